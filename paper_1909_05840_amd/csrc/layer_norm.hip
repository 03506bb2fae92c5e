// Layer norm and its backward.
//
//   mean = sum x / W;  rstd = 1 / sqrt(sum (x - mean)^2 / W + eps);  h = (x - mean) rstd;  y = h w + b
//   g = dy w;  dx = rstd (g - sum g / W - h sum g h / W) (+ residual);  dw = sum_t dy h;  db = sum_t dy
//
// A row stays in the registers of a wavefront or a workgroup between its loads and its stores; the squares are of x - mean, as the formula has
// them.  Bound by memory.  The backward's threads keep their columns from row to row and so hold their share of dw and db; a workgroup's share
// goes to the workspace, and a second launch adds these up in a fixed order.  32768 x 1024 in bf16 24.5 us forward, backward with a residual 50 and 4.7, 5.4 TB/s; as many values in
// rows of 4096 27, 45 and 4.8 (without a residual, 40 at the rate of a copy: eight wavefronts to a CU, which wait for each other's sums), in rows of 32768 38, 80 (read twice) and 4.8.
#include "qb_acts.hpp"
#include <algorithm>

namespace qb {
namespace {

struct NormArgs {
    const void *X, *dY, *residual;
    int64_t x_row, dy_row, residual_row;
    const int8_t *x_codes;  // X in 8 bits, instead of X
    const float *x_scales, *weight, *bias;
    float eps;
    int T, W;
    void *Y;  // backward: dX
    float *mean, *rstd;
    int8_t *codes;
    float *scales;
    float *part;  // [workgroups][2][W]: dw, db
    float *dweight, *dbias;
};

// the sum over R neighbouring lanes, in each of them
template <int R>
__device__ __forceinline__ float lanes_add(float x)
{
    const auto add = [&](auto ctrl) { x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    add(std::integral_constant<int, 0xB1>());   // lane ^ 1
    add(std::integral_constant<int, 0x4E>());   // lane ^ 2
    add(std::integral_constant<int, 0x141>());  // the other four of eight
    if constexpr (R >= 16) add(std::integral_constant<int, 0x140>());  // the other eight of sixteen
    if constexpr (R >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return x;
}
// R threads to a row, C chunks of eight values to a thread
template <int R, int C>
struct Row {
    static constexpr int kThreads = R > 256 ? R : 256, kRows = kThreads / R, kWaves = (R + 63) / 64;
    static __device__ __forceinline__ int col(int i) { return (i * R + (int)(threadIdx.x % R)) * 8; }
    // the sums of two values over a row's threads
    static __device__ __forceinline__ v2f sum(float a, float b, v2f *shared)
    {
        if constexpr (R < 64) return v2f{lanes_add<R>(a), lanes_add<R>(b)};
        a = wave_add(a);
        b = wave_add(b);
        if constexpr (R > 64) {
            __syncthreads();  // (the last sum has been read)
            if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v2f{a, b};
            __syncthreads();
            const int first = (int)(threadIdx.x / R) * kWaves;
            a = b = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                a += shared[first + i][0];
                b += shared[first + i][1];
            }
        }
        return v2f{a, b};
    }
};
__device__ __forceinline__ void columns(const float *p, float other, int col, int W, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = other;
    if (!p || col >= W) return;
    Eight<QB_TYPE_FP32> x;
    x.load(p, col, W - col);
    x.get(v);
}

// TAIL: the width is no multiple of eight, so that a chunk may be part of a row and not only all or nothing of it.
// Two workgroups of 1024 threads fit a CU with up to 80 scalar registers to a wavefront, which rows of 4097 to 8192 values take (20000 x 5000 in bf16 120 us, with two more 180).
template <int TYPE, int R, int C, bool TAIL>
__global__ __launch_bounds__((Row<R, C>::kThreads)) void layer_norm_kernel(const NormArgs a)
{
    typedef Row<R, C> L;
    __shared__ v2f shared[L::kThreads / 64];
    const float inv = 1.0f / (float)a.W;
    constexpr bool kHold = C < 4;  // the weights stay in registers
    float w[C][8], b[C][8];
    const auto weights = [&](int i) {
        columns(a.weight, 1.0f, L::col(i), a.W, w[i]);
        columns(a.bias, 0.0f, L::col(i), a.W, b[i]);
    };
#pragma unroll
    for (int i = 0; i < C; ++i)
        if (kHold) weights(i);
    for (int row0 = blockIdx.x * L::kRows; row0 < a.T; row0 += gridDim.x * L::kRows) {
        const int row = row0 + (int)(threadIdx.x / R);
        if (R <= 64 && row >= a.T) break;
        Eight<TYPE> x[C];
        float v[C][8], s = 0.0f;
#pragma unroll
        for (int i = 0; i < C; ++i) x[i].load(a.X, row * a.x_row + L::col(i), a.W - L::col(i));
#pragma unroll
        for (int i = 0; i < C; ++i) {
            x[i].get(v[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) s += v[i][e];
        }
        // the differences from a mean that is rounded say what it is off, and the squares are corrected for that (equal values have no variance)
        const float near = L::sum(s, 0.0f, shared)[0] * inv;
        float q = 0.0f;
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] -= L::col(i) + (TAIL ? e : 0) < a.W ? near : 0.0f;
                q = __builtin_fmaf(v[i][e], v[i][e], q);
                s += v[i][e];
            }
        const v2f both = L::sum(q, s, shared);
        const float more = both[1] / (float)a.W, mean = more == more ? near + more : near;  // (infinity stays: differences from it are no numbers)
        const float rstd = 1.0f / sqrtf(__builtin_elementwise_maximum(__builtin_fmaf(-more, more, both[0] * inv), 0.0f) + a.eps);  // (NaN stays)
        if (threadIdx.x % R == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if (!kHold) weights(i);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = __builtin_fmaf((v[i][e] - more) * rstd, w[i][e], b[i][e]);
            if (a.codes) keep8<false>(v[i], a.codes, a.scales, row, a.W, L::col(i));
            x[i].set(v[i]);
            x[i].store(a.Y, (int64_t)row * a.W + L::col(i), a.W - L::col(i));
        }
    }
}

// Rows that leave no registers for that (kWide values and more) are read once again by layer_norm_sums_kernel.
constexpr int kWide = 8192;
template <int TYPE, int R, int C>
__global__ __launch_bounds__((Row<R, C>::kThreads)) void layer_norm_bwd_kernel(const NormArgs a)
{
    typedef Row<R, C> L;
    constexpr bool kHold = R * C * 8 <= kWide;  // weights and sums stay in registers
    __shared__ v2f shared[L::kThreads / 64];
    const float inv = 1.0f / (float)a.W;
    float w[C][8], dw[C][8], db[C][8];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        if (kHold) columns(a.weight, 1.0f, L::col(i), a.W, w[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[i][e] = db[i][e] = 0.0f;
    }
    for (int row0 = blockIdx.x * L::kRows; row0 < a.T; row0 += gridDim.x * L::kRows) {
        const int row = row0 + (int)(threadIdx.x / R);
        if (R <= 64 && row >= a.T) break;
        Eight<TYPE> x[C], g[C], r[C];
        float h[C][8], v[C][8], s = 0.0f, sh = 0.0f;
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            g[i].load(a.dY, row * a.dy_row + L::col(i), a.W - L::col(i));
            if (a.x_codes) kept8(h[i], a.x_codes, a.x_scales, row, a.W, L::col(i));
            else x[i].load(a.X, row * a.x_row + L::col(i), a.W - L::col(i));
            if (a.residual) r[i].load(a.residual, row * a.residual_row + L::col(i), a.W - L::col(i));
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            g[i].get(v[i]);
            if (!a.x_codes) x[i].get(h[i]);
            if (!kHold) columns(a.weight, 1.0f, L::col(i), a.W, w[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[i][e] = (h[i][e] - mean) * rstd;  // (values past the row's end meet gradients of zero)
                if (kHold) {
                    dw[i][e] = __builtin_fmaf(v[i][e], h[i][e], dw[i][e]);
                    db[i][e] += v[i][e];
                }
                v[i][e] *= w[i][e];
                s += v[i][e];
                sh = __builtin_fmaf(v[i][e], h[i][e], sh);
            }
        }
        const v2f m = L::sum(s, sh, shared) * inv;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float past[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) past[e] = 0.0f;
            if (a.residual) r[i].get(past);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = __builtin_fmaf(v[i][e] - __builtin_fmaf(h[i][e], m[1], m[0]), rstd, past[e]);
            x[i].set(v[i]);
            x[i].store(a.Y, (int64_t)row * a.W + L::col(i), a.W - L::col(i));
        }
    }
    if (!kHold || !a.part) return;
    float *const to = a.part + (int64_t)blockIdx.x * 2 * a.W;
    if constexpr (L::kRows > 1) {  // the rows of a workgroup that worked side by side
        __shared__ float shares[2][L::kRows][R * 8];
        const int at = (int)(threadIdx.x % R), team = (int)(threadIdx.x / R);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                shares[0][team][e * R + at] = dw[i][e];
                shares[1][team][e * R + at] = db[i][e];
            }
            __syncthreads();
            for (int k = threadIdx.x; k < 2 * R * 8; k += L::kThreads) {
                const int which = k / (R * 8), c = k % (R * 8), col = (i * R + c % R) * 8 + c / R;
                float s = 0.0f;
#pragma unroll
                for (int t = 0; t < L::kRows; ++t) s += shares[which][t][c];
                if (col < a.W) to[which * a.W + col] = s;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (L::col(i) + e < a.W) {
                    to[L::col(i) + e] = dw[i][e];
                    to[a.W + L::col(i) + e] = db[i][e];
                }
    }
}

// Shares of dw and db of wide rows: 512 columns to a workgroup, every kSumParts-th set of four rows, one to a wavefront.
constexpr int kSumParts = 32;
template <int TYPE>
__global__ __launch_bounds__(256) void layer_norm_sums_kernel(const NormArgs a)
{
    __shared__ float shares[2][4][512];
    const int blocks = (a.W + 511) / 512, part = blockIdx.x / blocks, at = (threadIdx.x & 63) * 8, col = ((int)blockIdx.x - part * blocks) * 512 + at, wave = threadIdx.x >> 6;
    float dw[8], db[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = db[e] = 0.0f;
#pragma unroll 4
    for (int row = part * 4 + wave; row < a.T; row += kSumParts * 4) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        Eight<TYPE> g, x;
        float v[8], h[8];
        g.load(a.dY, row * a.dy_row + col, a.W - col);
        if (a.x_codes) {
            kept8(h, a.x_codes, a.x_scales, row, a.W, col);
        } else {
            x.load(a.X, row * a.x_row + col, a.W - col);
            x.get(h);
        }
        g.get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dw[e] = __builtin_fmaf(v[e], (h[e] - mean) * rstd, dw[e]);
            db[e] += v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        shares[0][wave][at + e] = dw[e];
        shares[1][wave][at + e] = db[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 1024; i += 256) {
        const int which = i >> 9, c = i & 511, to = col - at + c;
        if (to < a.W) a.part[((int64_t)part * 2 + which) * a.W + to] = shares[which][0][c] + shares[which][1][c] + shares[which][2][c] + shares[which][3][c];
    }
}

// dw and db from the workgroups' shares: 64 columns to a workgroup, sixteen wavefronts on shares of their own
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const NormArgs a, int parts)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane, all = 2 * a.W;
    float s = 0.0f;
    if (col < all) {
#pragma unroll 16
        for (int p = wave; p < parts; p += 16) s += a.part[(int64_t)p * all + col];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || col >= all) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sums[i][lane];
    if (col < a.W) {
        if (a.dweight) a.dweight[col] = s;
    } else if (a.dbias) {
        a.dbias[col - a.W] = s;
    }
}

// f with the threads to a row and the chunks to a thread that rows of W values take
template <typename F>
void by_width(int64_t W, const F &f)
{
    if (W <= 64) f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    else if (W <= 128) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    else if (W <= 256) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    else if (W <= 512) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    else if (W <= 1024) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    else if (W <= 2048) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    else if (W <= 4096) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    else if (W <= 8192) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
    else if (W <= 16384) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
}
template <typename F>
void by_type(int type, const F &f)
{
    if (type == QB_TYPE_BF16) f(std::integral_constant<int, QB_TYPE_BF16>{});
    else if (type == QB_TYPE_FP16) f(std::integral_constant<int, QB_TYPE_FP16>{});
    else f(std::integral_constant<int, QB_TYPE_FP32>{});
}
inline int rows_of(int64_t W) { return W <= 64 ? 32 : W <= 128 ? 16 : W <= 256 ? 8 : W <= 1024 ? 4 : 1; }  // that a workgroup works on at once
inline int bwd_groups(int64_t T, int64_t W) { return (int)std::min<int64_t>((T + rows_of(W) - 1) / rows_of(W), W <= 4096 ? 512 : 256); }

inline int sum_parts(int64_t T, int64_t W) { return W <= kWide ? bwd_groups(T, W) : T > 0 ? kSumParts : 0; }

bool shape_ok(int64_t T, int64_t W) { return T >= 0 && T <= kMostRows && W >= 1 && W <= QB_MAX_K; }

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" qb_status qb_layer_norm_fwd(const void *X, int64_t x_row, int type, int64_t T, int64_t W, const float *weight, const float *bias, float eps,
                                       void *Y, float *mean, float *rstd, int8_t *codes, float *scales, void *stream)
{
    if (!shape_ok(T, W)) return QB_ERR_SHAPE;
    if (!type_ok(type) || !stride_ok(x_row) || !(eps >= 0.0f && eps < __builtin_inff())) return QB_ERR_VALUE;
    if (T == 0) return QB_OK;
    if (!X || !Y || !mean || !rstd || !codes != !scales) return QB_ERR_NULL;
    if (misaligned(X, size_of(type)) || misaligned(Y, size_of(type)) || misaligned(weight, 4) || misaligned(bias, 4) || misaligned(mean, 4) || misaligned(rstd, 4) ||
        misaligned(scales, 4))
        return QB_ERR_VALUE;
    NormArgs a = {};
    a.X = X; a.x_row = x_row; a.T = (int)T; a.W = (int)W;
    a.weight = weight; a.bias = bias; a.eps = eps;
    a.Y = Y; a.mean = mean; a.rstd = rstd; a.codes = codes; a.scales = scales;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    by_type(type, [&](auto t) {
        by_width(W, [&](auto r, auto c) {
            typedef Row<decltype(r)::value, decltype(c)::value> L;
            const int64_t groups = (T + L::kRows - 1) / L::kRows;
            const int grid = (int)std::min<int64_t>(groups, 2048);
            if (W % 8) layer_norm_kernel<decltype(t)::value, decltype(r)::value, decltype(c)::value, true><<<grid, L::kThreads, 0, st>>>(a);
            else layer_norm_kernel<decltype(t)::value, decltype(r)::value, decltype(c)::value, false><<<grid, L::kThreads, 0, st>>>(a);
        });
    });
    return launch_status();
}

extern "C" size_t qb_layer_norm_bwd_workspace_nbytes(int64_t T, int64_t W)
{
    return shape_ok(T, W) ? (size_t)sum_parts(T, W) * 2 * (size_t)W * 4 : 0;
}

extern "C" qb_status qb_layer_norm_bwd(const qb_norm_grads *n, void *dX, float *dweight, float *dbias, void *workspace, void *stream)
{
    if (!n) return QB_ERR_NULL;
    if (!shape_ok(n->T, n->W)) return QB_ERR_SHAPE;
    if (!type_ok(n->type) || !stride_ok(n->dy_row) || !stride_ok(n->x_row) || !stride_ok(n->residual_row)) return QB_ERR_VALUE;
    const bool sums = dweight || dbias;
    if (n->T > 0) {
        if (!n->dY || !n->mean || !n->rstd || !dX || (!n->X) == (!n->x_codes) || !n->x_codes != !n->x_scales) return QB_ERR_NULL;
        const int size = size_of(n->type);
        if (misaligned(n->dY, size) || misaligned(n->X, size) || misaligned(n->residual, size) || misaligned(dX, size) || misaligned(n->x_scales, 4) || misaligned(n->weight, 4) ||
            misaligned(n->mean, 4) || misaligned(n->rstd, 4) || misaligned(dweight, 4) || misaligned(dbias, 4))
            return QB_ERR_VALUE;
        if (sums && (!workspace || misaligned(workspace, 256))) return QB_ERR_WORKSPACE;
    }
    NormArgs a = {};
    a.X = n->X; a.dY = n->dY; a.residual = n->residual;
    a.x_row = n->x_row; a.dy_row = n->dy_row; a.residual_row = n->residual_row;
    a.x_codes = n->x_codes; a.x_scales = n->x_scales; a.weight = n->weight;
    a.T = (int)n->T; a.W = (int)n->W;
    a.Y = dX; a.mean = const_cast<float *>(n->mean); a.rstd = const_cast<float *>(n->rstd);
    a.part = sums ? static_cast<float *>(workspace) : nullptr;
    a.dweight = dweight; a.dbias = dbias;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int groups = bwd_groups(n->T, n->W);
    if (sums && groups > 0 && a.W > kWide)  // (before dX, which may take dY's place)
        by_type(n->type, [&](auto t) { layer_norm_sums_kernel<decltype(t)::value><<<kSumParts * ((a.W + 511) / 512), 256, 0, st>>>(a); });
    if (groups > 0)
        by_type(n->type, [&](auto t) {
            by_width(n->W, [&](auto r, auto c) {
                layer_norm_bwd_kernel<decltype(t)::value, decltype(r)::value, decltype(c)::value><<<groups, Row<decltype(r)::value, decltype(c)::value>::kThreads, 0, st>>>(a);
            });
        });
    if (sums) layer_norm_join_kernel<<<(2 * a.W + 63) / 64, 1024, 0, st>>>(a, sum_parts(n->T, n->W));
    return launch_status();
}
