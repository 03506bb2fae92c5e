// Linear layer in 16 bits, forward: bias, activation and residual where the product ends.
//
//   z[t,n] = sum_j X[t,j] W[n,j] (+ bias[n]);  Y = act(z) (+ residual);  kept for the backward: z, or Y where there is no activation, in 8 bits, or z in 16
//
// Bound by the matrix cores with many tokens, by W's bytes with few.
#include "linear.hpp"
#include <algorithm>

namespace qb {
namespace {

struct LinearArgs {
    const uint16_t *X, *W, *residual;
    const float *bias;
    int64_t x_row, residual_row;
    int T, N, K, act;
    uint16_t *Y, *pre;
    int8_t *codes;
    float *scales;
    float *part;  // [parts][T][Np], or null
    int parts, Np;
};

// what becomes of two blocks of a row's sums, 64 neighbours: columns col .. of row `row`
template <typename T>
__device__ __forceinline__ void finish(const LinearArgs &a, int row, int col, int hf, float (&z)[2][16])
{
    typedef Block<T> B;
    const bool inside = row < a.T;
    const int64_t at = (int64_t)row * a.N;
    const auto keep = [&]() {
        const Coder c(halves_top(max(B::top(col, a.N, hf, z[0]), B::top(col + 32, a.N, hf, z[1]))));
        if (inside && hf == 0 && col < a.N) a.scales[(int64_t)row * ((a.N + kGroup - 1) / kGroup) + col / kGroup] = c.scale;
        B::store_codes(a.codes, at, col, a.N, inside, hf, c, z[0]);
        B::store_codes(a.codes, at, col + 32, a.N, inside, hf, c, z[1]);
    };
    if (a.act != QB_ACT_NONE) {
        if (a.codes) keep();
        if (a.pre) {
            B::store(a.pre, at, col, a.N, inside, hf, z[0]);
            B::store(a.pre, at, col + 32, a.N, inside, hf, z[1]);
        }
        activate(a.act, z[0]);
        activate(a.act, z[1]);
    }
    if (a.residual) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float r[16];
            B::load(a.residual, row * a.residual_row, col + 32 * i, a.N, inside, hf, r);
#pragma unroll
            for (int k = 0; k < 16; ++k) z[i][k] += r[k];
        }
    }
    if (a.act == QB_ACT_NONE && a.codes) keep();
    B::store(a.Y, at, col, a.N, inside, hf, z[0]);
    B::store(a.Y, at, col + 32, a.N, inside, hf, z[1]);
}

// Tiles of neurons by tokens: a lane's results are neighbours of a row of Y.
template <typename T, typename S>
__global__ __launch_bounds__(64 * S::kWaves, 2) void linear_kernel(const LinearArgs a)
{
    static_assert(S::TM % 2 == 0, "a wavefront holds whole groups of 64");
    __shared__ __align__(1024) uint8_t lds[S::kStages * S::kStage];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave - wm * S::WN;
    const int words = (a.N + S::BM - 1) / S::BM, tiles = words * ((a.T + S::BN - 1) / S::BN);
    const int id = tile_of(blockIdx.x, tiles * a.parts), part = id / tiles, tile = id - part * tiles;
    const int tt = tile / words, n0 = (tile - tt * words) * S::BM, t0 = tt * S::BN;
    const int steps = a.K / 64, s0 = (int)((int64_t)steps * part / a.parts), s1 = (int)((int64_t)steps * (part + 1) / a.parts);
    v16f z[S::TM][S::TN];
    clear(z);
    constexpr int NA = S::BM / 8 / S::kWaves, NB = S::BN / 8 / S::kWaves;
    multiply<T, S, false, false>(z, lds, s1 - s0, 64, 64, wave, lane, along<S, NA>(a.W, (int64_t)a.K * 2, n0, a.N, s0, wave, lane),
                                 along<S, NB>(a.X, a.x_row * 2, t0, a.T, s0, wave, lane));
    each<S::TM / 2>([&](auto half) {
        constexpr int i = 2 * half;
        const int col = n0 + (wm * S::TM + i) * 32;
        if (col >= a.N) return;
        float b[2][16];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int n = col + 32 * u + 8 * (k >> 2) + 4 * hf + (k & 3);
                b[u][k] = a.bias && !a.part && n < a.N ? a.bias[n] : 0.0f;
            }
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            const int row = t0 + (wn * S::TN + j) * 32 + l32;
            float v[2][16];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < 16; ++k) v[u][k] = z[i + u][j][k] + b[u][k];
            if (!a.part) {
                finish<T>(a, row, col, hf, v);
            } else if (row < a.T) {
                float *const to = a.part + ((int64_t)part * a.T + row) * a.Np + col;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int k = 0; k < 16; k += 4) *reinterpret_cast<v4f *>(to + 32 * u + 2 * k + 4 * hf) = v4f{v[u][k], v[u][k + 1], v[u][k + 2], v[u][k + 3]};
            }
        }
    });
}

// the parts of a contraction that was cut: 32 rows by 64 columns to a wavefront, in the order in which a product's results lie
template <typename T>
__global__ __launch_bounds__(64) void linear_join_kernel(const LinearArgs a)
{
    const int lane = threadIdx.x, hf = lane >> 5, groups = a.Np / 64, tt = (int)blockIdx.x / groups, col = ((int)blockIdx.x - tt * groups) * 64, row = tt * 32 + (lane & 31);
    float z[2][16];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int n = col + 32 * u + 8 * (k >> 2) + 4 * hf + (k & 3);
            z[u][k] = a.bias && n < a.N ? a.bias[n] : 0.0f;
        }
    const float *from = a.part + (int64_t)min(row, a.T - 1) * a.Np + col + 4 * hf;
    for (int p = 0; p < a.parts; ++p, from += (int64_t)a.T * a.Np)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 16; k += 4) {
                const v4f x = *reinterpret_cast<const v4f *>(from + 32 * u + 2 * k);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[u][k + e] += x[e];
            }
    finish<T>(a, row, col, hf, z);
}

typedef Shape<2, 4, 4, 2, 2> Large;  // 256 x 256
typedef Shape<2, 2, 2, 2, 2> Middle;  // 128 x 128
typedef Shape<1, 4, 2, 1, 3> Small;  // 64 x 128

struct Plan {
    int size, parts;  // 0 small, 1 middle, 2 large
};
template <typename S>
int64_t tiles_of(int64_t T, int64_t N) { return ((T + S::BN - 1) / S::BN) * ((N + S::BM - 1) / S::BM); }
Plan plan_of(const qb_linear &l)
{
    const int steps = (int)(l.K / 64);
    if (tiles_of<Large>(l.T, l.N) >= 192) return {2, 1};
    if (tiles_of<Middle>(l.T, l.N) >= 256) return {1, 1};
    return {0, best_parts(tiles_of<Small>(l.T, l.N), steps, 512, 8)};
}

size_t lay_out(const qb_linear &l, LinearArgs &a)
{
    const Plan p = plan_of(l);
    a.parts = p.parts;
    a.Np = (int)((l.N + 63) / 64 * 64);
    return p.parts > 1 ? round_up((size_t)p.parts * l.T * a.Np * 4) : 0;
}
bool shape_ok(const qb_linear &l) { return l.T >= 0 && l.T <= kMostRows && l.N >= 1 && l.N <= kMostOutputs && k_ok(l.K); }

template <typename T, typename S>
void launch(const LinearArgs &a, hipStream_t st)
{
    linear_kernel<T, S><<<(int)(tiles_of<S>(a.T, a.N) * a.parts), 64 * S::kWaves, 0, st>>>(a);
}
template <typename T>
qb_status launch(const LinearArgs &a, int size, hipStream_t st)
{
    if (size == 2) launch<T, Large>(a, st);
    else if (size == 1) launch<T, Middle>(a, st);
    else launch<T, Small>(a, st);
    if (a.parts > 1) linear_join_kernel<T><<<(a.T + 31) / 32 * (a.Np / 64), 64, 0, st>>>(a);
    return launch_status();
}

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" size_t qb_linear_fwd_workspace_nbytes(const qb_linear *l)
{
    LinearArgs a = {};
    return l && shape_ok(*l) && l->T > 0 ? lay_out(*l, a) : 0;
}

extern "C" qb_status qb_linear_fwd(const qb_linear *l, void *workspace, void *stream)
{
    if (!l) return QB_ERR_NULL;
    if (!shape_ok(*l)) return QB_ERR_SHAPE;
    if ((l->type != QB_TYPE_BF16 && l->type != QB_TYPE_FP16) || !act_ok(l->act) || !stride_ok(l->x_row) || l->x_row % 8 || !stride_ok(l->residual_row)) return QB_ERR_VALUE;
    if (l->pre && l->act == QB_ACT_NONE) return QB_ERR_VALUE;
    if (l->T == 0) return QB_OK;
    if (!l->X || !l->W || !l->Y || !l->codes != !l->scales) return QB_ERR_NULL;
    if (!aligned16(l->X) || !aligned16(l->W) || misaligned(l->Y, 2) || misaligned(l->pre, 2) || misaligned(l->residual, 2) || misaligned(l->bias, 4) || misaligned(l->scales, 4))
        return QB_ERR_VALUE;
    LinearArgs a = {};
    a.X = static_cast<const uint16_t *>(l->X); a.W = static_cast<const uint16_t *>(l->W); a.residual = static_cast<const uint16_t *>(l->residual);
    a.bias = l->bias; a.x_row = l->x_row; a.residual_row = l->residual_row;
    a.T = (int)l->T; a.N = (int)l->N; a.K = (int)l->K; a.act = l->act;
    a.Y = static_cast<uint16_t *>(l->Y); a.pre = static_cast<uint16_t *>(l->pre);
    a.codes = l->codes; a.scales = l->scales;
    if (lay_out(*l, a)) {
        if (!workspace || misaligned(workspace, 256)) return QB_ERR_WORKSPACE;
        a.part = static_cast<float *>(workspace);
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int size = plan_of(*l).size;
    return l->type == QB_TYPE_BF16 ? launch<Bf16>(a, size, st) : launch<Fp16>(a, size, st);
}
