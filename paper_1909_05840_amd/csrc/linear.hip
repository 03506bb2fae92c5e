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

// what becomes of two blocks of sums, 64 columns from `col` on of 32 rows from `row0` on; `room`: LDS of the wavefront's own
template <typename T, bool STREAM>
__device__ __forceinline__ void finish(const LinearArgs &a, int row0, int col, int lane, uint8_t *room, float (&z)[2][16])
{
    typedef Block<T> B;
    const int row = row0 + (lane & 31), hf = lane >> 5;
    const bool inside = row < a.T;
    const auto keep = [&]() {
        const Coder c(top_of(col, a.N, hf, z));
        if (inside && hf == 0) a.scales[(int64_t)row * ((a.N + kGroup - 1) / kGroup) + col / kGroup] = c.quick_scale();
        store_code_rows<STREAM>(a.codes, row0, a.T, col, a.N, lane, room, c, z);
    };
    if (a.act != QB_ACT_NONE) {
        if (a.codes) keep();
        if (a.pre) store_rows<T, STREAM>(a.pre, row0, a.T, col, a.N, lane, room, z);
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
    store_rows<T, STREAM>(a.Y, row0, a.T, col, a.N, lane, room, z);
}

constexpr int kMostCut = 128 * 128;  // results of a tile whose contraction may be cut; the parts are added up by a second launch
// Tiles of neurons by tokens: a lane's results are neighbours of a row of Y.  (Workgroups that stay and take tile after tile, the next one's first steps and this one's
// rows on their way meanwhile, measured the same within 2%, 16384 x 4096 by 1024 without and with GELU and codes; they need the registers.)
template <typename T, typename S, bool STREAM>
__global__ __launch_bounds__(64 * S::kWaves, 2) void linear_kernel(const LinearArgs a)
{
    static_assert(S::TM % 2 == 0, "a wavefront holds whole groups of 64");
    constexpr int kTeam = S::WM * S::WN;
    __shared__ __align__(1024) uint8_t lds[S::kLds];
    static_assert(S::kStages * S::kStage >= kTeam * kRowsRoom, "room for the rows on their way out, where the stages were");
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % kTeam / S::WN, wn = wave % S::WN;
    const int words = (a.N + S::BM - 1) / S::BM, rows = (a.T + S::BN - 1) / S::BN, tiles = words * rows, all = a.K / S::KS;
    const int id = tile_of(blockIdx.x, tiles * a.parts), part = id / tiles, s0 = all * part / a.parts, steps = all * (part + 1) / a.parts - s0;
    int tt, tn, stage = 0, next = 0;
    place_of(id - part * tiles, rows, words, tt, tn);
    const int n0 = tn * S::BM, t0 = tt * S::BN;
    const uint32_t lds0 = lds_address(lds);
    v16f z[S::TM][S::TN];
    float none[S::TN];
    clear(z);
    {
        Feed<S::NA> w = along<S, S::NA>(a.W, (int64_t)a.K * 2, n0, a.N, s0, wave, lane);
        Feed<S::NB> x = along<S, S::NB>(a.X, a.x_row * 2, t0, a.T, s0, wave, lane);
        const auto fetch = [&](int to) {
            if (next >= steps) return;
            ++next;
            copy_step<S, false>(w, lds0 + to * S::kStage, S::KS, wave, lane);
            copy_step<S, false>(x, lds0 + to * S::kStage + S::BM * S::KS * 2, S::KS, wave, lane);
        };
#pragma unroll
        for (int u = 0; u < S::kStages; ++u) fetch(u);
        Product<T, S, false, false, false>(lds0, wave, lane).run(z, none, steps, stage, fetch, [&](int s) { wait_step<S>(s, steps); });
    }
    gather<S>(z, lds + S::kStages * S::kStage, wave, lane);
    if (wave >= kTeam) return;
    each<S::TM / 2>([&](auto half) {
        constexpr int i = 2 * half;
        const int col = n0 + (wm * S::TM + i) * 32;
        if (col >= a.N) return;
        if constexpr (S::BM * S::BN <= kMostCut) {
            if (a.part) {  // (its rows have room for whole groups)
#pragma unroll
                for (int j = 0; j < S::TN; ++j) {
                    const int row = t0 + (wn * S::TN + j) * 32 + l32;
                    if (row >= a.T) continue;
                    float *const to = a.part + ((int64_t)part * a.T + row) * a.Np + col;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int k = 0; k < 16; k += 4)
                            *reinterpret_cast<v4f *>(to + 32 * u + 2 * k + 4 * hf) = v4f{z[i + u][j][k], z[i + u][j][k + 1], z[i + u][j][k + 2], z[i + u][j][k + 3]};
                }
                return;
            }
        }
        float b[2][16];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int n = col + 32 * u + 8 * (k >> 2) + 4 * hf + (k & 3);
                b[u][k] = a.bias ? a.bias[min(n, a.N - 1)] : 0.0f;
            }
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            float v[2][16];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < 16; ++k) v[u][k] = z[i + u][j][k] + b[u][k];
            finish<T, STREAM>(a, t0 + (wn * S::TN + j) * 32, col, lane, lds + wave * kRowsRoom, v);
        }
    });
}

// Few tokens: 16 * M neurons to a workgroup, whose wavefronts share the contraction, or a part of it; the weights go from memory straight into the matrix cores'
// operands, each read once.  G groups of sixteen tokens; kUnits of 64 values of the contraction under way to a wavefront (units that are not there cost as much as others:
// 1 x 4096 by 1024 4.5 us with four, 3.4 with two).  A CU is given about 45 GB/s, whatever it asks for: with few neurons the contraction is cut into parts, so that every CU
// takes its share of weights and tokens, and with many M makes the tokens' share small.
template <typename T, int M, int G, int kUnits>
__global__ __launch_bounds__(512) void linear_few_kernel(const LinearArgs a)
{
    __shared__ float sums[8][G * 16][M * 16 + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), blocks = (a.N + 16 * M - 1) / (16 * M);
    const int part = blockIdx.x / blocks, n0 = ((int)blockIdx.x - part * blocks) * (16 * M), r = lane & 15, k0 = 8 * (lane >> 4);
    const int units = a.K / 64, u0 = (int)((int64_t)units * part / a.parts), u1 = (int)((int64_t)units * (part + 1) / a.parts);
    const uint16_t *w[M], *x[G];
    v4f z[M][G];
#pragma unroll
    for (int m = 0; m < M; ++m) {
        w[m] = a.W + (int64_t)min(n0 + 16 * m + r, a.N - 1) * a.K + k0;
#pragma unroll
        for (int g = 0; g < G; ++g) z[m][g] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int g = 0; g < G; ++g) x[g] = a.X + min(16 * g + r, a.T - 1) * a.x_row + k0;
    for (int first = u0 + wave; first < u1; first += 8 * kUnits) {
        v8s p[kUnits][2][M], q[kUnits][2][G];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int k = min(first + 8 * u, u1 - 1) * 64;  // (past the end: the last unit again, not multiplied)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int m = 0; m < M; ++m) p[u][h][m] = *reinterpret_cast<const v8s *>(w[m] + k + 32 * h);
#pragma unroll
                for (int g = 0; g < G; ++g) q[u][h][g] = *reinterpret_cast<const v8s *>(x[g] + k + 32 * h);
            }
        }
        // (all loads before the first product)
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int m = 0; m < M; ++m) asm volatile("" : "+v"(p[u][h][m]));
#pragma unroll
                for (int g = 0; g < G; ++g) asm volatile("" : "+v"(q[u][h][g]));
            }
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (first + 8 * u < u1) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int g = 0; g < G; ++g) z[m][g] = T::mma16(p[u][h][m], q[u][h][g], z[m][g]);
            }
    }
    // a lane's results: token lane % 16, neurons 4 * (lane / 16) ..
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[wave][16 * g + r][16 * m + k0 / 2 + e] = z[m][g][e];
    __syncthreads();
    for (int i = threadIdx.x; i < M * G * 256; i += 512) {
        const int row = i / (16 * M), c = i % (16 * M), n = n0 + c;
        if (row >= a.T || n >= a.N) continue;
        float v[1] = {a.bias && !a.part ? a.bias[n] : 0.0f};
#pragma unroll
        for (int k = 0; k < 8; ++k) v[0] += sums[k][row][c];
        if (a.part) {
            a.part[((int64_t)part * a.T + row) * a.Np + n] = v[0];
            continue;
        }
        const int64_t at = (int64_t)row * a.N + n;
        if (a.pre) a.pre[at] = (uint16_t)T::pair(v[0], 0.0f);
        activate(a.act, v);
        if (a.residual) v[0] += T::lo(a.residual[row * a.residual_row + n]);
        a.Y[at] = (uint16_t)T::pair(v[0], 0.0f);
    }
}

// the parts of a contraction that was cut: four neighbours of a row to a thread, a group of 64 to sixteen lanes
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(const LinearArgs a)
{
    const uint32_t quads = (uint32_t)a.Np / 4, i = blockIdx.x * 256 + threadIdx.x;
    const int row = (int)min(i / quads, (uint32_t)a.T - 1), col = (int)(i % quads) * 4;  // (a group's lanes stay together)
    const bool inside = i / quads < (uint32_t)a.T;
    float z[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = a.bias && col + e < a.N ? a.bias[col + e] : 0.0f;
    add_parts(a.part + (int64_t)row * a.Np + col, (int64_t)a.T * a.Np, a.parts, z);
    if (a.act != QB_ACT_NONE) {
        if (a.codes) keep4(z, a.codes, a.scales, row, a.N, col, inside);
        if (a.pre && inside) store4<T>(a.pre, (int64_t)row * a.N + col, a.N - col, z);
        activate(a.act, z);
    }
    if (a.residual && inside) {
        float r[4];
        load4<T>(a.residual, row * a.residual_row + col, a.N - col, r);
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] += r[e];
    }
    if (a.act == QB_ACT_NONE && a.codes) keep4(z, a.codes, a.scales, row, a.N, col, inside);
    if (inside) store4<T>(a.Y, (int64_t)row * a.N + col, a.N - col, z);
}

typedef Tile<2, 4, 4, 2, 2> Large;     // 256 x 256
typedef Tile<2, 4, 2, 2, 3> Broad;     // 128 x 256
typedef Tile<2, 2, 2, 2, 2> Middle;    // 128 x 128
typedef Tile<1, 4, 2, 1, 3> Small;     // 64 x 128
typedef Tile<1, 2, 2, 1, 3, 2> Least;  // 64 x 64
struct Plan {
    int size, parts;  // 0 least .. 4 large; few tokens: -M
};
int64_t padded(int64_t N) { return (N + 63) / 64 * 64; }  // a part's rows: whole groups are written and read
template <typename S>
int64_t tiles_of(int64_t T, int64_t N) { return ((T + S::BN - 1) / S::BN) * ((N + S::BM - 1) / S::BM); }
// Few tokens: a launch's ends and the rounds of a wavefront's units, the largest share of a CU, at 45 KB a microsecond (with registers for 64 tokens 32), and what a second
// launch and the parts' bytes cost.  Measured over three sets of operands in turn (modelled), us: 1 x 1024 by 4096 uncut 8.1 (7.1), in 4 parts 7.2 (6.6); 24 x 1024 by 4096 12.9 (11.3),
// 8.8 (7.7); 32 x 1024 by 4096 14.2 (12.7), 9.2 (8.1); 16 x 4096 by 4096 11.2 (9.8), with 32 neurons in 2 parts 12.3 (11.3); 64 x 768 by 768 8.1 (7.8).
Plan few_plan(const qb_linear &l, double &least)
{
    Plan best = {-1, 1};
    for (const int m : {1, 2}) {
        for (const int p : {1, 2, 4, 8}) {
            if (p > 1 && p > l.K / 128) break;
            if (m > 1 && l.K / p < 1024) break;  // (two units for each wavefront)
            const int64_t groups = (l.N + 16 * m - 1) / (16 * m) * p, units = (l.K / 64 + 8 * p - 1) / (8 * p), at_once = m > 1 || l.T > 32 ? 2 : 4;
            const double share = (double)((groups + 255) / 256) * (double)((16 * m + l.T) * l.K * 2 / p) * 1e-3;
            double cost = (l.T > 32 ? 4.0 + share / 32.0 : 3.0 + share / 45.0) + (double)((units - 1) / at_once);
            if (p > 1 || l.codes) cost += 2.8 + p * l.T * padded(l.N) * 1e-6;
            if (cost < 0.95 * least) {  // (1 x 16384 by 4096, one and two of sixteen neurons: 26.3, 28.1 us)
                least = cost;
                best = {-m, p};
            }
        }
    }
    return best;
}
// Tiles, and into how many parts their contraction is cut.  Measured over three sets of operands in turn (modelled), us: 390 x 768 by 768 least 7.1 (7.2), small 9.0 (10.3);
// 1000 x 1024 by 1024 9.0 (8.3), 11.0 (11.9), middle 14.5 (15.7); 4000 x 1024 by 1024 19.2 (24.7), 16.8 (17.3), 16.6 (15.7), broad 18.9 (22.7); 8190 x 1024 by 4096 broad 69.1
// (72.8), large 92.6 (108), middle 68.6 (83.3); 16384 x 4096 by 1024 large 142 (122), broad 165 (182).  Least in parts: 65 x 1024 by 4096 uncut 18.6 (20.5), in 4 10.0 (10.5), in 8
// 9.2 (9.2); 390 x 768 by 3008 15.2 (16.1), in 2 13.1 (13.5), in 3 12.6 (12.3), in 4 13.6 (15.1); 64 x 4096 by 4096 19.2 (20.5), in 4 12.5 (12.7).
template <typename S>
void try_size(Plan &best, double &least, const Cost &c, const qb_linear &l)
{
    const int64_t tiles = tiles_of<S>(l.T, l.N), steps = l.K / 64;
    if (c.ends + (double)(tiles * steps) * ((S::BM + S::BN) / 8.0) / (256 * c.rate) >= least) return;
    for (const int p : {1, 2, 3, 4, 6, 8, 12, 16}) {
        if (p > 1 && (p > steps / 4 || S::BM * S::BN > kMostCut)) break;
        const int64_t length = (steps + p - 1) / p;
        const double share = (double)((tiles * p + 255) / 256 * length) * ((S::BM + S::BN) / 8.0);
        double cost = c.ends * (double)((tiles * p + c.room - 1) / c.room) + std::max(length * c.step, share / c.rate);
        if (p > 1) cost += 1.5 + p * (double)l.T * padded(l.N) * 2.8e-6;
        if (cost < least) {
            least = cost;
            best = {c.size, p};
        }
    }
}
Plan plan_of(const qb_linear &l)
{
    Plan p = {0, 1};
    double least = 1e300;
    if (l.T <= 64) p = few_plan(l, least);
    try_size<Least>(p, least, {0, 512, 4.2, 0.2, 63.0}, l);
    if (l.T <= 64) return p;
    try_size<Small>(p, least, {1, 512, 5.5, 0.4, 65.0}, l);
    try_size<Middle>(p, least, {2, 512, 6.0, 0.6, 53.0}, l);
    try_size<Broad>(p, least, {3, 256, 6.0, 1.0, 46.0}, l);
    try_size<Large>(p, least, {4, 256, 6.0, 1.6, 42.0}, l);
    return p;
}

size_t lay_out(const qb_linear &l, LinearArgs &a, Plan &p)
{
    p = plan_of(l);
    a.parts = p.parts;
    a.Np = (int)padded(l.N);
    return p.parts > 1 || (p.size < 0 && l.codes) ? round_up((size_t)p.parts * l.T * a.Np * 4) : 0;
}
bool shape_ok(const qb_linear &l) { return l.T >= 0 && l.T <= kMostRows && l.N >= 1 && l.N <= kMostOutputs && k_ok(l.K); }

template <typename T, typename S>
void launch(const LinearArgs &a, hipStream_t st)
{
    const int groups = (int)tiles_of<S>(a.T, a.N) * a.parts;
    if constexpr (S::kWaves == 8)  // (large results, which the L2 would not keep anyway)
        if (a.N % 64 == 0) return linear_kernel<T, S, true><<<groups, 64 * S::kWaves, 0, st>>>(a);
    linear_kernel<T, S, false><<<groups, 64 * S::kWaves, 0, st>>>(a);
}
template <typename T>
qb_status launch(const LinearArgs &a, int size, hipStream_t st)
{
    if (size < 0) {
        const int groups = (a.N + 16 * -size - 1) / (16 * -size) * a.parts, units = (a.K / 64 + 8 * a.parts - 1) / (8 * a.parts);  // (of a wavefront)
        const auto go = [&](auto g) {
            constexpr int G = decltype(g)::value;
            if (size == -2) return linear_few_kernel<T, 2, G, 2><<<groups, 512, 0, st>>>(a);
            if (units == 1) return linear_few_kernel<T, 1, G, 1><<<groups, 512, 0, st>>>(a);
            if constexpr (G < 4)
                if (units > 2) return linear_few_kernel<T, 1, G, 4><<<groups, 512, 0, st>>>(a);
            linear_few_kernel<T, 1, G, 2><<<groups, 512, 0, st>>>(a);
        };
        if (a.T <= 16) go(std::integral_constant<int, 1>{});
        else if (a.T <= 32) go(std::integral_constant<int, 2>{});
        else go(std::integral_constant<int, 4>{});
    } else if (size == 4) launch<T, Large>(a, st);
    else if (size == 3) launch<T, Broad>(a, st);
    else if (size == 2) launch<T, Middle>(a, st);
    else if (size == 1) launch<T, Small>(a, st);
    else launch<T, Least>(a, st);
    if (a.part) linear_join_kernel<T><<<(int)(((int64_t)a.T * (a.Np / 4) + 255) / 256), 256, 0, st>>>(a);
    return launch_status();
}

}  // namespace

// host, pure: Plan::size of a call, and into how many parts its contraction is cut
int linear_fwd_plan(const qb_linear *l, int *parts)
{
    const Plan p = plan_of(*l);
    *parts = p.parts;
    return p.size;
}

}  // namespace qb

using namespace qb;

extern "C" size_t qb_linear_fwd_workspace_nbytes(const qb_linear *l)
{
    LinearArgs a = {};
    Plan p;
    return l && shape_ok(*l) && l->T > 0 ? lay_out(*l, a, p) : 0;
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
    Plan p;
    if (lay_out(*l, a, p)) {
        if (!workspace || misaligned(workspace, 256)) return QB_ERR_WORKSPACE;
        a.part = static_cast<float *>(workspace);
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return l->type == QB_TYPE_BF16 ? launch<Bf16>(a, p.size, st) : launch<Fp16>(a, p.size, st);
}
