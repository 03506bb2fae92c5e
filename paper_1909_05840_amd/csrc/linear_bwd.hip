// Linear layer in 16 bits, backward.
//
//   dX = (dY W) o act'(pre)   where the input X was act(pre), or dY W;   dW = dY^T X;   dbias = sum_t dY[t]
//
// X is given in 16 bits, or in 8, or is formed again from pre, which is given in 16 bits or in 8.  One launch brings X and dY into the form that the
// products read, where they are not in it, and adds up dbias; one launch forms both products, their tiles dealt to the same workgroups; one adds up the parts
// of tiles whose contraction was cut.  Bound by the matrix cores.
#include "linear.hpp"
#include <algorithm>

namespace qb {
namespace {

struct GradArgs {
    const uint16_t *dY, *W, *X, *pre;
    const int8_t *x_codes, *pre_codes;
    const float *x_scales, *pre_scales;
    int64_t dy_row, x_row;
    int T, N, K, act, N8;  // N8: columns of the dY that the products read, a multiple of eight
    uint16_t *dX, *dW;
    float *dbias;
    uint16_t *dYs, *Xs;    // dY with rows that can be copied; X in 16 bits
    float *db;             // [row blocks][N]
    float *dXp, *dWp;      // [parts][T][K], [parts][N][K], or null
    int x_tiles, w_tiles, x_parts, w_parts, x_first;
    int x_blocks, n_blocks, t_blocks;  // of the first launch: for X; for dY, column blocks and row blocks
};

constexpr int kRowsAtOnce = 32;  // of X, to a workgroup of the first launch
constexpr int kRowBlock = 128;   // rows of dY whose sum is one part of dbias

template <typename T>
struct TypeOf;
template <>
struct TypeOf<Bf16> { static constexpr int value = QB_TYPE_BF16; };
template <>
struct TypeOf<Fp16> { static constexpr int value = QB_TYPE_FP16; };

template <typename T>
__global__ __launch_bounds__(256) void linear_prepare_kernel(const GradArgs a)
{
    typedef Eight<TypeOf<T>::value> E;
    if ((int)blockIdx.x < a.x_blocks) {
        const int row0 = blockIdx.x * kRowsAtOnce, rows = min(kRowsAtOnce, a.T - row0), chunks = a.K / 8;
        for (int c = threadIdx.x; c < rows * chunks; c += 256) {
            const int r = c / chunks, col = (c - r * chunks) * 8;
            const int64_t row = row0 + r;
            float v[8];
            E e;
            if (a.x_codes) {
                kept8(v, a.x_codes, a.x_scales, row, a.K, col);
            } else {
                if (a.pre_codes) {
                    kept8(v, a.pre_codes, a.pre_scales, row, a.K, col);
                } else {
                    e.load(a.pre, row * a.K + col, 8);
                    e.get(v);
                }
                activate(a.act, v);
            }
            e.set(v);
            e.store(a.Xs, row * a.K + col, 8);
        }
        return;
    }
    __shared__ float sums[8][256];
    const int id = blockIdx.x - a.x_blocks, block = id / a.n_blocks, lane = threadIdx.x & 31, team = threadIdx.x >> 5;
    const int n0 = (id - block * a.n_blocks) * 256, col = n0 + lane * 8, row0 = block * kRowBlock, row1 = min(a.T, row0 + kRowBlock);
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.0f;
    if (col < a.N) {
#pragma unroll 4
        for (int row = row0 + team; row < row1; row += 8) {
            E e;
            float v[8];
            e.load(a.dY, row * a.dy_row + col, a.N - col);
            if (a.dYs) e.store(a.dYs, (int64_t)row * a.N8 + col, 8);
            e.get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += v[i];
        }
    }
    if (!a.db) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[team][i * 32 + lane] = s[i];  // (lanes side by side)
    __syncthreads();
    const int n = n0 + (threadIdx.x & 31) * 8 + (threadIdx.x >> 5);
    if (n >= a.N) return;
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) x += sums[i][threadIdx.x];
    a.db[(int64_t)block * a.N + n] = x;
}

// dX's rows: 64 neighbours of what dY W gives
template <typename T>
__device__ __forceinline__ void finish(const GradArgs &a, int row, int col, int hf, float (&g)[2][16])
{
    typedef Block<T> B;
    const bool inside = row < a.T;
    const int64_t at = (int64_t)row * a.K;
    if (a.act != QB_ACT_NONE) {
        const float scale = a.pre_codes && inside ? a.pre_scales[(int64_t)row * (a.K / kGroup) + col / kGroup] : 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float z[16];
            if (a.pre_codes) B::load_codes(a.pre_codes, at, col + 32 * i, a.K, inside, hf, scale, z);
            else B::load(a.pre, at, col + 32 * i, a.K, inside, hf, z);
            slope(a.act, z, g[i]);
        }
    }
    B::store(a.dX, at, col, a.K, inside, hf, g[0]);
    B::store(a.dX, at, col + 32, a.K, inside, hf, g[1]);
}

template <typename T, typename S>
__global__ __launch_bounds__(64 * S::kWaves, 2) void linear_grads_kernel(const GradArgs a)
{
    static_assert(S::TM % 2 == 0, "a wavefront holds whole groups of 64");
    __shared__ __align__(1024) uint8_t lds[S::kStages * S::kStage];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave - wm * S::WN;
    constexpr int NA = S::BM / 8 / S::kWaves, NB = S::BN / 8 / S::kWaves;
    const int kt = (a.K + S::BM - 1) / S::BM, x_all = a.x_tiles * a.x_parts, w_all = a.w_tiles * a.w_parts;
    const bool of_x = a.x_first ? (int)blockIdx.x < x_all : (int)blockIdx.x >= w_all;
    const int tiles = of_x ? a.x_tiles : a.w_tiles, parts = of_x ? a.x_parts : a.w_parts;
    const int id = tile_of(of_x == (a.x_first != 0) ? blockIdx.x : blockIdx.x - (of_x ? w_all : x_all), tiles * parts), part = id / tiles, tile = id - part * tiles;
    const int row0 = tile / kt * S::BN, k0 = (tile - tile / kt * kt) * S::BM;  // of the results: tokens or neurons; inputs
    const int length = of_x ? a.N : a.T, all = (length + 63) / 64, s0 = (int)((int64_t)all * part / parts), s1 = (int)((int64_t)all * (part + 1) / parts);
    const int left = s1 == all ? length - (all - 1) * 64 : 64;
    v16f g[S::TM][S::TN];
    clear(g);
    const void *const dY = a.dYs ? a.dYs : a.dY;
    const int64_t dy_row = 2 * (a.dYs ? (int64_t)a.N8 : a.dy_row);
    if (of_x)
        multiply<T, S, true, false>(g, lds, s1 - s0, left, (left + 7) & ~7, wave, lane, across<S, NA>(a.W, 2ll * a.K, k0, a.K, s0, wave, lane),
                                    along<S, NB>(dY, dy_row, row0, a.T, s0, wave, lane));
    else
        multiply<T, S, true, true>(g, lds, s1 - s0, left, left, wave, lane, across<S, NA>(a.Xs ? a.Xs : a.X, 2 * (a.Xs ? (int64_t)a.K : a.x_row), k0, a.K, s0, wave, lane),
                                   across<S, NB>(dY, dy_row, row0, a.N8, s0, wave, lane));
    float *const sums = of_x ? a.dXp : a.dWp;
    const int rows = of_x ? a.T : a.N;
    each<S::TM / 2>([&](auto half) {
        constexpr int i = 2 * half;
        const int col = k0 + (wm * S::TM + i) * 32;
        if (col >= a.K) return;
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            const int row = row0 + (wn * S::TN + j) * 32 + l32;
            float v[2][16];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < 16; ++k) v[u][k] = g[i + u][j][k];
            if (sums) {
                if (row < rows) {
                    float *const to = sums + ((int64_t)part * rows + row) * a.K + col;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int k = 0; k < 16; k += 4) *reinterpret_cast<v4f *>(to + 32 * u + 2 * k + 4 * hf) = v4f{v[u][k], v[u][k + 1], v[u][k + 2], v[u][k + 3]};
                }
            } else if (of_x) {
                finish<T>(a, row, col, hf, v);
            } else {
                Block<T>::store(a.dW, (int64_t)row * a.K, col, a.K, row < a.N, hf, v[0]);
                Block<T>::store(a.dW, (int64_t)row * a.K, col + 32, a.K, row < a.N, hf, v[1]);
            }
        }
    });
}

// What was cut into parts: 32 rows by 64 columns of dX (x_blocks workgroups) or dW (w_blocks) to a wavefront; the last workgroups add up 64 columns of dbias each.
template <typename T>
__global__ __launch_bounds__(256) void linear_ends_kernel(const GradArgs a, int x_blocks, int w_blocks)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hf = lane >> 5;
    if ((int)blockIdx.x >= x_blocks + w_blocks) {
        __shared__ float sums[4][64];
        const int n = ((int)blockIdx.x - x_blocks - w_blocks) * 64 + lane;
        float s = 0.0f;
        if (n < a.N) {
#pragma unroll 8
            for (int p = wave; p < a.t_blocks; p += 4) s += a.db[(int64_t)p * a.N + n];
        }
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && n < a.N) a.dbias[n] = sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
        return;
    }
    const bool of_x = (int)blockIdx.x < x_blocks;
    const int rows = of_x ? a.T : a.N, parts = of_x ? a.x_parts : a.w_parts, groups = a.K / 64;
    const int64_t id = (int64_t)((int)blockIdx.x - (of_x ? 0 : x_blocks)) * 4 + wave;
    const int block = (int)(id / groups), col = (int)(id - (int64_t)block * groups) * 64, row = block * 32 + (lane & 31);
    if (block * 32 >= rows) return;
    float g[2][16];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int k = 0; k < 16; ++k) g[u][k] = 0.0f;
    const float *from = (of_x ? a.dXp : a.dWp) + (int64_t)min(row, rows - 1) * a.K + col + 4 * hf;
    for (int p = 0; p < parts; ++p, from += (int64_t)rows * a.K)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 16; k += 4) {
                const v4f x = *reinterpret_cast<const v4f *>(from + 32 * u + 2 * k);
#pragma unroll
                for (int e = 0; e < 4; ++e) g[u][k + e] += x[e];
            }
    if (of_x) {
        finish<T>(a, row, col, hf, g);
    } else {
        Block<T>::store(a.dW, (int64_t)row * a.K, col, a.K, row < rows, hf, g[0]);
        Block<T>::store(a.dW, (int64_t)row * a.K, col + 32, a.K, row < rows, hf, g[1]);
    }
}

// no token: gradients of zero
__global__ __launch_bounds__(256) void linear_zero_kernel(uint16_t *dW, float *dbias, int64_t n, int64_t N)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n || i < N; i += (int64_t)gridDim.x * 256) {
        if (dW && i < n) dW[i] = 0;
        if (dbias && i < N) dbias[i] = 0.0f;
    }
}

typedef Shape<2, 4, 4, 2, 2> Large;  // 256 x 256
typedef Shape<2, 2, 2, 2, 2> Middle;  // 128 x 128
typedef Shape<1, 4, 2, 1, 3> Small;  // 64 x 128

struct Plan {
    int size, x_tiles, w_tiles, x_parts, w_parts;
};
// Steps until the last of `room` workgroups is done with n1 tiles of a steps and, after them, n2 of b.
int64_t last_done(int64_t n1, int64_t a, int64_t n2, int64_t b, int room)
{
    const int64_t full = n1 / room, rest = n1 - full * room;
    if (rest == 0) return full * a + (n2 + room - 1) / room * b;
    const int64_t beside = (room - rest) * (a / b);  // tiles of b that fit beside the last round of a
    return (full + 1) * a + (n2 > beside ? (n2 - beside + room - 1) / room * b : 0);
}
template <typename S>
void parts_of(Plan &p, bool dx, bool dw, int64_t T, int64_t N, int64_t K, int room)
{
    const int64_t kt = (K + S::BM - 1) / S::BM;
    p.x_tiles = dx ? (int)(kt * ((T + S::BN - 1) / S::BN)) : 0;
    p.w_tiles = dw ? (int)(kt * ((N + S::BN - 1) / S::BN)) : 0;
    constexpr int kParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    constexpr int kTileCost = 5;
    const int x_steps = (int)((N + 63) / 64), w_steps = (int)((T + 63) / 64);
    p.x_parts = p.w_parts = 1;
    int64_t least = INT64_MAX;
    for (const int x : kParts)
        for (const int w : kParts) {
            if ((x > 1 && (!dx || x > x_steps / 2)) || (w > 1 && (!dw || w > w_steps / 2))) continue;
            const int64_t a = (x_steps + x - 1) / x + kTileCost, b = (w_steps + w - 1) / w + kTileCost, nx = (int64_t)p.x_tiles * x, nw = (int64_t)p.w_tiles * w;
            int64_t cost = a >= b ? last_done(nx, a, nw, b, room) : last_done(nw, b, nx, a, room);
            // the parts' sums: written and read once, at the rate at which a step's operands come
            cost += (x > 1 || w > 1 ? 4 : 0) + ((x > 1 ? x * T * K : 0) + (w > 1 ? w * N * K : 0)) / (room * 8192ll);
            if (cost < least) {
                least = cost;
                p.x_parts = x;
                p.w_parts = w;
            }
        }
}
Plan plan_of(const qb_linear_grads &l)
{
    const bool dx = l.dX != nullptr, dw = l.dW != nullptr;
    Plan p = {};
    const int64_t work = (dx ? l.T * l.K * ((l.N + 63) / 64) : 0) + (dw ? l.N * l.K * ((l.T + 63) / 64) : 0);  // results by steps
    p.size = work >= 256ll * 65536 * 16 ? 2 : work >= 256ll * 16384 * 16 ? 1 : 0;
    if (p.size == 2) parts_of<Large>(p, dx, dw, l.T, l.N, l.K, 256);
    else if (p.size == 1) parts_of<Middle>(p, dx, dw, l.T, l.N, l.K, 512);
    else parts_of<Small>(p, dx, dw, l.T, l.N, l.K, 512);
    return p;
}

bool shape_ok(const qb_linear_grads &l) { return l.T >= 0 && l.T <= kMostRows && l.N >= 1 && l.N <= kMostOutputs && k_ok(l.K); }
// rows of dY as the products read them: chunks of sixteen bytes at multiples of sixteen
bool readable(const qb_linear_grads &l) { return l.N % 8 == 0 && l.dy_row % 8 == 0 && aligned16(l.dY); }

// where everything lies in the workspace; returns its size
size_t lay_out(const qb_linear_grads &l, GradArgs &a, Plan &p, uint8_t *base)
{
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        uint8_t *const q = base + at;
        at += round_up(bytes);
        return q;
    };
    p = plan_of(l);
    a.T = (int)l.T; a.N = (int)l.N; a.K = (int)l.K;
    a.N8 = (a.N + 7) & ~7;
    a.x_tiles = p.x_tiles; a.w_tiles = p.w_tiles; a.x_parts = p.x_parts; a.w_parts = p.w_parts;
    a.t_blocks = (a.T + kRowBlock - 1) / kRowBlock;
    a.n_blocks = (a.N + 255) / 256;
    const bool stage = (l.dX || l.dW) && !readable(l), expand = l.dW && !l.X;
    a.x_blocks = expand ? (a.T + kRowsAtOnce - 1) / kRowsAtOnce : 0;
    if (!stage && !l.dbias) a.t_blocks = 0;
    if (expand) a.Xs = reinterpret_cast<uint16_t *>(take((size_t)a.T * a.K * 2));
    if (stage) a.dYs = reinterpret_cast<uint16_t *>(take((size_t)a.T * a.N8 * 2));
    if (l.dbias) a.db = reinterpret_cast<float *>(take((size_t)a.t_blocks * a.N * 4));
    if (p.x_parts > 1) a.dXp = reinterpret_cast<float *>(take((size_t)p.x_parts * a.T * a.K * 4));
    if (p.w_parts > 1) a.dWp = reinterpret_cast<float *>(take((size_t)p.w_parts * a.N * a.K * 4));
    return at;
}

template <typename T>
qb_status launch(const GradArgs &a, int size, hipStream_t st)
{
    const int64_t first = (int64_t)a.x_blocks + (int64_t)a.n_blocks * a.t_blocks;
    if (first > 0) linear_prepare_kernel<T><<<(int)first, 256, 0, st>>>(a);
    const int groups = a.x_tiles * a.x_parts + a.w_tiles * a.w_parts;
    if (groups > 0) {
        if (size == 2) linear_grads_kernel<T, Large><<<groups, 64 * Large::kWaves, 0, st>>>(a);
        else if (size == 1) linear_grads_kernel<T, Middle><<<groups, 64 * Middle::kWaves, 0, st>>>(a);
        else linear_grads_kernel<T, Small><<<groups, 64 * Small::kWaves, 0, st>>>(a);
    }
    const auto blocks = [&](int64_t rows) { return (int)(((rows + 31) / 32 * (a.K / 64) + 3) / 4); };
    const int x_blocks = a.dXp ? blocks(a.T) : 0, w_blocks = a.dWp ? blocks(a.N) : 0, ends = x_blocks + w_blocks + (a.dbias ? (a.N + 63) / 64 : 0);
    if (ends > 0) linear_ends_kernel<T><<<ends, 256, 0, st>>>(a, x_blocks, w_blocks);
    return launch_status();
}

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" size_t qb_linear_bwd_workspace_nbytes(const qb_linear_grads *l)
{
    GradArgs a = {};
    Plan p;
    return l && shape_ok(*l) && l->T > 0 ? lay_out(*l, a, p, nullptr) : 0;
}

extern "C" qb_status qb_linear_bwd(const qb_linear_grads *l, void *workspace, void *stream)
{
    if (!l) return QB_ERR_NULL;
    if (!shape_ok(*l)) return QB_ERR_SHAPE;
    if ((l->type != QB_TYPE_BF16 && l->type != QB_TYPE_FP16) || !act_ok(l->act) || !stride_ok(l->x_row) || l->x_row % 8 || !stride_ok(l->dy_row)) return QB_ERR_VALUE;
    const bool pre = l->pre || l->pre_codes;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (misaligned(l->dX, 2) || misaligned(l->dW, 2) || misaligned(l->dbias, 4)) return QB_ERR_VALUE;
    if (l->T == 0) {
        if (l->dW || l->dbias) linear_zero_kernel<<<(int)std::min<int64_t>(4096, (l->N * l->K + 255) / 256), 256, 0, st>>>(static_cast<uint16_t *>(l->dW), l->dbias, l->N * l->K, l->N);
        return launch_status();
    }
    if (!l->dY || (l->dX && !l->W)) return QB_ERR_NULL;
    if (!l->x_codes != !l->x_scales || !l->pre_codes != !l->pre_scales) return QB_ERR_NULL;
    if ((l->act != QB_ACT_NONE) != pre || (l->pre && l->pre_codes) || (l->X && l->x_codes)) return QB_ERR_VALUE;
    if (l->dW && !l->X && !l->x_codes && !pre) return QB_ERR_NULL;
    if (misaligned(l->dY, 2) || !aligned16(l->W) || !aligned16(l->X) || misaligned(l->x_scales, 4) || misaligned(l->pre, 2) || misaligned(l->pre_scales, 4)) return QB_ERR_VALUE;
    GradArgs a = {};
    Plan p;
    if (lay_out(*l, a, p, static_cast<uint8_t *>(workspace)) > 0 && (!workspace || misaligned(workspace, 256))) return QB_ERR_WORKSPACE;
    a.dY = static_cast<const uint16_t *>(l->dY); a.W = static_cast<const uint16_t *>(l->W); a.X = static_cast<const uint16_t *>(l->X);
    a.pre = static_cast<const uint16_t *>(l->pre);
    a.x_codes = l->x_codes; a.x_scales = l->x_scales; a.pre_codes = l->pre_codes; a.pre_scales = l->pre_scales;
    a.dy_row = l->dy_row; a.x_row = l->x_row; a.act = l->act;
    a.dX = static_cast<uint16_t *>(l->dX); a.dW = static_cast<uint16_t *>(l->dW); a.dbias = l->dbias;
    const int64_t x_steps = (l->N + 63) / 64 / a.x_parts, w_steps = (l->T + 63) / 64 / a.w_parts;
    a.x_first = x_steps >= w_steps;
    return l->type == QB_TYPE_BF16 ? launch<Bf16>(a, p.size, st) : launch<Fp16>(a, p.size, st);
}
