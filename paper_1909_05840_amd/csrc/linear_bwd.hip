// Linear layer in 16 bits, backward.
//
//   dX = (dY W) o act'(pre)   where the input X was act(pre), or dY W;   dW = dY^T X;   dbias = sum_t dY[t]
//
// X is given in 16 bits, or in 8, or is formed again from pre, which is given in 16 bits or in 8.  One launch brings X and dY into the form that the
// products read, where they are not in it; one launch forms both products, their tiles dealt to the same workgroups, and adds up dbias on the way; one adds up the
// parts of tiles whose contraction was cut.  Bound by the matrix cores.
#include "linear.hpp"
#include <algorithm>
#include <cmath>

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
    float *db;             // [db_parts][N]: parts of dbias
    float *dXp, *dWp;      // [parts][T][K], [parts][N][K], or null
    int x_tiles, w_tiles, x_parts, w_parts, x_first;
    int64_t x_blocks, y_blocks;        // of the first launch: for X; for dY's copy
    int n_blocks, t_blocks;            // for dbias where dW is not formed, column blocks and row blocks
    int db_parts;                      // of dbias: the first launch's row blocks, or the parts of dW's tiles, which then add it up
};

constexpr int kAtOnce = 2;       // chunks of eight values of X, or of dY, to a thread of the first launch
constexpr int kRowBlock = 128;   // rows of dY whose sum is one part of dbias
constexpr int64_t kMostBlocks = (1 << 24) - 1;  // of 256 threads: a launch has less than 2^32 of them, and a second one takes what is left

template <typename T>
struct TypeOf;
template <>
struct TypeOf<Bf16> { static constexpr int value = QB_TYPE_BF16; };
template <>
struct TypeOf<Fp16> { static constexpr int value = QB_TYPE_FP16; };

template <typename T>
__global__ __launch_bounds__(256) void linear_prepare_kernel(const GradArgs a, int64_t first_block)
{
    typedef Eight<TypeOf<T>::value> E;
    const int64_t at_block = first_block + blockIdx.x;
    if (at_block < a.x_blocks) {
        const int64_t chunks = (int64_t)a.T * (a.K / 8);
        int64_t at[kAtOnce];
        float v[kAtOnce][8];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            at[u] = min((at_block * kAtOnce + u) * 256 + threadIdx.x, chunks - 1);  // (past the end: the last chunk again)
            if (a.x_codes) {
                kept8(v[u], a.x_codes, a.x_scales, at[u]);
            } else if (a.pre_codes) {
                kept8(v[u], a.pre_codes, a.pre_scales, at[u]);
            } else {
                E e;
                e.load(a.pre, at[u] * 8, 8);
                e.get(v[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (!a.x_codes) activate(a.act, v[u]);
            E e;
            e.set(v[u]);
            e.store(a.Xs, at[u] * 8, 8);
        }
        return;
    }
    if (at_block < a.x_blocks + a.y_blocks) {
        const uint32_t chunks = (uint32_t)a.N8 / 8;
        const int64_t all = (int64_t)a.T * chunks;
        int64_t at[kAtOnce];
        E e[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            at[u] = min(((at_block - a.x_blocks) * kAtOnce + u) * 256 + threadIdx.x, all - 1);  // (past the end: the last chunk again)
            const int64_t row = all >> 32 ? at[u] / chunks : (uint32_t)at[u] / chunks;
            const int col = (int)(at[u] - row * chunks) * 8;
            e[u].load(a.dY, row * a.dy_row + col, a.N - col);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) e[u].store(a.dYs, at[u] * 8, 8);
        return;
    }
    __shared__ float sums[8][256];
    const int id = (int)(at_block - a.x_blocks - a.y_blocks), block = id / a.n_blocks, lane = threadIdx.x & 31, team = threadIdx.x >> 5;
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
            e.get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += v[i];
        }
    }
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

// dX's rows: 64 columns from `col` on of what dY W gives, 32 rows from `row0` on
template <typename T, bool STREAM>
__device__ __forceinline__ void finish(const GradArgs &a, int row0, int col, int lane, uint8_t *room, float (&g)[2][16])
{
    typedef Block<T> B;
    const int row = row0 + (lane & 31), hf = lane >> 5;
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
    store_rows<T, STREAM>(a.dX, row0, a.T, col, a.K, lane, room, g);
}

template <typename T, typename S>
__global__ __launch_bounds__(64 * S::kWaves, 2) void linear_grads_kernel(const GradArgs a)
{
    static_assert(S::TM % 2 == 0, "a wavefront holds whole groups of 64");
    __shared__ __align__(1024) uint8_t lds[S::kLds];
    static_assert(S::kStages * S::kStage >= S::kWaves * kRowsRoom, "room for the rows on their way out, where the stages were");
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % (S::WM * S::WN) / S::WN, wn = wave % S::WN;
    const int kt = (a.K + S::BM - 1) / S::BM, x_all = a.x_tiles * a.x_parts, w_all = a.w_tiles * a.w_parts;
    const bool of_x = a.x_first ? (int)blockIdx.x < x_all : (int)blockIdx.x >= w_all;
    const int tiles = of_x ? a.x_tiles : a.w_tiles, parts = of_x ? a.x_parts : a.w_parts;
    const int id = tile_of(of_x == (a.x_first != 0) ? blockIdx.x : blockIdx.x - (of_x ? w_all : x_all), tiles * parts), part = id / tiles, tile = id - part * tiles;
    int tr, tk;
    place_of(tile, tiles / kt, kt, tr, tk);
    const int row0 = tr * S::BN, k0 = tk * S::BM;  // of the results: tokens or neurons; inputs
    constexpr int KS = S::KS;
    const int length = of_x ? a.N : a.T, all = (length + KS - 1) / KS, s0 = (int)((int64_t)all * part / parts), s1 = (int)((int64_t)all * (part + 1) / parts);
    const int left = s1 == all ? length - (all - 1) * KS : KS;
    v16f g[S::TM][S::TN];
    clear(g);
    float db[S::TN];
#pragma unroll
    for (int j = 0; j < S::TN; ++j) db[j] = 0.0f;
    const void *const dY = a.dYs ? a.dYs : a.dY;
    const int64_t dy_row = 2 * (a.dYs ? (int64_t)a.N8 : a.dy_row);
    const uint32_t lds0 = lds_address(lds);
    const int steps = s1 - s0;
    int stage = 0;
    // f: the product, its operands on their way to LDS, how much of the last step there is
    const auto form = [&](const auto &product, auto a_across, auto b_across, auto fa, auto fb, int left_a, int left_b) {
        int next = 0;
        const auto fetch = [&](int to) {
            if (next >= steps) return;
            const bool last = ++next == steps;
            copy_step<S, decltype(a_across)::value>(fa, lds0 + to * S::kStage, last ? left_a : KS, wave, lane);
            copy_step<S, decltype(b_across)::value>(fb, lds0 + to * S::kStage + S::BM * KS * 2, last ? left_b : KS, wave, lane);
        };
#pragma unroll
        for (int u = 0; u < S::kStages; ++u) fetch(u);
        product.run(g, db, steps, stage, fetch, [&](int s) { wait_step<S>(s, steps); });
    };
    typedef std::true_type Across;
    typedef std::false_type Along;
    if (of_x) {
        form(Product<T, S, true, false, false>(lds0, wave, lane), Across(), Along(), across<S, S::NA>(a.W, 2ll * a.K, k0, a.K, s0, wave, lane),
             along<S, S::NB>(dY, dy_row, row0, a.T, s0, wave, lane), left, (left + 7) & ~7);
    } else {
        const auto x = across<S, S::NA>(a.Xs ? a.Xs : a.X, 2 * (a.Xs ? (int64_t)a.K : a.x_row), k0, a.K, s0, wave, lane);
        const auto y = across<S, S::NB>(dY, dy_row, row0, a.N8, s0, wave, lane);
        if (a.dbias && k0 == 0) {  // one tile of each row of tiles adds up dY on the way
            form(Product<T, S, true, true, true>(lds0, wave, lane), Across(), Across(), x, y, left, left);
            // the halves of the wavefront and the groups of wavefronts had shares of the contraction
            __shared__ float shares[S::KG][S::BN];
#pragma unroll
            for (int j = 0; j < S::TN; ++j) {
                const float sum = halves_sum(db[j]);
                if (wm == 0 && hf == 0) shares[wave / (S::WM * S::WN)][(wn * S::TN + j) * 32 + l32] = sum;
            }
            barrier();
            for (int i = threadIdx.x; i < S::BN; i += 64 * S::kWaves) {
                float sum = shares[0][i];
#pragma unroll
                for (int k = 1; k < S::KG; ++k) sum += shares[k][i];
                if (row0 + i < a.N) (parts > 1 ? a.db + (int64_t)part * a.N : a.dbias)[row0 + i] = sum;
            }
        } else {
            form(Product<T, S, true, true, false>(lds0, wave, lane), Across(), Across(), x, y, left, left);
        }
    }
    gather<S>(g, lds + S::kStages * S::kStage, wave, lane);
    if (wave >= S::WM * S::WN) return;
    float *const sums = of_x ? a.dXp : a.dWp;
    const int rows = of_x ? a.T : a.N;
    each<S::TM / 2>([&](auto half) {
        constexpr int i = 2 * half;
        const int col = k0 + (wm * S::TM + i) * 32;
        if (col >= a.K) return;
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            const int first = row0 + (wn * S::TN + j) * 32, row = first + l32;
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
                finish<T, S::kWaves == 8>(a, first, col, lane, lds + wave * kRowsRoom, v);
            } else {
                store_rows<T, false>(a.dW, first, a.N, col, a.K, lane, lds + wave * kRowsRoom, v);
            }
        }
    });
}

// What was cut into parts: rows of dX (x_blocks workgroups) or of dW (w_blocks), four neighbours to a thread; the last workgroups add up 64 columns of dbias each.
template <typename T>
__global__ __launch_bounds__(256) void linear_ends_kernel(const GradArgs a, int x_blocks, int w_blocks)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if ((int)blockIdx.x >= x_blocks + w_blocks) {
        __shared__ float sums[4][64];
        const int n = ((int)blockIdx.x - x_blocks - w_blocks) * 64 + lane;
        float s = 0.0f;
        if (n < a.N) {
#pragma unroll 8
            for (int p = wave; p < a.db_parts; p += 4) s += a.db[(int64_t)p * a.N + n];
        }
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && n < a.N) a.dbias[n] = sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
        return;
    }
    const bool of_x = (int)blockIdx.x < x_blocks;
    const int rows = of_x ? a.T : a.N, quads = a.K / 4;
    const int64_t i = (int64_t)((int)blockIdx.x - (of_x ? 0 : x_blocks)) * 256 + threadIdx.x;
    const int row = (int)(i / quads), col = (int)(i - (int64_t)row * quads) * 4;
    if (row >= rows) return;
    const int64_t at = (int64_t)row * a.K + col;
    float g[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    add_parts((of_x ? a.dXp : a.dWp) + at, (int64_t)rows * a.K, of_x ? a.x_parts : a.w_parts, g);
    if (of_x && a.act != QB_ACT_NONE) {
        float z[4];
        if (a.pre_codes) kept4(z, a.pre_codes, a.pre_scales, row, a.K, col);
        else load4<T>(a.pre, at, 4, z);
        slope(a.act, z, g);
    }
    store4<T>(of_x ? a.dX : a.dW, at, 4, g);
}

// no token: gradients of zero
__global__ __launch_bounds__(256) void linear_zero_kernel(uint16_t *dW, float *dbias, int64_t n, int64_t N)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n || i < N; i += (int64_t)gridDim.x * 256) {
        if (dW && i < n) dW[i] = 0;
        if (dbias && i < N) dbias[i] = 0.0f;
    }
}

typedef Tile<2, 4, 4, 2, 2> Large;     // 256 x 256
typedef Tile<2, 2, 2, 2, 2> Middle;    // 128 x 128
typedef Tile<1, 4, 2, 1, 3> Small;     // 64 x 128
typedef Tile<1, 2, 2, 1, 3, 2> Least;  // 64 x 64

struct Plan {
    int size, x_tiles, w_tiles, x_parts, w_parts;  // 0 least .. 3 large
};
// When `places` workgroups have done `n1` tasks of time `t1` and then `n2` shorter ones of `t2`, each taking the next as it gets free.
double done_at(int64_t n1, double t1, int64_t n2, double t2, int64_t places)
{
    const int64_t late = n1 % places;  // places with one long task more than the others
    const double early = (double)(n1 / places) * t1;
    int64_t a = 0, b = 0;  // short tasks behind the long ones of a late place, and of an early one
    double end = early + (late ? t1 : 0.0);
    while (late * a + (places - late) * b < n2) {
        const double next_a = early + t1 + (double)(a + 1) * t2, next_b = early + (double)(b + 1) * t2;
        if (late && next_a <= next_b) ++a, end = std::max(end, next_a);
        else ++b, end = std::max(end, next_b);
    }
    return end;
}
// Which tiles, and into how many parts their contractions are cut: the shortest time by that.  Parts cost the launch that adds them up, 3 us, and their bytes, twice, at 3 TB/s
// (4 where they leave the L2).  Measured over three sets of operands in turn (modelled), us: 390 x 768 by 768 least 8.1 (7.0), small 9.1 (10.3), middle 12.0 (13.2);
// 1000 x 1024 by 1024 13.3 (12.1), 13.9 (11.9), 18.4 (15.7); 390 x 2304 by 768 least 15.9 (13.0), with dX in 2 parts 16.8 (16.5), small with dX in 3 parts 15.2 (17.7).  Large, dW whole,
// in 2, 3 and 4 parts: 8190 x 1024 by 4096 232 (229), 162 (154), 154 (171), 155 (160); 16384 x 4096 by 1024 451 (446), 270 (247), 275 (284), 268 (253).
template <typename S>
void try_tiles(Plan &best, double &least, const Cost &c, bool dx, bool dw, int64_t T, int64_t N, int64_t K)
{
    constexpr bool kAlone = S::kWaves == 8;  // one workgroup to a CU
    const int64_t kt = (K + S::BM - 1) / S::BM, x_tiles = dx ? kt * ((T + S::BN - 1) / S::BN) : 0, w_tiles = dw ? kt * ((N + S::BN - 1) / S::BN) : 0;
    const int x_steps = dx ? (int)((N + 63) / 64) : 0, w_steps = dw ? (int)((T + 63) / 64) : 0, longest = std::max(x_steps, w_steps);
    const double kb = ((double)x_tiles * x_steps + (double)w_tiles * w_steps) * ((S::BM + S::BN) / 8.0);
    if (c.ends + kb / (256 * c.rate) >= least) return;
    for (const int cut : {1, 2, 3, 4, 6, 8, 12, 16}) {  // of the longer contraction; the other one is cut to the same length
        if (cut > 1 && cut > longest / 2) break;
        const int length = (longest + cut - 1) / cut, x = std::max(1, (x_steps + length - 1) / length), w = std::max(1, (w_steps + length - 1) / length);
        const double tasks = (double)(x_tiles * x + w_tiles * w), chain = length * c.step;
        const bool rounds = tasks > 1.1 * c.room;  // (the last of several is not full; of one, a CU has a whole number of workgroups)
        const double share = rounds ? kb / 256 : kb / tasks * (1 + (int)(tasks * (0.97 / 256)));
        double cost;
        if (kAlone && tasks < 64.0 * c.room) {
            const double tx = c.ends + (double)((x_steps + x - 1) / x) * c.step, tw = c.ends + (double)((w_steps + w - 1) / w) * c.step;
            cost = tx >= tw ? done_at(x_tiles * x, tx, w_tiles * w, tw, c.room) : done_at(w_tiles * w, tw, x_tiles * x, tx, c.room);
            if (dx && dw) cost += 0.1 * std::abs(tx - tw);  // (tiles of both kinds at once have less in common in the L2)
        } else {
            cost = c.ends * std::max(1.0, tasks / c.room) + std::max(chain, share / c.rate) + (rounds ? 0.25 * chain : 0.0);
        }
        if (x > 1 || w > 1) cost += 3.0 + ((x > 1 ? (double)x * T : 0.0) + (w > 1 ? (double)w * N : 0.0)) * K * (kAlone ? 2e-6 : 2.8e-6);
        if (cost < least) {
            least = cost;
            best = {c.size, (int)x_tiles, (int)w_tiles, x, w};
        }
        if (rounds && chain * c.rate < 0.5 * share) break;  // (many short tiles: cutting them gains nothing)
    }
}
Plan plan_of(const qb_linear_grads &l)
{
    const bool dx = l.dX != nullptr, dw = l.dW != nullptr;
    Plan p = {0, 0, 0, 1, 1};
    if (!dx && !dw) return p;
    double least = 1e300;
    try_tiles<Least>(p, least, {0, 512, 4.0, 0.25, 63.0}, dx, dw, l.T, l.N, l.K);
    try_tiles<Large>(p, least, {3, 256, 6.0, 1.6, 42.0}, dx, dw, l.T, l.N, l.K);
    try_tiles<Middle>(p, least, {2, 512, 6.0, 0.6, 53.0}, dx, dw, l.T, l.N, l.K);
    try_tiles<Small>(p, least, {1, 512, 5.5, 0.4, 65.0}, dx, dw, l.T, l.N, l.K);
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
    a.x_blocks = expand ? (l.T * (l.K / 8) + 256 * kAtOnce - 1) / (256 * kAtOnce) : 0;
    a.db_parts = !l.dbias ? 0 : l.dW ? p.w_parts : a.t_blocks;
    if (!l.dbias || l.dW) a.t_blocks = 0;
    a.y_blocks = stage ? (l.T * (a.N8 / 8) + 256 * kAtOnce - 1) / (256 * kAtOnce) : 0;
    if (expand) a.Xs = reinterpret_cast<uint16_t *>(take((size_t)a.T * a.K * 2));
    if (stage) a.dYs = reinterpret_cast<uint16_t *>(take((size_t)a.T * a.N8 * 2));
    if (l.dbias && !(l.dW && a.db_parts == 1)) a.db = reinterpret_cast<float *>(take((size_t)a.db_parts * a.N * 4));
    if (p.x_parts > 1) a.dXp = reinterpret_cast<float *>(take((size_t)p.x_parts * a.T * a.K * 4));
    if (p.w_parts > 1) a.dWp = reinterpret_cast<float *>(take((size_t)p.w_parts * a.N * a.K * 4));
    return at;
}

template <typename T>
qb_status launch(const GradArgs &a, int size, hipStream_t st)
{
    const int64_t first = a.x_blocks + a.y_blocks + (int64_t)a.n_blocks * a.t_blocks;
    for (int64_t at = 0; at < first; at += kMostBlocks) linear_prepare_kernel<T><<<(int)std::min(first - at, kMostBlocks), 256, 0, st>>>(a, at);
    const int groups = a.x_tiles * a.x_parts + a.w_tiles * a.w_parts;
    if (groups > 0) {
        if (size == 3) linear_grads_kernel<T, Large><<<groups, 64 * Large::kWaves, 0, st>>>(a);
        else if (size == 2) linear_grads_kernel<T, Middle><<<groups, 64 * Middle::kWaves, 0, st>>>(a);
        else if (size == 1) linear_grads_kernel<T, Small><<<groups, 64 * Small::kWaves, 0, st>>>(a);
        else linear_grads_kernel<T, Least><<<groups, 64 * Least::kWaves, 0, st>>>(a);
    }
    const auto blocks = [&](int64_t rows) { return (int)((rows * (a.K / 4) + 255) / 256); };
    const int x_blocks = a.dXp ? blocks(a.T) : 0, w_blocks = a.dWp ? blocks(a.N) : 0, ends = x_blocks + w_blocks + (a.dbias && !(a.dW && a.db_parts == 1) ? (a.N + 63) / 64 : 0);
    if (ends > 0) linear_ends_kernel<T><<<ends, 256, 0, st>>>(a, x_blocks, w_blocks);
    return launch_status();
}

}  // namespace

// host, pure: Plan::size of a call, and into how many parts the contractions of dX and dW are cut
int linear_bwd_plan(const qb_linear_grads *l, int *x_parts, int *w_parts)
{
    const Plan p = plan_of(*l);
    *x_parts = p.x_parts;
    *w_parts = p.w_parts;
    return p.size;
}

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
