// Softmax cross entropy behind the projection to the vocabulary, and its gradients.
//
//   z[t,v] = X[t].W[v] + bias[v];  lse[t] = log sum_v exp z;  loss[t] = lse[t] - z[t, target]
//   d[t,v] = dloss[t] (exp(z - lse[t]) - [v = target]);  dX = d W;  dW = d^T X;  dbias = sum_t d
//
// Only tokens that have a target take part: a first launch numbers them, the products fetch their rows of X through that list.
// The logits are formed tile by tile and never written: the forward keeps a maximum and a sum per token and tile, the
// backward forms them again, piece by piece of the vocabulary, and writes d of one piece in bfloat16, from which dX and dW take their share.
// d is held relative to the largest |dloss|, which multiplies the binary32 sums: the weight 1 / n of a mean over n tokens is
// then 1, where rounding d itself would put one error of up to 2^-8 on every token alike.
#include "qb_tiles.hpp"
#include <algorithm>

namespace qb {
namespace {

constexpr int64_t kMost = 1 << 24;              // tokens, words
constexpr int64_t kPieceBytes = 1024ll << 20;   // d of a piece, at most (16384 tokens: 32768 words), or of kRowPad words
constexpr float kLow = -1.0e30f;               // the maximum of no words (finite, also in powers of two)
constexpr int kRowPad = 256;                    // the list of tokens is padded to this

struct Counted {
    int n;        // tokens that have a target
    float scale;  // the largest |dloss| among them, and a normal number
    int slices;   // that the contraction of a tile of dX is cut into
    int pad[61];
};

// the shapes of the gradients' tiles and the number of workgroups at work
struct Work {
    int bm, bn, wbm, wbn, groups;
};
// Tiles of dX (x) and dW (w) come one after the other, id by id, to workgroups in turn.  A tile of dX runs over all words of the
// piece; it is cut into as many slices as make the longest share of a workgroup shortest, a tile counted as its steps and four more.
__device__ __host__ inline int most_slices(int x_tiles, int groups) { return x_tiles * 64 <= 2 * groups ? 64 : 2 * groups / x_tiles > 1 ? 2 * groups / x_tiles : 1; }
__device__ inline int best_slices(const Work &k, int n, int K, int words, int lane)  // (of one wavefront: a lane to a number)
{
    const int x_tiles = max(1, (n + k.bn - 1) / k.bn * ((K + k.bm - 1) / k.bm)), w_tiles = (words + k.wbn - 1) / k.wbn * ((K + k.wbm - 1) / k.wbm);
    const int steps = words / 64, most = min(most_slices(x_tiles, k.groups), max(1, steps / 4)), w = (n + 63) / 64 + 4;
    const int s = min(lane + 1, most), all = x_tiles * s, x = (steps + s - 1) / s + 4, full = all / k.groups, mixed = all % k.groups ? 1 : 0;
    const int64_t share = (int64_t)full * x + mixed * max(x, w) + (int64_t)max(0, (all + w_tiles + k.groups - 1) / k.groups - full - mixed) * w;
    int64_t best = share * 64 + s - 1;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = min(best, __shfl_xor(best, o));
    return (int)(best & 63) + 1;
}

// of 1024 tokens
struct Count {
    int n, someone;  // that have a target, and one of them or -1
    float top;       // the largest |dloss| among them
};

struct RowInfo {
    int token, target;
    float lse2, weight;  // backward: lse / ln 2, dloss
};

struct LossArgs {
    const uint16_t *X, *W;
    const float *bias, *dloss;
    const int64_t *targets;
    int T, V, K;
    Counted *counted;
    Count *counts;   // of every 1024 tokens, or null where these are few
    RowInfo *info;   // [Tp] of every counted row; padded
    int *place;      // [T] the row of a token; -1 where it has no target
    float *start;    // [Vp] the bias, -infinity behind the last word
    // forward
    float *loss, *lse;
    v2f *part;       // [vocabulary tiles][Tp] maximum, sum
    float *hit;      // [Tp] the target's logit
    // backward
    int v0, piece;   // this piece's first word and width (a multiple of kRowPad)
    uint16_t *d;     // [Tp][piece]
    uint16_t *Xc;    // [Tp][K] the rows that have a target
    float *db;       // [token tiles][V], or null
    float *dXs;      // tiles of dX: [tile][slice], binary32
    uint16_t *dX, *dW;
    float *dbias;
    int Tp, Vp;
    Work work;
};

__device__ __forceinline__ bool is_word(int64_t t, int V) { return t >= 0 && t < V; }

// Of many tokens a launch before the next counts every 1024.
template <bool BACKWARD>
__global__ __launch_bounds__(256) void loss_count_kernel(const LossArgs a)
{
    __shared__ Count each[4];
    const int tid = threadIdx.x, wave = tid >> 6;
    int n = 0, someone = -1;
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = (int)blockIdx.x * 1024 + i * 256 + tid;
        if (t >= a.T || !is_word(a.targets[t], a.V)) continue;
        ++n;
        someone = t;
        if constexpr (BACKWARD) top = fmaxf(top, fabsf(a.dloss[t]));
    }
    const uint64_t any = __builtin_amdgcn_ballot_w64(someone >= 0);
    const Count mine = {wave_sum(n), any ? __builtin_amdgcn_readlane(someone, __builtin_ctzll(any)) : -1, wave_max(top)};
    if ((tid & 63) == 0) each[wave] = mine;
    __syncthreads();
    if (tid != 0) return;
    Count c = each[0];
    for (int i = 1; i < 4; ++i) c = {c.n + each[i].n, max(c.someone, each[i].someone), fmaxf(c.top, each[i].top)};
    a.counts[blockIdx.x] = c;
}

// Numbers the tokens that have a target, in order.  A workgroup does 1024 tokens; it counts those before them itself, or adds up the counts.  The list
// is padded with one of them: a row of X that has no target may hold anything, and even with a weight of zero it would reach dW and dbias.
template <bool BACKWARD>
__global__ __launch_bounds__(1024) void loss_rows_kernel(const LossArgs a)
{
    __shared__ int sums[16];
    __shared__ float tops[16];
    __shared__ int someone[16];  // a token that has a target, or -1
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, groups = (a.T + 1023) / 1024;
    if ((int)blockIdx.x >= groups) {  // the further workgroups: where the sums start
        const int v = ((int)blockIdx.x - groups) * 1024 + tid;
        if (v < a.Vp) a.start[v] = v >= a.V ? -__builtin_inff() : a.bias ? a.bias[v] : 0.0f;
        return;
    }
    const int first = blockIdx.x * 1024, t = first + tid;
    const bool last = (int)blockIdx.x == groups - 1;
    int before = 0, counted = -1;
    float top = 0.0f;
    if (a.counts) {
#pragma unroll 4
        for (int i = tid; i < (int)blockIdx.x; i += 1024) {
            const Count c = a.counts[i];
            before += c.n;
            counted = max(counted, c.someone);
            top = fmaxf(top, c.top);
        }
    }
#pragma unroll 8
    for (int i = tid; i < (a.counts ? 0 : first); i += 1024) {
        const bool word = is_word(a.targets[i], a.V);
        before += word;
        if (BACKWARD && last && word) {
            top = fmaxf(top, fabsf(a.dloss[i]));
            counted = i;
        }
    }
    const bool mine = t < a.T && is_word(a.targets[t], a.V);
    if (BACKWARD && last && mine) {
        top = fmaxf(top, fabsf(a.dloss[t]));
        counted = t;
    }
    const uint64_t who = __builtin_amdgcn_ballot_w64(mine);
    before = wave_sum(before);
    if constexpr (BACKWARD) {
        top = wave_max(top);
        const uint64_t any = __builtin_amdgcn_ballot_w64(counted >= 0);
        if (any) counted = __builtin_amdgcn_readlane(counted, __builtin_ctzll(any));
    }
    if (lane == 0) {
        sums[wave] = before;
        tops[wave] = top;
        someone[wave] = counted;
    }
    __syncthreads();
    int start = 0;
    for (int i = 0; i < 16; ++i) start += sums[i];
    __syncthreads();
    if (lane == 0) sums[wave] = __builtin_popcountll(who);
    __syncthreads();
    int all = 0;
    for (int i = 0; i < 16; ++i) {
        if (i == wave) before = start + all;
        all += sums[i];
    }
    all += start;
    const int at = before + __builtin_popcountll(who & ((1ull << lane) - 1));
    if (t < a.T) {
        if (mine) {
            RowInfo r = {t, (int)a.targets[t], 0.0f, 0.0f};
            if constexpr (BACKWARD) {
                r.lse2 = a.lse[t] * 1.44269504088896341f;
                r.weight = a.dloss[t];
            }
            a.info[at] = r;
        }
        if constexpr (BACKWARD) {
            a.place[t] = mine ? at : -1;
        } else if (!mine) {
            a.loss[t] = 0.0f;
            a.lse[t] = 0.0f;
        }
    }
    if (!last) return;
    if (tid == 0) {
        a.counted->n = all;
        float s = 1.17549435e-38f;  // (one over less would be infinite)
        for (int i = 0; i < 16; ++i) s = fmaxf(s, tops[i]);
        a.counted->scale = s;
    }
    if (BACKWARD && wave == 1) {
        const int slices = best_slices(a.work, all, a.K, min(a.piece, (a.V + 63) / 64 * 64), lane);
        if (lane == 0) a.counted->slices = slices;
    }
    const int end = min(a.Tp, (all + kRowPad - 1) / kRowPad * kRowPad);
    int pad = 0;  // (forward: what padding gives is not written)
    if constexpr (BACKWARD)
        for (int i = 0; i < 16; ++i) pad = max(pad, someone[i]);
    if (all + tid < end) a.info[all + tid] = RowInfo{pad, -1, __builtin_inff(), 0.0f};  // (exponentials of zero)
}

// ---- products ------------------------------------------------------------------------------------------------------
// Tiles of BM x BN results by WM x WN wavefronts, TM x TN blocks of 32 x 32 each; the contraction goes in steps of 64 through a ring of
// stages in LDS, one multiplied while the others are under way.  An operand lies in LDS as it does in memory: rows of results with the
// contraction along them, or rows along the contraction (in blocks of 64 results), read turned.
template <int WM_, int WN_, int TM_, int TN_, int STAGES_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, kWaves = WM * WN, kStages = STAGES_;
    static constexpr int BM = 32 * WM * TM, BN = 32 * WN * TN;
    static constexpr int kStage = (BM + BN) * 128;
    // row number i that a lane copies
    static __device__ __forceinline__ int row(int i, int wave, int lane) { return (i * kWaves + wave) * 8 + (lane >> 3); }
};

// eight steps of the contraction in their own order: rows row0 + 8 * (lane / 32) ..
__device__ __forceinline__ v8s across_in_order(const uint8_t *tile, int row0, int col0, int lane)
{
    typedef Rows<64> R;
    typedef __attribute__((address_space(3))) v4s *turned;
    const int row = row0 + 8 * (lane >> 5) + ((lane >> 2) & 3), col = col0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const uint8_t *first = tile + R::at(row, col >> 3) + 2 * (col & 7), *second = tile + R::at(row + 4, col >> 3) + 2 * (col & 7);
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned)first), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned)second);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <bool ACROSS>
__device__ __forceinline__ v8s operand(const uint8_t *tile, int result, int sub, int lane)
{
    if constexpr (ACROSS) return across_in_order(tile + (result >> 6) * 8192, 16 * sub, result & 63, lane);
    else return *reinterpret_cast<const v8s *>(tile + Rows<64>::at(result + (lane & 31), 2 * sub + (lane >> 5)));
}

// acc += A B^T over one step, whose operands lie in a stage
template <typename S, bool A_ACROSS, bool B_ACROSS>
__device__ __forceinline__ void step(v16f (&acc)[S::TM][S::TN], const uint8_t *ta, int wave, int lane)
{
    const int wm = wave / S::WN, wn = wave - wm * S::WN;
    const uint8_t *const tb = ta + S::BM * 128;
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) {
        v8s x[S::TM], y[S::TN];
#pragma unroll
        for (int i = 0; i < S::TM; ++i) x[i] = operand<A_ACROSS>(ta, (wm * S::TM + i) * 32, sub, lane);
#pragma unroll
        for (int j = 0; j < S::TN; ++j) y[j] = operand<B_ACROSS>(tb, (wn * S::TN + j) * 32, sub, lane);
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int j = 0; j < S::TN; ++j) acc[i][j] = Bf16::mma32(x[i], y[j], acc[i][j]);
    }
}

// acc += A B^T over steps [s0, s1); row_a(r, s) is the address of LDS row r of step s: of result r (along), or for r = 64 * block + k of
// step k, result block `block` (across).  The addresses must not come from memory: a load between the copies waits for those before it.
template <typename S, bool A_ACROSS, bool B_ACROSS, typename FA, typename FB>
__device__ __forceinline__ void multiply(v16f (&acc)[S::TM][S::TN], uint8_t *lds, int s0, int s1, int wave, int lane, const FA &row_a, const FB &row_b)
{
    const uint32_t lds0 = lds_address(lds);
    constexpr int NA = S::BM / 8 / S::kWaves, NB = S::BN / 8 / S::kWaves, kAhead = S::kStages - 1;
    static_assert(NA * 8 * S::kWaves == S::BM && NB * 8 * S::kWaves == S::BN, "every wavefront copies the same number of times");
    const auto fetch = [&](int s, int stage) {
        const uint32_t to = lds0 + stage * S::kStage;
        typedef Rows<64> R;
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int first = (i * S::kWaves + wave) * 8, r = first + R::copy_row(lane);
            copy16(row_a(i, r, s) + 8 * R::copy_chunk(r, lane), to + first * 128);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int first = (i * S::kWaves + wave) * 8, r = first + R::copy_row(lane);
            copy16(row_b(i, r, s) + 8 * R::copy_chunk(r, lane), to + S::BM * 128 + first * 128);
        }
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (s0 + u < s1) fetch(s0 + u, u);
    int stage = 0;
    for (int s = s0; s < s1; ++s) {
        if (s + kAhead <= s1) wait_copies<(kAhead - 1) * (NA + NB)>();  // (younger steps' stay under way)
        else wait_copies<0>();
        barrier();
        if (s + kAhead < s1) fetch(s + kAhead, stage == 0 ? kAhead : stage - 1);  // (into the stage that the last step was multiplied from)
        step<S, A_ACROSS, B_ACROSS>(acc, lds + stage * S::kStage, wave, lane);
        stage = stage == kAhead ? 0 : stage + 1;
    }
    barrier();  // the stages are free again
}
template <int M, int N>
__device__ __forceinline__ void clear(v16f (&x)[M][N])
{
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) x[i][j][k] = 0.0f;
}
// Workgroups are dealt to the XCDs in turn: numbers that follow each other on one XCD get neighbouring tiles.
__device__ __forceinline__ int first_tile() { return (gridDim.x & 7) ? (int)blockIdx.x : (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)); }

// the sum over the 32 lanes of a half, in every lane
__device__ __forceinline__ float half_sum(float x)
{
    const auto add = [&](auto ctrl) { x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    add(std::integral_constant<int, 0xB1>());   // lane ^ 1
    add(std::integral_constant<int, 0x4E>());   // lane ^ 2
    add(std::integral_constant<int, 0x141>());  // the other four of eight
    add(std::integral_constant<int, 0x140>());  // the other eight of sixteen
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// Logits, a tile of words by tokens at a time: a lane's results belong to one token.  The sums start from the bias, and from
// -infinity for words past the end, which so have no weight.  A workgroup's tiles are one stream of steps: the first steps of a tile,
// what is known of its rows and where its sums start are on their way while the tile before is ended.  All of it comes
// through copies to LDS: a load into registers would have to wait for the copies in front of it.  Bound by the matrix cores, at the clock that
// power allows, and the exponentials behind each tile: 8192 tokens, 30522 words, 1024 units 482 us forward (1.06 PFLOP/s), 556 us backward, where
// d is written; a library's product of these sizes takes 504 us.  Few tokens are bound by W's bytes: 58 tokens, 768 units 10 us (4.6 TB/s).
template <typename S, bool BACKWARD>
__global__ __launch_bounds__(64 * S::kWaves, 1) void loss_logits_kernel(const LossArgs a)
{
    constexpr int kAhead = S::kStages - 1, kRing = S::kStages + 2;  // the tile at work, those ahead (of one step), and the next one's rows on their way
    constexpr int NA = S::BM / 8 / S::kWaves, NB = S::BN / 8 / S::kWaves;
    constexpr int kBoth = BACKWARD ? S::WN * S::BM * 4 : S::WM * S::BN * 8;
    __shared__ __align__(1024) uint8_t lds[S::kStages * S::kStage];
    __shared__ __align__(1024) RowInfo info[kRing][S::BN];
    __shared__ __align__(1024) float begin[kRing][S::BM > 256 ? S::BM : 256];  // (a copy fills 256)
    __shared__ __align__(16) uint8_t shared[kBoth];
    typedef Rows<64> R;
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave - wm * S::WN;
    const int n = a.counted->n, K = a.K, steps = K / 64, grid = (int)gridDim.x;
    const float inv = BACKWARD ? 1.0f / a.counted->scale : 0.0f;
    const int words = BACKWARD ? a.piece / S::BM : (a.V + S::BM - 1) / S::BM, tiles = words * ((n + S::BN - 1) / S::BN);
    const int tile0 = first_tile();
    if (BACKWARD && a.v0 == 0) {  // the rows that take part, side by side, for dW
        const int64_t chunks = (int64_t)((n + S::BN - 1) / S::BN * S::BN) * (K / 8);
        for (int64_t c = (int64_t)blockIdx.x * (64 * S::kWaves) + threadIdx.x; c < chunks; c += (int64_t)grid * (64 * S::kWaves)) {
            const int row = (int)(c / (K / 8)), k = (int)(c - (int64_t)row * (K / 8)) * 8;
            *reinterpret_cast<v4u *>(a.Xc + (int64_t)row * K + k) = *reinterpret_cast<const v4u *>(a.X + (int64_t)a.info[row].token * K + k);
        }
    }
    if (tile0 >= tiles) return;
    const auto words_of = [&](int tile) { return (BACKWARD ? a.v0 : 0) + tile % words * S::BM; };
    const auto rows_of = [&](int tile) { return tile / words * S::BN; };
    // a tile's rows and starts on their way (64 entries of 16 bytes a copy)
    const auto announce = [&](int tile, int ring) {
        constexpr int kInfo = S::BN / 64, kBegin = S::BM / 256 > 0 ? S::BM / 256 : 1;
        static_assert(kInfo + kBegin <= S::kWaves, "a copy to a wavefront");
        if (wave < kInfo) copy16(a.info + rows_of(tile) + wave * 64 + lane, lds_address(info[ring]) + wave * 1024);
        else if (wave < kInfo + kBegin) {  // (tiles of 64 words: a quarter of the copy is used)
            const int at = words_of(tile) + (wave - kInfo) * 256 + 4 * (S::BM >= 256 ? lane : lane & 15);
            copy16(a.start + at, lds_address(begin[ring]) + (wave - kInfo) * 1024);
        }
    };
    // ---- the copies' side of the stream: step `cs` of tile `ct`, the `cn`-th of this workgroup
    int ct = tile0, cs = 0, cn = 0;
    const uint16_t *x[NB], *w[NA];
    const auto enter = [&]() {
        const int v0 = words_of(ct);
#pragma unroll
        for (int i = 0; i < NB; ++i) x[i] = a.X + (int64_t)info[cn % kRing][S::row(i, wave, lane)].token * K + 8 * R::copy_chunk(S::row(i, wave, lane), lane);
#pragma unroll
        for (int i = 0; i < NA; ++i) w[i] = a.W + (int64_t)min(v0 + S::row(i, wave, lane), a.V - 1) * K + 8 * R::copy_chunk(S::row(i, wave, lane), lane);
        if (ct + grid < tiles) announce(ct + grid, (cn + 1) % kRing);
    };
    const uint32_t lds0 = lds_address(lds);
    const auto fetch = [&](int stage) {
        if (ct >= tiles) return;
        const uint32_t to = lds0 + stage * S::kStage;
#pragma unroll
        for (int i = 0; i < NA; ++i) copy16(w[i] + cs * 64, to + (i * S::kWaves + wave) * 1024);
#pragma unroll
        for (int i = 0; i < NB; ++i) copy16(x[i] + cs * 64, to + S::BM * 128 + (i * S::kWaves + wave) * 1024);
        if (++cs < steps) return;
        cs = 0;
        ct += grid;
        ++cn;
        if (ct >= tiles) return;
        if (steps <= kAhead) {  // the next tile's rows may not have come yet
            wait_copies<0>();
            barrier();
        }
        enter();
    };
    announce(ct, 0);
    wait_copies<0>();
    barrier();
    enter();
    for (int u = 0; u < kAhead; ++u) fetch(u);

    const int mine = (tiles - tile0 + grid - 1) / grid;  // tiles of this workgroup
    int stage = 0, left = mine * steps;
    constexpr float kLog2e = 1.44269504088896341f;
    for (int number = 0, tile = tile0; tile < tiles; tile += grid, ++number) {
        const int tt = tile / words, tv = tile - tt * words, t0 = tt * S::BN, v0 = words_of(tile), ring = number % kRing;
        v16f z[S::TM][S::TN];
        for (int s = 0; s < steps; ++s, --left) {
            constexpr int kStores = BACKWARD && kAhead == 1 ? S::TM * S::TN * 2 : 0;  // of d, at a tile's end, behind the copies that are waited for
            asm volatile("" ::: "memory");  // (the stores stay in front of the wait that counts them)
            if (kAhead == 1 && kStores > 0 && s == 0 && number > 0) wait_copies<kStores>();
            else if (left >= kAhead) wait_copies<(kAhead - 1) * (NA + NB)>();  // (younger steps' stay under way)
            else wait_copies<0>();
            barrier();
            fetch(stage == 0 ? kAhead : stage - 1);  // (into the stage that the last step was multiplied from)
            if (s == 0) {
#pragma unroll
                for (int i = 0; i < S::TM; ++i)
#pragma unroll
                    for (int k = 0; k < 16; k += 4) {
                        const v4f b = *reinterpret_cast<const v4f *>(&begin[ring][(wm * S::TM + i) * 32 + 2 * k + 4 * hf]);
#pragma unroll
                        for (int j = 0; j < S::TN; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) z[i][j][k + e] = b[e];
                    }
            }
            step<S, false, false>(z, lds + stage * S::kStage, wave, lane);
            stage = stage == kAhead ? 0 : stage + 1;
        }
        if constexpr (!BACKWARD) {
            v2f *const both = reinterpret_cast<v2f *>(shared);  // [WM][BN] maximum, sum of a wavefront's words
#pragma unroll
            for (int j = 0; j < S::TN; ++j) {
                float m = z[0][j][0];
#pragma unroll
                for (int i = 0; i < S::TM; ++i)
#pragma unroll
                    for (int k = 0; k < 16; k += 2) m = max3(m, z[i][j][k], z[i][j][k + 1]);
                m = fmaxf(halves_max(m), kLow);
                const float m2 = m * kLog2e;
                float l = 0.0f;
#pragma unroll
                for (int i = 0; i < S::TM; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) l += __builtin_amdgcn_exp2f(__builtin_fmaf(z[i][j][k], kLog2e, -m2));
                l = halves_sum(l);
                const int row = (wn * S::TN + j) * 32 + l32;
                if (hf == 0) both[wm * S::BN + row] = v2f{m, l};
                const int target = info[ring][row].target - v0 - wm * S::TM * 32;
                if (__builtin_amdgcn_ballot_w64(target >= 0 && target < S::TM * 32)) {  // (one wavefront in four at 30522 words)
                    bool have = false;
                    float hit = 0.0f;
#pragma unroll
                    for (int i = 0; i < S::TM; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (target - 4 * hf == i * 32 + 8 * (k >> 2) + (k & 3)) {
                                hit = z[i][j][k];
                                have = true;
                            }
                    if (have) a.hit[t0 + row] = hit;
                }
            }
            barrier();
            for (int r = threadIdx.x; r < S::BN; r += 64 * S::kWaves) {
                v2f x = both[r];
#pragma unroll
                for (int i = 1; i < S::WM; ++i) {
                    const v2f y = both[i * S::BN + r];
                    const float m = fmaxf(x[0], y[0]);
                    x = v2f{m, x[1] * __builtin_amdgcn_exp2f((x[0] - m) * kLog2e) + y[1] * __builtin_amdgcn_exp2f((y[0] - m) * kLog2e)};
                }
                a.part[(int64_t)tv * a.Tp + t0 + r] = x;
            }
        } else {
#pragma unroll
            for (int j = 0; j < S::TN; ++j) {
                const int row = (wn * S::TN + j) * 32 + l32;
                const RowInfo r = info[ring][row];
                const float w = r.weight * inv;
                const int target = r.target - v0 - wm * S::TM * 32;
#pragma unroll
                for (int i = 0; i < S::TM; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) z[i][j][k] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i][j][k], kLog2e, -r.lse2)) * w;
                if (__builtin_amdgcn_ballot_w64(target >= 0 && target < S::TM * 32)) {
#pragma unroll
                    for (int i = 0; i < S::TM; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) z[i][j][k] -= target - 4 * hf == i * 32 + 8 * (k >> 2) + (k & 3) ? w : 0.0f;
                }
                uint16_t *const to = a.d + (int64_t)(t0 + row) * a.piece + tv * S::BM + wm * S::TM * 32 + 8 * hf;
#pragma unroll
                for (int i = 0; i < S::TM; ++i)
#pragma unroll
                    for (int k = 0; k < 16; k += 8)
                        *reinterpret_cast<v4u *>(to + i * 32 + 2 * k) =
                            join_halves(v2u{Bf16::pair(z[i][j][k], z[i][j][k + 1]), Bf16::pair(z[i][j][k + 2], z[i][j][k + 3])},
                                        v2u{Bf16::pair(z[i][j][k + 4], z[i][j][k + 5]), Bf16::pair(z[i][j][k + 6], z[i][j][k + 7])});
            }
            if (a.db) {  // (uniform)
                float *const sums = reinterpret_cast<float *>(shared);  // [WN][BM] of d over a wavefront's tokens
#pragma unroll
                for (int i = 0; i < S::TM; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float x = z[i][0][k];
#pragma unroll
                        for (int j = 1; j < S::TN; ++j) x += z[i][j][k];
                        x = half_sum(x);
                        if (l32 == 0) sums[wn * S::BM + (wm * S::TM + i) * 32 + 8 * (k >> 2) + 4 * hf + (k & 3)] = x;
                    }
                barrier();
                for (int v = threadIdx.x; v < S::BM; v += 64 * S::kWaves) {
                    float x = 0.0f;
#pragma unroll
                    for (int i = 0; i < S::WN; ++i) x += sums[i * S::BM + v];
                    if (v0 + v < a.V) a.db[(int64_t)tt * a.V + v0 + v] = x;
                }
            }
        }
        // (the next step's barrier stands between these reads of `shared` and the next tile's writes)
    }
}

// loss and lse of 16 tokens from the maxima and sums of the vocabulary's tiles, sixteen threads to a token
__global__ __launch_bounds__(256) void loss_join_kernel(const LossArgs a, int words)
{
    __shared__ v2f both[16][16];
    const int n = a.counted->n, r = threadIdx.x & 15, q = threadIdx.x >> 4, row = blockIdx.x * 16 + r;
    if (blockIdx.x * 16 >= n) return;
    float m = kLow, l = 0.0f;
    const auto add = [&](v2f x) {
        const float top = fmaxf(m, x[0]);
        l = l * __expf(m - top) + x[1] * __expf(x[0] - top);
        m = top;
    };
    constexpr int kAtOnce = 8;
    for (int i = q; i < words; i += 16 * kAtOnce) {
        v2f x[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            x[u] = a.part[(int64_t)min(i + 16 * u, words - 1) * a.Tp + row];  // (rows past n are computed too)
            if (i + 16 * u >= words) x[u][1] = 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) add(x[u]);
    }
    both[q][r] = v2f{m, l};
    __syncthreads();
    if (q != 0 || row >= n) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) add(both[i][r]);
    const float lse = m + logf(l);
    const int token = a.info[row].token;
    a.lse[token] = lse;
    a.loss[token] = lse - a.hit[row];
}

// The piece's share of both gradients: results lie transposed in the products (hidden units by tokens or words), so that a lane
// holds neighbours of a row of dX or dW.  8192 tokens, 30522 words, 1024 units: 922 us, 1.11 PFLOP/s, the rate of a library's products of these sizes.
template <typename S, typename SW>  // tiles of dX, of dW
__global__ __launch_bounds__(64 * S::kWaves, 1) void loss_grads_kernel(const LossArgs a)
{
    static_assert(S::kWaves == SW::kWaves, "the same workgroups");
    constexpr int kX = S::kStages * S::kStage, kW = SW::kStages * SW::kStage;
    __shared__ __align__(1024) uint8_t lds[kX > kW ? kX : kW];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = a.counted->n, K = a.K;
    const float scale = a.counted->scale;
    const int kt = (K + S::BM - 1) / S::BM, kt_w = (K + SW::BM - 1) / SW::BM;
    const int words = min(a.piece, (a.V - a.v0 + 63) / 64 * 64);                 // of this piece, in whole steps
    const int x_tiles = kt * ((n + S::BN - 1) / S::BN), slices = a.counted->slices, x_steps = words / 64;
    const int w_tiles = kt_w * ((words + SW::BN - 1) / SW::BN), w_steps = (n + 63) / 64;
    for (int id = first_tile(); id < x_tiles * slices + w_tiles; id += gridDim.x) {
        if (id < x_tiles * slices) {
            const int wm = wave / S::WN, wn = wave - wm * S::WN;
            v16f acc[S::TM][S::TN];
            clear(acc);
            const int slice = id / x_tiles, tile = id - slice * x_tiles, tt = tile / kt,  // (neighbours read the same rows of W)
                      k0 = (tile - tt * kt) * S::BM, t0 = tt * S::BN;
            const int s0 = x_steps * slice / slices, s1 = x_steps * (slice + 1) / slices;
            if (s0 < s1)
                multiply<S, true, false>(acc, lds, s0, s1, wave, lane,
                    [&](int, int r, int s) { return a.W + (int64_t)min(a.v0 + s * 64 + (r & 63), a.V - 1) * K + min(k0 + (r & ~63), K - 64); },
                    [&](int, int r, int s) { return a.d + (int64_t)(t0 + r) * a.piece + s * 64; });
            float *const to = a.dXs + (int64_t)(tile * slices + slice) * S::BM * S::BN;
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
#pragma unroll
                for (int j = 0; j < S::TN; ++j)
#pragma unroll
                    for (int k = 0; k < 16; k += 4) {
                        v4f *const p = reinterpret_cast<v4f *>(to + ((wn * S::TN + j) * 32 + l32) * S::BM + (wm * S::TM + i) * 32 + 2 * k + 4 * hf);
                        v4f x = {acc[i][j][k], acc[i][j][k + 1], acc[i][j][k + 2], acc[i][j][k + 3]};
                        if (a.v0 > 0) x += *p;
                        *p = x;
                    }
        } else {
            const int wm = wave / SW::WN, wn = wave - wm * SW::WN;
            v16f acc[SW::TM][SW::TN];
            clear(acc);
            const int tile = id - x_tiles * slices, tv = tile / kt_w, k0 = (tile - tv * kt_w) * SW::BM, v0 = tv * SW::BN;
            if (w_steps > 0)
                multiply<SW, true, true>(acc, lds, 0, w_steps, wave, lane,
                    [&](int, int r, int s) { return a.Xc + (int64_t)(s * 64 + (r & 63)) * K + min(k0 + (r & ~63), K - 64); },
                    [&](int, int r, int s) { return a.d + (int64_t)(s * 64 + (r & 63)) * a.piece + v0 + (r & ~63); });
#pragma unroll
            for (int j = 0; j < SW::TN; ++j) {
                const int v = a.v0 + v0 + (wn * SW::TN + j) * 32 + l32;  // (words past the end are exchanged too, not written)
#pragma unroll
                for (int i = 0; i < SW::TM; ++i) {
                    const int k1 = k0 + (wm * SW::TM + i) * 32;
                    if (k1 >= K) continue;
#pragma unroll
                    for (int k = 0; k < 16; k += 8) {
                        const auto pairs = [&](int e) { return v2u{Bf16::pair(acc[i][j][e] * scale, acc[i][j][e + 1] * scale), Bf16::pair(acc[i][j][e + 2] * scale, acc[i][j][e + 3] * scale)}; };
                        const v4u w = join_halves(pairs(k), pairs(k + 4));
                        if (v < a.V) *reinterpret_cast<v4u *>(a.dW + (int64_t)v * K + k1 + 2 * k + 8 * hf) = w;
                    }
                }
            }
        }
    }
}

// dX from its slices, a zero row for a token without a target; the last workgroups join dbias
template <typename S>
__global__ __launch_bounds__(256) void loss_ends_kernel(const LossArgs a, int x_groups)
{
    const int n = a.counted->n, K = a.K, quads = K / 4;
    const float scale = a.counted->scale;
    if ((int)blockIdx.x >= x_groups) {
        const int v = ((int)blockIdx.x - x_groups) * 256 + threadIdx.x, tiles = (n + S::BN - 1) / S::BN;
        if (v >= a.V) return;
        float x = 0.0f;
#pragma unroll 8
        for (int i = 0; i < tiles; ++i) x += a.db[(int64_t)i * a.V + v];
        a.dbias[v] = x * scale;
        return;
    }
    const int kt = (K + S::BM - 1) / S::BM, slices = a.counted->slices;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)a.T * quads; i += (int64_t)x_groups * 256) {
        const int t = (int)(i / quads), k = (int)(i - (int64_t)t * quads) * 4, row = a.place[t];
        v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
        if (row >= 0) {
            const int tile = (row / S::BN) * kt + k / S::BM;
            const float *p = a.dXs + (int64_t)tile * slices * S::BM * S::BN + (row % S::BN) * S::BM + k % S::BM;
#pragma unroll 8
            for (int s = 0; s < slices; ++s) x += *reinterpret_cast<const v4f *>(p + (int64_t)s * S::BM * S::BN);
        }
        *reinterpret_cast<v2u *>(a.dX + (int64_t)t * K + k) = v2u{Bf16::pair(x[0] * scale, x[1] * scale), Bf16::pair(x[2] * scale, x[3] * scale)};
    }
}

// 256 x 256 fills a CU with one workgroup; with few tokens the weights' bytes are what counts, and 64 x 64 with four stages keeps
// 48 KB of them under way on every CU, two workgroups to a CU.  The host knows how many tokens there are, not how many have a target.
// 30522 words, 768 units, forward and backward, small and large: all of 128 tokens 81 and 108 us, of 256 118 and 114, of 512 195 and 146; but
// 58 of 390, the share of masked language modelling, 62 and about 108.  Up to 512 it is the share of the masked ones that counts.
typedef Shape<2, 4, 4, 2, 2> Large;
typedef Shape<2, 2, 1, 1, 4> Small;
typedef Shape<4, 1, 2, 2, 2> SmallW;  // dW of few tokens: one or two steps a tile, so larger ones
template <typename S> struct ForW { typedef S type; };
template <> struct ForW<Small> { typedef SmallW type; };
inline bool few(int64_t T) { return T <= 512; }

template <typename S>
constexpr int kAtWork = S::kWaves == 8 ? 256 : 512;  // workgroups of a launch: as many as are resident

inline size_t up(size_t v) { return (v + 255) / 256 * 256; }

// A workgroup that counts the tokens before its own reads all of their targets: work that grows with the square of T.  One launch and two, us: 32768
// tokens forward 6.9 and 3.6 + 3.9, backward 13.7 and 4.0 + 3.9; 4 194 304 tokens 6300 and 29 + 12.
inline bool count_apart(int64_t T) { return T > 32768; }

// where everything lies in the workspace; returns its size
size_t lay_out(LossArgs &a, uint8_t *base, bool backward)
{
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        uint8_t *p = base + at;
        at += up(bytes);
        return p;
    };
    const int bm = few(a.T) ? Small::BM : Large::BM, bn = few(a.T) ? Small::BN : Large::BN;
    a.work = few(a.T) ? Work{bm, bn, SmallW::BM, SmallW::BN, kAtWork<Small>} : Work{bm, bn, bm, bn, kAtWork<Large>};
    a.Tp = (int)((a.T + kRowPad - 1) / kRowPad * kRowPad);
    a.counted = reinterpret_cast<Counted *>(take(sizeof(Counted)));
    a.Vp = (int)(((int64_t)a.V + kRowPad - 1) / kRowPad * kRowPad);
    if (backward) {  // pieces of about one size
        const int64_t most = std::max<int64_t>(1, kPieceBytes / (2ll * a.Tp) / kRowPad), pieces = (a.Vp / kRowPad + most - 1) / most;
        a.piece = (int)((a.Vp / kRowPad + pieces - 1) / pieces * kRowPad);
        a.Vp = (int)(pieces * a.piece);
    }
    a.counts = count_apart(a.T) ? reinterpret_cast<Count *>(take((size_t)((a.T + 1023) / 1024) * sizeof(Count))) : nullptr;
    a.info = reinterpret_cast<RowInfo *>(take((size_t)a.Tp * sizeof(RowInfo)));
    a.start = reinterpret_cast<float *>(take((size_t)a.Vp * 4));
    if (!backward) {
        a.part = reinterpret_cast<v2f *>(take((size_t)((a.V + bm - 1) / bm) * a.Tp * 8));
        a.hit = reinterpret_cast<float *>(take((size_t)a.Tp * 4));
        return at;
    }
    a.place = reinterpret_cast<int *>(take((size_t)a.T * 4));
    a.d = reinterpret_cast<uint16_t *>(take((size_t)a.Tp * a.piece * 2));
    a.Xc = reinterpret_cast<uint16_t *>(take((size_t)a.Tp * a.K * 2));
    a.db = reinterpret_cast<float *>(take((size_t)(a.Tp / bn) * a.V * 4));
    const int64_t x_tiles = (int64_t)(a.Tp / bn) * ((a.K + bm - 1) / bm);
    int64_t slots = 0;  // the most tiles and slices that any number of counted tokens gives
    for (int64_t t = 1; t <= a.Tp / bn; ++t) {
        const int64_t tiles = t * ((a.K + bm - 1) / bm);
        slots = std::max(slots, tiles * most_slices((int)tiles, a.work.groups));
        if (tiles > 2 * a.work.groups) {
            slots = std::max(slots, x_tiles);
            break;
        }
    }
    a.dXs = reinterpret_cast<float *>(take((size_t)slots * bm * bn * 4));
    return at;
}

bool shape_ok(int64_t T, int64_t V, int64_t K) { return T >= 1 && T <= kMost && V >= 1 && V <= kMost && k_ok(K); }

template <typename S>
qb_status forward(const LossArgs &a, hipStream_t st)
{
    const int words = (a.V + S::BM - 1) / S::BM;
    const int64_t tiles = (int64_t)words * (a.Tp / S::BN);
    if (a.counts) loss_count_kernel<false><<<(a.T + 1023) / 1024, 256, 0, st>>>(a);
    loss_rows_kernel<false><<<(a.T + 1023) / 1024 + (a.Vp + 1023) / 1024, 1024, 0, st>>>(a);
    loss_logits_kernel<S, false><<<(int)std::min<int64_t>(tiles, kAtWork<S>), 64 * S::kWaves, 0, st>>>(a);
    loss_join_kernel<<<(a.T + 15) / 16, 256, 0, st>>>(a, words);
    return launch_status();
}

template <typename S>
qb_status backward(LossArgs a, hipStream_t st)
{
    if (a.counts) loss_count_kernel<true><<<(a.T + 1023) / 1024, 256, 0, st>>>(a);
    loss_rows_kernel<true><<<(a.T + 1023) / 1024 + (a.Vp + 1023) / 1024, 1024, 0, st>>>(a);
    for (a.v0 = 0; a.v0 < a.V; a.v0 += a.piece) {
        const int64_t tiles = (int64_t)(a.piece / S::BM) * (a.Tp / S::BN);
        loss_logits_kernel<S, true><<<(int)std::min<int64_t>(tiles, kAtWork<S>), 64 * S::kWaves, 0, st>>>(a);
        loss_grads_kernel<S, typename ForW<S>::type><<<kAtWork<S>, 64 * S::kWaves, 0, st>>>(a);
    }
    const int x_groups = (int)std::min<int64_t>(4096, ((int64_t)a.T * (a.K / 4) + 255) / 256);
    loss_ends_kernel<S><<<x_groups + (a.dbias ? (a.V + 255) / 256 : 0), 256, 0, st>>>(a, x_groups);
    return launch_status();
}

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" size_t qb_vocab_loss_workspace_nbytes(int64_t T, int64_t V, int64_t K, int backward)
{
    if (!shape_ok(T, V, K)) return 0;
    LossArgs a = {};
    a.T = (int)T;
    a.V = (int)V;
    a.K = (int)K;
    return lay_out(a, nullptr, backward != 0);
}

extern "C" qb_status qb_vocab_loss_fwd(const uint16_t *X, const uint16_t *W, const float *bias, const int64_t *targets,
                                       int64_t T, int64_t V, int64_t K, float *loss, float *lse, void *workspace, void *stream)
{
    if (!shape_ok(T, V, K)) return QB_ERR_SHAPE;
    if (!X || !W || !targets || !loss || !lse) return QB_ERR_NULL;
    if (!aligned16(X) || !aligned16(W) || (reinterpret_cast<uintptr_t>(targets) & 7)) return QB_ERR_VALUE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255)) return QB_ERR_WORKSPACE;
    LossArgs a = {};
    a.X = X; a.W = W; a.bias = bias; a.targets = targets;
    a.T = (int)T; a.V = (int)V; a.K = (int)K;
    a.loss = loss; a.lse = lse;
    lay_out(a, static_cast<uint8_t *>(workspace), false);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return few(T) ? forward<Small>(a, st) : forward<Large>(a, st);
}

extern "C" qb_status qb_vocab_loss_bwd(const float *dloss, const uint16_t *X, const uint16_t *W, const float *bias,
                                       const int64_t *targets, const float *lse, int64_t T, int64_t V, int64_t K,
                                       uint16_t *dX, uint16_t *dW, float *dbias, void *workspace, void *stream)
{
    if (!shape_ok(T, V, K)) return QB_ERR_SHAPE;
    if (!dloss || !X || !W || !targets || !lse || !dX || !dW) return QB_ERR_NULL;
    if (!aligned16(X) || !aligned16(W) || !aligned16(dX) || !aligned16(dW) || (reinterpret_cast<uintptr_t>(targets) & 7)) return QB_ERR_VALUE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255)) return QB_ERR_WORKSPACE;
    LossArgs a = {};
    a.X = X; a.W = W; a.bias = bias; a.targets = targets; a.dloss = dloss;
    a.T = (int)T; a.V = (int)V; a.K = (int)K;
    a.lse = const_cast<float *>(lse);
    a.dX = dX; a.dW = dW; a.dbias = dbias;
    lay_out(a, static_cast<uint8_t *>(workspace), true);
    if (!dbias) a.db = nullptr;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return few(T) ? backward<Small>(a, st) : backward<Large>(a, st);
}
