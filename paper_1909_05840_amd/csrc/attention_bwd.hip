// Attention of packed sequences, backward.
//
//   P = exp(S - lse);  dP = M (dO V^T);  delta = sum_k P dP;  dS = P (dP - delta)
//   dQ = scale dS K;  dK = scale dS^T Q;  dV = (P M)^T dO
//
// Two launches, each of which forms S and dP again: one goes over the keys of a tile of rows (dQ, delta), the other over the rows
// of a tile of keys (dK, dV; shared heads of keys sum over their queries there).  Seven products instead of the five
// that one launch would need, but nothing is added to memory by several workgroups: no atomics, the same bits every time.
// dS and P are rounded to the inputs' type for the last products only.
//
// float16 has normal numbers from 2^-14 on, and P is about 1 / keys, dS that times gradients of any size.  Both are rounded lifted by powers of two,
// which the binary32 results are taken back by: P 2^14 times, and dS that and a power for dP - delta besides, which keeps that at one or below.  dQ has such a
// power for every row, lowered when a block of keys has a larger |dP - delta| than those before, and the sums with it.  dK and dV sum over rows:
// theirs follows from |dP - delta| <= |dO| |V| / share + |delta|, norms over a row's values, with the largest of V among a wavefront's keys and the largest
// of dO and of delta that the launch for dQ leaves for the rows of the sequence and key head.  (A bound by the differences themselves would not do: where they
// vanish in the one launch, they are rounding errors in the other, which sums in another order.)  Unlifted, at 8192 keys and a spread of dO of
// 1e-4 dQ and dK were 11 times as far from exact as exact arithmetic rounded once; so 1.0 times, and 1.4 at a spread of 1e-2 and more.
#include "attention.hpp"
#include <algorithm>

namespace qb {
namespace {

constexpr int kKeys = 64, kRowsOfTile = 64;

struct GradArgs {
    const uint16_t *dO, *O;
    const float *lse;
    uint16_t *dQ, *dK, *dV;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    float *stat;  // [2][total_q * heads + 1]: -lse / scale (-infinity for a row that sees nothing, and for the last entry: P is zero), -delta
    float *part;  // [pairs][tiles of keys][splits][128][dK, dV] of tiles in parts
    v2f *most;    // float16: [pairs][tiles_q][4] of a wavefront's rows the largest squared norm of dO, the largest |delta|
    int tiles_q;  // tiles of 128 rows of a sequence of max_q (a longer one may have more, which there is no room for)
};

constexpr int kLift = 14;  // of P in float16, in powers of two: a weight that rounding has put a little above one, and any dS, stays below 65504

constexpr int kMostLift = 40;  // of dS besides, a row's before it has seen a key

template <int N>
__device__ __forceinline__ void clear(v16f (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) x[i][j] = 0.0f;
}
template <typename T>
__device__ __forceinline__ v8s rounded(const v16f &x, int half)
{
    v4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = T::pair(x[8 * half + 2 * i], x[8 * half + 2 * i + 1]);
    return __builtin_bit_cast(v8s, w);
}

template <typename T>
__device__ __forceinline__ float squares(v8s x)
{
    const v4u w = __builtin_bit_cast(v4u, x);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += T::lo(w[i]) * T::lo(w[i]) + T::hi(w[i]) * T::hi(w[i]);
    return sum;
}

// dQ and delta; 128 rows to a workgroup, 32 to a wavefront, a lane's results all of one row (as in the forward).
//
// delta = dO.O takes O as the forward rounded it, which moves dQ by -eps sum_k P K.  EXACT therefore sums eps = sum_k P (dP - delta)
// on the way, which is what delta lacks, and B = sum_k P K beside A = sum_k dS K: dQ = scale (A - eps B), and the second launch gets
// delta + eps.  Without it dQ is 1.5 to 1.6 times as far from exact as exact arithmetic rounded once at dim 64, whatever the number
// of keys (dS in 16 bits alone makes 1.41), and so at dim 128 with few; with many keys it is 1.43 to 1.49 times there, and tiles of rows that see
// more than kExactKeys are left to the other variant, which needs two thirds of the registers and three quarters of the products (whole backward, 8
// heads over 4000 keys: 344 us with it, 389 without; of 4 x 1024 the exact one's 114 us would be 104).  Bound as the forward is.  8192 causal keys, 16
// heads of 64: 288 us, 0.95 PFLOP/s of four products.
template <int D> constexpr int kExactKeys = D == 64 ? INT32_MAX : 1024;
template <typename T, int D, bool DROP, bool EXACT>
__global__ __launch_bounds__(256, D == 128 && EXACT ? 1 : 2) void attention_dq_kernel(const AttnArgs a, const GradArgs g, bool by_xcd)
{
    typedef Rows<D> R;
    constexpr int kTile = kKeys * R::kBytes, kStages = D == 64 ? 3 : 2, kCopies = 2 * kKeys / R::kPerCopy / 4;
    __shared__ __align__(1024) uint8_t lds[kStages][2 * kTile];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (EXACT && blockIdx.x == 0 && threadIdx.x < 2) g.stat[threadIdx.x ? 2 * (int64_t)a.total_q * a.heads + 1 : (int64_t)a.total_q * a.heads] = threadIdx.x ? 0.0f : -__builtin_inff();
    const Place at = place<false>(a, blockIdx.x, a.tiles, by_xcd, true, lane);
    if (at.none) return;
    const int kv = at.kv;
    const Segment &seg = at.seg;
    const int rows = seg.nq * a.group, first = at.tile * 128;
    if (first >= rows) return;
    const int row = first + wave * 32 + l32;
    const int token = min((unsigned)row / (unsigned)a.group, (unsigned)seg.nq - 1u);
    const int head = kv * a.group + (row - (int)((unsigned)row / (unsigned)a.group) * a.group);
    const int row_q = seg.q0 + token;
    const int64_t at_row = (int64_t)row_q * a.heads + head;

    v8s q[D / 16], dO[D / 16];
    const uint16_t *const q_from = a.Q + (int64_t)row_q * a.q_row + (int64_t)head * a.q_head + 8 * hf;
    const uint16_t *const do_from = g.dO + at_row * D + 8 * hf, *const o_from = g.O + at_row * D + 8 * hf;
    float delta = 0.0f, norm = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
        q[d] = *reinterpret_cast<const v8s *>(q_from + 16 * d);
        dO[d] = *reinterpret_cast<const v8s *>(do_from + 16 * d);
        const v4u x = __builtin_bit_cast(v4u, dO[d]), y = *reinterpret_cast<const v4u *>(o_from + 16 * d);
#pragma unroll
        for (int i = 0; i < 4; ++i) delta += T::lo(x[i]) * T::lo(y[i]) + T::hi(x[i]) * T::hi(y[i]);
        if constexpr (T::kNarrow) norm += squares<T>(dO[d]);
    }
    delta = halves_sum(delta);
    const float lse = g.lse[at_row];
    const float lse2 = lse == -__builtin_inff() ? __builtin_inff() : lse * 1.44269504088896341f - (T::kNarrow ? kLift : 0);

    const auto sees = [&](int t) { return a.causal ? min(seg.nk, max(0, seg.first_hidden(t))) : seg.nk; };
    const auto token_of = [&](int r) { return min(r / a.group, seg.nq - 1); };
    const int limit = sees(token);
    const int wave_least = __builtin_amdgcn_readfirstlane(sees(token_of(first + wave * 32)));
    const int wave_most = first + wave * 32 < rows ? __builtin_amdgcn_readfirstlane(sees(token_of(first + wave * 32 + 31))) : 0;  // (a wavefront without rows only copies)
    const int most = __builtin_amdgcn_readfirstlane(sees(token_of(first + 127)));
    if (EXACT != (most <= kExactKeys<D>)) return;
    const int tiles = (most + kKeys - 1) / kKeys;

    const uint16_t *const K = a.K + (int64_t)seg.k0 * a.k_row + (int64_t)kv * a.k_head;
    const uint16_t *const V = a.V + (int64_t)seg.k0 * a.v_row + (int64_t)kv * a.v_head;
    const uint32_t lds0 = lds_address(lds);
    const bool near = near_rows(a.k_row) && near_rows(a.v_row);
    const TileCopy<D, kKeys, 4> copy_k(wave, lane, [&](int r) { return (uint32_t)r * (uint32_t)a.k_row; }), copy_v(wave, lane, [&](int r) { return (uint32_t)r * (uint32_t)a.v_row; });
    const auto fetch = [&](int tile, int stage) {
        const uint32_t to = lds0 + stage * 2 * kTile;
        if (near && (tile + 1) * kKeys <= seg.nk) {
            copy_k.copy(K + (int64_t)tile * kKeys * a.k_row, to, wave);
            copy_v.copy(V + (int64_t)tile * kKeys * a.v_row, to + kTile, wave);
            return;
        }
        copy_rows<D, kKeys, 4>(to, wave, lane, [&](int r) { return K + (int64_t)min(tile * kKeys + r, seg.nk - 1) * a.k_row; });
        copy_rows<D, kKeys, 4>(to + kTile, wave, lane, [&](int r) { return V + (int64_t)min(tile * kKeys + r, seg.nk - 1) * a.v_row; });
    };
    const Threefry bits(DROP ? (uint64_t)*a.seed : 0);
    const Operands<D> op(lane, lds0);
    int lift = kMostLift;
    float lifted = __builtin_ldexpf(1.0f, kMostLift), lifted_delta = delta * lifted;
    v16f A[D / 32], B[EXACT ? D / 32 : 1];
    clear(A);
    clear(B);
    float eps = 0.0f;
    for (int t = 0; t < kStages - 1 && t < tiles; ++t) fetch(t, t);
    for (int t = 0, stage = 0; t < tiles; ++t, stage = stage == kStages - 1 ? 0 : stage + 1) {
        if (t + kStages - 1 <= tiles) wait_copies<(kStages - 2) * kCopies>();  // (the tiles behind this one may be under way)
        else wait_copies<0>();
        barrier();
        if (t + kStages - 1 < tiles) fetch(t + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
        if (t * kKeys >= wave_most) continue;
        const uint32_t tk = stage * 2 * kTile, tv = tk + kTile;
        const bool masked = (t + 1) * kKeys > wave_least;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            if (kb == 1 && t * kKeys + 32 >= wave_most) break;
            // (all operands are read in front of their products, those turned for the last one in front of the exponentials)
            v16f s, dp;
            {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.0f;
#pragma unroll
                for (int d0 = 0; d0 < D / 16; d0 += 4) {
                    v8s k[4], v[4];
#pragma unroll
                    for (int d = 0; d < 4; ++d) k[d] = op.along(tk, 32 * kb, d0 + d);
#pragma unroll
                    for (int d = 0; d < 4; ++d) v[d] = op.along(tv, 32 * kb, d0 + d);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        s = T::mma32(k[d], q[d0 + d], s);
                        dp = T::mma32(v[d], dO[d0 + d], dp);
                    }
                }
            }
            v8s turned[2][D / 32];
            const auto turn = [&](int h) {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) turned[h][i] = op.across(tk, 32 * kb + 16 * h, i);
            };
            if constexpr (D == 64) {
                turn(0);
                turn(1);
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = t * kKeys + 32 * kb + 8 * (i >> 2) + 4 * hf + (i & 3) < limit ? s[i] : -__builtin_inff();
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.c, -lse2));
            if constexpr (DROP) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const v2u w = weight_draws(bits, row_q, head, t * kKeys + 32 * kb + 2 * i + 4 * hf);
                    dp[i] = kept_low(w[0], a.threshold) ? dp[i] * a.inv_share : 0.0f;
                    dp[i + 1] = kept_high(w[0], a.threshold) ? dp[i + 1] * a.inv_share : 0.0f;
                    dp[i + 2] = kept_low(w[1], a.threshold) ? dp[i + 2] * a.inv_share : 0.0f;
                    dp[i + 3] = kept_high(w[1], a.threshold) ? dp[i + 3] * a.inv_share : 0.0f;
                }
            }
            if constexpr (T::kNarrow) {
                float top = 0.0f, other = 0.0f;  // (two chains)
#pragma unroll
                for (int i = 0; i < 16; ++i) dp[i] = __builtin_fmaf(dp[i], lifted, -lifted_delta);
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    top = max3(top, __builtin_fabsf(dp[i]), __builtin_fabsf(dp[i + 1]));
                    other = max3(other, __builtin_fabsf(dp[i + 2]), __builtin_fabsf(dp[i + 3]));
                }
                top = fmaxf(top, other);
                if (__builtin_amdgcn_ballot_w64(top > 1.0f)) {
                    top = halves_max(top);
                    const int down = top > 1.0f && top < __builtin_inff() ? __builtin_amdgcn_frexp_expf(top) + 2 : 0;  // (two powers of two to spare)
                    const float f = __builtin_ldexpf(1.0f, -down);
                    lift -= down;
                    lifted *= f;
                    lifted_delta *= f;
                    eps *= f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) dp[i] *= f;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i)
#pragma unroll
                        for (int j = 0; j < 16; ++j) A[i][j] *= f;
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                dp[i] = s[i] * (T::kNarrow ? dp[i] : dp[i] - delta);
                if constexpr (EXACT) eps += dp[i];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (D != 64) turn(h);
                const v8s ds = rounded<T>(dp, h);
                v8s p;
                if constexpr (EXACT) p = rounded<T>(s, h);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    A[i] = T::mma32(turned[h][i], ds, A[i]);
                    if constexpr (EXACT) B[i] = T::mma32(turned[h][i], p, B[i]);
                }
            }
        }
    }
    if constexpr (EXACT) {
        eps = halves_sum(eps);
        if constexpr (T::kNarrow) eps = __builtin_ldexpf(eps, -kLift);  // (B is as P is)
        delta += T::kNarrow ? __builtin_ldexpf(eps, -lift) : eps;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) A[i][j] -= eps * B[i][j];
    }
    if constexpr (T::kNarrow) {  // (rows that see no key have no gradient; one with infinities or NaN gives those whatever it is multiplied by)
        const float squared = halves_sum(norm);
        const bool counts = limit > 0 && squared < __builtin_inff() && __builtin_fabsf(delta) < __builtin_inff();
        const v2f most = {wave_max(counts ? squared : 0.0f), wave_max(counts ? __builtin_fabsf(delta) : 0.0f)};
        if (lane == 0 && at.tile < g.tiles_q) g.most[(((int64_t)at.seq * a.kv_heads + kv) * g.tiles_q + at.tile) * 4 + wave] = most;
    }
    write_row<T, D>(g.dQ + (int64_t)row_q * g.q_row + (int64_t)head * g.q_head, A, T::kNarrow ? __builtin_ldexpf(a.scale, -kLift - lift) : a.scale, hf, row < rows);
    if (row >= rows) return;
    if (hf == 0) {
        g.stat[at_row] = lse == -__builtin_inff() ? -__builtin_inff() : -lse / a.scale;
        g.stat[(int64_t)a.total_q * a.heads + 1 + at_row] = -delta;
    }
}

__device__ __forceinline__ void copy4(const void *from, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(lds) : "memory", "m0");
}
// word of lane B of every four, as a constant of the instruction
template <int B>
__device__ __forceinline__ uint32_t of_four(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, B * 0x55, 0xF, 0xF, true); }

// For dK and dV the rows of a key head are dealt to tiles of 64: `heads` of the group's heads of each of `tokens` tokens, so that a row's
// place in its tile tells its token and head without a division.  Rows of a tile that are none (three heads: the last of 64) have
// P = 0.  `chunks`: tiles to a group of more than 64.
struct RowTiling {
    int heads, tokens, chunks;
};
inline RowTiling row_tiling(int group)
{
    const int heads = group < kRowsOfTile ? group : kRowsOfTile;
    return {heads, kRowsOfTile / heads, (group + heads - 1) / heads};
}
// The tiles that a tile of 128 keys is seen by are cut into parts of `most` tiles, from the last row on (with causal masks the first keys
// are seen by many more rows than the last, but all by the last rows): part p of every tile of keys is the same rows, and the
// workgroups that are at work together, which take the parts in turn, find them in their L2.  There are at most `splits` parts, for which the
// workspace has room, however long the sequence is.
struct RowTiles {
    int begin, end, parts;
};
__host__ __device__ __forceinline__ RowTiles row_tiles(bool causal, const RowTiling &r, int nq, int nk, int first_key, int part, int most, int splits)
{
    const int token = causal ? min(nq, max(0, first_key - (nk - nq))) : 0;  // causal: key <= token + nk - nq
    const int all = (nq + r.tokens - 1) / r.tokens, first = token < nq ? token / r.tokens : all;
    const int n = (all - first) * r.chunks, end = all * r.chunks - part * most;
    return {max(first * r.chunks, end - most), end, max(1, min(splits, (n + most - 1) / most))};
}

// dK and dV; 128 keys to a workgroup, 32 to a wavefront: a lane's results all of one key.  Where tiles of keys are few, a workgroup does
// a part of the rows, and its binary32 sums go to the workspace for a third launch to join.  Scores are taken as S = Q K^T, so that a
// lane holds sixteen rows of its key and P and dS are, as they lie, the operands of dV^T = dO^T P and dK^T = Q^T dS.  8192 causal keys, 16 heads
// and 4 key heads of 64: 340 us and 11 to join the parts, 0.78 PFLOP/s of four products; a block of 32 x 32 takes about 1000 cycles of a SIMD, of
// which its products are 512 and its vector instructions 490: one after the other (counters of a run).  32 sequences of up to 384 with dropout: 43 us.
template <typename T, int D, bool DROP>
__global__ __launch_bounds__(256, 2) void attention_dkv_kernel(const AttnArgs a, const GradArgs g, const RowTiling tiling, int splits, int most, bool by_xcd)
{
    typedef Rows<D> R;
    constexpr int kTile = kRowsOfTile * R::kBytes, kStage = 2 * kTile + 2 * kRowsOfTile * 4, kStages = 3;
    __shared__ __align__(1024) uint8_t lds[kStages][kStage];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place<true>(a, blockIdx.x, a.tiles * splits, by_xcd, splits == 1, lane);
    if (at.none) return;
    const int kv = at.kv;
    const Segment &seg = at.seg;
    const int part = splits == 1 ? 0 : at.tile / a.tiles, key_tile = at.tile - part * a.tiles;  // part after part
    const int first = key_tile * 128;
    if (first >= seg.nk) return;
    const RowTiles todo = row_tiles(a.causal, tiling, seg.nq, seg.nk, first, part, most, splits);
    if (part >= todo.parts) return;
    const int begin = __builtin_amdgcn_readfirstlane(todo.begin), end = __builtin_amdgcn_readfirstlane(todo.end);
    const int key = first + wave * 32 + l32, key_in = min(key, seg.nk - 1);

    v8s k[D / 16], v[D / 16];
    const uint16_t *const k_from = a.K + (int64_t)(seg.k0 + key_in) * a.k_row + (int64_t)kv * a.k_head + 8 * hf;
    const uint16_t *const v_from = a.V + (int64_t)(seg.k0 + key_in) * a.v_row + (int64_t)kv * a.v_head + 8 * hf;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
        k[d] = *reinterpret_cast<const v8s *>(k_from + 16 * d);
        v[d] = *reinterpret_cast<const v8s *>(v_from + 16 * d);
    }
    // causal: the key is seen from this token on; the wavefront's last key from wave_token on
    const int from_token = a.causal ? key - (seg.nk - seg.nq) : INT32_MIN / 128;
    const int wave_token = __builtin_amdgcn_readfirstlane(a.causal ? first + wave * 32 + 31 - (seg.nk - seg.nq) : INT32_MIN / 128);

    const uint32_t lds0 = lds_address(lds);
    const int64_t stats = (int64_t)a.total_q * a.heads;
    const int head0 = kv * a.group, last_token = seg.nq - 1;
    const bool near = near_rows(a.q_row) && near_rows(a.q_head) && (int64_t)a.heads * D < (1 << 23);
    const auto token_in = [&](int r) { return r / tiling.heads; };
    const auto head_in = [&](int r) { return r - r / tiling.heads * tiling.heads; };
    const TileCopy<D, kRowsOfTile, 4> copy_q(wave, lane, [&](int r) { return (uint32_t)token_in(r) * (uint32_t)a.q_row + (uint32_t)head_in(r) * (uint32_t)a.q_head; }),
        copy_d(wave, lane, [&](int r) { return (uint32_t)(token_in(r) * a.heads + head_in(r)) * D; });
    const int stat_token = token_in(lane), stat_head = head_in(lane);  // of row `lane` of a tile
    const auto place_of = [&](int tile, int &token, int &head) __attribute__((always_inline)) {       // first token and head of a tile
        const int block = tiling.chunks == 1 ? tile : __builtin_amdgcn_readfirstlane(tile / tiling.chunks);
        token = block * tiling.tokens;
        head = (tile - block * tiling.chunks) * tiling.heads;
    };
    const auto fetch = [&](int tile, int stage) __attribute__((always_inline)) {
        const uint32_t to = lds0 + stage * kStage;
        int token, head;
        place_of(tile, token, head);
        if (near && token + kRowsOfTile / tiling.heads < seg.nq && head + tiling.heads <= a.group) {  // (a row that is none lies one token on)
            const int64_t at = seg.q0 + token, at_row = at * a.heads + head0 + head;
            copy_q.copy(a.Q + at * a.q_row + (int64_t)(head0 + head) * a.q_head, to, wave);
            copy_d.copy(g.dO + at_row * D, to + kTile, wave);
        } else {
            const auto row_of = [&](int r, int64_t &t, int64_t &h) {
                t = seg.q0 + min(token + token_in(r), last_token);
                h = head0 + min(head + head_in(r), a.group - 1);
            };
            copy_rows<D, kRowsOfTile, 4>(to, wave, lane, [&](int r) {
                int64_t t, h;
                row_of(r, t, h);
                return a.Q + t * a.q_row + h * a.q_head;
            });
            copy_rows<D, kRowsOfTile, 4>(to + kTile, wave, lane, [&](int r) {
                int64_t t, h;
                row_of(r, t, h);
                return g.dO + (t * a.heads + h) * D;
            });
        }
        if (wave < 2) {  // a row that is none takes the entry behind the last: P = 0
            const bool row = stat_token < tiling.tokens && token + stat_token <= last_token && head + stat_head < a.group;
            const int64_t at = row ? (int64_t)(seg.q0 + token + stat_token) * a.heads + head0 + head + stat_head : stats;
            copy4(g.stat + wave * (stats + 1) + at, to + 2 * kTile + wave * kRowsOfTile * 4);
        }
    };
    const Threefry bits(DROP ? (uint64_t)*a.seed : 0);
    int lift = 0;
    float lifted = 1.0f;
    v16f dK[D / 32], dV[D / 32];
    clear(dK);
    clear(dV);
    const Operands<D> op(lane, lds0);
    typedef const __attribute__((address_space(3))) v4f *lds_v4f;
    const uint32_t stat_at = lds0 + 2 * kTile + 16 * hf;

    // A block of 32 rows goes through three steps: its operands are read; scores and dP are formed; P, dS and their products.  The
    // second step of a block runs next to the exponentials of the block before it, the first next to that one's products: the matrix
    // cores work on the one while the vector units and the LDS work on the other.  (sched_barrier: the compiler keeps to the order
    // written here.)  The stage is a constant of the code, and with it every place in LDS.
    // The sums start from -lse / scale and -delta, as they lie in LDS: exp(S - lse) and dP - delta take a multiplication each.
    const auto start = [&](uint32_t tq, int rb, v16f &p, v16f &ds) __attribute__((always_inline)) {
        const uint32_t stat = stat_at + tq + 4 * (32 * rb);
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const v4f x = *(lds_v4f)(stat + 8 * i);
            v4f y = {0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (!DROP) y = *(lds_v4f)(stat + 4 * kRowsOfTile + 8 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[i + j] = x[j];
                ds[i + j] = y[j];
            }
        }
    };
    constexpr int kAhead = 2;  // operands that are read ahead of their products
    const auto read = [&](uint32_t tq, int rb, int d, v8s &x, v8s &y) __attribute__((always_inline)) {
        x = op.along(tq, 32 * rb, d);
        y = op.along(tq + kTile, 32 * rb, d);
    };
    const auto turn = [&](uint32_t tq, int rb, int h, v8s (&x)[D / 32], v8s (&y)[D / 32]) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            x[i] = op.across(tq + kTile, 32 * rb + 16 * h, i);
            y[i] = op.across(tq, 32 * rb + 16 * h, i);
        }
    };
    const auto hide = [&](int rb, int token, v16f &p) __attribute__((always_inline)) {
        const int from = (from_token - token) * tiling.heads - 32 * rb - 4 * hf;  // (row r's token is at or behind x if r >= x * heads)
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = 8 * (i >> 2) + (i & 3) >= from ? p[i] : -__builtin_inff();
    };
    // rows 8 * q + 4 * hf .. + 3 of a block: P and dS
    v2u bits_of[4];
    const auto draw = [&](int rb, int token, int head) __attribute__((always_inline)) {
        // Four neighbouring lanes need the four draws of the same counters: each of them forms the counters of every fourth row,
        // and they take each other's words.
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 32 * rb + 8 * i + 4 * hf + (lane & 3);
            bits_of[i] = weight_draws(bits, seg.q0 + token + token_in(r), head0 + head + head_in(r), key);
        }
    };
    const auto weights = [&](uint32_t tq, int rb, auto quarter, v16f &p, v16f &ds) __attribute__((always_inline)) {
        constexpr int q4 = decltype(quarter)::value, i0 = 4 * q4;
#pragma unroll
        for (int j = 0; j < 4; ++j) p[i0 + j] = __builtin_amdgcn_exp2f(T::kNarrow ? __builtin_fmaf(p[i0 + j], a.c, (float)kLift) : p[i0 + j] * a.c);
        if constexpr (!DROP) {
#pragma unroll
            for (int j = 0; j < 4; ++j) ds[i0 + j] *= T::kNarrow ? p[i0 + j] * lifted : p[i0 + j];
        } else {
            const v4f minus_delta = *(lds_v4f)(stat_at + tq + 4 * (kRowsOfTile + 32 * rb + 8 * q4));
            const auto take = [&](int j, uint32_t w0, uint32_t w1) {
                const uint32_t word = (lane & 2) ? w1 : w0;
                const bool in = ((lane & 1) ? word >> 16 : word & 0xFFFFu) >= a.threshold;
                ds[i0 + j] = (T::kNarrow ? p[i0 + j] * lifted : p[i0 + j]) * ((in ? ds[i0 + j] * a.inv_share : 0.0f) + minus_delta[j]);
                p[i0 + j] = in ? p[i0 + j] : 0.0f;
            };
            const v2u w = bits_of[q4];
            take(0, of_four<0>(w[0]), of_four<0>(w[1]));
            take(1, of_four<1>(w[0]), of_four<1>(w[1]));
            take(2, of_four<2>(w[0]), of_four<2>(w[1]));
            take(3, of_four<3>(w[0]), of_four<3>(w[1]));
        }
    };
    v16f p[2], ds[2];
    v8s x[kAhead], y[kAhead], tx[D / 32], ty[D / 32];
    int t = begin, token, head;
    // block rb of the tile at tq, whose scores are in p[rb] and ds[rb], next to the scores of the other block, whose operands are in x and y
    const auto exponentials = [&](uint32_t tq, auto block, uint32_t tn) __attribute__((always_inline)) {
        constexpr int rb = decltype(block)::value;
        int hidden = wave_token;
        asm volatile("" : "+s"(hidden));  // (or the compiler makes two copies of all that follows, for the tiles with and those without)
        if (token < hidden) hide(rb, token, p[rb]);
        if constexpr (DROP) draw(rb, token, head);
        __builtin_amdgcn_sched_barrier(0);
        each<D / 16>([&](auto number) __attribute__((always_inline)) {
            constexpr int d = decltype(number)::value;
            p[1 - rb] = T::mma32(x[d % kAhead], k[d], p[1 - rb]);
            ds[1 - rb] = T::mma32(y[d % kAhead], v[d], ds[1 - rb]);
            if constexpr (d + kAhead < D / 16) read(tn, 1 - rb, d + kAhead, x[d % kAhead], y[d % kAhead]);
            if constexpr (d % (D / 64) == 0) weights(tq, rb, std::integral_constant<int, d / (D / 64)>{}, p[rb], ds[rb]);
            if constexpr (d == D / 16 - 1) turn(tq, rb, 0, tx, ty);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // its products; meanwhile the operands of block rn of the tile at tn are read
    const auto products = [&](uint32_t tq, auto block, uint32_t tn, const auto &in_between) __attribute__((always_inline)) {
        constexpr int rb = decltype(block)::value;
        v8s pr[2] = {rounded<T>(p[rb], 0), rounded<T>(p[rb], 1)}, dr[2] = {rounded<T>(ds[rb], 0), rounded<T>(ds[rb], 1)};
        asm volatile("" : "+v"(pr[0]), "+v"(pr[1]), "+v"(dr[0]), "+v"(dr[1]));  // (formed here, and not moved behind the branch below)
        in_between();
        __builtin_amdgcn_sched_barrier(0);
        start(tn, rb, p[rb], ds[rb]);
#pragma unroll
        for (int d = 0; d < kAhead; ++d) read(tn, rb, d, x[d], y[d]);
        each<2>([&](auto half) __attribute__((always_inline)) {
            constexpr int h = decltype(half)::value;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                dV[i] = T::mma32(tx[i], pr[h], dV[i]);
                dK[i] = T::mma32(ty[i], dr[h], dK[i]);
            }
            if constexpr (h == 0) turn(tq, rb, 1, tx, ty);
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    place_of(t, token, head);
    if (begin < end) {
        fetch(begin, 0);
        if constexpr (T::kNarrow) {
            const v2f *const from = g.most + ((int64_t)at.seq * a.kv_heads + kv) * g.tiles_q * 4;
            v2f most = {0.0f, 0.0f};
            for (int i = lane, n = min(g.tiles_q, (seg.nq * a.group + 127) >> 7) * 4; i < n; i += 64) most = v2f{fmaxf(most[0], from[i][0]), fmaxf(most[1], from[i][1])};
            float norm = 0.0f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) norm += squares<T>(v[d]);
            norm = halves_sum(norm);
            norm = wave_max(norm < __builtin_inff() ? norm : 0.0f);
            const float bound = __builtin_sqrtf(wave_max(most[0])) * __builtin_sqrtf(norm) * (DROP ? a.inv_share : 1.0f) + wave_max(most[1]);
            if (bound > 0.0f) lift = __builtin_amdgcn_readfirstlane(-__builtin_amdgcn_frexp_expf(bound));
            lifted = __builtin_ldexpf(1.0f, lift);
        }
        if (begin + 1 < end) {
            fetch(begin + 1, 1);
            wait_copies<2 * decltype(copy_q)::N>();  // (the first tile's; the second's may be under way)
        } else {
            wait_copies<0>();
        }
        barrier();
        start(0, 0, p[0], ds[0]);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            read(0, 0, d, x[0], y[0]);
            p[0] = T::mma32(x[0], k[d], p[0]);
            ds[0] = T::mma32(y[0], v[d], ds[0]);
        }
        start(0, 1, p[1], ds[1]);
#pragma unroll
        for (int d = 0; d < kAhead; ++d) read(0, 1, d, x[d], y[d]);
    }
    const auto turn_over = [&](int next) __attribute__((always_inline)) {
        wait_copies<0>();
        barrier();  // the next tile has come, and everyone is done with the last one
        if (t + 2 < end) fetch(t + 2, next == kStages - 1 ? 0 : next + 1);
    };
    int stage = 0;
    if (first + wave * 32 >= seg.nk) {  // a wavefront without keys only copies
        for (; t < end; ++t) {
            stage = stage == kStages - 1 ? 0 : stage + 1;
            turn_over(stage);
        }
        return;
    }
    while (t < end) {
        const int next = stage == kStages - 1 ? 0 : stage + 1;
        const uint32_t tq = stage * kStage, tn = next * kStage;
        const std::integral_constant<int, 0> upper;
        const std::integral_constant<int, 1> lower;
        exponentials(tq, upper, tq);
        products(tq, upper, tn, [&]() __attribute__((always_inline)) { turn_over(next); });
        exponentials(tq, lower, tn);
        products(tq, lower, tn, []() {});  // (past the last tile: scores of what lies there, unused)
        place_of(++t, token, head);
        stage = next;
    }
    if constexpr (T::kNarrow) {
        const float of_k = __builtin_ldexpf(1.0f, -kLift - lift), of_v = __builtin_ldexpf(1.0f, -kLift);
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                dK[i][j] *= of_k;
                dV[i][j] *= of_v;
            }
    }
    if (todo.parts > 1) {
        if (key >= seg.nk) return;
        float *const to = g.part + ((int64_t)((at.pair * (int64_t)a.tiles + key_tile) * splits + part) * 128 + key - first) * (2 * D);
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                *reinterpret_cast<v4f *>(to + 32 * i + 2 * j + 4 * hf) = v4f{dK[i][j], dK[i][j + 1], dK[i][j + 2], dK[i][j + 3]};
                *reinterpret_cast<v4f *>(to + D + 32 * i + 2 * j + 4 * hf) = v4f{dV[i][j], dV[i][j + 1], dV[i][j + 2], dV[i][j + 3]};
            }
        return;
    }
    write_row<T, D>(g.dK + (int64_t)(seg.k0 + key) * g.k_row + (int64_t)kv * g.k_head, dK, a.scale, hf, key < seg.nk);
    write_row<T, D>(g.dV + (int64_t)(seg.k0 + key) * g.v_row + (int64_t)kv * g.v_head, dV, DROP ? a.inv_share : 1.0f, hf, key < seg.nk);
}

// dK and dV of 16 keys from their parts; a thread does eight neighbouring values
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_dkv_join_kernel(const AttnArgs a, const GradArgs g, const RowTiling tiling, int splits, int most, float inv_share)
{
    constexpr int kEach = 2 * D / 8;  // threads to a key
    const int pair = blockIdx.x / (a.tiles * (128 * kEach / 256)), in_pair = blockIdx.x - pair * (a.tiles * (128 * kEach / 256));
    const int id = in_pair * 256 + threadIdx.x, key = id / kEach, d = (id - key * kEach) * 8;
    const int b = pair / a.kv_heads, kv = pair - b * a.kv_heads;
    const Segment seg = segment(a, b);
    if (key >= seg.nk) return;
    const int tile = key / 128;
    const float *const from = g.part + ((int64_t)(pair * (int64_t)a.tiles + tile) * splits * 128 + key % 128) * (2 * D) + d;
    v4f x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    const int parts = row_tiles(a.causal, tiling, seg.nq, seg.nk, tile * 128, 0, most, splits).parts;
    if (parts == 1) return;  // (written whole)
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
        const v4f *const q = reinterpret_cast<const v4f *>(from + (int64_t)p * 128 * (2 * D));
        x[0] += q[0];
        x[1] += q[1];
    }
    const float f = d < D ? a.scale : inv_share;
    uint16_t *const to = d < D ? g.dK + (int64_t)(seg.k0 + key) * g.k_row + (int64_t)kv * g.k_head + d : g.dV + (int64_t)(seg.k0 + key) * g.v_row + (int64_t)kv * g.v_head + d - D;
    *reinterpret_cast<v4u *>(to) = v4u{T::pair(x[0][0] * f, x[0][1] * f), T::pair(x[0][2] * f, x[0][3] * f), T::pair(x[1][0] * f, x[1][1] * f), T::pair(x[1][2] * f, x[1][3] * f)};
}

// How many tiles of rows a part has at most: such that the parts come to about as many workgroups as this, but eight or more; and the
// most parts of a tile of keys.  Parts even out what tiles of keys have to do, and fill the CUs (two workgroups to each) where tiles are few:
// 8192 causal keys, 4 key heads of 64, whole backward: unsplit 842 us, for 256 workgroups 705, 512 668, 768 614, 1536 614.  But each part's sums are
// written and read again, 4 * 128 * 2 * dim bytes: 8 heads of 128 over 4000 keys 244 us unsplit and for 256, for 512 274, 768 287; 2 x 4000 causal, 4 key heads
// of 128: 719 unsplit, 576 for 256, 645 for 512.
inline int64_t parts_wanted(int dim) { return dim == 64 ? 768 : 256; }
struct Parts {
    int64_t most, splits;
};
inline Parts row_parts(int64_t pairs, int64_t max_q, int64_t group, int64_t max_k, bool causal, int dim)
{
    const RowTiling t = row_tiling((int)group);
    const int64_t tiles = pairs * ((max_k + 127) / 128), rows = (max_q + t.tokens - 1) / t.tokens * t.chunks, wanted = parts_wanted(dim);
    if (tiles > INT32_MAX / 256) return {rows, 1};  // (more than a launch takes: refused)
    const int64_t most = std::max<int64_t>(8, (tiles * rows / (causal ? 2 : 1) + wanted - 1) / wanted);
    return {most, std::max<int64_t>(1, (rows + most - 1) / most)};
}
inline size_t stat_bytes(const qb_attention *p) { return ((size_t)(p->total_q * p->heads + 1) * 8 + 255) / 256 * 256; }
inline size_t most_bytes(const qb_attention *p)  // (four wavefronts to a tile)
{
    const int64_t tiles = (p->max_q * (p->heads / p->kv_heads) + 127) / 128;
    return p->type == QB_TYPE_FP16 ? ((size_t)((int64_t)p->n_seqs * p->kv_heads * tiles) * 32 + 255) / 256 * 256 : 0;
}

template <typename T, int D>
qb_status backward(AttnArgs a, const GradArgs &g, int64_t max_q, int64_t max_k, bool drop, hipStream_t stream)
{
    const int64_t pairs = (int64_t)a.n_seqs * a.kv_heads;
    const bool by_xcd = deal_by_xcd(pairs);
    if (max_q > 0) {
        a.tiles = (int)((max_q * a.group + 127) / 128);
        const int64_t grid = dealt_workgroups(pairs, a.tiles);
        if (grid > INT32_MAX / 256) return QB_ERR_SHAPE;
        if (drop) attention_dq_kernel<T, D, true, true><<<(int)grid, 256, 0, stream>>>(a, g, by_xcd);
        else attention_dq_kernel<T, D, false, true><<<(int)grid, 256, 0, stream>>>(a, g, by_xcd);
        if constexpr (D == 128) if (max_k > kExactKeys<D>) {
            if (drop) attention_dq_kernel<T, D, true, false><<<(int)grid, 256, 0, stream>>>(a, g, by_xcd);
            else attention_dq_kernel<T, D, false, false><<<(int)grid, 256, 0, stream>>>(a, g, by_xcd);
        }
    }
    if (max_k > 0) {
        a.tiles = (int)((max_k + 127) / 128);
        const Parts parts = row_parts(pairs, max_q, a.group, max_k, a.causal, D);
        const int splits = (int)parts.splits, most = (int)parts.most;
        const int64_t grid = dealt_workgroups(pairs, (int64_t)a.tiles * splits);
        if (drop) attention_dkv_kernel<T, D, true><<<(int)grid, 256, 0, stream>>>(a, g, row_tiling(a.group), splits, most, by_xcd);
        else attention_dkv_kernel<T, D, false><<<(int)grid, 256, 0, stream>>>(a, g, row_tiling(a.group), splits, most, by_xcd);
        if (splits > 1) attention_dkv_join_kernel<T, D><<<(int)(pairs * a.tiles * (128 * 2 * D / 8 / 256)), 256, 0, stream>>>(a, g, row_tiling(a.group), splits, most, drop ? a.inv_share : 1.0f);
    }
    return launch_status();
}

}  // namespace

// Parts that the dK and dV of a tile of keys are written in, for a sequence of nq queries and nk keys in a call of these sizes; `reserved`:
// the parts that its workspace has room for.
int attention_row_parts(int64_t pairs, int64_t group, int64_t max_q, int64_t max_k, bool causal, int dim, int nq, int nk, int first_key, int *reserved)
{
    const Parts p = row_parts(pairs, max_q, group, max_k, causal, dim);
    *reserved = (int)p.splits;
    return row_tiles(causal, row_tiling((int)group), nq, nk, first_key, 0, (int)p.most, (int)p.splits).parts;
}

}  // namespace qb

using namespace qb;

extern "C" size_t qb_attention_bwd_workspace_nbytes(const qb_attention *p)
{
    AttnArgs a;
    if (attention_args(p, a) != QB_OK) return 0;
    const int64_t pairs = (int64_t)a.n_seqs * a.kv_heads, splits = row_parts(pairs, p->max_q, a.group, p->max_k, p->causal, p->dim).splits;
    return stat_bytes(p) + most_bytes(p) + (splits > 1 ? (size_t)(pairs * ((p->max_k + 127) / 128) * splits) * 128 * 2 * p->dim * 4 : 0);
}

extern "C" qb_status qb_attention_bwd(const qb_attention *p, const void *dO, const void *O, const float *lse,
                                      const qb_attention_grads *grads, void *workspace, void *stream)
{
    AttnArgs a;
    const qb_status s = attention_args(p, a);
    if (s != QB_OK) return s;
    if (!grads) return QB_ERR_NULL;
    if (p->k_len || (grads->q_row | grads->q_head | grads->k_row | grads->k_head | grads->v_row | grads->v_head) % 8 != 0) return QB_ERR_VALUE;
    if (p->n_seqs == 0 || (p->total_q == 0 && p->total_k == 0)) return QB_OK;
    if (p->total_q > 0 && (!dO || !O || !lse || !grads->dQ)) return QB_ERR_NULL;
    if (p->total_k > 0 && (!grads->dK || !grads->dV)) return QB_ERR_NULL;
    if (!aligned16(dO) || !aligned16(O) || !aligned16(grads->dQ) || !aligned16(grads->dK) || !aligned16(grads->dV)) return QB_ERR_VALUE;
    if ((p->total_q > 0 || p->max_q > 0) && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255))) return QB_ERR_WORKSPACE;
    const int64_t pairs = (int64_t)p->n_seqs * p->kv_heads;
    if (dealt_workgroups(pairs, (p->max_q * a.group + 127) / 128) > INT32_MAX / 256 || dealt_workgroups(pairs, (p->max_k + 127) / 128 * row_parts(pairs, p->max_q, a.group, p->max_k, p->causal, p->dim).splits) > INT32_MAX / 256) return QB_ERR_SHAPE;
    uint8_t *const ws = static_cast<uint8_t *>(workspace);
    const GradArgs g = {static_cast<const uint16_t *>(dO), static_cast<const uint16_t *>(O), lse, static_cast<uint16_t *>(grads->dQ), static_cast<uint16_t *>(grads->dK),
                        static_cast<uint16_t *>(grads->dV), grads->q_row, grads->q_head, grads->k_row, grads->k_head, grads->v_row, grads->v_head, reinterpret_cast<float *>(ws),
                        reinterpret_cast<float *>(ws + stat_bytes(p) + most_bytes(p)), reinterpret_cast<v2f *>(ws + stat_bytes(p)), (int)((p->max_q * a.group + 127) / 128)};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool drop = p->p > 0.0f;
    if (p->type == QB_TYPE_BF16) return p->dim == 64 ? backward<Bf16, 64>(a, g, p->max_q, p->max_k, drop, st) : backward<Bf16, 128>(a, g, p->max_q, p->max_k, drop, st);
    return p->dim == 64 ? backward<Fp16, 64>(a, g, p->max_q, p->max_k, drop, st) : backward<Fp16, 128>(a, g, p->max_q, p->max_k, drop, st);
}
