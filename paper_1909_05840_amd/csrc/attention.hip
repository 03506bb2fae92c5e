// Attention of packed sequences, forward.
//
//   S = scale q.k;  m = max S, l = sum exp(S - m) over the keys that are seen;  O = sum exp(S - m) M V / l;  lse = m + log l
//
// One pass over the keys with a running maximum and sum (binary32).  Scores are taken transposed, S^T = K Q^T: a lane of the
// 32 x 32 product holds sixteen keys of ONE query, so that maximum and sum are taken inside a lane, and its exponentials are, as
// they lie, the operand of O^T = V^T P^T, whose contraction may run over the keys in any order; V's operand is turned by the
// transposing LDS reads in the same order.  Exponentials are rounded to the inputs' type for that product only: l sums
// them unrounded.
#include "attention.hpp"
#include <algorithm>

namespace qb {

// scale: lse / scale, which the backward's sums start from, and kNothing * scale, which a row's exponentials start from, have to be finite
qb_status attention_args(const qb_attention *p, AttnArgs &a)
{
    if (!p) return QB_ERR_NULL;
    if (p->total_q < 0 || p->total_k < 0 || p->total_q > INT32_MAX - 4096 || p->total_k > INT32_MAX - 4096 || p->n_seqs < 0 || p->heads <= 0 ||
        p->kv_heads <= 0 || p->heads % p->kv_heads != 0 || p->heads > (1 << 16) || (p->dim != 64 && p->dim != 128) || p->max_q < 0 || p->max_k < 0 ||
        p->max_q > INT32_MAX || p->max_k > INT32_MAX - 4096 || p->max_q * (p->heads / p->kv_heads) >= (1 << 30) ||
        (int64_t)p->n_seqs * p->kv_heads > INT32_MAX)
        return QB_ERR_SHAPE;
    if ((p->type != QB_TYPE_BF16 && p->type != QB_TYPE_FP16) || !(p->scale >= 1e-36f && p->scale <= 2e8f) || !(p->p >= 0.0f && p->p < 1.0f) ||
        (p->q_row | p->q_head | p->k_row | p->k_head | p->v_row | p->v_head) % 8 != 0)
        return QB_ERR_VALUE;
    if (p->p > 0.0f) {
        if (p->heads > 512 || p->max_k > (1 << 24)) return QB_ERR_SHAPE;
        if (!p->seed) return QB_ERR_NULL;
    }
    if (!aligned16(p->Q) || !aligned16(p->K) || !aligned16(p->V)) return QB_ERR_VALUE;
    if (p->total_q > 0 && p->n_seqs > 0 && (!p->Q || !p->cu_q || !p->cu_k)) return QB_ERR_NULL;
    if (p->total_k > 0 && p->n_seqs > 0 && (!p->K || !p->V || !p->cu_q || !p->cu_k)) return QB_ERR_NULL;
    a.Q = static_cast<const uint16_t *>(p->Q);
    a.K = static_cast<const uint16_t *>(p->K);
    a.V = static_cast<const uint16_t *>(p->V);
    a.q_row = p->q_row; a.q_head = p->q_head;
    a.k_row = p->k_row; a.k_head = p->k_head;
    a.v_row = p->v_row; a.v_head = p->v_head;
    a.heads = p->heads;
    a.kv_heads = p->kv_heads;
    a.group = p->heads / p->kv_heads;
    a.total_q = (int)p->total_q;
    a.total_k = (int)p->total_k;
    a.n_seqs = p->n_seqs;
    a.causal = p->causal;
    a.cu_q = p->cu_q;
    a.cu_k = p->cu_k;
    a.k_len = p->k_len;
    a.tiles = 0;
    a.scale = p->scale;
    a.c = (float)(p->scale * 1.4426950408889634);
    a.seed = p->seed;
    a.threshold = drop_threshold(p->p);
    a.inv_share = (float)(65536.0 / (65536 - a.threshold));
    return QB_OK;
}

namespace {

// A running softmax of 32 rows over the keys, a wavefront's: m and l per lane's row (l of the half's own keys), O^T.
constexpr float kNothing = -1.0e30f;  // m before a row has seen a key (finite: -infinity less itself is no number)
// The accumulators are rescaled only when a maximum has grown by more than this (powers of two): until then the
// exponentials stay below 2^8, which costs no precision in either type.
constexpr float kLazy = 8.0f;
// In float16 exponentials, and with them l and O's sums, are held 2^7 times as large (so below 2^15): its normal numbers end at 2^-14, and keys
// of less weight count where those of more have little value.  A first key of 2^20 times the others' weight and no value had O 9 to 11 times
// as far from exact as exact arithmetic rounded once.
template <typename T> constexpr float kLift = T::kNarrow ? 7.0f : 0.0f;
template <typename T>
__device__ __forceinline__ float lse_of(float m, float l, float scale) { return l == 0.0f ? -__builtin_inff() : m * scale + __logf(T::kNarrow ? l * 0.0078125f : l); }

template <int D>
struct Softmax {
    float m, l;
    v16f o[D / 32];
    __device__ __forceinline__ void clear()
    {
        m = kNothing;
        l = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    }
};

constexpr int kKeys = 64;  // keys to a tile

// KB blocks of 32 keys from tile0 on, in LDS, of which the lane's row sees those below `limit` (masked: some row of the
// wavefront does not see all of them).
template <typename T, int D, bool DROP, int KB = 2>
__device__ __forceinline__ void attend(Softmax<D> &x, const v8s (&q)[D / 16], const Operands<D> &op, uint32_t tk, uint32_t tv, int tile0, int limit,
                                       bool masked, float c, const Threefry &bits, uint32_t threshold, int row_q, int head, int lane)
{
    const int hf = lane >> 5;
    // All operands of a product are read before its first multiplication (left to itself the compiler reads each just in front of its
    // use, and every multiplication waits for the LDS): the keys here, the values in front of the exponentials.
    v16f s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.0f;
#pragma unroll
    for (int d0 = 0; d0 < D / 16; d0 += 4) {
        v8s k[KB][4];
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) k[kb][d] = op.along(tk, 32 * kb, d0 + d);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) s[kb] = T::mma32(k[kb][d], q[d0 + d], s[kb]);
    }
    v8s v[D == 64 ? KB : 1][2][D / 32];
    const auto read_values = [&](int kb, v8s (&to)[2][D / 32]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) to[h][i] = op.across(tv, 32 * kb + 16 * h, i);
    };
    if (masked) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][i] = tile0 + 32 * kb + 8 * (i >> 2) + 4 * hf + (i & 3) < limit ? s[kb][i] : -__builtin_inff();
    }
    float top = s[0][0], other = s[KB - 1][1];  // (two chains)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        top = max3(top, s[0][i], s[0][i + 1]);
        if (KB == 2) other = max3(other, s[KB - 1][i], s[KB - 1][i + 1]);
    }
    top = fmaxf(top, other);
    top = halves_max(top);
    if (__builtin_amdgcn_ballot_w64((top - x.m) * c > kLazy)) {
        const float m = fmaxf(x.m, top), f = __builtin_amdgcn_exp2f((x.m - m) * c);
        x.m = m;
        x.l *= f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) x.o[i][j] *= f;
    }
    if constexpr (D == 64) {
        read_values(0, v[0]);
        if constexpr (KB == 2) read_values(1, v[KB - 1]);
        __builtin_amdgcn_sched_barrier(0);
    }
    const float mc = x.m * c - kLift<T>;
    float sum = 0.0f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], c, -mc));
            sum += s[kb][i];
        }
    x.l += sum;
    if constexpr (DROP) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const v2u d = weight_draws(bits, row_q, head, tile0 + 32 * kb + 2 * i + 4 * hf);
                s[kb][i] = kept_low(d[0], threshold) ? s[kb][i] : 0.0f;
                s[kb][i + 1] = kept_high(d[0], threshold) ? s[kb][i + 1] : 0.0f;
                s[kb][i + 2] = kept_low(d[1], threshold) ? s[kb][i + 2] : 0.0f;
                s[kb][i + 3] = kept_high(d[1], threshold) ? s[kb][i + 3] : 0.0f;
            }
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        if constexpr (D != 64) read_values(kb, v[0]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4u w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = T::pair(s[kb][8 * h + 2 * i], s[kb][8 * h + 2 * i + 1]);
            const v8s p = __builtin_bit_cast(v8s, w);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) x.o[i] = T::mma32(v[D == 64 ? kb : 0][h][i], p, x.o[i]);
        }
    }
}

// A workgroup does 128 rows, a wavefront 32 of them; tiles of 64 keys and values go through a ring of stages in LDS, one used while the
// others are under way (three where three workgroups fit a CU all the same).  Bound by the matrix cores and the vector unit in turn: a
// wavefront's products wait for its exponentials, and the two or three wavefronts of a SIMD overlap them in part.  8192 causal keys, 16
// heads of 64: 176 us, 0.78 PFLOP/s; sequences of up to 3999, 16 heads of 128: 108 us, 0.87.  Short sequences are bound by a workgroup's
// start: 32 of up to 512, 12 heads of 64: 26 us, and 12 without any keys (places, first loads, outputs).
template <typename T, int D, bool DROP>
__global__ __launch_bounds__(256, 2) void attention_kernel(const AttnArgs a, uint16_t *O, float *lse, bool by_xcd)
{
    typedef Rows<D> R;
    constexpr int kTile = kKeys * R::kBytes, kStages = D == 64 ? 3 : 2, kCopies = 2 * kKeys / R::kPerCopy / 4;
    __shared__ __align__(1024) uint8_t lds[kStages][2 * kTile];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place<false>(a, blockIdx.x, a.tiles, by_xcd, true, lane);
    if (at.none) return;
    const int kv = at.kv;
    const Segment &seg = at.seg;
    const int rows = seg.nq * a.group, first = at.tile * 128;
    if (first >= rows) return;
    const int row = first + wave * 32 + l32;
    const int token = min((unsigned)row / (unsigned)a.group, (unsigned)seg.nq - 1u);  // rows past the end compute the last token's, unstored
    const int head = kv * a.group + (row - (int)((unsigned)row / (unsigned)a.group) * a.group);
    const int row_q = seg.q0 + token;

    // the keys that the lane's row, the wavefront's first and last row, and the workgroup's last row see
    const auto sees = [&](int t) { return a.causal ? min(seg.nk, max(0, seg.first_hidden(t))) : seg.nk; };
    const auto token_of = [&](int r) { return min(r / a.group, seg.nq - 1); };
    const int limit = sees(token);
    const int wave_least = __builtin_amdgcn_readfirstlane(sees(token_of(first + wave * 32)));
    const int wave_most = first + wave * 32 < rows ? __builtin_amdgcn_readfirstlane(sees(token_of(first + wave * 32 + 31))) : 0;  // (a wavefront without rows only copies)
    const int most = __builtin_amdgcn_readfirstlane(sees(token_of(first + 127)));
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
        // rows past the last key repeat it: its scores are masked, its values meet weights of zero
        copy_rows<D, kKeys, 4>(to, wave, lane, [&](int r) { return K + (int64_t)min(tile * kKeys + r, seg.nk - 1) * a.k_row; });
        copy_rows<D, kKeys, 4>(to + kTile, wave, lane, [&](int r) { return V + (int64_t)min(tile * kKeys + r, seg.nk - 1) * a.v_row; });
    };
    if (tiles > 0) fetch(0, 0);
    v8s q[D / 16];
    const uint16_t *const from = a.Q + (int64_t)row_q * a.q_row + (int64_t)head * a.q_head + 8 * hf;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) q[d] = *reinterpret_cast<const v8s *>(from + 16 * d);
    const Threefry bits(DROP ? (uint64_t)*a.seed : 0);
    const Operands<D> op(lane, lds0);
    Softmax<D> x;
    x.clear();
    wait_copies<0>();  // the first products wait for Q and the first tile, not for what follows them
    for (int t = 1; t < kStages - 1 && t < tiles; ++t) fetch(t, t);
    for (int t = 0, stage = 0; t < tiles; ++t, stage = stage == kStages - 1 ? 0 : stage + 1) {
        if (t + kStages - 1 <= tiles) wait_copies<(kStages - 2) * kCopies>();  // (the tiles behind this one may be under way)
        else wait_copies<0>();
        barrier();
        if (t + kStages - 1 < tiles) fetch(t + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
        const int left = wave_most - t * kKeys;
        const uint32_t tk = stage * 2 * kTile;
        constexpr bool kHalves = D == 64 && DROP;  // (without dropout's arithmetic to save, both in the kernel cost more: 177 -> 190 us for 8192 causal keys)
        if (left > (kHalves ? 32 : 0)) attend<T, D, DROP>(x, q, op, tk, tk + kTile, t * kKeys, limit, (t + 1) * kKeys > wave_least, a.c, bits, a.threshold, row_q, head, lane);
        else if (kHalves && left > 0) attend<T, D, DROP, 1>(x, q, op, tk, tk + kTile, t * kKeys, limit, t * kKeys + 32 > wave_least, a.c, bits, a.threshold, row_q, head, lane);
    }
    const float l = halves_sum(x.l);  // (zero where no key is seen; NaN stays NaN, in O and lse)
    const int64_t at_row = (int64_t)row_q * a.heads + head;
    write_row<T, D>(O + at_row * D, x.o, l == 0.0f ? 0.0f : (DROP ? a.inv_share : 1.0f) / l, hf, row < rows);
    if (row >= rows) return;
    if (hf == 0) lse[at_row] = lse_of<T>(x.m, l, a.scale);
}

// ---- few rows: the new tokens over a cache
// Up to 32 rows of a key head are one wavefront's; its keys are what there is to share out.  They are cut into chunks, a workgroup
// each, whose four wavefronts take the chunk's tiles in turn, each through two stages of its own in LDS and with no barrier: it
// waits for its own copies only, the next stage's under way.  The wavefronts' sums are joined in LDS, the chunks' by a second launch.
// Bound by the keys' and values' bytes; the products of up to 31 idle rows cost nothing beside them.  16 sequences of up to 16384 keys, 8 key heads
// of 128: 118 us and 9 us to join the chunks, 530 MB (4.5 TB/s in the first).  Few keys are bound by the launch and one chain of loads: 4 sequences of up to 390, 5.8 us.
template <typename T, int D, bool SPLIT>
__global__ __launch_bounds__(256, 1) void attention_cache_kernel(const AttnArgs a, uint16_t *O, float *lse, int chunk, int chunks, float *part)
{
    typedef Rows<D> R;
    constexpr int KB = D == 64 ? 2 : 1, kTileKeys = 32 * KB, kTile = kTileKeys * R::kBytes, kCopies = kTileKeys / R::kPerCopy;
    constexpr int kJoin = 32 * (D + 4) * 4;  // a wavefront's O, m, l
    __shared__ __align__(1024) uint8_t lds_all[4][4 * kTile > kJoin ? 4 * kTile : kJoin];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pairs = a.n_seqs * a.kv_heads, pair = (int)(blockIdx.x % pairs), at_chunk = (int)(blockIdx.x / pairs) % chunks, tile_r = (int)(blockIdx.x / pairs) / chunks;
    const int b = pair / a.kv_heads, kv = pair - b * a.kv_heads;
    const Segment seg = segment(a, b);
    const int rows = seg.nq * a.group, first = tile_r * 32;
    if (first >= rows) return;
    const int row = first + l32;
    const int token = min((unsigned)row / (unsigned)a.group, (unsigned)seg.nq - 1u);
    const int head = kv * a.group + (row - (int)((unsigned)row / (unsigned)a.group) * a.group);
    const int row_q = seg.q0 + token;
    const auto sees = [&](int t) { return a.causal ? min(seg.nk, max(0, seg.first_hidden(t))) : seg.nk; };
    const int limit = sees(token);
    const int least = __builtin_amdgcn_readfirstlane(sees(min(first / a.group, seg.nq - 1))), most = __builtin_amdgcn_readfirstlane(sees(min((first + 31) / a.group, seg.nq - 1)));
    const int begin = SPLIT ? at_chunk * chunk : 0, end = SPLIT ? min(most, begin + chunk) : most;
    if (SPLIT && at_chunk > 0 && begin >= end) return;  // (the joining launch knows which chunks there are)

    const uint16_t *const K = a.K + (int64_t)seg.k0 * a.k_row + (int64_t)kv * a.k_head;
    const uint16_t *const V = a.V + (int64_t)seg.k0 * a.v_row + (int64_t)kv * a.v_head;
    uint8_t *const lds = lds_all[wave];
    const uint32_t lds0 = lds_address(lds);
    const auto fetch = [&](int key0, int stage) {
        const uint32_t to = lds0 + stage * 2 * kTile;
        copy_rows<D, kTileKeys, 1>(to, 0, lane, [&](int r) { return K + (int64_t)min(key0 + r, seg.nk - 1) * a.k_row; });
        copy_rows<D, kTileKeys, 1>(to + kTile, 0, lane, [&](int r) { return V + (int64_t)min(key0 + r, seg.nk - 1) * a.v_row; });
    };
    const Operands<D> op(lane, lds0);
    Softmax<D> x;
    x.clear();
    const int step = 4 * kTileKeys, mine = begin + wave * kTileKeys;
    if (mine < end) fetch(mine, 0);
    v8s q[D / 16];
    const uint16_t *const from = a.Q + (int64_t)row_q * a.q_row + (int64_t)head * a.q_head + 8 * hf;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) q[d] = *reinterpret_cast<const v8s *>(from + 16 * d);
    const Threefry bits(0);
    int stage = 0;
    for (int key0 = mine; key0 < end; key0 += step, stage ^= 1) {
        if (key0 + step < end) {
            fetch(key0 + step, stage ^ 1);
            wait_copies<2 * kCopies>();
        } else {
            wait_copies<0>();
        }
        asm volatile("" ::: "memory");
        attend<T, D, false, KB>(x, q, op, stage * 2 * kTile, stage * 2 * kTile + kTile, key0, limit, key0 + kTileKeys > least, a.c, bits, 0, row_q, head, lane);
        __builtin_amdgcn_s_waitcnt(0xC07F);  // this stage's reads have returned before the next copies into it
        asm volatile("" ::: "memory");
    }
    x.l = halves_sum(x.l);
    // joined in LDS: [row][D values, m, l]
    float *const own = reinterpret_cast<float *>(lds);
    constexpr int kPitch = D + 4;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; j += 4) *reinterpret_cast<v4f *>(own + l32 * kPitch + 32 * i + 2 * j + 4 * hf) = v4f{x.o[i][j], x.o[i][j + 1], x.o[i][j + 2], x.o[i][j + 3]};
    if (hf == 0) {
        own[l32 * kPitch + D] = x.m;
        own[l32 * kPitch + D + 1] = x.l;
    }
    barrier();
    // a thread does eight neighbouring values of a row
    constexpr int kThreads = D / 8;
    const int here = min(32, rows - first);
    for (int i = threadIdx.x; i < here * kThreads; i += 256) {
        const int r = i / kThreads, d = (i - r * kThreads) * 8;
        float m = kNothing, l = 0.0f;
        const float *const all = reinterpret_cast<const float *>(lds_all[0]) + r * kPitch;
        constexpr int kWaveFloats = (int)(sizeof(lds_all[0]) / 4);
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, all[w * kWaveFloats + D]);
        v4f o[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f((all[w * kWaveFloats + D] - m) * a.c);
            l += f * all[w * kWaveFloats + D + 1];
            o[0] += f * *reinterpret_cast<const v4f *>(all + w * kWaveFloats + d);
            o[1] += f * *reinterpret_cast<const v4f *>(all + w * kWaveFloats + d + 4);
        }
        const int t = (first + r) / a.group, h = kv * a.group + first + r - t * a.group;
        if constexpr (SPLIT) {
            float *const to = part + ((int64_t)((pair * (int64_t)a.tiles + tile_r) * chunks + at_chunk) * 32 + r) * kPitch;
            *reinterpret_cast<v4f *>(to + d) = o[0];
            *reinterpret_cast<v4f *>(to + d + 4) = o[1];
            if (d == 0) {
                to[D] = m;
                to[D + 1] = l;
            }
        } else {
            const float f = l == 0.0f ? 0.0f : 1.0f / l;
            const int64_t at_row = (int64_t)(seg.q0 + t) * a.heads + h;
            *reinterpret_cast<v4u *>(O + at_row * D + d) = v4u{T::pair(o[0][0] * f, o[0][1] * f), T::pair(o[0][2] * f, o[0][3] * f), T::pair(o[1][0] * f, o[1][1] * f), T::pair(o[1][2] * f, o[1][3] * f)};
            if (d == 0) lse[at_row] = lse_of<T>(m, l, a.scale);
        }
    }
}

// the chunks of every row joined: a wavefront to a row, D / 64 values a lane
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttnArgs a, uint16_t *O, float *lse, int chunk, int chunks, const float *part, int max_rows)
{
    constexpr int kPitch = D + 4, N = D / 64;
    const int lane = threadIdx.x & 63, id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pair = id / max_rows, r = id - pair * max_rows;
    if (pair >= a.n_seqs * a.kv_heads) return;
    const int b = pair / a.kv_heads, kv = pair - b * a.kv_heads;
    const Segment seg = segment(a, b);
    if (r >= seg.nq * a.group) return;
    const int tile_r = r >> 5, t = r / a.group, h = kv * a.group + r - t * a.group;
    const int last_token = min((tile_r * 32 + 31) / a.group, seg.nq - 1);  // the tile's chunks reach as far as its last row sees
    const int most = a.causal ? min(seg.nk, max(0, seg.first_hidden(last_token))) : seg.nk;
    const int n = min(chunks, max(1, (most + chunk - 1) / chunk));
    const float *const from = part + ((int64_t)(pair * (int64_t)a.tiles + tile_r) * chunks * 32 + (r & 31)) * kPitch;
    float m = kNothing, l = 0.0f, o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.0f;
    for (int c = 0; c < n; ++c) {
        const float *const p = from + (int64_t)c * 32 * kPitch;
        const float m1 = p[D], top = fmaxf(m, m1), f = __builtin_amdgcn_exp2f((m - top) * a.c), g = __builtin_amdgcn_exp2f((m1 - top) * a.c);
        m = top;
        l = l * f + p[D + 1] * g;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = o[i] * f + p[N * lane + i] * g;
    }
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t at_row = (int64_t)(seg.q0 + t) * a.heads + h;
    if constexpr (N == 2) *reinterpret_cast<uint32_t *>(O + at_row * D + 2 * lane) = T::pair(o[0] * f, o[N - 1] * f);
    else O[at_row * D + lane] = (uint16_t)T::pair(o[0] * f, 0.0f);
    if (lane == 0) lse[at_row] = lse_of<T>(m, l, a.scale);
}

// Few rows (without dropout, which serving has none of): up to 32 of a key head, or more where the other kernel would leave most CUs idle: it
// reads the keys once for 128 rows but has one workgroup for them.  16 sequences of 4096 keys, 8 key heads of 128: 32 rows 64 us here, 80 there; 64 rows 120
// here, 82 there, and 128 rows 222 and 82.  What it takes is that of one workgroup, what this one takes grows with the tiles of 32 rows: even at about 170.
// The chunks: as many as fill the GPU with about 2048 workgroups, half of which find no keys where lengths differ, of 512 keys or more.
constexpr int64_t kFewTiles = 160;
struct Chunks {
    int64_t size, count;
};
inline Chunks chunks_of(int64_t pairs, int64_t max_k)
{
    Chunks c;
    c.count = std::max<int64_t>(1, std::min((max_k + 511) / 512, (2048 + pairs - 1) / pairs));
    c.size = std::max<int64_t>(256, (((max_k + c.count - 1) / c.count) + 255) / 256 * 256);
    c.count = std::max<int64_t>(1, (max_k + c.size - 1) / c.size);
    return c;
}
inline bool few_rows(const AttnArgs &a, const qb_attention *p)
{
    const int64_t tiles = (p->max_q * a.group + 31) / 32;
    return (tiles <= 1 || tiles * a.n_seqs * a.kv_heads <= kFewTiles) && !(p->p > 0.0f);
}

template <typename T, int D>
qb_status forward_few(AttnArgs a, int64_t max_q, int64_t max_k, void *O, float *lse, void *workspace, hipStream_t stream)
{
    const int64_t pairs = (int64_t)a.n_seqs * a.kv_heads, rows = max_q * a.group;
    a.tiles = (int)((rows + 31) / 32);
    const Chunks c = chunks_of(pairs, max_k);
    const int64_t grid = pairs * a.tiles * c.count;
    if (grid > INT32_MAX / 256 || pairs * rows > INT32_MAX / 256) return QB_ERR_SHAPE;
    uint16_t *const out = static_cast<uint16_t *>(O);
    float *const part = static_cast<float *>(workspace);
    if (c.count == 1) {
        attention_cache_kernel<T, D, false><<<(int)grid, 256, 0, stream>>>(a, out, lse, 0, 1, nullptr);
    } else {
        attention_cache_kernel<T, D, true><<<(int)grid, 256, 0, stream>>>(a, out, lse, (int)c.size, (int)c.count, part);
        attention_join_kernel<T, D><<<(int)((pairs * rows + 3) / 4), 256, 0, stream>>>(a, out, lse, (int)c.size, (int)c.count, part, (int)rows);
    }
    return launch_status();
}

template <typename T, int D>
qb_status forward(AttnArgs a, int64_t max_q, bool drop, void *O, float *lse, hipStream_t stream)
{
    const int64_t pairs = (int64_t)a.n_seqs * a.kv_heads;
    a.tiles = (int)((max_q * a.group + 127) / 128);
    const int64_t grid = dealt_workgroups(pairs, a.tiles);
    if (grid > INT32_MAX / 256) return QB_ERR_SHAPE;
    const bool by_xcd = deal_by_xcd(pairs);
    if (drop) attention_kernel<T, D, true><<<(int)grid, 256, 0, stream>>>(a, static_cast<uint16_t *>(O), lse, by_xcd);
    else attention_kernel<T, D, false><<<(int)grid, 256, 0, stream>>>(a, static_cast<uint16_t *>(O), lse, by_xcd);
    return launch_status();
}

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" size_t qb_attention_fwd_workspace_nbytes(const qb_attention *p)
{
    AttnArgs a;
    if (attention_args(p, a) != QB_OK || p->max_q == 0 || p->n_seqs == 0 || !few_rows(a, p)) return 0;
    const int64_t pairs = (int64_t)a.n_seqs * a.kv_heads, tiles = (p->max_q * a.group + 31) / 32;
    const Chunks c = chunks_of(pairs, p->max_k);
    return c.count == 1 ? 0 : (size_t)(pairs * tiles * c.count) * 32 * (p->dim + 4) * 4;
}

namespace {
template <typename T, int D>
qb_status forward_any(const AttnArgs &a, const qb_attention *p, void *O, float *lse, void *workspace, hipStream_t stream)
{
    if (few_rows(a, p)) return forward_few<T, D>(a, p->max_q, p->max_k, O, lse, workspace, stream);
    return forward<T, D>(a, p->max_q, p->p > 0.0f, O, lse, stream);
}
}  // namespace

extern "C" qb_status qb_attention_fwd(const qb_attention *p, void *O, float *lse, void *workspace, void *stream)
{
    AttnArgs a;
    const qb_status s = attention_args(p, a);
    if (s != QB_OK) return s;
    if (p->total_q == 0 || p->n_seqs == 0 || p->max_q == 0) return QB_OK;
    if (!O || !lse) return QB_ERR_NULL;
    if (!aligned16(O)) return QB_ERR_VALUE;
    if (qb_attention_fwd_workspace_nbytes(p) > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255))) return QB_ERR_WORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (p->type == QB_TYPE_BF16) return p->dim == 64 ? forward_any<Bf16, 64>(a, p, O, lse, workspace, st) : forward_any<Bf16, 128>(a, p, O, lse, workspace, st);
    return p->dim == 64 ? forward_any<Fp16, 64>(a, p, O, lse, workspace, st) : forward_any<Fp16, 128>(a, p, O, lse, workspace, st);
}
