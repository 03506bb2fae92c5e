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
#include <cmath>

namespace qb {

qb_status attention_args(const qb_attention *p, AttnArgs &a)
{
    if (!p) return QB_ERR_NULL;
    if (p->total_q < 0 || p->total_k < 0 || p->total_q > INT32_MAX - 4096 || p->total_k > INT32_MAX - 4096 || p->n_seqs < 0 || p->heads <= 0 ||
        p->kv_heads <= 0 || p->heads % p->kv_heads != 0 || p->heads > (1 << 16) || (p->dim != 64 && p->dim != 128) || p->max_q < 0 || p->max_k < 0 ||
        p->max_q > INT32_MAX || p->max_k > INT32_MAX - 4096 || p->max_q * (p->heads / p->kv_heads) >= (1 << 30))
        return QB_ERR_SHAPE;
    if ((p->type != QB_TYPE_BF16 && p->type != QB_TYPE_FP16) || !(p->scale > 0.0f) || !std::isfinite(p->scale * 1.5f) || !(p->p >= 0.0f && p->p < 1.0f) ||
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

// One tile of keys: keys tile0 .. tile0 + 63 in LDS, of which the lane's row sees those below `limit` (masked: some row of the
// wavefront does not see all of them).
template <typename T, int D, bool DROP>
__device__ __forceinline__ void attend(Softmax<D> &x, const v8s (&q)[D / 16], const uint8_t *tk, const uint8_t *tv, int tile0, int limit,
                                       bool masked, float c, const Threefry &bits, uint32_t threshold, int row_q, int head, int lane)
{
    typedef Rows<D> R;
    const int hf = lane >> 5;
    v16f s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.0f;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) s[kb] = T::mma32(R::along(tk, 32 * kb, d, lane), q[d], s[kb]);
    }
    if (masked) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][i] = tile0 + 32 * kb + 8 * (i >> 2) + 4 * hf + (i & 3) < limit ? s[kb][i] : -__builtin_inff();
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, fmaxf(s[0][i], s[1][i]));
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
    const float mc = x.m * c;
    float sum = 0.0f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], c, -mc));
            sum += s[kb][i];
        }
    x.l += sum;
    if constexpr (DROP) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
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
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4u w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = T::pair(s[kb][8 * h + 2 * i], s[kb][8 * h + 2 * i + 1]);
            const v8s p = __builtin_bit_cast(v8s, w);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) x.o[i] = T::mma32(R::across(tv, 32 * kb + 16 * h, 32 * i, lane), p, x.o[i]);
        }
}

// O^T / l to a row of O: the lane holds four neighbouring values of its row at a time
template <typename T, int D>
__device__ __forceinline__ void write_row(uint16_t *row, const v16f (&o)[D / 32], float f, int hf)
{
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
            const v2u w = {T::pair(o[i][j] * f, o[i][j + 1] * f), T::pair(o[i][j + 2] * f, o[i][j + 3] * f)};
            *reinterpret_cast<v2u *>(row + 32 * i + 2 * j + 4 * hf) = w;
        }
}

// A workgroup does 128 rows, a wavefront 32 of them; tiles of 64 keys and values go through two stages in LDS, one under way
// while the other is used.
template <typename T, int D, bool DROP>
__global__ __launch_bounds__(256, 2) void attention_kernel(const AttnArgs a, uint16_t *O, float *lse, bool by_xcd)
{
    typedef Rows<D> R;
    constexpr int kTile = kKeys * R::kBytes;
    __shared__ __align__(1024) uint8_t lds[2][2 * kTile];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place(blockIdx.x, a.n_seqs * a.kv_heads, a.tiles, by_xcd);
    if (at.pair >= a.n_seqs * a.kv_heads) return;
    const int b = at.pair / a.kv_heads, kv = at.pair - b * a.kv_heads;
    const Segment seg = segment(a, b);
    const int rows = seg.nq * a.group, first = at.tile * 128;
    if (first >= rows) return;
    const int row = first + wave * 32 + l32;
    const int token = min((unsigned)row / (unsigned)a.group, (unsigned)seg.nq - 1u);  // rows past the end compute the last token's, unstored
    const int head = kv * a.group + (row - (int)((unsigned)row / (unsigned)a.group) * a.group);
    const int row_q = seg.q0 + token;

    v8s q[D / 16];
    const uint16_t *const from = a.Q + (int64_t)row_q * a.q_row + (int64_t)head * a.q_head + 8 * hf;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) q[d] = *reinterpret_cast<const v8s *>(from + 16 * d);

    // the keys that the lane's row, the wavefront's first and last row, and the workgroup's last row see
    const auto sees = [&](int t) { return a.causal ? min(seg.nk, max(0, seg.first_hidden(t))) : seg.nk; };
    const auto token_of = [&](int r) { return min(r / a.group, seg.nq - 1); };
    const int limit = sees(token);
    const int wave_least = __builtin_amdgcn_readfirstlane(sees(token_of(first + wave * 32)));
    const int wave_most = __builtin_amdgcn_readfirstlane(sees(token_of(first + wave * 32 + 31)));
    const int most = __builtin_amdgcn_readfirstlane(sees(token_of(first + 127)));
    const int tiles = (most + kKeys - 1) / kKeys;

    const uint16_t *const K = a.K + (int64_t)seg.k0 * a.k_row + (int64_t)kv * a.k_head;
    const uint16_t *const V = a.V + (int64_t)seg.k0 * a.v_row + (int64_t)kv * a.v_head;
    const uint32_t lds0 = lds_address(lds);
    const auto fetch = [&](int tile, int stage) {
        // rows past the last key repeat it: its scores are masked, its values meet weights of zero
        const uint32_t to = lds0 + stage * 2 * kTile;
        copy_rows<D, kKeys, 4>(to, wave, lane, [&](int r) { return K + (int64_t)min(tile * kKeys + r, seg.nk - 1) * a.k_row; });
        copy_rows<D, kKeys, 4>(to + kTile, wave, lane, [&](int r) { return V + (int64_t)min(tile * kKeys + r, seg.nk - 1) * a.v_row; });
    };
    const Threefry bits(DROP ? (uint64_t)*a.seed : 0);
    Softmax<D> x;
    x.clear();
    if (tiles) fetch(0, 0);
    for (int t = 0; t < tiles; ++t) {
        wait_copies<0>();
        barrier();
        if (t + 1 < tiles) fetch(t + 1, (t + 1) & 1);
        if (t * kKeys < wave_most)
            attend<T, D, DROP>(x, q, lds[t & 1], lds[t & 1] + kTile, t * kKeys, limit, (t + 1) * kKeys > wave_least, a.c, bits, a.threshold, row_q, head, lane);
    }
    if (row >= rows) return;
    const float l = halves_sum(x.l);
    const int64_t at_row = (int64_t)row_q * a.heads + head;
    write_row<T, D>(O + at_row * D, x.o, l > 0.0f ? (DROP ? a.inv_share : 1.0f) / l : 0.0f, hf);
    if (hf == 0) lse[at_row] = l > 0.0f ? x.m * a.scale + __logf(l) : -__builtin_inff();
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
    if (attention_args(p, a) != QB_OK) return 0;
    return 0;
}

extern "C" qb_status qb_attention_fwd(const qb_attention *p, void *O, float *lse, void *workspace, void *stream)
{
    AttnArgs a;
    const qb_status s = attention_args(p, a);
    if (s != QB_OK) return s;
    if (p->total_q == 0 || p->n_seqs == 0 || p->max_q == 0) return QB_OK;
    if (!O || !lse) return QB_ERR_NULL;
    if (!aligned16(O)) return QB_ERR_VALUE;
    (void)workspace;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool drop = p->p > 0.0f;
    if (p->type == QB_TYPE_BF16) return p->dim == 64 ? forward<Bf16, 64>(a, p->max_q, drop, O, lse, st) : forward<Bf16, 128>(a, p->max_q, drop, O, lse, st);
    return p->dim == 64 ? forward<Fp16, 64>(a, p->max_q, drop, O, lse, st) : forward<Fp16, 128>(a, p->max_q, drop, O, lse, st);
}
