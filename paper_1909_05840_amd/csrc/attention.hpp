// What the attention kernels' forward and backward share: their arguments, a sequence's part of the packed tensors, the order
// of the workgroups.
#pragma once
#include "qb_tiles.hpp"

namespace qb {

struct AttnArgs {
    const uint16_t *Q, *K, *V;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    int heads, kv_heads, group;  // group: query heads to a key head
    int total_q, total_k;
    int n_seqs, causal;
    const int32_t *cu_q, *cu_k, *k_len;
    int tiles;         // row (or key) tiles of the longest sequence
    float scale, c;    // c = scale / ln 2: exponentials are powers of two
    const int64_t *seed;
    uint32_t threshold;
    float inv_share;   // one over the share that dropout keeps
};

// Queries of one key head are laid end to end as rows r = token * group + head of the group, so that heads that share keys
// share the tiles of them too.
struct Segment {
    int q0, nq, k0, nk;
    __device__ __forceinline__ int first_hidden(int token) const { return token + 1 + nk - nq; }  // causal: keys below this are seen
};
__device__ __forceinline__ Segment segment(const AttnArgs &a, int b)
{
    Segment s;
    s.q0 = a.cu_q[b];
    s.nq = a.cu_q[b + 1];
    s.k0 = a.cu_k[b];
    s.nk = a.cu_k[b + 1];
    if (a.k_len) {
        const int n = a.k_len[b];
        s.nk = n < s.nk - s.k0 ? s.k0 + n : s.nk;
    }
    // (whatever the arrays say, nothing outside the tensors is touched)
    s.q0 = s.q0 > 0 ? s.q0 : 0;
    s.k0 = s.k0 > 0 ? s.k0 : 0;
    s.nq = (s.nq < a.total_q ? s.nq : a.total_q) - s.q0;
    s.nk = (s.nk < a.total_k ? s.nk : a.total_k) - s.k0;
    s.nk = s.nk > 0 ? s.nk : 0;
    return s;
}

// The nth longest sequence (of up to 64; of more, the nth): workgroups take the sequences in that order, so that those with the most tiles are
// at work first and every CU gets some of either kind.
__device__ __forceinline__ int nth_longest(const AttnArgs &a, int nth, int lane)
{
    if (a.n_seqs == 1 || a.n_seqs > 64) return nth;
    const int i = min(lane, a.n_seqs - 1), length = a.cu_q[i + 1] - a.cu_q[i] + a.cu_k[i + 1] - a.cu_k[i];
    int before = 0;
    for (int j = 0; j < a.n_seqs; ++j) {
        const int other = __builtin_amdgcn_readlane(length, j);
        before += other > length || (other == length && j < lane);
    }
    return __builtin_ctzll(__builtin_amdgcn_ballot_w64(before == nth && lane < a.n_seqs));
}

// Which tile of which (sequence, key head) a workgroup does.  Workgroups are dealt to the eight XCDs in turn, each with an L2
// of its own: where there are pairs enough, all tiles of a pair go to one XCD, which fetches its keys once.  Tiles of the largest number
// come first: with causal masks they see the most keys.
struct Place {
    int pair, tile;
};
__device__ __forceinline__ Place place(int id, int pairs, int tiles, bool by_xcd)
{
    if (by_xcd) {
        const int i = id >> 3;
        return {(i / tiles) * 8 + (id & 7), tiles - 1 - i % tiles};
    }
    return {id % pairs, tiles - 1 - id / pairs};
}
inline bool deal_by_xcd(int64_t pairs) { return pairs % 8 == 0 || pairs >= 64; }
inline int64_t dealt_workgroups(int64_t pairs, int64_t tiles) { return (deal_by_xcd(pairs) ? (pairs + 7) / 8 * 8 : pairs) * tiles; }

qb_status attention_args(const qb_attention *p, AttnArgs &a);  // checks and converts

// Tiles of `ROWS` rows of D values each from memory to LDS by WAVES wavefronts, 16 bytes a lane; row(i) is the address of tile row i.
template <int D, int ROWS, int WAVES, typename F>
__device__ __forceinline__ void copy_rows(uint32_t lds, int wave, int lane, const F &row)
{
    typedef Rows<D> R;
    constexpr int kCopies = ROWS / R::kPerCopy;
    static_assert(kCopies % WAVES == 0, "every wavefront copies the same number of times");
#pragma unroll
    for (int i = 0; i < kCopies / WAVES; ++i) {
        const int first = (i * WAVES + wave) * R::kPerCopy, r = first + R::copy_row(lane);
        copy16(row(r) + 8 * R::copy_chunk(r, lane), lds + first * R::kBytes);
    }
}

// The same for whole tiles of rows whose distances from the tile's first row do not change from tile to tile: the lane's offsets are
// formed once, and a copy takes no vector arithmetic.  (Formed anew they were a third of the forward's vector instructions, and with the
// division by the group more than half of those of dK and dV.)
template <int D, int ROWS, int WAVES>
struct TileCopy {
    typedef Rows<D> R;
    static constexpr int N = ROWS / R::kPerCopy / WAVES;
    uint32_t offset[N];
    template <typename F>  // values from the tile's first row to row i
    __device__ __forceinline__ TileCopy(int wave, int lane, const F &distance)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = (i * WAVES + wave) * R::kPerCopy + R::copy_row(lane);
            offset[i] = (uint32_t)(distance(r) + 8 * R::copy_chunk(r, lane)) * 2;
        }
    }
    __device__ __forceinline__ void copy(const uint16_t *base, uint32_t lds, int wave) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) copy16(base, offset[i], lds + (i * WAVES + wave) * (R::kPerCopy * R::kBytes));
    }
};
// whether the rows of a tile lie less than 2^31 bytes apart
__device__ __forceinline__ bool near_rows(int64_t stride) { return stride >= 0 && stride < (1 << 23); }

// The draws of four neighbouring keys of a query (k a multiple of 4).
__device__ __forceinline__ v2u weight_draws(const Threefry &bits, int row_q, int head, int k)
{
    return bits.draws((uint32_t)row_q, 0x80000000u + ((uint32_t)head << 22) + ((uint32_t)k >> 2));
}

}  // namespace qb
