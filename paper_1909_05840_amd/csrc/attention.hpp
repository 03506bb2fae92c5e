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
    s.nq = max(0, (s.nq < a.total_q ? s.nq : a.total_q) - s.q0);
    s.nk = max(0, (s.nk < a.total_k ? s.nk : a.total_k) - s.k0);
    return s;
}

// Which tile of which (sequence, key head) a workgroup does.  Workgroups are dealt to the eight XCDs in turn, each with an L2
// of its own: where there are pairs enough, all tiles of a pair go to one XCD, which fetches its keys once.  Tiles with the
// most work under a causal mask come first: the last rows, the first keys.  With 2 to 64 sequences a wavefront's lanes hold one
// each: sequences come by their lengths, the longest first, and the tiles that there are take the first workgroups, so that
// the empty ones of a ragged batch come last and cost next to nothing.
struct Place {
    int pair, tile;  // (pair: the sequence, or its rank by length, times kv_heads, and the key head)
    Segment seg;
    int seq, kv;
    bool none;
};
// KEYS: tiles of 128 keys, else of 128 rows; by_length: there is one workgroup to such a tile
template <bool KEYS>
__device__ __forceinline__ Place place(const AttnArgs &a, int id, int tiles, bool by_xcd, bool by_length, int lane)
{
    Place p;
    const int pairs = a.n_seqs * a.kv_heads;
    if (a.n_seqs > 64 || a.n_seqs == 1 || !by_xcd || !by_length) {
        const int i = by_xcd ? id >> 3 : id;
        p.pair = by_xcd ? (i / tiles) * 8 + (id & 7) : id % pairs;
        p.tile = by_xcd ? i % tiles : id / pairs;
        if (!KEYS) p.tile = tiles - 1 - p.tile;
        p.none = p.pair >= pairs;
        const int b = p.none ? 0 : p.pair / a.kv_heads;
        p.seq = b;
        p.kv = p.pair - b * a.kv_heads;
        p.seg = segment(a, b);
        return p;
    }
    const Segment mine = segment(a, min(lane, a.n_seqs - 1));
    const int length = mine.nq + mine.nk;
    int rank = 0;
    for (int j = 0; j < a.n_seqs; ++j) {
        const int other = __builtin_amdgcn_readlane(length, j);
        rank += other > length || (other == length && j < lane);
    }
    const bool in = lane < a.n_seqs;
    rank = in ? rank : lane;
    const int count = !in ? 0 : KEYS ? (mine.nk + 127) >> 7 : (mine.nq * a.group + 127) >> 7;
    // from here on a lane stands for a rank
    const int n = __builtin_amdgcn_ds_permute(rank << 2, count), who = __builtin_amdgcn_ds_permute(rank << 2, lane);
    const int xcd = id & 7, first = (xcd - lane * a.kv_heads) & 7, heads = first < a.kv_heads ? (a.kv_heads - first + 7) >> 3 : 0;  // of the rank's key heads on this XCD
    const int items = n * heads;
    int sum = items;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int before = __shfl_up(sum, o);
        sum += lane >= o ? before : 0;
    }
    const int slot = id >> 3;
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(sum > slot);
    p.none = beyond == 0;
    if (p.none) return p;
    const int r = __builtin_ctzll(beyond), of = __builtin_amdgcn_readlane(n, r), rest = slot - __builtin_amdgcn_readlane(sum - items, r);
    const int nth = __builtin_amdgcn_readfirstlane(rest / of), seq = __builtin_amdgcn_readlane(who, r);
    p.tile = KEYS ? rest - nth * of : of - 1 - (rest - nth * of);
    p.kv = __builtin_amdgcn_readlane(first, r) + 8 * nth;
    p.seq = seq;
    p.pair = r * a.kv_heads + p.kv;
    p.seg = {__builtin_amdgcn_readlane(mine.q0, seq), __builtin_amdgcn_readlane(mine.nq, seq), __builtin_amdgcn_readlane(mine.k0, seq), __builtin_amdgcn_readlane(mine.nk, seq)};
    return p;
}
inline bool deal_by_xcd(int64_t pairs) { return pairs % 8 == 0 || pairs >= 64; }
inline int64_t dealt_workgroups(int64_t pairs, int64_t tiles) { return (deal_by_xcd(pairs) ? (pairs + 7) / 8 * 8 : pairs) * tiles; }

// f times a row's D values, held as products hold them (value d of the row in the lane pair's result d), rounded to 16 bits, 16 bytes a store;
// every lane of the wavefront calls it, and `write` is the same for both lanes of a row
template <typename T, int D>
__device__ __forceinline__ void write_row(uint16_t *row, const v16f (&o)[D / 32], float f, int hf, bool write)
{
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; j += 8) {
            const v2u low = {T::pair(o[i][j] * f, o[i][j + 1] * f), T::pair(o[i][j + 2] * f, o[i][j + 3] * f)};
            const v2u high = {T::pair(o[i][j + 4] * f, o[i][j + 5] * f), T::pair(o[i][j + 6] * f, o[i][j + 7] * f)};
            const v4u w = join_halves(low, high);
            if (write) *reinterpret_cast<v4u *>(row + 32 * i + 2 * j + 8 * hf) = w;
        }
}

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
