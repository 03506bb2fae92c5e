// What the 16-bit linears' forward and backward share: the stream of steps through LDS, a product's results as rows.
#pragma once
#include "qb_acts.hpp"
#include "qb_products.hpp"

namespace qb {

// sixteen bytes that are zero, in place of what lies behind a contraction's end
static __device__ const uint4 kZeros = {0, 0, 0, 0};

// Tile number of a workgroup.  Workgroups are dealt to the eight XCDs in turn: those of one XCD get tiles that follow each other, so that what
// neighbours share is fetched once into its L2.
__device__ __forceinline__ int tile_of(int group, int tiles)
{
    const int xcd = group & 7, each = tiles >> 3, rest = tiles & 7;
    return xcd * each + min(xcd, rest) + (group >> 3);
}

// One operand of a product on its way to LDS.  `at` is the first step's place in memory, the same for all lanes; a lane's chunk of copy i lies `off[i]` bytes
// further on; each step moves on by `step` bytes.
template <int N>
struct Feed {
    const uint8_t *at;
    int64_t step;
    uint32_t off[N];
};
// Rows of results with the contraction along them: row r of the tile is row min(first + r, rows - 1) of the matrix (`row` bytes each).
template <typename S, int N>
__device__ __forceinline__ Feed<N> along(const void *base, int64_t row, int first, int rows, int s0, int wave, int lane)
{
    typedef Rows<64> R;
    Feed<N> f;
    f.at = static_cast<const uint8_t *>(base) + first * row + (int64_t)s0 * 128;
    f.step = 128;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = S::row(i, wave, lane);
        f.off[i] = (uint32_t)(min(r, rows - 1 - first) * row) + 16 * R::copy_chunk(r, lane);
    }
    return f;
}
// Rows along the contraction: LDS row r holds 64 results from 64 * (r / 64) on, of step r % 64; past the last column (a multiple of eight) the last eight again.
template <typename S, int N>
__device__ __forceinline__ Feed<N> across(const void *base, int64_t row, int first, int columns, int s0, int wave, int lane)
{
    typedef Rows<64> R;
    Feed<N> f;
    f.at = static_cast<const uint8_t *>(base) + (int64_t)s0 * 64 * row;
    f.step = 64 * row;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = S::row(i, wave, lane);
        f.off[i] = (uint32_t)((r & 63) * row) + 2 * min(first + (r & ~63) + 8 * R::copy_chunk(r, lane), columns - 8);
    }
    return f;
}

// acc += A B^T over `steps` steps.  Of the last one `left_a` and `left_b` values of the contraction are there (64, or fewer: a multiple of eight where the operand has it
// along its rows); zeros stand for the others.
template <typename T, typename S, bool A_ACROSS, bool B_ACROSS, int NA, int NB>
__device__ __forceinline__ void multiply(v16f (&acc)[S::TM][S::TN], uint8_t *lds, int steps, int left_a, int left_b, int wave, int lane, Feed<NA> a, Feed<NB> b)
{
    constexpr int kAhead = S::kStages - 1;
    static_assert(NA * 8 * S::kWaves == S::BM && NB * 8 * S::kWaves == S::BN, "every wavefront copies the same number of times");
    typedef Rows<64> R;
    const uint32_t lds0 = lds_address(lds);
    int next = 0;
    const auto fetch = [&](int stage) {
        if (next >= steps) return;
        const uint32_t to = lds0 + stage * S::kStage + wave * 1024;
        if (++next == steps && left_a < 64) {
            const auto there = [&](bool turned, int left, int i) {
                const int r = S::row(i, wave, lane);
                return turned ? (r & 63) < left : 8 * R::copy_chunk(r, lane) < left;
            };
#pragma unroll
            for (int i = 0; i < NA; ++i) copy16(there(A_ACROSS, left_a, i) ? static_cast<const void *>(a.at + a.off[i]) : &kZeros, to + i * S::kWaves * 1024);
#pragma unroll
            for (int i = 0; i < NB; ++i) copy16(there(B_ACROSS, left_b, i) ? static_cast<const void *>(b.at + b.off[i]) : &kZeros, to + S::BM * 128 + i * S::kWaves * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < NA; ++i) copy16(a.at, a.off[i], to + i * S::kWaves * 1024);
#pragma unroll
            for (int i = 0; i < NB; ++i) copy16(b.at, b.off[i], to + S::BM * 128 + i * S::kWaves * 1024);
        }
        a.at += a.step;
        b.at += b.step;
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u) fetch(u);
    int stage = 0;
    for (int s = 0; s < steps; ++s) {
        if (s + kAhead <= steps) wait_copies<(kAhead - 1) * (NA + NB)>();  // (younger steps' stay under way)
        else wait_copies<0>();
        barrier();
        fetch(stage == 0 ? kAhead : stage - 1);  // (into the stage that the last step was multiplied from)
        step<T, S, A_ACROSS, B_ACROSS>(acc, lds + stage * S::kStage, wave, lane);
        stage = stage == kAhead ? 0 : stage + 1;
    }
}

// The inverse of join_halves: eight neighbours a lane to two quads' words.
__device__ __forceinline__ void part_halves(v4u w, v2u &first, v2u &second)
{
    const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    first = v2u{a[0], b[0]};
    second = v2u{a[1], b[1]};
}
// Sixteen codes a lane (the lower half of the wavefront has the block's first sixteen) from the lane's four quads, and back.
__device__ __forceinline__ v4u join_codes(v4u quads)
{
    const auto a = __builtin_amdgcn_permlane32_swap(quads[0], quads[2], false, false), b = __builtin_amdgcn_permlane32_swap(quads[1], quads[3], false, false);
    return v4u{a[0], a[1], b[0], b[1]};
}
__device__ __forceinline__ v4u part_codes(v4u w)
{
    const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[1], false, false), b = __builtin_amdgcn_permlane32_swap(w[2], w[3], false, false);
    return v4u{a[0], b[0], a[1], b[1]};
}

// The values of one 32 x 32 block of results that a lane holds: of one row, columns 8 * q + 4 * (lane / 32) + 0 .. 3 for q = 0 .. 3.
// Rows in memory have `width` columns; the lane's row may be past the last one (`inside` false: not touched; all lanes take part in the exchanges).
template <typename T>
struct Block {
    static __device__ __forceinline__ void load(const uint16_t *p, int64_t at, int col, int width, bool inside, int hf, float (&v)[16])
    {
#pragma unroll
        for (int k = 0; k < 16; k += 8) {
            const int c = col + 2 * k + 8 * hf;
            v4u w = {0, 0, 0, 0};
            if (inside) {
                if (c + 8 <= width) w = load16(p + at, 2 * c);
                else each<8>([&](auto e) { if (c + e < width) w[e >> 1] |= (uint32_t)p[at + c + e] << (16 * (e & 1)); });
            }
            v2u a, b;
            part_halves(w, a, b);
            v[k] = T::lo(a[0]); v[k + 1] = T::hi(a[0]); v[k + 2] = T::lo(a[1]); v[k + 3] = T::hi(a[1]);
            v[k + 4] = T::lo(b[0]); v[k + 5] = T::hi(b[0]); v[k + 6] = T::lo(b[1]); v[k + 7] = T::hi(b[1]);
        }
    }
    static __device__ __forceinline__ void store(uint16_t *p, int64_t at, int col, int width, bool inside, int hf, const float (&v)[16])
    {
#pragma unroll
        for (int k = 0; k < 16; k += 8) {
            const v4u w = join_halves(v2u{T::pair(v[k], v[k + 1]), T::pair(v[k + 2], v[k + 3])}, v2u{T::pair(v[k + 4], v[k + 5]), T::pair(v[k + 6], v[k + 7])});
            const int c = col + 2 * k + 8 * hf;
            if (!inside) continue;
            if (c + 8 <= width) store16(p + at, 2 * c, w);
            else each<8>([&](auto e) { if (c + e < width) p[at + c + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1))); });
        }
    }
    static __device__ __forceinline__ void load_codes(const int8_t *p, int64_t at, int col, int width, bool inside, int hf, float scale, float (&v)[16])
    {
        const int c = col + 16 * hf;
        v4u w = {0, 0, 0, 0};
        if (inside) {
            if (c + 16 <= width) w = load16(p + at, c);
            else each<16>([&](auto e) { if (c + e < width) w[e >> 2] |= (uint32_t)(uint8_t)p[at + c + e] << (8 * (e & 3)); });
        }
        w = part_codes(w);
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = (float)(int8_t)(w[k >> 2] >> (8 * (k & 3))) * scale;
    }
    static __device__ __forceinline__ void store_codes(int8_t *p, int64_t at, int col, int width, bool inside, int hf, const Coder &coder, const float (&v)[16])
    {
        v4u w;
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = four(coder.code(v[4 * q]), coder.code(v[4 * q + 1]), coder.code(v[4 * q + 2]), coder.code(v[4 * q + 3]));
        w = join_codes(w);
        const int c = col + 16 * hf;
        if (!inside) return;
        if (c + 16 <= width) store16(p + at, c, w);
        else each<16>([&](auto e) { if (c + e < width) p[at + c + e] = (int8_t)(w[e >> 2] >> (8 * (e & 3))); });
    }
    static __device__ __forceinline__ uint32_t top(int col, int width, int hf, const float (&v)[16])
    {
        uint32_t t = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (col + 8 * (k >> 2) + 4 * hf + (k & 3) < width) t = max(t, magnitude(v[k]));
        return t;
    }
};
__device__ __forceinline__ uint32_t halves_top(uint32_t v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(s[0], s[1]);
}

constexpr int64_t kMostOutputs = 1 << 20;
inline size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

// How many parts to cut a contraction of `steps` steps into, so that the longest share of `room` workgroups is shortest: a tile costs its steps and
// about `kTileCost` more (the first copies' latency, its results' way out), and each part but a lone one is read again by a launch of its own.
inline int best_parts(int64_t tiles, int steps, int room, int most)
{
    constexpr int kTileCost = 5;
    int best = 1;
    double least = 0;
    for (int p = 1; p <= most && p <= steps; ++p) {
        const int64_t rounds = (tiles * p + room - 1) / room;
        const double cost = (double)rounds * ((steps + p - 1) / p + kTileCost) + (p > 1 ? 8 + 0.5 * p : 0);
        if (p == 1 || cost < least) {
            least = cost;
            best = p;
        }
    }
    return best;
}

}  // namespace qb
