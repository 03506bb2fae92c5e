// What the 16-bit linears' forward and backward share: the stream of steps through LDS, a product's results as rows.
#pragma once
#include "qb_acts.hpp"

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

// Tiles of BM x BN results by WM x WN wavefronts, TM x TN blocks of 32 x 32 each; the contraction goes in steps of KS through a ring of stages in LDS.  An operand lies in
// LDS as it does in memory: rows of results with the contraction along them (KS values), or rows along the contraction (64 results; KS rows to a block of these), read
// turned.  KG groups of wavefronts share a step's sixteens of the contraction: a small tile's step is a chain of reads and few instructions, which more wavefronts shorten.
template <int WM_, int WN_, int TM_, int TN_, int STAGES_, int KG_ = 1>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, KG = KG_, kWaves = WM * WN * KG, kStages = STAGES_, KS = 64;
    static constexpr int BM = 32 * WM * TM, BN = 32 * WN * TN;
    static constexpr int kStage = (BM + BN) * KS * 2, kSums = (KG - 1) * BM * BN * 4, kLds = kStages * kStage + kSums;
    static constexpr int NA = BM * KS / 512 / kWaves, NB = BN * KS / 512 / kWaves;  // copies of 1024 bytes that a wavefront makes
    static_assert(NA * 512 * kWaves == BM * KS && NB * 512 * kWaves == BN * KS, "every wavefront copies the same number of times");
};

// Rows of KS values along the contraction: the chunks of sixteen bytes are XORed with a key of the row such that sixteen consecutive rows at one chunk meet different banks.
template <int KS>
struct AlongRows {
    static_assert(KS == 64, "rows of 128 bytes");
    static constexpr int kBytes = 2 * KS, kChunks = KS / 8, kPerCopy = 64 / kChunks;
    static __device__ __forceinline__ int key(int row) { return Rows<64>::key(row); }
    static __device__ __forceinline__ int row(int copy, int lane) { return copy * kPerCopy + lane / kChunks; }
    static __device__ __forceinline__ int chunk(int copy, int lane) { return (lane % kChunks) ^ key(row(copy, lane)); }
};
// Blocks of KS rows of 64 results
template <int KS>
struct AcrossRows {
    static __device__ __forceinline__ int row(int copy, int lane) { return (copy * 8 + (lane >> 3)) % KS; }
    static __device__ __forceinline__ int block(int copy) { return copy * 8 / KS; }
    static __device__ __forceinline__ int chunk(int copy, int lane) { return (lane & 7) ^ Rows<64>::key(row(copy, lane)); }
};

// Where tile `id` of a matrix of `rows` x `columns` tiles lies: bands of four rows, a band column by column, so that the 32 workgroups that an XCD has at work read
// the operands of 4 x 8 tiles, not of 1 x 32.  Bands of 1, 2, 4, 8 rows, us: 16384 x 4096 by 1024 151, 147, 140, 149; 8192 x 8192 by 8192 953, 890, 855, 862.
__device__ __forceinline__ void place_of(int id, int rows, int columns, int &row, int &column)
{
    constexpr int kBand = 4;
    const int band = id / (kBand * columns), in = id - band * kBand * columns, wide = min(kBand, rows - band * kBand);
    column = in / wide;
    row = band * kBand + in - column * wide;
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
    typedef AlongRows<S::KS> R;
    Feed<N> f;
    f.at = static_cast<const uint8_t *>(base) + first * row + (int64_t)s0 * (2 * S::KS);
    f.step = 2 * S::KS;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int copy = i * S::kWaves + wave;
        f.off[i] = (uint32_t)(min(R::row(copy, lane), rows - 1 - first) * row) + 16 * R::chunk(copy, lane);
    }
    return f;
}
// Rows along the contraction; past the last column (a multiple of eight) the last eight again.
template <typename S, int N>
__device__ __forceinline__ Feed<N> across(const void *base, int64_t row, int first, int columns, int s0, int wave, int lane)
{
    typedef AcrossRows<S::KS> R;
    Feed<N> f;
    f.at = static_cast<const uint8_t *>(base) + (int64_t)s0 * S::KS * row;
    f.step = S::KS * row;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int copy = i * S::kWaves + wave;
        f.off[i] = (uint32_t)(R::row(copy, lane) * row) + 2 * min(first + 64 * R::block(copy) + 8 * R::chunk(copy, lane), columns - 8);
    }
    return f;
}

// A lane's places in the tiles of one operand, formed once: everything else is an offset in the instruction.
template <int KS, bool ACROSS>
struct Places {
    uint32_t at[ACROSS ? 4 : KS / 16];
    // second: the wavefront's results start at the second half of a block
    // sub0: the wavefront's first sixteen of a step
    __device__ __forceinline__ Places(int lane, bool second, int sub0)
    {
        if constexpr (ACROSS) {
            typedef Rows<64> R;
            const int row = 8 * (lane >> 5) + ((lane >> 2) & 3), col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
            for (int i = 0; i < 4; ++i) at[i] = R::at(row + 4 * (i & 1), (32 * ((i >> 1) ^ (second ? 1 : 0)) + col) >> 3) + 2 * (col & 7) + sub0 * 2048;
        } else {
            typedef AlongRows<KS> R;
            const int row = lane & 31;
#pragma unroll
            for (int c = 0; c < KS / 16; ++c) at[c] = row * R::kBytes + (((2 * ((sub0 + c) % (KS / 16)) + (lane >> 5)) ^ R::key(row)) << 4);
        }
    }
    // the operand of the 32 results from `result` on, sixteen of the contraction from 16 * sub on
    __device__ __forceinline__ v8s get(uint32_t tile, int result, int sub) const
    {
        if constexpr (ACROSS) {
            typedef __attribute__((address_space(3))) v4s *turned;
            const uint32_t from = tile + (result >> 6) * (KS * 128) + sub * 2048;
            const int odd = (result >> 5) & 1;
            const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned)(from + at[2 * odd])), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned)(from + at[2 * odd + 1]));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            return *(const __attribute__((address_space(3))) v8s *)(tile + at[sub] + result * AlongRows<KS>::kBytes);
        }
    }
};

// One step's copies of an operand; its last step may have fewer than KS values of the contraction (`left`, a multiple of eight where it runs along the rows): zeros
// stand for the others.
template <typename S, bool ACROSS, int N>
__device__ __forceinline__ void copy_step(Feed<N> &f, uint32_t to, int left, int wave, int lane)
{
    if (left < S::KS) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int copy = i * S::kWaves + wave;
            const bool there = ACROSS ? AcrossRows<S::KS>::row(copy, lane) < left : 8 * AlongRows<S::KS>::chunk(copy, lane) < left;
            copy16(there ? static_cast<const void *>(f.at + f.off[i]) : &kZeros, to + copy * 1024);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) copy16(f.at, f.off[i], to + (i * S::kWaves + wave) * 1024);
    }
    f.at += f.step;
}

// acc += A B^T over a tile's steps, which lie or will lie in the stages from `stage` on.  When the operands of a step's last instructions are in registers its stage is free:
// `fetch(stage)` starts the copies of the step that comes kStages later.  `arrived(s)` waits for the wavefront's copies of step
// s, behind which those of kStages - 1 further steps may be under way for s = 0, else kStages - 2.  With SUMS, sums[j] gets what B's rows add up to over the contraction, a
// lane's share of its column of block j.
// Of 256 x 256 tiles more than two stages (5 slots of an operand each, all of LDS) measured the same: 16384 x 1024 by 4096 112.3 us and 113.6, 8192 x 8192 by 8192 867
// and 851; what bounds them is the rate at which a CU is given its operands, 46 GB/s each, and the clock, 1.7 to 2.1 GHz under this load.
template <typename T, typename S, bool A_ACROSS, bool B_ACROSS, bool SUMS>
struct Product {
    static constexpr int KS = S::KS, kSubs = KS / 16 / S::KG;  // a wavefront's sixteens of a step
    static_assert(S::TM % 2 == 0 && (S::TN % 2 == 0 || S::TN == 1), "a wavefront's results start at a block, or are half of one");
    static_assert(kSubs == 1 || kSubs % 2 == 0, "the operands' two buffers");
    const Places<KS, A_ACROSS> pa;
    const Places<KS, B_ACROSS> pb;
    uint32_t first_a, first_b;
    __device__ __forceinline__ Product(uint32_t lds, int wave, int lane)
        : pa(lane, false, wave / (S::WM * S::WN) * kSubs), pb(lane, S::TN == 1 && (wave % S::WN & 1), wave / (S::WM * S::WN) * kSubs)
    {
        const int wm = wave % (S::WM * S::WN) / S::WN, wn = wave % S::WN, result_b = B_ACROSS ? wn * S::TN * 32 & ~63 : wn * S::TN * 32;
        first_a = lds + (uint32_t)(wm * S::TM * 32) * (KS * 2);
        first_b = lds + (uint32_t)(S::BM + result_b) * (KS * 2);
    }
    template <typename FF, typename FA>
    __device__ __forceinline__ void run(v16f (&acc)[S::TM][S::TN], float (&sums)[S::TN], int steps, int &stage, const FF &fetch, const FA &arrived) const
    {
        v8s x[2][S::TM], y[2][S::TN];
        const auto load = [&](auto buffer, auto sub) {
#pragma unroll
            for (int i = 0; i < S::TM; ++i) x[buffer][i] = pa.get(first_a + stage * S::kStage, 32 * i, sub);
#pragma unroll
            for (int j = 0; j < S::TN; ++j) y[buffer][j] = pb.get(first_b + stage * S::kStage, 32 * j, sub);
        };
        const auto step = [&](int s, auto first) {  // first: the buffer that the step's first operands are in
            each<kSubs>([&](auto sub) {
                constexpr int now = (first + sub) % 2, then = 1 - now;
                if constexpr (sub + 1 < kSubs) {
                    load(std::integral_constant<int, then>(), std::integral_constant<int, sub + 1>());
                } else {
                    if (s + 1 < steps) arrived(s + 1);
                    barrier();
                    fetch(stage);
                    stage = stage == S::kStages - 1 ? 0 : stage + 1;
                    if (s + 1 < steps) load(std::integral_constant<int, then>(), std::integral_constant<int, 0>());
                }
                if constexpr (SUMS) {
#pragma unroll
                    for (int j = 0; j < S::TN; ++j) {
                        const v4u w = __builtin_bit_cast(v4u, y[now][j]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sums[j] += T::lo(w[e]) + T::hi(w[e]);
                    }
                }
#pragma unroll
                for (int i = 0; i < S::TM; ++i)
#pragma unroll
                    for (int j = 0; j < S::TN; ++j) acc[i][j] = T::mma32(x[now][i], y[now][j], acc[i][j]);
            });
        };
        arrived(0);
        barrier();
        load(std::integral_constant<int, 0>(), std::integral_constant<int, 0>());
        for (int s = 0; s < steps; ++s) {
            step(s, std::integral_constant<int, 0>());
            if constexpr (kSubs % 2 != 0)
                if (++s < steps) step(s, std::integral_constant<int, 1>());
        }
    }
};
// Waits for the wavefront's copies of step s of a tile that is all that it copies.
template <typename S>
__device__ __forceinline__ void wait_step(int s, int steps)
{
    constexpr int kStep = S::NA + S::NB;
    if (s == 0 && steps >= S::kStages) wait_copies<(S::kStages - 1) * kStep>();
    else if (steps - s >= S::kStages - 1) wait_copies<(S::kStages - 2) * kStep>();
    else wait_copies<0>();
}
// The groups' shares of a tile's sums come together in the first group; `room`: S::kSums bytes that nothing else uses.
template <typename S>
__device__ __forceinline__ void gather(v16f (&acc)[S::TM][S::TN], uint8_t *room, int wave, int lane)
{
    if constexpr (S::KG > 1) {
        constexpr int kTeam = S::WM * S::WN, kValues = S::TM * S::TN * 16;
        const int group = wave / kTeam;
        v4f *const mine = reinterpret_cast<v4f *>(room) + (wave % kTeam * (kValues / 4)) * 64 + lane;
        constexpr int kNext = kTeam * (kValues / 4) * 64;
        if (group > 0) {
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
#pragma unroll
                for (int j = 0; j < S::TN; ++j)
#pragma unroll
                    for (int k = 0; k < 16; k += 4)
                        mine[(group - 1) * kNext + ((i * S::TN + j) * 4 + k / 4) * 64] = v4f{acc[i][j][k], acc[i][j][k + 1], acc[i][j][k + 2], acc[i][j][k + 3]};
        }
        barrier();
        if (group == 0) {
#pragma unroll
            for (int g = 0; g < S::KG - 1; ++g)
#pragma unroll
                for (int i = 0; i < S::TM; ++i)
#pragma unroll
                    for (int j = 0; j < S::TN; ++j)
#pragma unroll
                        for (int k = 0; k < 16; k += 4) {
                            const v4f x = mine[g * kNext + ((i * S::TN + j) * 4 + k / 4) * 64];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][j][k + e] += x[e];
                        }
        }
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
};
// the bits of the largest magnitude of a row's 64 columns from `col` on, those of the lane's row (NaN above all)
__device__ __forceinline__ uint32_t top_of(int col, int width, int hf, const float (&v)[2][16])
{
    float t = 0.0f;
    if (col + 64 <= width) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 16; k += 2) t = max3(t, fabsf(v[u][k]), fabsf(v[u][k + 1]));
    } else {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 16; ++k) t = __builtin_elementwise_maximum(t, col + 32 * u + 8 * (k >> 2) + 4 * hf + (k & 3) < width ? fabsf(v[u][k]) : 0.0f);
    }
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(t), __float_as_uint(t), false, false);
    return max(s[0], s[1]);
}

// The same 64 columns of 32 rows through LDS of the wavefront's own (kRowsRoom bytes), sixteen rows at a time, so that eight neighbouring lanes write 128 bytes of a
// row, where a lane alone would write 16 of its own.  STREAM: what is written leaves the L2 first (only whole lines may: pieces of them would
// go to memory one by one).  16384 x 4096 results of 1024, with GELU and codes, 166 us; without STREAM 175, and slower yet where a branch of the loop chooses.
constexpr int kRowsRoom = 2048;
template <bool STREAM>
__device__ __forceinline__ void put16(void *p, int64_t byte, v4u v)
{
    if constexpr (STREAM) store16_stream(p, byte, v);
    else store16(p, byte, v);
}
template <typename T, bool STREAM>
__device__ __forceinline__ void store_rows(uint16_t *p, int row0, int rows, int col, int width, int lane, uint8_t *room, const float (&v)[2][16])
{
    const int l32 = lane & 31, hf = lane >> 5;
    v4u w[4];  // chunks of eight columns: 2 * i + hf
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float *const x = v[i >> 1] + 8 * (i & 1);
        w[i] = join_halves(v2u{T::pair(x[0], x[1]), T::pair(x[2], x[3])}, v2u{T::pair(x[4], x[5]), T::pair(x[6], x[7])});
    }
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        __builtin_amdgcn_wave_barrier();
        if ((l32 >> 4) == pass) {
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<v4u *>(room + (l32 & 15) * 128 + (((2 * i + hf) ^ (l32 & 7)) << 4)) = w[i];
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int in = 8 * r + (lane >> 3), row = row0 + 16 * pass + in, c = col + 8 * (lane & 7);
            const v4u x = *reinterpret_cast<const v4u *>(room + in * 128 + (((lane & 7) ^ (in & 7)) << 4));
            if (row >= rows) continue;
            const int64_t at = (int64_t)row * width;
            if (c + 8 <= width) put16<STREAM>(p + at, 2 * c, x);
            else each<8>([&](auto e) { if (c + e < width) p[at + c + e] = (uint16_t)(x[e >> 1] >> (16 * (e & 1))); });
        }
    }
}
template <bool STREAM>
__device__ __forceinline__ void store_code_rows(int8_t *p, int row0, int rows, int col, int width, int lane, uint8_t *room, const Coder &coder, const float (&v)[2][16])
{
    const int l32 = lane & 31, hf = lane >> 5;
    v4u w[2];  // chunks of sixteen columns: 2 * u + hf
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        uint32_t q[4];
        coder.quick(v[u], q);
        w[u] = join_codes(v4u{q[0], q[1], q[2], q[3]});
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = 0; u < 2; ++u) *reinterpret_cast<v4u *>(room + l32 * 64 + (((2 * u + hf) ^ (l32 >> 2 & 3)) << 4)) = w[u];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int in = 16 * r + (lane >> 2), row = row0 + in, c = col + 16 * (lane & 3);
        const v4u x = *reinterpret_cast<const v4u *>(room + in * 64 + (((lane & 3) ^ (in >> 2 & 3)) << 4));
        if (row >= rows) continue;
        const int64_t at = (int64_t)row * width;
        if (c + 16 <= width) put16<STREAM>(p + at, c, x);
        else each<16>([&](auto e) { if (c + e < width) p[at + c + e] = (int8_t)(x[e >> 2] >> (8 * (e & 3))); });
    }
}

// ---- rows of sums: four neighbours to a thread, a group of 64 to sixteen lanes
__device__ __forceinline__ void add_parts(const float *p, int64_t step, int parts, float (&z)[4])
{
    constexpr int kAtOnce = 8;
    for (int first = 0; first < parts; first += kAtOnce) {
        v4f x[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) x[u] = *reinterpret_cast<const v4f *>(p + min(first + u, parts - 1) * step);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (first + u < parts) {
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] += x[u][e];
            }
    }
}
template <typename T>
__device__ __forceinline__ void load4(const uint16_t *p, int64_t at, int n, float (&v)[4])
{
    if (n >= 4) {
        struct __attribute__((packed)) Loose { v2u v; };
        const v2u w = reinterpret_cast<const Loose *>(p + at)->v;
        v[0] = T::lo(w[0]); v[1] = T::hi(w[0]); v[2] = T::lo(w[1]); v[3] = T::hi(w[1]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < n ? T::lo(p[at + e]) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(uint16_t *p, int64_t at, int n, const float (&v)[4])
{
    const v2u w = {T::pair(v[0], v[1]), T::pair(v[2], v[3])};
    if (n >= 4) {
        struct __attribute__((packed)) Loose { v2u v; };
        reinterpret_cast<Loose *>(p + at)->v = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) p[at + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}
__device__ __forceinline__ void keep4(const float (&z)[4], int8_t *codes, float *scales, int64_t row, int width, int col, bool inside)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < width) top = max(top, magnitude(z[e]));
    top = max8(top);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x140, 0xF, 0xF, true));  // the other eight of sixteen
    const Coder c(top);
    uint32_t w[1];
    c.quick(z, w);
    if (!inside || col >= width) return;
    if ((col & (kGroup - 1)) == 0) scales[row * ((width + kGroup - 1) / kGroup) + col / kGroup] = c.quick_scale();
    int8_t *const to = codes + row * width + col;
    if (col + 4 <= width) {
        struct __attribute__((packed)) Loose { uint32_t v; };
        reinterpret_cast<Loose *>(to)->v = w[0];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < width) to[e] = (int8_t)(w[0] >> (8 * e));
    }
}
__device__ __forceinline__ void kept4(float (&v)[4], const int8_t *codes, const float *scales, int64_t row, int width, int col)  // (all four inside)
{
    struct __attribute__((packed)) Loose { uint32_t v; };
    const uint32_t w = reinterpret_cast<const Loose *>(codes + row * width + col)->v;
    const float scale = scales[row * ((width + kGroup - 1) / kGroup) + col / kGroup];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)(int8_t)(w >> (8 * e)) * scale;
}

// What a size of tiles costs, in microseconds: a launch with a tile's ends; a step of a lone workgroup; the KB that a CU is given in one, by all the workgroups that it has
struct Cost {
    int size, room;  // workgroups at work at once
    double ends, step, rate;
};

constexpr int64_t kMostOutputs = 1 << 20;
inline size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace qb
