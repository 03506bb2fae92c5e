// What the kernels of attention, of the vocabulary loss and of the other 16-bit operators share: the 16-bit types with their matrix instructions, tiles
// of rows in LDS, copies into them, the generator of dropout's random bits.
#pragma once
#include "qb_common.hpp"

namespace qb {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));

// A 16-bit type: eight values as a matrix operand, two floats rounded to nearest even (the first in the low half), and back.
// kNarrow: the exponents of binary32 do not fit.
struct Bf16 {
    static constexpr bool kNarrow = false;
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ v16f mma32(v8s a, v8s b, v16f c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ v4f mma16(v8s a, v8s b, v4f c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi)
    {
        typedef __bf16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{lo, hi}, v2));
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
};
struct Fp16 {
    static constexpr bool kNarrow = true;
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ v16f mma32(v8s a, v8s b, v16f c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ v4f mma16(v8s a, v8s b, v4f c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{lo, hi}, v2)); }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(v2, w)[0]; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(v2, w)[1]; }
};

// f(0), .., f(N - 1) with the number as a constant (vector elements whose number is one only after unrolling end up in memory)
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(const F &f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
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

template <int N>
__device__ __forceinline__ void wait_copies()  // until at most N of this wavefront's vector memory operations are under way
{
    static_assert(N >= 0 && N < 64, "the counter has six bits");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | 0x0070 | 0x0F00);
}
// Every wavefront's LDS reads so far have returned and are not moved below, nor later ones above.
__device__ __forceinline__ void barrier()
{
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// sixteen bytes per lane from memory to LDS by the load unit: lane l's land at lds + 16 * l
__device__ __forceinline__ void copy16(const void *from, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(lds) : "memory", "m0");
}
// sixteen with the address as a base that the wavefront shares and an offset in bytes (the base is moved into registers of the block's
// own by a scalar instruction: a vector memory instruction may read what a VALU instruction wrote five wait states later only)
__device__ __forceinline__ void copy16(const void *base, uint32_t offset, uint32_t lds)
{
    const uint64_t at = reinterpret_cast<uint64_t>(base);  // (a quotient of uniform values lies in a vector register)
    const uint64_t uniform = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)) << 32;
    uint64_t own;
    asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 %0, %1\n\tglobal_load_lds_dwordx4 %2, %0" : "=&s"(own) : "s"(uniform), "v"(offset), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)p; }

// A tile of rows of D 16-bit values in LDS, rows dense.  The 16-byte chunks of a row are XORed with a key of the row such
// that both ways of reading meet different banks: sixteen consecutive rows at one chunk (an operand whose contraction runs
// along the row), and four consecutive rows at four neighbouring chunks (a turned operand, below).
template <int D>
struct Rows {
    static_assert(D == 64 || D == 128, "rows of 128 or 256 bytes");
    static constexpr int kBytes = 2 * D, kChunks = D / 8, kPerCopy = 1024 / kBytes;  // rows that one wavefront's copy fills
    static __device__ __forceinline__ int key(int row)
    {
        if constexpr (D == 64) return ((row >> 3) & 1) | ((row >> 1) & 2) | ((row << 1) & 4);
        else return ((row << 2) & 12) | ((row >> 2) & 3);
    }
    static __device__ __forceinline__ uint32_t at(int row, int chunk) { return (uint32_t)(row * kBytes + ((chunk ^ key(row)) << 4)); }
    // which row of a copy's rows, and which chunk of the row in memory, the lane fetches (row0: first row of the copy)
    static __device__ __forceinline__ int copy_row(int lane) { return lane / kChunks; }
    static __device__ __forceinline__ int copy_chunk(int row, int lane) { return (lane % kChunks) ^ key(row); }
};

// Operands out of such tiles.  The lane's places in a tile are formed once; rows further on by a multiple of 32 (16) are an offset in the instruction.
template <int D>
struct Operands {
    typedef Rows<D> R;
    uint32_t along_at[D / 16], across_at[D / 32][2];
    // base: the tiles' place in LDS
    __device__ __forceinline__ Operands(int lane, uint32_t base)
    {
#pragma unroll
        for (int c = 0; c < D / 16; ++c) along_at[c] = base + R::at(lane & 31, 2 * c + (lane >> 5));
        const int row = 4 * (lane >> 5) + ((lane >> 2) & 3), col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int part = 0; part < 2; ++part) across_at[i][part] = base + R::at(row + 8 * part, (32 * i + col) >> 3) + 2 * (col & 7);
    }
    // Contraction along the rows, 32 x 16: the lane's row (lane % 32 of `row0`), values 16 * c + 8 * (lane / 32) ..
    __device__ __forceinline__ v8s along(uint32_t tile, int row0, int c) const
    {
        return *(const __attribute__((address_space(3))) v8s *)(tile + along_at[c] + row0 * R::kBytes);
    }
    // Contraction across the rows, 32 x 16: the lane's column is 32 * i + lane % 32, its eight values are rows row0 + 4 * (lane / 32) + 0..3
    // and 8 further on: the order in which a product's result holds its rows.  The transposing read hands lane i of sixteen the
    // four rows of column i; lane i points at row i / 4, columns 4 * (i % 4)..
    __device__ __forceinline__ v8s across(uint32_t tile, int row0, int i) const
    {
        typedef __attribute__((address_space(3))) v4s *turned;
        const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned)(tile + across_at[i][0] + row0 * R::kBytes));
        const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned)(tile + across_at[i][1] + row0 * R::kBytes));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// the largest of three in one instruction (fmaxf has the compiler quieten its operands first, an instruction each)
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
// the value of the other half of the wavefront joined with the lane's own
__device__ __forceinline__ float halves_max(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float halves_sum(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// Eight bytes of each of two quads of results, one quad in the lower and one in the upper half of the wavefront, to sixteen neighbouring bytes a lane: a
// product's result holds four neighbours in a lane and the next four in the lane 32 further on.  first, second: the lane's words of
// rows 8 * q + 4 * (lane / 32) .. of quads q and q + 1; the lane is given the eight rows of quad q + (lane / 32).
__device__ __forceinline__ v4u join_halves(v2u first, v2u second)
{
    const auto a = __builtin_amdgcn_permlane32_swap(first[0], second[0], false, false), b = __builtin_amdgcn_permlane32_swap(first[1], second[1], false, false);
    return v4u{a[0], b[0], a[1], b[1]};
}

// Dropout's random bits: Threefry-2x32 with 13 rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", SC 2011; 13 rounds is the least that passed the authors' tests), key: the caller's 64-bit seed.  Additions,
// rotations and exclusive ors run at the full rate, the multiplications of the same paper's other generators at a quarter.
struct Threefry {
    uint32_t k[3];
    __device__ __forceinline__ explicit Threefry(uint64_t seed)
    {
        k[0] = (uint32_t)seed;
        k[1] = (uint32_t)(seed >> 32);
        k[2] = k[0] ^ k[1] ^ 0x1BD11BDAu;
    }
    // four 16-bit draws: word 0 low and high half, then word 1
    __device__ __forceinline__ v2u draws(uint32_t c0, uint32_t c1) const
    {
        constexpr int turn[8] = {13, 15, 26, 6, 17, 29, 16, 24};
        uint32_t x0 = c0 + k[0], x1 = c1 + k[1];
#pragma unroll
        for (int r = 0; r < 13; ++r) {
            x0 += x1;
            x1 = __builtin_amdgcn_alignbit(x1, x1, 32 - turn[r & 7]) ^ x0;
            if ((r & 3) == 3) {
                x0 += k[((r >> 2) + 1) % 3];
                x1 += k[((r >> 2) + 2) % 3] + (uint32_t)((r >> 2) + 1);
            }
        }
        return v2u{x0, x1};
    }
};
// a value is dropped where its draw is below this; p in [0, 1)
inline uint32_t drop_threshold(float p)
{
    const uint32_t t = (uint32_t)__builtin_nearbyint(p * 65536.0);
    return t < 65535u ? t : 65535u;
}
// The threshold in both places a draw can lie: the low half compares as it is, the high half with the threshold shifted up
// (the low half of the word only adds below its last bit).
__device__ __forceinline__ bool kept_low(uint32_t w, uint32_t threshold) { return (w & 0xFFFFu) >= threshold; }
__device__ __forceinline__ bool kept_high(uint32_t w, uint32_t threshold) { return w >= (threshold << 16); }

// Sixteen bytes at any address (the load unit takes them with the same instruction, aligned or not)
__device__ __forceinline__ v4u load16(const void *p, int64_t byte)
{
    struct __attribute__((packed)) Loose { v4u v; };
    return reinterpret_cast<const Loose *>(static_cast<const uint8_t *>(p) + byte)->v;
}
__device__ __forceinline__ void store16(void *p, int64_t byte, v4u v)
{
    struct __attribute__((packed)) Loose { v4u v; };
    reinterpret_cast<Loose *>(static_cast<uint8_t *>(p) + byte)->v = v;
}

// the same for what is not read again soon: it leaves the L2 first, and the operands that others read there stay
__device__ __forceinline__ void store16_stream(void *p, int64_t byte, v4u v)
{
    typedef v4u Loose __attribute__((aligned(1)));
    __builtin_nontemporal_store(v, reinterpret_cast<Loose *>(static_cast<uint8_t *>(p) + byte));
}
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace qb
