// What layer norm, the 16-bit linears and the 8-bit checkpoints share: eight neighbours of a row in registers, activations with their
// derivatives, the 8-bit codes of groups of 64.
#pragma once
#include "qb_tiles.hpp"

namespace qb {

constexpr int kGroup = QB_KEEP_GROUP;
static_assert(kGroup == 64, "a group is eight lanes' values, or two blocks of a product's results");

inline bool type_ok(int type) { return type >= QB_TYPE_BF16 && type <= QB_TYPE_FP32; }
template <int TYPE>
using Half = std::conditional_t<TYPE == QB_TYPE_BF16, Bf16, Fp16>;  // (of a 16-bit type)
template <int TYPE>
constexpr int kSizeOf = TYPE == QB_TYPE_FP32 ? 4 : 2;
constexpr int64_t kMostRows = 1 << 24;    // tokens
constexpr int64_t kMostStride = 1 << 22;  // values between rows (256 rows stay within 32 bits of bytes)
inline bool stride_ok(int64_t s) { return s >= 0 && s <= kMostStride; }
inline bool misaligned(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) != 0; }
inline int size_of(int type) { return type == QB_TYPE_FP32 ? 4 : 2; }

// Eight neighbours of a row, or the last `n` of it (the others zero).  Rows may start anywhere that their type allows.
template <int TYPE>
struct Eight {
    static constexpr int kWords = TYPE == QB_TYPE_FP32 ? 8 : 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void *p, int64_t at, int n)
    {
        const uint8_t *const from = static_cast<const uint8_t *>(p) + at * kSizeOf<TYPE>;
        if (n >= 8) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const v4u x = load16(from, 4 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[i + e] = x[e];
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= n) continue;
            if constexpr (TYPE == QB_TYPE_FP32) w[i] = reinterpret_cast<const uint32_t *>(from)[i];
            else w[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(from)[i] << (16 * (i & 1));
        }
    }
    __device__ __forceinline__ void store(void *p, int64_t at, int n) const
    {
        uint8_t *const to = static_cast<uint8_t *>(p) + at * kSizeOf<TYPE>;
        if (n >= 8) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) store16(to, 4 * i, v4u{w[i], w[i + 1], w[i + 2], w[i + 3]});
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= n) continue;
            if constexpr (TYPE == QB_TYPE_FP32) reinterpret_cast<uint32_t *>(to)[i] = w[i];
            else reinterpret_cast<uint16_t *>(to)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (TYPE == QB_TYPE_FP32) {
                v[i] = __uint_as_float(w[i]);
            } else {
                v[2 * i] = Half<TYPE>::lo(w[i]);
                v[2 * i + 1] = Half<TYPE>::hi(w[i]);
            }
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (TYPE == QB_TYPE_FP32) w[i] = __float_as_uint(v[i]);
            else w[i] = Half<TYPE>::pair(v[2 * i], v[2 * i + 1]);
        }
    }
};

// ---- 8 bits: scale = max |x| / 127 in binary32, code = the whole number nearest x / scale ----------------------------

// the magnitudes' bits order as the magnitudes do, NaN above infinity, so that either reaches the scale
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

struct Coder {
    float scale, inverse;
    bool fast;  // the scale has a reciprocal
    __device__ __forceinline__ explicit Coder(uint32_t top)
    {
        scale = __fdiv_rn(__uint_as_float(top), 127.0f);
        fast = scale >= 1.0e-30f && scale <= 1.0e37f;
        inverse = fast ? __builtin_amdgcn_rcpf(scale) : 0.0f;
    }
    // N codes, four to a word.  Adding 1.5 * 2^23 leaves the nearest whole number in the low bits of a sum that is rounded once; the reciprocal is within one unit in
    // the last place, so that x inverse is within 127.5 * 2^-23 = 1.6e-5 of the true quotient.  Where one of the quotients is closer than 2e-5 to half a step, all of the lane's are taken again, with care.
    template <int N>
    __device__ __forceinline__ void codes(const float (&x)[N], uint32_t (&w)[N / 4]) const
    {
        constexpr float kWhole = 12582912.0f;
        float far = fast ? 0.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            float k[4], d[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                k[e] = __builtin_fmaf(x[i + e], inverse, kWhole);
                d[e] = fabsf(__builtin_fmaf(x[i + e], inverse, kWhole - k[e]));
            }
            far = fmaxf(fmaxf(far, fmaxf(d[0], d[1])), fmaxf(d[2], d[3]));
            const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(k[1]), __float_as_uint(k[0]), 0x0C0C0400), hi = __builtin_amdgcn_perm(__float_as_uint(k[3]), __float_as_uint(k[2]), 0x04000C0C);
            w[i / 4] = lo | hi;
        }
        if (far <= 0.49998f) return;
#pragma unroll
        for (int i = 0; i < N; i += 4) w[i / 4] = four(careful(x[i]), careful(x[i + 1]), careful(x[i + 2]), careful(x[i + 3]));
    }
    // The same without the second look, for values that are themselves results of rounded arithmetic: a quotient closer than 2^-16 to half a step may go either way.
    // Groups whose scale has no reciprocal read back as zeros (magnitudes below 1.3e-28), or as NaN (infinities, NaN).
    __device__ __forceinline__ float quick_scale() const { return fast ? scale : scale * 0.0f; }
    template <int N>
    __device__ __forceinline__ void quick(const float (&x)[N], uint32_t (&w)[N / 4]) const
    {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            uint32_t k[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) k[e] = __float_as_uint(__builtin_fmaf(x[i + e], inverse, 12582912.0f));
            w[i / 4] = __builtin_amdgcn_perm(k[1], k[0], 0x0C0C0400) | __builtin_amdgcn_perm(k[3], k[2], 0x04000C0C);
        }
    }
    static __device__ __forceinline__ uint32_t four(int a, int b, int c, int d) { return (a & 0xFF) | (b & 0xFF) << 8 | (c & 0xFF) << 16 | (uint32_t)d << 24; }
    // next to half a step the sign of |x| - (k + 1/2) scale decides, which one fused multiply and add gives without error (of small scales both are
    // taken larger: half a subnormal step would be rounded to nothing)
    __device__ __forceinline__ int careful(float x) const
    {
        if (!(scale > 0.0f && scale < __builtin_inff())) return 0;
        const float up = scale < 1.0e-30f ? 0x1p60f : 1.0f, s = scale * up, m = fabsf(x) * up, t = fminf(__fdiv_rn(m, s), 127.0f), low = floorf(t);  // (subnormal scales are far from max |x| / 127)
        const float d = __builtin_fmaf(-(low + 0.5f), s, m);
        const int k = (int)low + (low < 127.0f && (d > 0.0f || (d == 0.0f && ((int)low & 1) != 0)) ? 1 : 0);
        return x < 0.0f ? -k : k;
    }
};

// the largest of eight neighbouring lanes, in each of them
__device__ __forceinline__ uint32_t max8(uint32_t v)
{
    const auto other = [&](auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true); };
    v = max(v, other(std::integral_constant<int, 0xB1>()));   // lane ^ 1
    v = max(v, other(std::integral_constant<int, 0x4E>()));   // lane ^ 2
    return max(v, other(std::integral_constant<int, 0x141>()));  // the other four of eight
}
// Codes of a group that lies in eight neighbouring lanes, eight values each, whole groups: `chunk` counts the eights.
__device__ __forceinline__ void keep8(const float (&v)[8], int8_t *codes, float *scales, int64_t chunk)
{
    uint32_t top = 0, q[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, magnitude(v[i]));
    const Coder c(max8(top));
    c.codes(v, q);
    if ((chunk & 7) == 0) scales[chunk >> 3] = c.scale;
    struct __attribute__((packed)) Loose { v2u v; };
    reinterpret_cast<Loose *>(codes)[chunk].v = v2u{q[0], q[1]};
}
__device__ __forceinline__ void kept8(float (&v)[8], const int8_t *codes, const float *scales, int64_t chunk)
{
    struct __attribute__((packed)) Loose { v2u v; };
    const v2u w = reinterpret_cast<const Loose *>(codes)[chunk].v;
    const float scale = scales[chunk >> 3];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(w[i >> 2] >> (8 * (i & 3))) * scale;
}
// The same of a row of any width: eight values from column `col` on, which may be past the end.
template <bool EXACT>
__device__ __forceinline__ void keep8(const float (&v)[8], int8_t *codes, float *scales, int64_t row, int width, int col)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < width) top = max(top, magnitude(v[i]));
    const Coder c(max8(top));
    if (col >= width) return;
    if ((col & (kGroup - 1)) == 0) scales[row * ((width + kGroup - 1) / kGroup) + col / kGroup] = EXACT ? c.scale : c.quick_scale();
    uint32_t q[2];
    if constexpr (EXACT) c.codes(v, q);
    else c.quick(v, q);
    const v2u w = {q[0], q[1]};
    int8_t *const to = codes + row * width + col;
    if (col + 8 <= width) {
        struct __attribute__((packed)) Loose { v2u v; };
        reinterpret_cast<Loose *>(to)->v = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < width) to[i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}
// and back: eight values of a row
__device__ __forceinline__ void kept8(float (&v)[8], const int8_t *codes, const float *scales, int64_t row, int width, int col)
{
    const int n = width - col;
    v2u w = {0, 0};
    float scale = 0.0f;
    if (n > 0) {
        const int8_t *const from = codes + row * width + col;
        scale = scales[row * ((width + kGroup - 1) / kGroup) + col / kGroup];
        if (n >= 8) {
            struct __attribute__((packed)) Loose { v2u v; };
            w = reinterpret_cast<const Loose *>(from)->v;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) w[i >> 2] |= (uint32_t)(uint8_t)from[i] << (8 * (i & 3));
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(w[i >> 2] >> (8 * (i & 3))) * scale;
}

// ---- activations ------------------------------------------------------------------------------------------------------

// The normal distribution's upper tail at x >= 0 is a power of two of a polynomial of degree seven: fitted to the tail's logarithm on [0, 7] for the least largest
// error, 1.4e-5 of the tail itself with the evaluation's roundings (below 2^-16).  Up to there, 7, GELU and the tail's share of its derivative are relative to themselves below the 16-bit types' half
// steps, 2^-9 and 2^-12, also where they are small.  Further out the polynomial falls faster than the tail: by 3.4e-4 of it at 7.5, 0.2% at 8, 0.6% at 8.5, 1.8% at 9, 9% at 10,
// most of it from 12 on, and from 16 on it is zero; GELU is -9e-12 at -7, zero in float16 from -6 on, and -5e-15 at -8, where bf16 begins to tell the difference.  (Degree eight: 1.0e-5 up to
// 7, or 4e-5 up to 6 and 6e-4 up to 13.  An instruction for each of 16384 x 4096 results takes 8 us when the matrix cores wait for it.)
constexpr float kTailEnd = 16.0f;
__device__ __forceinline__ float normal_tail(float x)
{
    float p = __builtin_fmaf(-1.58821490003902e-06f, x, 5.61533379368484e-05f);
    p = __builtin_fmaf(p, x, -0.0008832153398543596f);
    p = __builtin_fmaf(p, x, 0.008303219452500343f);
    p = __builtin_fmaf(p, x, -0.053501322865486145f);
    p = __builtin_fmaf(p, x, -0.4589643180370331f);
    p = __builtin_fmaf(p, x, -1.1510356664657593f);
    return __builtin_amdgcn_exp2f(__builtin_fmaf(p, x, -1.0000139474868774f));
}
__device__ __forceinline__ float hyperbolic_tangent(float z)
{
    if (fabsf(z) < 0.25f) {  // (the quotient's numerator would cancel; the next term of the series is 2.1e-9 at most)
        const float s = z * z;
        float p = __builtin_fmaf(s, 62.0f / 2835.0f, -17.0f / 315.0f);
        p = __builtin_fmaf(p, s, 2.0f / 15.0f);
        p = __builtin_fmaf(p, s, -1.0f / 3.0f);
        return __builtin_fmaf(p * s, z, z);
    }
    const float e = __builtin_amdgcn_exp2f(fabsf(z) * -2.88539008178f);
    return copysignf((1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e), z);
}
inline bool act_ok(int act) { return act >= QB_ACT_NONE && act <= QB_ACT_TANH; }

// (`act` is the same for all threads of a launch)
template <int N>
__device__ __forceinline__ void activate(int act, float (&z)[N])
{
    if (act == QB_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) {  // z - z tail, or below zero z tail
            const float x = fminf(fabsf(z[i]), kTailEnd);
            z[i] = __builtin_fmaf(-x, normal_tail(x), __builtin_elementwise_maximum(z[i], 0.0f));
        }
    } else if (act == QB_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i];
    } else if (act == QB_ACT_TANH) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = hyperbolic_tangent(z[i]);
    }
}
// g times the derivative at z
template <int N>
__device__ __forceinline__ void slope(int act, const float (&z)[N], float (&g)[N])
{
    if (act == QB_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float tail = normal_tail(fminf(fabsf(z[i]), kTailEnd)), share = z[i] < 0.0f ? tail : 1.0f - tail;  // (left of zero the tail itself: 1 / 2 - (1 / 2 - tail) would lose it)
            g[i] *= __builtin_fmaf(z[i] * __builtin_amdgcn_exp2f(z[i] * z[i] * -0.72134752044f), 0.3989422804f, share);
        }
    } else if (act == QB_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = z[i] > 0.0f ? g[i] : 0.0f;
    } else if (act == QB_ACT_TANH) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float e = __builtin_amdgcn_exp2f(fabsf(z[i]) * -2.88539008178f), r = __builtin_amdgcn_rcpf(1.0f + e);
            g[i] *= 4.0f * e * r * r;
        }
    }
}

// the sum over a wavefront whose lanes are all active, in every lane
__device__ __forceinline__ float wave_add(float v)
{
    const auto step = [&](auto ctrl, auto rows) { v += __int_as_float(dpp<decltype(ctrl)::value, decltype(rows)::value>(0, __float_as_int(v))); };
    step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());  // row_shr:1, 2, 4, 8
    step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());  // row_bcast:15, 31
    step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

}  // namespace qb
