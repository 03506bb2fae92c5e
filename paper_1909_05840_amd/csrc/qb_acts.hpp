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
        inverse = fast ? __fdiv_rn(1.0f, scale) : 0.0f;
    }
    // The product with the rounded reciprocal is within 127.5 * 3 * 2^-24 = 2.3e-5 of the true quotient; closer than 1e-4 to half a step the sign of
    // x - (k + 1/2) scale decides, which one fused multiply and add gives without error.
    __device__ __forceinline__ int code(float x) const
    {
        const float m = fabsf(x), t = fast ? m * inverse : __fdiv_rn(m, scale);
        float k = rintf(t);
        if (!(fabsf(t - k) <= 0.4999f)) k = near_half(m, t);
        k = fminf(k, 127.0f);  // (subnormal scales are far from max |x| / 127)
        return (int)(x < 0.0f ? -k : k);
    }
    __device__ __forceinline__ float near_half(float m, float t) const
    {
        if (!(scale > 0.0f && scale < __builtin_inff())) return 0.0f;
        const float low = floorf(t), d = __builtin_fmaf(-(low + 0.5f), scale, m);
        const bool odd = ((int)low & 1) != 0;
        return d > 0.0f || (d == 0.0f && odd) ? low + 1.0f : low;
    }
};
__device__ __forceinline__ uint32_t four(int a, int b, int c, int d) { return (a & 0xFF) | (b & 0xFF) << 8 | (c & 0xFF) << 16 | (uint32_t)d << 24; }

// the largest of eight neighbouring lanes, in each of them
__device__ __forceinline__ uint32_t max8(uint32_t v)
{
    const auto other = [&](auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true); };
    v = max(v, other(std::integral_constant<int, 0xB1>()));   // lane ^ 1
    v = max(v, other(std::integral_constant<int, 0x4E>()));   // lane ^ 2
    return max(v, other(std::integral_constant<int, 0x141>()));  // the other four of eight
}
// Codes of a group that lies in eight neighbouring lanes, eight values each; `n` of a lane's are inside the row.
__device__ __forceinline__ void keep8(const float (&v)[8], int8_t *codes, float *scales, int64_t row, int width, int col)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < width) top = max(top, magnitude(v[i]));
    const Coder c(max8(top));
    if (col >= width) return;
    if ((col & (kGroup - 1)) == 0) scales[row * ((width + kGroup - 1) / kGroup) + col / kGroup] = c.scale;
    const v2u w = {four(c.code(v[0]), c.code(v[1]), c.code(v[2]), c.code(v[3])), four(c.code(v[4]), c.code(v[5]), c.code(v[6]), c.code(v[7]))};
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

// The normal distribution's upper tail at |z| = exp(-z^2 / 2) M(|z|).  M falls like 1 / |z|; as a polynomial in u = 1 / (1 + 0.376 |z|) without a
// constant term (the form of C. Hastings, "Approximations for Digital Computers", 1955; coefficients: least largest relative error, fitted for |z| <= 14)
// it is within 3e-5 of itself, 2^-15, so that the share and GELU are below the 16-bit types' rounding steps, their tails included.
struct Normal {
    float bell, share;  // exp(-z^2 / 2); the distribution below z
    __device__ __forceinline__ explicit Normal(float z)
    {
        const float u = __builtin_amdgcn_rcpf(__builtin_fmaf(0.376f, fabsf(z), 1.0f));
        bell = __builtin_amdgcn_exp2f(z * z * -0.72134752044f);
        float m = __builtin_fmaf(-0.0908565548694444f, u, 0.19874278238977716f);
        m = __builtin_fmaf(m, u, 0.08471268883902303f);
        m = __builtin_fmaf(m, u, 0.15791362939227915f);
        m = __builtin_fmaf(m, u, 0.1494776113147777f);
        const float tail = m * u * bell;
        share = z < 0.0f ? tail : 1.0f - tail;
    }
};
__device__ __forceinline__ float hyperbolic_tangent(float z)
{
    if (fabsf(z) < 0.25f) {  // (the quotient's numerator would cancel; the next term of the series is below 2e-9)
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
        for (int i = 0; i < N; ++i) z[i] *= Normal(z[i]).share;
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
            const Normal n(z[i]);
            g[i] *= __builtin_fmaf(z[i] * n.bell, 0.3989422804f, n.share);
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
