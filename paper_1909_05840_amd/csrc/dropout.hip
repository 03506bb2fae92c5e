// Dropout with the residual added, and its backward; the mask is drawn again instead of stored.
//
//   Y[i] = X[i] * m[i] (+ residual[i]),  dX[i] = dY[i] * m[i],  m[i] = 0 or 65536 / (65536 - t)
//
// Bound by memory: three tensors of traffic forward, two backward.  A counter's four draws cost about 60 instructions, 15 a
// value, against the 2 to 12 bytes that it moves.  32768 x 1024 bfloat16: 35 us with the residual (5.8 TB/s), 25 us without (5.4).
#include "qb_tiles.hpp"
#include <cmath>

namespace qb {
namespace {

constexpr int kAtOnce = 4;  // chunks of sixteen bytes that a thread has under way, so that the loads' latency is hidden

struct DropArgs {
    const void *X, *residual;
    void *Y;
    int64_t n;
    const int64_t *seed;
    uint32_t threshold;
    float scale;
};

// sixteen bytes at any address (the load unit takes them with the same instruction, aligned or not)
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

// Sixteen bytes are a chunk: four values and one counter in 32 bits, eight values and two counters in 16.
template <int TYPE>
struct Chunk {
    static constexpr int kSize = TYPE == QB_TYPE_FP32 ? 4 : 2, kValues = 16 / kSize, kCounters = kValues / 4;
    typedef std::conditional_t<TYPE == QB_TYPE_BF16, Bf16, Fp16> T;
    float v[kValues];
    __device__ __forceinline__ explicit Chunk(v4u w)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == QB_TYPE_FP32) {
                v[i] = __uint_as_float(w[i]);
            } else {
                v[2 * i] = T::lo(w[i]);
                v[2 * i + 1] = T::hi(w[i]);
            }
        }
    }
    __device__ __forceinline__ v4u words() const
    {
        v4u w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == QB_TYPE_FP32) w[i] = __float_as_uint(v[i]);
            else w[i] = T::pair(v[2 * i], v[2 * i + 1]);
        }
        return w;
    }
    __device__ __forceinline__ void drop(const Threefry &bits, int64_t chunk, uint32_t threshold, float scale)
    {
#pragma unroll
        for (int c = 0; c < kCounters; ++c) {
            const uint64_t counter = (uint64_t)chunk * kCounters + c;
            const v2u d = bits.draws((uint32_t)counter, (uint32_t)(counter >> 32));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool keep = j & 1 ? kept_high(d[j >> 1], threshold) : kept_low(d[j >> 1], threshold);
                v[4 * c + j] = keep ? v[4 * c + j] * scale : 0.0f;
            }
        }
    }
    __device__ __forceinline__ void add(const Chunk &x)
    {
#pragma unroll
        for (int i = 0; i < kValues; ++i) v[i] += x.v[i];
    }
};
// the last values of a tensor, fewer than a chunk
template <int TYPE>
__device__ v4u load_some(const void *p, int64_t byte, int values)
{
    v4u w = {0, 0, 0, 0};
    for (int i = 0; i < values; ++i) {
        if constexpr (TYPE == QB_TYPE_FP32) w[i] = reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(p) + byte)[i];
        else w[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(static_cast<const uint8_t *>(p) + byte)[i] << (16 * (i & 1));
    }
    return w;
}
template <int TYPE>
__device__ void store_some(void *p, int64_t byte, v4u w, int values)
{
    for (int i = 0; i < values; ++i) {
        if constexpr (TYPE == QB_TYPE_FP32) reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(p) + byte)[i] = w[i];
        else reinterpret_cast<uint16_t *>(static_cast<uint8_t *>(p) + byte)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}

template <int TYPE, bool RESIDUAL>
__global__ __launch_bounds__(256) void dropout_kernel(const DropArgs a)
{
    typedef Chunk<TYPE> C;
    const Threefry bits((uint64_t)*a.seed);
    const int64_t whole = a.n / C::kValues, step = (int64_t)gridDim.x * (256 * kAtOnce);
    for (int64_t first = (int64_t)blockIdx.x * (256 * kAtOnce) + threadIdx.x; first < whole; first += step) {
        // all loads of a round before the bits of its first chunk
        v4u x[kAtOnce], r[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t c = min(first + u * 256, whole - 1);
            x[u] = load16(a.X, 16 * c);
            if constexpr (RESIDUAL) r[u] = load16(a.residual, 16 * c);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t c = first + u * 256;
            if (c >= whole) break;
            C v(x[u]);
            v.drop(bits, c, a.threshold, a.scale);
            if constexpr (RESIDUAL) v.add(C(r[u]));
            store16(a.Y, 16 * c, v.words());
        }
    }
    const int rest = (int)(a.n - whole * C::kValues);
    if (rest > 0 && blockIdx.x == gridDim.x - 1 && threadIdx.x == 255) {
        C v(load_some<TYPE>(a.X, 16 * whole, rest));
        v.drop(bits, whole, a.threshold, a.scale);
        if constexpr (RESIDUAL) v.add(C(load_some<TYPE>(a.residual, 16 * whole, rest)));
        store_some<TYPE>(a.Y, 16 * whole, v.words(), rest);
    }
}

template <bool RESIDUAL>
qb_status launch(const DropArgs &a, int type, hipStream_t stream)
{
    const int64_t chunks = a.n / (type == QB_TYPE_FP32 ? 4 : 8), need = (chunks + 256 * kAtOnce - 1) / (256 * kAtOnce);
    const int blocks = (int)(need < 1 ? 1 : need < 8192 ? need : 8192);
    if (type == QB_TYPE_BF16) dropout_kernel<QB_TYPE_BF16, RESIDUAL><<<blocks, 256, 0, stream>>>(a);
    else if (type == QB_TYPE_FP16) dropout_kernel<QB_TYPE_FP16, RESIDUAL><<<blocks, 256, 0, stream>>>(a);
    else dropout_kernel<QB_TYPE_FP32, RESIDUAL><<<blocks, 256, 0, stream>>>(a);
    return launch_status();
}

qb_status dropout(const void *X, const void *residual, int64_t n, int type, float p, const int64_t *seed, void *Y, void *stream)
{
    if (n < 0) return QB_ERR_SHAPE;
    if (!(p >= 0.0f && p < 1.0f) || type < QB_TYPE_BF16 || type > QB_TYPE_FP32) return QB_ERR_VALUE;
    if (n == 0) return QB_OK;
    if (!X || !Y || !seed) return QB_ERR_NULL;
    const uintptr_t mask = type == QB_TYPE_FP32 ? 3 : 1;
    if (((reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(Y) | reinterpret_cast<uintptr_t>(residual)) & mask) || (reinterpret_cast<uintptr_t>(seed) & 7)) return QB_ERR_VALUE;
    const uint32_t t = drop_threshold(p);
    const DropArgs a = {X, residual, Y, n, seed, t, (float)(65536.0 / (65536 - t))};
    return residual ? launch<true>(a, type, static_cast<hipStream_t>(stream)) : launch<false>(a, type, static_cast<hipStream_t>(stream));
}

}  // namespace
}  // namespace qb

extern "C" qb_status qb_dropout_fwd(const void *X, const void *residual, int64_t n, int type, float p, const int64_t *seed,
                                    void *Y, void *stream)
{
    return qb::dropout(X, residual, n, type, p, seed, Y, stream);
}

extern "C" qb_status qb_dropout_bwd(const void *dY, int64_t n, int type, float p, const int64_t *seed, void *dX, void *stream)
{
    return qb::dropout(dY, nullptr, n, type, p, seed, dX, stream);
}
