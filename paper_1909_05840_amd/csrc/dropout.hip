// Dropout with the residual added, and its backward; the mask is drawn again instead of stored.
//
//   Y[i] = X[i] * m[i] (+ residual[i]),  dX[i] = dY[i] * m[i],  m[i] = 0 or 65536 / (65536 - t)
//
// Bound by memory: three tensors of traffic forward, two backward.  A counter's four draws cost about 60 instructions, 15 a
// value, against the 2 to 12 bytes that it moves.
#include "qb_tiles.hpp"
#include <cmath>

namespace qb {
namespace {

struct DropArgs {
    const void *X, *residual;
    void *Y;
    int64_t n;
    const int64_t *seed;
    uint32_t threshold;
    float scale;
};

// one value of a type as a float, and back (rounded to nearest even)
template <int TYPE>
__device__ __forceinline__ float value(const void *p, int64_t i)
{
    if constexpr (TYPE == QB_TYPE_FP32) return static_cast<const float *>(p)[i];
    const uint32_t w = static_cast<const uint16_t *>(p)[i];
    return TYPE == QB_TYPE_BF16 ? Bf16::lo(w) : Fp16::lo(w);
}
template <int TYPE>
__device__ __forceinline__ void put(void *p, int64_t i, float v)
{
    if constexpr (TYPE == QB_TYPE_FP32) static_cast<float *>(p)[i] = v;
    else static_cast<uint16_t *>(p)[i] = (uint16_t)(TYPE == QB_TYPE_BF16 ? Bf16::pair(v, v) : Fp16::pair(v, v));
}

template <int TYPE, bool RESIDUAL>
__global__ __launch_bounds__(256) void dropout_kernel(const DropArgs a)
{
    const Threefry bits((uint64_t)*a.seed);
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; 4 * c < a.n; c += step) {
        const v2u d = bits.draws((uint32_t)c, (uint32_t)((uint64_t)c >> 32));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (4 * c + j >= a.n) break;
            const bool keep = j & 1 ? kept_high(d[j >> 1], a.threshold) : kept_low(d[j >> 1], a.threshold);
            float v = keep ? value<TYPE>(a.X, 4 * c + j) * a.scale : 0.0f;
            if constexpr (RESIDUAL) v += value<TYPE>(a.residual, 4 * c + j);
            put<TYPE>(a.Y, 4 * c + j, v);
        }
    }
}

template <bool RESIDUAL>
qb_status launch(const DropArgs &a, int type, hipStream_t stream)
{
    const int64_t need = (a.n + 1023) / 1024;
    const int blocks = (int)(need < 8192 ? need : 8192);
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
