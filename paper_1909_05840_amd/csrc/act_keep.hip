// Activations in 8 bits, and back.
//
//   scale = max |x| of 64 neighbours of a row / 127;  code = x / scale to the nearest whole number, half to even;  code * scale
//
// Bound by memory: a group is eight lanes with eight values each, all loads of a thread under way before the first is used.  16384 x 4096 in bf16 45 us and back 30, 41 each at the
// rate of a large copy (codes just written are partly in the last cache); 64 where rows lie apart, whose chunks need a division each.
#include "qb_acts.hpp"
#include <algorithm>

namespace qb {
namespace {

constexpr int kAtOnce = 4;  // chunks of eight values that a thread has under way

struct KeepArgs {
    const void *X;
    void *Y;
    int64_t x_row, T;
    int W, groups;  // groups of a row
    int8_t *codes;
    float *scales;
};

// Chunk c of eight values: group c / 8 of all rows' groups, in order; the lanes of a group are neighbours.  FLAT: rows of whole groups, side by side, need no row or
// column (and no division).
template <int TYPE, bool KEEP, bool FLAT>
__global__ __launch_bounds__(256) void act_keep_kernel(const KeepArgs a)
{
    const int64_t chunks = a.T * a.groups * 8, step = (int64_t)gridDim.x * (256 * kAtOnce);
    for (int64_t first = (int64_t)blockIdx.x * (256 * kAtOnce) + threadIdx.x; first < chunks; first += step) {
        int64_t row[kAtOnce], at[kAtOnce];
        int col[kAtOnce];
        Eight<TYPE> x[kAtOnce];
        float v[kAtOnce][8];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t c = min(first + u * 256, chunks - 8 + (threadIdx.x & 7));  // (past the end: the last group again)
            if constexpr (FLAT) {
                at[u] = c;
                if constexpr (KEEP) x[u].load(a.X, c * 8, 8);
                else kept8(v[u], a.codes, a.scales, c);
            } else {
                row[u] = (c >> 3) / a.groups;
                col[u] = (int)(c - row[u] * (a.groups * 8)) * 8;
                if constexpr (KEEP) x[u].load(a.X, row[u] * a.x_row + col[u], a.W - col[u]);
                else kept8(v[u], a.codes, a.scales, row[u], a.W, col[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if constexpr (KEEP) {
                x[u].get(v[u]);
                if constexpr (FLAT) keep8(v[u], a.codes, a.scales, at[u]);
                else keep8<true>(v[u], a.codes, a.scales, row[u], a.W, col[u]);
            } else {
                x[u].set(v[u]);
                if constexpr (FLAT) x[u].store(a.Y, at[u] * 8, 8);
                else x[u].store(a.Y, row[u] * a.W + col[u], a.W - col[u]);
            }
        }
    }
}

template <bool KEEP>
qb_status launch(const KeepArgs &a, int type, hipStream_t st)
{
    const int64_t need = (a.T * a.groups * 8 + 256 * kAtOnce - 1) / (256 * kAtOnce);
    const int blocks = (int)std::min<int64_t>(need, 8192);
    const auto go = [&](auto t) {
        if (a.W % kGroup == 0 && a.x_row == a.W) act_keep_kernel<decltype(t)::value, KEEP, true><<<blocks, 256, 0, st>>>(a);
        else act_keep_kernel<decltype(t)::value, KEEP, false><<<blocks, 256, 0, st>>>(a);
    };
    if (type == QB_TYPE_BF16) go(std::integral_constant<int, QB_TYPE_BF16>{});
    else if (type == QB_TYPE_FP16) go(std::integral_constant<int, QB_TYPE_FP16>{});
    else go(std::integral_constant<int, QB_TYPE_FP32>{});
    return launch_status();
}

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" qb_status qb_checkpoint_act(const void *X, int64_t x_row, int type, int64_t T, int64_t W, int8_t *codes, float *scales, void *stream)
{
    if (T < 0 || T > kMostRows || W < 1 || W > QB_MAX_K) return QB_ERR_SHAPE;
    if (!type_ok(type) || !stride_ok(x_row)) return QB_ERR_VALUE;
    if (T == 0) return QB_OK;
    if (!X || !codes || !scales) return QB_ERR_NULL;
    if (misaligned(X, size_of(type)) || misaligned(scales, 4)) return QB_ERR_VALUE;
    const KeepArgs a = {X, nullptr, x_row, T, (int)W, (int)((W + kGroup - 1) / kGroup), codes, scales};
    return launch<true>(a, type, static_cast<hipStream_t>(stream));
}

extern "C" qb_status qb_restore_act(const int8_t *codes, const float *scales, int64_t T, int64_t W, int type, void *X, void *stream)
{
    if (T < 0 || T > kMostRows || W < 1 || W > QB_MAX_K) return QB_ERR_SHAPE;
    if (!type_ok(type)) return QB_ERR_VALUE;
    if (T == 0) return QB_OK;
    if (!X || !codes || !scales) return QB_ERR_NULL;
    if (misaligned(X, size_of(type)) || misaligned(scales, 4)) return QB_ERR_VALUE;
    const KeepArgs a = {nullptr, X, W, T, (int)W, (int)((W + kGroup - 1) / kGroup), const_cast<int8_t *>(codes), const_cast<float *>(scales)};
    return launch<false>(a, type, static_cast<hipStream_t>(stream));
}
