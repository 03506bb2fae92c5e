// Products on the 16-bit matrix cores as the vocabulary loss and the 16-bit linears form them: tiles of results, their operands in LDS.
#pragma once
#include "qb_tiles.hpp"

namespace qb {

// Tiles of BM x BN results by WM x WN wavefronts, TM x TN blocks of 32 x 32 each; the contraction goes in steps of 64 through a ring of
// stages in LDS, one multiplied while the others are under way.  An operand lies in LDS as it does in memory: rows of results with the
// contraction along them, or rows along the contraction (in blocks of 64 results), read turned.
template <int WM_, int WN_, int TM_, int TN_, int STAGES_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, kWaves = WM * WN, kStages = STAGES_;
    static constexpr int BM = 32 * WM * TM, BN = 32 * WN * TN;
    static constexpr int kStage = (BM + BN) * 128;
    // row number i that a lane copies
    static __device__ __forceinline__ int row(int i, int wave, int lane) { return (i * kWaves + wave) * 8 + (lane >> 3); }
};

// eight steps of the contraction in their own order: rows row0 + 8 * (lane / 32) ..
__device__ __forceinline__ v8s across_in_order(const uint8_t *tile, int row0, int col0, int lane)
{
    typedef Rows<64> R;
    typedef __attribute__((address_space(3))) v4s *turned;
    const int row = row0 + 8 * (lane >> 5) + ((lane >> 2) & 3), col = col0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const uint8_t *first = tile + R::at(row, col >> 3) + 2 * (col & 7), *second = tile + R::at(row + 4, col >> 3) + 2 * (col & 7);
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned)first), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned)second);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <bool ACROSS>
__device__ __forceinline__ v8s operand(const uint8_t *tile, int result, int sub, int lane)
{
    if constexpr (ACROSS) return across_in_order(tile + (result >> 6) * 8192, 16 * sub, result & 63, lane);
    else return *reinterpret_cast<const v8s *>(tile + Rows<64>::at(result + (lane & 31), 2 * sub + (lane >> 5)));
}

// acc += A B^T over one step, whose operands lie in a stage
template <typename T, typename S, bool A_ACROSS, bool B_ACROSS>
__device__ __forceinline__ void step(v16f (&acc)[S::TM][S::TN], const uint8_t *ta, int wave, int lane)
{
    const int wm = wave / S::WN, wn = wave - wm * S::WN;
    const uint8_t *const tb = ta + S::BM * 128;
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) {
        v8s x[S::TM], y[S::TN];
#pragma unroll
        for (int i = 0; i < S::TM; ++i) x[i] = operand<A_ACROSS>(ta, (wm * S::TM + i) * 32, sub, lane);
#pragma unroll
        for (int j = 0; j < S::TN; ++j) y[j] = operand<B_ACROSS>(tb, (wn * S::TN + j) * 32, sub, lane);
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int j = 0; j < S::TN; ++j) acc[i][j] = T::mma32(x[i], y[j], acc[i][j]);
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
// Workgroups are dealt to the XCDs in turn: numbers that follow each other on one XCD get neighbouring tiles.
__device__ __forceinline__ int first_tile() { return (gridDim.x & 7) ? (int)blockIdx.x : (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)); }

}  // namespace qb
