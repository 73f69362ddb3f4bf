// Device-side pieces that the kernels of the Newton-Schulz products share.
#pragma once

#include "common.hpp"
#include "ns.hpp"

namespace fpo {

// A stack of equal matrices in the workspace: fp16, or pairs of fp16. A square one of
// single fp16 has `diag`: what its diagonal lost to rounding, in the same units.
// These matrices are near multiples of I, their diagonals the largest entries, so half
// of the rounding error of fp16 is there: 512 x 1382, five steps, 1.3e-3 against 64 bits
// without it, 6.4e-4 with it.
struct NsMat {
  uint16_t* hi;
  float* diag;
  int64_t lo_off;   // elements from a hi to its lo (which follow each other)
  int64_t stride;   // elements from one matrix to the next
  int64_t dstride;  // of diag
};

// One launch of products C = alpha A B over `count` matrices, for one or two sets of operands.
struct NsGemmArgs {
  NsMat a[2], b[2], c[2];
  int lda, ldb, ldc;
  int M, N, K;         // padded sizes (multiples of 64)
  int count, tiles;    // matrices; tiles a matrix
  int nbig;            // 128 x 128 launch: the 256 x 256 tiles before it (0: all tiles are 128 x 128)
  float alpha[2];      // by set
  float beta, eye;     // kPoly: C = alpha A A + beta A + eye I
};

// What a launch computes. kGram: X X^T, B K-contiguous ([N][K] rows); the others have B
// N-contiguous ([K][N]). kGram, kMul and kPoly: symmetric, tiles with tn <= tm. kApplyX: Q X.
enum { kGram = 0, kMul = 1, kPoly = 2, kApplyX = 3 };

__device__ __forceinline__ uint16_t to_f16(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ float f16_to_f32(uint16_t h) { return (float)__builtin_bit_cast(_Float16, h); }
__device__ __forceinline__ u32x2 pack4(const uint16_t (&h)[4]) {
  return u32x2{h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16};
}

// Tile (tm, tn), tn <= tm < n, of entry t of the lower triangle, taken in strips of four
// rows, column by column: neighbouring entries share row and column panels in L2 (a row
// at a time, sixteen tiles in a row read sixteen column panels).
__device__ __forceinline__ void tri_tile(int t, int n, int& tm, int& tn) {
  for (int first = 0;; first += 4) {
    const int h = min(4, n - first), square = first * h, count = square + h * (h + 1) / 2;
    if (t >= count && first + 4 < n) {
      t -= count;
      continue;
    }
    if (t < square) {
      tn = t / h;
      tm = first + t % h;
    } else {
      t -= square;
      int c = 0;
      while (t >= h - c) t -= h - c++;
      tn = first + c;
      tm = first + c + t;
    }
    return;
  }
}

// ---- what becomes of the orthogonal X
struct NsFinish {
  int R[2], C[2];            // rows and columns of the caller's matrix: [0] wide, [1] tall
  int mp;                    // X's row pitch
  uint64_t tall;
  float pow2;                // 2^-e of X
  // muon
  float decay, lr_wd;        // 1 - lr weight_decay, lr weight_decay
  float step[2];             // lr times the scale of O, by orientation
  int clip_update;
  double clip_frac;
  double* W_sumsq;
  float* clip_scale;
  double* part;              // [count][tiles]
  double* dsq;               // [count] ||delta||^2
};
struct NsOutPtrs {
  float* W[kMaxMats];
  void* o[kMaxMats];         // O, or the low-precision copy of W
  uint8_t id[kMaxMats];
};

enum { kWriteO = 0, kApply = 1, kDelta = 2 };

// Four entries v = O of the caller's matrix, from `at` on: written (kWriteO); the step on
// W, W' = decay W - step O (kApply; sum: ||W'||^2), or with the update clipped W' = W + k
// delta, delta = -lr_wd W - step O; or only ||delta||^2 (kDelta).
template <typename T, int WHAT>
__device__ __forceinline__ void finish4(const NsFinish& a, const NsOutPtrs& p, int mat, float step, float k, int64_t at,
                                        f32x4 v, double& sum) {
  if constexpr (WHAT == kWriteO) {
    st4<T>((T*)p.o[mat], at, v);
    return;
  }
  f32x4 w = ld4<float>(p.W[mat], at);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float delta = fmaf(-step, v[q], -a.lr_wd * w[q]);
    if constexpr (WHAT == kDelta)
      sum = fma((double)delta, (double)delta, sum);
    else
      w[q] = a.clip_update ? fmaf(k, delta, w[q]) : fmaf(-step, v[q], a.decay * w[q]);
  }
  if constexpr (WHAT == kApply) {
    st4<float>(p.W[mat], at, w);
    if (p.o[mat]) st4<T>((T*)p.o[mat], at, w);
#pragma unroll
    for (int q = 0; q < 4; ++q) sum = fma((double)w[q], (double)w[q], sum);
  }
}

// Where a small matrix (kernels_ns_small.hip) of `cols` columns has entries (row, col ..
// col + 7), col a multiple of 8: blocks of 32 rows x 16 columns, in each the first eight
// columns of the 32 rows, then the others.
__device__ __forceinline__ int64_t small_chunk(int row, int col, int cols) {
  return ((int64_t)(row >> 5) * (cols >> 4) + (col >> 4)) * 512 + ((col & 8) * 4 + (row & 31)) * 8;
}

// The products of small matrices: 64 x 64 tiles. B is given transposed: a symmetric one is
// its own transpose, for kApplyX it is X^T, and x_of_b X itself. kApplyX stores C^T in to_t
// if that has hi; with `rows` it stores C row by row, with `last` it does not store it but
// finishes the caller's matrices (kWriteO or kApply). One set of operands: ns_choose gives small
// matrices at most two steps a group, and only a third one's products make two.
struct NsLast {
  NsFinish f;
  NsOutPtrs p;
  int what;
};
hipError_t launch_small_product(int what, const char* name, NsGemmArgs g, bool pair, const NsMat& x_of_b,
                                const NsMat& to_t, bool rows, const NsLast* last, hipStream_t st);

}  // namespace fpo
