// Newton-Schulz products of matrices too small to fill the chip with large tiles, where a
// step is some twenty dependent launches and each launch's latency is what counts.
//
// A workgroup computes one 64 x 64 tile; its waves split K between them (each takes every
// eighth or fourth K step of 16), read their operands straight from memory and add their
// sums in LDS. Up to 256 tiles, one a CU, eight waves each load two or four K steps
// ahead, so that a launch takes little more than one memory latency, the sum and the
// store. With more tiles four waves each, and several workgroups a CU, whose sums and
// stores hide behind the others' products (eight 512 x 1376 283 -> 242 us). Both operands
// are read along K: a symmetric right operand is its own transpose, and X is kept both
// ways. All matrices are stored in MFMA operands, blocks of 32 rows x 16 K entries, 1 KB
// each in lane order (small_chunk): an operand is one contiguous load. (Row by row an
// operand is 32 pieces of 32 bytes, and a launch took about twice as long.) All sides are
// multiples of 64 here (padded with zeros), so nothing is checked.
#include "gemm2.hpp"
#include "ns_dev.hpp"
#include "prof.hpp"

namespace fpo {

namespace {

constexpr int kSmallEdge = 64;
constexpr int kRedLd = kSmallEdge + 4;  // row stride of the partial sums in LDS
constexpr int kTrLd = kSmallEdge + 8;   // of the transposed tile

// One K step's operands of a wave: 32 rows a fragment, 8 K entries a lane.
template <bool PAIR>
struct SmallFrag {
  u32x4 a[2], b[2], al[PAIR ? 2 : 1], bl[PAIR ? 2 : 1];
};

__device__ __forceinline__ void unpack8(u32x4 w, float (&v)[8]) {
  const f16x8 h = __builtin_bit_cast(f16x8, w);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = (float)h[k];
}
__device__ __forceinline__ u32x4 pack8(const uint16_t (&h)[8]) {
  return u32x4{h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16,
               h[6] | (uint32_t)h[7] << 16};
}

struct NsNotLast {};

// rows: C is stored row by row. Last = NsLast (kApplyX): C is not stored, the caller's
// matrices are finished. NW waves, 8 or 4.
template <int WHAT, bool PAIR, int NW, class Last>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 2 : 3) void ns_small_kernel(NsGemmArgs g, NsMat x_of_b, NsMat to_t,
                                                                                   int rows, Last last) {
  constexpr bool SYM = WHAT != kApplyX, LAST = !std::is_same<Last, NsNotLast>::value;
  constexpr int U = (NW == 4 ? 2 : 4) / (PAIR ? 2 : 1);  // K steps loaded together
  constexpr int E = 8 / NW, H = NW / 2;           // chunks of eight entries a thread stores; partial sums in LDS
  __shared__ __align__(16) float red[H][kSmallEdge][kRedLd];
  const int ntm = g.M / kSmallEdge;
  const int loc = blockIdx.x, mat = blockIdx.y;
  int tm, tn;
  if constexpr (SYM) {
    tri_tile(loc, ntm, tm, tn);
  } else {
    tn = loc / ntm;
    tm = loc - tn * ntm;
  }
  const int m0 = tm * kSmallEdge, n0 = tn * kSmallEdge;
  const NsMat a = g.a[0], b = g.b[0], c = g.c[0];
  const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), l = threadIdx.x & 63;
  const uint16_t* ah = a.hi + mat * a.stride;
  const uint16_t* bh = b.hi + mat * b.stride;
  // ---- what the epilogue adds, eight entries of a row a chunk, loaded ahead
  const int er = threadIdx.x & 63, row = m0 + er;  // in the tile; ec: its columns
  auto ec = [&](int e) { return 8 * ((int)(threadIdx.x >> 6) + NW * e); };
  u32x4 xw[E], yw[E];
  float adv = 0.f, bdv[E][8];
  auto load_diag = [&](int e) {
    if constexpr ((WHAT == kMul || WHAT == kPoly) && !PAIR) {
#pragma unroll
      for (int k = 0; k < 8; ++k) bdv[e][k] = b.diag[mat * b.dstride + n0 + ec(e) + k];
    }
  };
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int col = n0 + ec(e);
    const int64_t at = small_chunk(row, col, g.N);
    xw[e] = yw[e] = u32x4{0u, 0u, 0u, 0u};
    if constexpr (WHAT == kPoly || (WHAT == kMul && !PAIR)) xw[e] = *reinterpret_cast<const u32x4*>(ah + at);
    if constexpr (WHAT == kPoly && PAIR) yw[e] = *reinterpret_cast<const u32x4*>(ah + a.lo_off + at);
    if constexpr (WHAT == kMul && !PAIR) yw[e] = *reinterpret_cast<const u32x4*>(bh + at);
    if constexpr (WHAT == kApplyX && !PAIR)
      yw[e] = *reinterpret_cast<const u32x4*>(x_of_b.hi + mat * x_of_b.stride + at);
    if constexpr (NW == 8) load_diag(e);  // (four waves have no registers left to hold it)
  }
  if constexpr (WHAT != kGram && !PAIR) adv = a.diag[mat * a.dstride + row];
  // ---- the wave's share of K
  const int steps = g.K / 16;
  const uint16_t* ap = ah + (int64_t)m0 * g.K;
  const uint16_t* bp = bh + (int64_t)n0 * g.K;
  const int64_t r32 = (int64_t)32 * g.K;  // the next 32 rows
  f32x16 acc[2][2] = {{f32x16{}, f32x16{}}, {f32x16{}, f32x16{}}};
  auto load = [&](SmallFrag<PAIR> (&f)[U], int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + NW * u;
      if (s >= steps) break;  // (uniform)
      const uint16_t* pa = ap + 512 * (int64_t)s;
      const uint16_t* pb = bp + 512 * (int64_t)s;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f[u].a[h] = reinterpret_cast<const u32x4*>(pa + h * r32)[l];
        f[u].b[h] = reinterpret_cast<const u32x4*>(pb + h * r32)[l];
        if constexpr (PAIR) {
          f[u].al[h] = reinterpret_cast<const u32x4*>(pa + h * r32 + a.lo_off)[l];
          f[u].bl[h] = reinterpret_cast<const u32x4*>(pb + h * r32 + b.lo_off)[l];
        }
      }
    }
  };
  auto multiply = [&](const SmallFrag<PAIR> (&f)[U], int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + NW * u >= steps) break;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          acc[h][i] = mfma_16bit<true>(f[u].b[i], f[u].a[h], acc[h][i]);
          if constexpr (PAIR) {
            acc[h][i] = mfma_16bit<true>(f[u].bl[i], f[u].a[h], acc[h][i]);
            acc[h][i] = mfma_16bit<true>(f[u].b[i], f[u].al[h], acc[h][i]);
          }
        }
    }
  };
  SmallFrag<PAIR> f0[U], f1[U];
  constexpr int kAhead = NW * U;
  load(f0, w);
  for (int s = w; s < steps; s += 2 * kAhead) {
    load(f1, s + kAhead);
    multiply(f0, s);
    load(f0, s + 2 * kAhead);
    multiply(f1, s + kAhead);
  }
  // ---- sums: the upper half of the waves into LDS, the lower half adds its own, and the
  // H sums are added below. (The products are taken as B A^T, so that a lane has four
  // neighbouring columns of a row.)
  const int lr = l & 31, lc = 4 * (l >> 5);
  auto each = [&](auto&& f) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          f(f32x4{acc[h][i][r], acc[h][i][r + 1], acc[h][i][r + 2], acc[h][i][r + 3]},
            *reinterpret_cast<f32x4*>(&red[w % H][32 * h + lr][32 * i + 2 * r + lc]));
  };
  if (w >= H) each([](f32x4 v, f32x4& m) { m = v; });
  __syncthreads();
  if (w < H) each([](f32x4 v, f32x4& m) { m += v; });
  __syncthreads();
  // ---- epilogue
  const float alpha = g.alpha[0];
  uint16_t* ch = LAST ? nullptr : c.hi + mat * c.stride;
  uint16_t h[E][8], lo[E][8];
  float fin[LAST ? E : 1][8];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int col = n0 + ec(e);
    if constexpr (NW == 4) load_diag(e);
    float t[8], xv[8], yv[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      t[k] = red[0][er][ec(e) + k];
#pragma unroll
      for (int q = 1; q < H; ++q) t[k] += red[q][er][ec(e) + k];
    }
    unpack8(xw[e], xv);
    unpack8(yw[e], yv);
    if constexpr (WHAT == kPoly && PAIR) {
#pragma unroll
      for (int k = 0; k < 8; ++k) xv[k] += yv[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if constexpr (!PAIR && WHAT == kPoly) t[k] = fmaf(adv + bdv[e][k], xv[k], t[k]);
      if constexpr (!PAIR && WHAT == kMul) t[k] = fmaf(adv, yv[k], fmaf(bdv[e][k], xv[k], t[k]));
      if constexpr (!PAIR && WHAT == kApplyX) t[k] = fmaf(adv, yv[k], t[k]);
      t[k] *= alpha;
      if constexpr (WHAT == kPoly) {
        t[k] = fmaf(g.beta, xv[k], t[k]);
        if (row == col + k) t[k] += fmaf(g.beta, adv, g.eye);
      }
      if constexpr (LAST) {
        fin[e][k] = t[k];
        continue;
      }
      h[e][k] = to_f16(t[k]);
      const float rest = t[k] - f16_to_f32(h[e][k]);
      if constexpr (PAIR) lo[e][k] = to_f16(rest);
      if constexpr (!PAIR && SYM)
        if (row == col + k) c.diag[mat * c.dstride + row] = rest;
    }
    if constexpr (!LAST) {
      const int64_t out = rows ? (int64_t)row * g.N + col : small_chunk(row, col, g.N);
      *reinterpret_cast<u32x4*>(ch + out) = pack8(h[e]);
      if constexpr (PAIR) *reinterpret_cast<u32x4*>(ch + c.lo_off + out) = pack8(lo[e]);
    }
  }
  if constexpr (LAST) {
    using T = typename std::conditional<PAIR, float, uint16_t>::type;
    const NsFinish& fa = last.f;
    const bool tall = (fa.tall >> mat) & 1;
    // (r0, c0): of this tile in the caller's matrix, which for a tall one is the transpose
    const int R = fa.R[tall], C = fa.C[tall], r0 = tall ? n0 : m0, c0 = tall ? m0 : n0;
    if (tall) {
      float(*tr)[kRedLd] = red[0];
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int k = 0; k < 8; ++k) tr[ec(e) + k][er] = fin[e][k];
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int k = 0; k < 8; ++k) fin[e][k] = tr[er][ec(e) + k];
    }
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (r0 + er >= R || c0 + ec(e) >= C) continue;  // (C is a multiple of 8)
      const int64_t out = (int64_t)(r0 + er) * C + c0 + ec(e);
#pragma unroll
      for (int q = 0; q < 8; q += 4) {
        const f32x4 v = f32x4{fin[e][q], fin[e][q + 1], fin[e][q + 2], fin[e][q + 3]} * fa.pow2;
        if (last.what == kWriteO) finish4<T, kWriteO>(fa, last.p, mat, 0.f, 1.f, out + q, v, sum);
        else finish4<T, kApply>(fa, last.p, mat, fa.step[tall], 1.f, out + q, v, sum);
      }
    }
    if (last.what == kApply) {
      __shared__ double dred[NW];
      sum = block_sum_d(sum, dred);
      if (threadIdx.x == 0) fa.part[((int64_t)mat * ntm + tm) * (g.N / kSmallEdge) + tn] = sum;
    }
    return;
  }
  // the transposed tile: C's other half, or C^T
  const NsMat o = SYM ? c : to_t;
  if (SYM ? m0 == n0 : o.hi == nullptr) return;
  uint16_t* oh = o.hi + mat * o.stride;
  uint16_t(*tr)[kSmallEdge][kTrLd] = reinterpret_cast<uint16_t(*)[kSmallEdge][kTrLd]>(&red[0][0][0]);
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      tr[0][ec(e) + k][er] = h[e][k];
      if constexpr (PAIR) tr[1][ec(e) + k][er] = lo[e][k];
    }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int64_t to = small_chunk(n0 + er, m0 + ec(e), g.M);
    *reinterpret_cast<u32x4*>(oh + to) = *reinterpret_cast<const u32x4*>(&tr[0][er][ec(e)]);
    if constexpr (PAIR) *reinterpret_cast<u32x4*>(oh + o.lo_off + to) = *reinterpret_cast<const u32x4*>(&tr[1][er][ec(e)]);
  }
}

template <int WHAT, class Last>
void launch_small(const char* name, const NsGemmArgs& g, bool pair, const NsMat& x_of_b, const NsMat& to_t, int rows,
                  const Last& last, hipStream_t st) {
  const dim3 grid((unsigned)g.tiles, (unsigned)g.count);
  auto waves = [&](auto nw) {
    constexpr int NW = decltype(nw)::value;
    if (pair)
      FPO_LAUNCH(name, st,
                 (ns_small_kernel<WHAT, true, NW, Last><<<grid, dim3(64 * NW), 0, st>>>(
                     g, x_of_b, to_t, rows, last)));
    else
      FPO_LAUNCH(name, st,
                 (ns_small_kernel<WHAT, false, NW, Last><<<grid, dim3(64 * NW), 0, st>>>(
                     g, x_of_b, to_t, rows, last)));
  };
  if ((int64_t)g.tiles * g.count <= kCus) waves(std::integral_constant<int, 8>{});
  else waves(std::integral_constant<int, 4>{});
}

}  // namespace

hipError_t launch_small_product(int what, const char* name, NsGemmArgs g, bool pair, const NsMat& x_of_b,
                                const NsMat& to_t, bool rows, const NsLast* last, hipStream_t st) {
  g.tiles = (int)ns_tiles(g.M, g.N, kSmallEdge, what != kApplyX);
  const NsNotLast no;
  switch (what) {
    case kGram: launch_small<kGram>(name, g, pair, x_of_b, to_t, 0, no, st); break;
    case kMul: launch_small<kMul>(name, g, pair, x_of_b, to_t, 0, no, st); break;
    case kPoly: launch_small<kPoly>(name, g, pair, x_of_b, to_t, 0, no, st); break;
    default:
      if (last) launch_small<kApplyX>(name, g, pair, x_of_b, to_t, 0, *last, st);
      else launch_small<kApplyX>(name, g, pair, x_of_b, to_t, rows, no, st);
      break;
  }
  return hipGetLastError();
}

}  // namespace fpo
