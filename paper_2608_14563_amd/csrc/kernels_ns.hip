// Orthogonalisation by Newton-Schulz products and the optimizer step built on it.
//
// X = M / (||M||_F + eps), n x m with n <= m (a matrix with more rows than columns is
// taken transposed); each step X <- a X + b (X X^T) X + c (X X^T)^2 X. Every step is a
// polynomial of X X^T, so that several steps need X only twice: A = X X^T once, the
// steps' factors B_j = a I + b A_j + c A_j^2 and A_{j+1} = B_j A_j B_j among n x n
// matrices, then X <- (B_g ... B_1) X (ns.hpp: groups). All n x n matrices here are
// symmetric: only the tiles on and under the diagonal are computed, each stored at
// both places.
//
// Number formats. Products take fp16 operands and add in fp32. Every matrix is stored
// times a power of two that keeps a bound of its spectral norm under 2^13 (ns.hpp), so
// that fp16's range is no concern and its 11 bits count: with bf16 operands (8 bits)
// the five-step result of a 512 x 1536 normal matrix is off by 1.1e-2 against 64 bits,
// with fp16 by 1.3e-3, and half of that with what the diagonals lose to rounding kept
// (NsMat). The matrix instructions run at the same rate. With float32 operands every
// matrix is a pair hi + lo of fp16 and a product the three hi hi + hi lo + lo hi: 22 to
// 23 bits at three times the work, where fp32 matrix instructions take 16 times.
//
// Bound by the matrix pipes at the power limit: the Muon step of nine 4096 x 12288
// matrices takes 20.9 ms, of which the products 17.9 (1.10 PFLOP/s of 1.14 that a library
// product of 8192^3 reaches), the passes over gradient, momentum and weights 3.0 at 4.9
// to 5.2 TB/s.
#include "gemm2s.hpp"
#include "gemm.hpp"
#include "ns_dev.hpp"
#include "prof.hpp"
#include "upd.hpp"

namespace fpo {

namespace {

template <int EDGE, bool BNC>
struct NsCore;
template <bool BNC>
struct NsCore<256, BNC> {
  using Smem = G2Smem;
  using Map = AccMap2<BNC>;
  static constexpr int FM = 4, FN = 4, VEC = BNC ? 4 : 1;
};
template <bool BNC>
struct NsCore<128, BNC> {
  using Smem = G2SSmem;
  using Map = AccMap2S<BNC>;
  static constexpr int FM = G2SWave<BNC>::FM, FN = G2SWave<BNC>::FN, VEC = 1;
};

__device__ __forceinline__ void unpack4(u32x2 w, float (&v)[4]) {
  const f16x4 h = __builtin_bit_cast(f16x4, w);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = (float)h[k];
}

// What the epilogue of the 256 x 256 tiles adds at four rows (row .. row + 3) and four columns
// of an operand, as loaded.
struct NsBlock {
  u32x2 w[4];
  __device__ __forceinline__ void load(const uint16_t* p, int ld, int row, int col) {
#pragma unroll
    for (int r = 0; r < 4; ++r) w[r] = *reinterpret_cast<const u32x2*>(p + (int64_t)(row + r) * ld + col);
  }
  __device__ __forceinline__ void get(float (&v)[4][4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) unpack4(w[r], v[r]);
  }
};

__device__ __forceinline__ void unpack8(u32x4 w, float (&v)[8]) {
  const f16x8 h = __builtin_bit_cast(f16x8, w);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = (float)h[k];
}

template <int V>
__device__ __forceinline__ void store_f16(uint16_t* p, const uint16_t (&h)[V]) {
  if constexpr (V == 4) *reinterpret_cast<u32x2*>(p) = pack4(h);
  else *p = h[0];
}

// 128 x 128 tiles: the eight entries of a row that a thread finishes, eight times, and
// where they are in LDS: sums with the halves of 64 exchanged every four rows (which the
// two halves of a wave write), chunks of eight 16-bit entries exchanged every eight rows
// (so that rows eight apart are in different banks when a column is read).
__device__ __forceinline__ int ns_row(int q) { return (int)(threadIdx.x >> 4) + 16 * q; }
__device__ __forceinline__ int ns_col() { return 8 * (int)(threadIdx.x & 15); }
__device__ __forceinline__ int ns_sum_at(int row, int col) { return row * 128 + (col ^ ((row & 4) << 3)); }
__device__ __forceinline__ int ns_chunk_at(int row, int col) { return row * 16 + ((col >> 3) ^ (row >> 3)); }

// PAIR: operands and C are hi + lo, and a product is hi hi + hi lo + lo hi. Otherwise C =
// (A + diag(a)) (B + diag(b)) = A B + (a_i B_ij + A_ij b_j) with the products of two
// remainders left out, for square A (a) and B (b).
//
// Tiles of EDGE x EDGE, one a workgroup: those of the 256 grid from nbig on go as 128 x
// 128 quarters, in a launch of their own (ns.hpp: ns_split).
//
// Both cores leave one workgroup a CU, so that whatever follows the K loop is paid in
// full. 256 x 256: the entries of A and B that the epilogue adds are loaded ahead, those
// of the first rows before the K loop, the others while the rows before them are stored.
// What is left is that all workgroups write at once: six 2048 x 2048 products take 66 us,
// 58 of them the K loop, and write 50 MB (a quarter of the tile at a time through LDS, as
// below, halves the code but waits four times for its copies: 70 us).
// 128 x 128, where the K loop is short: what follows it runs once a launch, so that its
// instructions come from L2 and their number is what counts. The sums go to LDS, those
// entries of A and B too (after the K loop, which has just read them), and a short loop
// finishes eight entries of a row at a time: 11 KB of code instead of 26 KB, four 1024 x
// 1024 products 20.6 -> 15.2 us (loaded ahead into registers, eight entries at a time but
// unrolled, 33 KB: 23.4 us).
template <int EDGE, bool FAST, int WHAT, bool PAIR>
__global__ __launch_bounds__(256, 1) void ns_gemm_kernel(NsGemmArgs g) {
  constexpr bool SYM = WHAT != kApplyX, BNC = WHAT != kGram;
  using Core = NsCore<EDGE, BNC>;
  constexpr int VEC = Core::VEC, FM = Core::FM, FN = Core::FN / VEC;
  __shared__ typename Core::Smem sm;
  // ---- which tile
  const int edge = g.nbig ? 256 : EDGE;  // of the grid that `tiles` counts
  const int ntm = (g.M + edge - 1) / edge, ntn = (g.N + edge - 1) / edge;
  const bool part = EDGE == 128 && g.nbig;
  // a contiguous range of each 256 tiles to an XCD (which share its L2), all XCDs on the
  // same matrices (which share the Infinity Cache)
  const int win = (int)blockIdx.x & ~255;
  const int slot = win + xcd_remap((int)blockIdx.x - win, min(256, (int)gridDim.x - win));
  const int id = part ? g.nbig + (slot >> 2) : slot;
  int mat = id / g.tiles;
  const int loc = id - mat * g.tiles;
  const int set = mat / g.count;
  mat -= set * g.count;
  int tm, tn;
  if constexpr (SYM)
    tri_tile(loc, ntm, tm, tn);
  else
    grouped_tile(loc, ntm, ntn, 8, tm, tn);
  tm = to_scalar(tm);
  tn = to_scalar(tn);
  mat = to_scalar(mat);
  const int m0 = tm * edge + (part ? (slot & 1) * 128 : 0), n0 = tn * edge + (part ? (slot >> 1 & 1) * 128 : 0);
  if (part && (m0 >= g.M || n0 >= g.N || (SYM && n0 > m0))) return;
  const NsMat a = set ? g.a[1] : g.a[0], b = set ? g.b[1] : g.b[0], c = set ? g.c[1] : g.c[0];
  const uint16_t* ah = a.hi + mat * a.stride;
  const uint16_t* bh = b.hi + mat * b.stride;
  const typename Core::Map map;
  // ---- what the epilogue adds: x of A (its low half xl for pairs), y of B
  constexpr bool HAS_X = WHAT == kPoly || (WHAT == kMul && !PAIR), HAS_XL = WHAT == kPoly && PAIR;
  constexpr bool HAS_Y = !PAIR && (WHAT == kMul || WHAT == kApplyX);
  NsBlock x[2][FN][4], xl[2][FN][4], y[2][FN][4];  // 256
  auto inside = [&](int row, int col) { return FAST || (row < g.M && col < g.N); };  // (blocks are in or out)
  // pairs leave the 256 x 256 core no registers to load ahead of the K loop, products of
  // two operands' entries half of them
  constexpr bool AHEAD_X = !PAIR, AHEAD_Y = AHEAD_X && WHAT != kMul;
  auto fetch = [&](int f, auto& bx, auto& bxl, auto& by, bool dox, bool doy) {
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = m0 + map.row(f, 4 * q), col = n0 + map.col(i * VEC);
        if (!inside(row, col)) continue;
        if constexpr (HAS_X) if (dox) bx[i][q].load(ah, g.ldc, row, col);
        if constexpr (HAS_XL) if (dox) bxl[i][q].load(ah + a.lo_off, g.ldc, row, col);
        if constexpr (HAS_Y) if (doy) by[i][q].load(bh, g.ldc, row, col);
      }
  };
  if constexpr (EDGE == 256) {
    fetch(0, x[0], xl[0], y[0], AHEAD_X, AHEAD_Y);
  }
  // ---- products
  f32x16 acc[Core::FM][Core::FN];
  const Operand A{ah + (int64_t)m0 * g.lda, g.lda, band_bytes(g.M - m0, g.lda) + (PAIR ? (uint32_t)(2 * a.lo_off) : 0u)};
  const uint16_t* bp = bh + (BNC ? (int64_t)n0 : (int64_t)n0 * g.ldb);
  const Operand B{bp, g.ldb,
                  (BNC ? band_bytes(g.K, g.ldb, n0) : band_bytes(g.N - n0, g.ldb)) + (PAIR ? (uint32_t)(2 * b.lo_off) : 0u)};
  if constexpr (EDGE == 256) {
    zero_acc2(acc);
#pragma unroll 1
    for (int s = 0; s < (PAIR ? 3 : 1); ++s) {
      const Operand As{A.base + (s == 2 ? a.lo_off : 0), A.ld, A.bytes - (s == 2 ? (uint32_t)(2 * a.lo_off) : 0u)};
      const Operand Bs{B.base + (s == 1 ? b.lo_off : 0), B.ld, B.bytes - (s == 1 ? (uint32_t)(2 * b.lo_off) : 0u)};
      gemm2_mainloop<BNC, FAST, true>(sm, acc, As, Bs, g.M - m0, g.N - n0, g.K, 0, g.K / 64);
    }
  } else {
    zero_acc2s<BNC>(acc);
    if constexpr (PAIR) {
      const K3 seg{g.K / 64, (uint32_t)(2 * a.lo_off), (uint32_t)(2 * b.lo_off)};
      gemm2s_mainloop<BNC, true>(sm, acc, A, B, g.M - m0, g.N - n0, 3 * g.K, 0, 3 * (g.K / 64), seg);
    } else {
      gemm2s_mainloop<BNC, true>(sm, acc, A, B, g.M - m0, g.N - n0, g.K, 0, g.K / 64);
    }
  }
  // ---- epilogue (the mainloop ends with a barrier: LDS is free)
  const float alpha = set ? g.alpha[1] : g.alpha[0];
  uint16_t* ch = c.hi + mat * c.stride;
  const float* ad = !PAIR && WHAT != kGram ? a.diag + mat * a.dstride : nullptr;
  const float* bd = !PAIR && (WHAT == kMul || WHAT == kPoly) ? b.diag + mat * b.dstride : nullptr;
  float* cd = !PAIR && SYM ? c.diag + mat * c.dstride : nullptr;
  // the tile is symmetric with tile (tn, tm): off the diagonal it is stored twice, the
  // second time transposed, by way of LDS so that whole lines are written
  constexpr bool STAGE = SYM && EDGE == 256 && !PAIR;
  const bool mirror = SYM && m0 != n0;
  uint16_t* lds = reinterpret_cast<uint16_t*>(&sm);
  if constexpr (EDGE == 128) {
    // LDS: the sums, what was loaded of A and B (and in its place the tile of C, hi and
    // lo), the diagonals' remainders
    float* sums = reinterpret_cast<float*>(&sm);
    u32x4* xt = reinterpret_cast<u32x4*>(sums + 128 * 128);
    u32x4* yt = xt + 128 * 16;
    static_assert(sizeof(sm) >= 128 * 128 * 8, "sums and two tiles of 16 bits");
    __shared__ float rem[256];
    // (past the last row a copy reads zeros, past the last column what follows; neither is used)
    auto copy = [&](const uint16_t* from, u32x4* to) {
      const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), l = threadIdx.x & 63;
      const u32x4 r = make_rsrc(Operand{from + (int64_t)m0 * g.ldc + n0, g.ldc, band_bytes(g.M - m0, g.ldc, n0)});
      const uint32_t dst = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)to) + 8192u * w;
#pragma unroll
      for (int q = 0; q < 8; ++q) {  // ns_chunk_at: the lane's chunk of the row
        const int row = 32 * w + 4 * q + (l >> 4);
        dma16(r, dst + 1024u * q, 2u * (uint32_t)(row * g.ldc + 8 * ((l & 15) ^ (row >> 3))));
      }
    };
    if constexpr (HAS_X) copy(ah, xt);
    if constexpr (HAS_XL) copy(ah + a.lo_off, yt);
    if constexpr (HAS_Y) copy(bh, yt);
    float dv = 0.f;  // a remainder of A's diagonal, or B's
    if constexpr (!PAIR && WHAT != kGram) {
      const int t = threadIdx.x & 127;
      if (threadIdx.x < 128) {
        if (m0 + t < g.M) dv = a.diag[mat * a.dstride + m0 + t];
      } else if (WHAT != kApplyX && n0 + t < g.N) {
        dv = b.diag[mat * b.dstride + n0 + t];
      }
    }
#pragma unroll
    for (int f = 0; f < Core::FM; ++f)
#pragma unroll
      for (int i = 0; i < Core::FN; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[ns_sum_at(map.row(f, r), map.col(i))] = acc[f][i][r];
    if constexpr (!PAIR && WHAT != kGram) rem[threadIdx.x] = dv;
    wait_vmcnt<0>();
    __syncthreads();
    const int ec = ns_col(), col = n0 + ec;
#pragma unroll 1
    for (int q = 0; q < 8; ++q) {
      const int er = ns_row(q), row = m0 + er;
      if (!inside(row, col)) continue;
      const f32x4 t0 = *reinterpret_cast<const f32x4*>(sums + ns_sum_at(er, ec));
      const f32x4 t1 = *reinterpret_cast<const f32x4*>(sums + ns_sum_at(er, ec + 4));
      float t[8] = {t0[0], t0[1], t0[2], t0[3], t1[0], t1[1], t1[2], t1[3]}, xv[8], yv[8], adv = 0.f, bdv[8], rest = 0.f;
      const int own = ns_chunk_at(er, ec);
      if constexpr (HAS_X) unpack8(xt[own], xv);
      if constexpr (HAS_XL || HAS_Y) unpack8(yt[own], yv);
      if constexpr (HAS_XL) {
#pragma unroll
        for (int k = 0; k < 8; ++k) xv[k] += yv[k];
      }
      if constexpr (!PAIR && WHAT != kGram) adv = rem[er];
      if constexpr (!PAIR && (WHAT == kMul || WHAT == kPoly)) {
        const f32x4 b0 = *reinterpret_cast<const f32x4*>(rem + 128 + ec);
        const f32x4 b1 = *reinterpret_cast<const f32x4*>(rem + 132 + ec);
#pragma unroll
        for (int k = 0; k < 8; ++k) bdv[k] = k < 4 ? b0[k & 3] : b1[k & 3];
      }
      const int dk = SYM ? row - col : -1;  // which of the eight is on the diagonal
      f16x8 h, l;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if constexpr (!PAIR && WHAT == kPoly) t[k] = fmaf(adv + bdv[k], xv[k], t[k]);
        if constexpr (!PAIR && WHAT == kMul) t[k] = fmaf(adv, yv[k], fmaf(bdv[k], xv[k], t[k]));
        if constexpr (!PAIR && WHAT == kApplyX) t[k] = fmaf(adv, yv[k], t[k]);
        t[k] *= alpha;
        if constexpr (WHAT == kPoly) {
          t[k] = fmaf(g.beta, xv[k], t[k]);
          t[k] += dk == k ? fmaf(g.beta, adv, g.eye) : 0.f;
        }
        h[k] = (_Float16)t[k];
        const float lost = t[k] - (float)h[k];
        if constexpr (PAIR) l[k] = (_Float16)lost;
        if constexpr (!PAIR && SYM) rest = dk == k ? lost : rest;
      }
      if constexpr (!PAIR && SYM)
        if ((unsigned)dk < 8u) cd[row] = rest;
      const int64_t at = (int64_t)row * g.ldc + col;
      *reinterpret_cast<u32x4*>(ch + at) = __builtin_bit_cast(u32x4, h);
      if constexpr (PAIR) *reinterpret_cast<u32x4*>(ch + c.lo_off + at) = __builtin_bit_cast(u32x4, l);
      if constexpr (SYM) {
        xt[own] = __builtin_bit_cast(u32x4, h);  // (read above, by this thread alone)
        if constexpr (PAIR) yt[own] = __builtin_bit_cast(u32x4, l);
      }
    }
    if (!SYM || !mirror) return;
    __syncthreads();
    // the other half of C: the tile transposed
#pragma unroll 1
    for (int q = 0; q < 8; ++q) {
      const int er = ns_row(q);  // of the transposed tile
      if (!inside(m0 + ec, n0 + er)) continue;
      const int64_t at = (int64_t)(n0 + er) * g.ldc + m0 + ec;
      auto column = [&](const u32x4* tile) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(tile + ns_chunk_at(ec, er & ~7)) + (er & 7);
        uint16_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = p[k * 128];  // rows ec .. ec + 7 share the exchange
        return u32x4{v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16,
                     v[6] | (uint32_t)v[7] << 16};
      };
      *reinterpret_cast<u32x4*>(ch + at) = column(xt);
      if constexpr (PAIR) *reinterpret_cast<u32x4*>(ch + c.lo_off + at) = column(yt);
    }
    return;
  }
  auto finish = [&](int f, auto& bx, auto& bxl, auto& by) {
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int lr = map.row(f, 4 * q), lc = map.col(i * VEC), row = m0 + lr, col = n0 + lc;
        if (!inside(row, col)) continue;
        float xv[4][VEC], yv[4][VEC], bdv[VEC];
        f32x4 adv = {0.f, 0.f, 0.f, 0.f};
        if constexpr (HAS_X) bx[i][q].get(xv);
        if constexpr (HAS_XL) {
          bxl[i][q].get(yv);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int k = 0; k < VEC; ++k) xv[r][k] += yv[r][k];
        }
        if constexpr (HAS_Y) by[i][q].get(yv);
        if constexpr (!PAIR && WHAT != kGram) adv = *reinterpret_cast<const f32x4*>(ad + row);
        if constexpr (!PAIR && (WHAT == kMul || WHAT == kPoly)) {
#pragma unroll
          for (int k = 0; k < VEC; ++k) bdv[k] = bd[col + k];
        }
        float t[4][VEC];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            t[r][k] = acc[f][i * VEC + k][4 * q + r];
            if constexpr (!PAIR && WHAT == kPoly) t[r][k] = fmaf(adv[r] + bdv[k], xv[r][k], t[r][k]);
            if constexpr (!PAIR && WHAT == kMul) t[r][k] = fmaf(adv[r], yv[r][k], fmaf(bdv[k], xv[r][k], t[r][k]));
            if constexpr (!PAIR && WHAT == kApplyX) t[r][k] = fmaf(adv[r], yv[r][k], t[r][k]);
            t[r][k] *= alpha;
            if constexpr (WHAT == kPoly) t[r][k] = fmaf(g.beta, xv[r][k], t[r][k]);
          }
        if (SYM && !mirror) {  // (uniform) the diagonal's entries: the multiple of I, the remainders
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int k = 0; k < VEC; ++k)
              if (row + r == col + k) {
                if constexpr (WHAT == kPoly) t[r][k] += fmaf(g.beta, adv[r], g.eye);
                if constexpr (!PAIR) cd[col + k] = t[r][k] - f16_to_f32(to_f16(t[r][k]));
              }
        }
        uint16_t h[4][VEC], l[4][VEC];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            h[r][k] = to_f16(t[r][k]);
            if constexpr (PAIR) l[r][k] = to_f16(t[r][k] - f16_to_f32(h[r][k]));
          }
          const int64_t at = (int64_t)(row + r) * g.ldc + col;
          store_f16<VEC>(ch + at, h[r]);
          if constexpr (PAIR) store_f16<VEC>(ch + c.lo_off + at, l[r]);
        }
        if (SYM && mirror) {
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const uint16_t ht[4] = {h[0][k], h[1][k], h[2][k], h[3][k]};
            if constexpr (STAGE) {
              const int cc = lc + k;
              store_f16<4>(lds + cc * 256 + (((lr >> 3) ^ (BNC ? (cc >> 2) & 31 : cc & 31)) * 8 + (lr & 7)), ht);
            } else {
              const int64_t at = (int64_t)(col + k) * g.ldc + row;
              store_f16<4>(ch + at, ht);
              if constexpr (PAIR) {
                const uint16_t lt[4] = {l[0][k], l[1][k], l[2][k], l[3][k]};
                store_f16<4>(ch + c.lo_off + at, lt);
              }
            }
          }
        }
      }
  };
  if constexpr (EDGE == 256) {
    fetch(0, x[0], xl[0], y[0], !AHEAD_X, !AHEAD_Y);
#pragma unroll
    for (int f = 0; f < FM; ++f) {
      if (f + 1 < FM) fetch(f + 1, x[(f + 1) & 1], xl[(f + 1) & 1], y[(f + 1) & 1], true, true);
      finish(f, x[f & 1], xl[f & 1], y[f & 1]);
    }
  }
  if constexpr (STAGE) {
    if (!mirror) return;
    __syncthreads();
    const int p = threadIdx.x & 31;
    for (int cc = threadIdx.x >> 5; cc < 256; cc += 8)
      if (inside(m0 + 8 * p, n0 + cc))
        *reinterpret_cast<u32x4*>(ch + (int64_t)(n0 + cc) * g.ldc + m0 + 8 * p) =
            *reinterpret_cast<const u32x4*>(lds + cc * 256 + (p ^ (BNC ? (cc >> 2) & 31 : cc & 31)) * 8);
  }
}

// ---------------------------------------------------------------- elementwise passes
// The update's direction u of one element: the momentum buffer's new value b' = mu b +
// s g (s g at step 1), and u = s g + mu b' (Nesterov) or b'. Without a buffer u = s g.
struct Direction {
  float mu, s;
  bool first, nesterov;
  __device__ __forceinline__ float state(float g, float b) const { return first ? s * g : fmaf(mu, b, s * g); }
  __device__ __forceinline__ float u(float g, float b1) const { return nesterov ? fmaf(mu, b1, s * g) : b1; }
};

// Pointers of a batch, by value.
struct NsPtrs {
  const void* x[kMaxMats];   // X, or the gradient
  float* state[kMaxMats];
  uint8_t id[kMaxMats];
};

struct NsEw {
  int64_t numel;
  int rows_n, cols_m;        // n, m
  int np, mp;                // padded (mp on the large tiles: X's row pitch)
  uint64_t tall;
  double eps;
  float momentum;
  int first, nesterov;
  double clip_frac;          // > 0: clip the gradient against W_sumsq
  const double* grad_sumsq;
  const double* W_sumsq;
  float* clip_scale;
  double* part;              // [count][kNsNormBlocks]
};

template <bool MUON>
__device__ __forceinline__ Direction direction(const NsEw& a, const NsPtrs& p, int mat) {
  Direction d{};
  if constexpr (MUON) {
    const int id = p.id[mat];
    d.mu = p.state[mat] ? a.momentum : 0.f;
    d.first = a.first != 0 || !p.state[mat];
    d.nesterov = a.nesterov != 0 && p.state[mat];
    d.s = a.clip_frac > 0.0 ? clip_factor(a.grad_sumsq[id], a.W_sumsq[id], a.clip_frac) : 1.f;
  }
  return d;
}

// Momentum (MUON: the state in place) and the block's share of ||u||^2, in double.
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsEw a, NsPtrs p) {
  __shared__ double red[4];
  const int mat = blockIdx.y;
  const T* x = (const T*)p.x[mat];
  float* st = MUON ? p.state[mat] : nullptr;
  const Direction d = direction<MUON>(a, p, mat);
  double sum = 0.0;
  // every block takes an equal run of 1024-element pieces
  const int64_t pieces = (a.numel + 1023) / 1024, per = (pieces + gridDim.x - 1) / gridDim.x;
  const int64_t i1 = min(a.numel, (int64_t)(blockIdx.x + 1) * per * 1024);
  for (int64_t i = (int64_t)blockIdx.x * per * 1024 + threadIdx.x * 4; i < i1; i += 1024) {
    f32x4 v = ld4<T>(x, i);
    if constexpr (MUON) {
      f32x4 b = st && !d.first ? ld4<float>(st, i) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        b[k] = d.state(v[k], b[k]);
        v[k] = d.u(v[k], b[k]);
      }
      if (st) st4<float>(st, i, b);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) sum = fma((double)v[k], (double)v[k], sum);
  }
  sum = block_sum_d(sum, red);
  if (threadIdx.x == 0) {
    a.part[(int64_t)mat * kNsNormBlocks + blockIdx.x] = sum;
    if (MUON && blockIdx.x == 0 && a.clip_scale) a.clip_scale[p.id[mat]] = d.s;
  }
}

// X = 2^e u / (||u|| + eps) as fp16 (PAIR: hi + lo), n x m and padded with zeros, and X^T
// where it is wanted (XT.hi: small products, both then in their layout); one 64 x 64 tile
// a workgroup. The matrix that is laid out like the source (X, or X^T of a tall one) is
// stored as read, the other through LDS.
template <typename T, bool MUON, bool PAIR>
__global__ __launch_bounds__(256) void ns_convert_kernel(NsEw a, NsPtrs p, NsMat X, NsMat XT, float pow2, int nblk) {
  __shared__ float tile[kNsEdge][kNsEdge + 1];
  __shared__ double red[4];
  const int mat = blockIdx.z, t = threadIdx.x;
  const int i0 = blockIdx.y * kNsEdge, j0 = blockIdx.x * kNsEdge;  // rows and columns of X
  const T* x = (const T*)p.x[mat];
  const float* st = MUON ? p.state[mat] : nullptr;
  const Direction d = direction<MUON>(a, p, mat);
  const bool tall = (a.tall >> mat) & 1;
  // source rows and columns of this tile
  const int R = tall ? a.cols_m : a.rows_n, C = tall ? a.rows_n : a.cols_m;
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  // loaded ahead of the norm, which waits for the partials and the workgroup
  f32x4 v[4], b[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = k * 16 + (t >> 4), c = 4 * (t & 15);
    v[k] = b[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (r0 + r < R && c0 + c < C) {  // C is a multiple of 8
      const int64_t at = (int64_t)(r0 + r) * C + c0 + c;
      v[k] = ld4<T>(x, at);
      if constexpr (MUON)
        if (st) b[k] = ld4<float>(st, at);
    }
  }
  const double* part = a.part + (int64_t)mat * kNsNormBlocks;
  double s = 0.0;
  for (int k = t; k < nblk; k += 256) s += part[k];
  s = sqrt(block_sum_d(s, red)) + a.eps;
  const double f = s == 0.0 ? 0.0 : (double)pow2 / s;  // (double: beyond float's range for a norm under 2.4e-35)
  const NsMat straight = tall ? XT : X, turned = tall ? X : XT;
  const int ld_s = tall ? a.np : a.mp, ld_t = tall ? a.mp : a.np;
  auto put = [&](const NsMat& to, int i, int j, int ld, f32x4 v) {
    const int64_t at = XT.hi ? small_chunk(i, j & ~7, ld) + (j & 4) : (int64_t)i * ld + j;
    u32x2 h, l;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint16_t h0 = to_f16(v[2 * k]), h1 = to_f16(v[2 * k + 1]);
      h[k] = h0 | (uint32_t)h1 << 16;
      l[k] = to_f16(v[2 * k] - f16_to_f32(h0)) | (uint32_t)to_f16(v[2 * k + 1] - f16_to_f32(h1)) << 16;
    }
    uint16_t* hi = to.hi + mat * to.stride + at;
    *reinterpret_cast<u32x2*>(hi) = h;
    if constexpr (PAIR) *reinterpret_cast<u32x2*>(hi + to.lo_off) = l;
  };
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = k * 16 + (t >> 4), c = 4 * (t & 15);
    f32x4 u = v[k];
    if constexpr (MUON) {
#pragma unroll
      for (int q = 0; q < 4; ++q) u[q] = st ? d.u(u[q], b[k][q]) : d.s * u[q];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) u[q] = (float)((double)u[q] * f);
    if (straight.hi) put(straight, r0 + r, c0 + c, ld_s, u);
    if (turned.hi) {
#pragma unroll
      for (int q = 0; q < 4; ++q) tile[r][c + q] = u[q];
    }
  }
  if (!turned.hi) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c = k * 16 + (t >> 4), r = 4 * (t & 15);
    put(turned, c0 + c, r0 + r, ld_t, f32x4{tile[r][c], tile[r + 1][c], tile[r + 2][c], tile[r + 3][c]});
  }
}

// Four consecutive entries of X.
template <bool PAIR>
__device__ __forceinline__ f32x4 load_x4(const uint16_t* hi, const uint16_t* lo, int64_t at) {
  const f16x4 h = *reinterpret_cast<const f16x4*>(hi + at);
  f32x4 v = {(float)h[0], (float)h[1], (float)h[2], (float)h[3]};
  if constexpr (PAIR) {
    const f16x4 l = *reinterpret_cast<const f16x4*>(lo + at);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += (float)l[k];
  }
  return v;
}

// One 64 x 64 tile of the caller's matrix (finish4), by way of LDS where that is tall, and its
// share of a sum.
template <typename T, int WHAT, bool PAIR>
__global__ __launch_bounds__(256) void ns_finish_kernel(NsFinish a, NsOutPtrs p, NsMat X) {
  __shared__ float tile[kNsEdge][kNsEdge + 1];
  __shared__ double red[4];
  const int mat = blockIdx.z, t = threadIdx.x;
  const bool tall = (a.tall >> mat) & 1;
  const int i0 = blockIdx.y * kNsEdge, j0 = blockIdx.x * kNsEdge;  // of X
  const int R = a.R[tall], C = a.C[tall];
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  const uint16_t* hi = X.hi + mat * X.stride;
  const uint16_t* lo = hi + X.lo_off;
  if (tall) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = k * 16 + (t >> 4), j = 4 * (t & 15);
      const f32x4 v = load_x4<PAIR>(hi, lo, (int64_t)(i0 + i) * a.mp + j0 + j);
#pragma unroll
      for (int q = 0; q < 4; ++q) tile[j + q][i] = v[q];
    }
    __syncthreads();
  }
  const int id = p.id[mat];
  const float step = a.step[tall];
  float k_clip = 1.f;
  if constexpr (WHAT == kApply) {
    if (a.clip_update) k_clip = clip_factor(a.dsq[mat], a.W_sumsq[id], a.clip_frac);
  }
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = k * 16 + (t >> 4), c = 4 * (t & 15);
    if (r0 + r >= R || c0 + c >= C) continue;
    f32x4 v;
    if (tall)
      v = f32x4{tile[r][c], tile[r][c + 1], tile[r][c + 2], tile[r][c + 3]};
    else
      v = load_x4<PAIR>(hi, lo, (int64_t)(i0 + r) * a.mp + j0 + c);
    v *= a.pow2;
    const int64_t at = (int64_t)(r0 + r) * C + c0 + c;
    finish4<T, WHAT>(a, p, mat, step, k_clip, at, v, sum);
  }
  if constexpr (WHAT != kWriteO) {
    sum = block_sum_d(sum, red);
    if (t == 0) {
      a.part[((int64_t)mat * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x] = sum;
      if (WHAT == kApply && a.clip_update && a.clip_scale && blockIdx.x == 0 && blockIdx.y == 0)
        a.clip_scale[id] = k_clip;
    }
  }
}

// Per-matrix sums of the tiles' partials: into dsq, or W_sumsq of the caller's index.
__global__ __launch_bounds__(256) void ns_reduce_kernel(const double* part, int64_t tiles, double* dsq,
                                                        double* W_sumsq, NsOutPtrs p) {
  __shared__ double red[4];
  const int mat = blockIdx.x;
  const double s = block_sum_d(strided_sum_d(part + mat * tiles, 0, tiles), red);
  if (threadIdx.x == 0) {
    if (dsq)
      dsq[mat] = s;
    else
      W_sumsq[p.id[mat]] = s;
  }
}

// ---------------------------------------------------------------- workspace
constexpr int64_t kNsAlign = 256;

struct NsSpace {
  NsMat Xa, Xb;      // n x m: the iterates in turn
  NsMat Xat, Xbt;    // m x n: their transposes, for small products only
  NsMat A, C, P[3];  // n x n: Gram matrix, B A, and three for B and the product of the B
  double* norm_part;
  double* part;
  double* dsq;
  size_t bytes;
};

NsSpace ns_carve(int64_t n, int64_t m, int count, bool bf16, void* ws) {
  char* base = (char*)ws;
  size_t off = 0;
  auto take = [&](int64_t bytes) {
    char* p = base ? base + off : nullptr;
    off += (size_t)(ceil_div(bytes, kNsAlign) * kNsAlign);
    return p;
  };
  const int64_t np = ns_pad(n), mp = ns_pad(m);
  const bool small = ns_choose(n, m, count, bf16).small;
  auto mat = [&](int64_t rows, int64_t width) {
    const int64_t cols = small ? width : ns_pitch(width);
    NsMat x{};
    x.lo_off = rows * cols;
    x.stride = rows * cols * (bf16 ? 1 : 2);
    x.dstride = rows;
    x.hi = (uint16_t*)take(2 * x.stride * count);
    if (!bf16) return x;
    if (rows == np && width == np) x.diag = (float*)take(4 * np * count);
    return x;
  };
  NsSpace s{};
  s.Xa = mat(np, mp);
  s.Xb = mat(np, mp);
  if (small) {
    s.Xat = mat(mp, np);
    s.Xbt = mat(mp, np);
  }
  s.A = mat(np, np);
  s.C = mat(np, np);
  for (auto& q : s.P) q = mat(np, np);
  s.norm_part = (double*)take(8 * (int64_t)count * kNsNormBlocks);
  s.part = (double*)take(8 * (int64_t)count * (np / kNsEdge) * (mp / kNsEdge));
  s.dsq = (double*)take(8 * (int64_t)count);
  s.bytes = off;
  return s;
}

#define FPO_CHECK_LAUNCH()             \
  do {                                 \
    hipError_t e_ = hipGetLastError(); \
    if (e_ != hipSuccess) return e_;   \
  } while (0)

template <int EDGE, bool FAST, int WHAT, bool PAIR>
void launch_gemm(const char* name, const NsGemmArgs& g, int64_t grid, hipStream_t st) {
  FPO_LAUNCH(name, st, (ns_gemm_kernel<EDGE, FAST, WHAT, PAIR><<<dim3((unsigned)grid), dim3(256), 0, st>>>(g)));
}

template <int WHAT, bool PAIR>
hipError_t launch_product(const char* name, NsGemmArgs g, int sets, hipStream_t st) {
  const int mats = g.count * sets;
  const bool sym = WHAT != kApplyX;
  const NsSplit sp = ns_split(g.M, g.N, (int64_t)g.K * (PAIR ? 3 : 1), mats, sym);
  g.tiles = (int)ns_tiles(g.M, g.N, sp.nbig ? 256 : 128, sym);
  const int64_t all = (int64_t)g.tiles * mats;
  if (sp.nbig) {
    if (g.M % 256 == 0 && g.N % 256 == 0)
      launch_gemm<256, true, WHAT, PAIR>(name, g, sp.nbig, st);
    else
      launch_gemm<256, false, WHAT, PAIR>(name, g, sp.nbig, st);
  }
  if (sp.nbig < all) {
    g.nbig = (int)sp.nbig;
    launch_gemm<128, false, WHAT, PAIR>(name, g, sp.nbig ? 4 * (all - sp.nbig) : all, st);
  }
  return hipGetLastError();
}

template <typename T, bool PAIR>
hipError_t run_ns(const NsLaunch& a, const NsBatch& b) {
  hipStream_t st = (hipStream_t)a.stream;
  const int64_t n = b.n, m = b.m, np = ns_pad(n), mp = ns_pad(m);
  const NsSpace s = ns_carve(n, m, b.count, a.bf16, a.ws);
  const NsChoice choice = ns_choose(n, m, b.count, a.bf16);
  const NsPlan pl = ns_plan(a.steps, a.coef, choice.first);
  const bool small = choice.small;
  const int64_t ldn = small ? np : ns_pitch(np), ldm = small ? mp : ns_pitch(mp);  // row pitches
  NsPtrs p{};
  NsOutPtrs o{};
  for (int i = 0; i < b.count; ++i) {
    p.x[i] = a.muon ? (const void*)b.grad[i] : b.x[i];
    p.state[i] = b.state[i];
    p.id[i] = o.id[i] = (uint8_t)b.id[i];
    o.W[i] = b.W[i];
    o.o[i] = a.muon ? b.W_lp[i] : b.o[i];
  }
  NsEw e{};
  e.numel = n * m;
  e.rows_n = (int)n;
  e.cols_m = (int)m;
  e.np = (int)np;
  e.mp = (int)ldm;
  e.tall = b.tall;
  e.eps = a.eps;
  e.momentum = a.momentum;
  e.first = a.first;
  e.nesterov = a.nesterov;
  e.clip_frac = a.clip_update ? 0.0 : a.clip_frac;
  e.grad_sumsq = a.grad_sumsq;
  e.W_sumsq = a.W_sumsq;
  e.clip_scale = a.clip_update ? nullptr : a.clip_scale;
  e.part = s.norm_part;
  const int nblk = (int)std::min<int64_t>(kNsNormBlocks, ceil_div(n * m, 4096));
  const dim3 tiles((unsigned)(mp / kNsEdge), (unsigned)(np / kNsEdge), (unsigned)b.count);
  const float pow_in = (float)std::ldexp(1.0, pl.groups[0].e_X);
  if (a.muon) {
    FPO_LAUNCH("muon_momentum", st,
               (ns_norm_kernel<float, true><<<dim3(nblk, b.count), dim3(256), 0, st>>>(e, p)));
    FPO_CHECK_LAUNCH();
    FPO_LAUNCH("ns_convert", st,
               (ns_convert_kernel<float, true, PAIR><<<tiles, dim3(256), 0, st>>>(e, p, s.Xa, s.Xat, pow_in, nblk)));
  } else {
    FPO_LAUNCH("ns_norm", st, (ns_norm_kernel<T, false><<<dim3(nblk, b.count), dim3(256), 0, st>>>(e, p)));
    FPO_CHECK_LAUNCH();
    FPO_LAUNCH("ns_convert", st,
               (ns_convert_kernel<T, false, PAIR><<<tiles, dim3(256), 0, st>>>(e, p, s.Xa, s.Xat, pow_in, nblk)));
  }
  FPO_CHECK_LAUNCH();

  // what becomes of the last X
  NsFinish f{};
  f.R[0] = f.C[1] = (int)n;
  f.C[0] = f.R[1] = (int)m;
  f.mp = (int)ldm;
  f.tall = b.tall;
  f.pow2 = (float)std::ldexp(1.0, -pl.e_out);
  f.part = s.part;
  f.dsq = s.dsq;
  const auto scale = [&](double rows, double cols) {
    return a.scale == kNsScaleRms        ? 0.2 * std::sqrt(std::max(rows, cols))
           : a.scale == kNsScaleSpectral ? std::sqrt(std::max(1.0, rows / cols))
                                         : 1.0;
  };
  f.step[0] = (float)(a.lr * scale((double)n, (double)m));
  f.step[1] = (float)(a.lr * scale((double)m, (double)n));
  f.decay = (float)(1.0 - a.lr * a.weight_decay);
  f.lr_wd = (float)(a.lr * a.weight_decay);
  f.clip_update = a.clip_update;
  f.clip_frac = a.clip_frac;
  f.W_sumsq = a.W_sumsq;
  f.clip_scale = a.clip_scale;

  NsMat X = s.Xa, Y = s.Xb, XT = s.Xat, YT = s.Xbt;
  // C = 2^shift A B of square operands; more sets are added for the same launch
  const auto product = [&](const NsMat& l, const NsMat& r, const NsMat& out, double alpha) {
    NsGemmArgs g{};
    g.a[0] = l;
    g.b[0] = r;
    g.c[0] = out;
    g.lda = g.ldb = g.ldc = (int)ldn;
    g.M = g.N = g.K = (int)np;
    g.count = b.count;
    g.alpha[0] = (float)alpha;
    return g;
  };
  const auto launch = [&](auto what, const char* name, const NsGemmArgs& g, int sets) {
    constexpr int kWhat = decltype(what)::value;
    return small ? launch_small_product(kWhat, name, g, PAIR, NsMat{}, NsMat{}, false, nullptr, st)
                 : launch_product<kWhat, PAIR>(name, g, sets, st);
  };
  constexpr std::integral_constant<int, kGram> gram;
  constexpr std::integral_constant<int, kPoly> poly;
  constexpr std::integral_constant<int, kMul> mul;
  hipError_t err;
  for (int gi = 0; gi < pl.ngroups; ++gi) {
    const NsGroup& gr = pl.groups[gi];
    const NsStep* sp = &pl.steps[gr.first];
    {  // A = X X^T
      NsGemmArgs g = product(X, X, s.A, std::ldexp(1.0, sp[0].e_A - 2 * gr.e_X));
      g.lda = g.ldb = (int)ldm;
      g.K = (int)mp;
      if ((err = launch(gram, "ns_gram", g, 1)) != hipSuccess) return err;
    }
    int q = 0;  // P[q]: the product of the B so far; the other two are free
    for (int j = 0; j < gr.count; ++j) {
      const int bj = j ? (q + 1) % 3 : 0, qn = j ? (q + 2) % 3 : 0;
      {  // P[bj] = B_j = a I + b A + c A A
        NsGemmArgs g = product(s.A, s.A, s.P[bj], sp[j].c * std::ldexp(1.0, sp[j].e_B - 2 * sp[j].e_A));
        g.beta = (float)(sp[j].b * std::ldexp(1.0, sp[j].e_B - sp[j].e_A));
        g.eye = (float)(sp[j].a * std::ldexp(1.0, sp[j].e_B));
        if ((err = launch(poly, "ns_poly", g, 1)) != hipSuccess) return err;
      }
      // the product of the B, and B A on the way to the next A = B A B, in one launch
      const bool more = j + 1 < gr.count;
      int sets = 0;
      NsGemmArgs g = product(s.P[bj], s.A, s.C, 0.0);
      if (more) g.alpha[sets++] = (float)std::ldexp(1.0, sp[j].e_C - sp[j].e_B - sp[j].e_A);
      if (j) {
        g.a[sets] = s.P[bj];
        g.b[sets] = s.P[q];
        g.c[sets] = s.P[qn];
        g.alpha[sets++] = (float)std::ldexp(1.0, sp[j].e_Q - sp[j].e_B - sp[j - 1].e_Q);
      }
      if (sets && (err = launch(mul, "ns_mul", g, sets)) != hipSuccess) return err;
      if (more) {
        g = product(s.C, s.P[bj], s.A, std::ldexp(1.0, sp[j + 1].e_A - sp[j].e_C - sp[j].e_B));
        if ((err = launch(mul, "ns_mul", g, 1)) != hipSuccess) return err;
      }
      q = qn;
    }
    // X <- Q X
    const int e_next = gi + 1 < pl.ngroups ? pl.groups[gi + 1].e_X : pl.e_out;
    NsGemmArgs g = product(s.P[q], X, Y, std::ldexp(1.0, e_next - gr.e_X - sp[gr.count - 1].e_Q));
    g.ldb = g.ldc = (int)ldm;
    g.N = (int)mp;
    if (small) {
      g.b[0] = XT;
      // the last one finishes the caller's matrices, unless the clip needs the whole step's norm first
      const bool end = gi + 1 == pl.ngroups, fused = end && !a.clip_update;
      const NsLast last{f, o, a.muon ? kApply : kWriteO};
      err = launch_small_product(kApplyX, fused && a.muon ? "muon_apply" : "ns_apply", g, PAIR, X, end ? NsMat{} : YT,
                                 end, fused ? &last : nullptr, st);
    } else {
      err = launch_product<kApplyX, PAIR>("ns_apply", g, 1, st);
    }
    if (err != hipSuccess) return err;
    std::swap(X, Y);
    std::swap(XT, YT);
  }

  if (!a.muon) {
    if (!small) {
      FPO_LAUNCH("ns_write", st, (ns_finish_kernel<T, kWriteO, PAIR><<<tiles, dim3(256), 0, st>>>(f, o, X)));
      FPO_CHECK_LAUNCH();
    }
    return hipSuccess;
  }
  const int64_t ntiles = (np / kNsEdge) * (mp / kNsEdge);
  if (a.clip_update) {
    FPO_LAUNCH("muon_delta", st, (ns_finish_kernel<T, kDelta, PAIR><<<tiles, dim3(256), 0, st>>>(f, o, X)));
    FPO_CHECK_LAUNCH();
    FPO_LAUNCH("muon_reduce", st,
               ns_reduce_kernel<<<dim3(b.count), dim3(256), 0, st>>>(s.part, ntiles, s.dsq, nullptr, o));
    FPO_CHECK_LAUNCH();
  }
  if (!small || a.clip_update) {
    FPO_LAUNCH("muon_apply", st, (ns_finish_kernel<T, kApply, PAIR><<<tiles, dim3(256), 0, st>>>(f, o, X)));
    FPO_CHECK_LAUNCH();
  }
  if (a.W_sumsq) {
    FPO_LAUNCH("muon_reduce", st,
               ns_reduce_kernel<<<dim3(b.count), dim3(256), 0, st>>>(s.part, ntiles, nullptr, a.W_sumsq, o));
    FPO_CHECK_LAUNCH();
  }
  return hipSuccess;
}

}  // namespace

size_t ns_workspace(int64_t n, int64_t m, int count, bool bf16) { return ns_carve(n, m, count, bf16, nullptr).bytes; }

hipError_t launch_ns(const NsLaunch& a, const NsBatch& b) {
  return a.bf16 ? run_ns<uint16_t, false>(a, b) : run_ns<float, true>(a, b);
}

}  // namespace fpo
