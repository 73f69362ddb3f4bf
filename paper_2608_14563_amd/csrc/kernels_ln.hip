// Layer norm over the last dimension, forward and VJP with the gradients of gain and
// bias (fpo_layernorm, fpo_layernorm_vjp):
//   mu = mean x, sigma = sqrt(mean (x - mu)^2 + eps), y = gain (x - mu) / sigma + bias
//   v = gain dy, sigma~ = max(sigma, min_std), x^ = (x - mu) / sigma~
//   dx = (v - mean v - x^ mean(v x^)) / sigma~
//   dgain = sum_t dy (x - mu) / sigma, dbias = sum_t dy
// Both are bound by HBM: a row is read once into registers, its statistics are two
// reductions over the lanes that share it (the squares are of differences from the
// mean, so that a large mean costs only the digits of its own rounding), and everything else is elementwise.
//
// A row is shared by 16 lanes (d up to 128), 32 (256), 64 (1024 or 2048), 256 (up to 4096),
// 512 (8192) or 1024 (16384), each holding up to four chunks of eight neighbouring elements; longer rows are
// read again for every reduction. A workgroup takes every grid-th row, loading the next
// one before the current one's reductions, and keeps gain (and bias) in registers (8192 x
// 4096 bf16 forward 32 -> 27 us, 5.0 TB/s: they were as many bytes from L2 as x and y). In
// the VJP it also keeps its columns' sums of the two parameter gradients in registers; the
// workgroups' sums go to the workspace and a second launch adds them in a fixed order (no
// atomics: the same input gives the same bits). Next to HBM the vector instructions count
// too, some 14 an element in the VJP, a third of the memory time if nothing waits; hence
// the products are shared between the sums (8192 x 4096, bf16 x and dx_lp, float32 dy and
// dx: 87 us, 4.6 TB/s; a wave a row, 128 sums a lane and one wave a SIMD, had nothing to
// hide a row's loads behind, 112 us).
#include "common.hpp"
#include "launch.hpp"
#include "prof.hpp"

namespace fpo {

namespace {

typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Raw8;  // eight stored elements
template <>
struct Raw8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4*>(p);
    b = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ __forceinline__ f32x8 get() const { return f32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}; }
};
template <>
struct Raw8<uint16_t> {
  u32x4 a;
  __device__ __forceinline__ void load(const uint16_t* p) { a = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ f32x8 get() const {
    return f32x8{bf16_lo(a.x), bf16_hi(a.x), bf16_lo(a.y), bf16_hi(a.y),
                 bf16_lo(a.z), bf16_hi(a.z), bf16_lo(a.w), bf16_hi(a.w)};
  }
};
__device__ __forceinline__ void store8(float* p, f32x8 v) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(uint16_t* p, f32x8 v) {
  *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                       pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ float sum8(f32x8 v) {
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// Sum over the LANES lanes of a row; up to 64: within the wave, else the workgroup is one
// row's. `red` holds 3 x 16 floats.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* red) {
  if constexpr (LANES <= 64) return wave_sum<LANES>(v);
  else return block_sum(v, red);
}
// Three of them in one exchange.
template <int LANES>
__device__ __forceinline__ void row_sum3(float& a, float& b, float& c, float* red) {
  a = wave_sum<std::min(LANES, 64)>(a);
  b = wave_sum<std::min(LANES, 64)>(b);
  c = wave_sum<std::min(LANES, 64)>(c);
  if constexpr (LANES > 64) {
    const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
    __syncthreads();
    if (l == 0) {
      red[w] = a;
      red[16 + w] = b;
      red[32 + w] = c;
    }
    __syncthreads();
    a = b = c = 0.f;
    for (int i = 0; i < LANES / kWave; ++i) {  // fixed order
      a += red[i];
      b += red[16 + i];
      c += red[32 + i];
    }
  }
}

constexpr int ln_threads(int lanes) { return lanes < 256 ? 256 : lanes; }

// NV: chunks a lane (of 8 elements, LANES chunks apart); 0: any number, read again.
template <typename T, int LANES, int NV>
__global__ __launch_bounds__(ln_threads(LANES)) void ln_forward_kernel(const T* __restrict__ x, const T* __restrict__ gain,
                                                                      const T* __restrict__ bias, int64_t rows, int d,
                                                                      float eps, T* __restrict__ y,
                                                                      float* __restrict__ mean_out,
                                                                      float* __restrict__ rstd_out) {
  __shared__ float red[32];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  constexpr int SLOTS = ln_threads(LANES) / LANES;
  const int nc = d / 8;
  const float inv_d = 1.f / (float)d;
  constexpr int NR = NV ? NV : 1;
  Raw8<T> rx[NR], rg[NR], rb[NR];  // the next row; gain and bias, kept for all of a workgroup's rows
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int k = 0; k < NR; ++k)
      if (lane + k * LANES < nc) rx[k].load(x + row * d + 8 * (lane + k * LANES));
  };
  const int64_t step = (int64_t)gridDim.x * SLOTS;
  int64_t row = (int64_t)blockIdx.x * SLOTS + slot;
  if constexpr (NV > 0) {
    if (row < rows) fetch(row);
#pragma unroll
    for (int k = 0; k < NR; ++k)
      if (lane + k * LANES < nc) {
        if (gain) rg[k].load(gain + 8 * (lane + k * LANES));
        if (bias) rb[k].load(bias + 8 * (lane + k * LANES));
      }
  }
  // (with several slots a row's lanes are in one wave, and nothing in the loop is a barrier)
  for (; row < rows; row += step) {
    f32x8 v[NR];
    float s = 0.f;
    auto each = [&](auto&& f) {  // f(chunk, k, values): every chunk of the lane
      if constexpr (NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (lane + k * LANES < nc) f(lane + k * LANES, k, v[k]);
      } else {
        for (int c = lane; c < nc; c += LANES) {
          Raw8<T> r;
          r.load(x + row * d + 8 * c);
          f(c, 0, r.get());
        }
      }
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) v[k] = rx[k].get();
      if (row + step < rows) fetch(row + step);
    }
    each([&](int, int, const f32x8& t) { s += sum8(t); });
    const float mean = row_sum<LANES>(s, red) * inv_d;
    s = 0.f;
    each([&](int, int, f32x8 t) {
      t -= mean;
      s += sum8(t * t);
    });
    const float rstd = 1.f / sqrtf(row_sum<LANES>(s, red) * inv_d + eps);
    each([&](int c, int k, f32x8 t) {
      t = (t - mean) * rstd;
      if constexpr (NV == 0) {
        if (gain) rg[0].load(gain + 8 * c);
        if (bias) rb[0].load(bias + 8 * c);
      }
      if (gain) t *= rg[k].get();
      if (bias) t += rb[k].get();
      store8(y + row * d + 8 * c, t);
    });
    if (lane == 0) {
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
  }
}

struct LnVjp {
  const void* x;
  const void* gain;
  const void* dy;
  float* dx;
  void* dx_lp;
  float* pgain;  // [gridDim.x][d] sums of a workgroup's rows (the results, with one workgroup), or null
  float* pbias;
  int64_t rows;
  int d;
  float eps, min_std;
};

// PARAM: sums for dgain and dbias are kept, in registers, or with NV == 0 (very long
// rows) in the workgroup's partials themselves, each entry only ever touched by one lane.
template <typename T, typename TD, int LANES, int NV, bool PARAM>
__global__ __launch_bounds__(ln_threads(LANES)) void ln_vjp_kernel(LnVjp a) {
  constexpr int SLOTS = ln_threads(LANES) / LANES;
  constexpr int NR = NV ? NV : 1;
  constexpr bool AHEAD = NV > 0 && LANES < 1024;  // (1024 lanes have no registers left for it)
  __shared__ float red[48];
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
  const T* x = (const T*)a.x;
  const TD* dy = (const TD*)a.dy;
  const T* gain = (const T*)a.gain;
  T* dx_lp = (T*)a.dx_lp;
  const int d = a.d, nc = d / 8;
  const float inv_d = 1.f / (float)d;
  const int64_t step = (int64_t)gridDim.x * SLOTS;
  f32x8 pg[PARAM ? NR : 1], pb[PARAM ? NR : 1];
  if constexpr (PARAM) {
#pragma unroll
    for (int k = 0; k < NR; ++k) pg[k] = pb[k] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  }
  Raw8<T> rx[NR];
  Raw8<TD> rd[NR];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int k = 0; k < NR; ++k)
      if (lane + k * LANES < nc) {
        rx[k].load(x + row * d + 8 * (lane + k * LANES));
        rd[k].load(dy + row * d + 8 * (lane + k * LANES));
      }
  };
  auto gain8 = [&](int c) {
    f32x8 g = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (gain) {
      Raw8<T> r;
      r.load(gain + 8 * c);
      g = r.get();
    }
    return g;
  };
  constexpr bool KEEP_GAIN = (NV == 1 || NV == 2) && LANES < 1024;  // (else there are no registers left)
  f32x8 gv[KEEP_GAIN ? NR : 1];
  if constexpr (KEEP_GAIN) {
#pragma unroll
    for (int k = 0; k < NR; ++k)
      if (lane + k * LANES < nc) gv[k] = gain8(lane + k * LANES);
  }
  int64_t row = (int64_t)blockIdx.x * SLOTS + slot;
  if constexpr (AHEAD) {
    if (row < a.rows) fetch(row);
  }
  // with several slots a row's lanes are in one wave and nothing in the loop is a barrier
  for (; row < a.rows; row += step) {
    f32x8 vx[NR], vd[NR];
    auto each = [&](auto&& f) {  // f(chunk, k, x, dy, gain)
      if constexpr (NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (lane + k * LANES < nc) {
            if constexpr (KEEP_GAIN) f(lane + k * LANES, k, vx[k], vd[k], gv[k]);
            else f(lane + k * LANES, k, vx[k], vd[k], gain8(lane + k * LANES));
          }
      } else {
        for (int c = lane; c < nc; c += LANES) {
          Raw8<T> r;
          Raw8<TD> q;
          r.load(x + row * d + 8 * c);
          q.load(dy + row * d + 8 * c);
          f(c, 0, r.get(), q.get(), gain8(c));
        }
      }
    };
    if constexpr (NV > 0) {
      if constexpr (!AHEAD) fetch(row);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        vx[k] = rx[k].get();
        vd[k] = rd[k].get();
      }
    }
    if constexpr (AHEAD) {
      if (row + step < a.rows) fetch(row + step);
    }
    float s = 0.f;
    each([&](int, int, const f32x8& t, const f32x8&, const f32x8&) { s += sum8(t); });
    const float mean = row_sum<LANES>(s, red) * inv_d;
    float ss[2] = {0.f, 0.f}, c1[2] = {0.f, 0.f}, c2[2] = {0.f, 0.f};  // of (x - mean)^2, v, v (x - mean)
    each([&](int, int, const f32x8& t, const f32x8& g, const f32x8& gn) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xc = t[e] - mean;
        ss[e & 1] = fmaf(xc, xc, ss[e & 1]);
        c1[e & 1] = fmaf(g[e], gn[e], c1[e & 1]);
        c2[e & 1] = fmaf(g[e] * xc, gn[e], c2[e & 1]);
      }
    });
    float sq = ss[0] + ss[1], m1 = c1[0] + c1[1], m2 = c2[0] + c2[1];
    row_sum3<LANES>(sq, m1, m2, red);
    const float sigma = sqrtf(sq * inv_d + a.eps);
    const float rstd = 1.f / sigma, inv = 1.f / fmaxf(sigma, a.min_std);
    // dx = (v - mean v - x^ mean(v x^)) / sigma~ = inv v - o1 - o2 (x - mean)
    const float o1 = m1 * inv_d * inv, o2 = m2 * inv_d * inv * inv * inv;
    each([&](int c, int k, const f32x8& t, const f32x8& g, const f32x8& gn) {
      f32x8 o, pr;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xc = t[e] - mean;
        o[e] = fmaf(-o2, xc, fmaf(g[e], gn[e] * inv, -o1));
        if constexpr (PARAM) pr[e] = g[e] * xc;
      }
      if constexpr (PARAM && NV > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          pg[k][e] = fmaf(pr[e], rstd, pg[k][e]);
          pb[k][e] += g[e];
        }
      } else if constexpr (PARAM) {
        const int64_t at = (int64_t)blockIdx.x * d + 8 * c;
        const bool add = row != (int64_t)blockIdx.x;  // not the workgroup's first row
        auto keep = [&](float* p, f32x8 w) {
          if (!p) return;
          if (add) {
            Raw8<float> old;
            old.load(p + at);
            w += old.get();
          }
          store8(p + at, w);
        };
        keep(a.pgain, pr * rstd);
        keep(a.pbias, g);
      }
      if (a.dx) store8(a.dx + row * d + 8 * c, o);
      if (dx_lp) store8(dx_lp + row * d + 8 * c, o);
    });
  }
  if constexpr (PARAM && NV > 0) {
    if constexpr (SLOTS == 1) {
#pragma unroll
      for (int k = 0; k < NR; ++k)
        if (lane + k * LANES < nc) {
          const int64_t at = (int64_t)blockIdx.x * d + 8 * (lane + k * LANES);
          if (a.pgain) store8(a.pgain + at, pg[k]);
          if (a.pbias) store8(a.pbias + at, pb[k]);
        }
    } else {  // the slots' sums, in a fixed order
      __shared__ f32x8 part[SLOTS][LANES];
#pragma unroll
      for (int k = 0; k < NR; ++k)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          __syncthreads();
          part[slot][lane] = which ? pb[k] : pg[k];
          __syncthreads();
          float* out = which ? a.pbias : a.pgain;
          if (slot == 0 && out && lane + k * LANES < nc) {
            f32x8 t = part[0][lane];
#pragma unroll
            for (int w = 1; w < SLOTS; ++w) t += part[w][lane];
            store8(out + (int64_t)blockIdx.x * d + 8 * (lane + k * LANES), t);
          }
        }
    }
  }
}

// Column sums of the workgroups' partials, dgain with blockIdx.y == 0, dbias with 1: 32
// columns (a line) a workgroup, 16 rows of partials at a time, added in double; eight
// loads of a lane are in flight.
__global__ __launch_bounds__(512) void ln_reduce_kernel(const float* __restrict__ pgain, const float* __restrict__ pbias,
                                                        int n, int d, float* dgain, float* dbias) {
  __shared__ double part[16][32];
  const float* p = blockIdx.y ? pbias : pgain;
  float* out = blockIdx.y ? dbias : dgain;
  if (!out) return;
  const int c = threadIdx.x % 32, r = threadIdx.x / 32, col = blockIdx.x * 32 + c;
  double s = 0.0;
  if (col < d) {
    int i = r;
    for (; i + 112 < n; i += 128) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p[(int64_t)(i + 16 * k) * d + col];
#pragma unroll
      for (int k = 0; k < 8; ++k) s += (double)v[k];
    }
    for (; i < n; i += 16) s += (double)p[(int64_t)i * d + col];
  }
  part[r][c] = s;
  __syncthreads();
  if (r == 0 && col < d) {
    for (int i = 1; i < 16; ++i) s += part[i][c];
    out[col] = (float)s;
  }
}

constexpr int kLnForwardBlocks = 4 * kCus;  // workgroups of the forward pass
constexpr int kLnBlocks = 2048;              // workgroups of the VJP without parameter gradients

// How rows of d elements are held: lanes a row and chunks a lane (0: read again).
struct LnShape {
  int lanes, nv;
};
// Rows of up to 256 elements, as norms of single heads have them, share a wave (2^20 x 128
// bf16: forward 318 -> 107 us, VJP 617 -> 192 us, 4.9 and 5.5 TB/s).
// Rows too few for four of them to a workgroup on every CU have a workgroup each. Between
// 1032 and 2048 elements a wave a row is quicker in the forward pass (16384 x 2048: 26 us
// against 33 with 256 lanes) and slower in the VJP, whose sums then leave one wave a SIMD
// too few (84 against 72).
LnShape ln_shape(int64_t T, int64_t d, bool vjp) {
  const int64_t nc = d / 8;
  const bool few = T < 4 * kCus;
  if (nc <= 16) return {16, 1};
  if (nc <= 32) return {32, 1};
  if (nc <= 64) return {64, 1};
  if (nc <= 128) return few ? LnShape{256, 1} : LnShape{64, 2};
  if (nc <= 256) return few || vjp ? LnShape{256, 1} : LnShape{64, 4};
  if (nc <= 512) return {256, 2};
  if (nc <= 1024) return {512, 2};
  if (nc <= 2048) return {1024, 2};  // (1024 lanes leave 128 registers each)
  return {1024, 0};
}

// f(std::integral_constant lanes, nv) for the shape
template <class F>
void with_shape(LnShape s, F&& f) {
  if (s.lanes == 16) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
  else if (s.lanes == 32) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
  else if (s.lanes == 64 && s.nv == 1) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else if (s.lanes == 64 && s.nv == 2) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
  else if (s.lanes == 64) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
  else if (s.lanes == 256 && s.nv == 1) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  else if (s.lanes == 256 && s.nv == 2) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
  else if (s.lanes == 512) f(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
  else if (s.nv == 2) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 0>{});
}

#define FPO_CHECK_LAUNCH()             \
  do {                                 \
    hipError_t e_ = hipGetLastError(); \
    if (e_ != hipSuccess) return e_;   \
  } while (0)

template <typename T>
hipError_t run_forward(const LnLaunch& a) {
  hipStream_t st = (hipStream_t)a.stream;
  with_shape(ln_shape(a.T, a.d, false), [&](auto lanes, auto nv) {
    constexpr int kThreads = ln_threads(lanes), kSlots = kThreads / lanes;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.T, kSlots), kLnForwardBlocks));
    FPO_LAUNCH("ln_forward", st,
               (ln_forward_kernel<T, lanes, nv><<<grid, dim3(kThreads), 0, st>>>(
                   (const T*)a.x, (const T*)a.gain, (const T*)a.bias, a.T, (int)a.d, a.eps, (T*)a.y, a.mean, a.rstd)));
  });
  FPO_CHECK_LAUNCH();
  return hipSuccess;
}

template <typename T, typename TD>
hipError_t run_vjp(const LnLaunch& a) {
  hipStream_t st = (hipStream_t)a.stream;
  const LnShape sh = ln_shape(a.T, a.d, true);
  const bool param = a.dgain || a.dbias;
  const int64_t groups = ceil_div(a.T, ln_threads(sh.lanes) / sh.lanes);
  const int n = param ? ln_vjp_blocks(a.T, a.d) : (int)std::min<int64_t>(groups, kLnBlocks);
  const bool direct = n == 1;  // one workgroup's sums are the results
  LnVjp v{a.x, a.gain, a.dy, a.dx, a.dx_lp, nullptr, nullptr, a.T, (int)a.d, a.eps, a.min_std};
  if (a.dgain) v.pgain = direct ? a.dgain : a.part;
  if (a.dbias) v.pbias = direct ? a.dbias : a.part + (int64_t)n * a.d;
  with_shape(sh, [&](auto lanes, auto nv) {
    if (param)
      FPO_LAUNCH("ln_vjp", st,
                 (ln_vjp_kernel<T, TD, lanes, nv, true><<<dim3(n), dim3(ln_threads(lanes)), 0, st>>>(v)));
    else
      FPO_LAUNCH("ln_vjp", st,
                 (ln_vjp_kernel<T, TD, lanes, nv, false><<<dim3(n), dim3(ln_threads(lanes)), 0, st>>>(v)));
  });
  FPO_CHECK_LAUNCH();
  if (param && !direct) {
    FPO_LAUNCH("ln_reduce", st,
               ln_reduce_kernel<<<dim3((unsigned)ceil_div(a.d, 32), 2), dim3(512), 0, st>>>(v.pgain, v.pbias, n,
                                                                                           (int)a.d, a.dgain, a.dbias));
    FPO_CHECK_LAUNCH();
  }
  return hipSuccess;
}

}  // namespace

int ln_vjp_blocks(int64_t T, int64_t d) {
  const LnShape s = ln_shape(T, d, true);
  // about as many workgroups a CU as their registers let run at once; another one more has
  // another row of partials to write and read
  const int per_cu = s.lanes <= 64 ? 2 : s.lanes == 256 ? (s.nv == 1 ? 3 : 2) : 1;
  const int64_t groups = ceil_div(T, ln_threads(s.lanes) / s.lanes);
  // Few rows are left to one workgroup, whose sums are the results: another turn of it takes
  // 0.8 us (64 lanes a row) to 2 us (d 8192), the second launch 2.5 us and 3 us of the host.
  // Eager, T 16, d 512: 9.5 -> 6.7 us; 2 x 4096: 9.5 -> 6.8; 2 x 8192: 9.4 -> 6.9. From a graph
  // two turns gain (8 x 512: 5.3 -> 4.2 us; 2 x 4096: 6.3 -> 5.9; 2 x 8192: 7.1 -> 7.0), four lose
  // (16 x 512: 5.4 -> 6.0; 32 x 256: 5.5 -> 5.9; 64 x 128: 6.0 -> 6.2) less than they gain eager.
  if (groups <= (s.lanes <= 64 ? 4 : s.lanes <= 512 ? 2 : 1)) return 1;
  return (int)std::min<int64_t>(groups, kCus * per_cu);
}

hipError_t launch_layernorm(const LnLaunch& a) {
  return a.bf16 ? run_forward<uint16_t>(a) : run_forward<float>(a);
}

hipError_t launch_layernorm_vjp(const LnLaunch& a) {
  if (a.bf16) return a.dy_bf16 ? run_vjp<uint16_t, uint16_t>(a) : run_vjp<uint16_t, float>(a);
  return a.dy_bf16 ? run_vjp<float, uint16_t>(a) : run_vjp<float, float>(a);
}

}  // namespace fpo
