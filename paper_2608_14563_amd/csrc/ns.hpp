// Orthogonalisation by Newton-Schulz products (host side): how the steps are
// grouped into products, the power of two each matrix is stored with, and the
// launch description of fpo_orthogonalize and fpo_muon_update.
#pragma once

#include <stdint.h>

#include <cmath>
#include <algorithm>

#include "launch.hpp"

namespace fpo {

constexpr int kNsMaxSteps = 32;

// One step maps every singular value s of X to p(s) = a s + b s^3 + c s^5, that is
// X' = B X with B = a I + b A + c A^2 and A = X X^T (n x n, n the shorter side).
struct NsStep {
  double a, b, c;
  double r_in;      // bound of X's largest singular value before the step (X starts with Frobenius norm <= 1)
  double r_out;     // and after it
  double b_max;     // bound of B's largest eigenvalue magnitude
  int e_A, e_B, e_C, e_Q;  // stored as 2^e times the value: A, B, B A, the group's product of the B
};

// Steps [first, first + count) of one group: all their B are formed from A by n x n
// products (the next A is B A B), and X is multiplied once, by the product of the B.
struct NsGroup {
  int first, count;
  int e_X;  // exponent of the X that the group reads
};

struct NsPlan {
  int nsteps = 0, ngroups = 0;
  NsStep steps[kNsMaxSteps];
  NsGroup groups[kNsMaxSteps];
  int e_out = 0;     // exponent of the last X
  bool ok = false;   // false: the coefficients let X grow without bound
};

// Exponent for values of magnitude up to `bound`: 2^13 at most, an eighth of fp16's
// largest, so that rounding errors that a step enlarges have room too.
inline int ns_exponent(double bound) {
  int e = 0;
  std::frexp(bound > 1e-30 ? bound : 1e-30, &e);  // bound < 2^e
  const int r = 13 - e;
  return r > 40 ? 40 : r;
}

// Largest |a + b l + c l^2| over l in [0, top].
inline double ns_poly_max(double a, double b, double c, double top) {
  auto f = [&](double l) { return std::fabs(a + b * l + c * l * l); };
  double m = f(0.0) > f(top) ? f(0.0) : f(top);
  if (c != 0.0) {
    const double v = -b / (2 * c);
    if (v > 0.0 && v < top && f(v) > m) m = f(v);
  }
  return m;
}

// Largest |p(s)| over s in [0, top]: at the end or where p' = a + 3 b u + 5 c u^2 = 0, u = s^2.
inline double ns_value_max(double a, double b, double c, double top) {
  auto f = [&](double s) { return std::fabs(s * (a + b * s * s + c * s * s * s * s)); };
  double m = f(top);
  auto at = [&](double u) {
    if (u > 0.0 && u < top * top && f(std::sqrt(u)) > m) m = f(std::sqrt(u));
  };
  if (c != 0.0) {
    const double d = 9 * b * b - 20 * a * c;
    if (d >= 0.0) {
      at((-3 * b + std::sqrt(d)) / (10 * c));
      at((-3 * b - std::sqrt(d)) / (10 * c));
    }
  } else if (b != 0.0) {
    at(-a / (3 * b));
  }
  return m;
}

// Groups. With g steps in a group and r = m / n a group costs, in n x n x n half
// products, 3 r + 1 + 4 (g - 1): longer groups are cheaper, the more the wider X is.
// What limits them is rounding: A is rounded once a group, and B A B carries that error
// on, enlarged by up to b_max^2 a step, while X's small singular values rely on A's
// small eigenvalues. Relative error of five steps of (3.4445, -4.775, 2.0315) against
// 64 bits, fp16 with the diagonals' remainders (emulated), groups 3+2 / 2+1+2 / 2+2+1:
// token-summed outer products 512 x 1382 6.4e-4 / 5.3e-4 / 9.4e-4, 512 x 512 1.1e-3 /
// 1.0e-3 / 1.3e-3, 256 x 256 1.2e-3 / 9.7e-4 / 1.5e-3, 64 x 128 2.2e-3 / 7.4e-4 / 7.1e-4;
// six steps 2+2+2, 512 x 512 1.6e-3; five in one group overflow. So with fp16 products
// the first group takes three steps where that is cheaper by more than 7% (r >= 1.5,
// where the singular values of a matrix of full rank also keep away from zero) and the
// products' time is what counts (n >= 512: below, the launches' number, which is the
// same); otherwise, and with pairs, whose point is accuracy, it takes two. After it
// groups of one and two alternate, after one of three beginning with two. `first`: steps
// in the first group, 1: one in each. Coefficients that enlarge more close a group earlier
// (kNsGrowth is a little over 3.4445^4).
constexpr double kNsGrowth = 150.0;
constexpr double kNsMaxSigma = 1024.0;

inline NsPlan ns_plan(int steps, const double* coef, int first) {
  static const double kDefault[3] = {3.4445, -4.7750, 2.0315};
  NsPlan p;
  double r = 1.0;
  for (int i = 0; i < steps; ++i) {
    const double* k = coef ? coef + 3 * i : kDefault;
    NsStep s{};
    s.a = k[0];
    s.b = k[1];
    s.c = k[2];
    s.r_in = r;
    s.b_max = ns_poly_max(s.a, s.b, s.c, r * r);
    r = ns_value_max(s.a, s.b, s.c, r);
    s.r_out = r;
    if (!(r <= kNsMaxSigma) || !(s.b_max <= kNsMaxSigma * kNsMaxSigma)) return p;
    p.steps[p.nsteps++] = s;
  }
  for (int i = 0; i < steps;) {
    const int longest = i == 0 || first == 1 ? first : p.ngroups % 2 == first % 2 ? 2 : 1;
    NsGroup g{i, 1, ns_exponent(p.steps[i].r_in)};
    double growth = p.steps[i].b_max * p.steps[i].b_max, q = p.steps[i].b_max;
    while (g.count < longest && i + g.count < steps && growth <= kNsGrowth) {
      const double b = p.steps[i + g.count].b_max;
      growth *= b * b;
      ++g.count;
    }
    for (int j = 0; j < g.count; ++j) {
      NsStep& s = p.steps[i + j];
      if (j) q *= s.b_max;
      s.e_A = ns_exponent(s.r_in * s.r_in);
      s.e_B = ns_exponent(s.b_max);
      s.e_C = ns_exponent(s.b_max * s.r_in * s.r_in);
      s.e_Q = j ? ns_exponent(q) : s.e_B;
    }
    p.groups[p.ngroups++] = g;
    i += g.count;
  }
  p.e_out = ns_exponent(r);
  p.ok = true;
  return p;
}

// ---------------------------------------------------------------- launch
// Tiles of one M x N product (symmetric: M == N, those on and under the diagonal).
inline int64_t ns_tiles(int64_t M, int64_t N, int64_t edge, bool symmetric) {
  const int64_t tm = ceil_div(M, edge), tn = ceil_div(N, edge);
  return symmetric ? tm * (tm + 1) / 2 : tm * tn;
}

// How a launch of `mats` M x N products over K is cut, as big_tiles does: the first nbig
// 256 x 256 tiles as such, the others as 128 x 128 quarters; or (nbig 0) all as 128 x 128.
struct NsSplit {
  int64_t nbig;
  double us;
};
inline NsSplit ns_split(int64_t M, int64_t N, int64_t K, int64_t mats, bool symmetric) {
  const double kt = (double)ceil_div(K, 64);
  // (as in big_tiles, with this epilogue: stored twice, operands read again)
  auto big = [&](int64_t n) { return n ? (1.0 + 0.6 * (double)n / kCus) * kt + 20.0 : 0.0; };
  auto quarters = [&](int64_t n) { return (double)ceil_div(n, kCus) * (0.45 * kt + 8.0); };
  const int64_t n = mats * ns_tiles(M, N, 256, symmetric), rem = n % kCus, whole = n - rem;
  const double waves = (double)(n / kCus) * big(kCus);
  NsSplit best{n, waves + big(rem)};
  const double part = quarters(4 * rem) + 2.0;  // one more launch
  if (whole && rem && part < 0.85 * big(rem)) best = NsSplit{whole, waves + part};
  const double all = quarters(mats * ns_tiles(M, N, 128, symmetric));
  if (all < 0.85 * best.us) best = NsSplit{0, all};
  return best;
}

// How a batch of `count` matrices is computed: on 64 x 64 tiles (kernels_ns_small.hip) or
// large ones, and the number of steps in the first group (ns_plan), by the least estimated
// time of the products of five steps.
//  * Up to 256 small tiles take 4.2 us and 4.3 ns a K entry (pairs 4.6 and 9.5), more of
//    them 4.6 us and, per 256, 3.6 us and 2.7 ns a K entry (5 and 6.5). Measured, us small /
//    large: fp16, 64 x 168 75 / 116, 512 x 1376 125 / 199, eight of them 242 / 239, 1024 x
//    1024 137 / 238, eight 444 / 477, three 1536 x 4144 820 / 553. Pairs, 256 x 688 129 /
//    240, eight 512 x 1376 394 / 418, three 1536 x 4144 1810 / 1435.
//  * One step a group takes three launches a step (15), groups of 2, 1, 2 take 17: fewer
//    where a launch's latency is what counts.
//  * Three steps in the first group of the large tiles: see ns_plan.
struct NsChoice {
  bool small;
  int first;
};
inline double ns_small_us(int64_t tiles, int64_t K, bool bf16) {
  if (tiles <= kCus) return bf16 ? 4.2 + 0.0043 * (double)K : 4.6 + 0.0095 * (double)K;
  return 4.6 + (double)tiles / kCus * (bf16 ? 3.6 + 0.0027 * (double)K : 5.0 + 0.0065 * (double)K);
}
inline NsChoice ns_choose(int64_t n, int64_t m, int count, bool bf16) {
  const int64_t np = ceil_div(n, 64) * 64, mp = ceil_div(m, 64) * 64;
  auto small = [&](int64_t N, int64_t K, bool sym) { return ns_small_us(count * ns_tiles(np, N, 64, sym), K, bf16); };
  auto large = [&](int64_t N, int64_t K, bool sym) {
    return ns_split(np, N, K * (bf16 ? 1 : 3), count, sym).us + 1.5;
  };
  const double g = small(np, mp, true), s = small(np, np, true), x = small(mp, np, false);
  const double one = 5 * g + 5 * s + 5 * x, two = 3 * g + 11 * s + 3 * x;
  const double big = 3 * large(np, mp, true) + 11 * large(np, np, true) + 3 * large(mp, np, false);
  if (std::min(one, two) < big) return {true, one < two ? 1 : 2};
  return {false, bf16 && n >= 512 && 2 * m >= 3 * n ? 3 : 2};
}

constexpr int kNsNormBlocks = 512;   // workgroups (and partials) a matrix of the norm pass
constexpr int kNsEdge = 64;          // edge of the tiles of the elementwise passes; n and m are padded to it

inline int64_t ns_pad(int64_t v) { return ceil_div(v, kNsEdge) * kNsEdge; }

// Row pitch of a padded side p on the large tiles: an odd multiple of 256 bytes, so that
// the rows of a K tile lie in different L2 channels (X X^T of nine 4096 x 12288, whose
// plain pitch is 24 KB: 1805 -> 1541 us; products of 4096 x 4096 matrices 2% less).
inline int64_t ns_pitch(int64_t p) {
  const int64_t q = ceil_div(p, 128) * 128;
  return q / 128 % 2 ? q : q + 128;
}

// The matrices of one call that share (n, m), n the shorter side: one batch of launches.
struct NsBatch {
  int count;
  int64_t n, m;               // true sizes, n <= m
  int id[kMaxMats];           // the caller's index (of the per-matrix device arrays)
  uint64_t tall;              // bit i: matrix i has more rows than columns
  // fpo_orthogonalize: x read (f32 or bf16), o written in the same type.
  const void* x[kMaxMats];
  void* o[kMaxMats];
  // fpo_muon_update
  const float* grad[kMaxMats];
  float* state[kMaxMats];     // null entries: no momentum
  float* W[kMaxMats];
  void* W_lp[kMaxMats];
};

enum { kNsScaleNone = 0, kNsScaleSpectral = 1, kNsScaleRms = 2 };  // fpo_muon_scale

struct NsLaunch {
  int steps;
  const double* coef;
  bool bf16;                  // element type of x, o, W_lp; bf16: fp16 products, f32: pairs of fp16
  double eps;
  bool muon;
  bool first, nesterov;
  float momentum;
  double clip_frac;
  bool clip_update;
  double lr, weight_decay;
  int scale;                  // fpo_muon_scale
  const double* grad_sumsq;
  double* W_sumsq;
  float* clip_scale;
  void* ws;
  void* stream;
};

// Matrices of one batch at most. A batch's smallest launches (n x n, tiles on and under
// the diagonal) should fill the CUs several times; a larger one only costs workspace.
inline int ns_batch_limit(int64_t n) {
  const int64_t t = ceil_div(n, 256), tri = t * (t + 1) / 2;
  const int64_t want = ceil_div(8 * kCus, tri);
  return (int)std::min<int64_t>(kMaxMats, std::max<int64_t>(want, 4));
}

size_t ns_workspace(int64_t n, int64_t m, int count, bool bf16);
hipError_t launch_ns(const NsLaunch& a, const NsBatch& b);

}  // namespace fpo
