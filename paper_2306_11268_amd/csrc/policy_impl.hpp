// Policy over device levels: levels drawn for several rollouts, their
// log-probabilities, and the clipped policy loss with its gradient.
//
// All three are streaming passes over rows of logits [count][K].  A row of up
// to kPolicyRowMax levels sits in the registers of G lanes, N values each, as
// many lanes as keep N at 4 to 16 (32 past 1024 levels): several rows share a
// wave, so that the steps of a reduction over lanes serve all of them at once.
// A longer row takes a workgroup.  Memory bounds them (a large copy reaches 5.0
// TB/s on this card): draws of four rollouts for 200000 x 256 logits 175 us (5.9
// TB/s, reading only), log-probabilities of eight for 612500 x 64 41 us, the
// loss and gradient of 16 rollouts for 200000 x 256 97 us (4.6 TB/s).
#pragma once

#include "kernels.hpp"
#include "tile.hpp"

namespace lr {

constexpr int kPolicyRowMax = 2048;
constexpr int kPolicyThreads = 256;
constexpr int kPolicyCus = 256;  // of the MI355X
constexpr int kLdsUnit = 1280;   // bytes that shared memory is given out by
constexpr int kLdsUnits = 128;   // of a CU

// ---- reductions on the vector ALU (no shared memory) -----------------------
// Lanes 1, 2, 4, 8 apart through DPP (where pairs, quads, ... already agree, the
// mirrored lane is as good as the one 4 or 8 apart), 16 and 32 apart through
// the row swaps; every lane of the group ends with the result.
template <int G, class Op>
__device__ __forceinline__ float lanes_reduce(float x, Op op) {
  auto dpp = [&](auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  if constexpr (G >= 2) x = op(x, dpp(std::integral_constant<int, 0xB1>{}));   // quad_perm [1,0,3,2]
  if constexpr (G >= 4) x = op(x, dpp(std::integral_constant<int, 0x4E>{}));   // quad_perm [2,3,0,1]
  if constexpr (G >= 8) x = op(x, dpp(std::integral_constant<int, 0x141>{}));  // row_half_mirror
  if constexpr (G >= 16) x = op(x, dpp(std::integral_constant<int, 0x140>{})); // row_mirror
  if constexpr (G >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (G >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return x;
}
struct OpSum {
  __device__ float operator()(float a, float b) const { return a + b; }
};
struct OpMax {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct OpMin {
  __device__ float operator()(float a, float b) const { return fminf(a, b); }
};

template <int G>
__device__ __forceinline__ double lanes_sum_d(double x) {
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// N values over a workgroup of THREADS, in a fixed order.  One barrier: red is
// free for the next call only behind another one.
template <int THREADS, int N, class Op>
__device__ __forceinline__ void block_reduce(float (&x)[N], Op op, float (&red)[N][THREADS / 64]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = lanes_reduce<64>(x[i], op);
    if ((threadIdx.x & 63) == 0) red[i][threadIdx.x >> 6] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = red[i][0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) x[i] = op(x[i], red[i][w]);
  }
}
// (red: THREADS / 64 values, free again at the end)
template <int THREADS>
__device__ __forceinline__ double block_sum_d(double x, double* red) {
  x = lanes_sum_d<64>(x);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int i = 1; i < THREADS / 64; ++i) x += red[i];
  __syncthreads();
  return x;
}

// ---- rows in registers -----------------------------------------------------
// A lane's values are runs of four neighbouring levels: value i of lane l of G
// is column ((i / 4) G + l) 4 + i % 4.  16-byte loads need only the alignment
// of one float here, so that rows of any length and place are read alike; TAIL:
// the last run of a row that is no multiple of four goes value by value.
struct __attribute__((packed, aligned(4))) Quad {
  float v[4];
};
struct __attribute__((packed, aligned(2))) QuadBf16 {
  uint32_t v[2];
};
template <int G>
__device__ __forceinline__ int quad_col(int lane, int i) {
  return ((i / 4) * G + lane) * 4;
}
// Columns c .. c + 3 of a row of K; those past the end are `past`.
template <bool TAIL>
__device__ __forceinline__ void quad_read(const float* __restrict__ p, int K, int c, float past, float* v) {
  if (TAIL ? c + 4 <= K : c < K) {
    const Quad q = *reinterpret_cast<const Quad*>(p + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = q.v[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = TAIL && j < 3 && c + j < K ? p[c + j] : past;
  }
}
// (K = 0 for a row that is not there)
template <int G, bool TAIL, int N>
__device__ __forceinline__ void row_read(const float* __restrict__ p, int K, int lane, float past, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) quad_read<TAIL>(p, K, quad_col<G>(lane, i), past, &v[i]);
}

constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Barred levels: far below, but finite, so that 0 times their logarithm is 0.
// (The maximum drops a NaN; its exponential, formed from the value itself,
// keeps it.)
__device__ __forceinline__ float floor_d(float d) { return fmaxf(d, -1e30f); }

// Two values rounded to bf16, nearest even (gfx950 converts them in one
// instruction; in integer arithmetic it was six a value).
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){a, b}, b2));
}

// The tile that is worked as number t.  Workgroups go to the eight XCDs in turn,
// so that cache lines which the choices of neighbouring tiles share would be
// fetched or completed once for each XCD's L2: every XCD takes runs of tiles
// instead, ROWS rows long, as far as whole runs for all of them go.  (Draws of
// four rollouts, 200000 x 256: 180 -> 175 us, 50000 x 1000: 175 -> 166;
// log-probabilities of eight, 612500 x 64: 43.0 -> 41.4, of 16, 200000 x 256: 44 ->
// 39, of 32, 612500 x 16: 43.0 -> 40.3.  The loss keeps the plain order, though it
// fetches such lines more than once: 97 us either way at 256 levels and 71 at 16,
// 69 -> 73 at 32, 91 -> 95 at 2048.)
template <int T, int ROWS>
__device__ __forceinline__ long long tile_at(long long t, long long tiles) {
  constexpr int RUN = ROWS / T;
  const long long first = t / (8 * RUN) * (8 * RUN);
  if (first + 8 * RUN > tiles) return t;
  const int i = (int)(t - first);
  return first + i % 8 * RUN + i / 8;
}
constexpr int kRunRows = 2048;
constexpr int kRunLongRows = 32;

// ---- draw ------------------------------------------------------------------
// One lane of the row's holds the level drawn and its logit, and writes.
__device__ __forceinline__ void draw_write(const PolicyDrawArgs& a, long long o, int act, float d, float lz) {
  a.actions[o] = act;
  if (a.logp) a.logp[o] = d - lz;
  if (a.phi) a.phi[o] = a.levels[act];
}

// Best score of this lane's columns and its place: the first of equals (a
// lane's columns ascend with i); NaN compares false.
struct Best {
  float score = -INFINITY;
  float x = 0.f;
  int k;
  __device__ __forceinline__ explicit Best(int K) : k(K) {}
  __device__ __forceinline__ void take(float xi, float ni, int c) {
    const float v = xi + ni;
    const bool better = v > score;
    score = better ? v : score;
    k = better ? c : k;
    x = better ? xi : x;
  }
};
// The row's winner writes (level numbers are exact in float32): top and first
// are the reductions of all lanes' scores and of the columns that reach it.
__device__ __forceinline__ void best_write(const PolicyDrawArgs& a, long long o, const Best& b, float top, float first,
                                           bool lane0, float x0, float m, float lz) {
  const int act = (int)first;
  if (act < a.K) {
    if (b.k == act && b.score == top) draw_write(a, o, act, b.x - m, lz);
  } else if (lane0) {
    draw_write(a, o, 0, x0 - m, lz);
  }
}

template <int G, int N, bool TAIL>
__global__ void __launch_bounds__(kPolicyThreads) policy_draw_rows_kernel(PolicyDrawArgs a) {
  constexpr int T = kPolicyThreads / G;
  const int lane = threadIdx.x % G;
  const long long tiles = (a.count + T - 1) / T;
  for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
    const long long r = tile_at<T, kRunRows>(t, tiles) * T + threadIdx.x / G;
    const bool ok = r < a.count;
    const int K = ok ? a.K : 0;
    float x[N];
    row_read<G, TAIL>(a.logits + r * a.K, K, lane, -INFINITY, x);
    float n[2][N];
    row_read<G, TAIL>(a.noise + r * a.K, K, lane, 0.f, n[0]);
    float m = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
    m = lanes_reduce<G>(m, OpMax{});
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) z += exp_fast(x[i] - m);
    const float lz = logf(lanes_reduce<G>(z, OpSum{}));
    auto one = [&](int s, float (&now)[N], float (&next)[N]) {
      if (s + 1 < a.samples)
        row_read<G, TAIL>(a.noise + ((long long)(s + 1) * a.count + r) * a.K, K, lane, 0.f, next);
      Best b(a.K);
#pragma unroll
      for (int i = 0; i < N; ++i) b.take(x[i], now[i], quad_col<G>(lane, i) + i % 4);
      const float top = lanes_reduce<G>(b.score, OpMax{});
      const float first = lanes_reduce<G>(b.score == top ? (float)b.k : (float)a.K, OpMin{});
      if (ok) best_write(a, (long long)s * a.count + r, b, top, first, lane == 0, x[0], m, lz);
    };
    for (int s = 0; s < a.samples; s += 2) {
      one(s, n[0], n[1]);
      if (s + 1 < a.samples) one(s + 1, n[1], n[0]);
    }
  }
}

// ---- long rows: a workgroup each, streamed -----------------------------------
// Running maximum, sum of exponentials and of exponential times distance from
// the maximum; the maximum starts finite, so that barred levels (-inf) leave 0.
struct Running {
  float m = -3.402823466e38f;
  float z = 0.f;
  float zd = 0.f;
  __device__ __forceinline__ void rescale(float to) {
    const float d = m - to;  // <= 0
    const float f = exp_fast(d);
    zd = f > 0.f ? f * (zd + d * z) : 0.f;  // (nothing is left far below, where d z is beyond float32)
    z *= f;
    m = to;
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N]) {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
    if (top > m) rescale(top);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = x[i] - m;
      const float e = exp_fast(d);
      z += e;
      zd += e * floor_d(d);
    }
  }
};

// Threads of a row's workgroup, and values that each has in flight: with 512 of
// 16, rows of little more than 2048 levels leave most threads idle, and waves
// wait at the barriers (four rollouts of 10000 x 2500: 217 us against 110 with 256
// of 8, 10000 x 5000 227 against 183); longer ones need the bytes in flight when
// there are few of them (eight rollouts of 100 x 50000: 54 us against 104).
template <int THREADS_, int PER_>
struct LongShape {
  static constexpr int THREADS = THREADS_, PER = PER_, STEP = THREADS_ * PER_;
};
constexpr int kLongSamples = 4;  // rollouts that one pass over the logits serves

template <class S>
__global__ void __launch_bounds__(S::THREADS) policy_draw_long_kernel(PolicyDrawArgs a) {
  constexpr int THREADS = S::THREADS;
  constexpr int ALL = kLongSamples;
  __shared__ float red_max[ALL + 1][THREADS / 64];
  __shared__ float red_sum[1][THREADS / 64];
  __shared__ float red_min[ALL][THREADS / 64];
  const int lane = threadIdx.x;
  for (long long r = blockIdx.x; r < a.count; r += gridDim.x) {
    const float* __restrict__ row = a.logits + r * a.K;
    Running w;
    float lz = 0.f;
    for (int s0 = 0; s0 < a.samples; s0 += ALL) {
      Best b[ALL] = {Best(a.K), Best(a.K), Best(a.K), Best(a.K)};
      for (int k0 = 0; k0 < a.K; k0 += S::STEP) {
        float x[S::PER];
        row_read<THREADS, true>(row + k0, a.K - k0, lane, -INFINITY, x);
#pragma unroll
        for (int s = 0; s < ALL; ++s) {
          if (s0 + s >= a.samples) break;
          float n[S::PER];
          row_read<THREADS, true>(a.noise + ((long long)(s0 + s) * a.count + r) * a.K + k0, a.K - k0, lane, 0.f, n);
#pragma unroll
          for (int i = 0; i < S::PER; ++i) b[s].take(x[i], n[i], k0 + quad_col<THREADS>(lane, i) + i % 4);
        }
        if (s0 == 0) w.add(x);
      }
      float top[ALL + 1] = {b[0].score, b[1].score, b[2].score, b[3].score, w.m};
      block_reduce<THREADS>(top, OpMax{}, red_max);
      if (s0 == 0) {
        w.rescale(top[ALL]);
        float z[1] = {w.z};
        block_reduce<THREADS>(z, OpSum{}, red_sum);
        lz = logf(z[0]);
      }
      float first[ALL];
#pragma unroll
      for (int s = 0; s < ALL; ++s) first[s] = b[s].score == top[s] ? (float)b[s].k : (float)a.K;
      block_reduce<THREADS>(first, OpMin{}, red_min);
#pragma unroll
      for (int s = 0; s < ALL; ++s) {
        if (s0 + s >= a.samples) break;
        best_write(a, (long long)(s0 + s) * a.count + r, b[s], top[s], first[s], lane == 0, row[0], w.m, lz);
      }
    }
  }
}

// ---- log-probabilities of given levels ---------------------------------------
__device__ __forceinline__ float logp_of(const float* __restrict__ row, int act, int K, float m, float lz) {
  if (act < 0) return 0.f;
  return act < K ? (row[act] - m) - lz : __builtin_nanf("");
}

template <int G, int N, bool TAIL>
__global__ void __launch_bounds__(kPolicyThreads) policy_logp_rows_kernel(PolicyDrawArgs a) {
  constexpr int T = kPolicyThreads / G;
  __shared__ float2 stat[T];
  const int lane = threadIdx.x % G;
  const int row = threadIdx.x / G;
  const long long tiles = (a.count + T - 1) / T;
  for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
    const long long r0 = tile_at<T, kRunRows>(t, tiles) * T;
    float x[N];
    row_read<G, TAIL>(a.logits + (r0 + row) * a.K, r0 + row < a.count ? a.K : 0, lane, -INFINITY, x);
    float m = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
    m = lanes_reduce<G>(m, OpMax{});
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) z += exp_fast(x[i] - m);
    z = lanes_reduce<G>(z, OpSum{});
    if (lane == 0) stat[row] = make_float2(m, logf(z));
    __syncthreads();
    for (int q = threadIdx.x; q < a.samples * T; q += kPolicyThreads) {
      const long long r = r0 + q % T;
      if (r >= a.count) continue;
      const long long o = (long long)(q / T) * a.count + r;
      const float2 of = stat[q % T];
      a.logp[o] = logp_of(a.logits + r * a.K, a.actions[o], a.K, of.x, of.y);
    }
    __syncthreads();
  }
}

template <class S>
__global__ void __launch_bounds__(S::THREADS) policy_logp_long_kernel(PolicyDrawArgs a) {
  constexpr int THREADS = S::THREADS;
  __shared__ float red_max[1][THREADS / 64];
  __shared__ float red_sum[1][THREADS / 64];
  for (long long t = blockIdx.x; t < a.count; t += gridDim.x) {
    const long long r = tile_at<1, kRunLongRows>(t, a.count);
    const float* __restrict__ row = a.logits + r * a.K;
    Running w;
    for (int k0 = 0; k0 < a.K; k0 += S::STEP) {
      float x[S::PER];
      row_read<THREADS, true>(row + k0, a.K - k0, threadIdx.x, -INFINITY, x);
      w.add(x);
    }
    float m[1] = {w.m};
    block_reduce<THREADS>(m, OpMax{}, red_max);
    w.rescale(m[0]);
    float z[1] = {w.z};
    block_reduce<THREADS>(z, OpSum{}, red_sum);
    const float lz = logf(z[0]);
    for (int s = threadIdx.x; s < a.samples; s += THREADS) {
      const long long o = (long long)s * a.count + r;
      a.logp[o] = logp_of(row, a.actions[o], a.K, w.m, lz);
    }
  }
}

// ---- the loss ----------------------------------------------------------------
// One choice of a rollout.
struct Choice {
  int act;  // < 0: none
  float old, ref, adv;
};
// Place o of the [samples][count] arrays, k bytes on; o_adv and k_adv of the
// advantages, which may be [samples].  (o in scalar registers where a wave shares
// it: a load then needs no address arithmetic.)
template <class T>
__device__ __forceinline__ T read_at(const T* p, long long o, unsigned k) {
  return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(p + o) + k);
}
__device__ __forceinline__ void choice_read(const PolicyLossArgs& a, long long o, unsigned k, long long o_adv,
                                            unsigned k_adv, Choice& c) {
  c.act = read_at(a.actions, o, k);
  c.old = read_at(a.old_logp, o, k);
  if (a.ref_logp) c.ref = read_at(a.ref_logp, o, k);
  c.adv = read_at(a.adv, o_adv, k_adv);
}
// What the choices of one thread add to the loss's terms.
struct Terms {
  float gain = 0.f, kl = 0.f, entropy = 0.f, cut = 0.f;
};
// The wave's sums of them, in float32 over its lanes, added to sum in float64.
__device__ __forceinline__ void terms_add(const Terms& t, double* sum) {
  const float gain = lanes_reduce<64>(t.gain, OpSum{});
  const float kl = lanes_reduce<64>(t.kl, OpSum{});
  const float entropy = lanes_reduce<64>(t.entropy, OpSum{});
  const float cut = lanes_reduce<64>(t.cut, OpSum{});
  if ((threadIdx.x & 63) == 0) {
    sum[0] -= (double)gain;
    sum[1] += (double)kl;
    sum[2] += (double)entropy;
    sum[3] += (double)cut;
  }
}
// A choice under the present logits.  d: its level's logit minus the row's
// maximum.
struct Ratio {
  float logp, ratio, border;
  float over;  // > 0: on the clipped side
  __device__ __forceinline__ Ratio(const PolicyLossArgs& a, const Choice& c, float d, float lz) {
    logp = d - lz;
    ratio = exp_fast(logp - c.old);
    const bool up = c.adv >= 0.f;
    border = up ? a.border_high : a.border_low;
    over = ratio - border;
    over = up ? over : -over;
  }
  // So near to the border that float32 may put it on the wrong side.  With u = 2^-24 the ratio is off, relative to
  // itself, by
  //   |d| u + |logp| u       the roundings of d and of logp = d - lz (|d| <= |logp| + lz),
  //   2 lz u + s u           the logarithm, and the sum of exponentials before it: 191 u at 65536 levels (128 values of
  //                          a lane one after another, 6 steps of lanes, 7 of waves, 3 u in each of 8 rounds for a new
  //                          maximum, and 2 u + 2.22 u |d| of an exponential, |d| log 65536 in the mean at most),
  //   3.3 |logp - old| u + 4 u  the difference, its exponential and the border.
  // logp is at most 0 and the border at least u or 0, so logp - old is at least -16.7 beside a border, and at most |old|:
  // together within (3.3 |old| + 3 lz + 290) u.  row (of open_row) and the factor of |old| hold 436 u + 6 u lz and 6 u.
  __device__ __forceinline__ bool open(const Choice& c, float row) const {
    return fabsf(over) <= border * fmaf(fabsf(c.old), 3.6e-7f, row);
  }
  // A level out of range.
  __device__ __forceinline__ void spoil() { logp = ratio = over = __builtin_nanf(""); }
};
__device__ __forceinline__ float open_row(float lz) { return 3.6e-7f * lz + 2.6e-5f; }
// dl/dlogp (times scale) of a choice that was made; its gain and KL added to t.
__device__ __forceinline__ float choice_slope(const PolicyLossArgs& a, const Choice& c, const Ratio& r, Terms& t) {
  const bool cut = r.over > 0.f;
  const float g = r.ratio * c.adv;
  t.gain += cut ? r.border * c.adv : g;
  float slope = cut ? 0.f : -g;
  if (a.ref_logp) {
    // q = e^k - 1 - k: by its series where the difference would cancel; e = e^k - 1 from q there, and elsewhere
    // from itself (far below zero, down to the -inf of a level that the reference bars, k + q would lose its -1)
    const float k = c.ref - r.logp;
    float q = 1.f / 3628800;
    q = q * k + 1.f / 362880;
    q = q * k + 1.f / 40320;
    q = q * k + 1.f / 5040;
    q = q * k + 1.f / 720;
    q = q * k + 1.f / 120;
    q = q * k + 1.f / 24;
    q = q * k + 1.f / 6;
    q = (q * k + 0.5f) * k * k;
    float e = k + q;
    if (__builtin_amdgcn_ballot_w64(!(fabsf(k) < 1.f))) {
      asm volatile("");  // (a branch, or every wave forms both)
      if (!(fabsf(k) < 1.f)) {
        e = exp_fast(k) - 1.f;
        q = e - k;
      }
    }
    t.kl += q;
    if (a.kl_coef != 0.f) slope -= a.kl_coef * e;  // (not 0 times infinity)
  }
  return slope * a.scale;
}
// e^x for |x| < 700 to about 1e-13: 2^k times the series of the rest, at most
// ln(2) / 2 (0.35^12 / 12! < 1e-14).  Rolled, its coefficients in memory: the
// library's function, or the coefficients in registers, would cost every wave
// of the kernel 40 to 100 registers for a path that few rows take.
__constant__ double kExpSeries[12] = {1. / 39916800, 1. / 3628800, 1. / 362880, 1. / 40320, 1. / 5040, 1. / 720,
                                      1. / 120,      1. / 24,      1. / 6,      0.5,        1.,        1.};
__device__ __forceinline__ double exp_d(double x) {
  const double k = __builtin_rint(x * 1.4426950408889634074);
  const double r = __builtin_fma(k, -0.69314718055994530942, x);
  double p = 0.;
#pragma unroll 1
  for (int i = 0; i < 12; ++i) p = __builtin_fma(p, r, kExpSeries[i]);
  return __builtin_ldexp(p, (int)k);
}
// Ratio::over in 64 bits, times z: ratio = e^(x - m - old) / z against the
// border, from the level's logit, the row's maximum and its sum of exponentials.
__device__ __forceinline__ float over_d(const PolicyLossArgs& a, const Choice& c, float x, float m, double z) {
  const double u = exp_d(fmin(fmax(((double)x - (double)m) - (double)c.old, -690.), 690.));
  return (float)(c.adv >= 0.f ? u - (1. + (double)a.clip_high) * z : (1. - (double)a.clip_low) * z - u);
}
// Sum of a row's exponentials in 64 bits, read again from memory by G lanes.
template <int G>
__device__ __forceinline__ double sum_exp_d(const float* row, int K, int lane, float m) {
  double z = 0.;
#pragma unroll 1
  for (int k = lane; k < K; k += G) z += exp_d(fmax((double)row[k] - (double)m, -690.));
  return z;
}
__device__ __forceinline__ double wave_sum_exp_d(const float* row, int K, float m) {
  return lanes_sum_d<64>(sum_exp_d<64>(row, K, threadIdx.x & 63, m));
}
// dL/dlogit = (sum of the slopes of choices of this level) - p (all slopes -
// w (log p + H)), w = scale * entropy_coef * choices made, p = e / z and
// log p = d - lz: acc - e / z (base - w d) with the row's base.
struct RowGrad {
  float base, w, inv_z;
  __device__ __forceinline__ RowGrad(const PolicyLossArgs& a, float slopes, float made, float inv_z_, float lz, float h)
      : w(a.scale * a.entropy_coef * made), inv_z(inv_z_) {
    base = slopes - w * (h - lz);
  }
  __device__ __forceinline__ float at(float acc, float e, float d) const { return acc - (e * inv_z) * (base - w * d); }
};
__device__ __forceinline__ void grad_store(void* grad, int bf16, long long at, float g) {
  if (bf16) static_cast<uint16_t*>(grad)[at] = (uint16_t)bf16_pair(g, 0.f);
  else static_cast<float*>(grad)[at] = g;
}
// Columns c .. c + 3 of a row that starts at `row` in the gradient.
template <bool TAIL>
__device__ __forceinline__ void quad_store(void* grad, int bf16, long long row, int K, int c, const float* g) {
  if (!TAIL || c + 4 <= K) {
    if (bf16) {
      const QuadBf16 q{{bf16_pair(g[0], g[1]), bf16_pair(g[2], g[3])}};
      *reinterpret_cast<QuadBf16*>(static_cast<uint16_t*>(grad) + row + c) = q;
    } else {
      *reinterpret_cast<Quad*>(static_cast<float*>(grad) + row + c) = Quad{{g[0], g[1], g[2], g[3]}};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (c + j < K) grad_store(grad, bf16, row + c + j, g[j]);
  }
}

// T rows a workgroup.  1. Their log-sum-exp, in registers; the logits (minus the
// maximum) also go to shared memory.  2. The choices of all rollouts, a thread
// each whatever the row's lanes are, read along the rows, find their logits
// there.  Their slopes are added to the row's levels in shared memory, by one
// lane in the order of the rollouts (the adds of one lane keep their order, so
// results do not change from run to run, also where rollouts chose the same
// level).  3. The gradient from registers.
//
// PARTS > 0, rows of few levels: the thread that forms a slope adds it, into one
// of the PARTS tables that the threads of a row have; the gradient joins them.
// Otherwise the choices' levels and slopes go to shared memory, `chunk` rollouts
// at a time, and a lane per row adds them in the logits' place.  (612500 rows of
// 16 levels, 32 rollouts: 165 us through the list, whose one adding wave the
// others wait for.)
//
// The phases wait for each other, so that the pass lives from many workgroups
// on a CU: nothing is carried from tile to tile but the terms, and the thread's
// number and K are made new for each, or the compiler holds 70 registers of
// addresses and comparisons across the loop.  Dynamic shared memory (K rounded
// up to four, or padded): float [1 + PARTS][T][K], the logits first; without
// tables float2 [chunk][T] behind them.
//
// Rows whose quads of four levels are a multiple of a power of two start on few
// of the 64 banks.  With tables, their quads change places, by a number that goes
// through that power (16 at most) over the rows that would meet, its high bits
// first (for stores of neighbouring quads): choices of one level then meet as if
// the rows were padded, without the padding's memory (612500 rows of 16 levels:
// 80 us padded, with four workgroups on a CU, 72 with five).  The list's rows,
// fewer and longer, are padded.
template <bool DIRECT>
__host__ __device__ constexpr int loss_stride(int K) {
  return (K + 3) / 4 * 4 + (DIRECT || (K + 3) / 4 % 2 ? 0 : 4);
}
template <bool DIRECT>
__device__ __forceinline__ int loss_swap(int K, int row) {
  if (!DIRECT) return 0;
  const int bits = min(__builtin_ctz((K + 3) / 4), 4);
  return (int)(__brev((unsigned)row >> (4 - bits)) >> 1 >> (31 - bits));
}

template <int G, int N, int PARTS, int WAVES, bool TAIL>
__global__ void __launch_bounds__(kPolicyThreads, WAVES) policy_loss_rows_kernel(PolicyLossArgs a, int chunk) {
  constexpr bool DIRECT = PARTS > 0;
  constexpr int T = kPolicyThreads / G;
  constexpr int TABLES = DIRECT ? PARTS : 1;
  constexpr int STEP = DIRECT ? PARTS : G;  // rollouts of a round: threads that take a row's choices
  extern __shared__ __align__(16) float lds[];
  __shared__ float2 stat[T];         // log of the sum of exponentials, entropy
  __shared__ float2 sums[TABLES][T];  // of the row's slopes and choices
  __shared__ float stat_m[T];
  __shared__ double terms[kPolicyThreads / 64][4];  // of each wave
  if (threadIdx.x < kPolicyThreads / 64 * 4) (&terms[0][0])[threadIdx.x] = 0.;
  const long long tiles = (a.count + T - 1) / T;
#pragma unroll 1
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    unsigned tid = threadIdx.x;
    int K = a.K;
    asm volatile("" : "+v"(tid));
    asm volatile("" : "+s"(K));
    const int lane = tid % G;
    const int row = tid / G;
    const int stride = loss_stride<DIRECT>(K);
    const int table = T * stride;
    float2* pairs = reinterpret_cast<float2*>(lds + table);
    float4* mine = reinterpret_cast<float4*>(lds + row * stride);
    const int swap = loss_swap<DIRECT>(K, row);
    const long long r0 = tile * T;
    const bool ok = r0 + row < a.count;
    const int mine_row = tid % T;  // whose choices this thread takes, STEP rollouts apart
    int part = tid / T;
    if constexpr (T % 64 == 0) part = __builtin_amdgcn_readfirstlane(part);
    const bool live = r0 + mine_row < a.count;
    long long at = part * a.count + r0;
    long long adv_at = a.per_choice ? at : part;
    const long long adv_step = a.per_choice ? STEP * a.count : STEP;
    // The thread's next choice is read into c, or marked as none (its other numbers are then any).
    auto fetch = [&](int s, Choice& c) {
      c.act = -1;
      if (s < a.samples && part < STEP && live) {
        unsigned k = 4 * mine_row;
        if constexpr (T % 64 == 0) {
          asm volatile("" : "+v"(k));  // (or the arrays' places of this thread take eight registers)
          k &= 4 * T - 1;
        }
        choice_read(a, at, k, adv_at, a.per_choice ? k : 0u, c);
      }
    };
    Choice next{-1, 0.f, 0.f, 0.f};
    fetch(part, next);
    float d[N];
    row_read<G, TAIL>(a.logits + (r0 + row) * K, ok ? K : 0, lane, -INFINITY, d);
    float m = d[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, d[i]);
    m = lanes_reduce<G>(m, OpMax{});
    float z = 0.f;
    float zd = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      d[i] -= m;
      const float e = exp_fast(d[i]);
      d[i] = floor_d(d[i]);
      z += e;
      zd += e * d[i];
    }
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const int c = quad_col<G>(lane, i);
      if (c >= K) continue;
      mine[c / 4 ^ swap] = make_float4(d[i], d[i + 1], d[i + 2], d[i + 3]);
      if (DIRECT) {
#pragma unroll
        for (int p = 1; p <= TABLES; ++p) mine[p * (table / 4) + (c / 4 ^ swap)] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
    z = lanes_reduce<G>(z, OpSum{});
    zd = lanes_reduce<G>(zd, OpSum{});
    const float inv_z = 1.f / z;
    const float lz = logf(z);
    const float h = lz - zd * inv_z;
    if (lane == 0) {
      stat[row] = make_float2(lz, h);
      stat_m[row] = m;
    }
    float slopes = 0.f;
    float made = 0.f;
    Terms add;
    __syncthreads();
    const float2 row_stat = stat[mine_row];
    const float row_open = open_row(row_stat.x);
    const float row_m = stat_m[mine_row];
    const float* row_d = lds + mine_row * stride;
    float* row_add = lds + (DIRECT ? (1 + part) * table : 0) + mine_row * stride;
    const int swap_level = 4 * loss_swap<DIRECT>(K, mine_row);
    float chosen = 0.f;  // choices of this thread
    unsigned cuts = 0;   // of this wave, on the clipped side
    // The thread's next choice.  (A wave's lanes go through it together: those without one have act = -1.)
    auto choose = [&](int s, bool near_lds) {
      const Choice c = next;
      at += STEP * a.count;
      adv_at += adv_step;
      fetch(s + STEP, next);
      const int level = min(max(c.act, 0), K - 1);
      float dx;
      if (near_lds) dx = row_d[level ^ swap_level];
      else dx = floor_d(a.logits[live ? (r0 + mine_row) * K + level : 0] - row_m);
      Ratio ratio(a, c, dx, row_stat.x);
      const bool is_made = c.act >= 0;
      if (__builtin_amdgcn_ballot_w64(c.act >= K)) {
        asm volatile("");
        if (c.act >= K) {
          ratio.spoil();
          add.kl = add.entropy = add.cut = __builtin_nanf("");
        }
      }
      // undecided choices: the wave forms their rows' sums again, in 64 bits
      for (unsigned long long open = __builtin_amdgcn_ballot_w64(is_made && ratio.open(c, row_open)); open;
           open &= open - 1) {
        const int who = __builtin_ctzll(open);
        const float* p = a.logits + (r0 + __shfl(mine_row, who, 64)) * K;
        const double zr = wave_sum_exp_d(p, K, __shfl(row_m, who, 64));
        if ((int)(threadIdx.x & 63) == who) ratio.over = over_d(a, c, p[level], row_m, zr);
      }
      cuts += __popcll(__builtin_amdgcn_ballot_w64(is_made && ratio.over > 0.f));
      float slope = 0.f;
      if (is_made) {
        chosen += 1.f;
        slope = choice_slope(a, c, ratio, add);
      }
      return make_float2(__int_as_float(DIRECT ? (is_made ? level : -1) : c.act), slope);
    };
    auto collect = [&](float2 c) {
      const int act = __float_as_int(c.x);
      if (act >= 0) {
        made += 1.f;
        slopes += c.y;
        if (!DIRECT && act >= K) return;
        // (a place of this lane alone.  Where it has all of a row's rollouts, the atomic lets it go on without
        // the sum; where every lane adds, the atomics' rate would hold the pass: 612500 x 16, 32 rollouts 50 us more)
        if (DIRECT) row_add[act ^ swap_level] += c.y;
        else __hip_atomic_fetch_add(row_add + (act ^ swap_level), c.y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      }
    };
    if constexpr (DIRECT) {
      static_assert(T * PARTS % 64 == 0, "whole waves take choices");
      if (part < PARTS) {
#pragma unroll 1
        for (int s = 0; s < a.samples; s += STEP) collect(choose(s + part, true));
        sums[part][mine_row] = make_float2(slopes, made);
      }
    } else {
#pragma unroll 1
      for (int s0 = 0; s0 < a.samples; s0 += chunk) {
        const int s1 = min(s0 + chunk, a.samples);
#pragma unroll 1
        for (int s = s0; s < s1; s += STEP) {
          const float2 c = choose(s + part, s0 == 0);
          if (s + part < s1) pairs[(s + part - s0) * T + mine_row] = c;
        }
        __syncthreads();
        if (s0 == 0) {
#pragma unroll
          for (int i = 0; i < N; i += 4) {
            const int c = quad_col<G>(lane, i);
            if (c < K) mine[c / 4 ^ swap] = make_float4(0.f, 0.f, 0.f, 0.f);
          }
          __syncthreads();
        }
        if (tid < T) {
#pragma unroll 4
          for (int s = 0; s < s1 - s0; ++s) collect(pairs[s * T + mine_row]);
          sums[0][mine_row] = make_float2(slopes, made);
        }
        if (s1 < a.samples) __syncthreads();
      }
    }
    if (chosen > 0.f) add.entropy += chosen * row_stat.y;
    if (tid % 64 == 0) add.cut += (float)cuts;
    terms_add(add, terms[tid / 64]);
    __syncthreads();
    if (a.grad) {
      float2 all = sums[0][row];
#pragma unroll
      for (int p = 1; p < TABLES; ++p) {
        all.x += sums[p][row].x;
        all.y += sums[p][row].y;
      }
      const RowGrad to(a, all.x, all.y, inv_z, lz, h);
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const int c = quad_col<G>(lane, i);
        if (c >= K) continue;
        float4 q = mine[(DIRECT ? table / 4 : 0) + (c / 4 ^ swap)];
#pragma unroll
        for (int p = 2; p <= TABLES; ++p) {
          const float4 o = mine[p * (table / 4) + (c / 4 ^ swap)];
          q = make_float4(q.x + o.x, q.y + o.y, q.z + o.z, q.w + o.w);
        }
        const float s[4] = {q.x, q.y, q.z, q.w};
        float g[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          g[j] = all.y > 0.f ? to.at(s[j], exp_fast(d[i + j]), d[i + j]) : 0.f;
        if (ok) quad_store<TAIL>(a.grad, a.bf16, (r0 + row) * K, K, c, g);
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < 4) {
    double s = 0.;
    for (int w = 0; w < kPolicyThreads / 64; ++w) s += terms[w][threadIdx.x];
    a.part[4 * blockIdx.x + threadIdx.x] = s;
  }
}

// A workgroup per row of more than kPolicyRowMax levels.  HELD rounds of the
// row (16 values a thread each) stay in registers between the sums and the
// gradient, as many as still leave 16 waves to a CU, of two workgroups or more,
// so that one loads while another computes; what a longer row has beyond them is
// read again from the caches.  The gradient is written as if no level had been chosen;
// then the first rollout that chose a level adds the slopes of all that did, in
// their order, and writes that value again.  A thread's first choice and its
// logit are read before the row.
constexpr int kLongPer = 16;
template <int THREADS, int HELD>
__global__ void __launch_bounds__(THREADS, 4) policy_loss_long_kernel(PolicyLossArgs a) {
  constexpr int STEP = THREADS * kLongPer;
  __shared__ float red_max[1][THREADS / 64];
  __shared__ float red_sum[2][THREADS / 64];
  __shared__ double redd[THREADS / 64];
  __shared__ float2 pairs[kMaxRollouts];
  __shared__ double terms[THREADS / 64][4];  // of each wave
  if (threadIdx.x < THREADS / 64 * 4) (&terms[0][0])[threadIdx.x] = 0.;
#pragma unroll 1
  for (long long r = blockIdx.x; r < a.count; r += gridDim.x) {
    int tid = threadIdx.x;
    int K = a.K;
    asm volatile("" : "+v"(tid));
    asm volatile("" : "+s"(K));
    const float* __restrict__ row = a.logits + r * K;
    auto fetch = [&](int s, float& x) {
      Choice c{-1, 0.f, 0.f, 0.f};
      const long long at = (long long)s * a.count + r;
      choice_read(a, at, 0u, a.per_choice ? at : s, 0u, c);
      x = (unsigned)c.act < (unsigned)K ? row[c.act] : 0.f;
      return c;
    };
    auto slope_of = [&](const Choice& c, const Ratio& ratio, float h, Terms& t) {
      if (c.act < 0) return 0.f;
      t.entropy += h;
      t.cut += ratio.over > 0.f ? 1.f : 0.f;
      return choice_slope(a, c, ratio, t);
    };
    Choice c0{-1, 0.f, 0.f, 0.f};
    float x0 = 0.f;
    if (tid < a.samples) c0 = fetch(tid, x0);
    Running run;
    float held[HELD][kLongPer];
#pragma unroll
    for (int b = 0; b < HELD; ++b) {
      if ((b + 1) * STEP <= K) row_read<THREADS, false>(row + b * STEP, STEP, tid, -INFINITY, held[b]);
      else row_read<THREADS, true>(row + b * STEP, K - b * STEP, tid, -INFINITY, held[b]);
    }
#pragma unroll
    for (int b = 0; b < HELD; ++b)
      if (b * STEP < K) run.add(held[b]);
#pragma unroll 1
    for (int k0 = HELD * STEP; k0 < K; k0 += STEP) {
      float x[kLongPer];
      row_read<THREADS, true>(row + k0, K - k0, tid, -INFINITY, x);
      run.add(x);
    }
    float top[1] = {run.m};
    block_reduce<THREADS>(top, OpMax{}, red_max);
    run.rescale(top[0]);
    float z[2] = {run.z, run.zd};
    block_reduce<THREADS>(z, OpSum{}, red_sum);
    const float m = run.m;
    const float inv_z = 1.f / z[0];
    const float lz = logf(z[0]);
    const float h = lz - z[1] * inv_z;
    bool near = false;
    Terms add;
#pragma unroll 1
    for (int s = tid; s < a.samples; s += THREADS) {
      Choice c = c0;
      float x = x0;
      if (s != tid) c = fetch(s, x);
      const bool real = (unsigned)c.act < (unsigned)K;
      Ratio ratio(a, c, floor_d(x - m), lz);
      if (c.act >= K) {
        ratio.spoil();
        add.kl = add.entropy = add.cut = __builtin_nanf("");
      }
      const bool here = real && ratio.open(c, open_row(lz));
      near |= here;
      // (an undecided choice is left to the second pass)
      const float g = here ? 0.f : slope_of(c, ratio, h, add);
      pairs[s] = make_float2(__int_as_float(here ? -2 : (c.act < 0 ? -1 : c.act)), g);
    }
    if (__syncthreads_or(near)) {
      const double zr = block_sum_d<THREADS>(sum_exp_d<THREADS>(row, K, tid, m), redd);
#pragma unroll 1
      for (int s = tid; s < a.samples; s += THREADS) {
        if (__float_as_int(pairs[s].x) != -2) continue;
        float x;
        const Choice c = fetch(s, x);
        Ratio ratio(a, c, x - m, lz);
        ratio.over = over_d(a, c, x, m, zr);
        pairs[s] = make_float2(__int_as_float(c.act), slope_of(c, ratio, h, add));
      }
      __syncthreads();
    }
    terms_add(add, terms[tid / 64]);
    if (a.grad) {
      // (every wave for itself)
      float slopes = 0.f;
      float made = 0.f;
      for (int s = tid % 64; s < a.samples; s += 64) {
        const float2 c = pairs[s];
        made += __float_as_int(c.x) >= 0 ? 1.f : 0.f;
        slopes += __float_as_int(c.x) >= 0 ? c.y : 0.f;
      }
      slopes = lanes_reduce<64>(slopes, OpSum{});
      made = lanes_reduce<64>(made, OpSum{});
      const RowGrad to(a, slopes, made, inv_z, lz, h);
      auto write = [&](float (&x)[kLongPer], int k0) {
#pragma unroll
        for (int i = 0; i < kLongPer; ++i) {
          const float d = x[i] - m;
          x[i] = made > 0.f ? to.at(0.f, exp_fast(d), floor_d(d)) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kLongPer; i += 4)
          quad_store<true>(a.grad, a.bf16, r * K, K, k0 + quad_col<THREADS>(tid, i), &x[i]);
      };
#pragma unroll
      for (int b = 0; b < HELD; ++b)
        if (b * STEP < K) write(held[b], b * STEP);
#pragma unroll 1
      for (int k0 = HELD * STEP; k0 < K; k0 += STEP) {
        float x[kLongPer];
        row_read<THREADS, true>(row + k0, K - k0, tid, -INFINITY, x);
        write(x, k0);
      }
      __syncthreads();  // (the row's stores come before those below)
#pragma unroll 1
      for (int s = tid; s < a.samples; s += THREADS) {
        const int act = __float_as_int(pairs[s].x);
        if (act < 0 || act >= K) continue;
        float g = 0.f;
        bool first = true;
        for (int o = 0; o < a.samples; ++o) {
          const float2 c = pairs[o];
          if (__float_as_int(c.x) != act) continue;
          first &= o >= s;
          g += c.y;
        }
        if (!first) continue;
        const float d = (s == tid ? x0 : row[act]) - m;
        grad_store(a.grad, a.bf16, r * K + act, to.at(g, exp_fast(d), floor_d(d)));
      }
    }
    __syncthreads();
  }
  __syncthreads();
  if (threadIdx.x < 4) {
    double s = 0.;
    for (int w = 0; w < THREADS / 64; ++w) s += terms[w][threadIdx.x];
    a.part[4 * blockIdx.x + threadIdx.x] = s;
  }
}

// The loss and its four terms from n workgroups' partial sums [n][4], a thread
// for each and those of its kind a multiple of 1024 behind it.
__global__ void __launch_bounds__(1024) policy_finish_kernel(const double* __restrict__ part, int n, float kl, float ent,
                                                             float scale, float* loss, float* terms) {
  __shared__ double red[16][4];
  double s = 0.;
  for (int e = threadIdx.x; e < 4 * n; e += 1024) s += part[e];
#pragma unroll
  for (int o = 32; o >= 4; o >>= 1) s += __shfl_xor(s, o, 64);
  if (threadIdx.x % 64 < 4) red[threadIdx.x / 64][threadIdx.x % 64] = s;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  double t = 0.;
#pragma unroll
  for (int w = 0; w < 16; ++w) t += red[w][threadIdx.x % 4];
  t *= (double)scale;
  if (threadIdx.x < 4 && terms) terms[threadIdx.x] = (float)t;
  const double q = __shfl(t, 1, 64);
  const double h = __shfl(t, 2, 64);
  if (threadIdx.x == 0 && loss) *loss = (float)(t + (kl != 0.f ? (double)kl * q : 0.) - (double)ent * h);
}

// ---- launches ------------------------------------------------------------------
// Calls rows(Shape<G, N, TAIL>) for K <= kPolicyRowMax levels, else longs().
template <int G_, int N_, bool TAIL_>
struct Shape {
  static constexpr int G = G_, N = N_;
  static constexpr bool TAIL = TAIL_;
};
template <bool TAIL, class F>
static void policy_rows_shape(int K, F&& rows) {
  if (K <= 4) rows(Shape<1, 4, TAIL>{});
  else if (K <= 8) rows(Shape<2, 4, TAIL>{});
  else if (K <= 16) rows(Shape<4, 4, TAIL>{});
  else if (K <= 32) rows(Shape<4, 8, TAIL>{});
  else if (K <= 64) rows(Shape<8, 8, TAIL>{});
  else if (K <= 128) rows(Shape<8, 16, TAIL>{});
  else if (K <= 256) rows(Shape<16, 16, TAIL>{});
  else if (K <= 512) rows(Shape<32, 16, TAIL>{});
  else if (K <= 1024) rows(Shape<64, 16, TAIL>{});
  else rows(Shape<64, 32, TAIL>{});
}
// The loss's rows: also how many threads of a row add slopes, and the
// workgroups that a CU holds by their registers (without spilling any but two or
// three at 25 to 32 levels, where a sixth workgroup gives 3 %).  With tables every
// thread of a workgroup takes choices up to 24 levels, and half of them above, so
// rows share few lanes: 16 rollouts of 612500 x 17, 20, 24 61, 58, 59 us with four
// lanes a row, 49, 48, 50 with two, 32 rollouts of 612500 x 20 100, 85; 16 of 400000
// x 40 66 with eight, 51 with four, of 400000 x 64 82, 80.  Up to 48 levels rows of 12
// values a lane, not 16: 16 rollouts of 400000 x 33, 36, 40, 47, 48 55, 51, 52, 58, 52
// us with 16, 50, 47, 50, 55, 51 with 12.
template <int G_, int N_, int PARTS_, int WAVES_, bool TAIL_>
struct LossShape {
  static constexpr int G = G_, N = N_, PARTS = PARTS_, WAVES = WAVES_;
  static constexpr bool TAIL = TAIL_;
};
template <bool TAIL, class F>
static void loss_rows_shape(int K, F&& rows) {
  if (K <= 4) rows(LossShape<1, 4, 1, 6, TAIL>{});
  else if (K <= 8) rows(LossShape<1, 8, 1, 5, TAIL>{});
  else if (K <= 16) rows(LossShape<2, 8, 2, 5, TAIL>{});
  else if (K <= 24) rows(LossShape<2, 12, 2, 5, TAIL>{});
  else if (K <= 32) rows(LossShape<4, 8, 2, 6, TAIL>{});
  else if (K <= 48) rows(LossShape<4, 12, 2, 5, TAIL>{});
  else if (K <= 64) rows(LossShape<4, 16, 2, 4, TAIL>{});
  else if (K <= 128) rows(LossShape<8, 16, 0, 4, TAIL>{});
  else if (K <= 256) rows(LossShape<16, 16, 0, 4, TAIL>{});
  else if (K <= 512) rows(LossShape<32, 16, 0, 4, TAIL>{});
  else if (K <= 1024) rows(LossShape<64, 16, 0, 4, TAIL>{});
  else rows(LossShape<64, 32, 0, 3, TAIL>{});
}
template <class F, class L>
static void policy_shape(int K, F&& rows, L&& longs) {
  if (K > kPolicyRowMax) longs();
  else if (K % 4) policy_rows_shape<true>(K, rows);
  else policy_rows_shape<false>(K, rows);
}
template <int G>
static dim3 policy_grid(long long count, long long most) {
  const long long tiles = (count + kPolicyThreads / G - 1) / (kPolicyThreads / G);
  return dim3((unsigned)std::min(tiles, most));
}

hipError_t launch_policy_draw(const PolicyDrawArgs& a, hipStream_t st) {
  if (a.count <= 0 || a.samples <= 0) return hipSuccess;
  policy_shape(
      a.K,
      [&](auto s) {
        using S = decltype(s);
        const dim3 grid = policy_grid<S::G>(a.count, 1 << 16);
        if (a.noise) hipLaunchKernelGGL((policy_draw_rows_kernel<S::G, S::N, S::TAIL>), grid, dim3(kPolicyThreads), 0, st, a);
        else hipLaunchKernelGGL((policy_logp_rows_kernel<S::G, S::N, S::TAIL>), grid, dim3(kPolicyThreads), 0, st, a);
      },
      [&] {
        const dim3 grid((unsigned)std::min<long long>(a.count, 1 << 16));
        auto go = [&](auto s) {
          using S = decltype(s);
          if (a.noise) hipLaunchKernelGGL((policy_draw_long_kernel<S>), grid, dim3(S::THREADS), 0, st, a);
          else hipLaunchKernelGGL((policy_logp_long_kernel<S>), grid, dim3(S::THREADS), 0, st, a);
        };
        if (a.K <= 8192) go(LongShape<256, 8>{});
        else go(LongShape<512, 16>{});
      });
  return hipGetLastError();
}

hipError_t launch_policy_loss(const PolicyLossArgs& a, hipStream_t st) {
  if (a.count <= 0 || a.samples <= 0) return hipSuccess;
  dim3 grid;
  auto rows = [&](auto s) {
    using S = decltype(s);
    constexpr int T = kPolicyThreads / S::G;
    const int table = T * loss_stride<(S::PARTS > 0)>(a.K) * 4;
    // (the list: a whole number of the kernel's rounds of kPolicyThreads choices, in what leaves as many
    // workgroups to a CU's 160 KB as its registers do)
    const int fixed = 128 + (12 + 8 * std::max(1, S::PARTS)) * T;
    const int fit = (kLdsUnits / S::WAVES * kLdsUnit - fixed - table) / (8 * kPolicyThreads);
    const int rounds = (a.samples + S::G - 1) / S::G;
    const int chunk = std::max(1, std::min(rounds, std::min(fit, 8))) * S::G;
    const int lds = S::PARTS ? table * (1 + S::PARTS) : table + chunk * T * 8;
    // as many workgroups as run at once: a second, smaller round of them would leave CUs idle (400000 x 40, 16
    // rollouts: 64 us with one workgroup for each CU more than its shared memory takes, 51 without)
    static_assert(kPolicyCus * S::WAVES <= kPolicyParts, "partial sums");
    const int units = (lds + fixed + kLdsUnit - 1) / kLdsUnit;
    grid = policy_grid<S::G>(a.count, kPolicyCus * std::min(S::WAVES, kLdsUnits / units));
    hipLaunchKernelGGL((policy_loss_rows_kernel<S::G, S::N, S::PARTS, S::WAVES, S::TAIL>), grid, dim3(kPolicyThreads),
                       lds, st, a, chunk);
  };
  if (a.K > kPolicyRowMax) {
    grid = dim3((unsigned)std::min<long long>(a.count, kPolicyParts));
    // (Rounds held: what 128 registers a lane take, the most of which are a row's values, but for two or three that
    // workgroups of 128 and 256 spill; with a fourth round, or with 80 registers for six waves on a SIMD, many more.  1600 rows of 40007 in bf16 111 us with four
    // rounds, 97 with three; 1500 of 65536 194, 186.  Short rows in smaller workgroups, which wait for fewer waves:
    // 16 rollouts of 20000 x 2500 148 -> 121 us with 128 threads and two rounds after 256 with one, of 10000 x 5000
    // 134 -> 108 with 256 after 512.  1024 threads, which hold rows of 40007 whole but fill a CU alone: 139 -> 149.)
    auto go = [&](auto threads, auto held) {
      constexpr int THREADS = decltype(threads)::value;
      hipLaunchKernelGGL((policy_loss_long_kernel<THREADS, decltype(held)::value>), grid, dim3(THREADS), 0, st, a);
    };
    using std::integral_constant;
    if (a.K <= 2 * 128 * kLongPer) go(integral_constant<int, 128>{}, integral_constant<int, 2>{});
    else if (a.K <= 2 * 256 * kLongPer) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else go(integral_constant<int, 512>{}, integral_constant<int, 3>{});
  } else if (a.K % 4) {
    loss_rows_shape<true>(a.K, rows);
  } else {
    loss_rows_shape<false>(a.K, rows);
  }
  if (a.loss || a.terms)
    hipLaunchKernelGGL(policy_finish_kernel, dim3(1), dim3(1024), 0, st, a.part, (int)grid.x, a.kl_coef, a.entropy_coef,
                       a.scale, a.loss, a.terms);
  return hipGetLastError();
}

}  // namespace lr
