// Policy over device levels: levels drawn for several rollouts, their
// log-probabilities, and the clipped policy loss with its gradient.
#pragma once

#include "kernels.hpp"
#include "tile.hpp"

namespace lr {

__device__ __forceinline__ double block_sum_d(double x, double* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return ((red[0] + red[1]) + red[2]) + red[3];
}
__device__ __forceinline__ float block_max_f(float x, float* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

__device__ __forceinline__ uint16_t bf16_bits(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);  // (a NaN stays one)
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// One row per workgroup: the row's log-sum-exp in float64, then its samples.
__global__ void __launch_bounds__(256) policy_draw_kernel(PolicyDrawArgs a) {
  __shared__ double red[4];
  __shared__ float redf[4];
  __shared__ int best[256];
  for (long long r = blockIdx.x; r < a.count; r += gridDim.x) {
    const float* x = a.logits + r * a.K;
    float m = -INFINITY;
    for (int k = threadIdx.x; k < a.K; k += 256) m = fmaxf(m, x[k]);
    m = block_max_f(m, redf);
    double z = 0.;
    for (int k = threadIdx.x; k < a.K; k += 256) z += exp((double)x[k] - (double)m);
    const double lz = log(block_sum_d(z, red));
    for (int s = 0; s < a.samples; ++s) {
      const long long o = (long long)s * a.count + r;
      int act;
      if (a.noise) {
        const float* n = a.noise + o * a.K;
        float b = -INFINITY;
        int kb = a.K;
        for (int k = threadIdx.x; k < a.K; k += 256) {
          const float v = x[k] + n[k];
          if (v > b || (v == b && k < kb)) {
            b = v;
            kb = k;
          }
        }
        const float top = block_max_f(b, redf);
        best[threadIdx.x] = b == top ? kb : a.K;
        __syncthreads();
        act = a.K;
        for (int i = 0; i < 256; ++i) act = best[i] < act ? best[i] : act;
        if (act >= a.K) act = 0;
        __syncthreads();
      } else {
        act = a.actions[o];
      }
      if (threadIdx.x == 0) {
        if (a.noise) a.actions[o] = act;
        if (a.logp) {
          float lp = 0.f;
          if (act >= a.K) lp = __builtin_nanf("");
          else if (act >= 0) lp = (float)(((double)x[act] - (double)m) - lz);
          a.logp[o] = lp;
        }
        if (a.phi) a.phi[o] = a.levels[act];
      }
    }
  }
}

__global__ void __launch_bounds__(256) policy_loss_kernel(PolicyLossArgs a) {
  __shared__ double red[4];
  __shared__ float redf[4];
  double t[4] = {0., 0., 0., 0.};
  const double lo = 1. - (double)a.clip_low;
  const double hi = 1. + (double)a.clip_high;
  for (long long r = blockIdx.x; r < a.count; r += gridDim.x) {
    const float* x = a.logits + r * a.K;
    float m = -INFINITY;
    for (int k = threadIdx.x; k < a.K; k += 256) m = fmaxf(m, x[k]);
    m = block_max_f(m, redf);
    double z = 0.;
    double zd = 0.;
    for (int k = threadIdx.x; k < a.K; k += 256) {
      const double d = (double)x[k] - (double)m;
      const double e = exp(d);
      z += e;
      if (e > 0.) zd += e * d;
    }
    z = block_sum_d(z, red);
    const double lz = log(z);
    const double h = lz - block_sum_d(zd, red) / z;
    // every thread goes through all choices of the row
    double g_all = 0.;
    int made = 0;
    auto slope = [&](int s, double* terms) {
      const long long o = (long long)s * a.count + r;
      const int act = a.actions[o];
      if (act < 0) return 0.;
      if (act >= a.K) {
        terms[0] += __builtin_nan("");
        terms[1] += __builtin_nan("");
        terms[2] += __builtin_nan("");
        terms[3] += __builtin_nan("");
        return __builtin_nan("");
      }
      const double lp = ((double)x[act] - (double)m) - lz;
      const double ratio = exp(lp - (double)a.old_logp[o]);
      const double adv = a.per_choice ? a.adv[o] : a.adv[s];
      const bool cut = adv >= 0. ? ratio > hi : ratio < lo;
      double g = cut ? 0. : -ratio * adv;
      terms[0] -= (cut ? (adv >= 0. ? hi : lo) : ratio) * adv;
      if (a.ref_logp) {
        const double d = (double)a.ref_logp[o] - lp;
        terms[1] += expm1(d) - d;
        g -= (double)a.kl_coef * expm1(d);
      }
      terms[2] += h;
      terms[3] += cut ? 1. : 0.;
      return g;
    };
    double mine[4] = {0., 0., 0., 0.};
    for (int s = 0; s < a.samples; ++s) {
      g_all += slope(s, mine);
      made += a.actions[(long long)s * a.count + r] >= 0;
    }
    for (int i = 0; i < 4; ++i) t[i] += mine[i];
    if (a.grad) {
      for (int k = threadIdx.x; k < a.K; k += 256) {
        double g = 0.;
        if (made) {
          const double d = (double)x[k] - (double)m;
          const double p = exp(d - lz);
          g = -p * g_all;
          if (p > 0.) g += (double)a.entropy_coef * made * p * ((d - lz) + h);
          double unused[4];
          for (int s = 0; s < a.samples; ++s)
            if (a.actions[(long long)s * a.count + r] == k) g += slope(s, unused);
        }
        const float gf = (float)(g * (double)a.scale);
        if (a.bf16) static_cast<uint16_t*>(a.grad)[r * a.K + k] = bf16_bits(gf);
        else static_cast<float*>(a.grad)[r * a.K + k] = gf;
      }
    }
  }
  if (threadIdx.x == 0)
    for (int i = 0; i < 4; ++i) a.part[4 * blockIdx.x + i] = t[i];
}

// The loss and its four terms from the workgroups' partial sums.
__global__ void __launch_bounds__(256) policy_finish_kernel(const double* __restrict__ part, int n, float kl, float ent,
                                                            float scale, float* loss, float* terms) {
  __shared__ double red[4];
  double t[4];
  for (int i = 0; i < 4; ++i) {
    double s = 0.;
    for (int b = threadIdx.x; b < n; b += 256) s += part[4 * b + i];
    t[i] = block_sum_d(s, red) * (double)scale;
  }
  if (threadIdx.x == 0) {
    if (loss) *loss = (float)(t[0] + (double)kl * t[1] - (double)ent * t[2]);
    if (terms)
      for (int i = 0; i < 4; ++i) terms[i] = (float)t[i];
  }
}

hipError_t launch_policy_draw(const PolicyDrawArgs& a, hipStream_t st) {
  if (a.count <= 0 || a.samples <= 0) return hipSuccess;
  const unsigned grid = (unsigned)std::min<long long>(a.count, 1 << 20);
  hipLaunchKernelGGL(policy_draw_kernel, dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_policy_loss(const PolicyLossArgs& a, hipStream_t st) {
  if (a.count <= 0 || a.samples <= 0) return hipSuccess;
  const unsigned grid = (unsigned)std::min<long long>(a.count, kPolicyParts);
  hipLaunchKernelGGL(policy_loss_kernel, dim3(grid), dim3(256), 0, st, a);
  if (a.loss || a.terms)
    hipLaunchKernelGGL(policy_finish_kernel, dim3(1), dim3(256), 0, st, a.part, (int)grid, a.kl_coef, a.entropy_coef,
                       a.scale, a.loss, a.terms);
  return hipGetLastError();
}

}  // namespace lr
