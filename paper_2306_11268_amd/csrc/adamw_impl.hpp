// The optimiser step over many tensors: the 2-norm of their gradients, AdamW
// with float32 or 8-bit moments, and the values that 8-bit moments stand for.
#pragma once

#include "kernels.hpp"
#include "policy_impl.hpp"

namespace lr {

__device__ __forceinline__ float grad_at(const void* g, long long i, int bf16) {
  return bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(g)[i] << 16) : static_cast<const float*>(g)[i];
}

// Random bits: two rounds of multiply and shift (the odd integers next to
// 2^32 / golden ratio and 2^32 (sqrt 2 - 1)).
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x9E3779B1u;
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  return x ^ (x >> 16);
}

// Tensor of the list that chunk c of the launch belongs to.
__device__ __forceinline__ int tensor_of(const TensorList& l, long long c) {
  int lo = 0;
  for (int i = 1; i < l.num; ++i) lo = c >= l.t[i].chunk0 ? i : lo;
  return lo;
}

__global__ void __launch_bounds__(256) grad_norm_kernel(TensorList l, int bf16, double* __restrict__ part) {
  __shared__ double red[4];
  double s = 0.;
  for (long long c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const TensorEntry& t = l.t[tensor_of(l, c)];
    for (int j = threadIdx.x; j < kTensorChunk; j += 256) {
      const long long i = (c - t.chunk0) * kTensorChunk + j;
      const double g = i < t.count ? (double)grad_at(t.grad, i, bf16) : 0.;
      s += g * g;
    }
  }
  s = block_sum_d<256>(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ void __launch_bounds__(256) grad_norm_finish_kernel(const double* __restrict__ part, int n, float* norm) {
  __shared__ double red[4];
  double s = 0.;
  for (int b = threadIdx.x; b < n; b += 256) s += part[b];
  s = block_sum_d<256>(s, red);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

// Products and sums that are rounded one by one (never fused): the moments are
// defined by them.
__device__ __forceinline__ float mul_rn(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
__device__ __forceinline__ float add_rn(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}

// 8-bit codes: value / (2 u), in [0, 1], of the seven or eight bits c.
template <int LEAST>  // exponent of the smallest normal value
__device__ __forceinline__ float code_value(uint32_t c) {
  const uint32_t e = c >> 3;
  const float f = (float)(c & 7u);
  return e ? (8.f + f) * __uint_as_float((e + 126u + LEAST - 3u) << 23) : f * __uint_as_float((127u + LEAST - 3u) << 23);
}
// Code of the magnitude y in [0, 1) with 20 random bits.
template <int LEAST>
__device__ __forceinline__ uint32_t code_of(float y, uint32_t bits) {
  const float least = __uint_as_float((127u + LEAST) << 23);
  const bool small = y < least;
  const uint32_t z = (__float_as_uint(small ? y + least : y) + bits) >> 20;
  return z - ((126u + LEAST) << 3) - (small ? 8u : 0u);
}

// One block of LST values per workgroup.
__global__ void __launch_bounds__(256) adamw_kernel(TensorList l, AdamwArgs a) {
  __shared__ float redf[4];
  float clip = 1.f;
  if (a.norm) {
    const float n = *a.norm;
    if (!(fabsf(n) <= 3.402823466e38f)) return;
    if (n > a.max_norm) clip = a.max_norm / n;
  }
  for (long long c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const int ti = tensor_of(l, c);
    const TensorEntry& t = l.t[ti];
    for (int j = threadIdx.x; j < kTensorChunk; j += 256) {
      const long long i = (c - t.chunk0) * kTensorChunk + j;
      const bool in = i < t.count;
      const long long blk = ((c - t.chunk0) * kTensorChunk + (j & ~255)) / 256;
      const bool blk_in = blk * 256 < t.count;
      float m = 0.f;
      float v = 0.f;
      float g = 0.f;
      float p = 0.f;
      if (in) {
        g = grad_at(t.grad, i, a.bf16);
        p = t.param[i];
        if (a.bits8) {
          const uint32_t cm = static_cast<const uint8_t*>(t.m)[i];
          const uint32_t cv = static_cast<const uint8_t*>(t.v)[i];
          m = mul_rn(2.f * code_value<-14>(cm & 127u), t.scales[2 * blk]);
          if (cm & 128u) m = -m;
          v = mul_rn(2.f * code_value<-30>(cv), t.scales[2 * blk + 1]);
        } else {
          m = static_cast<const float*>(t.m)[i];
          v = static_cast<const float*>(t.v)[i];
        }
        if (a.norm) g = mul_rn(g, clip);
        m = add_rn(mul_rn(m, a.b1), mul_rn(g, a.c1));
        v = add_rn(mul_rn(v, a.b2), mul_rn(mul_rn(g, g), a.c2));
        t.param[i] = p * a.keep - a.rate * m / (sqrtf(v) * a.root + a.eps);
        if (!a.bits8) {
          static_cast<float*>(t.m)[i] = m;
          static_cast<float*>(t.v)[i] = v;
        }
      }
      if (a.bits8) {
        // (exponents are exact in float32)
        uint32_t em = (uint32_t)block_reduce<256>((float)((__float_as_uint(m) >> 23) & 255u), OpMax{}, redf);
        uint32_t ev = (uint32_t)block_reduce<256>((float)((__float_as_uint(v) >> 23) & 255u), OpMax{}, redf);
        em = em < 27u ? 27u : em;
        ev = ev < 27u ? 27u : ev;
        if (in) {
          const uint32_t key = mix32(t.key + (uint32_t)((unsigned long long)i >> 32));
          const uint32_t h = mix32((uint32_t)i + key);
          uint32_t cm = 0;
          uint32_t cv = 0;
          if (em < 253u) {
            cm = code_of<-14>(fabsf(m) * __uint_as_float((253u - em) << 23), h & 0xFFFFFu);
            if (m < 0.f) cm |= 128u;
          }
          if (ev < 253u) {
            cv = code_of<-30>(v * __uint_as_float((253u - ev) << 23), h >> 12);
            if (v > 0.f && cv == 0u) cv = 1u;
          }
          static_cast<uint8_t*>(t.m)[i] = (uint8_t)cm;
          static_cast<uint8_t*>(t.v)[i] = (uint8_t)cv;
        }
        if (threadIdx.x == 0 && blk_in) {
          t.scales[2 * blk] = em < 253u ? __uint_as_float(em << 23) : __builtin_nanf("");
          t.scales[2 * blk + 1] = ev < 253u ? __uint_as_float(ev << 23) : __builtin_nanf("");
        }
      }
    }
  }
}

__global__ void __launch_bounds__(256) moments_kernel(TensorList l) {
  for (long long c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const TensorEntry& t = l.t[tensor_of(l, c)];
    for (int j = threadIdx.x; j < kTensorChunk; j += 256) {
      const long long i = (c - t.chunk0) * kTensorChunk + j;
      if (i >= t.count) continue;
      const uint32_t cm = static_cast<const uint8_t*>(t.m)[i];
      const uint32_t cv = static_cast<const uint8_t*>(t.v)[i];
      const float m = 2.f * code_value<-14>(cm & 127u) * t.scales[2 * (i / 256)];
      t.param[i] = cm & 128u ? -m : m;
      const_cast<float*>(static_cast<const float*>(t.grad))[i] = 2.f * code_value<-30>(cv) * t.scales[2 * (i / 256) + 1];
    }
  }
}

hipError_t launch_grad_norm(const TensorList* lists, int num, int bf16, double* part, float* norm, hipStream_t st) {
  int parts = 0;
  for (int i = 0; i < num; ++i) {
    if (lists[i].chunks <= 0) continue;
    const int grid = (int)std::min<long long>(lists[i].chunks, kNormParts);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(grid), dim3(256), 0, st, lists[i], bf16, part + parts);
    parts += grid;
  }
  hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(256), 0, st, part, parts, norm);
  return hipGetLastError();
}

hipError_t launch_adamw(const TensorList& l, const AdamwArgs& a, hipStream_t st) {
  if (l.chunks <= 0) return hipSuccess;
  hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)std::min<long long>(l.chunks, 1 << 16)), dim3(256), 0, st, l, a);
  return hipGetLastError();
}

uint32_t tensor_key(uint32_t seed, uint32_t i) { return mix32(seed + 0x9E3779B9u * i); }

hipError_t launch_moments(const TensorList& l, hipStream_t st) {
  if (l.chunks <= 0) return hipSuccess;
  hipLaunchKernelGGL(moments_kernel, dim3((unsigned)std::min<long long>(l.chunks, 1 << 16)), dim3(256), 0, st, l);
  return hipGetLastError();
}

}  // namespace lr
