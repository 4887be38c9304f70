// The optimiser step over many tensors: the 2-norm of their gradients, AdamW
// with float32 or 8-bit moments, and the values that 8-bit moments stand for.
//
// Streaming passes over chunks of values, a workgroup each; the
// tensors of a launch are a kernel argument, so that hundreds of small ones
// take a few launches and a step can be recorded.  A wave takes runs of 256
// values, four neighbours a lane, which is also a block of the 8-bit moments:
// its largest exponents are found in the wave.  Nothing is read or written
// twice: 28 bytes a value with float32 moments and gradients, 14 with 8-bit
// moments and bf16 gradients.  Memory bounds them (a large copy: 5.0 TB/s):
// 165 M values with 8-bit moments 415 us (5.6 TB/s), their moments written out
// 264 us (6.3 TB/s, mostly stores), the norm of as many bf16 gradients 60 us
// (5.5 TB/s); 200 tensors of together 22.2 M values with float32 moments, three
// launches, 131 us (4.7 TB/s).  With 8-bit moments the vector instructions come
// next (66 a value, 308 us at the peak rate): 93 of them took 440 us.
#pragma once

#include "kernels.hpp"
#include "policy_impl.hpp"

namespace lr {

constexpr int kOptThreads = 256;
constexpr int kOptRuns = kStepChunk / kOptThreads / 4;  // of 256 values, a wave's in a chunk

// Random bits: two rounds of multiply and shift (the odd integers next to
// 2^32 / golden ratio and 2^32 (sqrt 2 - 1)).
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x9E3779B1u;
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  return x ^ (x >> 16);
}

// Tensor of the list that chunk c of the launch belongs to.
template <class F>
__device__ __forceinline__ int tensor_of(int num, uint32_t c, F&& chunk0) {
  int lo = 0;
  int hi = num;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (c >= chunk0(mid)) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ int tensor_of(const TensorList& l, uint32_t c) {
  return tensor_of(l.num, c, [&](int i) { return l.t[i].chunk0; });
}

// Values i .. i + 3 of a tensor, any alignment; FULL: all are there.
template <bool FULL>
__device__ __forceinline__ void quad_f32(const void* p, long long i, long long count, float (&v)[4]) {
  const float* __restrict__ x = static_cast<const float*>(p);
  if (FULL) {
    const Quad q = *reinterpret_cast<const Quad*>(x + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = q.v[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = i + j < count ? x[i + j] : 0.f;
  }
}
template <bool FULL>
__device__ __forceinline__ void quad_grad(const void* p, int bf16, long long i, long long count, float (&v)[4]) {
  if (!bf16) return quad_f32<FULL>(p, i, count, v);
  const uint16_t* __restrict__ x = static_cast<const uint16_t*>(p);
  if (FULL) {
    const QuadBf16 q = *reinterpret_cast<const QuadBf16*>(x + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(j % 2 ? q.v[j / 2] & 0xFFFF0000u : q.v[j / 2] << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = i + j < count ? __uint_as_float((uint32_t)x[i + j] << 16) : 0.f;
  }
}
struct __attribute__((packed, aligned(1))) Bytes4 {
  uint32_t w;
};
template <bool FULL>
__device__ __forceinline__ uint32_t quad_codes(const void* p, long long i, long long count) {
  const uint8_t* __restrict__ x = static_cast<const uint8_t*>(p);
  if (FULL) return reinterpret_cast<const Bytes4*>(x + i)->w;
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + j < count) w |= (uint32_t)x[i + j] << (8 * j);
  return w;
}
template <bool FULL>
__device__ __forceinline__ void put_f32(void* p, long long i, long long count, const float (&v)[4]) {
  float* x = static_cast<float*>(p);
  if (FULL) {
    *reinterpret_cast<Quad*>(x + i) = Quad{{v[0], v[1], v[2], v[3]}};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < count) x[i + j] = v[j];
  }
}
template <bool FULL>
__device__ __forceinline__ void put_codes(void* p, long long i, long long count, uint32_t w) {
  uint8_t* x = static_cast<uint8_t*>(p);
  if (FULL) {
    *reinterpret_cast<Bytes4*>(x + i) = Bytes4{w};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < count) x[i + j] = (uint8_t)(w >> (8 * j));
  }
}

// ---- norm ------------------------------------------------------------------
// Squares and sums in float64: no square of a float32 leaves its range.
template <int THREADS>
__device__ __forceinline__ double grad_square_sum(const GradList& l, int bf16, uint32_t chunk, uint32_t step) {
  double s = 0.;
  for (; chunk < l.chunks; chunk += step) {
    const int t = tensor_of(l.num, chunk, [&](int i) { return l.chunk0[i]; });
    const long long base = (long long)(chunk - l.chunk0[t]) * kNormChunk;
    const long long count = l.count[t];
    auto one = [&](auto full) {
      constexpr int QUADS = kNormChunk / THREADS / 4;
      float v[QUADS][4];
#pragma unroll
      for (int q = 0; q < QUADS; ++q)
        quad_grad<decltype(full)::value>(l.grad[t], bf16, base + 4 * (q * THREADS + (int)threadIdx.x), count, v[q]);
#pragma unroll
      for (int q = 0; q < QUADS; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) s += (double)v[q][j] * (double)v[q][j];
    };
    if (count - base >= kNormChunk) one(std::true_type{});
    else one(std::false_type{});
  }
  return s;
}
__global__ void __launch_bounds__(kOptThreads) grad_norm_kernel(GradList l, int bf16, double* __restrict__ part) {
  __shared__ double red[kOptThreads / 64];
  const double s = block_sum_d<kOptThreads>(grad_square_sum<kOptThreads>(l, bf16, blockIdx.x, gridDim.x), red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}
__global__ void __launch_bounds__(1024) grad_norm_finish_kernel(const double* __restrict__ part, int n, float* norm) {
  __shared__ double red[16];
  double s = 0.;
  for (int b = threadIdx.x; b < n; b += 1024) s += part[b];
  s = block_sum_d<1024>(s, red);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}
// A few chunks: one workgroup, one launch (one tensor of 4096, 16384, 32768, 49152
// values: 2.5, 3.2, 4.2, 5.3 us so, 4.0, 4.3, 4.5, 4.5 with partial sums and a second
// launch; three tensors of together six chunks 4.4, 4.5, of twelve 6.0, 4.7).
constexpr int kNormOneValues = 32768;
constexpr int kNormOneThreads = kNormChunk / 4;
__global__ void __launch_bounds__(kNormOneThreads) grad_norm_one_kernel(GradList l, int bf16, float* norm) {
  __shared__ double red[kNormOneThreads / 64];
  const double s = block_sum_d<kNormOneThreads>(grad_square_sum<kNormOneThreads>(l, bf16, 0, 1), red);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

// ---- AdamW -----------------------------------------------------------------
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

// 8-bit codes: with the code's seven or eight bits c in place (exponent and
// three mantissa bits, as float32 has them), float32's own subnormal numbers
// give the codes below the smallest normal value, 2^LEAST; two powers of two
// then bring the exponent right.
template <int LEAST>
__device__ __forceinline__ float code_value(uint32_t c, float u) {
  // (2^(127 + LEAST) times u: 2 u 2^LEAST over float32's 2^-126)
  return __uint_as_float(c << 20) * __uint_as_float((254u + LEAST) << 23) * u;
}
// Code of the magnitude y (the value over two scales and times 2^(-126 - LEAST),
// so that float32's subnormal numbers are the codes' too) with 20 random bits, in
// the upper byte.
__device__ __forceinline__ uint32_t code_of(float y, uint32_t bits) { return (__float_as_uint(y) + bits) << 4; }
// The upper bytes of four words.
__device__ __forceinline__ uint32_t upper_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(b, a, 0x0C0C0703u) | __builtin_amdgcn_perm(d, c, 0x07030C0Cu);
}
// Largest magnitude of the wave as bits (NaN and infinity the largest).
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t x) {
  auto dpp = [&](auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, true);
  };
  x = max(x, dpp(std::integral_constant<int, 0xB1>{}));
  x = max(x, dpp(std::integral_constant<int, 0x4E>{}));
  x = max(x, dpp(std::integral_constant<int, 0x141>{}));
  x = max(x, dpp(std::integral_constant<int, 0x140>{}));
  auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max((uint32_t)r[0], (uint32_t)r[1]);
  r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max((uint32_t)r[0], (uint32_t)r[1]);
}

// m and v after the step, p moved by them.  The root and the reciprocal are the
// hardware's instructions, each within one step of float32 (the exact ones take
// some ten instructions more each): with the other roundings the change is within
// 10 half steps of the formula's, and nothing that is kept builds on it but p.
__device__ __forceinline__ void adamw_values(const AdamwArgs& a, float clip, const float (&g4)[4], float (&m)[4],
                                             float (&v)[4], float (&p)[4]) {
  float root[4];
  uint32_t least = 0xFFFFFFFFu;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float g = mul_rn(g4[j], clip);  // (exact for clip = 1)
    m[j] = add_rn(mul_rn(m[j], a.b1), mul_rn(g, a.c1));
    v[j] = add_rn(mul_rn(v[j], a.b2), mul_rn(mul_rn(g, g), a.c2));
    root[j] = __builtin_amdgcn_sqrtf(v[j]);
    least = min(least, __float_as_uint(v[j]) - 1u);
  }
  // (the root's instruction takes no subnormal numbers, which are rare; zeros wrap around)
  if (__any(least < 0x007FFFFFu)) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (v[j] < 0x1p-100f) root[j] = __builtin_amdgcn_sqrtf(v[j] * 0x1p64f) * 0x1p-32f;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    p[j] = p[j] * a.keep - a.rate * m[j] * __builtin_amdgcn_rcpf(root[j] * a.root + a.eps);
}

template <bool BITS8, bool BF16, bool FULL>
__device__ __forceinline__ void adamw_chunk(const TensorEntry& t, const AdamwArgs& a, long long base) {
  constexpr int RUNS = kOptRuns;
  constexpr int AT_ONCE = BITS8 || RUNS < 2 ? RUNS : 2;  // runs in flight
  const int wave = threadIdx.x / 64;
  const int lane = threadIdx.x % 64;
  const float norm = a.norm ? *a.norm : 0.f;
#pragma unroll
  for (int r0 = 0; r0 < RUNS; r0 += AT_ONCE) {
    float p[AT_ONCE][4], g[AT_ONCE][4];
    float m[BITS8 ? 1 : AT_ONCE][4], v[BITS8 ? 1 : AT_ONCE][4];
    uint32_t cm[AT_ONCE], cv[AT_ONCE];
    float2 u[AT_ONCE];
    // (a block past the tensor's end has no scales)
    auto block = [&](int r) { return base / kStateBlock + (r0 + r) * (kOptThreads / 64) + wave; };
    auto at = [&](int r) { return base + ((r0 + r) * (kOptThreads / 64) + wave) * 256 + 4 * lane; };
#pragma unroll
    for (int r = 0; r < AT_ONCE; ++r) {
      const long long i = at(r);
      quad_f32<FULL>(t.param, i, t.count, p[r]);
      quad_grad<FULL>(t.grad, BF16, i, t.count, g[r]);
      if constexpr (BITS8) {
        cm[r] = quad_codes<FULL>(t.m, i, t.count);
        cv[r] = quad_codes<FULL>(t.v, i, t.count);
        u[r] = make_float2(0.f, 0.f);
        if (FULL || block(r) * kStateBlock < t.count)
          u[r] = make_float2(t.scales[2 * block(r)], t.scales[2 * block(r) + 1]);
      } else {
        quad_f32<FULL>(t.m, i, t.count, m[r]);
        quad_f32<FULL>(t.v, i, t.count, v[r]);
      }
    }
    // (behind the loads, so that they do not wait for it)
    if (!(fabsf(norm) <= 3.402823466e38f)) return;
    const float clip = norm > a.max_norm ? a.max_norm / norm : 1.f;
#pragma unroll
    for (int r = 0; r < AT_ONCE; ++r) {
      const long long i = at(r);
      if constexpr (!BITS8) {
        adamw_values(a, clip, g[r], m[r], v[r], p[r]);
        put_f32<FULL>(t.param, i, t.count, p[r]);
        put_f32<FULL>(t.m, i, t.count, m[r]);
        put_f32<FULL>(t.v, i, t.count, v[r]);
      } else {
        float mm[4], vv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t c = cm[r] >> (8 * j);
          const float x = code_value<-14>(c & 127u, u[r].x);
          mm[j] = __uint_as_float(__float_as_uint(x) ^ ((c & 128u) << 24));
          vv[j] = code_value<-30>((cv[r] >> (8 * j)) & 255u, u[r].y);
        }
        adamw_values(a, clip, g[r], mm, vv, p[r]);
        put_f32<FULL>(t.param, i, t.count, p[r]);
        uint32_t top_m = 0, top_v = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          top_m = max(top_m, __float_as_uint(fabsf(mm[j])));
          top_v = max(top_v, __float_as_uint(vv[j]));  // (a NaN's sign only makes it larger)
        }
        // exponents of the block, held where a scale and its inverse are normal numbers
        uint32_t em = wave_max_bits(top_m) >> 23;
        uint32_t ev = wave_max_bits(top_v) >> 23;
        em = max(em, 27u);
        ev = max(ev, 27u);
        const uint32_t key = mix32(t.key + (uint32_t)((unsigned long long)i >> 32));
        uint32_t zm[4], zv[4];
        uint32_t least = 0xFFFFFFFFu;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t h = mix32((uint32_t)i + j + key);
          zm[j] = code_of(__builtin_ldexpf(fabsf(mm[j]), 14 - (int)em), h & 0xFFFFFu);
          zv[j] = code_of(__builtin_ldexpf(vv[j], 30 - (int)ev), h >> 12);
          least = min(least, zv[j]);
        }
        if (__any(least < 1u << 24)) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (vv[j] > 0.f) zv[j] = max(zv[j], 1u << 24);
        }
        auto sign = [&](int j) { return __float_as_uint(mm[j] + 0.f); };  // (none of a negative zero)
        uint32_t wm = upper_bytes(zm[0], zm[1], zm[2], zm[3]) |
                      (upper_bytes(sign(0), sign(1), sign(2), sign(3)) & 0x80808080u);
        uint32_t wv = upper_bytes(zv[0], zv[1], zv[2], zv[3]);
        if (em >= 253u) wm = 0;
        if (ev >= 253u) wv = 0;
        put_codes<FULL>(t.m, i, t.count, wm);
        put_codes<FULL>(t.v, i, t.count, wv);
        if (lane == 0 && (FULL || block(r) * kStateBlock < t.count)) {
          t.scales[2 * block(r)] = em < 253u ? __uint_as_float(em << 23) : __builtin_nanf("");
          t.scales[2 * block(r) + 1] = ev < 253u ? __uint_as_float(ev << 23) : __builtin_nanf("");
        }
      }
    }
  }
}

template <bool BITS8, bool BF16>
__global__ void __launch_bounds__(kOptThreads) adamw_kernel(TensorList l, AdamwArgs a) {
  for (uint32_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const TensorEntry& t = l.t[tensor_of(l, c)];
    const long long base = (long long)(c - t.chunk0) * kStepChunk;
    if (t.count - base >= kStepChunk) adamw_chunk<BITS8, BF16, true>(t, a, base);
    else adamw_chunk<BITS8, BF16, false>(t, a, base);
  }
}

template <bool FULL>
__device__ __forceinline__ void moments_chunk(const TensorEntry& t, long long base) {
#pragma unroll
  for (int r = 0; r < kOptRuns; ++r) {
    const long long run = base + (r * (kOptThreads / 64) + threadIdx.x / 64) * 256;
    const long long i = run + 4 * (threadIdx.x % 64);
    if (!FULL && run >= t.count) break;
    const uint32_t cm = quad_codes<FULL>(t.m, i, t.count);
    const uint32_t cv = quad_codes<FULL>(t.v, i, t.count);
    const float um = t.scales[2 * (run / kStateBlock)];
    const float uv = t.scales[2 * (run / kStateBlock) + 1];
    float m[4], v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t c = cm >> (8 * j);
      m[j] = __uint_as_float(__float_as_uint(code_value<-14>(c & 127u, um)) ^ ((c & 128u) << 24));
      v[j] = code_value<-30>((cv >> (8 * j)) & 255u, uv);
    }
    put_f32<FULL>(t.param, i, t.count, m);
    put_f32<FULL>(const_cast<void*>(t.grad), i, t.count, v);
  }
}
__global__ void __launch_bounds__(kOptThreads) moments_kernel(TensorList l) {
  for (uint32_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const TensorEntry& t = l.t[tensor_of(l, c)];
    const long long base = (long long)(c - t.chunk0) * kStepChunk;
    if (t.count - base >= kStepChunk) moments_chunk<true>(t, base);
    else moments_chunk<false>(t, base);
  }
}

// ---- launches ----------------------------------------------------------------
hipError_t launch_grad_norm(const GradList* lists, int num, int bf16, double* part, float* norm, hipStream_t st) {
  if (num == 1 && lists[0].chunks <= kNormOneValues / kNormChunk) {
    hipLaunchKernelGGL(grad_norm_one_kernel, dim3(1), dim3(kNormOneThreads), 0, st, lists[0], bf16, norm);
    return hipGetLastError();
  }
  int parts = 0;
  for (int i = 0; i < num; ++i) {
    const int grid = (int)std::min<uint32_t>(lists[i].chunks, kNormParts);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(grid), dim3(kOptThreads), 0, st, lists[i], bf16, part + parts);
    parts += grid;
  }
  hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(1024), 0, st, part, parts, norm);
  return hipGetLastError();
}

uint32_t tensor_key(uint32_t seed, uint32_t i) { return mix32(seed + 0x9E3779B9u * i); }

static dim3 chunk_grid(const TensorList& l) { return dim3((unsigned)std::min<uint32_t>(l.chunks, 1u << 22)); }

hipError_t launch_adamw(const TensorList& l, const AdamwArgs& a, hipStream_t st) {
  if (l.chunks == 0) return hipSuccess;
  auto go = [&](auto bits8, auto bf16) {
    hipLaunchKernelGGL((adamw_kernel<decltype(bits8)::value, decltype(bf16)::value>), chunk_grid(l), dim3(kOptThreads),
                       0, st, l, a);
  };
  if (a.bits8 && a.bf16) go(std::true_type{}, std::true_type{});
  else if (a.bits8) go(std::true_type{}, std::false_type{});
  else if (a.bf16) go(std::false_type{}, std::true_type{});
  else go(std::false_type{}, std::false_type{});
  return hipGetLastError();
}

hipError_t launch_moments(const TensorList& l, hipStream_t st) {
  if (l.chunks == 0) return hipSuccess;
  hipLaunchKernelGGL(moments_kernel, chunk_grid(l), dim3(kOptThreads), 0, st, l);
  return hipGetLastError();
}

}  // namespace lr
