// Unit caches in 8 bits (Eq. 1 for policies that run their own units): the
// refresh of a unit for the samples whose lattice asks for it, and the reuse of
// a run of skipped units.
//
//   write: c[n] <- Q(r[n]), y[n] = x[n] + r[n]     refresh[n] != 0
//          y[n] = x[n], c[n] as it was             refresh[n] == 0
//   add:   y[n] = x[n] + sum over u with reuse[u][n] != 0 of c_u[n], in unit order
//
// Both are bound by DRAM: one pass, each thread 8 consecutive values (a 32-byte
// sector of fp32, 16 bytes of bf16, 8 codes), four lanes a scale group.
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_memory.h"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int THREADS = 256;
constexpr int BATCH = 6;                            // units whose loads a thread has in flight

template <typename T>
struct Eight;
template <>
struct Eight<float> {
  static __device__ __forceinline__ void load(const float* p, float4 (&v)[2]) {
    v[0] = reinterpret_cast<const float4*>(p)[0];
    v[1] = reinterpret_cast<const float4*>(p)[1];
  }
};
template <>
struct Eight<__nv_bfloat16> {
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float4 (&v)[2]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    v[0] = make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u));
    v[1] = make_float4(__uint_as_float(u.z << 16), __uint_as_float(u.z & 0xffff0000u), __uint_as_float(u.w << 16),
                       __uint_as_float(u.w & 0xffff0000u));
  }
};

__device__ __forceinline__ void add4(float4& a, const float4& b) {
  a.x += b.x;
  a.y += b.y;
  a.z += b.z;
  a.w += b.w;
}

// vectors of 8 values: `per` a sample, N * per in all
template <typename T>
__global__ void __launch_bounds__(THREADS) cache_write_kernel(const T* r, const uint8_t* refresh, int per, int total,
                                                              const float* x, float* y, uint8_t* codes,
                                                              uint8_t* scales) {
  const int i = blockIdx.x * THREADS + threadIdx.x;
  const bool in = i < total;                        // total is a multiple of 4: whole groups are in or out
  const bool on = in && (!refresh || refresh[i / per] != 0);
  const long long at = 8ll * i;
  float4 v[2] = {}, s[2] = {};
  if (on) Eight<T>::load(r + at, v);
  if (in && y && (on || y != x)) Eight<float>::load(x + at, s);
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) a = amax_bits(amax_bits(amax_bits(amax_bits(a, v[j].x), v[j].y), v[j].z), v[j].w);
  const uint32_t byte = scale_byte(group_umax<4>(a));
  if (on) {
    const uint2 c = make_uint2(quantise4(v[0], byte), quantise4(v[1], byte));
    *reinterpret_cast<uint2*>(codes + at) = c;
    if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)byte;
    add4(s[0], v[0]);
    add4(s[1], v[1]);
  }
  if (in && y && (on || y != x)) {
    reinterpret_cast<float4*>(y + at)[0] = s[0];
    reinterpret_cast<float4*>(y + at)[1] = s[1];
  }
}

__global__ void __launch_bounds__(THREADS) cache_add_kernel(const uint8_t* codes, const uint8_t* scales,
                                                            const uint8_t* reuse, int U, int N, int per, int total,
                                                            const float* x, float* y) {
  const int i = blockIdx.x * THREADS + threadIdx.x;
  if (i >= total) return;
  const int n = i / per;
  const long long at = 8ll * i;
  float4 s[2];
  Eight<float>::load(x + at, s);
  for (int u0 = 0; u0 < U; u0 += BATCH) {          // a batch of units' loads in flight at once
    uint2 c[BATCH];
    uint32_t f[BATCH];
    bool on[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) on[j] = u0 + j < U && (!reuse || reuse[(long long)(u0 + j) * N + n] != 0);
#pragma unroll
    for (int j = 0; j < BATCH; ++j)
      if (on[j]) {
        const long long v = (long long)(u0 + j) * total + i;
        c[j] = *reinterpret_cast<const uint2*>(codes + 8 * v);
        f[j] = scales[v >> 2];
      }
#pragma unroll
    for (int j = 0; j < BATCH; ++j)
      if (on[j]) {
        const float k = scale_value(f[j]);
        const float4 a = codes4(c[j].x), b = codes4(c[j].y);
        // a product by a power of two is exact: the fused form rounds as the sum does
        s[0] = make_float4(fmaf(a.x, k, s[0].x), fmaf(a.y, k, s[0].y), fmaf(a.z, k, s[0].z), fmaf(a.w, k, s[0].w));
        s[1] = make_float4(fmaf(b.x, k, s[1].x), fmaf(b.y, k, s[1].y), fmaf(b.z, k, s[1].z), fmaf(b.w, k, s[1].w));
      }
  }
  reinterpret_cast<float4*>(y + at)[0] = s[0];
  reinterpret_cast<float4*>(y + at)[1] = s[1];
}

}  // namespace

cudaError_t launch_cache_write(const void* r, int dtype, const uint8_t* refresh, int N, long long per, const float* x,
                               float* y, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  const int pv = (int)(per / 8), total = N * pv;
  const int grid = (total + THREADS - 1) / THREADS;
  if (dtype == EVO_DTYPE_F32)
    cache_write_kernel<<<grid, THREADS, 0, st>>>(static_cast<const float*>(r), refresh, pv, total, x, y, codes, scales);
  else
    cache_write_kernel<<<grid, THREADS, 0, st>>>(static_cast<const __nv_bfloat16*>(r), refresh, pv, total, x, y, codes,
                                                 scales);
  return cudaGetLastError();
}

cudaError_t launch_cache_add(const uint8_t* codes, const uint8_t* scales, const uint8_t* reuse, int U, int N,
                             long long per, const float* x, float* y, cudaStream_t st) {
  const int pv = (int)(per / 8), total = N * pv;
  cache_add_kernel<<<(total + THREADS - 1) / THREADS, THREADS, 0, st>>>(codes, scales, reuse, U, N, pv, total, x, y);
  return cudaGetLastError();
}

}  // namespace evo
