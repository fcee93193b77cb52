// Unit caches in 8 bits (Eq. 1 for policies that run their own units): the
// refresh of a unit for the samples whose lattice asks for it, and the reuse of
// a run of skipped units.
//
//   write: c[n] <- Q(r[n]), y[n] = x[n] + r[n]     refresh[n] != 0
//          y[n] = x[n], c[n] as it was             refresh[n] == 0
//   add:   y[n] = x[n] + sum over u with reuse[u][n] != 0 of c_u[n], in unit order
//
// Both are bound by DRAM, one pass.  A writing thread takes 8 consecutive values (a
// 32-byte sector of fp32, 16 bytes of bf16, 8 codes), four lanes a scale group; an
// adding one 16 (16 codes a load), because conversions and addresses, not bytes,
// bound it at 8.
#include <cstdint>
#include <type_traits>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_memory.h"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int THREADS = 256;
constexpr int BATCH = 4;                            // units whose loads a thread has in flight

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

// the reuse flags of units u0 .. u0 + 31 for sample n, one bit each
__device__ __forceinline__ uint32_t reuse_mask(const uint8_t* reuse, int u0, int U, int N, int n) {
  const int units = min(32, U - u0);
  if (!reuse) return 0xffffffffu >> (32 - units);
  const int lane = threadIdx.x & 31;
  if (__all_sync(0xffffffffu, n == __shfl_sync(0xffffffffu, n, 0)))      // a warp within one sample: a flag a lane
    return __ballot_sync(0xffffffffu, lane < units && reuse[(long long)(u0 + lane) * N + n] != 0);
  uint32_t m = 0;
  for (int u = 0; u < units; ++u) m |= (uint32_t)(reuse[(long long)(u0 + u) * N + n] != 0) << u;
  return m;
}

// vectors of V values: `per` a sample, N * per in all
template <int V>
__global__ void __launch_bounds__(THREADS) cache_add_kernel(const uint8_t* codes, const uint8_t* scales,
                                                            const uint8_t* reuse, int U, int N, int per, int total,
                                                            const float* x, float* y) {
  const int i = blockIdx.x * THREADS + threadIdx.x, at = min(i, total - 1), n = at / per;
  using Codes = typename std::conditional<V == 16, uint4, uint2>::type;
  constexpr int Q = V / 4, LANES = UNIT_GROUP / V;   // lanes that share a scale
  const float4* src = reinterpret_cast<const float4*>(x) + (long long)Q * at;
  float4 s[Q];
#pragma unroll
  for (int j = 0; j < Q; ++j) s[j] = src[j];
  for (int u0 = 0; u0 < U; u0 += 32) {
    const uint32_t mine = reuse_mask(reuse, u0, U, N, n);
    const uint8_t* c0 = codes + V * ((long long)u0 * total + at);
    const uint8_t* f0 = scales + ((long long)u0 * total + at) / LANES;
    // the units that some lane of the warp reuses, a batch of loads in flight at once
    for (uint32_t left = __reduce_or_sync(0xffffffffu, mine); left;) {
      Codes c[BATCH];
      uint32_t f[BATCH];
      bool on[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int u = __ffs(left) - 1;             // -1 behind the last one
        left &= left - 1;
        on[j] = u >= 0 && (mine >> (u & 31) & 1);
        if (on[j]) {
          c[j] = *reinterpret_cast<const Codes*>(c0 + (long long)V * u * total);
          f[j] = f0[(long long)u * (total / LANES)];
        }
      }
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
        if (on[j]) {
          const float k = scale_value(f[j]);
          const uint32_t* w = reinterpret_cast<const uint32_t*>(&c[j]);
#pragma unroll
          for (int e = 0; e < Q; ++e) {
            const float4 v = codes4(w[e]);
            // a product by a power of two is exact: the fused form rounds as the sum does
            s[e] = make_float4(fmaf(v.x, k, s[e].x), fmaf(v.y, k, s[e].y), fmaf(v.z, k, s[e].z), fmaf(v.w, k, s[e].w));
          }
        }
    }
  }
  if (i < total)
#pragma unroll
    for (int j = 0; j < Q; ++j) reinterpret_cast<float4*>(y)[(long long)Q * i + j] = s[j];
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
  // 16 values a thread once that gives every SM 4 blocks (16.8 million values, 11 units: 54.6 us
  // against 70.1 with 8); below, 8 and twice the threads (262,144 values, 5 units: 4.2 us against 6.1)
  const bool wide = N * per >= 152ll * 4 * THREADS * 16;
  const int pv = (int)(per / (wide ? 16 : 8)), total = N * pv, grid = (total + THREADS - 1) / THREADS;
  if (wide)
    cache_add_kernel<16><<<grid, THREADS, 0, st>>>(codes, scales, reuse, U, N, pv, total, x, y);
  else
    cache_add_kernel<8><<<grid, THREADS, 0, st>>>(codes, scales, reuse, U, N, pv, total, x, y);
  return cudaGetLastError();
}

}  // namespace evo
