// Expansion of a latent memory to the keys and values of an ordinary paged one:
//   k_h = (W_k,h c | k'),   v_h = W_v,h c
// for every head h and token of a range, with c the token's latent and k' its rotated key part,
// written to the token's page of the other memory.
//
// fp32: a block takes 64 tokens and the 192 products of a head, 16 of the rank at a time through shared
// memory; a thread has 8 tokens x 6 products in packed pairs of tokens.
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_mem_ptx.cuh"
#include "evo_rows.cuh"

namespace evo {
namespace {

constexpr int THREADS = 256, BM = 64, BN = LATENT_KEY + LATENT_VALUE, BK = 16;

// tokens of sequence n that are written: [lo, hi); what does not fit the call reports itself and gives none
__device__ __forceinline__ int2 token_range(const LatentExpandArgs& a, int n) {
  const int hi = seq_len(a.m, n, a.max_len), lo = a.first ? a.first[n] : 0;
  if (lo < 0 || lo > hi || hi - lo > a.max_new || hi > a.to.max_pages * a.to.page_tokens) {
    memory_fault(a.m);
    return make_int2(0, 0);
  }
  return make_int2(lo, hi);
}
// page i of a sequence in one of the memories, or -1 where the entry is outside the pool
__device__ __forceinline__ int page_or_none(const evo_memory& m, int32_t* status, int n, int i) {
  const int p = m.table[(long long)n * m.max_pages + i];
  if ((unsigned)p < (unsigned)m.n_pages) return p;
  if (status) *status = EVO_ERR_CORRUPT;
  return -1;
}

__device__ __forceinline__ float4 four(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 four(const __nv_bfloat16* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                     __uint_as_float(v.y & 0xffff0000u));
}
__device__ __forceinline__ void put2(float* p, float2 v) { *reinterpret_cast<float2*>(p) = v; }
__device__ __forceinline__ void put2(__nv_bfloat16* p, float2 v) {
  *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v.x, v.y);
}

template <typename T>
__global__ void __launch_bounds__(THREADS) latent_expand_kernel(const __grid_constant__ LatentExpandArgs a, int tiles) {
  __shared__ __align__(16) float as[BK][BM], bs[BK][BN];
  __shared__ long long from_row[BM], to_row[BM];             // rows of the pools; -1: none
  const int tid = threadIdx.x, H = a.to.n_kv_head, rank = a.m.head_dim;
  const int h = blockIdx.x % H, tile = blockIdx.x / H % tiles, n = blockIdx.x / H / tiles;
  const int2 range = token_range(a, n);
  const int t0 = range.x + tile * BM;
  if (t0 >= range.y) return;
  if (tid < BM) {
    const int t = t0 + tid;
    long long from = -1, to = -1;
    if (t < range.y) {
      const int p = page_or_none(a.m, a.m.status, n, t / a.m.page_tokens), q = page_or_none(a.to, a.m.status, n, t / a.to.page_tokens);
      if (p >= 0 && q >= 0) {
        from = (long long)p * a.m.page_tokens + t % a.m.page_tokens;
        to = ((long long)q * H + h) * a.to.page_tokens + t % a.to.page_tokens;
      }
    }
    from_row[tid] = from;
    to_row[tid] = to;
  }
  __syncthreads();
  const T* pool = static_cast<const T*>(a.m.k_pages);
  const int row = rank + LATENT_ROPE;
  // loads: a token's 4 values, and those of 3 products
  const int am = tid % BM, ak = tid / BM * 4;
  const T* asrc = from_row[am] >= 0 ? pool + from_row[am] * row + ak : nullptr;
  const T* bsrc[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int o = am + 64 * i;
    bsrc[i] = (o < LATENT_KEY ? static_cast<const T*>(a.w_k) + ((long long)h * LATENT_KEY + o) * rank
                              : static_cast<const T*>(a.w_v) + ((long long)h * LATENT_VALUE + o - LATENT_KEY) * rank) + ak;
  }
  float2 acc[4][6] = {};                                     // tokens 8 w + 2 i and the next x products 2 l + 64 j and the next
  const int lane = tid % 32, w = tid / 32;
  float4 av = asrc ? four(asrc) : make_float4(0.f, 0.f, 0.f, 0.f), bv[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) bv[i] = four(bsrc[i]);
  for (int k0 = 0; k0 < rank; k0 += BK) {
    as[ak][am] = av.x, as[ak + 1][am] = av.y, as[ak + 2][am] = av.z, as[ak + 3][am] = av.w;
#pragma unroll
    for (int i = 0; i < 3; ++i)
      bs[ak][am + 64 * i] = bv[i].x, bs[ak + 1][am + 64 * i] = bv[i].y, bs[ak + 2][am + 64 * i] = bv[i].z, bs[ak + 3][am + 64 * i] = bv[i].w;
    __syncthreads();
    if (k0 + BK < rank) {
      if (asrc) av = four(asrc + k0 + BK);
#pragma unroll
      for (int i = 0; i < 3; ++i) bv[i] = four(bsrc[i] + k0 + BK);
    }
#pragma unroll
    for (int k = 0; k < BK; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(&as[k][8 * w]), y = *reinterpret_cast<const float4*>(&as[k][8 * w + 4]);
      const float2 t2[4] = {make_float2(x.x, x.y), make_float2(x.z, x.w), make_float2(y.x, y.y), make_float2(y.z, y.w)};
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        const float2 b = *reinterpret_cast<const float2*>(&bs[k][2 * lane + 64 * j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[i][2 * j] = fma_pair(t2[i], make_float2(b.x, b.x), acc[i][2 * j]);
          acc[i][2 * j + 1] = fma_pair(t2[i], make_float2(b.y, b.y), acc[i][2 * j + 1]);
        }
      }
    }
    __syncthreads();
  }
  T* const kp = static_cast<T*>(a.to.k_pages);
  T* const vp = static_cast<T*>(a.to.v_pages);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long long to = to_row[8 * w + i], from = from_row[8 * w + i];
    if (to < 0) continue;
    const auto at = [&](int j) {
      return i % 2 ? make_float2(acc[i / 2][2 * j].y, acc[i / 2][2 * j + 1].y) : make_float2(acc[i / 2][2 * j].x, acc[i / 2][2 * j + 1].x);
    };
    put2(kp + to * 128 + 2 * lane, at(0));
    put2(vp + to * 128 + 2 * lane, at(1));
    put2(vp + to * 128 + 64 + 2 * lane, at(2));
    const T* turned = pool + from * row + rank + 2 * lane;
    kp[to * 128 + 64 + 2 * lane] = turned[0];
    kp[to * 128 + 65 + 2 * lane] = turned[1];
  }
}

}  // namespace

cudaError_t launch_latent_expand(const LatentExpandArgs& a, cudaStream_t st) {
  const int tiles = (a.max_new + BM - 1) / BM;
  const unsigned blocks = (unsigned)((long long)a.m.n_seq * tiles * a.to.n_kv_head);
  if (a.m.dtype == EVO_DTYPE_F32)
    latent_expand_kernel<float><<<blocks, THREADS, 0, st>>>(a, tiles);
  else
    latent_expand_kernel<__nv_bfloat16><<<blocks, THREADS, 0, st>>>(a, tiles);
  return cudaGetLastError();
}

}  // namespace evo
