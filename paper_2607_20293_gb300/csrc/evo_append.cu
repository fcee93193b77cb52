// Append to a paged memory: the norm of each head of the queries and keys, their
// rotation by position, and the write of keys and values to the sequence's pages
// in the memory's format, in one pass over the rows.
//
//   norm      u = x / sqrt(mean(x^2) + eps) * gain          (queries and keys, fp32)
//   rotation  (u_i, u_{i+D/2}) by the angle of (position, i): cosines and sines
//             come from a table that the caller computed in double precision
//   write     keys and values in the format's type, or e4m3 codes and a scale
//             byte for the head's row (evo_quant.cuh)
//
// One rounding per output: everything between the load and the store is fp32.
// A warp takes a row (a token).  D / 8 lanes hold one head, each the 4 values at
// 4l and the 4 at D/2 + 4l: both halves of every rotated pair are in one lane, so
// the rotation needs no exchange, and the norm and the largest magnitude are
// shuffles over those lanes.  The row's cosines and sines stay in registers for
// all its heads.  The work is bound by DRAM for long chunks and by the chain
// starts -> length -> table -> page for single tokens; short calls therefore
// spread a row's heads over several warps.
#include <algorithm>
#include <cstdint>
#include <type_traits>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_memory.h"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int BATCH = 4;                            // head groups whose loads a warp has in flight

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
// four values as they are in memory
template <typename T>
using Raw = typename std::conditional<sizeof(T) == 4, float4, uint2>::type;
__device__ __forceinline__ float4 values(float4 u) { return u; }
__device__ __forceinline__ float4 values(uint2 u) {
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                     __uint_as_float(u.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ float dot4(float4 a) { return (a.x * a.x + a.y * a.y) + (a.z * a.z + a.w * a.w); }

// the sequence that row belongs to: the last n with starts[n] <= row, found 32
// entries a step by the whole warp (two dependent loads for up to 1,024 sequences)
__device__ __forceinline__ int seq_of_row(const int* starts, int n_seq, int row, int lane) {
  int lo = 0, hi = n_seq;                             // starts[lo] <= row, starts[hi] > row
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int at = lo + (lane + 1) * step;
    const unsigned past = __ballot_sync(0xffffffffu, at >= hi || starts[min(at, n_seq)] > row);
    const int k = past ? __ffs(past) - 1 : 32;        // the first probe past the row
    const int from = lo + k * step;
    hi = min(hi, from + step);
    lo = from;
  }
  return lo;
}

template <typename T, int D, int FORMAT>
__global__ void __launch_bounds__(THREADS) append_kernel(const __grid_constant__ AppendArgs a, int parts) {
  constexpr int LH = D / 8, HEADS = 32 / LH;          // lanes a head, heads a warp takes at once
  const evo_memory& m = a.m;
  const int lane = threadIdx.x & 31, l = lane % LH;
  const long long w = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
  const int row = (int)(w / parts), part = (int)(w % parts);
  if (row >= a.rows) return;
  int n;
  if (m.starts) {
    if (row < m.starts[0] || row >= m.starts[m.n_seq]) return;    // behind the last sequence
    n = seq_of_row(m.starts, m.n_seq, row, lane);
  } else {
    n = row / (a.rows / m.n_seq);
  }
  const SeqRows s = seq_rows(m, n, a.rows, a.rows);
  if (row < s.first || row >= s.first + s.count) return;          // malformed starts
  const int pos = m.lens[n] - s.count + (row - s.first);
  const int turn = pos + (a.pos0 ? a.pos0[n] : 0);
  const int pi = pos / m.page_tokens;
  const bool stores = a.k != nullptr;
  if (pos < 0 || pi >= m.max_pages || (a.rotation && (turn < 0 || turn >= a.n_pos))) {
    memory_fault(m);
    return;
  }
  int page = 0;
  if (stores) {
    page = m.table[(long long)n * m.max_pages + pi];
    if ((unsigned)page >= (unsigned)m.n_pages) {
      memory_fault(m);
      return;
    }
  }
  float4 c, sn;
  if (a.rotation) {
    const float* t = a.rotation + (long long)turn * D + 4 * l;
    c = load4(t);
    sn = load4(t + D / 2);
  }
  const int nq = a.q ? m.n_head : 0, nk = stores ? m.n_kv_head : 0, heads = nq + 2 * nk;
  const int slot = pos % m.page_tokens;
  for (int h0 = part * HEADS; h0 < heads; h0 += parts * HEADS * BATCH) {
  Raw<T> raw[BATCH][2];                                           // a batch of heads' loads in flight at once
#pragma unroll
  for (int i = 0; i < BATCH; ++i) {
    const int h = h0 + i * parts * HEADS + lane / LH;
    if (h < heads) {
      const int kind = h < nq ? 0 : h < nq + nk ? 1 : 2;          // query, key, value
      const int hh = kind == 0 ? h : kind == 1 ? h - nq : h - nq - nk;
      const T* src = static_cast<const T*>(kind == 0 ? a.q : kind == 1 ? a.k : a.v) +
                     row * (kind == 0 ? a.ldq : kind == 1 ? a.ldk : a.ldv) + (long long)hh * D + 4 * l;
      raw[i][0] = *reinterpret_cast<const Raw<T>*>(src);
      raw[i][1] = *reinterpret_cast<const Raw<T>*>(src + D / 2);
    }
  }
#pragma unroll
  for (int i = 0; i < BATCH; ++i) {
    if (h0 + i * parts * HEADS >= heads) break;                   // the same for the whole warp
    const int h = h0 + i * parts * HEADS + lane / LH;
    const bool on = h < heads;
    const int kind = h < nq ? 0 : h < nq + nk ? 1 : 2;
    const int hh = kind == 0 ? h : kind == 1 ? h - nq : h - nq - nk;
    float4 x = {}, y = {};
    if (on) x = values(raw[i][0]), y = values(raw[i][1]);
    const float* gain = kind == 0 ? a.q_gain : kind == 1 ? a.k_gain : nullptr;
    float ss = dot4(x) + dot4(y);
#pragma unroll
    for (int o = LH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (gain) {
      const float f = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
      const float4 g = load4(gain + 4 * l), e = load4(gain + D / 2 + 4 * l);
      x = make_float4(x.x * f * g.x, x.y * f * g.y, x.z * f * g.z, x.w * f * g.w);
      y = make_float4(y.x * f * e.x, y.y * f * e.y, y.z * f * e.z, y.w * f * e.w);
    }
    if (a.rotation && kind != 2) {
      const float4 u = x;
      x = make_float4(x.x * c.x - y.x * sn.x, x.y * c.y - y.y * sn.y, x.z * c.z - y.z * sn.z, x.w * c.w - y.w * sn.w);
      y = make_float4(y.x * c.x + u.x * sn.x, y.y * c.y + u.y * sn.y, y.z * c.z + u.z * sn.z, y.w * c.w + u.w * sn.w);
    }
    uint32_t byte = 0;
    if constexpr (FORMAT == EVO_CACHE_E4M3) {
      uint32_t b = 0;
      b = amax_bits(amax_bits(amax_bits(amax_bits(b, x.x), x.y), x.z), x.w);
      b = amax_bits(amax_bits(amax_bits(amax_bits(b, y.x), y.y), y.z), y.w);
      byte = scale_byte(group_umax<LH>(b));
    }
    if (!on) continue;
    if (kind == 0) {
      T* dst = static_cast<T*>(a.q_out) + row * a.ldo + (long long)hh * D + 4 * l;
      store4(dst, x);
      store4(dst + D / 2, y);
      continue;
    }
    const long long at = ((long long)page * m.n_kv_head + hh) * m.page_tokens + slot;
    if constexpr (FORMAT == EVO_CACHE_E4M3) {
      uint8_t* dst = static_cast<uint8_t*>(kind == 1 ? m.k_pages : m.v_pages) + at * D + 4 * l;
      *reinterpret_cast<uint32_t*>(dst) = quantise4(x, byte);
      *reinterpret_cast<uint32_t*>(dst + D / 2) = quantise4(y, byte);
      if (l == 0) (kind == 1 ? m.k_scales : m.v_scales)[at] = (uint8_t)byte;
    } else {
      T* dst = static_cast<T*>(kind == 1 ? m.k_pages : m.v_pages) + at * D + 4 * l;
      store4(dst, x);
      store4(dst + D / 2, y);
    }
  }
  }
}

template <typename T, int D>
cudaError_t launch_as(const AppendArgs& a, int parts, cudaStream_t st) {
  const long long warps = (long long)a.rows * parts;
  const unsigned grid = (unsigned)((warps + WARPS - 1) / WARPS);
  if (a.m.format == EVO_CACHE_E4M3)
    append_kernel<T, D, EVO_CACHE_E4M3><<<grid, THREADS, 0, st>>>(a, parts);
  else
    append_kernel<T, D, EVO_CACHE_F32><<<grid, THREADS, 0, st>>>(a, parts);   // the activations' own type
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_append(const AppendArgs& a, cudaStream_t st) {
  const int D = a.m.head_dim, at_once = 256 / D;
  const int heads = (a.q ? a.m.n_head : 0) + (a.k ? 2 * a.m.n_kv_head : 0);
  const int most = (heads + at_once - 1) / at_once;
  // few rows: a row's heads over as many warps as keep the GPU's 152 x 32 warps busy
  const int parts = (int)std::max(1ll, std::min((long long)most, 152ll * 32 / a.rows));
  if (a.m.dtype == EVO_DTYPE_F32) return D == 64 ? launch_as<float, 64>(a, parts, st) : launch_as<float, 128>(a, parts, st);
  return D == 64 ? launch_as<__nv_bfloat16, 64>(a, parts, st) : launch_as<__nv_bfloat16, 128>(a, parts, st);
}

}  // namespace evo
