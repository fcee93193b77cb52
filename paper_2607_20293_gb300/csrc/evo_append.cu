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
// A warp takes a row (a token).  D / 16 lanes hold one head, each the 8 values at
// 8l and the 8 at D/2 + 8l: both halves of every rotated pair are in one lane, so
// the rotation needs no exchange, and the norm and the largest magnitude are
// shuffles over those lanes.
//
// Single tokens are bound by the chain starts -> length -> table -> page.  Calls of few
// rows spread a row's heads over several warps (64 tokens of 24 heads of 64: 6.2 us).
// Calls of many rows copy whole rows to shared memory by bulk copies, issued before the
// chain is walked, and walk it for all rows of a warp at once: 11,700 rows of 24 heads of
// 128 take 29.1 us (4.7 TB/s, 70 % of the copy rate), against 32.7 with loads to registers
// and one chain a row.  What bounds them is latency: a warp has one row at a time, so that
// nothing of its own is on the way while it computes and stores, and the warps take
// their four rows in step (half of the issue slots are empty, and DRAM has room).
#include <algorithm>
#include <cstdint>
#include <type_traits>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_mem_ptx.cuh"
#include "evo_memory.h"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int RING_WARPS = 4, RING_THREADS = 32 * RING_WARPS;
constexpr int STAGES = 1;                           // rows a warp holds: 20 warps a SM with one each are ahead of 16 with two (30.1 us)
// blocks a SM (6: 32.1 us).  Their 96 registers a thread hold bf16 rows over 8-bit pages; with bf16 pages 8 bytes
// a thread are spilled, with fp32 rows 56
constexpr int RING_BLOCKS = 5;
constexpr int BATCH = 2;                            // head groups whose loads a warp has in flight

// eight values of a row as they are in memory, and as four pairs of fp32
template <typename T>
struct Raw {
  uint4 u[sizeof(T) / 2];
};
__device__ __forceinline__ void values(const Raw<float>& r, float2 (&v)[4]) {
  v[0] = make_float2(__uint_as_float(r.u[0].x), __uint_as_float(r.u[0].y));
  v[1] = make_float2(__uint_as_float(r.u[0].z), __uint_as_float(r.u[0].w));
  v[2] = make_float2(__uint_as_float(r.u[1].x), __uint_as_float(r.u[1].y));
  v[3] = make_float2(__uint_as_float(r.u[1].z), __uint_as_float(r.u[1].w));
}
__device__ __forceinline__ void values(const Raw<__nv_bfloat16>& r, float2 (&v)[4]) {
  const uint32_t w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void store8(float* p, const float2 (&v)[4]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float2 (&v)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[i].x, v[i].y);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
enum { QUERY, KEY, VALUE };

// 8 + 8 values of a head (columns 8 l and D/2 + 8 l): norm, rotation and store
struct Lane {
  float2 c[4], s[4];              // cosines and sines of the row
  float2 g0[4], g1[4];            // gain
};
__device__ __forceinline__ void load_pairs(const float* p, float2 (&v)[4]) {
  Raw<float> r;
  r.u[0] = reinterpret_cast<const uint4*>(p)[0];
  r.u[1] = reinterpret_cast<const uint4*>(p)[1];
  values(r, v);
}

template <typename T, int D, int FORMAT, int KIND>
__device__ __forceinline__ void put_head(const AppendArgs& a, const Lane& t, const Raw<T>& r0, const Raw<T>& r1, bool norm,
                                         bool turn, bool on, long long at, int row, int head, int l) {
  constexpr int LH = D / 16;
  float2 x[4], y[4];
  values(r0, x);
  values(r1, y);
  if (KIND != VALUE && norm) {
    float2 ss = mul_pair(x[0], x[0]), sy = mul_pair(y[0], y[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) ss = fma_pair(x[i], x[i], ss), sy = fma_pair(y[i], y[i], sy);
    float sum = (ss.x + ss.y) + (sy.x + sy.y);
#pragma unroll
    for (int o = LH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float f = rsqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = mul_pair(mul_pair(x[i], make_float2(f, f)), t.g0[i]);
      y[i] = mul_pair(mul_pair(y[i], make_float2(f, f)), t.g1[i]);
    }
  }
  if (KIND != VALUE && turn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 u = x[i], s = t.s[i];
      x[i] = fma_pair(y[i], make_float2(-s.x, -s.y), mul_pair(u, t.c[i]));
      y[i] = fma_pair(u, s, mul_pair(y[i], t.c[i]));
    }
  }
  if constexpr (KIND == QUERY) {
    T* dst = static_cast<T*>(a.q_out) + row * a.ldo + head * D + 8 * l;
    if (on) store8(dst, x), store8(dst + D / 2, y);
  } else if constexpr (FORMAT == EVO_CACHE_E4M3) {
    uint32_t b = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) b = amax_bits(amax_bits(amax_bits(amax_bits(b, x[i].x), x[i].y), y[i].x), y[i].y);
    const uint32_t byte = scale_byte(group_umax<LH>(b));
    uint8_t* dst = static_cast<uint8_t*>(KIND == KEY ? a.m.k_pages : a.m.v_pages) + at * D + 8 * l;
    if (on) {
      *reinterpret_cast<uint2*>(dst) = make_uint2(quantise4(make_float4(x[0].x, x[0].y, x[1].x, x[1].y), byte),
                                                  quantise4(make_float4(x[2].x, x[2].y, x[3].x, x[3].y), byte));
      *reinterpret_cast<uint2*>(dst + D / 2) = make_uint2(quantise4(make_float4(y[0].x, y[0].y, y[1].x, y[1].y), byte),
                                                          quantise4(make_float4(y[2].x, y[2].y, y[3].x, y[3].y), byte));
      if (l == 0) (KIND == KEY ? a.m.k_scales : a.m.v_scales)[at] = (uint8_t)byte;
    }
  } else {
    T* dst = static_cast<T*>(KIND == KEY ? a.m.k_pages : a.m.v_pages) + at * D + 8 * l;
    if (on) store8(dst, x), store8(dst + D / 2, y);
  }
}

// heads [0, n) of one kind: a warp takes HEADS of them at once, every parts-th such group
// from `first` on, the loads of BATCH groups in flight
template <typename T, int D, int FORMAT, int KIND>
__device__ __forceinline__ void put_heads(const AppendArgs& a, Lane& t, const T* from, const float* gain, int n, int first,
                                          int parts, long long at0, int row, int lane) {
  constexpr int LH = D / 16, HEADS = 32 / LH;
  const int l = lane % LH, hl = lane / LH;
  const bool norm = KIND != VALUE && gain, turn = KIND != VALUE && a.rotation;
  if (first * HEADS >= n) return;
  if (norm) load_pairs(gain + 8 * l, t.g0), load_pairs(gain + D / 2 + 8 * l, t.g1);
  const T* src = from + 8 * l;
  for (int g0 = first; g0 * HEADS < n; g0 += parts * BATCH) {
    Raw<T> r[BATCH][2] = {};
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = (g0 + i * parts) * HEADS + hl;
      if (h < n) {
#pragma unroll
        for (int e = 0; e < (int)sizeof(T) / 2; ++e) {
          r[i][0].u[e] = reinterpret_cast<const uint4*>(src + h * D)[e];
          r[i][1].u[e] = reinterpret_cast<const uint4*>(src + h * D + D / 2)[e];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = (g0 + i * parts) * HEADS + hl;
      if ((g0 + i * parts) * HEADS >= n) break;      // the same for the whole warp
      put_head<T, D, FORMAT, KIND>(a, t, r[i][0], r[i][1], norm, turn, h < n, at0 + (long long)h * a.m.page_tokens, row, h, l);
    }
  }
}

// where a row belongs
struct Place {
  int turn;                       // position for the rotation, or -1: the row is not touched
  int page, slot;
};

// the place of this lane's row; reports what it cannot place
__device__ __forceinline__ Place place_of(const AppendArgs& a, int row) {
  const evo_memory& m = a.m;
  Place p{-1, 0, 0};
  if (row >= a.rows) return p;
  int n;
  if (m.starts) {
    if (row < m.starts[0] || row >= m.starts[m.n_seq]) return p;  // behind the last sequence
    int lo = 0, hi = m.n_seq;                                     // starts[lo] <= row < starts[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (m.starts[mid] <= row) lo = mid;
      else hi = mid;
    }
    n = lo;
  } else {
    n = row / (a.rows / m.n_seq);
  }
  const SeqRows s = seq_rows(m, n, a.rows, a.rows);
  if (row < s.first || row >= s.first + s.count) return p;        // malformed starts
  const int pos = m.lens[n] - s.count + (row - s.first);
  const int turn = a.rotation ? pos + (a.pos0 ? a.pos0[n] : 0) : 0;
  const int pi = pos >> (31 - __clz(m.page_tokens));
  if (pos < 0 || pi >= m.max_pages || turn < 0 || (a.rotation && turn >= a.n_pos)) {
    memory_fault(m);
    return p;
  }
  if (a.k) {
    p.page = m.table[(long long)n * m.max_pages + pi];
    if ((unsigned)p.page >= (unsigned)m.n_pages) {
      memory_fault(m);
      return p;
    }
  }
  p.turn = turn;
  p.slot = pos & (m.page_tokens - 1);
  return p;
}

// a row's heads, from wherever its queries, keys and values lie: groups of HEADS heads of one
// kind, of which this warp takes part, part + parts, ...
template <typename T, int D, int FORMAT>
__device__ __forceinline__ void put_row(const AppendArgs& a, const T* q, const T* k, const T* v, const float* rotation, int part,
                                        int parts, long long at, int row, int lane) {
  constexpr int HEADS = 512 / D;
  Lane t;
  if (a.rotation) {
    load_pairs(rotation + 8 * (lane % (D / 16)), t.c);
    load_pairs(rotation + D / 2 + 8 * (lane % (D / 16)), t.s);
  }
  const int nq = a.q ? a.m.n_head : 0, nk = a.k ? a.m.n_kv_head : 0;
  const int gq = (nq + HEADS - 1) / HEADS, gk = (nk + HEADS - 1) / HEADS;
  const int fk = (part + parts - gq % parts) % parts, fv = (fk + parts - gk % parts) % parts;
  put_heads<T, D, FORMAT, QUERY>(a, t, q, a.q_gain, nq, part, parts, 0, row, lane);
  put_heads<T, D, FORMAT, KEY>(a, t, k, a.k_gain, nk, fk, parts, at, row, lane);
  put_heads<T, D, FORMAT, VALUE>(a, t, v, nullptr, nk, fv, parts, at, row, lane);
}

// few rows: a row's heads over `parts` warps, straight from global memory
template <typename T, int D, int FORMAT>
__global__ void __launch_bounds__(THREADS) append_kernel(const __grid_constant__ AppendArgs a, int parts) {
  const int lane = threadIdx.x & 31;
  const int w = blockIdx.x * WARPS + (threadIdx.x >> 5), row = w / parts;
  if (row >= a.rows) return;
  const Place p = place_of(a, row);
  if (p.turn < 0) return;
  const long long at = (long long)p.page * a.m.n_kv_head * a.m.page_tokens + p.slot;
  put_row<T, D, FORMAT>(a, static_cast<const T*>(a.q) + row * a.ldq, static_cast<const T*>(a.k) + row * a.ldk,
                        static_cast<const T*>(a.v) + row * a.ldv, a.rotation + (long long)p.turn * D, w % parts, parts, at, row,
                        lane);
}

// many rows: a warp takes `each` rows behind one another.  Their places are looked up together, a
// lane each, and their data arrive in the warp's ring of STAGES rows by bulk copies, so that neither
// chain of loads is waited out once a row.
template <typename T, int D, int FORMAT>
__global__ void __launch_bounds__(RING_THREADS, RING_BLOCKS) append_ring_kernel(const __grid_constant__ AppendArgs a, int each) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ __align__(8) uint64_t full[RING_WARPS][STAGES];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int first = (blockIdx.x * RING_WARPS + warp) * each, count = min(each, a.rows - first);
  if (threadIdx.x == 0) {
    for (int i = 0; i < RING_WARPS * STAGES; ++i) tc::mbar_init1(&full[0][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  const int qb = a.q ? a.m.n_head * D * (int)sizeof(T) : 0, kb = a.k ? a.m.n_kv_head * D * (int)sizeof(T) : 0;
  const int rb = a.rotation ? D * 4 : 0, bytes = qb + 2 * kb + rb;
  uint8_t* const mine = ring + warp * STAGES * bytes;
  const auto copy_data = [&](int i) {
    if (i >= count || lane != 0) return;
    const long long row = first + i;
    const uint32_t dst = tc::su32(mine + i % STAGES * bytes), bar = tc::su32(&full[warp][i % STAGES]);
    if (qb) bulk_load(dst, static_cast<const T*>(a.q) + row * a.ldq, qb, bar);
    if (kb) bulk_load(dst + qb, static_cast<const T*>(a.k) + row * a.ldk, kb, bar);
    if (kb) bulk_load(dst + qb + kb, static_cast<const T*>(a.v) + row * a.ldv, kb, bar);
  };
  for (int i = 0; i < STAGES; ++i) copy_data(i);    // on their way while the places are looked up
  const Place place = place_of(a, lane < count ? first + lane : a.rows);
  const auto copy_rotation = [&](int i) {           // and the stage's count of bytes
    const int turn = __shfl_sync(0xffffffffu, place.turn, i & 31);
    if (i >= count || lane != 0) return;
    uint64_t* bar = &full[warp][i % STAGES];
    const int r = turn < 0 ? 0 : rb;                // a row that is not touched has none
    tc::mbar_expect_tx(bar, qb + 2 * kb + r);
    if (r) bulk_load(tc::su32(mine + i % STAGES * bytes + qb + 2 * kb), a.rotation + (long long)turn * D, r, tc::su32(bar));
  };
  for (int i = 0; i < STAGES; ++i) copy_rotation(i);
  bool ok = true;
  for (int i = 0; i < count && ok; ++i) {
    const int stage = i % STAGES, turn = __shfl_sync(0xffffffffu, place.turn, i);
    const int page = __shfl_sync(0xffffffffu, place.page, i), slot = __shfl_sync(0xffffffffu, place.slot, i);
    ok = __all_sync(0xffffffffu, wait_full(tc::su32(&full[warp][stage]), (i / STAGES) & 1));
    if (ok && turn >= 0) {
      const uint8_t* src = mine + stage * bytes;
      put_row<T, D, FORMAT>(a, reinterpret_cast<const T*>(src), reinterpret_cast<const T*>(src + qb),
                            reinterpret_cast<const T*>(src + qb + kb), reinterpret_cast<const float*>(src + qb + 2 * kb), 0, 1,
                            (long long)page * a.m.n_kv_head * a.m.page_tokens + slot, first + i, lane);
    }
    __syncwarp();                                   // every lane has read the stage
    if (ok) copy_data(i + STAGES), copy_rotation(i + STAGES);
  }
  if (__syncthreads_or(!ok)) settle(a.m.status);    // a copy did not arrive
}

template <typename T, int D, int FORMAT>
cudaError_t launch_as(const AppendArgs& a, cudaStream_t st) {
  const int row = ((a.q ? a.m.n_head : 0) + (a.k ? 2 * a.m.n_kv_head : 0)) * D * (int)sizeof(T) + (a.rotation ? 4 * D : 0);
  const int smem = RING_WARPS * STAGES * row, blocks = std::min(RING_BLOCKS, 220 * 1024 / std::max(smem, 1));
  const int warps = 152 * RING_WARPS * blocks;      // resident at once
  if (blocks >= 2 && a.rows >= 2 * warps) {
    const auto k = append_ring_kernel<T, D, FORMAT>;
    static std::atomic<uint64_t> done{0};           // the most that a call takes: calls of other sizes may launch meanwhile
    const cudaError_t e = allow_smem(k, 110 * 1024, done);
    if (e != cudaSuccess) return e;
    const int each = std::min(32, (a.rows + warps - 1) / warps);
    const int need = (a.rows + each - 1) / each;
    k<<<(need + RING_WARPS - 1) / RING_WARPS, RING_THREADS, smem, st>>>(a, each);
    return cudaGetLastError();
  }
  const int at_once = 512 / D;
  const int most = (a.q ? (a.m.n_head + at_once - 1) / at_once : 0) + (a.k ? 2 * ((a.m.n_kv_head + at_once - 1) / at_once) : 0);
  // a row's heads over as many warps as keep the GPU's 152 x 32 busy
  const int parts = (int)std::max(1ll, std::min((long long)most, 152ll * 32 / a.rows));
  const long long warps_needed = (long long)a.rows * parts;
  append_kernel<T, D, FORMAT><<<(unsigned)((warps_needed + WARPS - 1) / WARPS), THREADS, 0, st>>>(a, parts);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const AppendArgs& a, cudaStream_t st) {
  const bool d64 = a.m.head_dim == 64;              // EVO_CACHE_F32 stands for the rows' own type
  if (a.m.format == EVO_CACHE_E4M3) return d64 ? launch_as<T, 64, EVO_CACHE_E4M3>(a, st) : launch_as<T, 128, EVO_CACHE_E4M3>(a, st);
  return d64 ? launch_as<T, 64, EVO_CACHE_F32>(a, st) : launch_as<T, 128, EVO_CACHE_F32>(a, st);
}

}  // namespace

cudaError_t launch_append(const AppendArgs& a, cudaStream_t st) {
  return a.m.dtype == EVO_DTYPE_F32 ? launch_type<float>(a, st) : launch_type<__nv_bfloat16>(a, st);
}

}  // namespace evo
