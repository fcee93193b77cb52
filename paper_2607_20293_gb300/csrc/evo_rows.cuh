// What the appends to paged memories share: rows in registers as pairs of fp32, and
// the place of a row in its sequence's pages.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>

#include "evo_memory.h"

namespace evo {

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
__device__ __forceinline__ void load_pairs(const float* p, float2 (&v)[4]) {
  Raw<float> r;
  r.u[0] = reinterpret_cast<const uint4*>(p)[0];
  r.u[1] = reinterpret_cast<const uint4*>(p)[1];
  values(r, v);
}

// where a row belongs
struct Place {
  int turn;                       // position for the rotation, or -1: the row is not touched
  int page, slot;
};

// the place of this lane's row; reports what it cannot place.  Args has the call's memory view m, rows,
// rotation with n_pos and pos0, and k: whether there is something for the pages
template <typename Args>
__device__ __forceinline__ Place place_of(const Args& a, int row) {
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

}  // namespace evo
