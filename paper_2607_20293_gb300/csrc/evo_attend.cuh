// What the attention kernels over a paged memory share: which keys a row sees,
// the pieces that a memory is split into, and the partial results of a piece.
//
// The rows of a (sequence, key/value head) are its chunk's tokens times the
// `group` query heads that share the head, token-major: row i is token i / group,
// query head i % group of the group.  A block takes a tile of such rows and one
// piece of the keys that any of them sees.
#pragma once

#include <cuda_bf16.h>

#include "evo_memory.h"

namespace evo {

struct Tile {
  int n, kv_head, tile, split;
  int first, count;             // the sequence's rows of the call
  int len;                      // tokens in its memory
};

__device__ __forceinline__ Tile tile_of_block(const AttendArgs& a) {
  Tile t;
  int b = blockIdx.x;
  t.split = b % a.splits;
  b /= a.splits;
  t.tile = b % a.tiles;
  b /= a.tiles;
  t.kv_head = b % a.m.n_kv_head;
  t.n = b / a.m.n_kv_head;
  const SeqRows s = seq_rows(a.m, t.n, a.rows, a.max_new);
  t.first = s.first;
  t.count = s.count;
  t.len = seq_len(a.m, t.n, a.max_len);
  return t;
}

// keys [lo, hi) that token j of the chunk sees
struct Range { int lo, hi; };
__device__ __forceinline__ Range seen_by(const AttendArgs& a, const Tile& t, int j) {
  Range r;
  r.hi = a.causal ? min(t.len, t.len - t.count + j + 1) : t.len;
  r.hi = max(r.hi, 0);
  r.lo = a.window ? max(0, r.hi - a.window) : 0;
  return r;
}

// keys that some row of tokens j0 .. j1 sees
__device__ __forceinline__ Range seen_by_tile(const AttendArgs& a, const Tile& t, int j0, int j1) {
  return {seen_by(a, t, j0).lo, seen_by(a, t, j1).hi};
}

// this block's piece of the range, cut at multiples of `step` keys
__device__ __forceinline__ Range piece_of(const AttendArgs& a, const Tile& t, Range r, int step) {
  const int lo = r.lo / step, hi = (r.hi + step - 1) / step;
  const int each = (max(hi - lo, 0) + a.splits - 1) / a.splits;
  return {max(r.lo, (lo + t.split * each) * step), min(r.hi, (lo + (t.split + 1) * each) * step)};
}

// index of (row of the call, query head) in the partial results of a cluster's pieces
__device__ __forceinline__ long long part_index(const AttendArgs& a, int part, int row, int head) {
  return ((long long)part * a.rows + row) * a.m.n_head + head;
}

__device__ __forceinline__ void cluster_arrive_wait() {
  __syncwarp();                                    // the barrier wants whole warps; lanes left the loop before at their own times
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address of this block's shared memory at p in the block of another rank of the cluster
__device__ __forceinline__ uint32_t in_rank(const void* p, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ float2 remote_f2(uint32_t p) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(p));
  return v;
}
__device__ __forceinline__ float4 remote_f4(uint32_t p) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(p));
  return v;
}

__device__ __forceinline__ void store_out(float* p, float4 v, float f) {
  *reinterpret_cast<float4*>(p) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
}
__device__ __forceinline__ void store_out(__nv_bfloat16* p, float4 v, float f) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x * f, v.y * f), b = __floats2bfloat162_rn(v.z * f, v.w * f);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// The end of a block of few rows: 4 values d .. d + 3 of the sums of row R of the tile, its maximum
// m and sum l go to the output, or to the partial results where a join kernel follows.
template <typename T, int D>
__device__ __forceinline__ void put_result(const AttendArgs& a, const Tile& t, int R, int d, float4 x, float m, float l) {
  const int row = t.first + R / a.group, head = t.kv_head * a.group + R % a.group;
  if (a.splits == a.cluster) {
    store_out(static_cast<T*>(a.out) + row * a.ldo + (long long)head * D + d, x, l == 0.f ? 0.f : 1.f / l);
  } else {
    const long long at = part_index(a, t.split / a.cluster, row, head);
    *reinterpret_cast<float4*>(a.part + at * D + d) = x;
    if (d == 0) a.ml[at] = make_float2(m, l);
  }
}

// Joins the pieces of a cluster's blocks through their shared memory: `sums` [ROWS][ld] and `ml`
// [ROWS] hold each block's; every block finishes its share of the values.  All threads of all
// blocks of the cluster call it.
template <typename T, int D, int ROWS, int THREADS>
__device__ __forceinline__ void join_cluster(const AttendArgs& a, const Tile& t, const float* sums, int ld, const float2* ml, int r0,
                                             int rows) {
  cluster_arrive_wait();
  const int rank = t.split % a.cluster;
  for (int i = rank * THREADS + threadIdx.x; i < ROWS * D / 4; i += a.cluster * THREADS) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, R = r0 + r;
    if (R >= rows) break;
    float m = -INFINITY, l = 0.f;
    for (int c = 0; c < a.cluster; ++c) m = fmaxf(m, remote_f2(in_rank(ml + r, c)).x);
    const float ref = m == -INFINITY ? 0.f : m;
    float4 x = {};
#pragma unroll 4
    for (int c = 0; c < a.cluster; ++c) {
      const float2 o = remote_f2(in_rank(ml + r, c));
      const float4 y = remote_f4(in_rank(sums + r * ld + d, c));
      const float f = exp2f(o.x - ref);
      l = fmaf(o.y, f, l);
      x = make_float4(fmaf(y.x, f, x.x), fmaf(y.y, f, x.y), fmaf(y.z, f, x.z), fmaf(y.w, f, x.w));
    }
    put_result<T, D>(a, t, R, d, x, m, l);
  }
  cluster_arrive_wait();                           // no block ends while another reads its shared memory
}

// launches a block a piece, the pieces of a cluster as one
template <typename... K, typename... A>
cudaError_t launch_pieces(void (*kernel)(K...), const AttendArgs& a, int threads, int smem, std::atomic<uint64_t>& done,
                          cudaStream_t st, const A&... args) {
  const cudaError_t e = allow_smem(kernel, smem, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = (unsigned)((long long)a.m.n_seq * a.m.n_kv_head * a.tiles * a.splits);
  cfg.blockDim = threads;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = a.cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = a.cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, a, args...);
}

}  // namespace evo
