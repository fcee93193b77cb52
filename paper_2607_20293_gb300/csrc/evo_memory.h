// Internal declarations of the 8-bit unit caches, the paged memory and the latent
// memory: arguments of their kernels and the host functions that launch them.
#pragma once

#include <atomic>
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "evo.h"

namespace evo {

extern thread_local int g_last_cuda_error;   // evo_last_cuda_error (evo_api.cu)

constexpr int UNIT_GROUP = 32;               // values of a unit's cache that share a scale

cudaError_t launch_cache_write(const void* r, int dtype, const uint8_t* refresh, int N, long long per, const float* x,
                               float* y, uint8_t* codes, uint8_t* scales, cudaStream_t st);
cudaError_t launch_cache_add(const uint8_t* codes, const uint8_t* scales, const uint8_t* reuse, int U, int N,
                             long long per, const float* x, float* y, cudaStream_t st);

struct AppendArgs {
  evo_memory m;
  const void *q, *k, *v;
  void* q_out;
  long long ldq, ldk, ldv, ldo;   // elements between rows
  int rows;
  const float *q_gain, *k_gain;   // [head_dim] or null: no norm
  float eps;
  const float* rotation;          // [n_pos][head_dim]: cosines, then sines; null: no rotation
  int n_pos;
  const int* pos0;                // [N] or null
};
cudaError_t launch_append(const AppendArgs& a, cudaStream_t st);

struct AttendArgs {
  evo_memory m;
  const void* q;
  void* out;
  long long ldq, ldo;
  int rows, max_new, max_len;
  int group;                      // query heads a key/value head
  float scale_log2;               // scale * log2(e): the softmax runs on base-2 exponentials
  int causal, window;
  int tiles;                      // row tiles of a (sequence, key/value head): max_new * group rows
  int splits;                     // pieces of the memory that a tile's blocks share
  int cluster;                    // pieces that the blocks of a cluster join among themselves; divides splits
  float* part;                    // [splits / cluster][rows][n_head][head_dim]: unnormalised sums of a cluster's pieces
  float2* ml;                     // [splits / cluster][rows][n_head]: their maximum (base 2) and sum
};
// which kernel takes a call, and how it is cut up.  expand: 8-bit pages are first written out as
// bf16 pages of their own in the scratch, `expand` of them a sequence (0: no)
enum AttendKernel { ATTEND_F32, ATTEND_F32_ROWS, ATTEND_ROWS, ATTEND_TILES };
struct AttendPlan {
  AttendKernel kernel;
  int tile_rows, tiles, splits, cluster, expand;
  size_t scratch;
};
AttendPlan plan_attend(const evo_memory& m, int rows, int max_new, int max_len, int causal, int window);
cudaError_t launch_attend_rows(const AttendArgs& a, int tile_rows, cudaStream_t st);   // evo_attend_rows.cu
cudaError_t launch_attend_f32_rows(const AttendArgs& a, int tile_rows, cudaStream_t st);   // evo_attend_f32.cu
cudaError_t launch_attend_tiles(const AttendArgs& a, cudaStream_t st);                // evo_attend_tiles.cu
cudaError_t launch_attend(AttendArgs& a, const AttendPlan& p, void* scratch, cudaStream_t st);

// The latent memory.  Its calls run on the paged memory's arguments: one key/value head whose keys are a
// page's rows of rank + LATENT_ROPE values and whose values are the first head_dim = rank of them.
constexpr int LATENT_ROPE = 64, LATENT_KEY = 64, LATENT_VALUE = 128;
struct LatentAppendArgs {
  evo_memory m;                   // k_pages: the latent pages
  const void *c, *k, *q;          // c and k null: only queries; q null: only tokens
  void* q_out;
  long long ldc, ldk, ldq, hdq, ldo, hdo;   // elements between rows, and between a row's heads
  int rows;
  const float* c_gain;            // [rank] or null: no norm
  float eps;
  const float* rotation;          // [n_pos][LATENT_ROPE] or null
  int n_pos;
  const int* pos0;
};
cudaError_t launch_latent_append(const LatentAppendArgs& a, cudaStream_t st);   // evo_latent.cu
struct LatentPlan {
  int tile_rows, tiles;           // rows of an item, items of a sequence
  int splits, blocks;             // 2: the launch's blocks share items
  size_t scratch;
};
LatentPlan plan_latent(const evo_memory& m, int rows, int max_new, int max_len, int causal, int window);   // evo_latent.cu
cudaError_t launch_latent_attend(AttendArgs& a, const LatentPlan& p, void* scratch, cudaStream_t st);
cudaError_t launch_latent_tiles(const AttendArgs& a, const LatentPlan& p, cudaStream_t st);  // up to 64 bf16 rows an item: evo_latent_tiles.cu
cudaError_t launch_latent_wide(const AttendArgs& a, const LatentPlan& p, cudaStream_t st);   // 128: evo_latent_wide.cu
int latent_f32_rows(int rank, long long all, int n_seq);   // rows of an item of fp32 rows, evo_latent_f32.cu
cudaError_t launch_latent_f32(const AttendArgs& a, const LatentPlan& p, cudaStream_t st);
struct LatentExpandArgs {
  evo_memory m, to;               // the latent memory, and the one that its tokens are written to
  const void *w_k, *w_v;          // [n_head][LATENT_KEY][rank], [n_head][LATENT_VALUE][rank]
  const int* first;               // [n_seq] or null: the first token of each that is written
  int max_new, max_len;
};
cudaError_t launch_latent_expand(const LatentExpandArgs& a, cudaStream_t st);   // evo_latent_expand.cu

// tensor map of a pool of pages: its rows (a token of a head each) in boxes of
// box_rows rows x 128 bytes (64 where a row has no more), swizzled by the box's width
bool page_map(CUtensorMap* map, const evo_memory& m, const void* pages, int box_rows);
// the same of a latent memory's pages, a row a token
bool latent_map(CUtensorMap* map, const evo_memory& m, int box_rows);
// of a call's bf16 queries whose rows lie behind one another, a row a (token, head)
bool query_map(CUtensorMap* map, const AttendArgs& a, int box_rows);

// lets a kernel have this much dynamic shared memory; `done`: a bit for each device where it has it
template <typename K>
cudaError_t allow_smem(K kernel, int smem, std::atomic<uint64_t>& done) {
  int dev;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1))) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  return e;
}

// ---------------------------------------------------------------- device helpers

// rows of sequence n of a call: [first, first + count); a malformed entry reports
// itself and gives no rows
struct SeqRows { int first, count; };
__device__ __forceinline__ void memory_fault(const evo_memory& m) {
  if (m.status) *m.status = EVO_ERR_CORRUPT;
}
__device__ __forceinline__ SeqRows seq_rows(const evo_memory& m, int n, int rows, int max_new) {
  SeqRows s;
  if (!m.starts) {
    s.count = rows / m.n_seq;
    s.first = n * s.count;
    return s;
  }
  s.first = m.starts[n];
  s.count = m.starts[n + 1] - s.first;
  if (s.first < 0 || s.count < 0 || s.count > max_new || s.first > rows - s.count) {
    memory_fault(m);
    s.first = s.count = 0;
  }
  return s;
}
// tokens in the memory of sequence n, at most max_len (which the table's rows can name)
__device__ __forceinline__ int seq_len(const evo_memory& m, int n, int max_len) {
  const int len = m.lens[n];
  if (len < 0 || len > max_len) {
    memory_fault(m);
    return len < 0 ? 0 : max_len;
  }
  return len;
}
// page i of sequence n; an entry outside the pool reports itself and stands for page 0
__device__ __forceinline__ int seq_page(const evo_memory& m, int n, int i) {
  const int p = m.table[(long long)n * m.max_pages + i];
  if ((unsigned)p >= (unsigned)m.n_pages) {
    memory_fault(m);
    return 0;
  }
  return p;
}

}  // namespace evo
