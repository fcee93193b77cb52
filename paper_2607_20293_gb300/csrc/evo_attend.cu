// Attention over a paged memory: the fp32 kernel for many rows, the expansion of
// 8-bit pages, the join of split memories and the choice among the kernels:
//
//   rows a key/value head    bf16 rows                          fp32 rows
//   up to 32 (fp32: 16)      evo_attend_rows.cu (mma.sync)      evo_attend_f32.cu
//   more                     evo_attend_tiles.cu (tcgen05);     attend_kernel
//                            8-bit pages from 65 rows on
// (8-bit pages of 33 to 64 rows: two tiles of evo_attend_rows.cu).
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(s_j - max s),  s_j = scale log2(e) <q, k_j>
//
// over the keys j that the row sees, in one pass with a running maximum and sum
// (a row that sees none is zero).  A memory split over several blocks leaves each
// piece's maximum, sum and unnormalised values, which a second kernel joins.
//
// fp32 kernel: a block of 128 threads takes 8 RM rows and 64 keys at a time; the
// thread at (ty, tx) of an 8 x 16 grid computes RM rows x 4 keys of the scores and RM
// rows x D/16 columns of the output.  All products are fp32 (packed in pairs: half the
// issue slots); the multiply-add units bound it: 1,024 rows over 4,096 keys of 64, 8
// heads, 251 us = 34 TFLOP/s, registers leaving 12 warps a SM to hide their latency.  There is no tensor-core form of it:
// three tf32 products for one of fp32 are 170 multiply-adds a cycle and SM, against 128.
#include <algorithm>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
#include "evo_mem_ptx.cuh"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int BN = 64, THREADS = 128, JOIN_THREADS = 256;
// from this many rows a key/value head on, 8-bit pages are written out as bf16 pages for the tcgen05
// kernel (16 sequences of 8,192 keys of 64, us with / without: 64 rows 131 / 129, 96 rows 131 / 152,
// 256 rows 165 / 362; of 128: 237 / 196, 238 / 331, 267 / 693), while they fit this many bytes
constexpr int EXPAND_ROWS = 65;
constexpr long long EXPAND_MOST = 4ll << 30;

template <int D, int RM>
struct Smem {
  static constexpr int BM = 8 * RM;
  float q[BM][D];
  float k[BN][D + 4];           // rows 4 banks apart: 8 rows' float4 in a phase do not collide
  float v[BN][D];
  float p[BM][BN + 4];
};

__device__ __forceinline__ void copy16(float* dst, const float* src, bool on) {   // zeros where it is off
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
               "r"(on ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// (top, sum, o) joined with another piece's
__device__ __forceinline__ void join(float& top, float& sum, float4& o, float2 ml, float4 p) {
  const float now = fmaxf(top, ml.x), base = now == -INFINITY ? 0.f : now;
  const float f = exp2f(top - base), g = exp2f(ml.x - base);
  top = now;
  sum = sum * f + ml.y * g;
  o = make_float4(o.x * f + p.x * g, o.y * f + p.y * g, o.z * f + p.z * g, o.w * f + p.w * g);
}

template <int D, int FORMAT, int RM>
__global__ void __launch_bounds__(THREADS, D == 64 ? 3 : 2) attend_kernel(const __grid_constant__ AttendArgs a) {
  constexpr bool CODES = FORMAT == EVO_CACHE_E4M3;
  extern __shared__ __align__(16) uint8_t raw[];
  using S = Smem<D, RM>;
  S& sm = *reinterpret_cast<S*>(raw);
  constexpr int BM = 8 * RM, DC = D / 64;          // a thread's columns: 4 tx + 64 c .. + 3
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  const Tile t = tile_of_block(a);
  const int rows = t.count * a.group, r0 = t.tile * BM;
  if (r0 >= rows) return;
  const int last = min(r0 + BM, rows) - 1;
  const Range first_row = seen_by(a, t, r0 / a.group), last_row = seen_by(a, t, last / a.group);
  const Range all = piece_of(a, t, {first_row.lo, last_row.hi}, BN);
  const int whole_lo = max(last_row.lo, all.lo), whole_hi = min(first_row.hi, all.hi);
  const int shift = 31 - __clz(a.m.page_tokens);

  for (int i = tid; i < BM * D / 4; i += THREADS) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, R = r0 + r;
    float4 x = {};
    if (R < rows)
      x = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + (t.first + R / a.group) * a.ldq +
                                           (long long)(t.kv_head * a.group + R % a.group) * D + d);
    *reinterpret_cast<float4*>(&sm.q[r][d]) = x;
  }
  Range seen[RM];
  float mx[RM], sum[RM];
  float2 o[RM][DC][2];
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    const int R = r0 + ty * RM + i;
    seen[i] = R < rows ? seen_by(a, t, R / a.group) : Range{0, 0};
    seen[i] = {max(seen[i].lo, all.lo), min(seen[i].hi, all.hi)};
    mx[i] = -INFINITY;
    sum[i] = 0.f;
#pragma unroll
    for (int c = 0; c < DC; ++c) o[i][c][0] = o[i][c][1] = make_float2(0.f, 0.f);
  }
  // row of the pool that holds a key, or -1 outside the piece
  const auto row_of = [&](int key) -> long long {
    if (key < all.lo || key >= all.hi) return -1;
    return ((long long)seq_page(a.m, t.n, key >> shift) * a.m.n_kv_head + t.kv_head) * a.m.page_tokens +
           (key & (a.m.page_tokens - 1));
  };
  constexpr int CV = CODES ? BN * D / 16 / THREADS : 1;      // 16-code vectors a thread brings, keys and values each
  uint4 kc[CV], vc[CV];
  uint32_t kscale[CV], vscale[CV];
  const auto bring = [&](int k0) {
    if constexpr (CODES) {
#pragma unroll
      for (int i = 0; i < CV; ++i) {
        const int v = tid + i * THREADS, r = v / (D / 16), d = v % (D / 16) * 16;
        const long long at = row_of(k0 + r);
        kc[i] = vc[i] = make_uint4(0, 0, 0, 0);
        kscale[i] = vscale[i] = 1;
        if (at >= 0) {
          kc[i] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.m.k_pages) + at * D + d);
          vc[i] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.m.v_pages) + at * D + d);
          kscale[i] = a.m.k_scales[at];
          vscale[i] = a.m.v_scales[at];
        }
      }
    } else {
#pragma unroll 4
      for (int i = tid; i < BN * D / 4; i += THREADS) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        const long long at = row_of(k0 + r);
        copy16(&sm.k[r][d], static_cast<const float*>(a.m.k_pages) + max(at, 0ll) * D + d, at >= 0);
        copy16(&sm.v[r][d], static_cast<const float*>(a.m.v_pages) + max(at, 0ll) * D + d, at >= 0);
      }
    }
  };
  const auto unpack = [&] {                        // the codes in registers to shared memory
    if constexpr (CODES) {
#pragma unroll
      for (int i = 0; i < CV; ++i) {
        const int v = tid + i * THREADS, r = v / (D / 16), d = v % (D / 16) * 16;
        const float kf = scale_value(kscale[i]), vf = scale_value(vscale[i]);
        const uint32_t kw[4] = {kc[i].x, kc[i].y, kc[i].z, kc[i].w}, vw[4] = {vc[i].x, vc[i].y, vc[i].z, vc[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 k = codes4(kw[e]), x = codes4(vw[e]);
          *reinterpret_cast<float4*>(&sm.k[r][d + 4 * e]) = make_float4(k.x * kf, k.y * kf, k.z * kf, k.w * kf);
          *reinterpret_cast<float4*>(&sm.v[r][d + 4 * e]) = make_float4(x.x * vf, x.y * vf, x.z * vf, x.w * vf);
        }
      }
    }
  };
  for (int k0 = all.lo / BN * BN; k0 < all.hi; k0 += BN) {
    const bool whole = k0 >= whole_lo && k0 + BN <= whole_hi;
    __syncthreads();
    bring(k0);
    if constexpr (CODES) unpack();
    else copies_done();
    __syncthreads();
    float2 s2[RM][4] = {};                         // sums over the even and the odd dimensions
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
      float4 k[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][d]);
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const float4 q = *reinterpret_cast<const float4*>(&sm.q[ty * RM + i][d]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s2[i][j] = fma_pair(make_float2(q.x, q.y), make_float2(k[j].x, k[j].y), s2[i][j]);
          s2[i][j] = fma_pair(make_float2(q.z, q.w), make_float2(k[j].z, k[j].w), s2[i][j]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      float s[4], top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = k0 + tx + 16 * j;
        s[j] = (s2[i][j].x + s2[i][j].y) * a.scale_log2;
        if (!whole && (key < seen[i].lo || key >= seen[i].hi)) s[j] = -INFINITY;
        top = fmaxf(top, s[j]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
      const float now = fmaxf(mx[i], top), base = now == -INFINITY ? 0.f : now;
      const float keep = exp2f(mx[i] - base);
      mx[i] = now;
      float add = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2f(s[j] - base);
        add += p;
        sm.p[ty * RM + i][tx + 16 * j] = p;
      }
      sum[i] = sum[i] * keep + add;                // this thread's keys; joined at the end
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) o[i][c][h] = make_float2(o[i][c][h].x * keep, o[i][c][h].y * keep);
    }
    __syncwarp();               // a row's weights come from its own half warp
    if (whole) {
#pragma unroll 2
      for (int j = 0; j < BN; j += 4) {
        float4 v[4][DC];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < DC; ++c) v[e][c] = *reinterpret_cast<const float4*>(&sm.v[j + e][4 * tx + 64 * c]);
#pragma unroll
        for (int i = 0; i < RM; ++i) {
          const float4 p4 = *reinterpret_cast<const float4*>(&sm.p[ty * RM + i][j]);
          const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int c = 0; c < DC; ++c) {
              o[i][c][0] = fma_pair(make_float2(p[e], p[e]), make_float2(v[e][c].x, v[e][c].y), o[i][c][0]);
              o[i][c][1] = fma_pair(make_float2(p[e], p[e]), make_float2(v[e][c].z, v[e][c].w), o[i][c][1]);
            }
        }
      }
    } else {
      // some row does not see the whole block: what it does not see adds nothing, whatever it holds
      for (int j = 0; j < BN; ++j)
#pragma unroll
        for (int i = 0; i < RM; ++i) {
          const float p = sm.p[ty * RM + i][j];
          if (p != 0.f)
#pragma unroll
            for (int c = 0; c < DC; ++c) {
              const float4 v = *reinterpret_cast<const float4*>(&sm.v[j][4 * tx + 64 * c]);
              o[i][c][0] = fma_pair(make_float2(p, p), make_float2(v.x, v.y), o[i][c][0]);
              o[i][c][1] = fma_pair(make_float2(p, p), make_float2(v.z, v.w), o[i][c][1]);
            }
        }
    }
    __syncwarp();
  }
#pragma unroll
  for (int i = 0; i < RM; ++i) {
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], w);
    const int R = r0 + ty * RM + i;
    if (R >= rows) continue;
    const int row = t.first + R / a.group, head = t.kv_head * a.group + R % a.group;
    const float f = a.splits > 1 ? 1.f : sum[i] == 0.f ? 0.f : 1.f / sum[i];
    const long long at = part_index(a, t.split, row, head);
    float* dst = a.splits > 1 ? a.part + at * D : static_cast<float*>(a.out) + row * a.ldo + (long long)head * D;
#pragma unroll
    for (int c = 0; c < DC; ++c)
      *reinterpret_cast<float4*>(dst + 4 * tx + 64 * c) =
          make_float4(o[i][c][0].x * f, o[i][c][0].y * f, o[i][c][1].x * f, o[i][c][1].y * f);
    if (a.splits > 1 && tx == 0) a.ml[at] = make_float2(mx[i], sum[i]);
  }
}

// joins the pieces: D / 4 lanes a (row, head), or several such groups that share its
// pieces (groups > 1: few outputs of many pieces would else wait out one load after the other)
template <typename T, int D>
__global__ void __launch_bounds__(JOIN_THREADS) join_kernel(const __grid_constant__ AttendArgs a, int groups) {
  constexpr int LANES = D / 4, AT_ONCE = JOIN_THREADS / LANES, BATCH = 4;
  __shared__ float4 os[AT_ONCE][LANES];
  __shared__ float2 mls[AT_ONCE];
  const int slot = threadIdx.x / LANES, lane = threadIdx.x % LANES, d = lane * 4, group = slot % groups;
  const long long i = (long long)blockIdx.x * (AT_ONCE / groups) + slot / groups;
  const int row = (int)(i / a.m.n_head), head = (int)(i % a.m.n_head);
  const int parts = a.splits / a.cluster;
  tc::pdl_wait();
  bool on = row < a.rows;
  if (on && a.m.starts) on = row >= a.m.starts[0] && row < a.m.starts[a.m.n_seq];
  float top = -INFINITY, sum = 0.f;
  float4 o = {};
  if (on)
    for (int s0 = group; s0 < parts; s0 += groups * BATCH) {
      float2 ml[BATCH];
      float4 p[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int s = s0 + j * groups;
        ml[j] = make_float2(-INFINITY, 0.f);
        p[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s < parts) {
          const long long at = part_index(a, s, row, head);
          ml[j] = a.ml[at];
          p[j] = *reinterpret_cast<const float4*>(a.part + at * D + d);
        }
      }
#pragma unroll
      for (int j = 0; j < BATCH; ++j) join(top, sum, o, ml[j], p[j]);
    }
  if (groups > 1) {
    os[slot][lane] = o;
    if (lane == 0) mls[slot] = make_float2(top, sum);
    __syncthreads();
    if (group == 0)
      for (int g = 1; g < groups; ++g) join(top, sum, o, mls[slot + g], os[slot + g][lane]);
    on = on && group == 0;
  }
  if (!on) return;
  store_out(static_cast<T*>(a.out) + row * a.ldo + (long long)head * D + d, o, sum == 0.f ? 0.f : 1.f / sum);
}

// 8-bit pages of every sequence as bf16 pages n * cols + i (i < cols: what max_len tokens fill),
// keys and values: a power of two times a code is exact in bf16.  16 codes a thread.
template <int D>
__global__ void __launch_bounds__(JOIN_THREADS) expand_kernel(const __grid_constant__ evo_memory m, int cols, int max_len, __nv_bfloat16* k,
                                                              __nv_bfloat16* v, int* table) {
  const int page = blockIdx.x, n = page / cols, i = page % cols;
  if (threadIdx.x == 0 && blockIdx.y == 0) table[page] = page;
  if ((long long)i * m.page_tokens >= seq_len(m, n, max_len)) return;
  const long long head_rows = (long long)m.n_kv_head * m.page_tokens, from = seq_page(m, n, i) * head_rows, to = page * head_rows;
  const uint8_t* codes = static_cast<const uint8_t*>(blockIdx.y ? m.v_pages : m.k_pages);
  const uint8_t* scales = blockIdx.y ? m.v_scales : m.k_scales;
  __nv_bfloat16* out = blockIdx.y ? v : k;
  for (int x = threadIdx.x; x < head_rows * (D / 16); x += JOIN_THREADS) {
    const int r = x / (D / 16), d = x % (D / 16) * 16;
    const uint4 c = *reinterpret_cast<const uint4*>(codes + (from + r) * D + d);
    const float f = scale_value(scales[from + r]);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 y = codes4(w[e]);
      const __nv_bfloat162 a = __floats2bfloat162_rn(y.x * f, y.y * f), b = __floats2bfloat162_rn(y.z * f, y.w * f);
      h[2 * e] = *reinterpret_cast<const uint32_t*>(&a);
      h[2 * e + 1] = *reinterpret_cast<const uint32_t*>(&b);
    }
    uint4* dst = reinterpret_cast<uint4*>(out + (to + r) * D + d);
    dst[0] = make_uint4(h[0], h[1], h[2], h[3]);
    dst[1] = make_uint4(h[4], h[5], h[6], h[7]);
  }
}

template <int D, int FORMAT, int RM>
cudaError_t launch_f32_as(const AttendArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  return launch_pieces(attend_kernel<D, FORMAT, RM>, a, THREADS, (int)sizeof(Smem<D, RM>), done, st);
}

template <int D, int RM>
cudaError_t launch_f32(const AttendArgs& a, cudaStream_t st) {
  return a.m.format == EVO_CACHE_E4M3 ? launch_f32_as<D, EVO_CACHE_E4M3, RM>(a, st) : launch_f32_as<D, EVO_CACHE_F32, RM>(a, st);
}

template <typename T, int D>
cudaError_t launch_join(const AttendArgs& a, cudaStream_t st) {
  constexpr int AT_ONCE = JOIN_THREADS / (D / 4);
  const long long outputs = (long long)a.rows * a.m.n_head;
  int groups = 1;                                  // 16 pieces a group, while the GPU has threads to spare
  while (groups < AT_ONCE && groups * 16 < a.splits / a.cluster && outputs * groups < 152 * 8 * AT_ONCE) groups *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = (unsigned)((outputs * groups + AT_ONCE - 1) / AT_ONCE);
  cfg.blockDim = JOIN_THREADS;
  cfg.stream = st;
  cudaLaunchAttribute at[1];                       // the launch overlaps the pieces' end; the kernel waits for it
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, join_kernel<T, D>, a, groups);
}

}  // namespace

AttendPlan plan_attend(const evo_memory& m, int rows, int max_new, int max_len) {
  AttendPlan p;
  const long long all = (long long)max_new * (m.n_head / m.n_kv_head);
  const bool f32 = m.dtype == EVO_DTYPE_F32, few = all <= (f32 ? 16 : 32);
  // Many rows: 8-bit pages are written out as bf16 pages once, so that the tensor cores read them
  // as they lie
  const long long cols = (max_len + m.page_tokens - 1) / m.page_tokens;
  const long long expanded = 4ll * m.n_seq * cols * m.n_kv_head * m.page_tokens * m.head_dim;
  const bool expand = !f32 && m.format == EVO_CACHE_E4M3 && all >= EXPAND_ROWS && expanded <= EXPAND_MOST && cols > 0;
  const bool tiles = !f32 && !few && (m.format == EVO_CACHE_BF16 || expand);
  p.expand = expand ? (int)cols : 0;
  p.kernel = f32 ? (few ? ATTEND_F32_ROWS : ATTEND_F32) : tiles ? ATTEND_TILES : ATTEND_ROWS;
  if (tiles)
    p.tile_rows = 256;
  else if (!f32)
    p.tile_rows = all <= 8 ? 8 : all <= 16 ? 16 : 32;
  else if (few)   // 4 rows a tile while that fills the GPU sooner (3 x 16 rows over 333 keys: 8.3 us against 12.4 with 16)
    p.tile_rows = all == 1 ? 1 : all <= 4 || (long long)m.n_seq * m.n_kv_head < 152 ? 4 : 16;
  else            // 64 rows of 128 leave one block a SM
    p.tile_rows = all <= 32 || m.head_dim == 128 ? 32 : 64;
  p.tiles = (int)((all + p.tile_rows - 1) / p.tile_rows);
  const long long blocks = (long long)m.n_seq * m.n_kv_head * p.tiles;
  p.cluster = 1;
  if (p.kernel == ATTEND_ROWS || p.kernel == ATTEND_F32_ROWS) {
    // Pieces: enough blocks to fill the GPU, and with plenty of work several waves of them, so
    // that sequences of different lengths even out; tiles of 32 rows pay 10 us a wave of further
    // blocks (32 rows of 64 sequences: 99 us in one piece, 104 in two).  Up to 8 pieces of few
    // items are joined by a cluster, without a second kernel (3 x 16 rows over 333 fp32 keys: 8.3
    // us against 10.3); more, or those of many items, by a kernel (a cluster's blocks wait for
    // one another: 64 ragged sequences 147 us against 134).
    const long long most = std::max(1, max_len / (f32 ? 64 : 128));
    const long long target = blocks < 456 || p.tile_rows == 32 ? 456 : 1824;
    const long long want = std::max(1ll, std::min({most, (target + blocks / 2) / blocks, 64ll}));
    p.cluster = blocks < 456 && want <= 8 ? (int)want : 1;
    p.splits = (int)want;
  } else {
    const long long most = std::max(1, max_len / (tiles ? 512 : 64));
    const long long target = tiles ? 152 : 152 * 4;
    p.splits = (int)std::max(1ll, std::min({most, target / blocks, 64ll}));
  }
  const int parts = p.splits / p.cluster;
  p.scratch = parts == 1 ? 0 : (size_t)parts * rows * m.n_head * ((size_t)m.head_dim + 2) * sizeof(float);
  if (expand) p.scratch = (p.scratch + 15) / 16 * 16 + expanded + 4ll * m.n_seq * cols;
  return p;
}

cudaError_t launch_attend(AttendArgs& a, const AttendPlan& p, void* scratch, cudaStream_t st) {
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.cluster = p.cluster;
  const int parts = p.splits / p.cluster;
  a.part = static_cast<float*>(scratch);
  a.ml = reinterpret_cast<float2*>(a.part + (size_t)parts * a.rows * a.m.n_head * a.m.head_dim);
  const bool d64 = a.m.head_dim == 64;
  cudaError_t e = cudaSuccess;
  if (p.expand) {
    const size_t joined = parts == 1 ? 0 : (size_t)parts * a.rows * a.m.n_head * ((size_t)a.m.head_dim + 2) * sizeof(float);
    const size_t values = (size_t)a.m.n_seq * p.expand * a.m.n_kv_head * a.m.page_tokens * a.m.head_dim;
    __nv_bfloat16* k = reinterpret_cast<__nv_bfloat16*>(static_cast<uint8_t*>(scratch) + (joined + 15) / 16 * 16);
    int* table = reinterpret_cast<int*>(k + 2 * values);
    const dim3 grid(a.m.n_seq * p.expand, 2);
    if (d64)
      expand_kernel<64><<<grid, JOIN_THREADS, 0, st>>>(a.m, p.expand, a.max_len, k, k + values, table);
    else
      expand_kernel<128><<<grid, JOIN_THREADS, 0, st>>>(a.m, p.expand, a.max_len, k, k + values, table);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    a.m.format = EVO_CACHE_BF16;
    a.m.k_pages = k;
    a.m.v_pages = k + values;
    a.m.k_scales = a.m.v_scales = nullptr;
    a.m.table = table;
    a.m.max_pages = p.expand;
    a.m.n_pages = a.m.n_seq * p.expand;
  }
  if (p.kernel == ATTEND_F32)
    e = p.tile_rows == 32 ? d64 ? launch_f32<64, 4>(a, st) : launch_f32<128, 4>(a, st)
                          : d64 ? launch_f32<64, 8>(a, st) : launch_f32<128, 8>(a, st);
  else if (p.kernel == ATTEND_F32_ROWS)
    e = launch_attend_f32_rows(a, p.tile_rows, st);
  else if (p.kernel == ATTEND_ROWS)
    e = launch_attend_rows(a, p.tile_rows, st);
  else
    e = launch_attend_tiles(a, st);
  if (e != cudaSuccess || parts == 1) return e;
  if (a.m.dtype == EVO_DTYPE_F32) return d64 ? launch_join<float, 64>(a, st) : launch_join<float, 128>(a, st);
  return d64 ? launch_join<__nv_bfloat16, 64>(a, st) : launch_join<__nv_bfloat16, 128>(a, st);
}

}  // namespace evo
