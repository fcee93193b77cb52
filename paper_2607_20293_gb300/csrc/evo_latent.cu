// Latent memory: the append of new tokens and the choice among the attention kernels.
//
// A token is one row of rank + 64 values that all heads share: its latent c, normed, and a
// key part k, rotated by the token's position.  A query has been multiplied by its head's key map:
//   s_j = scale <(q | q'), (c_j | k_j)>,   out = sum_j softmax(s)_j c_j
//
// Append: u = c / sqrt(mean(c^2) + eps) * gain, and the pairs (i, i + 32) of k and of every query's
// last 64 values turned by (position, i); fp32 inside, one rounding.  A warp takes a row's latent
// and key part, or some of its queries: 4 lanes a head, each the 8 values at 8 l and the 8 at 32 + 8 l,
// so that the rotation needs no exchange.
//
// A token's append is a chain of loads (length, table, page), 4 us for 64 of them; long chunks are bound by
// the loads that a warp has on the way: 11,700 rows of 16 heads, rank 512, bf16, 16.6 us, 4.7 TB/s.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_mem_ptx.cuh"
#include "evo_rows.cuh"

namespace evo {
namespace {

// ---------------------------------------------------------------- append

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int HEADS = 8;                           // heads of a row that a warp takes at once
constexpr int BATCH = 2;                           // such groups whose loads are in flight

template <typename T>
__device__ __forceinline__ Raw<T> load8(const T* p) {
  Raw<T> r;
#pragma unroll
  for (int e = 0; e < (int)sizeof(T) / 2; ++e) r.u[e] = reinterpret_cast<const uint4*>(p)[e];
  return r;
}

// 8 + 8 values of a rotated part, columns 8 l and 32 + 8 l
template <typename T>
__device__ __forceinline__ void put_turned(T* dst, const Raw<T>& r0, const Raw<T>& r1, const float2 (&c)[4],
                                           const float2 (&s)[4], bool turn) {
  float2 x[4], y[4];
  values(r0, x);
  values(r1, y);
  if (turn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 u = x[i];
      x[i] = fma_pair(y[i], make_float2(-s[i].x, -s[i].y), mul_pair(u, c[i]));
      y[i] = fma_pair(u, s[i], mul_pair(y[i], c[i]));
    }
  }
  store8(dst, x);
  store8(dst + LATENT_ROPE / 2, y);
}

template <typename T, int RANK>
__global__ void __launch_bounds__(THREADS) latent_append_kernel(const __grid_constant__ LatentAppendArgs a, int parts) {
  constexpr int EACH = RANK > 256 ? 2 : 1;         // groups of 8 values of a latent a lane
  const int lane = threadIdx.x & 31, l = lane & 3;
  const int w = blockIdx.x * WARPS + (threadIdx.x >> 5), row = w / parts, part = w % parts;
  if (row >= a.rows) return;
  const bool mine = a.k && part == parts - 1;
  Raw<T> c[EACH], k0, k1;
  if (mine) {
    const T* src = static_cast<const T*>(a.c) + row * a.ldc;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (lane + 32 * i < RANK / 8) c[i] = load8(src + 8 * (lane + 32 * i));
    const T* kp = static_cast<const T*>(a.k) + row * a.ldk + 8 * l;
    k0 = load8(kp), k1 = load8(kp + LATENT_ROPE / 2);
  }
  const Place p = place_of(a, row);
  if (p.turn < 0) return;
  float2 cs[4] = {}, sn[4] = {};
  const bool turn = a.rotation != nullptr;
  if (turn) {
    const float* r = a.rotation + (long long)p.turn * LATENT_ROPE + 8 * l;
    load_pairs(r, cs);
    load_pairs(r + LATENT_ROPE / 2, sn);
  }
  if (mine) {
    T* dst = static_cast<T*>(a.m.k_pages) + ((long long)p.page * a.m.page_tokens + p.slot) * (RANK + LATENT_ROPE);
    float2 x[EACH][4];
    float2 ss = {};
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      values(c[i], x[i]);
      if (lane + 32 * i < RANK / 8)
#pragma unroll
        for (int e = 0; e < 4; ++e) ss = fma_pair(x[i][e], x[i][e], ss);
    }
    if (a.c_gain) {
      float sum = ss.x + ss.y;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float f = rsqrtf(sum * (1.0f / RANK) + a.eps);
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (lane + 32 * i < RANK / 8) {
          float2 g[4];
          load_pairs(a.c_gain + 8 * (lane + 32 * i), g);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[i][e] = mul_pair(mul_pair(x[i][e], make_float2(f, f)), g[e]);
        }
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (lane + 32 * i < RANK / 8) store8(dst + 8 * (lane + 32 * i), x[i]);
    if (lane < 4) put_turned(dst + RANK + 8 * l, k0, k1, cs, sn, turn);
  }
  if (!a.q) return;
  const T* q = static_cast<const T*>(a.q) + row * a.ldq + 8 * l;
  T* out = static_cast<T*>(a.q_out) + row * a.ldo + 8 * l;
  for (int h0 = part * HEADS; h0 < a.m.n_head; h0 += parts * HEADS * BATCH) {
    Raw<T> r[BATCH][2];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = h0 + i * parts * HEADS + lane / 4;
      if (h < a.m.n_head) r[i][0] = load8(q + h * a.hdq), r[i][1] = load8(q + h * a.hdq + LATENT_ROPE / 2);
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = h0 + i * parts * HEADS + lane / 4;
      if (h < a.m.n_head) put_turned(out + h * a.hdo, r[i][0], r[i][1], cs, sn, turn);
    }
  }
}

template <typename T, int RANK>
cudaError_t launch_append_as(const LatentAppendArgs& a, cudaStream_t st) {
  const int most = std::max(1, a.q ? (a.m.n_head + HEADS - 1) / HEADS : 1);
  // a row's heads over as many warps as keep the GPU's 152 x 32 busy
  const int parts = (int)std::max(1ll, std::min((long long)most, 152ll * 32 / a.rows));
  const long long warps = (long long)a.rows * parts;
  latent_append_kernel<T, RANK><<<(unsigned)((warps + WARPS - 1) / WARPS), THREADS, 0, st>>>(a, parts);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_append_type(const LatentAppendArgs& a, cudaStream_t st) {
  return a.m.head_dim == 128   ? launch_append_as<T, 128>(a, st)
         : a.m.head_dim == 256 ? launch_append_as<T, 256>(a, st)
                               : launch_append_as<T, 512>(a, st);
}

}  // namespace

cudaError_t launch_latent_append(const LatentAppendArgs& a, cudaStream_t st) {
  return a.m.dtype == EVO_DTYPE_F32 ? launch_append_type<float>(a, st) : launch_append_type<__nv_bfloat16>(a, st);
}

LatentPlan plan_latent(const evo_memory& m, int rows, int max_new, int max_len, int causal, int window) {
  LatentPlan p{};
  const long long all = (long long)max_new * m.n_head;
  const int moves = causal ? std::min(max_new, 128 / m.n_head + 1) : 0;
  const int keys = window ? (int)std::min<long long>(max_len, (long long)window + moves) : max_len;
  p.tile_rows = m.dtype == EVO_DTYPE_F32 ? latent_f32_rows(m.head_dim, all, m.n_seq)
                : all <= 16              ? 16
                : all <= 32 || m.head_dim == 512 ? 32
                : all <= 64              ? 64
                                         : 128;
  p.tiles = (int)((all + p.tile_rows - 1) / p.tile_rows);
  // Items go to the blocks whole where that takes little longer, in tiles of 128 tokens, than equal runs, their
  // pieces, the join of these, and the caller's time for its launch and the workspace (5 us).  4 / 60 items of 4 tiles,
  // whole against in runs: 10.3 to 9.2 / 10.8 to 13.1 us (bf16, rank 256, 32 rows), 13.6 to 9.4 / 14.0 to 12.5 (fp32, rank
  // 128); of 12 tiles: 20.9 to 9.6 / 24.0 to 22.9 and 30.8 to 9.9 / 33.6 to 26.3
  constexpr int SMS = 152, MOST_ITEMS = 2048;      // items that a block counts
  const int join = m.dtype == EVO_DTYPE_F32 ? (m.head_dim == 512 ? 1 : m.head_dim == 256 ? 2 : 3) : p.tile_rows == 128 ? 3 : m.head_dim == 512 ? 4 : 5;
  const long long items = (long long)m.n_seq * p.tiles, tiles = std::max(1, (keys + 127) / 128);
  const double whole = (double)((items + SMS - 1) / SMS) * (tiles + 2), even = (double)items * tiles / SMS + 2 + join;
  const bool split = items <= MOST_ITEMS && tiles > 1 && items * (tiles + 3) < INT_MAX && even < whole;
  p.splits = split ? 2 : 1;
  p.blocks = (int)std::min<long long>(SMS, split ? items * tiles : items);
  // sums, and maximum and sum of weights, of two pieces a block; where a block's last item goes on
  p.scratch = split ? (size_t)p.blocks * (2 * p.tile_rows * ((size_t)m.head_dim + 2) * sizeof(float) + sizeof(int4)) : 0;
  return p;
}

cudaError_t launch_latent_attend(AttendArgs& a, const LatentPlan& p, void* scratch, cudaStream_t st) {
  a.tiles = p.tiles;
  a.part = static_cast<float*>(scratch);
  a.ml = reinterpret_cast<float2*>(a.part + (size_t)2 * p.blocks * p.tile_rows * a.m.head_dim);
  return a.m.dtype == EVO_DTYPE_F32 ? launch_latent_f32(a, p, st) : p.tile_rows == 128 ? launch_latent_wide(a, p, st) : launch_latent_tiles(a, p, st);
}

}  // namespace evo
