// Latent memory: the append of new tokens, the attention of fp32 rows over the latents and
// the choice among the attention kernels.
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
// Attention of fp32 rows: a warp has 4 rows, and all of its lanes a share of the dimensions: 4 in each
// 128 of the latent and 2 of the key part.  The tokens of a stage (16, contiguous in their page) arrive
// by one bulk copy from a warp of its own, STAGES - 1 ahead.  The warp takes 4 of them at a time: 16 sums
// over the lanes by a transposing reduction, the 16 weights a lane pair each, and these once more to
// all lanes, which add them times their share of the latents.  A block is KW warps that share the
// tokens of a stage times RW that share the rows.
//
// The running maximum is lazy: sums are rescaled only when a score passes the row's reference by 2^8.
// A masked weight is none (not zero): what a token holds that a row does not see never meets its sums.
#include <algorithm>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
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

// ---------------------------------------------------------------- attention

constexpr int STAGE = 16;                          // tokens of a stage: a page holds whole ones
constexpr int R = 4;                               // rows a warp
constexpr int AT_ONCE = 4;                         // tokens that a warp takes at once
constexpr float LAZY = 8.f;                        // log2 of how far a weight may pass 1
constexpr float MASKED = -1.f;                     // in place of the weight of a token that a row does not see

template <int RANK, int KW, int RW>
struct Cfg {
  static constexpr int THREADS = 32 * (KW * RW + 1), ROWS = R * RW;
  static constexpr int ROW = (RANK + LATENT_ROPE) * 4, BYTES = STAGE * ROW;
  static constexpr int LD = RANK + 4;
  static constexpr int JOIN = KW * ROWS * LD * 4;
  static constexpr int STAGES = 108 * 1024 / BYTES > 8 ? 8 : 108 * 1024 / BYTES;
  static constexpr int SMEM = STAGES * BYTES > JOIN ? STAGES * BYTES : JOIN;
};

template <int RANK, int KW, int RW>
__global__ void __launch_bounds__(Cfg<RANK, KW, RW>::THREADS) latent_rows_kernel(const __grid_constant__ AttendArgs a) {
  using C = Cfg<RANK, KW, RW>;
  constexpr int N4 = RANK / 128, PAIRS = 2 * N4 + 1;         // float2 of a lane: its share of the latent, then of the key part
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ __align__(8) uint64_t full[8], empty[8];
  __shared__ float2 stat[KW][C::ROWS], block_ml[C::ROWS];
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const Tile t = tile_of_block(a);
  const int rows = t.count * a.group, r0 = t.tile * C::ROWS;
  if (r0 >= rows) return;
  const int last = min(r0 + C::ROWS, rows) - 1;
  const Range first_row = seen_by(a, t, r0 / a.group), last_row = seen_by(a, t, last / a.group);
  const Range all = piece_of(a, t, {first_row.lo, last_row.hi}, STAGE);
  // tokens that every row of the tile sees, of this piece
  const int whole_lo = max(last_row.lo, all.lo), whole_hi = min(first_row.hi, all.hi);
  const int from = all.lo / STAGE * STAGE, n = max(0, (all.hi - from + STAGE - 1) / STAGE);
  if (tid == 0) {
    for (int i = 0; i < C::STAGES; ++i) tc::mbar_init1(&full[i], 1), tc::mbar_init1(&empty[i], KW * RW);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  bool ok = true;
  const int kw = warp % KW, rw = warp / KW;
  float2 o[R][2 * N4];
  float sum = 0.f, mine_top = -INFINITY;             // sum, mine_top: of the row whose weights this lane makes
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < 2 * N4; ++i) o[r][i] = make_float2(0.f, 0.f);
  // after the reduction lane l has value (l / 2) of [token][row]: token l / 8, row l / 2 % 4
  const int my_key = lane / 8, my_row = lane / 2 % R;
  if (warp == KW * RW) {
    // ---------------------------------------------------------- copies: pages of 32 stages are looked up at once
    const int shift = 31 - __clz(a.m.page_tokens);
    for (int i0 = 0; i0 < n && ok; i0 += 32) {
      const int key = from + (i0 + lane) * STAGE;
      const int page = i0 + lane < n ? seq_page(a.m, t.n, key >> shift) : 0;
      for (int j = 0; j < min(32, n - i0) && ok; ++j) {
        const int i = i0 + j, slot = i % C::STAGES, use = i / C::STAGES;
        const long long at = (long long)__shfl_sync(0xffffffffu, page, j) * a.m.page_tokens + ((from + i * STAGE) & (a.m.page_tokens - 1));
        if (use > 0) ok = __all_sync(0xffffffffu, wait_full(tc::su32(&empty[slot]), (use - 1) & 1));
        if (ok && lane == 0) {
          tc::mbar_expect_tx(&full[slot], C::BYTES);
          bulk_load(tc::su32(ring + slot * C::BYTES), static_cast<const uint8_t*>(a.m.k_pages) + at * C::ROW, C::BYTES,
                    tc::su32(&full[slot]));
        }
        __syncwarp();
      }
    }
  } else {
    float2 q[R][PAIRS];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int Q = r0 + R * rw + r;
      const float* src = static_cast<const float*>(a.q) + (long long)(t.first + Q / a.group) * a.ldq + (long long)(Q % a.group) * (RANK + LATENT_ROPE);
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        const int d = i < 2 * N4 ? 128 * (i / 2) + 4 * lane + 2 * (i % 2) : RANK + 2 * lane;
        q[r][i] = Q < rows ? *reinterpret_cast<const float2*>(src + d) : make_float2(0.f, 0.f);
      }
    }
    const float f = a.scale_log2;
    for (int i = 0; i < n; ++i) {
      const int slot = i % C::STAGES;
      ok = __all_sync(0xffffffffu, wait_full(tc::su32(&full[slot]), (i / C::STAGES) & 1));
      if (!ok) break;
      const int k0 = from + i * STAGE;
      const bool odd = k0 < whole_lo || k0 + STAGE > whole_hi;
      const uint32_t base = tc::su32(ring + slot * C::BYTES);
      for (int g = kw; g < STAGE / AT_ONCE; g += KW) {
        float2 x[AT_ONCE][PAIRS];
        float v[AT_ONCE * R];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
          const uint32_t p = base + (g * AT_ONCE + k) * C::ROW;
#pragma unroll
          for (int j = 0; j < N4; ++j) {
            const float4 y = lds_f4(p + (128 * j + 4 * lane) * 4);
            x[k][2 * j] = make_float2(y.x, y.y), x[k][2 * j + 1] = make_float2(y.z, y.w);
          }
          x[k][2 * N4] = lds_f2(p + (RANK + 2 * lane) * 4);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            float2 s = mul_pair(x[k][0], q[r][0]);
#pragma unroll
            for (int j = 1; j < PAIRS; ++j) s = fma_pair(x[k][j], q[r][j], s);
            v[k * R + r] = s.x + s.y;
          }
        }
        // sums over the lanes: each step halves the values a lane holds
#pragma unroll
        for (int h = 8, m = 16; h > 0; h >>= 1, m >>= 1) {
          const bool up = lane & m;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < h) {
              const float keep = up ? v[j + h] : v[j], give = up ? v[j] : v[j + h];
              v[j] = keep + __shfl_xor_sync(0xffffffffu, give, m);
            }
        }
        float s = (v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1)) * f;
        bool masked = false;
        if (odd) {
          const int Q = r0 + R * rw + my_row, key = k0 + g * AT_ONCE + my_key;
          const Range see = Q < rows ? seen_by(a, t, Q / a.group) : Range{0, 0};
          masked = key < max(see.lo, all.lo) || key >= min(see.hi, all.hi);
          if (masked) s = -INFINITY;
        }
        if (__any_sync(0xffffffffu, s > mine_top + LAZY || (mine_top == -INFINITY && s > -INFINITY))) {
          float m = s;
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
          m = fmaxf(m, mine_top);
          const float down = m == -INFINITY ? 1.f : ex2_approx(mine_top - m);
          mine_top = m;
          sum *= down;
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float d = __shfl_sync(0xffffffffu, down, 2 * r);
#pragma unroll
            for (int j = 0; j < 2 * N4; ++j) o[r][j] = mul_pair(o[r][j], make_float2(d, d));
          }
        }
        float p = ex2_approx(s - (mine_top == -INFINITY ? 0.f : mine_top));
        if (masked) p = MASKED;
        else sum += p;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float w = __shfl_sync(0xffffffffu, p, 8 * k + 2 * r);
            if (odd && w == MASKED) continue;
#pragma unroll
            for (int j = 0; j < 2 * N4; ++j) o[r][j] = fma_pair(x[k][j], make_float2(w, w), o[r][j]);
          }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive1(&empty[slot]);
    }
#pragma unroll
    for (int m = 8; m < 32; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
  }
  if (__syncthreads_or(!ok)) settle(a.m.status);             // a copy did not arrive
  float* const sums = reinterpret_cast<float*>(ring);        // [KW][ROWS][LD]
  if (warp < KW * RW) {
    if (lane < 2 * R && lane % 2 == 0) stat[kw][R * rw + lane / 2] = make_float2(mine_top, sum);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < N4; ++j)
        *reinterpret_cast<float4*>(sums + (kw * C::ROWS + R * rw + r) * C::LD + 128 * j + 4 * lane) =
            make_float4(o[r][2 * j].x, o[r][2 * j].y, o[r][2 * j + 1].x, o[r][2 * j + 1].y);
  }
  __syncthreads();
  for (int i = tid; i < C::ROWS * RANK / 4; i += C::THREADS) {
    const int r = i / (RANK / 4), d = i % (RANK / 4) * 4;
    if (r0 + r >= rows) break;
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) m = fmaxf(m, stat[w][r].x);
    const float ref = m == -INFINITY ? 0.f : m;
    float4 x = {};
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const float2 ml = stat[w][r];
      const float4 y = *reinterpret_cast<const float4*>(sums + (w * C::ROWS + r) * C::LD + d);
      const float fw = ex2_approx(ml.x - ref);
      l = fmaf(ml.y, fw, l);
      x = make_float4(fmaf(y.x, fw, x.x), fmaf(y.y, fw, x.y), fmaf(y.z, fw, x.z), fmaf(y.w, fw, x.w));
    }
    if (a.cluster == 1) {
      put_result<float, RANK>(a, t, r0 + r, d, x, m, l);
    } else {                                                 // in place of the first warp's
      *reinterpret_cast<float4*>(sums + r * C::LD + d) = x;
      if (d == 0) block_ml[r] = make_float2(m, l);
    }
  }
  if (a.cluster > 1) join_cluster<float, RANK, C::ROWS, C::THREADS>(a, t, sums, C::LD, block_ml, r0, rows);
}

template <int RANK, int KW, int RW>
cudaError_t launch_rows_as(const AttendArgs& a, cudaStream_t st) {
  using C = Cfg<RANK, KW, RW>;
  static std::atomic<uint64_t> done{0};
  return launch_pieces(latent_rows_kernel<RANK, KW, RW>, a, C::THREADS, C::SMEM, done, st);
}
template <int RANK>
cudaError_t launch_rows_of(const AttendArgs& a, int tile_rows, cudaStream_t st) {
  return tile_rows == 4    ? launch_rows_as<RANK, 4, 1>(a, st)
         : tile_rows == 8  ? launch_rows_as<RANK, 4, 2>(a, st)
         : tile_rows == 16 ? launch_rows_as<RANK, 2, 4>(a, st)
                           : launch_rows_as<RANK, 1, 8>(a, st);
}
cudaError_t launch_rows(const AttendArgs& a, int tile_rows, cudaStream_t st) {
  return a.m.head_dim == 128   ? launch_rows_of<128>(a, tile_rows, st)
         : a.m.head_dim == 256 ? launch_rows_of<256>(a, tile_rows, st)
                               : launch_rows_of<512>(a, tile_rows, st);
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
  p.cluster = 1;
  if (m.dtype != EVO_DTYPE_F32) {
    plan_latent_tiles(p, m, all, keys);
    return p;
  }
  p.tile_rows = all <= 4 ? 4 : all <= 8 ? 8 : all <= 16 ? 16 : 32;
  p.tiles = (int)((all + p.tile_rows - 1) / p.tile_rows);
  const long long blocks = (long long)m.n_seq * p.tiles;
  p.splits = (int)std::max(1ll, std::min({(long long)keys / 64, 304 / blocks, 64ll}));
  p.scratch = p.splits == 1 ? 0 : (size_t)p.splits * rows * m.n_head * ((size_t)m.head_dim + 2) * sizeof(float);
  return p;
}

cudaError_t launch_latent_attend(AttendArgs& a, const LatentPlan& p, void* scratch, cudaStream_t st) {
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.cluster = p.cluster;
  if (a.m.dtype != EVO_DTYPE_F32) return launch_latent_tiles(a, p, scratch, st);
  const int parts = p.splits / p.cluster;
  a.part = static_cast<float*>(scratch);
  a.ml = reinterpret_cast<float2*>(a.part + (size_t)parts * a.rows * a.m.n_head * a.m.head_dim);
  const cudaError_t e = launch_rows(a, p.tile_rows, st);
  return e != cudaSuccess || parts == 1 ? e : launch_join(a, st);
}

}  // namespace evo
