// Attention over a paged memory for few fp32 rows a key/value head (at most 16):
// fp32 or 8-bit pages, all products in fp32.
//
// DRAM bounds these calls as long as every key and value is read from shared memory
// once: at 16 rows the multiply-adds (128 a cycle and SM) take 1.4 times as long as the
// 16 KB of 32 fp32 keys and values of 64 take to arrive, at 4 rows 0.35.
//
// A block is WARPS warps on one tile of R rows and one piece of the memory; each takes
// every WARPS-th run of 32 keys by itself, brought to its own part of shared memory by
// tiled bulk copies while the SM's other warps compute.
//   scores: a lane a key; its 16-byte chunks meet 8 different banks a phase through the
//           copies' swizzle, the queries are broadcast reads;
//   output: a lane D / 32 dimensions; a value's row is one conflict-free read, the
//           weights, 4 keys at a time, broadcast reads.
// A key's scale multiplies its score, a value's its weight, both in fp32.  Every warp
// keeps its own maximum (lazy: rescaled only when a score passes it by 2^8) and sums,
// joined through shared memory at the end.  Weights of zero are skipped in runs that
// some row does not see whole, so that what a masked token holds reaches no other row.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
#include "evo_mem_ptx.cuh"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int RUN = 32;
constexpr float LAZY = 8.f;

template <int D, bool E4M3, int R>
struct Cfg {
  static constexpr int ROW = D * (E4M3 ? 1 : 4);   // bytes of a key or value
  static constexpr int BOX = ROW < 128 ? ROW : 128;
  static constexpr int TILE = RUN * ROW, STAGE = 2 * TILE;
  static constexpr int STAGES = E4M3 ? 2 : 1;
  static constexpr int WARPS = STAGE > 16384 ? 2 : 4, THREADS = 32 * WARPS;
  static constexpr int JOIN = R * D * 4;
  static constexpr int RING = STAGES * STAGE > JOIN ? STAGES * STAGE : (JOIN + 1023) / 1024 * 1024;   // a warp's bytes
  static constexpr int P = R * RUN * 4;            // a warp's weights
  static constexpr int SCALES = E4M3 ? STAGES * 2 * RUN : 0;
  static constexpr int SMEM = 1024 + WARPS * (RING + P + SCALES) + R * D * 4;
};

template <int D, bool E4M3, int R>
__global__ void __launch_bounds__(Cfg<D, E4M3, R>::THREADS) f32_rows_kernel(const __grid_constant__ AttendArgs a,
                                                                            const __grid_constant__ CUtensorMap kmap,
                                                                            const __grid_constant__ CUtensorMap vmap) {
  using C = Cfg<D, E4M3, R>;
  constexpr int WARPS = C::WARPS, THREADS = C::THREADS, STAGES = C::STAGES, PD = D / 64;   // pairs of dimensions a lane
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t full[WARPS][STAGES];
  __shared__ float2 stat[WARPS][R];                // the warps' maxima and sums
  __shared__ float2 block_ml[R];
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  const uint32_t ring = tc::su32(mem) + warp * C::RING, psm = tc::su32(mem) + WARPS * C::RING + warp * C::P;
  const uint32_t qsm = tc::su32(mem) + WARPS * (C::RING + C::P), ssm = qsm + R * D * 4 + warp * C::SCALES;
  if (tid == 0) fetch_map(&kmap), fetch_map(&vmap);
  const Tile t = tile_of_block(a);
  const int rows = t.count * a.group, r0 = t.tile * R;
  if (r0 >= rows) return;
  const int last = min(r0 + R, rows) - 1;
  const Range first_row = seen_by(a, t, r0 / a.group), last_row = seen_by(a, t, last / a.group);
  const Range all = piece_of(a, t, {first_row.lo, last_row.hi}, RUN);
  const int whole_lo = max(last_row.lo, all.lo), whole_hi = min(first_row.hi, all.hi);
  if (tid == 0) {
    for (int i = 0; i < WARPS * STAGES; ++i) tc::mbar_init1(&full[0][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();

  // copies of a run: box keys each, lane i the i-th
  const int box = min(a.m.page_tokens, RUN), shift = 31 - __clz(a.m.page_tokens), step = WARPS * RUN;
  const int page_rows = a.m.n_kv_head * a.m.page_tokens, head_row = t.kv_head * a.m.page_tokens;
  const auto page_at = [&](int k0) {
    const int kb = k0 + lane * box;
    return lane * box < RUN && kb + box > all.lo && kb < all.hi ? seq_page(a.m, t.n, kb >> shift) : -1;
  };
  const auto issue = [&](int k0, int page, int stage) {
    const uint32_t bar = tc::su32(&full[warp][stage]);
    const int copies = __popc(__ballot_sync(0xffffffffu, page >= 0));
    if (lane == 0) tc::mbar_expect_tx(&full[warp][stage], copies * box * (2 * C::ROW + (E4M3 ? 2 : 0)));
    __syncwarp();
    if (page >= 0) {
      const int at = page * page_rows + head_row + ((k0 + lane * box) & (a.m.page_tokens - 1));
      const uint32_t dst = ring + stage * C::STAGE + lane * box * C::BOX;
#pragma unroll
      for (int x = 0; x < C::ROW / C::BOX; ++x) {
        tile_load(dst + x * RUN * C::BOX, &kmap, x * 32, at, bar);
        tile_load(dst + C::TILE + x * RUN * C::BOX, &vmap, x * 32, at, bar);
      }
      if constexpr (E4M3) {
        bulk_load(ssm + stage * 2 * RUN + lane * box, a.m.k_scales + at, box, bar);
        bulk_load(ssm + stage * 2 * RUN + RUN + lane * box, a.m.v_scales + at, box, bar);
      }
    }
  };
  int k0 = all.lo / RUN * RUN + warp * RUN;
#pragma unroll
  for (int i = 0; i < STAGES; ++i)
    if (k0 + i * step < all.hi) issue(k0 + i * step, page_at(k0 + i * step), i);
  int ahead = page_at(k0 + STAGES * step);

  for (int i = tid; i < R * D / 4; i += THREADS) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, q = r0 + r;
    float4 x = {};
    if (q < rows)
      x = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + (long long)(t.first + q / a.group) * a.ldq +
                                           (long long)(t.kv_head * a.group + q % a.group) * D + d);
    sts_f4(qsm + (r * D + d) * 4, x);
  }
  __syncthreads();

  float2 o[R][PD];
  float sum[R], top[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    sum[r] = 0.f;
    top[r] = -INFINITY;
#pragma unroll
    for (int i = 0; i < PD; ++i) o[r][i] = make_float2(0.f, 0.f);
  }
  int stage = 0;
  uint32_t phase = 0;
  bool dead = false;
  for (; k0 < all.hi; k0 += step) {
    if (!__all_sync(0xffffffffu, wait_full(tc::su32(&full[warp][stage]), phase))) {
      dead = true;
      break;
    }
    const uint32_t kt = ring + stage * C::STAGE, vt = kt + C::TILE, sc = ssm + stage * 2 * RUN;
    const bool odd = k0 < whole_lo || k0 + RUN > whole_hi;   // some row does not see the whole run
    float2 s2[R];
#pragma unroll
    for (int r = 0; r < R; ++r) s2[r] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int ch = 0; ch < C::ROW / 16; ++ch) {
      float4 k[E4M3 ? 4 : 1];
      if constexpr (E4M3) {
        const uint4 u = lds128(kt + chunk_at<C::ROW, RUN>(lane, ch));
        k[0] = codes4(u.x), k[1] = codes4(u.y), k[2] = codes4(u.z), k[3] = codes4(u.w);
      } else {
        k[0] = lds_f4(kt + chunk_at<C::ROW, RUN>(lane, ch));
      }
#pragma unroll
      for (int e = 0; e < (E4M3 ? 4 : 1); ++e)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float4 q = lds_f4(qsm + (r * D + ch * (E4M3 ? 16 : 4) + 4 * e) * 4);
          s2[r] = fma_pair(make_float2(q.x, q.y), make_float2(k[e].x, k[e].y), s2[r]);
          s2[r] = fma_pair(make_float2(q.z, q.w), make_float2(k[e].z, k[e].w), s2[r]);
        }
    }
    float ks = a.scale_log2, vs = 1.f;
    if constexpr (E4M3) ks *= scale_value(lds8(sc + lane)), vs = scale_value(lds8(sc + RUN + lane));
    float s[R];
    bool raise = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = (s2[r].x + s2[r].y) * ks;
      if (odd) {
        const int q = r0 + r;
        const Range see = q < rows ? seen_by(a, t, q / a.group) : Range{0, 0};
        const int key = k0 + lane;
        if (key < max(see.lo, all.lo) || key >= min(see.hi, all.hi)) s[r] = -INFINITY;
      }
      raise |= s[r] > top[r] + LAZY;
    }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float m = fmaxf(top[r], s[r]);
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
        const float f = exp2f(top[r] - (m == -INFINITY ? 0.f : m));
        top[r] = m;
        sum[r] *= f;
#pragma unroll
        for (int i = 0; i < PD; ++i) o[r][i] = make_float2(o[r][i].x * f, o[r][i].y * f);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float w = exp2f(s[r] - (top[r] == -INFINITY ? 0.f : top[r]));
      sum[r] += w;
      // the value's scale; a masked weight stays zero whatever the scale says
      sts_f1(psm + (r * RUN + lane) * 4, E4M3 ? (odd && w == 0.f ? 0.f : w * vs) : w);
    }
    __syncwarp();
#pragma unroll 2
    for (int j = 0; j < RUN; j += 4) {
      float2 v[4][PD];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = j + e;
        if constexpr (E4M3) {                      // 2 or 4 codes of the row
          const int b = lane * 2 * PD;
          const uint32_t at = vt + chunk_at<C::ROW, RUN>(r, b / 16) + b % 16;
          const float4 x = codes4(PD == 1 ? lds16(at) : lds32(at));
          v[e][0] = make_float2(x.x, x.y);
          if constexpr (PD == 2) v[e][1] = make_float2(x.z, x.w);
        } else if constexpr (PD == 1) {
          v[e][0] = lds_f2(vt + chunk_at<C::ROW, RUN>(r, lane / 2) + 8 * (lane % 2));
        } else {
          const float4 x = lds_f4(vt + chunk_at<C::ROW, RUN>(r, lane));
          v[e][0] = make_float2(x.x, x.y);
          v[e][1] = make_float2(x.z, x.w);
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float4 p4 = lds_f4(psm + (r * RUN + j) * 4);
        const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (odd && p[e] == 0.f) continue;        // the same for the whole warp
#pragma unroll
          for (int i = 0; i < PD; ++i) o[r][i] = fma_pair(make_float2(p[e], p[e]), v[e][i], o[r][i]);
        }
      }
    }
    __syncwarp();                                  // every lane has read the stage and the weights
    if (k0 + STAGES * step < all.hi) {
      issue(k0 + STAGES * step, ahead, stage);
      ahead = page_at(k0 + (STAGES + 1) * step);
    }
    if (++stage == STAGES) stage = 0, phase ^= 1;
  }
  if (__syncthreads_or(dead)) settle(a.m.status);  // a copy did not arrive: nothing more was asked for

  // the warps' sums, each in its own part of the ring
  float* const mine = reinterpret_cast<float*>(mem + warp * C::RING);
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], w);
#pragma unroll
    for (int i = 0; i < PD; ++i) reinterpret_cast<float2*>(mine + r * D)[lane * PD + i] = o[r][i];
    if (lane == 0) stat[warp][r] = make_float2(top[r], sum[r]);
  }
  __syncthreads();
  for (int i = tid; i < R * D / 4; i += THREADS) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, q = r0 + r;
    if (q >= rows) break;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) m = fmaxf(m, stat[w][r].x);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    float4 x = {};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float2 ml = stat[w][r];
      const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(mem + w * C::RING) + r * D + d);
      const float f = exp2f(ml.x - ref);
      l = fmaf(ml.y, f, l);
      x = make_float4(fmaf(y.x, f, x.x), fmaf(y.y, f, x.y), fmaf(y.z, f, x.z), fmaf(y.w, f, x.w));
    }
    if (a.cluster == 1) {
      put_result<float, D>(a, t, q, d, x, m, l);
    } else {                                       // in place of the first warp's
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(mem) + r * D + d) = x;
      if (d == 0) block_ml[r] = make_float2(m, l);
    }
  }
  if (a.cluster > 1) join_cluster<float, D, R, THREADS>(a, t, reinterpret_cast<const float*>(mem), D, block_ml, r0, rows);
}

template <int D, bool E4M3, int R>
cudaError_t launch_as(const AttendArgs& a, cudaStream_t st) {
  using C = Cfg<D, E4M3, R>;
  CUtensorMap km, vm;
  const int box = std::min(a.m.page_tokens, RUN);
  if (!page_map(&km, a.m, a.m.k_pages, box) || !page_map(&vm, a.m, a.m.v_pages, box)) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  return launch_pieces(f32_rows_kernel<D, E4M3, R>, a, C::THREADS, C::SMEM, done, st, km, vm);
}

template <int R>
cudaError_t launch_rows(const AttendArgs& a, cudaStream_t st) {
  const bool e = a.m.format == EVO_CACHE_E4M3;
  if (a.m.head_dim == 64) return e ? launch_as<64, true, R>(a, st) : launch_as<64, false, R>(a, st);
  return e ? launch_as<128, true, R>(a, st) : launch_as<128, false, R>(a, st);
}

}  // namespace

cudaError_t launch_attend_f32_rows(const AttendArgs& a, int tile_rows, cudaStream_t st) {
  return tile_rows == 1 ? launch_rows<1>(a, st) : tile_rows == 4 ? launch_rows<4>(a, st) : launch_rows<16>(a, st);
}

}  // namespace evo
