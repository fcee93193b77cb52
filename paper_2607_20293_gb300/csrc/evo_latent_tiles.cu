// Attention of bf16 rows over a latent memory, on tcgen05.
//
// All heads share a token's vector, so even one token's attention is a product of n_head rows, and a
// memory's bytes are used 2 n_head times each; keys and values are the same bytes, which are brought to
// shared memory once.  Both products have the memory as their first operand (128 tokens or 128
// dimensions are the 128 rows of an instruction) and the queries' rows as the second, so that 16 rows
// cost an eighth of what 128 do, and the output of 512 dimensions takes 4 N columns of tensor memory:
//   S^T = X Q^T   tokens x rows, X = (c | k) as it lies in its page
//   O^T += C^T P^T  dimensions x rows, C^T by the transposing form of the same tiles
// An item is N = 16 to 64 rows (tokens of a chunk times heads) of one sequence, and is taken 128
// tokens of memory at a time. The last warp brings these by tiled bulk copies into a ring of slots of 128
// dimensions (and one of key parts); the one before it issues the products; the others are the
// softmax: a thread has a token (its lane of tensor memory) and 8 to 32 of the rows, and writes the weights
// P^T, which are summed over the lanes only at the end of an item.
//
// Blocks stay resident and take equal runs of the tiles (evo_latent.cuh); the copies run ahead into the
// next item while the softmax still writes this one's output.
//
// The memory's bytes bound it: 64 single tokens of 16 heads over up to 8,192 tokens of rank 512 take 85 us, 5.2 TB/s (77 %
// of a copy's rate; the first tiles, the pieces and their join are the rest), 32 tokens of 64 heads over rank 256 39 us, 3.2 TB/s:
// with 64 rows two tiles fit the ring, and a tile's slots come free only behind its softmax.
//
// The running maximum is lazy: a row's reference is raised only when a score passes it by 2^8, so that
// the common tile has one vote in place of reductions over the lanes.  The reference m is subtracted from the
// product, and the difference multiplied by the factor: equal scores have equal weights at any size.
// Weights are rounded to bf16 for their product, 2^-8 of each at most.
//
// Masks are looked at only in tiles that some row does not see whole.  There, tokens outside the item's
// range are set to zero in shared memory; so is one with a value that is not finite (0 * NaN would reach
// rows that do not see it), whose score is then NaN for the rows that see it.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_latent.cuh"

namespace evo {
namespace {

template <int RANK, int N>
struct Cfg {
  static constexpr int PER = RANK / 128;           // slots of a tile
  static constexpr int Q = N * (RANK + LATENT_ROPE) * 2, P = BK * N * 2;
  static constexpr int FREE = 227 * 1024 - 1024 - 2048 - Q - P;   // alignment and static shared memory left out
  // tiles of 128 dimensions are one slot and one key part each; else one or two key parts, the rest slots
  static constexpr int EVEN = FREE / (SLOT + HALF), MOST = (FREE - HALF) / SLOT;
  static constexpr int SLOTS = PER == 1 ? EVEN : MOST > 6 ? 6 : MOST;
  static constexpr int PARTS = PER == 1 ? EVEN : FREE - SLOTS * SLOT >= 2 * HALF ? 2 : 1;
  static constexpr int SMEM = 1024 + Q + P + SLOTS * SLOT + PARTS * HALF;
  static constexpr int S_COL = PER * N, COLS = S_COL + 2 * N;     // tensor memory: O, then two buffers of S
  static constexpr int ALLOC = COLS <= 64 ? 64 : COLS <= 128 ? 128 : COLS <= 256 ? 256 : 512;
  static constexpr int WARPS = N >= 64 ? 16 : 8, SOFTMAX = 32 * WARPS, THREADS = SOFTMAX + 64;
  static constexpr int WEIGHTS16 = 16 * (N >= 64 ? 128 : 2 * N);  // bytes of 16 tokens' weights
  static constexpr int HC = N / (WARPS / 4);       // rows of a softmax thread
  static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(BK >> 4) << 24);
  static constexpr uint32_t IDESC_O = IDESC | (1u << 15) | (1u << 16);   // contiguous indexes: dimensions, rows
  static_assert(SLOTS >= PER && SLOTS <= 6 && COLS <= 512, "");
};

template <int N>
struct Shared : Roles {
  __align__(16) float ref[N];                      // what is subtracted from a row's scores
  int top[N];                                      // a new maximum (ordered as integers), then the factor of what was summed
  long long to[N];                                 // where a row's output begins
};

// the weights: min(N, 64) rows by 8 tokens, swizzled by that width
template <int N>
__device__ __forceinline__ uint64_t weight_desc(uint32_t saddr) {
  if constexpr (N >= 64) return latent_desc(saddr);
  return (uint64_t)((saddr & 0x3ffffu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(N * 16 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)(N == 32 ? 4 : 6) << 61;
}
// byte offset of 8 weights of token k, rows 8 i ..
template <int N>
__device__ __forceinline__ int weight_at(int k, int i) {
  if constexpr (N >= 64) return (i / 8) * HALF + k * 128 + ((i % 8 ^ (k & 7)) << 4);
  if constexpr (N == 32) return k * 64 + ((i ^ ((k >> 1) & 3)) << 4);
  return k * 32 + ((i ^ ((k >> 2) & 1)) << 4);
}
template <int RANK, int N>
__global__ void __launch_bounds__(Cfg<RANK, N>::THREADS, 1)
    latent_tiles_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map,
                        const __grid_constant__ CUtensorMap queries, const __grid_constant__ Run run) {
  using C = Cfg<RANK, N>;
  constexpr int PER = C::PER, HC = C::HC, SLOTS = C::SLOTS, PARTS = C::PARTS, SOFTMAX = C::SOFTMAX, THREADS = C::THREADS;
  extern __shared__ uint8_t raw[];
  __shared__ Shared<N> sh;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  uint8_t* const weights = mem + C::Q;
  uint8_t* const ring = weights + C::P;
  uint8_t* const parts = ring + SLOTS * SLOT;
  if (tid == 0) fetch_map(&map), fetch_map(&queries);
  __syncwarp();                                    // a whole warp's instruction, behind one lane's prefetch
  if (warp == 0) tc::tmem_alloc(&sh.tmem, C::ALLOC);
  if (tid == 32) {
    for (int i = 0; i < SLOTS; ++i) tc::mbar_init1(&sh.full[i], 1), tc::mbar_init1(&sh.empty[i], 1);
    for (int i = 0; i < PARTS; ++i) tc::mbar_init1(&sh.part_full[i], 1), tc::mbar_init1(&sh.part_empty[i], 1);
    tc::mbar_init1(&sh.s_full[0], 1), tc::mbar_init1(&sh.s_full[1], 1);
    tc::mbar_init1(&sh.p_full[0], C::WARPS);          // a warp each
    tc::mbar_init1(&sh.q_full, run.flat ? 1 : C::WARPS);
    tc::mbar_init1(&sh.o_full, 1);
    sh.dead = 0;
    sh.item = run.split ? run.items : blockIdx.x;
    sh.skip = 0;
    sh.tiles = run.split ? 0 : INT_MAX;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < N) sh.ref[tid] = NONE;
  tc::pdl_wait();                                  // what earlier kernels wrote is there
  if (run.split) tc::pdl_trigger();                // the join may take the places that become free, and waits there
  const Share share = count_tiles<N, THREADS>(a, run, sh);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;
  Walk<N> walk(a, run, sh);
  int g = 0;                                       // tiles so far

  if (warp == C::WARPS + 1) {
    // ------------------------------------------------------------ copies
    bring_tiles<RANK, SLOTS, PARTS>(a, walk, map, ring, parts, sh);
  } else if (warp == C::WARPS) {
    // ------------------------------------------------------------ products
    // Uniform over the warp and known to the compiler to be (a shuffle's result is), one elected lane issuing:
    // descriptors then stay in uniform registers, and an instruction costs an addition or two.
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t rows_desc = tc::sw128_desc(0), turned_desc = latent_desc(0), w_desc = weight_desc<N>(0);
    const uint32_t hi = (uint32_t)(rows_desc >> 32), whi = (uint32_t)(w_desc >> 32), at = tc::su32(ring) >> 4;
    const uint32_t xr = (uint32_t)rows_desc + at, xt = (uint32_t)turned_desc + at, q = (uint32_t)rows_desc + (tc::su32(mem) >> 4),
                   kp = (uint32_t)rows_desc + (tc::su32(parts) >> 4), w = (uint32_t)w_desc + (tc::su32(weights) >> 4);
    const uint32_t full = tc::su32(sh.full), empty = tc::su32(sh.empty), part_full = tc::su32(sh.part_full),
                   part_empty = tc::su32(sh.part_empty), dead_word = tc::su32(&sh.dead);
    const uint32_t s_full = tc::su32(sh.s_full), p_full = tc::su32(sh.p_full), o_full = tc::su32(&sh.o_full);
    uint32_t s_slot = 0, s_phase = 0, s_part = 0, s_part_phase = 0, o_slot = 0;
    const auto wait = [&](uint32_t bar, uint32_t parity) {
      if (!tc::mbar_test(bar, parity)) wait_slow(bar, parity, dead_word);
    };
    const auto scores = [&](uint32_t i) {
      const uint32_t d = tm + C::S_COL + (i & 1) * N;
#pragma unroll
      for (uint32_t j = 0; j < PER; ++j) {
        wait(full + 8 * s_slot, s_phase);
        tc::tc_fence_after();
        const uint32_t x = xr + s_slot * (SLOT >> 4);
        if (tc::elect_one())
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k)
            tc::mma_f16(d, desc64(x + (k / 4) * (HALF >> 4) + (k % 4) * 2, hi), desc64(q + (2 * j + k / 4) * (N * 128 >> 4) + (k % 4) * 2, hi),
                        C::IDESC, j | k);
        if (++s_slot == SLOTS) s_slot = 0, s_phase ^= 1;
      }
      wait(part_full + 8 * s_part, s_part_phase);
      tc::tc_fence_after();
      const uint32_t x = kp + s_part * (HALF >> 4);
      if (tc::elect_one()) {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
          tc::mma_f16(d, desc64(x + k * 2, hi), desc64(q + 2 * PER * (N * 128 >> 4) + k * 2, hi), C::IDESC, 1);
        commit(s_full + 8 * (i & 1));
        commit(part_empty + 8 * s_part);
      }
      if (++s_part == PARTS) s_part = 0, s_part_phase ^= 1;
    };
    const auto output = [&](uint32_t accumulate) {
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const uint32_t x = xt + o_slot * (SLOT >> 4);
        if (tc::elect_one()) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            tc::mma_f16(tm + j * N, desc64(x + k * (2048 >> 4), hi), desc64(w + k * (C::WEIGHTS16 >> 4), whi), C::IDESC_O, k ? 1 : accumulate);
          commit(empty + 8 * o_slot);
          if (j == PER - 1) commit(o_full);
        }
        if (++o_slot == SLOTS) o_slot = 0;
      }
    };
    // The next tile's scores go before this one's output where its tokens are there (its key parts come last) before
    // the weights are, and else behind it: the output frees the slots that further tokens wait for
    bool dead = false;
    while (!dead && walk.next()) {
      if (walk.n == 0) continue;
      const int n = __shfl_sync(0xffffffffu, walk.n, 0);
      wait(tc::su32(&sh.q_full), (walk.filled - 1) & 1);
      tc::tc_fence_after();
      scores(g);
      for (int i = 0; i < n; ++i, ++g) {
        bool early = i + 1 >= n;
        for (const long long since = clock64(); !early && !test(p_full, g & 1);) {
          early = test(part_full + 8 * s_part, s_part_phase);
          if (early) scores(g + 1);
          else if (clock64() - since > WAIT_CYCLES_DEFAULT) break;   // (the wait below reports it)
        }
        wait(p_full, g & 1);
        tc::tc_fence_after();
        dead = __any_sync(0xffffffffu, tc::block_dead(dead_word));
        if (dead) break;
        output(i);
        if (!early) scores(g + 1);
      }
    }
  } else {
    // ------------------------------------------------------------ softmax: a token and rows c0 .. c0 + HC - 1 a thread
    // A wait that is in vain ends no turn: the barriers of the softmax want all of its warps.
    const int k = tid % BK, part = warp / 4, c0 = part * HC;
    const uint32_t lanes = (uint32_t)(32 * (warp % 4)) << 16;
    const float f = factor_of(a), far = far_of(f), sign = sign_of(a);
    // the first warp looks the next item up for all of them
    bool shares = false;
    const auto look_up = [&](Segment& q) {
      bar_softmax<SOFTMAX>();                        // nobody is at the item before any more
      if (warp == 0) fill_segment(a, run, share, walk, q, shares);
      bar_softmax<SOFTMAX>();
    };
    float sum[HC];
    look_up(sh.seg[0]);
    if (sh.seg[0].more && sh.seg[0].n > 0) bring_queries<RANK, N, SOFTMAX>(a, run, queries, sh.seg[0].x, mem, sh);
    for (int s = 0; sh.seg[s].more; s ^= 1) {
      const Segment& q = sh.seg[s];
      const Segment& after = sh.seg[s ^ 1];
      if (q.n > 0) queries_there(run, sh);
      look_up(sh.seg[s ^ 1]);
      const Item& x = q.x;
      const Tile& t = x.t;
      const int n = q.n, key0 = q.key0;
#pragma unroll
      for (int j = 0; j < HC; ++j) sum[j] = 0.f;
      for (int i = 0; i < n; ++i, ++g) {
        wait_for(&sh.s_full[g & 1], (g >> 1) & 1, &sh.dead);
        __syncwarp();
        tc::tc_fence_after();
        float v[HC];
        const uint32_t scores = tmem + C::S_COL + (g & 1) * N + c0 + lanes;
        tmem_load(scores, v);
        if (sign != 1.f)
#pragma unroll
          for (int j = 0; j < HC; ++j) v[j] *= sign;
        const int key = key0 + i * BK + k;
        if (key0 + i * BK < x.last_row.lo || key0 + (i + 1) * BK > x.first_row.hi) {
          const bool alike = q.alike, out = key < x.all.lo || key >= x.all.hi;
          // this thread's share of the token's latent: 64 of each 128 dimensions of every second slot, or of all
          constexpr int SHARES = C::WARPS / 8;
          bool bad = false;
          for (int j = part / 2 % SHARES; j < PER; j += SHARES) {
            const int index = g * PER + j, slot = index % SLOTS;
            wait_for(&sh.full[slot], (index / SLOTS) & 1, &sh.dead);
            uint4* p = reinterpret_cast<uint4*>(ring + slot * SLOT + part % 2 * HALF + k * 128);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (out) {
                p[e ^ (k & 7)] = make_uint4(0, 0, 0, 0);
              } else if (!alike) {
                const uint4 u = p[e ^ (k & 7)];
                const uint32_t y[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int z = 0; z < 4; ++z) bad |= (y[z] & 0x7f80u) == 0x7f80u || (y[z] & 0x7f800000u) == 0x7f800000u;
              }
            }
          }
          if (alike) {
#pragma unroll
            for (int j = 0; j < HC; ++j) v[j] = out ? -INFINITY : v[j];
          } else {
            if (tid < 4) sh.bad[tid] = 0;
            bar_softmax<SOFTMAX>();
            if (bad) atomicOr(&sh.bad[k / 32], 1u << (k % 32));
            bar_softmax<SOFTMAX>();
            bad = sh.bad[k / 32] >> (k % 32) & 1;
            if (bad)
              for (int j = part / 2 % SHARES; j < PER; j += SHARES) {
                uint4* p = reinterpret_cast<uint4*>(ring + (g * PER + j) % SLOTS * SLOT + part % 2 * HALF + k * 128);
                for (int e = 0; e < 8; ++e) p[e] = make_uint4(0, 0, 0, 0);
              }
#pragma unroll
            for (int j = 0; j < HC; ++j) {
              const Range see = seen_by(a, t, min(x.r0 + c0 + j, x.last) / a.group);
              if (bad) v[j] = __builtin_nanf("");
              if (out || key < see.lo || key >= see.hi) v[j] = -INFINITY;
            }
          }
          tc::fence_async_smem();
        }
        if (sign != 1.f || key0 + i * BK < x.last_row.lo || key0 + (i + 1) * BK > x.first_row.hi) {
          for (int j = 0; j < HC; j += 8) tmem_store8(scores + j, v + j);   // where a new reference looks for them
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        }
        // scores less their references; a row that has seen nothing is far below any score
        const auto less = [&] {
          float top = -INFINITY;
#pragma unroll
          for (int j = 0; j < HC; j += 4) {
            const float4 r = *reinterpret_cast<const float4*>(&sh.ref[c0 + j]);
            const float2 d = add2(make_float2(v[j], v[j + 1]), make_float2(-r.x, -r.y));
            const float2 e = add2(make_float2(v[j + 2], v[j + 3]), make_float2(-r.z, -r.w));
            v[j] = d.x, v[j + 1] = d.y, v[j + 2] = e.x, v[j + 3] = e.y;
            top = fmaxf(fmaxf(top, fmaxf(d.x, d.y)), fmaxf(e.x, e.y));
          }
          return top;
        };
        const bool raise = less() > far;
        bool waited = i == 0;
        if (bar_softmax_or<SOFTMAX>(raise)) {
          if (tid < N) sh.top[tid] = ordered(-INFINITY);
          tmem_load(scores, v);
          bar_softmax<SOFTMAX>();
          int mine = 0;
#pragma unroll
          for (int j = 0; j < HC; ++j) {
            const int m = __reduce_max_sync(0xffffffffu, ordered(v[j]));
            if (lane == j) mine = m;
          }
          if (lane < HC) atomicMax(&sh.top[c0 + lane], mine);
          bar_softmax<SOFTMAX>();
          if (tid < N) {
            const float old = sh.ref[tid], m = fmaxf(old, unordered(sh.top[tid]));
            sh.top[tid] = __float_as_int(ex2_approx((old - m) * f));
            sh.ref[tid] = m;
          }
          bar_softmax<SOFTMAX>();
#pragma unroll
          for (int j = 0; j < HC; ++j) sum[j] *= __int_as_float(sh.top[c0 + j]);
          if (i > 0) {
            wait_for(&sh.o_full, (g - 1) & 1, &sh.dead);
            waited = true;
            __syncwarp();
            tc::tc_fence_after();
#pragma unroll 1
            for (int j = 0; j < PER * HC; j += 8) {
              const int col = c0 + j % HC;
              const uint32_t at = tmem + j / HC * N + col + lanes;
              float o[8];
              tmem_load(at, o);
#pragma unroll
              for (int e = 0; e < 8; ++e) o[e] *= __int_as_float(sh.top[col + e]);
              tmem_store8(at, o);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          }
          less();
        }
        uint32_t p[HC / 2];
#pragma unroll
        for (int j = 0; j < HC / 2; ++j) {
          const float2 y = mul2(make_float2(v[2 * j], v[2 * j + 1]), make_float2(f, f));
          const float2 e = make_float2(ex2_approx(y.x), ex2_approx(y.y)), s = add2(make_float2(sum[2 * j], sum[2 * j + 1]), e);
          sum[2 * j] = s.x, sum[2 * j + 1] = s.y;
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[j]) : "f"(e.y), "f"(e.x));
        }
        if (!waited) wait_for(&sh.o_full, (g - 1) & 1, &sh.dead);   // the product before has read its weights
#pragma unroll
        for (int j = 0; j < HC / 8; ++j)
          *reinterpret_cast<uint4*>(weights + weight_at<N>(k, c0 / 8 + j)) = make_uint4(p[4 * j], p[4 * j + 1], p[4 * j + 2], p[4 * j + 3]);
        tc::fence_async_smem();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive1(&sh.p_full[0]);
      }
      // the next item's queries take the place of these, whose scores are all there
      if (after.more && after.n > 0) bring_queries<RANK, N, SOFTMAX>(a, run, queries, after.x, mem, sh);
      if (n > 0) wait_for(&sh.o_full, (g - 1) & 1, &sh.dead);
      __syncwarp();
      tc::tc_fence_after();
      // sums of the weights over the lanes: each step halves the rows that a lane holds
      float* const lsum = reinterpret_cast<float*>(weights);   // [4][N]
      int m = 16;
#pragma unroll
      for (int h = HC / 2; h > 0; h >>= 1, m >>= 1) {
        const bool up = lane & m;
#pragma unroll
        for (int j = 0; j < HC / 2; ++j)
          if (j < h) {
            const float keep = up ? sum[j + h] : sum[j], give = up ? sum[j] : sum[j + h];
            sum[j] = keep + __shfl_xor_sync(0xffffffffu, give, m);
          }
      }
      for (; m > 0; m >>= 1) sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], m);
      if (lane % (32 / HC) == 0) lsum[warp % 4 * N + c0 + lane / (32 / HC)] = sum[0];
      bar_softmax<SOFTMAX>();
      if (tid < N) {
        const float l = n > 0 ? (lsum[tid] + lsum[N + tid]) + (lsum[2 * N + tid] + lsum[3 * N + tid]) : 0.f;
        if (q.whole)
          sh.top[tid] = __float_as_int(l == 0.f ? 0.f : 1.f / l);
        else
          a.ml[q.slot * N + tid] = make_float2(sh.ref[tid], l);
        sh.ref[tid] = NONE;
        const int R = min(x.r0 + tid, x.last), token = R / a.group;
        sh.to[tid] = (long long)(t.first + token) * a.ldo + (long long)(R - token * a.group) * RANK;
      }
      bar_softmax<SOFTMAX>();
      // (what is read of shared memory is read before the stores: they might write it, for all that the compiler knows)
      const int rows = min(HC, x.last - x.r0 - c0 + 1);
      const bool whole = q.whole;
      float* const part = a.part + (long long)(q.slot * N + c0) * RANK + k;
#pragma unroll 1
      for (int y = 0; y < PER; ++y) {
        float o[HC];
#pragma unroll
        for (int e = 0; e < HC; ++e) o[e] = 0.f;
        if (n > 0) tmem_load(tmem + y * N + c0 + lanes, o);
        if (!whole) {
#pragma unroll
          for (int e = 0; e < HC; ++e)
            if (e < rows) part[e * RANK + y * 128] = o[e];
        } else {
#pragma unroll
          for (int e0 = 0; e0 < HC; e0 += 8) {
            __nv_bfloat16* to[8];
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
              to[e] = static_cast<__nv_bfloat16*>(a.out) + sh.to[c0 + e0 + e] + y * 128 + k, f[e] = __int_as_float(sh.top[c0 + e0 + e]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e0 + e < rows) *to[e] = __float2bfloat16_rn(o[e0 + e] * f[e]);
          }
        }
      }
    }
    if (run.split && !run.by_item && tid == 0 && !shares) run.meta[blockIdx.x] = make_int4(-1, 0, 0, 0);
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (sh.dead) {                                   // a wait was in vain: what is in flight lands before memory is given back
    settle(a.m.status);
    __syncthreads();
  }
  if (warp == 0) tc::tmem_dealloc(tmem, C::ALLOC);
}

template <int RANK, int N>
cudaError_t launch_as(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  return launch_items<RANK, N>(latent_tiles_kernel<RANK, N>, Cfg<RANK, N>::THREADS, Cfg<RANK, N>::SMEM, a, p, st);
}
template <int RANK>
cudaError_t launch_of(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  if (p.tile_rows == 16) return launch_as<RANK, 16>(a, p, st);
  if constexpr (RANK < 512)
    if (p.tile_rows == 64) return launch_as<RANK, 64>(a, p, st);
  return launch_as<RANK, 32>(a, p, st);
}

}  // namespace

cudaError_t launch_latent_tiles(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  return a.m.head_dim == 128 ? launch_of<128>(a, p, st) : a.m.head_dim == 256 ? launch_of<256>(a, p, st) : launch_of<512>(a, p, st);
}

}  // namespace evo
