// Attention of many bf16 rows over a latent memory of rank 128 or 256, on tcgen05: items of 128 rows.
//
//   S = Q X^T     rows x tokens, X = (c | k) as it lies in its page
//   P = 2^(S - m) read from tensor memory and written over S as bf16
//   O += P C      P from tensor memory, C by the transposing form of the same tiles
// Here a row is a lane of tensor memory, so no reduction crosses lanes, and the weights need no shared memory, which
// leaves room for two tiles of the memory beside 128 queries (with the memory as first operand, evo_latent_tiles.cu,
// 128 rows leave one and a half, and each tile waits for the copies of the next).  What 512 columns of tensor memory
// hold: two buffers of S and an output of 256.
//
// A thread of the softmax has a row and half of a tile's 128 tokens.  A tile's products take 2,304 cycles for
// rank 256 at a library product's rate, 128 rows by 16 steps of 640 + 256 dimensions, a tile 3,570: with two in the ring
// the next tile's copies wait for this one's output every other time.  4 chunks of up to 250 tokens of 16 heads over 4,096
// tokens each: 67 us, 0.91 PFLOP/s; 64 chunks of 16 tokens of 8 heads over up to 2,050: 31 us, of which start, pieces and
// join are two thirds.
//
// Items, runs, references, roundings and masks are as in evo_latent_tiles.cu.
#include <algorithm>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_latent.cuh"

namespace evo {
namespace {

constexpr int ROWS = 128, WARPS = 8, SOFTMAX = 32 * WARPS, THREADS = SOFTMAX + 64;

template <int RANK>
struct Cfg {
  static constexpr int PER = RANK / 128;           // slots of a tile
  static constexpr int Q = ROWS * (RANK + LATENT_ROPE) * 2;
  static constexpr int FREE = 227 * 1024 - 1024 - 2048 - Q;   // alignment and static shared memory left out
  static constexpr int SLOTS = PER == 1 ? FREE / (SLOT + HALF) : 4, PARTS = PER == 1 ? SLOTS : 1;
  static constexpr int SMEM = 1024 + Q + SLOTS * SLOT + PARTS * HALF;
  static constexpr int O_COL = 256;                // tensor memory: two buffers of S, then O
  static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(ROWS >> 4) << 24);
  static constexpr uint32_t IDESC_S = IDESC | ((uint32_t)(BK >> 3) << 17);
  static constexpr uint32_t IDESC_O = IDESC | (1u << 16) | ((uint32_t)(RANK >> 3) << 17);   // C's contiguous index is N
  // A tile's slots lie behind one another, so that one instruction reads them all (an instruction a slot, which frees the
  // first one sooner: 3,790 cycles a tile against 3,570)
  static_assert(SLOTS * SLOT + PARTS * HALF <= FREE && SLOTS <= 6 && SLOTS % PER == 0, "");
};

struct Shared : Roles {
  int top[ROWS];                                   // a new maximum, ordered as integers
  float sum[ROWS];                                 // of the weights, at an item's end: a place of its own, because one thread of a row
                                                   // may be there before the other has read the last tile's maximum
};
static_assert(sizeof(Shared) <= 2048, "what Cfg::FREE leaves out");

__device__ __forceinline__ void mma_tmem_a(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
template <int RANK>
__global__ void __launch_bounds__(THREADS, 1)
    latent_wide_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map,
                        const __grid_constant__ CUtensorMap queries, const __grid_constant__ Run run) {
  using C = Cfg<RANK>;
  constexpr int PER = C::PER, SLOTS = C::SLOTS, PARTS = C::PARTS, N = ROWS;
  extern __shared__ uint8_t raw[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  uint8_t* const ring = mem + C::Q;
  uint8_t* const parts = ring + SLOTS * SLOT;
  if (tid == 0) fetch_map(&map), fetch_map(&queries);
  __syncwarp();                                    // a whole warp's instruction, behind one lane's prefetch
  if (warp == 0) tc::tmem_alloc(&sh.tmem, 512);
  if (tid == 32) {
    for (int i = 0; i < SLOTS; ++i) tc::mbar_init1(&sh.full[i], 1), tc::mbar_init1(&sh.empty[i], 1);
    for (int i = 0; i < PARTS; ++i) tc::mbar_init1(&sh.part_full[i], 1), tc::mbar_init1(&sh.part_empty[i], 1);
    tc::mbar_init1(&sh.s_full[0], 1), tc::mbar_init1(&sh.s_full[1], 1);
    // a warp each; one for even and one for odd tiles: the softmax may end a tile more before a late test of the first, and
    // two phases further on its parity would say that nothing has come
    tc::mbar_init1(&sh.p_full[0], WARPS), tc::mbar_init1(&sh.p_full[1], WARPS);
    tc::mbar_init1(&sh.q_full, run.flat ? 1 : WARPS);
    tc::mbar_init1(&sh.o_full, 1);
    sh.dead = 0;
    sh.item = run.split ? run.items : blockIdx.x;
    sh.skip = 0;
    sh.tiles = run.split ? 0 : INT_MAX;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc::pdl_wait();                                  // what earlier kernels wrote is there
  if (run.split) tc::pdl_trigger();                // the join may take the places that become free, and waits there
  const Share share = count_tiles<N, THREADS>(a, run, sh);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;
  Walk<N> walk(a, run, sh);
  int g = 0;                                       // tiles so far

  if (warp == WARPS + 1) {
    bring_tiles<RANK, SLOTS, PARTS>(a, walk, map, ring, parts, sh);
  } else if (warp == WARPS) {
    // ------------------------------------------------------------ products (descriptors in uniform registers)
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t rows_desc = tc::sw128_desc(0), turned_desc = latent_desc(0);
    const uint32_t hi = (uint32_t)(rows_desc >> 32), at = tc::su32(ring) >> 4;
    const uint32_t xr = (uint32_t)rows_desc + at, xt = (uint32_t)turned_desc + at, q = (uint32_t)rows_desc + (tc::su32(mem) >> 4),
                   kp = (uint32_t)rows_desc + (tc::su32(parts) >> 4);
    const uint32_t full = tc::su32(sh.full), empty = tc::su32(sh.empty), part_full = tc::su32(sh.part_full),
                   part_empty = tc::su32(sh.part_empty), dead_word = tc::su32(&sh.dead);
    const uint32_t s_full = tc::su32(sh.s_full), p_full = tc::su32(sh.p_full), o_full = tc::su32(&sh.o_full);
    uint32_t s_slot = 0, s_phase = 0, s_part = 0, s_part_phase = 0, o_slot = 0;
    const auto wait = [&](uint32_t bar, uint32_t parity) {
      if (!tc::mbar_test(bar, parity)) wait_slow(bar, parity, dead_word);
    };
    const auto scores = [&](uint32_t i) {          // of tile i, over the weights of tile i - 2, whose output is done
      const uint32_t d = tm + (i & 1) * BK;
#pragma unroll
      for (uint32_t j = 0; j < PER; ++j) {
        wait(full + 8 * s_slot, s_phase);
        tc::tc_fence_after();
        const uint32_t x = xr + s_slot * (SLOT >> 4);
        if (tc::elect_one())
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k)
            tc::mma_f16(d, desc64(q + (2 * j + k / 4) * (N * 128 >> 4) + (k % 4) * 2, hi), desc64(x + (k / 4) * (HALF >> 4) + (k % 4) * 2, hi),
                        C::IDESC_S, j | k);
        if (++s_slot == SLOTS) s_slot = 0, s_phase ^= 1;
      }
      wait(part_full + 8 * s_part, s_part_phase);
      tc::tc_fence_after();
      const uint32_t x = kp + s_part * (HALF >> 4);
      if (tc::elect_one()) {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
          tc::mma_f16(d, desc64(q + 2 * PER * (N * 128 >> 4) + k * 2, hi), desc64(x + k * 2, hi), C::IDESC_S, 1);
        commit(s_full + 8 * (i & 1));
        commit(part_empty + 8 * s_part);
      }
      if (++s_part == PARTS) s_part = 0, s_part_phase ^= 1;
    };
    const auto output = [&](uint32_t i, uint32_t accumulate) {
      const uint32_t x = xt + o_slot * (SLOT >> 4);
      if (tc::elect_one()) {
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
          mma_tmem_a(tm + C::O_COL, tm + (i & 1) * BK + 8 * k, desc64(x + k * (2048 >> 4), hi), C::IDESC_O, k ? 1 : accumulate);
#pragma unroll
        for (uint32_t j = 0; j < PER; ++j) commit(empty + 8 * (o_slot + j));
        commit(o_full);
      }
      o_slot += PER;
      if (o_slot == SLOTS) o_slot = 0;
    };
    bool dead = false;
    while (!dead && walk.next()) {
      if (walk.n == 0) continue;
      const int n = __shfl_sync(0xffffffffu, walk.n, 0);
      wait(tc::su32(&sh.q_full), (walk.filled - 1) & 1);
      tc::tc_fence_after();
      scores(g);
      for (int i = 0; i < n; ++i, ++g) {
        bool early = i + 1 >= n, done = g == 0;    // done: the output before this one is
        for (const long long since = clock64(); !early && !test(p_full + 8 * (g & 1), (g >> 1) & 1);) {
          early = test(part_full + 8 * s_part, s_part_phase) && (done || test(o_full, (g - 1) & 1));
          if (early) scores(g + 1), done = true;
          else if (clock64() - since > WAIT_CYCLES_DEFAULT) break;   // (the wait below reports it)
        }
        wait(p_full + 8 * (g & 1), (g >> 1) & 1);
        if (!done) wait(o_full, (g - 1) & 1);
        tc::tc_fence_after();
        dead = __any_sync(0xffffffffu, tc::block_dead(dead_word));
        if (dead) break;
        output(g, i);
        if (!early) scores(g + 1);
      }
    }
  } else {
    // ------------------------------------------------------------ softmax: a row and half of a tile's tokens a thread
    // A wait that is in vain ends no turn: the barriers of the softmax want all of its warps.
    const int r = tid % ROWS, half = tid / ROWS;
    const uint32_t lanes = (uint32_t)(32 * (warp % 4)) << 16;
    const float f = factor_of(a), far = far_of(f), sign = sign_of(a);
    // the first warp looks the next item up for all of them
    bool shares = false;
    const auto look_up = [&](Segment& q) {
      bar_softmax<SOFTMAX>();                        // nobody is at the item before any more
      if (warp == 0) fill_segment(a, run, share, walk, q, shares);
      bar_softmax<SOFTMAX>();
    };
    look_up(sh.seg[0]);
    if (sh.seg[0].more && sh.seg[0].n > 0) bring_queries<RANK, N, SOFTMAX>(a, run, queries, sh.seg[0].x, mem, sh);
    for (int s = 0; sh.seg[s].more; s ^= 1) {
      const Segment& q = sh.seg[s];
      const Segment& after = sh.seg[s ^ 1];
      if (q.n > 0) queries_there(run, sh);
      look_up(sh.seg[s ^ 1]);
      const Item& x = q.x;
      const int n = q.n, key0 = q.key0;
      const Range see = seen_by(a, x.t, min(x.r0 + r, x.last) / a.group);
      float ref = NONE, l = 0.f;
      for (int i = 0; i < n; ++i, ++g) {
        wait_for(&sh.s_full[g & 1], (g >> 1) & 1, &sh.dead);
        __syncwarp();
        tc::tc_fence_after();
        float v[64];
        const uint32_t buffer = tmem + (g & 1) * BK + lanes, scores = buffer + 64 * half;
        tmem_load(scores, v);
        if (sign != 1.f)
#pragma unroll
          for (int j = 0; j < 64; ++j) v[j] *= sign;
        const int k0 = key0 + i * BK;
        const bool odd = k0 < x.last_row.lo || k0 + BK > x.first_row.hi;
        if (odd) {
          const int k = r, key = k0 + k;             // of the cleaning: a token and 64 of each 128 dimensions
          const bool alike = q.alike, out = key < x.all.lo || key >= x.all.hi;
          bool bad = false;
          for (int j = 0; j < PER; ++j) {
            const int index = g * PER + j, slot = index % SLOTS;
            wait_for(&sh.full[slot], (index / SLOTS) & 1, &sh.dead);
            uint4* p = reinterpret_cast<uint4*>(ring + slot * SLOT + half * HALF + k * 128);
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
          uint32_t bits[2] = {0, 0};                 // of this thread's tokens, those that hold a value that is not finite
          if (!alike) {
            if (tid < 4) sh.bad[tid] = 0;
            bar_softmax<SOFTMAX>();
            if (bad) atomicOr(&sh.bad[k / 32], 1u << (k % 32));
            bar_softmax<SOFTMAX>();
            if (sh.bad[k / 32] >> (k % 32) & 1)
              for (int j = 0; j < PER; ++j) {
                uint4* p = reinterpret_cast<uint4*>(ring + (g * PER + j) % SLOTS * SLOT + half * HALF + k * 128);
                for (int e = 0; e < 8; ++e) p[e] = make_uint4(0, 0, 0, 0);
              }
            bits[0] = sh.bad[2 * half], bits[1] = sh.bad[2 * half + 1];
          }
          const int lo = see.lo - k0 - 64 * half, hi = see.hi - k0 - 64 * half;
#pragma unroll
          for (int j = 0; j < 64; ++j) {
            if (bits[j / 32] >> (j % 32) & 1) v[j] = __builtin_nanf("");
            if (j < lo || j >= hi) v[j] = -INFINITY;
          }
          tc::fence_async_smem();
        }
        if (odd || sign != 1.f) {                    // where a new reference looks for them
          tmem_store32(scores, reinterpret_cast<const uint32_t*>(v));
          tmem_store32(scores + 32, reinterpret_cast<const uint32_t*>(v + 32));
          tmem_wait_st();
        }
        const auto less = [&] {                      // scores less their reference; one of nothing is far below any
          float top = -INFINITY;
#pragma unroll
          for (int j = 0; j < 64; j += 2) {
            const float2 d = add2(make_float2(v[j], v[j + 1]), make_float2(-ref, -ref));
            v[j] = d.x, v[j + 1] = d.y;
            top = fmaxf(top, fmaxf(d.x, d.y));
          }
          return top;
        };
        // (the weights go over the scores of both threads of a row: behind this barrier everybody has his)
        bool waited = i + 1 < n || i == 0;
        if (bar_softmax_or<SOFTMAX>(less() > far)) {
          if (tid < ROWS) sh.top[tid] = ordered(-INFINITY);
          tmem_load(scores, v);
          float top = v[0];
#pragma unroll
          for (int j = 1; j < 64; ++j) top = fmaxf(top, v[j]);
          bar_softmax<SOFTMAX>();
          atomicMax(&sh.top[r], ordered(top));
          bar_softmax<SOFTMAX>();
          const float m = fmaxf(ref, unordered(sh.top[r])), down = ex2_approx((ref - m) * f);
          ref = m;
          l *= down;
          if (i > 0) {
            wait_for(&sh.o_full, (g - 1) & 1, &sh.dead);
            waited = true;
            __syncwarp();
            tc::tc_fence_after();
            if (__any_sync(0xffffffffu, down != 1.f))
#pragma unroll 1
              for (int j = 0; j < RANK / 2; j += 32) {
                const uint32_t at = tmem + C::O_COL + half * (RANK / 2) + j + lanes;
                float o[32];
                tmem_load(at, o);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] *= down;
                tmem_store32(at, reinterpret_cast<const uint32_t*>(o));
              }
            tmem_wait_st();
          }
          less();
        }
        uint32_t p[32];
        float2 sums[4] = {};                         // chains of their own
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float2 y = mul2(make_float2(v[2 * j], v[2 * j + 1]), make_float2(f, f));
          const float2 e = make_float2(ex2_approx(y.x), ex2_approx(y.y));
          sums[j % 4] = add2(sums[j % 4], e);
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[j]) : "f"(e.y), "f"(e.x));
        }
        const float2 all4 = add2(add2(sums[0], sums[1]), add2(sums[2], sums[3]));
        l += all4.x + all4.y;
        tmem_store32(buffer + 32 * half, p);
        tmem_wait_st();
        // The last output is waited for below.  A parity tells two phases apart, and so the output before has to be done
        // when that wait begins: the scores that came say so only of the one before that
        if (!waited) wait_for(&sh.o_full, (g - 1) & 1, &sh.dead);
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive1(&sh.p_full[g & 1]);
      }
      // a row's sum from its two threads
      if (half == 1) sh.sum[r] = l;
      bar_softmax<SOFTMAX>();
      if (half == 0) {
        l += sh.sum[r];
        sh.sum[r] = l;
      }
      bar_softmax<SOFTMAX>();
      l = sh.sum[r];
      if (n > 0) wait_for(&sh.o_full, (g - 1) & 1, &sh.dead);
      __syncwarp();
      tc::tc_fence_after();
      const bool whole = q.whole;
      const float norm = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
      float* const part = a.part + ((long long)q.slot * RANK + half * (RANK / 2)) * N + r;
      if (!whole && half == 0) a.ml[(long long)q.slot * N + r] = make_float2(ref, l);
#pragma unroll 1
      for (int j = 0; j < RANK / 2; j += 32) {
        float o[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0.f;
        if (n > 0) tmem_load(tmem + C::O_COL + half * (RANK / 2) + j + lanes, o);
        if (whole) {                                 // as bf16 to the queries' place, 64 dimensions behind one another
          const int d = half * (RANK / 2) + j;
          uint32_t v[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[e]) : "f"(o[2 * e + 1] * norm), "f"(o[2 * e] * norm));
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint4*>(mem + d / 64 * (N * 128) + r * 128 + (((d % 64 / 8 + e) ^ (r & 7)) << 4)) =
                make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) part[(j + e) * N] = o[e];
        }
      }
      if (whole) {                                   // and out in whole rows
        bar_softmax<SOFTMAX>();
        constexpr int PIECES = RANK / 8;
#pragma unroll 4
        for (int i = tid; i < N * PIECES; i += SOFTMAX) {
          const int y = i / PIECES, e = i % PIECES, R = x.r0 + y, token = R / a.group;
          if (R <= x.last)
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + (long long)(x.t.first + token) * a.ldo +
                                      (long long)(R - token * a.group) * RANK + 8 * e) =
                *reinterpret_cast<const uint4*>(mem + e / 8 * (N * 128) + y * 128 + ((e % 8 ^ (y & 7)) << 4));
        }
        tc::fence_async_smem();
        bar_softmax<SOFTMAX>();
      }
      if (after.more && after.n > 0) bring_queries<RANK, N, SOFTMAX>(a, run, queries, after.x, mem, sh);
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
  if (warp == 0) tc::tmem_dealloc(tmem, 512);
}

template <int RANK>
cudaError_t launch_as(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  return launch_items<RANK, ROWS>(latent_wide_kernel<RANK>, THREADS, Cfg<RANK>::SMEM, a, p, st);
}

}  // namespace

cudaError_t launch_latent_wide(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  return a.m.head_dim == 128 ? launch_as<128>(a, p, st) : launch_as<256>(a, p, st);
}

}  // namespace evo
