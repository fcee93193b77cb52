// Attention of bf16 rows over a latent memory, on tcgen05.
//
// All heads share a token's vector, so even one token's attention is a product of n_head rows, and a
// memory's bytes are used 2 n_head times each; keys and values are the same bytes, which are brought to
// shared memory once.  Both products have the memory as their first operand (128 tokens or 128
// dimensions are the 128 rows of an instruction) and the queries' rows as the second, so that 16 rows
// cost an eighth of what 128 do, and the output of 512 dimensions takes 4 N columns of tensor memory:
//   S^T = X Q^T   tokens x rows, X = (c | k) as it lies in its page
//   O^T += C^T P^T  dimensions x rows, C^T by the transposing form of the same tiles
// A block takes N = 16 to 128 rows (tokens of the chunk times heads) and one piece of the memory, 128
// tokens at a time.  Warp 9 brings them by tiled bulk copies into a ring of slots of 128 dimensions
// (and one of key parts); warp 8 issues the products; warps 0-7 are the softmax: a thread has a token
// (its lane of tensor memory) and half of the rows, and writes the weights P^T, which are summed
// over the lanes only at the end.
//
// The running maximum is lazy: a row's reference is raised only when a score passes it by 2^8, so that
// the common tile has one vote in place of reductions over the lanes.  The reference m is subtracted from the
// product, and the difference multiplied by the factor: equal scores have equal weights at any size.
// Weights are rounded to bf16 for their product, 2^-8 of each at most.
//
// Masks are looked at only in tiles that some row does not see whole.  There, tokens outside the piece
// are set to zero in shared memory; so is one with a value that is not finite (0 * NaN would reach
// rows that do not see it), whose score is then NaN for the rows that see it.
#include <algorithm>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
#include "evo_mem_ptx.cuh"

namespace evo {
namespace {

constexpr int BK = 128;                            // tokens of a tile
constexpr int SOFTMAX = 256, THREADS = SOFTMAX + 64;
constexpr int SLOT = BK * 256, HALF = BK * 128;    // bytes of 128 and of 64 dimensions of a tile
constexpr float LAZY = 8.f;                        // log2 of how far a weight may pass 1

template <int RANK, int N>
struct Cfg {
  static constexpr int PER = RANK / 128;           // slots of a tile
  static constexpr int Q = N * (RANK + LATENT_ROPE) * 2, P = BK * N * 2;
  static constexpr int FREE = 227 * 1024 - 1024 - 2048 - Q - P;   // alignment and static shared memory left out
  // tiles of 128 dimensions are one slot and one key part each; else one or two key parts, the rest slots
  static constexpr int EVEN = FREE / (SLOT + HALF), MOST = (FREE - HALF) / SLOT;
  static constexpr int SLOTS = PER == 1 ? EVEN : MOST > 6 ? 6 : MOST;
  static constexpr int PARTS = PER == 1 ? EVEN : FREE - SLOTS * SLOT >= 2 * HALF ? 2 : 1;
  static constexpr bool AHEAD = SLOTS >= 2 * PER && PARTS >= 2;   // the next scores before this output
  static constexpr int SMEM = 1024 + Q + P + SLOTS * SLOT + PARTS * HALF;
  static constexpr int S_COL = PER * N, COLS = S_COL + 2 * N;     // tensor memory: O, then two buffers of S
  static constexpr int ALLOC = COLS <= 64 ? 64 : COLS <= 128 ? 128 : COLS <= 256 ? 256 : 512;
  static constexpr int HC = N / 2;                 // rows of a softmax thread
  static constexpr int LD = RANK + 4;              // floats of a row where sums are handed over
  static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(BK >> 4) << 24);
  static constexpr uint32_t IDESC_O = IDESC | (1u << 15) | (1u << 16);   // contiguous indexes: dimensions, rows
  static_assert(SLOTS >= PER && SLOTS <= 6 && N * LD * 4 <= SMEM - 1024 && COLS <= 512, "");
};

template <int N>
struct Shared {
  uint64_t full[6], empty[6], part_full[6], part_empty[6], s_full[2], p_full, o_full;
  __align__(16) float2 ref[N];                     // what is subtracted from a row's scores, and the score that raises it
  int top[N];                                      // a new maximum (ordered as integers), then the factor of what was summed
  uint32_t bad[4];
  uint32_t tmem;
  int dead;
};

// ---------------------------------------------------------------- PTX wrappers
template <int C>
__device__ __forceinline__ void tmem_load(uint32_t taddr, float (&v)[C]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  if constexpr (C == 8) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr));
  } else if constexpr (C == 16) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
  } else {
#pragma unroll
    for (int i = 0; i < C / 32; ++i) {
      uint32_t* s = r + 32 * i;
      asm volatile(
          "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
          "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
          : "=r"(s[0]), "=r"(s[1]), "=r"(s[2]), "=r"(s[3]), "=r"(s[4]), "=r"(s[5]), "=r"(s[6]), "=r"(s[7]), "=r"(s[8]),
            "=r"(s[9]), "=r"(s[10]), "=r"(s[11]), "=r"(s[12]), "=r"(s[13]), "=r"(s[14]), "=r"(s[15]), "=r"(s[16]),
            "=r"(s[17]), "=r"(s[18]), "=r"(s[19]), "=r"(s[20]), "=r"(s[21]), "=r"(s[22]), "=r"(s[23]), "=r"(s[24]),
            "=r"(s[25]), "=r"(s[26]), "=r"(s[27]), "=r"(s[28]), "=r"(s[29]), "=r"(s[30]), "=r"(s[31])
          : "r"(taddr + 32 * i));
    }
  }
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < C; ++i) asm volatile("" : "+f"(v[i]));   // no use moves in front of the wait
}
__device__ __forceinline__ void tmem_store8(uint32_t taddr, const float* v) {
  const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void bar_softmax() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ bool bar_softmax_or(bool x) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, 1, 256, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"((uint32_t)x)
      : "memory");
  return r != 0;
}
// a bounded wait; false once any wait of the block was in vain
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, int* dead) {
  const uint32_t b = tc::su32(bar);
  return tc::mbar_test(b, parity) || wait_live(b, parity, tc::su32(dead));
}

// operands whose contiguous index is not the contraction's: 64 dimensions by 8 tokens a swizzled
// kilobyte, the next 8 tokens behind it, the next 64 dimensions HALF bytes on
__device__ __forceinline__ uint64_t latent_desc(uint32_t saddr) {
  return (tc::sw128_desc(saddr) & ~(0x3fffull << 16)) | (uint64_t)(HALF >> 4) << 16;
}
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
// floats in the order of integers; a NaN stands for none
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x == x ? x : -INFINITY);
  return b >= 0 ? b : b ^ 0x7fffffff;
}
__device__ __forceinline__ float unordered(int b) { return __int_as_float(b >= 0 ? b : b ^ 0x7fffffff); }

template <int RANK, int N>
__global__ void __launch_bounds__(THREADS, 1) latent_tiles_kernel(const __grid_constant__ AttendArgs a,
                                                                  const __grid_constant__ CUtensorMap map) {
  using C = Cfg<RANK, N>;
  constexpr int PER = C::PER, HC = C::HC, SLOTS = C::SLOTS, PARTS = C::PARTS;
  extern __shared__ uint8_t raw[];
  __shared__ Shared<N> sh;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  uint8_t* const weights = mem + C::Q;
  uint8_t* const ring = weights + C::P;
  uint8_t* const parts = ring + SLOTS * SLOT;
  if (tid == 0) fetch_map(&map);
  const Tile t = tile_of_block(a);
  const int rows = t.count * a.group, r0 = t.tile * N;
  if (r0 >= rows) return;
  const int last = min(r0 + N, rows) - 1;
  const Range first_row = seen_by(a, t, r0 / a.group), last_row = seen_by(a, t, last / a.group);
  const Range all = piece_of(a, t, {first_row.lo, last_row.hi}, BK);
  const int whole_lo = max(last_row.lo, all.lo), whole_hi = min(first_row.hi, all.hi);
  const bool alike = first_row.lo == last_row.lo && first_row.hi == last_row.hi;   // every row sees the same tokens
  const int key0 = all.lo / BK * BK, n = max(0, (all.hi - key0 + BK - 1) / BK);

  __syncwarp();                                    // a whole warp's instruction, behind one lane's prefetch
  if (warp == 0) tc::tmem_alloc(&sh.tmem, C::ALLOC);
  if (tid == 32) {
    for (int i = 0; i < SLOTS; ++i) tc::mbar_init1(&sh.full[i], 1), tc::mbar_init1(&sh.empty[i], 1);
    for (int i = 0; i < PARTS; ++i) tc::mbar_init1(&sh.part_full[i], 1), tc::mbar_init1(&sh.part_empty[i], 1);
    tc::mbar_init1(&sh.s_full[0], 1), tc::mbar_init1(&sh.s_full[1], 1);
    tc::mbar_init1(&sh.p_full, SOFTMAX / 32);      // a warp each
    tc::mbar_init1(&sh.o_full, 1);
    sh.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid >= 64 && tid < 64 + N) sh.ref[tid - 64] = make_float2(0.f, -INFINITY);
  // queries to shared memory; the softmax works with a positive factor
  const float f = a.scale_log2 == 0.f ? 1.f : fmaxf(fabsf(a.scale_log2), 1.1754944e-38f);
  {
    constexpr int PIECES = (RANK + LATENT_ROPE) / 8;
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;
    for (int i = tid; i < N * PIECES; i += THREADS) {
      const int r = i / PIECES, j = i % PIECES, R = r0 + r;
      uint4 u = make_uint4(0, 0, 0, 0);
      if (R < rows && a.scale_log2 != 0.f)
        u = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (long long)(t.first + R / a.group) * a.ldq +
                                           (long long)(R % a.group) * (RANK + LATENT_ROPE))[j];
      u.x ^= flip, u.y ^= flip, u.z ^= flip, u.w ^= flip;
      *reinterpret_cast<uint4*>(mem + (j / 8) * (N * 128) + r * 128 + ((j % 8 ^ (r & 7)) << 4)) = u;
    }
    tc::fence_async_smem();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;

  if (warp == 9) {
    // ------------------------------------------------------------ copies
    const int page_tokens = a.m.page_tokens, box = min(page_tokens, BK), shift = 31 - __clz(page_tokens);
    for (int i = 0; i < n; ++i) {
      const int key = key0 + i * BK + lane * box;
      const bool on = lane * box < BK && key + box > all.lo && key < all.hi;
      const int page = on ? seq_page(a.m, t.n, key >> shift) : 0;
      const int at = page * page_tokens + (key & (page_tokens - 1)), copies = __popc(__ballot_sync(0xffffffffu, on));
      const auto bring = [&](uint8_t* to, uint64_t* full, uint64_t* empty, int use, int column, int halves) {
        if (!__all_sync(0xffffffffu, use == 0 || wait_for(empty, (use - 1) & 1, &sh.dead))) return;
        if (lane == 0) tc::mbar_expect_tx(full, copies * box * 128 * halves);
        __syncwarp();
        if (on)
          for (int x = 0; x < halves; ++x)
            tile_load(tc::su32(to) + x * HALF + lane * box * 128, &map, column + 64 * x, at, tc::su32(full));
        __syncwarp();
      };
      for (int j = 0; j < PER; ++j) {
        const int index = i * PER + j, slot = index % SLOTS;
        bring(ring + slot * SLOT, &sh.full[slot], &sh.empty[slot], index / SLOTS, 128 * j, 2);
      }
      bring(parts + i % PARTS * HALF, &sh.part_full[i % PARTS], &sh.part_empty[i % PARTS], i / PARTS, RANK, 1);
    }
  } else if (warp == 8) {
    // ------------------------------------------------------------ products
    const uint32_t q = tc::su32(mem), w = tc::su32(weights);
    const auto scores = [&](int i) {
      const uint32_t d = tmem + C::S_COL + (i & 1) * N;
      for (int j = 0; j < PER; ++j) {
        const int index = i * PER + j, slot = index % SLOTS;
        wait_for(&sh.full[slot], (index / SLOTS) & 1, &sh.dead);
        tc::tc_fence_after();
        const uint32_t x = tc::su32(ring + slot * SLOT);
        if (tc::elect_one())
#pragma unroll
          for (int k = 0; k < 8; ++k)
            tc::mma_f16(d, tc::sw128_desc(x + (k / 4) * HALF + (k % 4) * 32),
                        tc::sw128_desc(q + (2 * j + k / 4) * (N * 128) + (k % 4) * 32), C::IDESC, j | k);
        __syncwarp();
      }
      wait_for(&sh.part_full[i % PARTS], (i / PARTS) & 1, &sh.dead);
      tc::tc_fence_after();
      const uint32_t x = tc::su32(parts + i % PARTS * HALF);
      if (tc::elect_one()) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          tc::mma_f16(d, tc::sw128_desc(x + k * 32), tc::sw128_desc(q + 2 * PER * (N * 128) + k * 32), C::IDESC, 1);
        tc::mma_commit(&sh.s_full[i & 1]);
        tc::mma_commit(&sh.part_empty[i % PARTS]);
      }
      __syncwarp();
    };
    const auto output = [&](int i) {
      if (tc::elect_one())
        for (int j = 0; j < PER; ++j) {
          const int slot = (i * PER + j) % SLOTS;
          const uint32_t x = tc::su32(ring + slot * SLOT);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            tc::mma_f16(tmem + j * N, latent_desc(x + k * 2048), weight_desc<N>(w + k * (N >= 64 ? 2048 : N * 32)), C::IDESC_O, i | k);
          tc::mma_commit(&sh.empty[slot]);
          if (j == PER - 1) tc::mma_commit(&sh.o_full);
        }
      __syncwarp();
    };
    if (n > 0) scores(0);
    for (int i = 0; i < n; ++i) {
      if (C::AHEAD && i + 1 < n) scores(i + 1);
      wait_for(&sh.p_full, i & 1, &sh.dead);
      tc::tc_fence_after();
      if (__any_sync(0xffffffffu, tc::block_dead(tc::su32(&sh.dead)))) break;
      output(i);
      if (!C::AHEAD && i + 1 < n) scores(i + 1);
    }
  } else {
    // ------------------------------------------------------------ softmax: a token and rows c0 .. c0 + HC - 1 a thread
    // A wait that is in vain ends no turn: the barriers of the softmax want all of its warps.
    const int k = tid % BK, c0 = warp / 4 * HC;
    const uint32_t lanes = (uint32_t)(32 * (warp % 4)) << 16;
    float sum[HC];
#pragma unroll
    for (int j = 0; j < HC; ++j) sum[j] = 0.f;
    for (int i = 0; i < n; ++i) {
      wait_for(&sh.s_full[i & 1], (i >> 1) & 1, &sh.dead);
      __syncwarp();
      tc::tc_fence_after();
      float v[HC];
      tmem_load(tmem + C::S_COL + (i & 1) * N + c0 + lanes, v);
      const int key = key0 + i * BK + k;
      if (key0 + i * BK < whole_lo || key0 + (i + 1) * BK > whole_hi) {
        const bool out = key < all.lo || key >= all.hi;
        // this thread's half of the token's latent
        bool bad = false;
        for (int j = 0; j < PER; ++j) {
          const int index = i * PER + j, slot = index % SLOTS;
          wait_for(&sh.full[slot], (index / SLOTS) & 1, &sh.dead);
          uint4* p = reinterpret_cast<uint4*>(ring + slot * SLOT + warp / 4 * HALF + k * 128);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (out) {
              p[e] = make_uint4(0, 0, 0, 0);
            } else if (!alike) {
              const uint4 u = p[e];
              const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
              for (int y = 0; y < 4; ++y) bad |= (x[y] & 0x7f80u) == 0x7f80u || (x[y] & 0x7f800000u) == 0x7f800000u;
            }
          }
        }
        if (alike) {
#pragma unroll
          for (int j = 0; j < HC; ++j) v[j] = out ? -INFINITY : v[j];
        } else {
          if (tid < 4) sh.bad[tid] = 0;
          bar_softmax();
          if (bad) atomicOr(&sh.bad[k / 32], 1u << (k % 32));
          bar_softmax();
          bad = sh.bad[k / 32] >> (k % 32) & 1;
          if (bad)
            for (int j = 0; j < PER; ++j) {
              uint4* p = reinterpret_cast<uint4*>(ring + (i * PER + j) % SLOTS * SLOT + warp / 4 * HALF + k * 128);
              for (int e = 0; e < 8; ++e) p[e] = make_uint4(0, 0, 0, 0);
            }
#pragma unroll
          for (int j = 0; j < HC; ++j) {
            const Range see = seen_by(a, t, min(r0 + c0 + j, last) / a.group);
            if (bad) v[j] = __builtin_nanf("");
            if (out || key < see.lo || key >= see.hi) v[j] = -INFINITY;
          }
        }
        tc::fence_async_smem();
      }
      bool raise = false;
#pragma unroll
      for (int j = 0; j < HC; j += 2) {
        const float4 r = *reinterpret_cast<const float4*>(&sh.ref[c0 + j]);
        raise |= v[j] > r.y || v[j + 1] > r.w;
      }
      bool waited = i == 0;
      if (bar_softmax_or(raise)) {
        if (tid < N) sh.top[tid] = ordered(-INFINITY);
        bar_softmax();
#pragma unroll
        for (int j0 = 0; j0 < HC; j0 += 32) {
          int mine = 0;
#pragma unroll
          for (int j = 0; j < (HC < 32 ? HC : 32); ++j) {
            const int m = __reduce_max_sync(0xffffffffu, ordered(v[j0 + j]));
            if (lane == j) mine = m;
          }
          if (lane < HC) atomicMax(&sh.top[c0 + j0 + lane], mine);
        }
        bar_softmax();
        if (tid < N) {
          const float2 r = sh.ref[tid];
          const float old = r.y == -INFINITY ? -INFINITY : r.x, m = fmaxf(old, unordered(sh.top[tid]));
          sh.top[tid] = __float_as_int(old == -INFINITY ? 1.f : ex2_approx((old - m) * f));
          if (m != -INFINITY) sh.ref[tid] = make_float2(m, m + LAZY / f);
        }
        bar_softmax();
#pragma unroll
        for (int j = 0; j < HC; ++j) sum[j] *= __int_as_float(sh.top[c0 + j]);
        if (i > 0) {
          wait_for(&sh.o_full, (i - 1) & 1, &sh.dead);
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
      }
      uint32_t p[HC / 2];
#pragma unroll
      for (int j = 0; j < HC; j += 2) {
        const float4 r = *reinterpret_cast<const float4*>(&sh.ref[c0 + j]);
        const float2 x = mul2(add2(make_float2(v[j], v[j + 1]), make_float2(-r.x, -r.z)), make_float2(f, f));
        const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y)), s = add2(make_float2(sum[j], sum[j + 1]), e);
        sum[j] = s.x, sum[j + 1] = s.y;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[j / 2]) : "f"(e.y), "f"(e.x));
      }
      if (!waited) wait_for(&sh.o_full, (i - 1) & 1, &sh.dead);   // the product before has read its weights
#pragma unroll
      for (int j = 0; j < HC / 8; ++j)
        *reinterpret_cast<uint4*>(weights + weight_at<N>(k, c0 / 8 + j)) = make_uint4(p[4 * j], p[4 * j + 1], p[4 * j + 2], p[4 * j + 3]);
      tc::fence_async_smem();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive1(&sh.p_full);
    }
    if (n > 0) wait_for(&sh.o_full, (n - 1) & 1, &sh.dead);
    __syncwarp();
    tc::tc_fence_after();
    // sums of the weights over the lanes: each step halves the rows that a lane holds
    constexpr int B = HC < 32 ? HC : 32;
    float* const lsum = reinterpret_cast<float*>(weights);   // [4][N]
#pragma unroll
    for (int j0 = 0; j0 < HC; j0 += 32) {
      int m = 16;
#pragma unroll
      for (int h = B / 2; h > 0; h >>= 1, m >>= 1) {
        const bool up = lane & m;
#pragma unroll
        for (int j = 0; j < B / 2; ++j)
          if (j < h) {
            const float keep = up ? sum[j0 + j + h] : sum[j0 + j], give = up ? sum[j0 + j] : sum[j0 + j + h];
            sum[j0 + j] = keep + __shfl_xor_sync(0xffffffffu, give, m);
          }
      }
      for (; m > 0; m >>= 1) sum[j0] += __shfl_xor_sync(0xffffffffu, sum[j0], m);
      if (lane % (32 / B) == 0) lsum[warp % 4 * N + c0 + j0 + lane / (32 / B)] = sum[j0];
    }
  }
  __syncthreads();                                 // nothing reads the queries, the ring or the weights any more
  float* const sums = reinterpret_cast<float*>(mem);   // [N][LD]
  float l = 0.f, m = -INFINITY;
  if (tid < N && n > 0) {
    const float* lsum = reinterpret_cast<const float*>(weights);
    l = (lsum[tid] + lsum[N + tid]) + (lsum[2 * N + tid] + lsum[3 * N + tid]);
    const float2 r = sh.ref[tid];
    m = r.y == -INFINITY ? -INFINITY : r.x * f;
  }
  __syncthreads();
  if (tid < N) sh.ref[tid] = make_float2(m, l);
  if (warp < 8) {
    const uint32_t lanes = (uint32_t)(32 * (warp % 4)) << 16;
    const int c0 = warp / 4 * HC;
#pragma unroll 1
    for (int j = 0; j < PER * HC; j += 8) {
      const int col = c0 + j % HC, d = j / HC * 128 + tid % 128;
      float o[8] = {};
      if (n > 0) tmem_load(tmem + j / HC * N + col + lanes, o);
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[(col + e) * C::LD + d] = o[e];
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (sh.dead) {                                   // a wait was in vain: what is in flight lands before memory is given back
    settle(a.m.status);
    __syncthreads();
  }
  if (warp == 0) tc::tmem_dealloc(tmem, C::ALLOC);
  if (a.cluster > 1) {
    join_cluster<__nv_bfloat16, RANK, N, THREADS>(a, t, sums, C::LD, sh.ref, r0, rows);
  } else {
    for (int i = tid; i < N * RANK / 4; i += THREADS) {
      const int r = i / (RANK / 4), d = i % (RANK / 4) * 4;
      if (r0 + r >= rows) break;
      const float2 ml = sh.ref[r];
      put_result<__nv_bfloat16, RANK>(a, t, r0 + r, d, *reinterpret_cast<const float4*>(sums + r * C::LD + d), ml.x, ml.y);
    }
  }
}

template <int RANK, int N>
cudaError_t launch_as(const AttendArgs& a, cudaStream_t st) {
  using C = Cfg<RANK, N>;
  CUtensorMap map;
  if (!latent_map(&map, a.m, std::min(a.m.page_tokens, BK))) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  return launch_pieces(latent_tiles_kernel<RANK, N>, a, THREADS, C::SMEM, done, st, map);
}
template <int RANK>
cudaError_t launch_of(const AttendArgs& a, int tile_rows, cudaStream_t st) {
  if (tile_rows == 16) return launch_as<RANK, 16>(a, st);
  if constexpr (RANK < 512) {
    if (tile_rows == 64) return launch_as<RANK, 64>(a, st);
    if (tile_rows == 128) return launch_as<RANK, 128>(a, st);
  }
  return launch_as<RANK, 32>(a, st);
}

}  // namespace

cudaError_t launch_latent_tiles(const AttendArgs& a, int tile_rows, cudaStream_t st) {
  return a.m.head_dim == 128   ? launch_of<128>(a, tile_rows, st)
         : a.m.head_dim == 256 ? launch_of<256>(a, tile_rows, st)
                               : launch_of<512>(a, tile_rows, st);
}

}  // namespace evo
