// Attention of fp32 rows over a latent memory, on mma.sync: a number is split into two of 11 bits
// and a product taken as three of tf32, off by 2^-21 of itself at most (2^-23 for what each low part
// loses, 2^-22 for the product of the low parts).
//
// As in the bf16 kernel both products have the memory as their first operand,
//   S^T = X Q^T (tokens x rows),   O^T += C^T P^T (dimensions x rows)
// so that the split of a token's values, three instructions each, serves all rows. A block is 8 teams (rank 512: 5) of one
// or two warps on an item of 8 NR rows, or its run's part of one (evo_latent.cuh).  A team takes every eighth (fifth) run of 16
// tokens by itself, which arrives in its own one or two slots by tiled bulk copies, so that no barrier of the block is met
// until the end: while one team waits for its run the others compute.  (Slots of all warps' in one ring would let one
// be two phases ahead of another's wait, which a parity does not show.)  Every team keeps its own maximum
// (lazy: rescaled only when a score passes it by 2^8) and sums, joined through shared memory.
//
// A run's chain of dependent products bounds a team: 14,700 cycles for rank 512 with one warp, whose 408 products need
// 3,300.  Two warps of a team have half of the dimensions each and exchange their parts of the scores: 206 single tokens of
// 2 heads over up to 689 tokens 109 -> 84 us (for rank 128 there is nothing to gain: 46.7 / 47.6).  48 single tokens of 8
// heads over up to 2,050 of rank 256: 35 us, 2.7 TB/s.
//
// Fragments are read 16 bytes at a time, because a contraction's index may be permuted at will (lane (g, c) =
// (lane / 4, lane % 4)):
//   scores   4 dimensions 16 h + 4 c .. of tokens t(g) and 8 + t(g) make two steps; t(g) = g / 2 + 4 (g % 2), so
//            that the 8 lanes of a phase meet 8 different chunks of the copies' swizzle
//   output   4 dimensions 32 b + 4 g .. of tokens 2 c, 2 c + 1 and 8 on: the rows g and g + 8 of two tiles
// The matrix unit cuts its sums off: those of the scores are five (four of high parts, one of the
// others), and the output's products of a run are added to its sums in fp32.
//
// Masks are looked at only in runs that some row does not see whole.  There, the values of tokens outside the piece
// count as zero, and so do those of a token that holds a value that is not finite or whose high part
// is not, whose scores are then no numbers for the rows that see it.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>
#include <new>

#include "evo_latent.cuh"

namespace evo {
namespace {

constexpr int RUN = 16;                            // tokens of a run: a page holds whole ones

template <int RANK, int NR>
struct Cfg {
  static constexpr int DIMS = RANK + LATENT_ROPE, ROWS = 8 * NR, BOXES = DIMS / 32;
  static constexpr int SHARE = RANK == 512 || (RANK == 256 && NR == 1) ? 2 : 1;   // warps that share a run
  static constexpr int BYTES = RUN * DIMS * 4, Q = DIMS / 16 * NR * 1024;   // a run; the queries' fragments, high and low
  static constexpr int ROOM = (225 * 1024 - 1024 - Q - (SHARE == 2 ? 8192 * NR : 0)) / BYTES, TEAMS = ROOM > 8 ? 8 : ROOM, WARPS = TEAMS * SHARE, THREADS = 32 * WARPS;
  static constexpr int HALF = SHARE == 2 ? WARPS * NR * 32 : 1;
  static constexpr int SLOTS = ROOM / TEAMS > 2 ? 2 : ROOM / TEAMS;   // of each team
  static constexpr int LD = RANK + 4, JOIN = TEAMS * ROWS * LD * 4;
  static constexpr int RING = TEAMS * SLOTS * BYTES > JOIN ? TEAMS * SLOTS * BYTES : JOIN;
  static constexpr int SMEM = 1024 + Q + RING;
  static_assert(SMEM <= 225 * 1024, "");
};

__device__ __forceinline__ void mma8(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the 11 leading bits of x, rounded, and what they leave
__device__ __forceinline__ void split(float x, uint32_t& hi, uint32_t& lo) {
  hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
  lo = __float_as_uint(x - __uint_as_float(hi));
}
// is x, or what split rounds it to, not finite?  The latter from 2^128 - 2^116 on
__device__ __forceinline__ bool odd_number(float x) { return (__float_as_uint(x) & 0x7fffffffu) >= 0x7f7ff000u; }

__device__ __forceinline__ void bar_team(int team) { asm volatile("bar.sync %0, 64;" ::"r"(team + 1) : "memory"); }
// of a ballot whose bit 4 g + c is a quarter of token t(g): the tokens
__device__ __forceinline__ uint32_t quarters(uint32_t b) {
  uint32_t x = 0;
#pragma unroll
  for (int y = 0; y < 8; ++y)
    if (b & 0xfu << (4 * y)) x |= 1u << (y / 2 + 4 * (y % 2));
  return x;
}

template <int RANK, int NR>
__global__ void __launch_bounds__(Cfg<RANK, NR>::THREADS, 1)
    latent_f32_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map, const __grid_constant__ Run run) {
  using C = Cfg<RANK, NR>;
  constexpr int WARPS = C::WARPS, TEAMS = C::TEAMS, SHARE = C::SHARE, THREADS = C::THREADS, SLOTS = C::SLOTS;
  constexpr int STEPS = C::DIMS / 16, MINE = STEPS / SHARE, BOXES = RANK / 32 / SHARE;   // steps of 16 dimensions, and those and the boxes of 32 dimensions of the latent that a warp has
  extern __shared__ uint8_t raw[];
  __shared__ Roles sh;
  __shared__ __align__(8) uint64_t full[TEAMS][SLOTS];
  __shared__ float2 stat[TEAMS][C::ROWS];
  __shared__ float4 half[C::HALF];                          // the warps' parts of their teams' scores
  __shared__ uint32_t half_bad[WARPS];
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4, team = warp / SHARE, part = warp % SHARE;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  const uint32_t ring = tc::su32(mem), queries = ring + C::RING;
  if (tid == 0) {
    fetch_map(&map);
    for (int i = 0; i < TEAMS * SLOTS; ++i) tc::mbar_init1(&full[0][i], 1);
    sh.item = run.split ? run.items : blockIdx.x;
    sh.skip = 0;
    sh.tiles = run.split ? 0 : INT_MAX;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  tc::pdl_wait();                                            // what earlier kernels wrote is there
  if (run.split) tc::pdl_trigger();                // the join may take the places that become free, and waits there
  const Share share = count_tiles<C::ROWS, THREADS>(a, run, sh);
  __syncthreads();
  __shared__ __align__(8) uint8_t walk_at[sizeof(Walk<C::ROWS>)];   // one thread's: registers are short
  Walk<C::ROWS>* const walk = reinterpret_cast<Walk<C::ROWS>*>(walk_at);
  bool shares = false, dead = false;
  if (tid == 0) new (walk) Walk<C::ROWS>(a, run, sh);
  if (tid == 0) fill_segment(a, run, share, *walk, sh.seg[0], shares);
  __syncthreads();
  int asked = 0;                                             // runs of this warp before this item's
  const float f = factor_of(a), far = far_of(f), sign = sign_of(a);
  const int shift = 31 - __clz(a.m.page_tokens);
  for (int item = 0; sh.seg[item & 1].more; ++item) {
    const Segment& seg = sh.seg[item & 1];
    const Tile& t = seg.x.t;
    const int rows = seg.x.rows, r0 = seg.x.r0;
    // this block's piece of the tokens, and of these the ones that every row sees
    const Range all = {max(seg.x.all.lo, seg.key0), seg.n == 0 ? 0 : min(seg.x.all.hi, seg.key0 + seg.n * BK)};
    const int whole_lo = max(seg.x.last_row.lo, all.lo), whole_hi = min(seg.x.first_row.hi, all.hi);
    const int from = all.lo / RUN * RUN, n = max(0, (all.hi - from + RUN - 1) / RUN);
    // the j-th run of this team is run i of the piece; only it waits for it and reads it, and its first warp asks for it
    const auto run_of = [&](int j) { return team + j * TEAMS; };
    const auto page_of = [&](int j) { return part == 0 && run_of(j) < n ? seq_page(a.m, t.n, (from + run_of(j) * RUN) >> shift) : 0; };
    const uint32_t mine = ring + team * (SLOTS * C::BYTES);
    const auto ask = [&](int j, int page) {          // to its slot, a lane a box
      if (part != 0 || run_of(j) >= n) return;
      const int slot = (asked + j) % SLOTS;
      uint64_t* bar = &full[team][slot];
      if (lane == 0) tc::mbar_expect_tx(bar, C::BYTES);
      __syncwarp();
      if (lane < C::BOXES)
        tile_load(mine + slot * C::BYTES + lane * (RUN * 128), &map, 32 * lane,
                  (page << shift) + ((from + run_of(j) * RUN) & (a.m.page_tokens - 1)), tc::su32(bar));
    };
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) ask(j, page_of(j));
    int ahead = page_of(SLOTS);
    if (tid == 0) fill_segment(a, run, share, *walk, sh.seg[(item + 1) & 1], shares);   // while copies are under way
    // queries, which take the scale's sign: the fragments of a step pair, high parts and low parts
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
      const int R = r0 + 8 * nr + g;
      const float* const src = static_cast<const float*>(a.q) + (long long)(t.first + R / a.group) * a.ldq + (long long)(R % a.group) * C::DIMS + 4 * c;
#pragma unroll 4
      for (int h = warp; h < STEPS; h += WARPS) {
        const float4 x = R < rows ? *reinterpret_cast<const float4*>(src + 16 * h) : make_float4(0.f, 0.f, 0.f, 0.f);
        uint4 hi, lo;
        split(x.x * sign, hi.x, lo.x), split(x.y * sign, hi.y, lo.y), split(x.z * sign, hi.z, lo.z), split(x.w * sign, hi.w, lo.w);
        uint4* dst = reinterpret_cast<uint4*>(mem + C::RING + (h * NR + nr) * 1024 + lane * 16);
        dst[0] = hi;
        dst[32] = lo;
      }
    }
    __syncthreads();

    float o[NR][2 * BOXES][4], sum[NR][2], top[NR][2];         // o: tile 2 b + j; rows 2 c, 2 c + 1
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
#pragma unroll
      for (int j = 0; j < 2 * BOXES; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nr][j][e] = 0.f;
      sum[nr][0] = sum[nr][1] = 0.f;
      top[nr][0] = top[nr][1] = -INFINITY;
    }
    const int tg = g / 2 + 4 * (g % 2);                        // the token of the scores' row g; row g + 8: 8 further
    int j = 0;
    for (; run_of(j) < n; ++j) {
      const int slot = (asked + j) % SLOTS;
      const uint32_t x = mine + slot * C::BYTES;
      // (after a wait in vain the turns go on, without copies: the other warp of the team is met in each)
      if (!dead) dead = !__all_sync(0xffffffffu, wait_full(tc::su32(&full[team][slot]), ((asked + j) / SLOTS) & 1));
      const int k0 = from + run_of(j) * RUN;
      const bool odd = k0 < whole_lo || k0 + RUN > whole_hi;
      float s[NR][4];
      uint32_t drop = 0;                                       // tokens whose values count as zero
      {
        constexpr int RESTS = NR == 1 ? 4 : 1;                 // sums of the other products: chains of their own, where registers are left
        float hh[NR][4][4] = {}, rest[NR][RESTS][4] = {};
        bool bad0 = false, bad1 = false;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
          const int h = part * MINE + i;
          const float4 x0 = lds_f4(x + h / 2 * (RUN * 128) + tg * 128 + (((4 * (h % 2) + c) ^ tg) << 4));
          const float4 x1 = lds_f4(x + h / 2 * (RUN * 128) + (8 + tg) * 128 + (((4 * (h % 2) + c) ^ tg) << 4));
          if (odd && h < RANK / 16) {
            bad0 |= odd_number(x0.x) || odd_number(x0.y) || odd_number(x0.z) || odd_number(x0.w);
            bad1 |= odd_number(x1.x) || odd_number(x1.y) || odd_number(x1.z) || odd_number(x1.w);
          }
          uint32_t hi[2][4], lo[2][4];
          split(x0.x, hi[0][0], lo[0][0]), split(x1.x, hi[0][1], lo[0][1]), split(x0.y, hi[0][2], lo[0][2]), split(x1.y, hi[0][3], lo[0][3]);
          split(x0.z, hi[1][0], lo[1][0]), split(x1.z, hi[1][1], lo[1][1]), split(x0.w, hi[1][2], lo[1][2]), split(x1.w, hi[1][3], lo[1][3]);
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            const uint4 qh = lds128(queries + (h * NR + nr) * 1024 + lane * 16), ql = lds128(queries + (h * NR + nr) * 1024 + 512 + lane * 16);
            mma8(hh[nr][2 * i % 4], hi[0], qh.x, qh.y);
            mma8(hh[nr][(2 * i + 1) % 4], hi[1], qh.z, qh.w);
            mma8(rest[nr][0], lo[0], qh.x, qh.y);
            mma8(rest[nr][1 % RESTS], hi[0], ql.x, ql.y);
            mma8(rest[nr][2 % RESTS], lo[1], qh.z, qh.w);
            mma8(rest[nr][3 % RESTS], hi[1], ql.z, ql.w);
          }
        }
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float low = rest[nr][0][e];
#pragma unroll
            for (int y = 1; y < RESTS; ++y) low += rest[nr][y][e];
            s[nr][e] = ((hh[nr][0][e] + hh[nr][1][e]) + (hh[nr][2][e] + hh[nr][3][e])) + low;
          }
        if constexpr (SHARE == 2) {                            // the other warp's part of the scores, and of what is no number
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) half[(warp * NR + nr) * 32 + lane] = make_float4(s[nr][0], s[nr][1], s[nr][2], s[nr][3]);
          const uint32_t bad = odd ? __ballot_sync(0xffffffffu, bad0) : 0, bad8 = odd ? __ballot_sync(0xffffffffu, bad1) : 0;
          if (odd && lane == 0) half_bad[warp] = quarters(bad) | quarters(bad8) << 8;
          bar_team(team);
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            const float4 y = half[((warp ^ 1) * NR + nr) * 32 + lane];
            s[nr][0] += y.x, s[nr][1] += y.y, s[nr][2] += y.z, s[nr][3] += y.w;
          }
          if (odd) drop = quarters(bad) | quarters(bad8) << 8 | half_bad[warp ^ 1];
        } else if (odd) {
          drop = quarters(__ballot_sync(0xffffffffu, bad0)) | quarters(__ballot_sync(0xffffffffu, bad1)) << 8;
        }
        if (odd) {
          const int k1 = k0 + tg, k2 = k1 + 8;
#pragma unroll
          for (int y = 0; y < RUN; ++y)
            if (k0 + y < all.lo || k0 + y >= all.hi) drop |= 1u << y;
#pragma unroll
          for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int R = r0 + 8 * nr + 2 * c + e;
              const Range see = R < rows ? seen_by(a, t, R / a.group) : Range{0, 0};
              const int lo = max(see.lo, all.lo), hi = min(see.hi, all.hi);
              if (drop >> tg & 1) s[nr][e] = __builtin_nanf("");
              if (drop >> (tg + 8) & 1) s[nr][2 + e] = __builtin_nanf("");
              if (k1 < lo || k1 >= hi) s[nr][e] = -INFINITY;
              if (k2 < lo || k2 >= hi) s[nr][2 + e] = -INFINITY;
            }
        }
      }
      bool raise = false;
#pragma unroll
      for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float m = fmaxf(s[nr][e], s[nr][2 + e]);
          raise |= m > top[nr][e] + far || (top[nr][e] == -INFINITY && m > -INFINITY);
        }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float m = fmaxf(s[nr][e], s[nr][2 + e]);
#pragma unroll
            for (int y = 4; y < 32; y *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, y));
            m = fmaxf(m, top[nr][e]);
            const float down = m == -INFINITY ? 1.f : ex2_approx((top[nr][e] - m) * f);
            top[nr][e] = m;
            sum[nr][e] *= down;
#pragma unroll
            for (int j = 0; j < 2 * BOXES; ++j) o[nr][j][e] *= down, o[nr][j][2 + e] *= down;
          }
      }
      // weights, and the output's second operand: steps z, tokens 8 z + 2 c and the next, row g
      uint32_t ph[NR][2][2], pl[NR][2][2];
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float m = top[nr][e % 2];
          p[e] = ex2_approx((s[nr][e] - (m == -INFINITY ? 0.f : m)) * f);
          sum[nr][e % 2] += p[e];
        }
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int token = 2 * c + b, src = ((token & 3) * 2 + token / 4) * 4 + g / 2;
            const float y0 = __shfl_sync(0xffffffffu, p[2 * z], src), y1 = __shfl_sync(0xffffffffu, p[2 * z + 1], src);
            split(g % 2 ? y1 : y0, ph[nr][z][b], pl[nr][z][b]);
          }
      }
#pragma unroll
      for (int b = 0; b < BOXES; ++b) {
        float y[NR][2][4] = {};
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int k1 = 8 * z + 2 * c;
          float4 x0 = lds_f4(x + (part * BOXES + b) * (RUN * 128) + k1 * 128 + ((g ^ (2 * c)) << 4));
          float4 x1 = lds_f4(x + (part * BOXES + b) * (RUN * 128) + (k1 + 1) * 128 + ((g ^ (2 * c + 1)) << 4));
          if (odd) {
            if (drop >> k1 & 1) x0 = make_float4(0.f, 0.f, 0.f, 0.f);
            if (drop >> (k1 + 1) & 1) x1 = make_float4(0.f, 0.f, 0.f, 0.f);
          }
          uint32_t hi[2][4], lo[2][4];
          split(x0.x, hi[0][0], lo[0][0]), split(x0.y, hi[0][1], lo[0][1]), split(x1.x, hi[0][2], lo[0][2]), split(x1.y, hi[0][3], lo[0][3]);
          split(x0.z, hi[1][0], lo[1][0]), split(x0.w, hi[1][1], lo[1][1]), split(x1.z, hi[1][2], lo[1][2]), split(x1.w, hi[1][3], lo[1][3]);
#pragma unroll
          for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              mma8(y[nr][j], hi[j], ph[nr][z][0], ph[nr][z][1]);
              mma8(y[nr][j], lo[j], ph[nr][z][0], ph[nr][z][1]);
              mma8(y[nr][j], hi[j], pl[nr][z][0], pl[nr][z][1]);
            }
        }
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nr][2 * b + j][e] += y[nr][j][e];
      }
      if constexpr (SHARE == 2) bar_team(team);                // everybody has read the slot
      __syncwarp();
      if (!dead) ask(j + SLOTS, ahead);
      ahead = page_of(j + 1 + SLOTS);
    }
    asked += j;
    dead = __syncthreads_or(dead);
    if (dead) {                                                // a copy did not arrive
      settle(a.m.status);
      if (tid == 0)                                            // (the join looks at every item's entry)
        while (sh.seg[(item + 1) & 1].more) fill_segment(a, run, share, *walk, sh.seg[(item + 1) & 1], shares);
      break;
    }
    float* const sums = reinterpret_cast<float*>(mem);         // [TEAMS][ROWS][LD], the warps of a team having their dimensions of a row; in place of the ring
    const int teams = min(n, TEAMS);                           // those that had a run
    if (team < teams)
#pragma unroll
      for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float l = sum[nr][e];
#pragma unroll
          for (int y = 4; y < 32; y *= 2) l += __shfl_xor_sync(0xffffffffu, l, y);
          const int r = 8 * nr + 2 * c + e;
          if (g == 0 && part == 0) stat[team][r] = make_float2(top[nr][e], l);
#pragma unroll
          for (int b = 0; b < BOXES; ++b)
            *reinterpret_cast<float4*>(sums + (team * C::ROWS + r) * C::LD + 32 * (part * BOXES + b) + 4 * g) =
                make_float4(o[nr][2 * b][e], o[nr][2 * b][2 + e], o[nr][2 * b + 1][e], o[nr][2 * b + 1][2 + e]);
        }
    __syncthreads();
    for (int i = tid; i < C::ROWS * RANK / 4; i += THREADS) {
      const int r = i / (RANK / 4), d = i % (RANK / 4) * 4;
      if (r0 + r >= rows) break;
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < TEAMS; ++w)
        if (w < teams) m = fmaxf(m, stat[w][r].x);
      const float ref = m == -INFINITY ? 0.f : m;
      float4 v = {};
#pragma unroll
      for (int w = 0; w < TEAMS; ++w) {
        if (w >= teams) break;
        const float2 ml = stat[w][r];
        const float4 y = *reinterpret_cast<const float4*>(sums + (w * C::ROWS + r) * C::LD + d);
        const float fw = ex2_approx((ml.x - ref) * f);
        l = fmaf(ml.y, fw, l);
        v = make_float4(fmaf(y.x, fw, v.x), fmaf(y.y, fw, v.y), fmaf(y.z, fw, v.z), fmaf(y.w, fw, v.w));
      }
      if (seg.whole) {
        const int R = r0 + r;
        store_out(static_cast<float*>(a.out) + (long long)(t.first + R / a.group) * a.ldo + (long long)(R % a.group) * RANK + d, v,
                  l == 0.f ? 0.f : 1.f / l);
      } else {
        const long long at = (long long)seg.slot * C::ROWS + r;
        *reinterpret_cast<float4*>(a.part + at * RANK + d) = v;
        if (d == 0) a.ml[at] = make_float2(m, l);
      }
    }
    tc::fence_async_smem();                                    // before further copies take the place of the sums
    __syncthreads();
  }
  if (run.split && !run.by_item && tid == 0 && !shares) run.meta[blockIdx.x] = make_int4(-1, 0, 0, 0);
}

template <int RANK, int NR>
cudaError_t launch_as(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  using C = Cfg<RANK, NR>;
  CUtensorMap map;
  if (!latent_map(&map, a.m, RUN)) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem(latent_f32_kernel<RANK, NR>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  const Run run = run_of_plan(a, p, C::ROWS);
  Launch launch(p.blocks, C::THREADS, C::SMEM, st);
  e = cudaLaunchKernelEx(&launch.cfg, latent_f32_kernel<RANK, NR>, a, map, run);
  return e != cudaSuccess || !run.split ? e : launch_join_of<float, RANK, C::ROWS>(a, p, run, st);
}

}  // namespace

// rows of a tile: what the registers hold, while that leaves a block for every SM
int latent_f32_rows(int rank, long long all, int n_seq) {
  int rows = rank == 512 ? 8 : rank == 256 ? 16 : 32;
  while (rows > 8 && (all <= rows / 2 || n_seq * ((all + rows - 1) / rows) < 152)) rows /= 2;
  return rows;
}

cudaError_t launch_latent_f32(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  if (a.m.head_dim == 512) return launch_as<512, 1>(a, p, st);
  if (a.m.head_dim == 256) return p.tile_rows == 8 ? launch_as<256, 1>(a, p, st) : launch_as<256, 2>(a, p, st);
  return p.tile_rows == 8 ? launch_as<128, 1>(a, p, st) : p.tile_rows == 16 ? launch_as<128, 2>(a, p, st) : launch_as<128, 4>(a, p, st);
}

}  // namespace evo
