// What the kernels of attention over a latent memory share: items and the runs of tiles that resident
// blocks take of them, the join of what they leave, the copies of the tcgen05 kernels, and wrappers.
//
// An item is a number of rows (tokens of a chunk times heads) of one sequence with the tokens of the memory that
// any of them sees, in tiles of 128.  Blocks stay resident, one a SM.  Where whole items would not fill
// them evenly, the tiles of all items are counted (every block does so, by itself) and each block takes an equal run of
// them, so that sequences of different lengths end at the same time; the first and the last item of a run are shared
// with other blocks, leave their sums in the workspace and are joined by a second kernel.
//
// The join is bound by the time of a load after another: a row's sums and statistics of several pieces are read at once, and
// there is a block only for what may be shared (one token of 16,389 in 129 pieces: 3.5 us of 11.3; 7 with a load behind
// the other).
#pragma once

#include <algorithm>
#include <atomic>
#include <climits>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
#include "evo_mem_ptx.cuh"

namespace evo {

constexpr int BK = 128;                            // tokens of a tile
constexpr int SMS = 152;
constexpr int SLOT = BK * 256, HALF = BK * 128;    // bytes of 128 and of 64 dimensions of a tile
constexpr float LAZY = 8.f;                        // log2 of how far a weight may pass 1
// The reference of a row that has seen nothing.  It is one like any other: scores next to it do not raise it, and have weights
constexpr float NONE = -3.402823466e38f;

// The softmax works on products <q, x> themselves, which are fp32 numbers where they times the scale need not be: 2^(f (s - m)) with
// a positive factor f, and the scale's sign in the products.  So are the maxima of pieces.
__device__ __forceinline__ float factor_of(const AttendArgs& a) {
  return a.scale_log2 == 0.f ? 1.f : fmaxf(fabsf(a.scale_log2), 1.1754944e-38f);
}
__device__ __forceinline__ float sign_of(const AttendArgs& a) { return a.scale_log2 < 0.f ? -1.f : a.scale_log2 == 0.f ? 0.f : 1.f; }
// how far a product may pass its reference
__device__ __forceinline__ float far_of(float f) { return fminf(LAZY / f, 1e38f); }

// An item's beginning and end, in tiles (items of N rows): they count in a run before its tiles.  (128 rows: 34.5 -> 31.3 us
// for 64 chunks of 16 tokens; 64 rows: 40.8 -> 39.0 for 32 tokens; fewer: 84.4 -> 86.0 with 1 for 64 tokens, whose tiles are long)
template <int N>
constexpr int EXTRA = N >= 64 ? 2 : 0;

// An item's rows and the tokens that they see
struct Item {
  Tile t;
  int rows, r0, last;             // rows of the sequence; the item's are r0 .. last
  Range first_row, last_row, all;
  int tile0, tiles;               // tiles of 128 tokens that some row sees
  // what it counts in a run (an item without tiles is written as zeros, and counts as one)
  template <int N>
  __device__ __forceinline__ int cost() const { return r0 >= rows ? 0 : EXTRA<N> + max(1, tiles); }
};
// what the softmax's warps have to know of one item, or of what this block has of it
struct Segment {
  Item x;
  int more, n, key0, slot, whole; // more: there is one.  n tiles from token key0 on; slot: of its sums, unless it is whole here
  bool alike;                     // every row sees the same tokens
};

struct Run {
  int items, split;                                // split: blocks take equal runs of tiles; else whole items, every gridDim-th
  int flat;                                        // queries lie row behind row: an item's come by tiled copies
  int by_item;                                     // there are fewer items than blocks: meta is by the item, else by the block that has an item's first tile
  int4* meta;                                      // of an item that goes on to other blocks: its piece's slot (else -1), the first block, the last, the item
};

// shared memory of the roles
struct Roles {
  uint64_t full[6], empty[6], part_full[6], part_empty[6], s_full[2], p_full[2], o_full, q_full;
  uint32_t bad[4];
  uint32_t tmem;
  int dead, item, skip;                            // the first item's number, and the tiles of it that others take
  int tiles, warp_tiles[32];                       // tiles that the block takes; sums of the warps' items
  Segment seg[2];
  Item begin;                                      // the block's first item
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
template <int THREADS>
__device__ __forceinline__ void bar_softmax() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }
template <int THREADS>
__device__ __forceinline__ bool bar_softmax_or(bool x) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"((uint32_t)x), "n"(THREADS)
      : "memory");
  return r != 0;
}
// a bounded wait; false once any wait of the block was in vain
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, int* dead) {
  const uint32_t b = tc::su32(bar);
  return tc::mbar_test(b, parity) || wait_live(b, parity, tc::su32(dead));
}

// does not suspend the warp, for the one that waits for either of two; one lane's answer for all
__device__ __forceinline__ bool test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return __shfl_sync(0xffffffffu, ok, 0) != 0;
}
// a wait behind a first test that failed
static __device__ __noinline__ void wait_slow(uint32_t bar, uint32_t parity, uint32_t dead) { wait_live(bar, parity, dead); }
__device__ __forceinline__ uint64_t desc64(uint32_t lo, uint32_t hi) { return ((uint64_t)hi << 32) | lo; }
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// operands whose contiguous index is not the contraction's: 64 dimensions by 8 tokens a swizzled
// kilobyte, the next 8 tokens behind it, the next 64 dimensions HALF bytes on
__device__ __forceinline__ uint64_t latent_desc(uint32_t saddr) {
  return (tc::sw128_desc(saddr) & ~(0x3fffull << 16)) | (uint64_t)(HALF >> 4) << 16;
}
// floats in the order of integers; a NaN stands for none
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x == x ? x : -INFINITY);
  return b >= 0 ? b : b ^ 0x7fffffff;
}
__device__ __forceinline__ float unordered(int b) { return __int_as_float(b >= 0 ? b : b ^ 0x7fffffff); }

template <int N>
__device__ __forceinline__ Item item_of(const AttendArgs& a, int i) {
  Item x;
  x.t = {};
  x.t.n = i / a.tiles;
  const SeqRows s = seq_rows(a.m, x.t.n, a.rows, a.max_new);
  x.t.first = s.first;
  x.t.count = s.count;
  x.t.len = seq_len(a.m, x.t.n, a.max_len);
  x.rows = s.count * a.group;
  x.r0 = i % a.tiles * N;
  x.last = min(x.r0 + N, x.rows) - 1;
  x.first_row = seen_by(a, x.t, x.r0 / a.group);
  x.last_row = seen_by(a, x.t, max(x.last, 0) / a.group);
  x.all = {x.first_row.lo, x.last_row.hi};
  x.tile0 = x.all.lo / BK;
  x.tiles = x.r0 >= x.rows || x.all.hi <= x.all.lo ? 0 : (x.all.hi + BK - 1) / BK - x.tile0;
  return x;
}

// `blocks` runs of `tiles` tiles, the first ones a tile longer: where run b begins, and which has tile t
__device__ __forceinline__ int run_from(int tiles, int blocks, int b) { return blocks ? b * (tiles / blocks) + min(b, tiles % blocks) : 0; }
__device__ __forceinline__ int block_of(int tiles, int blocks, int t) {
  const int each = tiles / blocks, longer = tiles % blocks * (each + 1);
  return t < longer ? t / (each + 1) : tiles % blocks + (t - longer) / each;
}

// The block's items one after the other, the same for every role
template <int N>
struct Walk {
  const AttendArgs& a;
  const Run& run;
  const Item& begin;
  int item, skip, left;
  bool fresh = true;
  // this segment: tiles from .. from + n - 1 of item x
  Item x;
  int index, from, n, segments = 0, filled = 0;   // filled: segments with tiles so far
  int after;                                       // tiles of the item that later blocks have

  template <typename S>
  __device__ __forceinline__ Walk(const AttendArgs& a, const Run& run, const S& sh)
      : a(a), run(run), begin(sh.begin), item(sh.item), skip(sh.skip), left(sh.tiles) {}
  __device__ __forceinline__ bool next() {
    for (; item < run.items && left > 0; item += run.split ? 1 : gridDim.x, skip = 0) {
      x = fresh ? begin : item_of<N>(a, item);
      fresh = false;
      const int cost = x.template cost<N>();
      if (cost == 0) {                             // behind the sequence's rows: so are the others up to the next sequence's
        if (!run.split) item += (((x.t.n + 1) * a.tiles - item + (int)gridDim.x - 1) / (int)gridDim.x - 1) * (int)gridDim.x;
        continue;
      }
      const int take = min(cost - skip, left), upto = min(max(skip + take - EXTRA<N>, 0), x.tiles);
      from = min(max(skip - EXTRA<N>, 0), x.tiles);
      n = upto - from;
      after = x.tiles - upto;
      if (run.split) left -= take;
      if (n == 0 && x.tiles > 0) continue;         // no tile, only of what goes before
      index = item;
      item += run.split ? 1 : gridDim.x;
      skip = 0;
      ++segments;
      filled += n > 0;
      return true;
    }
    return false;
  }
  __device__ __forceinline__ int key0() const { return (x.tile0 + from) * BK; }
};

// The tiles of all items, and the blocks that take some; the block's own part of them goes to sh (all threads call it,
// behind a barrier of the block that follows what set sh up, and wait for another one before they read it)
struct Share { int total, blocks; };
template <int N, int THREADS>
__device__ __forceinline__ Share count_tiles(const AttendArgs& a, const Run& run, Roles& sh) {
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  int total = 0, blocks = gridDim.x;
  if (!run.split) {
    if (tid == 0) sh.begin = item_of<N>(a, blockIdx.x);
  } else {
    // every thread counts the tiles of a few items; the block's run is the blockIdx-th of `blocks` equal ones
    const int each = (run.items + THREADS - 1) / THREADS, i0 = tid * each, i1 = min(i0 + each, run.items);
    Item x;
    if (i0 < i1) x = item_of<N>(a, i0);
    const int one = i0 < i1 ? x.template cost<N>() : 0;
    int mine = one;
    for (int i = i0 + 1; i < i1; ++i) mine += item_of<N>(a, i).template cost<N>();
    const auto up_to = [&](int v) {                // sum over the lanes up to this one
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int y = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += y;
      }
      return v;
    };
    int before = up_to(mine);
    if (lane == 31) sh.warp_tiles[warp] = before;
    __syncthreads();
    const int warps = up_to(lane < THREADS / 32 ? sh.warp_tiles[lane] : 0);
    total = __shfl_sync(0xffffffffu, warps, 31);
    before += (warp ? __shfl_sync(0xffffffffu, warps, max(warp - 1, 0)) : 0) - mine;
    blocks = min(blocks, total);
    const int lo = run_from(total, blocks, blockIdx.x), hi = run_from(total, blocks, blockIdx.x + 1);
    if (blockIdx.x < blocks && lo >= before && lo < before + mine) {   // the run begins in one of this thread's items
      int i = i0;
      for (int cost = one; lo >= before + cost; cost = x.template cost<N>()) before += cost, x = item_of<N>(a, ++i);
      sh.begin = x;
      sh.item = i;
      sh.skip = lo - before;
      sh.tiles = hi - lo;
    }
  }
  return {total, blocks};
}

// the copying warp: every tile of the block's, its latents to slots of 128 dimensions and its key parts
template <int RANK, int SLOTS, int PARTS, typename W>
__device__ __forceinline__ void bring_tiles(const AttendArgs& a, W& walk, const CUtensorMap& map, uint8_t* ring, uint8_t* parts, Roles& sh) {
  const int lane = threadIdx.x % 32;
  int g = 0;
  const int page_tokens = a.m.page_tokens, box = min(page_tokens, BK), shift = 31 - __clz(page_tokens), log_boxes = 7 - shift;   // 1 << log_boxes boxes a tile
  while (walk.next()) {
    const Range all = walk.x.all;
    // pages are looked up for 32 boxes of consecutive tiles at once, a lane each (-1: it holds no token of the item)
    const auto pages_from = [&](int i) {
      const int tile = i + (lane >> log_boxes), key = walk.key0() + i * BK + lane * box;
      return tile < walk.n && key + box > all.lo && key < all.hi ? seq_page(a.m, walk.x.t.n, key >> shift) : -1;
    };
    int batch = pages_from(0);
    for (int i = 0; i < walk.n; ++i, ++g) {
      const int at_lane = (i << log_boxes) & 31;
      if (at_lane == 0 && i > 0) batch = pages_from(i);
      const int page = __shfl_sync(0xffffffffu, batch, (at_lane + lane) & 31);
      const bool on = lane >> log_boxes == 0 && page >= 0;
      const int at = page * page_tokens + ((walk.key0() + i * BK + lane * box) & (page_tokens - 1));
      const int copies = __popc(__ballot_sync(0xffffffffu, on));
      const auto bring = [&](uint8_t* to, uint64_t* full, uint64_t* empty, int use, int column, int halves) {
        if (!__all_sync(0xffffffffu, use == 0 || wait_for(empty, (use - 1) & 1, &sh.dead))) return;
        if (lane == 0) tc::mbar_expect_tx(full, copies * box * 128 * halves);
        __syncwarp();
        if (on)
          for (int x = 0; x < halves; ++x)
            tile_load(tc::su32(to) + x * HALF + lane * box * 128, &map, column + 64 * x, at, tc::su32(full));
        __syncwarp();
      };
      for (int j = 0; j < RANK / 128; ++j) {
        const int index = g * (RANK / 128) + j, slot = index % SLOTS;
        bring(ring + slot * SLOT, &sh.full[slot], &sh.empty[slot], index / SLOTS, 128 * j, 2);
      }
      bring(parts + g % PARTS * HALF, &sh.part_full[g % PARTS], &sh.part_empty[g % PARTS], g / PARTS, RANK, 1);
    }
  }
}

// An item's queries to shared memory, 64 of their dimensions behind one another, 128-byte swizzle.  Flat ones are one
// lane's tiled copies (rows behind the sequence's are others', and nobody's result), others all threads' asynchronous ones,
// which queries_there waits for.
template <int RANK, int N, int SOFTMAX>
__device__ __forceinline__ void bring_queries(const AttendArgs& a, const Run& run, const CUtensorMap& map, const Item& x, uint8_t* mem, Roles& sh) {
  const int tid = threadIdx.x;
  if (run.flat) {
    if (tid == 0) {
      tc::mbar_expect_tx(&sh.q_full, N * (RANK + LATENT_ROPE) * 2);
      const int row = x.t.first * a.group + x.r0;
      for (int c = 0; c < (RANK + LATENT_ROPE) / 64; ++c) tile_load(tc::su32(mem + c * (N * 128)), &map, 64 * c, row, tc::su32(&sh.q_full));
    }
    return;
  }
  constexpr int PIECES = (RANK + LATENT_ROPE) / 8;
#pragma unroll 2
  for (int i = tid; i < N * PIECES; i += SOFTMAX) {
    const int r = i / PIECES, j = i % PIECES, R = x.r0 + r, on = R < x.rows ? 16 : 0, token = on ? R / a.group : 0;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + (long long)(x.t.first + token) * a.ldq +
                               (long long)(on ? R - token * a.group : 0) * (RANK + LATENT_ROPE) + 8 * j;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                     tc::su32(mem + (j / 8) * (N * 128) + r * 128 + ((j % 8 ^ (r & 7)) << 4))),
                 "l"(src), "r"(on)
                 : "memory");
  }
}
__device__ __forceinline__ void queries_there(const Run& run, Roles& sh) {
  if (run.flat) return;
  asm volatile("cp.async.wait_all;" ::: "memory");
  tc::fence_async_smem();
  __syncwarp();
  if (threadIdx.x % 32 == 0) tc::mbar_arrive1(&sh.q_full);
}

// the block's next item, by the first warp of the softmax for all; shares: an item goes on to further blocks
template <typename W>
__device__ __forceinline__ void fill_segment(const AttendArgs& a, const Run& run, const Share& share, W& walk, Segment& q, bool& shares) {
  const bool more = walk.next();
  if (threadIdx.x % 32 != 0) return;
  q.more = more;
  if (!more) return;
  const Item& x = walk.x;
  q.x = x;
  q.n = walk.n;
  q.key0 = walk.key0();
  q.slot = 2 * blockIdx.x + (walk.segments > 1 ? 1 : 0);   // of an item that other blocks share: the run's first or last
  q.whole = walk.from == 0 && walk.after == 0;
  q.alike = x.first_row.lo == x.last_row.lo && x.first_row.hi == x.last_row.hi;
  if (walk.from == 0 && walk.after > 0) {          // it goes on to the block that has the last of its tiles
    const int end = run_from(share.total, share.blocks, blockIdx.x + 1) + walk.after;
    run.meta[run.by_item ? walk.index : blockIdx.x] = make_int4(q.slot, blockIdx.x, block_of(share.total, share.blocks, end - 1), walk.index);
    shares = true;
  } else if (run.by_item && walk.from == 0) {
    run.meta[walk.index] = make_int4(-1, 0, 0, 0);
  }
}

// Joins the pieces of the items that blocks share: that of the block which has an item's first tile, and the first one of each
// block behind it up to the last.
struct Pieces {
  int slot, first, n;             // n: 0, nothing to join
  SeqRows s;
  int r0;                         // of the item, in its sequence's rows
  __device__ __forceinline__ long long at(int p) const { return p == 0 ? slot : 2 * (first + p); }
};
template <int N>
__device__ __forceinline__ Pieces pieces_of(const AttendArgs& a, const Run& run) {
  tc::pdl_wait();
  Pieces x;
  int item = blockIdx.x;
  const int4 m = run.meta[blockIdx.x];
  if (run.by_item) {                               // its rows are looked up beside its entry, not behind it
    x.s = seq_rows(a.m, item / a.tiles, a.rows, a.max_new);
    x.r0 = item % a.tiles * N;
  }
  // (an item without rows is nobody's, and has no entry)
  x.n = (run.by_item && x.r0 >= x.s.count * a.group) || m.x < 0 ? 0 : m.z - m.y + 1;
  x.slot = m.x, x.first = m.y;
  if (x.n > 0 && !run.by_item) {
    item = m.w;
    x.s = seq_rows(a.m, item / a.tiles, a.rows, a.max_new);
    x.r0 = item % a.tiles * N;
  }
  return x;
}
// a row's o and sum, with maximum top, and C further pieces of it; f: the scores' factor
template <int C, int D>
__device__ __forceinline__ void join_pieces(float f, float& top, float& sum, float (&o)[D], const float2 (&ml)[C], const float (&y)[C][D]) {
  float m = top;
#pragma unroll
  for (int i = 0; i < C; ++i) m = fmaxf(m, ml[i].x);
  const float ref = m == -INFINITY ? 0.f : m, down = ex2_approx((top - ref) * f);
  top = m;
  sum *= down;
#pragma unroll
  for (int e = 0; e < D; ++e) o[e] *= down;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const float g = ex2_approx((ml[i].x - ref) * f);
    sum = fmaf(ml[i].y, g, sum);
#pragma unroll
    for (int e = 0; e < D; ++e) o[e] = fmaf(y[i][e], g, o[e]);
  }
}

// RANK / 4 lanes a row, or several such groups that share its pieces.  The loads of several pieces, sums and statistics, are
// under way at once: a load's time is what bounds this kernel.
constexpr int JOIN_THREADS = 512;
template <typename T, int RANK, int N>
__global__ void __launch_bounds__(JOIN_THREADS, 1) latent_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Run run, int groups) {
  constexpr int LANES = RANK / 4, AT_ONCE = JOIN_THREADS / LANES;
  __shared__ float2 stat[AT_ONCE];
  __shared__ float4 os[AT_ONCE][LANES];
  const int at = threadIdx.x / LANES, lane = threadIdx.x % LANES, group = at % groups, row = at / groups;
  const int r = blockIdx.y * (AT_ONCE / groups) + row;
  const Pieces x = pieces_of<N>(a, run);
  if (x.n == 0) return;
  const int R = x.r0 + r;
  const bool on = r < N && R < x.s.count * a.group;
  const float f = factor_of(a);
  float top = -INFINITY, sum = 0.f, o[4] = {};
  if (on)
    for (int p0 = group; p0 < x.n; p0 += 8 * groups) {
      float2 ml[8];
      float y[8][4];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int p = p0 + i * groups;
        const long long at = x.at(p) * N + r;
        const bool there = p < x.n;
        ml[i] = there ? a.ml[at] : make_float2(-INFINITY, 0.f);
        const float4 v = there ? *reinterpret_cast<const float4*>(a.part + at * RANK + 4 * lane) : make_float4(0.f, 0.f, 0.f, 0.f);
        y[i][0] = v.x, y[i][1] = v.y, y[i][2] = v.z, y[i][3] = v.w;
      }
      join_pieces(f, top, sum, o, ml, y);
    }
  if (groups > 1) {
    os[at][lane] = make_float4(o[0], o[1], o[2], o[3]);
    if (lane == 0) stat[at] = make_float2(top, sum);
    __syncthreads();
    if (on && group == 0)
      for (int e = 1; e < groups; ++e) {
        const float4 v = os[at + e][lane];
        const float2 ml[1] = {stat[at + e]};
        const float y[1][4] = {{v.x, v.y, v.z, v.w}};
        join_pieces(f, top, sum, o, ml, y);
      }
  }
  if (!on || group != 0) return;
  store_out(static_cast<T*>(a.out) + (long long)(x.s.first + R / a.group) * a.ldo + (long long)(R % a.group) * RANK + 4 * lane,
            make_float4(o[0], o[1], o[2], o[3]), sum == 0.f ? 0.f : 1.f / sum);
}

// The same for items of 128 rows, whose pieces are [dimension][row]: a thread a row and 8 dimensions
template <int RANK>
__global__ void __launch_bounds__(256) latent_join_wide_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Run run) {
  const int r = threadIdx.x % 128, d = (blockIdx.y * 2 + threadIdx.x / 128) * 8;
  const Pieces x = pieces_of<128>(a, run);
  const int R = x.n == 0 ? 0 : x.r0 + r;
  if (x.n == 0 || R >= x.s.count * a.group) return;
  const float f = factor_of(a);
  float top = -INFINITY, sum = 0.f, o[8] = {};
  for (int p0 = 0; p0 < x.n; p0 += 4) {
    float2 ml[4];
    float y[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool there = p0 + i < x.n;
      ml[i] = there ? a.ml[x.at(p0 + i) * 128 + r] : make_float2(-INFINITY, 0.f);
      const float* part = a.part + (x.at(p0 + i) * RANK + d) * 128 + r;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[i][e] = there ? part[e * 128] : 0.f;
    }
    join_pieces(f, top, sum, o, ml, y);
  }
  const float norm = sum == 0.f ? 0.f : 1.f / sum;
  uint32_t v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[e]) : "f"(o[2 * e + 1] * norm), "f"(o[2 * e] * norm));
  *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + (long long)(x.s.first + R / a.group) * a.ldo + (long long)(R % a.group) * RANK + d) =
      make_uint4(v[0], v[1], v[2], v[3]);
}

// a launch whose kernel waits for the ones before it itself (griddepcontrol.wait)
struct Launch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[1];
  Launch(dim3 grid, int threads, int smem, cudaStream_t st) {
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cfg.stream = st;
    cfg.gridDim = grid;
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = smem;
  }
};
inline Run run_of_plan(const AttendArgs& a, const LatentPlan& p, int rows) {
  const int items = a.m.n_seq * a.tiles;
  return Run{items, p.splits > 1, 0, items < p.blocks, reinterpret_cast<int4*>(a.ml + 2 * p.blocks * rows)};
}

template <typename T, int RANK, int N>
cudaError_t launch_join_of(const AttendArgs& a, const LatentPlan& p, const Run& run, cudaStream_t st) {
  const int entries = std::min(run.items, p.blocks);
  if constexpr (N == 128) {
    Launch launch(dim3(entries, RANK / 16), 256, 0, st);
    return cudaLaunchKernelEx(&launch.cfg, latent_join_wide_kernel<RANK>, a, run);
  } else {
    constexpr int AT_ONCE = JOIN_THREADS / (RANK / 4);
    int groups = 1;
    while (groups < AT_ONCE && groups * 8 * run.items < p.blocks) groups *= 2;
    Launch launch(dim3(entries, (N * groups + AT_ONCE - 1) / AT_ONCE), JOIN_THREADS, 0, st);
    return cudaLaunchKernelEx(&launch.cfg, latent_join_kernel<T, RANK, N>, a, run, groups);
  }
}

// launches the bf16 kernel of items of N rows, and the join of those that blocks share
template <int RANK, int N, typename K>
cudaError_t launch_items(K kernel, int threads, int smem, const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  CUtensorMap map, queries;
  Run run = run_of_plan(a, p, N);
  run.flat = a.ldq == (long long)a.m.n_head * (RANK + LATENT_ROPE);
  if (!latent_map(&map, a.m, a.m.page_tokens)) return cudaErrorInvalidValue;
  queries = map;
  if (run.flat && !query_map(&queries, a, N)) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem(kernel, smem, done);
  if (e != cudaSuccess) return e;
  Launch launch(p.blocks, threads, smem, st);
  e = cudaLaunchKernelEx(&launch.cfg, kernel, a, map, queries, run);
  return e != cudaSuccess || !run.split ? e : launch_join_of<__nv_bfloat16, RANK, N>(a, p, run, st);
}

}  // namespace evo
