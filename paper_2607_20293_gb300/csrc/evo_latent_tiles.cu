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
// Blocks stay resident, one a SM.  Where items do not fill them evenly, the tiles of all items are counted
// (every block does so, by itself) and each block takes an equal run of them, so that sequences of different
// lengths end at the same time; the runs' first and last items are shared with other blocks, leave
// their sums in the workspace and are joined by a second kernel.  The copies run ahead into the next item
// while the softmax still writes this one's output.
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

#include "evo_attend.cuh"
#include "evo_mem_ptx.cuh"

namespace evo {
namespace {

constexpr int BK = 128;                            // tokens of a tile
constexpr int SMS = 152, MOST_ITEMS = 2048;        // items that a block counts
constexpr int SLOT = BK * 256, HALF = BK * 128;    // bytes of 128 and of 64 dimensions of a tile
constexpr float LAZY = 8.f;                        // log2 of how far a weight may pass 1
constexpr float NONE = -3.402823466e38f;           // the reference of a row that has seen nothing

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

// An item's rows and the tokens that they see
struct Item {
  Tile t;
  int rows, r0, last;             // rows of the sequence; the item's are r0 .. last
  Range first_row, last_row, all;
  int tile0, tiles;               // tiles of 128 tokens that some row sees
  // (an item without any is written as zeros, and counts as a tile)
  __device__ __forceinline__ int cost() const { return r0 >= rows ? 0 : max(1, tiles); }
};
// what the softmax's warps have to know of one item, or of what this block has of it
struct Segment {
  Item x;
  int more, n, key0, slot, whole; // more: there is one.  n tiles from token key0 on; slot: of its sums, unless it is whole here
  bool alike;                     // every row sees the same tokens
};

template <int N>
struct Shared {
  uint64_t full[6], empty[6], part_full[6], part_empty[6], s_full[2], p_full, o_full, q_full;
  __align__(16) float ref[N];                      // what is subtracted from a row's scores
  int top[N];                                      // a new maximum (ordered as integers), then the factor of what was summed
  uint32_t bad[4];
  uint32_t tmem;
  int dead, item, skip;                            // the first item's number, and the tiles of it that others take
  int tiles, warp_tiles[32];                       // tiles that the block takes; sums of the warps' items
  Segment seg[2];
  Item begin;                                      // the block's first item
  long long to[N];                                 // where a row's output begins
};

struct Run {
  int items, split;                                // split: blocks take equal runs of tiles; else whole items, every gridDim-th
  int4* meta;                                      // of each block from which an item goes on to others: its piece's slot (else -1), the last block, the item
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
__device__ __noinline__ void wait_slow(uint32_t bar, uint32_t parity, uint32_t dead) { wait_live(bar, parity, dead); }
__device__ __forceinline__ uint64_t desc64(uint32_t lo, uint32_t hi) { return ((uint64_t)hi << 32) | lo; }
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
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
      const int cost = x.cost();
      if (cost == 0) continue;
      index = item;
      from = skip;
      const int take = min(cost - skip, left);
      n = x.tiles == 0 ? 0 : take;
      after = cost - from - take;
      if (run.split) left -= take;
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

template <int RANK, int N>
__global__ void __launch_bounds__(Cfg<RANK, N>::THREADS, 1)
    latent_tiles_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map, const __grid_constant__ Run run) {
  using C = Cfg<RANK, N>;
  constexpr int PER = C::PER, HC = C::HC, SLOTS = C::SLOTS, PARTS = C::PARTS, SOFTMAX = C::SOFTMAX, THREADS = C::THREADS;
  extern __shared__ uint8_t raw[];
  __shared__ Shared<N> sh;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  uint8_t* const weights = mem + C::Q;
  uint8_t* const ring = weights + C::P;
  uint8_t* const parts = ring + SLOTS * SLOT;
  if (tid == 0) fetch_map(&map);
  __syncwarp();                                    // a whole warp's instruction, behind one lane's prefetch
  if (warp == 0) tc::tmem_alloc(&sh.tmem, C::ALLOC);
  if (tid == 32) {
    for (int i = 0; i < SLOTS; ++i) tc::mbar_init1(&sh.full[i], 1), tc::mbar_init1(&sh.empty[i], 1);
    for (int i = 0; i < PARTS; ++i) tc::mbar_init1(&sh.part_full[i], 1), tc::mbar_init1(&sh.part_empty[i], 1);
    tc::mbar_init1(&sh.s_full[0], 1), tc::mbar_init1(&sh.s_full[1], 1);
    tc::mbar_init1(&sh.p_full, C::WARPS);          // a warp each
    tc::mbar_init1(&sh.q_full, C::WARPS);
    tc::mbar_init1(&sh.o_full, 1);
    sh.dead = 0;
    sh.item = run.split ? run.items : blockIdx.x;
    sh.skip = 0;
    sh.tiles = run.split ? 0 : INT_MAX;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < N) sh.ref[tid] = NONE;
  tc::pdl_wait();                                  // what earlier kernels wrote is there
  if (run.split) tc::pdl_trigger();                // the join may take its places, and waits there
  int total = 0;
  int blocks = gridDim.x;                          // that take tiles
  if (!run.split) {
    if (tid == 0) sh.begin = item_of<N>(a, blockIdx.x);
  } else {
    // every thread counts the tiles of a few items; the block's run is the blockIdx-th of `blocks` equal ones
    const int each = (run.items + THREADS - 1) / THREADS, i0 = tid * each, i1 = min(i0 + each, run.items);
    Item x;
    if (i0 < i1) x = item_of<N>(a, i0);
    const int one = i0 < i1 ? x.cost() : 0;
    int mine = one;
    for (int i = i0 + 1; i < i1; ++i) mine += item_of<N>(a, i).cost();
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
      for (int cost = one; lo >= before + cost; cost = x.cost()) before += cost, x = item_of<N>(a, ++i);
      sh.begin = x;
      sh.item = i;
      sh.skip = lo - before;
      sh.tiles = hi - lo;
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;
  Walk<N> walk(a, run, sh);
  int g = 0;                                       // tiles so far

  if (warp == C::WARPS + 1) {
    // ------------------------------------------------------------ copies
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
        for (int j = 0; j < PER; ++j) {
          const int index = g * PER + j, slot = index % SLOTS;
          bring(ring + slot * SLOT, &sh.full[slot], &sh.empty[slot], index / SLOTS, 128 * j, 2);
        }
        bring(parts + g % PARTS * HALF, &sh.part_full[g % PARTS], &sh.part_empty[g % PARTS], g / PARTS, RANK, 1);
      }
    }
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
    const uint32_t s_full = tc::su32(sh.s_full), p_full = tc::su32(&sh.p_full), o_full = tc::su32(&sh.o_full);
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
    // the softmax works with a positive factor: the scale's sign goes to the scores
    const float f = a.scale_log2 == 0.f ? 1.f : fmaxf(fabsf(a.scale_log2), 1.1754944e-38f), far = fminf(LAZY / f, 1e38f);
    const float sign = a.scale_log2 < 0.f ? -1.f : a.scale_log2 == 0.f ? 0.f : 1.f;
    // an item's queries on their way to shared memory, and there
    const auto bring_queries = [&](const Item& x) {
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
    };
    const auto queries_there = [&] {
      asm volatile("cp.async.wait_all;" ::: "memory");
      tc::fence_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive1(&sh.q_full);
    };
    // the first warp looks the next item up for all of them
    bool shares = false;
    const auto look_up = [&](Segment& q) {
      bar_softmax<SOFTMAX>();                        // nobody is at the item before any more
      if (warp == 0) {
        const bool more = walk.next();
        if (lane == 0) {
          q.more = more;
          if (more) {
            const Item& x = walk.x;
            q.x = x;
            q.n = walk.n;
            q.key0 = walk.key0();
            q.slot = 2 * blockIdx.x + (walk.segments > 1 ? 1 : 0);   // of an item that other blocks share: the run's first or last
            q.whole = walk.from == 0 && walk.after == 0;
            q.alike = x.first_row.lo == x.last_row.lo && x.first_row.hi == x.last_row.hi;
            if (walk.from == 0 && walk.after > 0) {  // it goes on to the block that has the last of its tiles
              const int end = run_from(total, blocks, blockIdx.x + 1) + walk.after;
              run.meta[blockIdx.x] = make_int4(q.slot, block_of(total, blocks, end - 1), walk.index, 0);
              shares = true;
            }
          }
        }
      }
      bar_softmax<SOFTMAX>();
    };
    float sum[HC];
    look_up(sh.seg[0]);
    if (sh.seg[0].more && sh.seg[0].n > 0) bring_queries(sh.seg[0].x);
    for (int s = 0; sh.seg[s].more; s ^= 1) {
      const Segment& q = sh.seg[s];
      const Segment& after = sh.seg[s ^ 1];
      if (q.n > 0) queries_there();
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
            sh.top[tid] = __float_as_int(old == NONE ? 1.f : ex2_approx((old - m) * f));
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
        if (lane == 0) tc::mbar_arrive1(&sh.p_full);
      }
      // the next item's queries take the place of these, whose scores are all there
      if (after.more && after.n > 0) bring_queries(after.x);
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
          a.ml[q.slot * N + tid] = make_float2(sh.ref[tid] == NONE ? -INFINITY : sh.ref[tid] * f, l);
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
    if (run.split && tid == 0 && !shares) run.meta[blockIdx.x] = make_int4(-1, 0, 0, 0);
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

// Joins the pieces of the items that blocks share, from the block that has an item's first tile: its piece, and the
// first of each block behind it up to the last.  RANK / 4 lanes a row, or several such groups that share its pieces
// (few rows of many pieces would else wait out one load after the other).
constexpr int JOIN_THREADS = 512;
template <int RANK, int N>
__global__ void __launch_bounds__(JOIN_THREADS) latent_join_kernel(const __grid_constant__ AttendArgs a, const int4* meta, int groups) {
  constexpr int LANES = RANK / 4, AT_ONCE = JOIN_THREADS / LANES;
  __shared__ float weight[AT_ONCE][SMS];           // of a row's pieces
  __shared__ float total[AT_ONCE];
  __shared__ float4 os[AT_ONCE][LANES];
  const int at = threadIdx.x / LANES, lane = threadIdx.x % LANES, group = at % groups, row = at / groups;
  const int r = blockIdx.y * (AT_ONCE / groups) + row;
  tc::pdl_wait();
  const int4 m = meta[blockIdx.x];
  if (m.x < 0) return;
  const int n = m.z / a.tiles, pieces = m.y - blockIdx.x + 1;
  const SeqRows s = seq_rows(a.m, n, a.rows, a.max_new);
  const int R = m.z % a.tiles * N + r;
  const bool on = r < N && R < s.count * a.group;
  const auto place = [&](int p) { return (long long)(p == 0 ? m.x : 2 * (blockIdx.x + p)) * N + r; };
  if (on && group == 0 && lane < 32) {             // a warp a row: its pieces' weights
    float top = -INFINITY, sum = 0.f;
    for (int p = lane; p < pieces; p += 32) top = fmaxf(top, a.ml[place(p)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    for (int p = lane; p < pieces; p += 32) {
      const float2 ml = a.ml[place(p)];
      const float w = ex2_approx(ml.x - (top == -INFINITY ? 0.f : top));
      weight[row][p] = w;
      sum = fmaf(ml.y, w, sum);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) total[row] = sum;
  }
  __syncthreads();
  float4 o = {};
  if (on) {
#pragma unroll 8
    for (int p = group; p < pieces; p += groups) {
      const float4 y = *reinterpret_cast<const float4*>(a.part + place(p) * RANK + 4 * lane);
      const float w = weight[row][p];
      o = make_float4(fmaf(y.x, w, o.x), fmaf(y.y, w, o.y), fmaf(y.z, w, o.z), fmaf(y.w, w, o.w));
    }
  }
  if (groups > 1) {
    os[at][lane] = o;
    __syncthreads();
    if (group == 0)
      for (int e = 1; e < groups; ++e) {
        const float4 y = os[at + e][lane];
        o = make_float4(o.x + y.x, o.y + y.y, o.z + y.z, o.w + y.w);
      }
  }
  if (!on || group != 0) return;
  const float sum = total[row];
  store_out(static_cast<__nv_bfloat16*>(a.out) + (long long)(s.first + R / a.group) * a.ldo + (long long)(R % a.group) * RANK + 4 * lane, o,
            sum == 0.f ? 0.f : 1.f / sum);
}

template <int RANK, int N>
cudaError_t launch_as(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  using C = Cfg<RANK, N>;
  CUtensorMap map;
  if (!latent_map(&map, a.m, std::min(a.m.page_tokens, BK))) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem(latent_tiles_kernel<RANK, N>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  const Run run{a.m.n_seq * a.tiles, p.splits > 1, reinterpret_cast<int4*>(a.ml + 2 * p.blocks * N)};
  // both kernels wait for the ones before them themselves (griddepcontrol.wait)
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  cfg.stream = st;
  cfg.gridDim = p.blocks;
  cfg.blockDim = C::THREADS;
  cfg.dynamicSmemBytes = C::SMEM;
  e = cudaLaunchKernelEx(&cfg, latent_tiles_kernel<RANK, N>, a, map, run);
  if (e != cudaSuccess || !run.split) return e;
  constexpr int AT_ONCE = JOIN_THREADS / (RANK / 4);
  int groups = 1;
  while (groups < AT_ONCE && groups * 8 * run.items < p.blocks) groups *= 2;
  cfg.gridDim = dim3(p.blocks, (N * groups + AT_ONCE - 1) / AT_ONCE);
  cfg.blockDim = JOIN_THREADS;
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, latent_join_kernel<RANK, N>, a, (const int4*)run.meta, groups);
}
template <int RANK>
cudaError_t launch_of(const AttendArgs& a, const LatentPlan& p, cudaStream_t st) {
  if (p.tile_rows == 16) return launch_as<RANK, 16>(a, p, st);
  if constexpr (RANK < 512)
    if (p.tile_rows == 64) return launch_as<RANK, 64>(a, p, st);
  return launch_as<RANK, 32>(a, p, st);
}

}  // namespace

// Pieces: items go to the blocks whole where that takes little longer, in tiles, than equal runs and their join
void plan_latent_tiles(LatentPlan& p, const evo_memory& m, long long all, int keys) {
  p.tile_rows = all <= 16 ? 16 : all <= 32 || m.head_dim == 512 ? 32 : 64;
  p.tiles = (int)((all + p.tile_rows - 1) / p.tile_rows);
  const long long items = (long long)m.n_seq * p.tiles, tiles = std::max(1, (keys + BK - 1) / BK);
  const double whole = (double)((items + SMS - 1) / SMS) * (tiles + 2), even = (double)items * tiles / SMS + 3;
  const bool split = items <= MOST_ITEMS && tiles > 1 && items * (tiles + 1) < INT_MAX && even < whole;
  p.splits = split ? 2 : 1;
  p.blocks = (int)std::min<long long>(SMS, split ? items * tiles : items);
  // sums, and maximum and sum of weights, of two pieces a block; where a block's last item goes on
  p.scratch = split ? (size_t)p.blocks * (2 * p.tile_rows * ((size_t)m.head_dim + 2) * sizeof(float) + sizeof(int4)) : 0;
}

cudaError_t launch_latent_tiles(AttendArgs& a, const LatentPlan& p, void* scratch, cudaStream_t st) {
  a.part = static_cast<float*>(scratch);
  a.ml = reinterpret_cast<float2*>(a.part + (size_t)2 * p.blocks * p.tile_rows * a.m.head_dim);
  return a.m.head_dim == 128 ? launch_of<128>(a, p, st) : a.m.head_dim == 256 ? launch_of<256>(a, p, st) : launch_of<512>(a, p, st);
}

}  // namespace evo
