// Expansion of a latent memory to the keys and values of an ordinary paged one:
//   k_h = (W_k,h c | k'),   v_h = W_v,h c
// for every head h and token of a range, with c the token's latent and k' its rotated key part,
// written to the token's page of the other memory.
//
// bf16, on tcgen05: a block has one head's 192 products (rank 512, large pages: half of them; its maps stay in
// shared memory, 48 to 192 KB, and with 192 only two copies are on the way) and takes
// tiles of 128 tokens, whose latents arrive 64 dimensions at a time by tiled bulk copies.  The last warp looks tiles
// and pages up, for all, and brings the latents, the one before it issues the products into one of two accumulators,
// and eight warps each empty one of these, so that what a warp waits for (a tile's pages, tensor memory, room for
// its stores) is hidden by the others.  The output is 512 bytes a (token, head) against 2 rank
// that are read, mostly from L2, so the writes bound the kernel, and have to leave as whole lines: accumulators are read
// 16 tokens by 256 bits, four lanes a token, and the maps' rows stand in shared memory in the order that gives
// each of these lanes 8 products of its own in a row (a token a lane and 32 bytes a store were 32 lines an
// instruction: 101 us).  31,800 tokens of 16 heads, rank 256: 57 us, 4.9 TB/s of algorithmic bytes.
//
// fp32, on mma.sync: a number is split into two of 11 bits and a product taken as three of tf32 (evo_latent_f32.cu).
// A block has 32 tokens (16 where no sequence has more) and a head, a warp 48 of its 192 products; rows of 32
// dimensions of both arrive in a ring by asynchronous copies.  Two blocks a SM, so that one computes while the other starts
// or stores.  The matrix unit cuts its sums off: those of 32 dimensions are added in fp32 (906 tokens, rank 128: 3.3e-7 of the
// result, sums of fp32 multiply-adds 2.0e-7).  Rows stand in shared memory in
// the order that gives the lanes of a 16-byte load different banks, and each lane four products in a row of its tokens.
// The matrix unit bounds it, at three products each: 750 tokens of 64 heads, rank 256, 84 us, 56 TFLOP/s (one block of 64
// tokens a SM 100, fp32 multiply-adds 148); 68 x 2 tokens of 16 heads 38 us (in blocks of 64 tokens 122).
#include <algorithm>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_latent.cuh"

namespace evo {
namespace {

constexpr int BN = LATENT_KEY + LATENT_VALUE;        // products of a head

// tokens of sequence n that are written: [lo, hi); what does not fit the call reports itself and gives none
__device__ __forceinline__ int2 token_range(const LatentExpandArgs& a, int n) {
  const int hi = seq_len(a.m, n, a.max_len), lo = a.first ? a.first[n] : 0;
  if (lo < 0 || lo > hi || hi - lo > a.max_new || hi > a.to.max_pages * a.to.page_tokens) {
    memory_fault(a.m);
    return make_int2(0, 0);
  }
  return make_int2(lo, hi);
}
// page i of a sequence in one of the memories, or -1 where the entry is outside the pool
__device__ __forceinline__ int page_or_none(const evo_memory& m, int32_t* status, int n, int i) {
  const int p = m.table[(long long)n * m.max_pages + i];
  if ((unsigned)p < (unsigned)m.n_pages) return p;
  if (status) *status = EVO_ERR_CORRUPT;
  return -1;
}

// ---------------------------------------------------------------- bf16

constexpr int TM = 128, STAGE = TM * 128;          // tokens of a tile; bytes of 64 of their dimensions
template <int RANK, int PARTS>
struct Cfg {
  static constexpr int N = BN / PARTS, WRITERS = 16 / PARTS, THREADS = 32 * (WRITERS + 2);
  static constexpr int CHUNKS = RANK / 64, CHUNK = N * 128, W = CHUNKS * CHUNK;   // bytes of 64 dimensions of the maps, of all
  static constexpr int ROOM = (227 * 1024 - 2048 - W) / STAGE, STAGES = ROOM > 8 ? 8 : ROOM;
  static constexpr int SMEM = 1024 + W + STAGES * STAGE;
  static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(TM >> 4) << 24);
};
constexpr int INFOS = 4;                           // tiles that are looked up ahead
struct Info {
  int n, t0, lo, hi;              // sequence; the tile's tokens t0 .. t0 + 127, of which lo .. hi - 1 are written; n < 0: no more
  int from[8], to[8];             // pages of its tokens in either memory, -1: outside the pool
};
struct Shared {
  uint64_t full[8], empty[8], w_full, acc_full[2], acc_empty[2], info_full[INFOS], info_empty[INFOS];
  Info info[INFOS];
  uint32_t tmem;
  int dead;
};

// 32 columns of 16 lanes: of column 8 k + 2 c + e, lane (g, c) gets that of TMEM lane g in v[4 k + e] and of g + 8 in v[4 k + 2 + e]
__device__ __forceinline__ void tmem_ld16x32(uint32_t taddr, float (&v)[16]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ uint32_t pair_of(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// the product (0 .. 63 of the key, 64 .. of the value) that stands in column p of the accumulator: a lane's 8 in a row
__device__ __forceinline__ int product_of(int p) { return p & ~31 | (p & 6) << 2 | (p & 24) >> 2 | (p & 1); }

template <int RANK, int PARTS>
__global__ void __launch_bounds__(Cfg<RANK, PARTS>::THREADS, 1)
    latent_expand_tiles_kernel(const __grid_constant__ LatentExpandArgs a, const __grid_constant__ CUtensorMap map, int pairs, int groups) {
  using C = Cfg<RANK, PARTS>;
  constexpr int WRITERS = C::WRITERS, CHUNK = C::CHUNK;
  extern __shared__ uint8_t raw[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, H = a.to.n_kv_head, h = blockIdx.x / PARTS % H, half = blockIdx.x % PARTS;
  uint8_t* const maps = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  uint8_t* const ring = maps + C::W;
  if (tid == 0) fetch_map(&map);
  __syncwarp();                                              // a whole warp's instruction, behind one lane's prefetch
  if (warp == 0) tc::tmem_alloc(&sh.tmem, 512);
  if (tid == 32) {
    for (int i = 0; i < C::STAGES; ++i) tc::mbar_init1(&sh.full[i], 1), tc::mbar_init1(&sh.empty[i], 1);
    tc::mbar_init1(&sh.w_full, WRITERS + 1);                 // a warp each
    for (int i = 0; i < 2; ++i) tc::mbar_init1(&sh.acc_full[i], 1), tc::mbar_init1(&sh.acc_empty[i], WRITERS / 2);
    for (int i = 0; i < INFOS; ++i) tc::mbar_init1(&sh.info_full[i], 1), tc::mbar_init1(&sh.info_empty[i], WRITERS / 2 + 1);
    sh.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;
  tc::pdl_wait();                                            // what earlier kernels wrote is there

  if (warp == WRITERS + 1) {
    // ------------------------------------------------------------ tiles, pages and copies
    // The block's tiles: of pairs (tile, sequence), sequences first, every groups-th.  Tiles start at multiples of 128
    // tokens, so that pages fit them
    const int page_tokens = a.m.page_tokens, to_tokens = a.to.page_tokens, box = min(page_tokens, TM);
    const int l = lane % 8, size = lane < 8 ? page_tokens : to_tokens;   // lanes 0 .. 7: the latents' pages; 8 .. 15: the other memory's
    int index = 0, i = 0;
    const auto publish = [&](int n, int t0, int lo, int hi, int page) {
      Info& info = sh.info[i % INFOS];
      if (i >= INFOS && !__all_sync(0xffffffffu, wait_for(&sh.info_empty[i % INFOS], (i / INFOS - 1) & 1, &sh.dead))) return;
      if (lane < 8) info.from[l] = page;
      else if (lane < 16) info.to[l] = page;
      if (lane == 0) info.n = n, info.t0 = t0, info.lo = lo, info.hi = hi;
      __syncwarp();
      if (lane == 0) tc::mbar_arrive1(&sh.info_full[i % INFOS]);
      ++i;
    };
    // a lane a tile: 32 ranges are looked up at once, and pages a tile ahead of their use
    for (long long pair0 = blockIdx.x / (PARTS * H); pair0 < pairs; pair0 += 32ll * groups) {
      const long long pair = pair0 + (long long)lane * groups;
      int2 range = make_int2(0, 0);
      int my_t0 = 0;
      if (pair < pairs) {
        range = token_range(a, (int)(pair % a.m.n_seq));
        my_t0 = range.x / TM * TM + (int)(pair / a.m.n_seq) * TM;
      }
      uint32_t left = __ballot_sync(0xffffffffu, my_t0 < range.y);
      struct Ahead { int n, t0, lo, hi, entry; bool on; } next;
      const auto look_up = [&] {                             // the entry is looked at when the tile's turn comes
        const int from = left ? __ffs(left) - 1 : 0;
        next.n = (int)((pair0 + (long long)from * groups) % a.m.n_seq);
        next.t0 = __shfl_sync(0xffffffffu, my_t0, from);
        next.lo = __shfl_sync(0xffffffffu, range.x, from);
        next.hi = __shfl_sync(0xffffffffu, range.y, from);
        const int t = next.t0 + l * size;
        next.on = left && lane < 16 && l * size < TM && t + size > next.lo && t < next.hi;
        const evo_memory& m = lane < 8 ? a.m : a.to;
        next.entry = next.on ? m.table[(long long)next.n * m.max_pages + t / size] : 0;
      };
      look_up();
      while (left) {
        const Ahead now = next;
        left &= left - 1;
        if (left) look_up();
        int page = now.on ? now.entry : -1;
        if (now.on && (unsigned)page >= (unsigned)(lane < 8 ? a.m.n_pages : a.to.n_pages)) page = -1, memory_fault(a.m);
        publish(now.n, now.t0, now.lo, now.hi, page);
        const bool on = lane < 8 && page >= 0;
        const int copies = __popc(__ballot_sync(0xffffffffu, on)), row = page * page_tokens + ((now.t0 + l * size) & (page_tokens - 1));
        for (int c = 0; c < C::CHUNKS; ++c, ++index) {
          const int slot = index % C::STAGES, use = index / C::STAGES;
          if (!__all_sync(0xffffffffu, use == 0 || wait_for(&sh.empty[slot], (use - 1) & 1, &sh.dead))) continue;
          if (lane == 0) tc::mbar_expect_tx(&sh.full[slot], copies * box * 128);
          __syncwarp();
          if (on) tile_load(tc::su32(ring + slot * STAGE + lane * box * 128), &map, 64 * c, row, tc::su32(&sh.full[slot]));
          __syncwarp();
        }
      }
    }
    publish(-1, 0, 0, 0, -1);                                // no more, for the writers of even and of odd tiles
    publish(-1, 0, 0, 0, -1);
  } else {
    // the head's maps, 16 bytes a copy
    constexpr int PIECES = RANK / 8;
#pragma unroll 4
    for (int i = tid; i < C::N * PIECES; i += C::THREADS - 32) {
      const int p = i / PIECES, j = i % PIECES, o = product_of(half * C::N + p);
      const __nv_bfloat16* src = (o < LATENT_KEY ? static_cast<const __nv_bfloat16*>(a.w_k) + ((long long)h * LATENT_KEY + o) * RANK
                                                 : static_cast<const __nv_bfloat16*>(a.w_v) + ((long long)h * LATENT_VALUE + o - LATENT_KEY) * RANK) + 8 * j;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::su32(maps + j / 8 * CHUNK + p * 128 + ((j % 8 ^ (p & 7)) << 4))), "l"(src)
                   : "memory");
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    tc::fence_async_smem();
    __syncwarp();
    if (lane == 0) tc::mbar_arrive1(&sh.w_full);
    // the i-th tile's info; false: there is none, or a wait was in vain
    const auto info_of = [&](int i, Info& info) {
      const bool ok = __all_sync(0xffffffffu, wait_for(&sh.info_full[i % INFOS], (i / INFOS) & 1, &sh.dead));
      if (ok) info = sh.info[i % INFOS];
      return ok && info.n >= 0;
    };
    const auto done_with = [&](int i) {
      __syncwarp();
      if (lane == 0) tc::mbar_arrive1(&sh.info_empty[i % INFOS]);
    };
    Info info;
    if (warp == WRITERS) {
      // ---------------------------------------------------------- products
      // (uniform over the warp and known to the compiler to be: descriptors stay in uniform registers)
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), dead = tc::su32(&sh.dead), full = tc::su32(sh.full), empty = tc::su32(sh.empty);
      const uint64_t desc = tc::sw128_desc(0);
      const uint32_t hi = (uint32_t)(desc >> 32), x0 = (uint32_t)desc + (tc::su32(ring) >> 4), w = (uint32_t)desc + (tc::su32(maps) >> 4);
      const auto wait = [&](uint32_t bar, uint32_t parity) {
        if (!tc::mbar_test(bar, parity)) wait_slow(bar, parity, dead);
      };
      wait(tc::su32(&sh.w_full), 0);
      uint32_t slot = 0, phase = 0;
      for (int i = 0; info_of(i, info); ++i) {
        done_with(i);
        if (i >= 2) wait(tc::su32(&sh.acc_empty[i & 1]), (i / 2 - 1) & 1);
        if (__any_sync(0xffffffffu, tc::block_dead(dead))) break;
        const uint32_t d = tm + 256 * (i & 1);
#pragma unroll
        for (uint32_t c = 0; c < C::CHUNKS; ++c) {
          wait(full + 8 * slot, phase);
          tc::tc_fence_after();
          const uint32_t x = x0 + slot * (STAGE >> 4);
          if (tc::elect_one()) {
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k)
              tc::mma_f16(d, desc64(x + 2 * k, hi), desc64(w + c * (CHUNK >> 4) + 2 * k, hi), C::IDESC, c | k);
            commit(empty + 8 * slot);
            if (c == C::CHUNKS - 1) commit(tc::su32(&sh.acc_full[i & 1]));
          }
          if (++slot == C::STAGES) slot = 0, phase ^= 1;
        }
      }
    } else {
      // ---------------------------------------------------------- 96 columns of 32 tokens: warps 0-3 the key and a quarter of
      // the value, and the rotated half of the key; warps 4-7 the rest (rank 512: the other block does);
      // the second half of the warps the same of every second tile.
      // Lane (g, c) has tokens g, g + 8, .. and of each 32 products the 8 from 8 c on
      const bool second = PARTS == 1 ? warp / 4 % 2 : half;
      const int g = lane / 4, c = lane % 4, shift = 31 - __clz(a.m.page_tokens), to_shift = 31 - __clz(a.to.page_tokens);
      __nv_bfloat16* const keys = static_cast<__nv_bfloat16*>(a.to.k_pages) + 8 * c;
      __nv_bfloat16* const values = static_cast<__nv_bfloat16*>(a.to.v_pages) + 8 * c;
      const __nv_bfloat16* const pool = static_cast<const __nv_bfloat16*>(a.m.k_pages) + RANK + 8 * c;
      for (int i = warp / (WRITERS / 2); info_of(i, info); i += 2) {
        long long to[4];                                     // a token's row of either pool, -1: none
        uint4 turned[4][2];                                  // the rotated half of a key
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int y = 32 * (warp % 4) + 8 * j + g, t = info.t0 + y;
          const int p = sh.info[i % INFOS].from[y >> shift], q = sh.info[i % INFOS].to[y >> to_shift];
          to[j] = -1;
          if (t >= info.lo && t < info.hi && p >= 0 && q >= 0) {
            to[j] = ((((long long)q * H + h) << to_shift) + (t & (a.to.page_tokens - 1))) * 128;
            if (!second) {
              const uint4* src = reinterpret_cast<const uint4*>(pool + (((long long)p << shift) + (t & (a.m.page_tokens - 1))) * (RANK + LATENT_ROPE));
              turned[j][0] = src[0], turned[j][1] = src[4];
            }
          }
        }
        done_with(i);
        wait_for(&sh.acc_full[i & 1], (i / 2) & 1, &sh.dead);
        __syncwarp();
        tc::tc_fence_after();
#pragma unroll
        for (int x = 0; x < 3; ++x) {
          __nv_bfloat16* const out = second ? values + 32 * (x + 1) : x < 2 ? keys + 32 * x : values;
#pragma unroll
          for (int y = 0; y < 2; ++y) {                      // 16 lanes each
            float v[16];
            __syncwarp();                                    // whole warps before a collective load
            tmem_ld16x32(tmem + 256 * (i & 1) + (PARTS == 1 && second ? 96 : 0) + 32 * x + ((uint32_t)(32 * (warp % 4) + 16 * y) << 16), v);
#pragma unroll
            for (int z = 0; z < 2; ++z)
              if (to[2 * y + z] >= 0)
                *reinterpret_cast<uint4*>(out + to[2 * y + z]) =
                    make_uint4(pair_of(v[2 * z], v[2 * z + 1]), pair_of(v[4 + 2 * z], v[5 + 2 * z]), pair_of(v[8 + 2 * z], v[9 + 2 * z]),
                               pair_of(v[12 + 2 * z], v[13 + 2 * z]));
          }
        }
        __syncwarp();
        tc::tc_fence_before();
        if (lane == 0) tc::mbar_arrive1(&sh.acc_empty[i & 1]);
        if (!second)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (to[j] >= 0) {
              uint4* p = reinterpret_cast<uint4*>(keys + to[j] + LATENT_KEY);
              p[0] = turned[j][0], p[4] = turned[j][1];
            }
      }
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (sh.dead) {                                             // a wait was in vain: what is in flight lands first
    settle(a.m.status);
    __syncthreads();
  }
  if (warp == 0) tc::tmem_dealloc(tmem, 512);
}

template <int RANK, int PARTS>
cudaError_t launch_tiles(const LatentExpandArgs& a, cudaStream_t st) {
  using C = Cfg<RANK, PARTS>;
  CUtensorMap map;
  if (!latent_map(&map, a.m, a.m.page_tokens)) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(latent_expand_tiles_kernel<RANK, PARTS>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  const int pairs = a.m.n_seq * (a.max_new / TM + 2);        // a range may begin and end within a tile
  const int units = a.to.n_kv_head * PARTS, groups = std::max(1, std::min(pairs, 152 / units));
  Launch launch(groups * units, C::THREADS, C::SMEM, st);
  return cudaLaunchKernelEx(&launch.cfg, latent_expand_tiles_kernel<RANK, PARTS>, a, map, pairs, groups);
}

// ---------------------------------------------------------------- fp32

// BM tokens a block; a stage is 32 dimensions of its rows, of which two or three are on the way while one is used
template <int BM>
struct F32Cfg {
  static constexpr int MT = BM / 16, THREADS = 128, STAGES = BM == 16 ? 4 : 3;
  static constexpr int STAGE = (BM + BN) * 128, SMEM = 1024 + STAGES * STAGE;
  static constexpr int COPIES = (BM + BN) * 8 / THREADS, TOKENS = BM * 8 / THREADS;   // 16 bytes each, of a thread; those of tokens
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
// the place of row n of 8 of a fragment: those that the 8 lanes of a load's phase have are 4 rows apart
__device__ __forceinline__ int place8(int n) { return n / 2 + 4 * (n % 2); }
// the place of product p of 16: column 2 c + e of tile t is 4 c + 2 t + e
__device__ __forceinline__ int place16(int p) { return 8 * (p / 2 % 2) + place8(p / 4 * 2 + p % 2); }

// <x, w>, whatever they hold
__device__ __forceinline__ float plain_product(const float* x, const float* w, int n) {
  double sum = 0.;
#pragma unroll 1
  for (int i = 0; i < n; ++i) sum = fma((double)x[i], (double)w[i], sum);
  return (float)sum;
}

template <int BM>
__global__ void __launch_bounds__(F32Cfg<BM>::THREADS, 2) latent_expand_kernel(const __grid_constant__ LatentExpandArgs a, int tiles) {
  using C = F32Cfg<BM>;
  constexpr int THREADS = C::THREADS, MT = C::MT, COPIES = C::COPIES, TOKENS = C::TOKENS;
  extern __shared__ uint8_t raw[];
  __shared__ long long from_row[BM], to_row[BM];             // rows of the pools; -1: none
  const int tid = threadIdx.x, H = a.to.n_kv_head, rank = a.m.head_dim;
  const int h = blockIdx.x % H, tile = blockIdx.x / H % tiles, n = blockIdx.x / H / tiles;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  tc::pdl_wait();                                            // what earlier kernels wrote is there
  const int2 range = token_range(a, n);
  const int t0 = range.x + tile * BM;
  if (t0 >= range.y) return;
  if (tid < BM) {
    const int t = t0 + tid;
    long long from = -1, to = -1;
    if (t < range.y) {
      const int p = page_or_none(a.m, a.m.status, n, t / a.m.page_tokens), q = page_or_none(a.to, a.m.status, n, t / a.to.page_tokens);
      if (p >= 0 && q >= 0) {
        from = (long long)p * a.m.page_tokens + t % a.m.page_tokens;
        to = ((long long)q * H + h) * a.to.page_tokens + t % a.to.page_tokens;
      }
    }
    from_row[tid] = from;
    to_row[tid] = to;
  }
  __syncthreads();
  const float* const pool = static_cast<const float*>(a.m.k_pages);
  float* const keys = static_cast<float*>(a.to.k_pages);
  float* const values = static_cast<float*>(a.to.v_pages);
  const int row = rank + LATENT_ROPE, chunks = rank / 32;
  // copies: a thread has 16 bytes of its tokens and products in every chunk (tokens that are not there: zeros)
  const int piece = tid % 8, y0 = tid / 8;
  const float* src[COPIES];
  uint32_t dst[COPIES];
  bool none[TOKENS];
#pragma unroll
  for (int i = 0; i < COPIES; ++i) {
    const int y = y0 + THREADS / 8 * (i < TOKENS ? i : i - TOKENS), at = i < TOKENS ? (y & ~7) + place8(y & 7) : BM + (y & ~15) + place16(y & 15);
    src[i] = i < TOKENS ? pool + max(from_row[y], 0ll) * row
                        : (y < LATENT_KEY ? static_cast<const float*>(a.w_k) + ((long long)h * LATENT_KEY + y) * rank
                                          : static_cast<const float*>(a.w_v) + ((long long)h * LATENT_VALUE + y - LATENT_KEY) * rank);
    src[i] += 4 * piece;
    dst[i] = tc::su32(mem) + at * 128 + ((piece ^ (at & 7)) << 4);
    if (i < TOKENS) none[i] = from_row[y] < 0;
  }
  const auto bring = [&](int k) {
    if (k < chunks)
#pragma unroll
      for (int i = 0; i < COPIES; ++i)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst[i] + k % C::STAGES * C::STAGE), "l"(src[i] + 32 * k),
                     "r"(i < TOKENS && none[i < TOKENS ? i : 0] ? 0 : 16)
                     : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int k = 0; k < C::STAGES - 1; ++k) bring(k);
  for (int i = tid; i < BM * 16; i += THREADS) {             // the rotated half of the keys
    const int y = i / 16, e = i % 16 * 4;
    if (to_row[y] >= 0) *reinterpret_cast<float4*>(keys + to_row[y] * 128 + LATENT_KEY + e) = *reinterpret_cast<const float4*>(pool + from_row[y] * row + rank + e);
  }
  const int warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4;
  const int at = place8(g);
  float sum[MT][6][4] = {};                                  // tokens 16 i x columns 8 j of the warp's 48
  for (int k = 0; k < chunks; ++k) {
    asm volatile("cp.async.wait_group %0;" ::"n"(C::STAGES - 2) : "memory");
    __syncthreads();                                         // the chunk is there for all, and the one before is read
    bring(k + C::STAGES - 1);
    const uint32_t x = tc::su32(mem) + k % C::STAGES * C::STAGE, w = x + (BM + 48 * warp) * 128;
    float part[MT][6][4] = {};
#pragma unroll
    for (int u = 0; u < 2; ++u) {                            // 16 dimensions: two steps, 4 of them in a lane
      uint32_t hi[MT][2][4], lo[MT][2][4];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const float4 p = lds_f4(x + (16 * i + at) * 128 + (((4 * u + c) ^ at) << 4));
        const float4 q = lds_f4(x + (16 * i + 8 + at) * 128 + (((4 * u + c) ^ at) << 4));
        split(p.x, hi[i][0][0], lo[i][0][0]), split(q.x, hi[i][0][1], lo[i][0][1]), split(p.y, hi[i][0][2], lo[i][0][2]), split(q.y, hi[i][0][3], lo[i][0][3]);
        split(p.z, hi[i][1][0], lo[i][1][0]), split(q.z, hi[i][1][1], lo[i][1][1]), split(p.w, hi[i][1][2], lo[i][1][2]), split(q.w, hi[i][1][3], lo[i][1][3]);
      }
#pragma unroll
      for (int j = 0; j < 6; ++j) {
        const float4 p = lds_f4(w + (8 * j + at) * 128 + (((4 * u + c) ^ at) << 4));
        uint4 bh, bl;
        split(p.x, bh.x, bl.x), split(p.y, bh.y, bl.y), split(p.z, bh.z, bl.z), split(p.w, bh.w, bl.w);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          mma8(part[i][j], hi[i][0], bh.x, bh.y);
          mma8(part[i][j], hi[i][1], bh.z, bh.w);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          mma8(part[i][j], lo[i][0], bh.x, bh.y);
          mma8(part[i][j], lo[i][1], bh.z, bh.w);
          mma8(part[i][j], hi[i][0], bl.x, bl.y);
          mma8(part[i][j], hi[i][1], bl.z, bl.w);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 6; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[i][j][e] += part[i][j][e];
  }
  const auto out_of = [&](long long to, int o) { return o < LATENT_KEY ? keys + to * 128 + o : values + to * 128 + o - LATENT_KEY; };
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {                         // token 8 i + g: of each two tiles four products
    const long long to = to_row[8 * i + g];
    if (to < 0) continue;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const int o = 48 * warp + 16 * j + 4 * c, b = 2 * (i % 2);
      const float4 v = make_float4(sum[i / 2][2 * j][b], sum[i / 2][2 * j][b + 1], sum[i / 2][2 * j + 1][b], sum[i / 2][2 * j + 1][b + 1]);
      *reinterpret_cast<float4*>(out_of(to, o)) = v;
      odd |= !isfinite(v.x) || !isfinite(v.y) || !isfinite(v.z) || !isfinite(v.w);
    }
  }
  // An infinite number, one from 2^128 - 2^116 on (its high part is infinite) and a NaN make parts that are no numbers, and so
  // every sum with one of them: such sums are done again as they are written down (by the thread that stored them; never
  // where all is finite)
  if (odd)
#pragma unroll 1
    for (int i = 0; i < 6 * MT; ++i) {
      const int y = 8 * (i / 3) + g, o = 48 * warp + 16 * (i % 3) + 4 * c;
      if (to_row[y] < 0) continue;
      float* const out = out_of(to_row[y], o);
      const float* const token = pool + from_row[y] * row;
      const float* const map = o < LATENT_KEY ? static_cast<const float*>(a.w_k) + ((long long)h * LATENT_KEY + o) * rank
                                              : static_cast<const float*>(a.w_v) + ((long long)h * LATENT_VALUE + o - LATENT_KEY) * rank;
#pragma unroll 1
      for (int e = 0; e < 4; ++e)
        if (!isfinite(out[e])) out[e] = plain_product(token, map + (long long)e * rank, rank);
    }
}

template <int BM>
cudaError_t launch_f32(const LatentExpandArgs& a, cudaStream_t st) {
  using C = F32Cfg<BM>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(latent_expand_kernel<BM>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  const int tiles = (a.max_new + BM - 1) / BM;
  Launch launch((unsigned)((long long)a.m.n_seq * tiles * a.to.n_kv_head), C::THREADS, C::SMEM, st);
  return cudaLaunchKernelEx(&launch.cfg, latent_expand_kernel<BM>, a, tiles);
}

}  // namespace

cudaError_t launch_latent_expand(const LatentExpandArgs& a, cudaStream_t st) {
  if (a.m.dtype == EVO_DTYPE_F32) return a.max_new <= 16 ? launch_f32<16>(a, st) : launch_f32<32>(a, st);
  if (a.m.head_dim == 128) return launch_tiles<128, 1>(a, st);
  if (a.m.head_dim == 256) return launch_tiles<256, 1>(a, st);
  // two blocks a head bring every tile twice: not where it comes in many small copies (4 x 2,000 tokens of 20 heads, one
  // against two: pages of 128 53.2 / 46.0 us, of 32 54.1 / 57.1, of 16 56.8 / 73.7)
  return a.m.page_tokens >= 64 ? launch_tiles<512, 2>(a, st) : launch_tiles<512, 1>(a, st);
}

}  // namespace evo
