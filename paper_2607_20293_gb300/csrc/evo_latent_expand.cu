// Expansion of a latent memory to the keys and values of an ordinary paged one:
//   k_h = (W_k,h c | k'),   v_h = W_v,h c
// for every head h and token of a range, with c the token's latent and k' its rotated key part,
// written to the token's page of the other memory.
//
// bf16, on tcgen05: a block has one head's 192 products (its maps stay in shared memory: 48 to 192 KB) and takes
// tiles of 128 tokens, whose latents arrive 64 dimensions at a time by tiled bulk copies.  Warp 9 brings them, warp
// 8 issues the products into one of two accumulators, warps 0-7 empty the other: a thread has a token and
// either its key or its value, and writes whole 32-byte sectors of them.  The output is 512 bytes a
// (token, head) against 2 rank that are read, mostly from L2: what bounds the kernel is the writes.
//
// fp32: a block takes 64 tokens and the 192 products of a head, 16 of the rank at a time through shared
// memory; a thread has 8 tokens x 6 products in packed pairs of tokens.
#include <algorithm>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_mem_ptx.cuh"
#include "evo_rows.cuh"

namespace evo {
namespace {

constexpr int THREADS = 256, BM = 64, BN = LATENT_KEY + LATENT_VALUE, BK = 16;

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

__device__ __forceinline__ float4 four(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void put2(float* p, float2 v) { *reinterpret_cast<float2*>(p) = v; }

// ---------------------------------------------------------------- bf16

constexpr int TM = 128, TILE_THREADS = 320, STAGE = TM * 128, CHUNK = BN * 128;   // bytes of 64 dimensions of the tokens, of the maps
template <int RANK>
struct Cfg {
  static constexpr int CHUNKS = RANK / 64, W = CHUNKS * CHUNK;
  static constexpr int ROOM = (227 * 1024 - 2048 - W) / STAGE, STAGES = ROOM > 8 ? 8 : ROOM;
  static constexpr int SMEM = 1024 + W + STAGES * STAGE;
  static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(TM >> 4) << 24);
};
struct Shared {
  uint64_t full[8], empty[8], w_full, acc_full[2], acc_empty[2];
  uint32_t tmem;
  int dead;
};

__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, int* dead) {
  const uint32_t b = tc::su32(bar);
  return tc::mbar_test(b, parity) || wait_live(b, parity, tc::su32(dead));
}
// 16 values as bf16 to a 32-byte sector, or to two halves of 16 where rows start on these
__device__ __forceinline__ void put16(__nv_bfloat16* p, const uint32_t (&w)[8], bool whole) {
  if (whole) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

template <int RANK>
__global__ void __launch_bounds__(TILE_THREADS, 1)
    latent_expand_tiles_kernel(const __grid_constant__ LatentExpandArgs a, const __grid_constant__ CUtensorMap xmap,
                               const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, int pairs,
                               int groups) {
  using C = Cfg<RANK>;
  extern __shared__ uint8_t raw[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, H = a.to.n_kv_head, h = blockIdx.x % H, first = blockIdx.x / H;
  uint8_t* const maps = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  uint8_t* const ring = maps + C::W;
  if (warp == 0) tc::tmem_alloc(&sh.tmem, 512);
  if (tid == 32) {
    for (int i = 0; i < C::STAGES; ++i) tc::mbar_init1(&sh.full[i], 1), tc::mbar_init1(&sh.empty[i], 1);
    tc::mbar_init1(&sh.w_full, 1);
    for (int i = 0; i < 2; ++i) tc::mbar_init1(&sh.acc_full[i], 1), tc::mbar_init1(&sh.acc_empty[i], 8);   // a warp each
    sh.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;
  // The block's tiles: of pairs (tile, sequence), sequences first, every groups-th.  Tiles start at multiples of 128
  // tokens, so that pages fit them
  const auto tile_of = [&](int pair, int2& range) {
    const int n = pair % a.m.n_seq;
    range = token_range(a, n);
    return range.x / TM * TM + pair / a.m.n_seq * TM;
  };

  if (warp == 9) {
    // ------------------------------------------------------------ copies
    if (lane == 0) {
      tc::mbar_expect_tx(&sh.w_full, C::W);
      for (int c = 0; c < C::CHUNKS; ++c) {
        tile_load(tc::su32(maps + c * CHUNK), &kmap, 64 * c, h * LATENT_KEY, tc::su32(&sh.w_full));
        tile_load(tc::su32(maps + c * CHUNK + LATENT_KEY * 128), &vmap, 64 * c, h * LATENT_VALUE, tc::su32(&sh.w_full));
      }
    }
    __syncwarp();
    const int page_tokens = a.m.page_tokens, box = min(page_tokens, TM);
    int index = 0;
    for (int pair = first; pair < pairs; pair += groups) {
      int2 range;
      const int t0 = tile_of(pair, range);
      if (t0 >= range.y) continue;
      const int t = t0 + lane * box;
      int page = lane * box < TM && t + box > range.x && t < range.y ? page_or_none(a.m, a.m.status, pair % a.m.n_seq, t / page_tokens) : -1;
      const int copies = __popc(__ballot_sync(0xffffffffu, page >= 0));
      for (int c = 0; c < C::CHUNKS; ++c, ++index) {
        const int slot = index % C::STAGES, use = index / C::STAGES;
        if (!__all_sync(0xffffffffu, use == 0 || wait_for(&sh.empty[slot], (use - 1) & 1, &sh.dead))) continue;
        if (lane == 0) tc::mbar_expect_tx(&sh.full[slot], copies * box * 128);
        __syncwarp();
        if (page >= 0)
          tile_load(tc::su32(ring + slot * STAGE + lane * box * 128), &xmap, 64 * c, page * page_tokens + t % page_tokens,
                    tc::su32(&sh.full[slot]));
        __syncwarp();
      }
    }
  } else if (warp == 8) {
    // ------------------------------------------------------------ products
    wait_for(&sh.w_full, 0, &sh.dead);
    int index = 0, i = 0;
    for (int pair = first; pair < pairs; pair += groups) {
      int2 range;
      if (tile_of(pair, range) >= range.y) continue;
      if (i >= 2) wait_for(&sh.acc_empty[i & 1], (i / 2 - 1) & 1, &sh.dead);
      for (int c = 0; c < C::CHUNKS; ++c, ++index) {
        const int slot = index % C::STAGES;
        wait_for(&sh.full[slot], (index / C::STAGES) & 1, &sh.dead);
        tc::tc_fence_after();
        if (!tc::block_dead(tc::su32(&sh.dead)) && tc::elect_one()) {
          const uint32_t x = tc::su32(ring + slot * STAGE), w = tc::su32(maps + c * CHUNK);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            tc::mma_f16(tmem + 256 * (i & 1), tc::sw128_desc(x + 32 * k), tc::sw128_desc(w + 32 * k), C::IDESC, c | k);
          tc::mma_commit(&sh.empty[slot]);
          if (c == C::CHUNKS - 1) tc::mma_commit(&sh.acc_full[i & 1]);
        }
        __syncwarp();
      }
      ++i;
    }
  } else {
    // ------------------------------------------------------------ a token a thread: its key (warps 0-3) or its value
    const bool value = warp >= 4;
    __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(value ? a.to.v_pages : a.to.k_pages);
    const bool whole = reinterpret_cast<uintptr_t>(out) % 32 == 0;
    const uint32_t lanes = (uint32_t)(32 * (warp % 4)) << 16;
    // a thread's token: its row in either pool.  Looked up a tile ahead
    struct Token { long long from, to; };
    const auto next_of = [&](int pair, Token& token) {
      for (; pair < pairs; pair += groups) {
        int2 range;
        const int t0 = tile_of(pair, range), n = pair % a.m.n_seq, t = t0 + tid % TM;
        if (t0 >= range.y) continue;
        token = Token{-1, -1};
        if (t >= range.x && t < range.y) {
          const int p = page_or_none(a.m, a.m.status, n, t / a.m.page_tokens), q = page_or_none(a.to, a.m.status, n, t / a.to.page_tokens);
          if (p >= 0 && q >= 0)
            token = Token{(long long)p * a.m.page_tokens + t % a.m.page_tokens, ((long long)q * H + h) * a.to.page_tokens + t % a.to.page_tokens};
        }
        break;
      }
      return pair;
    };
    Token token;
    int pair = next_of(first, token);
    for (int i = 0; pair < pairs; ++i) {
      __nv_bfloat16* const dst = token.to >= 0 ? out + token.to * 128 : nullptr;
      uint32_t turned[4][8];                                 // the rotated half of a key
      if (dst && !value) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.m.k_pages) + token.from * (RANK + LATENT_ROPE) + RANK);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint4 u = src[j];
          uint32_t* w = &turned[j / 2][4 * (j % 2)];
          w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        }
      }
      pair = next_of(pair + groups, token);
      wait_for(&sh.acc_full[i & 1], (i / 2) & 1, &sh.dead);
      __syncwarp();
      tc::tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < (value ? 4 : 2); ++c) {
        float v[32];
        __syncwarp();                                        // whole warps before a collective load
        tc::tmem_ld32(tmem + 256 * (i & 1) + (value ? LATENT_KEY : 0) + 32 * c + lanes, v);
        if (!dst) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[16 * j + 2 * e], v[16 * j + 2 * e + 1]);
            w[e] = *reinterpret_cast<const uint32_t*>(&b);
          }
          put16(dst + 32 * c + 16 * j, w, whole);
        }
      }
      __syncwarp();
      tc::tc_fence_before();
      if (lane == 0) tc::mbar_arrive1(&sh.acc_empty[i & 1]);
      if (dst && !value)
#pragma unroll
        for (int j = 0; j < 4; ++j) put16(dst + LATENT_KEY + 16 * j, turned[j], whole);
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

template <int RANK>
cudaError_t launch_tiles(const LatentExpandArgs& a, cudaStream_t st) {
  using C = Cfg<RANK>;
  CUtensorMap x, k, v;
  if (!latent_map(&x, a.m, a.m.page_tokens) || !map_of(&k, a.w_k, (long long)a.m.n_head * LATENT_KEY, RANK, LATENT_KEY) ||
      !map_of(&v, a.w_v, (long long)a.m.n_head * LATENT_VALUE, RANK, LATENT_VALUE))
    return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(latent_expand_tiles_kernel<RANK>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  const int pairs = a.m.n_seq * (a.max_new / TM + 2);        // a range may begin and end within a tile
  const int groups = std::max(1, std::min(pairs, 152 / a.to.n_kv_head));
  latent_expand_tiles_kernel<RANK><<<groups * a.to.n_kv_head, TILE_THREADS, C::SMEM, st>>>(a, x, k, v, pairs, groups);
  return cudaGetLastError();
}

// ---------------------------------------------------------------- fp32

__global__ void __launch_bounds__(THREADS) latent_expand_kernel(const __grid_constant__ LatentExpandArgs a, int tiles) {
  __shared__ __align__(16) float as[BK][BM], bs[BK][BN];
  __shared__ long long from_row[BM], to_row[BM];             // rows of the pools; -1: none
  const int tid = threadIdx.x, H = a.to.n_kv_head, rank = a.m.head_dim;
  const int h = blockIdx.x % H, tile = blockIdx.x / H % tiles, n = blockIdx.x / H / tiles;
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
  const float* pool = static_cast<const float*>(a.m.k_pages);
  const int row = rank + LATENT_ROPE;
  // loads: a token's 4 values, and those of 3 products
  const int am = tid % BM, ak = tid / BM * 4;
  const float* asrc = from_row[am] >= 0 ? pool + from_row[am] * row + ak : nullptr;
  const float* bsrc[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int o = am + 64 * i;
    bsrc[i] = (o < LATENT_KEY ? static_cast<const float*>(a.w_k) + ((long long)h * LATENT_KEY + o) * rank
                              : static_cast<const float*>(a.w_v) + ((long long)h * LATENT_VALUE + o - LATENT_KEY) * rank) + ak;
  }
  float2 acc[4][6] = {};                                     // tokens 8 w + 2 i and the next x products 2 l + 64 j and the next
  const int lane = tid % 32, w = tid / 32;
  float4 av = asrc ? four(asrc) : make_float4(0.f, 0.f, 0.f, 0.f), bv[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) bv[i] = four(bsrc[i]);
  for (int k0 = 0; k0 < rank; k0 += BK) {
    as[ak][am] = av.x, as[ak + 1][am] = av.y, as[ak + 2][am] = av.z, as[ak + 3][am] = av.w;
#pragma unroll
    for (int i = 0; i < 3; ++i)
      bs[ak][am + 64 * i] = bv[i].x, bs[ak + 1][am + 64 * i] = bv[i].y, bs[ak + 2][am + 64 * i] = bv[i].z, bs[ak + 3][am + 64 * i] = bv[i].w;
    __syncthreads();
    if (k0 + BK < rank) {
      if (asrc) av = four(asrc + k0 + BK);
#pragma unroll
      for (int i = 0; i < 3; ++i) bv[i] = four(bsrc[i] + k0 + BK);
    }
#pragma unroll
    for (int k = 0; k < BK; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(&as[k][8 * w]), y = *reinterpret_cast<const float4*>(&as[k][8 * w + 4]);
      const float2 t2[4] = {make_float2(x.x, x.y), make_float2(x.z, x.w), make_float2(y.x, y.y), make_float2(y.z, y.w)};
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        const float2 b = *reinterpret_cast<const float2*>(&bs[k][2 * lane + 64 * j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[i][2 * j] = fma_pair(t2[i], make_float2(b.x, b.x), acc[i][2 * j]);
          acc[i][2 * j + 1] = fma_pair(t2[i], make_float2(b.y, b.y), acc[i][2 * j + 1]);
        }
      }
    }
    __syncthreads();
  }
  float* const kp = static_cast<float*>(a.to.k_pages);
  float* const vp = static_cast<float*>(a.to.v_pages);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long long to = to_row[8 * w + i], from = from_row[8 * w + i];
    if (to < 0) continue;
    const auto at = [&](int j) {
      return i % 2 ? make_float2(acc[i / 2][2 * j].y, acc[i / 2][2 * j + 1].y) : make_float2(acc[i / 2][2 * j].x, acc[i / 2][2 * j + 1].x);
    };
    put2(kp + to * 128 + 2 * lane, at(0));
    put2(vp + to * 128 + 2 * lane, at(1));
    put2(vp + to * 128 + 64 + 2 * lane, at(2));
    put2(kp + to * 128 + 64 + 2 * lane, *reinterpret_cast<const float2*>(pool + from * row + rank + 2 * lane));
  }
}

}  // namespace

cudaError_t launch_latent_expand(const LatentExpandArgs& a, cudaStream_t st) {
  if (a.m.dtype == EVO_DTYPE_BF16)
    return a.m.head_dim == 128 ? launch_tiles<128>(a, st) : a.m.head_dim == 256 ? launch_tiles<256>(a, st) : launch_tiles<512>(a, st);
  const int tiles = (a.max_new + BM - 1) / BM;
  latent_expand_kernel<<<(unsigned)((long long)a.m.n_seq * tiles * a.to.n_kv_head), THREADS, 0, st>>>(a, tiles);
  return cudaGetLastError();
}

}  // namespace evo
