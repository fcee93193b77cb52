// Attention over a paged memory for many rows a key/value head (long chunks,
// candidates that share a memory): bf16 rows and pages, on tcgen05.
//
// With 128 rows and more a key is used often enough that the tensor cores bound
// the call: 4 D operations a (row, key), 628 cycles for 128 rows x 128 keys of 64 at
// the measured bf16 rate, against 512 cycles for their 16,384 exponentials (32 a
// cycle and SM) and about 600 issue cycles a scheduler for the rest of the softmax.
// All three have to run at once.  A block keeps two streams of tiles in flight, and of
// each stream the next scores start as soon as the softmax has loaded these to registers:
//   * more than 128 rows: the streams are two tiles of 128 rows over the same keys;
//   * else: both are the same rows, over the even and the odd blocks of keys, and
//     are joined at the end.
// Roles: warps 0-3 and 4-7 are the softmax of streams A and B, a thread a row (the
// thread-per-lane layout of tensor memory: no reduction over lanes anywhere); warps 8
// and 10 issue a stream's MMAs each, so that neither waits for the other's weights; warp
// 9 brings keys and values, a block of BN at a time, by tiled bulk copies into a ring.
//
//   S = Q K^T      both operands from shared memory, 128-byte swizzle, fp32 in TMEM
//   P = 2^(S - m)  read from TMEM, written back to it as bf16, beside S
//   O += P V       P from TMEM, V as it lies in its page (rows of keys: the operand
//                  whose contiguous index is N)
// BN is what 512 columns of tensor memory hold of S, P and O of two streams: 128 keys
// of 64, 64 keys of 128.  Measured (2,048 rows over 16,384 keys of 64, 8 heads / four
// causal chunks of 1,000 tokens over 8,000, heads of 128): 87 us = 0.79 PFLOP/s / 135 us =
// 0.88; weights over the scores, so that the next ones wait for the product, 99 / 147; one
// issuing warp that takes both streams in turn 114 / 150.  What bounds it now is the
// softmax's issue: its two warps a scheduler are 85 % of the special-function unit while
// both are at their exponentials, and wait side by side when they are not (alternating them
// by a barrier, or a polynomial for some of the exponentials, measured slower).
//
// There is no running maximum: a row's reference is the maximum of its first block,
// and every further block's weights are summed before they are handed on.  Only where
// a sum passes 2^16 is a new maximum taken, O rescaled (a pass over TMEM, behind the
// product before) and the block done again, once: the common block reads no maximum (a fifth
// of the softmax's instructions, which bound it).  Weights are at most 2^16, and bf16
// holds them with the same relative rounding, 2^-8 at most of each.
//
// Masks are looked at only in blocks that some row does not see whole.  There, the
// values of keys outside the piece are set to zero in shared memory, and entries
// that are not finite too (0 * NaN would reach rows that do not see them); the rows
// that see them get them added at the end.
#include <algorithm>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
#include "evo_mem_ptx.cuh"

namespace evo {
namespace {

constexpr int BM = 128;
constexpr int THREADS = 384;                       // warps 10 and 11 only complete the third warpgroup
constexpr float LAZY = 8.f;                        // log2 of how far a block's maximum passes a reference that stays
constexpr int Q64 = BM * 128;                      // bytes of 64 columns of 128 queries

template <int D>
struct Cfg {
  static constexpr int BN = D == 64 ? 128 : 64;    // keys of a block: what 512 columns of tensor memory hold of S, P and O twice
  static constexpr int QTILE = BM * D * 2, TILE = BN * D * 2, K64 = BN * 128;   // bytes: 128 queries, BN keys or values, 64 columns of them
  static constexpr int SLOTS = D == 64 ? 8 : 10;
  static constexpr int LD = D + 4;                 // floats of a row where the streams are joined
  static constexpr int SMEM = 1024 + 2 * QTILE + SLOTS * TILE;
  static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BM >> 4) << 24);
  static constexpr uint32_t IDESC_S = IDESC | ((uint32_t)(BN >> 3) << 17);
  static constexpr uint32_t IDESC_O = IDESC | (1u << 16) | ((uint32_t)(D >> 3) << 17);   // B's contiguous index is N
  // TMEM columns of stream x: S at BN x, P (bf16, two a column) at P_COL + BN / 2 x, O at O_COL + D x
  static constexpr int P_COL = 2 * BN, O_COL = 512 - 2 * D;
};

struct Shared {
  uint64_t full[10], empty[10], s_full[2], s_free[2], p_full[2], o_full[2];
  uint32_t tmem;
  int dead, poison;
  float2 ml[BM];                                   // stream B's maximum and sum where the streams are joined
};

// ---------------------------------------------------------------- PTX wrappers
__device__ __forceinline__ void mma_tmem_a(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// 32 columns of this thread's lane, without waiting
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// the loads into v have landed: no use of v moves in front of this
template <int N>
__device__ __forceinline__ void tmem_wait_ld(float (&v)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// registers of a warpgroup: 8 softmax warps of 216 and 4 of 72 are the 12 warps of 168 of the launch
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void bar_softmax() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// descriptor of V as the operand whose contiguous index is N: 64 dimensions by 8 keys
// a swizzled kilobyte, the next 8 keys behind it, the next 64 dimensions k64 bytes on
__device__ __forceinline__ uint64_t v_desc(uint32_t saddr, int k64) {
  return (tc::sw128_desc(saddr) & ~(0x3fffull << 16)) | (uint64_t)(k64 >> 4) << 16;
}

// a bounded wait; false once any wait of the block was in vain
__device__ __forceinline__ bool wait_for(Shared& sh, uint64_t* bar, uint32_t parity) {
  const uint32_t b = tc::su32(bar);
  return tc::mbar_test(b, parity) || wait_live(b, parity, tc::su32(&sh.dead));
}

// the same behind a first test that failed, for the issuing warp
__device__ __noinline__ void wait_slow(uint32_t bar, uint32_t parity, uint32_t dead) { wait_live(bar, parity, dead); }
__device__ __forceinline__ uint64_t desc64(uint32_t lo, uint32_t hi) { return ((uint64_t)hi << 32) | lo; }
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ float2 exp2_of(float2 x) { return make_float2(ex2_approx(x.x), ex2_approx(x.y)); }
__device__ __forceinline__ uint32_t pack(float2 x) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(x.y), "f"(x.x));
  return r;
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1) tiles_kernel(const __grid_constant__ AttendArgs a,
                                                           const __grid_constant__ CUtensorMap kmap,
                                                           const __grid_constant__ CUtensorMap vmap) {
  using C = Cfg<D>;
  constexpr int SLOTS = C::SLOTS, BN = C::BN, K64 = C::K64;
  extern __shared__ uint8_t raw[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  uint8_t* const ring = mem + 2 * C::QTILE;
  if (tid == 0) fetch_map(&kmap), fetch_map(&vmap);
  const Tile t = tile_of_block(a);
  const int rows = t.count * a.group, r0 = t.tile * 2 * BM;
  if (r0 >= rows) return;
  const bool pair = r0 + BM < rows;                // two tiles of rows; else one, its keys over both streams
  const int ahead = pair ? 2 : 4;                  // blocks of keys whose scores are asked for before the first output
  const int last = min(r0 + 2 * BM, rows) - 1;
  const Range first_row = seen_by(a, t, r0 / a.group), last_row = seen_by(a, t, last / a.group);
  const Range all = piece_of(a, t, {first_row.lo, last_row.hi}, BN);
  const int whole_lo = max(last_row.lo, all.lo), whole_hi = min(first_row.hi, all.hi);
  const int key0 = all.lo / BN * BN, n = max(0, (all.hi - key0 + BN - 1) / BN);
  // operands in the ring: K 0 .. ahead - 1, then V i, K i + ahead
  const auto v_index = [&](int i) { return min(n, i + ahead) + i; };

  __syncwarp();                                    // a whole warp's instruction, behind one lane's prefetches
  if (warp == 0) tc::tmem_alloc(&sh.tmem, 512);
  if (tid == 32) {
    for (int i = 0; i < SLOTS; ++i) tc::mbar_init1(&sh.full[i], 1), tc::mbar_init1(&sh.empty[i], pair ? 2 : 1);
    for (int x = 0; x < 2; ++x) {
      tc::mbar_init1(&sh.s_full[x], 1);
      tc::mbar_init1(&sh.s_free[x], 4);        // a warp each
      tc::mbar_init1(&sh.p_full[x], 4);
      tc::mbar_init1(&sh.o_full[x], 1);
    }
    sh.dead = sh.poison = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // queries to shared memory, a row a thread; the softmax works with a positive scale
  const float sc = a.scale_log2 == 0.f ? 1.f : fmaxf(fabsf(a.scale_log2), 1.1754944e-38f);
  if (warp < 8 && (pair || warp < 4)) {
    const int r = tid % BM, R = r0 + tid;
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) +
                                                      (long long)(t.first + R / a.group) * a.ldq +
                                                      (long long)(t.kv_head * a.group + R % a.group) * D);
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      uint4 u = R < rows && a.scale_log2 != 0.f ? src[j] : make_uint4(0, 0, 0, 0);
      u.x ^= flip, u.y ^= flip, u.z ^= flip, u.w ^= flip;
      *reinterpret_cast<uint4*>(mem + (warp / 4) * C::QTILE + (j / 8) * Q64 + r * 128 + ((j % 8 ^ (r & 7)) << 4)) = u;
    }
    tc::fence_async_smem();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;

  if (warp >= 8) {
  fewer_registers<72>();
  if (warp == 9) {
    // ------------------------------------------------------------ copies
    const int page_tokens = a.m.page_tokens, box = min(page_tokens, BN), shift = 31 - __clz(page_tokens);
    const int head_row = t.kv_head * page_tokens, page_rows = a.m.n_kv_head * page_tokens;
    int index = 0;
    const auto bring = [&](const CUtensorMap* map, int i) {
      const int slot = index % SLOTS, use = index / SLOTS;
      ++index;
      const int key = key0 + i * BN + lane * box;
      const bool on = lane * box < BN && key + box > all.lo && key < all.hi;
      const int page = on ? seq_page(a.m, t.n, key >> shift) : 0;
      if (!__all_sync(0xffffffffu, use == 0 || wait_for(sh, &sh.empty[slot], (use - 1) & 1))) return;
      const int copies = __popc(__ballot_sync(0xffffffffu, on));
      if (lane == 0) tc::mbar_expect_tx(&sh.full[slot], copies * box * D * 2);
      __syncwarp();
      if (on)
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
          tc::tma_load_2d(ring + slot * C::TILE + x * K64 + lane * box * 128, map, x * 64,
                          page * page_rows + head_row + (key & (page_tokens - 1)), &sh.full[slot]);
      __syncwarp();
    };
    for (int i = 0; i < min(ahead, n); ++i) bring(&kmap, i);
    for (int i = 0; i < n; ++i) {
      bring(&vmap, i);
      if (i + ahead < n) bring(&kmap, i + ahead);
    }
  } else if (warp == 8 || warp == 10) {
    // ------------------------------------------------------------ MMAs of a stream
    // Uniform over the warp and known to the compiler to be (a shuffle's result is), one elected
    // lane issuing: descriptors then stay in uniform registers.
    const uint32_t x = __shfl_sync(0xffffffffu, warp == 8 ? 0 : 1, 0);
    const int blocks = __shfl_sync(0xffffffffu, n, 0), two = __shfl_sync(0xffffffffu, (int)pair, 0);
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t kdesc = tc::sw128_desc(0), vdesc = v_desc(0, K64);
    const uint32_t khi = (uint32_t)(kdesc >> 32), klo = (uint32_t)kdesc, vhi = (uint32_t)(vdesc >> 32), vlo = (uint32_t)vdesc;
    const uint32_t qd = klo + (tc::su32(mem) >> 4) + (two ? x : 0) * (C::QTILE >> 4), r0d = tc::su32(ring) >> 4;
    const uint32_t full = tc::su32(sh.full), empty = tc::su32(sh.empty), dead = tc::su32(&sh.dead);
    const uint32_t s_full = tc::su32(&sh.s_full[x]), s_free = tc::su32(&sh.s_free[x]), p_full = tc::su32(&sh.p_full[x]),
                   o_full = tc::su32(&sh.o_full[x]);
    const uint32_t lead = two ? 2 : 4;
    const auto wait = [&](uint32_t bar, uint32_t parity) {
      if (!tc::mbar_test(bar, parity)) wait_slow(bar, parity, dead);
    };
    // S of block i
    const auto scores = [&](uint32_t i) {
      const uint32_t index = i < lead ? i : 2 * i - lead + 1, slot = index % SLOTS;
      wait(full + 8 * slot, (index / SLOTS) & 1);
      tc::tc_fence_after();
      const uint32_t kd = klo + r0d + slot * (C::TILE >> 4);
      if (tc::elect_one()) {
#pragma unroll
        for (uint32_t k = 0; k < D / 16; ++k)
          tc::mma_f16(tm + BN * x, desc64(qd + (k / 4) * (Q64 >> 4) + (k % 4) * 2, khi),
                      desc64(kd + (k / 4) * (K64 >> 4) + (k % 4) * 2, khi), C::IDESC_S, k);
        commit(s_full);
        commit(empty + 8 * slot);
      }
    };
    // O += P V of block i
    const auto output = [&](uint32_t i, uint32_t accumulate) {
      const uint32_t index = min((uint32_t)blocks, i + lead) + i, slot = index % SLOTS;
      wait(full + 8 * slot, (index / SLOTS) & 1);
      tc::tc_fence_after();
      const uint32_t vd = vlo + r0d + slot * (C::TILE >> 4);
      if (tc::elect_one()) {
#pragma unroll
        for (uint32_t k = 0; k < BN / 16; ++k)
          mma_tmem_a(tm + C::O_COL + D * x, tm + C::P_COL + BN / 2 * x + 8 * k, desc64(vd + k * (2048 >> 4), vhi), C::IDESC_O,
                     accumulate | k);
        commit(empty + 8 * slot);
        commit(o_full);
      }
    };
    const int from = two ? 0 : x, by = two ? 1 : 2;
    if (from < blocks) scores(from);
    for (int it = 0; from + by * it < blocks; ++it) {
      if (from + by * (it + 1) < blocks) {
        wait(s_free, it & 1);                      // the softmax has this block's scores in registers
        scores(from + by * (it + 1));
      }
      wait(p_full, it & 1);
      output(from + by * it, it);
      if (__any_sync(0xffffffffu, tc::block_dead(dead))) break;
    }
  }
  } else {
    more_registers<216>();
    // ------------------------------------------------------------ softmax: stream x, a row a thread
    const int x = warp / 4, r = tid % BM, R = r0 + (pair ? tid : r);
    const uint32_t lanes = (uint32_t)(32 * (warp % 4)) << 16;
    const uint32_t s_at = tmem + BN * x + lanes, p_at = tmem + C::P_COL + BN / 2 * x + lanes, o_at = tmem + C::O_COL + D * x + lanes;
    Range see = R < rows ? seen_by(a, t, R / a.group) : Range{0, 0};
    see = {max(see.lo, all.lo), min(see.hi, all.hi)};
    const int from = pair ? 0 : x, by = pair ? 1 : 2;
    float top = -INFINITY;
    float l = 0.f;
    bool ok = true;
    int it = 0;
    for (int i = from; i < n; i += by, ++it) {
      ok = __all_sync(0xffffffffu, wait_for(sh, &sh.s_full[x], it & 1));
      if (!ok) break;
      tc::tc_fence_after();
      float v[BN];
#pragma unroll
      for (int j = 0; j < BN / 32; ++j) tmem_ld32_async(s_at + 32 * j, v + 32 * j);
      tmem_wait_ld(v);
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive1(&sh.s_free[x]);
      const int k0 = key0 + i * BN;
      const bool whole = k0 >= whole_lo && k0 + BN <= whole_hi;
      if (!whole) {
        const int lo = see.lo - k0, hi = see.hi - k0;
#pragma unroll
        for (int j = 0; j < BN; ++j) v[j] = j >= lo && j < hi ? v[j] : -INFINITY;
        {
          // this block's values, cleaned before the product may read them (two streams that share
          // them both do it, each for its own product: they write the same)
          const int index = v_index(i), slot = index % SLOTS;
          ok = __all_sync(0xffffffffu, wait_for(sh, &sh.full[slot], (index / SLOTS) & 1));
          if (!ok) break;
          const int vr = r % BN, part = r / BN;    // a value a thread, or its columns' half
          const bool drop = k0 + vr < all.lo || k0 + vr >= all.hi;
#pragma unroll
          for (int jj = 0; jj < D * BN / 1024; ++jj) {
            const int j = part * (D * BN / 1024) + jj;
            uint4* p = reinterpret_cast<uint4*>(ring + slot * C::TILE + (j / 8) * K64 + vr * 128 + ((j % 8 ^ (vr & 7)) << 4));
            uint4 u = *p;
            uint32_t* w = reinterpret_cast<uint32_t*>(&u);
            bool changed = drop, bad = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t keep = 0xffffffffu;
              if ((w[e] & 0x7f80u) == 0x7f80u) keep &= 0xffff0000u;
              if ((w[e] & 0x7f800000u) == 0x7f800000u) keep &= 0x0000ffffu;
              if (keep != 0xffffffffu) changed = true, bad |= !drop;
              w[e] = drop ? 0u : w[e] & keep;
            }
            if (bad) {                             // before the value goes: the other stream may find it clean already
              *reinterpret_cast<volatile int*>(&sh.poison) = 1;
              __threadfence_block();
            }
            if (changed) *p = u;
          }
          tc::fence_async_smem();
        }
      }
      if (it > 0) {                                // the product before this block has read its weights
        ok = __all_sync(0xffffffffu, wait_for(sh, &sh.o_full[x], (it - 1) & 1));
        if (!ok) break;
        tc::tc_fence_after();
      }
      // a row's reference is the maximum of the block where it was set.  The others are taken on
      // trust: a block whose weights sum to more than 2^16 sets it anew and is done again, once
      float s1 = sc;                               // factor that the scores in v still lack
      for (bool set = __any_sync(0xffffffffu, top == -INFINITY), again = true;; again = false) {
        if (set) {
          float m = v[0];
#pragma unroll
          for (int j = 1; j < BN; ++j) m = fmaxf(m, v[j]);
          m = __fmul_rn(m, s1);
          const float now = m - top > LAZY ? m : top;   // (top + LAZY may round to more than LAZY above top)
          const float f = ex2_approx(top - (now == -INFINITY ? 0.f : now));
          top = now;
          l *= f;
          if (it > 0) {
#pragma unroll 1
            for (int j = 0; j < D / 32; ++j) {
              float o[32];
              tmem_ld32_async(o_at + 32 * j, o);
              tmem_wait_ld(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= f;
              tmem_st32(o_at + 32 * j, reinterpret_cast<const uint32_t*>(o));
            }
          }
        }
        const float ref = top == -INFINITY ? 0.f : -top;
        // The reference is a rounded product, the fused ones below are not: past 2^24 they differ by more
        // than a step of the exponent, and the largest weight would not be 1.  Where a row of the warp is
        // that far, scores are rounded first, as the reference was
        if (__any_sync(0xffffffffu, fabsf(ref) >= 16777216.f)) {
#pragma unroll
          for (int j = 0; j < BN; ++j) v[j] = __fmul_rn(v[j], s1);
          s1 = 1.f;
        }
        const float2 sc2 = make_float2(s1, s1), ref2 = make_float2(ref, ref);
        float2 sums[4] = {};                       // chains of their own
#pragma unroll
        for (int h = 0; h < BN / 64; ++h) {
          uint32_t p[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float2 w = exp2_of(fma2(make_float2(v[64 * h + 2 * j], v[64 * h + 2 * j + 1]), sc2, ref2));
            sums[j % 4] = add2(sums[j % 4], w);
            p[j] = pack(w);
          }
          tmem_st32(p_at + 32 * h, p);
        }
        const float2 all4 = add2(add2(sums[0], sums[1]), add2(sums[2], sums[3]));
        set = __any_sync(0xffffffffu, all4.x + all4.y > 65536.f);
        if (!set || !again) {
          l += all4.x + all4.y;
          break;
        }
      }
      tmem_wait_st();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive1(&sh.p_full[x]);
    }
    if (ok && it > 0) ok = __all_sync(0xffffffffu, wait_for(sh, &sh.o_full[x], (it - 1) & 1));
    tc::tc_fence_after();
    bool mine = R < rows, scaled = false;
    float fa = 1.f, fb = 0.f;
    float* const joined = reinterpret_cast<float*>(ring) + r * C::LD;
    if (!pair) {
      // stream B hands its sums over once nothing reads the ring any more
      bar_softmax();
      if (x == 1) {
        sh.ml[r] = make_float2(top, l);
        if (it > 0 && ok)
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            float o[32];
            tmem_ld32_async(o_at + 32 * j, o);
            tmem_wait_ld(o);
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(joined + 32 * j + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        mine = false;
      }
      bar_softmax();
      if (x == 0 && n > 1) {
        const float2 b = sh.ml[r];
        const float m = fmaxf(top, b.x), ref = m == -INFINITY ? 0.f : m;
        fa = ex2_approx(top - ref), fb = ex2_approx(b.x - ref);
        top = m;
        l = l * fa + b.y * fb;
        scaled = true;
      }
    }
    if (ok && !tc::block_dead(tc::su32(&sh.dead))) {
      const int row = t.first + R / a.group, head = t.kv_head * a.group + R % a.group;
      const long long at = mine ? part_index(a, t.split, row, head) : 0;
      const float norm = l == 0.f ? 0.f : 1.f / l;
      const bool fix = sh.poison != 0;
#pragma unroll 1
      for (int j = 0; j < D / 32; ++j) {
        float o[32];
        __syncwarp();                              // lanes leave the turn before at their own times
        if (x == 0 || pair) {                      // (a warp's collective load: whole warps of stream B are out)
          if (it > 0) {
            tmem_ld32_async(o_at + 32 * j, o);
            tmem_wait_ld(o);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
        }
        if (!mine) continue;
        if (scaled)
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = o[e] * fa + joined[32 * j + e] * fb;
        if (fix) {
          for (int k = see.lo; k < see.hi; ++k) {
            const int k0 = k / BN * BN;
            if (k0 >= whole_lo && k0 + BN <= whole_hi) {
              k = k0 + BN - 1;
              continue;
            }
            const long long vr = ((long long)seq_page(a.m, t.n, k / a.m.page_tokens) * a.m.n_kv_head + t.kv_head) *
                                     a.m.page_tokens + k % a.m.page_tokens;
            const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(a.m.v_pages) + vr * D + 32 * j;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float y = __bfloat162float(p[e]);
              if (!isfinite(y)) o[e] += y;
            }
          }
        }
        if (a.splits == 1) {
          uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + row * a.ldo + (long long)head * D + 32 * j);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            dst[e] = make_uint4(pack(make_float2(o[8 * e] * norm, o[8 * e + 1] * norm)),
                                pack(make_float2(o[8 * e + 2] * norm, o[8 * e + 3] * norm)),
                                pack(make_float2(o[8 * e + 4] * norm, o[8 * e + 5] * norm)),
                                pack(make_float2(o[8 * e + 6] * norm, o[8 * e + 7] * norm)));
        } else {
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<float4*>(a.part + at * D + 32 * j + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
      }
      if (mine && a.splits > 1) a.ml[at] = make_float2(top, l);
    }
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

template <int D>
cudaError_t launch_as(const AttendArgs& a, cudaStream_t st) {
  using C = Cfg<D>;
  CUtensorMap km, vm;
  const int box = std::min(a.m.page_tokens, C::BN);
  if (!page_map(&km, a.m, a.m.k_pages, box) || !page_map(&vm, a.m, a.m.v_pages, box)) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  return launch_pieces(tiles_kernel<D>, a, THREADS, C::SMEM, done, st, km, vm);
}

}  // namespace

cudaError_t launch_attend_tiles(const AttendArgs& a, cudaStream_t st) {
  return a.m.head_dim == 64 ? launch_as<64>(a, st) : launch_as<128>(a, st);
}

}  // namespace evo
