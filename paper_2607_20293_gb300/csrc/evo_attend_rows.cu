// Attention over a paged memory for few rows a key/value head (single tokens,
// short action chunks): bf16 rows, bf16 or 8-bit pages.
//
// Such a call reads every key and value once for at most 8 NR rows, so DRAM
// bounds it as long as the tensor cores and the conversion of codes keep up:
// mma.sync (1,024 multiply-adds a cycle and SM, a quarter of what tcgen05 has)
// takes 16 of the 174 cycles in which 16 bf16 keys and values of 64 arrive for 8
// rows, without padding them to tcgen05's 128.
//
// Both products have the memory as their first operand, so that a tile is 16 keys
// (or dimensions) by 8 rows, and 8 rows cost half of what 16 do:
//   S^T = K Q^T  (keys x rows),  O^T = V^T P^T  (dimensions x rows)
// P^T leaves the first product as keys x rows and enters the second as its
// transpose's fragment: one movmatrix for 8 keys.
//
// A block is 4 warps on one tile of rows and one piece of the memory.  Each warp
// takes every 4th run of RUN keys by itself: it brings the run's keys, values and
// scale bytes to its own ring in shared memory by tiled bulk copies, STAGES - 1 runs
// ahead, so that no barrier of the block is met until the end (loads straight to
// registers, one run ahead, reached 2.8 TB/s on 64 sequences of 4,096-8,192 8-bit
// keys).  Fragments are read with 16-byte loads, because a contraction's index may
// be permuted at will: lane (g, c) = (lane / 4, lane % 4) holds 16 contiguous bytes
// of key g, the queries' fragments use the same permutation, and row g of an output
// tile stands for one of the 8 or 16 contiguous dimensions that the lane read of
// values 2c, 2c+1, 2c+8 and 2c+9: with the copies' 128-byte swizzle the 8 lanes of a
// phase meet 8 different chunks.  Every warp keeps its own running maximum and
// sums; they are joined through shared memory at the end.
//
// The running maximum is lazy: the sums are rescaled only when a score passes
// the row's reference by 2^8, so the common run has one vote instead of
// reductions over lanes and a pass over the accumulators.  Weights are then at
// most 2^8, which the 16-bit operand holds with the same relative rounding.
// The reference m is subtracted from the product, and the difference multiplied by
// the row's factor: equal scores have equal weights at any size.  (A fused product minus a
// rounded reference leaves the largest weight at 2^(rounding error): past fp16 from scores of 2^24.)
//
// 8-bit pages: codes become fp16 exactly (one conversion for two).  A key's scale
// multiplies its row of S^T in fp32; queries are brought to fp16 by an exact power of
// two per row.  A value's scale 2^k is added to the exponent of its weights,
// 2^(s - m + k - m'), with an offset m' of its own, so that the fp16 operand stays in
// range for any mixture of scales; the sum of weights uses 2^(s - m).  The weights'
// rounding is fp16's there: 2^-11 of each, or 2^-25 absolute for those that are, with
// their value's scale, below 2^-14 of the row's largest; bf16's (2^-8) with bf16 pages.
//
// Masks are looked at only in runs that some row does not see whole.  There, keys
// outside the piece give zero values, and a value that is not finite is taken out
// of the product (0 * NaN would reach rows that do not see it) and put back at the
// end for the rows that see it.
#include <algorithm>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
#include "evo_mem_ptx.cuh"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr float LAZY = 8.f;                        // log2 of how far a weight may pass 1
constexpr float SLACK = 7.f;                       // and, with its value's scale, pass the row's reference for those: 2^15 in all
constexpr float NO_NUMBER = __builtin_nanf("");

template <int D, bool E4M3, int NR>
struct Cfg {
  static constexpr int ROW = D * (E4M3 ? 1 : 2);   // bytes of a key or value
  static constexpr int BOX = ROW < 128 ? ROW : 128;   // bytes of a row that one copy brings (the swizzle's width)
  static constexpr int RUN = ROW == 64 ? 32 : 16;
  static constexpr int NB = RUN / 16;
  static constexpr int KP = ROW / 64;              // 16-byte pieces of a key a lane holds (4 lanes a key)
  static constexpr int VP = ROW < 128 ? 1 : ROW / 128;   // 16-byte (or one 8-byte) pieces of a value (8 lanes a value)
  static constexpr int TILE = RUN * ROW;           // bytes of a run's keys
  static constexpr int STAGE = 2 * TILE;
  static constexpr int STAGES = STAGE > 4096 ? 3 : 4;
  static constexpr int JOIN = 8 * NR * (D + 4) * 4;
  static constexpr int RING = (STAGES * STAGE > JOIN ? STAGES * STAGE : JOIN + 1023) / 1024 * 1024;   // a warp's bytes
  static constexpr bool QS = NR == 4;              // queries stay in shared memory: their fragments take 32 or 64 registers
  static constexpr int BLOCKS = NR == 4 ? (D == 64 ? 3 : 2) : 1;   // blocks a SM that the registers leave room for
  static constexpr int QB = QS ? NR * (D / 16) * 256 : 0;
  static constexpr int SCALES = E4M3 ? WARPS * STAGES * 2 * RUN : 0;
  static constexpr int SMEM = 1024 + WARPS * RING + QB + SCALES;
};

// ---------------------------------------------------------------- PTX wrappers
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool half) {
  if (half)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the transpose of an 8 x 8 matrix of 16-bit values, two of a row in a lane
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// two codes (low 16 bits of c) to two fp16
__device__ __forceinline__ uint32_t half2_of(uint32_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
  return h;
}
__device__ __forceinline__ uint32_t pack(float a, float b, bool half) {
  uint32_t r;
  if (half)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t finite_halves(uint32_t w, bool* bad) {
  uint32_t keep = 0xffffffffu;
  if ((w & 0x7f80u) == 0x7f80u) keep &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) keep &= 0x0000ffffu;
  *bad |= keep != 0xffffffffu;
  return w & keep;
}

template <int D, bool E4M3, int NR>
__global__ void __launch_bounds__(THREADS, Cfg<D, E4M3, NR>::BLOCKS) rows_kernel(const __grid_constant__ AttendArgs a,
                                                       const __grid_constant__ CUtensorMap kmap,
                                                       const __grid_constant__ CUtensorMap vmap) {
  using C = Cfg<D, E4M3, NR>;
  constexpr int RUN = C::RUN, NB = C::NB, KS = D / 16, DT = D / 16, LD = D + 4, STAGES = C::STAGES, ROWS = 8 * NR;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t full[WARPS][STAGES];
  __shared__ float2 stat[WARPS][ROWS];                       // the warps' maxima and sums
  __shared__ float vmax[E4M3 ? WARPS : 1][ROWS];
  __shared__ float2 block_ml[ROWS];
  __shared__ int poison;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4;
  uint8_t* const mem = raw + ((1024u - (tc::su32(raw) & 1023u)) & 1023u);
  const uint32_t ring = tc::su32(mem) + warp * C::RING;
  const uint32_t qsm = tc::su32(mem) + WARPS * C::RING;
  const uint32_t ssm = qsm + C::QB + warp * (STAGES * 2 * RUN);
  if (tid == 0) fetch_map(&kmap), fetch_map(&vmap);
  const Tile t = tile_of_block(a);
  const int rows = t.count * a.group, r0 = t.tile * ROWS;
  if (r0 >= rows) return;
  const int last = min(r0 + ROWS, rows) - 1;
  const Range first_row = seen_by(a, t, r0 / a.group), last_row = seen_by(a, t, last / a.group);
  const Range all = piece_of(a, t, {first_row.lo, last_row.hi}, RUN);
  // keys that every row of the tile sees, of this piece
  const int whole_lo = max(last_row.lo, all.lo), whole_hi = min(first_row.hi, all.hi);
  if (tid == 0) {
    poison = 0;
    for (int i = 0; i < WARPS * STAGES; ++i) tc::mbar_init1(&full[0][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();

  // copies of a run: box rows each, lane i the i-th; its page is looked up a run ahead
  const int box = min(a.m.page_tokens, RUN), shift = 31 - __clz(a.m.page_tokens), step = WARPS * RUN;
  const int page_rows = a.m.n_kv_head * a.m.page_tokens, head_row = t.kv_head * a.m.page_tokens;
  auto page_at = [&](int k0) {
    const int kb = k0 + lane * box;
    return lane * box < RUN && kb + box > all.lo && kb < all.hi ? seq_page(a.m, t.n, kb >> shift) : -1;
  };
  auto issue = [&](int k0, int page, int stage) {
    const uint32_t bar = tc::su32(&full[warp][stage]);
    const int copies = __popc(__ballot_sync(0xffffffffu, page >= 0));
    if (lane == 0) tc::mbar_expect_tx(&full[warp][stage], copies * box * (2 * C::ROW + (E4M3 ? 2 : 0)));
    __syncwarp();
    if (page >= 0) {
      const int at = page * page_rows + head_row + ((k0 + lane * box) & (a.m.page_tokens - 1));
      const uint32_t dst = ring + stage * C::STAGE + lane * box * C::BOX;
#pragma unroll
      for (int x = 0; x < C::ROW / C::BOX; ++x) {
        tile_load(dst + x * RUN * C::BOX, &kmap, x * 64, at, bar);
        tile_load(dst + C::TILE + x * RUN * C::BOX, &vmap, x * 64, at, bar);
      }
      if constexpr (E4M3) {
        bulk_load(ssm + stage * 2 * RUN + lane * box, a.m.k_scales + at, box, bar);
        bulk_load(ssm + stage * 2 * RUN + RUN + lane * box, a.m.v_scales + at, box, bar);
      }
    }
  };
  int k0 = all.lo / RUN * RUN + warp * RUN;
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i)
    if (k0 + i * step < all.hi) issue(k0 + i * step, page_at(k0 + i * step), i);
  int ahead = page_at(k0 + (STAGES - 1) * step);

  // queries: fragments in the keys' permutation; row 8 nr + g
  uint32_t q[C::QS ? 1 : NR][C::QS ? 1 : KS][2];
  float rf[NR][2];                                           // factor of rows 2 c, 2 c + 1 from a product to base-2 scores
#pragma unroll
  for (int nr = 0; nr < NR; ++nr) {
    const int R = r0 + 8 * nr + g;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + (long long)(t.first + R / a.group) * a.ldq +
                               (long long)(t.kv_head * a.group + R % a.group) * D;
    uint4 u[D / 32];                                         // 8 values each, in the order of the steps
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      u[i] = R < rows ? *reinterpret_cast<const uint4*>(src + (E4M3 ? 64 * (i / 2) + 16 * c + 8 * (i % 2) : 32 * i + 8 * c))
                      : make_uint4(0, 0, 0, 0);
    // the softmax works with a positive factor: the scale's sign goes to the queries
    float f = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u, keep = a.scale_log2 == 0.f ? 0u : ~0u;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      u[i] = make_uint4((u[i].x ^ flip) & keep, (u[i].y ^ flip) & keep, (u[i].z ^ flip) & keep, (u[i].w ^ flip) & keep);
    if constexpr (E4M3) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max(top, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // 2^(14 - e) for a largest magnitude in [2^e, 2^(e+1)), within fp32's exponents
      const int e = (int)(top >> 7);                         // e + 127
      const int up = top == 0 || e == 255 ? 0 : min(max(141 - e, -126), 126);
      const float s2 = __int_as_float((up + 127) << 23);
      f *= __int_as_float((127 - up) << 23);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&u[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = pack(__uint_as_float(w[j] << 16) * s2, __uint_as_float(w[j] & 0xffff0000u) * s2, true);
      }
    }
    f = fmaxf(f, 1.1754944e-38f);                            // (a factor that is flushed to zero would make a masked score none)
    rf[nr][0] = __shfl_sync(0xffffffffu, f, 8 * c);
    rf[nr][1] = __shfl_sync(0xffffffffu, f, 8 * c + 4);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint32_t b0 = ks % 2 ? u[ks / 2].z : u[ks / 2].x, b1 = ks % 2 ? u[ks / 2].w : u[ks / 2].y;
      if constexpr (C::QS) {
        if (warp == 0)
          asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(qsm + ((nr * KS + ks) * 32 + lane) * 8), "r"(b0), "r"(b1) : "memory");
      } else {
        q[nr][ks][0] = b0;
        q[nr][ks][1] = b1;
      }
    }
  }
  if constexpr (C::QS) __syncthreads();

  // o: dimensions g, g + 8 x rows 2 c, 2 c + 1 of a tile; top: the row's reference, in units of the product;
  // voff: what its values' sums stand in beside it, as an exponent (+infinity: it has seen no key)
  float o[NR][DT][4], sum[NR][2], top[NR][2], voff[NR][2];
#pragma unroll
  for (int nr = 0; nr < NR; ++nr) {
#pragma unroll
    for (int j = 0; j < DT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[nr][j][i] = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) sum[nr][e] = 0.f, top[nr][e] = -INFINITY, voff[nr][e] = INFINITY;
  }

  int stage = 0;
  uint32_t phase = 0;
  bool dead = false;
  for (; k0 < all.hi; k0 += step) {
    if (k0 + (STAGES - 1) * step < all.hi) {
      issue(k0 + (STAGES - 1) * step, ahead, stage == 0 ? STAGES - 1 : stage - 1);
      ahead = page_at(k0 + STAGES * step);
    }
    if (!__all_sync(0xffffffffu, wait_full(tc::su32(&full[warp][stage]), phase))) {
      dead = true;
      break;
    }
    const uint32_t kt = ring + stage * C::STAGE, vt = kt + C::TILE, sc = ssm + stage * 2 * RUN;
    // s[nr][b]: keys g, g + 8 of the b-th 16 x rows 2 c, 2 c + 1
    float s[NR][NB][4];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nr][b][e] = 0.f;
#pragma unroll
    for (int h = 0; h < C::KP; ++h) {
      uint4 kr[NB][2];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) kr[b][i] = lds128(kt + chunk_at<C::ROW, RUN>(16 * b + 8 * i + g, 4 * h + c));
#pragma unroll
      for (int j = 0; j < (E4M3 ? 4 : 2); ++j) {             // steps of 4 values a lane
        const int ks = (E4M3 ? 4 : 2) * h + j;
        uint32_t qf[NR][2];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
          if constexpr (C::QS) {
            const uint2 u = lds64(qsm + ((nr * KS + ks) * 32 + lane) * 8);
            qf[nr][0] = u.x, qf[nr][1] = u.y;
          } else {
            qf[nr][0] = q[nr][ks][0], qf[nr][1] = q[nr][ks][1];
          }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const uint32_t w0[4] = {kr[b][0].x, kr[b][0].y, kr[b][0].z, kr[b][0].w};
          const uint32_t w1[4] = {kr[b][1].x, kr[b][1].y, kr[b][1].z, kr[b][1].w};
          uint32_t f[4];
          if constexpr (E4M3) {
            f[0] = half2_of(w0[j]), f[1] = half2_of(w1[j]), f[2] = half2_of(w0[j] >> 16), f[3] = half2_of(w1[j] >> 16);
          } else {
            f[0] = w0[2 * j % 4], f[1] = w1[2 * j % 4], f[2] = w0[(2 * j + 1) % 4], f[3] = w1[(2 * j + 1) % 4];
          }
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) mma16(s[nr][b], f, qf[nr][0], qf[nr][1], E4M3);
        }
      }
    }
    // a key's scale; a value's as an exponent
    float vs[NB][2];
    bool odd = k0 < whole_lo || k0 + RUN > whole_hi;         // some row does not see the whole run
    float vs_top = 0.f;                                      // the largest value scale of the run
    if constexpr (E4M3) {
      const uint32_t kb = lane < RUN ? lds8(sc + lane) : 0, vb = lane < RUN ? lds8(sc + RUN + lane) : 0;
      const uint32_t top_byte = __reduce_max_sync(0xffffffffu, max(kb == SCALE_NAN ? SCALE_NAN : 0u, vb));
      vs_top = __uint_as_float(0x4b000000u | top_byte) - 8388735.f;
      odd |= top_byte == SCALE_NAN;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t kb = lds8(sc + 16 * b + 8 * i + g), vb = lds8(sc + RUN + 16 * b + 8 * i + g);
          float ks = __uint_as_float(kb << 23);
          vs[b][i] = __uint_as_float(0x4b000000u | vb) - 8388735.f;      // vb - 127
          // a key or value that is no number makes the key's scores none: the rows that see it,
          // and no other, then hold NaN
          if (odd && (kb == SCALE_NAN || vb == SCALE_NAN)) ks = NO_NUMBER, vs[b][i] = 0.f;
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            const float2 x = mul2(make_float2(s[nr][b][2 * i], s[nr][b][2 * i + 1]), make_float2(ks, ks));
            s[nr][b][2 * i] = x.x, s[nr][b][2 * i + 1] = x.y;
          }
        }
    }
    if (odd) {
#pragma unroll
      for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int R = r0 + 8 * nr + 2 * c + e;
          const Range see = R < rows ? seen_by(a, t, R / a.group) : Range{0, 0};
          const int lo = max(see.lo, all.lo), hi = min(see.hi, all.hi);
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int key = k0 + 16 * b + 8 * i + g;
              if (key < lo || key >= hi) s[nr][b][2 * i + e] = -INFINITY;
            }
        }
    }
    // does a score pass its row's reference by 2^LAZY?  The reference is subtracted before the factor is
    // multiplied in, here as for the weights, so that the largest weight is 1 at any size of the scores.
    // 8-bit pages: or could a weight times its value's scale pass what fp16 holds, 2^(LAZY + SLACK)
    bool raise = false;
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float m = fmaxf(s[nr][0][e], s[nr][0][2 + e]);
#pragma unroll
        for (int b = 1; b < NB; ++b) m = fmaxf(m, fmaxf(s[nr][b][e], s[nr][b][2 + e]));
        raise |= (m - top[nr][e]) * rf[nr][e] > LAZY;
        if constexpr (E4M3) raise |= vs_top > voff[nr][e] + SLACK;
      }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float m = s[nr][0][e];
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i) m = fmaxf(m, s[nr][b][2 * i + e]);
#pragma unroll
          for (int x = 4; x < 32; x *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
          m = fmaxf(m, top[nr][e]);
          const float base = m == -INFINITY ? 0.f : m, down = (top[nr][e] - base) * rf[nr][e];
          const float f = ex2_approx(down);
          float fv = f;
          if constexpr (E4M3) {
            // the values' reference: the row's own largest weight times scale so far, raised no further
            // than this run's weights need, so that no outlier of negligible weight pushes the others out
            float mv = -INFINITY;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int i = 0; i < 2; ++i) mv = fmaxf(mv, (s[nr][b][2 * i + e] - base) * rf[nr][e] + vs[b][i]);
#pragma unroll
            for (int x = 4; x < 32; x *= 2) mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, x));
            const float old = top[nr][e] == -INFINITY ? -INFINITY : voff[nr][e] + down;
            mv = fmaxf(mv, old);
            fv = ex2_approx(old - (mv == -INFINITY ? 0.f : mv));
            voff[nr][e] = m == -INFINITY ? INFINITY : mv;
          }
          top[nr][e] = m;
          sum[nr][e] *= f;
#pragma unroll
          for (int j = 0; j < DT; ++j) o[nr][j][e] *= fv, o[nr][j][2 + e] *= fv;
        }
    }
    // weights, and their transposes as the second product's fragments
    uint32_t p[NR][NB][2];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
      const float2 r2 = make_float2(rf[nr][0], rf[nr][1]);
      const float2 m2 = make_float2(top[nr][0] == -INFINITY ? 0.f : -top[nr][0], top[nr][1] == -INFINITY ? 0.f : -top[nr][1]);
      const float2 v2 = make_float2(-voff[nr][0], -voff[nr][1]);
      float2 l2 = make_float2(sum[nr][0], sum[nr][1]);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 x = add2(make_float2(s[nr][b][2 * i], s[nr][b][2 * i + 1]), m2);
          float2 w = mul2(x, r2);
          w = make_float2(ex2_approx(w.x), ex2_approx(w.y));
          l2 = add2(l2, w);
          if constexpr (E4M3) {
            w = fma2(x, r2, add2(make_float2(vs[b][i], vs[b][i]), v2));
            w = make_float2(ex2_approx(w.x), ex2_approx(w.y));
          }
          p[nr][b][i] = transposed(pack(w.x, w.y, E4M3));
        }
      sum[nr][0] = l2.x, sum[nr][1] = l2.y;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int h = 0; h < C::VP; ++h) {
        uint32_t w[4][4];                                    // values 2 c, 2 c + 1, 2 c + 8, 2 c + 9
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 16 * b + 8 * (i / 2) + 2 * c + i % 2;
          if constexpr (C::ROW == 64) {
            const uint2 u = lds64(vt + chunk_at<64, RUN>(r, g / 2) + 8 * (g % 2));
            w[i][0] = u.x, w[i][1] = u.y, w[i][2] = w[i][3] = 0;
          } else {
            const uint4 u = lds128(vt + chunk_at<C::ROW, RUN>(r, 8 * h + g));
            w[i][0] = u.x, w[i][1] = u.y, w[i][2] = u.z, w[i][3] = u.w;
          }
        }
        if (odd) {
          bool bad = false;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 16 * b + 8 * (i / 2) + 2 * c + i % 2, key = k0 + r;
            bool drop = key < all.lo || key >= all.hi;
            if constexpr (E4M3) drop |= lds8(sc + RUN + r) == SCALE_NAN || lds8(sc + r) == SCALE_NAN;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              if (drop) w[i][x] = 0;
              if constexpr (!E4M3) w[i][x] = finite_halves(w[i][x], &bad);
            }
          }
          if (!E4M3 && bad) poison = 1;
          __syncwarp();                                      // the products are a whole warp's
        }
        if constexpr (E4M3) {
#pragma unroll
          for (int x = 0; x < (C::ROW == 64 ? 2 : 4); ++x)   // 4 dimensions a word: two tiles
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint32_t a01 = __byte_perm(w[0][x], w[1][x], y ? 0x7362 : 0x5140);
              const uint32_t a23 = __byte_perm(w[2][x], w[3][x], y ? 0x7362 : 0x5140);
              const uint32_t f[4] = {half2_of(a01), half2_of(a01 >> 16), half2_of(a23), half2_of(a23 >> 16)};
#pragma unroll
              for (int nr = 0; nr < NR; ++nr) mma16(o[nr][2 * x + y], f, p[nr][b][0], p[nr][b][1], true);
            }
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x) {                      // 2 dimensions a word: a tile
            const uint32_t f[4] = {__byte_perm(w[0][x], w[1][x], 0x5410), __byte_perm(w[0][x], w[1][x], 0x7632),
                                   __byte_perm(w[2][x], w[3][x], 0x5410), __byte_perm(w[2][x], w[3][x], 0x7632)};
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) mma16(o[nr][4 * h + x], f, p[nr][b][0], p[nr][b][1], false);
          }
        }
      }
    __syncwarp();                                            // every lane has read the stage
    if (++stage == STAGES) stage = 0, phase ^= 1;
  }
  if (__syncthreads_or(dead)) settle(a.m.status);            // a copy did not arrive: nothing more was asked for

  // this warp's sums to its part of the ring: [row][dimension]; tile j holds, in its rows g and
  // g + 8, dimensions D/8 g + 2 j and the next (8-bit), 64 (j / 4) + 8 g + 2 (j % 4) and the next (bf16)
  float* const mine = reinterpret_cast<float*>(mem + warp * C::RING);
#pragma unroll
  for (int nr = 0; nr < NR; ++nr)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = sum[nr][e];
#pragma unroll
      for (int x = 4; x < 32; x *= 2) l += __shfl_xor_sync(0xffffffffu, l, x);
      const int r = 8 * nr + 2 * c + e;
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        const int d = E4M3 ? D / 8 * g + 2 * j : 64 * (j / 4) + 8 * g + 2 * (j % 4);
        *reinterpret_cast<float2*>(mine + r * LD + d) = make_float2(o[nr][j][e], o[nr][j][2 + e]);
      }
      if (g == 0) {
        stat[warp][r] = make_float2(top[nr][e] * rf[nr][e], l);
        if constexpr (E4M3) vmax[warp][r] = voff[nr][e];
      }
    }
  __syncthreads();
  for (int i = tid; i < ROWS * D / 4; i += THREADS) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, R = r0 + r;
    if (R >= rows) break;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) m = fmaxf(m, stat[w][r].x);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    float4 x = {};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float2 ml = stat[w][r];
      const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(mem + w * C::RING) + r * LD + d);
      const float f = ex2_approx(ml.x - ref);
      // 8-bit pages: the sums stand in units of 2^(m + m')
      const float fv = E4M3 ? (ml.x == -INFINITY ? 0.f : ex2_approx(vmax[E4M3 ? w : 0][r] + (ml.x - ref))) : f;
      l = fmaf(ml.y, f, l);
      x = make_float4(fmaf(y.x, fv, x.x), fmaf(y.y, fv, x.y), fmaf(y.z, fv, x.z), fmaf(y.w, fv, x.w));
    }
    if (!E4M3 && poison) {
      // values that are not finite, of the runs where they were taken out, for the rows that see them
      const Range see = seen_by(a, t, R / a.group);
      for (int k = max(see.lo, all.lo); k < min(see.hi, all.hi); ++k) {
        const int run = k / RUN * RUN;
        if (run >= whole_lo && run + RUN <= whole_hi) {
          k = run + RUN - 1;
          continue;
        }
        const long long at = (long long)seq_page(a.m, t.n, k >> shift) * page_rows + head_row + (k & (a.m.page_tokens - 1));
        const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.m.v_pages) + at * D + d;
        const float y[4] = {__bfloat162float(v[0]), __bfloat162float(v[1]), __bfloat162float(v[2]), __bfloat162float(v[3])};
        if (!isfinite(y[0])) x.x += y[0];
        if (!isfinite(y[1])) x.y += y[1];
        if (!isfinite(y[2])) x.z += y[2];
        if (!isfinite(y[3])) x.w += y[3];
      }
    }
    if (a.cluster == 1) {
      put_result<__nv_bfloat16, D>(a, t, R, d, x, m, l);
    } else {                                                 // in place of the first warp's
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(mem) + r * LD + d) = x;
      if (d == 0) block_ml[r] = make_float2(m, l);
    }
  }
  if (a.cluster > 1) join_cluster<__nv_bfloat16, D, ROWS, THREADS>(a, t, reinterpret_cast<const float*>(mem), LD, block_ml, r0, rows);
}

template <int D, bool E4M3, int NR>
cudaError_t launch_as(const AttendArgs& a, cudaStream_t st) {
  using C = Cfg<D, E4M3, NR>;
  CUtensorMap km, vm;
  const int box = std::min(a.m.page_tokens, C::RUN);
  if (!page_map(&km, a.m, a.m.k_pages, box) || !page_map(&vm, a.m, a.m.v_pages, box)) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  return launch_pieces(rows_kernel<D, E4M3, NR>, a, THREADS, C::SMEM, done, st, km, vm);
}

template <int NR>
cudaError_t launch_rows(const AttendArgs& a, cudaStream_t st) {
  const bool e = a.m.format == EVO_CACHE_E4M3;
  if (a.m.head_dim == 64) return e ? launch_as<64, true, NR>(a, st) : launch_as<64, false, NR>(a, st);
  return e ? launch_as<128, true, NR>(a, st) : launch_as<128, false, NR>(a, st);
}

}  // namespace

cudaError_t launch_attend_rows(const AttendArgs& a, int tile_rows, cudaStream_t st) {
  return tile_rows == 8 ? launch_rows<1>(a, st) : tile_rows == 16 ? launch_rows<2>(a, st) : launch_rows<4>(a, st);
}

}  // namespace evo
