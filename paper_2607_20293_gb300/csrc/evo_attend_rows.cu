// Attention over a paged memory for few rows a key/value head (single tokens,
// short action chunks): bf16 rows, bf16 or 8-bit pages.
//
// Such a call reads every key and value once for at most 16 MT rows, so DRAM
// bounds it as long as the tensor cores and the conversion of codes keep up:
// mma.sync (1,024 multiply-adds a cycle and SM, a quarter of what tcgen05 has)
// needs 32 of the 174 cycles that 16 bf16 keys and values of 64 take to arrive,
// without padding 16 rows to tcgen05's 128.
//
// A block is 4 warps on one tile of rows and one piece of the memory.  Each warp
// takes every 4th run of 16 NB keys by itself (no barrier until the end), loads
// keys and values from global memory straight into the fragments of
// mma.m16n8k16, and keeps its own running maximum and sums; the warps' results
// are joined through shared memory.  Neither operand goes through shared memory,
// because the contraction's index may be permuted at will:
//   scores: lane (g, c) = (lane / 4, lane % 4) holds key g's values at 16 bytes
//           contiguous per step; the queries' fragments use the same permutation;
//   output: the four keys of a lane's fragment are 4c .. 4c+3 and its column g
//           stands for 8 (or 16) contiguous dimensions, one n-tile each.
// Loads are issued for the next run as soon as the registers of this one are
// used: keys after the scores, values after the output.
//
// The running maximum is lazy: the sums are rescaled only when a score passes
// the row's reference by 2^8, so the common run has one vote instead of
// reductions over lanes and a pass over the accumulators.  Weights are then at
// most 2^8, which the 16-bit operand holds with the same relative rounding.
//
// 8-bit pages: codes become fp16 exactly (one conversion for two).  A key's scale
// multiplies its column of the scores in fp32; queries are brought to fp16 by an
// exact power of two per row.  A value's scale 2^k is added to the exponent of its
// weights, 2^(s + k - m'), with a reference m' of its own, so that the fp16
// operand stays in range for any mixture of scales; the sum of weights uses
// 2^(s - m).  The weights' rounding is fp16's (2^-12 of each) there, bf16's (2^-9)
// with bf16 pages.
//
// Masks are looked at only in runs of 16 keys that some row does not see whole.
// There, keys outside the piece give zero values, and a value that is not finite
// is taken out of the product (0 * NaN would reach rows that do not see it) and
// put back at the end for the rows that see it.
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr float LAZY = 8.f;                       // log2 of how far a weight may pass 1

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

// how many keys beyond the loads of a run its registers hold, per format
template <int D, bool E4M3>
struct Frag {
  static constexpr int ROW = D * (E4M3 ? 1 : 2);   // bytes of a key or value
  static constexpr int KP = ROW / 64;              // 16-byte pieces of a key a lane holds (4 lanes a key)
  static constexpr int VB = ROW / 8;               // bytes of a value a lane holds (8 lanes a value)
  static constexpr int VP = VB == 8 ? 1 : VB / 16; // 16-byte (or one 8-byte) pieces of them
};

template <int D, bool E4M3, int MT, int NB>
__global__ void __launch_bounds__(THREADS) rows_kernel(const __grid_constant__ AttendArgs a) {
  using F = Frag<D, E4M3>;
  constexpr int RUN = 16 * NB, NT = D / 8, KS = D / 16, LD = D + 4;
  extern __shared__ __align__(16) float joined[];            // [WARPS][16 MT][LD], then the warps' maxima and sums
  float2* const stat = reinterpret_cast<float2*>(joined + WARPS * 16 * MT * LD);   // [WARPS][16 MT]
  float* const vmax = reinterpret_cast<float*>(stat + WARPS * 16 * MT);            // [WARPS][16 MT], 8-bit pages
  __shared__ int poison;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4;
  const Tile t = tile_of_block(a);
  const int rows = t.count * a.group, r0 = t.tile * 16 * MT;
  if (r0 >= rows) return;
  const int last = min(r0 + 16 * MT, rows) - 1;
  const Range first_row = seen_by(a, t, r0 / a.group), last_row = seen_by(a, t, last / a.group);
  const Range all = piece_of(a, t, {first_row.lo, last_row.hi}, RUN);
  // keys that every row of the tile sees, of this piece
  const int whole_lo = max(last_row.lo, all.lo), whole_hi = min(first_row.hi, all.hi);
  if (tid == 0) poison = 0;
  __syncthreads();

  // queries: fragments in the keys' permutation
  uint32_t q[MT][KS][4];
  float rf[MT][2];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int R = r0 + mt * 16 + hf * 8 + g;
      const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + (long long)(t.first + R / a.group) * a.ldq +
                                 (long long)(t.kv_head * a.group + R % a.group) * D;
      rf[mt][hf] = a.scale_log2;
      if constexpr (E4M3) {
        uint4 u[D / 32];                                     // values 64 h + 16 c .. + 15
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          u[i] = R < rows ? *reinterpret_cast<const uint4*>(src + 64 * (i / 2) + 16 * c + 8 * (i % 2)) : make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) top = max(top, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^(14 - e) for a largest magnitude in [2^e, 2^(e+1)), within fp32's exponents
        const int e = (int)(top >> 7);                       // e + 127
        const int up = top == 0 || e == 255 ? 0 : min(max(141 - e, -126), 126);
        const float f = __int_as_float((up + 127) << 23);
        rf[mt][hf] = a.scale_log2 * __int_as_float((127 - up) << 23);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint4 v = u[ks / 2];
          const uint32_t lo = ks % 2 ? v.z : v.x, hi = ks % 2 ? v.w : v.y;
          q[mt][ks][hf] = pack(__uint_as_float(lo << 16) * f, __uint_as_float(lo & 0xffff0000u) * f, true);
          q[mt][ks][2 + hf] = pack(__uint_as_float(hi << 16) * f, __uint_as_float(hi & 0xffff0000u) * f, true);
        }
      } else {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {                   // values 32 i + 8 c .. + 7: two steps
          const uint4 u = R < rows ? *reinterpret_cast<const uint4*>(src + 32 * i + 8 * c) : make_uint4(0, 0, 0, 0);
          q[mt][2 * i][hf] = u.x;
          q[mt][2 * i][2 + hf] = u.y;
          q[mt][2 * i + 1][hf] = u.z;
          q[mt][2 * i + 1][2 + hf] = u.w;
        }
      }
    }

  float o[MT][NT][4], sum[MT][2], top[MT][2], vtop[MT][2];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[mt][j][i] = 0.f;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) sum[mt][hf] = 0.f, top[mt][hf] = vtop[mt][hf] = -INFINITY;
  }

  uint4 kr[NB][2][F::KP];                                    // keys 4 (g / 2) + 2 i + g % 2 of the 16, i = 0, 1
  uint4 vr[NB][4][F::VP];                                    // values 4 c + i of the 16
  uint32_t kscale[NB], vscale[NB];                           // scale bytes of keys 4 c .. 4 c + 3
  const long long head_rows = a.m.page_tokens, page_rows = (long long)a.m.n_kv_head * a.m.page_tokens;
  const int shift = 31 - __clz(a.m.page_tokens), mask = a.m.page_tokens - 1;

  // row of the pool at which 16 keys from k0 start, or -1 if none of them is in the piece
  auto locate = [&](int k0) -> long long {
    if (k0 + 16 <= all.lo || k0 >= all.hi) return -1;
    return seq_page(a.m, t.n, k0 >> shift) * page_rows + t.kv_head * head_rows + (k0 & mask);
  };
  auto load_keys = [&](int b, long long at) {
    if (at >= 0) {
      const uint8_t* p = static_cast<const uint8_t*>(a.m.k_pages) + at * F::ROW;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < F::KP; ++h)
          kr[b][i][h] = *reinterpret_cast<const uint4*>(p + (4 * (g / 2) + 2 * i + g % 2) * F::ROW + 64 * h + 16 * c);
      if constexpr (E4M3) kscale[b] = *reinterpret_cast<const uint32_t*>(a.m.k_scales + at + 4 * c);
    }
  };
  auto load_values = [&](int b, long long at) {
    if (at >= 0) {
      const uint8_t* p = static_cast<const uint8_t*>(a.m.v_pages) + at * F::ROW;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < F::VP; ++h) {
          const uint8_t* s = p + (4 * c + i) * F::ROW + (F::VB == 8 ? 8 * g : 128 * h + 16 * g);
          if constexpr (F::VB == 8) {
            const uint2 u = *reinterpret_cast<const uint2*>(s);
            vr[b][i][h] = make_uint4(u.x, u.y, 0, 0);
          } else {
            vr[b][i][h] = *reinterpret_cast<const uint4*>(s);
          }
        }
      if constexpr (E4M3) vscale[b] = *reinterpret_cast<const uint32_t*>(a.m.v_scales + at + 4 * c);
    }
  };

  const int step = WARPS * RUN;
  int k0 = all.lo / RUN * RUN + warp * RUN;
  long long here[NB], next[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) here[b] = locate(k0 + 16 * b), next[b] = locate(k0 + step + 16 * b);
#pragma unroll
  for (int b = 0; b < NB; ++b) load_keys(b, here[b]);
#pragma unroll
  for (int b = 0; b < NB; ++b) load_values(b, here[b]);

  for (; k0 < all.hi; k0 += step) {
    long long after[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) after[b] = locate(k0 + 2 * step + 16 * b);
    float s[MT][NB][2][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[mt][b][i][e] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < F::KP; ++h) {
          const uint32_t w[4] = {kr[b][i][h].x, kr[b][i][h].y, kr[b][i][h].z, kr[b][i][h].w};
          if constexpr (E4M3) {                              // 4 codes a step
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t b0 = half2_of(w[j]), b1 = half2_of(w[j] >> 16);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) mma16(s[mt][b][i], q[mt][4 * h + j], b0, b1, true);
            }
          } else {                                           // 4 values in two words a step
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) mma16(s[mt][b][i], q[mt][2 * h + j], w[2 * j], w[2 * j + 1], false);
          }
        }
    // scores in base 2; column 2 c + e of n-tile i is key 4 c + 2 i + e
    float ks[NB][4], vs[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (E4M3) {
          // a value that is no number makes the key's score one: the rows that see it, and no
          // other, then hold NaN
          const uint32_t v = (vscale[b] >> (8 * j)) & 255u;
          ks[b][j] = scale_value(v == SCALE_NAN ? SCALE_NAN : (kscale[b] >> (8 * j)) & 255u);
          vs[b][j] = v == SCALE_NAN ? 0.f : (float)((int)v - 127);
        }
      }
#pragma unroll
    for (int b = 0; b < NB; ++b) load_keys(b, next[b]);

    bool raise = false;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int kb = k0 + 16 * b;
      const bool whole = kb >= whole_lo && kb + 16 <= whole_hi;
      bool drop[4] = {};                                     // values of this lane's keys that must not be multiplied
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 4; ++j) drop[j] = kb + 4 * c + j < all.lo || kb + 4 * c + j >= all.hi;
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          Range see = {0, 0};
          if (!whole) {
            const int R = r0 + mt * 16 + hf * 8 + g;
            if (R < rows) see = seen_by(a, t, R / a.group);
            see = {max(see.lo, all.lo), min(see.hi, all.hi)};
          }
          float m = -INFINITY, mv = -INFINITY;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float& x = s[mt][b][j / 2][2 * hf + j % 2];
            if constexpr (E4M3) x *= ks[b][j];
            x *= rf[mt][hf];
            if (!whole) {
              const int key = kb + 4 * c + j;
              if (key < see.lo || key >= see.hi) x = -INFINITY;
            }
            m = fmaxf(m, x);
            if constexpr (E4M3) mv = fmaxf(mv, x + vs[b][j]);
          }
          raise |= m > top[mt][hf] + LAZY;
          if constexpr (E4M3) raise |= mv > vtop[mt][hf] + LAZY;
        }
      if constexpr (E4M3) {
#pragma unroll
        for (int j = 0; j < 4; ++j) drop[j] |= ks[b][j] != ks[b][j];
        if (__any_sync(0xffffffffu, drop[0] | drop[1] | drop[2] | drop[3])) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int h = 0; h < F::VP; ++h)
              if (drop[j]) vr[b][j][h] = make_uint4(0, 0, 0, 0);
        }
      } else if (!whole) {
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int h = 0; h < F::VP; ++h) {
            uint4& u = vr[b][j][h];
            if (drop[j]) u = make_uint4(0, 0, 0, 0);
            u = make_uint4(finite_halves(u.x, &bad), finite_halves(u.y, &bad), finite_halves(u.z, &bad),
                           finite_halves(u.w, &bad));
          }
        if (bad) poison = 1;
      }
    }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          float m = top[mt][hf], mv = vtop[mt][hf];
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x = s[mt][b][j / 2][2 * hf + j % 2];
              m = fmaxf(m, x);
              if constexpr (E4M3) mv = fmaxf(mv, x + vs[b][j]);
            }
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
          if constexpr (E4M3) {
            mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, 1));
            mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, 2));
          } else {
            mv = m;
          }
          const float f = ex2_approx(top[mt][hf] - (m == -INFINITY ? 0.f : m));
          const float fv = E4M3 ? ex2_approx(vtop[mt][hf] - (mv == -INFINITY ? 0.f : mv)) : f;
          top[mt][hf] = m;
          vtop[mt][hf] = mv;
          sum[mt][hf] *= f;
#pragma unroll
          for (int j = 0; j < NT; ++j) o[mt][j][2 * hf] *= fv, o[mt][j][2 * hf + 1] *= fv;
        }
    }
    uint32_t p[MT][NB][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const float m = top[mt][hf] == -INFINITY ? 0.f : top[mt][hf];
        const float mv = vtop[mt][hf] == -INFINITY ? 0.f : vtop[mt][hf];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          float w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = s[mt][b][j / 2][2 * hf + j % 2];
            w[j] = ex2_approx(x - m);
            sum[mt][hf] += w[j];
            if constexpr (E4M3) w[j] = ex2_approx(x + (vs[b][j] - mv));
          }
          p[mt][b][hf] = pack(w[0], w[1], E4M3);
          p[mt][b][2 + hf] = pack(w[2], w[3], E4M3);
        }
      }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int h = 0; h < F::VP; ++h) {
        const uint32_t w[4][4] = {{vr[b][0][h].x, vr[b][0][h].y, vr[b][0][h].z, vr[b][0][h].w},
                                  {vr[b][1][h].x, vr[b][1][h].y, vr[b][1][h].z, vr[b][1][h].w},
                                  {vr[b][2][h].x, vr[b][2][h].y, vr[b][2][h].z, vr[b][2][h].w},
                                  {vr[b][3][h].x, vr[b][3][h].y, vr[b][3][h].z, vr[b][3][h].w}};
        if constexpr (E4M3) {
#pragma unroll
          for (int x = 0; x < (F::VB == 8 ? 2 : 4); ++x)     // 4 dimensions of each word
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint32_t a01 = __byte_perm(w[0][x], w[1][x], y ? 0x7362 : 0x5140);
              const uint32_t a23 = __byte_perm(w[2][x], w[3][x], y ? 0x7362 : 0x5140);
#pragma unroll
              for (int z = 0; z < 2; ++z) {
                const uint32_t b0 = half2_of(a01 >> (16 * z)), b1 = half2_of(a23 >> (16 * z));
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) mma16(o[mt][4 * x + 2 * y + z], p[mt][b], b0, b1, true);
              }
            }
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint32_t b0 = __byte_perm(w[0][x], w[1][x], y ? 0x7632 : 0x5410);
              const uint32_t b1 = __byte_perm(w[2][x], w[3][x], y ? 0x7632 : 0x5410);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) mma16(o[mt][8 * h + 2 * x + y], p[mt][b], b0, b1, false);
            }
        }
      }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      load_values(b, next[b]);
      next[b] = after[b];
    }
  }

  // this warp's sums to shared memory: n-tile j, column n is dimension
  // 8-bit: D/8 n + j; bf16: 64 (j / 8) + 8 n + j % 8
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      float l = sum[mt][hf];
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      const int r = mt * 16 + hf * 8 + g;
      float* dst = joined + (warp * 16 * MT + r) * LD;
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int j = 0; j < NT; j += 4) {
          const int d = E4M3 ? D / 8 * (2 * c + e) + j : 64 * (j / 8) + 8 * (2 * c + e) + j % 8;
          *reinterpret_cast<float4*>(dst + d) = make_float4(o[mt][j][2 * hf + e], o[mt][j + 1][2 * hf + e],
                                                            o[mt][j + 2][2 * hf + e], o[mt][j + 3][2 * hf + e]);
        }
      if (c == 0) {
        stat[warp * 16 * MT + r] = make_float2(top[mt][hf], l);
        if constexpr (E4M3) vmax[warp * 16 * MT + r] = vtop[mt][hf];
      }
    }
  __syncthreads();
  for (int i = tid; i < 16 * MT * D / 4; i += THREADS) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, R = r0 + r;
    if (R >= rows) continue;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) m = fmaxf(m, stat[w * 16 * MT + r].x);
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    float4 x = {};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float2 ml = stat[w * 16 * MT + r];
      const float4 y = *reinterpret_cast<const float4*>(joined + (w * 16 * MT + r) * LD + d);
      const float f = ex2_approx(ml.x - base);
      // 8-bit pages: the sums stand in units of 2^m'
      const float fv = E4M3 ? (ml.x == -INFINITY ? 0.f : ex2_approx(vmax[w * 16 * MT + r] - base)) : f;
      l = fmaf(ml.y, f, l);
      x = make_float4(fmaf(y.x, fv, x.x), fmaf(y.y, fv, x.y), fmaf(y.z, fv, x.z), fmaf(y.w, fv, x.w));
    }
    if (!E4M3 && poison) {
      // values that are not finite, of the runs where they were taken out, for the rows that see them
      const Range see = seen_by(a, t, R / a.group);
      for (int k = max(see.lo, all.lo); k < min(see.hi, all.hi); ++k) {
        const int kb = k & ~15;
        if (kb >= whole_lo && kb + 16 <= whole_hi) {
          k = kb + 15;
          continue;
        }
        const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.m.v_pages) + (locate(kb) + (k - kb)) * D + d;
        const float y[4] = {__bfloat162float(v[0]), __bfloat162float(v[1]), __bfloat162float(v[2]), __bfloat162float(v[3])};
        if (!isfinite(y[0])) x.x += y[0];
        if (!isfinite(y[1])) x.y += y[1];
        if (!isfinite(y[2])) x.z += y[2];
        if (!isfinite(y[3])) x.w += y[3];
      }
    }
    const int row = t.first + R / a.group, head = t.kv_head * a.group + R % a.group;
    if (a.splits == 1) {
      const float f = l == 0.f ? 0.f : 1.f / l;
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.out) + row * a.ldo + (long long)head * D + d;
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack(x.x * f, x.y * f, false), pack(x.z * f, x.w * f, false));
    } else {
      const long long at = part_index(a, t.split, row, head);
      *reinterpret_cast<float4*>(a.part + at * D + d) = x;
      if (d == 0) a.ml[at] = make_float2(m, l);
    }
  }
}

template <int D, bool E4M3, int MT, int NB>
cudaError_t launch_as(const AttendArgs& a, unsigned grid, cudaStream_t st) {
  const auto k = rows_kernel<D, E4M3, MT, NB>;
  constexpr int smem = WARPS * 16 * MT * (D + 4) * 4 + WARPS * 16 * MT * 12;
  const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  k<<<grid, THREADS, smem, st>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_rows(const AttendArgs& a, int mt, cudaStream_t st) {
  const unsigned grid = (unsigned)((long long)a.m.n_seq * a.m.n_kv_head * a.tiles * a.splits);
  const bool e = a.m.format == EVO_CACHE_E4M3;
  if (a.m.head_dim == 64) {
    if (mt == 1) return e ? launch_as<64, true, 1, 2>(a, grid, st) : launch_as<64, false, 1, 1>(a, grid, st);
    return e ? launch_as<64, true, 2, 2>(a, grid, st) : launch_as<64, false, 2, 1>(a, grid, st);
  }
  if (mt == 1) return e ? launch_as<128, true, 1, 1>(a, grid, st) : launch_as<128, false, 1, 1>(a, grid, st);
  return e ? launch_as<128, true, 2, 1>(a, grid, st) : launch_as<128, false, 2, 1>(a, grid, st);
}

}  // namespace evo
