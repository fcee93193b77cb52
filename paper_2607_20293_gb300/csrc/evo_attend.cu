// Attention over a paged memory: the fp32 kernel for many rows, the expansion of
// 8-bit pages, the join of split memories and the choice among the kernels:
//
//   rows a key/value head    bf16 rows                          fp32 rows
//   up to 32 (fp32: 16)      evo_attend_rows.cu (mma.sync)      evo_attend_f32.cu
//   more                     evo_attend_tiles.cu (tcgen05);     attend_kernel
//                            8-bit pages from 65 rows on
// (8-bit pages of 33 to 64 rows: two tiles of evo_attend_rows.cu).
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(s_j - max s),  s_j = scale log2(e) <q, k_j>
//
// over the keys j that the row sees, in one pass with a running maximum and sum
// (a row that sees none is zero).  A memory split over several blocks leaves each
// piece's maximum, sum and unnormalised values, which a second kernel joins.
//
// fp32 kernel: a warp takes 16 rows, a block 64 (or 32), and 64 keys at a time.  fp32 multiply-adds
// bounded its first form (a register tile a thread: 1,024 rows over 4,096 keys of 64, 8 heads,
// 255 us = 34 TFLOP/s, of keys of 128 541 us).  So a number is split into two of 11 bits and a product
// taken as three of tf32, off by 2^-19 of itself at most (2 x 2^-21 for what the parts leave out, 2^-22
// for the product of the low parts): mma.sync has 512 of these multiply-adds a cycle and SM, 170 of
// the fp32 ones, against 85 to 110 of the plain ones: 170 us = 50 TFLOP/s and 338 us.  The matrix unit cuts
// its sums off, so products of high and of low parts have sums of their own, and those of 32 keys are added
// to the output in fp32: over 2,302 keys the result is off by 3.8e-7 of its norm (all in one sum, which takes
// 6 % less time, 2.3e-6; PyTorch's fp32 products 9e-7).  Codes are exact in 11 bits and take two products.  What bounds
// it now is issue: a warp's 384 products of a block of keys (51 % of the tensor pipe's time) stand beside some
// 2,100 other instructions, half of them the split of keys and values, which do not overlap much with them.
// Tiles of 32 rows a warp split half as often, but spill (194 us where 16 rows took 203).
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "evo_attend.cuh"
#include "evo_mem_ptx.cuh"
#include "evo_quant.cuh"

namespace evo {
namespace {

constexpr int BN = 64, JOIN_THREADS = 256;
// from this many rows a key/value head on, 8-bit pages are written out as bf16 pages for the tcgen05
// kernel (16 sequences of 8,192 keys of 64, us with / without: 64 rows 123 / 103, 96 rows 123 / 144,
// 256 rows 148 / 331; of 128: 239 / 191, 240 / 272, 251 / 638), while they fit this many bytes
constexpr int EXPAND_ROWS = 65;
constexpr long long EXPAND_MOST = 4ll << 30;

template <int D, int WARPS>
struct Smem {
  static constexpr int BM = 16 * WARPS;
  float q[BM * D], k[BN * D], v[BN * D];
  int row[2][BN];               // rows of the pool that hold the keys of this block and the next, or -1
};
// where 4 floats d .. d + 3 of row r lie, so that the 8 lanes of a phase meet 8 different chunks of 128
// bytes: 2 rows x 4 chunks of queries and keys, 4 pairs of rows x 2 chunks of values
template <int D>
__device__ __forceinline__ int key_at(int r, int d) { return r * D + (d ^ (r & 1) << 4); }
template <int D>
__device__ __forceinline__ int value_at(int r, int d) { return r * D + (d ^ (r >> 1 & 3) << 3); }

__device__ __forceinline__ void copy16(float* dst, const float* src, bool on) {   // zeros where it is off
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
               "r"(on ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }   // all but the last N groups

// x as two numbers of 11 bits: hi, x rounded to nearest, and lo, what is left of it, cut off:
// hi + lo = x (1 + e), |e| <= 2^-21.  In integers: a conversion has an eighth of their rate
struct Split { uint32_t hi, lo; };
__device__ __forceinline__ Split split(float x) {
  Split s;
  s.hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
  s.lo = __float_as_uint(x - __uint_as_float(s.hi)) & 0xffffe000u;
  return s;
}
__device__ __forceinline__ void mma8(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// four tiles (d + r)[i] += a b_i of fp32 numbers: the products of the high parts to d, those with a low
// part to r, for the matrix unit cuts its sums off and loses half a step of d with each; CODES: b is exact in
// 11 bits.  A product does not wait for the one before it on its tile
template <bool CODES>
__device__ __forceinline__ void mma_split(float (*d)[4], float (*r)[4], const uint32_t (&ah)[4], const uint32_t (&al)[4], float4 b0,
                                          float4 b1) {
  const float x[4] = {b0.x, b0.y, b0.z, b0.w}, y[4] = {b1.x, b1.y, b1.z, b1.w};
  uint32_t xh[4], xl[4], yh[4], yl[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const Split u = split(x[i]), w = split(y[i]);
    xh[i] = CODES ? __float_as_uint(x[i]) : u.hi, xl[i] = u.lo;
    yh[i] = CODES ? __float_as_uint(y[i]) : w.hi, yl[i] = w.lo;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) mma8(d[i], ah, xh[i], yh[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) mma8(r[i], al, xh[i], yh[i]);
  if constexpr (!CODES)
#pragma unroll
    for (int i = 0; i < 4; ++i) mma8(r[i], ah, xl[i], yl[i]);
}

// (top, sum, o) joined with another piece's
__device__ __forceinline__ void join(float& top, float& sum, float4& o, float2 ml, float4 p) {
  const float now = fmaxf(top, ml.x), base = now == -INFINITY ? 0.f : now;
  const float f = exp2f(top - base), g = exp2f(ml.x - base);
  top = now;
  sum = sum * f + ml.y * g;
  o = make_float4(o.x * f + p.x * g, o.y * f + p.y * g, o.z * f + p.z * g, o.w * f + p.w * g);
}

// A row whose sums are not finite, once more with plain fp32 products (an infinity's low part is no
// number, so that infinities that a row sees, and NaN in tokens that it does not see, spoil the split
// form).  A warp takes the row: a lane a key, then a lane D / 32 dimensions.
template <int D, int FORMAT>
__device__ __noinline__ void row_again(const AttendArgs& a, const Tile& t, const float* q, int r, Range see, float& top, float& sum,
                                       float (&o)[D / 32]) {
  constexpr bool CODES = FORMAT == EVO_CACHE_E4M3;
  const int lane = threadIdx.x & 31, page_tokens = a.m.page_tokens;
  top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = 0.f;
  for (int k0 = see.lo; k0 < see.hi; k0 += 32) {
    const int key = min(k0 + lane, see.hi - 1);
    const long long at =
        ((long long)seq_page(a.m, t.n, key / page_tokens) * a.m.n_kv_head + t.kv_head) * page_tokens + key % page_tokens;
    float s = 0.f;
    for (int d = 0; d < D; d += 4) {
      float4 k;
      if constexpr (CODES) k = codes4(*reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.m.k_pages) + at * D + d));
      else k = *reinterpret_cast<const float4*>(static_cast<const float*>(a.m.k_pages) + at * D + d);
      const float4 x = *reinterpret_cast<const float4*>(q + key_at<D>(r, d));
      s = fmaf(x.x, k.x, fmaf(x.y, k.y, fmaf(x.z, k.z, fmaf(x.w, k.w, s))));
    }
    if constexpr (CODES) s *= scale_value(a.m.k_scales[at]);
    s = k0 + lane < see.hi ? s * a.scale_log2 : -INFINITY;
    float m = s;
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
    m = fmaxf(m, top);
    const float base = m == -INFINITY ? 0.f : m, keep = exp2f(top - base), p = exp2f(s - base);
    top = m;
    sum = sum * keep + p;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] *= keep;
    for (int j = 0; j < min(32, see.hi - k0); ++j) {
      const float w = __shfl_sync(0xffffffffu, p, j);
      const long long from = __shfl_sync(0xffffffffu, at, j);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        float v;
        if constexpr (CODES)
          v = codes4(static_cast<const uint8_t*>(a.m.v_pages)[from * D + lane + 32 * i]).x * scale_value(a.m.v_scales[from]);
        else
          v = static_cast<const float*>(a.m.v_pages)[from * D + lane + 32 * i];
        o[i] = fmaf(w, v, o[i]);
      }
    }
  }
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
}

template <int D, int FORMAT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, (D == 64 ? 3 : 2) * (4 / WARPS)) attend_kernel(const __grid_constant__ AttendArgs a) {
  constexpr bool CODES = FORMAT == EVO_CACHE_E4M3;
  constexpr int THREADS = 32 * WARPS, BM = 16 * WARPS, NT = BN / 8, DT = D / 8;
  extern __shared__ __align__(16) uint8_t raw[];
  using S = Smem<D, WARPS>;
  S& sm = *reinterpret_cast<S*>(raw);
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4;
  const Tile t = tile_of_block(a);
  const int rows = t.count * a.group, r0 = t.tile * BM;
  if (r0 >= rows) return;
  const int last = min(r0 + BM, rows) - 1;
  const Range first_row = seen_by(a, t, r0 / a.group), last_row = seen_by(a, t, last / a.group);
  const Range all = piece_of(a, t, {first_row.lo, last_row.hi}, BN);
  const int whole_lo = max(last_row.lo, all.lo), whole_hi = min(first_row.hi, all.hi);
  const int shift = 31 - __clz(a.m.page_tokens);

  const auto look_up = [&](int k0) {               // the pool's rows for 64 keys from k0 on, a thread each
    if (tid >= BN) return;
    const int key = k0 + tid;
    int row = -1;
    if (key >= all.lo && key < all.hi)
      row = (seq_page(a.m, t.n, key >> shift) * a.m.n_kv_head + t.kv_head) * a.m.page_tokens + (key & (a.m.page_tokens - 1));
    sm.row[k0 / BN & 1][tid] = row;
  };
  // 64 keys or values from k0 on (zeros outside the piece): fp32 on their way, a group of copies;
  // 8-bit ones as numbers
  const auto bring = [&](int k0, const void* pages, const uint8_t* scales, float* tile, auto place) {
    const int* row = sm.row[k0 / BN & 1];
    if constexpr (CODES) {
#pragma unroll 4
      for (int i = tid; i < BN * D / 16; i += THREADS) {
        const int r = i / (D / 16), d = i % (D / 16) * 16, at = row[r];
        uint4 u = make_uint4(0, 0, 0, 0);
        float f = 0.f;
        if (at >= 0) u = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(pages) + (long long)at * D + d), f = scale_value(scales[at]);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 x = codes4(w[e]);
          *reinterpret_cast<float4*>(tile + place(r, d + 4 * e)) = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
        }
      }
    } else {
#pragma unroll 4
      for (int i = tid; i < BN * D / 4; i += THREADS) {
        const int r = i / (D / 4), d = i % (D / 4) * 4, at = row[r];
        copy16(tile + place(r, d), static_cast<const float*>(pages) + (long long)max(at, 0) * D + d, at >= 0);
      }
      copies_close();
    }
  };
  const auto bring_k = [&](int k0) { bring(k0, a.m.k_pages, a.m.k_scales, sm.k, key_at<D>); };
  const auto bring_v = [&](int k0) { bring(k0, a.m.v_pages, a.m.v_scales, sm.v, value_at<D>); };
  int k0 = all.lo / BN * BN;
  look_up(k0);
  __syncthreads();
  if (k0 < all.hi) bring_k(k0), bring_v(k0);

  for (int i = tid; i < BM * D / 4; i += THREADS) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, R = r0 + r;
    float4 x = {};
    if (R < rows)
      x = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + (t.first + R / a.group) * a.ldq +
                                           (long long)(t.kv_head * a.group + R % a.group) * D + d);
    *reinterpret_cast<float4*>(&sm.q[key_at<D>(r, d)]) = x;
  }
  Range seen[2];                                   // rows g and g + 8 of the warp's 16
  float mx[2], sum[2], o[DT][4];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int R = r0 + 16 * warp + g + 8 * e;
    seen[e] = R < rows ? seen_by(a, t, R / a.group) : Range{0, 0};
    seen[e] = {max(seen[e].lo, all.lo), min(seen[e].hi, all.hi)};
    mx[e] = -INFINITY;
    sum[e] = 0.f;
  }
#pragma unroll
  for (int j = 0; j < DT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[j][e] = 0.f;

  const bool busy = r0 + 16 * warp < rows;         // a warp without rows only copies
  for (; k0 < all.hi; k0 += BN) {
    const bool whole = k0 >= whole_lo && k0 + BN <= whole_hi, more = k0 + BN < all.hi;
    if (more) look_up(k0 + BN);
    copies_wait<1>();                              // the keys (their copies are older than the values')
    __syncthreads();
    // s[n]: keys 8 n + 2 c, 8 n + 2 c + 1 of rows g (0, 1) and g + 8 (2, 3).  A contraction's index may be
    // permuted at will: a lane's four dimensions 16 h + 4 c .. + 3 are its places c, c + 4 of two steps
    float s[NT][4], low[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = low[n][e] = 0.f;
#pragma unroll 1
    for (int h = busy ? 0 : D / 16; h < D / 16; ++h) {
      const float4 x = *reinterpret_cast<const float4*>(&sm.q[key_at<D>(16 * warp + g, 16 * h + 4 * c)]);
      const float4 y = *reinterpret_cast<const float4*>(&sm.q[key_at<D>(16 * warp + g + 8, 16 * h + 4 * c)]);
      const Split q[2][4] = {{split(x.x), split(y.x), split(x.y), split(y.y)}, {split(x.z), split(y.z), split(x.w), split(y.w)}};
      const uint32_t ah[2][4] = {{q[0][0].hi, q[0][1].hi, q[0][2].hi, q[0][3].hi}, {q[1][0].hi, q[1][1].hi, q[1][2].hi, q[1][3].hi}};
      const uint32_t al[2][4] = {{q[0][0].lo, q[0][1].lo, q[0][2].lo, q[0][3].lo}, {q[1][0].lo, q[1][1].lo, q[1][2].lo, q[1][3].lo}};
#pragma unroll
      for (int n = 0; n < NT; n += 4) {
        float4 k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = *reinterpret_cast<const float4*>(&sm.k[key_at<D>(8 * (n + i) + g, 16 * h + 4 * c)]);
        mma_split<CODES>(s + n, low + n, ah[0], al[0], make_float4(k[0].x, k[1].x, k[2].x, k[3].x),
                         make_float4(k[0].y, k[1].y, k[2].y, k[3].y));
        mma_split<CODES>(s + n, low + n, ah[1], al[1], make_float4(k[0].z, k[1].z, k[2].z, k[3].z),
                         make_float4(k[0].w, k[1].w, k[2].w, k[3].w));
      }
    }
    __syncthreads();                               // every warp has read the keys
    if (more) bring_k(k0 + BN);
    else copies_close();                           // an empty group, so that the count of groups stays
    if (busy)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float& x = s[n][2 * e + i];
          x = (x + low[n][2 * e + i]) * a.scale_log2;
          const int key = k0 + 8 * n + 2 * c + i;
          if (!whole && (key < seen[e].lo || key >= seen[e].hi)) x = -INFINITY;
          top = fmaxf(top, x);
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float now = fmaxf(mx[e], top), base = now == -INFINITY ? 0.f : now;
      const float keep = ex2_approx(mx[e] - base);
      mx[e] = now;
      float add = 0.f;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float& x = s[n][2 * e + i];
          x = ex2_approx(x - base);
          add += x;
        }
      sum[e] = sum[e] * keep + add;                // this lane's keys; joined at the end
#pragma unroll
      for (int j = 0; j < DT; ++j) o[j][2 * e] *= keep, o[j][2 * e + 1] *= keep;
    }
    copies_wait<1>();                              // the values
    __syncthreads();
    // weights enter as they left the scores: keys 2 c, 2 c + 1 of 8 are places c, c + 4.  Tile 4 x + y of o
    // holds dimensions 32 x + 8 c + y (0, 2) and 32 x + 8 c + 4 + y (1, 3) of rows g and g + 8
    // The sums of 32 keys are added to o in fp32 (sums over a long memory in the matrix unit would fall behind by a
    // half step each: 6e-6 of the values over 16,000 keys)
    if (busy)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint32_t ph[NT / 2][4], pl[NT / 2][4];
#pragma unroll
      for (int n = 0; n < NT / 2; ++n) {
        const float(&w)[4] = s[half * (NT / 2) + n];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Split u = split(w[e % 2 * 2 + e / 2]);
          ph[n][e] = u.hi, pl[n][e] = u.lo;
        }
      }
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        float d[4][4] = {}, r[4][4] = {};
#pragma unroll
        for (int n = 0; n < NT / 2; ++n) {
          const int key = 8 * (half * (NT / 2) + n) + 2 * c;
          const float4 u = *reinterpret_cast<const float4*>(&sm.v[value_at<D>(key, 32 * x + 4 * g)]);
          const float4 w = *reinterpret_cast<const float4*>(&sm.v[value_at<D>(key + 1, 32 * x + 4 * g)]);
          mma_split<CODES>(d, r, ph[n], pl[n], u, w);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[4 * x + y][e] += d[y][e] + r[y][e];
      }
    }
    __syncthreads();                               // every warp has read the values
    if (more) bring_v(k0 + BN);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 1);
    sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 2);
  }
  const auto place = [&](int R, long long& at) {   // where a row's sums go
    const int row = t.first + R / a.group, head = t.kv_head * a.group + R % a.group;
    at = part_index(a, t.split, row, head);
    return a.splits > 1 ? a.part + at * D : static_cast<float*>(a.out) + row * a.ldo + (long long)head * D;
  };
  uint32_t again = 0;                              // the warp's rows whose sums are not finite, a bit each
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    float bad = sum[e] * 0.f;                      // NaN if the sum or a value is not finite
#pragma unroll
    for (int j = 0; j < DT; ++j) bad += o[j][2 * e] * 0.f + o[j][2 * e + 1] * 0.f;
    const uint32_t lanes = __ballot_sync(0xffffffffu, bad != 0.f && r0 + 16 * warp + g + 8 * e < rows);
#pragma unroll
    for (int i = 0; i < 8; ++i) again |= (lanes >> (4 * i) & 15u ? 1u : 0u) << (8 * e + i);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int R = r0 + 16 * warp + g + 8 * e;
    if (R >= rows || (again >> (8 * e + g) & 1)) continue;
    const float f = a.splits > 1 ? 1.f : sum[e] == 0.f ? 0.f : 1.f / sum[e];
    long long at;
    float* dst = place(R, at);
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        *reinterpret_cast<float4*>(dst + 32 * x + 8 * c + 4 * i) =
            make_float4(o[4 * x][2 * e + i] * f, o[4 * x + 1][2 * e + i] * f, o[4 * x + 2][2 * e + i] * f, o[4 * x + 3][2 * e + i] * f);
    if (a.splits > 1 && c == 0) a.ml[at] = make_float2(mx[e], sum[e]);
  }
  for (; again; again &= again - 1) {
    const int r = 16 * warp + __ffs(again) - 1, R = r0 + r;
    Range see = seen_by(a, t, R / a.group);
    see = {max(see.lo, all.lo), min(see.hi, all.hi)};
    float top, l, x[D / 32];
    row_again<D, FORMAT>(a, t, sm.q, r, see, top, l, x);
    const float f = a.splits > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
    long long at;
    float* dst = place(R, at);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) dst[lane + 32 * i] = x[i] * f;
    if (a.splits > 1 && lane == 0) a.ml[at] = make_float2(top, l);
  }
}

// joins the pieces: D / 4 lanes a (row, head), or several such groups that share its
// pieces (groups > 1: few outputs of many pieces would else wait out one load after the other)
template <typename T, int D>
__global__ void __launch_bounds__(JOIN_THREADS) join_kernel(const __grid_constant__ AttendArgs a, int groups) {
  constexpr int LANES = D / 4, AT_ONCE = JOIN_THREADS / LANES, BATCH = 4;
  __shared__ float4 os[AT_ONCE][LANES];
  __shared__ float2 mls[AT_ONCE];
  const int slot = threadIdx.x / LANES, lane = threadIdx.x % LANES, d = lane * 4, group = slot % groups;
  const long long i = (long long)blockIdx.x * (AT_ONCE / groups) + slot / groups;
  const int row = (int)(i / a.m.n_head), head = (int)(i % a.m.n_head);
  const int parts = a.splits / a.cluster;
  tc::pdl_wait();
  bool on = row < a.rows;
  if (on && a.m.starts) on = row >= a.m.starts[0] && row < a.m.starts[a.m.n_seq];
  float top = -INFINITY, sum = 0.f;
  float4 o = {};
  if (on)
    for (int s0 = group; s0 < parts; s0 += groups * BATCH) {
      float2 ml[BATCH];
      float4 p[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int s = s0 + j * groups;
        ml[j] = make_float2(-INFINITY, 0.f);
        p[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s < parts) {
          const long long at = part_index(a, s, row, head);
          ml[j] = a.ml[at];
          p[j] = *reinterpret_cast<const float4*>(a.part + at * D + d);
        }
      }
#pragma unroll
      for (int j = 0; j < BATCH; ++j) join(top, sum, o, ml[j], p[j]);
    }
  if (groups > 1) {
    os[slot][lane] = o;
    if (lane == 0) mls[slot] = make_float2(top, sum);
    __syncthreads();
    if (group == 0)
      for (int g = 1; g < groups; ++g) join(top, sum, o, mls[slot + g], os[slot + g][lane]);
    on = on && group == 0;
  }
  if (!on) return;
  store_out(static_cast<T*>(a.out) + row * a.ldo + (long long)head * D + d, o, sum == 0.f ? 0.f : 1.f / sum);
}

// 8-bit pages of every sequence as bf16 pages n * cols + i (i < cols: what max_len tokens fill),
// keys and values: a power of two times a code is exact in bf16 (but for steps below 2^-133).  16 codes a thread.  Pages that no row
// sees are left out: their entries may name nothing (pages that left the window and were dropped).
template <int D>
__global__ void __launch_bounds__(JOIN_THREADS) expand_kernel(const __grid_constant__ AttendArgs a, int cols, __nv_bfloat16* k,
                                                              __nv_bfloat16* v, int* table) {
  const evo_memory& m = a.m;
  const int page = blockIdx.x, n = page / cols, i = page % cols;
  if (threadIdx.x == 0 && blockIdx.y == 0) table[page] = page;
  const SeqRows s = seq_rows(m, n, a.rows, a.max_new);
  const Tile t{n, 0, 0, 0, s.first, s.count, seq_len(m, n, a.max_len)};
  const long long at = (long long)i * m.page_tokens;
  if (s.count == 0 || at >= t.len || at + m.page_tokens <= seen_by(a, t, 0).lo) return;
  const long long head_rows = (long long)m.n_kv_head * m.page_tokens, from = seq_page(m, n, i) * head_rows, to = page * head_rows;
  const uint8_t* codes = static_cast<const uint8_t*>(blockIdx.y ? m.v_pages : m.k_pages);
  const uint8_t* scales = blockIdx.y ? m.v_scales : m.k_scales;
  __nv_bfloat16* out = blockIdx.y ? v : k;
  for (int x = threadIdx.x; x < head_rows * (D / 16); x += JOIN_THREADS) {
    const int r = x / (D / 16), d = x % (D / 16) * 16;
    const uint4 c = *reinterpret_cast<const uint4*>(codes + (from + r) * D + d);
    const float f = scale_value(scales[from + r]);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 y = codes4(w[e]);
      const __nv_bfloat162 a = __floats2bfloat162_rn(y.x * f, y.y * f), b = __floats2bfloat162_rn(y.z * f, y.w * f);
      h[2 * e] = *reinterpret_cast<const uint32_t*>(&a);
      h[2 * e + 1] = *reinterpret_cast<const uint32_t*>(&b);
    }
    uint4* dst = reinterpret_cast<uint4*>(out + (to + r) * D + d);
    dst[0] = make_uint4(h[0], h[1], h[2], h[3]);
    dst[1] = make_uint4(h[4], h[5], h[6], h[7]);
  }
}

template <int D, int FORMAT, int WARPS>
cudaError_t launch_f32_as(const AttendArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  return launch_pieces(attend_kernel<D, FORMAT, WARPS>, a, 32 * WARPS, (int)sizeof(Smem<D, WARPS>), done, st);
}

template <int D, int WARPS>
cudaError_t launch_f32(const AttendArgs& a, cudaStream_t st) {
  return a.m.format == EVO_CACHE_E4M3 ? launch_f32_as<D, EVO_CACHE_E4M3, WARPS>(a, st) : launch_f32_as<D, EVO_CACHE_F32, WARPS>(a, st);
}

template <typename T, int D>
cudaError_t launch_join(const AttendArgs& a, cudaStream_t st) {
  constexpr int AT_ONCE = JOIN_THREADS / (D / 4);
  const long long outputs = (long long)a.rows * a.m.n_head;
  int groups = 1;                                  // 16 pieces a group, while the GPU has threads to spare
  while (groups < AT_ONCE && groups * 16 < a.splits / a.cluster && outputs * groups < 152 * 8 * AT_ONCE) groups *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = (unsigned)((outputs * groups + AT_ONCE - 1) / AT_ONCE);
  cfg.blockDim = JOIN_THREADS;
  cfg.stream = st;
  // The join may start once every block of the pieces has ended, before what they wrote is visible to all, and
  // waits for that; none of them lets it start sooner
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, join_kernel<T, D>, a, groups);
}

// Pieces of an item for the kernels of many rows: as many as leave the fullest SM least to do, in keys: its
// blocks times (a piece's keys, and what a block costs beside them).
//   tcgen05: a block a SM; 450 keys, or 1,100 where the pieces are joined, which are of 512 keys at least
//     (100 items of 256 rows over 16,000 keys of 64: 148 us in one piece, 122 in 3, 143 in 4; over 4,000 49, 56, 68)
//   fp32: blocks of 64 keys and 100 beside them, and an SM with few blocks is slower at them (256 items of
//     64 rows over 8,000 keys of 64: 667 us in 2 pieces, which fill the places, 563 in 7; 96 over 700: 39
//     us in 3, 48 in 6).  Up to 32 rows leave half the warps without any: as many blocks as there are places
//     (96 items of 20 rows over 2,000 keys: 55 us in 6 pieces, 62 in 4), of 128 keys at least (8 items over 700: 17 us in 6, 19 in 10)
int pieces_of(bool tiles, long long blocks, long long rows, int max_len) {
  const bool half = !tiles && rows <= 32;
  const int most = std::min(64, std::max(1, max_len / (tiles ? 512 : half ? 128 : 64)));
  if (half) return (int)std::max(1ll, std::min((long long)most, 152 * 4 / blocks));
  int best = 1;
  double least = 1e300;
  for (int s = 1; s <= most; ++s) {
    const double each = (double)((blocks * s + 151) / 152), keys = (double)max_len / s;
    const double cost = tiles ? each * (keys + (s == 1 ? 450 : 1100))
                              : each * (64 * std::ceil(keys / 64) + 100) * (each == 1 ? 1.5 : each == 2 ? 1.07 : each == 3 ? 1.06 : 1);
    if (cost < least) least = cost, best = s;
  }
  return best;
}

}  // namespace

AttendPlan plan_attend(const evo_memory& m, int rows, int max_new, int max_len, int causal, int window) {
  AttendPlan p;
  const long long all = (long long)max_new * (m.n_head / m.n_kv_head);
  const bool f32 = m.dtype == EVO_DTYPE_F32, few = all <= (f32 ? 16 : 32);
  // Many rows: 8-bit pages are written out as bf16 pages once, so that the tensor cores read them
  // as they lie
  const long long cols = (max_len + m.page_tokens - 1) / m.page_tokens;
  const long long expanded = 4ll * m.n_seq * cols * m.n_kv_head * m.page_tokens * m.head_dim;
  const bool expand = !f32 && m.format == EVO_CACHE_E4M3 && all >= EXPAND_ROWS && expanded <= EXPAND_MOST && cols > 0;
  const bool tiles = !f32 && !few && (m.format == EVO_CACHE_BF16 || expand);
  p.expand = expand ? (int)cols : 0;
  p.kernel = f32 ? (few ? ATTEND_F32_ROWS : ATTEND_F32) : tiles ? ATTEND_TILES : ATTEND_ROWS;
  if (tiles)
    p.tile_rows = 256;
  else if (!f32)
    p.tile_rows = all <= 8 ? 8 : all <= 16 ? 16 : 32;
  else if (few)   // 4 rows a tile while that fills the GPU sooner (3 x 16 rows over 333 keys: 8.3 us against 12.4 with 16)
    p.tile_rows = all == 1 ? 1 : all <= 4 || (long long)m.n_seq * m.n_kv_head < 152 ? 4 : 16;
  else
    // 64 rows a block, of which up to 32 idle; blocks of 32 where there are items enough to fill the GPU with them
    // (64 x 32 rows over 4,000 keys of 64: 404 us against 581; of 128: 928 against 1,284, but 8-bit ones 1,658
    // against 1,234; 2 x 32 rows over 500 keys of 128: 28.8 against 24.7)
    p.tile_rows = all <= 32 && (m.head_dim == 64 || m.format == EVO_CACHE_F32) && (long long)m.n_seq * m.n_kv_head >= 152 ? 32 : 64;
  p.tiles = (int)((all + p.tile_rows - 1) / p.tile_rows);
  // keys that a tile's rows see: a window's, and one more a token behind the first where it moves with the rows.
  // Pieces by these, by all 16,000 keys: one token, window 256, 5.3 and 9.4 us; by all 8,192: 64 tokens, window 512,
  // 18.8 and 27.1 (8 x 4 fp32 tokens of 16 heads, keys of 128, window 128: 11.4 and 9.1)
  const int group = m.n_head / m.n_kv_head, moves = causal ? std::min(max_new, p.tile_rows / group + 1) : 0;
  const int keys = window ? (int)std::min<long long>(max_len, (long long)window + moves) : max_len;
  const long long blocks = (long long)m.n_seq * m.n_kv_head * p.tiles;
  p.cluster = 1;
  if (p.kernel == ATTEND_ROWS || p.kernel == ATTEND_F32_ROWS) {
    // Pieces of few items: as many as are resident at once, joined by the blocks of a cluster of up to 8
    // without a second kernel.  Of the 2, 3 or 6 blocks that a SM holds, whole clusters of up to 5 find at
    // least 288, 432 or 860 places, of up to 8 at least 264, 400 or 800; one cluster more is a wave of its own (56
    // items over 16,000 8-bit keys: 38 us in 6 pieces, 49 in 8; 65 over 12,000: 27 in 6, 39 in 7).
    // Long memories of fewer items take several clusters an item, whose results a kernel joins (8 items
    // over 16,389 keys: 26.7 us in 8 pieces, 16.5 in 40, and 20 in 57 without clusters; over 4,096 keys
    // 10.4 in 8, 12.4 in 24).
    const bool codes = m.format == EVO_CACHE_E4M3, wide = m.head_dim == 128;
    const int a_sm = f32 ? (p.tile_rows == 16 ? 2 : codes && !wide ? 6 : 3) : wide && (!codes || p.tile_rows == 32) ? 2 : 3;
    const long long places5 = a_sm == 2 ? 288 : a_sm == 3 ? 432 : 860, places8 = a_sm == 2 ? 264 : a_sm == 3 ? 400 : 800;
    if (2 * blocks <= places5) {
      const long long most = std::max(1, keys / (f32 ? 64 : 128));
      p.cluster = (int)std::min({8ll, std::max(std::min(5ll, places5 / blocks), places8 / blocks), most});
      const long long more = p.cluster == 8 ? std::min({8ll, places8 / (8 * blocks), keys / 2048ll}) : 1;
      p.splits = p.cluster * (int)std::max(1ll, more);
    } else {
      // More: several waves, so that sequences of different lengths even out (240 items over 16,000 keys:
      // 157 us in one piece, 116 in 7; 64 ragged sequences 134 us, in clusters 147), of pieces that are
      // worth the kernel that joins them (over 2,000 keys 26 us in one, 33 in 7).  Tiles of 32 rows pay
      // 10 us a wave of further blocks (64 ragged sequences to 4,099 keys: 90.4 us in one piece, 93.2 in two, though
      // 114 and 107 where all have 4,096; 45 of 16,000: 255 and 235).
      const long long most = std::max(1, keys / 1024);
      const long long want = p.tile_rows == 32 ? 900 / blocks : (1824 + blocks / 2) / blocks;
      p.splits = (int)std::max(1ll, std::min({most, want, 64ll}));
    }
  } else {
    // A window: the tcgen05 kernel's pieces as without one, but of 256 keys at least (4 x 256 rows of 16,000 keys of
    // 64, window 1,024: 20.0 us, 27.3 in one piece; 64 rows, window 128: 9.1 us, 15.8 in pieces of the whole memory's
    // number); the fp32 kernel's by what is seen (200 rows of 4 heads, keys of 128, window 512: 26.6 us, 32.9 by that rule)
    p.splits = tiles && window ? std::min(pieces_of(tiles, blocks, all, max_len), std::max(1, keys / 256))
                               : pieces_of(tiles, blocks, all, keys);
  }
  const int parts = p.splits / p.cluster;
  p.scratch = parts == 1 ? 0 : (size_t)parts * rows * m.n_head * ((size_t)m.head_dim + 2) * sizeof(float);
  if (expand) p.scratch = (p.scratch + 15) / 16 * 16 + expanded + 4ll * m.n_seq * cols;
  return p;
}

cudaError_t launch_attend(AttendArgs& a, const AttendPlan& p, void* scratch, cudaStream_t st) {
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.cluster = p.cluster;
  const int parts = p.splits / p.cluster;
  a.part = static_cast<float*>(scratch);
  a.ml = reinterpret_cast<float2*>(a.part + (size_t)parts * a.rows * a.m.n_head * a.m.head_dim);
  const bool d64 = a.m.head_dim == 64;
  cudaError_t e = cudaSuccess;
  if (p.expand) {
    const size_t joined = parts == 1 ? 0 : (size_t)parts * a.rows * a.m.n_head * ((size_t)a.m.head_dim + 2) * sizeof(float);
    const size_t values = (size_t)a.m.n_seq * p.expand * a.m.n_kv_head * a.m.page_tokens * a.m.head_dim;
    __nv_bfloat16* k = reinterpret_cast<__nv_bfloat16*>(static_cast<uint8_t*>(scratch) + (joined + 15) / 16 * 16);
    int* table = reinterpret_cast<int*>(k + 2 * values);
    const dim3 grid(a.m.n_seq * p.expand, 2);
    if (d64)
      expand_kernel<64><<<grid, JOIN_THREADS, 0, st>>>(a, p.expand, k, k + values, table);
    else
      expand_kernel<128><<<grid, JOIN_THREADS, 0, st>>>(a, p.expand, k, k + values, table);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    a.m.format = EVO_CACHE_BF16;
    a.m.k_pages = k;
    a.m.v_pages = k + values;
    a.m.k_scales = a.m.v_scales = nullptr;
    a.m.table = table;
    a.m.max_pages = p.expand;
    a.m.n_pages = a.m.n_seq * p.expand;
  }
  if (p.kernel == ATTEND_F32)
    e = p.tile_rows == 32 ? d64 ? launch_f32<64, 2>(a, st) : launch_f32_as<128, EVO_CACHE_F32, 2>(a, st)
        : d64 ? launch_f32<64, 4>(a, st) : launch_f32<128, 4>(a, st);
  else if (p.kernel == ATTEND_F32_ROWS)
    e = launch_attend_f32_rows(a, p.tile_rows, st);
  else if (p.kernel == ATTEND_ROWS)
    e = launch_attend_rows(a, p.tile_rows, st);
  else
    e = launch_attend_tiles(a, st);
  if (e != cudaSuccess || parts == 1) return e;
  if (a.m.dtype == EVO_DTYPE_F32) return d64 ? launch_join<float, 64>(a, st) : launch_join<float, 128>(a, st);
  return d64 ? launch_join<__nv_bfloat16, 64>(a, st) : launch_join<__nv_bfloat16, 128>(a, st);
}

}  // namespace evo
