// Device helpers of the paged-memory kernels: shared-memory loads, bulk copies,
// the bounded wait for them and packed arithmetic.
#pragma once

#include <cstdint>
#include <cuda.h>

#include "evo_tc.cuh"

namespace evo {

__device__ __forceinline__ uint4 lds128(uint32_t p) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(p));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t p) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(p));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t p) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(p));
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t p) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(p));
  return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t p) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(p));
  return v;
}
__device__ __forceinline__ float4 lds_f4(uint32_t p) {
  const uint4 v = lds128(p);
  return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ float2 lds_f2(uint32_t p) {
  const uint2 v = lds64(p);
  return make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
}
__device__ __forceinline__ void sts_f4(uint32_t p, float4 v) {
  asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(p), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void sts_f1(uint32_t p, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(p), "f"(v) : "memory"); }

// copies global -> shared whose bytes are counted on a barrier of this block
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::
          "r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
// a tensor map on its way to the copy unit while the first coordinates are looked up
__device__ __forceinline__ void fetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
// a bounded wait: false if the copies did not arrive within `limit` tests.  A test that fails suspends its
// warp for 3.8 us (measured on a barrier that nothing arrives at): about 2 s.  A clock in place of the count
// takes registers that the kernels do not have (64 x 32 rows over 8-bit pages of 64: 94 us against 91)
__device__ __forceinline__ bool wait_full(uint32_t bar, uint32_t parity, int limit = 1 << 19) {
  for (int i = 0; i < limit; ++i)
    if (tc::mbar_test(bar, parity)) return true;
  return false;
}
// the same behind a first test that failed, over as soon as any wait of the block was in vain: `dead`
// is a word of shared memory, zero at the start
__device__ __forceinline__ bool wait_live(uint32_t bar, uint32_t parity, uint32_t dead, long long limit = WAIT_CYCLES_DEFAULT) {
  const long long t0 = clock64();
  while (!tc::block_dead(dead)) {
    if (tc::mbar_test(bar, parity)) return true;
    if (clock64() - t0 > limit) asm volatile("st.volatile.shared::cta.b32 [%0], 1;" ::"r"(dead) : "memory");
  }
  return false;
}
// what a block does in which a wait was in vain, after its last one: it reports, and lets the
// copies in flight land before it ends
__device__ __forceinline__ void settle(int32_t* status) {
  if (threadIdx.x == 0 && status) *status = EVO_ERR_TIMEOUT;
  const long long t0 = clock64();
  while (clock64() - t0 < SETTLE_CYCLES) __nanosleep(1000);
}

// byte offset of 16-byte chunk `chunk` of row r in a tile of ROWS rows of ROW bytes that tiled copies
// brought: boxes of at most 128 bytes of a row, one behind the other, swizzled by their width
template <int ROW, int ROWS>
__device__ __forceinline__ int chunk_at(int r, int chunk) {
  if constexpr (ROW == 64) return r * 64 + ((chunk ^ ((r >> 1) & 3)) << 4);
  return (chunk >> 3) * (ROWS * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4);
}

// packed pairs, subnormals kept (mul2 and fma2 flush them)
__device__ __forceinline__ float2 mul_pair(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 ra, rb, rd;\n mov.b64 ra, {%2, %3};\n mov.b64 rb, {%4, %5};\n"
      " mul.rn.f32x2 rd, ra, rb;\n mov.b64 {%0, %1}, rd;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 ra, rb, rc, rd;\n mov.b64 ra, {%2, %3};\n mov.b64 rb, {%4, %5};\n mov.b64 rc, {%6, %7};\n"
      " fma.rn.f32x2 rd, ra, rb, rc;\n mov.b64 {%0, %1}, rd;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

}  // namespace evo
