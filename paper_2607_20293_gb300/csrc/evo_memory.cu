// Entry points of the 8-bit unit caches and the paged memory (include/evo.h):
// argument checks on the host, then the launch.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cuda_runtime.h>

#include "evo_memory.h"

using namespace evo;

namespace evo {

bool page_map(CUtensorMap* map, const evo_memory& m, const void* pages, int box_rows) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    cudaDriverEntryPointQueryResult q;
    void* p = nullptr;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return (Encode) nullptr;
    return reinterpret_cast<Encode>(p);
  }();
  if (!encode) return false;
  const bool codes = m.format == EVO_CACHE_E4M3;
  const cuuint32_t item = codes ? 1 : m.format == EVO_CACHE_BF16 ? 2 : 4;
  const cuuint64_t row = (cuuint64_t)m.head_dim * item;
  const cuuint64_t dims[2] = {(cuuint64_t)m.head_dim, (cuuint64_t)m.n_pages * m.n_kv_head * m.page_tokens};
  const cuuint64_t strides[1] = {row};
  const cuuint32_t width = (cuuint32_t)(row < 128 ? row : 128);
  const cuuint32_t box[2] = {width / item, (cuuint32_t)box_rows}, steps[2] = {1, 1};
  const CUtensorMapDataType type = codes       ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                   : item == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                               : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
  return encode(map, type, 2, const_cast<void*>(pages), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace evo

namespace {

#define EVO_CUDA(x)                       \
  do {                                    \
    const cudaError_t _e = (x);           \
    if (_e != cudaSuccess) {              \
      g_last_cuda_error = (int)_e;        \
      return EVO_ERR_CUDA;                \
    }                                     \
  } while (0)

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// do a_bytes at a and b_bytes at b share any?
bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + b_bytes && y < x + a_bytes;
}

// what evo_cache_write and evo_cache_add check alike; *per = values of a sample
evo_status cache_args(int32_t U, int32_t N, int32_t H, int32_t E, const float* x, const float* y,
                      const uint8_t* codes, const uint8_t* scales, long long* per) {
  if (N < 0 || H < 0 || E <= 0) return EVO_ERR_ARG;
  if (E % UNIT_GROUP) return EVO_ERR_SHAPE;
  *per = (long long)H * E;
  if (*per > (1ll << 33) || (N > 0 && *per > (1ll << 33) / N) || N * (*per / 8) > INT_MAX - 1024) return EVO_ERR_SHAPE;
  if (N == 0 || H == 0) return EVO_OK;
  if ((U > 0 && (!codes || !scales)) || (x == nullptr) != (y == nullptr)) return EVO_ERR_ARG;
  if (!aligned(codes, 16) || !aligned(x, 16) || !aligned(y, 16)) return EVO_ERR_ARG;
  const size_t values = (size_t)N * *per, held = (size_t)U * values;
  if (x && x != y && overlap(x, 4 * values, y, 4 * values)) return EVO_ERR_ARG;
  if (U > 0 && (overlap(codes, held, scales, held / UNIT_GROUP) ||
                (x && (overlap(x, 4 * values, codes, held) || overlap(x, 4 * values, scales, held / UNIT_GROUP) ||
                       overlap(y, 4 * values, codes, held) || overlap(y, 4 * values, scales, held / UNIT_GROUP)))))
    return EVO_ERR_ARG;
  return EVO_OK;
}

evo_status memory_ok(const evo_memory* m) {
  if (!m) return EVO_ERR_ARG;
  if (m->dtype != EVO_DTYPE_F32 && m->dtype != EVO_DTYPE_BF16) return EVO_ERR_ARG;
  if (m->format < EVO_CACHE_F32 || m->format > EVO_CACHE_E4M3) return EVO_ERR_ARG;
  if (m->n_head <= 0 || m->n_kv_head <= 0 || m->n_pages <= 0 || m->max_pages <= 0 || m->n_seq < 0) return EVO_ERR_ARG;
  if (m->format != EVO_CACHE_E4M3 && m->format != (m->dtype == EVO_DTYPE_F32 ? EVO_CACHE_F32 : EVO_CACHE_BF16))
    return EVO_ERR_UNSUPPORTED;
  if (m->head_dim != 64 && m->head_dim != 128) return EVO_ERR_SHAPE;
  if (m->n_head % m->n_kv_head || m->n_head > 1024) return EVO_ERR_SHAPE;
  if (m->page_tokens != 16 && m->page_tokens != 32 && m->page_tokens != 64 && m->page_tokens != 128) return EVO_ERR_SHAPE;
  // 2^30 tokens: the kernels look runs ahead in 32 bits
  if (m->max_pages > (1 << 30) / m->page_tokens) return EVO_ERR_SHAPE;
  if ((long long)m->n_pages * m->n_kv_head * m->page_tokens > INT_MAX) return EVO_ERR_SHAPE;
  if (!m->k_pages || !m->v_pages || (m->n_seq > 0 && (!m->table || !m->lens))) return EVO_ERR_ARG;
  if (!aligned(m->k_pages, 16) || !aligned(m->v_pages, 16)) return EVO_ERR_ARG;
  const bool scales = m->format == EVO_CACHE_E4M3;
  if ((m->k_scales != nullptr) != scales || (m->v_scales != nullptr) != scales) return EVO_ERR_ARG;
  if (!aligned(m->k_scales, 16) || !aligned(m->v_scales, 16)) return EVO_ERR_ARG;
  return EVO_OK;
}

// rows of `heads` heads, ld elements apart
bool rows_ok(const evo_memory* m, const void* p, int64_t ld, int heads) {
  const int item = m->dtype == EVO_DTYPE_F32 ? 4 : 2;
  return aligned(p, 16) && ld >= (int64_t)heads * m->head_dim && ld <= INT_MAX && ld * item % 16 == 0;
}

// do `rows` rows of a_heads heads, lda elements apart, at a share a byte with those at b?  (Column
// ranges of one buffer interleave without doing so.)
bool rows_overlap(const evo_memory* m, const void* a, int64_t lda, int a_heads, const void* b, int64_t ldb, int b_heads,
                  int32_t rows) {
  const uint64_t item = m->dtype == EVO_DTYPE_F32 ? 4 : 2, wide_a = a_heads * m->head_dim * item, wide_b = b_heads * m->head_dim * item;
  const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  const uint64_t end_a = x + (rows - 1) * lda * item + wide_a, end_b = y + (rows - 1) * ldb * item + wide_b;
  if (end_a <= y || end_b <= x) return false;
  if (lda != ldb) return true;
  const uint64_t step = lda * item, at = x <= y ? (y - x) % step : (step - (x - y) % step) % step;   // b's column, a's being 0
  return at < wide_a || at + wide_b > step;
}

// rows of a call: none, or chunks that the sequences can have
evo_status chunks_ok(const evo_memory* m, int32_t rows) {
  if (rows < 0) return EVO_ERR_ARG;
  if (rows > 0 && m->n_seq == 0) return EVO_ERR_ARG;
  if (!m->starts && m->n_seq > 0 && rows % m->n_seq) return EVO_ERR_SHAPE;
  if ((long long)rows * m->n_head > INT_MAX / 32) return EVO_ERR_SHAPE;
  return EVO_OK;
}

// sizes of an attention call
evo_status attend_sizes(const evo_memory* m, int32_t rows, int32_t max_new, int32_t max_len) {
  const evo_status s = chunks_ok(m, rows);
  if (s != EVO_OK) return s;
  if (max_new <= 0 || max_new > rows || max_len < 0) return EVO_ERR_ARG;
  if (!m->starts && max_new < rows / m->n_seq) return EVO_ERR_ARG;
  if (max_len > m->max_pages * m->page_tokens) return EVO_ERR_ARG;
  // blocks of the launch: the row tiles of every sequence and head, a piece each
  if (((long long)max_new * m->n_head / 16 + m->n_kv_head) * m->n_seq > INT_MAX / 128) return EVO_ERR_SHAPE;
  return EVO_OK;
}

}  // namespace

extern "C" {

evo_status evo_cache_write(const void* r, int32_t dtype, const uint8_t* refresh, int32_t N, int32_t H, int32_t E,
                           const float* x, float* y, uint8_t* codes, uint8_t* scales, void* stream) {
  if (dtype != EVO_DTYPE_F32 && dtype != EVO_DTYPE_BF16) return EVO_ERR_ARG;
  long long per;
  const evo_status s = cache_args(1, N, H, E, x, y, codes, scales, &per);
  if (s != EVO_OK || N == 0 || H == 0) return s;
  if (!r || !aligned(r, 16)) return EVO_ERR_ARG;
  // the stream may take the place of an fp32 residual (a thread reads what it writes), nothing else that is read
  const size_t values = (size_t)N * per, bytes = values * (dtype == EVO_DTYPE_F32 ? 4 : 2);
  if (overlap(r, bytes, codes, values) || overlap(r, bytes, scales, values / UNIT_GROUP) ||
      (y && !(y == r && dtype == EVO_DTYPE_F32) && overlap(r, bytes, y, 4 * values)))
    return EVO_ERR_ARG;
  EVO_CUDA(launch_cache_write(r, dtype, refresh, N, per, x, y, codes, scales, reinterpret_cast<cudaStream_t>(stream)));
  return EVO_OK;
}

evo_status evo_cache_add(const uint8_t* codes, const uint8_t* scales, const uint8_t* reuse, int32_t U, int32_t N,
                         int32_t H, int32_t E, const float* x, float* y, void* stream) {
  if (U < 0) return EVO_ERR_ARG;
  long long per;
  const evo_status s = cache_args(U, N, H, E, x, y, codes, scales, &per);
  if (s != EVO_OK || N == 0 || H == 0) return s;
  if (!x) return EVO_ERR_ARG;
  EVO_CUDA(launch_cache_add(codes, scales, reuse, U, N, per, x, y, reinterpret_cast<cudaStream_t>(stream)));
  return EVO_OK;
}

evo_status evo_rotation_table(int32_t n_pos, int32_t head_dim, double base, float* out) {
  if (n_pos <= 0 || head_dim <= 0 || head_dim % 2 || !(base > 0) || !std::isfinite(base) || !out) return EVO_ERR_ARG;
  const int half = head_dim / 2;
  for (int i = 0; i < half; ++i) {
    const double w = std::pow(base, -2.0 * i / head_dim);
    for (int p = 0; p < n_pos; ++p) {
      out[(size_t)p * head_dim + i] = (float)std::cos(p * w);
      out[(size_t)p * head_dim + half + i] = (float)std::sin(p * w);
    }
  }
  return EVO_OK;
}

evo_status evo_memory_append(const evo_memory* mem, const void* q, const void* k, const void* v, int64_t ldq,
                             int64_t ldk, int64_t ldv, int32_t rows, const float* q_gain, const float* k_gain,
                             float eps, const float* rotation, int32_t n_pos, const int32_t* pos0, void* q_out,
                             int64_t ldo, void* stream) {
  evo_status s = memory_ok(mem);
  if (s == EVO_OK) s = chunks_ok(mem, rows);
  if (s != EVO_OK) return s;
  if ((k == nullptr) != (v == nullptr) || (q == nullptr) != (q_out == nullptr) || !(eps >= 0.f)) return EVO_ERR_ARG;
  if (rotation ? n_pos <= 0 : pos0 != nullptr) return EVO_ERR_ARG;
  if (rows == 0 || (!q && !k)) return EVO_OK;
  if (q && (!rows_ok(mem, q, ldq, mem->n_head) || !rows_ok(mem, q_out, ldo, mem->n_head))) return EVO_ERR_ARG;
  if (k && (!rows_ok(mem, k, ldk, mem->n_kv_head) || !rows_ok(mem, v, ldv, mem->n_kv_head))) return EVO_ERR_ARG;
  // queries may be overwritten in place (a warp reads what it writes), nothing else that the call reads
  if (q && (q_out != q || ldo != ldq) && rows_overlap(mem, q_out, ldo, mem->n_head, q, ldq, mem->n_head, rows)) return EVO_ERR_ARG;
  if (q && k && (rows_overlap(mem, q_out, ldo, mem->n_head, k, ldk, mem->n_kv_head, rows) ||
                 rows_overlap(mem, q_out, ldo, mem->n_head, v, ldv, mem->n_kv_head, rows)))
    return EVO_ERR_ARG;
  if (!aligned(rotation, 16) || !aligned(q_gain, 16) || !aligned(k_gain, 16)) return EVO_ERR_ARG;
  const AppendArgs a{*mem, q, k, v, q_out, ldq, ldk, ldv, ldo, rows, q_gain, k_gain, eps, rotation, n_pos, pos0};
  EVO_CUDA(launch_append(a, reinterpret_cast<cudaStream_t>(stream)));
  return EVO_OK;
}

size_t evo_memory_scratch_bytes(const evo_memory* mem, int32_t rows, int32_t max_new, int32_t max_len) {
  if (memory_ok(mem) != EVO_OK || attend_sizes(mem, rows, max_new, max_len) != EVO_OK) return 0;
  return plan_attend(*mem, rows, max_new, max_len, 0, 0).scratch;
}

evo_status evo_memory_attend(const evo_memory* mem, const void* q, int64_t ldq, int32_t rows, int32_t max_new,
                             int32_t max_len, float scale, int32_t causal, int32_t window, void* out, int64_t ldo,
                             void* scratch, void* stream) {
  evo_status s = memory_ok(mem);
  if (s != EVO_OK) return s;
  if (rows == 0) return EVO_OK;
  s = attend_sizes(mem, rows, max_new, max_len);
  if (s != EVO_OK) return s;
  const float scale_log2 = scale * 1.4426950408889634f;
  if (!q || !out || !std::isfinite(scale_log2) || (causal != 0 && causal != 1) || window < 0) return EVO_ERR_ARG;
  if (!rows_ok(mem, q, ldq, mem->n_head) || !rows_ok(mem, out, ldo, mem->n_head)) return EVO_ERR_ARG;
  if (rows_overlap(mem, q, ldq, mem->n_head, out, ldo, mem->n_head, rows)) return EVO_ERR_ARG;
  // pieces by what a window leaves to see, where they fit the workspace that a call without one has
  AttendPlan p = plan_attend(*mem, rows, max_new, max_len, 0, 0);
  if (window) {
    const AttendPlan w = plan_attend(*mem, rows, max_new, max_len, causal, window);
    if (w.scratch <= p.scratch) p = w;
  }
  if (p.scratch && (!scratch || !aligned(scratch, 16))) return EVO_ERR_ARG;
  AttendArgs a{};
  a.m = *mem;
  a.q = q;
  a.out = out;
  a.ldq = ldq;
  a.ldo = ldo;
  a.rows = rows;
  a.max_new = max_new;
  a.max_len = max_len;
  a.group = mem->n_head / mem->n_kv_head;
  a.scale_log2 = scale_log2;
  a.causal = causal;
  a.window = window;
  EVO_CUDA(launch_attend(a, p, scratch, reinterpret_cast<cudaStream_t>(stream)));
  return EVO_OK;
}

}  // extern "C"
