// C entry points of the operators on 8-bit weights and on tokens sorted by expert
// (include/gleam.h): argument checks, then one launch each.
#include <atomic>

#include "host_checks.cuh"
#include "operators.cuh"

using namespace gleam;

namespace {

// Up to so many rows gleam_fp8_linear is one kernel.  Two groups of 8 rows are as many as its
// registers hold; an expert's rows are on average this few, and more of them read its weights
// again.
constexpr uint64_t kFewRows = 16, kFewRowsOfExpert = 4;

constexpr uint32_t kMaxAlign = 1u << 20, kMaxPerToken = 1u << 20;
constexpr uint64_t kMaxDim = 0x7fffff00ull;  // rows and columns fit 31 bits, tiles too
// More than any memory holds, and few enough that spans in bytes stay below 2^63.
constexpr uint64_t kMaxElements = 1ull << 50, kMaxAllElements = 1ull << 60, kMaxTiles = 1ull << 40;

uint64_t tiles_of(uint64_t n) { return (n + kTile - 1) / kTile; }

bool dtype_ok(int32_t t) { return t == GLEAM_BF16 || t == GLEAM_FP16 || t == GLEAM_FP32; }

// Shape of a matrix: known type, sizes and span in range, rows that do not overlap.
bool shape_ok(const gleam_matrix_t& x) {
  if (!dtype_ok(x.dtype) || x.count == 0 || x.rows > kMaxDim || x.cols > kMaxDim) return false;
  if (x.ld < x.cols || x.ld > (1ull << 40) || (x.rows > 1 && x.ld > kMaxElements / x.rows)) return false;
  if (x.count > 1 && (x.rows == 0 || x.stride < (x.rows - 1) * x.ld + x.cols || x.stride > kMaxAllElements / x.count))
    return false;
  return true;
}

// Bytes from the first element to the last of a matrix with elements.
uint64_t span_of(const gleam_matrix_t& x) {
  const uint64_t one = (x.rows - 1) * x.ld + x.cols;
  return ((x.count - 1) * (x.count > 1 ? x.stride : 0) + one) * (x.dtype == GLEAM_FP32 ? 4 : 2);
}

bool aligned(const void* p, uint64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Whether an element starts at a multiple of its own size.
bool element_aligned(const void* p, int32_t dtype) { return aligned(p, dtype == GLEAM_FP32 ? 4 : 2); }

int current_device(int* dev) { return cuda_err(cudaGetDevice(dev)); }

QuantizeArgs quantize_args(const gleam_matrix_t& x, const int32_t* src, uint32_t per_token, uint64_t rows,
                           uint8_t* q, float* s) {
  const uint64_t size = x.dtype == GLEAM_FP32 ? 4 : 2;
  QuantizeArgs a{};
  a.x = static_cast<const uint8_t*>(x.d);
  a.ld = x.ld * size;
  a.stride = x.count > 1 ? x.stride * size : 0;
  a.x_rows = x.rows;
  a.cols = x.cols;
  a.rows = rows;
  a.rt = tiles_of(rows);
  a.kb = tiles_of(x.cols);
  a.src = src;
  a.per_token = per_token;
  a.count = x.count;
  a.dtype = (uint32_t)x.dtype;
  a.form = GLEAM_FP8_GROUPS;
  a.vec = aligned(x.d, 4 * size) && x.ld % 4 == 0 && (x.count == 1 || x.stride % 4 == 0);
  a.q = q;
  a.s = s;
  return a;
}

// Rows to expect of one matrix: sorted rows are the slots' own and up to 127 more per expert.
uint64_t rows_to_expect(uint64_t rows, uint32_t experts) {
  if (experts == 0) return rows;
  const uint64_t fill = experts * (uint64_t)(kTile - 1);
  return rows > fill ? (rows - fill + experts - 1) / experts : 1;
}

// Whether gleam_fp8_linear runs as one kernel.
bool one_kernel(uint64_t rows, uint64_t cols, uint32_t experts) {
  return rows_to_expect(rows, experts) <= (experts == 0 ? kFewRows : kFewRowsOfExpert) &&
         few_fits(experts == 0 ? rows : 1, tiles_of(cols));
}

// Test hooks (gleam_operators_debug_set).
std::atomic<unsigned long long> g_wait_ns{kOperatorWaitNs};
std::atomic<uint32_t> g_skip{kNoSkip};
// It applies to one call.
uint32_t take_skip() {
  return g_skip.load(std::memory_order_relaxed) == kNoSkip ? kNoSkip : g_skip.exchange(kNoSkip);
}

// A failure that the device found, of a product whose caller gave no word for it.
__device__ int32_t g_failure;

// Its address on the current GPU.
int failure_word(int dev, int32_t** word) {
  static std::atomic<int32_t*> known[64] = {};
  const bool kept = dev >= 0 && dev < 64;
  *word = kept ? known[dev].load(std::memory_order_relaxed) : nullptr;
  if (*word != nullptr) return GLEAM_OK;
  void* p = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&p, g_failure);
  if (e != cudaSuccess) return cuda_err(e);
  *word = static_cast<int32_t*>(p);
  if (kept) known[dev].store(*word, std::memory_order_relaxed);
  return GLEAM_OK;
}

#define GLEAM_TRY(x)              \
  do {                            \
    const int rc_ = (x);          \
    if (rc_ != GLEAM_OK) return rc_; \
  } while (0)

}  // namespace

extern "C" {

int gleam_fp8_quantize(const gleam_matrix_t* x, int form, const int32_t* d_src, uint32_t per_token,
                       uint64_t rows_out, uint8_t* d_q, float* d_s, uint8_t* d_qt, float* d_st,
                       gleam_stream_t stream) {
  if (x == nullptr || (form != GLEAM_FP8_GROUPS && form != GLEAM_FP8_BLOCKS)) return GLEAM_ERR_INVALID_ARG;
  const bool blocks = form == GLEAM_FP8_BLOCKS;
  if (!shape_ok(*x) || (!blocks && x->count != 1) || (blocks && d_src != nullptr))
    return GLEAM_ERR_INVALID_ARG;
  if ((d_q == nullptr) != (d_s == nullptr) || (d_qt == nullptr) != (d_st == nullptr) ||
      (d_q == nullptr && d_qt == nullptr))
    return GLEAM_ERR_INVALID_ARG;
  const uint64_t rows = d_src == nullptr ? x->rows : rows_out;
  if (d_src == nullptr && rows_out != x->rows) return GLEAM_ERR_INVALID_ARG;
  if (rows > kMaxDim || per_token > 0x7fffffffu) return GLEAM_ERR_INVALID_ARG;
  if (rows == 0 || x->cols == 0) return GLEAM_OK;
  if (x->rows == 0 && d_src == nullptr) return GLEAM_OK;
  const uint64_t rt = tiles_of(rows), kb = tiles_of(x->cols);
  if (rt * kb > 0x7fffffffull / x->count) return GLEAM_ERR_INVALID_ARG;
  const uint64_t tiles = rt * kb * x->count;
  int dev = 0;
  GLEAM_TRY(current_device(&dev));
  PtrChecker chk(dev);
  if (x->rows != 0) {
    GLEAM_TRY(chk.check(x->d, span_of(*x)));
    if (!element_aligned(x->d, x->dtype)) return GLEAM_ERR_INVALID_ARG;
  }
  if (d_src != nullptr) {
    GLEAM_TRY(chk.check(d_src, rows * 4));
    if (!aligned(d_src, 4)) return GLEAM_ERR_INVALID_ARG;
  }
  if (d_q != nullptr) {
    GLEAM_TRY(chk.check(d_q, tiles * kTileBytes));
    GLEAM_TRY(chk.check(d_s, blocks ? tiles * 4 : tiles * kTile * 4));
  }
  if (d_qt != nullptr) {
    GLEAM_TRY(chk.check(d_qt, tiles * kTileBytes));
    GLEAM_TRY(chk.check(d_st, blocks ? tiles * 4 : tiles * kTile * 4));
  }
  if (!aligned(d_q, 16) || !aligned(d_s, 16) || !aligned(d_qt, 16) || !aligned(d_st, 16))
    return GLEAM_ERR_INVALID_ARG;

  QuantizeArgs a = quantize_args(*x, d_src, per_token, rows, d_q, d_s);
  a.form = (uint32_t)form;
  a.qt = d_qt;
  a.st = d_st;
  return cuda_err(launch_quantize(a, reinterpret_cast<cudaStream_t>(stream)));
}

int gleam_fp8_product(const gleam_fp8_product_t* p, gleam_stream_t stream) {
  if (p == nullptr || p->reserved != 0 || p->ex.reserved != 0 || !dtype_ok(p->dtype)) return GLEAM_ERR_INVALID_ARG;
  if (p->w_form != GLEAM_FP8_GROUPS && p->w_form != GLEAM_FP8_BLOCKS) return GLEAM_ERR_INVALID_ARG;
  if (p->m > kMaxDim || p->n > kMaxDim || p->k > kMaxDim || p->ld < p->n || p->ld > (1ull << 40))
    return GLEAM_ERR_INVALID_ARG;
  const uint32_t E = p->ex.experts;
  if (E > kMaxExperts || (p->over != GLEAM_OVER_ROWS && p->over != GLEAM_OVER_SUMS))
    return GLEAM_ERR_INVALID_ARG;
  const bool sums = E != 0 && p->over == GLEAM_OVER_SUMS, by_row = E != 0 && !sums;
  // a group's scale is one of a row, which a weight that is one of several has no array for
  if (by_row && p->w_form != GLEAM_FP8_BLOCKS) return GLEAM_ERR_INVALID_ARG;
  // a block's scale along sums over rows would span 128 rows of w
  if (sums && p->w_form != GLEAM_FP8_GROUPS) return GLEAM_ERR_INVALID_ARG;
  if (E == 0 && p->over != GLEAM_OVER_ROWS) return GLEAM_ERR_INVALID_ARG;
  if (p->m == 0 || p->n == 0) return GLEAM_OK;
  const uint64_t size = p->dtype == GLEAM_FP32 ? 4 : 2;
  const uint64_t matrices = sums ? E : 1;
  const uint64_t xrt = tiles_of(p->m), wrt = tiles_of(p->n), kb = tiles_of(p->k), weights = by_row ? E : 1;
  if (wrt * kb > kMaxTiles / weights || p->ld > kMaxAllElements / (matrices * p->m)) return GLEAM_ERR_INVALID_ARG;
  int dev = 0;
  GLEAM_TRY(current_device(&dev));
  PtrChecker chk(dev);
  if (kb != 0) {
    GLEAM_TRY(chk.check(p->d_xq, xrt * kb * kTileBytes));
    GLEAM_TRY(chk.check(p->d_xs, xrt * kb * kTile * 4));
    GLEAM_TRY(chk.check(p->d_wq, weights * wrt * kb * kTileBytes));
    GLEAM_TRY(chk.check(p->d_ws, weights * wrt * kb * 4 * (p->w_form == GLEAM_FP8_GROUPS ? kTile : 1)));
    if (!aligned(p->d_xq, 16) || !aligned(p->d_xs, 16) || !aligned(p->d_wq, 16) || !aligned(p->d_ws, 16))
      return GLEAM_ERR_INVALID_ARG;
  }
  GLEAM_TRY(chk.check(p->d_y, (((matrices - 1) * p->m + p->m - 1) * p->ld + p->n) * size));
  if (!element_aligned(p->d_y, p->dtype)) return GLEAM_ERR_INVALID_ARG;
  if (E != 0) {
    GLEAM_TRY(chk.check(p->ex.d_offsets, (E + 1) * 4ull));
    GLEAM_TRY(chk.check(p->ex.d_counts, E * 4ull));
    if (!aligned(p->ex.d_offsets, 4) || !aligned(p->ex.d_counts, 4)) return GLEAM_ERR_INVALID_ARG;
  }
  if (p->d_status != nullptr) {
    GLEAM_TRY(chk.check(p->d_status, 4));
    if (!aligned(p->d_status, 4)) return GLEAM_ERR_INVALID_ARG;
  }

  int32_t* status = p->d_status;
  if (status == nullptr) GLEAM_TRY(failure_word(dev, &status));

  ProductArgs a{};
  a.xq = p->d_xq;
  a.xs = p->d_xs;
  a.wq = p->d_wq;
  a.ws = p->d_ws;
  a.y = static_cast<uint8_t*>(p->d_y);
  a.ld = p->ld;
  a.ystride = p->m * p->ld;
  a.m = p->m;
  a.n = p->n;
  a.kb = kb;
  a.xrt = xrt;
  a.wrt = wrt;
  a.dtype = (uint32_t)p->dtype;
  a.w_form = (uint32_t)p->w_form;
  a.experts = E;
  a.vec = aligned(p->d_y, 16) && p->ld * size % 16 == 0;
  a.over = (uint32_t)p->over;
  a.offsets = p->ex.d_offsets;
  a.counts = p->ex.d_counts;
  a.status = status;
  a.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
  a.skip = take_skip();
  return cuda_err(launch_product(a, rows_to_expect(p->m, by_row ? E : 0), reinterpret_cast<cudaStream_t>(stream)));
}

uint64_t gleam_fp8_linear_work(uint64_t rows, uint64_t cols, uint32_t experts) {
  if (rows > kMaxDim || cols > kMaxDim || one_kernel(rows, cols, experts)) return 0;
  const uint64_t tiles = tiles_of(rows) * tiles_of(cols);
  return tiles * (kTileBytes + kTile * 4);
}

int gleam_fp8_linear(const gleam_fp8_linear_t* p, gleam_stream_t stream) {
  if (p == nullptr || p->reserved != 0 || p->ex.reserved != 0 || !shape_ok(p->x) || p->x.count != 1)
    return GLEAM_ERR_INVALID_ARG;
  const gleam_matrix_t& x = p->x;
  const uint32_t E = p->ex.experts;
  if (p->rows > kMaxDim || p->n > kMaxDim || p->ld < p->n || p->ld > (1ull << 40) || E > kMaxExperts ||
      p->per_token > 0x7fffffffu || (p->d_src == nullptr && p->rows != x.rows))
    return GLEAM_ERR_INVALID_ARG;
  if (p->rows == 0 || p->n == 0) return GLEAM_OK;
  const uint64_t size = x.dtype == GLEAM_FP32 ? 4 : 2;
  const uint64_t rt = tiles_of(p->rows), kb = tiles_of(x.cols), wrt = tiles_of(p->n), weights = E == 0 ? 1 : E;
  if (rt * kb > 0x7fffffffull || wrt * kb > kMaxTiles / weights || p->ld > kMaxAllElements / p->rows)
    return GLEAM_ERR_INVALID_ARG;
  int dev = 0;
  GLEAM_TRY(current_device(&dev));
  PtrChecker chk(dev);
  if (kb != 0) {
    if (x.rows != 0) GLEAM_TRY(chk.check(x.d, span_of(x)));
    GLEAM_TRY(chk.check(p->d_wq, weights * wrt * kb * kTileBytes));
    GLEAM_TRY(chk.check(p->d_ws, weights * wrt * kb * 4));
  }
  GLEAM_TRY(chk.check(p->d_y, ((p->rows - 1) * p->ld + p->n) * size));
  if (p->d_src != nullptr) GLEAM_TRY(chk.check(p->d_src, p->rows * 4));
  if (E != 0) {
    GLEAM_TRY(chk.check(p->ex.d_offsets, (E + 1) * 4ull));
    GLEAM_TRY(chk.check(p->ex.d_counts, E * 4ull));
  }
  if (p->d_status != nullptr) GLEAM_TRY(chk.check(p->d_status, 4));
  const uint64_t need = gleam_fp8_linear_work(p->rows, x.cols, E);
  if (p->work_bytes < need) return GLEAM_ERR_INVALID_ARG;
  if (need != 0) GLEAM_TRY(chk.check(p->d_work, need));
  if (!element_aligned(x.d, x.dtype) || !element_aligned(p->d_y, x.dtype) || !aligned(p->d_wq, 16) ||
      !aligned(p->d_ws, 16) || !aligned(p->d_work, 16) || !aligned(p->d_src, 4) || !aligned(p->ex.d_offsets, 4) ||
      !aligned(p->ex.d_counts, 4) || !aligned(p->d_status, 4))
    return GLEAM_ERR_INVALID_ARG;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int32_t* status = p->d_status;
  if (status == nullptr) GLEAM_TRY(failure_word(dev, &status));

  if (one_kernel(p->rows, x.cols, E)) {
    FewArgs f{};
    f.x = static_cast<const uint8_t*>(x.d);
    f.ld = x.ld * size;
    f.x_rows = x.rows;
    f.cols = x.cols;
    f.rows = p->rows;
    f.src = p->d_src;
    f.per_token = p->per_token;
    f.dtype = (uint32_t)x.dtype;
    f.vec = aligned(x.d, 16) && f.ld % 16 == 0;
    f.wq = p->d_wq;
    f.ws = p->d_ws;
    f.n = p->n;
    f.kb = kb;
    f.wrt = wrt;
    f.y = static_cast<uint8_t*>(p->d_y);
    f.y_ld = p->ld;
    f.experts = E;
    f.offsets = p->ex.d_offsets;
    f.counts = p->ex.d_counts;
    f.status = status;
    f.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
    f.skip = take_skip();
    return cuda_err(launch_few(f, s));
  }
  uint8_t* xq = static_cast<uint8_t*>(p->d_work);
  float* xs = reinterpret_cast<float*>(xq + rt * kb * kTileBytes);
  if (kb != 0) {
    QuantizeArgs q = quantize_args(x, p->d_src, p->per_token, p->rows, xq, xs);
    q.fill = E == 0 && p->d_src != nullptr;
    q.leads = 1;
    GLEAM_TRY(cuda_err(launch_quantize(q, s)));
  }
  ProductArgs a{};
  a.xq = xq;
  a.xs = xs;
  a.wq = p->d_wq;
  a.ws = p->d_ws;
  a.y = static_cast<uint8_t*>(p->d_y);
  a.ld = p->ld;
  a.m = p->rows;
  a.n = p->n;
  a.kb = kb;
  a.xrt = rt;
  a.wrt = wrt;
  a.dtype = (uint32_t)x.dtype;
  a.w_form = GLEAM_FP8_BLOCKS;
  a.experts = E;
  a.vec = aligned(p->d_y, 16) && p->ld * size % 16 == 0;
  // the quantisation starts after all work before it, which may have written the weights
  a.w_ready = E == 0 && kb != 0;
  a.over = GLEAM_OVER_ROWS;
  a.offsets = p->ex.d_offsets;
  a.counts = p->ex.d_counts;
  a.status = status;
  a.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
  a.skip = take_skip();
  return cuda_err(launch_product(a, rows_to_expect(p->rows, E), s));
}

int gleam_operators_status(gleam_stream_t stream) {
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int dev = 0;
  int32_t* word = nullptr;
  int32_t v = GLEAM_OK;
  GLEAM_TRY(current_device(&dev));
  GLEAM_TRY(failure_word(dev, &word));
  GLEAM_TRY(cuda_err(cudaMemcpyAsync(&v, word, sizeof(v), cudaMemcpyDeviceToHost, s)));
  GLEAM_TRY(cuda_err(cudaStreamSynchronize(s)));
  if (v == GLEAM_OK) return GLEAM_OK;
  GLEAM_TRY(cuda_err(cudaMemsetAsync(word, 0, sizeof(v), s)));
  return v;
}

int gleam_operators_debug_set(int what, int64_t value) {
  if (value <= 0) return GLEAM_ERR_INVALID_ARG;
  if (what == GLEAM_DEBUG_WAIT_LIMIT_NS) {
    g_wait_ns = (unsigned long long)value;
    return GLEAM_OK;
  }
  if (what == GLEAM_DEBUG_SKIP_ARRIVE && value < (int64_t)kNoSkip) {
    g_skip = (uint32_t)value;
    return GLEAM_OK;
  }
  return GLEAM_ERR_INVALID_ARG;
}

uint64_t gleam_expert_rows(uint64_t tokens, uint32_t per_token, uint32_t experts, uint32_t align) {
  if (align == 0 || align > kMaxAlign || tokens > kMaxDim || per_token > kMaxPerToken || experts > kMaxExperts)
    return 0;
  const uint64_t n = tokens * per_token, most = n < experts ? n : experts;
  return (n + most * (align - 1) + align - 1) / align * align;
}

int gleam_expert_sort(const void* d_ids, int id_bytes, uint64_t tokens, uint32_t per_token,
                      uint32_t experts, uint32_t align, int32_t* d_offsets, int32_t* d_counts,
                      int32_t* d_row_of, int32_t* d_src_of, gleam_stream_t stream) {
  if ((id_bytes != 4 && id_bytes != 8) || experts == 0 || experts > kMaxExperts || align == 0 ||
      align > kMaxAlign || tokens > kMaxDim || per_token > kMaxPerToken)
    return GLEAM_ERR_INVALID_ARG;
  const uint64_t slots = tokens * per_token, cap = gleam_expert_rows(tokens, per_token, experts, align);
  if (cap > kMaxDim) return GLEAM_ERR_INVALID_ARG;
  int dev = 0;
  GLEAM_TRY(current_device(&dev));
  PtrChecker chk(dev);
  GLEAM_TRY(chk.check(d_offsets, (experts + 1) * 4ull));
  GLEAM_TRY(chk.check(d_counts, experts * 4ull));
  if (slots != 0) {
    GLEAM_TRY(chk.check(d_ids, slots * id_bytes));
    GLEAM_TRY(chk.check(d_row_of, slots * 4));
    GLEAM_TRY(chk.check(d_src_of, cap * 4));
  }
  if (!aligned(d_ids, id_bytes) || !aligned(d_offsets, 4) || !aligned(d_counts, 4) ||
      !aligned(d_row_of, 4) || !aligned(d_src_of, 4))
    return GLEAM_ERR_INVALID_ARG;
  SortArgs a{};
  a.ids = d_ids;
  a.slots = slots;
  a.cap = cap;
  a.experts = experts;
  a.align = align;
  a.wide = id_bytes == 8;
  a.offsets = d_offsets;
  a.counts = d_counts;
  a.row_of = d_row_of;
  a.src_of = d_src_of;
  return cuda_err(launch_expert_sort(a, reinterpret_cast<cudaStream_t>(stream)));
}

int gleam_expert_gather(const gleam_matrix_t* x, const int32_t* d_src_of, uint32_t per_token,
                        uint64_t rows, void* d_out, gleam_stream_t stream) {
  if (x == nullptr || !shape_ok(*x) || x->count != 1 || per_token == 0 || per_token > 0x7fffffffu ||
      rows > kMaxDim)
    return GLEAM_ERR_INVALID_ARG;
  if (rows == 0 || x->cols == 0) return GLEAM_OK;
  const uint64_t size = x->dtype == GLEAM_FP32 ? 4 : 2;
  int dev = 0;
  GLEAM_TRY(current_device(&dev));
  PtrChecker chk(dev);
  if (x->rows != 0) {
    GLEAM_TRY(chk.check(x->d, span_of(*x)));
    if (!element_aligned(x->d, x->dtype)) return GLEAM_ERR_INVALID_ARG;
  }
  GLEAM_TRY(chk.check(d_src_of, rows * 4));
  GLEAM_TRY(chk.check(d_out, rows * x->cols * size));
  if (!aligned(d_src_of, 4) || !element_aligned(d_out, x->dtype)) return GLEAM_ERR_INVALID_ARG;
  RowsArgs a{};
  a.a = static_cast<const uint8_t*>(x->d);
  a.lda = x->ld * size;
  a.a_rows = x->rows;
  a.b_rows = rows;
  a.cols = x->cols;
  a.src_of = d_src_of;
  a.per_token = per_token;
  a.dtype = (uint32_t)x->dtype;
  a.vec = aligned(x->d, 16) && a.lda % 16 == 0 && aligned(d_out, 16) && x->cols * size % 16 == 0;
  a.out = static_cast<uint8_t*>(d_out);
  return cuda_err(launch_expert_gather(a, reinterpret_cast<cudaStream_t>(stream)));
}

int gleam_expert_combine(const gleam_matrix_t* rows, const int32_t* d_row_of, const float* d_weights,
                         uint64_t tokens, uint32_t per_token, void* d_out, gleam_stream_t stream) {
  if (rows == nullptr || !shape_ok(*rows) || rows->count != 1 || tokens > kMaxDim ||
      per_token > kMaxPerToken)
    return GLEAM_ERR_INVALID_ARG;
  if (tokens == 0 || rows->cols == 0) return GLEAM_OK;
  const uint64_t size = rows->dtype == GLEAM_FP32 ? 4 : 2, slots = tokens * per_token;
  int dev = 0;
  GLEAM_TRY(current_device(&dev));
  PtrChecker chk(dev);
  if (rows->rows != 0) {
    GLEAM_TRY(chk.check(rows->d, span_of(*rows)));
    if (!element_aligned(rows->d, rows->dtype)) return GLEAM_ERR_INVALID_ARG;
  }
  if (slots != 0) {
    GLEAM_TRY(chk.check(d_row_of, slots * 4));
    if (d_weights != nullptr) GLEAM_TRY(chk.check(d_weights, slots * 4));
  }
  GLEAM_TRY(chk.check(d_out, tokens * rows->cols * size));
  if (!aligned(d_row_of, 4) || !aligned(d_weights, 4) || !element_aligned(d_out, rows->dtype))
    return GLEAM_ERR_INVALID_ARG;
  RowsArgs a{};
  a.a = static_cast<const uint8_t*>(rows->d);
  a.lda = rows->ld * size;
  a.a_rows = rows->rows;
  a.cols = rows->cols;
  a.tokens = tokens;
  a.row_of = d_row_of;
  a.w = d_weights;
  a.per_token = per_token;
  a.dtype = (uint32_t)rows->dtype;
  a.vec = aligned(rows->d, 16) && a.lda % 16 == 0 && aligned(d_out, 16) && rows->cols * size % 16 == 0;
  a.out = static_cast<uint8_t*>(d_out);
  return cuda_err(launch_expert_combine(a, reinterpret_cast<cudaStream_t>(stream)));
}

int gleam_expert_combine_grad(const gleam_matrix_t* dy, const gleam_matrix_t* rows,
                              const int32_t* d_row_of, const int32_t* d_src_of,
                              const float* d_weights, uint32_t per_token, void* d_drows,
                              float* d_dweights, gleam_stream_t stream) {
  if (dy == nullptr || rows == nullptr || !shape_ok(*dy) || !shape_ok(*rows) || dy->count != 1 ||
      rows->count != 1 || dy->dtype != rows->dtype || dy->cols != rows->cols || per_token > kMaxPerToken)
    return GLEAM_ERR_INVALID_ARG;
  const uint64_t size = dy->dtype == GLEAM_FP32 ? 4 : 2, slots = dy->rows * per_token;
  if (dy->rows + rows->rows == 0) return GLEAM_OK;
  if (dy->rows + rows->rows > kMaxDim) return GLEAM_ERR_INVALID_ARG;
  int dev = 0;
  GLEAM_TRY(current_device(&dev));
  PtrChecker chk(dev);
  if (dy->cols != 0) {
    if (dy->rows != 0) GLEAM_TRY(chk.check(dy->d, span_of(*dy)));
    if (rows->rows != 0) {
      GLEAM_TRY(chk.check(rows->d, span_of(*rows)));
      GLEAM_TRY(chk.check(d_drows, rows->rows * rows->cols * size));
    }
    if (!element_aligned(dy->d, dy->dtype) || !element_aligned(rows->d, dy->dtype) ||
        !element_aligned(d_drows, dy->dtype))
      return GLEAM_ERR_INVALID_ARG;
  }
  if (slots != 0) {
    GLEAM_TRY(chk.check(d_row_of, slots * 4));
    GLEAM_TRY(chk.check(d_weights, slots * 4));
    GLEAM_TRY(chk.check(d_dweights, slots * 4));
  }
  if (rows->rows != 0) GLEAM_TRY(chk.check(d_src_of, rows->rows * 4));
  if (!aligned(d_row_of, 4) || !aligned(d_src_of, 4) || !aligned(d_weights, 4) || !aligned(d_dweights, 4))
    return GLEAM_ERR_INVALID_ARG;
  RowsArgs a{};
  a.a = static_cast<const uint8_t*>(dy->d);
  a.b = static_cast<const uint8_t*>(rows->d);
  a.lda = dy->ld * size;
  a.ldb = rows->ld * size;
  a.a_rows = dy->rows;
  a.b_rows = rows->rows;
  a.cols = dy->cols;
  a.tokens = dy->rows;
  a.row_of = d_row_of;
  a.src_of = d_src_of;
  a.w = d_weights;
  a.per_token = per_token;
  a.dtype = (uint32_t)dy->dtype;
  a.vec = aligned(dy->d, 16) && a.lda % 16 == 0 && aligned(rows->d, 16) && a.ldb % 16 == 0 &&
          aligned(d_drows, 16) && dy->cols * size % 16 == 0;
  a.out = static_cast<uint8_t*>(d_drows);
  a.dw = d_dweights;
  return cuda_err(launch_expert_combine_grad(a, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
