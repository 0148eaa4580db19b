// What the kernels on 8-bit weights and on tokens sorted by expert share: their
// arguments, element types and launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "gleam_internal.cuh"
#include "ring.cuh"

namespace gleam {

constexpr uint32_t kTile = 128;                // rows and columns of a tile, values of a group
constexpr uint32_t kTileBytes = kTile * kTile;  // e4m3
constexpr uint32_t kMaxExperts = 1024;
// Limit of a wait inside the product kernels (gleam_operators_debug_set may lower it), and of a
// wait for copies and products in flight once another has run out.
constexpr unsigned long long kOperatorWaitNs = 4000000000ULL;
constexpr uint32_t kNoSkip = 0xffffffffu;

struct QuantizeArgs {
  const uint8_t* x;
  uint64_t ld, stride;  // bytes
  uint64_t x_rows, cols;
  uint64_t rows;        // of the output
  uint64_t rt, kb;      // row tiles and column blocks
  const int32_t* src;
  uint32_t per_token;
  uint32_t count;
  uint32_t dtype, form;
  uint32_t vec;         // rows start 4-element aligned
  uint32_t fill;        // rows that are none are written as zeros
  uint32_t leads;       // a product of the same call follows and may start early
  uint8_t *q, *qt;
  float *s, *st;
};

struct ProductArgs {
  const uint8_t *xq, *wq;
  const float *xs, *ws;
  uint8_t* y;
  uint64_t ld, ystride;   // elements
  uint64_t m, n;
  uint64_t kb;            // blocks along the contraction
  uint64_t xrt, wrt;      // row tiles of x and of one w
  uint64_t tiles;         // without experts: all; over sums: all; over rows: from the offsets
  uint32_t dtype, w_form;
  uint32_t experts, over;
  uint32_t vec;           // y's rows start 16-byte aligned
  uint32_t w_ready;       // w is not written by the kernel before this one on the stream
  const int32_t *offsets, *counts;
  int32_t* status;        // the caller's word, or the GPU's
  unsigned long long wait_ns;
  uint32_t skip;          // test hook: block 0's first copying thread stops after so many stages
};

// y = quantised(x) W^T in one launch, for few rows.
struct FewArgs {
  const uint8_t* x;
  uint64_t ld;            // bytes
  uint64_t x_rows, cols;
  uint64_t rows;          // of y; with experts: sorted
  const int32_t* src;
  uint32_t per_token;
  uint32_t dtype, vec;    // vec: x's rows start 16-byte aligned
  uint32_t stages;        // of a warp's ring (the launch fills it in)
  const uint8_t* wq;
  const float* ws;
  uint64_t n, kb, wrt;
  uint8_t* y;
  uint64_t y_ld;          // elements
  uint32_t experts;
  const int32_t *offsets, *counts;
  int32_t* status;        // the caller's word, or the GPU's
  unsigned long long wait_ns;
  uint32_t skip;          // test hook: block 0 asks for no chunk after so many (kNoSkip: none)
};

struct SortArgs {
  const void* ids;
  uint64_t slots, cap;
  uint32_t experts, align, wide;
  int32_t *offsets, *counts, *row_of, *src_of;
};

struct RowsArgs {  // gather, combine and its gradient
  const uint8_t* a;       // x, rows, or dy
  const uint8_t* b;       // the gradient's rows
  uint64_t lda, ldb;      // bytes
  uint64_t a_rows, b_rows;
  uint64_t cols, tokens;
  const int32_t *row_of, *src_of;
  const float* w;
  uint32_t per_token;
  uint32_t dtype, vec;
  uint8_t* out;
  float* dw;
};

cudaError_t launch_quantize(const QuantizeArgs& a, cudaStream_t s);
cudaError_t launch_product(const ProductArgs& a, uint64_t rows_per_matrix, cudaStream_t s);
// Whether x (rows of one matrix, blocks along the contraction) fits a block of that kernel.
bool few_fits(uint64_t rows, uint64_t kb);
cudaError_t launch_few(const FewArgs& a, cudaStream_t s);
cudaError_t launch_expert_sort(const SortArgs& a, cudaStream_t s);
cudaError_t launch_expert_gather(const RowsArgs& a, cudaStream_t s);
cudaError_t launch_expert_combine(const RowsArgs& a, cudaStream_t s);
cudaError_t launch_expert_combine_grad(const RowsArgs& a, cudaStream_t s);

#ifdef __CUDACC__

__host__ __device__ constexpr uint32_t dtype_bytes(uint32_t dtype) {
  return dtype == GLEAM_FP32 ? 4 : 2;
}

// A bulk copy to shared memory; its bytes arrive at the barrier.
__device__ __forceinline__ void copy_in(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}

template <int DT>
__device__ __forceinline__ float load_value(const uint8_t* p) {
  if constexpr (DT == GLEAM_BF16) return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p));
  else if constexpr (DT == GLEAM_FP16) return __half2float(*reinterpret_cast<const __half*>(p));
  else return *reinterpret_cast<const float*>(p);
}

template <int DT>
__device__ __forceinline__ void store_value(uint8_t* p, float v) {
  if constexpr (DT == GLEAM_BF16) *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v);
  else if constexpr (DT == GLEAM_FP16) *reinterpret_cast<__half*>(p) = __float2half_rn(v);
  else *reinterpret_cast<float*>(p) = v;
}

// Two values of a 16-bit type in one word.
template <int DT>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (DT == GLEAM_BF16) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
  } else {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
}
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (DT == GLEAM_BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}

constexpr uint32_t kLeast = 0x0F800000u;  // 2^-96

// (scale s, factor of the values) of a group whose largest |x| has these bits.
// Bits of |x| order like the values, NaN above all.  Both are products with a
// reciprocal rounded by itself, as the definition in gleam.h has them: a value
// half way between two of e4m3 is common (two bf16 values and a ratio), and the
// last bit of the factor decides where it goes.
__device__ __forceinline__ float2 group_scale(uint32_t bits) {
  const float a = __uint_as_float(max(bits, kLeast));
  return make_float2(__fmul_rn(a, 1.0f / 448.0f), __fmul_rn(__frcp_rn(a), 448.0f));
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  return e4m3x2(a, b) | (e4m3x2(c, d) << 16);
}

// 16 bytes of a row as values (8 of a 16-bit type, 4 in 32 bits) and back.
template <int DT>
struct Piece {
  static constexpr int kValues = DT == GLEAM_FP32 ? 4 : 8;
  static __device__ __forceinline__ void load(const uint8_t* p, float (&v)[kValues]) {
    get(*reinterpret_cast<const uint4*>(p), v);
  }
  static __device__ __forceinline__ void get(uint4 w, float (&v)[kValues]) {
    if constexpr (DT == GLEAM_FP32) {
      v[0] = __uint_as_float(w.x);
      v[1] = __uint_as_float(w.y);
      v[2] = __uint_as_float(w.z);
      v[3] = __uint_as_float(w.w);
    } else {
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<DT>(u[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    }
  }
  static __device__ __forceinline__ void store(uint8_t* p, const float (&v)[kValues]) {
    *reinterpret_cast<uint4*>(p) = put(v);
  }
  static __device__ __forceinline__ uint4 put(const float (&v)[kValues]) {
    uint4 w;
    if constexpr (DT == GLEAM_FP32) {
      w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                     __float_as_uint(v[3]));
    } else {
      w = make_uint4(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]), pack2<DT>(v[4], v[5]),
                     pack2<DT>(v[6], v[7]));
    }
    return w;
  }
};

// Launches a kernel chained to the one before it on its stream: its blocks may
// start while that one ends, and wait (pdl_wait) before they touch memory.  A kernel that ends
// a public call does not let its dependents start early itself (pdl_trigger): what follows may
// read its results without a wait, as an upload with GLEAM_OVERLAP_CALLS reads its payload.
template <class... P>
cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s,
                           uint32_t cluster, P... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 1;
  if (cluster > 1) {
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  cfg.attrs = at;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

#endif  // __CUDACC__

}  // namespace gleam
