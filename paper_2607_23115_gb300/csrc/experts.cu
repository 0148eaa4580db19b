// Tokens sorted by expert and back: a stable counting sort of the router's slots,
// the rows' gather, their weighted sum per token and its gradients.
#include <cooperative_groups.h>

#include <algorithm>

#include "operators.cuh"

namespace gleam {
namespace {

namespace cg = cooperative_groups;

// ---- sort ------------------------------------------------------------------
//
// One cluster sorts all slots: each warp owns a contiguous range of them, counts
// its slots by expert, and, once the counts of the warps and blocks before it
// are known, gives its own out in order.  Slots of one expert in a batch of 32 are
// told apart by a match among the lanes, so no atomic decides an order.  Bound by its
// passes' latency: 38 slots 4.5 us, 32,768 slots of 64 experts 12.7 us.
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;

struct SortShared {
  uint32_t total[kMaxExperts];  // this block's slots by expert
  uint32_t before[kMaxExperts]; // offset, and the blocks before
  uint32_t scan[kSortWarps];
};

__device__ __forceinline__ uint32_t slot_expert(const SortArgs& a, uint64_t i) {
  if (i >= a.slots) return a.experts;
  if (a.wide) {
    const long long v = static_cast<const long long*>(a.ids)[i];
    return v < 0 || v >= (long long)a.experts ? a.experts : (uint32_t)v;
  }
  const uint32_t v = static_cast<const uint32_t*>(a.ids)[i];
  return min(v, a.experts);
}

__global__ void __launch_bounds__(kSortThreads, 1) k_expert_sort(const __grid_constant__ SortArgs a) {
  extern __shared__ uint32_t hist[];  // [warps][experts]
  __shared__ SortShared sh;
  pdl_wait();
  cg::cluster_group cl = cg::this_cluster();
  const uint32_t rank = cl.block_rank(), blocks = cl.num_blocks();
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, E = a.experts;
  const uint32_t own = blockDim.x / 32;  // warps of a block
  const uint64_t warps = (uint64_t)blocks * own;
  const uint64_t per = ((a.slots + warps - 1) / warps + 31) & ~31ull;
  const uint64_t i0 = (rank * (uint64_t)own + warp) * per, i1 = min(a.slots, i0 + per);
  uint32_t* mine = hist + warp * E;

  for (uint32_t i = threadIdx.x; i < own * E; i += blockDim.x) hist[i] = 0;
  __syncthreads();
  for (uint64_t i = i0; i < i1; i += 32) {
    const uint32_t e = slot_expert(a, i + lane < i1 ? i + lane : a.slots);
    const uint32_t same = __match_any_sync(0xffffffffu, e);
    if (e < E && lane == (uint32_t)(__ffs(same) - 1)) mine[e] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  const uint32_t e = threadIdx.x;
  if (e < E) {
    uint32_t sum = 0;
    for (uint32_t w = 0; w < own; ++w) {
      const uint32_t c = hist[w * E + e];
      hist[w * E + e] = sum;
      sum += c;
    }
    sh.total[e] = sum;
  }
  cl.sync();
  uint32_t count = 0, before = 0;
  if (e < E) {
    for (uint32_t b = 0; b < blocks; ++b) {
      const uint32_t c = cl.map_shared_rank(sh.total, b)[e];
      if (b < rank) before += c;
      count += c;
    }
  }
  // offsets: sums of the aligned counts
  const uint32_t room = (count + a.align - 1) / a.align * a.align;
  uint32_t up = room;
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, up, d);
    if (lane >= (uint32_t)d) up += o;
  }
  if (lane == 31) sh.scan[warp] = up;
  __syncthreads();
  uint32_t base = 0, used = 0;
  for (uint32_t w = 0; w < own; ++w) {
    if (w < warp) base += sh.scan[w];
    used += sh.scan[w];
  }
  const uint32_t at = base + up - room;
  if (e < E) {
    sh.before[e] = at + before;
    if (rank == 0) {
      a.offsets[e] = (int32_t)at;
      a.counts[e] = (int32_t)count;
    }
    // rows that pad the expert's
    if (e % blocks == rank)
      for (uint32_t r = at + count; r < at + room; ++r) a.src_of[r] = -1;
  }
  if (rank == 0 && threadIdx.x == 0) a.offsets[E] = (int32_t)used;
  for (uint64_t r = used + rank * (uint64_t)blockDim.x + threadIdx.x; r < a.cap;
       r += (uint64_t)blocks * blockDim.x)
    a.src_of[r] = -1;
  __syncthreads();
  for (uint64_t i = i0; i < i1; i += 32) {
    const uint64_t slot = i + lane;
    const uint32_t x = slot_expert(a, slot < i1 ? slot : a.slots);
    const uint32_t same = __match_any_sync(0xffffffffu, x);
    const uint32_t earlier = __popc(same & ((1u << lane) - 1));
    if (x < E) {
      const uint32_t row = sh.before[x] + mine[x] + earlier;
      a.row_of[slot] = (int32_t)row;
      a.src_of[row] = (int32_t)slot;
    } else if (slot < i1) {
      a.row_of[slot] = -1;
    }
    __syncwarp();
    if (x < E && earlier == 0) mine[x] += __popc(same);
    __syncwarp();
  }
  cl.sync();  // a block's counts stay until the others have read them
}

// ---- rows ------------------------------------------------------------------

// A thread takes 16 bytes of a row at a time (or, where rows start at no multiple of 16
// bytes, a value), a block 128 neighbouring ones; few rows spread over more blocks so.  Bound
// by memory, and for few rows by latency: the rows' numbers first, then all of a token's rows.
// 8192 tokens x 4 rows of 8 KiB: gather 75 us (5.4 TB/s), combine 53 (6.3), its gradient 102 (6.6,
// some of it from L2); of 8,190 bytes, value by value: 198, 360 and 211.
constexpr int kRowThreads = 128;
constexpr int kSlots = 4;  // rows of a token in flight

// The row that a slot or -1 names, or -1.
__device__ __forceinline__ int64_t row_in(int32_t r, uint64_t rows) {
  return r >= 0 && (uint64_t)r < rows ? (int64_t)r : -1;
}

// Blocks (x: row, y: part of it).
constexpr int kGatherPieces = 4;  // of a thread
__global__ void __launch_bounds__(kRowThreads) k_expert_gather(const __grid_constant__ RowsArgs a) {
  pdl_wait();
  const int32_t slot = a.src_of[blockIdx.x];
  const int64_t t = slot < 0 ? -1 : row_in((int32_t)((uint32_t)slot / a.per_token), a.a_rows);
  const uint64_t bytes = a.cols * dtype_bytes(a.dtype);
  uint8_t* out = a.out + blockIdx.x * bytes;
  const uint8_t* in = a.a + (t < 0 ? 0 : t) * a.lda;
  constexpr uint64_t kPart = kRowThreads * kGatherPieces * 16;
  const uint64_t end = min(bytes, (blockIdx.y + 1) * kPart);
  if (a.vec) {
    uint4 v[kGatherPieces];
#pragma unroll
    for (int i = 0; i < kGatherPieces; ++i) {
      const uint64_t c = blockIdx.y * kPart + (i * kRowThreads + threadIdx.x) * 16;
      v[i] = make_uint4(0, 0, 0, 0);
      if (t >= 0 && c < end) v[i] = __ldg(reinterpret_cast<const uint4*>(in + c));
    }
#pragma unroll
    for (int i = 0; i < kGatherPieces; ++i) {
      const uint64_t c = blockIdx.y * kPart + (i * kRowThreads + threadIdx.x) * 16;
      if (c < end) *reinterpret_cast<uint4*>(out + c) = v[i];
    }
  } else {
    for (uint64_t c = blockIdx.y * kPart + threadIdx.x * 2; c < end; c += kRowThreads * 2)
      *reinterpret_cast<uint16_t*>(out + c) = t < 0 ? 0 : *reinterpret_cast<const uint16_t*>(in + c);
  }
}

// Blocks (x: token, y: part of its row).
template <int DT>
__global__ void __launch_bounds__(kRowThreads) k_expert_combine(const __grid_constant__ RowsArgs a) {
  constexpr int kN = Piece<DT>::kValues;
  constexpr uint64_t kSize = dtype_bytes(DT);
  pdl_wait();
  const uint64_t t = blockIdx.x;
  const int32_t* row_of = a.row_of + t * a.per_token;
  const float* w = a.w == nullptr ? nullptr : a.w + t * a.per_token;
  uint8_t* out = a.out + t * a.cols * kSize;
  const uint64_t c0 = (uint64_t)blockIdx.y * kRowThreads * kN;
  if (a.vec) {
    const uint64_t c = c0 + threadIdx.x * kN;
    if (c >= a.cols) return;
    float sum[kN] = {};
    for (uint32_t j0 = 0; j0 < a.per_token; j0 += kSlots) {
      int32_t r[kSlots];
      float f[kSlots];
      uint4 v[kSlots];
#pragma unroll
      for (int j = 0; j < kSlots; ++j) {
        r[j] = j0 + j < a.per_token ? (int32_t)row_in(row_of[j0 + j], a.a_rows) : -1;
        f[j] = w != nullptr && j0 + j < a.per_token ? w[j0 + j] : 1.0f;
      }
#pragma unroll
      for (int j = 0; j < kSlots; ++j)
        if (r[j] >= 0) v[j] = __ldg(reinterpret_cast<const uint4*>(a.a + (uint64_t)r[j] * a.lda + c * kSize));
#pragma unroll
      for (int j = 0; j < kSlots; ++j) {
        if (r[j] < 0) continue;
        float u[kN];
        Piece<DT>::get(v[j], u);
#pragma unroll
        for (int i = 0; i < kN; ++i) sum[i] = fmaf(f[j], u[i], sum[i]);
      }
    }
    Piece<DT>::store(out + c * kSize, sum);
  } else {
    for (uint64_t c = c0 + threadIdx.x; c < min(a.cols, c0 + kRowThreads * kN); c += kRowThreads) {
      float sum = 0;
      for (uint32_t j = 0; j < a.per_token; ++j) {
        const int64_t r = row_in(row_of[j], a.a_rows);
        if (r >= 0) sum = fmaf(w == nullptr ? 1.0f : w[j], load_value<DT>(a.a + r * a.lda + c * kSize), sum);
      }
      store_value<DT>(out + c * kSize, sum);
    }
  }
}

// Blocks 0 .. tokens - 1: a token's slots, kSlots at a time, its dy read once for them; the
// others zero the rows of no slot, kFillRows each.
constexpr int kFillRows = 8;
template <int DT>
__global__ void __launch_bounds__(kRowThreads) k_expert_combine_grad(const __grid_constant__ RowsArgs a) {
  constexpr int kN = Piece<DT>::kValues;
  constexpr uint64_t kSize = dtype_bytes(DT);
  __shared__ float part[kRowThreads / 32][kSlots];
  pdl_wait();
  if (blockIdx.x >= a.tokens) {
    const uint64_t r0 = (blockIdx.x - a.tokens) * kFillRows;
    for (uint64_t row = r0; row < min(r0 + kFillRows, a.b_rows); ++row) {
      if (a.src_of[row] >= 0) continue;
      uint8_t* out = a.out + row * a.cols * kSize;
      const float none[kN] = {};
      if (a.vec)
        for (uint64_t c = threadIdx.x * kN; c < a.cols; c += kRowThreads * kN) Piece<DT>::store(out + c * kSize, none);
      else
        for (uint64_t c = threadIdx.x; c < a.cols; c += kRowThreads) store_value<DT>(out + c * kSize, 0.0f);
    }
    return;
  }
  const uint64_t t = blockIdx.x;
  const uint8_t* dy = a.a + t * a.lda;
  for (uint32_t j0 = 0; j0 < a.per_token; j0 += kSlots) {
    int32_t r[kSlots];
    float f[kSlots], dot[kSlots] = {};
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
      const bool is = j0 + j < a.per_token;
      r[j] = is ? (int32_t)row_in(a.row_of[t * a.per_token + j0 + j], a.b_rows) : -1;
      f[j] = is ? a.w[t * a.per_token + j0 + j] : 0.0f;
    }
    if (a.vec) {
      for (uint64_t c = threadIdx.x * kN; c < a.cols; c += kRowThreads * kN) {
        float d[kN];
        Piece<DT>::load(dy + c * kSize, d);
        uint4 v[kSlots];
#pragma unroll
        for (int j = 0; j < kSlots; ++j)
          if (r[j] >= 0) v[j] = __ldg(reinterpret_cast<const uint4*>(a.b + (uint64_t)r[j] * a.ldb + c * kSize));
#pragma unroll
        for (int j = 0; j < kSlots; ++j) {
          if (r[j] < 0) continue;
          float u[kN], o[kN];
          Piece<DT>::get(v[j], u);
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            dot[j] = fmaf(u[i], d[i], dot[j]);
            o[i] = d[i] * f[j];
          }
          Piece<DT>::store(a.out + ((uint64_t)r[j] * a.cols + c) * kSize, o);
        }
      }
    } else {
      for (uint64_t c = threadIdx.x; c < a.cols; c += kRowThreads) {
        const float d = load_value<DT>(dy + c * kSize);
#pragma unroll
        for (int j = 0; j < kSlots; ++j) {
          if (r[j] < 0) continue;
          dot[j] = fmaf(load_value<DT>(a.b + (uint64_t)r[j] * a.ldb + c * kSize), d, dot[j]);
          store_value<DT>(a.out + ((uint64_t)r[j] * a.cols + c) * kSize, d * f[j]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
      for (int d = 16; d; d >>= 1) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], d);
      if (threadIdx.x % 32 == 0) part[threadIdx.x / 32][j] = dot[j];
    }
    __syncthreads();
    if (threadIdx.x < kSlots && j0 + threadIdx.x < a.per_token) {
      float sum = 0;
      for (int i = 0; i < kRowThreads / 32; ++i) sum += part[i][threadIdx.x];
      a.dw[t * a.per_token + j0 + threadIdx.x] = sum;
    }
    __syncthreads();
  }
}

template <class K>
K by_dtype(uint32_t dtype, K bf16, K fp16, K fp32) {
  return dtype == GLEAM_BF16 ? bf16 : dtype == GLEAM_FP16 ? fp16 : fp32;
}

}  // namespace

// Few slots take one block of as many threads as there are slots or experts, which has
// no cluster to wait for.
cudaError_t launch_expert_sort(const SortArgs& a, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(k_expert_sort, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)(kSortWarps * kMaxExperts * 4));
  if (e != cudaSuccess) return e;
  const unsigned blocks = a.slots <= 4096 ? 1 : 8;
  uint64_t threads = kSortThreads;
  if (blocks == 1) threads = std::min<uint64_t>(threads, (std::max<uint64_t>({a.slots, a.experts, 1}) + 31) / 32 * 32);
  const size_t smem = threads / 32 * a.experts * 4;
  return launch_chained(k_expert_sort, dim3(blocks), dim3((unsigned)threads), smem, s, blocks, a);
}

// Blocks that go over a row of `bytes`.
static unsigned parts_of(uint64_t bytes, uint64_t part) { return (unsigned)((bytes + part - 1) / part); }

cudaError_t launch_expert_gather(const RowsArgs& a, cudaStream_t s) {
  const unsigned parts = parts_of(a.cols * dtype_bytes(a.dtype), kRowThreads * kGatherPieces * 16);
  if (parts > 65535) return cudaErrorInvalidValue;
  return launch_chained(k_expert_gather, dim3((unsigned)a.b_rows, parts), dim3(kRowThreads), 0, s, 1, a);
}

cudaError_t launch_expert_combine(const RowsArgs& a, cudaStream_t s) {
  const unsigned parts = parts_of(a.cols * dtype_bytes(a.dtype), kRowThreads * 16);
  if (parts > 65535) return cudaErrorInvalidValue;
  return launch_chained(by_dtype(a.dtype, k_expert_combine<GLEAM_BF16>, k_expert_combine<GLEAM_FP16>,
                                 k_expert_combine<GLEAM_FP32>),
                        dim3((unsigned)a.tokens, parts), dim3(kRowThreads), 0, s, 1, a);
}

cudaError_t launch_expert_combine_grad(const RowsArgs& a, cudaStream_t s) {
  const uint64_t blocks = a.tokens + (a.b_rows + kFillRows - 1) / kFillRows;
  return launch_chained(by_dtype(a.dtype, k_expert_combine_grad<GLEAM_BF16>,
                                 k_expert_combine_grad<GLEAM_FP16>, k_expert_combine_grad<GLEAM_FP32>),
                        dim3((unsigned)blocks), dim3(kRowThreads), 0, s, 1, a);
}

}  // namespace gleam
