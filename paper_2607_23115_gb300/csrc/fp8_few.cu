// y = quantised(x) W^T for few rows of x, in one launch.
//
// Bound by the weights' bytes and, below that, by the latency of a launch: no kernel runs
// before it.  A block takes slabs of 16 rows of w; its 16 warps share out the blocks of 128
// along the contraction.  Each warp quantises its own blocks of x once, into shared memory,
// and then multiplies slab after slab by mma.sync.m16n8k32: 8 rows of x are its columns, so 1
// costs what 8 cost, and 5th-generation tensor cores, whose tile has 128 lanes behind shared
// and tensor memory, would only add trips.  A warp's chunks of weights (2 KiB of a tile, in a
// row) come by bulk copies into a ring of its own, two to six ahead: held in registers, the
// next ones do not fit beside x's work.  The warps' sums of a slab meet in shared memory and
// are added in the order of the contraction.  1 x 14336 x 4096: 14.2 us, 4.1 TB/s; 1 x 1024 x
// 4096: 5.3 us, which is the launch, x's quantisation and the round trips.
//
// mma.sync pairs byte i of A's and B's registers whatever k they stand for: a lane takes 16
// neighbouring bytes of a row (its piece of the tile) for four registers of each operand.
#include <algorithm>

#include "operators.cuh"

namespace gleam {
namespace {

constexpr int kWarps = 16;
constexpr int kThreads = 32 * kWarps;
constexpr int kRows = 16;   // of w, for a block
constexpr uint32_t kChunk = kRows * kTile;  // a slab's bytes of one block of the contraction
constexpr uint32_t kMaxStages = 6;           // chunks of a warp on their way
constexpr uint32_t kAhead = 3;               // slabs whose weights are asked for to L2 before the wait

__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Waits for a phase for at most limit_ns.  The clock answers late, so it is asked after some looks.
__device__ __forceinline__ bool arrived(uint32_t bar, uint32_t parity, unsigned long long limit_ns) {
#pragma unroll 1
  for (int i = 0; i < 64; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  return mbar_wait(bar, parity, limit_ns);
}

// A lane's two pieces of a block: 16 values from column `col` and 16 from `col` + 64, as loaded.
template <int DT>
struct Pieces {
  static constexpr int kLoads = DT == GLEAM_FP32 ? 8 : 4;
  uint4 w[kLoads];
  __device__ __forceinline__ void load(const uint8_t* row, uint64_t col, bool present) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint64_t half = i >= kLoads / 2 ? 64 : 0;
      w[i] = make_uint4(0, 0, 0, 0);
      if (present)
        w[i] = __ldg(reinterpret_cast<const uint4*>(row + (col + half) * dtype_bytes(DT)) + i % (kLoads / 2));
    }
  }
  // value by value, zeros past the row's end
  __device__ __forceinline__ void load_some(const uint8_t* row, uint64_t col, uint64_t cols) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      float v[Piece<DT>::kValues];
#pragma unroll
      for (int j = 0; j < Piece<DT>::kValues; ++j) {
        const uint64_t c = col + (i >= kLoads / 2 ? 64 : 0) + i % (kLoads / 2) * Piece<DT>::kValues + j;
        v[j] = c < cols ? load_value<DT>(row + c * dtype_bytes(DT)) : 0.0f;
      }
      w[i] = Piece<DT>::put(v);
    }
  }
  __device__ __forceinline__ void get(float (&v)[32]) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      float u[Piece<DT>::kValues];
      Piece<DT>::get(w[i], u);
#pragma unroll
      for (int j = 0; j < Piece<DT>::kValues; ++j) v[i * Piece<DT>::kValues + j] = u[j];
    }
  }
};

__device__ __forceinline__ void prefetch(const uint8_t* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

struct Shared {
  unsigned long long full[kWarps][kMaxStages];
  uint32_t first[kMaxExperts + 1];  // an expert's first item
  uint32_t total;
};

// Shared memory of a block for x and the chunks (the rest is static).
constexpr uint32_t kFewMost = 184u << 10;
// Bytes of x's part of shared memory for a block of the contraction: 8 registers a lane, and 8 scales.
__host__ __device__ constexpr uint32_t x_bytes(int groups) { return groups * (32 * 32 + 8 * 4); }

template <int DT, int kGroups>
__global__ void __launch_bounds__(kThreads, 1) k_fp8_few(const __grid_constant__ FewArgs a) {
  extern __shared__ __align__(128) uint8_t chunks[];  // [warp][stage][kChunk], then x
  __shared__ Shared sh;
  __shared__ float part[2][kWarps][kGroups][kRows][9];  // 9: columns apart by no power of two
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const uint32_t slabs = (uint32_t)((a.n + kRows - 1) / kRows), kb = (uint32_t)a.kb;
  uint8_t* x_mem = chunks + (size_t)kWarps * a.stages * kChunk;
  uint4* xq = reinterpret_cast<uint4*>(x_mem);                                  // [kb][group][2][lane]
  float* xs = reinterpret_cast<float*>(x_mem + (size_t)kb * kGroups * 32 * 32);  // [kb][group][8]
  // The warp's ring of chunks: lane 0 asks for them and waits for them.
  uint8_t* ring = chunks + (size_t)warp * a.stages * kChunk;
  const uint32_t bars = (uint32_t)__cvta_generic_to_shared(&sh.full[warp][0]);
  uint32_t stage = 0, phase = 0;       // read next
  uint32_t to_stage = 0;                // filled next
  uint64_t asked = 0;                   // chunks so far
  bool ok = true;                       // no wait has run out: once one has, no chunk is asked for
  const uint32_t most = blockIdx.x == 0 && warp == 0 ? a.skip : kNoSkip;
  if (lane == 0) {
    for (uint32_t i = 0; i < a.stages; ++i) mbar_init(bars + 8 * i);
    mbar_fence_init();
  }
  // 16 rows of a tile are 2 KiB in a row; a warp asks for its own blocks'
  auto fetch = [&](const uint8_t* we, uint32_t slab) {
    const uint8_t* p = we + (uint64_t)(slab * kRows / kTile) * kb * kTileBytes + slab * kRows % kTile * kTile;
    for (uint32_t k = warp + lane * kWarps; k < kb; k += 32 * kWarps)
      prefetch(p + (uint64_t)k * kTileBytes, kRows * kTile);
  };
  if (a.experts == 0) {
    // which weights is known: they come to L2, whatever the kernel before this one writes
    const uint32_t s0 = (uint32_t)((uint64_t)slabs * blockIdx.x / gridDim.x);
    const uint32_t s1 = (uint32_t)((uint64_t)slabs * (blockIdx.x + 1) / gridDim.x);
    for (uint32_t s = s0; s < min(s0 + kAhead, s1); ++s) fetch(a.wq, s);
  }
  pdl_wait();
  uint32_t total = slabs;
  if (a.experts != 0) {
    // items: the slabs of each expert that has rows
    if (warp == 0) {
      uint32_t sum = 0;
      for (uint32_t e0 = 0; e0 < a.experts; e0 += 32) {
        const uint32_t e = e0 + lane;
        uint32_t mine = 0;
        if (e < a.experts) {
          const int32_t o = a.offsets[e], c = a.counts[e];
          const bool bad =
              c != 0 && (o < 0 || c < 0 || (o & (kTile - 1)) != 0 || (uint64_t)o + (uint64_t)c > a.rows);
          if (bad) *a.status = GLEAM_ERR_INVALID_ARG;
          mine = c != 0 && !bad ? slabs : 0;
        }
        uint32_t up = mine;
        for (int d = 1; d < 32; d <<= 1) {
          const uint32_t o = __shfl_up_sync(0xffffffffu, up, d);
          if (lane >= (uint32_t)d) up += o;
        }
        if (e < a.experts) sh.first[e] = sum + up - mine;
        sum += __shfl_sync(0xffffffffu, up, 31);
      }
      if (lane == 0) {
        sh.first[a.experts] = sum;
        sh.total = sum;
      }
    }
    __syncthreads();
    total = sh.total;
  }
  // this block's items: as many as the others', or one more
  const uint32_t item0 = (uint32_t)((uint64_t)total * blockIdx.x / gridDim.x);
  const uint32_t item1 = (uint32_t)((uint64_t)total * (blockIdx.x + 1) / gridDim.x);
  uint32_t side = 0;

  for (uint32_t item = item0; item < item1;) {
    // the slabs [slab0, slab1) of one expert
    uint32_t e = 0, slab0 = item, slab1 = item1, row0 = 0, rows = (uint32_t)a.rows;
    if (a.experts != 0) {
      uint32_t lo = 0, hi = a.experts;
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (sh.first[mid] <= item) lo = mid;
        else hi = mid;
      }
      e = lo;
      slab0 = item - sh.first[lo];
      slab1 = min(slabs, item1 - sh.first[lo]);
      row0 = (uint32_t)a.offsets[e];
      rows = (uint32_t)a.counts[e];
    }
    item += slab1 - slab0;
    const uint8_t* we = a.wq + (uint64_t)e * a.wrt * kb * kTileBytes;
    const float* wse = a.ws + (uint64_t)e * a.wrt * kb;
    for (uint32_t x0 = 0; x0 < rows; x0 += 8 * kGroups) {
      // Chunks: the warp's blocks of a slab, slab after slab, a.stages of them on their way.
      uint32_t lslab = slab0, lk = warp;  // asked for next
      auto ask = [&]() {
        if (lane == 0 && ok && lslab < slab1 && lk < kb && (most == kNoSkip || asked < most)) {
          ++asked;
          const uint32_t wt = lslab * kRows / kTile;
          mbar_expect_tx(bars + 8 * to_stage, kChunk);
          copy_in((uint32_t)__cvta_generic_to_shared(ring + to_stage * kChunk),
                  we + ((uint64_t)wt * kb + lk) * kTileBytes + lslab * kRows % kTile * kTile, kChunk,
                  bars + 8 * to_stage);
          if (++to_stage == a.stages) to_stage = 0;
          lk += kWarps;
          if (lk >= kb) {
            lk = warp;
            ++lslab;
          }
        }
      };
      for (uint32_t i = 0; i < a.stages; ++i) ask();
      // quantise the warp's blocks of these rows; lane (g, t) has row g's pieces t and t + 4
#pragma unroll
      for (int q = 0; q < kGroups; ++q) {
        int64_t from = -1;
        if (x0 + 8 * q + g < rows) {
          from = row0 + x0 + 8 * q + g;
          if (a.src != nullptr) {
            const int32_t slot = a.src[from];
            if (slot < 0) from = -1;
            else if (a.per_token != 0) from = (uint32_t)slot / a.per_token;
          }
          if (from >= (int64_t)a.x_rows) from = -1;
        }
        const uint8_t* xrow = a.x + (uint64_t)(from < 0 ? 0 : from) * a.ld;
        auto keep = [&](uint32_t k, const Pieces<DT>& raw) {
          float v[32];
          raw.get(v);
          uint32_t most = 0;
#pragma unroll
          for (int j = 0; j < 32; ++j) most = max(most, __float_as_uint(v[j]) & 0x7fffffffu);
          most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
          most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
          const float2 sc = group_scale(most);
          uint32_t b[8];
#pragma unroll
          for (int j = 0; j < 8; ++j)
            b[j] = e4m3x4(v[4 * j] * sc.y, v[4 * j + 1] * sc.y, v[4 * j + 2] * sc.y, v[4 * j + 3] * sc.y);
          xq[((k * kGroups + q) * 2) * 32 + lane] = make_uint4(b[0], b[1], b[2], b[3]);
          xq[((k * kGroups + q) * 2 + 1) * 32 + lane] = make_uint4(b[4], b[5], b[6], b[7]);
          if (t == 0) xs[(k * kGroups + q) * 8 + g] = sc.x;
        };
        // several blocks' loads before the first is used, where they are whole and aligned
        constexpr uint32_t kOnce = 2;
        const uint32_t whole = a.vec != 0 ? (uint32_t)(a.cols / kTile) : 0;
        uint32_t k = warp;
        for (; k + (kOnce - 1) * kWarps < whole; k += kOnce * kWarps) {
          Pieces<DT> raw[kOnce];
#pragma unroll
          for (uint32_t i = 0; i < kOnce; ++i) raw[i].load(xrow, (k + i * kWarps) * kTile + 16 * t, from >= 0);
#pragma unroll
          for (uint32_t i = 0; i < kOnce; ++i) keep(k + i * kWarps, raw[i]);
        }
#pragma unroll 1
        for (; k < kb; k += kWarps) {
          Pieces<DT> raw;
          if (k < whole) raw.load(xrow, k * kTile + 16 * t, from >= 0);
          else raw.load_some(xrow, k * kTile + 16 * t, from >= 0 ? a.cols : 0);
          keep(k, raw);
        }
      }
      __syncwarp();

      // this lane's two pieces of rows g and g + 8 of a chunk
      const uint32_t p0 = g * kTile + ((t ^ g) << 4), p1 = g * kTile + (((t + 4) ^ g) << 4);
      for (uint32_t slab = slab0; slab < slab1; ++slab) {
        const float* wsp = wse + (uint64_t)(slab * kRows / kTile) * kb;
        float acc[kGroups][4] = {};
        for (uint32_t k = warp; k < kb; k += kWarps) {
          const float sw = __ldg(wsp + k);
          if (lane == 0 && ok) ok = arrived(bars + 8 * stage, phase, a.wait_ns);
          __syncwarp();
          const uint8_t* c0 = ring + stage * kChunk;
          const uint4 w0 = *reinterpret_cast<const uint4*>(c0 + p0), w1 = *reinterpret_cast<const uint4*>(c0 + p1);
          const uint4 w2 = *reinterpret_cast<const uint4*>(c0 + 8 * kTile + p0),
                      w3 = *reinterpret_cast<const uint4*>(c0 + 8 * kTile + p1);
          if (++stage == a.stages) {
            stage = 0;
            phase ^= 1;
          }
#pragma unroll
          for (int q = 0; q < kGroups; ++q) {
            const uint4 b0 = xq[((k * kGroups + q) * 2) * 32 + lane];
            const uint4 b1 = xq[((k * kGroups + q) * 2 + 1) * 32 + lane];
            // columns 2t and 2t + 1 are rows 2t and 2t + 1 of x
            const float2 sx = *reinterpret_cast<const float2*>(&xs[(k * kGroups + q) * 8 + 2 * t]);
            float c[4] = {};
            mma_e4m3(c, w0.x, w2.x, w0.y, w2.y, b0.x, b0.y);
            mma_e4m3(c, w0.z, w2.z, w0.w, w2.w, b0.z, b0.w);
            mma_e4m3(c, w1.x, w3.x, w1.y, w3.y, b1.x, b1.y);
            mma_e4m3(c, w1.z, w3.z, w1.w, w3.w, b1.z, b1.w);
            const float s0 = sw * sx.x, s1 = sw * sx.y;
            acc[q][0] = fmaf(c[0], s0, acc[q][0]);
            acc[q][1] = fmaf(c[1], s1, acc[q][1]);
            acc[q][2] = fmaf(c[2], s0, acc[q][2]);
            acc[q][3] = fmaf(c[3], s1, acc[q][3]);
          }
          __syncwarp();  // the chunk has been read
          ask();
        }
        // the two sides take turns: one barrier a slab
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
          part[side][warp][q][g][2 * t] = acc[q][0];
          part[side][warp][q][g][2 * t + 1] = acc[q][1];
          part[side][warp][q][g + 8][2 * t] = acc[q][2];
          part[side][warp][q][g + 8][2 * t + 1] = acc[q][3];
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 8 * kGroups * kRows; i += kThreads) {
          const uint32_t col = i / kRows, rr = i % kRows;
          const uint64_t j = (uint64_t)slab * kRows + rr;
          if (x0 + col < rows && j < a.n) {
            float sum = 0;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) sum += part[side][k][col / 8][rr][col % 8];
            store_value<DT>(a.y + ((row0 + x0 + col) * a.y_ld + j) * dtype_bytes(DT), sum);
          }
        }
        side ^= 1;
      }
      __syncwarp();  // this warp's blocks of x have been read
    }
  }
  // a wait ran out: chunks on their way land before this block's memory goes to another
  if (lane == 0 && !ok) {
    *a.status = GLEAM_ERR_TIMEOUT;
    settle_ring(&asked, 1, a.stages, [](uint32_t) {},
                [&](uint32_t i, uint32_t parity) { mbar_wait(bars + 8 * i, parity, kOperatorWaitNs); });
  }
}

template <int kGroups>
cudaError_t start(const FewArgs& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  void (*k)(FewArgs) = a.dtype == GLEAM_BF16   ? k_fp8_few<GLEAM_BF16, kGroups>
                       : a.dtype == GLEAM_FP16 ? k_fp8_few<GLEAM_FP16, kGroups>
                                               : k_fp8_few<GLEAM_FP32, kGroups>;
  // x first, then as many stages as there is room for
  const uint32_t x = (uint32_t)a.kb * x_bytes(kGroups), room = kFewMost - x;
  FewArgs b = a;
  b.stages = std::min<uint32_t>(kMaxStages, room / (kWarps * kChunk));
  const uint32_t smem = x + b.stages * kWarps * kChunk;
  // the most that any call takes: another thread's call of the same kernel must not find it lowered
  if ((e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewMost)) != cudaSuccess)
    return e;
  const uint64_t slabs = (a.n + kRows - 1) / kRows;
  // the kernel counts items in 32 bits, whatever the offsets on the device say
  if (std::max<uint64_t>(a.experts, 1) * slabs >= 0x7fffffffull) return cudaErrorInvalidValue;
  const uint64_t items = a.experts == 0 ? slabs : std::min<uint64_t>(a.experts, a.rows) * slabs;
  const uint64_t at_once = (uint64_t)sms;
  return launch_chained(k, dim3((unsigned)std::min<uint64_t>(items, at_once)), dim3(kThreads), smem, s, 1, b);
}

}  // namespace

bool few_fits(uint64_t rows, uint64_t kb) {
  return kb * x_bytes(rows <= 8 ? 1 : 2) + 2 * kWarps * kChunk <= kFewMost;
}

cudaError_t launch_few(const FewArgs& a, cudaStream_t s) {
  return a.experts != 0 || a.rows <= 8 ? start<1>(a, s) : start<2>(a, s);
}

}  // namespace gleam
