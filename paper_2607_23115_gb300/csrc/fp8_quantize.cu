// Quantisation to e4m3 with a scale for each group of 128 values or block of
// 128 x 128, into the tiles that the product reads.
//
// A block of 256 threads takes one tile of 128 x 128 values and keeps it in
// registers as loaded (64 values a thread: 16 rows of 4 neighbouring columns, so that a
// warp reads 256 or 512 bytes of a row at once).  The tile holds every group that
// its rows, its columns or itself make up, so each value is read once whatever
// is asked for: the values along rows, those of the transpose, or both.  Bound by
// memory: size + 1 bytes a value (size + 2 with the transpose).  All of a tile's loads are
// made before the first is used, and four tiles of a 16-bit type fit an SM: 14336 x 4096 of bf16
// take 33 us, 5.3 TB/s, where loads and conversions in turn took 118 and three tiles 36.
#include "operators.cuh"

namespace gleam {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerWarp = 16;

// Four neighbouring values of a row, as loaded, and the largest |x| of several in the order of
// their bits (NaN above all).
template <int DT>
struct Four {
  uint2 w;
  static __device__ __forceinline__ Four zero() { return {make_uint2(0, 0)}; }
  __device__ __forceinline__ void load(const uint8_t* p) { w = __ldg(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ void load_some(const uint8_t* p, uint64_t n) {
    uint32_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = (uint64_t)j < n ? reinterpret_cast<const uint16_t*>(p)[j] : 0;
    w = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
  }
  __device__ __forceinline__ void get(float (&v)[4]) const {
    const float2 a = unpack2<DT>(w.x), b = unpack2<DT>(w.y);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
  }
  struct Most {
    uint2 m;  // of each of the four columns
    __device__ __forceinline__ void add(const Four& f) {
      m.x = __vmaxu2(m.x, f.w.x & 0x7fff7fffu);
      m.y = __vmaxu2(m.y, f.w.y & 0x7fff7fffu);
    }
    __device__ __forceinline__ uint4 each() const {
      return make_uint4(m.x & 0xffff, m.x >> 16, m.y & 0xffff, m.y >> 16);
    }
    __device__ __forceinline__ uint32_t all() const {
      const uint32_t v = __vmaxu2(m.x, m.y);
      return max(v & 0xffff, v >> 16);
    }
  };
  // the 32-bit float of a largest value
  static __device__ __forceinline__ uint32_t widen(uint32_t bits) {
    return __float_as_uint(unpack2<DT>(bits).x);
  }
};
template <>
struct Four<GLEAM_FP32> {
  uint4 w;
  static __device__ __forceinline__ Four zero() { return {make_uint4(0, 0, 0, 0)}; }
  __device__ __forceinline__ void load(const uint8_t* p) { w = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void load_some(const uint8_t* p, uint64_t n) {
    uint32_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = (uint64_t)j < n ? reinterpret_cast<const uint32_t*>(p)[j] : 0;
    w = make_uint4(h[0], h[1], h[2], h[3]);
  }
  __device__ __forceinline__ void get(float (&v)[4]) const {
    v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y);
    v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
  }
  struct Most {
    uint4 m;
    __device__ __forceinline__ void add(const Four& f) {
      m.x = max(m.x, f.w.x & 0x7fffffffu);
      m.y = max(m.y, f.w.y & 0x7fffffffu);
      m.z = max(m.z, f.w.z & 0x7fffffffu);
      m.w = max(m.w, f.w.w & 0x7fffffffu);
    }
    __device__ __forceinline__ uint4 each() const { return m; }
    __device__ __forceinline__ uint32_t all() const { return max(max(m.x, m.y), max(m.z, m.w)); }
  };
  static __device__ __forceinline__ uint32_t widen(uint32_t bits) { return bits; }
};

template <int DT>
__global__ void __launch_bounds__(kThreads, DT == GLEAM_FP32 ? 2 : 4) k_fp8_quantize(const __grid_constant__ QuantizeArgs a) {
  __shared__ uint32_t s_col[kThreads / 32][kTile];
  __shared__ __align__(16) uint8_t s_t[kTileBytes];
  pdl_wait();
  // in this order: the product that follows reads the weights before it waits
  if (a.leads != 0) pdl_trigger();
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  uint64_t id = blockIdx.x;
  const uint64_t kb = id % a.kb;
  id /= a.kb;
  const uint64_t rb = id % a.rt, e = id / a.rt;
  const uint64_t col = kb * kTile + 4 * lane, row0 = rb * kTile + warp * kRowsPerWarp;
  const bool blocks = a.form == GLEAM_FP8_BLOCKS;

  // the row that stands at row0 + i, kept by lane i
  int32_t from = -1;
  if (lane < kRowsPerWarp && row0 + lane < a.rows) {
    from = (int32_t)(row0 + lane);
    if (a.src != nullptr) {
      const int32_t slot = a.src[row0 + lane];
      if (slot < 0) from = -1;
      else if (a.per_token != 0) from = (int32_t)((uint32_t)slot / a.per_token);
    }
    if (from >= (int64_t)a.x_rows) from = -1;
  }
  const uint32_t present = __ballot_sync(0xffffffffu, from >= 0);
  if (a.qt == nullptr && !blocks && present == 0 && a.fill == 0) return;
  // all loads before the first use: a warp has 4 or 8 KiB on its way
  Four<DT> v[kRowsPerWarp];
  {
    int32_t r[kRowsPerWarp];
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) r[i] = __shfl_sync(0xffffffffu, from, i);
    const uint8_t* x = a.x + e * a.stride + col * dtype_bytes(DT);
    if (a.vec != 0 && col + 4 <= a.cols) {
#pragma unroll
      for (int i = 0; i < kRowsPerWarp; ++i) {
        v[i] = Four<DT>::zero();
        if (r[i] >= 0) v[i].load(x + (uint64_t)r[i] * a.ld);
      }
    } else {
      const uint64_t n = col < a.cols ? a.cols - col : 0;
#pragma unroll
      for (int i = 0; i < kRowsPerWarp; ++i) {
        v[i] = Four<DT>::zero();
        if (r[i] >= 0) v[i].load_some(x + (uint64_t)r[i] * a.ld, n);
      }
    }
  }

  // the place of this thread's 4 bytes in row r of a tile
  auto place = [&](uint32_t r) { return r * kTile + (((lane >> 2) ^ (r & 7)) << 4) + ((lane & 3) << 2); };
  auto scaled = [&](int i, float f) {
    float u[4];
    v[i].get(u);
    return e4m3x4(u[0] * f, u[1] * f, u[2] * f, u[3] * f);
  };

  if (!blocks && a.q != nullptr) {
    uint8_t* tile = a.q + (rb * a.kb + kb) * kTileBytes;
    float mine = 0;  // the scale of row `lane`
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) {
      typename Four<DT>::Most m{};
      m.add(v[i]);
      const float2 sc = group_scale(Four<DT>::widen(__reduce_max_sync(0xffffffffu, m.all())));
      if (lane == i) mine = sc.x;
      if ((present >> i & 1) || (a.fill != 0 && row0 + i < a.rows))
        *reinterpret_cast<uint32_t*>(tile + place(warp * kRowsPerWarp + i)) = scaled(i, sc.y);
    }
    if (from >= 0 || (a.fill != 0 && lane < kRowsPerWarp && row0 + lane < a.rows)) a.s[kb * (a.rt * kTile) + row0 + lane] = mine;
  }
  if (!blocks && a.qt == nullptr) return;

  typename Four<DT>::Most most{};
#pragma unroll
  for (int i = 0; i < kRowsPerWarp; ++i) most.add(v[i]);
  uint4 c = most.each();
  *reinterpret_cast<uint4*>(&s_col[warp][4 * lane]) = c;
  if (!__syncthreads_or(present != 0) && !blocks) return;  // no row: this block of the sum is not read
#pragma unroll
  for (int k = 0; k < kThreads / 32; ++k) {
    const uint4 o = *reinterpret_cast<const uint4*>(&s_col[k][4 * lane]);
    c = make_uint4(max(c.x, o.x), max(c.y, o.y), max(c.z, o.z), max(c.w, o.w));
  }
  float f[4];
  if (blocks) {
    const float2 sc = group_scale(
        Four<DT>::widen(__reduce_max_sync(0xffffffffu, max(max(c.x, c.y), max(c.z, c.w)))));
    f[0] = f[1] = f[2] = f[3] = sc.y;
    if (threadIdx.x == 0) {
      if (a.s != nullptr) a.s[(e * a.rt + rb) * a.kb + kb] = sc.x;
      if (a.st != nullptr) a.st[(e * a.kb + kb) * a.rt + rb] = sc.x;
    }
    if (a.q != nullptr) {
      uint8_t* tile = a.q + ((e * a.rt + rb) * a.kb + kb) * kTileBytes;
#pragma unroll
      for (int i = 0; i < kRowsPerWarp; ++i)
        *reinterpret_cast<uint32_t*>(tile + place(warp * kRowsPerWarp + i)) = scaled(i, sc.y);
    }
  } else {
    const uint32_t m[4] = {c.x, c.y, c.z, c.w};
    float sc4[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 sc = group_scale(Four<DT>::widen(m[j]));
      f[j] = sc.y;
      sc4[j] = sc.x;
    }
    if (warp == 0)
      *reinterpret_cast<float4*>(a.st + rb * (a.kb * kTile) + col) =
          make_float4(sc4[0], sc4[1], sc4[2], sc4[3]);
  }
  if (a.qt == nullptr) return;

  // The transpose: this thread's 16 rows are one 16-byte piece of each of its
  // columns.  The pieces meet in shared memory under a swizzle of their own (by
  // the lane, so that 8 lanes' pieces fall on all banks) and leave in order.
  uint32_t w[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float u[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[4 * i + k].get(u[k]);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j][i] = e4m3x4(u[0][j] * f[j], u[1][j] * f[j], u[2][j] * f[j], u[3][j] * f[j]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *reinterpret_cast<uint4*>(s_t + (4 * lane + j) * kTile + ((warp ^ (lane & 7)) << 4)) =
        make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
  __syncthreads();
  uint8_t* tile = a.qt + ((e * a.kb + kb) * a.rt + rb) * kTileBytes;
#pragma unroll
  for (int i = 0; i < (int)(kTileBytes / 16 / kThreads); ++i) {
    const uint32_t at = i * kThreads + threadIdx.x, r = at >> 3, piece = (at & 7) ^ (r & 7);
    *reinterpret_cast<uint4*>(tile + at * 16) =
        *reinterpret_cast<const uint4*>(s_t + r * kTile + ((piece ^ ((r >> 2) & 7)) << 4));
  }
}

}  // namespace

cudaError_t launch_quantize(const QuantizeArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)(a.rt * a.kb * a.count));
  void (*k)(QuantizeArgs) = a.dtype == GLEAM_BF16   ? k_fp8_quantize<GLEAM_BF16>
                            : a.dtype == GLEAM_FP16 ? k_fp8_quantize<GLEAM_FP16>
                                                    : k_fp8_quantize<GLEAM_FP32>;
  return launch_chained(k, grid, dim3(kThreads), 0, s, 1, a);
}

}  // namespace gleam
