// Products of 8-bit matrices with a scale for each block of 128 along the
// contraction: y[i, j] = sum over b of xs[i, b] ws[j, b] (sum over k in b of
// xq[i, k] wq[j, k]).
//
// The inner sums run on the tensor cores (tcgen05.mma, kind f8f6f4, exact to 32
// bits) and cannot leave them unscaled: each block's partial tile goes from tensor
// memory through registers, where it is scaled and added in 32 bits.  Two kernels
// differ in which operand's rows are the 128 lanes of that tile:
//
//   k_fp8_wide    many rows of x: x's rows are the lanes and 128 or 256 rows of w
//                 the columns.  A lane's factor for a block is then one number,
//                 x's scale times the weight block's.  8192 x 14336 x 4096: 361 us,
//                 2,660 TFLOP/s (the library's product with one scale: 3,480), bound by
//                 the trip of a part of tensor memory to the adding warps and back.
//   k_fp8_narrow  few rows of x (up to 64): w's rows are the lanes and 16 to 64 rows
//                 of x the columns, so that nothing is computed for rows that are
//                 not there.  It waits for the weights alone; the blocks along the
//                 contraction are shared out among a cluster until every SM reads.
//                 37 x 14336 x 4096 with its quantisation: 20.6 us, 2.9 TB/s of weights.
//
// Both: one block per SM, persistent.  Warps 0 and 2 copy (16 KiB tiles of w, 128 bytes a
// row of x, each one bulk copy, or for a pair's tile a tensor copy, in the order that the tensor
// cores read), warp 1, in the wide kernel with warp 3, issues the products into two alternating parts of tensor memory,
// warps 4 to 11 scale, add and store.
#include <cuda.h>

#include <algorithm>

#include "operators.cuh"

namespace gleam {
namespace {

constexpr int kThreads = 384;
constexpr int kAdders = 8;  // warps that scale and add
constexpr uint32_t kMaxStages = 12;

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void mbar_init_n(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

// Barriers and state that both kernels keep in shared memory.
struct Control {
  unsigned long long full[kMaxStages], empty[kMaxStages];    // stages of values
  unsigned long long peer[kMaxStages];                       // the second block's copies (pairs)
  unsigned long long tfull[2], tempty[2];                    // parts of tensor memory
  unsigned long long drain[2];       // an issuing thread's products, once a wait has run out
  uint64_t filled[2];                // stages that each copying thread has filled
  unsigned long long pfull, pfree;  // partial sums: all here; read
  uint32_t tmem;
  uint32_t dead;                    // a wait ran out (in the end: of any block of the cluster)
  uint32_t total;                   // tiles
  uint32_t first[kMaxExperts];      // an expert's first tile (over rows)
};

// Whether a phase is complete.  kPeers: it may have arrivals from other blocks of the cluster.
template <bool kPeers>
__device__ __forceinline__ bool try_phase(uint32_t bar, uint32_t parity) {
  if constexpr (!kPeers) return mbar_try_wait(bar, parity);
  uint32_t done;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
      " selp.u32 %0, 1, 0, p;\n}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
// Waits for a phase, at most a.wait_ns; false once any wait of the block ran out.  The
// clock is read only once a while: it answers late.
template <bool kPeers = false>
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, Control& sh, const ProductArgs& a) {
  if (try_phase<kPeers>(bar, parity)) return true;
  unsigned long long t0 = 0;
  for (uint32_t i = 1;; ++i) {
    if (try_phase<kPeers>(bar, parity)) return true;
    if ((i & 63) != 0) continue;
    if (*reinterpret_cast<volatile uint32_t*>(&sh.dead)) return false;
    const unsigned long long now = globaltimer_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > a.wait_ns) {
      *reinterpret_cast<volatile uint32_t*>(&sh.dead) = 1;
      *a.status = GLEAM_ERR_TIMEOUT;
      return false;
    }
  }
}

// Shared memory descriptor of rows of 128 bytes, swizzled over 128 bytes, contraction along
// the row: 8 rows are 1024 bytes apart from the next 8.
__device__ __forceinline__ uint64_t tile_descriptor(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) |
         (2ull << 61);
}

// kPair: the two blocks of a cluster work on one tile, issued by the first.
template <bool kPair>
__device__ __forceinline__ void mma_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  if constexpr (kPair)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}
// An arrival at the barrier (of both blocks) once this thread's products so far are done.
template <bool kPair>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  if constexpr (kPair)
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            bar),
        "h"((uint16_t)3)
        : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
                 : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// N columns of this warp's 32 lanes; tmem_wait makes them usable.
#define GLEAM_R8(o) "=f"(r[o]), "=f"(r[o + 1]), "=f"(r[o + 2]), "=f"(r[o + 3]), "=f"(r[o + 4]), "=f"(r[o + 5]), "=f"(r[o + 6]), "=f"(r[o + 7])
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&r)[N]) {
  static_assert(N == 8 || N == 16 || N == 32, "columns of one load");
  if constexpr (N == 8)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];" : GLEAM_R8(0) : "r"(addr));
  else if constexpr (N == 16)
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : GLEAM_R8(0), GLEAM_R8(8)
        : "r"(addr));
  else
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : GLEAM_R8(0), GLEAM_R8(8), GLEAM_R8(16), GLEAM_R8(24)
        : "r"(addr));
}
#undef GLEAM_R8
// The operands tie the values to the wait: nothing reads them before it.
#define GLEAM_R8(o) "+f"(r[o]), "+f"(r[o + 1]), "+f"(r[o + 2]), "+f"(r[o + 3]), "+f"(r[o + 4]), "+f"(r[o + 5]), "+f"(r[o + 6]), "+f"(r[o + 7])
template <int N>
__device__ __forceinline__ void tmem_wait(float (&r)[N]) {
  if constexpr (N == 8) asm volatile("tcgen05.wait::ld.sync.aligned;" : GLEAM_R8(0)::"memory");
  else if constexpr (N == 16) asm volatile("tcgen05.wait::ld.sync.aligned;" : GLEAM_R8(0), GLEAM_R8(8)::"memory");
  else
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : GLEAM_R8(0), GLEAM_R8(8), GLEAM_R8(16), GLEAM_R8(24)::"memory");
}
#undef GLEAM_R8

// 16 columns of this warp's 32 lanes in pieces of 8 rows by 8 columns: lane (g, t) of
// (lane / 4, lane % 4) gets columns 8i + 2t and the next of row g + 8j in r[4i + 2(j % 2) + 8(j / 2)]
// and the next.
__device__ __forceinline__ void tmem_load_pieces(uint32_t addr, float (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
               : "r"(addr));
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
               : "r"(addr + (16u << 16)));
}

// Two 32-bit values in one register pair, and d = a * b + c on both.
__device__ __forceinline__ unsigned long long pair(float lo, float hi) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 unpair(unsigned long long v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ void fma2(unsigned long long& d, unsigned long long a, unsigned long long b) {
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(a), "l"(b));
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address of block `rank`'s copy of a shared memory location.
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 peer_load(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}
__device__ __forceinline__ void peer_store(uint32_t addr, uint32_t v) {
  asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ uint64_t peer_load64(uint32_t addr) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
// An arrival that makes what this thread wrote, and what it saw arrive, visible to the cluster,
// and one that only says that tensor memory has been read: those reads are done
// (tcgen05.wait::ld) and ordered by the tcgen05 fences before the arrival and after the wait for
// it, for which PTX asks no more than a relaxed arrival (the first waits for every access
// that the thread has on its way: 900 cycles in an adding warp).  Whoever waits for either does so
// with the cluster as its scope (wait_phase<true>).
__device__ __forceinline__ void peer_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void peer_signal(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// An arrival that only says how many bytes to expect.
__device__ __forceinline__ void peer_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
}

// The tiles of the operands of a pair's product, as tensors of three dimensions, and the scales of their
// rows, as tensors of two.  A copy of a tensor, unlike one of bytes, may land in one block and arrive
// at the other's barrier, so that the first block, which issues the products, waits for the second's
// copies themselves.  (Told of them by a thread of the second, it takes a release in that thread,
// 1,100 cycles a stage: a call of 8192 x 14336 x 4096 took 546 us with one such thread, 460 with two and
// takes 383.)  The adding warps know of their scales by the products, as in a block on its own: a
// barrier of the scales' own to wait for cost the product 6%.
template <bool kPair>
struct Maps {};
template <>
struct Maps<true> {
  CUtensorMap x, w, xs, ws;
};
__device__ __forceinline__ void copy_tile(uint32_t dst, const CUtensorMap* map, uint64_t tile, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], "
      "[%1, {%2, %2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(0), "r"((uint32_t)tile), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void copy_scales(uint32_t dst, const CUtensorMap* map, uint64_t row, uint32_t kb,
                                            uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], "
      "[%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"((uint32_t)row), "r"(kb), "r"(bar)
      : "memory");
}
// Rows of expert e (or, over sums, its part of the contraction); none if they lie outside
// the matrix.
__device__ __forceinline__ void expert_rows(const ProductArgs& a, uint32_t e, uint64_t rows, uint32_t* at,
                                            uint32_t* count) {
  const int32_t o = __ldg(a.offsets + e), c = __ldg(a.counts + e);
  *at = (uint32_t)o;
  *count = (uint32_t)c;
  if (c == 0) return;
  if (o < 0 || c < 0 || (o & (kTile - 1)) != 0 || (uint64_t)o + (uint64_t)c > rows) {
    *count = 0;
    *a.status = GLEAM_ERR_INVALID_ARG;
  }
}

// One output tile: rows x0 .. x0 + rows - 1 of x against rows w0 .. of matrix e of w.
struct Tile {
  uint64_t x0;        // first row of x (and of y)
  uint64_t w0;        // first row of w within its matrix
  uint64_t wtile;     // its row tile, counted over all matrices
  uint32_t rows;      // of x: 1 .. kX
  uint32_t kb0, kb1;  // blocks along the contraction
  uint64_t y;         // first element of y's matrix
};

// Tile `id` of tiles of kX rows of x by kW of w; x's rows run fastest, so that blocks
// that run together read the same weights.
template <int kX, int kW>
__device__ __forceinline__ Tile decode(const ProductArgs& a, const Control& sh, uint32_t id) {
  Tile t;
  t.y = 0;
  t.kb0 = 0;
  t.kb1 = (uint32_t)a.kb;
  uint32_t wt;
  if (a.experts != 0 && a.over == GLEAM_OVER_ROWS) {
    uint32_t lo = 0, hi = a.experts;  // first[lo] <= id, and less than first[hi]
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (sh.first[mid] <= id) lo = mid;
      else hi = mid;
    }
    uint32_t at, count;
    expert_rows(a, lo, a.m, &at, &count);
    const uint32_t xt = (count + kX - 1) / kX, in = id - sh.first[lo];
    wt = in / xt;
    const uint32_t r = in % xt * kX;
    t.x0 = at + r;
    t.rows = min((uint32_t)kX, count - r);
    t.wtile = (uint64_t)lo * a.wrt;
  } else {
    const uint32_t xt = (uint32_t)((a.m + kX - 1) / kX), wts = (uint32_t)((a.n + kW - 1) / kW);
    uint32_t in = id;
    if (a.experts != 0) {
      const uint32_t per = xt * wts, e = id / per;
      in = id % per;
      t.y = e * a.ystride;
      uint32_t at, count;
      expert_rows(a, e, a.kb * kTile, &at, &count);
      t.kb0 = at / kTile;
      t.kb1 = t.kb0 + (count + kTile - 1) / kTile;
      if (count == 0) t.kb0 = t.kb1 = 0;
    }
    wt = in / xt;
    t.x0 = (uint64_t)(in % xt) * kX;
    t.rows = (uint32_t)min((uint64_t)kX, a.m - t.x0);
    t.wtile = 0;
  }
  t.w0 = (uint64_t)wt * kW;
  t.wtile += t.w0 / kTile;
  return t;
}

// Barriers and tensor memory.  In a cluster, the other blocks' barriers are ready too.
struct Counts {
  uint32_t stages;    // of values
  uint32_t copiers;   // threads that fill a stage
  uint32_t adders;    // warps that read a part of tensor memory
  uint32_t partials;  // warps that add to partial sums
};
template <bool kPair>
__device__ __forceinline__ void begin(Control& sh, const Counts& n, uint32_t columns, bool cluster) {
  const uint32_t warp = threadIdx.x / 32;
  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < n.stages; ++i) {
      mbar_init_n(smem_addr(&sh.full[i]), n.copiers);
      mbar_init_n(smem_addr(&sh.empty[i]), 1);
      mbar_init_n(smem_addr(&sh.peer[i]), n.copiers);
    }
    for (uint32_t i = 0; i < 2; ++i) {
      mbar_init_n(smem_addr(&sh.tfull[i]), 1);
      mbar_init_n(smem_addr(&sh.tempty[i]), n.adders);
    }
    for (uint32_t i = 0; i < 2; ++i) {
      mbar_init_n(smem_addr(&sh.drain[i]), 1);
      sh.filled[i] = 0;
    }
    mbar_init_n(smem_addr(&sh.pfull), n.partials);
    mbar_init_n(smem_addr(&sh.pfree), n.partials);
    sh.dead = 0;
    mbar_fence_init();
  }
  if (warp == 1) {
    if constexpr (kPair) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tmem)),
                   "r"(columns)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tmem)),
                   "r"(columns)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    fence_before();
  }
  __syncthreads();
  if (cluster) cluster_sync();
  fence_after();
}

// How many tiles there are, once the kernel before this one is done.
template <int kX, int kW>
__device__ __forceinline__ void count_tiles(const ProductArgs& a, Control& sh) {
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (a.experts != 0 && a.over == GLEAM_OVER_ROWS) {
    if (warp == 2) {
      const uint32_t wts = (uint32_t)((a.n + kW - 1) / kW);
      unsigned long long sum = 0;
      for (uint32_t e0 = 0; e0 < a.experts; e0 += 32) {
        uint32_t at, count = 0;
        if (e0 + lane < a.experts) expert_rows(a, e0 + lane, a.m, &at, &count);
        const unsigned long long mine = (unsigned long long)((count + kX - 1) / kX) * wts;
        unsigned long long up = mine;
        for (int d = 1; d < 32; d <<= 1) {
          const unsigned long long o = __shfl_up_sync(0xffffffffu, up, d);
          if (lane >= (uint32_t)d) up += o;
        }
        if (e0 + lane < a.experts) sh.first[e0 + lane] = (uint32_t)(sum + up - mine);
        sum += __shfl_sync(0xffffffffu, up, 31);
      }
      // more than the rows have room for: experts that share rows, whose tiles may pass 32 bits
      const bool bad = sum > a.tiles;
      if (lane == 0) {
        if (bad) *a.status = GLEAM_ERR_INVALID_ARG;
        sh.total = bad ? 0 : (uint32_t)sum;
      }
    }
  } else if (threadIdx.x == 64) {
    sh.total = (uint32_t)a.tiles;
  }
  __syncthreads();
}

// In a cluster, no block leaves while another may still write to it or read its memory.  Once a
// wait has run out, settle waits for all copies and products on their way, whichever threads asked
// for them, before memory and tensor memory go to another block.
template <bool kPair, class Settle>
__device__ __forceinline__ void finish(const Control& sh, uint32_t tmem, uint32_t columns, bool cluster,
                                       Settle settle) {
  __syncwarp();
  fence_before();
  __syncthreads();
  const volatile uint32_t* dead = &sh.dead;
  if (cluster) {
    if (threadIdx.x < cluster_size() && *dead) peer_store(peer_addr(smem_addr(&sh.dead), threadIdx.x), 1);
    __syncwarp();
    cluster_sync();
  }
  fence_after();
  if (*dead) {
    settle();
    __syncwarp();
    __syncthreads();
    if (cluster) cluster_sync();
  }
  if (threadIdx.x / 32 == 1) {
    if constexpr (kPair)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
  }
  if (kPair) cluster_sync();
}

// Products that this thread, the i-th that issues any, has asked for are done (in both blocks of a
// pair, of which the first issues).
template <bool kPair>
__device__ __forceinline__ void await_products(Control& sh, uint32_t i, bool issues) {
  if (issues) mma_commit<kPair>(smem_addr(&sh.drain[i]));
  mbar_wait(smem_addr(&sh.drain[i]), 0, kOperatorWaitNs);
}
// Copies on their way to a ring of n stages have landed.
__device__ __forceinline__ void await_copies(const uint64_t* filled, uint32_t threads, unsigned long long* bars,
                                             uint32_t n) {
  settle_ring(filled, threads, n, [&](uint32_t i) { mbar_arrive(smem_addr(&bars[i])); },
              [&](uint32_t i, uint32_t parity) { mbar_wait(smem_addr(&bars[i]), parity, kOperatorWaitNs); });
}

// One block of the contraction: 128 lanes (of each block) from `a`, NT columns from `b`.
template <int NT, bool kPair>
__device__ __forceinline__ void issue_block(uint32_t d, uint32_t a, uint32_t b) {
  constexpr uint32_t kM = kPair ? 2 * kTile : kTile;
  constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NT >> 3) << 17) | ((kM >> 4) << 24);
  const uint64_t da = tile_descriptor(a), db = tile_descriptor(b);
#pragma unroll
  for (uint32_t k = 0; k < 4; ++k) mma_f8<kPair>(d, da + 2 * k, db + 2 * k, idesc, k != 0);
}

// ---- wide ------------------------------------------------------------------

// Rows of y in shared memory on their way out: 256 bytes a row, 16 apart so that eight lanes'
// rows fall on all banks.
constexpr uint32_t kOutBytes = 256, kOutPitch = kOutBytes + 16;

// kPair: a cluster of two blocks on 256 rows of x, each with 128 of them and half of w's.
template <int NT, bool kPair>
struct Wide {
  static constexpr int kRows = kPair ? 2 * kTile : kTile;  // of x, in a tile
  static constexpr int kOwnW = kPair ? NT / 2 : NT;        // rows of w that a block holds
  static constexpr uint32_t kStage = kTileBytes + kOwnW * kTile;
  // More do not feed the tensor cores faster (8192 x 8192 x 8192 took 1% longer with six)
  static constexpr uint32_t kStages = kStage > (32u << 10) ? 3 : 4;
  // Whether two threads issue products in turns.  With an even number of stages each stage
  // belongs to one of them, which then sees every phase of its barrier; with an odd number a
  // thread would ask for a phase while the one before, the other thread's, is still to come, and
  // take the phase before that for it, as a barrier tells phases apart by parity alone.
  static constexpr bool kTurns = kStages % 2 == 0;
  static constexpr int kCols = NT / 2;  // of an adding warp
  // Scales come with the stage of their block and are read after its products are done, when
  // the stage may be filled again: by then the adding warps may have two blocks' products
  // before them, as tensor memory has two parts, and be in the middle of a third, whose part is
  // free already.  Three places more than stages keep the scales apart.
  static constexpr uint32_t kPlaces = kStages + 3;
  struct Shared {
    alignas(16) uint8_t out[kAdders][32 * kOutPitch];
    alignas(128) float xscales[kPlaces][kTile];
    alignas(128) float wscales[kPlaces][NT];  // with a scale for each row of w
    Control c;
  };
  static constexpr uint32_t kBytes = 1024 + kStages * kStage + sizeof(Shared);
  static_assert(kBytes <= 232448, "shared memory of a block");
};

// Stores kCols columns of this lane's row of y.  The warp's rows go through shared memory and
// leave row by row, 256 bytes at once: a store of 32 rows' pieces, and a bulk copy for each row
// (70 cycles to ask for one), held the tensor cores up for 2 us of 16 of a tile of 32 blocks.
// Rows that start or end at no multiple of 16 bytes leave word by word.
// kPieces: acc[4 i + j] is columns 8i + 2t and the next of row g + 8j (tmem_load_pieces) and not
// columns 2i and 2i + 1 of the lane's row.
template <int DT, int kCols, bool kPieces>
__device__ __forceinline__ void store_rows(const ProductArgs& a, const unsigned long long (&acc)[kCols / 2],
                                           uint64_t at, uint64_t col, uint32_t rows, uint32_t lane, uint8_t* out) {
  constexpr uint32_t kSize = dtype_bytes(DT);
  constexpr int kPiece = Piece<DT>::kValues;
  constexpr int kOnce = kCols * kSize < kOutBytes ? kCols : kOutBytes / kSize;  // columns at a time
  uint8_t* mine = out + lane * kOutPitch;
#pragma unroll
  for (int c0 = 0; c0 < kCols; c0 += kOnce) {
    const uint64_t left = a.n > col + c0 ? a.n - col - c0 : 0;
    const uint32_t cols = (uint32_t)min(left, (uint64_t)kOnce);
    if (cols == 0) break;
    if constexpr (kPieces) {
      uint8_t* at = out + lane / 4 * kOutPitch + lane % 4 * 2 * kSize;
#pragma unroll
      for (int c = 0; c < kOnce; c += 8)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 p = unpair(acc[(c0 + c) / 2 + j]);
          uint8_t* q = at + 8 * j * kOutPitch + c * kSize;
          if constexpr (DT == GLEAM_FP32) *reinterpret_cast<float2*>(q) = p;
          else *reinterpret_cast<uint32_t*>(q) = pack2<DT>(p.x, p.y);
        }
    } else {
#pragma unroll
      for (int c = 0; c < kOnce; c += kPiece) {
        float v[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece; i += 2) {
          const float2 p = unpair(acc[(c0 + c + i) / 2]);
          v[i] = p.x;
          v[i + 1] = p.y;
        }
        Piece<DT>::store(mine + c * kSize, v);
      }
    }
    uint8_t* y = a.y + (at + col + c0) * kSize;  // of the warp's first row
    __syncwarp();
    const uint32_t most = min(rows, 32u);
    if (a.vec && cols * kSize % 16 == 0) {
      constexpr uint32_t kOfRow = kOnce * kSize / 16, kRowsOnce = 32 / kOfRow;
      const uint32_t piece = lane % kOfRow, r0 = lane / kOfRow;
      const uint8_t* from = out + r0 * kOutPitch + piece * 16;
      uint8_t* to = y + r0 * a.ld * kSize + piece * 16;
      if (piece * 16 < cols * kSize) {
#pragma unroll
        for (uint32_t r = 0; r < 32; r += kRowsOnce)
          if (r + r0 < most)
            *reinterpret_cast<uint4*>(to + r * a.ld * kSize) = *reinterpret_cast<const uint4*>(from + r * kOutPitch);
      }
    } else if constexpr (DT == GLEAM_FP32) {
#pragma unroll 4
      for (uint32_t r = 0; r < most; ++r)
        for (uint32_t c = lane; c < cols; c += 32)
          *reinterpret_cast<float*>(y + r * a.ld * kSize + 4 * c) =
              *reinterpret_cast<const float*>(out + r * kOutPitch + 4 * c);
    } else {
      // a row's first value alone where it stands in the second half of a word, and its last
      // where it stands in the first
      if (lane < most) {
        uint16_t* p = reinterpret_cast<uint16_t*>(y + lane * a.ld * kSize);
        const uint16_t* h = reinterpret_cast<const uint16_t*>(mine);
        const uint32_t off = reinterpret_cast<uintptr_t>(p) / 2 % 2;
        if (off) p[0] = h[0];
        if ((cols - off) % 2 != 0) p[cols - 1] = h[cols - 1];
      }
#pragma unroll
      for (uint32_t w0 = 0; w0 < kOnce / 2; w0 += 32) {
#pragma unroll 8
        for (uint32_t r = 0; r < 32; ++r) {
          uint16_t* p = reinterpret_cast<uint16_t*>(y + r * a.ld * kSize);
          const uint32_t off = reinterpret_cast<uintptr_t>(p) / 2 % 2, c = off + 2 * (w0 + lane);
          const uint16_t* h = reinterpret_cast<const uint16_t*>(out + r * kOutPitch) + c;
          if (r < most && c + 1 < cols) *reinterpret_cast<uint32_t*>(p + c) = (uint32_t)h[0] | (uint32_t)h[1] << 16;
        }
      }
    }
    __syncwarp();
  }
}

template <int NT, bool kBlocks, bool kPair>
__global__ void __launch_bounds__(kThreads, 1)
    k_fp8_wide(const __grid_constant__ ProductArgs a, const __grid_constant__ Maps<kPair> maps) {
  using W = Wide<NT, kPair>;
  constexpr uint32_t kStages = W::kStages, kStage = W::kStage;
  constexpr int kCols = W::kCols;
  constexpr int kLoad = 16;  // columns read at once: 32 would not fit the registers
  constexpr uint32_t kBlocksOfTile = kPair ? 2 : 1;
  extern __shared__ uint8_t raw[];
  uint8_t* base = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
  typename W::Shared& ws = *reinterpret_cast<typename W::Shared*>(base + kStages * kStage);
  Control& sh = ws.c;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = kPair ? cluster_rank() : 0;
  const uint32_t id0 = blockIdx.x / kBlocksOfTile, ids = gridDim.x / kBlocksOfTile;

  begin<kPair>(sh, Counts{kStages, 2, kBlocksOfTile * kAdders, 1}, 2 * NT, kPair);
  pdl_wait();
  count_tiles<W::kRows, NT>(a, sh);
  const uint32_t tmem = sh.tmem, total = sh.total;
  // this block's rows of a tile's x
  auto own_rows = [&](const Tile& t) {
    return t.rows > rank * kTile ? min(t.rows - rank * kTile, kTile) : 0u;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if ((warp == 0 || warp == 2) && lane == 0) {
      // copies: warp 0 those of x, warp 2 those of w
      Ring st;
      uint32_t place = 0;
      uint64_t filled = 0;
      const uint64_t most = blockIdx.x == 0 && warp == 0 && a.skip != kNoSkip ? a.skip : ~0ull;
      bool ok = true;
      for (uint32_t id = id0; ok && id < total; id += ids) {
        const Tile t = decode<W::kRows, NT>(a, sh, id);
        const uint32_t xbytes = ((own_rows(t) + 7) & ~7u) * kTile;
        const uint64_t wrow = t.w0 / kTile + rank;  // row tiles of w that exist, of this block's
        const uint32_t wtiles = wrow < a.wrt ? (uint32_t)min((uint64_t)(W::kOwnW / kTile), a.wrt - wrow) : 0;
        // rows of w whose scales are read; a pair's copy fills up with zeros past the last
        const uint32_t wscales = kPair ? NT * 4 : (uint32_t)min((uint64_t)NT, (a.wrt - t.w0 / kTile) * kTile) * 4;
        const uint64_t xtile = (t.x0 / kTile + rank) * a.kb, wtile = (t.wtile + rank) * a.kb;
        const uint32_t bytes = warp != 0     ? wtiles * kTileBytes + (kBlocks ? 0 : wscales)
                               : xbytes == 0 ? 0
                                             : (kPair ? kTileBytes : xbytes) + kTile * 4;
        for (uint32_t kb = t.kb0; kb < t.kb1; ++kb) {
          if (!(ok = filled < most && wait_phase<kPair>(smem_addr(&sh.empty[st.i]), st.phase ^ 1, sh, a))) break;
          ++filled;
          const uint32_t dst = smem_addr(base + st.i * kStage);
          const uint32_t xs = smem_addr(ws.xscales[place]), wsc = smem_addr(ws.wscales[place]);
          if constexpr (kPair) {
            const uint32_t bar = rank == 0 ? smem_addr(&sh.full[st.i]) : peer_addr(smem_addr(&sh.peer[st.i]), 0);
            if (rank == 0) mbar_expect_tx(bar, bytes);
            else peer_expect_tx(bar, bytes);
            if (warp == 0 && xbytes != 0) {
              copy_tile(dst, &maps.x, xtile + kb, bar);
              copy_scales(xs, &maps.xs, t.x0 + rank * kTile, kb, bar);
            } else if (warp == 2) {
              if (wtiles != 0) copy_tile(dst + kTileBytes, &maps.w, wtile + kb, bar);
              if (!kBlocks) copy_scales(wsc, &maps.ws, t.w0, kb, bar);
            }
          } else {
            const uint32_t bar = smem_addr(&sh.full[st.i]);
            mbar_expect_tx(bar, bytes);
            if (warp == 0) {
              copy_in(dst, a.xq + (xtile + kb) * kTileBytes, xbytes, bar);
              copy_in(xs, a.xs + kb * (a.xrt * kTile) + t.x0, kTile * 4, bar);
            } else {
              for (uint32_t i = 0; i < wtiles; ++i)
                copy_in(dst + (1 + i) * kTileBytes, a.wq + (wtile + i * a.kb + kb) * kTileBytes, kTileBytes, bar);
              if (!kBlocks) copy_in(wsc, a.ws + kb * (a.wrt * kTile) + t.w0, wscales, bar);
            }
          }
          st.next(kStages);
          if (++place == W::kPlaces) place = 0;
        }
      }
      // the other block's arrivals for the last stages land before this block's memory goes to another
      if (kPair)
        for (uint32_t i = 0; ok && i < kStages; ++i, st.next(kStages))
          ok = wait_phase<true>(smem_addr(&sh.empty[st.i]), st.phase ^ 1, sh, a);
      sh.filled[warp / 2] = filled;
    } else if (rank == 0 && (warp == 1 || (W::kTurns && warp == 3)) && lane == 0) {
      // products: in turns, one thread's waits pass while the other's products run (a thread
      // stands still while it issues)
      Ring st, tm;
      bool ok = true;
      for (uint32_t id = id0; ok && id < total; id += ids) {
        const Tile t = decode<W::kRows, NT>(a, sh, id);
        for (uint32_t kb = t.kb0; kb < t.kb1; ++kb) {
          if (!W::kTurns || tm.i == warp / 2) {
            if (!(ok = wait_phase(smem_addr(&sh.full[st.i]), st.phase, sh, a))) break;
            if (kPair && !(ok = wait_phase<true>(smem_addr(&sh.peer[st.i]), st.phase, sh, a))) break;
            if (!(ok = wait_phase<kPair>(smem_addr(&sh.tempty[tm.i]), tm.phase ^ 1, sh, a))) break;
            fence_after();
            const uint32_t at = smem_addr(base + st.i * kStage);
            issue_block<NT, kPair>(tmem + tm.i * NT, at, at + kTileBytes);
            mma_commit<kPair>(smem_addr(&sh.empty[st.i]));
            mma_commit<kPair>(smem_addr(&sh.tfull[tm.i]));
          }
          st.next(kStages);
          tm.next(2);
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    const uint32_t half = (warp - 4) / 4, row = (warp % 4) * 32 + lane;
    const uint32_t taddr = tmem + ((warp % 4) * 32 << 16) + half * kCols;
    // part 0 of tensor memory is free once both blocks' adding warps say so to the first
    const uint32_t tempty = kPair ? peer_addr(smem_addr(&sh.tempty[0]), 0) : smem_addr(&sh.tempty[0]);
    Ring tm;
    uint32_t place = 0;
    bool ok = true;
    for (uint32_t id = id0; ok && id < total; id += ids) {
      const Tile t = decode<W::kRows, NT>(a, sh, id);
      unsigned long long acc[kCols / 2];
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) acc[i] = 0;
      // A weight block's scale is one number for the warp's columns: a lane holds one of 32
      // blocks'.  Columns past the matrix take the tile's first; their sums are not stored.
      const uint32_t wpart = half * kCols / kTile;
      const float* wsp = a.ws + (t.wtile + (t.w0 / kTile + wpart < a.wrt ? wpart : 0)) * a.kb;
      float sw32 = 0;
      for (uint32_t kb = t.kb0; kb < t.kb1; ++kb) {
        if (kBlocks && (kb - t.kb0) % 32 == 0) sw32 = __ldg(wsp + min(kb + lane, t.kb1 - 1));
        ok = __all_sync(0xffffffffu, wait_phase<kPair>(smem_addr(&sh.tfull[tm.i]), tm.phase, sh, a));
        if (!ok) break;
        fence_after();
        const uint32_t part = taddr + tm.i * NT;
        // the next columns are on their way while these are added; once the last are in
        // registers, the next products may come
        float v[2][kLoad];
        if constexpr (kBlocks) {
          const float f = ws.xscales[place][row] * __shfl_sync(0xffffffffu, sw32, (kb - t.kb0) % 32);
          const unsigned long long f2 = pair(f, f);
          tmem_load(part, v[0]);
#pragma unroll
          for (int c = 0; c < kCols; c += kLoad) {
            float(&u)[kLoad] = v[c / kLoad & 1];
            tmem_wait(u);
            if (c + kLoad < kCols) {
              tmem_load(part + c + kLoad, v[(c / kLoad + 1) & 1]);
            } else {
              fence_before();
              __syncwarp();
              if (lane == 0) {
                if (kPair) peer_signal(tempty + 8 * tm.i);
                else mbar_arrive(tempty + 8 * tm.i);
              }
            }
#pragma unroll
            for (int i = 0; i < kLoad; i += 2) fma2(acc[(c + i) / 2], pair(u[i], u[i + 1]), f2);
          }
        } else {
          // With a scale for each row of w too, a lane takes 4 rows of 2 columns in 8, so that it
          // reads 32 columns' scales and not 128 (whose reads took as long as the products).
          unsigned long long f2[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float f = ws.xscales[place][(warp % 4) * 32 + lane / 4 + 8 * j];
            f2[j] = pair(f, f);
          }
          const float* s = ws.wscales[place] + half * kCols + 2 * (lane % 4);
          tmem_load_pieces(part, v[0]);
#pragma unroll
          for (int c = 0; c < kCols; c += kLoad) {
            float(&u)[kLoad] = v[c / kLoad & 1];
            tmem_wait(u);
            if (c + kLoad < kCols) {
              tmem_load_pieces(part + c + kLoad, v[(c / kLoad + 1) & 1]);
            } else {
              fence_before();
              __syncwarp();
              if (lane == 0) {
                if (kPair) peer_signal(tempty + 8 * tm.i);
                else mbar_arrive(tempty + 8 * tm.i);
              }
            }
#pragma unroll
            for (int i = 0; i < kLoad / 8; ++i) {
              const unsigned long long g = *reinterpret_cast<const unsigned long long*>(s + c + 8 * i);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int r = 4 * i + 2 * (j % 2) + 8 * (j / 2);
                fma2(acc[c / 2 + 4 * i + j], pair(u[r], u[r + 1]), mul2(g, f2[j]));
              }
            }
          }
        }
        tm.next(2);
        if (++place == W::kPlaces) place = 0;
      }
      if (!ok) break;
      const uint32_t quarter = (warp % 4) * 32;
      const uint32_t rows = own_rows(t) > quarter ? own_rows(t) - quarter : 0;
      const uint64_t first = t.y + (t.x0 + rank * kTile + quarter) * a.ld, col = t.w0 + half * kCols;
      uint8_t* out = ws.out[warp - 4];
      if (a.dtype == GLEAM_BF16) store_rows<GLEAM_BF16, kCols, !kBlocks>(a, acc, first, col, rows, lane, out);
      else if (a.dtype == GLEAM_FP16) store_rows<GLEAM_FP16, kCols, !kBlocks>(a, acc, first, col, rows, lane, out);
      else store_rows<GLEAM_FP32, kCols, !kBlocks>(a, acc, first, col, rows, lane, out);
    }
  }
  finish<kPair>(sh, tmem, 2 * NT, kPair, [&] {
    if ((warp == 1 || (W::kTurns && warp == 3)) && lane == 0) await_products<kPair>(sh, warp / 2, rank == 0);
    if (threadIdx.x != 0) return;
    if (rank == 0) await_copies(sh.filled, 2, sh.full, kStages);
    if (kPair && rank == 0) {
      const uint64_t theirs[2] = {peer_load64(peer_addr(smem_addr(&sh.filled[0]), 1)),
                                  peer_load64(peer_addr(smem_addr(&sh.filled[1]), 1))};
      await_copies(theirs, 2, sh.peer, kStages);
    }
  });
}

// ---- narrow ----------------------------------------------------------------

// A part of tensor memory holds kGroup blocks of the contraction side by side: a round
// trip from the tensor cores through the adding warps and back costs the same for one
// as for all of them.  Each half of the adding warps takes half of the blocks, all
// columns, and keeps a sum of its own.
template <int NT>
struct Narrow {
  static constexpr uint32_t kGroup = 128 / NT;
  static constexpr uint32_t kStage = kTileBytes + NT * kTile;
  static constexpr uint32_t kPartial = 2 * NT * kTile * 4;  // bytes: both halves' sums
  static constexpr uint32_t kStages =
      ((216u << 10) - kPartial) / kStage > kMaxStages ? kMaxStages : ((216u << 10) - kPartial) / kStage;
  // scales of x, as in the wide kernel: at most two groups of blocks are not read
  static constexpr uint32_t kPlaces = kStages + 2 * kGroup;
  struct Shared {
    alignas(16) float partial[2 * NT * kTile];  // [half][column][row]
    alignas(16) float scales[kPlaces][NT];
    Control c;
  };
  static constexpr uint32_t kBytes = 1024 + kStages * kStage + sizeof(Shared);
  static_assert(kBytes <= 232448, "shared memory of a block");
};

// Four neighbouring values of a row of y.
template <int DT>
__device__ __forceinline__ void store_four(uint8_t* p, const float4& v, uint64_t left, bool vec) {
  constexpr uint64_t kSize = dtype_bytes(DT);
  if (vec && left >= 4) {
    if constexpr (DT == GLEAM_FP32) *reinterpret_cast<float4*>(p) = v;
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack2<DT>(v.x, v.y), pack2<DT>(v.z, v.w));
  } else {
    if (left >= 1) store_value<DT>(p, v.x);
    if (left >= 2) store_value<DT>(p + kSize, v.y);
    if (left >= 3) store_value<DT>(p + 2 * kSize, v.z);
    if (left >= 4) store_value<DT>(p + 3 * kSize, v.w);
  }
}

// Adds up and stores this block's columns of a tile, one to a warp at a time and four rows to
// a lane, from the partial sums of all blocks in the order of the contraction.
template <int DT, int NT>
__device__ __forceinline__ void store_sums(const ProductArgs& a, const Tile& t, const float* partial, uint32_t rank,
                                           uint32_t ranks) {
  constexpr uint64_t kSize = dtype_bytes(DT);
  const uint32_t lane = threadIdx.x % 32, mine = NT / ranks;
  const uint32_t end = min(t.rows, (rank + 1) * mine);
  const uint64_t col = t.w0 + 4 * lane, left = col < a.n ? a.n - col : 0;
  for (uint32_t c = rank * mine + threadIdx.x / 32 - 4; c < end; c += kAdders) {
    const uint32_t at = smem_addr(&partial[c * kTile + 4 * lane]);
    float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll 2
    for (uint32_t r = 0; r < ranks; ++r) {
      const uint32_t from = ranks == 1 ? at : peer_addr(at, r);
#pragma unroll
      for (uint32_t half = 0; half < 2; ++half) {
        const float4 v = peer_load(from + half * NT * kTile * 4);
        sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
      }
    }
    store_four<DT>(a.y + ((t.x0 + c) * a.ld + col) * kSize, sum, left, a.vec);
  }
}

template <int NT>
__global__ void __launch_bounds__(kThreads, 1) k_fp8_narrow(const __grid_constant__ ProductArgs a) {
  using N = Narrow<NT>;
  constexpr uint32_t kStages = N::kStages, kStage = N::kStage, kGroup = N::kGroup;
  constexpr int kLoad = NT < 32 ? NT : 32;
  extern __shared__ uint8_t raw[];
  uint8_t* base = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
  typename N::Shared& ns = *reinterpret_cast<typename N::Shared*>(base + kStages * kStage);
  Control& sh = ns.c;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = cluster_rank(), ranks = cluster_size();
  const uint32_t cluster = blockIdx.x / ranks, clusters = gridDim.x / ranks;

  begin<false>(sh, Counts{kStages, 2, kAdders, ranks * kAdders}, 256, ranks > 1);
  // this block's share of a tile's contraction
  auto share = [&](const Tile& t, uint32_t* k0, uint32_t* k1) {
    const uint32_t n = t.kb1 - t.kb0;
    *k0 = t.kb0 + (uint32_t)((uint64_t)n * rank / ranks);
    *k1 = t.kb0 + (uint32_t)((uint64_t)n * (rank + 1) / ranks);
  };
  uint32_t ahead = 0;  // stages whose weights are asked for already
  if (a.w_ready && threadIdx.x == 0 && cluster < a.tiles) {
    // the kernel before this one writes x alone: the weights need not wait for it
    const Tile t = decode<NT, kTile>(a, sh, cluster);
    uint32_t k0, k1;
    share(t, &k0, &k1);
    for (; ahead < kStages && k0 + ahead < k1; ++ahead) {
      const uint32_t bar = smem_addr(&sh.full[ahead]);
      mbar_expect_tx(bar, kTileBytes);
      copy_in(smem_addr(base + ahead * kStage), a.wq + (t.wtile * a.kb + k0 + ahead) * kTileBytes, kTileBytes, bar);
    }
  }
  pdl_wait();
  count_tiles<NT, kTile>(a, sh);
  const uint32_t tmem = sh.tmem, total = sh.total;

  if ((warp == 0 || warp == 2) && lane == 0) {
    // copies: warp 0 those of w, warp 2 those of x and its scales
    Ring st;
    uint32_t place = 0;
    uint64_t filled = ahead;
    const uint64_t most = blockIdx.x == 0 && warp == 0 && a.skip != kNoSkip ? a.skip : ~0ull;
    bool ok = true;
    for (uint32_t id = cluster; ok && id < total; id += clusters) {
      const Tile t = decode<NT, kTile>(a, sh, id);
      uint32_t k0, k1;
      share(t, &k0, &k1);
      const uint32_t xbytes = ((t.rows + 7) & ~7u) * kTile;
      const uint32_t ns4 = (uint32_t)min((uint64_t)NT, a.xrt * kTile - t.x0) * 4;
      const uint8_t* xq = a.xq + t.x0 / kTile * a.kb * kTileBytes + t.x0 % kTile * kTile;
      const uint8_t* wq = a.wq + t.wtile * a.kb * kTileBytes;
      for (uint32_t kb = k0; kb < k1; ++kb) {
        if (!(ok = filled < most && wait_phase(smem_addr(&sh.empty[st.i]), st.phase ^ 1, sh, a))) break;
        if (ahead == 0) ++filled;
        const uint32_t bar = smem_addr(&sh.full[st.i]);
        const uint32_t dst = smem_addr(base + st.i * kStage);
        if (warp == 2) {
          mbar_expect_tx(bar, xbytes + ns4);
          copy_in(dst + kTileBytes, xq + (uint64_t)kb * kTileBytes, xbytes, bar);
          copy_in(smem_addr(ns.scales[place]), a.xs + kb * (a.xrt * kTile) + t.x0, ns4, bar);
        } else if (ahead != 0) {
          --ahead;
        } else {
          mbar_expect_tx(bar, kTileBytes);
          copy_in(dst, wq + (uint64_t)kb * kTileBytes, kTileBytes, bar);
        }
        st.next(kStages);
        if (++place == N::kPlaces) place = 0;
      }
    }
    sh.filled[warp / 2] = filled;
  } else if (warp == 1 && lane == 0) {
    // products
    Ring st, tm;
    bool ok = true;
    for (uint32_t id = cluster; ok && id < total; id += clusters) {
      const Tile t = decode<NT, kTile>(a, sh, id);
      uint32_t k0, k1;
      share(t, &k0, &k1);
      for (uint32_t kb = k0; ok && kb < k1; kb += kGroup) {
        if (!(ok = wait_phase(smem_addr(&sh.tempty[tm.i]), tm.phase ^ 1, sh, a))) break;
        for (uint32_t j = 0; j < kGroup && kb + j < k1; ++j) {
          if (!(ok = wait_phase(smem_addr(&sh.full[st.i]), st.phase, sh, a))) break;
          fence_after();
          const uint32_t at = smem_addr(base + st.i * kStage);
          issue_block<NT, false>(tmem + tm.i * 128 + j * NT, at, at + kTileBytes);
          mma_commit<false>(smem_addr(&sh.empty[st.i]));
          st.next(kStages);
        }
        if (!ok) break;
        mma_commit<false>(smem_addr(&sh.tfull[tm.i]));
        tm.next(2);
      }
    }
  } else if (warp >= 4) {
    const uint32_t half = (warp - 4) / 4, row = (warp % 4) * 32 + lane;
    const uint32_t taddr = tmem + ((warp % 4) * 32 << 16);
    Ring tm;
    uint32_t place = 0;
    uint32_t parity = 0;               // of the partial sums' barriers
    bool ok = true;
    for (uint32_t id = cluster; ok && id < total; id += clusters) {
      const Tile t = decode<NT, kTile>(a, sh, id);
      uint32_t k0, k1;
      share(t, &k0, &k1);
      unsigned long long acc[NT / 2];
#pragma unroll
      for (int i = 0; i < NT / 2; ++i) acc[i] = 0;
      const float* wsp = a.ws + t.wtile * a.kb;
      float sw32 = 0;  // a weight block's scale, of 32 blocks: a lane each
      for (uint32_t kb = k0; ok && kb < k1; kb += kGroup) {
        if ((kb - k0) % 32 == 0) sw32 = __ldg(wsp + min(kb + lane, k1 - 1));
        const uint32_t n = min(kGroup, k1 - kb);
        const uint32_t j0 = half * (kGroup / 2);  // this half's first block of the group
        ok = __all_sync(0xffffffffu, wait_phase(smem_addr(&sh.tfull[tm.i]), tm.phase, sh, a));
        if (!ok) break;
        fence_after();
#pragma unroll
        for (uint32_t j = 0; j < kGroup / 2; ++j) {
          if (j0 + j >= n) break;
          const uint32_t at = place + j0 + j;
          const float* sx = ns.scales[at < N::kPlaces ? at : at - N::kPlaces];
          const float f = __shfl_sync(0xffffffffu, sw32, (kb - k0 + j0 + j) % 32);
          const unsigned long long f2 = pair(f, f);
#pragma unroll
          for (int c = 0; c < NT; c += kLoad) {
            float v[kLoad];
            tmem_load(taddr + tm.i * 128 + (j0 + j) * NT + c, v);
            tmem_wait(v);
#pragma unroll
            for (int i = 0; i < kLoad; i += 4) {
              const ulonglong2 g = *reinterpret_cast<const ulonglong2*>(sx + c + i);
              fma2(acc[(c + i) / 2], pair(v[i], v[i + 1]), mul2(g.x, f2));
              fma2(acc[(c + i) / 2 + 1], pair(v[i + 2], v[i + 3]), mul2(g.y, f2));
            }
          }
        }
        place += n;
        if (place >= N::kPlaces) place -= N::kPlaces;
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&sh.tempty[tm.i]));
        tm.next(2);
      }
      if (!ok) break;

      // Both halves of every block leave their sums in their own shared memory, and each block
      // adds up and stores its share of the columns.
      ok = __all_sync(0xffffffffu, ranks > 1 ? wait_phase<true>(smem_addr(&sh.pfree), parity ^ 1, sh, a)
                                             : wait_phase(smem_addr(&sh.pfree), parity ^ 1, sh, a));
      if (!ok) break;
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        if (c >= (int)t.rows) break;
        const float2 v = unpair(acc[c / 2]);
        ns.partial[(half * NT + c) * kTile + row] = c & 1 ? v.y : v.x;
      }
      __syncwarp();
      if (ranks == 1) {
        if (lane == 0) mbar_arrive(smem_addr(&sh.pfull));
        ok = __all_sync(0xffffffffu, wait_phase(smem_addr(&sh.pfull), parity, sh, a));
      } else {
        if (lane < ranks) peer_arrive(peer_addr(smem_addr(&sh.pfull), lane));
        ok = __all_sync(0xffffffffu, wait_phase<true>(smem_addr(&sh.pfull), parity, sh, a));
      }
      if (!ok) break;
      if (a.dtype == GLEAM_BF16) store_sums<GLEAM_BF16, NT>(a, t, ns.partial, rank, ranks);
      else if (a.dtype == GLEAM_FP16) store_sums<GLEAM_FP16, NT>(a, t, ns.partial, rank, ranks);
      else store_sums<GLEAM_FP32, NT>(a, t, ns.partial, rank, ranks);
      __syncwarp();
      if (ranks == 1) {
        if (lane == 0) mbar_arrive(smem_addr(&sh.pfree));
      } else if (lane < ranks) {
        peer_arrive(peer_addr(smem_addr(&sh.pfree), lane));
      }
      parity ^= 1;
    }
  }
  finish<false>(sh, tmem, 256, ranks > 1, [&] {
    if (warp == 1 && lane == 0) await_products<false>(sh, 0, true);
    if (threadIdx.x == 0) await_copies(sh.filled, 2, sh.full, kStages);
  });
}

// ---- launches --------------------------------------------------------------

struct Gpu {
  cudaError_t err = cudaSuccess;
  int sms = 1;
  Gpu() {
    int dev = 0;
    if ((err = cudaGetDevice(&dev)) == cudaSuccess)
      err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  }
};

template <class... P>
cudaError_t start(void (*kernel)(ProductArgs, P...), uint32_t bytes, const ProductArgs& a, uint64_t blocks,
                  uint32_t cluster, cudaStream_t s, P... more) {
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) return e;
  return launch_chained(kernel, dim3((unsigned)blocks), dim3(kThreads), bytes, s, cluster, a, more...);
}

typedef decltype(&cuTensorMapEncodeTiled) EncodeFn;

// The driver's function that describes a tensor to the copies; it needs no GPU work.
EncodeFn encode_fn() {
  static const EncodeFn fn = []() -> EncodeFn {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      return nullptr;
    }
    return reinterpret_cast<EncodeFn>(f);
  }();
  return fn;
}

// A tensor of 2 or 3 dimensions without gaps, of which a copy takes a box.
cudaError_t map_tensor(CUtensorMap* map, const void* d, CUtensorMapDataType type, uint64_t size, uint32_t rank,
                       const cuuint64_t (&dims)[3], const cuuint32_t (&box)[3]) {
  const EncodeFn fn = encode_fn();
  if (fn == nullptr) return cudaErrorNotSupported;
  const cuuint64_t strides[2] = {dims[0] * size, dims[0] * dims[1] * size};
  const cuuint32_t step[3] = {1, 1, 1};
  const CUresult r = fn(map, type, rank, const_cast<void*>(d), dims, strides, box, step,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}
// Tiles, one after the other (coordinates are of 31 bits).
cudaError_t map_tiles(CUtensorMap* map, const uint8_t* q, uint64_t tiles) {
  if (tiles > 0x7fffffffull) return cudaErrorInvalidValue;
  return map_tensor(map, q, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, 3, {kTile, kTile, tiles}, {kTile, kTile, 1});
}
// Scales of each row and block of the contraction, those of `rows` rows at a time.
cudaError_t map_scales(CUtensorMap* map, const float* s, uint64_t row_tiles, uint64_t kb, uint32_t rows) {
  return map_tensor(map, s, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, 2, {row_tiles * kTile, kb, 1}, {rows, 1, 1});
}

// Tiles of kX rows of x by kW of w (over rows: at most, as the offsets are on the device).
uint64_t tiles_of(const ProductArgs& a, uint64_t kx, uint64_t kw) {
  const uint64_t xt = (a.m + kx - 1) / kx, wt = (a.n + kw - 1) / kw;
  if (a.experts == 0) return xt * wt;
  if (a.over == GLEAM_OVER_SUMS) return xt * wt * a.experts;
  return (xt + a.experts) * wt;
}

template <int NT, bool kPair>
cudaError_t wide(ProductArgs a, int sms, cudaStream_t s) {
  using W = Wide<NT, kPair>;
  constexpr uint32_t per = kPair ? 2 : 1;
  a.tiles = tiles_of(a, W::kRows, NT);
  if (a.tiles >= 0x7fffffffull) return cudaErrorInvalidValue;
  const uint64_t blocks = per * std::min<uint64_t>(a.tiles, (uint64_t)sms / per);
  Maps<kPair> maps{};
  if constexpr (kPair) {
    const uint64_t weights = a.experts != 0 && a.over == GLEAM_OVER_ROWS ? a.experts : 1;
    cudaError_t e = cudaSuccess;
    // without a contraction nothing is copied
    if (a.kb != 0 &&
        ((e = map_tiles(&maps.x, a.xq, a.xrt * a.kb)) != cudaSuccess ||
         (e = map_tiles(&maps.w, a.wq, weights * a.wrt * a.kb)) != cudaSuccess ||
         (e = map_scales(&maps.xs, a.xs, a.xrt, a.kb, kTile)) != cudaSuccess ||
         (a.w_form == GLEAM_FP8_GROUPS && (e = map_scales(&maps.ws, a.ws, a.wrt, a.kb, NT)) != cudaSuccess)))
      return e;
  }
  return start(a.w_form == GLEAM_FP8_BLOCKS ? k_fp8_wide<NT, true, kPair> : k_fp8_wide<NT, false, kPair>, W::kBytes,
               a, blocks, per, s, maps);
}

// The contraction is shared out among 1, 2, 4 or 8 blocks, as many as keep the GPU's SMs
// busy with the tiles there are and have a group of blocks each.
template <int NT>
cudaError_t narrow(ProductArgs a, int sms, cudaStream_t s) {
  a.tiles = tiles_of(a, NT, kTile);
  if (a.tiles >= 0x7fffffffull) return cudaErrorInvalidValue;
  uint64_t tiles = a.tiles;
  uint32_t ranks = 1;
  while (ranks < 8 && tiles * ranks * 2 <= (uint64_t)sms && a.kb >= ranks * 2) ranks *= 2;
  const uint64_t clusters = std::min<uint64_t>(tiles, (uint64_t)sms / ranks);
  return start(k_fp8_narrow<NT>, Narrow<NT>::kBytes, a, clusters * ranks, ranks, s);
}

}  // namespace

// Rows of x (per matrix) decide: up to 64 leave most lanes of a wide tile idle.
cudaError_t launch_product(const ProductArgs& a, uint64_t rows, cudaStream_t s) {
  const Gpu gpu;
  if (gpu.err != cudaSuccess) return gpu.err;
  if (a.w_form == GLEAM_FP8_BLOCKS && rows <= 64) {
    if (rows <= 16) return narrow<16>(a, gpu.sms, s);
    if (rows <= 32) return narrow<32>(a, gpu.sms, s);
    return narrow<64>(a, gpu.sms, s);
  }
  // ... and up to 128 leave most SMs idle, unless w has many rows: two tiles of 64 share out the
  // contraction (128 x 4096 x 4096: 19 us wide)
  if (a.w_form == GLEAM_FP8_BLOCKS && rows <= 128 && 2 * tiles_of(a, 64, kTile) <= (uint64_t)gpu.sms)
    return narrow<64>(a, gpu.sms, s);
  // the tile that takes the least time, counted in waves of tiles over the SMs: at 8192 x 4096 x 4096
  // a wave of pairs' tiles of 256 x 256 takes 15.5 us, one of 128 x 256 16.9 and one of 128 x 128 12.9.
  // The ratio is that of 32 blocks to a tile; starts and stores weigh more with fewer.
  const uint64_t sms = (uint64_t)gpu.sms;
  auto waves = [](uint64_t tiles, uint64_t at_once) { return (tiles + at_once - 1) / at_once; };
  const uint64_t pair = 20 * waves(tiles_of(a, 256, 256), sms / 2), one = 22 * waves(tiles_of(a, 128, 256), sms),
                 half = 17 * waves(tiles_of(a, 128, 128), sms);
  if (pair <= one && pair <= half) return wide<256, true>(a, gpu.sms, s);
  return one <= half ? wide<256, false>(a, gpu.sms, s) : wide<128, false>(a, gpu.sms, s);
}

}  // namespace gleam
