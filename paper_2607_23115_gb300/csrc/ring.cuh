// Rings of barriers that copies fill in turn: positions, and what a block waits for that gave
// up in the middle.  No CUDA needed: the CPU tests run this code against a model of barriers.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define GLEAM_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define GLEAM_HOST_DEVICE inline
#endif

namespace gleam {

// A position in a ring of n barriers.
struct Ring {
  uint32_t i = 0, phase = 0;
  GLEAM_HOST_DEVICE void next(uint32_t n) {
    if (++i == n) {
      i = 0;
      phase ^= 1;
    }
  }
};

// How often stage i of a ring of n was filled by a thread that filled `fills` in turn.
GLEAM_HOST_DEVICE uint64_t fills_of(uint64_t fills, uint32_t n, uint32_t i) {
  return fills / n + (i < fills % n ? 1 : 0);
}

// Waits for the copies that are still on their way to the n stages of a ring.  fills[c]: of each
// of the threads that fill the stages together, each with one arrival and its own bytes.  Where
// one of them gave up before the others filled a stage (it cannot be further behind, as a
// stage is free again only once all have filled it), its arrival is made up for, so that the
// stage's phase ends with the others' bytes.  arrive(i), wait(i, parity).
template <class Arrive, class Wait>
GLEAM_HOST_DEVICE void settle_ring(const uint64_t* fills, uint32_t threads, uint32_t n, Arrive arrive, Wait wait) {
  for (uint32_t i = 0; i < n; ++i) {
    uint64_t most = 0;
    for (uint32_t c = 0; c < threads; ++c) {
      const uint64_t f = fills_of(fills[c], n, i);
      if (f > most) most = f;
    }
    if (most == 0) continue;
    for (uint32_t c = 0; c < threads; ++c)
      if (fills_of(fills[c], n, i) < most) arrive(i);
    wait(i, (uint32_t)(most - 1) & 1);
  }
}

}  // namespace gleam
