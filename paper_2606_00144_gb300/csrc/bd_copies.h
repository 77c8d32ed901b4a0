// Copies that complete on one barrier, a phase each, counted where they are issued: a CTA that gives up half-way waits for the
// last of them, whatever it had in mind for afterwards.  (Plain C++ as well, for the test that walks a producer's exits.)
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define BD_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define BD_HOST_DEVICE inline
#endif

namespace bd {

// The copies follow one another (each is issued after the one before has landed), so the last one's phase is all there is to wait for.
struct CopyCount {
  int issued;
  BD_HOST_DEVICE void add() { ++issued; }
  BD_HOST_DEVICE bool any() const { return issued > 0; }
  BD_HOST_DEVICE uint32_t last_parity() const { return (uint32_t)(issued - 1) & 1u; }
};

}  // namespace bd
