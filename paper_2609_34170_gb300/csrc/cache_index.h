// Index arithmetic of the 8-bit context cache's kernels that compiles for the
// host as well, where tests look it over.
#pragma once

#ifdef __CUDACC__
#define RAVEL_HD __host__ __device__ __forceinline__
#else
#define RAVEL_HD inline
#endif

namespace ravel {

// A ring of `slots` places that loads fill in turn, one barrier per place: load k (from 0)
// goes to place k % slots and completes the phase of this parity there.
RAVEL_HD unsigned load_parity(int k, int slots) { return (unsigned)(k / slots) & 1u; }

// The loads that may still be on their way when the wait for load `at` has run out: those
// before it have been waited for, and each of them, once read, let load + slots be issued, of
// `loads` in all.  Nothing is issued from then on.
struct LoadsLeft {
  int first, end;
};
RAVEL_HD LoadsLeft loads_left(int at, int loads, int slots) {
  return LoadsLeft{at, at + slots < loads ? at + slots : loads};
}

}  // namespace ravel
