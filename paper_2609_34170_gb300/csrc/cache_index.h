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

// Of the 64 rows from `first` on, those that see token j: lo .. hi - 1 of them (lo may be -1, for
// "all from before").  Row r is query r / G at position p0 + r / G of a robot with `len` tokens
// and rows below end_row.  A window reaches as far as the tokens do, so that its end may pass 32
// bits.
struct RowsThatSee {
  int lo, hi;
};
RAVEL_HD RowsThatSee rows_that_see(int j, int len, int p0, int G, int end_row, int causal, int window, int sinks, int first) {
  long long lo = 0, hi = j < len ? end_row : 0;
  if (causal) {
    lo = ((long long)j - p0) * G;
    if (window > 0 && j >= sinks) {
      const long long behind = ((long long)j + window - p0) * G;
      hi = behind < hi ? behind : hi;
    }
  }
  lo -= first;
  hi -= first;
  return RowsThatSee{(int)(lo < -1 ? -1 : (lo > 64 ? 64 : lo)), (int)(hi < 0 ? 0 : (hi > 64 ? 64 : hi))};
}

// Unit t of what a tile of rows sees: the first sink_units, then the window's from unit `from` on.
RAVEL_HD int unit_place(int t, int sink_units, int from) { return t < sink_units ? t : t - sink_units + from; }

// The longest run of neighbours among units t0 .. t0 + n - 1: where it begins and its units.
struct UnitRun {
  int at, units;
};
RAVEL_HD UnitRun longest_run(int t0, int n, int sink_units, int from) {
  if (sink_units == from) return UnitRun{t0, n};   // (no gap between the sinks and the window)
  const int sinks = sink_units <= t0 ? 0 : (sink_units - t0 < n ? sink_units - t0 : n);
  return sinks > n - sinks ? UnitRun{t0, sinks} : UnitRun{unit_place(t0 + sinks, sink_units, from), n - sinks};
}

}  // namespace ravel
