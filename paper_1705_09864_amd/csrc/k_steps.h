// Which steps of K a wave of w4_rows_kernel loads.  Plain arithmetic, on the host too: the tests walk it.
#pragma once

namespace bmx {

// A wave has the steps wave, wave + waves, ... below `full` (wave < full).  It requests its step number n (0, 1, ...) so many steps before its use;
// numbers that it no longer has are its reads of the last step again, so that nothing behind the weights is read.
__host__ __device__ static inline int k_step(int wave, int waves, int n, int full) {
  const int step = wave + n * waves;
  return step < full ? step : full - 1;
}

}  // namespace bmx
