// Host side of a kernel launch, shared by the files that hold kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "calibatt.h"

namespace calibatt_host {

struct FwdPtrs {
  const uint16_t *q, *k, *v;
  uint16_t *out;
  const int32_t *row_ptr, *col_idx, *work, *fan_ptr, *fan_dst;
  int32_t *counter;
  const int32_t *iv_ptr;  // interval form of the kept-block lists, or NULL
  const uint32_t *iv;
  const int32_t *head_map;  // tensor head of each pattern head, or NULL
  float *lse;               // log-sum-exp output, or NULL
  int dtype;                // CALIBATT_BF16 or CALIBATT_F16
};

// Per-device launch facts of one kernel: how many workgroups the whole device holds at a time.
// Looked up on the first call per device.  Concurrent first calls all compute the same figure, so
// the slot is a plain atomic (0 = not known yet) and no lock is taken.
struct DevInfo {
  std::atomic<int> slots[64];
};

template <typename Kernel>
int prepare(Kernel kernel, int threads, int smem, DevInfo &info, int &slots) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return CALIBATT_ERR_LAUNCH;
  slots = info.slots[dev].load(std::memory_order_acquire);
  if (slots > 0) return CALIBATT_OK;
  int cus = 0, per_cu = 0;
  if (hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, smem) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, (const void *)kernel, threads, smem) != hipSuccess ||
      cus <= 0 || per_cu <= 0)
    return CALIBATT_ERR_LAUNCH;
  slots = cus * per_cu;
  info.slots[dev].store(slots, std::memory_order_release);
  return CALIBATT_OK;
}

// Whether rows of `row` elements at every n[0] x n[1] x n[2] multiple of three distances s lie apart: an output's rows are
// written by different workgroups, in any order.  Axes whose rows are all within a step of the next one always do; of layouts
// that interleave otherwise, two indices collide if their rows start less than a row apart.  That is looked for along the two
// shorter axes, for up to 2^16 differences of indices; beyond that the answer is no.
inline bool rows_apart(const int64_t n[3], const int64_t s[3], int64_t row) {
  struct Axis {
    int64_t n, s;
  } axes[3];
  int m = 0;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (s[i] < row) return false;
    axes[m++] = Axis{n[i], s[i]};
  }
  std::sort(axes, axes + m, [](const Axis &a, const Axis &b) { return a.s < b.s; });
  __int128 extent = row;
  bool nested = true;
  for (int i = 0; i < m; ++i) {
    nested = nested && axes[i].s >= extent;
    extent += (__int128)(axes[i].n - 1) * axes[i].s;
  }
  if (nested) return true;
  for (; m < 3; ++m) axes[m] = Axis{1, 0};
  std::sort(axes, axes + 3, [](const Axis &a, const Axis &b) { return a.n < b.n; });
  const Axis &a = axes[0], &b = axes[1], &c = axes[2];
  if (a.n * (2 * (__int128)b.n - 1) > 1 << 16) return false;
  for (int64_t i = 0; i < a.n; ++i)
    for (int64_t j = 1 - b.n; j < b.n; ++j) {
      if (i == 0 && j == 0) continue;  // (rows of one axis are a row apart)
      // the multiples of c's distance next to what i and j make
      const __int128 x = (__int128)i * a.s + (__int128)j * b.s, k = x / c.s;
      for (__int128 t = k - 1; t <= k + 1; ++t) {
        const __int128 d = x - t * c.s;
        if (t > -c.n && t < c.n && d < row && -d < row) return false;
      }
    }
  return true;
}

// Launches through the call that reports its own status: the runtime's "last error" may still hold
// an unrelated error left by earlier calls of the host program.
template <typename Kernel, typename... Args>
int launch_kernel(Kernel kernel, unsigned grid, int threads, int smem, hipStream_t stream, Args... args) {
  void *argv[] = {(void *)&args...};
  return hipLaunchKernel((const void *)kernel, dim3(grid), dim3(threads), argv, smem, stream) == hipSuccess
             ? CALIBATT_OK
             : CALIBATT_ERR_LAUNCH;
}

}  // namespace calibatt_host
