// K and V rows into the pages of the cache: row r of the batch (or row
// keep_idx[r], after a selection) to the place that slot_map[r] names.
//
// HBM-bound bit copy: every row is read once and written once, in 16-byte
// units.  A row of one tensor is Hkv pieces of one head each, and a page keeps
// a head's tokens together, so a piece of 128 to 512 bytes is the run that lands
// in one place.  One row per group of threads: with two, four or eight rows in
// flight per group there were that many times fewer waves, and 15,000 rows of
// 8 heads of 128 (120 MB moved) took 27, 36 and 42 us instead of 19.5.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "avtp_internal.h"

namespace avtp {
namespace {

constexpr int kThreads = 256;

struct SArgs {
  const char *k, *v;
  char *kp, *vp;
  long long k_stride, v_stride, n_src;
  const int32_t *slot, *keep;
  long long n;
  int units;       // 16-byte units per row
  int lpr_shift;   // log2 of the threads that share a row
  int unit_shift;  // log2 of the units of one head
  int page_shift, Hkv;
  long long slots;  // of the pool
};

__global__ __launch_bounds__(kThreads) void page_store_kernel(SArgs a) {
  const int lane = threadIdx.x & ((1 << a.lpr_shift) - 1);
  const long long block = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  const long long r = block * (kThreads >> a.lpr_shift) + (threadIdx.x >> a.lpr_shift);
  if (r >= a.n) return;
  const long long s = a.slot[r], j = a.keep ? a.keep[r] : r;
  if (s < 0 || s >= a.slots || j < 0 || j >= a.n_src) return;
  const char *k = a.k + j * a.k_stride, *v = a.v + j * a.v_stride;
  const long long page = (s >> a.page_shift) * a.Hkv, at = s & ((1 << a.page_shift) - 1);
  for (int u = lane; u < a.units; u += 1 << a.lpr_shift) {
    const int h = u >> a.unit_shift, c = u & ((1 << a.unit_shift) - 1);
    const uint4 x = *reinterpret_cast<const uint4 *>(k + u * 16ll), y = *reinterpret_cast<const uint4 *>(v + u * 16ll);
    const long long o = (((((page + h) << a.page_shift) + at) << a.unit_shift) + c) * 16;
    *reinterpret_cast<uint4 *>(a.kp + o) = x;
    *reinterpret_cast<uint4 *>(a.vp + o) = y;
  }
}

}  // namespace

hipError_t launch_page_store(hipStream_t st, const avtp_pages &P, const void *k, int64_t k_stride,
                             const void *v, int64_t v_stride, int64_t n_src, const int32_t *slot_map,
                             const int32_t *keep_idx, int64_t n) {
  clear_pending_error();
  SArgs a;
  a.k = (const char *)k;
  a.v = (const char *)v;
  a.kp = (char *)P.k;
  a.vp = (char *)P.v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.n_src = n_src;
  a.slot = slot_map;
  a.keep = keep_idx;
  a.n = n;
  const int head_units = P.d * (P.dtype == AVTP_FP32 ? 4 : 2) / 16;  // a power of two
  a.units = P.Hkv * head_units;
  a.unit_shift = __builtin_ctz((unsigned)head_units);
  a.lpr_shift = 0;
  while ((1 << a.lpr_shift) < a.units && (1 << a.lpr_shift) < kThreads) ++a.lpr_shift;
  a.page_shift = __builtin_ctz((unsigned)P.page_size);
  a.Hkv = P.Hkv;
  a.slots = (long long)P.n_pages * P.page_size;
  const long long rows = kThreads >> a.lpr_shift, blocks = (n + rows - 1) / rows;
  constexpr long long kWide = 1 << 20;  // blocks side by side (2^32 threads are too many for one axis)
  const dim3 grid((unsigned)(blocks < kWide ? blocks : kWide), (unsigned)((blocks + kWide - 1) / kWide));
  hipLaunchKernelGGL(page_store_kernel, grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace avtp
