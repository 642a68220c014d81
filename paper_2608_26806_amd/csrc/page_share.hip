// Pages that several sequences name: new sequences that start from another's
// tokens, copies of whole pages, and pages handed back when no row of the table
// names them any more.
//
// No counts of a page's holders are kept between calls, where they could go out
// of step with the table: a release counts them from the rows, which it has to
// read in part anyway (64 sequences of 500 pages: 128 KB).  Forks and releases are
// bound by latency, copies by the memory's rate.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "avtp_internal.h"
#include "wave_ops.h"

namespace avtp {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ inline int pages_of(int tokens, int shift) { return (int)(((long long)tokens + (1 << shift) - 1) >> shift); }
__device__ inline bool in_pool(int id, int n_pages) { return (unsigned)id < (unsigned)n_pages; }

// the sum over the block's threads (every thread gets it)
template <int WAVES>
__device__ inline int block_sum(int v, int *wsum) {
  const int s = (int)wave::sum((uint32_t)v);
  __syncthreads();  // wsum's last readers are done
  if ((threadIdx.x & 63) == 0) wsum[threadIdx.x >> 6] = s;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) total += wsum[w];
  return total;
}

// ---- forks

struct Fork {
  int parent, len;  // parent < 0: the sequence stays as it was
  int need;         // 1: its last page is partly filled, it gets one of its own
  bool refused;
};
// N sequences b0 + i step (parent < 0 behind the last), whose loads are in flight
// together: with the four that a thread of the last block counts of 1,024 sequences one
// after the other 768 forks of up to 2,048 pages took 5.7 us instead of 4.8.
template <int N>
__device__ inline void forks_of(const PageFork &a, int b0, int step, int last, Fork *f) {
  int own[N], L[N], pp[N], gone[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int b = min(b0 + i * step, a.B - 1);
    f[i].parent = a.parent[b];
    f[i].len = a.fork_len[b];
    own[i] = a.seq_len[b];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = min(max(0, f[i].parent), a.B - 1);
    L[i] = max(0, a.seq_len[p]);
    pp[i] = a.parent[p];
    gone[i] = a.gone ? a.gone[p] : 0;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool asked = f[i].parent >= 0 && b0 + i * step < last;
    const bool ok = f[i].parent < a.B && own[i] <= 0 && pp[i] < 0 && f[i].len >= 0 && f[i].len <= L[i] &&
                    pages_of(max(0, f[i].len), a.page_shift) <= a.max_pages && (gone[i] <= 0 || f[i].len == L[i]);
    f[i].refused = asked && !ok;
    if (!asked || !ok) f[i].parent = -1;
    f[i].need = f[i].parent >= 0 && (f[i].len & ((1 << a.page_shift) - 1)) != 0;
  }
}

// Block i makes the forks of its per_block sequences (a wave each at a time),
// after counting the pages that the sequences before them take.  Rows that are
// read are not written: a parent is no fork of the same call.
struct FArgs {
  PageFork f;
  int per_block;
};
__global__ __launch_bounds__(kThreads) void page_fork_kernel(FArgs x) {
  __shared__ int wsum[kWaves];
  const PageFork &a = x.f;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int count = min(max(0, a.free_count[0]), a.n_pages);
  const int b0 = blockIdx.x * x.per_block, b1 = min(b0 + x.per_block, a.B);
  int sum = 0;
  constexpr int U = 4;
  for (int b = tid; b < b0; b += kThreads * U) {
    Fork f[U];
    forks_of<U>(a, b, kThreads, b0, f);
#pragma unroll
    for (int u = 0; u < U; ++u) sum += f[u].need;
  }
  const int before = block_sum<kWaves>(sum, wsum);
  // lane j: the block's sequence j (every wave holds them all)
  const int b = b0 + lane;
  Fork f;
  forks_of<1>(a, b, 0, b1, &f);
  const int end = before + (int)wave::prefix_sum((uint32_t)f.need);
  const bool fits = f.need == 0 || end <= count;
  int src = -1, dst = -1;
  if (f.parent >= 0 && f.need && fits) {
    src = a.table[(size_t)f.parent * a.max_pages + (f.len >> a.page_shift)];
    dst = a.free_pages[count - end];
  }
  for (int j = wave; j < b1 - b0; j += kWaves) {
    const int parent = __builtin_amdgcn_readlane(f.parent, j), len = __builtin_amdgcn_readlane(f.len, j);
    if (parent < 0 || !__builtin_amdgcn_readlane((int)fits, j)) continue;
    const int whole = len >> a.page_shift, fresh = __builtin_amdgcn_readlane(dst, j);
    const int32_t *from = a.table + (size_t)parent * a.max_pages;
    int32_t *to = a.table + (size_t)(b0 + j) * a.max_pages;
    constexpr int V = 8;  // entries in flight
    for (int i = lane; i < whole; i += 64 * V) {
      int32_t x[V];
#pragma unroll
      for (int u = 0; u < V; ++u) x[u] = from[min(i + 64 * u, whole - 1)];
#pragma unroll
      for (int u = 0; u < V; ++u)
        if (i + 64 * u < whole) to[i + 64 * u] = x[u];
    }
    if (lane == 0 && __builtin_amdgcn_readlane(f.need, j)) to[whole] = fresh;
  }
  if (wave == 0 && b < b1) {
    const bool made = f.parent >= 0 && fits;
    const bool good = in_pool(src, a.n_pages) && in_pool(dst, a.n_pages);
    a.seq_len_out[b] = made ? f.len : a.seq_len[b];
    a.src_page[b] = good ? src : -1;
    a.dst_page[b] = good ? dst : -1;
    if (a.gone) a.gone_out[b] = made ? a.gone[f.parent] : a.gone[b];
    const int flags = (f.refused ? AVTP_FLAG_REFUSED : 0) | (fits ? 0 : AVTP_FLAG_NO_PAGES) |
                      (made && f.need && !good ? AVTP_FLAG_BAD_PAGE : 0);
    if (flags && a.status) atomicOr(&a.status[b], flags);
  }
  if (b1 == a.B && tid == 63) a.free_count_out[0] = count - min(end, count);
}

// ---- copies of pages

struct CArgs {
  char *k, *v;
  const int32_t *src, *dst;
  long long page_bytes;
  int chunks, n_pages;  // chunks of a page, blocks of one page and tensor
};
__global__ __launch_bounds__(kThreads) void page_copy_kernel(CArgs a) {
  const unsigned i = blockIdx.x / (2 * a.chunks), part = blockIdx.x % (2 * a.chunks);
  const int src = a.src[i], dst = a.dst[i];
  if (!in_pool(src, a.n_pages) || !in_pool(dst, a.n_pages)) return;
  char *base = part & 1 ? a.v : a.k;
  const int u = (int)(part >> 1) * kThreads + threadIdx.x;
  if (u < (int)(a.page_bytes / 16))
    reinterpret_cast<uint4 *>(base + dst * a.page_bytes)[u] = reinterpret_cast<const uint4 *>(base + src * a.page_bytes)[u];
}

// ---- releases
//
// A sequence of L tokens whose tokens from the sinks to `gone` have left its window
// holds the pages [0, S) and [max(S, gone / page), ceil(L / page)) of its row, S the
// pages of the sinks.  A page goes back when all rows that held it before the call
// let it go: `holders` counts the rows before, `dropped` those that let go, both
// by integer atomics, whose order does not show.  Freed pages are pushed by number.
//
// Small pools are counted in the LDS of one block, in one launch: 64 requests that
// share eight prompts (15,000 entries) take 8.2 us, two requests 3.5; in four launches
// over the chip, which count in a workspace (clear, count, drop, push), 14.6 and 14.5,
// mostly the launches.  128 requests of 100 entries 8.3 against 15.0 (256 of them 16 us
// in a block of 1,024 rows).  1,024 requests behind a window, 68,000 entries: 16.3.

constexpr int kPer = 4;               // entries of a row per lane
constexpr int kSegment = 64 * kPer;   // and of a wave
constexpr int kChunk = kThreads * 4;  // pages whose freed ones are counted together

struct Held {
  int end, sinks, first;  // pages of the row: [0, sinks) and [first, end)
  __device__ inline int count() const { return sinks + max(0, end - first); }
  __device__ inline int entry(int i) const { return i < sinks ? i : first + i - sinks; }
};
__device__ inline Held held(const PageRelease &r, int tokens, int gone) {
  Held h;
  h.end = min(pages_of(tokens, r.page_shift), r.max_pages);
  const int s = pages_of(r.sinks, r.page_shift);
  h.sinks = min(s, h.end);
  h.first = max(s, gone >> r.page_shift);
  return h;
}
// what `before` holds and `after` does not: up to three runs of a row
struct Gone {
  int a0, a1, b0, b1, c0, c1;
  __device__ inline Gone(const Held &before, const Held &after)
      : a0(after.sinks), a1(before.sinks), b0(before.first), b1(max(b0, min(after.first, before.end))),
        c0(max(b1, after.end)), c1(before.end) {}
  __device__ inline int count() const { return max(0, a1 - a0) + (b1 - b0) + max(0, c1 - c0); }
  __device__ inline int entry(int i) const {
    const int a = max(0, a1 - a0);
    if (i < a) return a0 + i;
    return i - a < b1 - b0 ? b0 + i - a : c0 + i - a - (b1 - b0);
  }
};
struct Row {
  int L, gone, keep;  // before; keep: the tokens asked for, or kept
};
__device__ inline Row row_of(const PageRelease &r, int b) {
  const int L = max(0, r.seq_len[b]);
  return {L, r.gone ? max(0, r.gone[b]) : 0, min(max(0, r.keep_len[b]), L)};
}
// What row b keeps, and of its window; with `say` it is written down.
__device__ inline Row kept(const PageRelease &r, int b, const Row &x, const int *holders, bool say) {
  const int W = r.window;
  Row y = x;
  bool refused = false;
  if (x.keep > 0 && x.keep < x.L) {
    // no cut inside a page that others hold, none behind what the window has left
    const int at = x.keep >> r.page_shift;
    const bool inside = (x.keep & ((1 << r.page_shift) - 1)) && at < r.max_pages;
    const int id = inside ? r.table[(size_t)b * r.max_pages + at] : -1;
    refused = in_pool(id, r.n_pages) && holders[id] > 1;
    if (x.gone > 0 && (W == 0 || x.keep - W + 1 < x.gone)) refused = true;
  }
  if (refused) y.keep = x.L;
  else if (x.keep == 0) y.gone = 0;
  else if (W > 0) y.gone = max(x.gone, x.keep - W + 1);
  if (say) {
    r.seq_len_out[b] = y.keep;
    if (r.gone_out) r.gone_out[b] = y.gone;
    if (refused && r.status) atomicOr(&r.status[b], AVTP_FLAG_REFUSED);
  }
  return y;
}

// LANES lanes count the entries i0 .. of what row b holds, PER each, their loads in
// flight together.
template <int LANES, int PER>
__device__ inline void count_entries(const PageRelease &r, int b, const Held &h, int i0, int *holders) {
  const int32_t *row = r.table + (size_t)b * r.max_pages;
  const int n = h.count(), i = i0 + (int)(threadIdx.x % LANES);
  int id[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) id[u] = i + u * LANES < n ? row[h.entry(i + u * LANES)] : 0;
  bool bad = false;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    if (i + u * LANES >= n) break;
    if (in_pool(id[u], r.n_pages)) atomicAdd(&holders[id[u]], 1);
    else bad = true;
  }
  if (bad && r.status) atomicOr(&r.status[b], AVTP_FLAG_BAD_PAGE);
}
// And let go of the entries i0 .. of what it holds no longer; freed: by chunks, or null.
template <int LANES, int PER>
__device__ inline void drop_entries(const PageRelease &r, int b, const Gone &g, int i0, const int *holders,
                                    int *dropped, int *freed) {
  const int32_t *row = r.table + (size_t)b * r.max_pages;
  const int n = g.count(), i = i0 + (int)(threadIdx.x % LANES);
  int id[PER], before[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) id[u] = i + u * LANES < n ? row[g.entry(i + u * LANES)] : -1;
#pragma unroll
  for (int u = 0; u < PER; ++u) before[u] = in_pool(id[u], r.n_pages) ? atomicAdd(&dropped[id[u]], 1) : 0;
  if (!freed) return;
#pragma unroll
  for (int u = 0; u < PER; ++u)
    if (in_pool(id[u], r.n_pages) && before[u] + 1 == holders[id[u]]) atomicAdd(&freed[id[u] / kChunk], 1);
}
__device__ inline int stack_of(const PageRelease &r) { return min(max(0, r.free_count[0]), r.n_pages); }

// Four pages from p0 on for each of the block's threads: the freed ones go onto the
// stack from place `at` on, which moves up.
template <int WAVES>
__device__ inline void push_freed(const PageRelease &r, int p0, const int4 &h, const int4 &d, int &at, int *wsum) {
  const int tid = threadIdx.x, wave = tid >> 6;
  const bool f[4] = {h.x > 0 && h.x == d.x, h.y > 0 && h.y == d.y, h.z > 0 && h.z == d.z, h.w > 0 && h.w == d.w};
  const int n = f[0] + f[1] + f[2] + f[3];
  const int incl = (int)wave::prefix_sum((uint32_t)n);
  __syncthreads();  // wsum's last readers are done
  if ((tid & 63) == 63) wsum[wave] = incl;
  __syncthreads();
  int place = at + incl - n;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) place += wsum[w];
    at += wsum[w];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (f[i]) {
      if (place < r.n_pages) r.free_pages[place] = p0 + i;
      ++place;
    }
}

constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;
constexpr int kSmallRows = 128;
constexpr long long kSmallEntries = 1 << 17;  // of the table, of which few rows fill theirs
constexpr int kSmallPages = 16384;           // whose counts fill 128 KB of LDS
constexpr int kGroup = 32;                   // lanes that walk a row, kPer entries each at a time
__global__ __launch_bounds__(kSmallThreads) void page_release_small_kernel(PageRelease r) {
  __shared__ __attribute__((aligned(16))) int holders[kSmallPages], dropped[kSmallPages];
  __shared__ Row before[kSmallRows], after[kSmallRows];
  __shared__ int wsum[kSmallWaves];
  const int tid = threadIdx.x;
  int at = stack_of(r);
  if (tid < r.B) before[tid] = row_of(r, tid);
  for (int i = tid * 4; i < r.n_pages; i += kSmallThreads * 4)
    *reinterpret_cast<int4 *>(holders + i) = *reinterpret_cast<int4 *>(dropped + i) = make_int4(0, 0, 0, 0);
  __syncthreads();
  constexpr int kGroups = kSmallThreads / kGroup;
  for (int b = tid / kGroup; b < r.B; b += kGroups) {
    const Held h = held(r, before[b].L, before[b].gone);
    for (int i0 = 0; i0 < h.count(); i0 += kGroup * kPer) count_entries<kGroup, kPer>(r, b, h, i0, holders);
  }
  __syncthreads();
  if (tid < r.B) after[tid] = kept(r, tid, before[tid], holders, true);
  __syncthreads();
  for (int b = tid / kGroup; b < r.B; b += kGroups) {
    const Gone g(held(r, before[b].L, before[b].gone), held(r, after[b].keep, after[b].gone));
    for (int i0 = 0; i0 < g.count(); i0 += kGroup * kPer)
      drop_entries<kGroup, kPer>(r, b, g, i0, holders, dropped, nullptr);
  }
  __syncthreads();
  for (int p0 = 0; p0 < r.n_pages; p0 += kSmallThreads * 4) {
    const int p = p0 + tid * 4;
    int4 h = make_int4(0, 0, 0, 0), d = h;
    if (p < r.n_pages) {
      h = *reinterpret_cast<const int4 *>(holders + p);
      d = *reinterpret_cast<const int4 *>(dropped + p);
    }
    push_freed<kSmallWaves>(r, p, h, d, at, wsum);
  }
  if (tid == 0) r.free_count_out[0] = min(at, r.n_pages);
}

struct LArgs {
  PageRelease r;
  int *holders, *dropped, *freed;  // workspace
  int waves;                       // that share a row, kSegment entries each at a time
};
// the counts, which lie in one piece
__global__ __launch_bounds__(kThreads) void page_release_clear_kernel(int4 *ws, long long n) {
  const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) ws[i] = make_int4(0, 0, 0, 0);
}
// which row, and the wave's number in it
__device__ inline int row_wave(const LArgs &a, int &w) {
  const unsigned x = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  w = (int)(x % (unsigned)a.waves);
  return (int)(x / (unsigned)a.waves);
}
__global__ __launch_bounds__(kThreads) void page_release_count_kernel(LArgs a) {
  int w;
  const int b = row_wave(a, w);
  if (b >= a.r.B) return;
  const Row x = row_of(a.r, b);
  const Held h = held(a.r, x.L, x.gone);
  for (int i0 = w * kSegment; i0 < h.count(); i0 += a.waves * kSegment) count_entries<64, kPer>(a.r, b, h, i0, a.holders);
}
__global__ __launch_bounds__(kThreads) void page_release_drop_kernel(LArgs a) {
  int w;
  const int b = row_wave(a, w);
  if (b >= a.r.B) return;
  const Row x = row_of(a.r, b), y = kept(a.r, b, x, a.holders, w == 0 && (threadIdx.x & 63) == 0);
  const Gone g(held(a.r, x.L, x.gone), held(a.r, y.keep, y.gone));
  for (int i0 = w * kSegment; i0 < g.count(); i0 += a.waves * kSegment)
    drop_entries<64, kPer>(a.r, b, g, i0, a.holders, a.dropped, a.freed);
}
// Block i pushes the freed ones of the pages [1024 i, 1024 (i + 1)), four a thread.
__global__ __launch_bounds__(kThreads) void page_release_push_kernel(LArgs a) {
  __shared__ int wsum[kWaves];
  const int tid = threadIdx.x, p0 = blockIdx.x * kChunk + tid * 4;
  const int4 h = *reinterpret_cast<const int4 *>(a.holders + p0), d = *reinterpret_cast<const int4 *>(a.dropped + p0);
  int sum = 0;
  for (int i = tid; i < (int)blockIdx.x; i += kThreads) sum += a.freed[i];
  int at = stack_of(a.r) + block_sum<kWaves>(sum, wsum);
  push_freed<kWaves>(a.r, p0, h, d, at, wsum);
  if (blockIdx.x == gridDim.x - 1 && tid == 0) a.r.free_count_out[0] = min(at, a.r.n_pages);
}

}  // namespace

hipError_t launch_page_fork(hipStream_t st, const PageFork &F) {
  clear_pending_error();
  // four sequences a block (one per wave) up to 1,024 blocks, at most 64 (one per lane)
  int per = (F.B + 1023) / 1024;
  static_assert(AVTP_MAX_REQUESTS / 1024 <= 64, "a lane per sequence of a block");
  per = per < kWaves ? kWaves : per;
  const FArgs a{F, per};
  hipLaunchKernelGGL(page_fork_kernel, dim3((unsigned)((F.B + per - 1) / per)), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_copy(hipStream_t st, const avtp_pages &P, const int32_t *src_page,
                            const int32_t *dst_page, int64_t n) {
  clear_pending_error();
  CArgs a;
  a.k = (char *)P.k;
  a.v = (char *)P.v;
  a.src = src_page;
  a.dst = dst_page;
  a.page_bytes = (long long)P.Hkv * P.page_size * P.d * (P.dtype == AVTP_FP32 ? 4 : 2);
  constexpr int kBytes = kThreads * 16;
  a.chunks = (int)((a.page_bytes + kBytes - 1) / kBytes);
  a.n_pages = P.n_pages;
  // (blocks of 256 threads, fewer than 2^24 in a launch)
  const int64_t most = ((1 << 24) - 1) / (2 * a.chunks);
  for (int64_t i = 0; i < n; i += most) {
    const int64_t m = n - i < most ? n - i : most;
    hipLaunchKernelGGL(page_copy_kernel, dim3((unsigned)(m * 2 * a.chunks)), dim3(kThreads), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.src += m;
    a.dst += m;
  }
  return hipSuccess;
}

// holders and dropped, whole chunks of them, and freed
static size_t chunks_of(int n_pages) { return ((size_t)n_pages + kChunk - 1) / kChunk; }
size_t page_release_workspace_bytes(int n_pages) { return (2 * kChunk * 4 + 4) * chunks_of(n_pages) + 12; }

hipError_t launch_page_release(hipStream_t st, const PageRelease &R, int32_t *ws) {
  clear_pending_error();
  LArgs a;
  a.r = R;
  const size_t chunks = chunks_of(R.n_pages);
  a.holders = ws;
  a.dropped = ws + chunks * kChunk;
  a.freed = ws + 2 * chunks * kChunk;
  // enough waves to fill the chip, of which short rows use one
  const int most = (R.max_pages + kSegment - 1) / kSegment, want = (4096 + R.B - 1) / R.B;
  a.waves = most < want ? most : want;
  if (R.n_pages <= kSmallPages && R.B <= kSmallRows && (long long)R.B * R.max_pages <= kSmallEntries) {
    hipLaunchKernelGGL(page_release_small_kernel, dim3(1), dim3(kSmallThreads), 0, st, R);
    return hipGetLastError();
  }
  const long long units = (long long)((2 * chunks * kChunk + chunks + 3) / 4), waves = (long long)R.B * a.waves;
  const dim3 rows((unsigned)((waves + kWaves - 1) / kWaves));
  hipLaunchKernelGGL(page_release_clear_kernel, dim3((unsigned)((units + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                     st, (int4 *)ws, units);
  hipLaunchKernelGGL(page_release_count_kernel, rows, dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(page_release_drop_kernel, rows, dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(page_release_push_kernel, dim3((unsigned)chunks), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace avtp
