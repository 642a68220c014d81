// Block tables and slot maps of the paged K/V cache, and the way back: pages
// of sequences that end or are cut.
//
// A request with L cached tokens and n new ones holds ceil(L / page) pages and
// needs ceil((L + n) / page); the pages it lacks are the stack entries at the
// exclusive prefix sum of the needs before it.  Both kernels are bound by
// latency (a few dependent loads; 64 requests move 1.3 KB), so each is one
// launch in which no block waits for another: every block forms the prefix
// sums it needs itself, from the lengths, and only reads what no block writes.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "avtp_internal.h"
#include "wave_ops.h"

namespace avtp {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kPer = 4;                     // sequences per thread
constexpr int kChunk = kThreads * kPer;     // sequences whose prefix sums a block holds in LDS
constexpr int kSlots = 1024;                // slots per block

// Exclusive prefix sums over the block's threads, and the block's total.
__device__ inline int block_scan(int v, int *wsum, int &total) {
  const int tid = threadIdx.x, wave = tid >> 6;
  const int incl = (int)wave::prefix_sum((uint32_t)v);
  __syncthreads();  // wsum's last readers are done
  if ((tid & 63) == 63) wsum[wave] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += wsum[w];
    total += wsum[w];
  }
  return before + incl - v;
}

struct Need {
  int L, n, have, need;
  bool room;  // its row of the table and the slot map are long enough
};

struct TArgs {
  PageTables p;
  const int32_t *cu_new, *free_pages;
  int32_t *table, *slot_map, *kv_len;
  int n_new;
};

__device__ inline Need need_of(const TArgs &a, int b) {
  const int ps = a.p.page_shift, mask = (1 << ps) - 1;
  Need r;
  r.L = max(0, a.p.seq_len[b]);
  r.n = max(0, max(0, a.cu_new[b + 1]) - max(0, a.cu_new[b]));
  const long long want = ((long long)r.L + r.n + mask) >> ps;
  r.have = (int)(((long long)r.L + mask) >> ps);
  r.room = want <= a.p.max_pages && a.cu_new[b + 1] <= a.n_new;
  r.need = r.room ? (int)want - r.have : 0;
  return r;
}

// Block i writes the slots [1024 i, 1024 (i + 1)), the table entries of the
// pages that start in them, and the new lengths of the sequences [1024 i,
// 1024 (i + 1)).  It walks the sequences its slots belong to, 1,024 at a time,
// with their offsets, lengths and prefix sums in LDS.
__global__ __launch_bounds__(kThreads) void page_tables_kernel(TArgs a) {
  __shared__ int cu_s[kChunk + 1], len_s[kChunk], off_s[kChunk];
  __shared__ int wsum[kWaves];
  __shared__ int used_s;  // pages of the requests that got theirs (the last block visits every chunk)
  const int tid = threadIdx.x, B = a.p.B, ps = a.p.page_shift, mask = (1 << ps) - 1;
  const int count = min(max(0, a.p.free_count[0]), a.p.n_pages);
  const long long i0 = (long long)blockIdx.x * kSlots, i1 = min(i0 + kSlots, (long long)a.n_new);
  const int own0 = blockIdx.x * kChunk, own1 = min(own0 + kChunk, B);
  const bool last = own0 < B && own1 == B;
  const int n_tot = a.cu_new[B];

  // entries behind the batch
  for (long long i = max(i0, (long long)max(0, n_tot)) + tid; i < i1; i += kThreads) a.slot_map[i] = -1;

  const bool slots = i0 < min(i1, (long long)n_tot);
  if (!slots && own0 >= B) return;
  if (tid == 0) used_s = 0;  // (a barrier of the first scan lies before its first use)
  int base = 0;              // pages needed by the sequences before the chunk
  for (int c0 = 0; c0 < B; c0 += kChunk) {
    const int c1 = min(c0 + kChunk, B);
    const bool mine = c0 == own0;
    const bool here = slots && a.cu_new[c0] < i1 && a.cu_new[c1] > i0;
    const bool later = (own0 < B && own0 >= c1) || (slots && a.cu_new[c1] < i1);
    if (!mine && !here && !later) break;
    // thread t: sequences c0 + 4 t .. + 3
    Need r[kPer];
    int sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = c0 + tid * kPer + j;
      r[j] = b < c1 ? need_of(a, b) : Need{0, 0, 0, 0, true};
      sum += r[j].need;
    }
    int total;
    int off = base + block_scan(sum, wsum, total);
    int got = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = c0 + tid * kPer + j;
      if (b < c1) {
        const bool fits = r[j].room && (r[j].need == 0 || off + r[j].need <= count);
        if (fits && r[j].need > 0) got = off + r[j].need;  // (fitting requests are a prefix of those in need)
        if (mine) {
          a.p.seq_len_out[b] = fits ? r[j].L + r[j].n : r[j].L;
          if (a.kv_len && r[j].n > 0) a.kv_len[b] = fits ? r[j].L + r[j].n : 0;
          if (!fits && a.p.status) atomicOr(&a.p.status[b], AVTP_FLAG_NO_PAGES);
        }
        if (here) {
          cu_s[tid * kPer + j] = max(0, a.cu_new[b]);
          if (b + 1 == c1) cu_s[c1 - c0] = max(0, a.cu_new[c1]);
          len_s[tid * kPer + j] = r[j].L;
          off_s[tid * kPer + j] = fits ? off : -1;
        }
        off += r[j].need;
      }
    }
    if (last && got > 0) atomicMax(&used_s, got);
    if (here) {
      __syncthreads();
      const int m = c1 - c0;
      const int lo = (int)max(i0, (long long)cu_s[0]), hi = (int)min(i1, (long long)cu_s[m]);
      for (int i = lo + tid; i < hi; i += kThreads) {
        int x = 0, y = m;  // the sequence of slot i: the last one that starts at or before it
        while (y - x > 1) {
          const int h = (x + y) >> 1;
          if (cu_s[h] <= i) x = h;
          else y = h;
        }
        const int b = c0 + x, L = len_s[x], o = off_s[x], pos = L + (i - cu_s[x]);
        int slot = -1;
        if (o >= 0 && i < cu_s[x + 1]) {
          const int pg = pos >> ps, fresh = pg - (int)(((long long)L + mask) >> ps);
          const size_t e = (size_t)b * a.p.max_pages + pg;
          int id;
          if (fresh >= 0) {  // a page of this step, from the top of the stack
            id = a.free_pages[count - 1 - (o + fresh)];
            if ((pos & mask) == 0) a.table[e] = id;
          } else {
            id = a.table[e];
          }
          if ((unsigned)id < (unsigned)a.p.n_pages) slot = (id << ps) + (pos & mask);
          else if (a.p.status) atomicOr(&a.p.status[b], AVTP_FLAG_BAD_PAGE);
        }
        a.slot_map[i] = slot;
      }
      __syncthreads();
    }
    base += total;
  }
  if (last) {
    __syncthreads();
    if (tid == 0) a.p.free_count_out[0] = count - used_s;
  }
}

struct RArgs {
  PageTables p;
  const int32_t *keep_len, *table;
  int32_t *free_pages;
  int per_block;  // sequences per block
};

struct Back {
  int keep, first, n;  // kept tokens, first page handed back, pages handed back
};
__device__ inline Back back_of(const RArgs &a, int b) {
  const int ps = a.p.page_shift, mask = (1 << ps) - 1;
  const int L = max(0, a.p.seq_len[b]);
  Back r;
  r.keep = min(max(0, a.keep_len[b]), L);
  r.first = (int)(((long long)r.keep + mask) >> ps);
  const int have = min((int)(((long long)L + mask) >> ps), a.p.max_pages);
  r.n = max(0, have - r.first);
  return r;
}

// Block i hands back the pages of its per_block sequences (a wave each at a
// time), after summing what the sequences before them hand back.
__global__ __launch_bounds__(kThreads) void page_trim_kernel(RArgs a) {
  __shared__ int wsum[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = a.p.B;
  const int count = min(max(0, a.p.free_count[0]), a.p.n_pages);
  const int b0 = blockIdx.x * a.per_block, b1 = min(b0 + a.per_block, B);
  int sum = 0, before;
  for (int b = tid; b < b0; b += kThreads) sum += back_of(a, b).n;
  block_scan(sum, wsum, before);
  // lane j: the block's sequence j (every wave holds them all)
  Back r{0, 0, 0};
  if (b0 + lane < b1) r = back_of(a, b0 + lane);
  // (B * max_pages pages handed back onto n_pages: below 2^32)
  const uint32_t end = (uint32_t)count + (uint32_t)before + wave::prefix_sum((uint32_t)r.n);
  const uint32_t cap = (uint32_t)a.p.n_pages;
  for (int j = wave; j < b1 - b0; j += kWaves) {
    const int n = __builtin_amdgcn_readlane(r.n, j);
    const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)end, j) - (uint32_t)n;
    const int m = at < cap ? (int)min((uint32_t)n, cap - at) : 0;
    const int32_t *row = a.table + (size_t)(b0 + j) * a.p.max_pages + __builtin_amdgcn_readlane(r.first, j);
    for (int i = lane; i < m; i += 64) a.free_pages[at + i] = row[i];
    if (m < n && lane == 0 && a.p.status) atomicOr(&a.p.status[b0 + j], AVTP_FLAG_OUT_CAPACITY);
  }
  if (wave == 0 && b0 + lane < b1) a.p.seq_len_out[b0 + lane] = r.keep;
  if (b1 == B && tid == 63) a.p.free_count_out[0] = (int)min(end, cap);
}

}  // namespace

hipError_t launch_page_tables(hipStream_t st, const PageTables &P, const int32_t *cu_new,
                              const int32_t *free_pages, int32_t *block_table, int32_t *slot_map,
                              int64_t n_new, int32_t *kv_len) {
  clear_pending_error();
  const TArgs a{P, cu_new, free_pages, block_table, slot_map, kv_len, (int)n_new};
  const long long nb = (n_new + kSlots - 1) / kSlots, sb = (P.B + kChunk - 1) / kChunk;
  hipLaunchKernelGGL(page_tables_kernel, dim3((unsigned)(nb > sb ? nb : sb)), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_trim(hipStream_t st, const PageTables &P, const int32_t *keep_len,
                            const int32_t *block_table, int32_t *free_pages) {
  clear_pending_error();
  // four sequences a block (one per wave) up to 1,024 blocks, at most 64 (one per lane)
  int per = (P.B + 1023) / 1024;
  static_assert(AVTP_MAX_REQUESTS / 1024 <= 64, "a lane per sequence of a block");
  per = per < kWaves ? kWaves : per;
  const RArgs a{P, keep_len, block_table, free_pages, per};
  hipLaunchKernelGGL(page_trim_kernel, dim3((unsigned)((P.B + per - 1) / per)), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace avtp
