// Attention of new tokens over the paged K/V cache on gfx950 (MFMA, wave64).
//
// One pass over the keys with the running maximum m and sum l of each row's
// softmax: for a tile of keys, z = c q.k, and when a row's maximum rises from
// m to m' its sum and its output so far are scaled by exp(m - m').  Neither the
// logits nor the probabilities leave the registers:
//   S^T = K Q^T: keys are the MFMA's rows, query rows its columns, so a lane
//     owns one query row (half of its keys with the 32-row MFMA, the other half
//     is 32 lanes away; with the 16-row MFMA a quarter, 16 lanes apart) and the
//     softmax needs one exchange per tile, for the maximum;
//   O^T = V^T P^T: the probabilities a lane holds are its part of the second
//     product's operand as they are (the order of the keys inside a product is
//     free, as long as V's rows come in the same order), and scaling O by
//     exp(m - m') is one factor per lane.
// K and V tiles stream to LDS by direct loads (buffer form, 16 bytes per lane),
// double-buffered.  Rows of the wave tile are (token, head of the group) pairs,
// the G query heads of a key head side by side, so all of them share the tile.
//
// A page has 16 tokens or more and a wave loads 16 tokens or fewer at a time,
// so the page is uniform in a load: its address is the buffer's base, 64 bits.
// The buffer's size is what the sequence has of those tokens: the places behind
// the last token, and pages outside the pool, come as zeros.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <cmath>
#include <type_traits>

#include "avtp_internal.h"
#include "wave_ops.h"

namespace avtp {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t Rsrc;
#define AVTP_LDS __attribute__((address_space(3)))

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kTile = 32;  // keys of a tile
// A row's exponentials refer to the largest logit m of some earlier tile, not
// always of all: only when their sum over a tile leaves this range is m raised
// (and the sum and output so far scaled).  fp32 sums, and products with bf16 or
// fp32 probabilities of that size, are as exact as with the true maximum.  The limit
// holds for the keys of one lane, 8 of a tile's 32 at the fewest (the 16-row MFMA): a
// row's sum stays below 2^13 per key, and its output below 2^128 while |v| is at
// most 2^114 over the keys.
constexpr float kLazyLimit = 65536.f;

template <typename T, int D>
struct Geo {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int ROWB = D * (int)sizeof(T);  // bytes of a head row
  static constexpr int NCH = ROWB / 16;            // its 16-byte chunks
  static constexpr int RPL = 64 / NCH;             // rows of a wave's load
  // Chunk order inside an LDS row, XOR-ed with the row: 16 consecutive rows of
  // one chunk (a K fragment) lie in 16 different places of the 64 banks, and so
  // do the four 64-byte pieces of consecutive rows that a transposing read of
  // bf16 V takes (with those of the next four rows in the other lane half).
  static __device__ inline int swz(int row) {
    if (F32) return row & 15;
    return NCH == 16 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  }
};

// values dd .. dd + 3 of an output row
template <typename T>
__device__ inline void put4(char *row, int dd, f32x4 x) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4 *>(row + dd * 4) = x;
  } else {
    bf16x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (__bf16)x[i];
    *reinterpret_cast<bf16x4 *>(row + dd * 2) = y;
  }
}

struct KArgs {
  static constexpr bool WIN = false;
  const char *q, *k, *v;
  char *out;
  long long q_tok, out_tok, head_bytes;  // head_bytes: one head of one page
  float *lse, *po, *pl;
  const int32_t *cu_q, *kv_len, *table;
  int32_t *status;
  int B, Hkv, G, N_q, max_pages, n_pages, page_shift;
  int workers, nsplit, least;  // see PageAttnPlan
  float gain, from;
  int4 *meta;                  // two per possible cut tile
  float cl2e;
};
// Rows that see a window of the latest tokens and the first ones (PageWindow).
struct WArgs : KArgs {
  static constexpr bool WIN = true;
  int window, sinks;
};

// A buffer of `bytes` bytes at p, both the same in every lane (said once more
// here: left to the compiler's analysis, every load became a loop over lanes).
__device__ inline Rsrc make_rsrc(const char *p, int bytes) {
  const unsigned long long u = (unsigned long long)p;
  const unsigned long long lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)u);
  const unsigned long long hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(u >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void *)(lo | hi << 32), 0, __builtin_amdgcn_readfirstlane(bytes),
                                           0x00027000);
}

// wait for this wave's outstanding loads, direct-to-LDS ones included
__device__ inline void wait_vmem() {
  __builtin_amdgcn_s_waitcnt(0xF70);
  asm volatile("" ::: "memory");
}

// Over the lanes that hold the same row, 64 / M of them M lanes apart.
template <int M, typename F>
__device__ inline float over_row(float x, F f) {
  auto both = [&](auto p) __attribute__((always_inline)) {
    return f(__builtin_bit_cast(float, (unsigned)p[0]), __builtin_bit_cast(float, (unsigned)p[1]));
  };
  if (M == 16) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    x = both(__builtin_amdgcn_permlane16_swap(u, u, false, false));
  }
  const unsigned u = __builtin_bit_cast(unsigned, x);
  return both(__builtin_amdgcn_permlane32_swap(u, u, false, false));
}

// The MFMA of M rows and columns.  A lane holds column lane mod M; of the M rows
// it holds those with (row / 4) mod (64 / M) = lane / M, and of a product's
// inner index the share number lane / M.
template <int M>
struct Mma;
template <>
struct Mma<32> {
  typedef f32x16 acc;
  static __device__ inline acc run(bf16x8 a, bf16x8 b, acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ inline acc run(float a, float b, acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<16> {
  typedef f32x4 acc;
  static __device__ inline acc run(bf16x8 a, bf16x8 b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ inline acc run(float a, float b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
};

// The work.  A row tile is BM rows (token, head of the group) of one sequence
// and key head; a unit is one stage of KS keys of a tile, and a tile has the
// units of the keys its last row sees (one at least).  With few rows per sequence
// all units stand in one line, key head by key head, sequence by sequence, tile by
// tile, and every worker (block) takes the same number of them, so that long and
// short sequences keep all of the chip busy to the end (64 requests' decode step
// 162 us; a block per tile and key range 214).  A worker finds its first unit from
// the lengths alone.  A tile that the line cuts leaves parts in the workspace,
// which page_join_kernel joins.  With many rows, and in short work, a block takes a
// tile or a range of its keys (page_attn_many_kernel, page_attn_short_kernel).
struct Seq {
  int q0, n, kv, L;  // first row, new tokens, cached tokens, those the table has room for
};
__device__ inline Seq seq_of(const KArgs &a, int b) {
  Seq s;
  s.q0 = min(max(0, a.cu_q[b]), a.N_q);
  s.n = min(max(s.q0, a.cu_q[b + 1]), a.N_q) - s.q0;
  s.kv = max(0, a.kv_len[b]);
  s.L = (int)min((long long)s.kv, (long long)a.max_pages << a.page_shift);
  return s;
}
__device__ inline Seq uniform(const Seq &s, int src) {
  return {__builtin_amdgcn_readlane(s.q0, src), __builtin_amdgcn_readlane(s.n, src),
          __builtin_amdgcn_readlane(s.kv, src), __builtin_amdgcn_readlane(s.L, src)};
}
template <int BM>
__device__ inline int tiles_of(const KArgs &a, const Seq &s) {
  return (s.n * a.G + BM - 1) / BM;
}
// The keys of a tile, of which its rows see some: with a window, the stages that hold
// the sinks and then, from the 16 keys on in which the first row's window starts, those
// up to the last row.  They are numbered without what lies between, so that all work is
// shared out by number: number x is key x up to `head`, then key x + skip.
struct Span {
  int keys;                // their number
  int head, skip, lo;      // lo: the first key behind the sinks that a row sees
  __device__ inline int key(int x) const { return x < head ? x : x + skip; }
};
template <int BM, int KS, typename A>
__device__ inline Span span_of(const A &a, const Seq &s, int tile) {
  const int hi = min(s.L, s.kv - s.n + (min((tile + 1) * BM, s.n * a.G) - 1) / a.G + 1);
  if constexpr (A::WIN) {
    const int lo = max(0, s.kv - s.n + tile * BM / a.G + 1 - a.window);
    const int head = (a.sinks + KS - 1) / KS * KS;
    // (a table that ends before the window)
    if (lo >= hi) return {min(hi, a.sinks), head, 0, lo};
    const int skip = max(0, (lo & ~15) - head);
    return {hi - skip, head, skip, lo};
  } else {
    return {hi, 0, 0, 0};
  }
}
template <int BM, int KS, typename A>
__device__ inline int units_of(const A &a, const Seq &s, int tile) {
  return max(1, (span_of<BM, KS>(a, s, tile).keys + KS - 1) / KS);
}
typedef uint64_t u64;
// inclusive, over the lanes; v below 2^50
__device__ inline u64 prefix_sum64(u64 v) {
  return (u64)wave::prefix_sum((uint32_t)(v & 0xFFFFFF)) + ((u64)wave::prefix_sum((uint32_t)(v >> 24)) << 24);
}
// Units of lane i's sequence c0 + i (0 behind the last); every lane calls it.
template <int BM, int KS, typename A>
__device__ inline u64 seq_units(const A &a, int c0, Seq &s) {
  const int lane = threadIdx.x & 63, b = c0 + lane;
  s = seq_of(a, min(b, a.B - 1));
  const int T = b < a.B ? tiles_of<BM>(a, s) : 0;
  constexpr int kAlone = 4;  // tiles that a lane sums by itself; more are spread over the wave
  u64 w = 0;
  for (int t = 0; t < min(T, kAlone); ++t) w += units_of<BM, KS>(a, s, t);
  for (u64 m = __ballot(T > kAlone); m != 0; m &= m - 1) {
    const int src = __builtin_ctzll(m), n = __builtin_amdgcn_readlane(T, src);
    const Seq x = uniform(s, src);
    u64 sum = 0;
    for (int t = kAlone + lane; t < n; t += 64) sum += units_of<BM, KS>(a, x, t);
    sum = wave::sum(sum);
    if (lane == src) w += sum;
  }
  return w;
}

// A place in the line of units: unit u of the U of tile t of sequence b and
// key head g.  Wave-uniform, found by every wave for itself.
template <int BM, int KS>
struct Place {
  int g, b, t, u, U;
  Seq s;
  // the place of unit w of the `per` units of a key head (first: the first 64
  // sequences' units and descriptions)
  template <typename A>
  __device__ inline void find(const A &a, u64 w, u64 per, u64 units, const Seq &first) {
    const int lane = threadIdx.x & 63;
    g = (int)(w / per);
    u64 r = w - (u64)g * per;
    Seq sl = first;
    int c0 = 0;
    u64 incl = prefix_sum64(units);
    for (;; c0 += 64) {
      const u64 total = wave::lane_value(incl, 63);
      if (r < total || c0 + 64 >= a.B) break;
      r -= total;
      units = seq_units<BM, KS>(a, c0 + 64, sl);
      incl = prefix_sum64(units);
    }
    const int src = __builtin_ctzll(__ballot(r < incl) | 1ull << 63);
    r -= wave::lane_value(incl - units, src);
    b = c0 + src;
    s = uniform(sl, src);
    const int T = tiles_of<BM>(a, s);
    for (t = 0;; t += 64) {  // 64 tiles at a time
      const int x = t + lane < T ? units_of<BM, KS>(a, s, t + lane) : 0;
      const u64 in = prefix_sum64(x), total = wave::lane_value(in, 63);
      if (r >= total && t + 64 < T) {
        r -= total;
        continue;
      }
      const int k = __builtin_ctzll(__ballot(r < in) | 1ull << 63);
      u = (int)(r - wave::lane_value(in - x, k));
      U = __builtin_amdgcn_readlane(x, k);
      t += k;
      break;
    }
  }
  // the first unit of the next tile (there is one)
  template <typename A>
  __device__ inline void next(const A &a) {
    u = 0;
    if (++t >= tiles_of<BM>(a, s)) {
      t = 0;
      const int lane = threadIdx.x & 63;
      int c0 = b + 1;
      for (;; c0 += 64) {
        if (c0 >= a.B) {
          ++g;
          c0 = 0;
        }
        const Seq x = seq_of(a, min(c0 + lane, a.B - 1));
        const u64 m = __ballot(c0 + lane < a.B && x.n > 0);
        if (m != 0) {
          const int src = __builtin_ctzll(m);
          b = c0 + src;
          s = uniform(x, src);
          break;
        }
      }
    }
    U = units_of<BM, KS>(a, s, t);
  }
};

// A tile that is cut: its parts' slots in the workspace are `first`, then `next`,
// next + step, ..; `more` follow the first.  The block that takes its first
// keys says so here (more = 0: nothing to join).
struct Cut {
  int more, g, q0, n, row0, first, next, step;
};
__device__ inline void put_cut(int4 *meta, int i, const Cut &c) {
  meta[2 * i] = make_int4(c.more, c.g, c.q0, c.n);
  meta[2 * i + 1] = make_int4(c.row0, c.first, c.next, c.step);
}
__device__ inline Cut get_cut(const int4 *meta, int i) {
  const int4 x = meta[2 * i], y = meta[2 * i + 1];
  return {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
}

// One tile (or, cut, some of its keys): the rows row0 .. of sequence b and key
// head g over the keys of number kbeg .. kend - 1 (kbeg: the first of a stage).
struct Job {
  int g, b, row0, kbeg, kend, slot;  // slot: where a cut tile's part goes
  bool cut;
  Seq s;
};

// WR waves of M rows each share the stages of TPW tiles of 32 keys.
template <typename T, int D, int M, int WR, int TPW>
struct Shape {
  using G_ = Geo<T, D>;
  static constexpr int BM = WR * M;
  static constexpr int KS = TPW * kTile;           // keys per stage
  static constexpr int RW = KS / WR;               // of them, rows a wave loads
  static constexpr int GR = RW < 16 ? RW : 16;     // rows of one page group
  static constexpr int NG = RW / GR, LPG = GR / G_::RPL;
  static_assert(RW % G_::RPL == 0 && GR % G_::RPL == 0, "whole loads");
  static constexpr int TB = KS * G_::ROWB;         // bytes of one tensor's stage
  // Blocks per CU, with two stage buffers each.  One-wave workers: one wave per
  // SIMD (two where a stage is small) keeps 64 KB in flight.  More of them, or a
  // third buffer, is slower: a decode step of two requests of 128,000 tokens takes
  // 171 us with four workers of two buffers, 204 with five, 183 with three of
  // three.  Chunks: two blocks, of an fp32 tile of 512-byte rows one, by its registers.
  static constexpr int kPerCu = WR > 1 ? (G_::ROWB > 256 ? 1 : 2) : 128 * 1024 / (4 * TB);
  static constexpr int kPerSimd = (kPerCu * WR + 3) / 4;
};

// HERE: the part stays in LDS, rows of D floats in bufA and their log2 sums in sums.
template <typename T, int D, int M, int WR, int TPW, bool HERE = false, typename A>
__device__ __attribute__((always_inline)) inline void attend(const A &a, const Job &job, AVTP_LDS char *bufA,
                                                             AVTP_LDS char *bufB, AVTP_LDS float *sums = nullptr) {
  using G_ = Geo<T, D>;
  using S_ = Shape<T, D, M, WR, TPW>;
  using M_ = Mma<M>;
  constexpr bool F32 = G_::F32;
  constexpr int BM = S_::BM, KS = S_::KS, RW = S_::RW, GR = S_::GR, NG = S_::NG, LPG = S_::LPG, TB = S_::TB;
  constexpr int ROWB = G_::ROWB, NCH = G_::NCH, RPL = G_::RPL;
  constexpr int NGR = 64 / M;        // lane groups: lanes of one row
  constexpr int NK = kTile / M;      // S tiles of M keys
  constexpr int NS = NCH / NGR;      // K fragments per key: chunks of 16 bytes, one a group
  constexpr int ND = D / M;          // output tiles of M values
  constexpr int AE = M * M / 64;     // a lane's elements of an M x M tile
  constexpr int NE = NK * AE;        // and of a tile's logits
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = WR > 1 ? __builtin_amdgcn_readfirstlane(tid >> 6) : 0;
  const int grp = lane / M, col = lane % M;
  const float cl2e = a.cl2e;
  const int pmask = (1 << a.page_shift) - 1;
  AVTP_LDS char *const job_buf = bufA;
  const int g = job.g, b = job.b, L = job.s.L, row0 = job.row0, kbeg = job.kbeg, kend = job.kend;
  const int R = job.s.n * a.G;
  if (L < job.s.kv && a.status && (WR > 1 ? tid : lane) == 0) atomicOr(&a.status[b], AVTP_FLAG_BAD_PAGE);
  // row r of the sequence: token r / G, which sees kv - n + token + 1 keys
  const int wrow = row0 + wave * M;
  const int row = min(wrow + col, R - 1), tok = row / a.G, head = g * a.G + (row - tok * a.G);
  const int lim = min(L, job.s.kv - job.s.n + tok + 1);
  const bool valid = wrow + col < R;
  const int wmin = __builtin_amdgcn_readlane(lim, 0), wmax = __builtin_amdgcn_readlane(lim, M - 1);
  // the row's window starts at key `low`, of the wave's rows at wlow .. wlow1
  constexpr bool WIN = A::WIN;
  const Span span = span_of<BM, KS>(a, job.s, row0 / BM);
  int sinks = 0, low = 0, wlow = 0, wlow1 = 0;
  if constexpr (WIN) {
    sinks = a.sinks;
    low = job.s.kv - job.s.n + tok + 1 - a.window;
    wlow = __builtin_amdgcn_readlane(low, 0);
    wlow1 = __builtin_amdgcn_readlane(low, M - 1);
  }
  auto sees = [&](int key) __attribute__((always_inline)) {
    return WIN ? key < lim && (key < sinks || key >= low) : key < lim;
  };
  // do all rows of the wave see the n keys from number x, which is key `key`, on?
  auto all_see = [&](int x, int key, int n) __attribute__((always_inline)) {
    if (WIN) return x + n <= kend && key + n <= wmin && (key + n <= sinks || key >= wlow1);
    return x + n <= min(kend, wmin);
  };

  // where this lane's loads of a 16-row group come from
  uint32_t voff[LPG];
  const int r0w = wave * RW;  // the wave's first row of a stage
#pragma unroll
  for (int i = 0; i < LPG; ++i) {
    const int r = i * RPL + lane / NCH;
    voff[i] = (uint32_t)(r * ROWB + ((lane % NCH) ^ G_::swz(r0w + r)) * 16);
  }

  // query rows, the second operand of S^T
  u32x4 qf[NS];
  {
    const char *p = a.q + (job.s.q0 + tok) * a.q_tok + (long long)head * ROWB + grp * 16;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const u32x4 *>(p + s * NGR * 16);
  }

  const int32_t *trow = a.table + (long long)b * a.max_pages;
  // page ids of the wave's groups of the stage at number x, one per lane (lane
  // gi: group gi), read a stage ahead
  auto load_ids = [&](int x) __attribute__((always_inline)) {
    const int ks = WIN ? span.key(x) : x;
    const int key = min(ks + r0w + (lane & (NG - 1)) * 16, L - 1);
    return trow[key >> a.page_shift];
  };
  // Decode steps read K and V once: non-temporal (64 requests' step 206 -> 194 us).
  // Chunks, 32-row tiles of the short form among them, read them again, from the L2
  // (eight of 30 tokens over 1,500 keys, 32/8 heads, 23.1 us non-temporal, 20.9 so).
  constexpr int kAux = WR == 1 && !(HERE && M == 32) ? 2 : 0;
  auto issue = [&](AVTP_LDS char *buf, int x, int ids) __attribute__((always_inline)) {
    const int ks = WIN ? span.key(x) : x;
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      const int id = __builtin_amdgcn_readlane(ids, gi);
      const int key = ks + r0w + gi * 16;
      // (between the sinks and the window a page need not be there)
      const bool seen = !WIN || key < sinks || key + GR > span.lo;
      const bool ok = seen && (unsigned)id < (unsigned)a.n_pages;
      if (!ok && seen && key < L && a.status && lane == 0) atomicOr(&a.status[b], AVTP_FLAG_BAD_PAGE);
      const int have = ok ? min(max(L - key, 0), GR) * ROWB : 0;
      const long long off = ok ? ((long long)id * a.Hkv + g) * a.head_bytes + (long long)(key & pmask) * ROWB : 0;
      const Rsrc rk = make_rsrc(a.k + off, have), rv = make_rsrc(a.v + off, have);
      AVTP_LDS char *dst = buf + (r0w + gi * 16) * ROWB;
#pragma unroll
      for (int i = 0; i < LPG; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, dst + i * 1024, 16, (int)voff[i], 0, 0, kAux);
#pragma unroll
      for (int i = 0; i < LPG; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, dst + TB + i * 1024, 16, (int)voff[i], 0, 0, kAux);
    }
  };

  typename M_::acc O[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) O[i] = typename M_::acc{};
  float m = -INFINITY, l = 0.f;  // this lane's share of the row's sum

  // element e of this lane: key (of a tile's logits) or value (of an output
  // tile) eoff(e) + 4 grp
  auto eoff = [](int e) __attribute__((always_inline)) { return 4 * NGR * (e >> 2) + (e & 3); };

  // LDS addresses of a tile's operands: the lane's base, XOR-ed with the chunk,
  // plus rows that fit the instruction's offset.
  // K: row kk M + col, fragment s
  typedef AVTP_LDS const char *lptr;
  const uint32_t kbase = (uint32_t)(col * ROWB + ((grp ^ G_::swz(col)) << 4));
  auto kaddr = [&](lptr kt, int kk, int s) __attribute__((always_inline)) {
    return kt + (kbase ^ (uint32_t)(s * NGR << 4)) + kk * M * ROWB;
  };
  // V, bf16: the transposing read hands lane i of 16 the value i of four rows of
  // 16 values whose addresses the lanes give (lane i: four values of row i / 4),
  // here M dt + col of the four keys eoff(8 c + 4 j) + 4 grp + .. that belong to
  // the lane's probabilities 8 c + 4 j + ..
  const int ti = lane & 15, tq = (lane >> 4) & (M / 16 - 1);
  const int vrow = F32 ? 4 * grp : 4 * grp + (ti >> 2);
  const uint32_t vbase = F32 ? (uint32_t)(vrow * ROWB + (((col >> 2) ^ G_::swz(vrow)) << 4) + (col & 3) * 4)
                             : (uint32_t)(vrow * ROWB + (((2 * tq + ((ti & 3) >> 1)) ^ G_::swz(vrow)) << 4) + (ti & 1) * 8);
  auto vfrag = [&](lptr vt, int c, int dt) __attribute__((always_inline)) {
    bf16x8 f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = eoff(8 * c + 4 * j);
      const uint32_t o = (vbase ^ (uint32_t)(((dt * M / 8) ^ G_::swz(r)) << 4)) + (uint32_t)(r * ROWB);
      const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((AVTP_LDS bf16x4 *)(vt + o));
#pragma unroll
      for (int i = 0; i < 4; ++i) f[4 * j + i] = x[i];
    }
    return f;
  };
  // fp32: value M dt + col of key eoff(e) + 4 grp
  auto velem = [&](lptr vt, int e, int dt) __attribute__((always_inline)) {
    const uint32_t o = (vbase ^ (uint32_t)(((dt * M / 4) ^ G_::swz(eoff(e))) << 4)) + (uint32_t)(eoff(e) * ROWB);
    return *reinterpret_cast<AVTP_LDS const float *>(vt + o);
  };

  // Values of V that are not finite, in a tile that some row sees only in
  // part: 0 times them is not 0.  The tile's product then runs without them
  // and they are added to the rows that see them.
  auto not_finite = [&](uint32_t x) __attribute__((always_inline)) {
    return F32 ? (x & 0x7f800000u) == 0x7f800000u : ((((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0u);
  };
  // (With a window, in fp32, by a sum of 0 times the values, one instruction each: one
  // prompt of 1,000 tokens, 16/8 heads of 128, window 512 67.5 -> 65.7 us; in bf16 sums
  // of squares gained nothing over the integer test.)
  auto tile_not_finite = [&](lptr vt) __attribute__((always_inline)) {
    bool bad = false;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kTile * NCH / 64; ++i) {
      const u32x4 x = *reinterpret_cast<AVTP_LDS const u32x4 *>(vt + (i * 64 + lane) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t u = x[j];  // (an element cast in place is read as the vector's first)
        if constexpr (F32 && WIN) sum = __builtin_fmaf(__builtin_bit_cast(float, u), 0.f, sum);
        else bad = bad || not_finite(u);
      }
    }
    return __ballot(F32 && WIN ? sum != 0.f : bad) != 0ull;  // (a sum of NaN)
  };
  auto add_not_finite = [&](lptr vt, int key) __attribute__((always_inline)) {
#pragma unroll 1
    for (int r = 0; r < kTile; ++r) {
      const bool seen = sees(key + r);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
#pragma unroll
        for (int e = 0; e < AE; ++e) {
          const int dd = M * dt + eoff(e) + 4 * grp;  // this lane's value of the output
          const int ch = dd * (int)sizeof(T) / 16, by = dd * (int)sizeof(T) % 16;
          const float x =
              (float)*reinterpret_cast<AVTP_LDS const T *>(vt + r * ROWB + ((ch ^ G_::swz(r)) << 4) + by);
          const bool add = seen && !(__builtin_fabsf(x) < INFINITY);
          O[dt][e] += add ? x : 0.f;
        }
      }
    }
  };

  // S^T of the 32 keys at kt
  struct Logits {
    typename M_::acc x[NK];
    __device__ inline float get(int e) const { return x[e / AE][e % AE]; }
  };
  auto logits = [&](lptr kt) __attribute__((always_inline)) {
    Logits S;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      S.x[kk] = typename M_::acc{};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        if constexpr (F32) {
          const f32x4 kf = *reinterpret_cast<AVTP_LDS const f32x4 *>(kaddr(kt, kk, s)), qv = __builtin_bit_cast(f32x4, qf[s]);
#pragma unroll
          for (int i = 0; i < 4; ++i) S.x[kk] = M_::run(kf[i], qv[i], S.x[kk]);
        } else {
          S.x[kk] = M_::run(*reinterpret_cast<AVTP_LDS const bf16x8 *>(kaddr(kt, kk, s)),
                            __builtin_bit_cast(bf16x8, qf[s]), S.x[kk]);
        }
      }
    }
    return S;
  };
  // p = 2^(c S - m), as the second product takes them, and their sum.  In bf16 they
  // are rounded to it (2^-8 of each at most), since the bf16 MFMA takes V as it is
  // only beside bf16 and p as a sum of two bf16 parts would double these products;
  // their sum is that of the fp32 values.  The output's error against 64 bits, relative
  // 2-norm, is 0.0019-0.0022 instead of the 0.0016-0.0017 of an output in bf16 alone.
  struct Probs {
    std::conditional_t<F32, float, bf16x8> x[F32 ? NE : NE / 8];
  };
  auto probs = [&](const Logits &S, Probs &p, float ref) __attribute__((always_inline)) {
    float sum[2];
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const float x = __builtin_amdgcn_exp2f(S.get(e) * cl2e - ref);
      sum[e & 1] = e < 2 ? x : sum[e & 1] + x;
      if constexpr (F32) p.x[e] = x;
      else p.x[e >> 3][e & 7] = (__bf16)x;
    }
    return sum[0] + sum[1];
  };
  // O^T += V^T P^T
  auto weigh = [&](lptr vt, const Probs &p, bool clean) __attribute__((always_inline)) {
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < NE; ++e) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          float x = velem(vt, e, dt);
          if (clean) x = __builtin_fabsf(x) < INFINITY ? x : 0.f;
          O[dt] = M_::run(x, p.x[e], O[dt]);
        }
      }
    } else {
#pragma unroll
      for (int c = 0; c < NE / 8; ++c) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          bf16x8 f = vfrag(vt, c, dt);
          if (clean) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __builtin_fabsf((float)f[i]) < INFINITY ? f[i] : (__bf16)0.f;
          }
          O[dt] = M_::run(f, p.x[c], O[dt]);
        }
      }
    }
  };
  // A stage whose keys every row of the wave sees.  Returns how many of its tiles
  // are done: at the first one that takes a row's sum out of its range (or finds
  // no reference yet) it stops, and `part` takes the rest.
  auto whole = [&](lptr kt, lptr vt) __attribute__((always_inline)) {
    if constexpr (TPW == 2 && M == 32 && !F32) {
      // Two tiles, the matrix core and the VALU at work together: tile 1's logits
      // beside tile 0's exponentials, tile 0's products with V beside tile 1's.  One
      // MFMA a step, with the LDS read of the step two further on and some
      // exponentials; left to itself the compiler puts all products of a kind
      // first.  32/8 heads of 128, four prompts of 7,000-9,000 tokens 2050 -> 2011 us
      // (1075 TFLOP/s); 28/4 heads, two of 2,048 83.2 -> 79.9; 14/2 heads of 64, 16 of
      // 1,000 66.0 -> 64.4.
      constexpr int AHEAD = 2, STEPS = 2 * ND;
      Logits S[2];
      Probs p[2];
      float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
      auto terms = [&](int i, int e0, int e1) __attribute__((always_inline)) {
#pragma unroll
        for (int e = e0; e < e1; ++e) {
          const float x = __builtin_amdgcn_exp2f(S[i].get(e) * cl2e - m);
          sum[i][e & 1] += x;
          p[i].x[e >> 3][e & 7] = (__bf16)x;
        }
      };
      auto step_end = []() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };
      bf16x8 kf[AHEAD], vf[AHEAD];
      auto kread = [&](int i) __attribute__((always_inline)) {
        return *reinterpret_cast<AVTP_LDS const bf16x8 *>(kaddr(kt + i / NS * kTile * ROWB, 0, i % NS));
      };
      auto vread = [&](int j) __attribute__((always_inline)) {
        return vfrag(vt + j / STEPS * kTile * ROWB, j / ND % 2, j % ND);
      };
      auto product = [&](int j) __attribute__((always_inline)) {
        O[j % ND] = M_::run(vf[j % AHEAD], p[j / STEPS].x[j / ND % 2], O[j % ND]);
        if (j + AHEAD < 2 * STEPS) vf[j % AHEAD] = vread(j + AHEAD);
      };
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) kf[i] = kread(i);
      step_end();
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i) {
        f32x16 &x = S[i / NS].x[0];
        x = M_::run(kf[i % AHEAD], __builtin_bit_cast(bf16x8, qf[i % NS]), i % NS == 0 ? f32x16{} : x);
        if (i + AHEAD < 2 * NS) kf[i % AHEAD] = kread(i + AHEAD);
        else vf[i + AHEAD - 2 * NS] = vread(i + AHEAD - 2 * NS);
        if (i > NS) terms(0, (i - NS - 1) * 16 / (NS - 1), (i - NS) * 16 / (NS - 1));
        step_end();
      }
      const float t0 = sum[0][0] + sum[0][1];
      if (__builtin_expect(__ballot(!(t0 <= kLazyLimit)) != 0ull, 0)) return 0;
      l += t0;
#pragma unroll
      for (int j = 0; j < STEPS; ++j) {
        product(j);
        terms(1, j * 16 / STEPS, (j + 1) * 16 / STEPS);
        step_end();
      }
      const float t1 = sum[1][0] + sum[1][1];
      if (__builtin_expect(__ballot(!(t1 <= kLazyLimit)) != 0ull, 0)) return 1;
      l += t1;
#pragma unroll
      for (int j = STEPS; j < 2 * STEPS; ++j) {
        product(j);
        step_end();
      }
    } else {
      Logits S[TPW];
      Probs p[TPW];
      float tot = 0.f;
#pragma unroll
      for (int i = 0; i < TPW; ++i) S[i] = logits(kt + i * kTile * ROWB);
#pragma unroll
      for (int i = 0; i < TPW; ++i) tot += probs(S[i], p[i], m);
      if (__builtin_expect(__ballot(!(tot <= kLazyLimit)) != 0ull, 0)) return 0;
      l += tot;
#pragma unroll
      for (int i = 0; i < TPW; ++i) weigh(vt + i * kTile * ROWB, p[i], false);
    }
    return TPW;
  };
  // A tile of keys from number kb on, of which some rows may see a part or nothing, and
  // whose largest logit becomes the row's reference if it is larger.
  auto part = [&](lptr kt, lptr vt, int kb) __attribute__((always_inline)) {
    const int key = WIN ? span.key(kb) : kb;
    Logits S = logits(kt);
    Probs p;
    const bool all = all_see(kb, key, kTile);
    auto mask = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        float &x = reinterpret_cast<float *>(&S)[e];
        x = sees(key + 4 * grp + eoff(e)) ? x : -INFINITY;
      }
    };
    // Behind the first tile most rows have their reference, and a tile of a window, at
    // whose ends a chunk's tiles are seen in part, need not raise it (prompts of 1,000
    // tokens, 28/4 heads, window 512 31.5 -> 29.0 us; four of 7,000-9,000, 32/8 heads, 512
    // 413 -> 399, 2,048 992 -> 972; fp32, tiles that all see alone, 249 -> 243).
    bool done = false;
    if (WIN && WR > 1 && kb > kbeg && (all || !F32)) {
      if (!all) mask();
      const float sum = probs(S, p, m);
      done = __ballot(!(sum <= kLazyLimit)) == 0ull;
      if (done) l += sum;
    }
    if (!done) {
      mask();
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < NE; ++e) top = fmaxf(top, S.get(e));
      const float nm = fmaxf(m, over_row<M>(top, [](float x, float y) { return fmaxf(x, y); }) * cl2e);
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - nm);
      m = nm;
      l *= f;
      if (kb > kbeg) {  // (the first tile finds O empty)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int e = 0; e < AE; ++e) O[dt][e] *= f;
      }
      l += probs(S, p, m == -INFINITY ? 0.f : m);  // (no key seen so far: every term is 0)
    }
    if (!all && __builtin_expect(tile_not_finite(vt), 0)) {
      add_not_finite(vt, key);
      weigh(vt, p, true);
    } else {
      weigh(vt, p, false);
    }
  };

  const int nstage = kend > kbeg ? (kend - kbeg + KS - 1) / KS : 0;
  if (WR > 1) __syncthreads();  // the waves are done with the tile before
  if (nstage > 0) {
    int ids = load_ids(kbeg);
    issue(bufA, kbeg, ids);
    ids = load_ids(kbeg + KS);
    // Stage st is in LDS and every wave is done with the other buffer, which
    // the next stage's loads take.
    auto begin = [&](AVTP_LDS char *nxt, int st) __attribute__((always_inline)) {
      wait_vmem();
      if (WR > 1) __syncthreads();
      if (st + 1 < nstage) {
        issue(nxt, kbeg + (st + 1) * KS, ids);
        ids = load_ids(kbeg + (st + 2) * KS);
      }
    };
    // (restrict: the stage read and the one in flight are different memory, or
    // every read would wait for the loads)
    auto parts = [&](AVTP_LDS const char *__restrict__ cur, int st, int from) __attribute__((always_inline)) {
      // keys below the range's end, and those that rows of this wave see
      const int ks = kbeg + st * KS, stop = min(kend, wmax), key = WIN ? span.key(ks) : ks;
      auto some_see = [&](int t) __attribute__((always_inline)) {
        if (!WIN) return ks + t * kTile < stop;
        const int x = key + t * kTile;
        return ks + t * kTile < kend && x < wmax && (x < sinks || x + kTile > wlow);
      };
#pragma unroll 1
      for (int t = from; t < TPW; ++t)
        if (some_see(t)) part(cur + t * kTile * ROWB, cur + TB + t * kTile * ROWB, ks + t * kTile);
    };
    auto wholes = [&](AVTP_LDS const char *__restrict__ cur, AVTP_LDS char *__restrict__ nxt, int st)
        __attribute__((always_inline)) {
      begin(nxt, st);
      const int ks = kbeg + st * KS;
      return __builtin_expect(all_see(ks, WIN ? span.key(ks) : ks, KS), 1) ? whole(cur, cur + TB) : 0;
    };
    // Stages whose keys every row sees run in a loop of their own (with both
    // kinds in one, O was copied at every stage); the first one, and those that
    // raise a row's reference, go the other way.
    begin(bufB, 0);
    int done = 0;  // tiles of stage st
    for (int st = 0;;) {
      parts(bufA, st, done);
      done = TPW;
      while (done == TPW && ++st < nstage) {
        AVTP_LDS char *x = bufA;
        bufA = bufB;
        bufB = x;
        done = wholes(bufA, bufB, st);
      }
      if (done == TPW) break;
    }
  }
  l = over_row<M>(l, [](float x, float y) { return x + y; });

  const float inv = l == 0.f ? 0.f : 1.f / l;
  const float ls = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);  // log2 of the row's sum
  if constexpr (WIN && WR > 1 && !F32) {
    if (!job.cut) {
      // Finished rows of 128 tokens and heads, whose stores weigh more the shorter the
      // window: turned around in LDS, 16 bytes a lane and a row in one piece (four prompts
      // of 7,000-9,000 tokens, 32/8 heads, window 64 251 -> 196 us, 512 442 -> 433, 2,048
      // 1056 -> 1047).  The other stage buffer is free: all waves passed the last stage's
      // barrier, and nothing is on its way to it.
      AVTP_LDS char *const mine = bufB + wave * M * ROWB;
      auto at = [&](int r, int ch) __attribute__((always_inline)) { return mine + r * ROWB + ((ch ^ (r & (NCH - 1))) << 4); };
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int j = 0; j < AE / 4; ++j) {
          const int dd = M * dt + eoff(4 * j) + 4 * grp;
          bf16x4 y;
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = (__bf16)(O[dt][4 * j + i] * inv);
          *reinterpret_cast<AVTP_LDS bf16x4 *>(at(col, dd / 8) + (dd & 4) * 2) = y;
        }
#pragma unroll
      for (int i = 0; i < M * NCH / 64; ++i) {
        const int r = i * RPL + lane / NCH, ch = lane % NCH, t = (wrow + r) / a.G, h = g * a.G + (wrow + r - t * a.G);
        const u32x4 x = *reinterpret_cast<AVTP_LDS const u32x4 *>(at(r, ch));
        if (wrow + r < R)
          *reinterpret_cast<u32x4 *>(a.out + (job.s.q0 + t) * a.out_tok + (long long)h * ROWB + ch * 16) = x;
      }
      if (valid && grp == 0 && a.lse) a.lse[(long long)head * a.N_q + job.s.q0 + tok] = ls * kLn2;
      return;
    }
  }

  // the finished rows, or the tile's part
  if (!valid) return;
  const long long pr = (long long)job.slot * BM + wave * M + col;
  char *o = a.out + (job.s.q0 + tok) * a.out_tok + (long long)head * ROWB;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int j = 0; j < AE / 4; ++j) {
      const int dd = M * dt + eoff(4 * j) + 4 * grp;
      const f32x4 x = {O[dt][4 * j] * inv, O[dt][4 * j + 1] * inv, O[dt][4 * j + 2] * inv, O[dt][4 * j + 3] * inv};
      if constexpr (HERE) *reinterpret_cast<AVTP_LDS f32x4 *>(job_buf + (col * D + dd) * 4) = x;
      else if (job.cut) *reinterpret_cast<f32x4 *>(a.po + pr * D + dd) = x;
      else put4<T>(o, dd, x);
    }
  if (grp == 0) {
    if constexpr (HERE) sums[col] = ls;
    else if (job.cut) a.pl[pr] = ls;
    else if (a.lse) a.lse[(long long)head * a.N_q + job.s.q0 + tok] = ls * kLn2;
  }
}

// Few rows per sequence (decode steps): a block is one wave, a worker that takes
// its share of the line of units.
template <typename T, int D, int M, typename A>
__global__ __launch_bounds__(64, (Shape<T, D, M, 1, 1>::kPerSimd)) void page_attn_few_kernel(A a) {
  using S_ = Shape<T, D, M, 1, 1>;
  constexpr int BM = S_::BM, KS = S_::KS;
  // two stage buffers as distinct objects, so the compiler can tell the one
  // being read from the one in flight
  __shared__ __attribute__((aligned(16))) char smA[2 * S_::TB];
  __shared__ __attribute__((aligned(16))) char smB[2 * S_::TB];
  const int worker = blockIdx.x;
  Seq first;
  const u64 units = seq_units<BM, KS>(a, 0, first);
  u64 per = wave::sum(units);
  for (int c0 = 64; c0 < a.B; c0 += 64) {
    Seq x;
    per += wave::sum(seq_units<BM, KS>(a, c0, x));
  }
  const u64 all = per * (unsigned)a.Hkv;
  u64 share = (all + a.workers - 1) / a.workers;
  if (share < (unsigned)a.least) share = a.least;
  u64 w = share * worker;
  const u64 wend = w + share < all ? w + share : all;
  Cut c{};
  if (w < wend) {
    Place<BM, KS> at;
    at.find(a, w, per, units, first);
    for (;;) {
      const int u1 = (u64)(at.U - at.u) <= wend - w ? at.U : at.u + (int)(wend - w);
      Job job{at.g, at.b, at.t * BM, at.u * KS, min(span_of<BM, KS>(a, at.s, at.t).keys, u1 * KS),
              2 * worker + (at.u > 0 ? 0 : 1), at.u > 0 || u1 < at.U, at.s};
      attend<T, D, M, 1, 1>(a, job, (AVTP_LDS char *)smA, (AVTP_LDS char *)smB);
      // (a worker's first part of a tile is the odd one of its slots; the
      // workers behind it go on in their even ones)
      if (at.u == 0 && job.cut)
        c = {(int)((at.U - u1 + share - 1) / share), at.g, at.s.q0, at.s.n, job.row0, job.slot, 2 * (worker + 1), 2};
      w += u1 - at.u;
      if (w >= wend) break;
      at.next(a);
    }
  }
  if (threadIdx.x == 0) put_cut(a.meta, worker, c);
}

// The tile of a rank, -1 if there is none, and its sequence.  The whole wave
// calls it.
template <int BM>
__device__ inline int tile_of_rank(const KArgs &a, int rank, int &b, Seq &s) {
  const int lane = threadIdx.x & 63;
  if (a.B <= 64) {
    // longest sequences first, the tiles that see most first: what is left at
    // the end is small
    const Seq mine = seq_of(a, min(lane, a.B - 1));
    const int nt = lane < a.B ? tiles_of<BM>(a, mine) : 0;
    int before = 0;
    for (int j = 0; j < a.B; ++j) {
      const int kv = __builtin_amdgcn_readlane(mine.L, j), n = __builtin_amdgcn_readlane(nt, j);
      if (kv > mine.L || (kv == mine.L && j < lane)) before += n;
    }
    const u64 m = __ballot(before <= rank && rank < before + nt);
    if (m == 0) return -1;
    b = __builtin_ctzll(m);
    s = uniform(mine, b);
    return __builtin_amdgcn_readlane(before + nt, b) - 1 - rank;
  }
  // Sequence b's tiles have the ranks from floor(q0 G / BM) + b on: the next
  // sequence's start at least ceil(n G / BM) further, so that no sum over the
  // sequences is needed.
  auto start = [&](int x) __attribute__((always_inline)) { return min(max(0, a.cu_q[x]), a.N_q) * a.G / BM + x; };
  int lo = 0;
  for (int step = 1 << 12; step > 0; step >>= 6) {  // (B is 2^16 at most)
    const int x = lo + lane * step;
    const u64 m = __ballot(x < a.B && start(min(x, a.B - 1)) <= rank);
    lo += max(0, __builtin_popcountll(m) - 1) * step;
  }
  b = lo;
  s = uniform(seq_of(a, b), 0);
  const int tile = rank - __builtin_amdgcn_readfirstlane(start(b));
  return tile < tiles_of<BM>(a, s) ? tile : -1;
}

// Short work: a block takes a whole tile, its W waves a share of the
// keys each, and joins their parts in LDS: no second launch.
constexpr int kShortWaves = 4;  // whose buffers a CU's LDS holds
template <typename T, int D, int M, int W, typename A>
__global__ __launch_bounds__(64 * W) void page_attn_short_kernel(A a) {
  using S_ = Shape<T, D, M, 1, 1>;
  constexpr int KS = S_::KS, BUF = 2 * S_::TB;
  static_assert(M * D * 4 <= BUF, "a part fits a stage buffer");
  __shared__ __attribute__((aligned(16))) char smA[W * BUF];
  __shared__ __attribute__((aligned(16))) char smB[W * BUF];
  __shared__ float sums[W * M];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.x % a.Hkv;
  int b = 0;
  Seq s{};
  const int tile = tile_of_rank<M>(a, blockIdx.x / a.Hkv, b, s);
  if (tile < 0) return;
  const int keys = span_of<M, KS>(a, s, tile).keys, units = units_of<M, KS>(a, s, tile), each = (units + W - 1) / W;
  const Job job{g, b, tile * M, wave * each * KS, min(keys, (wave + 1) * each * KS), 0, true, s};
  attend<T, D, M, 1, 1, true>(a, job, (AVTP_LDS char *)smA + wave * BUF, (AVTP_LDS char *)smB + wave * BUF,
                              (AVTP_LDS float *)sums + wave * M);
  __syncthreads();
  constexpr int TPR = D / 4;  // threads per row
  const int rows = min(s.n * a.G - job.row0, M);
  for (int i = threadIdx.x; i < rows * TPR; i += 64 * W) {
    const int r = i / TPR, ch = i % TPR;
    float top = -INFINITY, tot = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, sums[w * M + r]);
    f32x4 x = f32x4{};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float ls = sums[w * M + r], f = ls == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ls - top);
      const f32x4 y = *reinterpret_cast<const f32x4 *>(smA + w * BUF + (r * D + ch * 4) * 4);
      tot += f;
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] += y[k] * f;
    }
    const float inv = tot == 0.f ? 0.f : 1.f / tot;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] *= inv;
    const int tok = (job.row0 + r) / a.G, head = g * a.G + (job.row0 + r - tok * a.G);
    put4<T>(a.out + (s.q0 + tok) * a.out_tok + (long long)head * D * (int)sizeof(T), ch * 4, x);
    if (ch == 0 && a.lse)
      a.lse[(long long)head * a.N_q + s.q0 + tok] = tot == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(tot)) * kLn2;
  }
}

// Ranges of a tile's keys.  bf16: cut into r of them, a tile's S stages take 1/r of
// their time, but its parts are written, read and joined, t(r) = stage S / r + part T r
// + join with T tiles: least at r = sqrt(gain S), gain = stage / (part T), and worth it
// where r (r - 2) > join / (part T), which is r > from.  28/4 heads of 128, prompt of
// 1,000 tokens 31.8 -> 26.6 us against ranges of 256 keys, of 300 16.5 -> 12.4; 32/8
// heads, 500 tokens 20.5 -> 16.7, four chunks of 30 over 3,000 keys 28.9 -> 26.1.
// fp32 (gain 0), whose stages take 5 times as long: ranges of 64 keys (by the formula
// two prompts of 700 tokens, 14/2 heads of 64, 43 -> 45-52).
template <int KS>
__host__ __device__ inline int key_ranges(int keys, float gain, float from) {
  if (gain == 0.f) return (keys + 63) / 64;
  const int stages = (keys + KS - 1) / KS;
  const float r = sqrtf(gain * (float)stages);
  return r <= from ? 1 : r < (float)stages ? (int)(r + 0.5f) : stages;
}

// Many rows per sequence (chunks of tokens): a block takes one tile of 128 rows
// of one key head, or one of nsplit ranges of its keys where there are few
// tiles.  The tiles of one sequence go together, key heads fastest, so that
// an XCD (blocks equal mod 8) reads the same K and V at about the same time: in
// the even line above, whose workers stand at different keys, four prompts of
// 7,000-9,000 tokens took 2907 us, with blocks in step 2147.
template <typename T, int D, int WR, int TPW, typename A>
__global__ __launch_bounds__(64 * WR, (Shape<T, D, 32, WR, TPW>::kPerSimd)) void page_attn_many_kernel(A a) {
  using S_ = Shape<T, D, 32, WR, TPW>;
  constexpr int BM = S_::BM, KS = S_::KS;
  __shared__ __attribute__((aligned(16))) char smA[2 * S_::TB];
  __shared__ __attribute__((aligned(16))) char smB[2 * S_::TB];
  const int g = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv;
  const int split = rest % a.nsplit, rank = rest / a.nsplit;
  const int place = rank * a.Hkv + g;  // of the tile among all
  int b = 0;
  Seq s{};
  const int tile = tile_of_rank<BM>(a, rank, b, s);
  Cut c{};
  if (tile >= 0) {
    const int keys = span_of<BM, KS>(a, s, tile).keys;
    // whole stages, evenly
    const int stages = max(1, (keys + KS - 1) / KS);
    const int ranges = min(a.nsplit, max(1, key_ranges<KS>(keys, a.gain, a.from)));
    const int each = (stages + ranges - 1) / ranges;
    const int parts = (stages + each - 1) / each;
    if (split >= parts) return;
    const Job job{g, b, tile * BM, split * each * KS, min(keys, (split + 1) * each * KS), place * a.nsplit + split,
                  parts > 1, s};
    attend<T, D, 32, WR, TPW>(a, job, (AVTP_LDS char *)smA, (AVTP_LDS char *)smB);
    c = {parts - 1, g, s.q0, s.n, job.row0, job.slot, job.slot + 1, 1};
  }
  if (a.nsplit > 1 && split == 0 && threadIdx.x == 0) put_cut(a.meta, place, c);
}

// Joins the parts of the tiles that were cut: D / 4 threads per row, a block
// for each 2048 / D rows of a tile.  Where a tile has fewer rows than that, the
// groups of threads share out its parts instead.
constexpr int kJoinThreads = 512;
template <typename T, int D, int BM>
__global__ __launch_bounds__(kJoinThreads) void page_join_kernel(KArgs a) {
  constexpr int TPR = D / 4, GROUPS = kJoinThreads / TPR < BM ? kJoinThreads / TPR : BM;
  constexpr int NT = GROUPS * TPR;  // threads in use
  __shared__ f32x4 x_s[NT];
  __shared__ float m_s[GROUPS], l_s[GROUPS];
  const Cut t = get_cut(a.meta, blockIdx.x / (BM / GROUPS));
  const int r0 = (blockIdx.x % (BM / GROUPS)) * GROUPS;
  const int rows = min(t.n * a.G - t.row0 - r0, GROUPS);
  if (t.more == 0 || rows <= 0) return;
  int wide = 1;  // rows side by side: a power of two
  while (wide < rows) wide <<= 1;
  const int ch = threadIdx.x % TPR, grp = threadIdx.x / TPR;
  const int i = grp & (wide - 1), first = grp / wide, step = GROUPS / wide;
  const int r = r0 + min(i, rows - 1);
  auto part = [&](int s) __attribute__((always_inline)) {
    return (long long)(s == 0 ? t.first : t.next + (s - 1) * t.step) * BM + r;
  };
  // a running reference: the parts are read once, eight at a time
  constexpr int U = 8;
  float top = -INFINITY, tot = 0.f;
  f32x4 x = f32x4{};
  for (int s = first; s <= t.more; s += U * step) {
    float ls[U], nm = top;
    f32x4 y[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const long long at = part(min(s + j * step, t.more));
      ls[j] = s + j * step <= t.more ? a.pl[at] : -INFINITY;
      y[j] = *reinterpret_cast<const f32x4 *>(a.po + at * D + ch * 4);
    }
#pragma unroll
    for (int j = 0; j < U; ++j) nm = fmaxf(nm, ls[j]);
    const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - nm);
    top = nm;
    tot *= f;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] *= f;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (ls[j] == -INFINITY) continue;  // nothing in this part (or there is none)
      const float e = __builtin_amdgcn_exp2f(ls[j] - top);
      tot += e;
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] += y[j][k] * e;
    }
  }
  if (step > 1) {
    x_s[threadIdx.x] = x;
    if (ch == 0) {
      m_s[grp] = top;
      l_s[grp] = tot;
    }
    __syncthreads();
    if (first > 0) return;
    for (int j = 0; j < step; ++j) top = fmaxf(top, m_s[i + j * wide]);
    tot = 0.f;
    x = f32x4{};
    for (int j = 0; j < step; ++j) {
      const float ms = m_s[i + j * wide], e = ms == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms - top);
      const f32x4 y = x_s[threadIdx.x + j * wide * TPR];
      tot += l_s[i + j * wide] * e;
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] += y[k] * e;
    }
  }
  if (i >= rows) return;
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] *= inv;
  const int tok = (t.row0 + r) / a.G, head = t.g * a.G + (t.row0 + r - tok * a.G);
  put4<T>(a.out + (t.q0 + tok) * a.out_tok + (long long)head * D * (int)sizeof(T), ch * 4, x);
  if (ch == 0 && a.lse)
    a.lse[(long long)head * a.N_q + t.q0 + tok] = tot == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(tot)) * kLn2;
}

constexpr int kManyWaves = 4;
// Short work in bf16: a block per tile of 16 or 32 rows that joins its waves' parts
// itself, while the tiles fit on the chip at once (of 512-byte parts one on a CU, of
// 256-byte ones two; the bound counts up to a tile too many per sequence) and four
// waves are enough for a tile's keys.
// One token, 28/4 heads of 128: 794 keys 10.2 -> 8.9 us, 1,500 keys 11.7 -> 16.9; 32
// requests of 300 keys, 32/8 heads, 17.1 -> 15.0, 64 of them 21.4 -> 33.6; 28 of 900,
// 16/16 heads of 64, 26.1 -> 20.4.  Prompts against blocks of 128 rows: 200 tokens, 28/4
// heads 12.3 -> 8.9 us, two of 200, 32/8 heads (416 tiles) 11.7 -> 13.9, 400, 16/16
// heads of 64 (416) 11.3 -> 7.3, two of 300 9.9 -> 8.2, four (656) 10.3 -> 12.6.
// Twice the keys where the tiles fill half of the chip, since ranges of keys gain less
// there: eight chunks of 30 over 1,500 keys, 32/8 heads (304 tiles) 37.7 -> 21.2 us,
// over 3,000 40.8 -> 37.0, two of 60 over 3,500 (136) 25.3 -> 32.0; one of 30 over 1,500,
// 28/4 heads (28) 16.6 -> 17.8.  Not for single tokens, whose sequences differ most in
// length (60 of 10-2,000 keys, 28/4 heads, 19.8 -> 27.2).
// fp32 keeps the line: 8 requests of 300 keys 16.6 -> 19.3.
constexpr int kShortTiles = 384, kShortTiles64 = 512, kShortKeys = 1024, kShortFull = 128, kShortFullKeys = 2048;
// single tokens behind a window (page_attn_plan)
constexpr int kAlikeKeys = 2560;
// and chunks in fp32
constexpr int kThreeStages = 320;
// 32-key tiles of a stage: fp32 rows of 512 bytes fill a stage with one
constexpr int many_tiles(int row_bytes) { return row_bytes > 256 ? 1 : 2; }

}  // namespace

PageAttnPlan page_attn_plan(const avtp_pages &P, int Hq, int B, int64_t N_q, int64_t max_kv_len,
                            const PageWindow &w) {
  PageAttnPlan L{};
  // (longer sequences run all the same)
  max_kv_len = max_kv_len < 1 ? 1 : max_kv_len < (1 << 30) ? max_kv_len : (1 << 30);
  // what a row sees (a tile's first rows see a few more keys than its last)
  const int64_t seen = (int64_t)w.window + w.sinks;
  const bool alike = w.window > 0 && max_kv_len >= 2 * seen;
  if (w.window > 0 && max_kv_len > seen) max_kv_len = seen;
  const int64_t rows = N_q * (Hq / P.Hkv);
  // one wave of 16 or 32 rows for a sequence, or blocks of 128; a tile's ranks: at most
  auto tiles_of = [&](int bm) { return (rows / bm + B) * P.Hkv; };
  const int small = rows <= (int64_t)B * 16 ? 16 : 32;
  const int64_t brief = tiles_of(small);
  L.brief = P.dtype == AVTP_BF16 && brief <= (P.d == 64 ? kShortTiles64 : kShortTiles) &&
            max_kv_len <= (small == 32 && brief >= kShortFull ? kShortFullKeys : kShortKeys);
  // (the tiles of sequences of equally many rows)
  const int64_t now = ((rows + small - 1) / small > B ? (rows + small - 1) / small : B) * P.Hkv;
  // Behind a window most sequences see equally much (told by a bound of twice the window
  // or more), so that blocks of single tokens end together: four waves or two a tile, where
  // they are on half of the CUs in one round or fill 0.7 of the places of several.  One
  // token, 32/8 heads of 128, window 1,024, the line against blocks: 8 requests (64
  // tiles) 16.8 / 17.0 us, 16 22.9 / 19.0, 32 33.4 / 28.4, 48 44.3 / 39.5 (two waves;
  // four 46.7), 64 of which some are short 49.6 / 44.7, 80 65.8 / 62.2 (two 67.7), 96 76.2
  // / 69.1 (two 71.7), 128 97.5 / 87.8; window 256, 64 24.3 / 24.4 (four 34.5), 96 29.4 /
  // 25.6 (four 30.9); 16/16 heads of 64, window 1,024, 8 (128 tiles) 17.5 / 14.1.  Longer
  // windows are not worth it where lengths differ after all (64 requests of 300-20,000
  // tokens, window 2,048 72.8 / 72.3, 4,096 111 / 115, 8,192 154 / 190; 16 4,096 36 / 48).
  // The line stays where two waves fill less and four lose: 80 requests, window 256 27.3, two
  // 24.2, four 28.5.
  if (alike && !L.brief && max_kv_len <= kAlikeKeys && P.dtype == AVTP_BF16 && small == 16) {
    // the part of their places that the blocks of the last round and those before fill
    auto fill = [&](int waves) {
      const int64_t places = 1024 / waves * (P.d == 64 ? 2 : 1), rounds = (now + places - 1) / places;
      const double f = (double)now / (double)(rounds * places);
      return (rounds == 1 ? now >= 128 : f >= 0.7) ? f : 0.;
    };
    const double four = fill(kShortWaves), two = fill(kShortWaves / 2);
    const bool once = now <= 256 * (P.d == 64 ? 2 : 1);
    L.half = !(four > 0 && (once || (max_kv_len > 512 && four > 1.12 * two)));
    L.brief = four > 0 || two > 0;
    if (L.half && two == 0.) L.brief = false;
  }
  // Tiles of 32 rows: in one round only, and from 80 tiles on of more keys (over 3,000 keys,
  // blocks that join / blocks of 128 rows: 300 tokens, window 64, 32/8 heads, 304 tiles 15.7
  // / 12.4, 1,024, 28/4 heads, 264 tiles 32.4 / 23.6; 100 tokens, 1,024, 104 and 88 tiles
  // 16.9 / 19.8 and 16.9 / 19.3; 30 tokens, 64 tiles 16.8 / 15.6).
  if (alike && P.dtype == AVTP_BF16 && small == 32)
    L.brief = now <= 256 * (P.d == 64 ? 2 : 1) && max_kv_len <= (now >= 80 ? kShortFullKeys : kShortKeys);
  // fp32 behind a window: where a block's waves (four, or two at d 128) have a few stages
  // each.  us, line or blocks of 128 rows against blocks that join, d 64 (14/2 heads) and
  // d 128 (16/8): 100 tokens, window 64 17.0 / 8.4 and 26.5 / 17.3, 256 18.9 / 14.2 and 27.6
  // / 32.6, 1,000 21.0 / 30.0; 300 tokens (131 tiles), 1,000 42.8 / 30.9; 1,000 tokens (440
  // tiles), 256 31.9 / 28.3, 1,000 57.8 / 60.1; one token, 64 11.0 / 5.5 and 15.0 / 10.4, 256
  // 11.3 / 9.0 and 15.2 / 18.5; 32 requests, 256 11.0 / 13.3 and (256 tiles) 32.1 / 27.2.
  // Between 257 and 512 tiles of d 64 up to three stages a wave, which hold 320 keys beside the
  // tile's own tokens and the ends of sinks and window (600 to 1,150 tokens and ten of 100, 14/2
  // heads, blocks of 128 rows / blocks that join: 260 keys 25.7-31.5 / 26.7-29.4, 304 27.9-33.7 /
  // 26.7-29.5, 344 27.5-38.0 / 29.2-34.2, 388 28.5-40.8 / 31.9-34.7; from there on now one, now
  // the other).
  if (w.window > 0 && P.dtype == AVTP_FP32) {
    const bool full = now >= kShortFull, narrow = P.d == 64;
    const int64_t most = narrow && small == 32 ? (full ? kShortFullKeys : 512) : !narrow && small == 16 && full && alike ? kAlikeKeys : 128;
    L.brief = now <= 256 ? max_kv_len <= most : narrow && small == 32 && now <= 512 && max_kv_len <= kThreeStages;
  }
  // Up to 32 rows a sequence is one tile of the even line; more rows read its keys once
  // per 32 there and once per 128 in a block.  us, line against blocks: 28/4 heads, 64
  // requests of 300-16,000 keys, 4 tokens (28 rows) 102 / 292, 5 (35 rows) 183 / 294, 9 (63)
  // 190 / 296, 18 (126) 362 / 296; eight of them, 28 rows 28.8 / 29.8, 35 rows 38.2 / 29.9; 32/8
  // heads, eight of 3,000 keys, 32 rows 34.0 / 32.4, 36 rows 43.1 / 34.1; one of 10,000,
  // 28/4 heads, 28 rows 24.8 / 19.4.  (It loses for 33 to 64 rows of many sequences of very
  // different length, and for 17 to 32 rows of a single long one.)
  L.few = L.brief || rows <= (int64_t)B * 32;
  const int bm = L.tile = L.few ? small : kManyWaves * 32;
  const int64_t tiles = tiles_of(bm);
  int64_t slots;
  if (L.brief) {
    L.blocks = tiles;
    slots = 0;
  } else if (L.few) {
    // As many workers as the CUs' LDS holds, with `least` units (of 32 keys) each or
    // more: a worker's time grows with its units, the join's with their number, so
    // their root.  28/4 heads, one token over 3,000 keys 15.1 -> 12.8 us against
    // single units, 10,000 22.1 -> 18.5, 40,000 36.7 -> 32.2.  Half of the root for tiles
    // of 32 rows, whose parts are more to join: 16/8 heads, 15 tokens over 3,000 keys
    // 25.0 -> 19.5, 10,000 36.2 -> 26.2, 40,000 51.7 -> 50.1.  The units are those of
    // max_kv_len, so a bound far above the lengths leaves few requests fewer workers
    // than would be best: one token over 794 keys 8.9 us at the exact bound, 16.2 at
    // 32,768, 22.0 at 131,072; 64 requests of 300-16,000 keys 163 and 169.
    auto per_cu = [&](auto m_tag) {
      constexpr int M = decltype(m_tag)::value;
      if (P.dtype == AVTP_FP32) return P.d == 64 ? Shape<float, 64, M, 1, 1>::kPerCu : Shape<float, 128, M, 1, 1>::kPerCu;
      return P.d == 64 ? Shape<__bf16, 64, M, 1, 1>::kPerCu : Shape<__bf16, 128, M, 1, 1>::kPerCu;
    };
    const int64_t most = 256 * (bm == 16 ? per_cu(std::integral_constant<int, 16>{}) : per_cu(std::integral_constant<int, 32>{}));
    const int64_t units = (max_kv_len + kTile - 1) / kTile;
    L.least = (int)(std::sqrt((double)units) / (bm == 16 ? 4 : 2));
    if (L.least < 1) L.least = 1;
    const int64_t need = (tiles * units + L.least - 1) / L.least;
    L.blocks = need < most ? need : most;
    L.cuts = (int)L.blocks;
    slots = 2 * L.blocks;
  } else {
    // Two blocks per CU.  In fp32 four (two of 512-byte rows): one chunk of 1,000
    // tokens, 16/8 heads of 128, 85 us with half as many, 70 with these, 88 with twice
    // as many.  (bf16 with twice as many: four chunks of 300 tokens 20 -> 31.)
    const bool f32 = P.dtype == AVTP_FP32;
    const int64_t want = f32 && P.d == 64 ? 1024 : 512;
    // us: a stage of 64 keys, a part written and read, the second launch (tiles of 64 rows
    // over 1,024 and 4,096 keys, 8-256 of them: a stage 1.09 at d 128, 0.77 at d 64; a fit over
    // one to 16 ranges gives 0.041 and 0.029 a part, 3.5 and 1.8 for the launch)
    const float part = 0.04f * P.d / 128 * tiles, join = 4.f;
    if (!f32) L.gain = (P.d == 64 ? 0.7f : 1.1f) / part;
    L.from = 1 + std::sqrt(1 + join / part);
    const int most = many_tiles(P.d * (f32 ? 4 : 2)) == 1 ? key_ranges<kTile>(max_kv_len, L.gain, L.from)
                                                          : key_ranges<2 * kTile>(max_kv_len, L.gain, L.from);
    const int64_t ns = want / tiles;
    L.nsplit = (int)(ns < 1 ? 1 : ns < most ? ns : most);
    L.blocks = tiles * L.nsplit;
    L.cuts = L.nsplit > 1 ? (int)tiles : 0;
    slots = L.nsplit > 1 ? L.blocks : 0;
  }
  if (N_q > 0 && L.cuts > 0) {
    L.off_lse = (size_t)slots * bm * P.d * 4;
    L.off_meta = L.off_lse + (size_t)slots * bm * 4;
    L.bytes = L.off_meta + (size_t)L.cuts * 32;
  }
  return L;
}

template <typename T, int D, typename A>
static hipError_t launch(hipStream_t st, const PageAttnPlan &L, const A &k) {
  constexpr int TPW = many_tiles(D * (int)sizeof(T));
  const dim3 grid((unsigned)L.blocks);
  if constexpr (sizeof(T) == 2 || A::WIN) {
    if (L.brief) {
      auto run = [&](auto m_tag, auto w_tag) {
        constexpr int M = decltype(m_tag)::value, W = decltype(w_tag)::value;
        hipLaunchKernelGGL((page_attn_short_kernel<T, D, M, W, A>), grid, dim3(64 * W), 0, st, k);
      };
      // (fp32 rows of 512 bytes: two waves' buffers fill the LDS)
      constexpr std::integral_constant<int, kShortWaves * (D * (int)sizeof(T) > 256 ? 2 : 4) / 4> all{};
      if (L.tile == 32) run(std::integral_constant<int, 32>{}, all);
      else if (!A::WIN || !L.half) run(std::integral_constant<int, 16>{}, all);
      else if constexpr (A::WIN) run(std::integral_constant<int, 16>{}, std::integral_constant<int, kShortWaves / 2>{});
      return hipGetLastError();
    }
  }
  if (L.tile == 16) hipLaunchKernelGGL((page_attn_few_kernel<T, D, 16, A>), grid, dim3(64), 0, st, k);
  else if (L.few) hipLaunchKernelGGL((page_attn_few_kernel<T, D, 32, A>), grid, dim3(64), 0, st, k);
  else hipLaunchKernelGGL((page_attn_many_kernel<T, D, kManyWaves, TPW, A>), grid, dim3(64 * kManyWaves), 0, st, k);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || L.cuts == 0) return e;
  // (a block per 2048 / D rows, one for a shorter tile)
  auto join = [&](auto bm_tag) {
    constexpr int BM = decltype(bm_tag)::value, ROWS = kJoinThreads * 4 / D < BM ? kJoinThreads * 4 / D : BM;
    hipLaunchKernelGGL((page_join_kernel<T, D, BM>), dim3((unsigned)(L.cuts * (BM / ROWS))), dim3(ROWS * D / 4), 0, st,
                       (const KArgs &)k);
  };
  if (L.tile == 16) join(std::integral_constant<int, 16>{});
  else if (L.few) join(std::integral_constant<int, 32>{});
  else join(std::integral_constant<int, kManyWaves * 32>{});
  return hipGetLastError();
}

template <typename A>
static hipError_t launch(hipStream_t st, const avtp_pages &P, const PageAttnPlan &L, const A &k) {
  if (P.dtype == AVTP_FP32) return P.d == 64 ? launch<float, 64>(st, L, k) : launch<float, 128>(st, L, k);
  return P.d == 64 ? launch<__bf16, 64>(st, L, k) : launch<__bf16, 128>(st, L, k);
}

hipError_t launch_page_attention(hipStream_t st, const avtp_pages &P, const PageAttnPlan &L,
                                 const PageAttnArgs &A, char *ws) {
  clear_pending_error();
  WArgs k;
  k.window = A.w.window;
  k.sinks = A.w.sinks;
  k.q = (const char *)A.q;
  k.k = (const char *)P.k;
  k.v = (const char *)P.v;
  k.out = (char *)A.out;
  k.q_tok = A.q_tok;
  k.out_tok = A.out_tok;
  k.head_bytes = (long long)P.page_size * P.d * (P.dtype == AVTP_FP32 ? 4 : 2);
  k.lse = A.lse;
  k.po = (float *)ws;
  k.pl = (float *)(ws + L.off_lse);
  k.meta = (int4 *)(ws + L.off_meta);
  k.cu_q = A.cu_q;
  k.kv_len = A.kv_len;
  k.table = A.table;
  k.status = A.status;
  k.B = A.B;
  k.Hkv = P.Hkv;
  k.G = A.Hq / P.Hkv;
  k.N_q = A.N_q;
  k.max_pages = A.max_pages;
  k.n_pages = P.n_pages;
  k.page_shift = __builtin_ctz((unsigned)P.page_size);
  k.workers = (int)L.blocks;
  k.nsplit = L.nsplit;
  k.least = L.least;
  k.gain = L.gain;
  k.from = L.from;
  k.cl2e = A.scale * kLog2e;
  return A.w.window > 0 ? launch(st, P, L, k) : launch(st, P, L, (const KArgs &)k);
}

}  // namespace avtp
