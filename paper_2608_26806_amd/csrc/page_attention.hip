// Attention of new tokens over the paged K/V cache on gfx950 (MFMA, wave64).
//
// One pass over the keys with the running maximum m and sum l of each row's
// softmax: for a tile of keys, z = c q.k, and when a row's maximum rises from
// m to m' its sum and its output so far are scaled by exp(m - m').  Neither the
// logits nor the probabilities leave the registers:
//   S^T = K Q^T: keys are the MFMA's rows, query rows its columns, so a lane
//     owns one query row (half of its keys; the other half is 32 lanes away)
//     and the softmax needs one exchange per tile, for the maximum;
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

#include <type_traits>

#include "avtp_internal.h"

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
constexpr int kTile = 32;  // query rows and keys of an MFMA tile
// A row's exponentials refer to the largest logit m of some earlier tile, not
// always of all: only when their sum over a tile leaves this range is m raised
// (and the sum and output so far scaled).  fp32 sums, and products with bf16 or
// fp32 probabilities of that size, are as exact as with the true maximum.
constexpr float kLazyLimit = 65536.f;

template <typename T, int D>
struct Geo {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int ROWB = D * (int)sizeof(T);  // bytes of a head row
  static constexpr int NCH = ROWB / 16;            // its 16-byte chunks
  static constexpr int RPL = 64 / NCH;             // rows of a wave's load
  static constexpr int NS = D * (int)sizeof(T) / 32;  // K fragments per key (16 bytes per lane half)
  static constexpr int ND = D / 32;                // output tiles of 32 values
  // Chunk order inside an LDS row, XOR-ed with the row: 16 consecutive rows of
  // one chunk (a K fragment) lie in 16 different places of the 64 banks, and so
  // do the four 64-byte pieces of consecutive rows that a transposing read of
  // bf16 V takes (with those of the next four rows in the other lane half).
  static __device__ inline int swz(int row) {
    if (F32) return row & 15;
    return NCH == 16 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  }
};

struct KArgs {
  const char *q, *k, *v;
  char *out;
  long long q_tok, out_tok, head_bytes;  // head_bytes: one head of one page
  float *lse, *po, *pl;
  const int32_t *cu_q, *kv_len, *table;
  int32_t *status;
  int B, Hq, Hkv, G, N_q, max_pages, n_pages, page_shift, nsplit, chunk;
  float cl2e;
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

__device__ inline void wait_vmem() {
  __builtin_amdgcn_s_waitcnt(0xF70);
  asm volatile("" ::: "memory");
}

// of both lane halves: combine(x, the value 32 lanes away)
__device__ inline float half_max(float x) {
  const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x),
                                                  false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)p[0]), __builtin_bit_cast(float, (unsigned)p[1]));
}
__device__ inline float half_sum(float x) {
  const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x),
                                                  false, false);
  return __builtin_bit_cast(float, (unsigned)p[0]) + __builtin_bit_cast(float, (unsigned)p[1]);
}

// Row tile slots: sequence b's tiles of BM rows are numbered from
// floor(cu_q[b] G / BM) + b on.  The next sequence's start is at least
// ceil(n_b G / BM) further, so every tile has a slot of its own, there are at
// most floor(N_q G / BM) + B, and no prefix sum is needed to find one.
struct Seq {
  int b, q0, q1, kv, base;
};
__device__ inline Seq find_seq(const KArgs &a, int slot, int bm_shift) {
  const int lane = threadIdx.x & 63;
  auto first = [&](int c, int b) __attribute__((always_inline)) {
    return ((min(max(0, c), a.N_q) * a.G) >> bm_shift) + b;
  };
  int w0 = 0;
  if (a.B > 64) {
    int step = 64;
    while (step * 64 < a.B) step *= 64;
    for (; step > 1; step >>= 6) {
      const int c = w0 + lane * step;
      const unsigned long long m = __ballot(c < a.B && first(a.cu_q[min(c, a.B)], c) <= slot);
      w0 += max(0, __builtin_popcountll(m) - 1) * step;
    }
  }
  const int c = min(w0 + lane, a.B - 1);
  const int lo = a.cu_q[c], hi = a.cu_q[c + 1], kv = a.kv_len[c];
  const unsigned long long m = __ballot(w0 + lane < a.B && first(lo, c) <= slot);
  const int src = max(0, __builtin_popcountll(m) - 1);
  Seq s;
  s.b = w0 + src;
  s.q0 = min(max(0, __builtin_amdgcn_readlane(lo, src)), a.N_q);
  s.q1 = min(max(s.q0, __builtin_amdgcn_readlane(hi, src)), a.N_q);
  s.kv = max(0, __builtin_amdgcn_readlane(kv, src));
  s.base = first(s.q0, s.b);
  return s;
}

// A block takes one row tile (WR waves of 32 rows) of one key head and one
// range of its keys; the keys of a stage are shared out over WK waves, whose
// results are joined at the end.  WK = 1: many rows, the waves share every
// stage.  WR = 1: few rows (a decode step), every wave streams keys of its
// own and waits for nobody.
template <typename T, int D, int WR, int WK, int TPW>
__global__ __launch_bounds__(64 * WR * WK, (WK > 1 || D * sizeof(T) > 256 ? 1 : 2)) void page_attn_kernel(KArgs a) {
  using G_ = Geo<T, D>;
  constexpr bool F32 = G_::F32;
  constexpr int NW = WR * WK, BM = WR * kTile, ROWB = G_::ROWB, NCH = G_::NCH, RPL = G_::RPL;
  constexpr int NS = G_::NS, ND = G_::ND;
  constexpr int KS = WK * TPW * kTile;             // keys per stage
  constexpr int RW = KS / NW;                      // of them, rows a wave loads (its own, if WK > 1)
  constexpr int GR = RW < 16 ? RW : 16;            // rows of one page group
  constexpr int NG = RW / GR, LPG = GR / RPL;
  static_assert(WR == 1 || WK == 1, "");
  static_assert(RW % RPL == 0 && GR % RPL == 0 && (WK == 1 || RW == TPW * kTile), "whole loads");
  constexpr int TB = KS * ROWB;                    // bytes of one tensor's stage
  // two stage buffers as distinct objects, so the compiler can tell the one
  // being read from the one in flight
  __shared__ __attribute__((aligned(16))) char smA[2 * TB];
  __shared__ __attribute__((aligned(16))) char smB[2 * TB];
  __shared__ float ml_s[WK > 1 ? WK * kTile * 2 : 1];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = WR > 1 ? wave : 0, wk = WK > 1 ? wave : 0;
  const int hi = lane >> 5, col = lane & 31;
  constexpr int kBmShift = BM == 32 ? 5 : (BM == 128 ? 7 : 8);
  static_assert(BM == 1 << kBmShift, "");

  // key heads fastest: blocks go to the XCDs in turn, so an XCD sees few heads.
  // The last tiles of a sequence see the most keys and go first.
  const int g = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv;
  const int nslots = gridDim.x / a.Hkv / a.nsplit;
  const int slot = nslots - 1 - rest / a.nsplit, split = rest % a.nsplit;
  const Seq sq = find_seq(a, slot, kBmShift);
  const int b = sq.b, n = sq.q1 - sq.q0;
  const int R = n * a.G, row0 = (slot - sq.base) * BM;
  if (slot < sq.base || row0 >= R) return;

  // tokens of the sequence that the table has room for
  const long long cap = (long long)a.max_pages << a.page_shift;
  const int L = (int)min((long long)sq.kv, cap);
  if (L < sq.kv && a.status && tid == 0) atomicOr(&a.status[b], AVTP_FLAG_BAD_PAGE);
  // row r of the sequence: token r / G, which sees kv - n + token + 1 keys
  const int wrow = row0 + wr * kTile;
  const int row = min(wrow + col, R - 1), tok = row / a.G, head = g * a.G + (row - tok * a.G);
  const int lim = min(L, sq.kv - n + tok + 1);
  const bool valid = wrow + col < R;
  const int wmin = __builtin_amdgcn_readlane(lim, 0), wmax = __builtin_amdgcn_readlane(lim, 31);
  const int blast = min(row0 + BM, R) - 1;
  const int bmax = min(L, sq.kv - n + blast / a.G + 1);  // keys the block's last row sees
  const int kbeg = split * a.chunk;
  const int kend = split + 1 < a.nsplit ? min(bmax, kbeg + a.chunk) : bmax;

  // (a row's place among all rows: token, then head)
  const long long orow = (long long)(sq.q0 + tok) * a.Hq + head;
  if (kbeg >= kend) {  // no key for any row of the block
    if (a.nsplit > 1) {
      if (wk == 0 && valid && hi == 0) a.pl[(long long)split * a.N_q * a.Hq + orow] = -INFINITY;
    } else if (wk == 0 && valid) {
      u32x4 *o = reinterpret_cast<u32x4 *>(a.out + (sq.q0 + tok) * a.out_tok + (long long)head * ROWB);
      for (int c = hi; c < NCH; c += 2) o[c] = u32x4{};
      if (a.lse && hi == 0) a.lse[(long long)head * a.N_q + sq.q0 + tok] = -INFINITY;
    }
    return;
  }

  // query rows, the second operand of S^T
  u32x4 qf[NS];
  {
    const char *p = a.q + (sq.q0 + tok) * a.q_tok + (long long)head * ROWB + hi * 16;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const u32x4 *>(p + s * 32);
  }

  // where this lane's loads of a 16-row group come from
  uint32_t voff[LPG];
  const int r0w = wave * RW;  // the wave's first row of a stage
#pragma unroll
  for (int i = 0; i < LPG; ++i) {
    const int r = i * RPL + lane / NCH;
    voff[i] = (uint32_t)(r * ROWB + ((lane % NCH) ^ G_::swz(r0w + r)) * 16);
  }
  const int32_t *trow = a.table + (long long)b * a.max_pages;
  const int pmask = (1 << a.page_shift) - 1;
  // page ids of the wave's groups of the stage at key ks, one per lane (lane
  // gi: group gi), read a stage ahead
  auto load_ids = [&](int ks) __attribute__((always_inline)) {
    const int key = min(ks + r0w + (lane & (NG - 1)) * 16, L - 1);
    return trow[key >> a.page_shift];
  };
  auto issue = [&](char *buf, int ks, int ids) __attribute__((always_inline)) {
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      const int id = __builtin_amdgcn_readlane(ids, gi);
      const int key = ks + r0w + gi * 16;
      const bool ok = (unsigned)id < (unsigned)a.n_pages;
      if (!ok && key < L && a.status && lane == 0) atomicOr(&a.status[b], AVTP_FLAG_BAD_PAGE);
      const int have = ok ? min(max(L - key, 0), GR) * ROWB : 0;
      const long long off = ok ? ((long long)id * a.Hkv + g) * a.head_bytes + (long long)(key & pmask) * ROWB : 0;
      const Rsrc rk = make_rsrc(a.k + off, have), rv = make_rsrc(a.v + off, have);
      char *dst = buf + (r0w + gi * 16) * ROWB;
#pragma unroll
      for (int i = 0; i < LPG; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (AVTP_LDS void *)(dst + i * 1024), 16, (int)voff[i], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < LPG; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (AVTP_LDS void *)(dst + TB + i * 1024), 16, (int)voff[i], 0, 0, 0);
    }
  };

  f32x16 O[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) O[i] = f32x16{};
  float m = -INFINITY, l = 0.f;  // this lane's share of the row's sum
  const float cl2e = a.cl2e;

  // element e of a tile of this lane: key eoff(e) + 4 hi of the tile
  auto eoff = [](int e) __attribute__((always_inline)) { return 8 * (e >> 2) + (e & 3); };

  // LDS addresses of a tile's operands: the lane's base, XOR-ed with the chunk,
  // plus rows that fit the instruction's offset.
  // K: row col, fragment s
  typedef AVTP_LDS const char *lptr;
  const uint32_t kbase = (uint32_t)(col * ROWB + ((hi ^ G_::swz(col)) << 4));
  auto kaddr = [&](lptr kt, int s) __attribute__((always_inline)) { return kt + (kbase ^ (uint32_t)(s << 5)); };
  // V, bf16: the transposing read hands lane i of 16 the value i of four rows of
  // 16 values whose addresses the lanes give (lane i: four values of row i / 4),
  // here 32 dt + col of the four keys 16 c + 8 j + 4 hi + .. that belong to the
  // lane's probabilities 8 c + 4 j + ..
  const int ti = lane & 15, tq = (lane >> 4) & 1;
  const int vrow = F32 ? 4 * hi : 4 * hi + (ti >> 2);
  const uint32_t vbase = F32 ? (uint32_t)(vrow * ROWB + (((col >> 2) ^ G_::swz(vrow)) << 4) + (col & 3) * 4)
                             : (uint32_t)(vrow * ROWB + (((2 * tq + ((ti & 3) >> 1)) ^ G_::swz(vrow)) << 4) + (ti & 1) * 8);
  auto vfrag = [&](lptr vt, int c, int dt) __attribute__((always_inline)) {
    bf16x8 f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t o = (vbase ^ (uint32_t)(dt << 6 | (G_::swz(8 * j) << 4))) + (uint32_t)((16 * c + 8 * j) * ROWB);
      const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((AVTP_LDS bf16x4 *)(vt + o));
#pragma unroll
      for (int i = 0; i < 4; ++i) f[4 * j + i] = x[i];
    }
    return f;
  };
  // fp32: value 32 dt + col of key eoff(e) + 4 hi
  auto velem = [&](lptr vt, int e, int dt) __attribute__((always_inline)) {
    const uint32_t o = (vbase ^ (uint32_t)(((8 * dt) ^ G_::swz(eoff(e))) << 4)) + (uint32_t)(eoff(e) * ROWB);
    return *reinterpret_cast<AVTP_LDS const float *>(vt + o);
  };

  // Values of V that are not finite, in a tile that some row sees only in
  // part: 0 times them is not 0.  The tile's product then runs without them
  // and they are added to the rows that see them.
  auto not_finite = [&](uint32_t x) __attribute__((always_inline)) {
    return F32 ? (x & 0x7f800000u) == 0x7f800000u : ((((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0u);
  };
  auto tile_not_finite = [&](lptr vt) __attribute__((always_inline)) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kTile * NCH / 64; ++i) {
      const u32x4 x = *reinterpret_cast<AVTP_LDS const u32x4 *>(vt + (i * 64 + lane) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) bad = bad || not_finite(x[j]);
    }
    return __ballot(bad) != 0ull;
  };
  auto add_not_finite = [&](lptr vt, int kb) __attribute__((always_inline)) {
#pragma unroll 1
    for (int r = 0; r < kTile; ++r) {
      const bool seen = kb + r < lim;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int dd = 32 * dt + eoff(e) + 4 * hi;  // this lane's value of the output
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
  auto logits = [&](lptr kt) __attribute__((always_inline)) {
    f32x16 S = f32x16{};
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      if constexpr (F32) {
        const f32x4 kf = *reinterpret_cast<AVTP_LDS const f32x4 *>(kaddr(kt, s)), qv = __builtin_bit_cast(f32x4, qf[s]);
#pragma unroll
        for (int i = 0; i < 4; ++i) S = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[i], qv[i], S, 0, 0, 0);
      } else {
        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<AVTP_LDS const bf16x8 *>(kaddr(kt, s)),
                                                    __builtin_bit_cast(bf16x8, qf[s]), S, 0, 0, 0);
      }
    }
    return S;
  };
  // p = 2^(c S - m), as the second product takes them, and their sum
  struct Bf {
    bf16x8 x[2];
  };
  typedef std::conditional_t<F32, f32x16, Bf> Probs;
  auto probs = [&](const f32x16 &S, Probs &p, float ref) __attribute__((always_inline)) {
    float sum[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = __builtin_amdgcn_exp2f(S[e] * cl2e - ref);
      sum[e & 1] = e < 2 ? x : sum[e & 1] + x;
      if constexpr (F32) p[e] = x;
      else p.x[e >> 3][e & 7] = (__bf16)x;
    }
    return sum[0] + sum[1];
  };
  // O^T += V^T P^T
  auto weigh = [&](lptr vt, const Probs &p, bool clean) __attribute__((always_inline)) {
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          float x = velem(vt, e, dt);
          if (clean) x = __builtin_fabsf(x) < INFINITY ? x : 0.f;
          O[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p[e], O[dt], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          bf16x8 f = vfrag(vt, c, dt);
          if (clean) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __builtin_fabsf((float)f[i]) < INFINITY ? f[i] : (__bf16)0.f;
          }
          O[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, p.x[c], O[dt], 0, 0, 0);
        }
      }
    }
  };
  // N tiles of 32 keys that every row of the wave sees.  false (nothing done):
  // a row's sum left its range, or has no reference yet; `part` takes them.
  auto whole = [&](lptr kt, lptr vt, auto n_tag) __attribute__((always_inline)) {
    constexpr int N = decltype(n_tag)::value;
    f32x16 S[N];
    Probs p[N];
    float tot = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) S[i] = logits(kt + i * kTile * ROWB);
#pragma unroll
    for (int i = 0; i < N; ++i) tot += probs(S[i], p[i], m);
    if (__builtin_expect(__ballot(!(tot <= kLazyLimit)) != 0ull, 0)) return false;
    l += tot;
#pragma unroll
    for (int i = 0; i < N; ++i) weigh(vt + i * kTile * ROWB, p[i], false);
    return true;
  };
  // A tile of keys from kb on, of which some rows may see a part or nothing, and
  // whose largest logit becomes the row's reference if it is larger.
  auto part = [&](lptr kt, lptr vt, int kb) __attribute__((always_inline)) {
    f32x16 S = logits(kt);
    Probs p;
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = kb + 4 * hi + eoff(e) < lim ? S[e] : -INFINITY;
    float top = S[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, S[e]);
    const float nm = fmaxf(m, half_max(top) * cl2e);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - nm);
    m = nm;
    l *= f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) O[dt][e] *= f;
    l += probs(S, p, m == -INFINITY ? 0.f : m);  // (no key seen so far: every term is 0)
    if (__builtin_expect(tile_not_finite(vt), 0)) {
      add_not_finite(vt, kb);
      weigh(vt, p, true);
    } else {
      weigh(vt, p, false);
    }
  };

  const int nstage = (kend - kbeg + KS - 1) / KS;
  int ids = load_ids(kbeg);
  issue(smA, kbeg, ids);
  ids = load_ids(kbeg + KS);
  auto step = [&](const char *buf, char *nxt, int st) __attribute__((always_inline)) {
    const int ks = kbeg + st * KS;
    wait_vmem();
    if (WK == 1) __syncthreads();  // stage st is in LDS; every wave is done with the other buffer
    if (st + 1 < nstage) {
      issue(nxt, ks + KS, ids);
      ids = load_ids(ks + 2 * KS);
    }
    // keys of this wave below the range's end, and the rows that see them
    const int kb = ks + wk * TPW * kTile, stop = min(kend, wmax);
    lptr kt = (lptr)(buf) + wk * TPW * kTile * ROWB, vt = kt + TB;
    if (__builtin_expect(kb + TPW * kTile <= min(kend, wmin), 1) &&
        __builtin_expect(whole(kt, vt, std::integral_constant<int, TPW>{}), 1))
      return;
#pragma unroll 1
    for (int t = 0; t < TPW; ++t)
      if (kb + t * kTile < stop) part(kt + t * kTile * ROWB, vt + t * kTile * ROWB, kb + t * kTile);
  };
  for (int st = 0; st < nstage; st += 2) {
    step(smA, smB, st);
    if (st + 1 < nstage) step(smB, smA, st + 1);
  }
  l = half_sum(l);

  // a finished row (or its part): values d .. d + 3, normalised
  auto put = [&](long long at_out, long long at_row, int dd, f32x4 x) __attribute__((always_inline)) {
    if (a.nsplit > 1) {
      *reinterpret_cast<f32x4 *>(a.po + ((long long)split * a.N_q * a.Hq + at_row) * D + dd) = x;
    } else if constexpr (F32) {
      *reinterpret_cast<f32x4 *>(a.out + at_out + dd * 4) = x;
    } else {
      bf16x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (__bf16)x[i];
      *reinterpret_cast<bf16x4 *>(a.out + at_out + dd * 2) = y;
    }
  };
  // log2 of the row's sum
  auto put_lse = [&](int t, int h, long long at_row, float x) __attribute__((always_inline)) {
    if (a.nsplit > 1) a.pl[(long long)split * a.N_q * a.Hq + at_row] = x;
    else if (a.lse) a.lse[(long long)h * a.N_q + sq.q0 + t] = x * kLn2;
  };

  if constexpr (WK == 1) {
    if (!valid) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const long long at_out = (sq.q0 + tok) * a.out_tok + (long long)head * ROWB;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        put(at_out, orow, 32 * dt + 8 * j + 4 * hi,
            f32x4{O[dt][4 * j] * inv, O[dt][4 * j + 1] * inv, O[dt][4 * j + 2] * inv, O[dt][4 * j + 3] * inv});
    if (hi == 0) put_lse(tok, head, orow, l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l));
  } else {
    // Join the waves' parts: each leaves its O in LDS (in 16-byte chunks, XOR-ed
    // with the row), its m and l beside it.
    constexpr int OB = kTile * D * 4;  // bytes of a wave's O
    static_assert(NW * OB <= 2 * TB, "the parts fit the first buffer");
    __syncthreads();
    char *mine = smA + wk * OB;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int ch = 8 * dt + 2 * j + hi;
        *reinterpret_cast<f32x4 *>(mine + col * (D * 4) + ((ch ^ (col & (D / 4 - 1))) << 4)) =
            f32x4{O[dt][4 * j], O[dt][4 * j + 1], O[dt][4 * j + 2], O[dt][4 * j + 3]};
      }
    if (hi == 0) {
      ml_s[(wk * kTile + col) * 2] = m;
      ml_s[(wk * kTile + col) * 2 + 1] = l;
    }
    __syncthreads();
    const int rows = min(R - row0, kTile);
    for (int i = tid; i < rows * (D / 4); i += NW * 64) {
      const int r = i / (D / 4), ch = i % (D / 4);
      float top = -INFINITY, tot = 0.f;
#pragma unroll
      for (int w = 0; w < WK; ++w) top = fmaxf(top, ml_s[(w * kTile + r) * 2]);
      f32x4 x = f32x4{};
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        const float mw = ml_s[(w * kTile + r) * 2];
        const float f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - top);
        tot += ml_s[(w * kTile + r) * 2 + 1] * f;
        const f32x4 y = *reinterpret_cast<const f32x4 *>(smA + w * OB + r * (D * 4) + ((ch ^ (r & (D / 4 - 1))) << 4));
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += y[j] * f;
      }
      const float inv = tot == 0.f ? 0.f : 1.f / tot;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] *= inv;
      const int t = (row0 + r) / a.G, h = g * a.G + (row0 + r - t * a.G);
      const long long ar = (long long)(sq.q0 + t) * a.Hq + h;
      put((sq.q0 + t) * a.out_tok + (long long)h * ROWB, ar, ch * 4, x);
      if (ch == 0) put_lse(t, h, ar, tot == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(tot));
    }
  }
}

// Joins the parts of the key ranges: a group of D / 4 threads per (token, head).
template <typename T, int D>
__global__ __launch_bounds__(256) void page_join_kernel(KArgs a) {
  constexpr int TPR = D / 4;
  const long long rows = (long long)a.N_q * a.Hq;
  const long long r = (long long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  const int ch = threadIdx.x % TPR;
  const int t = (int)(r / a.Hq), h = (int)(r - (long long)t * a.Hq);
  if (r >= rows || t < a.cu_q[0] || t >= a.cu_q[a.B]) return;
  float top = -INFINITY;
  for (int s = 0; s < a.nsplit; ++s) top = fmaxf(top, a.pl[s * rows + r]);
  float tot = 0.f;
  f32x4 x = f32x4{};
  for (int s = 0; s < a.nsplit; ++s) {
    const float ls = a.pl[s * rows + r];
    if (ls == -INFINITY) continue;  // no key in this range: nothing was written
    const float f = __builtin_amdgcn_exp2f(ls - top);
    const f32x4 y = *reinterpret_cast<const f32x4 *>(a.po + (s * rows + r) * D + ch * 4);
    tot += f;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] += y[j] * f;
  }
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
  char *o = a.out + t * a.out_tok + (long long)h * D * sizeof(T) + ch * 4 * sizeof(T);
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4 *>(o) = f32x4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
  } else {
    bf16x4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (__bf16)(x[j] * inv);
    *reinterpret_cast<bf16x4 *>(o) = y;
  }
  if (ch == 0 && a.lse)
    a.lse[(long long)h * a.N_q + t] = tot == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(tot)) * kLn2;
}

constexpr int kManyWaves = 4;                    // row waves of a block of many rows
constexpr int kManyRows = kManyWaves * kTile;

}  // namespace

PageAttnPlan page_attn_plan(const avtp_pages &P, int Hq, int B, int64_t N_q, int64_t max_kv_len) {
  PageAttnPlan L{};
  // (a longer sequence still runs: the last range takes the rest)
  max_kv_len = max_kv_len < (1 << 30) ? max_kv_len : (1 << 30);
  const int64_t G = Hq / P.Hkv, rows = N_q * G;
  L.few = rows <= (int64_t)B * kTile;
  const int bm = L.few ? kTile : kManyRows;
  const int64_t tiles = rows / bm + B;
  L.tiles = (int)tiles;
  // about 512 blocks, of 512 keys or more
  const int64_t blocks = tiles * P.Hkv;
  const int64_t most = (max_kv_len + 511) / 512;
  int64_t ns = 512 / (blocks < 1 ? 1 : blocks);
  ns = ns < 1 ? 1 : (ns > most ? (most < 1 ? 1 : most) : ns);
  int64_t chunk = (max_kv_len + ns - 1) / ns;
  chunk = (chunk + 127) / 128 * 128;
  if (chunk < 128) chunk = 128;
  L.nsplit = (int)ns;
  L.chunk = (int)chunk;
  if (L.nsplit > 1) {
    const size_t r = (size_t)N_q * Hq;
    L.off_lse = (r * L.nsplit * P.d * 4 + 255) / 256 * 256;
    L.bytes = L.off_lse + r * L.nsplit * 4;
  }
  return L;
}

template <typename T, int D>
static hipError_t launch(hipStream_t st, const PageAttnPlan &L, const KArgs &k) {
  const dim3 grid((unsigned)((long long)L.tiles * k.Hkv * L.nsplit));
  if (L.few) {
    constexpr int WK = sizeof(T) == 4 && D == 128 ? 2 : 4;
    hipLaunchKernelGGL((page_attn_kernel<T, D, 1, WK, 1>), grid, dim3(64 * WK), 0, st, k);
  } else {
    constexpr int TPW = sizeof(T) == 4 && D == 128 ? 1 : 2;
    hipLaunchKernelGGL((page_attn_kernel<T, D, kManyWaves, 1, TPW>), grid, dim3(64 * kManyWaves), 0, st, k);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || L.nsplit == 1) return e;
  const long long rows = (long long)k.N_q * k.Hq, per = 256 / (D / 4);
  hipLaunchKernelGGL((page_join_kernel<T, D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, k);
  return hipGetLastError();
}

hipError_t launch_page_attention(hipStream_t st, const avtp_pages &P, const PageAttnPlan &L,
                                 const PageAttnArgs &A, char *ws) {
  clear_pending_error();
  KArgs k;
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
  k.cu_q = A.cu_q;
  k.kv_len = A.kv_len;
  k.table = A.table;
  k.status = A.status;
  k.B = A.B;
  k.Hq = A.Hq;
  k.Hkv = P.Hkv;
  k.G = A.Hq / P.Hkv;
  k.N_q = A.N_q;
  k.max_pages = A.max_pages;
  k.n_pages = P.n_pages;
  k.page_shift = __builtin_ctz((unsigned)P.page_size);
  k.nsplit = L.nsplit;
  k.chunk = L.chunk;
  k.cl2e = A.scale * kLog2e;
  if (P.dtype == AVTP_FP32) {
    return P.d == 64 ? launch<float, 64>(st, L, k) : launch<float, 128>(st, L, k);
  }
  return P.d == 64 ? launch<__bf16, 64>(st, L, k) : launch<__bf16, 128>(st, L, k);
}

}  // namespace avtp
