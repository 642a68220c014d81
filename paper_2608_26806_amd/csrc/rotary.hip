// The norm of queries and keys head by head and their rotation by the tokens'
// positions, in one pass over the rows, with K and V on into their pages.
//
// Of a head's values x: y = x w rsqrt(mean(x^2) + eps), then for each pair (a, b)
// of the rotated ones, with t its angle,
//   a' = s (a cos t - b sin t),  b' = s (b cos t + a sin t).
// All of it in fp32, rounded once at the end.  The angle is counted in turns: a
// position times the turns of one position, a fraction in 64 bits, so that whole
// turns drop out of the integer product and what is left is as exact at position
// 10^9 as at 1.  Sine and cosine are Taylor sums on an eighth of a turn to either
// side: below 2^-28 behind the terms taken, about 2^-23 with their roundings.
//
// HBM-bound: every row is read once and written once.  133,120 rows of 32/8 heads of
// 128 take in bf16 465 us (2.73 GB, 5.9 TB/s; a plain copy of 4 GB 4.9), into pages with
// their values 551 (3.27 GB, 5.9), in fp32 924 and 1,106; 64 rows of a decode step 4.3 us,
// a launch and two dependent loads.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "avtp_internal.h"

namespace avtp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;

struct NArgs {
  RotaryArgs r;
  int heads;   // q, k and (into pages) v
  int groups;  // waves that share a token's heads
  int page_shift;
  long long slots;
};

// sine and cosine of h / 2^32 turns
__device__ inline void sincos_turns(int32_t h, float &s, float &c) {
  const uint32_t quarter = ((uint32_t)h + 0x20000000u) >> 30;
  const float x = (float)(int32_t)((uint32_t)h - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float z = x * x;
  float a = 1.f / 362880, b = -1.f / 3628800;
  a = __builtin_fmaf(a, z, -1.f / 5040);
  b = __builtin_fmaf(b, z, 1.f / 40320);
  a = __builtin_fmaf(a, z, 1.f / 120);
  b = __builtin_fmaf(b, z, -1.f / 720);
  a = __builtin_fmaf(a, z, -1.f / 6);
  b = __builtin_fmaf(b, z, 1.f / 24);
  a = __builtin_fmaf(a * z, x, x);
  b = __builtin_fmaf(b, z, -0.5f);
  b = __builtin_fmaf(b, z, 1.f);
  const bool odd = quarter & 1;
  s = odd ? b : a;
  c = odd ? a : b;
  s = quarter & 2 ? -s : s;
  c = (quarter + 1) & 2 ? -c : c;
}

// the sum over the N neighbouring lanes of a head
template <int N>
__device__ inline float over_head(float x) {
  auto add = [&](auto ctrl) __attribute__((always_inline)) {
    const int u = __builtin_bit_cast(int, x);
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  add(std::integral_constant<int, 0xB1>{});               // lane ^ 1
  add(std::integral_constant<int, 0x4E>{});               // lane ^ 2
  if constexpr (N >= 8) add(std::integral_constant<int, 0x141>{});  // the other four of eight
  if constexpr (N >= 16) add(std::integral_constant<int, 0x140>{});  // the other eight of sixteen
  return x;
}

// A head's row is TPH lanes wide, two pieces of 16 bytes each: where the row is
// rotated in halves the pieces that belong together, else neighbours.  A wave takes
// heads of one token, 64 / TPH at once.  The sines and cosines of a block's tokens,
// four at the most, are computed once, one a thread, while the first rows are on their
// way, and handed round in LDS with the norm weights: with each lane's eight angles in
// its registers a wave had 131 of them and the prompts above took 588 us.  One row a
// lane in flight, many waves: with two 64 rows took 4.6 us instead of 4.3, 2,000 rows
// 12.2 instead of 10.0.
template <typename T, int D, bool HALF, bool STREAM>
__global__ __launch_bounds__(kThreads) void norm_rotary_kernel(NArgs a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int E = 16 / (int)sizeof(T);  // values of a piece
  constexpr int TPH = D / (2 * E), HPW = 64 / TPH;
  constexpr int ROWB = D * (int)sizeof(T);
  __shared__ __attribute__((aligned(16))) float cs_s[kWaves][D / 2], sn_s[kWaves][D / 2], w_s[2][D];
  const RotaryArgs &r = a.r;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane % TPH;
  const unsigned w0 = (blockIdx.y * gridDim.x + blockIdx.x) * kWaves, t0 = w0 / a.groups, t = (w0 + wave) / a.groups;
  const int group = (int)(w0 + wave - t * a.groups);
  const bool here = t < r.n;
  const bool turned = c * E < r.rot / 2;
  const int pa = HALF && turned ? c * E : 2 * c * E, pb = HALF && turned ? r.rot / 2 + c * E : (2 * c + 1) * E;
  const long long slot = r.slot && here ? (long long)r.slot[t] : 0;
  const bool stored = slot >= 0 && slot < a.slots;
  const long long page = (slot >> a.page_shift) * r.Hk, at = slot & ((1 << a.page_shift) - 1);

  u32x4 x[2];
  char *to;
  int kind;  // 0: query, 1: key, 2: value, 3: nothing
  auto load = [&](int h) __attribute__((always_inline)) {
    kind = h < r.Hq ? 0 : h < r.Hq + r.Hk ? 1 : 2;
    const int g = h - (kind == 0 ? 0 : kind == 1 ? r.Hq : r.Hq + r.Hk);
    const char *from = kind == 0 ? r.q + t * r.q_tok : kind == 1 ? r.k + t * r.k_tok : r.v + t * r.v_tok;
    if (kind == 0) to = r.q_out + t * r.q_out_tok + g * ROWB;
    else if (!r.slot) to = r.k_out + t * r.k_out_tok + g * ROWB;
    else to = (kind == 1 ? r.k_out : r.v_out) + (((page + g) << a.page_shift) + at) * ROWB;
    if (!here || h >= a.heads || (kind != 0 && !stored)) kind = 3;
    x[0] = x[1] = u32x4{};
    if (kind != 3) {
      x[0] = *reinterpret_cast<const u32x4 *>(from + g * ROWB + pa * (int)sizeof(T));
      x[1] = *reinterpret_cast<const u32x4 *>(from + g * ROWB + pb * (int)sizeof(T));
    }
  };
  int h = group * HPW + lane / TPH;
  load(h);

  {
    const unsigned mine = t0 + wave;  // (the block's tokens are at most one a wave)
    if (lane < r.rot / 2 && mine < r.n) {
      const unsigned plane = r.plane ? (unsigned)r.plane[lane] : 0;
      const uint64_t pos = (uint64_t)r.pos[(plane < (unsigned)r.planes ? plane : 0) * r.pos_stride + mine];
      float s, k;
      sincos_turns((int32_t)((pos * r.turns[lane]) >> 32), s, k);
      cs_s[wave][lane] = k * r.scale;
      sn_s[wave][lane] = s * r.scale;
    }
    if (tid < D) w_s[0][tid] = r.q_weight ? r.q_weight[tid] : 1.f;
    else if (tid < 2 * D) w_s[1][tid - D] = r.k_weight ? r.k_weight[tid - D] : 1.f;
  }
  __syncthreads();
  if (!here) return;
  float cs[E], sn[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    cs[i] = turned ? cs_s[t - t0][c * E + i] : 1.f;
    sn[i] = turned ? sn_s[t - t0][c * E + i] : 0.f;
  }

  for (;;) {
    float y[2 * E];
#pragma unroll
    for (int i = 0; i < 2 * E; ++i) {
      if constexpr (F32) y[i] = __builtin_bit_cast(f32x4, x[i / E])[i % E];
      else y[i] = (float)__builtin_bit_cast(bf16x8, x[i / E])[i % E];
    }
    if (r.q_weight || r.k_weight) {  // (every lane of a head is here)
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) ss = __builtin_fmaf(y[i], y[i], ss);
      ss = over_head<TPH>(ss);
      const bool norm = kind == 0 ? r.q_weight != nullptr : r.k_weight != nullptr;
      const float f = norm ? 1.f / __builtin_sqrtf(ss / D + r.eps) : 1.f;
      const float *w = w_s[kind != 0];
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) y[i] = y[i] * f * w[i < E ? pa + i : pb + i - E];
    }
    if (turned) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        float &p = HALF ? y[i] : y[2 * i], &q = HALF ? y[E + i] : y[2 * i + 1];
        const float u = p * cs[i] - q * sn[i], v = q * cs[i] + p * sn[i];
        p = u;
        q = v;
      }
    }
    if (kind != 3) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        u32x4 o = x[j];
        if (kind != 2) {  // (values pass bit for bit)
          if constexpr (F32) {
            o = __builtin_bit_cast(u32x4, f32x4{y[j * E], y[j * E + 1], y[j * E + 2], y[j * E + 3]});
          } else {
            bf16x8 b;
#pragma unroll
            for (int i = 0; i < E; ++i) b[i] = (__bf16)y[j * E + i];
            o = __builtin_bit_cast(u32x4, b);
          }
        }
        u32x4 *dst = reinterpret_cast<u32x4 *>(to + (j == 0 ? pa : pb) * (int)sizeof(T));
        if constexpr (STREAM) __builtin_nontemporal_store(o, dst);
        else *dst = o;
      }
    }
    h += a.groups * HPW;
    if (h >= a.heads) break;
    load(h);
  }
}

template <typename T, int D>
hipError_t launch(hipStream_t st, NArgs a) {
  constexpr int HPW = 64 / (D * (int)sizeof(T) / 32);
  const int most = (a.heads + HPW - 1) / HPW;
  // A wave for each 64 / TPH heads of few tokens; of tokens that fill the chip two or
  // three times as many heads a wave, whose angles are computed less often (both with
  // cached stores: 133,120 rows 482 us, 540 with one round of heads a wave, 518 with all
  // five; 8,000 rows 37, 41 and 42).
  constexpr long long kFull = 4096;
  a.groups = most / 2 > 1 ? most / 2 : 1;
  while (a.groups < most && a.r.n * a.groups < kFull) ++a.groups;
  // Outputs of half of the Infinity Cache or more go past the caches (133,120 rows 482 ->
  // 463 us): with a reader behind them 16,000 rows (164 MB written) take 115 us instead of
  // 122, 8,000 rows 58.3 instead of 57.6, 2,000 rows 17.1 instead of 16.0.
  const bool stream = a.r.n * a.heads * D * (int)sizeof(T) >= 128ll << 20;
  const long long blocks = (a.r.n * a.groups + kWaves - 1) / kWaves;
  constexpr long long kWide = 1 << 20;  // blocks side by side (2^32 threads are too many for one axis)
  const dim3 grid((unsigned)(blocks < kWide ? blocks : kWide), (unsigned)((blocks + kWide - 1) / kWide));
  auto run = [&](auto half, auto streamed) {
    hipLaunchKernelGGL((norm_rotary_kernel<T, D, decltype(half)::value, decltype(streamed)::value>), grid, dim3(kThreads),
                       0, st, a);
  };
  auto form = [&](auto half) {
    if (stream) run(half, std::true_type{});
    else run(half, std::false_type{});
  };
  if (a.r.interleaved) form(std::false_type{});
  else form(std::true_type{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rotary(hipStream_t st, const RotaryArgs &R, int dtype, int d, int page_size, int64_t slots) {
  clear_pending_error();
  NArgs a;
  a.r = R;
  a.heads = R.Hq + (R.slot ? 2 : 1) * R.Hk;
  a.page_shift = R.slot ? __builtin_ctz((unsigned)page_size) : 0;
  a.slots = R.slot ? slots : 1;
  if (dtype == AVTP_FP32) return d == 64 ? launch<float, 64>(st, a) : launch<float, 128>(st, a);
  return d == 64 ? launch<__bf16, 64>(st, a) : launch<__bf16, 128>(st, a);
}

}  // namespace avtp
