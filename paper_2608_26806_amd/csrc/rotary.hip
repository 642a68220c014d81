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
// HBM-bound: every row is read once and written once.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "avtp_internal.h"

namespace avtp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kPlanes = AVTP_MAX_PLANES;

struct NArgs {
  RotaryArgs r;
  int heads;       // q, k and (into pages) v
  int groups;      // waves that share a token's heads
  long long waves; // waves with work: tokens taken at a time, times groups
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
// rotated in halves the pieces that belong together, else neighbours.  A wave
// takes 64 / TPH heads at once, U of them one after the other with their loads in
// flight together; angles and norm weights stay in its registers.
template <typename T, int D, bool HALF, int U>
__global__ __launch_bounds__(kThreads) void norm_rotary_kernel(NArgs a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int E = 16 / (int)sizeof(T);  // values of a piece
  constexpr int TPH = D / (2 * E), HPW = 64 / TPH;
  constexpr int ROWB = D * (int)sizeof(T);
  const RotaryArgs &r = a.r;
  const int lane = threadIdx.x & 63, c = lane % TPH;
  const long long w = (long long)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= a.waves) return;
  const int group = (int)(w % a.groups);
  const bool turned = c * E < r.rot / 2;
  const int pa = HALF && turned ? c * E : 2 * c * E, pb = HALF && turned ? r.rot / 2 + c * E : (2 * c + 1) * E;

  // of this lane's pairs c E + i: turns of a position, and which plane's
  uint64_t turns[E];
  int plane[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    turns[i] = turned ? r.turns[c * E + i] : 0;
    plane[i] = turned && r.plane ? r.plane[c * E + i] : 0;
  }
  float wq[2 * E], wk[2 * E];
#pragma unroll
  for (int i = 0; i < 2 * E; ++i) {
    const int at = i < E ? pa + i : pb + i - E;
    wq[i] = r.q_weight ? r.q_weight[at] : 1.f;
    wk[i] = r.k_weight ? r.k_weight[at] : 1.f;
  }

  for (long long t = w / a.groups; t < r.n; t += a.waves / a.groups) {
    float cs[E], sn[E];
    {
      uint64_t pos[kPlanes];
#pragma unroll
      for (int p = 0; p < kPlanes; ++p) pos[p] = p < r.planes ? (uint64_t)r.pos[p * r.pos_stride + t] : 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        uint64_t p = pos[0];
#pragma unroll
        for (int j = 1; j < kPlanes; ++j) p = plane[i] == j ? pos[j] : p;
        sincos_turns((int32_t)((p * turns[i]) >> 32), sn[i], cs[i]);
        sn[i] *= r.scale;
        cs[i] *= r.scale;
      }
    }
    const long long slot = r.slot ? (long long)r.slot[t] : 0;
    const bool stored = slot >= 0 && slot < a.slots;
    const long long page = (slot >> a.page_shift) * r.Hk, at = slot & ((1 << a.page_shift) - 1);
    for (int h0 = group * HPW + lane / TPH; h0 < a.heads; h0 += U * a.groups * HPW) {
      u32x4 x[U][2];
      char *to[U];
      int kind[U];  // 0: query, 1: key, 2: value, 3: nothing
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * a.groups * HPW;
        kind[u] = h < r.Hq ? 0 : h < r.Hq + r.Hk ? 1 : h < a.heads ? 2 : 3;
        const int g = h - (kind[u] == 0 ? 0 : kind[u] == 1 ? r.Hq : r.Hq + r.Hk);
        const char *from = kind[u] == 0 ? r.q + t * r.q_tok : kind[u] == 1 ? r.k + t * r.k_tok : r.v + t * r.v_tok;
        if (kind[u] == 0) to[u] = r.q_out + t * r.q_out_tok + g * ROWB;
        else if (!r.slot) to[u] = r.k_out + t * r.k_out_tok + g * ROWB;
        else to[u] = (kind[u] == 1 ? r.k_out : r.v_out) + (((page + g) << a.page_shift) + at) * ROWB;
        if (kind[u] != 0 && !stored) kind[u] = 3;
        if (kind[u] != 3) {
          x[u][0] = *reinterpret_cast<const u32x4 *>(from + g * ROWB + pa * (int)sizeof(T));
          x[u][1] = *reinterpret_cast<const u32x4 *>(from + g * ROWB + pb * (int)sizeof(T));
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float y[2 * E];
#pragma unroll
        for (int i = 0; i < 2 * E; ++i) {
          if constexpr (F32) y[i] = __builtin_bit_cast(f32x4, x[u][i / E])[i % E];
          else y[i] = (float)__builtin_bit_cast(bf16x8, x[u][i / E])[i % E];
        }
        const bool norm = kind[u] == 0 ? r.q_weight != nullptr : r.k_weight != nullptr;
        if (r.q_weight || r.k_weight) {  // (every lane of a head is here)
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * E; ++i) ss = __builtin_fmaf(y[i], y[i], ss);
          ss = over_head<TPH>(ss);
          const float f = norm ? 1.f / __builtin_sqrtf(ss / D + r.eps) : 1.f;
#pragma unroll
          for (int i = 0; i < 2 * E; ++i) y[i] = y[i] * f * (kind[u] == 0 ? wq[i] : wk[i]);
        }
        if (turned) {
#pragma unroll
          for (int i = 0; i < E; ++i) {
            float &p = HALF ? y[i] : y[2 * i], &q = HALF ? y[E + i] : y[2 * i + 1];
            const float u0 = p * cs[i] - q * sn[i], u1 = q * cs[i] + p * sn[i];
            p = u0;
            q = u1;
          }
        }
        if (kind[u] == 3) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          u32x4 o = x[u][j];
          if (kind[u] != 2) {
            if constexpr (F32) {
              o = __builtin_bit_cast(u32x4, f32x4{y[j * E], y[j * E + 1], y[j * E + 2], y[j * E + 3]});
            } else {
              bf16x8 b;
#pragma unroll
              for (int i = 0; i < E; ++i) b[i] = (__bf16)y[j * E + i];
              o = __builtin_bit_cast(u32x4, b);
            }
          }
          *reinterpret_cast<u32x4 *>(to[u] + (j == 0 ? pa : pb) * (int)sizeof(T)) = o;
        }
      }
    }
  }
}

template <typename T, int D>
hipError_t launch(hipStream_t st, NArgs a) {
  constexpr int HPW = 64 / (D * (int)sizeof(T) / 32);
  const int most = (a.heads + HPW - 1) / HPW;
  // a token's heads in one wave where tokens fill the chip, else spread over waves
  constexpr long long kWaves = 256 * 16;
  a.groups = 1;
  while (a.groups < most && a.r.n * a.groups < kWaves) ++a.groups;
  const long long tokens = a.r.n * a.groups < kWaves ? a.r.n : (kWaves + a.groups - 1) / a.groups;
  a.waves = tokens * a.groups;
  const dim3 grid((unsigned)((a.waves + kThreads / 64 - 1) / (kThreads / 64)));
  if (a.r.interleaved) hipLaunchKernelGGL((norm_rotary_kernel<T, D, false, 2>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((norm_rotary_kernel<T, D, true, 2>), grid, dim3(kThreads), 0, st, a);
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
