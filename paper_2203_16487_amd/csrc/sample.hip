// A token per row of logits: temperature, top-k, top-p and min-p, drawn with a given random number.
//
// Weights w_i = exp((x_i - max x) / temperature).  In the order of falling logits (equal ones: lowest index first) the first top_k tokens
// stay, of these the first whose weights before them sum to less than top_p of all that top-k left, of these those with w_i >= min_p; the
// first one always stays.  Every rule keeps a leading part of the same order, so what stays is a smallest logit, which of those
// equal to it, and a smallest weight.  The token drawn is the first one, in the order of the vocabulary, at which the sum of the weights that
// stay exceeds u of their total.
// Weights are whole numbers, w 2^38 to less than one from 64-bit floats, and their sums whole numbers of 64 bits: no order of
// summation changes a sum, so none changes a token.  (fp32 weights put the end of a nucleus one token off in about one row of a thousand:
// sums are off by 1e-7, tokens at the end weigh 1e-4.)
//
// A workgroup a row, which is read once and stays in registers where it fits; every wave owns a consecutive part of it, so that the order
// of the vocabulary is the order of the waves.  The end of top-k and of top-p is found without sorting: logits are counted (or weighed) in
// kBuckets equal steps of max - x over the range in which weights are above zero, and the one step that holds the end is settled
// among its own tokens.  Few tokens that stay are sorted instead, and all the rest is done on them alone.
// Weights are formed where something depends on them: of all tokens only for top-p alone and for a plain draw.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace sd {

typedef unsigned long long u64;
typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int kBuckets = 2048, kList = 1024;
// Tokens that stay are sorted where top-k or a count gives at most kFew of them, and what looks among them is at most kShort.  Sorting costs the
// square of their number, the steps passes over the row: 1408 rows of 32768, top-k 120: 72 us sorted, 85 by steps; 200: 98 and 88 (96 rows of 131072: 28 and 59).
constexpr int kFew = 192, kShort = 512;
constexpr double kOne = (double)(1ull << 38);   // (at most 2^24 tokens: sums stay below 2^62)

// Logits as whole numbers of the same order.
__device__ __forceinline__ unsigned order_key(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k); }

// 2^38 2^t, 0 >= t = d * per >= -46, as a whole number: 2^f for the fractional part |f| <= 1/2 by the polynomial that meets it
// in nine Chebyshev nodes (relative error 2^-39.7), so off by less than one.  The whole part comes out of the low bits of t + 1.5 2^52, goes
// into the exponent, and 2^52 added rounds what is behind the point away: fifteen 64-bit instructions with what comes before, of 4 cycles as
// any other (counted: 53 vector instructions for 64 tokens of 1408 rows with top-p, one every 4 cycles for 89 % of the time).
__device__ __forceinline__ u64 fixed_exp2(double d, double per) {
  constexpr double M = 6755399441055744.0;
  const double m = __builtin_fma(d, per, M), f = __builtin_fma(d, per, -(m - M));
  double p = 1.325497460306718e-06;
  p = __builtin_fma(p, f, 1.531007807039615e-05);
  p = __builtin_fma(p, f, 0.00015403457039410448);
  p = __builtin_fma(p, f, 0.0013333450573018062);
  p = __builtin_fma(p, f, 0.009618129157656703);
  p = __builtin_fma(p, f, 0.055504109412010456);
  p = __builtin_fma(p, f, 0.24022650695821055);
  p = __builtin_fma(p, f, 0.6931471805459343);
  p = __builtin_fma(p, f, 0.9999999999999997);
  const u64 bits = __builtin_bit_cast(u64, p);
  const unsigned hi = (unsigned)(bits >> 32) + (((unsigned)__builtin_bit_cast(u64, m) + 38u) << 20);
  return __builtin_bit_cast(u64, __builtin_bit_cast(double, (u64)hi << 32 | (unsigned)bits) + 4503599627370496.0) & 0xfffffffffffffull;
}

// Sum over the wave, to every lane (the moves of wave_sum).
template <int CTRL>
__device__ __forceinline__ u64 dpp_u64(u64 v) {
  return (u64)(unsigned)dpp_i<CTRL>((int)(v >> 32)) << 32 | (unsigned)dpp_i<CTRL>((int)v);
}
__device__ __forceinline__ u64 lane_u64(u64 v, int lane) {
  return (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ u64 sum_u64(u64 v) {
  v += dpp_u64<kDppSwap1>(v);
  v += dpp_u64<kDppSwap2>(v);
  v += dpp_u64<kDppHalfMirror>(v);
  v += dpp_u64<kDppMirror>(v);
  return lane_u64(v, 0) + lane_u64(v, 16) + lane_u64(v, 32) + lane_u64(v, 48);
}
// Inclusive running sum over the lanes: within rows of 16 by shifts, then the last lane of a row into the rows behind it.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp_add_u64(u64 v) {
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
  const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
  return v + ((u64)hi << 32 | lo);
}
__device__ __forceinline__ u64 scan_u64(u64 v) {
  v = dpp_add_u64<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8
  v = dpp_add_u64<0x112, 0xf>(v);
  v = dpp_add_u64<0x114, 0xf>(v);
  v = dpp_add_u64<0x118, 0xf>(v);
  v = dpp_add_u64<0x142, 0xa>(v);   // lane 15 of rows 0, 2 into 1, 3
  return dpp_add_u64<0x143, 0xc>(v);   // lane 31 into rows 2, 3
}

// The values of four bytes.  (As instructions that are not merged with those of another pass.)
__device__ __forceinline__ void unpack(unsigned raw, float* v, float) { v[0] = __builtin_bit_cast(float, raw); }
__device__ __forceinline__ void unpack(unsigned raw, float* v, bf16) {
  asm volatile("v_lshlrev_b32 %0, 16, %1" : "=v"(v[0]) : "v"(raw));
  asm volatile("v_and_b32 %0, 0xffff0000, %1" : "=v"(v[1]) : "v"(raw));
}
__device__ __forceinline__ void unpack(unsigned raw, float* v, f16) {
  asm volatile("v_cvt_f32_f16 %0, %1" : "=v"(v[0]) : "v"(raw));
  asm volatile("v_cvt_f32_f16_sdwa %0, %1 src0_sel:WORD_1" : "=v"(v[1]) : "v"(raw));
}

// HOLD 16-byte pieces a lane in registers; 0: read again for every pass.
template <class E, int WAVES, int HOLD>
__global__ __launch_bounds__(64 * WAVES, 4) void sample_kernel(SampleArgs a) {
  constexpr int VEC = 16 / sizeof(E), THREADS = 64 * WAVES, EACH = kBuckets / THREADS;
  constexpr int GROUP = HOLD > 9 ? 3 : 1, PARTS = HOLD > 0 ? (HOLD + GROUP - 1) / GROUP : 1;   // rounds whose sums a lane keeps as one
  typedef E Vec __attribute__((ext_vector_type(VEC)));
  typedef unsigned Raw __attribute__((ext_vector_type(4)));
  __shared__ alignas(16) u64 mass[kBuckets];      // (of counts, where the end of top-k is looked for)
  __shared__ alignas(16) float list[kList];
  __shared__ alignas(16) u64 list_w[kList];
  __shared__ u64 red[4][WAVES];         // (a place for each use: none waits until another one has been read)
  __shared__ float red_f[2][WAVES];
  __shared__ unsigned list_n;
  __shared__ struct { u64 over, w; float value; unsigned equal; int bucket, index; } end;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.x, V = a.vocab;

  // the row in 16-byte pieces of `VEC` tokens that start before it where it is not aligned; a wave's are consecutive
  const E* x0 = static_cast<const E*>(a.logits) + row * a.row_stride;
  const int shift = (int)((reinterpret_cast<uintptr_t>(x0) & 15) / sizeof(E));
  const int rounds = (V + shift + THREADS * VEC - 1) / (THREADS * VEC), first = wave * rounds * 64 * VEC - shift;
  auto load = [&](int r) {
    const int i = first + (r * 64 + lane) * VEC;
    if (i >= 0 && i + VEC <= V) return *reinterpret_cast<const Raw*>(x0 + i);
    Vec v;
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = i + e >= 0 && i + e < V ? x0[i + e] : (E)kNegInf;
    return __builtin_bit_cast(Raw, v);
  };
  Raw held[HOLD > 0 ? HOLD : 1];
  if constexpr (HOLD > 0) {
#pragma unroll
    for (int r = 0; r < HOLD; ++r)
      if (r < rounds) held[r] = load(r);
  }
  for (int i = tid; i < kBuckets; i += THREADS) mass[i] = 0;
  if (tid == 0) list_n = 0;
  float top = kNegInf;
  bool inf_top = false;   // only the infinite ones count: as zeros among -inf
  auto values = [&](Raw raw, float (&v)[VEC]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack(raw[i], v + i * (VEC / 4), E());
    if (inf_top)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = v[e] == -kNegInf ? 0.f : kNegInf;
  };
  // f(round, the lane's values) for every round.  NaN are among them: every use is a comparison that fails for them.
  auto all = [&](auto f) {
    float v[VEC];
    if constexpr (HOLD > 0) {
#pragma unroll
      for (int r = 0; r < HOLD; ++r) {
        // (rounds are not mixed, and conversions do not outlive their pass: it would not fit the registers)
        if (r < rounds) { values(held[r], v); f(r, v); }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      constexpr int AHEAD = 4;
      Raw next[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) next[i] = load(min(i, rounds - 1));
#pragma unroll 1
      for (int r = 0; r < rounds; r += AHEAD)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const Raw now = next[i];
          next[i] = load(min(r + i + AHEAD, rounds - 1));
          if (r + i < rounds) { values(now, v); f(r + i, v); }
        }
    }
  };
  // the same in few instructions, where it is seldom done
  auto again = [&](auto f) {
    float v[VEC];
#pragma unroll 1
    for (int r = 0; r < rounds; ++r) { values(load(r), v); f(r, v); }
  };
  auto block_sum = [&](u64 v) {   // to everyone
    v = sum_u64(v);
    if (lane == 0) red[0][wave] = v;
    __syncthreads();
    u64 s = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) s += red[0][i];
    return s;
  };
  auto block_range = [&](float& hi, float& lo) {
    hi = wave_max(hi);
    lo = -wave_max(-lo);
    if (lane == 0) { red_f[0][wave] = hi; red_f[1][wave] = lo; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) { hi = fmaxf(hi, red_f[0][i]); lo = fminf(lo, red_f[1][i]); }
  };
  auto any = [](const float (&v)[VEC], auto is) {   // (one branch a piece)
    bool r = false;
#pragma unroll
    for (int e = 0; e < VEC; ++e) r |= is(v[e]);
    return r;
  };

  const float temperature = a.temperature ? a.temperature[row] : 1.f, p = a.top_p ? a.top_p[row] : 1.f, min_p = a.min_p ? a.min_p[row] : 0.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  all([&](int, float (&v)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) top = v[e] > top ? v[e] : top;
  });
  // The smallest of the maxima of k or more groups of lanes: k tokens are at least as large, and few others, so only they are counted for top-k.
  float among = -kNegInf;
  if (k > 0 && k <= THREADS) {
    float m = top;
    if (k <= THREADS / 4) { m = fmaxf(m, dpp_f<kDppSwap1>(m)); m = fmaxf(m, dpp_f<kDppSwap2>(m)); }
    if (k <= THREADS / 16) { m = fmaxf(m, dpp_f<kDppHalfMirror>(m)); m = fmaxf(m, dpp_f<kDppMirror>(m)); }
    among = m;
  }
  const bool few_k = k > 1 && k <= kFew && k < V;
  if (few_k) list[tid] = top;   // (the lane's own)
  block_range(top, among);
  if (among == -kNegInf) among = kNegInf;
  if (few_k) {   // closer, by one wave: by halves between that and the largest, a value that k lanes still reach
    if (wave == 0) {
      float lo = among, hi = top, of[WAVES];
#pragma unroll
      for (int i = 0; i < WAVES; ++i) of[i] = list[i * 64 + lane];
#pragma unroll 1
      for (int turn = 0; turn < 8; ++turn) {
        const float mid = lo + (hi - lo) * 0.5f;
        int c = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(of[i] >= mid));
        if (c >= k) lo = mid; else hi = mid;
      }
      if (lane == 0) end.value = lo;
    }
    __syncthreads();
    among = end.value;
  }

  if (top == kNegInf) {   // nothing to draw from
    if (tid == 0) { a.token[row] = -1; if (a.logprob) a.logprob[row] = kNegInf; }
    return;
  }
  if (top == -kNegInf) { inf_top = true; top = 0.f; }

  const bool alone = !(temperature > 0.f) || k == 1 || p <= 0.f || min_p > 1.f;   // the first token is all that stays
  const double inv_t = 1.0 / (double)temperature, per_x = fmax(inv_t * 1.44269504088896340736, 1e-300);
  const u64 least = min_p > 0.f ? (u64)ceil((double)min_p * kOne) : 0;
  // below floor_0 nothing weighs anything, below floor_x not `least`, by margins far beyond the rounding of these lines
  // (in 64 bits: the product passes the largest fp32 for temperatures from 1e37, which logits of the type's range can need)
  auto floor_of = [&](float nats) {
    return (float)fmax((double)top - 1.0001 * (double)temperature * ((double)nats + 1e-4) - 1e-6 * fabs((double)top), -3.4028234663852886e38);
  };
  auto nats_of = [](float w) { return 0.6931472f * (38.f - __builtin_amdgcn_logf(w)); };   // from the largest down to a weight
  const float floor_0 = floor_of(27.1f), floor_x = least > 0 ? floor_of(nats_of((float)least)) : floor_0;
  const double weightless = -46.0 / per_x;
  auto weight = [&](float x) {   // (four waves of a SIMD hide the chain's latency; several chains at once would not fit the registers)
    const u64 w = fixed_exp2(fmax((double)x - (double)top, weightless), per_x);
    __builtin_amdgcn_sched_barrier(0);
    return w;
  };

  // the first token, in the order of the vocabulary, at which the wave's sum of mine(value, index) exceeds `target`, which all of it does; part: the lane's
  // sums by groups of rounds, where they are known.  Called by one wave.
  auto find = [&](u64 target, const u64* part, auto mine, float& value) {
    float v[VEC];
    auto of_round = [&](int r) {
      const int i0 = first + (r * 64 + lane) * VEC;
      values(load(r), v);
      u64 t = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e) t += mine(v[e], i0 + e);
      return t;
    };
    int r = 0;
    if (HOLD > 0 && part) {
      bool got = false;
#pragma unroll
      for (int q = 0; q < PARTS; ++q)
        if (!got) {
          const u64 total = sum_u64(part[q]);
          if (target < total) { got = true; r = q * GROUP; } else target -= total;
        }
    }
    u64 s = 0;
    for (; r < rounds; ++r) {
      s = of_round(r);
      const u64 total = sum_u64(s);
      if (target < total) break;
      target -= total;
    }
    if (r >= rounds) return -1;   // (only if the logits change meanwhile)
    const u64 upto = scan_u64(s);
    const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > target));
    const int i0 = first + (r * 64 + lane) * VEC;
    u64 left = target - (upto - s);
    int at = -1;
    float val = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const u64 m = mine(v[e], i0 + e);
      if (at < 0 && left < m) { at = i0 + e; val = v[e]; }
      else left -= m;
    }
    value = __shfl(val, who);
    return __shfl(at, who);
  };

  // the cut: tokens above it stay, and those equal to it up to an index
  float cut = alone ? top : kNegInf;
  u64 equal = 1;
  bool some = alone;   // not all of those equal to it
  const bool by_k = !alone && k > 0 && k < V, by_p = !alone && p < 1.f;
  if (by_k || by_p) {
    // (2^-39 = exp(-27.03): what is beyond weighs nothing.  Not 0 however large the temperature: a difference beyond fp32 is infinite, and in the last step)
    const float steps = fmaxf(fminf((float)(kBuckets - 1) / (27.1f * temperature), 1e38f), 1e-37f);
    const float floor_k = fmaxf(by_p ? floor_0 : floor_x, by_k && !inf_top ? among : kNegInf);   // (what min-p drops counts for top-p)
    auto bucket = [&](float x) { return (int)fminf((top - x) * steps, (float)(kBuckets - 1)); };
    // Few of many: the tokens that top-k looks among, put in their order (each counts the ones before it); all the rest is done on them alone.
    // (One row of 32768 with top-k 50 and top-p: 19.6 us by the steps below, 10.2 so.  Four others a read: one a read 11.6, and top-k 120 of 1408 rows 101 us for 72.)
    // `lowest`: below it is none that stays; `most` tokens at most stay, and of them the first until the weights before one reach `need` (0: p of all these).
    auto sorted = [&](float lowest, int most, u64 need) __attribute__((always_inline)) {
      int* list_i = reinterpret_cast<int*>(list_w);
      all([&](int r, float (&v)[VEC]) {
        if (!any(v, [&](float x) { return x >= lowest; })) return;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v[e] >= lowest) {
            const unsigned at = atomicAdd(&list_n, 1u);
            if (at < kShort) { list[at] = v[e]; list_i[at] = first + (r * 64 + lane) * VEC + e; }
          }
      });
      __syncthreads();
      const int n = (int)list_n;
      if (n > kShort) return false;
      {
        constexpr int SHARE = THREADS / kShort;   // lanes of a token: each looks at a part of the others
        static_assert(SHARE == 1 || SHARE == 2, "");
        const int mine = tid / SHARE;
        float x = kNegInf;
        int xi = 0, rank = 0;
        if (mine < n) {
          x = list[mine];
          xi = list_i[mine];
          for (int j = 4 * (tid % SHARE); j < n; j += 4 * SHARE) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(list + j);
            const i32x4 yi = *reinterpret_cast<const i32x4*>(list_i + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) rank += (j + e < n) & ((y[e] > x) | ((y[e] == x) & (yi[e] < xi)));
          }
        }
        if (SHARE == 2) rank += dpp_i<kDppSwap1>(rank);
        float* order_x = reinterpret_cast<float*>(mass);
        int* order_i = reinterpret_cast<int*>(mass) + kShort;
        u64* order_w = mass + kShort;
        __syncthreads();   // (mass: cleared before, read by none)
        if (mine < n && tid % SHARE == 0 && rank < most) { order_x[rank] = x; order_i[rank] = xi; }
        __syncthreads();
        const int m = min(n, most);
        u64 w = 0;
        if (tid < m) { w = weight(order_x[tid]); order_w[tid] = w; }
        const u64 upto = scan_u64(w);
        if (lane == 63) red[1][wave] = upto;
        __syncthreads();
        u64 before = upto - w, Z = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) { before += i < wave ? red[1][i] : 0; Z += red[1][i]; }
        if (need == 0) need = by_p ? (u64)ceil((double)p * (double)Z) : ~0ull;
        const bool in = tid < m && (tid == 0 || (before < need && w >= least));
        const u64 kept_w = sum_u64(in ? w : 0), kept_n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(in));
        if (lane == 0) { red[2][wave] = kept_w; red[3][wave] = kept_n; }
        __syncthreads();
        int kept = 0;
        Z = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) { Z += red[2][i]; kept += (int)red[3][i]; }
        // in the order of the vocabulary: the sum before a token, by SHARE lanes of it
        const int t = tid / SHARE;
        u64 below = 0;
        int ti = 0;
        if (t < kept) {
          ti = order_i[t];
          for (int j = 4 * (tid % SHARE); j < kept; j += 4 * SHARE) {
            const i32x4 yi = *reinterpret_cast<const i32x4*>(order_i + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const u64 w = order_w[j + e];
              below += ((j + e < kept) & (yi[e] < ti)) ? w : 0;
            }
          }
        }
        if (SHARE == 2) below += dpp_u64<kDppSwap1>(below);
        const double at = (double)a.u[row] * (double)Z;
        const u64 target = at > 0.0 ? (at < (double)Z ? min((u64)at, Z - 1) : Z - 1) : 0;   // (as below)
        if (t < kept && tid % SHARE == 0 && below <= target && target < below + order_w[t]) {
          a.token[row] = ti;
          if (a.logprob) a.logprob[row] = (float)(((double)order_x[t] - (double)top) * inv_t - log((double)Z / kOne));
        }
      }
      return true;
    };
    // by more than the rounding of a bucket; the last step has no end
    auto lower_edge = [&](int step) { return step == kBuckets - 1 ? kNegInf : top - ((float)step + 1.01f) / steps - 1e-6f * fabsf(top); };
    if (by_k && few_k && sorted(floor_k, k, 0)) return;
    // the step in which the running sum reaches `need`, behind a barrier; false: none does
    auto locate = [&](u64 need) {
      u64 n[EACH], sum = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) { n[i] = mass[tid * EACH + i]; sum += n[i]; }
      const u64 upto = scan_u64(sum);
      if (lane == 63) red[1][wave] = upto;
      if (tid == 0) { end.bucket = -1; list_n = 0; }
      __syncthreads();
      u64 before = upto - sum;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) before += i < wave ? red[1][i] : 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (before < need && before + n[i] >= need) { end.bucket = tid * EACH + i; end.over = before; }
        before += n[i];
      }
      __syncthreads();
      return end.bucket >= 0;
    };
    // settles the end within that step: value, the sum of what is above it, how many equal it; each token counts one or its weight
    auto settle = [&](u64 need, bool weighed) {
      const int B = end.bucket;
      const u64 over = end.over;
      // (every value of the step, and few others: by more than the rounding of a bucket)
      const float wide = 1e-6f * fabsf(top), from = fmaxf(floor_k, lower_edge(B)), to = B == kBuckets - 1 ? top : top - ((float)B - 0.01f) / steps + wide;
      all([&](int, float (&v)[VEC]) {
        if (!any(v, [&](float x) { return x >= from && x <= to; })) return;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v[e] >= from && v[e] <= to && bucket(v[e]) == B) {
            const unsigned at = atomicAdd(&list_n, 1u);
            if (at < kList) list[at] = v[e];
          }
      });
      __syncthreads();
      const int n = (int)list_n;
      if (n <= kList) {
        for (int i = tid; i < n; i += THREADS) list_w[i] = weighed ? weight(list[i]) : 1;
        __syncthreads();
        for (int i = tid; i < n; i += THREADS) {
          const float x = list[i];
          u64 c = over;
          unsigned same = 0;
          for (int j = 0; j < n; ++j) {
            const float y = list[j];
            if (y > x) c += list_w[j];
            same += y == x;
          }
          const u64 w = list_w[i];
          if (c < need && c + same * w >= need) { end.value = x; end.over = c; end.equal = same; end.w = w; }   // (every thread of this value: the same)
        }
        __syncthreads();
        return;
      }
      // too many tokens in one step (equal ones, or logits far closer than the temperature): by halves of the keys between its ends
      float hi = kNegInf, lo = -kNegInf;
      again([&](int, float (&v)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v[e] > kNegInf && bucket(v[e]) == B) { hi = fmaxf(hi, v[e]); lo = fminf(lo, v[e]); }
      });
      block_range(hi, lo);
      auto above = [&](float x) {
        u64 c = 0;
        again([&](int, float (&v)[VEC]) {
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (v[e] > x && bucket(v[e]) == B) c += weighed ? weight(v[e]) : 1;
        });
        __syncthreads();
        return over + block_sum(c);
      };
      unsigned in = order_key(hi), out = order_key(lo) - 1;   // the end is the smallest key above which too little lies
      while (in - out > 1) {
        const unsigned mid = out + (in - out) / 2;
        if (above(key_value(mid)) < need) in = mid; else out = mid;
      }
      const float x = key_value(in);
      const u64 c = above(x);
      u64 same = 0;
      again([&](int, float (&v)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) same += v[e] == x;
      });
      __syncthreads();
      same = block_sum(same);
      if (tid == 0) { end.value = x; end.over = c; end.equal = (unsigned)same; end.w = weighed ? weight(x) : 1; }
      __syncthreads();
    };
    bool cut_k = false;
    if (by_k) {
      all([&](int, float (&v)[VEC]) {
        if (!any(v, [&](float x) { return x >= floor_k; })) return;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v[e] >= floor_k) atomicAdd(&mass[bucket(v[e])], 1ull);
      });
      __syncthreads();
      cut_k = locate(k);   // (fewer tokens of any weight, or of the least that stays, than k: all stay)
      if (cut_k) {
        settle(k, false);
        cut = end.value;
        equal = k - end.over;
        some = equal < end.equal;
      }
    }
    if (by_p) {
      if (by_k) {
        for (int i = tid; i < kBuckets; i += THREADS) mass[i] = 0;   // (behind the barriers of locate and settle)
        __syncthreads();
      }
      u64 sum = 0;
      if (cut_k) {   // of the tokens that top-k leaves
        if (tid == 0) {
          sum = equal * weight(cut);
          atomicAdd(&mass[bucket(cut)], sum);
        }
        all([&](int, float (&v)[VEC]) {
          if (!any(v, [&](float x) { return x > cut; })) return;
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (v[e] > cut) {
              const u64 w = weight(v[e]);
              sum += w;
              atomicAdd(&mass[bucket(v[e])], w);
            }
        });
      } else {       // of all: what weighs less than half of (1 - p) / V cannot reach the end and is only summed
        const float light = floor_of(nats_of(fmaxf(0.49f * (1.f - p) / (float)V * (float)kOne, 1.f)));
        all([&](int, float (&v)[VEC]) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const u64 w = weight(v[e]);
            sum += w;
            if (v[e] >= light) atomicAdd(&mass[bucket(v[e])], w);
          }
        });
      }
      const u64 need = (u64)ceil((double)p * (double)block_sum(sum));
      if (locate(need)) {
        if (!cut_k) {   // all before the end are above a lower edge, and often few: counted first (flat rows put thousands in a list for nothing)
          const float lowest = fmaxf(floor_0, lower_edge(end.bucket));
          unsigned many = 0;
          all([&](int, float (&v)[VEC]) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) many += v[e] >= lowest;
          });
          const u64 mine = sum_u64(many);
          if (lane == 0) red[2][wave] = mine;
          __syncthreads();
          u64 n = 0;
#pragma unroll
          for (int i = 0; i < WAVES; ++i) n += red[2][i];
          if (n <= kFew) {   // (1408 rows of 32768, top-p 0.9: 79 us so, 101 without)
            __syncthreads();   // (red[2] is written again)
            if (sorted(lowest, kShort, need)) return;
          }
        }
        settle(need, true);
        const u64 w = end.w, ties = cut_k && end.value == cut ? equal : end.equal;
        equal = min(ties, (need - end.over + w - 1) / w);
        cut = end.value;
        some = equal < end.equal;
      }
    }
  }

  // which of those equal to the cut
  int last = 0x7fffffff;
  if (some) {
    unsigned count = 0;
    all([&](int, float (&v)[VEC]) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) count += v[e] == cut;
    });
    const u64 ties = sum_u64(count);
    if (lane == 0) red[2][wave] = ties;
    __syncthreads();
    u64 before = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) before += i < wave ? red[2][i] : 0;
    if (equal - 1 >= before && equal - 1 < before + ties) {
      float unused;
      const int at = find(equal - 1 - before, nullptr, [&](float x, int) { return (u64)(x == cut); }, unused);
      if (lane == 0) end.index = at;
    }
    __syncthreads();
    last = end.index;
  }
  if (alone) {
    if (tid == 0) { a.token[row] = last; if (a.logprob) a.logprob[row] = 0.f; }
    return;
  }

  // the draw
  const float from = fmaxf(cut, floor_x);   // (finite: what is -inf or NaN is not above it)
  auto stays = [&](float x, int i) -> u64 {
    if (!(x >= from) || (x == cut && i > last)) return 0;
    const u64 w = weight(x);
    return w >= least ? w : 0;
  };
  u64 part[PARTS] = {}, mine = 0;
  const bool few = cut > kNegInf || least > 0;
  all([&](int r, float (&v)[VEC]) {
    u64 t = 0;
    if (!few) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) t += weight(v[e]);
    } else if (any(v, [&](float x) { return x >= from; })) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) t += stays(v[e], first + (r * 64 + lane) * VEC + e);
    }
    if (HOLD > 0) part[HOLD > 0 ? r / GROUP : 0] += t;
    mine += t;
  });
  mine = sum_u64(mine);
  if (lane == 0) red[3][wave] = mine;
  __syncthreads();
  u64 before = 0, Z = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) { before += i < wave ? red[3][i] : 0; Z += red[3][i]; }
  const double at = (double)a.u[row] * (double)Z;
  const u64 target = at > 0.0 ? (at < (double)Z ? min((u64)at, Z - 1) : Z - 1) : 0;   // (u outside of [0, 1): the nearest end; NaN: the first)
  if (target < before || target >= before + mine) return;
  float x = 0.f;
  const int token = find(target - before, HOLD > 0 ? part : nullptr, stays, x);
  if (lane == 0) {
    a.token[row] = token;
    if (a.logprob) a.logprob[row] = (float)(((double)x - (double)top) * inv_t - log((double)Z / kOne));
  }
}

template <class E>
static void sample_launch(hipStream_t st, const SampleArgs& a) {
  // Pieces of 16 bytes, one more than the row's where it is not aligned.  A row of up to 144 KB stays in registers: with the rows for it two a compute
  // unit, one loading while the other one computes; a few rows have more lanes each.
  const int pieces = (a.vocab * (int)sizeof(E) + 15) / 16 + 1;
  if (pieces <= 512 * 4) hipLaunchKernelGGL((sample_kernel<E, 8, 4>), dim3(a.rows), dim3(512), 0, st, a);
  else if (pieces <= 512 * 18 && a.rows > 256) hipLaunchKernelGGL((sample_kernel<E, 8, 18>), dim3(a.rows), dim3(512), 0, st, a);
  else if (pieces <= 1024 * 9) hipLaunchKernelGGL((sample_kernel<E, 16, 9>), dim3(a.rows), dim3(1024), 0, st, a);
  else hipLaunchKernelGGL((sample_kernel<E, 16, 0>), dim3(a.rows), dim3(1024), 0, st, a);
}

// (a grid has fewer than 2^32 threads in a dimension: 2^21 rows of up to 1024 threads a launch)
hipError_t sample(hipStream_t st, const SampleArgs& all) {
  constexpr int most = 1 << 21;
  for (int r0 = 0; r0 < all.rows; r0 += std::min(most, all.rows - r0)) {
    SampleArgs a = all;
    a.rows = std::min(most, all.rows - r0);
    a.logits = static_cast<const char*>(all.logits) + r0 * all.row_stride * (all.dtype == 0 ? 4 : 2);
    auto from = [r0](auto& p) { if (p) p += r0; };
    from(a.temperature); from(a.top_k); from(a.top_p); from(a.min_p); from(a.u); from(a.token); from(a.logprob);
    if (a.dtype == 0) sample_launch<float>(st, a);
    else if (a.dtype == 1) sample_launch<bf16>(st, a);
    else sample_launch<f16>(st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace sd
