// A token per row of logits: temperature, top-k, top-p and min-p, drawn with a given random number.
//
// Weights w_i = exp((x_i - max x) / temperature).  In the order of falling logits (equal ones: lowest index first) the first top_k tokens
// stay, of these the first whose weights before them sum to less than top_p of all that top-k left, of these those with w_i >= min_p; the
// first one always stays.  Every rule keeps a leading part of the same order, so what stays is a smallest logit, which of those
// equal to it, and a smallest weight.  The token drawn is the first one, in the order of the vocabulary, at which the sum of the weights that
// stay exceeds u of their total.
// Weights are whole numbers, w 2^38 rounded to nearest from 64-bit floats, and their sums whole numbers of 64 bits: no order of
// summation changes a sum, so none changes a token.  (fp32 weights put the end of a nucleus one token off in about one row of a thousand:
// sums are off by 1e-7, tokens at the end weigh 1e-4.)
//
// A workgroup a row, which is read once and stays in registers where it fits; every wave owns a consecutive part of it, so that the order
// of the vocabulary is the order of the waves.  The end of top-k and of top-p is found without sorting: logits are counted (and weighed) in
// kBuckets equal steps of max - x over the range in which weights are above zero, and the one step that holds the end is settled
// among its own tokens.
#include "common.h"
#include "kernels.h"

namespace sd {

typedef unsigned long long u64;
constexpr int kBuckets = 2048, kList = 1024;
constexpr double kOne = (double)(1ull << 38);   // (at most 2^24 tokens: sums stay below 2^62)

// Logits as whole numbers of the same order.
__device__ __forceinline__ unsigned order_key(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k); }

// round(2^38 2^t), t <= 0: whole and fractional part, the series of exp(f ln 2) to the power 10 (|f| <= 1/2: 2e-13 off)
__device__ __forceinline__ u64 fixed_exp2(double t) {
  if (t < -40.0) return 0;
  constexpr double L = 0.69314718055994530942;
  constexpr double c2 = L * L / 2, c3 = c2 * L / 3, c4 = c3 * L / 4, c5 = c4 * L / 5, c6 = c5 * L / 6, c7 = c6 * L / 7, c8 = c7 * L / 8, c9 = c8 * L / 9, c10 = c9 * L / 10;
  const double n = __builtin_rint(t), f = t - n;
  double p = c10;
  p = __builtin_fma(p, f, c9); p = __builtin_fma(p, f, c8); p = __builtin_fma(p, f, c7); p = __builtin_fma(p, f, c6);
  p = __builtin_fma(p, f, c5); p = __builtin_fma(p, f, c4); p = __builtin_fma(p, f, c3); p = __builtin_fma(p, f, c2);
  p = __builtin_fma(p, f, L); p = __builtin_fma(p, f, 1.0);
  const double r = __builtin_ldexp(p, (int)n + 38) + 4503599627370496.0;   // (2^52: what is behind the point is rounded away)
  return __builtin_bit_cast(u64, r) & 0xfffffffffffffull;
}

__device__ __forceinline__ u64 shfl_u64(u64 v, int lane) { return __shfl(v, lane); }
__device__ __forceinline__ u64 sum_u64(u64 v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ u64 scan_u64(u64 v) {   // inclusive, over the lanes
  const int lane = threadIdx.x & 63;
  for (int o = 1; o < 64; o <<= 1) { const u64 x = __shfl_up(v, o); if (lane >= o) v += x; }
  return v;
}

// PER values a lane in registers; 0: read again for every pass.
template <class E, int WAVES, int PER>
__global__ __launch_bounds__(64 * WAVES) void sample_kernel(SampleArgs a) {
  constexpr int VEC = 16 / sizeof(E), HOLD = PER / VEC > 0 ? PER / VEC : 1, THREADS = 64 * WAVES, EACH = kBuckets / THREADS;
  typedef E Vec __attribute__((ext_vector_type(VEC)));
  __shared__ unsigned cnt[kBuckets];
  __shared__ u64 mass[kBuckets];
  __shared__ float list[kList];
  __shared__ u64 list_w[kList];
  __shared__ u64 red[2][WAVES];
  __shared__ unsigned list_n;
  __shared__ struct { u64 over_mass, w; float value; unsigned over, equal; int bucket, index; } end;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.x, V = a.vocab;

  // the row in 16-byte pieces of `VEC` tokens that start before it where it is not aligned; a wave's are consecutive
  const E* x0 = static_cast<const E*>(a.logits) + row * a.row_stride;
  const int shift = (int)((reinterpret_cast<uintptr_t>(x0) & 15) / sizeof(E));
  const int rounds = (V + shift + THREADS * VEC - 1) / (THREADS * VEC), first = wave * rounds * 64 * VEC - shift;
  auto load = [&](int r, float (&v)[VEC]) {
    const int i = first + (r * 64 + lane) * VEC;
    if (i >= 0 && i + VEC <= V) {
      const Vec p = *reinterpret_cast<const Vec*>(x0 + i);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = (float)p[e];
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = i + e >= 0 && i + e < V ? (float)x0[i + e] : kNegInf;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = v[e] == v[e] ? v[e] : kNegInf;
  };
  float held[HOLD][VEC];
  if constexpr (PER > 0) {
#pragma unroll
    for (int r = 0; r < HOLD; ++r)
      if (r < rounds) load(r, held[r]);
  }
  bool inf_top = false;
  auto get = [&](int r, float (&v)[VEC]) {   // (re-read)
    load(r, v);
    if (inf_top)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = v[e] == -kNegInf ? 0.f : kNegInf;
  };
  // f(round, the lane's values)
  auto all = [&](auto f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int r = 0; r < HOLD; ++r) {
        // (nothing that is formed of the values outlives its pass, and rounds are not mixed: both would take more registers than there are)
#pragma unroll
        for (int e = 0; e < VEC; ++e) asm volatile("" : "+v"(held[r][e]));
        if (r < rounds) f(r, held[r]);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      for (int r = 0; r < rounds; ++r) { float v[VEC]; get(r, v); f(r, v); }
    }
  };
  auto block_sum = [&](u64 v, u64 w, u64& sv, u64& sw) {   // both sums to everyone
    v = sum_u64(v);
    w = sum_u64(w);
    __syncthreads();
    if (lane == 0) { red[0][wave] = v; red[1][wave] = w; }
    __syncthreads();
    sv = sw = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) { sv += red[0][i]; sw += red[1][i]; }
  };

  float top = kNegInf, low = -kNegInf;
  all([&](int, float (&v)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) { top = fmaxf(top, v[e]); low = fminf(low, v[e] == kNegInf ? -kNegInf : v[e]); }
  });
  top = wave_max(top);
  low = -wave_max(-low);
  if (lane == 0) red[0][wave] = (u64)__builtin_bit_cast(unsigned, top) << 32 | __builtin_bit_cast(unsigned, low);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    top = fmaxf(top, __builtin_bit_cast(float, (unsigned)(red[0][i] >> 32)));
    low = fminf(low, __builtin_bit_cast(float, (unsigned)red[0][i]));
  }
  if (top == kNegInf) {   // nothing to draw from
    if (tid == 0) { a.token[row] = -1; if (a.logprob) a.logprob[row] = kNegInf; }
    return;
  }
  if (top == -kNegInf) {   // only the infinite ones count: as zeros among -inf
    inf_top = true;
    top = low = 0.f;
    if constexpr (PER > 0) {
#pragma unroll
      for (int r = 0; r < HOLD; ++r)
#pragma unroll
        for (int e = 0; e < VEC; ++e) held[r][e] = held[r][e] == -kNegInf ? 0.f : kNegInf;
    }
  }

  const float temperature = a.temperature ? a.temperature[row] : 1.f, p = a.top_p ? a.top_p[row] : 1.f, min_p = a.min_p ? a.min_p[row] : 0.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  const bool alone = !(temperature > 0.f) || k == 1 || p <= 0.f || min_p > 1.f;   // the first token is all that stays
  const double inv_t = 1.0 / (double)temperature, per_x = fmax(inv_t * 1.44269504088896340736, 1e-300);
  auto weight = [&](float x) {
    const u64 w = fixed_exp2(((double)x - (double)top) * per_x);
    __builtin_amdgcn_sched_barrier(0);
    return w;
  };
  const u64 least = min_p > 0.f ? (u64)ceil((double)min_p * kOne) : 0;

  // the f-th token, in the order of the vocabulary, that a wave's `mine`(x, index) counts add up to: its index; called by one wave
  auto find = [&](u64 target, auto mine, float& value) {
    int found = -1;
    auto look = [&](int r, float (&v)[VEC]) {
      if (found >= 0) return;
      const int i0 = first + (r * 64 + lane) * VEC;
      u64 m[VEC], s = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e) { m[e] = mine(v[e], i0 + e); s += m[e]; }
      const u64 upto = scan_u64(s), total = shfl_u64(upto, 63);
      if (target >= total) { target -= total; return; }
      const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > target));
      u64 left = target - (upto - s);
      int at = -1;
      float val = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (at < 0 && left < m[e]) { at = i0 + e; val = v[e]; }
        else left -= m[e];
      }
      found = __shfl(at, who);
      value = __shfl(val, who);
    };
    all(look);
    return found;
  };

  // the cut: tokens above it stay, and those equal to it up to an index
  float cut = alone ? top : kNegInf;
  u64 equal = 1;
  bool some = alone;   // not all of those equal to it
  const bool by_k = !alone && k > 0 && k < V, by_p = !alone && p < 1.f;
  if (by_k || by_p) {
    const float range = fminf(27.1f * temperature, (top - low) * 1.001f);   // (2^-39 = exp(-27.03))
    const float steps = (float)(kBuckets - 1) / range;
    auto bucket = [&](float x) {
      const float d = top - x;
      return d > 0.f ? (int)fminf(d * steps, (float)(kBuckets - 1)) : 0;
    };
    for (int i = tid; i < kBuckets; i += THREADS) { cnt[i] = 0; mass[i] = 0; }
    if (tid == 0) list_n = 0;
    __syncthreads();
    // (by top-p alone: what weighs less than half of (1 - p) / V cannot reach its end)
    const u64 light = by_p && !by_k ? (u64)(0.5 * (1.0 - (double)p) / V * kOne) : 0;
    u64 sum = 0, Z, dummy;
    all([&](int, float (&v)[VEC]) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int b = bucket(v[e]);
        if (by_p) {
          const u64 w = weight(v[e]);
          sum += w;
          if (w > light) atomicAdd(&mass[b], w);
          if (by_k && w > 0) atomicAdd(&cnt[b], 1u);
        } else if (b < kBuckets - 1) {   // (the last step: weights of zero)
          atomicAdd(&cnt[b], 1u);
        }
      }
    });
    if (by_p) block_sum(sum, 0, Z, dummy);
    else __syncthreads();
    // the step in which the running count reaches `need_n`, or the running weight `need_w`; false: none does
    auto locate = [&](u64 need_n, u64 need_w) {
      u64 n = 0, w = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) { n += cnt[tid * EACH + i]; w += mass[tid * EACH + i]; }
      const u64 un = scan_u64(n), uw = scan_u64(w);
      __syncthreads();
      if (lane == 63) { red[0][wave] = un; red[1][wave] = uw; }
      if (tid == 0) end.bucket = -1;
      __syncthreads();
      u64 bn = un - n, bw = uw - w;
      for (int i = 0; i < wave; ++i) { bn += red[0][i]; bw += red[1][i]; }
      if (bn < need_n && bw < need_w && (bn + n >= need_n || bw + w >= need_w)) {
        for (int i = 0; i < EACH; ++i) {
          const u64 cn = cnt[tid * EACH + i], cw = mass[tid * EACH + i];
          if (bn + cn >= need_n || bw + cw >= need_w) { end.bucket = tid * EACH + i; end.over = (unsigned)bn; end.over_mass = bw; break; }
          bn += cn; bw += cw;
        }
      }
      __syncthreads();
      return end.bucket >= 0;
    };
    // settles the end within that step: value, what is above it, how many equal it
    auto settle = [&](u64 need_n, u64 need_w) {
      const int B = end.bucket;
      const u64 over = end.over, over_mass = end.over_mass;
      __syncthreads();
      if (tid == 0) list_n = 0;
      __syncthreads();
      all([&](int, float (&v)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v[e] > kNegInf && bucket(v[e]) == B) {
            const unsigned at = atomicAdd(&list_n, 1u);
            if (at < kList) { list[at] = v[e]; list_w[at] = weight(v[e]); }
          }
      });
      __syncthreads();
      const int n = (int)list_n;
      if (n <= kList) {
        for (int i = tid; i < n; i += THREADS) {
          const float x = list[i];
          u64 cn = over, cw = over_mass;
          unsigned same = 0;
          for (int j = 0; j < n; ++j) {
            const float y = list[j];
            if (y > x) { ++cn; cw += list_w[j]; }
            same += y == x;
          }
          const u64 w = list_w[i];
          if (cn < need_n && cw < need_w && (cn + same >= need_n || cw + same * w >= need_w)) {   // (every thread of this value: the same)
            end.value = x; end.over = (unsigned)cn; end.over_mass = cw; end.equal = same; end.w = w;
          }
        }
        __syncthreads();
        return;
      }
      // too many tokens in one step (equal ones, or logits far closer than the temperature): by halves of the keys between its ends
      float hi = kNegInf, lo = -kNegInf;
      all([&](int, float (&v)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v[e] > kNegInf && bucket(v[e]) == B) { hi = fmaxf(hi, v[e]); lo = fminf(lo, v[e]); }
      });
      hi = wave_max(hi);
      lo = -wave_max(-lo);
      __syncthreads();
      if (lane == 0) red[0][wave] = (u64)__builtin_bit_cast(unsigned, hi) << 32 | __builtin_bit_cast(unsigned, lo);
      __syncthreads();
      for (int i = 0; i < WAVES; ++i) {
        hi = fmaxf(hi, __builtin_bit_cast(float, (unsigned)(red[0][i] >> 32)));
        lo = fminf(lo, __builtin_bit_cast(float, (unsigned)red[0][i]));
      }
      auto above = [&](float x, u64& cn, u64& cw) {
        u64 c = 0, w = 0;
        all([&](int, float (&v)[VEC]) {
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (v[e] > x && bucket(v[e]) == B) { ++c; w += weight(v[e]); }
        });
        block_sum(c, w, cn, cw);
        cn += over; cw += over_mass;
      };
      unsigned in = order_key(hi), out = order_key(lo) - 1;   // the end is the smallest key above which too little lies
      u64 cn, cw;
      while (in - out > 1) {
        const unsigned mid = out + (in - out) / 2;
        above(key_value(mid), cn, cw);
        if (cn < need_n && cw < need_w) in = mid; else out = mid;
      }
      const float x = key_value(in);
      above(x, cn, cw);
      u64 same = 0, d0;
      all([&](int, float (&v)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) same += v[e] == x;
      });
      block_sum(same, 0, same, d0);
      if (tid == 0) { end.value = x; end.over = (unsigned)cn; end.over_mass = cw; end.equal = (unsigned)same; end.w = weight(x); }
      __syncthreads();
    };
    const u64 never = ~0ull;
    bool cut_k = false;
    if (by_k && locate(k, never)) {   // (fewer tokens of any weight than k: all stay)
      if (by_p) {   // (its weights are summed: what of them k leaves)
        settle(k, never);
        Z = end.over_mass + (k - end.over) * end.w;
      } else {
        settle(k, never);
      }
      cut_k = true;
      cut = end.value;
      equal = k - end.over;
      some = equal < end.equal;
    }
    if (by_p) {
      const double reach = (double)p * (double)Z;
      const u64 need = (u64)ceil(reach);
      __syncthreads();
      if (locate(never, need)) {
        settle(never, need);
        const u64 w = end.w, ties = cut_k && end.value == cut ? equal : end.equal;
        const u64 stay = min(ties, (need - end.over_mass + w - 1) / w);
        cut = end.value;
        equal = stay;
        some = stay < end.equal;
      }
    }
  }

  // which of those equal to the cut
  int last = 0x7fffffff;
  float unused;
  if (some) {
    u64 ties = 0;
    all([&](int, float (&v)[VEC]) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) ties += v[e] == cut;
    });
    ties = sum_u64(ties);
    __syncthreads();
    if (lane == 0) red[0][wave] = ties;
    __syncthreads();
    u64 before = 0;
    for (int i = 0; i < wave; ++i) before += red[0][i];
    if (equal - 1 >= before && equal - 1 < before + ties) {
      const int at = find(equal - 1 - before, [&](float x, int) { return (u64)(x == cut); }, unused);
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
  auto stays = [&](float x, int i) -> u64 {
    if (!(x > cut || (x == cut && x > kNegInf && i <= last))) return 0;
    const u64 w = weight(x);
    return w >= least ? w : 0;
  };
  u64 mine = 0;
  all([&](int r, float (&v)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) mine += stays(v[e], first + (r * 64 + lane) * VEC + e);
  });
  mine = sum_u64(mine);
  __syncthreads();
  if (lane == 0) red[0][wave] = mine;
  __syncthreads();
  u64 before = 0, Z = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) { if (i < wave) before += red[0][i]; Z += red[0][i]; }
  const double at = (double)a.u[row] * (double)Z;
  const u64 target = at > 0.0 ? (at < (double)Z ? min((u64)at, Z - 1) : Z - 1) : 0;   // (u outside of [0, 1): the nearest end; NaN: the first)
  if (target < before || target >= before + mine) return;
  float x = 0.f;
  const int token = find(target - before, stays, x);
  if (lane == 0) {
    a.token[row] = token;
    if (a.logprob) a.logprob[row] = (float)(((double)x - (double)top) * inv_t - log((double)Z / kOne));
  }
}

template <class E>
static void sample_launch(hipStream_t st, const SampleArgs& a) {
  // (a piece more than the row's where it is not aligned)
  const int room = a.vocab + 16 / (int)sizeof(E) - 1;
  if (room <= 512 * 16) hipLaunchKernelGGL((sample_kernel<E, 8, 16>), dim3(a.rows), dim3(512), 0, st, a);
  else if (room <= 1024 * 32 + 16) hipLaunchKernelGGL((sample_kernel<E, 16, 32 + 16 / sizeof(E)>), dim3(a.rows), dim3(1024), 0, st, a);
  else hipLaunchKernelGGL((sample_kernel<E, 16, 0>), dim3(a.rows), dim3(1024), 0, st, a);
}

hipError_t sample(hipStream_t st, const SampleArgs& a) {
  if (a.dtype == 0) sample_launch<float>(st, a);
  else if (a.dtype == 1) sample_launch<bf16>(st, a);
  else sample_launch<f16>(st, a);
  return hipGetLastError();
}

}  // namespace sd
