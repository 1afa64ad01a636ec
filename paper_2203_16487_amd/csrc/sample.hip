// A token per row of logits: temperature, top-k, top-p and min-p, drawn with a given random number.
//
// Weights w_i = exp((x_i - max x) / temperature).  In the order of falling logits (equal ones: lowest index first) the first top_k tokens
// stay, of these the first whose weights before them sum to less than top_p of all that top-k left, of these those with w_i >= min_p; the
// first one always stays.  Every rule keeps a leading part of the same order, so what stays is a smallest logit and how many of those
// equal to it.  The token drawn is the first one, in the order of the vocabulary, at which the sum of the weights that stay exceeds u of it.
// Weights are whole numbers, w 2^38 rounded to nearest from 64-bit floats, and their sums whole numbers of 64 bits: no order of
// summation changes a sum, so none changes a token.
#include "common.h"
#include "kernels.h"

namespace sd {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;
constexpr double kWeightOne = (double)(1ull << 38);   // (at most 2^24 tokens: sums stay below 2^62)
typedef unsigned long long u64;

// Logits as whole numbers of the same order; -0 as +0, NaN as -inf.
__device__ __forceinline__ unsigned order_key(float x) {
  if (x != x) x = kNegInf;
  const unsigned u = __builtin_bit_cast(unsigned, x + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k); }
constexpr unsigned kKeyNone = 0x007fffffu;   // of -inf

__device__ __forceinline__ double exponent(unsigned key, unsigned top, double inv_t) {   // (x - max) / temperature
  return key == top ? 0.0 : ((double)key_value(key) - (double)key_value(top)) * inv_t;
}
__device__ __forceinline__ u64 weight(unsigned key, unsigned top, double inv_t) {
  return key <= kKeyNone ? 0 : (u64)__double2ll_rn(exp(exponent(key, top, inv_t)) * kWeightOne);
}

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
struct Sums { u64 count, mass; };
__device__ __forceinline__ Sums block_sums(u64 count, u64 mass, u64 (*red)[2]) {
  count = wave_sum_u64(count);
  mass = wave_sum_u64(mass);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6][0] = count; red[threadIdx.x >> 6][1] = mass; }
  __syncthreads();
  Sums s{0, 0};
  for (int w = 0; w < kSampleWaves; ++w) { s.count += red[w][0]; s.mass += red[w][1]; }
  return s;
}

template <class E>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
  __shared__ u64 red[kSampleWaves][2];
  __shared__ u64 per[kSampleThreads];
  const int row = blockIdx.x, tid = threadIdx.x, V = a.vocab;
  const E* x = static_cast<const E*>(a.logits) + row * a.row_stride;
  // consecutive tokens a thread: what a thread holds is in the order of the vocabulary
  const int each = (V + kSampleThreads - 1) / kSampleThreads, lo = min(tid * each, V), hi = min(lo + each, V);
  unsigned top = 0;
  for (int i = lo; i < hi; ++i) top = max(top, order_key((float)x[i]));
  top = (unsigned)wave_max_i((int)(top ^ 0x80000000u)) ^ 0x80000000u;
  __syncthreads();
  if ((tid & 63) == 0) red[tid >> 6][0] = top;
  __syncthreads();
  for (int w = 0; w < kSampleWaves; ++w) top = max(top, (unsigned)red[w][0]);
  if (top <= kKeyNone) {   // nothing to draw from
    if (tid == 0) { a.token[row] = -1; if (a.logprob) a.logprob[row] = kNegInf; }
    return;
  }
  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  const bool greedy = !(temperature > 0.f);
  const double inv_t = greedy ? 0.0 : 1.0 / (double)temperature;
  const u64 k = a.top_k && a.top_k[row] > 0 ? a.top_k[row] : ~0ull;
  const double p = a.top_p ? (double)a.top_p[row] : 1.0, least = a.min_p ? (double)a.min_p[row] * kWeightOne : 0.0;
  auto above = [&](unsigned key) {   // of the tokens of larger logits
    u64 count = 0, mass = 0;
    for (int i = lo; i < hi; ++i) {
      const unsigned q = order_key((float)x[i]);
      if (q > key) { ++count; mass += weight(q, top, inv_t); }
    }
    return block_sums(count, mass, red);
  };
  // the smallest logit for which `stays` holds, which holds for all larger ones
  auto smallest = [&](auto stays) {
    unsigned in = top, out = kKeyNone;   // stays(in), nothing at out
    while (in - out > 1) {
      const unsigned mid = out + (in - out) / 2;
      if (stays(mid)) in = mid; else out = mid;
    }
    return in;
  };
  unsigned cut = top;
  u64 equal = 1;   // of those equal to it, the first ones that stay
  if (!greedy) {
    // top-k: tokens of logits >= kth, of those equal to it the first k - count
    const unsigned kth = smallest([&](unsigned key) { return above(key).count < k; });
    const Sums over = above(kth), with = above(kth - 1);
    const u64 wk = weight(kth, top, inv_t);
    const u64 rest = min(with.count - over.count, k - over.count);
    const u64 all = over.mass + rest * wk;
    const double reach = p < 1.0 ? p * (double)all : 2.0 * (double)all;   // (NaN: off)
    auto stays = [&](unsigned key) {
      if (key < kth) return false;
      if ((double)weight(key, top, inv_t) < least) return key == top;
      return key == top || (double)above(key).mass < reach;
    };
    cut = smallest(stays);
    const Sums o = above(cut);
    const u64 there = cut == kth ? rest : above(cut - 1).count - o.count, wc = weight(cut, top, inv_t);
    if (wc && reach < (double)(o.mass + there * wc)) {   // the first j with o.mass + j wc >= reach
      u64 j = o.mass > 0 || reach > 0.0 ? (u64)fmax(0.0, (reach - (double)o.mass) / (double)wc) : 0;
      while ((double)(o.mass + j * wc) < reach) ++j;
      while (j > 0 && (double)(o.mass + (j - 1) * wc) >= reach) --j;
      equal = min(there, j);
    } else {
      equal = there;
    }
    if (cut == top) {
      if ((double)wc < least) equal = 1;
      equal = max(equal, (u64)1);
    }
  }
  // the draw: prefix sums over the threads, first of the tokens equal to the cut, then of the weights that stay
  auto prefix = [&](u64 v, u64& total) {
    per[tid] = v;
    __syncthreads();
    u64 before = 0;
    total = 0;
    for (int i = 0; i < kSampleThreads; ++i) { if (i < tid) before += per[i]; total += per[i]; }
    __syncthreads();
    return before;
  };
  u64 ties = 0, dummy;
  for (int i = lo; i < hi; ++i) ties += order_key((float)x[i]) == cut;
  const u64 ties_before = prefix(ties, dummy);
  auto each_kept = [&](auto f) {
    u64 tie = ties_before;
    for (int i = lo; i < hi; ++i) {
      const unsigned q = order_key((float)x[i]);
      if (q > cut || (q == cut && tie++ < equal)) f(i, q);
    }
  };
  u64 mass = 0, Z;
  each_kept([&](int, unsigned q) { mass += weight(q, top, inv_t); });
  u64 sum = prefix(mass, Z);
  const double at = greedy ? 0.0 : (double)a.u[row] * (double)Z;
  const u64 target = at > 0.0 ? (at < (double)Z ? min((u64)at, Z - 1) : Z - 1) : 0;   // (u outside of [0, 1): the nearest end; NaN: the first)
  if (sum <= target && target < sum + mass) {
    bool done = false;
    each_kept([&](int i, unsigned q) {
      sum += weight(q, top, inv_t);
      if (!done && target < sum) {
        done = true;
        a.token[row] = i;
        if (a.logprob) a.logprob[row] = greedy ? 0.f : (float)(exponent(q, top, inv_t) - log((double)Z / kWeightOne));
      }
    });
  }
}

hipError_t sample(hipStream_t st, const SampleArgs& a) {
  if (a.dtype == 0) hipLaunchKernelGGL(sample_kernel<float>, dim3(a.rows), dim3(kSampleThreads), 0, st, a);
  else if (a.dtype == 1) hipLaunchKernelGGL(sample_kernel<bf16>, dim3(a.rows), dim3(kSampleThreads), 0, st, a);
  else hipLaunchKernelGGL(sample_kernel<f16>, dim3(a.rows), dim3(kSampleThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace sd
