// Attention of the rows of a drafted tree over a cache.
//
// Sequence b has n_b cached keys / values and T_b rows of its own, whose keys / values lie behind them, at rows n_b + i of the same
// arena.  Row t sees every cached key and those rows i whose bit is set in visible[b][t] (a tree: itself and its ancestors):
//   o[b][t][h] = sum_s p_s v[b][s][h / G],  p = softmax over the visible s of scale * (q[b][t][h] . k[b][s][h / G]),  G = H / Hkv.
#include "common.h"
#include "kernels.h"

namespace sd {

template <class E> struct Pack;
template <> struct Pack<bf16> { typedef bf16 x8 __attribute__((ext_vector_type(8))); };
template <> struct Pack<f16> { typedef f16 x8 __attribute__((ext_vector_type(8))); };

// The simplest form: a wave a (sequence, row, query head), lanes over the head's dims, key after key with a running maximum and sum.
template <class E, int PER>
__global__ __launch_bounds__(64) void tree_attn_kernel(TreeAttnArgs a) {
  const int lane = threadIdx.x, h = blockIdx.x % a.H, t = blockIdx.x / a.H, b = blockIdx.y;
  const int rows = a.rows ? min(max(a.rows[b], 0), a.T) : a.T;
  if (t >= rows) return;
  const int n = a.cached[b];
  const bool fits = n >= 0 && n <= a.cap - rows;
  const int hk = h / (a.H / a.Hkv);
  const E* q = static_cast<const E*>(a.q) + b * a.q_s[0] + t * a.q_s[1] + h * a.q_s[2] + lane * PER;
  const E* k = static_cast<const E*>(a.k) + b * a.k_s[0] + hk * a.k_s[2] + lane * PER;
  const E* v = static_cast<const E*>(a.v) + b * a.v_s[0] + hk * a.v_s[2] + lane * PER;
  E* o = static_cast<E*>(a.o) + b * a.o_s[0] + t * a.o_s[1] + h * a.o_s[2] + lane * PER;
  const unsigned long long seen = a.visible ? a.visible[(size_t)b * a.T + t] : ~0ull >> (63 - t);
  float qv[PER], acc[PER], m = kNegInf, l = 0.f;
#pragma unroll
  for (int e = 0; e < PER; ++e) { qv[e] = (float)q[e] * a.scale; acc[e] = 0.f; }
  for (int s = 0; fits && s < n + rows; ++s) {
    if (s >= n && !(seen >> (s - n) & 1)) continue;
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) d += qv[e] * (float)k[s * a.k_s[1] + e];
    d = wave_sum(d);
    const float m2 = fmaxf(m, d), keep = m == kNegInf ? 0.f : __expf(m - m2), p = d == kNegInf ? 0.f : __expf(d - m2);
    l = l * keep + p;
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] = acc[e] * keep + p * (float)v[s * a.v_s[1] + e];
    m = m2;
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = (E)(l == 0.f ? 0.f : acc[e] / l);   // (nothing seen: zeros)
}

size_t tree_attn_bytes(const TreeAttnArgs&) { return 0; }

hipError_t tree_attn(hipStream_t st, const TreeAttnArgs& a) {
  const dim3 grid(a.T * a.H, a.B);
  if (a.f16) {
    if (a.dh == 128) hipLaunchKernelGGL((tree_attn_kernel<f16, 2>), grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL((tree_attn_kernel<f16, 1>), grid, dim3(64), 0, st, a);
  } else {
    if (a.dh == 128) hipLaunchKernelGGL((tree_attn_kernel<bf16, 2>), grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL((tree_attn_kernel<bf16, 1>), grid, dim3(64), 0, st, a);
  }
  return hipGetLastError();
}

// Masks of a tree from its rows' parents: a wave a sequence.  Row 0 is the root; row i (1 .. n) hangs on row parent[i - 1] < i and sees
// what that sees and itself.  A row whose parent is none of the rows before it, or has been left out, is left out: mask 0.
__global__ __launch_bounds__(64) void tree_visible_kernel(const int* __restrict__ parent, int n, unsigned long long* __restrict__ visible) {
  __shared__ unsigned long long mask[64];
  const int lane = threadIdx.x, b = blockIdx.x;
  const int p = lane >= 1 && lane <= n ? parent[(size_t)b * n + lane - 1] : -1;
  if (lane == 0) {
    mask[0] = 1;
    // (one lane: a row follows its parent)
  }
  for (int i = 1; i <= n; ++i) {
    const int pi = __builtin_amdgcn_readlane(p, i);
    __syncthreads();
    if (lane == 0) mask[i] = pi >= 0 && pi < i && mask[pi] ? mask[pi] | 1ull << i : 0ull;
  }
  __syncthreads();
  if (lane <= n) visible[(size_t)b * (n + 1) + lane] = mask[lane];
}
hipError_t tree_visible(hipStream_t st, const int* parent, int B, int n, unsigned long long* visible) {
  hipLaunchKernelGGL(tree_visible_kernel, dim3(B), dim3(64), 0, st, parent, n, visible);
  return hipGetLastError();
}

}  // namespace sd
