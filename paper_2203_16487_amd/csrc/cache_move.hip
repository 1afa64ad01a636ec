// Sequences and rows of a cache moved in place.  What could overwrite a source before it is read lies within one workgroup, which holds
// everything it moves in registers: all its loads are done before its first store.
#include "common.h"
#include "kernels.h"

namespace sd {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
constexpr int kMoveUnits = 8;   // 16-byte pieces a thread holds

// Every load of the workgroup has its value when this returns.
__device__ __forceinline__ void loads_done() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// A workgroup owns 2^shift consecutive pieces of one (layer, head) in every sequence: sequences exchange only what lies in the same place.
// `pieces` of them are a row; 0: rows follow each other without gaps (`of_row` pieces each) and no place has to be taken apart.
// WAVE: a wave's pieces are one sequence's (2^shift >= 64): what is asked of a sequence is read with scalar loads.
template <bool WAVE>
__global__ __launch_bounds__(1024) void fork_kernel(CacheSlabs c, int B, int n_src, const int* __restrict__ src, const int* __restrict__ len,
                                                    int per, int shift, unsigned pieces, unsigned of_row) {
  const int plane = blockIdx.y, kv = plane & 1, z = plane >> 1, layer = z / c.heads, head = z - layer * c.heads;
  char* base = static_cast<char*>(kv ? c.v : c.k);
  if (!base) return;
  base += layer * c.layer_s + head * c.head_s;
  const unsigned p0 = blockIdx.x << shift;
  int to[kMoveUnits], from[kMoveUnits];   // (from < 0: nothing to move)
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i) {
    int b = (i * (int)blockDim.x + (int)threadIdx.x) >> shift;
    if (WAVE) b = __builtin_amdgcn_readfirstlane(b);
    to[i] = b;
    from[i] = b < B ? src[b] : -1;
  }
  long rows[kMoveUnits];
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i) {
    if (from[i] == to[i] || (unsigned)from[i] >= (unsigned)n_src) from[i] = -1;
    rows[i] = from[i] < 0 ? 0 : min(((long)len[from[i]] + per - 1) / per, (long)c.capacity);
  }
  auto offset = [&](int i, unsigned& at) {
    at = p0 + ((i * blockDim.x + threadIdx.x) & ((1u << shift) - 1));
    if (!pieces) return at * 16l;
    const unsigned row = at / pieces;
    return row * c.row_s + (at - row * pieces) * 16l;
  };
  u32x4 held[kMoveUnits];
  bool moves[kMoveUnits];
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i) {
    unsigned at;
    const long off = offset(i, at);
    moves[i] = (long)at < rows[i] * of_row;
    held[i] = *reinterpret_cast<const u32x4*>(base + (moves[i] ? from[i] * c.seq_s + off : 0));   // (no branch: all requests go out at once)
  }
  loads_done();
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i) {
    unsigned at;
    if (moves[i]) *reinterpret_cast<u32x4*>(base + to[i] * c.seq_s + offset(i, at)) = held[i];
  }
}

hipError_t cache_fork(hipStream_t st, CacheSlabs c, int B, int n_src, const int* src, const int* len, int per) {
  if (c.heads > 1 && c.head_s == c.row_bytes && c.row_s >= (long)c.row_bytes * c.heads) {   // the heads' rows lie beside each other: one long row
    c.row_bytes *= c.heads;
    c.heads = 1;
  }
  const int threads = B <= 32 ? 256 : B <= 64 ? 512 : 1024, pieces = c.row_bytes / 16;   // (at least 1 KB of a sequence, up to 128 of them)
  int shift = 0;
  while (((long)B << (shift + 1)) <= (long)threads * kMoveUnits) ++shift;
  const long all = (long)c.capacity * pieces;
  if (all >= 1l << 31) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((all + (1l << shift) - 1) >> shift), (unsigned)(c.layers * c.heads * 2));
  hipLaunchKernelGGL(shift >= 6 ? fork_kernel<true> : fork_kernel<false>, grid, dim3(threads), 0, st, c, B, n_src, src, len, per, shift, c.row_s == c.row_bytes ? 0u : (unsigned)pieces, (unsigned)pieces);
  return hipGetLastError();
}

// A workgroup owns whole (layer, head) slabs of one sequence, as many as it has pieces for: rows exchange only what lies in the same slab.
// A thread has one piece (of `wide` = 2^shift pieces of all the workgroup's slabs side by side) of every 256 / wide-th row of the path.
// Bound by round trips: what depends on nothing is read first, all at once.
__global__ __launch_bounds__(256) void compact_kernel(CacheSlabs c, int n, const int* __restrict__ first, const int* __restrict__ path,
                                                      const int* __restrict__ count, int shift, int pieces) {
  const int b = blockIdx.y, planes = c.layers * c.heads * (c.v ? 2 : 1), w = (int)threadIdx.x & ((1 << shift) - 1), r0 = (int)threadIdx.x >> shift, step = 256 >> shift;
  const int f = first[b], m = min(count[b], n);
  int from[kMoveUnits];
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i) {
    const int r = r0 + i * step;
    from[i] = r < n ? path[(size_t)b * n + r] : 0;
  }
  const int slab = w / pieces, slabs = (1 << shift) / pieces, plane = (int)blockIdx.x * slabs + slab;
  if (slab >= slabs || plane >= planes) return;   // (with whole slabs: whoever moves rows of one meets below)
  const int z = c.v ? plane >> 1 : plane, layer = z / c.heads;
  char* base = static_cast<char*>(c.v && (plane & 1) ? c.v : c.k) + layer * c.layer_s + (z - layer * c.heads) * c.head_s + b * c.seq_s + (w - slab * pieces) * 16;
  u32x4 held[kMoveUnits];
  bool moves[kMoveUnits];
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i) {
    const int r = r0 + i * step;
    const long dst = (long)f + r, row = (long)f + from[i];
    moves[i] = r < m && row != dst && row >= 0 && row < c.capacity && dst >= 0 && dst < c.capacity;
    held[i] = *reinterpret_cast<const u32x4*>(base + (moves[i] ? row * c.row_s : 0));   // (no branch: all requests go out at once)
  }
  loads_done();
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i)
    if (moves[i]) *reinterpret_cast<u32x4*>(base + ((long)f + r0 + i * step) * c.row_s) = held[i];
}

hipError_t cache_compact(hipStream_t st, const CacheSlabs& c, int B, int n, const int* first, const int* path, const int* count) {
  static_assert(kCompactRows * (kCompactRowBytes / 16) <= 256 * kMoveUnits, "a slab's rows fit a workgroup");
  const int pieces = c.row_bytes / 16, planes = c.layers * c.heads * (c.v ? 2 : 1);
  int shift = 8;
  while ((n << shift) > 256 * kMoveUnits) --shift;
  const int slabs = (1 << shift) / pieces;
  hipLaunchKernelGGL(compact_kernel, dim3((planes + slabs - 1) / slabs, B), dim3(256), 0, st, c, n, first, path, count, shift, pieces);
  return hipGetLastError();
}

}  // namespace sd
