// Sequences and rows of a cache moved in place.  What could overwrite a source before it is read lies within one workgroup, which holds
// everything it moves in registers: all its loads are done before its first store.
#include "common.h"
#include "kernels.h"

namespace sd {

constexpr int kMoveUnits = 8;   // 16-byte pieces a thread holds

// Every load of the workgroup has its value when this returns.
__device__ __forceinline__ void loads_done() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// A workgroup owns 2^shift consecutive pieces of one (layer, head) in every sequence: sequences exchange only what lies in the same place.
__global__ __launch_bounds__(1024) void fork_kernel(CacheSlabs c, int B, int n_src, const int* __restrict__ src, const int* __restrict__ len,
                                                    int per, int shift, int pieces) {
  const int plane = blockIdx.y, kv = plane & 1, z = plane >> 1, layer = z / c.heads, head = z - layer * c.heads;
  char* base = static_cast<char*>(kv ? c.v : c.k);
  if (!base) return;
  base += layer * c.layer_s + head * c.head_s;
  const long p0 = (long)blockIdx.x << shift;
  uint4 held[kMoveUnits];
  char* to[kMoveUnits];
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i) {
    const int u = i * (int)blockDim.x + (int)threadIdx.x, b = u >> shift;
    const long at = p0 + (u & ((1 << shift) - 1)), row = at / pieces;
    to[i] = nullptr;
    if (b >= B || row >= c.capacity) continue;
    const int s = src[b];
    if (s == b || s < 0 || s >= n_src || row * per >= len[s]) continue;
    const long off = row * c.row_s + (at - row * pieces) * 16;
    to[i] = base + b * c.seq_s + off;
    held[i] = *reinterpret_cast<const uint4*>(base + s * c.seq_s + off);
  }
  loads_done();
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i)
    if (to[i]) *reinterpret_cast<uint4*>(to[i]) = held[i];
}

hipError_t cache_fork(hipStream_t st, const CacheSlabs& c, int B, int n_src, const int* src, const int* len, int per) {
  const int threads = 1024, pieces = c.row_bytes / 16;
  int shift = 0;
  while (((long)B << (shift + 1)) <= (long)threads * kMoveUnits) ++shift;
  const long all = (long)c.capacity * pieces;
  const dim3 grid((unsigned)((all + (1l << shift) - 1) >> shift), (unsigned)(c.layers * c.heads * 2));
  hipLaunchKernelGGL(fork_kernel, grid, dim3(threads), 0, st, c, B, n_src, src, len, per, shift, pieces);
  return hipGetLastError();
}

// A workgroup owns whole (layer, head) slabs of one sequence, as many as it has pieces for: rows exchange only what lies in the same slab.
__global__ __launch_bounds__(256) void compact_kernel(CacheSlabs c, int n, const int* __restrict__ first, const int* __restrict__ path,
                                                      const int* __restrict__ count, int slabs, int pieces) {
  const int b = blockIdx.y, planes = c.layers * c.heads * (c.v ? 2 : 1), f = first[b], m = min(count[b], n);
  uint4 held[kMoveUnits];
  char* to[kMoveUnits];
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i) {
    int u = i * 256 + (int)threadIdx.x;
    const int slab = u / (n * pieces);
    u -= slab * n * pieces;
    const int plane = (int)blockIdx.x * slabs + slab, r = u / pieces;
    to[i] = nullptr;
    if (slab >= slabs || plane >= planes || r >= m) continue;
    const long dst = (long)f + r, row = (long)f + path[(size_t)b * n + r];
    if (row == dst || row < 0 || row >= c.capacity || dst < 0 || dst >= c.capacity) continue;
    const int z = c.v ? plane >> 1 : plane, layer = z / c.heads;
    char* base = static_cast<char*>(c.v && (plane & 1) ? c.v : c.k) + layer * c.layer_s + (z - layer * c.heads) * c.head_s + b * c.seq_s +
                 (u - r * pieces) * 16;
    to[i] = base + dst * c.row_s;
    held[i] = *reinterpret_cast<const uint4*>(base + row * c.row_s);
  }
  loads_done();
#pragma unroll
  for (int i = 0; i < kMoveUnits; ++i)
    if (to[i]) *reinterpret_cast<uint4*>(to[i]) = held[i];
}

hipError_t cache_compact(hipStream_t st, const CacheSlabs& c, int B, int n, const int* first, const int* path, const int* count) {
  static_assert(kCompactRows * (kCompactRowBytes / 16) <= 256 * kMoveUnits, "a slab's rows fit a workgroup");
  const int pieces = c.row_bytes / 16, slabs = 256 * kMoveUnits / (n * pieces), planes = c.layers * c.heads * (c.v ? 2 : 1);
  hipLaunchKernelGGL(compact_kernel, dim3((planes + slabs - 1) / slabs, B), dim3(256), 0, st, c, n, first, path, count, slabs, pieces);
  return hipGetLastError();
}

}  // namespace sd
