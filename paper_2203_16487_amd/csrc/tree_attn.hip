// Attention of the rows of a drafted tree over a cache.
//
// Sequence b has n_b cached keys / values and T_b rows of its own, whose keys / values lie behind them, at rows n_b + i of the same
// arena.  Row t sees every cached key and those rows i whose bit is set in visible[b][t] (a tree: itself and its ancestors):
//   o[b][t][h] = sum_s p_s v[b][s][h / G],  p = softmax over the visible s of scale * (q[b][t][h] . k[b][s][h / G]),  G = H / Hkv.
//
// The G query heads of the T rows that share a key head are the G T columns of one pair of products, so a key and a value are read from
// memory once for all of them (once per block of 32 RW columns, from L2).  A workgroup takes tiles of KT keys through LDS, two buffers, the
// next tile's direct loads under way while this one is multiplied; its waves are RW groups of 32 columns times KW parts of a tile's keys.
// Scores are formed as S^T = K Q^T in 32 x 32 tiles: a lane then holds 16 keys of one column, the running maximum and sum are a lane's own up
// to one exchange of the wave's halves, and the weights are already the second operand of O^T += V^T P^T (the order in which keys are
// summed is free, so both operands take the one that S^T has).  V^T comes out of LDS by transposing reads.
#include <atomic>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace sd {

typedef unsigned long long u64;
typedef short s16x8 __attribute__((ext_vector_type(8)));

// What differs between the element types.  A column's reference (the running maximum of a softmax) follows its scores only when they exceed it by
// kSlack powers of two: sums are rescaled seldom.  kLift: weights are stored as 2^kLift exp2(s - reference), so that fp16, whose values end
// at 2^-24, keeps weights down to 2^-37 of the largest (without it 65536 keys of 2^-25 each would be lost) and none reaches 2^16.
template <class E> struct AttnType;
template <> struct AttnType<bf16> {
  typedef bf16 x8 __attribute__((ext_vector_type(8)));
  static constexpr float kLift = 0.f, kSlack = 8.f;
  static constexpr unsigned kExp = 0x7f807f80u, kUnit = 0x00800080u;
  static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
};
template <> struct AttnType<f16> {
  typedef f16 x8 __attribute__((ext_vector_type(8)));
  static constexpr float kLift = 13.f, kSlack = 2.f;
  static constexpr unsigned kExp = 0x7c007c00u, kUnit = 0x04000400u;
  static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
};

// How a call is cut: blocks of 32 rw columns, tiles of kt keys; split: the tiles of a column block are dealt out in chunks of a length
// that gives about `target` workgroups in all, whatever the lengths are (the workgroups work it out: the host does not know them), each
// leaves its maximum, sum and unnormalised output in a slot of the workspace, and tree_join_kernel adds them up.
// Rules, by what both sides take (us in a graph).  Split arenas of more than 1024 rows: the second launch costs 3.5, and one workgroup takes 9 for 700 keys
// of 16 heads (split 14), 1500 keys of two sequences of 8 heads 15.  Up to 32 columns on 128 keys a tile and four waves where a call is short (one token on
// 224 keys 5.3, on 64 keys and two waves 6.5), on 64 and two where it is long and heads have 128 dims, so that two workgroups are on a compute unit
// (65536 keys 92 / 78).  Chunks that fill the GPU once where the column blocks are fewer than three quarters of that, else twice as many, so that
// long sequences are cut (16 long ragged trees 225, chunks that begin a second round, / 186).
// Every workgroup goes over all sequences: little up to 64, whose lengths stay in a register, and most of the time beyond some hundred (one token, 8 heads
// of 64, 64 - 1000 keys, in arenas of 1088 rows and, not split, of 1024: 64 sequences 28 / 16, 256 94 / 48, 1024 651 / 195, 4096 6841 / 725).
struct TreePlan {
  int rw, kw, kt, row_blocks, target, slots;
  bool split;
};
constexpr int kSplitTarget = 512;   // workgroups that run at once: two a compute unit
// The workspace of a split call: tiles of a chunk, the first slot of every sequence (written by the first workgroup for tree_join_kernel); the slots.
__host__ __device__ static constexpr size_t tree_head_ints(int B) { return ((size_t)B + 1 + 63) / 64 * 64; }
static TreePlan tree_plan(const TreeAttnArgs& a) {
  TreePlan p;
  const int m = a.H / a.Hkv * a.T;
  p.rw = m <= 32 ? 1 : m <= 64 ? 2 : 4;
  p.split = a.cap > 1024;
  p.kw = p.rw == 4 ? 1 : p.rw == 2 || (p.split && a.dh == 128) ? 2 : 4;
  p.kt = p.kw == 4 ? 128 : 64;
  p.row_blocks = (m + 32 * p.rw - 1) / (32 * p.rw);
  const long whole = (long)a.B * a.Hkv * p.row_blocks;
  p.target = whole <= kSplitTarget * 3 / 4 ? kSplitTarget : 2 * kSplitTarget;
  p.slots = (int)(p.split ? p.target + whole : whole);
  return p;
}

// One sequence: rows there are, tiles, column blocks.
struct TreeSeq { int n, rows, tiles, blocks; };
__device__ __forceinline__ TreeSeq tree_seq(const TreeAttnArgs& a, const TreePlan& p, int b) {
  TreeSeq s;
  s.rows = a.rows ? min(max(a.rows[b], 0), a.T) : a.T;
  s.n = a.cached[b];
  if (s.n < 0 || s.n > a.cap - s.rows) s.n = -1;   // (no room for the rows: they see nothing)
  s.tiles = s.n < 0 ? 1 : (s.n + s.rows + p.kt - 1) / p.kt;
  s.blocks = (a.H / a.Hkv * s.rows + 32 * p.rw - 1) / (32 * p.rw);
  return s;
}

// Where a workgroup's work lies: chunk `chunk` of `chunks` of `per` tiles, in slot `slot`.
struct TreeWork { int b, hk, block, chunk, chunks, per, slot; bool none; };

__device__ __forceinline__ int wave_sum_i(int v) {   // (the moves of wave_sum)
  v += dpp_i<kDppSwap1>(v);
  v += dpp_i<kDppSwap2>(v);
  v += dpp_i<kDppHalfMirror>(v);
  v += dpp_i<kDppMirror>(v);
  return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48);
}

// (every wave for itself: lane i has sequences i, i + 64, ..)
struct TreeDeal { int per, all; };
template <class F>
__device__ __forceinline__ TreeDeal tree_deal(const TreeAttnArgs& a, const TreePlan& p, F seq) {
  const int lane = threadIdx.x & 63;
  double total = 0.0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const TreeSeq s = seq(b0 + lane);
    double t = b0 + lane < a.B ? (double)s.blocks * s.tiles : 0.0;
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    total += t;
  }
  TreeDeal d;
  d.per = max(1, (int)fmin(ceil(total * a.Hkv / p.target), 1073741824.0));
  // Last chunks are short ones, so there are more than that.  A workgroup more than run at once doubles the time of all: chunks that are longer, until they
  // fit, or until no sequence is cut any more.
  for (int turn = 0;; ++turn) {
    int all = 0, most = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      const TreeSeq s = seq(b0 + lane);
      const bool in = b0 + lane < a.B;
      all += wave_sum_i(in ? a.Hkv * s.blocks * ((s.tiles + d.per - 1) / d.per) : 0);
      most = max(most, wave_max_i(in && s.blocks ? s.tiles : 0));
    }
    d.all = all;
    if (all <= p.target || p.target > kSplitTarget || d.per >= most || turn == 8) break;
    d.per = max(d.per + 1, (int)fmin(ceil((double)d.per * all / p.target), (double)most));
  }
  return d;
}
// Running sums of the workgroups of the sequences: f(first slot of the lane's sequence, its slots, sequence) for 64 of them at a time.
template <class S, class F>
__device__ __forceinline__ void tree_slots(const TreeAttnArgs& a, int per, S seq, F f) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const TreeSeq s = seq(b0 + lane);
    const int mine = b0 + lane < a.B ? a.Hkv * s.blocks * ((s.tiles + per - 1) / per) : 0;
    int sum = mine;
    for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(sum, o); if (lane >= o) sum += v; }
    if (f(before + sum - mine, mine, b0, s)) return;
    before += __shfl(sum, 63);
  }
}

__device__ __forceinline__ TreeWork tree_work(const TreeAttnArgs& a, const TreePlan& p, TreeSeq& s) {
  TreeWork w;
  w.none = false;
  if (!p.split) {
    int id = blockIdx.x;
    w.block = id % p.row_blocks; id /= p.row_blocks;
    w.hk = id % a.Hkv;
    w.b = id / a.Hkv;
    w.chunk = 0; w.chunks = 1; w.per = 1 << 30; w.slot = 0;
    s = tree_seq(a, p, w.b);
    w.none = w.block >= s.blocks;
    return w;
  }
  const int lane = threadIdx.x & 63;
  const TreeSeq held = tree_seq(a, p, min(lane, a.B - 1));
  auto seq = [&](int b) { return a.B <= 64 ? held : tree_seq(a, p, min(b, a.B - 1)); };
  const TreeDeal d = tree_deal(a, p, seq);
  if (blockIdx.x == 0 && threadIdx.x < 64) {
    int* head = reinterpret_cast<int*>(a.ws);
    if (lane == 0) head[0] = d.per;
    tree_slots(a, d.per, seq, [&](int first, int, int b0, const TreeSeq&) {
      if (b0 + lane < a.B) head[1 + b0 + lane] = first;
      return false;
    });
  }
  // neighbours in slot order, which share keys where a key head has several column blocks, go to one XCD
  const int each = (d.all + 7) / 8, at = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  w.none = (int)(blockIdx.x >> 3) >= each || at >= d.all;
  if (w.none) return w;
  tree_slots(a, d.per, seq, [&](int first, int mine, int b0, const TreeSeq& q) {
    const unsigned long long in = __builtin_amdgcn_ballot_w64(at >= first && at < first + mine);
    if (!in) return false;
    const int from = __builtin_ctzll(in);
    w.b = b0 + from;
    s.n = __shfl(q.n, from); s.rows = __shfl(q.rows, from); s.tiles = __shfl(q.tiles, from); s.blocks = __shfl(q.blocks, from);
    int rest = at - __shfl(first, from);
    w.per = d.per;
    w.chunks = (s.tiles + d.per - 1) / d.per;
    w.chunk = rest / (s.blocks * a.Hkv); rest -= w.chunk * s.blocks * a.Hkv;
    w.hk = rest / s.blocks;
    w.block = rest - w.hk * s.blocks;
    w.slot = at;
    return true;
  });
  return w;
}

#define UNIFORM(x) x = __builtin_amdgcn_readfirstlane(x)

template <class E, int DH, int RW, int KW, int SUB>
__global__ __launch_bounds__(64 * RW * KW, 2) void tree_attn_kernel(TreeAttnArgs a, TreePlan p) {
  typedef AttnType<E> Ty;
  constexpr int WAVES = RW * KW, KT = 32 * KW * SUB, ROW = DH * 2, CH = DH / 8, TILE = KT * ROW;   // bytes of a key, its 16-byte chunks, bytes of a tile
  constexpr int RPI = 1024 / ROW, LOADS = TILE / 1024 / WAVES;                                     // keys a load of a wave covers, loads a wave
  constexpr int ET = DH / 32, JOIN = (DH + 4) * 4;                                                 // bytes of a joined row
  static_assert(LOADS * WAVES * 1024 == TILE, "");
  extern __shared__ __align__(1024) char lds[];   // [2 buffers][K, V][TILE]; at the end [WAVES][32][JOIN]
  TreeSeq s;
  TreeWork w = tree_work(a, p, s);
  if (w.none) return;
  UNIFORM(w.b); UNIFORM(w.hk); UNIFORM(w.block); UNIFORM(w.chunk); UNIFORM(w.chunks); UNIFORM(w.per); UNIFORM(w.slot);
  UNIFORM(s.n); UNIFORM(s.rows); UNIFORM(s.tiles);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave % RW, wk = wave / RW, col = lane & 31, half = lane >> 5;
  const int G = a.H / a.Hkv, M = G * s.rows;
  const int m = (w.block * RW + wr) * 32 + col, t = m / G, head = w.hk * G + m - t * G;   // this lane's column: row t, query head
  const bool there = m < M;

  // keys of this lane's loads: key i * WAVES * RPI + .. of the tile, 16-byte chunk swizzled so that neither the rows of 32 keys nor
  // the four keys of a transposing read fall on the same banks
  const int key0 = wave * RPI + lane / CH, last = s.n + s.rows - 1;
  auto swz = [](int key) { return DH == 128 ? (key & 3) << 2 | (key >> 2 & 3) : (key >> 1 & 1) << 2 | (key >> 2 & 3); };
  const char* kb = reinterpret_cast<const char*>(static_cast<const E*>(a.k) + w.b * a.k_s[0] + w.hk * a.k_s[2]);
  const char* vb = reinterpret_cast<const char*>(static_cast<const E*>(a.v) + w.b * a.v_s[0] + w.hk * a.v_s[2]);
  const long krow = a.k_s[1] * 2, vrow = a.v_s[1] * 2;
  // (a lane's place in a tile: the same for every load of it but for the swizzle where a wave's loads are 8 keys apart; rows so far apart
  // that it passes 32 bits take the products for every load, as does the last tile, whose keys end)
  constexpr int APART = WAVES * RPI;
  const bool near = (krow | vrow) < (1l << 26);
  unsigned kofs[2], vofs[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const unsigned chunk = ((lane % CH) ^ swz(key0 + i * APART)) * 16;
    kofs[i] = (unsigned)key0 * (unsigned)krow + chunk;
    vofs[i] = (unsigned)key0 * (unsigned)vrow + chunk;
  }
  static_assert(APART % 16 == 0 || APART == 8, "swizzles of every other load are alike");
  auto load_tile = [&](int tile, int buf) __attribute__((always_inline)) {
    char* dst = lds + buf * 2 * TILE + wave * 1024;
    if (near && tile * KT + KT - 1 <= last) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const long row = tile * KT + i * APART;
        __builtin_amdgcn_global_load_lds(SD_GLB_PTR(kb + row * krow + kofs[i & 1]), SD_LDS_PTR(dst + i * WAVES * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds(SD_GLB_PTR(vb + row * vrow + vofs[i & 1]), SD_LDS_PTR(dst + TILE + i * WAVES * 1024), 16, 0, 0);
      }
      return;
    }
#pragma unroll 1
    for (int i = 0; i < LOADS; ++i) {
      const int in = key0 + i * APART, key = min(tile * KT + in, last);
      const int chunk = ((lane % CH) ^ swz(in)) * 16;
      __builtin_amdgcn_global_load_lds(SD_GLB_PTR(kb + key * krow + chunk), SD_LDS_PTR(dst + i * WAVES * 1024), 16, 0, 0);
      __builtin_amdgcn_global_load_lds(SD_GLB_PTR(vb + key * vrow + chunk), SD_LDS_PTR(dst + TILE + i * WAVES * 1024), 16, 0, 0);
    }
  };
  int tile = w.chunk * w.per;
  const int end = s.n < 0 ? tile : min(s.tiles, tile + w.per);
  if (tile < end) load_tile(tile, 0);

  s16x8 q[DH / 16];
  {
    const E* qp = static_cast<const E*>(a.q) + w.b * a.q_s[0] + (there ? t : 0) * a.q_s[1] + (there ? head : w.hk * G) * a.q_s[2] + half * 8;
#pragma unroll
    for (int k = 0; k < DH / 16; ++k) q[k] = *reinterpret_cast<const s16x8*>(qp + k * 16);
    if (a.scale < 0.f)   // (a negative scale as queries of the other sign: the largest product is the largest score)
#pragma unroll
      for (int k = 0; k < DH / 16; ++k) q[k] ^= (short)0x8000;
  }
  u64 seen = 0;
  if (there) seen = (a.visible ? a.visible[(size_t)w.b * a.T + t] : ~0ull >> (63 - t)) & (~0ull >> (64 - s.rows));
  const float scale = fmaxf(fabsf(a.scale) * 1.44269504088896f, 1e-37f);   // (not 0: what is masked is -inf times this)

  f32x16 acc[ET];
#pragma unroll
  for (int e = 0; e < ET; ++e) acc[e] = f32x16{};
  float top = kNegInf, sum = 0.f;
  const int g = lane & 15, kkey = col, vkey = 4 * half + g / 4;
  const int kc = swz(kkey) ^ half, vc = ((lane >> 4 & 1) * 2 + (g >> 1 & 1)) ^ swz(vkey);

  // 32 N keys from key `first` of a tile, `key` of the sequence.  (N > 1: one product's chain of matrix instructions fills the other one's waits.)
  auto step = [&](auto masked, auto parts, const char* kt, const char* vt, int first, int key) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(masked)::value;
    constexpr int N = decltype(parts)::value;
    static_assert(!MASK || N == 1, "");
    f32x16 st[N] = {};
#pragma unroll
    for (int k = 0; k < DH / 16; ++k)
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const s16x8 kf = *reinterpret_cast<const s16x8*>(kt + (first + 32 * u + kkey) * ROW + ((kc ^ 2 * k) * 16));
        st[u] = Ty::mfma(kf, q[k], st[u]);
      }
    unsigned window = ~0u;   // which of keys 4 half .. + 31 this column sees
    if constexpr (MASK) {
      const int rel = key + 4 * half - s.n;
      window = rel >= 64 ? 0u : rel >= 0 ? (unsigned)(seen >> rel) : rel <= -32 ? ~0u : (unsigned)(seen << -rel) | ((1u << -rel) - 1);
    }
    float x[N][16], big = kNegInf;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[u][i] = st[u][i];
        if (MASK && !(window >> (8 * (i >> 2) + (i & 3)) & 1)) x[u][i] = kNegInf;
        big = fmaxf(big, x[u][i]);
      }
    big = half_max(big) * scale;
    if (__builtin_amdgcn_ballot_w64(big > top + Ty::kSlack)) {
      const float next = fmaxf(top, big);
      float keep = top == kNegInf ? 0.f : __builtin_amdgcn_exp2f(top - next);
      top = next;
      sum *= keep;
      asm volatile("" : "+v"(keep));   // (known here only: the products are not formed ahead for every tile)
#pragma unroll
      for (int e = 0; e < ET; ++e) acc[e] *= keep;
    } else {   // (a value of its own on this side, too: else all sums are moved to other registers and back, for every tile)
#pragma unroll
      for (int e = 0; e < ET; ++e) asm volatile("" : "+v"(acc[e]));
    }
    const float base = top == kNegInf ? 0.f : top - Ty::kLift;
    // The second product's matrix instructions take weights of the element type: each is off by half a step of it, its column's sum is of the unrounded ones.
    // (Outputs against 64 bits: bf16 2.3e-3, weights of 32 bits 1.6e-3; fp16 2.9e-4 and 2.1e-4.  Weights as two terms would double that product.)
    s16x8 pf[2 * N];
    float part = 0.f;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      typename Ty::x8 pv[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][i], scale, -base));
        part += x[u][i];
        pv[i >> 3][i & 7] = (E)x[u][i];
      }
      pf[2 * u] = __builtin_bit_cast(s16x8, pv[0]);
      pf[2 * u + 1] = __builtin_bit_cast(s16x8, pv[1]);
    }
    sum += part;
    if constexpr (MASK) {
      // Values that some columns see and others do not: 0 x infinity is not 0.  Where the tree's rows of this tile hold any, products one by one.
      if (a.T > 1 || a.visible) {
        unsigned odd = 0;
#pragma unroll
        for (int i = 0; i < 32 * ROW / 1024; ++i) {
          const uint4 v4 = *reinterpret_cast<const uint4*>(vt + first * ROW + i * 1024 + lane * 16);
          for (unsigned u : {v4.x, v4.y, v4.z, v4.w}) odd |= ((u & Ty::kExp) + Ty::kUnit) & 0x80008000u;
        }
        if (__builtin_amdgcn_ballot_w64(odd != 0)) {
#pragma unroll 1
          for (int i = 0; i < 32; ++i) {   // (seldom run, so short: the lane's weights move past, two keys each)
            const int reg = i >> 1, h2 = i & 1, row = first + 8 * (reg >> 2) + 4 * h2 + (reg & 3);
            const float pi = (float)(E)__shfl(x[0][0], col + 32 * h2);
            if (h2)
#pragma unroll
              for (int r = 0; r < 15; ++r) x[0][r] = x[0][r + 1];
            if (__shfl(window, col + 32 * h2) >> (8 * (reg >> 2) + (reg & 3)) & 1)
#pragma unroll
              for (int e = 0; e < ET; ++e)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                  const int dim = e * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                  acc[e][r] += pi * (float)*reinterpret_cast<const E*>(vt + row * ROW + ((dim / 8) ^ swz(row)) * 16 + (dim & 7) * 2);
                }
          }
          return;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 2 * N; ++k)
#pragma unroll
      for (int e = 0; e < ET; ++e) {
        s16x4 v4[2];
#pragma unroll
        for (int r = 0; r < 2; ++r)
          v4[r] = lds_tr16(reinterpret_cast<const bf16*>(vt + (first + 16 * k + 8 * r + vkey) * ROW + ((vc ^ 4 * e ^ 2 * r) * 16) + (g & 1) * 8));
        const s16x8 vf = {v4[0][0], v4[0][1], v4[0][2], v4[0][3], v4[1][0], v4[1][1], v4[1][2], v4[1][3]};
        acc[e] = Ty::mfma(vf, pf[k], acc[e]);
      }
  };

  const bool idle = (w.block * RW + wr) * 32 >= M;   // (a wave without columns: it loads and waits with the others)
  auto arrived = [&] {   // every wave's part of this tile is there, and every wave is done with the buffer loaded next
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  // the tiles that every column sees whole (which buffer is known to the compiler: addresses in LDS are a lane's own and a constant) ..
  const int whole_end = max(tile, min(end, s.n / KT));
  int buf = 0;
  auto tile_in = [&](auto buffer) __attribute__((always_inline)) {
    constexpr int BUF = decltype(buffer)::value;
    arrived();
    if (tile + 1 < end) load_tile(tile + 1, BUF ^ 1);
    const char* kt = lds + BUF * 2 * TILE;
    step(std::false_type{}, std::integral_constant<int, SUB>{}, kt, kt + TILE, wk * SUB * 32, 0);
    ++tile;
  };
  if (idle) {
#pragma unroll 1
    for (; tile < end; ++tile, buf ^= 1) {
      arrived();
      if (tile + 1 < end) load_tile(tile + 1, buf ^ 1);
    }
  }
  while (tile < whole_end) {
    tile_in(std::integral_constant<int, 0>{});
    if (tile == whole_end) { buf = 1; break; }
    tile_in(std::integral_constant<int, 1>{});
  }
  // .. and those with rows of the tree (a loop of its own: its registers are not the other one's)
#pragma unroll 1
  for (; tile < end; ++tile, buf ^= 1) {
    arrived();
    if (tile + 1 < end) load_tile(tile + 1, buf ^ 1);
    const char* kt = lds + buf * 2 * TILE;
    const int first = wk * SUB * 32, key = tile * KT + first;
#pragma unroll 1
    for (int u = 0; u < 32 * SUB && key + u < s.n + s.rows; u += 32) step(std::true_type{}, std::integral_constant<int, 1>{}, kt, kt + TILE, first + u, key + u);
  }
#pragma unroll
  for (int e = 0; e < ET; ++e) mfma_settle(acc[e]);
  sum = half_add(sum);

  const bool whole = w.chunks == 1;
  float* slot = a.ws + tree_head_ints(a.B) + (size_t)w.slot * 32 * RW * (DH + 2);   // [columns][DH], [columns] maxima, [columns] sums
  if constexpr (KW == 1) {
    if (!there) return;
    if (whole) {
      const float f = sum == 0.f ? 0.f : 1.f / sum;
      E* o = static_cast<E*>(a.o) + w.b * a.o_s[0] + t * a.o_s[1] + head * a.o_s[2] + 4 * half;
#pragma unroll
      for (int e = 0; e < ET; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          typedef E x4 __attribute__((ext_vector_type(4)));
          x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = (E)(acc[e][r * 4 + i] * f);
          *reinterpret_cast<x4*>(o + e * 32 + r * 8) = v;
        }
    } else {
      float* o = slot + (size_t)(wr * 32 + col) * DH + 4 * half;
#pragma unroll
      for (int e = 0; e < ET; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) *reinterpret_cast<f32x4*>(o + e * 32 + r * 8) = f32x4{acc[e][r * 4], acc[e][r * 4 + 1], acc[e][r * 4 + 2], acc[e][r * 4 + 3]};
      if (half == 0) {
        slot[32 * RW * DH + wr * 32 + col] = top;
        slot[32 * RW * (DH + 1) + wr * 32 + col] = sum;
      }
    }
  } else {
    // the waves of a column join what they have: [wave][column][DH + 4], the last four {maximum, sum}
    __syncthreads();
    char* mine = lds + (size_t)(wave * 32 + col) * JOIN;
#pragma unroll
    for (int e = 0; e < ET; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4*>(mine + (e * 32 + r * 8 + 4 * half) * 4) = f32x4{acc[e][r * 4], acc[e][r * 4 + 1], acc[e][r * 4 + 2], acc[e][r * 4 + 3]};
    if (half == 0) *reinterpret_cast<f32x4*>(mine + DH * 4) = f32x4{top, sum, 0.f, 0.f};
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * RW * (DH / 4); i += 64 * WAVES) {
      const int c = i / (DH / 4), d4 = i - c * (DH / 4), mm = w.block * RW * 32 + c;
      if (mm >= M) break;
      const char* part[KW];
      f32x4 st[KW];
      float all = kNegInf;
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        part[k] = lds + (size_t)((k * RW + c / 32) * 32 + (c & 31)) * JOIN;
        st[k] = *reinterpret_cast<const f32x4*>(part[k] + DH * 4);
        all = fmaxf(all, st[k][0]);
      }
      f32x4 o = {};
      float l = 0.f;
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        const float f = st[k][0] == kNegInf && st[k][1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(st[k][0] - all);
        l += f * st[k][1];
        const f32x4 v = *reinterpret_cast<const f32x4*>(part[k] + d4 * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += f * v[j];
      }
      if (whole) {
        const float f = l == 0.f ? 0.f : 1.f / l;
        const int t2 = mm / G;
        typedef E x4 __attribute__((ext_vector_type(4)));
        x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (E)(o[j] * f);
        *reinterpret_cast<x4*>(static_cast<E*>(a.o) + w.b * a.o_s[0] + t2 * a.o_s[1] + (w.hk * G + mm - t2 * G) * a.o_s[2] + d4 * 4) = v;
      } else {
        *reinterpret_cast<f32x4*>(slot + (size_t)c * DH + d4 * 4) = o;
        if (d4 == 0) { slot[32 * RW * DH + c] = all; slot[32 * RW * (DH + 1) + c] = l; }
      }
    }
  }
}

// The chunks of a column (row, query head) added up, kJoinAhead of them requested at once: bound by round trips.  JW waves a column, each every JW-th
// chunk: one, four columns a workgroup, where a column has few chunks, sixteen where it has many (64 chunks of 32 columns: 26 us with four waves
// that first looked for the largest maximum).
constexpr int kJoinAhead = 4;
template <class E, int PER, int JW>
__global__ __launch_bounds__(JW == 1 ? 256 : 64 * JW) void tree_join_kernel(TreeAttnArgs a, TreePlan p) {
  constexpr int DH = 64 * PER, COLS = JW == 1 ? 4 : 1;
  typedef float Part __attribute__((ext_vector_type(PER)));
  typedef E Out __attribute__((ext_vector_type(PER)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), cols = 32 * p.rw, G = a.H / a.Hkv;
  int id = blockIdx.x;
  const int c = id % (cols / COLS) * COLS + (JW == 1 ? wave : 0); id /= cols / COLS;
  const int block = id % p.row_blocks, hk = id / p.row_blocks, b = blockIdx.y;
  const int* head = reinterpret_cast<const int*>(a.ws);
  const int per = head[0], first = head[1 + b];
  const TreeSeq s = tree_seq(a, p, b);
  const int m = block * cols + c, chunks = (s.tiles + per - 1) / per;
  if (m >= G * s.rows || chunks == 1) return;   // (one chunk: written by its workgroup)
  const size_t step = (size_t)cols * (DH + 2) * s.blocks * a.Hkv;
  const float* slot = a.ws + tree_head_ints(a.B) + ((size_t)first + (size_t)hk * s.blocks + block) * cols * (DH + 2);
  Part o = {};
  float top = kNegInf, l = 0.f;
  auto add = [&](float mi, float li, const Part& v, float next) {
    const float f = mi == kNegInf && li == 0.f ? 0.f : __builtin_amdgcn_exp2f(mi - next);
    l += f * li;
    o += f * v;
  };
  for (int i0 = JW == 1 ? 0 : wave; i0 < chunks; i0 += JW * kJoinAhead) {
    Part v[kJoinAhead];
    float mi[kJoinAhead], li[kJoinAhead], next = top;
#pragma unroll
    for (int j = 0; j < kJoinAhead; ++j) {
      const float* from = slot + min(i0 + j * JW, chunks - 1) * step;
      v[j] = *reinterpret_cast<const Part*>(from + (size_t)c * DH + lane * PER);
      mi[j] = from[cols * DH + c];
      li[j] = from[cols * (DH + 1) + c];
    }
#pragma unroll
    for (int j = 0; j < kJoinAhead; ++j) next = fmaxf(next, mi[j]);
    const float keep = top == kNegInf && l == 0.f ? 0.f : __builtin_amdgcn_exp2f(top - next);
    l *= keep;
    o *= keep;
#pragma unroll
    for (int j = 0; j < kJoinAhead; ++j)
      if (i0 + j * JW < chunks) add(mi[j], li[j], v[j], next);
    top = next;
  }
  if constexpr (JW > 1) {
    __shared__ float part[JW][DH + 2];
#pragma unroll
    for (int e = 0; e < PER; ++e) part[wave][lane * PER + e] = o[e];
    if (lane == 0) { part[wave][DH] = top; part[wave][DH + 1] = l; }
    __syncthreads();
    if (wave != 0) return;
    float next = kNegInf;
#pragma unroll
    for (int j = 0; j < JW; ++j) next = fmaxf(next, part[j][DH]);
    l = 0.f;
    o = Part{};
#pragma unroll
    for (int j = 0; j < JW; ++j) add(part[j][DH], part[j][DH + 1], *reinterpret_cast<const Part*>(&part[j][lane * PER]), next);
  }
  const int t = m / G;
  Out x;
#pragma unroll
  for (int e = 0; e < PER; ++e) x[e] = (E)(l == 0.f ? 0.f : o[e] / l);
  *reinterpret_cast<Out*>(static_cast<E*>(a.o) + b * a.o_s[0] + t * a.o_s[1] + (hk * G + m - t * G) * a.o_s[2] + lane * PER) = x;
}

size_t tree_attn_bytes(const TreeAttnArgs& a) {
  const TreePlan p = tree_plan(a);
  return p.split ? (tree_head_ints(a.B) + (size_t)p.slots * 32 * p.rw * (a.dh + 2)) * sizeof(float) : 0;
}

template <class E, int DH, int RW, int KW, int SUB>
static hipError_t tree_launch(hipStream_t st, const TreeAttnArgs& a, const TreePlan& p) {
  constexpr int tiles = 4 * 32 * KW * SUB * DH * 2, join = KW > 1 ? RW * KW * 32 * (DH + 4) * 4 : 0, bytes = tiles > join ? tiles : join;
  const auto kernel = tree_attn_kernel<E, DH, RW, KW, SUB>;
  static std::atomic<bool> ready[64];   // (of each GPU; setting it twice does no harm)
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (bytes > 65536 && !(dev < 64 && ready[dev])) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    if (dev < 64) ready[dev] = true;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)(p.split ? (p.slots + 7) / 8 * 8 : p.slots)), dim3(64 * RW * KW), bytes, st, a, p);
  e = hipGetLastError();
  if (e != hipSuccess || !p.split) return e;
  // (a column has about as many chunks as the target is larger than the number of column blocks)
  // (sequences in y: columns of 64 - 1024 threads, batch x heads x rows of them, would pass the 2^32 threads of one dimension)
  const unsigned columns = (unsigned)a.Hkv * p.row_blocks * 32 * p.rw;
  if (p.target <= 8 * a.B * a.Hkv * p.row_blocks) hipLaunchKernelGGL((tree_join_kernel<E, DH / 64, 1>), dim3(columns / 4, a.B), dim3(256), 0, st, a, p);
  else hipLaunchKernelGGL((tree_join_kernel<E, DH / 64, 16>), dim3(columns, a.B), dim3(1024), 0, st, a, p);
  return hipGetLastError();
}

template <class E, int DH>
static hipError_t tree_launch_rows(hipStream_t st, const TreeAttnArgs& a) {
  const TreePlan p = tree_plan(a);
  return p.rw == 1 ? p.kw == 2 ? tree_launch<E, DH, 1, 2, 1>(st, a, p) : tree_launch<E, DH, 1, 4, 1>(st, a, p) : p.rw == 2 ? tree_launch<E, DH, 2, 2, 1>(st, a, p) : tree_launch<E, DH, 4, 1, 2>(st, a, p);
}

hipError_t tree_attn(hipStream_t st, const TreeAttnArgs& a) {
  if (a.f16) return a.dh == 128 ? tree_launch_rows<f16, 128>(st, a) : tree_launch_rows<f16, 64>(st, a);
  return a.dh == 128 ? tree_launch_rows<bf16, 128>(st, a) : tree_launch_rows<bf16, 64>(st, a);
}

// Masks of a tree from its rows' parents: a wave a sequence.  Row 0 is the root; row i (1 .. n) hangs on row parent[i - 1] < i and sees
// what that sees and itself.  A row whose parent is none of the rows before it, or has been left out, is left out: mask 0.
__global__ __launch_bounds__(64) void tree_visible_kernel(const int* __restrict__ parent, int n, u64* __restrict__ visible) {
  __shared__ u64 mask[64];
  const int lane = threadIdx.x, b = blockIdx.x;
  const int p = lane >= 1 && lane <= n ? parent[(size_t)b * n + lane - 1] : -1;
  if (lane == 0) mask[0] = 1;
  for (int i = 1; i <= n; ++i) {   // (one lane: a row follows its parent)
    const int pi = __builtin_amdgcn_readlane(p, i);
    if (lane == 0) mask[i] = pi >= 0 && pi < i && mask[pi] ? mask[pi] | 1ull << i : 0ull;
  }
  __syncthreads();
  if (lane <= n) visible[(size_t)b * (n + 1) + lane] = mask[lane];
}
hipError_t tree_visible(hipStream_t st, const int* parent, int B, int n, u64* visible) {
  constexpr int most = 1 << 24;   // (a grid has fewer than 2^32 threads in a dimension)
  for (int b0 = 0, now; b0 < B; b0 += now) {
    now = B - b0 < most ? B - b0 : most;
    hipLaunchKernelGGL(tree_visible_kernel, dim3(now), dim3(64), 0, st, parent + (size_t)b0 * n, n, visible + (size_t)b0 * (n + 1));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace sd
