// Trees of drafted tokens: what each node sees, and which nodes stand.
//
// Node 0 is the last token that was sampled, node i > 0 is drafted behind node parent[i] < i.
#include "tree.h"

namespace vidkv {

// Ancestors by doubling: a node's mask joins that of the node its pointer stands at, and the pointer moves on to where
// that one's stands; log2(depth) rounds.  A thread a node, a workgroup a tree: bound by the launch.
template <int WORDS>
__global__ __launch_bounds__(64 * WORDS) void tree_masks_kernel(TreeMasks a) {
  const int b = blockIdx.x, i = threadIdx.x;
  const int count = a.count ? min(max(a.count[b], 0), a.n) : a.n;
  __shared__ uint64_t mask[WORDS][64 * WORDS];
  __shared__ int at[64 * WORDS];
  uint64_t m[WORDS];
  const bool there = i < count;
  int up = there ? a.parent ? a.parent[(size_t)b * a.n + i] : i - 1 : -1;
  if (up >= i) up = -1;
#pragma unroll
  for (int w = 0; w < WORDS; ++w) m[w] = there && i >> 6 == w ? 1ull << (i & 63) : 0;
  for (;;) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) mask[w][i] = m[w];
    at[i] = up;
    if (!__syncthreads_or(up >= 0)) break;
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < WORDS; ++w) m[w] |= mask[w][up];
      up = at[up];
    }
    __syncthreads();
  }
  if (i >= a.n) return;
  int depth = 0;
#pragma unroll
  for (int w = 0; w < WORDS; ++w) {
    a.mask[((size_t)b * a.n + i) * WORDS + w] = m[w];
    depth += __popcll(m[w]);
  }
  if (a.pos) {
    const int p = a.base[b] + (there ? depth - 1 : 0);
    for (int x = 0; x < a.n_axes; ++x) a.pos[((size_t)x * gridDim.x + b) * a.n + i] = p;
  }
}

hipError_t launch_tree_masks(const TreeMasks& a, int batch, hipStream_t st) {
  const int words = (a.n + 63) / 64;
  auto go = [&](auto w) {
    constexpr int W = decltype(w)::value;
    hipLaunchKernelGGL(tree_masks_kernel<W>, dim3(batch), dim3(64 * W), 0, st, a);
  };
  if (words == 1) go(std::integral_constant<int, 1>{});
  else if (words == 2) go(std::integral_constant<int, 2>{});
  else if (words == 3) go(std::integral_constant<int, 3>{});
  else go(std::integral_constant<int, 4>{});
  return hipGetLastError();
}

// ---- verification -----------------------------------------------------------------------------
// The residual distribution of a node after its first children were turned down is kept in closed form: with R_0 = P and
// R' = max(R - s Q, 0) / sum, and max(max(x, 0) - y, 0) = max(x - y, 0) for y >= 0,
//   R_k(v) = max(P(v) - a_k Q(v), 0) / b_k,   a_0 = 0, b_0 = 1,   a' = a + b s,   b' = sum_v max(P(v) - a' Q(v), 0),
// s = 1, or, where siblings were drawn without putting back, 1 over what the tried ones left of Q.  (A token that was tried has
// a' Q > P and stays at zero by itself.)  So a child turned down costs one pass over a row of P and Q, and nothing is written
// back.  Without Q, R is P without the tried tokens, b what they left, and no pass is needed before the last.
// All sums, a and b are in 64 bits: a decision next to a border is that of the definition.

constexpr int SLAB = 1024;                 // probabilities that a wave takes in a turn: 16 a lane

struct PF32 { typedef float E; static __device__ __forceinline__ float widen(E e) { return e; } };
struct PF16 { typedef _Float16 E; static __device__ __forceinline__ float widen(E e) { return (float)e; } };
struct PBF16 { typedef __bf16 E; static __device__ __forceinline__ float widen(E e) { return (float)e; } };

__device__ __forceinline__ double weight(float p, float q, double a) { return fmax((double)p - a * (double)q, 0.0); }

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
  return v;
}

// A tree in LDS: thread i holds node i.
struct Nodes {
  int parent[VIDKV_TREE_NODES], token[VIDKV_TREE_NODES];
  float u[VIDKV_TREE_NODES], p[VIDKV_TREE_NODES], q[VIDKV_TREE_NODES];
};

// Where the walk stands; the same in every lane of the wave that walks.
struct Walk {
  int node, last;              // the node reached, its last child that was tried (or itself)
  double a, b, used;           // the residual there; what the tried ones took of Q
  double further;              // a of the residual that a pass is to sum up
  bool pending;                // ... which is asked for: else the walk is over
  bool summed;                 // b is that sum (where Q is): the residual's weights have been added up in a pass
};

template <class T>
__device__ __forceinline__ void load_nodes(Nodes& s, const TreeVerify& a, int b, int count, int i) {
  if (i >= VIDKV_TREE_NODES) return;
  const size_t at = (size_t)b * a.n + i;
  int up = -1, x = -1;
  float p = 0.0f, q = 1.0f, u = 0.0f;
  if (i < count) {
    up = a.parent ? a.parent[at] : i - 1;
    x = a.token[at];
    u = a.uniform[at];
    if (i == 0 || up < 0 || up >= i || x < 0 || x >= a.vocab) up = -1;           // (no child of any node)
    if (up >= 0) {
      typedef typename T::E E;
      p = fmaxf(T::widen(reinterpret_cast<const E*>(a.target.data + b * a.target.sb + up * a.target.st)[x]), 0.0f);
      if (a.draft.data) q = fmaxf(T::widen(reinterpret_cast<const E*>(a.draft.data + b * a.draft.sb + up * a.draft.st)[x]), 0.0f);
    }
  }
  s.parent[i] = up;
  s.token[i] = x;
  s.u[i] = u;
  s.p[i] = p;
  s.q[i] = q;
}

// One wave walks on from where w stands until a pass is needed or no child is left.  Lane: nodes lane, lane + 64, ...
__device__ __forceinline__ void walk_on(Walk& w, const Nodes& s, bool drawn, bool distinct, int lane) {
  int up[4], x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) { up[j] = s.parent[lane + 64 * j]; x[j] = s.token[lane + 64 * j]; }
  w.pending = false;
  for (;;) {
    int child = -1;
#pragma unroll
    for (int j = 3; j >= 0; --j) {
      const uint64_t m = __ballot(up[j] == w.node && lane + 64 * j > w.last);
      if (m) child = 64 * j + __builtin_ctzll(m);
    }
    if (child < 0) return;
    w.last = child;
    const int token = s.token[child];
    if (!drawn || distinct) {              // a token that an earlier sibling had is passed over
      bool had = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) had = had || (up[j] == w.node && x[j] == token && lane + 64 * j < child);
      if (__any(had)) continue;
    }
    const double u = s.u[child], p = s.p[child], q = s.q[child];
    if (!drawn) {
      if (u * w.b < p) { w.node = w.last = child; w.b = 1.0; continue; }
      w.b = fmax(w.b - p, 0.0);
      continue;
    }
    const double scale = !distinct ? 1.0 : w.used < 1.0 ? 1.0 / (1.0 - w.used) : 0.0;
    if (u * (w.b * scale * q) < fmax(p - w.a * q, 0.0)) {
      w.node = w.last = child;
      w.a = 0.0; w.b = 1.0; w.used = 0.0;
      w.summed = false;
      continue;
    }
    w.used += q;
    w.further = w.a + w.b * scale;
    w.pending = true;
    return;
  }
}

// ... with the sum it asked for.  A residual of nothing is not taken: what was there before stays, and no further child is tried.
__device__ __forceinline__ void take_sum(Walk& w, double z) {
  w.summed = z > 0.0;
  if (w.summed) { w.a = w.further; w.b = z; }
  else w.last = VIDKV_TREE_NODES;
}

// A row as a wave reads it.
template <class T>
struct Row {
  const typename T::E* p;
  const typename T::E* q;      // or nullptr
  double a;
  int vocab;
};

// Four elements from index e on, nothing behind the row's end.  (Rows begin where they like: element by element aligned.)
template <class T>
__device__ __forceinline__ void load4(const Row<T>& r, int e, float (&p)[4], float (&q)[4]) {
  typedef typename T::E E;
  typedef E Four __attribute__((ext_vector_type(4), aligned(sizeof(E))));
  Four x = 0, y = 0;
  if (e + 4 <= r.vocab) {
    x = *reinterpret_cast<const Four*>(r.p + e);
    if (r.q) y = *reinterpret_cast<const Four*>(r.q + e);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (e + k < r.vocab) {
        x[k] = r.p[e + k];
        if (r.q) y[k] = r.q[e + k];
      }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) { p[k] = T::widen(x[k]); q[k] = T::widen(y[k]); }
}

// The weights of a slab by one wave: lane takes elements 256 j + 4 lane + k.  tried: nodes whose tokens have no weight (no Q), as the
// lanes hold them (token or -1).
template <class T>
__device__ __forceinline__ void slab_weights(double (&v)[16], const Row<T>& r, int slab, const int (&tried)[4], int lane) {
  float p[4][4], q[4][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) load4(r, slab * SLAB + 256 * j + 4 * lane, p[j], q[j]);
#pragma unroll
  for (int j = 0; j < 16; ++j) v[j] = r.q ? weight(p[j >> 2][j & 3], q[j >> 2][j & 3], r.a) : fmax((double)p[j >> 2][j & 3], 0.0);
  if (r.q) return;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint64_t m = __ballot(tried[k] >= 0 && tried[k] / SLAB == slab);
    while (m) {
      const int e = __shfl(tried[k], __builtin_ctzll(m)) - slab * SLAB;
      m &= m - 1;
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (256 * (j >> 2) + 4 * lane + (j & 3) == e) v[j] = 0.0;
    }
  }
}

// One workgroup a sequence.
template <class T>
__global__ __launch_bounds__(1024) void tree_verify_kernel(TreeVerify a) {
  constexpr int W = 16;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int count = a.count ? min(max(a.count[b], 0), a.n) : a.n;
  const int slabs = (a.vocab + SLAB - 1) / SLAB;
  __shared__ Nodes s;
  __shared__ Walk shared;
  __shared__ double sums[VIDKV_TREE_VOCAB / SLAB];
  __shared__ double part[W];
  __shared__ int found;
  if (count == 0) {
    for (int i = tid; i < a.n; i += 1024) a.path[(size_t)b * a.n + i] = -1;
    if (tid == 0) { a.accepted[b] = 0; a.next[b] = -1; }
    return;
  }
  load_nodes<T>(s, a, b, count, tid);
  __syncthreads();
  const bool drawn = a.draft.data != nullptr;
  Walk w{0, 0, 0.0, 1.0, 0.0, 0.0, false, false};
  auto row = [&](double with) {
    typedef typename T::E E;
    return Row<T>{reinterpret_cast<const E*>(a.target.data + b * a.target.sb + w.node * a.target.st),
                  drawn ? reinterpret_cast<const E*>(a.draft.data + b * a.draft.sb + w.node * a.draft.st) : nullptr, with, a.vocab};
  };
  // the slabs' sums of a row's weights, and their total (in order of the slabs, the same in every thread)
  auto pass = [&](const Row<T>& r, const int (&tried)[4]) {
    for (int k = wv; k < slabs; k += W) {
      double v[16];
      slab_weights(v, r, k, tried, lane);
      double z = 0.0;
#pragma unroll
      for (int j = 0; j < 16; ++j) z += v[j];
      z = wave_sum(z);
      if (lane == 0) sums[k] = z;
    }
    __syncthreads();
    double z = 0.0;
    for (int k = tid; k < slabs; k += 1024) z += sums[k];
    z = wave_sum(z);
    if (lane == 0) part[wv] = z;
    __syncthreads();
    z = 0.0;
#pragma unroll
    for (int k = 0; k < W; ++k) z += part[k];
    __syncthreads();
    return z;
  };
  const int none[4] = {-1, -1, -1, -1};
  double total = 0.0;
  for (;;) {
    if (wv == 0) {
      walk_on(w, s, drawn, a.distinct, lane);
      if (lane == 0) shared = w;
    }
    __syncthreads();
    w = shared;
    if (!w.pending) break;
    total = pass(row(w.further), none);
    take_sum(w, total);
  }
  // the residual's weights at the last node
  int tried[4] = {-1, -1, -1, -1};
  if (!drawn) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (s.parent[lane + 64 * j] == w.node) tried[j] = s.token[lane + 64 * j];
  }
  Row<T> r = row(w.a);
  if (!w.summed) total = pass(r, tried);
  if (!(total > 0.0)) {                    // nothing left of it: the row as it was
#pragma unroll
    for (int j = 0; j < 4; ++j) tried[j] = -1;
    r.a = 0.0;
    total = pass(r, none);
  }
  // the slab in which the sum passes u times the total, or the last one that has any
  const double goal = (double)s.u[0] * total;
  double before = 0.0;                     // sum of the slabs before it
  int slab = -1;
  if (wv == 0) {
    double run = 0.0;
    int some = -1;
    for (int k0 = 0; k0 < slabs && slab < 0; k0 += 64) {
      const double mine = k0 + lane < slabs ? sums[k0 + lane] : 0.0;
      double in = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(in, d);
        if (lane >= d) in += o;
      }
      const uint64_t over = __ballot(mine > 0.0 && run + in > goal), any = __ballot(mine > 0.0);
      if (over) {
        const int l = __builtin_ctzll(over);
        slab = k0 + l;
        before = run + __shfl(in - mine, l);
      } else if (any) {
        const int l = 63 - __builtin_clzll(any);
        some = k0 + l;
        before = run + __shfl(in - mine, l);
      }
      run += __shfl(in, 63);
    }
    if (slab < 0) slab = some;
    int token = -1;
    if (slab >= 0) {
      // its elements in order: lane takes 16 that lie next to each other
      double v[16], in = 0.0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float p[4], q[4];
        load4(r, slab * SLAB + 16 * lane + 4 * j, p, q);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[4 * j + k] = drawn ? weight(p[k], q[k], r.a) : fmax((double)p[k], 0.0);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint64_t m = __ballot(tried[k] >= 0 && tried[k] / SLAB == slab);
        while (m) {
          const int e = __shfl(tried[k], __builtin_ctzll(m)) - slab * SLAB - 16 * lane;
          m &= m - 1;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j == e) v[j] = 0.0;
        }
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) in += v[j];
      const double mine = in;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(in, d);
        if (lane >= d) in += o;
      }
      double run2 = before + (in - mine);
      int hit = -1, last = -1;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        run2 += v[j];
        if (v[j] > 0.0) {
          last = j;
          if (hit < 0 && run2 > goal) hit = j;
        }
      }
      const uint64_t hits = __ballot(hit >= 0), lasts = __ballot(last >= 0);
      const int l = hits ? __builtin_ctzll(hits) : lasts ? 63 - __builtin_clzll(lasts) : 0;
      const int j = __shfl(hits ? hit : last, l);
      token = j >= 0 ? slab * SLAB + 16 * l + j : -1;
    }
    if (lane == 0) {
      a.next[b] = token;
      int depth = 0;
      for (int i = w.node; i > 0; i = s.parent[i]) ++depth;
      found = depth + 1;
      a.accepted[b] = depth + 1;
      for (int i = w.node, k = depth; k >= 0; i = s.parent[i], --k) a.path[(size_t)b * a.n + k] = i;
    }
  }
  __syncthreads();
  for (int i = found + tid; i < a.n; i += 1024) a.path[(size_t)b * a.n + i] = -1;
}

size_t tree_verify_ws_bytes(int, int, int) { return 256; }

hipError_t launch_tree_verify(const TreeVerify& a, int dtype, int batch, void*, hipStream_t st) {
  if (dtype == VIDKV_F32) hipLaunchKernelGGL(tree_verify_kernel<PF32>, dim3(batch), dim3(1024), 0, st, a);
  else if (dtype == VIDKV_F16) hipLaunchKernelGGL(tree_verify_kernel<PF16>, dim3(batch), dim3(1024), 0, st, a);
  else hipLaunchKernelGGL(tree_verify_kernel<PBF16>, dim3(batch), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace vidkv
