// Trees of drafted tokens: what each node sees, and which nodes stand.
//
// Node 0 is the last token that was sampled, node i > 0 is drafted behind node parent[i] < i.
#include "tree.h"
#include <algorithm>

namespace vidkv {

// Ancestors by doubling: a node's mask joins that of the node its pointer stands at, and the pointer moves on to where
// that one's stands; log2(depth) rounds.  A thread a node, a workgroup a tree: bound by the launch (one tree of 33 nodes 2.1 us,
// 64 of 256 with paths of some 130 nodes 5.6, of it eight rounds of two barriers).
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
// s = 1, or, where siblings were drawn without putting back, 1 over what the tried ones left of Q (of nothing no further child is
// tried: passing one over takes nothing from the target's probabilities, letting it stand without a chance to compare would).  (A
// token that was tried has a' Q > P and stays at zero by itself.)  So a child turned down costs one pass over a row of P and Q, and
// nothing is written back.  Without Q, R is P without the tried tokens, b what they left, and no pass is needed before the last.
// All sums, a and b are in 64 bits: a decision next to a border is that of the definition.
//
// Bound by round trips: nodes -> probabilities -> row -> slab.  A chain of 6 over 32000 float32 9 us in one launch; 16 trees of 64
// over 150001 7.7 and 4.9 (9.6 MB of rows are 1.9 at a copy's rate).

constexpr int SLAB = 1024;                 // probabilities that a wave takes in a turn: 16 a lane

struct PF32 { typedef float E; static __device__ __forceinline__ float widen(E e) { return e; } };
struct PF16 { typedef _Float16 E; static __device__ __forceinline__ float widen(E e) { return (float)e; } };
struct PBF16 { typedef __bf16 E; static __device__ __forceinline__ float widen(E e) { return (float)e; } };

__device__ __forceinline__ double weight(float p, float q, double a) { return fmax((double)p - a * (double)fmaxf(q, 0.0f), 0.0); }

// A double from another lane of a row of sixteen, or of another row; zero where there is none.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double from_lane(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Sums over the lanes up to each, and lane l's number as the wave's.  (Six register moves of two halves; as shuffles through LDS each step
// waits for it: a launch of few sequences 0.5 us longer.)
__device__ __forceinline__ double wave_scan(double v) {
  v += from_lane<0x111>(v);                // row_shr 1, 2, 4, 8
  v += from_lane<0x112>(v);
  v += from_lane<0x114>(v);
  v += from_lane<0x118>(v);
  v += from_lane<0x142, 0xa>(v);           // lane 15 of a row to the next one, in rows 1 and 3
  v += from_lane<0x143, 0xc>(v);           // lane 31 to rows 2 and 3
  return v;
}
__device__ __forceinline__ double lane_value(double v, int l) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, l), hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), l);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) { return lane_value(wave_scan(v), 63); }

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
  int sums;                    // ASKED for with `further`; HERE: those of the residual's weights are made; or NONE_MADE.  If not asked
                               // for, the walk is over
};
enum { NONE_MADE, HERE, ASKED };

// Thread i loads node i; what does not depend on one another is asked for at once.
struct NodeIn {
  int up, x;
  float u;
};
__device__ __forceinline__ NodeIn ask_node(const TreeVerify& a, int b, int i) {
  NodeIn o{-1, -1, 0.0f};
  if (i < a.n) {
    const size_t at = (size_t)b * a.n + i;
    o.up = a.parent ? a.parent[at] : i - 1;
    o.x = a.token[at];
    o.u = a.uniform[at];
  }
  return o;
}
template <class T>
__device__ __forceinline__ f2 gather(const NodeIn& o, const TreeVerify& a, int b) {
  typedef typename T::E E;
  f2 v{0.0f, 1.0f};
  if (o.up >= 0) {
    v[0] = fmaxf(T::widen(reinterpret_cast<const E*>(a.target.data + b * a.target.sb + o.up * a.target.st)[o.x]), 0.0f);
    if (a.draft.data) v[1] = fmaxf(T::widen(reinterpret_cast<const E*>(a.draft.data + b * a.draft.sb + o.up * a.draft.st)[o.x]), 0.0f);
  }
  return v;
}
__device__ __forceinline__ void keep_child(NodeIn& o, const TreeVerify& a, int count, int i) {
  if (i == 0 || i >= count || o.up < 0 || o.up >= i || o.x < 0 || o.x >= a.vocab) o.up = -1;           // (no child of any node)
}
__device__ __forceinline__ void put_node(Nodes& s, const NodeIn& o, f2 pq, int i) {
  if (i >= VIDKV_TREE_NODES) return;
  s.parent[i] = o.up;
  s.token[i] = o.x;
  s.u[i] = o.u;
  s.p[i] = pq[0];
  s.q[i] = pq[1];
}

// One wave walks on from where w stands until a pass is needed or no child is left.  Lane: nodes lane, lane + 64, ...
__device__ __forceinline__ void walk_on(Walk& w, const Nodes& s, bool drawn, bool distinct, int lane) {
  int up[4], x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) { up[j] = s.parent[lane + 64 * j]; x[j] = s.token[lane + 64 * j]; }
  for (;;) {
    if (distinct && !(w.used < 1.0)) return;         // nothing is left of Q that a further child could have come from
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
    const double scale = distinct ? 1.0 / (1.0 - w.used) : 1.0;
    if (u * (w.b * scale * q) < fmax(p - w.a * q, 0.0)) {
      w.node = w.last = child;
      w.a = 0.0; w.b = 1.0; w.used = 0.0;
      w.sums = NONE_MADE;
      continue;
    }
    w.used += q;
    w.further = w.a + w.b * scale;
    w.sums = ASKED;
    return;
  }
}

// The same for a wave's every lane, held as its scalars.
__device__ __forceinline__ Walk uniform(const Walk& w) {
  return Walk{__builtin_amdgcn_readfirstlane(w.node), __builtin_amdgcn_readfirstlane(w.last), lane_value(w.a, 0), lane_value(w.b, 0),
              lane_value(w.used, 0), lane_value(w.further, 0), __builtin_amdgcn_readfirstlane(w.sums)};
}

// ... with the sum it asked for.  A residual of nothing is not taken: what was there before stays, and no further child is tried.
__device__ __forceinline__ void take_sum(Walk& w, double z) {
  w.sums = z > 0.0 ? HERE : NONE_MADE;
  if (z > 0.0) { w.a = w.further; w.b = z; }
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

// What a wave takes of a slab: lane has elements 256 j + 4 lane + k of it.
struct Slab {
  float p[4][4], q[4][4];
};
template <class T>
__device__ __forceinline__ void load_slab(Slab& v, const Row<T>& r, int slab, int lane) {
#pragma unroll
  for (int j = 0; j < 4; ++j) load4(r, slab * SLAB + 256 * j + 4 * lane, v.p[j], v.q[j]);
}
// Tokens without weight (without Q: those tried), as the lanes hold them, become zeros: element(i) is the token of a lane's
// i-th place.
template <class F, class P>
__device__ __forceinline__ void clear_tried(const int (&tried)[4], int slab, F&& element, P&& place) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint64_t m = __ballot(tried[k] >= 0 && tried[k] / SLAB == slab);
    while (m) {
      const int e = __builtin_amdgcn_readlane(tried[k], __builtin_ctzll(m)) - slab * SLAB;
      m &= m - 1;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (element(i) == e) place(i) = 0.0f;
    }
  }
}
template <class T>
__device__ __forceinline__ double sum_of_slab(Slab& v, const Row<T>& r, const int (&tried)[4], int slab, int lane) {
  double z = 0.0;
  if (r.q) {
#pragma unroll
    for (int i = 0; i < 16; ++i) z += weight(v.p[i >> 2][i & 3], v.q[i >> 2][i & 3], r.a);
  } else {
    clear_tried(tried, slab, [&](int i) { return 256 * (i >> 2) + 4 * lane + (i & 3); }, [&](int i) -> float& { return v.p[i >> 2][i & 3]; });
#pragma unroll
    for (int i = 0; i < 16; ++i) z += (double)fmaxf(v.p[i >> 2][i & 3], 0.0f);
  }
  return wave_sum(z);
}

// What a sequence's launches hand on: where the walk stands, and whether the sums that it asked for last are the last ones
// (of the weights that the next token is drawn by).  `at`: which of the two arrays has them.
struct State {
  Walk w;
  int done, at;
};

struct TreeWork {
  State* state;                // [2][B]: a launch reads one and writes the other
  f2* pq;                      // [B][n]: the drafted tokens' probabilities, gathered by the first launch
  double* sums;                // [2][B][slabs]
  int slabs;
};

// (The weights before a child was turned down are the target's own: Q is not read.)
template <class T>
__device__ __forceinline__ Row<T> row_of(const TreeVerify& a, int b, int node, double with) {
  typedef typename T::E E;
  return Row<T>{reinterpret_cast<const E*>(a.target.data + b * a.target.sb + node * a.target.st),
                a.draft.data && with > 0.0 ? reinterpret_cast<const E*>(a.draft.data + b * a.draft.sb + node * a.draft.st) : nullptr,
                with, a.vocab};
}

// Tokens without weight at the last node, as the lanes of a wave hold them.
__device__ __forceinline__ void load_tried(int (&tried)[4], const Nodes& s, int node, bool drawn, int lane) {
#pragma unroll
  for (int j = 0; j < 4; ++j) tried[j] = !drawn && s.parent[lane + 64 * j] == node ? s.token[lane + 64 * j] : -1;
}

// Sums of slabs first, first + step, ... by one wave, each asked for while the one before is added up.
template <class T>
__device__ __forceinline__ void sum_slabs(double* sums, const Row<T>& r, const int (&tried)[4], int first, int step, int slabs, int lane) {
  Slab now, next;
  if (first < slabs) load_slab(now, r, first, lane);
  for (int k = first; k < slabs; k += step) {
    if (k + step < slabs) load_slab(next, r, k + step, lane);
    const double z = sum_of_slab(now, r, tried, k, lane);
    if (lane == 0) sums[k] = z;
    now = next;
  }
}

// Their total by one wave, the same whoever asks.
__device__ __forceinline__ double total_of(const double* sums, int slabs, int lane) {
  double z = 0.0;
  for (int k = lane; k < slabs; k += 64) z += sums[k];
  return wave_sum(z);
}

// One pass over a row, shared out to the workgroups of a sequence, each of which finds out for itself what is wanted: it
// goes on from where the launch before left the walk, with the sums that that one made.  grid (workgroups a sequence, B).
template <class T>
__global__ __launch_bounds__(256) void tree_pass_kernel(TreeVerify a, TreeWork k, int round) {
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  NodeIn in = ask_node(a, b, tid);
  f2 pq{0.0f, 0.0f};
  if (round > 0 && tid < a.n) pq = k.pq[(size_t)b * a.n + tid];
  const int now = round & 1;
  double z = 0.0;
  if (round > 0 && wv == 0) z = total_of(k.sums + ((size_t)(1 - now) * gridDim.y + b) * k.slabs, k.slabs, lane);
  const int count = a.count ? min(max(a.count[b], 0), a.n) : a.n;
  if (count == 0) return;
  __shared__ Nodes s;
  __shared__ State next;
  State from{Walk{0, 0, 0.0, 1.0, 0.0, 0.0, NONE_MADE}, 0, 0};
  if (round > 0) from = k.state[(size_t)(1 - now) * gridDim.y + b];
  if (from.done) {
    if (blockIdx.x == 0 && tid == 0) k.state[(size_t)now * gridDim.y + b] = from;
    return;
  }
  keep_child(in, a, count, tid);
  if (round == 0) {
    pq = gather<T>(in, a, b);
    if (blockIdx.x == 0 && tid < a.n) k.pq[(size_t)b * a.n + tid] = pq;
  }
  put_node(s, in, pq, tid);
  __syncthreads();
  const bool drawn = a.draft.data != nullptr;
  if (wv == 0) {
    Walk w = from.w;
    if (w.sums == ASKED) take_sum(w, z);
    walk_on(w, s, drawn, a.distinct, lane);
    State to{w, w.sums != ASKED, w.sums == HERE ? 1 - now : now};
    if (lane == 0) {
      next = to;
      if (blockIdx.x == 0) k.state[(size_t)now * gridDim.y + b] = to;
    }
  }
  __syncthreads();
  const Walk w = uniform(next.w);
  if (w.sums == HERE) return;       // (the sums of the launch before are the last ones)
  int tried[4] = {-1, -1, -1, -1};
  if (next.done) load_tried(tried, s, w.node, drawn, lane);
  sum_slabs(k.sums + ((size_t)now * gridDim.y + b) * k.slabs, row_of<T>(a, b, w.node, next.done ? w.a : w.further), tried,
            blockIdx.x * 4 + wv, gridDim.x * 4, k.slabs, lane);
}

// The rest: passes that are still wanted, the next token, the path.  One workgroup a sequence.
template <class T, int W>
__global__ __launch_bounds__(64 * W) void tree_finish_kernel(TreeVerify a, TreeWork k, int rounds) {
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int count = a.count ? min(max(a.count[b], 0), a.n) : a.n;
  const int slabs = k.slabs;
  NodeIn in = ask_node(a, b, tid);
  f2 pq{0.0f, 0.0f};
  if (rounds > 0 && tid < a.n) pq = k.pq[(size_t)b * a.n + tid];
  __shared__ Nodes s;
  __shared__ Walk shared;
  __shared__ double sums[VIDKV_TREE_VOCAB / SLAB];
  __shared__ int found;
  if (count == 0) {
    for (int i = tid; i < a.n; i += 64 * W) a.path[(size_t)b * a.n + i] = -1;
    if (tid == 0) { a.accepted[b] = 0; a.next[b] = -1; }
    return;
  }
  State from{Walk{0, 0, 0.0, 1.0, 0.0, 0.0, NONE_MADE}, 0, 0};
  if (rounds > 0) {
    const int last = (rounds - 1) & 1;
    from = k.state[(size_t)last * gridDim.x + b];
    // (both arrays are asked for, so that one does not wait for the state)
    const double* made = k.sums + (size_t)b * slabs;
    for (int i = tid; i < slabs; i += 64 * W) {
      const double even = made[i], odd = made[(size_t)gridDim.x * slabs + i];
      sums[i] = from.at ? odd : even;
    }
  }
  keep_child(in, a, count, tid);
  if (rounds == 0) pq = gather<T>(in, a, b);
  put_node(s, in, pq, tid);
  __syncthreads();
  const bool drawn = a.draft.data != nullptr;
  Walk w = from.w;
  int tried[4] = {-1, -1, -1, -1};
  // whose sums are wanted: 0: what the walk asks for, 1: the last node's weights, 2: its row as it was, where nothing is left of it
  int of = from.done ? 1 : 0;
  bool here = from.done;                   // they are made already
  double total = 0.0, with = w.a;
  if (of) load_tried(tried, s, w.node, drawn, lane);
  for (;;) {
    if (of == 0) {
      if (w.sums == ASKED) take_sum(w, total_of(sums, slabs, lane));
      if (wv == 0) {
        walk_on(w, s, drawn, a.distinct, lane);
        if (lane == 0) shared = w;
      }
      __syncthreads();
      w = uniform(shared);
      __syncthreads();
      with = w.further;
      if (w.sums != ASKED) {
        of = 1;
        with = w.a;
        here = w.sums == HERE;
        load_tried(tried, s, w.node, drawn, lane);
      }
    }
    if (!here) {
      sum_slabs(sums, row_of<T>(a, b, w.node, with), tried, wv, W, slabs, lane);
      __syncthreads();
    }
    here = false;
    if (of == 0) continue;
    total = total_of(sums, slabs, lane);
    if (total > 0.0 || of == 2) break;
    of = 2;
    with = 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) tried[j] = -1;
    __syncthreads();
  }
  // the slab in which the sum passes u times the total, or the last one that has any
  const double goal = (double)s.u[0] * total;
  if (wv == 0) {
    double run = 0.0, before = 0.0;        // sums of the slabs looked at, and of those before the one taken
    int slab = -1, some = -1;
    for (int k0 = 0; k0 < slabs && slab < 0; k0 += 64) {
      const double mine = k0 + lane < slabs ? sums[k0 + lane] : 0.0;
      const double in = wave_scan(mine);
      const uint64_t over = __ballot(mine > 0.0 && run + in > goal), any = __ballot(mine > 0.0);
      if (over | any) {
        const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(any);
        if (over) slab = k0 + l;
        else some = k0 + l;
        before = run + lane_value(in - mine, l);
      }
      run += lane_value(in, 63);
    }
    if (slab < 0) slab = some;
    int token = -1;
    if (slab >= 0) {
      // its elements in order: lane takes 16 that lie next to each other
      const Row<T> r = row_of<T>(a, b, w.node, with);
      float p[16], q[16];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x[4], y[4];
        load4(r, slab * SLAB + 16 * lane + 4 * j, x, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) { p[4 * j + e] = x[e]; q[4 * j + e] = y[e]; }
      }
      clear_tried(tried, slab, [&](int i) { return 16 * lane + i; }, [&](int i) -> float& { return p[i]; });
      double v[16], mine = 0.0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v[i] = r.q ? weight(p[i], q[i], with) : (double)fmaxf(p[i], 0.0f);
        mine += v[i];
      }
      const double in = wave_scan(mine);
      double sum = before + (in - mine);
      int hit = -1, last = -1;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        sum += v[j];
        if (v[j] > 0.0) {
          last = j;
          if (hit < 0 && sum > goal) hit = j;
        }
      }
      const uint64_t hits = __ballot(hit >= 0), lasts = __ballot(last >= 0);
      const int l = hits ? __builtin_ctzll(hits) : lasts ? 63 - __builtin_clzll(lasts) : 0;
      const int j = __builtin_amdgcn_readlane(hits ? hit : last, l);
      token = j >= 0 ? slab * SLAB + 16 * l + j : -1;
    }
    if (lane == 0) {
      a.next[b] = token;
      int depth = 0;
      const int node = __builtin_amdgcn_readfirstlane(w.node);           // (a copy: the compiler chases w's address with the nodes')
      for (int i = node; i > 0; i = s.parent[i]) ++depth;
      found = depth + 1;
      a.accepted[b] = depth + 1;
      for (int i = node, d = depth; d >= 0; i = s.parent[i], --d) a.path[(size_t)b * a.n + d] = i;
    }
  }
  __syncthreads();
  for (int i = found + tid; i < a.n; i += 64 * W) a.path[(size_t)b * a.n + i] = -1;
}

// Launches that share a pass out to a sequence's workgroups, in front of the last one.  A row of up to 32 slabs is two a wave for the
// last launch's workgroup itself (chains over 16000 and 32000 tokens 9.7 and 9.9 us, with a launch in front 10.4 and 9.7; over
// 150000 20 and 10.9; 16 trees without a draft 21 and 13.7).  Chains, and trees without a draft, ask for one pass at most; of a
// tree that was drawn each child turned down asks for one, which costs some 9 us in the last launch, 3 in one of its own, and such a
// launch 2 to 3 where it is not needed (8 sequences of 24 nodes over 150000 tokens, 0 to 4 and 6: 66, 58, 49, 39, 33, 33; 64 of 4 nodes
// over 64000: 31, 31, 28, 25, 27, 32).
static int tree_rounds(const TreeVerify& a, int slabs) {
  return slabs <= 32 ? 0 : a.draft.data && a.parent ? std::max(1, std::min(a.n - 1, 4)) : 1;
}

static int slabs_of(int vocab) { return (vocab + SLAB - 1) / SLAB; }

size_t tree_verify_ws_bytes(int batch, int n, int vocab) {
  return align256(2 * (size_t)batch * sizeof(State)) + align256((size_t)batch * n * sizeof(f2)) +
         align256(2 * (size_t)batch * slabs_of(vocab) * sizeof(double));
}

hipError_t launch_tree_verify(const TreeVerify& a, int dtype, int batch, void* ws, hipStream_t st) {
  uint8_t* at = static_cast<uint8_t*>(ws);
  TreeWork k;
  k.slabs = slabs_of(a.vocab);
  k.state = reinterpret_cast<State*>(at);
  at += align256(2 * (size_t)batch * sizeof(State));
  k.pq = reinterpret_cast<f2*>(at);
  at += align256((size_t)batch * a.n * sizeof(f2));
  k.sums = reinterpret_cast<double*>(at);
  const int rounds = tree_rounds(a, k.slabs);
  // a slab a wave, up to six workgroups a compute unit (64 sequences, 150001 tokens: 16, 24 and 37 workgroups each 18.9, 18.2 and 20.8 us)
  const int share = std::max(1, std::min((k.slabs + 3) / 4, 6 * device_cu_count() / batch));
  auto go = [&](auto t) {
    using T = decltype(t);
    for (int r = 0; r < rounds; ++r)
      hipLaunchKernelGGL(tree_pass_kernel<T>, dim3(share, batch), dim3(256), 0, st, a, k, r);
    // (four waves where no pass is left for it)
    if (rounds > 0 && !(a.draft.data && a.parent)) hipLaunchKernelGGL((tree_finish_kernel<T, 4>), dim3(batch), dim3(256), 0, st, a, k, rounds);
    else hipLaunchKernelGGL((tree_finish_kernel<T, 16>), dim3(batch), dim3(1024), 0, st, a, k, rounds);
  };
  if (dtype == VIDKV_F32) go(PF32{});
  else if (dtype == VIDKV_F16) go(PF16{});
  else go(PBF16{});
  return hipGetLastError();
}

}  // namespace vidkv
