// Attention of a tree of drafted tokens over the 8-bit cache and over the tree's own keys and values.
//
// The rows are those of the attention over the cache (row = node * rep + head): every node sees all cached tokens, and of
// the drafted ones those that its mask has.  These are given in 16 bits and never coded - tokens that will mostly be rejected do not
// touch a block's magnitude - and join the running sums as blocks of 32 behind the cached ones, so that they cost no
// launch and no pass of their own.  What bounds it is what bounds the attention of as many rows: 64 nodes x 28 heads over 196000
// tokens, int8, 205 us, 0.88 PFLOP/s; 16 x 28 over 64 sequences of 12544 to 25088 tokens, e4m3, 430; 6 x 32 over 16 of 3000 to 6001
// 26; one head of 1568 tokens 5.9.  The drafted blocks are 1.4 to 4 us of these (the last of a wave's work, by code that is
// fetched for it alone), 10 of the 430.
#include "cache8_attn.h"
#include "tree.h"
#include <algorithm>
#include <cmath>

namespace vidkv {

template <int NT, int CODE, int W, class T>
__global__ __launch_bounds__(64 * W, W > 4 ? W / 4 : NT < 3 ? 2 : 1) void c8_tree_few_kernel(C8Attn a, Tree<T>) {
  few_rows<NT, CODE, W, Tree<T>>(a);
}

template <int NT, int CODE, class T>
__global__ __launch_bounds__(256, 2) void c8_tree_many_kernel(C8Attn a, Tree<T>, int tiles) {
  __shared__ ManyLds<Tree<T>, (NT < 3), NT> lds;
  many_rows<NT, CODE, Tree<T>>(a, even_span<NT>(a, blockIdx.x, tiles), lds);
}

// Rows that are some tiles of 192 and a rest of up to 128: the rest's workgroups have one or two tiles a wave, a block takes them
// less time, and so the rest has fewer splits (`few` of a.splits).  Workgroups of the rest come first.
template <int REST, int CODE, class T>
__global__ __launch_bounds__(256, 2) void c8_tree_mixed_kernel(C8Attn a, Tree<T>, int full, int few) {
  __shared__ ManyLds<Tree<T>, true, 3> lds;
  int at = blockIdx.x;
  const int h = at % a.H; at /= a.H;
  const int b = at % a.B; at /= a.B;
  const bool rest = at < few;
  ManySpan span{b, h, full * 192, at, few};
  if (!rest) span = ManySpan{b, h, (at - few) % full * 192, (at - few) / full, a.splits};
  asm volatile("" : "+s"(span.b), "+s"(span.h), "+s"(span.tile0), "+s"(span.sp), "+s"(span.splits));
  if (rest) many_rows<REST, CODE, Tree<T>>(a, span, lds);
  else many_rows<3, CODE, Tree<T>>(a, span, lds);
}

struct TreePlan {
  C8Plan p;
  int full, few;               // mixed: tiles of 192 rows, splits of the rest; few = 0: tiles of one size
};

// The attention's plan, with splits of its own for more rows than a wave's: that one allows the next more than two workgroups a
// compute unit, and a tree's rows are seldom a divisor of them (64 nodes x 7 heads x 4 over 196000 tokens, three tiles: 43 splits are
// 516 workgroups, 329 us; 42 are 504, 217).  Costs as in c8_plan(); a round is two workgroups a compute unit, the last one's are alone if
// they are no more than one.  A rest of up to 128 rows behind tiles of 192 has one or two tiles a wave, and fewer splits in the ratio of
// what a block costs (those 448 rows: 49 splits of two tiles of 192, 30 of 64 rows, 205 us; 231 rows 160 -> 133).  No more splits than the
// size query has room for, which walks the attention's calls of up to n queries (1 to 6 us of the host's time: asked only
// for more than the attention's own splits, that are always there); whatever more a workspace holds, a call's sums keep their
// order.  (Trees of very different sizes leave tiles without rows, whose workgroups end at once, and so more splits would do for them.)
static TreePlan tree_plan(const C8Geom& g, int n) {
  TreePlan t{c8_plan(g, n), 0, 0};
  C8Plan& p = t.p;
  if (p.few) return t;
  const int own = p.splits;
  const long long heads = (long long)g.H * g.B, rows = (long long)n * g.rep, cu = device_cu_count();
  auto alone = [](int nt) { return 0.8f + 0.1f * nt; };
  auto beside = [](int nt) { return nt == 1 ? 1.0f : nt == 2 ? 1.25f : 1.65f; };
  const float blocks = (float)(g.nbc + (n + G - 1) / G), row_us = (float)heads * rows * (2 * 528 / 5e6f);
  const int full = (int)(rows / 192), rest = (int)(rows % 192), nt = rest <= 64 ? 1 : 2;
  const bool mixes = p.nt == 3 && full > 0 && rest > 0 && rest <= 128;
  // (splits beyond a round of workgroups are looked at where there is about one without)
  const long long enough = p.tiles * heads > cu ? 8 * cu : 2 * cu, step = (mixes ? full : p.tiles) * heads;
  auto cheapest = [&](long long most) {
    float least = 0.0f;
    for (int k = 1; k <= most && (k == 1 || step * (k - 1) < enough); ++k) {
      const float merge = k > 1 ? 4.0f + row_us * k : 0.0f;
      const long long all = p.tiles * heads * k, left = all % (2 * cu);
      const float rounds = (float)(all / (2 * cu)) * beside(p.nt) + (left == 0 ? 0.0f : left <= cu ? alone(p.nt) : beside(p.nt));
      const float us = blocks / k * rounds + merge;
      if (k == 1 || us < least) { least = us; p.splits = k; t.few = 0; }
      const int few = (int)ceilf(k * beside(nt) / beside(3));
      const long long both = heads * (full * (long long)k + few);
      const float mixed = blocks / k * (both <= cu ? alone(3) : beside(3)) + merge;
      if (mixes && both <= 2 * cu && mixed < least) { least = mixed; p.splits = k; t.few = few; t.full = full; }
    }
  };
  const long long most = std::min(256LL, (g.nbc + 7LL) / 8);
  cheapest(most);
  if (p.splits > own) {
    const long long room = (long long)((c8_attn_ws_bytes(g, n) - 256) / (heads * rows * (D + 2) * sizeof(float)));
    if (p.splits > room) cheapest(std::min(most, std::max(1LL, room)));
  }
  return t;
}

vidkv_status launch_c8_tree(const C8Geom& g, int layer, int n, float scale, const vidkv_view* q, const vidkv_view* K, const vidkv_view* V,
                            const uint64_t* mask, const uint8_t* cache, const int32_t* length, const int32_t* count,
                            const vidkv_view* out, void* ws, size_t ws_bytes, hipStream_t st) {
  const TreePlan plan = tree_plan(g, n);
  const C8Plan& p = plan.p;
  if (ws_bytes < c8_parts(g, (long long)n * g.rep, p.splits) + 256) return VIDKV_ENOSPACE;
  const C8Attn a = c8_args(g, p, layer, n, 0, scale, q, cache, length, count, out, ws);
  auto go = [&](auto t, auto code) {
    using T = decltype(t);
    constexpr int CODE = decltype(code)::value;
    const Tree<T> tree{make_view(K), make_view(V), reinterpret_cast<const uint32_t*>(mask), (n + 63) / 64 * 2};
    const dim3 blk(256), few(p.splits, g.H, g.B), many(p.tiles * p.splits * g.H * g.B);
    if (plan.few) {
      const dim3 mixed((unsigned)((long long)(plan.full * p.splits + plan.few) * g.H * g.B));
      if (n * g.rep % 192 <= 64) hipLaunchKernelGGL((c8_tree_mixed_kernel<1, CODE, T>), mixed, blk, 0, st, a, tree, plan.full, plan.few);
      else hipLaunchKernelGGL((c8_tree_mixed_kernel<2, CODE, T>), mixed, blk, 0, st, a, tree, plan.full, plan.few);
    } else if (p.few && p.waves == 12) hipLaunchKernelGGL((c8_tree_few_kernel<1, CODE, 12, T>), few, dim3(768), 0, st, a, tree);
    else if (p.few && p.nt == 1) hipLaunchKernelGGL((c8_tree_few_kernel<1, CODE, 4, T>), few, blk, 0, st, a, tree);
    else if (p.few && p.nt == 2) hipLaunchKernelGGL((c8_tree_few_kernel<2, CODE, 4, T>), few, blk, 0, st, a, tree);
    else if (p.few) hipLaunchKernelGGL((c8_tree_few_kernel<3, CODE, 4, T>), few, blk, 0, st, a, tree);
    else if (p.nt == 1) hipLaunchKernelGGL((c8_tree_many_kernel<1, CODE, T>), many, blk, 0, st, a, tree, p.tiles);
    else if (p.nt == 2) hipLaunchKernelGGL((c8_tree_many_kernel<2, CODE, T>), many, blk, 0, st, a, tree, p.tiles);
    else hipLaunchKernelGGL((c8_tree_many_kernel<3, CODE, T>), many, blk, 0, st, a, tree, p.tiles);
  };
  auto by_code = [&](auto t) {
    if (g.code == 0) go(t, std::integral_constant<int, 0>{});
    else go(t, std::integral_constant<int, 1>{});
  };
  if (q->dtype == VIDKV_F16) by_code(TF16{});
  else by_code(TBF16{});
  launch_c8_merge(a, st);
  return hipGetLastError() == hipSuccess ? VIDKV_OK : VIDKV_EHIP;
}

}  // namespace vidkv
