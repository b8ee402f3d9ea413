// Attention of a tree of drafted tokens over the 8-bit cache and over the tree's own keys and values.
//
// The rows are those of the attention over the cache (row = node * rep + head): every node sees all cached tokens, and of
// the drafted ones those that its mask has.  These are given in 16 bits and never coded - tokens that will mostly be rejected do not
// touch a block's magnitude - and join the running sums as blocks of 32 behind the cached ones, so that they cost no
// launch and no pass of their own.
#include "cache8_attn.h"
#include "tree.h"

namespace vidkv {

template <int NT, int CODE, int W, class T>
__global__ __launch_bounds__(64 * W, W > 4 ? W / 4 : NT < 3 ? 2 : 1) void c8_tree_few_kernel(C8Attn a, Tree<T>) {
  few_rows<NT, CODE, W, Tree<T>>(a);
}

template <int NT, int CODE, class T>
__global__ __launch_bounds__(256, 2) void c8_tree_many_kernel(C8Attn a, Tree<T>, int tiles) {
  many_rows<NT, CODE, Tree<T>>(a, tiles);
}

// The attention's plan, with fewer splits where its last workgroups would be a round of their own: it allows the next more
// than two a compute unit, and a tree's rows are seldom a divisor of them (64 nodes x 7 heads x 4 over 196000 tokens, three tiles: 43 splits
// are 516 workgroups, 329 us; 42 are 504, 220).  More than the plan's are not taken, so that its workspace does.  Costs as in
// c8_plan(); a round is two workgroups a compute unit, the last one's are alone if they are no more than one.  (Trees of very
// different sizes leave tiles without rows, whose workgroups end at once: two of 128 to 256 nodes, 25088 tokens, 7 splits 187 us, 6
// by this rule 206; both of 256 nodes 296 and 214.)
static C8Plan tree_plan(const C8Geom& g, int n) {
  C8Plan p = c8_plan(g, n);
  if (p.few) return p;
  const long long heads = (long long)g.H * g.B, wgs = p.tiles * heads, cu = device_cu_count();
  const float alone = 0.8f + 0.1f * p.nt, beside = p.nt == 1 ? 1.0f : p.nt == 2 ? 1.25f : 1.65f;
  const float blocks = (float)(g.nbc + (n + G - 1) / G), row_us = (float)heads * n * g.rep * (2 * 528 / 5e6f);
  float least = 0.0f;
  for (int k = 1, most = p.splits; k <= most; ++k) {
    const long long all = wgs * k, rest = all % (2 * cu);
    const float round = (float)(all / (2 * cu)) * beside + (rest == 0 ? 0.0f : rest <= cu ? alone : beside);
    const float us = blocks / k * round + (k > 1 ? 4.0f + row_us * k : 0.0f);
    if (k == 1 || us < least) { least = us; p.splits = k; }
  }
  return p;
}

hipError_t launch_c8_tree(const C8Geom& g, int layer, int n, float scale, const vidkv_view* q, const vidkv_view* K, const vidkv_view* V,
                          const uint64_t* mask, const uint8_t* cache, const int32_t* length, const int32_t* count,
                          const vidkv_view* out, void* ws, hipStream_t st) {
  const C8Plan p = tree_plan(g, n);
  const C8Attn a = c8_args(g, p, layer, n, 0, scale, q, cache, length, count, out, ws);
  auto go = [&](auto t, auto code) {
    using T = decltype(t);
    constexpr int CODE = decltype(code)::value;
    const Tree<T> tree{make_view(K), make_view(V), reinterpret_cast<const uint32_t*>(mask), (n + 63) / 64 * 2};
    const dim3 blk(256), few(p.splits, g.H, g.B), many(p.tiles * p.splits * g.H * g.B);
    if (p.few && p.waves == 12) hipLaunchKernelGGL((c8_tree_few_kernel<1, CODE, 12, T>), few, dim3(768), 0, st, a, tree);
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
  return hipGetLastError();
}

}  // namespace vidkv
