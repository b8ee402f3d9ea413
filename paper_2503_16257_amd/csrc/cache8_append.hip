// Accepted tokens of a tree appended to the 8-bit cache of every layer in one launch.
//
// The codes are those of c8_write_kernel: a workgroup per block that a path can reach, of a head, sequence and layer; the rows come from
// the path's nodes.  A few tokens a sequence: bound by the chain start, path -> rows, the begun block's codes -> maximum -> codes.
#include "cache8_write.h"
#include "tree.h"

namespace vidkv {

// grid: blocks that a path can reach x H x B x L, blocks fastest.
template <class T, int CODE>
__global__ __launch_bounds__(256) void c8_append_kernel(C8Write a, Path path) {
  write_block<T, CODE, false>(a, path);
}

// Whether a grid holds an append to all layers: HIP counts a dimension's threads in 32 bits.
bool c8_append_fits(const C8Geom& g, int n) {
  return (unsigned __int128)c8_reach(g, n) * g.H * g.B * g.L < (1 << 24);
}

hipError_t launch_c8_append(const C8Geom& g, int n, const vidkv_view* K, long long k_layer, const vidkv_view* V, long long v_layer,
                            const int32_t* path, const int32_t* count, const int32_t* start, uint8_t* cache, hipStream_t st) {
  C8Write a{};
  a.K = make_view(K); a.V = make_view(V);
  a.n = n; a.start = start; a.count = count;
  a.kc = cache; a.vc = cache + g.v_codes;
  a.km = reinterpret_cast<float*>(cache + g.k_mag);
  a.vm = reinterpret_cast<float*>(cache + g.v_mag);
  a.H = g.H; a.nbc = g.nbc; a.cap = g.cap;
  a.n_axes = 1;
  const Path p{path, g.B, c8_reach(g, n), k_layer * 2, v_layer * 2};
  const dim3 grid((unsigned)((size_t)p.reach * g.H * g.B * g.L)), blk(256);
  auto go = [&](auto t) {
    using T = decltype(t);
    if (g.code == 0) hipLaunchKernelGGL((c8_append_kernel<T, 0>), grid, blk, 0, st, a, p);
    else hipLaunchKernelGGL((c8_append_kernel<T, 1>), grid, blk, 0, st, a, p);
  };
  if (K->dtype == VIDKV_F16) go(TF16{});
  else go(TBF16{});
  return hipGetLastError();
}

}  // namespace vidkv
