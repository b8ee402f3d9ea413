// Accepted tokens of a tree appended to the 8-bit cache of every layer in one launch.
//
// The codes are those of c8_write_kernel; the rows come from the path's nodes.  A few tokens a sequence: bound by the chain start, path -> rows, the begun block's codes -> maximum -> codes.
#include "cache8_write.h"
#include "tree.h"

namespace vidkv {

// A workgroup a head of a sequence of a layer walks the blocks that the path reaches, mostly one.  28 x 64 x 4 heads, 64 nodes of which
// 1 to 8 stand: 41 us for 53 MB read and 38 written, 18 at a copy's rate (a begun block's value record is read and written whole: its
// bytes are in the attention's order), half of a wave's time waiting for them; 32 to 34 on a cache that the call before has just appended
// to.  On such a cache: a workgroup for each block that 64 nodes could reach, most of them without work, 51; live keys' codes
// asked for at once and not when they are to be coded anew, 34; two to five layers a workgroup, or two more workgroups a compute
// unit with some registers spilled, as this one.  grid (H x B x L), heads fastest.
template <class T, int CODE>
__global__ __launch_bounds__(256) void c8_append_kernel(C8Write a, Path path) {
  ask_arguments(a);
  const int tid = threadIdx.x;
  int at = blockIdx.x;
  const int h = at % a.H; at /= a.H;
  const int b = at % path.B, layer = at / path.B;
  const int node = tid < a.n ? path.path[(size_t)b * a.n + tid] : -1;
  const int start = a.start[b];
  __shared__ int nodes[VIDKV_TREE_NODES], ends[4];
  nodes[tid] = node;
  const uint64_t none = __ballot(node < 0 || node >= a.n);     // the path ends before the first entry that is no node
  if ((tid & 63) == 0) ends[tid >> 6] = none ? tid + __builtin_ctzll(none) : VIDKV_TREE_NODES;
  __syncthreads();
  const int count = min(min(min(ends[0], ends[1]), min(ends[2], ends[3])), a.count[b]);
  if (start < 0) return;
  for (int nth = 0; (start / G + nth) * (long long)G < (long long)start + count; ++nth) {
    write_block<T, CODE, false>(a, path, b, h, layer, nth, start, count, nodes);
    __syncthreads();                       // (its LDS is the next one's)
  }
}

// Whether a grid holds an append to all layers: HIP counts a dimension's threads in 32 bits.
bool c8_append_fits(const C8Geom& g) { return (unsigned __int128)g.H * g.B * g.L < (1 << 24); }

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
  const Path p{path, g.B, k_layer * 2, v_layer * 2};
  const dim3 grid((unsigned)((size_t)g.H * g.B * g.L)), blk(256);
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
