// Attention over the 8-bit cache, any number of queries a sequence: kernels, their merge, how a call is shared out.
#include "cache8_attn.h"
#include <algorithm>

namespace vidkv {

template <int NT, int CODE, int W>
__global__ __launch_bounds__(64 * W, W > 4 ? W / 4 : NT < 3 ? 2 : 1) void c8_few_kernel(C8Attn a) {
  few_rows<NT, CODE, W, NoTree>(a);
}

template <int NT, int CODE>
__global__ __launch_bounds__(256, 2) void c8_many_kernel(C8Attn a, int tiles) {
  __shared__ ManyLds<NoTree, false, NT> lds;
  many_rows<NT, CODE, NoTree>(a, even_span<NT>(a, blockIdx.x, tiles), lds);
}

// out of the splits' partials.  A row is taken by 32 SL threads, 32 channel quads x SL slices of its splits, eight
// splits asked for at a time; 256 / (32 SL) rows a workgroup.  grid (ceil(rows / rows a workgroup), H, B).
template <int SL>
__global__ __launch_bounds__(256) void c8_merge_kernel(C8Attn a) {
  // (all arguments in one round trip; left to itself the compiler asks for each where it is used)
  asm volatile("" :: "s"(a.out.data), "s"(a.out.sb), "s"(a.out.sh), "s"(a.out.st), "s"(a.po), "s"(a.pml), "s"(a.H), "s"(a.rep),
               "s"(a.n), "s"(a.splits), "s"(a.bf16), "s"(a.inv_level));
  const int b = blockIdx.z, h = blockIdx.y, c4 = threadIdx.x & 31, sl = (threadIdx.x >> 5) % SL, rr = (threadIdx.x >> 5) / SL;
  const int rows = a.n * a.rep, row = blockIdx.x * (8 / SL) + rr;
  const bool on = row < rows;
  const size_t at = (((size_t)b * a.H + h) * rows + (on ? row : 0)) * a.splits;
  const f4* po = reinterpret_cast<const f4*>(a.po) + at * (D / 4) + c4;
  const f2* pm = reinterpret_cast<const f2*>(a.pml) + at;
  float M = NONE, l = 0.0f;
  f4 o = f4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = sl; s0 < a.splits; s0 += 8 * SL) {
    f4 v[8];
    f2 ml[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int s = min(s0 + u * SL, a.splits - 1);           // (behind the last: a split again, not counted)
      ml[u] = pm[s];
      v[u] = po[(size_t)s * (D / 4)];
    }
    // (left to itself the compiler waits for (m, l) first, and for the sums only behind the maximum)
#pragma unroll
    for (int u = 0; u < 8; ++u) asm volatile("" : "+v"(v[u]), "+v"(ml[u]));
    float top = M;
#pragma unroll
    for (int u = 0; u < 8; ++u) top = fmaxf(top, ml[u][0]);
    const float al = __builtin_amdgcn_exp2f(M - top);
    M = top;
    o *= al;
    l *= al;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float wt = s0 + u * SL < a.splits ? __builtin_amdgcn_exp2f(ml[u][0] - M) : 0.0f;
      o += v[u] * wt;
      l = fmaf(ml[u][1], wt, l);
    }
  }
  if constexpr (SL > 1) {
    __shared__ f4 so[8][32];
    __shared__ float sm[8], sl_[8];
    const int k = threadIdx.x >> 5;
    so[k][c4] = o;
    if (c4 == 0) { sm[k] = M; sl_[k] = l; }
    __syncthreads();
    if (sl != 0) return;
    const int k0 = rr * SL;
    M = NONE;
    for (int i = 0; i < SL; ++i) M = fmaxf(M, sm[k0 + i]);
    o = f4{0.f, 0.f, 0.f, 0.f};
    l = 0.0f;
    for (int i = 0; i < SL; ++i) {
      const float wt = __builtin_amdgcn_exp2f(sm[k0 + i] - M);
      o += so[k0 + i][c4] * wt;
      l = fmaf(sl_[k0 + i], wt, l);
    }
  }
  if (on) put_out(a, b, h, row, 4 * c4, l != 0.0f ? o * (a.inv_level / l) : f4{0.f, 0.f, 0.f, 0.f});
}

// Up to 48 rows a head are a wave's, and waves share the blocks; more are shared out over waves, which walk the blocks together (e4m3,
// 24, 32, 40 and 48 rows of 4 heads, this way and that: one sequence of 98208 tokens 24.6, 25.2, 27.5, 27.3 and 32.1, 32.7, 33.2,
// 33.9 us; 16 of up to 6001 19.6, 19.2, 23.9, 25.0 and 26.9, 25.2, 26.6, 28.4; 64 of 6016 78, 80, 91, 89 and 100, 101, 103, 104; a
// fourth tile a wave, at 56 and 64 rows: 32.3, 33.0 against 35.0, 37.6; 30.6, 30.1 against 28.7, 28.5; 102, 104 against 107, 110).
// Waves that share blocks do best in one round of workgroups: each costs some 3 us before its first product and its partials as long
// behind the last (196000 tokens, 4 heads: 40.8 us with a workgroup a compute unit, 42.1 with two, 45.1 with four; 16 sequences of up to
// 6001 tokens, 40 rows: 23.8, 29.3, 38.8).
// Where the heads are three quarters of the compute units or more, for caches of up to 2048 tokens half of them, a workgroup
// of twelve waves takes a head and there is no merge (64 x 4 heads of 512 tokens 13.2 -> 8.9 us, of 8192 113 -> 91; 1024 heads of
// 2048 tokens 109 -> 100, but of 384 tokens 19 -> 29; 128 heads of 2048 tokens 16.5 -> 15.1, of 2048 to 4096 23.2 -> 27.8),
// and so it does for a cache of a block a wave (4 heads of 256 tokens 6.6 -> 5.6; of 1024 tokens 6.9 -> 9.0).  Its sequences
// may differ in length: then up to four a compute unit, while a wave keeps 16 blocks (64 sequences of 12544 to 25088 tokens:
// 173 us unsplit, 156 in four; 16 of up to 6272, a block a wave: 19 and 44).
C8Plan c8_plan(const C8Geom& g, int n) {
  C8Plan p{};
  const long long rows = (long long)n * g.rep, heads = (long long)g.H * g.B, cu = device_cu_count();
  p.few = rows <= 48;
  if (!p.few) {
    p.nt = rows <= 64 ? 1 : rows <= 128 ? 2 : 3;
    p.tiles = (int)((rows + 64 * p.nt - 1) / (64 * p.nt));
    // Splits, up to two workgroups a compute unit, by what they cost: a block takes a workgroup 0.9 to 1.1 us where it has
    // the unit for itself, 1.0 to 1.65 beside another; a row's partials are 528 bytes written and read, at 5 TB/s, the
    // merge's launch 4 us.  (112 rows of 256 heads over 1024 tokens: 31.0 us unsplit, 35.4 in two; 56 rows over 4096: 109 and 78;
    // 1372 rows of 32 heads over 512: 23 and 36.)
    const long long wgs = p.tiles * heads;
    p.most = (int)std::min({(2 * cu + wgs - 1) / wgs, (g.nbc + 7LL) / 8, 256LL});
    const float alone = 0.8f + 0.1f * p.nt, beside = p.nt == 1 ? 1.0f : p.nt == 2 ? 1.25f : 1.65f;
    float least = 0.0f;
    for (int k = 1; k <= p.most; ++k) {
      const float us = (float)g.nbc / k * (wgs * k <= cu ? alone : beside) +
                       (k > 1 ? 4.0f + (float)heads * (float)rows * k * (2 * 528 / 5e6f) : 0.0f);
      if (k == 1 || us < least) { least = us; p.splits = k; }
    }
    return p;
  }
  p.nt = (int)(rows + 15) / 16;
  p.tiles = 1;
  const bool filled = 4 * heads >= 3 * cu || (2 * heads >= cu && g.nbc <= 64);
  const bool wide = p.nt == 1 && (filled ? heads < 4 * cu || g.nbc >= 40 : g.nbc <= 12);
  p.waves = wide ? 12 : 4;
  const long long fill = (cu + heads - 1) / heads;
  long long s = wide ? 1 : fill;
  if (filled) s = std::max(s, std::min(g.B > 1 ? std::max(fill, 4 * cu / heads) : fill, (long long)g.nbc / (16 * p.waves)));
  p.splits = (int)std::max(1LL, std::min({s, (g.nbc + 3LL) / 4, 256LL}));
  return p;
}

// Bytes of a call's partials.
size_t c8_parts(const C8Geom& g, long long rows, int splits) {
  return splits > 1 ? align256((size_t)g.B * g.H * rows * splits * (D + 2) * sizeof(float)) : 0;
}
size_t c8_attn_ws_need(const C8Geom& g, int n) { return c8_parts(g, (long long)n * g.rep, c8_plan(g, n).splits) + 256; }

// ... and of the largest of the calls of up to n queries: fewer rows can mean more splits.  The plan changes with the
// tiles of 16 or 192 rows, and within a tile more rows never mean more splits (a split costs each row the same).  Over the tiles the
// splits do not fall steadily: where the workgroups pass the compute units a block takes longer, and a call is split again that was
// not with fewer tiles.  They end where no more than one can be: two workgroups a compute unit without, or eight blocks in all.
size_t c8_attn_ws_bytes(const C8Geom& g, int n) {
  size_t most = 0;
  for (long long q = 1; q <= n;) {
    const C8Plan p = c8_plan(g, (int)q);
    if (!p.few && p.most == 1) break;
    const long long rows = p.few ? 16LL * p.nt : 64LL * p.nt * p.tiles;          // the last of this plan
    const long long last = std::max(q, std::min<long long>(n, rows / g.rep));
    most = std::max(most, c8_parts(g, last * g.rep, p.splits));
    q = last + 1;
  }
  return most + 256;
}

// Whether a grid holds the call: HIP counts a dimension's threads in 32 bits.
bool c8_attn_fits(const C8Geom& g, int n) {
  const C8Plan p = c8_plan(g, n);
  return p.few || (long long)p.tiles * p.splits * g.H * g.B < (1 << 24);
}

C8Attn c8_args(const C8Geom& g, const C8Plan& p, int layer, int n, int causal, float scale, const vidkv_view* q, const uint8_t* cache,
               const int32_t* length, const int32_t* q_count, const vidkv_view* out, void* ws) {
  const size_t blk0 = (size_t)layer * g.B * g.H * g.nbc;
  C8Attn a{};
  a.q = make_view(q); a.out = make_view(out);
  a.kc = cache + blk0 * C8REC;
  a.vc = cache + g.v_codes + blk0 * C8REC;
  a.km = reinterpret_cast<const float*>(cache + g.k_mag) + blk0;
  a.vm = reinterpret_cast<const float*>(cache + g.v_mag) + blk0;
  a.length = length; a.q_count = q_count;
  if (p.splits > 1) {
    a.po = static_cast<float*>(ws);
    a.pml = a.po + (size_t)g.B * g.Hq * n * p.splits * D;
  }
  a.B = g.B; a.H = g.H; a.rep = g.rep; a.n = n; a.cap = g.cap; a.nbc = g.nbc; a.splits = p.splits; a.causal = causal;
  a.bf16 = q->dtype == VIDKV_BF16;
  const float level = g.code == 0 ? 127.0f : 448.0f;
  a.scale2 = scale * 1.4426950408889634f / level;
  a.inv_level = 1.0f / level;
  return a;
}

void launch_c8_merge(const C8Attn& a, hipStream_t st) {
  if (!a.po) return;
  const int rows = a.n * a.rep;
  auto merge = [&](auto sl) {
    constexpr int SL = decltype(sl)::value;
    hipLaunchKernelGGL(c8_merge_kernel<SL>, dim3((rows + 8 / SL - 1) / (8 / SL), a.H, a.B), dim3(256), 0, st, a);
  };
  if (a.splits > 32) merge(std::integral_constant<int, 8>{});
  else if (a.splits > 16) merge(std::integral_constant<int, 4>{});
  else if (a.splits > 8) merge(std::integral_constant<int, 2>{});
  else merge(std::integral_constant<int, 1>{});
}

hipError_t launch_c8_attn(const C8Geom& g, int layer, int n, int causal, float scale, const vidkv_view* q,
                          const uint8_t* cache, const int32_t* length, const int32_t* q_count, const vidkv_view* out,
                          void* ws, hipStream_t st) {
  const C8Plan p = c8_plan(g, n);
  const C8Attn a = c8_args(g, p, layer, n, causal, scale, q, cache, length, q_count, out, ws);
  const dim3 blk(256);
  auto by_code = [&](auto code) {
    constexpr int CODE = decltype(code)::value;
    const dim3 few(p.splits, g.H, g.B), many(p.tiles * p.splits * g.H * g.B);
    if (p.few && p.waves == 12) hipLaunchKernelGGL((c8_few_kernel<1, CODE, 12>), few, dim3(768), 0, st, a);
    else if (p.few && p.nt == 1) hipLaunchKernelGGL((c8_few_kernel<1, CODE, 4>), few, blk, 0, st, a);
    else if (p.few && p.nt == 2) hipLaunchKernelGGL((c8_few_kernel<2, CODE, 4>), few, blk, 0, st, a);
    else if (p.few) hipLaunchKernelGGL((c8_few_kernel<3, CODE, 4>), few, blk, 0, st, a);
    else if (p.nt == 1) hipLaunchKernelGGL((c8_many_kernel<1, CODE>), many, blk, 0, st, a, p.tiles);
    else if (p.nt == 2) hipLaunchKernelGGL((c8_many_kernel<2, CODE>), many, blk, 0, st, a, p.tiles);
    else hipLaunchKernelGGL((c8_many_kernel<3, CODE>), many, blk, 0, st, a, p.tiles);
  };
  if (g.code == 0) by_code(std::integral_constant<int, 0>{});
  else by_code(std::integral_constant<int, 1>{});
  launch_c8_merge(a, st);
  return hipGetLastError();
}

}  // namespace vidkv
