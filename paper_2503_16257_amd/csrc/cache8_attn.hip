// Attention over the 8-bit cache: out = softmax(scale q K'^T) V', any number of queries a sequence.
//
// The (query, query head) pairs of one KV head are the rows of one product, row = query * rep + head, so that the group
// shares what is read of the cache.  Per block of 32 tokens, on the matrix cores (codes as fp16 operands, exact):
//   x[token][row] = sum_c K[token][c] q[row][c]                       two tiles of 16 tokens
//   P = 2^(x ck + log2 A_v - m),  o[channel][row] += sum_t V[t][channel] P[t][row],  l += sum_t P / A_v
// with ck = A_k * scale * log2 e / level: the magnitude of a block's values goes into the exponent, where it costs an
// addition a row, and the accumulators stay in the codes' units.  out = o / (l level).  The maximum m of
// x ck + log2 A_v is a row's; it is raised only when a score exceeds it by 2^RISE, and P stays below 2^(RISE + UP) = 2^15, so
// that a P of 2^-29 of the largest still has fp16's 11 bits.
// bf16 queries become fp16 operands under a power of two of their own row.
#include "cache8.h"

namespace vidkv {

constexpr float RISE = 8.0f, UP = 7.0f;
constexpr float NONE = -1e30f;             // a maximum of nothing

struct C8Attn {
  View q, out;
  const uint8_t* kc;
  const uint8_t* vc;
  const float* km;
  const float* vm;
  const int32_t* length;
  const int32_t* q_count;      // or nullptr
  float* po;                   // partials [B * H * rows][splits][128], [..][splits][2]; nullptr: one split, straight to out
  float* pml;
  int H, rep, n, cap, nbc, splits, causal, bf16;
  float scale2;                // softmax scale * log2 e / level
  float inv_level;
};

__device__ __forceinline__ float max32(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max16(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum32(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum16(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Codes of one block as a lane takes them: 16 bytes of K for token x and x + 16 of channels 16 kb.. and 64 + 16 kb..; V as
// the record has them.
struct Block {
  u32x4 k[4], v[4];
  float km, vm;
};

template <int NT>
struct Rows {                  // a wave's 16 NT rows; lane: column x of each tile
  Op q[NT][4];
  float cq[NT];                // score factor of the row without A_k
  int limit[NT];               // tokens the row sees
  float m[NT], l[NT];
  f4 o[NT][8];
};

__device__ __forceinline__ void load_block(Block& f, const uint8_t* kc, const uint8_t* vc, const float* km, const float* vm,
                                           size_t blk, int lane) {
  const int x = lane & 15, kb = lane >> 4;
  const uint8_t* k = kc + blk * C8REC + x * D + kb * 16;
  const uint8_t* v = vc + blk * C8REC + lane * 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) f.k[i] = *reinterpret_cast<const u32x4*>(k + (i >> 1) * 16 * D + (i & 1) * 64);
#pragma unroll
  for (int i = 0; i < 4; ++i) f.v[i] = *reinterpret_cast<const u32x4*>(v + i * 1024);
  f.km = km[blk];
  f.vm = vm[blk];
}

// A row's denominator.  A query behind q_count went along where the others see every token: it has none.
template <int NT>
__device__ __forceinline__ float row_sum(const Rows<NT>& r, int t) {
  const float l = sum16(sum32(r.l[t]));
  return r.limit[t] > 0 ? l : 0.0f;
}

// Queries of 16 rows from `row0` on as operands; row = query * rep + head.
template <int NT>
__device__ __forceinline__ void load_rows(Rows<NT>& r, const C8Attn& a, int b, int h, int row0, int rows, int len, int nq, int lane) {
  const int x = lane & 15, kb = lane >> 4;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + 16 * t + x;
    const bool on = row < rows;
    const int i = on ? row / a.rep : 0, hd = on ? row - i * a.rep : 0;
    const char* p = a.q.data + b * a.q.sb + (long long)(h * a.rep + hd) * a.q.sh + i * a.q.st;
    f8v v[4];
    float big = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = (j >> 1) * 64 + kb * 16 + (j & 1) * 8;
      Op raw;
      raw.q = on ? *reinterpret_cast<const u32x4*>(p + 2 * c) : u32x4{0, 0, 0, 0};
      if (!a.bf16) {
        r.q[t][j] = raw;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[j][2 * e] = __uint_as_float(raw.u[e] << 16);
          v[j][2 * e + 1] = __uint_as_float(raw.u[e] & 0xffff0000u);
          big = fmaxf(big, fmaxf(fabsf(v[j][2 * e]), fabsf(v[j][2 * e + 1])));
        }
      }
    }
    float back = 1.0f;
    if (a.bf16) {                          // largest element to 2^14..2^15: eight bits are kept down to 2^-29 of it
      big = max16(max32(big));
      int e = 0;
      if (big > 0.0f && big < INFINITY) (void)frexpf(big, &e);
      const int up = min(max(15 - e, -120), 120);
      const float f = ldexpf(1.0f, up);
      back = ldexpf(1.0f, -up);
#pragma unroll
      for (int j = 0; j < 4; ++j) r.q[t][j].v = __builtin_convertvector(v[j] * f, h8);
    }
    r.cq[t] = a.scale2 * back;
    r.limit[t] = !on || i >= nq ? 0 : a.causal ? max(len - nq + i + 1, 0) : len;
    r.m[t] = NONE;
    r.l[t] = 0.0f;
#pragma unroll
    for (int m = 0; m < 8; ++m) r.o[t][m] = f4{0.f, 0.f, 0.f, 0.f};
  }
}

// One block's tokens t0 .. t0 + 31 into the running sums.  EDGE: some row does not see all of them.
template <int NT, int CODE, bool EDGE>
__device__ __forceinline__ void take_block(Rows<NT>& r, const Block& f, int t0, int len, int lane) {
  const int kb = lane >> 4;
  f4 s[NT][2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t][tt] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32x4 w = f.k[2 * tt + (j >> 1)];
      const Op k = decode8<CODE>(w[2 * (j & 1)], w[2 * (j & 1) + 1]);
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t][tt] = mma(k, r.q[t][j], s[t][tt]);
    }
  }
  const float lv = __log2f(f.vm) + UP, rv = __builtin_amdgcn_rcpf(f.vm);
  Op p[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float ck = r.cq[t] * f.km;
    float y[8], big = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v = s[t][i >> 2][i & 3] * ck;
      if (EDGE) v = t0 + slot_token(kb, i) < r.limit[t] ? v : -INFINITY;
      y[i] = v;
      big = fmaxf(big, v);
    }
    const float top = big + lv - UP;
    if (__any(top > r.m[t] + RISE)) {
      const float mn = fmaxf(r.m[t], max16(max32(top)));
      const float al = __builtin_amdgcn_exp2f(r.m[t] - mn);
      r.m[t] = mn;
      r.l[t] *= al;
#pragma unroll
      for (int m = 0; m < 8; ++m) r.o[t][m] *= al;
    }
    const float off = lv - r.m[t];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = __builtin_amdgcn_exp2f(y[i] + off);
      sum += y[i];
    }
    r.l[t] = fmaf(sum, rv, r.l[t]);
#pragma unroll
    for (int i = 0; i < 8; ++i) p[t].v[i] = (_Float16)y[i];
  }
#pragma unroll
  for (int m = 0; m < 8; ++m) {
    uint32_t u0 = f.v[m >> 1][2 * (m & 1)], u1 = f.v[m >> 1][2 * (m & 1) + 1];
    if (EDGE && CODE == 1) {               // bytes behind the length can be a NaN's
      const int n0 = len - t0 - 4 * kb, n1 = n0 - 16;
      u0 = n0 >= 4 ? u0 : n0 <= 0 ? 0u : u0 & ((1u << (8 * n0)) - 1);
      u1 = n1 >= 4 ? u1 : n1 <= 0 ? 0u : u1 & ((1u << (8 * n1)) - 1);
    }
    const Op v = decode8<CODE>(u0, u1);
#pragma unroll
    for (int t = 0; t < NT; ++t) r.o[t][m] = mma(v, p[t], r.o[t][m]);
  }
}

__device__ __forceinline__ void put_out(const C8Attn& a, int b, int h, int row, int c, const f4& v) {
  const int i = row / a.rep, hd = row - i * a.rep;
  char* p = a.out.data + b * a.out.sb + (long long)(h * a.rep + hd) * a.out.sh + i * a.out.st + 2 * c;
  if (a.bf16) {
    TBF16::store2(p, v[0], v[1]);
    TBF16::store2(p + 4, v[2], v[3]);
  } else {
    TF16::store2(p, v[0], v[1]);
    TF16::store2(p + 4, v[2], v[3]);
  }
}

// Waves share out the blocks of a split, for up to 16 NT rows a KV head.  grid (splits, H, B).
template <int NT, int CODE>
__global__ __launch_bounds__(256) void c8_few_kernel(C8Attn a) {
  const int b = blockIdx.z, h = blockIdx.y, sp = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, kb = lane >> 4;
  const int len = min(max(a.length[b], 0), a.cap);
  const int nq = a.q_count ? min(max(a.q_count[b], 0), a.n) : a.n;
  const int rows = a.n * a.rep;
  Rows<NT> r;
  load_rows<NT>(r, a, b, h, 0, rows, len, nq, lane);
  const int nb = (len + G - 1) / G, units = 4 * a.splits, un = 4 * sp + w;
  const int b0 = (int)((long long)un * nb / units), b1 = (int)((long long)(un + 1) * nb / units);
  const int all = a.causal ? max(len - nq + 1, 0) : len;          // tokens that every row sees
  const size_t head = ((size_t)b * a.H + h) * a.nbc;
  if (b0 < b1) {
    Block f, g;
    load_block(f, a.kc, a.vc, a.km, a.vm, head + b0, lane);
    for (int i = b0; i < b1; ++i) {
      if (i + 1 < b1) load_block(g, a.kc, a.vc, a.km, a.vm, head + i + 1, lane);
      if ((i + 1) * G <= all) take_block<NT, CODE, false>(r, f, i * G, len, lane);
      else take_block<NT, CODE, true>(r, f, i * G, len, lane);
      f = g;
    }
  }
  // the four waves' sums
  __shared__ f4 so[4][NT * 16][D / 4 + 1];
  __shared__ float sm[4][NT * 16], sl[4][NT * 16];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float l = row_sum(r, t);
    if (kb == 0) { sm[w][16 * t + x] = r.m[t]; sl[w][16 * t + x] = l; }
#pragma unroll
    for (int m = 0; m < 8; ++m) so[w][16 * t + x][4 * m + kb] = r.o[t][m];
  }
  __syncthreads();
  for (int e = tid; e < rows * (D / 4); e += 256) {
    const int row = e / (D / 4), c4 = e - row * (D / 4);
    float M = NONE;
#pragma unroll
    for (int k = 0; k < 4; ++k) M = fmaxf(M, sm[k][row]);
    f4 o = f4{0.f, 0.f, 0.f, 0.f};
    float l = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float wt = __builtin_amdgcn_exp2f(sm[k][row] - M);
      o += so[k][row][c4] * wt;
      l = fmaf(sl[k][row], wt, l);
    }
    if (a.po) {
      const size_t at = (((size_t)b * a.H + h) * rows + row) * a.splits + sp;
      reinterpret_cast<f4*>(a.po)[at * (D / 4) + c4] = o;
      if (c4 == 0) { a.pml[2 * at] = M; a.pml[2 * at + 1] = l; }
    } else {
      put_out(a, b, h, row, 4 * c4, l != 0.0f ? o * (a.inv_level / l) : f4{0.f, 0.f, 0.f, 0.f});
    }
  }
}

// Waves share out the rows: 16 NT a wave, 64 NT a workgroup, each walking the split's blocks.
// grid (row tiles x splits, H, B); the tiles that see most come first.
template <int NT, int CODE>
__global__ __launch_bounds__(256) void c8_many_kernel(C8Attn a, int tiles) {
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, kb = lane >> 4;
  const int tile = tiles - 1 - blockIdx.x / a.splits, sp = blockIdx.x % a.splits;
  const int len = min(max(a.length[b], 0), a.cap);
  const int nq = a.q_count ? min(max(a.q_count[b], 0), a.n) : a.n;
  const int rows = a.n * a.rep, row0 = tile * 64 * NT + w * 16 * NT;
  if (row0 >= rows) return;
  Rows<NT> r;
  load_rows<NT>(r, a, b, h, row0, rows, len, nq, lane);
  // tokens that the first of the wave's rows sees, and those that its last does
  const int i0 = row0 / a.rep, i1 = min((row0 + 16 * NT - 1) / a.rep, nq - 1);
  const int all = i1 < i0 ? 0 : a.causal ? max(len - nq + i0 + 1, 0) : len;
  const int most = i1 < i0 ? 0 : a.causal ? max(len - nq + i1 + 1, 0) : len;
  const int nb = (most + G - 1) / G;
  const int b0 = (int)((long long)sp * nb / a.splits), b1 = (int)((long long)(sp + 1) * nb / a.splits);
  const size_t head = ((size_t)b * a.H + h) * a.nbc;
  if (b0 < b1) {
    Block f, g;
    load_block(f, a.kc, a.vc, a.km, a.vm, head + b0, lane);
    for (int i = b0; i < b1; ++i) {
      if (i + 1 < b1) load_block(g, a.kc, a.vc, a.km, a.vm, head + i + 1, lane);
      if ((i + 1) * G <= all) take_block<NT, CODE, false>(r, f, i * G, len, lane);
      else take_block<NT, CODE, true>(r, f, i * G, len, lane);
      f = g;
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + 16 * t + x;
    const float l = row_sum(r, t);
    if (row >= rows) continue;
    if (a.po) {
      const size_t at = (((size_t)b * a.H + h) * rows + row) * a.splits + sp;
#pragma unroll
      for (int m = 0; m < 8; ++m) reinterpret_cast<f4*>(a.po)[at * (D / 4) + 4 * m + kb] = r.o[t][m];
      if (kb == 0) { a.pml[2 * at] = r.m[t]; a.pml[2 * at + 1] = l; }
    } else {
      const float f = l != 0.0f ? a.inv_level / l : 0.0f;
#pragma unroll
      for (int m = 0; m < 8; ++m) put_out(a, b, h, row, 16 * m + 4 * kb, l != 0.0f ? r.o[t][m] * f : f4{0.f, 0.f, 0.f, 0.f});
    }
  }
}

// out of the splits' partials: 32 lanes a row, eight rows a workgroup.  grid (ceil(rows / 8), H, B).
__global__ __launch_bounds__(256) void c8_merge_kernel(C8Attn a) {
  const int b = blockIdx.z, h = blockIdx.y, c4 = threadIdx.x & 31;
  const int rows = a.n * a.rep, row = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const size_t at = (((size_t)b * a.H + h) * rows + row) * a.splits;
  float M = NONE;
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, a.pml[2 * (at + s)]);
  f4 o = f4{0.f, 0.f, 0.f, 0.f};
  float l = 0.0f;
  for (int s = 0; s < a.splits; ++s) {
    const float wt = __builtin_amdgcn_exp2f(a.pml[2 * (at + s)] - M);
    o += reinterpret_cast<const f4*>(a.po)[(at + s) * (D / 4) + c4] * wt;
    l = fmaf(a.pml[2 * (at + s) + 1], wt, l);
  }
  put_out(a, b, h, row, 4 * c4, l != 0.0f ? o * (a.inv_level / l) : f4{0.f, 0.f, 0.f, 0.f});
}

// How a call is shared out.
struct C8Plan {
  int nt;                      // row tiles of 16 a wave
  bool few;                    // waves share blocks (all rows fit one wave), else rows
  int tiles, splits;
};

static C8Plan c8_plan(const C8Geom& g, int n) {
  C8Plan p{};
  const long long rows = (long long)n * g.rep;
  p.few = rows <= 32;
  p.nt = p.few && rows <= 16 ? 1 : 2;
  p.tiles = p.few ? 1 : (int)((rows + 64 * p.nt - 1) / (64 * p.nt));
  const long long wgs = (long long)p.tiles * g.H * g.B, want = 4LL * device_cu_count();
  long long s = (want + wgs - 1) / wgs;
  const long long most = p.few ? (g.nbc + 3) / 4 : (g.nbc + 7) / 8;
  p.splits = (int)std::max(1LL, std::min({s, most, 256LL}));
  return p;
}

size_t c8_attn_ws_bytes(const C8Geom& g, int n) {
  const C8Plan p = c8_plan(g, n);
  const size_t parts = p.splits > 1 ? (size_t)g.B * g.Hq * n * p.splits : 0;
  return align256(parts * (D + 2) * sizeof(float)) + 256;
}

hipError_t launch_c8_attn(const C8Geom& g, int layer, int n, int causal, float scale, const vidkv_view* q,
                          const uint8_t* cache, const int32_t* length, const int32_t* q_count, const vidkv_view* out,
                          void* ws, hipStream_t st) {
  const C8Plan p = c8_plan(g, n);
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
  a.H = g.H; a.rep = g.rep; a.n = n; a.cap = g.cap; a.nbc = g.nbc; a.splits = p.splits; a.causal = causal;
  a.bf16 = q->dtype == VIDKV_BF16;
  const float level = g.code == 0 ? 127.0f : 448.0f;
  a.scale2 = scale * 1.4426950408889634f / level;
  a.inv_level = 1.0f / level;
  const dim3 blk(256);
  auto by_code = [&](auto code) {
    constexpr int CODE = decltype(code)::value;
    const dim3 few(p.splits, g.H, g.B);
    if (p.few && p.nt == 1) hipLaunchKernelGGL((c8_few_kernel<1, CODE>), few, blk, 0, st, a);
    else if (p.few) hipLaunchKernelGGL((c8_few_kernel<2, CODE>), few, blk, 0, st, a);
    else hipLaunchKernelGGL((c8_many_kernel<2, CODE>), dim3(p.tiles * p.splits, g.H, g.B), blk, 0, st, a, p.tiles);
  };
  if (g.code == 0) by_code(std::integral_constant<int, 0>{});
  else by_code(std::integral_constant<int, 1>{});
  if (a.po) {
    const int rows = n * g.rep;
    hipLaunchKernelGGL(c8_merge_kernel, dim3((rows + 7) / 8, g.H, g.B), blk, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace vidkv
