// Attention over the 8-bit cache: out = softmax(scale q K'^T) V', any number of queries a sequence.
//
// The (query, query head) pairs of one KV head are the rows of one product, row = query * rep + head, so that the group
// shares what is read of the cache.  Per block of 32 tokens, on the matrix cores (codes as fp16 operands, exact):
//   x[token][row] = sum_c K[token][c] q[row][c]                       two tiles of 16 tokens
//   P = 2^(x ck + log2 A_v - m),  o[channel][row] += sum_t V[t][channel] P[t][row],  l += sum_t P / A_v
// with ck = A_k * scale * log2 e / level: the magnitude of a block's values goes into the exponent, where it costs an
// addition a row, and the accumulators stay in the codes' units.  out = o / (l level).  The maximum m of
// x ck + log2 A_v is a row's; it is raised only when a score exceeds it by 2^RISE, and P stays below 2^(RISE + UP) = 2^15.
// P is rounded to fp16, 11 bits down to 2^-14: down to 2^-21 of the largest where the maximum has just been raised (the largest is
// 2^UP then), 2^-29 where it is about to be; below, what is lost is 2^-32 of the largest at most.
// bf16 queries become fp16 operands under a power of two of their own row.
#include "cache8.h"
#include <algorithm>

namespace vidkv {

constexpr float RISE = 8.0f, UP = 7.0f;
constexpr float NONE = -1e30f;             // a maximum of nothing
constexpr uint32_t FAR = 3u << 23;         // a block's values are far below another's: by more than 2^3 (exponents, in place)

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
  int B, H, rep, n, cap, nbc, splits, causal, bf16;
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

// A block's magnitude as the sums take it, a wave's scalar.  A cleared buffer's, of a block that was never written, is zero: tokens
// of zeros, as they are read back, and no quotient by it.  (Magnitudes are not below zero, and compare as their bits do.)
__device__ __forceinline__ uint32_t held_bits(float mag) {
  return max((uint32_t)__builtin_amdgcn_readfirstlane(__float_as_uint(mag)), __float_as_uint(C8_LEAST));
}

// A row's maximum and denominator.  A query behind q_count went along where the others see every token: it has none, and
// whatever it is (an infinity times a weight of none would be no number) it gives zeros.
template <int NT>
__device__ __forceinline__ f2 row_stats(const Rows<NT>& r, int t) {
  return r.limit[t] > 0 ? f2{r.m[t], r.l[t]} : f2{NONE, 0.0f};
}

// The sum of a block's weights P over its tokens, in every lane, as a product with ones: of the weights as the other product
// takes them, rounded, so that equal ones are rounded alike above and below.  P carries A_v, the weight does not: where A_v is
// far below the largest before it, P can lose bits in fp16, or vanish, whose weight is as large as any (a block of zeros has
// A_v = 2^-40).  Such a block's sum is taken in float32; of others what fp16 loses is 2^-29 of the largest weight, a token.
// (196 queries over 98196 tokens, vector units the bound: no such block 271 us, every second one 302, all but the first 341; without
// the look at the magnitudes 268.  Few queries, memory the bound: the same times, 40 rows 25.4, 26.7, 25.7.)
__device__ __forceinline__ float sum_of(const Op& p) {
  Op ones;
#pragma unroll
  for (int i = 0; i < 4; ++i) ones.u[i] = 0x3c003c00u;
  return mma(ones, p, f4{0.f, 0.f, 0.f, 0.f})[0];
}
__device__ __forceinline__ float far_sum(const f4 (&s)[2], float ck, float off) {
  asm volatile("" : "+v"(off));            // (not seen to be off: nothing of the common path is moved up here and kept)
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) sum += __builtin_amdgcn_exp2f(fmaf(s[k >> 2][k & 3], ck, off));
  return sum16(sum32(sum));
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
    // (bounded so that its products with a magnitude, 2^-40..2^40, neither vanish nor leave float's range: a masked score times
    // them, or one of zero, would be no number.  Below the bound a row's weights are equal; above, a score that is not zero is 2^23 at
    // least, of sums of 2^-24 and up.)
    r.cq[t] = fminf(fmaxf(a.scale2 * back, 0x1p-86f), 0x1p87f);
    r.limit[t] = !on || i >= nq ? 0 : a.causal ? max(len - nq + i + 1, 0) : len;
    r.m[t] = NONE;
    r.l[t] = 0.0f;
#pragma unroll
    for (int m = 0; m < 8; ++m) r.o[t][m] = f4{0.f, 0.f, 0.f, 0.f};
  }
}

// Nothing is moved across it.
__device__ __forceinline__ void hold_order() { __builtin_amdgcn_sched_barrier(0); }

// One block's tokens t0 .. t0 + 31 into the running sums; k(tt, j), v(m): its operands, tile of 16 tokens and 32 channels
// of them, tile of 16 channels.  edge: some row does not see all of its tokens.  far: its values are far below others.
template <int NT, class K, class V>
__device__ __forceinline__ void take_block(Rows<NT>& r, const K& k, const V& v, float km, float vm, bool edge, bool far,
                                           int t0, int lane) {
  const int kb = lane >> 4;
  // operands are asked for two ahead of their products, and the order is held: left to itself the compiler asks for all of
  // them at once and has no registers left
  f4 s[NT][2];
  Op n0 = k(0, 0), n1 = k(0, 1);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const Op o0 = n0, o1 = n1;
    if (g < 3) { n0 = k((g + 1) >> 1, 2 * ((g + 1) & 1)); n1 = k((g + 1) >> 1, 2 * ((g + 1) & 1) + 1); }
    else { n0 = v(0); n1 = v(1); }
    hold_order();
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t][g >> 1] = mma(o0, r.q[t][2 * (g & 1)], g & 1 ? s[t][g >> 1] : f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t][g >> 1] = mma(o1, r.q[t][2 * (g & 1) + 1], s[t][g >> 1]);
    hold_order();
  }
  const float lv = __log2f(vm);
  float rv = __builtin_amdgcn_rcpf(vm);
  Op p[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float ck = r.cq[t] * km;
    if (edge) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (t0 + slot_token(kb, i) >= r.limit[t]) s[t][i >> 2][i & 3] = -INFINITY;
    }
    float big = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = fmaxf(big, s[t][i >> 2][i & 3]);
    const float top = fmaf(big, ck, lv);
    if (__any(top > r.m[t] + RISE)) {
      const float mn = fmaxf(r.m[t], max16(max32(top)));
      const float al = __builtin_amdgcn_exp2f(r.m[t] - mn);
      r.m[t] = mn;
      r.l[t] *= al;
#pragma unroll
      for (int m = 0; m < 8; ++m) r.o[t][m] *= al;
    }
    const float off = lv + UP - r.m[t];
    if (far) r.l[t] = fmaf(far_sum(s[t], ck, off), rv, r.l[t]);
#pragma unroll
    for (int i = 0; i < 8; ++i) p[t].v[i] = (_Float16)__builtin_amdgcn_exp2f(fmaf(s[t][i >> 2][i & 3], ck, off));
    hold_order();
  }
#pragma unroll
  for (int m = 0; m < 8; m += 2) {
    const Op o0 = n0, o1 = n1;
    if (m < 6) { n0 = v(m + 2); n1 = v(m + 3); }
    hold_order();
#pragma unroll
    for (int t = 0; t < NT; ++t) r.o[t][m] = mma(o0, p[t], r.o[t][m]);
#pragma unroll
    for (int t = 0; t < NT; ++t) r.o[t][m + 1] = mma(o1, p[t], r.o[t][m + 1]);
    hold_order();
  }
  if (far) rv = 0.0f;
#pragma unroll
  for (int t = 0; t < NT; ++t) r.l[t] = fmaf(sum_of(p[t]), rv, r.l[t]);
}

// The bytes of V codes (a lane group's eight tokens of a block, u0 and u1) of tokens that are there: n0 of the first four,
// n1 of the others.  What lies behind the length can be a NaN's code.
__device__ __forceinline__ uint32_t live(uint32_t u, int n) { return n >= 4 ? u : n <= 0 ? 0u : u & ((1u << (8 * n)) - 1); }

// A block out of a lane's registers.
template <int NT, int CODE>
__device__ __forceinline__ void take_codes(Rows<NT>& r, const Block& f, bool edge, bool far, int t0, int len, int lane) {
  const int n0 = len - t0 - 4 * (lane >> 4), n1 = n0 - 16;
  take_block<NT>(
      r, [&](int tt, int j) {
        const u32x4 w = f.k[2 * tt + (j >> 1)];
        return decode8<CODE>(w[2 * (j & 1)], w[2 * (j & 1) + 1]);
      },
      [&](int m) {
        uint32_t u0 = f.v[m >> 1][2 * (m & 1)], u1 = f.v[m >> 1][2 * (m & 1) + 1];
        if (CODE == 1 && edge) { u0 = live(u0, n0); u1 = live(u1, n1); }
        return decode8<CODE>(u0, u1);
      },
      f.km, f.vm, edge, far, t0, lane);
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

// W waves share out the blocks of a split, for up to 16 NT rows a KV head.  Bound by HBM, 256 bytes a token and KV head (int8,
// 28 heads over 196000 tokens, 4 KV heads: 37 us, 5.4 TB/s, and 4 the merge); a wave holds a block and asks for the next, 16 KB.  For
// short sequences by its chain of round trips: arguments, length, codes (one head of 1568 tokens 4.3 us, merge 2.2).
// grid (splits, H, B).
template <int NT, int CODE, int W>
__global__ __launch_bounds__(64 * W, W > 4 ? W / 4 : NT < 3 ? 2 : 1) void c8_few_kernel(C8Attn a) {
  const int b = blockIdx.z, h = blockIdx.y, sp = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, kb = lane >> 4;
  const int len = min(max(a.length[b], 0), a.cap);
  const int nq = a.q_count ? min(max(a.q_count[b], 0), a.n) : a.n;
  const int rows = a.n * a.rep;
  const int nb = (len + G - 1) / G, units = W * a.splits, un = W * sp + w;
  const int b0 = (int)((long long)un * nb / units), b1 = (int)((long long)(un + 1) * nb / units);
  const int all = a.causal ? max(len - nq + 1, 0) : len;          // tokens that every row sees
  const size_t head = ((size_t)b * a.H + h) * a.nbc;
  Rows<NT> r;
  Block f, g;
  if (b0 < b1) load_block(f, a.kc, a.vc, a.km, a.vm, head + b0, lane);      // (on its way while the queries are laid out)
  load_rows<NT>(r, a, b, h, 0, rows, len, nq, lane);
  if (b0 < b1) {
    uint32_t vmost = 0;                    // the largest magnitude so far
    for (int i = b0; i < b1; ++i) {
      if (i + 1 < b1) load_block(g, a.kc, a.vc, a.km, a.vm, head + i + 1, lane);
      const uint32_t kb = held_bits(f.km), vb = held_bits(f.vm);
      f.km = __uint_as_float(kb);
      f.vm = __uint_as_float(vb);
      vmost = max(vmost, vb);
      take_codes<NT, CODE>(r, f, (i + 1) * G > all, vb + FAR < vmost, i * G, len, lane);
      f = g;
    }
  }
  // the waves' sums, a tile of rows at a time
  __shared__ f4 so[W][16][D / 4 + 1];
  __shared__ float sm[W][16], sl[W][16];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const f2 ml = row_stats(r, t);
    if (t > 0) __syncthreads();
    if (kb == 0) { sm[w][x] = ml[0]; sl[w][x] = ml[1]; }
#pragma unroll
    for (int m = 0; m < 8; ++m) so[w][x][4 * m + kb] = r.o[t][m];
    __syncthreads();
#pragma unroll
    for (int e = tid; e < 16 * (D / 4); e += 64 * W) {
      const int rr = e / (D / 4), c4 = e % (D / 4), row = 16 * t + rr;
      if (row >= rows) continue;
      float M = NONE;
#pragma unroll
      for (int k = 0; k < W; ++k) M = fmaxf(M, sm[k][rr]);
      f4 o = f4{0.f, 0.f, 0.f, 0.f};
      float l = 0.0f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float wt = __builtin_amdgcn_exp2f(sm[k][rr] - M);
        o += so[k][rr][c4] * wt;
        l = fmaf(sl[k][rr], wt, l);
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
}

// Waves share out the rows: 16 NT a wave, 64 NT a workgroup, which walks the split's blocks together.  Each wave
// decodes a quarter of a block into LDS, where all four read it as operands, in their order, 16 bytes a lane.  The vector
// units are the bound, not the matrix cores: a 16 x 16 x 32 product keeps them from issuing for 8 of its 16 cycles, and a
// block costs a wave some 170 instructions of 4.6 cycles beside 51 products (a score: one multiply-add, an exponential of
// 8.6 cycles, half a conversion, half a maximum; the decoding: 40).  So: the more rows a wave, the fewer decodings and LDS
// reads a row - 48 rows are what 256 registers hold, two waves a SIMD (32 rows, three waves: 410 us where 48 took 352) -
// the weights of a block are made between the products of the block before, the decoding between those of the scores, and
// the denominators are products with ones.  196 queries x 28 heads over 98196 tokens, int8: 266 us, 1.04 PFLOP/s (1.16 with
// the rows that pad the last tile); 6272 over themselves, causal: 270 us, 1.04.  On the way there: each wave decoding for
// itself from memory 902 and 750; the weights in a phase of their own 340 and 350; eight waves to a workgroup, half the
// decoding each: the same.  32 x 32 x 16 products, which cost the vector units less, with 32 rows a wave: 460 and 355.
// grid (tiles of rows x splits x B x H), heads fastest: the tiles that see most come first, and what shares a head's
// codes runs at the same time, where the heads divide the eight dies' turns on the same die.
template <int NT, int CODE>
__global__ __launch_bounds__(256, 2) void c8_many_kernel(C8Attn a, int tiles) {
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, kb = lane >> 4;
  int at = blockIdx.x;
  const int h = at % a.H; at /= a.H;
  const int b = at % a.B; at /= a.B;
  const int sp = at % a.splits, tile = tiles - 1 - at / a.splits;
  const int len = min(max(a.length[b], 0), a.cap);
  const int nq = a.q_count ? min(max(a.q_count[b], 0), a.n) : a.n;
  const int rows = a.n * a.rep, tile0 = tile * 64 * NT, row0 = tile0 + w * 16 * NT;
  // tokens that the first row from `row` on sees, and those that the last of `n` rows does
  auto least = [&](int row) { return row / a.rep >= nq ? 0 : a.causal ? max(len - nq + row / a.rep + 1, 0) : len; };
  auto most = [&](int row, int n) {
    const int i1 = min((row + n - 1) / a.rep, nq - 1);
    return i1 < row / a.rep ? 0 : a.causal ? max(len - nq + i1 + 1, 0) : len;
  };
  const int all = least(row0), nb = (most(tile0, 64 * NT) + G - 1) / G;
  const int b0 = (int)((long long)sp * nb / a.splits), b1 = (int)((long long)(sp + 1) * nb / a.splits);
  const size_t head = ((size_t)b * a.H + h) * a.nbc;
  __shared__ Op ops[2][16][64];            // 0..7: K, tile of tokens tt, channels j at 4 tt + j; 8..15: V, tile of channels
  // this wave's quarter: K piece w (tt = w >> 1, j = 2 (w & 1) and the next), V piece w (m = 2 w and the next)
  const uint8_t* kc = a.kc + head * C8REC + ((w >> 1) * 16 + x) * D + (w & 1) * 64 + kb * 16;
  const uint8_t* vc = a.vc + head * C8REC + w * 1024 + lane * 16;
  u32x4 gk, gv;                            // codes on their way to LDS
  float gkm, gvm;                          // magnitudes of the block in gk
  auto ask_k = [&](int i) {
    i = min(i, b1 - 1);
    gk = *reinterpret_cast<const u32x4*>(kc + (size_t)i * C8REC);
    gkm = a.km[head + i];
    gvm = a.vm[head + i];
  };
  auto ask_v = [&](int i) { gv = *reinterpret_cast<const u32x4*>(vc + (size_t)min(i, b1 - 1) * C8REC); };
  auto clear_dead = [&](int i) {           // tokens behind the length
    if (CODE == 1 && (i + 1) * G > len) {
      const int n0 = len - i * G - 4 * kb, n1 = n0 - 16;
      gv[0] = live(gv[0], n0); gv[1] = live(gv[1], n1);
      gv[2] = live(gv[2], n0); gv[3] = live(gv[3], n1);
    }
  };
  auto put_k = [&](int i, int e) { ops[i & 1][2 * w + e][lane] = decode8<CODE>(gk[2 * e], gk[2 * e + 1]); };
  auto put_v = [&](int i, int e) { ops[i & 1][8 + 2 * w + e][lane] = decode8<CODE>(gv[2 * e], gv[2 * e + 1]); };
  // LDS alone is handed over: what is still on its way from memory goes on
  auto hand_over = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  // the first two blocks' codes, on their way while the queries are laid out
  u32x4 gk0{};
  float km = 1.0f, vm = 1.0f;
  if (b0 < b1) {
    ask_k(b0);
    gk0 = gk; km = gkm; vm = gvm;
    ask_v(b0);
    ask_k(b0 + 1);
  }
  Rows<NT> r;
  load_rows<NT>(r, a, b, h, row0, rows, len, nq, lane);
  f4 s[NT][2];
  Op p[NT], n0, n1;
  float al[NT];
  // x of block i; between its products, what goes to LDS meanwhile: fill(0..3)
  auto scores = [&](int i, auto&& fill) {
    const Op(*o)[64] = ops[i & 1];
    n0 = o[0][lane];
    n1 = o[1][lane];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const Op o0 = n0, o1 = n1;
      if (g < 3) { n0 = o[2 * g + 2][lane]; n1 = o[2 * g + 3][lane]; }
      hold_order();
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t][g >> 1] = mma(o0, r.q[t][2 * (g & 1)], g & 1 ? s[t][g >> 1] : f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t][g >> 1] = mma(o1, r.q[t][2 * (g & 1) + 1], s[t][g >> 1]);
      fill(g);
#pragma unroll
      for (int t = 0; t < 2 * NT; ++t) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 2, 0);
      }
      hold_order();
    }
  };
  // the weights' sums over a block's tokens; rv is 0 where far_sums had it
  auto sums = [&](float rv) {
#pragma unroll
    for (int t = 0; t < NT; ++t) r.l[t] = fmaf(sum_of(p[t]), rv, r.l[t]);
  };
  // masks, and the maxima where they have to rise; true: o is to be multiplied by al
  auto maxima = [&](int i, float km, float lv) {
    const int t0 = i * G;
    if (t0 + G > all) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (t0 + slot_token(kb, k) >= r.limit[t]) s[t][k >> 2][k & 3] = -INFINITY;
    }
    float top[NT];
    bool rise = false;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float big = -INFINITY;
#pragma unroll
      for (int k = 0; k < 8; ++k) big = fmaxf(big, s[t][k >> 2][k & 3]);
      top[t] = fmaf(big, r.cq[t] * km, lv);
      rise = rise || top[t] > r.m[t] + RISE;
    }
    rise = __any(rise);
    if (rise) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float mn = fmaxf(r.m[t], max16(max32(top[t])));
        al[t] = __builtin_amdgcn_exp2f(r.m[t] - mn);
        r.m[t] = mn;
        r.l[t] *= al[t];
      }
    }
    return rise;
  };
  // one score of the block as a weight
  float e0, ck[NT], off[NT];
  Op pn[NT];
  auto weight = [&](int t, int k) {
    const float e = __builtin_amdgcn_exp2f(fmaf(s[t][k >> 2][k & 3], ck[t], off[t]));
    if (k & 1) pn[t].p[k >> 1] = h2{(_Float16)e0, (_Float16)e};
    else e0 = e;
  };
  auto factors = [&](float km, float lv) {
#pragma unroll
    for (int t = 0; t < NT; ++t) { ck[t] = r.cq[t] * km; off[t] = lv + UP - r.m[t]; }
  };
  auto far_sums = [&](float rv) {
#pragma unroll
    for (int t = 0; t < NT; ++t) r.l[t] = fmaf(far_sum(s[t], ck[t], off[t]), rv, r.l[t]);
  };
  if (b0 < b1) {
    clear_dead(b0);
    put_v(b0, 0); put_v(b0, 1);
    put_k(b0 + 1, 0); put_k(b0 + 1, 1);
    uint32_t kn = held_bits(gkm), vn = held_bits(gvm);          // of the next block
    gk = gk0;
    put_k(b0, 0); put_k(b0, 1);
    ask_k(b0 + 2);
    ask_v(b0 + 1);
    hand_over();
    scores(b0, [](int) {});
    km = __uint_as_float(held_bits(km));
    vm = __uint_as_float(held_bits(vm));
    float lv = __log2f(vm);
    maxima(b0, km, lv);
    factors(km, lv);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int k = 0; k < 8; ++k) weight(t, k);
      p[t] = pn[t];
    }
    float rv = __builtin_amdgcn_rcpf(vm);
    uint32_t vmost = __float_as_uint(vm);  // the largest magnitude so far
    hand_over();
    // the weights of block i are there; block i + 1 is scored, and turned into weights between the products of block i
    for (int i = b0; i + 1 < b1; ++i) {
      // (of two waves on a SIMD the older one issues first, and its workgroup was done in two thirds of the younger's time;
      // turns of a block each: 322 -> 311 us)
      if ((i ^ (blockIdx.x >> 8)) & 1) __builtin_amdgcn_s_setprio(1);
      else __builtin_amdgcn_s_setprio(0);
      km = __uint_as_float(kn); vm = __uint_as_float(vn);
      const uint32_t vb = vn;
      kn = held_bits(gkm); vn = held_bits(gvm);
      clear_dead(i + 1);
      scores(i + 1, [&](int g) {
        if (g < 2) put_k(i + 2, g);
        else put_v(i + 1, g - 2);
      });
      ask_k(i + 3);
      ask_v(i + 2);
      sums(rv);
      rv = __builtin_amdgcn_rcpf(vm);
      lv = __log2f(vm);
      const bool rise = maxima(i + 1, km, lv);
      factors(km, lv);
      vmost = max(vmost, vb);
      if (vb + FAR < vmost) {
        far_sums(rv);
        rv = 0.0f;
      }
      const Op(*o)[64] = ops[i & 1] + 8;
      n0 = o[0][lane];
      n1 = o[1][lane];
      hold_order();
#pragma unroll
      for (int m = 0; m < 8; m += 2) {
        const Op o0 = n0, o1 = n1;
        if (m < 6) { n0 = o[m + 2][lane]; n1 = o[m + 3][lane]; }
#pragma unroll
        for (int t = 0; t < 2 * NT; ++t) {
          const int at = m * NT + t;
          r.o[t % NT][m + t / NT] = mma(t < NT ? o0 : o1, p[t % NT], r.o[t % NT][m + t / NT]);
          weight(at >> 3, at & 7);
          hold_order();
        }
      }
      // (else the compiler moves all of this behind the branch)
#pragma unroll
      for (int t = 0; t < NT; ++t) asm volatile("" : "+v"(pn[t].q));
#pragma unroll
      for (int t = 0; t < NT; ++t) p[t] = pn[t];
      if (rise) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int m = 0; m < 8; ++m) r.o[t][m] *= al[t];
      }
      hand_over();
    }
    sums(rv);
    const Op(*o)[64] = ops[(b1 - 1) & 1] + 8;
#pragma unroll
    for (int m = 0; m < 8; ++m) {
      const Op v = o[m][lane];
#pragma unroll
      for (int t = 0; t < NT; ++t) r.o[t][m] = mma(v, p[t], r.o[t][m]);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + 16 * t + x;
    const f2 ml = row_stats(r, t);
    if (row >= rows) continue;
    if (a.po) {
      const size_t at = (((size_t)b * a.H + h) * rows + row) * a.splits + sp;
#pragma unroll
      for (int m = 0; m < 8; ++m) reinterpret_cast<f4*>(a.po)[at * (D / 4) + 4 * m + kb] = r.o[t][m];
      if (kb == 0) { a.pml[2 * at] = ml[0]; a.pml[2 * at + 1] = ml[1]; }
    } else {
      const float l = ml[1], f = l != 0.0f ? a.inv_level / l : 0.0f;
#pragma unroll
      for (int m = 0; m < 8; ++m) put_out(a, b, h, row, 16 * m + 4 * kb, l != 0.0f ? r.o[t][m] * f : f4{0.f, 0.f, 0.f, 0.f});
    }
  }
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

// How a call is shared out.
struct C8Plan {
  int nt;                      // row tiles of 16 a wave
  bool few;                    // waves share blocks (all rows fit one wave), else rows
  int waves;                   // few: a workgroup's
  int tiles, splits;
  int most;                    // rows shared out: the splits that there can be
};

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
static C8Plan c8_plan(const C8Geom& g, int n) {
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
static size_t c8_parts(const C8Geom& g, long long rows, int splits) {
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
  a.B = g.B; a.H = g.H; a.rep = g.rep; a.n = n; a.cap = g.cap; a.nbc = g.nbc; a.splits = p.splits; a.causal = causal;
  a.bf16 = q->dtype == VIDKV_BF16;
  const float level = g.code == 0 ? 127.0f : 448.0f;
  a.scale2 = scale * 1.4426950408889634f / level;
  a.inv_level = 1.0f / level;
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
  if (a.po) {
    const int rows = n * g.rep;
    auto merge = [&](auto sl) {
      constexpr int SL = decltype(sl)::value;
      hipLaunchKernelGGL(c8_merge_kernel<SL>, dim3((rows + 8 / SL - 1) / (8 / SL), g.H, g.B), blk, 0, st, a);
    };
    if (p.splits > 32) merge(std::integral_constant<int, 8>{});
    else if (p.splits > 16) merge(std::integral_constant<int, 4>{});
    else if (p.splits > 8) merge(std::integral_constant<int, 2>{});
    else merge(std::integral_constant<int, 1>{});
  }
  return hipGetLastError();
}

}  // namespace vidkv
