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
#pragma once

#include "cache8.h"
#include <type_traits>

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

// ---- drafted tokens ---------------------------------------------------------------------------
// Behind the cached tokens a row can see drafted ones, whose keys and values are given beside the cache in 16 bits: blocks
// of 32 of them, of the magnitude `level`, so that their elements are in the codes' units as they are.
static_assert(sizeof(C8Attn) % 8 == 0 && alignof(C8Attn) == 8, "Tree::argument()");

struct NoTree {
  static constexpr bool ON = false;
};
template <class T>
struct Tree {
  static constexpr bool ON = true;
  typedef T Type;
  // A kernel's second argument, read where it is asked for: held over the cached tokens it costs the scalar registers that their
  // loop goes by (48 rows, 16 sequences of up to 6001 tokens: 29.4 us and 35 registers spilled, so 27.1).  Arguments lie behind each other.
  static __device__ __forceinline__ Tree argument() {
    typedef const __attribute__((address_space(4))) char* Args;
    Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const Tree*)(const char*)(p + sizeof(C8Attn));
  }
  View K, V;                   // [B][H][n][128]
  const uint32_t* mask;        // [B][n][words]: bit j % 32 of word j / 32: the node sees node j
  int words;
};

// ... and the first one, for what is left to do behind the blocks.  (Held over them it cost the mixed kernels 34 to 47 spilled scalars, now
// 8 to 12, and two of them a private segment; the times are the same.)
template <class TREE>
__device__ __forceinline__ C8Attn arguments(const C8Attn& a) {
  if constexpr (!TREE::ON) return a;
  typedef const __attribute__((address_space(4))) char* Args;
  Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const C8Attn*)(const char*)p;
}

// Nodes t0 .. t0 + 31 that a lane's rows see, as bits, of `nq` that there are.
template <int NT, class T>
__device__ __forceinline__ void load_sees(uint32_t (&sees)[NT], const Tree<T>& tree, const C8Attn& a, int b, int row0, int rows, int nq,
                                          int blk, int lane) {
  const uint32_t there = nq - blk * G >= G ? ~0u : (1u << (nq - blk * G)) - 1;
  asm volatile("" : "+s"(row0));           // (the rows' nodes are divided out again: not kept over the cached tokens)
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + 16 * t + (lane & 15), i = row / a.rep;
    sees[t] = row < rows && i < nq ? tree.mask[((size_t)b * a.n + i) * tree.words + blk] & there : 0;
  }
}

// 16 bytes of key `token`, a lane's operand of a tile's channels 32 j ..; eight values of two channels, those of lane group g.
// (Behind the last of nq nodes the last one is read, and taken as zeros.)
template <class T>
__device__ __forceinline__ u32x4 tree_key(const char* K, long long st, int token, int j, int nq, int kb) {
  const u32x4 k = *reinterpret_cast<const u32x4*>(K + min(token, nq - 1) * st + 2 * ((j >> 1) * 64 + kb * 16 + (j & 1) * 8));
  return token < nq ? k : u32x4{0, 0, 0, 0};
}
template <class T>
__device__ __forceinline__ void tree_values(uint32_t (&v)[8], const char* V, long long st, int t0, int g, int nq, int lane) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = t0 + slot_token(g, j);
    v[j] = *reinterpret_cast<const uint32_t*>(V + min(t, nq - 1) * st + 4 * lane);
    if (t >= nq) v[j] = 0;
  }
}

// Whether an element is beyond what a block of the cache holds (an infinity, a NaN): it is taken as the cache takes it.
template <class T, int N>
__device__ __forceinline__ us2 most_of(us2 m, const uint32_t (&u)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, u[i] & 0x7fff7fffu));
  return m;
}
template <class T>
__device__ __forceinline__ bool beyond(us2 m) { return __any(max(m[0], m[1]) > T::TOP); }

// The two channels' values as operands of their tiles of channels, at their places among `ops` [8][64].
__device__ __forceinline__ void put_values(u32x4* ops, const uint32_t (&v)[8], int g, int lane) {
  u32x4 lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x05040100u);
    hi[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x07060302u);
  }
  u32x4* at = ops + (lane >> 3) * 64 + 16 * g + 2 * (lane & 7);
  at[0] = lo;
  at[1] = hi;
}

// A block of drafted tokens into the running sums; k(tt, j), v(m): its operands, of type T.  bf16 queries are exact in bf16 again (what
// their fp16 form has dropped apart); weights of bf16 values are two bf16 numbers, 16 bits of any size, so none vanishes.
template <class T, int CODE, int NT, class K, class V>
__device__ __forceinline__ void take_tree(Rows<NT>& r, const K& k, const V& v, const uint32_t (&sees)[NT], bool far, int lane) {
  constexpr bool BF = std::is_same<T, TBF16>::value;
  constexpr float level = kLevel<CODE>, lv = CODE == 0 ? 6.98868468677217f : 8.80735492205760f;      // log2 of it
  auto mul = [](const Op& x, const Op& y, f4 c) { return BF ? mma_bf16(x, y, c) : mma(x, y, c); };
  const int kb = lane >> 4;
  f4 s[NT][2];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const Op k0 = k(0, j), k1 = k(1, j);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      Op q = r.q[t][j];
      if (BF) q.q = TBF16::pack8(__builtin_convertvector(q.v, f8v));
      s[t][0] = mul(k0, q, j ? s[t][0] : f4{0.f, 0.f, 0.f, 0.f});
      s[t][1] = mul(k1, q, j ? s[t][1] : f4{0.f, 0.f, 0.f, 0.f});
    }
    hold_order();
  }
  Op p[NT], lo[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float ck = r.cq[t] * level;
    const uint32_t w = sees[t] >> (4 * kb);
    float big = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (!(w >> (i < 4 ? i : 12 + i) & 1)) s[t][i >> 2][i & 3] = -INFINITY;
      big = fmaxf(big, s[t][i >> 2][i & 3]);
    }
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
    if (!BF && far) r.l[t] = fmaf(far_sum(s[t], ck, off), 1.0f / level, r.l[t]);
    if constexpr (BF) {
      f8v e, rest;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = __builtin_amdgcn_exp2f(fmaf(s[t][i >> 2][i & 3], ck, off));
        rest[i] = e[i] - (float)(__bf16)e[i];
      }
      p[t].q = TBF16::pack8(e);
      lo[t].q = TBF16::pack8(rest);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[t].v[i] = (_Float16)__builtin_amdgcn_exp2f(fmaf(s[t][i >> 2][i & 3], ck, off));
    }
    hold_order();
  }
#pragma unroll
  for (int m = 0; m < 8; ++m) {
    const Op o = v(m);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      r.o[t][m] = mul(o, p[t], r.o[t][m]);
      if (BF) r.o[t][m] = mul(o, lo[t], r.o[t][m]);
    }
    hold_order();
  }
  Op ones;
#pragma unroll
  for (int i = 0; i < 4; ++i) ones.u[i] = BF ? 0x3f803f80u : 0x3c003c00u;
  const float rv = !BF && far ? 0.0f : 1.0f / level;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    f4 l = mul(ones, p[t], f4{0.f, 0.f, 0.f, 0.f});
    if (BF) l = mul(ones, lo[t], l);
    r.l[t] = fmaf(l[0], rv, r.l[t]);
  }
}

// One such block by a wave for itself: operands through LDS, 8 KB each of its own (keys [8][64], values [8][64]).  TIGHT: keys are asked
// for when the values' registers are free again.
template <class T, bool TIGHT, int NT>
struct TreeBlock {
  u32x4 k[8];
  uint32_t v[4][8], sees[NT];
  const char* K;
  long long k_stride;
  int blk, nq;

  __device__ __forceinline__ void ask_keys(int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = tree_key<T>(K, k_stride, blk * G + 16 * (i >> 2) + (lane & 15), i & 3, nq, lane >> 4);
  }
  __device__ __forceinline__ void ask(const C8Attn& a, int b, int h, int rows, int nodes, int block, int lane) {
    const Tree<T> tree = Tree<T>::argument();
    blk = block;
    nq = nodes;
    asm volatile("" : "+s"(b), "+s"(h));                 // (addresses are made again at every block: not kept over the cached tokens)
    K = tree.K.data + b * tree.K.sb + h * tree.K.sh;
    k_stride = tree.K.st;
    const char* V = tree.V.data + b * tree.V.sb + h * tree.V.sh;
    load_sees(sees, tree, a, b, 0, rows, nq, blk, lane);
    if (!TIGHT) ask_keys(lane);
#pragma unroll
    for (int g = 0; g < 4; ++g) tree_values<T>(v[g], V, tree.V.st, blk * G, g, nq, lane);
  }
  __device__ __forceinline__ void put(u32x4* keys, u32x4* values, int lane) {
    us2 m{0, 0};
#pragma unroll
    for (int g = 0; g < 4; ++g) m = most_of<T>(m, v[g]);
    if (beyond<T>(m)) {
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i >> 3][i & 7] = held<T>(v[i >> 3][i & 7]);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) put_values(values, v[g], g, lane);
    if (TIGHT) {
      hold_order();
      ask_keys(lane);
    }
    m = us2{0, 0};
#pragma unroll
    for (int i = 0; i < 32; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, k[i >> 2][i & 3] & 0x7fff7fffu));
    if (beyond<T>(m)) {
#pragma unroll
      for (int i = 0; i < 32; ++i) k[i >> 2][i & 3] = held<T>(k[i >> 2][i & 3]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) keys[i * 64 + lane] = k[i];
  }
};

// W waves share out the blocks of a split, for up to 16 NT rows a KV head.  Bound by HBM, 256 bytes a token and KV head (int8,
// 28 heads over 196000 tokens, 4 KV heads: 37 us, 5.4 TB/s, and 4 the merge); a wave holds a block and asks for the next, 16 KB.  For
// short sequences by its chain of round trips: arguments, length, codes (one head of 1568 tokens 4.3 us, merge 2.2).
// grid (splits, H, B).
template <int NT, int CODE, int W, class TREE>
__device__ __forceinline__ void few_rows(const C8Attn a) {
  const int b = blockIdx.z, h = blockIdx.y, sp = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, kb = lane >> 4;
  const int len = min(max(a.length[b], 0), a.cap);
  const int nq = a.q_count ? min(max(a.q_count[b], 0), a.n) : a.n;
  const int rows = a.n * a.rep;
  const int nb = TREE::ON && nq == 0 ? 0 : (len + G - 1) / G, units = W * a.splits, un = W * sp + w;
  const int blocks = nb + (TREE::ON ? (nq + G - 1) / G : 0);      // cached ones, then drafted ones
  const int b0 = (int)((long long)un * blocks / units), end = (int)((long long)(un + 1) * blocks / units);
  const int b1 = TREE::ON ? min(end, nb) : end;
  const int all = a.causal ? max(len - nq + 1, 0) : len;          // tokens that every row sees
  const size_t head = ((size_t)b * a.H + h) * a.nbc;
  Rows<NT> r;
  Block f, g;
  __shared__ f4 so[W][16][D / 4 + 1];
  if (b0 < b1) load_block(f, a.kc, a.vc, a.km, a.vm, head + b0, lane);      // (on its way while the queries are laid out)
  // A drafted block, the wave's last work, is asked for now too and waits in LDS (48 rows of 16 sequences of
  // up to 6001 tokens 26 us; asked for at its turn 27.7).  NT tiles have at most two; a workgroup's second buffer is for the one that is not the last.
  constexpr int BUFS = TREE::ON ? NT == 1 ? 1 : 2 : 0;
  __shared__ u32x4 tree_keys[BUFS ? BUFS : 1][BUFS ? 512 : 1];
  auto tree_block = [&] {
    if constexpr (TREE::ON) return TreeBlock<typename TREE::Type, (W > 4), NT>{};
    else return 0;
  }();
  const int first = max(b0, nb), buf = BUFS == 2 && first + 1 < blocks ? 1 : 0;
  if constexpr (TREE::ON) {
    if (first < end) tree_block.ask(a, b, h, rows, nq, first - nb, lane);
  }
  load_rows<NT>(r, a, b, h, 0, rows, TREE::ON ? max(len, 1) : len, nq, lane);
  if constexpr (TREE::ON) {
    if (first < end) tree_block.put(tree_keys[buf], reinterpret_cast<u32x4*>(so[w]), lane);
  }
  uint32_t vmost = 0;                      // the largest magnitude so far
  if (b0 < b1) {
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
  if constexpr (TREE::ON) {
    const u32x4* keys = tree_keys[buf];
    const u32x4* values = reinterpret_cast<const u32x4*>(so[w]);
#pragma unroll 1
    for (int i = first; i < end; ++i) {
      if (i > first) {
        tree_block.ask(a, b, h, rows, nq, i - nb, lane);
        tree_block.put(tree_keys[buf], reinterpret_cast<u32x4*>(so[w]), lane);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      auto op = [&](const u32x4* at) {
        Op o;
        o.q = at[lane];
        return o;
      };
      take_tree<typename TREE::Type, CODE>(
          r, [&](int tt, int j) { return op(keys + (4 * tt + j) * 64); }, [&](int c) { return op(values + c * 64); }, tree_block.sees,
          __float_as_uint(kLevel<CODE>) + FAR < vmost, lane);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
  // the waves' sums, a tile of rows at a time
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
struct ManySpan {
  int b, h, tile0;             // the workgroup's first row
  int sp, splits;              // of the splits of its rows (the partials have a.splits)
};
// EARLY: a tree's first block waits here.  NT: the most tiles a wave.
template <class TREE, bool EARLY, int NT>
struct ManyLds {
  Op ops[2][16][64];           // 0..7: K, tile of tokens tt, channels j at 4 tt + j; 8..15: V, tile of channels
  // (arrays of nothing where they are not used)
  Op tree_ops[EARLY ? 16 : 0][64];
  uint32_t tree_sees[TREE::ON ? 2 : 0][4][NT][16];
};
template <int NT, int CODE, class TREE, class LDS>
__device__ __forceinline__ void many_rows(const C8Attn a, const ManySpan span, LDS& lds) {
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, kb = lane >> 4;
  const int b = span.b, h = span.h, sp = span.sp;
  const int len = min(max(a.length[b], 0), a.cap);
  const int nq = a.q_count ? min(max(a.q_count[b], 0), a.n) : a.n;
  const int rows = a.n * a.rep, tile0 = span.tile0, row0 = tile0 + w * 16 * NT;
  // tokens that the first row from `row` on sees, and those that the last of `n` rows does
  auto least = [&](int row) { return row / a.rep >= nq ? 0 : a.causal ? max(len - nq + row / a.rep + 1, 0) : len; };
  auto most = [&](int row, int n) {
    const int i1 = min((row + n - 1) / a.rep, nq - 1);
    return i1 < row / a.rep ? 0 : a.causal ? max(len - nq + i1 + 1, 0) : len;
  };
  const int all = least(row0), nb = (most(tile0, 64 * NT) + G - 1) / G;
  const int blocks = nb + (TREE::ON && tile0 / a.rep < nq ? (nq + G - 1) / G : 0);      // cached ones, then drafted ones
  const int b0 = (int)((long long)sp * blocks / span.splits), end = (int)((long long)(sp + 1) * blocks / span.splits);
  const int b1 = TREE::ON ? min(end, nb) : end;
  const size_t head = ((size_t)b * a.H + h) * a.nbc;
  Op(&ops)[2][16][64] = lds.ops;
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
  // drafted tokens: each wave lays a quarter of a block out in LDS, keys as the codes above, values of lane group w.  The first
  // block is asked for now and waits there; the others are asked for a block ahead, when the cached tokens are done (and the
  // first too where three tiles a wave have no registers for it: 196000 tokens, 64 nodes 453 us with those spilled, 337 so).
  constexpr bool EARLY = TREE::ON && NT < 3;
  const int d0 = max(b0 - nb, 0), d1 = end - nb;
  auto& tree_ops = lds.tree_ops;
  auto& tree_sees = lds.tree_sees;
  u32x4 tk[2];
  uint32_t tv[8], ts[NT];
  auto ask_tree = [&](int i) {
    if constexpr (TREE::ON) {
      typedef typename TREE::Type T;
      const TREE tree = TREE::argument();
      int seq = b, head = h;
      asm volatile("" : "+s"(seq), "+s"(head));          // (addresses are made again at every block: not kept over the cached tokens)
      const char* K = tree.K.data + seq * tree.K.sb + head * tree.K.sh;
      const char* V = tree.V.data + seq * tree.V.sb + head * tree.V.sh;
#pragma unroll
      for (int e = 0; e < 2; ++e) tk[e] = tree_key<T>(K, tree.K.st, i * G + 16 * (w >> 1) + x, 2 * (w & 1) + e, nq, kb);
      tree_values<T>(tv, V, tree.V.st, i * G, w, nq, lane);
      load_sees(ts, tree, a, b, row0, rows, nq, i, lane);
    }
  };
  auto put_tree = [&](Op(*to)[64], int i) {
    if constexpr (TREE::ON) {
      typedef typename TREE::Type T;
      us2 m = most_of<T>(us2{0, 0}, tv);
#pragma unroll
      for (int e = 0; e < 8; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, tk[e >> 2][e & 3] & 0x7fff7fffu));
      if (beyond<T>(m)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { tv[e] = held<T>(tv[e]); tk[e >> 2][e & 3] = held<T>(tk[e >> 2][e & 3]); }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) to[2 * w + e][lane].q = tk[e];
      put_values(&to[8][0].q, tv, w, lane);
      if (kb == 0) {
#pragma unroll
        for (int t = 0; t < NT; ++t) tree_sees[i & 1][w][t][x] = ts[t];
      }
    }
  };
  if (EARLY && d0 < d1) ask_tree(d0);
  Rows<NT> r;
  load_rows<NT>(r, a, b, h, row0, rows, TREE::ON ? max(len, 1) : len, nq, lane);
  if (EARLY && d0 < d1) put_tree(tree_ops, d0);
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
  uint32_t vmost = 0;                      // the largest magnitude so far
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
    vmost = __float_as_uint(vm);
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
  if constexpr (TREE::ON) {
    if (!EARLY && d0 < d1) {
      ask_tree(d0);
      hand_over();                         // (the last cached block's operands have been read)
      put_tree(ops[d0 & 1], d0);
    }
#pragma unroll 1
    for (int i = d0; i < d1; ++i) {
      if (i + 1 < d1) ask_tree(i + 1);
      hand_over();
      const Op(*o)[64] = EARLY && i == d0 ? tree_ops : ops[i & 1];
      uint32_t sees[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) sees[t] = tree_sees[i & 1][w][t][x];
      take_tree<typename TREE::Type, CODE>(
          r, [&](int tt, int j) { return o[4 * tt + j][lane]; }, [&](int c) { return o[8 + c][lane]; }, sees,
          __float_as_uint(kLevel<CODE>) + FAR < vmost, lane);
      if (i + 1 < d1) put_tree(ops[(i + 1) & 1], i + 1);
    }
  }
  const C8Attn e = arguments<TREE>(a);
  const int all_rows = e.n * e.rep;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    int row = row0 + 16 * t + x;
    if (TREE::ON) asm volatile("" : "+v"(row));          // (as in load_sees)
    const f2 ml = row_stats(r, t);
    if (row >= all_rows) continue;
    if (e.po) {
      const size_t at = (((size_t)b * e.H + h) * all_rows + row) * e.splits + sp;
#pragma unroll
      for (int m = 0; m < 8; ++m) reinterpret_cast<f4*>(e.po)[at * (D / 4) + 4 * m + kb] = r.o[t][m];
      if (kb == 0) { e.pml[2 * at] = ml[0]; e.pml[2 * at + 1] = ml[1]; }
    } else {
      const float l = ml[1], f = l != 0.0f ? e.inv_level / l : 0.0f;
#pragma unroll
      for (int m = 0; m < 8; ++m) put_out(e, b, h, row, 16 * m + 4 * kb, l != 0.0f ? r.o[t][m] * f : f4{0.f, 0.f, 0.f, 0.f});
    }
  }
  if constexpr (TREE::ON) {
    // fewer splits than the partials have: one of nothing for each behind them
    if (e.po && sp + span.splits < e.splits) {
      for (int i = tid; i < 64 * NT * (D / 4); i += 256) {
        const int row = tile0 + i / (D / 4);
        if (row >= all_rows) break;
        const size_t at = (((size_t)b * e.H + h) * all_rows + row) * e.splits + sp + span.splits;
        reinterpret_cast<f4*>(e.po)[at * (D / 4) + i % (D / 4)] = f4{0.f, 0.f, 0.f, 0.f};
        if (i % (D / 4) == 0) { e.pml[2 * at] = NONE; e.pml[2 * at + 1] = 0.0f; }
      }
    }
  }
}

// How a call is shared out.
struct C8Plan {
  int nt;                      // row tiles of 16 a wave
  bool few;                    // waves share blocks (all rows fit one wave), else rows
  int waves;                   // few: a workgroup's
  int tiles, splits;
  int most;                    // rows shared out: the splits that there can be
};
// Workgroup `at` of tiles x splits x B x H, heads fastest: the tiles that see most come first, and what shares a head's codes runs at
// the same time, where the heads divide the eight dies' turns on the same die.
template <int NT>
__device__ __forceinline__ ManySpan even_span(const C8Attn& a, int at, int tiles) {
  const int h = at % a.H; at /= a.H;
  const int b = at % a.B; at /= a.B;
  const int sp = at % a.splits, tile = tiles - 1 - at / a.splits;
  return ManySpan{b, h, tile * 64 * NT, sp, a.splits};
}

C8Plan c8_plan(const C8Geom& g, int n);
size_t c8_parts(const C8Geom& g, long long rows, int splits);
size_t c8_attn_ws_bytes(const C8Geom& g, int n);
// Arguments of a call whose plan it is, and the merge of its splits behind it (cache8_attn.hip).
C8Attn c8_args(const C8Geom& g, const C8Plan& p, int layer, int n, int causal, float scale, const vidkv_view* q, const uint8_t* cache,
               const int32_t* length, const int32_t* q_count, const vidkv_view* out, void* ws);
void launch_c8_merge(const C8Attn& a, hipStream_t st);

}  // namespace vidkv
