// Shared definitions of the rotary positions and the 8-bit cache: views, types, codes, geometry.
//
// Cache buffer: [K codes][V codes][K magnitudes][V magnitudes], heads = L*B*H, C = capacity:
//   K codes  heads x C/32 records of 4096 bytes, [32 tokens][128 channels]
//   V codes  heads x C/32 records of 4096 bytes, [4 mp][4 kb][16 x][2 mh][8 slots]: channel
//            32 mp + 16 mh + x, slot j < 4: token 4 kb + j, else 16 + 4 kb + j - 4 - the order in
//            which a lane of the attention kernels needs them as an operand
//   magnitudes  float32 [heads][C/32]
// Every section starts on a 256-byte boundary.
#pragma once

#include "mfma_util.h"

namespace vidkv {

constexpr int C8REC = G * D;                       // bytes of one block's codes of K or of V
constexpr float C8_LEAST = 0x1p-40f, C8_MOST = 0x1p40f;   // bounds of a block's magnitude

struct C8Geom {
  int L, B, H, Hq, rep, cap, nbc;                  // nbc: blocks a head
  int code;
  size_t v_codes, k_mag, v_mag, total;             // offsets; K codes are at 0
};

inline bool make_c8(const vidkv_cache8* p, C8Geom* g) {
  if (!p) return false;
  if (p->n_layers < 1 || p->batch < 1 || p->n_kv_heads < 1 || p->batch > 65535 || p->n_kv_heads > 65535) return false;
  if (p->n_q_heads < p->n_kv_heads || p->n_q_heads % p->n_kv_heads) return false;
  if (p->head_dim != D || p->capacity < G || p->capacity % G || p->capacity > (1 << 28)) return false;
  if (p->code != 0 && p->code != 1) return false;
  g->L = p->n_layers; g->B = p->batch; g->H = p->n_kv_heads; g->Hq = p->n_q_heads;
  g->rep = g->Hq / g->H;
  g->cap = p->capacity; g->nbc = g->cap / G; g->code = p->code;
  // (in 128 bits: the layers, sequences, heads and tokens of a mistaken call can be more than 2^64 bytes)
  const unsigned __int128 blocks = (unsigned __int128)g->L * g->B * g->H * g->nbc;
  if (blocks > ((unsigned __int128)1 << 48)) return false;
  const size_t nb = (size_t)blocks, codes = nb * C8REC, mags = align256(nb * sizeof(float));
  g->v_codes = codes;
  g->k_mag = 2 * codes;
  g->v_mag = g->k_mag + mags;
  g->total = g->v_mag + mags;
  return true;
}

// A view as a kernel takes it.
struct View {
  char* data;
  long long sb, sh, st;                            // strides in bytes
};

inline int dtype_bytes(int t) { return t == VIDKV_F32 ? 4 : 2; }

inline View make_view(const vidkv_view* v) {
  View r{nullptr, 0, 0, 0};
  if (v) {
    const long long e = dtype_bytes(v->dtype);
    r = View{static_cast<char*>(v->data), v->stride_batch * e, v->stride_head * e, v->stride_token * e};
  }
  return r;
}

// Rotation as a kernel argument; turn and axis as in vidkv_rotary.
struct Rot {
  uint64_t turn[VIDKV_ROTARY_PAIRS];
  uint8_t axis[VIDKV_ROTARY_PAIRS];
  const int32_t* pos;                              // [n_axes][B * n]; nullptr: no rotation
  long long rows;                                  // B * n
  int head_dim, rot_dim, adjacent;
};

inline Rot make_rot(const vidkv_rotary* r, const int32_t* pos, long long rows) {
  Rot o{};
  o.rows = rows;
  if (!r) return o;
  for (int i = 0; i < VIDKV_ROTARY_PAIRS; ++i) { o.turn[i] = r->turn[i]; o.axis[i] = r->axis[i]; }
  o.pos = pos;
  o.head_dim = r->head_dim; o.rot_dim = r->rot_dim; o.adjacent = r->adjacent;
  return o;
}

// ---- element types --------------------------------------------------------------------------
typedef float f8v __attribute__((ext_vector_type(8)));

// (Run: 16 bytes as they lie in memory, Run2: two elements)
struct TF16 {
  static constexpr int BYTES = 2;
  typedef h8 Run;
  static __device__ __forceinline__ Run load(const void* p) { return *static_cast<const h8*>(p); }
  static __device__ __forceinline__ f8v widen(Run v) { return __builtin_convertvector(v, f8v); }
  static __device__ __forceinline__ void store(void* p, f8v v) { store8(p, v); }
  static __device__ __forceinline__ void store8(void* p, f8v v) { *static_cast<h8*>(p) = __builtin_convertvector(v, h8); }
  typedef uint32_t Run2;
  static __device__ __forceinline__ Run2 load2(const void* p) { return *static_cast<const uint32_t*>(p); }
  static __device__ __forceinline__ f2 widen2(uint32_t u) {
    const h2 v = bits_h2(u);
    return f2{(float)v[0], (float)v[1]};
  }
  static __device__ __forceinline__ void store2(void* p, float a, float b) {
    *static_cast<h2*>(p) = h2{(_Float16)a, (_Float16)b};
  }
  static __device__ __forceinline__ u32x4 pack8(f8v v) { return __builtin_bit_cast(u32x4, __builtin_convertvector(v, h8)); }
  static __device__ __forceinline__ float of_bits(uint32_t u) { return (float)__builtin_bit_cast(_Float16, (uint16_t)u); }
  // bits of infinity, and of the largest magnitude that goes into a block: the type's
  static constexpr uint16_t INF = 0x7c00, TOP = 0x7bff;
};

struct TBF16 {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  static constexpr int BYTES = 2;
  typedef u32x4 Run;
  static __device__ __forceinline__ Run load(const void* p) { return *static_cast<const u32x4*>(p); }
  static __device__ __forceinline__ void store(void* p, f8v v) { store8(p, v); }
  static __device__ __forceinline__ f8v widen(Run u) {
    f8v r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[2 * i] = __uint_as_float(u[i] << 16);
      r[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
    return r;
  }
  static __device__ __forceinline__ void store8(void* p, f8v v) { *static_cast<b8*>(p) = __builtin_convertvector(v, b8); }
  typedef uint32_t Run2;
  static __device__ __forceinline__ Run2 load2(const void* p) { return *static_cast<const uint32_t*>(p); }
  static __device__ __forceinline__ f2 widen2(uint32_t u) {
    return f2{__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)};
  }
  static __device__ __forceinline__ void store2(void* p, float a, float b) {
    *static_cast<b2*>(p) = b2{(__bf16)a, (__bf16)b};
  }
  static __device__ __forceinline__ u32x4 pack8(f8v v) { return __builtin_bit_cast(u32x4, __builtin_convertvector(v, b8)); }
  static __device__ __forceinline__ float of_bits(uint32_t u) { return __uint_as_float(u << 16); }
  static constexpr uint16_t INF = 0x7f80, TOP = 0x5380;        // (C8_MOST)
};

struct TF32 {
  static constexpr int BYTES = 4;
  typedef f4 Run;
  static __device__ __forceinline__ Run load(const void* p) { return *static_cast<const f4*>(p); }
  static __device__ __forceinline__ f4 widen(Run v) { return v; }
  static __device__ __forceinline__ void store(void* p, f4 v) { *static_cast<f4*>(p) = v; }
  static __device__ __forceinline__ void store8(void* p, f8v v) {
    static_cast<f4*>(p)[0] = f4{v[0], v[1], v[2], v[3]};
    static_cast<f4*>(p)[1] = f4{v[4], v[5], v[6], v[7]};
  }
  typedef f2 Run2;
  static __device__ __forceinline__ Run2 load2(const void* p) { return *static_cast<const f2*>(p); }
  static __device__ __forceinline__ f2 widen2(Run2 v) { return v; }
  static __device__ __forceinline__ void store2(void* p, float a, float b) { *static_cast<f2*>(p) = f2{a, b}; }
};

// ---- rotation -------------------------------------------------------------------------------
// cos and sin of 2 pi t / 2^64 for t = position * turn modulo 2^64: the nearest quarter turn is taken
// off exactly, the rest y, at most pi/4, goes through the two Taylor sums (behind them: y^11/11! = 1.8e-9,
// y^12/12! = 1.2e-10).  Its top 32 bits are taken, 2^-32 turns at most are cut off, and a float keeps 24 bits of them: 2^-28 turns
// at an eighth of a turn, less of smaller angles.
__device__ __forceinline__ void turn_cos_sin(int pos, uint64_t turn, float* c, float* s) {
  const uint64_t t = (uint64_t)(int64_t)pos * turn;
  const uint32_t q = (uint32_t)((t + (1ull << 61)) >> 62);
  const int32_t r = (int32_t)(uint32_t)((t - ((uint64_t)q << 62)) >> 32);
  const float y = (float)r * (6.283185307179586f * 0x1p-32f), z = y * y;
  float si = fmaf(z, 1.0f / 362880, -1.0f / 5040);
  si = fmaf(si, z, 1.0f / 120);
  si = fmaf(si, z, -1.0f / 6);
  si = fmaf(si * z, y, y);
  float co = fmaf(z, -1.0f / 3628800, 1.0f / 40320);
  co = fmaf(co, z, -1.0f / 720);
  co = fmaf(co, z, 1.0f / 24);
  co = fmaf(co, z, -0.5f);
  co = fmaf(co, z, 1.0f);
  const float a = (q & 1) ? si : co, b = (q & 1) ? co : si;      // |cos|, |sin| up to sign
  *c = (q == 1 || q == 2) ? -a : a;
  *s = (q & 2) ? -b : b;
}

// A pair turned; in one order of roundings, so that every kernel that turns it leaves the same bits.
__device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s) {
  const float x1 = a, x2 = b;
  a = fmaf(x1, c, -(x2 * s));
  b = fmaf(x2, c, x1 * s);
}

// Two runs of N elements, the two sides of N pairs; or, adjacent, N / 2 pairs each.
template <int N, class V>
__device__ __forceinline__ void turn_runs(V& x, V& y, bool adjacent, const float* co, const float* si) {
  if (adjacent) {
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      float a = x[2 * e], b = x[2 * e + 1], c = y[2 * e], d = y[2 * e + 1];
      turn_pair(a, b, co[e], si[e]);
      turn_pair(c, d, co[N / 2 + e], si[N / 2 + e]);
      x[2 * e] = a; x[2 * e + 1] = b; y[2 * e] = c; y[2 * e + 1] = d;
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float a = x[e], b = y[e];
      turn_pair(a, b, co[e], si[e]);
      x[e] = a; y[e] = b;
    }
  }
}

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

// Two elements held to the largest magnitude that goes into a block: an infinity is the type's largest number, a NaN a zero,
// so that no code is one (a weight of zero times it would be a NaN in rows that do not see its token).
template <class T>
__device__ __forceinline__ uint32_t held(uint32_t u) {
  const uint32_t a = u & 0x7fffu, b = u >> 16 & 0x7fffu, lo = a > T::INF ? 0 : min(a, (uint32_t)T::TOP),
                 hi = b > T::INF ? 0 : min(b, (uint32_t)T::TOP);
  return (u & 0x80008000u) | lo | hi << 16;
}

// ---- codes ----------------------------------------------------------------------------------
template <int CODE> constexpr float kLevel = CODE == 0 ? 127.0f : 448.0f;

// The code's units of x: x * up / A to the last bit, where x has at most 16 significant bits and A 11 (both
// of a 16-bit type, or x a code's value and A = its old magnitude): x * up is exact, the quotient's first guess is
// within two units in the last place, its remainder exact, and the corrected quotient the nearest float.  A quotient
// that lies on the border of two codes is a float, so it comes out exactly, and no other one is within 2^-20 of a border.
__device__ __forceinline__ float units(float x, float up, float A, float rA) {
  const float n = x * up, q = n * rA;
  return fmaf(fmaf(-q, A, n), rA, q);
}

// Four values in the code's units as four codes.  int8: 1.5 * 2^23 added, which rounds to an integer, ties to even, and leaves it in
// the low byte.
template <int CODE>
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
  if constexpr (CODE == 0) {
    constexpr float R = 12582912.0f;
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b + R), __float_as_uint(a + R), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d + R), __float_as_uint(c + R), 0x04000c0cu);
    return lo | hi;
  } else {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  }
}

// Four codes as fp16 pairs, exact.  int8: a code plus 128 in the low byte of 0x6400 is the fp16 number 1024 + it.
template <int CODE>
__device__ __forceinline__ void decode4(uint32_t u, h2* lo, h2* hi) {
  if constexpr (CODE == 0) {
    const uint32_t w = u ^ 0x80808080u;
    const h2 off = h2{(_Float16)-1152.0f, (_Float16)-1152.0f};
    *lo = bits_h2(__builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + off;
    *hi = bits_h2(__builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + off;
  } else {
    *lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.0f, false);
    *hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.0f, true);
  }
}

template <int CODE>
__device__ __forceinline__ Op decode8(uint32_t u0, uint32_t u1) {
  Op o;
  decode4<CODE>(u0, &o.p[0], &o.p[1]);
  decode4<CODE>(u1, &o.p[2], &o.p[3]);
  return o;
}

}  // namespace vidkv
