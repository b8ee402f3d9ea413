// Coding new tokens into the 8-bit cache's blocks: what the kernels that write it share.
#pragma once

#include "cache8.h"
#include <algorithm>

namespace vidkv {

struct C8Write {
  View K, V;
  int n;                       // new tokens a sequence, at most
  const int32_t* start;
  const int32_t* count;        // or nullptr
  uint8_t* kc;                 // this layer's codes and magnitudes
  uint8_t* vc;
  float* km;
  float* vm;
  int H, nbc, cap, n_axes;
  Rot rot;
};

// Two maxima over the wave at once, each of 16 bits.
template <int CTRL>
__device__ __forceinline__ us2 max_dpp(us2 v) {
  const int u = __builtin_bit_cast(int, v);
  return __builtin_elementwise_max(v, __builtin_bit_cast(us2, __builtin_amdgcn_update_dpp(u, u, CTRL, 0xf, 0xf, true)));
}
__device__ __forceinline__ us2 wave_max(us2 v) {
  v = max_dpp<0x128>(max_dpp<0x124>(max_dpp<0x122>(max_dpp<0x121>(v))));      // row_ror 1, 2, 4, 8: a row of sixteen
  // (the elements through integers of their own: a bit cast of a vector's element takes the first one)
  auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  uint32_t r0 = r[0], r1 = r[1];
  v = __builtin_elementwise_max(__builtin_bit_cast(us2, r0), __builtin_bit_cast(us2, r1));
  r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  r0 = r[0]; r1 = r[1];
  return __builtin_elementwise_max(__builtin_bit_cast(us2, r0), __builtin_bit_cast(us2, r1));
}

// A block's magnitude as it is stored: never zero, and bounded, as its elements are, so that no product of them leaves float's range.
__device__ __forceinline__ float bounded(float a) { return fminf(fmaxf(a, C8_LEAST), C8_MOST); }

constexpr int FEW = 8;                     // new tokens of a block whose sines are shared out

// Which rows of K and V the new tokens are.  In order: row i of sequence b is its new token i.
struct InOrder {
  static constexpr bool PICKED = false;
};
// Picked: the nodes of a path through a tree, token i is row path[b][i]; of every layer in one launch.
struct Path {
  static constexpr bool PICKED = true;
  const int32_t* path;                     // [B][n]
  int B;
  long long k_layer, v_layer;              // strides in bytes
};

// The lane eight further on in its row of sixteen.
__device__ __forceinline__ uint32_t lane_xor8(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true);      // row_ror:8
}

// One workgroup per block that new tokens reach.  K: thread = 16 channels of one token (two runs of eight, the two
// sides of eight pairs where the keys are turned); V: wave = lane group kb of the record, lane = two channels of its eight
// tokens, so that its codes are whole 8-byte pieces of the record, and two lanes' four pieces two whole 16-byte ones.
// What a workgroup waits for - rows, positions, a begun block's magnitudes and codes - is asked for as soon as its block
// is known.  8 x 4 heads x 12544 tokens in fp16: 67 us for 308 MB, 4.6 TB/s; the vector units are the second bound, 9
// instructions an element of which the exact quotient is 4 (with a branch a row, values in 8-byte stores at every second place
// and maxima in float32: 84 us).  One token of 64 sequences, turned: 5.5 us.  grid (blocks a sequence can reach, H, B).
// Here: block `nth` of those that `count` new tokens of sequence b reach from `start` on, if it is one of them; nodes: the tokens' rows, if
// they are picked.
template <class T, int CODE, bool ROT, class ROWS>
__device__ __forceinline__ void write_block(const C8Write& a, const ROWS& rows, int b, int h, int layer, int nth, int start, int count,
                                            const int* nodes) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (start < 0 || count <= 0) return;
  const long long first = (long long)(start / G + (long long)nth) * G;
  const long long end = (long long)start + count;
  if (first >= end || first >= a.cap) return;
  const char* kin = a.K.data + b * a.K.sb + h * a.K.sh;
  const char* vin = a.V.data + b * a.V.sb + h * a.V.sh;        // (row addresses are the wave's: scalar)
  int seq = b;                             // of the cache: a layer's sequences lie behind those of the layer before it
  if constexpr (ROWS::PICKED) {
    kin += layer * rows.k_layer;
    vin += layer * rows.v_layer;
    seq += layer * rows.B;
  }
  auto row_of = [&](int token) {
    if constexpr (ROWS::PICKED) return nodes[token];
    else return token;
  };
  const int t0 = (int)first;
  const int lo = max(start, t0), hi = (int)min(min(end, (long long)t0 + G), (long long)a.cap);
  const size_t blk = ((size_t)seq * a.H + h) * a.nbc + t0 / G;
  const bool begun = t0 < start;           // live tokens stand before the new ones
  const bool whole = lo == t0 && hi == t0 + G;
  constexpr float LV = kLevel<CODE>;

  // keys
  const int kt = t0 + (tid >> 3), u = tid & 7;
  const bool knew = kt >= lo && kt < hi;
  int c0 = 16 * u, c1 = c0 + 8;
  const bool turns = ROT && u < a.rot.rot_dim / 16;
  if (turns && !a.rot.adjacent) { c0 = 8 * u; c1 = c0 + a.rot.rot_dim / 2; }
  uint2* pk0 = reinterpret_cast<uint2*>(a.kc + blk * C8REC + (tid >> 3) * D + c0);
  uint2* pk1 = reinterpret_cast<uint2*>(a.kc + blk * C8REC + (tid >> 3) * D + c1);
  // values: this lane's 16 bytes of the record, channels cv and cv + 16 of lane group w
  const int cv = (lane >> 4) * 32 + 2 * (lane & 7) + ((lane >> 3) & 1);
  u32x4* pv = reinterpret_cast<u32x4*>(a.vc + blk * C8REC + (((lane >> 4) * 4 + w) * 16 + (cv & 15)) * 16);
  typename T::Run rx{}, ry{};
  if (knew) {
    const char* in = kin + (long long)row_of(kt - start) * a.K.st;
    rx = T::load(in + 2 * c0);
    ry = T::load(in + 2 * c1);
  }
  uint32_t v[8];                           // two channels of a token, as they lie in memory
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = t0 + slot_token(w, j);
    v[j] = 0;
    if (whole || (t >= lo && t < hi)) v[j] = *reinterpret_cast<const uint32_t*>(vin + (long long)row_of(t - start) * a.V.st + 4 * lane);
  }
  float ko = 0.0f, vo = 0.0f;
  uint2 k0{}, k1{};
  u32x4 vold{};
  if (begun) {
    ko = a.km[blk]; vo = a.vm[blk];
    if constexpr (!ROWS::PICKED) { k0 = *pk0; k1 = *pk1; }
  }
  if (!whole) vold = *pv;
  auto sines = [&](int token, int pair, float* co, float* si) {           // of new token `token` of the sequence
    const long long row = (long long)b * a.n + token;
    int pos[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) pos[i] = a.rot.pos[min(i, a.n_axes - 1) * a.rot.rows + row];
    const int ax = a.rot.axis[pair];
    turn_cos_sin(ax & 2 ? (ax & 1 ? pos[3] : pos[2]) : (ax & 1 ? pos[1] : pos[0]), a.rot.turn[pair], co, si);
  };
  f8v x, y;
  if constexpr (ROT) {
    // A token's sines are eight threads' work; those of few tokens are shared out to all (one token of 64 sequences: 5.7 -> 5.3 us)
    __shared__ f2 table[FEW][D / 2];
    const int pairs = a.rot.rot_dim / 2, fresh = hi - lo;
    float co[8], si[8];
    if (fresh <= FEW) {
      for (int i = tid; i < fresh * pairs; i += 256) {
        const int t = i / pairs, e = i - t * pairs;
        float c, s;
        sines(lo - start + t, e, &c, &s);
        table[t][e] = f2{c, s};
      }
      __syncthreads();
    }
    x = T::widen(rx); y = T::widen(ry);
    if (turns && knew) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (fresh <= FEW) {
          const f2 v = table[kt - lo][8 * u + e];
          co[e] = v[0]; si[e] = v[1];
        } else {
          sines(kt - start, 8 * u + e, &co[e], &si[e]);
        }
      }
      turn_runs<8>(x, y, a.rot.adjacent, co, si);
    }
  }
  ko = bounded(ko); vo = bounded(vo);

  u32x4 bx = __builtin_bit_cast(u32x4, rx), by = __builtin_bit_cast(u32x4, ry);
  if constexpr (ROT) { bx = T::pack8(x); by = T::pack8(y); }   // rounded to the tensor's type, as the rotation by itself leaves them
  // magnitudes of 16-bit numbers compare as integers do, two at a time
  __shared__ us2 red[4];
  auto largest = [&] {
    us2 vm{0, 0}, km{0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) vm = __builtin_elementwise_max(vm, __builtin_bit_cast(us2, v[j] & 0x7fff7fffu));
#pragma unroll
    for (int e = 0; e < 4; ++e)
      km = __builtin_elementwise_max(km, __builtin_elementwise_max(__builtin_bit_cast(us2, bx[e] & 0x7fff7fffu),
                                                                   __builtin_bit_cast(us2, by[e] & 0x7fff7fffu)));
    const us2 most = wave_max(us2{std::max(km[0], km[1]), std::max(vm[0], vm[1])});
    if (lane == 0) red[w] = most;
    __syncthreads();
    const us2 all = __builtin_elementwise_max(__builtin_elementwise_max(red[0], red[1]), __builtin_elementwise_max(red[2], red[3]));
    return __builtin_bit_cast(us2, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, all)));
  };
  us2 most = largest();
  if (max(most[0], most[1]) > T::TOP) {    // (the whole workgroup's: all of it comes here or none)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = held<T>(v[j]);
#pragma unroll
    for (int e = 0; e < 4; ++e) { bx[e] = held<T>(bx[e]); by[e] = held<T>(by[e]); }
    __syncthreads();                       // red has been read
    most = largest();
  }
  x = T::widen(__builtin_bit_cast(typename T::Run, bx));
  y = T::widen(__builtin_bit_cast(typename T::Run, by));
  float ka = bounded(T::of_bits(most[0])), va = bounded(T::of_bits(most[1]));
  if (begun) { ka = fmaxf(ka, ko); va = fmaxf(va, vo); }
  const float rk = __builtin_amdgcn_rcpf(ka), rv = __builtin_amdgcn_rcpf(va);
  if (tid == 0) { a.km[blk] = ka; a.vm[blk] = va; }

  // a live token's codes under the new magnitude
  auto again = [](uint32_t c, float old, float A, float rA) {
    h2 l, g;
    decode4<CODE>(c, &l, &g);
    return code4<CODE>(units((float)l[0], old, A, rA), units((float)l[1], old, A, rA), units((float)g[0], old, A, rA),
                       units((float)g[1], old, A, rA));
  };
  if (knew) {
    uint2 p, q;
    p.x = code4<CODE>(units(x[0], LV, ka, rk), units(x[1], LV, ka, rk), units(x[2], LV, ka, rk), units(x[3], LV, ka, rk));
    p.y = code4<CODE>(units(x[4], LV, ka, rk), units(x[5], LV, ka, rk), units(x[6], LV, ka, rk), units(x[7], LV, ka, rk));
    q.x = code4<CODE>(units(y[0], LV, ka, rk), units(y[1], LV, ka, rk), units(y[2], LV, ka, rk), units(y[3], LV, ka, rk));
    q.y = code4<CODE>(units(y[4], LV, ka, rk), units(y[5], LV, ka, rk), units(y[6], LV, ka, rk), units(y[7], LV, ka, rk));
    *pk0 = p;
    *pk1 = q;
  } else if (kt < start && ka > ko) {      // (only in a begun block)
    if constexpr (ROWS::PICKED) { k0 = *pk0; k1 = *pk1; }
    *pk0 = uint2{again(k0.x, ko, ka, rk), again(k0.y, ko, ka, rk)};
    *pk1 = uint2{again(k1.x, ko, ka, rk), again(k1.y, ko, ka, rk)};
  }

  // the codes of channels 2 lane and 2 lane + 1; channel and channel + 16 go into one piece: lanes 0..7 of a row of 16 take
  // the even channels of both, lanes 8..15 the odd ones
  uint2 n[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = units(T::widen2(v[j])[i], LV, va, rv);
    n[i] = uint2{code4<CODE>(f[0], f[1], f[2], f[3]), code4<CODE>(f[4], f[5], f[6], f[7])};
  }
  const bool upper = lane & 8;
  const uint2 give = upper ? n[0] : n[1], keep = upper ? n[1] : n[0];
  const uint2 got{lane_xor8(give.x), lane_xor8(give.y)};
  u32x4 r = upper ? u32x4{got.x, got.y, keep.x, keep.y} : u32x4{keep.x, keep.y, got.x, got.y};
  if (!whole) {
    uint32_t fresh[2] = {0, 0}, live[2] = {0, 0};              // the bytes of new and of live tokens
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = t0 + slot_token(w, j);
      if (t >= lo && t < hi) fresh[j >> 2] |= 255u << (8 * (j & 3));
      else if (t < start) live[j >> 2] |= 255u << (8 * (j & 3));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t o = vold[i];
      if (begun && va > vo) o = (again(o, vo, va, rv) & live[i & 1]) | (o & ~live[i & 1]);
      r[i] = (r[i] & fresh[i & 1]) | (o & ~fresh[i & 1]);
    }
  }
  *pv = r;
}

// All arguments of a writing kernel in one round trip; left to itself the compiler asks for each where it is used.
__device__ __forceinline__ void ask_arguments(const C8Write& a) {
  asm volatile("" :: "s"(a.K.data), "s"(a.K.sb), "s"(a.K.sh), "s"(a.K.st), "s"(a.V.data), "s"(a.V.sb), "s"(a.V.sh), "s"(a.V.st),
               "s"(a.start), "s"(a.count), "s"(a.kc), "s"(a.vc), "s"(a.km), "s"(a.vm), "s"(a.H), "s"(a.nbc), "s"(a.cap), "s"(a.n));
}

// Blocks of a sequence that its n new tokens can touch, wherever they start; those behind the capacity are dropped.
inline int c8_reach(const C8Geom& g, int n) { return (int)std::min<long long>(((long long)n + 2 * G - 2) / G, g.nbc); }

}  // namespace vidkv
