// The 8-bit cache's codes: written as tokens arrive, read back as values.
//
// A block is 32 tokens x 128 channels of one head; for K and V each it has a magnitude A = max |x| and codes of
// x / A.  2 bytes in and 1 out an element (1 in and 2 or 4 out on the way back): bound by HBM; one token a sequence: by
// the chain start -> row -> maximum over the workgroup -> code.
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

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

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

// Two elements held to the largest magnitude that goes into a block: an infinity is the type's largest number, a NaN a zero,
// so that no code is one (a weight of zero times it would be a NaN in rows that do not see its token).
template <class T>
__device__ __forceinline__ uint32_t held(uint32_t u) {
  const uint32_t a = u & 0x7fffu, b = u >> 16 & 0x7fffu, lo = a > T::INF ? 0 : min(a, (uint32_t)T::TOP),
                 hi = b > T::INF ? 0 : min(b, (uint32_t)T::TOP);
  return (u & 0x80008000u) | lo | hi << 16;
}

constexpr int FEW = 8;                     // new tokens of a block whose sines are shared out

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
template <class T, int CODE, bool ROT>
__global__ __launch_bounds__(256) void c8_write_kernel(C8Write a) {
  // (all arguments in one round trip; left to itself the compiler asks for each where it is used)
  asm volatile("" :: "s"(a.K.data), "s"(a.K.sb), "s"(a.K.sh), "s"(a.K.st), "s"(a.V.data), "s"(a.V.sb), "s"(a.V.sh), "s"(a.V.st),
               "s"(a.start), "s"(a.count), "s"(a.kc), "s"(a.vc), "s"(a.km), "s"(a.vm), "s"(a.H), "s"(a.nbc), "s"(a.cap), "s"(a.n));
  if constexpr (ROT) asm volatile("" :: "s"(a.rot.pos), "s"(a.rot.rows), "s"(a.rot.rot_dim), "s"(a.rot.adjacent), "s"(a.n_axes));
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int start = a.start[b];
  const int count = a.count ? min(a.count[b], a.n) : a.n;
  if (start < 0 || count <= 0) return;
  const long long first = (long long)(start / G + (long long)blockIdx.x) * G;
  const long long end = (long long)start + count;
  if (first >= end || first >= a.cap) return;
  const int t0 = (int)first;
  const int lo = max(start, t0), hi = (int)min(min(end, (long long)t0 + G), (long long)a.cap);
  const size_t blk = ((size_t)b * a.H + h) * a.nbc + t0 / G;
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
    const char* in = a.K.data + b * a.K.sb + h * a.K.sh + (long long)(kt - start) * a.K.st;
    rx = T::load(in + 2 * c0);
    ry = T::load(in + 2 * c1);
  }
  const char* vin = a.V.data + b * a.V.sb + h * a.V.sh;        // (row addresses are the wave's: scalar)
  uint32_t v[8];                           // two channels of a token, as they lie in memory
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = t0 + slot_token(w, j);
    v[j] = 0;
    if (whole || (t >= lo && t < hi)) v[j] = *reinterpret_cast<const uint32_t*>(vin + (long long)(t - start) * a.V.st + 4 * lane);
  }
  float ko = 0.0f, vo = 0.0f;
  uint2 k0{}, k1{};
  u32x4 vold{};
  if (begun) {
    ko = a.km[blk]; vo = a.vm[blk];
    k0 = *pk0; k1 = *pk1;
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

hipError_t launch_c8_write(const C8Geom& g, int layer, int n, const vidkv_view* K, const vidkv_view* V,
                           const int32_t* start, const int32_t* count, const vidkv_rotary* rot, const int32_t* pos,
                           uint8_t* cache, hipStream_t st) {
  const size_t blk0 = (size_t)layer * g.B * g.H * g.nbc;
  C8Write a{};
  a.K = make_view(K); a.V = make_view(V);
  a.n = n; a.start = start; a.count = count;
  a.kc = cache + blk0 * C8REC;
  a.vc = cache + g.v_codes + blk0 * C8REC;
  a.km = reinterpret_cast<float*>(cache + g.k_mag) + blk0;
  a.vm = reinterpret_cast<float*>(cache + g.v_mag) + blk0;
  a.H = g.H; a.nbc = g.nbc; a.cap = g.cap;
  a.rot = make_rot(rot, pos, (long long)g.B * n);
  a.n_axes = rot ? rot->n_axes : 1;
  // tokens that do not fit are dropped: no more blocks than the cache has
  const long long reach = ((long long)n + 2 * G - 2) / G;
  const dim3 grid((unsigned)(reach < g.nbc ? reach : g.nbc), g.H, g.B), blk(256);
  auto go = [&](auto t, auto code) {
    using T = decltype(t);
    constexpr int CODE = decltype(code)::value;
    if (rot) hipLaunchKernelGGL((c8_write_kernel<T, CODE, true>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((c8_write_kernel<T, CODE, false>), grid, blk, 0, st, a);
  };
  auto by_code = [&](auto t) {
    if (g.code == 0) go(t, std::integral_constant<int, 0>{});
    else go(t, std::integral_constant<int, 1>{});
  };
  if (K->dtype == VIDKV_F16) by_code(TF16{});
  else by_code(TBF16{});
  return hipGetLastError();
}

struct C8Read {
  View K, V;
  int n;
  const int32_t* start;
  const uint8_t* kc;
  const uint8_t* vc;
  const float* km;
  const float* vm;
  int H, nbc, cap;
};

// One workgroup per block that the asked-for tokens lie in, threads as above.  8 x 4 heads x 12544 tokens as fp16: 56 us for
// 308 MB, 5.5 TB/s.
template <class T, int CODE>
__global__ __launch_bounds__(256) void c8_read_kernel(C8Read a) {
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int start = a.start[b];
  const long long t0 = ((long long)(start >> 5) + blockIdx.x) * G;      // (a negative start too: its block is below 0)
  const long long end = (long long)start + a.n;
  const bool there = t0 >= 0 && t0 < a.cap;
  const size_t blk = ((size_t)b * a.H + h) * a.nbc + (there ? t0 / G : 0);
  if (a.K.data) {
    const long long t = t0 + (tid >> 3);
    if (t >= start && t < end) {
      f8v x = f8v(0.0f), y = f8v(0.0f);
      if (there) {
        const float s = a.km[blk] * (1.0f / kLevel<CODE>);
        const u32x4 c = *reinterpret_cast<const u32x4*>(a.kc + blk * C8REC + tid * 16);
        x = __builtin_convertvector(decode8<CODE>(c[0], c[1]).v, f8v) * s;
        y = __builtin_convertvector(decode8<CODE>(c[2], c[3]).v, f8v) * s;
      }
      char* out = a.K.data + b * a.K.sb + h * a.K.sh + (t - start) * a.K.st + (tid & 7) * 16 * T::BYTES;
      T::store8(out, x);
      T::store8(out + 8 * T::BYTES, y);
    }
  }
  if (a.V.data) {
    f8v v[2] = {f8v(0.0f), f8v(0.0f)};
    if (there) {
      const float s = a.vm[blk] * (1.0f / kLevel<CODE>);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = 2 * lane + i;
        const uint2 o = *reinterpret_cast<const uint2*>(a.vc + blk * C8REC + (((c >> 5) * 4 + w) * 16 + (c & 15)) * 16 +
                                                        ((c >> 4) & 1) * 8);
        v[i] = __builtin_convertvector(decode8<CODE>(o.x, o.y).v, f8v) * s;
      }
    }
    char* out = a.V.data + b * a.V.sb + h * a.V.sh + 2 * lane * T::BYTES;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const long long t = t0 + slot_token(w, j);
      if (t >= start && t < end) T::store2(out + (t - start) * a.V.st, v[0][j], v[1][j]);
    }
  }
}

hipError_t launch_c8_read(const C8Geom& g, int layer, int n, const int32_t* start, const uint8_t* cache,
                          const vidkv_view* K, const vidkv_view* V, hipStream_t st) {
  const size_t blk0 = (size_t)layer * g.B * g.H * g.nbc;
  C8Read a{};
  a.K = make_view(K); a.V = make_view(V);
  a.n = n; a.start = start;
  a.kc = cache + blk0 * C8REC;
  a.vc = cache + g.v_codes + blk0 * C8REC;
  a.km = reinterpret_cast<const float*>(cache + g.k_mag) + blk0;
  a.vm = reinterpret_cast<const float*>(cache + g.v_mag) + blk0;
  a.H = g.H; a.nbc = g.nbc; a.cap = g.cap;
  const dim3 grid((unsigned)(((long long)n + 2 * G - 2) / G), g.H, g.B), blk(256);
  auto go = [&](auto t) {
    using T = decltype(t);
    if (g.code == 0) hipLaunchKernelGGL((c8_read_kernel<T, 0>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((c8_read_kernel<T, 1>), grid, blk, 0, st, a);
  };
  const int dt = K ? K->dtype : V->dtype;
  if (dt == VIDKV_F16) go(TF16{});
  else if (dt == VIDKV_BF16) go(TBF16{});
  else go(TF32{});
  return hipGetLastError();
}

}  // namespace vidkv
