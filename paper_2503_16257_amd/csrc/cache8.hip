// The 8-bit cache's codes: written as tokens arrive, read back as values.
//
// A block is 32 tokens x 128 channels of one head; for K and V each it has a magnitude A = max |x| and codes of
// x / A.  2 bytes in and 1 out an element (1 in and 2 or 4 out on the way back): bound by HBM; one token a sequence: by
// the chain start -> row -> maximum over the workgroup -> code.
#include "cache8.h"

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
  int H, nbc, cap;
  Rot rot;
};

// Lane maximum of non-negative numbers over the wave.
__device__ __forceinline__ float wave_max(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
#pragma unroll
  for (int m = 8; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
  return v;
}

// A block's magnitude as it is stored: never zero, and bounded so that no product with it leaves float's range.
__device__ __forceinline__ float bounded(float a) { return fminf(fmaxf(a, C8_LEAST), C8_MOST); }

// One workgroup per block that new tokens reach.  K: thread = 16 channels of one token (two runs of eight, the two
// sides of eight pairs where the keys are turned); V: wave = lane group kb of the record, lane = two channels of its eight
// tokens, so that its codes are whole 8-byte pieces of the record.  grid (blocks a sequence can reach, H, B).
template <class T, int CODE, bool ROT>
__global__ __launch_bounds__(256) void c8_write_kernel(C8Write a) {
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
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
  uint8_t* kc = a.kc + blk * C8REC;
  uint8_t* vc = a.vc + blk * C8REC;
  constexpr float LV = kLevel<CODE>;

  // keys
  const int kt = t0 + (tid >> 3), u = tid & 7;
  const bool knew = kt >= lo && kt < hi;
  int c0 = 16 * u, c1 = c0 + 8;
  const bool turns = ROT && u < a.rot.rot_dim / 16;
  if (turns && !a.rot.adjacent) { c0 = 8 * u; c1 = c0 + a.rot.rot_dim / 2; }
  f8v x = f8v(0.0f), y = f8v(0.0f);
  if (knew) {
    const char* in = a.K.data + b * a.K.sb + h * a.K.sh + (long long)(kt - start) * a.K.st;
    x = T::load8(in + 2 * c0);
    y = T::load8(in + 2 * c1);
  }
  // values
  const char* vin = a.V.data + b * a.V.sb + h * a.V.sh + 4 * lane;
  f2 v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = t0 + slot_token(w, j);
    v[j] = (t >= lo && t < hi) ? T::load2(vin + (long long)(t - start) * a.V.st) : f2{0.0f, 0.0f};
  }
  float ko = 0.0f, vo = 0.0f;
  if (begun) { ko = bounded(a.km[blk]); vo = bounded(a.vm[blk]); }
  if constexpr (ROT) {
    if (turns && knew) {
      const long long row = (long long)b * a.n + (kt - start);
      float co[8], si[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = 8 * u + e;
        turn_cos_sin(a.rot.pos[(long long)a.rot.axis[i] * a.rot.rows + row], a.rot.turn[i], &co[e], &si[e]);
      }
      // (rounded to the tensor's type, as the rotation by itself leaves them)
      if (a.rot.adjacent) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x1 = x[2 * e], x2 = x[2 * e + 1], y1 = y[2 * e], y2 = y[2 * e + 1];
          x[2 * e] = T::round(x1 * co[e] - x2 * si[e]);
          x[2 * e + 1] = T::round(x2 * co[e] + x1 * si[e]);
          y[2 * e] = T::round(y1 * co[4 + e] - y2 * si[4 + e]);
          y[2 * e + 1] = T::round(y2 * co[4 + e] + y1 * si[4 + e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x1 = x[e], x2 = y[e];
          x[e] = T::round(x1 * co[e] - x2 * si[e]);
          y[e] = T::round(x2 * co[e] + x1 * si[e]);
        }
      }
    }
  }

  float ka = 0.0f, va = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    ka = fmaxf(ka, fmaxf(fabsf(x[e]), fabsf(y[e])));
    va = fmaxf(va, fmaxf(fabsf(v[e][0]), fabsf(v[e][1])));
  }
  ka = wave_max(ka);
  va = wave_max(va);
  __shared__ float red[2][4];
  if (lane == 0) { red[0][w] = ka; red[1][w] = va; }
  __syncthreads();
  ka = bounded(fmaxf(fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3])), ko));
  va = bounded(fmaxf(fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3])), vo));
  const float rk = __builtin_amdgcn_rcpf(ka), rv = __builtin_amdgcn_rcpf(va);
  if (tid == 0) { a.km[blk] = ka; a.vm[blk] = va; }

  uint2* pk0 = reinterpret_cast<uint2*>(kc + (tid >> 3) * D + c0);
  uint2* pk1 = reinterpret_cast<uint2*>(kc + (tid >> 3) * D + c1);
  if (knew) {
    uint2 p, q;
    p.x = code4<CODE>(units(x[0], LV, ka, rk), units(x[1], LV, ka, rk), units(x[2], LV, ka, rk), units(x[3], LV, ka, rk));
    p.y = code4<CODE>(units(x[4], LV, ka, rk), units(x[5], LV, ka, rk), units(x[6], LV, ka, rk), units(x[7], LV, ka, rk));
    q.x = code4<CODE>(units(y[0], LV, ka, rk), units(y[1], LV, ka, rk), units(y[2], LV, ka, rk), units(y[3], LV, ka, rk));
    q.y = code4<CODE>(units(y[4], LV, ka, rk), units(y[5], LV, ka, rk), units(y[6], LV, ka, rk), units(y[7], LV, ka, rk));
    *pk0 = p;
    *pk1 = q;
  } else if (kt < start && ka > ko) {      // (only in a begun block) live tokens under the new magnitude
    auto again = [&](uint32_t c) {
      h2 l, g;
      decode4<CODE>(c, &l, &g);
      return code4<CODE>(units((float)l[0], ko, ka, rk), units((float)l[1], ko, ka, rk), units((float)g[0], ko, ka, rk),
                         units((float)g[1], ko, ka, rk));
    };
    const uint2 p = *pk0, q = *pk1;
    *pk0 = uint2{again(p.x), again(p.y)};
    *pk1 = uint2{again(q.x), again(q.y)};
  }

  // the record's bytes of channel 2 lane + i, lane group w
  const bool whole = lo == t0 && hi == t0 + G;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = 2 * lane + i;
    uint2* pv = reinterpret_cast<uint2*>(vc + (((c >> 5) * 4 + w) * 16 + (c & 15)) * 16 + ((c >> 4) & 1) * 8);
    uint2 n;
    n.x = code4<CODE>(units(v[0][i], LV, va, rv), units(v[1][i], LV, va, rv), units(v[2][i], LV, va, rv),
                      units(v[3][i], LV, va, rv));
    n.y = code4<CODE>(units(v[4][i], LV, va, rv), units(v[5][i], LV, va, rv), units(v[6][i], LV, va, rv),
                      units(v[7][i], LV, va, rv));
    if (!whole) {
      const uint2 o = *pv;
      uint2 m = o;                                            // live tokens' codes
      if (begun && va > vo) {
        h2 l, g;
        decode4<CODE>(o.x, &l, &g);
        m.x = code4<CODE>(units((float)l[0], vo, va, rv), units((float)l[1], vo, va, rv), units((float)g[0], vo, va, rv),
                          units((float)g[1], vo, va, rv));
        decode4<CODE>(o.y, &l, &g);
        m.y = code4<CODE>(units((float)l[0], vo, va, rv), units((float)l[1], vo, va, rv), units((float)g[0], vo, va, rv),
                          units((float)g[1], vo, va, rv));
      }
      auto pick = [&](uint32_t neu, uint32_t live, uint32_t old, int j0) {
        uint32_t r = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int t = t0 + slot_token(w, j0 + j);
          r |= (t >= lo && t < hi ? neu : t < start ? live : old) & (255u << (8 * j));
        }
        return r;
      };
      n = uint2{pick(n.x, m.x, o.x, 0), pick(n.y, m.y, o.y, 4)};
    }
    *pv = n;
  }
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

// One workgroup per block that the asked-for tokens lie in, threads as above.
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
