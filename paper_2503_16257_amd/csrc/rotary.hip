// Rotary positions on several axes: pair i of a head's first rot_dim channels is turned by pos[axis[i]] * freq_i,
//   y1 = x1 cos - x2 sin,  y2 = x2 cos + x1 sin,
// forward and inverse (the backward pass).  2 x the element's bytes of traffic an element and about four
// operations: bound by HBM, for single tokens by the launch.  cos and sin belong to a (token, pair), not to a head: a thread
// makes those of its pairs once and turns them in one or two heads.  6272 tokens of 32 heads x 128 in bf16: 18 us for 103 MB;
// 3 x 4097 of 32 x 80 in float32, inverse: 46 us for 252 MB, 5.5 TB/s; one token 2.7 us.
#include "cache8.h"

namespace vidkv {

struct RotaryArgs {
  View q, qo, k, ko;
  int Hq, Hk;
  int n;                       // tokens a sequence
  int rows;                    // sequences x tokens
  int per;                     // heads a thread
  float sign;                  // -1: inverse
  int n_axes;
  Rot rot;
};

// A unit is two runs of E elements of a token's head: the two sides of E pairs, or 2 E channels behind rot_dim.  Runs are 16
// bytes, or, where the tokens are few, two elements: what a thread then waits for is its chain of sines, not its bytes.
// Thread = one unit of one token in `per` heads.  What a thread waits for is asked for at once: the pairs'
// axes and turns, the positions of every axis, the first head's channels.
// grid (ceil(rows / tokens a workgroup), ceil(heads / per)).
template <class T, int E>
struct RotaryRun {                         // 16 bytes
  typedef typename T::Run Raw;
  static __device__ __forceinline__ Raw load(const char* p) { return T::load(p); }
  static __device__ __forceinline__ auto widen(Raw r) { return T::widen(r); }
  template <class V> static __device__ __forceinline__ void store(char* p, V v) { T::store(p, v); }
};
template <class T>
struct RotaryRun<T, 2> {
  typedef typename T::Run2 Raw;
  static __device__ __forceinline__ Raw load(const char* p) { return T::load2(p); }
  static __device__ __forceinline__ f2 widen(Raw r) { return T::widen2(r); }
  static __device__ __forceinline__ void store(char* p, f2 v) { T::store2(p, v[0], v[1]); }
};

template <class T, int E>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  // (all arguments in one round trip; left to itself the compiler asks for each where it is used)
  asm volatile("" :: "s"(a.q.data), "s"(a.q.sb), "s"(a.q.sh), "s"(a.q.st), "s"(a.k.data), "s"(a.k.sb), "s"(a.k.sh), "s"(a.k.st),
               "s"(a.qo.data), "s"(a.ko.data), "s"(a.Hq), "s"(a.Hk), "s"(a.n), "s"(a.rows), "s"(a.per), "s"(a.rot.pos),
               "s"(a.rot.head_dim), "s"(a.rot.rot_dim), "s"(a.rot.adjacent), "s"(a.n_axes));
  typedef RotaryRun<T, E> R;
  typedef float fe __attribute__((ext_vector_type(E)));
  const int U = a.rot.head_dim / (2 * E), tpw = 256 / U;
  const int tok = threadIdx.x / U, u = threadIdx.x - tok * U;
  const int row = blockIdx.x * tpw + tok;
  if (tok >= tpw || row >= a.rows) return;
  const int b = row / a.n, t = row - b * a.n;
  int c0 = 2 * E * u, c1 = c0 + E;         // the two runs
  const bool turns = c0 < a.rot.rot_dim;
  if (turns && !a.rot.adjacent) { c0 = E * u; c1 = c0 + a.rot.rot_dim / 2; }
  const int h0 = blockIdx.y * a.per, h1 = min(h0 + a.per, a.Hq + a.Hk);
  auto at = [&](int h, const View& q, const View& k) {
    const View& v = h < a.Hq ? q : k;
    const int hh = h < a.Hq ? h : h - a.Hq;
    return v.data + b * v.sb + hh * v.sh + t * v.st;
  };
  typename R::Raw r0 = R::load(at(h0, a.q, a.k) + c0 * T::BYTES), r1 = R::load(at(h0, a.q, a.k) + c1 * T::BYTES);
  float co[E], si[E];
  if (turns) {
    int pos[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) pos[x] = a.rot.pos[(long long)min(x, a.n_axes - 1) * a.rows + row];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int ax = a.rot.axis[E * u + e];
      turn_cos_sin(ax & 2 ? (ax & 1 ? pos[3] : pos[2]) : (ax & 1 ? pos[1] : pos[0]), a.rot.turn[E * u + e], &co[e], &si[e]);
      si[e] *= a.sign;
    }
  }
  for (int h = h0; h < h1; ++h) {
    fe x = R::widen(r0), y = R::widen(r1);
    if (h + 1 < h1) {                      // the next head's, in flight meanwhile
      r0 = R::load(at(h + 1, a.q, a.k) + c0 * T::BYTES);
      r1 = R::load(at(h + 1, a.q, a.k) + c1 * T::BYTES);
    }
    if (turns) turn_runs<E>(x, y, a.rot.adjacent, co, si);
    char* out = const_cast<char*>(at(h, a.qo, a.ko));
    R::store(out + c0 * T::BYTES, x);
    R::store(out + c1 * T::BYTES, y);
  }
}

hipError_t launch_rotary(const vidkv_rotary* r, int inverse, int B, int n, const int32_t* pos, int Hq, const vidkv_view* q,
                         const vidkv_view* qo, int Hk, const vidkv_view* k, const vidkv_view* ko, int dtype, hipStream_t st) {
  RotaryArgs a{};
  a.q = make_view(q); a.qo = make_view(qo); a.k = make_view(k); a.ko = make_view(ko);
  a.Hq = q ? Hq : 0; a.Hk = k ? Hk : 0;
  a.n = n; a.rows = B * n;
  a.sign = inverse ? -1.0f : 1.0f;
  a.n_axes = r->n_axes;
  a.rot = make_rot(r, pos, a.rows);
  const int heads = a.Hq + a.Hk;
  // (32 heads of one token, the kernel: 2.7 us with runs of two elements, 3.7 with 16 bytes; calls among others 4.9 and 5.5, of
  // 64 tokens 4.8 and 4.8, of 400 4.9 and 4.8)
  const bool short_runs = (long long)a.rows * heads <= 2048;
  const int run = short_runs ? 2 : 16 / dtype_bytes(dtype), tpw = 256 / (r->head_dim / (2 * run));
  const int tiles = (a.rows + tpw - 1) / tpw;
  // two heads a thread where that leaves a workgroup for every second compute unit (32 heads x 6272 tokens in bf16, one, two,
  // four and eight heads: 29.1, 22.8, 22.3, 23.7 us; x 1000: 6.4, 5.6, 5.7, 7.0; x 64 of one token: 4.5, 4.7, 4.7, 6.1); a thread
  // of float32 makes half as many sines (3 x 4097 tokens of 32 heads: 46.5, 47.9, 49.4, 50.9)
  a.per = dtype != VIDKV_F32 && !short_runs && (long long)tiles * heads >= device_cu_count() ? 2 : 1;
  const dim3 grid(tiles, (heads + a.per - 1) / a.per);
  auto go = [&](auto t) {
    using T = decltype(t);
    if (short_runs) hipLaunchKernelGGL((rotary_kernel<T, 2>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((rotary_kernel<T, 16 / T::BYTES>), grid, dim3(256), 0, st, a);
  };
  if (dtype == VIDKV_F16) go(TF16{});
  else if (dtype == VIDKV_BF16) go(TBF16{});
  else go(TF32{});
  return hipGetLastError();
}

}  // namespace vidkv
