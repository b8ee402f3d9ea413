// Rotary positions on several axes: pair i of a head's first rot_dim channels is turned by pos[axis[i]] * freq_i,
//   y1 = x1 cos - x2 sin,  y2 = x2 cos + x1 sin,
// forward and inverse (the backward pass).  2 x the element's bytes of traffic an element and about four
// operations: bound by HBM, for single tokens by the launch.  cos and sin belong to a (token, pair), not to a head: a thread
// makes those of eight pairs once and turns them in several heads.
#include "cache8.h"

namespace vidkv {

struct RotaryArgs {
  View q, qo, k, ko;
  int Hq, Hk;
  int n;                       // tokens a sequence
  int rows;                    // sequences x tokens
  int per;                     // heads a thread
  float sign;                  // -1: inverse
  Rot rot;
};

// Thread = 16 channels of one token (a unit) in `per` heads: eight pairs, or 16 channels behind rot_dim.
// grid (ceil(rows / tokens a workgroup), ceil(heads / per)).
template <class T>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  const int U = a.rot.head_dim / 16, tpw = 256 / U;
  const int tok = threadIdx.x / U, u = threadIdx.x - tok * U;
  const int row = blockIdx.x * tpw + tok;
  if (tok >= tpw || row >= a.rows) return;
  const int b = row / a.n, t = row - b * a.n;
  const int ur = a.rot.rot_dim / 16;
  int c0 = 16 * u, c1 = c0 + 8;            // the two runs of eight channels
  const bool turns = u < ur;
  if (turns && !a.rot.adjacent) { c0 = 8 * u; c1 = c0 + a.rot.rot_dim / 2; }
  float co[8], si[8];
  if (turns) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = 8 * u + e;
      turn_cos_sin(a.rot.pos[(long long)a.rot.axis[i] * a.rows + row], a.rot.turn[i], &co[e], &si[e]);
      si[e] *= a.sign;
    }
  }
  const int h0 = blockIdx.y * a.per, h1 = min(h0 + a.per, a.Hq + a.Hk);
#pragma unroll 4
  for (int h = h0; h < h1; ++h) {
    const bool isq = h < a.Hq;
    const View& vi = isq ? a.q : a.k;
    const View& vo = isq ? a.qo : a.ko;
    const int hh = isq ? h : h - a.Hq;
    const char* in = vi.data + b * vi.sb + hh * vi.sh + t * vi.st;
    char* out = vo.data + b * vo.sb + hh * vo.sh + t * vo.st;
    f8v x = T::load8(in + c0 * T::BYTES), y = T::load8(in + c1 * T::BYTES);
    if (turns) {
      if (a.rot.adjacent) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x1 = x[2 * e], x2 = x[2 * e + 1], y1 = y[2 * e], y2 = y[2 * e + 1];
          x[2 * e] = x1 * co[e] - x2 * si[e];
          x[2 * e + 1] = x2 * co[e] + x1 * si[e];
          y[2 * e] = y1 * co[4 + e] - y2 * si[4 + e];
          y[2 * e + 1] = y2 * co[4 + e] + y1 * si[4 + e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x1 = x[e], x2 = y[e];
          x[e] = x1 * co[e] - x2 * si[e];
          y[e] = x2 * co[e] + x1 * si[e];
        }
      }
    }
    T::store8(out + c0 * T::BYTES, x);
    T::store8(out + c1 * T::BYTES, y);
  }
}

hipError_t launch_rotary(const vidkv_rotary* r, int inverse, int B, int n, const int32_t* pos, int Hq, const vidkv_view* q,
                         const vidkv_view* qo, int Hk, const vidkv_view* k, const vidkv_view* ko, int dtype, hipStream_t st) {
  RotaryArgs a{};
  a.q = make_view(q); a.qo = make_view(qo); a.k = make_view(k); a.ko = make_view(ko);
  a.Hq = q ? Hq : 0; a.Hk = k ? Hk : 0;
  a.n = n; a.rows = B * n;
  a.sign = inverse ? -1.0f : 1.0f;
  a.rot = make_rot(r, pos, a.rows);
  const int heads = a.Hq + a.Hk, tpw = 256 / (r->head_dim / 16);
  const int tiles = (a.rows + tpw - 1) / tpw;
  a.per = 1;
  while (a.per < 8 && (long long)tiles * ((heads + 2 * a.per - 1) / (2 * a.per)) >= 2048) a.per *= 2;
  const dim3 grid(tiles, (heads + a.per - 1) / a.per);
  if (dtype == VIDKV_F16) hipLaunchKernelGGL(rotary_kernel<TF16>, grid, dim3(256), 0, st, a);
  else if (dtype == VIDKV_BF16) hipLaunchKernelGGL(rotary_kernel<TBF16>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(rotary_kernel<TF32>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace vidkv
