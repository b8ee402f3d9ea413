// The 8-bit cache's codes: written as tokens arrive, read back as values.
//
// A block is 32 tokens x 128 channels of one head; for K and V each it has a magnitude A = max |x| and codes of
// x / A.  2 bytes in and 1 out an element (1 in and 2 or 4 out on the way back): bound by HBM; one token a sequence: by
// the chain start -> row -> maximum over the workgroup -> code.
#include "cache8_write.h"

namespace vidkv {

template <class T, int CODE, bool ROT>
__global__ __launch_bounds__(256) void c8_write_kernel(C8Write a) {
  ask_arguments(a);
  if constexpr (ROT) asm volatile("" :: "s"(a.rot.pos), "s"(a.rot.rows), "s"(a.rot.rot_dim), "s"(a.rot.adjacent), "s"(a.n_axes));
  const int b = blockIdx.z;
  write_block<T, CODE, ROT>(a, InOrder{}, b, blockIdx.y, 0, blockIdx.x, a.start[b], a.count ? min(a.count[b], a.n) : a.n, nullptr);
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
  const dim3 grid((unsigned)c8_reach(g, n), g.H, g.B), blk(256);
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
