// C ABI of the rotary positions and the 8-bit cache: argument checks on the host, then launches on the caller's stream.
#include <cmath>

#include "cache8.h"

namespace vidkv {
hipError_t launch_rotary(const vidkv_rotary* r, int inverse, int B, int n, const int32_t* pos, int Hq, const vidkv_view* q,
                         const vidkv_view* qo, int Hk, const vidkv_view* k, const vidkv_view* ko, int dtype, hipStream_t st);
hipError_t launch_c8_write(const C8Geom& g, int layer, int n, const vidkv_view* K, const vidkv_view* V,
                           const int32_t* start, const int32_t* count, const vidkv_rotary* rot, const int32_t* pos,
                           uint8_t* cache, hipStream_t st);
hipError_t launch_c8_read(const C8Geom& g, int layer, int n, const int32_t* start, const uint8_t* cache,
                          const vidkv_view* K, const vidkv_view* V, hipStream_t st);
hipError_t launch_c8_attn(const C8Geom& g, int layer, int n, int causal, float scale, const vidkv_view* q,
                          const uint8_t* cache, const int32_t* length, const int32_t* q_count, const vidkv_view* out,
                          void* ws, hipStream_t st);
size_t c8_attn_ws_bytes(const C8Geom& g, int n);
size_t c8_attn_ws_need(const C8Geom& g, int n);
bool c8_attn_fits(const C8Geom& g, int n);
}  // namespace vidkv

using namespace vidkv;

namespace {
bool at(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// A view that a kernel can take: data there, 16 bytes at a time.
bool good_view(const vidkv_view* v, bool f32) {
  if (!v || !v->data || !at(v->data, 16)) return false;
  if (v->dtype != VIDKV_F16 && v->dtype != VIDKV_BF16 && !(f32 && v->dtype == VIDKV_F32)) return false;
  const int64_t e = 16 / dtype_bytes(v->dtype);
  const int64_t most = (int64_t)1 << 48;
  for (int64_t s : {v->stride_batch, v->stride_head, v->stride_token})
    if (s % e || s < -most || s > most) return false;
  return true;
}

bool good_rotary(const vidkv_rotary* r) {
  if (r->head_dim < 16 || r->head_dim > 256 || r->head_dim % 16) return false;
  if (r->rot_dim < 16 || r->rot_dim > r->head_dim || r->rot_dim % 16) return false;
  if ((r->adjacent != 0 && r->adjacent != 1) || r->n_axes < 1 || r->n_axes > 4) return false;
  for (int i = 0; i < r->rot_dim / 2; ++i)
    if (r->axis[i] >= r->n_axes) return false;
  return true;
}

// Tokens of a call, and rows (queries x heads of a group): HIP counts a grid dimension's threads in 32 bits.
constexpr int32_t MOST_TOKENS = 1 << 28;
bool few_enough(const C8Geom& g, int n) { return (long long)n * g.rep <= MOST_TOKENS; }
}  // namespace

extern "C" {

vidkv_status vidkv_rotary_init(vidkv_rotary* rot, int32_t head_dim, int32_t rot_dim, int32_t adjacent, int32_t n_axes,
                               const int32_t* sections, double theta, const double* freq) {
  if (!rot || !sections) return VIDKV_EINVAL;
  if (n_axes < 1 || n_axes > 4) return VIDKV_ESHAPE;
  vidkv_rotary r{};
  r.head_dim = head_dim; r.rot_dim = rot_dim; r.adjacent = adjacent; r.n_axes = n_axes;
  if (head_dim < 16 || head_dim > 256 || head_dim % 16 || rot_dim < 16 || rot_dim > head_dim || rot_dim % 16)
    return VIDKV_ESHAPE;
  if (adjacent != 0 && adjacent != 1) return VIDKV_EINVAL;
  const int pairs = rot_dim / 2;
  int i = 0;
  for (int x = 0; x < n_axes; ++x) {
    if (sections[x] < 0 || sections[x] > pairs - i) return VIDKV_EINVAL;
    for (int k = 0; k < sections[x]; ++k) r.axis[i++] = (uint8_t)x;
  }
  if (i != pairs) return VIDKV_EINVAL;
  if (!freq && !(theta > 0.0 && std::isfinite(theta))) return VIDKV_EINVAL;
  const long double two_pi = 6.283185307179586476925286766559L;
  for (i = 0; i < pairs; ++i) {
    const long double f = freq ? (long double)freq[i] : powl((long double)theta, -(long double)i / pairs);
    if (!std::isfinite((double)f)) return VIDKV_EINVAL;
    long double turns = f / two_pi;
    turns -= floorl(turns);                                   // [0, 1]
    const long double t = floorl(turns * 0x1p64L + 0.5L);
    r.turn[i] = t >= 0x1p64L ? 0 : (uint64_t)t;
  }
  *rot = r;
  return VIDKV_OK;
}

vidkv_status vidkv_rotary_apply(const vidkv_rotary* rot, int32_t inverse, int32_t batch, int32_t n_tokens,
                                const int32_t* pos, int32_t n_q_heads, const vidkv_view* q, const vidkv_view* q_out,
                                int32_t n_k_heads, const vidkv_view* k, const vidkv_view* k_out, void* stream) {
  if (!rot || !pos || (!q && !k) || (q && !q_out) || (k && !k_out)) return VIDKV_EINVAL;
  if (!good_rotary(rot) || (inverse != 0 && inverse != 1) || !at(pos, 4)) return VIDKV_EINVAL;
  if (batch < 0 || n_tokens < 0 || (q && n_q_heads < 0) || (k && n_k_heads < 0)) return VIDKV_EINVAL;
  if ((int64_t)batch * n_tokens > (1 << 26) || (q && n_q_heads > 65535) || (k && n_k_heads > 65535)) return VIDKV_ESHAPE;
  const long long heads = (q ? n_q_heads : 0) + (k ? n_k_heads : 0);
  if (heads > 65535) return VIDKV_ESHAPE;
  const int32_t dtype = q ? q->dtype : k->dtype;
  for (const vidkv_view* v : {q, q ? q_out : nullptr, k, k ? k_out : nullptr})
    if (v && (!good_view(v, true) || v->dtype != dtype)) return VIDKV_EINVAL;
  if (!stream_on_current_device(static_cast<hipStream_t>(stream))) return VIDKV_EINVAL;
  if (batch == 0 || n_tokens == 0 || heads == 0) return VIDKV_OK;
  const hipError_t e = launch_rotary(rot, inverse, batch, n_tokens, pos, n_q_heads, q, q_out, n_k_heads, k, k_out, dtype,
                                     static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VIDKV_OK : VIDKV_EHIP;
}

size_t vidkv_cache8_bytes(const vidkv_cache8* p) {
  C8Geom g;
  return make_c8(p, &g) ? g.total : 0;
}

size_t vidkv_cache8_workspace_bytes(const vidkv_cache8* p, int32_t n_query) {
  C8Geom g;
  if (!make_c8(p, &g) || n_query < 1 || !few_enough(g, n_query)) return 0;
  return c8_attn_ws_bytes(g, n_query);
}

vidkv_status vidkv_cache8_write(const vidkv_cache8* p, int32_t layer, int32_t n_tokens, const vidkv_view* K,
                                const vidkv_view* V, const int32_t* start, const int32_t* count, const vidkv_rotary* rot,
                                const int32_t* pos, void* cache, size_t cache_bytes, void* stream) {
  C8Geom g;
  if (!p || !cache || !start) return VIDKV_EINVAL;
  if (!make_c8(p, &g)) return VIDKV_ESHAPE;
  if (n_tokens > MOST_TOKENS) return VIDKV_ESHAPE;
  if (layer < 0 || layer >= g.L || n_tokens < 0) return VIDKV_EINVAL;
  if (!good_view(K, false) || !good_view(V, false) || K->dtype != V->dtype) return VIDKV_EINVAL;
  if ((rot != nullptr) != (pos != nullptr)) return VIDKV_EINVAL;
  if (rot && (!good_rotary(rot) || rot->head_dim != D)) return VIDKV_EINVAL;
  if (!at(cache, 256) || !at(start, 4) || !at(count, 4) || !at(pos, 4)) return VIDKV_EINVAL;
  if (cache_bytes < g.total) return VIDKV_ENOSPACE;
  if (!stream_on_current_device(static_cast<hipStream_t>(stream))) return VIDKV_EINVAL;
  if (n_tokens == 0) return VIDKV_OK;
  const hipError_t e = launch_c8_write(g, layer, n_tokens, K, V, start, count, rot, pos, static_cast<uint8_t*>(cache),
                                       static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VIDKV_OK : VIDKV_EHIP;
}

vidkv_status vidkv_cache8_read(const vidkv_cache8* p, int32_t layer, int32_t n_tokens, const int32_t* start,
                               const void* cache, size_t cache_bytes, const vidkv_view* K, const vidkv_view* V,
                               void* stream) {
  C8Geom g;
  if (!p || !cache || !start || (!K && !V)) return VIDKV_EINVAL;
  if (!make_c8(p, &g)) return VIDKV_ESHAPE;
  if (n_tokens > MOST_TOKENS) return VIDKV_ESHAPE;
  if (layer < 0 || layer >= g.L || n_tokens < 0) return VIDKV_EINVAL;
  if ((K && !good_view(K, true)) || (V && !good_view(V, true)) || (K && V && K->dtype != V->dtype)) return VIDKV_EINVAL;
  if (!at(cache, 256) || !at(start, 4)) return VIDKV_EINVAL;
  if (cache_bytes < g.total) return VIDKV_ENOSPACE;
  if (!stream_on_current_device(static_cast<hipStream_t>(stream))) return VIDKV_EINVAL;
  if (n_tokens == 0) return VIDKV_OK;
  const hipError_t e = launch_c8_read(g, layer, n_tokens, start, static_cast<const uint8_t*>(cache), K, V,
                                      static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VIDKV_OK : VIDKV_EHIP;
}

vidkv_status vidkv_cache8_attention(const vidkv_cache8* p, int32_t layer, int32_t n_query, int32_t causal,
                                    const vidkv_view* q, const void* cache, size_t cache_bytes, const int32_t* length,
                                    const int32_t* q_count, const vidkv_view* out, void* ws, size_t ws_bytes,
                                    void* stream) {
  C8Geom g;
  if (!p || !cache || !length || !ws) return VIDKV_EINVAL;
  if (!make_c8(p, &g)) return VIDKV_ESHAPE;
  if (layer < 0 || layer >= g.L || n_query < 0 || (causal != 0 && causal != 1)) return VIDKV_EINVAL;
  if (!(p->softmax_scale > 0.0f) || !(p->softmax_scale < 1e30f)) return VIDKV_EINVAL;
  if (!few_enough(g, n_query) || (n_query > 0 && !c8_attn_fits(g, n_query))) return VIDKV_ESHAPE;
  if (!good_view(q, false) || !good_view(out, false) || q->dtype != out->dtype) return VIDKV_EINVAL;
  if (!at(cache, 256) || !at(ws, 256) || !at(length, 4) || !at(q_count, 4)) return VIDKV_EINVAL;
  if (n_query == 0) return VIDKV_OK;
  if (cache_bytes < g.total || ws_bytes < c8_attn_ws_need(g, n_query)) return VIDKV_ENOSPACE;
  if (!stream_on_current_device(static_cast<hipStream_t>(stream))) return VIDKV_EINVAL;
  const hipError_t e = launch_c8_attn(g, layer, n_query, causal, p->softmax_scale, q, static_cast<const uint8_t*>(cache),
                                      length, q_count, out, ws, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VIDKV_OK : VIDKV_EHIP;
}

}  // extern "C"
