// Decode steps that need more than one pass over a cache's rows in plain form:
// the accumulated weights of a step, and attention over a shared prefix and
// the sequence's own rows.
#include <cmath>
#include <string>

#include "sckv_common.h"

namespace sckv {

struct StepFreq {
  double w[40];
};

template <typename T>
struct StepArgs {
  const T *q, *k_new, *v_new, *k_pre, *v_pre;
  T *k_cache, *v_cache, *o;
  const int32_t *pre_len, *kv_len, *cur_tok, *vu, *pos;
  const float* w_in;
  float *w_out, *scores;
  int32_t* status;
  int32_t per, P_cap, L_meta, H, L_cap, rotate;
  float c;
};

constexpr int STEP_THREADS = 256;

// one workgroup per slice: scores of prefix rows, own rows and the new row,
// their maximum and sum, then outputs and weights
template <typename T, int D>
__global__ __launch_bounds__(STEP_THREADS) void step_kernel(StepArgs<T> a, StepFreq tab) {
  constexpr int E = Piece<T>::E;
  __shared__ float qs[D], red[STEP_THREADS], acc[STEP_THREADS / 64][D];
  const int bh = blockIdx.x, s = bh / a.H, h = bh % a.H, tid = threadIdx.x;
  const int t = a.cur_tok[s];
  const int len = a.kv_len[s];
  const bool t_ok = t >= 0 && t < a.L_meta;
  const int kind = !t_ok ? 2 : a.vu[(int64_t)s * a.L_meta + t] == t ? 1 : (len < 0 || len >= a.L_cap) ? 3 : 0;
  const int n = min(max(len, 0), a.L_cap);
  const int64_t wo = (int64_t)bh * a.L_cap;
  T* o = a.o + (int64_t)bh * D;
  if (kind != 0) {
    if (kind > 1 && tid == 0 && h == 0 && a.status)
      atomicOr(a.status, kind == 2 ? SCKV_STATUS_TOKEN : SCKV_STATUS_CAP);
    for (int e = tid; e < D; e += STEP_THREADS) {
      if (kind == 1) o[e] = a.v_new[(int64_t)bh * D + e];
      else if constexpr (sizeof(T) == 2) o[e] = (T)0x7fc0;
      else o[e] = NAN;
    }
    if (a.w_out)
      for (int r = tid; r < n; r += STEP_THREADS) a.w_out[wo + r] = a.w_in ? a.w_in[wo + r] : 0.f;
    return;
  }
  T* kc = a.k_cache + wo * D;
  T* vc = a.v_cache + wo * D;
  auto val = [](const T* p, int i) {
    if constexpr (sizeof(T) == 2) return bf16_lo((uint32_t)p[i]);
    else return p[i];
  };
  if (tid < D) {
    const int64_t x = (int64_t)bh * D;
    const int p = tid < D / 2 ? tid + D / 2 : tid - D / 2;
    float qv = val(a.q + x, tid), kv = val(a.k_new + x, tid);
    if (a.rotate) {
      const double two_pi = 6.283185307179586476925286766559;
      double ang = (double)a.pos[(int64_t)s * a.L_meta + t] * tab.w[tid < D / 2 ? tid : p];
      ang -= two_pi * rint(ang / two_pi);
      float sn, cs;
      sincosf((float)ang, &sn, &cs);
      if (tid < D / 2) sn = -sn;
      qv = qv * cs + val(a.q + x, p) * sn;
      kv = kv * cs + val(a.k_new + x, p) * sn;
    }
    qs[tid] = qv * a.c;
    if constexpr (sizeof(T) == 2) kc[(int64_t)n * D + tid] = f32_to_bf16(kv);
    else kc[(int64_t)n * D + tid] = kv;
    vc[(int64_t)n * D + tid] = a.v_new[x + tid];
  }
  __threadfence_block();
  __syncthreads();
  const int g = s / a.per;
  const int np = a.k_pre ? min(max(a.pre_len[g], 0), a.P_cap) : 0;
  const int64_t po = ((int64_t)g * a.H + h) * a.P_cap * D;
  const int rows = np + n + 1;
  float* sc = a.scores + (int64_t)bh * ((int64_t)a.P_cap + a.L_cap);
  float m = -INFINITY;
  for (int r = tid; r < rows; r += STEP_THREADS) {
    const T* k = r < np ? a.k_pre + po + (int64_t)r * D : kc + (int64_t)(r - np) * D;
    float x = 0.f;
    for (int p = 0; p < D / E; ++p) {
      float f[E];
      Piece<T>::unpack(ld16(k + p * E), f);
#pragma unroll
      for (int e = 0; e < E; ++e) x = fmaf(f[e], qs[p * E + e], x);
    }
    sc[r] = x;
    m = fmaxf(m, x);
  }
  red[tid] = m;
  __threadfence_block();
  __syncthreads();
  for (int i = 0; i < STEP_THREADS; ++i) m = fmaxf(m, red[i]);
  __syncthreads();
  float l = 0.f;
  for (int r = tid; r < rows; r += STEP_THREADS) l += exp2f(sc[r] - m);
  red[tid] = l;
  __syncthreads();
  l = 0.f;
  for (int i = 0; i < STEP_THREADS; ++i) l += red[i];
  const int wave = tid >> 6, lane = tid & 63;
  float v0 = 0.f, v1 = 0.f;
  for (int r = wave; r < rows; r += STEP_THREADS / 64) {
    const T* v = r < np ? a.v_pre + po + (int64_t)r * D : vc + (int64_t)(r - np) * D;
    const float p = exp2f(sc[r] - m);
    v0 = fmaf(p, val(v, lane), v0);
    if (lane + 64 < D) v1 = fmaf(p, val(v, lane + 64), v1);
  }
  acc[wave][lane] = v0;
  if (lane + 64 < D) acc[wave][lane + 64] = v1;
  if (a.w_out)
    for (int r = tid; r < rows; r += STEP_THREADS)
      a.w_out[wo + r] = (a.w_in && r < n ? a.w_in[wo + r] : 0.f) + exp2f(sc[r] - m) / l;
  __syncthreads();
  if (tid < D) {
    float x = 0.f;
    for (int w = 0; w < STEP_THREADS / 64; ++w) x += acc[w][tid];
    x /= l;
    if constexpr (sizeof(T) == 2) o[tid] = f32_to_bf16(x);
    else o[tid] = x;
  }
}

static int step_checks(const std::string& w, const void* q, const void* k_new, const void* v_new,
                       const void* k_cache, const void* v_cache, const int32_t* kv_len,
                       const int32_t* cur_tok, const int32_t* vu, const int32_t* pos,
                       int32_t L_meta, const void* o, int32_t b, int32_t H, int32_t L_cap,
                       int32_t d_head, sckv_dtype dt, float scale, float rope_theta,
                       const void* ws) {
  if (!q || !k_new || !v_new || !k_cache || !v_cache || !kv_len || !cur_tok || !vu || !o || !ws)
    return fail(SCKV_EINVAL, w + ": null pointer");
  if (!valid_dtype(dt)) return fail(SCKV_EINVAL, w + ": unknown dtype");
  if (!supported_d(d_head)) return fail(SCKV_EUNSUP, w + ": d_head must be 64 or 80");
  if (b <= 0 || H <= 0 || L_cap <= 0 || L_meta <= 0)
    return fail(SCKV_EINVAL, w + ": sizes must be positive");
  if ((int64_t)b * H > 0x7fffffff) return fail(SCKV_EUNSUP, w + ": too many slices");
  if (!(scale > 0.f) || std::isinf(scale)) return fail(SCKV_EINVAL, w + ": scale must be finite and > 0");
  if (!(rope_theta >= 0.f) || std::isinf(rope_theta))
    return fail(SCKV_EINVAL, w + ": rope_theta must be finite and >= 0");
  if (rope_theta > 0.f && !pos) return fail(SCKV_EINVAL, w + ": null pos");
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) ||
      !aligned16(v_cache) || !aligned16(o) || !aligned16(ws))
    return fail(SCKV_EINVAL, w + ": buffers must be 16-byte aligned");
  return SCKV_OK;
}

template <typename T, int D>
static int launch_step(const void* q, const void* k_new, const void* v_new, const void* k_pre,
                       const void* v_pre, const int32_t* pre_len, int32_t per, int32_t P_cap,
                       void* k_cache, void* v_cache, const int32_t* kv_len,
                       const int32_t* cur_tok, const int32_t* vu, const int32_t* pos,
                       int32_t L_meta, void* o, const float* w_in, float* w_out, int32_t b,
                       int32_t H, int32_t L_cap, float scale, float theta, void* ws,
                       int32_t* status, const char* what, hipStream_t stream) {
  StepFreq tab;
  for (int i = 0; i < 40; ++i) tab.w[i] = 0.0;
  if (theta > 0.f)
    for (int i = 0; i < D / 2; ++i) tab.w[i] = std::pow((double)theta, -2.0 * i / D);
  StepArgs<T> a = {(const T*)q, (const T*)k_new, (const T*)v_new, (const T*)k_pre, (const T*)v_pre,
                   (T*)k_cache, (T*)v_cache, (T*)o, pre_len, kv_len, cur_tok, vu, pos, w_in, w_out,
                   (float*)ws, status, per, P_cap, L_meta, H, L_cap, theta > 0.f ? 1 : 0,
                   scale * 1.4426950408889634f};
  step_kernel<T, D><<<b * H, STEP_THREADS, 0, stream>>>(a, tab);
  return hip_check(hipGetLastError(), what);
}

}  // namespace sckv

using namespace sckv;

#define SCKV_STEP(T, D, KP, VP, PL, PER, PC, WI, WO, WHAT)                                         \
  launch_step<T, D>(q, k_new, v_new, KP, VP, PL, PER, PC, k_cache, v_cache, kv_len, cur_tok, vu,  \
                    pos, L_meta, o, WI, WO, b, H, L_cap, scale, rope_theta, ws, status, WHAT, stream)

extern "C" size_t sckv_decode_weights_workspace_bytes(int32_t b, int32_t H, int32_t L_cap,
                                                      int32_t d_head) {
  if (b <= 0 || H <= 0 || L_cap <= 0 || d_head <= 0) return 0;
  return (size_t)b * H * L_cap * sizeof(float);
}

extern "C" int compacted_decode_attn_weights(
    const void* q, const void* k_new, const void* v_new, void* k_cache, void* v_cache,
    const int32_t* kv_len, const int32_t* cur_tok, const int32_t* vu, const int32_t* pos,
    int32_t L_meta, void* o, const float* w_in, float* w_out, int32_t b, int32_t H, int32_t L_cap,
    int32_t d_head, sckv_dtype dt, float scale, float rope_theta, void* ws, size_t ws_bytes,
    int32_t* status, hipStream_t stream) {
  clear_error();
  const char* W = "compacted_decode_attn_weights";
  const int rc = step_checks(W, q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos, L_meta,
                             o, b, H, L_cap, d_head, dt, scale, rope_theta, ws);
  if (rc) return rc;
  if (!w_out) return fail(SCKV_EINVAL, std::string(W) + ": null pointer");
  if (!aligned4(w_out) || !aligned4(w_in))
    return fail(SCKV_EINVAL, std::string(W) + ": w_in and w_out must be 4-byte aligned");
  if (ws_bytes < sckv_decode_weights_workspace_bytes(b, H, L_cap, d_head))
    return fail(SCKV_EINVAL, std::string(W) + ": workspace too small");
  if (dt == SCKV_BF16)
    return d_head == 64 ? SCKV_STEP(uint16_t, 64, nullptr, nullptr, nullptr, 1, 0, w_in, w_out, W)
                        : SCKV_STEP(uint16_t, 80, nullptr, nullptr, nullptr, 1, 0, w_in, w_out, W);
  return d_head == 64 ? SCKV_STEP(float, 64, nullptr, nullptr, nullptr, 1, 0, w_in, w_out, W)
                      : SCKV_STEP(float, 80, nullptr, nullptr, nullptr, 1, 0, w_in, w_out, W);
}

extern "C" size_t sckv_shared_decode_workspace_bytes(int32_t b, int32_t H, int32_t n_prefix,
                                                     int32_t P_cap, int32_t L_cap,
                                                     int32_t d_head) {
  if (b <= 0 || H <= 0 || n_prefix <= 0 || P_cap <= 0 || L_cap <= 0 || d_head <= 0) return 0;
  return (size_t)b * H * ((size_t)P_cap + L_cap) * sizeof(float);
}

extern "C" int shared_prefix_decode_attn(
    const void* q, const void* k_new, const void* v_new, const void* k_prefix,
    const void* v_prefix, const int32_t* prefix_len, int32_t n_prefix, int32_t P_cap,
    void* k_cache, void* v_cache, const int32_t* kv_len, const int32_t* cur_tok,
    const int32_t* vu, const int32_t* pos, int32_t L_meta, void* o, int32_t b, int32_t H,
    int32_t L_cap, int32_t d_head, sckv_dtype dt, float scale, float rope_theta, void* ws,
    size_t ws_bytes, int32_t* status, hipStream_t stream) {
  clear_error();
  const char* W = "shared_prefix_decode_attn";
  const int rc = step_checks(W, q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos, L_meta,
                             o, b, H, L_cap, d_head, dt, scale, rope_theta, ws);
  if (rc) return rc;
  if (!k_prefix || !v_prefix || !prefix_len) return fail(SCKV_EINVAL, std::string(W) + ": null pointer");
  if (n_prefix <= 0 || P_cap <= 0 || b % n_prefix)
    return fail(SCKV_EINVAL, std::string(W) + ": b must be a multiple of n_prefix, sizes positive");
  if (!aligned16(k_prefix) || !aligned16(v_prefix))
    return fail(SCKV_EINVAL, std::string(W) + ": buffers must be 16-byte aligned");
  if (ws_bytes < sckv_shared_decode_workspace_bytes(b, H, n_prefix, P_cap, L_cap, d_head))
    return fail(SCKV_EINVAL, std::string(W) + ": workspace too small");
  const int per = b / n_prefix;
  if (dt == SCKV_BF16)
    return d_head == 64 ? SCKV_STEP(uint16_t, 64, k_prefix, v_prefix, prefix_len, per, P_cap, nullptr, nullptr, W)
                        : SCKV_STEP(uint16_t, 80, k_prefix, v_prefix, prefix_len, per, P_cap, nullptr, nullptr, W);
  return d_head == 64 ? SCKV_STEP(float, 64, k_prefix, v_prefix, prefix_len, per, P_cap, nullptr, nullptr, W)
                      : SCKV_STEP(float, 80, k_prefix, v_prefix, prefix_len, per, P_cap, nullptr, nullptr, W);
}
