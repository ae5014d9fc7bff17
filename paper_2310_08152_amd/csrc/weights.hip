// Accumulated attention weight of cache rows (what eviction goes by): the sum
// over queries of the softmax weight that each gives a row, under the mask of
// Section 3.1.
//
//   w[r] += sum_i exp2(c q_i.k_r - lse_i),  lse_i = log2 sum_r exp2(c q_i.k_r)
//
// with c = scale * log2(e).  Two passes over the scores, since a row's sum
// needs every query's normaliser first: stats takes each query's maximum and
// sum, sums adds up the weights of each row.  A <CL> query gives its own row
// weight 1; its lse is +inf, so that it gives the others exactly 0.
#include <cmath>

#include "sckv_common.h"

namespace sckv {

constexpr float W_LOG2E = 1.4426950408889634f;

template <typename T>
__device__ __forceinline__ float elem(const T* p, int i) {
  if constexpr (sizeof(T) == 2) return bf16_lo((uint32_t)p[i]);
  else return p[i];
}

template <typename T, int D>
__device__ __forceinline__ float row_dot(const T* __restrict__ k, const float* q) {
  constexpr int E = Piece<T>::E;
  float d = 0.f;
#pragma unroll
  for (int p = 0; p < D / E; ++p) {
    float f[E];
    Piece<T>::unpack(ld16(k + p * E), f);
#pragma unroll
    for (int e = 0; e < E; ++e) d = fmaf(f[e], q[p * E + e], d);
  }
  return d;
}

// one wave per (query, slice)
template <typename T, int D>
__global__ __launch_bounds__(64) void weight_stats_kernel(
    const T* __restrict__ q, const T* __restrict__ k, float* __restrict__ lse, int32_t b,
    int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float c, const int32_t* __restrict__ vu,
    int32_t L_meta, int32_t tok0, const int32_t* __restrict__ kv_len,
    const int32_t* __restrict__ tok_idx, int32_t L_cap) {
  __shared__ float qs[D];
  const int i = blockIdx.x;
  const int lane = threadIdx.x;
  for (int bh = blockIdx.y; bh < b * H; bh += gridDim.y) {
    const int s = bh / H;
    const int n = min(max(kv_len[s], 0), L_cap);
    const int t = tok0 + i;
    const int32_t* vus = vu + (int64_t)s * L_meta;
    __syncthreads();
    for (int e = lane; e < D; e += 64) qs[e] = elem(q + bh * q_s + (int64_t)i * D, e) * c;
    __syncthreads();
    float m = -INFINITY, l = 0.f;
    if (vus[t] != t)
      for (int r = lane; r < n; r += 64) {
        const int j = tok_idx[(int64_t)s * L_cap + r];
        if (j < 0 || j > t || vus[j] < t) continue;
        const float x = row_dot<T, D>(k + bh * k_s + (int64_t)r * D, qs);
        const float mn = fmaxf(m, x);
        l = l * exp2f(m - mn) + exp2f(x - mn);
        m = mn;
      }
    const float M = wave_max(m);
    l = wave_sum(m == -INFINITY ? 0.f : l * exp2f(m - M));
    if (lane == 0) lse[(int64_t)bh * nq + i] = M == -INFINITY ? INFINITY : M + log2f(l);
  }
}

// one thread per (row, slice)
template <typename T, int D>
__global__ __launch_bounds__(64) void weight_sums_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const float* __restrict__ lse,
    const float* w_in, float* w_out, int32_t b, int32_t H, int32_t nq, int64_t q_s, int64_t k_s,
    float c, const int32_t* __restrict__ vu, int32_t L_meta, int32_t tok0,
    const int32_t* __restrict__ kv_len, const int32_t* __restrict__ tok_idx, int32_t L_cap) {
  const int r = blockIdx.x * 64 + threadIdx.x;
  for (int bh = blockIdx.y; bh < b * H; bh += gridDim.y) {
    const int s = bh / H;
    const int n = min(max(kv_len[s], 0), L_cap);
    if (r >= n) continue;
    const int64_t at = (int64_t)bh * L_cap + r;
    float sum = 0.f;
    const int j = tok_idx[(int64_t)s * L_cap + r];
    const int v = j >= 0 && j < L_meta ? vu[(int64_t)s * L_meta + j] : -1;
    if (v == j && j >= tok0 && j < tok0 + nq) {
      sum = 1.f;
    } else if (v >= 0) {
      float kf[D];
#pragma unroll
      for (int e = 0; e < D; ++e) kf[e] = elem(k + bh * k_s + (int64_t)r * D, e) * c;
      const int i1 = min((int64_t)nq, (int64_t)v - tok0 + 1);
      for (int i = max(0, j - tok0); i < i1; ++i)
        sum += exp2f(row_dot<T, D>(q + bh * q_s + (int64_t)i * D, kf) - lse[(int64_t)bh * nq + i]);
    }
    w_out[at] = (w_in ? w_in[at] : 0.f) + sum;
  }
}

template <typename T, int D>
static int launch_weights(const void* q, const void* k, const float* w_in, float* w_out, int32_t b,
                          int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float scale,
                          const int32_t* vu, int32_t L_meta, int32_t tok0, const int32_t* kv_len,
                          const int32_t* tok_idx, int32_t L_cap, void* ws, hipStream_t stream) {
  const T* qq = static_cast<const T*>(q);
  const T* kk = static_cast<const T*>(k);
  float* lse = static_cast<float*>(ws);
  const unsigned y = (unsigned)(b * H < 65535 ? b * H : 65535);
  if (nq > 0) {
    weight_stats_kernel<T, D><<<dim3(nq, y), 64, 0, stream>>>(
        qq, kk, lse, b, H, nq, q_s, k_s, scale * W_LOG2E, vu, L_meta, tok0, kv_len, tok_idx, L_cap);
    const int rc = hip_check(hipGetLastError(), "cached_attn_weights: stats launch");
    if (rc) return rc;
  }
  weight_sums_kernel<T, D><<<dim3((L_cap + 63) / 64, y), 64, 0, stream>>>(
      qq, kk, lse, w_in, w_out, b, H, nq, q_s, k_s, scale * W_LOG2E, vu, L_meta, tok0, kv_len,
      tok_idx, L_cap);
  return hip_check(hipGetLastError(), "cached_attn_weights: sums launch");
}

}  // namespace sckv

using namespace sckv;

extern "C" size_t sckv_attn_weights_workspace_bytes(int32_t b, int32_t H, int32_t nq,
                                                    int32_t L_cap) {
  if (b <= 0 || H <= 0 || nq < 0 || L_cap <= 0) return 0;
  return (size_t)b * H * (nq > 0 ? nq : 1) * sizeof(float);
}

extern "C" int cached_attn_weights(const void* q, const void* k_cache, const float* w_in,
                                   float* w_out, int32_t b, int32_t H, int32_t nq, int32_t d_head,
                                   int64_t q_stride_bh, int64_t kv_stride_bh, sckv_dtype dt,
                                   float scale, const int32_t* vu, int32_t L_meta, int32_t tok0,
                                   const int32_t* kv_len, const int32_t* tok_idx, int32_t L_cap,
                                   void* ws, size_t ws_bytes, hipStream_t stream) {
  clear_error();
  if ((!q && nq != 0) || !k_cache || !w_out || !vu || !kv_len || !tok_idx || !ws)
    return fail(SCKV_EINVAL, "cached_attn_weights: null pointer");
  if (!valid_dtype(dt)) return fail(SCKV_EINVAL, "cached_attn_weights: unknown dtype");
  if (!supported_d(d_head)) return fail(SCKV_EUNSUP, "cached_attn_weights: d_head must be 64 or 80");
  if (b <= 0 || H <= 0 || L_cap <= 0 || L_meta <= 0 || nq < 0)
    return fail(SCKV_EINVAL, "cached_attn_weights: bad sizes");
  if (nq > 65536 || L_cap > 65536)
    return fail(SCKV_EUNSUP, "cached_attn_weights: nq or L_cap above 65536");
  if ((int64_t)b * H > 0x7fffffff) return fail(SCKV_EUNSUP, "cached_attn_weights: too many slices");
  if (tok0 < 0 || (int64_t)tok0 + nq > L_meta)
    return fail(SCKV_EINVAL, "cached_attn_weights: tokens [tok0, tok0+nq) exceed L_meta");
  if (q_stride_bh < (int64_t)nq * d_head || kv_stride_bh < (int64_t)L_cap * d_head)
    return fail(SCKV_EINVAL, "cached_attn_weights: slice stride smaller than its rows");
  if (!(scale > 0.f) || std::isinf(scale))
    return fail(SCKV_EINVAL, "cached_attn_weights: scale must be finite and > 0");
  if (ws_bytes < sckv_attn_weights_workspace_bytes(b, H, nq, L_cap))
    return fail(SCKV_EINVAL, "cached_attn_weights: workspace too small");
  if (!aligned16(q) || !aligned16(k_cache) || !aligned4(w_out) || !aligned4(w_in) ||
      !aligned16(ws) || q_stride_bh * elem_bytes(dt) % 16 || kv_stride_bh * elem_bytes(dt) % 16)
    return fail(SCKV_EINVAL, "cached_attn_weights: buffers and strides must be 16-byte aligned");
#define SCKV_WEIGHTS(T, D)                                                                        \
  launch_weights<T, D>(q, k_cache, w_in, w_out, b, H, nq, q_stride_bh, kv_stride_bh, scale, vu,   \
                       L_meta, tok0, kv_len, tok_idx, L_cap, ws, stream)
  if (dt == SCKV_BF16)
    return d_head == 64 ? SCKV_WEIGHTS(uint16_t, 64) : SCKV_WEIGHTS(uint16_t, 80);
  return d_head == 64 ? SCKV_WEIGHTS(float, 64) : SCKV_WEIGHTS(float, 80);
#undef SCKV_WEIGHTS
}
