// RMS norm of each head's queries and keys with the rotation at the tied
// positions in the same pass (rotary models: Section 4.1; the position tie:
// Section 3.1 "Input Transformation"):
//   y = x / sqrt(mean(x^2) + eps) * weight,
//   (y_i, y_{i+d/2}) turned by pos * theta^(-2i/d).
//
// Bound by HBM: a row is read and written once.  A thread owns one 16-byte
// piece of a row's first half and the matching piece of its second half, so
// both elements of a rotated pair are in one thread; the LANES threads of a
// row are neighbours and add up their squares by register moves.  The pair's
// angles are taken once and serve q and k of the HPT heads of the thread.
#include <cmath>

#include "sckv_common.h"

namespace sckv {

struct NormFreq {
  double w[40];  // theta^(-2i/d), i < d/2
};

template <typename T>
struct NormArgs {
  const T *q, *k, *v;
  T *q_out, *k_out, *v_out;
  const T *q_weight, *k_weight;
  int64_t xb, xh, xr, q_out_s, kv_s;
  const int32_t *pos, *cur_tok, *row0;
  int32_t* status;
  float eps;
  int32_t H, n, kv_rows, L_meta, tok0, rotate;
  int32_t n_hg, rows;  // groups of heads; (sequence, group, token) rows
  FastDiv by_n, by_hg;
};

// sum over the LANES neighbouring lanes that share a row
template <int LANES>
__device__ __forceinline__ float row_sum(float x, int lane) {
  if constexpr (LANES == 4 || LANES == 8) {
    x += dpp_mov<DPP_QUAD_XOR1>(x);
    x += dpp_mov<DPP_QUAD_XOR2>(x);
    if constexpr (LANES == 8) x += dpp_mov<DPP_ROW_HALF_MIRROR>(x);
    return x;
  } else {
    const int first = lane / LANES * LANES;
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < LANES; ++j) s += __shfl(x, (first + j) & 63, 64);
    return s;
  }
}

constexpr int NORM_THREADS = 256;

template <typename T, int D, int HPT>
__global__ __launch_bounds__(NORM_THREADS) void norm_rope_kernel(NormArgs<T> a, NormFreq tab) {
  constexpr int E = Piece<T>::E;
  constexpr int HALF = D / 2;
  constexpr int LANES = HALF / E;    // threads of a row
  constexpr int RPW = 64 / LANES;    // rows of a wave (its last lanes may be idle)
  static_assert(HALF % E == 0, "half a row is whole pieces");
  const int lane = threadIdx.x & 63;
  const int p = lane % LANES;
  const int64_t row = ((int64_t)blockIdx.x * (NORM_THREADS / 64) + (threadIdx.x >> 6)) * RPW + lane / LANES;
  const bool live = lane < RPW * LANES && row < a.rows;
  const int r = live ? (int)row : 0;
  const int sg = fast_div(r, a.by_n);
  const int t = r - sg * a.n;
  const int s = fast_div(sg, a.by_hg);
  const int h0 = (sg - s * a.n_hg) * HPT;

  // the row's token, its position, and where its key and value go
  const int64_t tok = (int64_t)(a.cur_tok ? a.cur_tok[s] : a.tok0) + t;
  const bool tok_ok = !a.cur_tok || (tok >= 0 && tok < a.L_meta);
  const int r0 = a.row0 ? a.row0[s] : 0;
  const bool kv_ok = r0 >= 0 && (int64_t)r0 + a.n <= a.kv_rows;
  if (live && h0 == 0 && p == 0 && a.status) {
    if (!tok_ok) atomicOr(a.status, SCKV_STATUS_TOKEN);
    if (!kv_ok && t == 0 && (a.k || a.v)) atomicOr(a.status, SCKV_STATUS_CAP);
  }
  float cs[E], sn[E];
  if (a.rotate) {
    const double two_pi = 6.283185307179586476925286766559;
    const double inv_two_pi = 0.15915494309189533576888376337251;
    const double ps = tok_ok ? (double)a.pos[(int64_t)s * a.L_meta + tok] : 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      double ang = ps * tab.w[p * E + e];
      ang -= two_pi * rint(ang * inv_two_pi);
      float si, co;
      sincosf((float)ang, &si, &co);
      sn[e] = si;
      cs[e] = co;
    }
  }
  const int64_t xo = s * a.xb + t * a.xr + p * E;
  const int64_t qo = (int64_t)s * a.H * a.q_out_s + (int64_t)t * D + p * E;
  const int64_t ko = (int64_t)s * a.H * a.kv_s + ((int64_t)r0 + t) * D + p * E;

  auto turn = [&](u32x4& lo, u32x4& hi, const float* wl, const float* wh) {
    float x1[E], x2[E], sq = 0.f;
    Piece<T>::unpack(lo, x1);
    Piece<T>::unpack(hi, x2);
#pragma unroll
    for (int e = 0; e < E; ++e) sq = fmaf(x2[e], x2[e], fmaf(x1[e], x1[e], sq));
    const float rms = 1.f / sqrtf(row_sum<LANES>(sq, lane) * (1.f / D) + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x1[e] *= rms * wl[e];
      x2[e] *= rms * wh[e];
    }
    if (a.rotate) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float y1 = fmaf(x1[e], cs[e], -(x2[e] * sn[e]));
        x2[e] = fmaf(x2[e], cs[e], x1[e] * sn[e]);
        x1[e] = y1;
      }
    }
    if (!tok_ok) {
#pragma unroll
      for (int e = 0; e < E; ++e) x1[e] = x2[e] = __builtin_nanf("");
    }
    lo = Piece<T>::pack(x1);
    hi = Piece<T>::pack(x2);
  };
  float qwl[E], qwh[E], kwl[E], kwh[E];
#pragma unroll
  for (int e = 0; e < E; ++e) qwl[e] = qwh[e] = kwl[e] = kwh[e] = 1.f;
  if (a.q_weight) {
    Piece<T>::unpack(ld16(a.q_weight + p * E), qwl);
    Piece<T>::unpack(ld16(a.q_weight + HALF + p * E), qwh);
  }
  if (a.k_weight) {
    Piece<T>::unpack(ld16(a.k_weight + p * E), kwl);
    Piece<T>::unpack(ld16(a.k_weight + HALF + p * E), kwh);
  }
  const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const int h = h0 + i;
    const bool on = live && h < a.H;
    const int64_t x = xo + h * a.xh;
    u32x4 ql = zero, qh = zero, kl = zero, kh = zero, vl = zero, vh = zero;
    if (on) {
      if (a.q) { ql = ld16(a.q + x); qh = ld16(a.q + x + HALF); }
      if (a.k) { kl = ld16(a.k + x); kh = ld16(a.k + x + HALF); }
      if (a.v) { vl = ld16(a.v + x); vh = ld16(a.v + x + HALF); }
    }
    if (a.q) {
      turn(ql, qh, qwl, qwh);
      if (on) {
        st16(a.q_out + qo + h * a.q_out_s, ql);
        st16(a.q_out + qo + h * a.q_out_s + HALF, qh);
      }
    }
    if (a.k) {
      turn(kl, kh, kwl, kwh);
      if (on && kv_ok) {
        st16(a.k_out + ko + h * a.kv_s, kl);
        st16(a.k_out + ko + h * a.kv_s + HALF, kh);
      }
    }
    if (a.v && on && kv_ok) {
      st16(a.v_out + ko + h * a.kv_s, vl);
      st16(a.v_out + ko + h * a.kv_s + HALF, vh);
    }
  }
}

template <typename T, int D, int HPT>
static int launch_norm(NormArgs<T> a, int32_t b, const NormFreq& tab, hipStream_t stream) {
  constexpr int RPB = NORM_THREADS / 64 * (64 / (D / 2 / Piece<T>::E));
  a.n_hg = (a.H + HPT - 1) / HPT;
  const int64_t rows = (int64_t)b * a.n_hg * a.n;
  if (rows > 0x7fffffff) return fail(SCKV_EUNSUP, "qk_norm_rope: too many rows");
  a.rows = (int32_t)rows;
  a.by_n = make_div((uint32_t)a.n);
  a.by_hg = make_div((uint32_t)a.n_hg);
  norm_rope_kernel<T, D, HPT><<<(unsigned)((rows + RPB - 1) / RPB), NORM_THREADS, 0, stream>>>(a, tab);
  return hip_check(hipGetLastError(), "qk_norm_rope: launch");
}

template <typename T, int D>
static int norm_typed(NormArgs<T> a, const void* q, const void* k, const void* v, void* q_out,
                      void* k_out, void* v_out, const void* q_weight, const void* k_weight,
                      int32_t b, float theta, hipStream_t stream) {
  a.q = static_cast<const T*>(q);
  a.k = static_cast<const T*>(k);
  a.v = static_cast<const T*>(v);
  a.q_out = static_cast<T*>(q_out);
  a.k_out = static_cast<T*>(k_out);
  a.v_out = static_cast<T*>(v_out);
  a.q_weight = static_cast<const T*>(q_weight);
  a.k_weight = static_cast<const T*>(k_weight);
  NormFreq tab;
  for (int i = 0; i < 40; ++i) tab.w[i] = 0.0;
  if (a.rotate)
    for (int i = 0; i < D / 2; ++i) tab.w[i] = std::pow((double)theta, -2.0 * i / D);
  return launch_norm<T, D, 1>(a, b, tab, stream);
}

}  // namespace sckv

using namespace sckv;

extern "C" int qk_norm_rope(const void* q, const void* k, const void* v, void* q_out, void* k_out,
                            void* v_out, const void* q_weight, const void* k_weight, float eps,
                            int32_t b, int32_t H, int32_t n, int64_t x_stride_b,
                            int64_t x_stride_h, int64_t x_stride_row, int64_t q_out_stride_bh,
                            int64_t kv_stride_bh, int32_t kv_rows, int32_t d_head, sckv_dtype dt,
                            const int32_t* pos, int32_t L_meta, int32_t tok0,
                            const int32_t* cur_tok, const int32_t* row0, float theta,
                            int32_t* status, hipStream_t stream) {
  clear_error();
  if ((!q && !k && !v) || !q != !q_out || !k != !k_out || !v != !v_out)
    return fail(SCKV_EINVAL, "qk_norm_rope: q, k and v each go with their output, and one is needed");
  if (!valid_dtype(dt)) return fail(SCKV_EINVAL, "qk_norm_rope: unknown dtype");
  if (!supported_d(d_head)) return fail(SCKV_EUNSUP, "qk_norm_rope: d_head must be 64 or 80");
  if (b <= 0 || H <= 0 || n < 0) return fail(SCKV_EINVAL, "qk_norm_rope: bad sizes");
  if (!(eps > 0.f) || std::isinf(eps)) return fail(SCKV_EINVAL, "qk_norm_rope: eps must be finite and > 0");
  if (x_stride_b < 0 || x_stride_h < 0 || x_stride_row < 0)
    return fail(SCKV_EINVAL, "qk_norm_rope: negative stride");
  if (q && q_out_stride_bh < (int64_t)n * d_head)
    return fail(SCKV_EINVAL, "qk_norm_rope: q_out slice smaller than its rows");
  if ((k || v) && (kv_rows < n || kv_stride_bh < (int64_t)kv_rows * d_head))
    return fail(SCKV_EINVAL, "qk_norm_rope: k_out or v_out slice smaller than its rows");
  if (!(theta >= 0.f) || std::isinf(theta))
    return fail(SCKV_EINVAL, "qk_norm_rope: theta must be finite and >= 0");
  if (theta > 0.f && !pos) return fail(SCKV_EINVAL, "qk_norm_rope: null pos");
  if (theta > 0.f || cur_tok) {
    if (L_meta <= 0 || (!cur_tok && (tok0 < 0 || (int64_t)tok0 + n > L_meta)))
      return fail(SCKV_EINVAL, "qk_norm_rope: rows [tok0, tok0+n) exceed L_meta");
  }
  const int64_t eb = elem_bytes(dt);
  const void* all[] = {q, k, v, q_out, k_out, v_out, q_weight, k_weight};
  for (const void* p : all)
    if (p && !aligned16(p)) return fail(SCKV_EINVAL, "qk_norm_rope: buffers must be 16-byte aligned");
  // (a dimension of one is never stepped over)
  if ((b > 1 && x_stride_b * eb % 16) || (H > 1 && x_stride_h * eb % 16) ||
      (n > 1 && x_stride_row * eb % 16) || (q && q_out_stride_bh * eb % 16) ||
      ((k || v) && kv_stride_bh * eb % 16))
    return fail(SCKV_EINVAL, "qk_norm_rope: strides must be multiples of 16 bytes");
  if (n == 0) return SCKV_OK;
  auto go = [&](auto a) {
    using T = std::remove_const_t<std::remove_pointer_t<decltype(a.q)>>;
    a.xb = x_stride_b;
    a.xh = x_stride_h;
    a.xr = x_stride_row;
    a.q_out_s = q_out_stride_bh;
    a.kv_s = kv_stride_bh;
    a.pos = pos;
    a.cur_tok = cur_tok;
    a.row0 = row0;
    a.status = status;
    a.eps = eps;
    a.H = H;
    a.n = n;
    a.kv_rows = (k || v) ? kv_rows : n;
    a.L_meta = L_meta;
    a.tok0 = tok0;
    a.rotate = theta > 0.f ? 1 : 0;
    return d_head == 64 ? norm_typed<T, 64>(a, q, k, v, q_out, k_out, v_out, q_weight, k_weight, b, theta, stream)
                        : norm_typed<T, 80>(a, q, k, v, q_out, k_out, v_out, q_weight, k_weight, b, theta, stream);
  };
  return dt == SCKV_BF16 ? go(NormArgs<uint16_t>()) : go(NormArgs<float>());
}
