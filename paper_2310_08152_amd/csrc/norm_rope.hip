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
// angles are taken once and serve the HPT heads of the thread.
#include <cmath>

#include "sckv_common.h"

namespace sckv {

struct NormFreq {
  double w[40];  // theta^(-2i/d), i < d/2
};

template <typename T>
struct NormArgs {
  const T* x[3];  // those of q, k and v that are given, in this order
  T* y[3];
  const T* weight[3];
  int64_t y_stride[3];
  int32_t kind[3];  // 0 q, 1 k, 2 v
  int64_t xb, xh, xr;
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
constexpr int NORM_SMALL = 2048;   // waves (a head a thread) that fill the SIMDs twice
constexpr int NORM_LARGE = 32768;  // 32 a SIMD

// Shapes, measured on token-major bf16 inputs, 32 heads of 80, us:
//   NZ = 3, HPT = 4 (a thread takes its heads' q, k and v): large launches,
//     16 x 4096 tokens 428 (4.7 TB/s) against 449 with a tensor a workgroup;
//     8 x 1024 47 against 44.
//   NZ = 1 (blockIdx.y picks the tensor), HPT = 4: from NORM_SMALL waves on;
//     HPT = 1 gives 70 at 8 x 1024, its angles taken for one row each.
//   NZ = 1, HPT = 1: the fewest rows a thread, one token's step 4.1 against 5.6.
// fp32 pieces hold 4 elements, so angles weigh half: NZ = 3 with HPT = 2 (16 x
// 1024 tokens 195, with a tensor a workgroup 204).
template <typename T, int D, int HPT, int NZ>
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

  // the tensors of this thread (all three, or one), their pieces and weights;
  // offsets are shared by those that share strides
  int kind[NZ];
  const T* from[NZ];
  u32x4 lo[NZ], hi[NZ], lo1[NZ], hi1[NZ], wlo[NZ], whi[NZ];
  bool weighed[NZ];
  int64_t xo = s * a.xb + h0 * a.xh + t * a.xr + p * E;
#pragma unroll
  for (int z = 0; z < NZ; ++z) {
    const int i = NZ == 1 ? (int)blockIdx.y : z;
    kind[z] = NZ == 3 ? z : i == 0 ? a.kind[0] : i == 1 ? a.kind[1] : a.kind[2];
    from[z] = i == 0 ? a.x[0] : i == 1 ? a.x[1] : a.x[2];
    lo[z] = hi[z] = lo1[z] = hi1[z] = wlo[z] = whi[z] = u32x4{0, 0, 0, 0};
    if (live) {
      lo[z] = ld16(from[z] + xo);
      hi[z] = ld16(from[z] + xo + HALF);
    }
    const T* w = i == 0 ? a.weight[0] : i == 1 ? a.weight[1] : a.weight[2];
    weighed[z] = w != nullptr;
    if (weighed[z]) {
      wlo[z] = ld16(w + p * E);
      whi[z] = ld16(w + HALF + p * E);
    }
  }
  // the row's token, its position, and where it goes
  const int64_t tok = (int64_t)(a.cur_tok ? a.cur_tok[s] : a.tok0) + t;
  const bool tok_ok = !a.cur_tok || (tok >= 0 && tok < a.L_meta);
  const int r0 = a.row0 ? a.row0[s] : 0;
  const bool room = r0 >= 0 && (int64_t)r0 + a.n <= a.kv_rows;
  bool turns = false, caches = false;
  T* to[NZ];
  int64_t ys[NZ], yo[NZ];  // (k and v: the same stride and offset)
#pragma unroll
  for (int z = 0; z < NZ; ++z) {
    const int i = NZ == 1 ? (int)blockIdx.y : z;
    turns = turns || kind[z] < 2;
    caches = caches || kind[z] > 0;
    to[z] = i == 0 ? a.y[0] : i == 1 ? a.y[1] : a.y[2];
    if (z == 2) {
      ys[z] = ys[1];
      yo[z] = yo[1];
    } else {
      ys[z] = i == 0 ? a.y_stride[0] : i == 1 ? a.y_stride[1] : a.y_stride[2];
      yo[z] = ((int64_t)s * a.H + h0) * ys[z] + ((int64_t)(kind[z] > 0 ? r0 : 0) + t) * D + p * E;
    }
  }
  if (live && h0 == 0 && p == 0 && a.status) {
    if (turns && !tok_ok) atomicOr(a.status, SCKV_STATUS_TOKEN);
    if (caches && !room && t == 0) atomicOr(a.status, SCKV_STATUS_CAP);
  }
  float cs[E], sn[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
  }
  const bool turned = turns && a.rotate;
  if (turned) {
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
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const bool on = live && h0 + i < a.H;
    // the next head's pieces are in flight while this one is computed
    if (i + 1 < HPT && live && h0 + i + 1 < a.H) {
      xo += a.xh;
#pragma unroll
      for (int z = 0; z < NZ; ++z) {
        lo1[z] = ld16(from[z] + xo);
        hi1[z] = ld16(from[z] + xo + HALF);
      }
    }
#pragma unroll
    for (int z = 0; z < NZ; ++z) {
      if (kind[z] < 2) {
        float x1[E], x2[E], w1[E], w2[E], sq = 0.f;
        Piece<T>::unpack(lo[z], x1);
        Piece<T>::unpack(hi[z], x2);
#pragma unroll
        for (int e = 0; e < E; ++e) sq = fmaf(x2[e], x2[e], fmaf(x1[e], x1[e], sq));
        const float rms = 1.f / sqrtf(row_sum<LANES>(sq, lane) * (1.f / D) + a.eps);
        if (weighed[z]) {
          Piece<T>::unpack(wlo[z], w1);
          Piece<T>::unpack(whi[z], w2);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            x1[e] *= rms * w1[e];
            x2[e] *= rms * w2[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            x1[e] *= rms;
            x2[e] *= rms;
          }
        }
        if (turned) {
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
        lo[z] = Piece<T>::pack(x1);
        hi[z] = Piece<T>::pack(x2);
      }
      if (on && (kind[z] == 0 || room)) {
        st16(to[z] + yo[z], lo[z]);
        st16(to[z] + yo[z] + HALF, hi[z]);
      }
      yo[z] += ys[z];
      lo[z] = lo1[z];
      hi[z] = hi1[z];
    }
  }
}

template <typename T, int D, int HPT, int NZ>
static int launch_norm(NormArgs<T> a, int32_t b, int count, const NormFreq& tab, hipStream_t stream) {
  constexpr int RPB = NORM_THREADS / 64 * (64 / (D / 2 / Piece<T>::E));
  a.n_hg = (a.H + HPT - 1) / HPT;
  const int64_t rows = (int64_t)b * a.n_hg * a.n;
  if (rows > 0x7fffffff) return fail(SCKV_EUNSUP, "qk_norm_rope: too many rows");
  a.rows = (int32_t)rows;
  a.by_n = make_div((uint32_t)a.n);
  a.by_hg = make_div((uint32_t)a.n_hg);
  const dim3 grid((unsigned)((rows + RPB - 1) / RPB), NZ == 1 ? (unsigned)count : 1u);
  norm_rope_kernel<T, D, HPT, NZ><<<grid, NORM_THREADS, 0, stream>>>(a, tab);
  return hip_check(hipGetLastError(), "qk_norm_rope: launch");
}

template <typename T, int D>
static int norm_typed(NormArgs<T> a, int32_t b, int count, float theta, hipStream_t stream) {
  NormFreq tab;
  for (int i = 0; i < 40; ++i) tab.w[i] = 0.0;
  if (a.rotate)
    for (int i = 0; i < D / 2; ++i) tab.w[i] = std::pow((double)theta, -2.0 * i / D);
  // waves of one tensor with a head a thread
  constexpr int RPW = 64 / (D / 2 / Piece<T>::E);
  const int64_t waves = ((int64_t)b * a.H * a.n + RPW - 1) / RPW;
  if (waves < NORM_SMALL) return launch_norm<T, D, 1, 1>(a, b, count, tab, stream);
  if (count < 3 || waves < NORM_LARGE) return launch_norm<T, D, 4, 1>(a, b, count, tab, stream);
  return launch_norm<T, D, sizeof(T) == 2 ? 4 : 2, 3>(a, b, count, tab, stream);
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
    using E = std::remove_pointer_t<decltype(+a.y[0])>;
    const void* xs[3] = {q, k, v};
    void* ys[3] = {q_out, k_out, v_out};
    const void* ws[3] = {q_weight, k_weight, nullptr};
    int count = 0;
    for (int i = 0; i < 3; ++i) {
      a.x[i] = nullptr;
      a.y[i] = nullptr;
      a.weight[i] = nullptr;
      a.y_stride[i] = 0;
      a.kind[i] = -1;
    }
    for (int i = 0; i < 3; ++i) {
      if (!xs[i]) continue;
      a.x[count] = static_cast<const E*>(xs[i]);
      a.y[count] = static_cast<E*>(ys[i]);
      a.weight[count] = static_cast<const E*>(ws[i]);
      a.y_stride[count] = i == 0 ? q_out_stride_bh : kv_stride_bh;
      a.kind[count++] = i;
    }
    a.xb = x_stride_b;
    a.xh = x_stride_h;
    a.xr = x_stride_row;
    a.pos = pos;
    a.cur_tok = cur_tok;
    a.row0 = row0;
    a.status = status;
    a.eps = eps;
    a.H = H;
    a.n = n;
    a.kv_rows = kv_rows;
    a.L_meta = L_meta;
    a.tok0 = tok0;
    a.rotate = theta > 0.f ? 1 : 0;
    return d_head == 64 ? norm_typed<E, 64>(a, b, count, theta, stream)
                        : norm_typed<E, 80>(a, b, count, theta, stream);
  };
  return dt == SCKV_BF16 ? go(NormArgs<uint16_t>()) : go(NormArgs<float>());
}
