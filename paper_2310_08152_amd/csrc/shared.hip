// Attention of decode steps over a prefix that several sequences share
// (several samples for one compressed document: Section 4.2), the part that
// reads the prefix: each of its rows once for all of its sequences.
//
// Per (prefix, head) the queries of its sequences form a matrix, so the scores
// S^T = K Q^T and the outputs O^T += V^T P^T are products on the matrix cores.
// A wave takes a tile of 32 queries (or two) and 32-row blocks of keys; lane l owns
// query l % 32 of S^T (16 of the block's 32 rows: 8a + 4(l/32) + c), hence the
// running maximum and sum of a softmax in registers, and the same rows of P^T
// are the B operand of the value product as they stand.  bf16 queries (after
// the rotation) and softmax weights are carried as two bf16 terms each (2^-17
// of them), so that a shared step is as exact as a decode step, which weighs
// in fp32; weights of one term cost half a step of the output's own type and
// saved 2% (64 sequences behind 12288 rows) or nothing (32 and fewer, bound by
// HBM).
//
// Bound by HBM while a tile of queries is not much larger than the card's
// flops per byte; the workgroup's four key waves split its rows, and the rows
// are split over workgroups (chunks) until the launch fills the CUs.  Each
// chunk leaves one partial (maximum, sum, output) a query, which the step over
// the sequences' own rows joins to its own at its end (decode.hip): two
// launches a step.
#include <algorithm>
#include <cmath>
#include <string>

#include "sckv_common.h"

namespace sckv {

constexpr int PRE_ROWS = 32;     // rows of a block
constexpr int PRE_QUERIES = 32;  // queries of a tile
constexpr int PRE_KEY_WAVES = 4;
constexpr float PRE_RESCALE = 8.f;  // lazy maximum, log2 units

struct PrefixFreq {
  double w[40];  // theta^(-2i/d)
};

// The 16 scores and weights of a lane, the wave's tile of queries and its
// outputs.  DB blocks of 32 output elements; in each, register v of lane l
// holds element 8 (v/4) + 4 (l/32) + v % 4 of query l % 32.
template <typename T, int D, int QT>
struct PrefixTile {
  static constexpr int DB = (D + 31) / 32;
  static constexpr int KS = D / 16;
  static constexpr int PITCH = 192;  // bytes of a value row in LDS: the transposing
                                     // reads' 8 rows x 64 bytes then meet no bank twice
  static constexpr int V_BYTES = sizeof(T) == 2 ? PRE_ROWS * PITCH : 0;
  static constexpr int NK = sizeof(T) == 2 ? KS : D / 8;   // 16-byte pieces of a key row per lane
  // A block's rows in registers, loaded a block ahead.  bf16 values pass
  // through LDS at the start of their block's step, so one set of them (`v`) is
  // enough, refilled at once.
  struct Rows {
    u32x4 k[NK];
    float v[sizeof(T) == 2 ? 1 : 16 * DB];
  };
  u32x4 v[sizeof(T) == 2 ? KS : 1];
  bf16x8 qhi[QT][sizeof(T) == 2 ? KS : 1], qlo[QT][sizeof(T) == 2 ? KS : 1];
  float qf[QT][sizeof(T) == 2 ? 1 : D / 2];
  f32x16 o[QT][DB];
  float M[QT], l[QT];

  // the lane's query of tile x, row `q` of D floats in LDS
  __device__ __forceinline__ void take_query(int x, const float* q, int h) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        u32x4 wh, wl;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = q[16 * kk + 8 * h + 2 * i], x1 = q[16 * kk + 8 * h + 2 * i + 1];
          wh[i] = pack_bf16x2(x0, x1);
          wl[i] = pack_bf16x2(x0 - bf16_lo(wh[i]), x1 - bf16_hi(wh[i]));
        }
        qhi[x][kk] = __builtin_bit_cast(bf16x8, wh);
        qlo[x][kk] = __builtin_bit_cast(bf16x8, wl);
      }
    } else {
#pragma unroll
      for (int p = 0; p < D / 8; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j) qf[x][4 * p + j] = q[8 * p + 4 * h + j];
    }
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[x][b][v] = 0.f;
    M[x] = -INFINITY;
    l[x] = 0.f;
  }

  // Rows r .. r + 31 of a slice (those past `last` read row `last`).  bf16:
  // pieces 16 kk + 8 h of the lane's row l % 32 of both.  fp32: pieces 2p + h
  // of the key row; of the values what the A operands of 32x32x2 take, element
  // 32 b + l % 32 of row 8a + 4h + c.
  __device__ __forceinline__ static void load(Rows& x, const T* kb, const T* vb, int r, int last,
                                              int lane) {
    const int h = lane >> 5;
    const int64_t row = min(r + (lane & 31), last);
    if constexpr (sizeof(T) == 2) {
      const T* kp = kb + row * D + 8 * h;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) x.k[kk] = ld16(kp + 16 * kk);
    } else {
      const T* kp = kb + row * D + 4 * h;
#pragma unroll
      for (int p = 0; p < D / 8; ++p) x.k[p] = ld16(kp + 8 * p);
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const T* vp = vb + (int64_t)min(r + 8 * (v / 4) + 4 * h + v % 4, last) * D;
#pragma unroll
        for (int b = 0; b < DB; ++b)  // (elements past the head size are never stored)
          x.v[v * DB + b] = vp[min(32 * b + (lane & 31), D - 1)];
      }
    }
  }
  __device__ __forceinline__ void load_values(const T* vb, int r, int last, int lane) {
    if constexpr (sizeof(T) == 2) {
      const T* vp = vb + (int64_t)min(r + (lane & 31), last) * D + 8 * (lane >> 5);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) v[kk] = ld16(vp + 16 * kk);
    }
  }

  // one block of rows r .. r + 31, of which those before r1 count; vt is the
  // wave's own value tile in LDS; the wave's next block starts at row `after`
  __device__ __forceinline__ void step(const Rows& x, const T* vb, int r, int after, int r1, float c,
                                       char* vt, int lane) {
    const int h = lane >> 5;
    f32x16 s[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[q][v] = 0.f;
    if constexpr (sizeof(T) == 2) {
      // the values go to LDS row by row while the scores are multiplied (the
      // wave's own tile, and LDS serves a wave in order: no barrier)
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) st16(vt + (lane & 31) * PITCH + 32 * kk + 16 * h, v[kk]);
      if (after < r1) load_values(vb, after, r1 - 1, lane);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const bf16x8 k = __builtin_bit_cast(bf16x8, x.k[kk]);
#pragma unroll
        for (int q = 0; q < QT; ++q) s[q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qhi[q][kk], s[q], 0, 0, 0);
#pragma unroll
        for (int q = 0; q < QT; ++q) s[q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qlo[q][kk], s[q], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int p = 0; p < D / 8; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int q = 0; q < QT; ++q)
            s[q] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x.k[p][j]), qf[q][4 * p + j], s[q], 0, 0, 0);
    }
    if (r + PRE_ROWS > r1) {
#pragma unroll
      for (int q = 0; q < QT; ++q)
#pragma unroll
        for (int v = 0; v < 16; ++v) s[q][v] = r + 8 * (v / 4) + 4 * h + v % 4 < r1 ? s[q][v] : -INFINITY;
    }
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      float mb = s[q][0];
#pragma unroll
      for (int v = 1; v < 16; ++v) mb = fmaxf(mb, s[q][v]);
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mb), __float_as_uint(mb), false, false);
      mb = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c;
      // finite in every lane from the first block on (its first row counts)
      if (__any(mb > M[q] + PRE_RESCALE)) {
        const float mn = fmaxf(M[q], mb);
        const float f = fast_exp2(M[q] - mn);  // 0 while M = -inf
        M[q] = mn;
        l[q] *= f;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[q][b][v] *= f;
      }
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bf16x8 pb[QT], pl[QT];
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          u32x4 p, e;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p0 = fast_exp2(fmaf(s[q][8 * t + 2 * i], c, -M[q]));
            const float p1 = fast_exp2(fmaf(s[q][8 * t + 2 * i + 1], c, -M[q]));
            p[i] = pack_bf16x2(p0, p1);
            e[i] = pack_bf16x2(p0 - bf16_lo(p[i]), p1 - bf16_hi(p[i]));
            l[q] += p0 + p1;
          }
          pb[q] = __builtin_bit_cast(bf16x8, p);
          pl[q] = __builtin_bit_cast(bf16x8, e);
        }
        // V^T: elements 32 b + 16 (l/16 % 2) .. of rows 16 t + 8 j + 4 h + 0..3
        const int i16 = lane & 15;
        const char* at = vt + (16 * t + 4 * h + i16 / 4) * PITCH + 32 * ((lane >> 4) & 1) + 8 * (i16 % 4);
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          const s16x4 lo = lds_read_tr16(at + 64 * b), hi = lds_read_tr16(at + 64 * b + 8 * PITCH);
          const s16x8 a = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
          for (int q = 0; q < QT; ++q)
            o[q][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), pb[q], o[q][b], 0, 0, 0);
#pragma unroll
          for (int q = 0; q < QT; ++q)
            o[q][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), pl[q], o[q][b], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          const float p = fast_exp2(fmaf(s[q][v], c, -M[q]));
          l[q] += p;
#pragma unroll
          for (int b = 0; b < DB; ++b)
            o[q][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.v[v * DB + b], p, o[q][b], 0, 0, 0);
        }
      }
    }
  }
};

// waves of a SIMD that the registers of a shape are held to
constexpr int prefix_waves(bool bf16, int D, int QT) { return !bf16 ? 1 : D == 64 && QT == 1 ? 3 : 2; }

// one workgroup per (prefix, head, chunk of rows, QT tiles of queries)
template <typename T, int D, int QT>
__global__ __launch_bounds__(64 * PRE_KEY_WAVES, prefix_waves(sizeof(T) == 2, D, QT)) void prefix_kernel(
    const T* __restrict__ q, const T* __restrict__ k_pre, const T* __restrict__ v_pre,
    const int32_t* __restrict__ pre_len, const int32_t* __restrict__ cur_tok,
    const int32_t* __restrict__ pos, int32_t L_meta, int32_t H, int32_t P_cap, int32_t per,
    int32_t n_chunk, int32_t n_slice, float c, int rotate, PrefixFreq tab, float* __restrict__ part_o,
    float2* __restrict__ part_ml) {
  using Tile = PrefixTile<T, D, QT>;
  constexpr int QUERIES = QT * PRE_QUERIES;
  constexpr int THREADS = 64 * PRE_KEY_WAVES;
  constexpr int HD = D / 2;
  constexpr int DB = Tile::DB;
  constexpr int QPITCH = D + 4;
  constexpr int Q_BYTES = QUERIES * QPITCH * 4;
  constexpr int V_BYTES = PRE_KEY_WAVES * Tile::V_BYTES;
  constexpr int O_BYTES = PRE_KEY_WAVES * 16 * DB * 64 * 4;
  __shared__ __align__(16) char lds[std::max(std::max(Q_BYTES, V_BYTES), O_BYTES)];
  __shared__ float2 meet[QT][PRE_KEY_WAVES][PRE_QUERIES];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int kw = __builtin_amdgcn_readfirstlane(tid >> 6);
  // chunks of a slice and slices first, tiles of queries behind: workgroups
  // that read the same rows are a multiple of the slices' chunks apart
  const int qt = blockIdx.x / (n_slice * n_chunk);
  const int rest = blockIdx.x - qt * (n_slice * n_chunk);
  const int slice = rest / n_chunk, chunk = rest - slice * n_chunk;
  const int g = slice / H, h_ = slice - g * H;
  const int q0 = qt * QUERIES;  // first query of the workgroup (of the prefix's `per`)

  // The tile's queries, element pairs (e, e + d/2) by thread; every load is
  // asked for before any is used (one pair after the other, with its token's
  // position, the prologue took longer than 1000 rows).
  constexpr int PAIRS = QUERIES * HD / THREADS;
  static_assert(PAIRS * THREADS == QUERIES * HD, "whole pairs a thread");
  T xr[PAIRS], yr[PAIRS];
  int tok[PAIRS];
  double freq[PAIRS];
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    const int f = tid + i * THREADS, j = f / HD, e = f - j * HD;
    const int s = g * per + min(q0 + j, per - 1);
    const T* src = q + ((int64_t)s * H + h_) * D;
    xr[i] = src[e];
    yr[i] = src[e + HD];
    tok[i] = rotate ? cur_tok[s] : 0;
    freq[i] = rotate ? tab.w[e] : 0.0;
  }
  const int n = min(max(pre_len[g], 0), P_cap);
  const int each = ((n + n_chunk - 1) / n_chunk + PRE_ROWS - 1) / PRE_ROWS * PRE_ROWS;
  const int r0 = min(chunk * (int64_t)each, (int64_t)n), r1 = min((int64_t)r0 + each, (int64_t)n);
  const int64_t at = ((int64_t)g * H + h_) * P_cap * D;
  const T* kb = k_pre + at;
  const T* vb = v_pre + at;
  typename Tile::Rows A, B;
  constexpr int STRIDE = PRE_ROWS * PRE_KEY_WAVES;
  int r = r0 + PRE_ROWS * kw;
  int ps[PAIRS];
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    const int s = g * per + min(q0 + (tid + i * THREADS) / HD, per - 1);
    // (a token outside the metadata: its step's output does not come from here)
    ps[i] = rotate && tok[i] >= 0 && tok[i] < L_meta ? pos[(int64_t)s * L_meta + tok[i]] : 0;
  }
  Tile st;
  if (r < r1) {
    Tile::load(A, kb, vb, r, r1 - 1, lane);
    st.load_values(vb, r, r1 - 1, lane);
  }
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    const int f = tid + i * THREADS, j = f / HD, e = f - j * HD;
    float x, y;
    if constexpr (sizeof(T) == 2) {
      x = bf16_lo((uint32_t)xr[i]);
      y = bf16_lo((uint32_t)yr[i]);
    } else {
      x = xr[i];
      y = yr[i];
    }
    if (rotate) {
      const double two_pi = 6.283185307179586476925286766559;
      const double inv_two_pi = 0.15915494309189533576888376337251;
      double ang = (double)ps[i] * freq[i];
      ang -= two_pi * rint(ang * inv_two_pi);
      float sn, cs;
      sincosf((float)ang, &sn, &cs);
      const float x1 = x;
      x = x1 * cs - y * sn;
      y = y * cs + x1 * sn;
    }
    float* dst = reinterpret_cast<float*>(lds) + j * QPITCH;
    dst[e] = x;
    dst[e + HD] = y;
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < QT; ++x)
    st.take_query(x, reinterpret_cast<const float*>(lds) + (PRE_QUERIES * x + (lane & 31)) * QPITCH, h);
  __syncthreads();  // every wave has its queries; the tiles of values take their place

  char* vt = lds + kw * Tile::V_BYTES;
  for (; r + 2 * STRIDE < r1; r += 2 * STRIDE) {
    Tile::load(B, kb, vb, r + STRIDE, r1 - 1, lane);
    st.step(A, vb, r, r + STRIDE, r1, c, vt, lane);
    Tile::load(A, kb, vb, r + 2 * STRIDE, r1 - 1, lane);
    st.step(B, vb, r + STRIDE, r + 2 * STRIDE, r1, c, vt, lane);
  }
  if (r < r1) {
    const bool more = r + STRIDE < r1;
    if (more) Tile::load(B, kb, vb, r + STRIDE, r1 - 1, lane);
    st.step(A, vb, r, r + STRIDE, r1, c, vt, lane);
    if (more) st.step(B, vb, r + STRIDE, r1, r1, c, vt, lane);
  }

  // The key waves meet: first their maxima and sums, then their outputs, each
  // taken to the common maximum, of which every wave adds up a quarter (both
  // halves of a wave hold a part of each query's sum).
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.l[x]), __float_as_uint(st.l[x]), false, false);
    st.l[x] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (lane < 32) meet[x][kw][lane] = make_float2(st.M[x], st.l[x]);
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    float M = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < PRE_KEY_WAVES; ++w) M = fmaxf(M, meet[x][w][lane & 31].x);
    const float m0 = M == -INFINITY ? 0.f : M;  // (no row at all)
#pragma unroll
    for (int w = 0; w < PRE_KEY_WAVES; ++w) {
      const float2 y = meet[x][w][lane & 31];
      l = fmaf(y.y, fast_exp2(y.x - m0), l);
    }
    const float f = fast_exp2(st.M[x] - m0);  // 0 for a wave without rows
    float* mine = reinterpret_cast<float*>(lds) + kw * 16 * DB * 64;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) mine[(16 * b + v) * 64 + lane] = st.o[x][b][v] * f;
    __syncthreads();
    const int j = q0 + PRE_QUERIES * x + (lane & 31);
    if (j < per) {
      const int64_t p = ((int64_t)(g * per + j) * H + h_) * n_chunk + chunk;
      if (tid < 32) part_ml[p] = make_float2(M, l);
      // wave w: registers 4 w .. 4 w + 3 of each block, elements 32 b + 8 w + 4 h + 0..3
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const int e = 32 * b + 8 * kw + 4 * h;
        if (e >= D) continue;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < PRE_KEY_WAVES; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            sum[i] += reinterpret_cast<const float*>(lds)[((w * DB + b) * 16 + 4 * kw + i) * 64 + lane];
        *reinterpret_cast<f32x4*>(part_o + p * D + e) = sum;
      }
    }
    if (x + 1 < QT) __syncthreads();  // the next tile's outputs take their place
  }
}

// Tiles of queries of a wave: two where it has them and holds both (bf16, 64
// elements a head: 254 registers), so that each row is loaded once for 64
// queries and two chains of softmax steps run beside each other (64 sequences
// behind 12288 rows: the prefix's part 32.7 -> 25.9 us).  At 80 elements two
// tiles leave one wave a SIMD, with the accumulators in the other half of the
// registers (64 behind 4000 rows: 32 us with one tile, 37 with two).
static int prefix_tiles(bool bf16, int32_t d, int32_t per) {
  return bf16 && d == 64 && per > PRE_QUERIES ? 2 : 1;
}
// Chunks of each prefix slice: as many as give every CU a workgroup, none of
// less than 128 rows.  Two workgroups a CU cost more at the ends (prologue,
// partials) than they hide: 64 behind 12288 rows 48 and 52 us, 32 behind 4000
// 20.6 and 21.5, 8 behind each of four of 2050 (80 elements) 28.8 and 28.2.
constexpr int PRE_WGS = 256;
int prefix_chunks(bool bf16, int32_t d, int32_t n_prefix, int32_t H, int32_t per, int32_t P_cap) {
  const int q = prefix_tiles(bf16, d, per) * PRE_QUERIES;
  const int64_t wgs = (int64_t)n_prefix * H * ((per + q - 1) / q);
  const int64_t want = std::max<int64_t>(1, PRE_WGS / wgs);
  return (int)std::min<int64_t>(want, (P_cap + 127) / 128);
}

template <typename T, int D>
static int launch_prefix_typed(const void* q, const void* k, const void* v, const int32_t* len,
                               int32_t n_prefix, int32_t P_cap, const int32_t* cur_tok,
                               const int32_t* pos, int32_t L_meta, int32_t b, int32_t H,
                               float scale, float theta, float* part_o, float* part_ml,
                               hipStream_t stream) {
  const int per = b / n_prefix;
  const int q_wg = prefix_tiles(sizeof(T) == 2, D, per) * PRE_QUERIES;
  const int qtiles = (per + q_wg - 1) / q_wg;
  const int nc = prefix_chunks(sizeof(T) == 2, D, n_prefix, H, per, P_cap);
  const int64_t wgs = (int64_t)n_prefix * H * nc * qtiles;
  if (wgs > 0x7fffffff) return fail(SCKV_EUNSUP, "shared_prefix_decode_attn: too many slices");
  PrefixFreq tab;
  for (int i = 0; i < 40; ++i) tab.w[i] = 0.0;
  if (theta > 0.f)
    for (int i = 0; i < D / 2; ++i) tab.w[i] = std::pow((double)theta, -2.0 * i / D);
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)wgs, 64 * PRE_KEY_WAVES, 0, stream>>>(
        static_cast<const T*>(q), static_cast<const T*>(k), static_cast<const T*>(v), len, cur_tok,
        pos, L_meta, H, P_cap, per, nc, n_prefix * H, scale * 1.4426950408889634f, theta > 0.f, tab,
        part_o, reinterpret_cast<float2*>(part_ml));
  };
  constexpr int MOST = sizeof(T) == 2 && D == 64 ? 2 : 1;
  if (q_wg > PRE_QUERIES) go(prefix_kernel<T, D, MOST>);
  else go(prefix_kernel<T, D, 1>);
  return hip_check(hipGetLastError(), "shared_prefix_decode_attn: prefix launch");
}

int launch_prefix(const void* q, const void* k, const void* v, const int32_t* len,
                  int32_t n_prefix, int32_t P_cap, const int32_t* cur_tok, const int32_t* pos,
                  int32_t L_meta, int32_t b, int32_t H, int32_t d_head, sckv_dtype dt, float scale,
                  float theta, float* part_o, float* part_ml, hipStream_t stream) {
#define SCKV_PREFIX(T, D)                                                                          \
  launch_prefix_typed<T, D>(q, k, v, len, n_prefix, P_cap, cur_tok, pos, L_meta, b, H, scale,      \
                            theta, part_o, part_ml, stream)
  if (dt == SCKV_BF16) return d_head == 64 ? SCKV_PREFIX(uint16_t, 64) : SCKV_PREFIX(uint16_t, 80);
  return d_head == 64 ? SCKV_PREFIX(float, 64) : SCKV_PREFIX(float, 80);
#undef SCKV_PREFIX
}

}  // namespace sckv
