// One decode step over the compacted cache, split over key chunks.
// Section 1 and Section 2 (the key/value memory read per step drives decode
// cost) and Section 4.3 (generation continues from the compressed cache).
//
// decode_chunk_kernel : one workgroup per (sequence, head, chunk of CH rows),
//   chunk-major (chunks of one slice share no data but q, so L2 placement
//   does not matter; idle workgroups past a slice's end go last).  A
//   workgroup streams its rows with a 16-byte piece per lane; a row is spread
//   over LPR lanes of an aligned power-of-two group of GRP lanes, so the row
//   dot product is a DPP butterfly inside the group.  Each lane group keeps an
//   online softmax; the groups of the workgroup are merged through LDS into
//   one partial (max, sum, unnormalised output) in log2 units.  The
//   workgroup whose chunk holds row kv_len also rotates the new key and writes
//   the new key/value pair there.
// decode_combine_kernel : merges the partials of each slice (log-sum-exp) and
//   writes the output; a <CL> step outputs v_new, a failed step NaN.  Being a
//   separate launch on the same stream, it sees every partial without any
//   device-wide cache flush inside the chunk kernel.
#include <math.h>

#include <algorithm>
#include <cmath>
#include <mutex>
#include <string>

#include "sckv_common.h"

namespace sckv {

// Launch shapes, measured on MI355X.  A slice is one (sequence, head) pair.
//  * bf16, fewer than DEC_SINGLE_MIN slices of a long cache: each slice is cut
//    into chunks, one 4-wave workgroup each, and a second kernel merges the
//    chunk partials.  A chunk has about DEC_CH rows at most; a launch of few
//    slices is cut finer, to DEC_FILL workgroups or chunks of DEC_CH_MIN rows,
//    as far as the workspace holds the partials (32 slices of 1000 rows,
//    d = 80: 18.2 us in chunks of DEC_CH, 9.6 us in chunks of 128; a target of
//    1024 workgroups was up to 27% slower, one of 256 within 3%).
//  * Otherwise one workgroup per slice writes the output itself (no second
//    launch).  Below DEC_SINGLE_MIN slices only over short caches, because a
//    batch's lengths differ and one long slice then outlasts the launch on its
//    one CU.  The host knows the cache's capacity alone: the line is at
//    DEC_ONE_ROWS + DEC_ONE_ROWS_PER_SLICE * slices rows, and at most
//    DEC_ONE_MAX_ROWS, up to which the most unequal batch (one sequence that
//    fills the cache, the others 500 rows) is not slower than in chunks of
//    DEC_CH and equal lengths are faster.  us split and so, d = 64: 192 slices
//    in a cache of 1536 rows 16.5 and 15.5 (equal lengths 22.0 and 17.2), 480
//    slices 20.7 and 22.6 (in chunks of DEC_CH 22.6; equal 39.5 and 35.1), 160
//    slices of 1500 10.7 and 13.9 (13.8; equal 18.2 and 16.6).  Above it the
//    loss grows without end: 192 slices, 3072 / 16000 rows 18.9 / 44.5 and
//    27.1 / 120 (equal 36.2 / 140 and 30.7 / 141), 384 slices of 2048 rows 22.1
//    and 25.6 (equal 40.8 and 43.1).  Fewer slices leave CUs idle (32 slices of
//    512 / 1000 rows, equal, d = 64: 7.7 / 7.8 split, 6.9 / 10.8 so).
//    Waves per slice (bf16): the most (4, 2 or 1; 1 only where d <= 64) with
//    which every wave of the launch is resident at once (the kernel holds two
//    waves per SIMD), so the launch runs in one round; where even one wave per
//    slice exceeds that, 4 waves, whose shorter workgroups balance the rounds
//    best.  Measured: 512 slices (d = 80) 4 waves; 2048 slices (d = 64) 1 wave
//    2% faster than 2 and 4% faster than 4; 8192 slices (d = 80) 4 waves 2.5%
//    faster than 2.
//  * fp32: split below DEC_SINGLE_MIN slices; from there on one workgroup per
//    slice of 512 threads, of 256 from DEC_NARROW_MIN slices on.
constexpr int DEC_CH = 1024;
constexpr int DEC_CH_MIN = 128;
constexpr int DEC_FILL = 512;
constexpr int DEC_ONE_ROWS = 512;
constexpr int DEC_ONE_ROWS_PER_SLICE = 8;
constexpr int DEC_ONE_MAX_ROWS = 1536;
constexpr int DEC_SINGLE_MIN = 512;
constexpr int DEC_NARROW_MIN = 1024;
constexpr int DEC_WAVES_PER_SIMD = 2;  // decode_mfma_kernel's occupancy (its register count)
constexpr size_t SCORE_LDS = 144 << 10;  // of a CU's 160 KB, for the scores of its workgroups
constexpr int DEC_SPEC2_ROWS = 512;    // cache rows per wave from which two blocks are speculated

// compute units of the current device, asked once per device
static int device_cus(int* cus) {
  static std::mutex mu;
  static int cached[64] = {0};
  int dev = 0;
  int rc = hip_check(hipGetDevice(&dev), "compacted_decode_attn: hipGetDevice");
  if (rc) return rc;
  if (dev < 0 || dev >= 64) return fail(SCKV_EUNSUP, "compacted_decode_attn: device index above 63");
  std::lock_guard<std::mutex> lock(mu);
  if (cached[dev] == 0) {
    int n = 0;
    rc = hip_check(hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev),
                   "compacted_decode_attn: hipDeviceGetAttribute");
    if (rc) return rc;
    cached[dev] = n > 0 ? n : 1;
  }
  *cus = cached[dev];
  return 0;
}
constexpr int DEC_THREADS = 256;  // fp32 split chunks
constexpr float LOG2E = 1.4426950408889634f;

struct RopeTab {
  double w[40];  // theta^(-2i/d), i < d/2
};

template <typename T, int D, int THREADS>
struct DecCfg {
  static constexpr int E = Piece<T>::E;           // elements per piece
  static constexpr int LPR = D / E;               // pieces per row
  static constexpr int GRP = LPR <= 8 ? 8 : (LPR <= 16 ? 16 : 32);
  static constexpr int RPW = 64 / GRP;            // rows per wave per step
  static constexpr int U = 4;                     // steps per trip (loads in flight per lane: 2U)
  static constexpr int NG = (THREADS / 64) * RPW;  // lane groups per workgroup
};

// rotated piece `seg` of a head vector x (global), rotate-half convention;
// inv[i] = theta^(-2i/d) (LDS)
template <typename T, int D>
__device__ __forceinline__ void load_rotated_piece(const T* x, int seg, bool rotate, double ps,
                                                   const double* inv, float* out) {
  constexpr int E = Piece<T>::E;
  constexpr int LPR = D / E;
  Piece<T>::unpack(ld16(x + seg * E), out);
  if (!rotate) return;
  const bool first = seg < LPR / 2;
  const int pseg = first ? seg + LPR / 2 : seg - LPR / 2;
  float partner[E];
  Piece<T>::unpack(ld16(x + pseg * E), partner);
  const double two_pi = 6.283185307179586476925286766559;
  const double inv_two_pi = 0.15915494309189533576888376337251;
  const int i0 = (first ? seg : pseg) * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    double ang = ps * inv[i0 + e];
    ang -= two_pi * rint(ang * inv_two_pi);
    float sn, cs;
    sincosf((float)ang, &sn, &cs);
    out[e] = first ? out[e] * cs - partner[e] * sn : out[e] * cs + partner[e] * sn;
  }
}

// two products and their sum, each rounded (never fused)
__device__ __forceinline__ float plain_turn(float x, float y, float cs, float sn) {
#pragma clang fp contract(off)
  const float a = x * cs;
  const float b = y * sn;
  return a + b;
}

// What a launch does beside the step itself.
struct StepOnly {
  static constexpr bool WEIGHTS = false, PREFIX = false, PLAIN_ROTATION = false;
};
// Adds the step's softmax weights to each row's accumulated weight.  A row's
// weight needs the whole slice's maximum and sum, so the scores (log2 units)
// are kept and turned into weights once those are known: by the slice's own
// workgroup where there is one, else by workgroups of the merge.  They are
// kept in LDS where one workgroup has the slice and the cache's capacity fits
// (`in_lds`), else in `scores`; computing them again would read the keys twice.
struct StepWeights {
  static constexpr bool WEIGHTS = true, PREFIX = false, PLAIN_ROTATION = true;
  const float* w_in;
  float* w_out;
  float* scores;  // [slice][L_cap]
  int32_t in_lds;
};
extern __shared__ float lds_scores[];  // [L_cap] (StepWeights, in_lds)

// keeps the score of a slice's row r
__device__ __forceinline__ void keep_score(const StepWeights& x, int64_t at, int r, float score) {
  if (x.in_lds) lds_scores[r] = score;
  else x.scores[at + r] = score;
}

// The first OLD_SUMS of a thread's accumulated weights, asked for before the
// workgroup's merge and used after it.
constexpr int OLD_SUMS = 8;
struct OldSums {
  float v[OLD_SUMS];
  __device__ __forceinline__ void load(const StepWeights& x, int64_t at, int n, int tid, int nthr) {
#pragma unroll
    for (int i = 0; i < OLD_SUMS; ++i) {
      const int r = tid + i * nthr;
      v[i] = x.w_in && r < n ? x.w_in[at + r] : 0.f;
    }
  }
};
// Joins the partials of a shared prefix (one per chunk of it) to the slice's.
struct StepPrefix {
  static constexpr bool WEIGHTS = false, PREFIX = true, PLAIN_ROTATION = true;
  const float* o;    // [slice][n][d], unnormalised
  const float2* ml;  // [slice][n]: maximum (log2 units), sum of weights
  int32_t n;
};

// w_out of rows [0, n) of a slice whose step adds nothing
__device__ __forceinline__ void keep_weights(const StepWeights& x, int64_t at, int n, int tid,
                                             int nthr) {
  for (int r = tid; r < n; r += nthr) x.w_out[at + r] = x.w_in ? x.w_in[at + r] : 0.f;
}

// w_out of rows [r0, r1) of a slice of n cache rows and the new one, from the
// slice's maximum M (log2 units) and sum of weights L
__device__ __forceinline__ void add_weights(const StepWeights& x, int64_t at, int n, int r0, int r1,
                                            float M, float L, int tid, int nthr,
                                            const OldSums& first) {
  const float inv = 1.f / L;
  for (int base = r0 + tid; base < r1; base += OLD_SUMS * nthr) {
    OldSums old;
    float sc[OLD_SUMS];
    if (base == r0 + tid) {
      old = first;
    } else {
      old.load(x, at, n, base, nthr);
    }
#pragma unroll
    for (int i = 0; i < OLD_SUMS; ++i) {
      const int r = min(base + i * nthr, r1 - 1);
      sc[i] = x.in_lds ? lds_scores[r] : x.scores[at + r];
    }
#pragma unroll
    for (int i = 0; i < OLD_SUMS; ++i) {
      const int r = base + i * nthr;
      if (r < r1) x.w_out[at + r] = fmaf(fast_exp2(sc[i] - M), inv, old.v[i]);
    }
  }
}

// Element e's share of a slice's prefix partials: the first ones are asked for
// ahead of the workgroup's merge.
template <int D>
struct PrefixParts {
  static constexpr int FIRST = 4;
  float2 ml[FIRST];
  float o[FIRST];
  __device__ __forceinline__ void load(const StepPrefix& x, int bh, int e, int c0) {
#pragma unroll
    for (int i = 0; i < FIRST; ++i) {
      const int64_t c = (int64_t)bh * x.n + min(c0 + i, x.n - 1);
      ml[i] = x.ml[c];
      o[i] = x.o[c * D + e];
    }
  }
  // joins them to the slice's maximum M, sum L and unnormalised output ov
  __device__ __forceinline__ void join(const StepPrefix& x, int bh, int e, float& M, float& L,
                                       float& ov) {
    for (int c0 = 0; c0 < x.n; c0 += FIRST) {
      if (c0 > 0) load(x, bh, e, c0);
      float Mx = M;
#pragma unroll
      for (int i = 0; i < FIRST; ++i) Mx = fmaxf(Mx, ml[i].x);
      const float f = exp2f(M - Mx);  // M is finite: the slice holds the new row
      L *= f;
      ov *= f;
#pragma unroll
      for (int i = 0; i < FIRST; ++i) {
        // 0 for a chunk without rows (its maximum -inf) and past the last one
        const float w = c0 + i < x.n ? exp2f(ml[i].x - Mx) : 0.f;
        L = fmaf(ml[i].y, w, L);
        ov = fmaf(o[i], w, ov);
      }
      M = Mx;
    }
  }
};

// 0: ordinary append step; 1: <CL> step; 2: token outside [0, L_meta);
// 3: no room for the new row
__device__ __forceinline__ int step_kind(const int32_t* cur_tok, const int32_t* vu,
                                         const int32_t* kv_len, int s, int L_meta, int L_cap) {
  const int t = cur_tok[s];
  if (t < 0 || t >= L_meta) return 2;
  if (vu[(int64_t)s * L_meta + t] == t) return 1;
  const int n = kv_len[s];
  if (n < 0 || n >= L_cap) return 3;
  return 0;
}

// A slice's rows split into n chunks of `rows` rows (the last one shorter).
// Chunk starts are multiples of 16 rows:
// a wave then reads whole 128-byte lines (a bf16 row of 80 elements is 160
// bytes, so only every fourth row starts on a line; a chunk that started
// between would make every load of its wave span one line more).
struct ChunkPlan {
  int n, rows;
};
constexpr int DEC_ALIGN = 16;
// How a launch splits its slices: at least one chunk for every DEC_CH rows,
// and up to `want` chunks of at least DEC_CH_MIN rows; never more than `most`
// (the partials the workspace holds for a slice).
struct Split {
  int32_t want, most;
};
// rows is a positive int, so every sum below fits in 32 unsigned bits
__device__ __forceinline__ ChunkPlan chunk_plan(int rows, Split sp) {
  const uint32_t r = (uint32_t)rows;
  const uint32_t fine = min((r + DEC_CH_MIN - 1) / DEC_CH_MIN, (uint32_t)sp.want);
  const uint32_t n0 = min(max((r + DEC_CH - 1) / DEC_CH, fine), (uint32_t)sp.most);
  const uint32_t per = (r + n0 - 1) / n0;
  const uint32_t cr = (per + DEC_ALIGN - 1) / DEC_ALIGN * DEC_ALIGN;
  ChunkPlan p;
  p.rows = (int)cr;
  p.n = (int)((r + cr - 1) / cr);  // <= n0
  return p;
}

// Writes the final output of a slice whose step is not an ordinary append
// (kind 1: <CL>, the output is v_new; kind 2/3: failure, NaN and a status
// bit).  `tid` runs over `nthr` threads.
template <typename T, int D>
__device__ __forceinline__ void write_special(int kind, const T* v_new, T* o, int32_t* status,
                                              int bh, int H, int tid, int nthr) {
  if (kind >= 2 && tid == 0 && (bh % H) == 0 && status)
    atomicOr(status, kind == 2 ? SCKV_STATUS_TOKEN : SCKV_STATUS_CAP);
  for (int i = tid; i < D; i += nthr) {
    if (kind == 1) o[(int64_t)bh * D + i] = v_new[(int64_t)bh * D + i];
    else if constexpr (sizeof(T) == 2) o[(int64_t)bh * D + i] = (T)0x7fc0;  // bf16 NaN
    else o[(int64_t)bh * D + i] = NAN;
  }
}

// FINAL: the workgroup covers the whole slice (one chunk) and
// writes the output itself; otherwise it writes a partial for the combine.
template <typename T, int D, int THREADS, bool FINAL, typename X>
__global__ __launch_bounds__(THREADS) void decode_chunk_kernel(
    const T* __restrict__ q, const T* __restrict__ k_new, const T* __restrict__ v_new,
    T* __restrict__ k_cache, T* __restrict__ v_cache, const int32_t* __restrict__ kv_len,
    const int32_t* __restrict__ cur_tok, const int32_t* __restrict__ vu,
    const int32_t* __restrict__ pos, int32_t L_meta, int32_t H, int32_t L_cap, float qscale,
    int rotate, RopeTab tab, float* __restrict__ part, int32_t n_chunk_max, int32_t n_work,
    Split sp, T* __restrict__ o, int32_t* __restrict__ status, X x) {
  using C = DecCfg<T, D, THREADS>;
  constexpr int E = C::E, LPR = C::LPR, GRP = C::GRP, RPW = C::RPW, U = C::U, NG = C::NG;
  // chunk-major order: every slice's first chunk is dispatched before any
  // slice's second chunk, so the workgroups that start past a slice's last
  // row (and exit at once) are dispatched last
  const int n_bh = n_work / n_chunk_max;
  const int chunk = blockIdx.x / n_bh;
  const int bh = blockIdx.x % n_bh;
  const int s = bh / H;
  const int kind = step_kind(cur_tok, vu, kv_len, s, L_meta, L_cap);
  if (kind != 0) {  // the combine handles it, or this workgroup when FINAL
    if constexpr (FINAL) write_special<T, D>(kind, v_new, o, status, bh, H, threadIdx.x, THREADS);
    if constexpr (FINAL && X::WEIGHTS)
      keep_weights(x, (int64_t)bh * L_cap, min(max(kv_len[s], 0), L_cap), threadIdx.x, THREADS);
    return;
  }
  const int n = kv_len[s];
  const int rows = n + 1;  // cache rows and the new row
  const ChunkPlan cp = chunk_plan(rows, sp);
  if (chunk >= cp.n) return;
  const int r0 = chunk * cp.rows;
  const int r1 = min(r0 + cp.rows, rows);
  const int rc = min(r1, n);  // cache rows of this chunk: [r0, rc)

  const int tid = threadIdx.x;
  const int wave = tid >> 6;
  const int lane = tid & 63;
  const int g = lane / GRP;      // row slot within the wave
  const int seg = lane % GRP;    // piece within the row
  const bool active = seg < LPR;

  const T* kb = k_cache + (int64_t)bh * L_cap * D;
  const T* vb = v_cache + (int64_t)bh * L_cap * D;
  constexpr int TRIP = (THREADS / 64) * U * RPW;  // rows per trip of the workgroup
  const int base0 = r0 + wave * U * RPW;

  // streamed rows: the 2U loads of one trip are issued together
  u32x4 kw[U], vw[U];
  auto issue = [&](int base, u32x4* kd, u32x4* vd) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = base + u * RPW + g;
      if (row < rc && active) {
        kd[u] = ld16(kb + (int64_t)row * D + seg * E);
        vd[u] = ld16(vb + (int64_t)row * D + seg * E);
      } else {
        kd[u] = u32x4{0, 0, 0, 0};
        vd[u] = u32x4{0, 0, 0, 0};
      }
    }
  };
  __shared__ double inv[D / 2];
  if (rotate && tid < D / 2) inv[tid] = tab.w[tid];
  __syncthreads();

  const double ps = rotate ? (double)pos[(int64_t)s * L_meta + cur_tok[s]] : 0.0;
  float qf[E];
#pragma unroll
  for (int e = 0; e < E; ++e) qf[e] = 0.f;
  if (active) {
    load_rotated_piece<T, D>(q + (int64_t)bh * D, seg, rotate, ps, inv, qf);
#pragma unroll
    for (int e = 0; e < E; ++e) qf[e] *= qscale;  // scores come out in log2 units
  }

  float m = -INFINITY, l = 0.f, acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;

  issue(base0, kw, vw);
  for (int base = base0; base < rc; base += TRIP) {
    float sc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float kf[E];
      Piece<T>::unpack(kw[u], kf);
      float d = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) d = fmaf(qf[e], kf[e], d);
      d = group_sum<GRP>(d);
      const int row = base + u * RPW + g;
      sc[u] = row < rc ? d : -INFINITY;
      if constexpr (X::WEIGHTS)
        if (row < rc && seg == 0) keep_score(x, (int64_t)bh * L_cap, row, d);
    }
    float mx = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mx = fmaxf(mx, sc[u]);
    if (mx != -INFINITY) {
      const float alpha = exp2f(m - mx);  // m == -inf gives 0
      l *= alpha;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= alpha;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float p = exp2f(sc[u] - mx);
        l += p;
        float vf[E];
        Piece<T>::unpack(vw[u], vf);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(p, vf[e], acc[e]);
      }
      m = mx;
    }
    if (base + TRIP < rc) issue(base + TRIP, kw, vw);
  }

  // the new row: rotated k_new, v_new; written to the cache by this chunk
  if (n >= r0 && n < r1 && wave == 0 && g == 0) {
    float kf[E], vf[E];
#pragma unroll
    for (int e = 0; e < E; ++e) { kf[e] = 0.f; vf[e] = 0.f; }
    if (active) {
      load_rotated_piece<T, D>(k_new + (int64_t)bh * D, seg, rotate, ps, inv, kf);
      // score with the stored (rounded) key, exactly as later steps will see it
      Piece<T>::unpack(Piece<T>::pack(kf), kf);
      Piece<T>::unpack(ld16(v_new + (int64_t)bh * D + seg * E), vf);
    }
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) d = fmaf(qf[e], kf[e], d);
    d = group_sum<GRP>(d);
    if constexpr (X::WEIGHTS)
      if (seg == 0) keep_score(x, (int64_t)bh * L_cap, n, d);
    const float mx = fmaxf(m, d);
    const float alpha = exp2f(m - mx);
    const float p = exp2f(d - mx);
    l = l * alpha + p;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(p, vf[e], acc[e] * alpha);
    m = mx;
    if (active) {
      st16(k_cache + ((int64_t)bh * L_cap + n) * D + seg * E, Piece<T>::pack(kf));
      st16(v_cache + ((int64_t)bh * L_cap + n) * D + seg * E,
           ld16(v_new + (int64_t)bh * D + seg * E));
    }
  }

  OldSums old;
  if constexpr (FINAL && X::WEIGHTS) old.load(x, (int64_t)bh * L_cap, n, tid, THREADS);
  PrefixParts<D> pre;
  if constexpr (FINAL && X::PREFIX) pre.load(x, bh, min(tid, D - 1), 0);
  // merge the lane groups of the workgroup into this chunk's partial
  __shared__ float sm[NG], sl[NG];
  __shared__ float sacc[NG][D];
  const int grp = wave * RPW + g;
  if (active) {
#pragma unroll
    for (int e = 0; e < E; ++e) sacc[grp][seg * E + e] = acc[e];
    if (seg == 0) { sm[grp] = m; sl[grp] = l; }
  }
  __syncthreads();
  __shared__ float res[D];
  if (X::WEIGHTS || tid < D) {  // with weights every thread takes the maximum and the sum
    const int e = min(tid, D - 1);
    float M = -INFINITY;
    for (int i = 0; i < NG; ++i) M = fmaxf(M, sm[i]);
    float Lsum = 0.f, ov = 0.f;
    for (int i = 0; i < NG; ++i) {
      if (sm[i] == -INFINITY) continue;
      const float w = exp2f(sm[i] - M);
      Lsum += sl[i] * w;
      ov += sacc[i][e] * w;
    }
    if constexpr (FINAL && X::PREFIX) pre.join(x, bh, tid, M, Lsum, ov);
    if constexpr (FINAL && X::WEIGHTS)
      add_weights(x, (int64_t)bh * L_cap, n, 0, rows, M, Lsum, tid, THREADS, old);
    if (tid >= D) {
    } else if constexpr (FINAL) {
      res[tid] = ov / Lsum;
    } else {
      float* out = part + ((int64_t)bh * n_chunk_max + chunk) * (D + 2);
      out[2 + tid] = ov;
      if (tid == 0) { out[0] = M; out[1] = Lsum; }
    }
  }
  if constexpr (FINAL) {
    __syncthreads();
    if (tid < D / E) {
      float f[E];
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = res[tid * E + e];
      st16(o + (int64_t)bh * D + tid * E, Piece<T>::pack(f));
    }
  }
}

// One workgroup of four waves per slice: log-sum-exp merge of the slice's
// chunk partials, 64 chunks at a time (lane c holds chunk c's weight; wave w
// adds chunks w, w + 4, ..., the output elements spread over its lanes; the
// waves' sums meet in LDS).
constexpr int COMBINE_WAVES = 4;
constexpr int WEIGHT_ROWS = 2048;  // rows of a workgroup that only adds weights
template <typename T, int D, typename X>
__global__ __launch_bounds__(64 * COMBINE_WAVES) void decode_combine_kernel(
    const T* __restrict__ v_new, const int32_t* __restrict__ kv_len,
    const int32_t* __restrict__ cur_tok, const int32_t* __restrict__ vu, int32_t L_meta,
    int32_t H, FastDiv by_H, int32_t L_cap, const float* __restrict__ part, int32_t n_chunk_max,
    Split sp, T* __restrict__ o, int32_t* __restrict__ status, int32_t ring, int32_t n_bh, X x) {
  // the workgroups behind the slices' add weights, WEIGHT_ROWS rows each
  const int blk = X::WEIGHTS ? (int)blockIdx.x / n_bh : 0;
  const int bh = (int)blockIdx.x - blk * n_bh;
  const int s = fast_div(bh, by_H);
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float* p = part + (int64_t)bh * n_chunk_max * (D + 2);
  // the first 64 chunks' maxima and sums are read along with the slice's
  // length (those past its chunks hold anything and are dropped below)
  float m0 = -INFINITY, l0 = 0.f;
  if (lane < n_chunk_max) {
    m0 = p[lane * (D + 2)];
    l0 = p[lane * (D + 2) + 1];
  }
  const int t = cur_tok[s];
  const int n = ring > 0 ? ring : kv_len[s];  // the ring is always full
  // rows of a workgroup that adds weights: asked for before the step's kind and
  // the slice's maximum and sum are known (a row past the last is read as it)
  const int64_t wat = (int64_t)bh * L_cap;
  const int r0 = (blk - 1) * WEIGHT_ROWS, r_end = min(max(n, 0), L_cap - 1);
  OldSums old;
  float sc[OLD_SUMS];
  if constexpr (X::WEIGHTS) {
    static_assert(WEIGHT_ROWS == OLD_SUMS * 64 * COMBINE_WAVES, "one batch of rows");
    if (blk > 0 && r0 <= r_end) {
      old.load(x, wat, r_end, r0 + tid, 64 * COMBINE_WAVES);
#pragma unroll
      for (int i = 0; i < OLD_SUMS; ++i) sc[i] = x.scores[wat + min(r0 + tid + i * 64 * COMBINE_WAVES, r_end)];
    }
  }
  // the step kind, as step_kind()
  const int kind = (t < 0 || t >= L_meta)                       ? 2
                   : vu[(int64_t)s * L_meta + t] == t           ? 1
                   : (ring == 0 && (n < 0 || n >= L_cap))       ? 3
                                                                : 0;
  if (kind != 0) {
    if (blk == 0) write_special<T, D>(kind, v_new, o, status, bh, H, tid, 64 * COMBINE_WAVES);
    if constexpr (X::WEIGHTS)
      if (blk == 1) keep_weights(x, wat, min(max(n, 0), L_cap), tid, 64 * COMBINE_WAVES);
    return;
  }
  const int nch = chunk_plan(n + 1, sp).n;
  if constexpr (X::WEIGHTS) {
    if (blk > 0) {
      if (r0 > n) return;
      float Mw = -INFINITY, lw = 0.f;
      for (int c0 = 0; c0 < nch; c0 += 64) {
        const int c = c0 + lane;
        const float mc = c >= nch ? -INFINITY : c0 == 0 ? m0 : p[c * (D + 2)];
        const float lc = c >= nch ? 0.f : c0 == 0 ? l0 : p[c * (D + 2) + 1];
        const float mn = fmaxf(Mw, wave_max(mc));
        lw = lw * exp2f(Mw - mn) + wave_sum(lc * exp2f(mc - mn));
        Mw = mn;
      }
      const float inv = 1.f / lw;
#pragma unroll
      for (int i = 0; i < OLD_SUMS; ++i) {
        const int row = r0 + tid + i * 64 * COMBINE_WAVES;
        if (row <= n) x.w_out[wat + row] = fmaf(fast_exp2(sc[i] - Mw), inv, old.v[i]);
      }
      return;
    }
  }
  PrefixParts<D> pre;
  if constexpr (X::PREFIX) pre.load(x, bh, min(tid, D - 1), 0);
  constexpr int PER = (D + 63) / 64;  // output elements per lane
  float M = -INFINITY, lsum = 0.f, acc[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) acc[j] = 0.f;
  for (int c0 = 0; c0 < nch; c0 += 64) {
    const int c = c0 + lane;
    float mc = -INFINITY, lc = 0.f;
    if (c < nch) {
      mc = c0 == 0 ? m0 : p[c * (D + 2)];
      lc = c0 == 0 ? l0 : p[c * (D + 2) + 1];
    }
    const float mb = wave_max(mc);
    const float mn = fmaxf(M, mb);    // finite: every chunk holds a row
    const float sc = exp2f(M - mn);   // 0 on the first block (M = -inf)
    lsum *= sc;
#pragma unroll
    for (int j = 0; j < PER; ++j) acc[j] *= sc;
    const float w = c < nch ? exp2f(mc - mn) : 0.f;
    lsum = fmaf(lc, w, lsum);
    const int cn = min(64, nch - c0);
#pragma unroll 4
    for (int i = wave; i < cn; i += COMBINE_WAVES) {
      const float wi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), i));
      const float* pc = p + (c0 + i) * (D + 2) + 2;
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (lane + 64 * j < D) acc[j] = fmaf(pc[lane + 64 * j], wi, acc[j]);
    }
    M = mn;
  }
  lsum = wave_sum(lsum);
  __shared__ float sums[COMBINE_WAVES][64 * PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) sums[wave][lane + 64 * j] = acc[j];
  __syncthreads();
  if (tid < D) {  // every wave holds the whole of lsum
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < COMBINE_WAVES; ++w) v += sums[w][tid];
    if constexpr (X::PREFIX) pre.join(x, bh, tid, M, lsum, v);
    v /= lsum;
    if constexpr (sizeof(T) == 2) o[(int64_t)bh * D + tid] = f32_to_bf16(v);
    else o[(int64_t)bh * D + tid] = v;
  }
}

// ---------------------------------------------------------------------------
// bf16 caches: scores on the matrix cores
// ---------------------------------------------------------------------------
// A wave takes 32-row blocks of the chunk (block i of the chunk goes to wave
// i mod NW).  Lane l owns key row l%32 of the block and elements
// 16kk + 8(l/32) .. +7 (kk < D/16) of that row's key and value: exactly the
// B operand of v_mfma_f32_32x32x16_bf16 for B[k][n] = K[n][k].  With the A
// operand holding q in every one of its 32 rows, every column n of the
// result is the score of key n, so each lane ends up with the score of its
// own key and weighs its own value elements with it (no cross-lane traffic
// per row).  q is split into two bf16 terms (hi + lo) so that the scores
// keep about fp32 accuracy.  The running maximum is raised only when a block
// maximum exceeds it by DM_RESCALE (log2 units), which keeps rescaling rare;
// accumulated weights stay below 2^DM_RESCALE per row.  The next block's
// rows are in flight while a block is computed.
constexpr float DM_RESCALE = 8.f;

template <int D, int NW, bool FINAL, bool SPEC2, typename X>
__global__ __launch_bounds__(NW * 64) void decode_mfma_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k_new,
    const uint16_t* __restrict__ v_new, uint16_t* __restrict__ k_cache,
    uint16_t* __restrict__ v_cache, const int32_t* __restrict__ kv_len,
    const int32_t* __restrict__ cur_tok, const int32_t* __restrict__ vu,
    const int32_t* __restrict__ pos, int32_t L_meta, int32_t H, int32_t L_cap, float qscale,
    int rotate, RopeTab tab, float* __restrict__ part, int32_t n_chunk_max, FastDiv by_H,
    FastDiv by_slices, int32_t n_bh, Split sp, uint16_t* __restrict__ o,
    int32_t* __restrict__ status, int32_t ring, X x) {
  constexpr int KS = D / 16;     // k steps of 16 elements
  constexpr int NA = 8 * KS;     // value elements per lane
  constexpr int THREADS = NW * 64;
  constexpr int HD = D / 2;
  // new-row elements: one per thread of the workgroup, then one or two per
  // lane of wave 0 for the score
  static_assert(D >= 64 && D <= 128 && D % 16 == 0 && D <= NW * 64, "head size");
  // chunk-major order (as in decode_chunk_kernel); a one-chunk launch has
  // one workgroup per slice
  const int chunk = FINAL ? 0 : fast_div(blockIdx.x, by_slices);
  const int bh = (int)blockIdx.x - chunk * n_bh;
  const int s = fast_div(bh, by_H);
  const int tid = threadIdx.x;
  const int wave = tid >> 6;
  const int lane = tid & 63;
  const int kr = lane & 31;
  const int h = lane >> 5;

  // The slice's length, token and position are wave-uniform and go through
  // scalar loads, whose counter is separate from that of the vector loads:
  // the first two blocks of key/value rows are issued as soon as the length
  // is known and arrive while q is prepared.  The block addresses use the
  // length clamped into the cache, so they are valid whatever the step turns
  // out to be.
  // ring > 0 (local-attention comparator): rows [0, ring) are a ring of the
  // ring most recent tokens, token t at row t mod ring; the new token
  // replaces the oldest, whose row is not attended
  const int n_raw = ring > 0 ? ring : kv_len[s];
  const int t_raw = cur_tok[s];
  // the query and the new row: thread tid < D takes element tid of q, k_new
  // and v_new, the elements q and k_new rotate against and their frequency
  // (from the argument block).  These vector loads go out before the block
  // loads (the counter retires in issue order), so they are ready before the
  // first block.  Picking q and the frequency out of scalar registers instead
  // cost about 1000 instructions a thread.  Threads past D re-read element
  // D - 1.
  const int te = min(tid, D - 1);
  const int tp = te < HD ? te + HD : te - HD;
  const uint16_t qx_raw = q[(int64_t)bh * D + te];
  const uint16_t qp_raw = q[(int64_t)bh * D + tp];
  double freq = 0.0;
  if (rotate) freq = tab.w[min(te, tp)];
  const uint16_t kx_raw = k_new[(int64_t)bh * D + te];
  const uint16_t kp_raw = k_new[(int64_t)bh * D + tp];
  const uint16_t vx_raw = v_new[(int64_t)bh * D + te];
  // A one-chunk launch (FINAL) starts its slice at row 0, so its first block
  // is rows 32*wave.. whatever the slice length: it is issued before the
  // length arrives (rows past the slice's end are neutralised below).
  const uint16_t* kb = k_cache + (int64_t)bh * L_cap * D;
  const uint16_t* vb = v_cache + (int64_t)bh * L_cap * D;
  auto load_row = [&](int row, u32x4* kd, u32x4* vd) {
    const uint16_t* kp = kb + (int64_t)row * D + 8 * h;
    const uint16_t* vp = vb + (int64_t)row * D + 8 * h;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) kd[kk] = ld16(kp + 16 * kk);
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) vd[kk] = ld16(vp + 16 * kk);
  };
  u32x4 kA[KS], vA[KS], kB[KS], vB[KS];
  if constexpr (FINAL) load_row(min(32 * wave + kr, L_cap - 1), kA, vA);
  // with SPEC2 (chosen by the host for caches large enough that slices are
  // taken to be long) the second block is issued before the length too
  if constexpr (FINAL && SPEC2) load_row(min(32 * (wave + NW) + kr, L_cap - 1), kB, vB);
  const bool t_ok = t_raw >= 0 && t_raw < L_meta;
  const int vu_t = t_ok ? vu[(int64_t)s * L_meta + t_raw] : 0;
  const int pos_t = (rotate && t_ok) ? pos[(int64_t)s * L_meta + t_raw] : 0;

  const int n = ring > 0 ? ring : min(max(n_raw, 0), L_cap - 1);
  const int slot = (ring > 0 && t_ok) ? t_raw % ring : -1;  // row of the new token (ring)
  const int rows = n + 1;
  const ChunkPlan cp = chunk_plan(rows, sp);
  const int r0 = chunk * cp.rows;
  const int r1 = min(r0 + cp.rows, rows);
  const int rc = min(r1, n);  // cache rows of this chunk: [r0, rc)
  const int nblk = chunk < cp.n ? (rc - r0 + 31) / 32 : 0;
  const bool holds_new = n >= r0 && n < r1;

  // rows past rc re-read row rc-1 (row 0 where the chunk has no rows);
  // their scores are masked
  auto load_blk = [&](int i, u32x4* kd, u32x4* vd) {
    load_row(max(min(r0 + 32 * i + kr, rc - 1), 0), kd, vd);
  };
  // issued whether or not the wave has these blocks, so that the counter
  // waits below stay exact on every path
  if constexpr (FINAL) {
    if constexpr (!SPEC2) load_blk(wave + NW, kB, vB);
    // a short slice: rows past its end were read too.  Their scores are
    // masked; their values are zeroed so that whatever those rows hold
    // (they may never have been written) adds exactly nothing.
    if (32 * wave + 32 > rc) {
      const bool a_in = 32 * wave + kr < rc;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) vA[kk] = a_in ? vA[kk] : u32x4{0, 0, 0, 0};
    }
    if constexpr (SPEC2) {
      if (32 * (wave + NW) + 32 > rc) {
        const bool b_in = 32 * (wave + NW) + kr < rc;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) vB[kk] = b_in ? vB[kk] : u32x4{0, 0, 0, 0};
      }
    }
  } else {
    load_blk(wave, kA, vA);
    load_blk(wave + NW, kB, vB);
  }

  // the step kind, with the precedence of step_kind()
  const int kind = !t_ok ? 2
                   : (vu_t == t_raw ? 1 : ((ring == 0 && (n_raw < 0 || n_raw >= L_cap)) ? 3 : 0));
  if (kind != 0) {
    if constexpr (FINAL) write_special<uint16_t, D>(kind, v_new, o, status, bh, H, tid, THREADS);
    if constexpr (FINAL && X::WEIGHTS)
      keep_weights(x, (int64_t)bh * L_cap, min(max(n_raw, 0), L_cap), tid, THREADS);
    return;
  }
  if (chunk >= cp.n) return;

  // rotated q and k elements tid (tid < D); both turn by the same angle.  The
  // key is rounded to bf16 as stored; its product with q and the value
  // element go to LDS.
  __shared__ float qs[D], kqs[D], vs[D];
  if (tid < D) {
    float x = bf16_lo((uint32_t)qx_raw);
    float kx = bf16_lo((uint32_t)kx_raw);
    if (X::PLAIN_ROTATION && rotate) {
      // sine and cosine in 64 bits, each rounded once, then two products and a
      // sum rounded to fp32: the stored key is that of plain fp32 arithmetic,
      // bit for bit.  (A key element rounded to its other bf16 neighbour moves
      // the fp32 weights by more than all their own rounding.)
      const float pv = bf16_lo((uint32_t)qp_raw), kp = bf16_lo((uint32_t)kp_raw);
      double turns = (double)pos_t * freq * 0.15915494309189533576888376337251;
      turns -= rint(turns);
      double sd, cd;
      sincospi(2.0 * turns, &sd, &cd);
      const float cs = (float)cd, sn = (float)(tid < HD ? -sd : sd);
      x = plain_turn(x, pv, cs, sn);
      kx = plain_turn(kx, kp, cs, sn);
    } else if (rotate) {
      const float pv = bf16_lo((uint32_t)qp_raw);
      const float kp = bf16_lo((uint32_t)kp_raw);
      const double two_pi = 6.283185307179586476925286766559;
      const double inv_two_pi = 0.15915494309189533576888376337251;
      double ang = (double)pos_t * freq;
      ang -= two_pi * rint(ang * inv_two_pi);
      float sn, cs;
      sincosf((float)ang, &sn, &cs);
      x = tid < HD ? x * cs - pv * sn : x * cs + pv * sn;
      kx = tid < HD ? kx * cs - kp * sn : kx * cs + kp * sn;
    }
    const uint16_t kq = f32_to_bf16(kx);
    qs[tid] = x;
    kqs[tid] = x * bf16_lo((uint32_t)kq);
    vs[tid] = bf16_lo((uint32_t)vx_raw);
    if (holds_new) {
      const int64_t dst = (int64_t)bh * L_cap + (ring > 0 ? slot : n);
      k_cache[dst * D + tid] = kq;
      v_cache[dst * D + tid] = vx_raw;
    }
  }
  __syncthreads();

  // Accumulated weights are fp32 sums: their launches carry q's last 8 bits
  // too, in a third term (two leave 2^-17 of a score).  There the three terms
  // lie in rows 0, 1 and 2 (mod 4) of one A operand: a lane's first three
  // results are its key's products with them, one MFMA a k step.
  bf16x8 qhi[KS], qlo[X::WEIGHTS ? 1 : KS];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {
    u32x4 wh, wl;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x0 = qs[16 * kk + 8 * h + 2 * i], x1 = qs[16 * kk + 8 * h + 2 * i + 1];
      const uint32_t hw = pack_bf16x2(x0, x1);
      wh[i] = hw;
      wl[i] = pack_bf16x2(x0 - bf16_lo(hw), x1 - bf16_hi(hw));
      if constexpr (X::WEIGHTS) {
        const uint32_t we = pack_bf16x2(x0 - bf16_lo(hw) - bf16_lo(wl[i]),
                                        x1 - bf16_hi(hw) - bf16_hi(wl[i]));
        const int term = kr & 3;
        wh[i] = term == 0 ? hw : term == 1 ? wl[i] : term == 2 ? we : 0;
      }
    }
    qhi[kk] = __builtin_bit_cast(bf16x8, wh);
    if constexpr (!X::WEIGHTS) qlo[kk] = __builtin_bit_cast(bf16x8, wl);
  }

  float M = -INFINITY, l = 0.f, acc[NA];
#pragma unroll
  for (int a = 0; a < NA; ++a) acc[a] = 0.f;
  // takes a score (wave-uniform block maximum over lanes); returns its weight
  auto weigh = [&](float sc) {
    const float mb = half_wave_max(sc);
    if (mb > M + DM_RESCALE) {
      const float f = exp2f(M - mb);  // 0 while M = -inf
      l *= f;
#pragma unroll
      for (int a = 0; a < NA; ++a) acc[a] *= f;
      M = mb;
    }
    return exp2f(sc - M);
  };
  auto compute = [&](int i, const u32x4* kd, const u32x4* vd) {
    f32x16 c;
#pragma unroll
    for (int v = 0; v < 16; ++v) c[v] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      const bf16x8 kv = __builtin_bit_cast(bf16x8, kd[kk]);
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qhi[kk], kv, c, 0, 0, 0);
      if constexpr (!X::WEIGHTS) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qlo[kk], kv, c, 0, 0, 0);
    }
    if constexpr (X::WEIGHTS) c[0] += c[1] + c[2];
    const int row = r0 + 32 * i + kr;
    const float sc = (row < rc && row != slot) ? c[0] * qscale : -INFINITY;
    if constexpr (X::WEIGHTS)
      if (h == 0 && row < rc) keep_score(x, (int64_t)bh * L_cap, row, sc);
    const float p = weigh(sc);
    if (h == 0) l += p;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = vd[kk][j];
        acc[8 * kk + 2 * j] = fmaf(p, bf16_lo(w), acc[8 * kk + 2 * j]);
        acc[8 * kk + 2 * j + 1] = fmaf(p, bf16_hi(w), acc[8 * kk + 2 * j + 1]);
      }
    }
  };

  // the new row opens the state of wave 0: its score is the sum of the
  // products in LDS; lanes 0 and 32 take the value elements they own and
  // lane 0 counts the weight
  if (holds_new && wave == 0) {
    float prod = kqs[lane];
    if (lane + 64 < D) prod += kqs[lane + 64];
    const float sc = wave_sum(prod) * qscale;
    const float p = weigh(sc);
    if (lane == 0) l += p;
    if constexpr (X::WEIGHTS)
      if (lane == 0) keep_score(x, (int64_t)bh * L_cap, n, sc);
    if (kr == 0) {
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[8 * kk + j] = p * vs[16 * kk + 8 * h + j];
      }
    }
  }

  // blocks wave, wave + NW are in flight; each computed buffer is refilled
  // with the block 2 NW further on.  The steady state loads without a
  // condition, so each buffer is written in place and the loop carries no
  // register copies (a copy would have to wait for its load to land).
  int i = wave;
  for (; i + 3 * NW < nblk; i += 2 * NW) {
    compute(i, kA, vA);
    load_blk(i + 2 * NW, kA, vA);
    compute(i + NW, kB, vB);
    load_blk(i + 3 * NW, kB, vB);
  }
  // at most three blocks remain: i and i + NW in flight, i + 2 NW to load
  if (i < nblk) {
    compute(i, kA, vA);
    if (i + 2 * NW < nblk) load_blk(i + 2 * NW, kA, vA);
  }
  if (i + NW < nblk) compute(i + NW, kB, vB);
  if (i + 2 * NW < nblk) compute(i + 2 * NW, kA, vA);

  OldSums old;
  if constexpr (FINAL && X::WEIGHTS) old.load(x, (int64_t)bh * L_cap, n, tid, THREADS);
  PrefixParts<D> pre;
  if constexpr (FINAL && X::PREFIX) pre.load(x, bh, min(tid, D - 1), 0);
  // wave partials: l over the wave, values over each half-wave
  l = wave_sum(l);
  int base = 0;
  half_wave_reduce<NA, 16>(acc, lane, base);
  constexpr int NF = half_wave_count<NA, 16>();
  __shared__ float sm[NW], sl[NW];
  __shared__ float sacc[NW][D];
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    const int a = base + j;
    sacc[wave][16 * (a / 8) + 8 * h + a % 8] = acc[j];
  }
  if (lane == 0) { sm[wave] = M; sl[wave] = l; }
  __syncthreads();
  if (X::WEIGHTS || tid < D) {  // with weights every thread takes the maximum and the sum
    const int e = min(tid, D - 1);
    float Mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) Mx = fmaxf(Mx, sm[w]);
    float Ls = 0.f, ov = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = exp2f(sm[w] - Mx);
      const bool any = sm[w] != -INFINITY;  // the wave had a row
      Ls += any ? sl[w] * f : 0.f;
      ov += any ? sacc[w][e] * f : 0.f;
    }
    if constexpr (FINAL && X::PREFIX) pre.join(x, bh, tid, Mx, Ls, ov);
    if constexpr (FINAL && X::WEIGHTS)
      add_weights(x, (int64_t)bh * L_cap, n, 0, rows, Mx, Ls, tid, THREADS, old);
    if (tid >= D) {
    } else if constexpr (FINAL) {
      o[(int64_t)bh * D + tid] = f32_to_bf16(ov / Ls);
    } else {
      float* out = part + ((int64_t)bh * n_chunk_max + chunk) * (D + 2);
      out[2 + tid] = ov;
      if (tid == 0) { out[0] = Mx; out[1] = Ls; }
    }
  }
}

// whether one workgroup per slice writes the output (no partials)
static bool one_workgroup(bool bf16, int64_t slices, int L_cap) {
  if (slices >= DEC_SINGLE_MIN) return true;
  return bf16 && L_cap <= std::min<int64_t>(DEC_ONE_ROWS + DEC_ONE_ROWS_PER_SLICE * slices,
                                            DEC_ONE_MAX_ROWS);
}

static int n_chunks(int L_cap) { return (L_cap + DEC_CH - 1) / DEC_CH; }

template <typename T, int D, typename X = StepOnly>
static int launch_decode(const void* q, const void* k_new, const void* v_new, void* k_cache,
                         void* v_cache, const int32_t* kv_len, const int32_t* cur_tok,
                         const int32_t* vu, const int32_t* pos, int32_t L_meta, void* o,
                         int32_t b, int32_t H, int32_t L_cap, float scale, float theta,
                         void* ws, size_t ws_bytes, int32_t* status, hipStream_t stream,
                         int32_t ring = 0, X x = X()) {
  RopeTab tab;
  for (int i = 0; i < 40; ++i) tab.w[i] = 0.0;
  const int rotate = theta > 0.f ? 1 : 0;
  if (rotate)
    for (int i = 0; i < D / 2; ++i) tab.w[i] = std::pow((double)theta, -2.0 * i / D);
  float* part = static_cast<float*>(ws);
  const T* qq = static_cast<const T*>(q);
  const T* kn = static_cast<const T*>(k_new);
  const T* vn = static_cast<const T*>(v_new);
  T* kc = static_cast<T*>(k_cache);
  T* vc = static_cast<T*>(v_cache);
  T* out = static_cast<T*>(o);
  const float qs = scale * LOG2E;
  const int slices = b * H;
  const FastDiv by_H = make_div((uint32_t)H), by_slices = make_div((uint32_t)slices);
  size_t lds = 0;
  // scores in LDS where all workgroups that a CU holds (`waves` of `of`) fit
  auto room = [&](int waves, int of) {
    if constexpr (X::WEIGHTS) {
      const size_t need = (size_t)L_cap * sizeof(float);
      x.in_lds = need <= (64 << 10) && need * (of / waves) <= SCORE_LDS;
      lds = x.in_lds ? need : 0;
    }
  };
  if (one_workgroup(sizeof(T) == 2, slices, L_cap)) {
    const bool narrow = slices >= DEC_NARROW_MIN;
    if constexpr (sizeof(T) == 2) {
      int cus = 0;
      const int rc = device_cus(&cus);
      if (rc) return rc;
      const int64_t slots = (int64_t)cus * 4 * DEC_WAVES_PER_SIMD;  // resident waves
      const int nw = (int64_t)slices * 4 <= slots   ? 4
                     : (int64_t)slices * 2 <= slots ? 2
                     : slices <= slots              ? (D <= 64 ? 1 : 2)
                                                    : 4;
      // A cache of at least DEC_SPEC2_ROWS rows per wave of a slice is taken
      // to hold long slices: both first blocks of every wave are then read
      // before the slice length arrives (rows past a shorter slice are read
      // for nothing, never used).
      const bool spec2 = ring == 0 && (int64_t)L_cap >= (int64_t)DEC_SPEC2_ROWS * nw;
      room(nw, 4 * DEC_WAVES_PER_SIMD);
#define SCKV_DECODE_LAUNCH(DD, NWW, SP)                                                          \
  decode_mfma_kernel<DD, NWW, true, SP, X><<<slices, NWW * 64, lds, stream>>>(                    \
      qq, kn, vn, kc, vc, kv_len, cur_tok, vu, pos, L_meta, H, L_cap, qs, rotate, tab, part, 1,  \
      by_H, by_slices, slices, Split{1, 1}, out, status, ring, x)
      constexpr int D1 = D <= 64 ? D : 64;  // nw == 1 only where D <= 64
      if (nw == 1 && spec2) SCKV_DECODE_LAUNCH(D1, 1, true);
      else if (nw == 1) SCKV_DECODE_LAUNCH(D1, 1, false);
      else if (nw == 2 && spec2) SCKV_DECODE_LAUNCH(D, 2, true);
      else if (nw == 2) SCKV_DECODE_LAUNCH(D, 2, false);
      else if (spec2) SCKV_DECODE_LAUNCH(D, 4, true);
      else SCKV_DECODE_LAUNCH(D, 4, false);
#undef SCKV_DECODE_LAUNCH
    } else {
      room(narrow ? 4 : 8, 24);
      if (narrow)
        decode_chunk_kernel<T, D, 256, true, X><<<slices, 256, lds, stream>>>(
            qq, kn, vn, kc, vc, kv_len, cur_tok, vu, pos, L_meta, H, L_cap, qs, rotate, tab, part,
            1, slices, Split{1, 1}, out, status, x);
      else
        decode_chunk_kernel<T, D, 512, true, X><<<slices, 512, lds, stream>>>(
            qq, kn, vn, kc, vc, kv_len, cur_tok, vu, pos, L_meta, H, L_cap, qs, rotate, tab, part,
            1, slices, Split{1, 1}, out, status, x);
    }
    return hip_check(hipGetLastError(), "compacted_decode_attn: launch");
  }
  // the caller's workspace holds at least n_chunks(L_cap) partials a slice
  // (checked); a larger one lets a launch of few slices split them finer
  const int fit = (int)std::min<size_t>(ws_bytes / ((size_t)slices * (D + 2) * sizeof(float)), 0x7fffffff);
  const int want = std::max(1, DEC_FILL / slices);
  const int nc = std::min(fit, std::max(n_chunks(L_cap), std::min(want, (L_cap + DEC_CH_MIN - 1) / DEC_CH_MIN)));
  const Split sp{want, nc};
  const int n_work = slices * nc;
  if constexpr (sizeof(T) == 2)
    decode_mfma_kernel<D, 4, false, false, X><<<n_work, 256, 0, stream>>>(
        qq, kn, vn, kc, vc, kv_len, cur_tok, vu, pos, L_meta, H, L_cap, qs, rotate, tab, part, nc,
        by_H, by_slices, slices, sp, out, status, ring, x);
  else
    decode_chunk_kernel<T, D, DEC_THREADS, false, X><<<n_work, DEC_THREADS, 0, stream>>>(
        qq, kn, vn, kc, vc, kv_len, cur_tok, vu, pos, L_meta, H, L_cap, qs, rotate, tab, part, nc,
        n_work, sp, out, status, x);
  int rc = hip_check(hipGetLastError(), "compacted_decode_attn: chunk launch");
  if (rc) return rc;
  const int wblk = X::WEIGHTS ? (int)((L_cap + (int64_t)WEIGHT_ROWS - 1) / WEIGHT_ROWS) : 0;
  decode_combine_kernel<T, D, X><<<slices * (1 + wblk), 64 * COMBINE_WAVES, 0, stream>>>(
      vn, kv_len, cur_tok, vu, L_meta, H, by_H, L_cap, part, nc, sp, out, status, ring, slices, x);
  return hip_check(hipGetLastError(), "compacted_decode_attn: combine launch");
}

}  // namespace sckv

using namespace sckv;

extern "C" size_t sckv_decode_workspace_bytes(int32_t b, int32_t H, int32_t L_cap, int32_t d_head) {
  if (b <= 0 || H <= 0 || L_cap <= 0 || d_head <= 0) return 0;
  return (size_t)b * H * n_chunks(L_cap) * (d_head + 2) * sizeof(float);
}

extern "C" int local_decode_attn(const void* q, const void* k_new, const void* v_new,
                                 void* k_cache, void* v_cache, int32_t W, const int32_t* cur_tok,
                                 const int32_t* vu, const int32_t* pos, int32_t L_meta, void* o,
                                 int32_t b, int32_t H, int32_t L_cap, int32_t d_head,
                                 sckv_dtype dt, float scale, float rope_theta, void* ws,
                                 size_t ws_bytes, int32_t* status, hipStream_t stream) {
  clear_error();
  if (!q || !k_new || !v_new || !k_cache || !v_cache || !cur_tok || !vu || !o || !ws)
    return fail(SCKV_EINVAL, "local_decode_attn: null pointer");
  if (dt != SCKV_BF16) return fail(SCKV_EUNSUP, "local_decode_attn: bf16 only");
  if (!supported_d(d_head)) return fail(SCKV_EUNSUP, "local_decode_attn: d_head must be 64 or 80");
  // W < L_cap: the W ring rows and the new token make W + 1 <= L_cap rows of
  // work, the most the launch and the workspace are sized for
  if (b <= 0 || H <= 0 || L_cap <= 0 || L_meta <= 0 || W <= 0 || W >= L_cap)
    return fail(SCKV_EINVAL, "local_decode_attn: need 0 < W < L_cap and positive sizes");
  if ((int64_t)b * H * n_chunks(L_cap) > 0x7fffffff)
    return fail(SCKV_EUNSUP, "local_decode_attn: b*H*chunks too large");
  if (!(scale > 0.f) || std::isinf(scale)) return fail(SCKV_EINVAL, "local_decode_attn: scale must be finite and > 0");
  if (!(rope_theta >= 0.f) || std::isinf(rope_theta))
    return fail(SCKV_EINVAL, "local_decode_attn: rope_theta must be finite and >= 0");
  if (rope_theta > 0.f && !pos) return fail(SCKV_EINVAL, "local_decode_attn: null pos");
  if (ws_bytes < sckv_decode_workspace_bytes(b, H, L_cap, d_head))
    return fail(SCKV_EINVAL, "local_decode_attn: workspace too small");
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) ||
      !aligned16(v_cache) || !aligned16(o) || !aligned16(ws))
    return fail(SCKV_EINVAL, "local_decode_attn: buffers must be 16-byte aligned");
  const int32_t* p = pos ? pos : vu;
  return d_head == 64
             ? launch_decode<uint16_t, 64>(q, k_new, v_new, k_cache, v_cache, nullptr, cur_tok, vu, p, L_meta, o, b, H, L_cap, scale, rope_theta, ws, ws_bytes, status, stream, W)
             : launch_decode<uint16_t, 80>(q, k_new, v_new, k_cache, v_cache, nullptr, cur_tok, vu, p, L_meta, o, b, H, L_cap, scale, rope_theta, ws, ws_bytes, status, stream, W);
}

// Host checks of compacted_decode_attn and its allocation-free variant
// (everything but the workspace); no HIP call is made here.
static int decode_checks(const char* W, const void* q, const void* k_new, const void* v_new,
                         const void* k_cache, const void* v_cache, const int32_t* kv_len,
                         const int32_t* cur_tok, const int32_t* vu, const int32_t* pos,
                         int32_t L_meta, const void* o, int32_t b, int32_t H, int32_t L_cap,
                         int32_t d_head, sckv_dtype dt, float scale, float rope_theta) {
  const std::string w(W);
  if (!q || !k_new || !v_new || !k_cache || !v_cache || !kv_len || !cur_tok || !vu || !o)
    return fail(SCKV_EINVAL, w + ": null pointer");
  if (!valid_dtype(dt)) return fail(SCKV_EINVAL, w + ": unknown dtype");
  if (!supported_d(d_head)) return fail(SCKV_EUNSUP, w + ": d_head must be 64 or 80");
  if (b <= 0 || H <= 0 || L_cap <= 0 || L_meta <= 0)
    return fail(SCKV_EINVAL, w + ": sizes must be positive");
  if ((int64_t)b * H * n_chunks(L_cap) > 0x7fffffff)
    return fail(SCKV_EUNSUP, w + ": b*H*chunks too large");
  if (!(scale > 0.f) || std::isinf(scale)) return fail(SCKV_EINVAL, w + ": scale must be finite and > 0");
  if (!(rope_theta >= 0.f) || std::isinf(rope_theta))
    return fail(SCKV_EINVAL, w + ": rope_theta must be finite and >= 0");
  if (rope_theta > 0.f && !pos) return fail(SCKV_EINVAL, w + ": null pos");
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) ||
      !aligned16(v_cache) || !aligned16(o))
    return fail(SCKV_EINVAL, w + ": buffers must be 16-byte aligned");
  return SCKV_OK;
}

template <typename X = StepOnly>
static int decode_dispatch(const void* q, const void* k_new, const void* v_new, void* k_cache,
                           void* v_cache, const int32_t* kv_len, const int32_t* cur_tok,
                           const int32_t* vu, const int32_t* pos, int32_t L_meta, void* o,
                           int32_t b, int32_t H, int32_t L_cap, int32_t d_head, sckv_dtype dt,
                           float scale, float rope_theta, void* ws, size_t ws_bytes,
                           int32_t* status, hipStream_t stream, X x = X()) {
  const int32_t* p = pos ? pos : vu;  // pos is read only when rotating
#define SCKV_DISPATCH(T, DD)                                                                       \
  launch_decode<T, DD, X>(q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, p, L_meta, o, b, \
                          H, L_cap, scale, rope_theta, ws, ws_bytes, status, stream, 0, x)
  if (dt == SCKV_BF16) return d_head == 64 ? SCKV_DISPATCH(uint16_t, 64) : SCKV_DISPATCH(uint16_t, 80);
  return d_head == 64 ? SCKV_DISPATCH(float, 64) : SCKV_DISPATCH(float, 80);
#undef SCKV_DISPATCH
}

extern "C" int compacted_decode_attn(const void* q, const void* k_new, const void* v_new,
                                     void* k_cache, void* v_cache, const int32_t* kv_len,
                                     const int32_t* cur_tok, const int32_t* vu,
                                     const int32_t* pos, int32_t L_meta, void* o, int32_t b,
                                     int32_t H, int32_t L_cap, int32_t d_head, sckv_dtype dt,
                                     float scale, float rope_theta, void* ws, size_t ws_bytes,
                                     int32_t* status, hipStream_t stream) {
  clear_error();
  const char* W = "compacted_decode_attn";
  int rc = decode_checks(W, q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos, L_meta,
                         o, b, H, L_cap, d_head, dt, scale, rope_theta);
  if (rc) return rc;
  if (!ws) return fail(SCKV_EINVAL, "compacted_decode_attn: null pointer");
  if (ws_bytes < sckv_decode_workspace_bytes(b, H, L_cap, d_head))
    return fail(SCKV_EINVAL, "compacted_decode_attn: workspace too small");
  if (!aligned16(ws)) return fail(SCKV_EINVAL, "compacted_decode_attn: buffers must be 16-byte aligned");
  return decode_dispatch(q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos, L_meta, o, b,
                         H, L_cap, d_head, dt, scale, rope_theta, ws, ws_bytes, status, stream);
}

// ---------------------------------------------------------------------------
// The same decode step without any allocation: the split-K partials go to a
// file-scope device array instead of a caller workspace.  Each device that
// runs the library holds its own copy of the array from module load until
// the process ends; its device address is looked up once per device (the
// array's name in host code is only a stand-in for that address) and kept.
// Every call on a device shares that device's array and leaves its partials
// in it; nothing in it has to start at zero (the merge reads only the chunk
// partials the same call wrote).  Calls that overlap on one device race.
// ---------------------------------------------------------------------------
static __device__ __align__(256) char scratch[SCKV_NOALLOC_SCRATCH_BYTES];

constexpr int NOALLOC_MAX_DEVICES = 64;
static std::mutex g_scratch_mu;
static void* g_scratch_ptr[NOALLOC_MAX_DEVICES];  // per device, set once

static int scratch_address(void** out) {
  int dev = -1;
  int rc = hip_check(hipGetDevice(&dev), "compacted_decode_attn_noalloc: hipGetDevice");
  if (rc) return rc;
  if (dev < 0 || dev >= NOALLOC_MAX_DEVICES)
    return fail(SCKV_EUNSUP, "compacted_decode_attn_noalloc: device index above 63");
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    rc = hip_check(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)),
                   "compacted_decode_attn_noalloc: hipGetSymbolAddress(scratch)");
    if (rc) return rc;
    if (!p || !aligned16(p))
      return fail(SCKV_EHIP, "compacted_decode_attn_noalloc: scratch array has no usable address");
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return SCKV_OK;
}

extern "C" int compacted_decode_attn_noalloc(const void* q, const void* k_new, const void* v_new,
                                             void* k_cache, void* v_cache, const int32_t* kv_len,
                                             const int32_t* cur_tok, const int32_t* vu,
                                             const int32_t* pos, int32_t L_meta, void* o,
                                             int32_t b, int32_t H, int32_t L_cap, int32_t d_head,
                                             sckv_dtype dt, float scale, float rope_theta,
                                             int32_t* status, hipStream_t stream) {
  clear_error();
  const char* W = "compacted_decode_attn_noalloc";
  int rc = decode_checks(W, q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos, L_meta,
                         o, b, H, L_cap, d_head, dt, scale, rope_theta);
  if (rc) return rc;
  // only a split launch writes partials; it splits as with the least workspace,
  // whose outputs it gives bit for bit
  const size_t need = one_workgroup(dt == SCKV_BF16, (int64_t)b * H, L_cap)
                          ? 0 : sckv_decode_workspace_bytes(b, H, L_cap, d_head);
  if (need > SCKV_NOALLOC_SCRATCH_BYTES)
    return fail(SCKV_EUNSUP, std::string(W) + ": the split-K partials need " +
                                 std::to_string(need) + " bytes, more than the " +
                                 std::to_string((size_t)SCKV_NOALLOC_SCRATCH_BYTES) +
                                 "-byte scratch array (use compacted_decode_attn with a workspace)");
  void* ws = nullptr;
  rc = scratch_address(&ws);
  if (rc) return rc;
  return decode_dispatch(q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos, L_meta, o, b,
                         H, L_cap, d_head, dt, scale, rope_theta, ws, need, status, stream);
}

// ---------------------------------------------------------------------------
// the step that also adds its weights; ws: chunk partials, then the scores
// ---------------------------------------------------------------------------
// Bytes of the partials: what a split launch needs at least, and room for the
// DEC_FILL workgroups that a launch of few slices is cut into.
static size_t partial_bytes(int32_t b, int32_t H, int32_t L_cap, int32_t d_head) {
  const size_t fine = (size_t)DEC_FILL * (d_head + 2) * sizeof(float);
  return (std::max(sckv_decode_workspace_bytes(b, H, L_cap, d_head), fine) + 15) / 16 * 16;
}

extern "C" size_t sckv_decode_weights_workspace_bytes(int32_t b, int32_t H, int32_t L_cap,
                                                      int32_t d_head) {
  if (b <= 0 || H <= 0 || L_cap <= 0 || d_head <= 0) return 0;
  return partial_bytes(b, H, L_cap, d_head) + (size_t)b * H * L_cap * sizeof(float);
}

extern "C" int compacted_decode_attn_weights(
    const void* q, const void* k_new, const void* v_new, void* k_cache, void* v_cache,
    const int32_t* kv_len, const int32_t* cur_tok, const int32_t* vu, const int32_t* pos,
    int32_t L_meta, void* o, const float* w_in, float* w_out, int32_t b, int32_t H, int32_t L_cap,
    int32_t d_head, sckv_dtype dt, float scale, float rope_theta, void* ws, size_t ws_bytes,
    int32_t* status, hipStream_t stream) {
  clear_error();
  const std::string W = "compacted_decode_attn_weights";
  const int rc = decode_checks(W.c_str(), q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu,
                               pos, L_meta, o, b, H, L_cap, d_head, dt, scale, rope_theta);
  if (rc) return rc;
  if (!w_out || !ws) return fail(SCKV_EINVAL, W + ": null pointer");
  if (!aligned4(w_out) || !aligned4(w_in))
    return fail(SCKV_EINVAL, W + ": w_in and w_out must be 4-byte aligned");
  if (!aligned16(ws)) return fail(SCKV_EINVAL, W + ": buffers must be 16-byte aligned");
  if (ws_bytes < sckv_decode_weights_workspace_bytes(b, H, L_cap, d_head))
    return fail(SCKV_EINVAL, W + ": workspace too small");
  const size_t part = partial_bytes(b, H, L_cap, d_head);
  const StepWeights x = {w_in, w_out, reinterpret_cast<float*>(static_cast<char*>(ws) + part), 0};
  return decode_dispatch(q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos, L_meta, o, b,
                         H, L_cap, d_head, dt, scale, rope_theta, ws, part, status, stream, x);
}

// ---------------------------------------------------------------------------
// the step behind shared prefixes; ws: chunk partials of the own rows, then
// the prefixes' partials
// ---------------------------------------------------------------------------
// (the size function is not told the element type)
static int most_chunks(int32_t d, int32_t n_prefix, int32_t H, int32_t per, int32_t P_cap) {
  return std::max(prefix_chunks(true, d, n_prefix, H, per, P_cap),
                  prefix_chunks(false, d, n_prefix, H, per, P_cap));
}

extern "C" size_t sckv_shared_decode_workspace_bytes(int32_t b, int32_t H, int32_t n_prefix,
                                                     int32_t P_cap, int32_t L_cap,
                                                     int32_t d_head) {
  if (b <= 0 || H <= 0 || n_prefix <= 0 || P_cap <= 0 || L_cap <= 0 || d_head <= 0 || b % n_prefix)
    return 0;
  return partial_bytes(b, H, L_cap, d_head) +
         (size_t)b * H * most_chunks(d_head, n_prefix, H, b / n_prefix, P_cap) * (d_head + 2) * sizeof(float);
}

extern "C" int shared_prefix_decode_attn(
    const void* q, const void* k_new, const void* v_new, const void* k_prefix,
    const void* v_prefix, const int32_t* prefix_len, int32_t n_prefix, int32_t P_cap,
    void* k_cache, void* v_cache, const int32_t* kv_len, const int32_t* cur_tok,
    const int32_t* vu, const int32_t* pos, int32_t L_meta, void* o, int32_t b, int32_t H,
    int32_t L_cap, int32_t d_head, sckv_dtype dt, float scale, float rope_theta, void* ws,
    size_t ws_bytes, int32_t* status, hipStream_t stream) {
  clear_error();
  const std::string W = "shared_prefix_decode_attn";
  int rc = decode_checks(W.c_str(), q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos,
                         L_meta, o, b, H, L_cap, d_head, dt, scale, rope_theta);
  if (rc) return rc;
  if (!k_prefix || !v_prefix || !prefix_len || !ws) return fail(SCKV_EINVAL, W + ": null pointer");
  if (n_prefix <= 0 || P_cap <= 0 || b % n_prefix)
    return fail(SCKV_EINVAL, W + ": b must be a multiple of n_prefix, sizes positive");
  if (!aligned16(k_prefix) || !aligned16(v_prefix) || !aligned16(ws))
    return fail(SCKV_EINVAL, W + ": buffers must be 16-byte aligned");
  if (ws_bytes < sckv_shared_decode_workspace_bytes(b, H, n_prefix, P_cap, L_cap, d_head))
    return fail(SCKV_EINVAL, W + ": workspace too small");
  const size_t own = partial_bytes(b, H, L_cap, d_head);
  const int n = prefix_chunks(dt == SCKV_BF16, d_head, n_prefix, H, b / n_prefix, P_cap);
  float* po = reinterpret_cast<float*>(static_cast<char*>(ws) + own);
  float* ml = po + (size_t)b * H * n * d_head;
  rc = launch_prefix(q, k_prefix, v_prefix, prefix_len, n_prefix, P_cap, cur_tok, pos ? pos : vu,
                     L_meta, b, H, d_head, dt, scale, rope_theta, po, ml, stream);
  if (rc) return rc;
  const StepPrefix x = {po, reinterpret_cast<const float2*>(ml), n};
  return decode_dispatch(q, k_new, v_new, k_cache, v_cache, kv_len, cur_tok, vu, pos, L_meta, o, b,
                         H, L_cap, d_head, dt, scale, rope_theta, ws, own, status, stream, x);
}
