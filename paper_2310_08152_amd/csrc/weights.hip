// Accumulated attention weight of cache rows (what eviction goes by): the sum
// over queries of the softmax weight that each gives a row, under the mask of
// Section 3.1.
//
//   w[r] += sum_i exp2(c q_i.k_r - lse_i),  lse_i = log2 sum_r exp2(c q_i.k_r)
//
// with c = scale * log2(e).  A row's sum needs every query's normaliser first,
// so the scores S^T = K Q^T are multiplied twice, on the matrix cores:
//   stats : a wave keeps a tile of queries in registers, reads key tiles and
//           holds each query's maximum and sum;
//   sums  : a wave keeps a tile of keys, reads query tiles and adds up the
//           weights of each row; the 32 queries of a tile meet once, at the end.
// Keeping the scores instead would write and read nq * 4 bytes a row, more
// than the 2 d of a bf16 key from 32 queries (d = 64) on.
//
//   plan  : the rows of each sequence in the order they are multiplied.  A row
//           is seen by the queries from its token to its vu, so rows are listed
//           by class: those that every later query sees; those enclosed by a
//           span that closes among the queries; those none sees (a <CL>,
//           rows freed before the first query, rows of later tokens).  Tiles
//           of 32 rows then are mostly seen whole or not at all: a tile's
//           least and greatest token and vu tell, and only mixed tiles are
//           masked by the element.
// A <CL> query gives its own row weight 1 and has no sum: it then gives the
// others exactly 0.
#include <algorithm>
#include <cmath>
#include <string>

#include "sckv_common.h"

namespace sckv {

constexpr float W_LOG2E = 1.4426950408889634f;
constexpr float W_RESCALE = 8.f;  // lazy maximum, log2 units
constexpr int W_TILE = 32;        // rows, or queries, of a tile
constexpr int W_CLASS = 64;       // classes of the list start at multiples of this
constexpr int W_CL = 1 << 20;     // list entry: a <CL> row among the queries' tokens

// ---------------------------------------------------------------------------
// plan
// ---------------------------------------------------------------------------
struct TileSum {
  int32_t tmin, tmax, vmin, vmax;  // tokens and vu of a tile's rows
};
struct WeightPlan {
  int32_t *row, *tok, *vu;  // [b][entries]
  TileSum* sum;             // [b][entries / W_TILE]
  int2* tiles;              // [b]: tiles that some query sees, all tiles
  int32_t entries;
};

// entries of a sequence's list: every row, and each class up to W_CLASS - 1 more
static int64_t plan_entries(int32_t L_cap) {
  return ((int64_t)L_cap + W_CLASS - 1) / W_CLASS * W_CLASS + 3 * W_CLASS;
}
static size_t plan_bytes(int32_t b, int32_t L_cap) {
  const size_t e = (size_t)plan_entries(L_cap);
  return (size_t)b * (3 * e * 4 + e / W_TILE * sizeof(TileSum) + 16);
}
static WeightPlan plan_at(void* ws, int32_t b, int32_t L_cap) {
  const size_t e = (size_t)plan_entries(L_cap);
  WeightPlan p;
  p.entries = (int32_t)e;
  p.row = static_cast<int32_t*>(ws);
  p.tok = p.row + (size_t)b * e;
  p.vu = p.tok + (size_t)b * e;
  p.sum = reinterpret_cast<TileSum*>(p.vu + (size_t)b * e);
  p.tiles = reinterpret_cast<int2*>(p.sum + (size_t)b * (e / W_TILE));
  return p;
}

constexpr int PLAN_WAVES = 16;
constexpr int PLAN_U = 4;  // rows of a thread in flight
constexpr int PLAN_THREADS = 64 * PLAN_WAVES;

__global__ __launch_bounds__(PLAN_THREADS) void weight_plan_kernel(
    WeightPlan p, const int32_t* __restrict__ vu, int32_t L_meta, int32_t tok0, int32_t nq,
    const int32_t* __restrict__ kv_len, const int32_t* __restrict__ tok_idx, int32_t L_cap) {
  constexpr int CHUNK = PLAN_THREADS * PLAN_U;
  static_assert(PLAN_U * PLAN_WAVES == 64, "one wave scans the counts of a class");
  // rows of class k that pass u of wave w holds, then those before them, at
  // [k][u * PLAN_WAVES + w]; the chunk's total behind them
  __shared__ int before[3][65];
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(kv_len[s], 0), L_cap);
  const int32_t* toks = tok_idx + (int64_t)s * L_cap;
  const int32_t* vus = vu + (int64_t)s * L_meta;
  const int64_t at = (int64_t)s * p.entries;
  const int last = tok0 + nq - 1;  // last query's token
  // classes: 0 seen by every later query, 1 by some, 2 by none (3: no row)
  int j[PLAN_U], v[PLAN_U], c[PLAN_U];
  uint64_t m[3][PLAN_U];
  auto classify = [&](int base) {
#pragma unroll
    for (int u = 0; u < PLAN_U; ++u) j[u] = toks[min(base + u * PLAN_THREADS + tid, n - 1)];
#pragma unroll
    for (int u = 0; u < PLAN_U; ++u) v[u] = vus[min(max(j[u], 0), L_meta - 1)];
#pragma unroll
    for (int u = 0; u < PLAN_U; ++u) {
      const bool none = j[u] < 0 || j[u] >= L_meta || v[u] == j[u] || j[u] > last || v[u] < tok0 || nq == 0;
      c[u] = base + u * PLAN_THREADS + tid >= n ? 3 : none ? 2 : v[u] >= last ? 0 : 1;
#pragma unroll
      for (int k = 0; k < 3; ++k) m[k][u] = __ballot(c[u] == k);
    }
  };
  // a chunk's counts become exclusive prefix sums
  auto scan = [&]() {
    __syncthreads();  // those of the chunk before have been read
#pragma unroll
    for (int u = 0; u < PLAN_U; ++u) {
      const int x0 = __popcll(m[0][u]), x1 = __popcll(m[1][u]), x2 = __popcll(m[2][u]);
      if (lane < 3) before[lane][u * PLAN_WAVES + wave] = lane == 0 ? x0 : lane == 1 ? x1 : x2;
    }
    __syncthreads();
    if (wave < 3) {
      const int x = before[wave][lane];
      int sum = x;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(sum, off, 64);
        if (lane >= off) sum += y;
      }
      before[wave][lane] = sum - x;
      if (lane == 63) before[wave][64] = sum;
    }
    __syncthreads();
  };
  // rows of each class
  int total[3] = {0, 0, 0};
  for (int base = 0; base < n; base += CHUNK) {
    classify(base);
    scan();
#pragma unroll
    for (int k = 0; k < 3; ++k) total[k] += before[k][64];
  }
  int start = 0, first[3], done[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    first[k] = done[k] = start;
    start += (total[k] + W_CLASS - 1) / W_CLASS * W_CLASS;
  }
  // the rows, in order within each class
  for (int base = 0; base < n; base += CHUNK) {
    if (n > CHUNK) {  // (else they are still held)
      classify(base);
      scan();
    }
#pragma unroll
    for (int u = 0; u < PLAN_U; ++u)
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (c[u] == k) {
          const int row = base + u * PLAN_THREADS + tid;
          const bool cl = k == 2 && v[u] == j[u] && j[u] >= tok0 && j[u] <= last;
          const int64_t e = at + done[k] + before[k][u * PLAN_WAVES + wave] + mask_rank(m[k][u]);
          p.row[e] = cl ? row | W_CL : row;
          p.tok[e] = j[u];
          p.vu[e] = k == 2 ? -1 : v[u];
        }
#pragma unroll
    for (int k = 0; k < 3; ++k) done[k] += before[k][64];
  }
  // what fills a class's last tiles: row -1, seen by none
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int end = k < 2 ? first[k + 1] : start;
    for (int e = first[k] + total[k] + tid; e < end; e += PLAN_THREADS) {
      p.row[at + e] = -1;
      p.tok[at + e] = 0x7fffffff;
      p.vu[at + e] = -1;
    }
  }
  __threadfence_block();
  __syncthreads();
  const int tiles = start / W_TILE;
  for (int t = tid / 32; t < tiles; t += PLAN_THREADS / 32) {
    const int j = p.tok[at + t * W_TILE + (tid & 31)], v = p.vu[at + t * W_TILE + (tid & 31)];
    TileSum x = {j, j, v, v};
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      x.tmin = min(x.tmin, __shfl_xor(x.tmin, off, 64));
      x.tmax = max(x.tmax, __shfl_xor(x.tmax, off, 64));
      x.vmin = min(x.vmin, __shfl_xor(x.vmin, off, 64));
      x.vmax = max(x.vmax, __shfl_xor(x.vmax, off, 64));
    }
    if ((tid & 31) == 0) p.sum[(int64_t)s * (p.entries / W_TILE) + t] = x;
  }
  if (tid == 0) p.tiles[s] = make_int2(first[2] / W_TILE, tiles);
}

// ---------------------------------------------------------------------------
// products of a 32-row and a 32-query tile: the lane holds its row's (query's)
// elements 16 i + 8 (l/32) .. + 7 in bf16, 8 i + 4 (l/32) .. + 3 in fp32, of
// row (query) l % 32, which is an MFMA operand either way (the order in which
// the products are summed is the same for both operands).  Register v of the
// result is row 8 (v/4) + 4 (l/32) + v % 4, query l % 32.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct Operand {
  static constexpr int N = sizeof(T) == 2 ? D / 16 : D / 8;
  u32x4 x[N];
  __device__ __forceinline__ void load(const T* row, int h) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = ld16(row + (D / N) * i + (D / N / 2) * h);
  }
};
template <typename T, int D>
__device__ __forceinline__ f32x16 scores(const Operand<T, D>& k, const Operand<T, D>& q) {
  f32x16 s;
#pragma unroll
  for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
  for (int i = 0; i < Operand<T, D>::N; ++i) {
    if constexpr (sizeof(T) == 2) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k.x[i]),
                                                  __builtin_bit_cast(bf16x8, q.x[i]), s, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.x[i][j]),
                                                 __uint_as_float(q.x[i][j]), s, 0, 0, 0);
    }
  }
  return s;
}

// scores of rows that token t does not see become -inf (whatever they were)
__device__ __forceinline__ void mask_scores(f32x16& s, const int32_t* tok, const int32_t* vu, int t,
                                            int h) {
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int4 j = *reinterpret_cast<const int4*>(tok + 8 * a + 4 * h);
    const int4 v = *reinterpret_cast<const int4*>(vu + 8 * a + 4 * h);
    const int js[4] = {j.x, j.y, j.z, j.w}, vs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) s[4 * a + e] = js[e] <= t && t <= vs[e] ? s[4 * a + e] : -INFINITY;
  }
}

__device__ __forceinline__ float other_half(float x, bool sum) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
  return sum ? a + b : fmaxf(a, b);
}

constexpr int W_WAVES = 4;

// ---------------------------------------------------------------------------
// stats: (maximum, sum) of each query over the rows of one of `splits` shares
// of its slice's tiles.  A unit is a wave: QT tiles of queries, one share; the
// waves of a workgroup are units next to one another, which read the same keys.
// ---------------------------------------------------------------------------
template <typename T, int D, int QT>
__global__ __launch_bounds__(64 * W_WAVES) void weight_stats_kernel(
    const T* __restrict__ q, const T* __restrict__ k, WeightPlan p, float2* __restrict__ ml,
    int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float c, const int32_t* __restrict__ vu,
    int32_t L_meta, int32_t tok0, int32_t n_slice, int32_t qtiles, int32_t splits) {
  const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
  // a slice's workgroups are n_slice apart, so that they share an XCD's L2
  const int wg = blockIdx.x / n_slice, slice = blockIdx.x - wg * n_slice;
  const int unit = __builtin_amdgcn_readfirstlane(wg * W_WAVES + (threadIdx.x >> 6));
  if (unit >= qtiles * splits) return;
  const int split = unit / qtiles;
  const int qt = qtiles - 1 - (unit - split * qtiles);  // the last queries see most: first
  const int s = slice / H;
  const int q0 = qt * QT * W_TILE;
  const T* qb = q + slice * q_s;
  const T* kb = k + slice * k_s;
  const int64_t at = (int64_t)s * p.entries;
  const int32_t *rows = p.row + at, *toks = p.tok + at, *vus = p.vu + at;
  const TileSum* sums = p.sum + (int64_t)s * (p.entries / W_TILE);
  const int n_tiles = p.tiles[s].x;

  Operand<T, D> Q[QT];
  int t[QT], ta[QT], tb[QT];  // the lane's token; first and last of the tile's
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int i = q0 + W_TILE * x;
    t[x] = tok0 + min(i + l32, nq - 1);
    ta[x] = tok0 + i;  // past the last token: sees nothing below
    tb[x] = i < nq ? min(ta[x] + W_TILE - 1, tok0 + nq - 1) : -1;
    Q[x].load(qb + (int64_t)min(i + l32, nq - 1) * D, h);
  }
  float M[QT], l[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) { M[x] = -INFINITY; l[x] = 0.f; }

  // the share's tiles that some query of the wave sees, 64 candidates at a time
  const int lo = ta[0], hi = tb[0] > tb[QT - 1] ? tb[0] : tb[QT - 1];
  struct Ref {
    int t;
    TileSum s;
  };
  int cand = 0;
  uint64_t seen = 0;
  TileSum held = {0, 0, 0, 0};
  int held0 = 0;
  auto next = [&]() {
    while (seen == 0 && cand * splits + split < n_tiles) {
      const int tile = (cand + lane) * splits + split;
      held0 = cand;
      cand += 64;
      bool see = false;
      if (tile < n_tiles) {
        held = sums[tile];
        see = held.tmin <= hi && held.vmax >= lo;
      }
      seen = __ballot(see);
    }
    Ref r;
    r.t = -1;
    r.s = TileSum{0, 0, 0, 0};
    if (seen != 0) {
      const int i = __builtin_ctzll(seen);
      seen &= seen - 1;
      r.t = (held0 + i) * splits + split;
      r.s.tmin = __builtin_amdgcn_readlane(held.tmin, i);
      r.s.tmax = __builtin_amdgcn_readlane(held.tmax, i);
      r.s.vmin = __builtin_amdgcn_readlane(held.vmin, i);
      r.s.vmax = __builtin_amdgcn_readlane(held.vmax, i);
    }
    return r;
  };
  auto index = [&](const Ref& r) { return r.t >= 0 ? max(rows[r.t * W_TILE + l32], 0) : 0; };
  auto compute = [&](const Operand<T, D>& K, const Ref& r) {
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      if (r.s.tmin > tb[x] || r.s.vmax < ta[x]) continue;
      f32x16 sc = scores<T, D>(K, Q[x]);
      if (r.s.tmax > ta[x] || r.s.vmin < tb[x])
        mask_scores(sc, toks + r.t * W_TILE, vus + r.t * W_TILE, t[x], h);
      float mb = sc[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) mb = fmaxf(mb, sc[v]);
      mb = other_half(mb, false) * c;
      if (__any(mb > M[x] + W_RESCALE)) {
        const float mn = fmaxf(M[x], mb);
        l[x] = mn == -INFINITY ? 0.f : l[x] * fast_exp2(M[x] - mn);
        M[x] = mn;
      }
      const float m0 = M[x] == -INFINITY ? 0.f : M[x];  // a lane that saw no row yet
      float a0 = 0.f, a1 = 0.f;
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        a0 += fast_exp2(fmaf(sc[v], c, -m0));
        a1 += fast_exp2(fmaf(sc[v + 1], c, -m0));
      }
      l[x] += a0 + a1;
    }
  };

  // keys one tile ahead, their row numbers two
  Operand<T, D> A, B;
  Ref r0 = next();
  int i0 = index(r0);
  Ref r1 = next();
  int i1 = index(r1);
  A.load(kb + (int64_t)i0 * D, h);
  while (r0.t >= 0) {
    B.load(kb + (int64_t)i1 * D, h);
    const Ref r2 = next();
    const int i2 = index(r2);
    compute(A, r0);
    if (r1.t < 0) break;
    A.load(kb + (int64_t)i2 * D, h);
    const Ref r3 = next();
    const int i3 = index(r3);
    compute(B, r1);
    r0 = r2;
    r1 = r3;
    i1 = i3;
  }
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const float sum = other_half(l[x], true);
    const int i = q0 + W_TILE * x + l32;
    if (lane < 32 && i < nq) {
      const bool cl = vu[(int64_t)s * L_meta + t[x]] == t[x];
      ml[((int64_t)slice * splits + split) * nq + i] = cl ? make_float2(-INFINITY, 0.f) : make_float2(M[x], sum);
    }
  }
}

// ---------------------------------------------------------------------------
// sums: KT tiles of rows a wave.  WQ = 1: the workgroup's waves take key tiles
// of their own; WQ = W_WAVES: they share theirs and take every WQ-th tile of
// queries each (launches of few keys).
// ---------------------------------------------------------------------------
template <typename T, int D, int KT, int WQ>
__global__ __launch_bounds__(64 * W_WAVES) void weight_sums_kernel(
    const T* __restrict__ q, const T* __restrict__ k, WeightPlan p, const float2* __restrict__ ml,
    const float* w_in, float* w_out, int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float c,
    int32_t tok0, int32_t L_cap, int32_t n_slice, int32_t splits) {
  const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wg = blockIdx.x / n_slice, slice = blockIdx.x - wg * n_slice;
  const int s = slice / H;
  const int n_tiles = p.tiles[s].y;  // a multiple of two
  const int t0 = (wg * (W_WAVES / WQ) + (WQ == 1 ? wave : 0)) * KT;
  if (t0 >= n_tiles) return;  // (all waves of a workgroup alike where WQ > 1)
  const T* qb = q + slice * q_s;
  const T* kb = k + slice * k_s;
  const int64_t at = (int64_t)s * p.entries + (int64_t)t0 * W_TILE;
  const TileSum* sums = p.sum + (int64_t)s * (p.entries / W_TILE) + t0;
  TileSum ts[KT];
  Operand<T, D> K[KT];
  f32x16 acc[KT];
  int a = 0x7fffffff, z = -1;  // first and last token that sees one of the rows
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    ts[x] = sums[x];
    if (ts[x].vmax >= 0) {
      a = min(a, ts[x].tmin);
      z = max(z, ts[x].vmax);
    }
    K[x].load(kb + (int64_t)(max(p.row[at + x * W_TILE + l32], 0) & (W_CL - 1)) * D, h);
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[x][v] = 0.f;
  }
  // query tiles [qa, qz]
  const int last = tok0 + nq - 1;
  z = min(z, last);
  const int qa = z < 0 || a > z ? 1 : max(a - tok0, 0) / W_TILE;
  const int qz = z < 0 || a > z ? 0 : (z - tok0) / W_TILE;
  const float2* mls = ml + (int64_t)slice * splits * nq;
  // a tile's queries, and the lane's normaliser (+inf: gives nothing)
  auto load_q = [&](Operand<T, D>& Q, int qt) { Q.load(qb + (int64_t)min(qt * W_TILE + l32, nq - 1) * D, h); };
  auto load_lse = [&](int qt) {
    const int i = qt * W_TILE + l32;
    float m = -INFINITY, l = 0.f;
    if (i < nq) {
      if (splits == 1) {
        const float2 x = mls[i];
        m = x.x;
        l = x.y;
      } else {  // the halves take every other share
        for (int j = h; j < splits; j += 2) {
          const float2 x = mls[(int64_t)j * nq + i];
          const float mn = fmaxf(m, x.x);
          if (mn != -INFINITY) l = l * fast_exp2(m - mn) + x.y * fast_exp2(x.x - mn);
          m = mn;
        }
      }
    }
    if (splits > 1) {
      const float mn = other_half(m, false);
      l = other_half(m == -INFINITY ? 0.f : l * fast_exp2(m - mn), true);
      m = mn;
    }
    return l > 0.f ? m + __builtin_amdgcn_logf(l) : INFINITY;
  };
  auto compute = [&](const Operand<T, D>& Q, float lse, int qt) {
    const int ta = tok0 + qt * W_TILE, tb = min(ta + W_TILE - 1, last);
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      if (ts[x].tmin > tb || ts[x].vmax < ta) continue;
      f32x16 sc = scores<T, D>(K[x], Q);
      if (ts[x].tmax > ta || ts[x].vmin < tb)
        mask_scores(sc, p.tok + at + x * W_TILE, p.vu + at + x * W_TILE, ta + l32, h);
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[x][v] += fast_exp2(fmaf(sc[v], c, -lse));
    }
  };
  Operand<T, D> A, B;
  int qt = qa + (WQ == 1 ? 0 : wave);
  if (qt <= qz) {
    load_q(A, qt);
    float la = load_lse(qt);
    for (;;) {
      const int n1 = min(qt + WQ, qz);
      load_q(B, n1);
      const float lb = load_lse(n1);
      compute(A, la, qt);
      if (qt + WQ > qz) break;
      const int n2 = min(qt + 2 * WQ, qz);
      load_q(A, n2);
      la = load_lse(n2);
      compute(B, lb, qt + WQ);
      if (qt + 2 * WQ > qz) break;
      qt += 2 * WQ;
    }
  }
  // over the queries: each lane ends with the sum of one row (lane pairs alike)
  __shared__ float meet[WQ == 1 ? 1 : WQ][KT * W_TILE];
  float sum[KT];
  int m[KT];
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = acc[x][i];
    int base = 0;
    half_wave_reduce<16, 16>(v, lane, base);
    static_assert(half_wave_count<16, 16>() == 1, "one row a lane");
    sum[x] = v[0];
    m[x] = 8 * (base / 4) + 4 * h + base % 4;
    if constexpr (WQ > 1)
      if (!(lane & 1)) meet[wave][x * W_TILE + m[x]] = sum[x];
  }
  if constexpr (WQ > 1) {
    __syncthreads();
    if (wave > 0) return;
  }
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    if (lane & 1) continue;
    float total = sum[x];
    if constexpr (WQ > 1)
#pragma unroll
      for (int w = 1; w < WQ; ++w) total += meet[w][x * W_TILE + m[x]];
    const int e = p.row[at + x * W_TILE + m[x]];
    if (e < 0) continue;
    const int64_t r = (int64_t)slice * L_cap + (e & (W_CL - 1));
    if (e & W_CL) total = 1.f;
    w_out[r] = (w_in ? w_in[r] : 0.f) + total;
  }
}

// Units of the stats launch: two waves a SIMD at least, where the queries (one
// tile a wave then, else two) and up to 64 shares of the rows, of 128 at
// least, give as many.
constexpr int W_FILL = 2048;
static int stats_tiles(bool bf16, int64_t slices, int32_t nq) {
  return bf16 && slices * ((nq + 2 * W_TILE - 1) / (2 * W_TILE)) >= W_FILL / 2 ? 2 : 1;
}
static int stats_splits(bool bf16, int64_t slices, int32_t nq, int32_t L_cap) {
  const int qt = stats_tiles(bf16, slices, nq) * W_TILE;
  const int64_t units = slices * ((nq + qt - 1) / qt);
  const int64_t want = (W_FILL + units - 1) / std::max<int64_t>(units, 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, 64, (L_cap + 127) / 128}));
}

template <typename T, int D>
static int launch_weights(const void* q, const void* k, const float* w_in, float* w_out, int32_t b,
                          int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float scale,
                          const int32_t* vu, int32_t L_meta, int32_t tok0, const int32_t* kv_len,
                          const int32_t* tok_idx, int32_t L_cap, void* ws, hipStream_t stream) {
  constexpr bool BF16 = sizeof(T) == 2;
  const T* qq = static_cast<const T*>(q);
  const T* kk = static_cast<const T*>(k);
  const WeightPlan p = plan_at(ws, b, L_cap);
  float2* ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + plan_bytes(b, L_cap));
  const int slices = b * H;
  const float c = scale * W_LOG2E;
  weight_plan_kernel<<<b, PLAN_THREADS, 0, stream>>>(p, vu, L_meta, tok0, nq, kv_len, tok_idx, L_cap);
  int rc = hip_check(hipGetLastError(), "cached_attn_weights: plan launch");
  if (rc) return rc;
  const int splits = nq > 0 ? stats_splits(BF16, slices, nq, L_cap) : 1;
  if (nq > 0) {
    const int qt = stats_tiles(BF16, slices, nq);
    const int qtiles = (nq + qt * W_TILE - 1) / (qt * W_TILE);
    const int64_t wgs = (int64_t)slices * (((int64_t)qtiles * splits + W_WAVES - 1) / W_WAVES);
    if (wgs > 0x7fffffff) return fail(SCKV_EUNSUP, "cached_attn_weights: too many tiles");
    auto go = [&](auto kernel) {
      kernel<<<(unsigned)wgs, 64 * W_WAVES, 0, stream>>>(qq, kk, p, ml, H, nq, q_s, k_s, c, vu, L_meta,
                                                         tok0, slices, qtiles, splits);
    };
    if constexpr (BF16) {
      if (qt == 2) go(weight_stats_kernel<T, D, 2>);
      else go(weight_stats_kernel<T, D, 1>);
    } else {
      go(weight_stats_kernel<T, D, 1>);
    }
    rc = hip_check(hipGetLastError(), "cached_attn_weights: stats launch");
    if (rc) return rc;
  }
  // Two key tiles a wave read the queries half as often; one where that leaves
  // SIMDs idle, shared by the workgroup's waves where it still does.
  const int64_t tiles = p.entries / W_TILE;
  const int kt = BF16 && slices * (tiles / 2) >= W_FILL ? 2 : 1;
  const int wq = kt == 1 && slices * tiles < W_FILL && nq > W_TILE ? W_WAVES : 1;
  const int64_t per_wg = (int64_t)kt * (W_WAVES / wq);
  const int64_t wgs = slices * ((tiles + per_wg - 1) / per_wg);
  if (wgs > 0x7fffffff) return fail(SCKV_EUNSUP, "cached_attn_weights: too many tiles");
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)wgs, 64 * W_WAVES, 0, stream>>>(qq, kk, p, ml, w_in, w_out, H, nq, q_s, k_s, c,
                                                       tok0, L_cap, slices, splits);
  };
  if constexpr (BF16) {
    if (kt == 2) go(weight_sums_kernel<T, D, 2, 1>);
  }
  if (kt == 1 && wq == 1) go(weight_sums_kernel<T, D, 1, 1>);
  if (kt == 1 && wq > 1) go(weight_sums_kernel<T, D, 1, W_WAVES>);
  return hip_check(hipGetLastError(), "cached_attn_weights: sums launch");
}

}  // namespace sckv

using namespace sckv;

extern "C" size_t sckv_attn_weights_workspace_bytes(int32_t b, int32_t H, int32_t nq,
                                                    int32_t L_cap) {
  if (b <= 0 || H <= 0 || nq < 0 || L_cap <= 0) return 0;
  // (the size function is not told the element type)
  const int64_t slices = (int64_t)b * H;
  const int splits = std::max(stats_splits(true, slices, nq, L_cap), stats_splits(false, slices, nq, L_cap));
  return plan_bytes(b, L_cap) + (size_t)slices * splits * nq * sizeof(float2);
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
