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
#include <type_traits>

#include "sckv_common.h"

namespace sckv {

constexpr float W_LOG2E = 1.4426950408889634f;
constexpr int W_TILE = 32;        // rows, or queries, of a tile
constexpr int W_WAVES = 4;        // of a workgroup
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
  int32_t* tiles;           // [b]: tiles listed
  int32_t entries;          // of a sequence
  int32_t chunk;            // of each PLAN_CHUNK rows
};

constexpr int PLAN_WAVES = 16;
constexpr int PLAN_THREADS = 64 * PLAN_WAVES;
constexpr int PLAN_U = 4;  // rows of a thread, in flight together
constexpr int PLAN_CHUNK = PLAN_THREADS * PLAN_U;
constexpr int PLAN_ENTRIES = PLAN_CHUNK + 3 * W_CLASS;  // the most of a chunk's list

// Entries of a sequence's list.  Each PLAN_CHUNK rows have a part of their own
// (a workgroup plans it): every row, and each class up to W_CLASS - 1 more.
static int32_t chunk_entries(int32_t L_cap) {
  return (std::min(L_cap, PLAN_CHUNK) + W_CLASS - 1) / W_CLASS * W_CLASS + 3 * W_CLASS;
}
static int32_t plan_chunks(int32_t L_cap) { return (L_cap + PLAN_CHUNK - 1) / PLAN_CHUNK; }
static int64_t plan_entries(int32_t L_cap) { return (int64_t)plan_chunks(L_cap) * chunk_entries(L_cap); }
static size_t plan_bytes(int32_t b, int32_t L_cap) {
  const size_t e = (size_t)plan_entries(L_cap);
  return (size_t)b * (3 * e * 4 + e / W_TILE * sizeof(TileSum) + 16);
}
static WeightPlan plan_at(void* ws, int32_t b, int32_t L_cap) {
  const size_t e = (size_t)plan_entries(L_cap);
  WeightPlan p;
  p.entries = (int32_t)e;
  p.chunk = chunk_entries(L_cap);
  p.row = static_cast<int32_t*>(ws);
  p.tok = p.row + (size_t)b * e;
  p.vu = p.tok + (size_t)b * e;
  p.sum = reinterpret_cast<TileSum*>(p.vu + (size_t)b * e);
  p.tiles = reinterpret_cast<int32_t*>(p.sum + (size_t)b * (e / W_TILE));
  return p;
}

// `of` over the 32 lanes of each half-wave; every lane gets it
template <typename F>
__device__ __forceinline__ int half_wave_of(int x, F of) {
  const auto mov = [](int y, auto ctrl) {
    return __builtin_bit_cast(int, dpp_mov<decltype(ctrl)::value>(__builtin_bit_cast(float, y)));
  };
  x = of(x, mov(x, std::integral_constant<int, DPP_QUAD_XOR1>()));
  x = of(x, mov(x, std::integral_constant<int, DPP_QUAD_XOR2>()));
  x = of(x, mov(x, std::integral_constant<int, DPP_ROW_HALF_MIRROR>()));
  x = of(x, mov(x, std::integral_constant<int, DPP_ROW_MIRROR>()));
  const auto r = __builtin_amdgcn_permlane16_swap((unsigned)x, (unsigned)x, false, false);
  return of((int)r[0], (int)r[1]);
}

// one workgroup per chunk of a sequence
__global__ __launch_bounds__(PLAN_THREADS) void weight_plan_kernel(
    WeightPlan p, const int32_t* __restrict__ vu, int32_t L_meta, int32_t tok0, int32_t nq,
    const int32_t* __restrict__ kv_len, const int32_t* __restrict__ tok_idx, int32_t L_cap,
    int32_t chunks) {
  static_assert(PLAN_U * PLAN_WAVES == 64, "one wave scans the counts of a class");
  // rows of class k that pass u of wave w holds, then those before them, at
  // [k][u * PLAN_WAVES + w]; the total behind them
  __shared__ int before[3][65];
  // tokens and vu of the chunk's list, for the summaries of its tiles
  __shared__ int list_tok[PLAN_ENTRIES], list_vu[PLAN_ENTRIES];
  const int s = blockIdx.x / chunks, chunk = blockIdx.x - s * chunks;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row0 = chunk * PLAN_CHUNK;
  const int32_t* toks = tok_idx + (int64_t)s * L_cap + row0;
  const int32_t* vus = vu + (int64_t)s * L_meta;
  // (asked for before the length is known: rows past it are read and dropped)
  int j[PLAN_U], v[PLAN_U], c[PLAN_U];
#pragma unroll
  for (int u = 0; u < PLAN_U; ++u) j[u] = toks[min(u * PLAN_THREADS + tid, L_cap - 1 - row0)];
  const int held = min(max(kv_len[s], 0), L_cap);
  if (chunk == 0 && tid == 0)
    p.tiles[s] = (held + PLAN_CHUNK - 1) / PLAN_CHUNK * (p.chunk / W_TILE);
  const int n = min(held - row0, PLAN_CHUNK);  // rows of this chunk
  if (n <= 0) return;
  const int64_t at = (int64_t)s * p.entries + (int64_t)chunk * p.chunk;
  const int last = tok0 + nq - 1;  // last query's token
  // classes: 0 seen by every later query, 1 by some, 2 by none (3: no row)
  uint64_t m[3][PLAN_U];
#pragma unroll
  for (int u = 0; u < PLAN_U; ++u) v[u] = vus[min(max(j[u], 0), L_meta - 1)];
#pragma unroll
  for (int u = 0; u < PLAN_U; ++u) {
    const bool none = j[u] < 0 || j[u] >= L_meta || v[u] == j[u] || j[u] > last || v[u] < tok0 || nq == 0;
    c[u] = u * PLAN_THREADS + tid >= n ? 3 : none ? 2 : v[u] >= last ? 0 : 1;
#pragma unroll
    for (int k = 0; k < 3; ++k) m[k][u] = __ballot(c[u] == k);
    const int x0 = __popcll(m[0][u]), x1 = __popcll(m[1][u]), x2 = __popcll(m[2][u]);
    if (lane < 3) before[lane][u * PLAN_WAVES + wave] = lane == 0 ? x0 : lane == 1 ? x1 : x2;
  }
  __syncthreads();
  if (wave < 3) {  // the counts become exclusive prefix sums
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
  // the rows, in order within each class; what is left of a class's last tiles
  // and of the chunk's part is row -1, seen by none
  int start = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int total = before[k][64];
#pragma unroll
    for (int u = 0; u < PLAN_U; ++u)
      if (c[u] == k) {
        const int row = row0 + u * PLAN_THREADS + tid;
        const bool cl = k == 2 && v[u] == j[u] && j[u] >= tok0 && j[u] <= last;
        const int e = start + before[k][u * PLAN_WAVES + wave] + mask_rank(m[k][u]);
        p.row[at + e] = cl ? row | W_CL : row;
        p.tok[at + e] = list_tok[e] = j[u];
        p.vu[at + e] = list_vu[e] = k == 2 ? -1 : v[u];
      }
    const int next = k == 2 ? p.chunk : start + (total + W_CLASS - 1) / W_CLASS * W_CLASS;
    for (int e = start + total + tid; e < next; e += PLAN_THREADS) {
      p.row[at + e] = -1;
      p.tok[at + e] = list_tok[e] = 0x7fffffff;
      p.vu[at + e] = list_vu[e] = -1;
    }
    start = next;
  }
  __syncthreads();
  for (int t = tid / 32; t < p.chunk / W_TILE; t += PLAN_THREADS / 32) {
    const int jt = list_tok[t * W_TILE + (tid & 31)], vt = list_vu[t * W_TILE + (tid & 31)];
    const auto least = [](int a, int b) { return min(a, b); };
    const auto most = [](int a, int b) { return max(a, b); };
    const TileSum x = {half_wave_of(jt, least), half_wave_of(jt, most), half_wave_of(vt, least),
                       half_wave_of(vt, most)};
    if ((tid & 31) == 0) p.sum[at / W_TILE + t] = x;
  }
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

// maximum and sum of a query (by lane) over one more tile of scores.  The
// maximum is only looked for where the weights of the tile, taken against the
// one so far, leave a lane's sum above 2^16 (or where a lane has none yet):
// sums then stay in range, and the comparison of 16 scores is spared.
__device__ __forceinline__ void add_tile(const f32x16& sc, float c, float& M, float& l) {
  const float m0 = M == -INFINITY ? 0.f : M;
  float a0 = 0.f, a1 = 0.f;
#pragma unroll
  for (int v = 0; v < 16; v += 2) {
    a0 += fast_exp2(fmaf(sc[v], c, -m0));
    a1 += fast_exp2(fmaf(sc[v + 1], c, -m0));
  }
  if (__any(!(a0 + a1 <= 65536.f) || M == -INFINITY)) {
    float mb = sc[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mb = fmaxf(mb, sc[v]);
    const float mn = fmaxf(M, other_half(mb, false) * c);
    l = mn == -INFINITY ? 0.f : l * fast_exp2(M - mn);
    M = mn;
    const float m1 = M == -INFINITY ? 0.f : M;
    a0 = a1 = 0.f;
#pragma unroll
    for (int v = 0; v < 16; v += 2) {
      a0 += fast_exp2(fmaf(sc[v], c, -m1));
      a1 += fast_exp2(fmaf(sc[v + 1], c, -m1));
    }
  }
  l += a0 + a1;
}


// ---------------------------------------------------------------------------
// stats: (maximum, sum) of each query over the rows of one of `splits` shares
// of its slice's tiles.  A unit is a wave: QT tiles of queries, one share; the
// waves of a workgroup are units next to one another, which read the same keys.
// ---------------------------------------------------------------------------
template <typename T, int D, int QT>
__global__ __launch_bounds__(64 * W_WAVES, 2) void weight_stats_kernel(
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
  const int n_tiles = p.tiles[s];

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
      add_tile(sc, c, M[x], l[x]);
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

// (maximum, sum) of two sets of rows, and the normaliser of one (+inf: the query
// gives nothing)
__device__ __forceinline__ float2 join_norm(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, 0.f);
  return make_float2(m, a.y * fast_exp2(a.x - m) + b.y * fast_exp2(b.x - m));
}
__device__ __forceinline__ float norm_lse(float2 a) {
  return a.y > 0.f ? a.x + __builtin_amdgcn_logf(a.y) : INFINITY;
}
// query i over the shares first, first + step, ..., the wave's halves together
__device__ __forceinline__ float2 tile_norm(const float2* __restrict__ ml, int i, int nq, int first,
                                            int step, int splits) {
  float2 a = make_float2(-INFINITY, 0.f);
  if (i < nq) {
#pragma unroll 4
    for (int j = first; j < splits; j += step) a = join_norm(a, ml[(int64_t)j * nq + i]);
  }
  const auto m = __builtin_amdgcn_permlane32_swap(__float_as_uint(a.x), __float_as_uint(a.x), false, false);
  const auto l = __builtin_amdgcn_permlane32_swap(__float_as_uint(a.y), __float_as_uint(a.y), false, false);
  return join_norm(make_float2(__uint_as_float(m[0]), __uint_as_float(l[0])),
                   make_float2(__uint_as_float(m[1]), __uint_as_float(l[1])));
}
__device__ __forceinline__ float tile_lse(const float2* __restrict__ ml, int i, int nq, int splits,
                                          int h) {
  if (splits == 1) return i < nq ? norm_lse(ml[i]) : INFINITY;
  return norm_lse(tile_norm(ml, i, nq, h, 2, splits));
}

// ---------------------------------------------------------------------------
// sums: KT tiles of rows a wave.  WQ = 1: the workgroup's waves take key tiles
// of their own; WQ = W_WAVES: they share theirs and take every WQ-th tile of
// queries each (launches of few keys).
// ---------------------------------------------------------------------------
template <typename T, int D, int KT, int WQ>
__global__ __launch_bounds__(64 * W_WAVES, 2) void weight_sums_kernel(
    const T* __restrict__ q, const T* __restrict__ k, WeightPlan p, const float2* __restrict__ ml,
    const float* w_in, float* w_out, int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float c,
    int32_t tok0, int32_t L_cap, int32_t n_slice, int32_t splits) {
  const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wg = blockIdx.x / n_slice, slice = blockIdx.x - wg * n_slice;
  const int s = slice / H;
  const int n_tiles = p.tiles[s];  // a multiple of two
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
  auto load_q = [&](Operand<T, D>& Q, int qt) { Q.load(qb + (int64_t)min(qt * W_TILE + l32, nq - 1) * D, h); };
  auto load_lse = [&](int qt) { return tile_lse(mls, qt * W_TILE + l32, nq, splits, h); };
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

// ---------------------------------------------------------------------------
// Stages: 64 rows (two tiles) that a workgroup's waves share through LDS,
// for long lists: a wave's own loads of an operand touch 32 cache lines an
// instruction, 32 bytes of each; staged, a line is read once a workgroup
// (16384 queries, 32 heads of 64: 1180 -> 970 us).  Short lists are slower so
// (16 x 1024 queries of 80: 152 -> 207 us): a workgroup's four waves go through
// the union of their lists, a barrier a stage.
// Piece g of row r lies at g ^ (r % 8) where a row is a power of two of
// pieces, at g otherwise (rows of 160 and 320 bytes fall on different banks by
// themselves), so that the 8 rows of a quarter wave's read share no bank.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct Stage {
  static constexpr int ROWS = 2 * W_TILE;
  static constexpr int PIECES = D * (int)sizeof(T) / 16;  // of a row
  static constexpr int BYTES = ROWS * PIECES * 16;
  static constexpr int THREADS = 64 * W_WAVES;
  static constexpr int PER = (ROWS * PIECES + THREADS - 1) / THREADS;  // of a thread
  __device__ __forceinline__ static int slot(int row, int g) {
    return (PIECES & (PIECES - 1)) == 0 ? g ^ (row & 7) : g;
  }
  u32x4 x[PER];
  // rows[i]: the row of the source that this thread's piece i belongs to
  __device__ __forceinline__ void load(const T* src, const int* rows, int tid) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int g = (tid + i * THREADS) % PIECES;
      x[i] = ld16(src + (int64_t)rows[i] * D + g * (16 / (int)sizeof(T)));
    }
  }
  __device__ __forceinline__ static int row_of(int tid, int i) {  // of the stage (clamped)
    return min((tid + i * THREADS) / PIECES, ROWS - 1);
  }
  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = tid + i * THREADS, row = e / PIECES, g = e % PIECES;
      if (e < ROWS * PIECES) st16(lds + (row * PIECES + slot(row, g)) * 16, x[i]);
    }
  }
  // a tile's operand (rows 32 half .. of the stage)
  __device__ __forceinline__ static void read(Operand<T, D>& o, const char* lds, int half, int lane) {
    const int row = half * W_TILE + (lane & 31), h = lane >> 5;
#pragma unroll
    for (int i = 0; i < Operand<T, D>::N; ++i) o.x[i] = ld16(lds + (row * PIECES + slot(row, 2 * i + h)) * 16);
  }
};

// stats of large launches: QT tiles of queries a wave, W_WAVES * QT a workgroup;
// four waves a SIMD where three registers less give them (d = 64; 2 x 32 heads of
// 4096 tokens 222 -> 213 us)
template <typename T, int D, int QT>
__global__ __launch_bounds__(64 * W_WAVES, sizeof(T) == 2 && D == 64 ? 4 : 2) void weight_stats_staged_kernel(
    const T* __restrict__ q, const T* __restrict__ k, WeightPlan p, float2* __restrict__ ml,
    int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float c, const int32_t* __restrict__ vu,
    int32_t L_meta, int32_t tok0, int32_t n_slice, int32_t qgroups, int32_t splits) {
  using S = Stage<T, D>;
  __shared__ __align__(16) char lds[2][S::BYTES];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wg = blockIdx.x / n_slice, slice = blockIdx.x - wg * n_slice;
  const int split = wg % splits;
  const int g0 = (qgroups - 1 - wg / splits) * W_WAVES * QT * W_TILE;  // first query; the last see most
  const int s = slice / H;
  const T* qb = q + slice * q_s;
  const T* kb = k + slice * k_s;
  const int64_t at = (int64_t)s * p.entries;
  const TileSum* sums = p.sum + (int64_t)s * (p.entries / W_TILE);
  const int n_stage = p.tiles[s] / 2;
  const int q0 = g0 + wave * QT * W_TILE;

  Operand<T, D> Q[QT];
  int t[QT], ta[QT], tb[QT];
  float M[QT], l[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int i = q0 + W_TILE * x;
    t[x] = tok0 + min(i + l32, nq - 1);
    ta[x] = tok0 + i;
    tb[x] = i < nq ? min(ta[x] + W_TILE - 1, tok0 + nq - 1) : -1;  // -1: sees nothing below
    Q[x].load(qb + (int64_t)min(i + l32, nq - 1) * D, h);
    M[x] = -INFINITY;
    l[x] = 0.f;
  }
  // the share's stages that some query of the workgroup sees, 64 at a time
  const int lo = tok0 + g0, hi = tok0 + min(g0 + W_WAVES * QT * W_TILE, nq) - 1;
  TileSum held[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  int cand = 0, held0 = 0;
  uint64_t seen = 0;
  struct Ref {
    int stage;
    TileSum s[2];
  };
  auto next = [&]() {
    while (seen == 0 && cand * splits + split < n_stage) {
      const int st = (cand + lane) * splits + split;
      held0 = cand;
      cand += 64;
      bool see = false;
      if (st < n_stage) {
        held[0] = sums[2 * st];
        held[1] = sums[2 * st + 1];
        see = (held[0].tmin <= hi && held[0].vmax >= lo) || (held[1].tmin <= hi && held[1].vmax >= lo);
      }
      seen = __ballot(see);
    }
    Ref r;
    r.stage = -1;
    if (seen != 0) {
      const int i = __builtin_ctzll(seen);
      seen &= seen - 1;
      r.stage = (held0 + i) * splits + split;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        r.s[y].tmin = __builtin_amdgcn_readlane(held[y].tmin, i);
        r.s[y].tmax = __builtin_amdgcn_readlane(held[y].tmax, i);
        r.s[y].vmin = __builtin_amdgcn_readlane(held[y].vmin, i);
        r.s[y].vmax = __builtin_amdgcn_readlane(held[y].vmax, i);
      }
    }
    return r;
  };
  S st;
  int rows[S::PER];
  auto number = [&](const Ref& r) {
#pragma unroll
    for (int i = 0; i < S::PER; ++i)
      rows[i] = r.stage >= 0 ? max(p.row[at + (int64_t)r.stage * S::ROWS + S::row_of(tid, i)], 0) : 0;
  };
  Ref cur = next();
  number(cur);
  if (cur.stage >= 0) st.load(kb, rows, tid);
  Ref nxt = next();
  number(nxt);
  int buf = 0;
  while (cur.stage >= 0) {
    st.store(lds[buf], tid);
    if (nxt.stage >= 0) st.load(kb, rows, tid);
    const Ref after = next();
    number(after);
    // one barrier a stage: the other buffer was read before the last one
    __syncthreads();
    Operand<T, D> K;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      S::read(K, lds[buf], y, lane);
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        if (cur.s[y].tmin > tb[x] || cur.s[y].vmax < ta[x]) continue;
        f32x16 sc = scores<T, D>(K, Q[x]);
        if (cur.s[y].tmax > ta[x] || cur.s[y].vmin < tb[x]) {
          const int64_t e = at + (int64_t)cur.stage * S::ROWS + y * W_TILE;
          mask_scores(sc, p.tok + e, p.vu + e, t[x], h);
        }
        add_tile(sc, c, M[x], l[x]);
      }
    }
    cur = nxt;
    nxt = after;
    buf ^= 1;
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

// sums of large launches: KT tiles of rows a wave, W_WAVES * KT a workgroup.
// The tiles are S = Q K^T here: the lane owns row l % 32 and its token, vu and
// sum, in four registers a tile of rows instead of 16 (16 x 4096 tokens of 80:
// 1586 -> 1486 us; 2 x 32 heads of 64: 187 -> 178).
template <typename T, int D, int KT>
__global__ __launch_bounds__(64 * W_WAVES, 2) void weight_sums_staged_kernel(
    const T* __restrict__ q, const T* __restrict__ k, WeightPlan p, const float2* __restrict__ ml,
    const float* w_in, float* w_out, int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float c,
    int32_t tok0, int32_t L_cap, int32_t n_slice, int32_t splits) {
  using S = Stage<T, D>;
  __shared__ __align__(16) char lds[2][S::BYTES];
  __shared__ __align__(16) float lse[2][S::ROWS];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wg = blockIdx.x / n_slice, slice = blockIdx.x - wg * n_slice;
  const int s = slice / H;
  const int n_tiles = p.tiles[s];
  const int g0 = wg * W_WAVES * KT;  // first tile of the workgroup
  if (g0 >= n_tiles) return;
  const T* qb = q + slice * q_s;
  const T* kb = k + slice * k_s;
  const int64_t at = (int64_t)s * p.entries;
  const TileSum* sums = p.sum + (int64_t)s * (p.entries / W_TILE);
  const int last = tok0 + nq - 1;
  // the workgroup's first and last token that sees one of its rows
  int a = 0x7fffffff, z = -1;
  for (int i = g0; i < min(g0 + W_WAVES * KT, n_tiles); ++i) {
    const TileSum x = sums[i];
    if (x.vmax >= 0) {
      a = min(a, x.tmin);
      z = max(z, x.vmax);
    }
  }
  z = min(z, last);
  const bool some = z >= 0 && a <= z;
  const int sa = some ? max(a - tok0, 0) / S::ROWS : 1, sz = some ? (z - tok0) / S::ROWS : 0;

  const int t0 = g0 + wave * KT;
  TileSum ts[KT];
  Operand<T, D> K[KT];
  // the lane's row of each tile: list entry, token, vu, sum
  int e[KT], tok[KT], vus[KT];
  float acc[KT];
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    const bool in = t0 + x < n_tiles;
    ts[x] = in ? sums[t0 + x] : TileSum{0x7fffffff, 0x7fffffff, -1, -1};
    const int64_t i = at + (int64_t)(t0 + x) * W_TILE + l32;
    e[x] = in ? p.row[i] : -1;
    tok[x] = in ? p.tok[i] : 0;
    vus[x] = in ? p.vu[i] : -1;
    K[x].load(kb + (int64_t)(max(e[x], 0) & (W_CL - 1)) * D, h);
    acc[x] = 0.f;
  }
  const float2* mls = ml + (int64_t)slice * splits * nq;
  S st;
  int rows[S::PER];
  auto load = [&](int stage) {
#pragma unroll
    for (int i = 0; i < S::PER; ++i) rows[i] = min(stage * S::ROWS + S::row_of(tid, i), nq - 1);
    st.load(qb, rows, tid);
  };
  // one wave takes the normalisers, 32 queries at a time
  float n0 = 0.f, n1 = 0.f;
  auto normalisers = [&](int stage) {
    if (wave == 0) {
      n0 = tile_lse(mls, stage * S::ROWS + l32, nq, splits, h);
      n1 = tile_lse(mls, stage * S::ROWS + W_TILE + l32, nq, splits, h);
    }
  };
  if (sa <= sz) {
    load(sa);
    normalisers(sa);
  }
  int buf = 0;
  for (int g = sa; g <= sz; ++g) {
    st.store(lds[buf], tid);
    if (wave == 0) lse[buf][lane] = h ? n1 : n0;
    if (g < sz) {
      load(g + 1);
      normalisers(g + 1);
    }
    __syncthreads();
    Operand<T, D> Q;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int ta = tok0 + g * S::ROWS + y * W_TILE, tb = min(ta + W_TILE - 1, last);
      if (ta > last) continue;
      S::read(Q, lds[buf], y, lane);
      float4 ls[4];  // of the lane's queries, as the registers of a score tile
#pragma unroll
      for (int i = 0; i < 4; ++i) ls[i] = *reinterpret_cast<const float4*>(&lse[buf][y * W_TILE + 8 * i + 4 * h]);
#pragma unroll
      for (int x = 0; x < KT; ++x) {
        if (ts[x].tmin > tb || ts[x].vmax < ta) continue;
        f32x16 sc = scores<T, D>(Q, K[x]);  // S = Q K^T: the lane owns a row
        if (ts[x].tmax > ta || ts[x].vmin < tb) {
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int tq = ta + 8 * (v / 4) + 4 * h + v % 4;
            sc[v] = tok[x] <= tq && tq <= vus[x] ? sc[v] : -INFINITY;
          }
        }
        // (a tile's sum first: the rounding of a long sum grows with its terms)
        float a0 = 0.f, a1 = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a0 += fast_exp2(fmaf(sc[4 * i], c, -ls[i].x));
          a1 += fast_exp2(fmaf(sc[4 * i + 1], c, -ls[i].y));
          a0 += fast_exp2(fmaf(sc[4 * i + 2], c, -ls[i].z));
          a1 += fast_exp2(fmaf(sc[4 * i + 3], c, -ls[i].w));
        }
        acc[x] += a0 + a1;
      }
    }
    buf ^= 1;
  }
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    const float total = other_half(acc[x], true);
    if (h || e[x] < 0) continue;
    const int64_t r = (int64_t)slice * L_cap + (e[x] & (W_CL - 1));
    w_out[r] = (w_in ? w_in[r] : 0.f) + (e[x] & W_CL ? 1.f : total);
  }
}

// ---------------------------------------------------------------------------
// sums of few queries (QT tiles): a wave keeps all queries and streams `run`
// key tiles, the next tile's keys and sums in flight while one is computed.
// With the keys kept instead, a wave's chain of loads (row numbers, keys, old
// sums) was paid every 64 rows: 49 us against 28 for 32 queries over
// 512 slices of 2050 rows of 80.
// ---------------------------------------------------------------------------
template <typename T, int D, int QT>
__global__ __launch_bounds__(64 * W_WAVES, 2) void weight_votes_kernel(
    const T* __restrict__ q, const T* __restrict__ k, WeightPlan p, const float2* __restrict__ ml,
    const float* w_in, float* w_out, int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float c,
    int32_t tok0, int32_t L_cap, int32_t n_slice, int32_t splits, int32_t run) {
  const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
  const int wg = blockIdx.x / n_slice, slice = blockIdx.x - wg * n_slice;
  const int unit = __builtin_amdgcn_readfirstlane(wg * W_WAVES + (threadIdx.x >> 6));
  const int s = slice / H;
  const int n_tiles = p.tiles[s];
  const int t0 = unit * run, t1 = min(t0 + run, n_tiles);
  // the normalisers: each wave joins a quarter of the shares
  __shared__ float2 meet[W_WAVES][QT * W_TILE];
  const int wave = threadIdx.x >> 6;
  const float2* mls = ml + (int64_t)slice * splits * nq;
  float lse[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const float2 part = tile_norm(mls, W_TILE * x + l32, nq, wave * 2 + h, 2 * W_WAVES, splits);
    if (lane < 32) meet[wave][W_TILE * x + l32] = part;
  }
  __syncthreads();
  if (t0 >= t1) return;
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    float2 all = meet[0][W_TILE * x + l32];
#pragma unroll
    for (int w = 1; w < W_WAVES; ++w) all = join_norm(all, meet[w][W_TILE * x + l32]);
    lse[x] = norm_lse(all);
  }
  const T* kb = k + slice * k_s;
  const int64_t at = (int64_t)s * p.entries;
  const TileSum* sums = p.sum + (int64_t)s * (p.entries / W_TILE);
  const int last = tok0 + nq - 1;
  // the row of a tile whose sum this lane ends with
  int base = 0;
  {
    float v[16] = {0.f};
    half_wave_reduce<16, 16>(v, lane, base);
  }
  const int m = 8 * (base / 4) + 4 * h + base % 4;

  Operand<T, D> A, B;
  auto number = [&](int t, int i) { return p.row[at + (int64_t)min(t, t1 - 1) * W_TILE + i]; };
  auto load = [&](Operand<T, D>& K, int e) { K.load(kb + (int64_t)(max(e, 0) & (W_CL - 1)) * D, h); };
  const int64_t wo = (int64_t)slice * L_cap;
  auto old = [&](int e) { return w_in ? w_in[wo + (max(e, 0) & (W_CL - 1))] : 0.f; };
  int e0 = number(t0, m), e1 = number(t0 + 1, m);
  int i1 = number(t0 + 1, l32);
  load(A, number(t0, l32));
  float o0 = old(e0);
  Operand<T, D> Q[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) Q[x].load(q + slice * q_s + (int64_t)min(W_TILE * x + l32, nq - 1) * D, h);
  auto compute = [&](const Operand<T, D>& K, int t, int e, float before) {
    const TileSum ts = sums[t];
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.f;
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      const int ta = tok0 + W_TILE * x, tb = min(ta + W_TILE - 1, last);
      if (ts.tmin > tb || ts.vmax < ta) continue;
      f32x16 sc = scores<T, D>(K, Q[x]);
      if (ts.tmax > ta || ts.vmin < tb)
        mask_scores(sc, p.tok + at + t * W_TILE, p.vu + at + t * W_TILE, ta + l32, h);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] += fast_exp2(fmaf(sc[i], c, -lse[x]));
    }
    int unused = 0;
    half_wave_reduce<16, 16>(v, lane, unused);
    if (!(lane & 1) && e >= 0)
      w_out[wo + (e & (W_CL - 1))] = before + (e & W_CL ? 1.f : v[0]);
  };
  for (int t = t0; t < t1; t += 2) {
    load(B, i1);
    const int i2 = number(t + 2, l32);
    const float o1 = old(e1);
    const int e2 = number(t + 2, m);
    compute(A, t, e0, o0);
    if (t + 1 >= t1) break;
    load(A, i2);
    i1 = number(t + 3, l32);
    o0 = old(e2);
    const int e3 = number(t + 3, m);
    compute(B, t + 1, e1, o1);
    e0 = e2;
    e1 = e3;
  }
}

// Launch shapes, by sizes alone (us; rows are the cache's capacity, the host's
// only hint of its length):
//  * stats: a wave keeps two tiles of bf16 queries where that leaves W_UNITS
//    waves (16 x 64 queries over 2048 rows of 64: 72 with one tile, 65 with two;
//    32 heads of 2048 tokens: 74, 67), else one.  The rows are cut into
//    up to 64 shares of at least 128 (fp32, whose products take eight times as
//    long: 64; 4 heads of 256 rows, 32 queries: 21.5 with 128, 17.6 with 64)
//    until there are W_FILL waves, two a SIMD.
//  * sums: up to 32 queries (bf16: 64) are kept by every wave, which streams
//    rows (`votes`: W_FILL waves, up to 16 tiles each; 16 x 64 queries over 2048
//    rows of 80: 66, with 4096 waves 69; 32 heads of 16000 rows 38, 41).
//    Beyond, a wave keeps two tiles of bf16 rows where W_FILL waves do, else
//    one, and the waves of a workgroup share theirs below W_SHARE tiles (32
//    heads of 2048 tokens: 93 a wave each, 74 shared).
//  * from W_LONG rows and W_LONG / 4 queries on, with W_WGS workgroups: both
//    staged in LDS.  A wave keeps two tiles of queries where 2 W_WGS workgroups
//    do (32 heads of 8192 tokens of 80: 558 with two, 587 with one), else one
//    (4096 tokens: 198, 179).  Two tiles of rows where 4 W_WGS workgroups do (32
//    heads of 16384 tokens of 64: 954, 971 with one; 16 x 32 of 4096 of 80: 1486,
//    1520; 2 x 32 of 4096 of 64: 204, 180).
constexpr int W_SPLITS = 64;
constexpr int W_MIN_SHARE = 64;
constexpr int W_FILL = 2048;
constexpr int W_UNITS = 512;
constexpr int W_SHARE = 4096;
constexpr int W_LONG = 4096;
constexpr int W_WGS = 512;

struct WeightShape {
  bool staged;
  int votes;   // tiles of queries that every wave of the second pass keeps (0: not so)
  int keep;    // tiles of queries that a wave of the first pass keeps
  int qtiles;  // units of queries (workgroups' where staged, else waves')
  int splits;  // shares of the rows in the first pass
};
static WeightShape weight_shape(bool bf16, int64_t slices, int32_t nq, int32_t L_cap) {
  WeightShape w = {false, 0, 1, 0, 1};
  if (nq == 0) return w;
  const int two = bf16 ? 2 : 1;
  w.votes = nq <= W_TILE ? 1 : nq <= two * W_TILE ? 2 : 0;
  const int group = W_WAVES * W_TILE * two;
  const int64_t groups = (nq + group - 1) / group;
  w.staged = nq >= W_LONG / 4 && L_cap >= W_LONG && slices * groups >= W_WGS;
  if (w.staged) {
    if (slices * groups >= 2 * W_WGS) w.keep = two;
    w.qtiles = (nq + W_WAVES * W_TILE * w.keep - 1) / (W_WAVES * W_TILE * w.keep);
    return w;
  }
  const int pair = two * W_TILE;
  if (nq > W_TILE && slices * ((nq + pair - 1) / pair) >= W_UNITS) w.keep = two;
  w.qtiles = (nq + w.keep * W_TILE - 1) / (w.keep * W_TILE);
  const int64_t units = slices * w.qtiles, want = (W_FILL + units - 1) / units;
  const int share = bf16 ? 2 * W_MIN_SHARE : W_MIN_SHARE;
  w.splits = (int)std::max<int64_t>(1, std::min<int64_t>({want, W_SPLITS, (L_cap + share - 1) / share}));
  return w;
}

template <typename T, int D>
static int launch_weights(const void* q, const void* k, const float* w_in, float* w_out, int32_t b,
                          int32_t H, int32_t nq, int64_t q_s, int64_t k_s, float scale,
                          const int32_t* vu, int32_t L_meta, int32_t tok0, const int32_t* kv_len,
                          const int32_t* tok_idx, int32_t L_cap, void* ws, hipStream_t stream) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int NT = BF16 ? 2 : 1;
  constexpr int THREADS = 64 * W_WAVES;
  const T* qq = static_cast<const T*>(q);
  const T* kk = static_cast<const T*>(k);
  const WeightPlan p = plan_at(ws, b, L_cap);
  float2* ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + plan_bytes(b, L_cap));
  const int slices = b * H;
  const float c = scale * W_LOG2E;
  const WeightShape sh = weight_shape(BF16, slices, nq, L_cap);
  const int chunks = plan_chunks(L_cap);
  if ((int64_t)b * chunks > 0x7fffffff) return fail(SCKV_EUNSUP, "cached_attn_weights: too many tiles");
  weight_plan_kernel<<<b * chunks, PLAN_THREADS, 0, stream>>>(p, vu, L_meta, tok0, nq, kv_len, tok_idx,
                                                             L_cap, chunks);
  int rc = hip_check(hipGetLastError(), "cached_attn_weights: plan launch");
  if (rc) return rc;
  unsigned g = 0;  // workgroups
  auto grid = [&](int64_t per_slice) {
    const int64_t n = per_slice * slices;
    g = (unsigned)n;
    return n > 0x7fffffff ? fail(SCKV_EUNSUP, "cached_attn_weights: too many tiles") : SCKV_OK;
  };
  if (nq > 0) {
    const int64_t units = (int64_t)sh.qtiles * sh.splits;
    rc = grid(sh.staged ? units : (units + W_WAVES - 1) / W_WAVES);
    if (rc) return rc;
    auto go = [&](auto kernel) {
      kernel<<<g, THREADS, 0, stream>>>(qq, kk, p, ml, H, nq, q_s, k_s, c, vu, L_meta, tok0, slices,
                                        sh.qtiles, sh.splits);
    };
    if (sh.staged && sh.keep == NT) go(weight_stats_staged_kernel<T, D, NT>);
    else if (sh.staged) go(weight_stats_staged_kernel<T, D, 1>);
    else if (sh.keep == NT) go(weight_stats_kernel<T, D, NT>);
    else go(weight_stats_kernel<T, D, 1>);
    rc = hip_check(hipGetLastError(), "cached_attn_weights: stats launch");
    if (rc) return rc;
  }
  const int64_t tiles = p.entries / W_TILE;
  auto go = [&](auto kernel) {
    kernel<<<g, THREADS, 0, stream>>>(qq, kk, p, ml, w_in, w_out, H, nq, q_s, k_s, c, tok0, L_cap,
                                      slices, sh.splits);
  };
  if (sh.votes > 0) {
    const int run = (int)std::min<int64_t>(16, std::max<int64_t>(1, slices * tiles / W_FILL));
    const int64_t units = (tiles + run - 1) / run;
    rc = grid((units + W_WAVES - 1) / W_WAVES);
    if (rc) return rc;
    auto vote = [&](auto kernel) {
      kernel<<<g, THREADS, 0, stream>>>(qq, kk, p, ml, w_in, w_out, H, nq, q_s, k_s, c, tok0, L_cap,
                                        slices, sh.splits, run);
    };
    if (sh.votes == NT) vote(weight_votes_kernel<T, D, NT>);
    else vote(weight_votes_kernel<T, D, 1>);
  } else if (sh.staged) {
    const int kt = slices * (tiles / (W_WAVES * NT)) >= 4 * W_WGS ? NT : 1;
    rc = grid((tiles + W_WAVES * kt - 1) / (W_WAVES * kt));
    if (rc) return rc;
    if (kt == NT) go(weight_sums_staged_kernel<T, D, NT>);
    else go(weight_sums_staged_kernel<T, D, 1>);
  } else {
    const int kt = slices * (tiles / NT) >= W_FILL ? NT : 1;
    const int wq = kt == 1 && slices * tiles < W_SHARE ? W_WAVES : 1;
    const int64_t per_wg = (int64_t)kt * (W_WAVES / wq);
    rc = grid((tiles + per_wg - 1) / per_wg);
    if (rc) return rc;
    if (wq > 1) go(weight_sums_kernel<T, D, 1, W_WAVES>);
    else if (kt == NT) go(weight_sums_kernel<T, D, NT, 1>);
    else go(weight_sums_kernel<T, D, 1, 1>);
  }
  return hip_check(hipGetLastError(), "cached_attn_weights: sums launch");
}

}  // namespace sckv

using namespace sckv;

extern "C" size_t sckv_attn_weights_workspace_bytes(int32_t b, int32_t H, int32_t nq,
                                                    int32_t L_cap) {
  if (b <= 0 || H <= 0 || nq < 0 || L_cap <= 0) return 0;
  // A bound that grows with nq, so that a workspace holds every smaller call
  // too (fewer queries may be cut into more shares).  Shares are at most S and
  // at most W_FILL / units + 1, of units of at most two tiles of queries.
  const size_t rows = (size_t)b * H * nq;
  const size_t S = std::min(W_SPLITS, (L_cap + W_MIN_SHARE - 1) / W_MIN_SHARE);
  return plan_bytes(b, L_cap) +
         (rows + std::min(rows * (S - 1), (size_t)W_FILL * 2 * W_TILE)) * sizeof(float2);
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
