// Eviction of cache rows by accumulated attention weight, and the move of the
// accumulated weights (Section 3, "Manipulating Key-Value Memory for
// Inference-time Compression": rows are freed, survivors keep their order).
//
// Kernels:
//   total  : total[s][r] = sum over layers and heads of w[m][s][h][r], in fp64
//            (the order of the sums then moves a total by 2^-53 of it, far
//            below the fp32 step in which rows are compared).
//   select : one workgroup per sequence; the heavy-th largest total by radix
//            selection (8 bits a pass over counts in LDS, which one wave
//            searches), then a stable scan over the rows as in the compaction,
//            with rows equal to that total taken from the lowest on (2048 rows:
//            9 us; 31 where one thread searched the counts).
//   move   : the compaction's mover, with one more workgroup per slice of
//            weights.
#include "sckv_common.h"

namespace sckv {

// A workgroup of total: 64 rows, its waves a share of the slices each, eight
// loads of a wave in flight (8 layers x 32 heads, 8 sequences of 2048 rows:
// 8.0 us; 28.9 with four waves and one load).
constexpr int SUM_ROWS = 64;
constexpr int SUM_WAVES = 16;
constexpr int SUM_U = 8;

__global__ __launch_bounds__(64 * SUM_WAVES) void evict_total_kernel(
    const float* __restrict__ w, int32_t slices, int32_t b, int32_t H, FastDiv by_H, int32_t L_cap,
    const int32_t* __restrict__ kv_len, float* __restrict__ total) {
  __shared__ double part[SUM_WAVES][SUM_ROWS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int s = blockIdx.y; s < b; s += gridDim.y) {
    const int n = min(max(kv_len[s], 0), L_cap);
    const int r0 = blockIdx.x * SUM_ROWS;
    if (r0 >= n) continue;
    const int r = r0 + lane;
    const float* ws = w + ((int64_t)s * H * L_cap + min(r, n - 1));
    double sum = 0.0;
    for (int i = wave; i < slices; i += SUM_WAVES * SUM_U) {
      float v[SUM_U];
#pragma unroll
      for (int u = 0; u < SUM_U; ++u) {
        const int k = i + u * SUM_WAVES;
        const int m = fast_div(k, by_H);
        v[u] = k < slices ? ws[((int64_t)m * b * H + (k - m * H)) * L_cap] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < SUM_U; ++u) sum += (double)v[u];
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && r < n) {
#pragma unroll
      for (int k = 1; k < SUM_WAVES; ++k) sum += part[k][lane];
      total[(int64_t)s * L_cap + r] = (float)sum;
    }
    __syncthreads();
  }
}

// order-preserving key of a float: larger floats have larger keys, -0 equals
// +0, every NaN is the largest
__device__ __forceinline__ uint32_t order_key(float f) {
  if (f != f) return 0xffffffffu;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int SEL_THREADS = 1024;
constexpr int SEL_WAVES = SEL_THREADS / 64;

// exclusive prefix of `mine` over the workgroup's threads that set `flag`, in
// thread order, and their number
__device__ __forceinline__ int flag_rank(bool flag, int* counts, int& total) {
  const int wave = threadIdx.x >> 6;
  const uint64_t m = __ballot(flag);
  __syncthreads();  // counts of the scan before have been read
  if ((threadIdx.x & 63) == 0) counts[wave] = __popcll(m);
  __syncthreads();
  int before = 0;
  total = 0;
  for (int k = 0; k < SEL_WAVES; ++k) {
    const int c = counts[k];
    if (k < wave) before += c;
    total += c;
  }
  return before + mask_rank(m);
}

__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(
    const float* __restrict__ total, int32_t* __restrict__ kv_len, int32_t* __restrict__ tok_idx,
    int32_t* __restrict__ pos_ids, int32_t L_cap, int32_t heavy, int32_t recent,
    int32_t* __restrict__ kept_src) {
  __shared__ int hist[256];
  __shared__ int counts[SEL_WAVES];
  __shared__ int pick[2];  // the pass's digit, and the rows still to take
  const int s = blockIdx.x;
  const int tid = threadIdx.x;
  const int n = min(max(kv_len[s], 0), L_cap);
  const float* tot = total + (int64_t)s * L_cap;
  int32_t* tok = tok_idx + (int64_t)s * L_cap;
  int32_t* pp = pos_ids + (int64_t)s * L_cap;
  int32_t* ks = kept_src + (int64_t)s * L_cap;
  const int first_recent = n - min(recent, n);  // rows from here on stay
  const bool all = (int64_t)heavy + recent >= n;
  // the heavy-th largest key of rows [0, first_recent), digit by digit; heavy
  // is below first_recent here
  uint32_t key = 0;
  int take = heavy;  // rows to take of those with the digits found so far
  if (!all && heavy > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int r = tid; r < first_recent; r += SEL_THREADS) {
        const uint32_t k = order_key(tot[r]);
        if (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8)))
          atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      // the largest digit with at least `take` rows from it upwards: lane l
      // has digits 255 - 4 l downwards
      if (tid < 64) {
        int c[4], sum = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += c[k] = hist[255 - 4 * tid - k];
        int upto = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const int x = __shfl_up(upto, off, 64);
          if (tid >= off) upto += x;
        }
        int left = take - (upto - sum);
        if (left > 0 && left <= sum) {  // one lane: take is at most the rows counted
          int k = 0;
          while (k < 3 && c[k] < left) left -= c[k++];
          pick[0] = 255 - 4 * tid - k;
          pick[1] = left;
        }
      }
      __syncthreads();
      key |= (uint32_t)pick[0] << shift;
      take = pick[1];
      __syncthreads();
    }
  }
  int kept = 0, equals = 0;
  for (int base = 0; base < n; base += SEL_THREADS) {
    const int r = base + tid;
    const bool in = r < n;
    const int t = in ? tok[r] : 0, p = in ? pp[r] : 0;
    bool keep = in && (all || r >= first_recent);
    bool eq = false;
    if (in && !keep && heavy > 0) {
      const uint32_t k = order_key(tot[r]);
      keep = k > key;
      eq = k == key;
    }
    int n_eq, n_keep;
    const int eq_rank = equals + flag_rank(eq, counts, n_eq);
    keep = keep || (eq && eq_rank < take);
    wait_vmem();  // the chunk's tokens and positions are read before any is written
    const int rank = kept + flag_rank(keep, counts, n_keep);
    if (keep) {
      tok[rank] = t;
      pp[rank] = p;
      ks[rank] = r;
    }
    equals += n_eq;
    kept += n_keep;
  }
  for (int r = kept + tid; r < L_cap; r += SEL_THREADS) ks[r] = -1;
  __syncthreads();  // every thread has read kv_len[s]
  if (tid == 0) kv_len[s] = kept;
}

__global__ __launch_bounds__(WMOVE_THREADS) void move_weights_kernel(
    const float* w, float* w_out, int32_t b, int32_t H, int32_t L_cap,
    const int32_t* __restrict__ kv_len, const int32_t* __restrict__ kept_src) {
  move_weights(w, w_out, blockIdx.x, b, H, L_cap, kv_len, kept_src);
}

}  // namespace sckv

using namespace sckv;

extern "C" int kv_compact_weights(float* w, float* w_out, int32_t M, int32_t b, int32_t H,
                                  int32_t L_cap, const int32_t* kv_len,
                                  const int32_t* kept_src_row, hipStream_t stream) {
  clear_error();
  if (!w || !kv_len || !kept_src_row) return fail(SCKV_EINVAL, "kv_compact_weights: null pointer");
  if (M <= 0 || b <= 0 || H <= 0 || L_cap <= 0)
    return fail(SCKV_EINVAL, "kv_compact_weights: sizes must be positive");
  if (L_cap > 65536) return fail(SCKV_EUNSUP, "kv_compact_weights: L_cap above 65536");
  if (!aligned4(w) || !aligned4(w_out))
    return fail(SCKV_EINVAL, "kv_compact_weights: w and w_out must be 4-byte aligned");
  const int64_t slices = (int64_t)M * b * H;
  if (slices > 0x7fffffff) return fail(SCKV_EUNSUP, "kv_compact_weights: too many slices");
  move_weights_kernel<<<(unsigned)slices, WMOVE_THREADS, 0, stream>>>(w, w_out ? w_out : w, b, H, L_cap,
                                                                      kv_len, kept_src_row);
  return hip_check(hipGetLastError(), "kv_compact_weights: launch");
}

extern "C" int kv_evict(void* kv, void* kv_out, float* w, float* w_out, int32_t M, int32_t b,
                        int32_t H, int32_t L_cap, int32_t d_head, sckv_dtype dt, int32_t* kv_len,
                        int32_t* tok_idx, int32_t* pos_ids, int32_t heavy, int32_t recent,
                        float* total, int32_t* kept_src_row, hipStream_t stream) {
  clear_error();
  if (!kv || !w || !kv_len || !tok_idx || !pos_ids || !total || !kept_src_row)
    return fail(SCKV_EINVAL, "kv_evict: null pointer");
  if (!valid_dtype(dt)) return fail(SCKV_EINVAL, "kv_evict: unknown dtype");
  if (!supported_d(d_head)) return fail(SCKV_EUNSUP, "kv_evict: d_head must be 64 or 80");
  if (M <= 0 || b <= 0 || H <= 0 || L_cap <= 0)
    return fail(SCKV_EINVAL, "kv_evict: sizes must be positive");
  if (L_cap > 65536) return fail(SCKV_EUNSUP, "kv_evict: L_cap above 65536");
  if (heavy < 0 || recent < 0 || (heavy == 0 && recent == 0))
    return fail(SCKV_EINVAL, "kv_evict: heavy and recent must be >= 0 and not both 0");
  if (kv_out == kv || w_out == w)
    return fail(SCKV_EINVAL, "kv_evict: an output must differ from its input (pass null for in place)");
  if (!aligned16(kv) || (kv_out && !aligned16(kv_out)) || !aligned4(w) || !aligned4(w_out))
    return fail(SCKV_EINVAL, "kv_evict: buffers must be 16-byte aligned");
  const int64_t slices = (int64_t)M * b * H;
  if (3 * slices > 0x7fffffff) return fail(SCKV_EUNSUP, "kv_evict: too many slices");
  const dim3 grid((unsigned)((L_cap + SUM_ROWS - 1) / SUM_ROWS), (unsigned)(b < 65535 ? b : 65535));
  evict_total_kernel<<<grid, 64 * SUM_WAVES, 0, stream>>>(w, M * H, b, H, make_div((uint32_t)H), L_cap,
                                                          kv_len, total);
  int rc = hip_check(hipGetLastError(), "kv_evict: total launch");
  if (rc) return rc;
  evict_select_kernel<<<b, SEL_THREADS, 0, stream>>>(total, kv_len, tok_idx, pos_ids, L_cap, heavy,
                                                     recent, kept_src_row);
  rc = hip_check(hipGetLastError(), "kv_evict: select launch");
  if (rc) return rc;
  return launch_move(kv, kv_out, M, b, H, L_cap, d_head, dt, kv_len, kept_src_row, "kv_evict: move launch",
                     stream, w, w_out ? w_out : w);
}
