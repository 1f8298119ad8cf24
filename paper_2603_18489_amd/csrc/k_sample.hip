// A token drawn from each row of logits: temperature, top-k, top-p and min-p, from a given uniform number.
//
// With e_i = exp((z_i - max z) / T) and the tokens in the order (z descending, id ascending), a row keeps the tokens of rank j
// with  j < top_k,  sum_{ranks < j} e < top_p * (sum of the top_k),  e >= min_p  and z > -inf: a prefix of that order.  The token
// drawn is the lowest id whose running sum of kept e, in the order of the ids, is above u times the sum of all kept.
//
// Sums decide between neighbours: in a nearly flat row of 126464 tokens the borders lie 8e-6 apart, and a running sum in float32
// would pick a neighbour in per cents of the rows.  So e is a 64-bit exponential, rounded to a multiple of 2^-46, and every sum is
// one of integers: exact, independent of the order, below 2^64 for the 163840 tokens a row may have.  (64-bit multiply-adds run at
// the rate of 32-bit ones that are not packed.)
#include "ec_internal.h"
#include "k_exp.h"

namespace ec {

typedef unsigned long long u64;

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;

// logits in order: larger for larger z, -0 and +0 the same
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// sum of the lanes below this one
__device__ __forceinline__ u64 wave_before_u64(u64 v) {
  const int lane = threadIdx.x & 63;
  u64 s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 t = __shfl_up(s, o, 64);
    s += lane >= o ? t : 0;
  }
  return s - v;
}

struct SampleRow {
  double m, scale;   // maximum; log2(e) / T
  __device__ __forceinline__ u64 weight(float z) const { return exp2_fixed46(((double)z - m) * scale); }
};

// One block a row, the row read from memory for every question asked of it.
template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(const T* __restrict__ logits, int V, size_t ld,
                                                                    const float* __restrict__ uniforms, SampleArgs a,
                                                                    int* __restrict__ tokens, float4* __restrict__ stats) {
  __shared__ uint32_t cnt[2048];
  __shared__ u64 mass[2048];
  __shared__ u64 wsum[kSampleWaves];
  __shared__ uint32_t wcnt[kSampleWaves];
  __shared__ u64 found_mass, found_above_mass;
  __shared__ uint32_t found_bin, found_cnt, found_above_cnt;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* z = logits + (size_t)blockIdx.x * ld;

  // maximum; a NaN anywhere or no finite maximum: no token
  float m = -INFINITY;
  bool nan = false;
  for (int i = tid; i < V; i += kSampleThreads) {
    const float v = load_f32(z + i);
    nan |= v != v;
    m = fmaxf(m, v);
  }
  m = wave_max_dpp(fmaxf(m, -INFINITY));
  const u64 any_nan = __builtin_amdgcn_ballot_w64(nan);
  if (lane == 0) { wsum[wave] = any_nan; wcnt[wave] = __float_as_uint(m); }
  __syncthreads();
  u64 nans = 0;
  for (int w = 0; w < kSampleWaves; ++w) { nans |= wsum[w]; m = fmaxf(m, __uint_as_float(wcnt[w])); }
  if (nans || !(fabsf(m) < INFINITY)) {
    if (tid == 0) {
      tokens[blockIdx.x] = -1;
      const float q = __builtin_nanf("");
      stats[blockIdx.x] = make_float4(q, q, q, q);
    }
    return;
  }
  const SampleRow row = {(double)m, a.scale};

  // block sum of u64, the same in every thread
  auto total = [&](u64 v) {
    v = wave_sum_u64(v);
    __syncthreads();
    if (lane == 0) wsum[wave] = v;
    __syncthreads();
    u64 s = 0;
    for (int w = 0; w < kSampleWaves; ++w) s += wsum[w];
    return s;
  };
  u64 part = 0;
  for (int i = tid; i < V; i += kSampleThreads) part += row.weight(load_f32(z + i));
  const u64 all = total(part);

  // The cut: tokens with a larger key are kept, and the first `ties` of those that have it.
  uint32_t cut = 0, ties = 0;   // (0: below every logit's key)
  // Digit by digit: of the keys that begin like the cut, how many have each next digit and what they weigh.
  auto select = [&](bool by_mass, u64 want) {
    uint32_t prefix = 0, above_cnt = 0;
    u64 above_mass = 0;
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
      for (int b = tid; b < 2048; b += kSampleThreads) { cnt[b] = 0; mass[b] = 0; }
      __syncthreads();
      for (int i = tid; i < V; i += kSampleThreads) {
        const float v = load_f32(z + i);
        const uint32_t k = key_of(v);
        if (v > -INFINITY && (pass == 0 || (k >> (shift + bits)) == prefix)) {
          const uint32_t b = (k >> shift) & ((1u << bits) - 1);
          atomicAdd(&cnt[b], 1u);
          atomicAdd(&mass[b], row.weight(v));
        }
      }
      __syncthreads();
      // two bins a thread, the largest keys first
      const int b0 = 2047 - 2 * tid, b1 = b0 - 1;
      const uint32_t c0 = cnt[b0], c1 = cnt[b1];
      const u64 m0 = mass[b0], m1 = mass[b1];
      const u64 cb = wave_before_u64(c0 + c1), mb = wave_before_u64(m0 + m1);
      if (lane == 63) { wcnt[wave] = (uint32_t)cb + c0 + c1; wsum[wave] = mb + m0 + m1; }
      __syncthreads();
      uint32_t cx = above_cnt + (uint32_t)cb;
      u64 mx = above_mass + mb;
      for (int w = 0; w < wave; ++w) { cx += wcnt[w]; mx += wsum[w]; }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t c = h ? c1 : c0;
        const u64 s = h ? m1 : m0;
        const bool here = by_mass ? mx < want && want <= mx + s : cx < want && want <= (u64)cx + c;
        if (here) {   // (one bin of all)
          found_bin = h ? b1 : b0;
          found_cnt = c; found_mass = s; found_above_cnt = cx; found_above_mass = mx;
        }
        cx += c; mx += s;
      }
      __syncthreads();
      prefix = (prefix << bits) | found_bin;
      above_cnt = found_above_cnt;
      above_mass = found_above_mass;
    }
    cut = prefix;
    if (by_mass) {
      const u64 each = found_mass / found_cnt;
      ties = (uint32_t)((want - above_mass + each - 1) / each);
    } else {
      ties = (uint32_t)want - above_cnt;
    }
    // what is kept of it
    const u64 sum = above_mass + (found_mass / found_cnt) * ties;
    __syncthreads();
    return sum;
  };
  u64 of_k = all;
  if (a.top_k > 0 && a.top_k < V) {
    part = 0;
    for (int i = tid; i < V; i += kSampleThreads) part += load_f32(z + i) > -INFINITY;
    if (total(part) > (u64)a.top_k) of_k = select(false, a.top_k);
  }
  if (a.top_p < 1.0) {
    const double want = ceil(a.top_p * (double)of_k);
    select(true, want < 1.0 ? 1 : (u64)want);
  }

  // Each wave goes through a range of the ids, so that running sums are those of the ids.
  const int per = ((V + kSampleWaves - 1) / kSampleWaves + 63) / 64 * 64;
  const int lo = min(wave * per, V), hi = min(lo + per, V);
  uint32_t before = 0;   // of the tokens at the cut, those with a lower id
  if (cut) {
    uint32_t n = 0;
    for (int i = lo + lane; i < hi; i += 64) n += key_of(load_f32(z + i)) == cut;
    n = (uint32_t)wave_sum_u64(n);
    if (lane == 0) wcnt[wave] = n;
    __syncthreads();
    for (int w = 0; w < wave; ++w) before += wcnt[w];
  }
  // weight of id i if it is kept, else 0; `seen` goes on with the tokens at the cut
  auto kept_weight = [&](int i, uint32_t& seen, uint32_t& n) -> u64 {
    const bool in = i < hi;
    const float v = in ? load_f32(z + i) : -INFINITY;
    const uint32_t k = key_of(v);
    const u64 tied = __builtin_amdgcn_ballot_w64(in && k == cut);
    const bool first = seen + (uint32_t)__builtin_popcountll(tied & ((1ull << lane) - 1)) < ties;
    seen += (uint32_t)__builtin_popcountll(tied);
    const u64 w = row.weight(v);
    const bool keep = in && v > -INFINITY && (k > cut || (k == cut && first)) && w >= a.min_weight;
    n += keep;
    return keep ? w : 0;
  };
  uint32_t seen = before, n_kept = 0;
  part = 0;
  for (int i0 = lo; i0 < hi; i0 += 64) part += kept_weight(i0 + lane, seen, n_kept);
  part = wave_sum_u64(part);
  n_kept = (uint32_t)wave_sum_u64(n_kept);
  __syncthreads();
  if (lane == 0) { wsum[wave] = part; wcnt[wave] = n_kept; }
  __syncthreads();
  u64 kept = 0, mine = 0;
  n_kept = 0;
  for (int w = 0; w < kSampleWaves; ++w) {
    if (w < wave) mine += wsum[w];
    kept += wsum[w];
    n_kept += wcnt[w];
  }
  // running sum > u * kept  <=>  running sum >= floor(u * kept) + 1
  const float u = uniforms[blockIdx.x];
  const double at = floor((u >= 0.f ? (double)fminf(u, 0x1.fffffep-1f) : 0.0) * (double)kept);
  const u64 want = min((u64)at + 1, kept);
  if (mine < want && want <= mine + part) {
    seen = before;
    uint32_t n = 0;
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const u64 w = kept_weight(i0 + lane, seen, n);
      const u64 upto = mine + wave_before_u64(w) + w;
      const u64 past = __builtin_amdgcn_ballot_w64(upto >= want);
      if (past) {
        if (lane == __builtin_ctzll(past)) {
          tokens[blockIdx.x] = i0 + lane;
          // (its own e unrounded: it may be a small one)
          const double e = exp2_times_2to46(((double)load_f32(z + i0 + lane) - row.m) * row.scale);
          stats[blockIdx.x] = make_float4((float)(e / (double)kept), (float)(e / (double)all), (float)n_kept,
                                          (float)((double)kept / (double)all));
        }
        break;
      }
      mine += wave_sum_u64(w);
    }
  }
}

void launch_sample_rows(const void* logits, bool bf16, int rows, int V, size_t ld, const float* uniforms, const SampleArgs& a,
                        int* tokens, float4* stats, hipStream_t s) {
  if (bf16)
    sample_row_kernel<<<rows, kSampleThreads, 0, s>>>((const bf16_t*)logits, V, ld, uniforms, a, tokens, stats);
  else
    sample_row_kernel<<<rows, kSampleThreads, 0, s>>>((const float*)logits, V, ld, uniforms, a, tokens, stats);
}

}  // namespace ec
