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
template <int CTRL> __device__ __forceinline__ u64 dpp_u64(u64 v) {
  return (u64)(uint32_t)dpp_i<CTRL>((int)(uint32_t)(v >> 32)) << 32 | (uint32_t)dpp_i<CTRL>((int)(uint32_t)v);
}
__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
  v += dpp_u64<0xB1>(v); v += dpp_u64<0x4E>(v); v += dpp_u64<0x141>(v); v += dpp_u64<0x140>(v);
  auto halves = [](u64 x, float (*other)(float)) {
    return (u64)__float_as_uint(other(__uint_as_float((uint32_t)(x >> 32)))) << 32 | __float_as_uint(other(__uint_as_float((uint32_t)x)));
  };
  v += halves(v, other_row);
  return v + halves(v, other_half);
}
// sum of the lanes below this one: inside rows of 16, then the rows' last lanes to the rows behind them
template <int CTRL, int ROWS> __device__ __forceinline__ u64 dpp_rows_u64(u64 v) {
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 wave_before_u64(u64 v) {
  u64 s = v;
  s += dpp_rows_u64<0x111, 0xf>(s); s += dpp_rows_u64<0x112, 0xf>(s); s += dpp_rows_u64<0x114, 0xf>(s); s += dpp_rows_u64<0x118, 0xf>(s);
  s += dpp_rows_u64<0x142, 0xa>(s);
  s += dpp_rows_u64<0x143, 0xc>(s);
  return s - v;
}

struct SampleRow {
  double m, scale;   // maximum; log2(e) / T
  __device__ __forceinline__ u64 weight(float z) const { return exp2_fixed46(((double)z - m) * scale); }
};

// What a block of 1024 threads works through, in the order of the ids: each wave has a range of its own, 64 neighbours at a time.
// each(f): f(place, logit, there) for the lane's elements; a place that is not there has a logit of -inf.
template <int NE> struct InRegisters {
  float v[NE];
  int first, n;   // the lane's first place; places in all
  template <typename T> __device__ __forceinline__ void fetch(const T* z, int count) {
    n = count;
    first = (threadIdx.x >> 6) * (64 * NE) + (threadIdx.x & 63);
#pragma unroll
    for (int e = 0; e < NE; ++e) v[e] = load_f32(z + min(first + e * 64, n - 1));
#pragma unroll
    for (int e = 0; e < NE; ++e) v[e] = first + e * 64 < n ? v[e] : -INFINITY;
  }
  template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int e = 0; e < NE; ++e) f(first + e * 64, v[e], first + e * 64 < n);
  }
};
template <typename T> struct InMemory {
  const T* z;
  int first, end, n;
  __device__ __forceinline__ void fetch(const T* from, int count) {
    z = from; n = count;
    const int per = ((n + kSampleWaves - 1) / kSampleWaves + 63) / 64 * 64, lo = min((int)(threadIdx.x >> 6) * per, n);
    first = lo + (threadIdx.x & 63);
    end = min(lo + per, n);
  }
  template <typename F> __device__ __forceinline__ void each(F f) const {
    const int rounds = (end - (first - (int)(threadIdx.x & 63)) + 63) / 64;   // (the same for all lanes)
    for (int e0 = 0; e0 < rounds; e0 += 8) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = load_f32(z + min(first + (e0 + e) * 64, n - 1));
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e0 + e < rounds) f(first + (e0 + e) * 64, first + (e0 + e) * 64 < end ? v[e] : -INFINITY, first + (e0 + e) * 64 < end);
    }
  }
};

// LDS of a block that looks for the cut
constexpr int kDigits = 2048;
struct Scratch {
  u64 mass[kDigits];
  uint32_t cnt[kDigits];
  u64 wsum[kSampleWaves];
  uint32_t wcnt[kSampleWaves];
  u64 found_mass, found_above_mass, few_mass[64];
  uint32_t found_bin, found_cnt, found_above_cnt, few_key[64], n_few;
  int found_id, few_place[64];
};

__device__ __forceinline__ u64 block_sum_u64(u64 v, Scratch& x) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) x.wsum[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) s += x.wsum[w];
  return s;
}
// the block's maximum; true: there is a NaN
__device__ __forceinline__ bool block_max(float& m, bool nan, Scratch& x) {
  m = wave_max_dpp(fmaxf(m, -INFINITY));
  const u64 any = __builtin_amdgcn_ballot_w64(nan);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) { x.wsum[threadIdx.x >> 6] = any; x.wcnt[threadIdx.x >> 6] = __float_as_uint(m); }
  __syncthreads();
  u64 nans = 0;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) { nans |= x.wsum[w]; m = fmaxf(m, __uint_as_float(x.wcnt[w])); }
  return nans != 0;
}

// Which tokens are kept: those with a larger key, and of those that have it the ones at a place up to `last`.
struct Cut {
  uint32_t key = 0;
  int last = INT_MAX;
  __device__ __forceinline__ bool keeps(uint32_t k, int place) const { return k > key || (k == key && place <= last); }
};

// Among kDigits bins, the largest logits first: the one of the token with which `want` tokens (by_mass: a weight of `want`) are reached.
__device__ __forceinline__ void find_bin(bool by_mass, u64 want, uint32_t above_cnt, u64 above_mass, Scratch& x) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b0 = 2 * threadIdx.x;
  const uint32_t c0 = x.cnt[b0], c1 = x.cnt[b0 + 1];
  const u64 m0 = x.mass[b0], m1 = x.mass[b0 + 1];
  u64 cx = wave_before_u64(c0 + c1), mx = wave_before_u64(m0 + m1);
  if (lane == 63) { x.wcnt[wave] = (uint32_t)cx + c0 + c1; x.wsum[wave] = mx + m0 + m1; }
  __syncthreads();
  cx += above_cnt;
  mx += above_mass;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) { cx += w < wave ? x.wcnt[w] : 0u; mx += w < wave ? x.wsum[w] : 0ull; }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t c = h ? c1 : c0;
    const u64 s = h ? m1 : m0;
    if (by_mass ? mx < want && want <= mx + s : cx < want && want <= cx + c) {   // (one of all)
      x.found_bin = b0 + h;
      x.found_cnt = c; x.found_mass = s; x.found_above_cnt = (uint32_t)cx; x.found_above_mass = mx;
    }
    cx += c; mx += s;
  }
  __syncthreads();
}
__device__ __forceinline__ void clear_bins(Scratch& x) {
  __syncthreads();
  for (int b = threadIdx.x; b < kDigits; b += kSampleThreads) { x.cnt[b] = 0; x.mass[b] = 0; }
  if (threadIdx.x == 0) x.n_few = 0;
  __syncthreads();
}

// The cut after which `want` tokens are kept (by_mass: after which what is kept first weighs `want` or more); there are as many.  Returns what is
// kept.  First bins of equal width in z, 32 T in all; if up to 64 tokens share the one of the cut, a wave ranks them.  Otherwise digit
// by digit of their keys: of those that begin like the cut, how many have each next digit and what they weigh.
template <typename S>
__device__ u64 select_cut(const S& src, const SampleRow& row, bool by_mass, u64 want, Cut& cut, Scratch& x) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // (a fixed order of operations on one logit: it falls into the same bin each time, and a larger one into none behind it)
  const float m = (float)row.m, wide = fminf((float)(row.scale * (kDigits / (32 * 1.4426950408889634))), 1e30f);
  auto bin = [&](float v) { return (int)fminf((m - v) * wide, (float)(kDigits - 1)); };
  clear_bins(x);
  uint32_t far = 0;
  u64 far_mass = 0;
  src.each([&](int, float v, bool) {
    if (v > -INFINITY) {
      const int b = bin(v);
      const u64 w = row.weight(v);
      if (b < kDigits - 1) { atomicAdd(&x.cnt[b], 1u); atomicAdd(&x.mass[b], w); }
      else { ++far; far_mass += w; }   // (most of a peaked row: not all to one address)
    }
  });
  far = (uint32_t)wave_sum_u64(far);
  far_mass = wave_sum_u64(far_mass);
  if (lane == 0 && far) { atomicAdd(&x.cnt[kDigits - 1], far); atomicAdd(&x.mass[kDigits - 1], far_mass); }
  __syncthreads();
  find_bin(by_mass, want, 0, 0, x);
  const int at = x.found_bin;
  const uint32_t n = x.found_cnt;
  uint32_t above_cnt = x.found_above_cnt;
  u64 above_mass = x.found_above_mass;
  if (n <= 64) {
    src.each([&](int place, float v, bool) {
      if (v > -INFINITY && bin(v) == at) {
        const uint32_t i = atomicAdd(&x.n_few, 1u);
        x.few_key[i] = key_of(v);
        x.few_place[i] = place;
        x.few_mass[i] = row.weight(v);
      }
    });
    __syncthreads();
    // every wave ranks them: a lane each, by key, then place
    const int mine = lane < (int)n ? lane : 0;
    const uint32_t key = x.few_key[mine];
    const int place = x.few_place[mine];
    uint32_t rank = above_cnt;
    u64 mass = above_mass;
    for (int j = 0; j < (int)n; ++j) {
      const bool ahead = x.few_key[j] > key || (x.few_key[j] == key && x.few_place[j] < place);
      rank += ahead;
      mass += ahead ? x.few_mass[j] : 0;
    }
    const u64 upto = mass + x.few_mass[mine];
    const u64 is = __builtin_amdgcn_ballot_w64(lane < (int)n && (by_mass ? mass < want && want <= upto : rank + 1 == (uint32_t)want));
    const int l = __builtin_ctzll(is);
    cut.key = (uint32_t)__builtin_amdgcn_readlane((int)key, l);
    cut.last = __builtin_amdgcn_readlane(place, l);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(upto >> 32), l), lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)upto, l);
    return (u64)hi << 32 | lo;
  }
  uint32_t prefix = 0;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    clear_bins(x);
    src.each([&](int, float v, bool) {
      const uint32_t k = key_of(v);
      if (v > -INFINITY && bin(v) == at && (pass == 0 || (k >> (shift + bits)) == prefix)) {
        const uint32_t b = (1u << bits) - 1 - ((k >> shift) & ((1u << bits) - 1));   // (the largest digit first)
        atomicAdd(&x.cnt[b], 1u);
        atomicAdd(&x.mass[b], row.weight(v));
      }
    });
    __syncthreads();
    find_bin(by_mass, want, above_cnt, above_mass, x);
    prefix = (prefix << bits) | ((1u << bits) - 1 - x.found_bin);
    above_cnt = x.found_above_cnt;
    above_mass = x.found_above_mass;
  }
  const u64 each = x.found_mass / x.found_cnt;   // (equal logits, equal weights)
  const uint32_t ties = by_mass ? (uint32_t)((want - above_mass + each - 1) / each) : (uint32_t)want - above_cnt;
  cut.key = prefix;
  cut.last = INT_MAX;
  if (ties < x.found_cnt) {   // the place of the last of them
    uint32_t tied = 0;
    src.each([&](int, float v, bool in) { tied += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(in && key_of(v) == prefix)); });
    __syncthreads();
    if (lane == 0) x.wcnt[wave] = tied;
    __syncthreads();
    uint32_t seen = 0;
    for (int w = 0; w < wave; ++w) seen += x.wcnt[w];
    if (seen < ties && ties <= seen + tied)
      src.each([&](int place, float v, bool in) {
        const u64 same = __builtin_amdgcn_ballot_w64(in && key_of(v) == prefix);
        const uint32_t nth = seen + (uint32_t)__builtin_popcountll(same & ((2ull << lane) - 1));
        if (in && key_of(v) == prefix && nth == ties) x.found_id = place;
        seen += (uint32_t)__builtin_popcountll(same);
      });
    __syncthreads();
    cut.last = x.found_id;
  }
  return above_mass + each * ties;
}

// what the tokens before one have to weigh for it to go
__device__ __forceinline__ u64 mass_wanted(double top_p, u64 total) {
  const double want = ceil(top_p * (double)total);
  return want < 1.0 ? 1 : min((u64)want, total);
}
// running sum > u * total  <=>  running sum >= this
__device__ __forceinline__ u64 draw_at(float u, u64 total) {
  const double at = floor((u >= 0.f ? (double)fminf(u, 0x1.fffffep-1f) : 0.0) * (double)total);
  return min((u64)at + 1, total);
}

// The place of the token: the first whose running sum of kept weights is `want` or more.  kept, count: of these tokens; `at` is called by
// every thread with them and says what is wanted.  Returns true to one lane.
template <typename S, typename W>
__device__ __forceinline__ bool draw_place(const S& src, const SampleRow& row, const Cut& cut, int shift, u64 min_weight, Scratch& x,
                                           u64& kept, uint32_t& count, W wanted, int& place, float& logit) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 part = 0;
  uint32_t n = 0;
  auto weight = [&](int at, float v) {
    const u64 w = row.weight(v);
    const bool keep = v > -INFINITY && w >= min_weight && cut.keeps(key_of(v), at + shift);
    n += keep;
    return keep ? w : 0;
  };
  src.each([&](int at, float v, bool) { part += weight(at, v); });
  part = wave_sum_u64(part);
  n = (uint32_t)wave_sum_u64(n);
  __syncthreads();
  if (lane == 0) { x.wsum[wave] = part; x.wcnt[wave] = n; }
  __syncthreads();
  u64 mine = 0;
  kept = 0;
  count = 0;
  for (int w = 0; w < kSampleWaves; ++w) {
    if (w < wave) mine += x.wsum[w];
    kept += x.wsum[w];
    count += x.wcnt[w];
  }
  const u64 want = wanted(kept);
  bool found = false, over = !(mine < want && want <= mine + part);
  if (!over)
    src.each([&](int at, float v, bool) {
      if (over) return;
      const u64 w = weight(at, v);
      const u64 upto = mine + wave_before_u64(w) + w;
      const u64 past = __builtin_amdgcn_ballot_w64(upto >= want);
      if (past) {
        over = true;
        if (lane == __builtin_ctzll(past)) { found = true; place = at; logit = v; }
      }
      mine += wave_sum_u64(w);
    });
  return found;
}

__device__ __forceinline__ void no_token(int* tokens, float4* stats, int r) {
  if (threadIdx.x == 0) {
    const float q = __builtin_nanf("");
    tokens[r] = -1;
    stats[r] = make_float4(q, q, q, q);
  }
}
__device__ __forceinline__ void put_token(int* tokens, float4* stats, int r, int id, float z, const SampleRow& row, u64 kept, uint32_t n,
                                          u64 all) {
  const double e = exp2_times_2to46(((double)z - row.m) * row.scale);   // (unrounded: it may be a small one)
  tokens[r] = id;
  stats[r] = make_float4((float)(e / (double)kept), (float)(e / (double)all), (float)n, (float)((double)kept / (double)all));
}

template <typename S> __device__ __forceinline__ u64 sum_weights(const S& src, const SampleRow& row, Scratch& x) {
  u64 sum = 0;
  src.each([&](int, float v, bool) { sum += row.weight(v); });   // (-inf: 0)
  return block_sum_u64(sum, x);
}

// All of a row by one block.
template <typename S>
__device__ void sample_whole(const S& src, const SampleRow& row, const SampleArgs& a, float u, int r, Scratch& x, int* tokens,
                             float4* stats) {
  const u64 all = sum_weights(src, row, x);
  Cut cut;
  u64 of_k = all;
  u64 finite = 0;
  src.each([&](int, float v, bool) { finite += v > -INFINITY; });
  finite = block_sum_u64(finite, x);
  for (int by_mass = 0; by_mass < 2; ++by_mass) {
    if (by_mass ? a.top_p >= 1.0 : a.top_k == 0 || (u64)a.top_k >= finite) continue;
    of_k = select_cut(src, row, by_mass, by_mass ? mass_wanted(a.top_p, of_k) : (u64)a.top_k, cut, x);
  }
  u64 kept;
  uint32_t n;
  int place;
  float z;
  if (draw_place(src, row, cut, 0, a.min_weight, x, kept, n, [&](u64 k) { return draw_at(u, k); }, place, z))
    put_token(tokens, stats, r, place, z, row, kept, n, all);
}

// A row of up to 1024 NE logits: one block, which reads it once.
template <typename T, int NE>
__global__ __launch_bounds__(kSampleThreads) void sample_small_kernel(const T* __restrict__ logits, int V, size_t ld,
                                                                      const float* __restrict__ uniforms, SampleArgs a,
                                                                      int* __restrict__ tokens, float4* __restrict__ stats) {
  __shared__ Scratch x;
  const int r = blockIdx.x;
  InRegisters<NE> src;
  src.fetch(logits + (size_t)r * ld, V);
  float m = -INFINITY;
  bool nan = false;
  src.each([&](int, float v, bool) { m = fmaxf(m, v); nan |= v != v; });
  if (block_max(m, nan, x) || !(fabsf(m) < INFINITY)) { no_token(tokens, stats, r); return; }
  sample_whole(src, SampleRow{(double)m, a.scale}, a, uniforms[r], r, x, tokens, stats);
}

// ---- longer rows: parts of 1024 NE logits to a block --------------------------------------------------
// A part's maximum and, without filters, its weights' sum.  With filters, how its weights spread over kBins bins of T / 16 in z, counted down
// from its largest logit; the last one is all that lies 32 T and more below it, which weighs nothing (less than 2^-46 of the maximum).  Bins
// begin at multiples of T / 16, so that a row's parts are put together by moving them by whole bins.  A weight of bin B is
// e^(B / 16) e^(rho / 16) with rho = z 16 / T - B in [0, 1], and what is added for it one number: 2^48 (a count) plus (e^(rho / 16) - 0.99) 2^36,
// whose sums over the 32768 logits of a part stay below 2^48.
constexpr int kBins = 512, kList = 8192, kPartsMax = 40, kSampleBatch = 1024;
struct PartSum {
  float m;
  int count;   // -1: a NaN.  With filters: the logits of the last bin, -2 where logits are too large for the bins (2^16 T).  Without: all above -inf
  u64 sum;     // (without filters)
};
typedef u64 Spread[kBins];

// number of the bin of a logit, counted up in z; whole, and monotonous whatever z
__device__ __forceinline__ float bin_of(float z, float per_z) { return floorf(fminf(fmaxf(z * per_z, -1e30f), 1e30f)); }
__device__ __forceinline__ int bins_below(float top, float b) { return (int)fminf(top - b, (float)(kBins - 1)); }
__device__ __forceinline__ u64 spread_of(float z, float b, double per_z) {
  const double rho = fma((double)z, per_z, -(double)b);
  // e^(rho / 16) - 0.99, degree 5 through the Chebyshev nodes of [-1/16, 17/16] (rounding z 16 / T may move a border that far): off by 9e-14
  double q = 0x1.19bf4680e8241p+9;
  q = fma(q, rho, 0x1.552f36e70099ep+15);
  q = fma(q, rho, 0x1.55559db67be1cp+21);
  q = fma(q, rho, 0x1.ffffff9698380p+26);
  q = fma(q, rho, 0x1.0000000009bfep+32);
  q = fma(q, rho, 0x1.47ae147aeca4fp+29);
  return (u64)__double_as_longlong(q + 0x1p52) + ((1ull << 48) - 0x4330000000000000ull);
}
// what a bin's sum weighs, as a whole number of 2^-46 of the weight at the maximum m of the row, whose bin is `top`
__device__ __forceinline__ double bin_unit(float m, float top, int b, double per_z) {
  return exp2_times_2to46((-fma((double)m, per_z, -(double)top) - b) * (1.4426950408889634 / 16));
}
__device__ __forceinline__ u64 bin_mass(u64 cnt, u64 frac, double unit) {
  return (u64)((0.99 * (double)cnt + (double)frac * 0x1p-36) * unit + 0.5);
}

template <typename T, int NE, bool FILTERS>
__global__ __launch_bounds__(kSampleThreads) void sample_parts_kernel(const T* __restrict__ logits, int V, size_t ld, double scale,
                                                                      double per_z, PartSum* __restrict__ sums,
                                                                      Spread* __restrict__ spreads) {
  __shared__ u64 spread[kBins], wsum[kSampleWaves];
  __shared__ float wmax[kSampleWaves];
  __shared__ int wnan[kSampleWaves], wcnt[kSampleWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int part = blockIdx.x, r = blockIdx.y, lo = part * (kSampleThreads * NE), out = r * gridDim.x + part;
  InRegisters<NE> src;
  src.fetch(logits + (size_t)r * ld + lo, min(V - lo, kSampleThreads * NE));
  if (FILTERS && threadIdx.x < kBins) spread[threadIdx.x] = 0;
  float m = -INFINITY;
  bool nan = false;
  src.each([&](int, float v, bool) { m = fmaxf(m, v); nan |= v != v; });
  m = wave_max_dpp(m);
  nan = __builtin_amdgcn_ballot_w64(nan) != 0;
  if (lane == 0) { wmax[wave] = m; wnan[wave] = nan; }
  __syncthreads();
  m = wave_max_dpp(wmax[lane & (kSampleWaves - 1)]);
  nan = __builtin_amdgcn_ballot_w64(wnan[lane & (kSampleWaves - 1)]) != 0;
  u64 sum = 0;
  int count = 0;
  if (nan || !(fabsf(m) < INFINITY)) {
    count = nan ? -1 : 0;
  } else if constexpr (FILTERS) {
    const float c = fminf((float)per_z, 1e30f), top = bin_of(m, c);
    src.each([&](int, float v, bool) {
      const float b = bin_of(v, c);
      const int below = bins_below(top, b);
      if (below < kBins - 1) atomicAdd(&spread[below], spread_of(v, b, per_z));
      else count += v > -INFINITY;
    });
    count = (int)wave_sum((float)count);   // (whole numbers below 2^24)
    if (lane == 0) wcnt[wave] = count;
    __syncthreads();
    count = 0;
#pragma unroll
    for (int w = 0; w < kSampleWaves; ++w) count += wcnt[w];
    if (fabsf(top) > 0x1p20f) count = -2;
    if (threadIdx.x < kBins) spreads[out][threadIdx.x] = spread[threadIdx.x];
  } else {
    const SampleRow row = {(double)m, scale};
    src.each([&](int, float v, bool) { sum += row.weight(v); count += v > -INFINITY; });
    sum = wave_sum_u64(sum);
    count = (int)wave_sum((float)count);
    if (lane == 0) { wsum[wave] = sum; wcnt[wave] = count; }
    __syncthreads();
    sum = 0;
    count = 0;
#pragma unroll
    for (int w = 0; w < kSampleWaves; ++w) { sum += wsum[w]; count += wcnt[w]; }
  }
  if (threadIdx.x == 0) sums[out] = PartSum{m, count, sum};
}

// Maximum of a row from its parts (a lane each); 0 as it should be, -1: none, or a NaN, -2: too large for bins.
__device__ __forceinline__ int join_parts(const PartSum* sums, int parts, float& m, PartSum& mine) {
  const int lane = threadIdx.x & 63;
  static_assert(kPartsMax <= 64, "a lane a part");
  mine = sums[min(lane, parts - 1)];
  m = wave_max_dpp(mine.m);
  if (__builtin_amdgcn_ballot_w64(mine.count == -1) || !(fabsf(m) < INFINITY)) return -1;
  return __builtin_amdgcn_ballot_w64(mine.count == -2) ? -2 : 0;
}

// What is known of a row once its bins are: the cut lies in bins lo .. hi, all above is kept and all below is not.  LISTED: bins 0 .. hi hold up to
// kList tokens, and these are listed; CUT: the tokens of bins lo .. hi are; WHOLE: neither will do.
enum { PLAN_NONE = 0, PLAN_LISTED = 1, PLAN_CUT = 2, PLAN_WHOLE = 3 };
struct Plan {
  float m;
  int mode, listed, by_k, by_p;   // by_k, by_p: top-k, top-p cut within the bins
  int fixed;                      // how many are kept, if that is known (else 0)
  uint32_t above_cnt;
  u64 all, above_mass;
  u64 above[kPartsMax];           // of above_mass, in each part
};

// Finds the bins of the cut and lists their tokens in the order of the ids.  One block a part; each of a row's blocks finds the same bins.
template <typename T, int NE>
__global__ __launch_bounds__(kSampleThreads) void sample_list_kernel(const T* __restrict__ logits, int V, size_t ld, SampleArgs a,
                                                                     const PartSum* __restrict__ sums, const Spread* __restrict__ spreads,
                                                                     Plan* __restrict__ plans, int2* __restrict__ lists) {
  __shared__ Scratch x;
  __shared__ u64 frac[kBins];
  __shared__ uint32_t cnt[kBins];
  __shared__ double unit[kBins];
  __shared__ int below[64], far[64];   // a part's bins lie so far below the row's; logits in its last
  __shared__ int bin_k, bin_p, at_hi_cnt, at_lo_cnt;
  __shared__ u64 at_lo_mass, above_s[kPartsMax];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int part = blockIdx.x, parts = gridDim.x, r = blockIdx.y, lo_id = part * (kSampleThreads * NE);
  InRegisters<NE> src;
  src.fetch(logits + (size_t)r * ld + lo_id, min(V - lo_id, kSampleThreads * NE));
  Plan& plan = plans[r];
  spreads += (size_t)r * parts;
  float m;
  PartSum mine;
  const int state = join_parts(sums + (size_t)r * parts, parts, m, mine);
  if (state) {
    if (part == 0 && tid == 0) { plan.m = m; plan.mode = state == -1 ? PLAN_NONE : PLAN_WHOLE; }
    return;
  }
  const float c = fminf((float)a.per_z, 1e30f), top = bin_of(m, c);
  if (tid < kBins) { frac[tid] = 0; cnt[tid] = 0; unit[tid] = tid < kBins - 1 ? bin_unit(m, top, tid, a.per_z) : 0.0; }
  if (tid < kPartsMax) above_s[tid] = 0;
  if (tid < 64) {
    below[tid] = tid < parts && mine.m > -INFINITY ? bins_below(top, bin_of(mine.m, c)) : -1;   // (-1: it has written none)
    far[tid] = tid < parts ? mine.count : 0;
  }
  if (tid == 0) bin_k = bin_p = kBins;
  __syncthreads();
  auto sum_of = [&](int p, int b) { return below[p] >= 0 ? spreads[p][b] : 0ull; };
  auto row_bin = [&](int p, int b) { return min(b + below[p], kBins - 1); };
  constexpr u64 kFrac = (1ull << 48) - 1;
  {
    const int b = tid % kBins;   // two parts at a time, a thread a bin of each
    for (int p0 = tid / kBins; p0 < parts; p0 += 8) {
      u64 s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = p0 + 2 * i < parts ? sum_of(p0 + 2 * i, b) : 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (s[i]) {
          const int to = row_bin(p0 + 2 * i, b);
          atomicAdd(&cnt[to], (uint32_t)(s[i] >> 48));
          atomicAdd(&frac[to], s[i] & kFrac);
        }
    }
    if (tid < parts && far[tid] > 0) atomicAdd(&cnt[kBins - 1], (uint32_t)far[tid]);
  }
  __syncthreads();
  // a bin a thread, the largest logits first
  const uint32_t n = tid < kBins ? cnt[tid] : 0;
  const u64 s = tid < kBins ? bin_mass(n, frac[tid], unit[tid]) : 0;
  u64 cb = wave_before_u64(n), mb = wave_before_u64(s);
  if (lane == 63) { x.wcnt[wave] = (uint32_t)cb + n; x.wsum[wave] = mb + s; }
  __syncthreads();
  u64 all = 0, finite = 0;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) {
    if (w < wave) { cb += x.wcnt[w]; mb += x.wsum[w]; }
    finite += x.wcnt[w];
    all += x.wsum[w];
  }
  bool by_k = a.top_k > 0 && (u64)a.top_k < finite;
  if (by_k && cb < (u64)a.top_k && (u64)a.top_k <= cb + n) bin_k = tid;
  __syncthreads();
  // Top-k that ends among tokens of no weight takes nothing from the others: all that it says is how many are kept, if nothing else does.
  const int fixed = by_k && bin_k == kBins - 1 && a.top_p >= 1.0 && a.min_weight == 0 ? a.top_k : 0;
  const int k_at = by_k && bin_k < kBins - 1 ? bin_k : kBins;
  by_k = k_at < kBins;
  const bool by_p = a.top_p < 1.0;
  const u64 want = by_p ? mass_wanted(a.top_p, all) : 0;
  if (by_p && !by_k && mb < want && want <= mb + s) bin_p = tid;
  __syncthreads();
  // kBins: no cut.  (The bin of min_p's border is known up to the rounding of its logarithm.  Where top-p goes by the sum of the top-k, these
  // have to be there.)
  int lo = min(k_at, bin_p), hi = lo;
  if (a.min_weight > 0 && !(by_k && by_p)) {
    const double border = log2((double)a.min_weight * 0x1p-46) / a.scale;   // (z of the border less the maximum: <= 0)
    const int bm = (int)fmax(fmin((double)top - floor(((double)m + border) * a.per_z), (double)kBins), 0.0);
    lo = min(lo, max(bm - 1, 0));
    hi = min(hi, bm + 1);
  }
  if (lo < kBins) hi = min(hi, kBins - 1);
  if (tid == 0) { at_hi_cnt = (int)finite; at_lo_cnt = (int)finite; at_lo_mass = all; }
  __syncthreads();
  if (tid == lo) { at_lo_cnt = (int)cb; at_lo_mass = mb; }
  if (tid == hi) at_hi_cnt = (int)cb + (int)n;
  __syncthreads();
  int mode = PLAN_WHOLE;
  if (lo < kBins && at_hi_cnt <= kList) mode = PLAN_LISTED;
  else if (!(by_k && by_p) && at_hi_cnt - at_lo_cnt <= kList) mode = PLAN_CUT;
  const int from = mode == PLAN_LISTED ? 0 : lo;
  if (mode != PLAN_WHOLE && lo < kBins) {
    uint32_t have = 0;
    u64 has[NE], sum = 0;
    int e = 0;
    src.each([&](int, float v, bool) {
      const int b = v > -INFINITY ? bins_below(top, bin_of(v, c)) : -1;
      has[e] = __builtin_amdgcn_ballot_w64(b >= from && b <= hi);
      have += (uint32_t)__builtin_popcountll(has[e++]);
    });
    // those of the parts before this one
    for (int i = tid; i < part * kBins; i += kSampleThreads) {
      const u64 v = sum_of(i / kBins, i % kBins);
      const int to = row_bin(i / kBins, i % kBins);
      sum += to >= from && to <= hi ? v >> 48 : 0;
    }
    if (hi == kBins - 1 && tid < part) sum += far[tid];
    const uint32_t before = (uint32_t)block_sum_u64(sum, x);
    __syncthreads();
    if (lane == 0) x.wcnt[wave] = have;
    __syncthreads();
    uint32_t at = before;
    for (int w = 0; w < wave; ++w) at += x.wcnt[w];
    int2* list = lists + (size_t)r * kList;
    e = 0;
    src.each([&](int place, float v, bool) {
      const u64 h = has[e++];
      const uint32_t to = at + (uint32_t)__builtin_popcountll(h & ((1ull << lane) - 1));
      if ((h >> lane & 1) && to < (uint32_t)kList) list[to] = make_int2(__float_as_int(v), lo_id + place);
      at += (uint32_t)__builtin_popcountll(h);
    });
  }
  if (part == 0) {
    if (mode == PLAN_CUT) {
      for (int i = tid; i < parts * kBins; i += kSampleThreads) {
        const int p = i / kBins, to = row_bin(p, i % kBins);
        const u64 v = to < lo && to < kBins - 1 ? sum_of(p, i % kBins) : 0;
        if (v) atomicAdd(&above_s[p], bin_mass(v >> 48, v & kFrac, unit[to]));
      }
      __syncthreads();
      if (tid < parts) plan.above[tid] = above_s[tid];
    }
    if (tid == 0) {
      plan.m = m;
      plan.mode = mode;
      plan.listed = mode == PLAN_LISTED ? at_hi_cnt : at_hi_cnt - at_lo_cnt;
      plan.by_k = by_k && k_at <= hi;
      plan.fixed = fixed;
      plan.by_p = by_p && (by_k || bin_p <= hi);
      plan.above_cnt = mode == PLAN_LISTED ? 0 : (uint32_t)at_lo_cnt;
      plan.above_mass = mode == PLAN_LISTED ? 0 : at_lo_mass;
      plan.all = all;
    }
  }
}

// The token of a row whose parts are known.  One block a row.
template <typename T, bool FILTERS>
__global__ __launch_bounds__(kSampleThreads) void sample_draw_kernel(const T* __restrict__ logits, int V, size_t ld, int parts, int part_size,
                                                                     const float* __restrict__ uniforms, SampleArgs a,
                                                                     const PartSum* __restrict__ sums, const Plan* __restrict__ plans,
                                                                     const int2* __restrict__ lists, int* __restrict__ tokens,
                                                                     float4* __restrict__ stats) {
  __shared__ Scratch x;
  __shared__ u64 part_kept[kPartsMax];
  const int r = blockIdx.x, tid = threadIdx.x;
  const float u = uniforms[r];
  const T* z = logits + (size_t)r * ld;
  Cut cut;
  u64 all = 0;
  uint32_t count = 0;
  float m;
  if constexpr (FILTERS) {
    const Plan& plan = plans[r];
    const int mode = plan.mode;
    if (mode == PLAN_NONE) { no_token(tokens, stats, r); return; }
    m = plan.m;
    const SampleRow row = {(double)m, a.scale};
    if (mode == PLAN_WHOLE) {
      InMemory<T> src;
      src.fetch(z, V);
      sample_whole(src, row, a, u, r, x, tokens, stats);
      return;
    }
    all = plan.all;
    const int2* list = lists + (size_t)r * kList;
    InRegisters<kList / kSampleThreads> src;
    src.n = plan.listed;
    src.first = (tid >> 6) * kList / kSampleWaves + (tid & 63);
#pragma unroll
    for (int e = 0; e < kList / kSampleThreads; ++e) {
      const int at = src.first + e * 64;
      src.v[e] = at < src.n ? __int_as_float(list[at].x) : -INFINITY;
    }
    const u64 listed = sum_weights(src, row, x);   // (may differ from the bins' by roundings)
    u64 of_k = mode == PLAN_LISTED ? all : 0;
    for (int by_mass = 0; by_mass < 2; ++by_mass) {
      u64 want;
      if (by_mass) {
        if (!plan.by_p) continue;
        want = min(mode == PLAN_LISTED ? mass_wanted(a.top_p, of_k) : mass_wanted(a.top_p, all) - plan.above_mass, listed);
      } else {
        if (!plan.by_k) continue;
        want = a.top_k - (int)plan.above_cnt;
        if (want >= (u64)src.n) { of_k = listed; continue; }
      }
      of_k = select_cut(src, row, by_mass, want, cut, x);
    }
    if (mode == PLAN_LISTED) {
      u64 kept;
      int place;
      float v;
      if (draw_place(src, row, cut, 0, a.min_weight, x, kept, count, [&](u64 k) { return draw_at(u, k); }, place, v))
        put_token(tokens, stats, r, list[place].y, v, row, kept, count, all);
      return;
    }
    // what is kept of each part: all above the bins, and some of the list
    if (tid < kPartsMax) part_kept[tid] = tid < parts ? plan.above[tid] : 0;
    __syncthreads();
    u64 n = 0;
    src.each([&](int at, float v, bool) {
      const u64 w = row.weight(v);
      if (v > -INFINITY && w >= a.min_weight && cut.keeps(key_of(v), at)) {
        ++n;
        atomicAdd(&part_kept[list[at].y / part_size], w);
      }
    });
    count = plan.above_cnt + (uint32_t)block_sum_u64(n, x);
    if (plan.fixed) count = plan.fixed;
    if (cut.last != INT_MAX) cut.last = list[cut.last].y;
  } else {
    PartSum mine;
    if (join_parts(sums + (size_t)r * parts, parts, m, mine)) { no_token(tokens, stats, r); return; }
    const bool some = (tid & 63) < parts && mine.m > -INFINITY;
    if (tid < kPartsMax)   // (the part's sum, seen from the row's maximum)
      part_kept[tid] = some ? (u64)((double)mine.sum * (exp2_times_2to46(((double)mine.m - (double)m) * a.scale) * 0x1p-46) + 0.5) : 0;
    count = (uint32_t)wave_sum_u64(some ? (u64)mine.count : 0);
  }
  __syncthreads();
  const SampleRow row = {(double)m, a.scale};
  const u64 kept = wave_sum_u64((tid & 63) < parts ? part_kept[tid & 63] : 0);
  if constexpr (!FILTERS) all = kept;
  // The part of the token, then the token.  The part's own weights, seen from the row's maximum, may come to a little less than its sum did, to
  // nothing where each rounds to 0: then the next part's first.
  const u64 want = draw_at(u, kept);
  u64 base = 0;
  int p = 0;
  while (p + 1 < parts && base + part_kept[p] < want) base += part_kept[p++];
  for (int tried = 0; tried <= parts; ++tried, p = p + 1 < parts ? p + 1 : 0) {
    const int lo = p * part_size;
    InMemory<T> src;
    src.fetch(z + lo, min(V - lo, part_size));
    u64 here;
    uint32_t n;
    int place;
    float v;
    const bool mine = draw_place(src, row, cut, lo, a.min_weight, x, here, n,
                                 [&](u64 k) { return tried ? min((u64)1, k) : min(want - base, k); }, place, v);
    if (mine) put_token(tokens, stats, r, lo + place, v, row, kept, count, all);
    if (here > 0) break;   // (the same for all threads)
  }
}

// ---- launchers ------------------------------------------------------------------------------------
struct SamplePlanSizes { int ne, parts; };
// Logits to a thread: the fewest with which a batch of rows makes about two blocks of 1024 threads for each compute unit.
static SamplePlanSizes sample_sizes(int rows, int V) {
  for (const int ne : {4, 8, 16, 32}) {
    const int parts = (V + kSampleThreads * ne - 1) / (kSampleThreads * ne);
    if (ne == 32 || (long)rows * parts <= 512) return {ne, parts};
  }
  return {32, 1};
}
constexpr int kSampleSmall = 16384;   // logits of a row that one block holds in registers
struct SampleBytes { size_t sums, spreads, plans, lists, all; };
static SampleBytes sample_bytes(int rows, int V) {
  SampleBytes b = {};
  if (rows <= 0 || V <= kSampleSmall) { b.all = 256; return b; }
  if (rows > kSampleBatch) rows = kSampleBatch;
  size_t most = 0;   // (fewer rows may have more parts between them)
  for (const int ne : {4, 8, 16, 32}) {
    const size_t parts = (V + kSampleThreads * ne - 1) / (kSampleThreads * ne);
    const size_t n = parts * (ne == 32 ? rows : rows * parts <= 512 ? rows : 512 / parts);
    if (n > most) most = n;
  }
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  b.sums = up(most * sizeof(PartSum));
  b.spreads = up(most * sizeof(Spread));
  b.plans = up(rows * sizeof(Plan));
  b.lists = up((size_t)rows * kList * sizeof(int2));
  b.all = b.sums + b.spreads + b.plans + b.lists;
  return b;
}
size_t sample_workspace(int rows, int V) { return sample_bytes(rows, V).all; }

template <typename T, int NE>
static void launch_sample_ne(const T* logits, int rows, int parts, int V, size_t ld, const float* uniforms, const SampleArgs& a, int* tokens,
                             float4* stats, char* ws, const SampleBytes& b, hipStream_t s) {
  PartSum* sums = (PartSum*)ws;
  Spread* spreads = (Spread*)(ws + b.sums);
  Plan* plans = (Plan*)(ws + b.sums + b.spreads);
  int2* lists = (int2*)(ws + b.sums + b.spreads + b.plans);
  const dim3 grid(parts, rows);
  if (a.top_k > 0 || a.top_p < 1.0 || a.min_weight > 0) {
    sample_parts_kernel<T, NE, true><<<grid, kSampleThreads, 0, s>>>(logits, V, ld, a.scale, a.per_z, sums, spreads);
    sample_list_kernel<T, NE><<<grid, kSampleThreads, 0, s>>>(logits, V, ld, a, sums, spreads, plans, lists);
    sample_draw_kernel<T, true><<<rows, kSampleThreads, 0, s>>>(logits, V, ld, parts, kSampleThreads * NE, uniforms, a, sums, plans, lists, tokens, stats);
  } else {
    sample_parts_kernel<T, NE, false><<<grid, kSampleThreads, 0, s>>>(logits, V, ld, a.scale, a.per_z, sums, spreads);
    sample_draw_kernel<T, false><<<rows, kSampleThreads, 0, s>>>(logits, V, ld, parts, kSampleThreads * NE, uniforms, a, sums, plans, lists, tokens, stats);
  }
}

template <typename T>
static void launch_sample_t(const T* logits, int rows, int V, size_t ld, const float* uniforms, const SampleArgs& a, int* tokens,
                            float4* stats, void* workspace, hipStream_t s) {
  if (V <= kSampleSmall) {
    if (V <= 1024) sample_small_kernel<T, 1><<<rows, kSampleThreads, 0, s>>>(logits, V, ld, uniforms, a, tokens, stats);
    else if (V <= 4096) sample_small_kernel<T, 4><<<rows, kSampleThreads, 0, s>>>(logits, V, ld, uniforms, a, tokens, stats);
    else sample_small_kernel<T, 16><<<rows, kSampleThreads, 0, s>>>(logits, V, ld, uniforms, a, tokens, stats);
    return;
  }
  const SampleBytes b = sample_bytes(rows, V);
  for (int r = 0; r < rows; r += kSampleBatch) {
    const int n = rows - r < kSampleBatch ? rows - r : kSampleBatch;
    const SamplePlanSizes w = sample_sizes(n, V);
    const T* z = logits + (size_t)r * ld;
    switch (w.ne) {
      case 4: launch_sample_ne<T, 4>(z, n, w.parts, V, ld, uniforms + r, a, tokens + r, stats + r, (char*)workspace, b, s); break;
      case 8: launch_sample_ne<T, 8>(z, n, w.parts, V, ld, uniforms + r, a, tokens + r, stats + r, (char*)workspace, b, s); break;
      case 16: launch_sample_ne<T, 16>(z, n, w.parts, V, ld, uniforms + r, a, tokens + r, stats + r, (char*)workspace, b, s); break;
      default: launch_sample_ne<T, 32>(z, n, w.parts, V, ld, uniforms + r, a, tokens + r, stats + r, (char*)workspace, b, s); break;
    }
  }
}
void launch_sample_rows(const void* logits, bool bf16, int rows, int V, size_t ld, const float* uniforms, const SampleArgs& a,
                        int* tokens, float4* stats, void* workspace, hipStream_t s) {
  if (bf16) launch_sample_t((const bf16_t*)logits, rows, V, ld, uniforms, a, tokens, stats, workspace, s);
  else launch_sample_t((const float*)logits, rows, V, ld, uniforms, a, tokens, stats, workspace, s);
}

}  // namespace ec
