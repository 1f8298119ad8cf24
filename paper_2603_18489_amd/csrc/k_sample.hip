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
#include <stddef.h>

#include "ec_internal.h"
#include "k_exp.h"

namespace ec {

typedef unsigned long long u64;

constexpr int kSampleThreads = 512;
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
__device__ __forceinline__ uint32_t wave_min_u32(uint32_t v) {   // (as wave_min_dpp, of unsigned numbers)
  return (uint32_t)wave_min_dpp((int)(v ^ 0x80000000u)) ^ 0x80000000u;
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

__device__ __forceinline__ uint32_t wave_upto_u32(uint32_t s) {   // (this lane's too)
  s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x111, 0xf, 0xf, false);
  s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x112, 0xf, 0xf, false);
  s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x114, 0xf, 0xf, false);
  s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x118, 0xf, 0xf, false);
  s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x142, 0xa, 0xf, false);
  s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x143, 0xc, 0xf, false);
  return s;
}
__device__ __forceinline__ int lanes_before(u64 mask) {   // of those in the mask
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

struct SampleRow {
  double m, scale;   // maximum; log2(e) / T
  __device__ __forceinline__ u64 weight(float z) const { return exp2_fixed46(((double)z - m) * scale); }
};

// What a block of 512 threads works through, in the order of the ids: each wave has a range of its own, 64 neighbours at a time.
// each(f): f(place, logit, there) for the lane's elements; a place that is not there has a logit of -inf.
template <int NE> struct InRegisters {
  float v[NE];
  int first, n;   // the lane's first place; places in all
  template <typename T> __device__ __forceinline__ void fetch(const T* z, int count) {
    n = count;
    first = (threadIdx.x >> 6) * (64 * NE) + (threadIdx.x & 63);
    if (n == kSampleThreads * NE) {
#pragma unroll
      for (int e = 0; e < NE; ++e) v[e] = load_f32(z + first + e * 64);
      return;
    }
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

struct InList {   // (logit, id) in LDS; places are those in the list
  const int2* list;
  int first, end, n;
  __device__ __forceinline__ void fetch(const int2* from, int count) {
    list = from; n = count;
    const int per = ((n + kSampleWaves - 1) / kSampleWaves + 63) / 64 * 64, lo = min((int)(threadIdx.x >> 6) * per, n);
    first = lo + (threadIdx.x & 63);
    end = min(lo + per, n);
  }
  template <typename F> __device__ __forceinline__ void each(F f) const {
    const int rounds = (end - (first - (int)(threadIdx.x & 63)) + 63) / 64;
    for (int e = 0; e < rounds; ++e) {
      const int at = first + e * 64;
      f(at, at < end ? __int_as_float(list[at].x) : -INFINITY, at < end);
    }
  }
};

// LDS of a block that looks for the cut
constexpr int kDigits = 1024;
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
  u64 total = above_mass;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) {
    const u64 s = x.wsum[w];
    cx += w < wave ? x.wcnt[w] : 0u;
    mx += w < wave ? s : 0ull;
    total += s;
  }
  if (by_mass) want = min(want, total);   // (sums by other bins and by tokens differ by roundings)
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

// The same among up to 64 tokens that x.few has.  Every wave ranks them, a lane each, by key, then place.  Returns what is kept.
__device__ __forceinline__ u64 rank_few(uint32_t n, uint32_t above_cnt, u64 above_mass, bool by_mass, u64 want, Cut& cut, Scratch& x) {
  __syncthreads();
  const int lane = threadIdx.x & 63, mine = lane < (int)n ? lane : 0;
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
  // (sums by bins and by tokens differ by roundings: a wanted weight past the last token's means the last)
  const u64 last = __builtin_amdgcn_ballot_w64(lane < (int)n && rank + 1 == above_cnt + n);
  const int l = __builtin_ctzll(is ? is : last);
  cut.key = (uint32_t)__builtin_amdgcn_readlane((int)key, l);
  cut.last = __builtin_amdgcn_readlane(place, l);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(upto >> 32), l), lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)upto, l);
  return (u64)hi << 32 | lo;
}

// The cut among the tokens for which in(z) holds; above_cnt, above_mass: of those ahead of them all.  Their keys' range in kDigits equal
// pieces, then the piece of the cut, until a piece is one key.  Returns what is kept.
template <typename S, typename P>
__device__ u64 select_digits(const S& src, const SampleRow& row, bool by_mass, u64 want, uint32_t above_cnt, u64 above_mass, P in_set, Cut& cut,
                             Scratch& x) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t high = 0, low = ~0u;
  src.each([&](int, float v, bool) {
    if (v > -INFINITY && in_set(v)) {
      const uint32_t k = key_of(v);
      high = max(high, k);
      low = min(low, k);
    }
  });
  high = ~(uint32_t)wave_min_u32(~high);
  low = wave_min_u32(low);
  __syncthreads();
  if (lane == 0) x.wsum[wave] = (u64)high << 32 | low;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) { high = max(high, (uint32_t)(x.wsum[w] >> 32)); low = min(low, (uint32_t)x.wsum[w]); }
  uint32_t span = high - low;   // of the keys from `high` down
  for (;;) {
    const int shift = max(0, 22 - __builtin_clz(span | 1));   // (span >> shift < kDigits)
    clear_bins(x);
    src.each([&](int, float v, bool) {
      const uint32_t k = key_of(v);
      if (v > -INFINITY && in_set(v) && k <= high && high - k <= span) {
        const uint32_t b = (high - k) >> shift;
        atomicAdd(&x.cnt[b], 1u);
        atomicAdd(&x.mass[b], row.weight(v));
      }
    });
    __syncthreads();
    find_bin(by_mass, want, above_cnt, above_mass, x);
    high -= x.found_bin << shift;
    above_cnt = x.found_above_cnt;
    above_mass = x.found_above_mass;
    if (shift == 0) break;
    span = (1u << shift) - 1;
  }
  const uint32_t prefix = high;
  const u64 each = x.found_mass / x.found_cnt;   // (equal logits, equal weights)
  const uint32_t ties = by_mass ? min((uint32_t)((want - above_mass + each - 1) / each), x.found_cnt) : (uint32_t)want - above_cnt;
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

// The cut after which `want` tokens are kept (by_mass: after which what is kept first weighs `want` or more); there are as many.  Returns what is
// kept.  First bins of equal width in z, 32 T in all; if up to 64 tokens share the one of the cut, a wave ranks them.
template <typename S>
__device__ u64 select_cut(const S& src, const SampleRow& row, bool by_mass, u64 want, Cut& cut, Scratch& x) {
  const int lane = threadIdx.x & 63;
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
    return rank_few(n, above_cnt, above_mass, by_mass, want, cut, x);
  }
  return select_digits(src, row, by_mass, want, above_cnt, above_mass, [&](float v) { return bin(v) == at; }, cut, x);
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

// The place of the token: the first whose running sum of kept weights is `want` or more.  kept, count: of these tokens; `wanted` is called by
// every thread with them and says what is wanted.  Returns true to one lane, whose `close` says that the token begins or ends within `near` of it.
template <typename S, typename W>
__device__ __forceinline__ bool draw_place(const S& src, const SampleRow& row, const Cut& cut, int shift, double least, Scratch& x,
                                           u64& kept, uint32_t& count, W wanted, int& place, float& logit, u64 near, bool& close) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 part = 0;
  uint32_t n = 0;
  auto weight = [&](int at, float v) {
    const u64 w = row.weight(v);
    const bool keep = v > -INFINITY && v >= least && cut.keeps(key_of(v), at + shift);
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
        if (lane == __builtin_ctzll(past)) { found = true; place = at; logit = v; close = want + w - upto < near || upto - want < near; }
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
  bool close;
  if (draw_place(src, row, cut, 0, row.m + a.min_z, x, kept, n, [&](u64 k) { return draw_at(u, k); }, place, z, 0, close))
    put_token(tokens, stats, r, place, z, row, kept, n, all);
}

// A row of up to 512 NE logits: one block, which reads it once and keeps it in registers.  A row of 4096, us by trace: 6.2 without filters (launch,
// load, maximum, sum, draw), 8.9 with top-k, 9.6 with top-p, 11.1 with both.  So each search for a cut takes 3: the weights of all logits once
// more and their LDS atomics, some barriers, and a wave that ranks what shares the cut's bin.  Weights are not kept: each step that wants one
// computes it again, five times and more a logit with both.
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

// ---- longer rows: parts of 4096 or 8192 logits to a block ---------------------------------------------
// One pass in which each block needs nothing of the others, then a block a row that joins what they found.  A part's maximum and, without
// filters, its weights' sum.  With filters, how its weights spread over kBins bins of T / 16 in z, counted down from its largest logit; the
// last one is all that lies about 32 T (at least 510 / 16 T) and more below it, which is taken to weigh nothing (it is up to 1.02 * 2^-46 of the
// maximum).  Bins begin at multiples of T / 16, so that a row's parts are put together by moving them by whole bins.  A weight of bin B is
// e^(B / 16) e^(rho / 16) with rho = z 16 / T - B in [0, 1] but for roundings, and what is added for it one number: 2^48 (a count) plus
// (e^(rho / 16) - 0.99) 2^36, whose sums over the 8192 logits of a part stay below 2^48.
// 544 rows of 126464 bf16 logits: 89 us, 1.5 TB/s; 36 of these are the loads and the maximum, the rest instructions: the 64-bit polynomial
// (26), bins, whose LDS atomics hide behind it, and the list below (23, for which the draw takes 50 us instead of 91; found by every wave for
// itself and with the logits in it: 28).  32 rows of float32 without filters: 8.6 us, about a launch and the latency of what a block does.
// (32 logits a thread, without the list: 75 us, 16: 68.)
constexpr int kBins = 512, kList = 5632, kPartsMax = 40, kSampleBatch = 1024;
constexpr int kChunk = 1024, kChunksMax = 192;   // logits that a wave goes through at a time; of the longest row
struct PartSum {
  float m;
  int count;   // -1: a NaN.  With filters: the logits of the last bin, -2 where logits are too large for the bins (2^16 T).  Without: all above -inf
  u64 sum;     // (without filters)
  float of_wave[kSampleWaves];   // the largest of each 64 NE logits in a row, NaN aside
  int listed, depth;             // with filters: how many tokens are listed, all of the first `depth` bins
};
typedef u64 Spread[kBins];
// With filters a part lists the tokens of its first bins, as many whole bins as have up to one in 32 of its logits, in the order of the ids: a
// cut that lies there in all parts needs the row's logits no more.
constexpr int kOfListed = 32, kListedMost = kSampleThreads * 16 / kOfListed;

// number of the bin of a logit, counted up in z; whole, and monotonous whatever z
__device__ __forceinline__ float bin_of(float z, float per_z) { return floorf(fminf(fmaxf(z * per_z, -1e30f), 1e30f)); }
__device__ __forceinline__ int bins_below(float top, float b) { return (int)fminf(top - b, (float)(kBins - 1)); }
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key); }
// The least key of the logits whose bin is at most b below the bin `top` (bins go with the logits' order): a few keys around where it should be,
// one a lane, or bisected.  c: 16 / T.
__device__ __forceinline__ uint32_t first_key(float top, float c, int b) {
  auto in = [&](uint32_t k) { return bins_below(top, bin_of(logit_of(k), c)) <= b; };
  const uint32_t guess = min(max(key_of((top - (float)b) / c), 0x00800020u), 0xff7fffdfu) - 32;
  const u64 yes = __builtin_amdgcn_ballot_w64(in(guess + (threadIdx.x & 63)));
  if (yes && !(yes & 1)) return guess + (uint32_t)__builtin_ctzll(yes);
  uint32_t i = 0x00800000u, j = 0xff7fffffu;   // (keys of the lowest and the highest finite value)
  while (i < j) {
    const uint32_t mid = i + (j - i) / 2;
    if (in(mid)) j = mid; else i = mid + 1;
  }
  return i;
}
__device__ __forceinline__ u64 spread_of(float z, float b, double per_z) {
  const double rho = fma((double)z, per_z, -(double)b);
  // e^(rho / 16) - 0.99, degree 5 through the Chebyshev nodes of [-1/16, 17/16]: off by 8.5e-14 there.  bin_of rounds 16 / T and its product with
  // z to float32, which moves a border by up to 1/8 at the largest bins, 2^20: off by 7.1e-13 in [-1/8, 9/8].
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
                                                                      Spread* __restrict__ spreads, int2* __restrict__ candidates) {
  __shared__ u64 spread[kBins], wsum[kSampleWaves];
  __shared__ uint16_t few[kSampleThreads * NE];   // (as far as it is used)
  __shared__ float list_from;
  __shared__ int list_depth;
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
  int count = 0, listed = 0, depth = 0;
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
    // how many bins are listed, and from which logit on: found by one wave for all
    constexpr uint32_t MOST = kSampleThreads * NE / kOfListed;
    if (wave == kSampleWaves - 1) {
      uint32_t before = 0;
      for (int b = 0; b < kBins; b += 64) {
        const uint32_t upto = before + wave_upto_u32((uint32_t)(spread[b + lane] >> 48));
        const u64 fits = __builtin_amdgcn_ballot_w64(upto <= MOST);
        depth += __builtin_popcountll(fits);
        if (~fits) break;
        before = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
      }
      const float from = depth ? logit_of(first_key(top, c, min(depth, kBins - 1) - 1)) : INFINITY;
      if (lane == 0) { list_from = from; list_depth = depth; }
    }
    __syncthreads();
    // each wave's tokens to where those of the waves before it end
    const float from = list_from;
    depth = list_depth;
    u64 has[NE];
    int mine = 0;
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      has[e] = __builtin_amdgcn_ballot_w64(src.v[e] >= from);
      mine += __builtin_popcountll(has[e]);
    }
    if (lane == 0) wcnt[wave] = mine;
    __syncthreads();
    int to = 0;
#pragma unroll
    for (int w = 0; w < kSampleWaves; ++w) { to += w < wave ? wcnt[w] : 0; listed += wcnt[w]; }
    listed = min(listed, (int)MOST);
#pragma unroll
    for (int e = 0; e < NE; ++e)
      if (has[e]) {
        if (src.v[e] >= from) few[to + lanes_before(has[e])] = (uint16_t)(src.first + e * 64);
        to += __builtin_popcountll(has[e]);
      }
    __syncthreads();
    if ((int)threadIdx.x < listed) {
      const int place = few[threadIdx.x];
      candidates[(size_t)out * MOST + threadIdx.x] = make_int2(__float_as_int(load_f32(logits + (size_t)r * ld + lo + place)), lo + place);
    }
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
  if (lane == 0) sums[out].of_wave[wave] = wmax[wave];
  if (threadIdx.x == 0) { sums[out].m = m; sums[out].count = count; sums[out].sum = sum; sums[out].listed = listed; sums[out].depth = depth; }
}

// Maximum of a row from its parts (a lane each); 0 as it should be, -1: none, or a NaN, -2: too large for bins.
struct PartHead { float m; int count; u64 sum; };   // (what every kernel wants of a PartSum)
__device__ __forceinline__ int join_parts(const PartSum* sums, int parts, float& m, PartHead& mine) {
  const int lane = threadIdx.x & 63;
  static_assert(kPartsMax <= 64, "a lane a part");
  mine = *(const PartHead*)&sums[min(lane, parts - 1)];
  m = wave_max_dpp(mine.m);
  if (__builtin_amdgcn_ballot_w64(mine.count == -1) || !(fabsf(m) < INFINITY)) return -1;
  return __builtin_amdgcn_ballot_w64(mine.count == -2) ? -2 : 0;
}

// LDS of a block that draws from a row whose parts are known, up to LIST tokens among which the cut is
template <int LIST> struct RowScratch {
  union {
    Scratch x;               // (of its arrays, mass is used only once these two are not)
    struct { u64 frac[kBins]; double unit[kBins]; } bins;
  };
  uint32_t cnt[kBins];
  int below[64], far[64];   // a part's bins lie so far below the row's (-1: it has none); logits in its last
  int bin_k, bin_p, redo;
  u64 cum_mass[kBins + 1], part_kept[64];   // cum: of the bins above
  uint32_t cum_cnt[kBins + 1];
  int chunk_cnt[kChunksMax], chunk_at[kChunksMax], chunk_id[kChunksMax], listed;
  int2 list[LIST];          // logit and id
};
static_assert(offsetof(Scratch, mass) == 0 && sizeof(Scratch::mass) >= kBins * 16, "frac and unit lie over mass");

// A sum of bins is off by up to 2^-36.5 of itself: in each of its logits, where 1 is the weight at the bin's lower end, by 2^-37 from rounding
// and 7.1e-13 from the polynomial, of 0.992 or more.  So a sum that is wanted and one that is compared with it are off by less than 2^-35 of
// the largest.  Where a border is as near (in rows of equal logits it may be met exactly: half of them kept, or u the share of the first
// ones), the block goes through the row, whose sums are exact.  34 rows of 152064 with top-p: 32.1 us as without the test.
constexpr int kNear = 35;

// Bins lo .. hi hold the cut: all above is kept and all below is not.  LISTED: the tokens of bins 0 .. hi are listed, up to LIST of them;
// CUT: those of lo .. hi; WHOLE: neither will do.
enum { PLAN_LISTED = 1, PLAN_CUT = 2, PLAN_WHOLE = 3 };

// Lists the tokens of bins `from` .. `hi` in the order of the ids.  A wave takes a chunk at a time, of those that reach so high; its
// tokens go to wherever the list has got to, and once all are there a chunk's are moved to behind those of the chunks before it.
template <typename T, int LIST>
__device__ __forceinline__ void list_bins(const T* z, int V, const PartSum* sums, int part_size, float c, float top, int from, int hi,
                                          RowScratch<LIST>& y) {
  constexpr int E = kChunk / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, chunks = (V + kChunk - 1) / kChunk;
  constexpr int CW = kChunksMax / 64;   // waves with a chunk a lane
  static_assert(kChunksMax % 64 == 0 && CW <= kSampleWaves, "a lane a chunk");
  // the lowest logit of bin hi, the highest of bin `from`
  uint32_t least = 0x00800000u, most = 0xff7fffffu;   // (keys of the lowest and the highest finite value)
  if (hi < kBins - 1) least = first_key(top, c, hi);
  if (from > 0) most = first_key(top, c, from - 1) - 1;
  const float vmin = logit_of(least), vmax = logit_of(most);
  // the chunks to go through, a lane each
  u64 n = 0;
  if (tid < chunks) {
    const int part = tid * kChunk / part_size, in = tid * kChunk - part * part_size, per = part_size / kSampleWaves;
    for (int w = in / per; w <= (in + kChunk - 1) / per; ++w) n |= sums[part].of_wave[w] >= vmin;
  }
  u64 before = 0;
  if (wave < CW) {
    before = wave_before_u64(n);
    if (lane == 63) y.x.wcnt[wave] = (uint32_t)(before + n);
  }
  __syncthreads();
  if (wave < CW) {
    for (int w = 0; w < wave; ++w) before += y.x.wcnt[w];
    if (n) y.chunk_id[before] = tid;
    if (tid < chunks) y.chunk_cnt[tid] = 0;
  }
  int active = 0;
#pragma unroll
  for (int w = 0; w < CW; ++w) active += (int)y.x.wcnt[w];
  __syncthreads();
  // (the last chunk begins early, so that all read whole chunks: rows here have more than one)
  auto begin = [&](int ch) { return min(ch * kChunk, V - kChunk); };
  auto fetch = [&](float (&v)[E], int i) {
    const T* from = z + begin(__builtin_amdgcn_readfirstlane(i < active ? y.chunk_id[i] : 0)) + lane;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = load_f32(from + e * 64);
  };
  auto put = [&](float (&v)[E], int i) {
    const int ch = __builtin_amdgcn_readfirstlane(y.chunk_id[i]), first = begin(ch);
    if (first < ch * kChunk)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = first + e * 64 + lane >= ch * kChunk ? v[e] : -INFINITY;
    u64 has[E];
    int n = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) has[e] = __builtin_amdgcn_ballot_w64(v[e] >= vmin);
    if (from)
#pragma unroll
      for (int e = 0; e < E; ++e) has[e] &= __builtin_amdgcn_ballot_w64(v[e] <= vmax);
#pragma unroll
    for (int e = 0; e < E; ++e) n += __builtin_popcountll(has[e]);
    if (!n) return;
    int at = 0;
    if (lane == 0) {
      at = atomicAdd(&y.listed, n);
      y.chunk_cnt[ch] = n;
      y.chunk_at[ch] = at;
    }
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (has[e]) {
        const int to = at + lanes_before(has[e]);
        if ((has[e] >> lane & 1) && to < LIST) y.list[to] = make_int2(__float_as_int(v[e]), first + e * 64 + lane);
        at += __builtin_popcountll(has[e]);
      }
  };
  float v[E], w[E];   // (one chunk on its way while the other is gone through)
  fetch(v, wave);
  for (int i = wave; i < active; i += 2 * kSampleWaves) {
    fetch(w, i + kSampleWaves);
    put(v, i);
    fetch(v, i + 2 * kSampleWaves);
    if (i + kSampleWaves < active) put(w, i + kSampleWaves);
  }
  __syncthreads();
  // where each chunk's tokens go
  if (wave < CW) {
    n = tid < chunks ? y.chunk_cnt[tid] : 0;
    before = wave_before_u64(n);
    if (lane == 63) y.x.wcnt[wave] = (uint32_t)(before + n);
  }
  int2 mine[LIST / kSampleThreads];
  static_assert(LIST % kSampleThreads == 0, "whole rounds");
  const int listed = min(y.listed, LIST);
#pragma unroll
  for (int e = 0; e < LIST / kSampleThreads; ++e)
    if (e * kSampleThreads < listed) mine[e] = y.list[min(e * kSampleThreads + tid, LIST - 1)];
  __syncthreads();
  if (tid < chunks && n) {
    for (int w = 0; w < wave; ++w) before += y.x.wcnt[w];
    y.chunk_cnt[tid] = (int)before - y.chunk_at[tid];   // how far they move
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < LIST / kSampleThreads; ++e) {
    const int at = e * kSampleThreads + tid;
    if (at < listed) y.list[at + y.chunk_cnt[mine[e].y / kChunk]] = mine[e];
  }
}

// The same from what the parts have listed, `most` places each: 64 at a time, a run of these to a wave.
template <int LIST>
__device__ __forceinline__ void list_candidates(const int2* candidates, int parts, int most, float c, float top, int from, int hi, RowScratch<LIST>& y) {
  constexpr int UNITS = kSampleThreads * 16 / kOfListed * (kPartsMax / 2) / 64, PER = (UNITS + kSampleWaves - 1) / kSampleWaves;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, each = most / 64, units = parts * each;   // (at most UNITS)
  const int per = (units + kSampleWaves - 1) / kSampleWaves;
  int2 v[PER];
  u64 has[PER];
  int n = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = candidates[(size_t)min(wave * per + i, units - 1) * 64 + lane];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int unit = min(wave * per + i, units - 1), part = unit / each;
    const int b = bins_below(top, bin_of(__int_as_float(v[i].x), c));
    has[i] = __builtin_amdgcn_ballot_w64(i < per && wave * per + i < units && (unit - part * each) * 64 + lane < y.chunk_at[part] && b >= from && b <= hi);
    n += __builtin_popcountll(has[i]);
  }
  if (lane == 0) y.x.wcnt[wave] = (uint32_t)n;
  __syncthreads();
  int to = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) { to += w < wave ? (int)y.x.wcnt[w] : 0; all += (int)y.x.wcnt[w]; }
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (has[i]) {
      const int at = to + lanes_before(has[i]);
      if ((has[i] >> lane & 1) && at < LIST) y.list[at] = v[i];
      to += __builtin_popcountll(has[i]);
    }
  if (threadIdx.x == 0) y.listed = min(all, LIST);
}

// The token of a row whose parts are known.  One block a row.  With filters, the parts' bins together say in which the cut lies; the tokens of
// these come from the parts' lists, or, where these are too short, from the row, and are then ranked.  Without, and where more is kept than can
// be listed, the parts' sums say in which part the token is, and only that is read.  34 rows of 152064 with top-p: 18 us, the chain from the bins to
// the token; 544 rows of 126464 bf16 with top-k, top-p and min-p: 51 us, two blocks to a compute unit and so two rounds.  Where all have to read
// their row again these take 91 us, 138 MB at 5.5 TB/s (three blocks with a list of half the length: 84 to 90 us, and spills; chunks of 512: 98).
// Where neither will do, the block goes through its row several times (sample_whole).  32 rows of 126464, us a call: top-p 0.9 at a spread of 2 66
// from bins and lists; by the row, min_p 0.05 at a spread of 1 and T 1.5 219, top-p 0.5 at T 2 420, top-k 10000 with top-p 510, and 375 where a part's
// largest logit is beyond 2^16 T (16384 neighbours at the type's lowest value, beside 63 with -inf there).
template <typename T, bool FILTERS, int LIST>
__global__ __launch_bounds__(kSampleThreads, FILTERS ? 4 : 1) void sample_draw_kernel(const T* __restrict__ logits, int V, size_t ld, int parts, int part_size,
                                                                     const float* __restrict__ uniforms, SampleArgs a,
                                                                     const PartSum* __restrict__ sums, const Spread* __restrict__ spreads,
                                                                     const int2* __restrict__ candidates, int* __restrict__ tokens, float4* __restrict__ stats) {
  extern __shared__ char lds_[];
  RowScratch<LIST>& y = *(RowScratch<LIST>*)lds_;
  Scratch& x = y.x;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float u = uniforms[r];
  const T* z = logits + (size_t)r * ld;
  spreads += (size_t)r * parts;
  sums += (size_t)r * parts;
  Cut cut;
  u64 all = 0;
  uint32_t count = 0;
  bool whole = false;   // the row is gone through by this block
  float m;
  PartHead mine;
  // (a thread a bin of each part; the first four asked for ahead of everything else)
  u64 s4[4];
  if constexpr (FILTERS) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s4[i] = spreads[min(i, parts - 1)][tid];
  }
  const int listed_of = FILTERS ? sums[min(lane, parts - 1)].listed : 0, depth_of = FILTERS ? sums[min(lane, parts - 1)].depth : 0;
  const int state = join_parts(sums, parts, m, mine);
  if (state == -1) { no_token(tokens, stats, r); return; }
  const SampleRow row = {(double)m, a.scale};
  if constexpr (FILTERS) {
    const float c = fminf((float)a.per_z, 1e30f), top = bin_of(m, c);
    int mode = PLAN_WHOLE, lo = 0, hi = 0, fixed = 0;
    bool by_k = false, by_p = a.top_p < 1.0;
    if (state == 0) {
      static_assert(kSampleThreads == kBins, "a thread a bin");
      y.bins.frac[tid] = 0;
      y.cnt[tid] = 0;
      y.bins.unit[tid] = tid < kBins - 1 ? bin_unit(m, top, tid, a.per_z) : 0.0;
      if (tid < 64) {
        y.below[tid] = tid < parts && mine.m > -INFINITY ? bins_below(top, bin_of(mine.m, c)) : -1;   // (-1: it has written none)
        y.far[tid] = tid < parts ? mine.count : 0;
        y.chunk_at[tid] = listed_of;
        y.part_kept[tid] = 0;
      }
      if (tid == 0) { y.bin_k = y.bin_p = kBins; y.listed = 0; y.redo = 0; }
      __syncthreads();
      auto row_bin = [&](int p, int b) { return min(b + y.below[p], kBins - 1); };
      constexpr u64 kFrac = (1ull << 48) - 1;
      for (int p0 = 0; p0 < parts; p0 += 4) {
        u64 next[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) next[i] = spreads[min(p0 + 4 + i, parts - 1)][tid];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = min(p0 + i, parts - 1);
          if (p0 + i < parts && y.below[p] >= 0 && s4[i]) {
            const int to = row_bin(p, tid);
            atomicAdd(&y.cnt[to], (uint32_t)(s4[i] >> 48));
            atomicAdd(&y.bins.frac[to], s4[i] & kFrac);
          }
          s4[i] = next[i];
        }
      }
      if (tid < parts && y.far[tid] > 0) atomicAdd(&y.cnt[kBins - 1], (uint32_t)y.far[tid]);
      __syncthreads();
      // a bin a thread, the largest logits first
      const uint32_t n = y.cnt[tid];
      const u64 s = bin_mass(n, y.bins.frac[tid], y.bins.unit[tid]);
      u64 cb = wave_before_u64(n), mb = wave_before_u64(s);
      if (lane == 63) { x.wcnt[wave] = (uint32_t)cb + n; x.wsum[wave] = mb + s; }
      __syncthreads();
      u64 finite = 0;
#pragma unroll
      for (int w = 0; w < kSampleWaves; ++w) {
        if (w < wave) { cb += x.wcnt[w]; mb += x.wsum[w]; }
        finite += x.wcnt[w];
        all += x.wsum[w];
      }
      by_k = a.top_k > 0 && (u64)a.top_k < finite;
      if (by_k && cb < (u64)a.top_k && (u64)a.top_k <= cb + n) y.bin_k = tid;
      __syncthreads();
      // the bin of min_p's border, up to one off by roundings
      const int bm = a.min_z > -INFINITY ? (int)fmax(fmin((double)top - floor((row.m + a.min_z) * a.per_z), (double)kBins), 0.0) : kBins;
      // Top-k that ends in the last bin, among tokens of no weight, takes nothing from the others: all that it says is how many are kept,
      // if nothing else does.  Where min_p's border may lie in that bin too, it cuts there like in any other.
      const int bin_k = y.bin_k;
      const bool both_last = !by_p && a.min_z > -INFINITY && bm + 1 >= kBins - 1;
      fixed = by_k && bin_k == kBins - 1 && !by_p && a.min_z == -INFINITY ? a.top_k : 0;
      by_k = by_k && (bin_k < kBins - 1 || both_last);
      const u64 want = by_p ? mass_wanted(a.top_p, all) : 0;
      if (by_p && !by_k && mb < want && want <= mb + s) y.bin_p = tid;
      __syncthreads();
      // kBins: no cut.  (Where top-p goes by the sum of the top-k, these have to be there.)
      const int k_at = by_k ? bin_k : kBins, p_at = y.bin_p;
      lo = hi = min(k_at, p_at);
      if (a.min_z > -INFINITY && !(by_k && by_p)) {
        lo = min(lo, max(bm - 1, 0));
        hi = min(hi, bm + 1);
      }
      if (lo < kBins) hi = min(hi, kBins - 1);
      y.cum_cnt[tid] = (uint32_t)cb;
      y.cum_mass[tid] = mb;
      if (tid == 0) { y.cum_cnt[kBins] = (uint32_t)finite; y.cum_mass[kBins] = all; }
      __syncthreads();
      // (hi < kBins wherever lo is)
      const int upto_hi = (int)y.cum_cnt[min(hi + 1, kBins)];
      if (lo < kBins && upto_hi <= LIST) mode = PLAN_LISTED;
      else if (!(by_k && by_p) && upto_hi - (int)y.cum_cnt[lo] <= LIST) mode = PLAN_CUT;
      by_k = by_k && k_at <= hi;
      by_p = by_p && (by_k || p_at <= hi);
      if (mode == PLAN_CUT) {
        // what lies above the bins, part by part
        for (int p0 = 0; p0 < parts; p0 += 8) {
          u64 v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int to = p0 + i < parts && y.below[p0 + i] >= 0 ? row_bin(p0 + i, tid) : kBins;
            v[i] = to < lo && to < kBins - 1 ? spreads[p0 + i][tid] : 0;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (p0 + i < parts) {
              const u64 sum = wave_sum_u64(v[i] ? bin_mass(v[i] >> 48, v[i] & kFrac, y.bins.unit[row_bin(p0 + i, tid)]) : 0);
              if (lane == 0 && sum) atomicAdd(&y.part_kept[p0 + i], sum);
            }
        }
      }
    }
    whole = mode == PLAN_WHOLE;
    if (!whole && lo < kBins) {
      // (the last bin is listed nowhere)
      const bool short_of = lane < parts && y.below[lane] >= 0 && y.below[lane] + depth_of <= hi;
      const int from = mode == PLAN_LISTED ? 0 : lo, most = part_size / kOfListed;
      if (hi < kBins - 1 && !__builtin_amdgcn_ballot_w64(short_of)) list_candidates(candidates + (size_t)r * parts * most, parts, most, c, top, from, hi, y);
      else list_bins(z, V, sums, part_size, c, top, from, hi, y);
    }
    __syncthreads();
    InList src;
    src.fetch(y.list, !whole && lo < kBins ? y.listed : 0);
    u64 of_k = all;
    for (int by_mass = 0; by_mass < 2; ++by_mass) {
      if (whole || !(by_mass ? by_p : by_k)) continue;
      const u64 want = by_mass ? mass_wanted(a.top_p, of_k) : (u64)a.top_k;
      int at = by_mass ? y.bin_p : y.bin_k;
      if (by_mass && by_k) {   // (the sum of the top-k is known only now)
        __syncthreads();
        if (y.cum_mass[tid] < want && want <= y.cum_mass[tid + 1]) y.bin_p = tid;
        __syncthreads();
        at = y.bin_p;
      }
      const uint32_t n = y.cnt[at];
      if (n <= 64) {
        if (tid == 0) x.n_few = 0;
        __syncthreads();
        src.each([&](int place, float v, bool in) {
          if (in && bins_below(top, bin_of(v, c)) == at) {
            const uint32_t i = atomicAdd(&x.n_few, 1u);
            x.few_key[i & 63] = key_of(v);
            x.few_place[i & 63] = place;
            x.few_mass[i & 63] = row.weight(v);
          }
        });
        of_k = rank_few(n, y.cum_cnt[at], y.cum_mass[at], by_mass, want, cut, x);
      } else {
        of_k = select_digits(src, row, by_mass, want, y.cum_cnt[at], y.cum_mass[at],
                             [&](float v) { return bins_below(top, bin_of(v, c)) == at; }, cut, x);
      }
      if (by_mass) {   // (what is kept, with the cut's token and without)
        const u64 without = of_k - row.weight(logit_of(cut.key)), near = all >> kNear;
        whole = want < without + near || of_k < want + near;
      }
    }
    if (!whole && mode == PLAN_LISTED) {
      u64 kept;
      int place;
      float v;
      bool close;
      if (draw_place(src, row, cut, 0, row.m + a.min_z, x, kept, count, [&](u64 k) { return draw_at(u, k); }, place, v, 0, close))
        put_token(tokens, stats, r, y.list[place].y, v, row, kept, count, all);
      return;
    }
    // what is kept of each part: all above the bins, and some of the list
    if (!whole) {
      u64 n = 0;
      src.each([&](int at, float v, bool) {
        const u64 w = row.weight(v);
        if (v > -INFINITY && v >= row.m + a.min_z && cut.keeps(key_of(v), at)) {
          ++n;
          atomicAdd(&y.part_kept[y.list[at].y / part_size], w);
        }
      });
      count = y.cum_cnt[lo] + (uint32_t)block_sum_u64(n, x);
      if (fixed) count = fixed;
      if (cut.last != INT_MAX) cut.last = y.list[cut.last].y;
    }
  } else {
    const bool some = lane < parts && mine.m > -INFINITY;
    if (tid < 64)   // (the part's sum, seen from the row's maximum)
      y.part_kept[tid] = some ? (u64)((double)mine.sum * (exp2_times_2to46(((double)mine.m - (double)m) * a.scale) * 0x1p-46) + 0.5) : 0;
    count = (uint32_t)wave_sum_u64(some ? (u64)mine.count : 0);
  }
  __syncthreads();
  if (!whole) {
    const u64 kept = wave_sum_u64(y.part_kept[lane]);
    if constexpr (!FILTERS) all = kept;
    // The part of the token, then the token.  The part's own weights, seen from the row's maximum, may come to a little less than its sum did, to
    // nothing where each rounds to 0: then the next part's first.  (With filters the row decides, as near a border.)
    const u64 want = draw_at(u, kept);
    u64 base = wave_before_u64(y.part_kept[lane]);
    int p = __builtin_ctzll(__builtin_amdgcn_ballot_w64(base + y.part_kept[lane] >= want));
    {
      const uint32_t bhi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(base >> 32), p), blo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)base, p);
      base = (u64)bhi << 32 | blo;
    }
    for (int tried = 0; tried <= parts; ++tried, p = p + 1 < parts ? p + 1 : 0) {
      const int first = p * part_size;
      InMemory<T> src;
      src.fetch(z + first, min(V - first, part_size));
      u64 here;
      uint32_t n;
      int place;
      float v;
      bool close;
      const bool found = draw_place(src, row, cut, first, row.m + a.min_z, x, here, n,
                                    [&](u64 k) { return tried ? min((u64)1, k) : min(want - base, k); }, place, v, FILTERS ? kept >> kNear : 0, close);
      if (found) {
        if (FILTERS && close) y.redo = 1;
        else put_token(tokens, stats, r, first + place, v, row, kept, count, all);
      }
      whole = FILTERS && here == 0;
      if (here > 0 || whole) break;   // (the same for all threads)
    }
    if constexpr (FILTERS) {
      __syncthreads();
      whole |= y.redo != 0;
    }
  }
  if constexpr (FILTERS) {
    if (whole) {
      InMemory<T> src;
      src.fetch(z, V);
      sample_whole(src, row, a, u, r, x, tokens, stats);
    }
  }
}

// ---- launchers ------------------------------------------------------------------------------------
struct SampleSizes { int ne, parts; };
// Logits to a thread: the fewest with which a batch of rows makes no more than two blocks for each compute unit; four where nothing is
// listed, as the part that the token is in is then read again.  us by trace, parts and draw, eight logits a thread against sixteen: 32 rows of
// 126464 without filters 8.5 + 6.6, 7.9 + 10.8; before parts listed tokens, 34 rows of 152064 with top-p (sixteen by the rule) 10.4 + 17.6, 10.0 + 16.9.
static SampleSizes sample_sizes(int rows, int V, bool filters) {
  const int parts = (V + kSampleThreads * 8 - 1) / (kSampleThreads * 8);
  if ((long)rows * parts <= (filters ? 512 : 1024)) return {8, parts};
  return {16, (V + kSampleThreads * 16 - 1) / (kSampleThreads * 16)};
}
// Logits of a row that one block holds in registers.  us of a call with top-k and top-p, by one block and in parts, for 24 and 591 rows: 4096
// logits 12 and 32, 15 and 30; 4097 62 and 173, 16 and 30 (32 logits a thread); 16384 68 and 195, 16 and 38.
constexpr int kSampleSmall = 4096;
struct SampleBytes { size_t sums, spreads, all; };   // where each ends
static SampleBytes sample_bytes(int rows, int V) {
  SampleBytes b = {};
  if (rows <= 0 || V <= kSampleSmall) return b;
  if (rows > kSampleBatch) rows = kSampleBatch;
  // Fewer rows may have more parts, of eight logits to a thread, up to 1024 in all: there is room for as many rows of these as it takes.  (The
  // last of several batches has few rows too.)
  const size_t p16 = (V + kSampleThreads * 16 - 1) / (kSampleThreads * 16), p8 = (V + kSampleThreads * 8 - 1) / (kSampleThreads * 8);
  const size_t small = ((size_t)rows < 1024 / p8 ? (size_t)rows : 1024 / p8) * p8;
  const size_t most = rows * p16 > small ? rows * p16 : small;
  b.sums = (most * sizeof(PartSum) + 255) / 256 * 256;
  b.spreads = b.sums + most * sizeof(Spread);
  b.all = b.spreads + most * kListedMost * sizeof(int2);
  return b;
}
size_t sample_workspace(int rows, int V) { return sample_bytes(rows, V).all; }

template <typename T, bool FILTERS, int LIST>
static void launch_sample_draw(const T* logits, int rows, int parts, int V, size_t ld, int part_size, const float* uniforms,
                               const SampleArgs& a, const PartSum* sums, const Spread* spreads, const int2* candidates, int* tokens, float4* stats,
                               hipStream_t s) {
  constexpr int smem = sizeof(RowScratch<LIST>);
  static_assert(smem <= 80 * 1024, "two blocks to a compute unit");
  static std::atomic<uint64_t> done{0};
  allow_lds((const void*)sample_draw_kernel<T, FILTERS, LIST>, smem, done);
  sample_draw_kernel<T, FILTERS, LIST><<<rows, kSampleThreads, smem, s>>>(logits, V, ld, parts, part_size, uniforms, a, sums, spreads, candidates,
                                                                          tokens, stats);
}
template <typename T, int NE>
static void launch_sample_ne(const T* logits, int rows, int parts, int V, size_t ld, const float* uniforms, const SampleArgs& a, int* tokens,
                             float4* stats, char* ws, const SampleBytes& b, hipStream_t s) {
  PartSum* sums = (PartSum*)ws;
  Spread* spreads = (Spread*)(ws + b.sums);
  int2* candidates = (int2*)(ws + b.spreads);
  const dim3 grid(parts, rows);
  if (a.top_k > 0 || a.top_p < 1.0 || a.min_z > -INFINITY) {
    sample_parts_kernel<T, NE, true><<<grid, kSampleThreads, 0, s>>>(logits, V, ld, a.scale, a.per_z, sums, spreads, candidates);
    launch_sample_draw<T, true, kList>(logits, rows, parts, V, ld, kSampleThreads * NE, uniforms, a, sums, spreads, candidates, tokens, stats, s);
  } else {
    sample_parts_kernel<T, NE, false><<<grid, kSampleThreads, 0, s>>>(logits, V, ld, a.scale, a.per_z, sums, spreads, candidates);
    launch_sample_draw<T, false, 1>(logits, rows, parts, V, ld, kSampleThreads * NE, uniforms, a, sums, spreads, candidates, tokens, stats, s);
  }
}

template <typename T>
static void launch_sample_t(const T* logits, int rows, int V, size_t ld, const float* uniforms, const SampleArgs& a, int* tokens,
                            float4* stats, void* workspace, hipStream_t s) {
  if (V <= kSampleSmall) {
    if (V <= 1024) sample_small_kernel<T, 2><<<rows, kSampleThreads, 0, s>>>(logits, V, ld, uniforms, a, tokens, stats);
    else sample_small_kernel<T, 8><<<rows, kSampleThreads, 0, s>>>(logits, V, ld, uniforms, a, tokens, stats);
    return;
  }
  const SampleBytes b = sample_bytes(rows, V);
  for (int r = 0; r < rows; r += kSampleBatch) {
    const int n = rows - r < kSampleBatch ? rows - r : kSampleBatch;
    const SampleSizes w = sample_sizes(n, V, a.top_k > 0 || a.top_p < 1.0 || a.min_z > -INFINITY);
    const T* z = logits + (size_t)r * ld;
    if (w.ne == 8) launch_sample_ne<T, 8>(z, n, w.parts, V, ld, uniforms + r, a, tokens + r, stats + r, (char*)workspace, b, s);
    else launch_sample_ne<T, 16>(z, n, w.parts, V, ld, uniforms + r, a, tokens + r, stats + r, (char*)workspace, b, s);
  }
}
void launch_sample_rows(const void* logits, bool bf16, int rows, int V, size_t ld, const float* uniforms, const SampleArgs& a,
                        int* tokens, float4* stats, void* workspace, hipStream_t s) {
  if (bf16) launch_sample_t((const bf16_t*)logits, rows, V, ld, uniforms, a, tokens, stats, workspace, s);
  else launch_sample_t((const float*)logits, rows, V, ld, uniforms, a, tokens, stats, workspace, s);
}

}  // namespace ec
