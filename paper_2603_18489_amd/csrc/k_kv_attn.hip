// Attention of a batch of sequences over a paged cache (k_kv.h), with a prefix that all of them share.
//
// out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale (q . k_j) - m),  m the largest of the exponents so far: one pass over the keys, with
// what was added up so far multiplied by exp(m_old - m_new) whenever m grows.  Per 32 keys (a chunk) and 16 rows of queries (a row of
// queries: one head of one row, the heads of a kv head's group next to each other):
//   S^T[keys x queries] = K . Q^T, softmax down the keys, O^T[components x queries] += V^T . P^T
// with the operands as they lie in the cache.  e4m3 keys are widened to bfloat16 with their power of two, exactly.  Values are widened
// so too where many queries share them; few queries' probabilities take it instead, an exact product again, before they are rounded to bfloat16 (2^-8 of them
// at most, 2^-16 with up to 16 queries).  Scores, maxima and sums are float32.  One part of a probability is off by less than the result's own rounding: together 0.0019 to
// 0.0022 of the result, where the result's rounding alone is 0.0017.  A second part for more than 16 queries too would take 16 x 34 rows from 36.8 to 40.0 us, 16 x 1536 from 624 to 826.
//
// Keys are cut into slices of chunks, a block each; the slices' (m, sum, O) meet in a second launch, in their order.  The prefix' slices take
// the rows of all sequences at once, so that its keys are read once for all.  A query that sees no key gets zeros: m begins so low
// that no score but -inf lies below, and a sum of 0 divides nothing.
#include <float.h>

#include <cmath>

#include "k_kv.h"
#include "k_maxima.h"

namespace ec {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 8 codes times a power of two, as bfloat16
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b, float f) {
  union { bf16x2 h[4]; bf16x8 v; } c;
  c.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, f, false);
  c.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, f, true);
  c.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, f, false);
  c.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, f, true);
  return c.v;
}
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) {
  union { u32x4 u; bf16x8 b; } c;
  c.u = v;
  return c.b;
}
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }   // (255: infinity, which makes NaN of 0)
__device__ __forceinline__ uint32_t byte_of(uint32_t word, int n) { return (word >> (8 * (n & 3))) & 255u; }

// what a kernel knows of the call
struct Args {
  const bf16_t* q; size_t q_ld, q_head;
  bf16_t* out; size_t out_ld, out_head;
  int rows, heads, group, seqs, max_rows, max_keys, each;
  const int *table, *lengths, *starts;
  size_t table_ld;
  const int* prefix; int prefix_len;
  bool causal;
  float scale;                       // with log2(e)
  float lag, low;                    // kLag / scale; what maxima begin at: the least that stays finite when it is scaled
  const uint8_t *data, *scales;
  KvPlace place; int pages;
  int split, prefix_split;           // chunks of a slice
  int slices, prefix_slices;         // slices at most
  float* part; float2* sums;         // [rows][heads][prefix_slices + slices][HD], and (m, sum)
};

// rows and keys of a sequence, kept inside what the call gave
struct Seq { int row0, n, keys; };
__device__ __forceinline__ Seq seq_of(const Args& a, int b) {
  Seq s;
  s.row0 = b * a.each;
  int end = s.row0 + a.each;
  if (a.starts) {
    s.row0 = min(max(a.starts[b], 0), a.rows);
    end = min(max(a.starts[b + 1], 0), a.rows);
  }
  s.row0 = __builtin_amdgcn_readfirstlane(s.row0);     // (of the block: no product of matrices may hang on a lane's condition)
  s.n = __builtin_amdgcn_readfirstlane(min(max(end - s.row0, 0), a.max_rows));
  s.keys = __builtin_amdgcn_readfirstlane(min(max(a.lengths[b], 0), a.max_keys));
  return s;
}

// What a block works on: rows of a sequence (or of the whole call, over the prefix) and a slice of its keys.
struct Part {
  Seq s;
  const int* table;
  int first, queries;         // its queries begin here; queries of the sequence and kv head
  int kvh, slice, c_lo, c_hi; // chunks
  int seen_first;             // keys that its first row sees
  bool causal;
  // row, head and keys seen of query `m`; behind the last query: the last one's
  __device__ __forceinline__ void query(const Args& a, int m, int* row, int* head, int* seen) const {
    m = min(m, queries - 1);
    const int r = m / a.group;
    *row = s.row0 + r;
    *head = kvh * a.group + (m - r * a.group);
    *seen = causal ? s.keys - s.n + 1 + r : s.keys;
  }
};
// false: nothing to do.  EACH: queries of a block.  Blocks that read the same keys are kv_heads apart, next to each other otherwise: mostly on one
// XCD, whose L2 they share.  Late rows, which see most under `causal`, go first.
template <int EACH, bool PREFIX>
__device__ __forceinline__ bool part_of(const Args& a, unsigned id, int tiles, Part& p) {
  p.kvh = id % a.place.kv_heads;
  id /= a.place.kv_heads;
  const int tile = tiles - 1 - (int)(id % tiles);
  id /= tiles;
  const int slices = PREFIX ? a.prefix_slices : a.slices, b = id / slices;
  p.slice = id % slices;
  p.s = PREFIX ? Seq{0, a.rows, a.prefix_len} : seq_of(a, b);
  p.first = tile * EACH;
  p.queries = p.s.n * a.group;
  if (p.first >= p.queries) return false;
  p.table = PREFIX ? a.prefix : a.table + (size_t)b * a.table_ld;
  const int split = PREFIX ? a.prefix_split : a.split;
  p.causal = !PREFIX && a.causal;
  p.c_lo = p.slice * split;
  if (p.slice > 0 && p.c_lo * 32 >= p.s.keys) return false;   // (the slices that are joined go by the keys too)
  const int last_row = (min(p.first + EACH, p.queries) - 1) / a.group;
  p.seen_first = p.causal ? p.s.keys - p.s.n + 1 + p.first / a.group : p.s.keys;
  const int seen_last = p.causal ? p.s.keys - p.s.n + 1 + last_row : p.s.keys;
  p.c_hi = min(p.c_lo + split, (max(seen_last, 0) + 31) >> 5);
  return true;
}

// The pages of every `step`-th chunk from `first` on, 64 of them in a wave's lanes
struct Pages {
  const int* table;
  int first, step, last, shift, ids;
  __device__ __forceinline__ int of(int i, int lane) {
    if ((i & 63) == 0) {
      ids = table[min(first + step * (i + lane), last) >> shift];
      asm volatile("" : "+v"(ids));   // (waited for here: where this path meets the other, every load on its way would be)
    }
    return __builtin_amdgcn_readlane(ids, i & 63);
  }
};

// The exponentials' reference is a maximum that lags behind by up to 2^kLag: moving it multiplies a whole tile of results, and with a lag the
// first chunks settle it for most queries.  (Probabilities of up to 2^kLag are as exact as those of up to 1: all of this is floating point.)
constexpr float kLag = 8.f;

// The scores of 16 queries and 32 keys (S^T: a lane has 8 neighbouring keys of query lane & 15): a lane's largest, which alone says whether the
// maximum has to move, and the query's, in each of its lanes
__device__ __forceinline__ float top_of_lane(const f32x4 (&sc)[2]) { return max_of_8(sc[0], sc[1]); }
__device__ __forceinline__ float top_of_query(float lane_top) { return max_of_swap32(max_of_swap16(lane_top)); }

// The maximum m is a score, not yet scaled, and a probability 2^(s scale - m scale) takes one multiplication and addition with the rounded m scale.  That
// is off from the exact one by up to 2^-24 of itself, for all keys alike, and cancels - but from a scaled maximum of 2^31 on by a factor of 2^128, which
// is no number, or zero.  From 2^24 on (`far`) exponents are (s - m) scale instead, where a score near m leaves no rounding.  (16 x 1536 rows over 1536 keys:
// 629 us without, 632 with; 16 x 34 rows: 34.9 and 35.3, in bfloat16 63.9 and 65.9.)
constexpr float kFar = 16777216.f;
__device__ __forceinline__ bool far(float m, float scale) { return !(fabsf(m * scale) < kFar); }
// the exponent by which what was added up with maximum m goes over to maximum m_new
__device__ __forceinline__ float moved_by(float m, float m_new, float scale) {
  const float a = m * scale, b = m_new * scale;
  return (m - m_new) * scale - (far(m, scale) ? 0.f : fmaf(m, scale, -a)) + (far(m_new, scale) ? 0.f : fmaf(m_new, scale, -b));
}
// The maximum m moves to mx, what has been added up goes with it, and the scores of far queries have it taken off.  ref: what probabilities subtract.
// some_far: the wave's queries that have been far, whose every chunk comes here.  (One branch for both: behind a second one the compiler keeps the results twice.)
template <int HT, typename Sum>
__device__ __forceinline__ void move_top(f32x4 (&acc)[HT], float& m, Sum& l, f32x4 (&sc)[2], float mx, float scale, float& ref, uint64_t& some_far) {
  const float m_new = max_of(m, mx), alpha = __builtin_amdgcn_exp2f(moved_by(m, m_new, scale));
  const bool off = far(m_new, scale);
  some_far |= __builtin_amdgcn_ballot_w64(off && m_new != m);    // (not where no key has been seen)
  m = m_new;
  ref = off ? 0.f : m * scale;
#pragma unroll
  for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] -= off ? m : 0.f;
  l *= alpha;
#pragma unroll
  for (int h = 0; h < HT; ++h) acc[h] *= alpha;
}
__device__ __forceinline__ bf16x8 pack8(const float (&p)[8]) {
  return u4_as_bf16x8(make_uint4(pack2_bf16(p[0], p[1]), pack2_bf16(p[2], p[3]), pack2_bf16(p[4], p[5]), pack2_bf16(p[6], p[7])));
}

// a piece of values, with the keys from `live` on (of its 8) as zeros: what lies behind the last key may be anything
template <int ES> __device__ __forceinline__ void cut_values(u32x4& v, int live) {
  if constexpr (ES == 1) {
    const uint64_t keep = live >= 8 ? ~0ull : (1ull << (8 * max(live, 0))) - 1;
    v &= (u32x4){(uint32_t)keep, (uint32_t)(keep >> 32), (uint32_t)keep, (uint32_t)(keep >> 32)};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] &= (2 * e < live ? 0xffffu : 0u) | (2 * e + 1 < live ? 0xffff0000u : 0u);
  }
}

// 8 neighbouring components of a query, o / l or, where slices are joined, o and (m, l)
template <int HD, bool DIRECT>
__device__ __forceinline__ void leave(const Args& a, int row, int head, int slice, int c, const float (&o)[8], float m, float l) {
  if constexpr (DIRECT) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    *(uint4*)(a.out + (size_t)row * a.out_ld + (size_t)head * a.out_head + c) =
        make_uint4(pack2_bf16(o[0] * inv, o[1] * inv), pack2_bf16(o[2] * inv, o[3] * inv), pack2_bf16(o[4] * inv, o[5] * inv),
                   pack2_bf16(o[6] * inv, o[7] * inv));
  } else {
    const size_t at = ((size_t)row * a.heads + head) * (a.prefix_slices + a.slices) + slice;
    float4* to = (float4*)(a.part + at * HD + c);
    to[0] = make_float4(o[0], o[1], o[2], o[3]);
    to[1] = make_float4(o[4], o[5], o[6], o[7]);
    if (c == 0) a.sums[at] = make_float2(m, l);
  }
}

// One chunk as a lane holds it
template <int ES, int HD> struct Chunk {
  static constexpr int U = KvChunk<ES, HD>::kUnits, V = HD / 32 * ES;
  u32x4 k[2 * U], v[V];
  uint32_t ks[2];
  u32x2 vs;
  const u32x4* data;
  const uint8_t* scales;
  bool there;
  __device__ __forceinline__ void at(const Args& a, int page, int no, int kvh) {
    there = page >= 0 && page < a.pages;
    const size_t chunk = ((((size_t)(there ? page : 0) * a.place.kv_heads + kvh) << a.place.shift) + (no & ((1 << a.place.shift) - 1)));
    data = (const u32x4*)(a.data + chunk * KvChunk<ES, HD>::kBytes);
    scales = a.scales + chunk * 64;
  }
  __device__ __forceinline__ void keys(int lane) {
#pragma unroll
    for (int i = 0; i < 2 * U; ++i) k[i] = data[i * 64 + lane];
    if constexpr (ES == 1) {
      ks[0] = ((const uint32_t*)scales)[((lane & 15) >> 2) * 2];
      ks[1] = ((const uint32_t*)scales)[((lane & 15) >> 2) * 2 + 1];
    }
  }
  __device__ __forceinline__ void values(int lane) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = data[(2 * U + i) * 64 + lane];
    vs = *(const u32x2*)(scales + 32 + (lane >> 4) * 8);
  }
};

}  // namespace

// Few queries: up to 48 of a sequence and kv head.  A block's waves go through the chunks of its slice in turn, each with all QT tiles of 16
// queries and a chunk's pieces in registers, and meet in LDS.  The next chunk's keys are on their way from when this one's are used, the values too; one tile of
// queries leaves registers for a second chunk.  The power of two of a key's values multiplies its probability.
// With one tile the matrix cores wait for memory, so that a probability can be two bfloat16 numbers, 2^-16 together, instead of one.
// DIRECT: there is one slice, and the block writes the result.
// 1 row over 131071 bfloat16 keys (28 heads on 4): 48 us, 5.7 TB/s.  16 sequences of up to 34 rows over up to 1536 e4m3 keys (32 heads): 33 us, 3 tiles,
// as long as their bytes and products take one after the other.  1 row over 1000 keys: 8.5, a chain of loads.
template <int HD, int QT> struct Few {
  static constexpr int W = 4;                   // waves
  static constexpr int HB = HD / 32, HT = HD / 16;
  static constexpr int SLOT = HT * 64 + 32;     // float4 of a wave's part of a tile
  static constexpr bool PARKED = QT > 2;        // queries in LDS, as a third tile's registers would spill others
  static constexpr int LDS = W * SLOT + (PARKED ? QT * HB * 64 : 0);
};
template <int ES, int HD, int QT, bool PREFIX, bool DIRECT>
__device__ __forceinline__ void attend_few(const Args& a, unsigned id, int tiles, u32x4* mem) {
  typedef Few<HD, QT> F;
  constexpr int W = F::W, HB = F::HB, HT = F::HT, U = KvChunk<ES, HD>::kUnits, SLOT = F::SLOT;
  constexpr bool PARKED = F::PARKED;
  typedef Chunk<ES, HD> C;
  float4* lds = (float4*)mem;
  u32x4* parked = mem + W * SLOT;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = lane >> 4, col = lane & 15;
  Part part;
  if (!part_of<16 * QT, PREFIX>(a, id, tiles, part)) return;

  bf16x8 qf[PARKED ? 1 : QT][HB];
  int seen[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    int row, head;
    part.query(a, part.first + t * 16 + col, &row, &head, &seen[t]);
    const bf16_t* p = a.q + (size_t)row * a.q_ld + (size_t)head * a.q_head + grp * (HD / 4);
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      if constexpr (!PARKED) qf[t][hb] = as_bf16x8(*(const u32x4*)(p + hb * 8));
      else if (hb % W == wave) parked[(t * HB + hb) * 64 + lane] = *(const u32x4*)(p + hb * 8);
    }
  }
  if constexpr (PARKED) __syncthreads();
  f32x4 acc[QT][HT];
  float m_run[QT], l_run[QT];
  uint64_t some_far = 0;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_run[t] = a.low;
    l_run[t] = 0.f;
#pragma unroll
    for (int h = 0; h < HT; ++h) acc[t][h] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  const int from = part.c_lo + wave;                                                        // this wave's first chunk
  const int mine = from < part.c_hi ? (part.c_hi - from + W - 1) / W : 0;         // and how many it has
  Pages pages = {part.table, from, W, from + W * (mine - 1), a.place.shift, 0};
  auto place = [&](C& c, int i) {
    const int n = min(i, mine - 1);     // (behind the last chunk it comes once more, from the cache)
    c.at(a, pages.of(n, lane), from + W * n, part.kvh);
  };
  f32x4 sc[QT][2];
  auto score = [&](const C& c) {
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2) {
      bf16x8 kf[HB];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const u32x4 k = c.k[t2 * U + u];
        if constexpr (ES == 1) {
          const float f = power_of(byte_of(c.ks[t2], lane));
          kf[2 * u] = widen8(k[0], k[1], f);
          kf[2 * u + 1] = widen8(k[2], k[3], f);
        } else {
          kf[u] = as_bf16x8(k);
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) sc[t][t2] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int hb = 0; hb < HB; ++hb) {      // (the tiles in turn: a product waits for the one before it on the same sums)
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          const bf16x8 q = PARKED ? as_bf16x8(parked[(t * HB + hb) * 64 + lane]) : qf[PARKED ? 0 : t][hb];
          sc[t][t2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[hb], q, sc[t][t2], 0, 0, 0);
        }
      }
    }
  };
  auto attend = [&](C& c, int i, bool there) {
    const int key0 = (from + W * i) * 32, k0 = key0 + grp * 8;
    const bool masked = key0 + 32 > part.seen_first || !there;
    if (masked) {
      const int live = there ? part.s.keys - k0 : 0;
#pragma unroll
      for (int h = 0; h < C::V; ++h) cut_values<ES>(c.v[h], live);
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (k0 + e >= seen[t] || !there) sc[t][e >> 2][e & 3] = -INFINITY;
    }
    float vs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) vs[e] = power_of((c.vs[e >> 2] >> (8 * (e & 3))) & 255u);
    bf16x8 pf[QT], pl[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float mx = top_of_lane(sc[t]);
      float ref = m_run[t] * a.scale;
      if ((__builtin_amdgcn_ballot_w64(mx > m_run[t] + a.lag) | some_far) != 0)
        move_top(acc[t], m_run[t], l_run[t], sc[t], top_of_query(mx), a.scale, ref, some_far);
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(sc[t][e >> 2][e & 3], a.scale, -ref));
        l_run[t] += p[e];
        p[e] *= vs[e];
      }
      if (masked) {   // (a hidden key's power of two may be none)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (k0 + e >= seen[t] || !there) p[e] = 0.f;
      }
      pf[t] = pack8(p);
      if constexpr (QT == 1) {
        union { bf16x8 b; uint32_t u[4]; } c = {pf[t]};
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] -= __uint_as_float(e & 1 ? c.u[e >> 1] & 0xffff0000u : c.u[e >> 1] << 16);
        pl[t] = pack8(p);
      }
    }
    if constexpr (QT == 3 && ES == 2) __builtin_amdgcn_sched_barrier(0);   // (values that are read ahead of this would be spilled)
#pragma unroll
    for (int h = 0; h < HT; ++h) {
      bf16x8 vf;
      if constexpr (ES == 1) vf = h & 1 ? widen8(c.v[h >> 1][2], c.v[h >> 1][3], 1.f) : widen8(c.v[h >> 1][0], c.v[h >> 1][1], 1.f);
      else vf = as_bf16x8(c.v[h]);
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        acc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t], acc[t][h], 0, 0, 0);
        if constexpr (QT == 1) acc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[t], acc[t][h], 0, 0, 0);
      }
    }
  };
  if constexpr (QT == 1) {
    C one, two;
    if (mine > 0) {
      place(one, 0);
      one.keys(lane);
      one.values(lane);
    }
    for (int i = 0; i < mine; i += 2) {
      place(two, i + 1);
      two.keys(lane);
      two.values(lane);
      __builtin_amdgcn_sched_barrier(0);
      score(one);
      attend(one, i, one.there);
      __builtin_amdgcn_sched_barrier(0);
      place(one, i + 2);
      one.keys(lane);
      one.values(lane);
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < mine) {
        score(two);
        attend(two, i + 1, two.there);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  } else {
    C c;
    if (mine > 0) {
      place(c, 0);
      c.keys(lane);
      c.values(lane);
    }
    for (int i = 0; i < mine; ++i) {
      score(c);
      __builtin_amdgcn_sched_barrier(0);
      const bool there = c.there;
      place(c, i + 1);
      c.keys(lane);
      __builtin_amdgcn_sched_barrier(0);
      attend(c, i, there);
      __builtin_amdgcn_sched_barrier(0);
      c.values(lane);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // ---- the waves' parts meet, tile by tile: (m, sum, O) of each, in their order
  float4* slot = lds + (size_t)wave * SLOT;
  const int at_slice = PREFIX ? part.slice : a.prefix_slices + part.slice;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    if (t > 0) __syncthreads();
    float l = l_run[t];
    l += other_row(l);
    l += other_half(l);
    ((float2*)(slot + HT * 64))[lane] = make_float2(m_run[t], l);
#pragma unroll
    for (int h = 0; h < HT; ++h) slot[h * 64 + lane] = make_float4(acc[t][h][0], acc[t][h][1], acc[t][h][2], acc[t][h][3]);
    __syncthreads();
    float m_all = a.low, l_all = 0.f, f[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      f[w] = ((const float2*)(lds + (size_t)w * SLOT + HT * 64))[lane].x;
      m_all = fmaxf(m_all, f[w]);
    }
#pragma unroll
    for (int w = 0; w < W; ++w) {
      f[w] = __builtin_amdgcn_exp2f(moved_by(f[w], m_all, a.scale));
      l_all += ((const float2*)(lds + (size_t)w * SLOT + HT * 64))[lane].y * f[w];
    }
    const int m = part.first + t * 16 + col;
    int row, head, unused;
    part.query(a, m, &row, &head, &unused);
    for (int p = wave; p < HT / 2 && m < part.queries; p += W) {
      float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float4 x = lds[(size_t)w * SLOT + 2 * p * 64 + lane], y = lds[(size_t)w * SLOT + (2 * p + 1) * 64 + lane];
        o[0] += x.x * f[w]; o[1] += x.y * f[w]; o[2] += x.z * f[w]; o[3] += x.w * f[w];
        o[4] += y.x * f[w]; o[5] += y.y * f[w]; o[6] += y.z * f[w]; o[7] += y.w * f[w];
      }
      leave<HD, DIRECT>(a, row, head, at_slice, p * 32 + grp * 8, o, m_all, l_all);
    }
  }
}

// 16 codes of values, of 8 keys whose powers of two are the bytes of vs, as bfloat16.  (The conversion takes a factor's exponent bits alone.)
__device__ __forceinline__ void widen_values(u32x4 v, u32x2 vs, u32x4& x, u32x4& y) {
  union { bf16x2 h; uint32_t u; } a, b;
#pragma unroll
  for (int k = 0; k < 4; ++k) {   // keys 2 k and 2 k + 1
    const uint32_t s = vs[k >> 1], w = v[k >> 1], z = v[2 + (k >> 1)];
    const float f = __uint_as_float(k & 1 ? s << 7 : s << 23), g = __uint_as_float(k & 1 ? s >> 1 : s << 15);
    a.h = k & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, false);
    b.h = k & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, g, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, g, false);
    x[k] = (a.u & 0xffffu) | (b.u & 0xffff0000u);
    a.h = k & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(z, f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(z, f, false);
    b.h = k & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(z, g, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(z, g, false);
    y[k] = (a.u & 0xffffu) | (b.u & 0xffff0000u);
  }
}

// Many queries: a wave owns QT tiles of 16, a block 64 QT, and its waves go through the keys together.  Each chunk comes through registers, where codes
// are widened once for all, values with their powers of two, into one of two stages of LDS; the next one's pieces are on their way meanwhile.  The
// probabilities' sums are a product of P^T with ones: what is rounded is what is added up.
// 16 x 1536 rows over 1536 e4m3 keys, 32 heads of 128: 620 to 640 us, 0.97 to 1.0 PFLOP/s.  What bounds it is the issue of instructions: the matrix cores are at work in 43 % of
// the cycles, and the other vector instructions, of softmax and widening, 3.6 to a product, issue in 43 % too, of which two waves a SIMD hide little behind products.
// Chunks that hold a key which some query does not see, or values that are NaN, go a slower way; the others' code has one rare branch.
template <int HD> constexpr int kManyLds = 2 * (2 * HD / 32 + HD / 16) * 64;
template <int ES, int HD, int QT, bool PREFIX, bool DIRECT>
__device__ __forceinline__ void attend_many(const Args& a, unsigned id, int tiles, u32x4* lds) {
  constexpr int HB = HD / 32, HT = HD / 16, U = KvChunk<ES, HD>::kUnits;
  constexpr int KP = 2 * U * 64, ALL = KvChunk<ES, HD>::kBytes / 16, N = ALL / 256;   // pieces of 16 bytes: keys, all, a thread's
  constexpr int KF = 2 * HB * 64, STAGE = KF + HT * 64;                                  // of a stage: keys, all
  static_assert(ALL % 256 == 0 && KP % 64 == 0 && 2 * STAGE == kManyLds<HD>, "a wave's pieces are keys or values");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = lane >> 4, col = lane & 15;
  Part part;
  if (!part_of<64 * QT, PREFIX>(a, id, tiles, part)) return;
  const int first = part.first + wave * 16 * QT;

  bf16x8 qf[QT][HB];
  int seen[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    int row, head;
    part.query(a, first + t * 16 + col, &row, &head, &seen[t]);
    const bf16_t* p = a.q + (size_t)row * a.q_ld + (size_t)head * a.q_head + grp * (HD / 4);
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) qf[t][hb] = as_bf16x8(*(const u32x4*)(p + hb * 8));
  }
  f32x4 acc[QT][HT], l_run[QT];
  float m_run[QT];
  uint64_t some_far = 0;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_run[t] = a.low;
    l_run[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < HT; ++h) acc[t][h] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  const int n = max(part.c_hi - part.c_lo, 0);
  Pages pages = {part.table, part.c_lo, 1, part.c_hi - 1, a.place.shift, 0};
  u32x4 piece[N];
  uint32_t ks[N], four = 0;     // (words: a byte would be widened, and waited for, long before it is used)
  u32x2 vs = {};
  bool there = false;
  // whether a wave's j-th pieces are keys: known when compiled, unless a chunk's keys are less than the block's threads
  auto is_keys = [&](int j) { return KP % 256 == 0 ? j * 256 < KP : j * 256 + wave * 64 < KP; };
  // (nothing here hangs on a condition: where loads and what was loaded before meet, the loads would be waited for.  Behind the last chunk it comes again.)
  auto load = [&](int i) {
    i = min(i, n - 1);
    const int page = pages.of(i, lane), no = part.c_lo + i;
    there = page >= 0 && page < a.pages;
    const size_t chunk = ((((size_t)(there ? page : 0) * a.place.kv_heads + part.kvh) << a.place.shift) + (no & ((1 << a.place.shift) - 1)));
    const u32x4* p = (const u32x4*)(a.data + chunk * KvChunk<ES, HD>::kBytes);
    const uint8_t* s = a.scales + chunk * 64;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int q = j * 256 + (int)threadIdx.x;
      piece[j] = p[q];
      if constexpr (ES == 1) {
        if (is_keys(j)) ks[j] = ((const uint32_t*)s)[(col >> 2) * 2 + q / (U * 64)];
      }
    }
    if constexpr (ES == 1) vs = *(const u32x2*)(s + 32 + grp * 8);
    four = ((const uint32_t*)s)[8 + (lane & 31) / 4];
  };
  // what a step has to know of the chunk that is in LDS: keys of no page, and a bit for each key whose values are NaN
  struct Known { bool there; uint32_t bad; };
  auto store = [&](u32x4* stage, int i) {
    const int k0 = (part.c_lo + i) * 32 + grp * 8, live = there ? part.s.keys - k0 : 0;
    Known known = {there, (uint32_t)__builtin_amdgcn_ballot_w64(byte_of(four, lane) == 255u)};
    if ((part.c_lo + i) * 32 + 32 > part.s.keys || !there || known.bad != 0) {
      asm volatile("; the last chunk, or one with values that are NaN");    // (a branch and no selections)
      if constexpr (ES == 1) {     // powers of two that are none, of keys that are not there or of zeros: any will do
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= live || ((vs[e >> 2] >> (8 * (e & 3))) & 255u) == 255u) vs[e >> 2] &= ~(255u << (8 * (e & 3)));
      }
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (!is_keys(j)) cut_values<ES>(piece[j], live);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int q = j * 256 + wave * 64;      // (of the wave: keys or values)
      union { bf16x8 b; u32x4 v; } x, y;
      if (is_keys(j)) {
        if constexpr (ES == 1) {
          const int t2 = q / (U * 64), u = q / 64 % U;
          const float f = power_of(byte_of(ks[j], lane));
          x.b = widen8(piece[j][0], piece[j][1], f);
          y.b = widen8(piece[j][2], piece[j][3], f);
          stage[(t2 * HB + 2 * u) * 64 + lane] = x.v;
          stage[(t2 * HB + 2 * u + 1) * 64 + lane] = y.v;
        } else {
          stage[q + lane] = piece[j];
        }
      } else {
        const int h = (q - KP) / 64;
        if constexpr (ES == 1) {
          widen_values(piece[j], vs, x.v, y.v);
          stage[KF + 2 * h * 64 + lane] = x.v;
          stage[KF + (2 * h + 1) * 64 + lane] = y.v;
        } else {
          stage[KF + h * 64 + lane] = piece[j];
        }
      }
    }
    return known;
  };
  const bf16x8 ones = u4_as_bf16x8(make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
  auto step = [&](const u32x4* stage, int i, Known known) {
    const bool slow = (part.c_lo + i) * 32 + 32 > part.seen_first || !known.there || known.bad;
    f32x4 sc[QT][2];
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2) {
      bf16x8 kf[HB];
#pragma unroll
      for (int hb = 0; hb < HB; ++hb) kf[hb] = as_bf16x8(stage[(t2 * HB + hb) * 64 + lane]);
#pragma unroll
      for (int t = 0; t < QT; ++t) sc[t][t2] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int hb = 0; hb < HB; ++hb)      // (the tiles in turn: a product waits for the one before it on the same sums)
#pragma unroll
        for (int t = 0; t < QT; ++t) sc[t][t2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[hb], qf[t][hb], sc[t][t2], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0x8);    // (products may pass; reads of values that are brought forward to here would take the registers of two tiles)
    const int k0 = (part.c_lo + i) * 32 + grp * 8;
    if (slow) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if ((known.bad >> (grp * 8 + e)) & 1u) sc[t][e >> 2][e & 3] = __uint_as_float(0x7fc00000u);
          if (k0 + e >= seen[t] || !known.there) sc[t][e >> 2][e & 3] = -INFINITY;
        }
    }
    float mx[QT], ref[QT];
    bool up = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      mx[t] = top_of_lane(sc[t]);
      up = up || mx[t] > m_run[t] + a.lag;
      ref[t] = m_run[t] * a.scale;
    }
    if ((__builtin_amdgcn_ballot_w64(up) | some_far) != 0) {
#pragma unroll
      for (int t = 0; t < QT; ++t) move_top(acc[t], m_run[t], l_run[t], sc[t], top_of_query(mx[t]), a.scale, ref[t], some_far);
    }
    bf16x8 pf[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(sc[t][e >> 2][e & 3], a.scale, -ref[t]));
      pf[t] = pack8(p);
      l_run[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[t], l_run[t], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int h = 0; h < HT; ++h) {
      const bf16x8 vf = as_bf16x8(stage[KF + h * 64 + lane]);
#pragma unroll
      for (int t = 0; t < QT; ++t) acc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t], acc[t][h], 0, 0, 0);
    }
  };
  Known next = {false, 0};
  if (n > 0) {
    load(0);
    next = store(lds, 0);
    load(1);
  }
  block_barrier_nofence();
  for (int i = 0; i < n; ++i) {
    const u32x4* stage = lds + (i & 1) * STAGE;
    const Known now = next;
    next = store(lds + (~i & 1) * STAGE, i + 1);     // (behind the last chunk: what no one reads)
    load(i + 2);
    step(stage, i, now);
    block_barrier_nofence();
  }

  const int at_slice = PREFIX ? part.slice : a.prefix_slices + part.slice;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float l = l_run[t][0];
    const int m = first + t * 16 + col;
    if (m >= part.queries) continue;
    int row, head, unused;
    part.query(a, m, &row, &head, &unused);
#pragma unroll
    for (int p = 0; p < HT / 2; ++p) {
      const f32x4 x = acc[t][2 * p], y = acc[t][2 * p + 1];
      const float o[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      leave<HD, DIRECT>(a, row, head, at_slice, p * 32 + grp * 8, o, m_run[t], l);
    }
  }
}

template <int ES, int HD, int QT, bool PREFIX, bool DIRECT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void kv_attention_few_kernel(Args a) {
  __shared__ u32x4 lds[Few<HD, QT>::LDS];
  attend_few<ES, HD, QT, PREFIX, DIRECT>(a, blockIdx.x, 1, lds);
}
template <int ES, int HD, int QT, bool PREFIX, bool DIRECT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void kv_attention_many_kernel(Args a, int tiles) {
  __shared__ u32x4 lds[kManyLds<HD>];
  attend_many<ES, HD, QT, PREFIX, DIRECT>(a, blockIdx.x, tiles, lds);
}
// The prefix, and sequences of up to 16 queries: one launch.  The sequences' blocks wait for memory and leave the matrix cores to the prefix', whose
// blocks go first, as they take longer (64 rows of 28 heads on 4, 16384 keys before 511 each: 54 us in two launches, 46 in one, 55 the other way round).
template <int ES, int HD, bool MANY, int QT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void kv_attention_both_kernel(Args a, int tiles, unsigned prefix) {
  constexpr int PRE = MANY ? kManyLds<HD> : Few<HD, QT>::LDS, OWN = Few<HD, 1>::LDS;
  __shared__ u32x4 lds[PRE > OWN ? PRE : OWN];
  if (blockIdx.x >= prefix) attend_few<ES, HD, 1, false, false>(a, blockIdx.x - prefix, 1, lds);
  else if constexpr (MANY) attend_many<ES, HD, QT, true, false>(a, blockIdx.x, tiles, lds);
  else attend_few<ES, HD, QT, true, false>(a, blockIdx.x, tiles, lds);
}

// The slices of a row of queries meet in their order (28 heads, 64 rows, 34 slices: 31 MB in 7.5 us): W waves take every W-th slice, a lane HD/64 components.  The slices' (m, sum) are a
// lane's each, two at most, so that all of them are on their way at once.
constexpr int kSlicesMax = 64;    // of the prefix, and of a sequence's own keys

template <int HD, int W>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(Args a) {
  constexpr int N = HD / 64;
  typedef float fN __attribute__((ext_vector_type(N)));
  __shared__ float meet[4][64][N];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = wave % W;
  const Seq s = seq_of(a, blockIdx.y);
  const int i = blockIdx.x * (4 / W) + wave / W, r = i / a.heads, head = i - r * a.heads;
  const int total = a.prefix_slices + a.slices;
  const int own = max(1, (((s.keys + 31) >> 5) + a.split - 1) / a.split), n = a.prefix_slices + own;
  const bool live = r < s.n;
  float o[N] = {}, inv = 0.f;
  if (live) {
    const size_t at = ((size_t)(s.row0 + r) * a.heads + head) * total;
    float2 x = make_float2(a.low, 0.f), y = x;
    if (lane < n) x = a.sums[at + lane];
    if (lane + 64 < n) y = a.sums[at + lane + 64];
    const float m = wave_max_dpp(fmaxf(x.x, y.x));
    const float fx = __builtin_amdgcn_exp2f(moved_by(x.x, m, a.scale)), fy = __builtin_amdgcn_exp2f(moved_by(y.x, m, a.scale));
    const float l = wave_sum_dpp(fmaf(x.y, fx, y.y * fy));
    inv = l == 0.f ? 0.f : 1.0f / l;
    const float* part = a.part + at * HD + lane * N;
    auto weight = [&](int z) {
      return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(z < 64 ? fx : fy), z & 63));
    };
    int z = sub;
    for (; z + 3 * W < n; z += 4 * W) {
      fN v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = *(const fN*)(part + (size_t)(z + k * W) * HD);
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] += v[k][e] * weight(z + k * W);
    }
    for (; z < n; z += W) {
      const fN v = *(const fN*)(part + (size_t)z * HD);
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] += v[e] * weight(z);
    }
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < N; ++e) meet[wave][lane][e] = o[e];
    __syncthreads();
    if (!live || sub != 0) return;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      o[e] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) o[e] += meet[wave + w][lane][e];
    }
  }
  if (!live) return;
  bf16_t* to = a.out + (size_t)(s.row0 + r) * a.out_ld + (size_t)head * a.out_head + lane * N;
  if constexpr (N == 2) *(uint32_t*)to = pack2_bf16(o[0] * inv, o[1] * inv);
  else *to = f32_to_bf16(o[0] * inv);
}

namespace {

// How a call's queries of one sequence and kv head, or of the prefix, are cut into blocks, and the keys into slices.
struct Cut {
  bool many;
  int qt, tiles, split, slices;
};
// Blocks that fill the compute units, and chunks of a slice at least.  (1 row over 20000 keys of 32 heads: 32.7 us, of 1024 blocks 34.5, of 256 33.2; 600 rows of 28 heads
// on 4 over 9000: 113, 127 and 167; 64 over 16384 shared ones: 42, 51 and 46.  1 row of 28 heads on 4 over 4096 keys: 7.6 us, slices of 4 chunks 8.1, of 16 8.8.)
constexpr int kBlocks = 512, kSliceChunks = 8;
constexpr int kUncut = 32;     // chunks that few queries' blocks take as one
Cut cut(long queries, int chunks, long others, bool joined) {
  Cut c;
  c.many = queries > 48;
  if (c.many) {
    // by what a tile takes (16 x 1536 rows over 1536 keys: 820, 646 and 630 us in tiles of 64, 128 and 192, 492, 403 and 380 with 64 components; 64 x 128 rows 323,
    // 264 and 353) and how full the last one is
    const double cost[3] = {1.29, 2 * 1.03, 3.0};
    double least = 0;
    for (int qt = 1; qt <= 3; ++qt) {
      const long tiles = (queries + 64 * qt - 1) / (64 * qt);
      if (qt == 1 || tiles * cost[qt - 1] < least) {
        least = tiles * cost[qt - 1];
        c.qt = qt;
        c.tiles = (int)tiles;
      }
    }
  } else {
    c.qt = (int)max(1L, (queries + 15) / 16);
    c.tiles = 1;
  }
  const long want = kBlocks / max(others * c.tiles, 1L);
  const long most = max(1, chunks / kSliceChunks);
  // Up to 1024 keys are not cut for few queries: a block is through them in 8.5 us where slices and their meeting take 7.1, but the second launch costs the
  // caller 4 (one row, 1000 keys, 28 heads on 4).
  const int n = !c.many && !joined && chunks <= kUncut ? 1 : (int)max(1L, min(min(want, most), (long)kSlicesMax));
  c.split = (chunks + n - 1) / n;
  c.slices = (chunks + c.split - 1) / c.split;
  return c;
}
struct Plan { Cut own, prefix; };
Plan plan_of(const KvCache& c, const KvAttention& a) {
  const long group = a.heads / c.kv_heads;
  Plan p = {};
  p.own = cut(a.max_rows * group, max(1, (a.max_keys + 31) / 32), (long)c.kv_heads * a.seqs, a.prefix_len > 0);
  if (a.prefix_len > 0) p.prefix = cut(a.rows * group, (a.prefix_len + 31) / 32, c.kv_heads, true);
  return p;
}
// `parts`: heads of rows times slices
size_t part_bytes(const KvCache& c, size_t parts) { return (parts * c.head_dim * 4 + 255) / 256 * 256; }
size_t parts_bytes(const KvCache& c, size_t parts) { return part_bytes(c, parts) + parts * sizeof(float2); }

// Most parts that cut() can make of up to `heads` heads of rows, `queries` queries and `chunks` chunks, 0: they are never cut.  Where there are slices at
// all, `others` x tiles x slices are at most kBlocks, so that there are that many parts to a query of a tile, of which a tile has 192 at most.
size_t most_parts(size_t heads, long queries, int chunks, bool joined) {
  const size_t slices = queries <= 48 && !joined && chunks <= kUncut ? 1 : max(1, min(chunks / kSliceChunks, kSlicesMax));
  return slices == 1 ? 0 : min(heads * slices, (size_t)min(queries, 192L) * kBlocks);
}

template <int ES, int HD, bool PREFIX, bool DIRECT>
void launch_cut(const Args& a, const Cut& c, hipStream_t s) {
  const long blocks = (long)a.place.kv_heads * (PREFIX ? 1 : a.seqs) * c.slices * c.tiles;
  if (c.many) {
    if (c.qt == 1) kv_attention_many_kernel<ES, HD, 1, PREFIX, DIRECT><<<(unsigned)blocks, 256, 0, s>>>(a, c.tiles);
    else if (c.qt == 2) kv_attention_many_kernel<ES, HD, 2, PREFIX, DIRECT><<<(unsigned)blocks, 256, 0, s>>>(a, c.tiles);
    else kv_attention_many_kernel<ES, HD, 3, PREFIX, DIRECT><<<(unsigned)blocks, 256, 0, s>>>(a, c.tiles);
  } else {
    if (c.qt == 1) kv_attention_few_kernel<ES, HD, 1, PREFIX, DIRECT><<<(unsigned)blocks, 256, 0, s>>>(a);
    else if (c.qt == 2) kv_attention_few_kernel<ES, HD, 2, PREFIX, DIRECT><<<(unsigned)blocks, 256, 0, s>>>(a);
    else kv_attention_few_kernel<ES, HD, 3, PREFIX, DIRECT><<<(unsigned)blocks, 256, 0, s>>>(a);
  }
}

template <int ES, int HD, bool MANY>
void launch_both(const Args& a, const Plan& p, hipStream_t s) {
  const unsigned prefix = (unsigned)(a.place.kv_heads * p.prefix.slices * p.prefix.tiles), blocks = prefix + (unsigned)(a.place.kv_heads * a.seqs * p.own.slices);
  if (p.prefix.qt == 1) kv_attention_both_kernel<ES, HD, MANY, 1><<<blocks, 256, 0, s>>>(a, p.prefix.tiles, prefix);
  else if (p.prefix.qt == 2) kv_attention_both_kernel<ES, HD, MANY, 2><<<blocks, 256, 0, s>>>(a, p.prefix.tiles, prefix);
  else kv_attention_both_kernel<ES, HD, MANY, 3><<<blocks, 256, 0, s>>>(a, p.prefix.tiles, prefix);
}

template <int ES, int HD>
void launch(const KvCache& c, const KvAttention& k, const Plan& p, void* workspace, hipStream_t s) {
  Args a;
  a.q = k.q; a.q_ld = k.q_ld; a.q_head = k.q_head;
  a.out = k.out; a.out_ld = k.out_ld; a.out_head = k.out_head;
  a.rows = k.rows; a.heads = k.heads; a.group = k.heads / c.kv_heads;
  a.seqs = k.seqs; a.max_rows = k.max_rows; a.max_keys = k.max_keys; a.each = k.max_rows;
  a.table = k.table; a.lengths = k.lengths; a.starts = k.starts; a.table_ld = k.table_ld;
  a.prefix = k.prefix; a.prefix_len = k.prefix_len; a.causal = k.causal; a.scale = k.scale * 1.4426950408889634f;
  a.lag = kLag / a.scale;
  a.low = a.scale > 1.f ? -std::nextafter(FLT_MAX / a.scale, 0.f) : -FLT_MAX;
  a.data = c.data; a.scales = c.data + kv_code_bytes(c);
  a.place = {c.page == 32 ? 0 : c.page == 64 ? 1 : c.page == 128 ? 2 : 3, c.kv_heads};
  a.pages = c.pages;
  a.split = p.own.split; a.slices = p.own.slices; a.prefix_split = p.prefix.split; a.prefix_slices = p.prefix.slices;
  const int total = a.slices + a.prefix_slices;
  a.part = (float*)workspace;
  a.sums = (float2*)((char*)workspace + part_bytes(c, (size_t)k.rows * k.heads * total));
  if (total == 1) return launch_cut<ES, HD, false, true>(a, p.own, s);
  if (a.prefix_slices && !p.own.many && p.own.qt == 1) {
    if (p.prefix.many) launch_both<ES, HD, true>(a, p, s);
    else launch_both<ES, HD, false>(a, p, s);
  } else {
    if (a.prefix_slices) launch_cut<ES, HD, true, false>(a, p.prefix, s);
    launch_cut<ES, HD, false, false>(a, p.own, s);
  }
  const long queries = (long)a.max_rows * a.heads;
  if (total > 8) kv_attention_join_kernel<HD, 4><<<dim3((unsigned)queries, a.seqs), 256, 0, s>>>(a);
  else kv_attention_join_kernel<HD, 1><<<dim3((unsigned)((queries + 3) / 4), a.seqs), 256, 0, s>>>(a);
}

}  // namespace

// Fewer rows have fewer tiles and more slices of keys: there is room for whatever calls of as many rows, sequences and keys or fewer need.  (Rows that are of no
// sequence have parts too; with them it is what the call itself needs.)
size_t kv_attention_workspace(const KvCache& c, const KvAttention& a) {
  const Plan p = plan_of(c, a);
  const int total = p.own.slices + p.prefix.slices;
  const long group = a.heads / c.kv_heads;
  const size_t heads = (size_t)a.rows * a.heads, here = total == 1 ? 0 : heads * total;
  size_t parts = most_parts(heads, a.max_rows * group, max(1, (a.max_keys + 31) / 32), a.prefix_len > 0);
  if (a.prefix_len > 0) parts = max(parts, heads) + max(most_parts(heads, a.rows * group, (a.prefix_len + 31) / 32, true), heads);
  return parts_bytes(c, max(parts, here));
}

void launch_kv_attention(const KvCache& c, const KvAttention& a, void* workspace, hipStream_t s) {
  const Plan p = plan_of(c, a);
  if (c.e4m3) {
    if (c.head_dim == 64) launch<1, 64>(c, a, p, workspace, s);
    else launch<1, 128>(c, a, p, workspace, s);
  } else {
    if (c.head_dim == 64) launch<2, 64>(c, a, p, workspace, s);
    else launch<2, 128>(c, a, p, workspace, s);
  }
}

}  // namespace ec
