// Attention of a batch of sequences over a paged cache (k_kv.h), with a prefix that all of them share.
//
// out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale (q . k_j) - m),  m the largest of the exponents so far: one pass over the keys, with
// what was added up so far multiplied by exp(m_old - m_new) whenever m grows.  Per 32 keys (a chunk) and 16 rows of queries (a row of
// queries: one head of one row, the heads of a kv head's group next to each other):
//   S^T[keys x queries] = K . Q^T, softmax down the keys, O^T[components x queries] += V^T . P^T
// with the operands as they lie in the cache.  e4m3 keys are widened to bfloat16 with their power of two, exactly; values are widened
// without it, exactly, and the probability takes it, an exact product again, before its one rounding to bfloat16 (2^-9 of it at most).
// Scores, maxima, sums and outputs are float32.
//
// Keys are cut into slices of chunks, a block each; the slices' (m, sum, O) meet in a second launch, in their order.  The prefix' slices take
// the rows of all sequences at once, so that its keys are read once for all.  A query that sees no key gets zeros: m begins at the lowest
// float, below which no score but -inf lies, and a sum of 0 divides nothing.
#include <float.h>

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

// what a kernel knows of the call
struct Args {
  const bf16_t* q; size_t q_ld, q_head;
  bf16_t* out; size_t out_ld, out_head;
  int rows, heads, group, seqs, max_rows, max_keys, each;
  const int *table, *lengths, *starts;
  int width; size_t table_ld;
  const int* prefix; int prefix_len;
  bool causal;
  float scale;                       // with log2(e)
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

// One chunk as a lane holds it
template <int ES, int HD> struct Chunk {
  static constexpr int U = KvChunk<ES, HD>::kUnits, V = HD / 32 * ES;
  u32x4 k[2 * U], v[V];
  uint32_t ks[2];
  u32x2 vs;
  __device__ __forceinline__ void load(const Args& a, size_t chunk, int lane) {
    const u32x4* p = (const u32x4*)(a.data + chunk * KvChunk<ES, HD>::kBytes) + lane;
#pragma unroll
    for (int i = 0; i < 2 * U; ++i) k[i] = p[i * 64];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = p[(2 * U + i) * 64];
    const uint8_t* s = a.scales + chunk * 64;
    const int w = ((lane & 15) >> 2) * 8 + (lane & 3);
    if constexpr (ES == 1) {
      ks[0] = s[w];
      ks[1] = s[w + 4];
    }
    vs = *(const u32x2*)(s + 32 + (lane >> 4) * 8);
  }
};

}  // namespace

constexpr int kWaves = 4;

// A block's waves go through the chunks of its slice in turn, each with QT tiles of 16 queries, and meet in LDS.  PREFIX: the rows of the
// whole call over the prefix.  DIRECT: there is one slice, and the block writes the result.
template <int ES, int HD, int QT, bool PREFIX, bool DIRECT>
__global__ __launch_bounds__(256) void kv_attention_kernel(Args a, int tiles) {
  constexpr int HB = HD / 32, HT = HD / 16, U = KvChunk<ES, HD>::kUnits;
  typedef Chunk<ES, HD> C;
  extern __shared__ float4 lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = lane >> 4, col = lane & 15;
  unsigned id = blockIdx.x;
  const int kvh = id % a.place.kv_heads;
  id /= a.place.kv_heads;
  const int slices = PREFIX ? a.prefix_slices : a.slices, slice = id % slices;
  id /= slices;
  const int tile = id % tiles, b = id / tiles;
  const Seq s = PREFIX ? Seq{0, a.rows, a.prefix_len} : seq_of(a, b);
  const int first = tile * 16 * QT, queries = s.n * a.group;    // of this sequence and kv head
  if (first >= queries) return;
  const int* table = PREFIX ? a.prefix : a.table + (size_t)b * a.table_ld;
  const int split = PREFIX ? a.prefix_split : a.split;
  const bool causal = !PREFIX && a.causal;
  const int c_lo = slice * split;
  if (slice > 0 && c_lo * 32 >= s.keys) return;
  // keys that the tile's first and last rows see
  const int last_row = (min(first + 16 * QT, queries) - 1) / a.group;
  const int seen_first = causal ? s.keys - s.n + 1 + first / a.group : s.keys;
  const int seen_last = causal ? s.keys - s.n + 1 + last_row : s.keys;
  const int c_hi = min(c_lo + split, (max(seen_last, 0) + 31) >> 5);

  bf16x8 qf[QT][HB];
  int seen[QT], row[QT], head[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int m = min(first + t * 16 + col, queries - 1), r = m / a.group;
    row[t] = s.row0 + r;
    head[t] = kvh * a.group + (m - r * a.group);
    seen[t] = causal ? s.keys - s.n + 1 + r : s.keys;
    const bf16_t* p = a.q + (size_t)row[t] * a.q_ld + (size_t)head[t] * a.q_head + grp * (HD / 4);
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) qf[t][hb] = as_bf16x8(*(const u32x4*)(p + hb * 8));
  }
  f32x4 acc[QT][HT];
  float m_run[QT], l_run[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_run[t] = -FLT_MAX;
    l_run[t] = 0.f;
#pragma unroll
    for (int h = 0; h < HT; ++h) acc[t][h] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  const int mine = c_lo + wave < c_hi ? (c_hi - c_lo - wave + kWaves - 1) / kWaves : 0;   // chunks of this wave
  auto chunk_no = [&](int i) { return c_lo + wave + kWaves * i; };
  int pids = 0;      // lane i: the page of the wave's i-th chunk (of the present 64)
  auto page_of = [&](int i) {
    if ((i & 63) == 0) pids = table[min(chunk_no(i + lane), chunk_no(mine - 1)) >> a.place.shift];
    return __builtin_amdgcn_readlane(pids, i & 63);
  };
  C cur, next;
  int page = 0, page_next = 0;
  auto fetch = [&](C& c, int i) {
    const int pg = page_of(i), no = chunk_no(i);
    const bool there = pg >= 0 && pg < a.pages;
    c.load(a, ((((size_t)(there ? pg : 0) * a.place.kv_heads + kvh) << a.place.shift) + (no & ((1 << a.place.shift) - 1))), lane);
    return there ? 1 : 0;
  };
  if (mine > 0) page = fetch(cur, 0);
  for (int i = 0; i < mine; ++i) {
    if (i + 1 < mine) page_next = fetch(next, i + 1);
    const int key0 = chunk_no(i) * 32, over = key0 + 32;
    // ---- scores
    f32x4 sc[QT][2];
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2) {
      bf16x8 kf[HB];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const u32x4 k = cur.k[t2 * U + u];
        if constexpr (ES == 1) {
          const float f = power_of(cur.ks[t2]);
          kf[2 * u] = widen8(k[0], k[1], f);
          kf[2 * u + 1] = widen8(k[2], k[3], f);
        } else {
          kf[u] = as_bf16x8(k);
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        sc[t][t2] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) sc[t][t2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[hb], qf[t][hb], sc[t][t2], 0, 0, 0);
      }
    }
    const int k0 = key0 + grp * 8;
    const bool masked = over > min(seen_first, s.keys) || !page;
    if (masked) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (k0 + e >= seen[t] || !page) sc[t][e >> 2][e & 3] = -INFINITY;
      // what lies behind the last key may be anything
      const int live = page ? min(max(s.keys - k0, 0), 8) : 0;
#pragma unroll
      for (int h = 0; h < C::V; ++h) {
        if constexpr (ES == 1) {
          const uint64_t keep = live == 8 ? ~0ull : (1ull << (8 * live)) - 1;
          cur.v[h] &= (u32x4){(uint32_t)keep, (uint32_t)(keep >> 32), (uint32_t)keep, (uint32_t)(keep >> 32)};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) cur.v[h][e] &= (2 * e < live ? 0xffffu : 0u) | (2 * e + 1 < live ? 0xffff0000u : 0u);
        }
      }
    }
    // ---- softmax
    float vs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) vs[e] = power_of((cur.vs[e >> 2] >> (8 * (e & 3))) & 255u);
    bf16x8 pf[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float mx = max_of_swap32(max_of_swap16(max_of_8(sc[t][0], sc[t][1]))) * a.scale;
      if (__builtin_amdgcn_ballot_w64(mx > m_run[t]) != 0) {
        const float m_new = max_of(m_run[t], mx), alpha = __builtin_amdgcn_exp2f(m_run[t] - m_new);
        m_run[t] = m_new;
        l_run[t] *= alpha;
#pragma unroll
        for (int h = 0; h < HT; ++h) acc[t][h] *= alpha;
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(sc[t][e >> 2][e & 3], a.scale, -m_run[t]));
        l_run[t] += p[e];
        p[e] *= vs[e];
      }
      if (masked)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (k0 + e >= seen[t] || !page) p[e] = 0.f;
      pf[t] = u4_as_bf16x8(make_uint4(pack2_bf16(p[0], p[1]), pack2_bf16(p[2], p[3]), pack2_bf16(p[4], p[5]), pack2_bf16(p[6], p[7])));
    }
    // ---- values
#pragma unroll
    for (int h = 0; h < HT; ++h) {
      bf16x8 vf;
      if constexpr (ES == 1) vf = h & 1 ? widen8(cur.v[h >> 1][2], cur.v[h >> 1][3], 1.f) : widen8(cur.v[h >> 1][0], cur.v[h >> 1][1], 1.f);
      else vf = as_bf16x8(cur.v[h]);
#pragma unroll
      for (int t = 0; t < QT; ++t) acc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t], acc[t][h], 0, 0, 0);
    }
    cur = next;
    page = page_next;
  }

  // ---- the waves' parts meet: (m, sum, O) of each, in their order
  constexpr int SLOT = QT * (HT * 64 + 32);   // float4
  float4* slot = lds + (size_t)wave * SLOT;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float l = l_run[t];
    l += other_row(l);
    l += other_half(l);
    ((float2*)(slot + QT * HT * 64))[t * 64 + lane] = make_float2(m_run[t], l);
#pragma unroll
    for (int h = 0; h < HT; ++h) slot[(t * HT + h) * 64 + lane] = make_float4(acc[t][h][0], acc[t][h][1], acc[t][h][2], acc[t][h][3]);
  }
  __syncthreads();
  const int total = a.prefix_slices + a.slices, at_slice = PREFIX ? slice : a.prefix_slices + slice;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float m_all = -FLT_MAX, l_all = 0.f, f[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 ml = ((const float2*)(lds + (size_t)w * SLOT + QT * HT * 64))[t * 64 + lane];
      f[w] = ml.x;
      m_all = fmaxf(m_all, ml.x);
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 ml = ((const float2*)(lds + (size_t)w * SLOT + QT * HT * 64))[t * 64 + lane];
      f[w] = __builtin_amdgcn_exp2f(f[w] - m_all);
      l_all += ml.y * f[w];
    }
    if (first + t * 16 + col >= queries) continue;
    const size_t at = ((size_t)row[t] * a.heads + head[t]) * total + at_slice;
    if (!DIRECT && wave == 0 && grp == 0) a.sums[at] = make_float2(m_all, l_all);
    for (int p = wave; p < HT / 2; p += kWaves) {
      float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float4 x = lds[(size_t)w * SLOT + (t * HT + 2 * p) * 64 + lane], y = lds[(size_t)w * SLOT + (t * HT + 2 * p + 1) * 64 + lane];
        o[0] += x.x * f[w]; o[1] += x.y * f[w]; o[2] += x.z * f[w]; o[3] += x.w * f[w];
        o[4] += y.x * f[w]; o[5] += y.y * f[w]; o[6] += y.z * f[w]; o[7] += y.w * f[w];
      }
      if constexpr (DIRECT) {
        const float inv = l_all == 0.f ? 0.f : 1.0f / l_all;
        *(uint4*)(a.out + (size_t)row[t] * a.out_ld + (size_t)head[t] * a.out_head + p * 32 + grp * 8) =
            make_uint4(pack2_bf16(o[0] * inv, o[1] * inv), pack2_bf16(o[2] * inv, o[3] * inv), pack2_bf16(o[4] * inv, o[5] * inv),
                       pack2_bf16(o[6] * inv, o[7] * inv));
      } else {
        float4* to = (float4*)(a.part + at * HD + p * 32 + grp * 8);
        to[0] = make_float4(o[0], o[1], o[2], o[3]);
        to[1] = make_float4(o[4], o[5], o[6], o[7]);
      }
    }
  }
}

// The slices of a row of queries meet: a wave each, a lane HD/64 components.
template <int HD>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(Args a) {
  constexpr int N = HD / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Seq s = seq_of(a, blockIdx.y);
  const int i = blockIdx.x * 4 + wave, r = i / a.heads, head = i - r * a.heads;
  if (r >= s.n) return;
  const int total = a.prefix_slices + a.slices;
  const int own = a.slices ? max(1, (((s.keys + 31) >> 5) + a.split - 1) / a.split) : 0;
  const size_t at = ((size_t)(s.row0 + r) * a.heads + head) * total;
  float m = -FLT_MAX, l = 0.f, o[N] = {};
  for (int z = 0; z < a.prefix_slices + own; ++z) m = fmaxf(m, a.sums[at + z].x);
  for (int z = 0; z < a.prefix_slices + own; ++z) {
    const float2 ml = a.sums[at + z];
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    l += ml.y * f;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] += a.part[(at + z) * HD + lane * N + e] * f;
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  bf16_t* to = a.out + (size_t)(s.row0 + r) * a.out_ld + (size_t)head * a.out_head + lane * N;
#pragma unroll
  for (int e = 0; e < N; ++e) to[e] = f32_to_bf16(o[e] * inv);
}

namespace {

// how the keys are cut
struct Plan { int split, slices, prefix_split, prefix_slices; };
int cut(int chunks, long others, int* split) {
  const long want = max(1L, 1024 / max(others, 1L));                       // blocks that fill the compute units
  const int most = max(1, chunks / 8);                                     // two chunks to a wave at least
  const int n = (int)min(want, (long)most);
  *split = (chunks + n - 1) / n;
  return (chunks + *split - 1) / *split;
}
Plan plan_of(const KvCache& c, const KvAttention& a) {
  const int group = a.heads / c.kv_heads;
  const long tiles = ((long)a.max_rows * group + 15) / 16, all = ((long)a.rows * group + 15) / 16;
  Plan p = {};
  p.slices = cut(max(1, (a.max_keys + 31) / 32), (long)c.kv_heads * a.seqs * tiles, &p.split);
  if (a.prefix_len > 0) p.prefix_slices = cut((a.prefix_len + 31) / 32, c.kv_heads * all, &p.prefix_split);
  return p;
}
size_t part_bytes(const KvCache& c, const KvAttention& a, int slices) {
  return ((size_t)a.rows * a.heads * slices * c.head_dim * 4 + 255) / 256 * 256;
}

template <int ES, int HD>
void launch(const KvCache& c, const KvAttention& k, const Plan& p, void* workspace, hipStream_t s) {
  Args a;
  a.q = k.q; a.q_ld = k.q_ld; a.q_head = k.q_head;
  a.out = k.out; a.out_ld = k.out_ld; a.out_head = k.out_head;
  a.rows = k.rows; a.heads = k.heads; a.group = k.heads / c.kv_heads;
  a.seqs = k.seqs; a.max_rows = k.max_rows; a.max_keys = k.max_keys; a.each = k.max_rows;
  a.table = k.table; a.lengths = k.lengths; a.starts = k.starts; a.width = k.width; a.table_ld = k.table_ld;
  a.prefix = k.prefix; a.prefix_len = k.prefix_len; a.causal = k.causal; a.scale = k.scale * 1.4426950408889634f;
  a.data = c.data; a.scales = c.data + kv_code_bytes(c);
  a.place = {c.page == 32 ? 0 : c.page == 64 ? 1 : c.page == 128 ? 2 : 3, c.kv_heads};
  a.pages = c.pages;
  a.split = p.split; a.slices = p.slices; a.prefix_split = p.prefix_split; a.prefix_slices = p.prefix_slices;
  const int total = p.slices + p.prefix_slices;
  a.part = (float*)workspace;
  a.sums = (float2*)((char*)workspace + part_bytes(c, k, total));
  constexpr int QT = 1;
  constexpr size_t lds = (size_t)kWaves * QT * (HD / 16 * 64 + 32) * 16;
  const long tiles = ((long)a.max_rows * a.group + 16 * QT - 1) / (16 * QT);
  if (total == 1) {
    kv_attention_kernel<ES, HD, QT, false, true><<<(unsigned)(c.kv_heads * a.slices * tiles * a.seqs), 256, lds, s>>>(a, (int)tiles);
    return;
  }
  if (p.prefix_slices) {
    const long all = ((long)a.rows * a.group + 16 * QT - 1) / (16 * QT);
    kv_attention_kernel<ES, HD, QT, true, false><<<(unsigned)(c.kv_heads * a.prefix_slices * all), 256, lds, s>>>(a, (int)all);
  }
  kv_attention_kernel<ES, HD, QT, false, false><<<(unsigned)(c.kv_heads * a.slices * tiles * a.seqs), 256, lds, s>>>(a, (int)tiles);
  kv_attention_join_kernel<HD><<<dim3((unsigned)(((long)a.max_rows * a.heads + 3) / 4), a.seqs), 256, 0, s>>>(a);
}

}  // namespace

size_t kv_attention_workspace(const KvCache& c, const KvAttention& a) {
  const Plan p = plan_of(c, a);
  const int total = p.slices + p.prefix_slices;
  return total == 1 ? 0 : part_bytes(c, a, total) + (size_t)a.rows * a.heads * total * 8;
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
