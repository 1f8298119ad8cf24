// Tokens' keys and values into a paged cache (k_kv.h), and back.
//
// To e4m3 (1 sign, 4 exponent bits with bias 7, 3 mantissa bits): each token's head is divided by the least power of two that leaves its
// largest magnitude at 448, the largest code, or below, and rounded to the nearest code, ties to the even one.  A floating code keeps its
// relative step down to 2^-15 of the largest magnitude whatever the scale is, so that a scale that is not a power of two, or more scales
// to a head, would gain nothing above that; and a power of two multiplies exactly.
#include "k_kv.h"

namespace ec {

namespace {

// s of a head whose largest magnitude has the bits `top`: 448 = 1.75 2^8.  From 248 2^120 on (0x7f780000) it would be rounded to 256 2^120 = 2^128,
// which is no float32: NaN, as what is not finite.
__device__ __forceinline__ uint32_t kv_scale(uint32_t top) {
  if (top >= 0x7f780000u) return 255;
  const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u);
  return (uint32_t)max(e, 1);
}

// N values as they lie in memory, and as float32
template <typename T, int N> struct Loaded {
  uint4 w[N * sizeof(T) / 16];
  __device__ __forceinline__ void load(const T* p, bool wide) {
    if (wide) {
#pragma unroll
      for (int j = 0; j < (int)(N * sizeof(T) / 16); ++j) w[j] = ((const uint4*)p)[j];
    } else {
      union { T v[N]; uint4 w[N * sizeof(T) / 16]; } c;
#pragma unroll
      for (int j = 0; j < N; ++j) c.v[j] = p[j];
#pragma unroll
      for (int j = 0; j < (int)(N * sizeof(T) / 16); ++j) w[j] = c.w[j];
    }
  }
  __device__ __forceinline__ void values(float (&v)[N]) const {
    const uint32_t* u = (const uint32_t*)w;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (sizeof(T) == 4) v[j] = __uint_as_float(u[j]);
      else v[j] = __uint_as_float(j & 1 ? u[j >> 1] & 0xffff0000u : u[j >> 1] << 16);
    }
  }
};

__device__ __forceinline__ uint32_t codes4(const float* v, float f) {
  int c = 0;
  c = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * f, v[1] * f, c, false);
  c = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * f, v[3] * f, c, true);
  return (uint32_t)c;
}

// A lane's N components of a token's head as they are stored, in words of 4 bytes; returns the head's scale byte, found by its HD/N lanes
// together.  bad: what a head that is not finite is filled with
template <int ES, int N, int HD>
__device__ __forceinline__ uint32_t stored(float (&v)[N], uint32_t (&w)[N * ES / 4], uint32_t bad) {
  if constexpr (ES == 2) {
    // (a value that is rounded to an infinity is one)
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = bf16_to_f32(f32_to_bf16(v[j]));
  }
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, (uint32_t)dpp_i<0xB1>((int)top));
  top = max(top, (uint32_t)dpp_i<0x4E>((int)top));
  if constexpr (HD / N >= 8) top = max(top, (uint32_t)dpp_i<0x141>((int)top));
  if constexpr (HD / N >= 16) top = max(top, (uint32_t)dpp_i<0x140>((int)top));
  const uint32_t s = ES == 1 ? kv_scale(top) : top >= 0x7f800000u ? 255u : 127u;
  if constexpr (ES == 1) {
    const float f = __uint_as_float((254 - min(s, 253u)) << 23);   // (s goes from 1 to 247, or is 255)
#pragma unroll
    for (int j = 0; j < N / 4; ++j) w[j] = s == 255 ? bad : codes4(v + 4 * j, f);
  } else {
#pragma unroll
    for (int j = 0; j < N / 2; ++j) w[j] = s == 255 ? bad : (__float_as_uint(v[2 * j]) >> 16) | (__float_as_uint(v[2 * j + 1]) & 0xffff0000u);
  }
  return s;
}

// N stored components as float32
template <int ES, int N>
__device__ __forceinline__ void values_of(const uint32_t (&w)[N * ES / 4], uint32_t s, float (&v)[N]) {
  if constexpr (ES == 1) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const float f = __uint_as_float(s == 255 ? 0x7fc00000u : s << 23);
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
      const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), y = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
      v[4 * j] = x[0] * f; v[4 * j + 1] = x[1] * f; v[4 * j + 2] = y[0] * f; v[4 * j + 3] = y[1] * f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      v[2 * j] = __uint_as_float(s == 255 ? 0x7fc00000u : w[j] << 16);
      v[2 * j + 1] = __uint_as_float(s == 255 ? 0x7fc00000u : w[j] & 0xffff0000u);
    }
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_values(T* p, bool wide, const float (&v)[N]) {
  if (!wide) {
#pragma unroll
    for (int j = 0; j < N; ++j) store_f32(p + j, v[j]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < N / 4; ++j) ((float4*)p)[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < N / 8; ++j)
      ((uint4*)p)[j] = make_uint4(pack2_bf16(v[8 * j], v[8 * j + 1]), pack2_bf16(v[8 * j + 2], v[8 * j + 3]),
                                  pack2_bf16(v[8 * j + 4], v[8 * j + 5]), pack2_bf16(v[8 * j + 6], v[8 * j + 7]));
  }
}

// 8 x 8 elements: row r's words -> column c's words
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&o)[4]) {
  const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05010400), y = __builtin_amdgcn_perm(b, a, 0x07030602);
  const uint32_t z = __builtin_amdgcn_perm(d, c, 0x05010400), w = __builtin_amdgcn_perm(d, c, 0x07030602);
  o[0] = __builtin_amdgcn_perm(z, x, 0x05040100); o[1] = __builtin_amdgcn_perm(z, x, 0x07060302);
  o[2] = __builtin_amdgcn_perm(w, y, 0x05040100); o[3] = __builtin_amdgcn_perm(w, y, 0x07060302);
}
template <int ES> __device__ __forceinline__ void transpose8(const uint32_t (&in)[8][2 * ES], uint32_t (&out)[8][2 * ES]) {
  if constexpr (ES == 1) {
#pragma unroll
    for (int half = 0; half < 2; ++half)        // columns 4 half .. 4 half + 3
#pragma unroll
      for (int part = 0; part < 2; ++part) {    // of rows 4 part ..
        uint32_t o[4];
        transpose4(in[4 * part][half], in[4 * part + 1][half], in[4 * part + 2][half], in[4 * part + 3][half], o);
#pragma unroll
        for (int c = 0; c < 4; ++c) out[4 * half + c][part] = o[c];
      }
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        out[2 * c][r] = __builtin_amdgcn_perm(in[2 * r + 1][c], in[2 * r][c], 0x05040100);
        out[2 * c + 1][r] = __builtin_amdgcn_perm(in[2 * r + 1][c], in[2 * r][c], 0x07060302);
      }
  }
}

}  // namespace

struct KvRows {
  const void *k, *v;
  size_t k_ld, k_head, v_ld, v_head;
  int rows, total;
  const int* slots;
  uint8_t *data, *scales;
  KvPlace place;
  bool wide;
};

// The rows of a block, with 7 on both sides: where they go, and which stretches of 8 rows are 8 neighbouring slots from a multiple of 8 on.
// In the cache the values of such a run are 8 x 8 blocks of elements that lie together, which a lane turns in its registers; the others go
// element by element.  A run belongs to the block that its first row is in.
template <int ROWS> struct Tile {
  static constexpr int SIDE = 7, ALL = ROWS + 2 * SIDE;
  int slot[ALL];          // -1: not in the cache, or (written) a later row has it
  int first[ROWS / 8];    // the runs' first rows
  int runs;
  bool there;             // all of the block's rows have a slot
  unsigned long long single;   // the block's rows that are in no run and have a slot, a bit each
  unsigned long long have[2], eight[2], linked[2];
  int low, high;          // written: of the rows' slots
  int row_of[2048];       // written: by slot % 2048, 1 + the row (of ALL) with it, 0: none, -1: several
};

// WRITE: of rows that name the same slot the last one is stored.  The rows behind the block's are gone through: few of them are in the block's slots'
// range, and of these one place of a table says whether they are any of them.
template <int ROWS, bool WRITE>
__device__ __forceinline__ void find_runs(const KvRows& a, int row0, Tile<ROWS>& t) {
  typedef Tile<ROWS> Tl;
  static_assert(ROWS <= 64 && Tl::ALL <= 128, "a bit for each row, a thread for each");
  const int i = threadIdx.x, r = row0 - Tl::SIDE + i;
  int s = -1;
  if (i < Tl::ALL) {
    s = r >= 0 && r < a.rows ? a.slots[r] : -1;
    s = s >= 0 && s < a.total ? s : -1;
    t.slot[i] = s;
  }
  if constexpr (WRITE) {
#pragma unroll
    for (int k = 0; k < 8; ++k) t.row_of[i + 256 * k] = 0;
    if (i == 0) { t.low = INT32_MAX; t.high = -1; }
    __syncthreads();
    if (s >= 0) {
      if (atomicCAS(&t.row_of[s & 2047], 0, i + 1) != 0) t.row_of[s & 2047] = -1;
      atomicMin(&t.low, s);
      atomicMax(&t.high, s);
    }
    __syncthreads();
    const int low = t.low, range = t.high - low, before = row0 - Tl::SIDE;
    auto compare = [&](int later, int slot) {
      const int r = t.row_of[slot & 2047];
      if (r > 0) {
        if (before + r - 1 < later && t.slot[r - 1] == slot) t.slot[r - 1] = -1;
      } else if (r < 0) {
        for (int j = 0; j < Tl::ALL && before + j < later; ++j)
          if (t.slot[j] == slot) t.slot[j] = -1;
      }
    };
    auto look = [&](int n, int slot) {
      if (slot >= 0 && (unsigned)(slot - low) <= (unsigned)range) compare(n, slot);
    };
    if (range >= 0) {
      // (pieces of 4 from the first multiple of 16 bytes on, 16 slots of a thread on their way at a time)
      constexpr int MANY = 4;
      const int from = max(before, 0), to = a.rows, lead = (int)(-((intptr_t)(a.slots + from) >> 2) & 3), even = min(from + lead, to);
      const int pieces = (to - even) >> 2;
      for (int p = i; p < pieces; p += 256 * MANY) {
        int4 x[MANY];
#pragma unroll
        for (int k = 0; k < MANY; ++k) x[k] = p + 256 * k < pieces ? ((const int4*)(a.slots + even))[p + 256 * k] : make_int4(-1, -1, -1, -1);
#pragma unroll
        for (int k = 0; k < MANY; ++k) {
          const int n = even + 4 * (p + 256 * k);
          look(n, x[k].x); look(n + 1, x[k].y); look(n + 2, x[k].z); look(n + 3, x[k].w);
        }
      }
      if (i < even - from) look(from + i, a.slots[from + i]);
      const int tail = even + 4 * pieces;
      if (i < to - tail) look(tail + i, a.slots[tail + i]);
    }
  }
  // a bit for each row: has a slot; has a multiple of 8; the row behind it has the slot behind it
  __syncthreads();
  if (i < 128) {
    const int at = i < Tl::ALL ? t.slot[i] : -1, next = i + 1 < Tl::ALL ? t.slot[i + 1] : -1;
    const unsigned long long have = __ballot(at >= 0), eight = __ballot(at >= 0 && (at & 7) == 0), linked = __ballot(at >= 0 && next == at + 1);
    if ((i & 63) == 0) { t.have[i >> 6] = have; t.eight[i >> 6] = eight; t.linked[i >> 6] = linked; }
  }
  __syncthreads();
  if (i < 64) {
    typedef unsigned __int128 Bits;
    auto bits = [](const unsigned long long (&w)[2]) { return (Bits)w[1] << 64 | w[0]; };
    const Bits have = bits(t.have), one = bits(t.linked), two = one & one >> 1, four = two & two >> 2;
    const Bits run = bits(t.eight) & four & two >> 4 & one >> 6;
    Bits in_run = run | run << 1;
    in_run |= in_run << 2;
    in_run |= in_run << 4;
    constexpr unsigned long long BLOCK = ~0ull >> (64 - ROWS);
    const unsigned long long runs = (unsigned long long)(run >> Tl::SIDE) & BLOCK;
    if (i < ROWS && ((runs >> i) & 1)) t.first[__popcll(runs & ((1ull << i) - 1))] = i;
    if (i == 0) {
      t.runs = __popcll(runs);
      t.single = (unsigned long long)((have & ~in_run) >> Tl::SIDE) & BLOCK;
      t.there = ((unsigned long long)(have >> Tl::SIDE) & BLOCK) == BLOCK;
    }
  }
  __syncthreads();
}

template <int HD> constexpr int kTileRows = 32 * (128 / HD);   // 64 lanes, 8 rows x 8 components each

// A wave takes the rows of a tile (SPREAD: a part of them) and goes through every (4 gridDim.y)-th head.  What bounds it is bytes: each is read and
// written once, in pieces of 16 bytes and more but for the values of rows in no run.  24576 rows of 32 heads of 128 from bfloat16 to e4m3 take 163 us in
// turn with their reading (111), 604 MB each way; 34 rows here and there 8.8 us, a chain of slots, table and data (read: 5.2).
template <typename T, int ES, int HD, bool SPREAD>
__global__ __launch_bounds__(256) void kv_write_kernel(KvRows a) {
  constexpr int ROWS = kTileRows<HD>, LK = HD / 16, LV = HD / 8;   // lanes of a row: keys, values
  constexpr uint32_t kNaN = ES == 1 ? 0x7f7f7f7fu : 0x7fc07fc0u;
  typedef KvChunk<ES, HD> L;
  __shared__ Tile<ROWS> t;
  const int row0 = blockIdx.x * ROWS, lane = threadIdx.x & 63;
  find_runs<ROWS, true>(a, row0, t);
  const int run = lane / LV, cv = lane % LV * 8;
  const bool has_run = run < t.runs;
  const int first = has_run ? t.first[run] : 0, run_slot = has_run ? t.slot[Tile<ROWS>::SIDE + first] : 0;
  for (int h = blockIdx.y * 4 + (threadIdx.x >> 6); h < a.place.kv_heads; h += gridDim.y * 4) {
    // values of the runs: 8 tokens x 8 components
    if (has_run && (!SPREAD || blockIdx.z == 0)) {
      const T* p = (const T*)a.v + (size_t)(row0 + first) * a.v_ld + (size_t)h * a.v_head + cv;
      Loaded<T, 8> x[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) x[r].load(p + (size_t)r * a.v_ld, a.wide);
      uint32_t w[8][2 * ES], o[8][2 * ES], s[2] = {0, 0};
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        float v[8];
        x[r].values(v);
        s[r >> 2] |= stored<ES, 8, HD>(v, w[r], 0) << (8 * (r & 3));
      }
      transpose8<ES>(w, o);
      const size_t chunk = a.place.chunk(run_slot, h);
      uint8_t* to = a.data + chunk * L::kBytes;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (ES == 1) {
          *(uint4*)(to + L::value_at(run_slot & 31, cv + r)) = make_uint4(o[r][0], o[r][1], o[r + 4][0], o[r + 4][1]);
        } else {
          *(uint4*)(to + L::value_at(run_slot & 31, cv + r)) = make_uint4(o[r][0], o[r][1], o[r][2], o[r][3]);
          *(uint4*)(to + L::value_at(run_slot & 31, cv + 4 + r)) = make_uint4(o[r + 4][0], o[r + 4][1], o[r + 4][2], o[r + 4][3]);
        }
      }
      if (cv == 0) *(uint2*)(a.scales + chunk * 64 + 32 + (run_slot & 31)) = make_uint2(s[0], s[1]);
    }
    // keys, 16 components of a token at a time
    constexpr int TURNS = ROWS * LK / 64, EACH = SPREAD ? 1 : TURNS;
    const int j0 = (SPREAD ? blockIdx.z * (64 / LK) : 0) + lane / LK, c0 = lane % LK * 16;
    Loaded<T, 16> x[EACH];
    int slot[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int j = j0 + i * (64 / LK);
      slot[i] = t.slot[Tile<ROWS>::SIDE + j];
      if (slot[i] >= 0) x[i].load((const T*)a.k + (size_t)(row0 + j) * a.k_ld + (size_t)h * a.k_head + c0, a.wide);
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (slot[i] >= 0) {
        const int w = slot[i] & 31;
        const size_t chunk = a.place.chunk(slot[i], h);
        uint8_t* to = a.data + chunk * L::kBytes;
        float v[16];
        uint32_t words[4 * ES];
        x[i].values(v);
        const uint32_t s = stored<ES, 16, HD>(v, words, kNaN);
#pragma unroll
        for (int n = 0; n < ES; ++n)
          *(uint4*)(to + L::key_at(w, c0 + n * 8)) = make_uint4(words[4 * n], words[4 * n + 1], words[4 * n + 2], words[4 * n + 3]);
        if (c0 == 0) a.scales[chunk * 64 + w] = (uint8_t)s;
      }
    }
    // values of the rows in no run
    if (t.single == 0) continue;
    for (int i = 0; i < EACH; ++i) {
      const int j = j0 + i * (64 / LK), at = t.slot[Tile<ROWS>::SIDE + j], w = at & 31;
      if ((t.single >> j) & 1) {
        const size_t chunk = a.place.chunk(at, h);
        uint8_t* to = a.data + chunk * L::kBytes;
        Loaded<T, 16> y;
        y.load((const T*)a.v + (size_t)(row0 + j) * a.v_ld + (size_t)h * a.v_head + c0, a.wide);
        float v[16];
        uint32_t words[4 * ES];
        y.values(v);
        const uint32_t s = stored<ES, 16, HD>(v, words, 0);
#pragma unroll
        for (int n = 0; n < 16; ++n) {
          if constexpr (ES == 1) to[L::value_at(w, c0 + n)] = (uint8_t)(words[n >> 2] >> (8 * (n & 3)));
          else *(uint16_t*)(to + L::value_at(w, c0 + n)) = (uint16_t)(words[n >> 1] >> (16 * (n & 1)));
        }
        if (c0 == 0) a.scales[chunk * 64 + 32 + w] = (uint8_t)s;
      }
    }
  }
}

template <typename T, int ES, int HD, bool SPREAD>
__global__ __launch_bounds__(256) void kv_read_kernel(KvRows a) {
  constexpr int ROWS = kTileRows<HD>, LK = HD / 16, LV = HD / 8;
  typedef KvChunk<ES, HD> L;
  __shared__ Tile<ROWS> t;
  const int row0 = blockIdx.x * ROWS, lane = threadIdx.x & 63;
  find_runs<ROWS, false>(a, row0, t);
  const int run = lane / LV, cv = lane % LV * 8;
  const bool has_run = run < t.runs;
  const int first = has_run ? t.first[run] : 0, run_slot = has_run ? t.slot[Tile<ROWS>::SIDE + first] : 0;
  for (int h = blockIdx.y * 4 + (threadIdx.x >> 6); h < a.place.kv_heads; h += gridDim.y * 4) {
    if (has_run && (!SPREAD || blockIdx.z == 0)) {
      const size_t chunk = a.place.chunk(run_slot, h);
      const uint8_t* from = a.data + chunk * L::kBytes;
      uint32_t w[8][2 * ES], o[8][2 * ES];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint4 x = *(const uint4*)(from + L::value_at(run_slot & 31, cv + r));
        if constexpr (ES == 1) {
          o[r][0] = x.x; o[r][1] = x.y; o[r + 4][0] = x.z; o[r + 4][1] = x.w;
        } else {
          const uint4 y = *(const uint4*)(from + L::value_at(run_slot & 31, cv + 4 + r));
          o[r][0] = x.x; o[r][1] = x.y; o[r][2] = x.z; o[r][3] = x.w;
          o[r + 4][0] = y.x; o[r + 4][1] = y.y; o[r + 4][2] = y.z; o[r + 4][3] = y.w;
        }
      }
      const uint2 s = *(const uint2*)(a.scales + chunk * 64 + 32 + (run_slot & 31));
      transpose8<ES>(o, w);
      T* p = (T*)a.v + (size_t)(row0 + first) * a.v_ld + (size_t)h * a.v_head + cv;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        float v[8];
        values_of<ES>(w[r], ((r < 4 ? s.x : s.y) >> (8 * (r & 3))) & 255u, v);
        store_values(p + (size_t)r * a.v_ld, a.wide, v);
      }
    }
    constexpr int TURNS = ROWS * LK / 64, EACH = SPREAD ? 1 : TURNS;
    const int j0 = (SPREAD ? blockIdx.z * (64 / LK) : 0) + lane / LK, c0 = lane % LK * 16;
    uint32_t kw[EACH][4 * ES], ks[EACH];
    int slot[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      slot[i] = t.slot[Tile<ROWS>::SIDE + j0 + i * (64 / LK)];
      if (slot[i] >= 0) {
        const size_t chunk = a.place.chunk(slot[i], h);
        const uint8_t* from = a.data + chunk * L::kBytes;
#pragma unroll
        for (int n = 0; n < ES; ++n) {
          const uint4 u = *(const uint4*)(from + L::key_at(slot[i] & 31, c0 + n * 8));
          kw[i][4 * n] = u.x; kw[i][4 * n + 1] = u.y; kw[i][4 * n + 2] = u.z; kw[i][4 * n + 3] = u.w;
        }
        ks[i] = a.scales[chunk * 64 + (slot[i] & 31)];
      }
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int j = j0 + i * (64 / LK);
      if (row0 + j < a.rows) {
        float x[16] = {};
        if (slot[i] >= 0) values_of<ES>(kw[i], ks[i], x);
        store_values((T*)a.k + (size_t)(row0 + j) * a.k_ld + (size_t)h * a.k_head + c0, a.wide, x);
      }
    }
    // values of the rows in no run, and of those that are not there
    if (t.single == 0 && t.there) continue;
    for (int i = 0; i < EACH; ++i) {
      const int j = j0 + i * (64 / LK), at = t.slot[Tile<ROWS>::SIDE + j];
      if (row0 + j < a.rows && (at < 0 || ((t.single >> j) & 1))) {
        float x[16] = {};
        if (at >= 0) {
          const size_t chunk = a.place.chunk(at, h);
          const uint8_t* from = a.data + chunk * L::kBytes;
          const uint32_t s = a.scales[chunk * 64 + 32 + (at & 31)];
          uint32_t words[4 * ES] = {};
#pragma unroll
          for (int n = 0; n < 16; ++n) {
            if constexpr (ES == 1) words[n >> 2] |= (uint32_t)from[L::value_at(at & 31, c0 + n)] << (8 * (n & 3));
            else words[n >> 1] |= (uint32_t) * (const uint16_t*)(from + L::value_at(at & 31, c0 + n)) << (16 * (n & 1));
          }
          values_of<ES>(words, s, x);
        }
        store_values((T*)a.v + (size_t)(row0 + j) * a.v_ld + (size_t)h * a.v_head + c0, a.wide, x);
      }
    }
  }
}

static KvRows rows_of(const KvCache& c, const void* k, const void* v, bool bf16, int rows, const size_t (&ld)[4], const int* slots) {
  KvRows a;
  a.k = k; a.v = v;
  a.k_ld = ld[0]; a.k_head = ld[1]; a.v_ld = ld[2]; a.v_head = ld[3];
  a.rows = rows; a.total = c.pages * c.page; a.slots = slots;
  a.data = c.data; a.scales = c.data + kv_code_bytes(c);
  a.place = {c.page == 32 ? 0 : c.page == 64 ? 1 : c.page == 128 ? 2 : 3, c.kv_heads};
  const size_t all = (ld[0] | ld[1] | ld[2] | ld[3]) * (bf16 ? 2 : 4) | (size_t)k | (size_t)v;
  a.wide = all % 16 == 0;
  return a;
}

// Blocks that share a tile of rows: as many as there are heads for, four to a block, up to `most` blocks in all; where few are made, some beside each
// other share the tile's rows too.  A block that writes goes through the rows behind its own for such that name the same slot: 24576 rows of 32 heads are
// written by 768 blocks of all heads in 152 us, by 1536 of half in 155, by 3840 in 189; read by 768 in 130, by 6144 in 122.  (That is rows times rows, which many rows
// feel: 131071 of 4 heads are written in 274 us, in four calls of a quarter in 187; 2^20 of one head in 11.0 ms, in 32 calls in 1.1.)
// Up to kSpread blocks have `turns` times as many, of a part of the rows each: 34 rows here and there of 32 heads are written in 8.3 us instead of 13.9 and read in 4.7
// instead of 9.5; of 376 blocks (1500 rows) writing takes 18.2 instead of 17.2 and reading 9.0 instead of 9.8, of 752 (3000 rows) 31.8 instead of 21.3 and 13.0 instead of 13.8.
constexpr int kSpread = 512;
static int kv_blocks(int tiles, int heads, int most) { return min((heads + 3) / 4, max(1, most / tiles)); }

#define EC_KV_LAUNCH(KERNEL, MOST, T, ES, HD)                                                                            \
  do {                                                                                                                   \
    constexpr int turns = kTileRows<HD> * (HD / 16) / 64;                                                                \
    const int tiles = (rows + kTileRows<HD> - 1) / kTileRows<HD>, y = kv_blocks(tiles, c.kv_heads, MOST);                 \
    if (tiles * y <= kSpread) KERNEL<T, ES, HD, true><<<dim3(tiles, y, turns), 256, 0, s>>>(a);                              \
    else KERNEL<T, ES, HD, false><<<dim3(tiles, y), 256, 0, s>>>(a);                                                     \
  } while (0)
#define EC_KV_PICK(KERNEL, MOST)                                                                      \
  do {                                                                                          \
    if (bf16) {                                                                                 \
      if (c.head_dim == 64) { if (c.e4m3) EC_KV_LAUNCH(KERNEL, MOST, bf16_t, 1, 64); else EC_KV_LAUNCH(KERNEL, MOST, bf16_t, 2, 64); }     \
      else { if (c.e4m3) EC_KV_LAUNCH(KERNEL, MOST, bf16_t, 1, 128); else EC_KV_LAUNCH(KERNEL, MOST, bf16_t, 2, 128); }                    \
    } else {                                                                                    \
      if (c.head_dim == 64) { if (c.e4m3) EC_KV_LAUNCH(KERNEL, MOST, float, 1, 64); else EC_KV_LAUNCH(KERNEL, MOST, float, 2, 64); }       \
      else { if (c.e4m3) EC_KV_LAUNCH(KERNEL, MOST, float, 1, 128); else EC_KV_LAUNCH(KERNEL, MOST, float, 2, 128); }                      \
    }                                                                                           \
  } while (0)

void launch_kv_write(const KvCache& c, const void* k, const void* v, bool bf16, int rows, const size_t (&ld)[4], const int* slots,
                     hipStream_t s) {
  const KvRows a = rows_of(c, k, v, bf16, rows, ld, slots);
  EC_KV_PICK(kv_write_kernel, 1024);
}

void launch_kv_read(const KvCache& c, void* k, void* v, bool bf16, int rows, const size_t (&ld)[4], const int* slots, hipStream_t s) {
  const KvRows a = rows_of(c, k, v, bf16, rows, ld, slots);
  EC_KV_PICK(kv_read_kernel, 8192);
}

}  // namespace ec
