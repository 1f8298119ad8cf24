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

template <typename T, int N>
__device__ __forceinline__ void load_values(const T* p, bool wide, float (&v)[N]) {
  if (wide) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < N / 4; ++j) {
        const float4 a = ((const float4*)p)[j];
        v[4 * j] = a.x; v[4 * j + 1] = a.y; v[4 * j + 2] = a.z; v[4 * j + 3] = a.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < N / 8; ++j) {
        const uint4 a = ((const uint4*)p)[j];
        const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[8 * j + 2 * k] = __uint_as_float(u[k] << 16);
          v[8 * j + 2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
        }
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = load_f32(p + j);
  }
}

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
  unsigned long long single;   // the block's rows that are in no run and have a slot, a bit each
  uint32_t seen[32];      // written: a bit for slot & 1023 of each row
  int low, high;
};

// WRITE: of rows that name the same slot the last one is stored.  The rows behind the block's are gone through; few of them are among the
// block's slots' range, and of these a bit for each of 1024 remainders leaves few to be compared.
template <int ROWS, bool WRITE>
__device__ __forceinline__ void find_runs(const KvRows& a, int row0, Tile<ROWS>& t) {
  typedef Tile<ROWS> Tl;
  static_assert(ROWS <= 64 && Tl::ALL <= 256, "a bit for each row, a thread for each");
  const int i = threadIdx.x, r = row0 - Tl::SIDE + i;
  int s = -1;
  if (i < Tl::ALL) {
    s = r >= 0 && r < a.rows ? a.slots[r] : -1;
    s = s >= 0 && s < a.total ? s : -1;
    t.slot[i] = s;
  }
  if constexpr (WRITE) {
    if (i < 32) t.seen[i] = 0;
    if (i == 32) { t.low = INT32_MAX; t.high = -1; }
    __syncthreads();
    if (s >= 0) {
      atomicOr(&t.seen[(s >> 5) & 31], 1u << (s & 31));
      atomicMin(&t.low, s);
      atomicMax(&t.high, s);
    }
    __syncthreads();
    const int low = t.low, range = t.high - low;
    auto compare = [&](int later, int slot) {
      if (!((t.seen[(slot >> 5) & 31] >> (slot & 31)) & 1u)) return;
      for (int j = 0; j < Tl::ALL && row0 - Tl::SIDE + j < later; ++j)
        if (t.slot[j] == slot) t.slot[j] = -1;
    };
    if (range >= 0)
      for (int n = max(row0 - Tl::SIDE, 0) + i; n < a.rows; n += 1024) {
        int x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = n + 256 * k < a.rows ? a.slots[n + 256 * k] : -1;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (x[k] >= 0 && (unsigned)(x[k] - low) <= (unsigned)range) compare(n + 256 * k, x[k]);
      }
  }
  __syncthreads();
  if (i < 64) {
    bool run = false, single = false;
    if (i < ROWS) {
      auto starts = [&](int at) {   // whether a run begins at row `at` of the tile
        const int s0 = t.slot[at];
        bool ok = s0 >= 0 && (s0 & 7) == 0;
        for (int k = 1; k < 8; ++k) ok = ok && t.slot[at + k] == s0 + k;
        return ok;
      };
      run = starts(Tl::SIDE + i);
      single = t.slot[Tl::SIDE + i] >= 0;
      for (int k = 0; k < 8 && single; ++k) single = !starts(Tl::SIDE + i - k);
    }
    const unsigned long long runs = __ballot(run), singles = __ballot(single);
    if (run) t.first[__popcll(runs & ((1ull << i) - 1))] = i;
    if (i == 0) { t.runs = __popcll(runs); t.single = singles; }
  }
  __syncthreads();
}

template <int HD> constexpr int kTileRows = 32 * (128 / HD);   // 64 lanes, 8 rows x 8 components each

// A wave takes the rows of a tile and goes through every (4 gridDim.y)-th head.  What bounds it is bytes: each is read and written once, in pieces of 16
// bytes and more but for the values of rows in no run.
template <typename T, int ES, int HD>
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
    if (has_run && blockIdx.z == 0) {
      const T* p = (const T*)a.v + (size_t)(row0 + first) * a.v_ld + (size_t)h * a.v_head + cv;
      float v[8][8];
#pragma unroll
      for (int r = 0; r < 8; ++r) load_values(p + (size_t)r * a.v_ld, a.wide, v[r]);
      uint32_t w[8][2 * ES], o[8][2 * ES], s[2] = {0, 0};
#pragma unroll
      for (int r = 0; r < 8; ++r) s[r >> 2] |= stored<ES, 8, HD>(v[r], w[r], 0) << (8 * (r & 3));
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
    // keys, and values of the rows in no run: 16 components of a token
    for (int i = blockIdx.z; i < ROWS * LK / 64; i += gridDim.z) {
      const int j = i * (64 / LK) + lane / LK, c0 = lane % LK * 16, slot = t.slot[Tile<ROWS>::SIDE + j], w = slot & 31;
      const bool single = (t.single >> j) & 1;
      if (slot >= 0) {
        const size_t chunk = a.place.chunk(slot, h);
        uint8_t* to = a.data + chunk * L::kBytes;
        float k[16], v[16];
        uint32_t words[4 * ES];
        load_values((const T*)a.k + (size_t)(row0 + j) * a.k_ld + (size_t)h * a.k_head + c0, a.wide, k);
        if (single) load_values((const T*)a.v + (size_t)(row0 + j) * a.v_ld + (size_t)h * a.v_head + c0, a.wide, v);
        uint32_t s = stored<ES, 16, HD>(k, words, kNaN);
#pragma unroll
        for (int n = 0; n < ES; ++n)
          *(uint4*)(to + L::key_at(w, c0 + n * 8)) = make_uint4(words[4 * n], words[4 * n + 1], words[4 * n + 2], words[4 * n + 3]);
        if (c0 == 0) a.scales[chunk * 64 + w] = (uint8_t)s;
        if (single) {
          s = stored<ES, 16, HD>(v, words, 0);
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
}

template <typename T, int ES, int HD>
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
    if (has_run && blockIdx.z == 0) {
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
    for (int i = blockIdx.z; i < ROWS * LK / 64; i += gridDim.z) {
      const int j = i * (64 / LK) + lane / LK, c0 = lane % LK * 16, slot = t.slot[Tile<ROWS>::SIDE + j], w = slot & 31;
      if (row0 + j < a.rows) {
        const bool there = slot >= 0, single = (t.single >> j) & 1;
        float k[16] = {}, v[16] = {};
        if (there) {
          const size_t chunk = a.place.chunk(slot, h);
          const uint8_t* from = a.data + chunk * L::kBytes;
          uint32_t kw[4 * ES], vw[4 * ES];
#pragma unroll
          for (int n = 0; n < ES; ++n) {
            const uint4 u = *(const uint4*)(from + L::key_at(w, c0 + n * 8));
            kw[4 * n] = u.x; kw[4 * n + 1] = u.y; kw[4 * n + 2] = u.z; kw[4 * n + 3] = u.w;
          }
          const uint32_t ks = a.scales[chunk * 64 + w], vs = a.scales[chunk * 64 + 32 + w];
#pragma unroll
          for (int n = 0; n < 4 * ES; ++n) vw[n] = 0;
          if (single) {
#pragma unroll
            for (int n = 0; n < 16; ++n) {
              if constexpr (ES == 1) vw[n >> 2] |= (uint32_t)from[L::value_at(w, c0 + n)] << (8 * (n & 3));
              else vw[n >> 1] |= (uint32_t) * (const uint16_t*)(from + L::value_at(w, c0 + n)) << (16 * (n & 1));
            }
          }
          values_of<ES>(kw, ks, k);
          values_of<ES>(vw, vs, v);
        }
        store_values((T*)a.k + (size_t)(row0 + j) * a.k_ld + (size_t)h * a.k_head + c0, a.wide, k);
        if (single || !there) store_values((T*)a.v + (size_t)(row0 + j) * a.v_ld + (size_t)h * a.v_head + c0, a.wide, v);
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

// Blocks that share a tile of rows: as many as there are heads for, four to a block, and four beside each other that share the rows in no run, as far as that
// makes no more than 2048 blocks.  (Each of them looks for rows that name the same slot.)
static dim3 kv_grid(int tiles, int heads) {
  const int y = min((heads + 3) / 4, max(1, 2048 / tiles));
  return dim3(tiles, y, tiles * y <= 512 ? 4 : 1);
}

#define EC_KV_LAUNCH(KERNEL, T, ES, HD) \
  KERNEL<T, ES, HD><<<kv_grid((rows + kTileRows<HD> - 1) / kTileRows<HD>, c.kv_heads), 256, 0, s>>>(a)
#define EC_KV_PICK(KERNEL)                                                                      \
  do {                                                                                          \
    if (bf16) {                                                                                 \
      if (c.head_dim == 64) { if (c.e4m3) EC_KV_LAUNCH(KERNEL, bf16_t, 1, 64); else EC_KV_LAUNCH(KERNEL, bf16_t, 2, 64); }     \
      else { if (c.e4m3) EC_KV_LAUNCH(KERNEL, bf16_t, 1, 128); else EC_KV_LAUNCH(KERNEL, bf16_t, 2, 128); }                    \
    } else {                                                                                    \
      if (c.head_dim == 64) { if (c.e4m3) EC_KV_LAUNCH(KERNEL, float, 1, 64); else EC_KV_LAUNCH(KERNEL, float, 2, 64); }       \
      else { if (c.e4m3) EC_KV_LAUNCH(KERNEL, float, 1, 128); else EC_KV_LAUNCH(KERNEL, float, 2, 128); }                      \
    }                                                                                           \
  } while (0)

void launch_kv_write(const KvCache& c, const void* k, const void* v, bool bf16, int rows, const size_t (&ld)[4], const int* slots,
                     hipStream_t s) {
  const KvRows a = rows_of(c, k, v, bf16, rows, ld, slots);
  EC_KV_PICK(kv_write_kernel);
}

void launch_kv_read(const KvCache& c, void* k, void* v, bool bf16, int rows, const size_t (&ld)[4], const int* slots, hipStream_t s) {
  const KvRows a = rows_of(c, k, v, bf16, rows, ld, slots);
  EC_KV_PICK(kv_read_kernel);
}

}  // namespace ec
