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

// 16 components of a token's head as they are stored, in words of 4 bytes; returns the head's scale byte, found by its LANES lanes
// together.  bad: what a head that is not finite is filled with
template <int ES, int LANES>
__device__ __forceinline__ uint32_t stored(float (&v)[16], uint32_t (&w)[4 * ES], uint32_t bad) {
  if constexpr (ES == 2) {
    // (a value that rounds to an infinity is one)
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = bf16_to_f32(f32_to_bf16(v[j]));
  }
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, (uint32_t)dpp_i<0xB1>((int)top));
  top = max(top, (uint32_t)dpp_i<0x4E>((int)top));
  if constexpr (LANES == 8) top = max(top, (uint32_t)dpp_i<0x141>((int)top));
  const uint32_t s = ES == 1 ? kv_scale(top) : top >= 0x7f800000u ? 255u : 127u;
  if constexpr (ES == 1) {
    const float f = __uint_as_float((254 - min(s, 253u)) << 23);   // (s goes from 1 to 247, or is 255)
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = s == 255 ? bad : codes4(v + 4 * j, f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = s == 255 ? bad : (__float_as_uint(v[2 * j]) >> 16) | (__float_as_uint(v[2 * j + 1]) & 0xffff0000u);
  }
  return s;
}

// Marks the rows of a block's tile that are stored: their slot is in the cache, and no later row of the call names it.  keep: [ROWS] in
// LDS, slot or -1.
template <int ROWS>
__device__ __forceinline__ void keep_last(const int* slots, int rows, int row0, int total, int* keep) {
  if (threadIdx.x < ROWS) {
    const int r = row0 + threadIdx.x, s = r < rows ? slots[r] : -1;
    keep[threadIdx.x] = s >= 0 && s < total ? s : -1;
  }
  __syncthreads();
  for (int i = row0 + threadIdx.x; i < rows; i += 256) {
    const int s = slots[i];
    for (int j = 0; j < ROWS && row0 + j < i; ++j)
      if (keep[j] == s) keep[j] = -1;
  }
  __syncthreads();
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

// A block takes 4096 components: the rows of a tile, and goes through the heads.
template <typename T, int ES, int HD>
__global__ __launch_bounds__(256) void kv_write_kernel(KvRows a, int heads_each) {
  constexpr int LANES = HD / 16, ROWS = 256 / LANES;
  constexpr uint32_t kNaN = ES == 1 ? 0x7f7f7f7fu : 0x7fc07fc0u;
  typedef KvChunk<ES, HD> L;
  __shared__ int keep[ROWS];
  const int row0 = blockIdx.x * ROWS;
  keep_last<ROWS>(a.slots, a.rows, row0, a.total, keep);
  const int j = threadIdx.x / LANES, c0 = threadIdx.x % LANES * 16, slot = keep[j];
  if (slot < 0) return;
  const int w = slot & 31;
  const int last = min((int)(blockIdx.y + 1) * heads_each, a.place.kv_heads);
  for (int h = blockIdx.y * heads_each; h < last; ++h) {
    const size_t chunk = a.place.chunk(slot, h);
    uint8_t* to = a.data + chunk * L::kBytes;
    float v[16];
    uint32_t words[4 * ES];
    load_values((const T*)a.k + (size_t)(row0 + j) * a.k_ld + (size_t)h * a.k_head + c0, a.wide, v);
    uint32_t s = stored<ES, LANES>(v, words, kNaN);
#pragma unroll
    for (int i = 0; i < ES; ++i)
      *(uint4*)(to + L::key_at(w, c0 + i * 8)) = make_uint4(words[4 * i], words[4 * i + 1], words[4 * i + 2], words[4 * i + 3]);
    if (c0 == 0) a.scales[chunk * 64 + w] = (uint8_t)s;
    load_values((const T*)a.v + (size_t)(row0 + j) * a.v_ld + (size_t)h * a.v_head + c0, a.wide, v);
    s = stored<ES, LANES>(v, words, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (ES == 1) to[L::value_at(w, c0 + i)] = (uint8_t)(words[i >> 2] >> (8 * (i & 3)));
      else *(uint16_t*)(to + L::value_at(w, c0 + i)) = (uint16_t)(words[i >> 1] >> (16 * (i & 1)));
    }
    if (c0 == 0) a.scales[chunk * 64 + 32 + w] = (uint8_t)s;
  }
}

// 16 stored components as float32
template <int ES>
__device__ __forceinline__ void values_of(const uint32_t (&w)[4 * ES], uint32_t s, float (&v)[16]) {
  if constexpr (ES == 1) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const float f = __uint_as_float(s << 23);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), y = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
      v[4 * j] = x[0] * f; v[4 * j + 1] = x[1] * f; v[4 * j + 2] = y[0] * f; v[4 * j + 3] = y[1] * f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
  if (s == 255)
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(0x7fc00000u);
}

template <typename T>
__device__ __forceinline__ void store_values(T* p, bool wide, const float (&v)[16]) {
  if (!wide) {
#pragma unroll
    for (int j = 0; j < 16; ++j) store_f32(p + j, v[j]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) ((float4*)p)[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      ((uint4*)p)[j] = make_uint4(pack2_bf16(v[8 * j], v[8 * j + 1]), pack2_bf16(v[8 * j + 2], v[8 * j + 3]),
                                  pack2_bf16(v[8 * j + 4], v[8 * j + 5]), pack2_bf16(v[8 * j + 6], v[8 * j + 7]));
  }
}

template <typename T, int ES, int HD>
__global__ __launch_bounds__(256) void kv_read_kernel(KvRows a, int heads_each) {
  constexpr int LANES = HD / 16, ROWS = 256 / LANES;
  typedef KvChunk<ES, HD> L;
  const int row = blockIdx.x * ROWS + threadIdx.x / LANES, c0 = threadIdx.x % LANES * 16;
  if (row >= a.rows) return;
  const int slot = a.slots[row], w = slot & 31;
  const bool there = slot >= 0 && slot < a.total;
  const int last = min((int)(blockIdx.y + 1) * heads_each, a.place.kv_heads);
  for (int h = blockIdx.y * heads_each; h < last; ++h) {
    float k[16], v[16];
    if (there) {
      const size_t chunk = a.place.chunk(slot, h);
      const uint8_t* from = a.data + chunk * L::kBytes;
      uint32_t words[4 * ES];
#pragma unroll
      for (int i = 0; i < ES; ++i) {
        const uint4 u = *(const uint4*)(from + L::key_at(w, c0 + i * 8));
        words[4 * i] = u.x; words[4 * i + 1] = u.y; words[4 * i + 2] = u.z; words[4 * i + 3] = u.w;
      }
      values_of<ES>(words, a.scales[chunk * 64 + w], k);
#pragma unroll
      for (int i = 0; i < 4 * ES; ++i) words[i] = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (ES == 1) words[i >> 2] |= (uint32_t)from[L::value_at(w, c0 + i)] << (8 * (i & 3));
        else words[i >> 1] |= (uint32_t) * (const uint16_t*)(from + L::value_at(w, c0 + i)) << (16 * (i & 1));
      }
      values_of<ES>(words, a.scales[chunk * 64 + 32 + w], v);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) k[i] = v[i] = 0.f;
    }
    store_values((T*)a.k + (size_t)row * a.k_ld + (size_t)h * a.k_head + c0, a.wide, k);
    store_values((T*)a.v + (size_t)row * a.v_ld + (size_t)h * a.v_head + c0, a.wide, v);
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

// heads that a block goes through: one where there are few tiles of rows
static int heads_each(int tiles, int heads) {
  const int parts = min(heads, max(1, 2048 / max(tiles, 1)));
  return (heads + parts - 1) / parts;
}

#define EC_KV_LAUNCH(KERNEL, T, ES, HD)                                                         \
  do {                                                                                          \
    const int tiles = (rows + 256 / (HD / 16) - 1) / (256 / (HD / 16)), each = heads_each(tiles, c.kv_heads); \
    KERNEL<T, ES, HD><<<dim3(tiles, (c.kv_heads + each - 1) / each), 256, 0, s>>>(a, each);     \
  } while (0)
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
