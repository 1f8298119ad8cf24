// Matrices in microscaled 4-bit floating point: to and from it, and the product with a matrix that is kept in it.
//
// 32 consecutive values of a row share a scale 2^(s - 127), s one byte (255: the block is NaN); a value is an e2m1 code (1 sign, 2
// exponent bits with bias 1, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) times the scale.  Row-major: codes [rows, k/2], an even k in the
// low four bits, scales [rows, k/32].
//
// Laid out for the products ("packed"): tiles of 16 rows x 128 k.  Of a tile lane g*16 + r holds row r's block g, k = 32 g .. 32 g + 31:
// 16 bytes of codes, so that a wave-wide load is one KiB, and one byte of scale.  Four tiles in a row along k have their scales in one
// dword a lane, tile t's in byte t.  Codes [tile row][tile of k][lane][16], then scales [tile row][4 tiles of k][lane][4].
#include "ec_internal.h"

namespace ec {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ---- to and from ------------------------------------------------------------------------------
// scale byte of a block whose largest magnitude is amax: floor(log2 amax) - 2, which brings the largest value into [4, 8);
// 0 for an amax below 2^-125 (zero among them), 255 for one that is not finite
__device__ __forceinline__ uint32_t mx_scale(float amax) {
  const uint32_t e = __float_as_uint(amax) >> 23;   // (biased exponent, 0 for subnormals)
  return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}
// 2^(127 - s): what brings a block of scale s to the codes' range.  s = 254 and 253 give subnormals, which are kept.
__device__ __forceinline__ float mx_to_codes(uint32_t s) {
  return s < 254 ? __uint_as_float((254 - s) << 23) : 0x1p-127f;
}
// 2^(s - 127) as the conversion from codes takes it: the exponent bits alone; NaN for 255
__device__ __forceinline__ float mx_to_values(uint32_t s) { return __uint_as_float(s << 23); }

template <typename T>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T* __restrict__ x, long rows, int kb, size_t ld,
                                                          uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;   // a block of 32 values
  if (i >= rows * kb) return;
  const long row = i / kb;
  const T* p = x + (size_t)row * ld + (size_t)(i - row * kb) * 32;
  float v[32], amax = 0.f;
  bool finite = true;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    v[j] = load_f32(p + j);
    finite &= fabsf(v[j]) < INFINITY;
    amax = fmaxf(amax, fabsf(v[j]));
  }
  const uint32_t s = finite ? mx_scale(amax) : 255u;
  const float f = mx_to_codes(s);
  uint32_t out[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[8 * d] * f, v[8 * d + 1] * f, 1.f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[8 * d + 2] * f, v[8 * d + 3] * f, 1.f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[8 * d + 4] * f, v[8 * d + 5] * f, 1.f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[8 * d + 6] * f, v[8 * d + 7] * f, 1.f, 3);
    out[d] = finite ? c : 0u;
  }
  *(uint4*)(codes + (size_t)i * 16) = make_uint4(out[0], out[1], out[2], out[3]);
  scales[i] = (uint8_t)s;
}

template <typename T>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                            long rows, int kb, T* __restrict__ out, size_t ld) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;   // 8 values
  if (i >= rows * kb * 4) return;
  const long row = i / (kb * 4);
  const int at = (int)(i - row * kb * 4);
  const uint32_t c = *(const uint32_t*)(codes + (size_t)i * 4);
  const float s = mx_to_values(scales[(size_t)row * kb + (at >> 2)]);
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
  const float v[8] = {a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
  T* p = out + (size_t)row * ld + (size_t)at * 8;
#pragma unroll
  for (int j = 0; j < 8; ++j) store_f32(p + j, v[j]);
}

// one thread a block of 32 of the packed matrix; past the matrix' rows and k: zeros
__global__ __launch_bounds__(256) void mx_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int n,
                                                      int kb, int nt, int kq4, uint8_t* __restrict__ packed) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const int kq = mx_tiles_of_k(kb);
  if (i >= (long)nt * kq4 * 4 * 64) return;
  const int lane = (int)(i & 63);
  const long t = i >> 6;
  const int tile = (int)(t / (kq4 * 4)), q = (int)(t % (kq4 * 4));
  const int row = tile * 16 + (lane & 15), b = q * 4 + (lane >> 4);
  const bool in = row < n && b < kb;
  const size_t from = (size_t)row * kb + b;
  if (q < kq) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (in) v = *(const uint4*)(codes + from * 16);
    *(uint4*)(packed + (((size_t)tile * kq + q) * 64 + lane) * 16) = v;
  }
  uint8_t* sc = packed + (size_t)nt * kq * 1024;
  sc[(((size_t)tile * kq4 + (q >> 2)) * 64 + lane) * 4 + (q & 3)] = in ? scales[from] : (uint8_t)127;
}

// ---- product ------------------------------------------------------------------------------------
struct MxProduct {
  const void* x;             // bf16 [M, K] with row stride ld, or codes [M, K/2]
  const uint8_t* x_scales;   // [M, K/32]
  size_t ld;
  const uint8_t* w;          // packed
  long M;
  int N, kb;                 // rows of W; blocks of 32 along k
  void* y; size_t ldy;
};

// One wave a 16 x 16 tile of the result, all of K.
template <bool X4, typename TY>
__global__ __launch_bounds__(64) void mx_product_simple_kernel(MxProduct p) {
  const int lane = threadIdx.x, g = lane >> 4, r = lane & 15;
  const int kq = mx_tiles_of_k(p.kb), kq4 = (kq + 3) / 4, nt = (p.N + 15) / 16;
  const int tile = blockIdx.x;
  const long row0 = (long)blockIdx.y * 16, row = row0 + r;
  const bool row_in = row < p.M;
  const u32x4* wc = (const u32x4*)p.w + (size_t)tile * kq * 64 + lane;
  const uint32_t* ws = (const uint32_t*)(p.w + (size_t)nt * kq * 1024) + (size_t)tile * kq4 * 64 + lane;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int q = 0; q < kq; ++q) {
    const u32x4 c = wc[(size_t)q * 64];
    const uint32_t s = ws[(size_t)(q >> 2) * 64] >> ((q & 3) * 8) & 255u;
    const int b = q * 4 + g;                       // the lane's block
    const bool in = row_in && b < p.kb;
    if constexpr (X4) {
      u32x4 v = {0u, 0u, 0u, 0u};
      uint32_t sx = 127;
      if (in) {
        v = *(const u32x4*)((const uint8_t*)p.x + ((size_t)row * p.kb + b) * 16);
        sx = p.x_scales[(size_t)row * p.kb + b];
      }
      const i32x8 a = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
      const i32x8 bb = {(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, bb, acc, 4, 4, 0, s, 0, sx);
    } else {
      const float f = mx_to_values(s);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        union { bf16x2 h[4]; bf16x8 v; } w;
        w.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], f, 0);
        w.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], f, 1);
        w.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], f, 2);
        w.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], f, 3);
        union { u32x4 u; bf16x8 v; } x = {};
        if (in) x.u = *(const u32x4*)((const bf16_t*)p.x + (size_t)row * p.ld + (size_t)b * 32 + j * 8);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v, x.v, acc, 0, 0, 0);
      }
    }
  }
  // the lane holds features 4 g .. 4 g + 3 of the tile for its row r
  if (row_in)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = tile * 16 + g * 4 + i;
      if (n < p.N) store_f32((TY*)p.y + (size_t)row * p.ldy + n, acc[i]);
    }
}

// ---- launchers ------------------------------------------------------------------------------------
size_t mx_packed_bytes(int n, int kb) {
  const size_t nt = (n + 15) / 16, kq = mx_tiles_of_k(kb), kq4 = (kq + 3) / 4;
  return nt * kq * 1024 + nt * kq4 * 256;
}

void launch_mx_quantize(const void* x, bool bf16, long rows, int kb, size_t ld, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const unsigned grid = (unsigned)((rows * kb + 255) / 256);
  if (bf16) mx_quantize_kernel<<<grid, 256, 0, s>>>((const bf16_t*)x, rows, kb, ld, codes, scales);
  else mx_quantize_kernel<<<grid, 256, 0, s>>>((const float*)x, rows, kb, ld, codes, scales);
}

void launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, long rows, int kb, void* out, bool bf16, size_t ld,
                          hipStream_t s) {
  const unsigned grid = (unsigned)((rows * kb * 4 + 255) / 256);
  if (bf16) mx_dequantize_kernel<<<grid, 256, 0, s>>>(codes, scales, rows, kb, (bf16_t*)out, ld);
  else mx_dequantize_kernel<<<grid, 256, 0, s>>>(codes, scales, rows, kb, (float*)out, ld);
}

void launch_mx_pack(const uint8_t* codes, const uint8_t* scales, int n, int kb, uint8_t* packed, hipStream_t s) {
  const int nt = (n + 15) / 16, kq4 = (mx_tiles_of_k(kb) + 3) / 4;
  mx_pack_kernel<<<(unsigned)(((long)nt * kq4 * 4 * 64 + 255) / 256), 256, 0, s>>>(codes, scales, n, kb, nt, kq4, packed);
}

void launch_mx_linear(const void* x, const uint8_t* x_scales, long M, size_t ld, const uint8_t* packed, int N, int kb, void* y,
                      bool y_bf16, size_t ldy, hipStream_t s) {
  const MxProduct p = {x, x_scales, ld, packed, M, N, kb, y, ldy};
  const dim3 grid((N + 15) / 16, (unsigned)((M + 15) / 16));
  if (x_scales) {
    if (y_bf16) mx_product_simple_kernel<true, bf16_t><<<grid, 64, 0, s>>>(p);
    else mx_product_simple_kernel<true, float><<<grid, 64, 0, s>>>(p);
  } else {
    if (y_bf16) mx_product_simple_kernel<false, bf16_t><<<grid, 64, 0, s>>>(p);
    else mx_product_simple_kernel<false, float><<<grid, 64, 0, s>>>(p);
  }
}

}  // namespace ec
