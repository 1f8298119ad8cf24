// Matrices in microscaled 4-bit floating point: to and from it, and the product with a matrix that is kept in it.
//
// 32 consecutive values of a row share a scale 2^(s - 127), s one byte (255: the block is NaN); a value is an e2m1 code (1 sign, 2
// exponent bits with bias 1, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) times the scale.  Row-major: codes [rows, k/2], an even k in the
// low four bits, scales [rows, k/32].
//
// Laid out for the products ("packed"): tiles of 16 rows x 128 k.  Of a tile lane g*16 + r holds row r's block g, k = 32 g .. 32 g + 31:
// 16 bytes of codes, so that a wave-wide load is one KiB, and one byte of scale.  Four tiles of rows make a group: at each 128 k a
// group has its codes [tile][lane][16], then its scales [lane][tile], 4352 bytes; groups go [64 rows][128 k].
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
// 2^(127 - s): what brings a block of scale s to the codes' range.  A finite block has s <= 252; the other value is for 255, whose codes are not used.
__device__ __forceinline__ float mx_to_codes(uint32_t s) {
  return s < 254 ? __uint_as_float((254 - s) << 23) : 0x1p-127f;
}
// 2^(s - 127) as the conversion from codes takes it: the exponent bits alone; NaN for 255
__device__ __forceinline__ float mx_to_values(uint32_t s) { return __uint_as_float(s << 23); }

// To and from move bytes: 24576 x 4096 float32 values to 4 bits and back 191 us, where a copy of as many bytes takes 159.
// A lane takes 8 values of a block, so that a wave reads 512 neighbours and writes 256 bytes; the block's four lanes find its largest
// together.  WIDE: rows lie so that 16 bytes can be read at a time.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T* __restrict__ x, long rows, int kb, size_t ld,
                                                          uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;   // eight values: four of these are a block
  if (i >= rows * kb * 4) return;                        // (the lanes of a block go together)
  const long row = i / (kb * 4);
  const T* p = x + (size_t)row * ld + (size_t)(i - row * (kb * 4)) * 8;
  float v[8];
  if constexpr (!WIDE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = load_f32(p + j);
  } else if constexpr (sizeof(T) == 4) {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const u32x4 a = *(const u32x4*)p;
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(a[j] << 16); v[2 * j + 1] = __uint_as_float(a[j] & 0xffff0000u); }
  }
  // (as integers, magnitudes order themselves and everything that is not finite is largest)
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, (uint32_t)dpp_i<0xB1>((int)top));
  top = max(top, (uint32_t)dpp_i<0x4E>((int)top));
  const bool finite = top < 0x7f800000u;
  const uint32_t s = finite ? mx_scale(__uint_as_float(top)) : 255u;
  const float f = mx_to_codes(s);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * f, v[1] * f, 1.f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * f, v[3] * f, 1.f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * f, v[5] * f, 1.f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * f, v[7] * f, 1.f, 3);
  ((uint32_t*)codes)[i] = finite ? c : 0u;
  if ((i & 3) == 0) scales[i >> 2] = (uint8_t)s;
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                            long rows, int kb, T* __restrict__ out, size_t ld) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;   // eight values
  if (i >= rows * kb * 4) return;
  const long row = i / (kb * 4);
  const uint32_t c = ((const uint32_t*)codes)[i];
  const float s = mx_to_values(scales[i >> 2]);
  T* p = out + (size_t)row * ld + (size_t)(i - row * (kb * 4)) * 8;
  if constexpr (sizeof(T) == 2 && WIDE) {
    union { bf16x2 h[4]; uint4 u; } o;
    o.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
    o.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
    o.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
    o.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
    *(uint4*)p = o.u;
  } else {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
    if constexpr (WIDE) {
      *(float4*)p = make_float4(a[0], a[1], b[0], b[1]);
      *(float4*)(p + 4) = make_float4(d[0], d[1], e[0], e[1]);
    } else {
      const float v[8] = {a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
#pragma unroll
      for (int j = 0; j < 8; ++j) store_f32(p + j, v[j]);
    }
  }
}

// one thread a block of 32 of the packed matrix; past the matrix' rows and k: zeros
__global__ __launch_bounds__(256) void mx_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int n,
                                                      int kb, long total, uint8_t* __restrict__ packed) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const int kq = mx_tiles_of_k(kb), lane = (int)(i & 63), t = (int)(i >> 6) & 3;
  const long part = i >> 8;                        // group and 128 k
  const int group = (int)(part / kq), q = (int)(part - (long)group * kq);
  const int row = group * 64 + t * 16 + (lane & 15), b = q * 4 + (lane >> 4);
  const bool in = row < n && b < kb;
  const size_t from = (size_t)row * kb + b;
  uint4 v = make_uint4(0, 0, 0, 0);
  if (in) v = *(const uint4*)(codes + from * 16);
  uint8_t* to = packed + (size_t)part * kMxGroupBytes;
  *(uint4*)(to + t * 1024 + lane * 16) = v;
  to[4096 + lane * 4 + t] = in ? scales[from] : (uint8_t)127;
}

// ---- product ------------------------------------------------------------------------------------
struct MxProduct {
  const void* x;             // bf16 [M, K] with row stride ld, or codes [M, K/2]
  const uint8_t* x_scales;   // [M, scale_ld]
  size_t ld;
  int scale_ld;
  const uint8_t* w;          // packed
  int M, N, kb;              // rows of x and of W; blocks of 32 along k
  void* y; size_t ldy;
  int wide, wide16;          // y takes the four features of a lane in one store; 16 bytes of bf16
  uint8_t* spread;           // room for the scales of 4-bit rows in whole dwords
  float* parts; int part_ld; // where K is split over blocks: their sums, [ranges][M][part_ld]; else NULL
};
constexpr int kMxParts = 4;  // most ranges
constexpr int kMxSplitRows = 1024;   // rows up to which K may be split

// 8 codes as 8 bf16 values, exactly (scale: the bits of 2^(s - 127))
__device__ __forceinline__ bf16x8 mx_widen(uint32_t codes, float scale) {
  union { bf16x2 h[4]; bf16x8 v; } w;
  w.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  w.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  w.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  w.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return w.v;
}
__device__ __forceinline__ i32x8 mx_operand(u32x4 v) {
  return (i32x8){(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) {
  union { u32x4 u; bf16x8 b; } c;
  c.u = v;
  return c.b;
}

// features n .. n + 3 of row m
template <typename TY>
__device__ __forceinline__ void mx_store(const MxProduct& p, int m, int n, f32x4 v) {
  TY* y = (TY*)p.y + (size_t)m * p.ldy + n;
  if (p.wide) {
    if (n < p.N) {   // (N is a multiple of 4)
      if constexpr (sizeof(TY) == 4) *(float4*)y = make_float4(v[0], v[1], v[2], v[3]);
      else *(uint2*)y = make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < p.N) store_f32(y + i, v[i]);
  }
}

enum { MX_RING = 0, MX_REGS = 1, MX_X4 = 2 };   // where a wave's rows go: bf16 to LDS or to registers, 4-bit ones to registers

// Few rows: a stream of W.  A block owns NTW tiles of 16 features, all MT tiles of 16 rows and one of gridDim.y ranges of K; its KS
// waves share that out, and their sums meet in LDS in the order of the waves.  What a wave multiplies next is on its way while
// it multiplies: R sets of operands, W in registers, bf16 rows by direct loads to a ring in LDS of the wave's own (which takes no
// registers and no barrier): rows of 256 bytes, their 16-byte chunks at their number XOR the row, so that 16 rows read at the same k hit all banks.
// NW > 1 is for many features: NW waves with tiles of their own share a ring, each bringing its part of the rows, and a barrier a step.  The
// rows then pass into LDS once for NW * NTW tiles, and the short sums let several blocks lie on a compute unit, whose waves together keep HBM
// busy.  Calls one behind the other: 34 x 24576 x 4096 18.2 us (53 MB of W: 2.9 TB/s, a compute unit's share of rows and W at about 50 KB/us, one wave
// a SIMD), 32 x 126464 x 4096 in float32 51.5 us (290 MB: 5.7 TB/s).  Three sets of operands, and rows in registers for more than 4 rows, were no
// faster.  4-bit rows lie in registers: 32 rows with 24576 features 12.5 us (bf16 rows 16), with 126464 and a bf16 result 57.5 (49: shared rows).
template <int XF, typename TY, int MT, int NTW, int KS, int NW>
__global__ __launch_bounds__(KS * NW * 64) void mx_rows_kernel(MxProduct p) {
  constexpr int R = 2;
  static_assert(NW == 1 || XF == MX_RING, "waves that share their rows");
  constexpr bool X4 = XF == MX_X4, RING = XF == MX_RING;
  extern __shared__ f32x4 red[];   // the rings; then [KS][NTW * MT][64]
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = wave_all / NW, wn = wave_all % NW;
  const int kq = mx_tiles_of_k(p.kb), groups = (p.N + 63) / 64, tile0 = (blockIdx.x * NW + wn) * NTW;
  const int klo = (int)((long)blockIdx.y * kq / gridDim.y), kn = (int)((long)(blockIdx.y + 1) * kq / gridDim.y) - klo;
  const int lo = klo + (int)((long)wave * kn / KS), n = klo + (int)((long)(wave + 1) * kn / KS) - lo;
  const uint8_t* wp[NTW];
#pragma unroll
  for (int i = 0; i < NTW; ++i) {
    const int t = tile0 + i < groups * 4 ? tile0 + i : 0;   // (a tile past the end is not stored)
    wp[i] = p.w + ((size_t)(t >> 2) * kq + lo) * kMxGroupBytes + (t & 3) * 1024 + lane * 16;
  }
  // A tile's scale is the byte of its number in its group's dword; NTW tiles lie in GW groups.
  constexpr int GW = NTW > 4 ? 2 : 1;
  static_assert(NTW == 1 || NTW == 2 || NTW == 4 || NTW == 6 || NTW == 8, "the bytes below");
  const uint8_t* sp[GW];
#pragma unroll
  for (int i = 0; i < GW; ++i) {
    const int gr = (tile0 >> 2) + i < groups ? (tile0 >> 2) + i : 0;
    sp[i] = p.w + ((size_t)gr * kq + lo) * kMxGroupBytes + 4096 + lane * 4;
  }
  const int first_byte = tile0 & 3;
  // To registers: the lane's own row of each tile.  To LDS: the row of which the lane brings 16 bytes, four rows a load.
  constexpr int XL = RING ? MT * 4 : MT, XN = X4 ? 1 : 4;
  const char* xp[XL / NW];
  const uint8_t* xs[MT];
#pragma unroll
  for (int j = 0; j < XL / NW; ++j) {
    const int row = RING ? (j * NW + wn) * 4 + g : j * 16 + r, m = row < p.M ? row : 0;
    xp[j] = X4 ? (const char*)p.x + (size_t)m * p.kb * 16 : (const char*)p.x + (size_t)m * p.ld * 2;
    if constexpr (X4) xs[j] = p.x_scales + (size_t)m * p.scale_ld;
  }
  char* ring = (char*)red + wave * (R * MT * 4096);

  f32x4 acc[NTW][MT];
#pragma unroll
  for (int i = 0; i < NTW; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

  struct Set {
    u32x4 w[NTW], x[RING ? 1 : MT][XN];
    uint32_t ws[GW], xs[X4 ? MT : 1];
  } set[R];
  constexpr int LOADS = NTW + GW + 4 * MT;   // of a set, where there is a ring
  // Blocks past K: their codes in W are 0; x is read where there is some, and set to 0 below.
  auto load = [&](int s, int it) {
    const int step = it < n ? it : n - 1, q = lo + step;
    if constexpr (!RING) {
      const int blk = min(q * 4 + g, p.kb - 1);
#pragma unroll
      for (int j = 0; j < MT; ++j) {
#pragma unroll
        for (int h = 0; h < XN; ++h) set[s].x[j][h] = *(const u32x4*)(xp[j] + (size_t)blk * (XN * 16) + h * 16);
        if constexpr (X4) set[s].xs[j] = xs[j][blk];
      }
    } else {
#pragma unroll
      for (int j0 = 0; j0 < XL; j0 += NW) {   // (waves with the same rows bring every NW-th)
        const int j = j0 + wn;
        int c = r ^ ((j * 4 + g) & 15);
        c = q * 4 + (c >> 2) < p.kb ? c : 0;
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(xp[j0 / NW] + (size_t)q * 256 + c * 16),
                                         (void __attribute__((address_space(3)))*)(ring + s * (MT * 4096) + j * 1024), 16, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < NTW; ++i) set[s].w[i] = __builtin_nontemporal_load((const u32x4*)(wp[i] + (size_t)step * kMxGroupBytes));
#pragma unroll
    for (int i = 0; i < GW; ++i) set[s].ws[i] = *(const uint32_t*)(sp[i] + (size_t)step * kMxGroupBytes);
  };
  auto mma = [&](int s, int it) {
    const bool tail = (lo + it + 1) * 4 > p.kb, in = (lo + it) * 4 + g < p.kb;
    uint32_t sc[NTW > 4 ? 2 : 1];
    if constexpr (NTW == 8) { sc[0] = set[s].ws[0]; sc[1] = set[s].ws[1]; }
    else if constexpr (NTW == 6) {
      sc[0] = __builtin_amdgcn_alignbyte(set[s].ws[1], set[s].ws[0], first_byte);
      sc[1] = set[s].ws[1] >> (8 * first_byte);
    } else {
      sc[0] = set[s].ws[0] >> (8 * first_byte);
    }
    if constexpr (!RING) {
      if (tail) {
#pragma unroll
        for (int j = 0; j < MT; ++j) {
#pragma unroll
          for (int h = 0; h < XN; ++h) set[s].x[j][h] = in ? set[s].x[j][h] : (u32x4){0u, 0u, 0u, 0u};
          if constexpr (X4) set[s].xs[j] = in ? set[s].xs[j] : 127u;
        }
      }
    }
    if constexpr (X4) {
#pragma unroll
      for (int i = 0; i < NTW; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          const i32x8 w = mx_operand(set[s].w[i]), x = mx_operand(set[s].x[j][0]);
          const int a = (int)sc[i >> 2], b = (int)set[s].xs[j];
          if ((i & 3) == 0) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc[i][j], 4, 4, 0, a, 0, b);
          else if ((i & 3) == 1) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc[i][j], 4, 4, 1, a, 0, b);
          else if ((i & 3) == 2) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc[i][j], 4, 4, 2, a, 0, b);
          else acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc[i][j], 4, 4, 3, a, 0, b);
        }
    } else {
      float f[NTW];
#pragma unroll
      for (int i = 0; i < NTW; ++i) f[i] = mx_to_values(sc[i >> 2] >> (8 * (i & 3)) & 255u);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        u32x4 x[MT];
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          if constexpr (RING) x[j] = *(const u32x4*)(ring + s * (MT * 4096) + (j * 16 + r) * 256 + ((g * 4 + h) ^ r) * 16);
          else x[j] = set[s].x[j][h];
        }
        if (RING && tail)
#pragma unroll
          for (int j = 0; j < MT; ++j) x[j] = in ? x[j] : (u32x4){0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < NTW; ++i) {
          const bf16x8 w = mx_widen(set[s].w[i][h], f[i]);
#pragma unroll
          for (int j = 0; j < MT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, as_bf16x8(x[j]), acc[i][j], 0, 0, 0);
        }
      }
    }
  };
  if constexpr (NW > 1) {
    // The waves that share a ring meet at each step, behind which its rows are there for both and the other place is free.
    const int most = (kn + KS - 1) / KS;
    if (n > 0) load(0, 0);
    for (int it = 0; it < most; it += 2) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (it + s < most) {
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          block_barrier_nofence();
          if (it + s + 1 < n) load(s ^ 1, it + s + 1);
          __builtin_amdgcn_sched_barrier(0);
          if (it + s < n) mma(s, it + s);
        }
      }
    }
  } else if (n > 0) {
#pragma unroll
    for (int s = 0; s < R - 1; ++s) load(s, s);
    for (int it = 0;; it += R) {
      bool done = false;
#pragma unroll
      for (int s = 0; s < R; ++s) {
        if (!done) {
          // (a slot of the ring is filled again once its reads have been waited for, by the products before this)
          load((s + R - 1) % R, it + s + R - 1);
          if constexpr (RING) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((R - 1) * LOADS) : "memory");
          __builtin_amdgcn_sched_barrier(0);
          mma(s, it + s);
          __builtin_amdgcn_sched_barrier(0);
          done = it + s + 1 >= n;
        }
      }
      if (done) break;
    }
  }
  constexpr int UNITS = NTW * MT;
  if constexpr (RING) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the last loads to the ring, asked for but not used)
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < NTW; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) red[(wave_all * UNITS + i * MT + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int o = threadIdx.x; o < NW * UNITS * 64; o += KS * NW * 64) {
    f32x4 v = red[o];
#pragma unroll
    for (int w = 1; w < KS; ++w) v += red[w * NW * UNITS * 64 + o];
    const int l = o & 63, unit = o >> 6, i = unit / MT, m = (unit - i * MT) * 16 + (l & 15);
    const int f = (blockIdx.x * NW * NTW + i) * 16 + (l >> 4) * 4;
    if (m < p.M) {
      if (p.parts) {
        if (f < p.N) *(f32x4*)(p.parts + ((size_t)blockIdx.y * p.M + m) * p.part_ld + f) = v;
      } else {
        mx_store<TY>(p, m, f, v);
      }
    }
  }
}

// Which block of the result: an XCD takes a run of the blocks in an order that goes down 8 blocks of rows, then on along the features, so
// that what its 32 compute units work on at a time shares rows and features.
__device__ __forceinline__ void mx_block_xy(int gx, int gy, int& bx, int& by) {
  const int nb = gx * gy, xcd = blockIdx.x & 7;
  const int j = xcd * (nb >> 3) + min(xcd, nb & 7) + (int)(blockIdx.x >> 3);
  const int panel = j / (8 * gx), high = min(8, gy - panel * 8), in = j - panel * 8 * gx;
  by = panel * 8 + in % high;
  bx = in / high;
}

// Many rows: 8 waves (WM x WN), a wave WTM tiles of 16 rows x 64 features.  QS steps of 128 k are a stage; S stages are in LDS, brought there by
// direct loads, one barrier a stage.  W lies there as it is packed.  Rows of bf16 (256 bytes a step) and of codes (128 bytes, two steps)
// have their 16-byte chunks at their number XOR the row, so that rows read at the same k hit all banks; the scales of 4-bit rows go
// [step][row], four bytes each.  561 x 37888 x 3584 in bf16: 150 us once the card has been at it for some ms (170 in the first launches of a
// process), 1.02 PFLOP/s of the 1.34 that a plain bf16 product reaches: the widening of W, done again by each block of rows, and the LDS reads
// beside the products.  (256 x 128 tiles: slower.)
template <bool X4, int WM, int WN, int WTM> struct MxTile {
  static constexpr int BM = WM * WTM * 16, BN = WN * 64, QS = X4 ? 2 : 1;
  static constexpr int XB = BM * (X4 ? 128 : 256), SB = X4 ? BM * 8 : 0, WB = WN * QS * (int)kMxGroupBytes;
  static constexpr int STAGE = XB + SB + WB;
  static constexpr int S = STAGE * 3 <= 160 * 1024 ? 3 : 2;
};
template <bool X4, typename TY, int WM, int WN, int WTM>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void mx_tiled_kernel(MxProduct p) {
  typedef MxTile<X4, WM, WN, WTM> T;
  static_assert(WM * WN == 8, "eight waves");
  constexpr int QS = T::QS, S = T::S;
  extern __shared__ char lds_[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
  const int wm = wave / WN, wn = wave % WN;
  const int kq = mx_tiles_of_k(p.kb), groups = (p.N + 63) / 64;
  const int gx = (p.N + T::BN - 1) / T::BN, gy = (p.M + T::BM - 1) / T::BM;
  int bx, by;
  mx_block_xy(gx, gy, bx, by);
  const int m0 = by * T::BM, group0 = bx * WN;
  const int st_all = (kq + QS - 1) / QS;
  const int st_lo = (int)((long)blockIdx.y * st_all / gridDim.y), ns = (int)((long)(blockIdx.y + 1) * st_all / gridDim.y) - st_lo;

  // loads of a stage: rows, then W, whole waves of 16 bytes a lane; what does not divide over the waves is shared by all of them
  constexpr int XL = T::XB / 1024 / 8, WU = T::WB / 16, WL = WU / 512, REST = WU % 512 / 8, UN = QS * 272;
  static_assert(T::XB % 8192 == 0 && WU % 8 == 0 && (REST == 0 || 64 % REST == 0), "whole loads, and as many lanes of one for each wave");
  const char* xsrc[XL];
  int xchunk[XL];
#pragma unroll
  for (int i = 0; i < XL; ++i) {
    const int u = (i * 8 + wave) * 64 + lane, row = X4 ? u >> 3 : u >> 4;
    const int m = min(m0 + row, p.M - 1);
    xchunk[i] = X4 ? (u & 7) ^ (row & 7) : (u & 15) ^ (row & 15);
    xsrc[i] = X4 ? (const char*)p.x + (size_t)m * p.kb * 16 : (const char*)p.x + (size_t)m * p.ld * 2;
  }
  auto w_unit = [&](int u, int& q) {   // where unit u of a stage's W comes from, at step 0
    const int gr = u / UN, off = u - gr * UN, group = group0 + gr < groups ? group0 + gr : 0;
    q = QS == 2 && off >= 272;
    return (const char*)p.w + (size_t)group * kq * kMxGroupBytes + (size_t)(off - q * 272) * 16;
  };
  const char* wsrc[WL + (REST > 0)];
  int wq[WL + (REST > 0)];
#pragma unroll
  for (int i = 0; i < WL; ++i) wsrc[i] = w_unit((i * 8 + wave) * 64 + lane, wq[i]);
  const int rest0 = wave * REST, rest_load = WL * 8 + (rest0 >> 6);
  const bool rest_mine = lane >= (rest0 & 63) && lane < (rest0 & 63) + REST;
  if constexpr (REST > 0) wsrc[WL] = w_unit(min(rest_load * 64 + lane, WU - 1), wq[WL]);
  // scales of 4-bit rows: a dword a row and step
  constexpr int SLOADS = X4 ? QS * T::BM / 64 : 0, SL = (SLOADS + 7) / 8;
  const uint8_t* ssrc[SL > 0 ? SL : 1];
  int sat[SL > 0 ? SL : 1];
#pragma unroll
  for (int i = 0; i < SL; ++i) {
    const int l = (i * 8 + wave) % (SLOADS ? SLOADS : 1);   // (brought twice where there are fewer than waves)
    sat[i] = l;
    ssrc[i] = p.x_scales + (size_t)min(m0 + (l % (T::BM / 64)) * 64 + lane, p.M - 1) * p.scale_ld;
  }
  constexpr int LOADS = XL + WL + (REST > 0) + SL;
  auto load = [&](int stage) {
    const int st = st_lo + min(stage, ns - 1), q0 = st * QS;
    char* to = lds_ + (stage % S) * T::STAGE;
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      int b = X4 ? q0 * 4 + xchunk[i] : q0 * 4 + (xchunk[i] >> 2);   // (past K: read something that is there, and see below)
      b = b < p.kb ? b : q0 * 4;
      const char* from = xsrc[i] + (X4 ? (size_t)b * 16 : (size_t)b * 64 + (xchunk[i] & 3) * 16);
      __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)from,
                                       (void __attribute__((address_space(3)))*)(to + (i * 8 + wave) * 1024), 16, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < SL; ++i) {
      const int q = min(q0 + sat[i] / (T::BM / 64), kq - 1);
      __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(ssrc[i] + (size_t)q * 4),
                                       (void __attribute__((address_space(3)))*)(to + T::XB + sat[i] * 256), 4, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < WL + (REST > 0); ++i) {
      const int q = min(q0 + wq[i], kq - 1), l = i < WL ? i * 8 + wave : rest_load;
      const char* from = wsrc[i] + (size_t)q * kMxGroupBytes;
      const auto slot = (void __attribute__((address_space(3)))*)(to + T::XB + T::SB + l * 1024);
      if (i < WL) __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)from, slot, 16, 0, 0);
      else if (rest_mine) __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)from, slot, 16, 0, 0);
    }
  };

  f32x4 acc[4][WTM];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < WTM; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int s = 0; s < S - 1; ++s) load(s);
  for (int s = 0; s < ns; ++s) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * LOADS) : "memory");
    char* at = lds_ + (s % S) * T::STAGE;
    if (!X4 && (st_lo + s + 1) * 4 > p.kb) {   // bf16 past K: zeros, by the wave that brought them
#pragma unroll
      for (int i = 0; i < XL; ++i)
        if ((st_lo + s) * 4 + (xchunk[i] >> 2) >= p.kb) *(u32x4*)(at + (i * 8 + wave) * 1024 + lane * 16) = (u32x4){0u, 0u, 0u, 0u};
    }
    block_barrier_nofence();
    load(s + S - 1);
    const char* wl = at + T::XB + T::SB + wn * QS * (int)kMxGroupBytes;
#pragma unroll
    for (int q = 0; q < QS; ++q) {
      if (QS == 2 && q == 1 && (st_lo + s) * 2 + 1 >= kq) break;
      u32x4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = *(const u32x4*)(wl + q * kMxGroupBytes + i * 1024 + lane * 16);
      const uint32_t ws = *(const uint32_t*)(wl + q * kMxGroupBytes + 4096 + lane * 4);
      if constexpr (X4) {
#pragma unroll
        for (int j = 0; j < WTM; ++j) {
          const int row = (wm * WTM + j) * 16 + r;
          const i32x8 x = mx_operand(*(const u32x4*)(at + row * 128 + (((q * 4 + g) ^ (row & 7)) * 16)));
          const int xs = (int)(*(const uint32_t*)(at + T::XB + (q * T::BM + row) * 4) >> (8 * g));
          acc[0][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(w[0]), x, acc[0][j], 4, 4, 0, (int)ws, 0, xs);
          acc[1][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(w[1]), x, acc[1][j], 4, 4, 1, (int)ws, 0, xs);
          acc[2][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(w[2]), x, acc[2][j], 4, 4, 2, (int)ws, 0, xs);
          acc[3][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(w[3]), x, acc[3][j], 4, 4, 3, (int)ws, 0, xs);
        }
      } else {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = mx_to_values(ws >> (8 * i) & 255u);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          bf16x8 x[WTM];
#pragma unroll
          for (int j = 0; j < WTM; ++j)
            x[j] = as_bf16x8(*(const u32x4*)(at + ((wm * WTM + j) * 16 + r) * 256 + ((g * 4 + h) ^ r) * 16));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bf16x8 v = mx_widen(w[i][h], f[i]);
#pragma unroll
            for (int j = 0; j < WTM; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, x[j], acc[i][j], 0, 0, 0);
          }
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the last loads, asked for but not used)
#pragma unroll
  for (int j = 0; j < WTM; ++j) {
    const int m = m0 + (wm * WTM + j) * 16 + r;
    if (m < p.M) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int f = (group0 + wn) * 64 + i * 16 + g * 4;
        if (p.parts) {
          if (f < p.N) *(f32x4*)(p.parts + ((size_t)blockIdx.y * p.M + m) * p.part_ld + f) = acc[i][j];
        } else {
          mx_store<TY>(p, m, f, acc[i][j]);
        }
      }
    }
  }
}

// Many rows in 4 bits.  As above, with v_mfma_scale_f32_32x32x64 (6.9 PFLOP/s from registers with random operands against 4.5 to 5.7 of
// 16x16x128, whose instructions one wave cannot issue often enough): 64 k a step, in which a lane has one block of 32 of one of 32 rows, 16
// bytes, and its scale.  A wave has MF x NF tiles of 32 x 32.  Four steps are a stage, two stages are in LDS.  The operands of a step are
// read while the step before it is multiplied; at a stage's last step the waves meet, behind which the next stage has landed and this
// one's place is free for the one after.  24576 x 12288 x 4096: 776 us, 3.2 PFLOP/s; a block of 256 x 256 takes 4 us to begin, 42 for 16 stages (30
// without the loads, 27 without the products, so neither alone: one stage is on its way and is waited for whole at each meeting; stages of 128 k,
// of which four would fit, have not been tried) and 3.4 to store.  With zeros for operands the whole takes 725 us: the clock under load is part
// of it.
template <int WM, int WN, int MF, int NF> struct MxTile4 {
  static constexpr int BM = WM * MF * 32, BN = WN * NF * 32;
  static constexpr int XB = BM * 128, SB = BM * 8, WB = BN / 64 * 2 * (int)kMxGroupBytes, STAGE = XB + SB + WB;
};
typedef float f32x16 __attribute__((ext_vector_type(16)));

// y in 16 bytes a lane where it can: lanes l and l + 32 hold row m, features 8 j + 4 (l >> 5) + 0 .. 3 of 32 from n on
template <typename TY>
__device__ __forceinline__ void mx_store32(const MxProduct& p, int m, int n, const f32x16& v, bool valid) {
  const bool hi = (threadIdx.x & 32) != 0;
  if constexpr (sizeof(TY) == 2) {
    if (p.wide16) {
#pragma unroll
      for (int j = 0; j < 4; j += 2) {   // the lower lane ends with both halves of eight features, the upper with those of the next eight
        const uint32_t a0 = pack2_bf16(v[4 * j], v[4 * j + 1]), a1 = pack2_bf16(v[4 * j + 2], v[4 * j + 3]);
        const uint32_t b0 = pack2_bf16(v[4 * j + 4], v[4 * j + 5]), b1 = pack2_bf16(v[4 * j + 6], v[4 * j + 7]);
        const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        const int f = n + 8 * (j + hi);
        if (valid && f < p.N) *(uint4*)((bf16_t*)p.y + (size_t)m * p.ldy + f) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
      }
      return;
    }
  }
  if (valid)
#pragma unroll
    for (int j = 0; j < 4; ++j) mx_store<TY>(p, m, n + 8 * j + (hi ? 4 : 0), (f32x4){v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]});
}

template <typename TY, int WM, int WN, int MF, int NF>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void mx_tiled4_kernel(MxProduct p) {
  typedef MxTile4<WM, WN, MF, NF> T;
  static_assert(WM * WN == 8 && T::BN % 64 == 0 && T::BM % 64 == 0, "eight waves, whole groups");
  extern __shared__ char lds_[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, r32 = lane & 31;
  const int wm = wave / WN, wn = wave % WN;
  const int kq = mx_tiles_of_k(p.kb), groups = (p.N + 63) / 64;
  const int gx = (p.N + T::BN - 1) / T::BN, gy = (p.M + T::BM - 1) / T::BM;
  int bx, by;
  mx_block_xy(gx, gy, bx, by);
  const int m0 = by * T::BM, group0 = bx * (T::BN / 64);
  const int st_all = (kq + 1) / 2;
  const int st_lo = (int)((long)blockIdx.y * st_all / gridDim.y), ns = (int)((long)(blockIdx.y + 1) * st_all / gridDim.y) - st_lo;

  // loads of a stage, 16 bytes a lane: rows, W, and what of W is left over, which several waves bring
  constexpr int XL = T::XB / 8192, WU = T::WB / 16, WL = WU / 512, RL = (WU % 512 + 63) / 64;
  static_assert(T::XB % 8192 == 0, "whole loads");
  const char* xsrc[XL];
  int xchunk[XL];
#pragma unroll
  for (int i = 0; i < XL; ++i) {
    const int u = (i * 8 + wave) * 64 + lane, row = u >> 3;
    xchunk[i] = (u & 7) ^ (row & 7);
    xsrc[i] = (const char*)p.x + (size_t)min(m0 + row, p.M - 1) * p.kb * 16;
  }
  const char* wsrc[WL + (RL > 0)];
  int wq[WL + (RL > 0)], wat[WL + (RL > 0)];
#pragma unroll
  for (int i = 0; i < WL + (RL > 0); ++i) {
    wat[i] = i < WL ? i * 8 + wave : WL * 8 + wave % (RL ? RL : 1);
    const int u = min(wat[i] * 64 + lane, WU - 1), gr = u / 544, off = u - gr * 544, group = group0 + gr < groups ? group0 + gr : 0;
    wq[i] = off >= 272;
    wsrc[i] = (const char*)p.w + (size_t)group * kq * kMxGroupBytes + (size_t)(off - wq[i] * 272) * 16;
  }
  const bool rest_in = WU % 64 == 0 || wat[WL + (RL > 0) - 1] * 64 + lane < WU;
  constexpr int SLOADS = T::BM / 32, SL = (SLOADS + 7) / 8;
  const uint8_t* ssrc[SL];
  int sat[SL];
#pragma unroll
  for (int i = 0; i < SL; ++i) {
    sat[i] = (i * 8 + wave) % SLOADS;
    ssrc[i] = p.x_scales + (size_t)min(m0 + (sat[i] % (T::BM / 64)) * 64 + lane, p.M - 1) * p.scale_ld;
  }
  auto load = [&](int stage) {
    const int q0 = (st_lo + min(stage, ns - 1)) * 2;
    char* to = lds_ + (stage & 1) * T::STAGE;
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      const int b = q0 * 4 + xchunk[i];   // (past K: codes that are there, times codes of W that are 0)
      __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(xsrc[i] + (size_t)(b < p.kb ? b : q0 * 4) * 16),
                                       (void __attribute__((address_space(3)))*)(to + (i * 8 + wave) * 1024), 16, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < SL; ++i)
      __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(ssrc[i] + (size_t)min(q0 + sat[i] / (T::BM / 64), kq - 1) * 4),
                                       (void __attribute__((address_space(3)))*)(to + T::XB + sat[i] * 256), 4, 0, 0);
#pragma unroll
    for (int i = 0; i < WL + (RL > 0); ++i) {
      const char* from = wsrc[i] + (size_t)min(q0 + wq[i], kq - 1) * kMxGroupBytes;
      const auto slot = (void __attribute__((address_space(3)))*)(to + T::XB + T::SB + wat[i] * 1024);
      if (i < WL || rest_in) __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)from, slot, 16, 0, 0);
    }
  };

  f32x16 acc[NF][MF];
#pragma unroll
  for (int i = 0; i < NF; ++i)
#pragma unroll
    for (int j = 0; j < MF; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  struct Step {
    u32x4 w[NF], x[MF];
    int ws[NF], xs[MF];
  } a, b;
  // step t of a stage: 64 k, blocks 2 (t & 1) and 2 (t & 1) + 1 of 128 k number t >> 1.  The scales of both steps of these lie in a dword, the
  // odd step's two bytes up.
  auto read = [&](Step& s, int stage, int t) {
    const char* at = lds_ + (stage & 1) * T::STAGE;
    const int q = t >> 1, blk = 2 * (t & 1) + half;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const int pair = wn * NF + i;   // 32 features: two tiles of a group
      const char* g = at + T::XB + T::SB + ((pair >> 1) * 2 + q) * (int)kMxGroupBytes;
      const int place = blk * 16 + (r32 & 15);
      s.w[i] = *(const u32x4*)(g + (2 * (pair & 1) + (r32 >> 4)) * 1024 + place * 16);
      s.ws[i] = *(const int*)(g + 4096 + place * 4);
    }
#pragma unroll
    for (int j = 0; j < MF; ++j) {
      const int row = (wm * MF + j) * 32 + r32;
      s.x[j] = *(const u32x4*)(at + row * 128 + (((q * 4 + blk) ^ (row & 7)) * 16));
      s.xs[j] = *(const int*)(at + T::XB + (q * T::BM + row) * 4);
    }
  };
  auto mma = [&](Step& s, bool odd) {
    // (the scales are shifted here and not where they are read, which would wait for them)
#pragma unroll
    for (int i = 0; i < NF; ++i) s.ws[i] >>= 16 * ((wn * NF + i) & 1) + 8 * (r32 >> 4);
#pragma unroll
    for (int j = 0; j < MF; ++j) s.xs[j] >>= 8 * half;
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
      for (int j = 0; j < MF; ++j)
        acc[i][j] = odd ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand(s.w[i]), mx_operand(s.x[j]), acc[i][j], 4, 4, 0, s.ws[i], 2, s.xs[j])
                        : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand(s.w[i]), mx_operand(s.x[j]), acc[i][j], 4, 4, 0, s.ws[i], 0, s.xs[j]);
    __builtin_amdgcn_sched_barrier(0);
  };
  // (an odd number of 128 k: the last stage's second half is 0)
  const bool short_end = (kq & 1) && blockIdx.y == gridDim.y - 1;
  load(0);
  load(1);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(XL + SL + WL + (RL > 0)) : "memory");
  block_barrier_nofence();
  read(a, 0, 0);
  for (int s = 0; s < ns; ++s) {
    const bool half_stage = short_end && s == ns - 1;
    read(b, s, 1);
    mma(a, false);
    if (!half_stage) {
      read(a, s, 2);
      mma(b, true);
      read(b, s, 3);
      mma(a, false);
    }
    // the next stage is there for every wave, and this one has been read by all
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    block_barrier_nofence();
    load(s + 2);
    read(a, s + 1, 0);
    mma(b, true);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the last loads, asked for but not used)
#pragma unroll
  for (int j = 0; j < MF; ++j) {
    const int m = m0 + (wm * MF + j) * 32 + r32;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const int n = group0 * 64 + (wn * NF + i) * 32;
      if (p.parts) {
        if (m < p.M)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int f = n + 8 * e + 4 * half;
            if (f < p.N)
              *(f32x4*)(p.parts + ((size_t)blockIdx.y * p.M + m) * p.part_ld + f) =
                  (f32x4){acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
          }
      } else {
        mx_store32<TY>(p, m, n, acc[i][j], m < p.M);
      }
    }
  }
}

// scales of 4-bit rows with whole dwords a row: [M][kq][4], 127 past K
__global__ __launch_bounds__(256) void mx_spread_scales_kernel(const uint8_t* __restrict__ scales, long total, int kb, int kq,
                                                               uint32_t* __restrict__ out) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const long m = i / kq;
  const int q = (int)(i - m * kq);
  uint32_t v = 0;
#pragma unroll
  for (int t = 0; t < 4; ++t) v |= (q * 4 + t < kb ? (uint32_t)scales[(size_t)m * kb + q * 4 + t] : 127u) << (8 * t);
  out[i] = v;
}

// y = the sum of the parts, in their order.  Four features a thread.
template <typename TY>
__global__ __launch_bounds__(256) void mx_join_kernel(MxProduct p, int parts) {
  const int f = (blockIdx.x * 256 + threadIdx.x) * 4, m = blockIdx.y;
  if (f >= p.N) return;
  const float* from = p.parts + (size_t)m * p.part_ld + f;
  f32x4 v[kMxParts];
#pragma unroll
  for (int z = 0; z < kMxParts; ++z) v[z] = *(const f32x4*)(from + (size_t)(z < parts ? z : 0) * p.M * p.part_ld);
#pragma unroll
  for (int z = 1; z < kMxParts; ++z)
    if (z < parts) v[0] += v[z];
  mx_store<TY>(p, m, f, v[0]);
}

// ---- launchers ------------------------------------------------------------------------------------
size_t mx_packed_bytes(int n, int kb) { return (size_t)((n + 63) / 64) * mx_tiles_of_k(kb) * kMxGroupBytes; }

// A launch takes fewer than 2^32 threads: rows of more go in several, each of up to 2^31 threads (`per_row` of them a row).
template <typename F> static void in_slices(long rows, long per_row, F launch) {
  const long most = (1l << 31) / per_row;   // (8192 and more)
  for (long r = 0; r < rows; r += most) {
    const long n = rows - r < most ? rows - r : most;
    launch(r, n, (unsigned)((n * per_row + 255) / 256));
  }
}
template <typename T>
static void launch_quantize_t(const T* x, long rows, int kb, size_t ld, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const bool wide = (uintptr_t)x % 16 == 0 && (ld * sizeof(T)) % 16 == 0;
  in_slices(rows, kb * 4, [&](long r, long n, unsigned grid) {
    const T* from = x + (size_t)r * ld;
    uint8_t *c = codes + (size_t)r * kb * 16, *e = scales + (size_t)r * kb;
    if (wide) mx_quantize_kernel<T, true><<<grid, 256, 0, s>>>(from, n, kb, ld, c, e);
    else mx_quantize_kernel<T, false><<<grid, 256, 0, s>>>(from, n, kb, ld, c, e);
  });
}
void launch_mx_quantize(const void* x, bool bf16, long rows, int kb, size_t ld, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  if (bf16) launch_quantize_t((const bf16_t*)x, rows, kb, ld, codes, scales, s);
  else launch_quantize_t((const float*)x, rows, kb, ld, codes, scales, s);
}

template <typename T>
static void launch_dequantize_t(const uint8_t* codes, const uint8_t* scales, long rows, int kb, T* out, size_t ld, hipStream_t s) {
  const bool wide = (uintptr_t)out % 16 == 0 && (ld * sizeof(T)) % 16 == 0;
  in_slices(rows, kb * 4, [&](long r, long n, unsigned grid) {
    const uint8_t *c = codes + (size_t)r * kb * 16, *e = scales + (size_t)r * kb;
    T* to = out + (size_t)r * ld;
    if (wide) mx_dequantize_kernel<T, true><<<grid, 256, 0, s>>>(c, e, n, kb, to, ld);
    else mx_dequantize_kernel<T, false><<<grid, 256, 0, s>>>(c, e, n, kb, to, ld);
  });
}
void launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, long rows, int kb, void* out, bool bf16, size_t ld,
                          hipStream_t s) {
  if (bf16) launch_dequantize_t(codes, scales, rows, kb, (bf16_t*)out, ld, s);
  else launch_dequantize_t(codes, scales, rows, kb, (float*)out, ld, s);
}

void launch_mx_pack(const uint8_t* codes, const uint8_t* scales, int n, int kb, uint8_t* packed, hipStream_t s) {
  const int kq = mx_tiles_of_k(kb);
  in_slices((n + 63) / 64, kq * 256l, [&](long g, long count, unsigned grid) {   // groups of 64 rows
    mx_pack_kernel<<<grid, 256, 0, s>>>(codes + (size_t)g * 64 * kb * 16, scales + (size_t)g * 64 * kb, (int)(n - g * 64), kb, count * kq * 256,
                                        packed + (size_t)g * kq * kMxGroupBytes);
  });
}

constexpr int mx_rows_lds(int xf, int mt, int ntw, int ks, int nw = 1) {
  const int ring = xf == MX_RING ? ks * 2 * mt * 4096 : 0, sums = ks * nw * ntw * mt * 1024;
  return ring > sums ? ring : sums;
}
template <int XF, typename TY, int MT, int NTW, int KS, int NW = 1>
static void launch_rows_t(const MxProduct& p, int parts, hipStream_t s) {
  constexpr int smem = mx_rows_lds(XF, MT, NTW, KS, NW);
  static_assert(smem <= 160 * 1024, "the rings and the waves' sums fit the LDS");
  if constexpr (smem > 48 * 1024) {
    static std::atomic<uint64_t> done{0};
    allow_lds((const void*)mx_rows_kernel<XF, TY, MT, NTW, KS, NW>, smem, done);
  }
  const int tiles = (p.N + 15) / 16;
  MxProduct q = p;
  if (parts == 1) q.parts = nullptr;
  mx_rows_kernel<XF, TY, MT, NTW, KS, NW><<<dim3((tiles + NW * NTW - 1) / (NW * NTW), parts), KS * NW * 64, smem, s>>>(q);
  if (parts > 1) mx_join_kernel<TY><<<dim3((p.N + 1023) / 1024, p.M), 256, 0, s>>>(p, parts);
}

constexpr int kMxRegisterRows = 4;   // rows of bf16 that a wave loads into registers, past LDS
// Where waves share their rows in LDS: from more features on than 256 blocks of 128 give each compute unit one (512 for up to 16 rows, whose
// share of the traffic is small).  Blocks of 256 features once there would be more than three blocks of 128 a unit, of which two share K where
// the registers let two blocks lie on a unit (up to 32 rows) and each unit has its two.  us at K 4096, f32 results, for 16 / 32 / 48 / 64 rows (256 features without / with halves of K):
//   features   alone            128 shared     256 shared     256 in halves
//     40960    21  47  57  66   26 27 31 34    36 40 43 49    30 33  38  42
//     65536    28  39  45  52   27 30 35 41    38 42 45 51    33 36  40  45
//     98304    41  57  66  75   38 45 52 68    45 51 59 72    43 46  75  83
//    131072    54  79  89 100   50 65 75 81    48 56 66 79    47 53  82  88
//    262144   113 149 170 196  102 125 135 160  93 117 134 155  99 109 157 171
enum { MX_ALONE, MX_SHARED_128, MX_SHARED_256, MX_SHARED_256_HALVES };
static int pick_shared(bool x4, int M, int N) {
  if (x4 || M <= kMxRegisterRows) return MX_ALONE;
  const int tiles = (N + 15) / 16, blocks128 = (tiles + 7) / 8, blocks256 = (tiles + 15) / 16;
  if (blocks128 <= (M <= 16 ? 512 : 256)) return MX_ALONE;
  if (blocks128 <= 768) return MX_SHARED_128;
  return M <= 32 && blocks256 <= 512 ? MX_SHARED_256_HALVES : MX_SHARED_256;
}
// Tiles of features to a block and ranges of K.  A compute unit pulls about 50 KB/us in these kernels, so that what counts is what goes
// through the busiest of the 256: its blocks' shares of W and, once a block, the rows; a join of K's ranges is another 3.5 us.  (Rows are counted by
// fours.  A ring brings whole tiles of 16, the first row's bytes for those that are not there; the rate is what fits the measured times so.)
struct MxRowsShape { int ntw, parts, shared; };
static MxRowsShape pick_rows(bool x4, int M, int N, int kb) {
  const int tiles = (N + 15) / 16, rows = (M + 3) / 4 * 4;
  MxRowsShape best = {4, 1, pick_shared(x4, M, N)};
  if (best.shared != MX_ALONE) return best;
  double least = 1e30;
  for (const int ntw : {1, 2, 4, 6, 8})
    for (const int parts : {1, 2, 4}) {
      if (parts > 1 && mx_tiles_of_k(kb) < 8 * parts) continue;
      const int blocks = (tiles + ntw - 1) / ntw * parts;
      const double kbytes = (ntw * 16 * 17.0 + rows * (x4 ? 17.0 : 64.0)) * kb / parts / 1000;
      const double us = (blocks + 255) / 256 * kbytes / 50 + (parts > 1 ? 3.5 : 0);
      if (us < least) { least = us; best = {ntw, parts, MX_ALONE}; }
    }
  return best;
}
template <int XF, typename TY, int MT>
static void launch_rows_mt(const MxProduct& p, hipStream_t s) {
  const MxRowsShape w = pick_rows(XF == MX_X4, p.M, p.N, p.kb);
  if constexpr (XF == MX_RING) {
    switch (w.shared) {
      case MX_SHARED_128: launch_rows_t<XF, TY, MT, 4, 2, 2>(p, 1, s); return;
      case MX_SHARED_256: launch_rows_t<XF, TY, MT, 4, 1, 4>(p, 1, s); return;
      case MX_SHARED_256_HALVES:
        if constexpr (MT <= 2) { launch_rows_t<XF, TY, MT, 4, 2, 4>(p, 1, s); return; }
        break;
      default: break;
    }
  }
  // (eight waves where a compute unit has one block, and LDS for it)
  const bool eight = MT == 1 && ((p.N + 15) / 16 + w.ntw - 1) / w.ntw * w.parts <= 256;
  constexpr int K1 = mx_rows_lds(XF, MT, 1, 8) <= 160 * 1024 ? 8 : 4, E = MT == 1 ? 8 : 4;
  switch (w.ntw) {
    case 1: launch_rows_t<XF, TY, MT, 1, K1>(p, w.parts, s); break;
    case 2: if (eight) launch_rows_t<XF, TY, MT, 2, E>(p, w.parts, s); else launch_rows_t<XF, TY, MT, 2, 4>(p, w.parts, s); break;
    case 4: if (eight) launch_rows_t<XF, TY, MT, 4, E>(p, w.parts, s); else launch_rows_t<XF, TY, MT, 4, 4>(p, w.parts, s); break;
    case 6: if (eight) launch_rows_t<XF, TY, MT, 6, E>(p, w.parts, s); else launch_rows_t<XF, TY, MT, 6, 4>(p, w.parts, s); break;
    default: if (eight) launch_rows_t<XF, TY, MT, 8, E>(p, w.parts, s); else launch_rows_t<XF, TY, MT, 8, 4>(p, w.parts, s); break;
  }
}

template <bool X4, typename TY, int WM, int WN, int WTM>
static void launch_tiled_t(const MxProduct& p, int parts, hipStream_t s) {
  typedef MxTile<X4, WM, WN, WTM> T;
  constexpr int smem = T::STAGE * T::S;
  static_assert(smem <= 160 * 1024, "the stages fit the LDS");
  static std::atomic<uint64_t> done{0};
  allow_lds((const void*)mx_tiled_kernel<X4, TY, WM, WN, WTM>, smem, done);
  MxProduct q = p;
  if (parts == 1) q.parts = nullptr;
  const int gx = (p.N + T::BN - 1) / T::BN, gy = (p.M + T::BM - 1) / T::BM;
  mx_tiled_kernel<X4, TY, WM, WN, WTM><<<dim3(gx * gy, parts), 512, smem, s>>>(q);
  if (parts > 1) mx_join_kernel<TY><<<dim3((p.N + 1023) / 1024, p.M), 256, 0, s>>>(p, parts);
}

template <typename TY, int WM, int WN, int MF, int NF>
static void launch_tiled4_t(const MxProduct& p, int parts, hipStream_t s) {
  typedef MxTile4<WM, WN, MF, NF> T;
  constexpr int smem = T::STAGE * 2;
  static_assert(smem <= 160 * 1024, "the stages fit the LDS");
  static std::atomic<uint64_t> done{0};
  allow_lds((const void*)mx_tiled4_kernel<TY, WM, WN, MF, NF>, smem, done);
  MxProduct q = p;
  if (parts == 1) q.parts = nullptr;
  const int gx = (p.N + T::BN - 1) / T::BN, gy = (p.M + T::BM - 1) / T::BM;
  mx_tiled4_kernel<TY, WM, WN, MF, NF><<<dim3(gx * gy, parts), 512, smem, s>>>(q);
  if (parts > 1) mx_join_kernel<TY><<<dim3((p.N + 1023) / 1024, p.M), 256, 0, s>>>(p, parts);
}

// Rows x features of a block and ranges of K, by what its rounds of 256 blocks take.  us a stage (128 k of bf16 rows, 256 k of 4-bit ones) and beside
// the stages, from whole products of K 4096:
//   bf16   128 x 256 1.65 + 3   64 x 256 1.05 + 3   128 x 128 1.05 + 3
//   4 bits 64 x 256 1.00 + 3    128 x 128 1.00 + 3  (16x16x128: quicker to start)
//          256 x 256 2.50 + 4.5 192 x 384 2.90 + 4.5  128 x 256 1.40 + 4.5  192 x 256 2.00 + 4.5  (32x32x64)
enum { MX_128x256, MX_64x256, MX_128x128, MX_256x256_4, MX_192x384_4, MX_128x256_4, MX_192x256_4, MX_SHAPES };
static const int kMxBlockRows[MX_SHAPES] = {128, 64, 128, 256, 192, 128, 192}, kMxBlockCols[MX_SHAPES] = {256, 256, 128, 256, 384, 256, 256};
struct MxTiledShape { int shape, parts; };
static MxTiledShape pick_tiled(bool x4, int M, int N, int kb) {
  const int *bm = kMxBlockRows, *bn = kMxBlockCols;
  static const double us16[MX_SHAPES] = {1.65, 1.05, 1.05}, us4[MX_SHAPES] = {0, 1.0, 1.0, 2.5, 2.9, 1.4, 2.0};
  const int stages = x4 ? (mx_tiles_of_k(kb) + 1) / 2 : mx_tiles_of_k(kb);
  MxTiledShape best = {MX_128x128, 1};
  double least = 1e30;
  for (int shape = x4 ? 1 : 0; shape < (x4 ? MX_SHAPES : 3); ++shape)
    for (const int parts : {1, 2, 4}) {
      if (parts > 1 && (M > kMxSplitRows || stages < 4 * parts)) continue;
      const long blocks = (long)((M + bm[shape] - 1) / bm[shape]) * ((N + bn[shape] - 1) / bn[shape]) * parts;
      const double us = (double)((blocks + 255) / 256) * (((stages + parts - 1) / parts) * (x4 ? us4 : us16)[shape] + (shape < 3 ? 3 : 4.5)) +
                        (parts > 1 ? 4 + (parts + 1) * 4.0 * M * N / 4e6 : 0);
      if (us < least) { least = us; best = {shape, parts}; }
    }
  return best;
}
template <bool X4, typename TY>
static void launch_tiled(const MxProduct& p, hipStream_t s) {
  const MxTiledShape w = pick_tiled(X4, p.M, p.N, p.kb);
  if (w.shape == MX_64x256) { launch_tiled_t<X4, TY, 2, 4, 2>(p, w.parts, s); return; }
  if (w.shape == MX_128x128) { launch_tiled_t<X4, TY, 4, 2, 2>(p, w.parts, s); return; }
  if constexpr (!X4) launch_tiled_t<false, TY, 2, 4, 4>(p, w.parts, s);
  else if (w.shape == MX_256x256_4) launch_tiled4_t<TY, 2, 4, 4, 2>(p, w.parts, s);
  else if (w.shape == MX_192x384_4) launch_tiled4_t<TY, 2, 4, 3, 3>(p, w.parts, s);
  else if (w.shape == MX_128x256_4) launch_tiled4_t<TY, 2, 4, 2, 2>(p, w.parts, s);
  else launch_tiled4_t<TY, 2, 4, 3, 2>(p, w.parts, s);
}

constexpr int kMxFewRows = 64;   // up to here W is streamed past all rows at once
void mx_linear_blocks(bool x4, long M, int N, int kb, int32_t shape[3]) {
  if (M <= kMxFewRows) {
    const MxRowsShape w = pick_rows(x4, (int)M, N, kb);
    shape[0] = (int)((M + 15) / 16 * 16);
    shape[1] = w.shared == MX_ALONE ? w.ntw * 16 : w.shared == MX_SHARED_128 ? 128 : 256;
    shape[2] = w.parts;
  } else {
    const MxTiledShape w = pick_tiled(x4, (int)M, N, kb);
    shape[0] = kMxBlockRows[w.shape];
    shape[1] = kMxBlockCols[w.shape];
    shape[2] = w.parts;
  }
}
template <bool X4, typename TY>
static void launch_linear_t(const MxProduct& p, hipStream_t s) {
  constexpr int XF = X4 ? MX_X4 : MX_RING;
  switch ((p.M + 15) / 16) {
    case 1: if (p.M <= kMxRegisterRows) launch_rows_mt<X4 ? MX_X4 : MX_REGS, TY, 1>(p, s); else launch_rows_mt<XF, TY, 1>(p, s); break;
    case 2: launch_rows_mt<XF, TY, 2>(p, s); break;
    case 3: launch_rows_mt<XF, TY, 3>(p, s); break;
    case 4: launch_rows_mt<XF, TY, 4>(p, s); break;
    default: {
      MxProduct q = p;
      if (X4 && (p.kb % 4 || (uintptr_t)p.x_scales % 4)) {
        const int kq = mx_tiles_of_k(p.kb);
        const long total = (long)p.M * kq;
        mx_spread_scales_kernel<<<(unsigned)((total + 255) / 256), 256, 0, s>>>(p.x_scales, total, p.kb, kq, (uint32_t*)p.spread);
        q.x_scales = p.spread;
        q.scale_ld = kq * 4;
      }
      launch_tiled<X4, TY>(q, s);
    }
  }
}

// parts' sums [ranges][M][N], then the scales of 4-bit rows in whole dwords.  (These may be wanted for scales that begin at any byte, which is not
// known here.)
static size_t mx_sums_bytes(int parts, long M, int N) {
  return parts > 1 ? ((size_t)parts * M * ((N + 3) / 4 * 4) * sizeof(float) + 255) / 256 * 256 : 0;
}
static size_t mx_parts_bytes(bool x4, long M, int N, int kb) {
  return mx_sums_bytes(M <= kMxFewRows ? pick_rows(x4, (int)M, N, kb).parts : pick_tiled(x4, (int)M, N, kb).parts, M, N);
}
// Ranges of K by the rows there are: pick_rows goes by fours of rows; of 64 that begin at a multiple of 64, what pick_tiled compares differs by the
// join alone, which costs more the more ranges and rows there are, so that the first row has the most ranges.  Found once for the shapes that
// a thread has in hand (2 us, where a call takes 9).
struct MxRanges {
  static constexpr int FEW = kMxFewRows / 4, ALL = FEW + (kMxSplitRows - kMxFewRows) / 64;
  int n = 0, kb = 0;
  bool x4 = false;
  uint8_t parts[ALL] = {};
  static long last(int i) { return i < FEW ? 4 * i + 4 : kMxFewRows + 64l * (i - FEW + 1); }
  static const MxRanges& of(bool x4, int N, int kb) {
    static thread_local MxRanges known[64];
    MxRanges& r = known[((uint32_t)N * 2654435761u ^ (uint32_t)(kb * 2 + x4) * 2246822519u) >> 26];
    if (r.n != N || r.kb != kb || r.x4 != x4) {
      for (int i = 0; i < ALL; ++i) {
        const int m = i ? (int)last(i - 1) + 1 : 1;
        r.parts[i] = (uint8_t)(i < FEW ? pick_rows(x4, m, N, kb).parts : pick_tiled(x4, m, N, kb).parts);
      }
      r.n = N; r.kb = kb; r.x4 = x4;
    }
    return r;
  }
};
// room for M rows or fewer
size_t mx_linear_workspace(bool x4, long M, int N, int kb) {
  const MxRanges& ranges = MxRanges::of(x4, N, kb);
  size_t most = 0;
  for (int i = 0; i < MxRanges::ALL && (i == 0 || MxRanges::last(i - 1) < M); ++i) {
    const long m = MxRanges::last(i) < M ? MxRanges::last(i) : M;
    if (ranges.parts[i] > 1) most = most > mx_sums_bytes(ranges.parts[i], m, N) ? most : mx_sums_bytes(ranges.parts[i], m, N);
  }
  return most + (x4 && M > kMxFewRows ? (size_t)M * mx_tiles_of_k(kb) * 4 : 0);
}

void launch_mx_linear(const void* x, const uint8_t* x_scales, long M, size_t ld, const uint8_t* packed, int N, int kb, void* y,
                      bool y_bf16, size_t ldy, void* workspace, hipStream_t s) {
  const int wide = N % 4 == 0 && ldy % 4 == 0 && (uintptr_t)y % (y_bf16 ? 8 : 16) == 0;
  const int wide16 = N % 8 == 0 && ldy % 8 == 0 && (uintptr_t)y % 16 == 0;
  uint8_t* spread = (uint8_t*)workspace + mx_parts_bytes(x_scales != nullptr, M, N, kb);
  const MxProduct p = {x, x_scales, ld, kb, packed, (int)M, N, kb, y, ldy, wide, wide16, spread, (float*)workspace, (N + 3) / 4 * 4};
  if (x_scales) {
    if (y_bf16) launch_linear_t<true, bf16_t>(p, s);
    else launch_linear_t<true, float>(p, s);
  } else {
    if (y_bf16) launch_linear_t<false, bf16_t>(p, s);
    else launch_linear_t<false, float>(p, s);
  }
}

}  // namespace ec
