// Rotary positions: pairs of a head's components turned by an angle that grows with the row's position.
//
// Pair i of dim/2 at position p turns by a = 2 pi p turns[i]:  (x, y) -> A (x cos a - y sin a, x sin a + y cos a), with -a for the
// inverse, which is the transposed rotation and so the gradient's.  The whole turns are dropped in 64 bits, where p turns[i] is exact
// to 2^-53 of itself: at position 2^20 and a turn in 6 positions the angle is off by 2^-33.
#include "ec_internal.h"

namespace ec {

namespace {

// cos and sin of 2 pi t.  t less its nearest quarter, exactly, leaves at most an eighth of a turn, y in [-pi/4, pi/4]; Taylor's series to
// y^9 and y^10 are off by less than 2e-9 there, below the rounding of float32 (6e-8).
__device__ __forceinline__ float2 cos_sin_of_turns(double t) {
  const double quarters = __builtin_rint(t * 4.0);
  const float y = (float)((t - 0.25 * quarters) * 6.283185307179586);
  const int q = (int)(quarters - 4.0 * __builtin_floor(quarters * 0.25));
  const float z = y * y;
  const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const float a = q & 1 ? s : c, b = q & 1 ? c : s;
  return make_float2(q == 1 || q == 2 ? -a : a, q == 2 || q == 3 ? -b : b);
}

template <typename T, int N> struct alignas(sizeof(T) * N) Words { T v[N]; };

}  // namespace

struct RotaryArgs {
  const void* x; void* out;
  size_t ld, ld_head, out_ld, out_ld_head;
  long rows;
  int heads, head_dim, dim;
  const int* positions; const double* turns;
  float amplitude, sign;   // sign: -1 for the inverse
};

// A block takes RB rows with all their heads: first the rows' cosines and sines into LDS, once for all heads, then the pairs, V of them to
// a thread at a time (V elements of each half, or 2 V neighbours).  Bytes bound it: 24576 rows of 64 heads of 128 in bfloat16 take 145 us, 5.5 TB/s
// both ways (a copy: 5.2); one row takes 3.3.
template <typename T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int RB) {
  extern __shared__ float2 cs[];   // [RB][dim/2]
  const int half = a.dim >> 1, per_head = half / V, per_row = a.heads * per_head;
  const long row0 = (long)blockIdx.x * RB;
  const int n = (int)min((long)RB, a.rows - row0);
  for (int i = threadIdx.x; i < n * half; i += 256) {
    const int r = i / half;
    const float2 v = cos_sin_of_turns((double)a.positions[row0 + r] * a.turns[i - r * half]);
    cs[i] = make_float2(v.x * a.amplitude, v.y * a.amplitude * a.sign);
  }
  __syncthreads();
  typedef Words<T, V> W;
  for (int i = threadIdx.x; i < n * per_row; i += 256) {
    const int r = i / per_row, j = i - r * per_row, head = j / per_head, p = (j - head * per_head) * V;
    const size_t at = (size_t)(row0 + r) * a.ld + (size_t)head * a.ld_head;
    const size_t to = (size_t)(row0 + r) * a.out_ld + (size_t)head * a.out_ld_head;
    const int c0 = INTERLEAVED ? 2 * p : p, c1 = INTERLEAVED ? 2 * p + V : p + half;
    alignas(16) T v[2 * V];
    *(W*)v = *(const W*)((const T*)a.x + at + c0);
    *(W*)(v + V) = *(const W*)((const T*)a.x + at + c1);
    const float2* f = cs + r * half + p;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      T &s = v[INTERLEAVED ? 2 * k : k], &t = v[INTERLEAVED ? 2 * k + 1 : k + V];
      const float x = load_f32(&s), y = load_f32(&t);
      store_f32(&s, fmaf(x, f[k].x, -(y * f[k].y)));
      store_f32(&t, fmaf(x, f[k].y, y * f[k].x));
    }
    *(W*)((T*)a.out + to + c0) = *(const W*)v;
    *(W*)((T*)a.out + to + c1) = *(const W*)(v + V);
  }
  // the components that do not turn
  const int rest = (a.head_dim - a.dim) / V;
  if (a.x == a.out || rest == 0) return;
  for (int i = threadIdx.x; i < n * a.heads * rest; i += 256) {
    const int r = i / (a.heads * rest), j = i - r * (a.heads * rest), head = j / rest, c = a.dim + (j - head * rest) * V;
    *(W*)((T*)a.out + (size_t)(row0 + r) * a.out_ld + (size_t)head * a.out_ld_head + c) =
        *(const W*)((const T*)a.x + (size_t)(row0 + r) * a.ld + (size_t)head * a.ld_head + c);
  }
}

// Where pairs do not lie on multiples of 16 bytes but heads do: a head goes through LDS, read and written in pieces of 16 bytes, and a thread
// finds the partners of its V components there.  Items of whole heads; HB of them to a block at a time.
template <typename T, int V>
__global__ __launch_bounds__(256) void rotary_any_kernel(RotaryArgs a, bool interleaved, int HB) {
  extern __shared__ float2 cs[];   // [HB][dim/2], then the heads
  const int half = a.dim >> 1, pieces = a.head_dim / V;
  T* x = (T*)(cs + (HB * half + 1) / 2 * 2);
  const long item0 = (long)blockIdx.x * HB, items = a.rows * a.heads;
  const int n = (int)min((long)HB, items - item0);
  const long row0 = item0 / a.heads;
  const int rows = (int)((item0 + n - 1) / a.heads - row0) + 1;
  typedef Words<T, V> W;
  for (int i = threadIdx.x; i < n * pieces; i += 256) {
    const int h = i / pieces, c = (i - h * pieces) * V;
    const long row = (item0 + h) / a.heads, head = item0 + h - row * a.heads;
    *(W*)(x + h * a.head_dim + c) = *(const W*)((const T*)a.x + (size_t)row * a.ld + (size_t)head * a.ld_head + c);
  }
  for (int i = threadIdx.x; i < rows * half; i += 256) {
    const int r = i / half;
    const float2 v = cos_sin_of_turns((double)a.positions[row0 + r] * a.turns[i - r * half]);
    cs[i] = make_float2(v.x * a.amplitude, v.y * a.amplitude * a.sign);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * pieces; i += 256) {
    const int h = i / pieces, c0 = (i - h * pieces) * V;
    const long row = (item0 + h) / a.heads, head = item0 + h - row * a.heads;
    if (c0 >= a.dim && a.x == a.out) continue;
    const T* p = x + h * a.head_dim;
    const float2* f = cs + (row - row0) * half;
    alignas(16) T v[V];
    *(W*)v = *(const W*)(p + c0);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int c = c0 + e;
      if (c < a.dim) {
        const int pair = interleaved ? c >> 1 : c < half ? c : c - half;
        const bool first = interleaved ? !(c & 1) : c < half;
        const float mine = load_f32(p + c), other = load_f32(p + (interleaved ? c ^ 1 : first ? c + half : c - half));
        store_f32(v + e, first ? fmaf(mine, f[pair].x, -(other * f[pair].y)) : fmaf(other, f[pair].y, mine * f[pair].x));
      }
    }
    *(W*)((T*)a.out + (size_t)row * a.out_ld + (size_t)head * a.out_ld_head + c0) = *(const W*)v;
  }
}

template <typename T, int V>
static void launch_rotary_any(const RotaryArgs& a, bool interleaved, hipStream_t s) {
  const int HB = min(min(2048 / (a.head_dim / V), 32), 60000 / (a.dim / 2 * (int)sizeof(float2) + a.head_dim * (int)sizeof(T)));   // (what fits LDS: 11 or more)
  const size_t lds = ((size_t)HB * (a.dim / 2) + 1) / 2 * 2 * sizeof(float2) + (size_t)HB * a.head_dim * sizeof(T);
  const long blocks = (a.rows * a.heads + HB - 1) / HB;
  rotary_any_kernel<T, V><<<(unsigned)blocks, 256, lds, s>>>(a, interleaved, HB);
}

template <typename T, int V>
static void launch_rotary_v(const RotaryArgs& a, bool interleaved, hipStream_t s) {
  // about 1024 pieces of V pairs to a block
  const long per_row = (long)a.heads * (a.dim / 2 / V);
  const int RB = (int)max(1L, min(16L, 1024 / per_row));
  const size_t lds = (size_t)RB * (a.dim / 2) * sizeof(float2);
  const long blocks = (a.rows + RB - 1) / RB;
  if (interleaved) rotary_kernel<T, V, true><<<(unsigned)blocks, 256, lds, s>>>(a, RB);
  else rotary_kernel<T, V, false><<<(unsigned)blocks, 256, lds, s>>>(a, RB);
}

static void launch_rotary_rows(const RotaryArgs& a, bool bf16, bool interleaved, hipStream_t s) {
  // the largest power of two that everything is a multiple of
  const size_t es = bf16 ? 2 : 4, strides = a.ld | a.ld_head | a.out_ld | a.out_ld_head;
  const size_t all = strides | (size_t)(a.dim / 2) | (size_t)(a.head_dim - a.dim) | (size_t)a.x / es | (size_t)a.out / es;
  const int v = all % 8 == 0 && bf16 ? 8 : all % 4 == 0 ? 4 : all % 2 == 0 ? 2 : 1;
  // (24576 x 64 heads of 128 in bfloat16, of which 38 components turn: 360 us pair by pair, 223 through LDS)
  const size_t whole = (strides | (size_t)a.head_dim) * es | (size_t)a.x | (size_t)a.out;
  if (v < (bf16 ? 4 : 2) && whole % 16 == 0 && (a.rows > 1 || a.heads > 1)) {
    if (bf16) launch_rotary_any<bf16_t, 8>(a, interleaved, s);
    else launch_rotary_any<float, 4>(a, interleaved, s);
    return;
  }
  if (bf16) {
    if (v == 8) launch_rotary_v<bf16_t, 8>(a, interleaved, s);
    else if (v == 4) launch_rotary_v<bf16_t, 4>(a, interleaved, s);
    else if (v == 2) launch_rotary_v<bf16_t, 2>(a, interleaved, s);
    else launch_rotary_v<bf16_t, 1>(a, interleaved, s);
  } else {
    if (v == 4) launch_rotary_v<float, 4>(a, interleaved, s);
    else if (v == 2) launch_rotary_v<float, 2>(a, interleaved, s);
    else launch_rotary_v<float, 1>(a, interleaved, s);
  }
}

void launch_rotary(const void* x, bool bf16, long rows, int heads, int head_dim, size_t ld, size_t ld_head, const int* positions,
                   const double* turns, int dim, bool interleaved, float amplitude, bool inverse, void* out, size_t out_ld,
                   size_t out_ld_head, hipStream_t s) {
  // A launch has less than 2^32 threads: of 2^23 heads, or of one row, both kernels take fewer than 2^23 blocks of 256
  const long most = max(1L, (1L << 23) / heads);
  const size_t es = bf16 ? 2 : 4;
  for (long r = 0; r < rows; r += most)
    launch_rotary_rows({(const char*)x + r * ld * es, (char*)out + r * out_ld * es, ld, ld_head, out_ld, out_ld_head, min(most, rows - r), heads,
                        head_dim, dim, positions + r, turns, amplitude, inverse ? -1.f : 1.f}, bf16, interleaved, s);
}

}  // namespace ec
