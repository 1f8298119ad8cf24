// A paged cache of keys and values, laid out as the attention's matrix products read it.
//
// A page holds `page` tokens (32, 64, 128 or 256) of every kv head; 32 tokens of a head are a chunk: [page][kv head][chunk of the page].
// A chunk has its keys, then its values, each 32 x HD elements of ES bytes (1: e4m3 codes, 2: bfloat16), in lanes' pieces of 16 bytes:
//   keys    tile t (2), unit u, lane g*16 + i: key (i/4)*8 + t*4 + (i%4) of the chunk, components g*HD/4 + u*(16/ES) and on.  A tile is
//           the A operand of S^T = K Q^T; after both a lane has the scores of 8 neighbouring keys of one query.
//   values  tile h of HD/16, lane g*16 + j, keys g*8 .. g*8+7: the A operand of O^T = V^T P^T.  Tile 2 p + s has component
//           p*32 + (j/4)*8 + s*4 + (j%4) in its row j, so that a lane ends up with 8 neighbouring components of its query.  e4m3: the
//           tiles 2 p and 2 p + 1 share a lane's 16 bytes.
// Behind all chunks their scale bytes, [chunk][keys, values][token of the chunk]: s, for a power of two 2^(s - 127), or 255: the token's
// head is NaN.  (bfloat16: 127 or 255.)  The elements of such keys are NaN, those of such values 0: a key that a query does not see
// leaves its scores as they are, but a product of matrices also multiplies the values it does not see, by 0.
#pragma once
#include "ec_internal.h"

namespace ec {

constexpr int kKvChunk = 32;

template <int ES, int HD> struct KvChunk {
  static constexpr int kPart = kKvChunk * HD * ES;   // bytes of a chunk's keys, or values
  static constexpr int kBytes = 2 * kPart;
  static constexpr int kPer = 16 / ES;               // elements of a piece
  static constexpr int kUnits = HD / 4 / kPer;       // pieces of a lane in a tile of keys
  // byte of component c of token w, in the keys and in the values
  __host__ __device__ static constexpr int key_at(int w, int c) {
    const int i = (w >> 3) * 4 + (w & 3), t = (w >> 2) & 1, g = c / (HD / 4), u = c % (HD / 4) / kPer, e = c % kPer;
    return ((t * kUnits + u) * 64 + g * 16 + i) * 16 + e * ES;
  }
  __host__ __device__ static constexpr int value_at(int w, int c) {
    const int p = c >> 5, s = (c >> 2) & 1, j = ((c >> 3) & 3) * 4 + (c & 3), lane = (w >> 3) * 16 + j;
    return ES == 1 ? kPart + (p * 64 + lane) * 16 + s * 8 + (w & 7) : kPart + ((2 * p + s) * 64 + lane) * 16 + (w & 7) * 2;
  }
};

// where a slot (page * tokens of a page + token of the page) is
struct KvPlace {
  int shift;      // log2 of a page's chunks
  int kv_heads;
  __device__ __forceinline__ size_t chunk(int slot, int head) const {
    const int c = slot >> 5, page = c >> shift;
    return ((((size_t)page * kv_heads + head) << shift) + (c & ((1 << shift) - 1)));
  }
};

}  // namespace ec
