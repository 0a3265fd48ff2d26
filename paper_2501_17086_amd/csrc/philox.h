// Which elements dropout leaves out: the counter-based generator Philox4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel
// random numbers: as easy as 1, 2, 3", 2011), so that a mask is made again wherever it is needed and stored nowhere.
#pragma once
#include "hbp_common.h"

namespace hbp {

// Eight consecutive elements of a row are one call, 16 bits each: an element is left out where its bits are below the threshold, so
// rates are multiples of 2^-16.  (32 bits each would be two calls of 20 wide products: 16384 x 2048 in bf16 onto a residual 28.3 -> 29.0 us with the same
// rows again and again, which the memory side's cache holds.)
struct DropoutKey {
  unsigned k0, k1;            // seed
  unsigned long offset;
  const unsigned long* counter;   // added to offset, or NULL
  unsigned threshold;         // 0: nothing is left out
  float factor;               // 65536 / (65536 - threshold), times what else multiplies every element
};

// the stream of a call: offset and the counter on the device, read once a thread
__device__ __forceinline__ unsigned long dropout_stream(const DropoutKey& k) { return k.offset + (k.counter ? *k.counter : 0ul); }

// bit j: element 8 block + j stays
__device__ __forceinline__ unsigned dropout_mask8(const DropoutKey& k, unsigned long stream, unsigned long block) {
  unsigned c0 = (unsigned)block, c1 = (unsigned)(block >> 32), c2 = (unsigned)stream, c3 = (unsigned)(stream >> 32);
  unsigned k0 = k.k0, k1 = k.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long a = (unsigned long)c0 * 0xD2511F53u, b = (unsigned long)c2 * 0xCD9E8D57u;
    c0 = (unsigned)(b >> 32) ^ c1 ^ k0;
    c1 = (unsigned)b;
    c2 = (unsigned)(a >> 32) ^ c3 ^ k1;
    c3 = (unsigned)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  const unsigned w[4] = {c0, c1, c2, c3};
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m |= (unsigned)((w[j] & 0xFFFFu) >= k.threshold) << (2 * j);
    m |= (unsigned)((w[j] >> 16) >= k.threshold) << (2 * j + 1);
  }
  return m;
}

}  // namespace hbp
