// What the attention kernels share: 32 x 32 products on the matrix cores, LDS tiles of rows that direct copies fill, and the
// operand fragments read from them.
#pragma once
#include "hbp_common.h"

namespace hbp {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// mfma(X, Y, acc): lane l, element r of acc  +=  sum_k X[8 (r/4) + 4 (l/32) + r%4][k] * Y[l % 32][k], where for one
// step of 16 k-values a lane's 8 operand elements are k = 8 (l/32) .. + 7 of row l % 32 of X and of Y.  Only the
// pairing matters: element i of lane half hh of X meets element i of lane half hh of Y.
__device__ __forceinline__ float16v mfma(bf16x8 x, bf16x8 y, float16v acc) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, acc, 0, 0, 0);
}
__device__ __forceinline__ int tile_row_of(int r, int hh) { return 8 * (r >> 2) + 4 * hh + (r & 3); }
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32: exp2(-inf) = 0

// An LDS tile: 32 rows of one head, DHP columns of bf16 (DHP = 32, 64 or 128: the head width rounded up).  The 16-byte
// chunks of a row are spread over the 64 banks by an XOR: within any four consecutive rows the XOR (with the row's
// place in the 256 bytes that the banks span) moves a group of four chunks to four different places, which is what a
// transposing read of four rows touches at once, and within any sixteen rows it moves a single chunk to all places, for
// the reads along a row.
template <int DHP>
struct Geo {
  static constexpr int RB = 2 * DHP;                 // bytes per row
  static constexpr int TB = 32 * RB;                 // ... per tile
  static constexpr int CPR = RB / 16;                // chunks per row
  static constexpr int RPC = 64 / CPR;               // rows per copy of 1 KB
  static constexpr int COPIES = TB / 1024;           // copies per tile
  static constexpr int PW = 2 * COPIES / 4;          // copies per wavefront of a pair of tiles, four wavefronts sharing it
  static constexpr int KK = DHP / 16;                // steps of 16 columns
  static constexpr int MB = DHP / 32;                // blocks of 32 columns
  static __device__ __forceinline__ int swz(int r) {
    if (DHP == 32) return (r >> 2) & 3;
    if (DHP == 64) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    return ((r & 3) << 2) | ((r >> 2) & 3);
  }
};

// Addresses: a wavefront-uniform pointer to row 0 of the 32-row tile plus one 32-bit byte offset per lane, which is
// the same for every whole tile (computed once); a tile that runs past the last row re-reads that row instead.  A head
// narrower than DHP: the chunks past its width repeat its last one (finite wherever the head is) and meet zeros in the
// other operand of every product that contracts over them; results in those columns are not stored.
//
// Tiles reach LDS by direct copies (global_load_lds_dwordx4: 16 bytes per lane from memory to lds_base + 16 lane,
// no staging registers), issued steps ahead into a ring of buffers.  The chunk swizzle is applied on the memory side:
// LDS position (row r, slot c) receives chunk c ^ swz(r) of the row.  The compiler sees neither the LDS write nor when
// it lands: a counted wait (copies_in_flight) and the workgroup's barrier (workgroup_handover) come before the reads.
__device__ __forceinline__ void copy16_to_lds(unsigned off, const void* sbase_in, unsigned lds_base) {
  // (the base is uniform by construction; say so where the register allocator has moved it to vector registers)
  const unsigned long long b = reinterpret_cast<unsigned long long>(sbase_in);
  const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)b);
  const unsigned hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(b >> 32));
  const void* sbase = reinterpret_cast<const void*>((unsigned long long)lo | ((unsigned long long)hi << 32));
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n"
               :: "v"(off), "s"(sbase), "s"(lds_base) : "memory");
}
// the same from a per-lane address
__device__ __forceinline__ void copy16_from_to_lds(const void* gptr, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off\n" :: "v"(gptr), "s"(lds_base) : "memory");
}
// 4 bytes per lane from a per-lane address to lds_base + 4 lane
__device__ __forceinline__ void copy4_to_lds(const void* gptr, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off\n" :: "v"(gptr), "s"(lds_base) : "memory");
}
// this lane's byte offset into a tile (row stride ldb) for copy u, rows from rows_left on repeating the last one;
// dh8: chunks that the head has
template <int DHP>
__device__ __forceinline__ unsigned copy_offset(unsigned ldb, int u, int rows_left, int dh8, int lane) {
  typedef Geo<DHP> G;
  const int r = G::RPC * u + lane / G::CPR;
  int c = (lane % G::CPR) ^ G::swz(r);
  c = c < dh8 ? c : dh8 - 1;
  return (unsigned)(r < rows_left ? r : rows_left - 1) * ldb + (unsigned)c * 16u;
}
// a whole tile by one wavefront
template <int DHP>
__device__ __forceinline__ void copy_tile(const unsigned char* base, unsigned ldb, int rows_left, int dh8, unsigned lds_tile,
                                          int lane) {
#pragma unroll
  for (int u = 0; u < Geo<DHP>::COPIES; ++u)
    copy16_to_lds(copy_offset<DHP>(ldb, u, rows_left, dh8, lane), base, lds_tile + 1024u * u);
}
// A pair of tiles filled by the four wavefronts of a workgroup together, PW copies each: half of them of either tile
// (32 columns: one copy each, of the first tile by wavefronts 0 and 1).
template <int DHP>
struct PairCopy {
  typedef Geo<DHP> G;
  static constexpr int H = G::PW < 2 ? 1 : G::PW / 2;
  unsigned off[G::PW];
  static __device__ __forceinline__ int tile(int w, int i) { return G::PW == 1 ? w >> 1 : i / H; }
  static __device__ __forceinline__ int part(int w, int i) { return G::PW == 1 ? w & 1 : w * H + i % H; }
  static __device__ __forceinline__ unsigned offset(unsigned ldb0, unsigned ldb1, int rows_left, int dh8, int w, int i, int lane) {
    return copy_offset<DHP>(tile(w, i) ? ldb1 : ldb0, part(w, i), rows_left, dh8, lane);
  }
  __device__ __forceinline__ PairCopy(unsigned ldb0, unsigned ldb1, int dh8, int w, int lane) {
#pragma unroll
    for (int i = 0; i < G::PW; ++i) off[i] = offset(ldb0, ldb1, 32, dh8, w, i, lane);
  }
  // rows_left < 32: the tile that runs past the last row
  __device__ __forceinline__ void issue(const unsigned char* t0, const unsigned char* t1, unsigned ldb0, unsigned ldb1, int rows_left,
                                        int dh8, unsigned lds_pair, int w, int lane) const {
    const unsigned dst = lds_pair + (unsigned)(G::PW == 1 ? w : w * H) * 1024u;
    if (rows_left >= 32) {
#pragma unroll
      for (int i = 0; i < G::PW; ++i)
        copy16_to_lds(off[i], tile(w, i) ? t1 : t0, dst + (G::PW == 1 ? 0u : (unsigned)(i / H) * G::TB + (unsigned)(i % H) * 1024u));
    } else {
#pragma unroll
      for (int i = 0; i < G::PW; ++i)
        copy16_to_lds(offset(ldb0, ldb1, rows_left, dh8, w, i, lane), tile(w, i) ? t1 : t0,
                      dst + (G::PW == 1 ? 0u : (unsigned)(i / H) * G::TB + (unsigned)(i % H) * 1024u));
    }
  }
};
// at most N of this wavefront's copies still in flight (they land in issue order)
template <int N>
__device__ __forceinline__ void copies_in_flight() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}
// ... and no LDS read either: the buffer that the next copies go to has been read
template <int N>
__device__ __forceinline__ void copies_in_flight_read() {
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// A value loaded from memory before the loop is made to arrive here.  Without this the compiler places its own counted
// waits for such loads at their first use inside the loop, and since it does not know of the direct copies, those
// waits would also drain the copies that were just issued for three steps ahead, on every step.
template <typename V>
__device__ __forceinline__ void landed(V& v) {
  asm volatile("" : "+v"(v));
}
// every wavefront of the workgroup has passed its wait: the tile is complete, and the buffer of the step before is free
__device__ __forceinline__ void workgroup_handover() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ unsigned lds_address(const void* p) {
  return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)p;
}
// operand fragment with the contraction along the tile's columns (step kk of 16 columns): lane holds row l % 32
template <int DHP>
__device__ __forceinline__ bf16x8 frag_cols_lds(const unsigned char* tile, int kk, int lane) {
  typedef Geo<DHP> G;
  const int r = lane & 31, ch = 2 * kk + (lane >> 5);
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(tile + r * G::RB + ((ch ^ G::swz(r)) << 4)));
}
// the same, zero past the head's width (the operand that is kept in registers)
template <int DHP>
__device__ __forceinline__ bf16x8 own_cols_lds(const unsigned char* tile, int kk, int dh8, int lane) {
  const uint4 v = __builtin_bit_cast(uint4, frag_cols_lds<DHP>(tile, kk, lane));
  const bool in = 2 * kk + (lane >> 5) < dh8;
  return __builtin_bit_cast(bf16x8, make_uint4(in ? v.x : 0u, in ? v.y : 0u, in ? v.z : 0u, in ? v.w : 0u));
}
// this lane's piece of a fragment into its place in the tile
template <int DHP>
__device__ __forceinline__ void put_cols_lds(unsigned char* tile, int kk, int lane, bf16x8 v) {
  typedef Geo<DHP> G;
  const int r = lane & 31, ch = 2 * kk + (lane >> 5);
  *reinterpret_cast<uint4*>(tile + r * G::RB + ((ch ^ G::swz(r)) << 4)) = __builtin_bit_cast(uint4, v);
}
// the same straight from memory; rows from rows_left on repeat the last one
__device__ __forceinline__ bf16x8 own_cols_mem(const unsigned char* base, unsigned ldb, int rows_left, int kk, int dh8, int lane) {
  const int r = lane & 31, ch = 2 * kk + (lane >> 5);
  const bool in = ch < dh8;
  const uint4 v = *reinterpret_cast<const uint4*>(base + (unsigned)(r < rows_left ? r : rows_left - 1) * ldb + 16u * (in ? ch : 0));
  return __builtin_bit_cast(bf16x8, make_uint4(in ? v.x : 0u, in ? v.y : 0u, in ? v.z : 0u, in ? v.w : 0u));
}
// operand fragment with the contraction along the tile's ROWS, in the order the accumulator of the first product
// holds them: lane holds column 32 m + l % 32; its element i of step t is tile row 16 t + 8 (i/4) + 4 (l/32) + i%4
// (= tile_row_of(8 t + i, l/32)).  ds_read_b64_tr_b16: within 16 lanes, lane j receives as element r' element j%4 of
// the 8 bytes addressed by lane 4 r' + j/4.
template <int DHP>
__device__ __forceinline__ bf16x8 frag_rows_lds(const unsigned char* tile, int m, int t, int lane) {
  typedef Geo<DHP> G;
  typedef __attribute__((address_space(3))) short4v* lds_p;
  const int s = lane & 15;
  const int e = 32 * m + 16 * ((lane >> 4) & 1) + 4 * (s & 3);
  const int r_lo = 16 * t + 4 * (lane >> 5) + (s >> 2), r_hi = r_lo + 8;
  const unsigned char* p_lo = tile + r_lo * G::RB + (((e >> 3) ^ G::swz(r_lo)) << 4) + (e & 7) * 2;
  const unsigned char* p_hi = tile + r_hi * G::RB + (((e >> 3) ^ G::swz(r_hi)) << 4) + (e & 7) * 2;
  const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(p_lo));
  const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(p_hi));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// 8 accumulator elements (r = 8 t .. 8 t + 7) rounded to bf16 as the second product's operand
__device__ __forceinline__ bf16x8 pack8(const float* v) {
  const uint4 w = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                             pack_bf16x2(v[6], v[7]));
  return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ void store4b(bf16_t* p, float a, float b, float c, float d) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}
template <int MB>
__device__ __forceinline__ void zero_acc(float16v (&acc)[MB]) {
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[m][r] = 0.f;
}
__device__ __forceinline__ float dot8(bf16x8 a, bf16x8 b) {
  const uint4 x = __builtin_bit_cast(uint4, a), y = __builtin_bit_cast(uint4, b);
  const unsigned xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
  float acc = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    acc = fmaf(__uint_as_float(xs[i] << 16), __uint_as_float(ys[i] << 16), acc);
    acc = fmaf(__uint_as_float(xs[i] & 0xFFFF0000u), __uint_as_float(ys[i] & 0xFFFF0000u), acc);
  }
  return acc;
}

}  // namespace

}  // namespace hbp
