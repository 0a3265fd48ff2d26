// Attention over packed sequences, forward and backward, whose key/value heads serve groups of query heads: bf16 storage, on the
// matrix cores; and the entry points of both storage types.
#include "attention_packed.h"

namespace hbp {

namespace {

// Fragments by LDS byte addresses.  The tiles' chunk swizzle is an XOR of address bits, so one register per direction holds all there
// is of a lane in an address: a step adds its stage, an XOR with a constant picks the fragment, and tiles of the same stage
// are constant offsets.  (Registers of the forward kernel at 128 channels: 235 with addresses formed from row and chunk, 216
// with these.)
template <int DHP>
struct Frags {
  typedef Geo<DHP> G;
  typedef unsigned uint4v __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) const uint4v* chunk_p;
  typedef __attribute__((address_space(3))) short4v* quad_p;
  static __device__ __forceinline__ unsigned cols_lane(int lane) {
    const int r = lane & 31;
    return (unsigned)(r * G::RB + (((lane >> 5) ^ G::swz(r)) << 4));
  }
  static __device__ __forceinline__ unsigned rows_lane(int lane) {
    const int q = lane & 15, e = 16 * ((lane >> 4) & 1) + 4 * (q & 3), r = 4 * (lane >> 5) + (q >> 2);
    return (unsigned)(r * G::RB + (((e >> 3) ^ G::swz(r)) << 4) + (e & 7) * 2);
  }
  // frag_cols_lds and frag_rows_lds of the tile at `tile` (a constant) behind the address `at` of a stage and lane
  static __device__ __forceinline__ bf16x8 cols(unsigned at, unsigned tile, int kk) {
    const uint4v v = *(chunk_p)(uintptr_t)((at ^ (32u * kk)) + tile);
    return __builtin_bit_cast(bf16x8, v);
  }
  static __device__ __forceinline__ bf16x8 rows(unsigned at, unsigned tile, int m, int t) {
    const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((quad_p)(uintptr_t)((at ^ (64u * m)) + (tile + 16 * t * G::RB)));
    const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((quad_p)(uintptr_t)((at ^ (64u * m + 32u)) + (tile + (16 * t + 8) * G::RB)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// A fragment of the rows that a wavefront owns: 8 channels of this lane's row, zero past the head's width.
__device__ __forceinline__ bf16x8 own_piece(const bf16_t* row, int kk, int dh8, int lane) {
  const int ch = 2 * kk + (lane >> 5);
  const bool in = ch < dh8;
  const uint4 v = *reinterpret_cast<const uint4*>(row + 8 * (in ? ch : 0));
  return __builtin_bit_cast(bf16x8, make_uint4(in ? v.x : 0u, in ? v.y : 0u, in ? v.z : 0u, in ? v.w : 0u));
}

constexpr int WAVES = 8;

// Streamed key and value tiles: a stage holds 32 NT keys, NT tiles of k, then NT of v, which a workgroup's wavefronts copy together, PW
// copies of 1 KB each, all of one tile or of whole ones.
template <int DHP, int NT, int NW>
struct KeyStream {
  typedef Geo<DHP> G;
  static constexpr int STAGE = 2 * NT * G::TB;
  static constexpr int PW = 2 * NT * G::COPIES / NW;
  unsigned off[PW];
  const unsigned char *k, *v;
  unsigned ldk, ldv, lds0;
  int nk, dh8;
  static __device__ __forceinline__ int tile(int w, int i) { return (w * PW + i) / G::COPIES; }
  static __device__ __forceinline__ int part(int w, int i) { return (w * PW + i) % G::COPIES; }
  __device__ __forceinline__ KeyStream(const PackedAttnArgs& a, const Seq& s, int hk, unsigned lds, int dh8_, int w, int lane) {
    k = reinterpret_cast<const unsigned char*>(row_of<bf16_t>(a.k, s.k0, hk));
    v = reinterpret_cast<const unsigned char*>(row_of<bf16_t>(a.v, s.k0, hk));
    ldk = (unsigned)(a.k.row * 2);
    ldv = (unsigned)(a.v.row * 2);
    lds0 = lds;
    nk = s.nk;
    dh8 = dh8_;
#pragma unroll
    for (int i = 0; i < PW; ++i) off[i] = copy_offset<DHP>(tile(w, i) < NT ? ldk : ldv, part(w, i), 32, dh8, lane);
  }
  // keys 32 NT step .. into stage `at`; keys past the last repeat it
  __device__ __forceinline__ void issue(int step, int at, int w, int lane) const {
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int t = tile(w, i), first = 32 * NT * step + 32 * (t % NT);
      const unsigned ld = t < NT ? ldk : ldv;
      const unsigned char* base = t < NT ? k : v;
      const unsigned dst = lds0 + (unsigned)at * STAGE + (unsigned)(w * PW + i) * 1024u;
      if (first + 32 <= nk) {
        copy16_to_lds(off[i], base + (long)first * ld, dst);
      } else {
        const int from = first < nk ? first : nk - 1;
        copy16_to_lds(copy_offset<DHP>(ld, part(w, i), nk - from, dh8, lane), base + (long)from * ld, dst);
      }
    }
  }
};

// How a workgroup's NW wavefronts (eight, or four) share rows and keys.  COLS = 1: 32 rows for each wavefront, which goes over all keys
// in steps of 64.  COLS = 4, for few rows: 64 rows, and of every step of 128 keys a wavefront takes 32; the four that share rows
// meet in LDS at the end.
template <int W, int COLS, int NW>
struct Shape {
  static constexpr int DHP = padded<W>();
  typedef Fit<W> G;
  static constexpr int ROWS = 32 * NW / COLS;
  static constexpr int NT = COLS == 1 ? 2 : 4, KEYS = 32 * NT, SUB = NT / COLS;
  typedef KeyStream<DHP, NT, NW> KS;
  static constexpr int NST = COLS == 1 ? (DHP == 128 || NW == 4 ? 3 : 4) : (DHP == 128 ? 2 : 3);
  static constexpr int SUMS = COLS == 1 ? 0 : NW * G::MB * 16 * 64 * 4;       // everyone's output, fp32
  static constexpr int RING = NST * KS::STAGE > SUMS ? NST * KS::STAGE : SUMS;
};

// The rows of a workgroup, and the keys that they see: steps from .. to - 1 of this workgroup's share of them.
template <int W, int COLS, int NW>
struct RowBlock {
  typedef Shape<W, COLS, NW> S;
  Tile x;
  int w0, rows_left, mine, fewest, most, from, to, share;
  RowPlace me;
  __device__ __forceinline__ bool find(const PackedAttnArgs& a, int rw, int lane) {
    x = find_tile<false>(a, S::ROWS, lane);
    if (!x.exists) return false;
    const int R = x.s.nq * a.group, r0 = S::ROWS * x.t;
    w0 = r0 + 32 * rw;
    rows_left = R - w0;
    auto seen = [&](int r) __attribute__((always_inline)) { return seen_by(x.s, place_of(a, x.hk, r).i, a.causal); };
    const int steps = (seen((R < r0 + S::ROWS ? R : r0 + S::ROWS) - 1) + S::KEYS - 1) / S::KEYS;
    share = (int)blockIdx.y;
    from = (int)((long)steps * share / a.shares);
    to = (int)((long)steps * (share + 1) / a.shares);
    const int r = rows_left > 0 ? w0 + ((lane & 31) < rows_left ? (lane & 31) : rows_left - 1) : R - 1;
    me = place_of(a, x.hk, r);
    mine = seen_by(x.s, me.i, a.causal);
    fewest = rows_left > 0 ? seen(w0) : 0;
    most = rows_left > 0 ? seen(w0 + (rows_left < 32 ? rows_left : 32) - 1) : 0;
    return true;
  }
};

// Scores into the second product's operand, rounded to bf16, or, in a sequence of few keys (queries), as two parts that hold 16 bits:
// a few roundings do not average out, and such sequences are not bound by their products.
constexpr int FEW = 64;
template <bool FEW_TERMS>
struct Operand {
  bf16x8 hi[2], lo[2];
  __device__ __forceinline__ explicit Operand(const float* p) {
#pragma unroll
    for (int t = 0; t < 2; ++t) hi[t] = pack8(p + 8 * t);
    if (FEW_TERMS) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint4 h = __builtin_bit_cast(uint4, hi[t]);
        const unsigned w[4] = {h.x, h.y, h.z, h.w};
        float rest[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          rest[2 * i] = p[8 * t + 2 * i] - __uint_as_float(w[i] << 16);
          rest[2 * i + 1] = p[8 * t + 2 * i + 1] - __uint_as_float(w[i] & 0xFFFF0000u);
        }
        lo[t] = pack8(rest);
      }
    }
  }
  // acc += the tile's columns (behind `at`, at `tile`) times the scores
  template <int DHP, int MB>
  __device__ __forceinline__ void times(unsigned at, unsigned tile, float16v (&acc)[MB]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) acc[mb] = mfma(Frags<DHP>::rows(at, tile, mb, t), hi[t], acc[mb]);
    if (FEW_TERMS) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) acc[mb] = mfma(Frags<DHP>::rows(at, tile, mb, t), lo[t], acc[mb]);
    }
  }
};

// A tile's results, scaled per row by f, to their rows (see store_tile in attention.hip: 64 bytes of a row per store).
// row(j): where row j of the tile goes; rows_left of them.  acc: blocks of 32 channels from block m0 on.
template <int MB, typename F>
__device__ __forceinline__ void store_rows(F row, int rows_left, const float16v (&acc)[MB], float f, int m0, int dh, unsigned char* stg,
                                           int lane) {
  const int r = lane & 31, hh = lane >> 5, rr = lane >> 2, ch = lane & 3;
  bf16_t* out[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) out[u] = rr + 16 * u < rows_left ? row(rr + 16 * u) : nullptr;
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    if (32 * (m0 + m) >= dh) break;
#pragma unroll
    for (int g = 0; g < 4; ++g)
      store4b(reinterpret_cast<bf16_t*>(stg + r * 64 + ((g ^ ((r >> 2) & 3)) << 4) + 8 * hh), acc[m][4 * g] * f,
              acc[m][4 * g + 1] * f, acc[m][4 * g + 2] * f, acc[m][4 * g + 3] * f);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int w = rr + 16 * u;
      const uint4 v = *reinterpret_cast<const uint4*>(stg + w * 64 + ((ch ^ ((w >> 2) & 3)) << 4));
      const int c = 32 * (m0 + m) + 8 * ch;
      if (out[u] && c < dh) *reinterpret_cast<uint4*>(out[u] + c) = v;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The outputs of the wavefronts that share rows (sums: [wavefront][block of 32 channels][element][lane]) into block `m` of the sum, each
// times its f.
template <int MB>
__device__ __forceinline__ void put_sums(float* sums, int wave, const float16v (&acc)[MB], int lane) {
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[((wave * MB + m) * 16 + e) * 64 + lane] = acc[m][e];
}
template <int MB, int COLS>
__device__ __forceinline__ void get_sums(const float* sums, int rw, int m, const float (&f)[COLS], float16v (&acc)[1], int lane) {
  constexpr int RW = WAVES / COLS;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < COLS; ++j) t = fmaf(f[j], sums[(((j * RW + rw) * MB + m) * 16 + e) * 64 + lane], t);
    acc[0][e] = t;
  }
}
// Forward.  A lane holds one row of q and half of that row's scores, so the running maximum and sum are scalars of the lane; the scores
// leave the first product in the places from which the second takes them.  Keys and values come through a ring of stages.
// The maximum that the exponents are taken from moves only when a row's has grown by more than a factor of 2^8 (probabilities
// then reach 2^8, sums 2^8 times the keys: far inside fp32, and bf16 rounds relatively), so the output is rarely rescaled.
// Few rows over long keys (a.shares > 1): a workgroup takes a share of the steps and leaves sums, maxima and outputs for
// packed_join_fwd_kernel.
template <int W, int COLS>
__global__ __launch_bounds__(64 * WAVES, W <= 64 ? 4 : 2) void packed_fwd_mfma_kernel(PackedAttnArgs a) {
  constexpr int NW = WAVES;
  constexpr int DHP = padded<W>();
  typedef Fit<W> G;
  typedef Shape<W, COLS, NW> S;
  typedef typename S::KS KS;
  constexpr int NST = S::NST, RW = NW / COLS;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[S::RING];
  __shared__ float stats[COLS == 1 ? 1 : WAVES][2][64];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), rw = wave % RW, col = wave / RW;
  RowBlock<W, COLS, NW> b;
  if (!b.find(a, rw, lane)) return;
  const Seq& sq = b.x.s;
  const int dh8 = a.dh >> 3;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const KS ks(a, sq, b.x.hk, lds0, dh8, wave, lane);
  for (int i = 0; i < NST - 1 && b.from + i < b.to; ++i) ks.issue(b.from + i, i, wave, lane);
  const long n = sq.q0 + b.me.i;
  const bf16_t* qrow = row_of<bf16_t>(a.q, n, b.me.h);
  bf16x8 fq[G::KK];
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) fq[kk] = own_piece(qrow, kk, dh8, lane);
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) landed(fq[kk]);
  const float c = a.scale * LOG2E;
  const unsigned ck = lds0 + Frags<DHP>::cols_lane(lane) + col * S::SUB * G::TB, rv = lds0 + Frags<DHP>::rows_lane(lane) + col * S::SUB * G::TB;
  float16v o[G::MB];
  zero_acc(o);
  float m = -FLT_MAX, l = 0.f;                             // m: in units of the exponent; l: this half's sum
  auto step = [&](int first, int at, bool masked, auto few) __attribute__((always_inline)) {
    const unsigned tk = ck + (unsigned)at * KS::STAGE, tv = rv + (unsigned)at * KS::STAGE;
    float16v s[S::SUB];
    zero_acc(s);
#pragma unroll
    for (int u = 0; u < S::SUB; ++u)
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) s[u] = mfma(Frags<DHP>::cols(tk, u * G::TB, kk), fq[kk], s[u]);
    if (masked) {
#pragma unroll
      for (int u = 0; u < S::SUB; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * u + tile_row_of(e, 0) >= b.mine - 4 * hh - first) s[u][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int e = 1; e < 16 * S::SUB; ++e) top = fmaxf(top, s[e >> 4][e & 15]);
    top = max_of_halves(top) * c;
    if (__any(top > m + 8.f)) {
      const float mn = fmaxf(m, top), alpha = fast_exp2(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int mb = 0; mb < G::MB; ++mb)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[mb][e] *= alpha;
    }
#pragma unroll
    for (int u = 0; u < S::SUB; ++u) {
      float p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = fast_exp2(fmaf(s[u][e], c, -m));
        l += p[e];
      }
      const Operand<decltype(few)::value> op(p);
      op.template times<DHP>(tv, (S::NT + u) * G::TB, o);
    }
  };
  auto walk = [&](auto few) __attribute__((always_inline)) {
    int at = 0;
    for (int i = b.from; i < b.to; ++i) {
      if (i + NST - 2 < b.to) copies_in_flight<KS::PW * (NST - 2)>();
      else copies_in_flight<0>();
      workgroup_handover();
      if (i + NST - 1 < b.to) ks.issue(i + NST - 1, at == 0 ? NST - 1 : at - 1, wave, lane);
      const int first = S::KEYS * i + 32 * S::SUB * col;
      if (first < b.most) step(first, at, first + 32 * S::SUB > b.fewest, few);
      at = at == NST - 1 ? 0 : at + 1;
    }
  };
  if (sq.nk <= FEW) walk(std::true_type());
  else walk(std::false_type());
  l += other_half(l);
  __syncthreads();                                         // the ring is free: results meet in it, or leave through it
  auto row = [&](int j) __attribute__((always_inline)) {
    const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
    return row_out<bf16_t>(a.o, sq.q0 + q.i, q.h);
  };
  const int c0 = COLS == 1 ? 0 : 32 * col, c1 = COLS == 1 || c0 + 32 > a.dh ? a.dh : c0 + 32;      // the channels that this wavefront leaves
  auto redo = [&](int j) {
    const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
    one_forward<bf16_t>(a, sq, q.i, q.h, c0, c1, lane);
  };
  const bool stat = lane < 32 && lane < b.rows_left;
  if constexpr (COLS == 1) {
    if (b.rows_left <= 0) return;
    const float f = inverse_sum(m, l);
    store_rows(row, b.rows_left, o, f, 0, a.dh, ring + wave * 2048, lane);
    if (stat) a.lse[n * a.heads + b.me.h] = l == 0.f ? -INFINITY : m + log2f(l);
    redo_rows(not_finite(o, f * 0.f), b.rows_left, redo);
  } else {
    float* const sums = reinterpret_cast<float*>(ring);
    put_sums<G::MB>(sums, wave, o, lane);
    stats[wave][0][lane] = m;
    stats[wave][1][lane] = l;
    __syncthreads();
    float f[COLS], top = stats[rw][0][lane], sum = 0.f;
#pragma unroll
    for (int j = 1; j < COLS; ++j) top = fmaxf(top, stats[j * RW + rw][0][lane]);
#pragma unroll
    for (int j = 0; j < COLS; ++j) {
      f[j] = fast_exp2(stats[j * RW + rw][0][lane] - top);
      sum = fmaf(f[j], stats[j * RW + rw][1][lane], sum);
    }
    float16v acc[1];
    if (col < G::MB) get_sums<G::MB, COLS>(sums, rw, col, f, acc, lane);
    __syncthreads();
    if (b.rows_left <= 0 || col >= G::MB) return;          // (a block of 32 channels each)
    if (a.shares > 1) {
      const long r = n * a.heads + b.me.h;
      const long p = (long)b.share * a.q_rows * a.heads + r;
      if ((lane & 31) < b.rows_left) store_share<1>(a.part, p, acc, col, a.dh, hh);
      if (stat && col == 0) {
        a.part_stats[2 * p] = top;
        a.part_stats[2 * p + 1] = sum;
      }
      return;
    }
    const float g = inverse_sum(top, sum);
    store_rows(row, b.rows_left, acc, g, col, a.dh, ring + wave * 2048, lane);
    if (stat && col == 0) a.lse[n * a.heads + b.me.h] = sum == 0.f ? -INFINITY : top + log2f(sum);
    redo_rows(not_finite(acc, g * 0.f), b.rows_left, redo);
  }
}

// More than 64 channels, many rows: 64 of them for a wavefront, so that a tile read from LDS meets two tiles of rows.  (32 rows each: the
// reads of LDS take as long as the products; 16384 positions, 32 heads of 128 on 8: 2115 us, with 64 1971, of which a long
// library product's rate would leave 1671.)  The steps are those of packed_fwd_mfma_kernel, 32 keys at a time; weights are rounded
// once even in a sequence of few keys among longer ones (see Operand; two parts have no registers here).
constexpr int TALL = 2 * 32 * WAVES;
template <int W>
__global__ __launch_bounds__(64 * WAVES, 2) void packed_fwd_tall_kernel(PackedAttnArgs a) {
  constexpr int DHP = padded<W>();
  typedef Fit<W> G;
  constexpr int RT = 2, NT = 2, KEYS = 32 * NT, ROWS = TALL, NST = 3;
  typedef KeyStream<DHP, NT, WAVES> KS;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[NST * KS::STAGE];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const Tile x = find_tile<false>(a, ROWS, lane);
  if (!x.exists) return;
  const Seq& sq = x.s;
  const int R = sq.nq * a.group, r0 = ROWS * x.t, w0 = r0 + 32 * RT * wave, rows_left = R - w0;
  auto seen = [&](int r) __attribute__((always_inline)) { return seen_by(sq, place_of(a, x.hk, r).i, a.causal); };
  const int steps = (seen((R < r0 + ROWS ? R : r0 + ROWS) - 1) + KEYS - 1) / KEYS;
  const int fewest = rows_left > 0 ? seen(w0) : 0, most = rows_left > 0 ? seen(w0 + (rows_left < 32 * RT ? rows_left : 32 * RT) - 1) : 0;
  const int dh8 = a.dh >> 3;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const KS ks(a, sq, x.hk, lds0, dh8, wave, lane);
  for (int i = 0; i < NST - 1 && i < steps; ++i) ks.issue(i, i, wave, lane);
  bf16x8 fq[RT][G::KK];
  int mine[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = w0 + 32 * t + (lane & 31);
    const RowPlace me = place_of(a, x.hk, r < R ? r : R - 1);
    mine[t] = seen_by(sq, me.i, a.causal) - 4 * hh;
    const bf16_t* qrow = row_of<bf16_t>(a.q, sq.q0 + me.i, me.h);
#pragma unroll
    for (int kk = 0; kk < G::KK; ++kk) fq[t][kk] = own_piece(qrow, kk, dh8, lane);
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int kk = 0; kk < G::KK; ++kk) landed(fq[t][kk]);
  const float c = a.scale * LOG2E;
  const unsigned ck = lds0 + Frags<DHP>::cols_lane(lane), rv = lds0 + Frags<DHP>::rows_lane(lane);
  float16v o[RT][G::MB];
  float m[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) { zero_acc(o[t]); m[t] = -FLT_MAX; l[t] = 0.f; }
  int at = 0;
  for (int i = 0; i < steps; ++i) {
    if (i + NST - 2 < steps) copies_in_flight<KS::PW * (NST - 2)>();
    else copies_in_flight<0>();
    workgroup_handover();
    if (i + NST - 1 < steps) ks.issue(i + NST - 1, at == 0 ? NST - 1 : at - 1, wave, lane);
    const unsigned tk = ck + (unsigned)at * KS::STAGE, tv = rv + (unsigned)at * KS::STAGE;
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const int first = KEYS * i + 32 * u;
      if (first < most) {
        float16v s[RT];
        zero_acc(s);
#pragma unroll
        for (int kk = 0; kk < G::KK; ++kk) {
          const bf16x8 f = Frags<DHP>::cols(tk, u * G::TB, kk);
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t] = mfma(f, fq[t][kk], s[t]);
        }
        if (first + 32 > fewest) {
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const int n = mine[t] - first;
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (tile_row_of(e, 0) >= n) s[t][e] = -INFINITY;
          }
        }
        float top[RT];
        bool more = false;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          top[t] = s[t][0];
#pragma unroll
          for (int e = 1; e < 16; ++e) top[t] = fmaxf(top[t], s[t][e]);
          top[t] = max_of_halves(top[t]) * c;
          more = more || top[t] > m[t] + 8.f;
        }
        if (__any(more)) {
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const float mn = fmaxf(m[t], top[t]), alpha = fast_exp2(m[t] - mn);
            m[t] = mn;
            l[t] *= alpha;
#pragma unroll
            for (int mb = 0; mb < G::MB; ++mb)
#pragma unroll
              for (int e = 0; e < 16; ++e) o[t][mb][e] *= alpha;
          }
        }
        bf16x8 p[RT][2];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          float w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            w[e] = fast_exp2(fmaf(s[t][e], c, -m[t]));
            l[t] += w[e];
          }
          p[t][0] = pack8(w);
          p[t][1] = pack8(w + 8);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int mb = 0; mb < G::MB; ++mb) {
            const bf16x8 f = Frags<DHP>::rows(tv, (NT + u) * G::TB, mb, g);
#pragma unroll
            for (int t = 0; t < RT; ++t) o[t][mb] = mfma(f, p[t][g], o[t][mb]);
          }
      }
    }
    at = at == NST - 1 ? 0 : at + 1;
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int left = rows_left - 32 * t, wt = w0 + 32 * t;
    if (left <= 0) return;
    l[t] += other_half(l[t]);
    const float f = inverse_sum(m[t], l[t]);
    store_rows([&](int j) __attribute__((always_inline)) {
      const RowPlace q = place_of(a, x.hk, wt + j);
      return row_out<bf16_t>(a.o, sq.q0 + q.i, q.h);
    }, left, o[t], f, 0, a.dh, ring + wave * 2048, lane);
    if (lane < 32 && lane < left) {
      const RowPlace me = place_of(a, x.hk, wt + lane);
      a.lse[(long)(sq.q0 + me.i) * a.heads + me.h] = l[t] == 0.f ? -INFINITY : m[t] + log2f(l[t]);
    }
    redo_rows(not_finite(o[t], f * 0.f), left, [&](int j) {
      const RowPlace q = place_of(a, x.hk, wt + j);
      one_forward<bf16_t>(a, sq, q.i, q.h, 0, a.dh, lane);
    });
  }
}

// dq, and for the other kernel minus D = sum_c dout (.) o and minus lse of every row.  As the forward pass: a lane holds a row of q and
// of dout, dS leaves the first two products in the places from which the third takes it.
// At up to 64 channels a workgroup of many rows has four wavefronts, and a compute unit three workgroups: rows are loaded, and results
// stored, while others compute (16 sequences of 1024, 16 heads on 4: 90 us with one workgroup of eight, of whose 22 us
// 7.4 are not spent on products; 77 with three of four).
template <int W, int COLS, int NW>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 3 : 2) void packed_dq_mfma_kernel(PackedAttnArgs a) {
  constexpr int DHP = padded<W>();
  typedef Fit<W> G;
  typedef Shape<W, COLS, NW> S;
  typedef typename S::KS KS;
  constexpr int NST = S::NST, RW = NW / COLS;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[S::RING];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), rw = wave % RW, col = wave / RW;
  RowBlock<W, COLS, NW> b;
  if (!b.find(a, rw, lane)) return;
  const Seq& sq = b.x.s;
  const int dh8 = a.dh >> 3;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const KS ks(a, sq, b.x.hk, lds0, dh8, wave, lane);
  for (int i = 0; i < NST - 1 && b.from + i < b.to; ++i) ks.issue(b.from + i, i, wave, lane);
  const long n = sq.q0 + b.me.i;
  const bf16_t* qrow = row_of<bf16_t>(a.q, n, b.me.h);
  const bf16_t* grow = row_of<bf16_t>(a.dout, n, b.me.h);
  const bf16_t* orow = row_of<bf16_t>(a.o, n, b.me.h);
  float L = a.lse[n * a.heads + b.me.h];                   // (asked for with the rows, not after them)
  bf16x8 fq[G::KK], fg[G::KK];
  float D = 0.f;
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) {
    fq[kk] = own_piece(qrow, kk, dh8, lane);
    fg[kk] = own_piece(grow, kk, dh8, lane);
    D += dot8(fg[kk], own_piece(orow, kk, dh8, lane));
  }
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) { landed(fq[kk]); landed(fg[kk]); }
  landed(L);
  D += other_half(D);
  L = stat_of(L);
  if (col == 0 && b.share == 0 && lane < 32 && lane < b.rows_left) {
    a.dsum[n * a.heads + b.me.h] = -D;
    a.nlse[n * a.heads + b.me.h] = -L;
  }
  const float c = a.scale * LOG2E;
  const unsigned ck = lds0 + Frags<DHP>::cols_lane(lane) + col * S::SUB * G::TB, rk = lds0 + Frags<DHP>::rows_lane(lane) + col * S::SUB * G::TB;
  float16v dq[G::MB], minus_D;
  zero_acc(dq);
#pragma unroll
  for (int e = 0; e < 16; ++e) minus_D[e] = -D;
  auto step = [&](int first, int at, bool masked, auto few) __attribute__((always_inline)) {
    const unsigned tc = ck + (unsigned)at * KS::STAGE, tr = rk + (unsigned)at * KS::STAGE;
#pragma unroll
    for (int u = 0; u < S::SUB; ++u) {
      float16v s[1], dp = minus_D;
      zero_acc(s);
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) {
        s[0] = mfma(Frags<DHP>::cols(tc, u * G::TB, kk), fq[kk], s[0]);
        dp = mfma(Frags<DHP>::cols(tc, (S::NT + u) * G::TB, kk), fg[kk], dp);
      }
      float ds[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) ds[e] = fast_exp2(fmaf(s[0][e], c, -L)) * dp[e];
      if (masked) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * u + tile_row_of(e, 0) >= b.mine - 4 * hh - first) ds[e] = 0.f;
      }
      const Operand<decltype(few)::value> op(ds);
      op.template times<DHP>(tr, u * G::TB, dq);
    }
  };
  auto walk = [&](auto few) __attribute__((always_inline)) {
    int at = 0;
    for (int i = b.from; i < b.to; ++i) {
      if (i + NST - 2 < b.to) copies_in_flight<KS::PW * (NST - 2)>();
      else copies_in_flight<0>();
      workgroup_handover();
      if (i + NST - 1 < b.to) ks.issue(i + NST - 1, at == 0 ? NST - 1 : at - 1, wave, lane);
      const int first = S::KEYS * i + 32 * S::SUB * col;
      if (first < b.most) step(first, at, first + 32 * S::SUB > b.fewest, few);
      at = at == NST - 1 ? 0 : at + 1;
    }
  };
  if (sq.nk <= FEW) walk(std::true_type());
  else walk(std::false_type());
  __syncthreads();
  auto row = [&](int j) __attribute__((always_inline)) {
    const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
    return row_out<bf16_t>(a.dq, sq.q0 + q.i, q.h);
  };
  const int c0 = COLS == 1 ? 0 : 32 * col, c1 = COLS == 1 || c0 + 32 > a.dh ? a.dh : c0 + 32;
  auto redo = [&](int j) {
    const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
    one_dq<bf16_t>(a, sq, q.i, q.h, row_dsum<bf16_t>(a, sq.q0 + q.i, q.h, lane), c0, c1, lane);
  };
  if constexpr (COLS == 1) {
    if (b.rows_left <= 0) return;
    store_rows(row, b.rows_left, dq, a.scale, 0, a.dh, ring + wave * 2048, lane);
    redo_rows(not_finite(dq, 0.f), b.rows_left, redo);
  } else {
    float* const sums = reinterpret_cast<float*>(ring);
    put_sums<G::MB>(sums, wave, dq, lane);
    __syncthreads();
    float f[COLS];
#pragma unroll
    for (int j = 0; j < COLS; ++j) f[j] = 1.f;
    float16v acc[1];
    if (col < G::MB) get_sums<G::MB, COLS>(sums, rw, col, f, acc, lane);
    __syncthreads();
    if (b.rows_left <= 0 || col >= G::MB) return;
    if (a.shares > 1) {
      if ((lane & 31) < b.rows_left)
        store_share<1>(a.part, (long)b.share * a.q_rows * a.heads + n * a.heads + b.me.h, acc, col, a.dh, hh);
      return;
    }
    store_rows(row, b.rows_left, acc, a.scale, col, a.dh, ring + wave * 2048, lane);
    redo_rows(not_finite(acc, 0.f), b.rows_left, redo);
  }
}

// dk, dv.  A workgroup's eight wavefronts own 32 keys each, TURNS wavefronts the same ones: they take every TURNS-th tile of 32 queries
// in turn, and their sums meet in LDS at the end.  A lane holds one key's k and v and half of that key's probabilities.
// TURNS = 2, 128 keys; 4, 64 keys, for few of them.  (128 keys with four wavefronts: half the wavefronts on a SIMD, or two
// workgroups on a compute unit that a causal mask leaves unequally long; 256 keys: half as many workgroups to share out.)
// Queries come from the last one down, all heads of the group for a tile of queries before the next tile: whatever the mask
// leaves them, the workgroups of a key head begin with the same tiles and stay in step, so that the tiles come from the XCD's L2.
// At 128 channels k stays in LDS, which leaves registers for two wavefronts on every SIMD.
template <int W, int TURNS>
__global__ __launch_bounds__(64 * WAVES, 2) void packed_dkdv_mfma_kernel(PackedAttnArgs a) {
  constexpr int DHP = padded<W>();
  typedef Fit<W> G;
  constexpr bool KLDS = DHP == 128;
  constexpr int NST = DHP == 128 && TURNS == 4 ? 2 : 3;
  constexpr int KW = WAVES / TURNS, KEYS = 32 * KW;
  constexpr int QT = DHP == 64 && TURNS == 2 ? 2 : 1;      // tiles of a wavefront in a step
  constexpr int NT = TURNS * QT;                           // tiles of a step
  constexpr int STAGE = 2 * NT * G::TB;                    // NT tiles of q, as many of dout
  constexpr int PW = 2 * NT * G::COPIES / WAVES;           // copies of a stage by one wavefront
  constexpr int SUMS = KW * (TURNS == 2 ? 2 : TURNS - 1) * G::MB * 16 * 64 * 4;    // of two turns dk and dv, of four one of them at a time
  constexpr int RING = NST * STAGE + (KLDS ? KW * G::TB : 0);
  __shared__ __attribute__((aligned(1024))) unsigned char ring[RING > SUMS ? RING : SUMS];
  __shared__ __attribute__((aligned(256))) float stats[NST][NT][2][64];          // [stage][tile][-lse | -D][32 rows, and again]
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), turn = wave / KW, kw = wave % KW;
  const Tile x = find_tile<true>(a, KEYS, lane);
  if (!x.exists) return;
  const int k0 = KEYS * x.t, w0 = k0 + 32 * kw;
  const int keys_left = x.s.nk - w0;
  const int dh8 = a.dh >> 3;
  const int nq = x.s.nq, shift = x.s.nk - nq;
  // the first query that sees a key (causal; the last query sees the last key)
  auto first_query = [&](int key) __attribute__((always_inline)) {
    const int i = key - shift;
    return !a.causal || i < 0 ? 0 : i;
  };
  const int top = (nq - 1) >> 5;                           // last tile of queries
  const int tiles = nq > 0 ? (top + 1 - (first_query(k0) >> 5)) * a.group : 0;     // times heads
  const int all_steps = (tiles + NT - 1) / NT, share = (int)blockIdx.y;
  const int from = (int)((long)all_steps * share / a.shares), to = (int)((long)all_steps * (share + 1) / a.shares);
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const unsigned lds1 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(stats));
  // this wavefront's copies: PW parts of one of the stage's tiles, and a statistic of another
  static_assert(G::COPIES % PW == 0, "a wavefront's copies are of one tile");
  const int ct = wave * PW / G::COPIES, cp = wave * PW % G::COPIES, st = (wave >> 1) % NT;
  const HeadRows& src = ct < NT ? a.q : a.dout;
  const unsigned ld = (unsigned)(src.row * 2);
  unsigned off[PW];
#pragma unroll
  for (int u = 0; u < PW; ++u) off[u] = copy_offset<DHP>(ld, cp + u, 32, dh8, lane);
  // a place in the list of (tile of queries, head of the group)
  struct Place {
    int h, q;
    __device__ __forceinline__ void on(int n, int group) {
      for (h += n; h >= group; h -= group) --q;
    }
  };
  const int skipped = (int)a.by_group.quotient((unsigned)(from * NT));
  const Place begin_at{from * NT - skipped * a.group, top - skipped};
  Place pc = begin_at, pt = begin_at;
  pc.on(ct % NT, a.group);
  pt.on(st, a.group);
  auto ask = [&](int at) __attribute__((always_inline)) {
    {
      const int first = pc.q < 0 ? 0 : 32 * pc.q, left = nq - first;               // (past the last: a tile that nobody reads)
      const unsigned char* base = reinterpret_cast<const unsigned char*>(row_of<bf16_t>(src, x.s.q0 + first, x.hk * a.group + pc.h));
      const unsigned dst = lds0 + (unsigned)at * STAGE + (unsigned)(wave * PW) * 1024u;
      if (left >= 32) {
#pragma unroll
        for (int u = 0; u < PW; ++u) copy16_to_lds(off[u], base, dst + 1024u * u);
      } else {
#pragma unroll
        for (int u = 0; u < PW; ++u) copy16_to_lds(copy_offset<DHP>(ld, cp + u, left, dh8, lane), base, dst + 1024u * u);
      }
    }
    // (every wavefront copies a statistic: the waits count the same for all)
    const int first = pt.q < 0 ? 0 : 32 * pt.q, r = first + (lane & 31) < nq ? first + (lane & 31) : nq - 1;
    copy4_to_lds((wave & 1 ? a.dsum : a.nlse) + (long)(x.s.q0 + r) * a.heads + x.hk * a.group + pt.h,
                 lds1 + (unsigned)at * (NT * 512u) + (unsigned)(2 * st + (wave & 1)) * 256u);
    pc.on(NT, a.group);
    pt.on(NT, a.group);
  };
  for (int i = 0; i < NST - 1 && from + i < to; ++i) ask(i);
  const int key = keys_left > 0 ? w0 + ((lane & 31) < keys_left ? (lane & 31) : keys_left - 1) : x.s.nk - 1;
  const bf16_t* krow = row_of<bf16_t>(a.k, x.s.k0 + key, x.hk);
  const bf16_t* vrow = row_of<bf16_t>(a.v, x.s.k0 + key, x.hk);
  const unsigned cl = Frags<DHP>::cols_lane(lane), cq = lds0 + cl + (unsigned)(turn * QT) * G::TB;
  const unsigned rq = lds0 + Frags<DHP>::rows_lane(lane) + (unsigned)(turn * QT) * G::TB;
  const unsigned kl = lds0 + NST * STAGE + (unsigned)kw * G::TB + cl;
  bf16x8 fk[G::KK], fv[G::KK];
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) { fk[kk] = own_piece(krow, kk, dh8, lane); fv[kk] = own_piece(vrow, kk, dh8, lane); }
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) {
    landed(fk[kk]);
    landed(fv[kk]);
    // (all wavefronts of these keys write the same)
    if (KLDS) put_cols_lds<DHP>(ring + NST * STAGE + kw * G::TB, kk, lane, fk[kk]);
  }
  const int mine = first_query(key);                       // the first query that sees this lane's key
  const int begin = keys_left > 0 ? first_query(w0) : nq, all = keys_left > 0 ? first_query(w0 + (keys_left < 32 ? keys_left : 32) - 1) : nq;
  const float c = a.scale * LOG2E;
  float16v dk[G::MB], dv[G::MB];
  zero_acc(dk);
  zero_acc(dv);
  // the wavefront's tiles of the stage: their first queries
  auto step = [&](const int (&first)[QT], int at, bool masked, auto few) __attribute__((always_inline)) {
    const unsigned tc = cq + (unsigned)at * STAGE, tr = rq + (unsigned)at * STAGE;
    float16v s[QT], dp[QT];
    float p[QT][16];
    zero_acc(s);
#pragma unroll
    for (int b = 0; b < QT; ++b)
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk)
        s[b] = mfma(Frags<DHP>::cols(tc, b * G::TB, kk), KLDS ? Frags<DHP>::cols(kl, 0, kk) : fk[kk], s[b]);
#pragma unroll
    for (int b = 0; b < QT; ++b) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 u = *reinterpret_cast<const float4*>(&stats[at][turn * QT + b][1][8 * g + 4 * hh]);
        dp[b][4 * g] = u.x; dp[b][4 * g + 1] = u.y; dp[b][4 * g + 2] = u.z; dp[b][4 * g + 3] = u.w;
      }
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) dp[b] = mfma(Frags<DHP>::cols(tc, (NT + b) * G::TB, kk), fv[kk], dp[b]);
    }
#pragma unroll
    for (int b = 0; b < QT; ++b) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 u = *reinterpret_cast<const float4*>(&stats[at][turn * QT + b][0][8 * g + 4 * hh]);
        p[b][4 * g] = fast_exp2(fmaf(s[b][4 * g], c, u.x));
        p[b][4 * g + 1] = fast_exp2(fmaf(s[b][4 * g + 1], c, u.y));
        p[b][4 * g + 2] = fast_exp2(fmaf(s[b][4 * g + 2], c, u.z));
        p[b][4 * g + 3] = fast_exp2(fmaf(s[b][4 * g + 3], c, u.w));
      }
    }
    if (masked) {
#pragma unroll
      for (int b = 0; b < QT; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int i = tile_row_of(e, 0);
          if (i < mine - 4 * hh - first[b] || i >= nq - 4 * hh - first[b]) p[b][e] = 0.f;
        }
    }
#pragma unroll
    for (int b = 0; b < QT; ++b) {
      const Operand<decltype(few)::value> op(p[b]);
      op.template times<DHP>(tr, (NT + b) * G::TB, dv);
#pragma unroll
      for (int e = 0; e < 16; ++e) p[b][e] *= dp[b][e];
      const Operand<decltype(few)::value> ds(p[b]);
      ds.template times<DHP>(tr, b * G::TB, dk);
    }
  };
  int at = 0;
  Place me[QT];                                            // this wavefront's next tiles
#pragma unroll
  for (int b = 0; b < QT; ++b) {
    me[b] = begin_at;
    me[b].on(turn * QT + b, a.group);
  }
  auto walk = [&](auto few) __attribute__((always_inline)) {
    for (int i = from; i < to; ++i) {
      if (i + NST - 2 < to) copies_in_flight<(PW + 1) * (NST - 2)>();
      else copies_in_flight<0>();
      workgroup_handover();
      if (i + NST - 1 < to) ask(at == 0 ? NST - 1 : at - 1);
      int first[QT];
      bool some = false, masked = false;
#pragma unroll
      for (int b = 0; b < QT; ++b) {
        const bool there = NT * i + turn * QT + b < tiles;
        first[b] = there ? 32 * me[b].q : nq;                // (a tile past the list: masked throughout)
        some = some || (there && first[b] + 32 > begin);
        masked = masked || first[b] < all || first[b] + 32 > nq;
        me[b].on(NT, a.group);
      }
      if (some && keys_left > 0) step(first, at, masked, few);
      at = at == NST - 1 ? 0 : at + 1;
    }
  };
  if (nq <= FEW) walk(std::true_type());
  else walk(std::false_type());
  // The turns' sums of dk meet in the first one, those of dv in the second, through LDS: two turns exchange them at once.
  constexpr bool AT_ONCE = TURNS == 2;
  float* const sums = reinterpret_cast<float*>(ring) + kw * (G::MB * 16 * 64) + lane;
  constexpr int SLOT = KW * G::MB * 16 * 64;
  auto put = [&](const float16v (&acc)[G::MB], int owner, int slot) __attribute__((always_inline)) {
    if (turn == owner) return;
    float* p = sums + (slot + (turn < owner ? turn : turn - 1)) * SLOT;
#pragma unroll
    for (int m = 0; m < G::MB; ++m)
#pragma unroll
      for (int e = 0; e < 16; ++e) p[(m * 16 + e) * 64] = acc[m][e];
  };
  auto get = [&](float16v (&acc)[G::MB], int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < TURNS - 1; ++j)
#pragma unroll
      for (int m = 0; m < G::MB; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[m][e] += sums[(slot + j) * SLOT + (m * 16 + e) * 64];
  };
  auto leave = [&](const float16v (&acc)[G::MB], const HeadRows& out, float f, int which) __attribute__((always_inline)) {
    if (a.shares > 1) {
      const long r = (long)(x.s.k0 + key) * a.kv_heads + x.hk, rows = (long)a.k_rows * a.kv_heads;
      if ((lane & 31) < keys_left) store_share<G::MB>(a.part, ((which == DV ? a.shares : 0) + share) * rows + r, acc, 0, a.dh, hh);
      return;
    }
    store_rows([&](int j) __attribute__((always_inline)) { return row_out<bf16_t>(out, x.s.k0 + w0 + j, x.hk); }, keys_left, acc, f, 0, a.dh,
               ring + wave * 2048, lane);
    redo_rows(not_finite(acc, 0.f), keys_left, [&](int j) { one_dkdv<bf16_t>(a, x.s, w0 + j, x.hk, which, 0, a.dh, lane); });
  };
  __syncthreads();
  put(dk, 0, 0);
  if (AT_ONCE) put(dv, 1, 1);
  __syncthreads();
  if (turn == 0) get(dk, 0);
  if (!AT_ONCE) {
    __syncthreads();
    put(dv, 1, 0);
    __syncthreads();
  }
  if (turn == 1) get(dv, AT_ONCE ? 1 : 0);
  __syncthreads();
  if (turn > 1 || keys_left <= 0) return;
  if (turn == 0) leave(dk, a.dk, a.scale, DK);
  else leave(dv, a.dv, 1.f, DV);
}

// ------------------------------------------------------------------------------------------------------------
// many short sequences: every wavefront by itself
// ------------------------------------------------------------------------------------------------------------
// With a few tiles on the other side, a workgroup spends its time starting, meeting and leaving, and most sequences do not fill it.
// Here each of its eight wavefronts has 32 rows (keys) of any sequence, a ring of its own and no barrier at all.  The other
// side's tiles then come to LDS once for every 32 rows instead of every 256: a short sequence's are in the L2.
template <int W>
struct Alone {
  static constexpr int DHP = padded<W>();
  typedef Fit<W> G;
  static constexpr int NST = DHP == 64 ? 2 : 1, STAGE = 2 * G::TB, COPIES = 2 * G::COPIES;
  unsigned ldx, ldy, off[DHP == 64 ? COPIES : 1];          // (64 channels: offsets of whole tiles, kept)
  int dh8;
  __device__ __forceinline__ Alone(unsigned ldx_, unsigned ldy_, int dh8_, int lane) : ldx(ldx_), ldy(ldy_), dh8(dh8_) {
    if (DHP == 64) {
#pragma unroll
      for (int u = 0; u < COPIES; ++u) off[u] = copy_offset<DHP>(u < G::COPIES ? ldx : ldy, u % G::COPIES, 32, dh8, lane);
    }
  }
  // tiles x and y, rows `first` .. of n, into the stage at `lds`
  __device__ __forceinline__ void issue(const unsigned char* x, const unsigned char* y, int first, int n, unsigned lds, int lane) const {
    x += (long)first * ldx;
    y += (long)first * ldy;
    if (DHP == 64 && first + 32 <= n) {
#pragma unroll
      for (int u = 0; u < COPIES; ++u) copy16_to_lds(off[u], u < G::COPIES ? x : y, lds + 1024u * u);
    } else {
      copy_tile<DHP>(x, ldx, n - first, dh8, lds, lane);
      copy_tile<DHP>(y, ldy, n - first, dh8, lds + G::TB, lane);
    }
  }
};
// The stage of step i, full; ask(step, stage) issues copies.
template <int W, typename F>
__device__ __forceinline__ int stage_alone(int i, int steps, F ask) {
  typedef Alone<W> A;
  if (A::NST == 1) {
    if (i > 0) {
      copies_in_flight_read<0>();                          // (what was read of the step before has arrived)
      ask(i, 0);
    }
    copies_in_flight_read<0>();
    return 0;
  }
  copies_in_flight_read<0>();                              // (step i has arrived, what was read of the step before as well)
  if (i + 1 < steps) ask(i + 1, (i + 1) & 1);
  return i & 1;
}

// this wavefront's rows and the keys that they see
struct OwnRows {
  Tile x;
  int w0, rows_left, mine, fewest, most;
  RowPlace me;
  __device__ __forceinline__ bool find(const PackedAttnArgs& a, unsigned id, int lane) {
    x = find_tile<false>(a, 32, lane, id);
    if (!x.exists) return false;
    const int R = x.s.nq * a.group;
    w0 = 32 * x.t;
    rows_left = R - w0;
    auto seen = [&](int r) __attribute__((always_inline)) { return seen_by(x.s, place_of(a, x.hk, r).i, a.causal); };
    me = place_of(a, x.hk, (lane & 31) < rows_left ? w0 + (lane & 31) : R - 1);
    mine = seen_by(x.s, me.i, a.causal);
    fewest = seen(w0);
    most = seen(w0 + (rows_left < 32 ? rows_left : 32) - 1);
    return true;
  }
};

template <int W>
__global__ __launch_bounds__(64 * WAVES, 2) void packed_fwd_short_kernel(PackedAttnArgs a) {
  constexpr int DHP = padded<W>();
  typedef Fit<W> G;
  typedef Alone<W> A;
  __shared__ __attribute__((aligned(1024))) unsigned char rings[WAVES * A::NST * A::STAGE];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  OwnRows b;
  if (!b.find(a, workgroup_id() * WAVES + wave, lane)) return;
  const Seq& sq = b.x.s;
  const int dh8 = a.dh >> 3, steps = (b.most + 31) >> 5;
  unsigned char* const ring = rings + wave * (A::NST * A::STAGE);
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const unsigned char* k = reinterpret_cast<const unsigned char*>(row_of<bf16_t>(a.k, sq.k0, b.x.hk));
  const unsigned char* v = reinterpret_cast<const unsigned char*>(row_of<bf16_t>(a.v, sq.k0, b.x.hk));
  const A ring_of((unsigned)(a.k.row * 2), (unsigned)(a.v.row * 2), dh8, lane);
  auto ask = [&](int i, int at) __attribute__((always_inline)) {
    ring_of.issue(k, v, 32 * i, sq.nk, lds0 + (unsigned)at * A::STAGE, lane);
  };
  if (steps > 0) ask(0, 0);
  const long n = sq.q0 + b.me.i;
  const bf16_t* qrow = row_of<bf16_t>(a.q, n, b.me.h);
  bf16x8 fq[G::KK];
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) fq[kk] = own_piece(qrow, kk, dh8, lane);
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) landed(fq[kk]);
  const float c = a.scale * LOG2E;
  const unsigned ck = lds0 + Frags<DHP>::cols_lane(lane), rv = lds0 + Frags<DHP>::rows_lane(lane);
  float16v o[G::MB];
  zero_acc(o);
  float m = -FLT_MAX, l = 0.f;
  auto walk = [&](auto few) __attribute__((always_inline)) {
    for (int i = 0; i < steps; ++i) {
      const unsigned at = (unsigned)stage_alone<W>(i, steps, ask) * A::STAGE;
      float16v s[1];
      zero_acc(s);
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) s[0] = mfma(Frags<DHP>::cols(ck + at, 0, kk), fq[kk], s[0]);
      if (32 * i + 32 > b.fewest) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * i + tile_row_of(e, hh) >= b.mine) s[0][e] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[0][e]);
      top = max_of_halves(top) * c;
      if (__any(top > m + 8.f)) {
        const float mn = fmaxf(m, top), alpha = fast_exp2(m - mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int mb = 0; mb < G::MB; ++mb)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[mb][e] *= alpha;
      }
      float p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = fast_exp2(fmaf(s[0][e], c, -m));
        l += p[e];
      }
      const Operand<decltype(few)::value> op(p);
      op.template times<DHP>(rv + at, G::TB, o);
    }
  };
  if (sq.nk <= FEW) walk(std::true_type());
  else walk(std::false_type());
  l += other_half(l);
  copies_in_flight_read<0>();                              // (the ring is free: results leave through it)
  const float f = inverse_sum(m, l);
  store_rows([&](int j) __attribute__((always_inline)) {
    const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
    return row_out<bf16_t>(a.o, sq.q0 + q.i, q.h);
  }, b.rows_left, o, f, 0, a.dh, ring, lane);
  if (lane < 32 && lane < b.rows_left) a.lse[n * a.heads + b.me.h] = l == 0.f ? -INFINITY : m + log2f(l);
  redo_rows(not_finite(o, f * 0.f), b.rows_left, [&](int j) {
    const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
    one_forward<bf16_t>(a, sq, q.i, q.h, 0, a.dh, lane);
  });
}

template <int W>
__global__ __launch_bounds__(64 * WAVES, 2) void packed_dq_short_kernel(PackedAttnArgs a) {
  constexpr int DHP = padded<W>();
  typedef Fit<W> G;
  typedef Alone<W> A;
  __shared__ __attribute__((aligned(1024))) unsigned char rings[WAVES * A::NST * A::STAGE];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  OwnRows b;
  if (!b.find(a, workgroup_id() * WAVES + wave, lane)) return;
  const Seq& sq = b.x.s;
  const int dh8 = a.dh >> 3, steps = (b.most + 31) >> 5;
  unsigned char* const ring = rings + wave * (A::NST * A::STAGE);
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const unsigned char* k = reinterpret_cast<const unsigned char*>(row_of<bf16_t>(a.k, sq.k0, b.x.hk));
  const unsigned char* v = reinterpret_cast<const unsigned char*>(row_of<bf16_t>(a.v, sq.k0, b.x.hk));
  const A ring_of((unsigned)(a.k.row * 2), (unsigned)(a.v.row * 2), dh8, lane);
  auto ask = [&](int i, int at) __attribute__((always_inline)) {
    ring_of.issue(k, v, 32 * i, sq.nk, lds0 + (unsigned)at * A::STAGE, lane);
  };
  if (steps > 0) ask(0, 0);
  const long n = sq.q0 + b.me.i, r = n * a.heads + b.me.h;
  const bf16_t* qrow = row_of<bf16_t>(a.q, n, b.me.h);
  const bf16_t* grow = row_of<bf16_t>(a.dout, n, b.me.h);
  const bf16_t* orow = row_of<bf16_t>(a.o, n, b.me.h);
  float L = a.lse[r], D = 0.f;
  bf16x8 fq[G::KK], fg[G::KK];
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) {
    fq[kk] = own_piece(qrow, kk, dh8, lane);
    fg[kk] = own_piece(grow, kk, dh8, lane);
    D += dot8(fg[kk], own_piece(orow, kk, dh8, lane));
  }
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) { landed(fq[kk]); landed(fg[kk]); }
  landed(L);
  D += other_half(D);
  L = stat_of(L);
  if (lane < 32 && lane < b.rows_left) {
    a.dsum[r] = -D;
    a.nlse[r] = -L;
  }
  const float c = a.scale * LOG2E;
  const unsigned ck = lds0 + Frags<DHP>::cols_lane(lane), rk = lds0 + Frags<DHP>::rows_lane(lane);
  float16v dq[G::MB];
  zero_acc(dq);
  auto walk = [&](auto few) __attribute__((always_inline)) {
    for (int i = 0; i < steps; ++i) {
      const unsigned at = (unsigned)stage_alone<W>(i, steps, ask) * A::STAGE;
      float16v s[1], dp;
      zero_acc(s);
#pragma unroll
      for (int e = 0; e < 16; ++e) dp[e] = -D;
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) {
        s[0] = mfma(Frags<DHP>::cols(ck + at, 0, kk), fq[kk], s[0]);
        dp = mfma(Frags<DHP>::cols(ck + at, G::TB, kk), fg[kk], dp);
      }
      float ds[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) ds[e] = fast_exp2(fmaf(s[0][e], c, -L)) * dp[e];
      if (32 * i + 32 > b.fewest) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * i + tile_row_of(e, hh) >= b.mine) ds[e] = 0.f;
      }
      const Operand<decltype(few)::value> op(ds);
      op.template times<DHP>(rk + at, 0, dq);
    }
  };
  if (sq.nk <= FEW) walk(std::true_type());
  else walk(std::false_type());
  copies_in_flight_read<0>();
  store_rows([&](int j) __attribute__((always_inline)) {
    const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
    return row_out<bf16_t>(a.dq, sq.q0 + q.i, q.h);
  }, b.rows_left, dq, a.scale, 0, a.dh, ring, lane);
  redo_rows(not_finite(dq, 0.f), b.rows_left, [&](int j) {
    const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
    one_dq<bf16_t>(a, sq, q.i, q.h, row_dsum<bf16_t>(a, sq.q0 + q.i, q.h, lane), 0, a.dh, lane);
  });
}

template <int W>
__global__ __launch_bounds__(64 * WAVES, 2) void packed_dkdv_short_kernel(PackedAttnArgs a) {
  constexpr int DHP = padded<W>();
  constexpr bool KLDS = DHP == 128;                        // (see packed_dkdv_mfma_kernel)
  typedef Fit<W> G;
  typedef Alone<W> A;
  constexpr int STATS = A::NST * A::STAGE, KEEP = STATS + A::NST * 512, OWN = KEEP + (KLDS ? G::TB : 0);
  constexpr int NW = DHP == 128 ? 4 : WAVES;               // wavefronts: what fits the LDS
  __shared__ __attribute__((aligned(1024))) unsigned char rings[NW * OWN];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const Tile x = find_tile<true>(a, 32, lane, workgroup_id() * NW + wave);
  if (!x.exists) return;
  const Seq& sq = x.s;
  const int w0 = 32 * x.t, keys_left = sq.nk - w0, nq = sq.nq, shift = sq.nk - nq, dh8 = a.dh >> 3;
  auto first_query = [&](int key) __attribute__((always_inline)) {
    const int i = key - shift;
    return !a.causal || i < 0 ? 0 : i;
  };
  unsigned char* const ring = rings + wave * OWN;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const int begin = first_query(w0) & ~31, each = (nq - begin + 31) >> 5, steps = nq > 0 ? each * a.group : 0;
  const A ring_of((unsigned)(a.q.row * 2), (unsigned)(a.dout.row * 2), dh8, lane);
  int ih = x.hk * a.group, iq = begin;                     // the next step to ask for
  auto ask = [&](int, int at) __attribute__((always_inline)) {
    ring_of.issue(reinterpret_cast<const unsigned char*>(row_of<bf16_t>(a.q, sq.q0, ih)),
                  reinterpret_cast<const unsigned char*>(row_of<bf16_t>(a.dout, sq.q0, ih)), iq, nq, lds0 + (unsigned)at * A::STAGE, lane);
    const long r = (long)(sq.q0 + (iq + (lane & 31) < nq ? iq + (lane & 31) : nq - 1)) * a.heads + ih;
    copy4_to_lds(a.nlse + r, lds0 + STATS + (unsigned)at * 512u);
    copy4_to_lds(a.dsum + r, lds0 + STATS + (unsigned)at * 512u + 256u);
    iq += 32;
    if (iq >= nq) { iq = begin; ++ih; }
  };
  if (steps > 0) ask(0, 0);
  const int key = (lane & 31) < keys_left ? w0 + (lane & 31) : sq.nk - 1;
  const bf16_t* krow = row_of<bf16_t>(a.k, sq.k0 + key, x.hk);
  const bf16_t* vrow = row_of<bf16_t>(a.v, sq.k0 + key, x.hk);
  bf16x8 fk[G::KK], fv[G::KK];
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) { fk[kk] = own_piece(krow, kk, dh8, lane); fv[kk] = own_piece(vrow, kk, dh8, lane); }
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) {
    landed(fk[kk]);
    landed(fv[kk]);
    if (KLDS) put_cols_lds<DHP>(ring + KEEP, kk, lane, fk[kk]);
  }
  const int mine = first_query(key), all = first_query(w0 + (keys_left < 32 ? keys_left : 32) - 1);
  const float c = a.scale * LOG2E;
  const unsigned cl = Frags<DHP>::cols_lane(lane), cq = lds0 + cl, rq = lds0 + Frags<DHP>::rows_lane(lane), kl = lds0 + KEEP + cl;
  float16v dk[G::MB], dv[G::MB];
  zero_acc(dk);
  zero_acc(dv);
  auto walk = [&](auto few) __attribute__((always_inline)) {
    int first = begin;
    for (int i = 0; i < steps; ++i) {
      const int st = stage_alone<W>(i, steps, ask);
      const unsigned at = (unsigned)st * A::STAGE;
      const float* stat = reinterpret_cast<const float*>(ring + STATS + st * 512);
      float16v s[1], dp;
      float p[16];
      zero_acc(s);
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) s[0] = mfma(Frags<DHP>::cols(cq + at, 0, kk), KLDS ? Frags<DHP>::cols(kl, 0, kk) : fk[kk], s[0]);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 u = *reinterpret_cast<const float4*>(stat + 64 + 8 * g + 4 * hh);
        dp[4 * g] = u.x; dp[4 * g + 1] = u.y; dp[4 * g + 2] = u.z; dp[4 * g + 3] = u.w;
      }
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) dp = mfma(Frags<DHP>::cols(cq + at, G::TB, kk), fv[kk], dp);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 u = *reinterpret_cast<const float4*>(stat + 8 * g + 4 * hh);
        p[4 * g] = fast_exp2(fmaf(s[0][4 * g], c, u.x));
        p[4 * g + 1] = fast_exp2(fmaf(s[0][4 * g + 1], c, u.y));
        p[4 * g + 2] = fast_exp2(fmaf(s[0][4 * g + 2], c, u.z));
        p[4 * g + 3] = fast_exp2(fmaf(s[0][4 * g + 3], c, u.w));
      }
      if (first < all || first + 32 > nq) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int q = first + tile_row_of(e, hh);
          if (q < mine || q >= nq) p[e] = 0.f;
        }
      }
      const Operand<decltype(few)::value> op(p);
      op.template times<DHP>(rq + at, G::TB, dv);
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] *= dp[e];
      const Operand<decltype(few)::value> ds(p);
      ds.template times<DHP>(rq + at, 0, dk);
      first += 32;
      if (first >= nq) first = begin;
    }
  };
  if (nq <= FEW) walk(std::true_type());
  else walk(std::false_type());
  copies_in_flight_read<0>();
  store_rows([&](int j) __attribute__((always_inline)) { return row_out<bf16_t>(a.dk, sq.k0 + w0 + j, x.hk); }, keys_left, dk, a.scale, 0,
             a.dh, ring, lane);
  store_rows([&](int j) __attribute__((always_inline)) { return row_out<bf16_t>(a.dv, sq.k0 + w0 + j, x.hk); }, keys_left, dv, 1.f, 0,
             a.dh, ring, lane);
  redo_rows(not_finite(dv, not_finite(dk, 0.f)), keys_left, [&](int j) { one_dkdv<bf16_t>(a, sq, w0 + j, x.hk, DK | DV, 0, a.dh, lane); });
}

// Wavefronts by themselves: many, and with little to stream each.  Per sequence 256 of the other side's rows; 1024 where there are enough
// wavefronts for all places (dk, dv), or where a sequence has one tile of rows, of which a workgroup's other wavefronts would have
// nothing.  Shared / alone, us: forward and backward of 256 sequences of 64, 12 heads of 64, 62 / 26 and 188 / 72; backward of 32 of
// 128 38 / 25, of 128 of 256, 4 heads, 86 / 55; 32 of 256, 32 heads of 128 on 8, 253 / 218; one token over 512 keys, 256
// sequences, 32 heads of 128 on 8, 118 / 94.  The other way round: dk, dv of 128 sequences of 256, 4 heads on 1 (1024 wavefronts, 32
// steps each), the whole backward pass 56 / 63; of 32 of 512, 16 heads of 64 on 4, 131 / 141.
template <bool KEYS>
bool alone(const PackedAttnArgs& a) {
  const long rows = KEYS ? (long)a.k_rows : (long)a.q_rows * a.group;
  const long other = KEYS ? (long)a.q_rows * a.group / a.seqs : a.k_rows / a.seqs;
  const long waves = (rows / 32 + a.seqs) * a.kv_heads;
  if (waves < 4 * (long)CUS) return false;
  return other <= 256 || (other <= 1024 && (KEYS ? waves >= 8 * (long)CUS : rows / a.seqs <= 32));
}

// 256 rows (128 keys) for a workgroup where that makes at least as many workgroups as there are compute units, otherwise 64; 512 of more
// than 64 channels where that makes two for every compute unit and sequences have twice as many rows (256 / 512, us, heads of 128:
// 8 sequences of 1024, 32 heads on 8, 93 / 85; 40 ragged ones of 400 159 / 148; the other way round one of 4096, 264 workgroups
// of which a causal mask makes the longest last, 142 / 206; 24 of 700, 16 heads of 96, 121 / 127)
template <int W>
hipError_t fwd_mfma(const PackedAttnArgs& a, hipStream_t s) {
  if (alone<false>(a))
    packed_fwd_short_kernel<W><<<grid_of((tile_grid<false>(a, 32) + WAVES - 1) / WAVES), 64 * WAVES, 0, s>>>(a);
  else if (W > 64 && wide_blocks<false>(a, TALL, 1024, 2 * CUS) && a.k_rows / a.seqs > FEW)
    packed_fwd_tall_kernel<(W > 64 ? W : 128)><<<grid_of(tile_grid<false>(a, TALL)), 64 * WAVES, 0, s>>>(a);
  else if (wide_blocks<false>(a, 256, 64, CUS))
    packed_fwd_mfma_kernel<W, 1><<<grid_of(tile_grid<false>(a, 256)), 64 * WAVES, 0, s>>>(a);
  else
    packed_fwd_mfma_kernel<W, 4><<<grid_of(tile_grid<false>(a, 64), a.shares), 64 * WAVES, 0, s>>>(a);
  return hipGetLastError();
}
template <int W>
hipError_t dq_mfma(const PackedAttnArgs& a, hipStream_t s) {
  constexpr int NW = W <= 64 ? 4 : 8;
  if (alone<false>(a))
    packed_dq_short_kernel<W><<<grid_of((tile_grid<false>(a, 32) + WAVES - 1) / WAVES), 64 * WAVES, 0, s>>>(a);
  else if (wide_blocks<false>(a, 256, 64, CUS))
    packed_dq_mfma_kernel<W, 1, NW><<<grid_of(tile_grid<false>(a, 32 * NW)), 64 * NW, 0, s>>>(a);
  else
    packed_dq_mfma_kernel<W, 4, WAVES><<<grid_of(tile_grid<false>(a, 64), a.shares), 64 * WAVES, 0, s>>>(a);
  return hipGetLastError();
}
template <int W>
hipError_t dkdv_mfma(const PackedAttnArgs& a, hipStream_t s) {
  if (alone<true>(a))
    packed_dkdv_short_kernel<W><<<grid_of((tile_grid<true>(a, 32) + (W > 64 ? 4 : WAVES) - 1) / (W > 64 ? 4 : WAVES)), 64 * (W > 64 ? 4 : WAVES), 0, s>>>(a);
  else if (wide_blocks<true>(a, 128, 64, CUS))
    packed_dkdv_mfma_kernel<W, 2><<<grid_of(tile_grid<true>(a, 128)), 64 * WAVES, 0, s>>>(a);
  else
    packed_dkdv_mfma_kernel<W, 4><<<grid_of(tile_grid<true>(a, 64), a.shares), 64 * WAVES, 0, s>>>(a);
  return hipGetLastError();
}

// Few rows (keys) leave compute units without a workgroup: the other side's steps are then shared out as well, for two workgroups on
// every compute unit (fp32: four, where products are all that counts and a causal mask's unequal tiles want evening out: forward of
// 1530 positions, 32 heads of 80 on 8, 261 us with two, 199 with four, 217 with eight; bf16 tokens over stored keys lose
// 9 % with four), but no fewer than four steps each.  Shares are fp32 sums that another kernel joins in a fixed order.
int shares_of(int dtype, long groups, long steps) {
  long n = (dtype == 0 ? 4 : 2) * CUS / groups;
  if (n > steps / 4) n = steps / 4;
  if (n > MOST_SHARES) n = MOST_SHARES;
  return n < 2 ? 1 : (int)n;
}
struct Shares { int rows, keys; };       // of the keys for a tile of rows (forward, dq), of the queries for a tile of keys (dk, dv)
Shares shares(int dtype, const PackedAttnArgs& a) {
  const long nq = a.q_rows / a.seqs, nk = a.k_rows / a.seqs;           // (of a sequence, on average)
  // rows (keys) of a workgroup, and keys (queries) of a step
  const bool f32 = dtype == 0, wide_r = f32 ? f32_wide<false>(a) : wide_blocks<false>(a, 256, 64, CUS);
  const bool wide_k = f32 ? f32_wide<true>(a) : wide_blocks<true>(a, 128, 64, CUS);
  const long rows = f32 ? (wide_r ? 128 : 32) : 64, keys = f32 ? (wide_k ? 128 : 32) : 64;
  const long key_step = f32 && wide_r ? 32 : 128, query_step = f32 && wide_k ? 32 : 128;
  const long row_blocks = ((long)a.q_rows * a.group / rows + a.seqs) * a.kv_heads, key_blocks = ((long)a.k_rows / keys + a.seqs) * a.kv_heads;
  return {!f32 && (wide_r || alone<false>(a)) ? 1 : shares_of(dtype, row_blocks, nk / key_step),
          !f32 && (wide_k || alone<true>(a)) ? 1 : shares_of(dtype, key_blocks, (nq + 31) / 32 * 32 * a.group / query_step)};
}

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

PackedAttnArgs with_divisors(const PackedAttnArgs& args) {
  PackedAttnArgs a = args;
  a.q_len = a.q_rows / a.seqs;
  a.k_len = a.k_rows / a.seqs;
  a.by_group = Divisor((unsigned)a.group);
  a.by_kv = Divisor((unsigned)a.kv_heads);
  a.by_seqs = Divisor((unsigned)a.seqs);
  return a;
}

// The workspace: minus D and minus lse of the rows (backward), the shares' maxima and sums (forward), the shares.
struct Layout { size_t stats, shares, total; };
Layout layout(const PackedAttnArgs& a, const Shares& n) {
  const size_t rows = (size_t)a.q_rows * a.heads, keys = (size_t)a.k_rows * a.kv_heads;
  Layout l{};
  l.stats = aligned(rows * 4);
  const size_t stats = 2 * l.stats > aligned(n.rows * rows * 8) || n.rows == 1 ? 2 * l.stats : aligned(n.rows * rows * 8);
  l.shares = stats;
  const size_t r = n.rows > 1 ? n.rows * rows * a.dh * 4 : 0, k = n.keys > 1 ? 2 * n.keys * keys * a.dh * 4 : 0;
  l.total = stats + aligned(r > k ? r : k);
  return l;
}

}  // namespace

size_t packed_attn_ws_bytes(int dtype, const PackedAttnArgs& a) { return layout(a, shares(dtype, a)).total; }

hipError_t launch_packed_attn_fwd(int dtype, const PackedAttnArgs& args, void* workspace, size_t bytes, hipStream_t s) {
  PackedAttnArgs a = with_divisors(args);
  if (a.q_rows == 0) return hipSuccess;
  const Shares n = shares(dtype, a);
  const Layout l = layout(a, n);
  if (bytes < l.total) return hipErrorInvalidValue;
  a.shares = n.rows;
  a.part_stats = reinterpret_cast<float*>(workspace);
  a.part = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + l.shares);
  const hipError_t e = dtype == 0 ? launch_packed_fwd_f32(a, s) : with_width(a.dh, [&](auto w) { return fwd_mfma<decltype(w)::value>(a, s); });
  if (e != hipSuccess || a.shares == 1) return e;
  const unsigned grid = (unsigned)(((long)a.q_rows * a.heads + 3) / 4);
  if (dtype == 0) packed_join_fwd_kernel<float><<<grid, 256, 0, s>>>(a);
  else packed_join_fwd_kernel<bf16_t><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_packed_attn_bwd(int dtype, const PackedAttnArgs& args, void* workspace, size_t bytes, hipStream_t s) {
  PackedAttnArgs a = with_divisors(args);
  const Shares n = shares(dtype, a);
  const Layout l = layout(a, n);
  if (bytes < l.total) return hipErrorInvalidValue;
  a.dsum = reinterpret_cast<float*>(workspace);
  a.nlse = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + l.stats);
  a.part = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + l.shares);
  hipError_t e = hipSuccess;
  if (a.q_rows > 0) {
    a.shares = n.rows;
    e = dtype == 0 ? launch_packed_dq_f32(a, s) : with_width(a.dh, [&](auto w) { return dq_mfma<decltype(w)::value>(a, s); });
    if (e != hipSuccess) return e;
    if (a.shares > 1) {
      const unsigned grid = (unsigned)(((long)a.q_rows * a.heads + 3) / 4);
      if (dtype == 0) packed_join_dq_kernel<float><<<grid, 256, 0, s>>>(a);
      else packed_join_dq_kernel<bf16_t><<<grid, 256, 0, s>>>(a);
    }
  }
  if (a.k_rows > 0) {
    a.shares = n.keys;
    e = dtype == 0 ? launch_packed_dkdv_f32(a, s) : with_width(a.dh, [&](auto w) { return dkdv_mfma<decltype(w)::value>(a, s); });
    if (e != hipSuccess) return e;
    if (a.shares > 1) {
      const unsigned grid = (unsigned)(((long)a.k_rows * a.kv_heads + 3) / 4);
      if (dtype == 0) packed_join_dkdv_kernel<float><<<grid, 256, 0, s>>>(a);
      else packed_join_dkdv_kernel<bf16_t><<<grid, 256, 0, s>>>(a);
    }
  }
  return hipGetLastError();
}

}  // namespace hbp
