// Attention over packed sequences in fp32 storage, on the matrix cores' fp32 products (v_mfma_f32_32x32x2_f32: a wavefront's
// 32 x 32 products of 2 take 64 clocks, 157 TFLOP/s in all, so that little else matters).
//
// The shapes are those of the bf16 kernels (attention_packed.hip): a lane owns one row (dk, dv: one key) and half of its scores, which
// enter the second product straight from the registers.  A product of contraction length 2 takes one number per lane from either
// side; which channel that is may be chosen freely as long as both sides agree, so four of them come from one 16-byte read.
// Four wavefronts; the other side streams in tiles of 32 rows through LDS.
#include "attention_packed.h"

namespace hbp {

namespace {

constexpr int WAVES = 4;

__device__ __forceinline__ float16v mfma_f32(float x, float y, float16v acc) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(x, y, acc, 0, 0, 0);
}

// W channels of fp32 in tiles of 64 or 128 are the bytes of twice as many of bf16: the tiles' layout is that.
template <int W>
struct Tiles {
  typedef Geo<2 * padded<W>()> G;
  typedef float floatv4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) const floatv4* chunk_p;
  typedef __attribute__((address_space(3))) const float* one_p;
  static constexpr int J = W / 8, MB = W / 32;
  // A tile's row l % 32: this half's four channels 8 j + 4 (l / 32) .. + 3.
  static __device__ __forceinline__ unsigned cols_lane(int lane) {
    const int r = lane & 31;
    return (unsigned)(r * G::RB + (((lane >> 5) ^ G::swz(r)) << 4));
  }
  static __device__ __forceinline__ floatv4 cols(unsigned at, unsigned tile, int j) {
    return *(chunk_p)(uintptr_t)((at ^ (32u * j)) + tile);
  }
  // Column 32 m + l % 32 of the tile's row tile_row_of(e, l / 32): what accumulator element e of the first product meets.
  static __device__ __forceinline__ unsigned rows_lane(int lane) {
    const int hh = lane >> 5;
    return (unsigned)(4 * hh * G::RB + ((((lane & 31) >> 2) ^ hh) << 4) + (lane & 3) * 4);
  }
  static __device__ __forceinline__ float rows(unsigned at, unsigned tile, int m, int e) {
    const unsigned bits = (unsigned)((8 * m) ^ ((e & 3) << 2) ^ (2 * ((e >> 2) & 1))) << 4;
    return *(one_p)(uintptr_t)((at ^ bits) + (tile + (unsigned)(8 * (e >> 2) + (e & 3)) * G::RB));
  }
  // this lane's own row: channels 8 j + 4 (l / 32) .. + 3, zero past the head's width
  static __device__ __forceinline__ void own(const float* row, int dh, int lane, float (&v)[4 * J]) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * j + 4 * (lane >> 5);
      const float4 x = *reinterpret_cast<const float4*>(row + (c < dh ? c : 0));
      v[4 * j] = c < dh ? x.x : 0.f;
      v[4 * j + 1] = c < dh ? x.y : 0.f;
      v[4 * j + 2] = c < dh ? x.z : 0.f;
      v[4 * j + 3] = c < dh ? x.w : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4 * J; ++i) landed(v[i]);
  }
  // acc += the tile's rows times the own row
  static __device__ __forceinline__ float16v product(unsigned at, unsigned tile, const float (&own)[4 * J], float16v acc) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const floatv4 x = cols(at, tile, j);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = mfma_f32(x[i], own[4 * j + i], acc);
    }
    return acc;
  }
  // acc += the tile's columns times the scores
  static __device__ __forceinline__ void add(unsigned at, unsigned tile, const float16v& s, float16v (&acc)[MB]) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int m = 0; m < MB; ++m) acc[m] = mfma_f32(rows(at, tile, m, e), s[e], acc[m]);
  }
};

// Stages of 2 NT tiles of 32 rows, NT of x, then NT of y, that the workgroup copies together, a wavefront whole tiles or parts of one; rows
// past the last (of n) repeat it.  NST stages: two, or one where two do not fit, which is then filled between two barriers.
template <int W, int NT>
struct PairStream {
  static constexpr int DHP = 2 * padded<W>();
  typedef Geo<DHP> G;
  static constexpr int STAGE = 2 * NT * G::TB, NST = 2 * STAGE <= 128 * 1024 ? 2 : 1;
  static constexpr int PW = 2 * NT * G::COPIES / WAVES, TILES = PW < G::COPIES ? 1 : PW / G::COPIES, PARTS = PW / TILES;
  unsigned lds, ldx, ldy;
  int first_tile, part, dh4;
  __device__ __forceinline__ PairStream(unsigned ldx_, unsigned ldy_, int dh, unsigned lds0, int w) {
    first_tile = w * PW / G::COPIES;
    part = w * PW % G::COPIES;
    dh4 = dh >> 2;
    ldx = ldx_;
    ldy = ldy_;
    lds = lds0 + (unsigned)(w * PW) * 1024u;
  }
  // this wavefront's copies of its i-th tile (of x: tile() < NT), whose row 0 is at `base` and which has n rows from there
  __device__ __forceinline__ int tile(int i) const { return first_tile + i; }
  __device__ __forceinline__ void issue(int i, const float* base, int n, int at, int lane) const {
    const unsigned ld = tile(i) < NT ? ldx : ldy, dst = lds + (unsigned)at * STAGE + (unsigned)(i * PARTS) * 1024u;
#pragma unroll
    for (int u = 0; u < PARTS; ++u) copy16_to_lds(copy_offset<DHP>(ld, part + u, n, dh4, lane), base, dst + 1024u * u);
  }
};
// Before the compute of step i of from .. to - 1: its stage is full.  ask(step, stage) issues the copies.
template <int NST, typename F>
__device__ __forceinline__ int next_stage(int i, int from, int to, F ask) {
  if (NST == 1) {
    if (i > from) {
      workgroup_handover();                                // everyone is done with the step before
      ask(i, 0);
    }
    copies_in_flight<0>();
    workgroup_handover();
    return 0;
  }
  copies_in_flight<0>();
  workgroup_handover();
  if (i + 1 < to) ask(i + 1, (i + 1) & 1);
  return i & 1;
}

// Blocks of 32 channels from block m0 on: a lane holds columns 32 m + 8 g + 4 (l / 32) .. + 3 of its row.
template <int MB>
__device__ __forceinline__ void store_row(float* row, const float16v (&acc)[MB], float f, int m0, int dh, int hh) {
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * (m0 + m) + 8 * g + 4 * hh;
      if (c < dh)
        *reinterpret_cast<float4*>(row + c) = make_float4(acc[m][4 * g] * f, acc[m][4 * g + 1] * f, acc[m][4 * g + 2] * f, acc[m][4 * g + 3] * f);
    }
}

// the end of N blocks' channels
template <int N> __device__ __forceinline__ int past_block(int m0, int dh) { return 32 * (m0 + N) < dh ? 32 * (m0 + N) : dh; }

// How the four wavefronts share rows and keys.  COLS = 1: 128 rows, 32 for each wavefront, steps of 32 keys.  COLS = 4, for few rows: 32 rows,
// steps of 128 keys of which a wavefront takes 32; they meet in LDS at the end.
template <int COLS> constexpr int rows_of_block() { return 32 * WAVES / COLS; }
template <int W, int COLS>
struct RowBlock {
  static constexpr int ROWS = rows_of_block<COLS>(), NT = COLS, KEYS = 32 * NT;
  typedef PairStream<W, NT> PS;
  Tile x;
  int w0, rows_left, mine, fewest, most, from, to, share;  // from .. to - 1: this workgroup's share of the steps
  RowPlace me;
  const float *k, *v;
  __device__ __forceinline__ bool find(const PackedAttnArgs& a, int rw, int lane) {
    x = find_tile<false>(a, ROWS, lane);
    if (!x.exists) return false;
    const int R = x.s.nq * a.group, r0 = ROWS * x.t;
    w0 = r0 + 32 * rw;
    rows_left = R - w0;
    auto seen = [&](int r) __attribute__((always_inline)) { return seen_by(x.s, place_of(a, x.hk, r).i, a.causal); };
    const int steps = (seen((R < r0 + ROWS ? R : r0 + ROWS) - 1) + KEYS - 1) / KEYS;
    share = (int)blockIdx.y;
    from = (int)((long)steps * share / a.shares);
    to = (int)((long)steps * (share + 1) / a.shares);
    const int r = rows_left > 0 ? w0 + ((lane & 31) < rows_left ? (lane & 31) : rows_left - 1) : R - 1;
    me = place_of(a, x.hk, r);
    mine = seen_by(x.s, me.i, a.causal);
    fewest = rows_left > 0 ? seen(w0) : 0;
    most = rows_left > 0 ? seen(w0 + (rows_left < 32 ? rows_left : 32) - 1) : 0;
    k = row_of<float>(a.k, x.s.k0, x.hk);
    v = row_of<float>(a.v, x.s.k0, x.hk);
    return true;
  }
  __device__ __forceinline__ void ask(const PS& ps, const PackedAttnArgs& a, int i, int at, int lane) const {
#pragma unroll
    for (int u = 0; u < PS::TILES; ++u) {
      const int t = ps.tile(u);
      int first = KEYS * i + 32 * (t % NT);
      first = first < x.s.nk ? first : x.s.nk - 1;
      ps.issue(u, (t < NT ? k : v) + (long)first * (t < NT ? a.k.row : a.v.row), x.s.nk - first < 32 ? x.s.nk - first : 32, at, lane);
    }
  }
};
// The wavefronts' outputs, [wavefront][block][element][lane], into block m of their sum, each times its f.
template <int MB>
__device__ __forceinline__ void put_sums(float* sums, int wave, const float16v (&acc)[MB], int lane) {
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[((wave * MB + m) * 16 + e) * 64 + lane] = acc[m][e];
}
template <int MB>
__device__ __forceinline__ void get_sums(const float* sums, int m, const float (&f)[WAVES], float16v (&acc)[1], int lane) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < WAVES; ++j) t = fmaf(f[j], sums[((j * MB + m) * 16 + e) * 64 + lane], t);
    acc[0][e] = t;
  }
}
template <int W, int NT> constexpr int ring_bytes() {
  typedef PairStream<W, NT> PS;
  constexpr int ring = PS::NST * PS::STAGE, sums = NT == 1 ? 0 : WAVES * Tiles<W>::MB * 16 * 64 * 4;
  return ring > sums ? ring : sums;
}

// what was read of LDS before has arrived, and all but N copies
template <int N>
__device__ __forceinline__ void read_and_in_flight() {
  asm volatile("" ::: "memory");
  copies_in_flight_read<N>();
}
// COLS = 4: a wavefront copies the tiles that it reads, its k and its v of every step, and waits for nobody.  (x: tile 0, y: tile 1 of its
// stage, each of Geo::COPIES copies.)  Two stages, or one where two do not fit: then k of the next step comes while v of this one is used.
// (One token for each of 44 sequences over 1910 keys, 8 heads of 128: 188 us, 3.7 TB/s; with stages that the workgroup fills together 238.  8
// heads of 64 on 2, 60 over 2000: 43 and 45; 2 over 10229, one head of 96, four steps a workgroup: 31 and 30.)
template <int W>
struct OwnStream {
  static constexpr int DHP = 2 * padded<W>();
  typedef Geo<DHP> G;
  static constexpr int NST = PairStream<W, 4>::NST, STAGE = PairStream<W, 4>::STAGE, N = G::COPIES;
  unsigned lds, ldk, ldv;
  const float *k, *v;
  int nk, dh4;
  // keys 32 t .. of the sequence, at most 32 of them, rows past the last repeat it
  __device__ __forceinline__ void tile(const float* x, unsigned ld, int first, unsigned dst, int lane) const {
    const int n = nk - first < 32 ? nk - first : 32;
    const float* base = x + (long)first * (ld >> 2);
#pragma unroll
    for (int u = 0; u < N; ++u) copy16_to_lds(copy_offset<DHP>(ld, u, n, dh4, lane), base, dst + 1024u * u);
  }
  __device__ __forceinline__ void ask_k(int first, int at, int lane) const { tile(k, ldk, first, lds + (unsigned)at * STAGE, lane); }
  __device__ __forceinline__ void ask_v(int first, int at, int lane) const { tile(v, ldv, first, lds + (unsigned)at * STAGE + 4 * G::TB, lane); }
};

template <int W, int COLS>
__global__ __launch_bounds__(64 * WAVES, COLS == 1 ? 2 : 1) void packed_fwd_f32_kernel(PackedAttnArgs a) {
  typedef Tiles<W> T;
  typedef RowBlock<W, COLS> RB;
  typedef typename RB::PS PS;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[ring_bytes<W, COLS>()];
  __shared__ float stats[COLS == 1 ? 1 : WAVES][2][64];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), rw = COLS == 1 ? wave : 0, col = COLS == 1 ? 0 : wave;
  RB b;
  if (!b.find(a, rw, lane)) return;
  const Seq& s = b.x.s;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const PS ps((unsigned)(a.k.row * 4), (unsigned)(a.v.row * 4), a.dh, lds0, wave);
  auto ask = [&](int i, int at) __attribute__((always_inline)) { b.ask(ps, a, i, at, lane); };
  typedef OwnStream<W> OS;
  const OS os{lds0 + (unsigned)wave * T::G::TB, (unsigned)(a.k.row * 4), (unsigned)(a.v.row * 4), b.k, b.v, s.nk, a.dh >> 2};
  // the last step in which this wavefront's keys are seen, and one
  int own_to = b.most > 32 * col ? (b.most - 32 * col + RB::KEYS - 1) / RB::KEYS : 0;
  own_to = own_to < b.to ? own_to : b.to;
  if constexpr (COLS == 1) {
    if (b.from < b.to) ask(b.from, PS::NST == 1 ? 0 : b.from & 1);
  } else if (b.from < own_to) {
    os.ask_k(RB::KEYS * b.from + 32 * col, 0, lane);
    os.ask_v(RB::KEYS * b.from + 32 * col, 0, lane);
  }
  float q[4 * T::J];
  T::own(row_of<float>(a.q, s.q0 + b.me.i, b.me.h), a.dh, lane, q);
  const unsigned ck = lds0 + T::cols_lane(lane) + (unsigned)col * T::G::TB, rv = lds0 + T::rows_lane(lane) + (unsigned)col * T::G::TB;
  const float c = a.scale * LOG2E;
  float16v o[T::MB];
  zero_acc(o);
  float m = -FLT_MAX, l = 0.f;
  // keys first .. + 31: their scores, which become weights, relative to the row's maximum
  auto weigh = [&](float16v (&sc)[1], int first) __attribute__((always_inline)) {
    if (first + 32 > b.fewest) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (first + tile_row_of(e, hh) >= b.mine) sc[0][e] = -INFINITY;
    }
    float top = sc[0][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, sc[0][e]);
    top = max_of_halves(top) * c;
    if (__any(top > m + 8.f)) {                            // (see the bf16 kernel)
      const float mn = fmaxf(m, top), alpha = fast_exp2(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[mb][e] *= alpha;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      sc[0][e] = fast_exp2(fmaf(sc[0][e], c, -m));
      l += sc[0][e];
    }
  };
  if constexpr (COLS == 1) {
    for (int i = b.from; i < b.to; ++i) {
      const unsigned at = (unsigned)next_stage<PS::NST>(i, b.from, b.to, ask) * PS::STAGE;
      const int first = RB::KEYS * i;
      if (first >= b.most) continue;
      float16v sc[1];
      zero_acc(sc);
      sc[0] = T::product(ck + at, 0, q, sc[0]);
      weigh(sc, first);
      T::add(rv + at, RB::NT * T::G::TB, sc[0], o);
    }
  } else {
    for (int i = b.from; i < own_to; ++i) {
      const int first = RB::KEYS * i + 32 * col, next = first + RB::KEYS, st = OS::NST == 1 ? 0 : (i - b.from) & 1;
      const bool more = i + 1 < own_to;
      const unsigned at = (unsigned)st * OS::STAGE;
      read_and_in_flight<OS::NST == 1 ? OS::N : 0>();   // (k is here; the other stage's reads as well)
      if (OS::NST == 2 && more) {
        os.ask_k(next, st ^ 1, lane);
        os.ask_v(next, st ^ 1, lane);
      }
      float16v sc[1];
      zero_acc(sc);
      sc[0] = T::product(ck + at, 0, q, sc[0]);
      if (OS::NST == 1) {
        read_and_in_flight<OS::N>();                    // (k has been read)
        if (more) os.ask_k(next, 0, lane);
      }
      weigh(sc, first);
      if (OS::NST == 1) {
        if (more) read_and_in_flight<OS::N>();
        else read_and_in_flight<0>();                   // (v is here)
      }
      T::add(rv + at, RB::NT * T::G::TB, sc[0], o);
      if (OS::NST == 1 && more) {
        read_and_in_flight<OS::N>();                    // (v has been read)
        os.ask_v(next, 0, lane);
      }
    }
  }
  l += other_half(l);
  const long n = s.q0 + b.me.i, r = n * a.heads + b.me.h, p = (long)b.share * a.q_rows * a.heads + r;
  const bool there = (lane & 31) < b.rows_left;
  // blocks m0 .. of the rows' outputs, sums l relative to m
  auto leave = [&](auto& acc, int m0, float m, float l) __attribute__((always_inline)) {
    constexpr int N = sizeof(acc) / sizeof(acc[0]);
    if (a.shares > 1) {
      if (there) {
        store_share<N>(a.part, p, acc, m0, a.dh, hh);
        if (hh == 0 && m0 == 0) {
          a.part_stats[2 * p] = m;
          a.part_stats[2 * p + 1] = l;
        }
      }
      return;
    }
    const float f = inverse_sum(m, l);
    if (there) {
      store_row(row_out<float>(a.o, n, b.me.h), acc, f, m0, a.dh, hh);
      if (hh == 0 && m0 == 0) a.lse[r] = l == 0.f ? -INFINITY : m + log2f(l);
    }
    redo_rows(not_finite(acc, f * 0.f), b.rows_left, [&](int j) {
      const RowPlace q = place_of(a, b.x.hk, b.w0 + j);
      one_forward<float>(a, s, q.i, q.h, 32 * m0, past_block<N>(m0, a.dh), lane);
    });
  };
  if constexpr (COLS == 1) {
    if (b.rows_left > 0) leave(o, 0, m, l);
  } else {
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(ring);
    put_sums(sums, wave, o, lane);
    stats[wave][0][lane] = m;
    stats[wave][1][lane] = l;
    __syncthreads();
    if (col >= T::MB) return;                              // (a block of 32 channels each)
    float f[WAVES], top = stats[0][0][lane], sum = 0.f;
#pragma unroll
    for (int j = 1; j < WAVES; ++j) top = fmaxf(top, stats[j][0][lane]);
#pragma unroll
    for (int j = 0; j < WAVES; ++j) {
      f[j] = fast_exp2(stats[j][0][lane] - top);
      sum = fmaf(f[j], stats[j][1][lane], sum);
    }
    float16v acc[1];
    get_sums<T::MB>(sums, col, f, acc, lane);
    leave(acc, col, top, sum);
  }
}

template <int W, int COLS>
__global__ __launch_bounds__(64 * WAVES, COLS > 1 || W > 96 ? 1 : 2) void packed_dq_f32_kernel(PackedAttnArgs a) {
  typedef Tiles<W> T;
  typedef RowBlock<W, COLS> RB;
  typedef typename RB::PS PS;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[ring_bytes<W, COLS>()];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), rw = COLS == 1 ? wave : 0, col = COLS == 1 ? 0 : wave;
  RB b;
  if (!b.find(a, rw, lane)) return;
  const Seq& s = b.x.s;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const PS ps((unsigned)(a.k.row * 4), (unsigned)(a.v.row * 4), a.dh, lds0, wave);
  auto ask = [&](int i, int at) __attribute__((always_inline)) { b.ask(ps, a, i, at, lane); };
  if (b.from < b.to) ask(b.from, PS::NST == 1 ? 0 : b.from & 1);
  const long n = s.q0 + b.me.i, r = n * a.heads + b.me.h;
  float L = a.lse[r];
  float q[4 * T::J], g[4 * T::J], D = 0.f;
  {
    float o[4 * T::J];
    T::own(row_of<float>(a.dout, n, b.me.h), a.dh, lane, g);
    T::own(row_of<float>(a.o, n, b.me.h), a.dh, lane, o);
#pragma unroll
    for (int i = 0; i < 4 * T::J; ++i) D = fmaf(g[i], o[i], D);
  }
  T::own(row_of<float>(a.q, n, b.me.h), a.dh, lane, q);
  landed(L);
  D += other_half(D);
  L = stat_of(L);
  if (hh == 0 && col == 0 && b.share == 0 && lane < b.rows_left) {
    a.dsum[r] = -D;
    a.nlse[r] = -L;
  }
  const unsigned ck = lds0 + T::cols_lane(lane) + (unsigned)col * T::G::TB, rk = lds0 + T::rows_lane(lane) + (unsigned)col * T::G::TB;
  const float c = a.scale * LOG2E;
  float16v dq[T::MB];
  zero_acc(dq);
  for (int i = b.from; i < b.to; ++i) {
    const unsigned at = (unsigned)next_stage<PS::NST>(i, b.from, b.to, ask) * PS::STAGE;
    const int first = RB::KEYS * i + 32 * col;
    if (first >= b.most) continue;
    float16v sc[1], dp;
    zero_acc(sc);
#pragma unroll
    for (int e = 0; e < 16; ++e) dp[e] = -D;
    sc[0] = T::product(ck + at, 0, q, sc[0]);
    dp = T::product(ck + at, RB::NT * T::G::TB, g, dp);
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[0][e] = fast_exp2(fmaf(sc[0][e], c, -L)) * dp[e];
    if (first + 32 > b.fewest) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (first + tile_row_of(e, hh) >= b.mine) sc[0][e] = 0.f;
    }
    T::add(rk + at, 0, sc[0], dq);
  }
  const bool there = (lane & 31) < b.rows_left;
  auto leave = [&](auto& acc, int m0) __attribute__((always_inline)) {
    constexpr int N = sizeof(acc) / sizeof(acc[0]);
    if (a.shares > 1) {
      if (there) store_share<N>(a.part, (long)b.share * a.q_rows * a.heads + r, acc, m0, a.dh, hh);
      return;
    }
    if (there) store_row(row_out<float>(a.dq, n, b.me.h), acc, a.scale, m0, a.dh, hh);
    redo_rows(not_finite(acc, 0.f), b.rows_left, [&](int j) {
      const RowPlace p = place_of(a, b.x.hk, b.w0 + j);
      one_dq<float>(a, s, p.i, p.h, row_dsum<float>(a, s.q0 + p.i, p.h, lane), 32 * m0, past_block<N>(m0, a.dh), lane);
    });
  };
  if constexpr (COLS == 1) {
    if (b.rows_left > 0) leave(dq, 0);
  } else {
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(ring);
    put_sums(sums, wave, dq, lane);
    __syncthreads();
    if (col >= T::MB) return;
    const float f[WAVES] = {1.f, 1.f, 1.f, 1.f};
    float16v acc[1];
    get_sums<T::MB>(sums, col, f, acc, lane);
    leave(acc, col);
  }
}

// Queries from the last tile down, all heads of the group for one tile before the next.  TURNS = 1: 128 keys, 32 for each wavefront; 4, for
// few keys: 32, and the wavefronts take every fourth tile of queries in turn.
template <int W, int TURNS>
__global__ __launch_bounds__(64 * WAVES, TURNS > 1 || W > 64 ? 1 : 2) void packed_dkdv_f32_kernel(PackedAttnArgs a) {
  typedef Tiles<W> T;
  typedef PairStream<W, TURNS> PS;
  constexpr int NT = TURNS, KEYS = 32 * WAVES / TURNS;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[ring_bytes<W, TURNS>()];
  __shared__ __attribute__((aligned(256))) float stats[PS::NST][NT][2][64];      // [stage][tile][-lse | -D][32 rows, and again]
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), turn = TURNS == 1 ? 0 : wave, kw = TURNS == 1 ? wave : 0;
  const Tile x = find_tile<true>(a, KEYS, lane);
  if (!x.exists) return;
  const Seq& s = x.s;
  const int w0 = KEYS * x.t + 32 * kw, keys_left = s.nk - w0;
  const int nq = s.nq, shift = s.nk - nq;
  auto first_query = [&](int key) __attribute__((always_inline)) {
    const int i = key - shift;
    return !a.causal || i < 0 ? 0 : i;
  };
  const int top = (nq - 1) >> 5;
  const int tiles = nq > 0 ? (top + 1 - (first_query(KEYS * x.t) >> 5)) * a.group : 0, all_steps = (tiles + NT - 1) / NT;
  const int share = (int)blockIdx.y;
  const int from = (int)((long)all_steps * share / a.shares), to = (int)((long)all_steps * (share + 1) / a.shares);
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const unsigned lds1 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(stats));
  const PS ps((unsigned)(a.q.row * 4), (unsigned)(a.dout.row * 4), a.dh, lds0, wave);
  // tile j of the list: its head of the group and its first query (past the list's end: one that nobody reads)
  struct Place { int h, first; };
  auto place = [&](int j) __attribute__((always_inline)) {
    const int down = (int)a.by_group.quotient((unsigned)j);
    return Place{x.hk * a.group + j - down * a.group, down > top ? 0 : 32 * (top - down)};
  };
  auto ask = [&](int i, int at) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < PS::TILES; ++u) {
      const int t = ps.tile(u);
      const Place p = place(NT * i + t % NT);
      ps.issue(u, row_of<float>(t < NT ? a.q : a.dout, s.q0 + p.first, p.h), nq - p.first < 32 ? nq - p.first : 32, at, lane);
    }
    // (NT = 1: the wavefronts copy the same two)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = wave % NT;
      const Place p = place(NT * i + t);
      const int r = p.first + (lane & 31) < nq ? p.first + (lane & 31) : nq - 1;
      copy4_to_lds((u ? a.dsum : a.nlse) + (long)(s.q0 + r) * a.heads + p.h, lds1 + (unsigned)at * (NT * 512u) + (unsigned)(2 * t + u) * 256u);
    }
  };
  if (from < to) ask(from, PS::NST == 1 ? 0 : from & 1);
  const int key = keys_left > 0 ? w0 + ((lane & 31) < keys_left ? (lane & 31) : keys_left - 1) : s.nk - 1;
  float k[4 * T::J], v[4 * T::J];
  T::own(row_of<float>(a.k, s.k0 + key, x.hk), a.dh, lane, k);
  T::own(row_of<float>(a.v, s.k0 + key, x.hk), a.dh, lane, v);
  const unsigned cq = lds0 + T::cols_lane(lane) + (unsigned)turn * T::G::TB, rq = lds0 + T::rows_lane(lane) + (unsigned)turn * T::G::TB;
  const int mine = first_query(key);
  const int begin = keys_left > 0 ? first_query(w0) : nq, all = keys_left > 0 ? first_query(w0 + (keys_left < 32 ? keys_left : 32) - 1) : nq;
  const float c = a.scale * LOG2E;
  float16v dk[T::MB], dv[T::MB];
  zero_acc(dk);
  zero_acc(dv);
  for (int i = from; i < to; ++i) {
    const int st = next_stage<PS::NST>(i, from, to, ask);
    const int j = NT * i + turn, first = place(j).first;
    if (j >= tiles || first + 32 <= begin || keys_left <= 0) continue;
    const unsigned at = (unsigned)st * PS::STAGE;
    float16v sc[1], dp;
    zero_acc(sc);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 u = *reinterpret_cast<const float4*>(&stats[st][turn][1][8 * g + 4 * hh]);
      dp[4 * g] = u.x; dp[4 * g + 1] = u.y; dp[4 * g + 2] = u.z; dp[4 * g + 3] = u.w;
    }
    sc[0] = T::product(cq + at, 0, k, sc[0]);
    dp = T::product(cq + at, NT * T::G::TB, v, dp);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 u = *reinterpret_cast<const float4*>(&stats[st][turn][0][8 * g + 4 * hh]);
      sc[0][4 * g] = fast_exp2(fmaf(sc[0][4 * g], c, u.x));
      sc[0][4 * g + 1] = fast_exp2(fmaf(sc[0][4 * g + 1], c, u.y));
      sc[0][4 * g + 2] = fast_exp2(fmaf(sc[0][4 * g + 2], c, u.z));
      sc[0][4 * g + 3] = fast_exp2(fmaf(sc[0][4 * g + 3], c, u.w));
    }
    if (first < all || first + 32 > nq) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int r = first + tile_row_of(e, hh);
        if (r < mine || r >= nq) sc[0][e] = 0.f;
      }
    }
    T::add(rq + at, NT * T::G::TB, sc[0], dv);
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[0][e] *= dp[e];
    T::add(rq + at, 0, sc[0], dk);
  }
  const bool there = (lane & 31) < keys_left;
  const long r = (long)(s.k0 + key) * a.kv_heads + x.hk, rows = (long)a.k_rows * a.kv_heads;
  auto leave = [&](auto& k_sum, auto& v_sum, int m0) __attribute__((always_inline)) {
    constexpr int N = sizeof(k_sum) / sizeof(k_sum[0]);
    if (a.shares > 1) {
      if (there) {
        store_share<N>(a.part, share * rows + r, k_sum, m0, a.dh, hh);
        store_share<N>(a.part, (a.shares + share) * rows + r, v_sum, m0, a.dh, hh);
      }
      return;
    }
    if (there) {
      store_row(row_out<float>(a.dk, s.k0 + key, x.hk), k_sum, a.scale, m0, a.dh, hh);
      store_row(row_out<float>(a.dv, s.k0 + key, x.hk), v_sum, 1.f, m0, a.dh, hh);
    }
    redo_rows(not_finite(v_sum, not_finite(k_sum, 0.f)), keys_left, [&](int j) {
      one_dkdv<float>(a, s, w0 + j, x.hk, DK | DV, 32 * m0, past_block<N>(m0, a.dh), lane);
    });
  };
  if constexpr (TURNS == 1) {
    if (keys_left > 0) leave(dk, dv, 0);
  } else {
    float* const sums = reinterpret_cast<float*>(ring);
    const float f[WAVES] = {1.f, 1.f, 1.f, 1.f};
    float16v k_sum[1], v_sum[1];
    __syncthreads();
    put_sums(sums, wave, dk, lane);
    __syncthreads();
    if (wave < T::MB) get_sums<T::MB>(sums, wave, f, k_sum, lane);
    __syncthreads();
    put_sums(sums, wave, dv, lane);
    __syncthreads();
    if (wave >= T::MB) return;
    get_sums<T::MB>(sums, wave, f, v_sum, lane);
    leave(k_sum, v_sum, wave);
  }
}

}  // namespace

hipError_t launch_packed_fwd_f32(const PackedAttnArgs& a, hipStream_t s) {
  return with_width(a.dh, [&](auto w) {
    constexpr int W = decltype(w)::value;
    if (f32_wide<false>(a)) packed_fwd_f32_kernel<W, 1><<<grid_of(tile_grid<false>(a, 128), a.shares), 64 * WAVES, 0, s>>>(a);
    else packed_fwd_f32_kernel<W, 4><<<grid_of(tile_grid<false>(a, 32), a.shares), 64 * WAVES, 0, s>>>(a);
    return hipGetLastError();
  });
}
hipError_t launch_packed_dq_f32(const PackedAttnArgs& a, hipStream_t s) {
  return with_width(a.dh, [&](auto w) {
    constexpr int W = decltype(w)::value;
    if (f32_wide<false>(a)) packed_dq_f32_kernel<W, 1><<<grid_of(tile_grid<false>(a, 128), a.shares), 64 * WAVES, 0, s>>>(a);
    else packed_dq_f32_kernel<W, 4><<<grid_of(tile_grid<false>(a, 32), a.shares), 64 * WAVES, 0, s>>>(a);
    return hipGetLastError();
  });
}
hipError_t launch_packed_dkdv_f32(const PackedAttnArgs& a, hipStream_t s) {
  return with_width(a.dh, [&](auto w) {
    constexpr int W = decltype(w)::value;
    if (f32_wide<true>(a)) packed_dkdv_f32_kernel<W, 1><<<grid_of(tile_grid<true>(a, 128), a.shares), 64 * WAVES, 0, s>>>(a);
    else packed_dkdv_f32_kernel<W, 4><<<grid_of(tile_grid<true>(a, 32), a.shares), 64 * WAVES, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace hbp
