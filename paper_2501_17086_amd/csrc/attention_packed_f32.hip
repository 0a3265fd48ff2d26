// Attention over packed sequences in fp32 storage, on the matrix cores' fp32 products (v_mfma_f32_32x32x2_f32: a wavefront's
// 32 x 32 products of 2 take 64 clocks, 157 TFLOP/s in all, so that little else matters).
//
// The shapes are those of the bf16 kernels (attention_packed.hip): a lane owns one row (dk, dv: one key) and half of its scores, which
// enter the second product straight from the registers.  A product of contraction length 2 takes one number per lane from either
// side; which channel that is may be chosen freely as long as both sides agree, so four of them come from one 16-byte read.
// Four wavefronts of 32 rows (keys); the other side streams in tiles of 32 through two stages of LDS.
#include "attention_packed.h"

namespace hbp {

namespace {

constexpr int WAVES = 4, ROWS = F32_ROWS;
static_assert(ROWS == 32 * WAVES, "a wavefront has 32 rows");

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
  static constexpr int STAGE = 2 * G::TB, J = W / 8, MB = W / 32;
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

// Two tiles of 32 rows, x then y, that the workgroup copies into a stage together; rows past the last (of n) repeat it.
template <int W>
struct PairStream {
  static constexpr int DHP = 2 * padded<W>();
  typedef Geo<DHP> G;
  static constexpr int PW = 2 * G::COPIES / WAVES;
  unsigned off[PW], ld, lds;
  int tile, part, dh4;
  __device__ __forceinline__ PairStream(unsigned ldx, unsigned ldy, int dh, unsigned lds0, int w, int lane) {
    static_assert(G::COPIES % PW == 0, "a wavefront's copies are of one tile");
    tile = w * PW / G::COPIES;
    part = w * PW % G::COPIES;
    dh4 = dh >> 2;
    ld = tile ? ldy : ldx;
    lds = lds0 + (unsigned)(w * PW) * 1024u;
#pragma unroll
    for (int u = 0; u < PW; ++u) off[u] = copy_offset<DHP>(ld, part + u, 32, dh4, lane);
  }
  // x, y: row 0; rows first .. into stage `at`
  __device__ __forceinline__ void issue(const float* x, const float* y, int first, int n, int at, int lane) const {
    const unsigned char* base = reinterpret_cast<const unsigned char*>(tile ? y : x) + (long)first * ld;
    const unsigned dst = lds + (unsigned)at * (2u * G::TB);
#pragma unroll
    for (int u = 0; u < PW; ++u)
      copy16_to_lds(first + 32 <= n ? off[u] : copy_offset<DHP>(ld, part + u, n - first, dh4, lane), base, dst + 1024u * u);
  }
};

// a lane holds columns 32 m + 8 g + 4 (l / 32) .. + 3 of its row
template <int MB>
__device__ __forceinline__ void store_row(float* row, const float16v (&acc)[MB], float f, int dh, int hh) {
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * m + 8 * g + 4 * hh;
      if (c < dh)
        *reinterpret_cast<float4*>(row + c) = make_float4(acc[m][4 * g] * f, acc[m][4 * g + 1] * f, acc[m][4 * g + 2] * f, acc[m][4 * g + 3] * f);
    }
}

// The rows of a workgroup and what its wavefronts see of the keys.
struct RowBlock {
  Tile x;
  int w0, rows_left, mine, fewest, most, from, to, share;  // from .. to - 1: this workgroup's share of the steps
  RowPlace me;
  __device__ __forceinline__ bool find(const PackedAttnArgs& a, int wave, int lane) {
    x = find_tile<false>(a, ROWS, lane);
    if (!x.exists) return false;
    const int R = x.s.nq * a.group, r0 = ROWS * x.t;
    w0 = r0 + 32 * wave;
    rows_left = R - w0;
    auto seen = [&](int r) __attribute__((always_inline)) { return seen_by(x.s, place_of(a, x.hk, r).i, a.causal); };
    const int steps = (seen((R < r0 + ROWS ? R : r0 + ROWS) - 1) + 31) >> 5;
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

template <int W>
__global__ __launch_bounds__(64 * WAVES, 2) void packed_fwd_f32_kernel(PackedAttnArgs a) {
  typedef Tiles<W> T;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[2 * T::STAGE];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  RowBlock b;
  if (!b.find(a, wave, lane)) return;
  const Seq& s = b.x.s;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const PairStream<W> ps((unsigned)(a.k.row * 4), (unsigned)(a.v.row * 4), a.dh, lds0, wave, lane);
  const float* k = row_of<float>(a.k, s.k0, b.x.hk);
  const float* v = row_of<float>(a.v, s.k0, b.x.hk);
  if (b.from < b.to) ps.issue(k, v, 32 * b.from, s.nk, b.from & 1, lane);
  float q[4 * T::J];
  T::own(row_of<float>(a.q, s.q0 + b.me.i, b.me.h), a.dh, lane, q);
  const unsigned ck = lds0 + T::cols_lane(lane), rv = lds0 + T::rows_lane(lane);
  const float c = a.scale * LOG2E;
  float16v o[T::MB];
  zero_acc(o);
  float m = -FLT_MAX, l = 0.f;
  for (int i = b.from; i < b.to; ++i) {
    copies_in_flight<0>();
    workgroup_handover();
    if (i + 1 < b.to) ps.issue(k, v, 32 * (i + 1), s.nk, (i + 1) & 1, lane);
    if (32 * i >= b.most) continue;
    const unsigned at = (unsigned)(i & 1) * T::STAGE;
    float16v sc[1];
    zero_acc(sc);
    sc[0] = T::product(ck + at, 0, q, sc[0]);
    if (32 * i + 32 > b.fewest) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (32 * i + tile_row_of(e, hh) >= b.mine) sc[0][e] = -INFINITY;
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
    T::add(rv + at, T::G::TB, sc[0], o);
  }
  if (b.rows_left <= 0) return;
  l += other_half(l);
  const float f = l == 0.f ? 0.f : 1.f / l;
  const long n = s.q0 + b.me.i;
  if (a.shares > 1) {
    const long p = (long)b.share * a.q_rows * a.heads + n * a.heads + b.me.h;
    if ((lane & 31) < b.rows_left) {
      store_share<T::MB>(a.part, p, o, 0, a.dh, hh);
      if (hh == 0) {
        a.part_stats[2 * p] = m;
        a.part_stats[2 * p + 1] = l;
      }
    }
    return;
  }
  if ((lane & 31) < b.rows_left) {
    store_row(row_out<float>(a.o, n, b.me.h), o, f, a.dh, hh);
    if (hh == 0) a.lse[n * a.heads + b.me.h] = l == 0.f ? -INFINITY : m + log2f(l);
  }
  redo_rows(not_finite(o, f * 0.f), b.rows_left, [&](int j) {
    const RowPlace p = place_of(a, b.x.hk, b.w0 + j);
    one_forward<float>(a, s, p.i, p.h, lane);
  });
}

template <int W>
__global__ __launch_bounds__(64 * WAVES, W > 96 ? 1 : 2) void packed_dq_f32_kernel(PackedAttnArgs a) {
  typedef Tiles<W> T;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[2 * T::STAGE];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  RowBlock b;
  if (!b.find(a, wave, lane)) return;
  const Seq& s = b.x.s;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const PairStream<W> ps((unsigned)(a.k.row * 4), (unsigned)(a.v.row * 4), a.dh, lds0, wave, lane);
  const float* k = row_of<float>(a.k, s.k0, b.x.hk);
  const float* v = row_of<float>(a.v, s.k0, b.x.hk);
  if (b.from < b.to) ps.issue(k, v, 32 * b.from, s.nk, b.from & 1, lane);
  const long n = s.q0 + b.me.i;
  float q[4 * T::J], g[4 * T::J], D = 0.f;
  {
    float o[4 * T::J];
    T::own(row_of<float>(a.dout, n, b.me.h), a.dh, lane, g);
    T::own(row_of<float>(a.o, n, b.me.h), a.dh, lane, o);
#pragma unroll
    for (int i = 0; i < 4 * T::J; ++i) D = fmaf(g[i], o[i], D);
  }
  T::own(row_of<float>(a.q, n, b.me.h), a.dh, lane, q);
  D += other_half(D);
  float L = stat_of(a.lse[n * a.heads + b.me.h]);
  landed(L);
  if (hh == 0 && b.share == 0 && lane < b.rows_left) {
    a.dsum[n * a.heads + b.me.h] = -D;
    a.nlse[n * a.heads + b.me.h] = -L;
  }
  const unsigned ck = lds0 + T::cols_lane(lane), rk = lds0 + T::rows_lane(lane);
  const float c = a.scale * LOG2E;
  float16v dq[T::MB];
  zero_acc(dq);
  for (int i = b.from; i < b.to; ++i) {
    copies_in_flight<0>();
    workgroup_handover();
    if (i + 1 < b.to) ps.issue(k, v, 32 * (i + 1), s.nk, (i + 1) & 1, lane);
    if (32 * i >= b.most) continue;
    const unsigned at = (unsigned)(i & 1) * T::STAGE;
    float16v sc[1], dp;
    zero_acc(sc);
#pragma unroll
    for (int e = 0; e < 16; ++e) dp[e] = -D;
    sc[0] = T::product(ck + at, 0, q, sc[0]);
    dp = T::product(ck + at, T::G::TB, g, dp);
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[0][e] = fast_exp2(fmaf(sc[0][e], c, -L)) * dp[e];
    if (32 * i + 32 > b.fewest) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (32 * i + tile_row_of(e, hh) >= b.mine) sc[0][e] = 0.f;
    }
    T::add(rk + at, 0, sc[0], dq);
  }
  if (b.rows_left <= 0) return;
  if (a.shares > 1) {
    if ((lane & 31) < b.rows_left)
      store_share<T::MB>(a.part, (long)b.share * a.q_rows * a.heads + n * a.heads + b.me.h, dq, 0, a.dh, hh);
    return;
  }
  if ((lane & 31) < b.rows_left) store_row(row_out<float>(a.dq, n, b.me.h), dq, a.scale, a.dh, hh);
  redo_rows(not_finite(dq, 0.f), b.rows_left, [&](int j) {
    const RowPlace p = place_of(a, b.x.hk, b.w0 + j);
    one_dq<float>(a, s, p.i, p.h, row_dsum<float>(a, s.q0 + p.i, p.h, lane), lane);
  });
}

// Queries from the last tile down, all heads of the group for one tile before the next.
template <int W>
__global__ __launch_bounds__(64 * WAVES, W > 64 ? 1 : 2) void packed_dkdv_f32_kernel(PackedAttnArgs a) {
  typedef Tiles<W> T;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[2 * T::STAGE];
  __shared__ __attribute__((aligned(256))) float stats[2][2][64];                // [stage][-lse | -D][32 rows, and again]
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const Tile x = find_tile<true>(a, ROWS, lane);
  if (!x.exists) return;
  const Seq& s = x.s;
  const int k0 = ROWS * x.t, w0 = k0 + 32 * wave, keys_left = s.nk - w0;
  const int nq = s.nq, shift = s.nk - nq;
  auto first_query = [&](int key) __attribute__((always_inline)) {
    const int i = key - shift;
    return !a.causal || i < 0 ? 0 : i;
  };
  const int top = (nq - 1) >> 5;
  const int steps = nq > 0 ? (top + 1 - (first_query(k0) >> 5)) * a.group : 0, share = (int)blockIdx.y;
  const int from = (int)((long)steps * share / a.shares), to = (int)((long)steps * (share + 1) / a.shares);
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const unsigned lds1 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(stats));
  const PairStream<W> ps((unsigned)(a.q.row * 4), (unsigned)(a.dout.row * 4), a.dh, lds0, wave, lane);
  int ih = from % a.group, iq = top - from / a.group;      // the next tile to ask for
  auto ask = [&](int at) __attribute__((always_inline)) {
    const int h = x.hk * a.group + ih, first = 32 * iq;
    ps.issue(row_of<float>(a.q, s.q0, h), row_of<float>(a.dout, s.q0, h), first, nq, at, lane);
    const int r = first + (lane & 31) < nq ? first + (lane & 31) : nq - 1;
    copy4_to_lds((wave & 1 ? a.dsum : a.nlse) + (long)(s.q0 + r) * a.heads + h, lds1 + (unsigned)at * 512u + (unsigned)(wave & 1) * 256u);
    if (++ih == a.group) { ih = 0; --iq; }
  };
  const int key = keys_left > 0 ? w0 + ((lane & 31) < keys_left ? (lane & 31) : keys_left - 1) : s.nk - 1;
  float k[4 * T::J], v[4 * T::J];
  T::own(row_of<float>(a.k, s.k0 + key, x.hk), a.dh, lane, k);
  T::own(row_of<float>(a.v, s.k0 + key, x.hk), a.dh, lane, v);
  const unsigned cq = lds0 + T::cols_lane(lane), rq = lds0 + T::rows_lane(lane);
  const int mine = first_query(key);
  const int begin = keys_left > 0 ? first_query(w0) : nq, all = keys_left > 0 ? first_query(w0 + (keys_left < 32 ? keys_left : 32) - 1) : nq;
  const float c = a.scale * LOG2E;
  float16v dk[T::MB], dv[T::MB];
  zero_acc(dk);
  zero_acc(dv);
  int sh = ih, first = 32 * iq;
  if (from < to) ask(from & 1);
  for (int i = from; i < to; ++i) {
    copies_in_flight<0>();
    workgroup_handover();
    if (i + 1 < to) ask((i + 1) & 1);
    if (first + 32 > begin && keys_left > 0) {
      const unsigned at = (unsigned)(i & 1) * T::STAGE;
      float16v sc[1], dp;
      zero_acc(sc);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 u = *reinterpret_cast<const float4*>(&stats[i & 1][1][8 * g + 4 * hh]);
        dp[4 * g] = u.x; dp[4 * g + 1] = u.y; dp[4 * g + 2] = u.z; dp[4 * g + 3] = u.w;
      }
      sc[0] = T::product(cq + at, 0, k, sc[0]);
      dp = T::product(cq + at, T::G::TB, v, dp);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 u = *reinterpret_cast<const float4*>(&stats[i & 1][0][8 * g + 4 * hh]);
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
      T::add(rq + at, T::G::TB, sc[0], dv);
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[0][e] *= dp[e];
      T::add(rq + at, 0, sc[0], dk);
    }
    if (++sh == a.group) { sh = 0; first -= 32; }
  }
  if (keys_left <= 0) return;
  if (a.shares > 1) {
    const long r = (long)(s.k0 + key) * a.kv_heads + x.hk, rows = (long)a.k_rows * a.kv_heads;
    if ((lane & 31) < keys_left) {
      store_share<T::MB>(a.part, share * rows + r, dk, 0, a.dh, hh);
      store_share<T::MB>(a.part, (a.shares + share) * rows + r, dv, 0, a.dh, hh);
    }
    return;
  }
  if ((lane & 31) < keys_left) {
    store_row(row_out<float>(a.dk, s.k0 + key, x.hk), dk, a.scale, a.dh, hh);
    store_row(row_out<float>(a.dv, s.k0 + key, x.hk), dv, 1.f, a.dh, hh);
  }
  redo_rows(not_finite(dv, not_finite(dk, 0.f)), keys_left, [&](int j) { one_dkdv<float>(a, s, w0 + j, x.hk, lane); });
}

}  // namespace

hipError_t launch_packed_fwd_f32(const PackedAttnArgs& a, hipStream_t s) {
  const dim3 grid(tile_grid<false>(a, ROWS), a.shares);
  return with_width(a.dh, [&](auto w) {
    packed_fwd_f32_kernel<decltype(w)::value><<<grid, 64 * WAVES, 0, s>>>(a);
    return hipGetLastError();
  });
}
hipError_t launch_packed_dq_f32(const PackedAttnArgs& a, hipStream_t s) {
  const dim3 grid(tile_grid<false>(a, ROWS), a.shares);
  return with_width(a.dh, [&](auto w) {
    packed_dq_f32_kernel<decltype(w)::value><<<grid, 64 * WAVES, 0, s>>>(a);
    return hipGetLastError();
  });
}
hipError_t launch_packed_dkdv_f32(const PackedAttnArgs& a, hipStream_t s) {
  const dim3 grid(tile_grid<true>(a, ROWS), a.shares);
  return with_width(a.dh, [&](auto w) {
    packed_dkdv_f32_kernel<decltype(w)::value><<<grid, 64 * WAVES, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace hbp
