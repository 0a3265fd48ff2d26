// What the kernels of the attention over packed sequences share (attention_packed.hip, attention_packed_f32.hip): sequences, tiles of
// rows, and the term-by-term computation of one row or key.
//
// A key/value head's `group` query heads see the same keys, so the rows that a sequence brings to it are its queries
// times its group, row r = query r / group of head r % group: tiles of rows then hold several heads of a query, the
// streamed keys serve all of them, and a single query fills `group` rows of a tile.
#pragma once
#include "attention_device.h"

#include <cfloat>
#include <type_traits>

namespace hbp {

namespace {

// One sequence: its first row and its length on either side.
struct Seq { int q0, nq, k0, nk; };
__device__ __forceinline__ int clamp_row(int v, int rows) { return v < 0 ? 0 : v > rows ? rows : v; }
__device__ __forceinline__ void span_of(const int* off, int rows, int len, int s, int& first, int& n) {
  if (!off) {
    n = len;
    first = s * n;
    return;
  }
  first = clamp_row(off[s], rows);
  n = clamp_row(off[s + 1], rows) - first;
  if (n < 0) n = 0;
}
__device__ __forceinline__ Seq seq_of(const PackedAttnArgs& a, int s) {
  Seq q;
  span_of(a.q_off, a.q_rows, a.q_len, s, q.q0, q.nq);
  span_of(a.k_off, a.k_rows, a.k_len, s, q.k0, q.nk);
  return q;
}
// the sequence that row n belongs to (offsets that do not decrease), -1: none
__device__ __forceinline__ int seq_with(const int* off, int len, int seqs, int n) {
  if (!off) return n / len;
  int lo = 0, hi = seqs;                                   // off[lo] <= n < off[hi], where there is such a sequence
  if (n < off[0] || n >= off[seqs]) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= n) lo = mid; else hi = mid;
  }
  return lo;
}

template <typename T> __device__ __forceinline__ const T* row_of(const HeadRows& x, long n, int h) {
  return reinterpret_cast<const T*>(x.p) + n * x.row + (long)h * x.head;
}
template <typename T> __device__ __forceinline__ T* row_out(const HeadRows& x, long n, int h) {
  return reinterpret_cast<T*>(x.p) + n * x.row + (long)h * x.head;
}
template <typename T>
__device__ __forceinline__ float dot_rows(const T* a, const T* b, int n) {
  float s = 0.f;
  for (int c = 0; c < n; c += 8) {
    float x[8], y[8];
    load8(a + c, x);
    load8(b + c, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(x[i], y[i], s);
  }
  return s;
}

// out[c] += sum over n rows of w (lane j: row j) times column c of `rows`; a lane holds columns lane and lane + 64
struct TwoColumns {
  float v[2] = {0.f, 0.f};
  template <typename T>
  __device__ __forceinline__ void add(float w, int n, const T* rows, long ld, int dh, int lane) {
    for (int j = 0; j < n; ++j) {
      const float wj = __shfl(w, j, 64);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < dh) v[u] = fmaf(wj, Elem<T>::load(rows + j * ld + lane + 64 * u), v[u]);
    }
  }
  // channels c0 .. c1 - 1 of the row at `out`
  template <typename T>
  __device__ __forceinline__ void store(T* out, float f, int c0, int c1, int lane) const {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (lane + 64 * u >= c0 && lane + 64 * u < c1) Elem<T>::store(out + lane + 64 * u, v[u] * f);
  }
  // NaN throughout: nothing that is added changes that
  __device__ __forceinline__ bool settled(int dh, int lane) const {
    bool nan = true;
#pragma unroll
    for (int u = 0; u < 2; ++u) nan = nan && (lane + 64 * u >= dh || v[u] != v[u]);
    return __all(nan);
  }
};

// keys that query i of a sequence sees
__device__ __forceinline__ int seen_by(const Seq& s, int i, int causal) {
  if (!causal) return s.nk;
  const int n = i + 1 + s.nk - s.nq;
  return n < 0 ? 0 : n;
}

// ------------------------------------------------------------------------------------------------------------
// term by term: one wavefront per (query, head), one per (key, key head), which leaves channels c0 .. c1 - 1 (and the statistic with c0 = 0)
// ------------------------------------------------------------------------------------------------------------
// Rows with scores past 2^31 may come here as well: there the rounding of the running maximum, which the kernels' fused multiply-add does
// not share, may take every weight of a row to 0 (or infinity), and the row does not come out finite; where it does, its
// weights keep their ratios.  So no contraction here: the largest score less itself is 0.
template <typename T>
__device__ __forceinline__ void one_forward(const PackedAttnArgs& a, const Seq& s, int i, int h, int c0, int c1, int lane) {
#pragma clang fp contract(off)
  const int hk = h / a.group, seen = seen_by(s, i, a.causal);
  const T* q = row_of<T>(a.q, s.q0 + i, h);
  const T* k = row_of<T>(a.k, s.k0, hk);
  const T* v = row_of<T>(a.v, s.k0, hk);
  const float c = a.scale * LOG2E;
  float m = -INFINITY, sum = 0.f;
  for (int j = lane; j < seen; j += 64) {
    const float x = c * dot_rows(q, k + j * a.k.row, a.dh);
    m = x > m || x != x ? x : m;                           // (a NaN stays)
    if (m != m) break;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float x = __shfl_xor(m, o, 64);
    m = x > m || x != x ? x : m;
  }
  const float base = m == -INFINITY ? 0.f : m;             // nothing seen, or minus infinity throughout: every weight is 0
  TwoColumns out;
  for (int j0 = 0; j0 < seen; j0 += 64) {
    float p = 0.f;
    if (j0 + lane < seen) {
      p = exp2f(c * dot_rows(q, k + (j0 + lane) * a.k.row, a.dh) - base);
      sum += p;
    }
    out.add(p, seen - j0 < 64 ? seen - j0 : 64, v + j0 * a.v.row, a.v.row, a.dh, lane);
    if (m != m && out.settled(a.dh, lane)) break;
  }
  sum = wave_sum(sum);
  const bool none = m == -INFINITY;
  if (none) out = TwoColumns();
  out.store(row_out<T>(a.o, s.q0 + i, h), none ? 0.f : 1.f / sum, c0, c1, lane);
  if (lane == 0 && c0 == 0) a.lse[(long)(s.q0 + i) * a.heads + h] = none ? -INFINITY : m + log2f(sum);
}
// the statistic that the backward pass subtracts: a row that weighs nothing keeps weighing nothing
__device__ __forceinline__ float stat_of(float lse) { return lse == -INFINITY ? INFINITY : lse; }

template <typename T>
__device__ __forceinline__ float row_dsum(const PackedAttnArgs& a, long n, int h, int lane) {
  const T* g = row_of<T>(a.dout, n, h);
  const T* o = row_of<T>(a.o, n, h);
  float d = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (lane + 64 * u < a.dh) d = fmaf(Elem<T>::load(g + lane + 64 * u), Elem<T>::load(o + lane + 64 * u), d);
  return wave_sum(d);
}

template <typename T>
__device__ __forceinline__ void one_dq(const PackedAttnArgs& a, const Seq& s, int i, int h, float D, int c0, int c1, int lane) {
  const int hk = h / a.group, seen = seen_by(s, i, a.causal);
  const long n = s.q0 + i;
  const T* q = row_of<T>(a.q, n, h);
  const T* g = row_of<T>(a.dout, n, h);
  const T* k = row_of<T>(a.k, s.k0, hk);
  const T* v = row_of<T>(a.v, s.k0, hk);
  const float c = a.scale * LOG2E, L = stat_of(a.lse[n * a.heads + h]);
  TwoColumns out;
  if (L != INFINITY)
    for (int j0 = 0; j0 < seen; j0 += 64) {
      float ds = 0.f;
      if (j0 + lane < seen) {
        const float p = exp2f(c * dot_rows(q, k + (j0 + lane) * a.k.row, a.dh) - L);
        ds = p * (dot_rows(g, v + (j0 + lane) * a.v.row, a.dh) - D);
      }
      out.add(ds, seen - j0 < 64 ? seen - j0 : 64, k + j0 * a.k.row, a.k.row, a.dh, lane);
      if (out.settled(a.dh, lane)) break;
    }
  out.store(row_out<T>(a.dq, n, h), a.scale, c0, c1, lane);
}

constexpr int DK = 1, DV = 2;
template <typename T>
__device__ __forceinline__ void one_dkdv(const PackedAttnArgs& a, const Seq& s, int j, int hk, int which, int c0, int c1, int lane) {
  const T* k = row_of<T>(a.k, s.k0 + j, hk);
  const T* v = row_of<T>(a.v, s.k0 + j, hk);
  const float c = a.scale * LOG2E;
  int i0 = a.causal ? j - (s.nk - s.nq) : 0;               // the first query that sees it
  if (i0 < 0) i0 = 0;
  TwoColumns dk, dv;
  for (int h = hk * a.group; h < (hk + 1) * a.group && !(dk.settled(a.dh, lane) && dv.settled(a.dh, lane)); ++h)
    for (int b = i0; b < s.nq; b += 64) {
      if (dk.settled(a.dh, lane) && dv.settled(a.dh, lane)) break;
      float p = 0.f, ds = 0.f;
      const int n = s.nq - b < 64 ? s.nq - b : 64;
      if (lane < n) {
        const long r = s.q0 + b + lane;
        const float L = a.nlse[r * a.heads + h];
        if (L != -INFINITY) {
          p = exp2f(c * dot_rows(row_of<T>(a.q, r, h), k, a.dh) + L);
          ds = p * (dot_rows(row_of<T>(a.dout, r, h), v, a.dh) + a.dsum[r * a.heads + h]);
        }
      }
      dk.add(ds, n, row_of<T>(a.q, s.q0 + b, h), a.q.row, a.dh, lane);
      dv.add(p, n, row_of<T>(a.dout, s.q0 + b, h), a.dout.row, a.dh, lane);
    }
  if (which & DK) dk.store(row_out<T>(a.dk, s.k0 + j, hk), a.scale, c0, c1, lane);
  if (which & DV) dv.store(row_out<T>(a.dv, s.k0 + j, hk), 1.f, c0, c1, lane);
}

// Heads of up to W channels (32, 64, 96 or 128): tiles of 64 or 128 channels, of which products and results take W.
template <int W> constexpr int padded() { return W <= 64 ? 64 : 128; }
template <int W>
struct Fit : Geo<padded<W>()> {
  static constexpr int KK = W / 16, MB = W / 32;
};
// f(the smallest such W, as a constant)
template <typename F>
hipError_t with_width(int dh, F f) {
  if (dh <= 32) return f(std::integral_constant<int, 32>());
  if (dh <= 64) return f(std::integral_constant<int, 64>());
  if (dh <= 96) return f(std::integral_constant<int, 96>());
  return f(std::integral_constant<int, 128>());
}

// sum over the 64 lanes
__device__ __forceinline__ int wave_total(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);     // row_shr:1, 2, 4, 8: every row's sum in its last lane
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
  return __builtin_amdgcn_readlane(v, 15) + __builtin_amdgcn_readlane(v, 31) + __builtin_amdgcn_readlane(v, 47) +
         __builtin_amdgcn_readlane(v, 63);
}

// Which key head, sequence and tile of `per` rows (KEYS: keys) a workgroup takes.  A causal mask leaves the tiles of a sequence unequally
// long: the last tile of rows and the first tile of keys see the whole sequence, the others less and less.  Level u of a sequence
// is its u-th shortest tile; ids go from the highest level down, all sequences that have one, so that compute units which are
// done early take the shorter tiles (sequence after sequence, a compute unit of two rounds got two long or two short ones: dk, dv of 16
// sequences of 1024 at 4 key heads left 43 % of the compute units' time unused).  Key heads are next to each other: all problems go on
// side by side, and with eight of them, or a multiple, consecutive ids, which go to the eight XCDs in turn, keep a problem's
// streamed tiles in one XCD's L2.
// Past LEVELLED sequences the search for a level costs more than it gives (a memory latency for 64 of them), and there are workgroups
// enough: tile t of sequence s then has the id first row / per + s + t, whose first two terms grow with s by at least the
// sequence's tiles, and s is found 64 candidates at a time.  Levels / this, us, ragged: forward of 16384 sequences of 9, 4 heads of
// 64, 1945 / 193; backward of 4096 of 64, 12 heads, 2870 / 1375; forward of 200 of 1000, 8 heads, 487 / 454; the other way round
// backward of 100 of 1000, 8 heads, 1062 / 1107; forward of 24 of 700, 16 heads on 4, 55 / 66.
// A dimension of a grid holds fewer than 2^32 threads, and what is launched beyond is cut off without an error: x has at most 2^22 workgroups
// (of 512 threads or fewer), more of them go on in z.  The last ones there may have no tile.
constexpr int GRID_X_LOG = 22;
__device__ __forceinline__ unsigned workgroup_id() { return (blockIdx.z << GRID_X_LOG) + blockIdx.x; }
inline dim3 grid_of(unsigned workgroups, int shares = 1) {
  const unsigned most = 1u << GRID_X_LOG, x = workgroups < most ? workgroups : most;
  return dim3(x, (unsigned)shares, (workgroups + most - 1) / most);
}
struct Tile { int hk, t; Seq s; bool exists; };
constexpr int LEVELLED = 128;
__device__ __forceinline__ int tiles_in(int len, int per) { return (int)((unsigned)(len + per - 1) / (unsigned)per); }   // (per: a power of two)
template <bool KEYS>
__device__ __forceinline__ Tile find_tile(const PackedAttnArgs& a, int per, int lane, unsigned id = workgroup_id()) {
  Tile x;
  int j = (int)a.by_kv.quotient(id);
  x.hk = (int)id - j * a.kv_heads;
  const int* off = KEYS ? a.k_off : a.q_off;
  const int mult = KEYS ? 1 : a.group, rows = KEYS ? a.k_rows : a.q_rows;
  int sq = -1, n = 0, level = 0;
  if (!off) {
    n = tiles_in((KEYS ? a.k_len : a.q_len) * mult, per);
    const int down = (int)a.by_seqs.quotient((unsigned)j);
    sq = j - down * a.seqs;
    level = n - down;
    if (level <= 0) sq = -1;
  } else if (a.seqs > LEVELLED) {
    int lo = 0, hi = a.seqs, base = 0;                     // base of lo <= j < base of hi, where there is such a sequence
    bool found = true;
    do {
      const int by = (hi - lo + 63) >> 6, at = lo + lane * by;
      const int b = at < hi ? (int)((unsigned)(clamp_row(off[at], rows) * mult) / (unsigned)per) + at : j + 1;
      const unsigned long long le = __ballot(b <= j);
      found = le != 0;
      if (!found) break;
      const int l = 63 - __clzll(le);
      base = __builtin_amdgcn_readlane(b, l);
      lo += l * by;
      hi = hi < lo + by ? hi : lo + by;
    } while (hi - lo > 1);
    if (found) {
      int first;
      span_of(off, rows, 0, lo, first, n);
      n = __builtin_amdgcn_readfirstlane(tiles_in(n * mult, per));
      const int t = j - base;
      if (t < n) {
        sq = lo;
        level = KEYS ? n - t : t + 1;
      }
    }
  } else {
    for (int s0 = 0; s0 < a.seqs; s0 += 64) {              // 64 sequences at a time, one per lane
      int first, m = 0;
      if (s0 + lane < a.seqs) span_of(off, rows, 0, s0 + lane, first, m);
      m = tiles_in(m * mult, per);
      const int all = wave_total(m);
      if (j >= all) {
        j -= all;
        continue;
      }
      // tiles of level u and above: sum of max(0, m - u + 1); the level of tile j is the highest u with more than j of them
      int lo = 1, hi = tiles_in(rows * mult, per);         // (no sequence has more)
      while (lo < hi) {
        const int u = lo + (hi - lo + 1) / 2;
        if (wave_total(m >= u ? m - u + 1 : 0) > j) lo = u;
        else hi = u - 1;
      }
      level = lo;
      const int rank = j - wave_total(m >= level + 1 ? m - level : 0);
      const unsigned long long has = __ballot(m >= level);
      const int before = __popcll(has & ((1ull << lane) - 1ull));
      const unsigned long long here = __ballot(m >= level && before == rank);
      if (here) {                                          // (offsets that do not decrease: always)
        const int l = __ffsll(here) - 1;
        sq = s0 + l;
        n = __builtin_amdgcn_readlane(m, l);
      }
      break;
    }
  }
  x.exists = sq >= 0;
  if (x.exists) {
    x.s = seq_of(a, sq);
    x.t = __builtin_amdgcn_readfirstlane(KEYS ? n - level : level - 1);
    x.s.q0 = __builtin_amdgcn_readfirstlane(x.s.q0);
    x.s.nq = __builtin_amdgcn_readfirstlane(x.s.nq);
    x.s.k0 = __builtin_amdgcn_readfirstlane(x.s.k0);
    x.s.nk = __builtin_amdgcn_readfirstlane(x.s.nk);
  }
  return x;
}
// the other half's value (lanes l and l + 32 hold one row's two halves), and the larger of the two
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }
__device__ __forceinline__ float max_of_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The rows of a tile: row r of the sequence at this key head is query r / group of head hk group + r % group.
struct RowPlace { int i, h; };
__device__ __forceinline__ RowPlace place_of(const PackedAttnArgs& a, int hk, int r) {
  RowPlace p;
  p.i = (int)a.by_group.quotient((unsigned)r);
  p.h = hk * a.group + (r - p.i * a.group);
  return p;
}

// Infinities and NaNs: a product on the matrix cores meets every element of a tile, also those that the mask or the sequence's end
// leaves out, and there 0 times an infinity is NaN.  A row of a result that did not come out finite is therefore computed
// once more, term by term over what it sees
// (wavefronts that hold blocks of 32 channels of a row each store, and compute once more, their own).
template <int MB>
__device__ __forceinline__ float not_finite(const float16v (&acc)[MB], float t) {
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) t = fmaf(acc[m][r], 0.f, t);
  return t;
}
// 1 / a row's sum of weights relative to its maximum m; 0 where it sees nothing.  (A sum of 0 with a maximum: infinity, which not_finite finds.)
__device__ __forceinline__ float inverse_sum(float m, float sum) { return sum == 0.f && m == -FLT_MAX ? 0.f : 1.f / sum; }
template <typename F>
__device__ __forceinline__ void redo_rows(float t, int rows_left, F f) {
  const unsigned long long b = __ballot(t != t);
  unsigned rows = (unsigned)b | (unsigned)(b >> 32);
  if (rows_left < 32) rows &= (1u << rows_left) - 1u;
  if (rows == 0) return;
  copies_in_flight<0>();                                   // (the tile's own stores, which these replace)
  for (; rows != 0; rows &= rows - 1) f(__ffs((int)rows) - 1);
}

// workgroups for tiles of `per` rows (keys), of which there are some
template <bool KEYS>
unsigned tile_grid(const PackedAttnArgs& a, int per) {
  const long rows = KEYS ? a.k_rows : (long)a.q_rows * a.group;
  const bool equal = KEYS ? !a.k_off : !a.q_off;
  const long each = (rows / a.seqs + per - 1) / per, tiles = equal ? a.seqs * each : rows / per + a.seqs;
  return (unsigned)(tiles * a.kv_heads);
}

// ------------------------------------------------------------------------------------------------------------
// shares: a workgroup that took part of the other side's steps leaves its sums in fp32, [share][row][dh]; a wavefront per row joins them
// ------------------------------------------------------------------------------------------------------------
constexpr int MOST_SHARES = 256;
template <int MB>
__device__ __forceinline__ void store_share(float* part, long row, const float16v (&acc)[MB], int m0, int dh, int hh) {
  float* p = part + row * dh;
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * (m0 + m) + 8 * g + 4 * hh;
      if (c < dh) *reinterpret_cast<float4*>(p + c) = make_float4(acc[m][4 * g], acc[m][4 * g + 1], acc[m][4 * g + 2], acc[m][4 * g + 3]);
    }
}
__device__ __forceinline__ void store2(float* p, float a, float b) { *reinterpret_cast<float2*>(p) = make_float2(a, b); }
__device__ __forceinline__ void store2(bf16_t* p, float a, float b) { *reinterpret_cast<unsigned*>(p) = pack_bf16x2(a, b); }
__device__ __forceinline__ bool all_finite(float a, float b) { return !__any(!(fabsf(a) < INFINITY && fabsf(b) < INFINITY)); }
// channels 2 lane, 2 lane + 1 of `shares` shares of a row, `stride` floats apart, each times f(share): eight at a time in flight
template <typename F>
__device__ __forceinline__ float2 sum_shares(const float* p, long stride, int shares, int dh, int lane, F f) {
  float2 v = make_float2(0.f, 0.f);
  const float* q = p + (2 * lane < dh ? 2 * lane : 0);
  for (int i = 0; i < shares; i += 8) {
    float2 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = *reinterpret_cast<const float2*>(q + (i + u < shares ? i + u : shares - 1) * stride);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float w = i + u < shares ? f(i + u) : 0.f;
      v.x = i + u < shares ? fmaf(w, x[u].x, v.x) : v.x;
      v.y = i + u < shares ? fmaf(w, x[u].y, v.y) : v.y;
    }
  }
  return v;
}
// The (query, head) of a wavefront and its sequence; false: it is in none.
__device__ __forceinline__ bool joined_row(const PackedAttnArgs& a, long r, Seq& s, int& n, int& h) {
  if (r >= (long)a.q_rows * a.heads) return false;
  n = (int)(r / a.heads);
  h = (int)(r - (long)n * a.heads);
  const int sq = seq_with(a.q_off, a.q_len, a.seqs, n);
  if (sq < 0) return false;
  s = seq_of(a, sq);
  return n >= s.q0 && n < s.q0 + s.nq;
}
template <typename T>
__global__ __launch_bounds__(256) void packed_join_fwd_kernel(PackedAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6), rows = (long)a.q_rows * a.heads;
  Seq s;
  int n, h;
  if (!joined_row(a, r, s, n, h)) return;
  // (a lane holds the factor of every 64th share, at most MOST_SHARES / 64 of them)
  float top = -FLT_MAX, sum = 0.f, f[MOST_SHARES / 64];
#pragma unroll
  for (int u = 0; u < MOST_SHARES / 64; ++u) {
    const int i = lane + 64 * u;
    f[u] = i < a.shares ? a.part_stats[(i * rows + r) * 2] : -FLT_MAX;
    top = fmaxf(top, f[u]);
  }
  top = wave_max(top);
#pragma unroll
  for (int u = 0; u < MOST_SHARES / 64; ++u) {
    const int i = lane + 64 * u;
    f[u] = fast_exp2(f[u] - top);
    if (i < a.shares) sum = fmaf(f[u], a.part_stats[(i * rows + r) * 2 + 1], sum);
  }
  sum = wave_sum(sum);
  const int c = 2 * lane;
  float2 w = make_float2(0.f, 0.f);
#pragma unroll
  for (int u = 0; u < MOST_SHARES / 64; ++u) {
    const int n64 = a.shares - 64 * u < 64 ? a.shares - 64 * u : 64;
    if (n64 <= 0) break;
    const float2 x = sum_shares(a.part + (64 * u * rows + r) * a.dh, rows * a.dh, n64, a.dh, lane,
                                [&](int i) __attribute__((always_inline)) { return __shfl(f[u], i, 64); });
    w.x += x.x;
    w.y += x.y;
  }
  const float v[2] = {w.x, w.y};
  const float g = inverse_sum(top, sum);
  if (!all_finite(v[0] * g, v[1] * g)) {                   // (see redo_rows)
    one_forward<T>(a, s, n - s.q0, h, 0, a.dh, lane);
    return;
  }
  if (c < a.dh) store2(row_out<T>(a.o, n, h) + c, v[0] * g, v[1] * g);
  if (lane == 0) a.lse[r] = sum == 0.f ? -INFINITY : top + log2f(sum);
}
template <typename T>
__global__ __launch_bounds__(256) void packed_join_dq_kernel(PackedAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6), rows = (long)a.q_rows * a.heads;
  Seq s;
  int n, h;
  if (!joined_row(a, r, s, n, h)) return;
  const auto one = [](int) { return 1.f; };
  const float2 v = sum_shares(a.part + r * a.dh, rows * a.dh, a.shares, a.dh, lane, one);
  if (!all_finite(v.x, v.y)) {
    one_dq<T>(a, s, n - s.q0, h, -a.dsum[r], 0, a.dh, lane);
    return;
  }
  if (2 * lane < a.dh) store2(row_out<T>(a.dq, n, h) + 2 * lane, v.x * a.scale, v.y * a.scale);
}
template <typename T>
__global__ __launch_bounds__(256) void packed_join_dkdv_kernel(PackedAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6), rows = (long)a.k_rows * a.kv_heads;
  if (r >= rows) return;
  const int n = (int)(r / a.kv_heads), hk = (int)(r - (long)n * a.kv_heads);
  const int sq = seq_with(a.k_off, a.k_len, a.seqs, n);
  if (sq < 0) return;
  const Seq s = seq_of(a, sq);
  if (n < s.k0 || n >= s.k0 + s.nk) return;
  const auto one = [](int) { return 1.f; };
  const float2 k = sum_shares(a.part + r * a.dh, rows * a.dh, a.shares, a.dh, lane, one);
  const float2 v = sum_shares(a.part + (a.shares * rows + r) * a.dh, rows * a.dh, a.shares, a.dh, lane, one);
  if (!all_finite(k.x + k.y, v.x + v.y)) {
    one_dkdv<T>(a, s, n - s.k0, hk, DK | DV, 0, a.dh, lane);
    return;
  }
  if (2 * lane < a.dh) {
    store2(row_out<T>(a.dk, n, hk) + 2 * lane, k.x * a.scale, k.y * a.scale);
    store2(row_out<T>(a.dv, n, hk) + 2 * lane, v.x, v.y);
  }
}

constexpr unsigned CUS = 256;
// Rows (keys) of a workgroup, `wide` or fewer of them with the other side's tiles shared out between its wavefronts: wide where that makes
// `least` workgroups (counted as with offsets, of which the workspace's size knows nothing) and where sequences have more rows than
// the narrow form takes at a time.
template <bool KEYS>
bool wide_blocks(const PackedAttnArgs& a, int wide, int narrow, long least) {
  const long rows = KEYS ? (long)a.k_rows : (long)a.q_rows * a.group;
  return (rows / wide + a.seqs) * a.kv_heads >= least && rows / a.seqs > narrow;
}
template <bool KEYS> bool f32_wide(const PackedAttnArgs& a) { return wide_blocks<KEYS>(a, 128, 32, CUS / 2); }

}  // namespace

hipError_t launch_packed_fwd_f32(const PackedAttnArgs& a, hipStream_t s);
hipError_t launch_packed_dq_f32(const PackedAttnArgs& a, hipStream_t s);
hipError_t launch_packed_dkdv_f32(const PackedAttnArgs& a, hipStream_t s);

}  // namespace hbp
