// Attention over packed sequences, forward and backward, whose key/value heads serve groups of query heads.
//
// A key/value head's `group` query heads see the same keys, so the rows that a sequence brings to it are its queries
// times its group, row r = query r / group of head r % group: tiles of rows then hold several heads of a query, the
// streamed keys serve all of them, dk and dv sum over the group by summing over rows, and a single query fills `group`
// rows of a tile.
#include "attention_device.h"

#include <cfloat>

namespace hbp {

namespace {

// One sequence: its first row and its length on either side.
struct Seq { int q0, nq, k0, nk; };
__device__ __forceinline__ int clamp_row(int v, int rows) { return v < 0 ? 0 : v > rows ? rows : v; }
__device__ __forceinline__ void span_of(const int* off, int rows, int seqs, int s, int& first, int& n) {
  if (!off) {
    n = rows / seqs;
    first = s * n;
    return;
  }
  first = clamp_row(off[s], rows);
  n = clamp_row(off[s + 1], rows) - first;
  if (n < 0) n = 0;
}
__device__ __forceinline__ Seq seq_of(const PackedAttnArgs& a, int s) {
  Seq q;
  span_of(a.q_off, a.q_rows, a.seqs, s, q.q0, q.nq);
  span_of(a.k_off, a.k_rows, a.seqs, s, q.k0, q.nk);
  return q;
}
// the sequence that row n belongs to (offsets that do not decrease), -1: none
__device__ __forceinline__ int seq_with(const int* off, int rows, int seqs, int n) {
  if (!off) return n / (rows / seqs);
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
  template <typename T>
  __device__ __forceinline__ void store(T* out, float f, int dh, int lane) const {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (lane + 64 * u < dh) Elem<T>::store(out + lane + 64 * u, v[u] * f);
  }
};

// keys that query i of a sequence sees
__device__ __forceinline__ int seen_by(const Seq& s, int i, int causal) {
  if (!causal) return s.nk;
  const int n = i + 1 + s.nk - s.nq;
  return n < 0 ? 0 : n;
}

// ------------------------------------------------------------------------------------------------------------
// term by term: one wavefront per (query, head), one per (key, key head)
// ------------------------------------------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void one_forward(const PackedAttnArgs& a, const Seq& s, int i, int h, int lane) {
  const int hk = h / a.group, seen = seen_by(s, i, a.causal);
  const T* q = row_of<T>(a.q, s.q0 + i, h);
  const T* k = row_of<T>(a.k, s.k0, hk);
  const T* v = row_of<T>(a.v, s.k0, hk);
  const float c = a.scale * LOG2E;
  float m = -INFINITY, sum = 0.f;
  for (int j = lane; j < seen; j += 64) {
    const float x = c * dot_rows(q, k + j * a.k.row, a.dh);
    m = x > m || x != x ? x : m;                           // (a NaN stays)
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
  }
  sum = wave_sum(sum);
  const bool none = m == -INFINITY;
  if (none) out = TwoColumns();
  out.store(row_out<T>(a.o, s.q0 + i, h), none ? 0.f : 1.f / sum, a.dh, lane);
  if (lane == 0) a.lse[(long)(s.q0 + i) * a.heads + h] = none ? -INFINITY : m + log2f(sum);
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
__device__ __forceinline__ void one_dq(const PackedAttnArgs& a, const Seq& s, int i, int h, float D, int lane) {
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
    }
  out.store(row_out<T>(a.dq, n, h), a.scale, a.dh, lane);
}

template <typename T>
__device__ __forceinline__ void one_dkdv(const PackedAttnArgs& a, const Seq& s, int j, int hk, int lane) {
  const T* k = row_of<T>(a.k, s.k0 + j, hk);
  const T* v = row_of<T>(a.v, s.k0 + j, hk);
  const float c = a.scale * LOG2E;
  int i0 = a.causal ? j - (s.nk - s.nq) : 0;               // the first query that sees it
  if (i0 < 0) i0 = 0;
  TwoColumns dk, dv;
  for (int h = hk * a.group; h < (hk + 1) * a.group; ++h)
    for (int b = i0; b < s.nq; b += 64) {
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
  dk.store(row_out<T>(a.dk, s.k0 + j, hk), a.scale, a.dh, lane);
  dv.store(row_out<T>(a.dv, s.k0 + j, hk), 1.f, a.dh, lane);
}

template <typename T>
__global__ __launch_bounds__(64) void packed_fwd_rows_kernel(PackedAttnArgs a) {
  const int n = (int)(blockIdx.x / (unsigned)a.heads), h = (int)(blockIdx.x % (unsigned)a.heads);
  const int sq = seq_with(a.q_off, a.q_rows, a.seqs, n);
  if (sq < 0) return;
  const Seq s = seq_of(a, sq);
  if (n < s.q0 || n >= s.q0 + s.nq) return;                // (offsets that decrease)
  one_forward<T>(a, s, n - s.q0, h, threadIdx.x);
}
template <typename T>
__global__ __launch_bounds__(64) void packed_dq_rows_kernel(PackedAttnArgs a) {
  const int n = (int)(blockIdx.x / (unsigned)a.heads), h = (int)(blockIdx.x % (unsigned)a.heads);
  const int sq = seq_with(a.q_off, a.q_rows, a.seqs, n);
  if (sq < 0) return;
  const Seq s = seq_of(a, sq);
  if (n < s.q0 || n >= s.q0 + s.nq) return;
  const float D = row_dsum<T>(a, n, h, threadIdx.x);
  if (threadIdx.x == 0) {
    a.dsum[(long)n * a.heads + h] = -D;
    a.nlse[(long)n * a.heads + h] = -stat_of(a.lse[(long)n * a.heads + h]);
  }
  one_dq<T>(a, s, n - s.q0, h, D, threadIdx.x);
}
template <typename T>
__global__ __launch_bounds__(64) void packed_dkdv_rows_kernel(PackedAttnArgs a) {
  const int n = (int)(blockIdx.x / (unsigned)a.kv_heads), hk = (int)(blockIdx.x % (unsigned)a.kv_heads);
  const int sq = seq_with(a.k_off, a.k_rows, a.seqs, n);
  if (sq < 0) return;
  const Seq s = seq_of(a, sq);
  if (n < s.k0 || n >= s.k0 + s.nk) return;
  one_dkdv<T>(a, s, n - s.k0, hk, threadIdx.x);
}

// ------------------------------------------------------------------------------------------------------------
// matrix-core kernels: bf16
// ------------------------------------------------------------------------------------------------------------
// Which key head, sequence and tile of `per` rows (keys: `per` keys) a workgroup takes.  The key heads of a tile are next to each
// other: all problems go on side by side, and with eight of them, or a multiple, consecutive ids, which go to the eight XCDs
// in turn, keep a problem's streamed tiles in one XCD's L2.
struct Tile { int hk, t, n; Seq s; bool exists; };          // t of the sequence's n tiles
__device__ __forceinline__ int tiles_in(int len, int per) { return (len + per - 1) / per; }
template <bool KEYS>
__device__ __forceinline__ Tile find_tile(const PackedAttnArgs& a, int per, int lane) {
  Tile x;
  const unsigned id = blockIdx.x;
  x.hk = (int)(id % (unsigned)a.kv_heads);
  x.t = (int)(id / (unsigned)a.kv_heads);
  const int* off = KEYS ? a.k_off : a.q_off;
  const int mult = KEYS ? 1 : a.group, rows = KEYS ? a.k_rows : a.q_rows;
  int sq = -1;
  if (!off) {
    x.n = tiles_in(rows / a.seqs * mult, per);
    sq = x.t / x.n;
    x.t -= sq * x.n;
    if (sq >= a.seqs) sq = -1;
  } else {
    for (int s0 = 0; s0 < a.seqs; s0 += 64) {              // 64 sequences at a time: a running sum of their tiles over the lanes
      int first, n = 0;
      if (s0 + lane < a.seqs) span_of(off, rows, a.seqs, s0 + lane, first, n);
      n = tiles_in(n * mult, per);
      int sum = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(sum, o, 64);
        if (lane >= o) sum += up;
      }
      const unsigned long long past = __ballot(sum > x.t);
      if (past) {
        const int l = __ffsll(past) - 1;
        sq = s0 + l;
        x.n = __builtin_amdgcn_readlane(n, l);
        x.t -= __builtin_amdgcn_readlane(sum, l) - x.n;
        break;
      }
      x.t -= __builtin_amdgcn_readlane(sum, 63);
    }
  }
  x.exists = sq >= 0;
  if (x.exists) {
    x.s = seq_of(a, sq);
    x.t = __builtin_amdgcn_readfirstlane(x.t);
    x.n = __builtin_amdgcn_readfirstlane(x.n);
    x.s.q0 = __builtin_amdgcn_readfirstlane(x.s.q0);
    x.s.nq = __builtin_amdgcn_readfirstlane(x.s.nq);
    x.s.k0 = __builtin_amdgcn_readfirstlane(x.s.k0);
    x.s.nk = __builtin_amdgcn_readfirstlane(x.s.nk);
  }
  return x;
}
// the other half's value (lanes l and l + 32 hold one row's two halves)
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

// Fragments by LDS byte addresses.  The tiles' chunk swizzle is an XOR of address bits, so one register per direction holds all there
// is of a lane in an address: a step adds its stage, an XOR with a constant picks the fragment, and tiles of the same stage
// are constant offsets.  (Addresses formed from the row and the chunk each time cost an addition per read, a third of
// the forward pass's vector instructions.)
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

// Streamed key and value tiles: a stage holds 64 keys, two tiles of 32 of k and two of v, which a workgroup's wavefronts copy together,
// PW copies of 1 KB each.
template <int DHP, int WAVES>
struct KeyStream {
  typedef Geo<DHP> G;
  static constexpr int STAGE = 4 * G::TB;
  static constexpr int PW = 4 * G::COPIES / WAVES;
  unsigned off[PW];
  const unsigned char *k, *v;
  unsigned ldk, ldv, lds0;
  int nk, dh8;
  static __device__ __forceinline__ int tile(int w, int i) { return (w * PW + i) / G::COPIES; }     // k, k, v, v
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
    for (int i = 0; i < PW; ++i) off[i] = copy_offset<DHP>(tile(w, i) < 2 ? ldk : ldv, part(w, i), 32, dh8, lane);
  }
  // keys 64 step .. into stage `at`; keys past the last repeat it
  __device__ __forceinline__ void issue(int step, int at, int w, int lane) const {
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int t = tile(w, i), first = 64 * step + 32 * (t & 1);
      const unsigned ld = t < 2 ? ldk : ldv;
      const unsigned char* base = t < 2 ? k : v;
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

// The rows of a tile: row r of the sequence at this key head is query r / group of head hk group + r % group.
struct RowPlace { int i, h; };
__device__ __forceinline__ RowPlace place_of(const PackedAttnArgs& a, int hk, int r) {
  RowPlace p;
  p.i = (int)((unsigned)r / (unsigned)a.group);
  p.h = hk * a.group + (r - p.i * a.group);
  return p;
}

// A tile's results, scaled per row by f, to their rows (see store_tile in attention.hip: 64 bytes of a row per store).
// row(j): where row j of the tile goes; rows_left of them.
template <int MB, typename F>
__device__ __forceinline__ void store_rows(F row, int rows_left, const float16v (&acc)[MB], float f, int dh, unsigned char* stg, int lane) {
  const int r = lane & 31, hh = lane >> 5, rr = lane >> 2, ch = lane & 3;
  bf16_t* out[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) out[u] = rr + 16 * u < rows_left ? row(rr + 16 * u) : nullptr;
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    if (32 * m >= dh) break;
#pragma unroll
    for (int g = 0; g < 4; ++g)
      store4b(reinterpret_cast<bf16_t*>(stg + r * 64 + ((g ^ ((r >> 2) & 3)) << 4) + 8 * hh), acc[m][4 * g] * f,
              acc[m][4 * g + 1] * f, acc[m][4 * g + 2] * f, acc[m][4 * g + 3] * f);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int w = rr + 16 * u;
      const uint4 v = *reinterpret_cast<const uint4*>(stg + w * 64 + ((ch ^ ((w >> 2) & 3)) << 4));
      if (out[u] && 32 * m + 8 * ch < dh) *reinterpret_cast<uint4*>(out[u] + 32 * m + 8 * ch) = v;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Infinities and NaNs: a product on the matrix cores meets every element of a tile, also those that the mask or the sequence's end
// leaves out, and there 0 times an infinity is NaN.  A row of a result that did not come out finite is therefore computed
// once more, term by term over what it sees.  Finite data never comes here.
template <int MB>
__device__ __forceinline__ float not_finite(const float16v (&acc)[MB], float t) {
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) t = fmaf(acc[m][r], 0.f, t);
  return t;
}
template <typename F>
__device__ __forceinline__ void redo_rows(float t, int rows_left, F f) {
  const unsigned long long b = __ballot(t != t);
  unsigned rows = (unsigned)b | (unsigned)(b >> 32);
  if (rows_left < 32) rows &= (1u << rows_left) - 1u;
  if (rows == 0) return;
  copies_in_flight<0>();                                   // (the tile's own stores, which these replace)
  for (; rows != 0; rows &= rows - 1) f(__ffs((int)rows) - 1);
}

constexpr int FWD_WAVES = 8;
template <int DHP> constexpr int key_stages() { return DHP == 128 ? 3 : 4; }

// Forward.  A workgroup of eight wavefronts owns 256 rows, a wavefront 32 of them: a lane holds one row of q and half of that row's
// scores, so the running maximum and sum are scalars of the lane; the scores leave the first product in the places from which the
// second takes them.  Keys and values come in steps of 64 through a ring of stages.  The maximum that the exponents are taken
// from moves only when a row's has grown by more than a factor of 2^8 (probabilities then reach 2^8, sums 2^8 times the keys:
// far inside fp32, and bf16 rounds relatively), so the output is rarely rescaled.
template <int DHP>
__global__ __launch_bounds__(64 * FWD_WAVES, 2) void packed_fwd_mfma_kernel(PackedAttnArgs a) {
  typedef Geo<DHP> G;
  typedef KeyStream<DHP, FWD_WAVES> KS;
  constexpr int NST = key_stages<DHP>();
  __shared__ __attribute__((aligned(1024))) unsigned char ring[NST * KS::STAGE];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  Tile x = find_tile<false>(a, 32 * FWD_WAVES, lane);
  if (!x.exists) return;
  x.t = x.n - 1 - x.t;                                     // (causal: long rows first)
  const int R = x.s.nq * a.group, r0 = 32 * FWD_WAVES * x.t, w0 = r0 + 32 * wave;
  const int rows_left = R - w0;                            // of this wavefront's 32; none: it only copies
  const int dh8 = a.dh >> 3;
  auto seen = [&](int r) __attribute__((always_inline)) { return seen_by(x.s, place_of(a, x.hk, r).i, a.causal); };
  const int last = (R < r0 + 32 * FWD_WAVES ? R : r0 + 32 * FWD_WAVES) - 1;
  const int steps = (seen(last) + 63) >> 6;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const KS ks(a, x.s, x.hk, lds0, dh8, wave, lane);
  for (int i = 0; i < NST - 1 && i < steps; ++i) ks.issue(i, i, wave, lane);
  const int r = rows_left > 0 ? w0 + ((lane & 31) < rows_left ? (lane & 31) : rows_left - 1) : R - 1;
  const RowPlace me = place_of(a, x.hk, r);
  const bf16_t* qrow = row_of<bf16_t>(a.q, x.s.q0 + me.i, me.h);
  bf16x8 fq[G::KK];
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) fq[kk] = own_piece(qrow, kk, dh8, lane);
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) landed(fq[kk]);
  const int mine = seen_by(x.s, me.i, a.causal);           // keys that this lane's row sees
  const int fewest = rows_left > 0 ? seen(w0) : 0, most = rows_left > 0 ? seen(w0 + (rows_left < 32 ? rows_left : 32) - 1) : 0;
  const float c = a.scale * LOG2E;
  const unsigned ck = lds0 + Frags<DHP>::cols_lane(lane), rv = lds0 + Frags<DHP>::rows_lane(lane);
  float16v o[G::MB];
  zero_acc(o);
  float m = -FLT_MAX, l = 0.f;                             // m: in units of the exponent; l: this half's sum
  auto step = [&](int i, int at, bool masked) __attribute__((always_inline)) {
    const unsigned tk = ck + (unsigned)at * KS::STAGE, tv = rv + (unsigned)at * KS::STAGE;
    float16v s[2];
    zero_acc(s);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) s[b] = mfma(Frags<DHP>::cols(tk, b * G::TB, kk), fq[kk], s[b]);
    if (masked) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (64 * i + 32 * b + tile_row_of(e, hh) >= mine) s[b][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int e = 1; e < 32; ++e) top = fmaxf(top, s[e >> 4][e & 15]);
    top = fmaxf(top, other_half(top)) * c;
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
    for (int b = 0; b < 2; ++b) {
      float p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = fast_exp2(fmaf(s[b][e], c, -m));
        l += p[e];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16x8 pt = pack8(p + 8 * t);                // rounded to bf16: the matrix cores' operand
#pragma unroll
        for (int mb = 0; mb < G::MB; ++mb) o[mb] = mfma(Frags<DHP>::rows(tv, (2 + b) * G::TB, mb, t), pt, o[mb]);
      }
    }
  };
  int at = 0;
  for (int i = 0; i < steps; ++i) {
    if (i + NST - 2 < steps) copies_in_flight<KS::PW * (NST - 2)>();
    else copies_in_flight<0>();
    workgroup_handover();
    if (i + NST - 1 < steps) ks.issue(i + NST - 1, at == 0 ? NST - 1 : at - 1, wave, lane);
    if (64 * i < most) step(i, at, 64 * i + 64 > fewest);
    at = at == NST - 1 ? 0 : at + 1;
  }
  __syncthreads();                                         // the ring is free: results leave through it
  if (rows_left <= 0) return;
  l += other_half(l);
  const float f = l == 0.f ? 0.f : 1.f / l;
  store_rows([&](int j) __attribute__((always_inline)) {
    const RowPlace q = place_of(a, x.hk, w0 + j);
    return row_out<bf16_t>(a.o, x.s.q0 + q.i, q.h);
  }, rows_left, o, f, a.dh, ring + wave * 2048, lane);
  if (lane < 32 && lane < rows_left) a.lse[(long)(x.s.q0 + me.i) * a.heads + me.h] = l == 0.f ? -INFINITY : m + log2f(l);
  redo_rows(not_finite(o, f * 0.f), rows_left, [&](int j) {
    const RowPlace q = place_of(a, x.hk, w0 + j);
    one_forward<bf16_t>(a, x.s, q.i, q.h, lane);
  });
}

// dq, and minus D = sum_c dout (.) o of every row for the other kernel.  As the forward pass: a lane holds a row of q and of dout,
// dS leaves the first two products in the places from which the third takes it.
template <int DHP>
__global__ __launch_bounds__(64 * FWD_WAVES, 2) void packed_dq_mfma_kernel(PackedAttnArgs a) {
  typedef Geo<DHP> G;
  typedef KeyStream<DHP, FWD_WAVES> KS;
  constexpr int NST = key_stages<DHP>();
  __shared__ __attribute__((aligned(1024))) unsigned char ring[NST * KS::STAGE];
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  Tile x = find_tile<false>(a, 32 * FWD_WAVES, lane);
  if (!x.exists) return;
  x.t = x.n - 1 - x.t;
  const int R = x.s.nq * a.group, r0 = 32 * FWD_WAVES * x.t, w0 = r0 + 32 * wave;
  const int rows_left = R - w0;
  const int dh8 = a.dh >> 3;
  auto seen = [&](int r) __attribute__((always_inline)) { return seen_by(x.s, place_of(a, x.hk, r).i, a.causal); };
  const int last = (R < r0 + 32 * FWD_WAVES ? R : r0 + 32 * FWD_WAVES) - 1;
  const int steps = (seen(last) + 63) >> 6;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const KS ks(a, x.s, x.hk, lds0, dh8, wave, lane);
  for (int i = 0; i < NST - 1 && i < steps; ++i) ks.issue(i, i, wave, lane);
  const int r = rows_left > 0 ? w0 + ((lane & 31) < rows_left ? (lane & 31) : rows_left - 1) : R - 1;
  const RowPlace me = place_of(a, x.hk, r);
  const long n = x.s.q0 + me.i;
  const bf16_t* qrow = row_of<bf16_t>(a.q, n, me.h);
  const bf16_t* grow = row_of<bf16_t>(a.dout, n, me.h);
  const bf16_t* orow = row_of<bf16_t>(a.o, n, me.h);
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
  D += other_half(D);
  float L = stat_of(a.lse[n * a.heads + me.h]);
  landed(L);
  if (rows_left > 0 && lane < 32 && lane < rows_left) {
    a.dsum[n * a.heads + me.h] = -D;
    a.nlse[n * a.heads + me.h] = -L;
  }
  const int mine = seen_by(x.s, me.i, a.causal);
  const int fewest = rows_left > 0 ? seen(w0) : 0, most = rows_left > 0 ? seen(w0 + (rows_left < 32 ? rows_left : 32) - 1) : 0;
  const float c = a.scale * LOG2E;
  const unsigned ck = lds0 + Frags<DHP>::cols_lane(lane), rk = lds0 + Frags<DHP>::rows_lane(lane);
  float16v dq[G::MB];
  zero_acc(dq);
  auto step = [&](int i, int at, bool masked) __attribute__((always_inline)) {
    const unsigned tc = ck + (unsigned)at * KS::STAGE, tr = rk + (unsigned)at * KS::STAGE;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float16v s[1], dp[1];
      zero_acc(s);
#pragma unroll
      for (int e = 0; e < 16; ++e) dp[0][e] = -D;
#pragma unroll
      for (int kk = 0; kk < G::KK; ++kk) {
        s[0] = mfma(Frags<DHP>::cols(tc, b * G::TB, kk), fq[kk], s[0]);
        dp[0] = mfma(Frags<DHP>::cols(tc, (2 + b) * G::TB, kk), fg[kk], dp[0]);
      }
      float ds[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = fast_exp2(fmaf(s[0][e], c, -L));
        ds[e] = p * dp[0][e];
      }
      if (masked) {
  #pragma unroll
        for (int e = 0; e < 16; ++e)
          if (64 * i + 32 * b + tile_row_of(e, hh) >= mine) ds[e] = 0.f;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16x8 dst = pack8(ds + 8 * t);
#pragma unroll
        for (int mb = 0; mb < G::MB; ++mb) dq[mb] = mfma(Frags<DHP>::rows(tr, b * G::TB, mb, t), dst, dq[mb]);
      }
    }
  };
  int at = 0;
  for (int i = 0; i < steps; ++i) {
    if (i + NST - 2 < steps) copies_in_flight<KS::PW * (NST - 2)>();
    else copies_in_flight<0>();
    workgroup_handover();
    if (i + NST - 1 < steps) ks.issue(i + NST - 1, at == 0 ? NST - 1 : at - 1, wave, lane);
    if (64 * i < most) step(i, at, 64 * i + 64 > fewest);
    at = at == NST - 1 ? 0 : at + 1;
  }
  __syncthreads();
  if (rows_left <= 0) return;
  store_rows([&](int j) __attribute__((always_inline)) {
    const RowPlace q = place_of(a, x.hk, w0 + j);
    return row_out<bf16_t>(a.dq, x.s.q0 + q.i, q.h);
  }, rows_left, dq, a.scale, a.dh, ring + wave * 2048, lane);
  redo_rows(not_finite(dq, 0.f), rows_left, [&](int j) {
    const RowPlace q = place_of(a, x.hk, w0 + j);
    one_dq<bf16_t>(a, x.s, q.i, q.h, row_dsum<bf16_t>(a, x.s.q0 + q.i, q.h, lane), lane);
  });
}

// dk, dv.  A workgroup owns 128 keys of a key head, and eight wavefronts: four times 32 keys, twice, for every other tile of 32
// queries; the two halves' sums meet in LDS at the end.  A lane holds one key's k and v and half of that key's probabilities.
// (128 keys with four wavefronts: half the wavefronts on a SIMD, or two workgroups on a compute unit that a causal mask leaves
// unequally long; 256 keys: half as many workgroups to share out.)  Queries come from the last one down, all heads of the group
// for a tile of queries before the next tile: whatever the mask leaves them, the workgroups of a key head begin with the same
// tiles and stay in step, so that the tiles come from the XCD's L2.
// At 128 channels k stays in LDS, which leaves registers for two wavefronts on every SIMD.
constexpr int KV_KEYS = 128, KV_WAVES = 8;
template <int DHP>
__global__ __launch_bounds__(64 * KV_WAVES, 2) void packed_dkdv_mfma_kernel(PackedAttnArgs a) {
  typedef Geo<DHP> G;
  constexpr bool KLDS = DHP == 128;
  constexpr int NST = 3;
  constexpr int STAGE = 4 * G::TB;                         // two tiles of q, two of dout
  constexpr int PW = 4 * G::COPIES / KV_WAVES;             // copies of a stage by one wavefront
  constexpr int SUMS = 4 * G::MB * 16 * 64 * 4;            // the sums of four wavefronts, dk or dv
  constexpr int RING = NST * STAGE + (KLDS ? 4 * G::TB : 0);
  __shared__ __attribute__((aligned(1024))) unsigned char ring[RING > SUMS ? RING : SUMS];
  __shared__ __attribute__((aligned(256))) float stats[NST][2][2][64];           // [stage][tile][-lse | -D][32 rows, and again]
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), turn = wave >> 2;
  const Tile x = find_tile<true>(a, KV_KEYS, lane);
  if (!x.exists) return;
  const int k0 = KV_KEYS * x.t, w0 = k0 + 32 * (wave & 3);
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
  const int steps = (tiles + 1) >> 1;
  const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(ring));
  const unsigned lds1 = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_address(stats));
  const unsigned ldq = (unsigned)(a.q.row * 2), ldg = (unsigned)(a.dout.row * 2);
  // copy u of this wavefront: of tile (q, q, dout, dout) wave PW / COPIES ..., the same one for all of them
  static_assert(G::COPIES % PW == 0, "a wavefront's copies are of one tile");
  const int ct = wave * PW / G::COPIES, cp = wave * PW % G::COPIES;
  const unsigned ld = ct < 2 ? ldq : ldg;
  unsigned off[PW];
#pragma unroll
  for (int u = 0; u < PW; ++u) off[u] = copy_offset<DHP>(ld, cp + u, 32, dh8, lane);
  int ih = 0, iq = top;                                    // the next tile to ask for: its head of the group, its tile of queries
  auto ask = [&](int at) __attribute__((always_inline)) {
    int h[2], t[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {                          // (an odd number of tiles: one that nobody reads, the first one below or tile 0)
      h[b] = x.hk * a.group + ih;
      t[b] = iq < 0 ? 0 : iq;
      if (++ih == a.group) { ih = 0; --iq; }
    }
    {
      const int b = ct & 1, first = 32 * (b ? t[1] : t[0]), left = nq - first;
      const unsigned char* base = reinterpret_cast<const unsigned char*>(row_of<bf16_t>(ct < 2 ? a.q : a.dout, x.s.q0 + first, b ? h[1] : h[0]));
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
    const int b = (wave >> 1) & 1, first = 32 * (b ? t[1] : t[0]), r = first + (lane & 31) < nq ? first + (lane & 31) : nq - 1;
    copy4_to_lds((wave & 1 ? a.dsum : a.nlse) + (long)(x.s.q0 + r) * a.heads + (b ? h[1] : h[0]),
                 lds1 + (unsigned)at * 1024u + (unsigned)(wave & 3) * 256u);
  };
  for (int i = 0; i < NST - 1 && i < steps; ++i) ask(i);
  const int key = keys_left > 0 ? w0 + ((lane & 31) < keys_left ? (lane & 31) : keys_left - 1) : x.s.nk - 1;
  const bf16_t* krow = row_of<bf16_t>(a.k, x.s.k0 + key, x.hk);
  const bf16_t* vrow = row_of<bf16_t>(a.v, x.s.k0 + key, x.hk);
  const unsigned cl = Frags<DHP>::cols_lane(lane), cq = lds0 + cl + (unsigned)turn * G::TB;
  const unsigned rq = lds0 + Frags<DHP>::rows_lane(lane) + (unsigned)turn * G::TB;
  const unsigned kl = lds0 + NST * STAGE + (unsigned)(wave & 3) * G::TB + cl;
  bf16x8 fk[G::KK], fv[G::KK];
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) { fk[kk] = own_piece(krow, kk, dh8, lane); fv[kk] = own_piece(vrow, kk, dh8, lane); }
#pragma unroll
  for (int kk = 0; kk < G::KK; ++kk) {
    landed(fk[kk]);
    landed(fv[kk]);
    // (both wavefronts of these keys write the same)
    if (KLDS) put_cols_lds<DHP>(ring + NST * STAGE + (wave & 3) * G::TB, kk, lane, fk[kk]);
  }
  const int mine = first_query(key);                       // the first query that sees this lane's key
  const int begin = keys_left > 0 ? first_query(w0) : nq, all = keys_left > 0 ? first_query(w0 + (keys_left < 32 ? keys_left : 32) - 1) : nq;
  const float c = a.scale * LOG2E;
  float16v dk[G::MB], dv[G::MB];
  zero_acc(dk);
  zero_acc(dv);
  auto step = [&](int first, int at, bool masked) __attribute__((always_inline)) {
    const unsigned tc = cq + (unsigned)at * STAGE, tr = rq + (unsigned)at * STAGE;
    float16v s[1], dp;
    float p[16];
    zero_acc(s);
#pragma unroll
    for (int kk = 0; kk < G::KK; ++kk) s[0] = mfma(Frags<DHP>::cols(tc, 0, kk), KLDS ? Frags<DHP>::cols(kl, 0, kk) : fk[kk], s[0]);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 u = *reinterpret_cast<const float4*>(&stats[at][turn][1][8 * g + 4 * hh]);
      dp[4 * g] = u.x; dp[4 * g + 1] = u.y; dp[4 * g + 2] = u.z; dp[4 * g + 3] = u.w;
    }
#pragma unroll
    for (int kk = 0; kk < G::KK; ++kk) dp = mfma(Frags<DHP>::cols(tc, 2 * G::TB, kk), fv[kk], dp);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 u = *reinterpret_cast<const float4*>(&stats[at][turn][0][8 * g + 4 * hh]);
      p[4 * g] = fast_exp2(fmaf(s[0][4 * g], c, u.x));
      p[4 * g + 1] = fast_exp2(fmaf(s[0][4 * g + 1], c, u.y));
      p[4 * g + 2] = fast_exp2(fmaf(s[0][4 * g + 2], c, u.z));
      p[4 * g + 3] = fast_exp2(fmaf(s[0][4 * g + 3], c, u.w));
    }
    if (masked) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int i = first + tile_row_of(e, hh);
        if (i < mine || i >= nq) p[e] = 0.f;
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 pt = pack8(p + 8 * t);
#pragma unroll
      for (int mb = 0; mb < G::MB; ++mb) dv[mb] = mfma(Frags<DHP>::rows(tr, 2 * G::TB, mb, t), pt, dv[mb]);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) p[e] *= dp[e];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 dst = pack8(p + 8 * t);
#pragma unroll
      for (int mb = 0; mb < G::MB; ++mb) dk[mb] = mfma(Frags<DHP>::rows(tr, 0, mb, t), dst, dk[mb]);
    }
  };
  int at = 0, sh = turn, sq = top;                         // this wavefront's next tile
  if (sh >= a.group) { sh -= a.group; --sq; }
  for (int i = 0; i < steps; ++i) {
    if (i + NST - 2 < steps) copies_in_flight<(PW + 1) * (NST - 2)>();
    else copies_in_flight<0>();
    workgroup_handover();
    if (i + NST - 1 < steps) ask(at == 0 ? NST - 1 : at - 1);
    const int first = 32 * sq;
    if (2 * i + turn < tiles && first + 32 > begin && keys_left > 0) step(first, at, first < all || first + 32 > nq);
    at = at == NST - 1 ? 0 : at + 1;
    sh += 2;
    if (sh >= a.group) {
      sh -= a.group;
      --sq;
      if (sh >= a.group) { sh -= a.group; --sq; }          // (a group of one)
    }
  }
  float* const sums = reinterpret_cast<float*>(ring) + (wave & 3) * (G::MB * 16 * 64) + lane;
  auto meet = [&](float16v (&acc)[G::MB]) __attribute__((always_inline)) {
    __syncthreads();                                       // (the ring, or the sums before, are free)
    if (turn == 1) {
#pragma unroll
      for (int m = 0; m < G::MB; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[(m * 16 + e) * 64] = acc[m][e];
    }
    __syncthreads();
    if (turn == 0) {
#pragma unroll
      for (int m = 0; m < G::MB; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[m][e] += sums[(m * 16 + e) * 64];
    }
  };
  meet(dk);
  meet(dv);
  __syncthreads();
  if (turn == 1 || keys_left <= 0) return;
  unsigned char* stg = ring + wave * 2048;
  store_rows([&](int j) __attribute__((always_inline)) { return row_out<bf16_t>(a.dk, x.s.k0 + w0 + j, x.hk); }, keys_left, dk, a.scale,
             a.dh, stg, lane);
  store_rows([&](int j) __attribute__((always_inline)) { return row_out<bf16_t>(a.dv, x.s.k0 + w0 + j, x.hk); }, keys_left, dv, 1.f, a.dh,
             stg, lane);
  redo_rows(not_finite(dv, not_finite(dk, 0.f)), keys_left, [&](int j) { one_dkdv<bf16_t>(a, x.s, w0 + j, x.hk, lane); });
}

// workgroups for tiles of `per` rows (keys)
template <bool KEYS>
unsigned tile_grid(const PackedAttnArgs& a, int per) {
  const long rows = KEYS ? a.k_rows : (long)a.q_rows * a.group;
  if (rows == 0) return 0;
  const bool equal = KEYS ? !a.k_off : !a.q_off;
  const long tiles = equal ? a.seqs * ((rows / a.seqs + per - 1) / per) : rows / per + a.seqs;
  return (unsigned)(tiles * a.kv_heads);
}
template <int DHP>
hipError_t fwd_mfma(const PackedAttnArgs& a, hipStream_t s) {
  if (const unsigned grid = tile_grid<false>(a, 32 * FWD_WAVES)) packed_fwd_mfma_kernel<DHP><<<grid, 64 * FWD_WAVES, 0, s>>>(a);
  return hipGetLastError();
}
template <int DHP>
hipError_t bwd_mfma(const PackedAttnArgs& a, hipStream_t s) {
  if (const unsigned grid = tile_grid<false>(a, 32 * FWD_WAVES)) packed_dq_mfma_kernel<DHP><<<grid, 64 * FWD_WAVES, 0, s>>>(a);
  if (const unsigned grid = tile_grid<true>(a, KV_KEYS)) packed_dkdv_mfma_kernel<DHP><<<grid, 64 * KV_WAVES, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t fwd_t(const PackedAttnArgs& a, hipStream_t s) {
  if (a.q_rows == 0) return hipSuccess;
  packed_fwd_rows_kernel<T><<<(unsigned)((long)a.q_rows * a.heads), 64, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T>
hipError_t bwd_t(const PackedAttnArgs& a, hipStream_t s) {
  if (a.q_rows > 0) packed_dq_rows_kernel<T><<<(unsigned)((long)a.q_rows * a.heads), 64, 0, s>>>(a);
  if (a.k_rows > 0) packed_dkdv_rows_kernel<T><<<(unsigned)((long)a.k_rows * a.kv_heads), 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t packed_attn_ws_bytes(int dtype, const PackedAttnArgs& a) {
  (void)dtype;
  return 2 * (((size_t)a.q_rows * a.heads * 4 + 255) / 256 * 256);
}
hipError_t launch_packed_attn_fwd(int dtype, const PackedAttnArgs& a, void*, hipStream_t s) {
  return dtype == 0 ? fwd_t<float>(a, s) : a.dh <= 64 ? fwd_mfma<64>(a, s) : fwd_mfma<128>(a, s);
}
hipError_t launch_packed_attn_bwd(int dtype, const PackedAttnArgs& a, void* workspace, hipStream_t s) {
  PackedAttnArgs b = a;
  b.dsum = reinterpret_cast<float*>(workspace);
  b.nlse = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + packed_attn_ws_bytes(dtype, a) / 2);
  return dtype == 0 ? bwd_t<float>(b, s) : a.dh <= 64 ? bwd_mfma<64>(b, s) : bwd_mfma<128>(b, s);
}

}  // namespace hbp
