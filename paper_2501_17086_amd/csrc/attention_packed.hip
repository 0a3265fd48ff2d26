// Attention over packed sequences, forward and backward, whose key/value heads serve groups of query heads.
//
// A key/value head's `group` query heads see the same keys, so the rows that a sequence brings to it are its queries
// times its group, row r = query r / group of head r % group: tiles of rows then hold several heads of a query, the
// streamed keys serve all of them, dk and dv sum over the group by summing over rows, and a single query fills `group`
// rows of a tile.
#include "hbp_common.h"

#include <cfloat>

namespace hbp {

namespace {

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
        const float L = stat_of(a.lse[r * a.heads + h]);
        if (L != INFINITY) {
          p = exp2f(c * dot_rows(row_of<T>(a.q, r, h), k, a.dh) - L);
          ds = p * (dot_rows(row_of<T>(a.dout, r, h), v, a.dh) - a.dsum[r * a.heads + h]);
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
  if (threadIdx.x == 0) a.dsum[(long)n * a.heads + h] = D;
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

size_t packed_attn_ws_bytes(int, const PackedAttnArgs& a) {
  return ((size_t)a.q_rows * a.heads * 4 + 255) / 256 * 256;
}
hipError_t launch_packed_attn_fwd(int dtype, const PackedAttnArgs& a, void*, hipStream_t s) {
  return dtype == 0 ? fwd_t<float>(a, s) : fwd_t<bf16_t>(a, s);
}
hipError_t launch_packed_attn_bwd(int dtype, const PackedAttnArgs& a, void* workspace, hipStream_t s) {
  PackedAttnArgs b = a;
  b.dsum = reinterpret_cast<float*>(workspace);
  return dtype == 0 ? bwd_t<float>(b, s) : bwd_t<bf16_t>(b, s);
}

}  // namespace hbp
