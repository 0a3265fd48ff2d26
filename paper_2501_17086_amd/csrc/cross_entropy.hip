// Softmax cross entropy of rows x against a vocabulary's weights W, and its gradients, in pieces of the vocabulary:
//   s = scale x W^T,  loss_n = log sum_v exp s_nv - s_n,t,   dS = g (softmax(s) - onehot(t)),  dx = scale dS W,  dW = scale dS^T x.
// A piece's logits are formed, their row sums taken and, for the gradients, turned into dS, which meets W and x; nothing of the size
// rows x vocabulary is kept.  Where the vocabulary takes several pieces the logits are formed twice, once for the sums.
//
// Logits lie [vocabulary][rows]: the vocabulary may have any size (it is the product's rows), the number of rows is filled up
// with zeros to a multiple of 8, and both gradients' products find their contraction where the kernels want it.
// Rows whose target is no token take no part: they are zeros in the copy of x that the products read, so that not even
// an infinity or a NaN in them reaches the others.
#include "hbp_common.h"

namespace hbp {

namespace {

constexpr int NTHR = 256;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int BLOCK_V = 256;                               // rows of the vocabulary whose sum is one number per row of x

struct Parts {
  void* x;                // [np, width], storage type: x, zeros where a row does not count
  float* target_logit;    // [np], times log2 e
  float* lse;             // [np], base 2; infinity where a row does not count: its probabilities are zeros
  int* target;            // [np], -1 where a row does not count
  float* rows;            // [np] row losses
  float* scalars;         // [4]: the factor on dS
  float* sums;            // [blocks][np]: base 2 logarithms of a block's sums
  float* logits;          // [piece][np]
  void* grad;             // [piece][np], storage type (fp32: the logits' place)
  float* dx;              // [shares][np, width]
  long np, piece;
  int blocks, pieces, shares;   // shares: products whose results lie side by side until they are added up
  size_t bytes;
};

struct CeArgs {
  CrossEntropyArgs c;
  Parts p;
  float to_log2;          // scale log2 e
  long v0, nv;            // the piece at hand
};

// x's copy, the target's logit: a wavefront a row
template <typename T>
__global__ __launch_bounds__(NTHR) void rows_kernel(CeArgs a) {
  const int lane = threadIdx.x & 63;
  const long n = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= a.p.np) return;
  const int t = n < a.c.rows ? a.c.targets[n] : -1;
  const bool counts = t >= 0 && t < a.c.vocab;
  T* copy = reinterpret_cast<T*>(a.p.x) + n * a.c.width;
  float dot = 0.f;
  for (int c = 8 * lane; c < a.c.width; c += 512) {
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (counts) {
      float w[8];
      load8(reinterpret_cast<const T*>(a.c.x.p) + n * a.c.x.row + c, v);
      load8(reinterpret_cast<const T*>(a.c.weight.p) + t * a.c.weight.row + c, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) dot = fmaf(v[j], w[j], dot);
    }
    store8(copy + c, v);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
  if (lane == 0) {
    a.p.target_logit[n] = dot * a.to_log2;
    a.p.target[n] = counts ? t : -1;
  }
}

// running maximum and sum of 2^v
struct Running {
  float m, l;
  __device__ __forceinline__ void add(float om, float ol) {
    const float n = fmaxf(m, om);
    if (n == -INFINITY) { l += ol; return; }               // (nothing yet: zeros, or a NaN, which stays)
    l = l * exp2f(m - n) + ol * exp2f(om - n);
    m = n;
  }
};
__device__ __forceinline__ float log2_sum(const Running& r) { return r.l == 0.f ? -INFINITY : r.m + log2f(r.l); }

// TB rows of x by 256 / TB parts of a block of the vocabulary a workgroup
template <int TB>
__device__ __forceinline__ Running meet(Running r, int part, int row, float (&sm)[NTHR / TB][TB], float (&sl)[NTHR / TB][TB]) {
  sm[part][row] = r.m;
  sl[part][row] = r.l;
  __syncthreads();
  Running t = {-INFINITY, 0.f};
  if (part == 0) {
    t = {sm[0][row], sl[0][row]};
    for (int i = 1; i < NTHR / TB; ++i) t.add(sm[i][row], sl[i][row]);
  }
  return t;
}
template <int TB>
__global__ __launch_bounds__(NTHR) void block_sums_kernel(CeArgs a) {
  constexpr int PARTS = NTHR / TB, PER = BLOCK_V / PARTS;
  __shared__ float sm[PARTS][TB], sl[PARTS][TB];
  const int row = threadIdx.x % TB, part = threadIdx.x / TB;
  const long n = (long)blockIdx.x * TB + row, nc = n < a.p.np ? n : a.p.np - 1;
  const long v0 = (long)blockIdx.y * BLOCK_V + part;
  Running r = {-INFINITY, 0.f};
  for (int i = 0; i < PER; i += 8) {
    float v[8];
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const long at = v0 + (long)(i + j) * PARTS;
      v[j] = at < a.nv ? a.p.logits[at * a.p.np + nc] * a.to_log2 : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, v[j]);
    float sum = 0.f;
    bool nan = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum += top == -INFINITY ? 0.f : exp2f(v[j] - top);
      nan = nan || v[j] != v[j];
    }
    r.add(top, nan ? NAN : sum);
  }
  const Running t = meet<TB>(r, part, row, sm, sl);
  if (part == 0 && n < a.p.np) a.p.sums[(a.v0 / BLOCK_V + blockIdx.y) * a.p.np + n] = log2_sum(t);
}
// all blocks of a row, its loss
template <int TB>
__global__ __launch_bounds__(NTHR) void row_loss_kernel(CeArgs a) {
  constexpr int PARTS = NTHR / TB;
  __shared__ float sm[PARTS][TB], sl[PARTS][TB];
  const int row = threadIdx.x % TB, part = threadIdx.x / TB;
  const long n = (long)blockIdx.x * TB + row, nc = n < a.p.np ? n : a.p.np - 1;
  Running r = {-INFINITY, 0.f};
  for (int b = part; b < a.p.blocks; b += PARTS) {
    const float v = a.p.sums[(long)b * a.p.np + nc];
    r.add(v, v == -INFINITY ? 0.f : v != v ? NAN : 1.f);
  }
  const Running t = meet<TB>(r, part, row, sm, sl);
  if (part != 0 || n >= a.p.np) return;
  const bool counts = a.p.target[n] >= 0;
  const float lse = log2_sum(t);
  const float loss = counts ? (lse - a.p.target_logit[n]) * LN2 : 0.f;
  a.p.lse[n] = counts ? lse : INFINITY;
  a.p.rows[n] = loss;
  if (a.c.row_loss && n < a.c.rows) a.c.row_loss[n] = loss;
}
// the loss, and what dS is multiplied by: one workgroup, sums in 64 bits in a fixed order
__global__ __launch_bounds__(1024) void loss_kernel(CeArgs a) {
  __shared__ double sum[1024];
  __shared__ int cnt[1024];
  const int tid = threadIdx.x;
  double s = 0.0;
  int c = 0;
  for (long n = tid; n < a.c.rows; n += 1024) {
    s += (double)a.p.rows[n];
    c += a.p.target[n] >= 0;
  }
  sum[tid] = s;
  cnt[tid] = c;
  __syncthreads();
  for (int o = 512; o > 0; o >>= 1) {
    if (tid < o) { sum[tid] += sum[tid + o]; cnt[tid] += cnt[tid + o]; }
    __syncthreads();
  }
  if (tid == 0) {
    const double f = (double)a.c.factor / (a.c.mean && cnt[0] > 1 ? cnt[0] : 1);
    a.c.loss[0] = (float)(sum[0] * f);
    a.p.scalars[0] = (float)(f * a.c.scale);
  }
}

// dS of a piece: 8 rows of x a thread
template <typename T>
__global__ __launch_bounds__(NTHR) void grad_kernel(CeArgs a) {
  const long per = a.p.np / 8, i = (long)blockIdx.x * NTHR + threadIdx.x;
  if (i >= per * a.nv) return;
  const long v = i / per, n = 8 * (i - v * per);
  float s[8], lse[8];
  load8(a.p.logits + v * a.p.np + n, s);
  load8(a.p.lse + n, lse);
  const float g = a.p.scalars[0];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float p = lse[j] == INFINITY ? 0.f : exp2f(fmaf(s[j], a.to_log2, -lse[j]));
    if (a.p.target[n + j] == a.v0 + v) p -= 1.f;
    s[j] = p * g;
  }
  store8(reinterpret_cast<T*>(a.p.grad) + v * a.p.np + n, s);
}

// the first share of dx += the others; elements of 8
__global__ __launch_bounds__(NTHR) void fold_kernel(float* dx, long n8, int shares) {
  const long i = (long)blockIdx.x * NTHR + threadIdx.x;
  if (i >= n8) return;
  float s[8];
  load8(dx + 8 * i, s);
  for (int k = 1; k < shares; ++k) {
    float v[8];
    load8(dx + 8 * (k * n8 + i), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] += v[j];
  }
  store8(dx + 8 * i, s);
}
// dx from its shares, rounded once; rows that do not count are zeros
template <typename T>
__global__ __launch_bounds__(NTHR) void dx_kernel(CeArgs a, Divisor by_row, int shares) {
  const long base = (long)blockIdx.x * NTHR;
  const unsigned per = (unsigned)(a.c.width / 8);
  const long row0 = base / per;
  const unsigned r = (unsigned)(base - row0 * per) + threadIdx.x, q = by_row.quotient(r);
  const long n = row0 + q;
  if (n >= a.c.rows) return;
  const long c = 8l * (r - q * per);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (a.p.target[n] >= 0) {
    for (int k = 0; k < shares; ++k) {
      float v[8];
      load8(a.p.dx + ((long)k * a.p.np + n) * a.c.width + c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += v[j];
    }
  }
  store8(reinterpret_cast<T*>(a.c.dx.p) + n * a.c.dx.row + c, s);
}
template <typename T>
__global__ __launch_bounds__(NTHR) void clear_kernel(T* p, long row, long rows, int width) {
  const long i = (long)blockIdx.x * NTHR + threadIdx.x, per = width / 8;
  if (i >= rows * per) return;
  const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  store8(p + i / per * row + 8 * (i % per), z);
}

// ---- sizes -----------------------------------------------------------------------------------------------------------
// A piece's logits take 1 GB at most (256 rows of the vocabulary: more, from 2^20 rows on), and four pieces' dx lie side by side.
constexpr long PIECE_LOGITS = 1l << 28, PIECE_ROWS = 1l << 20;
constexpr int SHARES = 4;
Parts carve(char* base, int dtype, long rows, long vocab, int width, bool gradients) {
  Parts p{};
  size_t off = 0;
  auto take = [&](size_t n) { char* q = base ? base + off : nullptr; off += (n + 255) / 256 * 256; return q; };
  const size_t es = dtype == 0 ? 4 : 2;
  p.np = (rows + 7) / 8 * 8;
  const long fit = PIECE_LOGITS / (p.np ? p.np : 1) / BLOCK_V * BLOCK_V;
  p.piece = fit < BLOCK_V ? BLOCK_V : fit < PIECE_ROWS ? fit : PIECE_ROWS;
  if (p.piece > vocab) p.piece = vocab;
  p.pieces = (int)((vocab + p.piece - 1) / p.piece);
  p.blocks = (int)((vocab + BLOCK_V - 1) / BLOCK_V);
  p.x = take(p.np * width * es);
  p.target_logit = reinterpret_cast<float*>(take(4 * p.np));
  p.lse = reinterpret_cast<float*>(take(4 * p.np));
  p.target = reinterpret_cast<int*>(take(4 * p.np));
  p.rows = reinterpret_cast<float*>(take(4 * p.np));
  p.scalars = reinterpret_cast<float*>(take(16));
  p.sums = reinterpret_cast<float*>(take((size_t)p.blocks * p.np * 4));
  p.logits = reinterpret_cast<float*>(take((size_t)p.piece * p.np * 4));
  p.grad = p.logits;
  if (gradients) {
    if (dtype == 1) p.grad = take((size_t)p.piece * p.np * 2);
    p.shares = p.pieces < SHARES ? p.pieces : SHARES;
    p.dx = reinterpret_cast<float*>(take((size_t)p.shares * p.np * width * 4));
  }
  p.bytes = off;
  return p;
}

hipError_t product(int dtype, const GemmArgs& g, hipStream_t s) {
  if (dtype == 1) {
    hipError_t e;
    if (launch_gemm_mfma(g, s, &e)) return e;
  } else if (gemm_f32_ok(g)) {
    return launch_gemm_f32(g, s);
  }
  return launch_gemm_generic(dtype, g, s);
}

#define CE_TRY(call)                      \
  do {                                    \
    const hipError_t e_ = (call);         \
    if (e_ != hipSuccess) return e_;      \
  } while (0)

template <typename T>
hipError_t run(int dtype, const CrossEntropyArgs& c, const Parts& p, hipStream_t s) {
  CeArgs a{};
  a.c = c; a.p = p; a.to_log2 = c.scale * LOG2E;
  const bool grads = c.dx.p || c.dweight.p;
  const T* weight = reinterpret_cast<const T*>(c.weight.p);
  if (c.rows == 0) {                                       // nothing counts
    loss_kernel<<<1, 1024, 0, s>>>(a);
    CE_TRY(hipGetLastError());
  } else {
    rows_kernel<T><<<(unsigned)((p.np + 3) / 4), NTHR, 0, s>>>(a);
    CE_TRY(hipGetLastError());
  }
  auto logits = [&](long v0, long nv) {
    GemmArgs g{};
    g.A = weight + v0 * c.weight.row; g.a_sm = c.weight.row; g.a_sk = 1;
    g.B = p.x; g.b_sn = c.width; g.b_sk = 1;
    g.C = p.logits; g.ldc = p.np; g.c_is_f32 = 1;
    g.M = nv; g.N = p.np; g.K = c.width;
    g.batch = 1; g.split_k = 1; g.mode = EPI_STORE;
    return product(dtype, g, s);
  };
  auto piece_at = [&](int i) { a.v0 = i * p.piece; a.nv = c.vocab - a.v0 < p.piece ? c.vocab - a.v0 : p.piece; };
  if (c.rows) {
    for (int i = 0; i < p.pieces; ++i) {
      piece_at(i);
      CE_TRY(logits(a.v0, a.nv));
      const unsigned nb = (unsigned)((a.nv + BLOCK_V - 1) / BLOCK_V);
      if (p.np >= 64) block_sums_kernel<64><<<dim3((unsigned)((p.np + 63) / 64), nb), NTHR, 0, s>>>(a);
      else block_sums_kernel<8><<<dim3((unsigned)(p.np / 8), nb), NTHR, 0, s>>>(a);
      CE_TRY(hipGetLastError());
    }
    if (p.np >= 4096) row_loss_kernel<64><<<(unsigned)((p.np + 63) / 64), NTHR, 0, s>>>(a);
    else row_loss_kernel<8><<<(unsigned)(p.np / 8), NTHR, 0, s>>>(a);
    loss_kernel<<<1, 1024, 0, s>>>(a);
    CE_TRY(hipGetLastError());
  }
  if (!grads) return hipSuccess;
  if (c.rows == 0) {
    if (!c.dweight.p) return hipSuccess;
    const unsigned blocks = (unsigned)((c.vocab * (c.width / 8) + NTHR - 1) / NTHR);
    if (c.grad_dtype == 0) clear_kernel<float><<<blocks, NTHR, 0, s>>>(reinterpret_cast<float*>(c.dweight.p), c.dweight.row, c.vocab, c.width);
    else clear_kernel<bf16_t><<<blocks, NTHR, 0, s>>>(reinterpret_cast<bf16_t*>(c.dweight.p), c.dweight.row, c.vocab, c.width);
    return hipGetLastError();
  }
  int shares = 0;
  for (int i = 0; i < p.pieces; ++i) {
    piece_at(i);
    if (p.pieces > 1) CE_TRY(logits(a.v0, a.nv));
    grad_kernel<T><<<(unsigned)((a.nv * (p.np / 8) + NTHR - 1) / NTHR), NTHR, 0, s>>>(a);
    CE_TRY(hipGetLastError());
    if (c.dweight.p) {
      GemmArgs g{};
      g.A = p.grad; g.a_sm = p.np; g.a_sk = 1;
      g.B = p.x; g.b_sk = c.width; g.b_sn = 1;
      g.c_is_f32 = c.grad_dtype == 0;
      if (g.c_is_f32) g.C = reinterpret_cast<float*>(c.dweight.p) + a.v0 * c.dweight.row;
      else g.C = reinterpret_cast<bf16_t*>(c.dweight.p) + a.v0 * c.dweight.row;
      g.ldc = c.dweight.row;
      g.M = a.nv; g.N = c.width; g.K = p.np;
      g.batch = 1; g.split_k = 1; g.mode = EPI_STORE;
      CE_TRY(product(dtype, g, s));
    }
    if (c.dx.p) {
      if (shares == p.shares) {
        const long n8 = p.np * c.width / 8;
        fold_kernel<<<(unsigned)((n8 + NTHR - 1) / NTHR), NTHR, 0, s>>>(p.dx, n8, shares);
        CE_TRY(hipGetLastError());
        shares = 1;
      }
      GemmArgs g{};
      g.A = p.grad; g.a_sm = 1; g.a_sk = p.np;
      g.B = weight + a.v0 * c.weight.row; g.b_sk = c.weight.row; g.b_sn = 1;
      g.C = p.dx + (long)shares++ * p.np * c.width; g.ldc = c.width; g.c_is_f32 = 1;
      g.M = p.np; g.N = c.width; g.K = a.nv;
      g.batch = 1; g.split_k = 1; g.mode = EPI_STORE;
      CE_TRY(product(dtype, g, s));
    }
  }
  if (c.dx.p) {
    const unsigned per = (unsigned)(c.width / 8);
    dx_kernel<T><<<(unsigned)((c.rows * per + NTHR - 1) / NTHR), NTHR, 0, s>>>(a, Divisor(per), shares);
    CE_TRY(hipGetLastError());
  }
  return hipSuccess;
}

}  // namespace

size_t cross_entropy_ws_bytes(int dtype, long rows, long vocab, int width, bool gradients) {
  return carve(nullptr, dtype, rows, vocab, width, gradients).bytes;
}

hipError_t launch_cross_entropy(int dtype, const CrossEntropyArgs& c, void* workspace, size_t bytes, hipStream_t s) {
  const Parts p = carve(reinterpret_cast<char*>(workspace), dtype, c.rows, c.vocab, c.width, c.dx.p || c.dweight.p);
  if (bytes < p.bytes) return hipErrorInvalidValue;
  return dtype == 0 ? run<float>(dtype, c, p, s) : run<bf16_t>(dtype, c, p, s);
}

}  // namespace hbp
