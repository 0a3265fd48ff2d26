// Softmax cross entropy of rows x against a vocabulary's weights W, and its gradients, in pieces of the vocabulary:
//   s = scale x W^T,  loss_n = log sum_v exp s_nv - s_n,t,   dS = g (softmax(s) - onehot(t)),  dx = scale dS W,  dW = scale dS^T x.
// A piece's logits are formed, their row sums taken and, for the gradients, turned into dS, which meets W and x; nothing of the size
// rows x vocabulary is kept.  Three forms, by sizes alone:
//   many tiles  (bf16) the logits meet no memory: the 256 x 256 kernel's epilogues take sums of 128 rows of the vocabulary from its
//               accumulators, and once more, when a row's sum is known, dS.  Four products of 2 rows x vocabulary x width where keeping the
//               logits would leave three; what bounds it are the matrix cores, busy for 70 to 80 % of the four products' cycles: 16384 rows against
//               131072 x 2048, kernel times on a card where a large product of the library reaches 1373 TFLOP/s, 6.79 ms for the sums, 7.14 dS, 6.40 dW,
//               6.65 dx, 27.2 in all, 1300 TFLOP/s over the four (cards differ by some 6 %).  With 256 channels a tile's exponentials and stores take
//               as long as its products: 32768 rows against 16384 x 256 275, 347, 243, 235 us, matrix cores busy for 50, 37, 54 and 52 %.
//   pieces      logits in memory in fp32, at most 1 GB at a time; with one piece they are formed once.  fp32, and few rows.
//   small       the same with logits and sums in one launch (small_logits_kernel): launches bound it, 2 to 10 us each.
//
// Logits lie [vocabulary][rows]: the vocabulary may have any size (it is the product's rows), the number of rows is filled up
// with zeros to a multiple of 8 or 256, and both gradients' products find their contraction where the kernels want it.
// Rows whose target is no token take no part: they are zeros in the copy of x that the products read, so that not even
// an infinity or a NaN in them reaches the others.  Logits, sums, dx and dweight are held in fp32; dS is rounded to the storage type once (twice the bits
// for few rows, TWO_TERMS), as the matrix instructions want it, with a power of two as its factor (the rest of the factor comes after the
// products), and dx gets back what that leaves out of the target's coefficient, the one that a confident row is made of.
#include "hbp_common.h"

namespace hbp {

namespace {

typedef float float16v __attribute__((ext_vector_type(16)));
constexpr int NTHR = 256;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int AFTER = 4;                                   // (16 bytes on)
constexpr int BLOCK_V = 64;                                // rows of the vocabulary whose sum is one number per row of x

struct Parts {
  void* x;                // [gp, wp], storage type: x, zeros where a row does not count and behind its channels; once for each term of dS
  void* weight;           // [vocab, wp]: the weights with zeros behind their channels, where wp is not the width; else NULL
  float* target_logit;    // [np]
  float* lse;             // [np], base 2; infinity where a row does not count: its probabilities are zeros
  int* target;            // [np], -1 where a row does not count
  float* rows;            // [np] row losses
  float* at_target;       // [np] the target's softmax less 1
  float* scalars;         // [0]: the factor on dS; [AFTER]: what dx and dweight are multiplied by afterwards
  float2* sums;           // [blocks][np]: a block's largest logit, and its sum of exponentials relative to that
  float* logits;          // [piece][np]
  void* grad;             // [piece][gp], storage type (fp32: the logits' place); of two terms the second behind the first
  float* dx;              // [shares][gp, wp]
  float* dweight;         // [shares of the contraction][rows at hand, width], where there are several
  long np, gp, piece;     // gp: np once for each term of dS
  int wp;                 // channels with those that fill up
  long fused;             // rows of the vocabulary whose logits meet no memory
  int blocks, pieces, shares;   // shares: products whose results lie side by side until they are added up
  size_t dweight_bytes, bytes;
};

struct CeArgs {
  CrossEntropyArgs c;
  Parts p;
  float to_log2;          // scale log2 e
  int power;              // bf16: dS has a power of two as its factor, the rest of it comes after the products
  long v0, nv;            // the rows of the vocabulary at hand
  long block0;            // their first block of sums
  long grad0;             // where their dS begins in its piece
  unsigned grad_blocks;   // grad_kernel's workgroups; those behind them copy x
};

// x's copy, a wavefront a row
template <typename T>
__device__ __forceinline__ void copy_row(const CeArgs& a, long n, int lane, bool counts) {
  T* copy = reinterpret_cast<T*>(a.p.x) + n * a.p.wp;
  const bool twice = a.p.gp > a.p.np;
  for (int c = 8 * lane; c < a.p.wp; c += 512) {
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (counts && c < a.c.width) load8(reinterpret_cast<const T*>(a.c.x.p) + n * a.c.x.row + c, v);
    store8(copy + c, v);
    if (twice) store8(copy + a.p.np * a.p.wp + c, v);
  }
}
__device__ __forceinline__ int target_of(const CeArgs& a, long n) {
  const int t = n < a.c.rows ? a.c.targets[n] : -1;
  return t >= 0 && t < a.c.vocab ? t : -1;
}
template <typename T>
__global__ __launch_bounds__(NTHR) void rows_kernel(CeArgs a) {
  const int lane = threadIdx.x & 63;
  const long n = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= a.p.np) return;
  const int t = target_of(a, n);
  copy_row<T>(a, n, lane, t >= 0);
  if (lane == 0) a.p.target[n] = t;
}

// the weights with their channels filled up
__global__ __launch_bounds__(NTHR) void weight_kernel(CeArgs a) {
  const long per = a.p.wp / 8, total = a.c.vocab * per;
  for (long i = (long)blockIdx.x * NTHR + threadIdx.x; i < total; i += (long)gridDim.x * NTHR) {
    const long v = i / per, c = 8 * (i - v * per);
    uint4 w = make_uint4(0, 0, 0, 0);
    if (c < a.c.width) w = *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16_t*>(a.c.weight.p) + v * a.c.weight.row + c);
    *reinterpret_cast<uint4*>(reinterpret_cast<bf16_t*>(a.p.weight) + v * a.p.wp + c) = w;
  }
}

// Running maximum of logits and sum of 2^(alpha (logit - maximum)).  The pair is kept as it is until a row's loss is made of it: one logarithm
// a block in its place is rounded at the logits' size, in every block (a vocabulary of 2000 equal logits of 105: 4e-6 of a loss of 7.6).
struct Running {
  float m, l;
  __device__ __forceinline__ void add(float om, float ol, float alpha) {
    const float n = fmaxf(m, om);
    if (n == -INFINITY) { l += ol; return; }               // (nothing yet: zeros, or a NaN, which stays)
    l = l * __builtin_amdgcn_exp2f((m - n) * alpha) + ol * __builtin_amdgcn_exp2f((om - n) * alpha);
    m = n;
  }
  // K pairs at once
  template <int K> __device__ __forceinline__ void add(const float (&v)[K], const float (&w)[K], float alpha) {
    float top = v[0], sum = 0.f;
#pragma unroll
    for (int j = 1; j < K; ++j) top = fmaxf(top, v[j]);
    const float shift = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int j = 0; j < K; ++j) sum += w[j] * __builtin_amdgcn_exp2f((v[j] - shift) * alpha);
    add(top, sum, alpha);
  }
  // K logits
  template <int K> __device__ __forceinline__ void add(const float (&v)[K], float alpha) {
    float one[K];
#pragma unroll
    for (int j = 0; j < K; ++j) one[j] = 1.f;
    add(v, one, alpha);
  }
};

// the parts' sums of TB rows meet in a fixed tree; thread = part TB + row, the result is part 0's
template <int TB, int NT>
__device__ __forceinline__ Running meet(Running r, float alpha, float (&sm)[NT], float (&sl)[NT]) {
  const int t = threadIdx.x;
  sm[t] = r.m;
  sl[t] = r.l;
  __syncthreads();
#pragma unroll
  for (int o = NT / 2; o >= TB; o /= 2) {
    if (t < o) {
      r.add(sm[t + o], sl[t + o], alpha);
      sm[t] = r.m;
      sl[t] = r.l;
    }
    __syncthreads();
  }
  return r;
}
// a block's sums from its logits, and the targets' among them: TB rows of x a workgroup
template <int TB>
__global__ __launch_bounds__(NTHR) void block_sums_kernel(CeArgs a) {
  constexpr int PARTS = NTHR / TB, PER = BLOCK_V / PARTS;
  __shared__ float sm[NTHR], sl[NTHR];
  const int row = threadIdx.x % TB, part = threadIdx.x / TB;
  const long n = (long)blockIdx.x * TB + row, nc = n < a.p.np ? n : a.p.np - 1;
  const long v0 = (long)blockIdx.y * BLOCK_V + part;
  float v[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const long at = v0 + j * PARTS;
    v[j] = at < a.nv ? a.p.logits[at * a.p.np + nc] : -INFINITY;
  }
  const long target = n < a.p.np ? a.p.target[n] - a.v0 : -1;
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (target == v0 + j * PARTS && target < a.nv) a.p.target_logit[n] = v[j];
  Running r = {-INFINITY, 0.f};
  r.add(v, a.to_log2);
  r = meet<TB>(r, a.to_log2, sm, sl);
  if (part == 0 && n < a.p.np) a.p.sums[(a.block0 + blockIdx.y) * a.p.np + n] = make_float2(r.m, r.l);
}

// Small problems: logits, a block's sums and the targets' logits in one launch, without x's copy.  A workgroup takes 64 rows of the vocabulary and
// 32 of x, its wavefronts a quarter of the channels each, straight from memory into the layout of the matrix instructions, and
// the quarters meet in LDS.  (8 rows against 16384 x 256: 16.0 -> 10.7 us.)
template <typename T> struct Frag;
template <> struct Frag<bf16_t> {                          // 16 channels a step, 8 of them in each half of the wavefront
  typedef __bf16 vec __attribute__((ext_vector_type(8)));
  static constexpr int STEP = 16;
  uint4 v;
  __device__ __forceinline__ void load(const bf16_t* row, int k, int h, int end, bool in) {
    v = make_uint4(0, 0, 0, 0);
    if (in && k + 8 * h < end) v = *reinterpret_cast<const uint4*>(row + k + 8 * h);
  }
  static __device__ __forceinline__ void multiply(float16v& acc, const Frag& a, const Frag& b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(vec, a.v), __builtin_bit_cast(vec, b.v), acc, 0, 0, 0);
  }
};
template <> struct Frag<float> {                           // 8 a step, 4 and 4
  static constexpr int STEP = 8;
  float4 v;
  __device__ __forceinline__ void load(const float* row, int k, int h, int end, bool in) {
    v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (in && k < end) v = *reinterpret_cast<const float4*>(row + k + 4 * h);
  }
  static __device__ __forceinline__ void multiply(float16v& acc, const Frag& a, const Frag& b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v.x, b.v.x, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v.y, b.v.y, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v.z, b.v.z, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v.w, b.v.w, acc, 0, 0, 0);
  }
};
template <typename T>
__global__ __launch_bounds__(NTHR) void small_logits_kernel(CeArgs a, int keep) {
  constexpr int STEP = Frag<T>::STEP, U = 4;
  __shared__ float part[4][BLOCK_V][33];
  __shared__ float sm[NTHR], sl[NTHR];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, h = lane >> 5;
  const long v0 = (long)blockIdx.x * BLOCK_V, n0 = (long)blockIdx.y * 32;
  const long va = v0 + r < a.c.vocab ? v0 + r : a.c.vocab - 1, vb = v0 + 32 + r < a.c.vocab ? v0 + 32 + r : a.c.vocab - 1;
  const T* wa = reinterpret_cast<const T*>(a.c.weight.p) + va * a.c.weight.row;
  const T* wb = reinterpret_cast<const T*>(a.c.weight.p) + vb * a.c.weight.row;
  const int t = target_of(a, n0 + r);
  const T* x = reinterpret_cast<const T*>(a.c.x.p) + (t >= 0 ? n0 + r : 0) * a.c.x.row;
  const int quarter = (a.c.width + 4 * STEP - 1) / (4 * STEP) * STEP;
  const int k0 = wave * quarter, end = k0 + quarter < a.c.width ? k0 + quarter : a.c.width;
  float16v acc0, acc1;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc0[i] = acc1[i] = 0.f;
  for (int k = k0; k < end; k += U * STEP) {
    Frag<T> fa[U], fb[U], fx[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      fa[u].load(wa, k + u * STEP, h, end, true);
      fb[u].load(wb, k + u * STEP, h, end, true);
      fx[u].load(x, k + u * STEP, h, end, t >= 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Frag<T>::multiply(acc0, fa[u], fx[u]);
      Frag<T>::multiply(acc1, fb[u], fx[u]);
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {                           // (the layout of a 32 x 32 result)
    const int row = 8 * (i / 4) + 4 * h + i % 4;
    part[wave][row][r] = acc0[i];
    part[wave][32 + row][r] = acc1[i];
  }
  __syncthreads();
  const int col = tid & 31, p8 = tid >> 5;
  const long n = n0 + col;
  const int tc = target_of(a, n);
  if (blockIdx.x == 0 && p8 == 0 && n < a.p.np) a.p.target[n] = tc;
  float v[BLOCK_V / 8];
#pragma unroll
  for (int j = 0; j < BLOCK_V / 8; ++j) {
    const int row = p8 + 8 * j;
    const float s = (part[0][row][col] + part[1][row][col]) + (part[2][row][col] + part[3][row][col]);
    const bool in = v0 + row < a.c.vocab;
    v[j] = in ? s : -INFINITY;
    if (in && n < a.p.np) {
      if (keep) a.p.logits[(v0 + row) * a.p.np + n] = s;
      if (tc == v0 + row) a.p.target_logit[n] = v[j];
    }
  }
  Running run = {-INFINITY, 0.f};
  run.add(v, a.to_log2);
  run = meet<32>(run, a.to_log2, sm, sl);
  if (p8 == 0 && n < a.p.np) a.p.sums[(long)blockIdx.x * a.p.np + n] = make_float2(run.m, run.l);
}

// The targets' logits where the others meet no memory: a wavefront takes 32 rows of x and their targets' rows of the weights, and of its 32 x 32 products
// keeps the diagonal.  Same instruction, same order along the channels: bit by bit the logits that the 256 x 256 kernel's epilogues see, so that where a
// target holds next to all of a row's mass its logit cancels against the sum's.  (A sum in another order, as a plain dot product is, leaves a
// rounding of the logit's size in the loss and in the target's coefficient, however small these are: fp32 dx, where the same was so, of 30000 rows against
// 1000 x 1000 3.7e-6 instead of 9.3e-7 off in relative L2.)  What bounds it is the wait for each row's channels in turn: 16384 rows of 2048 39 us, 32768 of 256 8.
__global__ __launch_bounds__(NTHR) void target_kernel(CeArgs a) {
  constexpr int STEP = Frag<bf16_t>::STEP, U = 4;
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const long n = ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) * 32 + r;
  if (n - r >= a.p.np) return;                             // (np: whole tiles of 256)
  const int t = a.p.target[n];
  const bool in = t >= 0 && t < a.p.fused;
  const bf16_t* w = a.p.weight ? reinterpret_cast<const bf16_t*>(a.p.weight) + (in ? t : 0l) * a.p.wp
                               : reinterpret_cast<const bf16_t*>(a.c.weight.p) + (in ? t : 0l) * a.c.weight.row;
  const bf16_t* x = reinterpret_cast<const bf16_t*>(a.p.x) + n * a.p.wp;
  float16v acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  for (int k = 0; k < a.p.wp; k += U * STEP) {             // (zeros behind the last channel change no sum)
    Frag<bf16_t> fw[U], fx[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      fw[u].load(w, k + u * STEP, h, a.p.wp, in);
      fx[u].load(x, k + u * STEP, h, a.p.wp, in);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) Frag<bf16_t>::multiply(acc, fw[u], fx[u]);
  }
  float own = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) own = 8 * (i / 4) + 4 * h + i % 4 == r ? acc[i] : own;
  if (in && ((r >> 2) & 1) == h) a.p.target_logit[n] = own;
}

// all blocks of TB rows from n0 on by NT threads, and their losses
template <int TB, int NT>
__device__ __forceinline__ void row_losses(const CeArgs& a, long n0, float (&sm)[NT], float (&sl)[NT]) {
  constexpr int PARTS = NT / TB, K = 8;
  const int row = threadIdx.x % TB, part = threadIdx.x / TB;
  const long n = n0 + row, nc = n < a.p.np ? n : a.p.np - 1;
  Running r = {-INFINITY, 0.f};
  for (int b = part; b < a.p.blocks; b += K * PARTS) {
    float2 f[K];
    float v[K], w[K];
#pragma unroll
    for (int j = 0; j < K; ++j)
      f[j] = b + j * PARTS < a.p.blocks ? a.p.sums[(long)(b + j * PARTS) * a.p.np + nc] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int j = 0; j < K; ++j) { v[j] = f[j].x; w[j] = f[j].y; }
    r.add(v, w, a.to_log2);
  }
  r = meet<TB>(r, a.to_log2, sm, sl);
  if (part != 0 || n >= a.p.np) return;
  const bool counts = a.p.target[n] >= 0;
  const float log2_l = __builtin_amdgcn_logf(r.l);
  float loss = counts ? fmaf(a.c.scale, r.m - a.p.target_logit[n], log2_l * LN2) : 0.f;
  if (loss < 0.f) loss = 0.f;                              // (a sum that is 1 may come out as 1 less a rounding; NaNs stay)
  a.p.lse[n] = counts ? fmaf(r.m, a.to_log2, log2_l) : INFINITY;
  a.p.at_target[n] = counts ? expm1f(-loss) : 0.f;
  a.p.rows[n] = loss;
  if (a.c.row_loss && n < a.c.rows) a.c.row_loss[n] = loss;
}
// the loss, and what dS is multiplied by: one workgroup, sums in 64 bits in a fixed order
__device__ __forceinline__ void whole_loss(const CeArgs& a, double (&sum)[1024], int (&cnt)[1024]) {
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
    // Most targets' coefficients are next to minus the factor, so that its own rounding would be all of theirs: up to 2^-8 of dweight.
    const double g = f * a.c.scale;
    int e = 0;
    const double m = frexp(g, &e);
    const bool apart = a.power && g != 0.0 && e > -100 && e < 100;
    a.p.scalars[0] = (float)(apart ? ldexp(1.0, e - 1) : g);
    a.p.scalars[AFTER] = apart ? (float)(2.0 * m) : 1.f;
  }
}
template <int TB>
__global__ __launch_bounds__(NTHR) void row_loss_kernel(CeArgs a) {
  __shared__ float sm[NTHR], sl[NTHR];
  row_losses<TB>(a, (long)TB * blockIdx.x, sm, sl);
}
__global__ __launch_bounds__(1024) void loss_kernel(CeArgs a) {
  __shared__ double sum[1024];
  __shared__ int cnt[1024];
  whole_loss(a, sum, cnt);
}
// few rows: both in one workgroup
__global__ __launch_bounds__(1024) void few_loss_kernel(CeArgs a) {
  __shared__ float sm[1024], sl[1024];
  __shared__ double sum[1024];
  __shared__ int cnt[1024];
  if (a.p.np <= 32)
    for (long n0 = 0; n0 < a.p.np; n0 += 8) row_losses<8>(a, n0, sm, sl);
  else
    for (long n0 = 0; n0 < a.p.np; n0 += 32) row_losses<32>(a, n0, sm, sl);
  __syncthreads();                                         // (the rows' losses, written above, are read below by other threads)
  whole_loss(a, sum, cnt);
}

__device__ __forceinline__ float bf16_of(float v) { return __uint_as_float(pack_bf16x2(0.f, v) & 0xFFFF0000u); }
// dS of a piece: 8 rows of x and GRAD_V rows of the vocabulary a thread, whose logits go out together.  (Four: 1000 rows against 32000 x 256 fp32, all
// in all, 664 us, one 703; a small problem, which needs the threads, 35.1 and 33.2.)
template <typename T, int GRAD_V>
__global__ __launch_bounds__(NTHR) void grad_kernel(CeArgs a, Divisor by_row) {
  if (blockIdx.x >= a.grad_blocks) {
    const long n = (long)(blockIdx.x - a.grad_blocks) * 4 + (threadIdx.x >> 6);
    if (n < a.p.np) copy_row<T>(a, n, threadIdx.x & 63, a.p.target[n] >= 0);
    return;
  }
  const unsigned per = by_row.d;
  const long base = (long)blockIdx.x * NTHR, row0 = base / per;
  const unsigned r = (unsigned)(base - row0 * per) + threadIdx.x, q = by_row.quotient(r);
  const long v = GRAD_V * (row0 + q), n = 8l * (r - q * per);
  if (v >= a.nv) return;
  Raw8<float> raw[GRAD_V];
#pragma unroll
  for (int i = 0; i < GRAD_V; ++i)
    if (v + i < a.nv) raw[i].load(a.p.logits + (v + i) * a.p.np + n);
  float lse[8];
  load8(a.p.lse + n, lse);
  const int4 t0 = *reinterpret_cast<const int4*>(a.p.target + n), t1 = *reinterpret_cast<const int4*>(a.p.target + n + 4);
  const int target[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
  const float g = a.p.scalars[0];
#pragma unroll
  for (int i = 0; i < GRAD_V; ++i) {
    if (v + i >= a.nv) continue;
    float s[8];
    raw[i].unpack(s);
    bool hit = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[j] = lse[j] == INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(s[j], a.to_log2, -lse[j])) * g;
      hit = hit || target[j] == a.v0 + v + i;
    }
    if (hit) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (target[j] == a.v0 + v + i) s[j] = a.p.at_target[n + j] * g;
    }
    T* to = reinterpret_cast<T*>(a.p.grad) + (a.grad0 + v + i) * a.p.gp + n;
    store8(to, s);
    if constexpr (sizeof(T) == 2)
      if (a.p.gp > a.p.np) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] -= bf16_of(s[j]);
        store8(to + a.p.np, s);
      }
  }
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
    const bool twice = a.p.gp > a.p.np;
#pragma unroll 4
    for (int k = 0; k < (twice ? 2 * shares : shares); ++k) {          // (two terms: 2 np rows a share, row n of either)
      float v[8];
      load8(a.p.dx + ((long)k * a.p.np + n) * a.p.wp + c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += v[j];
    }
    if constexpr (sizeof(T) == 2) {      // a confident row's dx is next to its target's coefficient times a row of the weights: what
      const float g = a.p.at_target[n] * a.p.scalars[0], rest = twice ? 0.f : g - bf16_of(g);   // its rounding left out
      float w[8];
      load8(reinterpret_cast<const T*>(a.c.weight.p) + (long)a.p.target[n] * a.c.weight.row + c, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = fmaf(rest, w[j], s[j]);
      const float f = a.p.scalars[AFTER];
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] *= f;
    }
  }
  store8(reinterpret_cast<T*>(a.c.dx.p) + n * a.c.dx.row + c, s);
}
// rows of dweight from their shares, n8 elements of 8
template <typename O>
__global__ __launch_bounds__(NTHR) void dweight_kernel(const float* part, O* out, long row, long n8, int shares, Divisor by_row, const float* scale) {
  const unsigned per = by_row.d;
  const long base = (long)blockIdx.x * NTHR, i = base + threadIdx.x, row0 = base / per;
  if (i >= n8) return;
  const unsigned r = (unsigned)(base - row0 * per) + threadIdx.x, q = by_row.quotient(r);
  float s[8];
  load8(part + 8 * i, s);
#pragma unroll 4
  for (int k = 1; k < shares; ++k) {
    float v[8];
    load8(part + 8 * (k * n8 + i), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] += v[j];
  }
  const float f = *scale;
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] *= f;
  store8(out + (row0 + q) * row + 8l * (r - q * per), s);
}
template <typename T>
__global__ __launch_bounds__(NTHR) void clear_kernel(T* p, long row, long rows, int width) {
  const long per = width / 8;
  const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (long i = (long)blockIdx.x * NTHR + threadIdx.x; i < rows * per; i += (long)gridDim.x * NTHR) store8(p + i / per * row + 8 * (i % per), z);
}

// ---- sizes -----------------------------------------------------------------------------------------------------------
// Rows and blocks whose losses and their sum are one workgroup's (8 rows of 782 blocks 5.7 us; 104 of 625 took it 16.6, with a workgroup for 8 rows
// and another for the sum 8).
constexpr long FEW_ROWS = 128, FEW_SUMS = 8192;
// small_logits_kernel's share: a product of its own and a launch for the sums cost more than its plain loads do up to a million logits of
// 512 channels.  Measured, us, the loss alone, this kernel / without: 64 rows against 16384 x 256 14.1 / 21.9, 1000 against 1000 x 256 13.4 /
// 20.4, 8 against 50000 x 1024 32.6 / 34.3, 32 (fp32) 88 / 119; beyond the lines: 100 against 10000 x 1024 34.8 / 31.3.
bool small_problem(const Parts& p, long vocab, int width) {
  return !p.fused && p.pieces == 1 && (p.np <= 32 || (p.np * vocab <= (1l << 20) && width <= 512));
}
// A piece of the vocabulary takes 1 GB of logits, or of dS where the logits are not written.  Measured, us, with gradients, 1 GB / 512 / 256 / 128
// MB: 32768 rows against 16384 x 256 1220 / 1450 / 1655 / 1889 (with its embedding), 8190 against 50021 x 1024 2818 / 2894 / 2985 / 3231, 16384 against
// 131072 x 2048 26830 / 27266 / 27659 / 29512: smaller pieces stay in the caches, but dx meets memory once a piece and launches end more often.
constexpr size_t PIECE_BYTES = 1ul << 30;
constexpr long PIECE_ROWS = 1l << 20;
constexpr int MAX_SPLIT = 16;
// bf16 of up to so many rows, their logits in memory: dS keeps two terms, what its rounding leaves out rounded in turn, side by side in one product
// each.  A row of dweight is the sum of few coefficients then, down to one, and would take over their roundings whole.  Relative L2 of dweight in bf16, of
// which 0.0017 is the result's own rounding, with two terms / one: 1 row against 50 x 64 0.0018 / 0.0034, 5 against 70 x 2048 0.0017 / 0.0028, 100 against
// 30000 x 264 0.0017 / 0.0020; beyond, 130 against 700 x 1024 - / 0.0021, 4000 against 256 x 1024 - / 0.0019.  Time, us: 64 against 5000 x 256 31.3 / 28.5, 32
// against 131072 x 2048 383 / 367, 100 against 131072 x 1024 346 / 329.
constexpr long TWO_TERMS = 128;

// Channels are filled up with zeros to a multiple of 32, and to one of 256 where that is an eighth more at most, for the sake of the
// 256 x 256 kernel; the weights are copied for it, which takes as long as one of the four products with 500 rows of x.
int padded_width(int width) {
  const int whole = (width + 255) / 256 * 256;
  if (whole <= width + width / 8) return whole;
  return width < 128 ? 128 : (width + 31) / 32 * 32;
}
// Rows of the vocabulary that the 256 x 256 kernel's own epilogues take: all whole tiles, where those fill the chip.
long fused_rows(int dtype, long np, long vocab) {
  if (dtype != 1 || np % 256 || np == 0) return 0;
  const long tiles = vocab / 256 * (np / 256);
  return gemm_fills_chip(tiles) && tiles < (1l << 28) ? vocab / 256 * 256 : 0;
}
// Rows of x are filled up with zeros, fp32 to a multiple of 8, bf16 to whole tiles of 256 where that is an eighth more at most, or three eighths and those epilogues then
// take the logits, else to 8.  Measured, us, with gradients, tiles / 8: 600 rows (768) against 40000 x 256 134 / 191, 100000 x 1024 617 / 830; 200
// (256) 84 / 101 and 298 / 346, against 40000 x 1024 161 / 154; beyond the line, 300 (512) against 40000 x 1024 229 / 192, 100 against 40000 x 1024
// 153 / 123.
long padded(int dtype, long rows, long vocab) {
  const long whole = (rows + 255) / 256 * 256;
  if (dtype == 1 && (whole <= rows + rows / 8 || (whole <= rows + rows * 3 / 8 && fused_rows(dtype, whole, vocab)))) return whole;
  return (rows + 7) / 8 * 8;
}
// A product of few tiles and a long contraction (dx: over the vocabulary, dweight: over the rows of x) is shared out until there is a tile for
// every compute unit, in MAX_SPLIT shares at most.  rows, cols: of its result; wide: the 256 x 256 kernel would take it.
int shares_of(int dtype, long rows, long cols, long k, bool wide) {
  const long t = dtype == 0 ? 64 : wide ? 256 : 128;
  const long tiles = (rows + t - 1) / t * ((cols + t - 1) / t);
  if (dtype != 0 && gemm_fills_chip(tiles)) return 1;
  // (fp32: 512 tiles, from where on they are the 64-wide ones)
  long n = dtype == 0 ? (511 + tiles) / tiles : 256 / tiles;
  if (n > MAX_SPLIT) n = MAX_SPLIT;
  // (at least 512 of the contraction: 512 rows of x against 2000 x 1024 59 us, with 256 72; 4096 against 8000 x 512 210, with 2048 218)
  if (n > k / 512) n = k / 512;
  // fp32 takes shares of 8192 at most, as many as that makes (up to 128; a piece's rows and columns are fewer then): it halves the error of sums over
  // 30000 (1000 x 1000 over 30000 756 us, in one share 881)
  if (dtype == 0 && n < (k + 8191) / 8192) n = (k + 8191) / 8192;
  return (int)(n < 1 ? 1 : n);
}
// Does the 256 x 256 kernel take whole tiles of such a product, in shares where it needs them?  (Else nothing is gained by keeping its
// rows, columns or contraction apart from the rest.)
bool wide(long rows, long cols, long k) {
  const long tiles = rows / 256 * (cols / 256);
  return tiles > 0 && gemm_fills_chip(tiles * shares_of(1, rows, cols / 256 * 256, k, true));
}
bool dx_wide(int dtype, long np, int wp, long nv) { return dtype == 1 && np % 256 == 0 && wide(np, wp, nv); }
int dx_split(int dtype, long np, int wp, long nv) {
  const bool w = dx_wide(dtype, np, wp, nv);
  return shares_of(dtype, np, w ? wp / 256 * 256 : wp, nv, w);
}
// dx of nv rows of the vocabulary: one product, or whole slices of 32 and the rest in one share (a contraction that is no multiple of 32 keeps the
// 256 x 256 kernel from all of it)
struct DxParts { long whole; int split, rest; };
DxParts dx_parts(int dtype, long np, int wp, long nv) {
  const long whole = nv / 32 * 32;
  if (whole > 0 && whole < nv && dx_wide(dtype, np, wp, whole)) return {whole, dx_split(dtype, np, wp, whole), 1};
  return {nv, dx_split(dtype, np, wp, nv), 0};
}
bool dweight_wide(int dtype, long np, int width, long nv) { return dtype == 1 && np % 32 == 0 && nv % 256 == 0 && wide(nv, width, np); }
int dweight_split(int dtype, long np, int width, long nv) {
  const bool w = dweight_wide(dtype, np, width, nv);
  return shares_of(dtype, nv, w ? width / 256 * 256 : width, np, w);
}
// How many of the next nv rows of the vocabulary have their dweight in one product: whole tiles of 256 (rows behind them would take all others to
// smaller tiles), and of those whole rounds of the compute units where little of another would be filled and a round is long.  Measured,
// with all else, us, so / all tiles together: 8190 rows of x against 50021 x 1024 (780 tiles) 2754 / 2858, 8192 against 20000 x 1024 1159 / 1234, 4096
// against 50000 x 1024 1445 / 1488; below the line 1024 against 70000 x 512 376 / 352.
long dweight_rows_of(int dtype, long np, int width, long nv) {
  if (!dweight_wide(dtype, np, width, nv / 256 * 256)) return nv;
  const long per = width / 256, tiles = nv / 256 * per, over = tiles % 256;
  const long take = np >= 4096 && tiles > 256 && over > 0 && over * 100 < 256 * 35 ? (tiles - over) / per : nv / 256;
  return take * 256;
}
size_t dweight_part(int dtype, long np, int width, long nv) {      // bytes of the shares of nv rows in one product
  const int n = dweight_split(dtype, np, width, nv);
  return n > 1 ? (size_t)n * nv * width * 4 : 0;
}
size_t dweight_room(int dtype, long np, int width, long nv) {      // ... and of a piece's products, one after the other
  size_t most = 0;
  for (long n; nv > 0; nv -= n) {
    n = dweight_rows_of(dtype, np, width, nv);
    const size_t b = dweight_part(dtype, np, width, n);
    most = b > most ? b : most;
  }
  return most;
}

Parts carve(char* base, int dtype, long rows, long vocab, int width, bool gradients) {
  Parts p{};
  size_t off = 0;
  auto take = [&](size_t n) { char* q = base ? base + off : nullptr; off += (n + 255) / 256 * 256; return q; };
  const size_t es = dtype == 0 ? 4 : 2;
  p.np = padded(dtype, rows, vocab);
  p.fused = fused_rows(dtype, p.np, vocab);
  p.wp = p.fused ? padded_width(width) : width;
  const size_t row = (p.fused ? 2 : 4) * (p.np ? p.np : 1);
  constexpr long TILE = 256;
  const long fit = (long)(PIECE_BYTES / row) / TILE * TILE;
  const long most = fit < TILE ? TILE : fit < PIECE_ROWS ? fit : PIECE_ROWS;
  p.pieces = (int)((vocab + most - 1) / most);             // of one size, as near as whole tiles allow
  p.piece = ((vocab + p.pieces - 1) / p.pieces + TILE - 1) / TILE * TILE;
  p.pieces = (int)((vocab + p.piece - 1) / p.piece);
  if (p.piece > vocab) p.piece = vocab;
  p.blocks = p.fused ? (int)(p.fused / 128 + (vocab - p.fused + BLOCK_V - 1) / BLOCK_V) : (int)((vocab + BLOCK_V - 1) / BLOCK_V);
  p.gp = gradients && dtype == 1 && !p.fused && p.np <= TWO_TERMS ? 2 * p.np : p.np;
  p.x = take(p.gp * p.wp * es);
  if (p.wp != width) p.weight = take((size_t)vocab * p.wp * es);
  p.target_logit = reinterpret_cast<float*>(take(4 * p.np));
  p.lse = reinterpret_cast<float*>(take(4 * p.np));
  p.target = reinterpret_cast<int*>(take(4 * p.np));
  p.rows = reinterpret_cast<float*>(take(4 * p.np));
  p.at_target = reinterpret_cast<float*>(take(4 * p.np));
  p.scalars = reinterpret_cast<float*>(take(4 * (AFTER + 1)));
  p.sums = reinterpret_cast<float2*>(take((size_t)p.blocks * p.np * 8));
  p.logits = reinterpret_cast<float*>(take((size_t)(p.fused ? vocab - p.fused : p.piece) * p.np * 4));
  p.grad = p.logits;
  if (gradients) {
    if (dtype == 1) p.grad = take((size_t)p.piece * p.gp * 2);
    // as many as there are, and of many pieces the largest product's, what was added up before it, and a rest, four at least
    const long last_piece = vocab - (p.pieces - 1) * p.piece;
    const DxParts each = dx_parts(dtype, p.gp ? p.gp : 8, p.wp, p.piece), end = dx_parts(dtype, p.gp ? p.gp : 8, p.wp, last_piece);
    const long all = (p.pieces - 1l) * (each.split + each.rest) + end.split + end.rest, split = each.split > end.split ? each.split : end.split;
    const long room = split + 2 < 4 ? 4 : split + 2;
    p.shares = (int)(all < room ? all : room);
    p.dx = reinterpret_cast<float*>(take((size_t)p.shares * p.gp * p.wp * 4));
    const size_t most = dweight_room(dtype, p.gp, width, p.piece), last = dweight_room(dtype, p.gp, width, last_piece);
    p.dweight_bytes = most > last ? most : last;
    p.dweight = reinterpret_cast<float*>(take(p.dweight_bytes));
  }
  p.bytes = off;
  return p;
}

// Have all products of the gradients their room?  Goes through them as the launches do (Run::dweight, Run::dx), and is asked before the first.
bool fits(const Parts& p, int dtype, long vocab, int width) {
  int shares = 0;
  for (int i = 0; i < p.pieces; ++i) {
    const long v0 = i * p.piece, nv = vocab - v0 < p.piece ? vocab - v0 : p.piece;
    for (long r = 0, n; r < nv; r += n) {
      n = dweight_rows_of(dtype, p.gp, width, nv - r);
      if (dweight_part(dtype, p.gp, width, n) > p.dweight_bytes) return false;
    }
    const DxParts d = dx_parts(dtype, p.gp, p.wp, nv);
    for (const int k : {d.split, d.rest}) {
      if (shares + k > p.shares) shares = 1;               // (Run::fold)
      if (shares + k > p.shares) return false;
      shares += k;
    }
  }
  return true;
}

hipError_t product(int dtype, const GemmArgs& g, hipStream_t s) {
  if (dtype == 1) {
    hipError_t e;
    if (launch_gemm_mfma(g, s, &e)) return e;
    if (g.mode == EPI_SCALED) return hipErrorInvalidValue;
  } else if (gemm_f32_ok(g)) {
    return launch_gemm_f32(g, s);
  }
  return launch_gemm_generic(dtype, g, s);
}
GemmArgs plain() {
  GemmArgs g{};
  g.batch = 1; g.split_k = 1; g.mode = EPI_STORE;
  return g;
}

#define CE_TRY(call)                      \
  do {                                    \
    const hipError_t e_ = (call);         \
    if (e_ != hipSuccess) return e_;      \
  } while (0)

template <typename T>
struct Run {
  static constexpr int DTYPE = sizeof(T) == 4 ? 0 : 1;
  const CrossEntropyArgs& c;
  const Parts& p;
  hipStream_t s;
  CeArgs a;
  int shares = 0;
  bool small;
  Run(const CrossEntropyArgs& c_, const Parts& p_, hipStream_t s_) : c(c_), p(p_), s(s_), a{}, small(small_problem(p_, c_.vocab, c_.width)) {
    a.c = c;
    a.p = p;
    a.to_log2 = c.scale * LOG2E;
    a.power = DTYPE == 1;
  }

  // the weights' rows from v0 on as the products read them
  long weight_row() const { return p.weight ? p.wp : c.weight.row; }
  const T* weight_at(long v0) const { return reinterpret_cast<const T*>(p.weight ? p.weight : c.weight.p) + v0 * weight_row(); }
  GemmArgs logits_args(long v0, long nv) const {
    GemmArgs g = plain();
    g.A = weight_at(v0); g.a_sm = weight_row(); g.a_sk = 1;
    g.B = p.x; g.b_sn = p.wp; g.b_sk = 1;
    g.ldc = p.np;
    g.M = nv; g.N = p.np; g.K = p.wp;
    return g;
  }
  // a product whose columns are the channels: whole tiles of 256 of them apart from the rest, on the 256 x 256 kernel
  hipError_t by_columns(GemmArgs g, bool apart) const {
    const long whole = apart ? g.N / 256 * 256 : 0, rest = g.N - whole;
    if (whole == 0 || rest == 0) return product(DTYPE, g, s);
    g.N = whole;
    CE_TRY(product(DTYPE, g, s));
    g.N = rest;
    g.B = reinterpret_cast<const T*>(g.B) + whole;
    if (g.c_is_f32) g.C = reinterpret_cast<float*>(g.C) + whole;
    else g.C = reinterpret_cast<T*>(g.C) + whole;
    return product(DTYPE, g, s);
  }
  void at(long v0, long nv) { a.v0 = v0; a.nv = nv; a.grad0 = 0; }
  hipError_t logits() {
    GemmArgs g = logits_args(a.v0, a.nv);
    g.C = p.logits; g.c_is_f32 = 1;
    return product(DTYPE, g, s);
  }
  hipError_t block_sums(long block0) {
    a.block0 = block0;
    const unsigned nb = (unsigned)((a.nv + BLOCK_V - 1) / BLOCK_V);
    if (p.np >= 32) block_sums_kernel<32><<<dim3((unsigned)((p.np + 31) / 32), nb), NTHR, 0, s>>>(a);
    else block_sums_kernel<8><<<dim3((unsigned)(p.np / 8), nb), NTHR, 0, s>>>(a);
    return hipGetLastError();
  }
  hipError_t softmax_grad() {
    const int rows = small ? 1 : 4;
    const Divisor per((unsigned)(p.np / 8));
    a.grad_blocks = (unsigned)(((a.nv + rows - 1) / rows * (p.np / 8) + NTHR - 1) / NTHR);
    if (small) grad_kernel<T, 1><<<a.grad_blocks + (unsigned)((p.np + 3) / 4), NTHR, 0, s>>>(a, per);
    else grad_kernel<T, 4><<<a.grad_blocks, NTHR, 0, s>>>(a, per);
    return hipGetLastError();
  }
  hipError_t fold() {
    const long n8 = p.gp * p.wp / 8;
    fold_kernel<<<(unsigned)((n8 + NTHR - 1) / NTHR), NTHR, 0, s>>>(p.dx, n8, shares);
    shares = 1;
    return hipGetLastError();
  }

  hipError_t sums() {
    if (p.fused) {
      GemmArgs g = logits_args(0, p.fused);
      g.C = p.sums; g.mode = EPI_VOCAB_SUMS; g.vocab.alpha = a.to_log2;
      CE_TRY(launch_gemm_vocab(g, s));
      target_kernel<<<(unsigned)((p.np + 127) / 128), NTHR, 0, s>>>(a);
      CE_TRY(hipGetLastError());
      if (p.fused == c.vocab) return hipSuccess;
      at(p.fused, c.vocab - p.fused);
      CE_TRY(logits());
      return block_sums(p.fused / 128);
    }
    for (int i = 0; i < p.pieces; ++i) {
      at(i * p.piece, c.vocab - i * p.piece < p.piece ? c.vocab - i * p.piece : p.piece);
      CE_TRY(logits());
      CE_TRY(block_sums(a.v0 / BLOCK_V));
    }
    return hipSuccess;
  }
  // dS of rows v0 .. v0 + nv of the vocabulary; the last ones, and with one piece all of them, have their logits in memory
  hipError_t piece_grad(long v0, long nv) {
    at(v0, nv);
    if (!p.fused) {
      if (p.pieces > 1) CE_TRY(logits());
      return softmax_grad();
    }
    const long nf = v0 + nv < p.fused ? nv : p.fused > v0 ? p.fused - v0 : 0;
    if (nf > 0) {
      GemmArgs g = logits_args(v0, nf);
      g.C = p.grad; g.mode = EPI_VOCAB_GRAD;
      g.vocab = {a.to_log2, p.lse, p.target, p.at_target, p.scalars, v0};
      CE_TRY(launch_gemm_vocab(g, s));
    }
    if (nf == nv) return hipSuccess;
    at(v0 + nf, nv - nf);
    a.grad0 = nf;
    return softmax_grad();
  }
  hipError_t dweight_rows(long v0, long r0, long nr) {
    const int n = dweight_split(DTYPE, p.gp, c.width, nr);
    GemmArgs g = plain();
    g.A = reinterpret_cast<const T*>(p.grad) + r0 * p.gp; g.a_sm = p.gp; g.a_sk = 1;
    g.B = p.x; g.b_sk = p.wp; g.b_sn = 1;
    g.M = nr; g.N = c.width; g.K = p.gp;
    const long o = (v0 + r0) * c.dweight.row;
    float* f = reinterpret_cast<float*>(c.dweight.p) + o;
    bf16_t* b = reinterpret_cast<bf16_t*>(c.dweight.p) + o;
    if (n == 1) {
      g.c_is_f32 = c.grad_dtype == 0;
      if (g.c_is_f32) g.C = f; else g.C = b;
      g.ldc = c.dweight.row;
      if (DTYPE == 1) { g.mode = EPI_SCALED; g.lambda = p.scalars + AFTER; }
      return by_columns(g, dweight_wide(DTYPE, p.gp, c.width, nr));
    }
    g.c_is_f32 = 1; g.C = p.dweight; g.ldc = c.width; g.c_sb = nr * c.width; g.split_k = n;
    CE_TRY(by_columns(g, dweight_wide(DTYPE, p.gp, c.width, nr)));
    const long n8 = nr * c.width / 8;
    const unsigned blocks = (unsigned)((n8 + NTHR - 1) / NTHR);
    const Divisor per((unsigned)(c.width / 8));
    if (c.grad_dtype == 0) dweight_kernel<float><<<blocks, NTHR, 0, s>>>(p.dweight, f, c.dweight.row, n8, n, per, p.scalars + AFTER);
    else dweight_kernel<bf16_t><<<blocks, NTHR, 0, s>>>(p.dweight, b, c.dweight.row, n8, n, per, p.scalars + AFTER);
    return hipGetLastError();
  }
  hipError_t dweight(long v0, long nv) {
    for (long r = 0, n; r < nv; r += n) {
      n = dweight_rows_of(DTYPE, p.gp, c.width, nv - r);
      CE_TRY(dweight_rows(v0, r, n));
    }
    return hipSuccess;
  }
  hipError_t dx_rows(long v0, long r0, long nr, int split) {
    GemmArgs g = plain();
    g.A = reinterpret_cast<const T*>(p.grad) + r0 * p.gp; g.a_sm = 1; g.a_sk = p.gp;
    g.B = weight_at(v0 + r0); g.b_sk = weight_row(); g.b_sn = 1;
    if (shares + split > p.shares) CE_TRY(fold());
    g.C = p.dx + (long)shares * p.gp * p.wp; g.ldc = p.wp; g.c_is_f32 = 1;
    g.c_sb = p.gp * p.wp;
    g.split_k = split;
    shares += split;
    g.M = p.gp; g.N = p.wp; g.K = nr;
    return by_columns(g, dx_wide(DTYPE, p.gp, p.wp, nr));
  }
  hipError_t dx(long v0, long nv) {
    const DxParts d = dx_parts(DTYPE, p.gp, p.wp, nv);
    CE_TRY(dx_rows(v0, 0, d.whole, d.split));
    return d.rest ? dx_rows(v0, d.whole, nv - d.whole, d.rest) : hipSuccess;
  }

  hipError_t without_rows() {
    loss_kernel<<<1, 1024, 0, s>>>(a);
    if (c.dweight.p) {
      const long all = (c.vocab * (c.width / 8) + NTHR - 1) / NTHR;
      const unsigned blocks = all < 65536 ? (unsigned)all : 65536u;
      if (c.grad_dtype == 0) clear_kernel<float><<<blocks, NTHR, 0, s>>>(reinterpret_cast<float*>(c.dweight.p), c.dweight.row, c.vocab, c.width);
      else clear_kernel<bf16_t><<<blocks, NTHR, 0, s>>>(reinterpret_cast<bf16_t*>(c.dweight.p), c.dweight.row, c.vocab, c.width);
    }
    return hipGetLastError();
  }
  hipError_t all() {
    if (c.rows == 0) return without_rows();
    if (small) {
      const dim3 grid((unsigned)((c.vocab + BLOCK_V - 1) / BLOCK_V), (unsigned)((p.np + 31) / 32));
      small_logits_kernel<T><<<grid, NTHR, 0, s>>>(a, c.dx.p || c.dweight.p);
    } else {
      rows_kernel<T><<<(unsigned)((p.np + 3) / 4), NTHR, 0, s>>>(a);
    }
    if (p.weight) {
      const long all = (c.vocab * (p.wp / 8) + NTHR - 1) / NTHR;
      weight_kernel<<<all < 65536 ? (unsigned)all : 65536u, NTHR, 0, s>>>(a);
    }
    CE_TRY(hipGetLastError());
    if (!small) CE_TRY(sums());
    if (p.np <= FEW_ROWS && p.np * p.blocks <= FEW_SUMS) {
      few_loss_kernel<<<1, 1024, 0, s>>>(a);
    } else {
      if (p.np <= 2048) row_loss_kernel<8><<<(unsigned)(p.np / 8), NTHR, 0, s>>>(a);
      else row_loss_kernel<32><<<(unsigned)((p.np + 31) / 32), NTHR, 0, s>>>(a);
      loss_kernel<<<1, 1024, 0, s>>>(a);
    }
    CE_TRY(hipGetLastError());
    if (!c.dx.p && !c.dweight.p) return hipSuccess;
    for (int i = 0; i < p.pieces; ++i) {
      const long v0 = i * p.piece, nv = c.vocab - v0 < p.piece ? c.vocab - v0 : p.piece;
      CE_TRY(piece_grad(v0, nv));
      if (c.dweight.p) CE_TRY(dweight(v0, nv));
      if (c.dx.p) CE_TRY(dx(v0, nv));
    }
    if (c.dx.p) {
      const unsigned per = (unsigned)(c.width / 8);
      dx_kernel<T><<<(unsigned)((c.rows * per + NTHR - 1) / NTHR), NTHR, 0, s>>>(a, Divisor(per), shares);
      CE_TRY(hipGetLastError());
    }
    return hipSuccess;
  }
};

}  // namespace

size_t cross_entropy_ws_bytes(int dtype, long rows, long vocab, int width, bool gradients) {
  const Parts p = carve(nullptr, dtype, rows, vocab, width, gradients);
  return rows && gradients && !fits(p, dtype, vocab, width) ? 0 : p.bytes;
}

hipError_t launch_cross_entropy(int dtype, const CrossEntropyArgs& c, void* workspace, size_t bytes, hipStream_t s) {
  const Parts p = carve(reinterpret_cast<char*>(workspace), dtype, c.rows, c.vocab, c.width, c.dx.p || c.dweight.p);
  if (bytes < p.bytes || (c.rows && (c.dx.p || c.dweight.p) && !fits(p, dtype, c.vocab, c.width))) return hipErrorInvalidValue;
  return dtype == 0 ? Run<float>(c, p, s).all() : Run<bf16_t>(c, p, s).all();
}

}  // namespace hbp
