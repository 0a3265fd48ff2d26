// The embedding of a language model's tokens, its gradient, and dropout.
//
// All of it is bound by memory: a unit of 8 channels is read once and written once, one product an element, and with dropout ten
// rounds of two wide integer products a unit.  Calls, one after the other: dropout of 16384 x 2048 bf16 onto a residual 36.7 us with rows from memory
// (5.5 TB/s; a copy: 5.1), 28.3 with the same rows again and again, which the memory side's cache holds; the embedding of 32768 tokens in 256 channels
// with dropout 8.0 us; calls of a few rows 6.7, which is the host's share of a launch.
//
// The gradient adds up rows of the same token, in 32 bits and in an order that does not change from run to run, so without atomics on
// its sums.  Tokens are sorted (least significant digit first, up to 9 bits a pass, stable, so that a token's rows stay in order);
// then a table's row has its stretch of the sorted list, found by bisection, and one group of lanes adds it up.
// Text repeats few tokens very often: 16 sorted places that begin at a multiple of 16 and hold one token are added up beforehand by a
// workgroup of their own, and the table's row adds that sum.  A table's row is written once, rows without tokens as zeros: that is most
// of the bytes.
// Measured: 16384 tokens, a tenth of them none, into 131072 x 2048 a call of 251 us, its kernels 24 for the sort, 13 chunks, 213 the table (1.07 GB
// written, 5 TB/s); 32768 into 16384 x 256 with dropout a call of 44, its kernels (traced) 26, 7 and 16.
#include "philox.h"

namespace hbp {

namespace {

constexpr int NTHR = 256;

// ---- dropout and lookup: a unit of 8 channels a thread and step ----------------------------------------------------------
// Units are counted along the rows, which is also the generator's count.  A workgroup's first unit is divided once in 64 bits, a
// thread's place behind it by a multiplication.
struct Units {
  long total;
  Divisor by_row;
  unsigned per_row;
};
struct Place { long row; unsigned unit; };
__device__ __forceinline__ Place place_of(const Units& u, long row0, unsigned rem0, unsigned local) {
  const unsigned r = rem0 + local, q = u.by_row.quotient(r);
  return {row0 + q, r - q * u.per_row};
}
__device__ __forceinline__ void keep8(unsigned mask, float factor, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (mask >> j) & 1u ? v[j] * factor : 0.f;
}

// (Kernel times, the same rows again and again: one unit a thread 16384 x 2048 bf16 onto a residual 30.1 us, two 30.4, four 32.0; 65536 x 2048 without 90,
// 100, 100.)
template <typename T, bool RES>
__global__ __launch_bounds__(NTHR) void dropout_kernel(DropoutArgs a, DropoutKey key, Units u) {
  const long base = (long)blockIdx.x * NTHR;
  if (base + threadIdx.x >= u.total) return;
  const long row0 = base / u.per_row;
  const Place p = place_of(u, row0, (unsigned)(base - row0 * u.per_row), threadIdx.x);
  Raw8<T> vx, vr;
  vx.load(reinterpret_cast<const T*>(a.x.p) + p.row * a.x.row + 8 * p.unit);
  if (RES) vr.load(reinterpret_cast<const T*>(a.residual.p) + p.row * a.residual.row + 8 * p.unit);
  const unsigned mask = key.threshold ? dropout_mask8(key, dropout_stream(key), base + threadIdx.x) : 255u;
  float v[8];
  vx.unpack(v);
  keep8(mask, key.factor, v);
  if (RES) {
    float w[8];
    vr.unpack(w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += w[j];
  }
  store8(reinterpret_cast<T*>(a.out.p) + p.row * a.out.row + 8 * p.unit, v);
}

// K units a thread, 256 apart: their loads go out together
template <typename T, int K>
__global__ __launch_bounds__(NTHR) void lookup_kernel(EmbeddingArgs a, DropoutKey key, Units u) {
  const long base = (long)blockIdx.x * (NTHR * K);
  const long row0 = base / u.per_row;
  const unsigned rem0 = (unsigned)(base - row0 * u.per_row);
  const unsigned long stream = key.threshold ? dropout_stream(key) : 0;
  const T* table = reinterpret_cast<const T*>(a.table.p);
  T* y = reinterpret_cast<T*>(a.out.p);
  Place p[K];
  int token[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const unsigned local = threadIdx.x + NTHR * k;
    token[k] = -1;
    if (base + local >= u.total) continue;
    p[k] = place_of(u, row0, rem0, local);
    token[k] = a.tokens[p[k].row];
  }
  Raw8<T> v[K];
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (token[k] >= 0 && token[k] < a.vocab) v[k].load(table + (long)token[k] * a.table.row + 8 * p[k].unit);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const unsigned local = threadIdx.x + NTHR * k;
    if (base + local >= u.total) continue;
    float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (token[k] >= 0 && token[k] < a.vocab) {
      v[k].unpack(w);
      keep8(key.threshold ? dropout_mask8(key, stream, base + local) : 255u, key.factor, w);
    }
    store8(y + p[k].row * a.out.row + 8 * p[k].unit, w);
  }
}

Units units_of(long rows, int width) {
  const unsigned per = (unsigned)(width / 8);
  return {rows * per, Divisor(per), per};
}
unsigned blocks_of(const Units& u, int k) { return (unsigned)((u.total + NTHR * k - 1) / (NTHR * k)); }

template <typename T, bool RES>
hipError_t launch_dropout_t(const DropoutArgs& a, const DropoutKey& key, hipStream_t s) {
  const Units u = units_of(a.rows, a.width);
  dropout_kernel<T, RES><<<blocks_of(u, 1), NTHR, 0, s>>>(a, key, u);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_lookup_t(const EmbeddingArgs& a, const DropoutKey& key, hipStream_t s) {
  const Units u = units_of(a.rows, a.width);
  // Two units a thread from a million on (a token's row is asked for only once the token is there): 16384 x 2048 18.0 us, one 22.7, four 18.1;
  // with dropout 20.6, 21.6, 21.6.
  if (u.total >= 1l << 20) lookup_kernel<T, 2><<<blocks_of(u, 2), NTHR, 0, s>>>(a, key, u);
  else lookup_kernel<T, 1><<<blocks_of(u, 1), NTHR, 0, s>>>(a, key, u);
  return hipGetLastError();
}

// ---- the gradient: tokens sorted -----------------------------------------------------------------------------------------
constexpr int SORT_PER = 4, SORT_E = NTHR * SORT_PER;      // places of a workgroup
constexpr int SORT_BITS = 9, SORT_D = 1 << SORT_BITS;
constexpr int CHUNK = 16;                                  // sorted places added up beforehand where they hold one token

// What a place sorts by: its token, or `vocab` for a token that is none (behind all others).
__device__ __forceinline__ unsigned key_of(int token, unsigned vocab) { return (unsigned)token < vocab ? (unsigned)token : vocab; }

struct SortArgs {
  const int* tokens;          // first pass: keys are made from these, places are their own numbers
  const unsigned *keys_in, *places_in;
  unsigned *keys_out, *places_out;
  unsigned* counts;           // [blocks][SORT_D]: keys with each digit, after scan_kernel those in earlier blocks
  unsigned* totals;           // [SORT_D], after scan_kernel
  long n;
  unsigned vocab;
  int shift, mask, blocks, scanned;
};
__device__ __forceinline__ unsigned load_key(const SortArgs& a, long i) {
  return a.tokens ? key_of(a.tokens[i], a.vocab) : a.keys_in[i];
}

__global__ __launch_bounds__(NTHR) void count_kernel(SortArgs a) {
  __shared__ unsigned cnt[SORT_D];
  for (int d = threadIdx.x; d < SORT_D; d += NTHR) cnt[d] = 0;
  __syncthreads();
  const long base = (long)blockIdx.x * SORT_E;
#pragma unroll
  for (int k = 0; k < SORT_PER; ++k) {
    const long i = base + threadIdx.x + NTHR * k;
    if (i < a.n) atomicAdd(&cnt[(load_key(a, i) >> a.shift) & a.mask], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < SORT_D; d += NTHR) a.counts[(long)blockIdx.x * SORT_D + d] = cnt[d];
}

// many blocks: their counts of a digit become the number of such keys in earlier blocks; a thread a digit
__global__ __launch_bounds__(64) void scan_kernel(SortArgs a) {
  const int d = blockIdx.x * 64 + threadIdx.x;
  unsigned sum = 0;
  int b = 0;
  for (; b + 8 <= a.blocks; b += 8) {
    unsigned c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = a.counts[(long)(b + j) * SORT_D + d];
#pragma unroll
    for (int j = 0; j < 8; ++j) { a.counts[(long)(b + j) * SORT_D + d] = sum; sum += c[j]; }
  }
  for (; b < a.blocks; ++b) {
    const unsigned c = a.counts[(long)b * SORT_D + d];
    a.counts[(long)b * SORT_D + d] = sum;
    sum += c;
  }
  a.totals[d] = sum;
}

// Lanes whose digits agree find each other by a ballot a bit.
__device__ __forceinline__ unsigned long same_digit(unsigned d, int bits, bool in) {
  unsigned long peers = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const unsigned long has = __ballot((d >> b) & 1u);
    peers &= (d >> b) & 1u ? has : ~has;
  }
  return peers;
}

// Every wavefront owns 256 consecutive places in 4 steps of 64.
__global__ __launch_bounds__(NTHR) void place_kernel(SortArgs a) {
  __shared__ unsigned cnt[4][SORT_D];                      // a wavefront's keys with each digit, then where they go
  __shared__ unsigned sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long base = (long)blockIdx.x * SORT_E + wave * (64 * SORT_PER) + lane;
  unsigned key[SORT_PER], rank[SORT_PER];
#pragma unroll
  for (int k = 0; k < SORT_PER; ++k) key[k] = base + 64 * k < a.n ? load_key(a, base + 64 * k) : 0u;
  // where the first key of each digit goes, two digits a thread (asked for before the keys are looked at)
  const unsigned d0 = 2 * tid;
  unsigned total[2], before[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    total[j] = before[j] = 0;
    if (a.scanned) {
      total[j] = a.totals[d0 + j];
      before[j] = a.counts[(long)blockIdx.x * SORT_D + d0 + j];
    }
  }
  if (!a.scanned) {
    for (int b = 0; b < a.blocks; b += 16) {               // (the loads of 16 blocks go out together)
      uint2 c[16];
#pragma unroll
      for (int j = 0; j < 16; ++j)
        c[j] = b + j < a.blocks ? *reinterpret_cast<const uint2*>(a.counts + (long)(b + j) * SORT_D + d0) : make_uint2(0, 0);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        total[0] += c[j].x; total[1] += c[j].y;
        if (b + j < (int)blockIdx.x) { before[0] += c[j].x; before[1] += c[j].y; }
      }
    }
  }
  for (int d = tid; d < 4 * SORT_D; d += NTHR) (&cnt[0][0])[d] = 0;
  __syncthreads();
  const int bits = 32 - __clz(a.mask);
#pragma unroll
  for (int k = 0; k < SORT_PER; ++k) {
    const bool in = base + 64 * k < a.n;
    const unsigned d = (key[k] >> a.shift) & a.mask;
    const unsigned long peers = same_digit(d, bits, in);
    const unsigned before = __popcll(peers & ((1ul << lane) - 1ul));
    rank[k] = in ? cnt[wave][d] + before : 0u;
    __builtin_amdgcn_wave_barrier();                       // (a wavefront's LDS operations execute in order)
    if (in && before == 0) cnt[wave][d] += __popcll(peers);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  unsigned pair = total[0] + total[1], scan = pair;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned t = __shfl_up(scan, o);
    if (lane >= o) scan += t;
  }
  if (lane == 63) sums[wave] = scan;
  __syncthreads();
  unsigned start = scan - pair;
  for (int w = 0; w < wave; ++w) start += sums[w];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    unsigned at = start + before[j];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const unsigned c = cnt[w][d0 + j];
      cnt[w][d0 + j] = at;
      at += c;
    }
    start += total[j];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < SORT_PER; ++k) {
    const long i = base + 64 * k;
    if (i >= a.n) continue;
    const unsigned at = cnt[wave][(key[k] >> a.shift) & a.mask] + rank[k];
    a.keys_out[at] = key[k];
    a.places_out[at] = a.tokens ? (unsigned)i : a.places_in[i];
  }
}

// Up to FEW places in one workgroup, all passes in one launch: each wavefront owns a consecutive sixteenth of the list, which goes round
// through LDS.  (The whole gradient of 4096 tokens into 16384 x 256: 24 us, with the launches of count and place 32.)
constexpr int FEW_PER = 4, FEW_THREADS = 1024, FEW = FEW_THREADS * FEW_PER, FEW_BITS = 8, FEW_D = 1 << FEW_BITS;
__global__ __launch_bounds__(FEW_THREADS) void sort_few_kernel(SortArgs a, int passes, int bits) {
  constexpr int NW = FEW_THREADS / 64;
  __shared__ unsigned cnt[NW][FEW_D], keys[FEW], places[FEW], sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = (int)a.n, steps = (n + FEW_THREADS - 1) / FEW_THREADS, base = wave * 64 * steps + lane;
  for (int i = tid; i < n; i += FEW_THREADS) {
    keys[i] = key_of(a.tokens[i], a.vocab);
    places[i] = i;
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    const unsigned mask = (1u << bits) - 1u;
    for (int i = tid; i < NW * FEW_D; i += FEW_THREADS) (&cnt[0][0])[i] = 0;
    __syncthreads();
    unsigned key[FEW_PER], place[FEW_PER], rank[FEW_PER];
#pragma unroll
    for (int k = 0; k < FEW_PER; ++k) {
      const int i = base + 64 * k;
      const bool in = k < steps && i < n;
      key[k] = in ? keys[i] : 0u;
      place[k] = in ? places[i] : 0u;
      if (k >= steps) continue;                            // (of the whole workgroup)
      const unsigned d = key[k] >> shift & mask;
      const unsigned long peers = same_digit(d, bits, in);
      const unsigned before = __popcll(peers & ((1ul << lane) - 1ul));
      rank[k] = in ? cnt[wave][d] + before : 0u;
      __builtin_amdgcn_wave_barrier();
      if (in && before == 0) cnt[wave][d] += __popcll(peers);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    unsigned total = 0, scan = 0;
    if (tid < FEW_D) {                                     // a thread a digit
#pragma unroll
      for (int w = 0; w < NW; ++w) total += cnt[w][tid];
      scan = total;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const unsigned t = __shfl_up(scan, o);
        if (lane >= o) scan += t;
      }
      if (lane == 63) sums[wave] = scan;
    }
    __syncthreads();
    if (tid < FEW_D) {
      unsigned at = scan - total;
      for (int w = 0; w < wave; ++w) at += sums[w];
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const unsigned c = cnt[w][tid];
        cnt[w][tid] = at;
        at += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < FEW_PER; ++k) {
      if (k >= steps || base + 64 * k >= n) continue;
      const unsigned at = cnt[wave][key[k] >> shift & mask] + rank[k];
      keys[at] = key[k];
      places[at] = place[k];
    }
    __syncthreads();
  }
  for (int i = tid; i < n; i += FEW_THREADS) {
    a.keys_out[i] = keys[i];
    a.places_out[i] = places[i];
  }
}

// ---- the gradient: sums --------------------------------------------------------------------------------------------------
struct SumArgs {
  EmbeddingArgs e;
  DropoutKey key;
  const unsigned *keys, *places;   // sorted
  float* chunk_sums;               // [chunks][width]
  unsigned* starts;                // [vocab + 1]: the first place of each token
  unsigned n, units;               // places; width / 8
  unsigned chunks, stride;         // stride: a wavefront's rows of the table are this many apart
};

// G lanes hold a row's channels, 8 each, so a wavefront works on 64 / G rows at a time; slice: blockIdx.y
template <typename T> struct Adder {
  const T* dout;
  const SumArgs& a;
  unsigned long stream;
  unsigned unit;                   // this lane's 8 channels
  bool in;
  __device__ __forceinline__ Adder(const SumArgs& a_, unsigned unit_)
      : dout(reinterpret_cast<const T*>(a_.e.dout.p)), a(a_), stream(a_.key.threshold ? dropout_stream(a_.key) : 0), unit(unit_),
        in(unit_ < a_.units) {}
  __device__ __forceinline__ void load(Raw8<T>& r, unsigned place) const {
    if (in) r.load(dout + (long)place * a.e.dout.row + 8 * unit);
  }
  // The masks of n <= 8 places (even n: one more), 8 bits each.  A loop of two: eight copies of the generator wherever rows are added are 16 KB
  // of instructions that a short launch has to fetch first, and a single one at a time waits for itself.
  template <typename F> __device__ __forceinline__ unsigned long masks(unsigned n, F place) const {
    if (!a.key.threshold) return ~0ul;
    unsigned long m = 0;
#pragma unroll 1
    for (unsigned k = 0; k < n; k += 2) {
      const unsigned long p = place(k), q = place(k + 1);
      const unsigned x = dropout_mask8(a.key, stream, p * a.units + unit), y = dropout_mask8(a.key, stream, q * a.units + unit);
      m |= (unsigned long)(x | y << 8) << (8 * k);
    }
    return m;
  }
  __device__ __forceinline__ void add(float (&acc)[8], const Raw8<T>& r, unsigned mask) const {
    if (!in) return;
    float v[8];
    r.unpack(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += (mask >> j) & 1u ? v[j] : 0.f;
  }
};

// Places of one token, CHUNK of them: each wavefront adds a quarter, and the four sums meet in LDS.  Workgroups behind those (and first
// slice): a thread a row of the table, where its places begin, by bisection.
template <typename T, int G>
__global__ __launch_bounds__(NTHR) void chunk_kernel(SumArgs a) {
  __shared__ float part[4][64 / G][8 * G];
  if (blockIdx.x >= a.chunks) {
    const unsigned v = (blockIdx.x - a.chunks) * NTHR + threadIdx.x;
    if (v > a.e.vocab || blockIdx.y) return;
    unsigned lo = 0, hi = a.n;
    while (lo < hi) {
      const unsigned m = (lo + hi) / 2;
      if (a.keys[m] < v) lo = m + 1; else hi = m;
    }
    a.starts[v] = lo;
    return;
  }
  const unsigned first = blockIdx.x * CHUNK;
  const unsigned v = a.keys[first];
  if (v >= a.e.vocab || a.keys[first + CHUNK - 1] != v) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane / G;
  constexpr int R = 64 / G, Q = CHUNK / 4, STEPS = Q / R > 0 ? Q / R : 1;     // (more lanes than a quarter's places: the others add none)
  const Adder<T> add(a, blockIdx.y * G + lane % G);
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (R <= Q || sub < Q) {
    const unsigned* places = a.places + first + Q * wave + sub;
    Raw8<T> r[STEPS];
    unsigned p[STEPS];
#pragma unroll
    for (int b = 0; b < STEPS; ++b) p[b] = places[b * R];
#pragma unroll
    for (int b = 0; b < STEPS; ++b) add.load(r[b], p[b]);
    const unsigned long masks = add.masks(STEPS, [&](unsigned k) { return p[k < STEPS ? k : 0]; });
#pragma unroll
    for (int b = 0; b < STEPS; ++b) add.add(acc, r[b], (unsigned)(masks >> (8 * b)));
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) part[wave][sub][8 * (lane % G) + j] = acc[j];
  __syncthreads();
  for (int c = threadIdx.x; c < 8 * G; c += NTHR) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int k = 0; k < R; ++k) t += part[w][k][c];
    const unsigned at = blockIdx.y * (8 * G) + c;
    if (at < 8 * a.units) a.chunk_sums[(long)blockIdx.x * (8 * a.units) + at] = t;
  }
}

template <typename O> __device__ __forceinline__ void put8(O* p, const float (&v)[8], bool accumulate) {
  if (accumulate) {
    float w[8];
    load8(p, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] += v[j];
    store8(p, w);
  } else store8(p, v);
}

// What every step-th of `n` places adds, eight on their way at once: the first `head` of them from b on, the rest from t on.  Eight lanes
// of the group read the places, one each.
template <typename T, int G>
__device__ __forceinline__ void add_places(const Adder<T>& add, float (&acc)[8], unsigned b, unsigned head, unsigned t, unsigned n,
                                           unsigned i, unsigned step) {
  constexpr unsigned B = 8;
  const unsigned lane = threadIdx.x & 63, first = lane / G * G;
  for (; i < n; i += B * step) {
    const unsigned at = i + lane % B * step;
    const unsigned mine = at < n ? add.a.places[at < head ? b + at : t + (at - head)] : 0;
    Raw8<T> r[B];
#pragma unroll
    for (unsigned k = 0; k < B; ++k)
      if (i + k * step < n) add.load(r[k], (unsigned)__shfl((int)mine, first + k));
    const unsigned left = (n - i + step - 1) / step;
    const unsigned long masks = add.masks(left < B ? left : B, [&](unsigned k) { return (unsigned)__shfl((int)mine, first + k); });
#pragma unroll
    for (unsigned k = 0; k < B; ++k)
      if (i + k * step < n) add.add(acc, r[k], (unsigned)(masks >> (8 * k)));
  }
}
// the same of chunks' sums
template <typename T>
__device__ __forceinline__ void add_chunks(const Adder<T>& add, float (&acc)[8], unsigned c, unsigned e, unsigned step) {
  constexpr unsigned B = 8;
  if (!add.in) return;
  while (c < e) {
    Raw8<float> r[B];
#pragma unroll
    for (unsigned k = 0; k < B; ++k)
      if (c + k * step < e) r[k].load(add.a.chunk_sums + (long)(c + k * step) * (8 * add.a.units) + 8 * add.unit);
#pragma unroll
    for (unsigned k = 0; k < B; ++k) {
      if (c + k * step >= e) continue;
      float w[8];
      r[k].unpack(w);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += w[j];
    }
    c += B * step;
  }
}
// the stretch b .. e of one token, this group of lanes every step-th of its places and chunks from the which-th on
template <typename T, int G>
__device__ __forceinline__ void add_stretch(const Adder<T>& add, float (&acc)[8], unsigned b, unsigned e, unsigned which, unsigned step) {
  const unsigned c0 = (b + CHUNK - 1) / CHUNK, c1 = e / CHUNK;
  unsigned head = e - b, t = 0, n = head;
  if (c0 < c1) {
    add_chunks(add, acc, c0 + which, c1, step);
    head = c0 * CHUNK - b;
    t = c1 * CHUNK;
    n = head + e - t;
  }
  add_places<T, G>(add, acc, b, head, t, n, which, step);
}
// A token is frequent if its stretch holds a whole chunk: a workgroup for every chunk looks whether it is the first of its token, and
// then adds the token's whole stretch, all lanes at it.  (One group of lanes takes 2 us for eight rows, half of it the generator.)
__device__ __forceinline__ bool frequent(unsigned b, unsigned e) { return (b + CHUNK - 1) / CHUNK < e / CHUNK; }

template <typename T, typename O, int G>
__device__ void frequent_row(const SumArgs& a) {
  __shared__ float part[4 * (64 / G)][8 * G];
  const unsigned c = blockIdx.x, v = a.keys[c * CHUNK];
  if (v >= a.e.vocab || a.keys[c * CHUNK + CHUNK - 1] != v) return;
  const unsigned b = a.starts[v], e = a.starts[v + 1];
  if ((b + CHUNK - 1) / CHUNK != c) return;
  constexpr int R = 64 / G;
  const int lane = threadIdx.x & 63, group = (threadIdx.x >> 6) * R + lane / G;
  const Adder<T> add(a, blockIdx.y * G + lane % G);
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  add_stretch<T, G>(add, acc, b, e, group, 4 * R);
  store8(&part[group][8 * (lane % G)], acc);
  __syncthreads();
  O* out = reinterpret_cast<O*>(a.e.dtable.p) + (long)v * a.e.dtable.row;
  for (int c = threadIdx.x; c < 8 * G; c += NTHR) {
    const unsigned at = blockIdx.y * (8 * G) + c;
    if (at >= 8 * a.units) continue;
    float t = 0.f;
    for (int k = 0; k < 4 * R; ++k) t += part[k][c];
    t *= a.key.factor;
    if (a.e.accumulate) t += Elem<O>::load(out + at);
    if constexpr (sizeof(O) == 2) out[at] = (O)pack_bf16x2(t, 0.f);
    else out[at] = t;
  }
}

// zeros, every store of a wavefront over consecutive places
template <int G> __device__ __forceinline__ void clear8(float* row, unsigned slice, unsigned l, unsigned units) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const unsigned c = slice * (8 * G) + k * (4 * G) + 4 * l;
    if (c < 8 * units) *reinterpret_cast<float4*>(row + c) = make_float4(0.f, 0.f, 0.f, 0.f);
  }
}
template <int G> __device__ __forceinline__ void clear8(bf16_t* row, unsigned slice, unsigned l, unsigned units) {
  const unsigned c = slice * (8 * G) + 8 * l;
  if (c < 8 * units) *reinterpret_cast<uint4*>(row + c) = make_uint4(0, 0, 0, 0);
}

// A wavefront's 64 / G groups of lanes own a row of the table each, and STEPS such rows `stride` apart: tokens of like frequency are
// often numbered next to each other.
template <typename T, typename O, int G, int STEPS>
__global__ __launch_bounds__(NTHR) void table_kernel(SumArgs a) {
  if (blockIdx.x < a.chunks) { frequent_row<T, O, G>(a); return; }
  const int lane = threadIdx.x & 63, sub = lane / G;
  constexpr int R = 64 / G;
  const unsigned v0 = ((blockIdx.x - a.chunks) * 4 + (threadIdx.x >> 6)) * R + sub;
  const Adder<T> add(a, blockIdx.y * G + lane % G);
  O* out = reinterpret_cast<O*>(a.e.dtable.p);
  unsigned from[STEPS], to[STEPS];
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    const unsigned v = v0 + t * a.stride;
    const bool mine = v0 < a.stride && v < a.e.vocab;
    from[t] = mine ? a.starts[v] : 0;
    to[t] = mine ? a.starts[v + 1] : 0;
  }
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    const unsigned v = v0 + t * a.stride;
    if (v0 >= a.stride || v >= a.e.vocab || frequent(from[t], to[t])) continue;
    O* row = out + (long)v * a.e.dtable.row;
    if (to[t] == from[t]) {
      if (!a.e.accumulate) clear8<G>(row, blockIdx.y, lane % G, a.units);
      continue;
    }
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    add_stretch<T, G>(add, acc, from[t], to[t], 0, 1);
    if (!add.in) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] *= a.key.factor;
    put8(row + 8 * add.unit, acc, a.e.accumulate);
  }
}

struct Sorted { unsigned *keys[2], *places[2], *counts, *totals, *starts; float* sums; size_t bytes; int blocks; };
Sorted carve(char* p, long rows, long vocab, int width) {
  Sorted w;
  size_t off = 0;
  auto take = [&](size_t n) { char* q = p ? p + off : nullptr; off += (n + 255) / 256 * 256; return q; };
  w.blocks = (int)((rows + SORT_E - 1) / SORT_E);
  for (int i = 0; i < 2; ++i) {
    w.keys[i] = reinterpret_cast<unsigned*>(take(4 * (size_t)rows));
    w.places[i] = reinterpret_cast<unsigned*>(take(4 * (size_t)rows));
  }
  w.counts = reinterpret_cast<unsigned*>(take((size_t)w.blocks * SORT_D * 4));
  w.totals = reinterpret_cast<unsigned*>(take(SORT_D * 4));
  w.starts = reinterpret_cast<unsigned*>(take(4 * (size_t)(vocab + 1)));
  w.sums = reinterpret_cast<float*>(take((size_t)(rows / CHUNK) * width * 4));
  w.bytes = off;
  return w;
}

template <typename T, typename O, int G>
hipError_t launch_sums(SumArgs a, hipStream_t s) {
  const unsigned slices = (a.units + G - 1) / G, searches = (unsigned)((a.e.vocab + NTHR) / NTHR);
  a.chunks = a.n / CHUNK;
  chunk_kernel<T, G><<<dim3(a.chunks + searches, slices), NTHR, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr unsigned PER = 4 * (64 / G);
  // Four rows a wavefront from 131072 wavefronts on: 131072 x 2048 249 us, with one each 320; 50000 x 1024 45.2, 43.8; 20000 x 512 27.0, 26.1.
  const bool four = a.e.vocab * slices >= 131072l * (64 / G);
  a.stride = (unsigned)(four ? (a.e.vocab + 3) / 4 : a.e.vocab);
  const dim3 grid(a.chunks + (a.stride + PER - 1) / PER, slices);
  if (four) table_kernel<T, O, G, 4><<<grid, NTHR, 0, s>>>(a);
  else table_kernel<T, O, G, 1><<<grid, NTHR, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, typename O>
hipError_t launch_sums_t(const SumArgs& a, hipStream_t s) {
  if (a.units <= 8) return launch_sums<T, O, 8>(a, s);
  if (a.units <= 16) return launch_sums<T, O, 16>(a, s);
  if (a.units <= 32) return launch_sums<T, O, 32>(a, s);
  return launch_sums<T, O, 64>(a, s);
}

}  // namespace

hipError_t launch_dropout(int dtype, const DropoutArgs& a, const DropoutKey& key, hipStream_t s) {
  if (dtype == 0) return a.residual.p ? launch_dropout_t<float, true>(a, key, s) : launch_dropout_t<float, false>(a, key, s);
  return a.residual.p ? launch_dropout_t<bf16_t, true>(a, key, s) : launch_dropout_t<bf16_t, false>(a, key, s);
}

hipError_t launch_embedding_fwd(int dtype, const EmbeddingArgs& a, const DropoutKey& key, hipStream_t s) {
  return dtype == 0 ? launch_lookup_t<float>(a, key, s) : launch_lookup_t<bf16_t>(a, key, s);
}

size_t embedding_ws_bytes(long rows, long vocab, int width) { return carve(nullptr, rows, vocab, width).bytes; }

hipError_t launch_embedding_bwd(int dtype, const EmbeddingArgs& a, const DropoutKey& key, void* workspace, size_t bytes, hipStream_t s) {
  const Sorted w = carve(reinterpret_cast<char*>(workspace), a.rows, a.vocab, a.width);
  if (bytes < w.bytes) return hipErrorInvalidValue;
  int bits = 1;
  while ((a.vocab >> bits) > 0) ++bits;                    // keys are 0 .. vocab
  const int most = a.rows <= FEW ? FEW_BITS : SORT_BITS, passes = (bits + most - 1) / most, per = (bits + passes - 1) / passes;
  SortArgs q{};
  q.n = a.rows; q.vocab = (unsigned)a.vocab; q.blocks = w.blocks; q.counts = w.counts; q.totals = w.totals;
  q.mask = (1 << per) - 1; q.scanned = w.blocks > 64;
  int last = 0;
  if (a.rows <= FEW) {
    q.tokens = a.tokens;
    q.keys_out = w.keys[0]; q.places_out = w.places[0];
    if (a.rows) sort_few_kernel<<<1, FEW_THREADS, 0, s>>>(q, passes, per);
  } else {
    for (int i = 0; i < passes; ++i) {
      q.tokens = i == 0 ? a.tokens : nullptr;
      q.keys_in = w.keys[(i + 1) & 1]; q.places_in = w.places[(i + 1) & 1];
      q.keys_out = w.keys[i & 1]; q.places_out = w.places[i & 1];
      q.shift = i * per;
      count_kernel<<<w.blocks, NTHR, 0, s>>>(q);
      if (q.scanned) scan_kernel<<<SORT_D / 64, 64, 0, s>>>(q);
      place_kernel<<<w.blocks, NTHR, 0, s>>>(q);
      last = i & 1;
    }
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  SumArgs m{};
  m.e = a; m.key = key;
  m.keys = w.keys[last]; m.places = w.places[last];
  m.chunk_sums = w.sums; m.starts = w.starts;
  m.n = (unsigned)a.rows; m.units = (unsigned)(a.width / 8);
  if (dtype == 0) return launch_sums_t<float, float>(m, s);
  return a.grad_dtype == 0 ? launch_sums_t<bf16_t, float>(m, s) : launch_sums_t<bf16_t, bf16_t>(m, s);
}

}  // namespace hbp
