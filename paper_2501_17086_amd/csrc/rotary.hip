// Rotary positions: channel pair i of every head of a row at position p turns by the angle p f_i, as a complex number times
// m exp(+-i p f_i).  All heads of a row turn alike, so a thread forms the angles of V pairs once and walks over heads.
//
// Bound: memory, every element read and written once; 3 flop an element.  The angle is a product of 64 bits in turns, whose
// whole part is dropped before it is rounded to 32: at position 10^6 the first pair has made 159 155 turns, and 32 bits would
// leave an angle 0.05 rad off.
#include "hbp_common.h"

namespace hbp {

namespace {

// V consecutive elements, V a power of two up to 8
template <typename T, int V> struct Chunk;
template <int V> struct Chunk<bf16_t, V> {
  typedef bf16_t vec __attribute__((ext_vector_type(V), aligned(2 * V)));
  vec w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<vec*>(p) = w; }
  __device__ __forceinline__ float get(int i) const { return bf16_to_f32(w[i]); }
  __device__ __forceinline__ void set2(int i, float a, float b) {
    const unsigned u = pack_bf16x2(a, b);
    w[i] = (bf16_t)u;
    w[i + 1] = (bf16_t)(u >> 16);
  }
};
template <> struct Chunk<bf16_t, 1> {
  bf16_t w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *p; }
  __device__ __forceinline__ void store(bf16_t* p) const { *p = w; }
  __device__ __forceinline__ float get(int) const { return bf16_to_f32(w); }
  __device__ __forceinline__ void set1(float v) { w = (bf16_t)pack_bf16x2(v, 0.f); }
};
template <int V> struct Chunk<float, V> {
  typedef float vec __attribute__((ext_vector_type(V), aligned(4 * V < 16 ? 4 * V : 16)));
  vec w;
  __device__ __forceinline__ void load(const float* p) { w = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<vec*>(p) = w; }
  __device__ __forceinline__ float get(int i) const { return w[i]; }
  __device__ __forceinline__ void set2(int i, float a, float b) { w[i] = a; w[i + 1] = b; }
};
template <> struct Chunk<float, 1> {
  float w;
  __device__ __forceinline__ void load(const float* p) { w = *p; }
  __device__ __forceinline__ void store(float* p) const { *p = w; }
  __device__ __forceinline__ float get(int) const { return w; }
  __device__ __forceinline__ void set1(float v) { w = v; }
};

// The pairs of a unit, V of them: HALF two chunks of V channels dims / 2 apart, INTERLEAVED one stretch of 2 V channels.
template <typename T, int V, bool HALF> struct Pairs;
template <typename T, int V> struct Pairs<T, V, true> {
  Chunk<T, V> a, b;
  __device__ __forceinline__ void load(const T* p, int half) { a.load(p); b.load(p + half); }
  __device__ __forceinline__ void turn(const float (&c)[V], const float (&s)[V]) {
    float x[V], y[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float u = a.get(i), w = b.get(i);
      x[i] = u * c[i] - w * s[i];
      y[i] = u * s[i] + w * c[i];
    }
    if constexpr (V == 1) {
      a.set1(x[0]);
      b.set1(y[0]);
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2) { a.set2(i, x[i], x[i + 1]); b.set2(i, y[i], y[i + 1]); }
    }
  }
  __device__ __forceinline__ void store(T* p, int half) const { a.store(p); b.store(p + half); }
};
template <typename T, int V> struct Pairs<T, V, false> {
  static constexpr int W = V < 8 ? 2 * V : 8, C = 2 * V / W;        // chunks of at most 8 channels
  Chunk<T, W> a[C];
  __device__ __forceinline__ void load(const T* p, int) {
#pragma unroll
    for (int j = 0; j < C; ++j) a[j].load(p + j * W);
  }
  __device__ __forceinline__ void turn(const float (&c)[V], const float (&s)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int j = 2 * i / W, e = 2 * i % W;
      const float u = a[j].get(e), w = a[j].get(e + 1);
      a[j].set2(e, u * c[i] - w * s[i], u * s[i] + w * c[i]);
    }
  }
  __device__ __forceinline__ void store(T* p, int) const {
#pragma unroll
    for (int j = 0; j < C; ++j) a[j].store(p + j * W);
  }
};

// A thread owns one unit of a row, V pairs or V channels that are only copied, in `per` consecutive heads.
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  const unsigned id = blockIdx.x * 256u + threadIdx.x;
  const unsigned n = id / (unsigned)a.units, u = id - n * (unsigned)a.units;
  if (n >= (unsigned)a.rows) return;
  const int h0 = (int)blockIdx.y * a.per, h1 = h0 + a.per < a.heads ? h0 + a.per : a.heads;
  const int half = a.dims / 2, turning = half / V;
  const T* x = reinterpret_cast<const T*>(a.x) + (long)n * a.x_row + (long)h0 * a.x_head;
  T* y = reinterpret_cast<T*>(a.y) + (long)n * a.y_row + (long)h0 * a.y_head;
  constexpr int B = 4;                               // heads whose loads go out together
  if ((int)u >= turning) {
    const int c0 = a.dims + ((int)u - turning) * V;
    for (int h = h0; h < h1; ++h, x += a.x_head, y += a.y_head) {
      Chunk<T, V> w;
      w.load(x + c0);
      w.store(y + c0);
    }
    return;
  }
  const int i0 = (int)u * V, c0 = HALF ? i0 : 2 * i0;
  const long place = a.period > 0 ? (long)(n % (unsigned)a.period) : (long)n;
  const double pos = (double)(a.positions ? (long)a.positions[n] : a.first + place);
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    double t = pos * a.turns[i0 + i];
    t -= rint(t);
    sincospif(2.f * (float)t, &s[i], &c[i]);
    c[i] *= a.magnitude;
    s[i] *= a.inverse ? -a.magnitude : a.magnitude;
  }
  int h = h0;
  for (; h + B <= h1; h += B) {
    Pairs<T, V, HALF> p[B];
#pragma unroll
    for (int b = 0; b < B; ++b) p[b].load(x + b * a.x_head + c0, half);
#pragma unroll
    for (int b = 0; b < B; ++b) {
      p[b].turn(c, s);
      p[b].store(y + b * a.y_head + c0, half);
    }
    x += B * a.x_head;
    y += B * a.y_head;
  }
  for (; h < h1; ++h, x += a.x_head, y += a.y_head) {
    Pairs<T, V, HALF> p;
    p.load(x + c0, half);
    p.turn(c, s);
    p.store(y + c0, half);
  }
}

template <typename T, int V>
hipError_t launch_v(RotaryArgs a, int layout, hipStream_t s) {
  a.units = a.dims / 2 / V + (a.x == a.y ? 0 : (a.dh - a.dims) / V);
  const long threads = a.rows * a.units;
  // Heads are shared out until there are 1024 threads for every compute unit: 72 heads of 32 channels in 3438 rows take 10.7 us (2048
  // threads, and a head each: 11.8, the angles formed 72 times), 40 of 64 with 6 channels turning in 2799 rows 16 us (512: 23).
  long split = (256L * 1024 + threads - 1) / threads;
  if (split > a.heads) split = a.heads;
  a.per = (int)((a.heads + split - 1) / split);
  const dim3 grid((unsigned)((threads + 255) / 256), (unsigned)((a.heads + a.per - 1) / a.per));
  if (layout == 0) rotary_kernel<T, V, true><<<grid, 256, 0, s>>>(a);
  else rotary_kernel<T, V, false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const RotaryArgs& a, int layout, hipStream_t s) {
  const int half = a.dims / 2;
  if (half % 8 == 0) return launch_v<T, 8>(a, layout, s);
  if (half % 4 == 0) return launch_v<T, 4>(a, layout, s);
  if (half % 2 == 0) return launch_v<T, 2>(a, layout, s);
  return launch_v<T, 1>(a, layout, s);
}

}  // namespace

hipError_t launch_rotary(int dtype, int layout, const RotaryArgs& a, hipStream_t s) {
  return dtype == 0 ? launch_t<float>(a, layout, s) : launch_t<bf16_t>(a, layout, s);
}

}  // namespace hbp
