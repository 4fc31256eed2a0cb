// Rotary positions (include/rope.h): queries and keys in one kernel, which
// reads and writes every row once.
//
// Angles: t = p f and its fraction of a turn in 64 bits (three roundings: 3.3e-16 of t),
// exactly reduced to an eighth of a turn; sine and cosine there by their Taylor series in 32
// bits (through x^9 and x^10, under 2e-9 off for |x| <= pi / 4).  A thread forms them once for
// its dims and turns four heads by them: 4 x 4096 tokens of 32 + 8 heads of 128 bf16 dims
// take 68 us with one head a thread, 61 with two, 56 with 4 and 57 with 8.  Up to 512
// workgroups latency wants every thread there is: the kernel takes 3.4 us for 8 tokens
// with one head a thread and 4.0 with four, 4.4 and 4.6 for 256, but 5.0 and 4.9 for
// 512, 10.8 and 8.5 for 3 x 512 (medians of a profiled run; calls in a row 10.0 and 8.4).
//
// Bound by HBM for many tokens: 335 MB in and out in 56 us, 6.0 TB/s (interleaved
// pairs out of a projection's [B, L, H, D] 61), by the launch for few (8 tokens: 3.4 us, a
// kernel that does nothing 2).  Calls with 64 MB of outputs or more, which leave the
// caches before anybody reads them, are streamed past them: 63 us without, 8192 tokens
// 34.1 against 29.3, 2 x 4096 of fp32 70.8 against 65.9 (but 4096 tokens, 42 MB, 14.2 and 16.1
// streamed).  Not where neighbouring loads share lines, which then are fetched again: 4 x
// 4096 tokens of 32 heads of 64, in halves of 64 bytes, 26.4 and 32.0 streamed.

#include "kernel_common.h"
#include "launch.h"

namespace attn {

namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 4;       // heads of a thread
constexpr int kFew = 512;       // workgroups of one head a thread up to which a thread has one

constexpr int64_t kStream = int64_t(64) << 20;   // bytes of outputs from which a call is streamed

// Whether a call is read and written past the caches: one whose outputs
// leave them before they are read again, and whose rows' parts are whole lines.
inline bool streamed(const RopeParams& p, int64_t size) {
  const int64_t part = p.interleaved ? p.R * size : p.R / 2 * size;
  return part % 128 == 0 && (p.D - p.R) * size % 128 == 0 && (int64_t)p.B * p.L * (p.H[0] + p.H[1]) * p.D * size >= kStream;
}

template <bool ONCE, typename R>
__device__ __forceinline__ R load(const R* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool ONCE, typename R>
__device__ __forceinline__ void store(R* p, const R& v) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// V elements of T as one register group, to and from fp32.
template <typename T, int V> struct Pack;
template <typename T> struct Pack<T, 1> {
  typedef T raw;
  static __device__ __forceinline__ void load(const raw& r, float* f) { f[0] = (float)r; }
  static __device__ __forceinline__ raw store(const float* f) { return (T)f[0]; }
};
template <typename T> struct Pack<T, 4> {   // 16-bit types: 8 bytes
  typedef uint32_t raw __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ void load(const raw& r, float* f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f[2 * i] = Elem<T>::lo(r[i]);
      f[2 * i + 1] = Elem<T>::hi(r[i]);
    }
  }
  static __device__ __forceinline__ raw store(const float* f) {
    return raw{Elem<T>::pack2(f[0], f[1]), Elem<T>::pack2(f[2], f[3])};
  }
};
template <typename T> struct Pack<T, 8> {
  typedef u32x4 raw;
  static __device__ __forceinline__ void load(const raw& r, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = Elem<T>::lo(r[i]);
      f[2 * i + 1] = Elem<T>::hi(r[i]);
    }
  }
  static __device__ __forceinline__ raw store(const float* f) {
    raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = Elem<T>::pack2(f[2 * i], f[2 * i + 1]);
    return r;
  }
};
template <> struct Pack<float, 4> {
  typedef f32x4 raw;
  static __device__ __forceinline__ void load(const raw& r, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = r[i];
  }
  static __device__ __forceinline__ raw store(const float* f) { return raw{f[0], f[1], f[2], f[3]}; }
};

// Sine and cosine of p * f radians.  (No products are contracted but those
// written as such: every kernel then gives the same bits.)
__device__ __forceinline__ void sin_cos(double p, double f, float& si, float& co) {
#pragma clang fp contract(off)
  double t = p * f * 0.15915494309189535;      // turns: 1 / (2 pi)
  t = 4.0 * (t - __builtin_rint(t));           // quarters of a turn, -2 .. 2
  const double q = __builtin_rint(t);
  const float x = (float)(t - q) * 1.5707963267948966f;
  const float z = x * x;
  const float s = x * __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 2.7557319e-6f, -1.9841270e-4f),
                                                                          8.3333333e-3f), -0.16666667f), 1.f);
  const float c = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f),
                                                                          -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  const int k = (int)q & 3;
  const float a = k & 1 ? c : s, b = k & 1 ? s : c;
  si = k & 2 ? -a : a;
  co = (k + 1) & 2 ? -b : b;
}

// Threads that copy the dims behind the rotated ones: as many vectors each as a
// thread that turns has, one or two.
template <int V, bool ONE>
__device__ __host__ __forceinline__ int copying_threads(const RopeParams& p) {
  const int copied = (p.D - p.R) / V;
  return ONE ? copied : (copied + 1) / 2;
}

// The threads of a token: those that turn kPairs pairs each, then those that copy
// the dims behind.  A thread has the pairs' a's in one vector of V elements and their b's in
// another, or, interleaved, V / 2 pairs in one vector (one pair in two elements where V =
// 1): so the lanes of a row cover it without gaps either way.  Its heads are
// kBatch neighbours, all loaded before the angles are formed.
template <typename T, int V, bool INTER, int kBatch, bool ONCE>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeParams p) {
  typedef Pack<T, V> P;
  typedef typename P::raw raw;
  constexpr bool kOne = INTER && V > 1;              // both of a pair in one vector
  constexpr int kPairs = kOne ? V / 2 : V;
  const uint32_t turning = (uint32_t)p.R / (2 * kPairs);
  const int copying = copying_threads<V, kOne>(p);
  const uint32_t per = turning + (uint32_t)copying;
  const uint32_t idx = blockIdx.x * kThreads + threadIdx.x;
  const uint32_t token = idx / per;
  if (token >= (uint32_t)p.B * (uint32_t)p.L) return;
  const int w = (int)(idx - token * per);
  const int b = (int)(token / (uint32_t)p.L), l = (int)(token - (uint32_t)b * (uint32_t)p.L);
  const bool turns = w < (int)turning;
  const int d0 = turns ? (INTER ? 2 * kPairs * w : V * w) : p.R + V * (w - (int)turning);
  const int next = turns ? (INTER ? V : p.R / 2) : V * copying;
  const int d1 = kOne || d0 + next >= p.D ? d0 : d0 + next;    // (a lone vector is copied twice)
  const int heads = p.H[0] + p.H[1], first = blockIdx.y * kBatch;

  const T* x[kBatch];
  T* y[kBatch];
  raw r0[kBatch], r1[kBatch];
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const int hh = min(first + u, heads - 1);          // past the last: that head again, not stored
    const int k = hh >= p.H[0];
    const int h = k ? hh - p.H[0] : hh;
    x[u] = static_cast<const T*>(p.x[k]) + b * p.sb[k] + h * p.sh[k] + l * p.sl[k];
    y[u] = static_cast<T*>(p.y[k]) + (((int64_t)b * p.H[k] + h) * p.L + l) * p.D;
  }
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    r0[u] = load<ONCE>(reinterpret_cast<const raw*>(x[u] + d0));
    if (!kOne) r1[u] = load<ONCE>(reinterpret_cast<const raw*>(x[u] + d1));
  }
  if (!turns) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (first + u < heads) {
        store<ONCE>(reinterpret_cast<raw*>(y[u] + d0), r0[u]);
        if (!kOne) store<ONCE>(reinterpret_cast<raw*>(y[u] + d1), r1[u]);
      }
    return;
  }
  const int64_t at = b * p.pos_stride + l;
  const double pos = p.pos64 ? (double)static_cast<const int64_t*>(p.pos)[at]
                             : (double)static_cast<const int*>(p.pos)[at];
  float si[kPairs], co[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    float s, c;
    sin_cos(pos, p.freqs[kPairs * w + i], s, c);
    si[i] = s * p.magnitude * p.sign;
    co[i] = c * p.magnitude;
  }
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    if (first + u >= heads) break;
    float f[2 * V], g[2 * V];
    P::load(r0[u], f);
    if (!kOne) P::load(r1[u], f + V);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const int a = INTER ? 2 * i : i, c = INTER ? 2 * i + 1 : V + i;
      g[a] = __builtin_fmaf(f[a], co[i], -(f[c] * si[i]));
      g[c] = __builtin_fmaf(f[a], si[i], f[c] * co[i]);
    }
    store<ONCE>(reinterpret_cast<raw*>(y[u] + d0), P::store(g));
    if (!kOne) store<ONCE>(reinterpret_cast<raw*>(y[u] + d1), P::store(g + V));
  }
}

template <typename T, int V, int kBatch, bool ONCE>
hipError_t launch_batch(const RopeParams& p, int64_t blocks, hipStream_t stream) {
  const dim3 grid((unsigned)blocks, (unsigned)((p.H[0] + p.H[1] + kBatch - 1) / kBatch)), block(kThreads);
  if (p.interleaved)
    hipLaunchKernelGGL((rope_kernel<T, V, true, kBatch, ONCE>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((rope_kernel<T, V, false, kBatch, ONCE>), grid, block, 0, stream, p);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t launch(const RopeParams& p, hipStream_t stream) {
  const bool one = p.interleaved && V > 1;             // as the kernel divides a row
  const int64_t threads = (int64_t)p.B * p.L *
                          (p.R / (one ? V : 2 * V) + (one ? copying_threads<V, true>(p) : copying_threads<V, false>(p)));
  const int64_t blocks = (threads + kThreads - 1) / kThreads;
  if (blocks * (p.H[0] + p.H[1]) <= kFew) return launch_batch<T, V, 1, false>(p, blocks, stream);
  if constexpr (V * sizeof(T) == 16)
    if (streamed(p, sizeof(T))) return launch_batch<T, V, kHeads, true>(p, blocks, stream);
  return launch_batch<T, V, kHeads, false>(p, blocks, stream);
}

// Every row starts at a multiple of n elements, and pairs fill vectors of n.
bool vectors(const RopeParams& p, int n, int size) {
  if (p.D % n || p.R % (p.interleaved ? n : 2 * n)) return false;
  for (int k = 0; k < 2; ++k) {
    if (!p.x[k]) continue;
    if (p.sb[k] % n || p.sh[k] % n || p.sl[k] % n) return false;
    if ((reinterpret_cast<uintptr_t>(p.x[k]) | reinterpret_cast<uintptr_t>(p.y[k])) % (size_t)(n * size)) return false;
  }
  return true;
}

template <typename T>
hipError_t launch16(const RopeParams& p, hipStream_t stream) {
  if (vectors(p, 8, 2)) return launch<T, 8>(p, stream);
  if (vectors(p, 4, 2)) return launch<T, 4>(p, stream);
  return launch<T, 1>(p, stream);
}

}  // namespace

hipError_t launch_rope(const RopeParams& p, hipStream_t stream) {
  if (p.dtype == 0) return launch16<_Float16>(p, stream);
  if (p.dtype == 1) return launch16<__bf16>(p, stream);
  return vectors(p, 4, 4) ? launch<float, 4>(p, stream) : launch<float, 1>(p, stream);
}

}  // namespace attn
