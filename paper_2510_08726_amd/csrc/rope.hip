// Rotary positions (include/rope.h): queries and keys in one kernel, which
// reads and writes every row once.
//
// A thread takes V pairs of one token (the same dims of every head turn by the
// same angle), forms their sines and cosines once, and turns those pairs in
// `heads` heads.  Angles: t = p f and its fraction of a turn in 64 bits, exactly
// reduced to an eighth of a turn; sine and cosine there by their Taylor series
// in 32 bits (through x^9 and x^10, under 2e-9 off for |x| <= pi / 4).
// Bound by HBM for many tokens (a row in and out), by the launch for few.

#include "kernel_common.h"
#include "launch.h"

namespace attn {

namespace {

constexpr int kThreads = 256;

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

// Sine and cosine of p * f radians.
__device__ __forceinline__ void sin_cos(double p, double f, float& si, float& co) {
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

// The threads of a token: R / (2 V) of V pairs each, then (D - R) / V that copy.
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeParams p) {
  typedef Pack<T, V> P;
  typedef typename P::raw raw;
  const int turning = p.R / (2 * V), per = turning + (p.D - p.R) / V;
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t token = idx / per;
  if (token >= (int64_t)p.B * p.L) return;
  const int w = (int)(idx - token * per);
  const int b = (int)(token / p.L), l = (int)(token - (int64_t)b * p.L);
  const bool turns = w < turning;
  // The two vectors of V elements: a's and b's of the pairs, or neighbours.
  const int d0 = turns ? (INTER ? 2 * V * w : V * w) : p.R + V * (w - turning);
  const int d1 = turns ? (INTER ? d0 + V : d0 + p.R / 2) : d0;

  float si[V], co[V];
  if (turns) {
    const int64_t at = b * p.pos_stride + l;
    const double pos = p.pos64 ? (double)static_cast<const int64_t*>(p.pos)[at]
                               : (double)static_cast<const int*>(p.pos)[at];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float s, c;
      sin_cos(pos, p.freqs[V * w + i], s, c);
      si[i] = s * p.magnitude * p.sign;
      co[i] = c * p.magnitude;
    }
  }
  const int first = blockIdx.y * p.heads, last = min(first + p.heads, p.H[0] + p.H[1]);
  for (int hh = first; hh < last; ++hh) {
    const int k = hh >= p.H[0];
    const int h = k ? hh - p.H[0] : hh;
    const T* x = static_cast<const T*>(p.x[k]) + b * p.sb[k] + h * p.sh[k] + l * p.sl[k];
    T* y = static_cast<T*>(p.y[k]) + (((int64_t)b * p.H[k] + h) * p.L + l) * p.D;
    const raw r0 = *reinterpret_cast<const raw*>(x + d0);
    if (!turns) {
      *reinterpret_cast<raw*>(y + d0) = r0;
      continue;
    }
    const raw r1 = *reinterpret_cast<const raw*>(x + d1);
    float f[2 * V], g[2 * V];
    P::load(r0, f);
    P::load(r1, f + V);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int a = INTER ? 2 * i : i, c = INTER ? 2 * i + 1 : V + i;
      g[a] = f[a] * co[i] - f[c] * si[i];
      g[c] = __builtin_fmaf(f[a], si[i], f[c] * co[i]);
    }
    *reinterpret_cast<raw*>(y + d0) = P::store(g);
    *reinterpret_cast<raw*>(y + d1) = P::store(g + V);
  }
}

template <typename T, int V>
hipError_t launch(RopeParams p, hipStream_t stream) {
  const int64_t threads = (int64_t)p.B * p.L * (p.R / (2 * V) + (p.D - p.R) / V);
  const int heads = p.H[0] + p.H[1];
  const int64_t blocks = (threads + kThreads - 1) / kThreads;
  p.heads = 1;
  const dim3 grid((unsigned)blocks, (unsigned)((heads + p.heads - 1) / p.heads)), block(kThreads);
  if (p.interleaved)
    hipLaunchKernelGGL((rope_kernel<T, V, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((rope_kernel<T, V, false>), grid, block, 0, stream, p);
  return hipGetLastError();
}

// Every row starts at a multiple of n elements, and pairs fill vectors of n.
bool vectors(const RopeParams& p, int n, int size) {
  if (p.D % n || p.R % (2 * n)) return false;
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
