// The root-mean-square norm between a model's layers for gfx950 (include/rmsnorm.h):
//
//   h = x + residual,  rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd (w + offset)
//
// in one pass: a row's h stays in the registers of the 64 to 1024 lanes that
// hold the row (8 elements a lane and step), so every byte is read once and written
// once.  Bound by memory; small calls by the launch and one reduction's latency.
//
// The squares are summed in fp64 (vector fp64 runs at the rate of plain fp32 here: two
// instructions an element, hidden behind the loads), so no row of fp32 or bf16 overflows.
// The 8-bit form takes y and its quotient by the scale in fp64 too: a code is then that of the
// definition, which fp32 misses for the one element in a million that lies next to a border.

#include <algorithm>
#include <type_traits>

#include "kernel_common.h"
#include "launch.h"

namespace attn {

namespace {

constexpr int kMaxThreads = 1024;
constexpr int kMaxWaves = kMaxThreads / 64;

// 16 bytes at any address that an element may have (the hardware takes them so).
template <typename T> struct Packed {
  typedef u32x4 vec;
  struct __attribute__((packed, aligned(sizeof(T)))) type { vec v; };
};

template <typename T> __device__ __forceinline__ float to_float(T x) { return (float)x; }

// 8 elements at `at`, the first n of which are the row's; zeros for the others.
template <typename T>
__device__ __forceinline__ void get8(const T* at, int n, float (&x)[8]) {
  if (n >= 8) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const u32x4 w = reinterpret_cast<const typename Packed<T>::type*>(at + 4 * k)->v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned u = w[i];
          x[4 * k + i] = __builtin_bit_cast(float, u);
        }
      }
    } else {
      const u32x4 w = reinterpret_cast<const typename Packed<T>::type*>(at)->v;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned u = w[i];
        x[2 * i] = Elem<T>::lo(u);
        x[2 * i + 1] = Elem<T>::hi(u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? to_float(at[i]) : 0.f;
  }
}

// The first n of 8 values, rounded to T.
template <typename T>
__device__ __forceinline__ void put8(T* at, int n, const float (&x)[8]) {
  if (n >= 8) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = x[4 * k + i];
          w[i] = __builtin_bit_cast(unsigned, f);
        }
        reinterpret_cast<typename Packed<T>::type*>(at + 4 * k)->v = w;
      }
    } else {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = Elem<T>::pack2(x[2 * i], x[2 * i + 1]);
      reinterpret_cast<typename Packed<T>::type*>(at)->v = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) at[i] = (T)x[i];
  }
}

// Values as T holds them.
template <typename T>
__device__ __forceinline__ void round8(float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)(T)x[i];
}

struct Sum {
  static __device__ __forceinline__ double join(double a, double b) { return a + b; }
  static __device__ __forceinline__ float join(float a, float b) { return a + b; }
};
// Of magnitudes, by their bits: a NaN is larger than all others.
struct Most {
  static __device__ __forceinline__ double join(double a, double b) {
    return __builtin_bit_cast(uint64_t, a) > __builtin_bit_cast(uint64_t, b) ? a : b;
  }
};

// Joins x over the `lanes` lanes of a row (of several waves through `shared`, which the caller's next
// join has to differ from).
template <typename J, typename V>
__device__ __forceinline__ V join_row(V x, int lanes, V* shared) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) x = J::join(x, __shfl_xor(x, m, 64));
  if (lanes > 64) {
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    const V* own = shared + threadIdx.x / lanes * (lanes / 64);      // the row's waves
    x = own[0];
    for (int w = 1; w < lanes / 64; ++w) x = J::join(x, own[w]);
  }
  return x;
}

// z in fp32, rounded to odd: toward zero, its last bit set where that lost something, so that a
// second rounding to fewer bits gives what one rounding of z would.
__device__ __forceinline__ float to_odd(double z) {
  const float f = (float)z;
  const double d = (double)f;
  unsigned b = __builtin_bit_cast(unsigned, f);
  b -= __builtin_fabs(d) > __builtin_fabs(z) ? 1u : 0u;
  b |= d != z ? 1u : 0u;
  return __builtin_bit_cast(float, b);
}

// 8 codes of z, in two words.
__device__ __forceinline__ uint2 codes8(const double (&z)[8], bool int8) {
  unsigned w[2] = {0u, 0u};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = to_odd(z[4 * k + i]);
    if (int8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = (int)__builtin_rintf(fminf(fmaxf(f[i], -127.f), 127.f));
        w[k] |= ((unsigned)c & 255u) << (8 * i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = fminf(fmaxf(f[i], -448.f), 448.f);
      w[k] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
      w[k] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], (int)w[k], true);
    }
  }
  return make_uint2(w[0], w[1]);
}

struct __attribute__((packed, aligned(1))) Bytes8 { uint2 v; };

// T: the type of x, the weight and y; R: that of the residual and h.  C: steps of 8 elements a
// lane.  QUANT: y in 8 bits.
template <typename T, typename R, int C, bool QUANT>
__global__ __launch_bounds__(kMaxThreads) void rmsnorm_add_kernel(RmsnormParams p) {
  __shared__ double sums[kMaxWaves];
  __shared__ double tops[kMaxWaves];
  const int lanes = p.lanes, rpb = blockDim.x / lanes;
  const int sub = threadIdx.x / lanes, t = threadIdx.x % lanes;
  const int M = p.M;
  for (int64_t first = (int64_t)blockIdx.x * rpb; first < p.N; first += (int64_t)gridDim.x * rpb) {
    const int64_t row = first + sub;
    const bool in = row < p.N;
    const int m = in ? M : 0;
    const int64_t base = (in ? row : 0) * M;
    float h[C][8];
    double ss = 0.0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (c * lanes + t);
      get8(reinterpret_cast<const T*>(p.x) + base + col, m - col, h[c]);
    }
    if (p.residual) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = 8 * (c * lanes + t);
        float r[8];
        get8(reinterpret_cast<const R*>(p.residual) + base + col, m - col, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] += r[i];
        put8(reinterpret_cast<R*>(p.h) + base + col, m - col, h[c]);
        round8<R>(h[c]);
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)h[c][i], (double)h[c][i], ss);
    ss = join_row<Sum>(ss, lanes, sums);
    const double rstd = 1.0 / __builtin_sqrt(ss / M + p.eps);
    if (p.rstd && in && t == 0) p.rstd[row] = (float)rstd;
    if constexpr (!QUANT) {
      const float r = (float)rstd;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = 8 * (c * lanes + t);
        float w[8], y[8];
        if (p.weight) get8(reinterpret_cast<const T*>(p.weight) + col, m - col, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = p.weight ? h[c][i] * r * (w[i] + p.offset) : h[c][i] * r;
        put8(reinterpret_cast<T*>(p.y) + base + col, m - col, y);
      }
    } else {
      const double most = p.int8 ? 127.0 : 448.0;
      const int G = p.group;
      double top = 0.0;
      double g = 0.0;          // rstd over the scale
      auto weighed = [&](int c, double (&z)[8]) __attribute__((always_inline)) {    // h (w + offset)
        const int col = 8 * (c * lanes + t);
        float w[8];
        if (p.weight) get8(reinterpret_cast<const T*>(p.weight) + col, m - col, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = p.weight ? (double)h[c][i] * ((double)w[i] + (double)p.offset) : (double)h[c][i];
      };
      auto scaled = [&](double a, int64_t at, bool writes) {
        float s = (float)(a * rstd / most);
        const bool fine = s <= 3.4028234663852886e38f;     // (not an infinity or NaN)
        if (!fine) s = __builtin_nanf("");
        if (writes) p.scales[at] = s;
        return fine && s > 0.f ? rstd / (double)s : 0.0;
      };
      if (G == 0) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          double z[8];
          weighed(c, z);
#pragma unroll
          for (int i = 0; i < 8; ++i) top = Most::join(top, __builtin_fabs(z[i]));
        }
        top = join_row<Most>(top, lanes, tops);
        g = scaled(top, row, in && t == 0);
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = 8 * (c * lanes + t);
        double z[8];
        weighed(c, z);
        if (G != 0) {
          double a = 0.0;
#pragma unroll
          for (int i = 0; i < 8; ++i) a = Most::join(a, __builtin_fabs(z[i]));
          for (int k = G / 16; k > 0; k >>= 1) a = Most::join(a, __shfl_xor(a, k, 64));
          g = scaled(a, row * p.groups + col / G, col < m && col % G == 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = g == 0.0 ? 0.0 : z[i] * g;
        const uint2 w = codes8(z, p.int8);
        unsigned char* at = reinterpret_cast<unsigned char*>(p.y) + base + col;
        if (m - col >= 8) {
          reinterpret_cast<Bytes8*>(at)->v = w;
        } else {
          for (int i = 0; i < m - col; ++i) at[i] = (unsigned char)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
        }
      }
    }
    if (lanes > 64) __syncthreads();      // before the next row's sums
  }
}

// Gradients.  A workgroup takes rows in turn, and its lanes keep the sum of dY n of their columns over
// them: [partials, M] in fp32, summed by rmsnorm_dweight_kernel in a fixed order.
template <typename T, typename R, int C>
__global__ __launch_bounds__(kMaxThreads) void rmsnorm_add_bwd_kernel(RmsnormBwdParams p) {
  __shared__ float sums[2][kMaxWaves];
  const int lanes = p.lanes, rpb = blockDim.x / lanes;
  const int sub = threadIdx.x / lanes, t = threadIdx.x % lanes;
  const int M = p.M;
  float dw[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[c][i] = 0.f;
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * rpb; first < p.N; first += (int64_t)gridDim.x * rpb, turn ^= 1) {
    const int64_t row = first + sub;
    const bool in = row < p.N;
    const int m = in ? M : 0;
    const int64_t base = (in ? row : 0) * M;
    const float r = in ? p.rstd[row] : 0.f;
    float g[C][8], n[C][8];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (c * lanes + t);
      get8(reinterpret_cast<const T*>(p.dy) + base + col, m - col, g[c]);
      get8(reinterpret_cast<const R*>(p.h) + base + col, m - col, n[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (c * lanes + t);
      float w[8];
      if (p.weight) get8(reinterpret_cast<const T*>(p.weight) + col, m - col, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        n[c][i] *= r;
        dw[c][i] = __builtin_fmaf(g[c][i], n[c][i], dw[c][i]);
        if (p.weight) g[c][i] *= w[i] + p.offset;
        s = __builtin_fmaf(g[c][i], n[c][i], s);
      }
    }
    s = join_row<Sum>(s, lanes, sums[turn]) / (float)M;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (c * lanes + t);
      float d[8];
      if (p.dh) get8(reinterpret_cast<const R*>(p.dh) + base + col, m - col, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = r * __builtin_fmaf(-n[c][i], s, g[c][i]);
        d[i] = p.dh ? d[i] + x : x;
      }
      if (p.dresidual) put8(reinterpret_cast<R*>(p.dresidual) + base + col, m - col, d);
      put8(reinterpret_cast<T*>(p.dx) + base + col, m - col, d);
    }
  }
  if (!p.ws) return;
  float* at = p.ws + ((int64_t)blockIdx.x * rpb + sub) * M;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = 8 * (c * lanes + t);
    put8(at + col, M - col, dw[c]);
  }
}

// Columns summed over the partials: 32 columns a workgroup, every eighth partial a row of lanes.
__global__ __launch_bounds__(256) void rmsnorm_dweight_kernel(const float* ws, float* out, int parts, int M) {
  __shared__ float part[8][32];
  const int col = blockIdx.x * 32 + threadIdx.x % 32, k = threadIdx.x / 32;
  float s = 0.f;
  if (col < M)
    for (int i = k; i < parts; i += 8) s += ws[(int64_t)i * M + col];
  part[k][threadIdx.x % 32] = s;
  __syncthreads();
  if (k == 0 && col < M) {
    for (int i = 1; i < 8; ++i) s += part[i][threadIdx.x];
    out[col] = s;
  }
}

// What codes stand for: 8 of them a lane.
template <typename T>
__global__ __launch_bounds__(256) void quant8_load_kernel(Quant8LoadParams p) {
  const int chunks = (p.M + 7) / 8;
  const int64_t all = (int64_t)p.N * chunks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / chunks;
    const int col = 8 * (int)(i - row * chunks), n = p.M - col;
    const unsigned char* at = p.codes + row * p.M + col;
    unsigned w[2] = {0u, 0u};
    if (n >= 8) {
      const uint2 v = reinterpret_cast<const Bytes8*>(at)->v;
      w[0] = v.x;
      w[1] = v.y;
    } else {
      for (int k = 0; k < n; ++k) w[k / 4] |= (unsigned)at[k] << (8 * (k & 3));
    }
    const float s = p.scales[row * p.groups + (p.group ? col / p.group : 0)];
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const unsigned b = w[k / 4] >> (8 * (k & 3));
      y[k] = s * (p.int8 ? (float)(signed char)(b & 255u) : __builtin_amdgcn_cvt_f32_fp8((int)b, 0));
    }
    put8(reinterpret_cast<T*>(p.y) + row * p.M + col, n, y);
  }
}

// Lanes of a row, and steps of 8 elements of a lane.
struct Split {
  int lanes, steps;
};
// By the row's length alone, so that a row's bits do not depend on how many there are.
Split split(int M) {
  int lanes = 64;
  while (lanes < kMaxThreads && 8 * lanes < M) lanes *= 2;
  const int s = (M + 8 * lanes - 1) / (8 * lanes);
  return {lanes, s <= 1 ? 1 : s <= 2 ? 2 : 4};
}

template <typename T, typename R, bool QUANT>
void launch_add(const RmsnormParams& p, const Split& s, dim3 grid, dim3 block, hipStream_t stream) {
  if (s.steps == 1) hipLaunchKernelGGL((rmsnorm_add_kernel<T, R, 1, QUANT>), grid, block, 0, stream, p);
  else if (s.steps == 2) hipLaunchKernelGGL((rmsnorm_add_kernel<T, R, 2, QUANT>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((rmsnorm_add_kernel<T, R, 4, QUANT>), grid, block, 0, stream, p);
}

template <typename T, typename R>
void launch_bwd(const RmsnormBwdParams& p, const Split& s, dim3 grid, dim3 block, hipStream_t stream) {
  if (s.steps == 1) hipLaunchKernelGGL((rmsnorm_add_bwd_kernel<T, R, 1>), grid, block, 0, stream, p);
  else if (s.steps == 2) hipLaunchKernelGGL((rmsnorm_add_bwd_kernel<T, R, 2>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((rmsnorm_add_bwd_kernel<T, R, 4>), grid, block, 0, stream, p);
}

// The call's types: dtype 0 fp16, 1 bf16, 2 fp32, and whether the residual stream is fp32.
template <typename F>
void with_types(int dtype, bool wide, F&& f) {
  if (dtype == 2) f(float{}, float{});
  else if (dtype == 1 && wide) f(__bf16{}, float{});
  else if (dtype == 1) f(__bf16{}, __bf16{});
  else if (wide) f(_Float16{}, float{});
  else f(_Float16{}, _Float16{});
}

int rows_per_block(const Split& s) { return std::max(256 / s.lanes, 1); }

constexpr int64_t kMaxBlocks = 1 << 20;      // more rows than that many workgroups take in turn
constexpr int64_t kBwdBlocks = 1024;         // workgroups of the backward pass, each a partial of dweight

}  // namespace

int64_t rmsnorm_bwd_partials(int64_t N, int M) {
  const int rpb = rows_per_block(split(M));
  return std::min((N + rpb - 1) / rpb, kBwdBlocks) * rpb;
}

hipError_t launch_rmsnorm_add(const RmsnormParams& p, hipStream_t stream) {
  const Split s = split(p.M);
  RmsnormParams q = p;
  q.lanes = s.lanes;
  const int rpb = rows_per_block(s);
  const dim3 grid((unsigned)std::min(((int64_t)p.N + rpb - 1) / rpb, kMaxBlocks)), block(s.lanes * rpb);
  with_types(p.dtype, p.wide, [&](auto t, auto r) {
    if (p.scales) launch_add<decltype(t), decltype(r), true>(q, s, grid, block, stream);
    else launch_add<decltype(t), decltype(r), false>(q, s, grid, block, stream);
  });
  return hipGetLastError();
}

hipError_t launch_rmsnorm_add_bwd(const RmsnormBwdParams& p, float* dweight, hipStream_t stream) {
  const Split s = split(p.M);
  RmsnormBwdParams q = p;
  q.lanes = s.lanes;
  const int rpb = rows_per_block(s);
  const int64_t parts = rmsnorm_bwd_partials(p.N, p.M);
  with_types(p.dtype, p.wide, [&](auto t, auto r) {
    launch_bwd<decltype(t), decltype(r)>(q, s, dim3((unsigned)(parts / rpb)), dim3(s.lanes * rpb), stream);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !dweight) return e;
  hipLaunchKernelGGL(rmsnorm_dweight_kernel, dim3((p.M + 31) / 32), dim3(256), 0, stream, p.ws, dweight, (int)parts, p.M);
  return hipGetLastError();
}

hipError_t launch_quant8_load(const Quant8LoadParams& p, hipStream_t stream) {
  const int64_t all = (int64_t)p.N * ((p.M + 7) / 8);
  const dim3 grid((unsigned)std::min((all + 255) / 256, kMaxBlocks)), block(256);
  if (p.dtype == 2) hipLaunchKernelGGL((quant8_load_kernel<float>), grid, block, 0, stream, p);
  else if (p.dtype == 1) hipLaunchKernelGGL((quant8_load_kernel<__bf16>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((quant8_load_kernel<_Float16>), grid, block, 0, stream, p);
  return hipGetLastError();
}

}  // namespace attn
