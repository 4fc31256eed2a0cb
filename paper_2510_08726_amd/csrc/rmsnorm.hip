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
constexpr int kMaxSteps = 4;
constexpr int kMaxChunks = kMaxSteps * 8 * kMaxThreads;      // elements of the chunks that a workgroup's lanes hold

// 8 elements as they lie in memory.
template <typename T>
struct Raw {
  static constexpr int W = sizeof(T) / 2;      // 16-byte words
  u32x4 w[W];
};

// 16 bytes at any address that an element may have (the hardware takes them so).
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Packed { u32x4 v; };

// The chunk of a row that a lane holds: 8 columns from `col` on, of which [lo, hi) are the row's.  Without
// ODD (M a multiple of 8) all or none.
template <bool ODD>
struct Chunk {
  int col, lo, hi;
  __device__ __forceinline__ bool whole() const { return ODD ? lo == 0 && hi == 8 : hi == 8; }
  __device__ __forceinline__ bool part() const { return ODD && !whole(); }
};

// Elements at .. at + 7 of p, which has `end` of them; those outside the chunk are anything.  A chunk of part of a row is read
// whole where its memory is the matrix's.
template <typename T, bool ODD>
__device__ __forceinline__ Raw<T> load(const void* ptr, int64_t at, int64_t end, const Chunk<ODD>& c) {
  const T* p = reinterpret_cast<const T*>(ptr) + at;
  Raw<T> r;
#pragma unroll
  for (int k = 0; k < Raw<T>::W; ++k) r.w[k] = u32x4{0u, 0u, 0u, 0u};
  if (c.whole() || (ODD && c.lo < c.hi && at >= 0 && at + 8 <= end)) {
#pragma unroll
    for (int k = 0; k < Raw<T>::W; ++k) r.w[k] = reinterpret_cast<const Packed<T>*>(p + 16 / sizeof(T) * k)->v;
  } else if constexpr (ODD) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < c.lo || i >= c.hi) continue;
      if constexpr (sizeof(T) == 4) r.w[i / 4][i % 4] = reinterpret_cast<const unsigned*>(p)[i];
      else r.w[0][i / 2] |= (unsigned)reinterpret_cast<const unsigned short*>(p)[i] << (16 * (i % 2));
    }
  }
  return r;
}

// Its values, zeros outside the chunk.
template <typename T, bool ODD>
__device__ __forceinline__ void values(const Raw<T>& r, const Chunk<ODD>& c, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      const unsigned a = r.w[0][i], b = r.w[1][i];
      x[i] = __builtin_bit_cast(float, a);
      x[4 + i] = __builtin_bit_cast(float, b);
    } else {
      const unsigned u = r.w[0][i];
      x[2 * i] = Elem<T>::lo(u);
      x[2 * i + 1] = Elem<T>::hi(u);
    }
  }
  if (c.part()) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i >= c.lo && i < c.hi ? x[i] : 0.f;
  }
}

// The chunk's values, rounded to T.
template <typename T, bool ODD>
__device__ __forceinline__ void put8(void* ptr, int64_t index, const Chunk<ODD>& c, const float (&x)[8]) {
  T* at = reinterpret_cast<T*>(ptr) + index;
  if (c.whole()) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = x[4 * k + i];
          w[i] = __builtin_bit_cast(unsigned, f);
        }
        reinterpret_cast<Packed<T>*>(at + 4 * k)->v = w;
      }
    } else {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = Elem<T>::pack2(x[2 * i], x[2 * i + 1]);
      reinterpret_cast<Packed<T>*>(at)->v = w;
    }
  } else if constexpr (ODD) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= c.lo && i < c.hi) at[i] = (T)x[i];
  }
}

// A lane's chunk number i of a row of M that begins `shift` elements behind a multiple of 8: the chunks begin at
// multiples of 8 of the matrix, so that they are whole 16-byte words of a matrix of any M.  (Rows of 5119: 277 us of a
// backward pass over 8191 of them with chunks from the row's first element, whose words lie across two.)
template <bool ODD>
__device__ __forceinline__ Chunk<ODD> chunk_of(int i, int shift, int M) {
  if constexpr (!ODD) return {8 * i, 0, 8 * i < M ? 8 : 0};
  const int col = 8 * i - shift;
  return {col, max(-col, 0), max(min(M - col, 8), 0)};
}

// Elements that a row of M at element `index` of the matrix begins behind a multiple of 8.  Of the few widths of which that
// would take one chunk more than the lanes hold none: their chunks begin at the row's first element.
template <int C>
__device__ __forceinline__ int shift_of(int64_t index, int M) {
  return C == kMaxSteps && M + 7 > kMaxChunks ? 0 : (int)(index & 7);
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

// x of the lane that a DPP control names.
template <int CTRL, typename V>
__device__ __forceinline__ V of_lane(V x) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
  } else {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint64_t lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)b, CTRL, 0xf, 0xf, true);
    const uint64_t hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(V, hi << 32 | lo);
  }
}

// x joined over groups of `n` lanes (4 to 64), each of which gets all of it.  By lane exchanges in the vector unit (six steps of
// an fp64 sum 0.1 us; through LDS 0.4).
template <typename J, typename V>
__device__ __forceinline__ V join_lanes(V x, int n) {
  x = J::join(x, of_lane<0xB1>(x));              // pairs
  x = J::join(x, of_lane<0x4E>(x));              // fours
  if (n > 4) x = J::join(x, of_lane<0x141>(x));  // eights: mirrored, the fours being alike
  if (n > 8) x = J::join(x, of_lane<0x140>(x));  // sixteens
  auto swap = [&](auto&& exchange) __attribute__((always_inline)) {
    if constexpr (sizeof(V) == 4) {
      const auto r = exchange(__builtin_bit_cast(unsigned, x));
      const unsigned a = r[0], b = r[1];
      x = J::join(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b));
    } else {
      const uint64_t v = __builtin_bit_cast(uint64_t, x);
      const auto lo = exchange((unsigned)v), hi = exchange((unsigned)(v >> 32));
      const unsigned a0 = lo[0], a1 = hi[0], b0 = lo[1], b1 = hi[1];
      x = J::join(__builtin_bit_cast(V, (uint64_t)a1 << 32 | a0), __builtin_bit_cast(V, (uint64_t)b1 << 32 | b0));
    }
  };
  if (n > 16) swap([](unsigned u) __attribute__((always_inline)) { return __builtin_amdgcn_permlane16_swap(u, u, false, false); });
  if (n > 32) swap([](unsigned u) __attribute__((always_inline)) { return __builtin_amdgcn_permlane32_swap(u, u, false, false); });
  return x;
}

// Joins x over the `lanes` lanes of a row (of several waves through `shared`, which the caller's next join
// has to differ from).
template <typename J, typename V>
__device__ __forceinline__ V join_row(V x, int lanes, V* shared) {
  x = join_lanes<J>(x, 64);
  if (lanes > 64) {
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    const V* own = shared + threadIdx.x / lanes * (lanes / 64);      // the row's waves
    x = own[0];
    for (int w = 1; w < lanes / 64; ++w) x = J::join(x, own[w]);
  }
  return x;
}

// 1 / x and 1 / sqrt(x) in fp64, by Newton's method from the hardware's estimates: off by an ulp or so, in a
// fifth of the instructions of an exactly rounded division.
__device__ __forceinline__ double inverse(double x) {
  double r = __builtin_amdgcn_rcp(x);
  r = __builtin_fma(__builtin_fma(-x, r, 1.0), r, r);
  return __builtin_fma(__builtin_fma(-x, r, 1.0), r, r);
}
__device__ __forceinline__ double inverse_root(double x) {
  const double y = __builtin_amdgcn_rsq(x);
  double r = y;
  r = __builtin_fma(0.5 * r, __builtin_fma(-x * r, r, 1.0), r);
  r = __builtin_fma(0.5 * r, __builtin_fma(-x * r, r, 1.0), r);
  return x > 0.0 && x < __builtin_inf() ? r : y;
}

// z in fp32, rounded to odd at 20 bits of mantissa (the upper word of z, its last bit set where the lower
// one is not zero), so that a second rounding to fewer bits gives what one rounding of z would.
__device__ __forceinline__ float to_odd(double z) {
  const uint64_t b = __builtin_bit_cast(uint64_t, z);
  const unsigned lo = (unsigned)b;
  const uint64_t odd = (uint64_t)((unsigned)(b >> 32) | (lo < 1u ? lo : 1u)) << 32;
  return (float)__builtin_bit_cast(double, odd);
}

// 8 codes of z, in two words.  (Only under a scale that is no normal number is |z| over the largest code.)
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
        const int c = (int)__builtin_rintf(__builtin_amdgcn_fmed3f(f[i], -127.f, 127.f));
        w[k] |= ((unsigned)c & 255u) << (8 * i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_fmed3f(f[i], -448.f, 448.f);
      w[k] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
      w[k] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], (int)w[k], true);
    }
  }
  return make_uint2(w[0], w[1]);
}

struct __attribute__((packed, aligned(1))) Bytes8 { uint2 v; };

// A row of a matrix as its lanes load and store it: chunk i begins 8 i elements behind the multiple of 8 at or before the
// row, and what a lane does not have, or a row that is not there, needs no branch: the buffer resource ends with the row,
// loads behind it give zeros, and stores are dropped.  Under branches the compiler's waits could not count what is on its
// way, and would wait for all of it, the next rows' words and the stores among them.
template <typename T, bool ODD>
struct Row {
  static constexpr int S = sizeof(T);
  static constexpr int kNowhere = 1 << 30;       // an offset behind any row
  char* base;
  int bytes;
  // The row from element `index` of the matrix on, `shift` behind a multiple of 8.  M = 0: none.
  __device__ __forceinline__ Row(const void* ptr, int64_t index, int shift, int M)
      : base(reinterpret_cast<char*>(const_cast<void*>(ptr)) + (index - shift) * S), bytes(ptr && M > 0 ? (shift + M) * S : 0) {}
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t until(int n) const {
    return __builtin_amdgcn_make_buffer_rsrc(base, 0, n, 0x00027000);
  }

  // Half a word at the row's end is no word of its own: last() has it.
  __device__ __forceinline__ Raw<T> load(int i) const {
    const __amdgpu_buffer_rsrc_t row = until(bytes & ~3);
    Raw<T> r;
#pragma unroll
    for (int k = 0; k < Raw<T>::W; ++k) r.w[k] = __builtin_amdgcn_raw_buffer_load_b128(row, 8 * S * i + 16 * k, 0, 0);
    return r;
  }
  __device__ __forceinline__ unsigned last() const {
    if constexpr (!ODD || S == 4) return 0u;
    else return (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(until(bytes), bytes ? bytes - S : 0, 0, 0);
  }

  // Chunk i, rounded to T: a whole one at once, of part of a row at most 4, 2 and 1 elements, in as many stores for
  // every lane.
  __device__ __forceinline__ void store(int i, const Chunk<ODD>& c, const float (&x)[8]) const {
    const __amdgpu_buffer_rsrc_t row = until(bytes);
    const int at = 8 * S * i;
    words<8>(row, c.whole() ? at : kNowhere, x);
    if constexpr (ODD) {
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = x[k];
      const int n = c.part() ? max(c.hi - c.lo, 0) : 0;
      if (n > 0) {                               // the row's elements to the front
#pragma unroll
        for (int b = 1; b < 8; b *= 2)
          if (c.lo & b) {
#pragma unroll
            for (int k = 0; k + b < 8; ++k) y[k] = y[k + b];
          }
      }
      const int from = at + S * c.lo;
      words<4>(row, n & 4 ? from : kNowhere, y);
      const float two[2] = {n & 4 ? y[4] : y[0], n & 4 ? y[5] : y[1]};
      words<2>(row, n & 2 ? from + S * (n & 4) : kNowhere, two);
      const float one[1] = {n & 4 ? n & 2 ? y[6] : y[4] : n & 2 ? y[2] : y[0]};
      words<1>(row, n & 1 ? from + S * (n & 6) : kNowhere, one);
    }
  }
  // 8 codes.
  __device__ __forceinline__ void store(int i, const Chunk<ODD>& c, uint2 codes) const {
    const __amdgpu_buffer_rsrc_t row = until(bytes);
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{codes.x, codes.y}, row, c.whole() ? 8 * i : kNowhere, 0, 0);
    if constexpr (ODD) {
      const int n = c.part() ? max(c.hi - c.lo, 0) : 0, from = 8 * i + c.lo;
      const uint64_t w = ((uint64_t)codes.y << 32 | codes.x) >> (8 * (c.lo & 7));
      __builtin_amdgcn_raw_buffer_store_b32((unsigned)w, row, n & 4 ? from : kNowhere, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(w >> (8 * (n & 4))), row, n & 2 ? from + (n & 4) : kNowhere, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b8((unsigned char)(w >> (8 * (n & 6))), row, n & 1 ? from + (n & 6) : kNowhere, 0, 0);
    }
  }
  // One element; i < 0: none.
  __device__ __forceinline__ void put(int i, float x) const {
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, x), until(bytes), i < 0 ? kNowhere : S * i, 0, 0);
  }
  template <int N, int K>
  static __device__ __forceinline__ void words(__amdgpu_buffer_rsrc_t row, int at, const float (&x)[K]) {
    unsigned w[N * S / 4 + 1];
    if constexpr (S == 4) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float f = x[k];
        w[k] = __builtin_bit_cast(unsigned, f);
      }
    } else {
#pragma unroll
      for (int k = 0; k < N; k += 2) w[k / 2] = Elem<T>::pack2(x[k], x[k + 1 < N ? k + 1 : k]);
    }
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    if constexpr (N * S >= 16) {
#pragma unroll
      for (int k = 0; k < N * S / 16; ++k)
        __builtin_amdgcn_raw_buffer_store_b128(u32x4{w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]}, row, at + 16 * k, 0, 0);
    } else if constexpr (N * S == 8) {
      __builtin_amdgcn_raw_buffer_store_b64(u32x2{w[0], w[1]}, row, at, 0, 0);
    } else if constexpr (N * S == 4) {
      __builtin_amdgcn_raw_buffer_store_b32(w[0], row, at, 0, 0);
    } else {
      __builtin_amdgcn_raw_buffer_store_b16((unsigned short)w[0], row, at, 0, 0);
    }
  }
};

// The values of a chunk as Row loads it, with the row's last element, of a row that ends at column M.
template <typename T, bool ODD>
__device__ __forceinline__ void values(const Raw<T>& r, unsigned last, int M, const Chunk<ODD>& c, float (&x)[8]) {
  values(r, c, x);
  if constexpr (ODD && sizeof(T) == 2) {
    if (c.part() && c.lo < c.hi && c.col + c.hi == M) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i == c.hi - 1 ? Elem<T>::lo(last) : x[i];
    }
  }
}

// The rows that a lane's place in its workgroup takes: from `first` in steps of `step`, those below `last`.  (A run
// of rows for each XCD instead, so that the words which two rows share pass through one L2, was 3 to 10 % slower, rows
// of 5119 among them.)
struct Turns {
  int64_t first, step, last;
};
__device__ __forceinline__ Turns turns_of(int64_t N, int rpb, int sub) {
  return {(int64_t)blockIdx.x * rpb + sub, (int64_t)gridDim.x * rpb, N};
}

// T: the type of x, the weight and y; R: that of the residual and h.  C: steps of 8 elements a lane.  QUANT: y in 8 bits.  A
// workgroup takes rows in turn, the words of two rows on their way while one is worked on (of one in more steps: of none until
// that one's are stored where QUANT leaves no registers: 4096 rows of 16384 with a scale each 163 us, 206 with them).  For 1024
// lanes there are 128 registers: none is spilled in one step, 22 to 25 in two to 8 bits, 12 to 268 in four.  8192 rows
// of 5120 in bf16 take 62 us, 5.4 TB/s in and out (a large copy 5.1), 8191 of 5119 76, 101 with branches at the rows' ends;
// to 8 bits, 8192 of 8192 95 us with a scale for each 128 (102 to 108 under a profiler, which keeps the calls apart), 120 with one row ahead.  That is bound by
// fp64 (the codes are those of the exact quotients), and a scale a row by its second join as well: 125 (127 with h taken
// through fp64 twice, as more steps of a lane do).
template <typename T, typename R, int C, bool QUANT, bool ODD>
__global__ __launch_bounds__(kMaxThreads) void rmsnorm_add_kernel(RmsnormParams p) {
  constexpr bool LATE = QUANT && C > 1;          // (no registers for it beside the fp64 values)
  __shared__ double sums[2][kMaxWaves];
  __shared__ double tops[2][kMaxWaves];
  const int lanes = p.lanes, rpb = blockDim.x / lanes;
  const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / lanes), t = threadIdx.x % lanes;
  const int M = p.M;
  const Turns turns = turns_of(p.N, rpb, sub);
  // Of all its rows: a lane's columns stay the same.  (Groups begin at a chunk's first element.)
  const int shift = !ODD || (QUANT && p.group) ? 0 : shift_of<C>(turns.first * M, M);
  Raw<T> weight[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const auto k = chunk_of<ODD>(c * lanes + t, shift, M);
    if (p.weight) weight[c] = load<T>(p.weight, k.col, M, k);
  }
  struct Words {
    Raw<T> x[C];
    Raw<R> r[C];
    unsigned x_last, r_last;
  };
  auto fetch = [&](int64_t row, Words& w) __attribute__((always_inline)) {
    const int m = row < turns.last ? M : 0;
    const Row<T, ODD> x(p.x, row * M, shift, m);
    const Row<R, ODD> r(p.residual, row * M, shift, m);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      w.x[c] = x.load(c * lanes + t);
      w.r[c] = r.load(c * lanes + t);
    }
    w.x_last = x.last();
    w.r_last = r.last();
  };
  int turn = 0;
  // One row.  As its words are taken apart, those of the row `ahead` take their place.
  auto one = [&](int64_t row, int64_t ahead, Words& now) __attribute__((always_inline)) {
    const int m = row < turns.last ? M : 0;
    auto chunk = [&](int c) __attribute__((always_inline)) { return chunk_of<ODD>(c * lanes + t, shift, m); };
    float h[C][8];
    double ss = 0.0;
    const Row<R, ODD> stream(p.residual ? p.h : nullptr, row * M, shift, m);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const auto k = chunk(c);
      float y[8];
      values(now.x[c], now.x_last, M, k, h[c]);
      values(now.r[c], now.r_last, M, k, y);
      if (p.residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] += y[i];
      }
    }
    if constexpr (!LATE) fetch(ahead, now);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      stream.store(c * lanes + t, chunk(c), h[c]);
      if (p.residual) round8<R>(h[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)h[c][i], (double)h[c][i], ss);
    ss = join_row<Sum>(ss, lanes, sums[turn]);
    const double rstd = inverse_root(__builtin_fma(ss, p.inv, p.eps));
    Row<float, false>(p.rstd, row, 0, m ? 1 : 0).put(t == 0 ? 0 : -1, (float)rstd);
    turn ^= 1;                                   // (of the tops behind it too)
    if constexpr (!QUANT) {
      const float r = (float)rstd;
      const Row<T, ODD> out(p.y, row * M, shift, m);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const auto k = chunk(c);
        float w[8], y[8];
        values(weight[c], k, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = p.weight ? h[c][i] * r * (w[i] + p.offset) : h[c][i] * r;
        out.store(c * lanes + t, k, y);
      }
    } else {
      const double unit = p.int8 ? rstd * (1.0 / 127.0) : rstd * (1.0 / 448.0);
      const int G = p.group;
      auto weighed = [&](int c, double (&z)[8]) __attribute__((always_inline)) {    // h (w + offset)
        float w[8];
        if (p.weight) {
          values(weight[c], chunk(c), w);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = (double)h[c][i] * ((double)w[i] + (double)p.offset);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = (double)h[c][i];
        }
      };
      // The largest magnitude, NaN where one of them is an infinity or NaN.
      auto largest = [](const double (&z)[8]) __attribute__((always_inline)) {
        double a = __builtin_fabs(z[0]), bad = z[0] * 0.0;
#pragma unroll
        for (int i = 1; i < 8; ++i) {
          a = __builtin_fmax(a, __builtin_fabs(z[i]));
          bad = __builtin_fma(z[i], 0.0, bad);
        }
        return __builtin_fabs(a + bad);
      };
      // rstd over the scale of a group whose largest |h (w + offset)| is a; 0 where its codes are zeros.
      const Row<float, false> scales(p.scales, row * p.groups, 0, m ? p.groups : 0);
      auto scaled = [&](double a, int at) __attribute__((always_inline)) {
        float s = (float)(a * unit);
        const bool fine = s <= 3.4028234663852886e38f;     // (not an infinity or NaN)
        if (!fine) s = __builtin_nanf("");
        scales.put(at, s);
        return fine && s > 0.f ? rstd * inverse((double)s) : 0.0;
      };
      const Row<unsigned char, ODD> codes(p.y, row * M, shift, m);
      auto put = [&](int c, double (&z)[8], double g) __attribute__((always_inline)) {
        const auto k = chunk(c);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= g;
        const uint2 w = g == 0.0 ? make_uint2(0u, 0u) : codes8(z, p.int8);
        codes.store(c * lanes + t, k, w);
      };
      if (G == 0) {
        if constexpr (C == 1) {
          double z[8];
          weighed(0, z);
          const double top = join_row<Most>(largest(z), lanes, tops[turn]);
          put(0, z, scaled(top, t == 0 ? 0 : -1));
        } else {                                 // (h (w + offset) twice: there are no registers for all of it in 64 bits)
          double top = 0.0;
#pragma unroll
          for (int c = 0; c < C; ++c) {
            double z[8];
            weighed(c, z);
            top = Most::join(top, largest(z));
          }
          top = join_row<Most>(top, lanes, tops[turn]);
          const double g = scaled(top, t == 0 ? 0 : -1);
#pragma unroll
          for (int c = 0; c < C; ++c) {
            double z[8];
            weighed(c, z);
            put(c, z, g);
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int col = 8 * (c * lanes + t);
          double z[8];
          weighed(c, z);
          double a = largest(z);
          a = join_lanes<Most>(a, G / 8);
          put(c, z, scaled(a, col < m && col % G == 0 ? col / G : -1));
        }
      }
    }
    if constexpr (LATE) fetch(ahead, now);
  };
  Words a, b;
  int64_t row = turns.first;
  fetch(row, a);
  if constexpr (C == 1) {
    __builtin_amdgcn_sched_barrier(0);           // (as below)
    fetch(row + turns.step, b);
    __builtin_amdgcn_sched_barrier(0);
    for (;; row += 2 * turns.step) {             // (all rows of a workgroup take as many turns as its first)
      one(row, row + 2 * turns.step, a);
      if (row - sub + turns.step >= turns.last) break;
      one(row + turns.step, row + 3 * turns.step, b);
      if (row - sub + 2 * turns.step >= turns.last) break;
    }
  } else {
    for (; row - sub < turns.last; row += turns.step) one(row, row + turns.step, a);
  }
}

// Gradients.  A workgroup takes rows in turn, and its lanes keep the sum of dY n of their columns over
// them: [workgroups, M] in fp32, summed by rmsnorm_dweight_kernel in a fixed order.  Two rows of words are on their way while
// one is worked on: 8192 rows of 5120 in bf16 take 66 us, 5.1 TB/s in and out as a large copy has, 87 with one ahead.
// 8191 of 5119 take 85; 98 with branches at the rows' ends in place of Row.  In more steps of a lane the next row's words come
// behind one's stores (4096 rows of 12289 97 us, 2048 of 32768 222; 125 and 387 as soon as that one's are taken apart, which
// spills more: as it is 3 to 5 registers in two steps of odd widths, 69 to 404 in four).
template <typename T, typename R, int C, bool ODD>
__global__ __launch_bounds__(kMaxThreads) void rmsnorm_add_bwd_kernel(RmsnormBwdParams p) {
  __shared__ float sums[2][kMaxWaves];
  __shared__ float joined[C == 1 ? 2048 : 1];      // rpb rows of at most 64 or 128 lanes
  const int lanes = p.lanes, rpb = blockDim.x / lanes;
  const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / lanes), t = threadIdx.x % lanes;
  const int M = p.M;
  const Turns turns = turns_of(p.N, rpb, sub);
  const int shift = ODD ? shift_of<C>(turns.first * M, M) : 0;       // of all its rows: a lane's columns stay the same
  auto chunk = [&](int c, bool in) __attribute__((always_inline)) { return chunk_of<ODD>(c * lanes + t, shift, in ? M : 0); };
  float dw[C][8];
  Raw<T> weight[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const auto k = chunk(c, true);
    if (p.weight) weight[c] = load<T>(p.weight, k.col, M, k);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[c][i] = 0.f;
  }
  struct Words {
    Raw<T> dy[C];
    Raw<R> h[C], dh[C];
    unsigned dy_last, h_last, dh_last;
    float rstd;
  };
  auto fetch = [&](int64_t row, Words& w) __attribute__((always_inline)) {
    const int m = row < turns.last ? M : 0;
    const Row<T, ODD> dy(p.dy, row * M, shift, m);
    const Row<R, ODD> h(p.h, row * M, shift, m);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      w.dy[c] = dy.load(c * lanes + t);
      w.h[c] = h.load(c * lanes + t);
    }
    w.dy_last = dy.last();
    w.h_last = h.last();
    w.rstd = p.rstd[min(row, turns.last - 1)];
  };
  auto fetch_dh = [&](int64_t row, Words& w) __attribute__((always_inline)) {
    const Row<R, ODD> dh(p.dh, row * M, shift, row < turns.last ? M : 0);
#pragma unroll
    for (int c = 0; c < C; ++c) w.dh[c] = dh.load(c * lanes + t);
    w.dh_last = dh.last();
  };
  int turn = 0;
  // One row.  As its words are taken apart, those of the row `ahead` take their place.
  auto one = [&](int64_t row, int64_t ahead, Words& now) __attribute__((always_inline)) {
    const bool in = row < turns.last;
    const float r = in ? now.rstd : 0.f;
    float g[C][8], n[C][8];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const auto k = chunk(c, in);
      float w[8];
      values(now.dy[c], now.dy_last, M, k, g[c]);
      values(now.h[c], now.h_last, M, k, n[c]);
      values(weight[c], k, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        n[c][i] *= r;
        dw[c][i] = __builtin_fmaf(g[c][i], n[c][i], dw[c][i]);
        if (p.weight) g[c][i] *= w[i] + p.offset;
        s = __builtin_fmaf(g[c][i], n[c][i], s);
      }
    }
    if constexpr (C == 1) fetch(ahead, now);
    s = join_row<Sum>(s, lanes, sums[turn]) / (float)M;
    turn ^= 1;
    const Row<R, ODD> dresidual(p.dresidual, row * M, shift, in ? M : 0);
    const Row<T, ODD> dx(p.dx, row * M, shift, in ? M : 0);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const auto k = chunk(c, in);
      float d[8];
      values(now.dh[c], now.dh_last, M, k, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = r * __builtin_fmaf(-n[c][i], s, g[c][i]);
        d[i] = p.dh ? d[i] + x : x;
      }
      dresidual.store(c * lanes + t, k, d);
      dx.store(c * lanes + t, k, d);
    }
    if constexpr (C > 1) fetch(ahead, now);
    fetch_dh(ahead, now);
  };
  Words a, b;
  int64_t row = turns.first;
  fetch(row, a);
  fetch_dh(row, a);
  if constexpr (C == 1) {
    // (In this order, for the waits that the loop begins with.)
    __builtin_amdgcn_sched_barrier(0);
    fetch(row + turns.step, b);
    fetch_dh(row + turns.step, b);
    __builtin_amdgcn_sched_barrier(0);
    for (;; row += 2 * turns.step) {
      one(row, row + 2 * turns.step, a);
      if (row - sub + turns.step >= turns.last) break;
      one(row + turns.step, row + 3 * turns.step, b);
      if (row - sub + 2 * turns.step >= turns.last) break;
    }
  } else {
    for (; row - sub < turns.last; row += turns.step) one(row, row + turns.step, a);
  }
  if (!p.ws) return;
  float* at = p.ws + (int64_t)blockIdx.x * M;
  if (C > 1 || rpb == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) put8<float>(at, chunk(c, true).col, chunk(c, true), dw[c]);
    return;
  }
  // Several rows at a time: their sums are joined first.
  const auto k = chunk(0, true);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i >= k.lo && i < k.hi) joined[sub * M + k.col + i] = dw[0][i];
  __syncthreads();
  for (int i = threadIdx.x; i < M; i += blockDim.x) {
    float x = joined[i];
    for (int u = 1; u < rpb; ++u) x += joined[u * M + i];
    at[i] = x;
  }
}

// Columns summed over the partials: 32 columns a workgroup, every eighth partial a row of lanes.  256 of 5119 take
// 4.1 us, the latency of four loads one after the other.
__global__ __launch_bounds__(256) void rmsnorm_dweight_kernel(const float* ws, float* out, int parts, int M) {
  __shared__ float part[8][32];
  const int col = blockIdx.x * 32 + threadIdx.x % 32, k = threadIdx.x / 32;
  float s = 0.f;
  if (col < M) {
    int i = k;
    for (; i + 56 < parts; i += 64) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = ws[(int64_t)(i + 8 * u) * M + col];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += x[u];
    }
    for (; i < parts; i += 8) s += ws[(int64_t)i * M + col];
  }
  part[k][threadIdx.x % 32] = s;
  __syncthreads();
  if (k == 0 && col < M) {
    for (int i = 1; i < 8; ++i) s += part[i][threadIdx.x];
    out[col] = s;
  }
}

// What codes stand for: 8 of them a lane.  Bound by memory: 8192 x 8192 to bf16 (203 MB) 35 us, 5.8 TB/s.
template <typename T, bool ODD>
__global__ __launch_bounds__(256) void quant8_load_kernel(Quant8LoadParams p) {
  const int chunks = (ODD && !p.group ? p.M + 14 : p.M + 7) / 8;
  const int64_t all = (int64_t)p.N * chunks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / chunks, base = row * p.M;
    const auto c = chunk_of<ODD>((int)(i - row * chunks), p.group ? 0 : (int)(base & 7), p.M);
    if (c.lo >= c.hi) continue;
    const unsigned char* at = p.codes + base + c.col;
    unsigned w[2] = {0u, 0u};
    if (c.whole()) {
      const uint2 v = reinterpret_cast<const Bytes8*>(at)->v;
      w[0] = v.x;
      w[1] = v.y;
    } else {
      for (int k = c.lo; k < c.hi; ++k) w[k / 4] |= (unsigned)at[k] << (8 * (k & 3));
    }
    const float s = p.scales[row * p.groups + (p.group ? c.col / p.group : 0)];
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const unsigned b = w[k / 4] >> (8 * (k & 3));
      y[k] = s * (p.int8 ? (float)(signed char)(b & 255u) : __builtin_amdgcn_cvt_f32_fp8((int)b, 0));
    }
    put8<T>(p.y, base + c.col, c, y);
  }
}

// Lanes of a row, and steps of 8 elements of a lane.
struct Split {
  int lanes, steps;
};
// By the row's length alone, so that a row's bits do not depend on how many there are.  One step of a lane
// up to 8192 elements, by as many waves as it takes.
Split split(int M) {
  const int m = M % 8 && M + 7 <= kMaxChunks ? M + 7 : M;      // (a row may begin within a chunk: shift_of)
  const int s = (m + 8 * kMaxThreads - 1) / (8 * kMaxThreads), steps = s <= 2 ? s : kMaxSteps;
  return {((m + 8 * steps - 1) / (8 * steps) + 63) / 64 * 64, steps};
}

template <typename T, typename R, bool QUANT, bool ODD>
void launch_add(const RmsnormParams& p, const Split& s, dim3 grid, dim3 block, hipStream_t stream) {
  if (s.steps == 1) hipLaunchKernelGGL((rmsnorm_add_kernel<T, R, 1, QUANT, ODD>), grid, block, 0, stream, p);
  else if (s.steps == 2) hipLaunchKernelGGL((rmsnorm_add_kernel<T, R, 2, QUANT, ODD>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((rmsnorm_add_kernel<T, R, 4, QUANT, ODD>), grid, block, 0, stream, p);
}

template <typename T, typename R, bool ODD>
void launch_bwd(const RmsnormBwdParams& p, const Split& s, dim3 grid, dim3 block, hipStream_t stream) {
  if (s.steps == 1) hipLaunchKernelGGL((rmsnorm_add_bwd_kernel<T, R, 1, ODD>), grid, block, 0, stream, p);
  else if (s.steps == 2) hipLaunchKernelGGL((rmsnorm_add_bwd_kernel<T, R, 2, ODD>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((rmsnorm_add_bwd_kernel<T, R, 4, ODD>), grid, block, 0, stream, p);
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

// Rows of a workgroup: of at least 256 lanes, where that many divide alike.
int rows_per_block(const Split& s) { return s.lanes == 64 ? 4 : s.lanes == 128 ? 2 : 1; }

// Workgroups that take rows in turn: as many as 256 compute units hold at a time with `hold` waves each, a multiple of 8.
int64_t resident(const Split& s, int hold) {
  const int waves = s.lanes * rows_per_block(s) / 64;
  return 256 * std::max(hold / waves, 1);
}

}  // namespace

int64_t rmsnorm_bwd_partials(int64_t N, int M) {
  const Split s = split(M);
  const int rpb = rows_per_block(s);
  // 8 waves, or one workgroup: 16384 rows of 4096 100 us (109 with 16), of 1024 29 (34; 34 with 6).
  return std::min((N + rpb - 1) / rpb, resident(s, 8));
}

hipError_t launch_rmsnorm_add(const RmsnormParams& p, hipStream_t stream) {
  const Split s = split(p.M);
  RmsnormParams q = p;
  q.lanes = s.lanes;
  q.inv = 1.0 / p.M;
  const int rpb = rows_per_block(s);
  // 8 waves a compute unit, or one workgroup: 16384 rows of 4096 94 us, 101 with 16.  To 8 bits 16: 108, with 8 144.
  const dim3 grid((unsigned)std::min(((int64_t)p.N + rpb - 1) / rpb, resident(s, p.scales ? 16 : 8))), block(s.lanes * rpb);
  with_types(p.dtype, p.wide, [&](auto t, auto r) {
    typedef decltype(t) T;
    typedef decltype(r) R;
    if (p.M % 8 == 0) {
      if (p.scales) launch_add<T, R, true, false>(q, s, grid, block, stream);
      else launch_add<T, R, false, false>(q, s, grid, block, stream);
    } else {
      if (p.scales) launch_add<T, R, true, true>(q, s, grid, block, stream);
      else launch_add<T, R, false, true>(q, s, grid, block, stream);
    }
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
    const dim3 grid((unsigned)parts), block(s.lanes * rpb);
    if (p.M % 8 == 0) launch_bwd<decltype(t), decltype(r), false>(q, s, grid, block, stream);
    else launch_bwd<decltype(t), decltype(r), true>(q, s, grid, block, stream);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !dweight) return e;
  hipLaunchKernelGGL(rmsnorm_dweight_kernel, dim3((p.M + 31) / 32), dim3(256), 0, stream, p.ws, dweight, (int)parts, p.M);
  return hipGetLastError();
}

hipError_t launch_quant8_load(const Quant8LoadParams& p, hipStream_t stream) {
  const int64_t all = (int64_t)p.N * ((p.M % 8 && !p.group ? p.M + 14 : p.M + 7) / 8);
  const dim3 grid((unsigned)std::min((all + 255) / 256, (int64_t)1 << 20)), block(256);     // (more chunks in turn)
  with_types(p.dtype, false, [&](auto t, auto) {
    if (p.M % 8 == 0) hipLaunchKernelGGL((quant8_load_kernel<decltype(t), false>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((quant8_load_kernel<decltype(t), true>), grid, block, 0, stream, p);
  });
  return hipGetLastError();
}

}  // namespace attn
