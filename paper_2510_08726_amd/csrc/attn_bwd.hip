// Attention's backward pass for gfx950 (include/attn_bwd.h).  With the scores
// s = mod(scale q k^T) + bias and each row's log-sum-exp from the forward pass,
//
//   P = exp(s - lse)                  recomputed, never in memory
//   dV = P^T dO
//   dS = P (dO V^T - delta) mod'(s) scale,   delta_i = dO_i . O_i
//   dQ = dS K,  dK = dS^T Q           dK and dV summed over the query heads of a KV head
//
// Three kernels, without atomics, so that a call's bits do not depend on timing:
//   bwd_rows_kernel  what a row brings into its scores: (delta, lse), once
//   bwd_kernel       dkv_block: a workgroup owns 128 keys and streams the tiles of 32 queries that see them;
//                    dq_block: a workgroup owns 128 query rows and streams the tiles of 32 keys
//   bwd_sum_kernel   adds up the blocks that were divided into parts, where few blocks are long
// Both kinds of blocks form S and dP, seven products in the place of five (and dQ's in two halves, below).  (One loop for
// both would need the partial dQ of every key block in memory, 1 KB a row and block of 256 keys
// against 131 kflop saved: no less time at this card's rates, and a sum over blocks.)
//
// A wave owns 32 keys (or rows) for the whole loop, 32x32x16 MFMAs with fp32
// accumulators in registers; Q and dO (or K and V) tiles pass through LDS, swizzled
// as prefill.hip's, filled by buffer loads that write LDS directly.  The products
// are arranged so that the lane is the wave's own index (key or row): S and dP come out in the
// layout in which P and dS go into the second products, in registers alone.
//
// Rounding.  P and dS go to the matrix unit in the type of Q: 2^-9 (bf16) or 2^-12 (fp16) relative to
// each, as much as the outputs' own rounding.  That holds for dV and dK (1.4 times the error that a
// result rounded once has).  dQ's sums cancel more, since the dS of a row sum to nothing, and
// with dS rounded once it was off by 1.5 times that error: there dS goes in as two values of the type, the
// second what the first leaves (1.00 times, for an eighth more time: 32 heads of 8192 causal rows 1856 us in
// place of 1649).  Sums are in fp32.  fp16 holds 5
// exponent bits, and both get small in long rows (dS also with the loss's scale), so there P is
// held times 2^15 and dS times a power of two from a bound on |dO| |V| of its KV head
// (bwd_scale), taken out of the fp32 sums at the end.

#include <algorithm>
#include <type_traits>
#include <utility>

#include "kernel_common.h"
#include "launch.h"

namespace attn {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int TN = 32;                  // rows of a streamed tile, and of a wave's own block
constexpr int BLK = TN * kWaves;        // keys (rows) that a workgroup owns
constexpr int kXcds = 8;
constexpr int kRowsBlock = 64;          // rows of a workgroup of bwd_rows_kernel
constexpr int kShift = 15;              // fp16: P is held times 2^kShift
constexpr double kLog2e64 = 1.4426950408889634;

typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
typedef __attribute__((address_space(3))) float lds_float;

template <typename T> constexpr bool is_half = std::is_same_v<T, _Float16>;

// A tile of 32 rows of D 16-bit values in LDS, 16-byte chunks swizzled (swz).
template <int D, typename T>
struct Tile {
  typedef typename Elem<T>::vec8 vec8;
  static constexpr int BYTES = TN * D * 2;
  static constexpr int NBLK = BYTES / 1024;     // 1 KB copies
  static constexpr int CPR = D / 8;             // 16-byte chunks of a row
  static constexpr int KX = D / 16;             // MFMA steps over D
  static constexpr int DB = D / 32;             // 32-dim blocks
  // Operand with the rows along M (or N) and the dims along K, step kx: lane (n, hh)
  // reads row n, dims 16 kx + 8 hh ...  row_offset is the lane's LDS address for step 0 of a tile at 0; step kx
  // is at its xor with 32 kx, which leaves the tile's own address (a multiple of 256) alone.
  static __device__ __forceinline__ int row_offset(int lane) {
    const int n = lane & 31, hh = lane >> 5;
    return 2 * n * D + 16 * (hh ^ swz<D>(n));
  }
  template <int KX0>
  static __device__ __forceinline__ vec8 rows(uint32_t at, int imm) {
    return __builtin_bit_cast(vec8, *(lds_u32x4*)(uintptr_t)(flip<32 * KX0>(at) + imm));
  }
  // Operand with the dims along M and the rows along K: block db, rows 16 c16 ..:
  // lane (m, hh) receives rows 16 c16 + 4 hh + 0..3 and 16 c16 + 8 + 4 hh + 0..3 of dim 32 db + m, the
  // order in which an accumulator of 32 rows by 32 holds them.
  static __device__ __forceinline__ int dim_offset(int lane) {
    const int G = lane >> 4, i = lane & 15;
    const int d = 16 * (G & 1) + 4 * (i & 3), k = 4 * (G >> 1) + (i >> 2);
    return 2 * k * D + 16 * ((d >> 3) ^ swz<D>(k)) + 2 * (d & 7);
  }
  template <int C16, int DB0>
  static __device__ __forceinline__ vec8 dims(uint32_t at, int imm) {
    const uint2 lo = read_tr(flip<64 * DB0>(at) + imm + C16 * 32 * D);
    const uint2 hi = read_tr(flip<64 * DB0 ^ 32>(at) + imm + C16 * 32 * D + 16 * D);
    return __builtin_bit_cast(vec8, make_uint4(lo.x, lo.y, hi.x, hi.y));
  }
  // at ^ X, here and now: as an ordinary expression the compiler computes all of a tile's addresses before the
  // loop and keeps them in registers that the loop does not have.
  template <int X>
  static __device__ __forceinline__ uint32_t flip(uint32_t at) {
    if constexpr (X == 0) return at;
    uint32_t r;
    asm volatile("v_xor_b32 %0, %2, %1" : "=v"(r) : "v"(at), "n"(X));
    return r;
  }
  static __device__ __forceinline__ uint2 read_tr(uint32_t at) {
    const v4s r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(uintptr_t)at);
    return __builtin_bit_cast(uint2, r);
  }
};

template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  [&]<int... Is>(std::integer_sequence<int, Is...>) { (f(std::integral_constant<int, Is>{}), ...); }(
      std::make_integer_sequence<int, N>{});
}

// Rows of an accumulator: register r of lane (n, hh) is row kconst(r) + 4 hh of column n.
constexpr __host__ __device__ int kconst(int r) { return 8 * (r / 4) + r % 4; }

__device__ __forceinline__ u32x4 resource(const void* base, unsigned bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu)),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}

// 16 (or 4) bytes a lane from `off` of a resource to LDS address dst + 16 (4) lane;
// past the resource's end zeros.
__device__ __forceinline__ void copy16(const u32x4& rs, uint32_t dst, int off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               : : "s"(__builtin_amdgcn_readfirstlane((int)dst)), "v"(off), "s"(rs) : "memory", "m0");
}
__device__ __forceinline__ void copy4(const u32x4& rs, uint32_t dst, int off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               : : "s"(__builtin_amdgcn_readfirstlane((int)dst)), "v"(off), "s"(rs) : "memory", "m0");
}

template <typename T>
__device__ __forceinline__ typename Elem<T>::vec8 load8(const T* at, unsigned sign = 0) {
  u32x4 w = *reinterpret_cast<const u32x4*>(at);
  w ^= sign;
  return __builtin_bit_cast(typename Elem<T>::vec8, w);
}

// 32 x 32 weights of a wave as two operands of 16 rows.
template <typename T>
struct Weights {
  uint32_t w[2][4];
  __device__ __forceinline__ void set(int r, float a, float b) { w[r / 8][(r % 8) / 2] = Elem<T>::pack2(a, b); }
  // What that leaves of a and b.
  __device__ __forceinline__ void rest(const Weights& of, int r, float a, float b) {
    const uint32_t u = of.w[r / 8][(r % 8) / 2];
    set(r, a - Elem<T>::lo(u), b - Elem<T>::hi(u));
  }
  __device__ __forceinline__ typename Elem<T>::vec8 operand(int c16) const {
    return __builtin_bit_cast(typename Elem<T>::vec8, make_uint4(w[c16][0], w[c16][1], w[c16][2], w[c16][3]));
  }
};

// SoftCap of a score x: the exponent of its weight, cap tanh(s / cap) log2 e - lse log2 e, where `add` is cap log2 e
// less the latter, and a quarter of the derivative of the cap: 1 - tanh^2 = 4 r (1 - r) with r = 1 / (1 + e^2t).
__device__ __forceinline__ float capped(float x, const BwdParams& p, float add, float& quarter) {
  const float r = __builtin_amdgcn_rcpf(1.f + fast_exp2(x * p.cap_k2));
  quarter = __builtin_fmaf(-r, r, r);
  return __builtin_fmaf(-2.f * p.cap_cl, r, add);
}

// What item of `n` workgroup g takes: an XCD a contiguous share (workgroup g runs on XCD g mod
// 8), so that those that read the same rows share its L2; -1 for none.
__device__ __forceinline__ int item_of(int g, int n, bool shares) {
  if (!shares) return g < n ? g : -1;
  const int x = g % kXcds;
  const int s0 = (int)((long long)n * x / kXcds), s1 = (int)((long long)n * (x + 1) / kXcds);
  const int i = s0 + g / kXcds;
  return i < s1 ? i : -1;
}

// The block and the part of it that is number r of a unit's list, and its first piece (of the blocks in several parts).
struct Place {
  int block, part, parts, piece;
};
__device__ __forceinline__ Place place_of(const BwdSplit& s, int r) {
  if (s.multi == 0) return {r, 0, 1, 0};
  int block = 0, piece = 0;
  for (;; ++block) {
    const int n = s.parts[block];
    if (r < n) return {block, r, n, piece};
    r -= n;
    piece += n > 1 ? n : 0;
  }
}

// fp16: the power of two that dS is held times, as an exponent: |dS| <= 2 |dO| |V| of the
// largest rows of the KV head stays below 2^15.  The workgroup's threads each look at a part of the rows'
// largest squares.
template <typename T>
__device__ __forceinline__ int bwd_scale(const BwdParams& p, int unit, float* shared) {
  if constexpr (!is_half<T>) return 0;
  const int nq = p.group * p.row_blocks, nk = p.key_blocks;
  const float* a = p.peaks + (size_t)unit * nq;
  const float* b = p.peaks + (size_t)p.B * p.Hq * p.row_blocks + (size_t)unit * nk;
  float x = 0.f, y = 0.f;
  for (int i = threadIdx.x; i < nq; i += kThreads) x = fmaxf(x, a[i]);
  for (int i = threadIdx.x; i < nk; i += kThreads) y = fmaxf(y, b[i]);
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) {
    x = fmaxf(x, __shfl_xor(x, m, 64));
    y = fmaxf(y, __shfl_xor(y, m, 64));
  }
  if ((threadIdx.x & 63) == 0) {
    shared[threadIdx.x / 64] = x;
    shared[kWaves + threadIdx.x / 64] = y;
  }
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    x = fmaxf(x, shared[w]);
    y = fmaxf(y, shared[kWaves + w]);
  }
  __syncthreads();
  const float bound = 2.02f * __builtin_sqrtf(x) * __builtin_sqrtf(y);
  if (!(bound > 0.f && bound < 3e38f)) return 0;
  return __builtin_amdgcn_readfirstlane(min(max(14 - __builtin_amdgcn_frexp_expf(bound), -100), 100));
}

// A row's part of its scores and of dP, in tiles of 32 rows: [B Hq, tiles, 64] floats,
// first what is added to a score before its exponential, (2^15's exponent - lse log2 e) over the scale, so that it starts the
// accumulator of Q K^T (with SoftCap: not over the scale, and with the cap: see capped; with ALiBi what the bias at
// the tile's origin leaves of lse, by a difference in 64 bits, for lse is as large as the bias: alibi_origin); then -delta, which starts that of dO V^T.  fp16: the largest square sums of
// the rows of dO and V in each block of 64.  Rows that see no key (the first Lq - Lk with the causal mask)
// take no part: their dQ is zero.  One pass over dO and O: bound by memory, 32 heads of 8192 rows of 128 in bf16 (134 MB) 28 us,
// 4.8 TB/s.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void bwd_rows_kernel(BwdParams p) {
  constexpr int LANES = D / 8, RPP = kThreads / LANES;     // lanes of a row, rows of a pass
  __shared__ float top[kWaves];
  const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  const int nheads = p.B * p.Hq, nkv = p.B * p.Hkv;
  int blk = blockIdx.x;
  float peak = 0.f;
  float* peak_at = nullptr;
  if (blk < nheads * p.row_blocks) {
    const int head = blk / p.row_blocks, b = head / p.Hq, h = head - b * p.Hq;
    const int i0 = (blk - head * p.row_blocks) * kRowsBlock;
    peak_at = p.peaks + blk;
    const float slope = p.slopes ? p.slopes[h] : 0.f;
    const AlibiOrigin o = alibi_origin(slope, p.causal, p.window, p.Lk);
    const T* og = reinterpret_cast<const T*>(p.o) + ((size_t)head * p.Lq + p.row0) * D + 8 * lane;
    const T* dg = reinterpret_cast<const T*>(p.d_o) + b * p.do_sb + h * p.do_sh + p.row0 * p.do_sl + 8 * lane;
#pragma unroll
    for (int u = 0; u < kRowsBlock / RPP; ++u) {
      const int i = i0 + u * RPP + sub, row = min(i, p.rows - 1);
      const u32x4 x = *reinterpret_cast<const u32x4*>(og + (size_t)row * D);
      const u32x4 y = *reinterpret_cast<const u32x4*>(dg + (int64_t)row * p.do_sl);
      float dot = 0.f, sq = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned xw = x[k], yw = y[k];
        const float ylo = Elem<T>::lo(yw), yhi = Elem<T>::hi(yw);
        dot = __builtin_fmaf(ylo, Elem<T>::lo(xw), dot);
        dot = __builtin_fmaf(yhi, Elem<T>::hi(xw), dot);
        if (is_half<T>) sq = __builtin_fmaf(ylo, ylo, __builtin_fmaf(yhi, yhi, sq));
      }
#pragma unroll
      for (int m = LANES / 2; m > 0; m >>= 1) {
        dot += __shfl_xor(dot, m, 64);
        if (is_half<T>) sq += __shfl_xor(sq, m, 64);
      }
      peak = fmaxf(peak, sq);
      if (lane == 0 && i < p.row_tiles * TN) {
        float start = kNegInf, nd = 0.f;
        if (i < p.rows) {
          const float lse = p.lse[(size_t)head * p.Lq + p.row0 + i];
          constexpr float shift = is_half<T> ? (float)kShift : 0.f;
          float e = shift - lse * kLog2e;
          if (p.slopes) {
            const int at = p.Lk - p.rows + i;     // off + i
            const double rest = (double)slope * (double)-from_origin(at, at - i % TN, o, p.causal) - (double)lse;
            e = (float)(rest * kLog2e64 + (double)shift);
          }
          e = p.cap_cl == 0.f ? e / p.c : e + p.cap_cl;
          start = lse == kNegInf ? kNegInf : e;
          nd = -dot;
        }
        float* at = p.stats + ((size_t)head * p.row_tiles + i / TN) * (2 * TN) + i % TN;
        at[0] = start;
        at[TN] = nd;
      }
    }
  } else if (is_half<T> && (blk -= nheads * p.row_blocks) < nkv * p.key_blocks) {
    const int unit = blk / p.key_blocks, j0 = (blk - unit * p.key_blocks) * kRowsBlock;
    peak_at = p.peaks + (size_t)nheads * p.row_blocks + blk;
    const T* vg = reinterpret_cast<const T*>(p.v) + (size_t)unit * p.Lk * D + 8 * lane;
#pragma unroll
    for (int u = 0; u < kRowsBlock / RPP; ++u) {
      const u32x4 y = *reinterpret_cast<const u32x4*>(vg + (size_t)min(j0 + u * RPP + sub, p.Lk - 1) * D);
      float sq = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned yw = y[k];
        const float ylo = Elem<T>::lo(yw), yhi = Elem<T>::hi(yw);
        sq = __builtin_fmaf(ylo, ylo, __builtin_fmaf(yhi, yhi, sq));
      }
#pragma unroll
      for (int m = LANES / 2; m > 0; m >>= 1) sq += __shfl_xor(sq, m, 64);
      peak = fmaxf(peak, sq);
    }
  } else {
    if (is_half<T>) blk -= nkv * p.key_blocks;
    else blk -= nheads * p.row_blocks;
    const int per = (p.row0 + kRowsBlock - 1) / kRowsBlock;
    const int head = blk / per, i0 = (blk - head * per) * kRowsBlock;
    T* at = reinterpret_cast<T*>(p.dq) + (size_t)head * p.Lq * D + 8 * lane;
    for (int i = i0 + sub; i < min(i0 + kRowsBlock, p.row0); i += RPP)
      *reinterpret_cast<u32x4*>(at + (size_t)i * D) = u32x4{0u, 0u, 0u, 0u};
    return;
  }
  if constexpr (is_half<T>) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) peak = fmaxf(peak, __shfl_xor(peak, m, 64));
    if ((threadIdx.x & 63) == 0) top[threadIdx.x / 64] = peak;
    __syncthreads();
    if (threadIdx.x == 0) *peak_at = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  }
}

// Store a wave's transposed accumulators (register r of block db, lane (n, hh): dim
// 32 db + kconst(r) + 4 hh of row n), times f: rounded, or as a partial in fp32.
template <int D, typename T>
__device__ __forceinline__ void store(const f32x16 (&acc)[D / 32], float f, T* out, float* part, int hh) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * db + 8 * g + 4 * hh;
      const f32x4 v = {acc[db][4 * g] * f, acc[db][4 * g + 1] * f, acc[db][4 * g + 2] * f, acc[db][4 * g + 3] * f};
      if (part) *reinterpret_cast<f32x4*>(part + d) = v;
      else *reinterpret_cast<uint2*>(out + d) = make_uint2(Elem<T>::pack2(v[0], v[1]), Elem<T>::pack2(v[2], v[3]));
    }
}

// Stages of a workgroup's ring, a tile pair and 64 floats each: two workgroups
// share a compute unit's 160 KB.
constexpr int kStages = 4;
template <int D> constexpr int kStage = 2 * TN * D * 2 + 256;
// Operands of V (of KX a wave) that a key block keeps in LDS behind the ring and not in registers, of which a bias or a cap
// needs more, and fp16's factor of dS one: spilled by the compiler, they came back from memory through waits for the copies
// of later tiles (what the one more costs and saves came out even, 268 us either way at 32 / 16 heads of 3001 rows on 4099 keys
// with a cap).
template <int D, typename T, bool MOD> constexpr int kHome = D == 128 ? (MOD ? 2 : 0) + (is_half<T> ? 1 : 0) : 0;
// Operands read ahead of their MFMA (LDS takes about four MFMAs' time, and two waves share a SIMD), and the registers of 16
// bytes a lane that they pass through: kAhead + 1, and one more beside the first product, where the others are short by it
// of a whole number of turns.
constexpr int kAhead = 2;
constexpr int kFrags = 4;
template <int N1, int NF>
constexpr int frag_of(int i) {
  constexpr int R = kAhead + 1;
  i %= NF;
  if constexpr (NF % R == 0) return i % R;
  else return i < N1 ? i % (R + 1) : (i - N1) % R;
}
// Operands i .. i + kAhead lie in different ones, also from one tile to the next.
template <int N1, int NF>
constexpr bool frags_apart() {
  for (int i = 0; i < NF; ++i)
    for (int j = 1; j <= kAhead; ++j)
      if (frag_of<N1, NF>(i) == frag_of<N1, NF>(i + j)) return false;
  return true;
}

// Where a half of a wave's lanes read what belongs to their rows: an address, computed here, behind which constants are
// offsets of the loads.
__device__ __forceinline__ uint32_t stats_at(uint32_t at, int hh) {
  uint32_t to;
  asm volatile("v_lshl_add_u32 %0, %1, 4, %2" : "=v"(to) : "v"(hh), "s"(__builtin_amdgcn_readfirstlane((int)at)));
  return to;
}

// x as it is, computed here: the compiler otherwise adds the constants behind it before the loop, each into a register
// of its own.
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+s"(x));
  return x;
}

// dK and dV of 128 keys of a KV head: the tiles of 32 queries that see them, of all query heads of
// the group, or a part of them (a partial in fp32, summed by bwd_sum_kernel).
template <int D, typename T, bool CAUSAL, bool ALIBI, bool CAP>
__device__ __forceinline__ void dkv_block(const BwdParams& p, char* lds, int item) {
  typedef Elem<T> E;
  typedef Tile<D, T> TL;
  typedef typename E::vec8 vec8;
  constexpr int TB = TL::BYTES, STAGE = kStage<D>, CPR = TL::CPR;
  constexpr int CB = TL::NBLK / kWaves;            // 1 KB copies of a tile that a wave makes
  constexpr int CPW = 2 * CB + 1;                  // copies in flight of a stage
  static_assert(CB >= 1, "a tile's copies divide over the waves");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, hh = lane >> 5;

  // Key blocks in order: the first ones see the most queries.
  const int units = p.B * p.Hkv;
  const int unit = p.shares ? item / p.dkv.list : item % units;
  const Place at = place_of(p.dkv, p.shares ? item - unit * p.dkv.list : item / units);
  const int kb = at.block, part = at.part, S = at.parts;
  const int b = unit / p.Hkv, h0 = (unit - b * p.Hkv) * p.group;   // batch and first query head
  const int rows = p.rows, off = p.Lk - rows, W = p.window;
  const int j0 = kb * BLK, jw = j0 + TN * wave;
  // The queries that see keys [j0, j0 + 128): tiles [ta, ta + nt) of each head.
  int ilo = 0, ihi = rows;
  if (CAUSAL) {
    ilo = max(0, j0 - off);
    if (W > 0) ihi = min(rows, min(j0 + BLK, p.Lk) - off + W - 1);
  }
  const int ta = ilo / TN, nt = ihi > ilo ? (ihi + TN - 1) / TN - ta : 0;
  const int total = nt * p.group;
  const int u0 = (int)((long long)total * part / S), u1 = (int)((long long)total * (part + 1) / S);

  const int key = jw + n, krow = min(key, p.Lk - 1);
  int scale_exp = 0;
  if (is_half<T>) scale_exp = bwd_scale<T>(p, unit, reinterpret_cast<float*>(lds));

  // K and V of the wave's keys: lane (n, hh) holds key n, dims 16 kx + 8 hh ...  (A negative scale: K
  // negated, which only the scores see.)
  constexpr int VL = kHome<D, T, ALIBI || CAP>;
  vec8 kf[TL::KX], vf[TL::KX - VL];
  const uint32_t home = (uint32_t)(uintptr_t)(lds_void*)lds + kStages * STAGE + wave * VL * 1024;
  {
    const T* kg = reinterpret_cast<const T*>(p.k) + ((size_t)unit * p.Lk + krow) * D + 8 * hh;
    const T* vg = reinterpret_cast<const T*>(p.v) + ((size_t)unit * p.Lk + krow) * D + 8 * hh;
#pragma unroll
    for (int kx = 0; kx < TL::KX; ++kx) {
      kf[kx] = load8(kg + 16 * kx, p.sign);
      const vec8 v = load8(vg + 16 * kx);
      if (kx < TL::KX - VL) vf[kx] = v;
      else *(lds_u32x4*)(uintptr_t)(home + (kx - TL::KX + VL) * 1024 + 16 * lane) = __builtin_bit_cast(u32x4, v);
    }
  }

  // Copies: this wave's blocks of the Q and dO tiles and, every wave alike, the tile's 64 floats.
  // Blocks wave, wave + 4 of a tile: 16 rows apart, where the swizzle is the same.
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)lds;
  int qoff, goff;
  {
    const int r = wave * (1024 / (2 * D)) + lane / CPR, c = 8 * ((lane % CPR) ^ swz<D>(r));
    qoff = (r * D + c) * 2;
    goff = (int)(r * p.do_sl + c) * 2;
  }
  static_assert(CB == 1 || kWaves * 1024 / (2 * D) == 16, "a wave's blocks lie 16 rows apart");
  const int gstep = (int)(TN * p.do_sl) * 2;
  // The next tile to copy, tile ct of head h0 + cg; cut off the resources of its head's rows.
  int cu = u0, cg = nt ? u0 / nt : 0, ct = ta + (nt ? u0 % nt : 0);
  u32x4 rq, rg;
  auto next_head = [&]() __attribute__((always_inline)) {
    const size_t head = (size_t)b * p.Hq + h0 + cg;
    rq = resource(reinterpret_cast<const T*>(p.q) + (head * p.Lq + p.row0) * D, (unsigned)rows * D * 2);
    rg = resource(reinterpret_cast<const T*>(p.d_o) + b * p.do_sb + (h0 + cg) * p.do_sh + p.row0 * p.do_sl,
                  (unsigned)((rows - 1) * p.do_sl + D) * 2);
  };
  next_head();
  const u32x4 rx = resource(p.stats + ((size_t)b * p.Hq + h0) * p.row_tiles * (2 * TN),
                            (unsigned)(p.group * p.row_tiles) * (8 * TN));
  auto copy_next = [&]() __attribute__((always_inline)) {
    if (cu >= u1) return;
    const uint32_t dst = lds0 + (uint32_t)(cu - u0) % kStages * STAGE;
#pragma unroll
    for (int u = 0; u < CB; ++u) {
      copy16(rq, dst + (uint32_t)((wave + u * kWaves) * 1024), qoff + here(ct * TB + u * (TB / 2)));
      copy16(rg, dst + (uint32_t)(TB + (wave + u * kWaves) * 1024), goff + here(ct * gstep + u * (gstep / 2)));
    }
    copy4(rx, dst + 2 * TB, 4 * lane + here((cg * p.row_tiles + ct) * (8 * TN)));
    ++cu;
    if (++ct == ta + nt) {
      ct = ta;
      ++cg;
      next_head();
    }
  };

  const int roff = TL::row_offset(lane), doff = TL::dim_offset(lane);
  f32x16 dk[TL::DB], dv[TL::DB];
#pragma unroll
  for (int db = 0; db < TL::DB; ++db) dk[db] = dv[db] = f32x16{};
  const float c = p.c;
  const float held = __builtin_ldexpf(1.f, scale_exp - (is_half<T> ? kShift : 0));

  // A tile's MFMAs, each with one operand from LDS: first S (rows of Q), dP (rows of dO), dV (dims of
  // dO) and dK (dims of Q), n of each.  Operand i is read kAhead MFMAs before its own, the first ones of a tile
  // at the end of the tile before, and so are the starts of its scores.
  constexpr int n1 = TL::KX, n2 = 2 * TL::KX, n3 = 3 * TL::KX, NF = 4 * TL::KX;
  static_assert(2 * TL::DB == TL::KX, "as many steps over dims as over rows");
  static_assert(frags_apart<n1, NF>(), "an operand is not read into another's place");
  vec8 fr[kFrags], vl[VL ? VL : 1];
  f32x16 s, x;
  // dP's steps begin with those whose V comes from LDS.
  auto step = [](int j) constexpr { return (j + TL::KX - VL) % TL::KX; };
  auto read = [&](auto ic, uint32_t st, uint32_t next) __attribute__((always_inline)) {
    constexpr int i = decltype(ic)::value;
    vec8& f = fr[frag_of<n1, NF>(i)];
    if constexpr (i < n1) f = TL::template rows<i>(st + roff, 0);
    else if constexpr (i < n2) f = TL::template rows<step(i - n1)>(st + roff, TB);
    else if constexpr (i < n3) f = TL::template dims<(i - n2) / TL::DB, (i - n2) % TL::DB>(st + doff, TB);
    else if constexpr (i < NF) f = TL::template dims<(i - n3) / TL::DB, (i - n3) % TL::DB>(st + doff, 0);
    else f = TL::template rows<i - NF>(next + roff, 0);
  };
  auto starts = [&](f32x16& a, uint32_t at) __attribute__((always_inline)) {
    const uint32_t to = stats_at(at, hh);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 v = *(lds_f32x4*)(uintptr_t)(to + 32 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) a[4 * g + i] = v[i];
    }
  };
  auto prime = [&](uint32_t st) __attribute__((always_inline)) {
    if constexpr (CAP) s = f32x16{};
    else starts(s, st + 2 * TB);
    static_for<kAhead>([&](auto ic) { read(ic, st, st); });
  };

  // One tile: queries i0 .. i0 + 31 of a head against the wave's keys.  The vector work runs beside the MFMAs that do not
  // wait for it: the exponentials beside dP (and the start of dV), dS beside dV (and the start of dK).
  auto tile = [&](auto masked, uint32_t st, uint32_t next, int i0, float sl2, AlibiOrigin o) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    // Query i sees this lane's key: lo <= i - i0 - 4 hh < hi.
    const int lo = key - off - i0 - 4 * hh, hi = W > 0 ? lo + W : 1 << 30;
    const float bias = ALIBI ? sl2 * (float)(key + here(from_origin(0, off + i0, o, CAUSAL))) : 0.f;
    Weights<T> pw, dw;
    uint32_t sx = 0;
    if constexpr (CAP) sx = stats_at(st + 2 * TB, hh);
    auto weigh = [&](auto kc) __attribute__((always_inline)) {       // registers 2 k, 2 k + 1
      constexpr int r = 2 * decltype(kc)::value;
      float y[2], f[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (CAP) {
          const float a = *(lds_float*)(uintptr_t)(sx + 4 * kconst(r + i));
          y[i] = fast_exp2(capped(s[r + i], p, a, f[i]));
        } else {
          y[i] = fast_exp2(ALIBI ? __builtin_fmaf(s[r + i], c, bias) : s[r + i] * c);
        }
        if (MASKED && (kconst(r + i) < lo || kconst(r + i) >= hi)) y[i] = 0.f;
        s[r + i] = CAP ? y[i] * f[i] : y[i];
      }
      pw.set(r, y[0], y[1]);
    };
    auto differ = [&](auto kc) __attribute__((always_inline)) {
      constexpr int r = 2 * decltype(kc)::value;
      float y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        y[i] = s[r + i] * x[r + i];
        if (is_half<T>) y[i] *= held;
        if (MASKED && (kconst(r + i) < lo || kconst(r + i) >= hi)) y[i] = 0.f;   // (0 times an infinity is NaN)
      }
      dw.set(r, y[0], y[1]);
    };
    static_for<NF>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      read(std::integral_constant<int, i + kAhead>{}, st, next);
      if constexpr (i == n1 - 2) starts(x, st + 2 * TB + 4 * TN);
      if constexpr (VL > 0 && i == n1 - 2) {
        uint32_t to;
        asm volatile("v_lshl_add_u32 %0, %1, 4, %2" : "=v"(to) : "v"(lane), "s"(home));
        static_for<VL>([&](auto uc) {
          constexpr int u = decltype(uc)::value;
          vl[u] = __builtin_bit_cast(vec8, *(lds_u32x4*)(uintptr_t)(to + u * 1024));
        });
      }
      const vec8 f = fr[frag_of<n1, NF>(i)];
      if constexpr (i < n1) s = E::mfma(f, kf[i], s);
      else if constexpr (i < n1 + VL) x = E::mfma(f, vl[i - n1], x);
      else if constexpr (i < n2) x = E::mfma(f, vf[step(i - n1)], x);
      else if constexpr (i < n3) dv[(i - n2) % TL::DB] = E::mfma(f, pw.operand((i - n2) / TL::DB), dv[(i - n2) % TL::DB]);
      else dk[(i - n3) % TL::DB] = E::mfma(f, dw.operand((i - n3) / TL::DB), dk[(i - n3) % TL::DB]);
      // Pair k of the weights after MFMA n1 + lag + k / per, of dS n MFMAs later.
      constexpr int per = 8 / TL::KX, lag = TL::KX / 4;
      static_for<per>([&](auto uc) {
        constexpr int u = decltype(uc)::value;
        constexpr int k = (i - n1 - lag) * per + u, j = (i - n2 - lag) * per + u;
        if constexpr (i >= n1 + lag && k < 8) weigh(std::integral_constant<int, k>{});
        if constexpr (i >= n2 + lag && j < 8) differ(std::integral_constant<int, j>{});
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (CAP) s = f32x16{};
    else starts(s, next + 2 * TB);
  };

  // This wave's tiles of a head: none of a row sees a key before tile va and from vb on, and from wa to wb every row sees
  // every key.
  int va = ta, vb = ta + nt, wa = ta, wb = ta + nt;
  if (CAUSAL) {
    va = max(ta, (jw - off) / TN);                        // (a row i sees key jw from i = jw - off on)
    if (jw < off) va = ta;
    wa = max(va, (jw + TN - 1 - off + TN - 1) / TN);
    if (jw + TN - 1 <= off) wa = va;
    if (W > 0) {
      vb = min(vb, max(va, (jw + TN - 1 - off + W - 1 + TN) / TN));     // rows below jw + 31 - off + W see some
      wb = min(vb, max(0, jw - off + W) / TN);                          // rows below jw - off + W see all
    }
    wa = min(wa, vb);
    wb = max(wa, min(wb, vb));
  }
  int g = nt ? u0 / nt : 0, t = ta + (nt ? u0 % nt : 0);
  // Behind this tile u + 2 is in LDS (every wave has waited for its own copies), and the stage of tile u is free.
  auto advance = [&](int u) __attribute__((always_inline)) {
    if (u + kStages - 1 < u1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)\n\ts_barrier" : : "n"((kStages - 3) * CPW), "n"(0) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    copy_next();
  };
  if (u1 > u0) {
    for (int u = 0; u < kStages - 1; ++u) copy_next();
    advance(u0 - 1);
    prime(lds0);
  }
  // Runs of tiles of one kind, each its own loop: the kinds side by side in one loop cost moves of the
  // accumulators at every tile.
  int u = u0;
  auto run = [&](auto kind, int end, float sl2, AlibiOrigin o) __attribute__((always_inline)) {      // to tile `end` of the head
    constexpr int KIND = decltype(kind)::value;        // 0: no row sees a key, 1: some, 2: all
    end = min(end, t + u1 - u);
    for (; t < end; ++t, ++u) {
      const uint32_t st = lds0 + (uint32_t)(u - u0) % kStages * STAGE, next = lds0 + (uint32_t)(u + 1 - u0) % kStages * STAGE;
      if constexpr (KIND == 0) prime(next);
      else tile(std::integral_constant<bool, KIND == 1>{}, st, next, t * TN, sl2, o);
      advance(u);
    }
  };
  while (u < u1) {
    const float slope = ALIBI ? p.slopes[h0 + g] : 0.f, sl2 = slope * kLog2e;
    const AlibiOrigin o = alibi_origin(slope, CAUSAL, W, p.Lk);
    if constexpr (CAUSAL) {
      run(std::integral_constant<int, 0>{}, va, sl2, o);
      for (int k = 0; k < 2; ++k) {      // (in a window a second time behind the whole ones)
        run(std::integral_constant<int, 1>{}, k ? vb : wa, sl2, o);
        run(std::integral_constant<int, 2>{}, wb, sl2, o);
      }
      run(std::integral_constant<int, 0>{}, ta + nt, sl2, o);
    } else {
      run(std::integral_constant<int, 2>{}, ta + nt, sl2, o);
    }
    t = ta;
    ++g;
  }

  if (key < p.Lk) {
    const size_t to = ((size_t)unit * p.Lk + key) * D;
    float* pk = S > 1 ? p.ws_dkv + (((size_t)unit * p.dkv.pieces + at.piece + part) * 2 * BLK + (key - j0)) * D : nullptr;
    store<D, T>(dk, __builtin_ldexpf(CAP ? 4.f * p.scale : p.scale, -scale_exp), reinterpret_cast<T*>(p.dk) + to, pk, hh);
    store<D, T>(dv, is_half<T> ? __builtin_ldexpf(1.f, -kShift) : 1.f, reinterpret_cast<T*>(p.dv) + to,
                pk ? pk + BLK * D : nullptr, hh);
  }
}

// dQ of 128 query rows (of p.hg heads that share a KV head, 128 / hg rows each): the tiles of 32
// keys that they see, or a part of them.
template <int D, typename T, bool CAUSAL, bool ALIBI, bool CAP>
__device__ __forceinline__ void dq_block(const BwdParams& p, char* lds, int item) {
  typedef Elem<T> E;
  typedef Tile<D, T> TL;
  typedef typename E::vec8 vec8;
  constexpr int TB = TL::BYTES, STAGE = kStage<D>, CPR = TL::CPR;
  constexpr int CB = TL::NBLK / kWaves, CPW = 2 * CB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, hh = lane >> 5;

  const int hg = p.hg, bm = TN * (kWaves / hg), ngrp = p.group / hg;
  const int rows = p.rows, off = p.Lk - rows, W = p.window;
  const int units = p.B * p.Hkv, nqb = (rows + bm - 1) / bm;
  // Row blocks from the last, which sees the most keys; the head groups of a block beside each other.
  const int unit = p.shares ? item / (p.dq_.list * ngrp) : item / ngrp % units;
  const int rest = p.shares ? item - unit * p.dq_.list * ngrp : item / (ngrp * units) * ngrp + item % ngrp;
  const int grp = rest % ngrp;
  const Place at = place_of(p.dq_, rest / ngrp);
  const int rb = nqb - 1 - at.block, part = at.part, S = at.parts;
  const int b = unit / p.Hkv, hq = (unit - b * p.Hkv) * p.group + grp * hg + wave % hg;
  const size_t head = (size_t)b * p.Hq + hq;
  const int i0 = rb * bm, iw = i0 + TN * (wave / hg), wlast = min(iw + TN, rows) - 1;
  int jlo = 0, jhi = p.Lk;
  if (CAUSAL) {
    jhi = min(p.Lk, min(i0 + bm, rows) + off);
    if (W > 0) jlo = max(0, i0 + off + 1 - W);
  }
  const int ta = jlo / TN, nt = (jhi + TN - 1) / TN - ta;
  const int t0 = ta + (int)((long long)nt * part / S), t1 = ta + (int)((long long)nt * (part + 1) / S);

  int scale_exp = 0;
  if (is_half<T>) scale_exp = bwd_scale<T>(p, unit, reinterpret_cast<float*>(lds));

  const int row = min(iw + n, rows - 1);
  vec8 qf[TL::KX], gf[TL::KX];
  {
    const T* qg = reinterpret_cast<const T*>(p.q) + (head * p.Lq + p.row0 + row) * D + 8 * hh;
    const T* gg = reinterpret_cast<const T*>(p.d_o) + b * p.do_sb + hq * p.do_sh + (p.row0 + row) * p.do_sl + 8 * hh;
#pragma unroll
    for (int kx = 0; kx < TL::KX; ++kx) {
      qf[kx] = load8(qg + 16 * kx, p.sign);
      gf[kx] = load8(gg + 16 * kx);
    }
  }
  const float* sx = p.stats + (head * p.row_tiles + row / TN) * (2 * TN) + row % TN;
  const float start = sx[0], nd = sx[TN];
  const float slope = ALIBI ? p.slopes[hq] : 0.f, sl2 = slope * kLog2e;
  const int from = -from_origin(0, off + iw, alibi_origin(slope, CAUSAL, W, p.Lk), CAUSAL);
  const float c = p.c, add = CAP ? start : start * c;

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)lds;
  int coff;
  {
    const int r = wave * (1024 / (2 * D)) + lane / CPR;
    coff = (r * D + 8 * ((lane % CPR) ^ swz<D>(r))) * 2;
  }
  const u32x4 rk = resource(reinterpret_cast<const T*>(p.k) + (size_t)unit * p.Lk * D, (unsigned)p.Lk * D * 2);
  const u32x4 rv = resource(reinterpret_cast<const T*>(p.v) + (size_t)unit * p.Lk * D, (unsigned)p.Lk * D * 2);
  auto copy_tile = [&](int t) __attribute__((always_inline)) {
    if (t >= t1) return;
    const uint32_t dst = lds0 + (uint32_t)(t - t0) % kStages * STAGE;
#pragma unroll
    for (int u = 0; u < CB; ++u) {
      const int at = coff + here(t * TB + u * (TB / 2));
      copy16(rk, dst + (uint32_t)((wave + u * kWaves) * 1024), at);
      copy16(rv, dst + (uint32_t)(TB + (wave + u * kWaves) * 1024), at);
    }
  };

  const int roff = TL::row_offset(lane), doff = TL::dim_offset(lane);
  f32x16 dq[TL::DB];
#pragma unroll
  for (int db = 0; db < TL::DB; ++db) dq[db] = f32x16{};
  const float held = __builtin_ldexpf(1.f, scale_exp - (is_half<T> ? kShift : 0));

  // A tile's MFMAs as in dkv_block: S (rows of K), dP (rows of V), dQ (dims of K).
  constexpr int n1 = TL::KX, n2 = 2 * TL::KX, NF = 3 * TL::KX;
  static_assert(frags_apart<n1, NF>(), "an operand is not read into another's place");
  vec8 fr[kFrags];
  auto read = [&](auto ic, uint32_t st, uint32_t next) __attribute__((always_inline)) {
    constexpr int i = decltype(ic)::value;
    vec8& f = fr[frag_of<n1, NF>(i)];
    if constexpr (i < n1) f = TL::template rows<i>(st + roff, 0);
    else if constexpr (i < n2) f = TL::template rows<i - n1>(st + roff, TB);
    else if constexpr (i < NF) f = TL::template dims<(i - n2) / TL::DB, (i - n2) % TL::DB>(st + doff, 0);
    else f = TL::template rows<i - NF>(next + roff, 0);
  };
  auto prime = [&](uint32_t st) __attribute__((always_inline)) {
    static_for<kAhead>([&](auto ic) { read(ic, st, st); });
  };
  auto tile = [&](auto masked, uint32_t st, uint32_t next, int j0) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    f32x16 s = f32x16{}, x = f32x16{};
    // This lane's row sees key j: lo < j - j0 - 4 hh <= hi.
    int hi = p.Lk - 1, lo = -1;
    if (CAUSAL) hi = min(hi, row + off);
    if (CAUSAL && W > 0) lo = row + off - W;
    hi -= j0 + 4 * hh;
    lo -= j0 + 4 * hh;
    const float base = ALIBI ? __builtin_fmaf(sl2, (float)(j0 + 4 * hh - from), add) : add;
    Weights<T> w, rest;
    auto weigh = [&](auto kc) __attribute__((always_inline)) {       // registers 2 k, 2 k + 1
      constexpr int r = 2 * decltype(kc)::value;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        constexpr int r0 = r;
        const int k = kconst(r0 + i);
        float f = 1.f;
        if constexpr (CAP) {
          s[r + i] = fast_exp2(capped(s[r + i], p, add, f));
          s[r + i] *= f;
        } else {
          s[r + i] = fast_exp2(__builtin_fmaf(s[r + i], c, ALIBI ? __builtin_fmaf(sl2, (float)k, base) : base));
        }
      }
    };
    auto differ = [&](auto kc) __attribute__((always_inline)) {
      constexpr int r = 2 * decltype(kc)::value;
      float y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = kconst(r + i);
        y[i] = s[r + i] * (x[r + i] + nd);
        if (is_half<T>) y[i] *= held;
        if (MASKED && (k > hi || k <= lo)) y[i] = 0.f;
      }
      w.set(r, y[0], y[1]);
      rest.rest(w, r, y[0], y[1]);
    };
    static_for<NF>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      read(std::integral_constant<int, i + kAhead>{}, st, next);
      const vec8 f = fr[frag_of<n1, NF>(i)];
      constexpr int per = 8 / TL::KX, lag = TL::KX / 4;
      // What the first half of dQ's MFMAs takes comes before them, the rest beside them.
      if constexpr (i == n2) static_for<4>([&](auto kc) { differ(kc); });
      if constexpr (i < n1) s = E::mfma(f, qf[i], s);
      else if constexpr (i < n2) x = E::mfma(f, gf[i - n1], x);
      else {
        constexpr int c16 = (i - n2) / TL::DB, db = (i - n2) % TL::DB;
        dq[db] = E::mfma(f, w.operand(c16), dq[db]);
        dq[db] = E::mfma(f, rest.operand(c16), dq[db]);
      }
      // The exponentials beside dP, the last ones in its last place.
      static_for<per>([&](auto uc) {
        constexpr int k = (i - n1 - lag) * per + decltype(uc)::value;
        if constexpr (i >= n1 + lag && i < n2) weigh(std::integral_constant<int, k>{});
      });
      if constexpr (i == n2 - 1) static_for<lag * per>([&](auto uc) { weigh(std::integral_constant<int, 8 - lag * per + decltype(uc)::value>{}); });
      if constexpr (i >= n2 && i < n2 + TL::DB) {
        constexpr int per2 = 4 / TL::DB;
        static_for<per2>([&](auto uc) { differ(std::integral_constant<int, 4 + (i - n2) * per2 + decltype(uc)::value>{}); });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  // This wave's tiles: its rows see keys of tiles [va, vb), each of them all keys of [wa, wb).
  int va = t0, vb = t1, wa = t0, wb = min(t1, p.Lk / TN);
  if (CAUSAL) {
    vb = min(vb, (wlast + off) / TN + 1);
    wb = min(wb, (iw + off + 1) / TN);
    if (W > 0) {
      va = max(va, max(0, iw + off - W + 1) / TN);
      wa = max(va, (max(0, wlast + off - W + 1) + TN - 1) / TN);
    }
  }
  if (iw >= rows) vb = va;
  va = min(va, t1);
  vb = max(va, min(vb, t1));
  wa = min(max(wa, va), vb);
  wb = max(wa, min(wb, vb));
  auto advance = [&](int t) __attribute__((always_inline)) {     // as in dkv_block
    if (t + kStages - 1 < t1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)\n\ts_barrier" : : "n"((kStages - 3) * CPW), "n"(0) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    copy_tile(t + kStages);
  };
  int t = t0;
  if (t1 > t0) {
    for (int u = 0; u < kStages - 1; ++u) copy_tile(t0 + u);
    advance(t0 - 1);
    prime(lds0);
  }
  auto run = [&](auto kind, int end) __attribute__((always_inline)) {
    constexpr int KIND = decltype(kind)::value;        // 0: no row sees a key, 1: some, 2: all
    for (; t < end; ++t) {
      const uint32_t st = lds0 + (uint32_t)(t - t0) % kStages * STAGE, next = lds0 + (uint32_t)(t + 1 - t0) % kStages * STAGE;
      if constexpr (KIND == 0) prime(next);
      else tile(std::integral_constant<bool, KIND == 1>{}, st, next, t * TN);
      advance(t);
    }
  };
  run(std::integral_constant<int, 0>{}, va);
  for (int k = 0; k < 2; ++k) {      // (the masked ones come before the whole ones in a window, and behind them)
    run(std::integral_constant<int, 1>{}, k ? vb : wa);
    run(std::integral_constant<int, 2>{}, wb);
  }
  run(std::integral_constant<int, 0>{}, t1);

  if (iw + n < rows) {
    const size_t to = (head * p.Lq + p.row0 + iw + n) * D;
    float* pq = nullptr;
    if (S > 1) pq = p.ws_dq + ((((size_t)unit * ngrp + grp) * p.dq_.pieces + at.piece + part) * BLK + TN * wave + n) * D;
    store<D, T>(dq, __builtin_ldexpf(CAP ? 4.f * p.scale : p.scale, -scale_exp), reinterpret_cast<T*>(p.dq) + to, pq, hh);
  }
}

// Both in one launch, the key blocks first: the row blocks fill what they leave free.  32 heads of 8192 causal rows of 128 in
// bf16 take 1856 us (here and below up to 6 % more on other GPUs), 0.74 PFLOP/s of the formula's five products and 1.18 of the eight that are formed, the matrix unit busy 0.66 of the cycles (at
// 1.72 GHz under that load); with fp16, a cap and a window of 1025 (32 / 16 heads of 3001 on 4099) 255, the vector unit 0.55
// and the matrix unit 0.40; 16 heads of 64 dims have the exponentials of twice as many products: 0.44 and 0.28.
template <int D, typename T, bool CAUSAL, bool ALIBI, bool CAP>
__global__ __launch_bounds__(kThreads, 2) void bwd_kernel(BwdParams p) {
  __shared__ __attribute__((aligned(1024))) char lds[kStages * kStage<D> + kWaves * 1024 * kHome<D, T, ALIBI || CAP>];
  const int units = p.B * p.Hkv, nk = units * p.dkv.list, gk = p.shares ? (nk + kXcds - 1) / kXcds * kXcds : nk;
  const int g = blockIdx.x;
  if (g < gk) {
    const int item = item_of(g, nk, p.shares);
    if (item >= 0) dkv_block<D, T, CAUSAL, ALIBI, CAP>(p, lds, item);
  } else {
    const int item = item_of(g - gk, units * (p.group / p.hg) * p.dq_.list, p.shares);
    if (item >= 0) dq_block<D, T, CAUSAL, ALIBI, CAP>(p, lds, item);
  }
}

// The partials of the blocks in several parts, summed in their order and rounded: 1024 values a workgroup,
// first of dK and dV, then of dQ.  Bound by memory: 11 us for 46 MB of them (2 x 32 / 8 heads of 2048 rows).
template <int D, typename T>
__global__ __launch_bounds__(256) void bwd_sum_kernel(BwdParams p) {
  constexpr int PER = BLK * D / 1024;                      // workgroups of a piece
  const int units = p.B * p.Hkv, nk = units * p.dkv.multi * 2 * PER;
  int g = blockIdx.x;
  const bool keys = g < nk;
  const BwdSplit& s = keys ? p.dkv : p.dq_;
  if (!keys) g -= nk;
  const int sub = g % PER;
  g /= PER;
  int which = 0;
  if (keys) {
    which = g % 2;
    g /= 2;
  }
  const int of = g / s.multi;                              // the unit (and head group)
  int m = g - of * s.multi, block = 0, piece = 0;          // the m-th block in several parts
  for (;; ++block) {
    const int c = s.parts[block];
    if (c > 1 && m-- == 0) break;
    piece += c > 1 ? c : 0;
  }
  const int parts = s.parts[block], i = sub * 1024 + 4 * threadIdx.x, r = i / D, d = i % D;
  const size_t step = (size_t)(keys ? 2 : 1) * BLK * D;
  const float* at = (keys ? p.ws_dkv : p.ws_dq) + ((size_t)of * s.pieces + piece) * step + which * BLK * D + i;
  T* out;
  if (keys) {
    const int key = block * BLK + r;
    if (key >= p.Lk) return;
    out = reinterpret_cast<T*>(which ? p.dv : p.dk) + ((size_t)of * p.Lk + key) * D + d;
  } else {
    const int hg = p.hg, bm = TN * (kWaves / hg), ngrp = p.group / hg, wave = r / TN;
    const int unit = of / ngrp, row = ((p.rows + bm - 1) / bm - 1 - block) * bm + TN * (wave / hg) + r % TN;
    if (row >= p.rows) return;
    const size_t head = (size_t)unit * p.group + (of - unit * ngrp) * hg + wave % hg;
    out = reinterpret_cast<T*>(p.dq) + (head * p.Lq + p.row0 + row) * D + d;
  }
  f32x4 a = *reinterpret_cast<const f32x4*>(at);
  for (int k = 1; k < parts; ++k) a += *reinterpret_cast<const f32x4*>(at + k * step);
  *reinterpret_cast<uint2*>(out) = make_uint2(Elem<T>::pack2(a[0], a[1]), Elem<T>::pack2(a[2], a[3]));
}

template <int D, typename T, bool CAUSAL, bool ALIBI, bool CAP>
hipError_t launch_t(const BwdParams& p, hipStream_t stream) {
  const int64_t units = (int64_t)p.B * p.Hkv, heads = (int64_t)p.B * p.Hq;
  int64_t pre = heads * p.row_blocks + heads * ((p.row0 + kRowsBlock - 1) / kRowsBlock);
  if (is_half<T>) pre += units * p.key_blocks;
  hipLaunchKernelGGL((bwd_rows_kernel<D, T>), dim3((unsigned)pre), dim3(kThreads), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const auto whole = [&](int64_t n) { return p.shares ? (n + kXcds - 1) / kXcds * kXcds : n; };
  const int64_t n = whole(units * p.dkv.list) + whole(units * (p.group / p.hg) * p.dq_.list);
  hipLaunchKernelGGL((bwd_kernel<D, T, CAUSAL, ALIBI, CAP>), dim3((unsigned)n), dim3(kThreads), 0, stream, p);
  if ((e = hipGetLastError()) != hipSuccess || p.dkv.multi + p.dq_.multi == 0) return e;
  const int64_t sums = (units * p.dkv.multi * 2 + units * (p.group / p.hg) * p.dq_.multi) * (BLK * D / 1024);
  hipLaunchKernelGGL((bwd_sum_kernel<D, T>), dim3((unsigned)sums), dim3(256), 0, stream, p);
  return hipGetLastError();
}

template <int D, typename T>
hipError_t launch_d(const BwdParams& p, hipStream_t s) {
  if (p.cap_cl != 0.f) return launch_t<D, T, true, false, true>(p, s);
  if (p.causal) return p.slopes ? launch_t<D, T, true, true, false>(p, s) : launch_t<D, T, true, false, false>(p, s);
  return p.slopes ? launch_t<D, T, false, true, false>(p, s) : launch_t<D, T, false, false, false>(p, s);
}

}  // namespace

int bwd_block_keys() { return BLK; }
int bwd_rows_per_block() { return kRowsBlock; }

hipError_t launch_attn_bwd(const BwdParams& p, hipStream_t stream) {
  if (p.D == 64) return p.bf16 ? launch_d<64, __bf16>(p, stream) : launch_d<64, _Float16>(p, stream);
  return p.bf16 ? launch_d<128, __bf16>(p, stream) : launch_d<128, _Float16>(p, stream);
}

}  // namespace attn
