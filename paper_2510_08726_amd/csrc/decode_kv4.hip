// Single-token decode over the paged 4-bit cache (include/kv4.h): split-k update
// (Section "Split-K Update", Algorithm 2) on tiles of 32 tokens.
//
// Work.  A row is (sequence b, KV head, column tile of its query heads); its
// tiles are those of the tokens that b sees.  All tiles of all rows, row
// after row, are one list, and workgroup w of W takes the tiles from w T / W to
// (w + 1) T / W: equal shares whatever the lengths.  A row inside one share is
// finished there; others leave a partial (O, max, sum) for each share that they
// lie in, and the second kernel joins those.
//
// Tile.  The wave's lanes are n = lane % 16 and g = lane / 16.  S^T = K Q^T runs on
// 16x16x32 MFMAs over the heads as columns: lane (n, g) holds dims [g D / 4, (g + 1) D / 4)
// of token n as the A operand and the same dims of head n as B (the order
// of the summed dims is free), so K goes from its rows to registers
// in one load a lane, with the lane's scale (one at D = 128, half of one at D = 64), and the result has tokens 4 g + r of
// head n in lane (n, g).  That is the B operand of O^T += V^T P^T if the summed
// tokens are taken as 4 g + r of both 16-token halves; for its A operand lane (i, g) loads
// dims [i D / 16, (i + 1) D / 16) of those eight tokens, and pairs of tokens are
// permuted together after conversion.  No LDS and no cross-lane move in the
// loop but for a new maximum.
//
// Bound: 17 / 32 bytes a value and 4 flops a value and head leave it an HBM
// stream; conversion is a VALU instruction for two values of K and two for two of V.

#include <algorithm>
#include <type_traits>

#include "kernel_common.h"
#include "kv4_common.h"
#include "launch.h"

namespace attn {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTile = 32;          // tokens
constexpr int kLeast = kWaves;     // tiles a share holds at least: one for each wave
constexpr float kLazy = 8.f;       // log2 units that a score may exceed its reference by

template <typename T> struct Mfma16;
template <> struct Mfma16<_Float16> {
  static __device__ __forceinline__ f32x4 mul(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Mfma16<__bf16> {
  static __device__ __forceinline__ f32x4 mul(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};

// Tokens [lo, hi) that a sequence sees, and its tiles: whole ones from lo / kTile on.
struct Seen {
  int lo, hi, tiles;
};

__device__ __forceinline__ Seen seen_of(const Kv4DecodeParams& p, int n) {
  Seen s;
  s.hi = min(max(n, 0), p.M << p.shift);
  s.lo = p.window > 0 ? max(s.hi - p.window, 0) : 0;
  s.tiles = s.hi > 0 ? (s.hi + kTile - 1) / kTile - s.lo / kTile : 0;
  return s;
}

// The list of all tiles and its shares: the first `more` hold one tile more
// than the others.  (The entry point keeps the list below 2^31 tiles.)
struct Shares {
  int total, count, each, more;
  __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
  __device__ __forceinline__ int of(int tile) const {
    const int big = more * (each + 1);
    return tile < big ? tile / (each + 1) : more + (tile - big) / each;
  }
};

__device__ __forceinline__ Shares shares_of(const Kv4DecodeParams& p, int total) {
  Shares s;
  s.total = total;
  s.count = min(p.shares, (total + kLeast - 1) / kLeast);
  s.each = s.count ? total / s.count : 0;
  s.more = total - s.each * s.count;
  return s;
}

// Tiles of one row of all sequences, and of those before sequence b; by one wave.
__device__ __forceinline__ int row_tiles(const Kv4DecodeParams& p, int lane, int b, int& before) {
  int all = 0, some = 0;
  for (int i = lane; i < p.B; i += 64) {
    const int t = seen_of(p, p.lens[i]).tiles;
    all += t;
    some += i < b ? t : 0;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    all += __shfl_xor(all, d, 64);
    some += __shfl_xor(some, d, 64);
  }
  before = __builtin_amdgcn_readfirstlane(some);
  return __builtin_amdgcn_readfirstlane(all);
}

// What a lane loads of a tile: of both 16-token halves its token's dims of K and
// their scale, and of eight tokens its dims of V and their scales (a byte each).
template <int D> struct Raw;
template <> struct Raw<128> {
  typedef u32x4 kvec;
  typedef uint32_t vvec;
  kvec k[2];
  vvec v[8];
  uint32_t ks[2], vs[2];
};
template <> struct Raw<64> {
  typedef uint32_t kvec __attribute__((ext_vector_type(2)));
  typedef uint16_t vvec;
  kvec k[2];
  vvec v[8];
  uint32_t ks[2], vs[2];
};

__device__ __forceinline__ float as_float(uint32_t bits) { return __builtin_bit_cast(float, bits); }

template <int D, typename T, int NC, bool ALIBI, bool CAP>
__global__ __launch_bounds__(kThreads) void decode_kv4_kernel(Kv4DecodeParams p) {
  typedef typename Elem<T>::vec8 vec8;
  typedef typename Raw<D>::kvec kvec;
  typedef typename Raw<D>::vvec vvec;
  constexpr int COLS = 16 * NC;
  constexpr int KS = D / 32;          // MFMA steps of K Q^T
  constexpr int DL = D / 16;          // dims of V that a lane holds, and MFMAs of O^T
  __shared__ __attribute__((aligned(16))) float sh_o[kWaves][COLS][D];
  __shared__ float sh_m[kWaves][COLS], sh_l[kWaves][COLS];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int rows_b = p.Hkv * p.head_tiles;

  int none;
  const Shares shares = shares_of(p, row_tiles(p, lane, 0, none) * rows_b);
  const int w = blockIdx.x;
  if (w >= shares.count) return;
  int at = shares.begin(w);
  const int end = shares.begin(w + 1);

  // The sequence of the first tile: the first whose tiles end behind it.
  int b = -1, before = 0;
  for (int c = 0; c < p.B; c += 64) {
    const int i = c + lane;
    const int mine = i < p.B ? seen_of(p, p.lens[i]).tiles * rows_b : 0;
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(upto, d, 64);
      if (lane >= d) upto += y;
    }
    upto += before;
    const uint64_t past = __ballot(upto > at);
    if (past) {
      const int k = __builtin_ctzll(past);
      b = c + k;
      before = __builtin_amdgcn_readlane(upto - mine, k);
      break;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  if (b < 0) return;
  Seen seen = seen_of(p, __builtin_amdgcn_readfirstlane(p.lens[b]));
  int row = (at - before) / max(seen.tiles, 1);    // of the sequence
  int t0 = (at - before) - row * seen.tiles;

  // (The lengths are read again for each sequence; were they changed meanwhile,
  // the conditions on row and b still keep every access in bounds.)
  for (bool first = true; row < rows_b; first = false) {
    const int t1 = min(seen.tiles, t0 + (end - at));
    const int hk = row / p.head_tiles, ht = row - hk * p.head_tiles;
    const int hq0 = hk * p.group + ht * COLS;
    const int heads = min(p.group - ht * COLS, COLS);
    const int tok0 = seen.lo & ~(kTile - 1);
    const int* table = p.table + (int64_t)b * p.M;

    vec8 q[NC][KS];
    float slope[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int h = 16 * c + n;
      const T* qp = static_cast<const T*>(p.q) + ((int64_t)b * p.Hq + hq0 + h) * D + g * (D / 4);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        u32x4 x = {0u, 0u, 0u, 0u};
        if (h < heads) x = *reinterpret_cast<const u32x4*>(qp + 8 * s);
        q[c][s] = __builtin_bit_cast(vec8, x);
      }
      slope[c] = ALIBI && h < heads ? p.slopes[hq0 + h] * kLog2e : 0.f;
    }

    float m[NC], l[NC];
    f32x4 o[NC][DL];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      m[c] = kNegInf;
      l[c] = 0.f;
#pragma unroll
      for (int j = 0; j < DL; ++j) o[c][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // The pages of a tile's halves, -1 for none.
    auto pages = [&](int t, int (&pg)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int pi = (tok0 + t * kTile + 16 * s) >> p.shift;
        const int x = table[min(pi, p.M - 1)];
        pg[s] = pi < p.M && (unsigned)x < (unsigned)p.pages ? x : -1;
      }
    };
    // A half without a page is read from page 0, and masked.
    auto fetch = [&](int t, const int (&pg)[2], Raw<D>& x) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int r = (tok0 + t * kTile + 16 * s) & ((1 << p.shift) - 1);
        const int page = __builtin_amdgcn_readfirstlane(max(pg[s], 0));
        const unsigned char* base = p.cache + ((int64_t)page * p.Hkv + hk) * (int64_t)kv4_block_bytes<D>(p.shift);
        const unsigned char* vc = base + kv4_code_bytes<D>(p.shift);
        const unsigned char* ks = vc + kv4_code_bytes<D>(p.shift);
        const unsigned char* vs = ks + kv4_scale_bytes<D>(p.shift);
        x.k[s] = *reinterpret_cast<const kvec*>(base + (uint32_t)((r + n) * (D / 2) + g * (D / 8)));
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x.v[4 * s + i] = *reinterpret_cast<const vvec*>(vc + (uint32_t)((r + 4 * g + i) * (D / 2) + n * (D / 32)));
        x.ks[s] = ks[(uint32_t)(((g * (D / 4) / 32) << p.shift) + r + n)];
        x.vs[s] = *reinterpret_cast<const uint32_t*>(vs + (uint32_t)(((n * DL / 32) << p.shift) + r + 4 * g));
      }
    };

    auto compute = [&](int t, const int (&pg)[2], Raw<D>& x) __attribute__((always_inline)) {
      const int tok = tok0 + t * kTile;
      const bool whole = tok >= seen.lo && tok + kTile <= seen.hi && (pg[0] | pg[1]) >= 0;
      // Scores.
      float sc[NC][8];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const float scale = as_float(x.ks[s] << 23);
        f32x4 acc[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < KS; ++st) {
          const uint32_t word = x.k[s][st];
          const u32x4 a = {Fp4<T>::template cvt<0>(word, scale), Fp4<T>::template cvt<1>(word, scale),
                           Fp4<T>::template cvt<2>(word, scale), Fp4<T>::template cvt<3>(word, scale)};
#pragma unroll
          for (int c = 0; c < NC; ++c) acc[c] = Mfma16<T>::mul(__builtin_bit_cast(vec8, a), q[c][st], acc[c]);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float v = acc[c][r] * p.c;
            if (CAP) v = soft_cap(v, p.cap_k2, p.cap_cl);
            if (ALIBI) v = __builtin_fmaf(slope[c], (float)(tok + 16 * s + 4 * g + r - (seen.hi - 1)), v);
            sc[c][4 * s + r] = v;
          }
      }
      if (!whole) {
        // What is not seen: no weight, and no NaN from what its bytes hold.
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = tok + 16 * s + 4 * g + r;
            if (key < seen.lo || key >= seen.hi || pg[s] < 0) {
#pragma unroll
              for (int c = 0; c < NC; ++c) sc[c][4 * s + r] = kNegInf;
              x.vs[s] &= ~(0xffu << (8 * r));
            }
          }
      }
      // Lazy repair: the reference moves when a score exceeds it by more than kLazy.
      vec8 pb[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float top = sc[c][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[c][i]);
        if (__ballot(top > m[c] + kLazy)) {
          top = fmaxf(top, __shfl_xor(top, 16, 64));
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float mn = fmaxf(m[c], top);
          const float alpha = m[c] == kNegInf ? 0.f : fast_exp2(m[c] - mn);
          m[c] = mn;
          l[c] *= alpha;
#pragma unroll
          for (int j = 0; j < DL; ++j) o[c][j] *= alpha;
        }
        const float ref = m[c] == kNegInf ? 0.f : m[c];
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          e[i] = fast_exp2(sc[c][i] - ref);
          l[c] += e[i];
        }
        const u32x4 pw = {Elem<T>::pack2(e[0], e[1]), Elem<T>::pack2(e[2], e[3]), Elem<T>::pack2(e[4], e[5]),
                          Elem<T>::pack2(e[6], e[7])};
        pb[c] = __builtin_bit_cast(vec8, pw);
      }
      // O^T: byte h of a lane's dims of tokens 2 i and 2 i + 1 gives word i of
      // the operands of dims 2 h and 2 h + 1.
      float vscale[8];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        vscale[4 * s] = as_float(x.vs[s] << 23);
        vscale[4 * s + 1] = as_float(x.vs[s] << 15);
        vscale[4 * s + 2] = as_float(x.vs[s] << 7);
        vscale[4 * s + 3] = as_float(x.vs[s] >> 1);
      }
      auto block = [&](auto byte) __attribute__((always_inline)) {
        constexpr int h = decltype(byte)::value;
        u32x4 a0, a1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t u = Fp4<T>::template cvt<h>(x.v[2 * i], vscale[2 * i]);
          const uint32_t v = Fp4<T>::template cvt<h>(x.v[2 * i + 1], vscale[2 * i + 1]);
          a0[i] = __builtin_amdgcn_perm(v, u, 0x05040100u);
          a1[i] = __builtin_amdgcn_perm(v, u, 0x07060302u);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          o[c][2 * h] = Mfma16<T>::mul(__builtin_bit_cast(vec8, a0), pb[c], o[c][2 * h]);
          o[c][2 * h + 1] = Mfma16<T>::mul(__builtin_bit_cast(vec8, a1), pb[c], o[c][2 * h + 1]);
        }
      };
      block(std::integral_constant<int, 0>{});
      block(std::integral_constant<int, 1>{});
      if constexpr (D == 128) {
        block(std::integral_constant<int, 2>{});
        block(std::integral_constant<int, 3>{});
      }
    };

    // A tile ahead in registers, its pages two ahead.
    int t = t0 + wave;
    if (t < t1) {
      Raw<D> x;
      int pg[2], next_pg[2];
      pages(t, pg);
      pages(t + kWaves, next_pg);
      fetch(t, pg, x);
      for (; t < t1; t += kWaves) {
        Raw<D> next = x;
        int far[2];
        pages(t + 2 * kWaves, far);
        if (t + kWaves < t1) fetch(t + kWaves, next_pg, next);
        compute(t, pg, x);
        x = next;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          pg[s] = next_pg[s];
          next_pg[s] = far[s];
        }
      }
    }

    // The waves' states, through LDS.  Lane (n, g) holds dims DL (4 g + r) + j of
    // head n in element r of block j.
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      l[c] += __shfl_xor(l[c], 16, 64);
      l[c] += __shfl_xor(l[c], 32, 64);
      float* to = sh_o[wave][16 * c + n];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < DL; j += 4)
          *reinterpret_cast<f32x4*>(to + DL * (4 * g + r) + j) =
              f32x4{o[c][j][r], o[c][j + 1][r], o[c][j + 2][r], o[c][j + 3][r]};
      if (g == 0) {
        sh_m[wave][16 * c + n] = m[c];
        sh_l[wave][16 * c + n] = l[c];
      }
    }
    __syncthreads();
    const bool done = t0 == 0 && t1 == seen.tiles;
    const int64_t part = 2 * (int64_t)w + (first ? 0 : 1);
    for (int idx = threadIdx.x; idx < heads * (D / 4); idx += kThreads) {
      const int h = idx / (D / 4), d = idx % (D / 4) * 4;
      float M = kNegInf;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) M = fmaxf(M, sh_m[i][h]);
      float L = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float f = sh_m[i][h] == kNegInf ? 0.f : fast_exp2(sh_m[i][h] - M);
        L = __builtin_fmaf(sh_l[i][h], f, L);
        acc += f * *reinterpret_cast<const f32x4*>(&sh_o[i][h][d]);
      }
      if (done) {
        const float r = L == 0.f ? 0.f : 1.f / L;
        uint2 out;
        out.x = Elem<T>::pack2(acc[0] * r, acc[1] * r);
        out.y = Elem<T>::pack2(acc[2] * r, acc[3] * r);
        *reinterpret_cast<uint2*>(static_cast<T*>(p.o) + ((int64_t)b * p.Hq + hq0 + h) * D + d) = out;
      } else {
        *reinterpret_cast<f32x4*>(p.ws_o + (part * COLS + h) * D + d) = acc;
        if (d == 0) {
          p.ws_m[part * COLS + h] = M;
          p.ws_l[part * COLS + h] = L;
        }
      }
    }
    at += t1 - t0;
    if (at >= end) break;
    __syncthreads();
    t0 = 0;
    if (++row == rows_b) {
      row = 0;
      do {
        if (++b == p.B) return;
        seen = seen_of(p, __builtin_amdgcn_readfirstlane(p.lens[b]));
      } while (seen.tiles == 0);
    }
  }
}

// Rows in several shares: one workgroup per (sequence, query head).  D / 4 lanes
// hold a row's dims, and the lane groups take its parts in turn.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void decode_kv4_combine_kernel(Kv4DecodeParams p) {
  constexpr int CH = D / 4, NG = kThreads / CH;
  __shared__ float sh_m[NG], sh_l[NG];
  __shared__ f32x4 sh_o[NG][CH];
  const int lane = threadIdx.x & 63;
  const int b = blockIdx.x / p.Hq, hq = blockIdx.x - b * p.Hq;
  const int cols = kv4_columns(p.group);
  const int hk = hq / p.group, in = hq - hk * p.group, ht = in / cols, h = in - ht * cols;
  const int rows_b = p.Hkv * p.head_tiles;
  int before;
  const Shares shares = shares_of(p, row_tiles(p, lane, b, before) * rows_b);
  const int tiles = seen_of(p, __builtin_amdgcn_readfirstlane(p.lens[b])).tiles;
  const int ch = threadIdx.x % CH, g = threadIdx.x / CH;
  T* out = static_cast<T*>(p.o) + (int64_t)blockIdx.x * D + 4 * ch;
  if (tiles == 0) {
    if (g == 0) *reinterpret_cast<uint2*>(out) = make_uint2(0u, 0u);
    return;
  }
  const int from = before * rows_b + (hk * p.head_tiles + ht) * tiles;
  const int w0 = shares.of(from), w1 = shares.of(from + tiles - 1);
  if (w0 == w1) return;                       // the split kernel has written it

  float M = kNegInf, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int w = w0 + g; w <= w1; w += NG) {
    // A share's first row is its part 0, its last (if another) part 1.
    const int64_t at = (2 * (int64_t)w + (w == w0 && shares.begin(w) < from ? 1 : 0)) * cols + h;
    const float m = p.ws_m[at], l = p.ws_l[at];
    const f32x4 v = *reinterpret_cast<const f32x4*>(p.ws_o + at * D + 4 * ch);
    const float mn = fmaxf(M, m);
    const float f = M == kNegInf ? 0.f : fast_exp2(M - mn), e = m == kNegInf ? 0.f : fast_exp2(m - mn);
    L = L * f + l * e;
    acc = acc * f + v * e;
    M = mn;
  }
  sh_o[g][ch] = acc;
  if (ch == 0) {
    sh_m[g] = M;
    sh_l[g] = L;
  }
  __syncthreads();
  if (g) return;
  M = kNegInf;
#pragma unroll
  for (int i = 0; i < NG; ++i) M = fmaxf(M, sh_m[i]);
  L = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const float e = sh_m[i] == kNegInf ? 0.f : fast_exp2(sh_m[i] - M);
    L = __builtin_fmaf(e, sh_l[i], L);
    acc += e * sh_o[i][ch];
  }
  const float r = L == 0.f ? 0.f : 1.f / L;
  *reinterpret_cast<uint2*>(out) =
      make_uint2(Elem<T>::pack2(acc[0] * r, acc[1] * r), Elem<T>::pack2(acc[2] * r, acc[3] * r));
}

template <int D, typename T, int NC>
hipError_t launch(const Kv4DecodeParams& p, int64_t blocks, hipStream_t stream) {
  const dim3 grid((unsigned)blocks), block(kThreads);
  if (p.slopes && p.cap_cl != 0.f)
    hipLaunchKernelGGL((decode_kv4_kernel<D, T, NC, true, true>), grid, block, 0, stream, p);
  else if (p.slopes)
    hipLaunchKernelGGL((decode_kv4_kernel<D, T, NC, true, false>), grid, block, 0, stream, p);
  else if (p.cap_cl != 0.f)
    hipLaunchKernelGGL((decode_kv4_kernel<D, T, NC, false, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((decode_kv4_kernel<D, T, NC, false, false>), grid, block, 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((decode_kv4_combine_kernel<D, T>), dim3((unsigned)(p.B * p.Hq)), block, 0, stream, p);
  return hipGetLastError();
}

template <int D, typename T>
hipError_t launch_cols(const Kv4DecodeParams& p, int64_t blocks, hipStream_t stream) {
  return kv4_columns(p.group) == 16 ? launch<D, T, 1>(p, blocks, stream) : launch<D, T, 2>(p, blocks, stream);
}

}  // namespace

int kv4_shares(int group, int cus) { return cus * (kv4_columns(group) == 16 ? 4 : 2); }

hipError_t launch_decode_kv4(const Kv4DecodeParams& p, hipStream_t stream) {
  // No more workgroups than the longest contexts that the tables hold could use.
  const int64_t most = (((int64_t)p.M << p.shift) / kTile + 2) * p.B * p.Hkv * p.head_tiles;
  const int64_t blocks = std::min<int64_t>(p.shares, (most + kLeast - 1) / kLeast);
  if (p.D == 64) return p.bf16 ? launch_cols<64, __bf16>(p, blocks, stream) : launch_cols<64, _Float16>(p, blocks, stream);
  return p.bf16 ? launch_cols<128, __bf16>(p, blocks, stream) : launch_cols<128, _Float16>(p, blocks, stream);
}

}  // namespace attn
