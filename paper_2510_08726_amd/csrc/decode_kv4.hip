// Single-token decode over the paged 4-bit cache (include/kv4.h): split-k update
// (Section "Split-K Update", Algorithm 2) on tiles of 32 tokens.
//
// Work.  A row is (sequence b, KV head, column tile of its query heads); its
// tiles are those of the tokens that b sees.  All tiles of all rows, row
// after row, are one list, and workgroup w of W takes an equal share of it, whatever
// the lengths.  A row inside one share is finished there; others leave a
// partial (O, max, sum) for each share that they lie in, and the second kernel joins
// those.
//
// Tile.  Each wave copies its tiles from HBM straight to LDS, kRing ahead, and
// needs no other wave until the end of a row.  The wave's lanes are n = lane % 16 and g =
// lane / 16.  S^T = K Q^T runs on 16x16x32 MFMAs over the heads as columns: lane (n, g)
// holds dims [g D / 4, (g + 1) D / 4) of a token as the A operand and the same dims of head
// n as B (the order of the summed dims is free), so the codes of a lane are
// neighbours and have one scale.  MFMA row 4 g + r is token 4 r + g of its 16: the result
// has tokens 4 r + g of head n in lane (n, g), which is the B operand of O^T += V^T P^T
// if the summed tokens are taken in that order; for its A operand lane (i, g) reads dims
// [i D / 16, (i + 1) D / 16) of its eight tokens, which at one r are four rows in line,
// and pairs of tokens are permuted together after conversion.  No lane
// needs another's values in the loop, but for a new maximum.
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
constexpr int kStart = kKv4RowStart;   // units of a row's start and end
// Units that a share holds at least, one row's start or two tiles a wave: one request
// of 3001 tokens takes 9 us, 10.7 with 16 units, 12.6 with 24, 15.4 with 40, and 64 requests of up
// to 200 tokens 11.6, 13.5, 15.1 and 20.0 (one of 32768 tokens would rather have longer
// shares: 17.4 against 16.9, 16.6 and 15.9).
constexpr int kLeast = 8;

// How many workgroups share a compute unit, and the tiles that a wave has in LDS: as
// many waves as the registers allow, then the tiles that 160 KB hold.  16 x 32768
// tokens of 8 KV heads at D = 128 take 96.9 us with 4 workgroups of 2 tiles a wave, 100.5 with
// 3 of 3 and with 2 of 4.  At D = 64 a fifth workgroup takes 8 x 16 heads of 16384
// tokens with ALiBi from 40.7 to 40.0, but spills registers in five of eight kernels.
constexpr int per_unit(int D, int cols) { return cols == 16 ? 4 : D == 64 ? 3 : 2; }
constexpr int ring_tiles(int D, int cols) { return D == 128 && cols == 16 ? 2 : 4; }
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

// Inclusive sum over the wave's lanes, by DPP: within rows of 16 lanes, then the
// last lane of a row to the rows behind it.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int x) {
  x = dpp_add<0x111, 0xf>(x);   // row_shr:1
  x = dpp_add<0x112, 0xf>(x);   // row_shr:2
  x = dpp_add<0x114, 0xf>(x);   // row_shr:4
  x = dpp_add<0x118, 0xf>(x);   // row_shr:8
  x = dpp_add<0x142, 0xa>(x);   // row_bcast:15
  x = dpp_add<0x143, 0xc>(x);   // row_bcast:31
  return x;
}

// The list of all rows' tiles.  A row counts kStart more: what its start
// and end cost a workgroup beside its tiles, so that shares of many short rows take as long
// as shares of one long one.  (The entry point keeps the list below 2^31.)
__device__ __forceinline__ int units_of(const Seen& s) { return s.tiles ? s.tiles + kStart : 0; }

// The shares of a list of `total`: the first `more` hold one unit more than the others.
struct Shares {
  int count, each, more;
  __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
  __device__ __forceinline__ int of(int unit) const {
    const int big = more * (each + 1);
    return unit < big ? unit / (each + 1) : more + (unit - big) / each;
  }
};

__device__ __forceinline__ Shares shares_of(const Kv4DecodeParams& p, int total) {
  Shares s;
  s.count = min(p.shares, (total + kLeast - 1) / kLeast);
  s.each = s.count ? total / s.count : 0;
  s.more = total - s.each * s.count;
  return s;
}

// A tile in LDS: the codes of K and of V, row by row, with the 16-byte chunks of
// a row in an order that keeps the reads free of bank conflicts (chunk c of row r at c ^ chunk_xor(r)),
// then the scale bytes [K, V][D / 32][32].
template <int D> struct Tile {
  static constexpr int kRow = D / 2, kChunks = kRow / 16;
  static constexpr int kCodes = kTile * kRow, kScales = 2 * kCodes, kBytes = kScales + 256;
  static constexpr int kCopies = D == 128 ? 5 : 3;      // instructions that fill it
  static __device__ __forceinline__ int chunk_xor(int r) { return (r >> 2) & (kChunks - 1); }
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Read through the scalar cache: uniform addresses, not written by the kernel.
typedef const __attribute__((address_space(4))) int* ScalarInts;
__device__ __forceinline__ ScalarInts scalar(const int* p) {
  return (ScalarInts)reinterpret_cast<uintptr_t>(p);
}

// soft_cap of a cap above kKv4HighCap.  There 1 - 2 / (1 + e^2t) loses the score in
// the cap: it is off by 2^-22 of the cap.  Up to half the cap: the series of tanh t /
// t, t = x / cl, to t^12 (the next term is under 1e-7 there); beyond, the loss is under 3e-7 of the score.
__device__ __forceinline__ float high_cap(float x, const Kv4DecodeParams& p) {
  const float t = x * p.cap_inv, z = t * t;
  float s = 3.5921280e-3f;                       // 21844 / 6081075
  s = __builtin_fmaf(s, z, -8.8632355e-3f);      // -1382 / 155925
  s = __builtin_fmaf(s, z, 2.1869489e-2f);       // 62 / 2835
  s = __builtin_fmaf(s, z, -5.3968254e-2f);      // -17 / 315
  s = __builtin_fmaf(s, z, 1.3333333e-1f);       // 2 / 15
  s = __builtin_fmaf(s, z, -3.3333333e-1f);      // -1 / 3
  return fabsf(t) < 0.5f ? __builtin_fmaf(x * z, s, x) : soft_cap(x, p.cap_k2, p.cap_cl);
}

__device__ __forceinline__ float as_float(uint32_t bits) { return __builtin_bit_cast(float, bits); }

template <int D, typename T, int NC, bool ALIBI, bool CAP>
__global__ __launch_bounds__(kThreads, per_unit(D, 16 * NC)) void decode_kv4_kernel(Kv4DecodeParams p) {
  typedef typename Elem<T>::vec8 vec8;
  typedef Tile<D> TL;
  constexpr int COLS = 16 * NC;
  constexpr int KS = D / 32;          // MFMA steps of K Q^T
  constexpr int DL = D / 16;          // dims of V that a lane holds, and MFMAs of O^T
  // The waves' rings; at the end of a row their states, 16 columns at a time.
  constexpr int kRing = ring_tiles(D, COLS);
  constexpr int kLds = kWaves * kRing * TL::kBytes;
  constexpr int kPad = D + 4;         // floats of a state's row: 16 lanes write 16 bytes to 16 rows without conflicts
  static_assert(kWaves * 16 * (kPad + 2) * 4 <= kLds, "the states fit into the rings");
  __shared__ __attribute__((aligned(1024))) char lds[kLds];
  float (*sh_o)[16][kPad] = reinterpret_cast<float (*)[16][kPad]>(lds);
  float (*sh_m)[16] = reinterpret_cast<float (*)[16]>(lds + kWaves * 16 * kPad * 4);
  float (*sh_l)[16] = sh_m + kWaves;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int rows_b = p.Hkv * p.head_tiles;
  char* const ring = lds + wave * (kRing * TL::kBytes);
  const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void*)ring;

  // What a lane copies: a 16-byte chunk of K and of V (of both halves at D =
  // 64), and four scale bytes (at D = 64 by half the lanes, the others again).
  const int copy_row = lane / TL::kChunks;
  const uint32_t copy_codes =
      (uint32_t)((copy_row & 15) * TL::kRow + (((lane % TL::kChunks) ^ TL::chunk_xor(copy_row)) * 16));
  const int copy_kv = (lane / (D / 4)) & 1, copy_blk = (lane >> 3) & (D / 32 - 1), copy_word = lane & 7;
  const uint32_t copy_scales = (uint32_t)(2 * kv4_code_bytes<D>(p.shift) + copy_kv * kv4_scale_bytes<D>(p.shift) +
                                          (copy_blk << p.shift) + 4 * (copy_word & 3));
  // What it reads: its token's chunk of K and the scale, and its dims of V and
  // the scales of their block.
  const int tok_k = 4 * (n & 3) + (n >> 2);
  const int read_k = tok_k * TL::kRow + (D == 128 ? (g ^ TL::chunk_xor(tok_k)) * 16
                                                  : ((g >> 1) ^ TL::chunk_xor(tok_k)) * 16 + (g & 1) * 8);
  const int read_ks = TL::kScales + (g * (D / 4) / 32) * kTile + tok_k;
  const int read_vs = TL::kScales + (D / 32 + n * DL / 32) * kTile;
  int read_v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = 4 * r + g, at = n * (D / 32);         // the byte of its row
    read_v[r] = TL::kCodes + row * TL::kRow + ((at >> 4) ^ TL::chunk_xor(row)) * 16 + (at & 15);
  }
  const uint32_t scale_turn = (uint32_t)(8 * g + 9) & 31;   // rotates byte g into the exponent's place

  // The list's length, and the sequence in which this share begins: the
  // first whose units end behind its first.  64 lengths at a time, a lane each.
  const int w = blockIdx.x;
  const int len0 = lane < p.B ? p.lens[lane] : 0;
  const int mine0 = units_of(seen_of(p, len0)), upto0 = wave_scan(mine0);
  int total = __builtin_amdgcn_readlane(upto0, 63);
  for (int i = 64; i < p.B; i += 64)
    total += __builtin_amdgcn_readlane(wave_scan(i + lane < p.B ? units_of(seen_of(p, p.lens[i + lane])) : 0), 63);
  const Shares shares = shares_of(p, total * rows_b);
  if (w >= shares.count) return;
  int at = shares.begin(w);
  const int end = shares.begin(w + 1);
  int b = -1, before = 0;
  Seen seen;
  for (int i = 0; i < p.B; i += 64) {
    const int len = i ? (i + lane < p.B ? p.lens[i + lane] : 0) : len0;
    const int mine = i ? units_of(seen_of(p, len)) : mine0;
    const int upto = before + (i ? wave_scan(mine) : upto0);
    const uint64_t past = __ballot(upto * rows_b > at);
    if (past) {
      const int k = __builtin_ctzll(past);
      b = i + k;
      before = __builtin_amdgcn_readlane(upto - mine, k);
      seen = seen_of(p, __builtin_amdgcn_readlane(len, k));
      break;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  if (b < 0) return;
  int row = (at - before * rows_b) / max(units_of(seen), 1);    // of the sequence
  int u0 = (at - before * rows_b) - row * units_of(seen);

  // From unit u1 of this row to the next row of the share; false at its end.  (The
  // lengths are read again for further sequences; were they changed meanwhile,
  // the conditions on row and b still keep every access in bounds.)
  auto next_row = [&](int u1) __attribute__((always_inline)) {
    at += u1 - u0;
    u0 = 0;
    if (at >= end) return false;
    if (++row < rows_b) return true;
    row = 0;
    do {
      if (++b == p.B) return false;
      seen = seen_of(p, scalar(p.lens)[b]);
    } while (seen.tiles == 0);
    return true;
  };
  for (bool wrote = false; row < rows_b;) {
    const int u1 = min(units_of(seen), u0 + (end - at));
    const int t0 = max(u0 - kStart, 0), t1 = max(u1 - kStart, 0);
    if (t0 >= t1) {                    // the start of a row, and none of its tiles
      if (!next_row(u1)) return;
      continue;
    }
    if (wrote) __syncthreads();        // the states of the row before have been read
    wrote = true;
    const int hk = row / p.head_tiles, ht = row - hk * p.head_tiles;
    const int hq0 = hk * p.group + ht * COLS;
    const int heads = min(p.group - ht * COLS, COLS);
    const int tok0 = seen.lo & ~(kTile - 1);
    const ScalarInts table = scalar(p.table + (int64_t)b * p.M);
    const uint32_t page_bytes = (uint32_t)p.Hkv * (uint32_t)kv4_block_bytes<D>(p.shift);    // under 2^31
    const uint64_t head = reinterpret_cast<uint64_t>(p.cache) + (uint32_t)(hk * kv4_block_bytes<D>(p.shift));

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

    // What the table has for a tile's halves (past its end: the last entry again);
    // in pages of 32 tokens or more both lie in one.
    const bool paired = (1 << p.shift) >= kTile;
    auto pages = [&](int t, int (&pg)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
        pg[s] = s && paired ? pg[0] : table[min((tok0 + t * kTile + 16 * s) >> p.shift, p.M - 1)];
    };
    // Start the copies of a tile into a slot of the ring.  A half without a page
    // is read from page 0, and masked: returns bit s for it.
    auto copy = [&](int t, const int (&pg)[2], int slot) __attribute__((always_inline)) {
      uint64_t codes[2], scales[2];
      uint32_t none = 0;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s && paired) {
          none |= none << 1;
          codes[1] = codes[0] + 16 * TL::kRow;
          scales[1] = scales[0] + 16;
          break;
        }
        const int first = tok0 + t * kTile + 16 * s;
        const int r = first & ((1 << p.shift) - 1);
        const bool there = (unsigned)pg[s] < (unsigned)p.pages && (first >> p.shift) < p.M;
        none |= there ? 0u : 1u << s;
        const uint64_t base = head + (uint64_t)(uint32_t)(there ? pg[s] : 0) * page_bytes;
        codes[s] = base + (uint32_t)(r * TL::kRow);
        scales[s] = base + (uint32_t)r;
      }
      const uint32_t to = ring_at + (uint32_t)(slot * TL::kBytes);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const uint32_t off = copy_codes + (uint32_t)(kv * kv4_code_bytes<D>(p.shift));
        if constexpr (D == 128) {
#pragma unroll
          for (int s = 0; s < 2; ++s)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                         : : "s"(to + (uint32_t)(kv * TL::kCodes + s * 1024)), "v"(off), "s"(codes[s]) : "memory", "m0");
        } else {
          const uint64_t at = (lane < 32 ? codes[0] : codes[1]) + off;
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt"
                       : : "s"(to + (uint32_t)(kv * TL::kCodes)), "v"(at) : "memory", "m0");
        }
      }
      const uint64_t at = (copy_word < 4 ? scales[0] : scales[1]) + copy_scales;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                   : : "s"(to + (uint32_t)TL::kScales), "v"(at) : "memory", "m0");
      return none;
    };

    // The wave's tiles: t0 + wave, and every kWaves-th from there.
    const int mine = t1 > t0 + wave ? (t1 - t0 - wave + kWaves - 1) / kWaves : 0;
    uint32_t missing = 0;           // two bits for each tile in flight, the next one's lowest
    int far[2] = {0, 0};
    int near[kRing][2];
#pragma unroll
    for (int k = 0; k < kRing; ++k) pages(t0 + wave + k * kWaves, near[k]);
    pages(t0 + wave + kRing * kWaves, far);
    // The loop's waits count copies: were what was loaded above still on its way, or a
    // spill among them, they would wait for more than their tile (never for less: in order).
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[c][s]));
      if (ALIBI) asm volatile("" : "+v"(slope[c]));
    }
#pragma unroll
    for (int k = 0; k < kRing; ++k)
      if (k < mine) missing |= copy(t0 + wave + k * kWaves, near[k], k) << (2 * k);
    int slot = 0;
    for (int k = 0; k < mine; ++k) {
      const int t = t0 + wave + k * kWaves;
      // This tile has arrived when only those behind it are in flight.
      const int behind = min(mine - 1 - k, kRing - 1);
      if (behind >= 3) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(3 * TL::kCopies) : "memory");
      else if (behind == 2) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * TL::kCopies) : "memory");
      else if (behind == 1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(TL::kCopies) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      static_assert(kRing <= 4, "the cases above");

      const char* tile = ring + slot * TL::kBytes;
      uint32_t kw[2][KS], vw[8], ks[2];
      u32x4 vs[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if constexpr (D == 128) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(tile + read_k + s * 16 * TL::kRow);
#pragma unroll
          for (int i = 0; i < KS; ++i) kw[s][i] = x[i];
        } else {
          const u32x2 x = *reinterpret_cast<const u32x2*>(tile + read_k + s * 16 * TL::kRow);
#pragma unroll
          for (int i = 0; i < KS; ++i) kw[s][i] = x[i];
        }
        ks[s] = *reinterpret_cast<const uint8_t*>(tile + read_ks + 16 * s);
        vs[s] = *reinterpret_cast<const u32x4*>(tile + read_vs + 16 * s);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const char* at = tile + read_v[r] + s * 16 * TL::kRow;
          if constexpr (D == 128) vw[4 * s + r] = *reinterpret_cast<const uint32_t*>(at);
          else vw[4 * s + r] = *reinterpret_cast<const uint16_t*>(at);
        }
      }
      const uint32_t lost = missing & 3;
      missing >>= 2;
      if (k + kRing < mine) {
        // The slot is free once its reads have returned.
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        missing |= copy(t + kRing * kWaves, far, slot) << (2 * (kRing - 1));
        pages(t + (kRing + 1) * kWaves, far);
      }
      if (++slot == kRing) slot = 0;

      const int tok = tok0 + t * kTile;
      // Scores: element 4 s + r is token 16 s + 4 r + g of the tile.
      float sc[NC][8], vscale[8], far_bias[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) far_bias[c] = ALIBI ? slope[c] * (float)(tok + g - (seen.hi - 1)) : 0.f;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const float scale = as_float(ks[s] << 23);
        f32x4 acc[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < KS; ++st) {
          const uint32_t word = kw[s][st];
          const u32x4 a = {Fp4<T>::template cvt<0>(word, scale), Fp4<T>::template cvt<1>(word, scale),
                           Fp4<T>::template cvt<2>(word, scale), Fp4<T>::template cvt<3>(word, scale)};
#pragma unroll
          for (int c = 0; c < NC; ++c) acc[c] = Mfma16<T>::mul(__builtin_bit_cast(vec8, a), q[c][st], acc[c]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t word = vs[s][r];
          vscale[4 * s + r] = as_float(__builtin_amdgcn_alignbit(word, word, scale_turn));
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            // The bias from the tile's and the token's part of the distance, one
            // rounding each.
            const float bias = ALIBI ? __builtin_fmaf(slope[c], (float)(16 * s + 4 * r), far_bias[c]) : 0.f;
            if (CAP) sc[c][4 * s + r] = acc[c][r] * p.c;
            else sc[c][4 * s + r] = ALIBI ? __builtin_fmaf(acc[c][r], p.c, bias) : acc[c][r] * p.c;
          }
        }
      }
      if (CAP) {
        auto capped = [&](auto cap) __attribute__((always_inline)) {
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float bias = ALIBI ? __builtin_fmaf(slope[c], (float)(16 * (i >> 2) + 4 * (i & 3)), far_bias[c]) : 0.f;
              sc[c][i] = cap(sc[c][i], bias);
            }
        };
        if (p.cap_inv != 0.f) capped([&](float x, float bias) { return high_cap(x, p) + bias; });
        else capped([&](float x, float bias) { return soft_cap(x, p.cap_k2, p.cap_cl, p.cap_cl + bias); });
      }
      if (tok < seen.lo || tok + kTile > seen.hi || lost) {
        // What is not seen: no weight, and no NaN from what its bytes hold.
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = tok + 16 * s + 4 * r + g;
            if (key < seen.lo || key >= seen.hi || (lost >> s & 1)) {
#pragma unroll
              for (int c = 0; c < NC; ++c) sc[c][4 * s + r] = kNegInf;
              vscale[4 * s + r] = 0.f;
            }
          }
      }
      // Lazy repair: the reference moves when a score exceeds it by more than kLazy.  A
      // weight goes to the matrix unit as two values of T, itself rounded and what that
      // leaves, so that P . V has the 32 bits of its sum and of its division: one value
      // alone, half a step of bf16 off, is most of the output's error (16 x 32768 tokens then
      // take 94.7 us, 96.9 with both; with 32 heads a KV head 122 and 143).
      vec8 pb[NC], pr[NC];
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
        u32x4 pw, rw;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pw[i] = Elem<T>::pack2(e[2 * i], e[2 * i + 1]);
          rw[i] = Elem<T>::pack2(e[2 * i] - Elem<T>::lo(pw[i]), e[2 * i + 1] - Elem<T>::hi(pw[i]));
        }
        pb[c] = __builtin_bit_cast(vec8, pw);
        pr[c] = __builtin_bit_cast(vec8, rw);
      }
      // O^T: byte h of a lane's dims of tokens 2 i and 2 i + 1 gives word i of
      // the operands of dims 2 h and 2 h + 1.
      auto block = [&](auto byte) __attribute__((always_inline)) {
        constexpr int h = decltype(byte)::value;
        u32x4 a0, a1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t u = Fp4<T>::template cvt<h>(vw[2 * i], vscale[2 * i]);
          const uint32_t v = Fp4<T>::template cvt<h>(vw[2 * i + 1], vscale[2 * i + 1]);
          a0[i] = __builtin_amdgcn_perm(v, u, 0x05040100u);
          a1[i] = __builtin_amdgcn_perm(v, u, 0x07060302u);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          o[c][2 * h] = Mfma16<T>::mul(__builtin_bit_cast(vec8, a0), pb[c], o[c][2 * h]);
          o[c][2 * h + 1] = Mfma16<T>::mul(__builtin_bit_cast(vec8, a1), pb[c], o[c][2 * h + 1]);
          o[c][2 * h] = Mfma16<T>::mul(__builtin_bit_cast(vec8, a0), pr[c], o[c][2 * h]);
          o[c][2 * h + 1] = Mfma16<T>::mul(__builtin_bit_cast(vec8, a1), pr[c], o[c][2 * h + 1]);
        }
      };
      block(std::integral_constant<int, 0>{});
      block(std::integral_constant<int, 1>{});
      if constexpr (D == 128) {
        block(std::integral_constant<int, 2>{});
        block(std::integral_constant<int, 3>{});
      }
    }

    // The waves' states, through LDS, 16 columns at a time.  Lane (n, g) holds
    // dims DL (4 g + r) + j of head n in element r of block j.
    const bool done = t0 == 0 && t1 == seen.tiles;
    const int64_t part = 2 * (int64_t)w + (t0 == 0 ? 1 : 0);    // the share's last row, or its first
    if (t0 == 0 && threadIdx.x == 0)   // the shares of the row: this one to the one of its last tile
      p.ws_rows[b * rows_b + row] = make_int2(w, done ? w : shares.of(at - u0 + units_of(seen) - 1));
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      l[c] += __shfl_xor(l[c], 16, 64);
      l[c] += __shfl_xor(l[c], 32, 64);
      __syncthreads();                 // every wave is done with its ring, or with the columns before
      if (16 * c + n < heads) {
        float* to = sh_o[wave][n];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < DL; j += 4)
            *reinterpret_cast<f32x4*>(to + DL * (4 * g + r) + j) =
                f32x4{o[c][j][r], o[c][j + 1][r], o[c][j + 2][r], o[c][j + 3][r]};
        if (g == 0) {
          sh_m[wave][n] = m[c];
          sh_l[wave][n] = l[c];
        }
      }
      __syncthreads();
      // (Not known to be the same at every row: its addresses would be held in
      // registers through the tile loops, which have none to spare.)
      int tid = threadIdx.x;
      asm volatile("" : "+v"(tid));
      for (int idx = tid; idx < min(heads - 16 * c, 16) * (D / 4); idx += kThreads) {
        const int in = idx / (D / 4), d = idx % (D / 4) * 4, h = 16 * c + in;
        float M = kNegInf;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) M = fmaxf(M, sh_m[i][in]);
        float L = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          const float f = sh_m[i][in] == kNegInf ? 0.f : fast_exp2(sh_m[i][in] - M);
          L = __builtin_fmaf(sh_l[i][in], f, L);
          acc += f * *reinterpret_cast<const f32x4*>(&sh_o[i][in][d]);
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
    }
    if (!next_row(u1)) return;
  }
}

// Rows in several shares: one workgroup per (sequence, query head).  D / 4 lanes
// hold a row's dims, and the lane groups take its parts in turn.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void decode_kv4_combine_kernel(Kv4DecodeParams p) {
  constexpr int CH = D / 4, NG = kThreads / CH, kBatch = 4;
  __shared__ float sh_m[NG], sh_l[NG];
  __shared__ f32x4 sh_o[NG][CH];
  const int b = blockIdx.x / p.Hq, hq = blockIdx.x - b * p.Hq;
  const int cols = kv4_columns(p.group);
  const int hk = hq / p.group, in = hq - hk * p.group, ht = in / cols, h = in - ht * cols;
  const int ch = threadIdx.x % CH, g = threadIdx.x / CH;
  int2 span = p.ws_rows[(b * p.Hkv + hk) * p.head_tiles + ht];   // (of a row without tiles: not looked at)
  span.x = min(max(span.x, 0), p.shares - 1);                    // (and in bounds whatever it says)
  span.y = min(max(span.y, 0), p.shares - 1);
  T* out = static_cast<T*>(p.o) + (int64_t)blockIdx.x * D + 4 * ch;
  if (p.lens[b] <= 0) {
    if (g == 0) *reinterpret_cast<uint2*>(out) = make_uint2(0u, 0u);
    return;
  }
  if (span.x == span.y) return;               // the split kernel has written it

  float M = kNegInf, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int w0 = span.x + g; w0 <= span.y; w0 += NG * kBatch) {
    float m[kBatch], l[kBatch];
    f32x4 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {   // past the last part: that part again, left out below
      const int w = min(w0 + u * NG, span.y);
      const int64_t at = (2 * (int64_t)w + (w == span.x ? 1 : 0)) * cols + h;
      m[u] = p.ws_m[at];
      l[u] = p.ws_l[at];
      v[u] = *reinterpret_cast<const f32x4*>(p.ws_o + at * D + 4 * ch);
    }
    // (Not loaded under the conditions below, one after another.)
#pragma unroll
    for (int u = 0; u < kBatch; ++u) asm volatile("" : "+v"(v[u]), "+v"(l[u]), "+v"(m[u]));
    float mn = M;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) mn = fmaxf(mn, m[u]);
    const float a = M == kNegInf ? 0.f : fast_exp2(M - mn);
    L *= a;
    acc *= a;
    M = mn;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (w0 + u * NG <= span.y) {       // (weight 0 where m is -inf: a NaN there stays one)
        const float e = m[u] == kNegInf ? 0.f : fast_exp2(m[u] - mn);
        L = __builtin_fmaf(e, l[u], L);
        acc += e * v[u];
      }
    }
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

int kv4_shares(int D, int group, int cus) { return cus * per_unit(D, kv4_columns(group)); }

hipError_t launch_decode_kv4(const Kv4DecodeParams& p, hipStream_t stream) {
  // No more workgroups than the longest contexts that the tables hold could use.
  const int64_t most = (((int64_t)p.M << p.shift) / kTile + 2 + kStart) * p.B * p.Hkv * p.head_tiles;
  const int64_t blocks = std::min<int64_t>(p.shares, (most + kLeast - 1) / kLeast);
  if (p.D == 64) return p.bf16 ? launch_cols<64, __bf16>(p, blocks, stream) : launch_cols<64, _Float16>(p, blocks, stream);
  return p.bf16 ? launch_cols<128, __bf16>(p, blocks, stream) : launch_cols<128, _Float16>(p, blocks, stream);
}

}  // namespace attn
