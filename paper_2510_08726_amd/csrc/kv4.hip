// The paged 4-bit cache (include/kv4.h): where new tokens go, writing them, and
// reading them back.  The conversions between E2M1 and 16 bits are gfx950
// instructions, which take the block's power of two as an operand.

#include <algorithm>

#include "kernel_common.h"
#include "kv4_common.h"
#include "launch.h"

namespace attn {

namespace {

constexpr int kThreads = 256;

// Inclusive sum over the workgroup; every thread must call.  `total` is the
// last one's.  sh: one int per wave.
__device__ __forceinline__ int block_scan(int x, int* sh, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  __syncthreads();                       // sh is free
  if (lane == 63) sh[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const int y = sh[w];
    before += w < wave ? y : 0;
    all += y;
  }
  total = all;
  return x + before;
}

struct Need {
  int n, count, held, need;   // tokens now and new, pages now and new
};

__device__ __forceinline__ Need need_of(const SlotsParams& p, int b) {
  const int page = 1 << p.shift, room = p.M << p.shift;
  Need r;
  r.n = min(max(p.lens[b], 0), room);
  r.count = min(max(p.counts[b], 0), p.L);
  r.held = (int)(((int64_t)r.n + page - 1) >> p.shift);
  const int64_t want = min((int64_t)r.n + r.count, (int64_t)room);
  r.need = (int)((want + page - 1) >> p.shift) - r.held;
  return r;
}

// A workgroup takes kItems consecutive (sequence, token) items.  It sums the needs
// of the sequences before its first (those of whole 256s at once, the others in
// the scan of its own), and writes each item's slot; the item in a new page's
// first row writes the page into the table.  No workgroup waits for another: each reads the
// lengths before its own, which the caches hold.  Latency bound: three dependent
// reads (lengths, page, and the table's or the list's) and three barriers (two more for each further
// 256 sequences, and two for those before), 2.1 us for 64 requests of one token;
// 256 requests of up to 2048 tokens write 6.3 MB in 4.8 us.
constexpr int kItems = 512;

__global__ __launch_bounds__(kThreads) void kv_slots_kernel(SlotsParams p) {
  __shared__ int wave_sum[kThreads / 64];
  __shared__ int start[kItems], held[kItems], stored[kItems], len[kItems];
  const uint32_t L = (uint32_t)p.L, items = (uint32_t)p.B * L, i0 = blockIdx.x * kItems;
  const uint32_t i1 = min(i0 + kItems, items);
  const int b0 = (int)(i0 / L), b1 = (int)((i1 - 1) / L);
  const int c0 = b0 & ~(kThreads - 1);
  int base = 0;
  if (c0 > 0) {
    int before = 0;
    for (int b = threadIdx.x; b < c0; b += kThreads) before += need_of(p, b).need;
    block_scan(before, wave_sum, base);
  }
  for (int c = c0; c <= b1; c += kThreads) {
    const int b = c + threadIdx.x;
    Need r{};
    if (b <= b1) r = need_of(p, b);
    int total;
    const int from = base + block_scan(r.need, wave_sum, total) - r.need;
    if (b >= b0 && b <= b1) {
      const int got = min(max(p.nfree - from, 0), r.need);
      const int64_t fit = ((int64_t)(r.held + got) << p.shift) - r.n;
      start[b - b0] = from;
      held[b - b0] = r.held;
      stored[b - b0] = (int)min(fit, (int64_t)r.count);
      len[b - b0] = r.n;
    }
    base += total;
  }
  __syncthreads();
  if (i1 == items && threadIdx.x == 0) *p.taken = min(base, p.nfree);
  const int mask = (1 << p.shift) - 1;
#pragma unroll
  for (int u = 0; u < kItems / kThreads; ++u) {
    const uint32_t i = i0 + u * kThreads + threadIdx.x;
    if (i >= i1) break;
    const uint32_t b = i / L, l = i - b * L;
    const int k = (int)b - b0;
    const int64_t pos = (int64_t)len[k] + l;
    int64_t slot = -1;
    if ((int)l < stored[k]) {
      const int pi = (int)(pos >> p.shift), row = (int)pos & mask;
      int* entry = p.table + (int64_t)b * p.M + pi;
      const bool fresh = pi >= held[k];
      const int page = fresh ? p.free_pages[start[k] + pi - held[k]] : *entry;
      if (fresh && row == 0) *entry = page;
      if (page >= 0) slot = ((int64_t)page << p.shift) + row;
    }
    p.slots[i] = slot;
    p.positions[i] = (int)pos;
    if (l == 0) p.new_lens[b] = len[k] + stored[k];
  }
}

// Grids of the two kernels below: a workgroup's lanes are the rows of neighbouring
// tokens of one head, blockIdx.y is the head, and blockIdx.z strides the sequences.
// (More tokens a thread, 2, 4 and 8 with all their loads in flight, took 4, 13 and 27 % longer
// than one: the rows of a workgroup then lie further apart.)

// Four lanes hold a block of 32 dims, 8 each: 16 bytes in, 4 bytes out, K and V in
// one thread.  The input is streamed past the caches, which the cache's lines need until
// all rows of a line are written (47.1 us for 8 prompts of up to 4095 tokens and their reading
// back, 51.9 without).  The slot decides whether a row is read at all, so that padding is
// not: two round trips in a row, where kv4_load's codes have one (88 MB in 21.6 us, 4.1
// TB/s; kv4_load 6.6).
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(Kv4AppendParams p) {
  constexpr int LPR = D / 8;                 // lanes per row
  constexpr int kTop = __is_same(T, _Float16) ? 13 : 125;
  const int lig = threadIdx.x % LPR, h = blockIdx.y;
  const int l = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  if (l >= p.L) return;
  for (int b = blockIdx.z; b < p.B; b += gridDim.z) {
    const int64_t slot = p.slots[(int64_t)b * p.L + l];
    if (slot < 0 || slot >= (int64_t)p.pages << p.shift) continue;    // the lanes of a row agree
    u32x4 x[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      x[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
          static_cast<const T*>(p.x[k]) + b * p.sb[k] + h * p.sh[k] + l * p.sl[k] + 8 * lig));
    const int r = (int)slot & ((1 << p.shift) - 1);
    unsigned char* base = p.cache + ((slot >> p.shift) * p.H + h) * (int64_t)kv4_block_bytes<D>(p.shift);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = Elem<T>::lo(x[k][i]);
        f[2 * i + 1] = Elem<T>::hi(x[k][i]);
      }
      // The largest magnitude as bits: ordered as the values are, infinities
      // and NaN above them.
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = f[i];
        top = max(top, __builtin_bit_cast(uint32_t, v) & 0x7fffffffu);
      }
      top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));   // quad_perm [1,0,3,2]
      top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));   // quad_perm [2,3,0,1]
      const bool fine = top < 0x7f800000u;
      // 2^e with a <= 7 2^e: the exponent of a less 2, one more over 1.75 of its binade.
      int e = (int)((top + 0x1fffffu) >> 23) - 129;
      e = min(max(e, -kTop), kTop);
      const uint32_t inv = (uint32_t)(127 - e) << 23;
      const float s = __builtin_bit_cast(float, inv);
      // Scaled first: the products are exact.
      uint32_t code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f[0] * s, f[1] * s, 1.f, 0);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[2] * s, f[3] * s, 1.f, 1);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[4] * s, f[5] * s, 1.f, 2);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[6] * s, f[7] * s, 1.f, 3);
      if (!fine) code = 0;
      *reinterpret_cast<uint32_t*>(base + k * kv4_code_bytes<D>(p.shift) + r * (D / 2) + 4 * lig) = code;
      if ((lig & 3) == 0)
        base[2 * kv4_code_bytes<D>(p.shift) + k * kv4_scale_bytes<D>(p.shift) + ((lig >> 2) << p.shift) + r] =
            (unsigned char)(fine ? e + 127 : 255);
    }
  }
}

// 8 dims a lane: 4 bytes of codes and a scale byte in, 16 bytes out.  The stores are
// ordinary ones, since attention reads K and V next: 30000 tokens, 36 us, and a piece of 64
// queries take 81 us together, 92 with streamed stores (the load alone 35).
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv4_load_kernel(Kv4LoadParams p) {
  constexpr int LPR = D / 8;
  const int lig = threadIdx.x % LPR, h = blockIdx.y;
  const int l = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  if (l >= p.L) return;
  for (int b = blockIdx.z; b < p.B; b += gridDim.z) {
    const int64_t t = (int64_t)(p.starts ? max(p.starts[b], 0) : 0) + l;
    const int64_t n = min((int64_t)p.lens[b], (int64_t)p.M << p.shift);
    const int pg = t < n ? p.table[(int64_t)b * p.M + (t >> p.shift)] : -1;
    uint32_t code[2] = {0u, 0u}, scale[2] = {0u, 0u};
    if ((unsigned)pg < (unsigned)p.pages) {
      const int r = (int)t & ((1 << p.shift) - 1);
      const unsigned char* base = p.cache + ((int64_t)pg * p.H + h) * (int64_t)kv4_block_bytes<D>(p.shift);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        code[k] = *reinterpret_cast<const uint32_t*>(base + k * kv4_code_bytes<D>(p.shift) + r * (D / 2) + 4 * lig);
        scale[k] = base[2 * kv4_code_bytes<D>(p.shift) + k * kv4_scale_bytes<D>(p.shift) + ((lig >> 2) << p.shift) + r];
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t bits = scale[k] << 23;
      const float s = __builtin_bit_cast(float, bits);
      const u32x4 out = {Fp4<T>::template cvt<0>(code[k], s), Fp4<T>::template cvt<1>(code[k], s),
                         Fp4<T>::template cvt<2>(code[k], s), Fp4<T>::template cvt<3>(code[k], s)};
      *reinterpret_cast<u32x4*>(static_cast<T*>(p.y[k]) + (((int64_t)b * p.H + h) * p.L + l) * D + 8 * lig) = out;
    }
  }
}

template <int D>
dim3 grid_of(int B, int H, int L) {
  constexpr int kTokens = kThreads / (D / 8);
  return dim3((unsigned)((L + kTokens - 1) / kTokens), (unsigned)H, (unsigned)std::min(B, 65535));
}

template <int D, typename T>
hipError_t append(const Kv4AppendParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((kv4_append_kernel<D, T>), grid_of<D>(p.B, p.H, p.L), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

template <int D, typename T>
hipError_t load(const Kv4LoadParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((kv4_load_kernel<D, T>), grid_of<D>(p.B, p.H, p.L), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_slots(const SlotsParams& p, hipStream_t stream) {
  const int64_t blocks = ((int64_t)p.B * p.L + kItems - 1) / kItems;
  hipLaunchKernelGGL(kv_slots_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_kv4_append(const Kv4AppendParams& p, hipStream_t stream) {
  if (p.D == 64) return p.bf16 ? append<64, __bf16>(p, stream) : append<64, _Float16>(p, stream);
  return p.bf16 ? append<128, __bf16>(p, stream) : append<128, _Float16>(p, stream);
}

hipError_t launch_kv4_load(const Kv4LoadParams& p, hipStream_t stream) {
  if (p.D == 64) return p.bf16 ? load<64, __bf16>(p, stream) : load<64, _Float16>(p, stream);
  return p.bf16 ? load<128, __bf16>(p, stream) : load<128, _Float16>(p, stream);
}

}  // namespace attn
