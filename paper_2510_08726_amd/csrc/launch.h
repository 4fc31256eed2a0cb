// Host-side launch interface between the C ABI (attn_api.cpp) and the kernels.
#pragma once

#include <hip/hip_runtime_api.h>
#include <hip/hip_vector_types.h>
#include <stddef.h>
#include <stdint.h>

namespace attn {

struct PrefillParams {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  const float* slopes;  // device, [Hq], or nullptr
  int B, Hq, Hkv, Lq, Lk, D;
  int group;            // Hq / Hkv
  bool causal, bf16;
  bool sorted;          // prefill.hip: a share's items go out heaviest first, set by the launcher
  float c;              // |scale| * log2(e) without ALiBi or SoftCap, scale * log2(e) with either
  unsigned qsign;       // 0x80008000 to negate Q (negative scale, no ALiBi or SoftCap), else 0
  float cap_k2;         // SoftCap: 2 / cap
  float cap_cl;         // SoftCap: cap * log2(e), or 0 for no cap
  int window;           // sliding window (keys per row, causal only), 0 for none
  int nqb;              // query blocks per head
  int nheads;           // B * Hq, set by the launcher
  int nitems;           // nqb * nheads, set by the launcher
  int nxcd;             // shares of the items, each with its own workgroups: the XCDs, or 1; set by the launcher
  int hg;               // query heads per workgroup (sharing one KV head), set by the launcher
};
// The kernel reads its arguments and, behind them, the grid size: within two
// cache lines here.  (24 bytes more, and one of the next line, were 0.2 us of a
// 25.9 us call.)
static_assert(sizeof(PrefillParams) + 4 <= 128, "arguments and grid size within two lines");

struct PrefillSplitParams : PrefillParams {
  int splits;           // key ranges (1: none)
  float* ws;            // partials, for splits > 1: [splits, B*Hq*Lq, D], then (max, sum) [splits, B*Hq*Lq, 2]
};

struct DecodeParams {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  const float* slopes;  // device, [Hq], or nullptr
  float* ws_o;          // [B*Hq*S, D]
  float* ws_m;          // [B*Hq*S]
  float* ws_l;          // [B*Hq*S]
  int B, Hq, Hkv, Lk, D;
  int group;            // Hq / Hkv
  int splits;           // S
  int chunk;            // ceil(Lk / S)
  int bf16;
  float c;              // scale * log2(e)
  float cap_k2;         // SoftCap: 2 / cap
  float cap_cl;         // SoftCap: cap * log2(e), or 0 for no cap
};

// Template flags of the prefill kernel that a call launches.  SoftCap and the
// sliding window are built for the causal mask (the entry point rejects the
// other combinations), SoftCap without ALiBi.
struct PrefillFlags {
  bool causal, alibi, cap, win;
};
inline PrefillFlags prefill_flags(bool causal, bool alibi, bool cap, bool win) {
  return {causal || cap || win, alibi && !cap, cap, win};
}

// Decode kernel for a GQA group of `group` query heads per KV head: 0 for the
// grouped matrix-unit kernel (2..32 heads), else the heads per workgroup of
// the vector split kernel (the largest of 8, 4, 2, 1 dividing the group).
inline int decode_split_heads(int group) {
  if (group >= 2 && group <= 32) return 0;
  if (group % 8 == 0) return 8;
  if (group % 4 == 0) return 4;
  if (group % 2 == 0) return 2;
  return 1;
}

int prefill_block_rows();
// Order of the items of prefill.hip: 0 KV head major, 1 heaviest first within
// each XCD's share, 2 heaviest first over all.
int prefill_order(int nitems, int nqb, int slots, bool causal, int window, int Lk, int64_t kv_bytes);
hipError_t launch_prefill(const PrefillParams& p, hipStream_t stream);
// Few query rows: keys split inside the workgroup, and with a workspace over
// workgroups (prefill_split.hip), where the plan of the call says so.
constexpr int kMaxPrefillSplits = 32;
struct PrefillSplitPlan {
  int kgroups;          // key groups of its workgroups (2 or 4), or 0: prefill.hip runs
  int splits;           // key ranges over workgroups that it wants (needs a workspace when > 1)
};
PrefillSplitPlan prefill_split_plan(int B, int Hq, int Hkv, int Lq, int Lk, int D, bool causal, int window, bool alibi,
                                    bool cap, int cus, int max_splits);
hipError_t launch_prefill_split(const PrefillSplitParams& p, int kgroups, hipStream_t stream);
// One per (head dim, element type); launch_prefill dispatches to them.
hipError_t launch_prefill_d128_f16(const PrefillParams& p, hipStream_t stream);
hipError_t launch_prefill_d128_bf16(const PrefillParams& p, hipStream_t stream);
hipError_t launch_prefill_d64_f16(const PrefillParams& p, hipStream_t stream);
hipError_t launch_prefill_d64_bf16(const PrefillParams& p, hipStream_t stream);
hipError_t launch_decode(const DecodeParams& p, hipStream_t stream);

// Bytes of the static decode workspace of attn_decode_noalloc.
constexpr size_t kDecodeScratchBytes = size_t(16) << 20;
// Device address of that workspace on the current device (resolved once per
// device, then cached).
hipError_t decode_scratch(void** ptr);

// Row reductions (norms.hip): the stable L2 norm, or RMSNorm with its row max.
struct NormParams {
  const void* x;
  void* y;              // RMSNorm output [N, M], or nullptr
  float* out;           // [N]: the norms, or the row maxima of y
  float* ws_r;          // [N * chunks] partials r
  float* ws_t;          // [N * chunks] partials t
  int N, M;
  int chunks;           // chunks per row
  int chunk;            // elements per chunk (whole 16-byte vectors)
  int dtype;            // 0 fp16, 1 bf16, 2 fp32
  int rms;              // 1: RMSNorm with row max, 0: L2 norm
  float eps;
  float invM;           // 1 / M
  int lanes;            // lanes per row of the row kernels, set by the launcher
};
hipError_t launch_norm(const NormParams& p, hipStream_t stream);
// Longest row (bytes) that RMSNorm with one chunk per row holds in the
// registers of one workgroup (1024 lanes x 16 vectors of 16 bytes), reading X once.
constexpr long long kNormRowBytes = 1024LL * 16 * 16;
// True when a row reduction with `chunks` chunks per row runs one kernel
// (a wave or a workgroup per row: the L2 norm always, RMSNorm when the row fits)
// rather than the chunk partials and a second kernel.
inline bool norm_one_kernel(bool rms, long long M, int elem, int chunks) {
  return chunks == 1 && (!rms || M * elem <= kNormRowBytes);
}

// Rotary positions (rope.hip).
struct RopeParams {
  const void* x[2];     // queries, keys (or nullptr)
  void* y[2];
  int64_t sb[2], sh[2], sl[2];   // strides in elements of x
  int H[2];
  int B, L, D, R;       // R: rotary dim
  const void* pos;
  int64_t pos_stride;
  const double* freqs;
  float magnitude, sign;   // sign -1: the transposed rotation
  bool pos64, interleaved;
  int dtype;            // 0 fp16, 1 bf16, 2 fp32
};
hipError_t launch_rope(const RopeParams& p, hipStream_t stream);

// The paged 4-bit cache (kv4.hip).
struct SlotsParams {
  const int* lens;
  const int* counts;
  int* table;
  const int* free_pages;
  int64_t* slots;
  int* positions;
  int* new_lens;
  int* taken;
  int nfree, B, M, L, shift;   // shift: log2 of the page size
};
hipError_t launch_slots(const SlotsParams& p, hipStream_t stream);

struct Kv4AppendParams {
  const void* x[2];     // K, V
  int64_t sb[2], sh[2], sl[2];   // strides in elements
  unsigned char* cache;
  const int64_t* slots;
  int B, H, L, D, pages, shift;
  bool bf16;
};
hipError_t launch_kv4_append(const Kv4AppendParams& p, hipStream_t stream);

struct Kv4LoadParams {
  const unsigned char* cache;
  const int* table;
  const int* starts;    // or nullptr
  const int* lens;
  void* y[2];           // K, V
  int B, H, L, D, pages, shift, M;
  bool bf16;
};
hipError_t launch_kv4_load(const Kv4LoadParams& p, hipStream_t stream);

// Decode attention over it (decode_kv4.hip).
struct Kv4DecodeParams {
  const void* q;
  const unsigned char* cache;
  const int* table;
  const int* lens;
  void* o;
  const float* slopes;  // device, [Hq], or nullptr
  float* ws_o;          // [2 * shares, columns, D]
  float* ws_m;          // [2 * shares, columns], log2 units
  float* ws_l;
  int2* ws_rows;        // [B, Hkv, head_tiles]: a row's first and last share
  int B, Hq, Hkv, D, group;
  int pages, shift, M;
  int window;           // 0 for none
  int head_tiles;       // column tiles of the query heads of a KV head
  int shares;           // most workgroups
  int bf16;
  float c;              // scale * log2(e)
  float cap_k2, cap_cl; // as DecodeParams, both finite
  float cap_inv;        // 1 / cap_cl for a cap above kKv4HighCap, else 0
};
// What a row of the list of tiles counts beside them: 32 uneven requests of 16
// KV heads take 66.6 us with 0, 28.5 with 4, 25.7 with 8, 26.3 with 12, 27.4 with 16 and 29.3 with 24.
constexpr int kKv4RowStart = 8;
// SoftCap caps up to which cap tanh(s / cap) is formed as 1 - 2 / (1 + e^2t), which is off
// by 2^-22 of the cap: 1.5e-5 at 64, as a score of 60 in 32 bits is, but 0.01 at 1e5.
// Above, scores far under the cap take a series: 8 x 32 / 16 heads of 8192 tokens 36.7 us
// instead of 33.3.
constexpr float kKv4HighCap = 64.f;
// Query heads that one workgroup serves: 16 or 32 matrix columns.  More than 16
// in two workgroups of 16 read K and V twice: 16 x 40 / 2 heads of 32768 tokens 53.7 us
// against 43.5, 16 x 256 / 8 196 against 143 (but 8 x 40 / 2 of 1500 10.3 against 12.0).
constexpr int kv4_columns(int group) { return group <= 16 ? 16 : 32; }
// Workgroups of the split kernel on a device of `cus` compute units.
int kv4_shares(int D, int group, int cus);
hipError_t launch_decode_kv4(const Kv4DecodeParams& p, hipStream_t stream);

// Compute units of the current device, 256 if it cannot be queried (attn_api.cpp).
int compute_units();
// Keeps the error for attn_last_hip_error; returns ATTN_ERR_HIP (attn_api.cpp).
int hip_fail(hipError_t e);

// Achievable-peak probes (peaks.hip).
hipError_t launch_hbm_read(const void* buf, size_t bytes, float* sink, hipStream_t stream);
int hbm_read_sink_floats();
hipError_t launch_mfma_loop(int bf16, int iters, const void* operands, float* sink, unsigned long long* clocks,
                            hipStream_t stream);
int mfma_loop_waves();
size_t mfma_loop_operand_bytes();

}  // namespace attn
