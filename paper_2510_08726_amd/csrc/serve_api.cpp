// C ABI of the operators around the 4-bit cache (include/rope.h, include/kv4.h):
// argument validation on the host, before anything is enqueued.

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <limits>

#include "../../include/attn.h"
#include "../../include/kv4.h"
#include "../../include/rope.h"
#include "launch.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kMaxInt = std::numeric_limits<int32_t>::max();
constexpr int64_t kMaxElements = int64_t(1) << 40;
constexpr int64_t kMaxTokens = int64_t(1) << 30;   // that a sequence's table row may hold

constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;   // workgroups of 256 threads in a row of a grid: under 2^32 threads

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

// log2 of a page size, or -1.
int page_shift(int page) {
  if (page < 16 || page > 32768 || (page & (page - 1))) return -1;
  return __builtin_ctz((unsigned)page);
}

int done(hipError_t e) { return e == hipSuccess ? ATTN_OK : attn::hip_fail(e); }

int rope(const void* Q, const long long* q_strides, void* Qo, int Hq, const void* K, const long long* k_strides,
         void* Ko, int Hkv, int B, int L, int D, const void* positions, int positions_bits,
         long long positions_stride, const double* freqs, int rotary_dim, int interleaved, float magnitude, int dtype,
         float sign, hipStream_t stream) {
  if (!Q || !q_strides || !Qo || !positions || !freqs || (K && (!k_strides || !Ko))) return ATTN_ERR_NULL;
  if (B < 1 || L < 1 || Hq < 1 || D < 2 || rotary_dim < 2 || rotary_dim > D || rotary_dim % 2) return ATTN_ERR_SHAPE;
  if ((K ? Hkv < 1 : Hkv != 0) || !std::isfinite(magnitude) || positions_stride < 0) return ATTN_ERR_SHAPE;
  if (positions_bits != 32 && positions_bits != 64) return ATTN_ERR_SHAPE;
  if (dtype < ROPE_F16 || dtype > ROPE_F32) return ATTN_ERR_UNSUPPORTED;
  // At most a thread for each pair or copied element, and a grid row for each head.
  if ((int64_t)B * L > kMaxInt / D || (int64_t)Hq + Hkv > 65535) return ATTN_ERR_SHAPE;
  attn::RopeParams p{};
  p.x[0] = Q; p.y[0] = Qo; p.H[0] = Hq;
  p.sb[0] = q_strides[0]; p.sh[0] = q_strides[1]; p.sl[0] = q_strides[2];
  if (K) {
    p.x[1] = K; p.y[1] = Ko; p.H[1] = Hkv;
    p.sb[1] = k_strides[0]; p.sh[1] = k_strides[1]; p.sl[1] = k_strides[2];
  }
  p.B = B; p.L = L; p.D = D; p.R = rotary_dim;
  p.pos = positions; p.pos64 = positions_bits == 64; p.pos_stride = positions_stride;
  p.freqs = freqs;
  p.magnitude = magnitude;
  p.sign = sign;
  p.interleaved = interleaved != 0;
  p.dtype = dtype;
  return done(attn::launch_rope(p, stream));
}

// Sizes of calls on a cache: a grid row for each head, and elements that stay addressable.
bool cache_ok(int B, int Hkv, int L, int pages) {
  return B >= 1 && Hkv >= 1 && Hkv <= 65535 && L >= 1 && pages >= 1 && (int64_t)B * L <= kMaxInt &&
         (int64_t)B * L <= kMaxElements / (128 * (int64_t)Hkv);
}

// A thread for every 8 dims of L tokens in a row of the grid of kv4_append and kv4_load.
bool tokens_ok(int L, int D) { return L <= kMaxGroups * (2048 / D); }

bool kv4_type(int D, attn_dtype dtype) {
  return (D == 64 || D == 128) && (dtype == ATTN_F16 || dtype == ATTN_BF16);
}

// The bytes that an operand spans.
struct Span {
  uintptr_t begin, end;
};

Span span(const void* p, int64_t bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at, p ? at + (uintptr_t)bytes : at};
}

// Those of rows of D 16-bit elements, with strides of batches, heads and tokens of either sign.
Span span(const void* p, const long long* strides, int B, int H, int L, int D) {
  const int n[3] = {B, H, L};
  __int128 low = 0, high = D;
  for (int i = 0; i < 3; ++i) {
    const __int128 reach = (__int128)(n[i] - 1) * strides[i];
    (reach < 0 ? low : high) += reach;
  }
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at + (uintptr_t)(2 * low), at + (uintptr_t)(2 * high)};
}

// Whether `out`, which a call writes, lies apart from all the others.
bool apart(Span out, std::initializer_list<Span> others) {
  for (const Span& x : others)
    if (x.begin < out.end && out.begin < x.end) return false;
  return true;
}

// (More than 2^62 bytes are no cache.)
int64_t cache_bytes(int pages, int Hkv, int page, int D) {
  return (int64_t)std::min((__int128)kv4_page_bytes(page, D) * Hkv * pages, (__int128)1 << 62);
}

}  // namespace

extern "C" {

int rope_frequencies(int rotary_dim, double base, int scaling, double factor, double original_length, double slow,
                     double fast, double* freqs) {
  if (!freqs) return ATTN_ERR_NULL;
  if (scaling < ROPE_PLAIN || scaling > ROPE_PARTS) return ATTN_ERR_UNSUPPORTED;
  if (rotary_dim < 2 || rotary_dim % 2 || !std::isfinite(base) || base <= 0) return ATTN_ERR_SHAPE;
  if (scaling != ROPE_PLAIN && (!std::isfinite(factor) || factor <= 0)) return ATTN_ERR_SHAPE;
  if (scaling == ROPE_BASE && rotary_dim < 4) return ATTN_ERR_SHAPE;
  if (scaling == ROPE_PARTS && (!std::isfinite(original_length) || original_length <= 0 || !std::isfinite(slow) ||
                                !std::isfinite(fast) || slow < 0 || fast <= slow))
    return ATTN_ERR_SHAPE;
  if (scaling == ROPE_BASE) base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
  if (!std::isfinite(base)) return ATTN_ERR_SHAPE;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rotary_dim);
    if (scaling == ROPE_LINEAR) f /= factor;
    if (scaling == ROPE_PARTS) {
      const double turns = original_length * f / 6.283185307179586;
      const double w = std::min(std::max((turns - slow) / (fast - slow), 0.0), 1.0);
      f = f * w + f / factor * (1.0 - w);
    }
    if (!std::isfinite(f)) return ATTN_ERR_SHAPE;
    freqs[i] = f;
  }
  return ATTN_OK;
}

int rope_fwd(const void* Q, const long long* q_strides, void* Qo, int Hq, const void* K, const long long* k_strides,
             void* Ko, int Hkv, int B, int L, int D, const void* positions, int positions_bits,
             long long positions_stride, const double* freqs, int rotary_dim, int interleaved, float magnitude,
             rope_dtype dtype, hipStream_t stream) {
  return rope(Q, q_strides, Qo, Hq, K, k_strides, Ko, Hkv, B, L, D, positions, positions_bits, positions_stride, freqs,
              rotary_dim, interleaved, magnitude, dtype, 1.f, stream);
}

int rope_bwd(const void* dQ, const long long* q_strides, void* dQo, int Hq, const void* dK, const long long* k_strides,
             void* dKo, int Hkv, int B, int L, int D, const void* positions, int positions_bits,
             long long positions_stride, const double* freqs, int rotary_dim, int interleaved, float magnitude,
             rope_dtype dtype, hipStream_t stream) {
  return rope(dQ, q_strides, dQo, Hq, dK, k_strides, dKo, Hkv, B, L, D, positions, positions_bits, positions_stride,
              freqs, rotary_dim, interleaved, magnitude, dtype, -1.f, stream);
}

size_t kv4_page_bytes(int page, int D) {
  if (page_shift(page) < 0 || (D != 64 && D != 128)) return 0;
  return (size_t)page * D / 16 * 17;
}

int kv_slots(const int* lens, const int* counts, int* table, const int* free_pages, int nfree, int B, int max_pages,
             int page, int L, long long* slots, int* positions, int* new_lens, int* taken, hipStream_t stream) {
  if (!lens || !counts || !table || !slots || !positions || !new_lens || !taken || (nfree > 0 && !free_pages))
    return ATTN_ERR_NULL;
  const int shift = page_shift(page);
  if (B < 1 || L < 1 || max_pages < 1 || nfree < 0 || shift < 0 || new_lens == lens) return ATTN_ERR_SHAPE;
  if ((int64_t)B * L > kMaxInt || (int64_t)B * max_pages > kMaxInt || ((int64_t)max_pages << shift) > kMaxTokens)
    return ATTN_ERR_SHAPE;
  if (((int64_t)max_pages << shift) + L > kMaxInt + 1) return ATTN_ERR_SHAPE;    // positions are int
  attn::SlotsParams p{};
  p.lens = lens; p.counts = counts; p.table = table; p.free_pages = free_pages; p.nfree = nfree;
  p.B = B; p.M = max_pages; p.L = L; p.shift = shift;
  static_assert(sizeof(long long) == sizeof(int64_t), "slots are 64 bits");
  p.slots = reinterpret_cast<int64_t*>(slots);
  p.positions = positions; p.new_lens = new_lens; p.taken = taken;
  return done(attn::launch_slots(p, stream));
}

int kv4_append(const void* K, const long long* k_strides, const void* V, const long long* v_strides, void* cache,
               const long long* slots, int B, int Hkv, int L, int D, int pages, int page, attn_dtype dtype,
               hipStream_t stream) {
  if (!K || !k_strides || !V || !v_strides || !cache || !slots) return ATTN_ERR_NULL;
  const int shift = page_shift(page);
  if (!cache_ok(B, Hkv, L, pages) || shift < 0) return ATTN_ERR_SHAPE;
  if (!kv4_type(D, dtype)) return ATTN_ERR_UNSUPPORTED;
  if (!tokens_ok(L, D) || misaligned(K) || misaligned(V) || misaligned(cache)) return ATTN_ERR_SHAPE;
  for (int i = 0; i < 3; ++i)
    if (k_strides[i] % 8 || v_strides[i] % 8) return ATTN_ERR_SHAPE;
  if (!apart(span(cache, cache_bytes(pages, Hkv, page, D)),
             {span(K, k_strides, B, Hkv, L, D), span(V, v_strides, B, Hkv, L, D), span(slots, 8LL * B * L)}))
    return ATTN_ERR_SHAPE;
  attn::Kv4AppendParams p{};
  p.x[0] = K; p.x[1] = V;
  p.sb[0] = k_strides[0]; p.sh[0] = k_strides[1]; p.sl[0] = k_strides[2];
  p.sb[1] = v_strides[0]; p.sh[1] = v_strides[1]; p.sl[1] = v_strides[2];
  p.cache = static_cast<unsigned char*>(cache);
  p.slots = reinterpret_cast<const int64_t*>(slots);
  p.B = B; p.H = Hkv; p.L = L; p.D = D; p.pages = pages; p.shift = shift;
  p.bf16 = dtype == ATTN_BF16;
  return done(attn::launch_kv4_append(p, stream));
}

int kv4_load(const void* cache, const int* table, const int* starts, const int* lens, void* K, void* V, int B, int Hkv,
             int L, int D, int pages, int page, int max_pages, attn_dtype dtype, hipStream_t stream) {
  if (!cache || !table || !lens || !K || !V) return ATTN_ERR_NULL;
  const int shift = page_shift(page);
  if (!cache_ok(B, Hkv, L, pages) || shift < 0 || max_pages < 1 || ((int64_t)max_pages << shift) > kMaxTokens)
    return ATTN_ERR_SHAPE;
  if (!kv4_type(D, dtype)) return ATTN_ERR_UNSUPPORTED;
  if (!tokens_ok(L, D) || misaligned(K) || misaligned(V) || misaligned(cache)) return ATTN_ERR_SHAPE;
  const int64_t rows = 2LL * B * Hkv * L * D;
  const Span in[] = {span(cache, cache_bytes(pages, Hkv, page, D)), span(table, 4LL * B * max_pages),
                     span(starts, 4LL * B), span(lens, 4LL * B)};
  if (!apart(span(K, rows), {span(V, rows), in[0], in[1], in[2], in[3]}) ||
      !apart(span(V, rows), {in[0], in[1], in[2], in[3]}))
    return ATTN_ERR_SHAPE;
  attn::Kv4LoadParams p{};
  p.cache = static_cast<const unsigned char*>(cache);
  p.table = table; p.starts = starts; p.lens = lens;
  p.y[0] = K; p.y[1] = V;
  p.B = B; p.H = Hkv; p.L = L; p.D = D; p.pages = pages; p.shift = shift; p.M = max_pages;
  p.bf16 = dtype == ATTN_BF16;
  return done(attn::launch_kv4_load(p, stream));
}

size_t attn_decode_kv4_workspace_bytes(int B, int Hq, int Hkv, int D) {
  if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || (D != 64 && D != 128)) return 0;
  const size_t parts = 2 * (size_t)attn::kv4_shares(D, Hq / Hkv, attn::compute_units());
  const size_t cols = attn::kv4_columns(Hq / Hkv), tiles = (Hq / Hkv + cols - 1) / cols;
  const size_t bytes = parts * cols * (size_t)(D + 2) * sizeof(float) + (size_t)B * Hkv * tiles * sizeof(int2);
  return (bytes + 255) & ~(size_t)255;
}

int attn_decode_kv4(const void* Q, const void* cache, const int* table, const int* lens, void* O, int B, int Hq,
                    int Hkv, int D, int pages, int page, int max_pages, float scale, const float* alibi_slopes,
                    float softcap, int window, void* workspace, size_t workspace_bytes, attn_dtype dtype,
                    hipStream_t stream) {
  if (!Q || !cache || !table || !lens || !O || !workspace) return ATTN_ERR_NULL;
  const int shift = page_shift(page);
  if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || pages < 1 || max_pages < 1 || shift < 0 || window < 0 ||
      !std::isfinite(scale) || !std::isfinite(softcap) || softcap < 0.f)
    return ATTN_ERR_SHAPE;
  if (!kv4_type(D, dtype)) return ATTN_ERR_UNSUPPORTED;
  if (misaligned(Q) || misaligned(cache) || misaligned(O)) return ATTN_ERR_SHAPE;
  const int group = Hq / Hkv, cols = attn::kv4_columns(group), tiles = (group + cols - 1) / cols;
  const int64_t rows = (int64_t)B * Hkv * tiles;
  // The list of all tiles is counted in 32 bits, and so is a page of all heads.
  if ((int64_t)B * Hq > kMaxGroups || ((int64_t)max_pages << shift) > kMaxTokens ||
      (int64_t)(kv4_page_bytes(page, D) * Hkv) > kMaxInt || rows > kMaxInt / ((((int64_t)max_pages << shift) + 31) / 32 + attn::kKv4RowStart))
    return ATTN_ERR_SHAPE;
  const size_t need = attn_decode_kv4_workspace_bytes(B, Hq, Hkv, D);
  if (workspace_bytes < need || misaligned(workspace)) return ATTN_ERR_WORKSPACE;
  const int64_t heads = 2LL * B * Hq * D;
  const Span ws = span(workspace, (int64_t)need);
  const Span in[] = {span(Q, heads), span(cache, cache_bytes(pages, Hkv, page, D)), span(table, 4LL * B * max_pages),
                     span(lens, 4LL * B), span(alibi_slopes, 4LL * Hq)};
  // In place: a query head's output is written when all that read its query are done.
  if ((O != Q && !apart(span(O, heads), {in[0]})) || !apart(span(O, heads), {ws, in[1], in[2], in[3], in[4]}) ||
      !apart(ws, {in[0], in[1], in[2], in[3], in[4]}))
    return ATTN_ERR_SHAPE;
  attn::Kv4DecodeParams p{};
  p.q = Q; p.cache = static_cast<const unsigned char*>(cache); p.table = table; p.lens = lens; p.o = O;
  p.slopes = alibi_slopes;
  p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.D = D; p.group = group;
  p.pages = pages; p.shift = shift; p.M = max_pages;
  p.window = window;
  p.head_tiles = tiles;
  p.shares = attn::kv4_shares(D, group, attn::compute_units());
  const size_t parts = 2 * (size_t)p.shares * cols;
  p.ws_o = static_cast<float*>(workspace);
  p.ws_m = p.ws_o + parts * D;
  p.ws_l = p.ws_m + parts;
  p.ws_rows = reinterpret_cast<int2*>(p.ws_l + parts);
  p.bf16 = dtype == ATTN_BF16;
  p.c = scale * kLog2e;
  // Finite for every cap, and twice as well: an infinity times 0 (a score, or what is left of
  // one at infinity) would be NaN.
  constexpr float kTop = std::numeric_limits<float>::max() / 2;
  p.cap_k2 = softcap > 0.f ? std::min(2.f / softcap, kTop) : 0.f;
  p.cap_cl = softcap > 0.f ? std::min(softcap * kLog2e, kTop) : 0.f;
  p.cap_inv = softcap > attn::kKv4HighCap ? 1.f / p.cap_cl : 0.f;
  return done(attn::launch_decode_kv4(p, stream));
}

}  // extern "C"
