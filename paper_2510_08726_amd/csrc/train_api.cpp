// C ABI of the operators of a training step (include/attn_bwd.h, include/rmsnorm.h):
// argument validation on the host, before anything is enqueued.

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "../../include/attn.h"
#include "../../include/attn_bwd.h"
#include "../../include/rmsnorm.h"
#include "launch.h"
#include "span.h"

namespace {

using attn::apart;
using attn::misaligned;
using attn::Span;
using attn::span;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kMaxInt = std::numeric_limits<int32_t>::max();
constexpr int64_t kMaxElements = int64_t(1) << 40;
constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;   // workgroups of 256 threads in a row of a grid: under 2^32 threads

int done(hipError_t e) { return e == hipSuccess ? ATTN_OK : attn::hip_fail(e); }

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Sizes that both passes take: a head's rows are addressed with 32-bit byte offsets.
bool sizes_ok(int B, int Hq, int Hkv, int Lq, int Lk, int D) {
  if (B < 1 || Hq < 1 || Hkv < 1 || Lq < 1 || Lk < 1 || Hq % Hkv) return false;
  // (To the end of the last tile, and of the group's rows of 256 bytes a tile.)
  if (((int64_t)Lq + 32) * D * 2 > kMaxInt || ((int64_t)Lk + 32) * D * 2 > kMaxInt) return false;
  if (((int64_t)Lq + 32) * 8 * (Hq / Hkv) > kMaxInt) return false;
  return (int64_t)B * Hq <= kMaxInt && (int64_t)B * Hq * Lq <= kMaxElements / D && (int64_t)B * Hkv * Lk <= kMaxElements / D;
}

// What both passes refuse beside their pointers; ATTN_OK for none.
int check(int B, int Hq, int Hkv, int Lq, int Lk, int D, int causal, float scale, const float* alibi_slopes,
          float softcap, int window, attn_dtype dtype) {
  if ((D != 64 && D != 128) || (dtype != ATTN_F16 && dtype != ATTN_BF16)) {
    return B < 1 || Hq < 1 || Hkv < 1 || Lq < 1 || Lk < 1 || Hq % Hkv ? ATTN_ERR_SHAPE : ATTN_ERR_UNSUPPORTED;
  }
  if (!sizes_ok(B, Hq, Hkv, Lq, Lk, D) || !std::isfinite(scale)) return ATTN_ERR_SHAPE;
  if (!std::isfinite(softcap) || softcap < 0.f || window < 0) return ATTN_ERR_SHAPE;
  if (softcap > 0.f && (!causal || alibi_slopes)) return ATTN_ERR_UNSUPPORTED;
  if (window > 0 && !causal) return ATTN_ERR_UNSUPPORTED;
  if (softcap > ATTN_TRAIN_MAX_SOFTCAP) return ATTN_ERR_UNSUPPORTED;
  return ATTN_OK;
}

// Sizes, parts and workspace of a backward pass.
struct BwdPlan {
  attn::BwdParams p;
  int64_t stats, peaks, dkv, dq;     // floats of each part of the workspace
  size_t bytes() const { return (size_t)(stats + peaks + dkv + dq) * sizeof(float); }
  int64_t groups;                    // the most workgroups of a kernel
};

// Tiles of 32 queries (of one head) that see keys [128 i, 128 (i + 1)), and of 32 keys that row block i sees, as
// attn_bwd.hip counts them.
int64_t query_tiles(const attn::BwdParams& p, int i) {
  const int off = p.Lk - p.rows, j0 = i * attn::bwd_block_keys();
  int64_t lo = 0, hi = p.rows;
  if (p.causal) {
    lo = std::max(0, j0 - off);
    if (p.window > 0) hi = std::min<int64_t>(hi, (int64_t)std::min(j0 + attn::bwd_block_keys(), p.Lk) - off + p.window - 1);
  }
  return hi > lo ? (hi + 31) / 32 - lo / 32 : 0;
}
int64_t key_tiles(const attn::BwdParams& p, int i) {
  const int bm = attn::bwd_block_keys() / p.hg, off = p.Lk - p.rows;
  const int rb = (p.rows + bm - 1) / bm - 1 - i;             // (from the last)
  int64_t lo = 0, hi = p.Lk;
  if (p.causal) {
    hi = std::min(p.Lk, std::min((rb + 1) * bm, p.rows) + off);
    if (p.window > 0) lo = std::max(0, rb * bm + off + 1 - p.window);
  }
  return (hi + 31) / 32 - lo / 32;
}

// Parts of about `share` tiles.
template <typename F>
void divide(attn::BwdSplit& s, int blocks, double share, F&& tiles) {
  s.list = blocks;
  if (blocks > attn::kBwdSplitBlocks) return;
  int list = 0;
  for (int i = 0; i < blocks; ++i) {
    const double w = (double)tiles(i);
    const int n = w > 1.25 * share ? (int)std::min(std::ceil(w / share), 255.0) : 1;
    s.parts[i] = (unsigned char)n;
    list += n;
    if (n > 1) {
      ++s.multi;
      s.pieces += n;
    }
  }
  s.list = list;
}

BwdPlan plan(int B, int Hq, int Hkv, int Lq, int Lk, int D, bool causal, int window) {
  BwdPlan r{};
  attn::BwdParams& p = r.p;
  p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.Lq = Lq; p.Lk = Lk; p.D = D;
  p.group = Hq / Hkv;
  p.causal = causal;
  p.window = std::min(window, Lk);      // (that many mask nothing)
  p.row0 = causal ? std::max(0, Lq - Lk) : 0;
  p.rows = Lq - p.row0;
  p.row_tiles = (int)ceil_div(p.rows, 32);
  p.row_blocks = (int)ceil_div(p.rows, attn::bwd_rows_per_block());
  p.key_blocks = (int)ceil_div(Lk, attn::bwd_rows_per_block());
  p.hg = 1;
  while (p.hg < 4 && p.group % (2 * p.hg) == 0) p.hg *= 2;
  const int64_t units = (int64_t)B * Hkv, heads = (int64_t)B * Hq;
  p.shares = units % 8 == 0;
  const int bm = attn::bwd_block_keys() / p.hg, nkb = (int)ceil_div(Lk, attn::bwd_block_keys()), nqb = (int)ceil_div(p.rows, bm);
  // The whole call's tiles (either side's are 4 products of 32 x 32 x D a wave), for each workgroup that runs at a time.
  double all = 0.0;
  for (int i = 0; i < nkb; ++i) all += (double)p.group * query_tiles(p, i);
  for (int i = 0; i < nqb; ++i) all += (double)(p.group / p.hg) * key_tiles(p, i);
  // A longer block would be the last to end, and is divided.  Three quarters of an even share: 2 x 32 / 8 heads of 2048 rows
  // (causal) take 283 us, 290 with half of it, 280 with all; 40 / 2 heads 181, 194 and 197; 128 rows of 32 / 8 heads on
  // 8192 keys 92, 100 and 101.  At least 8 tiles: 8 heads of 1024 rows 39 us, with 4 and 16 a tenth to a fifth more.
  const double share = std::max(0.75 * all * units / (2.0 * attn::compute_units()), 8.0);
  divide(p.dkv, nkb, share, [&](int i) { return p.group * query_tiles(p, i); });
  divide(p.dq_, nqb, share, [&](int i) { return key_tiles(p, i); });
  const auto floats = [](int64_t n) { return (n + 63) / 64 * 64; };
  r.stats = floats(heads * p.row_tiles * 64);
  r.peaks = floats(heads * p.row_blocks + units * p.key_blocks);
  const int64_t block = (int64_t)attn::bwd_block_keys() * D;
  r.dkv = 2 * units * p.dkv.pieces * block;
  r.dq = heads / p.hg * p.dq_.pieces * block;
  r.groups = std::max({heads * (p.row_blocks + ceil_div(p.row0, attn::bwd_rows_per_block())) + units * p.key_blocks,
                       units * p.dkv.list + heads / p.hg * p.dq_.list + 16,
                       (2 * units * p.dkv.multi + heads / p.hg * p.dq_.multi) * (block / 1024)});
  return r;
}

int element_size(norm_dtype t) { return t == NORM_F32 ? 4 : 2; }

// Rows of a norm, their types; ATTN_OK for none refused.
int check_norm(int N, int M, float offset, norm_dtype dtype, norm_dtype stream_dtype, bool alone) {
  if (N < 1 || M < 1 || M > RMSNORM_MAX_M || !std::isfinite(offset)) return ATTN_ERR_SHAPE;
  if ((int64_t)N * M >= kMaxElements) return ATTN_ERR_SHAPE;
  if (dtype < NORM_F16 || dtype > NORM_F32 || (stream_dtype != dtype && (alone || stream_dtype != NORM_F32)))
    return ATTN_ERR_UNSUPPORTED;
  return ATTN_OK;
}

// Scales of a row of M with one for each `group` elements, 0 for a group that is none.
int groups_of(int M, int group) {
  if (group == 0) return 1;
  return group == 32 || group == 64 || group == 128 || group == 256 ? (int)ceil_div(M, group) : 0;
}

// Whether `out` is apart from what else is given, or is `same` itself.
bool apart_or(Span out, Span same, std::initializer_list<Span> others) {
  return ((out.begin == same.begin && out.end == same.end) || apart(out, {same})) && apart(out, others);
}

int norm_add(const void* X, const void* residual, const void* weight, void* Y, float* scales, void* H, float* rstd, int N,
             int M, int group, int code, double eps, float offset, norm_dtype dtype, norm_dtype stream_dtype,
             hipStream_t stream) {
  if (!X || !Y || (residual && !H)) return ATTN_ERR_NULL;
  if (int rc = check_norm(N, M, offset, dtype, stream_dtype, !residual); rc != ATTN_OK) return rc;
  if (!std::isfinite(eps) || eps < 0.0) return ATTN_ERR_SHAPE;
  const int groups = scales ? groups_of(M, group) : 1;
  if (!groups) return ATTN_ERR_SHAPE;
  const int64_t n = (int64_t)N * M, e = element_size(dtype), r = element_size(stream_dtype);
  const Span x = span(X, n * e), res = span(residual, n * r), w = span(weight, M * e), y = span(Y, scales ? n : n * e),
             sc = span(scales, 4LL * N * groups), h = span(residual ? H : nullptr, n * r), rs = span(rstd, 4LL * N);
  // In place: a lane reads what it writes before it writes it.
  if (!(scales ? apart(y, {x, res, w, sc, h, rs}) : apart_or(y, x, {res, w, h, rs}))) return ATTN_ERR_SHAPE;
  if (!apart_or(h, res, {x, w, sc, rs}) || !apart(sc, {x, res, w, rs}) || !apart(rs, {x, res, w})) return ATTN_ERR_SHAPE;
  attn::RmsnormParams p{};
  p.x = X; p.residual = residual; p.weight = weight; p.y = Y; p.scales = scales; p.h = H; p.rstd = rstd;
  p.eps = eps;
  p.N = N; p.M = M; p.group = group; p.groups = groups;
  p.offset = offset;
  p.dtype = dtype;
  p.wide = stream_dtype == NORM_F32;
  p.int8 = code == QUANT8_INT8;
  return done(attn::launch_rmsnorm_add(p, stream));
}

}  // namespace

extern "C" {

int attn_fwd_lse(const void* Q, const void* K, const void* V, void* O, float* lse, int B, int Hq, int Hkv, int Lq,
                 int Lk, int D, int causal, float scale, const float* alibi_slopes, float softcap, int window,
                 attn_dtype dtype, hipStream_t stream) {
  if (!Q || !K || !V || !O || !lse) return ATTN_ERR_NULL;
  if (int rc = check(B, Hq, Hkv, Lq, Lk, D, causal, scale, alibi_slopes, softcap, window, dtype); rc != ATTN_OK) return rc;
  // (Copies to LDS of 16 bytes a lane; attn_bwd takes no others either.)
  for (const void* x : {Q, K, V, (const void*)O})
    if (misaligned(x)) return ATTN_ERR_SHAPE;
  const int64_t nqb = ceil_div(Lq, attn::prefill_block_rows());
  if (nqb * 4 * B * Hq > kMaxInt) return ATTN_ERR_SHAPE;
  const int64_t q = 2LL * B * Hq * Lq * D, k = 2LL * B * Hkv * Lk * D, l = 4LL * B * Hq * Lq;
  const Span in[] = {span(Q, q), span(K, k), span(V, k), span(alibi_slopes, 4LL * Hq)};
  if (!apart(span(O, q), {in[0], in[1], in[2], in[3], span(lse, l)}) || !apart(span(lse, l), {in[0], in[1], in[2], in[3]}))
    return ATTN_ERR_SHAPE;
  attn::PrefillLseParams p{};
  p.q = Q; p.k = K; p.v = V; p.o = O; p.lse = lse;
  p.slopes = alibi_slopes;
  p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.Lq = Lq; p.Lk = Lk; p.D = D;
  p.group = Hq / Hkv;
  p.causal = causal != 0;
  p.bf16 = dtype == ATTN_BF16;
  p.cap_k2 = softcap > 0.f ? 2.f / softcap : 0.f;
  p.cap_cl = softcap > 0.f ? softcap * kLog2e : 0.f;
  p.window = std::min(window, Lk);
  if (alibi_slopes || softcap > 0.f) {
    p.c = scale * kLog2e;
  } else {     // above zero, so that masked (-inf) scores stay so
    p.c = std::fmax(std::fabs(scale) * kLog2e, 1e-30f);
    p.qsign = std::signbit(scale) ? 0x80008000u : 0u;
  }
  return done(attn::launch_prefill_lse(p, stream));
}

size_t attn_bwd_workspace_bytes(int B, int Hq, int Hkv, int Lq, int Lk, int D, int causal, int window) {
  if ((D != 64 && D != 128) || !sizes_ok(B, Hq, Hkv, Lq, Lk, D) || window < 0) return 0;
  return plan(B, Hq, Hkv, Lq, Lk, D, causal != 0, window).bytes();
}

int attn_bwd(const void* dO, const long long* do_strides, const void* Q, const void* K, const void* V, const void* O,
             const float* lse, void* dQ, void* dK, void* dV, int B, int Hq, int Hkv, int Lq, int Lk, int D, int causal,
             float scale, const float* alibi_slopes, float softcap, int window, void* workspace,
             size_t workspace_bytes, attn_dtype dtype, hipStream_t stream) {
  if (!dO || !do_strides || !Q || !K || !V || !O || !lse || !dQ || !dK || !dV || !workspace) return ATTN_ERR_NULL;
  if (int rc = check(B, Hq, Hkv, Lq, Lk, D, causal, scale, alibi_slopes, softcap, window, dtype); rc != ATTN_OK) return rc;
  for (const void* x : {dO, Q, K, V, O, (const void*)dQ, (const void*)dK, (const void*)dV})
    if (misaligned(x)) return ATTN_ERR_SHAPE;
  const int n[3] = {B, Hq, Lq};
  for (int i = 0; i < 3; ++i)
    if (do_strides[i] < 0 || do_strides[i] % 8 || do_strides[i] > kMaxElements / n[i]) return ATTN_ERR_SHAPE;
  const long long row = Lq > 1 ? do_strides[2] : D;
  if (2 * row * ((int64_t)Lq + 32) > kMaxInt) return ATTN_ERR_SHAPE;
  BwdPlan w = plan(B, Hq, Hkv, Lq, Lk, D, causal != 0, window);
  if (w.groups > kMaxGroups) return ATTN_ERR_SHAPE;
  if (workspace_bytes < w.bytes() || misaligned(workspace)) return ATTN_ERR_WORKSPACE;
  const int64_t q = 2LL * B * Hq * Lq * D, k = 2LL * B * Hkv * Lk * D;
  const Span out[] = {span(dQ, q), span(dK, k), span(dV, k), span(workspace, (int64_t)w.bytes())};
  const Span in[] = {span(dO, do_strides, B, Hq, Lq, D), span(Q, q), span(K, k), span(V, k), span(O, q),
                     span(lse, 4LL * B * Hq * Lq), span(alibi_slopes, 4LL * Hq)};
  for (int i = 0; i < 4; ++i) {
    if (!apart(out[i], {in[0], in[1], in[2], in[3], in[4], in[5], in[6]})) return ATTN_ERR_SHAPE;
    for (int j = 0; j < i; ++j)
      if (!apart(out[i], {out[j]})) return ATTN_ERR_SHAPE;
  }
  attn::BwdParams& p = w.p;
  p.q = Q; p.k = K; p.v = V; p.o = O; p.d_o = dO; p.lse = lse;
  p.slopes = alibi_slopes;
  p.dq = dQ; p.dk = dK; p.dv = dV;
  p.stats = static_cast<float*>(workspace);
  p.peaks = p.stats + w.stats;
  p.ws_dkv = p.peaks + w.peaks;
  p.ws_dq = p.ws_dkv + w.dkv;
  p.do_sb = do_strides[0]; p.do_sh = do_strides[1]; p.do_sl = row;
  p.bf16 = dtype == ATTN_BF16;
  p.sign = std::signbit(scale) ? 0x80008000u : 0u;
  // Above zero: a row's log-sum-exp starts its scores, divided by it.
  p.c = std::fmax(std::fabs(scale) * kLog2e, 1e-30f);
  p.scale = scale;
  p.cap_k2 = softcap > 0.f ? 2.f / softcap * p.c : 0.f;
  p.cap_cl = softcap > 0.f ? softcap * kLog2e : 0.f;
  return done(attn::launch_attn_bwd(p, stream));
}

int rmsnorm_add(const void* X, const void* residual, const void* weight, void* Y, void* H, float* rstd, int N, int M,
                double eps, float weight_offset, norm_dtype dtype, norm_dtype stream_dtype, hipStream_t stream) {
  return norm_add(X, residual, weight, Y, nullptr, H, rstd, N, M, 0, 0, eps, weight_offset, dtype, stream_dtype, stream);
}

int rmsnorm_add_quant(const void* X, const void* residual, const void* weight, void* codes, float* scales, void* H,
                      float* rstd, int N, int M, int group, quant8_code code, double eps, float weight_offset,
                      norm_dtype dtype, norm_dtype stream_dtype, hipStream_t stream) {
  if (!scales) return ATTN_ERR_NULL;
  if (code != QUANT8_E4M3 && code != QUANT8_INT8) return ATTN_ERR_UNSUPPORTED;
  return norm_add(X, residual, weight, codes, scales, H, rstd, N, M, group, code, eps, weight_offset, dtype, stream_dtype,
                  stream);
}

int quant8_load(const void* codes, const float* scales, void* Y, int N, int M, int group, quant8_code code,
                norm_dtype dtype, hipStream_t stream) {
  if (!codes || !scales || !Y) return ATTN_ERR_NULL;
  if (int rc = check_norm(N, M, 0.f, dtype, dtype, true); rc != ATTN_OK) return rc;
  if (code != QUANT8_E4M3 && code != QUANT8_INT8) return ATTN_ERR_UNSUPPORTED;
  const int groups = groups_of(M, group);
  if (!groups) return ATTN_ERR_SHAPE;
  const int64_t n = (int64_t)N * M;
  if (!apart(span(Y, n * element_size(dtype)), {span(codes, n), span(scales, 4LL * N * groups)})) return ATTN_ERR_SHAPE;
  attn::Quant8LoadParams p{};
  p.codes = static_cast<const unsigned char*>(codes);
  p.scales = scales; p.y = Y;
  p.N = N; p.M = M; p.group = group; p.groups = groups;
  p.dtype = dtype;
  p.int8 = code == QUANT8_INT8;
  return done(attn::launch_quant8_load(p, stream));
}

size_t rmsnorm_add_bwd_workspace_bytes(int N, int M) {
  if (N < 1 || M < 1 || M > RMSNORM_MAX_M) return 0;
  return ((size_t)attn::rmsnorm_bwd_partials(N, M) * M * sizeof(float) + 255) & ~(size_t)255;
}

int rmsnorm_add_bwd(const void* dY, const void* H, const float* rstd, const void* weight, const void* dH, void* dX,
                    void* dresidual, float* dweight, int N, int M, float weight_offset, void* workspace,
                    size_t workspace_bytes, norm_dtype dtype, norm_dtype stream_dtype, hipStream_t stream) {
  if (!dY || !H || !rstd || !dX) return ATTN_ERR_NULL;
  if (int rc = check_norm(N, M, weight_offset, dtype, stream_dtype, false); rc != ATTN_OK) return rc;
  if (dresidual && dtype == stream_dtype) return ATTN_ERR_SHAPE;       // dX is that
  const size_t need = dweight ? rmsnorm_add_bwd_workspace_bytes(N, M) : 0;
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace))) return ATTN_ERR_WORKSPACE;
  const int64_t n = (int64_t)N * M, e = element_size(dtype), r = element_size(stream_dtype);
  const Span dy = span(dY, n * e), h = span(H, n * r), rs = span(rstd, 4LL * N), w = span(weight, M * e),
             dh = span(dH, n * r), dx = span(dX, n * e), dres = span(dresidual, n * r), dw = span(dweight, 4LL * M),
             ws = span(need ? workspace : nullptr, (int64_t)need);
  // In place: dX may be dY or a dH of its type, dresidual may be dH.
  const bool on_dh = dtype == stream_dtype && dX == dH;
  if (!(on_dh ? apart(dx, {dy, h, rs, w, dres, dw, ws}) : apart_or(dx, dy, {h, rs, w, dh, dres, dw, ws}))) return ATTN_ERR_SHAPE;
  if (!apart_or(dres, dh, {dy, h, rs, w, dw, ws}) || !apart(dw, {dy, h, rs, w, dh, ws}) || !apart(ws, {dy, h, rs, w, dh}))
    return ATTN_ERR_SHAPE;
  attn::RmsnormBwdParams p{};
  p.dy = dY; p.h = H; p.rstd = rstd; p.weight = weight; p.dh = dH; p.dx = dX; p.dresidual = dresidual;
  p.ws = need ? static_cast<float*>(workspace) : nullptr;
  p.N = N; p.M = M;
  p.offset = weight_offset;
  p.dtype = dtype;
  p.wide = stream_dtype == NORM_F32;
  return done(attn::launch_rmsnorm_add_bwd(p, dweight, stream));
}

}  // extern "C"
