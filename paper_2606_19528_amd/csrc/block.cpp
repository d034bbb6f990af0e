// block.cpp -- entry points of what stands between the linears of a decoder block
// and of what is kept of it: activations in 8 bits, and the norms with gate and
// residual sum.  Every argument is checked before any work is enqueued; nothing
// here allocates device memory, throws or aborts.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "api_util.hpp"

using namespace lora;

namespace {

static_assert(BN_GATE_CHANNEL == (int)BLOCK_GATE_CHANNEL && BN_GATE_TOKEN == (int)BLOCK_GATE_TOKEN &&
                  BN_GATE_FULL == (int)BLOCK_GATE_FULL && BN_GATE_NONE == (int)BLOCK_GATE_NONE,
              "the header's gate modes are the kernels'");

constexpr int64_t kMaxT = int64_t(1) << 22;       // rows of a norm
constexpr int64_t kMaxGroups = int64_t(1) << 29;  // groups of 128 values
constexpr int64_t kMaxActT = int64_t(1) << 40;    // rows of an activation (keeps their product with D in 64 bits)

bool finite32(double x) { return std::isfinite((float)x); }  // (bf16 rows and gradients take it in 32 bits)
bool bad_dtype(lora_dtype_t dt) { return dt != LORA_BF16 && dt != LORA_F32; }
Dtype dtype(lora_dtype_t dt) { return dt == LORA_BF16 ? DT_BF16 : DT_F32; }

lora_status_t check_act8(const void *x, const void *codes, const void *scale, int64_t T, int64_t D, lora_dtype_t dt) {
  if (bad_dtype(dt)) return fail(LORA_EINVAL, "unknown dtype");
  if (T < 1 || D < 1) return fail(LORA_EINVAL, "T and D must be >= 1");
  if (D % 8) return fail(LORA_EUNSUPPORTED, "D must be a multiple of 8");
  if (D > kMaxDim) return fail(LORA_EUNSUPPORTED, "D must be at most 2^20");
  if (T > kMaxActT || T * act8_groups(D) > kMaxGroups) return fail(LORA_EUNSUPPORTED, "at most 2^29 groups of 128 values");
  if (!x || !codes || !scale) return fail(LORA_EINVAL, "x, codes and scale are required");
  if (!aligned16(x) || !aligned16(codes) || !aligned16(scale)) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
  return LORA_OK;
}

// The sizes and parts that both directions take from the struct.
lora_status_t check_block(const block_norm_t *b) {
  if (!b) return fail(LORA_EINVAL, "the block's description is NULL");
  if (bad_dtype(b->dt) || bad_dtype(b->res_dt)) return fail(LORA_EINVAL, "unknown dtype");
  if (b->dt == LORA_F32 && b->res_dt != LORA_F32) return fail(LORA_EUNSUPPORTED, "an fp32 block has an fp32 stream");
  if (b->T < 1 || b->D < 1) return fail(LORA_EINVAL, "T and D must be >= 1");
  if (b->D % 8) return fail(LORA_EUNSUPPORTED, "D must be a multiple of 8");
  if (b->D > BN_MAX_D || b->T > kMaxT) return fail(LORA_EUNSUPPORTED, "D at most 16384, T at most 2^22");
  if (b->gate_mode < BLOCK_GATE_NONE || b->gate_mode > BLOCK_GATE_FULL) return fail(LORA_EINVAL, "unknown gate mode");
  if ((b->gate_mode != BLOCK_GATE_NONE) != (b->gate != nullptr)) return fail(LORA_EINVAL, "a gate and its mode go together");
  if (b->post_norm != 0 && b->post_norm != 1) return fail(LORA_EINVAL, "post_norm must be 0 or 1");
  if (b->w_post && !b->post_norm) return fail(LORA_EINVAL, "w_post is the gain of a post norm");
  if (!finite32(b->res_scale) || !finite32(b->gain_offset)) return fail(LORA_EINVAL, "res_scale and gain_offset must be finite");
  return LORA_OK;
}

int64_t gate_elems(const block_norm_t *b) {
  switch (b->gate_mode) {
    case BLOCK_GATE_CHANNEL: return b->D;
    case BLOCK_GATE_TOKEN: return b->T;
    case BLOCK_GATE_FULL: return b->T * b->D;
  }
  return 0;
}

// Ranges of a call, with their alignment checked as they are listed.
struct Ranges {
  Range in[16], out[16];
  size_t ni = 0, no = 0;
  bool aligned = true;
  void add_in(const void *p, int64_t bytes) {
    aligned = aligned && aligned16(p);
    in[ni++] = rng(p, bytes);
  }
  void add_out(const void *p, int64_t bytes) {
    aligned = aligned && aligned16(p);
    out[no++] = rng(p, bytes);
  }
  lora_status_t check() const {
    if (!aligned) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
    if (any_overlap(out, no, in, ni)) return fail(LORA_EINVAL, "an output overlaps an input or another output");
    return LORA_OK;
  }
};

bool whole(const lora_act8_t *k) { return !k || (k->codes && k->scale); }  // both parts, or not asked for
Act8Out act8_out(const lora_act8_t *k) { return k ? Act8Out{k->codes, k->scale} : Act8Out{}; }
Act8In act8_in(const lora_act8_t *k) { return k ? Act8In{k->codes, k->scale} : Act8In{}; }

size_t block_ws(int64_t T, int64_t D) { return round256((size_t)2 * block_norm_parts(T, D) * D * 4); }

}  // namespace

extern "C" {

lora_status_t act8_quantize(const void *x, int8_t *codes, float *scale, int64_t T, int64_t D, lora_dtype_t dt, void *hip_stream) {
  const lora_status_t s = check_act8(x, codes, scale, T, D, dt);
  if (s != LORA_OK) return s;
  const Range ins[] = {rng(x, T * D * (int64_t)esize(dt))}, outs[] = {rng(codes, T * D), rng(scale, T * act8_groups(D) * 4)};
  if (any_overlap(outs, 2, ins, 1)) return fail(LORA_EINVAL, "an output overlaps an input or another output");
  hipStream_t st = (hipStream_t)hip_stream;
  Timed t(K_ACT8_QUANTIZE, st);
  const hipError_t e = launch_act8_quantize(x, codes, scale, T, D, dtype(dt), st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "act8_quantize launch");
}

lora_status_t act8_dequantize(const int8_t *codes, const float *scale, void *x, int64_t T, int64_t D, lora_dtype_t dt,
                              void *hip_stream) {
  const lora_status_t s = check_act8(x, codes, scale, T, D, dt);
  if (s != LORA_OK) return s;
  const Range outs[] = {rng(x, T * D * (int64_t)esize(dt))}, ins[] = {rng(codes, T * D), rng(scale, T * act8_groups(D) * 4)};
  if (any_overlap(outs, 1, ins, 2)) return fail(LORA_EINVAL, "an output overlaps an input or another output");
  hipStream_t st = (hipStream_t)hip_stream;
  Timed t(K_ACT8_DEQUANTIZE, st);
  const hipError_t e = launch_act8_dequantize(codes, scale, x, T, D, dtype(dt), st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "act8_dequantize launch");
}

lora_status_t block_norm_fwd(const block_norm_t *b, const void *h, const void *y, void *h_out, void *n, float *rstd_post,
                             float *rstd_pre, const lora_act8_t *y8, const lora_act8_t *h8, const lora_act8_t *n8, double eps,
                             void *hip_stream) {
  lora_status_t s = check_block(b);
  if (s != LORA_OK) return s;
  if (!(eps >= 1e-30) || !finite32(eps)) return fail(LORA_EINVAL, "eps must be finite and at least 1e-30");
  if (!h) return fail(LORA_EINVAL, "h is required");
  if (!whole(y8) || !whole(h8) || !whole(n8)) return fail(LORA_EINVAL, "a copy in 8 bits needs codes and scale");
  if (!y && (b->post_norm || b->gate || y8 || rstd_post)) return fail(LORA_EINVAL, "a post norm, a gate and y8 need y");
  if (rstd_post && !b->post_norm) return fail(LORA_EINVAL, "rstd_post belongs to a post norm");
  if (!h_out && !n && !h8 && !n8 && !rstd_pre && !y8 && !rstd_post) return fail(LORA_EINVAL, "no output is given");
  const int64_t n_ = b->T * b->D, e = (int64_t)esize(b->dt), r = (int64_t)esize(b->res_dt), ng = act8_groups(b->D);
  Ranges g;
  if (h_out != h) g.add_in(h, n_ * r);  // (the stream may be updated in place)
  g.add_in(y, y ? n_ * e : 0);
  g.add_in(b->gate, gate_elems(b) * e);
  g.add_in(b->w_post, b->D * e);
  g.add_in(b->w_pre, b->D * e);
  g.add_out(h_out, n_ * r);
  g.add_out(n, n_ * e);
  g.add_out(rstd_post, b->T * 4);
  g.add_out(rstd_pre, b->T * 4);
  for (const lora_act8_t *k : {y8, h8, n8}) {
    if (!k) continue;
    g.add_out(k->codes, n_);
    g.add_out(k->scale, b->T * ng * 4);
  }
  if ((s = g.check()) != LORA_OK) return s;
  BlockNormFwd a{};
  a.y = y; a.h = h; a.gate = b->gate; a.w_post = b->w_post; a.w_pre = b->w_pre;
  a.h_out = h_out; a.n = n; a.rstd_post = rstd_post; a.rstd_pre = rstd_pre;
  a.y8 = act8_out(y8); a.h8 = act8_out(h8); a.n8 = act8_out(n8);
  a.T = b->T; a.D = (int)b->D; a.ng = (int)ng; a.gate_mode = b->gate_mode; a.post = b->post_norm;
  a.eps = eps; a.off = b->gain_offset; a.res_scale = b->res_scale;
  hipStream_t st = (hipStream_t)hip_stream;
  Timed t(K_BLOCK_NORM_FWD, st);
  const hipError_t err = launch_block_norm_fwd(a, dtype(b->dt), dtype(b->res_dt), st);
  t.done();
  return err == hipSuccess ? LORA_OK : hip_fail(err, "block_norm_fwd launch");
}

size_t block_norm_workspace_bytes(int64_t T, int64_t D) {
  if (T < 1 || D < 1 || D % 8 || D > BN_MAX_D || T > kMaxT) {
    fail(LORA_EUNSUPPORTED, "D a multiple of 8 up to 16384, T from 1 to 2^22");
    return (size_t)-1;
  }
  return block_ws(T, D);
}

lora_status_t block_norm_bwd(const block_norm_t *b, const void *dn, const void *dh_out, const void *h, const lora_act8_t *h8,
                             const void *y, const lora_act8_t *y8, const float *rstd_post, const float *rstd_pre, void *dh,
                             void *dy, float *dw_pre, float *dw_post, void *dgate, void *ws, size_t ws_bytes, void *hip_stream) {
  lora_status_t s = check_block(b);
  if (s != LORA_OK) return s;
  if (!dh) return fail(LORA_EINVAL, "dh is required");
  if (!dn && !dh_out) return fail(LORA_EINVAL, "dn or dh_out is required");
  if (!whole(y8) || !whole(h8)) return fail(LORA_EINVAL, "a copy in 8 bits needs codes and scale");
  if ((h && h8) || (y && y8)) return fail(LORA_EINVAL, "h and y are given whole or in 8 bits, not both");
  if (dn && ((!h && !h8) || !rstd_pre)) return fail(LORA_EINVAL, "dn needs h (or h8) and rstd_pre");
  if (dw_pre && !dn) return fail(LORA_EINVAL, "dw_pre needs dn");
  if (dgate && !b->gate) return fail(LORA_EINVAL, "dgate needs a gate");
  if (dw_post && !b->post_norm) return fail(LORA_EINVAL, "dw_post needs a post norm");
  const bool block = dy || dw_post || dgate;
  if (block && b->post_norm && !rstd_post) return fail(LORA_EINVAL, "a post norm needs rstd_post");
  if (((block && b->post_norm) || dgate) && !y && !y8) return fail(LORA_EINVAL, "a post norm and dgate need y (or y8)");
  const bool sums = dw_pre || dw_post || (dgate && b->gate_mode == BLOCK_GATE_CHANNEL);
  const size_t need = sums ? block_ws(b->T, b->D) : 0;
  if ((s = check_ws(ws, ws_bytes, need)) != LORA_OK) return s;
  const int64_t n_ = b->T * b->D, e = (int64_t)esize(b->dt), r = (int64_t)esize(b->res_dt), ng = act8_groups(b->D);
  Ranges g;
  g.add_in(dn, n_ * e);
  if (dh_out != dh) g.add_in(dh_out, n_ * r);  // (the stream's gradient may be updated in place)
  g.add_in(h, n_ * r);
  g.add_in(y, n_ * e);
  for (const lora_act8_t *k : {h8, y8}) {
    if (!k) continue;
    g.add_in(k->codes, n_);
    g.add_in(k->scale, b->T * ng * 4);
  }
  g.add_in(rstd_post, b->T * 4);
  g.add_in(rstd_pre, b->T * 4);
  g.add_in(b->gate, gate_elems(b) * e);
  g.add_in(b->w_post, b->D * e);
  g.add_in(b->w_pre, b->D * e);
  g.add_out(dh, n_ * r);
  g.add_out(dy, n_ * e);
  g.add_out(dw_pre, b->D * 4);
  g.add_out(dw_post, b->D * 4);
  g.add_out(dgate, gate_elems(b) * (b->gate_mode == BLOCK_GATE_FULL ? e : 4));
  g.add_out(need ? ws : nullptr, (int64_t)need);
  if ((s = g.check()) != LORA_OK) return s;
  BlockNormBwd a{};
  a.dn = dn; a.dh_out = dh_out; a.h = h; a.y = y; a.gate = b->gate; a.w_post = b->w_post; a.w_pre = b->w_pre;
  a.h8 = act8_in(h8); a.y8 = act8_in(y8);
  a.rstd_post = rstd_post; a.rstd_pre = rstd_pre;
  a.dh = dh; a.dy = dy; a.dgate = dgate;
  a.want_w1 = dw_pre; a.want_w2 = dw_post;
  a.want_gate = b->gate_mode == BLOCK_GATE_CHANNEL ? (float *)dgate : nullptr;
  a.part = (float *)ws;
  a.T = b->T; a.D = (int)b->D; a.ng = (int)ng; a.gate_mode = b->gate_mode; a.post = block ? b->post_norm : 0;
  a.off = (float)b->gain_offset; a.res_scale = (float)b->res_scale;
  hipStream_t st = (hipStream_t)hip_stream;
  Timed t(K_BLOCK_NORM_BWD, st);
  const hipError_t err = launch_block_norm_bwd(a, dtype(b->dt), dtype(b->res_dt), st);
  t.done();
  return err == hipSuccess ? LORA_OK : hip_fail(err, "block_norm_bwd launch");
}

}  // extern "C"
