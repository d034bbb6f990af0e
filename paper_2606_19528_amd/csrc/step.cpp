// step.cpp -- entry points of what surrounds the linears in a fine-tuning
// step: embedding lookup and gradient, losses over the targets'
// log-probabilities, and the clipping of a list of gradients by their norm.
// Every argument is checked before any work is enqueued; nothing here
// allocates device memory, throws or aborts.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "api_util.hpp"

using namespace lora;

namespace {

constexpr int64_t kMaxMatrix = int64_t(1) << 40;  // elements; offsets are 64-bit
constexpr int64_t kMaxRows = int64_t(1) << 30;    // a vocabulary, a row
// A launch has fewer than 2^32 threads: positions of an embedding (64 threads each for 4 KB of
// row, and in the gradient 4 for each 512 columns), of a loss (256 each), pairs (512 each).
constexpr int64_t kMaxEmbedT = int64_t(1) << 25, kMaxEmbedElems = int64_t(1) << 35;
constexpr int64_t kMaxLossT = int64_t(1) << 23, kMaxPairs = int64_t(1) << 22;

bool bad_dtype(lora_dtype_t dt) { return dt != LORA_BF16 && dt != LORA_F32; }
Dtype dtype(lora_dtype_t dt) { return dt == LORA_BF16 ? DT_BF16 : DT_F32; }

template <size_t N>
bool misaligned(const void *const (&ptrs)[N]) {
  for (const void *p : ptrs)
    if (p && !aligned16(p)) return true;
  return false;
}
template <size_t NO, size_t NI>
bool clash(const Range (&outs)[NO], const Range (&ins)[NI]) {
  return any_overlap(outs, NO, ins, NI);
}

// ----- embedding ---------------------------------------------------------------
lora_status_t check_embed(int64_t T, int64_t V, int64_t D, lora_dtype_t dt) {
  if (bad_dtype(dt)) return fail(LORA_EINVAL, "unknown dtype");
  if (T < 1 || V < 1 || D < 1) return fail(LORA_EINVAL, "T, V and D must be >= 1");
  if (D % 8) return fail(LORA_EUNSUPPORTED, "D must be a multiple of 8");
  if (D > kMaxDim) return fail(LORA_EUNSUPPORTED, "D must be at most 2^20");
  if (T > kMaxEmbedT || T > kMaxEmbedElems / D) return fail(LORA_EUNSUPPORTED, "T at most 2^25, T times D at most 2^35");
  if (V > kMaxRows || V > kMaxMatrix / D) return fail(LORA_EUNSUPPORTED, "V at most 2^30, the table at most 2^40 elements");
  return LORA_OK;
}
lora_status_t embed_grad(const int32_t *ids, const void *dout, float *out, int32_t *tokens, bool compact, int64_t T,
                         int64_t V, int64_t D, float scale, int accumulate, lora_dtype_t dt, void *ws, size_t ws_bytes,
                         void *hip_stream) {
  lora_status_t s = check_embed(T, V, D, dt);
  if (s != LORA_OK) return s;
  if (!ids || !dout || !out || (compact && !tokens)) return fail(LORA_EINVAL, "ids, dout and the outputs are required");
  if (!std::isfinite(scale)) return fail(LORA_EINVAL, "scale must be finite");
  const void *ptrs[] = {ids, dout, out, tokens};
  if (misaligned(ptrs)) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
  const EmbedPlan p = embed_plan(T, V, D);
  if ((s = check_ws(ws, ws_bytes, p.total)) != LORA_OK) return s;
  const int64_t rows = compact ? std::min(T, V) : V;
  const Range ins[] = {rng(ids, T * 4), rng(dout, T * D * (int64_t)esize(dt))};
  const Range outs[] = {rng(out, rows * D * 4), rng(tokens, rows * 4), rng(ws, (int64_t)p.total)};
  if (clash(outs, ins)) return fail(LORA_EINVAL, "an output overlaps an input or another output");
  hipStream_t st = (hipStream_t)hip_stream;
  if (p.scan) {
    Timed t(K_EMBED_GRAD, st);
    const hipError_t e = launch_embed_scan(ids, dout, out, tokens, (int)T, (int)V, (int)D, scale, accumulate != 0, dtype(dt), p,
                                           (char *)ws, st);
    t.done();
    return e == hipSuccess ? LORA_OK : hip_fail(e, "embed_grad launch");
  }
  {
    Timed t(K_EMBED_SORT, st);
    const hipError_t e = launch_embed_sort(ids, (int)T, (int)V, p, (char *)ws, tokens, st);
    t.done();
    if (e != hipSuccess) return hip_fail(e, "embed_sort launch");
  }
  Timed t(K_EMBED_GRAD, st);
  const hipError_t e = launch_embed_grad(dout, out, tokens, (int)T, (int)V, (int)D, scale, accumulate != 0, dtype(dt), p,
                                         (char *)ws, st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "embed_grad launch");
}

// ----- losses over the targets' log-probabilities ---------------------------------
struct LossLayout {
  LossPlan plan;
  size_t stat, ztgt, coef, rows, sync, total;
};
LossLayout loss_layout(int op, int64_t T, int64_t V, int64_t pairs, lora_dtype_t dt) {
  LossLayout L{};
  L.plan = loss_plan(T, V, dtype(dt), op == TOKEN_LOSS_OP_LOGP);
  const bool pref = op == TOKEN_LOSS_OP_PREFERENCE;
  size_t off = 0;
  L.stat = off;  // of the parts, and of the rows
  off += pref || L.plan.parts > 1 ? round256((size_t)T * (L.plan.parts + (pref ? 1 : 0)) * 8) : 0;
  L.ztgt = off;
  off += pref || L.plan.parts > 1 ? round256((size_t)T * 4) : 0;
  L.coef = off;
  off += pref ? round256((size_t)(T + 1) * 4) : 0;  // (and a word for offsets that are not ascending)
  L.rows = off;
  off += op == TOKEN_LOSS_OP_LOGP ? 0 : round256((size_t)(pref ? pairs : T) * 4);
  L.sync = off;
  off += op == TOKEN_LOSS_OP_LOGP && L.plan.parts > 1 ? round256((size_t)T * L.plan.parts * sizeof(meet_word)) : 0;
  L.total = off;
  return L;
}

lora_status_t check_loss_sizes(int op, int64_t T, int64_t V, int64_t ldz, int64_t pairs, lora_dtype_t dt) {
  if (op != TOKEN_LOSS_OP_LOGP && op != TOKEN_LOSS_OP_POLICY && op != TOKEN_LOSS_OP_PREFERENCE)
    return fail(LORA_EINVAL, "unknown operation");
  if (bad_dtype(dt)) return fail(LORA_EINVAL, "unknown dtype");
  if (T < 1 || V < 1 || ldz < V) return fail(LORA_EINVAL, "need T >= 1, V >= 1 and ldz >= V");
  if (op == TOKEN_LOSS_OP_PREFERENCE && pairs < 1) return fail(LORA_EINVAL, "need at least one pair");
  if (ldz % (dt == LORA_BF16 ? 8 : 4)) return fail(LORA_EUNSUPPORTED, "rows of logits must be whole 16-byte vectors");
  if (T > kMaxLossT || ldz > kMaxRows || T > kMaxMatrix / ldz || (op == TOKEN_LOSS_OP_PREFERENCE && pairs > kMaxPairs))
    return fail(LORA_EUNSUPPORTED, "T at most 2^23, ldz 2^30, pairs 2^22, logits 2^40 elements");
  return LORA_OK;
}

// What the three calls share once their sizes are checked: pointers, workspace, overlaps.  `more`
// are the inputs and `out` the outputs of one of them, besides logits, targets,
// weights, logp and dlogits.
lora_status_t check_loss(int op, const void *logits, int64_t ldz, const int32_t *targets, const float *weights, float *logp,
                         void *dlogits, int64_t T, int64_t V, int64_t pairs, lora_dtype_t dt, const Range *more,
                         size_t n_more, const Range *out, size_t n_out, void *ws, size_t ws_bytes, LossLayout *L) {
  lora_status_t s;
  if (!logits || !targets || !logp) return fail(LORA_EINVAL, "logits, targets and logp are required");
  const void *ptrs[] = {logits, targets, weights, logp, dlogits};
  if (misaligned(ptrs)) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
  *L = loss_layout(op, T, V, pairs, dt);
  if ((s = check_ws(ws, ws_bytes, L->total)) != LORA_OK) return s;
  const int64_t zb = T * ldz * (int64_t)esize(dt);
  Range ins[8], outs[8];
  size_t ni = 0, no = 0;
  ins[ni++] = rng(targets, T * 4);
  ins[ni++] = rng(weights, T * 4);
  if (dlogits != logits) ins[ni++] = rng(logits, zb);  // (dlogits may take the logits' place)
  for (size_t i = 0; i < n_more; ++i) ins[ni++] = more[i];
  outs[no++] = rng(logp, T * 4);
  outs[no++] = rng(dlogits, zb);
  outs[no++] = rng(ws, (int64_t)L->total);
  if (!dlogits) outs[1] = rng(nullptr, 0);
  for (size_t i = 0; i < n_out; ++i) outs[no++] = out[i];
  if (any_overlap(outs, no, ins, ni)) return fail(LORA_EINVAL, "an output overlaps an input or another output");
  return LORA_OK;
}

TokenLoss loss_args(const void *logits, int64_t ldz, const int32_t *targets, const float *weights, float *logp, void *dlogits,
                    float *loss, int64_t T, int64_t V, const LossLayout &L, void *ws) {
  char *wsb = (char *)ws;
  TokenLoss a{};
  a.z = logits;
  a.ld = ldz;
  a.T = (int)T;
  a.V = (int)V;
  a.y = targets;
  a.w = weights;
  a.logp = logp;
  a.dz = dlogits;
  a.loss = loss;
  a.parts = L.plan.parts;
  a.part_vecs = L.plan.part_vecs;
  a.stat = (float *)(wsb + L.stat);
  a.ztgt = (float *)(wsb + L.ztgt);
  a.coef = L.coef == L.rows ? nullptr : (float *)(wsb + L.coef);
  a.rows = (float *)(wsb + L.rows);
  a.sync = (meet_word *)(wsb + L.sync);
  return a;
}

// ----- gradient lists ---------------------------------------------------------------
constexpr int64_t kMaxGrads = int64_t(1) << 20;
constexpr int kChunkUnit = 4096;  // elements

// Chunks of about a fifteenth of a workgroup's share, so that the last round of
// chunks leaves few workgroups waiting.
int chunk_elems(int64_t elems) {
  const int64_t c = (elems / (16 * (int64_t)GRAD_PARTS) + kChunkUnit - 1) / kChunkUnit * kChunkUnit;
  return (int)std::min<int64_t>(std::max<int64_t>(c, kChunkUnit), 64 * kChunkUnit);
}

struct GradSizes {
  int64_t elems, nchunk;
  int chunk;
  size_t part, total;  // bytes: chunks, then partial sums
};
lora_status_t grad_sizes(const lora_grad_t *grads, int64_t n, GradSizes *z) {
  if (!grads) return fail(LORA_EINVAL, "grads is NULL");
  if (n < 1) return fail(LORA_EINVAL, "need at least one gradient");
  if (n > kMaxGrads) return fail(LORA_EUNSUPPORTED, "at most 2^20 gradients");
  *z = GradSizes{};
  for (int64_t i = 0; i < n; ++i) {
    const lora_grad_t &g = grads[i];
    if (g.n < 0) return fail(LORA_EINVAL, "a gradient's size is negative");
    if (g.n > kMaxMatrix) return fail(LORA_EUNSUPPORTED, "a gradient has more than 2^40 elements");
    if (g.n == 0) continue;
    if (!g.g) return fail(LORA_EINVAL, "a gradient is NULL");
    if (bad_dtype(g.dt) || (g.out && bad_dtype(g.out_dt))) return fail(LORA_EINVAL, "unknown dtype");
    if (!aligned16(g.g) || (g.out && !aligned16(g.out))) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
    if (g.out == g.g && g.out_dt != g.dt) return fail(LORA_EINVAL, "a gradient clipped in place keeps its type");
    z->elems += g.n;
    if (z->elems > kMaxMatrix) return fail(LORA_EUNSUPPORTED, "the gradients have more than 2^40 elements");
  }
  z->chunk = chunk_elems(z->elems);
  for (int64_t i = 0; i < n; ++i) z->nchunk += (grads[i].n + z->chunk - 1) / z->chunk;
  if (z->nchunk > kMaxRows) return fail(LORA_EUNSUPPORTED, "the gradients have too many elements");
  z->part = round256((size_t)z->nchunk * sizeof(GradChunk));
  z->total = z->part + (size_t)GRAD_PARTS * 8;
  return LORA_OK;
}

// Whether any output range overlaps another or any other gradient: the
// gradients' ranges in address order, each against the reach of those before it.
lora_status_t check_grad_ranges(const lora_grad_t *grads, int64_t n, const Range &mem) {
  struct Item {
    uintptr_t lo, hi;
    bool out;
  };
  Item *it = new (std::nothrow) Item[2 * n];
  if (!it) return fail(LORA_EUNSUPPORTED, "no host memory to check the list");
  int64_t m = 0;
  bool bad = false;
  for (int64_t i = 0; i < n; ++i) {
    const lora_grad_t &g = grads[i];
    if (g.n == 0) continue;
    const Range a = rng(g.g, g.n * (int64_t)esize(g.dt));
    const Range b = rng(g.out, g.out ? g.n * (int64_t)esize(g.out_dt) : 0);
    bad = bad || overlap(a, mem) || overlap(b, mem);
    const bool in_place = g.out == g.g;
    it[m++] = {a.lo, a.hi, in_place};
    if (b.set && !in_place) it[m++] = {b.lo, b.hi, true};
  }
  std::sort(it, it + m, [](const Item &x, const Item &y) { return x.lo < y.lo; });
  uintptr_t reach = 0, out_reach = 0;  // ends of all ranges, and of the outputs, so far
  for (int64_t i = 0; i < m && !bad; ++i) {
    bad = it[i].out ? it[i].lo < reach : it[i].lo < out_reach;
    reach = std::max(reach, it[i].hi);
    if (it[i].out) out_reach = std::max(out_reach, it[i].hi);
  }
  delete[] it;
  return bad ? fail(LORA_EINVAL, "an output overlaps an input or another output") : LORA_OK;
}

lora_status_t check_list(const lora_grad_list_t *list, const float *norm, int64_t norm_bytes) {
  if (!list || !norm) return fail(LORA_EINVAL, "list and norm are required");
  if (!list->mem || list->chunk < 1 || list->nchunk < 0) return fail(LORA_EINVAL, "the list has not been laid out");
  if (!aligned16(norm)) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
  const size_t bytes = round256((size_t)list->nchunk * sizeof(GradChunk)) + (size_t)GRAD_PARTS * 8;
  if (overlap(rng(norm, norm_bytes), rng(list->mem, (int64_t)bytes)))
    return fail(LORA_EINVAL, "norm overlaps the list's memory");
  return LORA_OK;
}
double *list_parts(const lora_grad_list_t *list) {
  return (double *)((char *)list->mem + round256((size_t)list->nchunk * sizeof(GradChunk)));
}

// One workgroup takes the list (16 chunks took as long as the two launches' 9 us).
bool few_chunks(const lora_grad_list_t *list) { return list->nchunk <= GRAD_FEW && list->chunk == kChunkUnit; }

}  // namespace

extern "C" {

lora_status_t embed_fwd(const void *table, const int32_t *ids, void *out, int64_t T, int64_t V, int64_t D, float scale,
                        lora_dtype_t dt, void *hip_stream) {
  lora_status_t s = check_embed(T, V, D, dt);
  if (s != LORA_OK) return s;
  if (!table || !ids || !out) return fail(LORA_EINVAL, "table, ids and out are required");
  if (!std::isfinite(scale)) return fail(LORA_EINVAL, "scale must be finite");
  const void *ptrs[] = {table, ids, out};
  if (misaligned(ptrs)) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
  const int64_t es = (int64_t)esize(dt);
  const Range ins[] = {rng(table, V * D * es), rng(ids, T * 4)}, outs[] = {rng(out, T * D * es)};
  if (clash(outs, ins)) return fail(LORA_EINVAL, "an output overlaps an input or another output");
  hipStream_t st = (hipStream_t)hip_stream;
  Timed t(K_EMBED_FWD, st);
  const hipError_t e = launch_embed_fwd(table, ids, out, (int)T, (int)V, (int)D, scale, dtype(dt), st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "embed_fwd launch");
}

size_t embed_bwd_workspace_bytes(int64_t T, int64_t V, int64_t D) {
  if (check_embed(T, V, D, LORA_BF16) != LORA_OK) return (size_t)-1;
  return embed_plan(T, V, D).total;
}

lora_status_t embed_bwd(const int32_t *ids, const void *dout, float *dtable, int64_t T, int64_t V, int64_t D, float scale,
                        int accumulate, lora_dtype_t dt, void *ws, size_t ws_bytes, void *hip_stream) {
  return embed_grad(ids, dout, dtable, nullptr, false, T, V, D, scale, accumulate, dt, ws, ws_bytes, hip_stream);
}

lora_status_t embed_bwd_rows(const int32_t *ids, const void *dout, int32_t *tokens, float *rows, int64_t T, int64_t V,
                             int64_t D, float scale, lora_dtype_t dt, void *ws, size_t ws_bytes, void *hip_stream) {
  return embed_grad(ids, dout, rows, tokens, true, T, V, D, scale, 0, dt, ws, ws_bytes, hip_stream);
}

size_t token_loss_workspace_bytes(token_loss_op_t op, int64_t T, int64_t V, int64_t ldz, int64_t npairs, lora_dtype_t dt) {
  if (check_loss_sizes(op, T, V, ldz, npairs, dt) != LORA_OK) return (size_t)-1;
  return loss_layout(op, T, V, npairs, dt).total;
}

lora_status_t token_logp(const void *logits, int64_t ldz, const int32_t *targets, const float *weights, float *logp,
                         int64_t T, int64_t V, lora_dtype_t dt, void *ws, size_t ws_bytes, void *hip_stream) {
  LossLayout L;
  lora_status_t s = check_loss_sizes(TOKEN_LOSS_OP_LOGP, T, V, ldz, 0, dt);
  if (s != LORA_OK) return s;
  s = check_loss(TOKEN_LOSS_OP_LOGP, logits, ldz, targets, weights, logp, nullptr, T, V, 0, dt, nullptr, 0, nullptr, 0, ws,
                 ws_bytes, &L);
  if (s != LORA_OK) return s;
  TokenLoss a = loss_args(logits, ldz, targets, weights, logp, nullptr, nullptr, T, V, L, ws);
  a.gen = next_tag();
  hipStream_t st = (hipStream_t)hip_stream;
  Timed t(K_TOKEN_LOGP, st);
  const hipError_t e = launch_token_logp(a, dtype(dt), st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "token_logp launch");
}

lora_status_t policy_loss(const void *logits, int64_t ldz, const int32_t *targets, const float *weights,
                          const float *advantages, const float *old_logp, const float *ref_logp, float *loss, float *logp,
                          void *dlogits, int64_t T, int64_t V, float clip_lo, float clip_hi, float kl_coef, lora_dtype_t dt,
                          void *ws, size_t ws_bytes, void *hip_stream) {
  lora_status_t s = check_loss_sizes(TOKEN_LOSS_OP_POLICY, T, V, ldz, 0, dt);
  if (s != LORA_OK) return s;
  if (!advantages || !old_logp || !loss) return fail(LORA_EINVAL, "advantages, old_logp and loss are required");
  if (!(clip_lo >= 0.0f) || !(clip_hi >= 0.0f)) return fail(LORA_EINVAL, "clip_lo and clip_hi must be >= 0");
  if (!std::isfinite(kl_coef)) return fail(LORA_EINVAL, "kl_coef must be finite");
  if (kl_coef != 0.0f && !ref_logp) return fail(LORA_EINVAL, "ref_logp is required with a kl_coef");
  const void *ptrs[] = {advantages, old_logp, ref_logp, loss};
  if (misaligned(ptrs)) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
  const Range ins[] = {rng(advantages, T * 4), rng(old_logp, T * 4), rng(ref_logp, T * 4)}, outs[] = {rng(loss, 4)};
  LossLayout L;
  s = check_loss(TOKEN_LOSS_OP_POLICY, logits, ldz, targets, weights, logp, dlogits, T, V, 0, dt, ins, 3, outs, 1, ws, ws_bytes,
                 &L);
  if (s != LORA_OK) return s;
  const TokenLoss a = loss_args(logits, ldz, targets, weights, logp, dlogits, loss, T, V, L, ws);
  const PolicyArgs p{advantages, old_logp, kl_coef != 0.0f ? ref_logp : nullptr, 1.0f - clip_lo, 1.0f + clip_hi, kl_coef};
  hipStream_t st = (hipStream_t)hip_stream;
  Timed t(K_POLICY_LOSS, st);
  const hipError_t e = launch_policy_loss(a, p, dtype(dt), st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "policy_loss launch");
}

lora_status_t preference_loss(const void *logits, int64_t ldz, const int32_t *targets, const float *weights,
                              const float *ref_logp, const int32_t *seq, int64_t npairs, float *loss, float *margins,
                              float *logp, void *dlogits, int64_t T, int64_t V, float beta, float label_smoothing,
                              lora_dtype_t dt, void *ws, size_t ws_bytes, void *hip_stream) {
  lora_status_t s = check_loss_sizes(TOKEN_LOSS_OP_PREFERENCE, T, V, ldz, npairs, dt);
  if (s != LORA_OK) return s;
  if (!seq || !loss || !margins) return fail(LORA_EINVAL, "seq, loss and margins are required");
  if (!std::isfinite(beta)) return fail(LORA_EINVAL, "beta must be finite");
  if (!(label_smoothing >= 0.0f && label_smoothing <= 1.0f)) return fail(LORA_EINVAL, "label_smoothing must be in [0, 1]");
  const void *ptrs[] = {ref_logp, seq, loss, margins};
  if (misaligned(ptrs)) return fail(LORA_EINVAL, "pointers must be 16-byte aligned");
  const Range ins[] = {rng(ref_logp, T * 4), rng(seq, (2 * npairs + 1) * 4)}, outs[] = {rng(loss, 4), rng(margins, npairs * 4)};
  LossLayout L;
  s = check_loss(TOKEN_LOSS_OP_PREFERENCE, logits, ldz, targets, weights, logp, dlogits, T, V, npairs, dt, ins, 2, outs, 2, ws,
                 ws_bytes, &L);
  if (s != LORA_OK) return s;
  const TokenLoss a = loss_args(logits, ldz, targets, weights, logp, dlogits, loss, T, V, L, ws);
  const PairArgs p{ref_logp, seq, (int)npairs, beta, label_smoothing, margins};
  hipStream_t st = (hipStream_t)hip_stream;
  Timed t(K_PREFERENCE_LOSS, st);
  const hipError_t e = launch_preference_loss(a, p, dtype(dt), st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "preference_loss launch");
}

size_t grad_list_bytes(const lora_grad_t *grads, int64_t n) {
  GradSizes z;
  return grad_sizes(grads, n, &z) == LORA_OK ? z.total : (size_t)-1;
}

lora_status_t grad_list_init(lora_grad_list_t *list, const lora_grad_t *grads, int64_t n, void *mem, size_t mem_bytes,
                             void *hip_stream) {
  if (!list) return fail(LORA_EINVAL, "list is NULL");
  GradSizes z;
  lora_status_t s = grad_sizes(grads, n, &z);
  if (s != LORA_OK) return s;
  if ((s = check_ws(mem, mem_bytes, z.total)) != LORA_OK) return s;
  if ((s = check_grad_ranges(grads, n, rng(mem, (int64_t)z.total))) != LORA_OK) return s;
  hipStream_t st = (hipStream_t)hip_stream;
  GradEntries es{};
  int count = 0, first = 0;
  bool outs = true;
  for (int64_t i = 0; i <= n; ++i) {
    if (count == GRAD_ENTRIES || (i == n && count > 0)) {
      const hipError_t e = launch_grad_layout(es, count, z.chunk, (GradChunk *)mem, st);
      if (e != hipSuccess) return hip_fail(e, "grad_layout launch");
      count = 0;
    }
    if (i == n || grads[i].n == 0) continue;
    const lora_grad_t &g = grads[i];
    outs = outs && g.out;
    es.e[count++] = {g.g, g.out, g.n, first, (g.dt == LORA_F32 ? 1 : 0) | (g.out && g.out_dt == LORA_F32 ? 2 : 0)};
    first += (int)((g.n + z.chunk - 1) / z.chunk);
  }
  *list = lora_grad_list_t{mem, z.elems, (int32_t)z.nchunk, z.chunk, outs ? 1 : 0};
  return LORA_OK;
}

lora_status_t grad_norm(const lora_grad_list_t *list, float *norm, void *hip_stream) {
  lora_status_t s = check_list(list, norm, 4);
  if (s != LORA_OK) return s;
  hipStream_t st = (hipStream_t)hip_stream;
  const GradChunk *c = (const GradChunk *)list->mem;
  Timed t(K_GRAD_NORM, st);
  const hipError_t e = few_chunks(list) ? launch_grad_few(c, list->nchunk, false, 0.0f, norm, st)
                                        : launch_grad_norm(c, list->nchunk, list_parts(list), norm, st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "grad_norm launch");
}

lora_status_t grad_clip(const lora_grad_list_t *list, float max_norm, float *norm, void *hip_stream) {
  lora_status_t s = check_list(list, norm, 8);
  if (s != LORA_OK) return s;
  if (!(max_norm >= 0.0f)) return fail(LORA_EINVAL, "max_norm must be >= 0");
  if (!list->has_out) return fail(LORA_EINVAL, "a gradient of the list has no output");
  hipStream_t st = (hipStream_t)hip_stream;
  hipError_t e;
  if (few_chunks(list)) {
    Timed t(K_GRAD_SCALE, st);
    e = launch_grad_few((const GradChunk *)list->mem, list->nchunk, true, max_norm, norm, st);
    t.done();
    return e == hipSuccess ? LORA_OK : hip_fail(e, "grad_scale launch");
  }
  {
    Timed t(K_GRAD_NORM, st);
    e = launch_grad_norm((const GradChunk *)list->mem, list->nchunk, list_parts(list), nullptr, st);
    t.done();
    if (e != hipSuccess) return hip_fail(e, "grad_norm launch");
  }
  Timed t(K_GRAD_SCALE, st);
  e = launch_grad_clip((const GradChunk *)list->mem, list->nchunk, list_parts(list), max_norm, norm, st);
  t.done();
  return e == hipSuccess ? LORA_OK : hip_fail(e, "grad_scale launch");
}

}  // extern "C"
