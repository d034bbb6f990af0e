"""What a fine-tuning program does around this package's linears, as cases that
can be timed and compared: the embedding lookup and its gradient, the
log-probabilities of given tokens, the clipped policy loss and the preference loss
with their gradients with respect to the logits, and the clipping of all adapter
gradients by their global norm.

A case is a dict of plain values; `prepare` makes its inputs on the GPU from a
seed, `run` is one pass: through the package's entry points where `own` is true,
else in the operators' plain form; `exact` is what a pass returns in 64-bit
arithmetic.
"""
from __future__ import annotations

import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DTYPES = {"bf16": BF16, "fp32": F32}
VOCAB_A, VOCAB_B = 128256, 151936  # the two 3B decoders' vocabularies
# (d_in, d_out) of the adapted linears of one decoder layer of either model.
LAYER_A = [(3072, 3072), (3072, 1024), (3072, 1024), (3072, 3072), (3072, 8192), (3072, 8192), (8192, 3072)]
LAYER_B = [(2048, 2048), (2048, 256), (2048, 256), (2048, 2048), (2048, 11008), (2048, 11008), (11008, 2048)]
LINEAR = [(256, 256)]
STACKS = {"a": LAYER_A, "b": LAYER_B, "linear": LINEAR}


def listed():
    return [
        # A short prompt's tokens looked up: latency counts.
        {"name": "lookup_prompt", "kind": "embed_fwd", "T": 24, "V": VOCAB_A, "D": 3072, "dt": "bf16", "scaled": False},
        # The longest context the method's memory tables sweep, scaled embeddings.
        {"name": "lookup_context", "kind": "embed_fwd", "T": 16384, "V": VOCAB_B, "D": 2048, "dt": "bf16", "scaled": True},
        # The gradient of a trained embedding in its compact form, an ordinary step.
        {"name": "embed_grad_rows", "kind": "embed_rows", "T": 4096, "V": VOCAB_A, "D": 3072, "dt": "bf16", "scaled": False},
        # The same as one dense matrix, an odd number of tokens.
        {"name": "embed_grad_dense", "kind": "embed_dense", "T": 1891, "V": VOCAB_B, "D": 2048, "dt": "bf16", "scaled": True},
        # Log-probabilities of a short answer under the reference weights.
        {"name": "logp_answer", "kind": "logp", "T": 24, "V": VOCAB_A, "pad": 0, "dt": "bf16", "live": 1.0},
        # The same of a whole batch of rollouts, prompts masked.
        {"name": "logp_rollouts", "kind": "logp", "T": 4096, "V": VOCAB_B, "pad": 0, "dt": "bf16", "live": 0.75},
        # A policy step on one short rollout over a small vocabulary, full precision.
        {"name": "policy_short", "kind": "policy", "T": 97, "V": 8192, "pad": 0, "dt": "fp32", "live": 1.0, "kl": 0.0},
        # A policy step on the rollouts of a group: the largest case.
        {"name": "policy_group", "kind": "policy", "T": 4096, "V": VOCAB_A, "pad": 0, "dt": "bf16", "live": 0.75, "kl": 0.04},
        # One preference pair over an odd vocabulary padded to whole vectors, full precision.
        {"name": "pair_odd", "kind": "preference", "T": 203, "V": 32001, "pad": 7, "dt": "fp32", "live": 0.6, "pairs": 1},
        # A batch of preference pairs.
        {"name": "pair_batch", "kind": "preference", "T": 2048, "V": VOCAB_B, "pad": 0, "dt": "bf16", "live": 0.6, "pairs": 4},
        # The gradients of a single small linear: launches and host work count.
        {"name": "clip_linear", "kind": "clip", "stack": "linear", "layers": 1, "r": 8, "out": "fp32"},
        # Every dA and dB of the 28-layer stack.
        {"name": "clip_stack", "kind": "clip", "stack": "a", "layers": 28, "r": 32, "out": "fp32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed_fwd", "embed_rows", "embed_dense", "logp", "policy", "policy", "preference", "preference", "clip"])
    dt = rng.choice(["bf16", "bf16", "fp32"])
    e = 2 if dt == "bf16" else 4
    if kind.startswith("embed"):
        V = _log_int(rng, 500, VOCAB_B)
        D = 8 * _log_int(rng, 8, 512)
        if kind == "embed_dense":
            V = max(2, min(V, 1200 * 10**6 // (4 * D)))
        T = _log_int(rng, 1 if kind == "embed_fwd" else 16, 32768)
        return {"kind": kind, "T": min(T, 10**9 // (8 * D)), "V": V, "D": D, "dt": dt, "scaled": rng.random() < 0.5}
    if kind == "clip":
        stack = rng.choice(["a", "b", "b", "linear"])
        layers = _log_int(rng, 1, {"a": 28, "b": 36, "linear": 8}[stack])
        return {"kind": kind, "stack": stack, "layers": layers, "r": rng.choice([4, 8, 13, 16, 32]), "out": rng.choice(["fp32", "fp32", "bf16"])}
    V = _log_int(rng, 1000, VOCAB_B)
    pad = -V % 8 + 8 * rng.choice([0, 0, 0, 3])
    T = _log_int(rng, 4, 4096)
    T = max(4, min(T, 900 * 10**6 // ((V + pad) * e)))
    c = {"kind": kind, "T": T, "V": V, "pad": pad, "dt": dt, "live": rng.choice([1.0, rng.uniform(0.2, 0.9)])}
    if kind == "policy":
        c["kl"] = rng.choice([0.0, 0.01, 0.1])
    if kind == "preference":
        c["pairs"] = max(1, min(rng.choice([1, 2, 4, 16]), T // 4))
    return c


# ---- inputs ------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _zipf(V):
    """Token frequencies of a text: inversely proportional to the rank."""
    p = 1.0 / (torch.arange(V, dtype=F64) + 3.0)
    return p / p.sum()


def _embed_inputs(c, seed):
    g = _gen(seed)
    T, V, D, dt = c["T"], c["V"], c["D"], DTYPES[c["dt"]]
    rank = torch.multinomial(_zipf(V).to("cuda"), T, replacement=True, generator=g)
    ids = torch.randperm(V, generator=g, device="cuda")[rank].to(torch.int32)
    s = {"ids": ids, "scale": math.sqrt(D) if c["scaled"] else 1.0}
    if c["kind"] == "embed_fwd":
        s["table"] = torch.empty(V, D, dtype=dt, device="cuda").normal_(0.0, 0.02, generator=g)
    else:
        s["dout"] = torch.randn(T, D, generator=g, device="cuda", dtype=F32).to(dt)
    return s


def _live_count(c, n):
    return max(1, int(round(n * c["live"])))


def _ends(c):
    """Where the sequences of a preference case end: pairs of a longer and a
    shorter answer, 2 pairs + 1 offsets into the T positions."""
    n = 2 * c["pairs"]
    share = [1.0 + 0.4 * math.sin(1.0 + 2.3 * i) for i in range(n)]
    ends, run_ = [0], 0.0
    for s in share:
        run_ += s
        ends.append(int(round(run_ / sum(share) * c["T"])))
    return ends


def _live_rows(c):
    """The trainable positions: the last of the batch, or of each sequence."""
    if c["kind"] != "preference":
        return list(range(c["T"] - _live_count(c, c["T"]), c["T"]))
    ends, rows = _ends(c), []
    for lo, hi in zip(ends, ends[1:]):
        if hi > lo:
            rows += range(hi - _live_count(c, hi - lo), hi)
    return rows


def _logit_inputs(c, seed):
    """Logits with a spread like a decoder's; each target drawn from its
    position's own distribution, as a rollout's tokens are."""
    g = _gen(seed)
    T, V, ld, dt = c["T"], c["V"], c["V"] + c["pad"], DTYPES[c["dt"]]
    z = torch.empty(T, ld, dtype=dt, device="cuda")
    y = torch.empty(T, dtype=torch.int32, device="cuda")
    logp = torch.empty(T, dtype=F64, device="cuda")
    for a in range(0, T, 512):
        b = min(T, a + 512)
        z[a:b] = torch.randn(b - a, ld, generator=g, device="cuda", dtype=F32) * 2.5
        zf = z[a:b, :V].float()
        noise = torch.empty_like(zf).exponential_(generator=g).log_()
        t = (zf - noise).argmax(1)
        y[a:b] = t.to(torch.int32)
        zd = zf.double()
        logp[a:b] = zd.gather(1, t[:, None])[:, 0] - torch.logsumexp(zd, 1)
    rows = torch.tensor(_live_rows(c), dtype=torch.int64, device="cuda")
    w = torch.zeros(T, dtype=F32, device="cuda")
    w[rows] = 1.0
    return {"z": z, "y": y, "rows": rows, "weights": w}, logp, g


CLIP_LO, CLIP_HI, BETA, SMOOTH = 0.2, 0.28, 0.1, 0.05


def _policy_inputs(c, seed):
    s, logp, g = _logit_inputs(c, seed)
    T = c["T"]
    # A few optimizer steps since the rollout: most ratios near one, some clipped.  They
    # keep a thousandth clear of the clip's edges, where the gradient jumps and
    # either side of the jump is right.
    lr = 0.15 * torch.randn(T, generator=g, device="cuda", dtype=F64)
    for edge in (1.0 - CLIP_LO, 1.0 + CLIP_HI):
        d = lr.exp() - edge
        lr = torch.where(d.abs() < 1e-3, (edge + torch.where(d < 0, -1e-3, 1e-3)).log(), lr)
    s["old"] = (logp - lr).float()
    s["ref"] = (logp + 0.3 * torch.randn(T, generator=g, device="cuda", dtype=F64)).float() if c["kl"] else None
    adv = torch.randn(-(-T // 128), generator=g, device="cuda", dtype=F32)  # one per rollout
    s["adv"] = adv.repeat_interleave(128)[:T].contiguous()
    s["weights"] /= s["rows"].numel()  # the mean over the trainable positions
    s["kl"] = c["kl"]
    return s


def _preference_inputs(c, seed):
    s, logp, g = _logit_inputs(c, seed)
    s["ref"] = (logp + 0.3 * torch.randn(c["T"], generator=g, device="cuda", dtype=F64)).float()
    s["seq"] = torch.tensor(_ends(c), dtype=torch.int32, device="cuda")
    s["ends"] = _ends(c)
    return s


def _clip_shapes(c):
    shapes = []
    for d_in, d_out in STACKS[c["stack"]] * c["layers"]:
        shapes += [(c["r"], d_in), (d_out, c["r"])]
    return shapes


def _clip_inputs(c, seed):
    """Adapter gradients whose size differs from layer to layer."""
    g = _gen(seed)
    grads = []
    for i, shape in enumerate(_clip_shapes(c)):
        grads.append(torch.randn(*shape, generator=g, device="cuda", dtype=F32) * (0.002 * (1.0 + (i % 7))))
    return {"grads": grads, "max_norm": 1.0e-2}


def prepare(case, seed):
    c = dict(case)
    kind = c["kind"]
    T = c.get("T", 0)

    def new(*shape, dtype=F32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if kind.startswith("embed"):
        s = _embed_inputs(c, seed)
        if kind == "embed_fwd":
            s["out"] = new(T, c["D"], dtype=DTYPES[c["dt"]])
        elif kind == "embed_rows":
            n = min(T, c["V"])
            s["tokens"], s["out"] = new(n, dtype=torch.int32), new(n, c["D"])
        else:
            s["out"] = new(c["V"], c["D"])
    elif kind == "clip":
        s = _clip_inputs(c, seed)
        # The clipped gradients go into one flat buffer, as an optimizer or a data-parallel
        # reduction over all adapters takes them.
        s["out"] = new(sum(x.numel() for x in s["grads"]), dtype=DTYPES[c["out"]])
        s["norm"] = new(2)
        if own:
            import paper_2606_19528_amd as lm

            parts = s["out"].split([x.numel() for x in s["grads"]])
            s["list"] = lm.grad_list(s["grads"], parts)  # kept by the program, as the buffers are
    else:
        s = {"logp": _logit_inputs, "policy": _policy_inputs, "preference": _preference_inputs}[kind](c, seed)
        if kind == "logp":
            s = s[0]
        else:
            s["dz"] = torch.empty_like(s["z"])
            s["loss"] = new(1)
            if kind == "preference":
                s["margins"] = new(c["pairs"])
        s["logp"] = new(T)
    if own and kind not in ("embed_fwd", "clip"):
        import paper_2606_19528_amd as lm

        if kind.startswith("embed"):
            n = lm.embed_bwd_workspace_bytes(T, c["V"], c["D"])
        else:
            op = {"logp": lm.TOKEN_LOSS_OP_LOGP, "policy": lm.TOKEN_LOSS_OP_POLICY, "preference": lm.TOKEN_LOSS_OP_PREFERENCE}[kind]
            n = lm.token_loss_workspace_bytes(op, T, c["V"], c["V"] + c["pad"], c.get("pairs", 0),
                                              lm.LORA_BF16 if c["dt"] == "bf16" else lm.LORA_F32)
        s["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    s["case"] = c
    return s


# ---- one pass: the package's entry points --------------------------------------
def _run_own(s):
    import paper_2606_19528_amd as lm

    c = s["case"]
    kind = c["kind"]
    if kind == "embed_fwd":
        return lm.embed_fwd(s["table"], s["ids"], s["out"], scale=s["scale"])
    if kind == "embed_rows":
        lm.embed_bwd_rows(s["ids"], s["dout"], c["V"], s["tokens"], s["out"], scale=s["scale"], ws=s["ws"])
        return [s["tokens"], s["out"]]
    if kind == "embed_dense":
        return lm.embed_bwd(s["ids"], s["dout"], s["out"], scale=s["scale"], ws=s["ws"])
    if kind == "logp":
        return lm.token_logp(s["z"], s["y"], s["logp"], weights=s["weights"], vocab=c["V"], ws=s["ws"])
    if kind == "policy":
        lm.policy_loss(s["z"], s["y"], s["weights"], s["adv"], s["old"], s["ref"], s["loss"], s["logp"], s["dz"],
                       clip_lo=CLIP_LO, clip_hi=CLIP_HI, kl_coef=s["kl"], vocab=c["V"], ws=s["ws"])
        return [s["loss"], s["logp"], s["dz"]]
    if kind == "preference":
        lm.preference_loss(s["z"], s["y"], s["weights"], s["ref"], s["seq"], s["loss"], s["margins"], s["logp"], s["dz"],
                           beta=BETA, label_smoothing=SMOOTH, vocab=c["V"], ws=s["ws"])
        return [s["loss"], s["margins"], s["logp"], s["dz"]]
    lm.grad_clip(s["list"], s["max_norm"], s["norm"])
    return [s["norm"], s["out"]]


# ---- one pass: the plain forms, in 32 bits ---------------------------------------
def _segments(ids):
    """Sorted order of the tokens, and for each place in it the number of its
    token among the distinct ones."""
    order = torch.argsort(ids, stable=True)
    sid = ids[order]
    first = torch.ones_like(sid)
    first[1:] = (sid[1:] != sid[:-1]).to(sid.dtype)
    return order, sid, torch.cumsum(first, 0) - 1


def _plain_logp(z, y):
    """(log-probability, log-sum-exp) of rows of logits."""
    m = z.amax(1, keepdim=True)
    lse = m + (z - m).exp().sum(1, keepdim=True).log()
    return (z.gather(1, y[:, None]) - lse)[:, 0], lse


def _plain_dz(s, z, lse, y, coef):
    """coef_t ([j = y_t] - softmax(z_t)_j) in the live rows, zeros elsewhere."""
    d = (z - lse).exp() * -coef[:, None]
    d.scatter_add_(1, y[:, None], coef[:, None])
    out = torch.zeros_like(s["z"])
    out[s["rows"], : z.shape[1]] = d.to(out.dtype)
    return out


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "embed_fwd":
        return (s["table"][s["ids"]].float() * s["scale"]).to(s["table"].dtype)
    if kind == "embed_rows":
        n = s["out"].shape[0]
        order, sid, seg = _segments(s["ids"])
        tokens = torch.full_like(s["tokens"], -1)
        tokens[seg] = sid
        rows = torch.zeros(n, c["D"], dtype=F32, device="cuda")
        rows.index_add_(0, seg, s["dout"][order].float())
        return [tokens, rows * s["scale"]]
    if kind == "embed_dense":
        out = torch.zeros(c["V"], c["D"], dtype=F32, device="cuda")
        return out.index_add_(0, s["ids"], s["dout"].float() * s["scale"])
    if kind == "clip":
        flat = torch.cat([g.view(-1) for g in s["grads"]])
        norm = (flat * flat).sum().sqrt()
        coef = torch.where(norm <= s["max_norm"], torch.ones_like(norm), s["max_norm"] / norm)
        return [torch.stack([norm, coef]), (flat * coef).to(s["out"].dtype)]
    rows, V = s["rows"], c["V"]
    z, y, w = s["z"][rows][:, :V].float(), s["y"][rows].long(), s["weights"][rows]
    logp, lse = _plain_logp(z, y)
    full = torch.zeros(c["T"], dtype=F32, device="cuda")
    full[rows] = logp
    if kind == "logp":
        return full
    if kind == "policy":
        adv = s["adv"][rows]
        ratio = (logp - s["old"][rows]).exp()
        free, held = ratio * adv, ratio.clamp(1.0 - CLIP_LO, 1.0 + CLIP_HI) * adv
        loss = -torch.minimum(free, held)
        grad = torch.where(free <= held, -free, torch.zeros_like(free))
        if s["kl"]:
            d = s["ref"][rows] - logp
            loss = loss + s["kl"] * (d.exp() - d - 1.0)
            grad = grad + s["kl"] * (1.0 - d.exp())
        return [(w * loss).sum()[None], full, _plain_dz(s, z, lse, y, w * grad)]
    diff = torch.zeros_like(full)
    diff[rows] = w * (logp - s["ref"][rows])
    sums = torch.stack([diff[a:b].sum() for a, b in zip(s["ends"], s["ends"][1:])])
    margin = BETA * (sums[0::2] - sums[1::2])
    up, down = 1.0 / (1.0 + (-margin).exp()), 1.0 / (1.0 + margin.exp())
    loss = (-(1.0 - SMOOTH) * up.log() - SMOOTH * down.log()).mean()
    g = BETA * (SMOOTH * up - (1.0 - SMOOTH) * down) / c["pairs"]
    coef = torch.zeros_like(full)
    for i, (a, b) in enumerate(zip(s["ends"], s["ends"][1:])):
        coef[a:b] = g[i // 2] if i % 2 == 0 else -g[i // 2]
    return [loss[None], margin, full, _plain_dz(s, z, lse, y, w * coef[rows])]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ----------------------------------------------
def work(case):
    c = case
    kind = c["kind"]
    if kind == "clip":
        n = sum(a * b for a, b in _clip_shapes(c))
        return {"bytes": n * (4 + (2 if c["out"] == "bf16" else 4)) + 8, "flops": 3 * n}
    e = 2 if c["dt"] == "bf16" else 4
    T, V = c["T"], c["V"]
    if kind.startswith("embed"):
        D = c["D"]
        if kind == "embed_fwd":  # the distinct tokens' rows, as many as are expected
            distinct = float((-torch.expm1(T * torch.log1p(-_zipf(V)))).sum())
            return {"bytes": int(4 * T + (distinct + T) * D * e), "flops": T * D}
        n = min(T, V)
        wr = 4 * V * D if kind == "embed_dense" else n * (4 * D + 4)
        return {"bytes": 4 * T + T * D * e + wr, "flops": 2 * T * D}
    live = len(_live_rows(c))
    if kind == "logp":
        return {"bytes": live * (V * e + 4) + 8 * T, "flops": 3 * live * V}
    extra = (4 if kind == "policy" else 2) * 4 * T
    return {"bytes": live * V * e + T * (V + c["pad"]) * e + extra, "flops": 6 * live * V}


# ---- the operators' definitions in 64 bits ---------------------------------------
def _exact_rows(z, y, V):
    """log p(y_t | t) and the softmax of each row, both in 64 bits."""
    zd = z[:, :V].double()
    p = torch.softmax(zd, 1)
    return torch.log_softmax(zd, 1)[torch.arange(z.shape[0], device=z.device), y.long()], p


def exact(case, seed):
    c = dict(case)
    kind = c["kind"]
    if kind == "embed_fwd":
        s = _embed_inputs(c, seed)
        return s["table"].double()[s["ids"].long()] * s["scale"]
    if kind.startswith("embed"):
        s = _embed_inputs(c, seed)
        ids, dout = s["ids"].long(), s["dout"].double() * s["scale"]
        if kind == "embed_dense":
            return torch.zeros(c["V"], c["D"], dtype=F64, device="cuda").index_add_(0, ids, dout)
        n = min(c["T"], c["V"])
        tok, inv = torch.unique(ids, sorted=True, return_inverse=True)
        tokens = torch.cat([tok.to(torch.int32), torch.full((n - tok.numel(),), -1, dtype=torch.int32, device="cuda")])
        return [tokens, torch.zeros(n, c["D"], dtype=F64, device="cuda").index_add_(0, inv, dout)]
    if kind == "clip":
        s = _clip_inputs(c, seed)
        norm = math.sqrt(sum(float(g.double().square().sum()) for g in s["grads"]))
        coef = min(1.0, s["max_norm"] / norm)
        return [torch.tensor([norm, coef], dtype=F64, device="cuda"), torch.cat([g.flatten().double() * coef for g in s["grads"]])]
    T, V = c["T"], c["V"]
    s = {"logp": lambda *a: _logit_inputs(*a)[0], "policy": _policy_inputs, "preference": _preference_inputs}[kind](c, seed)
    w, live = s["weights"].double(), s["weights"] != 0
    logp = torch.zeros(T, dtype=F64, device="cuda")
    for a in range(0, T, 256):
        logp[a:a + 256] = _exact_rows(s["z"][a:a + 256], s["y"][a:a + 256], V)[0]
    logp = torch.where(live, logp, torch.zeros_like(logp))
    if kind == "logp":
        return logp
    if kind == "policy":
        A, ratio = s["adv"].double(), torch.exp(logp - s["old"].double())
        bound = torch.where(A >= 0, torch.full_like(A, 1.0 + CLIP_HI), torch.full_like(A, 1.0 - CLIP_LO))
        inside = torch.where(A >= 0, ratio <= bound, ratio >= bound)
        loss = -A * torch.where(inside, ratio, bound)
        coef = torch.where(inside, -A * ratio, torch.zeros_like(A))
        if c["kl"]:
            d = s["ref"].double() - logp
            loss, coef = loss + c["kl"] * (torch.expm1(d) - d), coef - c["kl"] * torch.expm1(d)
        head, coef = [torch.where(live, w * loss, 0.0).sum()[None], logp], torch.where(live, w * coef, 0.0)
    else:
        diff = torch.where(live, w * (logp - s["ref"].double()), 0.0)
        ends = s["ends"]
        coef, margins, total = torch.zeros_like(logp), [], 0.0
        for i in range(c["pairs"]):
            a, b, d = ends[2 * i], ends[2 * i + 1], ends[2 * i + 2]
            m = BETA * float(diff[a:b].sum() - diff[b:d].sum())
            margins.append(m)
            total += (1.0 - SMOOTH) * math.log1p(math.exp(-m)) + SMOOTH * math.log1p(math.exp(m))
            g = BETA / c["pairs"] * (1.0 / (1.0 + math.exp(-m)) - (1.0 - SMOOTH))
            coef[a:b], coef[b:d] = g, -g
        coef = torch.where(live, w * coef, 0.0)
        head = [torch.tensor([total / c["pairs"]], dtype=F64, device="cuda"), torch.tensor(margins, dtype=F64, device="cuda"), logp]
    dz = torch.zeros(T, V + c["pad"], dtype=F64, device="cuda")
    for a in range(0, T, 256):
        b = min(T, a + 256)
        d = -coef[a:b, None] * _exact_rows(s["z"][a:b], s["y"][a:b], V)[1]
        d[torch.arange(b - a, device="cuda"), s["y"][a:b].long()] += coef[a:b]
        dz[a:b, :V] = d
    return [*head, dz]
