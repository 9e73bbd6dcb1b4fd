"""Cases that time the training operators of this package: the log-probabilities of given tokens with their gradient,
the junction of a block's output with the residual stream (norm after the block, gate, residual scale, norm before the
next block) with its gradient, and the orthogonalised update of a weight matrix.

`run` computes them from elementary torch operations, or, where `own` is true, through the package's entry points.
`exact` states the same operators in 64 bits from their definitions."""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
NS = (3.4445, -4.7750, 2.0315)      # coefficients of the Newton-Schulz polynomial a s + b s^3 + c s^5


def listed():
    return [
        # one decoded position scored against the whole vocabulary: latency
        {"name": "logp_one_row_32000", "op": "logp", "rows": 1, "vocab": 32000, "ld": 32000, "type": "bf16", "temp": 0.7, "top": 8},
        # every position of a fine-tuning batch (8 x 512) of the GPT-2-shaped model; rows of 50257 are not 16-byte multiples
        {"name": "logp_4096x50257", "op": "logp", "rows": 4096, "vocab": 50257, "ld": 50257, "type": "bf16", "temp": 1.0, "top": 5},
        # the answer tokens of one short example in single precision
        {"name": "logp_bwd_37x50257_fp32", "op": "logp_bwd", "rows": 37, "vocab": 50257, "ld": 50257, "type": "fp32", "temp": 1.0, "ent": True},
        # gradient of a whole batch (4 x 512) of the LLaMA-shaped model into its logits
        {"name": "logp_bwd_2048x32000", "op": "logp_bwd", "rows": 2048, "vocab": 32000, "ld": 32000, "type": "bf16", "temp": 1.0, "ent": True},
        # the classifier's 16 first tokens, each with a gate of its own
        {"name": "join_16x768_ln", "op": "join", "rows": 16, "cols": 768, "kind": 0, "type": "fp32", "gate": 1, "post": True, "pre": True, "scale": 1.0},
        # a junction of the LLaMA-shaped model, one learned gate vector
        {"name": "join_2048x4096_rms", "op": "join", "rows": 2048, "cols": 4096, "kind": 1, "type": "bf16", "gate": 2048, "post": True, "pre": True, "scale": 1.0},
        # the encoder's batch (16 x 128), a gate per sequence, scaled residual
        {"name": "join_bwd_2048x768_ln", "op": "join_bwd", "rows": 2048, "cols": 768, "kind": 0, "type": "bf16", "gate": 128, "post": True, "pre": True, "scale": 0.5},
        # a long batch of the LLaMA-shaped model
        {"name": "join_bwd_16384x4096_rms", "op": "join_bwd", "rows": 16384, "cols": 4096, "kind": 1, "type": "bf16", "gate": 16384, "post": True, "pre": True, "scale": 1.0},
        # the attention projection of the encoder: a small square matrix
        {"name": "orth_768x768", "op": "orth", "rows": 768, "cols": 768, "type": "bf16", "steps": 5},
        # the feed-forward matrix of the GPT-2-shaped model, taller than wide
        {"name": "orth_5120x1280_fp32", "op": "orth", "rows": 5120, "cols": 1280, "type": "fp32", "steps": 5},
        # one whole update of an odd-sized matrix
        {"name": "muon_1000x777", "op": "muon", "rows": 1000, "cols": 777, "steps": 5, "nesterov": True},
        # one whole update of the LLaMA-shaped down projection
        {"name": "muon_4096x11008", "op": "muon", "rows": 4096, "cols": 11008, "steps": 5, "nesterov": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logp", "logp_bwd", "join", "join_bwd", "orth", "muon"])
    kind = rng.choice(["fp32", "bf16"])
    if op in ("logp", "logp_bwd"):
        vocab = _log_int(rng, 2, 131072)
        most = 2048 * 32000 if op == "logp_bwd" else 4096 * 50257
        rows = _log_int(rng, 1, max(1, min(4096, most // (vocab * (2 if kind == "fp32" else 1)))))
        case = {"op": op, "rows": rows, "vocab": vocab, "ld": vocab if rng.random() < 0.5 else (vocab + 63) // 64 * 64,
                "type": kind, "temp": rng.choice([1.0, 0.7, 1.5])}
        return dict(case, top=rng.randint(0, 20)) if op == "logp" else dict(case, ent=rng.random() < 0.7)
    if op in ("join", "join_bwd"):
        cols = 8 * _log_int(rng, 1, 1024)
        rows = _log_int(rng, 1, min(16384, 16384 * 4096 // (cols * (2 if kind == "fp32" else 1))))
        post, pre = rng.choice([(True, True), (True, True), (True, False), (False, True)])
        return {"op": op, "rows": rows, "cols": cols, "kind": rng.randint(0, 1), "type": kind,
                "gate": rng.choice([0, 1, rows, max(1, rows // 3)]), "post": post, "pre": pre, "scale": rng.choice([1.0, 0.5])}
    rows, cols = _log_int(rng, 1, 11008), _log_int(rng, 1, 11008)
    if min(rows, cols) > 4096:
        rows = 4096
    case = {"op": op, "rows": rows, "cols": cols, "steps": 5}
    return dict(case, type=kind) if op == "orth" else dict(case, nesterov=rng.random() < 0.5)


def work(case):
    op = case["op"]
    es = 2 if case.get("type") == "bf16" else 4
    if op in ("logp", "logp_bwd"):
        n = case["rows"] * case["vocab"]
        if op == "logp":
            return {"bytes": n * es + case["rows"] * (20 + 8 * case["top"]), "flops": 6 * n}
        return {"bytes": 2 * n * es + 24 * case["rows"], "flops": 8 * n}
    if op in ("join", "join_bwd"):
        n = case["rows"] * case["cols"]
        vec = case["cols"] * (2 + 2 * case["post"] + 2 * case["pre"]) * 4
        if op == "join":
            return {"bytes": n * (8 + es + (es if case["pre"] else 0)) + vec, "flops": 14 * n}
        # in: the two gradients, the stream (for the norm before the next block), the block's output; out: two gradients
        return {"bytes": n * (8 + 2 * es + ((4 + es) if case["pre"] else 0)) + 2 * vec, "flops": 30 * n}
    m, n = sorted((case["rows"], case["cols"]))
    # per step: the Gram matrix and its square are symmetric (half the products), then one full product
    flops = case["steps"] * (3.0 * m * m * n + 1.0 * m * m * m)
    if op == "orth":
        return {"bytes": m * n * (es + 2), "flops": flops}
    return {"bytes": m * n * (4 * 5 + 2), "flops": flops}     # gradient in; master and momentum in and out; model copy out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device="cuda") * std + mean

    s = dict(case)
    if case["op"] in ("logp", "logp_bwd"):
        rows, vocab, ld = case["rows"], case["vocab"], case["ld"]
        dt = TYPES[case["type"]]
        # a model's logits: spread of a few units, a common word-frequency profile, the model sure of some of its tokens
        x = normal(rows, ld, std=2.0)
        x[:, :vocab] += normal(vocab, std=1.5)
        tok = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        sure = torch.rand(rows, generator=g, device="cuda")
        x[torch.arange(rows, device="cuda"), tok] += 14.0 * sure
        if vocab >= 64:                                      # words that decoding forbids
            x[:, torch.randint(0, vocab, (vocab // 64,), generator=g, device="cuda")] = -math.inf
        tok = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.1, -1, tok) if rows > 1 else tok
        s["logits"], s["tokens"] = x.to(dt), tok.to(torch.int32)
        if case["op"] == "logp_bwd":
            z = s["logits"][:, :vocab].double()
            m = z.amax(1, keepdim=True)
            e = (z - m) / case["temp"]
            lsum = torch.logsumexp(e, 1, keepdim=True)
            p = torch.exp(e - lsum)
            ent = -(p * torch.where(p > 0, e - lsum, 0.0)).sum(1)
            live = tok >= 0
            s["stats"] = torch.cat([torch.where(live, m[:, 0], 0.0), torch.where(live, lsum[:, 0], 0.0)]).float()
            s["entropy"] = torch.where(live, ent, 0.0).float()
            s["dlogp"] = normal(rows) / rows                 # advantages over the batch
            s["dent"] = torch.full((rows,), -0.01 / rows, device="cuda") if case["ent"] else None
        return s
    if case["op"] in ("join", "join_bwd"):
        rows, cols = case["rows"], case["cols"]
        dt = TYPES[case["type"]]
        s["x"] = normal(rows, cols, std=1.5)
        s["h"] = normal(rows, cols, std=0.7, mean=0.1).to(dt)
        s["eps"] = 1e-5 if case["kind"] == 0 else 1e-6
        for n in (("1",) if case["post"] else ()) + (("2",) if case["pre"] else ()):
            s["gain" + n] = normal(cols, std=0.1, mean=1.0).to(dt)
            s["bias" + n] = normal(cols, std=0.1).to(dt) if case["kind"] == 0 else None
        s["gatev"] = normal(-(-rows // case["gate"]), cols, std=0.3, mean=0.5).to(dt) if case["gate"] else None
        if case["op"] == "join_bwd":
            s["dy"] = normal(rows, cols, std=1e-2).to(dt) if case["pre"] else None
            s["dxo"] = normal(rows, cols, std=1e-2)
            # what the forward pass leaves: the joined stream and the statistics of the two norms
            xo, _, st = _join_plain(s, torch.float64)
            s["xo"], s["stats"] = xo.float(), st.float()
        return s
    rows, cols = case["rows"], case["cols"]
    # a gradient: a few strong directions over the products of a batch's activations and errors, and noise
    r = max(1, min(rows, cols) // 8)
    decay = torch.arange(1, r + 1, device="cuda").float() ** -0.5
    grad = (normal(rows, r) * decay) @ normal(r, cols) * 1e-3 + normal(rows, cols, std=3e-4)
    if case["op"] == "orth":
        s["g"] = grad.to(TYPES[case["type"]])
        return s
    s["grad"] = grad
    s["master"] = normal(rows, cols, std=0.02)
    s["mom"] = normal(rows, cols, std=1e-3)
    s["param"] = s["master"].to(torch.bfloat16)
    s["hp"] = {"lr": 1e-4, "momentum": 0.95, "weight_decay": 0.01}
    return s


# ------------------------------------------------------------------ plain forms
def _ordered_keys(x, n):
    """int64 keys that order by value and, among equal values, by lower index first."""
    i = (x.float() + 0.0).view(torch.int32)
    i = torch.where(i < 0, i ^ 0x7FFFFFFF, i).long()
    return (i << 32) + (n - 1 - torch.arange(n, device=x.device))


def _logp_plain(s):
    vocab, scale, top = s["vocab"], 1.0 / s["temp"], s["top"]
    raw = s["logits"][:, :vocab]
    live = s["tokens"] >= 0
    x = raw.float()
    m = x.amax(1, keepdim=True)
    e = (x - m) * scale
    w = torch.exp(e)
    total = w.sum(1, keepdim=True, dtype=torch.float64)     # the largest logit's 1 must not swallow a small rest
    lsum = torch.log1p(total - 1.0).float()
    ent = lsum[:, 0] - (w * torch.where(w > 0, e, 0.0)).sum(1) / total[:, 0].float()
    logp = e.gather(1, s["tokens"].clamp(min=0).long()[:, None])[:, 0] - lsum[:, 0]
    out = {"logp": torch.where(live, logp, 0.0), "entropy": torch.where(live, ent, 0.0),
           "stats": torch.cat([torch.where(live, m[:, 0], 0.0), torch.where(live, lsum[:, 0], 0.0)])}
    if top:
        k = min(top, vocab)
        ids = vocab - 1 - (torch.topk(_ordered_keys(raw, vocab), k, dim=1).values & 0xFFFFFFFF)
        v = e.gather(1, ids) - lsum
        none = (v == -math.inf) | ~live[:, None]
        full_i = torch.full((s["rows"], top), -1, dtype=torch.int32, device=x.device)
        full_v = torch.full((s["rows"], top), -math.inf, device=x.device)
        full_i[:, :k] = torch.where(none, -1, ids).int()
        full_v[:, :k] = torch.where(none, -math.inf, v)
        out["top_ids"], out["top_logp"] = full_i, full_v
    return out


def _logp_bwd_plain(s):
    vocab, rows, scale = s["vocab"], s["rows"], 1.0 / s["temp"]
    live = (s["tokens"] >= 0)[:, None]
    lp = (s["logits"][:, :vocab].float() - s["stats"][:rows, None]) * scale - s["stats"][rows:, None]
    p = torch.exp(lp)
    d = -p * s["dlogp"][:, None]
    t = s["tokens"].clamp(min=0).long()[:, None]
    d.scatter_(1, t, -torch.expm1(lp.gather(1, t)) * s["dlogp"][:, None])      # 1 - p of a token that is nearly sure
    if s["dent"] is not None:
        d = d - s["dent"][:, None] * p * (torch.where(p > 0, lp, 0.0) + s["entropy"][:, None])
    out = torch.zeros(rows, s["ld"], dtype=s["logits"].dtype, device=d.device)
    out[:, :vocab] = torch.where(live, d * scale, 0.0).to(out.dtype)
    return {"dlogits": out}


def _norm_plain(v, kind, eps, gain, bias, dt):
    mean = v.mean(1, keepdim=True) if kind == 0 else torch.zeros_like(v[:, :1])
    rstd = 1.0 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)
    out = (v - mean) * rstd * gain.to(dt)
    return (out if bias is None else out + bias.to(dt)), mean[:, 0], rstd[:, 0]


def _gate_rows(s, dt):
    if s["gatev"] is None:
        return None
    return s["gatev"].to(dt).repeat_interleave(s["gate"], 0)[: s["rows"]]


def _join_plain(s, dt=torch.float32):
    u, zero = s["h"].to(dt), torch.zeros(s["rows"], dtype=dt, device="cuda")
    st = [zero] * 4
    if s["post"]:
        u, st[0], st[1] = _norm_plain(u, s["kind"], s["eps"], s["gain1"], s["bias1"], dt)
    gate = _gate_rows(s, dt)
    xo = s["scale"] * s["x"].to(dt) + (u if gate is None else u * gate)
    y = None
    if s["pre"]:
        y, st[2], st[3] = _norm_plain(xo, s["kind"], s["eps"], s["gain2"], s["bias2"], dt)
    return xo, y, torch.cat(st)


def _norm_back_plain(g, hat, rstd, kind):
    out = g - hat * (g * hat).mean(1, keepdim=True)
    if kind == 0:
        out = out - g.mean(1, keepdim=True)
    return out * rstd


def _join_bwd_plain(s):
    rows, st = s["rows"], s["stats"]
    out, dt = {}, s["h"].dtype
    d = s["dxo"]
    if s["pre"]:
        dy = s["dy"].float()
        hat2 = (s["xo"] - st[2 * rows:3 * rows, None]) * st[3 * rows:, None]
        out["dgain2"] = (dy * hat2).sum(0)
        if s["kind"] == 0:
            out["dbias2"] = dy.sum(0)
        d = d + _norm_back_plain(dy * s["gain2"].float(), hat2, st[3 * rows:, None], s["kind"])
    out["dx"] = s["scale"] * d
    u = s["h"].float()
    if s["post"]:
        hat1 = (u - st[:rows, None]) * st[rows:2 * rows, None]
        u = hat1 * s["gain1"].float()
        if s["kind"] == 0:
            u = u + s["bias1"].float()
    gate = _gate_rows(s, torch.float32)
    du = d
    if gate is not None:
        n_gates = s["gatev"].shape[0]
        pad = n_gates * s["gate"] - rows
        t = torch.nn.functional.pad(d * u, (0, 0, 0, pad)) if pad else d * u
        out["dgate"] = t.view(n_gates, s["gate"], -1).sum(1)
        du = d * gate
    if s["post"]:
        out["dgain1"] = (du * hat1).sum(0)
        if s["kind"] == 0:
            out["dbias1"] = du.sum(0)
        du = _norm_back_plain(du * s["gain1"].float(), hat1, st[rows:2 * rows, None], s["kind"])
    out["dh"] = du.to(dt)
    return out


def _ns_plain(g, steps):
    a, b, c = NS
    x = g.float()
    x = x / x.double().square().sum().sqrt().clamp(min=1e-30).float()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    for _ in range(steps):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.T if tall else x


def _muon_plain(s):
    hp = s["hp"]
    s["mom"].mul_(hp["momentum"]).add_(s["grad"])
    u = s["grad"] + hp["momentum"] * s["mom"] if s["nesterov"] else s["mom"]
    o = _ns_plain(u, s["steps"])
    size = hp["lr"] * 0.2 * math.sqrt(max(s["rows"], s["cols"]))
    s["master"].mul_(1.0 - hp["lr"] * hp["weight_decay"]).sub_(size * o)
    s["param"].copy_(s["master"])
    return {"master": s["master"], "momentum": s["mom"], "param": s["param"]}


# ------------------------------------------------------------------ the framework's calls
def _keep(s, name, make):
    if name not in s:
        s[name] = make()
    return s[name]


def _own(s):
    import paper_2401_15207_b200 as P
    op, rows = s["op"], s["rows"]
    code = 1 if s.get("type") == "bf16" else 0

    def new(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if op == "logp":
        top = s["top"]
        o = _keep(s, "out", lambda: {"logp": new(rows), "entropy": new(rows), "stats": new(2 * rows),
                                     **({"top_ids": new(rows, top, dtype=torch.int32), "top_logp": new(rows, top)} if top else {})})
        P.k_token_logprobs(code, rows, s["vocab"], s["ld"], s["logits"], s["tokens"], s["temp"], top,
                           o["logp"], o["entropy"], o["stats"], o.get("top_ids"), o.get("top_logp"))
        return o
    if op == "logp_bwd":
        o = _keep(s, "out", lambda: {"dlogits": torch.empty_like(s["logits"])})
        P.k_token_logprobs_bwd(code, rows, s["vocab"], s["ld"], s["logits"], s["tokens"], s["temp"], s["stats"],
                               s["entropy"], s["dlogp"], s["dent"], o["dlogits"])
        return o
    if op in ("join", "join_bwd"):
        cols, kind = s["cols"], s["kind"]
        v = {n: s.get(n) for n in ("gain1", "bias1", "gain2", "bias2")}
        if op == "join":
            o = _keep(s, "out", lambda: [new(rows, cols), new(rows, cols, dtype=s["h"].dtype) if s["pre"] else None, new(4 * rows)])
            P.k_join_fwd(code, kind, rows, cols, s["eps"], s["scale"], s["x"], s["h"], v["gain1"], v["bias1"], s["gatev"],
                         s["gate"], v["gain2"], v["bias2"], o[0], o[1], o[2])
            return {"x_out": o[0], "y": o[1], "stats": o[2]}

        def make():
            o = {"dx": new(rows, cols), "dh": new(rows, cols, dtype=s["h"].dtype)}
            if s["gatev"] is not None:
                o["dgate"] = new(*s["gatev"].shape)
            for n in ("gain1", "bias1", "gain2", "bias2"):
                if v[n] is not None:
                    o["d" + n] = new(cols)
            return o
        o = _keep(s, "out", make)
        w = _keep(s, "scratch", lambda: new(P.join_bwd_scratch_bytes(rows, cols, s["gate"]), dtype=torch.uint8))
        P.k_join_bwd(code, kind, rows, cols, s["scale"], s["dy"], s["dxo"], s["xo"], s["h"], s["stats"], v["gain1"], v["bias1"],
                     s["gatev"], s["gate"], v["gain2"], o["dx"], o["dh"], o.get("dgain1"), o.get("dbias1"), o.get("dgate"),
                     o.get("dgain2"), o.get("dbias2"), w)
        return o
    w = _keep(s, "scratch", lambda: new(P.orthogonalize_scratch_bytes(rows, s["cols"]), dtype=torch.uint8))
    if op == "orth":
        o = _keep(s, "out", lambda: new(rows, s["cols"], dtype=torch.bfloat16))
        P.k_orthogonalize(code, rows, s["cols"], s["g"], o, s["steps"], w)
        return {"o": o}
    P.muon_step(rows, s["cols"], s["param"], s["master"], s["grad"], s["mom"], w, steps=s["steps"], nesterov=s["nesterov"], **s["hp"])
    return {"master": s["master"], "momentum": s["mom"], "param": s["param"]}


def run(state):
    if own:
        return _own(state)
    op = state["op"]
    if op == "logp":
        return _logp_plain(state)
    if op == "logp_bwd":
        return _logp_bwd_plain(state)
    if op == "join":
        xo, y, st = _join_plain(state)
        return {"x_out": xo, "y": None if y is None else y.to(state["h"].dtype), "stats": st}
    if op == "join_bwd":
        return _join_bwd_plain(state)
    if op == "orth":
        return {"o": _ns_plain(state["g"], state["steps"]).to(torch.bfloat16)}
    return _muon_plain(state)


# ------------------------------------------------------------------ 64 bits
def _exact_polar(g, steps):
    a, b, c = NS
    x = g.double() / g.double().norm().clamp(min=1e-30)
    for _ in range(steps):                                   # a X + b (X X^T) X + c (X X^T)^2 X, from the short side
        if x.shape[0] <= x.shape[1]:
            left = x @ x.mT
            y = left @ x
            x = a * x + b * y + c * (left @ y)
        else:
            right = x.mT @ x
            y = x @ right
            x = a * x + b * y + c * (y @ right)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    op, rows = case["op"], case["rows"]
    if op == "logp":
        live = s["tokens"] >= 0
        z = s["logits"][:, :case["vocab"]].double()
        peak = z.amax(1)
        q = torch.log_softmax(z / case["temp"], 1)
        ent = torch.where(q.exp() > 0, -q * q.exp(), 0.0).sum(1)
        lsum = torch.logsumexp((z - peak[:, None]) / case["temp"], 1)
        pick = q.take_along_dim(s["tokens"].clamp(min=0).long()[:, None], 1)[:, 0]
        out = {"logp": pick.where(live, 0.0), "entropy": ent.where(live, 0.0), "stats": torch.cat([peak.where(live, 0.0), lsum.where(live, 0.0)])}
        if case["top"]:
            best = torch.full((rows, case["top"]), -math.inf, dtype=torch.float64, device="cuda")
            k = min(case["top"], case["vocab"])
            best[:, :k] = q.topk(k, 1).values.where(live[:, None], -math.inf)
            out["top_ids"], out["top_logp"] = None, best
        return out
    if op == "logp_bwd":
        # derivatives of log p_t and of -sum p log p, through the logits
        z = s["logits"][:, :case["vocab"]].double()
        q = torch.log_softmax(z / case["temp"], 1)
        p = q.exp()
        d = torch.nn.functional.one_hot(s["tokens"].clamp(min=0).long(), case["vocab"]).double()
        d.sub_(p).mul_(s["dlogp"].double()[:, None])
        if s["dent"] is not None:
            pq = torch.where(p > 0, p * q, 0.0)
            d -= s["dent"].double()[:, None] * (pq - p * pq.sum(1, keepdim=True))
        full = torch.zeros(rows, case["ld"], dtype=torch.float64, device="cuda")
        full[:, :case["vocab"]] = torch.where((s["tokens"] >= 0)[:, None], d / case["temp"], 0.0)
        return {"dlogits": full}
    if op in ("join", "join_bwd"):
        # the definition in 64 bits; the gradient by differentiating it
        x, h = s["x"].double(), s["h"].double()
        names = [n for n in ("gain1", "bias1", "gain2", "bias2", "gatev") if s.get(n) is not None]
        v = {n: s[n].double() for n in names}

        def normed(t, gain, bias):
            mu = t.mean(-1, keepdim=True) if case["kind"] == 0 else 0.0
            r = ((t - mu).pow(2).mean(-1, keepdim=True) + s["eps"]).rsqrt()
            t = (t - mu) * r * gain
            return t if bias is None else t + bias, mu, r

        def gated(t):
            return t if "gatev" not in v else t * v["gatev"][torch.arange(rows, device="cuda") // case["gate"]]

        zero = torch.zeros(rows, 1, dtype=torch.float64, device="cuda")
        if op == "join":
            st = [zero] * 4
            if case["post"]:
                h, st[0], st[1] = normed(h, v["gain1"], v.get("bias1"))
            xo, y = case["scale"] * x + gated(h), None
            if case["pre"]:
                y, st[2], st[3] = normed(xo, v["gain2"], v.get("bias2"))
            return {"x_out": xo, "y": y, "stats": torch.cat([(zero + t)[:, 0] for t in st])}
        for t in [h] + list(v.values()):
            t.requires_grad_()
        xo = s["xo"].double().requires_grad_()               # the stream as the forward pass stored it
        d = s["dxo"].double()
        out = {}
        if case["pre"]:
            y = normed(xo, v["gain2"], v.get("bias2"))[0]
            on = [n for n in ("gain2", "bias2") if n in v]
            got = torch.autograd.grad(y, [xo] + [v[n] for n in on], s["dy"].double())
            d = d + got[0]
            out.update({"d" + n: t for n, t in zip(on, got[1:])})
        out["dx"] = case["scale"] * d
        branch = gated(normed(h, v["gain1"], v.get("bias1"))[0] if case["post"] else h)
        on = [n for n in ("gain1", "bias1", "gatev") if n in v]
        got = torch.autograd.grad(branch, [h] + [v[n] for n in on], d)
        out["dh"] = got[0]
        out.update({"dgate" if n == "gatev" else "d" + n: t for n, t in zip(on, got[1:])})
        return out
    if op == "orth":
        return {"o": _exact_polar(s["g"], case["steps"])}
    hp = s["hp"]
    mom = hp["momentum"] * s["mom"].double() + s["grad"].double()
    u = s["grad"].double() + hp["momentum"] * mom if case["nesterov"] else mom
    master = (1 - hp["lr"] * hp["weight_decay"]) * s["master"].double()
    master -= hp["lr"] * 0.2 * math.sqrt(max(rows, case["cols"])) * _exact_polar(u, case["steps"])
    return {"master": master, "momentum": mom, "param": master}
