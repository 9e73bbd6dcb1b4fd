"""Cases that time the block operators of this package: rotary positions, differential attention with its gradient, and activations
that keep their inputs in 8 bits for the backward pass.

`run` computes them from elementary torch operations, or, where `own` is true, through the package's entry points.
`exact` states the same operators in 64 bits from their definitions."""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32                          # columns that share a scale
EPS = 1e-5


def listed():
    return [
        # the q and k heads of one token of the LLaMA-shaped model: latency
        {"name": "rope_1_token", "op": "rope", "rows": 1, "heads": 64, "extra": 32, "d": 128, "rot": 128, "layout": 0, "type": "bf16", "packed": False, "seq": 512, "inverse": False},
        # gradient of a long batch with grouped heads, sequences packed behind one another, half of each head rotated in adjacent pairs
        {"name": "rope_bwd_16384_packed", "op": "rope", "rows": 16384, "heads": 40, "extra": 8, "d": 128, "rot": 64, "layout": 1, "type": "bf16", "packed": True, "seq": 4096, "inverse": True},
        # two short sequences of odd length in single precision
        {"name": "dattn_2x131_fp32", "op": "dattn", "batch": 2, "seq": 131, "heads": 4, "kv": 4, "d": 32, "causal": True, "lens": True, "norm": True, "type": "fp32"},
        # the encoder's batch, padded on the right, no causal mask
        {"name": "dattn_16x128_encoder", "op": "dattn", "batch": 16, "seq": 128, "heads": 12, "kv": 12, "d": 64, "causal": False, "lens": True, "norm": False, "type": "bf16"},
        # two long sequences through heads of the LLaMA-shaped model, four query heads to a key head
        {"name": "dattn_2x2048_gqa", "op": "dattn", "batch": 2, "seq": 2048, "heads": 32, "kv": 8, "d": 128, "causal": True, "lens": False, "norm": True, "type": "bf16"},
        # gradients of the first of these
        {"name": "dattn_bwd_2x131_fp32", "op": "dattn_bwd", "batch": 2, "seq": 131, "heads": 4, "kv": 2, "d": 32, "causal": True, "lens": True, "norm": True, "type": "fp32"},
        # a fine-tuning batch of the GPT-2-shaped model, padded on the right
        {"name": "dattn_bwd_8x512", "op": "dattn_bwd", "batch": 8, "seq": 512, "heads": 20, "kv": 20, "d": 64, "causal": True, "lens": True, "norm": False, "type": "bf16"},
        # one very long sequence
        {"name": "dattn_bwd_1x4096", "op": "dattn_bwd", "batch": 1, "seq": 4096, "heads": 16, "kv": 16, "d": 128, "causal": True, "lens": False, "norm": True, "type": "bf16"},
        # the classifier's 16 first tokens kept in 8 bits
        {"name": "act8_pack_16x768_fp32", "op": "act8", "kind": 0, "rows": 16, "f": 768, "format": 0, "type": "fp32"},
        # gated activation of a long batch of the LLaMA-shaped model, gate and up kept as e4m3
        {"name": "act8_swiglu_8192x11008", "op": "act8", "kind": 2, "rows": 8192, "f": 11008, "format": 1, "type": "bf16"},
        # one short example through the GPT-2-shaped feed-forward, single precision
        {"name": "act8_bwd_gelu_37x5120_fp32", "op": "act8_bwd", "kind": 1, "rows": 37, "f": 5120, "format": 0, "type": "fp32", "again": True},
        # gradient of the gated activation of a long batch, its output formed once more for the next weight's gradient
        {"name": "act8_bwd_swiglu_8192x11008", "op": "act8_bwd", "kind": 2, "rows": 8192, "f": 11008, "format": 0, "type": "bf16", "again": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "dattn", "dattn", "dattn_bwd", "dattn_bwd", "act8", "act8_bwd"])
    kind = rng.choice(["fp32", "bf16"]) if not op.startswith("dattn") else rng.choice(["fp32", "bf16", "bf16"])
    if op == "rope":
        d = rng.choice([32, 64, 80, 128])
        heads = _log_int(rng, 1, 96)
        rows = _log_int(rng, 1, min(16384, (1 << 26) // (heads * d)))
        return {"op": op, "rows": rows, "heads": heads, "extra": rng.choice([0, heads // 2]), "d": d, "rot": rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)]),
                "layout": rng.randint(0, 1), "type": kind, "packed": rng.random() < 0.5, "seq": rng.choice([512, 1000, 4096]), "inverse": rng.random() < 0.5}
    if op.startswith("dattn"):
        d = rng.choice([32, 64, 128]) if kind == "fp32" else rng.choice([64, 128])
        most = 1 << 24 if kind == "fp32" else 1 << 28           # scores of one map
        seq = _log_int(rng, 1, 1024 if kind == "fp32" else 4096)
        kv = _log_int(rng, 1, 16)
        heads = kv * rng.choice([1, 1, 2, 4])
        batch = _log_int(rng, 1, max(1, min(16, most // (heads * seq * seq))))
        while batch * heads * seq * seq > most:
            heads, kv = max(1, heads // kv), 1
            seq = min(seq, int(math.sqrt(most / (batch * heads))))
        return {"op": op, "batch": batch, "seq": seq, "heads": heads, "kv": kv, "d": d, "causal": rng.random() < 0.6,
                "lens": rng.random() < 0.4, "norm": rng.random() < 0.6, "type": kind}
    f = _log_int(rng, 1, 12000)
    case = {"op": op, "kind": rng.randint(0, 2), "rows": _log_int(rng, 1, min(16384, 8192 * 11008 // (f * (2 if kind == "fp32" else 1)))), "f": f,
            "format": rng.randint(0, 1), "type": kind}
    return case if op == "act8" else dict(case, again=rng.random() < 0.5)


def work(case):
    op = case["op"]
    es = 2 if case["type"] == "bf16" else 4
    if op == "rope":
        n = case["rows"] * case["heads"] * case["d"]
        return {"bytes": 2 * n * es + min(case["rows"], case["seq"]) * case["rot"] * 4 + 4 * case["rows"] * case["packed"], "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    if op.startswith("dattn"):
        B, S, H, K, D = (case[n] for n in ("batch", "seq", "heads", "kv", "d"))
        pairs = B * H * (S * (S + 1) // 2 if case["causal"] else S * S)
        tok, sets = B * S, 3 if case["norm"] else 2
        if op == "dattn":
            return {"bytes": tok * D * es * (H + 2 * K + sets * H) + 8 * B * H * S, "flops": 6 * D * pairs}
        return {"bytes": tok * D * es * (2 * (H + 2 * K) + 3 * H) + 8 * B * H * S, "flops": 10 * D * pairs}
    n, two = case["rows"] * case["f"], 2 if case["kind"] == 2 else 1
    packed = two * (n + case["rows"] * (-(-case["f"] // BLOCK)))
    if op == "act8":
        return {"bytes": n * es * two + packed + (n * es if case["kind"] else 0), "flops": 12 * n}
    grads = n * es * (1 + two) if case["kind"] else n * es
    return {"bytes": packed + grads + (n * es if case["kind"] and case["again"] else 0), "flops": 20 * n}


def _lens(g, batch, seq):
    return torch.randint(max(1, seq // 2), seq + 1, (batch,), generator=g, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device="cuda") * std + mean

    s = dict(case)
    op, dt = case["op"], TYPES[case["type"]]
    if op == "rope":
        rows, d, rot, seq = case["rows"], case["d"], case["rot"], case["seq"]
        s["ld"] = (case["heads"] + case["extra"]) * d
        s["x"] = normal(rows, s["ld"]).to(dt)
        angle = torch.arange(seq, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device="cuda").double() / rot)
        s["cs"] = torch.stack([angle.cos(), angle.sin()]).float().contiguous()          # cosines, then sines
        if case["packed"]:                                     # positions start again where a sequence does
            start = torch.randint(0, seq, (1,), generator=g, device="cuda")
            s["positions"] = ((torch.arange(rows, device="cuda") + start) % max(1, seq - 7)).to(torch.int32)
        else:
            s["positions"] = None
        return s
    if op.startswith("dattn"):
        B, S, H, K, D = (case[n] for n in ("batch", "seq", "heads", "kv", "d"))
        x = normal(B * S, (H + 2 * K) * D)
        x[:, : (H + K) * D] *= 1.5                             # scores that prefer some keys
        s["qkv"] = x.to(dt)
        s["lam"] = normal(H, std=0.1, mean=0.6)
        s["gain"] = normal(D, std=0.1, mean=1.0).to(dt) if case["norm"] else None
        s["c"] = 0.4
        s["key_lens"] = _lens(g, B, S) if case["lens"] else None
        if op == "dattn_bwd":
            s["dy"] = normal(B * S, H * D, std=1e-2).to(dt)
            # what the forward pass leaves
            o, o2, lse, _ = _dattn_forward(s, torch.float32)
            s["o"], s["o2"], s["lse"] = o.to(dt), o2.to(dt), lse.float()
        return s
    rows, f = case["rows"], case["f"]
    two = 2 if case["kind"] == 2 else 1
    # pre-activations: a spread of columns, a few columns far larger than the rest
    x = normal(rows, two * f) * (0.5 + normal(two * f).abs())
    x[:, torch.randint(0, two * f, (max(1, f // 500),), generator=g, device="cuda")] *= 20.0
    if op == "act8":
        s["x"] = x.to(dt)
        return s
    s["q"], s["scales"] = _pack(x.to(dt), two, case["format"])
    s["dy"] = normal(rows, f, std=1e-2).to(dt)
    return s


# ------------------------------------------------------------------ plain forms
def _rope_plain(s):
    heads, d, rot = s["heads"], s["d"], s["rot"]
    x = s["x"][:, : heads * d].float().view(-1, heads, d)
    pos = torch.arange(s["rows"], device="cuda") % s["seq"] if s["positions"] is None else s["positions"].long()
    c, n = s["cs"][0][pos][:, None], s["cs"][1][pos][:, None]
    n = -n if s["inverse"] else n
    r = x[..., :rot]
    a, b = (r[..., : rot // 2], r[..., rot // 2:]) if s["layout"] == 0 else (r[..., 0::2], r[..., 1::2])
    a, b = a * c - b * n, b * c + a * n
    r = torch.cat([a, b], -1) if s["layout"] == 0 else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([r, x[..., rot:]], -1).to(s["x"].dtype).view(-1, heads * d)


def _split(s, dt):
    """q, k [2 maps, batch, heads, seq, d / 2], v [batch, heads, seq, d], the keys' heads repeated."""
    B, S, H, K, D = (s[n] for n in ("batch", "seq", "heads", "kv", "d"))
    q, k, v = s["qkv"].to(dt).view(B, S, H + 2 * K, D).transpose(1, 2).split([H, K, K], 1)
    k, v = k.repeat_interleave(H // K, 1), v.repeat_interleave(H // K, 1)
    return q.unflatten(3, (2, D // 2)).movedim(3, 0), k.unflatten(3, (2, D // 2)).movedim(3, 0), v


def _hidden(s):
    """True where a query may not see a key; [batch or 1, 1, seq, seq]."""
    i = torch.arange(s["seq"], device="cuda")
    hide = (i[None, :] > i[:, None])[None, None] if s["causal"] else torch.zeros(1, 1, 1, s["seq"], dtype=torch.bool, device="cuda")
    return hide if s["key_lens"] is None else hide | (i[None, :] >= s["key_lens"][:, None])[:, None, None]


def _rows(t):
    """[batch, heads, seq, d] as rows of heads."""
    return t.transpose(1, 2).flatten(2).flatten(0, 1)


def _dattn_forward(s, dt):
    q, k, v = _split(s, dt)
    x = (q @ k.mT).mul_((s["d"] // 2) ** -0.5).masked_fill_(_hidden(s), -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    om = (x @ v).div_(total)
    o = om[0] - s["lam"].to(dt)[:, None, None] * om[1]
    y = None
    if s["norm"]:
        y = _rows(o * torch.rsqrt((o * o).mean(-1, keepdim=True) + EPS) * (s["gain"].to(dt) * s["c"]))
    return _rows(o), _rows(om[1]), (top + total.log())[..., 0], y


def _dattn_plain(s):
    o, o2, lse, y = _dattn_forward(s, torch.float32)
    dt = s["qkv"].dtype
    return {"o": o.to(dt), "o2": o2.to(dt), "lse": lse, "y": None if y is None else y.to(dt)}


def _heads_of(t, s):
    return t.float().view(s["batch"], s["seq"], s["heads"], s["d"]).transpose(1, 2)


def _dattn_bwd_plain(s):
    B, S, H, K, D = (s[n] for n in ("batch", "seq", "heads", "kv", "d"))
    q, k, v = _split(s, torch.float32)
    lam = s["lam"][:, None, None]
    g, o, o2 = _heads_of(s["dy"], s), _heads_of(s["o"], s), _heads_of(s["o2"], s)
    out = {}
    if s["norm"]:
        w = g * (s["gain"].float() * s["c"])
        r = torch.rsqrt((o * o).mean(-1, keepdim=True) + EPS)
        out["dgain"] = (g * o * r).sum((0, 1, 2), dtype=torch.float64).mul_(s["c"]).float()
        g = r * (w - o * (r * r * (w * o).mean(-1, keepdim=True)))
    d2 = (g * o2).sum(-1, keepdim=True)
    d1 = (g * (o + lam * o2)).sum(-1, keepdim=True)
    out["dlam"] = -d2.sum((0, 2, 3), dtype=torch.float64).float()
    p = (q @ k.mT).mul_((D // 2) ** -0.5).masked_fill_(_hidden(s), -math.inf).sub_(s["lse"][..., None]).exp_()
    dv = (p[0] - lam * p[1]).mT @ g
    dp = g @ v.mT
    p[0].mul_(dp - d1)
    p[1].mul_(dp.sub_(d2)).mul_(-lam)
    p.mul_((D // 2) ** -0.5)
    dq, dk = p @ k, p.mT @ q
    whole = [t.movedim(0, 3).flatten(3) for t in (dq, dk)] + [dv]
    whole[1:] = [t.view(B, K, H // K, S, D).sum(2) for t in whole[1:]]
    out["dqkv"] = torch.cat(whole, 1).transpose(1, 2).reshape(B * S, -1).to(s["qkv"].dtype)
    return out


def _blocks(x, two):
    """[rows, two halves, blocks, 32], padded with zeros."""
    f = x.shape[1] // two
    return torch.nn.functional.pad(x.view(-1, two, f), (0, -f % BLOCK)).unflatten(2, (-1, BLOCK))


def _power(e):
    """2 ** e as fp32, from its bits: pow() may be a rounding off, which breaks ties."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _pack(x, two, form):
    """8-bit values and scale bytes: 2 ** (byte - 127) is the least power of two that brings a block into the range, 2 ** -110 at least."""
    b = _blocks(x.float(), two)
    most = 448.0 if form else 127.0
    top = b.abs().amax(-1)
    m, e = torch.frexp(top)                                   # top = m 2^e, m in [0.5, 1)
    head, shift = (0.875, 9) if form else (127.0 / 128.0, 7)  # most = head 2^shift
    e = torch.where(m > head, e - shift + 1, e - shift)
    e = torch.where(top == 0, -110, e).clamp(min=-110)
    v = (b * _power(-e[..., None])).clamp(-most, most)
    q = v.to(torch.float8_e4m3fn) if form else v.round().to(torch.int8)
    return q.flatten(2)[..., : x.shape[1] // two].reshape(x.shape).contiguous(), (e + 127).to(torch.uint8).view(x.shape[0], -1)


def _unpack(s, dt):
    two = 2 if s["kind"] == 2 else 1
    b = _blocks(s["q"].to(dt), two)
    scale = _power(s["scales"].int().view(s["rows"], two, -1, 1) - 127)
    return (b * scale.to(dt)).flatten(2)[..., : s["f"]]


def _act8_plain(s):
    x, f = s["x"].float(), s["f"]
    q, scales = _pack(s["x"], 2 if s["kind"] == 2 else 1, s["format"])
    out = {"q": q, "scales": scales}
    if s["kind"] == 1:
        out["y"] = (0.5 * x * torch.special.erfc(-x * math.sqrt(0.5))).to(s["x"].dtype)
    elif s["kind"] == 2:
        out["y"] = (x[:, :f] * torch.sigmoid(x[:, :f]) * x[:, f:]).to(s["x"].dtype)
    return out


def _act8_bwd_plain(s):
    x, dt = _unpack(s, torch.float32), s["dy"].dtype
    if s["kind"] == 0:
        return {"x": x[:, 0].to(dt)}
    g = s["dy"].float()
    if s["kind"] == 1:
        x = x[:, 0]
        cdf = 0.5 * torch.special.erfc(-x * math.sqrt(0.5))
        out = {"dx": (g * (cdf + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2 * math.pi)))).to(dt)}
        y = x * cdf
    else:
        a, u = x[:, 0], x[:, 1]
        sig = torch.sigmoid(a)
        out = {"dx": torch.cat([g * u * sig * (1 + a * torch.sigmoid(-a)), g * a * sig], 1).to(dt)}
        y = a * sig * u
    return dict(out, y=y.to(dt)) if s["again"] else out


# ------------------------------------------------------------------ the framework's calls
def _keep(s, name, make):
    if name not in s:
        s[name] = make()
    return s[name]


def _own(s):
    import paper_2401_15207_b200 as P
    op, dt = s["op"], TYPES[s["type"]]
    code = 1 if s["type"] == "bf16" else 0

    def new(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if op == "rope":
        o = _keep(s, "out", lambda: new(s["rows"], s["heads"] * s["d"], dtype=dt))
        P.k_rope(code, s["layout"], s["rows"], s["heads"], s["d"], s["rot"], s["x"], s["ld"], o, s["heads"] * s["d"], s["cs"], s["seq"],
                 positions=s["positions"], inverse=s["inverse"])
        return o
    if op.startswith("dattn"):
        B, S, H, K, D = (s[n] for n in ("batch", "seq", "heads", "kv", "d"))
        args = (code, B, S, H, K, D, s["causal"], s["qkv"], s["lam"], s["gain"], EPS, s["c"])
        if op == "dattn":
            o = _keep(s, "out", lambda: {"o": new(B * S, H * D, dtype=dt), "o2": new(B * S, H * D, dtype=dt), "lse": new(2, B, H, S),
                                         "y": new(B * S, H * D, dtype=dt) if s["norm"] else None})
            P.k_diff_attention_fwd(*args, o["o"], o["o2"], o["y"], o["lse"], key_lens=s["key_lens"])
            return o
        o = _keep(s, "out", lambda: {**({"dgain": new(D)} if s["norm"] else {}), "dlam": new(H), "dqkv": torch.empty_like(s["qkv"])})
        w = _keep(s, "scratch", lambda: new(P.diff_attention_bwd_scratch_bytes(code, B, S, H, D, s["norm"]), dtype=torch.uint8))
        P.k_diff_attention_bwd(*args, s["o"], s["o2"], s["lse"], s["dy"], o["dqkv"], o["dlam"], o.get("dgain"), w, key_lens=s["key_lens"])
        return o
    rows, f, kind, form = s["rows"], s["f"], s["kind"], s["format"]
    two = 2 if kind == 2 else 1
    if op == "act8":
        o = _keep(s, "out", lambda: {"q": new(rows, two * f, dtype=torch.float8_e4m3fn if form else torch.int8),
                                     "scales": new(rows, two * -(-f // BLOCK), dtype=torch.uint8), **({"y": new(rows, f, dtype=dt)} if kind else {})})
        if kind == 0:
            P.k_act8_pack(code, form, rows, f, s["x"], f, o["q"], o["scales"])
        else:
            P.k_act8_fwd(code, form, kind, rows, f, s["x"], o["y"], o["q"], o["scales"])
        return o
    if kind == 0:
        o = _keep(s, "out", lambda: {"x": new(rows, f, dtype=dt)})
        P.k_act8_unpack(code, form, rows, f, s["q"], s["scales"], o["x"], f)
        return o
    o = _keep(s, "out", lambda: {"dx": new(rows, two * f, dtype=dt), **({"y": new(rows, f, dtype=dt)} if s["again"] else {})})
    P.k_act8_bwd(code, form, kind, rows, f, s["dy"], s["q"], s["scales"], o["dx"], o.get("y"))
    return o


def run(state):
    if own:
        return _own(state)
    return {"rope": _rope_plain, "dattn": _dattn_plain, "dattn_bwd": _dattn_bwd_plain, "act8": _act8_plain, "act8_bwd": _act8_bwd_plain}[state["op"]](state)


# ------------------------------------------------------------------ 64 bits
def _exact_maps(s):
    """For each map: scale, q, k (keys' heads repeated), scores in 64 bits; and v."""
    B, S, H, K, D = (s[n] for n in ("batch", "seq", "heads", "kv", "d"))
    x = s["qkv"].double().view(B, S, -1, D)
    group = torch.arange(H, device="cuda") // (H // K)
    q, k, v = x[:, :, :H], x[:, :, H:H + K][:, :, group], x[:, :, H + K:][:, :, group]
    seen = torch.ones(B, 1, S, S, dtype=torch.bool, device="cuda")
    if s["causal"]:
        seen = seen.tril()
    if s["key_lens"] is not None:
        seen = seen & (torch.arange(S, device="cuda") < s["key_lens"][:, None])[:, None, None]
    for m in range(2):
        a, b = q[..., m * D // 2:(m + 1) * D // 2], k[..., m * D // 2:(m + 1) * D // 2]
        z = torch.einsum("bihd,bjhd->bhij", a, b) / math.sqrt(D / 2)
        yield a, b, v, torch.where(seen, z, -math.inf)


def _exact_dattn(s):
    o, lse = [], []
    for _, _, v, z in _exact_maps(s):
        lse.append(torch.logsumexp(z, -1))
        o.append(torch.einsum("bhij,bjhd->bihd", torch.softmax(z, -1), v))
    full = o[0] - s["lam"].double()[:, None] * o[1]
    y = None
    if s["norm"]:
        y = full / torch.sqrt(full.pow(2).mean(-1, keepdim=True) + EPS) * s["gain"].double() * s["c"]
        y = y.reshape(len(s["qkv"]), -1)
    return {"o": full.reshape(len(s["qkv"]), -1), "o2": o[1].reshape(len(s["qkv"]), -1), "lse": torch.stack(lse), "y": y}


def _exact_dattn_bwd(s):
    B, S, H, K, D = (s[n] for n in ("batch", "seq", "heads", "kv", "d"))
    shape = (B, S, H, D)
    g, o, o2, lam = (s[n].double() for n in ("dy", "o", "o2", "lam"))
    g, o, o2 = g.view(shape), o.view(shape), o2.view(shape)
    out = {}
    if s["norm"]:                                             # by differentiating the norm
        o, gain = o.detach().requires_grad_(), s["gain"].double().requires_grad_()
        y = o / torch.sqrt(o.pow(2).mean(-1, keepdim=True) + EPS) * gain * s["c"]
        g, out["dgain"] = torch.autograd.grad(y, [o, gain], g)
        o = o.detach()
    out["dlam"] = -torch.einsum("bihd,bihd->h", g, o2)
    dqkv = torch.zeros(B, S, H + 2 * K, D, dtype=torch.float64, device="cuda")
    group = torch.arange(H, device="cuda") // (H // K)
    weight = [torch.ones_like(lam), -lam]
    held = [o + lam[:, None] * o2, o2]
    for m, (q, k, v, z) in enumerate(_exact_maps(s)):
        at = slice(m * D // 2, (m + 1) * D // 2)
        p = torch.exp(z - s["lse"][m].double()[..., None]) * weight[m][:, None, None]
        del z
        dqkv[:, :, H + K:].index_add_(2, group, torch.einsum("bhij,bihd->bjhd", p, g))
        dz = p * (torch.einsum("bihd,bjhd->bhij", g, v) - torch.einsum("bihd,bihd->bhi", g, held[m])[..., None]) / math.sqrt(D / 2)
        dqkv[:, :, :H, at] = torch.einsum("bhij,bjhd->bihd", dz, k)
        dqkv[:, :, H:H + K, at].index_add_(2, group, torch.einsum("bhij,bihd->bjhd", dz, q))
    out["dqkv"] = dqkv.view(B * S, -1)
    return out


def _exact_unpacked(s):
    n, f = (2 if s["kind"] == 2 else 1), s["f"]
    col = torch.arange(n * f, device="cuda")
    byte = s["scales"][:, col // f * -(-f // BLOCK) + col % f // BLOCK]
    return s["q"].double() * ((byte.long() - 127 + 1023) << 52).view(torch.float64)


def _exact_packed(x, f, form):
    """The 8-bit values, from the quotients by the blocks' powers of two."""
    rows, cols = x.shape
    x = x.double()
    top = torch.zeros(rows, cols // f, -(-f // BLOCK), dtype=torch.float64, device="cuda")
    col = torch.arange(cols, device="cuda")
    block = (col // f * top.shape[2] + col % f // BLOCK).expand(rows, -1)
    top = top.flatten(1).scatter_reduce_(1, block, x.abs(), "amax")
    m, e = torch.frexp(top / (448.0 if form else 127.0))
    def power(k):                                             # its bits in 64
        return ((k.long() + 1023) << 52).view(torch.float64)

    v = x / power(torch.where(m == 0.5, e - 1, e).clamp(min=-110)).gather(1, block)
    step = power(torch.frexp(v).exponent.clamp(min=-5) - 4) if form else 1.0
    return (v / step).round() * step


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rope":
        x = s["x"].double()[:, : case["heads"] * case["d"]].reshape(case["rows"], case["heads"], case["d"])
        pos = torch.arange(case["rows"], device="cuda") % case["seq"] if s["positions"] is None else s["positions"].long()
        i = torch.arange(case["rot"] // 2, device="cuda")
        first, second = (i, i + case["rot"] // 2) if case["layout"] == 0 else (2 * i, 2 * i + 1)
        angle = pos.double()[:, None] * 10000.0 ** (-2.0 * i.double() / case["rot"])
        turn = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)[:, None]
        z = torch.complex(x[..., first], x[..., second]) * turn
        out = x.clone()
        out[..., first], out[..., second] = z.real, z.imag
        return out.reshape(case["rows"], -1)
    if op == "dattn":
        return _exact_dattn(s)
    if op == "dattn_bwd":
        return _exact_dattn_bwd(s)
    f, kind = case["f"], case["kind"]
    normal = torch.distributions.Normal(torch.zeros((), dtype=torch.float64, device="cuda"), 1.0)
    if op == "act8":
        x = s["x"].double()
        out = {"q": _exact_packed(s["x"], f, case["format"]), "scales": None}
        if kind == 1:
            out["y"] = x * torch.special.ndtr(x)
        elif kind == 2:
            out["y"] = torch.nn.functional.silu(x[:, :f]) * x[:, f:]
        return out
    x, g = _exact_unpacked(s), s["dy"].double()
    if kind == 0:
        return {"x": x}
    if kind == 1:
        y = x * torch.special.ndtr(x)
        out = {"dx": g * (torch.special.ndtr(x) + x * normal.log_prob(x).exp())}
    else:
        x.requires_grad_()
        y = torch.nn.functional.silu(x[:, :f]) * x[:, f:]
        out = {"dx": torch.autograd.grad(y, x, g)[0]}
        y = y.detach()
    return dict(out, y=y) if case["again"] else out
