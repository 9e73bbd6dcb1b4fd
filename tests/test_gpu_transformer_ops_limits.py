"""The block operators beside the step at the ends of their ranges: far tails, the largest values, tiny eps, positions outside the table,
buffers off the 16-byte grid, and the sums over all rows at lengths where a missing part would not show in a norm."""
import math

import pytest

import block_ops_ref as R
from test_gpu_transformer_ops import _dattn_case, _dattn_check, _dattn_run, _types

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def _torch():
    import torch
    return torch


def _unit(code):
    return R.UB if code else R.U32


# ------------------------------------------------------------------ 8 bits
def _act8(code, fmt, kind, pre, dy):
    """Forward and backward: act, the packed values as numbers, scale bytes, dpre, the activation formed again."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    rows, f = dy.shape
    dt, nb = _types(code), -(-f // 32)
    act, again, dpre = (torch.full((rows, n * f), NAN, dtype=dt, device="cuda") for n in (1, 1, kind))
    q, sc = torch.zeros(rows, kind * f, dtype=torch.int8, device="cuda"), torch.zeros(rows, kind * nb, dtype=torch.uint8, device="cuda")
    P.k_act8_fwd(code, fmt, kind, rows, f, pre, act, q, sc)
    P.k_act8_bwd(code, fmt, kind, rows, f, dy, q, sc, dpre, again)
    return act, (q if fmt == 0 else q.view(torch.float8_e4m3fn)).double(), sc, dpre, again


def _near(got, want, err, unit, what):
    """Within err, half a step of the stored type, and the smallest normal fp32."""
    off = (got.double() - want).abs() - err - 1.001 * unit * want.abs() - 2.0 ** -126
    assert bool((off <= 0).all()), (what, float(off.max()), want.flatten()[int(off.argmax())].item())


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("f", [256, 251])
def test_gelu_tail_keeps_its_digits(code, fmt, f):
    """GELU and its derivative from -12 to 12, every value within a bound relative to itself: in 1 + erf(x) nothing is left at a = -5.5.
    Half steps of fp32 in the smaller of cdf and 1 - cdf, exp(-a^2/2) t Q(t): t carries 5 (a product and sum of one rounding, a quick division of two steps), which
    t Q amplifies up to 2.6 times; 6 of Q and its fit; 4 of the quick exponential; its argument three roundings, a^2 / 2 of each; two products.  So 25 + 2 a^2,
    then 2 of the cdf itself and of its product with a."""
    torch = _torch()
    rows = 40
    # rows of like magnitudes, so that the 8 bits keep them apart: -12 .. -0.3, and as far up
    top = torch.linspace(0.3, 12.0, rows, device="cuda")[:, None]
    pre = top * torch.linspace(-1.0, 1.0, f, device="cuda")[None]
    pre = pre.to(_types(code))
    dy = torch.full((rows, f), 0.01, device="cuda").to(_types(code)) * (1 + torch.arange(f, device="cuda") % 3).to(_types(code))
    act, num, sc, dpre, again = _act8(code, fmt, 1, pre, dy)
    kept = R.unpack(num, sc)
    assert float(kept.min()) < -11 and bool(((kept < -5) & (kept > -6)).any())

    def normal(x):                                           # (ndtr is 1 + erf in 64 bits, which loses digits from -7 on)
        low = 0.5 * torch.special.erfc(x.abs() / math.sqrt(2))
        return torch.where(x < 0, low, 1 - low), (25 + 2 * x * x) * low
    for x, got in ((R.f64(pre), act), (kept, again)):
        cdf, half_steps = normal(x)
        _near(got, x * cdf, x.abs() * (half_steps + 3 * cdf) * R.U32, _unit(code), "gelu")
    (cdf, half_steps), pdf = normal(kept), torch.exp(-kept * kept / 2) / math.sqrt(2 * math.pi)
    err = half_steps + 4 * cdf + (12 + 1.5 * kept * kept) * kept.abs() * pdf
    _near(dpre, R.f64(dy) * (cdf + kept * pdf), R.f64(dy) * err * R.U32, _unit(code), "derivative")


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("f", [128, 77])
def test_pack_the_largest_values(code, fmt, f):
    """Blocks whose largest magnitude would round to 2^128 keep the largest code that is finite: what comes back is finite, and off by less than a step."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    dt = _types(code)
    most = float(torch.finfo(dt).max)
    step = 2.0 ** 122 if fmt == 0 else 2.0 ** 124            # of the topmost scale, near 2^128
    vals = [most, -most, 1.9375 * 2.0 ** 127, 1.96875 * 2.0 ** 127, 1.75 * 2.0 ** 127, -1.984375 * 2.0 ** 127, 2.0 ** 127, -1.8125 * 2.0 ** 127, 1e38, 1.0]
    x = torch.zeros(len(vals), f, dtype=dt, device="cuda")
    x[:, ::32] = torch.tensor(vals, dtype=dt, device="cuda")[:, None]
    x[:, 5::32] = torch.tensor(-3e37, dtype=dt, device="cuda")
    x[:, 9] = 1.0
    nb = -(-f // 32)
    q, sc = torch.zeros(len(vals), f, dtype=torch.int8, device="cuda"), torch.zeros(len(vals), nb, dtype=torch.uint8, device="cuda")
    P.k_act8_pack(code, fmt, len(vals), f, x, f, q, sc)
    want, byte = R.pack(R.f64(x), fmt)
    assert torch.equal(sc.long(), byte)
    limit = 63.0 if fmt == 0 else 240.0                      # times 2^(249 - 127), or 2^(247 - 127): the last step below 2^128
    topmost = (byte == (249 if fmt == 0 else 247)).repeat_interleave(32, 1)[:, :f]
    want = torch.where(topmost, want.clamp(-limit, limit), want)
    num = (q if fmt == 0 else q.view(torch.float8_e4m3fn)).double()
    assert torch.equal(num, want) and bool(topmost.any())
    for out_code in (0, 1):
        back = torch.full((len(vals), f), NAN, dtype=_types(out_code), device="cuda")
        P.k_act8_unpack(out_code, fmt, len(vals), f, q, sc, back, f)
        assert bool(back.isfinite().all()) and torch.equal(back.double(), R.unpack(want, byte))
        assert float((back.double() - x.double()).abs().max()) < step
    # through the activations: no infinity or NaN out of finite values
    for kind in (1, 2):
        pre = x if kind == 1 else torch.cat([x, torch.full_like(x, 0.5)], 1)
        act, _, _, dpre, again = _act8(code, fmt, kind, pre.contiguous(), torch.full_like(x, 1e-3))
        assert bool(dpre.isfinite().all()) and bool(again.isfinite().all())


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("f", [64, 45])
def test_swiglu_of_far_negative_gates(code, fmt, f):
    """Gates at which sigmoid(a) is below the smallest normal number, times a large `up`: values that the type can hold are not lost.
    exp(a): 2 (2 + 1.173 |a|) half steps and |a| of its argument's rounding, a division of 4, three products; below 2^-126 half a unit of 2^-149 for each of
    the exponential, the quotient and their products."""
    torch = _torch()
    rows = 6
    a = torch.tensor([-80.0, -88.0, -92.0, -96.0, -60.0, -100.0], device="cuda")[:, None].expand(rows, f).clone()
    a[:, ::5] = -72.0
    u = torch.full((rows, f), 2.0 ** 100, device="cuda")
    u[:, ::3] = -(2.0 ** 98)
    pre = torch.cat([a, u], 1).to(_types(code))
    dy = torch.full((rows, f), 1.0, device="cuda").to(_types(code))
    act, num, sc, dpre, again = _act8(code, fmt, 2, pre, dy)
    tiny = 3 * 2.0 ** -149

    def rel(x):
        return (16 + 4.4 * x.abs()) * R.U32
    kept = R.unpack(num, sc, 2)
    for x, got in ((R.f64(pre), act), (kept, again)):
        g, w = x[:, :f], x[:, f:]
        y = g * torch.sigmoid(g) * w
        assert float(y.abs().min()) > 2.0 ** -60
        _near(got, y, rel(g) * y.abs() + tiny * (1 + g.abs()) * w.abs(), _unit(code), "swiglu")
    g, w = kept[:, :f], kept[:, f:]
    s = torch.sigmoid(g)
    d = w * s * (1 + g * torch.sigmoid(-g))
    _near(dpre[:, :f], d, (rel(g) * w * s * (1 + g.abs())).abs() + tiny * w.abs() * (1 + g.abs()), _unit(code), "gate")
    _near(dpre[:, f:], g * s, rel(g) * (g * s).abs() + tiny * (1 + g.abs()), _unit(code), "up")


# ------------------------------------------------------------------ differential attention
@pytest.mark.parametrize("code,D", [(0, 16), (0, 64), (1, 32), (1, 64), (1, 128)])
@pytest.mark.parametrize("size", [1.0, 1e-20])
@pytest.mark.parametrize("eps", [1e-30, 2e-38])
def test_differential_attention_norm_with_a_tiny_eps(code, D, size, eps):
    """An eps whose power of -3/2 fp32 does not hold: entries of length 0 (rows of zeros) and rows far below sqrt(eps) have the gradients of the formula."""
    torch = _torch()
    B, S, H, K = 3, 70, 2, 1
    s = _dattn_case(code, B, S, H, K, D, True, 31, [70, 0, 33])
    s["qkv"].view(B * S, H + 2 * K, D)[:, H + K:] *= size
    out = _dattn_check(code, B, S, H, K, D, True, s, eps=eps)
    for n in ("dqkv", "dlam", "dgain"):
        assert bool(out[n].isfinite().all()), n
    assert not bool(out["dqkv"][S:2 * S].any())              # the entry of length 0


# ------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (10, 6)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rope_leaves_rows_outside_the_table_as_they_are(code, layout, d, rot, in_place):
    """Bit for bit: infinities, NaN and zeros of either sign beside one another in a pair."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    rows, heads, n_pos = 24, 3, 9
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(rows, heads * d, generator=g, device="cuda")
    odd = torch.tensor([INF, -INF, NAN, -0.0, 0.0, 1.0], device="cuda")
    x = torch.where(torch.rand(x.shape, generator=g, device="cuda") < 0.6, odd[torch.randint(0, 6, x.shape, generator=g, device="cuda")], x).to(_types(code))
    pos = torch.randint(0, n_pos, (rows,), generator=g, device="cuda", dtype=torch.int32)
    out_of = torch.arange(rows, device="cuda") % 4 == 1
    pos[out_of] = torch.tensor([-1, n_pos, 2 ** 31 - 1, -2 ** 31, n_pos + 7, -5], dtype=torch.int32, device="cuda")
    cs = torch.empty(2, n_pos, rot // 2, device="cuda")
    P.rope_table(n_pos, rot, cs)
    bits = torch.int16 if code else torch.int32
    for inverse in (False, True):
        src, bad = x.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        out = src if in_place else torch.empty_like(x)
        P.k_rope(code, layout, rows, heads, d, rot, src, heads * d, out, heads * d, cs, n_pos, positions=pos, inverse=inverse, bad=bad)
        assert torch.equal(out[out_of].view(bits), x[out_of].view(bits)) and int(bad) == 1


def _yarn(n_pos, rot, base, factor, orig_len, fast, slow):
    """Cosines and sines, the ramp's ends found by looking for them: the last whole pair index that turns at least `fast` times over orig_len, the
    first one that turns at most `slow` times."""
    torch = _torch()

    def turns(j):
        return orig_len * base ** (-2.0 * j / rot) / (2 * math.pi)
    wide = range(-4 * rot, 5 * rot)
    lo = max(max((j for j in wide if turns(j) >= fast), default=wide[0]), 0)
    hi = min(min((j for j in wide if turns(j) <= slow), default=wide[-1]), rot - 1)
    f = []
    for j in range(rot // 2):
        share = 1.0 if j >= hi else 0.0 if j <= lo else (j - lo) / (hi - lo)
        f.append(base ** (-2.0 * j / rot) * (1 - share + share / factor))
    ang = torch.arange(n_pos, dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
    return torch.stack([ang.cos(), ang.sin()]) * (1 + 0.1 * math.log(factor))


@pytest.mark.parametrize("orig_len,fast,slow", [(1.0, 32.0, 1.0), (6.0, 32.0, 1.0), (6.5, 32.0, 1.0), (50.0, 9.0, 8.0), (100.0, 32.0, 1.0), (2048.0, 32.0, 1.0), (4096.0, 8.0, 0.5),
                                                (1e6, 2.0, 1.0), (1e9, 32.0, 1.0)])
@pytest.mark.parametrize("rot,base", [(2, 1e4), (8, 1e4), (64, 1e4), (128, 5e5)])
def test_yarn_table_from_its_definition(orig_len, fast, slow, rot, base):
    """Short trained lengths, over which even the first pair turns at most `slow` times, and long ones, over which the last turns `fast` times, among them."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    n_pos, factor = 300, 4.0
    cs = torch.full((2, n_pos, rot // 2), NAN, device="cuda")
    P.rope_table(n_pos, rot, cs, base=base, scaling=P.binding.ROPE_YARN, factor=factor, orig_len=orig_len, fast=fast, slow=slow)
    want = _yarn(n_pos, rot, base, factor, orig_len, fast, slow)
    assert float((cs.double().cpu() - want).abs().max()) <= 1.2 * 2 * R.U32 + 1e-12 * n_pos       # two roundings of values up to 1.14; the angles'


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("norm", [False, True])
def test_differential_attention_gradient_reads_o_and_o2_anywhere(D, norm):
    """The products of the gradient do not read o and o_2: where these start decides nothing, and the results have the same bits."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    B, S, H, K = 2, 150, 4, 2
    s = _dattn_case(1, B, S, H, K, D, norm, 33, [150, 71])
    a = _dattn_run(1, B, S, H, K, D, True, s)
    w = torch.empty(P.diff_attention_bwd_scratch_bytes(1, B, S, H, D, norm), dtype=torch.uint8, device="cuda")

    def off_grid(t):
        n = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape)
        n.copy_(t)
        assert n.data_ptr() % 16 == 2
        return n
    for o, o2 in ((off_grid(a["o"]), a["o2"]), (a["o"], off_grid(a["o2"]))):
        dqkv, dlam = torch.full_like(s["qkv"], NAN), torch.empty(H, device="cuda")
        P.k_diff_attention_bwd(1, B, S, H, K, D, True, s["qkv"], s["lam"], s["gain"], 1e-5, 0.4, o, o2, a["lse"], s["dy"], dqkv, dlam, None, w, key_lens=s["lens"])
        assert torch.equal(dqkv, a["dqkv"]) and torch.equal(dlam, a["dlam"][0])


@pytest.mark.parametrize("code,B,S,H,K,D", [(1, 2, 1500, 24, 6, 128), (1, 1, 9001, 2, 1, 64), (0, 3, 700, 4, 4, 16), (0, 64, 33, 5, 1, 32), (1, 300, 40, 3, 3, 32),
                                            (0, 1, 2000, 1, 1, 128)])
@pytest.mark.parametrize("norm", [False, True])
def test_differential_attention_sums_over_all_rows(code, B, S, H, K, D, norm):
    """dlambda and dgain at lengths of many partial sums, within the roundings that a term meets on its way: those of one thread's terms, of the lanes and rows
    of a block, of the blocks' sums.  That is a small part of the sums themselves, so that no missing part goes by."""
    torch = _torch()
    s = _dattn_case(code, B, S, H, K, D, norm, 35, [S - 3 * (i % 2) for i in range(B)])
    out = _dattn_run(code, B, S, H, K, D, True, s)
    heads = lambda t: R.f64(t).view(B * S, H, D)                                  # noqa: E731
    g, o, o2 = heads(s["dy"]), heads(out["o"]), heads(out["o2"])
    # a block takes at least 32 rows and at most what gives each head ceil(1184 / H) blocks, 256 / (D / 8) rows at a time
    rows = B * S
    per_block = max(32, -(-rows // -(-1184 // H))) + 1
    chunks, at_once = -(-rows // (per_block - 1)), 2048 // D
    turns = -(-per_block // at_once)
    size = g.abs()
    if norm:
        gain = R.f64(s["gain"]) * 0.4
        r = 1 / torch.sqrt((o * o).mean(-1, keepdim=True) + 1e-5)
        t = o * r
        want = (g * t).sum((0, 1)) * 0.4
        # the norm: 8 + 4 terms' sums, a root, a few products: 24 half steps of each term
        bound = (turns + at_once + H * chunks // 128 + 128 + 32) * R.U32 * (g * t).abs().sum((0, 1)) * 0.4
        assert float(bound.max()) <= 0.1 * float(want.abs().mean()), (float(bound.max()), float(want.abs().mean()))
        assert bool(((out["dgain"][0].double() - want).abs() <= bound).all())
        w = g * gain
        size = r * (w.abs() + t.abs() * (w * t).abs().mean(-1, keepdim=True))
        g = r * (w - t * (w * t).mean(-1, keepdim=True))
    want = -(g * o2).sum((0, 2))
    bound = (8 * turns + 4 + at_once + chunks // 1024 + 16 + 24) * R.U32 * (size * o2.abs()).sum((0, 2))
    assert float(bound.max()) <= 0.1 * float(want.abs().mean()), (float(bound.max()), float(want.abs().mean()))
    assert bool(((out["dlam"][0].double() - want).abs() <= bound).all())
