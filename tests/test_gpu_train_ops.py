"""The operators beside the step against their 64-bit definitions: token log-probabilities, the residual junction and the
orthogonalised update, forward and backward, at the sizes, masks and layouts where they can go wrong."""
import numpy as np
import pytest

import train_ops_ref as R
from gpu_util import U_BF16, assert_elem, rel_l2

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def _torch():
    import torch
    return torch


def _dt(code):
    return _torch().bfloat16 if code else _torch().float32


def _half_step(code):
    return U_BF16 if code else R.U32


def _dev(a, dtype=None):
    t = _torch().from_numpy(np.array(a, copy=True)).cuda()
    return t if dtype is None else t.to(dtype)


class Guarded:
    """An output tensor inside a larger one whose other bytes must keep their value."""

    def __init__(self, shape, dtype, shift=0):
        torch = _torch()
        n = int(np.prod(shape))
        self.n, self.lo = n, 64 + shift
        self.whole = torch.full((n + 128 + shift,), 77.0 if dtype.is_floating_point else 77, dtype=dtype, device="cuda")
        self.t = self.whole[self.lo:self.lo + n].view(*shape)

    def np(self):
        assert bool((self.whole[:self.lo] == 77).all()) and bool((self.whole[self.lo + self.n:] == 77).all()), "written outside the output"
        t = self.t
        return (t.double() if t.is_floating_point() else t).cpu().numpy()


# ------------------------------------------------------------------ token log-probabilities
def _logits(rows, vocab, ld, code, shift, seed, std=2.0):
    """Rows of logits in a buffer that starts `shift` elements past an aligned address; returns (tensor, fp64 image)."""
    torch = _torch()
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, ld)) * std
    flat = torch.zeros(rows * ld + shift + 8, dtype=_dt(code), device="cuda")
    t = flat[shift:shift + rows * ld].view(rows, ld)
    t.copy_(_dev(x).to(t.dtype))
    return t, t[:, :vocab].double().cpu().numpy()


def _run_logp(t, tok, vocab, temp, top, code, flag=None, shift=0):
    from paper_2401_15207_b200 import k_token_logprobs
    torch = _torch()
    rows, ld = t.shape
    f, i = torch.float32, torch.int32
    logp, ent, st = Guarded((rows,), f, shift), Guarded((rows,), f, shift), Guarded((2, rows), f, shift)
    ids, vals = (Guarded((rows, top), i, shift), Guarded((rows, top), f, shift)) if top else (None, None)
    k_token_logprobs(code, rows, vocab, ld, t, _dev(np.asarray(tok, np.int32)), temp, top, logp.t, ent.t, st.t,
                     ids.t if top else None, vals.t if top else None, flag)
    torch.cuda.synchronize()
    return logp.np(), ent.np(), st.np(), ids.np() if top else None, vals.np() if top else None


def _logp_slack(x, temp, st):
    """What fp32 arithmetic may put on log p, L and H of a row, absolute.  t = (x - m) / T carries three roundings; the
    exponential sees |t| log2 e rounded twice more and is itself good to 2^-22; a sum of V positive terms, taken by one
    thread in runs of V / 128 at most and then by trees (the tail of the runs is shorter than V), is off by (V / 128 + 20) 2^-24.
    Through L = log1p(r) relative errors of r count at most once, weighted by p."""
    rows, vocab = x.shape
    out = np.zeros(rows)
    for r in range(rows):
        m = x[r].max()
        if not np.isfinite(m):
            continue
        t = (x[r][np.isfinite(x[r])] - m) / temp
        p = np.exp(t - st[1, r])
        out[r] = 2.0 ** -22 + R.U32 * (vocab / 128 + 20) + 8 * R.U32 * (p * np.abs(t)).sum()
    return out


def _check_logp(got, x, tok, temp, top, what=""):
    logp, ent, st, ids, vals = got
    rl, re, rs, ri, rv = R.token_logprobs(x, tok, temp, top)
    # the outputs are fp32: lowest / 0.7 lies beyond its range and is -inf there
    rl, rv = (np.where(a < -float(np.finfo(np.float32).max), -np.inf, a) for a in (rl, rv))
    with np.errstate(invalid="ignore", over="ignore"):
        sl = _logp_slack(np.where(np.isnan(x), -np.inf, x), temp, rs)
    for g, ref, s, n in ((logp, rl, sl, "logp"), (st[0], rs[0], 0, "max"), (st[1], rs[1], sl, "L"),
                         (ent, re, sl * (1 + np.abs(re)) + 8 * R.U32 * np.abs(re), "entropy")):
        fin = np.isfinite(ref)
        assert np.array_equal(np.isnan(g), np.isnan(ref)) and np.array_equal(np.isneginf(g), np.isneginf(ref)), (what, n, g, ref)
        assert_elem(g[fin], ref[fin], 6 * R.U32, s[fin] if np.ndim(s) else 0.0, f"{what} {n}")
    if top:
        assert np.array_equal(ids, ri), (what, ids, ri)
        fin = np.isfinite(rv)
        assert np.array_equal(np.isnan(vals), np.isnan(rv)) and np.array_equal(np.isneginf(vals), np.isneginf(rv)), what
        assert_elem(vals[fin], rv[fin], 6 * R.U32, np.broadcast_to(sl[:, None], rv.shape)[fin], f"{what} alternatives")


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("rows,vocab,ld,shift,top,temp", [
    (1, 1, 1, 0, 3, 1.0), (2, 2, 2, 1, 1, 0.7), (5, 7, 9, 3, 20, 1.5), (3, 31, 31, 0, 32, 1.0), (4, 64, 64, 0, 0, 1.0),
    (33, 257, 264, 2, 5, 0.7), (7, 1000, 1003, 5, 8, 1.0), (2, 4095, 4095, 1, 32, 1.0), (1, 4097, 4104, 0, 1, 2.0),
    (9, 32000, 32000, 0, 5, 1.0), (1, 32000, 32001, 1, 20, 0.7), (3, 50257, 50257, 7, 8, 1.0), (160, 50257, 50264, 0, 2, 1.0),
    (1, 131072, 131072, 0, 32, 1.0), (2, 262147, 262147, 3, 5, 1.0), (700, 130, 130, 1, 4, 1.0)])
def test_logprobs_match_the_definition(code, rows, vocab, ld, shift, top, temp):
    t, x = _logits(rows, vocab, ld, code, shift, seed=rows + vocab)
    rng = np.random.default_rng(vocab)
    tok = rng.integers(0, vocab, rows)
    tok[::7] = x[::7].argmax(1)                     # some sure tokens
    if rows > 2:
        tok[1] = -1
    _check_logp(_run_logp(t, tok, vocab, temp, top, code, shift=shift % 4), x, tok, temp, top)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("vocab", [40, 1000, 9000, 40000])
def test_logprobs_masks_ties_and_bad_rows(code, vocab):
    torch = _torch()
    rows, top = 19, 9
    t, _ = _logits(rows, vocab, vocab, code, 0, seed=vocab)
    lowest = torch.finfo(t.dtype).min
    tok = np.arange(rows) % vocab
    t[0] = -INF                                     # nothing left
    t[1] = lowest                                   # the type's lowest value everywhere: uniform
    t[2, :] = -INF
    t[2, vocab - 1] = 3.0                           # one token left; the given one cannot occur
    t[3] = 1.25                                     # all equal: the lowest ids win
    t[4, 5] = NAN
    t[5, vocab - 2] = INF
    t[6, 5] = NAN
    tok[6] = -1                                     # an ignored row may hold anything
    t[7, ::2] = -INF
    t[8] = lowest
    t[8, 11] = 0.5
    t[9] = 0.0
    t[9, 1::2] = -0.0                               # zeros of both signs are equal
    t[10] = torch.round(t[10])                      # many ties
    t[11, 3] = 60.0                                 # nearly sure
    tok[11] = 3
    t[12] *= 3000.0                                 # far apart
    t[13] = t[13] * 0.01 + 10000.0                  # large and close
    tok[14] = vocab                                 # no such token
    tok[15] = 2 ** 31 - 1
    t[16] = -INF
    t[16, 7] = NAN
    t[17, :vocab - 8] = -INF                        # fewer left than asked for
    t[18] = torch.finfo(t.dtype).max
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = t.double().cpu().numpy()
    got = _run_logp(t, tok, vocab, 0.7, top, code, flag)
    # row 18: all at the type's largest value is a uniform row
    _check_logp(got, x, tok, 0.7, top)
    assert int(flag) == 1
    flag.zero_()
    tok[14] = tok[15] = -1
    _run_logp(t, tok, vocab, 0.7, top, code, flag)
    assert int(flag) == 0


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("stride", [1, 2, 31, 128, 256, 512, 1024, 2048, 4096])
def test_logprobs_alternatives_that_one_thread_holds(code, stride):
    """The largest logits a fixed distance apart: side by side, or in different loads of one and the same thread."""
    from paper_2401_15207_b200 import k_token_logprobs
    torch = _torch()
    rows, vocab, n = 600, 90000, 20                  # enough rows for one block each
    t, _ = _logits(rows, vocab, vocab, code, 0, seed=stride)
    t.clamp_(max=3.0)
    first = np.arange(rows) * 5 % 7001
    ids = first[:, None] + stride * np.arange(n)[None]
    order = np.argsort(np.random.default_rng(stride).random((rows, n)), axis=1)
    t.scatter_(1, _dev(ids.astype(np.int64)), _dev((8.0 + 0.5 * order).astype(np.float32)).to(t.dtype))
    e = lambda *s, d=torch.float32: torch.empty(*s, dtype=d, device="cuda")  # noqa: E731
    lp, en, st, got, val = e(rows), e(rows), e(2 * rows), e(rows, n + 3, d=torch.int32), e(rows, n + 3)
    k_token_logprobs(code, rows, vocab, vocab, t, _dev(ids[:, 0].astype(np.int32)), 1.0, n + 3, lp, en, st, got, val)
    want = np.take_along_axis(ids, np.argsort(-order, axis=1), axis=1)
    assert np.array_equal(got.cpu().numpy()[:, :n], want)
    rest = torch.topk(t.float().scatter(1, _dev(ids.astype(np.int64)), -INF), 3, dim=1).values
    assert torch.equal(torch.gather(t.float(), 1, got[:, n:].long()), rest)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("vocab,ld", [(2001, 2001), (8100, 8104), (16001, 16001)])
def test_logprobs_of_many_short_rows(code, vocab, ld):
    """Rows enough to fill the GPU with small blocks.  A thread's run of a sum is up to V / 64 terms there: V / 128 roundings more."""
    rows, top = 8192, 6
    t, _ = _logits(rows, vocab, ld, code, 1, seed=vocab)
    tok = np.random.default_rng(vocab).integers(0, vocab, rows)
    logp, ent, st, ids, vals = _run_logp(t, tok, vocab, 0.9, top, code)
    some = np.r_[0:16, 4000:4016, rows - 16:rows]
    x = t[some][:, :vocab].double().cpu().numpy()
    rl, re, rs, ri, rv = R.token_logprobs(x, tok[some], 0.9, top)
    sl = _logp_slack(x, 0.9, rs) + R.U32 * vocab / 128
    assert np.array_equal(ids[some], ri) and np.array_equal(st[0, some], rs[0].astype(np.float32))
    for g, ref, s in ((logp[some], rl, sl), (st[1, some], rs[1], sl), (ent[some], re, sl * (1 + np.abs(re)) + 8 * R.U32 * np.abs(re)),
                      (vals[some], rv, np.broadcast_to(sl[:, None], rv.shape))):
        assert_elem(g, ref, 6 * R.U32, s, "short rows")
    all_top = _torch().topk(t[:, :vocab].float(), top, dim=1).values.double().cpu().numpy()
    lse = _torch().logsumexp(t[:, :vocab].double() / 0.9, dim=1).cpu().numpy()
    assert np.abs(vals - (all_top / 0.9 - lse[:, None])).max() < 1e-4       # every row: alternatives of the right logits


def test_logprobs_read_no_padding_and_keep_the_logits():
    torch = _torch()
    t, _ = _logits(6, 1000, 1032, 1, 0, seed=5)
    t[:, 1000:] = NAN
    keep = t.clone()
    tok = np.array([0, 999, 5, -1, 7, 8])
    _check_logp(_run_logp(t, tok, 1000, 1.0, 5, 1), t[:, :1000].double().cpu().numpy(), tok, 1.0, 5)
    assert torch.equal(t.view(torch.int16), keep.view(torch.int16))


def test_logprobs_optional_outputs_and_no_rows():
    from paper_2401_15207_b200 import k_token_logprobs, k_token_logprobs_bwd
    torch = _torch()
    t, x = _logits(5, 300, 300, 0, 0, seed=6)
    tok = _dev(np.arange(5, dtype=np.int32))
    lp = torch.empty(5, device="cuda")
    k_token_logprobs(0, 5, 300, 300, t, tok, 1.0, 0, lp, None, None)
    ref = R.token_logprobs(x, np.arange(5), 1.0, 0)[0]
    assert rel_l2(lp.cpu().numpy(), ref) < 1e-6
    k_token_logprobs(0, 0, 300, 300, t, tok, 1.0, 0, lp, None, None)
    k_token_logprobs_bwd(0, 0, 300, 300, t, tok, 1.0, lp, lp, lp, lp, t)
    torch.cuda.synchronize()


def _bwd_slack(x, st, ent, g, h, temp):
    """fp32 error of the gradient per element: p is off by its exponent's error (three roundings of |x - m| / T, one of the
    difference with L, the exponential 2^-22 and its argument's two roundings), log p + H by the same absolute error."""
    t = np.abs(np.where(np.isfinite(x), (x - st[0][:, None]) / temp, 0.0))
    lp = t + st[1][:, None]
    p = np.exp(np.where(np.isfinite(x), (x - st[0][:, None]) / temp - st[1][:, None], -np.inf))
    e = 2.0 ** -22 + R.U32 * (6 * lp + 8)
    return (e * p * (np.abs(g)[:, None] + np.abs(h)[:, None] * (lp + np.abs(ent)[:, None] + 1)) + 4 * R.U32 * p) / temp


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("rows,vocab,ld,shift,oshift,temp,mode", [
    (1, 1, 1, 0, 0, 1.0, "both"), (2, 2, 2, 1, 1, 0.7, "both"), (5, 7, 9, 3, 2, 1.5, "g"), (33, 257, 264, 2, 2, 0.7, "h"),
    (7, 1000, 1003, 5, 5, 1.0, "both"), (2, 4095, 4095, 1, 0, 1.0, "both"), (9, 32000, 32000, 0, 0, 1.0, "both"),
    (3, 50257, 50257, 7, 7, 1.0, "both"), (160, 50257, 50264, 0, 0, 1.0, "g"), (700, 130, 130, 1, 1, 1.0, "both"),
    (2, 262147, 262147, 3, 3, 1.0, "h"), (4, 64, 80, 0, 8, 1.0, "both")])
def test_logprobs_gradient_matches_the_formula(code, rows, vocab, ld, shift, oshift, temp, mode):
    from paper_2401_15207_b200 import k_token_logprobs_bwd
    torch = _torch()
    t, x = _logits(rows, vocab, ld, code, shift, seed=rows * 3 + vocab)
    t[:, vocab:] = NAN
    rng = np.random.default_rng(vocab + 1)
    if vocab > 50:
        t[:, 17:vocab:23] = -INF
        x = t[:, :vocab].double().cpu().numpy()
    tok = rng.integers(0, vocab, rows)
    tok[::5] = x[::5].argmax(1)
    _, ent, st, _, _ = R.token_logprobs(x, tok, temp, 0)
    g, h = (rng.standard_normal(rows).astype(np.float32) for _ in range(2))
    if rows > 3:
        tok[2] = -1
        t[2] = NAN
    st32, ent32 = st.astype(np.float32), ent.astype(np.float32)
    out = Guarded((rows, ld), t.dtype, oshift)
    k_token_logprobs_bwd(code, rows, vocab, ld, t, _dev(tok.astype(np.int32)), temp, _dev(st32), _dev(ent32),
                         _dev(g) if mode != "h" else None, _dev(h) if mode != "g" else None, out.t)
    torch.cuda.synchronize()
    g0, h0 = (g if mode != "h" else 0 * g).astype(np.float64), (h if mode != "g" else 0 * h).astype(np.float64)
    s64, e64 = st32.astype(np.float64), ent32.astype(np.float64)
    ref = R.token_logprobs_bwd(x, tok, temp, s64, e64, g0, h0, ld)
    slack = np.zeros((rows, ld))
    slack[:, :vocab] = _bwd_slack(x, s64, e64, g0, h0, temp)
    got = out.np()
    assert_elem(got, ref, _half_step(code) + 6 * R.U32, slack + 1e-38, "dlogits")
    assert not got[:, vocab:].any()


@pytest.mark.parametrize("code", [0, 1])
def test_logprobs_gradient_in_place_rows_without_tokens_and_large_logits(code):
    from paper_2401_15207_b200 import k_token_logprobs_bwd
    torch = _torch()
    rows, vocab = 6, 5001
    t, _ = _logits(rows, vocab, vocab, code, 0, seed=3)
    t[0] = -INF
    t[1] *= 3000.0
    t[2] = t[2] * 0.01 + 10000.0
    t[3, 3] = 40.0
    tok = np.array([4, 5, 6, 3, vocab, 9])
    x = t.double().cpu().numpy()
    a = _run_logp(t, tok, vocab, 1.0, 0, code)
    g, h = np.ones(rows, np.float32), np.full(rows, -0.5, np.float32)
    st, ent = a[2].astype(np.float32), a[1].astype(np.float32)
    sep = torch.empty_like(t)
    args = (1.0, _dev(st), _dev(ent), _dev(g), _dev(h))
    tk = _dev(tok.astype(np.int32))
    k_token_logprobs_bwd(code, rows, vocab, vocab, t, tk, *args, sep)
    k_token_logprobs_bwd(code, rows, vocab, vocab, t, tk, *args, t)
    torch.cuda.synchronize()
    assert torch.equal(sep, t)
    ref = R.token_logprobs_bwd(x, tok, 1.0, st.astype(np.float64), ent.astype(np.float64), g, h, vocab)
    assert_elem(t.double().cpu().numpy()[[0, 1, 2, 3, 4, 5]], ref, _half_step(code) + 6 * R.U32,
                np.where(np.isfinite(x), _bwd_slack(x, np.where(np.isfinite(st), st, 0).astype(np.float64), ent, g, h, 1.0), 0.0) + 1e-38)
    assert not sep[0].any() and not sep[4].any()


@pytest.mark.parametrize("temp", [1e-30, 1e-3, 1e3, 1e30])
def test_logprobs_extreme_temperatures(temp):
    t, x = _logits(5, 3000, 3000, 0, 0, seed=12)
    tok = np.array([0, int(x[1].argmax()), 5, 7, int(x[4].argmax())])
    got = _run_logp(t, tok, 3000, temp, 3, 0)
    scale = float(np.float32(1.0 / temp))              # what the kernel multiplies by
    _check_logp(got, x, tok, 1.0 / scale, 3)


def test_logprobs_gradient_against_differences_of_the_objective():
    """The kernel's gradient against central differences of the 64-bit objective along random directions."""
    from paper_2401_15207_b200 import k_token_logprobs_bwd
    torch = _torch()
    rows, vocab, temp = 4, 777, 0.8
    t, x = _logits(rows, vocab, vocab, 0, 0, seed=11)
    rng = np.random.default_rng(4)
    tok, g, h = rng.integers(0, vocab, rows), rng.standard_normal(rows), rng.standard_normal(rows)
    lp, ent, st, _, _ = _run_logp(t, tok, vocab, temp, 0, 0)
    d = torch.empty_like(t)
    f32 = np.float32
    k_token_logprobs_bwd(0, rows, vocab, vocab, t, _dev(tok.astype(np.int32)), temp, _dev(st.astype(f32)), _dev(ent.astype(f32)),
                         _dev(g.astype(f32)), _dev(h.astype(f32)), d)
    got = d.double().cpu().numpy()

    def f(z):
        a, b, *_ = R.token_logprobs(z, tok, temp, 0)
        return (g.astype(f32) * a + h.astype(f32) * b).sum()
    for k in range(5):
        v = rng.standard_normal((rows, vocab))
        num = (f(x + 1e-5 * v) - f(x - 1e-5 * v)) / 2e-5
        # third derivatives are of the order of the objective's scale: 1e-10 of it; fp32 error of the gradient 1e-6 per element
        assert abs(num - (got * v).sum()) < 1e-5 * np.abs(got * v).sum() + 1e-7


# ------------------------------------------------------------------ the junction
def _join_inputs(rows, cols, code, kind, rpg, post, pre, seed, offset=0.0):
    rng = np.random.default_rng(seed)
    dt = _dt(code)

    def op(a):
        t = _dev(a.astype(np.float32)).to(dt)
        return t, t.double().cpu().numpy()
    v = {}
    x = (rng.standard_normal((rows, cols)) * 1.5 + offset).astype(np.float32)
    v["x"] = (_dev(x), x.astype(np.float64))
    v["h"] = op(rng.standard_normal((rows, cols)) * 0.7 + 0.3 + offset)
    for n, on in (("1", post), ("2", pre)):
        v["gain" + n] = op(1 + 0.2 * rng.standard_normal(cols)) if on else (None, None)
        v["bias" + n] = op(0.2 * rng.standard_normal(cols)) if on and kind == 0 else (None, None)
    v["gate"] = op(0.5 + 0.4 * rng.standard_normal((-(-rows // rpg), cols))) if rpg else (None, None)
    v["dy"] = op(rng.standard_normal((rows, cols))) if pre else (None, None)
    dxo = rng.standard_normal((rows, cols)).astype(np.float32)
    v["dxo"] = (_dev(dxo), dxo.astype(np.float64))
    return v


def _norm_slack(hat, gain, bias, mean, rstd, cols):
    """fp32 error of a normalised row: the moments are sums in runs of at most 32 and trees (relative (32 + 20) 2^-24, the mean's
    also of the row's absolute mean), and five roundings of the element."""
    w = np.abs(gain) * (np.abs(hat) * 64 + 64 * (np.abs(mean) * rstd)[:, None] + 64)
    return R.U32 * (w + (np.abs(bias) if bias is not None else 0))


JOIN_SHAPES = [(1, 8), (3, 16), (5, 264), (37, 768), (130, 1280), (64, 2048), (9, 4096), (5, 5120), (3, 8192), (2, 12296), (2, 16384)]


@pytest.mark.parametrize("code,kind", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("rows,cols", JOIN_SHAPES)
@pytest.mark.parametrize("post,pre,gated", [(True, True, True), (True, False, False), (False, True, True), (False, False, True)])
def test_join_forward_matches_the_definition(code, kind, rows, cols, post, pre, gated):
    from paper_2401_15207_b200 import k_join_fwd
    torch = _torch()
    rpg = max(1, rows // 3) if gated else 0
    v = _join_inputs(rows, cols, code, kind, rpg, post, pre, seed=rows + cols)
    eps, scale = 1e-5, 0.75
    xo, st = Guarded((rows, cols), torch.float32), Guarded((4, rows), torch.float32)
    y = Guarded((rows, cols), _dt(code)) if pre else None
    k_join_fwd(code, kind, rows, cols, eps, scale, v["x"][0], v["h"][0], v["gain1"][0], v["bias1"][0], v["gate"][0], rpg,
               v["gain2"][0], v["bias2"][0], xo.t, y.t if pre else None, st.t)
    torch.cuda.synchronize()
    a = {n: t[1] for n, t in v.items()}
    rx, ry, rs, (hat1, hat2, u, q) = R.join_fwd(kind, eps, scale, a["x"], a["h"], a["gain1"], a["bias1"], a["gate"], rpg or 1, a["gain2"], a["bias2"])
    s1 = np.abs(q) * _norm_slack(hat1, a["gain1"], a["bias1"], rs[0], rs[1], cols) if post else 0.0
    s1 = s1 + 4 * R.U32 * (np.abs(scale * a["x"]) + np.abs(q * u))
    assert_elem(xo.np(), rx, R.U32, s1, "x_out")
    assert_elem(st.np()[[1, 3]], rs[[1, 3]], 64 * R.U32, 1e-30, "rstd")
    assert_elem(st.np()[[0, 2]], rs[[0, 2]], 64 * R.U32, 64 * R.U32 * (np.abs(a["x"]).max() + np.abs(u).max()), "mean")
    if pre:
        s2 = _norm_slack(hat2, a["gain2"], a["bias2"], rs[2], rs[3], cols)
        # an error of x_out comes through the norm: at most rstd (|e| + mean |e| (1 + |hat|)) per element
        e = np.abs(s1) * rs[3][:, None]
        s2 = s2 + np.abs(a["gain2"]) * (e + e.mean(1, keepdims=True) + np.abs(hat2) * (e * np.abs(hat2)).mean(1, keepdims=True))
        assert_elem(y.np(), ry, _half_step(code), s2, "y")


def _run_join_bwd(v, xo, st, code, kind, rows, cols, rpg, scale, want=("dgain1", "dbias1", "dgate", "dgain2", "dbias2"), dx=None):
    from paper_2401_15207_b200 import join_bwd_scratch_bytes, k_join_bwd
    torch = _torch()
    f = torch.float32
    o = {"dx": Guarded((rows, cols), f), "dh": Guarded((rows, cols), _dt(code))}
    for n, src in (("dgain1", "gain1"), ("dbias1", "bias1"), ("dgain2", "gain2"), ("dbias2", "bias2"), ("dgate", "gate")):
        if n in want and v[src][0] is not None:
            o[n] = Guarded(tuple(v[src][0].shape), f)
    w = Guarded((join_bwd_scratch_bytes(rows, cols, rpg or rows),), torch.uint8, shift=448)   # 512-byte aligned
    g = lambda n: o[n].t if n in o else None  # noqa: E731
    k_join_bwd(code, kind, rows, cols, scale, v["dy"][0], v["dxo"][0], xo, v["h"][0], st, v["gain1"][0], v["bias1"][0], v["gate"][0],
               rpg, v["gain2"][0], o["dx"].t if dx is None else dx, o["dh"].t, g("dgain1"), g("dbias1"), g("dgate"), g("dgain2"), g("dbias2"), w.t)
    torch.cuda.synchronize()
    w.np()
    return {n: t.np() for n, t in o.items()}


def _join_saved(v, kind, eps, scale, rpg):
    """The forward pass's outputs as a program holds them: fp32, and their 64-bit images."""
    a = {n: t[1] for n, t in v.items()}
    xo, _, st, _ = R.join_fwd(kind, eps, scale, a["x"], a["h"], a["gain1"], a["bias1"], a["gate"], rpg or 1, a["gain2"], a["bias2"])
    xo, st = xo.astype(np.float32), st.astype(np.float32)
    return _dev(xo), _dev(st), xo.astype(np.float64), st.astype(np.float64)


def _check_join_bwd(got, v, kind, scale, rpg, xo, st, code):
    a = {n: t[1] for n, t in v.items()}
    rows, cols = xo.shape
    ref = R.join_bwd(kind, scale, a["dy"], a["dxo"], xo, a["h"], st, a["gain1"], a["bias1"], a["gate"], rpg or 1, a["gain2"])
    k = 64 * R.U32      # ten roundings of an element and row means in runs of 32 and trees

    def norm_slack(w, hat, rstd, e):
        """|error| of rstd (w - mean w - hat mean(w hat)) when w is off by e."""
        aw, ah = np.abs(w), np.abs(hat)
        t = k * aw + e
        return rstd[:, None] * (t + (t + k * aw).mean(1, keepdims=True) + ah * ((t + k * aw) * ah).mean(1, keepdims=True))
    e = np.zeros_like(xo)
    if a["gain2"] is not None:
        hat2 = (xo - st[2][:, None]) * st[3][:, None]
        e = norm_slack(a["dy"] * a["gain2"], hat2, st[3], 4 * R.U32 * np.abs(a["dy"] * a["gain2"]))
    if a["dxo"] is not None:
        e = e + 2 * R.U32 * np.abs(a["dxo"])
    e = e + 4 * R.U32 * np.abs(ref["d"])
    assert_elem(got["dx"], ref["dx"], 2 * R.U32, abs(scale) * e, "dx")
    q = np.ones_like(xo) if a["gate"] is None else a["gate"][np.arange(rows) // rpg]
    eu = np.abs(q) * e + 2 * R.U32 * np.abs(ref["du"])
    hat1 = None
    if a["gain1"] is not None:
        hat1 = (a["h"] - st[0][:, None]) * st[1][:, None]
        eh = norm_slack(ref["du"] * a["gain1"], hat1, st[1], np.abs(a["gain1"]) * eu)
    else:
        eh = eu
    assert_elem(got["dh"], ref["dh"], _half_step(code), eh, "dh")
    # column sums: each term's error, and rows + 20 roundings of the running sum of magnitudes (fewer: chunks, then doubles)
    n = (min(rows, 256) + 20) * R.U32
    if "dgain2" in got:
        assert_elem(got["dgain2"], ref["dgain2"], 2 * R.U32, (n * np.abs(a["dy"] * hat2)).sum(0) + 6 * R.U32 * np.abs(a["dy"] * hat2).sum(0), "dgain2")
    if "dbias2" in got:
        assert_elem(got["dbias2"], ref["dbias2"], 2 * R.U32, (n * np.abs(a["dy"])).sum(0), "dbias2")
    if "dgain1" in got:
        assert_elem(got["dgain1"], ref["dgain1"], 2 * R.U32, ((n + 6 * R.U32) * np.abs(ref["du"] * hat1) + eu * np.abs(hat1)).sum(0), "dgain1")
    if "dbias1" in got:
        assert_elem(got["dbias1"], ref["dbias1"], 2 * R.U32, (n * np.abs(ref["du"]) + eu).sum(0), "dbias1")
    if "dgate" in got:
        u = a["h"] if hat1 is None else hat1 * a["gain1"] + (a["bias1"] if kind == 0 else 0)
        t = (n + 8 * R.U32) * np.abs(ref["d"] * u) + e * np.abs(u) + 8 * R.U32 * np.abs(ref["d"]) * (np.abs(hat1 * a["gain1"]) if hat1 is not None else 0)
        assert_elem(got["dgate"], ref["dgate"], 2 * R.U32, np.stack([t[i:i + rpg].sum(0) for i in range(0, rows, rpg)]), "dgate")


@pytest.mark.parametrize("code,kind", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("rows,cols", JOIN_SHAPES)
@pytest.mark.parametrize("post,pre,gated", [(True, True, True), (True, False, False), (False, True, True), (False, False, True)])
def test_join_backward_matches_the_formula(code, kind, rows, cols, post, pre, gated):
    rpg = max(1, rows // 3) if gated else 0
    v = _join_inputs(rows, cols, code, kind, rpg, post, pre, seed=rows + cols + 1)
    xo_d, st_d, xo, st = _join_saved(v, kind, 1e-5, 0.75, rpg)
    got = _run_join_bwd(v, xo_d, st_d, code, kind, rows, cols, rpg, 0.75)
    _check_join_bwd(got, v, kind, 0.75, rpg, xo, st, code)


@pytest.mark.parametrize("rows,rpg", [(1, 1), (7, 1), (7, 100), (1000, 1), (1300, 2), (601, 1), (2500, 7), (2500, 600), (2500, 2499), (5000, 5000)])
def test_join_backward_gate_groups(rows, rpg):
    v = _join_inputs(rows, 72, 0, 0, rpg, True, True, seed=rows * 7 + rpg)
    xo_d, st_d, xo, st = _join_saved(v, 0, 1e-5, 1.0, rpg)
    _check_join_bwd(_run_join_bwd(v, xo_d, st_d, 0, 0, rows, 72, rpg, 1.0), v, 0, 1.0, rpg, xo, st, 0)


def test_join_backward_wants_and_missing_gradients():
    """Gradients that are not wanted, no gradient past the norm, no gradient into y, dx in the place of dx_out; the same bits."""
    torch = _torch()
    rows, cols, rpg = 300, 512, 50
    v = _join_inputs(rows, cols, 1, 0, rpg, True, True, seed=9)
    xo_d, st_d, xo, st = _join_saved(v, 0, 1e-5, 1.0, rpg)
    full = _run_join_bwd(v, xo_d, st_d, 1, 0, rows, cols, rpg, 1.0)
    again = _run_join_bwd(v, xo_d, st_d, 1, 0, rows, cols, rpg, 1.0)
    assert all(np.array_equal(full[n], again[n]) for n in full)
    some = _run_join_bwd(v, xo_d, st_d, 1, 0, rows, cols, rpg, 1.0, want=("dgate", "dbias2"))
    assert set(some) == {"dx", "dh", "dgate", "dbias2"} and all(np.array_equal(full[n], some[n]) for n in some)
    none = _run_join_bwd(v, xo_d, st_d, 1, 0, rows, cols, rpg, 1.0, want=())
    assert all(np.array_equal(full[n], none[n]) for n in none)
    place = v["dxo"][0].clone()
    w = dict(v, dxo=(place, None))
    inp = _run_join_bwd(w, xo_d, st_d, 1, 0, rows, cols, rpg, 1.0, dx=place)
    assert np.array_equal(place.double().cpu().numpy(), full["dx"]) and np.array_equal(inp["dh"], full["dh"])
    w = dict(v, dxo=(None, None))
    _check_join_bwd(_run_join_bwd(w, xo_d, st_d, 1, 0, rows, cols, rpg, 1.0), w, 0, 1.0, rpg, xo, st, 1)
    assert torch.equal(xo_d.cpu(), torch.from_numpy(xo.astype(np.float32)))


@pytest.mark.parametrize("kind", [0, 1])
def test_join_rows_far_from_zero_and_constant_rows(kind):
    from paper_2401_15207_b200 import k_join_fwd
    torch = _torch()
    rows, cols = 6, 1024
    v = _join_inputs(rows, cols, 0, kind, 0, True, True, seed=21, offset=300.0)
    v["h"][0][0] = 0.0                              # a row of zeros, and a constant row: the variance is 0, eps decides
    v["h"][0][1] = 5.0
    v["h"] = (v["h"][0], v["h"][0].double().cpu().numpy())
    xo, y, st = (torch.empty(rows, cols, device="cuda") for _ in range(3))
    st = torch.empty(4, rows, device="cuda")
    k_join_fwd(0, kind, rows, cols, 1e-5, 1.0, v["x"][0], v["h"][0], v["gain1"][0], v["bias1"][0], None, 0, v["gain2"][0], v["bias2"][0], xo, y, st)
    a = {n: t[1] for n, t in v.items()}
    rx, ry, rs, (hat1, hat2, u, q) = R.join_fwd(kind, 1e-5, 1.0, a["x"], a["h"], a["gain1"], a["bias1"], None, 1, a["gain2"], a["bias2"])
    s1 = _norm_slack(hat1, a["gain1"], a["bias1"], rs[0], rs[1], cols) + 4 * R.U32 * (np.abs(a["x"]) + np.abs(u))
    assert_elem(xo.double().cpu().numpy(), rx, R.U32, s1, "x_out")
    e = s1 * rs[3][:, None]
    s2 = _norm_slack(hat2, a["gain2"], a["bias2"], rs[2], rs[3], cols) + np.abs(a["gain2"]) * (e + e.mean(1, keepdims=True) + np.abs(hat2) * (e * np.abs(hat2)).mean(1, keepdims=True))
    assert_elem(y.double().cpu().numpy(), ry, R.U32, s2, "y")


def test_join_in_place_and_no_rows():
    from paper_2401_15207_b200 import k_join_bwd, k_join_fwd
    torch = _torch()
    rows, cols = 50, 768
    v = _join_inputs(rows, cols, 1, 1, 10, True, True, seed=4)
    outs = []
    for place in (False, True):
        x = v["x"][0].clone()
        xo = x if place else torch.empty_like(x)
        y, st = torch.empty_like(v["h"][0]), torch.empty(4 * rows, device="cuda")
        k_join_fwd(1, 1, rows, cols, 1e-6, 1.0, x, v["h"][0], v["gain1"][0], None, v["gate"][0], 10, v["gain2"][0], None, xo, y, st)
        outs.append((xo, y, st))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    sums = [torch.full((cols,), 7.0, device="cuda") for _ in range(2)]
    k_join_fwd(1, 1, 0, cols, 1e-6, 1.0, x, v["h"][0], v["gain1"][0], None, v["gate"][0], 10, v["gain2"][0], None, xo, y, st)
    k_join_bwd(1, 1, 0, cols, 1.0, None, None, None, None, None, v["gain1"][0], None, None, 0, v["gain2"][0], None, None, sums[0], None, None,
               sums[1], None, None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and not sums[0].any() and not sums[1].any()


# ------------------------------------------------------------------ the orthogonalised update
# What the products may put on the result, relative to its Frobenius norm: the products' operands are rounded to 16 bits
# with 11 significant (2^-12 rms at most 2^-11 / sqrt 3 each), the iterate itself and the diagonals of A and of the polynomial
# stay fp32.  A CPU model of exactly these roundings over Gaussian, low-rank (rank 1 to 8), decaying, one-row, outlier and sparse
# matrices of 4 x 40 to 512 x 512 gives 2e-4 to 2.4e-3, with the result's own rounding (1.7e-3) up to 2.9e-3; 2^-8 is the documented bound.
NS_TOL = 2.0 ** -8


def _ns_tol(n):
    """For a bf16 result of n elements.  Many elements: rounding errors are spread over the half step (2^-8 relative at most), their
    norm is at most 2^-8 / sqrt 3 = 2.3e-3 of the result's, with the products' 2.4e-3 together 3.3e-3 < 2^-8.  A few elements can all
    be half a step off: 2^-8 more."""
    return NS_TOL if n >= 100 else 2 * NS_TOL


def _matrix(kind, rows, cols, seed):
    rng = np.random.default_rng(seed)
    k = min(rows, cols)
    if kind == "gauss":
        g = rng.standard_normal((rows, cols))
    elif kind == "lowrank":
        r = max(1, k // 16)
        g = rng.standard_normal((rows, r)) @ rng.standard_normal((r, cols))
    elif kind.startswith("rank"):
        r = int(kind[4:])
        g = rng.standard_normal((rows, r)) @ rng.standard_normal((r, cols))
    elif kind == "onerow":
        g = np.zeros((rows, cols))
        g[rows // 2] = rng.standard_normal(cols)
    elif kind == "decay":
        u, v = np.linalg.qr(rng.standard_normal((rows, k)))[0], np.linalg.qr(rng.standard_normal((cols, k)))[0]
        g = (u * np.arange(1, k + 1) ** -1.0) @ v.T
    elif kind == "outlier":
        g = rng.standard_normal((rows, cols))
        g[:, 0] *= 100
        g[-1] *= 30
    else:
        g = np.zeros((rows, cols))
        g[::5] = rng.standard_normal(g[::5].shape)
    return g.astype(np.float32)


def _orth(g, code, steps=5, shift=1):
    from paper_2401_15207_b200 import k_orthogonalize, orthogonalize_scratch_bytes
    torch = _torch()
    rows, cols = g.shape
    o = Guarded((rows, cols), torch.bfloat16, shift=shift)
    w = Guarded((orthogonalize_scratch_bytes(rows, cols),), torch.uint8, shift=448)
    k_orthogonalize(code, rows, cols, g, o.t, steps, w.t)
    torch.cuda.synchronize()
    w.np()
    return o.np()


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 9), (9, 1), (2, 3), (16, 16), (63, 65), (64, 64), (127, 129), (128, 128), (129, 300), (300, 129),
                                       (513, 255), (768, 768), (257, 1000), (1100, 600), (40, 3001), (3001, 40), (1300, 2600), (2600, 1300),
                                       (700, 4000), (4000, 330), (50, 11008), (2100, 1400), (9000, 200)])
def test_orthogonalize_matches_the_definition(code, rows, cols):
    g = _dev(_matrix("gauss", rows, cols, rows * 7 + cols), _dt(code))
    assert rel_l2(_orth(g, code), R.orthogonalize(g.double().cpu().numpy())) < _ns_tol(rows * cols)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("rows,cols", [(512, 640), (640, 512), (132, 260), (128, 4096), (4096, 128), (100, 4100), (129, 129)])
def test_orthogonalize_rows_that_move_as_vectors(code, rows, cols):
    """The same bits from aligned buffers (16-byte accesses where the columns allow it) and from displaced ones."""
    torch = _torch()
    base = _dev(_matrix("gauss", rows, cols, rows + 3 * cols), _dt(code))
    flat = torch.zeros(rows * cols + 1, dtype=base.dtype, device="cuda")
    moved = flat[1:].view(rows, cols)
    moved.copy_(base)
    a, b = _orth(base, code, shift=0), _orth(moved, code, shift=1)
    assert np.array_equal(a, b)
    assert rel_l2(a, R.orthogonalize(base.double().cpu().numpy())) < NS_TOL


@pytest.mark.parametrize("kind", ["rank1", "rank2", "rank3", "lowrank", "decay", "outlier", "sparse", "onerow"])
@pytest.mark.parametrize("rows,cols", [(16, 16), (16, 300), (300, 16), (100, 100), (60, 900), (900, 60), (256, 256), (300, 700), (700, 300)])
def test_orthogonalize_spectra(kind, rows, cols):
    g = _dev(_matrix(kind, rows, cols, rows + cols))
    assert rel_l2(_orth(g, 0), R.orthogonalize(g.double().cpu().numpy())) < NS_TOL


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_orthogonalize_steps(steps):
    g = _dev(_matrix("gauss", 200, 333, 5))
    assert rel_l2(_orth(g, 0, steps), R.orthogonalize(g.double().cpu().numpy(), steps)) < NS_TOL


@pytest.mark.parametrize("rows,cols", [(130, 200), (200, 130)])
def test_orthogonalize_scales_zeros_and_bad_values(rows, cols):
    torch = _torch()
    base = _matrix("gauss", rows, cols, 8)
    ref = R.orthogonalize(base.astype(np.float64))
    for s in (1e-25, 1e-6, 1e6, 1e30):              # squares beyond fp32 both ways
        assert rel_l2(_orth(_dev((base.astype(np.float64) * s).astype(np.float32)), 0), ref) < NS_TOL
    assert not _orth(torch.zeros(rows, cols, device="cuda"), 0).any()
    assert not _orth(torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16), 1).any()
    for bad in (NAN, INF, -INF):
        g = _dev(base)
        g[3, 5] = bad
        assert np.isnan(_orth(g, 0)).all()


@pytest.mark.parametrize("rows,cols,nesterov,wd,has_param", [(1, 1, True, 0.0, True), (64, 64, True, 0.1, True), (77, 300, False, 0.0, True),
                                                             (1000, 130, True, 0.01, False), (301, 301, False, 0.1, True), (256, 512, True, 0.1, True), (512, 132, False, 0.0, True),
                                                             (20, 3000, True, 0.1, True), (3000, 20, False, 0.1, True), (128, 128, True, 0.0, False)])
def test_muon_step_matches_the_definition(rows, cols, nesterov, wd, has_param):
    from paper_2401_15207_b200 import muon_step, orthogonalize_scratch_bytes
    torch = _torch()
    rng = np.random.default_rng(rows + cols)
    master = (rng.standard_normal((rows, cols)) * 0.02).astype(np.float32)
    mom = (rng.standard_normal((rows, cols)) * 1e-3).astype(np.float32)
    tm, tb = Guarded((rows, cols), torch.float32), Guarded((rows, cols), torch.float32)
    tm.t.copy_(_dev(master)), tb.t.copy_(_dev(mom))
    tp = Guarded((rows, cols), torch.bfloat16, shift=rows % 2)          # an even number of rows: aligned
    w = torch.empty(orthogonalize_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    for k in range(3):
        grad = (_matrix("gauss", rows, cols, k) * np.float32(1e-3)).astype(np.float32)
        before, b_before = tm.np(), tb.np()
        muon_step(rows, cols, tp.t if has_param else None, tm.t, _dev(grad), tb.t, w, 1e-2, momentum=0.9, nesterov=nesterov, weight_decay=wd)
        torch.cuda.synchronize()
        m64, b64 = R.muon_step(before, grad.astype(np.float64), b_before, 1e-2, 0.9, nesterov, wd)
        # one fused multiply-add with mu rounded to fp32: at most two half steps of its terms, which may cancel in the sum
        assert_elem(tb.np(), b64, R.U32, 2 * R.U32 * (0.9 * np.abs(b_before) + np.abs(grad.astype(np.float64))), "momentum")
        # the update to the orthogonalisation's tolerance, plus the roundings of the stored master
        assert np.linalg.norm(tm.np() - m64) <= NS_TOL * np.linalg.norm(m64 - before * (1 - 1e-2 * wd)) + 4 * R.U32 * np.linalg.norm(m64)
        if has_param:
            assert np.array_equal(tp.np(), tm.t.to(torch.bfloat16).double().cpu().numpy())
    if not has_param:
        assert (tp.np() == 77).all()


@pytest.mark.parametrize("rows,cols", [(100, 60), (200, 300)])
def test_orthogonalize_writes_nothing_after_a_time_out(rows, cols):
    """With the tensor-core time-out flag raised, results and master stay as they are; cleared, the calls work again."""
    from paper_2401_15207_b200 import k_orthogonalize, muon_step, orthogonalize_scratch_bytes, tc_error_flag
    torch = _torch()
    g = _dev(_matrix("gauss", rows, cols, 3))
    o = torch.full((rows, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    master, mom = torch.full((rows, cols), 0.5, device="cuda"), torch.zeros(rows, cols, device="cuda")
    w = torch.empty(orthogonalize_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    assert tc_error_flag(1) == 1
    try:
        k_orthogonalize(0, rows, cols, g, o, 5, w)
        muon_step(rows, cols, None, master, g, mom, w, 1e-2)
        torch.cuda.synchronize()
        assert bool((o == 7).all()) and bool((master == 0.5).all())
    finally:
        assert tc_error_flag(0) == 0
    k_orthogonalize(0, rows, cols, g, o, 5, w)
    assert rel_l2(o.double().cpu().numpy(), R.orthogonalize(g.double().cpu().numpy())) < NS_TOL


# ------------------------------------------------------------------ offsets beyond 32 bits
def _same_bits(a, b):
    torch = _torch()
    i = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(i), b.contiguous().view(i))


def test_logprobs_of_rows_beyond_32_bit_offsets():
    """Rows 2^30 + 8 elements apart: the last starts beyond 2^31.  Same bits as the rows side by side; padding gets zeros."""
    from paper_2401_15207_b200 import k_token_logprobs, k_token_logprobs_bwd
    torch = _torch()
    rows, vocab, ld = 3, 1003, 2 ** 30 + 8
    near, _ = _logits(rows, vocab, 1008, 1, 0, seed=6)
    far = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    far[:, :vocab] = near[:, :vocab]
    far[:, vocab:vocab + 40] = NAN
    far[:, -40:] = NAN
    tok, w = _dev(np.array([1002, 0, 500], np.int32)), _dev(np.array([1.0, -2.0, 0.5], np.float32))
    outs = []
    for t, d in ((near, 1008), (far, ld)):
        o = [torch.zeros(n, device="cuda") for n in (rows, rows, 2 * rows)] + [torch.zeros(rows, 5, dtype=torch.int32, device="cuda"), torch.zeros(rows, 5, device="cuda")]
        k_token_logprobs(1, rows, vocab, d, t, tok, 1.0, 5, *o)
        k_token_logprobs_bwd(1, rows, vocab, d, t, tok, 1.0, o[2], o[1], w, w, t)
        outs.append(o)
    assert all(_same_bits(a, b) for a, b in zip(*outs))
    assert _same_bits(near[:, :vocab], far[:, :vocab])
    assert all(not bool(far[r, vocab:].any()) for r in range(rows))


def test_join_of_a_tensor_beyond_32_bit_offsets():
    """2.1e9 elements: the rows around and behind the 2^31st give the bits of the same rows alone."""
    from paper_2401_15207_b200 import join_bwd_scratch_bytes, k_join_bwd, k_join_fwd
    torch = _torch()
    cols, rows, n = 16384, 2 ** 17 + 40, 64
    v = _join_inputs(n, cols, 1, 0, n, True, True, seed=12)
    f, h = torch.float32, torch.bfloat16

    def run(x, hh, dy, dxo, r):
        y, st, dh = torch.zeros(r, cols, dtype=h, device="cuda"), torch.zeros(4 * r, device="cuda"), torch.zeros(r, cols, dtype=h, device="cuda")
        g = [torch.zeros(cols, device="cuda") for _ in range(4)]
        dq = torch.zeros(1, cols, device="cuda")
        k_join_fwd(1, 0, r, cols, 1e-5, 1.0, x, hh, v["gain1"][0], v["bias1"][0], v["gate"][0], r, v["gain2"][0], v["bias2"][0], x, y, st)
        w = torch.empty(join_bwd_scratch_bytes(r, cols, r), dtype=torch.uint8, device="cuda")
        k_join_bwd(1, 0, r, cols, 1.0, dy, dxo, x, hh, st, v["gain1"][0], v["bias1"][0], v["gate"][0], r, v["gain2"][0], dxo, dh, g[0], g[1], dq, g[2], g[3], w)
        return dict(x=x, y=y, dx=dxo, dh=dh), g + [dq]
    few, sums = run(v["x"][0].clone(), v["h"][0], v["dy"][0], v["dxo"][0].clone(), n)
    big = [torch.zeros(rows, cols, dtype=d, device="cuda") for d in (f, h, h, f)]
    for t, name in zip(big, ("x", "h", "dy", "dxo")):
        t[-n:] = v[name][0]                          # the rows before them are zeros, with gradients of zero: they add nothing to the sums
    many, msums = run(*big, rows)
    for name in few:
        assert _same_bits(many[name][-n:], few[name]), name
    assert not bool(many["dx"][:-n].any()) and not bool(many["dh"][:-n].any())
    for a, b in zip(msums, sums):                    # fp32 sums of at most 64 terms, in two orders
        assert float((a - b).norm()) <= 64 * 2 * R.U32 * float(b.abs().sum())
    del big, many
    torch.cuda.empty_cache()


def test_orthogonalize_of_a_matrix_beyond_32_bit_offsets():
    """65536 x 33000 with values in few rows and columns, the last ones among them: their submatrix is orthogonalised, the rest stays zero."""
    from paper_2401_15207_b200 import k_orthogonalize, orthogonalize_scratch_bytes
    torch = _torch()
    rows, cols = 65536, 33000
    r = [0, 1, 17, 40000, 65000, 65534, 65535]
    c = torch.cat([torch.arange(0, 33000, 331, device="cuda"), torch.tensor([32998, 32999], device="cuda")])
    sub = _dev(_matrix("gauss", len(r), len(c), 7))
    g = torch.zeros(rows, cols, device="cuda")
    for i, k in enumerate(r):
        g[k][c] = sub[i]
    w = torch.empty(orthogonalize_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    o = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    k_orthogonalize(0, rows, cols, g, o, 5, w)
    got = torch.stack([o[k][c] for k in r])
    assert rel_l2(got.double().cpu().numpy(), R.orthogonalize(sub.double().cpu().numpy())) < NS_TOL
    for k in r:
        o[k][c] = 0
    assert int(torch.count_nonzero(o)) == 0
    del g, w, o
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ streams, graphs, and the whole run
def test_operators_captured_in_a_graph_give_the_bits_of_the_calls():
    from paper_2401_15207_b200 import (join_bwd_scratch_bytes, k_join_bwd, k_join_fwd, k_token_logprobs, k_token_logprobs_bwd,
                                       k_orthogonalize, orthogonalize_scratch_bytes)
    torch = _torch()
    rows, cols, vocab = 40, 512, 1001
    v = _join_inputs(rows, cols, 1, 0, 8, True, True, seed=2)
    t, _ = _logits(rows, vocab, vocab, 1, 0, seed=2)
    tok = _dev((np.arange(rows) * 7 % vocab).astype(np.int32))
    g, small = _dev(_matrix("gauss", 200, 130, 1)), _dev(_matrix("gauss", 90, 700, 1))

    def buffers():
        f = torch.float32
        e = lambda *s, d=f: torch.full(s, 9, dtype=d, device="cuda")  # noqa: E731
        return dict(xo=e(rows, cols), y=e(rows, cols, d=torch.bfloat16), st=e(4 * rows), dx=e(rows, cols), dh=e(rows, cols, d=torch.bfloat16),
                    dg1=e(cols), db1=e(cols), dq=e(5, cols), dg2=e(cols), db2=e(cols), lp=e(rows), en=e(rows), ls=e(2 * rows),
                    ids=e(rows, 4, d=torch.int32), tv=e(rows, 4), dl=torch.full_like(t, 9), o=e(200, 130, d=torch.bfloat16), os=e(90, 700, d=torch.bfloat16),
                    w1=e(join_bwd_scratch_bytes(rows, cols, 8), d=torch.uint8), w2=e(orthogonalize_scratch_bytes(200, 130), d=torch.uint8),
                    w3=e(orthogonalize_scratch_bytes(90, 700), d=torch.uint8))

    def run(b):
        k_join_fwd(1, 0, rows, cols, 1e-5, 1.0, v["x"][0], v["h"][0], v["gain1"][0], v["bias1"][0], v["gate"][0], 8, v["gain2"][0], v["bias2"][0],
                   b["xo"], b["y"], b["st"])
        k_join_bwd(1, 0, rows, cols, 1.0, v["dy"][0], v["dxo"][0], b["xo"], v["h"][0], b["st"], v["gain1"][0], v["bias1"][0], v["gate"][0], 8,
                   v["gain2"][0], b["dx"], b["dh"], b["dg1"], b["db1"], b["dq"], b["dg2"], b["db2"], b["w1"])
        k_token_logprobs(1, rows, vocab, vocab, t, tok, 1.0, 4, b["lp"], b["en"], b["ls"], b["ids"], b["tv"])
        k_token_logprobs_bwd(1, rows, vocab, vocab, t, tok, 1.0, b["ls"], b["en"], b["lp"], b["en"], b["dl"])
        k_orthogonalize(0, 200, 130, g, b["o"], 5, b["w2"])
        k_orthogonalize(0, 90, 700, small, b["os"], 5, b["w3"])
    eager = buffers()
    run(eager)
    side, b = torch.cuda.Stream(), buffers()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                   # on a stream that is not the default one
        run(b)
    side.synchronize()
    names = [n for n in b if not n.startswith("w")]
    assert all(torch.equal(eager[n], b[n]) for n in names)
    # two graphs with scratch of their own, replayed on two streams at once
    graphs, bufs = [], [buffers(), buffers()]
    for b in bufs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            run(b)
        graphs.append(gr)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    for b in bufs:
        assert all(torch.equal(eager[n], b[n]) for n in names)


@pytest.mark.parametrize("rows,cols,vocab", [(8, 64, 129), (300, 1024, 4099)])
def test_calls_behind_one_another_wait_for_what_they_read(rows, cols, vocab):
    """A kernel may be resident before its predecessor has ended.  Each call here reads what the one before it wrote, over buffers
    and scratch that the next round writes again; the bits are those of a run that waits for the device after every call."""
    from paper_2401_15207_b200 import (join_bwd_scratch_bytes, k_join_bwd, k_join_fwd, k_orthogonalize, k_token_logprobs, k_token_logprobs_bwd, muon_step,
                                       orthogonalize_scratch_bytes)
    torch = _torch()
    f, h = torch.float32, torch.bfloat16
    v = _join_inputs(rows, cols, 1, 0, rows, True, True, seed=rows)
    logits0, _ = _logits(rows, vocab, vocab, 1, 0, seed=3)
    tok = _dev((np.arange(rows) * 11 % vocab).astype(np.int32))
    shapes = [(12, 700), (90, 260), (rows, cols)]      # the last of 300 x 1024 goes through tiled products, the others are single launches
    mats = [_dev(_matrix("gauss", r, c, 4)) for r, c in shapes]
    need = max(orthogonalize_scratch_bytes(r, c) for r, c in shapes)

    def buffers():
        e = lambda *s, d=f: torch.zeros(*s, dtype=d, device="cuda")  # noqa: E731
        return dict(xo=e(rows, cols), x2=v["x"][0].clone(), y=e(rows, cols, d=h), st=e(4 * rows), dx=v["dxo"][0].clone(), dx2=e(rows, cols), dh=e(rows, cols, d=h),
                    dg1=e(cols), db1=e(cols), dq=e(1, cols), dg2=e(cols), db2=e(cols), w1=e(join_bwd_scratch_bytes(rows, cols, rows), d=torch.uint8),
                    t=logits0.clone(), lp=e(rows), en=e(rows), ls=e(2 * rows), ids=e(rows, 3, d=torch.int32), tv=e(rows, 3), w2=e(need, d=torch.uint8),
                    **{f"{n}{i}": e(r, c, d=h if n == "o" else f) for i, (r, c) in enumerate(shapes) for n in ("o", "master", "mom")})

    def run(b, done):
        for k in range(4):
            xin, xout = (b["x2"], b["xo"]) if k % 2 == 0 else (b["xo"], b["x2"])
            k_join_fwd(1, 0, rows, cols, 1e-5, 1.0, xin, v["h"][0], v["gain1"][0], v["bias1"][0], v["gate"][0], rows, v["gain2"][0], v["bias2"][0],
                       xout, b["y"], b["st"])
            done()
            din, dout = (b["dx"], b["dx2"]) if k % 2 == 0 else (b["dx2"], b["dx"])
            k_join_bwd(1, 0, rows, cols, 1.0, b["y"], din, xout, v["h"][0], b["st"], v["gain1"][0], v["bias1"][0], v["gate"][0], rows,
                       v["gain2"][0], dout, b["dh"], b["dg1"], b["db1"], b["dq"], b["dg2"], b["db2"], b["w1"])
            done()
            k_token_logprobs(1, rows, vocab, vocab, b["t"], tok, 1.0, 3, b["lp"], b["en"], b["ls"], b["ids"], b["tv"])
            done()
            k_token_logprobs_bwd(1, rows, vocab, vocab, b["t"], tok, 1.0, b["ls"], b["en"], b["lp"], b["en"], b["t"])      # in place: the next round's logits
            done()
            for i, (r, c) in enumerate(shapes):
                muon_step(r, c, None, b[f"master{i}"], mats[i] if i < 2 else b["dx2"], b[f"mom{i}"], b["w2"], 1e-2)
                done()
                k_orthogonalize(0, r, c, b[f"master{i}"], b[f"o{i}"], 5, b["w2"])
                done()
    want, got = buffers(), buffers()
    torch.cuda.synchronize()
    run(want, torch.cuda.synchronize)
    run(got, lambda: None)
    names = [n for n in got if not n.startswith("w")]
    torch.cuda.synchronize()
    assert [n for n in names if not torch.equal(want[n], got[n])] == []
    assert all(bool(torch.isfinite(want[n].float()).all()) for n in names if n not in ("ids", "tv"))
    again = buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(again, lambda: None)
    fresh = buffers()
    for _ in range(3):                               # the copies are other people's kernels between two replays
        for n in again:
            again[n].copy_(fresh[n])
        graph.replay()
    torch.cuda.synchronize()
    assert [n for n in names if not torch.equal(want[n], again[n])] == []


@pytest.mark.parametrize("code", [0, 1])
def test_a_fine_tuning_step_out_of_the_operators(code):
    """Junction -> head product -> log-probabilities with entropy -> their gradient -> head products' gradients -> junction backward
    -> orthogonalised update of the head, as an objective on given tokens uses them; against the same in 64 bits."""
    from paper_2401_15207_b200 import (join_bwd_scratch_bytes, k_join_bwd, k_join_fwd, k_linear, k_token_logprobs, k_token_logprobs_bwd,
                                       muon_step, orthogonalize_scratch_bytes)
    torch = _torch()
    rows, cols, vocab, kind, eps = 192, 256, 640, 1, 1e-6
    dt, f = _dt(code), torch.float32
    v = _join_inputs(rows, cols, code, kind, 64, True, True, seed=31)
    rng = np.random.default_rng(32)
    wm = (rng.standard_normal((vocab, cols)) * 0.05).astype(np.float32)
    w = _dev(wm).to(dt)
    tok = rng.integers(0, vocab, rows).astype(np.int32)
    tok[::9] = -1
    adv = (rng.standard_normal(rows) / rows).astype(np.float32)
    hent = np.full(rows, -0.01 / rows, np.float32)
    e = lambda *s, d=f: torch.empty(*s, dtype=d, device="cuda")  # noqa: E731
    xo, y, st = e(rows, cols), e(rows, cols, d=dt), e(4 * rows)
    k_join_fwd(code, kind, rows, cols, eps, 1.0, v["x"][0], v["h"][0], v["gain1"][0], None, v["gate"][0], 64, v["gain2"][0], None, xo, y, st)
    logits, lp, en, ls = e(rows, vocab, d=dt), e(rows), e(rows), e(2 * rows)
    k_linear(0, code, rows, vocab, cols, y, w, logits)
    k_token_logprobs(code, rows, vocab, vocab, logits, _dev(tok), 1.0, 0, lp, en, ls)
    k_token_logprobs_bwd(code, rows, vocab, vocab, logits, _dev(tok), 1.0, ls, en, _dev(adv), _dev(hent), logits)
    dy, dw = e(rows, cols, d=dt), e(vocab, cols)
    k_linear(1, code, rows, vocab, cols, logits, w, dy)
    k_linear(2, code, rows, vocab, cols, logits, y, dw)
    o = {n: e(cols) for n in ("dgain1", "dgain2")}
    o["dgate"] = e(3, cols)
    dx, dh = e(rows, cols), e(rows, cols, d=dt)
    scr = e(join_bwd_scratch_bytes(rows, cols, 64), d=torch.uint8)
    zero = torch.zeros(rows, cols, device="cuda")
    k_join_bwd(code, kind, rows, cols, 1.0, dy, zero, xo, v["h"][0], st, v["gain1"][0], None, v["gate"][0], 64, v["gain2"][0], dx, dh,
               o["dgain1"], None, o["dgate"], o["dgain2"], None, scr)
    master, mom, par = _dev(wm), torch.zeros(vocab, cols, device="cuda"), e(vocab, cols, d=torch.bfloat16)
    sc2 = e(orthogonalize_scratch_bytes(vocab, cols), d=torch.uint8)
    muon_step(vocab, cols, par, master, dw, mom, sc2, 1e-3)
    torch.cuda.synchronize()
    # the same in 64 bits
    a = {n: t[1] for n, t in v.items()}
    w64 = w.double().cpu().numpy()
    rxo, ry, rst, _ = R.join_fwd(kind, eps, 1.0, a["x"], a["h"], a["gain1"], None, a["gate"], 64, a["gain2"], None)
    z = ry @ w64.T
    rlp, ren, rls, _, _ = R.token_logprobs(z, tok, 1.0, 0)
    dz = R.token_logprobs_bwd(z, tok, 1.0, rls, ren, adv.astype(np.float64), hent.astype(np.float64), vocab)
    rdw, rdy = dz.T @ ry, dz @ w64
    rb = R.join_bwd(kind, 1.0, rdy, np.zeros_like(rdy), rxo, a["h"], rst, a["gain1"], None, a["gate"], 64, a["gain2"])
    # fp32: sums of 256 to 640 products; bf16: y, the logits, their gradient and dy are each rounded to bf16 (2^-8 at most)
    tol = 2e-2 if code else 2e-5
    for got, ref, n in ((xo, rxo, "x_out"), (lp, rlp, "logp"), (en, ren, "entropy"), (dw, rdw, "dW"), (dx, rb["dx"], "dx"), (dh, rb["dh"], "dh"),
                        (o["dgain1"], rb["dgain1"], "dgain1"), (o["dgain2"], rb["dgain2"], "dgain2"), (o["dgate"], rb["dgate"], "dgate")):
        assert rel_l2(got.double().cpu().numpy(), ref) < tol, n
    rm, _ = R.muon_step(wm.astype(np.float64), dw.double().cpu().numpy(), np.zeros((vocab, cols)), 1e-3, 0.95, True, 0.0)
    assert np.linalg.norm(master.double().cpu().numpy() - rm) < NS_TOL * np.linalg.norm(rm - wm) + 4 * R.U32 * np.linalg.norm(rm)
