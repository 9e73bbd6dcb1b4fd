"""What the operators beside the step refuse, and the sizes they report: host logic, no GPU needed (a call that is
refused launches nothing, so the pointers below are never read)."""
import numpy as np
import pytest

import train_ops_ref as R
from paper_2401_15207_b200 import binding as B, build

CFG, INPUT, CAPACITY = 1, 4, 8
P = 1 << 20            # a well-aligned address that nothing reads


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.load_library()


def _logp(L, **kw):
    a = dict(dtype=1, rows=4, vocab=100, ld=100, logits=P, tokens=P, temp=1.0, top=3, logp=P, ent=P, stats=P, ids=P, vals=P, bad=None)
    a.update(kw)
    return L.hift_k_token_logprobs(a["dtype"], a["rows"], a["vocab"], a["ld"], a["logits"], a["tokens"], a["temp"], a["top"], a["logp"],
                                   a["ent"], a["stats"], a["ids"], a["vals"], a["bad"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), CFG), (dict(rows=-1), CFG), (dict(rows=1 << 31), CFG), (dict(vocab=0), CFG), (dict(ld=99), CFG),
    (dict(vocab=1 << 31, ld=1 << 31), CFG), (dict(temp=0.0), CFG), (dict(temp=-1.0), CFG), (dict(temp=float("nan")), CFG),
    (dict(temp=float("inf")), CFG), (dict(temp=1e-40), CFG), (dict(temp=3.2e-39), CFG), (dict(temp=1e40), CFG), (dict(top=-1), CFG), (dict(top=33), CAPACITY),
    (dict(logits=None), INPUT), (dict(tokens=None), INPUT), (dict(logp=None), INPUT), (dict(ids=None), INPUT), (dict(vals=None), INPUT),
    (dict(logits=P + 1), CFG), (dict(dtype=0, logits=P + 2), CFG), (dict(rows=0, logits=None, tokens=None, logp=None), 0)])
def test_token_logprobs_refuses(L, kw, want):
    assert _logp(L, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=-1), CFG), (dict(ld=10), CFG), (dict(temp=0.0), CFG), (dict(logits=None), INPUT), (dict(tokens=None), INPUT),
    (dict(stats=None), INPUT), (dict(g=None, h=None), INPUT), (dict(ent=None), INPUT), (dict(out=None), INPUT), (dict(out=P + 1), CFG),
    (dict(rows=0), 0)])
def test_token_logprobs_bwd_refuses(L, kw, want):
    a = dict(dtype=1, rows=4, vocab=100, ld=100, logits=P, tokens=P, temp=1.0, stats=P, ent=P, g=P, h=P, out=P)
    a.update(kw)
    assert L.hift_k_token_logprobs_bwd(a["dtype"], a["rows"], a["vocab"], a["ld"], a["logits"], a["tokens"], a["temp"], a["stats"],
                                       a["ent"], a["g"], a["h"], a["out"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), CFG), (dict(kind=2), CFG), (dict(rows=-1), CFG), (dict(cols=12), CFG), (dict(cols=0), CFG), (dict(cols=16392), CAPACITY),
    (dict(eps=-1.0), CFG), (dict(eps=float("nan")), CFG), (dict(scale=float("inf")), CFG), (dict(rpg=0), CFG), (dict(x=None), INPUT),
    (dict(h=None), INPUT), (dict(xo=None), INPUT), (dict(y=None), INPUT), (dict(stats=None), INPUT), (dict(b1=None), INPUT),
    (dict(b2=None), INPUT), (dict(x=P + 4), CFG), (dict(h=P + 2), CFG), (dict(gate=P + 8), CFG), (dict(g1=P + 8), CFG), (dict(y=P + 2), CFG),
    (dict(rows=0), 0)])
def test_join_fwd_refuses(L, kw, want):
    a = dict(dtype=1, kind=0, rows=4, cols=64, eps=1e-5, scale=1.0, x=P, h=P, g1=P, b1=P, gate=P, rpg=2, g2=P, b2=P, xo=P, y=P, stats=P)
    a.update(kw)
    assert L.hift_k_join_fwd(a["dtype"], a["kind"], a["rows"], a["cols"], a["eps"], a["scale"], a["x"], a["h"], a["g1"], a["b1"],
                             a["gate"], a["rpg"], a["g2"], a["b2"], a["xo"], a["y"], a["stats"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), CFG), (dict(kind=-1), CFG), (dict(cols=4), CFG), (dict(cols=16392), CAPACITY), (dict(rpg=0), CFG),
    (dict(scale=float("nan")), CFG), (dict(dy=None), INPUT), (dict(xo=None), INPUT), (dict(h=None), INPUT), (dict(stats=None), INPUT),
    (dict(g2=None, dg2=None, db2=None, dxo=None), INPUT), (dict(dx=None), INPUT), (dict(dh=None), INPUT), (dict(scratch=None), INPUT),
    (dict(nbytes=0), CAPACITY), (dict(gate=None), INPUT), (dict(g1=None), INPUT), (dict(g2=None), INPUT), (dict(kind=1), INPUT),
    (dict(b1=None), INPUT), (dict(dxo=P + 4), CFG), (dict(dh=P + 8), CFG), (dict(scratch=P + 8), CFG)])
def test_join_bwd_refuses(L, kw, want):
    a = dict(dtype=1, kind=0, rows=4, cols=64, scale=1.0, dy=P, dxo=P, xo=P, h=P, stats=P, g1=P, b1=P, gate=P, rpg=2, g2=P, dx=P, dh=P,
             dg1=P, db1=P, dgate=P, dg2=P, db2=P, scratch=P, nbytes=1 << 30)
    a.update(kw)
    assert L.hift_k_join_bwd(a["dtype"], a["kind"], a["rows"], a["cols"], a["scale"], a["dy"], a["dxo"], a["xo"], a["h"], a["stats"],
                             a["g1"], a["b1"], a["gate"], a["rpg"], a["g2"], a["dx"], a["dh"], a["dg1"], a["db1"], a["dgate"], a["dg2"],
                             a["db2"], a["scratch"], a["nbytes"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), CFG), (dict(rows=0), CFG), (dict(cols=-3), CFG), (dict(rows=65537), CAPACITY), (dict(steps=0), CFG), (dict(steps=21), CFG),
    (dict(g=None), INPUT), (dict(o=None), INPUT), (dict(scratch=None), INPUT), (dict(scratch=P + 16), CFG), (dict(nbytes=64), CAPACITY),
    (dict(dtype=0, g=P + 2), CFG), (dict(o=P + 1), CFG)])
def test_orthogonalize_refuses(L, kw, want):
    a = dict(dtype=1, rows=4, cols=64, g=P, o=P, steps=5, scratch=P, nbytes=1 << 30)
    a.update(kw)
    assert L.hift_k_orthogonalize(a["dtype"], a["rows"], a["cols"], a["g"], a["o"], a["steps"], a["scratch"], a["nbytes"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(rows=0), CFG), (dict(lr=float("nan")), CFG), (dict(wd=float("inf")), CFG), (dict(mu=1.0), CFG), (dict(mu=-0.1), CFG),
    (dict(master=None), INPUT), (dict(grad=None), INPUT), (dict(mom=None), INPUT), (dict(master=P + 2), CFG), (dict(param=P + 1), CFG),
    (dict(nbytes=64), CAPACITY), (dict(steps=0), CFG)])
def test_muon_step_refuses(L, kw, want):
    a = dict(rows=4, cols=64, param=P, master=P, grad=P, mom=P, scratch=P, nbytes=1 << 30, lr=1e-3, mu=0.95, wd=0.0, steps=5)
    a.update(kw)
    assert L.hift_muon_step(a["rows"], a["cols"], a["param"], a["master"], a["grad"], a["mom"], a["scratch"], a["nbytes"], a["lr"],
                            a["mu"], 1, a["wd"], a["steps"], None) == want


def test_scratch_sizes(L):
    assert L.hift_orthogonalize_scratch_bytes(0, 5) == 0 and L.hift_orthogonalize_scratch_bytes(65537, 5) == 0
    for r, c in ((1, 1), (1000, 777), (777, 1000), (4096, 11008)):
        assert L.hift_orthogonalize_scratch_bytes(r, c) >= 4 * r * c
        assert L.hift_orthogonalize_scratch_bytes(r, c) == L.hift_orthogonalize_scratch_bytes(c, r)
    assert L.hift_join_bwd_scratch_bytes(0, 64, 1) == 0
    for rows in (1, 7, 1000, 70000):
        for rpg in (1, 3, 512, rows, rows + 5):
            assert L.hift_join_bwd_scratch_bytes(rows, 64, rpg) > 0
    # no rows per gate given means one gate
    assert L.hift_join_bwd_scratch_bytes(1000, 64, 0) == L.hift_join_bwd_scratch_bytes(1000, 64, 1000)


# ------------------------------------------------------------------ the 64-bit definitions themselves
def test_reference_gradient_of_logprobs_is_the_derivative():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 11)) * 2
    x[1, 4] = -np.inf
    tok, g, h, temp = np.array([3, 7, 0]), rng.standard_normal(3), rng.standard_normal(3), 0.7

    def f(z):
        lp, ent, *_ = R.token_logprobs(z, tok, temp, 0)
        return (g * lp + h * ent).sum()
    _, ent, st, _, _ = R.token_logprobs(x, tok, temp, 0)
    d = R.token_logprobs_bwd(x, tok, temp, st, ent, g, h, 11)
    for r in range(3):
        for c in range(11):
            if np.isneginf(x[r, c]):
                assert d[r, c] == 0
                continue
            e = np.zeros_like(x)
            e[r, c] = 1e-6
            assert abs((f(x + e) - f(x - e)) / 2e-6 - d[r, c]) < 1e-7


@pytest.mark.parametrize("kind", [0, 1])
def test_reference_gradient_of_the_junction_is_the_derivative(kind):
    rng = np.random.default_rng(1)
    rows, cols, rpg = 5, 8, 2
    v = {n: rng.standard_normal((rows, cols)) for n in ("x", "h")}
    v.update({n: 1 + 0.3 * rng.standard_normal(cols) for n in ("gain1", "bias1", "gain2", "bias2")})
    v["gate"] = rng.standard_normal((3, cols))
    dy, dxo = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))

    def f(w):
        xo, y, *_ = R.join_fwd(kind, 1e-5, 0.7, w["x"], w["h"], w["gain1"], w["bias1"], w["gate"], rpg, w["gain2"], w["bias2"])
        return (xo * dxo).sum() + (y * dy).sum()
    xo, y, st, _ = R.join_fwd(kind, 1e-5, 0.7, v["x"], v["h"], v["gain1"], v["bias1"], v["gate"], rpg, v["gain2"], v["bias2"])
    got = R.join_bwd(kind, 0.7, dy, dxo, xo, v["h"], st, v["gain1"], v["bias1"], v["gate"], rpg, v["gain2"])
    for n in v:
        if kind == 1 and n.startswith("bias"):
            continue
        for i in np.ndindex(v[n].shape):
            up, dn = ({m: t.copy() for m, t in v.items()} for _ in range(2))
            up[n][i] += 1e-6
            dn[n][i] -= 1e-6
            assert abs((f(up) - f(dn)) / 2e-6 - got["d" + n][i]) < 2e-6, (n, i)


def test_reference_orthogonalisation_maps_singular_values():
    rng = np.random.default_rng(2)
    for shape in ((6, 9), (9, 6), (1, 5), (5, 1)):
        g = rng.standard_normal(shape)
        u, s, vt = np.linalg.svd(g, full_matrices=False)
        s = s / np.linalg.norm(s)
        for _ in range(5):
            s = R.NS[0] * s + R.NS[1] * s ** 3 + R.NS[2] * s ** 5
        assert np.abs(R.orthogonalize(g) - (u * s) @ vt).max() < 1e-9


@pytest.mark.parametrize("rows,cols", [(1000, 16392), (1000, 2 ** 40), (1000, 2 ** 63 - 8), (2 ** 31, 64), (2 ** 62, 16384)])
def test_join_scratch_of_sizes_that_are_refused(L, rows, cols):
    """No size for rows and columns that the call does not take (their products wrapped around)."""
    assert L.hift_join_bwd_scratch_bytes(rows, cols, rows) == 0
    assert L.hift_join_bwd_scratch_bytes(1000, 16384, 1000) > 0


def test_current_stream_without_torchs_private_call(monkeypatch):
    """The stream of a call is torch's current one, also with a torch that lacks the private call which tells it sooner."""
    import types

    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    assert B._stream_ptr() == 103
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert B._stream_ptr() == 77


@pytest.mark.parametrize("steps,want", [(1, INPUT), (8, INPUT), (9, CFG), (20, CFG)])
def test_orthogonalisation_takes_eight_steps_at_most(L, steps, want):
    """Noise in directions that a matrix lacks grows by 3.44 a step, in fp32 too: more steps would keep no digit of a low-rank matrix.
    (INPUT: the scratch buffer is missing, which is looked at after the steps.)"""
    assert L.hift_k_orthogonalize(0, 4, 64, P, P, steps, None, 1 << 30, None) == want
    assert L.hift_muon_step(4, 64, P, P, P, P, None, 1 << 30, 1e-3, 0.95, 1, 0.0, steps, None) == want


@pytest.mark.parametrize("cols", [1, 4, 12, 4095])
def test_join_scratch_of_columns_that_are_refused(L, cols):
    """Columns that are no multiple of 8 have no size either."""
    assert L.hift_join_bwd_scratch_bytes(100, cols, 100) == 0
    assert L.hift_join_bwd_scratch_bytes(100, 8, 100) > 0


@pytest.mark.parametrize("name", ["tokens", "logp", "ent", "stats", "ids", "vals", "bad"])
def test_token_logprobs_refuses_displaced_buffers(L, name):
    """A buffer that does not start where its elements may is refused, not read."""
    assert _logp(L, **{name: P + 2}) == CFG


@pytest.mark.parametrize("name", ["tokens", "stats", "ent", "g", "h"])
def test_token_logprobs_bwd_refuses_displaced_buffers(L, name):
    a = dict(tokens=P, stats=P, ent=P, g=P, h=P)
    a[name] = P + 1
    assert L.hift_k_token_logprobs_bwd(1, 4, 100, 100, P, a["tokens"], 1.0, a["stats"], a["ent"], a["g"], a["h"], P, None) == CFG


def test_join_refuses_displaced_statistics_and_sums(L):
    assert L.hift_k_join_fwd(1, 0, 4, 64, 1e-5, 1.0, P, P, P, P, P, 2, P, P, P, P, P + 2, None) == CFG
    names = ("stats", "dg1", "db1", "dg2", "db2")
    for name in names:
        a = {n: P + 2 if n == name else P for n in names}
        assert L.hift_k_join_bwd(1, 0, 4, 64, 1.0, P, P, P, P, a["stats"], P, P, P, 2, P, P, P, a["dg1"], a["db1"], P, a["dg2"], a["db2"], P,
                                 1 << 30, None) == CFG, name
    assert L.hift_k_join_bwd(1, 0, 0, 64, 1.0, P, P, P, P, P, P, P, P, 2, P, P, P, P + 2, P, P, P, P, P, 1 << 30, None) == CFG


def test_factors_beyond_fp32_are_refused(L):
    """Finite numbers that the kernels' fp32 would hold as infinity: 0 times them would be NaN."""
    def join(scale, eps):
        return L.hift_k_join_fwd(1, 0, 4, 64, eps, scale, None, P, P, P, P, 2, P, P, P, P, P, None)
    assert join(-3e38, 1e38) == INPUT                       # (x is missing, which is looked at later)
    assert join(1e39, 1e-5) == CFG and join(-1e300, 1e-5) == CFG and join(1.0, 1e39) == CFG
    assert L.hift_k_join_bwd(1, 0, 4, 64, 1e39, P, P, P, P, P, P, P, P, 2, P, P, P, P, P, P, P, P, P, 1 << 30, None) == CFG

    def muon(lr, wd):
        return L.hift_muon_step(4, 64, P, None, P, P, P, 1 << 30, lr, 0.95, 1, wd, 5, None)
    assert muon(1e38, 0.0) == INPUT and muon(1e-3, 1e40) == INPUT
    assert muon(1e39, 0.0) == CFG and muon(2.2e38, 0.0) == CFG and muon(1e-3, 1e42) == CFG and muon(1e200, 1e200) == CFG
