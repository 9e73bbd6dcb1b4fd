"""What the block operators beside the step refuse, the sizes they report, and their 64-bit definitions against differences: host logic, no
GPU needed (a call that is refused launches nothing, so the pointers below are never read)."""
import math

import pytest
import torch

import block_ops_ref as R
from paper_2401_15207_b200 import binding as B, build

CFG, INPUT, CAPACITY = 1, 4, 8
P = 1 << 20            # a well-aligned address that nothing reads
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.load_library()


@pytest.mark.parametrize("kw,want", [
    (dict(kind=5), CFG), (dict(kind=-1), CFG), (dict(n=-1), CFG), (dict(n=1 << 31), CFG), (dict(rot=3), CFG), (dict(rot=0), CFG), (dict(base=1.0), CFG),
    (dict(base=NAN), CFG), (dict(base=INF), CFG), (dict(kind=1, factor=0.5), CFG), (dict(kind=2, factor=INF), CFG), (dict(kind=3, orig=0.0), CFG),
    (dict(kind=4, slow=0.0), CFG), (dict(kind=3, slow=32.0), CFG), (dict(kind=3, fast=INF), CFG), (dict(cs=None), INPUT), (dict(cs=P + 2), CFG),
    (dict(n=0, cs=None), 0)])
def test_rope_table_refuses(L, kw, want):
    a = dict(kind=0, n=16, rot=8, base=1e4, factor=4.0, orig=512.0, fast=32.0, slow=1.0, cs=P)
    a.update(kw)
    assert L.hift_rope_table(a["kind"], a["n"], a["rot"], a["base"], a["factor"], a["orig"], a["fast"], a["slow"], a["cs"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), CFG), (dict(layout=2), CFG), (dict(rows=-1), CFG), (dict(rows=1 << 31), CFG), (dict(heads=0), CFG), (dict(d=1), CFG),
    (dict(rot=7), CFG), (dict(rot=18), CFG), (dict(rot=0), CFG), (dict(ld=31), CFG), (dict(ldo=31), CFG), (dict(n_pos=0), CFG), (dict(seq=0), CFG),
    (dict(seq=17), CFG), (dict(heads=1 << 20, ld=1 << 30, ldo=1 << 30), CAPACITY), (dict(x=None), INPUT), (dict(out=None), INPUT), (dict(cs=None), INPUT),
    (dict(x=P + 1), CFG), (dict(dtype=0, out=P + 2), CFG), (dict(cs=P + 2), CFG), (dict(pos=P + 2), CFG), (dict(bad=P + 1), CFG),
    (dict(out=P, ldo=48), CFG), (dict(rows=0, x=None, out=None, cs=None), 0)])
def test_rope_refuses(L, kw, want):
    a = dict(dtype=1, layout=0, rows=4, heads=2, d=16, rot=16, x=P, ld=32, out=2 * P, ldo=32, cs=P, n_pos=16, seq=16, pos=None, inv=0, bad=None)
    a.update(kw)
    assert L.hift_k_rope(a["dtype"], a["layout"], a["rows"], a["heads"], a["d"], a["rot"], a["x"], a["ld"], a["out"], a["ldo"], a["cs"], a["n_pos"],
                         a["seq"], a["pos"], a["inv"], a["bad"], None) == want


DATTN = [(dict(dtype=2), CFG), (dict(B=-1), CFG), (dict(S=-1), CFG), (dict(H=0), CFG), (dict(K=0), CFG), (dict(H=4, K=3), CFG), (dict(D=48), CFG),
         (dict(D=256), CFG), (dict(eps=0.0), CFG), (dict(eps=NAN), CFG), (dict(eps=1e-42), CFG), (dict(c=INF), CFG), (dict(B=1 << 16, S=1 << 16), CAPACITY),
         (dict(H=1 << 26, K=1 << 26), CAPACITY), (dict(B=1 << 20, S=64, H=1 << 12, K=1 << 12, D=16), CAPACITY), (dict(qkv=None), INPUT), (dict(lam=None), INPUT),
         (dict(o=None), INPUT), (dict(lse=None), INPUT), (dict(qkv=P + 1), CFG), (dict(lam=P + 2), CFG), (dict(lse=P + 2), CFG), (dict(lens=P + 2), CFG),
         (dict(dtype=0, o=P + 2), CFG), (dict(gain=P + 1), CFG)]


@pytest.mark.parametrize("kw,want", DATTN + [(dict(y=None), INPUT), (dict(gain=None), INPUT), (dict(gain=None, y=None, eps=0.0, B=0), 0), (dict(S=0, qkv=None), 0)])
def test_diff_attention_fwd_refuses(L, kw, want):
    a = dict(dtype=1, B=2, S=8, H=4, K=2, D=64, qkv=P, lam=P, gain=P, eps=1e-5, c=0.5, o=P, o2=P, y=P, lse=P, lens=None)
    a.update(kw)
    assert L.hift_k_diff_attention_fwd(a["dtype"], a["B"], a["S"], a["H"], a["K"], a["D"], 1, a["qkv"], a["lam"], a["gain"], a["eps"], a["c"], a["o"],
                                       a["o2"], a["y"], a["lse"], a["lens"], None) == want


@pytest.mark.parametrize("kw,want", DATTN + [(dict(o2=None), INPUT), (dict(dy=None), INPUT), (dict(dqkv=None), INPUT), (dict(scratch=None), INPUT),
                                             (dict(gain=None), INPUT), (dict(scratch=P + 16), CFG), (dict(nbytes=100), CAPACITY), (dict(dlam=P + 2), CFG),
                                             (dict(dqkv=P + 1), CFG), (dict(B=0, dlam=None, dgain=None), 0)])
def test_diff_attention_bwd_refuses(L, kw, want):
    a = dict(dtype=1, B=2, S=8, H=4, K=2, D=64, qkv=P, lam=P, gain=P, eps=1e-5, c=0.5, o=P, o2=P, lse=P, dy=P, dqkv=P, dlam=P, dgain=P, scratch=P,
             nbytes=1 << 40, lens=None)
    a.update(kw)
    assert L.hift_k_diff_attention_bwd(a["dtype"], a["B"], a["S"], a["H"], a["K"], a["D"], 1, a["qkv"], a["lam"], a["gain"], a["eps"], a["c"], a["o"],
                                       a["o2"], a["lse"], a["dy"], a["dqkv"], a["dlam"], a["dgain"], a["scratch"], a["nbytes"], a["lens"], None) == want


def test_diff_attention_scratch(L):
    f = L.hift_diff_attention_bwd_scratch_bytes
    assert f(1, 0, 8, 4, 64, 1) == 0 and f(1, 2, 8, 4, 48, 1) == 0 and f(2, 2, 8, 4, 64, 1) == 0
    for B_, S, H, D in ((1, 1, 1, 16), (2, 131, 4, 32), (8, 512, 20, 64), (1, 4096, 16, 128)):
        for code in (0, 1):
            plain, norm = f(code, B_, S, H, D, 0), f(code, B_, S, H, D, 1)
            assert plain >= 8 * B_ * H * S and norm >= plain + B_ * S * H * D * (2 if code else 4) and norm % 256 == 0


@pytest.mark.parametrize("kw,want", [(dict(H=0), CFG), (dict(d=0), CFG), (dict(sets=2), CFG), (dict(init=INF), CFG), (dict(w=None), INPUT), (dict(lam=None), INPUT),
                                     (dict(w=P + 2), CFG)])
def test_diff_lambda_refuses(L, kw, want):
    a = dict(H=4, sets=1, d=8, init=0.8, w=P, lam=P)
    a.update(kw)
    assert L.hift_k_diff_lambda(a["H"], a["sets"], a["d"], a["init"], a["w"], a["lam"], None) == want
    if "init" not in kw:
        assert L.hift_k_diff_lambda_bwd(a["H"], a["sets"], a["d"], a["w"], a["lam"], P, None) == want


@pytest.mark.parametrize("kw,want", [(dict(dtype=2), CFG), (dict(fmt=2), CFG), (dict(rows=-1), CFG), (dict(rows=1 << 31), CFG), (dict(f=0), CFG),
                                     (dict(f=(1 << 23) + 1), CAPACITY), (dict(x=None), INPUT), (dict(q=None), INPUT), (dict(s=None), INPUT), (dict(x=P + 1), CFG),
                                     (dict(rows=0, x=None, q=None, s=None), 0)])
def test_act8_refuses(L, kw, want):
    a = dict(dtype=1, fmt=0, rows=4, f=40, x=P, q=P, s=P)
    a.update(kw)
    ld = max(a["f"], 1)
    assert L.hift_k_act8_pack(a["dtype"], a["fmt"], a["rows"], a["f"], a["x"], ld, a["q"], a["s"], None) == want
    assert L.hift_k_act8_unpack(a["dtype"], a["fmt"], a["rows"], a["f"], a["q"], a["s"], a["x"], ld, None) == want
    for kind in (1, 2):
        assert L.hift_k_act8_fwd(a["dtype"], a["fmt"], kind, a["rows"], a["f"], a["x"], P, a["q"], a["s"], None) == want
        assert L.hift_k_act8_bwd(a["dtype"], a["fmt"], kind, a["rows"], a["f"], P, a["q"], a["s"], a["x"], None, None) == want
    if not kw:
        return
    good = dict(dtype=1, fmt=0, rows=4, f=40)
    assert L.hift_k_act8_pack(*good.values(), P, 39, P, P, None) == CFG
    assert L.hift_k_act8_unpack(*good.values(), P, P, P, 39, None) == CFG
    for kind in (0, 3):
        assert L.hift_k_act8_fwd(1, 0, kind, 4, 40, P, P, P, P, None) == CFG
        assert L.hift_k_act8_bwd(1, 0, kind, 4, 40, P, P, P, P, None, None) == CFG
    assert L.hift_k_act8_fwd(1, 0, 1, 4, 40, P, None, P, P, None) == INPUT
    assert L.hift_k_act8_bwd(1, 0, 1, 4, 40, None, P, P, P, None, None) == INPUT
    assert L.hift_k_act8_bwd(1, 0, 1, 4, 40, P, P, P, P, P + 1, None) == CFG


# ------------------------------------------------------------------ the 64-bit definitions themselves
def _dd(f, x, v, h=1e-6):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("H,K,causal,norm,lens", [(2, 1, True, True, None), (2, 2, False, False, [5, 3]), (4, 2, True, True, [0, 7])])
def test_reference_gradient_of_differential_attention_is_the_derivative(H, K, causal, norm, lens):
    B_, S, D = 2, 7, 8
    g = torch.Generator().manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)       # noqa: E731
    qkv, lam, gain, dy = rnd(B_ * S, (H + 2 * K) * D), rnd(H), (rnd(D) if norm else None), rnd(B_ * S, H * D)
    lens = None if lens is None else torch.tensor(lens)

    def out(x, la, ga):
        o, o2, y, lse, *_ = R.dattn_fwd(x, la, ga, 1e-3, 0.4, B_, S, H, K, D, causal, lens)
        return (dy * (y if norm else o)).sum(), o, o2, lse
    _, o, o2, lse = out(qkv, lam, gain)
    dqkv, dlam, dgain, _, _ = R.dattn_bwd(qkv, lam, gain, 1e-3, 0.4, o, o2, lse, dy, B_, S, H, K, D, causal, lens)
    v = rnd(*qkv.shape)
    assert float((dqkv * v).sum()) == pytest.approx(float(_dd(lambda x: out(x, lam, gain)[0], qkv, v)), rel=1e-6)
    v = rnd(H)
    assert float((dlam * v).sum()) == pytest.approx(float(_dd(lambda x: out(qkv, x, gain)[0], lam, v)), rel=1e-6)
    if norm:
        v = rnd(D)
        assert float((dgain * v).sum()) == pytest.approx(float(_dd(lambda x: out(qkv, lam, x)[0], gain, v)), rel=1e-6)


@pytest.mark.parametrize("layout", [0, 1])
def test_reference_rotation_keeps_lengths_and_its_inverse_is_its_transpose(layout):
    g = torch.Generator().manual_seed(1)
    x, y = torch.randn(5, 24, generator=g, dtype=torch.float64), torch.randn(5, 24, generator=g, dtype=torch.float64)
    cs, pos = R.rope_table(9, 6), torch.tensor([0, 8, 3, 11, -1])
    rx = R.rope(x, layout, 2, 12, 6, cs, pos, False)
    assert torch.allclose((rx ** 2).sum(1), (x ** 2).sum(1)) and torch.equal(rx[3:], x[3:])
    assert torch.allclose((rx * y).sum(), (x * R.rope(y, layout, 2, 12, 6, cs, pos, True)).sum())


def test_reference_rope_scalings():
    plain, _ = R.rope_frequencies(64, 1e4)
    lin, _ = R.rope_frequencies(64, 1e4, scaling=1, factor=4.0)
    ntk, _ = R.rope_frequencies(64, 1e4, scaling=2, factor=4.0)
    yarn, mag = R.rope_frequencies(64, 1e4, scaling=3, factor=4.0, orig_len=2048.0)
    band, _ = R.rope_frequencies(64, 1e4, scaling=4, factor=4.0, orig_len=2048.0, fast=4.0, slow=1.0)
    assert lin == [f / 4 for f in plain] and ntk[0] == plain[0] and ntk[-1] == pytest.approx(plain[-1] / 4)
    for f in (yarn, band):
        assert f[0] == plain[0] and f[-1] == pytest.approx(plain[-1] / 4) and all(p / 4 * 0.999 <= x <= p * 1.001 for x, p in zip(f, plain))
    assert mag == pytest.approx(1 + 0.1 * math.log(4.0))


@pytest.mark.parametrize("kind", [1, 2])
def test_reference_activation_derivatives(kind):
    x = torch.linspace(-6, 6, 26, dtype=torch.float64)[None]
    v = torch.cos(3 * x)
    _, parts = R.activation(kind, x)
    d = (torch.cat(parts, 1) if kind == 2 else parts[0]) * v
    got = d.sum() if kind == 1 else (d[:, :13] + d[:, 13:]).sum()
    assert float(got) == pytest.approx(float(_dd(lambda z: R.activation(kind, z)[0].sum(), x, v)), rel=1e-6)


def test_reference_packing():
    x = torch.zeros(1, 70, dtype=torch.float64)
    x[0, :3] = torch.tensor([127.0, -63.5, 0.5])
    x[0, 32:35] = torch.tensor([127.5, 1.0, 3.0])
    x[0, 64] = INF
    q, b = R.pack(x, 0)
    assert q[0, :3].tolist() == [127, -64, 0] and b[0].tolist() == [127, 128, 255] and q[0, 32:35].tolist() == [64, 0, 2] and q[0, 64] == 0
    assert bool(R.unpack(q, b)[0, 64:].isnan().all())
    x[0, :2], x[0, 64] = torch.tensor([448.0, 449.0]), 2.0 ** -130
    q, b = R.pack(x, 1)
    assert b[0].tolist() == [128, 126, 17] and q[0, :2].tolist() == [224, 224] and q[0, 64] == 0
