"""The block operators beside the step on the GPU, against their 64-bit definitions: rotary positions, differential attention and
activations in 8 bits."""
import itertools

import pytest

import block_ops_ref as R

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def _torch():
    import torch
    return torch


def _types(code):
    torch = _torch()
    return torch.bfloat16 if code else torch.float32


# ------------------------------------------------------------------ differential attention
def _dattn_case(code, B, S, H, K, D, norm, seed, lens=None, spread=1.5):
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")             # noqa: E731
    qkv = rnd(B * S, (H + 2 * K) * D)
    qkv[:, :(H + K) * D] *= spread
    dt = _types(code)
    return dict(qkv=qkv.to(dt), lam=0.5 + 0.3 * rnd(H), gain=(1 + 0.2 * rnd(D)).to(dt) if norm else None,
                dy=rnd(B * S, H * D).to(dt), lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))


def _dattn_run(code, B, S, H, K, D, causal, s, eps=1e-5, c=0.4, back=True, o2=True):
    """Outputs in buffers of NaN with a guard row behind each."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    dt = _types(code)

    def new(rows, cols, dtype=dt):
        return torch.full((rows + 1, cols), NAN, dtype=dtype, device="cuda")

    T, norm = B * S, s["gain"] is not None
    out = {"o": new(T, H * D), "o2": new(T, H * D) if o2 else None, "y": new(T, H * D) if norm else None, "lse": new(2 * B * H, S, torch.float32)}
    args = (code, B, S, H, K, D, causal, s["qkv"], s["lam"], s["gain"], eps, c)
    P.k_diff_attention_fwd(*args, out["o"], out["o2"], out["y"], out["lse"], key_lens=s["lens"])
    if back:
        out.update(dqkv=new(T, (H + 2 * K) * D), dlam=new(1, H, torch.float32), dgain=new(1, D, torch.float32) if norm else None)
        w = torch.empty(P.diff_attention_bwd_scratch_bytes(code, B, S, H, D, norm), dtype=torch.uint8, device="cuda")
        P.k_diff_attention_bwd(*args, out["o"], out["o2"], out["lse"], s["dy"], out["dqkv"], out["dlam"], out["dgain"], w, key_lens=s["lens"])
    torch.cuda.synchronize()
    assert P.tc_error_flag() == 0
    for n, t in out.items():
        if t is not None:
            assert bool(t[-1].isnan().all()), n              # nothing behind the last row
            out[n] = t[:-1]
    return out


def _inside(got, want, bound, unit, name):
    """Every element within the bound and half a step of its own type."""
    torch = _torch()
    got = got.double()
    nan = want.isnan()
    assert bool((got.isnan() == nan).all()), name
    off = torch.where(nan, 0.0, (got - want).abs() - bound - unit * want.abs())
    assert float(off.max()) <= 1e-30, (name, float(off.max()), float((got - want).abs().nan_to_num().max()))


def _dattn_check(code, B, S, H, K, D, causal, s, eps=1e-5, c=0.4, back=True):
    torch = _torch()
    out = _dattn_run(code, B, S, H, K, D, causal, s, eps, c, back)
    d = {n: None if s[n] is None else R.f64(s[n]) for n in ("qkv", "lam", "gain", "dy")}
    u, unit = (R.UB, R.UB) if code else (0.0, 2 * R.U32)
    shape = (B, S, H, K, D, causal, s["lens"])
    o, o2, y, lse, b_o, b_o2, b_y, b_lse = R.dattn_fwd(d["qkv"], d["lam"], d["gain"], eps, c, *shape, u=u)
    _inside(out["o"], o, b_o, unit, "o")
    _inside(out["o2"], o2, b_o2, unit, "o2")
    if y is not None:
        _inside(out["y"], y, b_y, unit, "y")
    got = out["lse"].view(2, B, H, S).double()
    none = lse == -INF
    assert bool(((got == -INF) == none).all())
    assert float(torch.where(none, 0.0, (got - lse).abs()).max()) <= b_lse
    if not back:
        return out
    dqkv, dlam, dgain, bound, terms = R.dattn_bwd(d["qkv"], d["lam"], d["gain"], eps, c, R.f64(out["o"]), R.f64(out["o2"]), got, d["dy"], *shape, u=u)
    _inside(out["dqkv"], dqkv, bound, unit, "dqkv")
    # sums of n fp32 products: n roundings of the terms' sum at most, and the few of each term
    n = B * S * D
    assert bool(((out["dlam"][0].double() - dlam).abs() <= (n + 64) * R.U32 * terms + 1e-30).all())
    if dgain is not None:
        t = R.f64(s["dy"]).abs().view(-1, D).sum(0) * 2.0                   # |o r| is at most sqrt(D), mostly about 1
        assert bool(((out["dgain"][0].double() - dgain).abs() <= (B * S * H + 64) * R.U32 * t * D ** 0.5).all())
    return out


@pytest.mark.parametrize("code,D", [(0, 16), (0, 32), (0, 64), (0, 128), (1, 16), (1, 32), (1, 64), (1, 128)])
@pytest.mark.parametrize("B,S,H,K,causal,norm,lens", [
    (1, 1, 1, 1, True, True, None), (2, 3, 2, 1, False, False, None), (1, 64, 2, 2, True, True, None), (3, 65, 3, 1, True, False, [65, 1, 0]),
    (2, 127, 4, 2, False, True, [127, 100]), (2, 128, 2, 2, True, False, [128, 64]), (1, 129, 2, 2, True, True, None),
    (2, 200, 2, 1, False, True, [0, 129]), (1, 300, 4, 4, True, True, [257])])
def test_differential_attention(code, D, B, S, H, K, causal, norm, lens):
    s = _dattn_case(code, B, S, H, K, D, norm, B * S + D, lens)
    _dattn_check(code, B, S, H, K, D, causal, s, back=code == 0 or D < 64 or BACK_TC)


BACK_TC = True
