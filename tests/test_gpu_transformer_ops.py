"""The block operators beside the step on the GPU, against their 64-bit definitions: rotary positions, differential attention and
activations in 8 bits."""
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
    _dattn_check(code, B, S, H, K, D, causal, s)


@pytest.mark.parametrize("code,D", [(0, 32), (1, 64), (1, 128)])
def test_differential_attention_long(code, D):
    """Many key blocks, grouped heads, lengths inside a tile, several items for a CTA."""
    B, S, H, K = (1, 700, 4, 1) if code == 0 else (2, 1500, 24, 6)
    s = _dattn_case(code, B, S, H, K, D, True, 3, [S - 37, S - 200][:B])
    _dattn_check(code, B, S, H, K, D, True, s)


@pytest.mark.parametrize("code,D", [(0, 32), (1, 64), (1, 128)])
@pytest.mark.parametrize("spread", [0.0, 12.0])
def test_differential_attention_flat_and_sharp_maps(code, D, spread):
    """All scores equal, and scores of hundreds, where the running maximum jumps and one key takes nearly all."""
    s = _dattn_case(code, 2, 190, 2, 1, D, False, 4, [190, 77], spread)
    _dattn_check(code, 2, 190, 2, 1, D, False, s)


@pytest.mark.parametrize("code,D", [(0, 64), (1, 64), (1, 128)])
def test_differential_attention_rising_maximum(code, D):
    """Every later key scores far more than all before it: the accumulators are rescaled in every block."""
    torch = _torch()
    B, S, H, K = 1, 520, 2, 2
    s = _dattn_case(code, B, S, H, K, D, True, 5)
    ramp = torch.arange(S, device="cuda")[:, None] / 8.0
    s["qkv"].view(S, H + 2 * K, D)[:, :H] = 1.0
    s["qkv"].view(S, H + 2 * K, D)[:, H:H + K] = (ramp / (D / 2) ** 0.5)[:, None].to(s["qkv"].dtype)
    _dattn_check(code, B, S, H, K, D, False, s)


@pytest.mark.parametrize("code,D", [(0, 64), (1, 64), (1, 128)])
def test_differential_attention_bad_values_stay_in_their_entry(code, D):
    """NaN and infinity in one batch entry leave the others as they are, bit for bit, where tiles reach beyond an entry's end."""
    torch = _torch()
    B, S, H, K = 3, 100, 2, 1
    s = _dattn_case(code, B, S, H, K, D, True, 6, [100, 100, 60])
    clean = _dattn_run(code, B, S, H, K, D, True, s)
    s["qkv"][S + 3:S + 40] = NAN
    s["qkv"][S + 50] = INF
    got = _dattn_run(code, B, S, H, K, D, True, s)
    for n in ("o", "o2", "y", "dqkv"):
        for b in (0, 2):
            assert torch.equal(got[n][b * S:(b + 1) * S], clean[n][b * S:(b + 1) * S]), (n, b)
        assert bool(got[n][S + 60:2 * S].isnan().any())


@pytest.mark.parametrize("code,D", [(0, 32), (0, 64), (1, 32), (1, 64), (1, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_differential_attention_whatever_padded_keys_hold(code, D, causal):
    """NaN and infinity in k and v at padded keys change no bit of any output; lengths of 0, inside a tile, at its end, and whole."""
    torch = _torch()
    B, S, H, K = 5, 210, 4, 2
    lens = [0, 70, 128, 210, 1]
    s = _dattn_case(code, B, S, H, K, D, True, 14, lens)
    kv = s["qkv"].view(B, S, H + 2 * K, D)[:, :, H:]
    clean = _dattn_run(code, B, S, H, K, D, causal, s)
    for b, n in enumerate(lens):
        kv[b, n:] = NAN
        kv[b, n + 1::3] = INF
    got = _dattn_run(code, B, S, H, K, D, causal, s)
    for n in got:
        assert torch.equal(got[n], clean[n]), n


@pytest.mark.parametrize("code,D", [(0, 32), (1, 32), (1, 64), (1, 128)])
def test_differential_attention_repeats_its_bits(code, D):
    torch = _torch()
    s = _dattn_case(code, 3, 333, 8, 2, D, True, 7, [333, 1, 200])
    a = _dattn_run(code, 3, 333, 8, 2, D, True, s)
    for _ in range(3):
        b = _dattn_run(code, 3, 333, 8, 2, D, True, s)
        for n in a:
            assert torch.equal(a[n].nan_to_num(7.0), b[n].nan_to_num(7.0)), n


@pytest.mark.parametrize("D", [64, 128])
def test_differential_attention_without_what_it_need_not_write(D):
    """No o_2 (nothing will be differentiated), no dlambda and dgain; and the same bits as with them."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    for code in (0, 1):
        for norm in (False, True):
            B, S, H, K = 2, 150, 2, 2
            s = _dattn_case(code, B, S, H, K, D, norm, 8)
            a = _dattn_run(code, B, S, H, K, D, True, s)
            b = _dattn_run(code, B, S, H, K, D, True, s, back=False, o2=False)
            assert torch.equal(a["o"], b["o"]) and (not norm or torch.equal(a["y"], b["y"]))
            w = torch.empty(P.diff_attention_bwd_scratch_bytes(code, B, S, H, D, norm), dtype=torch.uint8, device="cuda")
            dqkv = torch.empty_like(s["qkv"])
            P.k_diff_attention_bwd(code, B, S, H, K, D, True, s["qkv"], s["lam"], s["gain"], 1e-5, 0.4, a["o"], a["o2"], a["lse"], s["dy"], dqkv, None, None, w)
            assert torch.equal(dqkv, a["dqkv"])


@pytest.mark.parametrize("D", [64, 128])
def test_differential_attention_off_the_16_byte_grid(D):
    """bf16 buffers that start at any element take the CUDA-core kernels."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    B, S, H, K = 2, 70, 2, 1
    s = _dattn_case(1, B, S, H, K, D, True, 9, [70, 33])
    n = s["qkv"].numel()
    flat = torch.empty(n + 1, dtype=torch.bfloat16, device="cuda")
    flat[1:] = s["qkv"].flatten()
    s["qkv"] = flat[1:].view(B * S, -1)
    assert s["qkv"].data_ptr() % 16 == 2
    _dattn_check(1, B, S, H, K, D, True, s)
    assert P.tc_error_flag() == 0


@pytest.mark.parametrize("code,D", [(0, 32), (1, 64), (1, 128)])
@pytest.mark.parametrize("norm", [False, True])
def test_differential_attention_every_buffer_off_the_grid(code, D, norm):
    """Every buffer one element behind a 16-byte boundary; and each alone, the others on it, with the same results within the types' roundings."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    B, S, H, K, dt = 2, 90, 2, 1, _types(code)
    s = _dattn_case(code, B, S, H, K, D, norm, 15, [90, 41])
    T = B * S
    w = torch.empty(P.diff_attention_bwd_scratch_bytes(code, B, S, H, D, norm), dtype=torch.uint8, device="cuda")

    def run(shifted):
        def at(name, shape, src=None, dtype=dt):
            n = int(torch.Size(shape).numel())
            k = 1 if name in shifted else 0
            t = torch.full((n + 8,), 3.0, dtype=dtype, device="cuda")[k:k + n].view(shape)
            if src is not None:
                t.copy_(src)
            return t
        qkv, dy = at("qkv", s["qkv"].shape, s["qkv"]), at("dy", s["dy"].shape, s["dy"])
        gain = at("gain", (D,), s["gain"]) if norm else None
        lam = at("lam", (H,), s["lam"], torch.float32)
        o, o2 = at("o", (T, H * D)), at("o2", (T, H * D))
        y = at("y", (T, H * D)) if norm else None
        lse, dlam = at("lse", (2 * B * H, S), dtype=torch.float32), at("dlam", (H,), dtype=torch.float32)
        dgain = at("dgain", (D,), dtype=torch.float32) if norm else None
        dqkv = at("dqkv", s["qkv"].shape)
        args = (code, B, S, H, K, D, True, qkv, lam, gain, 1e-5, 0.4)
        P.k_diff_attention_fwd(*args, o, o2, y, lse, key_lens=s["lens"])
        P.k_diff_attention_bwd(*args, o, o2, lse, dy, dqkv, dlam, dgain, w, key_lens=s["lens"])
        torch.cuda.synchronize()
        return [t.double() for t in (o, o2, y, lse, dqkv, dlam, dgain) if t is not None]
    names = ["qkv", "dy", "gain", "lam", "o", "o2", "y", "lse", "dlam", "dgain", "dqkv"]
    want = run([])
    for shifted in [names] + [[n] for n in names]:
        for g, r in zip(run(shifted), want):
            # the tensor cores' way and the CUDA cores' differ by roundings of P, dS and the results: a few half steps of the type, relative to the whole
            assert float((g - r).norm()) <= (4 * R.UB if code else 1e-5) * float(r.norm()), shifted


@pytest.mark.parametrize("D", [64, 128])
def test_differential_attention_of_9001_tokens(D):
    s = _dattn_case(1, 1, 9001, 1, 1, D, True, 16, [8900])
    _dattn_check(1, 1, 9001, 1, 1, D, True, s)


def test_differential_attention_beyond_2_31_elements():
    """The last entry of a batch whose qkv has more than 2^31 elements, against the same entry alone."""
    torch = _torch()
    B, S, H, K, D = 90, 1024, 64, 64, 128
    assert (B - 1) * S * (H + 2 * K) * D > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(10)
    one = torch.randn(S, (H + 2 * K) * D, generator=g, device="cuda").to(torch.bfloat16)
    dy1 = torch.randn(S, H * D, generator=g, device="cuda").to(torch.bfloat16)
    s = dict(qkv=torch.zeros(B * S, (H + 2 * K) * D, dtype=torch.bfloat16, device="cuda"), lam=torch.rand(H, generator=g, device="cuda"), gain=None, lens=None,
             dy=torch.zeros(B * S, H * D, dtype=torch.bfloat16, device="cuda"))
    s["qkv"][-S:], s["dy"][-S:] = one, dy1
    big = _dattn_run(1, B, S, H, K, D, True, s)
    last = {n: big[n][-S:].clone() for n in ("o", "o2", "dqkv")}
    del big
    small = _dattn_run(1, 1, S, H, K, D, True, dict(s, qkv=one, dy=dy1))
    for n in last:
        assert torch.equal(last[n], small[n]), n


@pytest.mark.parametrize("code,D", [(0, 32), (1, 64), (1, 128)])
def test_differential_attention_captured_and_on_two_streams(code, D):
    """Two graphs that share the scratch buffer, replayed behind one another; then both calls at once on two streams with scratch of their own."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    B, S, H, K = 2, 260, 4, 2
    cases = [_dattn_case(code, B, S, H, K, D, True, i, [260, 130 + i]) for i in (11, 12)]
    want = [_dattn_run(code, B, S, H, K, D, True, s) for s in cases]
    nbytes = P.diff_attention_bwd_scratch_bytes(code, B, S, H, D, True)
    dt = _types(code)

    def buffers():
        return dict(o=torch.empty(B * S, H * D, dtype=dt, device="cuda"), o2=torch.empty(B * S, H * D, dtype=dt, device="cuda"),
                    y=torch.empty(B * S, H * D, dtype=dt, device="cuda"), lse=torch.empty(2 * B * H, S, device="cuda"),
                    dqkv=torch.empty(B * S, (H + 2 * K) * D, dtype=dt, device="cuda"), dlam=torch.empty(1, H, device="cuda"), dgain=torch.empty(1, D, device="cuda"))

    def calls(s, b, w, stream=None):
        args = (code, B, S, H, K, D, True, s["qkv"], s["lam"], s["gain"], 1e-5, 0.4)
        P.k_diff_attention_fwd(*args, b["o"], b["o2"], b["y"], b["lse"], key_lens=s["lens"], stream=stream)
        P.k_diff_attention_bwd(*args, b["o"], b["o2"], b["lse"], s["dy"], b["dqkv"], b["dlam"], b["dgain"], w, key_lens=s["lens"], stream=stream)
    shared = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    outs, graphs = [buffers(), buffers()], []
    for s, b in zip(cases, outs):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            calls(s, b, shared)
        graphs.append(gr)
    for _ in range(2):
        for b in outs:
            for t in b.values():
                t.fill_(NAN)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for w, b in zip(want, outs):
            for n in b:
                assert torch.equal(b[n], w[n]), n
    streams = [torch.cuda.Stream() for _ in cases]
    own = [torch.empty(nbytes, dtype=torch.uint8, device="cuda") for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, b, w, st in zip(cases, outs, own, streams):
            calls(s, b, w, st.cuda_stream)
    torch.cuda.synchronize()
    for w, b in zip(want, outs):
        for n in b:
            assert torch.equal(b[n], w[n]), n


@pytest.mark.parametrize("D", [64, 128])
def test_differential_attention_after_a_time_out(D):
    """With the tensor-core time-out flag raised nothing is written by the tensor-core kernels; cleared, the calls work again."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    s = _dattn_case(1, 1, 140, 2, 1, D, False, 13)
    o, o2 = (torch.full((140, 2 * D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros(2, 2, 140, device="cuda")
    assert P.tc_error_flag(1) == 1
    try:
        P.k_diff_attention_fwd(1, 1, 140, 2, 1, D, True, s["qkv"], s["lam"], None, 1e-5, 1.0, o, o2, None, lse)
        w = torch.empty(P.diff_attention_bwd_scratch_bytes(1, 1, 140, 2, D, False), dtype=torch.uint8, device="cuda")
        dqkv = torch.full_like(s["qkv"], 7.0)
        P.k_diff_attention_bwd(1, 1, 140, 2, 1, D, True, s["qkv"], s["lam"], None, 1e-5, 1.0, o, o2, lse, s["dy"], dqkv, None, None, w)
        torch.cuda.synchronize()
        assert bool((o == 7).all()) and bool((o2 == 7).all()) and bool((dqkv == 7).all())
    finally:
        assert P.tc_error_flag(0) == 0
    _dattn_check(1, 1, 140, 2, 1, D, True, s)


@pytest.mark.parametrize("H,sets,d", [(1, 1, 1), (5, 1, 33), (12, 12, 64), (70, 1, 100)])
def test_diff_lambda(H, sets, d):
    import paper_2401_15207_b200 as P
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(d)
    w = torch.randn(4, sets, d, generator=g, device="cuda") * 0.3
    lam, dw, dlam = torch.empty(H, device="cuda"), torch.full_like(w, NAN), torch.randn(H, generator=g, device="cuda")
    P.k_diff_lambda(H, sets, d, 0.8, w, lam)
    P.k_diff_lambda_bwd(H, sets, d, w, dlam, dw)
    x = w.double().requires_grad_()
    e1, e2 = torch.exp((x[0] * x[1]).sum(1)), torch.exp((x[2] * x[3]).sum(1))
    want = (e1 - e2 + 0.8).expand(H)
    grad, = torch.autograd.grad(want, x, dlam.double())
    # the exponent: d roundings of its terms' sum, an exponential's error of two steps; a difference and a sum behind it
    rel = (d * R.U32 * ((w[0] * w[1]).abs().sum(1) + (w[2] * w[3]).abs().sum(1)).double() + 8 * R.U32).max()
    assert bool(((lam.double() - want).abs() <= rel * (e1 + e2 + 1).max()).all())
    size = dlam.abs().double().sum() if sets == 1 else dlam.abs().double().max()
    assert bool(((dw.double() - grad).abs() <= (rel + H * R.U32) * size * torch.maximum(e1, e2).max() * w.abs().max()).all())


# ------------------------------------------------------------------ rotary positions
def _rope_table(n_pos, rot, **kw):
    import paper_2401_15207_b200 as P
    torch = _torch()
    cs = torch.full((2, n_pos, rot // 2), NAN, device="cuda")
    P.rope_table(n_pos, rot, cs, **kw)
    return cs


@pytest.mark.parametrize("kw", [dict(), dict(base=5e5), dict(scaling=1, factor=4.0), dict(scaling=2, factor=8.0),
                                dict(scaling=3, factor=4.0, orig_len=2048.0), dict(scaling=3, factor=16.0, orig_len=4096.0, fast=8.0, slow=0.5),
                                dict(scaling=4, factor=8.0, orig_len=8192.0, fast=4.0, slow=1.0)])
@pytest.mark.parametrize("n_pos,rot", [(1, 2), (77, 6), (5000, 64), (300000, 128)])
def test_rope_table(kw, n_pos, rot):
    """Angles in 64 bits: one rounding of cosine and sine, also far out; the definition's own angles differ by 64-bit roundings of pow (1e-14 relative)."""
    torch = _torch()
    got, want = _rope_table(n_pos, rot, **kw).double().cpu(), R.rope_table(n_pos, rot, **kw)
    assert float((got - want).abs().max()) <= 1.5 * 2 * R.U32 + 1e-13 * n_pos
    assert bool(torch.isfinite(got).all())


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("rows,heads,d,rot,pad", [(1, 1, 2, 2, 0), (3, 5, 7, 6, 1), (130, 3, 80, 40, 0), (64, 8, 128, 128, 128), (65, 9, 64, 32, 64), (33, 2, 96, 18, 3),
                                                  (1000, 12, 64, 64, 8), (3000, 40, 128, 64, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rope(code, layout, rows, heads, d, rot, pad, in_place):
    import paper_2401_15207_b200 as P
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    n_pos = 50
    ld, width = heads * d + pad, heads * d
    x = torch.randn(rows, ld, generator=g, device="cuda").to(_types(code))
    pos = torch.randint(-3, n_pos + 3, (rows,), generator=g, device="cuda", dtype=torch.int32) if rows > 1 else None
    cs = _rope_table(n_pos, rot)
    for inverse in (False, True):
        for p in (pos, None):
            src = x.clone()
            out = src if in_place else torch.full((rows, width + 5), NAN, dtype=x.dtype, device="cuda")
            bad = torch.zeros(1, dtype=torch.int32, device="cuda")
            P.k_rope(code, layout, rows, heads, d, rot, src, ld, out, ld if in_place else width + 5, cs, n_pos, seq=37, positions=p, inverse=inverse, bad=bad)
            at = torch.arange(rows, device="cuda") % 37 if p is None else p
            want = R.rope(x.double(), layout, heads, d, rot, cs.double(), at, inverse)
            got = out[:, :width].double()
            # two fp32 products and a sum: three half steps of fp32 of the terms; one of the result's own type
            half = R.rope(x.double().abs(), layout, heads, d, rot, torch.stack([cs[0].double().abs(), -cs[1].double().abs()]), at, False).abs()
            terms = half + x[:, :width].double().abs() * 2
            assert bool(((got - want).abs() <= 3 * R.U32 * terms + (R.UB if code else R.U32) * want.abs() * 1.001).all())
            assert int(bad) == int(p is not None and bool(((p < 0) | (p >= n_pos)).any()))
            rest = out[:, width:]
            assert torch.equal(rest, x[:, width:]) if in_place else bool(rest.isnan().all())
            keep = torch.arange(heads * d, device="cuda") % d >= rot
            assert torch.equal(out[:, :width][:, keep], x[:, :width][:, keep])


@pytest.mark.parametrize("shift", [1, 2, 4])
def test_rope_off_the_16_byte_grid(shift):
    import paper_2401_15207_b200 as P
    torch = _torch()
    cs = _rope_table(64, 64)
    base = torch.randn(40 * 256 + 8, device="cuda").to(torch.bfloat16)
    x = base[shift:shift + 40 * 256].view(40, 256)
    a, b = torch.empty(40, 256, dtype=torch.bfloat16, device="cuda"), torch.empty(40, 256, dtype=torch.bfloat16, device="cuda")
    P.k_rope(1, 0, 40, 4, 64, 64, x, 256, a, 256, cs, 64)
    P.k_rope(1, 0, 40, 4, 64, 64, x.clone(), 256, b, 256, cs, 64)
    assert torch.equal(a, b)


def test_rope_beyond_2_31_elements():
    import paper_2401_15207_b200 as P
    torch = _torch()
    rows, ld = 300000, 8192
    x = torch.zeros(rows, ld, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, ld, device="cuda").to(torch.bfloat16)
    want = torch.empty(3, ld, dtype=torch.bfloat16, device="cuda")
    cs, pos = _rope_table(100, 128), torch.full((rows,), 99, dtype=torch.int32, device="cuda")
    P.k_rope(1, 1, 3, 64, 128, 128, x[-3:].clone(), ld, want, ld, cs, 100, positions=pos[:3])
    P.k_rope(1, 1, rows, 64, 128, 128, x, ld, x, ld, cs, 100, positions=pos)
    assert torch.equal(x[-3:], want) and not bool(x[:-3].any())


def test_rope_agrees_with_the_fused_projection():
    """Against hift_k_linear_rope, whose table this is too: the one rounds before the rotation as well."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    M, K, heads, S = 256, 256, 2, 64
    N = heads * 128
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = (torch.randn(n, K, generator=g, device="cuda").to(torch.bfloat16) for n in (M, N))
    cs = _rope_table(S, 128)
    fused, plain = (torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    P.k_linear_rope(M, N, K, x, w, fused, None, cs, S, 128, N)
    P.k_linear(0, 1, M, N, K, x, w, plain)
    size = R.rope(plain.double().abs(), 0, heads, 128, 128, torch.stack([cs[0].double().abs(), -cs[1].double().abs()]), torch.arange(M, device="cuda") % S, False).abs()
    size = size + 2 * plain.double().abs()
    P.k_rope(1, 0, M, heads, 128, 128, plain, N, plain, N, cs, S)
    assert bool(((fused.double() - plain.double()).abs() <= 2 * R.UB * size + 2.0 ** -16).all())


# ------------------------------------------------------------------ 8 bits
def _values(rows, f, dt, seed=0):
    """Ordinary blocks; zeros, huge, tiny and mixed ones; ties; the formats' largest values; NaN and infinities."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, f, generator=g, device="cuda") * torch.exp(torch.randn(rows, f, generator=g, device="cuda"))
    b = torch.arange(f, device="cuda") // 32
    x = torch.where((b % 11 == 3)[None], x * 1e30, x)
    x = torch.where((b % 11 == 5)[None], x * 1e-30, x)
    x = torch.where((b % 11 == 6)[None], x * 1e-44, x)
    x = torch.where((b % 11 == 7)[None], 0.0, x)
    x = torch.where((b % 11 == 8)[None], torch.randint(-254, 255, x.shape, generator=g, device="cuda") / 2.0, x)
    if rows > 2:
        x[1, ::32] = torch.tensor([127.0, 127.5, 448.0, 448.5, 3e38, 256.0], device="cuda").repeat(len(x[1, ::32]) // 6 + 1)[:len(x[1, ::32])]
        x[2, f // 2], x[rows - 1, 0], x[rows - 1, f - 1] = NAN, INF, -INF
    return x.to(dt)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("rows,f,pad", [(1, 1, 0), (3, 31, 1), (5, 32, 0), (4, 33, 0), (7, 1000, 24), (300, 776, 0), (64, 4099, 3), (2000, 40, 8)])
def test_pack_and_unpack(code, fmt, rows, f, pad):
    import paper_2401_15207_b200 as P
    torch = _torch()
    dt = _types(code)
    x = torch.full((rows, f + pad), 9.0, dtype=dt, device="cuda")
    x[:, :f] = _values(rows, f, dt, f)
    nb = -(-f // 32)
    q = torch.full((rows + 1, f), 77, dtype=torch.int8, device="cuda")
    sc = torch.full((rows + 1, nb), 77, dtype=torch.uint8, device="cuda")
    P.k_act8_pack(code, fmt, rows, f, x, f + pad, q, sc)
    assert bool((q[-1] == 77).all()) and bool((sc[-1] == 77).all())
    q, sc = q[:-1], sc[:-1]
    want, byte = R.pack(R.f64(x[:, :f]), fmt)
    got = (q if fmt == 0 else q.view(torch.float8_e4m3fn)).double()
    assert torch.equal(got, want) and torch.equal(sc.long(), byte)
    for out_code in (0, 1):                                  # exact in either type
        back = torch.full((rows, f + pad), 9.0, dtype=_types(out_code), device="cuda")
        P.k_act8_unpack(out_code, fmt, rows, f, q, sc, back, f + pad)
        assert torch.equal(back[:, :f].double().nan_to_num(1e300), R.unpack(want, byte).nan_to_num(1e300)) and bool((back[:, f:] == 9).all())


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("rows,f", [(1, 1), (3, 33), (130, 96), (9, 1001), (37, 5120), (600, 264)])
def test_activations_in_8_bits(code, fmt, kind, rows, f):
    import paper_2401_15207_b200 as P
    torch = _torch()
    dt, parts = _types(code), kind
    g = torch.Generator(device="cuda").manual_seed(f)
    pre = (torch.randn(rows, parts * f, generator=g, device="cuda") * 3).to(dt)
    pre[:, ::17] *= 20
    dy = torch.randn(rows, f, generator=g, device="cuda").to(dt)
    nb = -(-f // 32)
    act, act2, dpre = (torch.full((rows, n * f), NAN, dtype=dt, device="cuda") for n in (1, 1, parts))
    q = torch.zeros(rows, parts * f, dtype=torch.int8, device="cuda")
    sc = torch.zeros(rows, parts * nb, dtype=torch.uint8, device="cuda")
    P.k_act8_fwd(code, fmt, kind, rows, f, pre, act, q, sc)
    P.k_act8_bwd(code, fmt, kind, rows, f, dy, q, sc, dpre, act2)
    want, byte = R.pack(R.f64(pre), fmt, parts)
    num = (q if fmt == 0 else q.view(torch.float8_e4m3fn)).double()
    assert torch.equal(num, want) and torch.equal(sc.long(), byte)
    unit = R.UB if code else R.U32
    # the quick division gives 0 for divisors 1 + exp(-a) beyond 2^126: a sigmoid below 2^-126 is 0 instead, off by that much, times its factors
    gone = 2.0 ** -126

    def near(got, val, err):
        assert bool(((got.double() - val).abs() <= err + unit * 1.001 * val.abs() + 1e-36).all()), float(((got.double() - val).abs() - err - unit * val.abs()).max())
    for x, got in ((R.f64(pre), act), (R.unpack(num, byte, parts), act2)):
        y, d = R.activation(kind, x)
        if kind == 1:
            # 0.5 a (1 + erf): the error function within 2 steps, a sum of about 1, two products
            near(got, y, 8 * R.U32 * x.abs())
        else:
            # __expf(a): 2 + 1.16 |a| steps of 2^-23; a division of 2, three products
            near(got, y, (12 + 2.4 * x[:, :f].abs()) * 2 * R.U32 * y.abs() + gone * (x[:, :f] * x[:, f:]).abs())
    gr = R.f64(dy)
    if kind == 1:
        pdf = torch.exp(-x * x / 2) * 0.3989422804014327
        near(dpre, gr * d[0], gr.abs() * (8 + (16 + 2.4 * x * x) * x.abs() * pdf) * R.U32)
    else:
        a, u = x[:, :f], x[:, f:]
        s, rel = torch.sigmoid(a), (16 + 2.4 * a.abs()) * 2 * R.U32
        near(dpre[:, :f], gr * d[0], gr.abs() * u.abs() * s * (1 + a.abs() * (1 - s)) * 2 * rel + gone * gr.abs() * u.abs() * (1 + a.abs()))
        near(dpre[:, f:], gr * d[1], (gr * d[1]).abs() * rel + gone * (gr * a).abs())
    again = torch.full_like(dpre, NAN)
    P.k_act8_bwd(code, fmt, kind, rows, f, dy, q, sc, again)                 # without the activation
    assert torch.equal(again, dpre)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("kind", [1, 2])
def test_activations_in_8_bits_with_bad_values(fmt, kind):
    """A NaN or infinity spoils its block of 32 and nothing else; the forward value is the exact pre-activation's."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    rows, f = 6, 96
    for code in (0, 1):
        dt = _types(code)
        pre = torch.randn(rows, kind * f, device="cuda").to(dt)
        pre[1, 40], pre[2, 0], pre[3, 95] = NAN, INF, -INF
        act, dpre = torch.empty(rows, f, dtype=dt, device="cuda"), torch.empty(rows, kind * f, dtype=dt, device="cuda")
        q, sc = torch.empty(rows, kind * f, dtype=torch.int8, device="cuda"), torch.empty(rows, kind * 3, dtype=torch.uint8, device="cuda")
        P.k_act8_fwd(code, fmt, kind, rows, f, pre, act, q, sc)
        P.k_act8_bwd(code, fmt, kind, rows, f, torch.ones(rows, f, dtype=dt, device="cuda"), q, sc, dpre)
        bad = torch.zeros(rows, f, dtype=torch.bool, device="cuda")
        bad[1, 32:64] = bad[2, :32] = bad[3, 64:] = True
        for part in range(kind):
            assert torch.equal(dpre[:, part * f:(part + 1) * f].isnan(), bad)
        assert bool(act[1, 40].isnan()) and bool(act[1, 41].isfinite()) and (sc == 255).sum() == 3


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("kind", [1, 2])
def test_activations_in_8_bits_off_the_16_byte_grid(code, kind):
    """Buffers that start at any element (any byte for the packed values) give the same bits as aligned ones."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    rows, f, dt = 19, 128, _types(code)
    g = torch.Generator(device="cuda").manual_seed(3)
    pre, dy = (torch.randn(rows, n * f, generator=g, device="cuda").to(dt) for n in (kind, 1))

    def run(shifted):
        def at(name, cols, dtype, src=None):
            k = int(name in shifted)
            t = torch.zeros(rows * cols + 16, dtype=dtype, device="cuda")[k:k + rows * cols].view(rows, cols)
            if src is not None:
                t.copy_(src)
            return t
        x, d, q, sc = at("pre", kind * f, dt, pre), at("dy", f, dt, dy), at("q", kind * f, torch.int8), at("sc", kind * f // 32, torch.uint8)
        act, dpre, act2, back = at("act", f, dt), at("dpre", kind * f, dt), at("act2", f, dt), at("back", kind * f, dt)
        P.k_act8_fwd(code, 0, kind, rows, f, x, act, q, sc)
        P.k_act8_bwd(code, 0, kind, rows, f, d, q, sc, dpre, act2)
        P.k_act8_unpack(code, 0, rows, kind * f, q, sc, back, kind * f)      # (f is a multiple of 32: the parts' blocks are those of whole rows)
        return [t.clone() for t in (act, q, sc, dpre, act2, back)]
    names = ["pre", "dy", "q", "sc", "act", "dpre", "act2", "back"]
    want = run([])
    for shifted in [names] + [[n] for n in names]:
        for a, b in zip(run(shifted), want):
            assert torch.equal(a, b), shifted


def test_pack_beyond_2_31_elements():
    import paper_2401_15207_b200 as P
    torch = _torch()
    rows, f = 270000, 8192
    x = torch.zeros(rows, f, dtype=torch.bfloat16, device="cuda")
    x[-2:] = torch.randn(2, f, device="cuda").to(torch.bfloat16)
    q, sc = torch.empty(rows, f, dtype=torch.int8, device="cuda"), torch.empty(rows, f // 32, dtype=torch.uint8, device="cuda")
    P.k_act8_pack(1, 0, rows, f, x, f, q, sc)
    want, byte = R.pack(R.f64(x[-2:]), 0)
    assert torch.equal(q[-2:].double(), want) and torch.equal(sc[-2:].long(), byte) and not bool(q[:-2].any())
    P.k_act8_unpack(1, 0, rows, f, q, sc, x, f)
    assert torch.equal(x[-2:].double(), R.unpack(want, byte)) and not bool(x[:-2].any())


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("code,dh,K", [(0, 32, 4), (1, 128, 2), (1, 64, 4)])
def test_a_block_of_them(code, dh, K):
    """A block as these operators make one: qkv projection, rotation of both maps' halves, differential attention with its learned lambda, output projection,
    SwiGLU with its pre-activations in 8 bits; then backward from what was kept.  Every gradient against automatic differentiation of the same block in
    64 bits, its pre-activations replaced by the packed values where the backward pass reads them."""
    import paper_2401_15207_b200 as P
    torch = _torch()
    B, S, H, f = 2, 96, 4, 512
    T, d, cols = B * S, H * dh, (H + 2 * K) * dh
    dt = _types(code)
    g = torch.Generator(device="cuda").manual_seed(21)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).to(dt)       # noqa: E731
    new = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device="cuda")                     # noqa: E731
    x, wqkv, wo = rnd(T, d), rnd(cols, d, std=d ** -0.5), rnd(d, d, std=d ** -0.5)
    wgu, wd, dout = rnd(2 * f, d, std=d ** -0.5), rnd(d, f, std=f ** -0.5), rnd(T, d)
    lw = torch.randn(4, 1, dh // 2, generator=g, device="cuda") * 0.1
    gain = (1 + 0.1 * torch.randn(dh, generator=g, device="cuda")).to(dt)
    lens = torch.tensor([S, S - 40], dtype=torch.int32, device="cuda")
    cs = _rope_table(S, dh // 2)
    lin = lambda form, M, N, KK, a, b, o: P.k_linear(form, code, M, N, KK, a, b, o)            # noqa: E731
    # forward
    qkv, lam = new(T, cols), new(H, dtype=torch.float32)
    lin(0, T, cols, d, x, wqkv, qkv)
    P.k_rope(code, 0, T, 2 * (H + K), dh // 2, dh // 2, qkv, cols, qkv, cols, cs, S)
    P.k_diff_lambda(H, 1, dh // 2, 0.5, lw, lam)
    o, o2, y, lse = new(T, d), new(T, d), new(T, d), new(2, B, H, S, dtype=torch.float32)
    P.k_diff_attention_fwd(code, B, S, H, K, dh, True, qkv, lam, gain, 1e-5, 0.5, o, o2, y, lse, key_lens=lens)
    z, gu, act, out = new(T, d), new(T, 2 * f), new(T, f), new(T, d)
    lin(0, T, d, d, y, wo, z)
    lin(0, T, 2 * f, d, z, wgu, gu)
    q8, s8 = new(T, 2 * f, dtype=torch.int8), new(T, 2 * f // 32, dtype=torch.uint8)
    P.k_act8_fwd(code, 0, 2, T, f, gu, act, q8, s8)
    lin(0, T, d, f, act, wd, out)
    # what a checkpoint of qkv in 8 bits gives back (kept beside: the comparison below reads the exact one)
    c8, cb, back = new(T, cols, dtype=torch.int8), new(T, -(-cols // 32), dtype=torch.uint8), new(T, cols)
    P.k_act8_pack(code, 0, T, cols, qkv, cols, c8, cb)
    P.k_act8_unpack(code, 0, T, cols, c8, cb, back, cols)
    # half a step of the least power of two that is at least top / 127, so less than 2 top / 127
    assert bool(((back - qkv).abs().float() <= 1 / 127 * qkv.abs().float().view(T, -1, 32).amax(2).repeat_interleave(32, 1) * 1.001).all())
    # backward
    dact, dgu, act8, dz, dy, dqkv = new(T, f), new(T, 2 * f), new(T, f), new(T, d), new(T, d), new(T, cols)
    lin(1, T, d, f, dout, wd, dact)
    P.k_act8_bwd(code, 0, 2, T, f, dact, q8, s8, dgu, act8)
    grads = {n: new(*w.shape, dtype=torch.float32) for n, w in (("wd", wd), ("wgu", wgu), ("wo", wo), ("wqkv", wqkv))}
    lin(2, T, d, f, dout, act8, grads["wd"])
    lin(2, T, 2 * f, d, dgu, z, grads["wgu"])
    lin(1, T, 2 * f, d, dgu, wgu, dz)
    lin(2, T, d, d, dz, y, grads["wo"])
    lin(1, T, d, d, dz, wo, dy)
    dlam, dgain, dlw = new(H, dtype=torch.float32), new(dh, dtype=torch.float32), new(4, 1, dh // 2, dtype=torch.float32)
    w = new(P.diff_attention_bwd_scratch_bytes(code, B, S, H, dh, True), dtype=torch.uint8)
    P.k_diff_attention_bwd(code, B, S, H, K, dh, True, qkv, lam, gain, 1e-5, 0.5, o, o2, lse, dy, dqkv, dlam, dgain, w, key_lens=lens)
    P.k_rope(code, 0, T, 2 * (H + K), dh // 2, dh // 2, dqkv, cols, dqkv, cols, cs, S, inverse=True)
    P.k_diff_lambda_bwd(H, 1, dh // 2, lw, dlam, dlw)
    lin(2, T, cols, d, dqkv, x, grads["wqkv"])
    dx = new(T, d)
    lin(1, T, cols, d, dqkv, wqkv, dx)
    # the same in 64 bits, from the stored values at each operator's entrance (so that one operator's roundings do not count against the next)
    leaf = lambda t: R.f64(t).clone().requires_grad_()                        # noqa: E731
    X, WQ, WO, WG, WD, LW, GA = (leaf(t) for t in (x, wqkv, wo, wgu, wd, lw, gain))
    pos = torch.arange(T, device="cuda") % S
    pre = X @ WQ.T
    i = torch.arange(dh // 4, device="cuda")
    v = pre[:, :(H + K) * dh].view(T, 2 * (H + K), dh // 2)
    c, s = (cs[k].double()[pos][:, None] for k in (0, 1))
    a, b = v[..., i], v[..., i + dh // 4]
    rot = torch.cat([torch.cat([a * c - b * s, b * c + a * s], -1).view(T, -1), pre[:, (H + K) * dh:]], 1)
    la = (torch.exp((LW[0] * LW[1]).sum()) - torch.exp((LW[2] * LW[3]).sum()) + 0.5).expand(H)
    qh, kh, vh, _ = R.dattn_split(rot, B, S, H, K, dh)
    seen = R.dattn_seen(B, S, True, lens, "cuda")
    om = []
    for m in range(2):
        h = slice(m * dh // 2, (m + 1) * dh // 2)
        om.append(torch.softmax(torch.where(seen, qh[..., h] @ kh[..., h].mT / (dh / 2) ** 0.5, -INF), -1) @ vh)
    full = om[0] - la[:, None, None] * om[1]
    Y = full / torch.sqrt((full ** 2).mean(-1, keepdim=True) + 1e-5) * GA * 0.5
    Y = Y.transpose(1, 2).reshape(T, d)
    Z = Y @ WO.T
    G = Z @ WG.T
    kept = R.unpack(q8.double(), s8, 2)
    Gk = G + (kept - G).detach()                              # the packed values, with G's gradient
    A = torch.nn.functional.silu(Gk[:, :f]) * Gk[:, f:]
    names = dict(wqkv=WQ, wo=WO, wgu=WG, wd=WD, lw=LW, gain=GA, x=X)
    ref = dict(zip(names, torch.autograd.grad(A @ WD.T, list(names.values()), R.f64(dout))))
    got = dict(grads, lw=dlw, gain=dgain, x=dx)
    # a chain of at most 12 operators, each with a few roundings of its type that do not line up: 12 half steps and as many of the norm's gradient
    tol = 24 * R.UB if code else 3e-5
    for n in names:
        rel = float((got[n].double().view_as(ref[n]) - ref[n]).norm() / ref[n].norm())
        assert rel <= tol, (n, rel)
    exact = (torch.nn.functional.silu(G[:, :f]) * G[:, f:]) @ WD.T
    assert float((out.double() - exact.detach()).norm() / out.double().norm()) <= tol
