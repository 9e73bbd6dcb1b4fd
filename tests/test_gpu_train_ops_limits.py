"""The orthogonalised update at its limits: every one of its three paths (one fp32 launch for a short side of at most 16, one launch
for one of at most 128, tiled products), both orientations, with inputs whose roundings line up, zeros, bad values, extreme scales
and a raised time-out flag."""
import numpy as np
import pytest

import train_ops_ref as R
from gpu_util import rel_l2
from test_gpu_train_ops import INF, NAN, NS_TOL, _dev, _matrix, _ns_tol, _orth, _torch

pytestmark = pytest.mark.gpu
# one fp32 launch, one CTA and several; one launch on tensor cores, one CTA, several, two column blocks a CTA; tiled
PATHS = [(1, 1), (2, 3), (16, 300), (9000, 16), (64, 64), (120, 500), (40, 3001), (3001, 40), (130, 200), (200, 130)]


def _unrounded(g, steps=5):
    """The result before its rounding to bf16: the update of a matrix of zeros without momentum is -lr 0.2 sqrt(max(rows, cols)) X."""
    from paper_2401_15207_b200 import muon_step, orthogonalize_scratch_bytes
    torch = _torch()
    rows, cols = g.shape
    master, mom = torch.zeros(rows, cols, device="cuda"), torch.zeros(rows, cols, device="cuda")
    w = torch.empty(orthogonalize_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    muon_step(rows, cols, None, master, g, mom, w, 1.0, momentum=0.0, nesterov=False, steps=steps)
    torch.cuda.synchronize()
    return -master.double().cpu().numpy() / (0.2 * np.sqrt(max(rows, cols)))


def _few_values(kind, rows, cols):
    if kind == "constant":
        return np.ones((rows, cols), np.float32)
    if kind == "diagonal":
        return np.eye(rows, cols, dtype=np.float32)
    n, g = int(kind[6:]), np.zeros((rows, cols), np.float32)
    for i in range(0, rows, n):
        j = i * cols // rows
        g[i:i + n, j:j + n] = 1
    return g


@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 3), (16, 300), (300, 2), (9000, 16), (64, 64), (40, 3001), (3001, 40), (130, 200)])
def test_no_path_writes_after_a_time_out(rows, cols):
    """With the tensor-core time-out flag raised, results, master and model copy stay as they are on every path, the one without
    tensor cores among them: a model's small matrices stand still with its large ones.  Cleared, the calls work again."""
    from paper_2401_15207_b200 import k_orthogonalize, muon_step, orthogonalize_scratch_bytes, tc_error_flag
    torch = _torch()
    g = _dev(_matrix("gauss", rows, cols, 3))
    o = torch.full((rows, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    master, mom = torch.full((rows, cols), 0.5, device="cuda"), torch.zeros(rows, cols, device="cuda")
    param = torch.full((rows, cols), 3.0, dtype=torch.bfloat16, device="cuda")
    w = torch.empty(orthogonalize_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    assert tc_error_flag(1) == 1
    try:
        k_orthogonalize(0, rows, cols, g, o, 5, w)
        muon_step(rows, cols, param, master, g, mom, w, 1e-2)
        torch.cuda.synchronize()
        assert bool((o == 7).all()) and bool((master == 0.5).all()) and bool((param == 3).all())
        assert torch.equal(mom, g)                       # the momentum has been updated
    finally:
        assert tc_error_flag(0) == 0
    k_orthogonalize(0, rows, cols, g, o, 5, w)
    assert rel_l2(o.double().cpu().numpy(), R.orthogonalize(g.double().cpu().numpy())) < _ns_tol(rows * cols)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 3), (5, 700), (16, 300), (9000, 16), (16, 16384), (64, 64), (120, 500), (40, 3001), (3001, 40)])
def test_small_matrices_on_the_tiled_products(code, rows, cols):
    """What runs where a device cannot hold the one launch's cluster: the products of the large matrices, with the short side padded to
    128.  One to six elements do not average the products' roundings out: 2^-4 there, and half a step of the result's own."""
    from paper_2401_15207_b200 import code_path_switch
    from paper_2401_15207_b200.binding import SWITCH_NS_ONE_LAUNCH
    torch = _torch()
    g = _dev(_matrix("gauss", rows, cols, rows + cols), torch.bfloat16 if code else None)
    ref = R.orthogonalize(g.double().cpu().numpy())
    one = _orth(g, code)
    assert code_path_switch(SWITCH_NS_ONE_LAUNCH, 0) == 1
    try:
        tiled = _orth(g, code)
    finally:
        assert code_path_switch(SWITCH_NS_ONE_LAUNCH, 1) == 0
    assert rel_l2(tiled, ref) < (NS_TOL if rows * cols >= 100 else 2.0 ** -4 + 2.0 ** -8)
    assert rel_l2(one, ref) < _ns_tol(rows * cols)
    if min(rows, cols) <= 16 and rows * cols >= 100:     # fp32 there, 16-bit operands here: the switch reached another kernel
        assert not (tiled == one).all()


@pytest.mark.parametrize("kind", ["constant", "diagonal", "blocks4", "blocks16"])
@pytest.mark.parametrize("rows,cols", [(16, 300), (20, 100), (32, 32), (48, 48), (64, 67), (128, 128), (64, 200), (300, 40), (200, 512), (512, 200), (300, 700)])
def test_orthogonalize_where_roundings_line_up(kind, rows, cols):
    """Few distinct values: every entry is rounded the same way, so nothing averages out.  The bounds are those of the header: a scalar
    model of the products' roundings (X to fp16 in both products, E, F; 1.2e7 blocks of ones of random sizes and scales) is at most 3.6e-2
    off after five steps and 1.4e-1 after eight.  With everything in fp32 the same line-up has 2^-24 in the place of 2^-11, 2^-4 becomes
    2^-17, and sums of up to 300 equal terms, whose partial sums are all rounded alike, put at most 8 times that on it."""
    g = _few_values(kind, rows, cols)
    for steps, tol in ((1, 2.0 ** -4), (3, 2.0 ** -4), (5, 2.0 ** -4), (8, 2.0 ** -2)):
        if min(rows, cols) <= 16:
            tol *= 2.0 ** -10
        assert rel_l2(_unrounded(_dev(g), steps), R.orthogonalize(g.astype(np.float64), steps)) < tol, steps


@pytest.mark.parametrize("kind", ["gauss", "rank1", "rank3"])
@pytest.mark.parametrize("rows,cols", PATHS + [(300, 700)])
def test_orthogonalize_steps_on_every_path(kind, rows, cols):
    """Where roundings average out 2^-8 up to five steps.  Three more multiply the null space's noise by 3.44 each, 41 in all, the rest
    by up to 1.6: 2^-4."""
    g = _matrix(kind, rows, cols, 5)
    for steps in (1, 2, 3, 5, 8):
        assert rel_l2(_unrounded(_dev(g), steps), R.orthogonalize(g.astype(np.float64), steps)) < (NS_TOL if steps <= 5 else 2.0 ** -4), steps


@pytest.mark.parametrize("kind", ["gauss", "rank1"])
@pytest.mark.parametrize("rows,cols", [(3, 16384), (16384, 16), (1, 16384), (3, 16385), (16385, 16), (16, 20000), (1, 50257), (65536, 2)])
def test_orthogonalize_both_sides_of_the_fp32_limit(kind, rows, cols):
    """A short side of at most 16: all in fp32 up to a long side of 16384, where five steps leave noise of 2^-24 in each of up to 16
    directions, grown by 3.44^5: 1.2e-4 < 2^-12.  Longer ones take the 16-bit products: 2^-8."""
    g = _matrix(kind, rows, cols, 5)
    tol = 2.0 ** -12 if max(rows, cols) <= 16384 else NS_TOL
    assert rel_l2(_unrounded(_dev(g)), R.orthogonalize(g.astype(np.float64))) < tol


@pytest.mark.parametrize("tiled", [False, True])
@pytest.mark.parametrize("rows,cols", PATHS)
def test_scales_zeros_and_bad_values_on_every_path(rows, cols, tiled):
    """Squares beyond fp32 both ways, zeros, and a NaN or an infinity in a corner, on the path that a matrix takes and on the tiled one."""
    from paper_2401_15207_b200 import code_path_switch
    from paper_2401_15207_b200.binding import SWITCH_NS_ONE_LAUNCH
    torch = _torch()
    base = _matrix("gauss", rows, cols, 8)
    ref = R.orthogonalize(base.astype(np.float64))
    tol = _ns_tol(rows * cols) if not tiled or rows * cols >= 100 else 2.0 ** -4 + 2.0 ** -8    # a few elements on 16-bit products
    old = code_path_switch(SWITCH_NS_ONE_LAUNCH, 0 if tiled else 1)
    try:
        for s in (1e-25, 1e-6, 1e6, 1e30, 1e37):
            assert rel_l2(_orth(_dev((base.astype(np.float64) * s).astype(np.float32)), 0), ref) < tol, s
        assert not _orth(torch.zeros(rows, cols, device="cuda"), 0).any()
        assert not _orth(torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16), 1).any()
        for bad in (NAN, INF, -INF):
            g = _dev(base)
            g[rows - 1, cols - 1] = bad
            assert np.isnan(_orth(g, 0)).all()
            g = _dev(base).bfloat16()
            g[0, cols // 2] = bad
            assert np.isnan(_orth(g, 1)).all()
    finally:
        code_path_switch(SWITCH_NS_ONE_LAUNCH, old)
