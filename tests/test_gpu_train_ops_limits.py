"""The orthogonalised update at its limits: every one of its three paths (one fp32 launch for a short side of at most 16, one launch
for one of at most 128, tiled products), both orientations, with inputs whose roundings line up, zeros, bad values, extreme scales
and a raised time-out flag."""
import pytest

import train_ops_ref as R
from gpu_util import rel_l2
from test_gpu_train_ops import NS_TOL, _dev, _matrix, _ns_tol, _orth, _torch

pytestmark = pytest.mark.gpu


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
