"""The orthogonalised update at its limits: every one of its three paths (one fp32 launch for a short side of at most 16, one launch
for one of at most 128, tiled products), both orientations, with inputs whose roundings line up, zeros, bad values, extreme scales
and a raised time-out flag."""
import pytest

import train_ops_ref as R
from gpu_util import rel_l2
from test_gpu_train_ops import _dev, _matrix, _ns_tol, _torch

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
