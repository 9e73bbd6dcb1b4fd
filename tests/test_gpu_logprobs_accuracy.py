"""Log-probabilities where the mass lies far below the largest logit: what the factor inside the exponentials may put on them."""
import numpy as np
import pytest

import train_ops_ref as R
from test_gpu_train_ops import _dev, _run_logp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temp", [0.67, 1.34])
@pytest.mark.parametrize("vocab", [32000, 262144])
def test_logprobs_far_below_the_largest_logit(temp, vocab):
    """exp(z - z_max) is taken as 2 to the power (x - m) (log2(e) / T), and an error of that factor counts |z - z_max| times in L.  It is
    the factor's own rounding to fp32, 1e-8 at these temperatures (a product of two rounded factors is 1e-7 off).  Beside it L and
    log p carry their last roundings, and the exponentials' and sums' own errors, which are spread over so many random
    terms, less than another."""
    rng = np.random.default_rng(vocab)
    spread = -np.log(vocab) * temp + rng.uniform(-1.5, 1.5, (2, vocab)) * temp
    spread[:, 17] = 0.0                                        # the largest, with about a third of the mass
    x = spread.astype(np.float32)
    tok = np.array([17, 5])
    logp, _, st, _, _ = _run_logp(_dev(x), tok, vocab, temp, 0, 0)
    z = (x.astype(np.float64) - x.max(1, keepdims=True).astype(np.float64)) / temp
    L = np.log(np.exp(z).sum(1))
    away = (np.exp(z - L[:, None]) * -z).sum(1)                # mean |z - z_max|
    off = abs(float(np.float32(np.log2(np.e) / temp)) / (np.log2(np.e) / temp) - 1)
    assert (np.abs(st[1] - L) <= off * away + 2 * R.U32 * L).all()
    want = z[np.arange(2), tok] - L
    assert (np.abs(logp - want) <= off * away + 2 * R.U32 * L + 4 * R.U32 * np.abs(z[np.arange(2), tok])).all()
