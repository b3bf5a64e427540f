"""GPU tests of the sampler where its sums, bins and cuts are at their edges, against the float64 model."""
import math

import numpy as np
import pytest

from tests import block_oracle as O
from tests.test_gpu_block_operators import _sample

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

FLT_MAX = float(np.finfo(np.float32).max)


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _lowest(f32):
    return float(torch.finfo(torch.float32 if f32 else torch.bfloat16).min)


def _check(x, f32=True, ld=None, shift=0, **par):
    got, lp, v = _sample(x, f32, ld, shift, **par)
    kinds = {k: np.int32 if k == "top_k" else np.float32 for k in par if par[k] is not None}
    cols = {k: np.broadcast_to(np.asarray(par[k], t), (len(v),)) for k, t in kinds.items()}
    for r in range(len(v)):
        p = {k: c[r].item() for k, c in cols.items()}
        token, want = O.sample(v[r], **p)
        assert got[r] == token, (r, p, got[r], token)
        # a weight and a sum of weights right to 2^-36 each, one rounding of the logarithm to fp32
        assert lp[r] == want or abs(lp[r] - want) <= 2.0**-24 * abs(want) + 2.0**-35, (r, p, lp[r], want)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("temperature", [1e35, 1e36, 1e37, 1e38, FLT_MAX])
def test_top_p_over_slices_of_the_lowest_value(temperature, f32):
    """Slices whose largest logit is far below -2^100, at temperatures at which that is no distance: their bins count
    from that logit.  Whole pieces only, and nothing that is not finite."""
    rng = np.random.default_rng([int(math.log10(temperature)), f32])
    n, low = 40960, _lowest(f32)
    x = rng.standard_normal((5, n))
    x[0, 8192:] = low                                        # all slices but the first
    x[1] = low
    x[2, :30000] = low * rng.uniform(0.5, 1.0, 30000)
    x[3] = np.clip(x[3] * 1e38, low, -low)
    x[4, ::2] = low
    for p in (0.3, 0.9, 0.9999):
        _check(x, f32, temperature=temperature, top_p=p, u=rng.random(5))
