"""GPU test of the 4-bit products: every code under every scale byte, alone in its row, through every kernel."""
import numpy as np
import pytest

from tests import block_oracle as O
from tests.test_gpu_block_operators import Weights

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("m", [1, 12, 24, 40, 130])
def test_product_of_every_code_under_every_scale(m):
    """Row (b, c): code c at k = 5 and zeros, under scale byte b.  With ones for activations each output is that weight as
    a bf16 number: exact up to b = 252, infinite where 253 and 254 take it past bf16's range, NaN for 255."""
    b, c = np.divmod(np.arange(256 * 16), 16)
    codes = np.zeros((4096, 16), np.uint8)
    codes[:, 2] = c << 4
    w = Weights(4096, 32, codes=codes, scales=b.astype(np.uint8)[:, None])
    got = w.product(torch.ones(m, 32, dtype=torch.bfloat16, device="cuda"), m, 32, True).cpu().double().numpy()
    value = np.where(c >= 8, -1.0, 1.0) * O.E2M1[c & 7] * np.exp2(b - 127.0)
    want = np.where(np.abs(value) >= 2.0**128, np.copysign(np.inf, value), value)
    assert np.isinf(want[(b == 253) | (b == 254)]).sum() == 4 + 8          # 4 and 6 of 2^126; 2, 3, 4 and 6 of 2^127
    assert np.isnan(got[:, b == 255]).all()
    fine = b < 255
    assert (got[:, fine] == want[fine]).all(), np.argwhere(got[:, fine] != want[fine])[:8].tolist()
