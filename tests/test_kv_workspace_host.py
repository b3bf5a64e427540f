"""What the cache operators cost an iteration in workspace (CPU)."""
import pytest

from paper_2609_07883_amd import api

ROWS = ((0, 1), (0, 256), (128, 4), (1500, 16), (4096, 8))   # (chunk rows, decodes)
# (layers, d_model, q heads, kv heads, head dim, FFN, max_pos): bytes before there was an 8-bit cache
BF16 = {(1, 4096, 32, 8, 128, 14336, 32768): (4379904, 54817280, 83797760, 251703808, 486258688),
        (2, 256, 4, 4, 64, 704, 4096): (558080, 2434816, 22897408, 31548928, 47838464),
        (2, 256, 8, 2, 64, 256, 4096): (2190080, 4238336, 22456320, 32211456, 50203136)}


def _ctx(shape):
    n, d, hq, hkv, hd, f, max_pos = shape
    return api.Context(n, d, hq, hkv, hd, f, 1e-5, 10000.0, max_pos)


@pytest.mark.parametrize("shape", BF16)
def test_bf16_iteration(shape):
    """An iteration over the full bf16 cache needs the workspace it needed without the operators: nothing in it holds
    lists of theirs."""
    c = _ctx(shape)
    c.kv_init(64, 64, 4)
    assert tuple(c.workspace_size(*r) for r in ROWS) == BF16[shape]


@pytest.mark.parametrize("shape", BF16)
def test_8bit_iteration(shape):
    """Over the 8-bit cache an iteration's workspace holds longer lists and no second copy of its K/V rows."""
    c = _ctx(shape)
    for C, B in ROWS:
        c.kv_init(64, 64, 4)
        it, op = c.workspace_size(C, B), c.attn_workspace_size(C, B)
        c.kv_init_8bit(64, 64, 64, 64, 4)
        lists = c.attn_workspace_size(C, B) - op + 16 * (C + B) + 2 * 256     # at most one append (four words) a row
        assert it <= c.workspace_size(C, B) <= it + lists
