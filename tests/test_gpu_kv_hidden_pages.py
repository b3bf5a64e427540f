"""GPU tests of windowed attention over the 8-bit cache where blocks that the window hides whole hold scales that are no
powers of two, as where a caller installs the window's tokens alone."""
import pytest

from paper_2609_07883_amd import api
from tests import kv_oracle as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SCALES = [0.0, float("nan"), -1.0, float("inf"), 3e38]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _rig(*a, **k):
    from tests.kv_rig import Rig
    return Rig(*a, **k)


def _check(rig, batch, scale, rows=None, q_std=2.0):
    """The batch against the model with `scale` for K and V in every block that no row of its sequence sees; some of
    those blocks lie in the 64-key tile of a token that is seen."""
    beside = 0
    for sid, at, _ in rig.runs(batch):
        for i, blk in enumerate(rig.ctx.block_table(sid)):
            first, last = 16 * i, 16 * i + 15
            if last <= at - rig.window and first >= rig.sinks:
                rig.k_scale[:, blk] = scale
                rig.v_scale[:, blk] = scale
                beside += max(at - rig.window + 1, 0) // 64 == i // 4
    assert beside
    x, q, k, v = rig.rows(batch.rows, q_std)
    plan = rig.begin(batch)
    rig.append(plan, 0, x)
    out = rig.attend(plan, 0, x)
    rig.model_append(0, batch, k, v)
    want, bound = rig.model_attend(0, batch, q, rows)
    got = rig.float_rows(out)
    O.check_rows(got if rows is None else got[sorted(rows)], want, bound)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("hq,hkv,hd,window,sinks", [(4, 4, 64, 50, 3), (8, 2, 128, 200, 70), (16, 1, 128, 1, 0)])
def test_decodes(hq, hkv, hd, window, sinks, scale):
    """Decodes that are one item each: their hidden blocks beside seen ones have no part in any row."""
    ctxs = [17, 63, 64, 90, 127, 130, 200, 256, 300, 420, 511, 700]
    seqs = {10 + i: n for i, n in enumerate(ctxs)}
    rig = _rig(hq, hkv, hd, seqs, window=window, sinks=sinks, grow=1)
    _check(rig, api.Batch(0, 0, 0, tuple(seqs), tuple(ctxs)), scale)


@pytest.mark.parametrize("scale", SCALES)
def test_long_decodes(scale):
    """Decodes of several items, whose partial sums are merged."""
    rig = _rig(8, 2, 128, {2: 4095, 3: 6001}, window=2500, sinks=5, grow=1)
    _check(rig, api.Batch(0, 0, 0, (2, 3), (4095, 6001)), scale)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("hq,hkv,hd,window,sinks", [(4, 4, 64, 50, 3), (8, 2, 128, 200, 70), (16, 1, 128, 1, 0), (8, 1, 64, 333, 0)])
def test_chunks(hq, hkv, hd, window, sinks, scale):
    """Prompts behind cached prefixes beside decodes."""
    pre = [(1, 90, 1), (2, 155, 65), (3, 333, 40), (4, 430, 70)]
    rig = _rig(hq, hkv, hd, {1: 90, 2: 155, 3: 333, 4: 430, 20: 90, 21: 700}, window=window, sinks=sinks, grow=80)
    _check(rig, api.Batch.batched(pre, (20, 21), (90, 700)), scale)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("hq,hkv,C,P,window,sinks", [(64, 16, 1024, 5003, 3500, 0), (128, 16, 512, 5000, 3001, 64),
                                                      (256, 16, 256, 5000, 2100, 1), (32, 8, 200, 16390, 9001, 5)])
def test_long_items(hq, hkv, C, P, window, sinks, scale):
    """The two-phase kernel, query tiles whole and split."""
    from paper_2609_07883_amd.synth import ModelShape
    shape = ModelShape(1, 256, hq, hkv, 128, 256, max_pos=32768)
    assert api.attention_plan(shape, [700], [(P, C)], window, sinks, kv="e4m3")["chunk_two_phase"]
    rig = _rig(hq, hkv, 128, {1: P, 2: 700}, window=window, sinks=sinks, grow=C + 1, max_pos=32768)
    tile = 256 * hkv // hq
    rows = {0, 1, 15, 16, 17, 31, 33, tile - 1, tile, C // 2, C - 1, C}
    _check(rig, api.Batch(C, 1, P, (2,), (700,)), scale, rows)
