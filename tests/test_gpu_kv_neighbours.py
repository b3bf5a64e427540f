"""GPU tests of what the cache operators leave alone: other sequences' slots and scales, blocks that no sequence owns."""
import pytest

from paper_2609_07883_amd import api

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 4, 64), (8, 2, 128)])
def test_blocks_of_others(cache, hq, hkv, hd):
    """An append and an attention in the middle layer of three: the model's cache in the blocks appended to, and every
    other byte of the pools and scales as it was."""
    from tests.kv_rig import Rig
    rig = Rig(hq, hkv, hd, {1: 10, 2: 90, 3: 33, 4: 64}, cache, layers=3, window=16, sinks=1, grow=20, spare=7)
    batch = api.Batch(9, 1, 10, (2,), (90,))
    pools = [rig.k_pool, rig.v_pool] + ([rig.k_scale, rig.v_scale] if cache == "e4m3" else [])
    before = [p.clone() for p in pools]
    x, q, k, v = rig.rows(batch.rows)
    plan = rig.begin(batch)
    rig.append(plan, 1, x)
    rig.attend(plan, 1, x)
    rig.model_append(1, batch, k, v)
    rig.check_cache(1)
    own = {rig.ctx.block_table(sid)[t // 16] for sid, at, n in rig.runs(batch) for t in range(at, at + n)}
    assert len(own) == 3
    others = torch.tensor([b for b in range(rig.blocks) if b not in own], device="cuda")
    for p, b in zip(pools, before):
        for layer in range(3):
            pick = others if layer == 1 else slice(None)
            assert torch.equal(p[layer][pick].contiguous().view(torch.uint8), b[layer][pick].contiguous().view(torch.uint8))
