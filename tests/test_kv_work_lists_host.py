"""Work lists of windowed layers against those of full attention over what the window leaves (CPU)."""
import numpy as np
from hypothesis import given, settings, strategies as st

from paper_2609_07883_amd import api
from paper_2609_07883_amd.synth import ModelShape

HEADS = [(8, 2, 64), (32, 8, 128), (16, 1, 128)]


def _skip(first, window, sinks):
    """Keys in whole 64-key tiles between the sinks and the window of a row at `first`."""
    lo = first - window + 1
    return max(0, lo // 64 - -(-sinks // 64)) * 64 if lo > 0 else 0


def _run(padded, waves):
    """Keys of an equal run: a multiple of 64, at least 128 where there are so many."""
    per = -(-padded // min(waves, max(1, padded // 128)))
    return -(-per // 64) * 64


@settings(max_examples=150, deadline=None)
@given(heads=st.sampled_from(HEADS), window=st.integers(1, 3000), sinks=st.integers(0, 400), seed=st.integers(0, 10**6))
def test_decodes(heads, window, sinks, seed):
    """A windowed decode's work is that of a decode over the keys left; every key is in one run, and no run is longer
    than an equal share asks for, or than one and a half of it and 128 where each decode is one run."""
    hq, hkv, hd = heads
    rng = np.random.default_rng(seed)
    shape = ModelShape(1, 4096, hq, hkv, hd, 256, max_pos=1 << 15)
    ctxs = [int(c) for c in rng.integers(0, rng.choice([200, 8000]), rng.integers(1, 80))]
    left = [c - _skip(c, window, sinks) for c in ctxs]
    plan = api.attention_plan(shape, ctxs, (), window, sinks, kv="e4m3")
    assert plan == api.attention_plan(shape, ctxs, (), window, sinks)      # a window alone: the same lists
    assert plan == api.attention_plan(shape, left, (), kv="e4m3")          # full attention over the 8-bit cache
    total, padded = sum(left) + len(left), sum(-(-(n + 1) // 64) * 64 for n in left)
    run, slots = _run(padded, max(1, 768 // hkv)), plan["decode_slots"]
    assert plan["decode_min_keys"] * slots <= total <= plan["decode_max_keys"] * slots
    if slots == len(ctxs) == plan["decode_items"]:
        assert plan["decode_max_keys"] == max(left) + 1 and 2 * plan["decode_max_keys"] <= 3 * run + 256
        assert plan["decode_min_keys"] == min(left) + 1
    else:
        assert plan["decode_max_keys"] <= run and slots == -(-padded // run)


@settings(max_examples=100, deadline=None)
@given(heads=st.sampled_from(HEADS), window=st.integers(1, 3000), sinks=st.integers(0, 400), prefix=st.integers(0, 20000),
       seed=st.integers(0, 10**6))
def test_a_query_tile(heads, window, sinks, prefix, seed):
    """A prompt of one query tile: the work of the same rows behind the prefix that is left."""
    hq, hkv, hd = heads
    rows = int(np.random.default_rng(seed).integers(1, 256 * hkv // hq + 1))
    shape = ModelShape(1, 4096, hq, hkv, hd, 256, max_pos=1 << 15)
    plan = api.attention_plan(shape, (), [(prefix, rows)], window, sinks, kv="e4m3")
    assert plan == api.attention_plan(shape, (), [(prefix - _skip(prefix, window, sinks), rows)], kv="e4m3")
    assert plan["query_tiles"] == 1
