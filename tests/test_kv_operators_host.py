"""The KV-cache operators on the CPU: refusals, work lists under a window, and the float64 model of the 8-bit cache."""
import numpy as np
import pytest
from hypothesis import given, settings, strategies as st

from paper_2609_07883_amd import api
from paper_2609_07883_amd.synth import ModelShape
from tests import kv_oracle as O

torch = pytest.importorskip("torch")


def _ctx(layers=2, max_pos=4096):
    return api.Context(layers, 256, 8, 2, 64, 256, 1e-5, 10000.0, max_pos)


def _refused(code, f, *a, **k):
    with pytest.raises(api.SloweaveError) as e:
        f(*a, **k)
    assert e.value.code == code, e.value


def test_pool_refusals():
    c = _ctx()
    for bad in ((0, 64, 64, 64), (64, 0, 64, 64), (64, 64, 0, 64), (64, 64, 64, 0), (8, 64, 64, 64), (64, 72, 64, 64),
                (64, 64, 66, 64), (64, 64, 64, 65)):
        _refused(api.EINVAL, c.kv_init_8bit, *bad, 4)
    _refused(api.EINVAL, c.kv_init_8bit, 64, 64, 64, 64, 0)
    c.kv_init_8bit(64, 64, 64, 64, 7)
    assert c.free_blocks() == 7
    c.kv_init(64, 64, 5)
    assert c.free_blocks() == 5


def test_window_refusals():
    c = _ctx()
    _refused(api.EINVAL, c.set_window, -1)
    _refused(api.EINVAL, c.set_window, 8, -1)
    _refused(api.EINVAL, c.set_window, 8, 4097)
    _refused(api.EINVAL, c.set_window, 0, 4)
    with pytest.raises(ValueError):
        c.set_window(8, 0, [1])
    c.set_window(2**31 - 1, 4096, [0, 1])
    c.set_window(0)


def test_batch_refusals():
    c = _ctx()
    b = api.Batch(0, 0, 0, (1,), (0,))
    _refused(api.EINVAL, c.attn_begin, b, 256, 1 << 30)                     # no pools
    c.kv_init_8bit(64, 64, 64, 64, 4)
    _refused(api.EINVAL, c.attn_begin, b, 256, 1 << 30)                     # unknown sequence
    c.seq_create(1)
    c.seq_create(2)
    n = c.attn_workspace_size(0, 1)
    _refused(api.EINVAL, c.attn_begin, b, 0, n)                             # null workspace
    _refused(api.EINVAL, c.attn_begin, b, 264, n)                           # misaligned
    _refused(api.ENOMEM, c.attn_begin, b, 256, n - 1)                       # short
    _refused(api.EINVAL, c.attn_begin, api.Batch(0, 0, 0, (1, 1), (0, 0)), 256, 1 << 30)      # twice
    _refused(api.EINVAL, c.attn_begin, api.Batch(0, 0, 0, (1,), (3,)), 256, 1 << 30)          # past its tokens
    _refused(api.EINVAL, c.attn_begin, api.Batch(-1, 1, 0, (), ()), 256, 1 << 30)
    _refused(api.ERANGE, c.attn_begin, api.Batch(4097, 1, 0, (), ()), 256, 1 << 30)           # above max_pos
    assert c.free_blocks() == 4
    _refused(api.EINVAL, c.attn_workspace_size, -1, 0)
    plan = c.attn_begin(api.Batch(0, 0, 0, (), ()), 0, 0)                   # no rows: calls do nothing
    plan.append(0, 0, 0, 0)
    plan.attend(1, 0, 0, 0)
    _refused(api.ERANGE, plan.append, 2, 0, 0, 0)
    c.set_window(16)
    _refused(api.EINVAL, plan.attend, 0, 0, 0, 0)
    c.set_window(0)
    plan.attend(0, 0, 0, 0)
    c.kv_init_8bit(64, 64, 64, 64, 4)
    _refused(api.EINVAL, plan.attend, 0, 0, 0, 0)
    c.close()
    _refused(api.EINVAL, plan.attend, 0, 0, 0, 0)
    other = _ctx()
    other.kv_init_8bit(64, 64, 64, 64, 4)
    plan._ctx = other
    _refused(api.EINVAL, plan.append, 0, 0, 0, 0)


def test_workspace_grows_with_what_is_set():
    c = _ctx()
    c.kv_init(64, 64, 4)
    full = c.attn_workspace_size(100, 3)
    it = c.workspace_size(100, 3)
    c.set_window(64, 4, [0, 1])
    assert c.attn_workspace_size(100, 3) > full and c.workspace_size(100, 3) > it
    c.set_window(0)
    assert c.attn_workspace_size(100, 3) == full and c.workspace_size(100, 3) == it
    c.kv_init_8bit(64, 64, 64, 64, 4)
    assert c.workspace_size(100, 3) > it


def _tiles(first, last, window, sinks):
    """64-key tiles that hold a key some row from position first to last sees, or that lie beside the sinks."""
    s = -(-sinks // 64) if window else 0
    lo = max(first - window + 1, 0) // 64 if window else 0
    return len([t for t in range(last // 64 + 1) if t < s or t >= lo])


@settings(max_examples=150, deadline=None)
@given(window=st.integers(0, 3000), sinks=st.integers(0, 400), seed=st.integers(0, 10**6))
def test_window_work_lists(window, sinks, seed):
    sinks = sinks if window else 0
    rng = np.random.default_rng(seed)
    shape = ModelShape(1, 256, 8, 2, 64, 256, max_pos=8192)
    ctxs = rng.integers(0, 8000, rng.integers(0, 20)).tolist()
    pre = [(int(rng.integers(0, 4000)), int(rng.integers(1, 900))) for _ in range(rng.integers(0, 4))]
    plan = api.attention_plan(shape, ctxs, pre, window, sinks, kv="e4m3")
    if window:
        assert plan == api.attention_plan(shape, ctxs, pre, window, sinks)
    else:  # the keys of full attention, divided by other rules
        full = api.attention_plan(shape, ctxs, pre)
        assert plan["chunk_tiles"] == full["chunk_tiles"]
    chunk = sum(_tiles(p + j, min(p + j + 64, p + c) - 1, window, sinks) for p, c in pre for j in range(0, c, 64))
    assert plan["chunk_tiles"] == chunk
    assert plan["decode_max_keys"] * plan["decode_slots"] >= 0
    if ctxs:
        keys = sum(64 * _tiles(c, c, window, sinks) for c in ctxs)
        assert plan["decode_min_keys"] <= keys / plan["decode_slots"] <= plan["decode_max_keys"] + 64
        assert len(ctxs) <= plan["decode_items"] < plan["decode_slots"] + len(ctxs)


def test_decode_runs():
    shape = ModelShape(1, 4096, 32, 8, 128, 256, max_pos=1 << 15)

    def runs(ctxs, pre=()):
        p = api.attention_plan(shape, ctxs, pre, kv="e4m3")
        return p["decode_items"], p["decode_slots"]

    assert runs([250]) == (1, 1) and runs([500]) == (4, 4)  # short: one run; else 128 keys each
    assert runs([830] * 64) == (64, 64)                     # alike: one run each, also where the lengths differ a little
    assert runs([600, 830] * 32) == (64, 64)
    items, slots = runs([300] * 63 + [8000])                # unlike: equal runs for 768 waves
    assert slots <= 96 and items > 64
    assert runs([3000] * 300)[1] <= 96                      # more decodes than wave slots
    full = api.attention_plan(shape, [300] * 63 + [8000], [(8192, 300)])
    assert runs([300] * 63 + [8000], [(8192, 300)]) == (full["decode_items"], full["decode_slots"])
    assert runs([190] * 5, [(50, 77)]) == (5, 5) and runs([300] * 5, [(50, 77)])[0] > 5


def test_plan_window_refusals():
    shape = ModelShape(1, 256, 8, 2, 64, 256, max_pos=512)
    for w, s in ((-1, 0), (4, -1), (4, 513), (0, 4)):
        _refused(api.EINVAL, api.attention_plan, shape, [3], (), w, s)


def test_model_rounding_is_the_formats():
    """Every e4m3 value, every midpoint between two and values beside it: the model's rounding against torch's."""
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    v = torch.unique(v[torch.isfinite(v)])
    mid = (v[1:] + v[:-1]) / 2
    x = torch.cat([v, mid, mid * (1 + 2.0**-20), mid * (1 - 2.0**-20)])
    want = x.float().to(torch.float8_e4m3fn).double()
    assert np.array_equal(O.round_e4m3(x.numpy()), want.numpy())


def test_model_exponent():
    for x, e in ((448.0, 0), (449.0, 1), (224.0, -1), (0.0, -100), (3.3e38, 120), (1e-40, -100), (1.75 * 2.0**-90, -98)):
        assert O.block_exponent(np.array([x, np.nan, np.inf])) == e, x
