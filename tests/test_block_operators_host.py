"""The operators round the cache on the CPU: refusals, sizes, and the float64 models on cases worked by hand."""
import math

import numpy as np
import pytest

from paper_2609_07883_amd import api
from tests import block_oracle as O


def _refused(code, f, *a, **k):
    with pytest.raises(api.SloweaveError) as e:
        f(*a, **k)
    assert e.value.code == code, e.value


# -- residual norm ------------------------------------------------------------------

def _norm(rows=1, d=64, resid=64, block=64, resid_out=64, gain=64, out=64, **k):
    api.residual_norm(rows, d, resid, block, resid_out, gain, out, **k)


def test_norm_refusals():
    for d in (0, 4, 12, 32776, -8):
        _refused(api.EUNSUPPORTED, _norm, d=d)
    _refused(api.EINVAL, _norm, rows=-1)
    _refused(api.EINVAL, _norm, resid=0)
    _refused(api.EINVAL, _norm, gain=0)
    _refused(api.EINVAL, _norm, out=0, resid_out=0)
    _refused(api.EINVAL, _norm, block=0, gate=64)
    _refused(api.EINVAL, _norm, block=0, post_gain=64)
    for name in ("resid", "block", "resid_out", "gain", "out", "gate", "post_gain"):
        _refused(api.EINVAL, _norm, **{name: 72})
    for name in ("ld_resid", "ld_block", "ld_resid_out", "ld_out"):
        _refused(api.EINVAL, _norm, **{name: 56})
        _refused(api.EINVAL, _norm, **{name: 68})
    _refused(api.EINVAL, _norm, gate=64, ld_gate=56)
    for eps in (-1e-6, math.nan, math.inf):
        _refused(api.EINVAL, _norm, eps=eps)
    _refused(api.EINVAL, _norm, scale=math.nan)
    _norm(rows=0)                                                # nothing to do


# -- products -----------------------------------------------------------------------

def test_w4_sizes_and_refusals():
    assert api.w4_packed_bytes(16, 128) == 1024 + 256
    assert api.w4_packed_bytes(17, 160) == 2 * (2 * 1024 + 256)   # padded to tiles of 16 rows, steps of 128
    assert api.w4_packed_bytes(34, 128, True) == 4 * (1024 + 256)  # 17 gate rows and 17 up rows, padded each
    for n, k, gated in ((0, 32, 0), (1, 0, 0), (1, 16, 0), (1, 33, 0), (3, 32, 1), (1, 65568, 0), ((1 << 22) + 1, 32, 0), (-16, 32, 0)):
        _refused(api.EUNSUPPORTED, api.w4_packed_bytes, n, k, bool(gated))
    w = api.W4(64, 32, 64)
    for m in (1, 16, 100, 5000):
        assert w.workspace_size(m) >= 0
    _refused(api.EINVAL, w.workspace_size, -1)
    _refused(api.EINVAL, w.pack, 0, 64)
    _refused(api.EINVAL, w.pack, 64, 0)
    _refused(api.EINVAL, w.pack, 72, 64)
    _refused(api.EINVAL, api.W4(0, 32, 64).pack, 64, 64)
    _refused(api.EINVAL, api.W4(72, 32, 64).pack, 64, 64)
    w.product(0, 0, 0, 0, 0)                                      # no rows
    ws = dict(ws=64, ws_bytes=1 << 40)
    _refused(api.EINVAL, w.product, 64, 64, -1, 64, 32, **ws)
    _refused(api.EUNSUPPORTED, w.product, 64, 64, (1 << 20) + 1, 64, 32, **ws)
    for a, lda, out, ldo, f32 in ((0, 64, 64, 32, 0), (72, 64, 64, 32, 0), (64, 56, 64, 32, 0), (64, 68, 64, 32, 0),
                                  (64, 64, 0, 32, 0), (64, 64, 65, 32, 0), (64, 64, 66, 32, 1), (64, 64, 64, 31, 0)):
        _refused(api.EINVAL, w.product, a, lda, 1, out, ldo, out_f32=bool(f32), **ws)
    _refused(api.EINVAL, api.W4(64, 32, 64, True).product, 64, 64, 1, 64, 15, **ws)
    _refused(api.EUNSUPPORTED, api.W4(64, 33, 64, True).product, 64, 64, 1, 64, 32, **ws)


def test_w4_model_by_hand():
    codes = np.zeros((1, 16), np.uint8)
    codes[0, :8] = [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]
    w = O.weights(codes, np.array([[128]], np.uint8))[0]
    assert w[:16].tolist() == [0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12]
    a = np.zeros((1, 32))
    a[0, 1], a[0, 15] = 3, 0.5
    assert O.product(a, w[None])[0][0, 0] == 3 * 1 + 0.5 * -12


# -- rotary rows --------------------------------------------------------------------

def _plan():
    c = api.Context(2, 256, 8, 2, 64, 256, 1e-5, 10000.0, 4096)
    c.kv_init(64, 64, 4)
    return c, c.attn_begin(api.Batch(0, 0, 0, (), ()), 0, 0)       # an empty batch needs no GPU


def test_rotate_refusals():
    c, plan = _plan()
    good = api.Rope(64, 10000.0)
    call = lambda rope=good, q=64, k=64, ld=768, qo=64, ko=64, ldo=768: plan.rotate(rope, q, k, ld, qo, ko, ldo)
    call()
    call(k=0, ko=0)
    call(q=0, qo=0, ld=128, ldo=128)
    for rot in (0, 8, 24, 80, 128, -16):
        _refused(api.EUNSUPPORTED, call, rope=api.Rope(rot, 10000.0))
    for theta in (0.0, -1.0, math.nan, math.inf):
        _refused(api.EINVAL, call, rope=api.Rope(64, theta))
    for scaling in ("linear", "ntk", "by_parts"):
        for factor in (0.0, -2.0, math.nan, math.inf):
            _refused(api.EINVAL, call, rope=api.Rope(64, 1e4, scaling=scaling, factor=factor, original_len=8192))
        call(rope=api.Rope(64, 1e4, scaling=scaling, factor=4.0, original_len=8192))
    _refused(api.EINVAL, call, rope=api.Rope(64, 1e4, scaling="by_parts", factor=2.0, original_len=0))
    _refused(api.EINVAL, call, rope=api.Rope(64, 1e4, scaling="by_parts", factor=2.0, low=4.0, high=4.0, original_len=8))
    _refused(api.EINVAL, call, rope=api.Rope(64, scaling="table"))
    _refused(api.EINVAL, call, rope=api.Rope(64, scaling="table", freq=68))
    _refused(api.EINVAL, call, rope=api.Rope(64, 1e4, mscale=math.inf))
    bad = api.Rope(64, 1e4)
    bad.c.interleaved = 2
    _refused(api.EINVAL, call, rope=bad)
    bad = api.Rope(64, 1e4)
    bad.c.scaling = 5
    _refused(api.EINVAL, call, rope=bad)
    _refused(api.EINVAL, call, q=0, k=0, qo=0, ko=0)
    _refused(api.EINVAL, call, qo=0)
    _refused(api.EINVAL, call, k=0)
    for name in ("q", "k", "qo", "ko"):
        _refused(api.EINVAL, call, **{name: 72})
    for name in ("ld", "ldo"):
        _refused(api.EINVAL, call, **{name: 504})
        _refused(api.EINVAL, call, **{name: 772})
    c.kv_init(64, 64, 4)
    _refused(api.EINVAL, call)                                     # a plan of other pools


def test_rotary_models_by_hand():
    f = O.frequencies(4, 100.0)
    assert np.allclose(f, [1.0, 0.1])
    assert np.allclose(O.frequencies(4, 100.0, "linear", 4.0), [0.25, 0.025])
    assert np.allclose(O.frequencies(4, 100.0, "ntk", 3.0), [1.0, 900.0**-0.5])     # theta 100 * 3^(4/2)
    # original length 2 pi * 8: the first pair turns 8 times in it (kept), the second 0.8 times (all slowed down)
    n = 2 * math.pi * 8
    assert np.allclose(O.frequencies(4, 100.0, "by_parts", 4.0, 1.0, 4.0, n), [1.0, 0.025])
    assert np.allclose(O.frequencies(4, 100.0, "by_parts", 4.0, 0.4, 1.2, n), [1.0, 0.1 * (0.5 / 4 + 0.5)])
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    y, _ = O.rotate(x, [math.pi / 2], np.array([1.0, 0.0]), mscale=2.0)
    assert np.allclose(y, [[[-6.0, 4.0, 2.0, 8.0, 5.0]]])
    y, _ = O.rotate(x, [math.pi / 2], np.array([1.0, 0.0]), interleaved=True)
    assert np.allclose(y, [[[-2.0, 1.0, 3.0, 4.0, 5.0]]])


# -- sampling -----------------------------------------------------------------------

def test_sample_refusals():
    call = lambda logits=64, rows=1, vocab=100, ld=100, u=64, tokens=64, **k: api.sample(
        logits, rows, vocab, ld, u, tokens, **{"ws": 64, "ws_bytes": 1 << 40, **k})
    for vocab in (0, -1, (1 << 20) + 1):
        _refused(api.EUNSUPPORTED, call, vocab=vocab, ld=1 << 21)
        _refused(api.EUNSUPPORTED, api.sample_workspace_size, 1, vocab)
    _refused(api.EINVAL, call, rows=-1)
    _refused(api.EINVAL, api.sample_workspace_size, -1, 100)
    for name in ("logits", "u", "tokens"):
        _refused(api.EINVAL, call, **{name: 0})
    _refused(api.EINVAL, call, logits=65)
    _refused(api.EINVAL, call, logits=66, logits_f32=True)
    _refused(api.EINVAL, call, ld=99)
    for name in ("u", "tokens", "temperature", "top_k", "top_p", "min_p", "logprob"):
        _refused(api.EINVAL, call, **{name: 66})
    call(rows=0)


def test_sample_workspace_refusals():
    call = lambda **k: api.sample(64, 4, 1000, 1000, 64, 64, **k)
    size = api.sample_workspace_size(4, 1000)
    assert size > 0 and api.sample_workspace_size(0, 1000) == 0
    _refused(api.EINVAL, call, ws=0, ws_bytes=size)
    _refused(api.EINVAL, call, ws=72, ws_bytes=size)
    _refused(api.ENOMEM, call, ws=64, ws_bytes=0)
    _refused(api.ENOMEM, lambda: api.sample(64, 4, 1 << 20, 1 << 20, 64, 64, ws=64, ws_bytes=size))


@pytest.mark.parametrize("vocab", [1, 8192, 8193, 50000, 1 << 20])
def test_sample_workspace_grows_with_the_rows(vocab):
    """What fits some rows fits fewer, whatever slices those are cut into."""
    sizes = [api.sample_workspace_size(r, vocab) for r in (1, 2, 63, 64, 65, 127, 128, 129, 500, 512, 513, 1023, 1024, 1025, 5000)]
    assert sizes == sorted(sizes)


def test_rows_beyond_the_most():
    most = 1 << 20
    _refused(api.EUNSUPPORTED, _norm, rows=most + 1)
    _refused(api.EUNSUPPORTED, api.sample, 64, most + 1, 8, 8, 64, 64, ws=64, ws_bytes=1 << 50)
    _refused(api.EUNSUPPORTED, api.sample_workspace_size, most + 1, 8)
    _refused(api.EUNSUPPORTED, api.W4(64, 32, 64).product, 64, 64, most + 1, 64, 32, ws=64, ws_bytes=1 << 50)


def test_w4_workspace_refusals():
    """A k that is split needs its workspace; what fits some rows fits fewer."""
    w = api.W4(64, 4096, 14336)
    sizes = [w.workspace_size(m) for m in range(0, 5000, 7)]
    assert sizes[0] == 0 and sizes == sorted(sizes)
    m = 48
    need = w.workspace_size(m)
    assert need > 0
    _refused(api.EINVAL, w.product, 64, 14336, m, 64, 4096)
    _refused(api.EINVAL, w.product, 64, 14336, m, 64, 4096, ws=72, ws_bytes=need)
    _refused(api.ENOMEM, w.product, 64, 14336, m, 64, 4096, ws=64, ws_bytes=16)


def test_sample_model_by_hand():
    x = np.log([0.5, 0.125, 0.25, 0.125])
    assert [O.sample(x, u=u)[0] for u in (0.0, 0.49, 0.51, 0.63, 0.7, 0.9)] == [0, 0, 1, 2, 2, 3]
    assert O.sample(x, temperature=0.0) == (0, 0.0)
    assert [O.sample(x, top_k=2, u=u)[0] for u in (0.6, 0.7)] == [0, 2]
    assert [O.sample(x, top_k=3, u=u)[0] for u in (0.56, 0.58, 0.99)] == [0, 1, 2]  # of the equal ones the lower index
    assert math.isclose(O.sample(x, top_k=2, u=0.9)[1], math.log(1 / 3))
    assert [O.sample(x, top_p=0.7, u=u)[0] for u in (0.6, 0.7)] == [0, 2]            # 0.5 is short of 0.7, 0.75 is not
    assert O.sample(x, top_p=0.5, u=0.9)[0] == 0
    assert [O.sample(x, min_p=0.4, u=u)[0] for u in (0.6, 0.7)] == [0, 2]
    assert O.sample(np.full(3, -np.inf)) == (-1, -math.inf)
    assert O.sample(np.array([math.nan, 1.0]), u=0.999)[0] == 1
    assert O.sample(np.array([0.0, math.inf, math.inf]), u=0.6) == (2, math.log(0.5))
