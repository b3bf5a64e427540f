"""GPU tests of the operators round the cache against their float64 models (tests/block_oracle.py): residual norms, 4-bit
products, rotary rows, sampling; and a decoder block made of them and the cache operators."""
import math

import numpy as np
import pytest

from paper_2609_07883_amd import api
from tests import block_oracle as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _bf16(x):
    """float64 array -> (bf16 tensor on the GPU, its values)."""
    t = torch.from_numpy(np.ascontiguousarray(x, np.float64)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def _f64(t):
    return t.detach().cpu().double().numpy()


def _padded(t, ld, fill=math.nan):
    """The rows of t in a buffer of row stride ld, other values `fill`."""
    buf = torch.full((t.shape[0], ld), fill, dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t
    return buf


def _within(got, want, bound, kind):
    tol = bound + O.ROUND[kind] * (np.abs(want) + bound)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])


# -- residual norm ------------------------------------------------------------------

@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("post,gate", [(False, None), (True, None), (False, "row"), (True, "channel")])
@pytest.mark.parametrize("rows,d", [(1, 8), (5, 256), (3, 512), (2, 520), (7, 2048), (1, 4096), (9, 4104), (2, 8192), (3, 8200),
                                    (2, 32768)])
def test_residual_norm(rows, d, post, gate, f32):
    rng = np.random.default_rng([rows, d, post, f32])
    kind = "f32" if f32 else "bf16"
    resid = torch.from_numpy(rng.standard_normal((rows, d)) * 4).to(torch.float32 if f32 else torch.bfloat16).cuda()
    r = _f64(resid)
    block, o = _bf16(rng.standard_normal((rows, d)))
    gain, g = _bf16(1 + 0.2 * rng.standard_normal(d))
    pg, p = _bf16(0.5 + 0.2 * rng.standard_normal(d))
    gt, t = _bf16(rng.standard_normal((rows if gate == "row" else 1, d)))
    lds = dict(ld_resid=d + 8, ld_block=d + 16, ld_resid_out=d + 24, ld_out=d + 32)
    resid, block = _padded(resid, d + 8), _padded(block, d + 16)
    resid_out = torch.full((rows, d + 24), 7.0, dtype=resid.dtype, device="cuda")
    out = torch.full((rows, d + 32), 7.0, dtype=torch.bfloat16, device="cuda")
    api.residual_norm(rows, d, resid.data_ptr(), block.data_ptr(), resid_out.data_ptr(), gain.data_ptr(), out.data_ptr(),
                      resid_f32=f32, eps=1e-6, post_gain=pg.data_ptr() if post else 0, gate=gt.data_ptr() if gate else 0,
                      ld_gate=d if gate == "row" else 0, scale=0.7, stream=_stream(), **lds)
    new, nb, y, yb = O.norm(r, o, g, p if post else None, t if gate else None, np.float32(0.7), 1e-6)
    _within(_f64(resid_out[:, :d]), new, nb, kind)
    _within(_f64(out[:, :d]), y, yb, "bf16")
    assert (resid_out[:, d:] == 7).all() and (out[:, d:] == 7).all()


@pytest.mark.parametrize("d", [64, 1024, 4096, 16384])
def test_residual_norm_parts_and_in_place(d):
    """The norm alone, the sum alone, outputs over the inputs; all as the call that does everything."""
    rng = np.random.default_rng(d)
    resid, r = _bf16(rng.standard_normal((6, d)))
    block, o = _bf16(rng.standard_normal((6, d)))
    gain, g = _bf16(1 + 0.2 * rng.standard_normal(d))
    want_r, want_y = torch.empty_like(resid), torch.empty_like(resid)
    api.residual_norm(6, d, resid.data_ptr(), block.data_ptr(), want_r.data_ptr(), gain.data_ptr(), want_y.data_ptr(), stream=_stream())
    _, _, y, yb = O.norm(r, o, g)
    _within(_f64(want_y), y, yb, "bf16")
    only = torch.empty_like(resid)
    api.residual_norm(6, d, resid.data_ptr(), block.data_ptr(), only.data_ptr(), 0, 0, stream=_stream())
    assert torch.equal(only, want_r)
    api.residual_norm(6, d, resid.data_ptr(), block.data_ptr(), 0, gain.data_ptr(), only.data_ptr(), stream=_stream())
    assert torch.equal(only, want_y)
    api.residual_norm(6, d, resid.data_ptr(), 0, 0, gain.data_ptr(), only.data_ptr(), stream=_stream())
    _, _, y, yb = O.norm(r, None, g)
    _within(_f64(only), y, yb, "bf16")
    api.residual_norm(6, d, resid.data_ptr(), block.data_ptr(), resid.data_ptr(), gain.data_ptr(), block.data_ptr(), stream=_stream())
    assert torch.equal(resid, want_r) and torch.equal(block, want_y)


def test_residual_norm_of_zeros_infinities_and_nan():
    x = torch.zeros(5, 256, dtype=torch.bfloat16, device="cuda")
    x[1, 3], x[2, 5], x[3] = math.nan, math.inf, 1e-30
    x[4] = torch.arange(256)
    gain = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    api.residual_norm(5, 256, x.data_ptr(), 0, 0, gain.data_ptr(), y.data_ptr(), stream=_stream())
    assert (y[0] == 0).all() and y[1].isnan().all()
    assert y[2, 5].isnan() and (y[2, :5] == 0).all() and (y[2, 6:] == 0).all()
    _, _, want, b = O.norm(_f64(x[3:]), None, np.ones(256))
    _within(_f64(y[3:]), want, b, "bf16")


# -- products -----------------------------------------------------------------------

class Weights:
    """Random codes and scales on the GPU, packed, and their values."""

    def __init__(self, n, k, gated=False, seed=0, lo=118, hi=124, codes=None, scales=None):
        rng = np.random.default_rng([n, k, gated, seed])
        self.codes = rng.integers(0, 256, (n, k // 2), dtype=np.uint8) if codes is None else codes
        self.scales = rng.integers(lo, hi, (n, k // 32), dtype=np.uint8) if scales is None else scales
        c, s = torch.from_numpy(self.codes).cuda(), torch.from_numpy(self.scales).cuda()
        self.packed = torch.full((api.w4_packed_bytes(n, k, gated) + 64,), 255, dtype=torch.uint8, device="cuda")
        self.w = api.W4(self.packed.data_ptr(), n, k, gated)
        self.w.pack(c.data_ptr(), s.data_ptr(), _stream())
        torch.cuda.synchronize()
        assert (self.packed[-64:] == 255).all()
        self.n, self.k, self.gated, self.n_out = n, k, gated, n // 2 if gated else n
        self.values = O.weights(self.codes, self.scales)

    def product(self, a, m, lda, f32=False, ldo=None, guard=7.0):
        ldo = ldo or self.n_out
        out = torch.full((m + 1, ldo), guard, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        size = self.w.workspace_size(m)
        ws = torch.full((size + 64,), 255, dtype=torch.uint8, device="cuda")
        self.w.product(a.data_ptr(), lda, m, out.data_ptr(), ldo, out_f32=f32, ws=ws.data_ptr(), ws_bytes=size, stream=_stream())
        torch.cuda.synchronize()
        assert (out[m:] == guard).all() and (out[:, self.n_out:] == guard).all() and (ws[size:] == 255).all()
        return out[:m, :self.n_out]


SHAPES = [(16, 32, False), (1, 64, False), (2, 128, True), (256, 704, False), (1408, 256, True), (250, 160, True), (33, 1056, False),
          (768, 256, False), (4096, 512, False), (130, 4096, False), (96, 14336, False), (62, 2080, True)]


@pytest.mark.parametrize("n,k,gated", SHAPES)
@pytest.mark.parametrize("m", [1, 3, 16, 17, 31, 40, 64, 65, 130, 300])
def test_product(n, k, gated, m):
    w = Weights(n, k, gated)
    rng = np.random.default_rng([n, k, m])
    a, av = _bf16(rng.standard_normal((m, k)))
    want, bound = O.product(av, w.values, gated)
    for f32 in (False, True):
        got = w.product(_padded(a, k + 8), m, k + 8, f32, ldo=w.n_out + 3 if m % 2 else None)
        _within(_f64(got), want, bound, "f32" if f32 else "bf16")


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (5, 6144, 4096), (24, 28672, 4096), (48, 4096, 14336), (100, 5000, 4096),
                                   (257, 6144, 4096), (600, 4096, 4096), (1025, 2050, 1056), (2080, 4096, 4096)])
def test_product_of_whole_numbers_is_exact(m, n, k):
    """Weights of k/32 groups with one scale and small whole activations: sums stay below 2^24 in any order."""
    rng = np.random.default_rng([m, n, k])
    w = Weights(n, k, False, scales=np.full((n, k // 32), 128, np.uint8))
    a = rng.integers(-4, 5, (m, k))
    t = torch.from_numpy(a).to(torch.bfloat16).cuda()
    want = t.float() @ torch.from_numpy(w.values).float().cuda().T        # whole numbers: exact
    assert torch.equal(w.product(t, m, k, True), want)


@pytest.mark.parametrize("m,n,k", [(12, 70001, 288), (20, 64, 8448), (16, 300, 10016), (32, 9000, 160), (50, 100, 8224), (68, 17, 928),
                                   (1038, 16, 4192), (196, 10918, 96), (102, 2108, 4000), (132, 10962, 32), (2056, 16, 4064),
                                   (265, 13112, 160), (65, 8578, 1952), (4673, 1549, 32), (2210, 277, 7904), (392, 13064, 64),
                                   (3129, 131, 5920), (514, 13223, 32), (129, 6451, 5792), (661, 13249, 160), (2732, 260, 10240),
                                   (770, 13149, 288)])
def test_product_of_every_shape_of_work_group_is_exact(m, n, k):
    """The same where the rows, columns and k ask for each size of tile, with k whole and split."""
    test_product_of_whole_numbers_is_exact(m, n, k)


@pytest.mark.parametrize("m,n,k", [(11, 131074, 64), (23, 66, 8224), (64, 514, 4128), (131, 272, 9472), (263, 13124, 32), (648, 1082, 288)])
def test_gated_product_of_more_shapes(m, n, k):
    w = Weights(n, k, True)
    a, av = _bf16(np.random.default_rng([m, n, k]).standard_normal((m, k)))
    _within(_f64(w.product(a, m, k, True)), *O.product(av, w.values, True), "f32")


def test_product_columns_do_not_mix():
    """Row i of a picks column i of W: every code of every lane comes back, once a group of scales."""
    n, k = 112, 384
    w = Weights(n, k, False, lo=100, hi=150)
    a = torch.eye(k, dtype=torch.bfloat16, device="cuda")
    assert np.array_equal(_f64(w.product(a, k, k, True)), w.values.T)
    assert np.array_equal(_f64(w.product(a[5:6], 1, k, True)), w.values.T[5:6])


def test_product_of_every_scale():
    """Scales from the smallest to the largest: a weight is its value as a bf16 number."""
    scales = np.arange(256, dtype=np.uint8).reshape(128, 2)
    codes = np.tile(np.array([0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE], np.uint8), (128, 4))
    w = Weights(128, 64, False, codes=codes, scales=scales)
    a = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    with np.errstate(over="ignore"):
        want = torch.from_numpy(w.values).to(torch.bfloat16)
    want[127, 32:] = math.nan
    got = w.product(a, 64, 64, True).cpu().T
    zero_inf = want.isinf().any(1, keepdim=True)       # 0 * inf in a row that has infinities is NaN
    ok = torch.isclose(got, want.float(), rtol=0, atol=0, equal_nan=True)
    bad = (scales >= 253).any(1)
    assert ok[~bad].all()
    assert got[127].isnan().all() and zero_inf[126].all()


@pytest.mark.parametrize("m", [1, 30, 40])
def test_product_of_rows_far_apart(m):
    """A row stride past what 32-bit offsets within a tile reach."""
    w = Weights(48, 64)
    ld = (1 << 22) + 8
    buf = torch.zeros(m * ld, dtype=torch.bfloat16, device="cuda").view(m, ld)
    a, av = _bf16(np.random.default_rng(m).standard_normal((m, 64)))
    buf[:, :64] = a
    want, bound = O.product(av, w.values)
    _within(_f64(w.product(buf, m, ld, True)), want, bound, "f32")


def test_product_rows_keep_to_themselves():
    """Infinities and NaN in a row of a, and rows behind the last, stay out of the others."""
    w = Weights(320, 512)
    rng = np.random.default_rng(2)
    for m in (5, 20, 70, 200):
        a, av = _bf16(rng.standard_normal((m + 8, 512)))
        want = w.product(a, m, 512, True).clone()
        a[m:], a[m // 2, 7], a[m // 3, 0] = math.nan, math.inf, math.nan
        got = w.product(a, m, 512, True)
        keep = torch.ones(m, dtype=torch.bool)
        keep[m // 2] = keep[m // 3] = False
        assert torch.equal(got[keep], want[keep])
        assert got[m // 3].isnan().all()


def test_gated_product_of_large_values():
    """silu far out: 0 for large negative gates, the gate itself for large positive ones; no NaN."""
    codes = np.zeros((4, 16), np.uint8)
    codes[:, 0] = 0x02                                           # 1.0 at k = 0
    w = Weights(4, 32, True, codes=codes, scales=np.full((4, 1), 127, np.uint8))
    x = torch.tensor([-1e30, -200.0, -90.0, 0.0, 90.0, 1e15], dtype=torch.bfloat16, device="cuda")
    a = torch.zeros(6, 32, dtype=torch.bfloat16, device="cuda")
    a[:, 0] = x
    got, v = _f64(w.product(a, 6, 32, True)), _f64(x)
    want = O.silu(v) * v
    assert np.allclose(got, want[:, None], rtol=2.0**-20, atol=1e-30)


# -- rotary rows --------------------------------------------------------------------

def _plan(hd, hq, hkv, prompts, decodes, max_pos=1 << 20):
    ctx = api.Context(1, 256, hq, hkv, hd, 256, 1e-5, 10000.0, max_pos)
    blocks = sum(-(-(p + n) // 16) for p, n in prompts) + sum(p // 16 + 1 for p in decodes)
    # the pools are not touched: only their addresses are kept
    pool = torch.empty(64, dtype=torch.bfloat16, device="cuda")
    ctx.kv_init(pool.data_ptr(), pool.data_ptr(), max(blocks, 1))
    ids = list(range(1, 1 + len(prompts) + len(decodes)))
    for sid, p in zip(ids, [p for p, _ in prompts] + decodes):
        ctx.seq_create(sid)
        ctx.seq_reserve(sid, p)
    batch = api.Batch.batched([(s, p, n) for s, (p, n) in zip(ids, prompts)], ids[len(prompts):], decodes)
    ws = torch.empty(ctx.attn_workspace_size(batch.chunk, len(decodes)), dtype=torch.uint8, device="cuda")
    plan = ctx.attn_begin(batch, ws.data_ptr(), ws.numel(), _stream())
    pos = [p + j for p, n in prompts for j in range(n)] + decodes
    return plan, pos, (ctx, pool, ws)


BATCHES = [([], [0]), ([], [1048575, 3, 70000]), ([(0, 1)], []), ([(100, 37)], [5, 900]), ([(1000, 5), (0, 70), (0, 1), (0, 30)], [64] * 9)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd,hq,hkv,rot", [(64, 4, 4, 64), (64, 8, 2, 16), (128, 32, 8, 128), (128, 8, 8, 48), (128, 16, 1, 64)])
@pytest.mark.parametrize("batch", range(len(BATCHES)))
def test_rotate(hd, hq, hkv, rot, interleaved, batch):
    prompts, decodes = BATCHES[batch]
    plan, pos, keep = _plan(hd, hq, hkv, prompts, decodes)
    rows, heads = len(pos), hq + hkv
    rng = np.random.default_rng([hd, hq, rot, batch])
    qkv, v = _bf16(rng.standard_normal((rows, (heads + hkv) * hd)))
    ld, ldo = qkv.shape[1], heads * hd + 16
    x = v[:, :heads * hd].reshape(rows, heads, hd)
    for scaling, factor in (("none", 1.0), ("linear", 3.3), ("ntk", 4.0), ("by_parts", 8.0), ("table", 1.0)):
        f = O.frequencies(rot, 500000.0, scaling, factor) if scaling != "table" else rng.uniform(0, 3, rot // 2)
        table = torch.from_numpy(f).cuda()
        rope = api.Rope(rot, 500000.0, interleaved=interleaved, scaling=scaling, factor=factor, original_len=8192,
                        freq=table.data_ptr(), mscale=1.25)
        want, bound = O.rotate(x, pos, f, interleaved, 1.25)
        out = torch.full((rows, ldo), 7.0, dtype=torch.bfloat16, device="cuda")
        plan.rotate(rope, qkv.data_ptr(), qkv.data_ptr() + 2 * hq * hd, ld, out.data_ptr(), out.data_ptr() + 2 * hq * hd, ldo, _stream())
        _within(_f64(out[:, :heads * hd]).reshape(x.shape), want, bound, "bf16")
        assert (out[:, heads * hd:] == 7).all()
        assert torch.equal(out[:, :heads * hd].view(rows, heads, hd)[..., rot:], qkv[:, :heads * hd].view(rows, heads, hd)[..., rot:])
        place = qkv.clone()
        plan.rotate(rope, place.data_ptr(), place.data_ptr() + 2 * hq * hd, ld, place.data_ptr(), place.data_ptr() + 2 * hq * hd, ld, _stream())
        assert torch.equal(place[:, :heads * hd], out[:, :heads * hd]) and torch.equal(place[:, heads * hd:], qkv[:, heads * hd:])
        for part in range(2):
            alone = torch.full_like(out, 7.0)
            q = [qkv.data_ptr(), 0] if part == 0 else [0, qkv.data_ptr() + 2 * hq * hd]
            o = [alone.data_ptr(), 0] if part == 0 else [0, alone.data_ptr() + 2 * hq * hd]
            plan.rotate(rope, *q, ld, *o, ldo, _stream())
            lo, hi = (0, hq * hd) if part == 0 else (hq * hd, heads * hd)
            assert torch.equal(alone[:, lo:hi], out[:, lo:hi]) and (alone[:, :lo] == 7).all() and (alone[:, hi:] == 7).all()


# -- sampling -----------------------------------------------------------------------

def _sample(x, f32=True, ld=None, shift=0, **par):
    """tokens and logprobs of rows x (float64), drawn with the parameters in par (arrays, or None: left out)."""
    rows, vocab = x.shape
    ld = ld or vocab
    buf = torch.full((rows * ld + shift + 8,), 1e30, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    t = torch.from_numpy(x).to(buf.dtype).cuda()
    view = buf[shift:shift + rows * ld].view(rows, ld)
    view[:, :vocab] = t
    dev = {}
    for name, dtype in (("temperature", np.float32), ("top_k", np.int32), ("top_p", np.float32), ("min_p", np.float32), ("u", np.float32)):
        if par.get(name) is not None:
            dev[name] = torch.from_numpy(np.broadcast_to(np.asarray(par[name], dtype), (rows,)).copy()).cuda()
    tokens = torch.full((rows + 1,), -7, dtype=torch.int32, device="cuda")
    logprob = torch.full((rows + 1,), 7.0, dtype=torch.float32, device="cuda")
    size = api.sample_workspace_size(rows, vocab)
    ws = torch.full((size + 64,), 255, dtype=torch.uint8, device="cuda")
    api.sample(view.data_ptr(), rows, vocab, ld, dev["u"].data_ptr(), tokens.data_ptr(), logits_f32=f32, logprob=logprob.data_ptr(),
               ws=ws.data_ptr(), ws_bytes=size, stream=_stream(), **{k: v.data_ptr() for k, v in dev.items() if k != "u"})
    torch.cuda.synchronize()
    assert tokens[rows] == -7 and logprob[rows] == 7 and (ws[size:] == 255).all()
    return tokens[:rows].cpu().numpy(), logprob[:rows].cpu().double().numpy(), t.double().cpu().numpy()


def _check(x, f32=True, ld=None, shift=0, **par):
    got, lp, v = _sample(x, f32, ld, shift, **par)
    names = [k for k in ("temperature", "top_k", "top_p", "min_p", "u") if par.get(k) is not None]
    cols = [np.broadcast_to(np.asarray(par[k], np.int32 if k == "top_k" else np.float32), (len(v),)) for k in names]
    for r in range(len(v)):
        p = {k: (int(c[r]) if k == "top_k" else float(c[r])) for k, c in zip(names, cols)}
        token, want = O.sample(v[r], **p)
        assert got[r] == token, (r, p, got[r], token)
        # one rounding to fp32 of a logarithm right to 2^-40
        assert lp[r] == want or abs(lp[r] - want) <= 2.0**-24 * abs(want) + 2.0**-40, (r, p, lp[r], want)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 65, 511, 513, 1000, 4099, 8191, 32768, 50001])
def test_sample(vocab, f32):
    """Rows of every kind of parameters over vocabularies of every fit to the pieces."""
    rng = np.random.default_rng([vocab, f32])
    rows = 24
    x = rng.standard_normal((rows, vocab)) * rng.choice([0.3, 1.0, 3.0], (rows, 1))
    t = rng.uniform(0.5, 1.5, rows)
    t[::6] = 0
    k = np.where(rng.random(rows) < 0.5, rng.integers(1, 60, rows), 0)
    p = np.where(rng.random(rows) < 0.5, rng.uniform(0.3, 0.99, rows), 1.0)
    low = np.where(rng.random(rows) < 0.3, rng.uniform(0.01, 0.3, rows), 0.0)
    _check(x, f32, ld=vocab + 5, shift=3, temperature=t, top_k=k, top_p=p, min_p=low, u=rng.random(rows))


@pytest.mark.parametrize("par", [dict(), dict(top_k=5000), dict(top_k=20000), dict(top_p=0.97), dict(top_p=0.5), dict(min_p=0.5),
                                 dict(top_k=9000, top_p=0.9), dict(top_k=9000, top_p=0.2, min_p=0.9), dict(top_k=30),
                                 dict(temperature=50.0, top_p=0.3), dict(temperature=1e30, top_k=7000)])
@pytest.mark.parametrize("f32", [False, True])
def test_sample_of_flat_rows(par, f32):
    """Many tokens kept, with equal logits at the cuts."""
    rng = np.random.default_rng(4)
    x = rng.standard_normal((6, 30011)) * 0.4
    x[1] = 0
    x[2] = np.where(rng.random(30011) < 0.3, -1.5, 2.5)
    x[3] = np.round(x[3] * 4) / 4
    _check(x, f32, u=[0.0, 0.25, 0.5, 0.999, 0.9999999, 0.3], **par)


def test_sample_of_equal_logits_keeps_the_lower_indices():
    x = np.zeros((5, 100))
    u = np.array([0.0, 0.2, 0.5, 0.8, 0.999])
    got, _, _ = _sample(x, top_k=10, u=u)
    assert got.tolist() == [0, 2, 5, 8, 9]
    got, _, _ = _sample(x, top_p=0.5, u=u)
    assert got.tolist() == [0, 10, 25, 40, 49]
    got, _, _ = _sample(x, u=u)
    assert got.tolist() == [0, 20, 50, 80, 99]


@pytest.mark.parametrize("f32", [False, True])
def test_sample_of_masked_rows(f32):
    """-inf, +inf, NaN and the type's lowest value among the logits; a row of nothing; one token left."""
    rng = np.random.default_rng(8)
    low = float(torch.finfo(torch.float32 if f32 else torch.bfloat16).min)
    x = rng.standard_normal((10, 777))
    x[0] = -np.inf
    x[1, 5:] = -np.inf
    x[2, 100:] = low
    x[3, [7, 9]] = np.inf
    x[4] = np.nan
    x[5, ::2] = np.nan
    x[6] = -np.inf
    x[6, 776] = -3
    x[7] = low
    x[8, 3] = -low
    x[9] = np.where(np.arange(777) % 2, 0.0, -0.0)
    for par in (dict(), dict(top_k=3), dict(top_p=0.6), dict(min_p=0.2), dict(temperature=0.0), dict(top_k=700, top_p=0.9)):
        for u in (0.0, 0.3, 0.77, 0.99999994):
            _check(x, f32, u=u, **par)


def test_sample_of_odd_parameters():
    rng = np.random.default_rng(9)
    x = rng.standard_normal((1, 2000)) * 2
    nan, inf = math.nan, math.inf
    for par in (dict(temperature=nan), dict(temperature=-1.0), dict(temperature=inf), dict(temperature=1e-30), dict(temperature=1e-44),
                dict(temperature=1e-3), dict(top_k=-5), dict(top_k=2000), dict(top_k=1999), dict(top_k=2**31 - 1), dict(top_k=1),
                dict(top_p=nan), dict(top_p=-1.0), dict(top_p=0.0), dict(top_p=1e-30), dict(top_p=2.0), dict(top_p=0.99999994),
                dict(min_p=nan), dict(min_p=-1.0), dict(min_p=1.0), dict(min_p=7.0), dict(min_p=1e-30), dict()):
        for u in (nan, -1.0, 0.0, 0.5, 0.99999994, 1.0, inf):
            _check(x, u=u, **par)


@pytest.mark.parametrize("temperature", [1e-44, 1e-38, 7e-38, 1e-30, 1e-20])
def test_sample_of_tiny_temperatures_with_0_on_top(temperature):
    """The largest logit 0 is no sixteenth of an octave from itself at any temperature, and all others are beyond any count."""
    rng = np.random.default_rng(15)
    x = -np.abs(rng.standard_normal((4, 20000)))
    x[0, 7] = x[0, 19000] = 0
    x[1, :4] = -0.0
    x[2] = 0
    x[3] = np.where(rng.random(20000) < 0.5, 0.0, -1e-38)
    for par in (dict(top_p=0.9), dict(top_p=0.5, min_p=0.1), dict(top_k=3, top_p=0.9), dict()):
        _check(x, True, temperature=temperature, u=rng.random(4), **par)


def test_sample_of_the_largest_vocabulary():
    rng = np.random.default_rng(10)
    x = rng.standard_normal((3, 1 << 20)) * 2
    x[2] = 0
    for par in (dict(), dict(top_p=0.9), dict(top_k=50)):
        _check(x, False, u=[0.1, 0.6, 0.9], **par)


@pytest.mark.parametrize("rows,vocab", [(1, 131072), (3, 100003), (40, 70001), (70, 40000), (130, 20011), (300, 12001), (600, 9000), (1100, 4100)])
def test_sample_of_many_rows(rows, vocab):
    """Batches whose rows are cut into sixteen slices down to one."""
    rng = np.random.default_rng([rows, vocab])
    x = rng.standard_normal((rows, vocab)) * rng.choice([0.5, 2.0, 6.0], (rows, 1))
    k = np.where(rng.random(rows) < 0.4, rng.integers(1, 3000, rows), 0)
    p = np.where(rng.random(rows) < 0.5, rng.uniform(0.1, 0.99, rows), 1.0)
    low = np.where(rng.random(rows) < 0.3, rng.uniform(0.001, 0.3, rows), 0.0)
    for f32 in (False, True):
        _check(x, f32, temperature=rng.uniform(0.5, 1.5, rows), top_k=k, top_p=p, min_p=low, u=rng.random(rows))


@pytest.mark.parametrize("f32", [False, True])
def test_sample_of_slices_that_hold_nothing(f32):
    """Long rows with +inf in one part, with only -inf or NaN in others, and with the mass at either end."""
    rng = np.random.default_rng(12)
    n = 140001
    x = rng.standard_normal((6, n)) * 2
    x[0, [70000, 139999]] = np.inf
    x[1, 20000:] = -np.inf
    x[2, :130000] = np.nan
    x[3, : n - 3] = -1e30
    x[4, 9000:100000] = -np.inf
    x[4, 5] = 30.0
    x[5] = -np.inf
    x[5, n - 1] = np.inf
    for par in (dict(), dict(top_k=2), dict(top_k=1500, top_p=0.8), dict(top_p=0.6), dict(top_p=0.999, min_p=0.001), dict(min_p=0.05)):
        _check(x, f32, u=rng.random(6), **par)


@pytest.mark.parametrize("scale,shift,temperature", [(0.1, 1000.0, 0.05), (0.1, -1000.0, 0.05), (1.0, 3e4, 0.5), (1e-3, 0.0, 1e-4), (40.0, 0.0, 0.7)])
def test_sample_far_from_zero(scale, shift, temperature):
    """Large logits over small temperatures: their sixteenths of an octave are beyond what single precision tells apart."""
    rng = np.random.default_rng(13)
    x = shift + scale * rng.standard_normal((4, 50000))
    for par in (dict(top_p=0.9), dict(top_p=0.3), dict(top_k=40, top_p=0.9), dict(top_p=0.95, min_p=0.01), dict()):
        _check(x, True, temperature=temperature, u=rng.random(4), **par)


def test_two_streams_at_once():
    """A product and a draw on each of two streams, every call with a workspace of its own: as one after the other."""
    rng = np.random.default_rng(14)
    w = Weights(2048, 4096, lo=121, hi=123)
    rows, vocab = 24, 30000
    a, _ = _bf16(rng.standard_normal((rows, 4096)))
    x = torch.from_numpy(rng.standard_normal((2, rows, vocab)) * 3).to(torch.bfloat16).cuda()
    u = torch.from_numpy(rng.random(rows).astype(np.float32)).cuda()
    p = torch.full((rows,), 0.9, device="cuda")
    wsize, ssize = max(16, w.w.workspace_size(rows)), api.sample_workspace_size(rows, vocab)

    def both(st, i):
        out = torch.empty(rows, 2048, dtype=torch.float32, device="cuda")
        tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
        ws, ws2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (wsize, ssize))
        torch.cuda.synchronize()
        yield
        for _ in range(20):
            w.w.product(a.data_ptr(), 4096, rows, out.data_ptr(), 2048, out_f32=True, ws=ws.data_ptr(), ws_bytes=wsize, stream=st)
            api.sample(x[i].data_ptr(), rows, vocab, vocab, u.data_ptr(), tokens.data_ptr(), top_p=p.data_ptr(), ws=ws2.data_ptr(),
                       ws_bytes=ssize, stream=st)
            yield
        torch.cuda.synchronize()
        yield out, tokens

    alone = [list(both(_stream(), i))[-1] for i in (0, 1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    together = list(zip(*(both(s.cuda_stream, i) for i, s in enumerate(streams))))[-1]
    for (o, t), (o2, t2) in zip(alone, together):
        assert torch.equal(o, o2) and torch.equal(t, t2)


def test_sample_is_the_same_every_time_and_in_every_batch():
    rng = np.random.default_rng(11)
    x = rng.standard_normal((40, 30000)) * 2
    par = dict(temperature=0.9, top_p=np.where(np.arange(40) % 2, 0.9, 1.0), u=rng.random(40))
    got, lp, _ = _sample(x, False, **par)
    for _ in range(3):
        again, lp2, _ = _sample(x, False, **par)
        assert np.array_equal(got, again) and np.array_equal(lp, lp2)
    for r in (0, 17, 39):
        one, lp1, _ = _sample(x[r:r + 1], False, temperature=0.9, top_p=par["top_p"][r], u=par["u"][r])
        assert one[0] == got[r] and lp1[0] == lp[r]


# -- together -----------------------------------------------------------------------

class Block:
    """A decoder block of another make than the iteration's: norms on both sides of each part, half of each head
    rotated, 4-bit projections, over the 8-bit cache; with a head and a sampler behind it."""
    D, HQ, HKV, HD, F, VOCAB, ROT = 256, 4, 2, 64, 416, 1003, 32

    def __init__(self):
        from tests.kv_rig import Rig
        rng = np.random.default_rng(21)
        self.rig = Rig(self.HQ, self.HKV, self.HD, {1: 0, 2: 40, 3: 17}, grow=20)
        qw = (self.HQ + 2 * self.HKV) * self.HD
        self.wqkv, self.wo = Weights(qw, self.D, lo=121, hi=123), Weights(self.D, self.HQ * self.HD, lo=121, hi=123)
        self.wgu, self.wd = Weights(2 * self.F, self.D, True, lo=121, hi=123), Weights(self.D, self.F, lo=121, hi=123)
        self.head = Weights(self.VOCAB, self.D, lo=121, hi=123)
        self.gains = [_bf16(1 + 0.1 * rng.standard_normal(self.D)) for _ in range(5)]
        self.rope = api.Rope(self.ROT, 10000.0, scaling="linear", factor=2.0)


def test_a_block_of_them():
    """Each step against its model, given what the step before left on the GPU; then the whole captured into a graph and
    replayed between eager work: the same bits."""
    B = Block
    b = Block()
    rig = b.rig
    batch = api.Batch(20, 1, 0, (2, 3), (40, 17))
    rows, qw = batch.rows, (B.HQ + 2 * B.HKV) * B.HD
    plan = rig.begin(batch)
    rng = np.random.default_rng(22)
    x, xv = _bf16(rng.standard_normal((rows, B.D)))
    u = torch.from_numpy(rng.random(rows).astype(np.float32)).cuda()
    temp = torch.full((rows,), 0.8, device="cuda")
    top_p = torch.full((rows,), 0.9, device="cuda")
    new = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")
    y, qkv, att, o, r1, y1, act, down, r2, y2 = (new(rows, w) for w in (B.D, qw, B.HQ * B.HD, B.D, B.D, B.D, B.F, B.D, B.D, B.D))
    qk = new(rows, qw)
    logits, tokens, logprob = new(rows, B.VOCAB, dtype=torch.float32), new(rows, dtype=torch.int32), new(rows, dtype=torch.float32)
    size = max([w.w.workspace_size(rows) for w in (b.wqkv, b.wo, b.wgu, b.wd, b.head)] + [api.sample_workspace_size(rows, B.VOCAB), 16])
    ws = new(size, dtype=torch.uint8)
    g = [t.data_ptr() for t, _ in b.gains]

    def step(st):
        w = dict(ws=ws.data_ptr(), ws_bytes=size, stream=st)
        api.residual_norm(rows, B.D, x.data_ptr(), 0, 0, g[0], y.data_ptr(), stream=st)
        b.wqkv.w.product(y.data_ptr(), B.D, rows, qkv.data_ptr(), qw, **w)
        qk.copy_(qkv)
        k = qk.data_ptr() + 2 * B.HQ * B.HD
        plan.rotate(b.rope, qk.data_ptr(), k, qw, qk.data_ptr(), k, qw, st)
        plan.append(0, k, k + 2 * B.HKV * B.HD, qw, st)
        plan.attend(0, qk.data_ptr(), qw, att.data_ptr(), st)
        b.wo.w.product(att.data_ptr(), B.HQ * B.HD, rows, o.data_ptr(), B.D, **w)
        api.residual_norm(rows, B.D, x.data_ptr(), o.data_ptr(), r1.data_ptr(), g[2], y1.data_ptr(), post_gain=g[1], stream=st)
        b.wgu.w.product(y1.data_ptr(), B.D, rows, act.data_ptr(), B.F, **w)
        b.wd.w.product(act.data_ptr(), B.F, rows, down.data_ptr(), B.D, **w)
        api.residual_norm(rows, B.D, r1.data_ptr(), down.data_ptr(), r2.data_ptr(), g[4], y2.data_ptr(), post_gain=g[3], stream=st)
        b.head.w.product(y2.data_ptr(), B.D, rows, logits.data_ptr(), B.VOCAB, out_f32=True, **w)
        api.sample(logits.data_ptr(), rows, B.VOCAB, B.VOCAB, u.data_ptr(), tokens.data_ptr(), logits_f32=True,
                   temperature=temp.data_ptr(), top_p=top_p.data_ptr(), logprob=logprob.data_ptr(), **w)

    step(_stream())
    torch.cuda.synchronize()
    gv = [v for _, v in b.gains]
    _, _, want, bd = O.norm(xv, None, gv[0])
    _within(_f64(y), want, bd, "bf16")
    _within(_f64(qkv), *O.product(_f64(y), b.wqkv.values), "bf16")
    pos = list(range(20)) + [40, 17]
    heads = _f64(qkv).reshape(rows, -1, B.HD)
    want, bd = O.rotate(heads[:, :B.HQ + B.HKV], pos, O.frequencies(B.ROT, 10000.0, "linear", 2.0))
    turned = _f64(qk).reshape(rows, -1, B.HD)
    _within(turned[:, :B.HQ + B.HKV], want, bd, "bf16")
    rig.model_append(0, batch, turned[:, B.HQ:B.HQ + B.HKV], turned[:, B.HQ + B.HKV:])
    rig.check_cache(0, "after the append")
    want, bd = rig.model_attend(0, batch, turned[:, :B.HQ])
    from tests import kv_oracle
    kv_oracle.check_rows(rig.float_rows(att), want, bd)
    _within(_f64(o), *O.product(_f64(att), b.wo.values), "bf16")
    new_r, nb, want, bd = O.norm(xv, _f64(o), gv[2], gv[1])
    _within(_f64(r1), new_r, nb, "bf16")
    _within(_f64(y1), want, bd, "bf16")
    _within(_f64(act), *O.product(_f64(y1), b.wgu.values, True), "bf16")
    _within(_f64(down), *O.product(_f64(act), b.wd.values), "bf16")
    new_r, nb, want, bd = O.norm(_f64(r1), _f64(down), gv[4], gv[3])
    _within(_f64(r2), new_r, nb, "bf16")
    _within(_f64(y2), want, bd, "bf16")
    _within(_f64(logits), *O.product(_f64(y2), b.head.values), "f32")
    lv = _f64(logits)
    for r in range(rows):
        t, lp = O.sample(lv[r], temperature=float(np.float32(0.8)), top_p=float(np.float32(0.9)), u=float(u[r]))
        assert tokens[r].item() == t
        assert abs(logprob[r].item() - lp) <= 2.0**-24 * abs(lp) + 2.0**-40

    outs = (y, qkv, qk, att, o, r1, y1, act, down, r2, y2, logits, tokens, logprob)
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(3):
        for t in outs:
            t.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(outs, want):
            assert torch.equal(t, w)
        step(_stream())
        torch.cuda.synchronize()
        for t, w in zip(outs, want):
            assert torch.equal(t, w)
