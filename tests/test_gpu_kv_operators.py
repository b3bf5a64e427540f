"""GPU tests of the KV-cache operators against the float64 model: the 8-bit append bit for bit, attention over 8-bit
and windowed caches within a bound derived in tests/kv_oracle.py."""
import numpy as np
import pytest

from paper_2609_07883_amd import api
from tests import kv_oracle as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def Rig(*a, **k):
    from tests.kv_rig import Rig as R
    return R(*a, **k)


def _run(rig, batch, layer=0, q_std=1.0, rows=None, x=None):
    x, q, k, v = rig.put(x) if x is not None else rig.rows(batch.rows, q_std)
    plan = rig.begin(batch)
    rig.append(plan, layer, x)
    out = rig.attend(plan, layer, x)
    rig.model_append(layer, batch, k, v)
    rig.check_cache(layer, "after the append")
    want, bound = rig.model_attend(layer, batch, q, rows)
    got = rig.float_rows(out)
    return O.check_rows(got if rows is None else got[sorted(rows)], want, bound)


# -- the append ---------------------------------------------------------------------

@pytest.mark.parametrize("hd", [64, 128])
def test_append_every_bf16_value(hd):
    """All 65536 bf16 values as K and V, in blocks of like magnitude and in mixed ones."""
    n = 65536 // (2 * hd)
    rig = Rig(2, 2, hd, {1: 0, 2: 0})
    rig.ctx.seq_free(1), rig.ctx.seq_free(2)
    rig.blocks = 2 * n // 16
    rig.attach()
    bits = np.arange(65536, dtype=np.uint16)
    order = np.argsort(bits & 0x7FFF, kind="stable")
    x = np.zeros((2 * n, 6, hd), np.uint16)
    x[:n, 2:4] = bits[order].reshape(n, 2, hd)
    x[:n, 4:6] = bits[order][::-1].reshape(n, 2, hd)
    x[n:, 2:4] = np.random.default_rng(3).permutation(bits & 0x7FFF | (bits & 1) << 15).reshape(n, 2, hd)
    x[n:, 4:6] = bits.reshape(n, 2, hd)
    t = torch.from_numpy(x.reshape(2 * n, -1).view(np.int16)).cuda().view(torch.bfloat16)
    f = torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).double().numpy()
    rig.k, rig.v = (np.zeros((1, rig.blocks, 2, 16, hd)) for _ in range(2))
    rig.ke, rig.ve = (np.zeros((1, rig.blocks, 2)) for _ in range(2))
    rig.upload()
    rig.ctx.seq_create(1)
    batch = api.Batch(2 * n, 1, 0, (), ())
    plan = rig.begin(batch)
    rig.append(plan, 0, t)
    rig.model_append(0, batch, f[:, 2:4], f[:, 4:6])
    rig.check_cache(0)


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 4, 64), (8, 2, 128), (16, 1, 64)])
def test_append_token_by_token(cache, hq, hkv, hd):
    """Sequences that grow by one token, by several and over block borders, each append's rows 2^-12 to 2^12 times the
    last one's: scales grow and stay, older tokens are rounded again; other slots keep their bits."""
    rig = Rig(hq, hkv, hd, {1: 0, 2: 15, 3: 16, 4: 37}, cache, layers=2, window=8, grow=60)
    at = dict(rig.len)
    rng = np.random.default_rng(5)
    for step in range(24):
        grow = {1: 1, 2: 1, 3: int(rng.integers(1, 4)), 4: 1 if step % 5 else 20}
        pre = [(s, at[s], grow[s]) for s in (3, 4) if at[s] + grow[s] < 90]
        dec = [s for s in (1, 2)]
        batch = api.Batch.batched(pre, dec, [at[s] for s in dec])
        x, _, k, v = rig.put(rng.standard_normal((batch.rows, hq + 2 * hkv, hd)) *
                             np.exp2(rng.integers(-12, 13, (batch.rows, 1, 1))))
        plan = rig.begin(batch)
        layer = step % 2
        for l in range(2):
            rig.append(plan, l, x)
            rig.model_append(l, batch, k, v)
        rig.check_cache(layer, f"step {step}")
        for s in [p[0] for p in pre] + dec:
            at[s] += grow[s]


def test_append_extremes():
    """Blocks of zeros, of the smallest and the largest values, with NaN and infinities, alone and after each other."""
    hd = 64
    rig = Rig(2, 1, hd, {s: 0 for s in range(1, 9)}, grow=40)
    big = 3.3895313892515355e38  # the largest finite bf16
    kinds = [np.zeros(hd), np.full(hd, 2.0**-133), np.full(hd, big), np.r_[np.nan, np.inf, -np.inf, np.ones(hd - 3)],
             np.full(hd, np.nan), np.full(hd, -np.inf), np.r_[big, np.full(hd - 1, 2.0**-133)], np.r_[448.0, np.full(hd - 1, -449)]]
    at = {s: 0 for s in range(1, 9)}
    for step in range(20):
        x = np.zeros((8, 4, hd))
        for s in range(8):
            x[s, 2] = kinds[(s + step) % 8]
            x[s, 3] = kinds[(3 * s + 5 * step) % 8]
        batch = api.Batch(0, 0, 0, tuple(at), tuple(at.values()))
        t, _, k, v = rig.put(x)
        plan = rig.begin(batch)
        rig.append(plan, 0, t)
        rig.model_append(0, batch, k, v)
        rig.check_cache(0, f"step {step}")
        at = {s: n + 1 for s, n in at.items()}
    assert torch.isfinite(rig.k_scale[0, rig.ctx.block_table(1)[:2]]).all()


def test_append_again_at_the_same_positions():
    """The same rows twice leave the same cache; other rows at an earlier position overwrite from there on."""
    rig = Rig(4, 2, 64, {1: 20, 2: 3}, grow=30)
    b = api.Batch(13, 1, 20, (2,), (3,))
    for seed in (0, 0, 1):
        x, _, k, v = rig.put(np.random.default_rng(seed).standard_normal((14, 8, 64)))
        for _ in range(2):
            rig.append(rig.begin(b), 0, x)
            rig.model_append(0, b, k, v)
            rig.check_cache(0)
    b = api.Batch(5, 1, 24, (2,), (1,))
    x, _, k, v = rig.put(np.random.default_rng(2).standard_normal((6, 8, 64)) * 40)
    rig.append(rig.begin(b), 0, x)
    rig.model_append(0, b, k, v)
    rig.check_cache(0)


# -- attention ----------------------------------------------------------------------

HEADS = [(4, 4, 64), (2, 2, 128), (8, 4, 64), (8, 4, 128), (8, 2, 64), (8, 2, 128), (16, 2, 64), (8, 1, 128), (16, 1, 64),
         (16, 1, 128)]
WINDOWS = {"e4m3": [(0, 0), (1, 0), (50, 3), (200, 70)], "bf16": [(1, 0), (50, 3), (200, 70)]}


@pytest.mark.parametrize("cache,window,sinks", [(c, *w) for c in WINDOWS for w in WINDOWS[c]])
@pytest.mark.parametrize("hq,hkv,hd", HEADS)
def test_decodes(hq, hkv, hd, cache, window, sinks):
    """Single tokens over contexts from none to many tiles, ends at every kind of border."""
    ctxs = [0, 1, 15, 16, 17, 63, 64, 65, 127, 130, 200, 256, 300, 511, 700]
    seqs = {10 + i: n for i, n in enumerate(ctxs)}
    rig = Rig(hq, hkv, hd, seqs, cache, window=window, sinks=sinks, grow=1)
    _run(rig, api.Batch(0, 0, 0, tuple(seqs), tuple(ctxs)), q_std=2.0)


@pytest.mark.parametrize("cache,window", [("e4m3", 0), ("bf16", 400)])
@pytest.mark.parametrize("hq,hkv,ctxs", [(16, 16, [3 * i % 130 for i in range(150)]), (8, 4, [600 + 3 * i for i in range(64)]),
                                         (8, 4, [30 + i for i in range(63)] + [1900])])
def test_many_decodes(hq, hkv, ctxs, cache, window):
    """More decodes than a launch has runs, decodes of like lengths, one long decode among short ones."""
    seqs = {10 + i: n for i, n in enumerate(ctxs)}
    rig = Rig(hq, hkv, 64, seqs, cache, window=window, grow=1, max_pos=2048)
    _run(rig, api.Batch(0, 0, 0, tuple(seqs), tuple(ctxs)), q_std=2.0)


@pytest.mark.parametrize("cache,window,sinks", [(c, *w) for c in WINDOWS for w in WINDOWS[c]])
@pytest.mark.parametrize("hq,hkv,hd", HEADS)
def test_chunks(hq, hkv, hd, cache, window, sinks):
    """Prompts of one row to several query tiles behind prefixes, beside decodes, in one batch."""
    pre = [(1, 0, 1), (2, 70, 65), (3, 0, 150), (4, 333, 40), (5, 15, 17)]
    seqs = {1: 0, 2: 70, 3: 0, 4: 333, 5: 15, 20: 77, 21: 400}
    rig = Rig(hq, hkv, hd, seqs, cache, window=window, sinks=sinks, grow=150)
    batch = api.Batch.batched(pre, (20, 21), (77, 400))
    rows = set(range(0, batch.rows, 7)) | {0, 1, 64, 65, 66, 215, 216, 217, 255, 256, 272, 273, 274}
    _run(rig, batch, q_std=2.0, rows={r for r in rows if r < batch.rows})


@pytest.mark.parametrize("cache,window,sinks", [("e4m3", 0, 0), ("e4m3", 1000, 5), ("bf16", 1000, 5), ("bf16", 2500, 300),
                                                ("e4m3", 64, 64), ("bf16", 128, 0), ("e4m3", 2**31 - 1, 0)])
def test_long_prefix(cache, window, sinks):
    """A chunk behind a long prefix, query tiles split over work-groups, and long decodes."""
    rig = Rig(8, 2, 128, {1: 5000, 2: 4095, 3: 6001}, cache, window=window, sinks=sinks, grow=200)
    batch = api.Batch(200, 1, 5000, (2, 3), (4095, 6001))
    _run(rig, batch, q_std=2.0, rows={0, 1, 63, 64, 100, 198, 199, 200, 201})


# (q heads, kv heads, chunk, prefix, window, sinks): work items long enough for the two-phase kernel
LONG = [(16, 16, 257, 25001, 0, 0), (32, 16, 140, 20020, 0, 0), (32, 8, 200, 16390, 0, 0), (64, 8, 100, 16401, 0, 0),
        (128, 8, 50, 16383, 0, 0), (16, 16, 4096, 5000, 4000, 3), (32, 16, 2048, 4000, 3001, 70), (64, 16, 1024, 5003, 3500, 0),
        (128, 16, 512, 5000, 3001, 64), (256, 16, 256, 5000, 2100, 1)]


def _long_rig(case, cache, grow=0):
    hq, hkv, C, P, window, sinks = case
    rig = Rig(hq, hkv, 128, {1: P, 2: 700, 3: 5}, cache, window=window, sinks=sinks, grow=C + 1, max_pos=32768)
    from paper_2609_07883_amd.synth import ModelShape
    shape = ModelShape(1, 256, hq, hkv, 128, 256, max_pos=32768)
    plan = api.attention_plan(shape, [700, 5], [(P, C)], window, sinks, kv=cache)
    assert plan["chunk_two_phase"]
    tile = 256 * hkv // hq
    rows = {0, 1, 33, tile - 1, tile, C // 2, C - 2, C - 1, C, C + 1}
    return rig, api.Batch(C, 1, P, (2, 3), (700, 5)), {r for r in rows if 0 <= r < C + 2}


def _with_caches(cases):  # full attention over bf16 pages is the iteration's own kernel
    return [pytest.param(c, t, id=f"hq{c[0]}_hkv{c[1]}_w{c[4]}_{t}") for c in cases for t in ("e4m3", "bf16") if c[4] or t == "e4m3"]


@pytest.mark.parametrize("case,cache", _with_caches(LONG))
def test_long_items(case, cache):
    """The two-phase kernel for every group size, whole and split query tiles, beside decodes."""
    rig, batch, rows = _long_rig(case, cache)
    _run(rig, batch, q_std=2.0, rows=rows)


@pytest.mark.parametrize("case,cache", _with_caches([LONG[2], LONG[7], LONG[9]]))
def test_long_items_with_tokens_that_are_not_finite(case, cache):
    """V values that are not finite, cached and new, in tiles that some rows see whole, some in part and some not at
    all: exactly the rows that see them have them."""
    hq, hkv, C, P, window, sinks = case
    rig, batch, rows = _long_rig(case, cache)
    bt = rig.ctx.block_table(1)
    bad = [P + C // 3 - window, P - 20] if window else [P - 20]
    for i, t in enumerate(bad):
        rig.v[0, bt[t // 16], :, t % 16, 3 + i] = np.nan if cache == "e4m3" else [np.inf, -np.inf][i]
    rig.upload()
    if window:
        rows |= {C // 3 - 3, C // 3 - 2, C // 3 - 1, C // 3, C // 3 + 1}
    x = rig.rng.standard_normal((batch.rows, hq + 2 * hkv, 128))
    x[C // 2, hq + hkv:, 7] = np.nan
    rows |= {C // 2 - 1, C // 2, C // 2 + 1}
    _run(rig, batch, x=x, rows=rows)


def test_large_values_and_far_scores():
    """Scores hundreds apart (the running maximum moves by more than the lazy threshold at every tile)."""
    rig = Rig(4, 2, 128, {1: 600, 2: 700}, "e4m3", window=0, grow=64)
    rig.ke += 6
    rig.upload()
    _run(rig, api.Batch(64, 1, 600, (2,), (700,)), q_std=8.0)


@pytest.mark.parametrize("cache,window", [("e4m3", 0), ("e4m3", 100), ("bf16", 100)])
@pytest.mark.parametrize("bad", ["nan_v", "inf_v", "nan_k", "inf_k"])
def test_not_finite_tokens(cache, window, bad):
    """Tokens whose K or V is not finite: rows that see them have what the definition gives, rows that do not (earlier
    ones, those past the window) have none of it, also inside the same 64-key tile."""
    rig = Rig(8, 2, 64, {1: 200, 2: 150, 3: 230, 4: 400}, cache, window=window, sinks=3 if window else 0, grow=130)
    val = np.nan if bad.startswith("nan") else np.inf
    is_k = bad.endswith("k")
    for sid, toks in ((1, (30, 190)), (3, (200,)), (4, (110, 333))):
        bt = rig.ctx.block_table(sid)
        for i, t in enumerate(toks):
            x = rig.k if is_k else rig.v
            if cache == "e4m3":  # the format has NaN alone
                x[0, bt[t // 16], :, t % 16, 5:9] = np.nan
            else:
                x[0, bt[t // 16], :, t % 16, 5:9] = val if is_k or i == 0 else -val
    rig.upload()
    batch = api.Batch.batched([(1, 200, 130), (2, 150, 100)], (3, 4), (230, 400))
    x = rig.rng.standard_normal((batch.rows, 12, 64))
    sel = (8 + (0 if is_k else 2))
    x[40, sel:sel + 2, 3] = val       # new tokens too: in the middle of the first prompt, and of the second
    x[180, sel, 60] = -val
    _run(rig, batch, x=x)


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_every_score_seen_not_a_number(cache):
    """A tile in which a row sees NaN scores alone, the sequence split over work items: the row is NaN."""
    rig = Rig(4, 1, 64, {1: 3000, 2: 3000}, cache, window=2900, sinks=0, grow=20)
    bt = rig.ctx.block_table(2)
    rig.k[0, bt[1024 // 16:1152 // 16]] = np.nan
    rig.upload()
    _run(rig, api.Batch(20, 1, 3000, (2,), (3000,)))


@pytest.mark.parametrize("cache,window", [("e4m3", 0), ("bf16", 30)])
def test_query_that_is_not_a_number(cache, window):
    """One head of one row's query holds NaN: that head of that row is NaN, every other output is as it was."""
    rig = Rig(8, 2, 128, {1: 100, 2: 60}, cache, window=window, grow=40)
    batch = api.Batch(40, 1, 100, (2,), (60,))
    x = rig.rng.standard_normal((41, 12, 128))
    x[7, 3, 5] = np.nan
    x[40, 6, 0] = np.nan
    _run(rig, batch, x=x)


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_pools_past_32_bits(cache):
    """Blocks whose pages lie more than 2^32 bytes into the pools: the same bits as in a small pool."""
    hq, hkv, hd, page = 8, 8, 128, 16 * 128 * (1 if cache == "e4m3" else 2)
    first = 2**32 // (hkv * page) + 5
    outs = []
    for spare in (0, first):
        blocks = spare + 40
        ctx = api.Context(1, 256, hq, hkv, hd, 256, 1e-5, 10000.0, 1 << 20)
        k = torch.empty(blocks * hkv * page, dtype=torch.uint8, device="cuda")
        v = torch.empty_like(k)
        k[-40 * hkv * page:].fill_(0x7F)
        v[-40 * hkv * page:].fill_(0x7F)
        if cache == "e4m3":
            ks = torch.full((blocks * hkv,), float("nan"), device="cuda")
            vs = torch.full_like(ks, float("nan"))
            ctx.kv_init_8bit(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), blocks)
        else:
            ctx.kv_init(k.data_ptr(), v.data_ptr(), blocks)
        ctx.set_window(200, 3)
        left, sid = spare, 100
        while left > 0:
            ctx.seq_create(sid)
            ctx.seq_reserve(sid, 16 * min(left, 65536))
            left, sid = left - min(left, 65536), sid + 1
        ctx.seq_create(1)
        ctx.seq_create(2)
        gen = torch.Generator(device="cuda").manual_seed(3)
        got = []
        for batch in (api.Batch.batched([(1, 0, 300), (2, 0, 70)]), api.Batch(90, 1, 300, (2,), (70,))):
            x = torch.randn((batch.rows, 3 * hq * hd), device="cuda", generator=gen).bfloat16()
            n = ctx.attn_workspace_size(batch.chunk, len(batch.decode_seqs))
            ws = torch.empty(n, dtype=torch.uint8, device="cuda")
            out = torch.empty((batch.rows, hq * hd), dtype=torch.bfloat16, device="cuda")
            plan = ctx.attn_begin(batch, ws.data_ptr(), n)
            p = x.data_ptr()
            plan.append(0, p + 2 * hq * hd, p + 4 * hq * hd, 3 * hq * hd)
            plan.attend(0, p, 3 * hq * hd, out.data_ptr())
            torch.cuda.synchronize()
            got.append(out.clone())
        got += [k[-40 * hkv * page:].clone(), v[-40 * hkv * page:].clone()]
        outs.append(got)
        assert min(ctx.block_table(1)) >= spare
        del k, v
    assert torch.isfinite(outs[0][0]).all() and torch.isfinite(outs[0][1]).all()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


# -- use ------------------------------------------------------------------------------

@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_layers_strides_and_runs_in_a_row(cache):
    """Three layers, windows on one of them, rows of their own strides, several iterations of one server."""
    rig = Rig(8, 2, 128, {1: 100, 2: 33, 3: 64}, cache, layers=3, window=40, sinks=2, windowed=[0, 1, 0], grow=90)
    at = {1: 100, 2: 33, 3: 64}
    for step in range(4):
        n = [17, 0, 1, 30][step]
        batch = api.Batch(n, 1, at[1], (2, 3), (at[2], at[3]))
        plan = rig.begin(batch)
        for layer in range(3):
            x, q, k, v = rig.rows(batch.rows)
            wide = torch.zeros((batch.rows, x.shape[1] + 8 * layer), dtype=torch.bfloat16, device="cuda")
            wide[:, : x.shape[1]] = x
            rig.append(plan, layer, wide)
            out = rig.attend(plan, layer, wide)
            rig.model_append(layer, batch, k, v)
            rig.check_cache(layer)
            O.check_rows(rig.float_rows(out), *rig.model_attend(layer, batch, q))
        at = {1: at[1] + n, 2: at[2] + 1, 3: at[3] + 1}


def test_rows_behind_the_batch_and_slots_of_others_keep_their_bits():
    rig = Rig(4, 4, 64, {1: 10, 2: 90}, "e4m3", window=16, sinks=1, grow=20)
    batch = api.Batch(9, 1, 10, (2,), (90,))
    x, *_ = rig.rows(batch.rows)
    out = torch.full((batch.rows + 3, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    plan = rig.begin(batch)
    rig.append(plan, 0, x)
    rig.attend(plan, 0, x, out=out)
    torch.cuda.synchronize()
    assert (out[batch.rows:] == 7.0).all() and torch.isfinite(out).all()


def test_graph_replays_with_other_rows():
    """One captured layer, replayed with new rows and between eager work: every replay equals the eager result."""
    rig = Rig(8, 2, 128, {1: 300, 2: 500}, "e4m3", window=128, sinks=4, grow=64)
    batch = api.Batch(50, 1, 300, (2,), (500,))
    plan = rig.begin(batch)
    x, _, k, v = rig.rows(batch.rows)
    out = torch.empty((batch.rows, 1024), dtype=torch.bfloat16, device="cuda")
    rig.append(plan, 0, x)
    rig.model_append(0, batch, k, v)
    rig.attend(plan, 0, x, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            st = torch.cuda.current_stream().cuda_stream
            with pytest.raises(api.SloweaveError):
                rig.begin(batch, st)
            rig.append(plan, 0, x, st)
            rig.attend(plan, 0, x, out, st)
    for i in range(5):
        y, q, k, v = rig.rows(batch.rows)
        x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        rig.model_append(0, batch, k, v)
        rig.check_cache(0, f"replay {i}")
        rig.append(plan, 0, x)
        want = rig.attend(plan, 0, x)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        O.check_rows(rig.float_rows(got), *rig.model_attend(0, batch, q))
        torch.ones(1 << 20, device="cuda").sum().item()


def test_two_plans_on_two_streams():
    rig = Rig(8, 2, 64, {1: 700, 2: 900, 3: 100, 4: 20}, "e4m3", grow=40)
    bs = [api.Batch(33, 1, 700, (3,), (100,)), api.Batch(21, 2, 900, (4,), (20,))]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    xs = [rig.rows(b.rows) for b in bs]
    outs = [torch.empty((b.rows, 512), dtype=torch.bfloat16, device="cuda") for b in bs]
    torch.cuda.synchronize()
    plans = [rig.begin(b, s.cuda_stream) for b, s in zip(bs, streams)]
    for _ in range(3):
        for p, s, x, o in zip(plans, streams, xs, outs):
            rig.append(p, 0, x[0], s.cuda_stream)
            rig.attend(p, 0, x[0], o, s.cuda_stream)
    torch.cuda.synchronize()
    for b, x in zip(bs, xs):
        rig.model_append(0, b, x[2], x[3])
    rig.check_cache(0)
    for b, x, o in zip(bs, xs, outs):
        O.check_rows(rig.float_rows(o), *rig.model_attend(0, b, x[1]))


def test_alignment_refusals():
    rig = Rig(4, 4, 64, {1: 10}, grow=8)
    plan = rig.begin(api.Batch(3, 1, 10, (), ()))
    x = torch.zeros((4, 776), dtype=torch.bfloat16, device="cuda")
    p, out = x.data_ptr(), torch.zeros((4, 264), dtype=torch.bfloat16, device="cuda").data_ptr()
    for args in ((p + 2, p, 768), (p, p + 8, 768), (p, p, 772), (p, p, 248), (0, p, 768), (p, 0, 768), (p, p, 2**31)):
        with pytest.raises(api.SloweaveError) as e:
            plan.append(0, *args)
        assert e.value.code == api.EINVAL
    for args in ((p + 2, 768, out), (p, 772, out), (p, 248, out), (p, 768, out + 8), (p, 768, 0), (0, 768, out)):
        with pytest.raises(api.SloweaveError) as e:
            plan.attend(0, *args)
        assert e.value.code == api.EINVAL


def test_full_bf16_layers_use_the_iterations_kernels():
    """Over bf16 pools without a window the operators give the definition too (the iteration's own attention)."""
    rig = Rig(8, 2, 128, {1: 300, 2: 500}, "bf16", grow=100)
    _run(rig, api.Batch(90, 1, 300, (2,), (500,)), q_std=2.0)


# -- the iteration on an 8-bit or windowed cache --------------------------------------

def _session(**k):
    from paper_2609_07883_amd import synth
    from paper_2609_07883_amd.runtime import Session
    shape = synth.ModelShape(n_layers=2, d_model=256, n_q_heads=8, n_kv_heads=2, head_dim=64, ffn_dim=704, max_pos=4096)
    return Session(shape, num_blocks=120, max_c=200, max_b=4, qk_std=0.16, **k)


def _step(sess, batch, x, entry="run"):
    from paper_2609_07883_amd.runtime import bits_to_tensor
    if entry == "run":
        sess.run(batch, x)
    else:
        sess.x_in[:batch.rows].copy_(bits_to_tensor(x, sess.dev))
        sess.ctx.mixed_iteration_static(batch, sess.x_in.data_ptr(), sess.x_out.data_ptr(), sess.stream())
    return sess.output(batch.rows)


@pytest.mark.parametrize("kv,window,sinks,layers", [("e4m3", 0, 0, None), ("e4m3", 60, 4, None), ("e4m3", 60, 4, [1, 0]),
                                                    ("bf16", 60, 4, [0, 1]), ("bf16", 9, 0, None)])
def test_iteration(kv, window, sinks, layers):
    """The mixed iteration on such a cache: its last layer's attention is the definition's on the layer's own q and the
    cache's values, the cache holds the layer's own k and v, and the rest of the layer follows from it; the entry point
    without a workspace and the one with stage events give the same bits."""
    from paper_2609_07883_amd import synth
    from oracle import layer as OL
    from tests.parity import check
    opts = dict(kv=kv, window=window, sinks=sinks, window_layers=layers)
    sessions = [_session(**opts) for _ in range(3)]
    sessions[2].ctx.set_stage_timing(4)
    at = {1: 0, 2: 0, 3: 0}
    todo = [api.Batch(150, 1, 0, (), ()), api.Batch(33, 2, 0, (1,), (150,)), api.Batch(70, 3, 0, (1, 2), (151, 33)),
            api.Batch.batched([(2, 34, 50), (3, 70, 9)], (1,), (152,)), api.Batch(0, 0, 0, (1, 2, 3), (153, 84, 79))]
    for s in sessions:
        for sid in at:
            s.ctx.seq_create(sid)
    shape = sessions[0].shape
    hq, hkv, hd = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    for i, b in enumerate(todo):
        x = synth.embeddings(b.rows, shape.d_model, seed=1, stream=i)
        outs = [_step(s, b, x, e) for s, e in zip(sessions, ("run", "static", "run"))]
        assert np.array_equal(outs[0], outs[1]) and np.array_equal(outs[0], outs[2]), f"iteration {i}"
        assert np.isfinite(outs[0]).all()
        s = sessions[0]
        args = (b.chunk, len(b.decode_seqs))
        qkv = s.view(api.VIEW_QKV, *args, (hq + 2 * hkv) * hd).reshape(b.rows, -1, hd)
        attn = s.view(api.VIEW_ATTN, *args, hq * hd).reshape(b.rows, hq, hd)
        seq_rows = [(sid, p, c) for sid, p, c in b.prefill_list] + [(sid, c, 1) for sid, c in zip(b.decode_seqs, b.context_lens)]
        row, last = 0, shape.n_layers - 1
        w = (window, sinks) if window and (layers is None or layers[last]) else (0, 0)
        for sid, p, c in seq_rows:
            k, v = s.read_kv(last, sid, np.arange(p + c))
            fresh = qkv[row:row + c, hq:]
            for got, new in ((k[p:], fresh[:, :hkv]), (v[p:], fresh[:, hkv:])):
                if kv == "bf16":
                    assert np.array_equal(got, new)
                else:   # half a step of e4m3 (2^-4 of the value, 2^-10 of the scale), the scale at most amax / 224
                    amax = np.abs(got).max()
                    assert (np.abs(got - new) <= 2.0**-4 * np.abs(new) + 2.0**-10 * 2 * amax / 224).all()
            O.check_rows(attn[row:row + c], *O.attend(qkv[row:row + c, :hq], k, v, np.arange(p, p + c), *w), f"iteration {i}")
            row += c
        from tests.parity import oracle_weights
        lw = oracle_weights(s.layer_bits[last])
        h = s.view(api.VIEW_H, *args, shape.d_model, fp32=True)
        wn = OL.rms_norm(h, lw.g2, shape.rms_eps)
        gu = wn @ lw.wgu.T
        y = h + (OL.silu(gu[:, :shape.ffn_dim]) * gu[:, shape.ffn_dim:]) @ lw.wd.T
        check(outs[0], y, f"iteration {i}", layers=1)
    t = sessions[2].ctx.stage_times()
    assert t["decode_attn"] > 0 and t["qkv_gemm"] > 0


def test_serve_on_an_8bit_windowed_cache():
    """The serving loop on the GPU executor, profiler's table and all, over such a cache."""
    sess = _session(kv="e4m3", window=100, sinks=4)
    ctx = sess.ctx
    table = ctx.build_cost_table([0, 32, 128], [0, 2, 4], prefix_len=64, ctx_lo=16, ctx_hi=128, seed=1, warmup=1, repeats=2,
                                 x_in=sess.x_in.data_ptr(), x_out=sess.x_out.data_ptr(), ws=sess.ws.data_ptr(),
                                 ws_bytes=sess.ws_bytes, stream=sess.stream())
    free = ctx.free_blocks()
    tok, its = api.serve([1, 2, 3], [0, 0, 1000], [150, 40, 77], [5, 9, 3], policy=api.POLICY_SLOWEAVE, tpot_ns=10**9,
                         max_decode=4, c_max=128, table=table, executor=api.EXEC_GPU, ctx=ctx, x_in=sess.x_in.data_ptr(),
                         x_out=sess.x_out.data_ptr(), max_rows=204, ws=sess.ws.data_ptr(), ws_bytes=sess.ws_bytes,
                         stream=sess.stream())
    assert all((t > 0).all() for t in tok) and ctx.free_blocks() == free
    assert int(its["chunk"].sum()) == 150 + 40 + 77
