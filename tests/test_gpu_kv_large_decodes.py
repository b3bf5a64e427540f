"""GPU tests of decode batches whose keys and values exceed the last-level cache (256 MB over all layers), where the
cache kernels load pages as data that is read once."""
import pytest

from paper_2609_07883_amd import api
from paper_2609_07883_amd.synth import ModelShape
from tests import kv_oracle as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LIMIT = 256 << 20
WINDOW, SINKS = 30000, 3     # hides nothing from the decodes: bf16 layers need a window to use these kernels


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class _Server:
    """A context over the first `layers` layers of pools, with its sequences."""

    def __init__(self, shape, cache, pools, blocks, lens, layers):
        hq, hkv, hd = shape
        self.shape, self.cache, self.pools = shape, cache, pools
        self.ctx = c = api.Context(layers, 256, hq, hkv, hd, 256, 1e-5, 10000.0, 32768)
        if cache == "e4m3":
            c.kv_init_8bit(*(p.data_ptr() for p in pools), blocks)
        else:
            c.kv_init(*(p.data_ptr() for p in pools[:2]), blocks)
            c.set_window(WINDOW, SINKS)
        for sid, n in lens.items():
            c.seq_create(sid)
            c.seq_reserve(sid, n)

    def layer(self, batch, layer, x):
        """Append and attention of one layer; the outputs."""
        hq, hkv, hd = self.shape
        n = self.ctx.attn_workspace_size(batch.chunk, len(batch.decode_seqs))
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        out = torch.empty((batch.rows, hq * hd), dtype=torch.bfloat16, device="cuda")
        plan = self.ctx.attn_begin(batch, ws.data_ptr(), n)
        p = x.data_ptr()
        plan.append(layer, p + 2 * hq * hd, p + 2 * (hq + hkv) * hd, x.stride(0))
        plan.attend(layer, p, x.stride(0), out.data_ptr())
        torch.cuda.synchronize()
        return out

    def dense(self, layer, sid, n):
        """K and V of a sequence's first n tokens as float64 [n][hkv][hd]."""
        ids = torch.tensor(self.ctx.block_table(sid)[: -(-n // 16)], device="cuda")
        r = []
        for i in range(2):
            y = O.pages(self.pools[i][layer, ids], i == 0)
            if self.cache == "e4m3":
                y = y * self.pools[2 + i][layer, ids].cpu().double().numpy()[..., None, None]
            r.append(y.transpose(0, 2, 1, 3).reshape(-1, *self.shape[1:])[:n])
        return r


# (q heads, kv heads, head dim), (prefix, rows) of a prompt beside the decodes
CASES = [((16, 8, 128), None), ((8, 8, 64), None), ((16, 8, 128), (100, 33)), ((8, 8, 64), (100, 33)), ((16, 8, 128), (24000, 300))]


@pytest.mark.parametrize("shape,prompt", CASES)
@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_decodes_past_the_last_level_cache(cache, shape, prompt):
    """Each layer of a two-layer context, whose decodes exceed the limit together, against the model; its first layer
    bit for bit against a context of that layer alone, whose decodes do not exceed it and whose work is split alike."""
    hq, hkv, hd = shape
    wide = 64 if cache == "e4m3" else 32
    key = 2 * hkv * hd * (1 if cache == "e4m3" else 2)
    n_dec = 64
    mean = int(0.6 * LIMIT / key / n_dec)
    ctxs = [mean - 32 + (17 * i) % 64 for i in range(n_dec)]
    seqs = {10 + i: n for i, n in enumerate(ctxs)}
    keys = sum(n + 1 for n in ctxs)
    assert keys * key < LIMIT < 2 * keys * key and max(ctxs) < WINDOW
    batch = api.Batch(prompt[1] if prompt else 0, 1, prompt[0] if prompt else 0, tuple(seqs), tuple(ctxs))
    lens = {sid: n + 1 for sid, n in seqs.items()}
    if prompt:
        lens[1] = sum(prompt)
        plan = api.attention_plan(ModelShape(1, 256, hq, hkv, hd, 256, max_pos=32768), ctxs, [prompt],
                                  *((WINDOW, SINKS) if cache == "bf16" else (0, 0)), kv=cache)
        assert plan["chunk_two_phase"] == (prompt[0] > 10000)
    blocks = sum(-(-n // 16) for n in lens.values())
    gen = torch.Generator(device="cuda").manual_seed(5)

    def random(*dims):
        return torch.randn(dims, device="cuda", generator=gen)

    if cache == "e4m3":
        pools = [(random(2, blocks, *page) * 32).to(torch.float8_e4m3fn) for page in ((hkv, hd // wide, 16, wide), (hkv, hd, 16))]
        pools += [torch.exp2(torch.randint(-7, -3, (2, blocks, hkv), device="cuda", generator=gen).float()) for _ in range(2)]
    else:
        pools = [random(2, blocks, *page).bfloat16() for page in ((hkv, hd // wide, 16, wide), (hkv, hd, 16))]
    rows = [random(batch.rows, (hq + 2 * hkv) * hd).bfloat16() for _ in range(2)]
    start = [p.clone() for p in pools]

    one = _Server(shape, cache, pools, blocks, lens, 1).layer(batch, 0, rows[0])
    for p, s in zip(pools, start):
        p.copy_(s)
    server = _Server(shape, cache, pools, blocks, lens, 2)
    outs = [server.layer(batch, layer, rows[layer]) for layer in range(2)]
    assert torch.equal(one, outs[0])
    runs = ([(1, *prompt)] if prompt else []) + [(sid, n, 1) for sid, n in seqs.items()]
    for layer in range(2):
        got = outs[layer].cpu().double().numpy().reshape(batch.rows, hq, hd)
        q = rows[layer].cpu().double().numpy().reshape(batch.rows, -1, hd)[:, :hq]
        row = 0
        for i, (sid, at, n) in enumerate(runs):
            if n > 1 or i % 13 == 1:
                pick = sorted({0, n // 2, n - 1})
                want, bound = O.attend(q[[row + r for r in pick]], *server.dense(layer, sid, at + n), [at + r for r in pick], 0, 0)
                O.check_rows(got[[row + r for r in pick]], want, bound, f"layer {layer}, sequence {sid}")
            row += n
