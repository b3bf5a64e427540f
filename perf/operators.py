"""Performance cases of the KV-cache operators: the append that quantises K/V
rows into a paged cache held in 8 bits, and attention over the paged cache
(8 bits or bf16), causal, with an optional sliding window and sink tokens.

One pass is what a server's iteration does with them for its batch (C prompt
rows of one or several prompts behind cached prefixes, B single-token
decodes): hand the batch over, then per layer append the rows' K/V and, but
for the append-only cases, attend.  Head layouts are this repository's own:
the 8B-shaped layer (32 / 8 heads of 128) and the Tiny model (4 / 4 of 64).

The definition:
  * the 8-bit cache holds, per block of 16 tokens and kv head, e4m3 codes and
    one power-of-two scale 2^e.  Appending tokens t0 .. t0 + n - 1 of a block
    takes e = the least integer >= -100 with max |x| <= 448 2^e over the new
    finite values, or the block's present e where that is larger and t0 > 0;
    codes are x 2^-e rounded to nearest even, and the tokens before t0 are
    rounded again to the new scale;
  * row at position p sees key t if t <= p and, with a window W > 0, t > p - W
    or t < sinks; out = softmax(q k / sqrt(hd)) v, heads in groups.
"""
import math

import numpy as np
import torch

own = False

HEADS = {"8b": dict(hq=32, hkv=8, hd=128, max_pos=32768), "tiny": dict(hq=4, hkv=4, hd=64, max_pos=4096)}
MODEL = {"8b": dict(d=4096, f=14336, theta=500000.0), "tiny": dict(d=256, f=704, theta=10000.0)}
PROMPT, DECODE = 1, 100     # sequence ids: prompts PROMPT, PROMPT + 1, ..., decodes DECODE, ...
MIN_EXP = -100


def _case(name, op="attend", shape="8b", cache="e4m3", layers=1, chunk=0, prefix=0, prompts=1, decodes=0, ctx="none",
          window=0, sinks=0):
    """op: append alone, or append and attend; chunk: prompt rows in all, of `prompts` prompts; prefix: cached
    tokens of the first prompt; ctx: distribution of the decodes' cached tokens."""
    return dict(name=name, op=op, shape=shape, cache=cache, layers=layers, chunk=chunk, prefix=prefix, prompts=prompts,
                decodes=decodes, ctx=ctx, window=window, sinks=sinks)


def listed():
    return [
        # The smallest call: one decode of the Tiny model over the 8-bit cache; launches and latency count.
        _case("tiny_b1_e4m3", shape="tiny", decodes=1, ctx="u64_256"),
        # A Tiny chunk beside decodes under a window that ends inside a tile.
        _case("tiny_c128_b4_w96_bf16", shape="tiny", cache="bf16", chunk=128, prefix=128, decodes=4, ctx="u64_256",
              window=96, sinks=4),
        # One user's decode through four layers.
        _case("decode_b1_stack4_e4m3", layers=4, decodes=1, ctx="chat"),
        # A chat server's decode batch with no prompt waiting.
        _case("decode_b64_e4m3", decodes=64, ctx="chat"),
        # The largest decode batch of a chat burst.
        _case("decode_b256_e4m3", decodes=256, ctx="chat"),
        # Longer decodes of a model with windowed layers over the bf16 cache.
        _case("decode_b32_w1024_bf16", cache="bf16", decodes=32, ctx="u1024_10240", window=1024, sinks=16),
        # One token for each of 256 blocks that are partly filled: every scale may grow.
        _case("append_b256_e4m3", op="append", decodes=256, ctx="chat"),
        # A whole chunk's K/V taken into the cache, from the middle of a block on.
        _case("append_c4096_e4m3", op="append", chunk=4096, prefix=1000),
        # A short ragged chunk, no multiple of anything, beside a few decodes.
        _case("ragged_c77_p50_b5_e4m3", chunk=77, prefix=50, decodes=5, ctx="chat"),
        # Several prompts in one iteration of a model with windowed layers.
        _case("batched4_c1500_b16_w512_bf16", cache="bf16", chunk=1500, prefix=2000, prompts=4, decodes=16, ctx="chat",
              window=512, sinks=64),
        # The last chunk of a 32 K prompt beside long decodes, windowed.
        _case("long_c4096_b8_w4096_e4m3", chunk=4096, prefix=28672, decodes=8, ctx="u16384_32768", window=4096, sinks=4),
        # The largest: the same over the whole context.
        _case("long_c4096_b8_e4m3", chunk=4096, prefix=28672, decodes=8, ctx="u16384_32768"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tiny", "decode", "decode", "decode_window", "append", "chunk", "chunk_window", "long"])
    window, sinks = _log_int(rng, 1, 8192), rng.choice([0, 1, 4, rng.randint(0, 200)])
    cache = rng.choice(["e4m3", "e4m3", "bf16"])
    if kind == "tiny":
        windowed = cache == "bf16" or rng.random() < 0.5
        c = _case("", shape="tiny", cache=cache, layers=rng.randint(1, 3), chunk=rng.choice([0, _log_int(rng, 1, 512)]),
                  prefix=rng.randint(0, 512), decodes=rng.randint(1, 8), ctx="u64_256",
                  window=_log_int(rng, 1, 300) if windowed else 0, sinks=rng.randint(0, 20) if windowed else 0)
    elif kind == "decode":
        c = _case("", layers=rng.randint(1, 2), decodes=_log_int(rng, 1, 256), ctx=rng.choice(["chat", "u512_2048", "u1024_10240"]))
    elif kind == "decode_window":
        c = _case("", cache=cache, decodes=_log_int(rng, 1, 256), ctx=rng.choice(["chat", "u512_2048", "u1024_10240"]),
                  window=window, sinks=sinks)
    elif kind == "append":
        c = _case("", op="append", chunk=rng.choice([0, _log_int(rng, 1, 4096)]), prefix=rng.randint(0, 8192),
                  decodes=_log_int(rng, 1, 256), ctx="chat")
    elif kind == "chunk":
        c = _case("", chunk=_log_int(rng, 16, 2048), prefix=rng.choice([0, _log_int(rng, 16, 8192)]),
                  prompts=rng.choice([1, 1, rng.randint(2, 8)]), decodes=rng.randint(0, 32), ctx="u512_2048")
    elif kind == "chunk_window":
        c = _case("", cache=cache, chunk=_log_int(rng, 16, 2048), prefix=rng.choice([0, _log_int(rng, 16, 8192)]),
                  prompts=rng.choice([1, 1, rng.randint(2, 8)]), decodes=rng.randint(0, 32), ctx="u512_2048",
                  window=window, sinks=sinks)
    else:
        c = _case("", chunk=_log_int(rng, 512, 4096), prefix=rng.randint(4096, 28600), decodes=rng.randint(0, 7),
                  ctx="u16384_32768", window=rng.choice([0, window]), sinks=0)
        c["sinks"] = sinks if c["window"] else 0
    del c["name"]
    return c


def _contexts(case):
    """Cached tokens of each decode: fixed by the case."""
    n = case["decodes"]
    rng = np.random.default_rng([2, n])
    if n == 0:
        return []
    if case["ctx"] == "chat":  # log-normal, median 700, sigma 0.8, cap 8192
        v = np.clip(np.rint(700 * np.exp(0.8 * rng.standard_normal(n))), 1, 8192)
    else:
        lo, hi = (int(s) for s in case["ctx"][1:].split("_"))
        v = rng.integers(lo, hi + 1, size=n)
    return [min(int(x), HEADS[case["shape"]]["max_pos"] - 1) for x in v]


def _prompts(case):
    """(prefix, rows) of each prompt: the rows split unevenly, the first prompt behind its cached prefix."""
    c, n = case["chunk"], min(case["prompts"], case["chunk"])
    if n <= 1:
        return [(case["prefix"], c)] if c else []
    share = np.random.default_rng([7, c, n]).uniform(0.5, 1.5, size=n)
    cut = [0] + [int(x) for x in np.rint(np.cumsum(share) / share.sum() * c)]
    for i in range(1, n + 1):  # every prompt has a row
        cut[i] = min(max(cut[i], cut[i - 1] + 1), c - (n - i))
    return [(case["prefix"] if i == 0 else 0, cut[i + 1] - cut[i]) for i in range(n)]


def _sequences(case):
    """[(id, first new position, new rows)] in row order: prompts, then decodes."""
    seqs = [(PROMPT + i, p, c) for i, (p, c) in enumerate(_prompts(case))]
    return seqs + [(DECODE + i, n, 1) for i, n in enumerate(_contexts(case))]


def _reservations(seqs):
    """The reservations (id, positions) that grow all sequences together, a block at a time: pages of a sequence
    are scattered through the pool, as a server leaves them."""
    todo = {sid: at + new for sid, at, new in seqs}
    k = 1
    while todo:
        for sid in list(todo):
            yield sid, min(todo[sid], 16 * k)
            if 16 * k >= todo[sid]:
                del todo[sid]
        k += 1


def _tables(seqs):
    """Block table of each sequence: a reservation takes the lowest free block."""
    tables = {sid: [] for sid, _, _ in seqs}
    for blk, (sid, _) in enumerate(_reservations(seqs)):
        tables[sid].append(blk)
    return tables


def _inputs(case, seed):
    """Rows and cached K/V, made on the GPU from the seed: q, k, v rows as a fused projection leaves them (a few
    channels larger than the rest, as keys have them), and pools that hold cached tokens in every block."""
    h, n = HEADS[case["shape"]], case["layers"]
    hq, hkv, hd = h["hq"], h["hkv"], h["hd"]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen)

    seqs = _sequences(case)
    blocks = sum(-(-(at + new) // 16) for _, at, new in seqs)
    channel = torch.exp(0.4 * normal(1, 1, hkv, 1, hd))
    rows = case["chunk"] + case["decodes"]
    qkv = normal(n, rows, hq + 2 * hkv, hd)
    qkv[:, :, hq:hq + hkv] *= channel[0, :, :, 0]
    qkv = qkv.reshape(n, rows, -1).to(torch.bfloat16)
    pools = []
    for scaled in (True, False):
        x = normal(n, blocks, hkv, 16, hd)
        if scaled:
            x *= channel
        if case["cache"] == "e4m3":
            e = torch.ceil(torch.log2(x.abs().amax((3, 4)) / 448)).clamp_(min=MIN_EXP)
            x = (x * torch.exp2(-e)[..., None, None]).clamp_(-448, 448).to(torch.float8_e4m3fn)
            wide, scale = 64, torch.exp2(e).contiguous()
        else:
            x, wide, scale = x.to(torch.bfloat16), 32, None
        if scaled:   # K pages: slabs of dims, token-major
            x = x.reshape(n, blocks, hkv, 16, hd // wide, wide).transpose(3, 4).contiguous()
        else:        # V pages: dim-major
            x = x.transpose(3, 4).contiguous()
        pools.append((x, scale))
    return dict(h, n=n, rows=rows, blocks=blocks, seqs=seqs, qkv=qkv, k=pools[0][0], ks=pools[0][1], v=pools[1][0],
                vs=pools[1][1])


def _groups(seqs, tables, is_prompt):
    """Index tensors of the prompts, or of the decodes, padded to the longest: rows [s][r], positions, block tables."""
    row, picked, at_row = [], [], 0
    for sid, at, new in seqs:
        if (sid < DECODE) == is_prompt:
            picked.append((sid, at, new, at_row))
        at_row += new
    if not picked:
        return None
    most, blocks = max(p[2] for p in picked), max(len(tables[p[0]]) for p in picked)
    row = np.zeros((len(picked), most), np.int64)
    pos = np.zeros((len(picked), most), np.int64)
    real = np.zeros((len(picked), most), bool)
    table = np.zeros((len(picked), blocks), np.int64)
    for i, (sid, at, new, r) in enumerate(picked):
        row[i, :new], pos[i, :new], real[i, :new] = np.arange(r, r + new), np.arange(at, at + new), True
        table[i, :len(tables[sid])] = tables[sid]
    return {k: torch.from_numpy(a).cuda() for k, a in (("row", row), ("pos", pos), ("real", real), ("table", table))}


def prepare(case, seed):
    s = _inputs(case, seed)
    seqs, tables = s["seqs"], _tables(s["seqs"])
    s.update(op=case["op"], cache=case["cache"], window=case["window"], sinks=case["sinks"])
    s["out"] = torch.empty((s["n"], s["rows"], s["hq"] * s["hd"]), dtype=torch.bfloat16, device="cuda")
    if own:
        from paper_2609_07883_amd import api
        m = MODEL[case["shape"]]
        ctx = api.Context(s["n"], m["d"], s["hq"], s["hkv"], s["hd"], m["f"], 1e-5, m["theta"], s["max_pos"])
        if case["cache"] == "e4m3":
            ctx.kv_init_8bit(s["k"].data_ptr(), s["v"].data_ptr(), s["ks"].data_ptr(), s["vs"].data_ptr(), s["blocks"])
        else:
            ctx.kv_init(s["k"].data_ptr(), s["v"].data_ptr(), s["blocks"])
        ctx.set_window(case["window"], case["sinks"])
        for sid, _, _ in seqs:
            ctx.seq_create(sid)
        for sid, n in _reservations(seqs):
            ctx.seq_reserve(sid, n)
        s["ctx"] = ctx
        s["batch"] = api.Batch.batched([q for q in seqs if q[0] < DECODE], [q[0] for q in seqs if q[0] >= DECODE],
                                       [q[1] for q in seqs if q[0] >= DECODE])
        s["ws"] = torch.empty(ctx.attn_workspace_size(case["chunk"], case["decodes"]), dtype=torch.uint8, device="cuda")
        s["stream"] = torch.cuda.current_stream().cuda_stream
        return s
    # the blocks that the batch writes: their ids, the row of each token (-1: none) and the first new token
    ids, rows, first, r = [], [], [], 0
    for sid, at, new in seqs:
        for b in range(at // 16, (at + new - 1) // 16 + 1):
            t = np.arange(16 * b, 16 * b + 16)
            ids.append(tables[sid][b])
            rows.append(np.where((t >= at) & (t < at + new), r + t - at, -1))
            first.append(max(at - 16 * b, 0))
        r += new
    s["w_blk"], s["w_row"], s["w_first"] = (torch.from_numpy(np.asarray(a, np.int64)).cuda() for a in (ids, np.stack(rows), first))
    s["prompts"], s["decodes"] = _groups(seqs, tables, True), _groups(seqs, tables, False)
    return s


def _append(s, pool, scale, x, is_k):
    """The plain append: x [n][rows][hkv][hd] float32."""
    blk, row, first = s["w_blk"], s["w_row"], s["w_first"]
    token = torch.arange(16, device="cuda")
    new = (row >= 0)[None, :, None, :, None]
    old = (token < first[:, None])[None, :, None, :, None]
    rows = x[:, row.clamp(min=0)].transpose(2, 3)                                # [n][blocks][hkv][16][hd]
    n, nb, hkv, _, hd = rows.shape
    held = pool[:, blk].transpose(3, 4).reshape(n, nb, hkv, 16, hd).float()
    if scale is None:
        put = torch.where(new, rows, held)
    else:
        amax = torch.where(new & torch.isfinite(rows), rows.abs(), 0.0).amax((3, 4))
        mantissa, e = torch.frexp(amax)                                          # amax = mantissa 2^e, mantissa in [1/2, 1)
        e = torch.where(mantissa > 448 / 512, e - 8, e - 9).clamp(min=MIN_EXP)
        e = torch.where(amax > 0, e, MIN_EXP)
        e_old = torch.frexp(scale[:, blk])[1] - 1
        e = torch.where((first > 0)[None, :, None], torch.maximum(e, e_old), e)
        rows = torch.where(torch.isfinite(rows), rows, math.nan)
        put = torch.where(new, rows * torch.exp2(-e.float())[..., None, None], held)
        put = torch.where(old, held * torch.exp2((e_old - e).float())[..., None, None], put)
        scale[:, blk] = torch.exp2(e.float())
    put = put.to(pool.dtype)
    if is_k:
        put = put.reshape(n, nb, hkv, 16, hd // pool.shape[-1], pool.shape[-1])
    pool[:, blk] = put.transpose(3, 4)


def _attend(s, g):
    """The plain attention of a group of sequences padded to the longest, in float32."""
    if g is None:
        return
    n, hq, hkv, hd = s["n"], s["hq"], s["hkv"], s["hd"]
    ns, most = g["row"].shape
    keys = 16 * g["table"].shape[1]

    def gather(pool, scale):
        x = pool[:, g["table"]].float()                                          # [n][s][blocks][hkv][..]
        if scale is not None:
            x *= scale[:, g["table"]].reshape(x.shape[:4] + (1,) * (x.dim() - 4))
        return x

    k = gather(s["k"], s["ks"]).transpose(4, 5).reshape(n, ns, -1, hkv, 16, hd)  # slabs of dims back together
    k = k.transpose(2, 3).reshape(n, ns, hkv, keys, hd)
    v = gather(s["v"], s["vs"]).permute(0, 1, 3, 2, 5, 4).reshape(n, ns, hkv, keys, hd)
    q = s["qkv"][:, g["row"], :hq * hd].float().reshape(n, ns, most, hkv, hq // hkv, hd).permute(0, 1, 3, 4, 2, 5)
    sc = (q.reshape(n, ns, hkv, -1, hd) @ k.transpose(3, 4)).div_(math.sqrt(hd)).reshape(n, ns, hkv, hq // hkv, most, keys)
    t, p = torch.arange(keys, device="cuda")[None, None], g["pos"][:, :, None]
    seen = t <= p
    if s["window"] > 0:
        seen &= (t > p - s["window"]) | (t < s["sinks"])
    sc.masked_fill_(~seen[None, :, None, None], -math.inf)
    sc -= sc.amax(-1, keepdim=True)
    sc.exp_()
    total = sc.sum(-1, keepdim=True)
    o = (sc.reshape(n, ns, hkv, -1, keys) @ v).reshape(n, ns, hkv, hq // hkv, most, hd) / total
    o = o.permute(0, 1, 4, 2, 3, 5).reshape(n, ns, most, hq * hd).to(torch.bfloat16)
    s["out"][:, g["row"][g["real"]]] = o[:, g["real"]]


def run(state):
    s = state
    hq, hkv, hd, n = s["hq"], s["hkv"], s["hd"], s["n"]
    if own:
        ctx, ws, st = s["ctx"], s["ws"], s["stream"]
        width = (hq + 2 * hkv) * hd
        plan = ctx.attn_begin(s["batch"], ws.data_ptr(), ws.numel(), st)
        q, out = s["qkv"].data_ptr(), s["out"].data_ptr()
        for layer in range(n):
            plan.append(layer, q + 2 * hq * hd, q + 2 * (hq + hkv) * hd, width, st)
            if s["op"] == "attend":
                plan.attend(layer, q, width, out, st)
            q, out = q + 2 * s["rows"] * width, out + 2 * s["rows"] * hq * hd
    else:
        x = s["qkv"].reshape(n, s["rows"], hq + 2 * hkv, hd)
        _append(s, s["k"], s["ks"], x[:, :, hq:hq + hkv].float(), True)
        _append(s, s["v"], s["vs"], x[:, :, hq + hkv:].float(), False)
        if s["op"] == "attend":
            _attend(s, s["prompts"])
            _attend(s, s["decodes"])
    r = {"k": s["k"], "v": s["v"]}
    if s["ks"] is not None:
        r.update(k_scale=s["ks"], v_scale=s["vs"])
    if s["op"] == "attend":
        r["out"] = s["out"]
    return r


def _visible(at, new, window, sinks):
    """(distinct keys, pairs) that rows at .. at + new - 1 see."""
    p = np.arange(at, at + new, dtype=np.int64)
    lo = np.maximum(p - window + 1, 0) if window > 0 else np.zeros_like(p)
    pairs = int((p - lo + 1 + np.minimum(lo, sinks)).sum())
    return int(at + new - lo[0] + min(lo[0], sinks)), pairs


def work(case):
    """The rows' q, k, v read and their outputs written once, the new tokens' codes written (beside older tokens of
    their blocks, which a new scale changes), the cached tokens that some row sees read once; the products."""
    h, n = HEADS[case["shape"]], case["layers"]
    hq, hkv, hd = h["hq"], h["hkv"], h["hd"]
    one = 1 if case["cache"] == "e4m3" else 2
    rows = case["chunk"] + case["decodes"]
    row = 2 * hkv * hd
    nbytes, flops = rows * row * (2 + one), 0
    for _, at, new in _sequences(case):
        if case["cache"] == "e4m3":
            nbytes += 8 * hkv * ((at + new - 1) // 16 - at // 16 + 1) + row * (at % 16)
        if case["op"] == "attend":
            keys, pairs = _visible(at, new, case["window"], case["sinks"])
            nbytes += max(keys - new, 0) * row * one + (max(keys - new, 0) // 16 * 8 * hkv if one == 1 else 0)
            flops += 4 * hq * hd * pairs
    if case["op"] == "attend":
        nbytes += 2 * 2 * rows * hq * hd
    return {"bytes": n * nbytes, "flops": n * flops}


def _e4m3(x):
    """float64 values of magnitude <= 448 to the nearest e4m3 value, ties to even: steps of 2^(exponent - 3), at least 2^-9."""
    step = torch.exp2((torch.frexp(x)[1].double() - 4).clamp(min=-9))
    return torch.round(x / step) * step


def exact(case, seed):
    """The definition in float64, sequence by sequence and head by head."""
    s = _inputs(case, seed)
    hq, hkv, hd, n = s["hq"], s["hkv"], s["hd"], s["n"]
    group, tables = hq // hkv, _tables(s["seqs"])
    eight = case["cache"] == "e4m3"
    x = s["qkv"].reshape(n, s["rows"], hq + 2 * hkv, hd)
    # pages as [n][block][hkv][16][hd]
    k = s["k"].double().permute(0, 1, 2, 4, 3, 5).reshape(n, s["blocks"], hkv, 16, hd)
    v = s["v"].double().transpose(3, 4).contiguous()
    scales = [t.double() for t in (s["ks"], s["vs"])] if eight else [None, None]
    # each row's block and token; first rows of a block, whole blocks at once by their number of new tokens
    jobs, r = {}, 0
    for sid, at, new in s["seqs"]:
        p = at
        while p < at + new:
            m = min(16 - p % 16, at + new - p)
            jobs.setdefault((p % 16, m), []).append((tables[sid][p // 16], r + p - at))
            p += m
        r += new
    for (t0, m), todo in jobs.items():
        blk = torch.tensor([b for b, _ in todo], device="cuda")
        row = torch.tensor([q for _, q in todo], device="cuda")[:, None] + torch.arange(m, device="cuda")
        for page, scale, lo in ((k, scales[0], hq), (v, scales[1], hq + hkv)):
            fresh = x[:, row][..., lo:lo + hkv, :].double().transpose(2, 3)      # [n][jobs][hkv][m][hd]
            if not eight:
                page[:, blk, :, t0:t0 + m] = fresh
                continue
            e = torch.ceil(torch.log2(fresh.abs().amax((3, 4)) / 448)).clamp(min=MIN_EXP)
            if t0 > 0:
                e = torch.maximum(e, torch.log2(scale[:, blk]))
                page[:, blk, :, :t0] = _e4m3(page[:, blk][:, :, :, :t0] * (scale[:, blk] / torch.exp2(e))[..., None, None])
            page[:, blk, :, t0:t0 + m] = _e4m3(fresh / torch.exp2(e)[..., None, None])
            scale[:, blk] = torch.exp2(e)
    wide = s["k"].shape[-1]
    r = {"k": k.reshape(n, s["blocks"], hkv, 16, hd // wide, wide).transpose(3, 4), "v": v.transpose(3, 4)}
    if eight:
        r.update(k_scale=scales[0], v_scale=scales[1])
    if case["op"] != "attend":
        return r
    out = torch.zeros((n, s["rows"], hq, hd), dtype=torch.float64, device="cuda")
    for layer in range(n):
        row = 0
        for sid, at, new in s["seqs"]:
            ids = torch.tensor(tables[sid], device="cuda")
            p = torch.arange(at, at + new, device="cuda")[:, None]
            t = torch.arange(at + new, device="cuda")[None]
            hidden = t > p
            if case["window"] > 0:
                hidden |= (t <= p - case["window"]) & (t >= case["sinks"])
            for g in range(hkv):
                kk, vv = k[layer, ids, g], v[layer, ids, g]
                if eight:
                    kk, vv = kk * scales[0][layer, ids, g, None, None], vv * scales[1][layer, ids, g, None, None]
                kk, vv = kk.reshape(-1, hd)[:at + new], vv.reshape(-1, hd)[:at + new]
                q = x[layer, row:row + new, g * group:(g + 1) * group].double().transpose(0, 1)
                sc = torch.matmul(q, kk.T) / math.sqrt(hd)
                sc.masked_fill_(hidden, -math.inf)
                out[layer, row:row + new, g * group:(g + 1) * group] = torch.matmul(torch.softmax(sc, -1), vv).transpose(0, 1)
            row += new
    r["out"] = out.reshape(n, s["rows"], hq * hd)
    return r
