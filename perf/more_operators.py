"""Performance cases of the operators that stand round the cache operators in a
decoder block other than the iteration's, and behind its last layer:

  * residual_norm: the block's output joins the residual stream, through its own
    norm, a gate and a scale where the model has them, and the next block's
    RMSNorm is taken of the sum;
  * product: rows times weights held in 4 bits with a scale for each group of
    32, as a plain projection or as a gated pair (SiLU(gate) * up);
  * rotate: rotary positions of the batch's query and key rows, either layout,
    part of the head, frequencies scaled for long contexts;
  * sample: the next tokens from logits and given random numbers, with
    temperature, top-k, top-p and min-p for each row.

Sizes are this repository's own: the 8B-shaped layer (d 4096, 32 / 8 heads of
128, f 14336) and the Tiny model (d 256, 4 / 4 heads of 64, f 704); vocabularies,
which it has none of, are generic.

The definitions:
  * residual_norm: r' = r + scale * gate * P(o), P(o) = o or
    o / sqrt(mean(o^2) + eps) * post_gain; y = r' / sqrt(mean(r'^2) + eps) * gain,
    of r' before it is rounded to the residual's type;
  * product: out = a W^T, W[n][k] = code * 2^(scale - 127), codes e2m1 (a sign,
    then 0, 1/2, 1, 3/2, 2, 3, 4, 6), one scale byte for 32 values of a row;
    gated: W holds f gate rows, then f up rows, out = silu(a Wg^T) * (a Wu^T);
  * rotate: at position p, pair i of the first rot values of a head turns by
    p f_i and is multiplied by mscale; pairs are (i, i + rot / 2), or
    (2i, 2i + 1) in the interleaved layout.  f_i = theta^(-2i / rot); linear:
    f_i / s; ntk: theta s^(rot / (rot - 2)) for theta; by_parts:
    f_i ((1 - g) / s + g), g = clamp((L f_i / 2 pi - lo) / (hi - lo), 0, 1);
  * sample: w_t = exp((x_t - max x) / temperature); tokens in the order of their
    logits (ties: the lower index first), the first top_k of them, of those
    the ones with less than top_p of the mass before them, of those the ones with
    w_t >= min_p; then the first token, by index, at which the running sum of
    the kept w exceeds u times their sum.  Temperature 0: the first largest.
"""
import math

import numpy as np
import torch

own = False

MODEL = {"8b": dict(d=4096, hq=32, hkv=8, hd=128, f=14336, theta=500000.0),
         "tiny": dict(d=256, hq=4, hkv=4, hd=64, f=704, theta=10000.0)}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _norm(name, rows, d, resid="bf16", post=False, gate="none", scale=1.0):
    """gate: none, a row of d values for all rows ("channel"), or one for each row ("row")."""
    return dict(name=name, op="residual_norm", rows=rows, d=d, resid=resid, post=post, gate=gate, scale=scale)


def _product(name, m, n, k, gated=False, out="bf16"):
    return dict(name=name, op="product", m=m, n=n, k=k, gated=gated, out=out)


def _rotate(name, shape="8b", chunk=0, prefix=0, prompts=1, decodes=0, far=8192, rot=128, interleaved=False,
            scaling="none", factor=1.0, mscale=1.0):
    """chunk rows of `prompts` prompts, the first behind `prefix` tokens; decodes at positions up to `far`."""
    return dict(name=name, op="rotate", shape=shape, chunk=chunk, prefix=prefix, prompts=prompts, decodes=decodes, far=far,
                rot=rot, interleaved=interleaved, scaling=scaling, factor=factor, mscale=mscale)


def _sample(name, rows, vocab, logits="bf16", kind="mixed", spread=3.0):
    """kind: which filters the rows use; spread: standard deviation of the logits."""
    return dict(name=name, op="sample", rows=rows, vocab=vocab, logits=logits, kind=kind, spread=spread)


def listed():
    return [
        # One user's decode: one row between two blocks; launch and latency.
        _norm("norm_r1_d4096", 1, 4096),
        # A whole chunk beside decodes, in a model with norms on both sides of its blocks and a gate, fp32 stream.
        _norm("norm_r4104_d4096_sandwich", 4104, 4096, resid="f32", post=True, gate="channel"),
        # One user's decode: the output projection of one layer, the smallest of an 8B-shaped layer.
        _product("product_m1_o", 1, 4096, 4096),
        # One user's decode: gate and up, most of a layer's weights.
        _product("product_m1_gateup", 1, 28672, 4096, gated=True),
        # A chat server's decode batch: the down projection.
        _product("product_m32_down", 32, 4096, 14336),
        # The logits of a ragged batch over an odd vocabulary, in fp32 for the sampler.
        _product("product_m23_head", 23, 100003, 4096, out="f32"),
        # A prefill chunk beside decodes: gate and up; the largest.
        _product("product_m2080_gateup", 2080, 28672, 4096, gated=True),
        # One token of the Tiny model.
        _rotate("rotate_tiny_b1", shape="tiny", decodes=1, far=256, rot=64),
        # The last chunk of a long prompt beside long decodes, half of each head, interleaved, scaled.
        _rotate("rotate_c4096_b8_scaled", chunk=4096, prefix=100000, decodes=8, far=120000, rot=64, interleaved=True,
                scaling="by_parts", factor=8.0, mscale=1.2079),
        # One user's next token.
        _sample("sample_b1_v32768", 1, 32768, kind="topk_topp"),
        # A chat burst's decode batch, every row with parameters of its own.
        _sample("sample_b256_v131072", 256, 131072),
        # No filter: the whole odd vocabulary, fp32 logits.
        _sample("sample_b23_v100003_f32", 23, 100003, logits="f32", kind="plain"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["residual_norm", "product", "product", "rotate", "sample", "sample"])
    if op == "residual_norm":
        d = 8 * _log_int(rng, 8, 2048)
        c = _norm("", _log_int(rng, 1, min(8192, (4104 * 4096) // d)), d, resid=rng.choice(["bf16", "f32"]),
                  post=rng.random() < 0.5, gate=rng.choice(["none", "channel", "row"]),
                  scale=rng.choice([1.0, round(rng.uniform(0.1, 2.0), 3)]))
    elif op == "product":
        gated = rng.random() < 0.4
        n, k = rng.choice([(6144, 4096), (4096, 4096), (28672, 4096), (4096, 14336), (256, 704), (768, 256), None, None, None]) or \
            (_log_int(rng, 16, 32768), 32 * _log_int(rng, 2, 448))
        n = 2 * ((n + 1) // 2) if gated else n
        most = min(4096, max(1, (2080 * 28672 * 4096) // (n * k)))
        c = _product("", rng.choice([1, _log_int(rng, 1, min(64, most)), _log_int(rng, 1, most)]), n, k, gated=gated,
                     out=rng.choice(["bf16", "bf16", "f32"]))
    elif op == "rotate":
        shape = rng.choice(["8b", "8b", "tiny"])
        hd = MODEL[shape]["hd"]
        scaling = rng.choice(["none", "linear", "ntk", "by_parts"])
        c = _rotate("", shape=shape, chunk=rng.choice([0, _log_int(rng, 1, 4096)]), prefix=_log_int(rng, 1, 100000),
                    prompts=rng.randint(1, 6), decodes=_log_int(rng, 1, 200) if rng.random() < 0.5 else 8,
                    far=_log_int(rng, 300, 10000), rot=rng.choice([hd, hd, 16 * rng.randint(1, hd // 16)]),
                    interleaved=rng.random() < 0.5, scaling=scaling,
                    factor=1.0 if scaling == "none" else round(rng.uniform(1.0, 16.0), 2),
                    mscale=rng.choice([1.0, round(rng.uniform(1.0, 1.4), 4)]))
    else:
        vocab = _log_int(rng, 1000, 160000)
        c = _sample("", _log_int(rng, 1, min(256, (256 * 131072) // vocab)), vocab, logits=rng.choice(["bf16", "f32"]),
                    kind=rng.choice(["mixed", "mixed", "plain", "topk", "topp", "minp", "topk_topp", "greedy"]),
                    spread=round(rng.uniform(1.0, 5.0), 2))
        if c["logits"] == "f32":
            c["rows"] = min(c["rows"], max(1, (128 * 131072) // vocab))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen)


def _uniform(gen, *shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(generator=gen)


def _norm_inputs(case, seed):
    """A residual stream some layers deep (a few channels far above the rest), a block's output beside it."""
    g, rows, d = _generator(seed), case["rows"], case["d"]
    channel = torch.exp(0.6 * _normal(g, d))
    s = {"resid": (_normal(g, rows, d) * 2 * channel).to(torch.bfloat16 if case["resid"] == "bf16" else torch.float32),
         "block": (_normal(g, rows, d) * 0.5).to(torch.bfloat16),
         "gain": (1 + 0.2 * _normal(g, d)).to(torch.bfloat16), "post_gain": None, "gate": None}
    if case["post"]:
        s["post_gain"] = (0.3 + 0.1 * _normal(g, d)).to(torch.bfloat16)
    if case["gate"] != "none":
        s["gate"] = (0.5 * _normal(g, rows if case["gate"] == "row" else 1, d)).to(torch.bfloat16)
    return s


def _quantise(w):
    """Codes (two a byte, the even one low) and scale bytes of float32 rows [n][k]: the least scale that holds a
    group's largest, each value to the nearest code."""
    n, k = w.shape
    x = w.reshape(n, k // 32, 32)
    mantissa, e = torch.frexp(x.abs().amax(-1) / 6)
    e = torch.where(mantissa > 0.5, e, e - 1).clamp(-100, 100)
    x = x * torch.exp2(-e.float())[..., None]
    step = torch.tensor([(a + b) / 2 for a, b in zip(E2M1, E2M1[1:])], device=w.device)
    code = torch.bucketize(x.abs(), step).to(torch.uint8) | ((x < 0).to(torch.uint8) << 3)
    code = code.reshape(n, k // 2, 2)
    return code[..., 0] | (code[..., 1] << 4), (e + 127).to(torch.uint8)


def _product_inputs(case, seed):
    g, m, n, k = _generator(seed), case["m"], case["n"], case["k"]
    codes = torch.empty((n, k // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n, k // 32), dtype=torch.uint8, device="cuda")
    for at in range(0, n, 16384):  # rows at a time: the float32 weights of a whole vocabulary are gigabytes
        rows = min(16384, n - at)
        w = _normal(g, rows, k) * (0.02 * torch.exp(0.3 * _normal(g, rows, 1)))
        codes[at:at + rows], scales[at:at + rows] = _quantise(w)
    a = (_normal(g, m, k) * torch.exp(0.3 * _normal(g, k))).to(torch.bfloat16)
    return {"codes": codes, "scales": scales, "a": a}


def _sequences(case):
    """[(first position, rows)]: the prompts' parts of the chunk, then one row for each decode."""
    c, n = case["chunk"], min(case["prompts"], case["chunk"])
    rng = np.random.default_rng([5, c, n, case["decodes"], case["far"]])
    cut = [0] + sorted(int(x) for x in rng.choice(np.arange(1, c), size=n - 1, replace=False)) + [c] if n > 0 else [0]
    prompts = [(case["prefix"] if i == 0 else 0, cut[i + 1] - cut[i]) for i in range(n)]
    return prompts, [int(x) for x in rng.integers(0, case["far"], size=case["decodes"])]


def _rotate_inputs(case, seed):
    m, rows = MODEL[case["shape"]], case["chunk"] + case["decodes"]
    g = _generator(seed)
    return {"qkv": _normal(g, rows, (m["hq"] + 2 * m["hkv"]) * m["hd"]).to(torch.bfloat16)}


def _positions(case):
    prompts, decodes = _sequences(case)
    return [p + j for p, rows in prompts for j in range(rows)] + decodes


def _frequencies(case):
    """f_i in 64 bits."""
    theta, rot, s = MODEL[case["shape"]]["theta"], case["rot"], case["factor"]
    if case["scaling"] == "ntk":
        theta *= s ** (rot / (rot - 2))
    f = [theta ** (-2.0 * i / rot) for i in range(rot // 2)]
    if case["scaling"] == "linear":
        f = [x / s for x in f]
    if case["scaling"] == "by_parts":
        g = [min(1.0, max(0.0, (8192 * x / (2 * math.pi) - 1.0) / (4.0 - 1.0))) for x in f]
        f = [x * ((1 - h) / s + h) for x, h in zip(f, g)]
    return f


def _sample_inputs(case, seed):
    """Logits as a model gives them: most far below a few; parameters of each row as users set them."""
    g, rows, vocab = _generator(seed), case["rows"], case["vocab"]
    x = _normal(g, rows, vocab) * case["spread"]
    x += 3 * torch.relu(_normal(g, rows, vocab) - 2.5)
    s = {"logits": x.to(torch.bfloat16 if case["logits"] == "bf16" else torch.float32)}
    pick = _uniform(g, 4, rows)
    kind = case["kind"]
    s["temperature"] = (0.6 + 0.7 * _uniform(g, rows)) if kind != "greedy" else torch.zeros(rows, device="cuda")
    s["top_k"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
    s["top_p"] = torch.ones(rows, device="cuda")
    s["min_p"] = torch.zeros(rows, device="cuda")
    k = torch.exp(math.log(5) + (math.log(1000) - math.log(5)) * _uniform(g, rows)).to(torch.int32)
    p = 0.8 + 0.19 * _uniform(g, rows)
    low = 0.02 + 0.13 * _uniform(g, rows)
    if kind == "mixed":
        s["temperature"] = torch.where(pick[0] < 0.1, 0.0, s["temperature"])
        s["top_k"] = torch.where(pick[1] < 0.4, k, 0)
        s["top_p"] = torch.where(pick[2] < 0.6, p, 1.0)
        s["min_p"] = torch.where(pick[3] < 0.2, low, 0.0)
    if kind in ("topk", "topk_topp"):
        s["top_k"] = k
    if kind in ("topp", "topk_topp"):
        s["top_p"] = p
    if kind == "minp":
        s["min_p"] = low
    s["u"] = _uniform(g, rows)
    return s


INPUTS = {"residual_norm": _norm_inputs, "product": _product_inputs, "rotate": _rotate_inputs, "sample": _sample_inputs}


def prepare(case, seed):
    s = INPUTS[case["op"]](case, seed)
    s["op"], s["case"] = case["op"], case
    if case["op"] == "rotate":
        s["pos"] = torch.tensor(_positions(case), dtype=torch.float64, device="cuda")
        s["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    if case["op"] == "product":
        s["value"] = torch.tensor(E2M1 + tuple(-x for x in E2M1), device="cuda")
    if own:
        from paper_2609_07883_amd import api
        s["api"] = api
        s["stream"] = torch.cuda.current_stream().cuda_stream
        {"residual_norm": _own_norm, "product": _own_product, "rotate": _own_rotate, "sample": _own_sample}[case["op"]](s, case, api)
    return s


def _own_norm(s, case, api):
    s["resid_out"] = torch.empty_like(s["resid"])
    s["out"] = torch.empty_like(s["block"])


def _own_product(s, case, api):
    n, k, st = case["n"], case["k"], s["stream"]
    s["packed"] = torch.empty(api.w4_packed_bytes(n, k, case["gated"]), dtype=torch.uint8, device="cuda")
    s["w"] = api.W4(s["packed"].data_ptr(), n, k, case["gated"])
    s["w"].pack(s["codes"].data_ptr(), s["scales"].data_ptr(), st)
    torch.cuda.current_stream().synchronize()  # the codes are not kept
    s["codes"] = s["scales"] = None
    s["out"] = torch.empty((case["m"], n // 2 if case["gated"] else n),
                           dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device="cuda")
    s["ws"] = torch.empty(s["w"].workspace_size(case["m"]), dtype=torch.uint8, device="cuda")


def _own_rotate(s, case, api):
    m = MODEL[case["shape"]]
    prompts, decodes = _sequences(case)
    blocks = sum(-(-(p + n) // 16) for p, n in prompts) + sum(p // 16 + 1 for p in decodes)
    ctx = api.Context(1, m["d"], m["hq"], m["hkv"], m["hd"], m["f"], 1e-5, m["theta"], 262144)
    pool = (blocks, m["hkv"], 16 * m["hd"])
    s["k_pool"], s["v_pool"] = (torch.empty(pool, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.kv_init(s["k_pool"].data_ptr(), s["v_pool"].data_ptr(), blocks)
    ids = list(range(1, 1 + len(prompts) + len(decodes)))
    for sid, p in zip(ids, [p for p, _ in prompts] + decodes):  # the tokens before the batch's
        ctx.seq_create(sid)
        ctx.seq_reserve(sid, p)
    batch = api.Batch.batched([(sid, p, n) for sid, (p, n) in zip(ids, prompts)], ids[len(prompts):], decodes)
    s["ws"] = torch.empty(ctx.attn_workspace_size(case["chunk"], case["decodes"]), dtype=torch.uint8, device="cuda")
    s["plan"] = ctx.attn_begin(batch, s["ws"].data_ptr(), s["ws"].numel(), s["stream"])
    s["rope"] = api.Rope(case["rot"], m["theta"], interleaved=case["interleaved"], scaling=case["scaling"],
                         factor=case["factor"], low=1.0, high=4.0, original_len=8192, mscale=case["mscale"])
    s["out"] = torch.empty((case["chunk"] + case["decodes"], (m["hq"] + m["hkv"]) * m["hd"]), dtype=torch.bfloat16, device="cuda")


def _own_sample(s, case, api):
    rows = case["rows"]
    s["tokens"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    s["logprob"] = torch.empty(rows, dtype=torch.float32, device="cuda")
    s["ws"] = torch.empty(api.sample_workspace_size(rows, case["vocab"]), dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

EPS = 1e-5


def _run_norm(s, case):
    if own:
        s["api"].residual_norm(case["rows"], case["d"], s["resid"].data_ptr(), s["block"].data_ptr(), s["resid_out"].data_ptr(),
                               s["gain"].data_ptr(), s["out"].data_ptr(), resid_f32=case["resid"] == "f32", eps=EPS,
                               post_gain=s["post_gain"].data_ptr() if case["post"] else 0,
                               gate=s["gate"].data_ptr() if case["gate"] != "none" else 0,
                               ld_gate=case["d"] if case["gate"] == "row" else 0, scale=case["scale"], stream=s["stream"])
        return {"resid": s["resid_out"], "out": s["out"]}
    o = s["block"].float()
    if s["post_gain"] is not None:
        o = o * torch.rsqrt((o * o).mean(-1, keepdim=True) + EPS) * s["post_gain"].float()
    if s["gate"] is not None:
        o = o * s["gate"].float()
    r = s["resid"].float() + case["scale"] * o
    y = r * torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS) * s["gain"].float()
    return {"resid": r.to(s["resid"].dtype), "out": y.to(torch.bfloat16)}


def _run_product(s, case):
    if own:
        a = s["a"]
        s["w"].product(a.data_ptr(), case["k"], case["m"], s["out"].data_ptr(), s["out"].shape[1], out_f32=case["out"] == "f32",
                       ws=s["ws"].data_ptr(), ws_bytes=s["ws"].numel(), stream=s["stream"])
        return {"out": s["out"]}
    codes, n, k = s["codes"], case["n"], case["k"]
    w = torch.stack((s["value"][(codes & 15).int()], s["value"][(codes >> 4).int()]), -1).reshape(n, k // 32, 32)
    w = w * torch.exp2(s["scales"].float() - 127)[..., None]
    out = s["a"].float() @ w.reshape(n, k).T
    if case["gated"]:
        gate, up = out[:, :n // 2], out[:, n // 2:]
        out = gate / (1 + torch.exp(-gate)) * up
    return {"out": out.to(torch.bfloat16) if case["out"] == "bf16" else out}


def _run_rotate(s, case):
    m = MODEL[case["shape"]]
    hq, hkv, hd, rot = m["hq"], m["hkv"], m["hd"], case["rot"]
    if own:
        q = s["qkv"].data_ptr()
        out = s["out"].data_ptr()
        s["plan"].rotate(s["rope"], q, q + 2 * hq * hd, (hq + 2 * hkv) * hd, out, out + 2 * hq * hd, (hq + hkv) * hd, s["stream"])
        return {"qk": s["out"]}
    x = s["qkv"].reshape(-1, hq + 2 * hkv, hd)[:, :hq + hkv].float()
    angle = s["pos"][:, None] * s["freq"]
    cos, sin = ((case["mscale"] * f(angle)).float()[:, None] for f in (torch.cos, torch.sin))
    if case["interleaved"]:
        x0, x1 = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((x0 * cos - x1 * sin, x1 * cos + x0 * sin), -1).flatten(-2)
    else:
        x0, x1 = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((x0 * cos - x1 * sin, x1 * cos + x0 * sin), -1)
    return {"qk": torch.cat((y, x[..., rot:]), -1).to(torch.bfloat16).reshape(-1, (hq + hkv) * hd)}


def _run_sample(s, case):
    if own:
        s["api"].sample(s["logits"].data_ptr(), case["rows"], case["vocab"], case["vocab"], s["u"].data_ptr(),
                        s["tokens"].data_ptr(), logits_f32=case["logits"] == "f32", temperature=s["temperature"].data_ptr(),
                        top_k=s["top_k"].data_ptr(), top_p=s["top_p"].data_ptr(), min_p=s["min_p"].data_ptr(),
                        logprob=s["logprob"].data_ptr(), ws=s["ws"].data_ptr(), ws_bytes=s["ws"].numel(), stream=s["stream"])
        return {"token": s["tokens"], "logprob": s["logprob"]}
    x = s["logits"].double()
    vocab = x.shape[1]
    t = s["temperature"].double()[:, None]
    greedy = t <= 0
    sorted_x, order = torch.sort(x, dim=-1, descending=True, stable=True)
    w = torch.exp((sorted_x - sorted_x[:, :1]) / torch.where(greedy, 1.0, t))
    rank = torch.arange(vocab, device="cuda")[None]
    k = s["top_k"][:, None]
    keep = rank < torch.where(greedy, 1, torch.where(k > 0, k, vocab))
    w = torch.where(keep, w, 0.0)
    p = s["top_p"].double()[:, None]
    before = torch.cumsum(w, -1) - w
    keep = (p >= 1) | (before < p * w.sum(-1, keepdim=True)) | (rank == 0)
    keep &= w >= s["min_p"].double()[:, None]
    w = torch.where(keep, w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)  # by index again
    total = torch.cumsum(w, -1)
    z = total[:, -1:]
    token = (total <= s["u"].double()[:, None] * z).sum(-1, keepdim=True).clamp(max=vocab - 1)
    logprob = torch.log(w.gather(1, token) / z)
    return {"token": token[:, 0].to(torch.int32), "logprob": logprob[:, 0].float()}


RUN = {"residual_norm": _run_norm, "product": _run_product, "rotate": _run_rotate, "sample": _run_sample}


def run(state):
    return RUN[state["op"]](state, state["case"])


def work(case):
    """Each input read once, each output written once; the products."""
    if case["op"] == "residual_norm":
        rows, d, one = case["rows"], case["d"], 2 if case["resid"] == "bf16" else 4
        gates = {"none": 0, "channel": 1, "row": rows}[case["gate"]]
        return {"bytes": rows * d * (2 * one + 4) + 2 * d * (1 + case["post"] + gates), "flops": 8 * rows * d}
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        out = m * (n // 2 if case["gated"] else n) * (2 if case["out"] == "bf16" else 4)
        return {"bytes": n * k // 2 + n * k // 32 + 2 * m * k + out, "flops": 2 * m * n * k}
    if case["op"] == "rotate":
        m, rows = MODEL[case["shape"]], case["chunk"] + case["decodes"]
        values = rows * (m["hq"] + m["hkv"]) * m["hd"]
        return {"bytes": 4 * values, "flops": 3 * values}
    one = 2 if case["logits"] == "bf16" else 4
    return {"bytes": case["rows"] * (case["vocab"] * one + 28), "flops": 4 * case["rows"] * case["vocab"]}


# ---------------------------------------------------------------------------
# in 64 bits
# ---------------------------------------------------------------------------

def _exact_norm(case, s):
    o, r = s["block"].double(), s["resid"].double()
    if case["post"]:
        o = o / torch.linalg.vector_norm(o, dim=1, keepdim=True).div(math.sqrt(case["d"])).square().add(EPS).sqrt() * s["post_gain"].double()
    if case["gate"] != "none":
        o = o * s["gate"].double()
    r = r.add(o, alpha=case["scale"])
    ms = torch.linalg.vector_norm(r, dim=1, keepdim=True).square() / case["d"]
    return {"resid": r, "out": r / torch.sqrt(ms + EPS) * s["gain"].double()}


def _exact_product(case, s):
    n, k, m = case["n"], case["k"], case["m"]
    a = s["a"].double()
    out = torch.empty((m, n), dtype=torch.float64, device="cuda")
    for at in range(0, n, 8192):
        codes = s["codes"][at:at + 8192]
        w = torch.empty((codes.shape[0], k), dtype=torch.float64, device="cuda")
        for half in range(2):
            c = (codes >> (4 * half)) & 15
            e, f = (c >> 1) & 3, (c & 1).double()      # exponent and mantissa bit: 2^(e - 1) (1 + f / 2), f / 2 where e is 0
            v = torch.where(e > 0, torch.exp2(e.double() - 1) * (1 + f / 2), f / 2)
            w[:, half::2] = torch.where(c >= 8, -v, v)
        w *= torch.exp2(s["scales"][at:at + 8192].double() - 127).repeat_interleave(32, 1)
        out[:, at:at + 8192] = a @ w.T.contiguous()
    if case["gated"]:
        out = out[:, :n // 2] * torch.sigmoid(out[:, :n // 2]) * out[:, n // 2:]
    return {"out": out}


def _exact_rotate(case, s):
    m = MODEL[case["shape"]]
    heads, rot = m["hq"] + m["hkv"], case["rot"]
    x = s["qkv"].double()[:, :heads * m["hd"]].reshape(-1, heads, m["hd"])
    angle = torch.outer(torch.tensor(_positions(case), dtype=torch.float64), torch.tensor(_frequencies(case), dtype=torch.float64))
    turn = torch.polar(torch.full_like(angle, case["mscale"]), angle).cuda()[:, None]
    i = torch.arange(rot // 2, device="cuda")
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
    z = torch.complex(x[..., first], x[..., second]) * turn
    x[..., first], x[..., second] = z.real, z.imag
    return {"qk": x.reshape(-1, heads * m["hd"])}


def _exact_sample(case, s):
    """Row by row on the host."""
    rows, vocab = case["rows"], case["vocab"]
    x = s["logits"].float().cpu().numpy().astype(np.float64)
    par = {key: s[key].cpu().numpy().astype(np.float64) for key in ("temperature", "top_k", "top_p", "min_p", "u")}
    token, logprob = np.zeros(rows, np.int32), np.zeros(rows)
    for r in range(rows):
        t, k, p, low, u = (par[key][r] for key in ("temperature", "top_k", "top_p", "min_p", "u"))
        best = int(np.argmax(x[r]))
        if t <= 0:
            token[r] = best
            continue
        ids = np.lexsort((np.arange(vocab), -x[r]))
        ids = ids[:int(k)] if k > 0 else ids
        w = np.exp((x[r, ids] - x[r, best]) / t)
        if p < 1:
            mass = np.concatenate([[0.0], np.cumsum(w)])
            last = int(np.searchsorted(mass[:-1], p * mass[-1], side="left"))
            ids, w = ids[:max(1, last)], w[:max(1, last)]
        ids, w = ids[w >= low], w[w >= low]
        by_index = np.argsort(ids)
        ids, w = ids[by_index], w[by_index]
        mass = np.cumsum(w)
        j = min(int(np.searchsorted(mass, u * mass[-1], side="right")), len(ids) - 1)
        token[r], logprob[r] = ids[j], math.log(w[j] / mass[-1])
    return {"token": torch.from_numpy(token), "logprob": torch.from_numpy(logprob)}


def exact(case, seed):
    s = INPUTS[case["op"]](case, seed)
    return {"residual_norm": _exact_norm, "product": _exact_product, "rotate": _exact_rotate, "sample": _exact_sample}[case["op"]](case, s)
