"""A context over random pools on the GPU with its float64 twin, for the KV-cache operator tests."""
from __future__ import annotations

import numpy as np
import torch

from paper_2609_07883_amd import api
from tests import kv_oracle as O


class Rig:
    """hq / hkv heads of hd; seqs: {id: cached tokens}; blocks of the sequences are interleaved in the pool.  Slots
    that no token owns hold NaN, and the scales of blocks that no sequence owns too."""

    def __init__(self, hq, hkv, hd, seqs, cache="e4m3", layers=1, window=0, sinks=0, windowed=None, spare=3, seed=0,
                 max_pos=8192, grow=0):
        self.hq, self.hkv, self.hd, self.cache, self.layers = hq, hkv, hd, cache, layers
        self.window, self.sinks = window, sinks
        self.windowed = list(windowed) if windowed is not None else [window > 0] * layers
        self.ctx = api.Context(layers, 256, hq, hkv, hd, 256, 1e-5, 10000.0, max_pos)
        need = sum(-(-(n + grow) // 16) for n in seqs.values())
        self.blocks = need + spare
        gen = np.random.default_rng(seed)
        self.rng = gen
        shape = (layers, self.blocks, hkv, 16, hd)
        self.k, self.v = gen.standard_normal(shape), gen.standard_normal(shape)
        self.ke = self.ve = None
        if cache == "e4m3":
            self.ke, self.ve = (gen.integers(-9, -4, shape[:3]).astype(np.float64) for _ in range(2))
            self.k, self.v = (O.round_e4m3(np.clip(x * 100, -448, 448)) for x in (self.k, self.v))
        else:
            self.k, self.v = (torch.from_numpy(x).bfloat16().double().numpy() for x in (self.k, self.v))
        self.attach()
        self.ctx.set_window(window, sinks, self.windowed if window else None)
        self.len = dict(seqs)
        todo = dict(seqs)
        for sid in seqs:
            self.ctx.seq_create(sid)
        step = 16
        while todo:
            for sid in list(todo):
                self.ctx.seq_reserve(sid, min(step, todo[sid]))
                if step >= todo[sid]:
                    del todo[sid]
            step += 16
        owned = np.zeros((self.blocks, 16), bool)
        for sid, n in seqs.items():
            bt = self.ctx.block_table(sid)
            for t in range(n):
                owned[bt[t // 16], t % 16] = True
        for x in (self.k, self.v):
            x[:, ~owned.any(1)] = np.nan
            x.transpose(1, 3, 0, 2, 4)[~owned] = np.nan
        for e in (self.ke, self.ve):
            if e is not None:
                e[:, ~owned.any(1)] = np.nan
        self.upload()

    def attach(self):
        n, b, hkv, hd = self.layers, self.blocks, self.hkv, self.hd
        dt, w = (torch.float8_e4m3fn, 64) if self.cache == "e4m3" else (torch.bfloat16, 32)
        self.k_pool = torch.empty((n, b, hkv, hd // w, 16, w), dtype=dt, device="cuda")
        self.v_pool = torch.empty((n, b, hkv, hd, 16), dtype=dt, device="cuda")
        if self.cache == "e4m3":
            self.k_scale = torch.empty((n, b, hkv), dtype=torch.float32, device="cuda")
            self.v_scale = torch.empty_like(self.k_scale)
            self.ctx.kv_init_8bit(self.k_pool.data_ptr(), self.v_pool.data_ptr(), self.k_scale.data_ptr(),
                                  self.v_scale.data_ptr(), b)
        else:
            self.ctx.kv_init(self.k_pool.data_ptr(), self.v_pool.data_ptr(), b)

    def upload(self):
        n, b, hkv, hd = self.layers, self.blocks, self.hkv, self.hd
        w = self.k_pool.shape[-1]
        dt = self.k_pool.dtype
        k = torch.from_numpy(self.k.reshape(n, b, hkv, 16, hd // w, w).transpose(0, 1, 2, 4, 3, 5).copy()).float()
        v = torch.from_numpy(self.v.transpose(0, 1, 2, 4, 3).copy()).float()
        self.k_pool.copy_(k.to(dt))
        self.v_pool.copy_(v.to(dt))
        if self.cache == "e4m3":
            self.k_scale.copy_(torch.from_numpy(2.0 ** self.ke).float())
            self.v_scale.copy_(torch.from_numpy(2.0 ** self.ve).float())
        torch.cuda.synchronize()

    def rows(self, n, q_std=1.0):
        """Random fused q, k, v rows (bf16) on the GPU, and as float64 [n][heads][hd] each."""
        x = self.rng.standard_normal((n, self.hq + 2 * self.hkv, self.hd))
        x[:, : self.hq] *= q_std
        x *= np.exp2(self.rng.integers(-3, 3, (n, 1, 1)))
        return self.put(x)

    def put(self, x):
        t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)
        f = t.double().numpy()
        return t.reshape(len(x), -1).cuda(), f[:, : self.hq], f[:, self.hq:self.hq + self.hkv], f[:, self.hq + self.hkv:]

    # -- the definition ---------------------------------------------------------
    def model_append(self, layer, batch, k, v):
        row = 0
        for sid, at, n in self.runs(batch):
            bt = self.ctx.block_table(sid)
            p = at
            while p < at + n:
                m = min(16 - p % 16, at + n - p)
                blk = bt[p // 16]
                for x, e, new in ((self.k, self.ke, k), (self.v, self.ve, v)):
                    for h in range(self.hkv):
                        r = new[row:row + m, h]
                        if e is None:
                            x[layer, blk, h, p % 16:p % 16 + m] = r
                        else:
                            old = e[layer, blk, h]
                            e[layer, blk, h] = O.append_block(x[layer, blk, h], 0 if np.isnan(old) else int(old), p % 16, r)
                p += m
                row += m

    @staticmethod
    def runs(batch):
        return list(batch.prefill_list) + [(s, c, 1) for s, c in zip(batch.decode_seqs, batch.context_lens)]

    def dense(self, layer, sid, n):
        bt = np.asarray(self.ctx.block_table(sid))[: -(-n // 16)]
        out = []
        for x, e in ((self.k, self.ke), (self.v, self.ve)):
            y = x[layer, bt]
            if e is not None:
                y = y * (2.0 ** e[layer, bt])[..., None, None]
            out.append(y.transpose(0, 2, 1, 3).reshape(-1, self.hkv, self.hd)[:n])
        return out

    def model_attend(self, layer, batch, q, rows=None):
        """(out, bound) [rows][hq][hd] of the rows asked for (all)."""
        w = (self.window, self.sinks) if self.windowed[layer] else (0, 0)
        outs, bounds, row = [], [], 0
        for sid, at, n in self.runs(batch):
            k, v = self.dense(layer, sid, at + n)
            pick = [r for r in range(n) if rows is None or row + r in rows]
            o, b = O.attend(q[[row + r for r in pick]], k, v, [at + r for r in pick], *w)
            outs.append(o)
            bounds.append(b)
            row += n
        return np.concatenate(outs), np.concatenate(bounds)

    # -- the library --------------------------------------------------------------
    def begin(self, batch, stream=0):
        n = self.ctx.attn_workspace_size(batch.chunk, len(batch.decode_seqs))
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        plan = self.ctx.attn_begin(batch, ws.data_ptr(), n, stream)
        plan.ws = ws
        return plan

    def append(self, plan, layer, x, stream=0):
        p = x.data_ptr()
        plan.append(layer, p + 2 * self.hq * self.hd, p + 2 * (self.hq + self.hkv) * self.hd, x.stride(0), stream)

    def attend(self, plan, layer, x, out=None, stream=0):
        if out is None:
            out = torch.full((x.shape[0], self.hq * self.hd), float("nan"), dtype=torch.bfloat16, device="cuda")
        plan.attend(layer, x.data_ptr(), x.stride(0), out.data_ptr(), stream)
        return out

    def float_rows(self, out):
        torch.cuda.synchronize()
        return out.cpu().double().numpy().reshape(out.shape[0], self.hq, self.hd)

    def check_cache(self, layer, what=""):
        """Every slot and scale of the layer's pools, bit for bit (NaN as NaN)."""
        torch.cuda.synchronize()
        for name, pool, x, is_k in (("k", self.k_pool, self.k, True), ("v", self.v_pool, self.v, False)):
            got = O.pages(pool[layer], is_k)
            assert np.array_equal(got, x[layer], equal_nan=True), f"{what}: {name} pages differ"
        if self.cache == "e4m3":
            for name, s, e in (("k", self.k_scale, self.ke), ("v", self.v_scale, self.ve)):
                assert np.array_equal(s[layer].cpu().double().numpy(), 2.0 ** e[layer], equal_nan=True), f"{what}: {name} scales"
