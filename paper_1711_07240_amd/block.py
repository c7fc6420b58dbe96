"""A small example: an attention block over the pixels of channels-last feature maps, trained and served through the library's
layers.

    y  = fixed-statistics norm of x                      cgbn_frozen_forward
    q, k, v = slices of y Wqkv^T + b                     cgbn_linear_forward
    q, k = per-head norm, rotated by position            cgbn_head_norm_forward, in place on the slices
    a  = softmax(q k^T / sqrt(D)) v                      under training plain torch; from pages cgbn_prefix_attention
    x1 = a Wo^T + x                                      cgbn_linear_forward, x as the residual
    h  = silu(y1 Wg^T) * (y1 Wu^T), y1 = norm of x1      cgbn_frozen_forward, cgbn_gated_forward
    out = h Wd^T + x1                                    cgbn_linear_forward, x1 as the residual

`Block.forward` keeps what `Block.backward` needs; `Block.token` takes one new token of each sequence and a cache of the earlier ones'
keys and values.  With a `context` queries and keys are not normed but rotated by frequencies that are scaled for long contexts
(cgbn_rotary_frequencies, cgbn_rotate_forward).  `Pages` serves a batch of requests of any lengths behind a prefix that they share, from a cache in pages
(cgbn_page_plan, cgbn_page_store, cgbn_prefix_attention).  `python -m paper_1711_07240_amd.block` trains a block for a few steps and serves a few tokens."""

from __future__ import annotations

import math

import torch

from . import cgbn

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


class Block:
    def __init__(self, channels, heads, head_size, width, positions, dtype="bf16", seed=0, device="cuda", context=None):
        """context: None, or (scaling, factor, trained positions) of a block without the heads' norm, whose contexts are `factor` times as long as
        those that it was trained on; its positions have no bound."""
        gen = torch.Generator(device=device).manual_seed(seed)
        self.C, self.H, self.D, self.F, self.dtype, self.device = channels, heads, head_size, width, dtype, device
        self.dt, inner = DTYPES[dtype], heads * head_size

        def weight(n, k):
            return torch.randn(n, k, device=device, generator=gen).mul_(k ** -0.5).to(self.dt)

        self.p = {"qkv": weight(3 * inner, channels), "o": weight(channels, inner), "gate": weight(width, channels),
                  "up": weight(width, channels), "down": weight(channels, width), "bias": torch.zeros(3 * inner, device=device),
                  "wq": torch.ones(head_size, device=device), "wk": torch.ones(head_size, device=device)}
        one, zero = torch.ones(channels, device=device), torch.zeros(channels, device=device)
        self.norm = {"mean": zero, "var": one, "gamma": one, "beta": zero}          # statistics and affine parameters are constants
        angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] \
            * 10000.0 ** (-torch.arange(0, head_size, 2, device=device, dtype=torch.float64) / head_size)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.workspace = torch.empty(256, dtype=torch.uint8, device=device)
        self.freq = None
        if context is not None:
            scaling, factor, trained = context
            freq = torch.empty(head_size // 2, dtype=torch.float64)
            cgbn.cgbn_rotary_frequencies(head_size, 10000.0, scaling, factor, trained, 32.0, 1.0, freq)
            self.freq = freq.to(device)
            self.magnitude = 0.1 * math.log(factor) + 1 if scaling == "parts" else 1.0
            del self.p["wq"], self.p["wk"]

    # ---- the layers ----

    def _room(self, nbytes):
        if self.workspace.numel() < nbytes:
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return self.workspace

    def _empty(self, *shape, dtype=None):
        return torch.empty(*shape, device=self.device, dtype=dtype or self.dt)

    def _frozen(self, x):
        n, y = self.norm, torch.empty_like(x)
        cgbn.cgbn_frozen_forward(x, x.shape[0], self.C, 1, 1, "NHWC", self.dtype, n["mean"], n["var"], n["gamma"], n["beta"], EPS, y)
        return y

    def _frozen_back(self, dy):
        dx = torch.empty_like(dy)
        cgbn.cgbn_frozen_backward(dy, dy.shape[0], self.C, 1, 1, "NHWC", self.dtype, self.norm["var"], self.norm["gamma"], EPS, dx)
        return dx

    def _linear(self, x, w, bias=None, residual=None, room=None):
        """room: in the place of _room(), if the workspace is another's"""
        m, n, k = x.shape[0], *w.shape
        y = self._empty(m, n)
        ws = (room or self._room)(cgbn.cgbn_linear_workspace_bytes(m, n, k, self.dtype, False))
        cgbn.cgbn_linear_forward(x, w, bias, residual, m, n, k, "none", y, None, self.dtype, ws)
        return y

    def _linear_back(self, dy, x, w, dbias=None):
        m, n, k = x.shape[0], *w.shape
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        ws = self._room(cgbn.cgbn_linear_workspace_bytes(m, n, k, self.dtype, True))
        cgbn.cgbn_linear_backward(dy, x, w, None, m, n, k, "none", dx, dw, dbias, None, self.dtype, ws)
        return dx, dw

    def _rotate(self, qkv, positions, out):
        """Norm and rotation of the q and k slices of rows [q, k, v]; `out` may be `qkv` itself."""
        m, inner, row = qkv.shape[0], self.H * self.D, qkv.shape[1]
        if self.freq is not None:
            cgbn.cgbn_rotate_forward(qkv, row, qkv[:, inner:], row, m, self.H, self.H, self.D, self.D, "halves", positions, self.freq, self.magnitude, out,
                                     out.shape[1], out[:, inner:], out.shape[1], self.dtype)
            return
        cgbn.cgbn_head_norm_forward(qkv, row, qkv[:, inner:], row, m, self.H, self.H, self.D, self.D, "halves", positions, self.cos, self.sin,
                                    self.cos.shape[0], self.p["wq"], self.p["wk"], EPS, out, out.shape[1], out[:, inner:], out.shape[1],
                                    self.dtype)

    def _gated(self, y, save, room=None):
        m = y.shape[0]
        h = self._empty(m, self.F)
        gate, up = (torch.empty_like(h), torch.empty_like(h)) if save else (None, None)
        ws = (room or self._room)(cgbn.cgbn_gated_workspace_bytes(m, self.F, self.C, self.dtype, False))
        cgbn.cgbn_gated_forward(y, self.p["gate"], self.p["up"], m, self.F, self.C, "silu", h, gate, up, self.dtype, ws)
        return h, gate, up

    def _heads(self, rows, sequences):
        """[sequences * S, H * D] -> float [sequences * H, S, D]"""
        s = rows.shape[0] // sequences
        return rows.float().view(sequences, s, self.H, self.D).transpose(1, 2).reshape(sequences * self.H, s, self.D)

    def _rows(self, heads, sequences):
        s = heads.shape[1]
        return heads.view(sequences, self.H, s, self.D).transpose(1, 2).reshape(sequences * s, self.H * self.D)

    # ---- training ----

    def forward(self, x, sequences):
        """x [sequences * S, C]: a token attends to those of its sequence up to itself."""
        inner, s = self.H * self.D, x.shape[0] // sequences
        positions = torch.arange(s, device=self.device, dtype=torch.int32).repeat(sequences)
        y = self._frozen(x)
        qkv = self._linear(y, self.p["qkv"], self.p["bias"])
        qk = self._empty(x.shape[0], 2 * inner)
        self._rotate(qkv, positions, qk)
        q, k, v = (self._heads(t, sequences) for t in (qk[:, :inner], qk[:, inner:], qkv[:, 2 * inner:]))
        later = torch.ones(s, s, dtype=torch.bool, device=self.device).triu(1)
        prob = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(self.D ** -0.5).masked_fill_(later, float("-inf")), dim=-1)
        a = self._rows(torch.bmm(prob, v), sequences).to(self.dt)
        x1 = self._linear(a, self.p["o"], residual=x)
        y1 = self._frozen(x1)
        h, gate, up = self._gated(y1, True)
        out = self._linear(h, self.p["down"], residual=x1)
        self.kept = (sequences, positions, y, qkv, q, k, v, prob, a, y1, h, gate, up)
        return out

    def backward(self, dout):
        """Gradients of the parameters, and of x, from that of the last forward's output."""
        sequences, positions, y, qkv, q, k, v, prob, a, y1, h, gate, up = self.kept
        m, inner, g = y.shape[0], self.H * self.D, {}
        dh, g["down"] = self._linear_back(dout, h, self.p["down"])
        dy1, g["gate"], g["up"] = torch.empty_like(y1), torch.empty_like(self.p["gate"]), torch.empty_like(self.p["up"])
        ws = self._room(cgbn.cgbn_gated_workspace_bytes(m, self.F, self.C, self.dtype, True))
        cgbn.cgbn_gated_backward(dh, y1, self.p["gate"], self.p["up"], gate, up, m, self.F, self.C, "silu", dy1, g["gate"], g["up"], self.dtype, ws)
        dx1 = dout + self._frozen_back(dy1)
        da, g["o"] = self._linear_back(dx1, a, self.p["o"])
        do = self._heads(da, sequences)
        dv = torch.bmm(prob.transpose(1, 2).contiguous(), do)
        dp = torch.bmm(do, v.transpose(1, 2).contiguous())
        ds = prob * (dp - (dp * prob).sum(-1, keepdim=True)) * self.D ** -0.5
        dqkv = torch.empty_like(qkv)
        for n, t in enumerate((torch.bmm(ds, k), torch.bmm(ds.transpose(1, 2).contiguous(), q), dv)):
            dqkv[:, n * inner:(n + 1) * inner] = self._rows(t, sequences)
        row = qkv.shape[1]
        # in place: the gradients of q and k where those of the rotated ones were
        if self.freq is not None:
            cgbn.cgbn_rotate_backward(dqkv, row, dqkv[:, inner:], row, m, self.H, self.H, self.D, self.D, "halves", positions, self.freq, self.magnitude,
                                      dqkv, row, dqkv[:, inner:], row, self.dtype)
        else:
            g["wq"], g["wk"] = (self._empty(self.D, dtype=torch.float32) for _ in range(2))
            ws = self._room(cgbn.cgbn_head_norm_workspace_bytes(m, self.H, self.H, self.D, self.dtype))
            cgbn.cgbn_head_norm_backward(dqkv, row, dqkv[:, inner:], row, qkv, row, qkv[:, inner:], row, m, self.H, self.H, self.D, self.D, "halves",
                                         positions, self.cos, self.sin, self.cos.shape[0], self.p["wq"], self.p["wk"], EPS, dqkv, row,
                                         dqkv[:, inner:], row, g["wq"], g["wk"], self.dtype, ws)
        g["bias"] = self._empty(3 * inner, dtype=torch.float32)
        dy, g["qkv"] = self._linear_back(dqkv, y, self.p["qkv"], g["bias"])
        return dx1 + self._frozen_back(dy), g

    # ---- serving ----

    def token(self, x, cache):
        """x [sequences, C]: one token of each; cache: what earlier calls returned (None: nothing yet).  -> output, cache"""
        sequences, inner = x.shape[0], self.H * self.D
        at = 0 if cache is None else cache[0].shape[1]
        positions = torch.full((sequences,), at, dtype=torch.int32, device=self.device)
        qkv = self._linear(self._frozen(x), self.p["qkv"], self.p["bias"])
        self._rotate(qkv, positions, qkv)
        q, k, v = (self._heads(t, sequences) for t in qkv.split(inner, dim=1))
        if cache is not None:
            k, v = torch.cat([cache[0], k], dim=1), torch.cat([cache[1], v], dim=1)
        prob = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(self.D ** -0.5), dim=-1)
        x1 = self._linear(self._rows(torch.bmm(prob, v), sequences).to(self.dt), self.p["o"], residual=x)
        h, _, _ = self._gated(self._frozen(x1), False)
        return self._linear(h, self.p["down"], residual=x1), (k, v)


class Pages:
    """Requests that a block answers, behind a prefix that they share: a cache in `pages` pages of `page` tokens, up to `rows` new tokens a step.

    `step` can be captured into a graph and replayed: x, `fresh` (how many tokens each request gets) and the cache change in place.
    `taken` has the pages that are taken and how many of the step's tokens got no place or row: those are answered without what they would have left in the
    cache.  Requests do not end here and give no pages back: for others a program makes another cache."""

    def __init__(self, block, requests, rows, pages, page=16, most=64):
        self.block, self.B, self.T, self.pages, self.page, self.most, self.prefix = block, requests, rows, pages, page, most, 0
        shape = (pages, block.H, page, block.D)
        # (zeros: what a place holds before its token is stored is never looked at)
        self.k, self.v = (torch.zeros(*shape, device=block.device, dtype=block.dt) for _ in range(2))
        self.free, self.taken = torch.arange(pages, device=block.device, dtype=torch.int32), self._ints(2)
        self.have, self.fresh, self.table = self._ints(requests), self._ints(requests), self._ints(requests, most)
        self.rows, self.lengths, self.prefix_table = self._ints(requests + 1), self._ints(requests), self._ints(1)
        self.slots, self.positions = self._ints(rows), self._ints(rows)
        plan = cgbn.cgbn_page_plan_workspace_bytes(requests, rows)
        self.plan_room = torch.empty(plan, device=block.device, dtype=torch.uint8)
        self.room, self.layers, self.kept, self.stepped = None, None, [], False

    def _ints(self, *shape):
        return torch.zeros(*shape, device=self.block.device, dtype=torch.int32)

    def _plan(self, table, have, fresh, requests, rows, lengths, slots, positions):
        cgbn.cgbn_page_plan(have, fresh, requests, self.prefix, self.free, self.pages, self.taken, self.taken, table, table.shape[1], self.pages, self.page,
                            slots.shape[0], rows, lengths, slots, positions, self.plan_room)

    def _layers(self, nbytes):
        """The layers' workspace.  Not the block's, which another call may replace by a larger one while a captured step still uses it, or use at the same time."""
        self.layers = self._at_least(self.layers, nbytes)
        return self.layers

    def _at_least(self, room, nbytes):
        if room is not None and room.numel() >= nbytes:
            return room
        if room is not None:
            self.kept.append(room)          # (a captured step of fewer rows may still use it)
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.block.device)

    def _check(self, x, rows):
        """The kernels go by the sizes that they are given: of other rows they would read or store what is not theirs."""
        if x.shape != (rows, self.block.C) or x.dtype != self.block.dt or not x.is_contiguous():
            raise ValueError(f"rows side by side, {rows} x {self.block.C} of {self.block.dt}, and not {tuple(x.shape)} of {x.dtype}")

    def _answer(self, x, table, requests, rows, lengths, slots, positions):
        b, m, inner = self.block, x.shape[0], self.block.H * self.block.D
        qkv = b._linear(b._frozen(x), b.p["qkv"], b.p["bias"], room=self._layers)
        b._rotate(qkv, positions, qkv)
        row = 3 * inner
        cgbn.cgbn_page_store(qkv[:, inner:], row, qkv[:, 2 * inner:], row, m, b.H, b.D, slots, self.k, self.v, self.pages, self.page, b.dtype)
        a = torch.zeros(m, inner, device=b.device, dtype=b.dt)          # rows behind the last token stay zero
        need = cgbn.cgbn_prefix_attention_workspace_bytes(m, requests, b.H, b.H, b.D, self.prefix, table.shape[1] * self.page, b.dtype)
        self.room = self._at_least(self.room, need)
        cgbn.cgbn_prefix_attention(qkv, row, m, requests, rows, lengths, b.H, b.H, b.D, b.D ** -0.5, self.k, self.v, self.pages, self.page, self.prefix_table,
                                   self.prefix, table, table.shape[1], a, inner, None, b.dtype, self.room)
        x1 = b._linear(a, b.p["o"], residual=x, room=self._layers)
        h, _, _ = b._gated(b._frozen(x1), False, self._layers)
        return b._linear(h, b.p["down"], residual=x1, room=self._layers)

    def share(self, x):
        """x [S, C]: the prefix of all requests, once and before the first step.  -> the block's output for it"""
        s = x.shape[0]
        self._check(x, s)
        if s == 0:
            return torch.empty_like(x)
        if self.prefix or self.stepped:
            raise ValueError("a prefix is shared once, before the first step")
        if s > self.pages * self.page:
            raise ValueError(f"{s} tokens, and room for {self.pages * self.page}")
        table = self._ints(1, -(-s // self.page))
        have, fresh, rows, lengths = self._ints(1), self._ints(1) + s, self._ints(2), self._ints(1)
        slots, positions = self._ints(s), self._ints(s)
        plan = cgbn.cgbn_page_plan_workspace_bytes(1, s)
        if self.plan_room.numel() < plan:
            self.plan_room = torch.empty(plan, device=self.block.device, dtype=torch.uint8)
        self._plan(table, have, fresh, 1, rows, lengths, slots, positions)
        out = self._answer(x, table, 1, rows, lengths, slots, positions)
        self.prefix_table, self.prefix = table.view(-1), s
        return out

    def step(self, x):
        """x [rows, C], or fewer rows: the new tokens, request by request, `fresh` says how many of each; rows behind them are padding.  -> output, row by row"""
        m = x.shape[0]
        self._check(x, min(max(m, 1), self.T))
        self.stepped = True
        slots, positions = self.slots[:m], self.positions[:m]
        self._plan(self.table, self.have, self.fresh, self.B, self.rows, self.lengths, slots, positions)
        out = self._answer(x, self.table, self.B, self.rows, self.lengths, slots, positions)
        self.have.copy_(self.lengths)
        return out


def main(steps=8):
    block = Block(channels=256, heads=8, head_size=32, width=683, positions=128)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, target = (torch.randn(8 * 49, 256, device="cuda", generator=gen).to(block.dt) for _ in range(2))
    for step in range(steps):                     # eight 7 x 7 crops, a sequence of pixels each
        error = block.forward(x, 8).float() - target.float()
        _, grads = block.backward((error * (2 / error.numel())).to(block.dt))
        for name, g in grads.items():
            block.p[name] -= (5 * g).to(block.p[name].dtype)          # at 20 the loss grows without bound from the fifth step on
        print(f"step {step}: loss {error.square().mean().item():.4f}", flush=True)
    pages = Pages(block, requests=8, rows=8, pages=40)
    token = pages.share(x[:40])[-8:]
    pages.fresh.fill_(1)
    for _ in range(16):
        token = pages.step(token)
        token = token / token.float().square().mean(-1, keepdim=True).sqrt().to(block.dt)
    print("served 16 tokens of 8 requests behind 40 that they share:", bool(torch.isfinite(token).all()))
    cache, token = None, x[:8].clone()
    for _ in range(16):
        token, cache = block.token(token, cache)
        token = token / token.float().square().mean(-1, keepdim=True).sqrt().to(block.dt)
    print("served 16 tokens of 8 sequences:", bool(torch.isfinite(token).all()))


if __name__ == "__main__":
    main()
