"""A small example: an attention block over the pixels of channels-last feature maps, trained and served through the library's
layers.

    y  = fixed-statistics norm of x                      cgbn_frozen_forward
    q, k, v = slices of y Wqkv^T + b                     cgbn_linear_forward
    q, k = per-head norm, rotated by position            cgbn_head_norm_forward, in place on the slices
    a  = softmax(q k^T / sqrt(D)) v                      plain torch: the library has no attention
    x1 = a Wo^T + x                                      cgbn_linear_forward, x as the residual
    h  = silu(y1 Wg^T) * (y1 Wu^T), y1 = norm of x1      cgbn_frozen_forward, cgbn_gated_forward
    out = h Wd^T + x1                                    cgbn_linear_forward, x1 as the residual

`Block.forward` keeps what `Block.backward` needs; `Block.token` takes one new token of each sequence and a cache of the earlier ones'
keys and values.  `python -m paper_1711_07240_amd.block` trains a block for a few steps and serves a few tokens."""

from __future__ import annotations

import torch

from . import cgbn

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


class Block:
    def __init__(self, channels, heads, head_size, width, positions, dtype="bf16", seed=0, device="cuda"):
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

    def _linear(self, x, w, bias=None, residual=None):
        m, n, k = x.shape[0], *w.shape
        y = self._empty(m, n)
        ws = self._room(cgbn.cgbn_linear_workspace_bytes(m, n, k, self.dtype, False))
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
        cgbn.cgbn_head_norm_forward(qkv, row, qkv[:, inner:], row, m, self.H, self.H, self.D, self.D, "halves", positions, self.cos, self.sin,
                                    self.cos.shape[0], self.p["wq"], self.p["wk"], EPS, out, out.shape[1], out[:, inner:], out.shape[1],
                                    self.dtype)

    def _gated(self, y, save):
        m = y.shape[0]
        h = self._empty(m, self.F)
        gate, up = (torch.empty_like(h), torch.empty_like(h)) if save else (None, None)
        ws = self._room(cgbn.cgbn_gated_workspace_bytes(m, self.F, self.C, self.dtype, False))
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
        g["wq"], g["wk"] = (self._empty(self.D, dtype=torch.float32) for _ in range(2))
        row, ws = qkv.shape[1], self._room(cgbn.cgbn_head_norm_workspace_bytes(m, self.H, self.H, self.D, self.dtype))
        # in place: the gradients of q and k where those of the rotated ones were
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
    cache, token = None, x[:8].clone()
    for _ in range(16):
        token, cache = block.token(token, cache)
        token = token / token.float().square().mean(-1, keepdim=True).sqrt().to(block.dt)
    print("served 16 tokens of 8 sequences:", bool(torch.isfinite(token).all()))


if __name__ == "__main__":
    main()
