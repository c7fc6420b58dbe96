"""The example block against the same block in 64 bits, differentiated by autograd, and its serving path against its training path."""

import pytest
import torch

from layers_harness import DEV
from paper_1711_07240_amd import block as B

pytestmark = pytest.mark.gpu


def _reference(blk, x, sequences):
    """The block's definition in 64 bits on the CPU; leaves that ask for gradients."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in blk.p.items()}
    x = x.detach().cpu().double().requires_grad_()
    H, D, inner, s = blk.H, blk.D, blk.H * blk.D, x.shape[0] // sequences
    norm = lambda t: t / (1 + B.EPS) ** 0.5
    qkv = norm(x) @ p["qkv"].T + p["bias"]
    cos, sin = (t.cpu().double()[:s].repeat(sequences, 1)[:, None] for t in (blk.cos, blk.sin))

    def rotated(t, w):
        t = t.reshape(-1, H, D)
        t = t / (t.pow(2).mean(-1, keepdim=True) + B.EPS).sqrt() * w
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    split = lambda t: t.reshape(sequences, s, H, D).transpose(1, 2)
    q, k, v = split(rotated(qkv[:, :inner], p["wq"])), split(rotated(qkv[:, inner:2 * inner], p["wk"])), split(qkv[:, 2 * inner:])
    score = (q @ k.transpose(-1, -2) / D ** 0.5).masked_fill(torch.ones(s, s, dtype=torch.bool).triu(1), float("-inf"))
    a = (score.softmax(-1) @ v).transpose(1, 2).reshape(-1, inner)
    x1 = x + a @ p["o"].T
    y1 = norm(x1)
    out = x1 + (torch.nn.functional.silu(y1 @ p["gate"].T) * (y1 @ p["up"].T)) @ p["down"].T
    return out, x, p


def _off(got, want):
    got, want = got.detach().cpu().double(), want.detach().double()
    return float((got - want).norm() / want.norm())


# float: a few dozen roundings of 2^-24 in a row, grown by softmax and norms; bfloat16: eight roundings of 2^-9 (root mean square) of
# tensors on the way forward and as many back, each at most the size of the result
@pytest.mark.parametrize("dtype,tol", [("f32", 2e-5), ("bf16", 3e-2)])
@pytest.mark.parametrize("sequences,s", [(1, 1), (3, 7), (2, 49)])
def test_forward_and_backward(sequences, s, dtype, tol):
    blk = B.Block(channels=72, heads=3, head_size=16, width=101, positions=64, dtype=dtype)
    gen = torch.Generator(device=DEV).manual_seed(s)
    x, dout = (torch.randn(sequences * s, 72, device=DEV, generator=gen).to(blk.dt) for _ in range(2))
    blk.p["bias"].normal_(generator=gen)
    blk.p["wq"].add_(0.3), blk.p["wk"].sub_(0.2)
    out = blk.forward(x, sequences)
    dx, grads = blk.backward(dout)
    want, x64, p64 = _reference(blk, x, sequences)
    want.backward(dout.cpu().double())
    assert _off(out, want) <= tol
    assert _off(dx, x64.grad) <= tol
    for name in grads:
        if s == 1 and name in ("wq", "wk"):          # one token attends to itself alone: these gradients are zero
            assert float(grads[name].abs().max()) <= tol
            continue
        assert _off(grads[name], p64[name].grad) <= (2 * tol if name in ("qkv", "bias", "wq", "wk") else tol), name


@pytest.mark.parametrize("dtype,tol", [("f32", 2e-5), ("bf16", 3e-2)])
def test_tokens_one_by_one_as_all_at_once(dtype, tol):
    blk = B.Block(channels=64, heads=2, head_size=32, width=96, positions=16, dtype=dtype)
    x = torch.randn(3, 9, 64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).to(blk.dt)
    want = blk.forward(x.reshape(27, 64), 3).view(3, 9, 64)
    cache = None
    for t in range(9):
        out, cache = blk.token(x[:, t].contiguous(), cache)
        assert _off(out, want[:, t].cpu()) <= tol


def test_the_command(capsys):
    B.main(steps=4)
    lines = capsys.readouterr().out.splitlines()
    losses = [float(line.split()[-1]) for line in lines if line.startswith("step")]
    assert len(losses) == 4 and losses[-1] < losses[0] and lines[-1].endswith("True")
