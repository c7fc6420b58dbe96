"""The serving operators together, as the example block uses them: a shared prefix, requests of any lengths in pages, rotation by scaled positions;
against the block's training path and against the block in 64 bits."""

import pytest
import torch

from layers_harness import DEV
from paper_1711_07240_amd import block as B
from paper_1711_07240_amd import cgbn as L
from test_gpu_block import _off

pytestmark = pytest.mark.gpu
# as in test_gpu_block.py, which see for what they count
TOLERANCES = [("f32", 2e-5), ("bf16", 3e-2)]


def _rows(n, channels, dtype, seed):
    return torch.randn(n, channels, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype,tol", TOLERANCES)
@pytest.mark.parametrize("context", [None, ("parts", 8.0, 16.0), ("base", 4.0, 16.0)])
@pytest.mark.parametrize("prefix", [0, 1, 37])
def test_steps_of_requests_as_all_at_once(prefix, context, dtype, tol):
    blk = B.Block(channels=64, heads=2, head_size=32, width=96, positions=128, dtype=dtype, context=context)
    shared = _rows(prefix, 64, blk.dt, 1)
    steps = [[3, 1, 0, 5], [1, 1, 1, 1], [0, 2, 9, 0], [1, 1, 1, 1]]
    lengths = [sum(s[b] for s in steps) for b in range(4)]
    own = [_rows(n, 64, blk.dt, 2 + b) for b, n in enumerate(lengths)]
    want = [blk.forward(torch.cat([shared, x]), 1) for x in own]
    pages = B.Pages(blk, requests=4, rows=13, pages=30, page=4, most=6)
    if prefix:
        assert _off(pages.share(shared), want[0][:prefix].cpu()) <= tol
    at = [0] * 4
    for s in steps:
        pages.fresh.copy_(torch.tensor(s))
        x = torch.cat([own[b][at[b]:at[b] + s[b]] for b in range(4)] + [torch.full((13 - sum(s), 64), 9.0, device=DEV, dtype=blk.dt)])
        out, row = pages.step(x), 0
        for b in range(4):
            if s[b]:
                got, ref = out[row:row + s[b]], want[b][prefix + at[b]:prefix + at[b] + s[b]]
                assert _off(got, ref.cpu()) <= tol, (s, b)
            row, at[b] = row + s[b], at[b] + s[b]
    assert pages.taken.tolist() == [-(-prefix // 4) + sum(-(-n // 4) for n in lengths), 0] and pages.have.tolist() == lengths


def test_a_step_in_a_graph():
    blk = B.Block(channels=64, heads=2, head_size=32, width=96, positions=128, dtype="bf16")
    shared = _rows(21, 64, blk.dt, 1)
    eager, captured = (B.Pages(blk, requests=3, rows=6, pages=30, page=4, most=6) for _ in range(2))
    for p in (eager, captured):
        p.share(shared)
    x = _rows(6, 64, blk.dt, 2)
    captured.fresh.zero_()
    captured.step(x)                    # (makes its workspaces; of no tokens nothing is kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = captured.step(x)
    for n, fresh in enumerate([[1, 1, 1], [4, 0, 2], [1, 1, 1], [0, 0, 0], [2, 3, 1], [1, 1, 1]]):
        x.copy_(_rows(6, 64, blk.dt, 10 + n))
        for p in (eager, captured):
            p.fresh.copy_(torch.tensor(fresh))
        want = eager.step(x)
        graph.replay()
        torch.cuda.synchronize()
        rows = sum(fresh)
        assert torch.equal(out[:rows], want[:rows]) and torch.equal(captured.table, eager.table) and torch.equal(captured.have, eager.have)
        assert all(torch.equal(a, b) for a, b in ((captured.k, eager.k), (captured.v, eager.v), (captured.taken, eager.taken)))


@pytest.mark.parametrize("dtype,tol", TOLERANCES)
@pytest.mark.parametrize("sequences,s", [(1, 1), (3, 7), (2, 49)])
def test_training_with_a_long_context(sequences, s, dtype, tol):
    blk = B.Block(channels=72, heads=3, head_size=16, width=101, positions=64, dtype=dtype, context=("parts", 4.0, 32.0))
    x, dout = _rows(sequences * s, 72, blk.dt, s), _rows(sequences * s, 72, blk.dt, s + 1)
    out = blk.forward(x, sequences)
    dx, grads = blk.backward(dout)
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in blk.p.items()}
    x64 = x.cpu().double().requires_grad_()
    H, D, inner = 3, 16, 48
    norm = lambda t: t / (1 + B.EPS) ** 0.5
    qkv = norm(x64) @ p["qkv"].T + p["bias"]
    angle = (torch.arange(s, dtype=torch.float64)[:, None] * blk.freq.cpu()).repeat(sequences, 1)[:, None]

    def turned(t):
        a, b = t.reshape(-1, H, D).chunk(2, dim=-1)
        return blk.magnitude * torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)

    split = lambda t: t.reshape(sequences, s, H, D).transpose(1, 2)
    q, k, v = split(turned(qkv[:, :inner])), split(turned(qkv[:, inner:2 * inner])), split(qkv[:, 2 * inner:])
    score = (q @ k.transpose(-1, -2) / D ** 0.5).masked_fill(torch.ones(s, s, dtype=torch.bool).triu(1), float("-inf"))
    x1 = x64 + (score.softmax(-1) @ v).transpose(1, 2).reshape(-1, inner) @ p["o"].T
    y1 = norm(x1)
    want = x1 + (torch.nn.functional.silu(y1 @ p["gate"].T) * (y1 @ p["up"].T)) @ p["down"].T
    want.backward(dout.cpu().double())
    assert _off(out, want) <= tol and _off(dx, x64.grad) <= tol and set(grads) == set(p)
    for name in grads:
        assert _off(grads[name], p[name].grad) <= (2 * tol if name in ("qkv", "bias") else tol), name


def test_a_cache_that_is_full():
    """Tokens without a place are counted, the others are served as before."""
    blk = B.Block(channels=64, heads=2, head_size=32, width=96, positions=128, dtype="f32")
    pages = B.Pages(blk, requests=2, rows=4, pages=2, page=2, most=3)
    pages.fresh.fill_(2)
    x = _rows(4, 64, blk.dt, 1)
    first = pages.step(x)
    assert pages.taken.tolist() == [2, 0] and _off(first[:2], blk.forward(x[:2], 1).cpu()) <= 2e-5
    pages.fresh.copy_(torch.tensor([1, 0]))
    before = pages.k.clone()
    pages.step(x)
    assert pages.taken.tolist() == [2, 1] and torch.equal(pages.k, before) and pages.slots.tolist() == [-1] * 4
