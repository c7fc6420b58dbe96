"""Attention over a shared prefix and pages of each request's own against the definition in 64 bits: types, heads, widths, lengths from none to
long ones, pages that end inside a tile, rows that see nothing, what nobody may look at, splits over keys, tiles of rows."""

import numpy as np
import pytest
import torch

from layers_harness import DEV, f64, workspace
from paper_1711_07240_amd import cgbn as L
from serving_harness import Attention, ints

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [8, 32, 40, 64, 80, 96, 128, 136, 192, 256])
def test_widths(D, dtype):
    a = Attention(dtype, [1, 1, 1], [37, 1, 150], 70, 16, 4, 2, D, stride=8)
    a.check(*a.call())
    a.check(*a.call(single=True, lse=False))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (3, 3), (8, 1), (6, 2), (17, 1), (40, 1), (130, 1)])
def test_heads(Hq, Hk, dtype):
    a = Attention(dtype, [1, 1], [90, 13], 100, 32, Hq, Hk, 32)
    a.check(*a.call(single=True))
    a = Attention(dtype, [2, 5], [90, 13], 33, 8, Hq, Hk, 32)
    a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [1, 2, 8, 64, 256, 1024])
def test_pages(page, dtype):
    a = Attention(dtype, [1, 3], [130, 257], 193, page, 4, 2, 64)
    a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 700])
def test_lengths(length, dtype):
    a = Attention(dtype, [1, 1], [length, 3], 0, 16, 4, 2, 64)
    a.check(*a.call())
    a = Attention(dtype, [1, 1], [0, 3], length, 16, 4, 2, 64)
    a.check(*a.call(single=True))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fresh,lengths,prefix", [([3, 0, 1, 7], [3, 0, 1, 7], 0), ([20, 1, 130], [55, 1, 130], 40), ([5, 5, 5], [2, 0, 5], 0),
                                                  ([64, 65], [300, 65], 129), ([33, 2], [20, 2], 65)])
def test_several_tokens_of_a_request(fresh, lengths, prefix, dtype):
    """Among them requests whose new tokens are more than the cache holds (the first ones see nothing of their own) and without any."""
    for heads in ((2, 2), (8, 2)):
        a = Attention(dtype, fresh, lengths, prefix, 16, *heads, 64, pad=5, stride=16)
        a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
def test_prompts_in_tiles_of_their_own(dtype):
    """So many rows that a workgroup takes the prefix and then its request's own keys."""
    fresh = [300, 1, 511, 128, 129, 640, 37, 0, 256, 700]
    a = Attention(dtype, fresh, [n + 50 * i for i, n in enumerate(fresh)], 200, 16, 16, 8, 32, pad=3)
    a.check(*a.call(), rows=[0, 1, 127, 128, 300, 509, 510, 639, 699])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("prefix,D,fresh", [(1500, 32, [400, 1, 129, 600, 0, 870]), (0, 64, [700, 700, 3, 500]), (2100, 136, [900, 900])])
def test_tiles_that_workgroups_share(prefix, D, fresh, dtype):
    """The last tiles of many: their keys, the prefix's and a request's own as one, are dealt to several workgroups."""
    a = Attention(dtype, fresh, [n + 900 * (i % 2) for i, n in enumerate(fresh)], prefix, 16, 16, 8, D, pad=9)
    got = a.call()
    a.check(*got, rows=[0, 1, 63, 64, 127, 128, 255, 399, 599, 869, 899])
    assert all(torch.equal(x, y) for x, y in zip(got, a.call()))


@pytest.mark.parametrize("dtype", TYPES)
def test_short_contexts_of_many_requests(dtype):
    rng = np.random.default_rng(6)
    a = Attention(dtype, [1] * 90, [int(n) for n in rng.integers(0, 200, 90)], 190, 16, 6, 3, 64)
    a.check(*a.call(single=True))
    a = Attention(dtype, [40] * 9, [int(n) for n in rng.integers(0, 300, 9)], 100, 16, 4, 2, 40)
    a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.125, 1e-30])
def test_scales(scale, dtype):
    """Of zero all keys weigh the same; a negative one turns the order around."""
    a = Attention(dtype, [1, 3], [100, 70], 600, 16, 4, 2, 64)
    a.scale = scale
    a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
def test_long_keys_in_many_parts(dtype):
    a = Attention(dtype, [1, 1, 2], [9000, 30, 4099], 20001, 64, 4, 1, 64, spread=3.0)
    a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("prefix", [0, 300])
@pytest.mark.parametrize("B,most", [(3, 30000), (64, 9000), (65, 9000), (300, 6001), (1024, 5000), (1025, 3000)])
def test_one_request_much_longer_than_the_others(B, most, prefix, dtype):
    """Keys are dealt to workgroups by the lengths, which only the device knows; among the others are requests without keys and without new tokens."""
    rng = np.random.default_rng(B)
    lengths = [int(n) for n in rng.integers(0, 90, B)]
    lengths[B // 3] = most
    a = Attention(dtype, [1] * B, lengths, prefix, 16, 4, 2, 32)
    got = a.call(single=True)
    a.check(*got)
    assert all(torch.equal(x, y) for x, y in zip(got, a.call(single=True)))
    fresh = [int(n) for n in rng.integers(0, 4, B)]
    fresh[B // 3] = 3
    a = Attention(dtype, fresh, [n + m for n, m in zip(fresh, lengths)], prefix, 16, 4, 2, 32, pad=2)
    a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fresh", [[7, 0, 90, 1], [300, 2, 1, 33]])
def test_a_long_request_with_many_new_tokens(fresh, dtype):
    a = Attention(dtype, fresh, [fresh[0] + 5000, 40, fresh[2], 700], 600, 16, 4, 2, 40, pad=1)
    a.check(*a.call(), rows=[0, 1, 6, 15, 16, 31, 32, 63, 64, 89, 127, 128, 255, 299])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths", [[128] * 64, [129] * 64, [512, 513, 1, 0] * 16, [2048] * 16, [16, 32, 48, 640] * 32])
def test_lengths_at_the_ends_of_parts(lengths, dtype):
    """In tables with room for far more; a request of one part is stored without a join."""
    a = Attention(dtype, [1] * len(lengths), lengths, 0, 16, 8, 4, 32, extra=3000)
    a.check(*a.call(single=True))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_requests(dtype):
    rng = np.random.default_rng(5)
    fresh = [int(n) for n in rng.integers(0, 4, 150)]
    a = Attention(dtype, fresh, [n + int(m) for n, m in zip(fresh, rng.integers(0, 90, 150))], 64, 8, 4, 2, 32, pad=1)
    a.check(*a.call())
    a = Attention(dtype, [1] * 150, [1 + int(m) for m in rng.integers(0, 90, 150)], 300, 8, 4, 2, 32)
    a.check(*a.call(single=True))


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores(dtype):
    """One key takes nearly all of the weight, and its place moves: what came before is scaled away."""
    a = Attention(dtype, [1, 2], [400, 70], 130, 16, 4, 2, 64, spread=40.0)
    a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
def test_no_keys_at_all(dtype):
    for prefix in (0, 50):
        a = Attention(dtype, [1, 2], [0, 0], prefix, 16, 4, 2, 32, extra=0)
        assert a.most == 0
        a.check(*a.call())


@pytest.mark.parametrize("dtype", TYPES)
def test_pages_that_are_not_there_are_not_seen(dtype):
    a = Attention(dtype, [1, 2], [100, 64], 70, 16, 4, 2, 64)
    a.table[0, 2], a.table[1, 0], a.prefix_table[1] = a.pages, -1, 1 << 30
    keep0, keep1, shared = np.r_[0:32, 48:100], np.r_[16:64], np.r_[0:16, 32:70]
    got, total = a.call()
    a.own = [tuple(x[:, keep0] for x in a.own[0]), tuple(x[:, keep1] for x in a.own[1])]
    a.shared = tuple(x[:, shared] for x in a.shared)
    a.prefix, a.lengths = len(shared), [len(keep0), len(keep1)]
    a.check(got, total)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fresh,length,heads", [(5, 40, (4, 2)), (5, 900, (4, 2)), (100, 130, (2, 1)), (200, 200, (16, 8)), (300, 1400, (16, 8))])
def test_infinities_of_later_tokens_stay_out(fresh, length, heads, dtype):
    """A later token's key and value reach the rows that see it and no others."""
    bad = length - 3
    a = Attention(dtype, [fresh] * 6, [length] * 6, 30, 16, *heads, 32)
    for b, (what, value) in enumerate([("v", np.inf), ("v", np.nan), ("v", -np.inf), ("k", np.nan), ("v", np.inf)]):
        page, at = a.place(b, bad)
        getattr(a, what)[page, :, at] = value
        a.own[b][0 if what == "k" else 1][:, bad] = value
    page, at = a.place(4, bad + 1)
    a.v[page, :, at] = -np.inf
    out, total = a.call()
    got = f64(out)[:, :a.Hq * a.D]
    for b, want in enumerate([np.inf, np.nan, -np.inf, np.nan, np.nan, None]):
        first = a.rows[b]
        seen = first + bad - (length - fresh)
        assert np.isfinite(got[first:seen]).all(), b
        if want is None:
            assert np.isfinite(got[first:first + fresh]).all()
        else:
            last = got[seen + 1:first + fresh]
            assert np.isnan(last).all() if np.isnan(want) else (last == want).all(), b
            assert np.isnan(got[seen]).all() if want is np.nan and b != 4 else np.isinf(got[seen]).all(), b
    a.check(out, total, rows=[0, 1, bad - (length - fresh) - 1])


@pytest.mark.parametrize("dtype", TYPES)
def test_the_same_bits_every_time(dtype):
    a = Attention(dtype, [1] * 10, list(range(1, 3000, 333)), 5000, 16, 8, 2, 64)
    first = a.call(single=True)
    for _ in range(3):
        again = a.call(single=True)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(first, again))


def test_a_cache_beyond_2_to_the_32_bytes():
    """Places whose byte and element offsets pass 32 bits: two pages far apart, the rest is never touched."""
    page, Hk, D = 1024, 8, 128
    pages = (1 << 31) // page - 1                                # 4 TB of bfloat16 would be all of it: as many as 9 GB hold
    pages = min(pages, 4500)
    k, v = (torch.empty(pages, Hk, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    a = Attention("bf16", [1, 2], [40, 9], 17, page, 8, Hk, D)
    moved = {int(p): pages - 1 - i for i, p in enumerate(sorted(set(a.prefix_table) | {int(a.table[0, 0]), int(a.table[1, 0])}))}
    for old, new in moved.items():
        k[new], v[new] = a.k[old], a.v[old]
    a.prefix_table = np.array([moved[int(p)] for p in a.prefix_table], np.int32)
    for b in range(2):
        a.table[b, 0] = moved[int(a.table[b, 0])]
    assert k.numel() * 2 > 1 << 32 and min(moved.values()) * page * Hk * D > 1 << 32
    a.k, a.v, a.pages = k, v, pages
    a.check(*a.call())


def test_two_streams_and_a_replayed_graph():
    """Two calls at once with a workspace each; a captured one follows lengths, tables and keys that change between its replays."""
    a, b = Attention("bf16", [1] * 4, [900, 40, 1, 300], 700, 16, 8, 2, 64), Attention("f32", [2, 3], [50, 600], 900, 16, 4, 2, 64)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s, x in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            x.got = x.call()
    for x in (a, b):
        x.check(*x.got)
    out, total = torch.full((4, a.ld), 7.0, dtype=torch.bfloat16, device=DEV), torch.empty(4, a.Hq, device=DEV)
    lengths, shared, table = ints(a.lengths), ints(a.prefix_table), ints(a.table)
    nb = L.cgbn_prefix_attention_workspace_bytes(4, 4, 8, 2, 64, a.prefix, a.most * 16, "bf16")
    ws = workspace(nb)

    def step():
        L.cgbn_prefix_attention(a.q, a.ld, 4, 4, None, lengths, 8, 2, 64, a.scale, a.k, a.v, a.pages, 16, shared, a.prefix, table, a.most, out, a.ld, total,
                                "bf16", ws, nb)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    full = list(a.lengths)
    for cut in (0, 1, 33, 250, 0):
        a.lengths = [max(n - cut, 0) for n in full]
        lengths.copy_(ints(a.lengths))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        a.check(out, total)
        eager = a.call(single=True)
        assert torch.equal(eager[0], out) and torch.equal(eager[1], total)
