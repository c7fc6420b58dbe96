"""The operators that serve an attention block to a batch of requests: the plan of a paged cache (tables, slots, positions), the rotation of
queries and keys by scaled positions with its backward, the store of new keys and values into pages, and attention of all requests'
new tokens over a prefix that they share and pages of their own.

`listed()` names the cases, `draw(rng)` gives more of the same ranges, `prepare` makes what a program has in hand before the
call, `run` is one pass (the plain form, or the library's entry points where `own` is true), `exact` the same results from the
definitions in 64 bits and `work` the bytes and operations a pass cannot do without."""

import json
import math
import random

import torch

own = False

DEVICE = "cuda"
TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}

# What a pass does ("op"):
#   page_plan          from the requests' lengths: where each one's new tokens start, the pages they take from the free list, and each token's
#                      position and place in the cache
#   rotate_forward     q and k (slices of a joint projection's rows) turned by position, the first R values of each head
#   rotate_backward    gradients turned back
#   page_store         keys and values of new tokens to their places in the pages
#   prefix_attention   softmax attention of every new token over the shared prefix and its own request's pages; the logarithm of the sum too


def _plan(name, b, t, page, max_pages, prompts, prompt):
    return {"name": name, "op": "page_plan", "B": b, "T": t, "page": page, "max_pages": max_pages, "prompts": prompts, "prompt": prompt}


def _rotate(name, op, dtype, t, hq, hk, d, r, style, far, scaling, factor):
    return {"name": name, "op": op, "dtype": dtype, "T": t, "Hq": hq, "Hk": hk, "D": d, "R": r, "style": style, "far": far, "scaling": scaling,
            "factor": factor}


def _store(name, dtype, t, hk, d, page):
    return {"name": name, "op": "page_store", "dtype": dtype, "T": t, "Hk": hk, "D": d, "page": page}


def _attention(name, dtype, b, hq, hk, d, page, prefix, shortest, longest, fresh, pad=0):
    return {"name": name, "op": "prefix_attention", "dtype": dtype, "B": b, "Hq": hq, "Hk": hk, "D": d, "page": page, "prefix": prefix,
            "shortest": shortest, "longest": longest, "fresh": fresh, "pad": pad}


def listed():
    return [
        # one decoding step of sixteen requests: latency is all there is to it
        _plan("plan_16_requests", 16, 16, 16, 256, 0.0, 1),
        # a step that mixes decoding with prompts, the batch padded to a fixed number of rows
        _plan("plan_1024_requests", 1024, 131072, 16, 512, 0.25, 960),
        # eight sequences, one token each, a million tokens into a context scaled by parts
        _rotate("rotate_8_far_tokens_bf16", "rotate_forward", "bf16", 8, 32, 8, 128, 128, "halves", 1 << 20, "parts", 32.0),
        # a prompt batch: q and k are slices of the joint projection's rows
        _rotate("rotate_32k_bf16", "rotate_forward", "bf16", 32768, 32, 8, 128, 128, "halves", 131072, "base", 8.0),
        # training in full precision with heads of 80 values, of which 32 are turned, pair by pair
        _rotate("rotate_8k_bwd_f32", "rotate_backward", "f32", 8191, 20, 20, 80, 32, "interleaved", 8192, "positions", 4.0),
        # a decoding step's keys and values, 64 requests
        _store("store_64_tokens_bf16", "bf16", 64, 8, 128, 16),
        # a prompt batch's, in full precision, heads of 80
        _store("store_20k_f32", "f32", 20011, 20, 80, 32),
        # three sequences of a small block: a short prompt, a few tokens of their own
        _attention("attend_3_small_bf16", "bf16", 3, 8, 8, 32, 16, 100, 1, 60, 1),
        # decoding 64 requests behind one long prompt: its keys are read once, for 256 rows of each head
        _attention("attend_64_shared_32k_bf16", "bf16", 64, 32, 8, 128, 16, 32768, 64, 2048, 1),
        # four long conversations, a short common start: the read of the requests' own pages is all there is to it
        _attention("attend_4_long_bf16", "bf16", 4, 32, 8, 128, 64, 1000, 65536, 131072, 1),
        # questions of up to 512 tokens put to one document, rows padded to a round number: products count
        _attention("attend_prompts_bf16", "bf16", 16, 32, 8, 128, 16, 8191, 1, 700, 512, 300),
        # three drafted tokens a request in full precision, heads of 80 without sharing
        _attention("attend_drafts_f32", "f32", 24, 20, 20, 80, 32, 4001, 3, 1500, 3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["page_plan", "rotate_forward", "rotate_backward", "page_store", "prefix_attention", "prefix_attention", "prefix_attention"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    page = rng.choice([8, 16, 32, 64, 128])
    if op == "page_plan":
        b = _log(rng, 1, 4096)
        prompts = rng.choice([0.0, 0.1, 0.5])
        prompt = _log(rng, 2, 2048) if prompts else 1
        t = min(131072, int(b * (1 + prompts * prompt / 2)) + rng.randrange(0, 100))
        return {"op": op, "B": b, "T": t, "page": page, "max_pages": rng.randrange(4, 512), "prompts": prompts, "prompt": prompt}
    if op.startswith("rotate"):
        d = rng.choice([32, 64, 80, 96, 128, 256, rng.randrange(33, 200)])
        r = rng.choice([d // 2 * 2, d // 4 * 2])
        hk = rng.choice([1, 2, 4, 8, 16])
        hq = hk * rng.choice([1, 2, 4, 8])
        t = max(1, min(_log(rng, 1, 32768), 160_000_000 // ((hq + hk) * d)))
        return {"op": op, "dtype": dtype, "T": t, "Hq": hq, "Hk": hk, "D": d, "R": r, "style": rng.choice(["halves", "interleaved"]),
                "far": _log(rng, 512, 1 << 20), "scaling": rng.choice(["none", "positions", "base", "parts"]), "factor": rng.choice([2.0, 8.0, 40.0])}
    d, hk = rng.choice([32, 64, 80, 96, 128, 256]), rng.choice([1, 2, 4, 8, 20])
    if op == "page_store":
        t = max(1, min(_log(rng, 1, 65536), 40_000_000 // (hk * d)))
        return {"op": op, "dtype": dtype, "T": t, "Hk": hk, "D": d, "page": page}
    hq = hk * rng.choice([1, 2, 3, 4, 8])
    b, fresh = _log(rng, 1, 128), rng.choice([1, 1, 1, 2, 5, 100])
    prefix = rng.choice([0, _log(rng, 1, 65536)])
    longest = _log(rng, fresh, 32768)
    case = {"op": op, "dtype": dtype, "B": b, "Hq": hq, "Hk": hk, "D": d, "page": page, "prefix": prefix, "shortest": max(1, longest // rng.choice([1, 3, 50])),
            "longest": longest, "fresh": fresh, "pad": rng.choice([0, 7]) if fresh > 1 else 0}
    # no more than a part of the largest listed ones (full precision, with a tenth of the rate, a tenth of the products)
    while True:
        cost = work(case)
        dense = 4 * case["B"] * hk * case["longest"] * (2 * d + case["fresh"] * hq // hk)          # what a padded batch holds in full precision
        if cost["bytes"] <= 1e9 and cost["flops"] <= (1.5e11 if dtype == "bf16" else 1.5e10) and dense <= 8e9:
            return case
        for key in ("prefix", "longest"):
            case[key] = case[key] * 3 // 4 if key == "prefix" else max(fresh, case[key] * 3 // 4)
        case["B"] = max(1, case["B"] * 3 // 4)
        case["shortest"] = min(case["shortest"], case["longest"])


def _lengths(case):
    """New tokens and private keys (the new ones among them) of each request, from the case alone."""
    rng = random.Random(json.dumps({k: v for k, v in case.items() if k != "name"}, sort_keys=True))
    fresh = [case["fresh"] if case["fresh"] < 8 else rng.randrange(1, case["fresh"] + 1) for _ in range(case["B"])]
    return fresh, [max(n, rng.randrange(case["shortest"], case["longest"] + 1)) for n in fresh]


# ---- inputs -----------------------------------------------------------------------------------------------------


def _frequencies(case):
    """Radians a position of each pair, for a context of 4096 positions stretched by `factor`."""
    r, base, factor, trained, fast, slow = case["R"], 10000.0, case["factor"], 4096.0, 32.0, 1.0
    if case["scaling"] == "base" and r > 2:
        base *= factor ** (r / (r - 2))
    found = []
    for i in range(r // 2):
        f = base ** (-2.0 * i / r)
        if case["scaling"] == "positions":
            f /= factor
        elif case["scaling"] == "parts":
            keep = min(1.0, max(0.0, (trained * f / (2 * math.pi) - slow) / (fast - slow)))
            f = f * keep + f / factor * (1 - keep)
        found.append(f)
    return found


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    op = case["op"]
    dt = TORCH_DTYPE[case.get("dtype", "f32")]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, device=DEVICE, generator=gen).mul_(scale).to(dt)

    def whole(lo, hi, *shape):
        return torch.randint(lo, hi, shape, device=DEVICE, generator=gen, dtype=torch.int32)

    def shuffled(n):
        return torch.randperm(n, device=DEVICE, generator=gen, dtype=torch.int64).int()

    if op == "page_plan":
        b, page, most = case["B"], case["page"], case["max_pages"]
        room = most * page
        fresh = torch.ones(b, device=DEVICE, dtype=torch.int32)
        if case["prompts"]:
            asks = torch.rand(b, device=DEVICE, generator=gen) < case["prompts"]
            fresh = torch.where(asks, whole(1, case["prompt"] + 1, b), fresh)
        have = torch.minimum(whole(0, room // 2 + 1, b), room - fresh).clamp_(min=0)
        held = (have + page - 1) // page
        wanted = (have + fresh + page - 1) // page - held
        pages = int(held.sum()) + int(wanted.sum()) + 64
        order = shuffled(pages)
        table = torch.full((b, most), -1, device=DEVICE, dtype=torch.int32)
        place = torch.arange(most, device=DEVICE)[None] < held[:, None]
        table[place] = order[:int(held.sum())]
        free = order[int(held.sum()):].contiguous()
        taken = whole(0, 32, 1)
        return {"have": have, "fresh": fresh, "free": free, "taken": taken, "table": table, "pages": pages}
    if op.startswith("rotate"):
        t, hq, hk, d = case["T"], case["Hq"], case["Hk"], case["D"]
        a = {"positions": whole(0, case["far"], t), "freq": torch.tensor(_frequencies(case), dtype=torch.float64, device=DEVICE)}
        a["magnitude"] = 0.1 * math.log(case["factor"]) + 1 if case["scaling"] == "parts" else 1.0
        if op == "rotate_forward":
            a["qkv"] = normal(t, (hq + 2 * hk) * d)              # the joint projection's rows: q, k, v side by side
        else:
            a["dyq"], a["dyk"] = normal(t, hq * d, scale=1e-2), normal(t, hk * d, scale=1e-2)
        return a
    hk, d, page = case["Hk"], case["D"], case["page"]
    if op == "page_store":
        t = case["T"]
        pages = (t + t // 4 + page - 1) // page + 2
        slots = shuffled(pages * page)[:t].contiguous()          # requests' tokens lie all over the pool
        slots[t - t // 50:] = -1                                 # the batch's padding
        return {"kv": normal(t, 2 * hk * d), "slots": slots, "pages": pages,
                "k_pages": normal(pages, hk, page, d), "v_pages": normal(pages, hk, page, d)}
    fresh, lengths = _lengths(case)
    shared = (case["prefix"] + page - 1) // page
    most = (case["longest"] + page - 1) // page + 1
    need = [(n + page - 1) // page for n in lengths]
    pages = shared + sum(need) + 3
    order = shuffled(pages)
    a = {"prefix_table": order[:shared].contiguous(), "pages": pages}
    held = torch.tensor(need, device=DEVICE)
    a["table"] = torch.full((case["B"], most), -1, device=DEVICE, dtype=torch.int32)
    a["table"][torch.arange(most, device=DEVICE)[None] < held[:, None]] = order[shared:shared + sum(need)]
    rows = [0]
    for n in fresh:
        rows.append(rows[-1] + n)
    a["rows"] = torch.tensor(rows, device=DEVICE, dtype=torch.int32)
    a["lengths"] = torch.tensor(lengths, device=DEVICE, dtype=torch.int32)
    a["q"] = normal(rows[-1] + case["pad"], case["Hq"] * d, scale=1.5)
    a["k_pages"], a["v_pages"] = normal(pages, hk, page, d), normal(pages, hk, page, d)
    return a


def prepare(case, seed):
    a = _inputs(case, seed)
    op = case["op"]
    dt = TORCH_DTYPE[case.get("dtype", "f32")]

    def ints(*shape):
        return torch.zeros(*shape, device=DEVICE, dtype=torch.int32)

    # buffers that a program keeps from step to step
    if op == "page_plan":
        out = {"counts": ints(2), "table": a["table"], "rows": ints(case["B"] + 1), "lengths": ints(case["B"]), "slots": ints(case["T"]),
               "positions": ints(case["T"])}
    elif op.startswith("rotate"):
        nq, nk = case["Hq"] * case["D"], case["Hk"] * case["D"]
        if op == "rotate_forward":
            a["q"], a["k"] = a["qkv"][:, :nq], a["qkv"][:, nq:nq + nk]
            names = ("yq", "yk")
        else:
            names = ("dq", "dk")
        out = {name: torch.empty(case["T"], n, device=DEVICE, dtype=dt) for name, n in zip(names, (nq, nk))}
    elif op == "page_store":
        n = case["Hk"] * case["D"]
        a["k"], a["v"] = a["kv"][:, :n], a["kv"][:, n:]
        out = {"k_pages": a["k_pages"], "v_pages": a["v_pages"]}
    else:
        # rows behind the last request's stay as they are
        out = {"out": torch.zeros_like(a["q"]), "lse": torch.zeros(a["q"].shape[0], case["Hq"], device=DEVICE)}
    return {"case": case, "in": a, "out": out}


# ---- the plain form: elementary operations in 32 bits, rounded once at the end ------------------------------------


def _plain_plan(case, a, out):
    b, t, page, most, pages = case["B"], case["T"], case["page"], case["max_pages"], a["pages"]
    have = a["have"].long().clamp(0, most * page)
    fresh = a["fresh"].long().clamp(min=0)
    ends = fresh.cumsum(0)
    rows = torch.cat([ends.new_zeros(1), ends]).clamp(max=t)
    lengths = have + rows[1:] - rows[:-1]
    held = (have + page - 1) // page
    need = ((lengths + page - 1) // page).clamp(max=most)
    wanted = (need - held).clamp(min=0)
    first = a["taken"].long() + wanted.cumsum(0) - wanted
    given = torch.minimum(wanted, (a["free"].numel() - first).clamp(min=0))
    col = torch.arange(most, device=DEVICE)[None]
    new = (col >= held[:, None]) & (col < need[:, None])
    at = first[:, None] + col - held[:, None]
    ok = new & (at < a["free"].numel())
    source = a["free"].long()[at.clamp(0, a["free"].numel() - 1)]
    table = torch.where(new, torch.where(ok & (source >= 0) & (source < pages), source, -1), a["table"].long())
    token = torch.arange(t, device=DEVICE)
    seq = torch.searchsorted(rows[1:].contiguous(), token, right=True)
    real = seq < b
    seq = seq.clamp(max=b - 1)
    key = have[seq] + token - rows[seq]
    entry = table[seq, (key // page).clamp(max=most - 1)]
    fits = real & (key < most * page) & (entry >= 0) & (entry < pages)
    placed = torch.minimum((held + given) * page, lengths) - have
    out["counts"][0] = torch.clamp(a["taken"].long()[0] + wanted.sum(), max=a["free"].numel())
    out["counts"][1] = (fresh - placed.clamp(min=0)).sum()
    out["table"].copy_(table)
    out["rows"].copy_(rows)
    out["lengths"].copy_(lengths)
    out["slots"].copy_(torch.where(fits, entry * page + key % page, -1))
    out["positions"].copy_(torch.where(real, key, 0))
    return out


def _turn(case, x, c, s):
    r = case["R"]
    x = x.float().reshape(case["T"], -1, case["D"])
    if case["style"] == "halves":
        p, q = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([p * c - q * s, q * c + p * s], dim=-1)
    else:
        p, q = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([p * c - q * s, q * c + p * s], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., r:]], dim=-1).reshape(case["T"], -1).to(TORCH_DTYPE[case["dtype"]])


def _plain_rotate(case, a):
    angle = a["positions"].double()[:, None] * a["freq"]         # a far position in 32 bits would be off by whole hundredths
    c, s = ((f * a["magnitude"]).float()[:, None] for f in (angle.cos(), angle.sin()))
    if case["op"] == "rotate_forward":
        return {"yq": _turn(case, a["q"], c, s), "yk": _turn(case, a["k"], c, s)}
    return {"dq": _turn(case, a["dyq"], c, -s), "dk": _turn(case, a["dyk"], c, -s)}


def _plain_store(case, a, out):
    keep = a["slots"] >= 0
    slot = a["slots"][keep].long()
    page, row = slot // case["page"], slot % case["page"]
    for pool, x in (("k_pages", a["k"]), ("v_pages", a["v"])):
        out[pool][page, :, row] = x[keep].reshape(-1, case["Hk"], case["D"])
    return out


def _part(score, seen, v):
    """Unnormalised attention over one part of the keys: the rows' largest scores, sums of exponentials and products."""
    score = score.masked_fill_(~seen, float("-inf")) if seen is not None else score
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(score - top)
    return top, p.sum(-1, keepdim=True), torch.matmul(p, v)


def _plain_attention(case, a, out):
    b, hq, hk, d, page = case["B"], case["Hq"], case["Hk"], case["D"], case["page"]
    g, scale = hq // hk, d ** -0.5
    rows, lengths = a["rows"].long(), a["lengths"].long()
    t = a["q"].shape[0] - case["pad"]
    q = a["q"][:t].float().view(t, hk, g, d).mul(scale).transpose(0, 1)                                         # [Hk, T, g, D]
    parts = []
    if case["prefix"]:
        k, v = (pool[a["prefix_table"].long()].float().transpose(0, 1).reshape(hk, -1, d)[:, :case["prefix"]] for pool in (a["k_pages"], a["v_pages"]))
        top, total, o = _part(torch.matmul(q.reshape(hk, t * g, d), k.transpose(1, 2).contiguous()), None, v.contiguous())
        parts.append((top.view(hk, t, g, 1), total.view(hk, t, g, 1), o.view(hk, t, g, d)))
    # the requests' own keys: a padded batch
    n = rows[1:] - rows[:-1]
    most = case["fresh"]
    seq = torch.repeat_interleave(torch.arange(b, device=DEVICE), n, output_size=t)
    step = torch.arange(t, device=DEVICE) - rows[seq]
    padded = q.new_zeros(b, hk, most, g, d)
    padded[seq, :, step] = q.transpose(0, 1)
    table = a["table"].long()
    longest = table.shape[1] * page
    k, v = (pool[table.clamp(min=0)].float().transpose(1, 2).reshape(b, hk, longest, d) for pool in (a["k_pages"], a["v_pages"]))
    score = torch.matmul(padded.reshape(b, hk, most * g, d), k.transpose(2, 3).contiguous()).view(b, hk, most, g, longest)
    last = lengths[:, None] - n[:, None] + torch.arange(most, device=DEVICE)                                  # the last key a row sees
    seen = (torch.arange(longest, device=DEVICE) <= last[..., None])[:, None, :, None]
    v = v.masked_fill(~(torch.arange(longest, device=DEVICE) < lengths[:, None])[:, None, :, None], 0.0)
    score = score.masked_fill_(~seen, float("-inf"))
    top, total, o = _part(score.view(b, hk, most * g, longest), None, v)
    parts.append(tuple(x.view(b, hk, most, g, -1)[seq, :, step].transpose(0, 1) for x in (top, total, o)))
    top = parts[0][0] if len(parts) == 1 else torch.maximum(parts[0][0], parts[1][0])
    total = sum(p[1] * torch.exp(p[0] - top) for p in parts)
    o = sum(p[2] * torch.exp(p[0] - top) for p in parts) / total
    out["out"][:t] = o.transpose(0, 1).reshape(t, hq * d).to(out["out"].dtype)
    out["lse"][:t] = (total.log() + top).transpose(0, 1).reshape(t, hq)
    return out


def _plain(state):
    case, a, out = state["case"], state["in"], state["out"]
    if case["op"] == "page_plan":
        return _plain_plan(case, a, out)
    if case["op"].startswith("rotate"):
        return _plain_rotate(case, a)
    if case["op"] == "page_store":
        return _plain_store(case, a, out)
    return _plain_attention(case, a, out)


# ---- the library's calls ------------------------------------------------------------------------------------------


def _workspace(state, need, *args):
    """The program's scratch, made at its first step and kept."""
    if "workspace" not in state:
        state["workspace"] = torch.empty(max(need(*args), 256), dtype=torch.uint8, device=DEVICE)
    return state["workspace"]


def _own(state):
    from paper_1711_07240_amd import cgbn
    case, a, o = state["case"], state["in"], state["out"]
    op = case["op"]
    if op == "page_plan":
        ws = _workspace(state, cgbn.cgbn_page_plan_workspace_bytes, case["B"], case["T"])
        cgbn.cgbn_page_plan(a["have"], a["fresh"], case["B"], 0, a["free"], a["free"].numel(), a["taken"], o["counts"], o["table"], case["max_pages"],
                            a["pages"], case["page"], case["T"], o["rows"], o["lengths"], o["slots"], o["positions"], ws)
    elif op.startswith("rotate"):
        heads = (case["T"], case["Hq"], case["Hk"], case["D"])
        turn = (case["R"], case["style"], a["positions"], a["freq"], a["magnitude"])
        nq, nk = case["Hq"] * case["D"], case["Hk"] * case["D"]
        if op == "rotate_forward":
            row = a["qkv"].shape[1]
            cgbn.cgbn_rotate_forward(a["q"], row, a["k"], row, *heads, *turn, o["yq"], nq, o["yk"], nk, case["dtype"])
        else:
            cgbn.cgbn_rotate_backward(a["dyq"], nq, a["dyk"], nk, *heads, *turn, o["dq"], nq, o["dk"], nk, case["dtype"])
    elif op == "page_store":
        row = a["kv"].shape[1]
        cgbn.cgbn_page_store(a["k"], row, a["v"], row, case["T"], case["Hk"], case["D"], a["slots"], o["k_pages"], o["v_pages"], a["pages"], case["page"],
                             case["dtype"])
    else:
        t, most = a["q"].shape[0], a["table"].shape[1]
        hq, hk, d = case["Hq"], case["Hk"], case["D"]
        ws = _workspace(state, cgbn.cgbn_prefix_attention_workspace_bytes, t, case["B"], hq, hk, d, case["prefix"], most * case["page"], case["dtype"])
        cgbn.cgbn_prefix_attention(a["q"], hq * d, t, case["B"], None if t == case["B"] else a["rows"], a["lengths"], hq, hk, d, d ** -0.5, a["k_pages"],
                                   a["v_pages"], a["pages"], case["page"], a["prefix_table"], case["prefix"], a["table"], most, o["out"], hq * d, o["lse"],
                                   case["dtype"], ws)
    return o


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------


def _exact_rotate(case, a):
    """The rotation as a product of complex numbers."""
    r, back = case["R"], case["op"] == "rotate_backward"
    angle = a["positions"].double()[:, None] * a["freq"]
    turn = torch.polar(torch.full_like(angle, a["magnitude"]), -angle if back else angle)[:, None]
    nq, nk = case["Hq"] * case["D"], case["Hk"] * case["D"]
    found = {}
    for name, x in (("dq", a["dyq"]), ("dk", a["dyk"])) if back else (("yq", a["qkv"][:, :nq]), ("yk", a["qkv"][:, nq:nq + nk])):
        x = x.double().reshape(case["T"], -1, case["D"])
        head = x[..., :r]
        if case["style"] == "halves":
            z = torch.complex(head[..., :r // 2].contiguous(), head[..., r // 2:].contiguous()) * turn
            head = torch.cat([z.real, z.imag], dim=-1)
        else:
            z = torch.view_as_complex(head.reshape(*head.shape[:-1], r // 2, 2).contiguous()) * turn
            head = torch.view_as_real(z).reshape(*head.shape)
        found[name] = torch.cat([head, x[..., r:]], dim=-1).reshape(case["T"], -1)
    return found


def _exact_attention(case, a):
    hq, hk, d, page = case["Hq"], case["Hk"], case["D"], case["page"]
    g = hq // hk
    fresh, lengths = _lengths(case)

    def keys(pool, table, n):
        return pool[table.long()].double().permute(1, 0, 2, 3).reshape(hk, -1, d)[:, :n]

    shared = [keys(a[pool], a["prefix_table"], case["prefix"]) for pool in ("k_pages", "v_pages")]
    out = torch.zeros(a["q"].shape[0], hq * d, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(a["q"].shape[0], hq, dtype=torch.float64, device=DEVICE)
    at = 0
    for b, (n, length) in enumerate(zip(fresh, lengths)):
        own_pages = a["table"][b, :(length + page - 1) // page]
        k, v = (torch.cat([s, keys(a[pool], own_pages, length)], dim=1) for s, pool in zip(shared, ("k_pages", "v_pages")))
        q = a["q"][at:at + n].double().view(n, hk, g, d).permute(1, 2, 0, 3).reshape(hk, g * n, d)
        score = (torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)).view(hk, g, n, -1)
        later = torch.ones(n, length, dtype=torch.bool, device=DEVICE).triu(length - n + 1)
        score[..., case["prefix"]:].masked_fill_(later, float("-inf"))
        o = torch.matmul(torch.softmax(score, -1).view(hk, g * n, -1), v.contiguous())
        out[at:at + n] = o.view(hk, g, n, d).permute(2, 0, 1, 3).reshape(n, hq * d)
        lse[at:at + n] = torch.logsumexp(score, -1).permute(2, 0, 1).reshape(n, hq)
        at += n
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["op"] == "page_plan":
        return None                                              # whole numbers
    a = _inputs(case, seed)
    if case["op"].startswith("rotate"):
        return _exact_rotate(case, a)
    if case["op"] == "page_store":
        n = case["Hk"] * case["D"]
        at = torch.nonzero(a["slots"] >= 0).flatten()
        slots, found = a["slots"][at].long(), {}
        for pool, x in (("k_pages", a["kv"][:, :n]), ("v_pages", a["kv"][:, n:])):
            rows = a[pool].double().transpose(1, 2).reshape(-1, n)               # a token's row of all heads
            rows.index_copy_(0, slots, x[at].double())
            found[pool] = rows.view(a["pages"], case["page"], case["Hk"], case["D"]).transpose(1, 2).contiguous()
        return found
    return _exact_attention(case, a)


def work(case):
    """Every input read once, every output written once; two operations a multiply-add, and a handful an element beside them."""
    op = case["op"]
    if op == "page_plan":
        t, b = case["T"], case["B"]
        return {"bytes": 8 * b + 8 * b + 8 * t + 8 * (t // case["page"]), "flops": 4 * (b + t)}
    eb, d, hk = (4 if case["dtype"] == "f32" else 2), case["D"], case["Hk"]
    if op.startswith("rotate"):
        rows = case["T"] * (case["Hq"] + hk)
        return {"bytes": eb * 2 * rows * d + 4 * case["T"] + 4 * case["R"], "flops": 3 * rows * case["R"]}
    if op == "page_store":
        stored = case["T"] - case["T"] // 50
        return {"bytes": eb * 4 * stored * hk * d + 4 * case["T"], "flops": 0}
    fresh, lengths = _lengths(case)
    t, hq = sum(fresh), case["Hq"]
    pairs = sum(n * (case["prefix"] + m - n) + n * (n + 1) // 2 for n, m in zip(fresh, lengths))
    return {"bytes": 2 * eb * d * (hk * (case["prefix"] + sum(lengths)) + hq * t) + 4 * hq * t + 4 * (case["prefix"] + sum(lengths)) // case["page"],
            "flops": 4 * d * hq * pairs}
