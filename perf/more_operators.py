"""The operators that answer with several continuations of one prompt (beams, samples, the options of a question): what they
compute, in plain torch, and calls of the library's kernels for the same inputs.

  beam     the next beams of every request: the best continuations over its beams and the vocabulary, from the logits
  fork     the requests of a paged cache go on as copies of one another: tables shared, blocks that nobody holds given back, and
           in every layer's pages the last, unfinished block copied for each request that goes on from it beside another
  compact  the blocks that requests hold move to the front of the pool, tables and pages
  prefix   attention of one new token per row over the paged cache, for groups of rows that share the beginning of their cache

With own = False, run() computes them from elementary torch operations in 32 bits (64 for the values that beams are ranked by);
with own = True it calls the library.
"""
import math

import torch

own = False

BF16, F8 = "bf16", "e4m3"
TYPES = {BF16: torch.bfloat16, F8: torch.float8_e4m3fn}


def listed():
    return [
        # one request of the tiny configuration, four beams: latency
        dict(name="beam 1x4 of 1024", op="beam", B=1, W=4, V=1024, pad=0, first=False, done=0.0, power=0.0, banned=0.0),
        # a batch of the 7B-shaped model, four beams each
        dict(name="beam 16x4 of 32000", op="beam", B=16, W=4, V=32000, pad=0, first=False, done=0.1, power=0.0, banned=0.001),
        # a large batch over the larger vocabulary, eight beams, ranked by length, some of them at their end
        dict(name="beam 64x8 of 50272", op="beam", B=64, W=8, V=50272, pad=0, first=False, done=0.2, power=0.7, banned=0.001),
        # one request of the tiny configuration, four beams: latency
        dict(name="fork 1x4 tiny", op="fork", B=1, W=4, layers=2, Hkv=4, dh=64, block=16, longest=40, made=9, gone=0.0),
        # sixteen requests of four beams in layers of the 7B shape: the unfinished blocks are what is copied
        dict(name="fork 16x4, 4 layers", op="fork", B=16, W=4, layers=4, Hkv=32, dh=128, block=16, longest=300, made=24, gone=0.0),
        # many beams with long tables: the bookkeeping
        dict(name="fork 128x8 of 4096", op="fork", B=128, W=8, layers=1, Hkv=1, dh=64, block=16, longest=4000, made=90, gone=0.1),
        # the tiny configuration's pool after some requests left
        dict(name="compact 4 tiny", op="compact", B=4, W=1, layers=2, Hkv=4, dh=64, block=16, longest=60, made=0, spread=2.0),
        # a pool of the 7B shape, half of it free, before memory goes back to training
        dict(name="compact 24, 4 layers", op="compact", B=12, W=2, layers=4, Hkv=32, dh=128, block=16, longest=400, made=20, spread=2.0),
        # four beams of the tiny configuration: latency
        dict(name="prefix 4 rows on 40", op="prefix", R=4, groups=1, pad=0, H=4, Hkv=4, dh=64, block=16, cache=BF16, shared=40, least=40, more=20),
        # sixteen prompts of the 7B-shaped model, four beams each
        dict(name="prefix 64 rows on 16", op="prefix", R=64, groups=16, pad=0, H=32, Hkv=32, dh=128, block=16, cache=BF16, shared=1800, least=200, more=64),
        # answers to one long document in 8-bit pages, a padded batch
        dict(name="prefix 40 rows on 8191 e4m3", op="prefix", R=40, groups=1, pad=3, H=32, Hkv=8, dh=128, block=32, cache=F8, shared=8191, least=8191, more=200),
        # two long documents, many answers, few key heads: the products bind
        dict(name="prefix 128 rows on 2 of 16384", op="prefix", R=128, groups=2, pad=0, H=32, Hkv=4, dh=128, block=64, cache=BF16, shared=16384, least=16000, more=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("beam", "fork", "compact", "prefix"))
    if op == "beam":
        W, V = _log(rng, 1, 16), _log(rng, 100, 50272)
        B = _log(rng, 1, max(1, min(64, int(12e6 / (W * V)))))
        return dict(op=op, B=B, W=W, V=V, pad=rng.choice((0, 0, 3, 16)), first=rng.random() < 0.2, done=rng.choice((0.0, 0.1, 0.5)),
                    power=rng.choice((0.0, 0.0, 0.7, 1.0)), banned=rng.choice((0.0, 0.001, 0.5)))
    if op in ("fork", "compact"):
        Hkv, dh, layers = rng.choice(((1, 64, 3), (4, 64, 2), (8, 128, 5), (32, 128, 2)))
        block = rng.choice((16, 32, 64, 128))
        B, W, longest, made = _log(rng, 1, 64), _log(rng, 1, 8), _log(rng, 1, 2000), _log(rng, 1, 100)
        spread = rng.uniform(1.2, 3.0) if op == "compact" else 1.25
        while layers * 2 * Hkv * dh * block * 2 * spread * (B * (longest / block + 1) + B * W * (made / block + 2)) > 4e8:
            B, longest = (B + 1) // 2, (longest + 1) // 2
            if B == 1 and longest == 1:
                break
        case = dict(op=op, B=B, W=W, layers=layers, Hkv=Hkv, dh=dh, block=block, longest=longest, made=made)
        return dict(case, spread=spread) if op == "compact" else dict(case, gone=rng.choice((0.0, 0.1, 0.5)))
    H, Hkv = rng.choice(((4, 4), (32, 32), (40, 40), (32, 8), (8, 1), (12, 4), (40, 8), (24, 1)))
    groups = _log(rng, 1, 16)
    R = max(groups, _log(rng, 2, 128))
    shared, more = _log(rng, 16, 16384), _log(rng, 1, 300)
    while R * (shared + more) * Hkv * 128 > 4e8 or groups * shared * Hkv * 128 > 2e8 or R * H * (shared + more) > 4e7:
        shared = (shared + 1) // 2
        if shared < 64:
            R, groups, more = (R + 1) // 2, (groups + 1) // 2, (more + 1) // 2
    pad = rng.choice((0, 0, 3))
    return dict(op=op, R=R + pad, groups=groups, pad=pad, H=H, Hkv=Hkv, dh=rng.choice((64, 128)), block=rng.choice((16, 32, 64, 128)),
                cache=rng.choice((BF16, F8)), shared=shared, least=1 if rng.random() < 0.5 else shared, more=more)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _randint(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    return {"beam": _prepare_beam, "fork": _prepare_pool, "compact": _prepare_pool, "prefix": _prepare_prefix}[case["op"]](case, _gen(seed))


END = 2  # the token that ends a beam


def _prepare_beam(case, g):
    st = dict(case)
    B, W, V = case["B"], case["W"], case["V"]
    # logits as a language model gives them: a few tokens far above the rest; some tokens are not allowed
    x = 2.0 * _randn(g, B * W, V)
    x += 6.0 * torch.rand(B * W, V, generator=g, device="cuda").pow(40)
    if case["banned"]:
        x[torch.rand(B * W, V, generator=g, device="cuda") < case["banned"]] = -math.inf
        x[:, 7] = 1.0
    rows = torch.empty(B * W, V + case["pad"], device="cuda")
    rows[:, :V] = x
    st["logits"] = rows[:, :V]
    scores = -20 * torch.rand(B, W, generator=g, device="cuda")
    last = torch.where(torch.rand(B, W, generator=g, device="cuda") < case["done"], END, 5).to(torch.int32)
    lengths = _randint(g, 1, 60, B, W)
    if case["first"]:  # behind the prompt only the first beam is there
        scores[:, 0], scores[:, 1:], last[:], lengths[:] = 0.0, -math.inf, 5, 0
    st["scores"], st["last"], st["lengths"] = scores, last, lengths
    if own:
        from paper_2505_13430_b200 import qzo
        st["ws"] = torch.empty(qzo.qzo_beam_select_workspace_bytes(B, W, V), dtype=torch.uint8, device="cuda")
    return st


def _prepare_pool(case, g):
    """Tables and pages of B requests with W beams each, as earlier steps left them: the blocks that the prompt fills are shared."""
    st = dict(case)
    B, W, block, layers, Hkv, dh = (case[k] for k in ("B", "W", "block", "layers", "Hkv", "dh"))
    prompt = _randint(g, max(1, case["longest"] // 2), case["longest"] + 1, B).long()
    lens = (prompt + case["made"]).repeat_interleave(W)
    common = (prompt // block)
    held = -(-lens // block)
    width = -(-(case["longest"] + case["made"] + 1) // block)
    alone = held - common.repeat_interleave(W)
    n_live = int(common.sum() + alone.sum())
    most = B * (case["longest"] // block) + B * W * (case["made"] // block + 2)
    n_blocks = int(most * case.get("spread", 1.25)) + B * W + 4
    ids = torch.randperm(n_blocks, generator=g, device="cuda").to(torch.int32)
    j = torch.arange(width, device="cuda")
    group = torch.arange(B * W, device="cuda") // W
    at_common = (common.cumsum(0) - common)[group][:, None] + j
    at_alone = common.sum() + (alone.cumsum(0) - alone)[:, None] + j - common[group][:, None]
    at = torch.where(j < common[group][:, None], at_common, at_alone)
    st["table"] = torch.where(j < held[:, None], ids[at.clamp(0, n_blocks - 1)], -1).to(torch.int32).contiguous()
    st["lens"] = lens.to(torch.int32)
    st["n_blocks"] = n_blocks
    st["free"] = torch.full((n_blocks,), -1, dtype=torch.int32, device="cuda")
    st["free"][:n_blocks - n_live] = ids[n_live:]
    st["n_free"] = torch.tensor([n_blocks - n_live], dtype=torch.int32, device="cuda")
    # every layer's keys and values; made in one go, so that a program may look at them as one
    st["pool"] = _randn(g, layers * 2, n_blocks, Hkv, block, dh).bfloat16()
    if case["op"] == "fork":
        best = _randint(g, 0, W, B, W)  # which beams go on: some of them twice, some not at all
        parents = best + W * torch.arange(B, device="cuda", dtype=torch.int32)[:, None]
        over = torch.rand(B, generator=g, device="cuda") < case["gone"]
        st["parents"] = torch.where(over[:, None], -1, parents).to(torch.int32).view(-1).contiguous()
    else:
        st["keep"] = n_live + B * W
    if own:
        from paper_2505_13430_b200 import qzo
        st["caches"] = [qzo.KvCache(st["pool"][2 * i], st["pool"][2 * i + 1]) for i in range(layers)]
        st["table_out"] = torch.empty_like(st["table"])
        st["free_out"], st["n_free_out"] = torch.full_like(st["free"], -1), st["n_free"].clone()
    return st


def _prepare_prefix(case, g):
    st = dict(case)
    R, n, H, Hkv, dh, block = (case[k] for k in ("R", "groups", "H", "Hkv", "dh", "block"))
    live = R - case["pad"]
    st["q"] = _randn(g, R, H, dh).bfloat16()
    bounds = [round(i * live / n) for i in range(n + 1)]
    st["group_rows"] = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    group = torch.searchsorted(st["group_rows"].long(), torch.arange(live, device="cuda"), right=True) - 1
    shared = _randint(g, case["least"], case["shared"] + 1, n)
    shared[0] = case["shared"]
    st["prefix_len"], st["prefix_seq"] = shared, st["group_rows"][:n].clone()
    mine = _randint(g, 1, case["more"] + 1, live)
    lens = shared[group] + mine
    st["positions"] = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    st["positions"][:live] = lens - 1
    # a group's full blocks are its requests' common ones; each request has a copy of the last, unfinished one
    width = -(-(case["shared"] + case["more"]) // block)
    common = (shared // block).long()
    j = torch.arange(width, device="cuda")
    own_most = -(-case["more"] // block) + 1
    first_own = int(common.sum())
    blocks = first_own + live * own_most + 5
    ids = torch.randperm(blocks, generator=g, device="cuda")
    at_common = (common.cumsum(0) - common)[group][:, None] + j
    at_own = first_own + own_most * torch.arange(live, device="cuda")[:, None] + j - common[group][:, None]
    at = torch.where(j < common[group][:, None], at_common, at_own)
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    table[:live] = torch.where(j < -(-lens.long() // block)[:, None], ids[at.clamp(0, blocks - 1)], -1).to(torch.int32)
    st["table"] = table
    st["cs"] = (0.5, 0.25) if case["cache"] == F8 else (1.0, 1.0)
    shape = (blocks, Hkv, block, dh)
    st["ck"], st["cv"] = ((_randn(g, *shape) / s).to(TYPES[case["cache"]]) for s in st["cs"])
    last = table[torch.arange(live, device="cuda"), common[group]].long()  # the block where a row's own tokens begin
    source = last[st["group_rows"][:n].long()][group]
    rest = (shared.long() % block)[group]
    for pages in (st["ck"], st["cv"]):
        raw = pages.view(torch.uint8 if case["cache"] == F8 else torch.int16)
        raw[last] = torch.where((torch.arange(block, device="cuda") < rest[:, None])[:, None, :, None], raw[source], raw[last])
    if own:
        from paper_2505_13430_b200 import qzo
        st["cache_of"] = qzo.KvCache(st["ck"], st["cv"], *st["cs"])
        st["ws"] = torch.empty(qzo.qzo_shared_prefix_attention_workspace_bytes(R, n, H, Hkv, dh, width * block), dtype=torch.uint8, device="cuda")
    return st


def run(st):
    return {"beam": _beam, "fork": _fork, "compact": _compact, "prefix": _prefix}[st["op"]](st)


def _beam(st):
    if own:
        from paper_2505_13430_b200 import qzo
        return qzo.qzo_beam_select(st["logits"], st["scores"], last_tokens=st["last"], end_token=END, lengths=st["lengths"], length_power=st["power"],
                                   workspace=st["ws"])
    B, W, V = st["B"], st["W"], st["V"]
    x = st["logits"].view(B, W, V)
    top = x.amax(-1, keepdim=True)
    norm = top.double() + torch.exp(x - top).double().sum(-1, keepdim=True).log()
    done = (st["last"] == END)[..., None]
    score = st["scores"].double()[..., None]
    value = score + (x.double() - norm)
    token = torch.arange(V, device="cuda")
    value = torch.where(done, torch.where(token == END, score, -math.inf), value)
    length = (st["lengths"][..., None] + torch.where(done, 0, 1)).double()
    rank = value / length ** st["power"]
    at = rank.view(B, W * V).sort(dim=-1, descending=True, stable=True)[1][:, :W]
    best = value.view(B, W * V).gather(1, at)
    some = best > -math.inf
    beam = at // V
    parents = torch.where(some, beam + W * torch.arange(B, device="cuda")[:, None], -1).to(torch.int32)
    tokens = torch.where(some, at % V, -1).to(torch.int32)
    lengths = torch.where(some, length.view(B, W).gather(1, beam), 0).to(torch.int32)
    return parents, tokens, best.float(), lengths


def _move(pool, copies, count, block):
    """pool[:, dst, :, :tokens] = pool[:, src, :, :tokens] for the listed copies; what stands behind them goes where the first does."""
    some = torch.arange(copies.shape[0], device="cuda") < count
    first = torch.where(count > 0, copies[0], 0)
    src, dst, tokens = torch.where(some[:, None], copies, first).long().unbind(1)
    taken = (torch.arange(block, device="cuda") < tokens[:, None])[:, None, :, None]
    pool[:, dst] = torch.where(taken, pool[:, src], pool[:, dst])


def _fork(st):
    if own:
        from paper_2505_13430_b200 import qzo
        table, lens, n_free, copies, count = qzo.qzo_fork_requests(st["lens"], st["parents"], st["table"], st["free"], st["n_free"], st["block"],
                                                                   st["n_blocks"], table_out=st["table_out"])
        qzo.qzo_copy_blocks(st["caches"], copies, count)
        return table, lens, n_free, st["free"], copies, count, st["pool"]
    table, parents, lens, block, n = st["table"], st["parents"].long(), st["lens"].long(), st["block"], st["n_blocks"]
    T, width = table.shape
    r, j = torch.arange(T, device="cuda"), torch.arange(width, device="cuda")
    goes_on = parents >= 0
    parent = parents.clamp(min=0)
    first = torch.full((T + 1,), T, device="cuda").scatter_reduce(0, torch.where(goes_on, parent, T), r, "amin")[:T]
    held = -(-lens // block)
    entries = j < held[:, None]

    def marked(which):
        at = torch.where(entries & which[:, None], table.long(), n)
        return torch.zeros(n + 1, dtype=torch.bool, device="cuda").index_fill(0, at.view(-1), True)[:n]

    # blocks that nobody holds any more go on the stack, the lowest first
    given = marked(first == T) & ~marked(first < T)
    place = torch.where(given, st["n_free"].long() + given.long().cumsum(0) - 1, n)
    stack = torch.cat((st["free"], st["free"][:1])).index_copy(0, place, torch.arange(n, device="cuda", dtype=torch.int32))[:n]
    st["free"].copy_(stack)
    top = st["n_free"].long() + given.sum()
    # the first request that goes on from another keeps its unfinished block, the others take one
    lens_out = torch.where(goes_on, lens[parent], 0)
    held_out = -(-lens_out // block)
    rest = lens_out % block
    takes = goes_on & (rest > 0) & (first[parent] != r)
    order = takes.long().cumsum(0)
    fresh = stack[(top - order).clamp(0, n - 1)]
    old = table[parent, (held_out - 1).clamp(min=0)]
    out = torch.where(j < held_out[:, None], table[parent], -1)
    out = torch.where((j == held_out[:, None] - 1) & takes[:, None], fresh[:, None], out)
    at = torch.where(takes, order - 1, T)
    copies = torch.full((T + 1, 3), -1, dtype=torch.int32, device="cuda").index_copy(0, at, torch.stack((old, fresh, rest.to(torch.int32)), 1))[:T].contiguous()
    count = order[-1:].to(torch.int32)
    _move(st["pool"], copies, count, block)
    return out, lens_out.to(torch.int32), (top - count).to(torch.int32), st["free"], copies, count, st["pool"]


def _compact(st):
    if own:
        from paper_2505_13430_b200 import qzo
        table, n_free, copies, count = qzo.qzo_compact_blocks(st["lens"], st["table"], st["free_out"], st["block"], st["n_blocks"], st["keep"],
                                                              free_count=st["n_free_out"], table_out=st["table_out"])
        qzo.qzo_copy_blocks(st["caches"], copies, count)
        return table, n_free, st["free_out"], copies, count, st["pool"]
    table, block, n, keep = st["table"], st["block"], st["n_blocks"], st["keep"]
    j = torch.arange(table.shape[1], device="cuda")
    entries = j < -(-st["lens"].long() // block)[:, None]
    at = torch.where(entries, table.long(), n)
    live = torch.zeros(n + 1, dtype=torch.bool, device="cuda").index_fill(0, at.view(-1), True)[:n]
    ids = torch.arange(n, device="cuda")
    n_live = live.sum()
    moves, hole = live & (ids >= n_live), ~live & (ids < n_live)
    count = moves.sum()
    src = torch.full((n + 1,), -1, device="cuda").index_copy(0, torch.where(moves, moves.long().cumsum(0) - 1, n), ids)[:n]
    dst = torch.full((n + 1,), -1, device="cuda").index_copy(0, torch.where(hole, hole.long().cumsum(0) - 1, n), ids)[:n]
    to = torch.where(moves, dst[(moves.long().cumsum(0) - 1).clamp(min=0)], ids)
    out = torch.where(entries, to[table.long().clamp(0, n - 1)], -1).to(torch.int32)
    listed_ = ids < count
    copies = torch.where(listed_[:, None], torch.stack((src, dst, torch.full_like(src, block)), 1), -1).to(torch.int32)
    free = torch.where(ids < keep - n_live, keep - 1 - ids, -1).to(torch.int32)
    _move(st["pool"], copies, count, block)
    return out, (keep - n_live).to(torch.int32).view(1), free, copies, count.to(torch.int32).view(1), st["pool"]


def _prefix(st):
    if own:
        from paper_2505_13430_b200 import qzo
        return qzo.qzo_shared_prefix_attention(st["q"], st["cache_of"], st["table"], st["positions"], st["group_rows"], st["prefix_seq"], st["prefix_len"],
                                               workspace=st["ws"])
    R, H, Hkv, dh, block = (st[k] for k in ("R", "H", "Hkv", "dh", "block"))
    width = st["table"].shape[1]
    pages = st["table"].long()
    seen = (torch.arange(width * block, device="cuda") <= st["positions"][:, None])[:, None, :]
    k = (st["ck"][pages].float() * st["cs"][0]).transpose(1, 2).reshape(R, Hkv, width * block, dh)
    q = st["q"].float().view(R, Hkv, H // Hkv, dh)
    s = (q @ k.transpose(2, 3)) / math.sqrt(dh)
    del k
    s = torch.where(seen[:, :, None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    v = (st["cv"][pages].float() * st["cs"][1]).transpose(1, 2).reshape(R, Hkv, width * block, dh)
    v = torch.where(seen[..., None], v, 0.0)
    o = p @ v / torch.where(total == 0, 1.0, total)
    return o.view(R, H, dh).bfloat16()


def work(case):
    op = case["op"]
    if op == "beam":
        rows = case["B"] * case["W"]
        return {"bytes": 4 * rows * case["V"] * (1 - case["done"]) + 28 * rows, "flops": 4 * rows * case["V"]}
    if op == "prefix":
        size = 1 if case["cache"] == F8 else 2
        live, H, Hkv, dh = case["R"] - case["pad"], case["H"], case["Hkv"], case["dh"]
        shared, more = (case["shared"] + case["least"]) / 2, (1 + case["more"]) / 2
        return {"bytes": 2 * Hkv * dh * size * (case["groups"] * shared + live * more) + 4 * case["R"] * H * dh, "flops": 4 * live * (shared + more) * H * dh}
    T, block = case["B"] * case["W"], case["block"]
    held = (0.75 * case["longest"] + case["made"]) / block + 0.5
    token = case["layers"] * 2 * case["Hkv"] * case["dh"] * 2
    if op == "fork":
        # beams that go on from another's unfinished block: W - 1 choices of W are spoken for with this chance
        second = T * (1 - case["gone"]) - case["B"] * (1 - case["gone"]) * case["W"] * (1 - (1 - 1 / case["W"]) ** case["W"])
        return {"bytes": 8 * T * held + 24 * T + 2 * second * token * block / 2, "flops": T * held}
    blocks = case["B"] * 0.75 * case["longest"] / block + T * (case["made"] / block + 1)
    moved = blocks * (1 - 1 / case["spread"])
    return {"bytes": 8 * T * held + 2 * moved * token * block, "flops": T * held}


def exact(case, seed):
    """The operators' definitions in 64 bits."""
    st = prepare(case, seed)
    if case["op"] == "prefix":
        H, Hkv, dh, block = (case[k] for k in ("H", "Hkv", "dh", "block"))
        out = torch.zeros(case["R"], H, dh, dtype=torch.float64, device="cuda")
        for r, last in enumerate(st["positions"].tolist()):
            if last < 0:
                continue
            t = torch.arange(last + 1, device="cuda")
            page = st["table"][r].long()[t // block]
            for h in range(Hkv):
                k = st["ck"][page, h, t % block].double() * st["cs"][0]
                v = st["cv"][page, h, t % block].double() * st["cs"][1]
                mine = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
                out[r, mine] = torch.softmax(st["q"][r, mine].double() @ k.T / dh ** 0.5, -1) @ v
        return out
    if case["op"] != "beam":
        return None
    B, W, V = case["B"], case["W"], case["V"]
    parents = torch.full((B, W), -1, dtype=torch.int32)
    tokens, scores, lengths = parents.clone(), torch.full((B, W), -math.inf, dtype=torch.float64), torch.zeros(B, W, dtype=torch.int32)
    x = torch.log_softmax(st["logits"].double(), -1).view(B, W, V)
    for b in range(B):
        found = []  # (rank, value, beam, token, length) of every beam's best
        for w in range(W):
            score, length = float(st["scores"][b, w]), int(st["lengths"][b, w])
            if int(st["last"][b, w]) == END:
                found.append((score / length ** case["power"], score, w, END, length))
                continue
            if score == -math.inf:
                continue
            y, at = x[b, w].sort(dim=-1, descending=True, stable=True)
            for v, t in zip(y[:W].tolist(), at[:W].tolist()):
                if v > -math.inf:
                    found.append(((score + v) / (length + 1) ** case["power"], score + v, w, t, length + 1))
        found.sort(key=lambda f: (-f[0], f[2], f[3]))
        for i, (_, value, w, t, length) in enumerate(found[:W]):
            parents[b, i], tokens[b, i], scores[b, i], lengths[b, i] = b * W + w, t, value, length
    return parents.cuda(), tokens.cuda(), scores.cuda(), lengths.cuda()
