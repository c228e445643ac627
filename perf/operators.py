"""The serving operators of an int4 model tuned with QZO: what they compute, in plain torch, and calls of the
library's kernels for the same inputs.

  gemv    y = x W for a few rows of x and int4 weights with one scale per 128 rows
  rope    norms of queries and keys for each head, the rotation by the row's position, and the write of keys and
          values into a paged cache, in one pass
  attend  attention of one new token per row over the paged cache
  slots   block tables and slot maps of a step, from the requests' lengths

With own = False, run() computes them from elementary torch operations in 32 bits; with own = True it calls the library.
"""
import math

import torch

own = False

BF16, F8 = "bf16", "e4m3"
TYPES = {BF16: torch.bfloat16, F8: torch.float8_e4m3fn}
GROUP = 128


def listed():
    return [
        # the smallest linear of the tiny configuration, one token: latency
        dict(name="gemv 1x256x688", op="gemv", M=1, K=256, N=688, bias=False),
        # one token through the 7B-shaped model's widest linear
        dict(name="gemv 1x4096x11008", op="gemv", M=1, K=4096, N=11008, bias=False),
        # five sequences through its down projection
        dict(name="gemv 5x11008x4096", op="gemv", M=5, K=11008, N=4096, bias=False),
        # a batch of sixteen through the 13B-shaped model's widest linear, with a bias
        dict(name="gemv 16x5120x13824", op="gemv", M=16, K=5120, N=13824, bias=True),
        # one token of the tiny configuration: latency
        dict(name="rope 1 row", op="rope", T=1, pad=0, H=4, Hkv=4, dh=64, block=16, cache=BF16, norm=False, rotate=True, far=64),
        # a prompt chunk: shared key heads, head norms, an 8-bit cache, positions far out, some padding rows
        dict(name="rope 4099 rows e4m3", op="rope", T=4099, pad=29, H=32, Hkv=8, dh=128, block=32, cache=F8, norm=True, rotate=True, far=131072),
        # one sequence of the 7B-shaped model's length: latency
        dict(name="attend 1 row of 250", op="attend", R=1, pad=0, H=32, Hkv=32, dh=128, block=16, cache=BF16, longest=250, shortest=250),
        # sixteen sequences of the 7B-shaped model, ragged
        dict(name="attend 16 rows to 2048", op="attend", R=16, pad=0, H=32, Hkv=32, dh=128, block=16, cache=BF16, longest=2048, shortest=100),
        # a larger batch over shared key heads and an 8-bit cache, padded to 64 rows
        dict(name="attend 64 rows to 4096 e4m3", op="attend", R=64, pad=3, H=32, Hkv=8, dh=128, block=32, cache=F8, longest=4096, shortest=1),
        # one long document: the cache's length is the only axis to split
        dict(name="attend 1 row of 131071", op="attend", R=1, pad=0, H=32, Hkv=8, dh=128, block=64, cache=BF16, longest=131071, shortest=131071),
        # a decode step of sixteen requests
        dict(name="slots 16 requests", op="slots", B=16, block=16, longest=2048, rows=16, fresh=0.0),
        # a step that takes many new prompts in and lets finished requests go
        dict(name="slots 1024 requests", op="slots", B=1024, block=16, longest=4096, rows=65536, fresh=0.3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("gemv", "rope", "attend", "slots"))
    if op == "gemv":
        return dict(op=op, M=rng.randint(1, 16), K=8 * _log(rng, 8, 1728), N=8 * _log(rng, 1, 640), bias=rng.random() < 0.5)
    if op == "slots":
        B = _log(rng, 1, 1024)
        return dict(op=op, B=B, block=rng.choice((16, 32, 64, 128)), longest=_log(rng, 16, 4096), rows=max(B, _log(rng, 1, 65536)), fresh=rng.choice((0.0, 0.3, 0.8)))
    H, Hkv = rng.choice(((1, 1), (4, 4), (32, 32), (40, 40), (32, 8), (8, 1), (12, 4), (40, 8), (24, 1)))
    dh, block, cache = rng.choice((64, 128)), rng.choice((16, 32, 64, 128)), rng.choice((BF16, F8))
    if op == "rope":
        T = _log(rng, 1, 1500 if H > 32 else 3000)
        return dict(op=op, T=T, pad=rng.randint(0, T // 4), H=H, Hkv=Hkv, dh=dh, block=block, cache=cache, norm=rng.random() < 0.5,
                    rotate=rng.random() < 0.8, far=_log(rng, 64, 131072))
    R = _log(rng, 1, 64)
    longest = _log(rng, 1, 16384)
    while R * longest * Hkv * dh > 64e6:
        longest = (longest + 1) // 2
    return dict(op=op, R=R, pad=rng.randint(0, R // 4), H=H, Hkv=Hkv, dh=dh, block=block, cache=cache, longest=longest,
                shortest=1 if rng.random() < 0.7 else longest)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _randint(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def _cache(g, case, blocks):
    """Key and value pages [block][key head][slot][dimension]; an 8-bit page holds value / scale."""
    shape = (blocks, case["Hkv"], case["block"], case["dh"])
    scales = (0.5, 0.25) if case["cache"] == F8 else (1.0, 1.0)
    return [(_randn(g, *shape) / s).to(TYPES[case["cache"]]) for s in scales], scales


THETA, NORM_EPS = 10000.0, 1e-5


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    st = dict(case)
    if op == "gemv":
        M, K, N = case["M"], case["K"], case["N"]
        st["x"] = _randn(g, M, K).bfloat16()
        # eight 4-bit values of a column to a word, as a checkpoint's interchange layout holds them
        st["words"] = torch.randint(-2 ** 31, 2 ** 31, (K // 8, N), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
        st["scales"] = (torch.rand((-(-K // GROUP), N), generator=g, device="cuda") * 0.015 + 0.005).bfloat16()
        st["b"] = _randn(g, N) if case["bias"] else None
        if own:  # the layout that a program makes once, when it loads its weights
            from paper_2505_13430_b200 import qzo
            st["wq"] = qzo.qzo_repack_int4(st["words"], K, N)
        return st
    if op == "rope":
        T, H, Hkv, dh, block, far = (case[k] for k in ("T", "H", "Hkv", "dh", "block", "far"))
        # queries, keys and values as one projection gives them: views of the rows of one tensor
        qkv = _randn(g, T, (H + 2 * Hkv) * dh).bfloat16()
        st["q"] = qkv[:, :H * dh].view(T, H, dh)
        st["k"] = qkv[:, H * dh:(H + Hkv) * dh].view(T, Hkv, dh)
        st["v"] = qkv[:, (H + Hkv) * dh:].view(T, Hkv, dh)
        blocks = 2 * (-(-T // block)) + 1
        (st["ck"], st["cv"]), st["cs"] = _cache(g, case, blocks)
        st["slots"] = torch.randperm(blocks * block, generator=g, device="cuda")[:T].to(torch.int32)
        st["positions"] = _randint(g, 0, far, T)
        if case["pad"]:  # the padding of a batch stands behind its rows
            st["slots"][T - case["pad"]:] = -1
            st["positions"][T - case["pad"]:] = -1
        st["q_gain"] = 1 + 0.1 * _randn(g, dh) if case["norm"] else None
        st["k_gain"] = 1 + 0.1 * _randn(g, dh) if case["norm"] else None
        st["table"] = None
        if case["rotate"]:
            angle = _angles(torch.arange(far, device="cuda"), dh)
            st["table"] = torch.stack((angle.cos(), angle.sin()), -1).float()
        st["q_out"] = _randn(g, T, H, dh).bfloat16()
        if own:
            from paper_2505_13430_b200 import qzo
            st["cache_of"] = qzo.KvCache(st["ck"], st["cv"], *st["cs"])
        return st
    if op == "attend":
        R, H, Hkv, dh, block = (case[k] for k in ("R", "H", "Hkv", "dh", "block"))
        st["q"] = _randn(g, R, H, dh).bfloat16()
        lens = _randint(g, case["shortest"], case["longest"] + 1, R)
        lens[0] = case["longest"]
        width = -(-case["longest"] // block)
        # pages of a pool that has served for a while: any order, some of them another request's
        blocks = R * width + 7
        (st["ck"], st["cv"]), st["cs"] = _cache(g, case, blocks)
        st["block_table"] = torch.randperm(blocks, generator=g, device="cuda")[:R * width].to(torch.int32).view(R, width).contiguous()
        st["positions"] = lens - 1
        if case["pad"]:
            st["positions"][R - case["pad"]:] = -1
        if own:
            from paper_2505_13430_b200 import qzo
            st["cache_of"] = qzo.KvCache(st["ck"], st["cv"], *st["cs"])
            st["ws"] = torch.empty(qzo.qzo_paged_attention_workspace_bytes(R, H, Hkv, dh, width * block), dtype=torch.uint8, device="cuda")
        return st
    B, block, longest, rows = (case[k] for k in ("B", "block", "longest", "rows"))
    width = -(-(longest + rows) // block)
    lens = _randint(g, 0, longest + 1, B)
    new = torch.ones(B, dtype=torch.int32, device="cuda")
    if case["fresh"]:
        kind = torch.rand(B, generator=g, device="cuda")
        prompts = kind < case["fresh"]
        lens[prompts] = 0
        # what the step's rows leave beside one for every running request goes to the prompts
        most = max(1, 2 * (rows - B) // max(1, int(case["fresh"] * B)))
        long_new = _randint(g, 1, most + 1, B)
        new = torch.where(prompts, long_new, torch.where(kind > 1 - 0.1 * case["fresh"], -1, 1)).to(torch.int32)
        new = torch.where((new > 0) & (new.clamp(min=0).long().cumsum(0) > rows), 0, new.long()).to(torch.int32)
    held = -(-lens.long() // block)
    need = B * (-(-longest // block) + 2) + -(-rows // block)
    ids = torch.randperm(need, generator=g, device="cuda").to(torch.int32)
    # tables as earlier steps left them, and the blocks that are free as a stack
    ends = held.cumsum(0)
    j = torch.arange(width, device="cuda")
    at = (ends - held)[:, None] + j
    st["block_table"] = torch.where(j < held[:, None], ids[at.clamp(max=need - 1)], -1).to(torch.int32).contiguous()
    st["free"] = torch.full((need,), -1, dtype=torch.int32, device="cuda")
    n_free = need - int(ends[-1])
    st["free"][:n_free] = ids[need - n_free:]
    st["n_free"] = torch.tensor([n_free], dtype=torch.int32, device="cuda")
    st["lens"], st["new"] = lens, new
    return st


def _angles(positions, dh):
    """Angle of each position and pair of dimensions, in 64 bits: far positions lose it in 32."""
    i = torch.arange(dh // 2, device="cuda", dtype=torch.float64)
    return positions.double()[:, None] * THETA ** (-i / (dh // 2))


def run(st):
    return {"gemv": _gemv, "rope": _rope, "attend": _attend, "slots": _slots}[st["op"]](st)


def _gemv(st):
    if own:
        from paper_2505_13430_b200 import qzo
        return qzo.qzo_gemv_int4(st["x"], st["wq"], st["scales"], st["K"], st["N"], bias=st["b"])
    K, N = st["K"], st["N"]
    nibble = torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)
    q = ((st["words"][:, None, :] >> nibble[:, None]) & 15).view(K, N) - 8
    w = q.float() * st["scales"].float().repeat_interleave(GROUP, 0)[:K]
    y = st["x"].float() @ w
    return (y if st["b"] is None else y + st["b"]).bfloat16()


def _rope(st):
    if own:
        from paper_2505_13430_b200 import qzo
        q = qzo.qzo_qk_norm_rope_cache(st["q"], st["k"], st["v"], st["positions"], st["slots"], st["cache_of"], q_gain=st["q_gain"],
                                       k_gain=st["k_gain"], norm_eps=NORM_EPS, table=st["table"], q_out=st["q_out"])
        return {"q": q, "keys": st["ck"], "values": st["cv"]}
    live = st["slots"] >= 0
    at = st["slots"].long().clamp(min=0)
    cs = None if st["table"] is None else st["table"][st["positions"].long().clamp(min=0)][:, None]
    q, k = _turned(st["q"].float(), st["q_gain"], cs), _turned(st["k"].float(), st["k_gain"], cs)
    st["q_out"].copy_(torch.where(live[:, None, None], q.bfloat16(), st["q_out"]))
    # rows without a slot are written where the first row goes, with the first row's values
    block = st["block"]
    at = torch.where(live, at, at[0])
    for pages, rows, scale in ((st["ck"], k, st["cs"][0]), (st["cv"], st["v"].float(), st["cs"][1])):
        rows = torch.where(live[:, None, None], rows, rows[:1])
        codes = (rows / scale).clamp(-448, 448) if st["cache"] == F8 else rows
        as_bytes = torch.uint8 if st["cache"] == F8 else torch.int16
        pages.view(as_bytes)[at // block, :, at % block] = codes.to(pages.dtype).view(as_bytes)
    return {"q": st["q_out"], "keys": st["ck"], "values": st["cv"]}


def _turned(x, gain, cs):
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + NORM_EPS) * gain
    if cs is None:
        return x
    a, b = x.chunk(2, -1)
    c, s = cs[..., 0], cs[..., 1]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def _attend(st):
    if own:
        from paper_2505_13430_b200 import qzo
        return qzo.qzo_paged_attention(st["q"], st["cache_of"], st["block_table"], st["positions"], workspace=st["ws"])
    R, H, Hkv, dh, block = (st[k] for k in ("R", "H", "Hkv", "dh", "block"))
    width = st["block_table"].shape[1]
    pages = st["block_table"].long()
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


def _slots(st):
    if own:
        from paper_2505_13430_b200 import qzo
        lens, n_free = torch.empty_like(st["lens"]), torch.empty_like(st["n_free"])
        maps = qzo.qzo_assign_slots(st["lens"], st["new"], st["block_table"], st["free"], st["n_free"], st["block"], st["rows"],
                                    lens_out=lens, free_count_out=n_free)
        return (*maps, lens, n_free, st["block_table"], st["free"])
    block, rows = st["block"], st["rows"]
    table, free, n_free = st["block_table"], st["free"], st["n_free"].long()
    lens, new = st["lens"].long(), st["new"].long()
    gone = new < 0
    add = new.clamp(min=0)
    held = (lens + block - 1) // block
    lens_out = torch.where(gone, 0, lens + add)
    need = torch.where(gone, 0, (lens_out + block - 1) // block - held)
    back = torch.where(gone, held, 0)
    # the stack of free blocks, the blocks of finished requests on top, in their order
    ends = back.cumsum(0)
    i = torch.arange(free.numel(), device="cuda")
    from_free = i < n_free
    r = torch.searchsorted(ends, i - n_free, right=True).clamp(max=len(ends) - 1)
    j = (i - n_free - (ends - back)[r]).clamp(0, table.shape[1] - 1)
    stack = torch.where(from_free, free, torch.where(i < n_free + ends[-1], table[r, j], -1))
    top = n_free + ends[-1]
    free.copy_(torch.where(from_free | (i >= top), free, stack))
    # each request takes what it needs from the top, in order
    first = need.cumsum(0) - need
    col = torch.arange(table.shape[1], device="cuda")
    taken = (top - 1 - (first[:, None] + col - held[:, None])).clamp(0, free.numel() - 1)
    table.copy_(torch.where((col >= held[:, None]) & (col < (held + need)[:, None]), stack[taken], table))
    # one row for each new token
    row_ends = add.cumsum(0)
    t = torch.arange(rows, device="cuda")
    live = t < row_ends[-1]
    seq = torch.searchsorted(row_ends, t, right=True).clamp(max=len(add) - 1)
    pos = lens[seq] + t - (row_ends - add)[seq]
    slot = table[seq, (pos // block).clamp(0, table.shape[1] - 1)].long() * block + pos % block
    maps = [torch.where(live, v, -1).to(torch.int32) for v in (seq, pos, slot)]
    return (*maps, lens_out.to(torch.int32), (top - need.sum()).to(torch.int32), table, free)


def work(case):
    op = case["op"]
    if op == "gemv":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": K * N / 2 + 2 * -(-K // GROUP) * N + 2 * M * (K + N) + (4 * N if case["bias"] else 0), "flops": 2 * M * K * N}
    if op == "slots":
        width = case["rows"] / case["block"] + case["B"]
        return {"bytes": 16 * case["B"] + 12 * case["rows"] + 8 * width, "flops": 10 * case["rows"]}
    size = 1 if case["cache"] == F8 else 2
    H, Hkv, dh = case["H"], case["Hkv"], case["dh"]
    if op == "rope":
        T = case["T"] - case["pad"]
        angles = 4 * dh * T if case["rotate"] else 0
        return {"bytes": T * (2 * H * dh * 2 + 2 * Hkv * dh * (2 + size) + 8) + angles, "flops": T * (H + Hkv) * dh * 8}
    keys = (case["R"] - case["pad"]) * (case["longest"] + case["shortest"]) / 2
    return {"bytes": 2 * keys * Hkv * dh * size + 4 * case["R"] * H * dh, "flops": 4 * keys * H * dh}


def exact(case, seed):
    """The operators' definitions in 64 bits."""
    st = prepare(case, seed)
    if case["op"] == "gemv":
        K, N = case["K"], case["N"]
        y = torch.zeros(case["M"], N, dtype=torch.float64, device="cuda")
        for j in range(8):  # rows j, j + 8, ... of the weights sit in nibble j of the words
            q = ((st["words"].long() >> (4 * j)) & 15) - 8
            k = torch.arange(j, K, 8, device="cuda")
            y += st["x"][:, j::8].double() @ (q.double() * st["scales"][k // GROUP].double())
        return y if st["b"] is None else y + st["b"].double()
    if case["op"] == "rope":
        dh, block, n = case["dh"], case["block"], case["T"] - case["pad"]
        out = {"q": st["q_out"].double(), "keys": st["ck"].double(), "values": st["cv"].double()}
        angle = _angles(st["positions"][:n].long(), dh)[:, None]
        new = {}
        for name in ("q", "k"):
            x = st[name][:n].double()
            if case["norm"]:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / dh + NORM_EPS) * st[name + "_gain"].double()
            if case["rotate"]:
                z = torch.complex(x[..., :dh // 2], x[..., dh // 2:]) * torch.polar(torch.ones_like(angle), angle)
                x = torch.cat((z.real, z.imag), -1)
            new[name] = x
        out["q"][:n] = new["q"]
        slot = st["slots"][:n].long()
        top = 448.0 if case["cache"] == F8 else math.inf
        for h in range(case["Hkv"]):
            out["keys"][slot // block, h, slot % block] = (new["k"][:, h] / st["cs"][0]).clamp(-top, top)
            out["values"][slot // block, h, slot % block] = (st["v"][:n, h].double() / st["cs"][1]).clamp(-top, top)
        return out
    if case["op"] == "attend":
        H, Hkv, dh, block = (case[k] for k in ("H", "Hkv", "dh", "block"))
        out = torch.zeros(case["R"], H, dh, dtype=torch.float64, device="cuda")
        for r, last in enumerate(st["positions"].tolist()):
            if last < 0:
                continue
            t = torch.arange(last + 1, device="cuda")
            page = st["block_table"][r].long()[t // block]
            for h in range(Hkv):
                k = st["ck"][page, h, t % block].double() * st["cs"][0]
                v = st["cv"][page, h, t % block].double() * st["cs"][1]
                mine = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
                out[r, mine] = torch.softmax(st["q"][r, mine].double() @ k.T / dh ** 0.5, -1) @ v
        return out
    return None
