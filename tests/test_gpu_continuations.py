"""GPU parity of the operators for several continuations of one prompt against the oracle: what is whole is equal, what is computed
is within bounds that count the roundings."""
import math

import numpy as np
import pytest
import torch

from oracle import continuations as oracle, serving
from paper_2505_13430_b200 import inputs

pytestmark = pytest.mark.gpu

BF16_STEP, F16_STEP, F32_STEP = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24
INF = math.inf


@pytest.fixture(scope="module")
def lib():
    from paper_2505_13430_b200 import qzo
    return qzo


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _gen(seed):
    return np.random.default_rng(seed)


# ------------------------------------------------------------------ selection of beams

def _check_beams(lib, logits, scores, rows=None, last=None, end_token=-1, lengths=None, power=0.0, reported=0, **kw):
    """logits: CUDA tensor or view; the rest numpy."""
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = lib.qzo_beam_select(logits, dev(scores), rows=dev(rows), last_tokens=dev(last), end_token=end_token, lengths=dev(lengths),
                              length_power=power, status=status, **kw)
    parents, tokens, out, out_lengths = (None if t is None else t.cpu().numpy() for t in got)
    want = oracle.beam_select(logits.cpu().numpy(), scores, rows, last, end_token, lengths, power)
    size = float(np.abs(np.where(np.isfinite(scores), scores, 0)).max()) + 100.0
    for b, best in enumerate(want):
        assert parents[b].tolist() == [f[0] for f in best] and tokens[b].tolist() == [f[1] for f in best], (b, best)
        if lengths is not None:
            assert out_lengths[b].tolist() == [f[3] for f in best]
        for w, f in enumerate(best):
            # rounded once (score + logit - norm); the norm's exponentials are off by 2^-22 each, their products with log2 e by 2^-23
            # of an exponent below 150 that counts for e^-100 then, their sums by 2^-24 for each of at most 256 + 14 terms
            assert out[b, w] == f[2] or abs(out[b, w] - f[2]) <= F32_STEP * abs(f[2]) + (2 ** -22 + 2 ** -22 + 270 * F32_STEP), (b, w, out[b, w], f[2])
    assert int(status) == reported
    return got


def _logits(rng, rows, V, pad=0, scale=2.0):
    x = torch.from_numpy((rng.standard_normal((rows, V + pad)) * scale).astype(np.float32)).cuda()
    return x[:, :V]


@pytest.mark.parametrize("B,W,V,pad", [(1, 1, 1, 0), (1, 1, 5, 3), (2, 4, 3, 0), (1, 4, 1024, 0), (3, 5, 1000, 1), (2, 32, 4097, 0), (1, 32, 50, 2), (5, 7, 8195, 1),
                                       (16, 4, 32000, 0), (1, 8, 50272, 0), (40, 3, 2049, 7), (1, 2, 262144, 0), (70, 16, 999, 1)])
def test_beams_follow_the_oracle(lib, B, W, V, pad):
    rng = _gen(B * W + V)
    scores = (-20 * rng.random((B, W))).astype(np.float32)
    got = _check_beams(lib, _logits(rng, B * W, V, pad), scores)
    assert got[3] is None


@pytest.mark.parametrize("power", [0.0, 0.7, 1.0, 8.0])
def test_ended_beams_lengths_and_missing_ones(lib, power):
    rng = _gen(int(10 * power))
    B, W, V = 9, 6, 3001
    scores = (-5 * rng.random((B, W))).astype(np.float32)
    last = np.where(rng.random((B, W)) < 0.4, 2, 7).astype(np.int32)
    lengths = rng.integers(0, 30, (B, W)).astype(np.int32)
    scores[1, 1:] = -INF                                # behind a prompt only the first beam is there
    last[1] = 7
    scores[2] = -INF                                    # nothing at all
    last[3] = 2                                         # every beam has ended: they come out in order
    rows = rng.permutation(B * W + 5)[:B * W].astype(np.int32).reshape(B, W)
    rows[4, 2:] = -1                                    # beams without logits
    x = _logits(rng, B * W + 5, V, 3)
    x[rows[5, 0], 5:] = -INF                            # five tokens allowed
    x[rows[6]] = -INF                                   # none
    _check_beams(lib, x, scores, rows=rows, last=last, end_token=2, lengths=lengths, power=power)


def test_equal_candidates_go_to_the_lowest_beam_and_token(lib):
    B, W, V = 2, 4, 9000
    x = torch.zeros(B * W, V, device="cuda")
    x[4:, 17] = 1.0
    x[4:, 8999] = 1.0
    x[5, 3] = -0.0
    scores = np.zeros((B, W), np.float32)
    parents, tokens, _, _ = _check_beams(lib, x, scores)
    assert parents[0].tolist() == [0] * 4 and tokens[0].tolist() == [0, 1, 2, 3]
    assert parents[1].tolist() == [4, 4, 5, 5] and tokens[1].tolist() == [17, 8999] * 2
    x = torch.full((1, 100), -1.0, device="cuda")       # zeros of either sign are one value
    x[0, 40], x[0, 60], x[0, 50] = -0.0, 0.0, 0.0
    _check_beams(lib, x.repeat(3, 1), np.array([[0.0, -INF, -INF]], np.float32))


def test_logits_and_scores_out_of_range_are_reported(lib):
    rng = _gen(3)
    B, W, V = 3, 2, 5000
    scores = -rng.random((B, W)).astype(np.float32)
    for where, value in ((4999, float("nan")), (0, INF)):
        x = _logits(rng, B * W, V)
        x[2, where] = value
        x[3] = value
        _check_beams(lib, x, scores, reported=2)
    x = _logits(rng, B * W, V)
    bad = scores.copy()
    bad[1] = float("nan"), INF
    _check_beams(lib, x, bad, reported=2)
    rows = np.arange(B * W, dtype=np.int32).reshape(B, W)
    rows[2, 1] = B * W
    _check_beams(lib, x, scores, rows=rows, reported=2)


def test_large_and_small_logits(lib):
    # sums far apart, logits of 1e30, a row whose chunks differ by more than fp32's exponent range
    rng = _gen(4)
    x = _logits(rng, 4, 6000)
    x[0] *= 1e29
    x[1, :4000] -= 1e4
    x[2] = 3.0e38
    x[2, 77] = 3.4e38
    x[3] = -3.0e38
    x[3, 5500] = -2.9e38
    _check_beams(lib, x, np.array([[0.0], [-1.0], [-2.0], [-3.0]], np.float32))


def test_zeros_of_either_sign_are_one_rank(lib):
    scores = np.array([[-0.0, 0.0, -1.0], [0.0, -0.0, -0.0]], np.float32)
    _check_beams(lib, torch.zeros((6, 8), device="cuda"), scores, last=np.full((2, 3), 5, np.int32), end_token=5)


@pytest.mark.parametrize("size", [0.0, 1e9, 1e15])
@pytest.mark.parametrize("power", [0.0, 0.7])
def test_candidates_whose_ranks_round_to_one(lib, size, power):
    # logits next to zero, and scores so low that logits vanish beside them: a beam's candidates go by their logits all the same, beams of one rank by their number
    W, V = 4, 5000
    x = torch.full((2 * W, V), -1.0, device="cuda")
    x[:, [10, 20, 30, 40, 4900]] = torch.tensor([0.0, 1e-18, 2e-18, 2e-18, 4e-18], device="cuda")
    x[W:, [7, 4000, 3000]] = torch.tensor([0.01, 0.02, 0.03], device="cuda")
    scores = np.full((2, W), -INF, np.float32)
    scores[0, 1] = scores[1, 2] = scores[1, 3] = -size
    lengths = np.full((2, W), 5, np.int32)
    _check_beams(lib, x, scores, lengths=lengths, power=power)
    rows = np.zeros((2, W), np.int32)                    # beams of one row and one score: the first has all places
    _check_beams(lib, x, np.full((2, W), -size, np.float32), rows=rows, lengths=lengths, power=power)


def test_beams_in_place(lib):
    rng = _gen(5)
    B, W, V = 3, 4, 2000
    x = _logits(rng, B * W, V)
    scores = torch.from_numpy(-rng.random((B, W)).astype(np.float32)).cuda()
    last, lengths = ints(rng.integers(0, 3, (B, W)).tolist()), ints(rng.integers(1, 9, (B, W)).tolist())
    want = lib.qzo_beam_select(x, scores, last_tokens=last, end_token=2, lengths=lengths, length_power=0.5)
    got = lib.qzo_beam_select(x, scores, last_tokens=last, end_token=2, lengths=lengths, length_power=0.5, tokens=last, scores_out=scores, lengths_out=lengths)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert got[1] is last and got[2] is scores and got[3] is lengths


# ------------------------------------------------------------------ forked requests

def _pool_state(rng, B, block, longest, n_blocks, spare=0):
    """Lengths, a table of blocks in any order, the stack of free ones."""
    lens = rng.integers(0, longest + 1, B)
    width = -(-longest // block) + spare
    held = -(-lens // block)
    ids = rng.permutation(n_blocks)
    assert held.sum() <= n_blocks
    table = np.full((B, max(1, width)), -9, np.int32)
    at = 0
    for r in range(B):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    free = np.full(n_blocks, -7, np.int32)
    free[:n_blocks - at] = ids[at:]
    return lens.astype(np.int32), table, free, n_blocks - at


def _fork(lib, lens, parents, table, free, count, block, n_blocks, in_place=False, want_served=True):
    """Runs the call, compares with the oracle, returns the new state in numpy."""
    d_lens, d_free, d_count, status = ints(lens.tolist()), ints(free.tolist()), ints([count]), ints([0])
    kw = dict(lens_out=d_lens, free_count_out=d_count) if in_place else {}
    table_out, lens_out, count_out, copies, n = lib.qzo_fork_requests(d_lens, ints(parents.tolist()), torch.from_numpy(table).cuda(), d_free, d_count, block,
                                                                      n_blocks, status=status, **kw)
    want = oracle.fork_requests(lens, parents, table, free, count, block, n_blocks)
    assert (want is not None) == want_served
    if want is None:
        assert int(status) == 4 and int(n) == 0 and (copies == -1).all() and int(count_out) == count
        assert np.array_equal(lens_out.cpu(), lens) and np.array_equal(table_out.cpu(), table) and np.array_equal(d_free.cpu(), free)
        return None
    assert int(status) == 0 and int(n) == len(want["copies"]) and int(count_out) == want["free_count"]
    assert [tuple(c) for c in copies.tolist()] == want["copies"] + [(-1, -1, -1)] * (len(lens) - len(want["copies"]))
    assert lens_out.tolist() == want["lens"]
    assert np.array_equal(table_out.cpu(), want["table"]) and np.array_equal(d_free.cpu(), want["free"])
    return np.array(want["lens"], np.int32), want["table"], want["free"], want["free_count"], want["copies"]


@pytest.mark.parametrize("B,block,longest,n_blocks,in_place", [(1, 16, 40, 7, False), (4, 16, 70, 40, True), (33, 32, 300, 500, False), (200, 16, 400, 9000, True),
                                                               (4096, 64, 500, 40000, False), (3, 256, 9000, 524288, False), (40, 16, 3000, 9001, True)])
def test_forks_follow_the_oracle_step_after_step(lib, B, block, longest, n_blocks, in_place):
    rng = _gen(B + block)
    lens, table, free, count = _pool_state(rng, B, block, longest, n_blocks, spare=2)
    for step in range(4):
        # within groups of up to four, as beams are, and now and then from anywhere, some ending
        parents = np.minimum(np.arange(B) // 4 * 4 + rng.integers(0, 4, B), B - 1)
        parents = np.where(rng.random(B) < 0.2, rng.integers(0, B, B), parents)
        parents = np.where(rng.random(B) < 0.15, -1, parents).astype(np.int32)
        lens, table, free, count, _ = _fork(lib, lens, parents, table, free, count, block, n_blocks, in_place)
        table[table < 0] = -9                           # what stands behind a request's blocks means nothing
        grown = [r for r in range(B) if lens[r] % block]        # a token more in the blocks that are not full
        lens[grown] += 1


def test_forks_that_cannot_be_served(lib):
    lens, table = np.array([20, 16, 5], np.int32), np.array([[3, 1], [0, -1], [2, -1]], np.int32)
    free = np.array([5, 4, -1, -1, -1, -1], np.int32)
    ok = np.array([0, 0, 0], np.int32)
    _fork(lib, lens, ok, table, free, 2, 16, 6)
    _fork(lib, lens, np.array([0, 0, 2], np.int32), table, free, 0, 16, 6)             # the block that request 1 leaves is enough
    _fork(lib, lens, np.array([0, 1, 0], np.int32), table, free, 0, 16, 6)
    for change in (dict(parents=np.array([0, 0, 3], np.int32)), dict(lens=np.array([20, -1, 5], np.int32)), dict(lens=np.array([33, 16, 5], np.int32)),
                   dict(table=np.array([[3, 6], [0, -1], [2, -1]], np.int32)), dict(table=np.array([[3, -1], [0, -1], [2, -1]], np.int32)),
                   dict(free=np.array([5, 4], np.int32)), dict(count=-1)):
        args = dict(lens=lens, parents=ok, table=table, free=free, count=2)
        args.update(change)
        for in_place in (False, True):
            _fork(lib, block=16, n_blocks=6, in_place=in_place, want_served=False, **args)
    # too few blocks: all three go on from one with an unfinished block, nothing is free and nobody leaves any
    lens, table = np.array([20, 0, 0], np.int32), np.array([[3, 1], [0, -1], [2, -1]], np.int32)
    _fork(lib, lens, ok, table, free, 1, 16, 6, want_served=False)
    _fork(lib, lens, ok, table, free, 2, 16, 6)


# ------------------------------------------------------------------ compaction

@pytest.mark.parametrize("B,block,longest,n_blocks", [(1, 16, 40, 30), (5, 16, 200, 100), (300, 32, 400, 20000), (64, 16, 2000, 524288), (7, 256, 3000, 97), (1, 16, 1, 1)])
def test_compaction_follows_the_oracle(lib, B, block, longest, n_blocks):
    rng = _gen(B + n_blocks)
    lens, table, _, count = _pool_state(rng, B, block, longest, n_blocks, spare=1)
    if B > 2:                                           # two requests share their first blocks
        a, b = np.argsort(lens)[-2:]
        table[b, :lens[a] // block] = table[a, :lens[a] // block]
    held = len({int(v) for r in range(B) for v in table[r, :-(-lens[r] // block)]})
    for keep in {max(1, held), max(1, (held + n_blocks) // 2), n_blocks}:
        want = oracle.compact_blocks(lens, table, block, n_blocks, keep)
        for in_place in (False, True):
            d_table, free, n_free, status = torch.from_numpy(table.copy()).cuda(), torch.full((n_blocks,), -7, dtype=torch.int32, device="cuda"), ints([-3]), ints([0])
            out, n_free, copies, n = lib.qzo_compact_blocks(ints(lens.tolist()), d_table, free, block, n_blocks, keep, free_count=n_free,
                                                            table_out=d_table if in_place else torch.empty_like(d_table), status=status)
            assert int(status) == 0 and int(n) == len(want[2]) and int(n_free) == len(want[1]) == keep - held
            assert np.array_equal(out.cpu(), want[0])
            assert free.tolist() == want[1] + [-7] * (n_blocks - len(want[1]))
            assert [tuple(c) for c in copies[:int(n)].tolist()] == want[2] and (copies[int(n):] == -1).all()


@pytest.mark.parametrize("B,block,longest,n_blocks", [(1, 16, 40, 16383), (2, 16, 100, 16384), (5, 32, 200, 131072), (3, 16, 300, 524288), (1, 16, 1, 524288)])
def test_few_requests_in_a_large_pool(lib, B, block, longest, n_blocks):
    # how many CTAs take a call goes by the pool too
    test_compaction_follows_the_oracle(lib, B, block, longest, n_blocks)
    test_forks_follow_the_oracle_step_after_step(lib, B, block, longest, n_blocks, False)


def test_compactions_that_cannot_be_done(lib):
    lens, table = np.array([20, 16, 5], np.int32), np.array([[13, 1], [0, -1], [9, -1]], np.int32)
    good = dict(lens=lens, table=table, keep=5, room=5, most=20)
    for change, served in ((dict(), True), (dict(keep=4), True), (dict(keep=3), False), (dict(keep=10, room=5), False), (dict(keep=9), True), (dict(most=2), True),
                           (dict(most=1), False), (dict(lens=np.array([20, -16, 5], np.int32)), False), (dict(lens=np.array([33, 16, 5], np.int32)), False),
                           (dict(table=np.array([[20, 1], [0, -1], [9, -1]], np.int32)), False), (dict(table=np.array([[-1, 1], [0, -1], [9, -1]], np.int32)), False)):
        a = dict(good, **change)
        d_table, free, n_free, status = torch.from_numpy(a["table"]).cuda(), torch.full((a["room"],), -7, dtype=torch.int32, device="cuda"), ints([-3]), ints([0])
        out, n_free, copies, n = lib.qzo_compact_blocks(ints(a["lens"].tolist()), d_table, free, 16, 20, a["keep"], free_count=n_free, table_out=torch.empty_like(d_table),
                                                        copies=torch.empty((a["most"], 3), dtype=torch.int32, device="cuda"), status=status)
        assert int(status) == (0 if served else 4)
        if served:
            assert int(n) == 2 and copies[:2].tolist() == [[9, 2, 16], [13, 3, 16]] and int(n_free) == a["keep"] - 4
        else:
            assert int(n) == 0 and (copies == -1).all() and int(n_free) == -3 and (free == -7).all() and torch.equal(out, d_table)


# ------------------------------------------------------------------ copies of pages

@pytest.mark.parametrize("layers,heads,block,dh,dtype", [(1, 1, 16, 64, torch.float8_e4m3fn), (3, 5, 32, 64, torch.bfloat16), (2, 32, 16, 128, torch.bfloat16),
                                                         (130, 2, 16, 64, torch.bfloat16), (2, 3, 256, 128, torch.float8_e4m3fn)])
def test_copies_move_the_listed_tokens_and_nothing_else(lib, layers, heads, block, dh, dtype):
    rng = _gen(layers + heads)
    n_blocks = 41
    raw = torch.from_numpy(rng.integers(0, 256, (layers, 2, n_blocks, heads, block, dh * dtype.itemsize), dtype=np.uint8)).cuda()
    caches = [lib.KvCache(raw[i, 0].view(dtype), raw[i, 1].view(dtype)) for i in range(layers)]
    ids = rng.permutation(n_blocks)
    copies = [(int(ids[i % 7]), int(ids[7 + i]), int(rng.integers(0, block + 1))) for i in range(30)]
    copies[3] = (copies[3][0], copies[3][1], block)
    copies[4] = (copies[4][0], copies[4][1], 1)
    want = raw.cpu().numpy()
    for page in want.reshape(-1, n_blocks, heads, block, dh * dtype.itemsize):
        oracle.copy_blocks(page, copies[:25])
    status = ints([0])
    lib.qzo_copy_blocks(caches, ints(copies), ints([25]), status=status)
    assert np.array_equal(raw.cpu().numpy(), want) and int(status) == 0
    for count in (0, -5):
        lib.qzo_copy_blocks(caches, ints(copies), ints([count]))
    assert np.array_equal(raw.cpu().numpy(), want)
    # what is out of range is left out and reported, the rest is copied; a count beyond the list ends with it
    bad = [(n_blocks, copies[25][1], 2), (copies[25][0], -1, 2), (copies[25][0], copies[25][1], block + 1), (copies[26][0], copies[26][1], -1), copies[27]]
    lib.qzo_copy_blocks(caches, ints(bad), ints([1000]), status=status)
    for page in want.reshape(-1, n_blocks, heads, block, dh * dtype.itemsize):
        oracle.copy_blocks(page, bad[4:])
    assert np.array_equal(raw.cpu().numpy(), want) and int(status) == 2


def test_copies_beyond_32_bit_offsets(lib):
    heads, block, dh = 8, 64, 128
    n_blocks = (1 << 32) // (heads * block * dh * 2) + 9          # 4 GB and a little of keys
    k, v = (torch.zeros((n_blocks, heads, block, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[3], v[n_blocks - 2] = 1.5, 2.5
    lib.qzo_copy_blocks([lib.KvCache(k, v)], ints([(3, n_blocks - 1, 40), (n_blocks - 2, 5, 64)]), ints([2]))
    assert (k[n_blocks - 1, :, :40] == 1.5).all() and (k[n_blocks - 1, :, 40:] == 0).all() and (v[5] == 2.5).all() and (v[n_blocks - 1] == 0).all() and (k[5] == 0).all()


# ------------------------------------------------------------------ attention over shared beginnings

# how prefixes are taken: by the rows through their own tables, in units of few queries, in units of 128
@pytest.fixture(params=[1, 2, 3], ids=["own-tables", "few", "many"])
def path(request, lib):
    lib.qzo_debug_prefix_path(request.param)
    yield request.param
    lib.qzo_debug_prefix_path(0)


@pytest.fixture(params=[2, 3], ids=["few", "many"])
def units(request, lib):
    lib.qzo_debug_prefix_path(request.param)
    yield request.param
    lib.qzo_debug_prefix_path(0)


CACHES = {"bf16": (torch.bfloat16, 1.0, 1.0), "e4m3": (torch.float8_e4m3fn, 0.25, 0.5)}


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Shared:
    """Rows of groups whose requests share the beginning of their cache.  groups: (rows, prefix, what each row has beyond it, a number or a
    list; None = padding, negative = the row sees that much less than the prefix).  Requests 0 .. n - 1 hold the prefixes and do nothing
    else, request n + t is row t's.  Full blocks of a prefix are shared, the rest of it is copied."""

    def __init__(self, groups, H, Hkv, dh, block, kind, seed, q_std=1.0, loose=0):
        rng = _gen(seed)
        dt, self.ks, self.vs = CACHES[kind]
        n = len(groups)
        own = [(i, o) for i, (rows, _, more) in enumerate(groups) for o in (more if isinstance(more, list) else [more] * rows)]
        own += [(None, o) for o in rng.integers(1, 200, loose)]
        bounds = np.cumsum([0] + [g[0] for g in groups])
        self.R, self.H, self.block, self.dh = len(own), H, block, dh
        assert bounds[-1] + loose == self.R
        self.lens = [0 if o is None else (groups[i][1] if i is not None else 0) + int(o) for i, o in own]
        self.prefix = [g[1] for g in groups]
        width = max(1, -(-max(self.lens + self.prefix) // block))
        count = lambda tokens: -(-tokens // block)
        need = sum(count(p) for p in self.prefix) + sum(count(v) for v in self.lens)
        n_blocks = need + 3
        shape = (n_blocks, Hkv, block, dh)
        self.ck, self.cv = (inputs.normal_fp32(shape, 1.0, seed + i).numpy() / s for i, s in enumerate((self.ks, self.vs)))
        ids = iter(rng.permutation(n_blocks).tolist())
        table = np.full((n + self.R, width), -1, np.int32)
        for i, p in enumerate(self.prefix):
            table[i, :count(p)] = [next(ids) for _ in range(count(p))]
        for t, (i, o) in enumerate(own):
            p = 0 if i is None else self.prefix[i]
            whole, rest = min(p, self.lens[t]) // block, p % block
            table[n + t, :whole] = table[i, :whole] if i is not None else []
            table[n + t, whole:count(self.lens[t])] = [next(ids) for _ in range(count(self.lens[t]) - whole)]
            if i is not None and self.lens[t] > whole * block and whole < count(p):
                n_copied = rest if whole == p // block else block
                for pages in (self.ck, self.cv):
                    pages[table[n + t, whole], :, :n_copied] = pages[table[i, whole], :, :n_copied]
        # nothing behind a request's length is looked at
        for r, length in enumerate(self.prefix + self.lens):
            if length % block:
                for pages in (self.ck, self.cv):
                    pages[table[r, length // block], :, length % block:] = float("nan")
        self.ck, self.cv = (torch.from_numpy(v).to(dt).cuda() for v in (self.ck, self.cv))
        self.q = inputs.normal_fp32((self.R, H, dh), q_std, seed + 5).bfloat16()
        self.table, self.seqs = table, np.arange(n, n + self.R)
        self.positions = [v - 1 for v in self.lens]
        self.rows = bounds.tolist()
        self.kind, self.scale = kind, dh ** -0.5

    def run(self, lib, reported=0, **change):
        a = dict(rows=self.rows, prefix=self.prefix, seq=list(range(len(self.prefix))))
        a.update(change)
        status = ints([0])
        out = lib.qzo_shared_prefix_attention(self.q.cuda(), lib.KvCache(self.ck, self.cv, self.ks, self.vs), torch.from_numpy(self.table).cuda(),
                                              ints(self.positions), ints(a["rows"]), ints(a["seq"]), ints(a["prefix"]), row_seq=ints(self.seqs.tolist()),
                                              scale=self.scale, status=status)
        assert int(status) == reported
        return out

    def check(self, out, only=None):
        kp, vp = f64(self.ck) * self.ks, f64(self.cv) * self.vs
        want, spread = serving.paged_attention(f64(self.q), kp, vp, self.table, self.seqs, self.positions, self.scale)
        kmax = np.nanmax(np.abs(kp[np.unique(self.table[self.table >= 0])])) if (self.table >= 0).any() else 0.0
        # score: dh exact products summed in fp32 (truncated at worst), one scaling; weight: exp2 within 4 steps, and as it enters the product:
        # the sum of two bf16 (2^-15), or of one fp16 (2^-11) where a row's own keys are 8-bit; the sums: two additions for every 16 keys
        score = np.abs(f64(self.q)).sum(-1, keepdims=True) * kmax * self.scale * (self.dh / 16 + 18) * 2 * F32_STEP
        p_step = 2.0 ** -15 if self.kind == "bf16" else F16_STEP
        keys = max(self.lens) + 1
        allowed = BF16_STEP * np.abs(want) + (p_step + 2 * score + (16 + keys / 4) * F32_STEP) * spread * (1 + BF16_STEP) + 1e-30
        off = np.abs(f64(out) - want)
        rows = range(self.R) if only is None else only
        assert all((off[r] <= allowed[r]).all() for r in rows), [(off / allowed)[r].max() for r in rows]
        for r in rows:
            if self.positions[r] < 0:
                assert (out[r] == 0).all()


SHARED_CASES = [
    # groups, H, Hkv, dh, block, cache, rows without a group
    ([(4, 40, [1, 5, 20, 7])], 4, 4, 64, 16, "bf16", 0),            # shorter than a tile: nothing is shared
    ([(4, 64, 1)], 4, 4, 64, 16, "bf16", 0),
    ([(1, 130, 3)], 1, 1, 128, 16, "bf16", 0),
    ([(3, 1000, [24, 1, 300])], 2, 2, 128, 16, "bf16", 2),
    ([(5, 999, [None, 1, 0, -1, 50]), (0, 500, 1), (2, 64, 0), (1, 63, 9)], 8, 2, 64, 32, "bf16", 3),
    ([(33, 700, 17)], 12, 3, 128, 64, "bf16", 0),                   # 132 queries of a key head: a tile of 128 and one of 4
    ([(20, 500, 33), (3, 2000, 1), (16, 64, 5)], 24, 1, 64, 128, "bf16", 1),
    ([(2, 300, 70)], 71, 1, 128, 16, "bf16", 0),
    ([(4, 9000, [1, 70, 200, 64])], 8, 2, 128, 256, "bf16", 0),
    ([(70, 2048, 1)], 8, 2, 128, 16, "bf16", 5),
    ([(4, 200, [1, 5, 20, 7])], 4, 4, 64, 16, "e4m3", 0),
    ([(6, 1000, [24, None, 1, 300, -900, 2]), (9, 321, 3)], 8, 2, 128, 32, "e4m3", 2),
    ([(40, 600, 30)], 16, 4, 64, 64, "e4m3", 0),
    ([(3, 6000, 257)], 4, 1, 128, 256, "e4m3", 0),
    ([(2, 130 + 7 * i, i) for i in range(70)], 2, 2, 64, 16, "bf16", 4),        # more groups than a warp has lanes
]


@pytest.mark.parametrize("groups,H,Hkv,dh,block,kind,loose", SHARED_CASES)
def test_shared_prefix_attention_matches_oracle(lib, path, groups, H, Hkv, dh, block, kind, loose):
    case = Shared(groups, H, Hkv, dh, block, kind, 300 + H + dh, loose=loose)
    out = case.run(lib)
    case.check(out)
    assert torch.equal(out.view(torch.int16), case.run(lib).view(torch.int16))


@pytest.mark.parametrize("kind,dh", [("bf16", 64), ("bf16", 128), ("e4m3", 64), ("e4m3", 128)])
@pytest.mark.parametrize("rising", [False, True])
def test_long_runs_of_tiles(lib, units, kind, dh, rising):
    # so many groups that a prefix is not split: dozens of tiles one after the other, two CTAs on an SM.  Rising: scores that pass the
    # running maximum again and again, so that the sums are rescaled between products; some rows fall instead
    case = Shared([(2, 450 + 13 * i, 1 + 3 * i) for i in range(40)], 8, 8, dh, 32, kind, 900 + dh)
    if rising:
        case.q[:, :, 0] = torch.tensor([60.0, -60.0, 0.0, 30.0]).repeat(20)[:, None].bfloat16()
        for r, length in enumerate(case.prefix + case.lens):
            j = np.arange(length)
            page = torch.from_numpy(case.table[r][j // case.block].astype(np.int64)).cuda()
            case.ck[page, :, torch.from_numpy(j % case.block).cuda(), 0] = torch.from_numpy((j // 64 * 0.75).astype(np.float32)).cuda()[:, None].to(case.ck.dtype)
    out = case.run(lib)
    case.check(out)
    for _ in range(20):
        assert torch.equal(out.view(torch.int16), case.run(lib).view(torch.int16))


@pytest.mark.parametrize("dh", [64, 128])
def test_every_code_of_8_bit_pages(lib, units, dh):
    # a dimension has one code in all keys, so that a row's result is that code's value: the weights' roundings leave less than half a bf16 step of it
    for first in range(0, 256, dh):
        case = Shared([(5, 200, [1, 3, 60, 7, 1])], 8, 4, dh, 16, "e4m3", 39)
        codes = torch.arange(first, first + dh, dtype=torch.uint8)
        case.cv.view(torch.uint8)[:] = codes.cuda()
        out = case.run(lib)
        want = codes.view(torch.float8_e4m3fn).float() * case.vs
        assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want).expand(out.shape))
        assert torch.equal(torch.nan_to_num(out.cpu().float()), torch.nan_to_num(want).expand(out.shape))


def test_peaked_scores_over_a_shared_prefix(lib, units):
    case = Shared([(5, 1500, 100), (4, 300, 3)], 8, 2, 128, 16, "bf16", 31, q_std=12.0)
    case.check(case.run(lib))
    case.scale = 0.7
    case.check(case.run(lib))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_large_scores_that_are_equal_in_a_prefix_and_behind_it(lib, units, kind):
    # every key has the same score, which fp32 holds in steps of 2 and more: what is rounded of it has to be the same on either side
    case = Shared([(4, 900, [60, 500, 1, 300]), (3, 200, 200)], 8, 2, 128, 16, kind, 38)
    case.ck.zero_()
    case.ck[..., 0] = 128.0
    case.q[:] = 0.0
    case.q[..., 0] = 2.0 ** 18 * 1.375
    case.scale = 0.3
    out = f64(case.run(lib))
    want, spread = serving.paged_attention(f64(case.q), f64(case.ck) * case.ks, f64(case.cv) * case.vs, case.table, case.seqs, case.positions, case.scale)
    # weights of one, which 16 bits hold; sums: two additions for every 16 keys, a join of up to 30 parts
    allowed = BF16_STEP * np.abs(want) + ((2.0 ** -15 if kind == "bf16" else F16_STEP) + (64 + max(case.lens) / 4) * F32_STEP) * spread * (1 + BF16_STEP)
    assert (np.abs(out - want) <= allowed).all(), (np.abs(out - want) / allowed).max()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_leading_keys_of_no_value_in_a_prefix(lib, units, kind):
    # keys that lead and whose values are zero leave the row to the others, whose weights are 2^-10 to 2^-40 of theirs
    case = Shared([(4, 900, 60)], 8, 2, 64, 16, kind, 32)
    case.ck[..., 0] = 0.0
    for j in [1] + list(range(70, 900, 97)):
        for r in range(5):
            page = int(case.table[r, j // 16])
            case.ck[page, :, j % 16, 0], case.cv[page, :, j % 16] = 16.0 / case.ks, 0.0
    leads = torch.tensor([7.0, 14.0, 21.0, 28.0, 3.0, 10.0, 17.0, 24.0])
    case.q[:, :, 0] = (leads / (16.0 * case.scale)).bfloat16()
    case.check(case.run(lib))


def test_infinite_values_and_scores_in_a_prefix(lib, units):
    case = Shared([(3, 500, [1, 64, 300])], 4, 2, 64, 16, "bf16", 33)
    for j, dim, v in ((0, 3, "inf"), (200, 17, "-inf"), (447, 63, "inf"), (0, 40, "inf"), (300, 40, "-inf"), (100, 5, "nan")):
        case.cv[int(case.table[0, j // 16]), :, j % 16, dim] = float(v)
    out = f64(case.run(lib))
    with np.errstate(invalid="ignore"):
        want, _ = serving.paged_attention(f64(case.q), f64(case.ck), f64(case.cv), case.table, case.seqs, case.positions, case.scale)
    special = ~np.isfinite(want)
    assert special.any() and np.isfinite(want).any()
    assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(out[special & ~np.isnan(want)], want[special & ~np.isnan(want)])
    # a key of -inf scores is left out where it counts against a query, and makes the row NaN where it counts for it
    case = Shared([(3, 500, [1, 64, 300])], 4, 2, 64, 16, "bf16", 34)
    case.ck[int(case.table[0, 3]), :, 5, 0] = -INF
    case.q[:2, :, 0], case.q[2, :, 0] = 1.0, -1.0
    out = case.run(lib)
    assert torch.isnan(out[2]).all() and torch.isfinite(out[:2]).all()
    case.ck[int(case.table[0, 3]), :, 5, 0] = -3e4      # as good as nothing too, and the oracle can take it
    case.check(out, only=[0, 1])


def test_what_is_out_of_range_in_groups_is_reported(lib, units):
    groups = [(3, 500, [1, 64, 300]), (2, 200, 30), (2, 300, 5)]
    case = Shared(groups, 8, 2, 64, 16, "bf16", 35)
    plain = case.run(lib)
    case.check(plain)
    # a group whose request or length is impossible reads its rows' own tables; so do all when the bounds do not ascend
    n, width = case.table.shape
    for change in (dict(seq=[0, n, 2]), dict(seq=[-1, 1, 2]), dict(prefix=[500, -1, 300]), dict(prefix=[500, 200, width * 16 + 1])):
        case.check(case.run(lib, reported=2, **change))
    low, high = -2 ** 31, 2 ** 31 - 1
    for rows in ([0, 5, 3, 7], [-1, 3, 5, 7], [0, 3, 5, 8], [7, 5, 3, 0], [0, 3, low, 7], [high, low, 5, 7], [0, high, low, 7], [low, 3, 5, high]):
        case.check(case.run(lib, reported=2, rows=rows))
    # bounds that leave rows out, and groups that are smaller than what shares the prefix
    for rows, prefix in (([1, 3, 5, 7], case.prefix), ([0, 2, 2, 2], [500, 1, 1]), ([0, 3, 5, 5], [400, 200, 0]), ([3, 3, 5, 7], [0, 128, 300])):
        case.check(case.run(lib, rows=rows, prefix=prefix))
    # a block outside the cache: nothing of it is seen, through either table
    for bad in (-1, case.ck.shape[0], 2 ** 31 - 1):
        broken = Shared(groups, 8, 2, 64, 16, "bf16", 35)
        page = broken.table[0, 7]
        broken.table[broken.table == page] = bad
        out = broken.run(lib, reported=2)
        for t in range(3):
            seen = np.setdiff1d(np.arange(broken.lens[t]), np.arange(7 * 16, 8 * 16))
            for h in range(8):
                pages = broken.table[3 + t][seen // 16]
                k, v = f64(broken.ck)[pages, h // 4, seen % 16], f64(broken.cv)[pages, h // 4, seen % 16]
                s = k @ f64(broken.q)[t, h] * broken.scale
                w = np.exp(s - s.max())
                want = w @ v / w.sum()
                assert np.abs(f64(out[t, h]) - want).max() <= BF16_STEP * np.abs(want).max() + 1e-3


def test_several_rows_of_a_request_and_strided_rows(lib, units):
    # the options of a question: every request has several new rows, which see the shared prefix and their own tokens up to themselves
    case = Shared([(4, 333, [40, 41, 42, 43])], 8, 4, 128, 16, "bf16", 36)
    take = [(t, p) for t in range(4) for p in range(330 + 20 * t, case.lens[t], 3)]
    R = len(take)
    q = inputs.normal_fp32((R, 8, 128), 1.0, 9).bfloat16()
    wide = torch.full((R, 3, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 1] = q.cuda()
    out = torch.full((R, 9, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    status = ints([0])
    lib.qzo_shared_prefix_attention(wide[:, 1], lib.KvCache(case.ck, case.cv), torch.from_numpy(case.table).cuda(), ints([p for _, p in take]), ints([0, R]), ints([0]),
                                    ints([333]), row_seq=ints([1 + t for t, _ in take]), out=out[:, :8], status=status)
    assert int(status) == 0 and (out[:, 8] == 5.0).all()
    case.R, case.q, case.seqs, case.positions, case.lens = R, q, np.array([1 + t for t, _ in take]), [p for _, p in take], [p + 1 for _, p in take]
    case.check(out[:, :8])


def test_calls_one_behind_the_other_see_what_was_written_before_them(lib, units):
    # the rows' own keys are read while the kernel in front runs: queries and positions that are written just before a call, and queries that are
    # the call before's output, in a stream and in a replayed graph
    case = Shared([(3, 500, [64, 300, 90]), (3, 200, [400, 17, 20])], 8, 4, 128, 16, "bf16", 40)
    cache, table, rows, seq, prefix, of = lib.KvCache(case.ck, case.cv), torch.from_numpy(case.table).cuda(), ints(case.rows), ints([0, 1]), ints(case.prefix), ints(case.seqs.tolist())
    R, n = case.R, 4
    queries = [inputs.normal_fp32((R, 8, 128), 1.0, 60 + i).bfloat16().cuda() for i in range(n)]
    places = [ints([p - 5 * i for p in case.positions]) for i in range(n)]
    q, positions = torch.empty_like(queries[0]), torch.empty_like(places[0])
    ws = torch.empty(lib.qzo_shared_prefix_attention_workspace_bytes(R, 2, 8, 4, 128, case.table.shape[1] * 16), dtype=torch.uint8, device="cuda")

    def call(q, out):
        return lib.qzo_shared_prefix_attention(q, cache, table, positions, rows, seq, prefix, row_seq=of, workspace=ws, out=out)

    def steps(outs, wait=lambda: None):
        for i in range(n):
            q.copy_(queries[i])
            positions.copy_(places[i])
            wait()
            call(q, outs[i][0])
            wait()
            call(outs[i][0], outs[i][1])
            wait()
    outs, want = ([[torch.empty_like(q) for _ in range(2)] for _ in range(n)] for _ in range(2))
    steps(want, torch.cuda.synchronize)
    same = lambda: all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for pair in zip(outs, want) for a, b in zip(*pair))  # noqa: E731
    for _ in range(10):
        steps(outs)
        assert same()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(stream):
        steps(outs)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            steps(outs)
    for _ in range(10):
        for pair in outs:
            for t in pair:
                t.zero_()
        graph.replay()
        assert same()


@pytest.mark.parametrize("H,Hkv,dh,block,kind", [(8, 8, 64, 16, "bf16"), (32, 8, 128, 32, "bf16"), (96, 8, 64, 16, "bf16"), (80, 4, 64, 16, "bf16"), (8, 8, 128, 16, "e4m3"), (32, 8, 64, 64, "e4m3")])
def test_rows_with_many_tokens_of_their_own_among_rows_with_few(lib, units, H, Hkv, dh, block, kind):
    # many rows and key heads, each of which has one CTA for its own keys, whatever their number: from none to thousands, with a prefix, without one and in
    # front of its end
    owns = [[3, 700, None, 2100], [513, 512, 514, 1], [5, -20, 40, 1500], [1200, 1030, 1025, 2049], [0, 0, 1, 0], [2048, 1024, 17, 16], [1, 2, 3, 4], [9, 9, 600, 9]]
    groups = [(4, 130 + 41 * i, owns[i % len(owns)]) for i in range(14)] + [(5, 0, [3000, 5, 513, 4000, 1])]
    case = Shared(groups, H, Hkv, dh, block, kind, 43)
    out = case.run(lib)
    case.check(out)
    for _ in range(5):
        assert torch.equal(out.view(torch.int16), case.run(lib).view(torch.int16))


def test_one_workspace_as_requests_end_and_groups_become_fewer(lib):
    # sized once for 64 rows in 64 groups; then fewer rows in fewer groups, which take other ways; none writes behind the workspace's end
    H = Hkv = 8
    case = Shared([(64, 1500, 40)], H, Hkv, 128, 16, "bf16", 42)
    cache, table, q, pos, of = lib.KvCache(case.ck, case.cv), torch.from_numpy(case.table).cuda(), case.q.cuda(), ints(case.positions), ints(case.seqs.tolist())
    need = lib.qzo_shared_prefix_attention_workspace_bytes(64, 64, H, Hkv, 128, case.table.shape[1] * 16)
    buffer = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    want = case.run(lib)
    case.check(want)
    lens = np.array(case.lens)
    for path in (0, 2, 3):
        lib.qzo_debug_prefix_path(path)
        assert path == 0 or lib.qzo_shared_prefix_attention_workspace_bytes(64, 64, H, Hkv, 128, case.table.shape[1] * 16) <= need
        try:
            for R, n in ((64, 64), (64, 16), (64, 2), (64, 1), (37, 37), (37, 5), (32, 2), (18, 18), (18, 1), (5, 2), (1, 1)):
                status = ints([0])
                out = lib.qzo_shared_prefix_attention(q[:R], cache, table, pos[:R].contiguous(), ints([R * i // n for i in range(n + 1)]), ints([0] * n), ints([1500] * n),
                                                      row_seq=of, workspace=buffer[:need], status=status)
                assert int(status) == 0 and (buffer[need:] == 77).all(), (path, R, n)
                few = Shared.__new__(Shared)
                few.__dict__.update(case.__dict__, R=R, q=case.q[:R], seqs=case.seqs[:R], positions=case.positions[:R], lens=lens[:R].tolist())
                few.check(out)
        finally:
            lib.qzo_debug_prefix_path(0)


def test_a_prefix_of_a_cache_beyond_32_bit_offsets(lib, units):
    Hkv, block, dh = 8, 64, 128
    n_blocks = (1 << 32) // (Hkv * block * dh * 2) + 6            # 4 GB and a little of keys, as many of values
    small = Shared([(3, 640, [5, 70, 1])], 16, Hkv, dh, block, "bf16", 37)
    k, v = (torch.zeros((n_blocks, Hkv, block, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    used = np.unique(small.table[small.table >= 0])
    to = np.concatenate([np.arange(n_blocks - (len(used) + 1) // 2, n_blocks), np.arange(len(used) // 2)])
    far = small.table.copy()
    for a, b in zip(used, to):
        k[int(b)], v[int(b)] = small.ck[int(a)], small.cv[int(a)]
        far[small.table == a] = b
    near = small.run(lib)
    small.table, small.ck, small.cv = far, k, v
    assert torch.equal(near, small.run(lib))
    del k, v


# ------------------------------------------------------------------ together

def _model(lib, name, max_tokens):
    from tests.helpers import build_oracle_model
    cfg = inputs.model_cfg(name)
    raw = inputs.raw_model_tensors(cfg, seed=1000)
    return cfg, build_oracle_model(raw), lib.build_model_from_raw(raw, max_tokens)


def _oracle_logits(om, tokens):
    from oracle import model as omodel
    cap, tok = {}, np.asarray(tokens)[None]
    omodel.forward_loss(om, tok, np.full_like(tok, -100), 0, 0, 1e-3, capture=cap)
    return cap["logits"]


@pytest.mark.parametrize("name,block,dtype", [("tiny_dh128", 16, torch.bfloat16), ("tiny", 16, torch.bfloat16), ("tiny_opt", 32, torch.bfloat16)])
def test_beam_search_with_a_model(lib, path, name, block, dtype):
    # two prompts, four beams each, over one pool: prompts by the first beam, then select, fork, copy, decode, step by step, with a
    # compaction on the way; every live row's logits are those of the oracle's forward of that beam's whole text
    cfg, om, gm = _model(lib, name, 4096)
    B, W, n_blocks, steps, power = 2, 4, 90, 9, 0.6
    H, dh = cfg["n_heads"], cfg["d_model"] // cfg["n_heads"]
    pages = lambda: torch.full((n_blocks, H, block, dh), float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    caches = [lib.KvCache(pages(), pages()) for _ in range(cfg["n_layers"])]
    rng = _gen(7)
    longest = cfg["max_seq"] - steps - 1
    prompts = [rng.integers(0, cfg["vocab"], n).tolist() for n in (longest, longest // 2 + 3)]
    width = -(-cfg["max_seq"] // block)
    lens, count, table = ints([0] * (B * W)), ints([n_blocks]), torch.full((B * W, width), -1, dtype=torch.int32, device="cuda")
    free = torch.from_numpy(rng.permutation(n_blocks).astype(np.int32)).cuda()
    status = ints([0])
    end = 3
    # the prompts: rows of the first beam of each request
    new = [len(prompts[r // W]) if r % W == 0 else 0 for r in range(B * W)]
    logits, maps = gm.qzo_decode_requests(caches, ints(sum(prompts, [])), lens, ints(new), table, free, count, status=status)
    rows = np.full((B, W), -1, np.int32)
    rows[:, 0] = np.cumsum([len(p) for p in prompts]) - 1
    text = [list(prompts[r // W]) if r % W == 0 else None for r in range(B * W)]
    scores = torch.full((B, W), -INF, device="cuda")
    scores[:, 0] = 0.0
    last, lengths = ints([[0] * W] * B), ints([[0] * W] * B)
    groups = dict(group_rows=ints([0, W, 2 * W]), prefix_seq=ints([0, W]), prefix_len=ints([len(p) for p in prompts]))
    for step in range(steps):
        host = logits.cpu().numpy()
        for b in range(B):
            for w in range(W):
                r = int(rows[b, w])
                if r >= 0 and text[b * W + w] is not None:
                    want = _oracle_logits(om, text[b * W + w])[-1]
                    assert np.abs(host[r] - want).max() <= 2e-2 * np.abs(want).max(), (step, b, w)
        want = oracle.beam_select(host, scores.cpu().numpy(), rows, last.cpu().numpy(), end, lengths.cpu().numpy(), power)
        parents, tokens, scores, lengths = lib.qzo_beam_select(logits, scores, rows=torch.from_numpy(rows).cuda(), last_tokens=last, end_token=end,
                                                               lengths=lengths, length_power=power, status=status)
        assert parents.tolist() == [[f[0] for f in best] for best in want] and tokens.tolist() == [[f[1] for f in best] for best in want]
        table, lens, count, copies, n_copies = lib.qzo_fork_requests(lens, parents, table, free, count, block, n_blocks, status=status)
        lib.qzo_copy_blocks(caches, copies, n_copies, status=status)
        if step == 4:
            table, count, copies, n_copies = lib.qzo_compact_blocks(lens, table, free, block, n_blocks, 60, free_count=count, status=status)
            lib.qzo_copy_blocks(caches, copies, n_copies, status=status)
            assert int(table.max()) < 60 and int(count) == 60 - len(set(table[table >= 0].tolist()))
        was_end = [bool(v) for v in (last.view(-1) == end).tolist()]
        text = [None if p < 0 else text[p] + ([] if was_end[p] else [t]) for p, t in zip(parents.view(-1).tolist(), tokens.view(-1).tolist())]
        last = tokens
        # every beam that goes on adds its token; the others have no row of their own, and padding stands in its place
        goes = (tokens != end) & (parents >= 0)
        seq, pos, slots = lib.qzo_assign_slots(lens, goes.to(torch.int32).view(-1).contiguous(), table, free, count, block, B * W, status=status)
        step_tokens = torch.where(seq >= 0, tokens.view(-1)[seq.clamp(min=0).long()], 0).to(torch.int32)
        n_rows = [int(goes[:b].sum()) for b in range(B + 1)]
        groups["group_rows"] = ints(n_rows)
        # the request that holds the prefix: any of its beams that is still there
        groups["prefix_seq"] = ints([b * W + int((parents[b] >= 0).int().argmax()) for b in range(B)])
        logits = gm.qzo_decode_groups(caches, step_tokens, seq, pos, slots, table, **groups)
        assert int(status) == 0 and gm.qzo_device_status() == 0
        rows = np.full(B * W, -1, np.int32)
        live = [r for r in seq.tolist() if r >= 0]
        rows[live] = np.arange(len(live))
        rows = rows.reshape(B, W)
        assert lens.tolist() == [0 if t is None else len(t) for t in text]
    gm.close()


def test_decode_of_groups_refuses_and_reports(lib):
    cfg, _, gm = _model(lib, "tiny", 64)
    cache = [lib.KvCache(*(torch.zeros((8, 4, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))) for _ in range(2)]
    table, z, one = ints([[0, 1, 2, 3], [4, 5, 6, 7]]), ints([0, 0]), ints([0, 1])
    a = dict(tokens=z, row_seq=one, positions=z, slots=ints([0, 64]), block_table=table)
    for rows, seq, length, ok in ((ints([0, 2]), ints([0]), ints([1]), True), (ints([0]), ints([0]), ints([1]), False), (ints([0, 2]), ints([0]).float(), ints([1]), False),
                                  (torch.tensor([0, 2], dtype=torch.int32), ints([0]), ints([1]), False)):
        if ok:
            assert gm.qzo_decode_groups(cache, group_rows=rows, prefix_seq=seq, prefix_len=length, **a).shape == (2, cfg["vocab"])
        else:
            with pytest.raises(AssertionError):
                gm.qzo_decode_groups(cache, group_rows=rows, prefix_seq=seq, prefix_len=length, **a)
    lib.qzo_debug_prefix_path(2)
    try:                                                # a workspace that holds no prefix: own tables; and none is touched beyond its end
        plain = gm.qzo_decode(cache, **a)
        assert torch.equal(plain, gm.qzo_decode_groups(cache, group_rows=ints([0, 2]), prefix_seq=z[:1], prefix_len=ints([1]), **a))
    finally:
        lib.qzo_debug_prefix_path(0)
    for bad in (-1, 4):
        with pytest.raises(lib.QzoError):
            lib.qzo_debug_prefix_path(bad)
    gm.close()


def test_a_search_step_in_a_replayed_graph_and_on_two_streams(lib, path):
    # select, fork, copy and attend, captured behind a side stream's work, replayed with new inputs; then two streams at once with a workspace each
    case = Shared([(4, 500, [9, 20, 33, 70]), (4, 300, [1, 2, 3, 4])], 8, 2, 128, 16, "bf16", 51)
    R, V, block, n_blocks = case.R, 3000, 16, case.ck.shape[0]
    rng = _gen(52)
    side = torch.cuda.Stream()

    def state(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        s = dict(logits=torch.randn(R, V, generator=g, device="cuda"), scores=-torch.rand(2, 4, generator=g, device="cuda"), q=torch.randn(R, 8, 128, generator=g, device="cuda").bfloat16(),
                 k=case.ck.clone(), v=case.cv.clone(), table=torch.from_numpy(case.table[2:]).cuda(), lens=ints(case.lens), count=ints([60]))
        s["free"] = torch.full((n_blocks + 70,), -1, dtype=torch.int32, device="cuda")
        s["free"][:60] = torch.arange(n_blocks, n_blocks + 60)
        s["k"] = torch.cat((s["k"], torch.zeros_like(s["k"][:60].repeat(60 // s["k"].shape[0] + 1, 1, 1, 1)[:60])))
        s["v"] = torch.cat((s["v"], torch.zeros_like(s["v"][:60].repeat(60 // s["v"].shape[0] + 1, 1, 1, 1)[:60])))
        return s

    def step(s, ws):
        cache = lib.KvCache(s["k"], s["v"])
        parents, tokens, scores, _ = lib.qzo_beam_select(s["logits"], s["scores"], workspace=ws[0])
        table, lens, count, copies, n = lib.qzo_fork_requests(s["lens"], parents, s["table"], s["free"], s["count"], block, n_blocks + 60)
        lib.qzo_copy_blocks([cache], copies, n)
        positions = lens - 1
        out = lib.qzo_shared_prefix_attention(s["q"], cache, table, positions, s["rows"], s["seq"], s["prefix"], workspace=ws[1])
        return parents, tokens, scores, table, lens, count, copies, n, out

    def workspaces():
        return (torch.empty(lib.qzo_beam_select_workspace_bytes(2, 4, V), dtype=torch.uint8, device="cuda"),
                torch.empty(max(1, lib.qzo_shared_prefix_attention_workspace_bytes(R, 2, 8, 2, 128, case.table.shape[1] * block)), dtype=torch.uint8, device="cuda"))
    states = [state(i) for i in range(4)]
    for s in states:
        s["rows"], s["seq"], s["prefix"] = ints([0, 4, 8]), ints([0, 4]), ints([500, 300])
    ws = workspaces()
    # what each state gives by itself, on copies (a step changes pages and stack)
    want = [[t.clone() for t in step({k: v.clone() for k, v in s.items()}, ws)] for s in states]
    for w in want:
        assert not torch.isnan(w[-1].float()).any()
    live = {k: v.clone() for k, v in states[0].items()}
    fresh = {k: v.clone() for k, v in states[0].items()}
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step({k: v.clone() for k, v in states[0].items()}, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for k in live:
                live[k].copy_(fresh[k])
            got = step(live, ws)
        for i in (1, 0, 2, 3, 1):
            for k in fresh:
                fresh[k].copy_(states[i][k])
            graph.replay()
            side.synchronize()
            for a, b in zip(got, want[i]):
                assert torch.equal(a, b)
    # two streams at once
    other = torch.cuda.Stream()
    mine = [{k: v.clone() for k, v in s.items()} for s in states[:2]]
    both = [workspaces(), workspaces()]
    torch.cuda.synchronize()
    got = [[], []]
    for turn in range(10):
        for i, st in enumerate((side, other)):
            with torch.cuda.stream(st):
                got[i].append(step({k: v.clone() for k, v in mine[i].items()}, both[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            for a, b in zip(g, want[i]):
                assert torch.equal(a, b)
    del graph


def test_tensors_off_the_device_or_of_another_shape_are_refused(lib):
    case = Shared([(2, 100, 5)], 2, 2, 64, 16, "bf16", 61)
    cache, table, pos = lib.KvCache(case.ck, case.cv), torch.from_numpy(case.table).cuda(), ints(case.positions)
    good = dict(q=case.q.cuda(), cache=cache, block_table=table, positions=pos, group_rows=ints([0, 2]), prefix_seq=ints([0]), prefix_len=ints([100]), row_seq=ints([1, 2]))
    lib.qzo_shared_prefix_attention(**good)
    for change in (dict(q=case.q), dict(positions=pos.cpu()), dict(group_rows=ints([0])), dict(prefix_len=ints([])), dict(prefix_seq=ints([0]).long()), dict(row_seq=ints([1])),
                   dict(out=torch.empty(2, 2, 32, dtype=torch.bfloat16, device="cuda")), dict(q=case.q.cuda().float())):
        with pytest.raises(AssertionError):
            lib.qzo_shared_prefix_attention(**{**good, **change})
    lib.qzo_debug_prefix_path(3)
    with pytest.raises(lib.QzoError):
        lib.qzo_shared_prefix_attention(**good, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    lib.qzo_debug_prefix_path(0)
    x, scores = torch.randn(4, 50, device="cuda"), torch.zeros(2, 2, device="cuda")
    lib.qzo_beam_select(x, scores)
    for change in (dict(logits=x.cpu()), dict(logits=x.half()), dict(scores=scores.cpu()), dict(scores=scores.double()), dict(last_tokens=ints([1])), dict(logits=x.t()),
                   dict(rows=ints([[0, 1]])), dict(scores_out=torch.zeros(1, device="cuda"))):
        with pytest.raises(AssertionError):
            lib.qzo_beam_select(**{**dict(logits=x, scores=scores), **change})
    lens, tab, free, n = ints([5, 20]), ints([[0, 1], [2, 3]]), ints([4, 5, -1, -1, -1, -1]), ints([2])
    for change in (dict(parents=ints([0])), dict(lens=lens.cpu()), dict(block_table=tab.long()), dict(table_out=ints([[0, 1]])), dict(copies=ints([0, 0, 0]))):
        with pytest.raises(AssertionError):
            lib.qzo_fork_requests(**{**dict(lens=lens, parents=ints([0, 1]), block_table=tab, free=free, free_count=n, block_size=16, n_blocks=6), **change})
    with pytest.raises(lib.QzoError):                   # never in place
        lib.qzo_fork_requests(lens, ints([0, 1]), tab, free, n, 16, 6, table_out=tab)
    with pytest.raises(AssertionError):
        lib.qzo_copy_blocks([], ints([[0, 1, 2]]), ints([1]))


def test_a_chain_of_serving_calls_sees_what_the_calls_before_wrote(lib, units):
    # slots, head norms, cache write and attention right behind one another, step after step in the same buffers, with no other kernel between them: each
    # may start while the one before it ends.  What a step gives is what it gives when every call is waited for
    case = Shared([(4, 500, [9, 20, 33, 60]), (4, 200, [1, 30, 5, 100])], 8, 4, 128, 16, "bf16", 41)
    R, n, steps, spare = case.R, len(case.prefix), 6, 2 * case.R
    n_blocks = case.ck.shape[0]
    more = torch.full((spare, 4, 16, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    first = dict(k=torch.cat((case.ck, more)), v=torch.cat((case.cv, more)), lens=ints(case.prefix + case.lens), count=ints([spare]),
                 free=torch.arange(n_blocks, n_blocks + spare, dtype=torch.int32, device="cuda"),
                 table=torch.nn.functional.pad(torch.from_numpy(case.table).cuda(), (0, 2), value=-1))
    live = {name: t.clone() for name, t in first.items()}
    cache, new = lib.KvCache(live["k"], live["v"]), ints([0] * n + [1] * R)
    given = [[inputs.normal_fp32((R, h, 128), 1.0, 70 + 3 * i + j).bfloat16().cuda() for j, h in enumerate((8, 4, 4))] for i in range(steps)]
    gain, angles = torch.linspace(0.5, 1.5, 128, device="cuda"), lib.qzo_rope_table(4096, 128)
    seq, pos, slots = (ints([0] * R) for _ in range(3))
    q, status, rows, prefix, of = torch.empty_like(given[0][0]), ints([0]), ints(case.rows), ints(case.prefix), ints(list(range(n)))
    ws = torch.empty(lib.qzo_shared_prefix_attention_workspace_bytes(R, n, 8, 4, 128, live["table"].shape[1] * 16), dtype=torch.uint8, device="cuda")

    def run(outs, wait):
        for name, t in first.items():
            live[name].copy_(t)
        torch.cuda.synchronize()
        for i in range(steps):
            lib.qzo_assign_slots(live["lens"], new, live["table"], live["free"], live["count"], 16, R, row_seq=seq, positions=pos, slots=slots, status=status)
            wait()
            lib.qzo_qk_norm_rope_cache(*given[i], pos, slots, cache, q_gain=gain, k_gain=gain, table=angles, q_out=q, status=status)
            wait()
            lib.qzo_shared_prefix_attention(q, cache, live["table"], pos, rows, of, prefix, row_seq=seq, out=outs[i], workspace=ws, status=status)
            wait()
    want, outs = ([torch.empty_like(q) for _ in range(steps)] for _ in range(2))
    run(want, torch.cuda.synchronize)
    assert int(status) == 0 and live["lens"].tolist() == case.prefix + [v + steps for v in case.lens]
    for _ in range(20):
        run(outs, lambda: None)
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(outs, want))
    case.q, case.ck, case.cv, case.table = q, live["k"], live["v"], live["table"].cpu().numpy()
    case.lens = [v + steps for v in case.lens]
    case.positions = [v - 1 for v in case.lens]
    case.check(outs[-1])


# ------------------------------------------------------------------ a decode step over shared prefixes

class Step:
    """One decode step of R rows of a model whose caches hold `prefix` random tokens that all rows share and some of their own."""

    def __init__(self, lib, name, R, prefix, max_tokens, kind="bf16", width=None, **override):
        cfg = inputs.model_cfg(name, **override)
        self.gm = lib.build_model_from_raw(inputs.raw_model_tensors(cfg, seed=1000), max_tokens)
        H, dh, block = cfg["n_heads"], cfg["d_model"] // cfg["n_heads"], 16
        dt, ks, vs = CACHES[kind]
        own = [prefix + 1 + 7 * (r % 5) for r in range(R)]                      # tokens of a row behind this step
        common, most = prefix // block, -(-max(own) // block)
        n_blocks = common + R * (most - common)
        self.caches = [lib.KvCache(*((inputs.normal_fp32((n_blocks, H, block, dh), 1.0, 80 + 2 * i + j) / s).to(dt).cuda() for j, s in enumerate((ks, vs))), ks, vs)
                       for i in range(cfg["n_layers"])]
        table = np.full((R, width or most), -1, np.int32)
        table[:, :common] = np.arange(common)
        table[:, common:most] = common + np.arange(R * (most - common)).reshape(R, -1)
        for c in self.caches:                                                   # the rest of the prefix stands in every row's own block
            for pages in (c.k.view(torch.uint8), c.v.view(torch.uint8)):
                pages[table[1:, common].tolist(), :, :prefix % block] = pages[int(table[0, common]), :, :prefix % block].clone()
        pos = np.array(own) - 1
        slots = table[np.arange(R), pos // block] * block + pos % block
        self.args = [ints(a.tolist()) for a in (_gen(81).integers(0, cfg["vocab"], R), np.arange(R), pos, slots)] + [torch.from_numpy(table).cuda()]
        self.groups = dict(group_rows=ints([0, R]), prefix_seq=ints([0]), prefix_len=ints([prefix]))

    def plain(self):
        return self.gm.qzo_decode(self.caches, *self.args)

    def shared(self):
        out = self.gm.qzo_decode_groups(self.caches, *self.args, **self.groups)
        assert self.gm.qzo_device_status() == 0
        return out


    def reads_once(self):
        """Whether the prefix is read through the first row's table alone: without the other rows' entries for it nothing is missed, while a row that reads
        its own table meets blocks that no cache has.  The last thing a step is used for (the status stays)."""
        want = self.shared()
        self.args[4][1:, :int(self.groups["prefix_len"]) // 16] = -1
        got = self.gm.qzo_decode_groups(self.caches, *self.args, **self.groups)
        missed = self.gm.qzo_device_status() != 0
        assert missed or torch.equal(got, want)
        return not missed


def _close(a, b):
    return ((a - b).abs().max() <= 2e-2 * b.abs().max()).item()


def test_decode_of_groups_takes_the_next_way_where_the_first_does_not_fit(lib):
    # a table so wide that units of 128 are the choice, and a buffer of 1008 results that holds units of 16 only
    step = Step(lib, "tiny_dh128", 64, 150, 64, width=3000)
    plain, rule = step.plain(), step.shared()
    lib.qzo_debug_prefix_path(2)
    try:
        few = step.shared()
    finally:
        lib.qzo_debug_prefix_path(0)
    assert torch.equal(rule, few) and _close(rule, plain) and step.reads_once()
    step.gm.close()


@pytest.mark.parametrize("max_tokens", [2, 3, 4, 5, 6, 9, 40])
def test_decode_of_groups_in_buffers_of_any_size(lib, path, max_tokens):
    # 62 results of a query and upwards: the smallest has room for the few-query way without splits at most, none for units of 128: own tables then
    step = Step(lib, "tiny", 2, 1000, max_tokens, width=256, max_seq=2048)
    plain, shared = step.plain(), step.shared()
    assert _close(shared, plain)
    assert path == 2 or torch.equal(shared, plain)
    assert torch.equal(step.plain(), plain), "what stands behind the buffer, the table of rotations among it, is as it was"
    assert step.reads_once() == (path == 2), "only units of few queries fit"
    step.gm.close()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("name,R,prefix", [("tiny", 3, 40), ("tiny_dh128", 21, 150), ("tiny_opt", 9, 33)])
def test_decode_of_groups_over_either_cache(lib, units, name, R, prefix, kind):
    step = Step(lib, name, R, prefix, 4096, kind)         # units of 128 leave 37888 results of 520 bytes at least: 20 MB of the 32
    assert _close(step.shared(), step.plain()) and step.reads_once()
    step.gm.close()
