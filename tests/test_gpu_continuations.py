"""GPU parity of the operators for several continuations of one prompt against the oracle: what is whole is equal, what is computed
is within bounds that count the roundings."""
import math

import numpy as np
import pytest
import torch

from oracle import continuations as oracle

pytestmark = pytest.mark.gpu

F32_STEP = 2.0 ** -24
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
