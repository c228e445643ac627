"""Pins of the oracle of the operators for several continuations (no GPU), and the refusals of their entry points, which come
before any device call."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

from oracle import continuations as oracle, serving


def test_beam_search_of_full_width_finds_the_most_probable_sequences():
    # with as many beams as there are sequences, the search is the enumeration of all of them
    rng = np.random.default_rng(1)
    V, steps = 3, 3
    W = V ** steps
    table = {}                                          # a model whose logits depend on everything before

    def logits(seq):
        return table.setdefault(seq, rng.standard_normal(V) * 2)
    beams = [((), 0.0)] + [((), -math.inf)] * (W - 1)
    for _ in range(steps):
        x = np.stack([logits(seq) for seq, _ in beams])
        best = oracle.beam_select(x, np.array([[s for _, s in beams]]))[0]
        beams = [(beams[p][0] + (t,), s) if p >= 0 else ((), -math.inf) for p, t, s, _, _ in best]
    every = {}
    for a in range(V):
        for b in range(V):
            for c in range(V):
                lp = 0.0
                for i, t in enumerate((a, b, c)):
                    x = logits((a, b, c)[:i])
                    lp += x[t] - math.log(np.exp(x).sum())
                every[(a, b, c)] = lp
    want = sorted(every, key=lambda s: -every[s])
    assert [seq for seq, _ in beams] == want
    np.testing.assert_allclose([s for _, s in beams], [every[s] for s in want], rtol=1e-12)
    assert abs(sum(math.exp(s) for _, s in beams) - 1) < 1e-12


def test_an_ended_beam_stays_and_is_ranked_by_its_own_length():
    x = np.log(np.array([[0.7, 0.3], [0.5, 0.5]]))
    scores, last, lengths = np.array([[-1.0, -1.2]]), np.array([[1, 0]]), np.array([[2, 5]])
    best = oracle.beam_select(x, scores, last=last, end_token=1, lengths=lengths, power=1.0)[0]
    # per token: the ended one -1 / 2, the others (-1.2 - log 2) / 6
    assert [(p, t, n) for p, t, _, n, _ in best] == [(1, 0, 6), (1, 1, 6)]
    best = oracle.beam_select(x, scores, last=last, end_token=1, lengths=lengths, power=0.0)[0]
    assert [(p, t, s) for p, t, s, _, _ in best][0] == (0, 1, -1.0)


def test_forks_keep_what_requests_hold_apart_from_each_other():
    # against a cache of plain lists: every request's tokens, after forks, endings, growth and compaction
    rng = np.random.default_rng(2)
    B, width, block, n_blocks = 6, 8, 16, 64
    table, free, count, lens = np.full((B, width), -1), np.arange(n_blocks), n_blocks, [0] * B
    pages = np.zeros((n_blocks, 1, block, 1))
    said = [[] for _ in range(B)]
    for step in range(120):
        new = rng.integers(0, 20, B).tolist()
        st = serving.assign_slots(lens, new, table, free, count, block, 6 * 20)
        if st is not None:
            for s, r, p in zip(st["slots"], st["row_seq"], st["positions"]):
                if s >= 0:
                    value = float(rng.integers(1, 1 << 30))
                    pages[s // block, 0, s % block, 0] = value
                    assert p == len(said[r])
                    said[r].append(value)
            lens, count, table, free = st["lens"], st["free_count"], st["table"], st["free"]
        parents = rng.integers(-1 if st is not None else -3, B, B)
        out = oracle.fork_requests(lens, parents, table, free, count, block, n_blocks)
        if out is None:
            parents[:] = -1
            out = oracle.fork_requests(lens, parents, table, free, count, block, n_blocks)
        oracle.copy_blocks(pages, out["copies"])
        said = [list(said[p]) if p >= 0 else [] for p in parents]
        lens, table, free, count = out["lens"], out["table"], out["free"], out["free_count"]
        if step % 7 == 0:
            table, stack, copies = oracle.compact_blocks(lens, table, block, n_blocks, n_blocks)
            oracle.copy_blocks(pages, copies)
            free, count = np.array(stack + [-1] * (n_blocks - len(stack))), len(stack)
        held = {int(v) for r in range(B) for v in table[r, :-(-lens[r] // block)]}
        assert sorted(held) + sorted(free[:count]) == sorted(held) + sorted(set(range(n_blocks)) - held)
        if step % 7 == 0:
            assert held == set(range(len(held)))
        for r in range(B):
            assert [pages[table[r, t // block], 0, t % block, 0] for t in range(lens[r])] == said[r]


# ---- refusals: a wrong argument is turned away before the device is touched ----

def _lib():
    from paper_2505_13430_b200 import qzo
    return qzo


P, Q, ODD, NONE = (ctypes.c_void_p(v) for v in (0x10000, 0x20000, 0x10002, 0))


def _no_gpu():
    import torch
    return not torch.cuda.is_available()


made_up = pytest.mark.skipif(not _no_gpu(), reason="made-up pointers: only where no device would follow them")


def _cache(**kw):
    qzo = _lib()
    f = dict(k=0x10000, v=0x20000, dtype=0, n_blocks=8, block_size=16, n_kv_heads=2, head_dim=64, k_scale=1.0, v_scale=1.0)
    f.update(kw)
    return qzo.KvCacheDesc(*[f[n] for n, _ in qzo.KvCacheDesc._fields_])


def _refused(call, good, changes):
    qzo = _lib()
    assert call(**good) in (qzo.QZO_OK, qzo.ERR_UNSUPPORTED_DEVICE), "the unchanged call is a valid one"
    for change in changes:
        assert call(**{**good, **change}) == qzo.ERR_BAD_ARG, change


@made_up
def test_beam_select_refusals():
    qzo = _lib()
    need = qzo.qzo_beam_select_workspace_bytes(3, 4, 1000)
    assert 0 < need < qzo.qzo_beam_select_workspace_bytes(3, 4, 32000)
    for args in ((0, 4, 10), (1, 0, 10), (1, 33, 10), (1, 4, 0), (1 << 24, 32, 10), (1, 4, (1 << 30) + 1)):
        with pytest.raises(qzo.QzoError):
            qzo.qzo_beam_select_workspace_bytes(*args)

    def call(x, ld, n, rows, s, last, end, lens, power, B, W, V, p, t, so, lo, ws=P, b=need):
        return qzo._lib.qzo_beam_select(x, ld, n, rows, s, last, end, lens, power, B, W, V, p, t, so, lo, ws, b, None, None)
    good = dict(x=P, ld=1000, n=12, rows=NONE, s=P, last=NONE, end=2, lens=NONE, power=0.0, B=3, W=4, V=1000, p=P, t=P, so=P, lo=NONE)
    bad = [{n: v} for n in ("x", "s", "p", "t", "so") for v in (NONE, ODD)] + [{n: ODD} for n in ("rows", "last", "lens", "lo")]
    bad += [dict(ld=999), dict(n=11), dict(n=0), dict(B=0), dict(W=0), dict(W=33), dict(V=0), dict(power=1.0), dict(lo=P), dict(power=-0.5, lens=P),
            dict(power=8.5, lens=P), dict(power=float("nan"), lens=P)]
    _refused(call, good, bad)
    for change in (dict(n=1, rows=P), dict(lens=P, power=8.0), dict(lens=P, lo=P, last=P)):
        assert call(**{**good, **change}) in (qzo.QZO_OK, qzo.ERR_UNSUPPORTED_DEVICE)
    for change in (dict(ws=NONE), dict(b=need - 1), dict(ws=ctypes.c_void_p(0x10080))):
        assert call(**{**good, **change}) == qzo.ERR_WORKSPACE


@made_up
def test_fork_compact_and_copy_refusals():
    lib = _lib()._lib

    def fork(lens=P, par=P, B=4, tab=P, w=4, bs=16, n=64, free=P, cap=64, cnt=P, lo=P, to=Q, co=P, cp=P, cc=P):
        return lib.qzo_fork_requests(lens, par, B, tab, w, bs, n, free, cap, cnt, lo, to, co, cp, cc, None, None)
    table = [dict(B=0), dict(B=4097), dict(w=0), dict(w=(1 << 26) + 1), dict(bs=8), dict(bs=24), dict(bs=512), dict(n=0), dict(n=524289), dict(cap=0)]
    names = ("lens", "par", "tab", "free", "cnt", "lo", "to", "co", "cp", "cc")
    _refused(fork, {}, [{n: v} for n in names for v in (NONE, ODD)] + table + [dict(to=P)])

    def compact(lens=P, B=4, tab=P, w=4, bs=16, n=64, keep=32, to=P, free=P, cap=64, co=P, cp=P, most=64, cc=P):
        return lib.qzo_compact_blocks(lens, B, tab, w, bs, n, keep, to, free, cap, co, cp, most, cc, None, None)
    names = ("lens", "tab", "to", "free", "co", "cp", "cc")
    _refused(compact, {}, [{n: v} for n in names for v in (NONE, ODD)] + table + [dict(keep=0), dict(keep=65), dict(most=0), dict(most=524289)])

    def copy(caches=(_cache(), _cache()), cp=P, cc=P, most=8):
        arr = (type(caches[0]) * len(caches))(*caches) if caches else None
        return lib.qzo_copy_blocks(arr, len(caches), cp, cc, most, None, None)
    bad = [dict(cp=NONE), dict(cp=ODD), dict(cc=NONE), dict(cc=ODD), dict(most=0), dict(most=524289), dict(caches=())]
    other = (dict(n_blocks=9), dict(block_size=32), dict(n_kv_heads=4), dict(head_dim=128), dict(dtype=4), dict(k=0), dict(v=0x20008), dict(dtype=1), dict(k_scale=2.0))
    _refused(copy, {}, bad + [dict(caches=(_cache(), _cache(**c))) for c in other] + [dict(caches=(_cache(**c), _cache())) for c in other])


@made_up
def test_shared_prefix_attention_refusals():
    qzo = _lib()
    sizes = {}
    for path in (0, 1, 2, 3):
        qzo.qzo_debug_prefix_path(path)
        sizes[path] = qzo.qzo_shared_prefix_attention_workspace_bytes(3, 2, 4, 2, 64, 64)
    qzo.qzo_debug_prefix_path(0)
    assert sizes[0] == sizes[1] == 0 < sizes[2] < sizes[3]              # by rule, little that is shared stays with the rows
    assert qzo.qzo_shared_prefix_attention_workspace_bytes(64, 1, 32, 32, 128, 4096) > 0
    for path in (-1, 4):
        with pytest.raises(qzo.QzoError):
            qzo.qzo_debug_prefix_path(path)
    for args in ((0, 1, 4, 2, 64, 64), (1, 0, 4, 2, 64, 64), (1, 1, 3, 2, 64, 64), (1, 1, 4, 0, 64, 64), (1, 1, 4, 2, 80, 64), (1, 1, 4, 2, 64, 0),
                 (1, 1, 4, 2, 64, (1 << 30) + 1), (1, (1 << 20) + 1, 4, 2, 64, 64)):
        with pytest.raises(qzo.QzoError):
            qzo.qzo_shared_prefix_attention_workspace_bytes(*args)

    def call(q, ldq, cache, tab, n, w, seq, pos, rows, pseq, plen, g, scale, out, ldo, R, H, ws=NONE, b=0, status=NONE):
        return qzo._lib.qzo_shared_prefix_attention(q, ldq, None if cache is None else ctypes.byref(cache), tab, n, w, seq, pos, rows, pseq, plen, g, scale, out,
                                                    ldo, R, H, ws, b, status, None)
    good = dict(q=P, ldq=256, cache=_cache(), tab=P, n=3, w=4, seq=NONE, pos=P, rows=P, pseq=P, plen=P, g=2, scale=0.125, out=Q, ldo=256, R=3, H=4)
    bad = [{n: v} for n in ("q", "tab", "pos", "rows", "pseq", "plen", "out") for v in (NONE, ODD)] + [dict(seq=ODD), dict(status=ODD)]
    bad += [dict(ldq=248), dict(ldq=260), dict(ldo=64), dict(n=0), dict(w=0), dict(w=(1 << 26) + 1), dict(R=0), dict(R=4), dict(H=3), dict(H=0), dict(g=0), dict(g=(1 << 20) + 1),
            dict(scale=0.0), dict(scale=float("nan")), dict(cache=None)]
    caches = (dict(k=0), dict(v=0x20008), dict(dtype=1), dict(block_size=8), dict(head_dim=96), dict(k_scale=2.0), dict(dtype=4, v_scale=0.0), dict(n_blocks=1 << 27))
    assert call(**good) in (qzo.QZO_OK, qzo.ERR_UNSUPPORTED_DEVICE)
    for change in bad + [dict(cache=_cache(**c)) for c in caches]:
        assert call(**{**good, **change}) == qzo.ERR_BAD_ARG, change


@made_up
def test_decode_of_groups_refuses_before_the_model_is_looked_at():
    lib, qzo = _lib()._lib, _lib()
    def call(m=NONE, tok=P, seq=P, pos=P, slots=P, tab=P, rows=P, pseq=P, plen=P, n=2, out=P):
        return lib.qzo_decode_groups(m, ctypes.byref(_cache()), tok, seq, pos, slots, 2, tab, 2, 4, rows, pseq, plen, n, out)
    for change in [{n: v} for n in ("tok", "seq", "pos", "slots", "tab", "rows", "pseq", "plen") for v in (NONE, ODD)] + [dict(n=0), dict(n=(1 << 20) + 1), dict(out=NONE), dict(m=NONE)]:
        assert call(**change) == qzo.ERR_BAD_ARG, change


def test_the_binding_names_the_limits_of_the_header():
    qzo = _lib()
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qzo.h")).read()
    for name in ("MAX_BEAMS", "MAX_POOL_BLOCKS"):
        assert getattr(qzo, name) == int(re.search(rf"#define QZO_{name} (\d+)", header).group(1))


def test_candidates_of_a_beam_whose_ranks_round_to_one_stay_in_the_order_of_their_logits():
    x = np.full((3, 50), -1.0)
    x[:, [10, 20, 30, 40]] = 0.0, 1e-18, 2e-18, 2e-18
    picked = lambda *scores: [(p, t) for p, t, *_ in oracle.beam_select(x, np.array([scores]))[0]]  # noqa: E731
    assert picked(-1.0, -math.inf, -math.inf) == [(0, 30), (0, 40), (0, 20)]      # equal logits: by token
    x[:, [30, 20]] = 0.01, 0.02
    assert picked(-1e15, -math.inf, -math.inf) == [(0, 20), (0, 30), (0, 40)]
    assert picked(-math.inf, -1e18, -1e18) == [(1, 20), (1, 30), (1, 40)]         # equal ranks of several beams: by beam


def test_a_workspace_for_the_largest_call_is_one_for_smaller_calls():
    qzo = _lib()
    size = qzo.qzo_shared_prefix_attention_workspace_bytes
    rng = np.random.default_rng(3)
    shapes = [(64, 64, 32, 32, 128, 2048), (64, 8, 32, 32, 128, 2048), (64, 2, 32, 32, 128, 2048), (128, 16, 32, 4, 128, 16384), (9, 1, 64, 1, 64, 70000)]
    for R, n, H, Hkv, dh, longest in shapes + [(int(rng.integers(1, 300)), int(rng.integers(1, 300)), 8 * g, 8, 128, int(rng.integers(1, 30000))) for g in (1, 2, 5, 12) for _ in range(5)]:
        most = size(R, n, H, Hkv, dh, longest)
        for _ in range(200):
            fewer = int(rng.integers(1, R + 1)), int(rng.integers(1, n + 1)), H, Hkv, dh, int(rng.integers(1, longest + 1))
            assert size(*fewer) <= most, (R, n, H, Hkv, dh, longest, fewer)
        assert most <= 4 * (dh + 2) * (5 * R * H + 8 * 296 * 16)     # results of every query, own keys in four splits, what the SMs hold eight times
