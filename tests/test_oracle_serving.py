"""Pins of the serving oracle (no GPU) and the refusals of the serving entry points, which come before any device call."""
import ctypes

import numpy as np
import pytest

from oracle import model as omodel, serving


def test_paged_attention_over_a_scattered_cache_is_causal_attention():
    rng = np.random.default_rng(3)
    B, S, H, dh, block = 2, 37, 4, 64, 16
    q, k, v = (rng.standard_normal((B, S, H, dh)) for _ in range(3))
    want = omodel.causal_attention(q, k, v)
    width = -(-S // block)
    ids = rng.permutation(B * width + 3)[:B * width].reshape(B, width)
    kp, vp = (np.full((B * width + 3, H, block, dh), np.nan) for _ in range(2))
    for b in range(B):
        slots = [int(ids[b, t // block]) * block + t % block for t in range(S)]
        serving.write_cache(kp, k[b], slots)
        serving.write_cache(vp, v[b], slots)
    row_seq = np.repeat(np.arange(B), S)
    got, _ = serving.paged_attention(q.reshape(B * S, H, dh), kp, vp, ids, row_seq, np.tile(np.arange(S), B), dh ** -0.5)
    np.testing.assert_allclose(got.reshape(B, S, H, dh), want, rtol=1e-12, atol=1e-12)


def test_rotation_is_the_models_and_the_norm_has_unit_rms():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((1, 9, 3, 64))
    np.testing.assert_allclose(serving.rotate(x[0], np.arange(9), 10000.0), omodel.rope(x, 10000.0)[0], rtol=1e-13, atol=1e-13)
    q, _ = serving.qk_norm_rope(x[0], x[0], np.arange(9) + 500, np.ones(64), None, 1e-12, 10000.0)
    np.testing.assert_allclose((q * q).mean(-1), 1.0, rtol=1e-9)


def test_assigned_slots_are_distinct_and_blocks_are_kept():
    rng = np.random.default_rng(5)
    B, width, block, cap = 5, 6, 16, 24
    table, free = np.full((B, width), -1), np.arange(cap)
    lens, count, owner = [0] * B, cap, {}
    for _ in range(200):
        new = [int(rng.integers(-1, 20)) if rng.random() < 0.7 else 1 for _ in range(B)]
        st = serving.assign_slots(lens, new, table, free, count, block, 64)
        if st is None:
            new = [-1] * B
            st = serving.assign_slots(lens, new, table, free, count, block, 64)
        for r, a in enumerate(new):
            if a < 0:
                owner = {s: o for s, o in owner.items() if o[0] != r}
        for s, r, p in zip(st["slots"], st["row_seq"], st["positions"]):
            if s >= 0:
                assert s not in owner
                owner[s] = (r, p)
        lens, count, table, free = st["lens"], st["free_count"], st["table"], st["free"]
        held = [b for r in range(B) for b in table[r, :-(-lens[r] // block)]]
        assert sorted(held + list(free[:count])) == list(range(cap))
        assert sorted(owner.values()) == [(r, p) for r in range(B) for p in range(lens[r])]


# ---- refusals: a wrong argument is turned away before the device is touched ----

P = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10002)
NONE = ctypes.c_void_p(0)


def _lib():
    from paper_2505_13430_b200 import qzo
    return qzo


def _cache(**kw):
    qzo = _lib()
    f = dict(k=0x10000, v=0x20000, dtype=0, n_blocks=8, block_size=16, n_kv_heads=2, head_dim=64, k_scale=1.0, v_scale=1.0)
    f.update(kw)
    return qzo.KvCacheDesc(*[f[n] for n, _ in qzo.KvCacheDesc._fields_])


BAD_CACHES = (dict(k=0), dict(v=0x20008), dict(dtype=1), dict(n_blocks=0), dict(block_size=8), dict(block_size=48), dict(block_size=512),
              dict(n_kv_heads=0), dict(head_dim=96), dict(k_scale=2.0), dict(dtype=4, v_scale=0.0), dict(dtype=4, k_scale=float("inf")),
              dict(n_blocks=1 << 27))


def _refused(call, good, changes):
    qzo = _lib()
    assert call(**good) in (qzo.QZO_OK, qzo.ERR_UNSUPPORTED_DEVICE), "the unchanged call is a valid one"
    for change in changes:
        assert call(**{**good, **change}) == qzo.ERR_BAD_ARG, change


def _no_gpu():
    import torch
    return not torch.cuda.is_available()


pytestmark = pytest.mark.skipif(not _no_gpu(), reason="made-up pointers: only where no device would follow them")


def test_gemv_refusals():
    def call(x, ldx, w, s, b, y, ldy, M, K, N):
        return _lib()._lib.qzo_gemv_int4(x, ldx, w, s, b, y, ldy, M, K, N, None)
    good = dict(x=P, ldx=256, w=P, s=P, b=NONE, y=P, ldy=64, M=2, K=256, N=64)
    _refused(call, good, [dict(x=NONE), dict(w=NONE), dict(s=NONE), dict(y=NONE), dict(x=ODD), dict(w=ODD), dict(s=ODD), dict(b=ODD), dict(M=0), dict(M=17),
                          dict(K=0), dict(K=252), dict(N=0), dict(N=60), dict(ldx=248), dict(ldx=260), dict(ldy=56)])


def test_rope_table_refusals():
    def call(t, n, dh, th):
        return _lib()._lib.qzo_rope_table(t, n, dh, th, None)
    _refused(call, dict(t=P, n=64, dh=64, th=1e4), [dict(t=NONE), dict(n=0), dict(dh=96), dict(th=0.0), dict(th=float("nan")),
                                                    dict(n=1 << 25), dict(t=ODD)])


def test_qk_norm_rope_cache_refusals():
    def call(q, ldq, k, ldk, v, ldv, qg, kg, eps, tab, mp, pos, slots, out, ldo, cache, T, H):
        return _lib()._lib.qzo_qk_norm_rope_cache(q, ldq, k, ldk, v, ldv, qg, kg, eps, tab, mp, pos, slots, out, ldo,
                                                  None if cache is None else ctypes.byref(cache), T, H, None, None)
    good = dict(q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, qg=P, kg=NONE, eps=1e-5, tab=P, mp=64, pos=P, slots=P, out=P, ldo=256,
                cache=_cache(), T=3, H=4)
    bad = [dict(q=NONE), dict(k=NONE), dict(v=NONE), dict(pos=NONE), dict(slots=NONE), dict(out=NONE), dict(q=ODD), dict(out=ODD), dict(qg=ODD),
           dict(tab=ODD), dict(eps=0.0), dict(mp=0), dict(T=0), dict(H=0), dict(H=3), dict(ldq=252), dict(ldq=258), dict(ldk=64),
           dict(ldv=64), dict(ldo=128), dict(ldo=260), dict(cache=None)]
    _refused(call, good, bad + [dict(cache=_cache(**c)) for c in BAD_CACHES])


def test_paged_attention_refusals():
    qzo = _lib()
    def call(q, ldq, cache, tab, n, w, seq, pos, scale, out, ldo, R, H, ws, b):
        return qzo._lib.qzo_paged_attention(q, ldq, None if cache is None else ctypes.byref(cache), tab, n, w, seq, pos, scale, out, ldo, R,
                                            H, ws, b, None, None)
    good = dict(q=P, ldq=256, cache=_cache(), tab=P, n=3, w=4, seq=NONE, pos=P, scale=0.125, out=ctypes.c_void_p(0x20000), ldo=256, R=3, H=4,
                ws=NONE, b=0)
    bad = [dict(q=NONE), dict(tab=NONE), dict(pos=NONE), dict(out=NONE), dict(q=ODD), dict(out=ODD), dict(ldq=248), dict(ldq=260), dict(ldo=64),
           dict(n=0), dict(w=0), dict(w=(1 << 26) + 1), dict(R=0), dict(R=4), dict(H=3), dict(H=0), dict(scale=0.0), dict(scale=float("nan")),
           dict(cache=None)]
    _refused(call, good, bad + [dict(cache=_cache(**c)) for c in BAD_CACHES])
    # workspace: asked for where a long cache is split
    need = qzo.qzo_paged_attention_workspace_bytes(1, 4, 2, 64, 1 << 16)
    assert need > 0 and qzo.qzo_paged_attention_workspace_bytes(3, 4, 2, 64, 64) == 0
    for args in ((0, 4, 2, 64, 64), (1, 3, 2, 64, 64), (1, 4, 0, 64, 64), (1, 4, 2, 80, 64), (1, 4, 2, 64, 0), (1, 4, 2, 64, (1 << 30) + 1)):
        with pytest.raises(qzo.QzoError):
            qzo.qzo_paged_attention_workspace_bytes(*args)


def test_index_arrays_off_their_boundary_are_refused():
    lib = _lib()._lib
    cache = _cache()
    def rope(pos=P, slots=P, status=NONE):
        return lib.qzo_qk_norm_rope_cache(P, 256, P, 128, P, 128, NONE, NONE, 0.0, NONE, 0, pos, slots, P, 256, ctypes.byref(cache), 3, 4, status, None)
    def attend(tab=P, seq=NONE, pos=P, status=NONE):
        return lib.qzo_paged_attention(P, 256, ctypes.byref(cache), tab, 3, 4, seq, pos, 0.1, ctypes.c_void_p(0x20000), 256, 3, 4, NONE, 0, status, None)
    def slots(lens=P, new=P, tab=P, free=P, cnt=P, a=P, b=P, c=P, lo=P, co=P, status=NONE):
        return lib.qzo_assign_slots(lens, new, 4, tab, 4, 16, free, 16, cnt, 8, a, b, c, lo, co, status, None)
    for call in (rope, attend, slots):
        names = call.__code__.co_varnames[:call.__code__.co_argcount]
        _refused(call, {}, [{n: ODD} for n in names])


def test_gains_and_angles_off_their_32_bytes_are_refused():
    cache, half = _cache(), ctypes.c_void_p(0x10010)
    def rope(qg=P, kg=P, tab=P):
        return _lib()._lib.qzo_qk_norm_rope_cache(P, 256, P, 128, P, 128, qg, kg, 1e-5, tab, 64, P, P, P, 256, ctypes.byref(cache), 3, 4, NONE, None)
    _refused(rope, {}, [dict(qg=half), dict(kg=half), dict(tab=half)])


def test_a_table_off_its_32_bytes_is_refused_where_it_is_made():
    def call(t):
        return _lib()._lib.qzo_rope_table(t, 64, 64, 1e4, None)
    _refused(call, dict(t=P), [dict(t=ctypes.c_void_p(0x10010)), dict(t=ctypes.c_void_p(0x10008))])


def test_scales_whose_reciprocal_or_product_leaves_fp32_are_refused():
    qzo = _lib()
    def rope(cache):
        return qzo._lib.qzo_qk_norm_rope_cache(P, 256, P, 128, P, 128, NONE, NONE, 0.0, NONE, 0, P, P, P, 256, ctypes.byref(cache), 3, 4, None, None)
    def attend(cache, scale):
        return qzo._lib.qzo_paged_attention(P, 256, ctypes.byref(cache), P, 3, 4, NONE, P, scale, ctypes.c_void_p(0x20000), 256, 3, 4, NONE, 0, None, None)
    for side in ("k_scale", "v_scale"):
        _refused(rope, dict(cache=_cache(dtype=4, **{side: 2.0 ** -64})),
                 [dict(cache=_cache(dtype=4, **{side: v})) for v in (1e-40, 2.0 ** -65, 2.0 ** 65, -1.0, float("nan"))])
    _refused(attend, dict(cache=_cache(dtype=4, k_scale=2.0 ** 64), scale=2.0 ** 40),
             [dict(scale=s) for s in (2.0 ** 41, 2.0 ** -41, -1.0, float("inf"))])


def test_assign_slots_refusals():
    def call(lens, new, B, tab, w, bs, free, cap, cnt, rows, a, b, c, lo, co):
        return _lib()._lib.qzo_assign_slots(lens, new, B, tab, w, bs, free, cap, cnt, rows, a, b, c, lo, co, None, None)
    good = dict(lens=P, new=P, B=4, tab=P, w=4, bs=16, free=P, cap=16, cnt=P, rows=8, a=P, b=P, c=P, lo=P, co=P)
    bad = [{n: NONE} for n in ("lens", "new", "tab", "free", "cnt", "a", "b", "c", "lo", "co")]
    bad += [dict(B=0), dict(B=4097), dict(w=0), dict(bs=8), dict(bs=24), dict(cap=0), dict(rows=0), dict(rows=(1 << 30) + 1), dict(w=1 << 28), dict(cap=1 << 28)]
    _refused(call, good, bad)


def test_the_binding_names_the_limits_of_the_header():
    import os
    import re
    qzo = _lib()
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qzo.h")).read()
    for name in ("GEMV_MAX_ROWS", "MAX_REQUESTS"):
        assert getattr(qzo, name) == int(re.search(rf"#define QZO_{name} (\d+)", header).group(1))
