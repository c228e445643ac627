"""GPU parity of the serving operators against the fp64 oracle, element by element, with bounds that follow from the
arithmetic: every rounding counts half a step (bf16 2^-8, e4m3 2^-4 of the value), fp32 sums what their terms allow."""
import numpy as np
import pytest
import torch

from oracle import int4, linear as olinear, serving
from paper_2505_13430_b200 import inputs

pytestmark = pytest.mark.gpu

BF16_STEP, F16_STEP, F32_STEP = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    from paper_2505_13430_b200 import qzo
    return qzo


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _randn(shape, seed, std=1.0):
    return inputs.normal_fp32(shape, std, seed).bfloat16()


# ------------------------------------------------------------------ matrix-vector products

GEMV_CASES = [(1, 128, 8), (1, 64, 128), (3, 8, 16), (1, 256, 688), (2, 688, 256), (5, 1032, 136), (8, 4096, 384), (9, 200, 72), (16, 1920, 1000),
              (1, 4096, 4096), (7, 11008, 264), (16, 72, 2056), (12, 13824, 128),
              (10, 384, 4808), (4, 1096, 4808), (1, 136, 9608)]


def _gemv_case(lib, M, K, N, seed):
    x, q, s = inputs.gemm_case(M, K, N, seed=seed)
    wq = lib.qzo_repack_int4(torch.from_numpy(int4.pack_int4(q.numpy()).view(np.int32)).cuda(), K, N)
    return x, q, s, wq


def _gemv_check(got, x, q, s, bias=None):
    x, q = f64(x), q.numpy().astype(np.float64)
    K, N = q.shape
    w = f64(s)[np.arange(K) // 128] * q
    want = x @ w + (0 if bias is None else f64(bias))
    # products exact; a chain of at most K/128 + 9 sums of up to 16 terms each, truncated at worst (one whole step each)
    size = np.abs(x) @ np.abs(w) + (0 if bias is None else np.abs(f64(bias)))
    allowed = BF16_STEP * np.abs(want) + (128 + K / 128 + 16) * 2 * F32_STEP * size * (1 + BF16_STEP)
    off = np.abs(f64(got) - want)
    assert (off <= allowed).all(), (off / allowed).max()


@pytest.mark.parametrize("M,K,N", GEMV_CASES)
def test_gemv_matches_oracle(lib, M, K, N):
    x, q, s, wq = _gemv_case(lib, M, K, N, M + K + N)
    bias = inputs.normal_fp32((N,), 0.5, 3) if N % 16 else None
    y = lib.qzo_gemv_int4(x.cuda(), wq, s.cuda(), K, N, bias=None if bias is None else bias.cuda())
    _gemv_check(y, x, q, s, bias)
    again = lib.qzo_gemv_int4(x.cuda(), wq, s.cuda(), K, N, bias=None if bias is None else bias.cuda())
    assert torch.equal(y.view(torch.int16), again.view(torch.int16))
    ref = olinear.perturbed_linear(f64(x), q.numpy(), f64(s), 0, 0, 0, 1e-3, None if bias is None else bias.numpy())
    assert np.abs(f64(y) - ref).max() <= 2e-2 * np.abs(ref).max()


def test_gemv_strides_leave_the_rest_alone(lib):
    M, K, N = 6, 688, 264
    x, q, s, wq = _gemv_case(lib, M, K, N, 1)
    wide = torch.full((M, K + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :K] = x.cuda()
    out = torch.full((M, N + 7), 5.0, dtype=torch.bfloat16, device="cuda")
    lib.qzo_gemv_int4(wide[:, :K], wq, s.cuda(), K, N, y=out[:, :N])
    _gemv_check(out[:, :N], x, q, s)
    assert (out[:, N:] == 5.0).all()


def test_gemv_extreme_activations(lib):
    # one huge activation beside small ones, rows of zeros, and rows that hold an infinity or a NaN beside clean ones
    M, K, N = 5, 512, 128
    x, q, s, wq = _gemv_case(lib, M, K, N, 2)
    x[0, 77] = 3e37
    x[1] = 0
    x[2, 5] = float("inf")
    x[3, 300] = float("nan")
    y = lib.qzo_gemv_int4(x.cuda(), wq, s.cuda(), K, N)
    _gemv_check(y[[0, 1, 4]], x[[0, 1, 4]], q, s)
    with np.errstate(invalid="ignore"):
        col = f64(s)[0] * q[5].numpy().astype(np.float64) * np.inf
    got = f64(y[2])
    assert np.array_equal(np.isnan(got), np.isnan(col)) and np.array_equal(got[~np.isnan(col)], col[~np.isnan(col)])
    assert torch.isnan(y[3]).all()


# ------------------------------------------------------------------ head norms, rotation, cache write

CACHES = {"bf16": (torch.bfloat16, 1.0, 1.0), "e4m3": (torch.float8_e4m3fn, 0.25, 0.5)}


def _pages(kind, shape, seed, std=1.0):
    dt, ks, vs = CACHES[kind]
    k = (inputs.normal_fp32(shape, std, seed) / ks).to(dt).cuda()
    v = (inputs.normal_fp32(shape, std, seed + 1) / vs).to(dt).cuda()
    return k, v, ks, vs


ROPE_CASES = [
    # T, padding rows, H, Hkv, dh, block, cache, q gain, k gain, rotation
    (1, 0, 4, 4, 64, 16, "bf16", False, False, True),
    (1, 0, 1, 1, 128, 16, "e4m3", True, True, True),
    (7, 2, 8, 2, 128, 32, "bf16", True, True, True),
    (33, 5, 12, 4, 64, 16, "e4m3", True, False, True),
    (50, 0, 5, 1, 128, 256, "bf16", False, True, False),
    (257, 40, 32, 8, 128, 64, "e4m3", True, True, True),
    (19, 19, 4, 4, 64, 16, "bf16", True, True, True),
    (600, 3, 3, 3, 64, 128, "bf16", False, False, False),
]


@pytest.mark.parametrize("T,pad,H,Hkv,dh,block,kind,qg,kg,rot", ROPE_CASES)
def test_qk_norm_rope_cache_matches_oracle(lib, T, pad, H, Hkv, dh, block, kind, qg, kg, rot):
    rng = np.random.default_rng(T)
    n_blocks = -(-T // block) + 2
    ck, cv, ks, vs = _pages(kind, (n_blocks, Hkv, block, dh), T)
    before = [f64(ck), f64(cv)]
    qkv = _randn((T, (H + 2 * Hkv) * dh + 8), T + 1, 2.0).cuda()
    q, k, v = (qkv[:, a * dh:b * dh].view(T, b - a, dh) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    max_pos = 70000
    positions = rng.integers(0, max_pos, T).astype(np.int32)
    slots = rng.permutation(n_blocks * block)[:T].astype(np.int32)
    positions[T - pad:], slots[T - pad:] = -1, -1
    if T > 1 and T > pad:
        positions[0] = max_pos - 1
    gains = [1 + inputs.normal_fp32((dh,), 0.2, 9 + i) if on else None for i, on in enumerate((qg, kg))]
    table = lib.qzo_rope_table(max_pos, dh, 10000.0) if rot else None
    q_out = torch.full((T, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = lib.KvCache(ck, cv, ks, vs)
    lib.qzo_qk_norm_rope_cache(q, k, v, torch.from_numpy(positions).cuda(), torch.from_numpy(slots).cuda(), cache,
                               q_gain=None if gains[0] is None else gains[0].cuda(), k_gain=None if gains[1] is None else gains[1].cuda(),
                               norm_eps=1e-5, table=table, q_out=q_out, status=status)
    assert int(status.item()) == 0
    live = T - pad
    assert (q_out[live:] == 7.0).all()
    wq, wk = serving.qk_norm_rope(f64(q)[:live], f64(k)[:live], positions[:live], *(None if g is None else g.numpy() for g in gains), 1e-5,
                                  10000.0 if rot else None)

    def slack(x, gain):   # fp32: the mean's sum, its root, three products and a sum: less than 32 steps of the pair's size
        if gain is not None:
            x = serving.head_norm(x, gain.numpy().astype(np.float64), 1e-5)
        a = np.abs(x)
        return 32 * F32_STEP * (a + np.roll(a, dh // 2, axis=-1))

    got = f64(q_out)[:live]
    assert (np.abs(got - wq) <= BF16_STEP * np.abs(wq) + slack(f64(q)[:live], gains[0])).all()
    for pages, old, rows, extra, scale in ((ck, before[0], wk, slack(f64(k)[:live], gains[1]), ks), (cv, before[1], f64(v)[:live], 0.0, vs)):
        want, room = old.copy(), np.zeros_like(old)
        serving.write_cache(want, np.clip(rows / scale, -448, 448) if kind == "e4m3" else rows, slots[:live])
        serving.write_cache(room, np.broadcast_to(np.asarray(extra) / scale, rows.shape), slots[:live])
        if kind == "e4m3":       # half a step: 2^-4 of the value, 2^-10 where the format's steps stop shrinking
            touched = np.zeros_like(old)
            serving.write_cache(touched, np.ones_like(rows), slots[:live])
            room = room * (1 + 2.0 ** -4) + touched * np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10)
        else:
            touched = np.zeros_like(old)
            serving.write_cache(touched, np.ones_like(rows), slots[:live])
            room = room + touched * BF16_STEP * np.abs(want)
        assert (np.abs(f64(pages) - want) <= room).all()


def test_values_are_stored_exactly_or_saturated(lib):
    T, H, dh = 4, 2, 64
    v = _randn((T, H, dh), 5)
    v[0, 0, :4] = torch.tensor([1000.0, -1000.0, 448.0, 0.0])
    for kind in CACHES:
        ck, cv, ks, vs = _pages(kind, (1, H, 16, dh), 6)
        q = _randn((T, H, dh), 7).cuda()
        i = torch.arange(T, dtype=torch.int32, device="cuda")
        lib.qzo_qk_norm_rope_cache(q, q, v.cuda(), i, i, lib.KvCache(ck, cv, ks, vs))
        want = v.cuda() if kind == "bf16" else (v.float() / vs).clamp(-448, 448).to(torch.float8_e4m3fn).cuda()
        assert torch.equal(cv[0, :, :T].transpose(0, 1).float(), want.float())


def test_queries_in_place_and_bad_indices(lib):
    T, H, dh, block = 5, 4, 128, 16
    ck, cv, ks, vs = _pages("bf16", (2, H, block, dh), 1)
    cache = lib.KvCache(ck, cv, ks, vs)
    table = lib.qzo_rope_table(64, dh, 10000.0)
    q, k, v = (_randn((T, H, dh), 20 + i).cuda() for i in range(3))
    pos = torch.tensor([0, 3, 63, 9, 1], dtype=torch.int32, device="cuda")
    slots = torch.tensor([0, 31, 5, 6, 7], dtype=torch.int32, device="cuda")
    want = lib.qzo_qk_norm_rope_cache(q, k, v, pos, slots, cache, table=table)
    mine = q.clone()
    lib.qzo_qk_norm_rope_cache(mine, k, v, pos, slots, cache, table=table, q_out=mine)
    assert torch.equal(mine, want)
    # a slot beyond the cache is not written, a position beyond the table turns by the nearest; both are reported
    kept = ck.clone(), cv.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.qzo_qk_norm_rope_cache(q, k, v, pos, torch.full_like(slots, 32), cache, table=table, status=status)
    assert int(status.item()) == 2 and torch.equal(ck, kept[0]) and torch.equal(cv, kept[1])
    status.zero_()
    far = lib.qzo_qk_norm_rope_cache(q, k, v, torch.full_like(pos, 64), slots, cache, table=table, status=status)
    assert int(status.item()) == 2
    near = lib.qzo_qk_norm_rope_cache(q, k, v, torch.full_like(pos, 63), slots, cache, table=table)
    assert torch.equal(far, near)


@pytest.mark.parametrize("rot,kind", [(True, "bf16"), (False, "bf16"), (True, "e4m3")])
def test_a_negative_position_is_padding_whatever_its_slot(lib, rot, kind):
    T, H, dh = 4, 2, 64
    ck, cv, ks, vs = _pages(kind, (2, H, 16, dh), 2)
    kept = ck.clone(), cv.clone()
    table = lib.qzo_rope_table(64, dh, 10000.0) if rot else None
    q, k, v = (_randn((T, H, dh), 30 + i).cuda() for i in range(3))
    pos = torch.tensor([0, -1, 5, -2 ** 31], dtype=torch.int32, device="cuda")
    slots = torch.tensor([-1, 3, 4, 31], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((T, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.qzo_qk_norm_rope_cache(q, k, v, pos, slots, lib.KvCache(ck, cv, ks, vs), table=table, q_out=out, status=status)
    assert int(status.item()) == 0
    assert (out[[0, 1, 3]] == 7.0).all() and (out[2] != 7.0).any()
    for pages, old in zip((ck, cv), kept):
        assert not torch.equal(pages[0, :, 4].float(), old[0, :, 4].float())
        pages[0, :, 4] = old[0, :, 4]
        assert torch.equal(pages.float(), old.float())


# ------------------------------------------------------------------ attention over the paged cache

ATTEND_CASES = [
    # rows' last positions, H, Hkv, dh, block, cache, tokens the table has room for beyond the longest
    ([0], 1, 1, 64, 16, "bf16", 0),
    ([0, 1, 15, 16, 17, -1, 62, 63, 64], 4, 4, 64, 16, "bf16", 0),
    ([249], 32, 32, 128, 16, "bf16", 0),
    ([5, -1, 300, 127, 128], 8, 1, 128, 32, "bf16", 1000),
    ([777, 0, 63], 12, 4, 64, 64, "e4m3", 0),
    ([1029], 24, 1, 128, 128, "e4m3", 0),
    ([2500, 1], 40, 8, 128, 16, "bf16", 5000),
    ([4095, 33, -1], 16, 1, 64, 256, "bf16", 0),
    ([9000], 2, 2, 128, 16, "e4m3", 0),
    ([3001], 20, 1, 64, 16, "e4m3", 0),
    ([100, 900] * 20, 2, 1, 128, 16, "bf16", 0),
    ([700], 71, 1, 64, 32, "bf16", 0),
]


def _attend_case(positions, H, Hkv, dh, block, kind, room, seed, q_std=1.0):
    rng = np.random.default_rng(seed)
    R = len(positions)
    width = -(-(max(positions) + 1 + room) // block)
    n_blocks = R * width + 3
    ck, cv, ks, vs = _pages(kind, (n_blocks, Hkv, block, dh), seed)
    table = rng.permutation(n_blocks)[:R * width].reshape(R, width).astype(np.int32)
    # whatever stands behind a request's length is not looked at: NaN in its last page, no block at all behind that
    nan = torch.tensor(float("nan")).to(ck.dtype)
    for r, last in enumerate(positions):
        n = last + 1
        if n % block:
            page = int(table[r, n // block])
            for pages in (ck, cv):
                pages[page, :, n % block:] = nan.cuda()
        table[r, -(-n // block):] = -1
    q = _randn((R, H, dh), seed + 5, q_std)
    return q, ck, cv, ks, vs, table


def _attend_check(got, q, ck, cv, ks, vs, table, row_seq, positions, scale):
    kp, vp = f64(ck) * ks, f64(cv) * vs
    want, spread = serving.paged_attention(f64(q), kp, vp, table, row_seq, positions, scale)
    dh = q.shape[-1]
    kmax = np.nanmax(np.abs(kp[np.unique(table[table >= 0])])) if (table >= 0).any() else 0.0
    # score: dh exact products summed in fp32, one scaling; weight: exp2 within 4 steps, its rounding to 16 bits
    score = np.abs(f64(q)).sum(-1, keepdims=True) * kmax * scale * (dh / 16 + 18) * 2 * F32_STEP
    p_step = BF16_STEP if ck.dtype == torch.bfloat16 else F16_STEP
    keys = max(positions) + 1
    allowed = BF16_STEP * np.abs(want) + (p_step + 2 * score + (16 + keys / 8) * F32_STEP) * spread * (1 + BF16_STEP) + 1e-30
    off = np.abs(f64(got) - want)
    assert (off <= allowed).all(), (off / allowed).max()


@pytest.mark.parametrize("positions,H,Hkv,dh,block,kind,room", ATTEND_CASES)
def test_paged_attention_matches_oracle(lib, positions, H, Hkv, dh, block, kind, room):
    q, ck, cv, ks, vs, table = _attend_case(positions, H, Hkv, dh, block, kind, room, 100 + len(positions) + H)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (q.cuda(), lib.KvCache(ck, cv, ks, vs), torch.from_numpy(table).cuda(), torch.tensor(positions, dtype=torch.int32, device="cuda"))
    out = lib.qzo_paged_attention(*args, status=status)
    assert int(status.item()) == 0
    _attend_check(out, q, ck, cv, ks, vs, table, np.arange(len(positions)), positions, dh ** -0.5)
    for r, last in enumerate(positions):
        if last < 0:
            assert (out[r] == 0).all()
    again = lib.qzo_paged_attention(*args)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("dh,kind", [(64, "bf16"), (128, "bf16"), (128, "e4m3")])
def test_many_rows_of_different_lengths(lib, dh, kind):
    # more rows than the SMs hold, whose keys are taken in pieces of equal length: rows that need none, one and several
    longest = [9000, 4501, 77]
    q, ck, cv, ks, vs, table = _attend_case([n - 1 for n in longest], 4, 4, dh, 16, kind, 0, 21)
    rng = np.random.default_rng(2)
    R = 150
    row_seq = rng.integers(0, 3, R).astype(np.int32)
    positions = np.array([rng.integers(-1, longest[s] if r % 5 == 0 else min(longest[s], 300)) for r, s in enumerate(row_seq)], dtype=np.int32)
    row_seq[:2], positions[:2] = [0, 1], [8999, 4500]
    q = _randn((R, 4, dh), 22)
    assert lib.qzo_paged_attention_workspace_bytes(R, 4, 4, dh, table.shape[1] * 16) > 0
    out = lib.qzo_paged_attention(q.cuda(), lib.KvCache(ck, cv, ks, vs), torch.from_numpy(table).cuda(), torch.from_numpy(positions).cuda(),
                                  row_seq=torch.from_numpy(row_seq).cuda())
    _attend_check(out, q, ck, cv, ks, vs, table, row_seq, positions.tolist(), dh ** -0.5)


@pytest.mark.parametrize("kind,H,Hkv", [("bf16", 4, 4), ("e4m3", 16, 2)])
def test_peaked_scores_and_a_given_scale(lib, kind, H, Hkv):
    # large scores: the maximum moves from tile to tile and single keys carry a row
    positions = [500, 1800]
    q, ck, cv, ks, vs, table = _attend_case(positions, H, Hkv, 128, 16, kind, 0, 7, q_std=20.0)
    out = lib.qzo_paged_attention(q.cuda(), lib.KvCache(ck, cv, ks, vs), torch.from_numpy(table).cuda(),
                                  torch.tensor(positions, dtype=torch.int32, device="cuda"), scale=0.3)
    _attend_check(out, q, ck, cv, ks, vs, table, np.arange(2), positions, 0.3)


def test_rows_of_one_request_and_strided_rows(lib):
    # a prompt's rows: each sees the keys up to its own; queries and outputs inside wider rows
    H, Hkv, dh, block, S = 8, 2, 64, 16, 70
    q, ck, cv, ks, vs, table = _attend_case([S - 1, 30], H, Hkv, dh, block, "bf16", 0, 8)
    rows = np.concatenate([np.arange(S), [30, -1]]).astype(np.int32)
    row_seq = np.concatenate([np.zeros(S), [1, -1]]).astype(np.int32)
    R = len(rows)
    wide = torch.full((R, H * dh + 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    q = _randn((R, H, dh), 9)
    wide[:, :H * dh] = q.view(R, -1).cuda()
    out = torch.full((R, H * dh + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.qzo_paged_attention(wide[:, :H * dh].view(R, H, dh), lib.KvCache(ck, cv, ks, vs), torch.from_numpy(table).cuda(),
                            torch.from_numpy(rows).cuda(), row_seq=torch.from_numpy(row_seq).cuda(), out=out[:, :H * dh].view(R, H, dh),
                            status=status)
    assert int(status.item()) == 0 and (out[:, H * dh:] == 3.0).all()
    _attend_check(out[:, :H * dh].reshape(R, H, dh), q, ck, cv, ks, vs, table, row_seq, rows, dh ** -0.5)


def test_infinite_scores_of_live_keys(lib):
    # keys that score -inf carry no weight; a row with nothing but such keys gives zeros; NaN keys make the row NaN
    H, dh, block = 2, 64, 16
    positions = [300, 40, 200]
    q, ck, cv, ks, vs, table = _attend_case(positions, H, H, dh, block, "bf16", 0, 11)
    q = q.abs() + 0.1
    ninf = float("-inf")
    for page in table[0][:9]:
        ck[int(page)] = ninf
    for page in table[1]:
        ck[int(page)] = ninf
    ck[int(table[2, 3]), 0, 5] = float("nan")
    out = lib.qzo_paged_attention(q.cuda(), lib.KvCache(ck, cv, ks, vs), torch.from_numpy(table).cuda(),
                                  torch.tensor(positions, dtype=torch.int32, device="cuda"))
    short = table[:1, 9:].copy()
    _attend_check(out[:1], q[:1], ck, cv, ks, vs, short, np.zeros(1, int), [300 - 9 * block], dh ** -0.5)
    assert (out[1] == 0).all()
    assert torch.isnan(out[2, 0]).all() and not torch.isnan(out[2, 1]).any()


def test_blocks_and_requests_out_of_range_are_reported_and_not_read(lib):
    H, dh, block = 2, 128, 16
    positions = [100, 100, 100, 100]
    q, ck, cv, ks, vs, table = _attend_case(positions, H, H, dh, block, "bf16", 0, 12)
    bad = table.copy()
    bad[0, 2] = ck.shape[0]               # a block beyond the cache: its keys are not seen
    bad[1, :] = -5                        # no block at all
    row_seq = np.array([0, 1, 2, 9], np.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pos = torch.tensor([100, 100, 1000, 100], dtype=torch.int32, device="cuda")
    out = lib.qzo_paged_attention(q.cuda(), lib.KvCache(ck, cv, ks, vs), torch.from_numpy(bad).cuda(), pos,
                                  row_seq=torch.from_numpy(row_seq).cuda(), status=status)
    assert int(status.item()) == 2
    assert (out[1] == 0).all() and (out[3] == 0).all()
    gone = np.delete(table[:1], 2, axis=1)
    _attend_check(out[:1], q[:1], ck, cv, ks, vs, gone, np.zeros(1, int), [100 - block], dh ** -0.5)
    # a position beyond the table sees the table's tokens: here NaN stands behind the request's own
    assert torch.isnan(out[2]).all()


def test_caches_beyond_32_bit_offsets(lib):
    # pages at the far end of a cache of more than 2^32 bytes per side
    Hkv, block, dh = 32, 16, 128
    n_blocks = (2 ** 32 + 2 ** 28) // (Hkv * block * dh * 2)
    ck = torch.empty((n_blocks, Hkv, block, dh), dtype=torch.bfloat16, device="cuda")
    cv = torch.empty_like(ck)
    S = 40
    table = torch.tensor([[n_blocks - 1, n_blocks - 3, n_blocks - 2]], dtype=torch.int32, device="cuda")
    k, v = _randn((S, Hkv, dh), 1), _randn((S, Hkv, dh), 2)
    pos = torch.arange(S, dtype=torch.int32, device="cuda")
    slots = (table[0, (pos // block).long()] * block + pos % block).to(torch.int32)
    cache = lib.KvCache(ck, cv)
    q = _randn((S, Hkv, dh), 3)
    lib.qzo_qk_norm_rope_cache(q.cuda(), k.cuda(), v.cuda(), pos, slots, cache)
    out = lib.qzo_paged_attention(q[-1:].cuda(), cache, table, pos[-1:])
    small_k, small_v = ck[-3:].clone(), cv[-3:].clone()
    del cache, ck, cv
    _attend_check(out, q[-1:], small_k, small_v, 1.0, 1.0, np.array([[2, 0, 1]]), np.zeros(1, int), [S - 1], dh ** -0.5)


# ------------------------------------------------------------------ slots

def _slots_run(lib, lens, new, table, free, count, block, rows, in_place=True):
    t = [torch.as_tensor(np.asarray(a), dtype=torch.int32, device="cuda").contiguous() for a in (lens, new, table, free, [count])]
    kw = {} if in_place else dict(lens_out=torch.empty_like(t[0]), free_count_out=torch.empty_like(t[4]))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    maps = lib.qzo_assign_slots(*t, block, rows, status=status, **kw)
    lens_out, count_out = (t[0], t[4]) if in_place else (kw["lens_out"], kw["free_count_out"])
    got = dict(zip(("row_seq", "positions", "slots"), maps), lens=lens_out, table=t[2], free=t[3])
    got = {n: v.cpu().numpy() for n, v in got.items()}
    got["free_count"] = int(count_out.item())
    return got, int(status.item())


@pytest.mark.parametrize("B,block,rows,in_place", [(1, 16, 1, True), (3, 16, 50, False), (40, 32, 700, True), (1000, 16, 5000, True),
                                                   (4096, 64, 9000, False), (1025, 128, 2000, True), (64, 16, 40000, True)])
def test_assign_slots_follows_the_oracle_step_after_step(lib, B, block, rows, in_place):
    rng = np.random.default_rng(B)
    width, cap = max(4, 2 * rows // block), 4 * B + 4 * rows // block
    table, free = np.full((B, width), -1, np.int32), rng.permutation(cap).astype(np.int32)
    lens, count, served = np.zeros(B, np.int32), cap, 0
    for step in range(6):
        kind = rng.random(B)
        new = np.where(kind < 0.15, -1, np.where(kind < 0.3, 0, np.where(kind < 0.6, 1, rng.integers(1, max(2, rows // B * 2), B))))
        new[np.cumsum(np.maximum(new, 0)) > rows] = 0
        if step == 4:
            new[-1] = rows + 1            # more rows than there is room for
        want = serving.assign_slots(lens, new, table, free, count, block, rows)
        got, status = _slots_run(lib, lens, new, table, free, count, block, rows, in_place)
        if want is None:
            assert status == 4 and np.array_equal(got["lens"], lens) and got["free_count"] == count
            assert np.array_equal(got["table"], table) and np.array_equal(got["free"], free)
            assert all((got[n] == -1).all() for n in ("row_seq", "positions", "slots"))
            continue
        served += 1
        assert status == 0
        for n in ("row_seq", "positions", "slots", "lens", "table"):
            assert np.array_equal(got[n], want[n]), n
        assert got["free_count"] == want["free_count"]
        assert np.array_equal(got["free"][:got["free_count"]], want["free"][:got["free_count"]])
        lens, table, free, count = got["lens"], got["table"], got["free"], got["free_count"]
    assert served >= 4


@pytest.mark.parametrize("lens,new,count,rows", [([5], [1], 0, 4), ([16], [1], 0, 4), ([-1], [1], 4, 4), ([60], [9], 4, 16), ([0], [5], 4, 4),
                                                 ([0], [2 ** 31 - 1], 4, 4), ([0], [3], -1, 4), ([20], [-1], 3, 4)])
def test_steps_that_cannot_be_served(lib, lens, new, count, rows):
    table, free = np.array([[3, 2, 1, 0]], np.int32), np.array([4, 5, 6, 7], np.int32)
    want = serving.assign_slots(lens, new, table, free, count, 16, rows)
    got, status = _slots_run(lib, lens, new, table, free, count, 16, rows)
    if want is None:
        assert status == 4 and got["lens"][0] == lens[0] and got["free_count"] == count and (got["slots"] == -1).all()
        assert np.array_equal(got["table"], table) and np.array_equal(got["free"], free)
    else:
        assert status == 0 and got["lens"][0] == want["lens"][0] and np.array_equal(got["slots"], want["slots"])


@pytest.mark.parametrize("block", [16, 256])
@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, "first"])
def test_ids_that_no_cache_can_hold_do_not_become_slots(lib, block, bad):
    bad = 2 ** 31 // block if bad == "first" else bad
    # request 0 holds a block with such an id, request 1 takes one from the stack, request 2 is clean
    table = np.array([[bad, -1], [-1, -1], [3, -1]], np.int32)
    got, status = _slots_run(lib, [2, 0, 5], [1, 1, 1], table, [1, bad], 2, block, 4)
    assert status == 0 and got["free_count"] == 1
    assert got["slots"].tolist() == [2 ** 31 - 1, 2 ** 31 - 1, 3 * block + 5, -1]
    assert got["positions"].tolist() == [2, 0, 5, -1] and got["table"][1, 0] == bad
    # the largest id that has slots: the same as any other
    top = 2 ** 31 // block - 1
    got, _ = _slots_run(lib, [0], [2], np.full((1, 1), -1, np.int32), [top], 1, block, 2)
    assert got["slots"].tolist() == [top * block, top * block + 1]


# ------------------------------------------------------------------ streams, graphs, together

def test_operators_on_a_side_stream_and_in_a_replayed_graph(lib):
    H, Hkv, dh, block, B = 8, 2, 128, 16, 3
    M, K, N = B, (H + 2 * Hkv) * dh, H * dh
    x, qw, s, wq = _gemv_case(lib, M, K, N, 4)
    xs = x.cuda()
    s = s.cuda()
    ck, cv, ks, vs = _pages("bf16", (40, Hkv, block, dh), 1)
    cache = lib.KvCache(ck, cv, ks, vs)
    table = torch.full((B, 8), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(40, dtype=torch.int32, device="cuda")
    rope = lib.qzo_rope_table(128, dh)
    ws = torch.empty(max(1, lib.qzo_paged_attention_workspace_bytes(B, H, Hkv, dh, 128)), dtype=torch.uint8, device="cuda")
    maps = torch.empty((3, B), dtype=torch.int32, device="cuda")
    new = torch.ones(B, dtype=torch.int32, device="cuda")
    out, y = torch.empty((B, H, dh), dtype=torch.bfloat16, device="cuda"), torch.empty((B, N), dtype=torch.bfloat16, device="cuda")
    q_out = torch.empty((B, H, dh), dtype=torch.bfloat16, device="cuda")

    def step(lens, count):
        lib.qzo_assign_slots(lens, new, table, free, count, block, B, row_seq=maps[0], positions=maps[1], slots=maps[2])
        qkv = xs.view(B, H + 2 * Hkv, dh)
        lib.qzo_qk_norm_rope_cache(qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], maps[1], maps[2], cache, table=rope, q_out=q_out)
        lib.qzo_paged_attention(q_out, cache, table, maps[1], row_seq=maps[0], out=out, workspace=ws)
        lib.qzo_gemv_int4(out.view(B, H * dh) if H * dh == K else xs, wq, s, K, N, y=y)

    def states():
        return torch.tensor([17, 0, 15], dtype=torch.int32, device="cuda"), torch.tensor([38], dtype=torch.int32, device="cuda")

    def fill():
        ck.copy_(base[0]), cv.copy_(base[1])
        table.fill_(-1)
        table[0, :2] = torch.tensor([39, 38], dtype=torch.int32, device="cuda")
        table[2, 0] = 0
        free.copy_(torch.arange(1, 41, dtype=torch.int32, device="cuda"))
        out.zero_(), y.zero_()

    base = ck.clone(), cv.clone()
    results = []
    for way in ("plain", "side", "graph"):
        fill()
        lens, count = states()
        torch.cuda.synchronize()
        if way == "plain":
            for _ in range(3):
                step(lens, count)
        else:
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                if way == "side":
                    for _ in range(3):
                        step(lens, count)
                else:
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=side):
                        step(lens, count)
                    for _ in range(3):
                        graph.replay()
        torch.cuda.synchronize()
        results.append([t.clone() for t in (lens, count, table, maps, ck, cv, out, y)])
    assert results[0][0].tolist() == [20, 3, 18]
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


def test_tensors_off_the_current_device_or_of_another_shape_are_refused(lib):
    x, q, s, wq = _gemv_case(lib, 2, 128, 64, 1)
    with pytest.raises(AssertionError):
        lib.qzo_gemv_int4(x, wq, s.cuda(), 128, 64)                  # host tensor
    with pytest.raises(AssertionError):
        lib.qzo_gemv_int4(x.cuda().float(), wq, s.cuda(), 128, 64)
    with pytest.raises(AssertionError):
        lib.qzo_gemv_int4(x.cuda(), wq, s.cuda(), 128, 256)          # weights too short
    with pytest.raises(lib.QzoError):
        lib.qzo_gemv_int4(x.cuda().repeat(9, 1), wq, s.cuda(), 128, 64)
    ck, cv, ks, vs = _pages("bf16", (4, 2, 16, 64), 1)
    cache = lib.KvCache(ck, cv)
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    table = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    with pytest.raises(AssertionError):
        lib.qzo_paged_attention(_randn((1, 2, 128), 1).cuda(), cache, table, pos)
    with pytest.raises(AssertionError):
        lib.qzo_paged_attention(_randn((1, 2, 64), 1).cuda(), cache, table, pos.long())
    with pytest.raises(AssertionError):
        lib.qzo_paged_attention(_randn((1, 64, 2), 1).cuda().transpose(1, 2), cache, table, pos)


def test_captured_behind_copies_and_behind_another_stream(lib):
    # the kernel in front of a captured call may be no kernel at all (a copy of device memory), or run on another stream
    M, K, N, H, dh, block = 3, 512, 512, 4, 128, 16
    x, qw, s, wq = _gemv_case(lib, M, K, N, 31)
    s = s.cuda()
    ck, cv, ks, vs = _pages("bf16", (8, H, block, dh), 32)
    cache = lib.KvCache(ck, cv, ks, vs)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(M, 2)
    given = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    at, pos = torch.empty((M, K), dtype=torch.bfloat16, device="cuda"), torch.empty(M, dtype=torch.int32, device="cuda")
    pos_given = torch.empty(M, dtype=torch.int32, device="cuda")
    y, out, z = (torch.empty((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    side, other = torch.cuda.Stream(), torch.cuda.Stream()

    def run(main, second):
        at.copy_(given)                                        # a copy, then a kernel
        lib.qzo_gemv_int4(at, wq, s, K, N, y=y)
        second.wait_stream(main)
        with torch.cuda.stream(second):
            pos.copy_(pos_given)
            lib.qzo_gemv_int4(y, wq, s, K, N, y=z)
        main.wait_stream(second)
        lib.qzo_paged_attention(z.view(M, H, dh), cache, table, pos, out=out.view(M, H, dh))

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        given.zero_(), pos_given.zero_()
        run(side, other)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            run(side, other)
    for seed in range(3):
        fresh, last = _randn((M, K), 40 + seed, 0.1).cuda(), torch.tensor([seed, 9 + seed, 29 + seed], dtype=torch.int32, device="cuda")
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            given.copy_(fresh), pos_given.copy_(last)
            graph.replay()
        torch.cuda.synchronize()
        first = lib.qzo_gemv_int4(fresh, wq, s, K, N)
        second = lib.qzo_gemv_int4(first, wq, s, K, N)
        want = lib.qzo_paged_attention(second.view(M, H, dh), cache, table, last).view(M, N)
        assert torch.equal(y, first) and torch.equal(z, second) and torch.equal(out, want)


def test_calls_on_two_streams_at_once(lib):
    # the same caches and weights read from two streams, a workspace each: what one stream gives alone
    positions = [6000, 4097]
    q, ck, cv, ks, vs, table = _attend_case(positions, 8, 2, 128, 16, "bf16", 0, 51)
    cache, table, pos = lib.KvCache(ck, cv, ks, vs), torch.from_numpy(table).cuda(), torch.tensor(positions, dtype=torch.int32, device="cuda")
    x, _, s, wq = _gemv_case(lib, 9, 2048, 4096, 52)
    x, s = x.cuda(), s.cuda()
    need = lib.qzo_paged_attention_workspace_bytes(2, 8, 2, 128, table.shape[1] * 16)
    assert need > 0
    queries = [q.cuda(), _randn((2, 8, 128), 53).cuda()]
    want = [(lib.qzo_paged_attention(a, cache, table, pos), lib.qzo_gemv_int4(x[i:i + 8], wq, s, 2048, 4096)) for i, a in enumerate(queries)]
    streams, spaces = [torch.cuda.Stream() for _ in queries], [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in queries]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, a in enumerate(queries):
            with torch.cuda.stream(streams[i]):
                got[i].append((lib.qzo_paged_attention(a, cache, table, pos, workspace=spaces[i]), lib.qzo_gemv_int4(x[i:i + 8], wq, s, 2048, 4096)))
    torch.cuda.synchronize()
    for i in range(2):
        for pair in got[i]:
            assert torch.equal(pair[0], want[i][0]) and torch.equal(pair[1], want[i][1])


# nats by which some keys lead the others, one per query head
LEADS = [0.0, 9.0, 14.0, 17.2, 20.0, 24.0, 28.0, 60.0]


@pytest.mark.parametrize("kind,heads,Hkv,dh,positions,room", [
    ("e4m3", 8, 1, 128, [2047], 0), ("e4m3", 8, 1, 64, [300, 5000, 0, 40], 0), ("e4m3", 16, 1, 128, [700], 0), ("e4m3", 8, 8, 128, [1500, 3], 9000),
    ("bf16", 8, 1, 128, [2047], 0), ("bf16", 16, 1, 64, [300, 5000], 0)])
def test_leading_keys_of_no_value(lib, kind, heads, Hkv, dh, positions, room):
    # keys that lead and whose values are zero leave the row to the others, whose weights are small beside theirs
    ks = CACHES[kind][1]
    block, scale = 16, dh ** -0.5
    q, ck, cv, ks, vs, table = _attend_case(positions, heads, Hkv, dh, block, kind, room, 61)
    ck[..., 0] = 0.0
    for r, last in enumerate(positions):
        for j in [1] + list(range(70, last + 1, 97)):
            if j <= last:
                page = int(table[r, j // block])
                ck[page, :, j % block, 0], cv[page, :, j % block] = 16.0 / ks, 0.0
    q[:, :, 0] = (torch.tensor(LEADS * 2)[:heads] / (16.0 * scale)).bfloat16()
    out = lib.qzo_paged_attention(q.cuda(), lib.KvCache(ck, cv, ks, vs), torch.from_numpy(table).cuda(),
                                  torch.tensor(positions, dtype=torch.int32, device="cuda"))
    kp, vp = f64(ck) * ks, f64(cv) * vs
    want, spread = serving.paged_attention(f64(q), kp, vp, table, np.arange(len(positions)), positions, scale)
    kmax = np.nanmax(np.abs(kp[np.unique(table[table >= 0])]))
    # as in _attend_check, and what the weights leave out: 2^-60 of the largest weight for each key
    score = np.abs(f64(q)).sum(-1, keepdims=True) * kmax * scale * (dh / 16 + 18) * 2 * F32_STEP
    p_step = BF16_STEP if kind == "bf16" else F16_STEP
    keys = max(positions) + 1
    allowed = BF16_STEP * np.abs(want) + (p_step + 2 * score + (16 + keys / 8) * F32_STEP) * spread * (1 + BF16_STEP) + keys * np.nanmax(np.abs(vp)) * 2.0 ** -60
    off = np.abs(f64(out) - want)
    assert (off <= allowed).all(), [(off / allowed)[:, h].max() for h in range(heads)]


@pytest.mark.parametrize("H,Hkv,dh,positions", [(2, 2, 64, [0, 1, 300]), (12, 1, 128, [40, 2500]), (4, 4, 128, [0, 900] * 30)])
def test_infinite_values_of_live_keys(lib, H, Hkv, dh, positions):
    # an infinite value makes its dimension infinite, both signs make it NaN, the other dimensions stay as they are
    q, ck, cv, ks, vs, table = _attend_case(positions, H, Hkv, dh, 16, "bf16", 0, 71)
    for r, last in enumerate(positions):
        for j, dim, v in ((0, 3, "inf"), (last // 2, 17, "-inf"), (last, dh - 1, "inf"), (0, 40, "inf"), (last, 40, "-inf"), (last, 5, "nan")):
            cv[int(table[r, j // 16]), :, j % 16, dim] = float(v)
    out = f64(lib.qzo_paged_attention(q.cuda(), lib.KvCache(ck, cv), torch.from_numpy(table).cuda(),
                                      torch.tensor(positions, dtype=torch.int32, device="cuda")))
    with np.errstate(invalid="ignore"):
        want, _ = serving.paged_attention(f64(q), f64(ck), f64(cv), table, np.arange(len(positions)), positions, dh ** -0.5)
    special = ~np.isfinite(want)
    assert special.any() and np.isfinite(want).any()
    assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(out[special & ~np.isnan(want)], want[special & ~np.isnan(want)])
    clean = f64(cv)
    clean[~np.isfinite(clean)] = 0.0
    for dim in (3, 17, dh - 1, 40, 5):
        out[..., dim] = want[..., dim] = 0.0
        clean[..., dim] = 0.0
    _attend_check(torch.from_numpy(out), q, ck, torch.from_numpy(clean), 1.0, 1.0, table, np.arange(len(positions)), positions, dh ** -0.5)


@pytest.mark.parametrize("positions,H,Hkv,dh", [([2000, 70], 8, 8, 128), ([3000], 12, 1, 64), ([300], 4, 4, 128)])
def test_weights_over_bf16_pages_keep_more_bits_than_their_type(lib, positions, H, Hkv, dh):
    # values of both signs that cancel: the weights' rounding shows beside the output's
    q, ck, cv, ks, vs, table = _attend_case(positions, H, Hkv, dh, 16, "bf16", 0, 81)
    sign = torch.where(torch.rand(cv.shape[:3], generator=torch.Generator().manual_seed(1)) < 0.5, -1.0, 1.0)[..., None].cuda()
    cv.copy_(torch.where(torch.isnan(cv), cv, (40.0 * sign + 0.5 * cv.float()).bfloat16()))
    out = lib.qzo_paged_attention(q.cuda(), lib.KvCache(ck, cv), torch.from_numpy(table).cuda(),
                                  torch.tensor(positions, dtype=torch.int32, device="cuda"))
    want, spread = serving.paged_attention(f64(q), f64(ck), f64(cv), table, np.arange(len(positions)), positions, dh ** -0.5)
    assert np.median(np.abs(want) / spread) < 0.1
    # score: dh exact products summed in fp32 (chains of 16, truncated at worst), one scaling; its exponential within 4 steps
    kmax = np.nanmax(np.abs(f64(ck)[np.unique(table[table >= 0])]))
    score = np.abs(f64(q)).sum(-1, keepdims=True) * kmax * dh ** -0.5 * (dh / 16 + 18) * 2 * F32_STEP
    # weights as the sum of two bf16: the first off by less than 2^-7 of the weight, the second by 2^-8 of that
    keys = max(positions) + 1
    allowed = BF16_STEP * np.abs(want) + (2.0 ** -15 + 2 * score + (16 + keys / 8) * F32_STEP) * spread * (1 + BF16_STEP)
    off = np.abs(f64(out) - want)
    assert (off <= allowed).all(), (off / allowed).max()


def test_keys_of_zeros_under_the_largest_queries_and_scales(lib):
    # every score is 0, however large the factors that stand before it: the mean of the values
    H, dh, positions = 2, 64, [50]
    q, ck, cv, ks, vs, table = _attend_case(positions, H, H, dh, 16, "e4m3", 0, 91)
    ck.zero_()
    q = q.sign() * torch.tensor(3.0e38).bfloat16()
    out = lib.qzo_paged_attention(q.cuda(), lib.KvCache(ck, cv, 2.0 ** 64, vs), torch.from_numpy(table).cuda(),
                                  torch.tensor(positions, dtype=torch.int32, device="cuda"), scale=2.0 ** 40)
    _attend_check(out, q * 0, ck, cv, ks, vs, table, np.arange(1), positions, 1.0)


def test_8_bit_codes_at_ordinary_scales(lib):
    # scales as a program takes them, the largest value over 448: every code within half a step of value / scale
    T, H, dh = 300, 2, 128
    q, k, v = (_randn((T, H, dh), 90 + i, 2.0) for i in range(3))
    ks, vs = float(k.abs().max().float()) / 448, float(v.abs().max().float()) / 448
    ck, cv = (torch.zeros((20, H, 16, dh), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    i = torch.arange(T, dtype=torch.int32, device="cuda")
    lib.qzo_qk_norm_rope_cache(q.cuda(), k.cuda(), v.cuda(), i, i, lib.KvCache(ck, cv, ks, vs))
    for pages, rows, scale in ((ck, k, ks), (cv, v, vs)):
        got = f64(pages).transpose(0, 2, 1, 3).reshape(-1, H, dh)[:T]
        want = np.clip(f64(rows) / np.float64(np.float32(scale)), -448, 448)
        step = 2.0 ** np.maximum(np.floor(np.log2(np.maximum(np.abs(want), 1e-30))), -6) * 2.0 ** -3
        # in fp32 the reciprocal and the product are off by half a step each
        assert (np.abs(got - want) <= step / 2 + 2 * F32_STEP * 1.001 * np.abs(want)).all()
        assert np.abs(got).max() == 448


@pytest.mark.parametrize("M", [1, 3, 8, 16])
def test_gemv_of_the_largest_activations(lib, M):
    # groups whose products without the scales pass fp32's largest number, and whose outputs do not
    K, N = 512, 72
    x, q, s, wq = _gemv_case(lib, M, K, N, 3)
    big = torch.finfo(torch.bfloat16).max
    x[0, 130:140], x[M - 1, 511] = big, -big
    s = (s.float() * 2.0 ** -5).bfloat16()
    want = f64(x) @ (f64(s)[np.arange(K) // 128] * q.numpy().astype(np.float64))
    assert (np.abs(f64(x)[0, 130:140] @ q.numpy()[130:140].astype(np.float64)) > 3.5e38).any() and np.abs(want).max() < 3e38
    _gemv_check(lib.qzo_gemv_int4(x.cuda(), wq, s.cuda(), K, N), x, q, s)


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("big", [2.0 ** 24, 2.0 ** 25, 2.0 ** 27])
@pytest.mark.parametrize("n,low", [(200, 0), (1500, 300)])
def test_small_differences_of_the_largest_scores(lib, kind, big, n, low):
    # scores in whole steps of fp32 (in powers of two, all products exact), a step or two apart from one warp's keys to another's,
    # behind some small ones: the differences are what counts, however the scores are kept
    H, dh = 1, 128
    step = big * 2.0 ** -23
    blocks = -(-n // 256) * 16
    k, v = torch.zeros((blocks, H, 16, dh)), torch.zeros((blocks, H, 16, dh))
    keys = torch.arange(16 * blocks)
    k.view(-1, dh)[:, 0] = torch.where(keys < low, 0.0, 128.0)
    k.view(-1, dh)[:, 1] = torch.tensor([1.0, 2.0, 0.0, 3.0])[(keys // 32) % 4]
    v.view(-1, dh)[:, :8] = torch.eye(8).repeat_interleave(32, 0).repeat(blocks // 16, 1)
    q = torch.zeros((1, H, dh))
    q[..., 0], q[..., 1] = big / 128, step
    ck, cv = (t.to(CACHES[kind][0]).cuda() for t in (k, v))
    table, scale = np.arange(blocks, dtype=np.int32)[None], float(np.float32(np.log(2.0)))
    out = f64(lib.qzo_paged_attention(q.bfloat16().cuda(), lib.KvCache(ck, cv), torch.from_numpy(table).cuda(),
                                      torch.tensor([n - 1], dtype=torch.int32, device="cuda"), scale=scale))
    want, spread = serving.paged_attention(f64(q), f64(ck), f64(cv), table, np.zeros(1, int), [n - 1], scale)
    # at most three steps between scores: a scale half a fp32 step off, exp2 within 4 steps, sums of n weights, weights in 16 bits
    p_step = 2.0 ** -15 if kind == "bf16" else F16_STEP
    allowed = BF16_STEP * want + (p_step + (4 * 3 * step * np.log(2.0) + 16 + n / 8) * F32_STEP) * spread * (1 + BF16_STEP)
    assert (np.abs(out - want) <= allowed).all(), (np.abs(out - want) / np.maximum(allowed, 1e-30)).max()


@pytest.mark.parametrize("M", [1, 16])
def test_gemv_of_tiny_activations(lib, M):
    # products below fp32's smallest normal number: what is lost is steps of 2^-149, taken 2^10 higher at the end
    K, N = 512, 72
    x, q, s, wq = _gemv_case(lib, M, K, N, 4)
    x, s = (x.float() * 2.0 ** -118).bfloat16(), torch.full_like(s, 4.0)
    want = f64(x) @ (4.0 * q.numpy().astype(np.float64))
    got = f64(lib.qzo_gemv_int4(x.cuda(), wq, s.cuda(), K, N))
    steps = 2 * K * 4.0 * 2.0 ** (10 - 149)
    off, size = np.abs(got - want), np.abs(f64(x)) @ np.abs(4.0 * q.numpy().astype(np.float64))
    assert (off <= BF16_STEP * np.abs(want) + (128 + K / 128 + 16) * 2 * F32_STEP * size + steps).all() and steps < 2.0 ** -9 * np.abs(want).max()
