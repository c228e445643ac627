"""The tuned model answering: qzo_assign_slots and qzo_decode, prompts and single tokens of several requests over the paged
caches, against the oracle's whole forward on each request's tokens."""
import numpy as np
import pytest
import torch

from oracle import model as omodel
from paper_2505_13430_b200 import inputs
from tests.helpers import build_oracle_model

pytestmark = pytest.mark.gpu

TOL = 2e-2       # max |a - b| / max |b| per row of logits, as for the logits of the training forwards


def _logits(om, tokens):
    cap = {}
    tok = np.asarray(tokens)[None]
    omodel.forward_loss(om, tok, np.full_like(tok, -100), 0, 0, 1e-3, capture=cap)
    return cap["logits"]


class Server:
    def __init__(self, qzo, gm, cfg, B, block, n_blocks, dtype=torch.bfloat16):
        H, dh = cfg["n_heads"], cfg["d_model"] // cfg["n_heads"]
        self.qzo, self.gm, self.B, self.block = qzo, gm, B, block
        scale = 1.0 if dtype == torch.bfloat16 else 2.0 ** -5
        shape = (n_blocks, H, block, dh)
        self.caches = [qzo.KvCache(*(torch.full(shape, float("nan"), device="cuda").to(dtype) for _ in range(2)), scale, scale)
                       for _ in range(cfg["n_layers"])]
        i32 = dict(dtype=torch.int32, device="cuda")
        self.lens, self.count = torch.zeros(B, **i32), torch.tensor([n_blocks], **i32)
        self.table = torch.full((B, -(-cfg["max_seq"] // block)), -1, **i32)
        self.free = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
        self.text = [[] for _ in range(B)]

    def step(self, new, rows):
        """new: request -> its new tokens, None when it is finished.  Returns (request, position, logits) of the rows."""
        add = torch.zeros(self.B, dtype=torch.int32)
        flat = []
        for r in range(self.B):
            toks = new.get(r, [])
            add[r] = -1 if toks is None else len(toks)
            self.text[r] = [] if toks is None else self.text[r] + list(toks)
            flat += [] if toks is None else list(toks)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        seq, pos, slots = self.qzo.qzo_assign_slots(self.lens, add.cuda(), self.table, self.free, self.count, self.block, rows, status=status)
        assert int(status.item()) == 0
        tokens = torch.full((rows,), -12345, dtype=torch.int32)       # what stands in padding rows is not looked at
        tokens[:len(flat)] = torch.tensor(flat, dtype=torch.int32)
        logits = self.gm.qzo_decode(self.caches, tokens.cuda(), seq, pos, slots, self.table)
        assert self.gm.qzo_device_status() == 0
        return [(int(r), int(p), l) for r, p, l in zip(seq[:len(flat)].tolist(), pos[:len(flat)].tolist(), logits.cpu().numpy())]


@pytest.mark.parametrize("name,block,dtype,tol", [("tiny", 16, torch.bfloat16, TOL), ("tiny_opt", 32, torch.bfloat16, TOL),
                                                  ("tiny_dh128", 16, torch.bfloat16, TOL)])
def test_decode_follows_the_oracle(name, block, dtype, tol):
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg(name)
    raw = inputs.raw_model_tensors(cfg, seed=1000)
    gm = qzo.build_model_from_raw(raw, 256)
    om = build_oracle_model(raw)
    rng = np.random.default_rng(3)
    srv = Server(qzo, gm, cfg, B=3, block=block, n_blocks=3 * -(-cfg["max_seq"] // block), dtype=dtype)
    take = lambda n: rng.integers(0, cfg["vocab"], n).tolist()  # noqa: E731
    steps = [({0: take(5)}, 8),                                  # one short prompt: the matrix-vector path
             ({0: take(1), 1: take(40)}, 48),                    # a token beside a long prompt: the GEMM path
             ({0: take(1), 1: take(1)}, 2),
             ({0: take(1), 2: take(11)}, 16),
             ({0: None, 1: take(3), 2: take(1)}, 4),             # a finished request gives its blocks back
             ({0: take(19), 2: take(1)}, 20),
             ({0: take(1), 1: take(1), 2: take(1)}, 16)]
    for new, rows in steps:
        for r, p, got in srv.step(new, rows):
            want = _logits(om, srv.text[r][:p + 1])[-1]
            assert np.abs(got - want).max() <= tol * np.abs(want).max(), (r, p)
    gm.close()


@pytest.mark.parametrize("name,block", [("tiny", 16), ("tiny_opt", 64), ("tiny_dh128", 32)])
def test_decode_over_8_bit_pages(monkeypatch, name, block):
    # the oracle attends to the keys and values that stand in the pages, and these are its own within half a step of their
    # type (2^-4 of the value, 2^-10 of the scale where steps no longer shrink) and what the linears before may differ by
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg(name)
    raw = inputs.raw_model_tensors(cfg, seed=1000)
    gm = qzo.build_model_from_raw(raw, 256)
    om = build_oracle_model(raw)
    rng = np.random.default_rng(11)
    srv = Server(qzo, gm, cfg, B=2, block=block, n_blocks=2 * -(-cfg["max_seq"] // block), dtype=torch.float8_e4m3fn)
    take = lambda n: rng.integers(0, cfg["vocab"], n).tolist()  # noqa: E731
    plain, calls = omodel.causal_attention, []

    def over_pages(q, k, v):
        cache, r = srv.caches[len(calls) % cfg["n_layers"]], calls.append(0) or srv.asked
        S = k.shape[1]
        at = np.arange(S)
        page = srv.table.cpu().numpy()[r][at // block]
        held = [(t.float().cpu().numpy().astype(np.float64) * c)[page, :, at % block][None] for t, c in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
        for got, want, scale in zip(held, (k, v), (cache.k_scale, cache.v_scale)):
            assert (np.abs(got - want) <= 2.0 ** -4 * np.abs(want) + scale * 2.0 ** -10 + TOL * (1 + 2.0 ** -3) * np.abs(want).max()).all()
        return plain(q, *held)

    monkeypatch.setattr(omodel, "causal_attention", over_pages)
    for new, rows in (({0: take(5)}, 8), ({0: take(1), 1: take(40)}, 48), ({0: take(1), 1: take(1)}, 2), ({0: None, 1: take(1)}, 4), ({0: take(9), 1: take(1)}, 12)):
        for r, p, got in srv.step(new, rows):
            srv.asked = r
            want = _logits(om, srv.text[r][:p + 1])[-1]
            assert np.abs(got - want).max() <= TOL * np.abs(want).max(), (r, p)
    assert len(calls) % cfg["n_layers"] == 0
    gm.close()


def test_long_context_in_a_small_workspace():
    # a prompt of several steps; the workspace holds fewer splits of the cache than the attention would take
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg("tiny", max_seq=4096)
    raw = inputs.raw_model_tensors(cfg, seed=1000)
    gm = qzo.build_model_from_raw(raw, 64)
    om = build_oracle_model(raw)
    srv = Server(qzo, gm, cfg, B=2, block=16, n_blocks=300)
    rng = np.random.default_rng(5)
    for step in range(10):
        rows = srv.step({1: rng.integers(0, cfg["vocab"], 64).tolist()}, 64)
    rows += srv.step({0: [3, 4], 1: [5]}, 3)
    want = _logits(om, srv.text[1])
    assert len(srv.text[1]) == 641
    for r, p, got in rows:
        ref = want[p] if r == 1 else _logits(om, srv.text[0])[p]
        assert np.abs(got - ref).max() <= TOL * np.abs(ref).max(), (r, p)
    gm.close()


def test_decode_of_requests_is_the_two_calls_in_one():
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg("tiny")
    gm = qzo.build_model_from_raw(inputs.raw_model_tensors(cfg, seed=1000), 64)
    one, two = (Server(qzo, gm, cfg, 2, 16, 6) for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for new, toks, rows in (([5, 9], list(range(14)), 14), ([1, 1], [7, 8], 4), ([-1, 20], list(range(20)), 20), ([3, 1], [1, 2, 3, 4], 4)):
        add = torch.tensor(new, dtype=torch.int32, device="cuda")
        tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        tokens[:len(toks)] = torch.tensor(toks, dtype=torch.int32, device="cuda")
        maps = qzo.qzo_assign_slots(one.lens, add, one.table, one.free, one.count, 16, rows)
        want = gm.qzo_decode(one.caches, tokens, *maps, one.table)
        got, got_maps = gm.qzo_decode_requests(two.caches, tokens, two.lens, add, two.table, two.free, two.count, status=status)
        assert torch.equal(got_maps, torch.stack(maps)) and torch.equal(got[:len(toks)], want[:len(toks)])
        for a, b in ((one.lens, two.lens), (one.count, two.count), (one.table, two.table)):
            assert torch.equal(a, b)
        for a, b in zip(one.caches, two.caches):
            assert torch.equal(a.k.view(torch.int16), b.k.view(torch.int16)) and torch.equal(a.v.view(torch.int16), b.v.view(torch.int16))
    assert int(status.item()) == 0
    # more than the free blocks hold: reported, nothing changes, and the model's own status stays clear
    lens, kept = two.lens.clone(), two.caches[0].k.clone()
    add = torch.tensor([60, 4], dtype=torch.int32, device="cuda")
    _, maps = gm.qzo_decode_requests(two.caches, torch.zeros(64, dtype=torch.int32, device="cuda"), two.lens, add, two.table, two.free,
                                     two.count, status=status)
    assert int(status.item()) == 4 and torch.equal(two.lens, lens) and (maps == -1).all() and gm.qzo_device_status() == 0
    assert torch.equal(two.caches[0].k.view(torch.int16), kept.view(torch.int16))
    gm.close()


def test_decode_agrees_with_the_training_forward_and_leaves_it_alone():
    # the same tokens through qzo_forward_loss and qzo_decode; a training step after decoding gives what it gives without
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg("tiny")
    raw = inputs.raw_model_tensors(cfg, seed=1000)
    tok, lab = inputs.tokens_and_labels(cfg, 2, 32, seed=9)
    outs = []
    for decode_between in (False, True):
        gm = qzo.build_model_from_raw(raw, 256)
        first = gm.qzo_step(tok.cuda(), lab.cuda(), 5, 1e-3, 1e-3, 100.0)
        if decode_between:
            srv = Server(qzo, gm, cfg, 2, 16, 16)
            rows = srv.step({0: tok[0].tolist(), 1: tok[1].tolist()}, 64)
            gm.qzo_forward_loss(tok.cuda(), lab.cuda(), 0, 0, 1e-3)
            full = gm.qzo_debug_layer_output(0, 1, 64)
            got = np.stack([l for _, _, l in rows])
            want = full.cpu().numpy()
            assert np.abs(got - want).max() <= 1e-2 * np.abs(want).max()
        second = gm.qzo_step(tok.cuda(), lab.cuda(), 6, 1e-3, 1e-3, 100.0)
        outs.append((first, second, gm.scales.clone()))
        gm.close()
    assert outs[0][:2] == outs[1][:2] and torch.equal(outs[0][2], outs[1][2])


def test_captured_decode_steps_replay():
    # a model on a stream of its own: one captured step, replayed token after token, gives what direct steps give
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg("tiny_dh128")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        gm = qzo.build_model_from_raw(inputs.raw_model_tensors(cfg, seed=1000), 64)
        direct, replayed = (Server(qzo, gm, cfg, 2, 16, 26) for _ in range(2))
        prompt = {0: list(range(30)), 1: [5, 6, 7]}
        for srv in (direct, replayed):
            srv.step(prompt, 33)
        new, tokens = (torch.ones(2, dtype=torch.int32, device="cuda") for _ in range(2))
        logits = torch.empty((2, cfg["vocab"]), dtype=torch.float32, device="cuda")
        step = lambda srv, out: gm.qzo_decode_requests(srv.caches, tokens, srv.lens, new, srv.table, srv.free, srv.count, logits=out)  # noqa: E731
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(replayed, logits)
        for _ in range(20):                                   # across a block's end
            want, _ = step(direct, None)
            graph.replay()
            assert torch.equal(logits, want)
            tokens.copy_(want.argmax(-1))
        assert torch.equal(direct.lens, replayed.lens) and replayed.lens.tolist() == [50, 23] and gm.qzo_device_status() == 0
        side.synchronize()
        del graph
        gm.close()


@pytest.mark.parametrize("name,layers", [("llama7b", 2), ("opt6.7b", 1), ("llama13b", 1)])
def test_full_width_decode_agrees_with_the_training_forward(name, layers):
    # prompts by the GEMM path, then their last tokens again, one by one, by the matrix-vector path
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg(name, n_layers=layers)
    gm = qzo.build_random_model_gpu(cfg, 128)
    tok, lab = inputs.tokens_and_labels(cfg, 3, 40, seed=4)
    gm.qzo_forward_loss(tok.cuda(), lab.cuda(), 0, 0, 1e-3)
    want = gm.qzo_debug_layer_output(0, 1, 120).view(3, 40, -1).cpu().numpy()
    srv = Server(qzo, gm, cfg, 3, 16, 12)
    rows = srv.step({r: tok[r, :38].tolist() for r in range(3)}, 114)
    for t in (38, 39):
        rows += srv.step({r: tok[r, t:t + 1].tolist() for r in range(3)}, 3)
    assert len(rows) == 120
    for r, p, got in rows:
        assert np.abs(got - want[r, p]).max() <= TOL * np.abs(want[r, p]).max(), (r, p)
    gm.close()


def test_decode_refusals_and_reports():
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg("tiny")
    raw = inputs.raw_model_tensors(cfg, seed=1000)
    gm = qzo.build_model_from_raw(raw, 64)
    srv = Server(qzo, gm, cfg, 1, 16, 4)
    i32 = dict(dtype=torch.int32, device="cuda")
    one = torch.zeros(1, **i32)
    table = torch.zeros((1, 4), **i32)

    def refused(status, caches=srv.caches, n=1, width=4):
        z = torch.zeros(n, **i32)
        with pytest.raises(qzo.QzoError) as e:
            gm.qzo_decode(caches, z, z, z, z, torch.zeros((1, width), **i32))
        assert e.value.status == status

    refused(qzo.ERR_WORKSPACE, n=65)
    wrong = [qzo.KvCache(torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda"))] * 2
    refused(qzo.ERR_BAD_ARG, caches=wrong)
    other = qzo.KvCache(*(torch.zeros((2, 4, 32, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    refused(qzo.ERR_BAD_ARG, caches=[srv.caches[0], other])
    with torch.cuda.stream(torch.cuda.Stream()), pytest.raises(AssertionError):
        gm.qzo_decode(srv.caches, one, one, one, one, table)
    # indices out of range: reported through the status word
    for tokens, pos, slot in ((cfg["vocab"], 0, 0), (0, cfg["max_seq"], 0), (0, 0, 64)):
        gm.qzo_decode(srv.caches, one + tokens, one, one + pos, one + slot, table)
        assert gm.qzo_device_status() == 2
        gm.qzo_debug_set_status(0)
    assert gm.qzo_device_status() == 0
    gm.close()


@pytest.mark.parametrize("name", ["tiny", "tiny_opt"])
@pytest.mark.parametrize("rows", [8, 24])
def test_rows_without_a_slot_are_padding_whatever_else_they_hold(name, rows):
    # slot -1 beside a position, a token, a request and a block table that nothing can look up: as position and slot -1
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg(name)
    gm = qzo.build_model_from_raw(inputs.raw_model_tensors(cfg, seed=1000), 64)
    results = []
    for junk in (False, True):
        srv = Server(qzo, gm, cfg, 2, 16, 6)
        live = [0, 2, 3, 5]
        i32 = dict(dtype=torch.int32, device="cuda")
        table = torch.full((3, 4), -1, **i32)
        table[0, 0], table[1, 0] = 5, 2
        tokens, seq, pos, slots = (torch.full((rows,), v, **i32) for v in (-12345, -1, -1, -1))
        if junk:
            seq[1::2], seq[4::4], pos[:] = 2, 77, torch.arange(rows, **i32) * 7
            pos[rows - 1], slots[rows - 2] = 10 ** 6, -2 ** 31
        for t, (s, p) in zip(live, ((0, 0), (0, 1), (1, 0), (0, 2))):
            tokens[t], seq[t], pos[t], slots[t] = 3 + t, s, p, int(table[s, 0]) * 16 + p
        logits = gm.qzo_decode(srv.caches, tokens, seq, pos, slots, table)
        assert gm.qzo_device_status() == 0
        results.append([logits[live].clone()] + [c.view(torch.int16).clone() for kv in srv.caches for c in (kv.k, kv.v)])
    assert torch.isfinite(results[0][0]).all()
    for a, b in zip(*results):
        assert torch.equal(a, b)
    gm.close()


def test_training_goes_on_after_a_decode_that_met_a_bad_index():
    # what a decode reports is said by the status word until it is cleared; training steps give what they give without it
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg("tiny")
    raw = inputs.raw_model_tensors(cfg, seed=1000)
    tok, lab = inputs.tokens_and_labels(cfg, 2, 32, seed=9)
    i32 = dict(dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, **i32)
    outs = []
    for bad in (False, True):
        gm = qzo.build_model_from_raw(raw, 256)
        steps = [gm.qzo_step(tok.cuda(), lab.cuda(), 5, 1e-3, 1e-3, 100.0)]
        before = gm.scales.clone()
        if bad:
            srv = Server(qzo, gm, cfg, 1, 16, 4)
            for tokens, pos, slot, block in ((cfg["vocab"], 0, 0, 0), (0, cfg["max_seq"], 0, 0), (0, 0, 64, 0), (0, 0, 0, 4)):
                gm.qzo_decode(srv.caches, zero + tokens, zero, zero + pos, zero + slot, torch.full((1, 4), block, **i32))
                assert gm.qzo_device_status() == 2
        steps += [gm.qzo_step(tok.cuda(), lab.cuda(), 6 + i, 1e-3, 1e-3, 100.0) for i in range(2)]     # the second is replayed
        assert not torch.equal(gm.scales, before)
        assert gm.qzo_device_status() == (2 if bad else 0)
        gm.qzo_debug_set_status(0)
        assert gm.qzo_device_status() == 0
        outs.append((steps, gm.scales.clone()))
        gm.close()
    assert outs[0][0] == outs[1][0] and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("name", ["tiny", "tiny_opt"])
def test_decode_behind_joint_updates_uses_what_they_wrote(name):
    # joint mode changes norms and matrices on the device: the decode in the queue behind it answers with the new ones
    from paper_2505_13430_b200 import qzo
    cfg = inputs.model_cfg(name)
    gm = qzo.build_model_from_raw(inputs.raw_model_tensors(cfg, seed=1000), 64)
    gm.qzo_enable_joint_spsa(0.05)
    tok, lab = inputs.tokens_and_labels(cfg, 2, 32, seed=9)
    tok, lab = tok.cuda(), lab.cuda()
    srv = Server(qzo, gm, cfg, 2, 16, 16)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.arange(8, **i32).view(2, 4)
    pos = torch.arange(32, **i32).repeat(2)
    seq = torch.arange(2, **i32).repeat_interleave(32)
    slots = table[seq.long(), (pos // 16).long()] * 16 + pos % 16
    one = lambda r, p: [t[32 * r + p:32 * r + p + 1].contiguous() for t in (tok.view(-1), seq, pos, slots)]  # noqa: E731
    answers = []
    for step in range(3):
        if step:
            gm.qzo_step(tok, lab, 5 + step, 1e-3, 1e-3, 100.0)
        many = gm.qzo_decode(srv.caches, tok.view(-1), seq, pos, slots, table)
        few = gm.qzo_decode(srv.caches, *one(1, 31), table)
        torch.cuda.synchronize()
        assert torch.equal(gm.qzo_decode(srv.caches, tok.view(-1), seq, pos, slots, table), many)
        torch.cuda.synchronize()
        assert torch.equal(gm.qzo_decode(srv.caches, *one(1, 31), table), few)
        gm.qzo_forward_loss(tok, lab, 0, 0, 1e-3)
        want = gm.qzo_debug_layer_output(0, 1, 64)
        # each side within TOL of the exact logits: two of them within twice that of one another
        assert (many - want).abs().max() <= 2 * TOL * want.abs().max()
        assert (few - want[63:]).abs().max() <= 2 * TOL * want.abs().max()
        answers.append(want.clone())
    for a, b in zip(answers, answers[1:]):
        assert (a - b).abs().max() > 0.1 * a.abs().max()
    assert gm.qzo_device_status() == 0
    gm.close()
