"""Steps of a model whose cache stores keys and values in 8 bits, against a 64-bit decoder with the same rounding on store (tests/kv8_model_ref.py).

The bar for logits is that of the bf16 models, 3e-2 of a row's RMS.  A key or value that lies where two codes are as near is stored one step apart (an eighth of it) by two sides whose inputs
differ in the 17th bit: 2^-17 / 2^-4 = 1.2e-4 of the numbers in the first layer, which have exact inputs, and a few percent further on."""
import numpy as np
import pytest

import pv_inputs
from kv8_model_ref import Decoder

pytestmark = pytest.mark.gpu

S = pv_inputs.ModelShape
GQA = S("kv8_gqa", 2, 512, 8, 2, 128, 1376, 1008, rope_base=500000.0, dtype="bf16", seed=9101)
MHA = S("kv8_mha", 2, 512, 8, 8, 64, 1376, 1008, dtype="bf16", seed=9102)
PAGES = S("kv8_pages", 2, 256, 8, 2, 64, 704, 1024, rope_base=500000.0, dtype="bf16", page_tokens=64, seed=9103)
Q4 = S("kv8_q4", 2, 512, 8, 2, 64, 1408, 1008, rope_base=500000.0, dtype="bf16", seed=9104, weight_bits=4)
WIDE_GROUP = S("kv8_wide", 1, 1024, 32, 1, 64, 352, 512, dtype="bf16", seed=9105)


@pytest.fixture(scope="module")
def pvlib():
    import torch
    assert torch.cuda.is_available()
    import paper_2505_01572_amd as pv
    return pv


def pair(pv, shape, max_gamma=64, room=512):
    from gpu_helpers import gpu_model
    tensors = None
    if shape.weight_bits == 4:
        from oracle import ref
        tensors = {}
        for kind, layer in pv_inputs.iter_tensors(shape):
            a = pv_inputs.fill_tensor(shape, kind, layer, gains="perturbed").reshape(pv_inputs.tensor_shape(shape, kind))
            a = ref.dequant_q4(*pv_inputs.quantize_q4(a)) if kind in pv_inputs.Q4_KINDS else pv_inputs.bf16_bits_to_f32(a)
            tensors[kind, layer] = a.astype(np.float64)
    gm = gpu_model(shape, gains="perturbed", max_gamma=max_gamma)
    return gm, pv.Cache(gm, room, kv_bits=8), Decoder(shape, "perturbed", room, tensors)


def err(got, want):
    return (np.abs(got - want) / np.sqrt((want ** 2).mean(-1, keepdims=True))).max()


def same_cache(gc, rc, share=0.03):
    got, want = pv_inputs.bf16_bits_to_f32(gc.export()).astype(np.float64), rc.export()
    assert got.shape == want.shape
    assert np.mean(got[0] != want[0]) < 1e-3 and np.mean(got != want) < share
    # one step apart at most in the first layer.  Further on the numbers themselves differ before they are rounded, by up to the bar for what the hidden state gives, 3e-2 of their RMS
    # (a number near zero by many of its own steps), and rounding adds a step at most
    slack = np.arange(got.shape[0]).clip(max=1).reshape(-1, 1, 1, 1) * 3e-2 * np.sqrt((want ** 2).mean((2, 3), keepdims=True))
    assert (np.abs(got - want) <= np.maximum(np.abs(got), np.abs(want)) / 8 + 2.0 ** -9 * np.abs(want).max() / 224 + slack).all()


def step(gc, rc, draft):
    T = rc.len
    n_r, t_r, pred, lg = rc.verify(draft)
    n_g, t_g = gc.verify(T, draft)
    got = gc.debug_logits()
    e = err(got, lg)
    assert e < 3e-2, e
    top = np.sort(lg, 1)
    safe = top[:, -1] - top[:, -2] > 4 * np.abs(got - lg).max()
    assert np.array_equal(gc.debug_pred()[safe], pred[safe])
    if safe[:max(n_r, 1)].all():
        assert (n_g, t_g) == (n_r, t_r) and gc.state() == (rc.len, rc.pending)
    else:
        gc.rollback(T)
        rc.rollback(T)
    return e


@pytest.mark.parametrize("shape", [GQA, MHA, PAGES, Q4, WIDE_GROUP], ids=lambda s: s.name)
def test_steps_match_the_decoder(pvlib, shape):
    _, gc, rc = pair(pvlib, shape)
    prompt = pv_inputs.uniform_tokens(61, 37, shape.vocab)
    gc.prefill(prompt)
    assert err(gc.debug_logits()[-1:], rc.prefill(prompt)[None]) < 3e-2
    for i, gamma in enumerate((8, 13, 1, 5, 16, 3, 33, 64, 2)):
        d = pv_inputs.uniform_tokens(62 + i, gamma, shape.vocab)
        if rc.pending >= 0:
            d[0] = rc.pending
        step(gc, rc, d)
    # and what greedy decoding gives is taken whole
    if rc.pending < 0:
        step(gc, rc, pv_inputs.uniform_tokens(99, 1, shape.vocab))
    T, start = rc.len, rc.pending
    greedy = [start]
    for _ in range(7):
        greedy.append(gc.verify(len(gc), [greedy[-1]])[1])
    gc.rollback(T)
    assert gc.verify(T, greedy[:-1])[0] >= 6          # (a tie within the arithmetic's noise may end it)
    gc.rollback(T)
    rc.rollback(T)
    same_cache(gc, rc)


def test_long_prompts_and_contexts(pvlib):
    """A prompt of 300 in one pass, steps whose keys are cut into chunks, and a prompt on top of a context."""
    gm, gc, rc = pair(pvlib, GQA, room=1600)
    prompt = pv_inputs.uniform_tokens(71, 300, GQA.vocab)
    gc.prefill(prompt)
    assert err(gc.debug_logits()[-1:], rc.prefill(prompt)[None]) < 3e-2
    step(gc, rc, pv_inputs.uniform_tokens(72, 8, GQA.vocab))
    gc.rollback(300)
    rc.rollback(300)
    more = pv_inputs.uniform_tokens(73, 1100, GQA.vocab)
    gc.prefill(more)
    assert err(gc.debug_logits()[-1:], rc.prefill(more)[None]) < 3e-2
    for gamma in (1, 4, 24, 64):
        step(gc, rc, pv_inputs.uniform_tokens(74 + gamma, gamma, GQA.vocab))
        gc.rollback(1400)
        rc.rollback(1400)
    same_cache(gc, rc, 0.06)


def test_a_prompt_of_many_packed_rows(pvlib):
    """1500 tokens of 32 query heads on one kv head in one pass."""
    _, gc, rc = pair(pvlib, WIDE_GROUP, room=1600)
    prompt = pv_inputs.uniform_tokens(75, 1500, WIDE_GROUP.vocab)
    gc.prefill(prompt)
    assert err(gc.debug_logits()[-1:], rc.prefill(prompt, 1500)[None]) < 3e-2
    step(gc, rc, pv_inputs.uniform_tokens(76, 64, WIDE_GROUP.vocab))
    gc.rollback(1500)
    rc.rollback(1500)
    same_cache(gc, rc)


LONG = S("kv8_long", 1, 256, 4, 1, 128, 352, 512, dtype="bf16", seed=9106)


def test_steps_over_a_long_context(pvlib):
    """More keys than an XCD's L2 holds: blocks of one row, of 12 and of 40 and more are worked through in three ways."""
    _, gc, rc = pair(pvlib, LONG, room=8900)
    for i in range(8):
        piece = pv_inputs.uniform_tokens(77 + i, 1050, LONG.vocab)
        gc.prefill(piece)
        last = rc.prefill(piece, 1050)
    assert err(gc.debug_logits()[-1:], last[None]) < 3e-2
    for gamma in (1, 8, 12, 40, 64):
        step(gc, rc, pv_inputs.uniform_tokens(90 + gamma, gamma, LONG.vocab))
        gc.rollback(8400)
        rc.rollback(8400)
    same_cache(gc, rc)


def test_graphs_static_steps_and_shuffled_pages_change_nothing(pvlib):
    gm, a, _ = pair(pvlib, MHA)
    caches = [a] + [pvlib.Cache(gm, 512, kv_bits=8) for _ in range(3)]
    caches[1].use_graphs(False)
    caches[2].set_page_table(np.random.default_rng(0).permutation(32).astype(np.int32))
    prompt = pv_inputs.uniform_tokens(81, 90, MHA.vocab)
    for c in caches:
        c.prefill(prompt)
    for i, gamma in enumerate((5, 1, 16, 40, 5)):
        d = pv_inputs.uniform_tokens(82 + i, gamma, MHA.vocab)
        d[0] = caches[0].pending
        want = caches[0].verify(len(a), d)
        logits = caches[0].debug_logits()
        for c in caches[1:3]:
            assert c.verify(len(c), d) == want and np.array_equal(c.debug_logits(), logits)
        caches[3].verify_async_static(len(caches[3]), d)
        assert caches[3].verify_wait() == want
    out = [c.export() for c in caches]
    assert all(np.array_equal(o, out[0]) for o in out[1:])


def test_rollback_and_readmission(pvlib):
    gm, a, _ = pair(pvlib, GQA)
    b = pvlib.Cache(gm, 512, kv_bits=8)
    prompt, d = pv_inputs.uniform_tokens(91, 50, GQA.vocab), pv_inputs.uniform_tokens(92, 20, GQA.vocab)
    for c in (a, b):
        c.prefill(prompt)
    a.set_pending(int(d[0]) ^ 1)
    assert a.verify(50, d)[0] == 0
    a.readmit(70)
    b.prefill(d)
    want = b.debug_logits()                            # (an export takes them away)
    assert len(a) == len(b) == 70 and np.array_equal(a.export(), b.export())
    a.rollback(50)
    a.prefill(d)
    assert np.array_equal(a.debug_logits(), want)
    a.rollback(33)
    a.prefill(prompt[33:])
    a.prefill(d)
    e = a.export() != b.export()                       # a block whose scale an earlier, longer sequence raised may have rounded its smallest numbers
    assert e.mean() < 0.01


@pytest.mark.parametrize("shape", [GQA, PAGES], ids=lambda s: s.name)
def test_draft_trees(pvlib, shape):
    """A tree's logits are the decoder's, and what it leaves behind is what its path leaves as a chain."""
    gm, gc, rc = pair(pvlib, shape)
    twin = pvlib.Cache(gm, 512, kv_bits=8)
    prompt = pv_inputs.uniform_tokens(101, 75, shape.vocab)
    for c in (gc, twin):
        c.prefill(prompt)
    rc.prefill(prompt)
    greedy = [gc.pending]
    for _ in range(12):
        greedy.append(twin.verify(len(twin), [greedy[-1]])[1])
    twin.rollback(75)
    twin.set_pending(greedy[0])
    r = np.random.default_rng(5)
    tokens, parents, at = [], [], -1
    for g in greedy[:10]:                              # the path, behind a wrong sibling or two each time
        for _ in range(r.integers(0, 4)):
            tokens.append((g + 1 + int(r.integers(0, 50))) % shape.vocab)
            parents.append(at)
        tokens.append(g)
        parents.append(at)
        at = len(tokens) - 1
    want = rc.forward(tokens, parents)
    n, nxt, path = gc.verify_tree(75, tokens, parents)
    assert err(gc.debug_logits(), want) < 3e-2
    assert n >= 9 and [tokens[i] for i in path] == greedy[:n]
    assert twin.verify(75, greedy[:n]) == (n, nxt)
    e, f = gc.export(), twin.export()
    assert np.mean(e[0] != f[0]) < 1e-3 and np.mean(e != f) < 0.05
    d = pv_inputs.uniform_tokens(103, 6, shape.vocab)
    gc.rollback(75 + n)
    twin.rollback(75 + n)
    gc.verify(75 + n, d)
    twin.verify(75 + n, d)
    assert err(gc.debug_logits(), twin.debug_logits()) < 3e-2


def test_batches(pvlib):
    """Every sequence of a batch gets what it gets alone."""
    gm, a, _ = pair(pvlib, GQA)
    sets = [[a] + [pvlib.Cache(gm, 512, kv_bits=8) for _ in range(3)], [pvlib.Cache(gm, 512, kv_bits=8) for _ in range(4)]]
    drafts = []
    for i, n in enumerate((5, 130, 47, 300)):
        prompt = pv_inputs.uniform_tokens(111 + i, n, GQA.vocab)
        for s in sets:
            if i == 2:
                s[i].set_page_table(np.random.default_rng(2).permutation(32).astype(np.int32))
            s[i].prefill(prompt)
        d = pv_inputs.uniform_tokens(121 + i, (7, 1, 20, 16)[i], GQA.vocab)
        d[0] = sets[0][i].pending
        drafts.append(d)
    got = pvlib.verify_batch(sets[0], drafts)
    logits, at = sets[0][0].debug_logits(), 0
    for i, (c, d) in enumerate(zip(sets[1], drafts)):
        want = c.verify(len(c), d)
        lg = c.debug_logits()
        assert err(logits[at:at + len(d)], lg) < 1e-2
        top = np.sort(lg, 1)
        if (top[:, -1] - top[:, -2] > 4 * np.abs(logits[at:at + len(d)] - lg).max()).all():
            assert got[i] == want
            assert np.mean(sets[0][i].export() != c.export()) < 0.03
        at += len(d)
    plain = pvlib.Cache(gm, 512)
    plain.prefill(drafts[0])
    with pytest.raises(pvlib.PVError):
        pvlib.verify_batch([sets[0][0], plain], [drafts[0], drafts[1]])


def test_what_has_no_8_bit_cache(pvlib):
    from gpu_helpers import gpu_model
    for shape, kw in ((pv_inputs.CONFIGS["tiny"], {}), (S("kv8_hd32", 1, 128, 4, 2, 32, 352, 512, dtype="bf16", seed=9110), {}), (MHA, {"kernel_path": pvlib.PATH_VECTOR})):
        with pytest.raises(pvlib.PVError):
            pvlib.Cache(gpu_model(shape, **kw), 128, kv_bits=8)
    gm = gpu_model(MHA)
    for bits in (4, 16, -8):
        with pytest.raises(pvlib.PVError):
            pvlib.Cache(gm, 128, kv_bits=bits)


def test_half_the_memory(pvlib):
    gm, a, _ = pair(pvlib, GQA)
    b = pvlib.Cache(gm, 512)
    assert a.pool.numel() <= b.pool.numel() * (1 / 2 + 1 / (16 * 128 * 2) + 1e-3)
    a.prefill(pv_inputs.uniform_tokens(1, 100, GQA.vocab))
    b.prefill(pv_inputs.uniform_tokens(1, 100, GQA.vocab))
    assert b.step_bytes(8) - a.step_bytes(8) == GQA.n_layers * 2 * (GQA.n_kv_heads * 128 * (108 + 8) - GQA.n_kv_heads * (7 + 1))


@pytest.mark.parametrize("bits", [0, 8])
def test_log_probabilities_of_a_step(pvlib, bits):
    """Of the drafts and of others, for chains and prompts; the rows' logits are the ones debug_logits returns."""
    gm, _, _ = pair(pvlib, GQA)
    c = pvlib.Cache(gm, 512, kv_bits=bits)
    assert c.logprobs().entropy.shape == (0,)
    c.prefill(pv_inputs.uniform_tokens(131, 100, GQA.vocab))
    for gamma in (1, 8, 40):
        d = pv_inputs.uniform_tokens(132 + gamma, gamma, GQA.vocab)
        c.verify(len(c), d)
        lg = c.debug_logits().astype(np.float64)
        lp = lg - np.log(np.exp(lg - lg.max(1, keepdims=True)).sum(1, keepdims=True)) - lg.max(1, keepdims=True)
        ask = np.stack([np.roll(d, -1), np.zeros(gamma, np.int32), np.full(gamma, -1, np.int32)], 1)
        got = c.logprobs(ask, top=7)
        assert np.abs(got.logprobs[:, :2] - np.take_along_axis(lp, ask[:, :2], 1)).max() < 1e-5 and np.isnan(got.logprobs[:, 2]).all()
        assert np.array_equal(got.top_ids, np.argsort(-lg, 1, kind="stable")[:, :7]) and np.array_equal(got.top_ids[:, 0], c.debug_pred())
        assert np.abs(got.top_logprobs - np.take_along_axis(lp, got.top_ids, 1)).max() < 1e-5
        assert np.abs(got.entropy + (np.exp(lp) * lp).sum(1)).max() < 1e-4
        assert c.logprobs(np.roll(d, -1)).logprobs.shape == (gamma,)
        c.rollback(100)
    with pytest.raises(pvlib.PVError):
        c.logprobs(np.zeros((3, 1), np.int32))
    with pytest.raises(pvlib.PVError):
        c.logprobs(top=33)
