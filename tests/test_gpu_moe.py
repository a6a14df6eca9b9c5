"""Engines of models with sparse layers (ee_moe_create): parity with the oracle,
and the properties every engine has (lossless greedy stream, batches and
trees bit for bit, graphs as eager launches)."""

import numpy as np
import pytest

from oracle import OracleSession
from tests.helpers import reuse_session_parity
from workloads import gen_weights, get_shape, inject_edits, planted_draft, random_tree, tree_tokens, zipf_tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2506_02780_amd as mod
    return mod


ROUTINGS = [dict(), dict(score="sigmoid", router_bias=True, route_scale=2.5), dict(renormalize=False, top_k=1),
            dict(score="sigmoid", router_bias=True, n_experts=16, top_k=4, n_groups=4, top_groups=2, group_top=2),
            dict(n_experts=5, top_k=5)]


@pytest.mark.parametrize("routing", ROUTINGS)
def test_fp32_reuse_session_matches_the_oracle(ee, routing):
    """64-token prompt, then 10 verify steps of K = 8, logits within 1e-4 (fp32
    sums of 256 and 352 columns; a row's experts differ only where two keys
    lie closer than that, and then the logits would say so)."""
    shape = get_shape("tiny-moe", **routing)
    w = gen_weights(shape, seed=1234, gains="random", std=0.05)
    code = zipf_tokens(shape.vocab, 160, seed=42)
    eng = ee.Engine(shape, w, max_ctx=256, k_max=8)
    _, compared, _ = reuse_session_parity(eng, shape, w, code[:64], code, steps=10, k=8, tol=1e-4)
    assert compared == 10
    eng.close()


def _bf16(**kw):
    base = dict(n_layers=2, d_model=512, n_heads=4, n_kv_heads=2, head_dim=128, ffn=192, vocab=2048, dtype="bf16",
                n_experts=16, top_k=4)
    base.update(kw)
    return get_shape("tiny-moe", **base)


def test_bf16_matches_the_oracle_where_every_expert_is_chosen(ee):
    """With top_k = n_experts no selection can flip on a rounding, and the
    logits follow the oracle's like a dense bf16 model's (the dense tests'
    tolerance at this size, 2e-2)."""
    shape = _bf16(n_experts=4, top_k=4)
    w = gen_weights(shape, seed=5, std=0.03)
    code = zipf_tokens(shape.vocab, 100, seed=6)
    eng, ref = ee.Engine(shape, w, max_ctx=256, k_max=16), OracleSession(shape, w)
    eng.prefill(0, code[:60])
    ref.prefill(code[:60])
    lg = eng.logits()
    assert np.abs(lg - ref.last_logits[-len(lg):]).max() <= 2e-2
    eng.close()


@pytest.mark.parametrize("make", [lambda: get_shape("tiny-moe"), lambda: _bf16(),
                                  lambda: _bf16(d_model=4608, ffn=64, n_layers=1)])
def test_greedy_stream_is_lossless(ee, make):
    """Verify steps with planted drafts of many lengths reproduce the stream of
    K = 0 steps, logits bit for bit; so do blocks of several sequences."""
    shape = make()
    w = gen_weights(shape, seed=11, std=0.08)
    prompt = zipf_tokens(shape.vocab, 150, seed=12)
    eng = ee.Engine(shape, w, max_ctx=400, max_seqs=3, k_max=96)
    first = eng.prefill(0, prompt)
    stream, rows = [first], []
    for _ in range(100):
        stream.append(eng.verify(0, [])[1])
        rows.append(eng.logits()[0])
    for k, good in ((1, 0), (3, 3), (8, 5), (17, 17), (33, 20), (64, 64), (96, 40)):
        eng.rollback(0, 150, first)
        d = planted_draft(stream[1:], good, k, shape.vocab, seed=k)
        a, nxt, _ = eng.verify(0, d)
        assert a == good and nxt == stream[good + 1]
        assert np.array_equal(eng.logits()[:good + 1], np.stack(rows[:good + 1])), k
    # three sequences in one block: as each alone
    for s in (1, 2):
        assert eng.prefill(s, prompt) == first
    eng.rollback(0, 150, first)
    drafts = [planted_draft(stream[1:], g, 12, shape.vocab, seed=g) for g in (2, 12, 7)]
    got = eng.verify_batch([0, 1, 2], drafts)
    assert [(a, n) for a, n, _ in got] == [(2, stream[3]), (12, stream[13]), (7, stream[8])]
    lg = eng.logits().reshape(3, 13, -1)
    for b, g in enumerate((2, 12, 7)):
        assert np.array_equal(lg[b, :g + 1], np.stack(rows[:g + 1]))
    eng.close()


def test_tree_graphs_and_noalloc(ee):
    shape = _bf16()
    w = gen_weights(shape, seed=21, std=0.08)
    prompt = zipf_tokens(shape.vocab, 130, seed=22)
    eng = ee.Engine(shape, w, max_ctx=400, k_max=64)
    first = eng.prefill(0, prompt)
    stream = [first] + [eng.verify(0, [])[1] for _ in range(10)]
    parent = random_tree(40, max_depth=6, max_branch=3, seed=3)
    toks = tree_tokens(parent, stream[1:7], shape.vocab, seed=3)
    draft = planted_draft(stream[1:], 6, 20, shape.vocab, seed=9)
    results = []
    for graphs in (True, False, True):
        eng.use_graphs(graphs)
        for _ in range(2):
            eng.rollback(0, 130, first)
            a = eng.verify(0, toks, parent)
            la = eng.logits()
            eng.rollback(0, 130, first)
            b = eng.verify(0, draft)
            results.append((a[0], a[1], list(a[2]), b[0], b[1], la, eng.logits()))
    eng.rollback(0, 130, first)
    c = eng.verify_noalloc(0, draft)
    assert c[:2] == results[0][3:5] and np.array_equal(eng.logits(), results[0][6])
    for r in results[1:]:
        assert r[:5] == results[0][:5]
        assert np.array_equal(r[5], results[0][5]) and np.array_equal(r[6], results[0][6])
    # the chain along the tree's accepted path gives the same tokens
    assert results[0][1] == stream[results[0][0] + 1]
    eng.close()


def test_prompt_blocks_do_not_change_results(ee):
    """A prompt of several blocks (k_max 600 rows at a time are one) and the
    same tokens committed piece by piece leave the same cache."""
    shape = _bf16()
    w = gen_weights(shape, seed=31, std=0.05)
    prompt = zipf_tokens(shape.vocab, 700, seed=32)
    eng = ee.Engine(shape, w, max_ctx=1024, max_seqs=2, k_max=64)
    p0 = eng.prefill(0, prompt)
    t = eng.prefill(1, prompt[:3])
    eng.rollback(1, 3, int(prompt[3]))
    at = 3
    for n in (0, 1, 30, 64, 200):
        t = eng.extend(1, prompt[at + 1:at + 1 + n])
        at += 1 + n
        eng.rollback(1, at, int(prompt[at]))
    t = eng.extend(1, prompt[at + 1:])
    assert t == p0
    for l in range(shape.n_layers):
        for x, y in zip(eng.read_kv(0, l), eng.read_kv(1, l)):
            assert np.array_equal(x, y)
    eng.close()


def test_other_verifications_and_an_edit_session(ee):
    """Top-1 and low-temperature sampled verification accept what the greedy one
    does, and an edit session with a sparse target and a sparse draft model
    emits the target's own greedy stream."""
    shape, dshape = _bf16(), _bf16(n_layers=1, n_experts=8, top_k=2)
    w = gen_weights(shape, seed=41, std=0.08)
    prompt = zipf_tokens(shape.vocab, 120, seed=42)
    eng = ee.Engine(shape, w, max_ctx=600, k_max=32)
    first = eng.prefill(0, prompt)
    stream = [first] + [eng.verify(0, [])[1] for _ in range(160)]
    g = np.random.default_rng(43)
    for k, good in ((1, 1), (7, 3), (20, 20), (32, 11)):
        d = planted_draft(stream[1:], good, k, shape.vocab, seed=k)
        eng.rollback(0, 120, first)
        assert eng.verify_topk([0], [d], 1, dynamic=False)[0][:2] == (good, stream[good + 1])
        eng.rollback(0, 120, first)
        assert eng.verify_sample(0, d, g.random(k) * 0.99, g.random(k + 1) * 0.99, None, 1e-4, True) == (good, stream[good + 1])
    eng.rollback(0, 120, first)
    original, _ = inject_edits(np.asarray(stream, dtype=np.int32), shape.vocab, seed=44, frac=0.1)
    drf = ee.Engine(dshape, gen_weights(dshape, seed=45, std=0.08), max_ctx=600, k_max=32)
    drf.prefill(0, prompt)
    s = ee.EditSession(eng, 0, original, drf, 0, k_reuse=16, gamma=5)
    while s.n < 160:
        s.step()
    assert s.output[:160] == stream[:160]
    eng.close()
    drf.close()


def test_refused_on_sparse_models(ee):
    eng = ee.Engine(get_shape("tiny-moe"), gen_weights(get_shape("tiny-moe"), seed=1), max_ctx=64, k_max=4)
    for call in (lambda: eng.capture(4), lambda: eng.time_gemm("gateup", 4), lambda: eng.time_gemm("down", 4)):
        with pytest.raises(ee.EEError):
            call()
    eng.prefill(0, [1, 2, 3])
    eng.profile(ee.PROF_CLASSES)
    eng.verify(0, [5, 6])
    times = eng.profile_read()
    assert times["gateup"][1] == 2 and times["down"][1] == 0
    assert eng.time_gemm("qkv", 4) > 0
    eng.close()


def test_blocks_of_fewer_rows_stay_inside_the_workspace(ee, monkeypatch):
    """Blocks on both sides of a step of the down products' columns: 64 sequences of
    65 rows hold 1792 columns, 63 of them 2048, of more bytes.  Bytes behind the
    workspace stay as they were, and the rows are those of single sequences."""
    shape = _bf16(n_layers=1, d_model=2048, ffn=64, vocab=256, n_experts=16, top_k=8)
    size, guard = ee.ee_moe_workspace_bytes, 64 << 20
    monkeypatch.setattr(ee, "ee_moe_workspace_bytes", lambda *a: size(*a) + guard)
    eng = ee.Engine(shape, gen_weights(shape, seed=51, std=0.05), max_ctx=128, max_seqs=64, k_max=64)
    behind = eng.workspace[-guard:]
    behind.fill_(165)
    prompts = [zipf_tokens(shape.vocab, 3 + s % 5, seed=60 + s) for s in range(64)]
    first = [eng.prefill(s, p) for s, p in enumerate(prompts)]
    drafts = [zipf_tokens(shape.vocab, 64, seed=200 + s) for s in range(64)]
    for n in (64, 63, 62, 33):
        got = eng.verify_batch(list(range(n)), drafts[:n])
        assert (behind == 165).all(), n
        rows = eng.logits().reshape(n, 65, -1)
        for s in range(n):
            eng.rollback(s, len(prompts[s]), first[s])
        for s in (0, n // 2, n - 1):
            a, nxt, _ = eng.verify(s, drafts[s])
            assert (a, nxt) == got[s][:2] and np.array_equal(eng.logits(), rows[s])
            eng.rollback(s, len(prompts[s]), first[s])
    eng.close()
