"""The oracle's sparse layers against a token-by-token evaluation, and the sizes
and refusals of ee_moe_create (no GPU)."""

import ctypes
import os

import numpy as np
import pytest

from oracle.model import route, silu, sparse_ffn
from workloads import gen_weights, get_shape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2506_02780_amd", "libee.so")


@pytest.mark.parametrize("kw", [dict(), dict(score="sigmoid", router_bias=True, route_scale=2.0),
                                dict(renormalize=False, top_k=3),
                                dict(score="sigmoid", router_bias=True, n_experts=12, n_groups=3, top_groups=2, group_top=2)])
def test_sparse_ffn_token_by_token(kw):
    shape = get_shape("tiny-moe", **kw)
    lw = gen_weights(shape, seed=3, std=0.1).layer(1)
    x = np.random.default_rng(4).standard_normal((9, shape.d_model))
    got = sparse_ffn(x, lw, shape, lambda z: z)
    f = shape.ffn
    for t in range(9):
        l = [float(x[t] @ lw["router"][e].astype(np.float64)) for e in range(shape.n_experts)]
        if shape.score == "softmax":
            s = [np.exp(v) / sum(np.exp(u) for u in l) for v in l]
        else:
            s = [1 / (1 + np.exp(-v)) for v in l]
        key = [s[e] + (float(lw["router_bias"][e]) if shape.router_bias else 0.0) for e in range(shape.n_experts)]
        per = shape.n_experts // shape.n_groups
        value = [sum(sorted(key[g * per:(g + 1) * per])[-shape.group_top:]) for g in range(shape.n_groups)]
        kept = sorted(range(shape.n_groups), key=lambda g: -value[g])[:shape.top_groups]
        ids = sorted((e for e in range(shape.n_experts) if e // per in kept), key=lambda e: -key[e])[:shape.top_k]
        tot = sum(s[e] for e in ids) if shape.renormalize else 1.0
        want = np.zeros(shape.d_model)
        for e in ids:
            gu = lw["w_gate_up"][e].astype(np.float64) @ x[t]
            want += s[e] / tot * shape.route_scale * (lw["w_down"][e].astype(np.float64) @ (silu(gu[:f]) * gu[f:]))
        np.testing.assert_allclose(got[t], want, rtol=1e-11, atol=1e-13)


def test_route_ties_go_to_the_lower_index():
    shape = get_shape("tiny-moe", n_experts=6, top_k=3)
    ids, w = route(np.array([[1.0, 2.0, 2.0, 0.0, 2.0, 2.0]]), shape)
    assert ids.tolist() == [[1, 2, 4]]
    np.testing.assert_allclose(w, 1 / 3)


def test_dense_weights_are_unchanged_by_the_sparse_fields():
    a, b = gen_weights(get_shape("tiny"), seed=9), gen_weights(get_shape("tiny-moe"), seed=9)
    assert all(np.array_equal(a.layer(1)[n], b.layer(1)[n]) for n in ("wq", "wk", "wv", "wo"))
    assert "w_gate" not in b.layer(0) and b.layer(0)["w_gate_up"].shape == (8, 704, 256)


@pytest.mark.skipif(not os.path.exists(LIB), reason="libee.so not built")
def test_sizes_and_refusals():
    import paper_2506_02780_amd as ee
    shape = get_shape("1b-moe")
    cfg, moe = ee.make_config(shape, max_ctx=2048, k_max=32), ee.make_moe_config(shape)
    pc, pm = ctypes.byref(cfg), ctypes.byref(moe)
    bank = 128 * 3 * 2048 * 768 * 2
    other = 2 * (2 * 32256 * 2048 + 16 * (2048 * (16 + 8) * 128 + 2048 * 2048 + 128 * 2048))
    assert 16 * bank + other < ee.ee_moe_packed_weight_bytes(pc, pm) < 16 * bank + other + (1 << 20)
    assert ee.ee_moe_workspace_bytes(pc, pm) > 0
    assert ee.ee_moe_packed_weight_bytes(pc, None) == ee.ee_moe_workspace_bytes(None, pm) == 0
    ctx, w, mw = ctypes.c_void_p(), ee.EEWeights(), ee.EEMoeWeights()

    def create(**kw):
        bad = ee.make_moe_config(shape)
        for k, v in kw.items():
            setattr(bad, k, v)
        assert not kw or ee.ee_moe_workspace_bytes(pc, ctypes.byref(bad)) == 0
        rc = ee.ee_moe_create(pc, ctypes.byref(bad), ctypes.byref(w), ctypes.byref(mw), 1, 1, 1, None, ctypes.byref(ctx))
        assert rc == ee.EE_EINVAL
        return ee.ee_last_error(None).decode()

    for kw, word in ((dict(n_experts=0), "n_experts"), (dict(n_experts=2000), "n_experts"), (dict(top_k=0), "top_k"),
                     (dict(top_k=33), "top_k"), (dict(score=3), "score"), (dict(n_groups=3), "n_groups"),
                     (dict(n_groups=8, top_groups=9), "top_groups"), (dict(group_top=0), "group_top"),
                     (dict(n_groups=64, top_groups=1), "top_k exceeds"), (dict(scale=float("nan")), "scale"), ({}, "NULL")):
        assert word in create(**kw), kw
    rc = ee.ee_moe_create(pc, pm, ctypes.byref(w), None, 1, 1, 1, None, ctypes.byref(ctx))
    assert rc == ee.EE_EINVAL and "NULL" in ee.ee_last_error(None).decode()
