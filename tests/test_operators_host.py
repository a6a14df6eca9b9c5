"""Refusals of the stand-alone operators, without a GPU: every bad argument is
reported before anything is launched, and zero rows are no work.  (The pointers
are plausible numbers that nothing may follow.)"""

import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2506_02780_amd", "libee.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libee.so not built")

P = 1 << 20   # an aligned address


@pytest.fixture(scope="module")
def ee():
    import paper_2506_02780_amd as mod
    return mod


def _linear(ee, **kw):
    d = dict(x=P, w=P, bias=P, residual=P, y=P, ldx=64, ldw=64, ldr=48, ldy=48, rows=0, in_=64, out=48,
             dtype=ee.EE_BF16, out_dtype=ee.EE_BF16, act=0)
    d.update(kw)
    return ee.ee_linear(ctypes.byref(ee.EELinearArgs(**d)), None)


def _route(ee, **kw):
    d = dict(logits=P, bias=P, ids=P, weights=P, ld=64, rows=0, n_experts=64, top_k=8, dtype=ee.EE_F32, score=0,
             renormalize=1, n_groups=1, top_groups=1, group_top=1, scale=1.0)
    d.update(kw)
    return ee.ee_moe_route(ctypes.byref(ee.EEMoeRouteArgs(**d)), None)


def _ffn(ee, **kw):
    d = dict(x=P, w_gate_up=P, w_down=P, ids=P, weights=P, residual=P, out=P, workspace=P, workspace_bytes=1 << 30,
             ldx=64, ldr=64, ldo=64, rows=0, n_experts=8, top_k=2, d_model=64, ffn=32, dtype=ee.EE_BF16,
             out_dtype=ee.EE_BF16)
    d.update(kw)
    return ee.ee_moe_ffn(ctypes.byref(ee.EEMoeFfnArgs(**d)), None)


def test_zero_rows_are_no_work(ee):
    assert _linear(ee) == _route(ee) == _ffn(ee) == ee.EE_OK
    assert _linear(ee, x=None, w=None, y=None) == ee.EE_OK
    assert ee.ee_linear(None, None) == ee.ee_moe_route(None, None) == ee.ee_moe_ffn(None, None) == ee.EE_EINVAL


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "rows"), (dict(rows=(1 << 22) + 1), "rows"), (dict(in_=0), "in and out"), (dict(out=0), "in and out"),
    (dict(out=(1 << 20) + 1), "in and out"), (dict(in_=48), "multiple of 32"), (dict(in_=24, dtype=0, out_dtype=0), "multiple of 32"),
    (dict(dtype=2), "dtype"), (dict(dtype=0, out_dtype=1), "dtype"), (dict(out_dtype=-1), "dtype"),
    (dict(act=5), "activation"), (dict(act=-1), "activation"),
    (dict(x=None, rows=1), "non-NULL"), (dict(w=None, rows=1), "non-NULL"), (dict(y=None, rows=1), "non-NULL"),
    (dict(x=P + 8, rows=1), "16-byte"), (dict(w=P + 2, rows=1), "16-byte"), (dict(ldx=63, rows=1), "16-byte"),
    (dict(ldw=56, rows=1), "16-byte"), (dict(ldx=68, rows=1), "16-byte"), (dict(ldx=-64, rows=1), "16-byte"),
    (dict(ldx=(1 << 21) + 64, rows=1), "16-byte"), (dict(ldw=(1 << 21) + 64, rows=1), "16-byte"),
    (dict(y=P + 1, rows=1), "y must"), (dict(ldy=47, rows=1), "y must"), (dict(ldr=47, rows=1), "residual"),
    (dict(residual=P + 1, rows=1), "residual"), (dict(bias=P + 2, rows=1), "bias"),
    (dict(rows=1 << 22, out=1 << 20, ldy=1 << 20, ldr=1 << 20), "tiles"),
])
def test_linear_refusals(ee, kw, word):
    assert _linear(ee, **kw) == ee.EE_EINVAL and word in ee.ee_last_error(None).decode()


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "rows"), (dict(n_experts=0), "n_experts"), (dict(n_experts=1025), "n_experts"),
    (dict(top_k=0), "top_k"), (dict(top_k=33), "top_k"), (dict(n_experts=4, top_k=5), "top_k"), (dict(dtype=7), "dtype"),
    (dict(score=2), "score"), (dict(n_groups=0), "n_groups"), (dict(n_groups=5), "n_groups"),
    (dict(n_experts=260, n_groups=65), "n_groups"), (dict(n_groups=4, top_groups=5), "top_groups"),
    (dict(top_groups=0), "top_groups"), (dict(n_groups=4, group_top=3), "group_top"), (dict(group_top=0), "group_top"),
    (dict(n_groups=16, top_groups=1), "top_k exceeds"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(logits=None, rows=1), "non-NULL"), (dict(ids=None, rows=1), "non-NULL"),
    (dict(weights=None, rows=1), "non-NULL"), (dict(logits=P + 2, rows=1), "logits"), (dict(ld=63, rows=1), "logits"),
    (dict(ids=P + 2, rows=1), "aligned"), (dict(weights=P + 1, rows=1), "aligned"), (dict(bias=P + 2, rows=1), "aligned"),
])
def test_route_refusals(ee, kw, word):
    assert _route(ee, **kw) == ee.EE_EINVAL and word in ee.ee_last_error(None).decode()


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "rows"), (dict(rows=1 << 24, top_k=2), "rows"), (dict(n_experts=0), "n_experts"),
    (dict(n_experts=1025), "n_experts"), (dict(top_k=0), "top_k"), (dict(top_k=9), "top_k"),
    (dict(n_experts=64, top_k=33), "top_k"), (dict(d_model=48), "multiples"), (dict(ffn=16), "multiples"),
    (dict(ffn=0), "d_model"), (dict(d_model=32800), "d_model"), (dict(dtype=3), "dtype"),
    (dict(dtype=0, out_dtype=1), "out_dtype"), (dict(x=None, rows=1), "non-NULL"), (dict(w_gate_up=None, rows=1), "non-NULL"),
    (dict(w_down=None, rows=1), "non-NULL"), (dict(ids=None, rows=1), "non-NULL"), (dict(weights=None, rows=1), "non-NULL"),
    (dict(out=None, rows=1), "non-NULL"), (dict(workspace=None, rows=1), "non-NULL"), (dict(x=P + 2, rows=1), "x must"),
    (dict(d_model=32768, ffn=16384), "2 GiB"), (dict(ldx=(1 << 21) + 64, rows=1), "x must"), (dict(ldx=65, rows=1), "x must"), (dict(ldx=56, rows=1), "x must"), (dict(w_gate_up=P + 2, rows=1), "w_gate_up"),
    (dict(w_down=P + 8, rows=1), "w_down"), (dict(ids=P + 2, rows=1), "ids"), (dict(ldo=63, rows=1), "out must"),
    (dict(out=P + 1, rows=1), "out must"), (dict(ldr=63, rows=1), "residual"), (dict(workspace=P + 128, rows=1), "workspace"),
])
def test_ffn_refusals(ee, kw, word):
    assert _ffn(ee, **kw) == ee.EE_EINVAL and word in ee.ee_last_error(None).decode()


def test_ffn_workspace(ee):
    n = ee.ee_moe_ffn_workspace_bytes(100, 8, 2, 64, 32, ee.EE_BF16)
    assert n >= 100 * 2 * 32 * 2
    assert _ffn(ee, rows=100, workspace_bytes=n - 1) == ee.EE_ECAPACITY
    assert ee.ee_moe_ffn_workspace_bytes(100, 8, 9, 64, 32, ee.EE_BF16) == 0
    assert ee.ee_moe_ffn_workspace_bytes(100, 8, 2, 48, 32, ee.EE_BF16) == 0
    assert ee.ee_moe_ffn_workspace_bytes(-1, 8, 2, 64, 32, ee.EE_BF16) == 0


def test_python_refusals_without_a_gpu(ee):
    import torch
    x, w = torch.zeros(2, 64), torch.zeros(48, 64)
    for call in (lambda: ee.linear(x, w), lambda: ee.moe_route(x, 4), lambda: ee.linear(None, w),
                 lambda: ee.moe_ffn(x, w, w, None, None)):
        with pytest.raises(ee.EEError) as e:
            call()
        assert e.value.code == ee.EE_EINVAL


@pytest.mark.parametrize("op,name", [("_OP_LINEAR", "EELinearArgs"), ("_OP_ROUTE", "EEMoeRouteArgs"), ("_OP_FFN", "EEMoeFfnArgs")])
def test_packed_arguments_are_the_struct(ee, op, name):
    # every field with a value of its own, the last byte of the struct included
    args = getattr(ee, name)
    values = [1 + i * (1 << 40 if ctypes.sizeof(t) == 8 else 1 << 20) for i, (_, t) in enumerate(args._fields_)]
    packed = getattr(ee, op)[0](*values)
    assert len(packed) == ctypes.sizeof(args)
    back = args.from_buffer_copy(packed)
    assert [getattr(back, n) or 0 for n, _ in args._fields_] == values


def test_arguments_past_their_type_are_refused(ee):
    for bad in (1 << 31, -(1 << 31) - 1):
        with pytest.raises(ee.EEError) as e:
            ee._operator(ee._OP_ROUTE, 0, 0, 0, 0, 0, 0, bad, 1, 1, 0, 0, 0, 1, 1, 1, 1.0)
        assert e.value.code == ee.EE_EINVAL


def test_outputs_that_are_inputs_are_refused(ee):
    apart = dict(rows=1, w=2 * P, bias=3 * P, residual=4 * P, y=5 * P)
    for kw in (dict(y=P), dict(y=2 * P), dict(y=3 * P), dict(y=4 * P, ldr=56)):
        assert _linear(ee, **{**apart, **kw}) == ee.EE_EINVAL, kw
        assert b"must not be an input" in ee.ee_last_error(None)
    apart = dict(rows=1, w_gate_up=2 * P, w_down=3 * P, ids=4 * P, weights=5 * P, residual=6 * P, out=7 * P, workspace=8 * P)
    for kw in (dict(out=P), dict(out=5 * P), dict(out=8 * P), dict(out=6 * P, ldr=72)):
        assert _ffn(ee, **{**apart, **kw}) == ee.EE_EINVAL, kw
        assert b"must not be an input" in ee.ee_last_error(None)


def _rows_around_steps(k, most):
    # (the columns that are held at once fall in steps of 256 as the pairs grow past 2^26 / 256 n)
    steps = {(1 << 26) // (256 * n) // k for n in range(1, 130)}
    return sorted({r for s in steps for r in (s - 1, s, s + 1, s + 2) if 0 < r <= most} | {1, 2, 17, 100, 512, 4095, 4160, most})


@pytest.mark.parametrize("E,k,d,f,dtype", [(128, 8, 2048, 768, "bf16"), (8, 2, 256, 352, "f32"), (256, 8, 7168, 2048, "bf16"),
                                           (32, 32, 8192, 32, "bf16"), (8, 2, 32768, 32, "bf16"), (8, 2, 32768, 16, "f32"),
                                           (4, 3, 1056, 96, "bf16"), (6, 1, 4096, 64, "bf16")])
def test_a_workspace_serves_fewer_rows(ee, E, k, d, f, dtype):
    """The size never falls as the rows grow: a caller may size one workspace for its
    largest call, an engine does, and a call in parts uses the whole call's."""
    dt = ee.EE_BF16 if dtype == "bf16" else ee.EE_F32
    last, at = 0, 0
    for rows in _rows_around_steps(k, min((1 << 24) // k, (2 ** 31 - 1) * 16 // (k * max(d, f)))):
        n = ee.ee_moe_ffn_workspace_bytes(rows, E, k, d, f, dt)
        assert n >= max(last, 1), f"{rows} rows need {n} bytes, {at} rows {last}"
        last, at = n, rows


ROUTE_APART = dict(rows=1, logits=P, bias=2 * P, ids=3 * P, weights=4 * P)
FFN_APART = dict(rows=1, x=P, w_gate_up=2 * P, w_down=3 * P, ids=4 * P, weights=5 * P, residual=6 * P, out=7 * P, workspace=8 * P)


@pytest.mark.parametrize("kw", [dict(ids=P), dict(ids=2 * P), dict(weights=P), dict(weights=2 * P), dict(ids=4 * P)])
def test_route_outputs_at_an_inputs_or_the_others_address(ee, kw):
    assert _route(ee, **{**ROUTE_APART, **kw}) == ee.EE_EINVAL
    assert b"must not be an input" in ee.ee_last_error(None)


@pytest.mark.parametrize("name", ["out", "workspace"])
@pytest.mark.parametrize("at", range(1, 8))
def test_ffn_outputs_at_an_inputs_address(ee, name, at):
    if name == "out" and at >= 6:   # (the residual's address is allowed with its stride; 7 is its own)
        at, kw = 6, dict(ldr=72)
    else:
        kw = {}
    assert _ffn(ee, **{**FFN_APART, name: at * P, **kw}) == ee.EE_EINVAL
    assert b"must not be an input" in ee.ee_last_error(None)


def test_a_single_row_may_carry_any_stride(ee):
    import torch
    for rows, stride, ld in ((1, 70001, 64), (1, 1 << 22, 64), (1, 3, 64), (2, 96, 96), (2, 70001, 70001)):
        t = torch.empty(2 * max(stride, 64) + 64).as_strided((rows, 64), (stride, 1))
        assert ee._rows_of(t, "w", (rows, 64), torch.float32, -1) == ld


def test_tangents_are_refused(ee):
    import torch
    from torch.autograd import forward_ad
    x = torch.zeros(2, 64)
    with forward_ad.dual_level():
        ee._refuse_tangents(x=x, bias=None, out=5)
        with pytest.raises(ee.EEError) as e:
            ee._refuse_tangents(x=x, w=forward_ad.make_dual(x, torch.ones(2, 64)))
        assert e.value.code == ee.EE_EINVAL and "w carries a tangent" in str(e.value)


def test_an_output_given_counts_as_written(ee, monkeypatch):
    """A tensor that autograd saved must not be overwritten unnoticed: out's version
    grows.  (No GPU: the calls themselves are left out.)"""
    import torch
    monkeypatch.setattr(ee, "_operand", lambda t, what: (-1, ee.EE_F32, *t.shape, t.stride(0)))
    monkeypatch.setattr(ee, "_operator", lambda *a: None)
    x, w, y = torch.zeros(4, 64), torch.zeros(64, 64), torch.zeros(8, 64)
    ids, wt = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for n, call in ((1, lambda: ee.linear(x, w, out=y[:4])),
                    (2, lambda: ee.moe_ffn(x, torch.zeros(3, 64, 64), torch.zeros(3, 64, 32), ids, wt, out=y[4:]))):
        call()
        assert y._version == n
    p = torch.ones(8, 64, requires_grad=True)
    loss = (p * y).sum()
    with torch.no_grad():
        ee.linear(x, w, residual=y[:4], out=y[:4])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():   # (such tensors have no version)
        ee.linear(x, w, out=torch.zeros(4, 64))


def test_one_expert_per_row_holds_no_down_products(ee):
    # (they are stored as they are made: what is left is z, the order and the tiles)
    rows, f = 8192, 96
    assert ee.ee_moe_ffn_workspace_bytes(rows, 2, 1, 3776, f, ee.EE_BF16) < rows * (2 * f + 4) + (16 << 10)
