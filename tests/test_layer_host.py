"""Refusals of the 8-bit and paged-cache operators, without a GPU: every bad argument
is reported before anything is launched, and no rows are no work.  (The pointers are
plausible numbers that nothing may follow.)"""

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2506_02780_amd", "libee.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libee.so not built")

P = 1 << 20   # an aligned address


@pytest.fixture(scope="module")
def ee():
    import paper_2506_02780_amd as mod
    return mod


def _call(ee, name, args, defaults, kw):
    unknown = set(kw) - {n for n, _ in args._fields_}
    assert not unknown, unknown
    return getattr(ee, name)(ctypes.byref(args(**{**defaults, **kw})), None)


def _quant(ee, **kw):
    return _call(ee, "ee_fp8_quant", ee.EEFp8QuantArgs,
                 dict(x=P, codes=2 * P, scales=3 * P, ldx=64, ldc=64, rows=0, in_=64, block_rows=1, dtype=ee.EE_BF16), kw)


def _linear(ee, **kw):
    return _call(ee, "ee_fp8_linear", ee.EEFp8LinearArgs,
                 dict(x=P, x_scales=2 * P, w=3 * P, w_scales=4 * P, bias=5 * P, residual=6 * P, y=7 * P, ldx=64, ldw=64, ldr=48, ldy=48,
                      rows=0, in_=64, out=48, out_dtype=ee.EE_BF16, act=0), kw)


CACHE = dict(k_cache=8 * P, v_cache=9 * P, tables=10 * P, k_page=2048, k_slot=128, k_head=64, v_page=2048, v_slot=128, v_head=64,
             ld=4, n_seqs=2, n_pages=8, max_pages=4, page_size=16)


def _append(ee, **kw):
    return _call(ee, "ee_kv_append", ee.EEKvAppendArgs,
                 dict(q=P, k=2 * P, v=3 * P, q_out=4 * P, **CACHE, seqs=5 * P, positions=6 * P, inv_freq=7 * P, ldq=256, ldk=128, ldv=128,
                      ldqo=256, rows=0, n_heads=4, n_kv_heads=2, head_dim=64, rot_dim=64, interleaved=0, dtype=ee.EE_BF16), kw)


def _attend(ee, **kw):
    return _call(ee, "ee_paged_attention", ee.EEPagedAttentionArgs,
                 dict(q=P, **CACHE, lens=2 * P, out=3 * P, lse=4 * P, workspace=5 * P, workspace_bytes=1 << 30, ldq=256, ldo=256, rows=1,
                      n_heads=4, n_kv_heads=2, head_dim=64, window=0, dtype=ee.EE_BF16, out_dtype=ee.EE_BF16, scale=0.125), kw)


def _refused(ee, call, kw, word):
    assert call(ee, **kw) == ee.EE_EINVAL and word in ee.ee_last_error(None).decode(), ee.ee_last_error(None)


def test_no_rows_are_no_work(ee):
    assert _quant(ee) == _linear(ee) == _append(ee) == _attend(ee, n_seqs=0) == ee.EE_OK
    assert _quant(ee, x=None) == _linear(ee, w=None) == _append(ee, k=None, seqs=None, n_seqs=0) == ee.EE_OK
    for f in (ee.ee_fp8_quant, ee.ee_fp8_linear, ee.ee_kv_append, ee.ee_paged_attention):
        assert f(None, None) == ee.EE_EINVAL


def test_declared_functions_are_exported(ee):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ee.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(ee_[a-z0-9_]+)\s*\(", src))
    assert {"ee_fp8_quant", "ee_fp8_linear", "ee_kv_append", "ee_paged_attention", "ee_paged_attention_workspace_bytes"} <= names
    for n in names:
        assert hasattr(ee._lib, n), n


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "rows"), (dict(rows=(1 << 22) + 1), "rows"), (dict(in_=0), "in in"), (dict(in_=(1 << 20) + 16), "in in"),
    (dict(in_=40), "multiple of 16"), (dict(block_rows=0), "block_rows"), (dict(block_rows=64), "block_rows"), (dict(dtype=2), "dtype"),
    (dict(x=None, rows=1), "non-NULL"), (dict(codes=None, rows=1), "non-NULL"), (dict(scales=None, rows=1), "non-NULL"),
    (dict(x=P + 8, rows=1), "x must"), (dict(ldx=63, rows=1), "x must"), (dict(ldx=68, rows=1), "x must"), (dict(ldx=(1 << 21) + 64, rows=1), "x must"),
    (dict(codes=P + 8, rows=1), "codes must"), (dict(ldc=48, rows=1), "codes must"), (dict(ldc=72, rows=1), "codes must"),
    (dict(ldc=(1 << 21) + 64, rows=1), "codes must"), (dict(scales=P + 2, rows=1), "scales must"),
    (dict(codes=P, rows=1), "not be x"), (dict(scales=P, rows=1), "not be x"), (dict(scales=2 * P, rows=1), "each other"),
])
def test_quant_refusals(ee, kw, word):
    _refused(ee, _quant, kw, word)


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "rows"), (dict(rows=(1 << 22) + 1), "rows"), (dict(in_=0), "in and out"), (dict(out=0), "in and out"),
    (dict(out=(1 << 20) + 1), "in and out"), (dict(in_=72), "multiple of 16"), (dict(out_dtype=2), "out_dtype"), (dict(act=5), "activation"),
    (dict(act=-1), "activation"), (dict(x=None, rows=1), "non-NULL"), (dict(w=None, rows=1), "non-NULL"), (dict(y=None, rows=1), "non-NULL"),
    (dict(x_scales=None, rows=1), "non-NULL"), (dict(w_scales=None, rows=1), "non-NULL"), (dict(x=P + 8, rows=1), "16-byte"),
    (dict(w=P + 4, rows=1), "16-byte"), (dict(ldx=48, rows=1), "16-byte"), (dict(ldw=72, rows=1), "16-byte"), (dict(ldw=(1 << 21) + 64, rows=1), "16-byte"),
    (dict(x_scales=P + 2, rows=1), "scales"), (dict(w_scales=P + 1, rows=1), "scales"), (dict(bias=P + 2, rows=1), "bias"),
    (dict(y=P + 1, rows=1), "y must"), (dict(ldy=47, rows=1), "y must"), (dict(ldr=47, rows=1), "residual"), (dict(residual=P + 1, rows=1), "residual"),
    (dict(rows=1 << 22, out=1 << 20, ldy=1 << 20, ldr=1 << 20), "tiles"), (dict(y=6 * P, ldr=56, rows=1), "must not be an input"),
    *((dict(y=i * P, rows=1), "must not be an input") for i in range(1, 6)),
])
def test_linear_refusals(ee, kw, word):
    _refused(ee, _linear, kw, word)


CACHE_REFUSALS = [
    (dict(dtype=2), "dtype"), (dict(head_dim=96), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(n_heads=0), "n_heads"),
    (dict(n_heads=1026), "n_heads"), (dict(n_kv_heads=0), "n_heads"), (dict(n_heads=5), "n_heads"), (dict(n_seqs=-1), "n_seqs"),
    (dict(page_size=0), "page_size"), (dict(page_size=24), "page_size"), (dict(page_size=65552), "page_size"), (dict(max_pages=-1), "max_pages"),
    (dict(max_pages=(1 << 26) + 1), "max_pages"), (dict(n_pages=-1), "n_pages"),
]
MEMORY_REFUSALS = [
    (dict(k_cache=None), "non-NULL"), (dict(v_cache=None), "non-NULL"), (dict(tables=None), "non-NULL"), (dict(k_page=2049), "16 bytes"),
    (dict(k_slot=-128), "not negative"), (dict(v_head=68), "16 bytes"), (dict(v_page=1 << 40), "below"), (dict(k_cache=P + 8), "cache must be 16-byte"),
    (dict(v_cache=P + 2), "cache must be 16-byte"), (dict(k_slot=1 << 27), "2 GiB"), (dict(tables=P + 2), "tables"), (dict(ld=3), "tables"),
]


@pytest.mark.parametrize("kw,word", CACHE_REFUSALS + [({**kw, "rows": 1}, word) for kw, word in MEMORY_REFUSALS] + [
    (dict(rows=-1), "rows"), (dict(rows=(1 << 22) + 1), "rows"), (dict(rot_dim=-16), "rot_dim"), (dict(rot_dim=80), "rot_dim"), (dict(rot_dim=24), "rot_dim"),
    (dict(seqs=None, rows=3), "n_seqs"), (dict(seqs=None, rows=3, n_seqs=0), "n_seqs"), (dict(k=None, rows=1), "non-NULL"),
    (dict(v=None, rows=1), "non-NULL"), (dict(positions=None, rows=1), "non-NULL"), (dict(q=None, rows=1), "together"),
    (dict(q_out=None, rows=1), "together"), (dict(inv_freq=None, rows=1), "inv_freq"), (dict(inv_freq=P + 4, rows=1), "inv_freq"),
    (dict(k=P + 8, rows=1), "q, k, v"), (dict(ldk=120, rows=1), "q, k, v"), (dict(ldv=132, rows=1), "q, k, v"), (dict(ldq=248, rows=1), "q, k, v"),
    (dict(ldqo=252, rows=1), "q, k, v"), (dict(positions=P + 2, rows=1), "positions"), (dict(seqs=P + 2, rows=1), "positions"),
    (dict(k_slot=64, rows=1), "share memory"), (dict(k_page=1024, rows=1), "share memory"), (dict(v_head=0, rows=1), "share memory"),
    (dict(v_page=0, rows=1), "share memory"), (dict(v_cache=8 * P, rows=1), "the same"), (dict(k_cache=2 * P, rows=1), "must not be an input"),
    (dict(v_cache=6 * P, rows=1), "must not be an input"), (dict(q_out=3 * P, rows=1), "must not be an input"), (dict(q_out=10 * P, rows=1), "must not be an input"),
    (dict(q_out=P, ldqo=264, rows=1), "must not be an input"), (dict(q_out=8 * P, rows=1), "must not be the cache"), (dict(q=9 * P, rows=1), "must not be the cache"),
])
def test_append_refusals(ee, kw, word):
    _refused(ee, _append, kw, word)


@pytest.mark.parametrize("kw,word", CACHE_REFUSALS + MEMORY_REFUSALS + [
    (dict(rows=0), "rows"), (dict(rows=1025), "rows"), (dict(rows=1024, n_seqs=4097), "rows"), (dict(window=-1), "window"),
    (dict(n_seqs=1 << 22, n_heads=1024, n_kv_heads=1), "too many"), (dict(n_seqs=1 << 22, n_heads=8), "too many"),
    (dict(n_seqs=(1 << 14) + 1, rows=1024, n_heads=1, n_kv_heads=1), "rows"), (dict(out_dtype=2), "out_dtype"), (dict(dtype=0, out_dtype=1), "out_dtype"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(q=None), "non-NULL"), (dict(out=None), "non-NULL"),
    (dict(lens=None), "non-NULL"), (dict(workspace=None), "non-NULL"), (dict(q=P + 8), "q must"), (dict(ldq=248), "q must"), (dict(ldq=260), "q must"),
    (dict(ldq=(1 << 21) + 64), "q must"), (dict(out=P + 1), "out must"), (dict(ldo=255), "out must"), (dict(lens=P + 2), "lens"), (dict(lse=P + 2), "lens"),
    (dict(workspace=P + 128), "workspace"), (dict(out=P), "must not be an input"), (dict(out=8 * P), "must not be an input"),
    (dict(lse=2 * P), "must not be an input"), (dict(workspace=10 * P), "must not be an input"), (dict(workspace=P), "must not be an input"),
    (dict(out=4 * P), "each other"), (dict(workspace=3 * P), "each other"), (dict(workspace=4 * P), "each other"),
])
def test_attention_refusals(ee, kw, word):
    _refused(ee, _attend, kw, word)


def _workspace(ee, n_seqs=2, rows=1, n_heads=4, n_kv_heads=2, head_dim=64, page_size=16, max_pages=4, window=0):
    return ee.ee_paged_attention_workspace_bytes(n_seqs, rows, n_heads, n_kv_heads, head_dim, page_size, max_pages, window)


def test_attention_workspace(ee):
    n = _workspace(ee)
    assert n >= 2 * 4 * 66 * 4
    assert _attend(ee, workspace_bytes=n - 1) == ee.EE_ECAPACITY
    for bad in (dict(n_seqs=-1), dict(rows=0), dict(rows=1025), dict(n_heads=3), dict(head_dim=32), dict(page_size=8), dict(max_pages=-1),
                dict(window=-1), dict(max_pages=1 << 30)):
        assert _workspace(ee, **bad) == 0, bad


@pytest.mark.parametrize("window", [0, 1, 255, 256, 257, 4096, 2 ** 31 - 1])
def test_an_attention_workspace_serves_smaller_calls(ee, window):
    for name, values in (("n_seqs", (1, 2, 3, 64, 1000)), ("rows", (1, 2, 33, 255, 256, 257, 1024)), ("max_pages", (0, 1, 15, 16, 17, 33, 1000, 1 << 20))):
        last = 0
        for v in values:
            n = _workspace(ee, **{name: v, "window": window})
            assert n >= max(last, 1), (name, v)
            last = n


@pytest.mark.parametrize("kw", [
    dict(n_seqs=64, rows=33, max_pages=8192), dict(n_seqs=1, rows=1024, max_pages=8192), dict(n_seqs=8, rows=1024, max_pages=8192),
    dict(n_seqs=64, rows=1024, max_pages=512, n_heads=8), dict(n_seqs=4096, rows=1, max_pages=8192), dict(n_seqs=64, rows=33, max_pages=8192, window=100_000),
])
def test_attention_workspace_of_wide_tables(ee, kw):
    """It stays below 2 GiB however many rows and sequences share tables of up to 131072 positions, where all their chunks'
    states at once took up to 70 GB; below that it is what they take."""
    at = dict(n_heads=32, n_kv_heads=8, head_dim=128, page_size=16)
    assert 0 < _workspace(ee, **{**at, **kw}) <= 2 << 30
    assert _workspace(ee, **{**at, "n_seqs": 64, "rows": 1, "max_pages": 8192}) == 64 * 512 * 32 * 520
    # (a row of one sequence is not parted)
    assert _workspace(ee, **{**at, "n_seqs": 3, "rows": 7, "max_pages": 1 << 25}) == (1 << 21) * 32 * 520


@pytest.mark.parametrize("op,name", [("_OP_FP8_QUANT", "EEFp8QuantArgs"), ("_OP_FP8_LINEAR", "EEFp8LinearArgs"),
                                     ("_OP_KV_APPEND", "EEKvAppendArgs"), ("_OP_PAGED_ATTENTION", "EEPagedAttentionArgs")])
def test_packed_arguments_are_the_struct(ee, op, name):
    # every field with a value of its own that a float32 holds too, the last byte of the struct included
    args = getattr(ee, name)
    values = [1 + i * (1 << 40 if ctypes.sizeof(t) == 8 else 1 << 19) for i, (_, t) in enumerate(args._fields_)]
    packed = getattr(ee, op)[0](*values)
    assert len(packed) == ctypes.sizeof(args)
    back = args.from_buffer_copy(packed)
    assert [getattr(back, n) or 0 for n, _ in args._fields_] == values


def test_python_refusals_without_a_gpu(ee):
    import torch
    x = torch.zeros(2, 64)
    c = torch.zeros(2, 16, 1, 64)
    t = torch.zeros(2, 1, dtype=torch.int32)
    for call in (lambda: ee.fp8_quant(x), lambda: ee.fp8_quant(None), lambda: ee.fp8_linear(x, x, x, x),
                 lambda: ee.kv_append(x, x, c, c.clone(), t, t[:, 0]), lambda: ee.paged_attention(x, c, c, t, t[:, 0])):
        with pytest.raises(ee.EEError) as e:
            call()
        assert e.value.code == ee.EE_EINVAL


def test_outputs_given_count_as_written(ee, monkeypatch):
    """(No GPU: the calls themselves are left out.)"""
    import torch
    monkeypatch.setattr(ee, "_operand", lambda t, what: (-1, ee.EE_F32, *t.shape, t.stride(0)))
    monkeypatch.setattr(ee, "_codes", lambda t, what: (-1, *t.shape, t.stride(0)))
    monkeypatch.setattr(ee, "_operator", lambda *a: None)
    x = torch.zeros(2, 128)
    codes, scales = torch.zeros(2, 128).to(torch.float8_e4m3fn), torch.zeros(2, 1)
    ee.fp8_quant(x, codes=codes, scales=scales)
    assert codes._version == scales._version == 1
    y = torch.zeros(2, 2)
    ee.fp8_linear(codes, scales, codes, scales[:1], out=y)
    assert y._version == 1
    kc, vc = torch.zeros(2, 16, 2, 64), torch.zeros(2, 16, 2, 64)
    t = torch.zeros(2, 1, dtype=torch.int32)
    ee.kv_append(x, x, kc, vc, t, t[:, 0].contiguous(), q=x, q_out=x)
    assert kc._version == vc._version == x._version == 1
    out, lse = torch.zeros(2, 128), torch.zeros(2, 2)
    ee.paged_attention(x, kc, vc, t, t[:, 0].contiguous(), out=out, lse=lse)
    assert out._version == lse._version == 1 and kc._version == 1


def test_attention_of_no_rows_is_no_work(ee, monkeypatch):
    """A batch that has no new rows is checked as any other, and answered with no rows, as the other operators do.
    (Without a GPU: the C call returns before it would launch anything.)"""
    import torch

    def operator(op, dev, *args):
        pack, call = op
        ee._check(call(pack(*args), None))
    monkeypatch.setattr(ee, "_operand", lambda t, what: (-1, ee.EE_F32, *t.shape, t.stride(0)))
    monkeypatch.setattr(ee, "_operator", operator)
    q, kc, vc = torch.zeros(0, 256), torch.zeros(2, 16, 2, 64), torch.zeros(2, 16, 2, 64)
    for n in (0, 1, 3):
        t, lens, out, lse = torch.zeros(n, 4, dtype=torch.int32), torch.zeros(n, dtype=torch.int32), torch.zeros(0, 256), torch.zeros(0, 4)
        assert ee.paged_attention(q, kc, vc, t, lens).shape == (0, 256)
        assert ee.paged_attention(q, kc, vc, t, lens, out=out, lse=lse, window=7) is out and out._version == lse._version == 1
        for kw in (dict(window=-1), dict(lens=lens.long()), dict(scale=float("nan")), dict(out=torch.zeros(0, 255)), dict(k_cache=kc[..., :48], v_cache=vc[..., :48])):
            with pytest.raises(ee.EEError) as e:
                ee.paged_attention(**{**dict(q=q, k_cache=kc, v_cache=vc, tables=t, lens=lens), **kw})
            assert e.value.code == ee.EE_EINVAL, kw


def test_tangents_are_refused(ee):
    import torch
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        t = forward_ad.make_dual(torch.zeros(2, 64), torch.ones(2, 64))
        with pytest.raises(ee.EEError):
            ee._refuse_tangents(x=t)
