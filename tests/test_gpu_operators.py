"""The stand-alone operators (linear, moe_route, moe_ffn) on the GPU against
plain float64 implementations written here.

Tolerances.  A product element is a float32 sum of n = K products in order,
each partial sum rounded (2^-24 of it): at most n 2^-24 sum |x w| off (and the
products of bf16 values are exact).  An output in bf16 is then off by half a
step, 2^-8 of the value's magnitude at most.  The experts' inner product z is rounded to the model
dtype, half a step of each z again, which the down product carries into
sum |z w| 2^-8.  The weighted sum of k terms adds k 2^-24.  (An MFMA fp32
accumulation rounds no worse than one rounding per term.)"""

import itertools

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U32, UBF = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ee():
    import paper_2506_02780_amd as mod
    return mod


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rand(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def _padded(t, pad):
    """The same values on the GPU with `pad` more elements between rows."""
    rows, cols = t.shape
    base = torch.full((rows, cols + pad), float("nan"), dtype=t.dtype, device="cuda")
    base[:, :cols] = t.cuda()
    return base[:, :cols]


def _act64(v, act):
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v / 2.0 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh((2 / np.pi) ** 0.5 * (v + 0.044715 * v ** 3)))
    return v.clamp(min=0) if act == "relu" else v


def _close(got, want, bound):
    err = (got.double().cpu() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((err / bound).max())} x the bound"


# ------------------------------------------------------------------- linear --

def _linear_case(ee, rows, k, n, dtype, out, act="none", bias=False, residual=False, pad=0, opad=0, seed=0):
    g = _gen(seed)
    x, w = _rand(g, rows, k, dtype=DT[dtype]), _rand(g, n, k, std=k ** -0.5, dtype=DT[dtype])
    b = _rand(g, n) if bias else None
    r = _rand(g, rows, n, dtype=DT[out]) if residual else None
    ldout = torch.full((rows, n + opad), 7.0, dtype=DT[out], device="cuda")
    y = ldout[:, :n]
    got = ee.linear(_padded(x, pad), _padded(w, pad), bias=b.cuda() if bias else None, act=act,
                    residual=_padded(r, opad) if residual else None, out=y)
    assert got is y
    pre = x.double() @ w.double().T
    err = (k + 2) * U32 * (x.double().abs() @ w.double().abs().T)
    if bias:
        pre = pre + b.double()
        err = err + 2 * U32 * pre.abs()
    want = _act64(pre, act)
    # the activations' slopes are below 1.2; their own evaluation takes a few float32 roundings
    err = 1.2 * err + 16 * U32 * (pre.abs() if act != "none" else 0 * pre)
    if residual:
        want = want + r.double()
    err = err + (UBF if out == "bf16" else U32) * (want.abs() + err) + U32 * want.abs()
    _close(y, want, err + 1e-30)
    assert (ldout[:, n:] == 7.0).all(), "columns past the output were written"
    return got


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 65, 129, 257, 513])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_linear_rows(ee, rows, dtype, out):
    _linear_case(ee, rows, 256, 272, dtype, out, bias=True, seed=rows)


@pytest.mark.parametrize("n", [1, 3, 4, 15, 16, 17, 63, 64, 65, 100, 127, 255, 512, 513, 528, 777, 1040])
@pytest.mark.parametrize("rows", [1, 20, 300])
def test_linear_columns(ee, rows, n):
    _linear_case(ee, rows, 128, n, "bf16", "bf16", act="silu", residual=True, seed=n)
    _linear_case(ee, rows, 64, n, "f32", "f32", act="relu", bias=True, seed=n)


@pytest.mark.parametrize("k", [32, 64, 96, 224, 256, 288, 512, 544, 1056, 2080, 8192])
@pytest.mark.parametrize("rows,n", [(1, 48), (5, 600), (40, 640), (270, 530)])
def test_linear_reduction(ee, rows, n, k):
    _linear_case(ee, rows, k, n, "bf16", "f32", seed=k)
    _linear_case(ee, rows, k // 2, n, "f32", "f32", seed=k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,k,n", [(700, 128, 500), (2100, 1088, 40), (3000, 64, 17), (9000, 576, 130), (8300, 1024, 512),
                                      (4000, 2080, 300), (5000, 96, 256)])
def test_narrow_linears_of_many_rows(ee, dtype, rows, k, n):
    # reductions of fewer stages than chains, of many, and of an odd number of
    # super-steps; every tile against single rows, and float64
    k = k if dtype == "bf16" else k // 2
    got = _linear_case(ee, rows, k, n, dtype, "f32", act="silu", bias=True, residual=True, seed=n)
    g = _gen(n + 1)
    x, w = _rand(g, rows, k, dtype=DT[dtype]).cuda(), _rand(g, n, k, dtype=DT[dtype]).cuda()
    whole = ee.linear(x, w)
    for lo, m in ((0, 1), (rows // 2, 20), (rows - 300, 300), (0, rows - 1)):
        assert torch.equal(ee.linear(x[lo:lo + m], w), whole[lo:lo + m]), (lo, m)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("rows,n", [(3, 130), (70, 1030), (300, 770)])
def test_linear_epilogues(ee, rows, n, act):
    for bias, residual in itertools.product((False, True), repeat=2):
        _linear_case(ee, rows, 160, n, "bf16", "bf16", act=act, bias=bias, residual=residual, seed=5)
        _linear_case(ee, rows, 160, n, "f32", "f32", act=act, bias=bias, residual=residual, seed=6)


@pytest.mark.parametrize("rows,n", [(1, 64), (19, 129), (300, 1024)])
def test_linear_strides(ee, rows, n):
    for opad in (0, 1, 4, 5):
        _linear_case(ee, rows, 96, n, "bf16", "bf16", bias=True, residual=True, pad=8, opad=opad, seed=7)
        _linear_case(ee, rows, 96, n, "bf16", "f32", residual=True, pad=40, opad=opad, seed=8)
        _linear_case(ee, rows, 80, n, "f32", "f32", residual=True, pad=4, opad=opad, seed=9)


def test_linear_residual_in_place(ee):
    g = _gen(3)
    x, w, h = _rand(g, 33, 64).cuda(), _rand(g, 96, 64).cuda(), _rand(g, 33, 96).cuda()
    want = ee.linear(x, w, residual=h.clone())
    assert ee.linear(x, w, residual=h, out=h) is h
    assert torch.equal(h, want)


def test_linear_large_values_and_nan(ee):
    """Infinities and NaN stay in their own row and column."""
    g = _gen(4)
    x, w = _rand(g, 20, 64, dtype=torch.bfloat16), _rand(g, 40, 64, dtype=torch.bfloat16)
    clean = ee.linear(x.cuda(), w.cuda())
    x[7, 3], x[11, 5] = float("nan"), float("inf")
    got = ee.linear(x.cuda(), w.cuda())
    assert torch.isnan(got[7]).all()
    assert (torch.isinf(got[11]) | torch.isnan(got[11])).all()
    rest = [i for i in range(20) if i not in (7, 11)]
    assert torch.equal(got[rest], clean[rest])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 128, 512, 600, 2048])
def test_linear_rows_do_not_depend_on_the_others(ee, dtype, n):
    g = _gen(n)
    x, w = _rand(g, 700, 512, dtype=DT[dtype]).cuda(), _rand(g, n, 512, dtype=DT[dtype]).cuda()
    whole = ee.linear(x, w, act="silu")
    for rows in (1, 7, 16, 17, 33, 64, 65, 130, 256, 513):
        assert torch.equal(ee.linear(x[:rows], w, act="silu"), whole[:rows]), rows
        assert torch.equal(ee.linear(x[700 - rows:], w, act="silu"), whole[700 - rows:]), rows


# -------------------------------------------------------------------- route --

def _route64(logits, k, score, bias, renorm, scale, groups, top_groups, group_top):
    """Row by row, from the definition."""
    big = float(np.finfo(np.float32).max)
    ids, ws = [], []
    for row in logits.double().cpu().numpy():
        live = ~(np.isnan(row) | (row == -np.inf))
        l = np.minimum(np.where(live, row, 0), big)
        if score == "softmax":
            e = np.where(live, np.exp(l - (l[live].max() if live.any() else 0)), 0)
            s = e / e.sum() if live.any() else e
        else:
            s = np.where(live, 1 / (1 + np.exp(-l)), 0)
        key = s.copy()
        ok = live.copy()
        if bias is not None:
            b = bias.double().cpu().numpy()
            ok &= ~(np.isnan(b) | (b == -np.inf))
            key = key + np.minimum(np.where(ok, b, 0), big)
        E = len(row)
        if groups > 1:
            per = E // groups
            val = []
            for g in range(groups):
                keys = sorted((key[e] for e in range(g * per, (g + 1) * per) if ok[e]), reverse=True)
                val.append(sum(keys[:group_top]) if keys else -np.inf)
            kept = sorted(range(groups), key=lambda g: (-val[g], g))[:top_groups]
            ok &= np.isin(np.arange(E) // per, kept)
        order = sorted((e for e in range(E) if ok[e]), key=lambda e: (-key[e], e))[:k]
        w = np.array([s[e] for e in order])
        if renorm:
            w = w / w.sum() if len(w) and w.sum() > 0 else 0 * w
        ids.append(order + [-1] * (k - len(order)))
        ws.append(np.concatenate([w * scale, np.zeros(k - len(order))]))
    return np.array(ids, np.int32).reshape(-1, k), np.array(ws).reshape(-1, k)


def _route_case(ee, logits, k, score="softmax", bias=None, renorm=True, scale=1.0, groups=1, top_groups=1, group_top=1):
    ids, w = ee.moe_route(logits, k, score=score, bias=bias, renormalize=renorm, scale=scale, n_groups=groups,
                          top_groups=top_groups, group_top=group_top)
    assert ids.dtype == torch.int32 and w.dtype == torch.float32
    ri, rw = _route64(logits, k, score, bias, renorm, scale, groups, top_groups, group_top)
    assert np.array_equal(ids.cpu().numpy(), ri)
    # float64 up to the one rounding of the stored weight
    np.testing.assert_allclose(w.cpu().numpy(), rw, rtol=U32 * (1 + 1e-6), atol=2.0 ** -149)
    return ids, w


@pytest.mark.parametrize("rows", [1, 3, 4, 5, 64, 513])
@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (7, 3), (63, 6), (64, 8), (65, 1), (128, 8), (200, 10), (256, 8),
                                 (300, 32), (512, 16), (513, 5), (1024, 32)])
def test_route_sizes(ee, rows, E, k):
    g = _gen(E + rows)
    l = _rand(g, rows, E, std=2.0).cuda()
    for score, renorm in itertools.product(("softmax", "sigmoid"), (True, False)):
        _route_case(ee, l, k, score, None, renorm)
    _route_case(ee, l, k, "sigmoid", _rand(g, E, std=0.1).cuda(), True, 2.5)


@pytest.mark.parametrize("E,groups", [(8, 2), (64, 8), (96, 3), (256, 8), (320, 64), (1024, 16), (64, 64), (2, 2)])
@pytest.mark.parametrize("group_top", [1, 2])
def test_route_groups(ee, E, groups, group_top):
    g = _gen(E + groups)
    l, b = _rand(g, 40, E, std=2.0).cuda(), _rand(g, E, std=0.2).cuda()
    for top_groups in {1, (groups + 1) // 2, groups}:
        k = min(8, E // groups * top_groups)
        _route_case(ee, l, k, "sigmoid", b, True, 1.0, groups, top_groups, group_top)
        _route_case(ee, l, k, "softmax", None, False, 1.0, groups, top_groups, group_top)


def test_route_bf16_logits_tie_to_the_lower_index(ee):
    g = _gen(1)
    l = (torch.randint(-3, 4, (200, 128), generator=g).float() * 0.5).to(torch.bfloat16).cuda()
    _route_case(ee, l, 8)
    _route_case(ee, l, 8, "sigmoid", None, False)
    _route_case(ee, l, 4, "sigmoid", None, True, 1.0, 8, 3, 2)
    _route_case(ee, torch.zeros(5, 300, dtype=torch.bfloat16, device="cuda"), 32)


def test_route_masked_rows(ee):
    """-inf, NaN, +inf and the lowest finite value among the logits; rows with
    fewer experts than slots, and with none."""
    g = _gen(2)
    inf, low = float("inf"), float(np.finfo(np.float32).min)
    l = _rand(g, 12, 96)
    l[0] = -inf
    l[1] = float("nan")
    l[2, 3:] = -inf
    l[3, ::2] = float("nan")
    l[4] = low
    l[5, 10] = inf
    l[6, 10], l[6, 4] = inf, inf
    l[7, :90] = low
    l[8, 1:] = low
    l[9] = -inf
    l[9, 95] = low
    l[10, :48] = -inf
    bias = _rand(g, 96, std=0.1)
    masked = bias.clone()
    masked[5], masked[6], masked[7], masked[8] = -inf, float("nan"), inf, low
    for score, b, renorm in itertools.product(("softmax", "sigmoid"), (None, bias, masked), (True, False)):
        b = None if b is None else b.cuda()
        ids, w = _route_case(ee, l.cuda(), 8, score, b, renorm)
        assert (ids[0] == -1).all() and (w[0] == 0).all() and (ids[1] == -1).all()
        _route_case(ee, l.cuda(), 4, score, b, renorm, 1.0, 4, 2, 2)
        _route_case(ee, l.cuda(), 4, score, b, renorm, 1.0, 4, 1, 1)


def test_route_strided_rows(ee):
    g = _gen(8)
    for dt in DT.values():
        l = _padded(_rand(g, 21, 130, dtype=dt), 3)
        a = ee.moe_route(l, 6)
        b = ee.moe_route(l.contiguous(), 6)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ experts --

def _ffn_inputs(rows, d, f, E, k, dtype, seed, skew=1.0, std=1.0):
    g = _gen(seed)
    x = _rand(g, rows, d, std=std, dtype=DT[dtype])
    gu, dn = _rand(g, E, 2 * f, d, std=d ** -0.5, dtype=DT[dtype]), _rand(g, E, d, f, std=f ** -0.5, dtype=DT[dtype])
    ids = (_rand(g, rows, E) + skew * _rand(g, E)).topk(k, dim=-1)[1].to(torch.int32)
    w = torch.rand(rows, k, generator=g)
    return x, gu, dn, ids, w


def _ffn64(x, gu, dn, ids, w, residual, dtype):
    """(value, bound) in float64: see the tolerances above."""
    rows, d = x.shape
    E, f = gu.shape[0], gu.shape[1] // 2
    uz = UBF if dtype == "bf16" else U32
    out, err = (torch.zeros(rows, d, dtype=torch.float64, device=x.device) for _ in range(2))
    for e in range(E):
        row, slot = torch.nonzero(ids == e, as_tuple=True)
        if not len(row):
            continue
        xe, ge, ue, de = x[row].double(), gu[e, :f].double(), gu[e, f:].double(), dn[e].double()
        gate, up = xe @ ge.T, xe @ ue.T
        eg, eu = ((d + 2) * U32 * (xe.abs() @ m.abs().T) for m in (ge, ue))
        s = gate * torch.sigmoid(gate)
        z = s * up
        # silu's slope is below 1.1; its evaluation and the product take a few float32 roundings
        ez = (1.1 * eg) * (up.abs() + eu) + s.abs() * eu + 16 * U32 * z.abs()
        ez = ez + uz * (z.abs() + ez)
        wt = w[row, slot].double()[:, None]
        out.index_add_(0, row, wt * (z @ de.T))
        mag = z.abs() @ de.abs().T
        err.index_add_(0, row, wt * (ez @ de.abs().T + (f + 2) * U32 * (mag + ez @ de.abs().T)))
        err.index_add_(0, row, wt * mag * (ids.shape[1] + 1) * U32)
    if residual is not None:
        out = out + residual.double()
    return out, err


def _ffn_check(ee, x, gu, dn, ids, w, dtype, out="same", residual=None, pad=0):
    odt = DT[dtype] if out == "same" else torch.float32
    y = torch.full((x.shape[0], x.shape[1] + pad), 7.0, dtype=odt, device="cuda")
    o = y[:, :x.shape[1]]
    got = ee.moe_ffn(_padded(x, pad * 16), gu.cuda(), dn.cuda(), ids.cuda(), w.cuda(),
                     residual=None if residual is None else _padded(residual, pad), out=o)
    want, err = _ffn64(x, gu, dn, ids, w, residual, dtype)
    u = UBF if odt == torch.bfloat16 else U32
    _close(got, want, err + u * (want.abs() + err) + 2 * U32 * want.abs() + 1e-30)
    assert (y[:, x.shape[1]:] == 7.0).all()
    return got


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 9, 16, 17, 33, 64, 100, 260])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ffn_rows(ee, rows, dtype):
    a = _ffn_inputs(rows, 128, 96, 8, 2, dtype, seed=rows)
    _ffn_check(ee, *a, dtype)
    _ffn_check(ee, *a, dtype, out="f32", residual=_rand(_gen(1), rows, 128))


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (3, 1), (16, 16), (40, 32), (64, 8), (129, 5), (300, 10), (1024, 4)])
def test_ffn_experts(ee, E, k):
    for rows in (1, 12, 150):
        _ffn_check(ee, *_ffn_inputs(rows, 64, 32, E, k, "bf16", seed=E + rows), "bf16",
                   residual=_rand(_gen(2), rows, 64, dtype=torch.bfloat16))


@pytest.mark.parametrize("d,f", [(32, 32), (32, 512), (512, 32), (96, 160), (544, 224), (1024, 288), (2048, 64), (64, 2080)])
def test_ffn_widths(ee, d, f):
    for rows in (1, 6, 70, 600):
        _ffn_check(ee, *_ffn_inputs(rows, d, f, 4, 2, "bf16", seed=d + rows), "bf16")
    _ffn_check(ee, *_ffn_inputs(40, d // 2, f // 2, 4, 2, "f32", seed=d), "f32")


@pytest.mark.parametrize("rows", [1, 4, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ffn_skipped_slots_and_rows(ee, rows, dtype):
    """Ids outside the bank: single slots, whole rows (their residual, or zeros), everything."""
    x, gu, dn, ids, w = _ffn_inputs(rows, 64, 64, 6, 3, dtype, seed=rows)
    ids[::2, 1] = -1
    ids[1::3] = torch.tensor([6, -5, 2 ** 31 - 1], dtype=torch.int32)
    w[1::3] = float("nan")     # a skipped slot's weight is not read into the sum
    clean = torch.where((ids < 0) | (ids >= 6), torch.zeros_like(w), w)
    res = _rand(_gen(5), rows, 64, dtype=DT[dtype])
    for r in (None, res):
        want, err = _ffn64(x, gu, dn, ids, clean, r, dtype)
        got = ee.moe_ffn(x.cuda(), gu.cuda(), dn.cuda(), ids.cuda(), w.cuda(), residual=None if r is None else r.cuda())
        u = UBF if dtype == "bf16" else U32
        _close(got, want, err + u * (want.abs() + err) + 2 * U32 * want.abs() + 1e-30)
    none = torch.full_like(ids, -1)
    assert (ee.moe_ffn(x.cuda(), gu.cuda(), dn.cuda(), none.cuda(), w.cuda()) == 0).all()
    assert torch.equal(ee.moe_ffn(x.cuda(), gu.cuda(), dn.cuda(), none.cuda(), w.cuda(), residual=res.cuda()).cpu(), res)


def test_ffn_one_expert_takes_every_row_and_repeats(ee):
    """The most uneven load, and one expert in several slots of a row."""
    x, gu, dn, ids, w = _ffn_inputs(500, 64, 96, 16, 4, "bf16", seed=9)
    ids[:] = 11
    _ffn_check(ee, x, gu, dn, ids, w, "bf16")
    ids[:, 0] = 3
    _ffn_check(ee, x, gu, dn, ids, w, "bf16")


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_ffn_strides_and_residual_in_place(ee, rows):
    a = _ffn_inputs(rows, 96, 64, 8, 2, "bf16", seed=3)
    for pad in (1, 2, 4):
        _ffn_check(ee, *a, "bf16", residual=_rand(_gen(4), rows, 96, dtype=torch.bfloat16), pad=pad)
        _ffn_check(ee, *a, "bf16", out="f32", residual=_rand(_gen(4), rows, 96), pad=pad)
    h = _rand(_gen(6), rows, 96).cuda()
    c = [t.cuda() for t in a]
    want = ee.moe_ffn(*c, residual=h.clone(), out_dtype=torch.float32)
    assert ee.moe_ffn(*c, residual=h, out=h) is h
    assert torch.equal(h, want)


def test_ffn_nan_stays_in_its_row(ee):
    x, gu, dn, ids, w = _ffn_inputs(50, 64, 64, 4, 2, "bf16", seed=7)
    c = [gu.cuda(), dn.cuda(), ids.cuda(), w.cuda()]
    clean = ee.moe_ffn(x.cuda(), *c)
    x[13, 2] = float("nan")
    got = ee.moe_ffn(x.cuda(), *c)
    assert torch.isnan(got[13]).all()
    rest = [i for i in range(50) if i != 13]
    assert torch.equal(got[rest], clean[rest])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,k", [(8, 2), (64, 6)])
def test_ffn_rows_do_not_depend_on_the_others(ee, dtype, E, k):
    x, gu, dn, ids, w = [t.cuda() for t in _ffn_inputs(900, 256, 160, E, k, dtype, seed=E)]
    whole = ee.moe_ffn(x, gu, dn, ids, w)
    for rows in (1, 2, 5, 9, 17, 33, 65, 130, 257, 513):
        for lo in (0, 900 - rows):
            s = slice(lo, lo + rows)
            assert torch.equal(ee.moe_ffn(x[s], gu, dn, ids[s].contiguous(), w[s].contiguous()), whole[s]), (rows, lo)


@pytest.mark.parametrize("rows,d,f,E,k", [(6000, 512, 512, 8, 2), (5001, 544, 288, 3, 1), (3000, 1024, 256, 64, 4), (9000, 288, 2080, 2, 2)])
def test_ffn_many_tiles_per_workgroup(ee, rows, d, f, E, k):
    # more row and feature tiles than compute units, experts of very different size,
    # rows without an expert: the same bits as a few of the rows alone, which the
    # tests above compare with float64
    x, gu, dn, ids, w = [t.cuda() for t in _ffn_inputs(rows, d, f, E, k, "bf16", seed=rows, skew=2.0)]
    ids[::97] = -1
    whole = ee.moe_ffn(x, gu, dn, ids, w)
    for lo in (0, 1000, rows // 2 - 13, rows - 31):
        s = slice(lo, lo + 31)
        assert torch.equal(ee.moe_ffn(x[s], gu, dn, ids[s].contiguous(), w[s].contiguous()), whole[s]), lo
    pick = torch.arange(0, rows, rows // 50, device="cuda")
    want, err = _ffn64(x[pick], gu, dn, ids[pick], w[pick], None, "bf16")
    _close(whole[pick], want.cpu(), (err + UBF * (want.abs() + err) + 2 * U32 * want.abs() + 1e-30).cpu())
    for _ in range(3):
        assert torch.equal(ee.moe_ffn(x, gu, dn, ids, w), whole)


@pytest.mark.parametrize("rows", [300, 1000, 5000])
@pytest.mark.parametrize("dtype,out,pad", [("bf16", "same", 0), ("bf16", "f32", 1), ("bf16", "same", 3), ("f32", "same", 8), ("f32", "same", 5)])
def test_ffn_one_expert_per_row(ee, rows, dtype, out, pad):
    # stored as they are made: strides, residuals, rows without an expert, and the
    # bits that few rows give
    x, gu, dn, ids, w = _ffn_inputs(rows, 544, 160, 5, 1, dtype, seed=rows, skew=1.5)
    ids[::11] = -1
    ids[5::101] = 5
    odt = DT[dtype] if out == "same" else torch.float32
    res = _rand(_gen(pad), rows, 544, dtype=odt)
    for r in (None, res):
        got = _ffn_check(ee, x, gu, dn, ids, w, dtype, out=out, residual=r, pad=pad)
        if r is not None:
            assert torch.equal(got[ids[:, 0] < 0].cpu(), r[ids[:, 0] < 0])
        else:
            assert not got[ids[:, 0] < 0].any()
        for lo in (0, rows - 33):
            s = slice(lo, lo + 33)
            some = ee.moe_ffn(x[s].cuda(), gu.cuda(), dn.cuda(), ids[s].cuda(), w[s].cuda(),
                              residual=None if r is None else r[s].cuda(), out_dtype=odt)
            assert torch.equal(some, got[s])
    whole = res.cuda()
    assert torch.equal(ee.moe_ffn(x.cuda(), gu.cuda(), dn.cuda(), ids.cuda(), w.cuda(), residual=whole, out=whole), got)


@pytest.mark.parametrize("d,f", [(32, 256), (240, 272), (256, 240), (272, 528), (528, 1040), (1040, 512), (2064, 784)])
def test_ffn_fp32_chains(ee, d, f):
    # reductions that end before, at and behind a chain of 256 columns, by the kernels
    # of few pairs and of every tile
    x, gu, dn, ids, w = [t.cuda() for t in _ffn_inputs(1200, d, f, 4, 2, "f32", seed=d)]
    whole = ee.moe_ffn(x, gu, dn, ids, w)
    for rows in (1, 7, 40, 200):
        assert torch.equal(ee.moe_ffn(x[:rows], gu, dn, ids[:rows].contiguous(), w[:rows].contiguous()), whole[:rows]), rows


@pytest.mark.parametrize("rows", [9, 300])
@pytest.mark.parametrize("d,f", [(7168, 256), (256, 4096)])
def test_ffn_fp32_long_reductions(ee, rows, d, f):
    # A chain of 256 columns adds its four-column steps one after another: at most 256
    # roundings of 0.29 ulp (rms, 2^-24 sqrt(1/3)) of partial sums whose rms is
    # sqrt(1/2) of the whole: 16 * 0.58 * 0.71 * 2^-24 = 4e-7, the chains' own sum
    # (28 of them) 1.3e-7 more; the gate's, the up's and the down's errors add as
    # squares: below 7.3e-7.  (One chain of 7168 columns: 2.3e-6.)
    x, gu, dn, ids, w = [t.cuda() for t in _ffn_inputs(rows, d, f, 4, 2, "f32", seed=rows)]
    want, _ = _ffn64(x, gu, dn, ids, w, None, "f32")
    err = (ee.moe_ffn(x, gu, dn, ids, w).double() - want).norm() / want.norm()
    assert err < 1e-6, float(err)


# ---------------------------------------------------------- as they are used --

def _layer(ee, h, gain, router, gu, dn, k, **kw):
    """Norm, router logits, routing and experts of one sparse layer, residual in place."""
    x = (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5) * gain).to(gu.dtype)
    ids, w = ee.moe_route(ee.linear(x, router, out_dtype=torch.float32), k, **kw)
    return ee.moe_ffn(x, gu, dn, ids, w, residual=h, out=h), x, ids, w


@pytest.mark.parametrize("rows", [1, 33, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_three_in_a_row(ee, rows, dtype):
    g = _gen(rows)
    d, f, E, k = 256, 96, 32, 4
    h = _rand(g, rows, d)
    gain, router = 1 + 0.1 * _rand(g, d), _rand(g, E, d, std=d ** -0.5, dtype=DT[dtype])
    gu, dn = _rand(g, E, 2 * f, d, std=d ** -0.5, dtype=DT[dtype]), _rand(g, E, d, f, std=f ** -0.5, dtype=DT[dtype])
    hc = h.cuda()
    out, x, ids, w = _layer(ee, hc, gain.cuda(), router.cuda(), gu.cuda(), dn.cuda(), k, score="sigmoid", n_groups=4,
                            top_groups=2, group_top=2)
    assert out is hc
    x, ids, w = x.cpu(), ids.cpu(), w.cpu()
    logits = ee.linear(x.cuda(), router.cuda(), out_dtype=torch.float32)
    ri, rw = _route64(logits, k, "sigmoid", None, True, 1.0, 4, 2, 2)
    assert np.array_equal(ids.numpy(), ri)
    want, err = _ffn64(x, gu, dn, ids, w, h, dtype)
    _close(out, want, err + 4 * U32 * want.abs())


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_captured_and_replayed(ee, rows):
    """The three operators in one graph, replayed with other contents between
    eager calls: every replay equals the eager result."""
    g = _gen(rows)
    d, f, E, k = 256, 96, 32, 4
    gain, router = (1 + 0.1 * _rand(g, d)).cuda(), _rand(g, E, d, std=d ** -0.5, dtype=torch.bfloat16).cuda()
    gu = _rand(g, E, 2 * f, d, std=d ** -0.5, dtype=torch.bfloat16).cuda()
    dn = _rand(g, E, d, f, std=f ** -0.5, dtype=torch.bfloat16).cuda()
    h = _rand(g, rows, d).cuda()

    def layer():
        x = (h * gain).to(torch.bfloat16)
        ids, w = ee.moe_route(ee.linear(x, router, out_dtype=torch.float32), k)
        return ee.moe_ffn(x, gu, dn, ids, w, residual=h, out_dtype=torch.float32)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer()
    for i in range(4):
        h.copy_(_rand(_gen(100 + i), rows, d).cuda())
        want = layer().clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_two_streams_at_once(ee):
    """Calls on two streams with workspaces of their own do not meet."""
    a = [t.cuda() for t in _ffn_inputs(200, 256, 128, 16, 4, "bf16", seed=1)]
    b = [t.cuda() for t in _ffn_inputs(300, 256, 128, 16, 4, "bf16", seed=2)]
    wa, wb = ee.moe_ffn(*a), ee.moe_ffn(*b)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(5):
        with torch.cuda.stream(s1):
            o1 = ee.moe_ffn(*a)
        with torch.cuda.stream(s2):
            o2 = ee.moe_ffn(*b)
        outs.append((o1, o2))
    torch.cuda.synchronize()
    for o1, o2 in outs:
        assert torch.equal(o1, wa) and torch.equal(o2, wb)


def test_rows_and_columns_past_the_output_stay(ee):
    g = _gen(12)
    for rows in (1, 20, 70, 300):
        for n in (40, 600):
            big = torch.full((rows + 40, n + 8), 5.0, dtype=torch.bfloat16, device="cuda")
            ee.linear(_rand(g, rows, 64, dtype=torch.bfloat16).cuda(), _rand(g, n, 64, dtype=torch.bfloat16).cuda(),
                      out=big[20:20 + rows, :n])
            assert (big[:20] == 5).all() and (big[20 + rows:] == 5).all() and (big[:, n:] == 5).all()
        a = [t.cuda() for t in _ffn_inputs(rows, 64, 64, 8, 2, "bf16", seed=rows)]
        big = torch.full((rows + 40, 72), 5.0, dtype=torch.bfloat16, device="cuda")
        ee.moe_ffn(*a, out=big[20:20 + rows, :64])
        assert (big[:20] == 5).all() and (big[20 + rows:] == 5).all() and (big[:, 64:] == 5).all()


def test_a_workspace_of_the_callers(ee):
    """Whatever it holds, and whichever call used it before."""
    most = ee.ee_moe_ffn_workspace_bytes(400, 16, 4, 128, 96, ee.EE_BF16)
    ws = torch.full((most + 512,), 255, dtype=torch.uint8, device="cuda")
    for rows in (400, 3, 90, 400):
        a = [t.cuda() for t in _ffn_inputs(rows, 128, 96, 16, 4, "bf16", seed=rows)]
        assert torch.equal(ee.moe_ffn(*a, workspace=ws), ee.moe_ffn(*a))
        assert (ws[most:] == 255).all(), "written past the stated size"
    with pytest.raises(ee.EEError) as e:
        ee.moe_ffn(*a, workspace=ws[:most - 256])
    assert e.value.code == ee.EE_ECAPACITY


def test_offsets_past_32_bits(ee):
    """Rows 2^21 elements apart: x, w, y and the residual each span more than
    4 GiB."""
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GiB")
    ld, g = 1 << 21, _gen(13)

    def spread(t):
        base = torch.empty(t.shape[0] * ld, dtype=t.dtype, device="cuda")
        v = base.as_strided((t.shape[0], t.shape[1]), (ld, 1))
        v.copy_(t)
        return v

    x, w = _rand(g, 1200, 96, dtype=torch.bfloat16).cuda(), _rand(g, 1100, 96, std=0.1, dtype=torch.bfloat16).cuda()
    r = _rand(g, 1200, 1100, dtype=torch.bfloat16).cuda()
    want = ee.linear(x, w, residual=r)
    xs, ws, rs = spread(x), spread(w), spread(r)
    assert torch.equal(ee.linear(xs, ws, residual=rs, out=rs), want)
    assert torch.equal(ee.linear(xs[1190:], w), ee.linear(x[1190:], w))
    assert torch.equal(ee.linear(xs, w[:300], out_dtype=torch.float32), ee.linear(x, w[:300], out_dtype=torch.float32))
    del ws
    a = [t.cuda() for t in _ffn_inputs(1200, 96, 64, 8, 2, "bf16", seed=14)]
    want = ee.moe_ffn(*a, residual=r[:, :96].contiguous())
    h = rs[:, :96]
    h.copy_(r[:, :96])
    assert torch.equal(ee.moe_ffn(spread(a[0]), *a[1:], residual=h, out=h), want)
    ids, wt = ee.moe_route(x, 8)
    assert all(torch.equal(p, q) for p, q in zip(ee.moe_route(xs, 8), (ids, wt)))


def test_an_expert_bank_of_more_than_4_gib(ee):
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GiB")
    E, d, f, k = 640, 2048, 1024, 4
    g = torch.Generator(device="cuda").manual_seed(15)
    gu = torch.empty(E, 2 * f, d, dtype=torch.bfloat16, device="cuda").normal_(0, d ** -0.5, generator=g)
    dn = torch.empty(E, d, f, dtype=torch.bfloat16, device="cuda").normal_(0, f ** -0.5, generator=g)
    for rows in (1, 7, 150):
        x = torch.randn(rows, d, generator=g, device="cuda").to(torch.bfloat16)
        ids = torch.randint(E - 40, E, (rows, k), generator=g, device="cuda", dtype=torch.int32)
        w = torch.rand(rows, k, generator=g, device="cuda")
        want, err = _ffn64(x, gu, dn, ids, w, None, "bf16")
        got = ee.moe_ffn(x, gu, dn, ids, w)
        _close(got, want.cpu(), (err + UBF * (want.abs() + err) + 2 * U32 * want.abs() + 1e-30).cpu())


def test_many_rows(ee):
    """Pairs sorted by many workgroups, down products in several groups of
    columns, and long grids."""
    a = [t.cuda() for t in _ffn_inputs(9000, 1056, 32, 16, 8, "bf16", seed=16)]
    res = _rand(_gen(17), 9000, 1056, dtype=torch.bfloat16).cuda()
    want, err = _ffn64(*a, res, "bf16")
    got = ee.moe_ffn(*a, residual=res)
    _close(got, want.cpu(), (err + UBF * (want.abs() + err) + 2 * U32 * want.abs() + 1e-30).cpu())
    g = _gen(18)
    l = _rand(g, 70001, 24, std=2.0).cuda()
    ids, w = ee.moe_route(l, 3)
    top = torch.sort(l, dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), top[1][:, :3])
    e = torch.exp(top[0][:, :3].double() - top[0][:, :1].double())
    assert ((w.double() - e / e.sum(1, keepdim=True)).abs() <= U32 * (1 + 1e-6)).all()
    x, wt = _rand(g, 70001, 64).cuda(), _rand(g, 24, 64).cuda()
    y = ee.linear(x, wt)
    assert ((y.double() - x.double() @ wt.double().T).abs() <= 66 * U32 * (x.double().abs() @ wt.double().abs().T)).all()


def test_python_refusals(ee):
    x, w = torch.zeros(4, 64, device="cuda"), torch.zeros(48, 64, device="cuda")
    ids, wt = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    gu, dn = torch.zeros(3, 64, 64, device="cuda"), torch.zeros(3, 64, 32, device="cuda")
    bad = [lambda: ee.linear(x.double(), w.double()), lambda: ee.linear(x, w.bfloat16()), lambda: ee.linear(x, w[:, :32]),
           lambda: ee.linear(x, w.cpu()), lambda: ee.linear(x, w, act="tanh"), lambda: ee.linear(x.t(), w),
           lambda: ee.linear(x, w, bias=torch.zeros(48, device="cuda", dtype=torch.bfloat16)),
           lambda: ee.linear(x, w, residual=torch.zeros(4, 47, device="cuda")), lambda: ee.linear(x, w, out_dtype=torch.bfloat16),
           lambda: ee.linear(x, w, out=torch.zeros(4, 96, device="cuda")[:, ::2]), lambda: ee.linear(x[0], w),
           lambda: ee.linear(x[:, :40].contiguous(), w[:, :40].contiguous()),
           lambda: ee.linear(x, w.clone().requires_grad_()),
           lambda: ee.moe_route(x, 0), lambda: ee.moe_route(x, 65), lambda: ee.moe_route(x, 4, score="tanh"),
           lambda: ee.moe_route(x, 4, n_groups=5), lambda: ee.moe_route(x, 4, bias=torch.zeros(63, device="cuda")),
           lambda: ee.moe_ffn(x, gu, dn, ids.long(), wt), lambda: ee.moe_ffn(x, gu, dn, ids, wt[:3]),
           lambda: ee.moe_ffn(x, gu[:2], dn, ids, wt), lambda: ee.moe_ffn(x, gu, dn.transpose(1, 2), ids, wt),
           lambda: ee.moe_ffn(x.bfloat16(), gu, dn, ids, wt), lambda: ee.moe_ffn(x, gu, dn, ids, wt, workspace=x)]
    for i, call in enumerate(bad):
        with pytest.raises(ee.EEError) as e:
            call()
        assert e.value.code == ee.EE_EINVAL, i
    with torch.no_grad():
        ee.linear(x, w.clone().requires_grad_())


def test_more_python_refusals(ee):
    x, w = torch.zeros(4, 64, device="cuda"), torch.zeros(64, 64, device="cuda")
    for i, call in enumerate((lambda: ee.linear(x, w, out=x), lambda: ee.linear(x, w, out=5), lambda: ee.linear(x, w, out=np.zeros((4, 64))),
                              lambda: ee.moe_route(x, 1 << 40), lambda: ee.moe_route(x, 4, n_groups=1 << 40),
                              lambda: ee.moe_route(x, 4, scale=float("inf")), lambda: ee.moe_route(x, 4, scale=None),
                              lambda: ee.linear(x.expand(4, 64)[:1].expand(4, 64), w))):
        with pytest.raises(ee.EEError) as e:
            call()
        assert e.value.code == ee.EE_EINVAL, i


def test_empty_calls(ee):
    w = torch.randn(48, 64, device="cuda")
    assert ee.linear(torch.empty(0, 64, device="cuda"), w).shape == (0, 48)
    ids, wt = ee.moe_route(torch.empty(0, 16, device="cuda"), 4)
    assert ids.shape == wt.shape == (0, 4)
    y = ee.moe_ffn(torch.empty(0, 64, device="cuda"), torch.randn(4, 64, 64, device="cuda"),
                   torch.randn(4, 64, 32, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"),
                   torch.empty(0, 2, device="cuda"))
    assert y.shape == (0, 64)


def _steps_case(rows, d, E, k, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, d, generator=g, device="cuda").to(torch.bfloat16)
    gu = (torch.randn(E, 64, d, generator=g, device="cuda") * d ** -0.5).to(torch.bfloat16)
    dn = (torch.randn(E, d, 32, generator=g, device="cuda") * 0.2).to(torch.bfloat16)
    ids = torch.randint(-1, E, (rows, k), generator=g, device="cuda", dtype=torch.int32)
    return x, gu, dn, ids, torch.rand(rows, k, generator=g, device="cuda")


def test_a_workspace_of_the_callers_around_a_step(ee):
    """Fewer rows that hold more columns of down products, in a workspace for the
    most rows; the bytes behind it stay."""
    d, E, k = 2048, 16, 8
    most = ee.ee_moe_ffn_workspace_bytes(4160, E, k, d, 32, ee.EE_BF16)
    ws = torch.full((most + (64 << 20),), 165, dtype=torch.uint8, device="cuda")
    a = _steps_case(4160, d, E, k, 31)
    whole = ee.moe_ffn(*a)
    for rows in (4160, 4097, 4096, 4095, 3641, 3640, 33):
        x, gu, dn, ids, w = a
        assert torch.equal(ee.moe_ffn(x[:rows], gu, dn, ids[:rows], w[:rows], workspace=ws[:most]), whole[:rows]), rows
        assert (ws[most:] == 165).all(), rows


def test_a_call_in_parts_stays_inside_its_workspace(ee):
    """1030 rows, 2^21 elements apart, run as 1023 and 7: the first part holds 2048
    columns of down products where the whole call would hold 1792."""
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GiB")
    rows, d, E, k, ld = 1030, 8192, 32, 32, 1 << 21
    x, gu, dn, ids, w = _steps_case(rows, d, E, k, 32)
    apart = torch.empty(rows * ld, dtype=x.dtype, device="cuda").as_strided((rows, d), (ld, 1))
    apart.copy_(x)
    most = ee.ee_moe_ffn_workspace_bytes(rows, E, k, d, 32, ee.EE_BF16)
    ws = torch.full((most + (64 << 20),), 165, dtype=torch.uint8, device="cuda")
    want = ee.moe_ffn(x, gu, dn, ids, w)
    assert torch.equal(ee.moe_ffn(apart, gu, dn, ids, w, workspace=ws[:most]), want)
    assert (ws[most:] == 165).all()


def test_one_row_of_any_stride(ee):
    """The last position of one sequence: its row's stride is past what the library
    takes, or no multiple of 16 bytes."""
    g = _gen(33)
    d, f, E, k = 256, 64, 8, 2
    w, gu, dn = _rand(g, 96, d).cuda(), _rand(g, E, 2 * f, d, std=0.1).cuda(), _rand(g, E, d, f, std=0.1).cuda()
    for stride in ((1 << 21) + 4, 1001):
        h = torch.zeros(stride + d, device="cuda").as_strided((1, d), (stride, 1))
        h.copy_(_rand(g, 1, d))
        x, r = h.clone(), _rand(g, 1, 96).cuda()
        assert torch.equal(ee.linear(h, w), ee.linear(x, w))
        assert torch.equal(ee.linear(x, h), ee.linear(x, x))
        ids, wt = ee.moe_route(h[:, :32], k)
        assert torch.equal(ids, ee.moe_route(x[:, :32].contiguous(), k)[0])
        ids = ids % E
        want = ee.moe_ffn(x, gu, dn, ids, wt, residual=x)
        assert torch.equal(ee.moe_ffn(h, gu, dn, ids, wt, residual=h), want)
        want = ee.linear(x, w, residual=r)
        y = torch.zeros(stride + 96, device="cuda").as_strided((1, 96), (stride, 1))
        y.copy_(r)
        assert ee.linear(h, w, residual=y, out=y) is y and torch.equal(y, want)


def test_forward_mode_tangents_are_refused(ee):
    """A tangent would be lost without a word."""
    from torch.autograd import forward_ad
    g = _gen(34)
    x, w, b, r = _rand(g, 4, 64).cuda(), _rand(g, 64, 64).cuda(), _rand(g, 64).cuda(), _rand(g, 4, 64).cuda()
    gu, dn = _rand(g, 3, 64, 64).cuda(), _rand(g, 3, 64, 32).cuda()
    ids, wt = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.rand(4, 2, device="cuda")
    want = ee.linear(x, w, bias=b, residual=r), ee.moe_route(x, 2), ee.moe_ffn(x, gu, dn, ids, wt, residual=r)
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))
        for i, call in enumerate((lambda: ee.linear(dual(x), w), lambda: ee.linear(x, dual(w)), lambda: ee.linear(x, w, bias=dual(b)),
                                  lambda: ee.linear(x, w, residual=dual(r)), lambda: ee.linear(x, w, out=dual(r)),
                                  lambda: ee.moe_route(dual(x), 2), lambda: ee.moe_route(x, 2, bias=dual(b)),
                                  lambda: ee.moe_ffn(dual(x), gu, dn, ids, wt), lambda: ee.moe_ffn(x, dual(gu), dn, ids, wt),
                                  lambda: ee.moe_ffn(x, gu, dual(dn), ids, wt), lambda: ee.moe_ffn(x, gu, dn, ids, dual(wt)),
                                  lambda: ee.moe_ffn(x, gu, dn, ids, wt, residual=dual(r)),
                                  lambda: ee.moe_ffn(x, gu, dn, ids, wt, out=dual(r)))):
            with pytest.raises(ee.EEError) as e:
                call()
            assert e.value.code == ee.EE_EINVAL and "tangent" in str(e.value), i
        # operands without one are served
        assert torch.equal(ee.linear(x, w, bias=b, residual=r), want[0])
        assert torch.equal(ee.moe_route(x, 2)[0], want[1][0])
        assert torch.equal(ee.moe_ffn(x, gu, dn, ids, wt, residual=r), want[2])


def test_autograd_notices_an_output_that_it_saved(ee):
    g = _gen(35)
    x, w = _rand(g, 4, 64).cuda(), _rand(g, 64, 64).cuda()
    for call in (lambda h: ee.linear(x, w, residual=h, out=h),
                 lambda h: ee.moe_ffn(x, w.expand(3, 64, 64).contiguous(), w[None, :, :32].expand(3, 64, 32).contiguous(),
                                      torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.ones(4, 2, device="cuda"), out=h)):
        p, h = torch.ones(4, 64, device="cuda", requires_grad=True), torch.ones(4, 64, device="cuda")
        loss = (p * h).sum()
        assert call(h) is h
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()


@pytest.mark.parametrize("rows", [5, 300, 3000])
def test_one_expert_per_row_stays_inside_its_workspace(ee, rows):
    x, gu, dn, ids, w = [t.cuda() for t in _ffn_inputs(rows, 544, 96, 5, 1, "bf16", seed=rows)]
    most = ee.ee_moe_ffn_workspace_bytes(rows, 5, 1, 544, 96, ee.EE_BF16)
    ws = torch.full((most + (16 << 20),), 165, dtype=torch.uint8, device="cuda")
    assert torch.equal(ee.moe_ffn(x, gu, dn, ids, w, workspace=ws[:most]), ee.moe_ffn(x, gu, dn, ids, w))
    assert (ws[most:] == 165).all()


@pytest.mark.parametrize("rows,E,k", [(131073, 64, 4), (300007, 5, 2), (600011, 3, 1)])
def test_pairs_sorted_in_longer_chunks(ee, rows, E, k):
    """From 2^19 pairs on the sorting workgroups' chunks grow: every pair is in the
    order once, so every row is what few of them alone give."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, 32, generator=g, device="cuda").to(torch.bfloat16)
    gu = (torch.randn(E, 64, 32, generator=g, device="cuda") * 0.2).to(torch.bfloat16)
    dn = (torch.randn(E, 32, 32, generator=g, device="cuda") * 0.2).to(torch.bfloat16)
    ids = torch.randint(-1, E, (rows, k), generator=g, device="cuda", dtype=torch.int32)
    w = torch.rand(rows, k, generator=g, device="cuda")
    want = torch.cat([ee.moe_ffn(x[i:i + 50000], gu, dn, ids[i:i + 50000], w[i:i + 50000]) for i in range(0, rows, 50000)])
    out = torch.full((rows, 32), 7.0, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(ee.moe_ffn(x, gu, dn, ids, w, out=out), want)
    pick = torch.arange(0, rows, 997, device="cuda")
    ref, err = _ffn64(x[pick], gu, dn, ids[pick], w[pick], None, "bf16")
    _close(out[pick], ref.cpu(), (err + UBF * (ref.abs() + err) + 2 * U32 * ref.abs() + 1e-30).cpu())


@pytest.mark.parametrize("make", [lambda m: -np.log((1 + m) * 2.0 ** -52), lambda m: -np.log((30000 + m) * 2.0 ** -52),
                                  lambda m: -np.log(((1 << 20) + m) * 2.0 ** -52), lambda m: -709.78 + m * 1.3e-3,
                                  lambda m: -708.3 + m * 0.02])
def test_route_distinct_scores_near_their_bounds(ee, make):
    """Sigmoid scores one or a few steps of float64 apart, just below 1 (logits of 22
    to 36) and where they are about to leave the normal numbers: the order is the
    definition's, and equal scores go to the lower index."""
    l = make(np.arange(1024)).astype(np.float32)
    rng = np.random.default_rng(36)
    rows = np.stack([rng.permutation(l) for _ in range(16)])
    for E in (64, 1024):
        part = rows[:, :E]
        ids, w = ee.moe_route(torch.from_numpy(part).contiguous().cuda(), 32, score="sigmoid", renormalize=False)
        score = 1 / (1 + np.exp(-part.astype(np.float64)))
        want = np.argsort(-score, axis=1, kind="stable")[:, :32]
        assert np.array_equal(ids.cpu().numpy(), want)
        np.testing.assert_allclose(w.cpu().numpy(), np.take_along_axis(score, want, 1), rtol=U32 * (1 + 1e-6), atol=2.0 ** -149)
