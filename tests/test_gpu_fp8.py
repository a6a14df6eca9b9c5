"""The 8-bit operators (fp8_quant, fp8_linear) on the GPU against plain float64
implementations written here.

Tolerances.  Codes and scales have a definition whose steps are single IEEE
roundings, so they are compared bit for bit.  A product: a block's sum of 128
products, times a scale that is one rounding off, joined to the chain by one fma per block:
with n = ceil(in / 128) blocks and s = sum over blocks of scale sum |x w|, (128 + n + 3)
2^-24 s where the sums are float32.  The 8-bit matrix instruction aligns every eight
columns' products to the largest of them and drops what lies 2^13 below its power of
two: seven dropped parts of less than 2^-13 of the largest each, so 7 2^-13 times the
sum of every eight columns' largest product.  An output in bf16 is half a step off, 2^-8 of the value at most."""

import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu

U32, UBF = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ee():
    import paper_2506_02780_amd as mod
    return mod


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rand(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def _padded(t, pad, fill=float("nan")):
    rows, cols = t.shape
    base = torch.full((rows, cols + pad), fill, dtype=torch.float32, device="cuda").to(t.dtype)
    base[:, :cols] = t.cuda()
    return base[:, :cols]


def _e4m3_64(v):
    """Nearest e4m3 values (even on ties) of float64 within its range."""
    a = v.abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(v) * (torch.round(a / step) * step)


def _blocks64(t, block_rows):
    """[row blocks, block_rows, column blocks, 128], zeros behind the ends."""
    R, C = t.shape
    out = torch.zeros(-(-R // block_rows) * block_rows, -(-C // 128) * 128, dtype=torch.float64, device=t.device)
    out[:R, :C] = t.double()
    return out.reshape(-1, block_rows, out.shape[1] // 128, 128)


def _scaled64(codes, scales, block_rows):
    R, C = codes.shape
    b = _blocks64(codes.float(), block_rows) * scales.double()[:, None, :, None]
    return b.reshape(-1, b.shape[2] * 128)[:R, :C]


# ----------------------------------------------------------------- quantise --

def _quant_case(ee, x, block_rows, **kw):
    codes, scales = ee.fp8_quant(x, block_rows=block_rows, **kw)
    assert codes.dtype is E4M3 and scales.dtype is torch.float32 and codes.shape == x.shape
    b = _blocks64(x.float(), block_rows)
    size = b.abs()
    amax = torch.where(torch.isfinite(size), size, 0.0).amax((1, 3))
    # one float32 rounding of the quotient (a float64 quotient of float32 values rounds to float32 as the exact one would)
    want = torch.maximum((amax / 448.0).float(), torch.tensor(2.0 ** -126, device="cuda"))
    assert torch.equal(scales, want)
    q = (b / want.double()[:, None, :, None]).float().double().clamp(-448.0, 448.0)
    q = q.reshape(-1, q.shape[2] * 128)[:x.shape[0], :x.shape[1]]
    got = codes.float().double()
    nan = torch.isnan(x)
    assert torch.isnan(got[nan]).all()
    assert torch.equal(got[~nan], _e4m3_64(q)[~nan])
    assert torch.equal(torch.signbit(got[~nan]), torch.signbit(x[~nan]))
    return codes, scales


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows", [1, 2, 3, 31, 33, 127, 128, 129, 300])
@pytest.mark.parametrize("cols", [16, 112, 128, 144, 256, 1024, 1040, 2064])
def test_quant_sizes(ee, rows, cols, block_rows, dtype):
    g = _gen(rows + cols)
    x = (_rand(g, rows, cols) * torch.exp2(_rand(g, 1, cols, std=4.0))).to(DT[dtype]).cuda()
    _quant_case(ee, x, block_rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quant_special_values(ee, block_rows, dtype):
    """NaN, infinities, zeros, the smallest and largest values, and ties."""
    g = _gen(3)
    x = _rand(g, 140, 512)
    x[0, :128] = 0.0
    x[1, 5], x[1, 200] = float("nan"), float("inf")
    x[2, 130] = -float("inf")
    x[3] = float("nan")
    x[4] = float("inf")
    x[5, :128] = 2.0 ** -133        # below the smallest scale times the largest code
    x[6] = torch.finfo(DT[dtype]).max
    x[7] = -0.0
    x[8, :128] = torch.arange(128) * 3.5 + 3.5      # 448 at the end: scale 1, ties between codes
    x[9, :128] = -x[8, :128]
    x[10, 0], x[10, 1:128] = 448.0, 2.0 ** -10      # half of the smallest code
    x[11, 0], x[11, 1:128] = 448.0, 2.0 ** -10 * 1.0078125
    x = x.to(DT[dtype]).cuda()
    _quant_case(ee, x, block_rows)
    _quant_case(ee, x[:12].contiguous(), block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quant_quotients_at_ties(ee, block_rows):
    """Quotients at, just above and just below the middle between two codes, at scales from the
    smallest to the largest: each rounds as the IEEE quotient does."""
    g = _gen(11)
    rows = 128 * 70
    amax = torch.exp2(torch.linspace(-149, 127.9, rows // block_rows, dtype=torch.float64)) * (1 + torch.rand(rows // block_rows, generator=g).double())
    amax = amax.float().clamp(max=3.4e38).repeat_interleave(block_rows)
    scale = torch.maximum((amax.double() / 448).float(), torch.tensor(2.0 ** -126)).double()
    codes = torch.arange(0, 126, dtype=torch.uint8)
    low, high = codes.view(E4M3).double(), (codes + 1).view(E4M3).double()
    mid = torch.cat([(low + high) / 2, high])[torch.randint(0, 252, (rows, 384), generator=g)]
    x = (mid * scale[:, None]).float()
    x = torch.where(x.abs() > amax[:, None], amax[:, None], x)
    step = torch.randint(-2, 3, (rows, 384), generator=g)
    x = (x.view(torch.int32) + step.to(torch.int32)).clamp(min=0).view(torch.float32)
    x = torch.minimum(x, amax[:, None]) * (1 - 2 * torch.randint(0, 2, (rows, 384), generator=g))
    x[:, ::128] = amax[:, None]
    _quant_case(ee, x.cuda(), block_rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quant_many_blocks(ee, dtype):
    x = _rand(_gen(12), 20001, 2064, std=3.0, dtype=DT[dtype])
    x[::7] *= 2.0 ** -100
    x[5::11, ::3] = -0.0
    x[3, 7], x[20000, 2063], x[19999, 100] = float("nan"), float("inf"), -float("inf")
    _quant_case(ee, x.cuda(), 1)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quant_strides_and_outputs(ee, block_rows):
    g = _gen(4)
    for dtype, pad in (("bf16", 8), ("f32", 4), ("bf16", 40)):
        x = _rand(g, 133, 272, dtype=DT[dtype])
        a, s = _quant_case(ee, _padded(x, pad), block_rows)
        base = torch.full((133, 304), 9.0, device="cuda").to(E4M3)
        scales = torch.empty_like(s)
        got = ee.fp8_quant(x.cuda(), block_rows=block_rows, codes=base[:, :272], scales=scales)
        assert got[1] is scales and torch.equal(scales, s)
        assert torch.equal(base[:, :272].float(), a.float()) and (base[:, 272:].float() == 9.0).all()


def test_quant_rows_do_not_depend_on_the_others(ee):
    x = _rand(_gen(5), 200, 400, dtype=torch.bfloat16).cuda()
    codes, scales = ee.fp8_quant(x)
    for lo, n in ((0, 1), (7, 33), (199, 1), (50, 128)):
        c, s = ee.fp8_quant(x[lo:lo + n])
        assert torch.equal(c.float(), codes[lo:lo + n].float()) and torch.equal(s, scales[lo:lo + n])


def test_quant_past_32_bit_offsets(ee):
    rows = 70000
    x = torch.zeros(rows, 65536, dtype=torch.bfloat16, device="cuda")      # 9.2 GB; codes past 2^32
    x[-1] = _rand(_gen(6), 1, 65536, dtype=torch.bfloat16).cuda()[0]
    x[rows // 2] = x[-1] * 2
    codes, scales = ee.fp8_quant(x)
    for r in (0, rows // 2, rows - 1):
        c, s = ee.fp8_quant(x[r:r + 1].clone())
        assert torch.equal(codes[r:r + 1].float(), c.float()) and torch.equal(scales[r:r + 1], s)
    assert (scales[1:rows // 2] == 2.0 ** -126).all()
    codes, scales = ee.fp8_quant(x, block_rows=128)
    c, s = ee.fp8_quant(x[-(rows % 128):].clone(), block_rows=128)
    assert torch.equal(codes[-(rows % 128):].float(), c.float()) and torch.equal(scales[-1:], s)


# ------------------------------------------------------------------- linear --

def _act64(v, act):
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v / 2.0 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3)))
    return v.clamp(min=0) if act == "relu" else v


def _operands(g, rows, k, n, spread=1.0):
    """Codes of every size and scales far apart, made without the library."""
    def one(r, scale_rows, std):
        v = (_rand(g, r, k, std=60.0) * torch.exp2(_rand(g, r, k, std=spread))).clamp(-448, 448)
        return v.to(E4M3).cuda(), (std * torch.exp2(_rand(g, scale_rows, -(-k // 128)))).cuda()
    x, xs = one(rows, rows, 1.0 / 60)
    w, ws = one(n, -(-n // 128), k ** -0.5 / 60)
    return x, xs, w, ws


def _sum_of_largest(x, w):
    """sum over every eight columns of the largest |x w|, [rows, out] in float64."""
    rows, k = x.shape
    out = torch.zeros(rows, w.shape[0], dtype=torch.float64, device=x.device)
    for c in range(0, k, 8):
        best = torch.zeros_like(out)
        for i in range(c, min(c + 8, k)):
            best = torch.maximum(best, x[:, i, None].abs() * w[None, :, i].abs())
        out += best
    return out


def _product64(x, xs, w, ws, out):
    """(x w^T, its bound) in float64."""
    a, b = _scaled64(x, xs, 1), _scaled64(w, ws, 128)
    pre = torch.mm(a, b.T.contiguous())
    err = (128 + a.shape[1] // 128 + 4) * U32 * torch.mm(a.abs(), b.abs().T.contiguous())
    if out == "bf16":
        err = err + 7 * 2.0 ** -13 * _sum_of_largest(a, b)
    return pre, err


def _linear_case(ee, rows, k, n, out, act="none", bias=False, residual=False, pad=0, opad=0, seed=0, spread=1.0):
    g = _gen(seed)
    x, xs, w, ws = _operands(g, rows, k, n, spread)
    b = _rand(g, n).cuda() if bias else None
    r = _rand(g, rows, n, dtype=DT[out]) if residual else None
    whole = torch.full((rows, n + opad), 7.0, dtype=DT[out], device="cuda")
    y = whole[:, :n]
    got = ee.fp8_linear(_padded(x, pad), xs, _padded(w, pad), ws, bias=b, act=act,
                        residual=_padded(r, opad) if residual else None, out=y)
    assert got is y
    pre, err = _product64(x, xs, w, ws, out)
    if bias:
        pre = pre + b.double()
        err = err + 2 * U32 * pre.abs()
    want = _act64(pre, act)
    # the activations' slopes are below 1.2; their own evaluation takes a few float32 roundings
    err = 1.2 * err + 16 * U32 * (pre.abs() if act != "none" else 0 * pre)
    if residual:
        want = want + r.cuda().double()
    err = err + (UBF if out == "bf16" else U32) * (want.abs() + err) + U32 * want.abs() + 1e-30
    bad = ~((y.double() - want).abs() <= err)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float(((y.double() - want).abs() / err).max())} x the bound"
    assert (whole[:, n:] == 7.0).all(), "columns past the output were written"
    return y


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 65, 129, 257, 513])
def test_linear_rows(ee, rows, out):
    _linear_case(ee, rows, 256, 272, out, bias=True, seed=rows)


@pytest.mark.parametrize("n", [1, 3, 4, 15, 16, 17, 63, 64, 100, 127, 128, 129, 255, 257, 528, 777])
@pytest.mark.parametrize("rows", [1, 20, 300])
def test_linear_columns(ee, rows, n):
    _linear_case(ee, rows, 128, n, "bf16", act="silu", residual=True, seed=n)
    _linear_case(ee, rows, 144, n, "f32", act="relu", bias=True, seed=n)


@pytest.mark.parametrize("k", [16, 32, 64, 80, 112, 128, 144, 240, 256, 272, 384, 400, 640, 1024, 1040, 2064, 4112])
@pytest.mark.parametrize("rows,n", [(1, 48), (5, 300), (40, 160), (270, 130)])
def test_linear_reduction(ee, rows, n, k):
    _linear_case(ee, rows, k, n, "bf16", seed=k)
    _linear_case(ee, rows, k, n, "f32", seed=k)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("rows,n", [(3, 130), (70, 530), (300, 258)])
def test_linear_epilogues(ee, rows, n, act):
    for bias, residual in itertools.product((False, True), repeat=2):
        _linear_case(ee, rows, 160, n, "bf16", act=act, bias=bias, residual=residual, seed=5)
        _linear_case(ee, rows, 160, n, "f32", act=act, bias=bias, residual=residual, seed=6)


@pytest.mark.parametrize("rows,n", [(1, 64), (19, 129), (300, 512)])
def test_linear_strides(ee, rows, n):
    for opad in (0, 1, 4, 5, 8):
        _linear_case(ee, rows, 96, n, "bf16", bias=True, residual=True, pad=16, opad=opad, seed=7)
        _linear_case(ee, rows, 272, n, "f32", residual=True, pad=48, opad=opad, seed=8)


def test_linear_products_of_very_different_size(ee):
    for rows in (1, 33, 200):
        _linear_case(ee, rows, 512, 96, "bf16", seed=rows, spread=4.0)
        _linear_case(ee, rows, 512, 96, "f32", seed=rows, spread=4.0)


def _dropped(x, xs, w, ws):
    """What the 8-bit instruction may drop, [rows, out] in float64: of every eight columns' products those with bits
    below 2^-13 of the largest one's power of two lose less than that each."""
    x64, w64 = x.float().double(), w.float().double()
    rows, k = x.shape
    out = torch.zeros(rows, w.shape[0], dtype=torch.float64, device=x.device)
    for c in range(0, k, 8):
        p = (x64[:, None, c:c + 8] * w64[None, :, c:c + 8]).abs()
        cut = torch.exp2(torch.floor(torch.log2(p.amax(-1).clamp(min=2.0 ** -18))) - 13)      # (2^-18: the least product)
        part = (p / cut[..., None]).frac().ne(0).sum(-1)
        out += part * cut * xs[:, c // 128, None].double() * ws[torch.arange(len(w), device=w.device) // 128, c // 128].double()
    return out


@pytest.mark.parametrize("rows", [1, 33, 200])
@pytest.mark.parametrize("k", [8 * 16, 272, 1040])
def test_linear_drops_no_more_than_its_instruction(ee, rows, k):
    """Random codes, product by product."""
    for spread in (0.0, 1.0, 3.0):
        x, xs, w, ws = _operands(_gen(rows + k), rows, k, 70, spread)
        y = ee.fp8_linear(x, xs, w, ws).double()
        a, b = _scaled64(x, xs, 1), _scaled64(w, ws, 128)
        want = torch.mm(a, b.T.contiguous())
        err = (128 + k // 128 + 4) * U32 * torch.mm(a.abs(), b.abs().T.contiguous()) + _dropped(x, xs, w, ws)
        assert ((y - want).abs() <= err + UBF * (want.abs() + err)).all()


@pytest.mark.parametrize("rows", [1, 33, 200])
def test_linear_loud_columns(ee, rows):
    """One product of 2^16 beside seven of 7.5 in every eight columns, which is where bf16's shortened sums lose most (7 2^-13 of the
    largest); then the loud ones cancel, and what is left is what an output in float32 keeps."""
    k, n = 256, 40
    quiet, ones = torch.full((rows, k), 7.5), torch.ones(n, k)
    scale = torch.ones(rows, 2, device="cuda"), torch.ones(1, 2, device="cuda")
    for cancel in (False, True):
        for at in range(8):
            x, w = quiet.clone(), ones.clone()
            x[:, at::8], w[:, at::8] = 256.0, 256.0
            if cancel:
                w[:, at + 8::16] = -256.0
            want = torch.mm(x.double(), w.double().T)
            most = float(torch.mm(x.double().abs(), w.double().abs().T).max())
            x8, w8 = x.to(E4M3).cuda(), w.to(E4M3).cuda()
            exact = ee.fp8_linear(x8, scale[0], w8, scale[1], out_dtype=torch.float32).cpu().double()
            assert ((exact - want).abs() <= (128 + 2 + 4) * U32 * most).all()
            y = ee.fp8_linear(x8, scale[0], w8, scale[1]).cpu().double()
            bound = 7 * 2.0 ** -13 * (k // 8) * 65536.0
            assert ((y - want).abs() <= bound + UBF * (want.abs() + bound)).all(), (at, cancel)


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_linear_nan_stays_in_its_row_and_column(ee, out):
    x, xs, w, ws = _operands(_gen(4), 40, 320, 150)
    clean = ee.fp8_linear(x, xs, w, ws, out_dtype=DT[out])
    x.view(torch.uint8)[7, 3] = 0x7f
    xs[11, 1] = float("inf")
    w.view(torch.uint8)[20, 319] = 0xff
    got = ee.fp8_linear(x, xs, w, ws, out_dtype=DT[out])
    assert torch.isnan(got[7]).all() and torch.isnan(got[:, 20]).all() and not torch.isfinite(got[11]).any()
    rows, cols = [i for i in range(40) if i not in (7, 11)], [i for i in range(150) if i != 20]
    assert torch.equal(got[rows][:, cols], clean[rows][:, cols])


def test_linear_does_not_read_behind_its_reduction(ee):
    """Codes past `in` of a wider operand may be anything."""
    for k in (16, 48, 144, 208):
        x, xs, w, ws = _operands(_gen(k), 37, k, 70)
        wide_x, wide_w = _padded(x, 112), _padded(w, 112)     # (NaN behind)
        for out in DT.values():
            assert torch.equal(ee.fp8_linear(wide_x, xs, wide_w, ws, out_dtype=out), ee.fp8_linear(x, xs, w, ws, out_dtype=out))


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("n,k", [(1, 512), (128, 1040), (600, 384), (2048, 512), (300, 8320)])
def test_linear_rows_do_not_depend_on_the_others(ee, out, n, k):
    x, xs, w, ws = _operands(_gen(n), 1100, k, n)
    whole = ee.fp8_linear(x, xs, w, ws, act="silu", out_dtype=DT[out])
    for rows in (1, 7, 16, 17, 33, 48, 64, 65, 130, 256, 513, 1024):
        for lo in (0, 1100 - rows):
            part = ee.fp8_linear(x[lo:lo + rows], xs[lo:lo + rows], w, ws, act="silu", out_dtype=DT[out])
            assert torch.equal(part, whole[lo:lo + rows]), (rows, lo)


@pytest.mark.parametrize("k", [272, 512])
@pytest.mark.parametrize("rows,n", [(7, 10240), (17, 4200), (21, 10241), (33, 10300), (65, 10250), (135, 11001), (1537, 1303), (261, 10245),
                                    (515, 10250), (4201, 1303), (2049, 4205), (3001, 11008)])
def test_linear_of_every_tile(ee, rows, n, k):
    """Sizes at which each of the tiles runs (the last one's features in two launches), with
    ragged edges: against float64, and bit for bit the rows alone."""
    for out in ("bf16", "f32"):
        y = _linear_case(ee, rows, k, n, out, act="silu", bias=True, residual=True, seed=rows)
        g = _gen(rows)
        x, xs, w, ws = _operands(g, rows, k, n)
        b = _rand(g, n).cuda()
        r = _rand(g, rows, n, dtype=DT[out]).cuda()
        for lo, hi in ((0, 1), (rows // 2, rows // 2 + 3), (rows - 6, rows)):
            part = ee.fp8_linear(x[lo:hi], xs[lo:hi], w, ws, bias=b, act="silu", residual=r[lo:hi], out_dtype=DT[out])
            assert torch.equal(part, y[lo:hi]), (out, lo)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("n", [2048, 2049, 2052])
def test_linear_epilogues_of_all_kernels(ee, n, act, out):
    """Bit for bit, each activation with and without bias and residual: rows alone (blocks of the reduction spread over waves)
    and among 150 (tiles; their stores 16 and 8 bytes wide and one value at a time)."""
    g = _gen(n)
    x, xs, w, ws = _operands(g, 150, 272, n)
    b, r = _rand(g, n).cuda(), _rand(g, 150, n, dtype=DT[out]).cuda()
    for bias, residual in itertools.product((None, b), (None, r)):
        y = ee.fp8_linear(x, xs, w, ws, bias=bias, act=act, residual=residual, out_dtype=DT[out])
        for lo, hi in ((0, 1), (63, 67), (148, 150)):
            part = ee.fp8_linear(x[lo:hi], xs[lo:hi], w, ws, bias=bias, act=act, residual=None if residual is None else r[lo:hi],
                                 out_dtype=DT[out])
            assert torch.equal(part, y[lo:hi]), (bias is not None, residual is not None, lo)


def test_linear_residual_in_place(ee):
    x, xs, w, ws = _operands(_gen(3), 33, 256, 96)
    h = _rand(_gen(1), 33, 96, dtype=torch.bfloat16).cuda()
    want = ee.fp8_linear(x, xs, w, ws, residual=h.clone())
    assert ee.fp8_linear(x, xs, w, ws, residual=h, out=h) is h
    assert torch.equal(h, want)


def test_linear_past_32_bit_offsets(ee):
    """Weights of 4.4 GB, and outputs past 2^32 bytes."""
    n, k = 270000, 16384
    x, xs, _, _ = _operands(_gen(8), 20, k, 16)
    w = torch.zeros(n, k, dtype=torch.uint8, device="cuda").view(E4M3)
    _, _, part, _ = _operands(_gen(9), 1, k, 300)
    w.view(torch.uint8)[-300:] = part.view(torch.uint8)
    ws = torch.full((-(-n // 128), 128), 0.001, device="cuda")
    for rows in (1, 20):
        y = ee.fp8_linear(x[:rows], xs[:rows], w, ws)
        assert (y[:, :-300] == 0).all()
        # (their scales are all one number, so the block borders do not matter)
        want, err = _product64(x[:rows], xs[:rows], part, ws[:3], "bf16")
        assert ((y[:, -300:].double() - want).abs() <= err + UBF * (want.abs() + err)).all()
    del w, y
    x, xs, w, ws = _operands(_gen(10), 40000, 16, 65536)
    y = ee.fp8_linear(x, xs, w, ws)
    for lo in (0, 20000, 39990):
        assert torch.equal(y[lo:lo + 10], ee.fp8_linear(x[lo:lo + 10], xs[lo:lo + 10], w, ws))


def test_quant_then_linear(ee):
    """As they are used: the product of quantised operands, near that of the originals."""
    g = _gen(11)
    a, b = _rand(g, 50, 1000 // 16 * 16).cuda(), _rand(g, 200, 1000 // 16 * 16, std=0.03).cuda()
    x, xs = ee.fp8_quant(a)
    w, ws = ee.fp8_quant(b, block_rows=128)
    y = ee.fp8_linear(x, xs, w, ws, out_dtype=torch.float32)
    want = torch.mm(_scaled64(x, xs, 1), _scaled64(w, ws, 128).T.contiguous())
    assert float((y.double() - want).abs().max()) < 1e-5
    # codes are half a step off, 2^-4 of a value (or of the smallest normal code's: 2^-10 scale)
    ea, eb = a.double().abs() * 2.0 ** -4 + 2.0 ** -10 * _scaled64(torch.ones_like(x.float()), xs, 1), b.double().abs() * 2.0 ** -4 + 2.0 ** -10 * _scaled64(torch.ones_like(w.float()), ws, 128)
    bound = torch.mm(ea, (b.double().abs() + eb).T.contiguous()) + torch.mm(a.double().abs(), eb.T.contiguous())
    assert ((y.double() - torch.mm(a.double(), b.double().T.contiguous())).abs() <= bound + 1e-5).all()


def test_captured_into_a_graph(ee):
    g = _gen(12)
    a, b = _rand(g, 33, 512, dtype=torch.bfloat16).cuda(), _rand(g, 260, 512, dtype=torch.bfloat16).cuda()
    w, ws = ee.fp8_quant(b, block_rows=128)

    def step():
        x, xs = ee.fp8_quant(a)
        return ee.fp8_linear(x, xs, w, ws, act="gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    for i in range(4):
        a.copy_(_rand(_gen(20 + i), 33, 512, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, step()), i


def test_python_refusals(ee):
    x, xs, w, ws = _operands(_gen(13), 20, 256, 200)
    h = torch.zeros(20, 256, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: ee.fp8_linear(x.float(), xs, w, ws), lambda: ee.fp8_linear(x, xs[:, :1], w, ws),
                 lambda: ee.fp8_linear(x, xs, w, ws[:1]), lambda: ee.fp8_linear(x, xs, w.view(torch.uint8), ws),
                 lambda: ee.fp8_linear(x, xs.double(), w, ws), lambda: ee.fp8_linear(x, xs, w, ws, act="tanh"),
                 lambda: ee.fp8_linear(x, xs, w, ws, out_dtype=torch.float16), lambda: ee.fp8_linear(x, xs.t().contiguous().t(), w, ws),
                 lambda: ee.fp8_linear(x, xs, w, ws, out=h), lambda: ee.fp8_linear(x[:, :250], xs, w[:, :250], ws),
                 lambda: ee.fp8_linear(x.cpu(), xs, w, ws), lambda: ee.fp8_linear(x, xs.requires_grad_(True), w, ws),
                 lambda: ee.fp8_quant(h.half()), lambda: ee.fp8_quant(h, block_rows=64), lambda: ee.fp8_quant(h[:, :250]),
                 lambda: ee.fp8_quant(h.t()), lambda: ee.fp8_quant(h, codes=x[:10]), lambda: ee.fp8_quant(h, scales=xs[:1]),
                 lambda: ee.fp8_quant(h[0])):
        with pytest.raises(ee.EEError) as e:
            call()
        assert e.value.code == ee.EE_EINVAL


def test_no_rows(ee):
    x, xs, w, ws = _operands(_gen(14), 4, 128, 64)
    assert ee.fp8_linear(x[:0], xs[:0], w, ws).shape == (0, 64)
    c, s = ee.fp8_quant(torch.empty(0, 256, device="cuda"))
    assert c.shape == (0, 256) and s.shape == (0, 2)
