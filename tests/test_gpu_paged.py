"""The operators around a paged cache (kv_append, paged_attention) on the GPU
against plain float64 implementations written here.

Tolerances.  Appending: the rotation's two products and their sum, with factors
that are each 2^-23 off (float64 angle, float32 sine and cosine of it within two roundings): 6
2^-24 (|a| + |b|), and half a step of the type.  Values and what is not rotated
are copied.
Attention: a score is a float32 sum of head_dim products, (hd + 2) 2^-24 sum |q k|
off, and its weight's exponent is formed with three more roundings of the score and
of the largest score, each 2^-24 of |s| log2 e; the exponential is 2^-22 off.  With
d_j the sum of these (relative, of weight j), the result is sum_j p_j d_j (|v_j| +
|o|) off, besides its own sums over n positions, (n + 8) 2^-24 sum p |v|, the 2^-16 of
weights as two bf16 parts, and the rounding to its type."""

import itertools

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def ee():
    import paper_2506_02780_amd as mod
    return mod


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rand(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def _cache(g, n_pages, page, heads, hd, dtype, layout="slots", fill=None):
    """(k, v) [n_pages, page, heads, hd] in one of several memory orders."""
    if layout == "slots":          # [page][slot][head]
        t = _rand(g, 2, n_pages, page, heads, hd, dtype=dtype).cuda()
    elif layout == "heads":        # [page][head][slot]
        t = _rand(g, 2, n_pages, heads, page, hd, dtype=dtype).cuda().transpose(2, 3)
    elif layout == "pairs":        # k and v of a page side by side
        t = _rand(g, n_pages, 2, page, heads, hd, dtype=dtype).cuda().transpose(0, 1)
    else:                          # room between the vectors
        t = _rand(g, 2, n_pages, page, heads + 1, hd + 16, dtype=dtype).cuda()[:, :, :, :heads, :hd]
    if fill is not None:
        t.fill_(fill)
    return t[0], t[1]


def _tables(g, lens, page, most=None, spare=2):
    """Pages of sequences in no order; -1 past their ends."""
    held = [-(-n // page) for n in lens]
    most = max(most or 0, max(held, default=0), 1)
    order = torch.randperm(sum(held) + spare, generator=g).tolist()
    t = torch.full((len(lens), most), -1, dtype=torch.int32)
    for i, n in enumerate(held):
        t[i, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    return t.cuda(), sum(held) + spare


# ------------------------------------------------------------------- append --

def _turn64(x, positions, inv_freq, interleaved):
    """(value, |a| + |b|) of rotated vectors [rows, heads, hd] in float64."""
    x = x.double().clone()
    size = torch.zeros_like(x)
    rot = 2 * len(inv_freq)
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    angle = positions.double()[:, None] * inv_freq
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = x[..., first].clone(), x[..., second].clone()
    x[..., first], x[..., second] = a * cos - b * sin, a * sin + b * cos
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return x, size


def _freq(rot, theta=10000.0):
    return theta ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / max(1, rot))


def _append_case(ee, *, rows, heads, kv, hd, dtype, page=64, rot=None, interleaved=False, layout="slots", n_seqs=3, queries=True,
                 far=0, positions=None, seqs=None, tables=None, seed=0, pad=0, in_place=False):
    g, dt = _gen(seed), DT[dtype]
    rot = hd if rot is None else rot
    if positions is None:
        at = [far + 5 * i for i in range(n_seqs)]
        seqs = torch.tensor([i % n_seqs for i in range(rows)], dtype=torch.int32, device="cuda")
        positions = torch.tensor([at[i % n_seqs] + i // n_seqs for i in range(rows)], dtype=torch.int32, device="cuda")
    most = max(0, int(positions.max())) // page + 1
    if tables is None:
        t = torch.full((n_seqs, most), -1, dtype=torch.int32)
        used = sorted({(int(s), int(p) // page) for s, p in zip(seqs, positions) if p >= 0 and 0 <= s < n_seqs})
        n_pages = len(used) + 2
        for (s, p), at in zip(used, torch.randperm(n_pages, generator=g).tolist()):
            t[s, p] = at
        tables = t.cuda()
    else:
        n_pages = 5
    kc, vc = _cache(g, n_pages, page, kv, hd, dt, layout)
    was_k, was_v = kc.clone(), vc.clone()
    width = (heads + 2 * kv) * hd
    qkv = _rand(g, rows, width + pad, dtype=dt).cuda()
    q, k, v = qkv[:, :heads * hd], qkv[:, heads * hd:(heads + kv) * hd], qkv[:, (heads + kv) * hd:width]
    before = qkv.clone()
    freq = _freq(rot) if rot else None
    out = ee.kv_append(k, v, kc, vc, tables, positions, seqs=seqs, q=q if queries else None, inv_freq=freq,
                       interleaved=interleaved, q_out=q if in_place else None)
    if not in_place:
        assert torch.equal(qkv, before)
    f = _freq(rot)

    def check(got, x):
        want, size = _turn64(x.reshape(rows, -1, hd), positions, f, interleaved)
        err = 6 * U32 * size + HALF[dt] * (want.abs() + 6 * U32 * size) * (size > 0)
        off = (got.double().reshape(rows, -1, hd) - want).abs()
        assert (off <= err).all(), float((off - err).max())
    if queries:
        assert (out is q) == in_place
        check(out, before[:, :heads * hd])
    else:
        assert out is None
    # the rows' slots
    ok, slots = [], []
    s_list = seqs.tolist() if seqs is not None else [i // (rows // n_seqs) for i in range(rows)]
    for i, (s, p) in enumerate(zip(s_list, positions.tolist())):
        if 0 <= s < len(tables) and 0 <= p < tables.shape[1] * page and 0 <= int(tables[s, p // page]) < n_pages:
            ok.append(i)
            slots.append((int(tables[s, p // page]), p % page))
    got_k = torch.zeros(rows, kv, hd, dtype=dt, device="cuda")
    kb = before[:, heads * hd:(heads + kv) * hd].reshape(rows, kv, hd)
    vb = before[:, (heads + kv) * hd:width].reshape(rows, kv, hd)
    if ok:
        pg, sl = (torch.tensor(z, device="cuda") for z in zip(*slots))
        got_k[ok] = kc[pg, sl]
        want, size = _turn64(kb, positions, f, interleaved)
        err = 6 * U32 * size + HALF[dt] * (want.abs() + 6 * U32 * size) * (size > 0)
        assert ((got_k.double() - want).abs() <= err)[ok].all()
        assert torch.equal(vc[pg, sl], vb[ok])
        was_k[pg, sl], was_v[pg, sl] = kc[pg, sl], vc[pg, sl]
    # nothing else was written
    assert torch.equal(kc, was_k) and torch.equal(vc, was_v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 2, 7, 70])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_sizes(ee, rows, hd, dtype, interleaved):
    for heads, kv in ((1, 1), (4, 4), (6, 2), (32, 8), (5, 1)):
        _append_case(ee, rows=rows, heads=heads, kv=kv, hd=hd, dtype=dtype, interleaved=interleaved, seed=rows + heads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["slots", "heads", "pairs", "room"])
@pytest.mark.parametrize("page", [16, 48, 64, 256])
def test_append_layouts(ee, layout, page, dtype):
    _append_case(ee, rows=61, heads=6, kv=3, hd=64, dtype=dtype, page=page, layout=layout, pad=16, seed=page)
    _append_case(ee, rows=61, heads=6, kv=3, hd=128, dtype=dtype, page=page, layout=layout, far=300, interleaved=True, queries=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", [0, 16, 32, 64, 96, 128])
def test_append_partial_rotation(ee, rot, dtype):
    for interleaved in (False, True):
        _append_case(ee, rows=9, heads=4, kv=2, hd=128, dtype=dtype, rot=rot, interleaved=interleaved, far=1000)
        _append_case(ee, rows=9, heads=4, kv=2, hd=128, dtype=dtype, rot=rot, interleaved=interleaved, in_place=True)


def test_append_far_positions(ee):
    """Angles of position 10^6 in float32 would be 2^-5 of a radian off."""
    for far in (99_990, 1_000_003, 2 ** 24 + 11):
        _append_case(ee, rows=6, heads=4, kv=4, hd=128, dtype="f32", page=1024, far=far)
        _append_case(ee, rows=6, heads=4, kv=4, hd=128, dtype="bf16", page=1024, far=far, interleaved=True)


def test_append_rows_that_name_no_slot(ee):
    """Padding: sequences, positions and pages that are not there are rotated but not stored."""
    seqs = torch.tensor([0, -1, 3, 2, 1, 1, 2, 2 ** 31 - 1, -2 ** 31, 0, 2], dtype=torch.int32, device="cuda")
    pos = torch.tensor([3, 4, 5, -1, 64, 200, 2, 7, 9, 2 ** 31 - 1, 70], dtype=torch.int32, device="cuda")
    tables = torch.tensor([[0, 1], [5, -1], [2, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")   # five pages
    for dtype, hd in (("bf16", 128), ("f32", 64)):
        _append_case(ee, rows=11, heads=2, kv=2, hd=hd, dtype=dtype, positions=pos, seqs=seqs, tables=tables)
    none = torch.full((4,), -1, dtype=torch.int32, device="cuda")
    _append_case(ee, rows=4, heads=2, kv=1, hd=64, dtype="bf16", positions=none.clone(), seqs=none, tables=tables)


def test_append_consecutive_rows_of_every_sequence(ee):
    pos = torch.tensor([10, 11, 12, 0, 1, 2, 63, 64, 65], dtype=torch.int32, device="cuda")
    tables = torch.tensor([[3, -1], [0, 4], [1, 2]], dtype=torch.int32, device="cuda")
    _append_case(ee, rows=9, heads=4, kv=2, hd=64, dtype="bf16", positions=pos, seqs=None, tables=tables)


def test_append_past_32_bit_offsets(ee):
    pages, page, kv, hd = 2200, 64, 64, 256      # 4.6 GB each of k and v
    kc, vc = (torch.zeros(pages, page, kv, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tables = torch.tensor([[2199, 0], [7, 2150]], dtype=torch.int32, device="cuda")
    g = _gen(0)
    k, v = (_rand(g, 2, kv * hd, dtype=torch.bfloat16).cuda() for _ in range(2))
    pos = torch.tensor([63, 127], dtype=torch.int32, device="cuda")
    ee.kv_append(k, v, kc, vc, tables, pos)
    assert torch.equal(kc[2199, 63], k[0].reshape(kv, hd)) and torch.equal(vc[2150, 63], v[1].reshape(kv, hd))
    assert int(kc.count_nonzero()) == int(k.count_nonzero()) and int(vc.count_nonzero()) == int(v.count_nonzero())


# ---------------------------------------------------------------- attention --

def _attend64(q, kc, vc, tables, lens, rows, heads, window, scale, split):
    """(value, its bound, lse, its bound), from the definition: gather what each row sees."""
    n, most = tables.shape
    page, kv, hd = kc.shape[1:]
    out = torch.zeros(n * rows, heads, hd, dtype=torch.float64, device="cuda")
    err = torch.zeros_like(out)
    lse = torch.full((n * rows, heads), -float("inf"), dtype=torch.float64, device="cuda")
    lerr = torch.zeros_like(lse)
    table = tables.cpu().numpy()
    for s in range(n):
        length = min(max(int(lens[s]), 0), most * page)
        for t in range(rows):
            end = length - rows + 1 + t
            at = np.arange(max(0, end - window) if window else 0, max(end, 0))
            pg = table[s, at // page] if len(at) else at
            keep = (pg >= 0) & (pg < len(kc))
            at, pg = torch.from_numpy(at[keep] % page).cuda(), torch.from_numpy(pg[keep].astype(np.int64)).cuda()
            if not len(at):
                continue
            k, v = kc[pg, at].double(), vc[pg, at].double()          # [m, kv, hd]
            x = q[s * rows + t].double().reshape(kv, heads // kv, hd)
            score = torch.einsum("hgd,mhd->hgm", x, k) * scale
            size = torch.einsum("hgd,mhd->hgm", x.abs(), k.abs()) * abs(scale)
            top = score.amax(-1, keepdim=True)
            d = (hd + 2) * U32 * size + 4 * U32 * (score.abs() + top.abs()) + 2.0 ** -22
            w = torch.exp(score - torch.where(torch.isinf(top) & (top < 0), torch.zeros_like(top), top))
            total = w.sum(-1, keepdim=True)
            p = torch.where(total > 0, w / total, torch.zeros_like(w))
            o = torch.einsum("hgm,mhd->hgd", p, v)
            r = s * rows + t
            out[r] = o.reshape(heads, hd)
            pd = (p * d).sum(-1, keepdim=True)
            e = torch.einsum("hgm,mhd->hgd", p * (d + (len(at) + 8) * U32 + (2.0 ** -16 if split else 0)), v.abs()) + o.abs() * (pd + (len(at) + 8) * U32)
            err[r] = e.reshape(heads, hd)
            lse[r] = (top + torch.log(total))[..., 0].reshape(heads)
            lerr[r] = (pd[..., 0] + (len(at) + 8) * U32).reshape(heads) + 8 * U32 * lse[r].abs().nan_to_num(0, 0, 0)
    return out.reshape(n * rows, -1), err.reshape(n * rows, -1), lse, lerr


def _attend_case(ee, *, lens, heads, kv, hd, dtype="bf16", rows=1, page=64, window=0, layout="slots", out=None, scale=None, most=None,
                 seed=0, pad=0, opad=0, tables=None, poison=True, std=1.0):
    g, dt = _gen(seed), DT[dtype]
    odt = DT[out or dtype]
    if tables is None:
        tables, n_pages = _tables(g, [min(n, most * page) if most else n for n in lens], page, most)
    else:
        n_pages = 9
    kc, vc = _cache(g, n_pages, page, kv, hd, dt, layout)
    n = len(lens)
    if poison:      # what no row may see: slots past a sequence's end, pages of nobody
        free = torch.ones(n_pages, page, dtype=torch.bool)
        for s in range(n):
            for p in range(min(lens[s], tables.shape[1] * page)):
                if 0 <= int(tables[s, p // page]) < n_pages:
                    free[int(tables[s, p // page]), p % page] = False
        kc[free.cuda()], vc[free.cuda()] = float("nan"), float("nan")
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = _rand(g, n * rows, heads * hd + pad, std=std, dtype=dt).cuda()[:, :heads * hd]
    whole = torch.full((n * rows, heads * hd + opad), 7.0, dtype=odt, device="cuda")
    y = whole[:, :heads * hd]
    lse = torch.empty(n * rows, heads, device="cuda")
    got = ee.paged_attention(q, kc, vc, tables, length, window=window, scale=scale, out=y, lse=lse)
    assert got is y
    want, err, wl, lerr = _attend64(q, kc, vc, tables, lens, rows, heads, window, hd ** -0.5 if scale is None else scale, dtype == "bf16")
    err = err + HALF[odt] * (want.abs() + err) + 1e-30
    off = (y.double() - want).abs()
    assert (off <= err).all(), f"{int((~(off <= err)).sum())} of {off.numel()} off, worst {float((off / err).max())} x the bound"
    empty = torch.isinf(wl)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
    assert ((lse.double() - wl).abs()[~empty] <= lerr[~empty]).all()
    assert (whole[:, heads * hd:] == 7.0).all(), "columns past the output were written"
    return dict(q=q, k_cache=kc, v_cache=vc, tables=tables, lens=length, y=y)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_attend_lengths(ee, hd, dtype, out):
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 200, 255, 256, 257, 300, 511, 512, 513, 1000]
    _attend_case(ee, lens=lens, heads=4, kv=2, hd=hd, dtype=dtype, out=out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 2), (3, 1), (8, 2), (15, 5), (16, 1), (17, 1), (40, 1), (32, 8), (64, 4), (33, 3), (7, 7)])
def test_attend_head_groups(ee, heads, kv, dtype):
    _attend_case(ee, lens=[70, 300, 1], heads=heads, kv=kv, hd=64, dtype=dtype, seed=heads)
    _attend_case(ee, lens=[70, 300, 4], heads=heads, kv=kv, hd=128, dtype=dtype, seed=heads, rows=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 48, 80, 128, 1024])
@pytest.mark.parametrize("layout", ["slots", "heads", "pairs", "room"])
def test_attend_pages_and_layouts(ee, layout, page, dtype):
    _attend_case(ee, lens=[1, 47, 48, 49, 333, 700], heads=4, kv=2, hd=128, dtype=dtype, page=page, layout=layout, pad=8, opad=3)
    _attend_case(ee, lens=[5, 260], heads=4, kv=4, hd=64, dtype=dtype, page=page, layout=layout, rows=5, window=40, most=9000 // page)


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 128), ("bf16", 256), ("f32", 256)])
@pytest.mark.parametrize("rows", [2, 3, 4, 5, 9, 16, 33, 65, 100])
def test_attend_blocks_of_rows(ee, rows, dtype, hd):
    for heads, kv in ((4, 1), (3, 3), (10, 2)):
        _attend_case(ee, lens=[rows, 300, 256 + rows, 64, rows - 1, 0, 1], heads=heads, kv=kv, hd=hd, dtype=dtype, rows=rows, seed=rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 255, 256, 257, 600, 5000])
def test_attend_windows(ee, window, dtype):
    _attend_case(ee, lens=[1, 64, 65, 300, 900], heads=4, kv=2, hd=64, dtype=dtype, window=window)
    _attend_case(ee, lens=[1, 64, 65, 300, 900], heads=4, kv=2, hd=128, dtype=dtype, window=window, rows=7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 6])
def test_attend_missing_pages(ee, rows, dtype):
    """Pages outside the pool hold nothing, given back ones of a window or bad ones; lengths past the tables are cut."""
    tables = torch.tensor([[0, -1, 2, 3], [9, 1, 2 ** 31 - 1, 8], [-1, -1, -1, -1], [4, 5, 6, 7], [-2 ** 31, -1, -1, 8]],
                          dtype=torch.int32, device="cuda")
    for hd, page, window in ((64, 64, 0), (128, 64, 0), (128, 96, 100), (64, 16, 0), (256, 64, 20)):
        _attend_case(ee, lens=[4 * page, 3 * page + 5, 200, 10 * page, 4 * page - 1], heads=4, kv=2, hd=hd, dtype=dtype, rows=rows,
                     page=page, window=window, tables=tables)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30])
def test_attend_windows_past_every_position(ee, window):
    """Sequences shorter than the block, whose first rows stand before position 0."""
    for rows in (1, 6, 40):
        a, b = (_attend_case(ee, lens=[3, 1, 100, 0], heads=4, kv=2, hd=64, rows=rows, window=w) for w in (window, 0))
        assert torch.equal(a["y"], b["y"])


def test_attend_negative_lengths_and_empty_batches(ee):
    _attend_case(ee, lens=[-5, -2 ** 31, 0, 3], heads=2, kv=1, hd=64, tables=torch.zeros(4, 1, dtype=torch.int32, device="cuda"))
    kc, vc = _cache(_gen(0), 2, 16, 1, 64, torch.float32)
    none = torch.zeros(0, 3, dtype=torch.int32, device="cuda")
    y = ee.paged_attention(torch.zeros(0, 64, device="cuda"), kc, vc, none, none[:, 0].contiguous())
    assert y.shape == (0, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pages,most", [(0, 0), (0, 5), (3, 0)])
def test_empty_pools_and_tables(ee, pages, most, dtype):
    """Sequences that hold nothing, from memory that there is none of: rows are rotated and not stored, and see nothing."""
    dt = DT[dtype]
    kc, vc = (torch.ones(pages, 16, 2, 64, dtype=dt, device="cuda") for _ in range(2))
    tables = torch.zeros(3, most, dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 17, 100], dtype=torch.int32, device="cuda")
    q, k, v = (_rand(_gen(i), 3, n, dtype=dt).cuda() for i, n in enumerate((256, 128, 128)))
    full = tuple(torch.empty(9, 16, 2, 64, dtype=dt, device="cuda") for _ in range(2))
    want = ee.kv_append(k, v, *full, torch.arange(24, dtype=torch.int32, device="cuda").reshape(3, 8), pos, q=q, inv_freq=_freq(64))
    assert torch.equal(ee.kv_append(k, v, kc, vc, tables, pos, q=q, inv_freq=_freq(64)), want)
    assert (kc == 1).all() and (vc == 1).all()
    for rows in (1, 3):
        for window in (0, 9):
            lens, lse = pos[:3 // rows].contiguous(), torch.empty(3, 4, device="cuda")
            y = ee.paged_attention(q, kc, vc, tables[:3 // rows], lens, window=window, lse=lse)
            assert (y == 0).all() and (lse == -float("inf")).all()


def test_attend_no_rows(ee):
    kc, vc = _cache(_gen(0), 2, 16, 1, 64, torch.bfloat16)
    for n in (0, 1, 3):
        tables = torch.zeros(n, 3, dtype=torch.int32, device="cuda")
        q = torch.zeros(0, 128, dtype=torch.bfloat16, device="cuda")
        assert ee.paged_attention(q, kc, vc, tables, tables[:, 0].contiguous()).shape == (0, 128)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_sharp_and_flat_scores(ee, dtype):
    _attend_case(ee, lens=[1000, 700], heads=4, kv=2, hd=128, dtype=dtype, std=30.0)
    _attend_case(ee, lens=[1000, 700], heads=4, kv=2, hd=128, dtype=dtype, std=0.0, rows=3)
    _attend_case(ee, lens=[1000, 700], heads=4, kv=2, hd=64, dtype=dtype, scale=-0.3)
    _attend_case(ee, lens=[1000, 700], heads=4, kv=2, hd=64, dtype=dtype, scale=0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_infinities(ee, dtype):
    """Scores of -inf count nothing; a row with no other is zeros; NaN and +inf reach who sees them."""
    g, dt = _gen(7), DT[dtype]
    kc, vc = _cache(g, 8, 64, 1, 64, dt)
    tables = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([500], dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 128, dtype=dt, device="cuda")
    q[0, 0], q[0, 64] = 1.0, -1.0       # scores: +- the keys' first dimension
    kc[..., 1:] = 0
    kc[..., 0] = -float("inf")
    kc[2, 5], vc[2, 5] = 0.0, 3.0       # one position that both see
    lse = torch.empty(1, 2, device="cuda")
    y = ee.paged_attention(q[:, :64].contiguous(), kc, vc, tables, lens, lse=lse[:, :1].contiguous())
    assert (y == 3.0).all()
    y = ee.paged_attention(q, kc, vc, tables, lens, lse=lse)
    assert (y[0, :64] == 3.0).all() and torch.isnan(y[0, 64:]).all()
    kc[2, 5] = 0
    kc[2, 5, 0, 0] = -float("inf")
    one = torch.empty(1, 1, device="cuda")
    y = ee.paged_attention(q[:, :64].contiguous(), kc, vc, tables, lens, lse=one)
    assert (y == 0).all() and one.item() == -float("inf")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("rows,lens,most", [
    (1, [700, 90, 300], None),           # chunks to workgroups
    (1, [700, 90, 1300], 300_000),       # runs to waves
    (1, [2100, 700] + [600] * 70, 2112),  # chunks to waves
    (7, [700, 90, 300], None),
    (40, [700, 90, 300], None),
])
def test_attend_infinite_values(ee, rows, lens, most, hd, dtype):
    """An infinite value that a row sees is the infinity of its sign in the row's result, values of both
    signs are NaN; who does not see it, and the other dimensions, keep their bits."""
    kv = 2
    s = _attend_case(ee, lens=lens, heads=3 * kv, kv=kv, hd=hd, dtype=dtype, rows=rows, most=most // 64 if most else None, seed=hd)
    clean = s["y"].reshape(len(lens), rows, kv, 3, hd)
    want = clean.clone()
    inf = float("inf")
    for b, head, dim, at, value in ((0, 0, 5, (lens[0] - 3,), inf), (0, 1, hd - 1, (0,), -inf), (0, 1, 17, (130, 131, 400), inf),
                                    (1, 0, 0, (2, 70), -inf), (1, 1, 33, tuple(range(64)), inf)):
        for p in at:
            s["v_cache"][int(s["tables"][b, p // 64]), p % 64, head, dim] = value
        for t in range(rows):
            if lens[b] - rows + t >= at[0]:
                want[b, t, head, :, dim] = value
    for p, value in ((10, inf), (250, -inf)):       # of both signs
        s["v_cache"][int(s["tables"][2, p // 64]), p % 64, 0, 9] = value
    want[2, :, 0, :, 9] = float("nan")
    got = ee.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["tables"], s["lens"]).reshape(want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(7.0, inf, -inf), want.nan_to_num(7.0, inf, -inf))


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 3000])
def test_attend_an_infinite_value_of_each_chunk(ee, hd, window):
    """One head has it in its first chunk, the next one in its second and so on, where waves take ten chunks in turn."""
    kv, length = 32, 5000
    s = _attend_case(ee, lens=[length] + [3] * 63, heads=kv, kv=kv, hd=hd, window=window, most=80, seed=hd)
    want, inf = s["y"].reshape(64, kv, hd).clone(), float("inf")
    for h in range(kv):
        for p in (h % 20 * 256 + 17, h % 20 * 256 + 130):
            if p < length:
                s["v_cache"][int(s["tables"][0, p // 64]), p % 64, h, 5] = inf
                if not window or p >= length - window:
                    want[0, h, 5] = inf
    got = ee.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["tables"], s["lens"], window=window).reshape(want.shape)
    assert torch.isinf(want).any() and torch.equal(got, want)


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64), ("bf16", 256)])
@pytest.mark.parametrize("window", [0, 50])
def test_attend_a_block_equals_its_rows(ee, dtype, hd, window):
    """Bit for bit, though later positions (and, with a window, older ones) hold NaN and infinities when the row is alone in seeing the others."""
    rows = 37
    for heads, kv in ((4, 1), (2, 2), (9, 3)):
        s = _attend_case(ee, lens=[330, 37, 290, 600], heads=heads, kv=kv, hd=hd, dtype=dtype, rows=rows, window=window, seed=heads)
        for t in (0, 1, 5, 15, 16, 31, 36):
            q = s["q"].reshape(4, rows, -1)[:, t].contiguous()
            one = ee.paged_attention(q, s["k_cache"], s["v_cache"], s["tables"], s["lens"] - rows + 1 + t, window=window)
            assert torch.equal(one, s["y"].reshape(4, rows, -1)[:, t]), (heads, t)
        # a position that only the rows from t on see: the others' bits stay
        t = 21
        for b in range(4):
            p = int(s["lens"][b]) - rows + t
            page, at = int(s["tables"][b, p // 64]), p % 64
            s["v_cache"][page, at], s["k_cache"][page, at] = float("nan"), float("inf")
        again = ee.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["tables"], s["lens"], window=window).reshape(4, rows, -1)
        assert torch.equal(again[:, :t], s["y"].reshape(4, rows, -1)[:, :t])
        assert torch.isnan(again[:, t:]).any(-1).all()


def test_attend_does_not_depend_on_the_batch(ee):
    """Nor on the tables' width."""
    s = _attend_case(ee, lens=[1000, 40, 2100, 700, 1], heads=8, kv=2, hd=128)
    for b in range(5):
        one = ee.paged_attention(s["q"][b:b + 1], s["k_cache"], s["v_cache"], s["tables"][b:b + 1], s["lens"][b:b + 1])
        assert torch.equal(one, s["y"][b:b + 1])
    wide = torch.full((5, 3000), -1, dtype=torch.int32, device="cuda")
    wide[:, :s["tables"].shape[1]] = s["tables"]
    assert torch.equal(ee.paged_attention(s["q"], s["k_cache"], s["v_cache"], wide, s["lens"]), s["y"])
    assert torch.equal(ee.paged_attention(s["q"], s["k_cache"], s["v_cache"], wide[:, :50], s["lens"]), s["y"])
    many = [t.repeat(70, *[1] * (t.dim() - 1)) for t in (s["q"], s["tables"], s["lens"])]
    got = ee.paged_attention(many[0], s["k_cache"], s["v_cache"], many[1].contiguous(), many[2])
    assert torch.equal(got, s["y"].repeat(70, 1))


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 256)])
@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("lens,kv,capacity", [
    ([0, 1, 64, 65, 256, 257, 5000], 2, 300_000),                      # short ones in wide tables: shared out by runs
    ([1024, 700, 256, 257, 255, 0, 1] + [30] * 33, 8, 1024),           # some by runs, some by chunks
    ([2048, 1700, 900, 300, 513, 0, 1, 256] + [5] * 56, 32, 2048),     # several chunks in turn
    ([1300, 40], 3, 270_000),
])
def test_attend_shared_out_over_waves(ee, dtype, hd, window, lens, kv, capacity):
    """Against float64, and bit for bit as alone with tables no wider than the sequence."""
    s = _attend_case(ee, lens=lens, heads=2 * kv, kv=kv, hd=hd, dtype=dtype, window=window, most=capacity // 64, seed=kv)

    def alone(tables, y):
        for b in range(min(len(lens), 8)):
            pages = max(1, -(-lens[b] // 64))
            one = ee.paged_attention(s["q"][b:b + 1], s["k_cache"], s["v_cache"], tables[b:b + 1, :pages].contiguous(), s["lens"][b:b + 1],
                                     window=window)
            got = y[b:b + 1]
            assert torch.equal(torch.isnan(one), torch.isnan(got)) and torch.equal(one[~torch.isnan(one)], got[~torch.isnan(got)]), b
    alone(s["tables"], s["y"])
    gone = s["tables"].clone()      # pages that are not there, and values of no number that all see
    gone[:, 1::3] = -1
    gone[-1, 0] = -1
    s["v_cache"][int(s["tables"][0, 0]) if lens[0] else 0, 40] = float("inf")
    alone(gone, ee.paged_attention(s["q"], s["k_cache"], s["v_cache"], gone, s["lens"], window=window))


@pytest.mark.parametrize("heads,kv", [(20, 1), (33, 3)])
def test_attend_many_heads_shared_out_over_waves(ee, heads, kv):
    """More queries of a KV head than a tile has columns."""
    _attend_case(ee, lens=[300, 1100, 0, 5], heads=heads, kv=kv, hd=128, most=300_000 // 64)
    _attend_case(ee, lens=[300, 1100, 0, 5] + [3] * 300, heads=heads, kv=kv, hd=64, most=1100 // 16, page=16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_long(ee, dtype):
    _attend_case(ee, lens=[70001, 3], heads=2, kv=1, hd=64, dtype=dtype, page=128, poison=False)
    _attend_case(ee, lens=[40000], heads=4, kv=2, hd=128, dtype=dtype, page=64, poison=False, window=9000)


def test_attend_more_rows_than_a_launch_of_workgroups(ee):
    """1.1 million rows and heads, whose states of 33 chunks take 9.8 GB."""
    seqs, rows, heads, page = 17, 1024, 64, 64
    lens = [1024 + 64 * i for i in range(seqs)]
    g = _gen(0)
    tables, n_pages = _tables(g, lens, page)
    kc, vc = _cache(g, n_pages, page, 1, 64, torch.bfloat16)
    q = _rand(g, 1024, heads * 64, dtype=torch.bfloat16).cuda().repeat(seqs, 1)
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    wide = torch.full((seqs, 132 + 1), -1, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = tables
    y = ee.paged_attention(q, kc, vc, wide, length)
    for b in (0, 8, 16):
        one = ee.paged_attention(q[:rows], kc, vc, tables[b:b + 1].contiguous(), length[b:b + 1])
        assert torch.equal(y[b * rows:(b + 1) * rows], one), b


def test_attend_past_32_bit_offsets(ee):
    pages, page, kv, hd = 2200, 64, 64, 256      # 4.6 GB each of k and v
    kc, vc = (torch.zeros(pages, page, kv, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = _gen(0)
    for p in (2199, 2150, 3):
        kc[p], vc[p] = (_rand(g, page, kv, hd, dtype=torch.bfloat16).cuda() for _ in range(2))
    q = _rand(g, 1, kv * hd, dtype=torch.bfloat16).cuda()
    lens = torch.tensor([180], dtype=torch.int32, device="cuda")
    far = ee.paged_attention(q, kc, vc, torch.tensor([[2199, 2150, 3]], dtype=torch.int32, device="cuda"), lens)
    near = ee.paged_attention(q, kc[[2199, 2150, 3]], vc[[2199, 2150, 3]], torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda"), lens)
    assert torch.equal(far, near)


def test_attend_workspaces(ee):
    s = _attend_case(ee, lens=[1000, 40, 600], heads=8, kv=2, hd=128)
    n = ee.ee_paged_attention_workspace_bytes(3, 1, 8, 2, 128, 64, s["tables"].shape[1], 0)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    args = (s["q"], s["k_cache"], s["v_cache"], s["tables"], s["lens"])
    for _ in range(2):
        assert torch.equal(ee.paged_attention(*args, workspace=ws), s["y"])
    with pytest.raises(ee.EEError) as e:
        ee.paged_attention(*args, workspace=ws[:n - 1])
    assert e.value.code == ee.EE_ECAPACITY


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,rows,heads,page,positions,window", [
    ([0, 1, 33, 300, 2, 700, 40, 257, 20, 1000, 32, 0, 64, 90, 34, 5, 600, 31, 256, 1500], 33, 8, 64, 1 << 20, 0),   # parts of 7 sequences
    ([700, 350, 0], 600, 8, 64, 1 << 20, 0),            # parts of 200 rows, those of the second before its first position
    ([70_000, 1, 2], 2, 64, 65536, 1 << 25, 0),         # of one row: a row's states are more than 2 GiB
    ([400_000, 50], 600, 8, 1024, 1 << 20, 300_000),    # of one sequence, which a window decides
])
def test_attend_in_parts(ee, lens, rows, heads, page, positions, window, dtype):
    """Calls whose tables are so wide that their states would not fit: bit for bit as alone with tables
    no wider than the sequence, in a workspace of the size that is asked for and no further."""
    g, dt, kv = _gen(rows), DT[dtype], 1
    tables, n_pages = _tables(g, lens, page)
    kc, vc = _cache(g, n_pages, page, kv, 64, dt)
    wide = torch.full((len(lens), positions // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = tables
    q = _rand(g, len(lens) * rows, heads * 64, dtype=dt).cuda()
    n = ee.ee_paged_attention_workspace_bytes(len(lens), rows, heads, kv, 64, page, positions // page, window)
    ws = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
    length, lse = _i32(lens), torch.full((len(lens) * rows, heads), 7.0, device="cuda")
    y = ee.paged_attention(q, kc, vc, wide, length, window=window, lse=lse, workspace=ws[:n], out=torch.full_like(q, 7.0))
    assert (ws[n:] == 77).all()
    for b in range(len(lens)):
        at = slice(b * rows, (b + 1) * rows)
        pages = max(1, -(-lens[b] // page))
        ends = torch.empty(rows, heads, device="cuda")
        one = ee.paged_attention(q[at], kc, vc, tables[b:b + 1, :pages].contiguous(), length[b:b + 1], window=window, lse=ends)
        assert torch.equal(y[at], one) and torch.equal(lse[at], ends), b


def test_two_streams(ee):
    a = _attend_case(ee, lens=[3000, 40], heads=8, kv=2, hd=128, seed=1)
    b = _attend_case(ee, lens=[1500, 2500], heads=8, kv=2, hd=128, seed=2)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(ee.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["tables"], s["lens"]))
    torch.cuda.synchronize()
    assert all(torch.equal(y, a["y"]) for y in got[0]) and all(torch.equal(y, b["y"]) for y in got[1])


# ------------------------------------------------------------------ together --

class _Layer:
    """The attention half of a layer, of the library's operators: 8-bit projections around the paged cache."""

    def __init__(self, ee, seed, d=256, heads=8, kv=2, hd=64, page=16, seqs=3, capacity=128):
        g = _gen(seed)
        self.ee, self.d, self.heads, self.kv, self.hd, self.page, self.seqs = ee, d, heads, kv, hd, page, seqs
        self.wqkv = ee.fp8_quant(_rand(g, (heads + 2 * kv) * hd, d, std=d ** -0.5).cuda(), block_rows=128)
        self.wo = ee.fp8_quant(_rand(g, d, heads * hd, std=(heads * hd) ** -0.5).cuda(), block_rows=128)
        per = capacity // page
        self.tables = torch.randperm(seqs * per, generator=g).to(torch.int32).reshape(seqs, per).cuda()
        self.k, self.v = _cache(g, seqs * per, page, kv, hd, torch.bfloat16, "heads", fill=float("nan"))
        self.freq = _freq(hd)

    def step(self, h, seqs, positions, lens, tables=None):
        ee, hd, qd, kd = self.ee, self.hd, self.heads * self.hd, self.kv * self.hd
        tables = self.tables if tables is None else tables
        qkv = ee.fp8_linear(*ee.fp8_quant(h), *self.wqkv)
        q = ee.kv_append(qkv[:, qd:qd + kd], qkv[:, qd + kd:], self.k, self.v, tables, positions, seqs=seqs, q=qkv[:, :qd],
                         inv_freq=self.freq)
        o = ee.paged_attention(q, self.k, self.v, tables, lens)
        return ee.fp8_linear(*ee.fp8_quant(o), *self.wo, residual=h)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _deq(codes, scales, block_rows):
    r, c = codes.shape
    s = scales.double().repeat_interleave(block_rows, 0)[:r].repeat_interleave(128, 1)[:, :c]
    return codes.float().double() * s


def test_decoding_with_all_operators(ee):
    """Prompts of three sequences, then single tokens, against the same layer in
    float64 on the operators' quantised weights: the difference is what rounding activations to
    e4m3 and bf16 leaves (half a step each: 2^-4 and 2^-8 of values; averaged over the
    products, a few hundredths of a result's typical size)."""
    L = _Layer(ee, 3)
    g = _gen(4)
    wqkv, wo = _deq(*L.wqkv, 128), _deq(*L.wo, 128)
    past = [[] for _ in range(3)]       # rows of h of every sequence
    lens = [0, 0, 0]

    def reference(s, h_all):
        qkv = torch.mm(_deq(*ee.fp8_quant(h_all.bfloat16()), 1), wqkv.T.contiguous())
        pos = torch.arange(len(h_all), device="cuda")
        q, _ = _turn64(qkv[:, :512].reshape(-1, 8, 64), pos, L.freq, False)
        k, _ = _turn64(qkv[:, 512:640].reshape(-1, 2, 64), pos, L.freq, False)
        v = qkv[:, 640:].reshape(-1, 2, 64)
        score = torch.einsum("tgd,mgd->gtm", q, k.repeat_interleave(4, 1)) / 8.0
        score = score.masked_fill(torch.ones_like(score[0]).triu(1).bool(), -float("inf"))
        o = torch.einsum("gtm,mgd->tgd", torch.softmax(score, -1), v.repeat_interleave(4, 1)).reshape(-1, 512)
        return h_all.double() + torch.mm(o, wo.T.contiguous())

    for rows in (20, 1, 1, 7, 1):
        h = _rand(g, 3 * rows, 256, dtype=torch.bfloat16).cuda()
        seqs, pos = [], []
        for s in range(3):
            past[s].append(h[s * rows:(s + 1) * rows])
            pos += range(lens[s], lens[s] + rows)
            seqs += [s] * rows
            lens[s] += rows
        y = L.step(h, _i32(seqs), _i32(pos), _i32(lens))
        for s in range(3):
            want = reference(s, torch.cat(past[s]))[-rows:]
            off = (y[s * rows:(s + 1) * rows].double() - want)
            assert float(off.pow(2).mean().sqrt()) < 0.05 * float((want - past[s][-1].double()).pow(2).mean().sqrt())


def test_a_verified_block_equals_single_steps(ee):
    """Bit for bit through all the operators, after a rollback that overwrites rejected positions."""
    L = _Layer(ee, 5, seqs=1)
    g = _gen(6)
    prompt, draft = _rand(g, 50, 256, dtype=torch.bfloat16).cuda(), _rand(g, 9, 256, dtype=torch.bfloat16).cuda()
    L.step(prompt, _i32([0] * 50), _i32(range(50)), _i32([50]))
    block = L.step(draft, _i32([0] * 9), _i32(range(50, 59)), _i32([59]))
    for t in range(9):
        one = L.step(draft[t:t + 1], _i32([0]), _i32([50 + t]), _i32([51 + t]))
        assert torch.equal(one, block[t:t + 1]), t


def test_steps_replayed_from_a_graph(ee):
    """A decoding step captured once, replayed with new tokens, positions and lengths,
    eager work between the replays; a second graph shares nothing with it."""
    L, M = _Layer(ee, 7), _Layer(ee, 7)
    M.k.copy_(L.k)
    M.v.copy_(L.v)
    g = _gen(8)
    prompt = _rand(g, 3 * 30, 256, dtype=torch.bfloat16).cuda()
    seqs, pos = _i32([0] * 30 + [1] * 30 + [2] * 30), _i32(list(range(30)) * 3)
    for x in (L, M):
        x.step(prompt, seqs, pos, _i32([30, 30, 30]))
    h, at, lens, sq = torch.zeros(3, 256, dtype=torch.bfloat16, device="cuda"), _i32([127] * 3), _i32([1] * 3), _i32([-1, -1, -1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.step(h, sq, at, lens)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = L.step(h, sq, at, lens)
        graphs.append((graph, y))
    sq.copy_(_i32([0, 1, 2]))
    for i in range(6):
        token = _rand(_gen(30 + i), 3, 256, dtype=torch.bfloat16).cuda()
        h.copy_(token)
        at.fill_(30 + i)
        lens.fill_(31 + i)
        graph, y = graphs[i % 2]
        graph.replay()
        torch.cuda.synchronize()
        want = M.step(token, _i32([0, 1, 2]), _i32([30 + i] * 3), _i32([31 + i] * 3))
        assert torch.equal(y, want), i
        assert torch.equal(L.k.nan_to_num(7.0), M.k.nan_to_num(7.0)) and torch.equal(L.v.nan_to_num(7.0), M.v.nan_to_num(7.0))


def test_python_refusals(ee):
    g = _gen(9)
    kc, vc = _cache(g, 6, 16, 2, 64, torch.bfloat16)
    q, k, v = (_rand(g, 2, n, dtype=torch.bfloat16).cuda() for n in (256, 128, 128))
    t, lens, pos = _i32([[0, 1], [2, 3]]), _i32([3, 20]), _i32([2, 19])
    A = lambda **kw: ee.paged_attention(**{**dict(q=q, k_cache=kc, v_cache=vc, tables=t, lens=lens), **kw})  # noqa: E731
    P = lambda **kw: ee.kv_append(**{**dict(k=k, v=v, k_cache=kc, v_cache=vc, tables=t, positions=pos, q=q, inv_freq=_freq(64)), **kw})  # noqa: E731
    A(), P()
    for kw in (dict(q=q.float()), dict(q=q[:, :200]), dict(q=q[:1]), dict(lens=lens.long()), dict(lens=lens[:1]), dict(tables=t.long()),
               dict(tables=t.t()), dict(k_cache=kc.float()), dict(v_cache=vc[:, :, :1]), dict(k_cache=kc[..., :32], v_cache=vc[..., :32]),
               dict(window=-1), dict(window=2 ** 40), dict(scale=float("nan")), dict(out=q.float()[:, :100]), dict(lse=torch.empty(2, 2, device="cuda")),
               dict(workspace=torch.empty(10, device="cuda")), dict(k_cache=kc.transpose(2, 3), v_cache=vc.transpose(2, 3)), dict(out=q),
               dict(k_cache=kc.cpu()), dict(q=q.clone().requires_grad_(True)), dict(k_cache=kc.clone().requires_grad_(True)),
               dict(k_cache=kc[:, :8], v_cache=vc[:, :8])):
        with pytest.raises(ee.EEError) as e:
            A(**kw)
        assert e.value.code == ee.EE_EINVAL, kw
    for kw in (dict(k=k.float()), dict(k=k[:, :64]), dict(v=v[:1]), dict(q=q[:, :100]), dict(positions=pos.long()), dict(positions=pos[:1]),
               dict(seqs=lens.long()), dict(inv_freq=_freq(64).float()), dict(inv_freq=_freq(16)[:3]), dict(inv_freq=_freq(256)),
               dict(q=None, q_out=q), dict(q_out=q[:, :128]), dict(k_cache=vc), dict(k_cache=kc[:1].expand(6, -1, -1, -1)), dict(k=k.clone().requires_grad_(True)),
               dict(tables=_i32([[0, 1], [2, 3], [4, 5]]))):
        with pytest.raises(ee.EEError) as e:
            P(**kw)
        assert e.value.code == ee.EE_EINVAL, kw
