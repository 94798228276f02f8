"""The MXFP4 operators on the GPU against the plain 64-bit form (tests/mx4_plain.py), and models whose projections are kept in MXFP4
against the oracle holding the numbers that they then stand for."""
import dataclasses

import numpy as np
import pytest
import torch

import synthetic_inputs as si
from tests import helpers as hp
from tests import mx4_plain as plain

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def P():
    import paper_2410_06916_amd as P
    return P


def _randn(seed, *shape, scale=1.0, dtype=FP):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def _weight(seed, rows, depth, dtype=BF):
    """Weights of sizes that differ from row to row, with a block of zeros in every ninth row."""
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(rows, depth, generator=g) * 0.05 * torch.exp(torch.randn(rows, 1, generator=g))
    w[::9, :32] = 0.0
    return w.to(dtype).cuda()


def _apart(t, pad, lead=0):
    """t's values in rows that lie `pad` elements further apart, the first `lead` elements into their memory."""
    big = torch.full((t.shape[0], t.shape[1] + pad + lead), 777.0, dtype=t.dtype, device=t.device)
    v = big[:, lead:lead + t.shape[1]]
    v.copy_(t)
    return v


def _close(got, want, bound, what):
    err = (got.detach().cpu().double() - want).abs()
    assert got.shape == want.shape and bool((err <= bound).all()), (what, float((err / bound).max()), int((err > bound).sum()))


# ------------------------------------------------------------------------------------------
# quantising and reading back
# ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,depth", [(1, 1), (1, 31), (3, 32), (16, 128), (17, 33), (15, 127), (40, 129), (100, 777), (33, 4104)])
@pytest.mark.parametrize("dtype", [FP, BF], ids=["fp32", "bf16"])
def test_quantised_values_are_the_formats(P, rows, depth, dtype):
    """Every value equals the definition's in 64 bits, whatever the row length, the distance of the rows and their alignment, in both types
    and out of both types; reading back and quantising again changes nothing."""
    w = _weight(rows + depth, rows, depth, dtype)
    want = plain.values(w)
    for src in (w, _apart(w, 7), _apart(w, 8), _apart(w, 3, lead=1)):
        packed = P.mx4_quantize(src)
        for out in (FP, BF):
            got = P.mx4_dequantize(packed, out)
            assert got.dtype == out and torch.equal(got.cpu().double(), want), (rows, depth, out)
    wide = torch.full((rows, depth + 9), 5.0, dtype=dtype, device="cuda")
    got = P.mx4_dequantize(packed, dtype, out=wide[:, 4:4 + depth])
    assert torch.equal(got.cpu().double(), want) and bool((wide[:, :4] == 5).all()) and bool((wide[:, 4 + depth:] == 5).all())
    again = P.mx4_quantize(P.mx4_dequantize(packed, dtype))
    assert torch.equal(P.mx4_dequantize(again).cpu().double(), want)


@pytest.mark.parametrize("rows,depth", [(1, 1), (8, 128), (7, 33), (9, 200), (172, 264)])
def test_gate_and_up_are_packed_side_by_side(P, rows, depth):
    gate, up = _weight(1, rows, depth), _apart(_weight(2, rows, depth), 5)
    packed = P.mx4_quantize_gated(gate, up)
    assert torch.equal(P.mx4_dequantize(packed).cpu().double(), torch.cat([plain.values(gate), plain.values(up)]))


def test_every_element_scale_and_tie(P):
    """All magnitudes a block can hold on a grid finer than the format's, one ulp to either side of each, at the scales of both ends of the
    range: the smallest (subnormal weights), around 1, the largest finite."""
    base = np.arange(0, 4096, dtype=np.float64) / 512.0              # 0 .. 8 in steps of 2^-9: every tie among them
    for e in (-127, -126, -125, -100, -1, 0, 7, 100, 124):
        with np.errstate(over="ignore", under="ignore"):
            mid = np.ldexp(base, e).astype(np.float32)
        for v in (mid, np.nextafter(mid, np.float32(np.inf), dtype=np.float32), np.nextafter(mid, np.float32(0), dtype=np.float32)):
            v = np.where(np.arange(v.size) % 3 == 0, -v, v)
            blocks = np.zeros((v.size // 31 + 1, 32), np.float32)
            blocks[:, 1:].flat[:v.size] = v
            # the block's first element sets its scale: the largest below 8 x 2^e
            blocks[:, 0] = np.nextafter(np.float32(np.ldexp(1.0, min(e + 3, 127)) if e < 125 else np.finfo(np.float32).max), np.float32(0))
            w = torch.from_numpy(blocks).cuda()
            assert torch.equal(P.mx4_dequantize(P.mx4_quantize(w)).cpu().double(), plain.values(w)), e


def test_blocks_that_hold_an_infinity_or_a_nan(P):
    w = _weight(3, 20, 100, FP)
    w[2, 5], w[3, 40], w[4, 99], w[7, 70] = float("inf"), float("-inf"), float("nan"), float("nan")
    for t in (w, w.to(BF)):
        got, want = P.mx4_dequantize(P.mx4_quantize(t)).cpu().double(), plain.values(t)
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(1.0), want.nan_to_num(1.0))
        assert int(got.isnan().sum()) == 32 + 32 + 4 + 32


# ------------------------------------------------------------------------------------------
# products
# ------------------------------------------------------------------------------------------
# rows of x around every change of kernel, widths and depths off every tile
_LINEAR = [(1, 1, 1), (1, 16, 128), (1, 17, 4104), (2, 100, 777), (3, 256, 256), (5, 40, 32), (5, 1001, 520), (6, 48, 1000), (8, 33, 31), (9, 4096, 1376),
           (10, 64, 4096), (11, 130, 700), (16, 513, 96), (17, 100, 2049), (21, 40, 640), (31, 272, 1160), (32, 96, 11008), (33, 96, 160), (42, 50, 130),
           (43, 50, 130), (48, 80, 384), (63, 70, 333), (64, 128, 512), (65, 128, 512), (100, 300, 264), (127, 17, 1000), (128, 256, 4096), (129, 31, 640),
           (200, 1000, 136), (255, 257, 300), (300, 640, 1024), (513, 384, 392), (1030, 96, 72)]


@pytest.mark.parametrize("n,rows,depth", _LINEAR)
@pytest.mark.parametrize("x_dtype", [FP, BF], ids=["x32", "x16"])
def test_linear_against_64_bits(P, n, rows, depth, x_dtype):
    w = _weight(n + rows, rows, depth)
    x = _randn(depth, n, depth, dtype=x_dtype)
    x[:, depth // 2] *= 30.0
    packed, vals = P.mx4_quantize(w), plain.values(w)
    r = _randn(5, n, rows, scale=2.0)
    want, size = plain.linear(x, vals)
    for out in (FP, BF):
        bound = plain.linear_bound(want, size, depth, 3 if x_dtype == FP else 1, out)
        _close(P.mx4_linear(x, packed, out_dtype=out), want, bound, (n, rows, depth, out))
    with_r, _ = plain.linear(x, vals, r.to(BF))
    bound = plain.linear_bound(with_r, size, depth, 3 if x_dtype == FP else 1, BF)
    _close(P.mx4_linear(x, packed, residual=r.to(BF), out_dtype=BF), with_r, bound, "residual")
    # rows apart and off 16 bytes, into rows apart, onto the residual itself
    y = _apart(r, 5, lead=3)
    got = P.mx4_linear(_apart(x, 3, lead=1), packed, residual=y, out=y)
    with_r, _ = plain.linear(x, vals, r)
    assert got.data_ptr() == y.data_ptr()
    _close(got, with_r, plain.linear_bound(with_r, size, depth, 3 if x_dtype == FP else 1, FP), "in place")
    whole = y._base if y._base is not None else y
    assert bool((whole[:, :3] == 777).all()) and bool((whole[:, 3 + rows:] == 777).all())


# rows of weights on either side of one, two, three and six row groups a compute unit (256 of them), depths on either side of what a
# wavefront's window holds (an eighth of 4, 8 and 12 super-tiles), and the column counts that go with them
@pytest.mark.parametrize("rows", [4096, 4112, 8208, 12304, 24600])
@pytest.mark.parametrize("depth", [520, 4104, 4736, 8456, 12680])
def test_few_rows_against_wide_and_deep_matrices(P, rows, depth):
    g = torch.Generator(device="cuda").manual_seed(rows + depth)
    w = (torch.randn(rows, depth, device="cuda", generator=g) * 0.05).to(BF)
    packed = P.mx4_quantize(w)
    vals = P.mx4_dequantize(packed).double()   # (tested against the definition above)
    some = torch.randint(0, rows, (7,), generator=torch.Generator().manual_seed(1)).cuda()
    assert torch.equal(vals[some].cpu(), plain.values(w[some]))
    for n, dt in ((1, BF), (1, FP), (3, FP), (5, FP), (9, BF), (9, FP), (16, BF), (13, FP), (20, FP), (40, BF), (30, FP), (90, BF)):
        x = torch.randn(n, depth, device="cuda", generator=g).to(dt)
        want, size = x.double() @ vals.t(), x.double().abs() @ vals.abs().t()
        got = P.mx4_linear(x, packed, out_dtype=FP)
        bound = plain.linear_bound(want, size, depth, 3 if dt == FP else 1, FP)
        err = (got.double() - want).abs()
        assert bool((err <= bound).all()), (n, dt, float((err / bound).max()))


# as many weight rows as make workgroups that share their columns worth while (5, 9, 11 and 14 row groups a compute unit), with depths on
# either side of what such a workgroup has in flight, of eight slices, and of 32 super-tiles
@pytest.mark.parametrize("rows,depth", [(18011, 40), (18011, 264), (18011, 1000), (18011, 2200), (33000, 40), (33000, 264), (33000, 1000), (33000, 2200),
                                        (45008, 40), (45008, 264), (45008, 1000), (45008, 2200), (53300, 4136)])
def test_many_columns_against_wide_matrices(P, rows, depth):
    g = torch.Generator(device="cuda").manual_seed(rows + depth)
    w = (torch.randn(rows, depth, device="cuda", generator=g) * 0.05).to(BF)
    packed = P.mx4_quantize(w)
    gated = P.mx4_quantize_gated(w[:rows // 2], w[rows // 2:2 * (rows // 2)])
    vals = P.mx4_dequantize(packed).double()   # (tested against the definition above)
    x96 = torch.randn(96, depth, device="cuda", generator=g)
    r96 = torch.randn(96, rows, device="cuda", generator=g)
    for dt, counts in ((BF, (96, 81, 65, 64, 50, 33, 32, 17)), (FP, (32, 27, 22, 21, 12, 11, 10, 6))):
        terms = 3 if dt == FP else 1
        for n in counts:
            x = x96[:n].to(dt)
            want, size = x.double() @ vals.t(), x.double().abs() @ vals.abs().t()
            got = P.mx4_linear(x, packed, residual=r96[:n], out_dtype=FP)
            with_r = want + r96[:n].double()
            assert bool(((got.double() - with_r).abs() <= plain.linear_bound(with_r, size, depth, terms, FP)).all()), (n, dt)
            half = rows // 2
            a, b, sa, sb = want[:, :half], want[:, half:2 * half], size[:, :half], size[:, half:2 * half]
            ref = (a / (1 + torch.exp(-a)) * b, a, b, sa, sb)
            got_h = P.mx4_swiglu(x, gated, out_dtype=BF)
            assert bool(((got_h.double() - ref[0]).abs() <= plain.swiglu_bound(*ref, depth, terms, BF)).all()), (n, dt)
            if n == counts[0]:
                full, full_h = got, got_h
            assert torch.equal(got, full[:n]) and torch.equal(got_h, full_h[:n]), (n, dt)
        one = P.mx4_linear(x96[:1].to(dt), packed, residual=r96[:1], out_dtype=FP)
        assert torch.equal(one, full[:1]) and torch.equal(P.mx4_swiglu(x96[:1].to(dt), gated, out_dtype=BF), full_h[:1])


# more than 64 super-tiles: slices of the depth in workgroups of their own, some of them short or empty; up to 768 row groups, and one more
@pytest.mark.parametrize("rows,depth", [(1, 8200), (40, 8200), (300, 9300), (4096, 11008), (2050, 16500), (12288, 8328), (12289, 8328)])
def test_many_columns_against_deep_matrices(P, rows, depth):
    g = torch.Generator(device="cuda").manual_seed(rows + depth)
    w = (torch.randn(rows, depth, device="cuda", generator=g) * 0.05).to(BF)
    packed = P.mx4_quantize(w)
    vals = P.mx4_dequantize(packed).double()   # (tested against the definition above)
    x96 = torch.randn(96, depth, device="cuda", generator=g)
    r96 = torch.randn(96, rows, device="cuda", generator=g)
    for dt, counts in ((BF, (96, 65, 64, 33, 32, 17, 16, 1)), (FP, (32, 22, 21, 11, 10, 6, 5, 1))):
        for n in counts:
            x = x96[:n].to(dt)
            want, size = x.double() @ vals.t() + r96[:n].double(), x.double().abs() @ vals.abs().t()
            y = torch.full((n, rows + 5), 3.0, device="cuda")
            got = P.mx4_linear(x, packed, residual=r96[:n], out=y[:, 1:1 + rows])
            assert bool(((got.double() - want).abs() <= plain.linear_bound(want, size, depth, 3 if dt == FP else 1, FP)).all()), (n, dt)
            assert bool((y[:, 0] == 3).all()) and bool((y[:, 1 + rows:] == 3).all())
            if n == counts[0]:
                full = got.clone()
            assert torch.equal(got, full[:n]), (n, dt)


def test_slices_of_calls_on_several_streams_and_in_graphs(P):
    """Two captured products whose slices meet in workspaces, replayed on two streams at once with eager ones between."""
    w = P.mx4_quantize(_weight(1, 600, 9000))
    xs = [_randn(i, 20, 9000) for i in range(3)]
    want = [P.mx4_linear(x, w) for x in xs]
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in (0, 1):
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            outs.append(P.mx4_linear(xs[i], w))
    for _ in range(4):
        for y in outs:
            y.zero_()
        torch.cuda.synchronize()
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        eager = P.mx4_linear(xs[2], w)
        torch.cuda.synchronize()
        assert torch.equal(eager, want[2]) and all(torch.equal(outs[i], want[i]) for i in (0, 1))


def test_a_row_does_not_depend_on_the_rows_beside_it(P):
    """Up to 96 columns every kernel adds a row's products in the same order (three columns an fp32 row)."""
    for rows, depth in ((300, 1160), (4400, 4736), (8300, 520)):
        packed, gated = P.mx4_quantize(_weight(1, rows, depth)), P.mx4_quantize_gated(_weight(2, rows, depth), _weight(3, rows, depth))
        for dt, counts in ((FP, (1, 2, 5, 6, 9, 16, 17, 22, 32)), (BF, (1, 8, 16, 17, 33, 49, 65, 96))):
            x = _randn(4, 96, depth, dtype=dt)
            full, fullg = P.mx4_linear(x[:counts[-1]], packed), P.mx4_swiglu(x[:counts[-1]], gated)
            for n in counts[:-1]:
                assert torch.equal(P.mx4_linear(x[:n], packed), full[:n]), (rows, depth, dt, n)
                assert torch.equal(P.mx4_swiglu(x[:n], gated), fullg[:n]), (rows, depth, dt, n)


_GLU = [(1, 1, 1), (1, 344, 1032), (2, 8, 128), (5, 17, 100), (9, 688, 256), (10, 100, 777), (16, 72, 4096), (32, 200, 640), (40, 129, 264), (64, 96, 1000),
        (70, 65, 130), (128, 40, 512), (150, 344, 136), (520, 100, 264)]


@pytest.mark.parametrize("n,rows,depth", _GLU)
@pytest.mark.parametrize("x_dtype", [FP, BF], ids=["x32", "x16"])
def test_swiglu_against_64_bits(P, n, rows, depth, x_dtype):
    gate, up = _weight(rows, rows, depth), _weight(rows + 1, rows, depth)
    x = _randn(depth + 1, n, depth, dtype=x_dtype)
    packed = P.mx4_quantize_gated(gate, up)
    ref = plain.swiglu(x, plain.values(gate), plain.values(up))
    for out in (FP, BF):
        bound = plain.swiglu_bound(*ref, depth, 3 if x_dtype == FP else 1, out)
        _close(P.mx4_swiglu(x, packed, out_dtype=out), ref[0], bound, (n, rows, depth, out))
    y = torch.full((n, rows + 4), 3.0, dtype=x_dtype, device="cuda")
    P.mx4_swiglu(_apart(x, 9), packed, out=y[:, 2:2 + rows])
    _close(y[:, 2:2 + rows], ref[0], plain.swiglu_bound(*ref, depth, 3 if x_dtype == FP else 1, x_dtype), "rows apart")
    assert bool((y[:, :2] == 3).all()) and bool((y[:, 2 + rows:] == 3).all())


@pytest.mark.parametrize("n", [1, 4, 9, 20, 40, 70, 140, 300])
@pytest.mark.parametrize("depth", [40, 300, 1160])
def test_a_row_of_ones_and_zeros_picks_an_element_exactly(P, n, depth):
    """Weights with one 1 in each row: the product is that element of x, bit for bit in fp32 (all three terms arrive, at the right place
    of a block), numbers near the largest and the smallest among them; in bf16 its
    rounding."""
    rows = 70
    at = [(7 * i * i + 3 * i) % depth for i in range(rows)]
    w = torch.zeros(rows, depth, device="cuda")
    for i, k in enumerate(at):
        w[i, k] = 1.0
    packed = P.mx4_quantize(w)
    x = _randn(n + depth, n, depth) * torch.exp(4.0 * _randn(9, n, depth))
    x[0, at[0]], x[n - 1, at[1]], x[n // 2, at[2]] = 3.4e38, -1.17549435e-38, 1.0000001
    got = P.mx4_linear(x, packed)
    assert torch.equal(got, x[:, at])
    assert torch.equal(P.mx4_linear(x, packed, out_dtype=BF), x[:, at].to(BF))
    # (3.4e38 is past bf16's largest number and half a step, 3.396e38: an infinity there, whose products with the row's zeros are NaN)
    want = (x.to(BF).cpu().double() @ w.cpu().double().t()).to(BF)
    assert torch.allclose(P.mx4_linear(x.to(BF), packed).cpu(), want, rtol=0.0, atol=0.0, equal_nan=True)


@pytest.mark.parametrize("n", [3, 12, 40, 80, 200])
@pytest.mark.parametrize("x_dtype", [FP, BF], ids=["x32", "x16"])
def test_infinities_and_nans_stay_in_their_rows(P, n, x_dtype):
    """A row of x with an infinity or a NaN, also in its last elements and next to the padding of a ragged depth, changes no other row; an
    infinity times a positive weight is an infinity; a NaN block of a weight row makes that result NaN for every row of x, no other."""
    rows, depth = 37, 200
    w = _weight(4, rows, depth).abs().clamp(min=0.01)
    x = _randn(6, n, depth, dtype=x_dtype)
    clean = P.mx4_linear(x, P.mx4_quantize(w))
    x2 = x.clone()
    x2[1, depth - 1] = float("inf")
    x2[n - 1, 0] = float("nan")
    packed = P.mx4_quantize(w)
    vals = plain.values(w)
    got = P.mx4_linear(_apart(x2, 5), packed)
    keep = [r for r in range(n) if r not in (1, n - 1)]
    assert torch.equal(got[keep], clean[keep]) and bool(got[n - 1].isnan().all())
    hit = (vals[:, depth - 1] > 0).tolist()
    assert got[1].isinf().tolist() == hit and got[1].isnan().tolist() == [not h for h in hit]
    w[5, 70] = float("nan")
    bad = P.mx4_linear(x, P.mx4_quantize(w))
    others = [o for o in range(rows) if o != 5]
    assert bool(bad[:, 5].isnan().all()) and torch.equal(bad[:, others], clean[:, others])


def test_shapes_of_activations_and_no_rows(P):
    w = _weight(1, 48, 160)
    packed, gated = P.mx4_quantize(w), P.mx4_quantize_gated(w, w)
    x = _randn(2, 2, 3, 160, dtype=BF)
    y = P.mx4_linear(x, packed)
    assert y.shape == (2, 3, 48) and torch.equal(y.view(6, 48), P.mx4_linear(x.view(6, 160), packed))
    assert torch.equal(P.mx4_linear(x[0, 0], packed), P.mx4_linear(x[0, :1], packed)[0])
    assert P.mx4_swiglu(x, gated).shape == (2, 3, 48)
    for shape in ((0, 160), (2, 0, 160)):
        e = torch.empty(*shape, dtype=BF, device="cuda")
        assert P.mx4_linear(e, packed).shape == (*shape[:-1], 48) and P.mx4_swiglu(e, gated).shape == (*shape[:-1], 48)
    # x that every row shares
    same = x[0, :1].expand(4, 160)
    with pytest.raises(ValueError, match="overlap"):
        P.mx4_linear(same, packed)


def test_refusals_on_device(P):
    w = P.mx4_quantize(_weight(1, 48, 160))
    g = P.mx4_quantize_gated(_weight(1, 48, 160), _weight(2, 48, 160))
    x = _randn(2, 4, 160, dtype=BF)
    for bad in (x[:, :159], x.t(), x.t().contiguous().t(), x[:, ::2], x.cpu()):
        with pytest.raises(ValueError):
            P.mx4_linear(bad, w)
        with pytest.raises(ValueError):
            P.mx4_swiglu(bad, g)
    with pytest.raises(TypeError):
        P.mx4_linear(x.half(), w)
    with pytest.raises(TypeError):
        P.mx4_linear(x, w, out_dtype=torch.float16)
    with pytest.raises(ValueError, match="gradient"):
        P.mx4_linear(x.float().requires_grad_(), w)
    with torch.no_grad():
        P.mx4_linear(x.float().requires_grad_(), w)
    r = _randn(3, 4, 48, dtype=BF)
    for kw in (dict(residual=r.float()), dict(residual=r[:3]), dict(residual=r[:, :47]), dict(out=r.float(), out_dtype=BF), dict(out=r[:3]), dict(out=r.cpu()),
               dict(residual=r.cpu())):
        with pytest.raises(ValueError):
            P.mx4_linear(x, w, **kw)
    with pytest.raises(ValueError):
        P.mx4_quantize_gated(_weight(1, 48, 160), _weight(1, 48, 161))
    with pytest.raises(ValueError):
        P.mx4_quantize_gated(_weight(1, 48, 160), _weight(1, 48, 160, FP))
    with pytest.raises(ValueError):
        P.mx4_quantize(_weight(1, 48, 160).t())
    with pytest.raises(P.SwiftError):
        P.mx4_quantize(torch.empty(0, 5, device="cuda"))
    with pytest.raises(ValueError):
        P.mx4_dequantize(w, out=torch.empty(47, 160, device="cuda"))


def test_overlaps_and_row_counts_that_are_refused(P):
    w = P.mx4_quantize(_weight(1, 64, 64))
    x = _randn(2, 4, 64)
    with pytest.raises(ValueError):
        P.mx4_linear(x, w, out=x)
    with pytest.raises(ValueError):
        P.mx4_swiglu(x, P.mx4_quantize_gated(_weight(1, 64, 64), _weight(2, 64, 64)), out=x)
    base = _randn(3, 4, 128)
    with pytest.raises(ValueError):
        P.mx4_linear(x, w, residual=base.view(8, 64)[:4], out=base[:, :64])
    thin = P.mx4_quantize(_weight(1, 16, 1))
    with pytest.raises(ValueError):
        P.mx4_linear(torch.zeros(1, 1, device="cuda").expand((1 << 32) + 5, 1), thin)
    with pytest.raises(ValueError):
        P.mx4_quantize(torch.zeros(1, 1, device="cuda").expand((1 << 32) + 5, 1))
    host = P.mx4_quantize(_weight(1, 64, 64)).to("cpu")
    with pytest.raises(ValueError):
        P.mx4_dequantize(host)
    with pytest.raises(ValueError):
        P.mx4_linear(x, host)


@pytest.mark.parametrize("n,pitch", [(2, (1 << 31) + 8), (9, (1 << 28) + 8), (13, (1 << 28) + 4), (40, (1 << 26) + 8), (140, (1 << 24) + 8)])
def test_rows_whose_distances_pass_32_bits(P, n, pitch):
    """Rows of x, results and residuals (in place) so far apart that the last lie past 2^31 elements or 2^32 bytes."""
    rows, depth = 70, 200
    w = P.mx4_quantize(_weight(1, rows, depth))
    gated = P.mx4_quantize_gated(_weight(2, rows, depth), _weight(3, rows, depth))
    memory = torch.empty((n - 1) * pitch + 512, device="cuda")
    for dt in (FP, BF):
        far = memory.view(dt)
        x, y = far.as_strided((n, depth), (pitch, 1)), far.as_strided((n, rows), (pitch, 1), 256)
        near = _randn(n, n, depth, dtype=dt)
        r = _randn(n + 1, n, rows, dtype=dt)
        x.copy_(near)
        y.copy_(r)
        assert torch.equal(P.mx4_linear(x, w, residual=y, out=y), P.mx4_linear(near, w, residual=r)), dt
        assert torch.equal(y, P.mx4_linear(near, w, residual=r))
        P.mx4_swiglu(x, gated, out=y)
        assert torch.equal(y, P.mx4_swiglu(near, gated))


def test_a_matrix_of_more_than_2_to_the_32_weights(P):
    """Rows past 2^32 weights and past 2^32 bytes of codes: as the same rows by themselves, packed, read back and multiplied."""
    rows, depth = 1048600, 8200
    w = torch.empty(rows, depth, dtype=BF, device="cuda")
    for i in range(0, rows, 1 << 17):
        w[i:i + (1 << 17)].normal_()
    packed = P.mx4_quantize(w)
    assert packed.data.numel() > 1 << 32
    at = rows - 1000
    tail = P.mx4_quantize(w[at:])
    back = P.mx4_dequantize(packed, out=w)
    assert torch.equal(back[at:], P.mx4_dequantize(tail, BF))
    del back, w
    for n, dt in ((1, BF), (5, FP), (20, BF), (64, BF), (96, BF), (130, BF)):
        x = _randn(n, n, depth, dtype=dt)
        got = P.mx4_linear(x, packed)[:, at:]
        want = P.mx4_linear(x, tail)
        if n < 100:
            assert torch.equal(got, want), n
        else:  # (other tiles, the same products in other sums)
            vals = P.mx4_dequantize(tail).double()
            exact, size = x.double() @ vals.t(), x.double().abs() @ vals.abs().t()
            assert bool(((got.double() - exact).abs() <= plain.linear_bound(exact, size, depth, 1, BF)).all())


def test_a_feed_forward_block_in_a_row(P):
    """The calls as they follow one another: gate and up of a normalised row, its down projection onto the residual stream, for one
    token, a verification block and a prompt, against 64 bits on the stored bf16 values in between."""
    hidden, ffn = 520, 1400
    gate, up, down = _weight(1, ffn, hidden), _weight(2, ffn, hidden), _weight(3, hidden, ffn)
    gu, dn = P.mx4_quantize_gated(gate, up), P.mx4_quantize(down)
    vals = [plain.values(t) for t in (gate, up, down)]
    for n in (1, 9, 300):
        x = _randn(n, n, hidden, dtype=BF)
        h = P.mx4_swiglu(x, gu)
        ref = plain.swiglu(x, vals[0], vals[1])
        _close(h, ref[0], plain.swiglu_bound(*ref, hidden, 1, BF), n)
        y = P.mx4_linear(h, dn, residual=x)
        want, size = plain.linear(h, vals[2], x)
        _close(y, want, plain.linear_bound(want, size, ffn, 1, BF), n)


@pytest.mark.parametrize("n", [1, 9, 40, 200])
def test_calls_on_another_stream_and_captured_ones(P, n):
    """Work goes to the current stream; a captured call replays with new inputs, several times, with eager calls between the replays; two
    graphs and eager calls do not share a workspace."""
    w = _weight(1, 352, 700)
    packed, gated = P.mx4_quantize(w), P.mx4_quantize_gated(w, _weight(2, 352, 700))
    xs = [_randn(10 + i, n, 700) for i in range(4)]
    want = [(P.mx4_linear(x, packed), P.mx4_swiglu(x, gated)) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = (P.mx4_linear(xs[0], packed), P.mx4_swiglu(xs[0], gated))
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0][0]) and torch.equal(got[1], want[0][1])
    x1, x2 = xs[0].clone(), xs[1].clone()
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        y1 = P.mx4_linear(x1, packed)
    with torch.cuda.graph(g2):
        y2 = P.mx4_swiglu(x2, gated)
    for i in range(4):
        x1.copy_(xs[i])
        x2.copy_(xs[3 - i])
        g1.replay()
        g2.replay()
        eager = P.mx4_linear(xs[i], packed)
        torch.cuda.synchronize()
        assert torch.equal(y1, want[i][0]) and torch.equal(y2, want[3 - i][1]) and torch.equal(eager, want[i][0]), i


def test_results_do_not_change_from_call_to_call(P):
    w = P.mx4_quantize(_weight(1, 1000, 1160))
    for n in (1, 9, 33, 150):
        x = _randn(n, n, 1160, dtype=BF)
        first = P.mx4_linear(x, w)
        for _ in range(3):
            assert torch.equal(P.mx4_linear(x, w), first)


# ------------------------------------------------------------------------------------------
# models
# ------------------------------------------------------------------------------------------
def _read_back(P, weights):
    """The bf16 tensors that an MXFP4 model's stand for."""
    out = {}
    for name, t in weights.items():
        matrix = name.split(".")[-1] in ("wq", "wk", "wv", "wo", "wg", "wu", "wd")
        out[name] = P.mx4_dequantize(P.mx4_quantize(t.cuda()), BF).cpu() if matrix else t
    return out


def _pair(P, oracle_lib, shape, weights, max_seq, threads=4):
    """The oracle on the numbers, and the library on the original tensors as an MXFP4 model."""
    o = oracle_lib.Oracle(shape, max_seq, threads=threads)
    o.set_weights(_read_back(P, weights))
    g = P.SwiftModel(dataclasses.replace(shape, dtype="mxfp4"), max_seq)
    g.load_weights(weights)
    return o, g


SHAPES = {
    # a depth below one super-tile; grouped heads; ragged everywhere
    "small-gqa": hp.SMALL_GQA_BF16,
    # heads of 64: matrix-core attention; depths that end inside a block
    "d64": si.ModelShape("mx4-d64", 2, 224, 4, 2, 64, 344, 300, "bf16", 1e-5),
    # heads of 128, depths of several super-tiles
    "d128": si.ModelShape("mx4-d128", 2, 520, 8, 4, 128, 1416, 500, "bf16", 1e-5),
}


@pytest.mark.parametrize("case", list(SHAPES))
def test_model_decodes_as_the_oracle_does(P, oracle_lib, case):
    """Prompts of every block kind, greedy continuation, drafting, verification and acceptance under masks, poisoned slots."""
    shape = SHAPES[case]
    weights = hp.shaped_weights(shape, seed=8)
    o, g = _pair(P, oracle_lib, shape, weights, 700)
    rng = np.random.default_rng(1)
    for n_prompt in (1, 5, 16, 17, 40, 64, 65, 130, 200, 600):
        prompt = si.uniform_ids(n_prompt, n_prompt, shape.vocab)
        mask = (rng.random(2 * shape.n_layers) < 0.4).astype(np.uint8)
        r = hp.lockstep_swift(o, g, prompt, 14, mask, 8, 0.3, 2e-2, poison=True)
        assert r["rows_checked"] > 0
    g.close()


def test_model_at_7b_width_against_oracle(P, oracle_lib):
    shape = si.LLAMA2_7B.with_layers(2)
    weights = hp.shaped_weights(shape, seed=2)
    o, g = _pair(P, oracle_lib, shape, weights, 400, threads=8)
    mask = np.array([0, 1, 1, 0], np.uint8)
    for n_prompt in (20, 140):
        hp.lockstep_swift(o, g, si.uniform_ids(3, n_prompt, shape.vocab), 20, mask, 8, 0.0, 2e-2)
    g.close()


@pytest.mark.parametrize("case", list(SHAPES) + ["7b-width"])
def test_model_rows_equal_single_rows_bit_for_bit(P, case):
    """A token's logits do not depend on how many rows share its pass: chains of 2..32 rows, and trees, against one-row passes."""
    shape = SHAPES.get(case) or si.LLAMA2_7B.with_layers(2)
    g = P.SwiftModel(dataclasses.replace(shape, dtype="mxfp4"), 96)
    if case == "7b-width":
        for nm, t in si.iter_weights(shape, 0, "cuda:0"):
            g.load_tensor(nm, t)
    else:
        g.load_weights(hp.shaped_weights(shape, seed=3))
    g.prefill(si.uniform_ids(4, 12, shape.vocab))
    n0, t0 = g.cache_len, g.pending
    toks, rows = [t0], []
    for _ in range(32):
        tgt, lg = g.verify([g.pending], True)
        g.accept()
        toks.append(int(tgt[0]))
        rows.append(lg[0].copy())
    for R in (2, 3, 5, 6, 9, 10, 11, 16, 17, 21, 22, 26, 32):
        g.rollback(n0, t0)
        tgt, lg = g.verify(toks[:R], True)
        assert [int(x) for x in tgt] == toks[1:R + 1]
        for r in range(R):
            assert np.array_equal(lg[r], rows[r]), (case, R, r, np.abs(lg[r] - rows[r]).max())
        g.rollback(n0, t0)
        ts, ls = g.verify_static(toks[:R], True)
        assert np.array_equal(ls, lg) and np.array_equal(ts, tgt)
    rng = np.random.default_rng(8)
    for widths in ((3, 1, 5, 2), (10, 10, 10, 1), (2,) * 8):
        g.rollback(n0, t0)
        levels = [rng.integers(0, shape.vocab, w).astype(np.int32) for w in widths]
        tgt, lg = g.verify_tree(levels, True)
        row, spine = 1, [t0]
        for lv in levels:
            for i, tok in enumerate(lv):
                g.rollback(n0, t0)
                _, clg = g.verify(spine + [int(tok)], True)
                assert np.array_equal(clg[-1], lg[row + i]), (case, widths, row + i)
            row += len(lv)
            spine.append(int(lv[0]))
    g.close()


@pytest.mark.parametrize("intermediate", [8456, 9000, 18000, 22600])
def test_model_blocks_with_a_wide_feed_forward_layer(P, oracle_lib, intermediate):
    """Gate and up of enough rows that blocks share their columns between row groups: equal to one row at a time bit for bit, and to the
    oracle's."""
    shape = si.ModelShape("mx4-wide", 2, 520, 8, 4, 64, intermediate, 300, "bf16", 1e-5)
    weights = hp.shaped_weights(shape, seed=6)
    o, g = _pair(P, oracle_lib, shape, weights, 96, threads=8)
    hp.lockstep_swift(o, g, si.uniform_ids(2, 20, shape.vocab), 12, np.array([0, 1, 1, 0], np.uint8), 8, 0.0, 2e-2)
    g.close()
    g = P.SwiftModel(dataclasses.replace(shape, dtype="mxfp4"), 96)
    g.load_weights(weights)
    g.prefill(si.uniform_ids(4, 12, shape.vocab))
    n0, t0 = g.cache_len, g.pending
    toks, rows = [t0], []
    for _ in range(32):
        tgt, lg = g.verify([g.pending], True)
        g.accept()
        toks.append(int(tgt[0]))
        rows.append(lg[0].copy())
    for R in (6, 10, 11, 17, 21, 22, 31, 32):
        g.rollback(n0, t0)
        tgt, lg = g.verify(toks[:R], True)
        assert [int(x) for x in tgt] == toks[1:R + 1]
        for r in range(R):
            assert np.array_equal(lg[r], rows[r]), (R, r, np.abs(lg[r] - rows[r]).max())
    g.close()


def test_model_candidate_evaluation_against_oracle(P, oracle_lib):
    shape = SHAPES["d64"]
    weights = hp.shaped_weights(shape, seed=21)
    n_prompt, n_gen = 12, 140
    o, g = _pair(P, oracle_lib, shape, weights, n_prompt + n_gen + 8, threads=1)
    prompt = si.uniform_ids(5, n_prompt, shape.vocab)
    want = oracle_lib.generate_ar(o, prompt, n_gen)
    assert np.array_equal(P.generate_ar(g, prompt, n_gen), want)
    seq = np.concatenate([prompt, want]).astype(np.int32)
    rng = np.random.default_rng(2)
    masks = [np.zeros(4, np.uint8), np.ones(4, np.uint8)] + [(rng.random(4) < 0.5).astype(np.uint8) for _ in range(3)]
    for gamma in (1, 4, 16, 17, 32, 33, 64, 65, 128):
        for mi, mask in enumerate(masks):
            po, mo = o.eval_mask(mask, seq[-(gamma + 1):])
            pg, mg = g.eval_mask(mask, seq[-(gamma + 1):])
            assert np.array_equal(pg, po) and mg == mo, (gamma, mi)
    g.close()


def test_model_prompts_leave_the_cache_the_oracle_does(P, oracle_lib):
    """Keys and values of a prompt of macro blocks: equal up to one bf16 rounding step where a value lies next to a border."""
    shape = SHAPES["d128"]
    weights = hp.shaped_weights(shape, seed=5)
    o, g = _pair(P, oracle_lib, shape, weights, 1300)
    for n_prompt in (200, 1100):
        prompt = si.uniform_ids(n_prompt, n_prompt, shape.vocab)
        o.prefill(prompt)
        g.prefill(prompt)
        for layer in range(shape.n_layers):
            for pos in (0, 63, 64, n_prompt // 2, n_prompt - 1):
                for got_v, want_v in zip(g.read_kv(layer, pos), o.read_kv(layer, pos)):
                    assert np.all(np.abs(got_v - want_v) <= 2.0 ** -7 * np.abs(want_v) + 2.0 ** -10 * np.abs(want_v).max()), (n_prompt, layer, pos)
                    assert (got_v != want_v).mean() < 0.1, (n_prompt, layer, pos)
    g.close()


@pytest.mark.parametrize("name,n_prompt,n_new", [("7b", 300, 48), ("13b", 700, 24), ("70b", 160, 10)])
def test_full_size_models_are_lossless(P, name, n_prompt, n_new):
    """Plain greedy decoding, speculation with every kind of block, and dynamic verification emit the same tokens."""
    w = si.WORKLOADS[name]
    g = P.SwiftModel(dataclasses.replace(w.shape, dtype="mxfp4"), n_prompt + n_new + 24)
    for nm, t in si.iter_weights(w.shape, w.weight_seed, "cuda:0"):
        g.load_tensor(nm, t)
    prompt, mask = si.uniform_ids(w.prompt_seed, n_prompt, w.shape.vocab), si.workload_mask(w)
    ar = P.generate_ar(g, prompt, n_new)
    for eps, max_k in ((w.conf_threshold, w.max_k), (0.0, w.max_k), (0.0, 15)):
        out, trace = P.generate_swift(g, prompt, n_new, mask, max_k, eps)
        assert np.array_equal(out, ar), (name, eps, max_k)
    out, trace = P.generate_swift_tree(g, prompt, n_new, mask, w.max_k, w.conf_threshold)
    assert np.array_equal(out, ar), (name, "tree")
    out, trace = P.generate_swift(g, prompt, n_new, np.zeros_like(mask), w.max_k, 0.0)
    assert np.array_equal(out, ar) and all(t["m"] == len(t["draft"]) for t in trace)
    g.close()


def test_model_refuses_tensors_of_other_types(P):
    shape = dataclasses.replace(hp.SMALL_GQA_BF16, dtype="mxfp4")
    g = P.SwiftModel(shape, 32)
    with pytest.raises(P.SwiftError, match="dtype"):
        g.load_tensor("l0.wq", torch.zeros(64, 96, device="cuda"))
    with pytest.raises(P.SwiftError, match="count"):
        g.load_tensor("l0.wq", torch.zeros(64, 95, device="cuda", dtype=BF))
    g.close()
