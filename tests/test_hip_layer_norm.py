"""Layer norm (csrc/layer_norm.hip) against its formulas in 64 bits on the CPU.

Tolerances, U = 2^-24 (half a step of fp32), H = half a step of the rows' type (2^-8 of bf16, U of fp32):
mean: a sum of d terms in fp32, at most 40 of them in a chain (up to 32 per lane, then a tree), about a rounded first mean:
within 64 U of the mean magnitude.  rstd: within 64 U and half of the relative change that the mean's error makes.  y, d_x:
terms and sums in fp32, 64 U of the magnitudes that are added up, and one rounding H of the result."""
import pytest
import torch

import paper_2505_16710_amd as seco

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

# Row lengths: both sides of what a group of 16 lanes, a wavefront and a workgroup hold, and of a word (8 bf16, 4 fp32)
LENGTHS = {"bf16": [1, 3, 7, 8, 9, 127, 128, 129, 256, 257, 511, 512, 1000, 1024, 1027, 2048, 2049, 4096, 4099, 8192, 8200,
                    16384, 16385, 20001],
           "f32": [1, 3, 4, 5, 64, 66, 128, 131, 256, 257, 512, 777, 1024, 1026, 2048, 2050, 4096, 4097, 8192, 8193, 9999]}
CASES = [(t, d) for t in LENGTHS for d in LENGTHS[t]]


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _rows(seed, rows, d, dtype, pad=0, mean=0.0, lead=()):
    g = torch.Generator().manual_seed(seed)
    wide = torch.empty(*lead, rows, d + pad, dtype=dtype)
    wide[..., :d] = (torch.randn(*lead, rows, d, generator=g) + mean).to(dtype)
    wide[..., d:] = float("nan")                              # what lies between the rows is never read
    return wide[..., :d]


def _on_gpu(x):
    """The same values and strides on the GPU."""
    out = torch.empty(x.untyped_storage().nbytes() // x.element_size(), dtype=x.dtype, device=DEV)
    whole = torch.as_strided(x, (out.numel(),), (1,), 0)
    out.copy_(whole)
    return torch.as_strided(out, x.shape, x.stride(), x.storage_offset())


def _forward64(x, gain, bias, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    n = (x - mean) * rstd
    return mean[..., 0], rstd[..., 0], n * (1 if gain is None else gain.double()) + (0 if bias is None else bias.double())


def _check_forward(x, gain, bias, eps, got, dtype):
    mean, rstd, y = _forward64(x, gain, bias, eps)
    gy, gm, gr = (t.cpu().double() for t in got[:3])
    x = x.double()
    size = x.abs().mean(-1)
    assert ((gm - mean).abs() <= 64 * U * size).all()
    # a deviation is off by U of the element and what the mean is off by; the variance by twice the sum of their products
    off = 64 * U * size
    spread = (x - mean[..., None]).abs().mean(-1)
    rel = 64 * U + rstd ** 2 * (off ** 2 + U * (x.abs() * (x - mean[..., None]).abs()).mean(-1) + off * U * size + 4 * U * spread ** 2)
    assert ((gr - rstd).abs() <= rel * rstd).all()
    g = 1.0 if gain is None else gain.double().abs()
    b = 0.0 if bias is None else bias.double().abs()
    n = ((x - mean[..., None]) * rstd[..., None]).abs()
    slack = (rel[..., None] + 8 * U) * n * g + (4 * U * x.abs() + off[..., None]) * rstd[..., None] * g + 4 * U * b
    assert ((gy - y).abs() <= slack * (1 + _half(dtype)) + _half(dtype) * y.abs()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t,d", CASES)
@pytest.mark.parametrize("residual", ["none", "apart", "in place"])
def test_forward(t, d, residual):
    dtype, rows = TYPES[t], 5 if d > 300 else 37
    pad = (0, 3)[d % 2]
    x, r = _rows(d, rows, d, dtype, pad), _rows(d + 1, rows, d, dtype, 1)
    gain, bias = _rows(d + 2, 1, d, dtype)[0].contiguous() + 1, _rows(d + 3, 1, d, dtype)[0].contiguous()
    dx = _on_gpu(x)
    kw = {} if residual == "none" else {"residual": _on_gpu(r), "x_out": dx if residual == "in place" else None}
    got = seco.layer_norm_fwd(dx, gain.to(DEV), bias.to(DEV), eps=1e-5, **kw)
    s = x if residual == "none" else (x.float() + r.float()).to(dtype)
    if residual != "none":
        assert torch.equal(got[3].cpu(), s)
    if residual != "in place":
        assert torch.equal(dx.cpu(), x)
    if pad:                                                       # ... nor written
        assert torch.isnan(torch.as_strided(dx, (rows - 1, pad), (d + pad, 1), d)).all()
    _check_forward(s, gain, bias, 1e-5, got, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("t,d", CASES)
@pytest.mark.parametrize("rows,d_in", [(1, "none"), (7, "in place"), (300, "apart"), (1030, "none"), (1301, "apart")])
def test_backward(t, d, rows, d_in):
    if rows * d > 1 << 22:
        rows = max(2, (1 << 22) // d)
    _check_backward(t, d, rows, d_in)


def _check_backward(t, d, rows, d_in):
    dtype = TYPES[t]
    x, dy, extra = _rows(d + 4, rows, d, dtype, 2), _rows(d + 5, rows, d, dtype), _rows(d + 6, rows, d, dtype)
    gain = _rows(d + 7, 1, d, dtype)[0].contiguous() + 1
    mean, rstd, _ = _forward64(x, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    din = None if d_in == "none" else _on_gpu(extra)
    got = seco.layer_norm_bwd(_on_gpu(x), gain.to(DEV), mean.to(DEV), rstd.to(DEV), _on_gpu(dy), d_in=din,
                              d_x=din if d_in == "in place" else None)
    if d_in == "in place":
        assert got[0] is din
    gx, gg, gb = (a.cpu().double() for a in got)
    x64, dy64, r = x.double(), dy.double(), rstd.double()[:, None]
    n, e = (x64 - mean.double()[:, None]) * r, dy64 * gain.double()
    base = torch.zeros_like(e) if d_in == "none" else extra.double()
    ref = base + r * (e - e.mean(1, keepdim=True) - n * (e * n).mean(1, keepdim=True))
    n_size = n.abs() + 2 * (x64.abs() + mean.double().abs()[:, None]) * r / 64          # (x - mean is off by a step of either)
    size = base.abs() + r * (e.abs() + e.abs().mean(1, keepdim=True) + n_size * (e.abs() * n_size).mean(1, keepdim=True))
    assert ((gx - ref).abs() <= 64 * U * size + _half(dtype) * ref.abs()).all()
    # sums of a column: up to 16 rows in a chain in a workgroup's share, then a tree and at most 40 shares
    for got_sum, terms, bound in ((gg, dy64 * n, dy64.abs() * n_size), (gb, dy64, dy64.abs())):
        assert ((got_sum - terms.sum(0)).abs() <= 64 * U * bound.sum(0) + _half(dtype) * terms.sum(0).abs()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t,d,rows,d_in", [("f32", 8197, 1027, "in place"), ("f32", 16384, 100, "apart"), ("f32", 12003, 300, "none"),
                                           ("bf16", 16400, 1030, "none"), ("bf16", 16411, 1301, "apart"), ("f32", 16385, 768, "in place")])
def test_backward_of_long_rows(t, d, rows, d_in):
    _check_backward(t, d, rows, d_in)


@pytest.mark.gpu
@pytest.mark.parametrize("t,d", [("bf16", 5), ("bf16", 96), ("bf16", 250), ("bf16", 1027), ("bf16", 2056), ("bf16", 4099), ("bf16", 12001), ("bf16", 20001),
                                 ("f32", 1027), ("f32", 8002), ("f32", 17001)])
@pytest.mark.parametrize("rows", [3, 2100])
def test_forward_results_in_the_place_of_either_input(t, d, rows):
    """y in the place of x or of the residual, x_out in that of the other, or apart: the same bits."""
    dtype = TYPES[t]
    x, r = (_on_gpu(_rows(64 + i, min(rows, (1 << 23) // d), d, dtype)) for i in range(2))
    want = seco.layer_norm_fwd(x, residual=r)
    for y_at, out_at in (("x", None), ("r", None), ("x", "r"), ("r", "x")):
        a = {"x": x.clone(), "r": r.clone(), None: None}
        got = seco.layer_norm_fwd(a["x"], residual=a["r"], y=a[y_at], x_out=a[out_at])
        assert got[0] is a[y_at] and all(torch.equal(p, q) for p, q in zip(got, want))
    place = x.clone()
    alone = seco.layer_norm_fwd(x)
    assert all(torch.equal(p, q) for p, q in zip(seco.layer_norm_fwd(place, y=place), alone))


@pytest.mark.gpu
@pytest.mark.parametrize("t,d,rows,d_in", [("bf16", 2056, 1301, "none"), ("bf16", 4099, 1301, "in place"), ("bf16", 8192, 1290, "apart"),
                                           ("bf16", 12001, 1301, "in place"), ("bf16", 12001, 1400, "apart"), ("bf16", 16384, 1281, "none"),
                                           ("f32", 2051, 1301, "in place"), ("f32", 4097, 1301, "in place"), ("f32", 8192, 1283, "apart")])
def test_backward_of_more_wide_rows_than_one_launch_takes(t, d, rows, d_in):
    """A workgroup to several rows in turn, at every number of words to a lane; what is left over does not come out even."""
    _check_backward(t, d, rows, d_in)


@pytest.mark.gpu
@pytest.mark.parametrize("t,d,rows", [("bf16", 1024, 1500), ("bf16", 2056, 1500), ("bf16", 4099, 700), ("bf16", 4099, 1301), ("bf16", 8192, 1290),
                                      ("bf16", 12001, 1301), ("bf16", 16400, 600), ("f32", 2051, 1301), ("f32", 8192, 1283), ("f32", 8195, 1400)])
def test_shares_of_a_training_step_are_added_to(t, d, rows):
    """As the step calls it: shares of the sums on top of what is there, chunk after chunk, d_x in the place of d_in."""
    import ctypes as C
    dtype, U1 = TYPES[t], 64 * U
    gain = _rows(d + 7, 1, d, dtype)[0].contiguous()
    parts = torch.randn(2, 256, d, generator=torch.Generator().manual_seed(d)).to(DEV)
    want, size = parts.double().sum(1).cpu(), parts.double().abs().sum(1).cpu()
    lib = seco.load_library()
    gd = gain.to(DEV)
    for k in range(2):
        x, dy, extra = (_rows(10 * k + i, rows, d, dtype) for i in range(3))
        mean, rstd, _ = _forward64(x, None, None, 1e-5)
        mean, rstd = mean.float(), rstd.float()
        at = [a.to(DEV) for a in (x, mean, rstd, dy, extra)]
        p = [C.c_void_p(a.data_ptr()) for a in at]
        apart = seco.layer_norm_bwd(at[0], gd, at[1], at[2], at[3], d_in=at[4])[0]
        rc = lib.dec_layer_norm_bwd(C.c_int(1 if t == "bf16" else 0), p[0], C.c_void_p(gd.data_ptr()), p[1], p[2], p[3], p[4], p[4],
                                    C.c_void_p(parts.data_ptr()), C.c_int64(rows), C.c_int64(d),
                                    C.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == 0 and torch.equal(at[4], apart)
        n = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        n_size = n.abs() + 2 * (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None] / 64
        want += torch.stack([(dy.double() * n).sum(0), dy.double().sum(0)])
        size += torch.stack([(dy.double().abs() * n_size).sum(0), dy.double().abs().sum(0)])
        assert ((parts.double().sum(1).cpu() - want).abs() <= U1 * size).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", [(1, 3), (2, 1024), (129, 45), (513, 260), (1024, 1027), (1280, 1027), (1281, 1027), (1900, 333), (1400, 4100), (300, 16384), (40, 16390), (100, 12001), (1040, 16391)])
def test_where_the_results_lie_changes_nothing(t, rows, d):
    """d_x apart, in the place of x, of d_y or (one row apart in the same buffer) beside x: the same bits; one sum without the other."""
    dtype = TYPES[t]
    x, dy = _on_gpu(_rows(60, rows, d, dtype)), _on_gpu(_rows(61, rows, d, dtype))
    gain = _rows(62, 1, d, dtype)[0].contiguous().to(DEV)
    _, mean, rstd = seco.layer_norm_fwd(x, gain)
    first = seco.layer_norm_bwd(x, gain, mean, rstd, dy)
    for place in ("x", "d_y"):
        x2, dy2 = x.clone(), dy.clone()
        got = seco.layer_norm_bwd(x2, gain, mean, rstd, dy2, d_x=x2 if place == "x" else dy2)
        assert got[0] is (x2 if place == "x" else dy2)
        assert all(torch.equal(a, b) for a, b in zip(got, first)), place
    wide = torch.empty(rows, 2 * d, dtype=dtype, device=DEV)
    wide[:, :d] = x
    got = seco.layer_norm_bwd(wide[:, :d], gain, mean, rstd, dy, d_x=wide[:, d:])
    assert all(torch.equal(a, b) for a, b in zip(got, first)) and torch.equal(wide[:, :d], x)
    only = seco.layer_norm_bwd(x, gain, mean, rstd, dy, with_bias=False)
    assert only[2] is None and torch.equal(only[1], first[1]) and torch.equal(only[0], first[0])
    only = seco.layer_norm_bwd(x, gain, mean, rstd, dy, with_gain=False)
    assert only[1] is None and torch.equal(only[2], first[2]) and torch.equal(only[0], first[0])


@pytest.mark.gpu
@pytest.mark.parametrize("t,rows,d", [("bf16", 700, 4099), ("bf16", 2500, 4099), ("bf16", 1100, 12001), ("f32", 300, 4102), ("f32", 3000, 2051)])
def test_gradient_added_in_place(t, rows, d):
    """d_x in the place of d_in, rows whose last words overlap across wavefronts: the same bits as apart."""
    dtype = TYPES[t]
    x, dy, extra = (_on_gpu(_rows(63 + i, rows, d, dtype)) for i in range(3))
    _, mean, rstd = seco.layer_norm_fwd(x, None)
    apart = seco.layer_norm_bwd(x, None, mean, rstd, dy, d_in=extra)
    place = extra.clone()
    got = seco.layer_norm_bwd(x, None, mean, rstd, dy, d_in=place, d_x=place)
    assert got[0] is place and all(torch.equal(a, b) for a, b in zip(got, apart))


@pytest.mark.gpu
@pytest.mark.parametrize("t,rows,d", [("bf16", 1400, 12001), ("bf16", 1300, 8203), ("bf16", 1301, 16381), ("f32", 1300, 8190)])
def test_gradient_added_in_place_of_more_rows(t, rows, d):
    test_gradient_added_in_place(t, rows, d)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [700, 1500])
@pytest.mark.parametrize("t,d", [("bf16", 1024), ("bf16", 4096), ("bf16", 130), ("bf16", 20001), ("f32", 8192), ("f32", 63)])
def test_results_are_the_same_every_time(t, d, rows):
    dtype = TYPES[t]
    x, dy = _on_gpu(_rows(1, rows, d, dtype)), _on_gpu(_rows(2, rows, d, dtype))
    gain = torch.ones(d, dtype=dtype, device=DEV)
    y, mean, rstd = seco.layer_norm_fwd(x, gain)
    first = seco.layer_norm_bwd(x, gain, mean, rstd, dy)
    for _ in range(3):
        again = seco.layer_norm_fwd(x, gain)
        assert all(torch.equal(a, b) for a, b in zip(again, (y, mean, rstd)))
        assert all(torch.equal(a, b) for a, b in zip(seco.layer_norm_bwd(x, gain, mean, rstd, dy), first))


@pytest.mark.gpu
def test_gradients_against_differences():
    """Central differences of a weighted sum of y, in 64 bits, at the same inputs."""
    rows, d, eps, h = 6, 45, 1e-5, 1e-5
    x, w = _rows(20, rows, d, torch.float32), _rows(21, rows, d, torch.float32)
    gain, bias = _rows(22, 1, d, torch.float32)[0] + 1, _rows(23, 1, d, torch.float32)[0]
    _, mean, rstd = seco.layer_norm_fwd(x.to(DEV), gain.contiguous().to(DEV), bias.contiguous().to(DEV), eps=eps)
    got = seco.layer_norm_bwd(x.to(DEV), gain.contiguous().to(DEV), mean, rstd, w.to(DEV))

    def value(x, gain, bias):
        return float((_forward64(x, gain, bias, eps)[2] * w.double()).sum())
    args = [x.double(), gain.double(), bias.double()]
    for k, g in enumerate(got):
        flat = args[k].reshape(-1)
        for i in range(0, flat.numel(), 7):
            ends = []
            for sign in (1, -1):
                moved = flat.clone()
                moved[i] += sign * h
                ends.append(value(*[moved.view_as(args[k]) if j == k else args[j] for j in range(3)]))
            # (the third derivative's share h^2 and the rounding of the values over 2 h are below 1e-8)
            assert abs((ends[0] - ends[1]) / (2 * h) - float(g.reshape(-1)[i])) < 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("t,d", [("bf16", 256), ("bf16", 4096), ("f32", 1000), ("f32", 30000)])
def test_rows_with_a_mean_far_from_zero(t, d):
    """Variance about the mean: with a mean of 300 deviations, rows keep what their own rounding leaves."""
    dtype = TYPES[t]
    x = _rows(30, 4, d, dtype, mean=300.0)
    _check_forward(x, None, None, 1e-5, seco.layer_norm_fwd(x.to(DEV)), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_rows_of_one_value_and_of_none(t):
    dtype = TYPES[t]
    x = torch.full((3, 512), 7.0, dtype=dtype, device=DEV)
    gain, bias = torch.full((512,), 2.0, dtype=dtype, device=DEV), torch.full((512,), 0.5, dtype=dtype, device=DEV)
    y, mean, rstd = seco.layer_norm_fwd(x, gain, bias, eps=1e-5)
    assert (y == 0.5).all() and (mean == 7).all() and ((rstd - 1e-5 ** -0.5).abs() < 64 * U * 317).all()
    # no rows: empty results, sums of nothing
    none = torch.empty(0, 512, dtype=dtype, device=DEV)
    y, mean, rstd = seco.layer_norm_fwd(none, gain, bias)
    assert y.shape == (0, 512) and mean.shape == rstd.shape == (0,)
    dx, dg, db = seco.layer_norm_bwd(none, gain, mean, rstd, none)
    assert dx.shape == (0, 512) and not dg.any() and not db.any() and dg.shape == db.shape == (512,)


@pytest.mark.gpu
@pytest.mark.parametrize("t,d", [("bf16", 96), ("bf16", 1024), ("bf16", 5000), ("f32", 17000)])
def test_infinities_and_nan_stay_in_their_row(t, d):
    dtype = TYPES[t]
    x, dy = _rows(40, 9, d, dtype), _rows(41, 9, d, dtype)
    bad = x.clone()
    bad[2, d // 2], bad[5, 0], bad[7, d - 1] = float("inf"), float("nan"), float("-inf")
    good = [i for i in range(9) if i not in (2, 5, 7)]
    clean, mean, rstd = seco.layer_norm_fwd(x.to(DEV))
    y, m2, r2 = seco.layer_norm_fwd(bad.to(DEV))
    assert torch.equal(y[good], clean[good]) and torch.isnan(y[[2, 5, 7]]).all()
    dx = seco.layer_norm_bwd(x.to(DEV), None, mean, rstd, dy.to(DEV))[0]
    dx2 = seco.layer_norm_bwd(bad.to(DEV), None, m2, r2, dy.to(DEV))[0]
    assert torch.equal(dx[good], dx2[good]) and torch.isnan(dx2[[2, 5, 7]]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t,d", [("bf16", 5), ("bf16", 96), ("bf16", 1024), ("bf16", 1027), ("bf16", 5000), ("f32", 4096), ("f32", 17000)])
@pytest.mark.parametrize("residual", [False, True])
def test_statistics_of_rows_that_are_not_finite(t, d, residual):
    """The formulas': rstd is NaN, the mean the infinity of the row's sum, or NaN."""
    dtype, inf = TYPES[t], float("inf")
    x, r = _rows(42, 9, d, dtype), _rows(43, 9, d, dtype)
    bad = x.clone()
    bad[2, d // 2], bad[5, 0], bad[7, d - 1] = inf, float("nan"), -inf
    bad[8, 0], bad[8, d - 1] = inf, -inf
    kw = {"residual": r.to(DEV)} if residual else {}
    good = [0, 1, 3, 4, 6]
    _, mean, rstd, *_ = seco.layer_norm_fwd(x.to(DEV), **kw)
    _, m2, r2, *_ = seco.layer_norm_fwd(bad.to(DEV), **kw)
    assert torch.equal(m2[good], mean[good]) and torch.equal(r2[good], rstd[good])
    assert torch.isnan(r2[[2, 5, 7, 8]]).all()
    assert m2[2] == inf and m2[7] == -inf and torch.isnan(m2[[5, 8]]).all()


@pytest.mark.gpu
def test_gain_types_missing_gain_and_wanted_sums():
    d, rows = 1000, 600
    x, dy = _rows(50, rows, d, torch.bfloat16), _rows(51, rows, d, torch.bfloat16)
    gain, bias = _rows(52, 1, d, torch.float32)[0].contiguous() + 1, _rows(53, 1, d, torch.float32)[0].contiguous()
    xd, dyd = x.to(DEV), dy.to(DEV)
    got = seco.layer_norm_fwd(xd, gain.to(DEV), bias.to(DEV))
    _check_forward(x, gain, bias, 1e-5, got, torch.bfloat16)
    _check_forward(x, None, bias, 1e-5, seco.layer_norm_fwd(xd, None, bias.to(DEV)), torch.bfloat16)
    dx, dg, db = seco.layer_norm_bwd(xd, gain.to(DEV), got[1], got[2], dyd)
    assert dg.dtype == db.dtype == torch.float32
    for kw in ({"with_gain": False}, {"with_bias": False}, {"with_gain": False, "with_bias": False}):
        dx2, dg2, db2 = seco.layer_norm_bwd(xd, gain.to(DEV), got[1], got[2], dyd, **kw)
        assert torch.equal(dx, dx2)
        assert dg2 is None if "with_gain" in kw else torch.equal(dg, dg2)
        assert db2 is None if "with_bias" in kw else torch.equal(db, db2)
    # a gain of ones is no gain
    ones = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    a, b = (seco.layer_norm_bwd(xd, g, got[1], got[2], dyd) for g in (ones, None))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [700, 1500])
def test_a_bias_without_a_gain_has_a_gradient_of_its_type(rows):
    """An fp32 bias on bf16 rows: the sum over the rows in fp32, not rounded to bf16 on its way."""
    from paper_2505_16710_amd.chunk_loop import LayerNorm
    d = 96
    x, dy = _rows(54, rows, d, torch.bfloat16), _rows(55, rows, d, torch.bfloat16)
    bias = _rows(56, 1, d, torch.float32)[0].contiguous().to(DEV).requires_grad_()
    LayerNorm.apply(x.to(DEV), None, bias).backward(dy.to(DEV))
    bound = 64 * U * dy.double().abs().sum(0)
    assert ((bias.grad.cpu().double() - dy.double().sum(0)).abs() <= bound).all()
    _, mean, rstd = seco.layer_norm_fwd(x.to(DEV), None, bias.detach())
    _, dg, db = seco.layer_norm_bwd(x.to(DEV), None, mean, rstd, dy.to(DEV), dtype=torch.float32)
    assert dg.dtype == torch.float32 and torch.equal(db, bias.grad)
    _, dg, db = seco.layer_norm_bwd(x.to(DEV), None, mean, rstd, dy.to(DEV))
    assert dg.dtype == db.dtype == torch.bfloat16 and torch.equal(db, bias.grad.bfloat16())


def test_refused_types_of_sums():
    x, g, m = torch.zeros(4, 16), torch.ones(16), torch.zeros(4)
    for args, dtype in (((x, g, m, m, x), torch.bfloat16), ((x, None, m, m, x), torch.bfloat16), ((x, None, m, m, x), torch.float16),
                        ((x, None, m, m, x), 1)):
        with pytest.raises(TypeError):
            seco.layer_norm_bwd(*args, dtype=dtype)
    with pytest.raises(ValueError, match="on one GPU"):
        seco.layer_norm_bwd(x, g, m, m, x, dtype=torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 1024, 4096])
def test_layouts(d):
    """Leading dimensions, rows of a wider buffer, a row for all, unaligned starts."""
    base = _rows(60, 2 * 3 * 5, d + 24, torch.bfloat16).contiguous()
    gain = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    want = seco.layer_norm_fwd(base[:, 3:3 + d].contiguous().to(DEV), gain)
    wide = base.view(2, 3, 5, d + 24).to(DEV)[..., 3:3 + d]
    got = seco.layer_norm_fwd(wide, gain)
    assert got[0].shape == (2, 3, 5, d) and got[1].shape == (2, 3, 5)
    assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip(got, want))
    out = torch.zeros(30, d + 24, dtype=torch.bfloat16, device=DEV)
    seco.layer_norm_fwd(wide.reshape(30, d), gain, y=out[:, 5:5 + d])
    assert torch.equal(out[:, 5:5 + d], want[0]) and not out[:, :5].any() and not out[:, 5 + d:].any()
    one = wide[0, 0, 0].expand(7, d)                          # a stride of 0
    assert torch.equal(seco.layer_norm_fwd(one, gain)[0], want[0][:1].expand(7, d))
    row = seco.layer_norm_fwd(wide[0, 0, 0], gain)            # a single row, no leading dimension
    assert torch.equal(row[0], want[0][0]) and row[1].shape == ()


@pytest.mark.gpu
@pytest.mark.parametrize("t,d", [("bf16", 5), ("bf16", 100), ("bf16", 250), ("bf16", 1027), ("bf16", 2048), ("bf16", 4100), ("bf16", 8200),
                                 ("bf16", 20001), ("f32", 1027), ("f32", 4096), ("f32", 8000)])
@pytest.mark.parametrize("rows", [1, 2, 5, 31, 1030, 1300])
def test_what_lies_behind_the_rows_stays(t, d, rows):
    dtype = TYPES[t]
    rows = min(rows, max(2, (1 << 21) // d))
    x, r, dy = (_rows(90 + i, rows, d, dtype).to(DEV) for i in range(3))
    gain = torch.ones(d, dtype=dtype, device=DEV)

    def room():
        return torch.full((rows + 8, d + 3), 77.0, dtype=dtype, device=DEV)
    bufs = [room() for _ in range(3)]
    y, out, dx = (b[4:4 + rows, 1:1 + d] for b in bufs)
    _, mean, rstd, _ = seco.layer_norm_fwd(x, gain, residual=r, y=y, x_out=out)
    seco.layer_norm_bwd(out, gain, mean, rstd, dy, d_in=r, d_x=dx)
    seco.layer_norm_bwd(out, gain, mean, rstd, dy, d_x=dx)
    for b in bufs:
        assert (b[4:4 + rows, 1:1 + d] != 77).any()
        b[4:4 + rows, 1:1 + d] = 77
        assert (b == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t,d", [("bf16", 2048), ("bf16", 8192), ("bf16", 16384), ("f32", 4096)])
def test_results_that_no_cache_holds(t, d):
    """256 MiB and more of them take other accesses: every row is what it is in a call of a few rows."""
    dtype = TYPES[t]
    rows = (1 << 28) // (d * torch.finfo(dtype).bits // 8) + 3
    g = torch.Generator(device=DEV).manual_seed(d)
    x, r, dy = (torch.randn(rows, d, generator=g, device=DEV, dtype=dtype) for _ in range(3))
    gain = torch.ones(d, dtype=dtype, device=DEV)
    y, mean, rstd, out = seco.layer_norm_fwd(x, gain, residual=r)
    dx, dg, db = seco.layer_norm_bwd(out, gain, mean, rstd, dy, d_in=r)
    dx2 = seco.layer_norm_bwd(out, gain, mean, rstd, dy, with_gain=False, with_bias=False)[0]
    for at in (slice(0, 600), slice(rows // 2, rows // 2 + 600), slice(rows - 600, rows)):
        few = seco.layer_norm_fwd(x[at], gain, residual=r[at])
        assert all(torch.equal(a[at], b) for a, b in zip((y, mean, rstd, out), few))
        assert torch.equal(dx[at], seco.layer_norm_bwd(out[at], gain, mean[at], rstd[at], dy[at], d_in=r[at])[0])
        assert torch.equal(dx2[at], seco.layer_norm_bwd(out[at], gain, mean[at], rstd[at], dy[at])[0])
    ref, size = torch.zeros(2, d, dtype=torch.float64, device=DEV), torch.zeros(2, d, dtype=torch.float64, device=DEV)
    for at in range(0, rows, 4096):
        y64 = dy[at:at + 4096].double()
        n = (out[at:at + 4096].double() - mean[at:at + 4096, None].double()) * rstd[at:at + 4096, None].double()
        ref += torch.stack([(y64 * n).sum(0), y64.sum(0)])
        size += torch.stack([(y64 * n).abs().sum(0), y64.abs().sum(0)])
    # a share's chain is up to rows / 256 long, 64 U for 40 terms above
    bound = 64 * U * max(1, rows / 256 / 40) * size + _half(dtype) * ref.abs()
    assert ((torch.stack([dg, db]).double() - ref).abs() <= bound).all()


@pytest.mark.gpu
def test_more_rows_than_a_grid_holds_along_x():
    """16 short rows to a workgroup, 2^22 workgroups along x: the rows behind them."""
    rows = (1 << 26) + 5
    x = torch.ones(rows, 4, dtype=torch.bfloat16, device=DEV)
    x[-3:] = torch.tensor([1.0, 2.0, 3.0, 6.0], device=DEV)
    y, mean, rstd = seco.layer_norm_fwd(x)
    assert (mean[:-3] == 1).all() and (mean[-3:] == 3).all() and torch.isfinite(rstd).all()
    assert not y[:-3].any() and (y[-1, 3] > 1).item()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", [(300, 1024), (1500, 1024), (1400, 4099), (30, 20001)])
def test_captured_and_replayed(rows, d):
    x, dy = _rows(70, rows, d, torch.bfloat16).to(DEV), _rows(71, rows, d, torch.bfloat16).to(DEV)
    gain = torch.ones(d, dtype=torch.bfloat16, device=DEV)

    def both():
        y, mean, rstd = seco.layer_norm_fwd(x, gain)
        return (y, *seco.layer_norm_bwd(x, gain, mean, rstd, dy))
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(3):
        x.normal_(generator=torch.Generator(device=DEV).manual_seed(k))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, both()))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [300, 1500])
def test_two_graphs_side_by_side(rows):
    """Two captured backwards replayed at once on two streams: each has its own shares and sums."""
    gain = torch.ones(1024, dtype=torch.bfloat16, device=DEV)
    graphs, outs, want, streams = [], [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(2):
        x, dy = _rows(72 + i, rows, 1024, torch.bfloat16).to(DEV), _rows(74 + i, rows, 1024, torch.bfloat16).to(DEV)
        _, mean, rstd = seco.layer_norm_fwd(x, gain)
        want.append(seco.layer_norm_bwd(x, gain, mean, rstd, dy))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(10):
                out = seco.layer_norm_bwd(x, gain, mean, rstd, dy)
        graphs.append((graph, x, dy, mean, rstd))
        outs.append(out)
    for _ in range(3):
        for t in outs[0] + outs[1]:
            t.zero_()
        torch.cuda.synchronize()
        for (graph, *_), stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for out, ref in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(out, ref))


@pytest.mark.gpu
def test_another_stream():
    x = _rows(80, 64, 4096, torch.bfloat16).to(DEV)
    want = seco.layer_norm_fwd(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a = seco.layer_norm_fwd(x, stream=side)
    with torch.cuda.stream(side):
        b = seco.layer_norm_fwd(x)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, want)) and all(torch.equal(p, q) for p, q in zip(b, want))


def test_refusals():
    """Before anything is launched (host tensors: the last thing looked at is where they are)."""
    x = torch.zeros(4, 16)
    g, m = torch.ones(16), torch.zeros(4)
    fwd, bwd = seco.layer_norm_fwd, seco.layer_norm_bwd
    for bad in (torch.zeros(()), torch.zeros(4, 0), torch.zeros(16, 4).t()[:, :3], torch.zeros(4, 32)[:, ::2],
                torch.zeros(4, 6, 16)[::1, ::2].transpose(0, 1)):
        with pytest.raises(ValueError):
            fwd(bad)
    with pytest.raises(TypeError):
        fwd(x.half())
    with pytest.raises(TypeError):
        fwd(x.bfloat16(), g.half())
    with pytest.raises(TypeError):
        fwd(x, g.bfloat16())
    for bad in (torch.ones(15), torch.ones(1, 16), torch.ones(32)[::2]):
        with pytest.raises(ValueError, match="gain"):
            fwd(x, bad)
        with pytest.raises(ValueError, match="bias"):
            fwd(x, g, bad)
    with pytest.raises(ValueError, match="bias"):
        fwd(x.bfloat16(), g.bfloat16(), g)
    with pytest.raises(ValueError, match="residual"):
        fwd(x, residual=torch.zeros(4, 15))
    with pytest.raises(ValueError, match="residual"):
        fwd(x, residual=x.bfloat16())
    with pytest.raises(ValueError, match="x_out"):
        fwd(x, x_out=x)
    wide = torch.zeros(256)
    there, other = wide.view(8, 32)[:4, :16], wide.view(4, 64)[:, :16]      # rows from one place on, at two distances
    for kw in (dict(y=other), dict(residual=there, x_out=other)):
        with pytest.raises(ValueError, match="strides"):
            fwd(there, **kw)
    with pytest.raises(ValueError, match="strides"):
        bwd(there, None, torch.zeros(4), torch.zeros(4), x, d_x=other)
    with pytest.raises(ValueError, match="mean"):
        bwd(x, g, m[:3], m, x)
    with pytest.raises(ValueError, match="mean"):
        bwd(x, g, m.double(), m, x)
    with pytest.raises(ValueError, match="d_y"):
        bwd(x, g, m, m, x[:3])
    with pytest.raises(ValueError, match="d_in"):
        bwd(x, g, m, m, x, d_in=x.bfloat16())
    with pytest.raises(TypeError):
        fwd([1.0])
    for call in (lambda: fwd(x), lambda: bwd(x, g, m, m, x)):
        with pytest.raises(ValueError, match="on one GPU"):
            call()


def test_results_that_overlap_are_refused():
    """Two results in one place, rows that another row's workgroup may have overwritten; beside each other they may lie."""
    m, flat = torch.zeros(4), torch.zeros(400)
    buf = flat[:320].view(5, 64)
    x, next_row, beside, across = buf[:4, :16], buf[1:, :16], buf[:4, 16:32], buf[:4, 8:24]
    apart = torch.zeros(4, 16)
    fwd = seco.layer_norm_fwd

    def bwd(x, dy, **kw):
        seco.layer_norm_bwd(x, None, m, m, dy, **kw)
    for call in (lambda: fwd(x, residual=apart, y=beside, x_out=beside), lambda: fwd(x, residual=apart, y=x, x_out=x),
                 lambda: fwd(x, residual=apart, y=beside, x_out=buf[:4, 24:40]), lambda: fwd(x, y=next_row), lambda: fwd(x, y=across),
                 lambda: fwd(apart, residual=x, x_out=next_row), lambda: fwd(flat[:64].view(4, 16), y=flat[4:68].view(4, 16)),
                 lambda: fwd(x[:1].expand(4, 16), y=flat[4:68].view(4, 16)), lambda: bwd(x, apart, d_x=next_row),
                 lambda: bwd(next_row, apart, d_x=x), lambda: bwd(apart, x, d_x=across), lambda: bwd(apart, apart, d_in=x, d_x=next_row),
                 lambda: bwd(flat[8:72].view(4, 16), apart, d_x=flat[:256].view(4, 64)[:, :16])):
        with pytest.raises(ValueError, match="overlaps"):
            call()
    rows3 = torch.zeros(2, 5, 3, 16)
    for call in (lambda: fwd(x, y=beside), lambda: fwd(x, residual=apart, y=beside, x_out=x), lambda: fwd(x, residual=beside, x_out=beside),
                 lambda: fwd(flat[:64].view(4, 16), y=flat[64:128].view(4, 16)), lambda: fwd(buf[:2, :16], y=buf[2:4, :16]),
                 lambda: fwd(flat[:320].view(10, 32)[::2, :16], y=flat[:320].view(10, 32)[1::2, :16]),
                 lambda: fwd(flat[:320].view(5, 4, 16)[:, 0], y=flat[:320].view(10, 2, 16)[:5, 1]),
                 lambda: fwd(rows3[..., 0, :], y=rows3[..., 1, :]), lambda: bwd(x, apart, d_x=x), lambda: bwd(x, beside, d_x=beside),
                 lambda: bwd(x, apart, d_in=beside, d_x=beside), lambda: bwd(x, apart, d_x=beside), lambda: bwd(x, x, d_x=x)):
        with pytest.raises(ValueError, match="on one GPU"):
            call()


def test_status_codes():
    import ctypes as C
    lib = seco.load_library()

    class Desc(C.Structure):
        _fields_ = [(n, C.c_int64) for n in ("rows", "d", "x_stride", "residual_stride", "out_stride", "y_stride")] + [
            ("dtype", C.c_int32), ("gain_dtype", C.c_int32), ("eps", C.c_float)]

    def desc(**kw):
        return Desc(**{**dict(rows=4, d=16, x_stride=16, residual_stride=16, out_stride=16, y_stride=16, dtype=1, gain_dtype=1,
                              eps=1e-5), **kw})
    P = C.c_void_p(0x1000)

    def fwd(d, x=P, r=None, out=None, y=P, mean=P):
        return lib.layer_norm_fwd(C.byref(d) if d else None, x, r, P, P, out, y, mean, P, None)

    def bwd(d, ws=P, n=1 << 20, dg=P, dx=P):
        return lib.layer_norm_bwd(C.byref(d), P, P, P, P, P, None, dx, dg, P, ws, C.c_size_t(n), None)
    assert fwd(None) == -1 and fwd(desc(), x=None) == -1 and fwd(desc(), mean=None) == -1
    assert fwd(desc(), r=P) == -1 and fwd(desc(), out=P) == -1
    assert fwd(desc(dtype=2)) == -4 and fwd(desc(dtype=0)) == -4 and fwd(desc(gain_dtype=3)) == -4
    assert fwd(desc(d=0)) == -2 and fwd(desc(rows=-1)) == -2 and fwd(desc(x_stride=-1)) == -2 and fwd(desc(y_stride=15)) == -2
    assert fwd(desc(eps=-1.0)) == -8 and fwd(desc(eps=float("nan"))) == -8
    assert fwd(desc(d=(1 << 30) + 1)) == -10 and fwd(desc(rows=(1 << 31) + 1)) == -10
    assert fwd(desc(), x=C.c_void_p(0x1001)) == -5 and fwd(desc(), mean=C.c_void_p(0x1002)) == -5
    assert fwd(desc(rows=0)) == 0                                   # nothing to do
    many = desc(rows=2000)                                          # (few rows take no workspace; these addresses are never read)
    assert bwd(many, ws=None) == -6 and bwd(many, n=16) == -6 and bwd(many, ws=C.c_void_p(0x1008)) == -6
    assert bwd(desc(), dx=None) == -1 and bwd(desc(), dg=C.c_void_p(0x1001)) == -5
    lib.layer_norm_workspace_bytes.restype = C.c_size_t
    assert lib.layer_norm_workspace_bytes(C.byref(desc())) == 0 and lib.layer_norm_workspace_bytes(C.byref(desc(rows=1280))) == 0
    assert lib.layer_norm_workspace_bytes(C.byref(desc(rows=0))) == 2 * 16 * 4
    assert lib.layer_norm_workspace_bytes(C.byref(desc(rows=1281))) > 0 and lib.layer_norm_workspace_bytes(C.byref(desc(d=16385))) > 0
    assert lib.layer_norm_workspace_bytes(C.byref(desc(rows=100000))) == 2 * 256 * 16 * 4
    assert lib.layer_norm_workspace_bytes(C.byref(desc(d=-1))) == C.c_size_t(-1).value
