"""Rotary positions with several axes (csrc/rope_axes.hip) against a complex product in 64 bits on the CPU.

Tolerances: angles and products are fp64, so that a result is its exact value rounded to fp32 and then to the storage type: half
a step of that (2^-8 in bf16, 2^-24 in fp32), 2^-24 of the pair's length for the first rounding, and 2^-30 of it for an angle of up to
2^21, which fp64 and the frequency behind it hold to 2^-31."""
import ctypes as C
import math

import pytest
import torch

import paper_2505_16710_amd as seco

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE = 10000.0


def _axis_of(sections, interleaved):
    if not interleaved:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    rounds = [(k, a) for a, n in enumerate(sections) for k in range(n)]        # the k-th pair of axis a comes in round k
    return [a for _, a in sorted(rounds)]


def _angles(positions, sections, base, interleaved, own):
    """[B, rows, pairs] in 64 bits."""
    axis, seen, freq = _axis_of(sections, interleaved), [0] * len(sections), []
    for i, a in enumerate(axis):
        freq.append(base ** -(seen[a] / sections[a] if own else i / len(axis)))
        seen[a] += 1
    return positions.double()[axis].permute(1, 2, 0) * torch.tensor(freq, dtype=torch.float64)


def _turn64(x, angles, sign=1):
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half].double(), x[..., half:].double())
    z = z * torch.polar(torch.ones_like(angles), sign * angles)[:, None]
    return torch.cat((z.real, z.imag), -1)


def _near(got, ref, x, scale=1.0):
    half = x.shape[-1] // 2
    length = torch.hypot(x[..., :half].double(), x[..., half:].double()) * abs(scale)
    step = torch.finfo(got.dtype).eps / 2
    tol = step * ref.abs() + (2.0 ** -24 + 2.0 ** -30) * torch.cat((length, length), -1) * 1.01
    assert ((got.cpu().double() - ref).abs() <= tol).all()


def _rows(seed, *shape, dtype):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _positions(seed, axes, B, rows, most=1 << 20):
    return torch.randint(-most, most, (axes, B, rows), generator=torch.Generator().manual_seed(seed))


# head_dim, sections: pairs in eights and in fours, one axis alone, an axis without pairs, one pair of an axis
SHAPES = [(128, (16, 24, 24)), (128, (64,)), (64, (11, 21)), (80, (20, 20)), (72, (12, 24)), (8, (1, 3)), (24, (4, 4, 4)),
          (256, (32, 32, 31, 33)), (256, (0, 128)), (16, (1, 1, 5, 1)), (200, (50, 50))]


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved,own", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("D,sections", SHAPES)
def test_rotation_and_its_inverse(t, D, sections, interleaved, own):
    dtype, B, H, rows = TYPES[t], 2, 5, 37
    if own and 0 in sections:
        sections = tuple(n for n in sections if n)
    axes = seco.RopeAxes(sections, BASE, interleaved=interleaved, own_frequencies=own)
    x, pos = _rows(D, B, H, rows, D, dtype=dtype), _positions(D + 1, len(sections), B, rows)
    ang = _angles(pos, sections, BASE, interleaved, own)
    out = seco.rope_rotate_axes(x.to(DEV), pos.to(DEV), axes)
    _near(out, _turn64(x, ang), x)
    back = seco.rope_rotate_axes(x.to(DEV), pos.to(DEV), axes, inverse=True)
    _near(back, _turn64(x, ang, -1), x)
    place = x.to(DEV)
    assert seco.rope_rotate_axes(place, pos.to(DEV), axes, out=place) is place and torch.equal(place, out)


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_equal_positions_turn_as_one_axis(t):
    """Text: the same position on every axis is the rotation with one axis, to the rounding of a tie."""
    x = _rows(3, 1, 4, 300, 128, dtype=TYPES[t]).to(DEV)
    pos = torch.arange(5000, 5300, device=DEV).expand(3, 1, 300)
    for interleaved in (False, True):
        got = seco.rope_rotate_axes(x, pos, seco.RopeAxes((16, 24, 24), 500000.0, interleaved=interleaved))
        want = seco.rope_rotate(x, 5000, 500000.0)
        step = torch.finfo(TYPES[t]).eps
        assert ((got.double() - want.double()).abs() <= step * want.double().abs() + 2.0 ** -24).all()
        assert (got != want).double().mean() < 1e-3


def _layer(t, B, Hq, Hkv, C, D, N, seed):
    dtype = TYPES[t]
    mk = lambda k, h: _rows(seed + k, B, C, h, D, dtype=dtype).transpose(1, 2)          # as a projection leaves it  # noqa: E731
    return mk(0, Hq), mk(1, Hkv), mk(2, Hkv), _rows(seed + 3, B, Hkv, N, D, dtype=dtype), _rows(seed + 4, B, Hkv, N, D, dtype=dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("t,B,Hq,Hkv,C,D,q_start", [
    ("bf16", 1, 32, 8, 1, 128, 511), ("bf16", 2, 6, 3, 77, 80, 13), ("bf16", 1, 1, 1, 33, 64, 0), ("bf16", 3, 5, 5, 16, 128, 100),
    ("f32", 2, 9, 3, 50, 40, 7), ("f32", 1, 4, 4, 129, 128, 1), ("bf16", 1, 8, 2, 300, 72, 40),
])
def test_append_and_readout(t, B, Hq, Hkv, C, D, q_start):
    sections = (D // 8, D // 4, D // 8)
    axes = seco.RopeAxes(sections, BASE, interleaved=C % 2 == 1)
    N = q_start + C + 9
    q, kn, vn, kc, vc = _layer(t, B, Hq, Hkv, C, D, N, 10 * D)
    pos = _positions(C, 3, B, C)
    ang = _angles(pos, sections, BASE, C % 2 == 1, False)
    dkc, dvc = kc.to(DEV), vc.to(DEV)
    out = seco.rope_append_axes(q.to(DEV), kn.to(DEV), vn.to(DEV), dkc, dvc, q_start, pos.to(DEV), axes)
    _near(out, _turn64(q, ang), q)
    here = slice(q_start, q_start + C)
    _near(dkc[:, :, here], _turn64(kn, ang), kn)
    assert torch.equal(dvc[:, :, here].cpu(), vn)
    for d, h in ((dkc, kc), (dvc, vc)):                       # the other rows stay
        d[:, :, here] = 0
        h = h.clone()
        h[:, :, here] = 0
        assert torch.equal(d.cpu(), h)
    # without queries, and in place
    d2 = kc.to(DEV), vc.to(DEV)
    assert seco.rope_append_axes(None, kn.to(DEV), vn.to(DEV), *d2, q_start, pos.to(DEV), axes) is None
    qd = q.to(DEV)
    d3 = kc.to(DEV), vc.to(DEV)
    assert seco.rope_append_axes(qd, kn.to(DEV), vn.to(DEV), *d3, q_start, pos.to(DEV), axes, q_out=qd) is qd
    assert torch.equal(qd, out) and torch.equal(d2[0], d3[0]) and torch.equal(d2[1], d3[1])
    # the way back
    gk, gv = _rows(5, B, Hkv, N, D, dtype=torch.float32), _rows(6, B, Hkv, N, D, dtype=torch.float32)
    for scaler in (1.0, 1.75):
        dq, dk, dv = seco.rope_readout_axes(q.to(DEV), gk.to(DEV), gv.to(DEV), q_start, pos.to(DEV), axes, scaler=scaler)
        assert dk.dtype == dv.dtype == dq.dtype == TYPES[t] and dk.shape == dv.shape == (B, Hkv, C, D)
        _near(dq, _turn64(q, ang, -1), q)
        _near(dk, scaler * _turn64(gk[:, :, here], ang, -1), gk[:, :, here], scaler)
        assert torch.equal(dv.cpu(), (gv[:, :, here] * scaler).to(TYPES[t]))
    none, dk2, dv2 = seco.rope_readout_axes(None, gk.to(DEV), gv.to(DEV), q_start, pos.to(DEV), axes, scaler=1.75, dtype=TYPES[t])
    assert none is None and torch.equal(dk2, dk) and torch.equal(dv2, dv)


@pytest.mark.gpu
def test_gradient_of_the_rotation():
    """The inverse is the transpose: <R x, y> = <x, R^T y>, and central differences of <R x, y>."""
    sections = (4, 8, 4)
    axes = seco.RopeAxes(sections, BASE)
    x, y = (_rows(k, 1, 2, 5, 32, dtype=torch.float32) for k in (1, 2))
    pos = _positions(3, 3, 1, 5, most=100)
    ang = _angles(pos, sections, BASE, False, False)
    grad = seco.rope_rotate_axes(y.to(DEV), pos.to(DEV), axes, inverse=True).cpu().double()
    flat, h = x.double().reshape(-1), 1e-4
    for i in range(0, flat.numel(), 11):
        ends = []
        for sign in (1, -1):
            moved = flat.clone()
            moved[i] += sign * h
            ends.append(float((_turn64(moved.view_as(x), ang) * y.double()).sum()))
        assert abs((ends[0] - ends[1]) / (2 * h) - float(grad.reshape(-1)[i])) < 1e-6     # (linear: rounding of fp32 only)


@pytest.mark.gpu
def test_positions_of_any_layout():
    axes = seco.RopeAxes((16, 24, 24), BASE)
    x = _rows(1, 2, 3, 40, 128, dtype=torch.bfloat16).to(DEV)
    pos = _positions(2, 3, 2, 40)
    want = seco.rope_rotate_axes(x, pos.to(DEV), axes)
    assert torch.equal(seco.rope_rotate_axes(x, pos.permute(2, 1, 0).contiguous().permute(2, 1, 0).to(DEV), axes), want)
    wide = torch.zeros(3, 2, 80, dtype=torch.int64)
    wide[..., ::2] = pos
    assert torch.equal(seco.rope_rotate_axes(x, wide.to(DEV)[..., ::2], axes), want)
    one = seco.rope_rotate_axes(x, pos[:, :1].to(DEV), axes)                               # for all batches
    assert torch.equal(one, seco.rope_rotate_axes(x, pos[:, :1].expand(3, 2, 40).contiguous().to(DEV), axes))
    # a tensor whose heads are part of a wider row, and one whose batches are one
    joint = _rows(3, 2, 40, 7 * 128, dtype=torch.bfloat16).to(DEV)
    part = joint[..., 2 * 128:5 * 128].view(2, 40, 3, 128).transpose(1, 2)
    before = joint.clone()
    got = seco.rope_rotate_axes(part, pos.to(DEV), axes, out=part)
    assert torch.equal(got, seco.rope_rotate_axes(before[..., 2 * 128:5 * 128].reshape(2, 40, 3, 128).transpose(1, 2), pos.to(DEV), axes))
    assert torch.equal(joint[..., :2 * 128], before[..., :2 * 128]) and torch.equal(joint[..., 5 * 128:], before[..., 5 * 128:])
    single = x[:1].expand(2, 3, 40, 128)
    assert torch.equal(seco.rope_rotate_axes(single, pos.to(DEV), axes)[1], seco.rope_rotate_axes(x[:1], pos[:, 1:].to(DEV), axes)[0])


@pytest.mark.gpu
def test_far_positions_and_far_rows():
    """Positions up to 2^39 (fp64 holds their angles to 2^-13: 2^-12 of a pair's length); cache rows behind 2^31 elements."""
    axes = seco.RopeAxes((32, 32), BASE)
    x = _rows(1, 1, 2, 9, 128, dtype=torch.float32)
    pos = _positions(2, 2, 1, 9, most=1 << 39)
    got = seco.rope_rotate_axes(x.to(DEV), pos.to(DEV), axes).cpu().double()
    half = torch.hypot(x[..., :64].double(), x[..., 64:].double())
    assert ((got - _turn64(x, _angles(pos, (32, 32), BASE, False, False))).abs() <= 2.0 ** -12 * torch.cat((half, half), -1)).all()
    N, row = (1 << 23) + 40, (1 << 23) + 3                    # 2 heads x 2^23 rows x 128 = 2^31 elements
    kc, vc = (torch.zeros(1, 2, N, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    kn = _rows(3, 1, 2, 20, 128, dtype=torch.bfloat16).to(DEV)
    p20 = _positions(4, 2, 1, 20).to(DEV)
    seco.rope_append_axes(None, kn, kn, kc, vc, row, p20, axes)
    assert torch.equal(kc[:, :, row:row + 20], seco.rope_rotate_axes(kn, p20, axes)) and torch.equal(vc[:, :, row:row + 20], kn)
    assert not kc[:, :, :row].any() and not kc[:, :, row + 20:].any() and not vc[:, :, row + 20:].any()


@pytest.mark.gpu
def test_more_rows_than_a_grid_holds_along_y():
    """8 rows of head_dim 256 to a workgroup, 65535 of these along a dimension of the grid: the rows behind them, two batches."""
    rows = 8 * 65535 + 11
    axes = seco.RopeAxes((64, 64), BASE)
    x = torch.zeros(2, 1, rows, 256, dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros(2, 1, rows, dtype=torch.int64, device=DEV)
    x[:, :, -20:] = _rows(1, 2, 1, 20, 256, dtype=torch.bfloat16).to(DEV)
    pos[:, :, -20:] = _positions(2, 2, 1, 20).to(DEV)
    got = seco.rope_rotate_axes(x, pos, axes)
    assert torch.equal(got[:, :, -20:], seco.rope_rotate_axes(x[:, :, -20:], pos[:, :, -20:], axes)) and not got[:, :, :-20].any()


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_pair():
    axes = seco.RopeAxes((32, 32), BASE)
    x = _rows(1, 1, 3, 20, 128, dtype=torch.bfloat16)
    pos = _positions(2, 2, 1, 20).to(DEV)
    clean = seco.rope_rotate_axes(x.to(DEV), pos, axes).cpu()
    x[0, 1, 7, 5], x[0, 2, 9, 70] = float("inf"), float("nan")
    got = seco.rope_rotate_axes(x.to(DEV), pos, axes).cpu()
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[0, 1, 7, [5, 69]] = bad[0, 2, 9, [6, 70]] = True
    assert torch.equal(got[~bad], clean[~bad]) and not torch.isfinite(got[bad]).any()


@pytest.mark.gpu
def test_no_rows():
    axes = seco.RopeAxes((32, 32), BASE)
    x = torch.empty(2, 3, 0, 128, dtype=torch.bfloat16, device=DEV)
    pos = torch.empty(2, 2, 0, dtype=torch.int64, device=DEV)
    assert seco.rope_rotate_axes(x, pos, axes).shape == x.shape
    kc = torch.ones(2, 3, 10, 128, dtype=torch.bfloat16, device=DEV)
    assert seco.rope_append_axes(x, x, x, kc, kc.clone(), 4, pos, axes).shape == x.shape and (kc == 1).all()
    g = torch.ones(2, 3, 10, 128, device=DEV)
    assert all(t.shape == x.shape for t in seco.rope_readout_axes(x, g, g.clone(), 4, pos, axes))


@pytest.mark.gpu
def test_captured_and_replayed():
    axes = seco.RopeAxes((16, 24, 24), BASE)
    q, kn, vn, kc, vc = (t.to(DEV) for t in _layer("bf16", 1, 8, 2, 64, 128, 200, 1))
    pos = _positions(2, 3, 1, 64).to(DEV)
    gk, gv = torch.randn(1, 2, 200, 128, device=DEV), torch.randn(1, 2, 200, 128, device=DEV)

    def both():
        out = seco.rope_append_axes(q, kn, vn, kc, vc, 30, pos, axes)
        return (out, *seco.rope_readout_axes(out, gk, gv, 30, pos, axes))
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(3):
        pos.random_(-1000, 100000, generator=torch.Generator(device=DEV).manual_seed(k))
        kc.zero_()
        graph.replay()
        torch.cuda.synchronize()
        cache = kc.clone()
        kc.zero_()
        assert all(torch.equal(a, b) for a, b in zip(out, both())) and torch.equal(cache, kc)


@pytest.mark.gpu
def test_another_stream():
    axes = seco.RopeAxes((64,), BASE)
    x = _rows(1, 1, 8, 500, 128, dtype=torch.bfloat16).to(DEV)
    pos = _positions(2, 1, 1, 500).to(DEV)
    want = seco.rope_rotate_axes(x, pos, axes)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = seco.rope_rotate_axes(x, pos, axes, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


# ---- refusals (no GPU)

def test_refusals():
    """Before anything is launched (host tensors: the last thing looked at is where they are)."""
    A = seco.RopeAxes
    for args in (((),), ((1, 2, 3, 4, 6),), ((-4, 68),), ((1, 2),), ((128, 4),)):
        with pytest.raises(ValueError):
            A(*args, BASE)
    for base in (1.0, -2.0, float("inf"), float("nan")):
        with pytest.raises(ValueError):
            A((64,), base)
    axes, pos = A((32, 32), BASE), torch.zeros(2, 1, 10, dtype=torch.int64)
    x, c, g = torch.zeros(1, 2, 10, 128), torch.zeros(1, 2, 50, 128), torch.zeros(1, 2, 50, 128)

    def rot(x=x, pos=pos, axes=axes, **kw):
        seco.rope_rotate_axes(x, pos, axes, **kw)

    def app(q=x, k=x, v=x, kc=c, vc=c, row=0, pos=pos, axes=axes, **kw):
        seco.rope_append_axes(q, k, v, kc, vc, row, pos, axes, **kw)

    def rea(q=x, gk=g, gv=g, row=0, pos=pos, axes=axes, **kw):
        seco.rope_readout_axes(q, gk, gv, row, pos, axes, **kw)
    for bad in (x[0], x[..., :120], torch.zeros(1, 2, 128, 10).transpose(2, 3)):
        with pytest.raises(ValueError):
            rot(bad)
    with pytest.raises(ValueError, match="strides"):
        rot(x, out=x.view(1, 10, 2, 128).transpose(1, 2))          # in the place of x, its rows in another order
    with pytest.raises(ValueError, match="strides"):
        app(q_out=x.view(1, 10, 2, 128).transpose(1, 2))
    with pytest.raises(ValueError, match="strides"):
        rea(dq_out=x.view(1, 10, 2, 128).transpose(1, 2))
    with pytest.raises(ValueError, match="at least one head"):
        app(k=x[:, :0], v=x[:, :0], kc=c[:, :0], vc=c[:, :0])
    with pytest.raises(ValueError, match="at least one head"):
        rea(gk=g[:, :0], gv=g[:, :0])
    for row in (-1, 41, 2 ** 63 - 1, 2 ** 63 - 5):
        for call in (app, rea):
            with pytest.raises(ValueError, match="holds rows"):
                call(row=row)
    for bad in (pos[:1], pos[..., :9], pos.int(), pos[0], torch.zeros(2, 3, 10, dtype=torch.int64)):
        for call in (rot, app):
            with pytest.raises(ValueError):
                call(pos=bad)
    for kw in (dict(out=x[:, :1]), dict(out=x.bfloat16()), dict(out=x[:, :1].expand(1, 2, 10, 128)), dict(axes=A((64, 64), BASE))):
        with pytest.raises(ValueError):
            rot(**kw)
    for kw in (dict(row=-1), dict(row=41), dict(v=x[:, :1]), dict(kc=c.bfloat16(), vc=c.bfloat16()), dict(kc=c[:, :1], vc=c[:, :1]),
               dict(vc=torch.zeros(1, 2, 60, 128)), dict(q=x[..., :64]), dict(q=None, q_out=x), dict(q_out=x[:, :1]),
               dict(kc=c[:, :, :1].expand(1, 2, 50, 128), vc=c[:, :, :1].expand(1, 2, 50, 128))):
        with pytest.raises(ValueError):
            app(**kw)
    for kw in (dict(row=-1), dict(row=41), dict(gk=g.bfloat16(), gv=g.bfloat16()), dict(gv=g[:, :1]), dict(q=None), dict(d_k=x),
               dict(d_k=x[:, :1], d_v=x[:, :1]), dict(dq_out=x[:, :1]), dict(q=None, dq_out=x, dtype=torch.float32)):
        with pytest.raises(ValueError):
            rea(**kw)
    with pytest.raises(TypeError):
        rea(q=None, dtype=torch.float16)
    with pytest.raises(TypeError):
        rot(x.half())
    for call in (rot, app, rea):
        with pytest.raises(ValueError, match="on one GPU"):
            call()


def test_results_that_overlap_are_refused():
    """Layouts drawn at random over one buffer, compared element by element: a result that shares some with the input is refused
    unless it lies in its place, and no other one is."""
    axes, room = seco.RopeAxes((2, 2), BASE), torch.zeros(4000)
    g = torch.Generator().manual_seed(5)

    def draw(n):
        return int(torch.randint(0, n, (1,), generator=g))
    numbers, seen = torch.arange(4000), {True: 0, False: 0}
    for _ in range(600):
        B, H, C = 1 + draw(3), 1 + draw(3), 1 + draw(4)
        pos, pair = torch.zeros(2, 1, C, dtype=torch.int64), []
        strides = None
        for _ in range(2):
            order = [(0, 1, 2), (0, 2, 1), (1, 0, 2), (2, 0, 1)][draw(4)]           # from the outermost dimension in
            if strides is None or draw(3) == 0:
                strides, step = [0, 0, 0, 1], 8 + 8 * draw(3) * draw(2)
                for i in reversed(order):
                    strides[i] = step
                    step *= (B, H, C)[i] + draw(2) * draw(3)
            pair.append((strides, 8 * draw(40) if draw(2) else draw(60)))
        if max(st[0] * B + st[1] * H + st[2] * C + off + 8 for st, off in pair) > 4000:
            continue
        x, out = (torch.as_strided(room, (B, H, C, 8), st, off) for st, off in pair)
        used = [set(torch.as_strided(numbers, (B, H, C, 8), st, off).flatten().tolist()) for st, off in pair]
        if pair[0][1] == pair[1][1]:
            same = all(n == 1 or a == b for n, a, b in zip((B, H, C), pair[0][0], pair[1][0]))
            want = "on one GPU" if same else "strides"
        else:
            want = "overlaps" if used[0] & used[1] else "on one GPU"
            seen[want == "overlaps"] += 1
        with pytest.raises(ValueError, match=want):
            seco.rope_rotate_axes(x, pos, axes, out=out)
    assert min(seen.values()) > 100
    joint = torch.zeros(1, 12, 6 * 8)
    q, k, v = (joint[..., a:b].unflatten(2, (-1, 8)).transpose(1, 2) for a, b in ((0, 16), (16, 32), (32, 48)))
    cache = torch.zeros(1, 2, 20, 8)
    pos = torch.zeros(2, 1, 10, dtype=torch.int64)
    q, k, v = (t[:, :, :10] for t in (q, k, v))
    for bad in (k, v, joint[:, 2:, :16].unflatten(2, (-1, 8)).transpose(1, 2), joint[:, :10, 8:24].unflatten(2, (-1, 8)).transpose(1, 2)):
        with pytest.raises(ValueError, match="overlaps"):
            seco.rope_append_axes(q, k, v, cache, cache.clone(), 4, pos, axes, q_out=bad)
    for kw in (dict(k=k[..., ::2]), dict(v=torch.zeros(1, 2, 8, 10).transpose(2, 3)), dict(vc=cache.transpose(2, 3).contiguous().transpose(2, 3)),
               dict(vc=cache[:, :, :1].expand(1, 2, 20, 8))):
        with pytest.raises(ValueError, match="head_dim|expanded"):
            seco.rope_append_axes(None, kw.get("k", k), kw.get("v", v), cache, kw.get("vc", cache.clone()), 4, pos, axes)
    with pytest.raises(ValueError, match="overlaps"):
        seco.rope_readout_axes(q, cache, cache, 4, pos, axes, dq_out=joint[:, 2:, :16].unflatten(2, (-1, 8)).transpose(1, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("t,C", [("bf16", 10), ("f32", 1)])
def test_keys_and_values_in_layouts_of_their_own(t, C):
    """Keys that a norm has made contiguous beside values in the joint projection; caches, gradient buffers and results likewise."""
    axes, B, Hq, H, D, N, dtype = seco.RopeAxes((32, 32), BASE), 2, 4, 2, 128, 40, TYPES[t]
    joint = _rows(1, B, C, (Hq + 2 * H) * D, dtype=dtype).to(DEV)
    q, k, v = (x.unflatten(2, (-1, D)).transpose(1, 2) for x in joint.split((Hq * D, H * D, H * D), 2))
    pos = _positions(3, 2, B, C).to(DEV)

    def caches(kind):
        a = torch.zeros(B, H, N, D, dtype=dtype, device=DEV)
        return a, (torch.zeros(B, N, H, D, dtype=dtype, device=DEV).transpose(1, 2) if kind else a.clone())
    want = caches(0)
    out = seco.rope_append_axes(q, k, v, *want, 7, pos, axes)
    for kn, vn, kind in ((k.contiguous(), v, 0), (k, v.contiguous(), 0), (k, v, 1), (k.contiguous(), v, 1)):
        got = caches(kind)
        assert torch.equal(seco.rope_append_axes(q, kn, vn, *got, 7, pos, axes), out)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    gk, gv = (torch.randn(B, H, N, D, device=DEV) for _ in range(2))
    want = seco.rope_readout_axes(q, gk, gv, 7, pos, axes, scaler=1.5)
    rows = gv.transpose(1, 2).contiguous().transpose(1, 2)
    for ga, gb, kw in ((gk, rows, {}), (gk, gv, dict(d_k=torch.empty_like(k.contiguous()), d_v=v)), (gk, rows, dict(d_k=k, d_v=v))):
        got = seco.rope_readout_axes(q, ga, gb, 7, pos, axes, scaler=1.5, **kw)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    # what the values' own launch would refuse is refused in front of both
    flat = torch.zeros(B * H * C * D + 8, dtype=dtype, device=DEV)
    for odd in (flat[1:1 + B * H * C * D].view(B, H, C, D), torch.zeros(B, H, C, D + 1, dtype=dtype, device=DEV)[..., :D]):
        got = caches(1)
        with pytest.raises(seco.SecoError):
            seco.rope_append_axes(q, k, odd, *got, 7, pos, axes)
        assert not got[0].any() and not got[1].any()


@pytest.mark.gpu
def test_caches_and_results_that_share_memory():
    """Keys and values in one tensor, halves of it or rows in turn; a projection that lies in the cache already; one place for both
    is refused."""
    axes, B, H, C, D, N = seco.RopeAxes((32, 32), BASE), 2, 3, 10, 128, 40
    kn, vn = (_rows(k, B, H, C, D, dtype=torch.bfloat16).to(DEV) for k in (1, 2))
    pos = _positions(3, 2, B, C).to(DEV)
    kc, vc = (torch.zeros(B, H, N, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    seco.rope_append_axes(None, kn, vn, kc, vc, 7, pos, axes)
    for shape, at in (((2, B, H, N, D), 0), ((B, 2, H, N, D), 1), ((B, H, 2, N, D), 2), ((B, H, N, 2, D), 3), ((B, H, N, D, 2), None)):
        both = torch.zeros(*shape, dtype=torch.bfloat16, device=DEV)
        if at is None:                                       # (elements in turn: no head_dim is contiguous)
            with pytest.raises(ValueError, match="head_dim"):
                seco.rope_append_axes(None, kn, vn, both[..., 0], both[..., 1], 7, pos, axes)
            continue
        k, v = both.unbind(at)
        seco.rope_append_axes(None, kn, vn, k, v, 7, pos, axes)
        assert torch.equal(k, kc) and torch.equal(v, vc)
    there = [torch.zeros(B, H, N, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for t, new in zip(there, (kn, vn)):
        t[:, :, 7:17] = new
    seco.rope_append_axes(None, there[0][:, :, 7:17], there[1][:, :, 7:17], *there, 7, pos, axes)
    assert torch.equal(there[0], kc) and torch.equal(there[1], vc)
    for bad in ((kc, kc), (kc[:, :2], kc[:, 1:])):
        with pytest.raises(ValueError, match="overlaps"):
            seco.rope_append_axes(None, kn[:, :bad[0].shape[1]], vn[:, :bad[0].shape[1]], *bad, 7, pos, axes)
    spare = torch.zeros_like(kc)[:, :, :C]
    for args in ((kc[:, :, 8:18], spare), (vc[:, :, 7:17], spare), (spare, kc[:, :, 16:26])):
        with pytest.raises(ValueError, match="overlaps"):
            seco.rope_append_axes(None, *args, kc, vc, 7, pos, axes)
    with pytest.raises(ValueError, match="overlaps"):
        seco.rope_append_axes(kc[:, :, 7:17], kn, vn, kc, vc, 7, pos, axes)
    with pytest.raises(ValueError, match="overlaps"):
        seco.rope_append_axes(kn, kn, vn, kc, vc, 7, pos, axes, q_out=kc[:, :, 3:13])
    g = torch.randn(B, H, N, D, device=DEV)
    for kw in (dict(d_k=kn, d_v=kn), dict(d_k=kn, d_v=vn, dq_out=kn)):
        with pytest.raises(ValueError, match="overlaps"):
            seco.rope_readout_axes(kn.clone(), g, g, 7, pos, axes, **kw)
    with pytest.raises(ValueError, match="overlaps"):
        seco.rope_readout_axes(None, g, g, 7, pos, axes, d_k=g[:, :, 8:18], d_v=torch.zeros_like(g)[:, :, :C])
    want = seco.rope_readout_axes(None, g, 2 * g, 7, pos, axes, dtype=torch.float32)
    gk, gv = g.clone(), 2 * g
    seco.rope_readout_axes(None, gk, gv, 7, pos, axes, d_k=gk[:, :, 7:17], d_v=gv[:, :, 7:17])
    assert torch.equal(gk[:, :, 7:17], want[1]) and torch.equal(gv[:, :, 7:17], want[2]) and torch.equal(gk[:, :, 17:], g[:, :, 17:])


def test_the_base_is_fp32():
    for base in (1.00000001, 1e39, 1.0, float("nan")):
        with pytest.raises(ValueError, match="fp32"):
            seco.RopeAxes((64,), base)
    assert seco.RopeAxes((64,), 500000).base == 500000.0
    assert seco.RopeAxes((64,), 1e6 / 3).base == float(torch.tensor(1e6 / 3)) and seco.RopeAxes((64,), 3.4028234663852886e38).base < math.inf


def test_status_codes():
    lib = seco.load_library()
    from paper_2505_16710_amd.binding import SecoDesc

    class Axes(C.Structure):
        _fields_ = [("n_axes", C.c_int32), ("interleaved", C.c_int32), ("own", C.c_int32), ("base", C.c_float), ("sections", C.c_int32 * 4)]
    P = C.c_void_p(0x1000)
    three = (C.c_int64 * 3)

    def desc(**kw):
        d = SecoDesc()
        d.batch, d.n_q_heads, d.n_kv_heads, d.head_dim, d.chunk_len, d.dtype = 1, 4, 2, 128, 16, 1
        for name in ("q_stride", "o_stride", "kv_stride", "g_stride"):
            setattr(d, name, three(4 * 512 * 128, 512 * 128, 128))
        for k, v in kw.items():
            setattr(d, k, v)
        return d

    def axes(n=2, base=1e4, sections=(32, 32, 0, 0)):
        return Axes(n, 0, 0, base, (C.c_int32 * 4)(*sections))

    def rot(d=None, a=None, x=P, out=P, pos=P, ps=(0, 0, 1), heads=4):
        return lib.rope_rotate_axes(C.byref(d or desc()), C.byref(a or axes()), heads, x, out, pos, three(*ps) if ps else None, 0, None)

    def app(d, q=P, k=P, v=P, kc=P):
        return lib.rope_append_axes(C.byref(d), C.byref(axes()), q, P, k, v, kc, P, P, three(0, 0, 1), None)

    def rea(d, scaler, gk=P):
        return lib.rope_readout_axes(C.byref(d), C.byref(axes()), P, P, gk, P, P, P, C.c_float(scaler), P, three(0, 0, 1), None)
    assert rot(x=None) == -1 and rot(pos=None) == -1 and rot(ps=None) == -1
    assert rot(desc(dtype=3)) == -4 and rot(desc(batch=0)) == -2 and rot(desc(chunk_len=0)) == -2 and rot(desc(q_start=-1)) == -2
    assert rot(desc(head_dim=100)) == -3 and rot(desc(head_dim=264)) == -3
    assert rot(a=axes(n=0)) == -8 and rot(a=axes(n=5)) == -8 and rot(a=axes(base=1.0)) == -8 and rot(a=axes(base=math.nan)) == -8
    assert rot(a=axes(sections=(32, 31, 0, 0))) == -8 and rot(a=axes(sections=(-1, 65, 0, 0))) == -8
    assert rot(pos=C.c_void_p(0x1004)) == -5 and rot(x=C.c_void_p(0x1008)) == -5 and rot(ps=(0, -1, 1)) == -2
    assert rot(desc(q_stride=three(0, 0, 132))) == -5 and rot(desc(q_stride=three(0, 0, 64))) == -5 and rot(desc(o_stride=three(0, 4, 128))) == -5
    assert rot(heads=0) == -2 and rot(heads=70000) == -10 and rot(desc(batch=70000)) == -10 and rot(desc(chunk_len=(1 << 27) + 1)) == -10
    assert app(desc(q_start=1 << 30)) == -10 and app(desc(), k=None) == -1 and app(desc(), kc=None) == -1
    assert app(desc(kv_stride=three(0, 0, 130))) == -5
    assert rea(desc(), math.inf) == -8 and rea(desc(), 1.0, gk=None) == -1
    assert rea(desc(g_stride=three(0, 0, 130)), 1.0) == -5                               # (fp32 rows: 4 elements to 16 bytes)
