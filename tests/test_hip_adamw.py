"""The AdamW update (csrc/adamw.hip, optimizer.py) against its formulas in 64 bits on the CPU, step by step: each step is
computed from the state that the GPU left after the one before.

Tolerances, U = 2^-24 (half a step of fp32): m and v are a product, a product and a fused addition with factors that are
rounded to fp32 once: 4 U of the magnitudes added.  The update's factors (rate, reciprocal root of the correction: U each),
its root and its reciprocal (a step, 2 U, each) and products: 16 U, with m's error in it, of the update's magnitude; p: that and 4 U of
itself, and half a step of bf16 where it is stored so.  States of 8 bits: half a step of e4m3, 2^-4 of the value or 2^-10
of the unit, (1 + 2^-12) for what the value in front was off by; the unit is the largest magnitude / 448 within 8 U."""
import ctypes as C

import pytest
import torch

import paper_2505_16710_amd as seco
from paper_2505_16710_amd.optimizer import AdamW

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BETAS, EPS = (0.9, 0.95), 1e-8


def _state(sizes, p_type, g_type, master, bits, seed=0, off=0):
    """Lists of tensors on the GPU, each between guard elements, `off` elements behind an aligned place."""
    g = torch.Generator().manual_seed(seed)
    s = {"p": [], "g": [], "m": [], "v": [], "masters": [] if master else None, "ms": [] if bits == 8 else None,
         "vs": [] if bits == 8 else None, "guards": []}

    def place(x, dtype):
        room = torch.full((x.numel() + off + 300,), 77.0, device=DEV).to(dtype)
        t = room[off:off + x.numel()]
        s["guards"].append((room, off, x.numel(), float(room[-1])))
        t.copy_(x.to(dtype))
        return t
    for n in sizes:
        w = torch.randn(n, generator=g) * 0.05
        s["p"].append(place(w, p_type))
        s["g"].append(place(torch.randn(n, generator=g) * 1e-3, g_type))
        state = torch.float8_e4m3fn if bits == 8 else torch.float32
        for k in ("m", "v"):
            s[k].append(place(torch.zeros(n), state))
        if master:
            s["masters"].append(place(w, torch.float32))
        if bits == 8:
            for k in ("ms", "vs"):
                s[k].append(place(torch.zeros(-(-n // 256)), torch.float32))
    s["step"] = torch.zeros(2, dtype=torch.int64, device=DEV)
    return s


def _go(s, lr=1e-3, wd=0.1, scale=None, **kw):
    seco.adamw_step(s["p"], s["g"], s["m"], s["v"], s["step"], lr, betas=BETAS, eps=EPS, weight_decay=wd, masters=s["masters"],
                    m_scales=s["ms"], v_scales=s["vs"], grad_scale=scale, **kw)


def _host(s):
    return {k: [t.cpu() for t in s[k]] if isinstance(s[k], list) else s[k] for k in ("p", "g", "m", "v", "masters", "ms", "vs")}


def _unpack(codes, scale):
    n = codes.numel()
    return codes.double() * scale.double().repeat_interleave(256)[:n]


def _check(before, after, i, t, lr, wd, scale=1.0):
    """Tensor i: `after` is one step from `before`, step number t."""
    eight = before["ms"] is not None
    b, a = ({k: None if x[k] is None else x[k][i] for k in x} for x in (before, after))
    m, v = (_unpack(b["m"], b["ms"]), _unpack(b["v"], b["vs"]) ** 2) if eight else (b["m"].double(), b["v"].double())
    w = (b["p"] if b["masters"] is None else b["masters"]).double()
    g = b["g"].double() * scale
    m_size = BETAS[0] * m.abs() + (1 - BETAS[0]) * g.abs()
    m, v = BETAS[0] * m + (1 - BETAS[0]) * g, BETAS[1] * v + (1 - BETAS[1]) * g * g
    den = v.sqrt() / (1 - BETAS[1] ** t) ** 0.5 + EPS
    rate = lr / (1 - BETAS[0] ** t)
    p = w * (1 - lr * wd) - rate * m / den
    tol = 4 * U * w.abs() + 16 * U * rate * m_size / den
    if b["masters"] is not None:
        assert ((a["masters"].double() - p).abs() <= tol).all()
        assert torch.equal(a["p"], a["masters"].to(a["p"].dtype))
    else:
        half = torch.finfo(a["p"].dtype).eps / 2
        assert ((a["p"].double() - p).abs() <= tol * (1 + half) + half * p.abs()).all()
    if not eight:
        assert ((a["m"].double() - m).abs() <= 4 * U * m_size).all()
        assert ((a["v"].double() - v).abs() <= 6 * U * v).all()
        return
    for name, x, size in (("m", m, m_size), ("v", v.sqrt(), v.sqrt())):
        n = x.numel()
        blocks = torch.zeros(-(-n // 256) * 256, dtype=torch.float64)
        blocks[:n] = x.abs()
        unit = (blocks.view(-1, 256).amax(1) / 448).clamp_min(2.0 ** -126)
        sizes = torch.zeros_like(blocks)
        sizes[:n] = size
        got = a[name + "s"].double()
        assert ((got - unit).abs() <= 8 * U * (unit + sizes.view(-1, 256).amax(1) / 448)).all()
        wide = got.repeat_interleave(256)[:n]
        off = (2.0 ** -4 * x.abs()).maximum(2.0 ** -10 * wide) * (1 + 2.0 ** -12) + 8 * U * size
        code = a[name].double()
        if name == "v":
            small = (x > 0) & (x < 2.0 ** -9 * wide)
            assert (code[x > 0] >= 2.0 ** -9).all() and (code[small] == 2.0 ** -9).all()
            off = torch.where(small, wide, off)
        assert ((code * wide - x).abs() <= off).all()


def _guards(s):
    return all((room[:off].float() == value).all() and (room[off + n:].float() == value).all() for room, off, n, value in s["guards"])


SIZES = [1, 3, 4, 255, 256, 257, 511, 1000, 1024, 4095, 4096, 4097, 5 * 4096, 3 * 4096 + 770, 30001]
KINDS = [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "f32", False), ("bf16", "bf16", False), ("bf16", "f32", True),
         ("bf16", "bf16", True)]


@pytest.mark.gpu
@pytest.mark.parametrize("off", [0, 3])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p,g,master", KINDS)
def test_steps(p, g, master, bits, off):
    s = _state(SIZES, TYPES[p], TYPES[g], master, bits, off=off)
    for t in range(1, 5):
        before = _host(s)
        wd = [0.1 * (i % 3) for i in range(len(SIZES))]
        _go(s, wd=wd)
        after = _host(s)
        assert s["step"].tolist() == [t, 0] and _guards(s)
        for i in range(len(SIZES)):
            _check(before, after, i, t, 1e-3, wd[i])
        for x in s["g"]:
            x.normal_(std=1e-3 * 3.0 ** t)


@pytest.mark.gpu
def test_many_tensors_of_several_kinds():
    """More than two launches hold (48 each), kinds in turn, empty tensors among them; scaled gradients, lr on the GPU."""
    sizes = [(7 * i) % 600 for i in range(130)]
    parts = [_state(sizes, TYPES[p], TYPES[g], master, 32, seed=k) for k, (p, g, master) in enumerate(KINDS)]
    s = {k: [x for group in zip(*(q[k] for q in parts)) for x in group] for k in ("p", "g", "m", "v")}
    s["masters"] = [x for group in zip(*(q["masters"] or [None] * len(sizes) for q in parts)) for x in group]
    s["ms"] = s["vs"] = None
    s["step"] = torch.tensor([41, 0], device=DEV)

    def host():
        h = {k: [None if t is None else t.cpu() for t in s[k]] for k in ("p", "g", "m", "v", "masters")}
        return {**h, "ms": None, "vs": None}
    before = host()
    _go(s, lr=torch.tensor([2e-3], device=DEV), scale=torch.tensor(0.25, device=DEV))
    after = host()
    assert s["step"].tolist() == [42, 0] and all(_guards(q) for q in parts)
    for i in range(len(s["p"])):
        if s["p"][i].numel():
            _check(before, after, i, 42, float(torch.tensor(2e-3)), 0.1, 0.25)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_the_same_every_time_and_late_steps(bits):
    """Two runs give the same bits; step numbers up to 2^40 (the corrections are 1 there)."""
    runs = []
    for _ in range(2):
        s = _state([70001, 513], torch.bfloat16, torch.bfloat16, True, bits)
        for t in (0, 5, 999999, 1 << 40):
            s["step"][0] = t
            before = _host(s)
            _go(s)
            for i in range(2):
                _check(before, _host(s), i, t + 1, 1e-3, 0.1)
        assert s["step"].tolist() == [(1 << 40) + 1, 0]
        runs.append(_host(s))
    for k in ("p", "m", "v", "masters", "ms", "vs"):
        if runs[0][k] is not None:
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(runs[0][k], runs[1][k]))


@pytest.mark.gpu
def test_no_tensors_counts_the_step():
    step = torch.zeros(2, dtype=torch.int64, device=DEV)
    for _ in range(3):
        seco.adamw_step([], [], [], [], step, 1e-3)
    assert step.tolist() == [3, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_finite(bits):
    """The element's parameter is NaN; every other one, in its block too, is what it is without it."""
    n = 3000
    a, b = (_state([n], torch.float32, torch.float32, False, bits, seed=4) for _ in range(2))
    at = torch.tensor([0, 300, 700, n - 1])
    for s in (a, b):
        s["g"][0][at.to(DEV)] = 0.0                           # (so that a block's largest magnitude is another's)
        _go(s)
    a["g"][0][at.to(DEV)] = torch.tensor([float("nan"), float("inf"), float("-inf"), float("nan")], device=DEV)
    for s in (a, b):
        _go(s)
    rest = torch.ones(n, dtype=torch.bool)
    rest[at] = False
    pa, pb = a["p"][0].cpu(), b["p"][0].cpu()
    assert torch.isnan(pa[at]).all() and torch.equal(pa[rest], pb[rest])
    ma, mb = a["m"][0].float().cpu(), b["m"][0].float().cpu()
    va, vb = a["v"][0].float().cpu(), b["v"][0].float().cpu()
    assert torch.equal(ma[rest], mb[rest]) and torch.equal(va[rest], vb[rest])
    if bits == 8:
        assert torch.equal(a["ms"][0], b["ms"][0]) and torch.equal(a["vs"][0], b["vs"][0])


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("huge", [1e20, -3e38, float("inf"), float("nan")])
def test_squares_that_overflow(huge, bits):
    """An infinite v stays that in 32 bits, and is NaN in 8: never a finite code, beside which the next step would be unbounded."""
    s, n, at = _state([600], torch.float32, torch.float32, False, bits, seed=6), 600, 300
    s["g"][0][at] = huge
    w = s["p"][0].clone()
    _go(s, wd=0.0)
    rest = torch.arange(n, device=DEV) != at
    m, v = s["m"][0].float()[at], s["v"][0].float()[at]
    finite = abs(huge) < 1e39
    if bits == 32:
        assert torch.isinf(v) if huge == huge else torch.isnan(v)
    else:
        assert torch.isnan(v) and torch.isfinite(s["vs"][0]).all() and (finite or torch.isnan(m))
    assert s["p"][0][at] == w[at] if finite else torch.isnan(s["p"][0][at])
    assert ((s["p"][0] - w)[rest].abs() < 1.01e-3).all()
    s["g"][0].zero_()
    for _ in range(3):
        before = s["p"][0].clone()
        _go(s, wd=0.0)
        if finite and bits == 32:
            assert s["p"][0][at] == w[at]
        else:
            assert torch.isnan(s["p"][0][at])
        assert ((s["p"][0] - before)[rest].abs() < 1.5e-3).all()      # (m / sqrt(v) of one gradient falls from 1 by less than its sum)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_whose_squares_are_subnormal(bits):
    """Gradients of 1e-21, eps = 0: the first step's update is lr, whatever they are, and a code of sqrt(v) is that of its root.  v is a
    multiple of 2^-149, half a step of that off: (g^2)(1 - beta2) of 1e-21 by 2^-149 / 2 / 5e-44 = 0.014, its root by 0.007."""
    s = _state([3000], torch.float32, torch.float32, False, bits, seed=8)
    g = s["g"][0]
    g.copy_(g.sign() * (1 + torch.rand(3000, generator=torch.Generator().manual_seed(1)).to(DEV)) * 1e-21)
    w = s["p"][0].clone()
    seco.adamw_step(s["p"], s["g"], s["m"], s["v"], s["step"], 1e-3, betas=BETAS, eps=0.0, weight_decay=0.0, m_scales=s["ms"], v_scales=s["vs"])
    moved = (w - s["p"][0]).cpu().double() / 1e-3 * g.sign().cpu()
    assert ((moved - 1).abs() < 0.008 + 4 * U * 0.2 / 1e-3).all()               # (and p's own rounding)
    if bits == 8:
        # half a step of e4m3 and a unit above 2^-126, in which 1e-21 has a code of its own
        r = _unpack(s["v"][0].cpu(), s["vs"][0].cpu())
        want = g.cpu().double().abs() * (1 - BETAS[1]) ** 0.5
        assert ((r / want - 1).abs() < 2.0 ** -4 + 0.008).all()


@pytest.mark.gpu
@pytest.mark.parametrize("low,high", [(-8, 4), (-22, -16), (14, 18)])
def test_units_and_codes_are_the_formulas(low, high):
    """With betas of zero m is g and sqrt(v) is sqrt(g^2): units and codes are, bit by bit, those of fp32 operations to the nearest."""
    n = 256 * 400
    gen = torch.Generator().manual_seed(high)
    g = (torch.randn(n // 256, 256, generator=gen) * 10.0 ** (low + (high - low) * torch.rand(n // 256, 1, generator=gen))).reshape(-1)
    s = _state([n], torch.float32, torch.float32, False, 8)
    s["g"][0].copy_(g)
    seco.adamw_step(s["p"], s["g"], s["m"], s["v"], s["step"], 1e-3, betas=(0.0, 0.0), m_scales=s["ms"], v_scales=s["vs"])
    for x, codes, scale in ((g, s["m"][0], s["ms"][0]), ((g * g).sqrt(), s["v"][0], s["vs"][0])):
        x = x.view(-1, 256)
        unit = (x.abs().amax(1) * torch.tensor(1 / 448)).clamp_min(2.0 ** -126)
        assert torch.equal(scale.cpu(), unit)
        want = (x / unit[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).float()
        if scale is s["vs"][0]:
            want = torch.where((x > 0) & (want < 2.0 ** -9), 2.0 ** -9, want)
        assert torch.equal(codes.float().cpu().view(-1, 256), want)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_zero_gradients_and_decay(bits):
    """Nothing but the decay moves; states stay zero; eps = 0 would divide zero by zero."""
    s = _state([5000], torch.float32, torch.float32, False, bits)
    s["g"][0].zero_()
    w = s["p"][0].cpu().double()
    _go(s, lr=0.01, wd=0.5)
    assert ((s["p"][0].cpu().double() - w * (1 - 0.005)).abs() <= 4 * U * w.abs()).all()
    assert not s["m"][0].float().any() and not s["v"][0].float().any()


@pytest.mark.gpu
def test_blocks_whose_squares_decay_follow_in_their_unit():
    """Without gradients v falls by beta2 a step: the codes stay, the unit falls, over 200 steps and within their roundings."""
    s = _state([1024], torch.float32, torch.float32, False, 8, seed=9)
    _go(s)
    r0 = _unpack(s["v"][0].cpu(), s["vs"][0].cpu())
    s["g"][0].zero_()
    for _ in range(200):
        _go(s)
    r = _unpack(s["v"][0].cpu(), s["vs"][0].cpu())
    big = r0 > 2.0 ** -5 * r0.max()                           # (normal codes)
    ratio = r[big] / r0[big] / BETAS[1] ** 100
    assert ((ratio - 1).abs() < 200 * 32 * U).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """A tensor of 2^31 + 5 elements: its last block and a short one."""
    n = (1 << 31) + 5
    p = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = (torch.zeros(-(-n // 256), device=DEV) for _ in range(2))
    tail = 5 + 256
    g[-tail:] = torch.randn(tail, generator=torch.Generator().manual_seed(1)).to(DEV) * 1e-3
    p[-tail:] = 0.5
    p[:256] = 0.25
    step = torch.zeros(2, dtype=torch.int64, device=DEV)

    def host():
        return {"p": [p[-tail:].cpu()], "g": [g[-tail:].cpu()], "m": [m[-tail:].cpu()], "v": [v[-tail:].cpu()], "masters": None,
                "ms": [ms[-2:].cpu()], "vs": [vs[-2:].cpu()]}
    before = host()
    seco.adamw_step([p], [g], [m], [v], step, 1e-2, betas=BETAS, eps=EPS, weight_decay=0.0, m_scales=[ms], v_scales=[vs])
    _check(before, host(), 0, 1, 1e-2, 0.0)
    assert (p[:256] == 0.25).all() and not p[256:4096].any() and not p[n - tail - 4096:n - tail].any()
    assert step.tolist() == [1, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_captured_and_replayed(bits):
    """A replay counts the step and reads gradients, lr and scale anew; another graph of the same optimizer in between."""
    a, b = (_state([5000, 300], torch.bfloat16, torch.bfloat16, True, bits, seed=2) for _ in range(2))
    lr, scale = torch.tensor(1e-3, device=DEV), torch.tensor(1.0, device=DEV)
    _go(a, lr=lr, scale=scale)
    _go(b, lr=lr, scale=scale)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            _go(a, lr=lr, scale=scale)
    assert a["step"].tolist() == [1, 0]                       # (capturing runs nothing)
    for k in range(6):
        lr.fill_(1e-3 / (k + 1))
        scale.fill_(0.5 + k)
        for s in (a, b):
            for i, x in enumerate(s["g"]):
                x.normal_(std=1e-3, generator=torch.Generator(device=DEV).manual_seed(k * 2 + i))
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        _go(b, lr=lr, scale=scale)
        assert a["step"].tolist() == b["step"].tolist() == [k + 2, 0]
        ha, hb = _host(a), _host(b)
        for key in ("p", "m", "v", "masters", "ms", "vs"):
            if ha[key] is not None:
                assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(ha[key], hb[key]))


@pytest.mark.gpu
def test_another_stream():
    a, b = (_state([50000], torch.float32, torch.float32, False, 32, seed=5) for _ in range(2))
    _go(a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    _go(b, stream=side)
    side.synchronize()
    assert torch.equal(a["p"][0], b["p"][0]) and b["step"].tolist() == [1, 0]


# ---- the optimizer

def _params(seed=0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return {"w": torch.randn(30, 50, generator=g).to(dtype), "b": torch.randn(77, generator=g).to(dtype),
            "t": torch.randn(40, 20, generator=g).to(dtype)}


@pytest.mark.gpu
def test_optimizer_follows_a_plain_one():
    """Ten steps in fp32 beside torch.optim.AdamW in 64 bits.  Both walk in steps of about lr; a step is off by 32 U of itself
    and 4 U of the parameter, and the states by as much: ten steps stay within 10 (64 U 10 lr + 8 U |p|)."""
    host = {n: t.double().requires_grad_() for n, t in _params().items()}
    dev = {n: t.to(DEV).requires_grad_() for n, t in _params().items()}
    dev["t"] = dev["t"].detach().t().contiguous().t().requires_grad_()              # columns first
    plain = torch.optim.AdamW(host.values(), lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    opt = AdamW(dev, lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    for k in range(10):
        g = torch.Generator().manual_seed(100 + k)
        grads = {n: torch.randn(t.shape, generator=g) for n, t in host.items()}
        for n in host:
            host[n].grad = grads[n].double()
            dev[n].grad = grads[n].to(DEV)
        plain.step()
        opt.step() if k % 2 else opt.step({n: x.to(DEV) for n, x in grads.items()})
    assert opt.steps.tolist() == [10, 0]
    for n in host:
        x, y = dev[n].detach().cpu().double(), host[n].detach()
        assert ((x - y).abs() <= 10 * (64 * U * 10 * 1e-2 + 8 * U * y.abs())).all(), n


@pytest.mark.gpu
def test_optimizer_with_shared_and_idle_parameters():
    p = {n: t.to(DEV).requires_grad_() for n, t in _params(dtype=torch.bfloat16).items()}
    p["again"] = p["w"]
    opt = AdamW(p, lr=1e-2, weight_decay=lambda n, t: 0.5 if t.dim() > 1 else 0.0, state_bits=8)
    assert opt.names == ["w", "b", "t"] and opt.weight_decay == [0.5, 0.0, 0.5]
    b = p["b"].detach().clone()
    w, version = p["w"].detach().clone(), p["w"]._version
    g = torch.ones_like(p["w"])
    opt.step({"w": g, "again": g, "t": torch.zeros_like(p["t"])})
    assert torch.equal(p["b"], b) and not opt.m[1].float().any()                     # no gradient: as it was
    assert not torch.equal(p["w"], w) and p["w"]._version > version
    assert torch.equal(p["w"].detach(), opt.masters[0].to(torch.bfloat16))
    with pytest.raises(KeyError):
        opt.step({"nobody": g})
    with pytest.raises(ValueError):
        opt.step([g])
    with torch.no_grad():
        p["w"].fill_(3.0)
    opt.sync_masters()
    assert (opt.masters[0] == 3).all()


@pytest.mark.gpu
def test_steps_without_every_gradient():
    """Beside torch.optim.AdamW in 64 bits: a parameter's correction goes by the steps that it has taken, whether its gradients begin
    late, are missing now and then, or all are.  Bounds as in test_optimizer_follows_a_plain_one, for 24 steps."""
    host = {n: t.double().requires_grad_() for n, t in _params().items()}
    dev = {n: t.to(DEV).requires_grad_() for n, t in _params().items()}
    kw = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    plain, opt = torch.optim.AdamW(host.values(), **kw), AdamW(dev, **kw)
    taken = dict.fromkeys(host, 0)
    for k in range(24):
        g = torch.Generator().manual_seed(200 + k)
        grads = {n: torch.randn(t.shape, generator=g) for n, t in host.items()}
        there = [n for n in host if not (n == "b" and k < 10 or n == "t" and k % 3 == 1 or k in (4, 17))]
        for n in host:
            host[n].grad = grads[n].double() if n in there else None
            taken[n] += n in there
        plain.step()
        opt.step({n: grads[n].to(DEV) for n in there})
        if k == 12:                                               # through a state saved here
            saved = {a: {n: x.clone() for n, x in b.items()} if isinstance(b, dict) else b for a, b in opt.state_dict().items()}
            opt = AdamW(dev, **kw)
            opt.load_state_dict(saved)
    counts = {"w": opt.steps, **opt.state_dict()["late"]}
    assert opt.steps.tolist() == [22, 0] and {n: int(c[0]) for n, c in counts.items()} == taken
    for n in host:
        x, y = dev[n].detach().cpu().double(), host[n].detach()
        assert ((x - y).abs() <= 24 * (64 * U * 10 * 1e-2 + 8 * U * y.abs())).all(), n


@pytest.mark.gpu
def test_captured_step_without_every_gradient():
    """Captured behind a step with the same gradients, a replay counts the steps of those parameters alone."""
    dev = [t.to(DEV) for t in _params().values()]
    ref = [t.clone() for t in dev]
    a, b = AdamW(dev, lr=1e-2), AdamW(ref, lr=1e-2)
    g = [torch.randn_like(t) for t in dev]
    some = [g[0], None, g[2]]
    a.step(some)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(some)
    b.step(some)
    for k in range(3):
        for x in g:
            x.normal_(generator=torch.Generator(device=DEV).manual_seed(k))
        graph.replay()
        torch.cuda.synchronize()
        b.step(some)
    a.step(g)
    b.step(g)
    assert all(torch.equal(x, y) for x, y in zip(dev, ref)) and a.steps.tolist() == b.steps.tolist() == [5, 0]
    assert a.state_dict()["late"]["1"].tolist() == [1, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer_state_saved_and_loaded(bits):
    def new():
        return {n: t.to(DEV) for n, t in _params(dtype=torch.bfloat16).items()}

    def grads(k):
        return {n: torch.randn(t.shape, generator=torch.Generator().manual_seed(k)).to(DEV, torch.bfloat16)
                for n, t in _params().items()}
    pa, pb = new(), new()
    a, b = (AdamW(p, lr=1e-2, state_bits=bits) for p in (pa, pb))
    a.step(grads(1))
    saved = {k: {n: x.clone() for n, x in v.items()} if isinstance(v, dict) else v for k, v in a.state_dict().items()}
    b.load_state_dict(saved)
    for n in pb:
        pb[n].copy_(pa[n])
    a.step(grads(2))
    b.step(grads(2))
    assert all(torch.equal(pa[n], pb[n]) for n in pa) and a.steps.tolist() == b.steps.tolist()
    with pytest.raises(ValueError):
        AdamW(new(), state_bits=40 - bits).load_state_dict(saved)
    with pytest.raises(ValueError):
        AdamW({"w": pa["w"]}, state_bits=bits).load_state_dict(saved)


# ---- refusals (no GPU)

def test_refusals():
    """Before anything is launched (host tensors: the last thing looked at is where they are)."""
    def call(**kw):
        a = {"p": [torch.zeros(300)], "g": [torch.zeros(300)], "m": [torch.zeros(300)], "v": [torch.zeros(300)],
             "step": torch.zeros(2, dtype=torch.int64), "lr": 1e-3}
        a.update({k: kw.pop(k) for k in list(kw) if k in a})
        seco.adamw_step(a["p"], a["g"], a["m"], a["v"], a["step"], a["lr"], **kw)
    x, half, f8 = torch.zeros(300), torch.zeros(300).bfloat16(), torch.zeros(300).to(torch.float8_e4m3fn)
    u = [torch.zeros(2)]
    for kw in (dict(g=[]), dict(m=[x, x]), dict(masters=[]), dict(m_scales=u), dict(m=[f8], v=[f8], m_scales=u, v_scales=[]),
               dict(step=torch.zeros(1, dtype=torch.int64)), dict(step=torch.zeros(2)), dict(weight_decay=[0.1, 0.1]),
               dict(g=[torch.zeros(299)]), dict(m=[torch.zeros(600)[::2]]), dict(p=[torch.zeros(600)[::2]]),
               dict(m=[f8], v=[f8], m_scales=u, v_scales=[torch.zeros(3)]), dict(lr=torch.zeros(2)),
               dict(lr=torch.zeros(1, dtype=torch.float64)), dict(grad_scale=torch.zeros(2)),
               dict(p=[x, x], g=[x, x], m=[x, x], v=[x, x]), dict(p=[x, x[5:]], g=[x, x[5:]], m=[x, x[5:]], v=[x, x[5:]])):
        with pytest.raises(ValueError):
            call(**kw)
    y, w = torch.zeros(300), torch.zeros(600)
    for kw in (dict(p=[y], m=[x], v=[x]), dict(p=[y], m=[y], v=[x]), dict(p=[half], m=[w[:300]], v=[x], masters=[w[299:599]]),
               dict(p=[y], m=[f8], v=[f8.clone()], m_scales=u, v_scales=u)):
        with pytest.raises(ValueError, match="overlap"):
            call(**kw)
    for kw in (dict(p=[x.half()]), dict(g=[x.double()]), dict(m=[half]), dict(m=[f8], v=[f8]), dict(m_scales=u, v_scales=u),
               dict(masters=[x]), dict(p=[half], masters=[half]), dict(p=[1.0]), dict(lr="fast")):
        with pytest.raises(TypeError):
            call(**kw)
    with pytest.raises(ValueError, match="on one GPU"):
        call()
    with pytest.raises(ValueError):
        AdamW({"w": x}, state_bits=16)
    with pytest.raises(TypeError):
        AdamW({"w": x.half()})
    with pytest.raises(ValueError):
        AdamW({})


def test_states_that_do_not_fit_are_refused():
    p = {"a": torch.zeros(4, 6), "b": torch.zeros(8)}
    state = AdamW(p).state_dict()
    for wrong in ({"late": {"c": torch.zeros(2)}}, {"late": {n: torch.zeros(2) for n in p}}, {"m": {}}, {"more": {}}):
        with pytest.raises(ValueError):
            AdamW(p).load_state_dict({**state, **wrong})
    opt = AdamW(p)
    for bad, error in ((torch.zeros(9), ValueError), (torch.zeros(8).half(), TypeError)):
        with pytest.raises(error, match="b: "):
            opt.step([None, bad])
    assert "late" not in state and "late" not in opt.state_dict()
    AdamW(p).load_state_dict(state)


@pytest.mark.parametrize("bits", [32, 8])
def test_states_of_another_order_of_dimensions(bits):
    """Units of 8-bit states belong to blocks in the order of memory: codes of the same shape in another order do not fit them."""
    rows, columns, one = torch.zeros(40, 20), torch.zeros(20, 40).t(), torch.zeros(40, 1, 20).transpose(0, 1)
    state = AdamW({"w": columns}, state_bits=bits).state_dict()
    state["m"]["w"].copy_(torch.arange(800.0).view(40, 20))
    opt = AdamW({"w": rows}, state_bits=bits)
    if bits == 8:
        with pytest.raises(ValueError, match="order"):
            opt.load_state_dict(state)
        opt.load_state_dict(AdamW({"w": rows.clone()}, state_bits=8).state_dict())
    else:
        opt.load_state_dict(state)
        assert torch.equal(opt.m[0], torch.arange(800.0).view(40, 20))
    AdamW({"w": one}, state_bits=bits).load_state_dict(AdamW({"w": torch.zeros(1, 40, 20)}, state_bits=bits).state_dict())


def test_status_codes():
    lib = seco.load_library()

    class Tensor(C.Structure):
        _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "master")] + [
            ("n", C.c_int64), ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("weight_decay", C.c_float)]

    class Desc(C.Structure):
        _fields_ = [(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps")] + [
            ("lr_device", C.c_void_p), ("grad_scale_device", C.c_void_p), ("state_bits", C.c_int32)]
    A = 0x1000

    def call(n=1, step=A, tensors=True, desc=True, **kw):
        d = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, state_bits=32)
        t = dict(param=A, grad=A, m=A, v=A, n=10, param_dtype=0, grad_dtype=0)
        for k, v in kw.items():
            (d if k in dict(Desc._fields_) else t)[k] = v
        return lib.adamw_step(C.byref(Desc(**d)) if desc else None, C.byref(Tensor(**t)) if tensors else None, n,
                              C.c_void_p(step), None)
    assert call(desc=False) == -1 and call(step=None) == -1 and call(tensors=False) == -1
    assert call(n=-1) == -2 and call(**{"n": 1}, grad=None) == -1 and call(m=None) == -1
    assert call(state_bits=16) == -4 and call(param_dtype=2) == -4 and call(grad_dtype=-1) == -4 and call(master=A) == -4
    assert call(state_bits=8) == -1 and call(state_bits=8, m_scale=A) == -1
    assert call(lr=-1.0) == -8 and call(lr=float("inf")) == -8 and call(beta1=1.0) == -8 and call(beta2=-0.1) == -8
    assert call(beta2=float("nan")) == -8 and call(eps=-1e-8) == -8 and call(weight_decay=-0.1) == -8
    assert call(step=A + 4) == -5 and call(param=A + 2) == -5 and call(grad=A + 1) == -5 and call(m=A + 1) == -5
    assert call(param_dtype=1, master=A + 2) == -5 and call(lr_device=A + 1) == -5
    assert call(state_bits=8, m_scale=A + 2, v_scale=A) == -5
