"""The operators around a decoder's training step, as cases that can be timed: the AdamW update of many tensors at once,
layer norm in both directions, and the hand-over of queries, keys and values between a projection and the KV cache under
rotary positions with several axes, in both directions.

    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program holds before the call (tensors on the GPU)
    run(state)          one pass: elementary torch operations, or (`own`) the library's entry points
    work(case)          bytes and floating-point operations that a pass cannot do without
    exact(case, seed)   what a pass gives, in 64 bits

Formulas.  AdamW, t = steps taken before + 1, g the scaled gradient: m <- b1 m + (1 - b1) g, v <- b2 v + (1 - b2) g^2,
p <- p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps).  With states in 8 bits a block of 256 consecutive
elements holds m and r = sqrt(v) as e4m3 values times max|.| / 448 of the block, an r > 0 at least 2^-9 of that unit.
Layer norm: s = x + residual (rounded), y = (s - mean) rstd gain + bias; backward, n = (x - mean) rstd, e = d_y gain:
d_x = d_in + rstd (e - mean(e) - n mean(e n)), d_gain = sum d_y n, d_bias = sum d_y.  Rotary positions: the pair
(x[i], x[i + D/2]) turns by positions[axis of i] * frequency of i.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LR, BETAS, EPS, DECAY, CLIP = 3e-4, (0.9, 0.95), 1e-8, 0.1, 0.5
BLOCK, TOP, LEAST = 256, 448.0, 2.0 ** -9      # of the 8-bit states: elements of a block, the largest e4m3 value, the smallest
NORM_EPS = 1e-5
ROPE_BASE = 500000.0


# ---- cases -------------------------------------------------------------------------------------------------------------

def _adamw(name, sizes, **kw):
    c = {"op": "adamw", "sizes": ",".join(map(str, sizes)), "dtype": "bf16", "master": True, "bits": 32, **kw}
    return {"name": name, **c} if name else c


def _norm(name, direction, rows, d, **kw):
    c = {"op": "norm", "dir": direction, "rows": rows, "d": d, "dtype": "bf16", "gain": "bf16", "residual": True, "pad": 0, **kw}
    return {"name": name, **c} if name else c


def _rope(name, direction, chunk, q_start, **kw):
    c = {"op": "rope", "dir": direction, "chunk": chunk, "q_start": q_start, "dtype": "bf16", "batch": 1, "q_heads": 32,
         "kv_heads": 8, "head_dim": 128, "sections": "16,24,24", "interleaved": False, "own_frequencies": False, **kw}
    return {"name": name, **c} if name else c


def _decoder_sizes(layers, dm, heads, kv, ff, vocab):
    layer = [dm, dm, dm * heads, dm * kv, dm * kv, heads * dm, dm * ff, ff * dm]
    return [vocab * dm, dm * vocab, dm] * (vocab > 0) + layer * layers


def listed():
    return [
        # The update of the gains alone (five norms of a two-layer decoder): a call of a few microseconds.
        _adamw("adamw_gains", [1024] * 5),
        # Every parameter of that decoder (d_model 1024, 8 / 2 heads of 128, vocabulary 1024), with fp32 masters.
        _adamw("adamw_decoder_2l", _decoder_sizes(2, 1024, 1024, 256, 4096, 1024)),
        # fp32 parameters whose sizes fit no block, states in 8 bits: heads, gains and biases of odd widths.
        _adamw("adamw_8bit_ragged_f32", [29, 1027, 50257, 1003 * 777, 255, 1, 4099 * 1031, 2 ** 20 + 3], dtype="f32", master=False,
               bits=8),
        # Three layers of the width of the benchmark's attention (d_model 4096, MLP 14336), masters, states in 8 bits.
        _adamw("adamw_8bit_3l_4096", _decoder_sizes(3, 4096, 4096, 1024, 14336, 0), bits=8),
        # Residual add and norm of the shortest chunk of the chunk-size study: latency.
        _norm("norm_fwd_c32", "fwd", 32, 4096),
        # Rows that start on no 16-byte boundary, inside wider rows.
        _norm("norm_fwd_ragged_f32", "fwd", 9001, 1027, dtype="f32", gain="f32", pad=14),
        # Backward of a 2048-token chunk of the two-layer decoder.
        _norm("norm_bwd_2k_1024", "bwd", 2048, 1024),
        # Backward of a whole 16K-token sequence, wide rows, fp32 gains.
        _norm("norm_bwd_16k_8192", "bwd", 16384, 8192, gain="f32", residual=False),
        # Rows of one chunk to the cache: a single token at the end of 16K, and a 2048-token chunk of video at 32K, pairs
        # dealt to time, height and width in turn.
        _rope("rope_append_c1", "append", 1, 16383),
        _rope("rope_append_c2048", "append", 2048, 30720, interleaved=True),
        # The way back: a whole 16K-token sequence; image rows and columns with a ladder of frequencies each, fp32, two
        # sequences, sizes that fit nothing.
        _rope("rope_readout_16k", "readout", 16384, 0),
        _rope("rope_readout_ragged_f32", "readout", 777, 1031, dtype="f32", batch=2, q_heads=6, kv_heads=3, head_dim=80,
              sections="20,20", own_frequencies=True),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(("adamw", "norm", "norm", "rope", "rope"))
    if op == "adamw":
        total, sizes = _log(rng, 1000, 200_000_000), []
        for _ in range(_log(rng, 1, 100)):
            sizes.append(_log(rng, 1, max(2, total // 4)))
        sizes.append(total)
        while sum(sizes) > 250_000_000:
            sizes.pop(0)
        rng.shuffle(sizes)
        dtype = rng.choice(("bf16", "bf16", "f32"))
        return _adamw(None, sizes, dtype=dtype, master=dtype == "bf16" and rng.random() < 0.7, bits=rng.choice((32, 8)))
    if op == "norm":
        d = rng.choice((_log(rng, 16, 16384), 8 * _log(rng, 8, 2048)))
        rows = _log(rng, 1, max(64, min(65536, 2 ** 27 // d)))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        return _norm(None, rng.choice(("fwd", "bwd")), rows, d, dtype=dtype, gain=rng.choice((dtype, "f32")),
                     residual=rng.random() < 0.5, pad=rng.choice((0, 0, _log(rng, 1, 64))))
    hq, hkv = rng.choice(((32, 8), (32, 8), (16, 2), (8, 8), (5, 5), (1, 1)))
    D = rng.choice((128, 128, 128, 64, 80, 256))
    batch = rng.choice((1, 1, 2, 3))
    chunk = _log(rng, 1, min(32768, 16384 * 48 * 128 // (batch * (hq + 2 * hkv) * D)))
    n = rng.choice((2, 3, 3, 3, 4))
    cuts = sorted(rng.sample(range(1, D // 2), n - 1))
    sections = [b - a for a, b in zip([0] + cuts, cuts + [D // 2])]
    return _rope(None, rng.choice(("append", "readout")), chunk, rng.choice((0, _log(rng, 1, 16384))),
                 dtype=rng.choice(("bf16", "bf16", "f32")), batch=batch, q_heads=hq, kv_heads=hkv, head_dim=D,
                 sections=",".join(map(str, sections)), interleaved=rng.random() < 0.5, own_frequencies=rng.random() < 0.3)


def _sizes(case):
    return [int(n) for n in case["sizes"].split(",")]


def _places(sizes):
    """Where each tensor begins in a buffer that holds them all, every one from a multiple of BLOCK elements on; its length."""
    at, places = 0, []
    for n in sizes:
        places.append(at)
        at += -(-n // BLOCK) * BLOCK
    return places, at


def _axis_of_pair(sections, interleaved):
    """The axis of every pair of a head: one run of pairs per axis, or (interleaved) dealt in turn among the axes that still
    lack some."""
    left, axis = list(sections), []
    while interleaved and any(left):
        for a, n in enumerate(left):
            if n:
                axis.append(a)
                left[a] -= 1
    return axis or [a for a, n in enumerate(sections) for _ in range(n)]


def _exponents(sections, axis, own_frequencies):
    """Of every pair: the frequency is base ** -exponent.  One ladder over all pairs, or one for each axis' pairs."""
    if not own_frequencies:
        return [i / len(axis) for i in range(len(axis))]
    seen, out = [0] * len(sections), []
    for a in axis:
        out.append(seen[a] / sections[a])
        seen[a] += 1
    return out


# ---- inputs ------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    c, dt = case, _TYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32) * std).to(dtype)

    if c["op"] == "adamw":
        sizes = _sizes(c)
        places, n = _places(sizes)
        inside = torch.zeros(n, device=DEV, dtype=torch.bool)
        for at, size in zip(places, sizes):
            inside[at:at + size] = True
        # gradients as backpropagation leaves them: magnitudes that differ between rows, means m that have seen about ten of
        # them and mean squares v of that scale
        level = torch.exp(torch.randn(n // BLOCK, 1, generator=gen, device=DEV)).expand(-1, BLOCK).reshape(-1) * inside
        master = normal(n, std=0.02, dtype=torch.float32) * inside
        flat = {"p": master.to(dt), "g": (normal(n, std=1e-3, dtype=torch.float32) * level).to(dt)}
        if c["master"]:
            flat["master"] = master
        m = normal(n, std=3e-4, dtype=torch.float32) * level
        v = (normal(n, std=1e-3, dtype=torch.float32) * level).square_() + 1e-8 * level.square()
        if c["bits"] == 8:
            flat["m"], flat["m_scale"] = _to_8(m)
            flat["v"], flat["v_scale"] = _to_8(v.sqrt_())
        else:
            flat["m"], flat["v"] = m, v
        s = {"case": c, "flat": flat, "step": torch.tensor([seed % 1000, 0], device=DEV), "clip": torch.full((), CLIP, device=DEV)}
        for name, t in flat.items():
            unit = BLOCK if name.endswith("_scale") else 1
            s[name] = [t[at // unit:-(-(at + size) // unit)] for at, size in zip(places, sizes)]
        return s
    if c["op"] == "norm":
        rows, d, pad = c["rows"], c["d"], c["pad"]
        # rows of a residual stream: a few columns far larger than the rest, another mean and size in every row
        column = 1 + 30 * (torch.rand(d, generator=gen, device=DEV) < 0.002)
        x = (torch.randn(rows, d + pad, generator=gen, device=DEV) + normal(rows, 1, dtype=torch.float32))[:, :d] * column
        s = {"case": c, "x": torch.empty(rows, d + pad, device=DEV, dtype=dt)[:, :d].copy_(x),
             "gain": (1 + normal(d, std=0.1, dtype=torch.float32)).to(_TYPES[c["gain"]]), "bias": normal(d, std=0.1, dtype=_TYPES[c["gain"]])}
        if c["residual"]:
            s["r"] = normal(rows, d)                 # forward: the layer's output; backward: the stream's own gradient
        if c["dir"] == "bwd":
            s["dy"] = normal(rows, d)
            wide = s["x"].double()
            s["mean"] = wide.mean(1)
            s["rstd"] = ((wide - s["mean"][:, None]).square().mean(1) + NORM_EPS).rsqrt().float()
            s["mean"] = s["mean"].float()
        return s
    B, Hq, Hkv, D, C = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["chunk"]
    N = c["q_start"] + C

    def projected(H):           # as a projection leaves it: [B, rows, H, D] seen as [B, H, rows, D]
        return normal(B, C, H, D).transpose(1, 2)

    sections = [int(n) for n in c["sections"].split(",")]
    # text, where all axes count the rows, and frames of 24 x 32 patches, where the first axis counts the frames
    r = torch.arange(c["q_start"], N, device=DEV) + torch.randint(0, 5000, (B, 1), generator=gen, device=DEV)
    grid = [r // 768, r // 32 % 24, r % 32, r % 7]
    text = r % 1536 < 200
    s = {"case": c, "positions": torch.stack([torch.where(text, r, g + r // 1536 * 232) for g in grid[:len(sections)]]),
         "sections": sections, "q": projected(Hq)}
    axis = _axis_of_pair(sections, c["interleaved"])
    s["axis"] = torch.tensor(axis, device=DEV)
    s["frequency"] = float(ROPE_BASE) ** -torch.tensor(_exponents(sections, axis, c["own_frequencies"]), device=DEV, dtype=torch.float64)
    if c["dir"] == "append":
        s.update(k_new=projected(Hkv), v_new=projected(Hkv), k=normal(B, Hkv, N, D), v=normal(B, Hkv, N, D))
    else:
        s.update(gk=normal(B, Hkv, N, D, dtype=torch.float32), gv=normal(B, Hkv, N, D, dtype=torch.float32))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(state):
    return {"adamw": _run_adamw, "norm": _run_norm, "rope": _run_rope}[state["case"]["op"]](state)


def _to_8(x):
    """(e4m3 codes, scales): blocks of BLOCK elements in units of their largest magnitude / TOP."""
    x = x.view(-1, BLOCK)
    scale = (x.abs().amax(1, keepdim=True) / TOP).clamp_min(2.0 ** -126)
    return (x / scale).clamp(-TOP, TOP).to(torch.float8_e4m3fn).view(-1), scale.view(-1)


def _run_adamw(s):
    c, flat = s["case"], s["flat"]
    if own:
        import paper_2505_16710_amd as seco
        seco.adamw_step(s["p"], s["g"], s["m"], s["v"], s["step"], LR, betas=BETAS, eps=EPS, weight_decay=DECAY,
                        masters=s.get("master"), m_scales=s.get("m_scale"), v_scales=s.get("v_scale"), grad_scale=s["clip"])
        return {**{k: t for k, t in flat.items() if k != "g"}, "step": s["step"]}
    s["step"][0] += 1
    t = s["step"][0].double()
    rate, root = (LR / (1 - BETAS[0] ** t)).float(), (1 - BETAS[1] ** t).sqrt().float()
    g = flat["g"].float() * s["clip"]
    if c["bits"] == 8:
        m = (flat["m"].float().view(-1, BLOCK) * flat["m_scale"][:, None]).view(-1)
        v = (flat["v"].float().view(-1, BLOCK) * flat["v_scale"][:, None]).view(-1).square_()
    else:
        m, v = flat["m"], flat["v"]
    m.mul_(BETAS[0]).add_(g, alpha=1 - BETAS[0])
    v.mul_(BETAS[1]).add_(g.square_(), alpha=1 - BETAS[1])
    r = v.sqrt()
    p = flat["master"] if c["master"] else flat["p"].float()
    p.mul_(1 - LR * DECAY).sub_(m / (r / root + EPS) * rate)
    if p is not flat["p"]:
        flat["p"].copy_(p)
    if c["bits"] == 8:
        codes, scale = _to_8(m)
        flat["m"].copy_(codes), flat["m_scale"].copy_(scale)
        codes, scale = _to_8(r)
        least = (r > 0) & (codes.float() < LEAST)
        flat["v"].copy_(torch.where(least, LEAST, codes.float())), flat["v_scale"].copy_(scale)
    return {**{k: t for k, t in flat.items() if k != "g"}, "step": s["step"]}


def _run_norm(s):
    c, x = s["case"], s["x"]
    if c["dir"] == "fwd":
        if own:
            import paper_2505_16710_amd as seco
            return seco.layer_norm_fwd(x, s["gain"], s["bias"], eps=NORM_EPS, residual=s.get("r"))
        if c["residual"]:
            x = (x.float() + s["r"].float()).to(x.dtype)
        wide = x.float()
        mean = wide.mean(1)
        off = wide - mean[:, None]
        rstd = (off.square().mean(1) + NORM_EPS).rsqrt()
        y = (off * rstd[:, None] * s["gain"].float() + s["bias"].float()).to(x.dtype)
        return (y, mean, rstd, x) if c["residual"] else (y, mean, rstd)
    if own:
        import paper_2505_16710_amd as seco
        return seco.layer_norm_bwd(x, s["gain"], s["mean"], s["rstd"], s["dy"], d_in=s.get("r"))
    n, dy = (x.float() - s["mean"][:, None]) * s["rstd"][:, None], s["dy"].float()
    e = dy * s["gain"].float()
    dx = (e - e.mean(1, keepdim=True) - n * (e * n).mean(1, keepdim=True)) * s["rstd"][:, None]
    if c["residual"]:
        dx += s["r"].float()
    return dx.to(x.dtype), (dy * n).sum(0).to(s["gain"].dtype), dy.sum(0).to(s["gain"].dtype)


def _run_rope(s):
    c = s["case"]
    here = slice(c["q_start"], c["q_start"] + c["chunk"])
    if own:
        import paper_2505_16710_amd as seco
        if "axes" not in s:
            s["axes"] = seco.RopeAxes(s["sections"], ROPE_BASE, interleaved=c["interleaved"], own_frequencies=c["own_frequencies"])
        if c["dir"] == "append":
            q = seco.rope_append_axes(s["q"], s["k_new"], s["v_new"], s["k"], s["v"], c["q_start"], s["positions"], s["axes"])
            return {"q": q, "k": s["k"], "v": s["v"]}
        return seco.rope_readout_axes(s["q"], s["gk"], s["gv"], c["q_start"], s["positions"], s["axes"])
    angle = s["positions"][s["axis"]].permute(1, 2, 0).double() * s["frequency"]          # [B, rows, pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    half = c["head_dim"] // 2

    def turned(x, sin):
        a, b = x[..., :half].float(), x[..., half:].float()
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(s["q"].dtype)

    if c["dir"] == "append":
        s["k"][:, :, here] = turned(s["k_new"], sin)
        s["v"][:, :, here] = s["v_new"]
        return {"q": turned(s["q"], sin), "k": s["k"], "v": s["v"]}
    return turned(s["q"], -sin), turned(s["gk"][:, :, here], -sin), s["gv"][:, :, here].to(s["q"].dtype)


# ---- what it takes, and what it gives -------------------------------------------------------------------------------------

def _elem(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    c, e = case, _elem(case["dtype"])
    if c["op"] == "adamw":
        sizes = _sizes(c)
        n, blocks = sum(sizes), sum(-(-x // BLOCK) for x in sizes)
        states = 16 * n if c["bits"] == 32 else 4 * n + 16 * blocks
        return {"bytes": n * e + (n * (8 + e) if c["master"] else 2 * n * e) + states, "flops": 14 * n}
    if c["op"] == "norm":
        n, g = c["rows"] * c["d"], c["d"] * _elem(c["gain"])
        if c["dir"] == "fwd":
            return {"bytes": n * e * (4 if c["residual"] else 2) + 8 * c["rows"] + 2 * g, "flops": 8 * n}
        return {"bytes": n * e * (4 if c["residual"] else 3) + 8 * c["rows"] + 3 * g, "flops": 14 * n}
    rows = c["batch"] * c["chunk"]
    q, kv = rows * c["q_heads"] * c["head_dim"], rows * c["kv_heads"] * c["head_dim"]
    at = 8 * rows * len(c["sections"].split(","))
    return {"bytes": 2 * q * e + 2 * kv * (2 * e if c["dir"] == "append" else 4 + e) + at, "flops": 3 * (q + kv)}


def _e4m3(x):
    """float64 values rounded to the nearest e4m3 value, ties to even."""
    unit = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return (x / unit).round() * unit


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "adamw":
        flat = {k: t.double() for k, t in s["flat"].items()}
        t = int(s["step"][0]) + 1
        eight = c["bits"] == 8
        g = flat["g"] * CLIP
        wide = lambda k: flat[k] * flat[k + "_scale"].repeat_interleave(BLOCK) if eight else flat[k]  # noqa: E731
        m = BETAS[0] * wide("m") + (1 - BETAS[0]) * g
        v = BETAS[1] * (wide("v") ** 2 if eight else wide("v")) + (1 - BETAS[1]) * g * g
        old = flat["master"] if c["master"] else flat["p"]
        p = old - LR * DECAY * old - LR * (m / (1 - BETAS[0] ** t)) / (torch.sqrt(v / (1 - BETAS[1] ** t)) + EPS)
        out = {"p": p, "m": m, "v": v, "step": torch.tensor([t, 0])}
        if c["master"]:
            out["master"] = p
        if eight:
            for name, x in (("m", m), ("v", v.sqrt())):
                unit = x.view(-1, BLOCK).abs().max(1).values / TOP
                code = _e4m3(x / unit.clamp_min(2.0 ** -126).repeat_interleave(BLOCK))
                out[name] = torch.where((x > 0) & (code < LEAST), LEAST, code) if name == "v" else code
                out[name + "_scale"] = unit.clamp_min(2.0 ** -126)
        return out
    if c["op"] == "norm":
        x, gain = s["x"].double(), s["gain"].double()
        if c["dir"] == "fwd":
            if c["residual"]:
                x = (x + s["r"].double()).to(s["x"].dtype).double()
            rstd = 1 / torch.sqrt(x.var(1, unbiased=False, keepdim=True) + NORM_EPS)
            y = (x - x.mean(1, keepdim=True)) * rstd * gain + s["bias"].double()
            out = (y, x.mean(1), rstd[:, 0])
            return (*out, x) if c["residual"] else out
        dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
        n = (x - s["mean"].double()[:, None]) * rstd
        e = dy * gain
        dx = rstd * (e - e.sum(1, keepdim=True) / c["d"] - n * ((e * n).sum(1, keepdim=True) / c["d"]))
        return (dx + s["r"].double() if c["residual"] else dx), torch.einsum("rd,rd->d", dy, n), dy.sum(0)
    # as a product with a complex number per pair
    axis = _axis_of_pair(s["sections"], c["interleaved"])
    frequency = [math.exp(-x * math.log(ROPE_BASE)) for x in _exponents(s["sections"], axis, c["own_frequencies"])]
    at = s["positions"].cpu().numpy().astype(np.float64)
    angle = torch.from_numpy(np.stack([at[a] * f for a, f in zip(axis, frequency)], -1)).to(DEV)[:, None]
    half, here = c["head_dim"] // 2, slice(c["q_start"], None)

    def turned(x, sign):
        z = torch.complex(x[..., :half].double(), x[..., half:].double()) * torch.polar(torch.ones_like(angle), sign * angle)
        return torch.cat((z.real, z.imag), -1)

    if c["dir"] == "append":
        k, v = s["k"].double(), s["v"].double()
        k[:, :, here], v[:, :, here] = turned(s["k_new"], 1), s["v_new"].double()
        return {"q": turned(s["q"], 1), "k": k, "v": v}
    return turned(s["q"], -1), turned(s["gk"][:, :, here], -1), s["gv"][:, :, here].double()
