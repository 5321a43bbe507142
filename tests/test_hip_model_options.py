"""The training step with layer norms and positions on several axes, and AdamW behind it, against the fp64 model oracle: the
operators together, as a multimodal decoder is trained.

Tolerances of the gradients, per tensor max|x - ref| / max|ref|: as the other end-to-end tests of the step, fp32 5e-4 and bf16
6e-2 (the roundings of about 20 activations and gradients in a chain, 2^-8 each); the layer norms and the rotation round as
often as what they stand for.  The update is compared with its formula at the step's own gradients."""
import pytest
import torch

import paper_2505_16710_amd as seco
from oracle import model as om

DEV = "cuda:0"
F32 = dict(n_layers=3, d_model=64, n_q_heads=4, n_kv_heads=2, head_dim=32, d_ff=96, vocab=29)
BF16 = dict(n_layers=2, d_model=64, n_q_heads=2, n_kv_heads=1, head_dim=128, d_ff=96, vocab=29)


def _setup(seed, B, N, dtype, biases=True, **options):
    from paper_2505_16710_amd.chunk_loop import ChunkedDecoder
    cfg = om.ModelConfig(**(F32 if dtype is torch.float32 else BF16), **options)
    p64 = om.init_params(cfg, seed)
    g = torch.Generator().manual_seed(seed + 50)
    if cfg.layer_norm and biases:
        for n in ["norm_f"] + [f"l{l}.norm{k}" for l in range(cfg.n_layers) for k in (1, 2)]:
            p64[n + "_b"] = (0.1 * torch.randn(cfg.d_model, generator=g, dtype=torch.float64)).requires_grad_()
    p64 = {n: t.detach().to(dtype).to(torch.float64).requires_grad_() for n, t in p64.items()}
    params = {n: t.detach().to(dtype).to(DEV).requires_grad_() for n, t in p64.items()}
    tok, tgt = (torch.randint(0, cfg.vocab, (B, N), generator=g) for _ in range(2))
    pos = None
    kw = {}
    if cfg.rope_sections:
        pos = torch.randint(0, 3000, (len(cfg.rope_sections), B, N), generator=g)
        kw["rope_axes"] = seco.RopeAxes(cfg.rope_sections, cfg.rope_base, interleaved=cfg.rope_interleaved)
    dec = ChunkedDecoder(params, cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim,
                         norm="layer" if cfg.layer_norm else "rms", norm_eps=cfg.norm_eps, **kw)
    return cfg, p64, params, dec, tok, tgt, pos


def _compare(ref, got, tol):
    assert set(ref) == set(got)
    for n, r in ref.items():
        err = float((got[n].detach().double().cpu() - r).abs().max() / r.abs().max().clamp_min(1e-30))
        assert err < tol, (n, err)


OPTIONS = {"layer": dict(layer_norm=True), "axes": dict(rope_base=10000.0),
           "both": dict(layer_norm=True, rope_base=10000.0, rope_interleaved=True)}


def _options(name, dtype):
    o = dict(OPTIONS[name])
    if "rope_base" in o:
        o["rope_sections"] = (4, 6, 6) if dtype is torch.float32 else (16, 24, 24)
    return o


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(OPTIONS))
@pytest.mark.parametrize("dtype,tol,N,C", [(torch.float32, 5e-4, 100, 32), (torch.bfloat16, 6e-2, 256, 64)])
def test_gradients_of_the_whole_sequence(name, dtype, tol, N, C):
    cfg, p64, params, dec, tok, tgt, pos = _setup(3, 2, N, dtype, **_options(name, dtype))
    loss_ref, ref = om.monolithic_grads(cfg, p64, tok, tgt, pos)
    loss, got = dec.step(tok.to(DEV), tgt.to(DEV), C, positions=None if pos is None else pos.to(DEV))
    assert abs(loss - float(loss_ref)) < (1e-4 if dtype is torch.float32 else 1e-2) * abs(float(loss_ref))
    _compare(ref, got, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 5e-4), (torch.bfloat16, 6e-2)])
def test_selected_chunks(dtype, tol):
    N, C, sel, f = 320, 64, [4, 2, 1], 5.0 / 3.0
    cfg, p64, params, dec, tok, tgt, pos = _setup(5, 1, N, dtype, **_options("both", dtype))
    _, ref = om.spaco_grads(cfg, p64, tok, tgt, C, sel, f, positions=pos)
    _, got = dec.step(tok.to(DEV), tgt.to(DEV), C, selected=sel, factor=f, positions=pos.to(DEV))
    _compare(ref, got, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_schedules_agree(dtype):
    """Kept attention outputs give the same bits; a whole-sequence first stage and the transposed order agree to rounding."""
    N, C = 256, 64
    cfg, p64, params, dec, tok, tgt, pos = _setup(7, 1, N, dtype, **_options("both", dtype))
    args = (tok.to(DEV), tgt.to(DEV), C)
    _, first = dec.step(*args, positions=pos.to(DEV))
    first = {n: t.clone() for n, t in first.items()}
    _, kept = dec.step(*args, positions=pos.to(DEV), keep_attention_outputs=True)
    assert all(torch.equal(first[n], kept[n]) for n in first)
    more = [dict(stage1_chunk_len=N, keep_attention_outputs=True)] + ([dict(transposed_backward=True)] if dtype is torch.bfloat16 else [])
    for kw in more:
        _, got = dec.step(*args, positions=pos.to(DEV), **kw)
        _compare({n: t.double().cpu() for n, t in first.items()}, got, 1e-4 if dtype is torch.float32 else 6e-2)


@pytest.mark.gpu
def test_layer_norms_without_biases_and_one_gain_for_all_columns():
    cfg, p64, params, dec, tok, tgt, pos = _setup(9, 1, 96, torch.float32, biases=False, layer_norm=True)
    del p64["l1.norm2"], params["l1.norm2"]
    p64["l1.norm2"] = torch.tensor([1.25], dtype=torch.float64, requires_grad=True)
    params["l1.norm2"] = torch.tensor([1.25], device=DEV, requires_grad=True)
    _, ref = om.monolithic_grads(cfg, p64, tok, tgt)
    _, got = dec.step(tok.to(DEV), tgt.to(DEV), 32)
    _compare(ref, got, 5e-4)


@pytest.mark.gpu
def test_long_and_short_chunks():
    """2600 rows to a chunk, then 800: the norms' gradients are formed in two ways, and added up."""
    cfg, p64, params, dec, tok, tgt, pos = _setup(25, 2, 1700, torch.float32, **_options("both", torch.float32))
    _, ref = om.monolithic_grads(cfg, p64, tok, tgt, pos)
    _, got = dec.step(tok.to(DEV), tgt.to(DEV), 1300, positions=pos.to(DEV))
    _compare(ref, got, 5e-4)


@pytest.mark.gpu
@pytest.mark.parametrize("layers", [0, 1])
def test_few_layers(layers, monkeypatch):
    for sizes in (F32, BF16):
        monkeypatch.setitem(sizes, "n_layers", layers)
    for dtype, tol in ((torch.float32, 5e-4), (torch.bfloat16, 6e-2)):
        cfg, p64, params, dec, tok, tgt, pos = _setup(21, 2, 96, dtype, **_options("both", dtype))
        _, ref = om.monolithic_grads(cfg, p64, tok, tgt, pos)
        _, got = dec.step(tok.to(DEV), tgt.to(DEV), 32, positions=pos.to(DEV))
        _compare(ref, got, tol)


@pytest.mark.gpu
def test_an_fp32_tail_behind_a_bf16_body():
    """Final norm (its bias too) and head in fp32: the logits are fp32."""
    cfg, p64, params, dec, tok, tgt, pos = _setup(23, 1, 128, torch.bfloat16, **_options("both", torch.bfloat16))
    for n in ("norm_f", "norm_f_b", "head"):
        params[n] = params[n].detach().float().requires_grad_()
    _, ref = om.monolithic_grads(cfg, p64, tok, tgt, pos)
    _, got = dec.step(tok.to(DEV), tgt.to(DEV), 64, positions=pos.to(DEV))
    assert all(got[n].dtype == torch.float32 for n in ("norm_f", "norm_f_b", "head"))
    _compare(ref, got, 6e-2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_text_positions_are_those_of_one_axis(dtype):
    """Without positions every axis counts the tokens: the step of rope_base, to rounding."""
    from paper_2505_16710_amd.chunk_loop import ChunkedDecoder
    o = _options("axes", dtype)
    cfg, p64, params, dec, tok, tgt, _ = _setup(11, 2, 128, dtype, **o)
    _, got = dec.step(tok.to(DEV), tgt.to(DEV), 64)
    got = {n: t.clone() for n, t in got.items()}
    one = ChunkedDecoder(params, cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, rope_base=cfg.rope_base)
    _, want = one.step(tok.to(DEV), tgt.to(DEV), 64)
    _compare({n: t.double().cpu() for n, t in want.items()}, got, 1e-4 if dtype is torch.float32 else 6e-2)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_steps_with_the_update(dtype, bits):
    """Three steps: each update is AdamW's at the step's gradients, and the next step starts from the updated parameters."""
    from paper_2505_16710_amd.optimizer import AdamW
    N, C, lr, wd = 128, 64, 1e-2, 0.1
    cfg, p64, params, dec, tok, tgt, pos = _setup(13, 2, N, dtype, **_options("both", dtype))
    opt = AdamW(params, lr=lr, weight_decay=lambda n, t: wd if t.dim() > 1 else 0.0, state_bits=bits)
    args = (tok.to(DEV), tgt.to(DEV), C)
    for t in range(1, 4):
        before = {n: (p.detach() if w is None else w).double() for n, p, w in zip(opt.names, opt.params, opt.masters)}
        old_m = {n: m.double() if bits == 32 else m.double() * opt.m_scales[i].double().repeat_interleave(256)[:m.numel()].view_as(m)
                 for i, (n, m) in enumerate(zip(opt.names, opt.m))}
        old_v = {n: v.double() if bits == 32 else (v.double() * opt.v_scales[i].double().repeat_interleave(256)[:v.numel()].view_as(v)) ** 2
                 for i, (n, v) in enumerate(zip(opt.names, opt.v))}
        _, grads = dec.step(*args, positions=pos.to(DEV), optimizer=opt)
        grads = {n: g.clone().double() for n, g in grads.items()}
        for i, n in enumerate(opt.names):
            m = 0.9 * old_m[n] + 0.1 * grads[n]
            v = 0.999 * old_v[n] + 0.001 * grads[n] ** 2
            decay = wd if opt.params[i].dim() > 1 else 0.0
            ref = before[n] * (1 - lr * decay) - lr / (1 - 0.9 ** t) * m / ((v / (1 - 0.999 ** t)).sqrt() + 1e-8)
            now = opt.params[i].detach().double() if opt.masters[i] is None else opt.masters[i].double()
            # 32 steps of fp32 of the update's magnitude, whose m may cancel, and of the parameter
            size = before[n].abs() + lr / (1 - 0.9 ** t) * (0.9 * old_m[n].abs() + 0.1 * grads[n].abs()) / ((v / (1 - 0.999 ** t)).sqrt() + 1e-8)
            assert ((now - ref).abs() <= 32 * 2.0 ** -24 * size).all(), n
            if opt.masters[i] is not None:
                assert torch.equal(opt.params[i].detach(), opt.masters[i].to(dtype))
    assert opt.steps.tolist() == [3, 0]
    p64 = {n: p.detach().double().cpu().requires_grad_() for n, p in params.items()}
    _, ref = om.monolithic_grads(cfg, p64, tok, tgt, pos)
    _, got = dec.step(*args, positions=pos.to(DEV))
    _compare(ref, got, 5e-4 if dtype is torch.float32 else 6e-2)


@pytest.mark.gpu
def test_a_token_outside_the_table_updates_nothing():
    from paper_2505_16710_amd.optimizer import AdamW
    cfg, p64, params, dec, tok, tgt, pos = _setup(15, 1, 96, torch.float32, **_options("both", torch.float32))
    opt = AdamW(params)
    tok[0, 50] = cfg.vocab
    before = {n: t.detach().clone() for n, t in params.items()}
    with pytest.raises(IndexError):
        dec.step(tok.to(DEV), tgt.to(DEV), 32, positions=pos.to(DEV), optimizer=opt)
    assert all(torch.equal(before[n], params[n].detach()) for n in params) and opt.steps.tolist() == [0, 0]
    tok[0, 50] = -1                                             # counted from the end
    dec.step(tok.to(DEV), tgt.to(DEV), 32, positions=pos.to(DEV), optimizer=opt)
    assert opt.steps.tolist() == [1, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_updates_of_parameters_with_hooks(bits):
    """Gradients that come through autograd are the step's own, step after step: the same bits as without hooks."""
    from paper_2505_16710_amd.optimizer import AdamW
    ends = []
    for hooked in (False, True):
        cfg, p64, params, dec, tok, tgt, pos = _setup(17, 1, 96, torch.float32, **_options("both", torch.float32))
        if hooked:
            params["l0.wq"].register_hook(lambda g: None)
            params["l1.norm1_b"].register_post_accumulate_grad_hook(lambda t: None)
        opt = AdamW(params, lr=1e-2, state_bits=bits)
        for _ in range(3):
            dec.step(tok.to(DEV), tgt.to(DEV), 32, positions=pos.to(DEV), optimizer=opt)
        ends.append({n: t.detach().clone() for n, t in params.items()})
    assert all(torch.equal(ends[0][n], ends[1][n]) for n in ends[0])


@pytest.mark.gpu
def test_another_optimizer_behind_the_step():
    """Whatever has a step() that takes .grad."""
    cfg, p64, params, dec, tok, tgt, pos = _setup(18, 1, 96, torch.float32, **_options("layer", torch.float32))
    before = {n: t.detach().clone() for n, t in params.items()}
    _, grads = dec.step(tok.to(DEV), tgt.to(DEV), 32, optimizer=torch.optim.SGD(params.values(), lr=0.5))
    assert all(torch.equal(params[n].detach(), before[n] - 0.5 * grads[n]) for n in params)


@pytest.mark.gpu
def test_updates_of_leaves_behind_computed_parameters():
    """A matrix computed from a leaf, anew for every step: the optimizer's leaf holds the last step's gradient alone; one that
    the optimizer does not hold adds up, as in backward()."""
    from paper_2505_16710_amd.optimizer import AdamW
    cfg, p64, params, dec, tok, tgt, pos = _setup(19, 1, 96, torch.float32, **_options("layer", torch.float32))
    base, other = (params[n].detach().clone().requires_grad_() for n in ("l0.w1", "l0.w2"))
    opt = AdamW({**{n: t for n, t in params.items() if n not in ("l0.w1", "l0.w2")}, "base": base}, lr=1e-2)
    total = torch.zeros_like(other)
    for _ in range(3):
        params["l0.w1"], params["l0.w2"] = 2 * base, 1 * other
        _, grads = dec.step(tok.to(DEV), tgt.to(DEV), 32, optimizer=opt)
        assert torch.equal(base.grad, 2 * grads["l0.w1"])
        total += grads["l0.w2"]
        assert torch.equal(other.grad, total)


@pytest.mark.gpu
def test_functions_for_autograd():
    """LayerNorm and RopeMulti inside a graph of framework operators: gradients against the same formulas in 64 bits."""
    from paper_2505_16710_amd.chunk_loop import LayerNorm, RopeMulti
    g = torch.Generator().manual_seed(1)
    x, r, w, u = (torch.randn(2, 3, 40, 64, generator=g) for _ in range(4))
    gain, bias = torch.randn(64, generator=g), torch.randn(64, generator=g)
    pos = torch.randint(0, 500, (2, 1, 40), generator=g)
    axes = seco.RopeAxes((16, 16), 10000.0)
    leaves = [t.to(DEV).requires_grad_() for t in (x, r, gain, bias)]
    y, s = LayerNorm.apply(leaves[0], leaves[2], leaves[3], 1e-5, leaves[1])
    (RopeMulti.apply(y, pos.to(DEV), axes) * w.to(DEV) + s * u.to(DEV)).sum().backward()
    host = [t.double().requires_grad_() for t in (x, r, gain, bias)]
    s64 = host[0] + host[1]
    c = s64 - s64.mean(-1, keepdim=True)
    y64 = c * torch.rsqrt((c * c).mean(-1, keepdim=True) + 1e-5) * host[2] + host[3]
    th = torch.cat([pos[a].double()[:, None, :, None] * 10000.0 ** (-torch.arange(16 * a, 16 * a + 16, dtype=torch.float64) / 32)
                    for a in range(2)], -1)
    lo, hi = y64[..., :32], y64[..., 32:]
    t64 = torch.cat([lo * th.cos() - hi * th.sin(), hi * th.cos() + lo * th.sin()], -1)
    (t64 * w.double() + s64 * u.double()).sum().backward()
    for a, b in zip(leaves, host):
        # (sums of up to 240 rows of products of three roundings: 1e-5 of the largest)
        assert float((a.grad.cpu().double() - b.grad).abs().max()) < 1e-5 * float(b.grad.abs().max())
    only = LayerNorm.apply(leaves[0].detach().requires_grad_(), None)
    only.sum().backward()
    frozen = leaves[2].detach()
    z = leaves[0].detach().requires_grad_()
    LayerNorm.apply(z, frozen).square().sum().backward()
    assert z.grad is not None and frozen.grad is None


# ---- refusals (no GPU)

def test_refusals():
    from paper_2505_16710_amd.chunk_loop import ChunkedDecoder
    from paper_2505_16710_amd import binding as B
    for kw in (dict(norm="batch"), dict(rope_base=1e4, rope_axes=seco.RopeAxes((8, 8), 1e4)), dict(rope_axes=seco.RopeAxes((32, 32), 1e4))):
        with pytest.raises(ValueError):
            ChunkedDecoder({}, 1, 2, 1, 32, **kw)
    ext = B._ext or B._load_ext()
    dm, V, D = 64, 40, 32
    mats = [torch.zeros(V, dm), torch.zeros(dm, V), torch.ones(dm), torch.ones(dm), torch.ones(dm), torch.zeros(dm, 2 * D), torch.zeros(dm, D),
            torch.zeros(dm, D), torch.zeros(2 * D, dm), torch.zeros(dm, 96), torch.zeros(96, dm)]
    packed = seco.RopeAxes((8, 8), 1e4).packed
    pos = torch.zeros(2, 1, 64, dtype=torch.int64)

    def new(norms=None, rope=None, base=None):
        return ext.step_new((1, 2, 1, D, D ** -0.5, base, 1, 64, 32, 32, False, norms, rope), mats)
    none = [None] * 3
    for norms in ((1e-5,), (1e-5, none[:2]), (1e-5, tuple(none)), 1e-5):
        with pytest.raises(TypeError):
            new(norms)
    for norms in ((-1.0, none), (float("nan"), none), (1e-5, [torch.zeros(dm + 1), None, None]), (1e-5, [None, torch.zeros(2, dm), None])):
        with pytest.raises(ValueError):
            new(norms)
    with pytest.raises(TypeError):
        new((1e-5, [None, torch.zeros(dm, dtype=torch.float64), None]))
    for rope in ((packed[:-1], pos), (packed,), packed):
        with pytest.raises(TypeError):
            new(rope=rope)
    for rope in ((packed, pos[:1]), (packed, pos.int()), (packed, pos[..., :63]), (seco.RopeAxes((32, 32), 1e4).packed, pos)):
        with pytest.raises(ValueError):
            new(rope=rope)
    with pytest.raises(ValueError):
        new(rope=(packed, pos), base=1e4)
    with pytest.raises(ValueError, match="on one GPU"):
        new((1e-5, none), (packed, pos))
