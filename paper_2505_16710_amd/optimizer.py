"""AdamW over a model's parameters: the state that `binding.adamw_step` updates, and one call per training step.

    opt = AdamW(params, lr=3e-4, weight_decay=0.1, state_bits=8)
    loss, grads = decoder.step(tokens, targets, chunk_len)      # leaves the gradients in .grad
    opt.step()                                                  # or decoder.step(..., optimizer=opt)

Per parameter the state is m and v in fp32 (8 bytes) or in 8 bits (2.03 bytes), and for bf16 parameters, unless
masters=False, an fp32 master (4 bytes).  Without a master a bf16 parameter is rounded after every step, and an update below
2^-9 of it is lost.
"""
from __future__ import annotations

import torch

from . import binding as _b

BLOCK = 256                                      # elements that share a unit of the 8-bit states


def _order(t):
    """Where the elements of a dense tensor lie, beside their shape."""
    return [(n, s) for n, s in zip(t.shape, t.stride()) if n > 1] if t.numel() else []


class AdamW:
    """params: a dict name -> tensor, or an iterable of tensors (bf16 or fp32, dense in memory, on one GPU); a tensor that is
    there under several names is updated once.  lr: a float, or a one-element fp32 tensor on the GPU, which a captured step
    reads anew at every replay; the attribute may be changed between steps.  weight_decay: a float, or a callable
    (name, tensor) -> float, asked once per parameter (names of an iterable: "0", "1", ...)."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, masters=True):
        if state_bits not in (8, 32):
            raise ValueError("state_bits is 8 or 32")
        named = dict(params) if isinstance(params, dict) else {str(i): t for i, t in enumerate(params)}
        if not named:
            raise ValueError("no parameters")
        self.names, self.params, self._of = [], [], {}
        for n, t in named.items():
            if not torch.is_tensor(t) or t.dtype not in (torch.bfloat16, torch.float32):
                raise TypeError(f"{n}: parameters are bfloat16 or float32 tensors")
            if id(t) not in self._of:
                self._of[id(t)] = len(self.params)
                self.names.append(n)
                self.params.append(t)
        self._named = named
        self.lr, self.betas, self.eps, self.state_bits = lr, betas, eps, state_bits
        self.weight_decay = [float(weight_decay(n, t)) if callable(weight_decay) else float(weight_decay)
                             for n, t in zip(self.names, self.params)]

        def zeros(dtype):
            return [torch.zeros_like(t, dtype=dtype, requires_grad=False) for t in self.params]
        self.m, self.v = (zeros(torch.float8_e4m3fn if state_bits == 8 else torch.float32) for _ in range(2))
        self.m_scales = self.v_scales = None
        if state_bits == 8:
            self.m_scales, self.v_scales = ([torch.zeros(-(-t.numel() // BLOCK), device=t.device) for t in self.params]
                                            for _ in range(2))
        self.masters = [t.detach().float() if masters and t.dtype == torch.bfloat16 else None for t in self.params]
        # steps taken, on the GPU: a counter for the parameters that have had their gradients in the same calls
        self.steps = torch.zeros(2, dtype=torch.int64, device=self.params[0].device)
        self._counted = [(self.steps, list(range(len(self.params))))]

    def step(self, grads=None, grad_scale=None):
        """One update.  grads: None (every parameter's .grad), or a dict by the names of the parameters, or a list in their
        order; a parameter without a gradient (None, or not in the dict) stays as it is, its states and the number of its steps
        too, while one whose gradient is zero decays.  Parameters whose numbers differ take launches of their own; a captured
        step does not tell them apart if none in front of it has had gradients of the same ones.  grad_scale: a one-element fp32
        tensor on the GPU that the gradients are multiplied by (clipping, loss scaling), or None."""
        if grads is None:
            found = [t.grad for t in self.params]
        elif isinstance(grads, dict):
            found = [None] * len(self.params)
            for n, g in grads.items():           # (under several names: each holds the sum, as ChunkedDecoder.step returns it)
                if n not in self._named:
                    raise KeyError(f"{n}: no such parameter")
                found[self._of[id(self._named[n])]] = g
        else:
            found = list(grads)
            if len(found) != len(self.params):
                raise ValueError("one gradient (or None) per parameter")
        missing = any(g is None for g in found)
        if missing or len(self._counted) > 1:    # (what the update would refuse, before the first of several launches)
            for n, t, g in zip(self.names, self.params, found):
                if g is not None and (g.shape != t.shape or g.device != t.device):
                    raise ValueError(f"{n}: the gradient must have the parameter's shape and device")
                if g is not None and g.dtype not in (torch.bfloat16, torch.float32):
                    raise TypeError(f"{n}: gradients are bfloat16 or float32 tensors")
        for i, (g, t) in enumerate(zip(found, self.params)):
            if g is not None and g.stride() != t.stride() and g.shape == t.shape:     # (a dense copy in the parameter's order)
                found[i] = torch.empty_like(t, dtype=g.dtype, requires_grad=False).copy_(g)
        with torch.no_grad():
            for steps, members in self._counted[:]:
                at = [i for i in members if found[i] is not None] if missing else members
                if not at:
                    continue
                if len(at) < len(members) and not (steps.is_cuda and torch.cuda.is_current_stream_capturing()):
                    self._counted.append((steps.clone(), [i for i in members if found[i] is None]))
                    members[:] = at
                every = len(at) == len(self.params)

                def of(values):
                    return values if every or values is None else [values[i] for i in at]
                _b.adamw_step(of(self.params), of(found), of(self.m), of(self.v), steps, self.lr, self.betas, self.eps,
                              of(self.weight_decay), of(self.masters), of(self.m_scales), of(self.v_scales), grad_scale)

    def sync_masters(self):
        """Takes the masters from the parameters again (after a program has written to these itself)."""
        for t, w in zip(self.params, self.masters):
            if w is not None:
                w.copy_(t.detach())

    def state_dict(self):
        """The state by the parameters' names: tensors that are the optimizer's own.  late: counters of the parameters whose number
        of steps is not `steps`, where there are any."""
        out = {"state_bits": self.state_bits, "steps": self.steps}
        late = {self.names[i]: steps for steps, members in self._counted[1:] for i in members}
        if late:
            out["late"] = late
        for key in ("m", "v", "m_scales", "v_scales", "masters"):
            values = getattr(self, key)
            if values is not None:
                out[key] = {n: x for n, x in zip(self.names, values) if x is not None}
        return out

    def load_state_dict(self, state):
        """Copies a state of the same parameters and state_bits; parameters are the program's to load."""
        mine, late = self.state_dict(), state.get("late", {})
        keys = set(mine) - {"state_bits", "steps", "late"}
        if state["state_bits"] != self.state_bits or set(state) - {"late"} != keys | {"state_bits", "steps"}:
            raise ValueError("the state is of another kind (state_bits)")
        for key in keys:
            if set(state[key]) != set(mine[key]) or any(x.shape != mine[key][n].shape or x.dtype != mine[key][n].dtype
                                                        for n, x in state[key].items()):
                raise ValueError(f"{key}: other parameters, or of another shape")
            if self.state_bits == 8 and key in ("m", "v") and any(_order(x) != _order(mine[key][n]) for n, x in state[key].items()):
                raise ValueError(f"{key}: saved from parameters whose dimensions lie in another order, and with it their blocks")
        if not set(late) < set(self.names) and late:
            raise ValueError("late: other parameters")
        for key in keys:
            for n, x in state[key].items():
                mine[key][n].copy_(x)
        self.steps.copy_(state["steps"])
        groups = {}                              # of those whose numbers are equal
        for i, n in enumerate(self.names):
            groups.setdefault(int(late[n][0]) if n in late else None, []).append(i)
        self._counted = [(self.steps, groups.pop(None))] + [(torch.zeros_like(self.steps), members) for members in groups.values()]
        for (counter, _), number in zip(self._counted[1:], groups):
            counter[0] = number
