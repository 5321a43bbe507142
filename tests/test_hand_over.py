"""How the training step leaves gradients at the parameters (chunk_loop.hand_over); no GPU needed."""
import pytest
import torch

from paper_2505_16710_amd.chunk_loop import hand_over, leaves_behind


def _leaf(v=0.0):
    return torch.full((3,), v, requires_grad=True)


def test_plain_parameters_take_the_gradient_itself():
    a, b, frozen, idle = _leaf(), _leaf(), torch.zeros(3), _leaf()
    ga, gb = torch.ones(3), 2 * torch.ones(3)
    out = hand_over({"a": a, "b": b, "frozen": frozen, "idle": idle}, {"a": ga, "b": gb, "frozen": ga, "idle": None})
    assert a.grad is ga and out["a"] is ga and b.grad is gb and frozen.grad is None and idle.grad is None
    assert not out["frozen"].any() and not out["idle"].any()


def test_a_tensor_under_two_names_gets_the_sum():
    a = _leaf()
    out = hand_over({"l0.w1": a, "l1.w1": a}, {"l0.w1": torch.ones(3), "l1.w1": 2 * torch.ones(3)})
    assert torch.equal(a.grad, torch.full((3,), 3.0)) and out["l0.w1"] is a.grad and out["l1.w1"] is a.grad


def test_hooks_run_once_and_their_result_counts():
    a, b, c = _leaf(), _leaf(), _leaf()
    seen = []
    a.register_hook(lambda g: (seen.append("a"), 10 * g)[1])

    def take(t):
        seen.append("b")
        t.grad = None
    b.register_post_accumulate_grad_hook(take)
    node = c.view_as(c).grad_fn.next_functions[0][0]
    node.register_hook(lambda *_: seen.append("c"))
    g = {n: torch.ones(3) for n in "abc"}
    out = hand_over({"a": a, "b": b, "c": c}, g)
    assert sorted(seen) == ["a", "b", "c"]
    assert torch.equal(a.grad, torch.full((3,), 10.0)) and torch.equal(out["a"], a.grad)
    assert b.grad is None and not out["b"].any()
    assert torch.equal(c.grad, torch.ones(3))


def test_a_computed_parameter_passes_its_gradient_on():
    a = _leaf(1.0)
    out = hand_over({"w": 2 * a}, {"w": torch.ones(3)})
    assert torch.equal(a.grad, torch.full((3,), 2.0)) and torch.equal(out["w"], torch.ones(3))


def test_a_second_step_takes_the_place_of_the_first():
    a, b, c = _leaf(), _leaf(), _leaf()
    a.register_hook(lambda g: 10 * g)
    b.register_post_accumulate_grad_hook(lambda t: None)
    for k in (1.0, 2.0):
        out = hand_over({"a": a, "b": b, "c": c}, {n: torch.full((3,), k) for n in "abc"})
        assert torch.equal(a.grad, torch.full((3,), 10 * k)) and torch.equal(out["a"], a.grad)
        assert torch.equal(b.grad, torch.full((3,), k)) and torch.equal(c.grad, torch.full((3,), k))
    out = hand_over({"a": a, "b": b, "c": c}, {"a": None, "b": None, "c": None})       # (no chunk reached them)
    assert a.grad is None and b.grad is None and c.grad is None and not any(t.any() for t in out.values())


@pytest.mark.parametrize("hooked", [False, True])
@pytest.mark.parametrize("order", [("emb", "head"), ("head", "emb")])
def test_a_parameter_beside_one_computed_from_it(order, hooked):
    """Tied weights: the leaf holds both shares, whichever name comes first; its hook runs once, with the sum."""
    emb, seen = torch.zeros(2, 3, requires_grad=True), []
    if hooked:
        emb.register_hook(lambda g: seen.append(g.clone()))
    for _ in range(2):
        p, g = {"emb": emb, "head": emb.t()}, {"emb": torch.ones(2, 3), "head": torch.full((3, 2), 2.0)}
        out = hand_over({n: p[n] for n in order}, g)
        assert torch.equal(emb.grad, torch.full((2, 3), 3.0)) and torch.equal(out["emb"], emb.grad)
        assert torch.equal(out["head"], g["head"])
    assert len(seen) == 2 * hooked and all(torch.equal(x, torch.full((2, 3), 3.0)) for x in seen)


def test_parameters_computed_by_one_operation():
    """Two pieces of a product: one backward pass, which would find the product's factors gone the second time."""
    a = _leaf(2.0)
    x, y = torch.stack([a * a, 3 * a]).unbind()
    hand_over({"x": x, "y": y}, {"x": torch.ones(3), "y": torch.ones(3)})
    assert torch.equal(a.grad, torch.full((3,), 7.0))
    u = (a * a).view(3, 1)
    hand_over({"first": u[:1], "rest": u[1:]}, {"first": torch.ones(1, 1), "rest": torch.ones(2, 1)})
    assert torch.equal(a.grad, torch.full((3,), 11.0))              # (a is no parameter: what it holds is the program's to clear)


def test_leaves_behind_computed_parameters():
    a, b, c, d = _leaf(), _leaf(), _leaf(), _leaf()
    s = a * b
    found = leaves_behind([s[:2], s + c.detach(), d, torch.zeros(3), a.detach()])
    assert len(found) == 2 and {id(t) for t in found} == {id(a), id(b)}
    assert leaves_behind([d, c]) == []
