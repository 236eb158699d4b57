"""The example that learns merge coefficients: plan, merge, a layer's forward and backward pass and the coefficients'
gradient in one loop.  With the full read the coefficients are those of the teacher, whose outputs the loss compares
with: the loss is a square in alpha near them, and ends at the level of bf16 rounding (2^-9 of outputs of order one, as
a mean square 4e-6 at most); under a budget some of the teacher's blocks are not read, and the loss falls all the same."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("learn_coefficients", os.path.join(ROOT, "examples", "learn_coefficients.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_full_read_finds_the_teacher(example):
    found, hidden, losses = example.learn(K=4, steps=60, tokens=256)
    assert losses[-1] < 1e-2 * losses[0]
    assert max(abs(a - b) for a, b in zip(found, hidden)) < 0.05


def test_a_budget_still_lowers_the_loss(example):
    _, _, losses = example.learn(K=4, steps=40, tokens=64, budget=0.5)
    assert losses[-1] < 0.9 * losses[0]


def test_one_gradient_is_the_slope_of_the_loss(example):
    """two steps of the loop's own loss, alpha moved along the gradient's first entry only: the difference quotient over
    0.2 in alpha of a loss that is nearly quadratic, within a tenth (bf16 weights and activations)"""
    mp = example.mp
    fam, places, rnd = example.family(2, 3)
    index = mp.mp_index_blocks(fam)
    merged, grad = torch.empty_like(fam.base), torch.zeros_like(fam.base)
    w, g = example.views(merged, places), example.views(grad, places)
    x = torch.randn((200, example.HIDDEN), generator=rnd, device="cuda").bfloat16()

    def at(alpha):
        op = mp.make_op(mp.MP_OP_TA, alpha=alpha)
        plan = mp.mp_plan(index, op, mp.mp_budget_from_fraction(fam, 1.0))
        mp.mp_merge(fam, index, plan, merged)
        y, kept = example.forward(w, x)
        return plan, y, kept, y.double().square().mean().item()

    plan, y, kept, _ = at([0.5, 0.5])
    example.backward(w, g, x, kept, (y.float() * (2.0 / y.numel())).bfloat16())
    slope = mp.mp_coef_grad(fam, index, plan, grad).double().sum(1).cpu()
    quotient = (at([0.6, 0.5])[3] - at([0.4, 0.5])[3]) / 0.2
    assert abs(slope[0].item() - quotient) < 0.1 * abs(quotient) + 1e-6
