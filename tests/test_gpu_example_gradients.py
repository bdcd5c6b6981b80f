"""The examples' autograd functions as a training program may use them beyond the examples' own loops."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _load(name):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location(name, os.path.join(ROOT, "examples", name + ".py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(scope="module")
def latent():
    return _load("latent_transformer")


@pytest.fixture(scope="module")
def trajectory():
    return _load("trajectory_transformer")


def _rand(shape, seed):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("which", ["latent", "trajectory"])
def test_rotary_leaves_the_gradients_that_reach_it(which, latent, trajectory):
    """They may be another consumer's too: here they reach the sum's other operands as well."""
    shape = (2, 12, 3, 8)
    q, k, a, b = (_rand(shape, i).requires_grad_() for i in range(4))
    gq, gk = _rand(shape, 5), _rand(shape, 6)
    table = _rand((20, 4, 2), 7)
    if which == "latent":
        at = torch.stack([torch.arange(12), torch.arange(12).flip(0)], 1).int().cuda()
        q2, k2 = latent.Rotary.apply(q, k, at, table, [2, 2])
    else:
        q2, k2 = trajectory.Rotary.apply(q, k, torch.arange(12, device="cuda", dtype=torch.int32), table)
    kept = gq.clone(), gk.clone()
    torch.autograd.backward([q2 + a, k2 + b], [gq, gk])
    assert torch.equal(gq, kept[0]) and torch.equal(gk, kept[1])
    assert torch.equal(a.grad, kept[0]) and torch.equal(b.grad, kept[1])
    # linear in q and k: <dq, q> is <gq, q2>, in float32 sums of 576 terms
    for x, y, g in ((q, q2, gq), (k, k2, gk)):
        assert abs(float((x.grad * x).sum() - (g * y).sum())) <= 1e-5 * float(g.norm() * y.norm())


def test_dropout_gradient_has_its_own_forward_passes_mask(latent):
    """The step may be counted up between a forward pass and its gradient, as where gradients are accumulated."""
    x, res = _rand((2, 30, 64), 10).requires_grad_(), _rand((2, 30, 64), 11)
    step = torch.zeros(1, device="cuda", dtype=torch.int32)
    ys = []
    for _ in range(2):
        ys.append(latent.Add.apply(x, res, 0.5, 3, 1, step))
        step += 1
    masks = [(y != res).detach() for y in ys]              # (no kept x is 0, or too small to see)
    assert not torch.equal(*masks)
    for y, m in zip(ys, masks):
        dx, = torch.autograd.grad(y, x, torch.ones_like(y))
        assert torch.equal(dx, 2.0 * m)                    # (p = 1/2: kept values are doubled)
