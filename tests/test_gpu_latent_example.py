"""examples/latent_transformer.py: the block's operators together, as they are used."""
import importlib.util
import os

import pytest
import torch

from oracle import block as ob

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("latent_transformer", os.path.join(ROOT, "examples", "latent_transformer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_example_runs(ex, dtype):
    r = ex.main(steps=5, batch=2, dtype=dtype)
    print(r, flush=True)
    assert all(v == v and abs(v) != float("inf") for v in r.values())
    assert 1 <= r["picard_rounds"] and r["sequential_rounds"] == 25


def _plain(model, x, n, keep):
    """The model in float64 with elementary operations; keep: the dropout mask of each site."""
    d = {k: v.detach().double().requires_grad_() for k, v in model.named_parameters()}
    f = torch.exp(-torch.log(torch.tensor(10000.0)) * torch.arange(model.width // 2, device="cuda") / (model.width // 2))
    a = (n[:, None].float() * f).double()
    t = torch.cat([a.sin(), a.cos()], 1) @ d["time"]
    t = t * torch.sigmoid(t)
    H, D, R = model.heads, model.dim, model.dim // 2
    cs, sn = (torch.cat([model.table[model.positions[:, a].long()][:, a * R // 2:(a + 1) * R // 2, i] for a in range(2)], 1).double()[:, None]
              for i in range(2))

    def norm(v, scale, shift):
        mean = v.mean(2, keepdim=True)
        var = ((v - mean) ** 2).mean(2, keepdim=True)
        return (v - mean) * (var + 1e-6) ** -0.5 * (1 + scale)[:, None] + shift[:, None]

    def turn(v):
        u, w = v[..., :R], v[..., R:]
        return torch.cat([u * cs - w * sn, u * sn + w * cs], -1)

    def drop(v, site):
        under = round(model.p * 65536)
        return torch.where(keep[site].view(v.shape), v * 65536 / (65536 - under), 0.0)
    h = x.double() @ d["enter"]
    for i in range(len(model.blocks)):
        p = "blocks.%d." % i
        s1, b1, s2, b2 = (t @ d[p + "modulation"]).chunk(4, 1)
        q, k, v = (norm(h, s1, b1) @ d[p + "qkv"]).unflatten(2, (3 * H, D)).split(H, 2)
        q, k, v = (u.transpose(1, 2) for u in (turn(q), turn(k), v))
        o = ((q @ k.transpose(2, 3)) * D ** -0.5).softmax(3) @ v
        h = h + drop(o.transpose(1, 2).flatten(2) @ d[p + "out"], 2 * i)
        y = norm(h, s2, b2)
        g = y @ d[p + "gate"]
        h = h + drop((g * torch.sigmoid(g) * (y @ d[p + "up"])) @ d[p + "down"], 2 * i + 1)
    s, b = (t @ d["modulation"]).chunk(2, 1)
    return norm(h, s, b) @ d["leave"], d


def test_example_gradients_match_float64(ex):
    model = ex.Model(dtype=torch.float32, seed=7)
    model.train()
    model.step += 5
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w = torch.randn(3, 48, 8, device="cuda", generator=g), torch.randn(3, 48, 8, device="cuda", generator=g)
    n = torch.tensor([3, 50, 99], device="cuda")
    keep = [torch.from_numpy(ob.kept(3 * 48, model.width, model.p, model.seed, site, 5)).cuda() for site in range(4)]
    out = model(x, n)
    (out * w).sum().backward()
    ref, d = _plain(model, x, n, keep)
    (ref * w.double()).sum().backward()
    assert float((out.detach().double() - ref.detach()).norm() / ref.detach().norm()) < 2e-5
    for name, p in model.named_parameters():
        rel = float((p.grad.double() - d[name].grad).norm() / d[name].grad.norm())
        print(name, rel, flush=True)
        # two layers of float32 sums of up to 336 terms: some 1e-6
        assert rel < 2e-5, name
