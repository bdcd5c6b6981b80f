"""examples/trajectory_transformer.py: the transformer operators together, as they are used."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("trajectory_transformer",
                                                  os.path.join(ROOT, "examples", "trajectory_transformer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_trains_samples_and_decodes(ex):
    """float32: the token-by-token form is the same sums in another order, a few roundings of 2^-24 a
    layer apart; the loss of predicting unit noise starts at about 1."""
    torch.manual_seed(0)
    r = ex.main(steps=120, batch=4, history=70, dtype=torch.float32)
    print(r, flush=True)
    assert r["loss_last"] < 0.6 * r["loss_first"]
    assert r["picard_rounds"] < r["sequential_rounds"]
    assert r["picard_vs_sequential"] < 0.05
    assert r["tokens_vs_whole"] < 2e-5


def test_example_in_eight_bits(ex):
    """bfloat16 and e4m3 norms: a rounding of e4m3 is 2^-4 at most, 2.6e-2 in the root mean square,
    and four rounded products a layer pair add up to under 0.1 of the output."""
    m = ex.Model(causal=True, window=32, sinks=4, seed=5)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = ex.trajectories(4, 40, 10, g)
    with torch.no_grad():
        whole = m(x)
    for eight, tol in ((False, 2e-2), (True, 0.1)):
        dec = ex.Decoder(m, 4, 40, eight)
        one = torch.stack([dec.step(x[:, i]) for i in range(40)], 1)
        rel = float((one - whole).norm() / whole.norm())
        print(eight, rel, flush=True)
        assert rel < tol


def test_example_gradients_match_float64(ex):
    """The whole model's gradient against autograd through the same model in float64 with plain operators."""
    def plain(model, x, n):
        d = {k: v.detach().double().requires_grad_() for k, v in model.named_parameters()}
        h = x.double() @ d["enter"] + model._times(n).double()
        more = torch.zeros_like(h)
        L, D, R = x.shape[1], model.dim, model.dim // 2
        cs, sn = model.table[:L].double().unbind(2)

        def norm(a, w):
            return a * torch.rsqrt(a.square().mean(2, keepdim=True) + 1e-6) * w

        def turn(a):
            u, v = a[..., :R], a[..., R:]
            c, s = cs[:, None], sn[:, None]
            return torch.cat([u * c - v * s, u * s + v * c], -1)
        for i in range(len(model.blocks)):
            p = "blocks.%d." % i
            h = h + more
            qkv = (norm(h, d[p + "norm1"]) @ d[p + "qkv"]).unflatten(2, (-1, D))
            q, k, v = qkv.split([model.heads, model.kv, model.kv], 2)
            G = model.heads // model.kv
            k, v = (t.repeat_interleave(G, 2).transpose(1, 2) for t in (turn(k), v))
            s = (turn(q).transpose(1, 2) @ k.transpose(2, 3)) * D ** -0.5
            a = (s.softmax(3) @ v).transpose(1, 2).flatten(2)
            h = h + a @ d[p + "out"]
            more = torch.nn.functional.gelu(norm(h, d[p + "norm2"]) @ d[p + "up"]) @ d[p + "down"]
        return norm(h + more, d["norm"]) @ d["leave"], d
    model = ex.Model(dtype=torch.float32, seed=7)
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w = torch.randn(3, 16, 10, device="cuda", generator=g), torch.randn(3, 16, 10, device="cuda", generator=g)
    n = torch.tensor([3, 50, 99], device="cuda")
    (model(x, n) * w).sum().backward()
    out, d = plain(model, x, n)
    (out * w.double()).sum().backward()
    for name, p in model.named_parameters():
        ref = d[name].grad
        rel = float((p.grad.double() - ref).norm() / ref.norm())
        print(name, rel, flush=True)
        # two layers of float32 sums of up to 1024 terms: some 1e-6
        assert rel < 2e-5, name
