"""Networks as experts whose weights are of 16 bits, in training: steps that are smaller than the weights' own."""
import numpy as np
import pytest

from paper_2201_00194_amd.networks import NetworkMixture

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2201_00194_amd import api as A
    return A


def study(api, k, experts, features, hidden, dtype, seed=3, programs=50):
    import torch
    rng = np.random.default_rng(seed)
    off = np.concatenate(([0], np.cumsum(rng.integers(0, 9, programs)))).astype(np.int32)
    rows = torch.from_numpy(rng.standard_normal((off[-1], features)).astype(np.float32)).cuda().to(dtype)
    return rng, off, torch.from_numpy(off).cuda(), rows, NetworkMixture(api, features, experts, hidden, k, dtype, seed)


def host(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_small_steps_add_up(api, dtype):
    """64 steps, each of about a fifth of what separates two weights of the type: weights are those that the same steps lead to in 64 bits, rounded."""
    import torch
    typ = getattr(torch, dtype)
    eps = torch.finfo(typ).eps
    rng, off, o, rows, mix = study(api, 2, 5, 32, 24, typ)
    target = torch.from_numpy(rng.standard_normal(off.size - 1).astype(np.float32)).cuda()
    w, v = mix.w.double(), mix.v.double()
    rate = None
    for _ in range(64):
        program, way = mix.forward(rows, o)
        _, d_w, d_v = mix.gradients(way, (program - target) * (2.0 / (off.size - 1)))
        if rate is None:
            rate = 0.2 * eps * float(mix.w.float().abs().median() / d_w.abs().median())
            start = mix.w.double()
        w -= rate * d_w.double()
        v -= rate * d_v.double()
        mix.step(rows, o, target, rate=rate)
    for got, exact in ((mix.w, w), (mix.v, v)):
        assert got.dtype == typ
        # Half a step, and three roundings to fp32 of each of the 64.
        assert bool(((got.double() - exact).abs() <= (eps / 2 + 200 * EPS) * exact.abs().clamp(min=2.0 ** -14) + 2.0 ** -25).all())
    assert float((w - start).abs().max()) > 4 * eps * float(start.abs().median())          # far enough to be seen


def test_other_weights_put_in_between(api):
    """What rounding left of the old ones is not added to new ones."""
    import torch
    rng, off, o, rows, mix = study(api, 2, 5, 32, 24, torch.bfloat16)
    target = torch.from_numpy(rng.standard_normal(off.size - 1).astype(np.float32)).cuda()
    for _ in range(3):
        mix.step(rows, o, target)
    mix.w = (mix.w.float() * 1e-4).bfloat16()
    before = mix.w.clone()
    mix.step(rows, o, target, rate=0.0)
    assert torch.equal(mix.w, before)
