"""Products of rows with their expert's weights, and the weights' gradient, against the definition in 64 bits.

A sum of n products in fp32, in any order, is off by at most (n + 1) * 2^-24 of the products' absolute sum (each product and each
addition rounds once; sums of 16-bit numbers' products round less); the rounding to the output's type by half a step."""
import numpy as np
import pytest

from oracle import experts_oracle as XO

pytestmark = pytest.mark.gpu
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LEAST = {"fp32": 1e-36, "bf16": 1e-36, "fp16": 2.0 ** -25}


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2201_00194_amd import api as A
    return A


def of(typ):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[typ]


def plan_of(api, counts, nobody=0):
    """A plan whose experts have so many slots, and so many behind them that nobody has."""
    import torch
    first = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device="cuda")
    slots = int(sum(counts)) + nobody
    return api.ExpertPlan(first, torch.empty(slots, dtype=torch.int32, device="cuda"), torch.empty((slots, 1), dtype=torch.int32, device="cuda"))


def strided(shape, typ, seed, extra=0, at=0, value=None):
    """A matrix, or matrices, whose rows are `extra` elements further apart than they are wide, `at` elements into memory."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    stride = shape[-1] + extra
    rows = int(np.prod(shape[:-1]))
    buf = torch.full((rows * stride + at + 8,), 5.0, dtype=of(typ), device="cuda")
    view = buf[at: at + rows * stride].view(*shape[:-1], stride)[..., :shape[-1]]
    if value is None:
        view.copy_(torch.randn(shape, generator=gen, device="cuda"))
    else:
        view.fill_(value)
    return buf, view


def untouched(buf, view):
    mask = buf.clone()
    rows = int(np.prod(view.shape[:-1]))
    mask[view.storage_offset(): view.storage_offset() + rows * view.stride(-2)].view(rows, -1)[:, :view.shape[-1]] = 5.0
    return bool((mask == 5.0).all())


def exact_product(x, plan, w, turned):
    """(y, the sums of absolute products) in 64 bits."""
    import torch
    out = w.shape[2] if turned else w.shape[1]
    y = torch.zeros(x.shape[0], out, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(y)
    for e, (a, b) in enumerate(XO.bounds(plan.first.tolist(), x.shape[0])[:-1]):
        we = w[e].double() if turned else w[e].double().t().contiguous()
        y[a:b] = x[a:b].double() @ we
        size[a:b] = x[a:b].double().abs() @ we.abs()
    return y, size


def exact_weights(g, x, plan):
    import torch
    d = torch.zeros(plan.n_experts, g.shape[1], x.shape[1], dtype=torch.float64, device="cuda")
    size = torch.zeros_like(d)
    for e, (a, b) in enumerate(XO.bounds(plan.first.tolist(), x.shape[0])[:-1]):
        ge = g[a:b].double().t().contiguous()
        d[e] = ge @ x[a:b].double()
        size[e] = ge.abs() @ x[a:b].double().abs()
    return d, size


def close(got, exact, size, terms, typ):
    import torch
    off = (terms + 1) * 2.0 ** -24 * size
    bad = (got.double() - exact).abs() > off + HALF[typ] * (exact.abs() + off) + LEAST[typ]
    assert not bool(bad.any()) and bool(torch.isfinite(got).all()), \
        (torch.nonzero(bad)[:5].tolist(), int(bad.sum()), float((got.double() - exact).abs().max()))


# counts of slots, nobody's, in, out, extra elements between rows, elements into memory
SHAPES = [
    ([1], 0, 1, 1, 0, 0), ([1], 0, 8, 16, 0, 0), ([0, 1, 0], 0, 64, 64, 0, 0), ([3, 0, 5, 1], 2, 16, 24, 0, 0), ([2, 1], 1, 17, 3, 0, 0),
    ([0, 0, 0], 4, 32, 32, 0, 0), ([15, 16, 17], 0, 40, 33, 0, 0), ([64, 65, 63, 1], 7, 63, 65, 0, 0), ([128, 127, 129, 0, 1], 3, 128, 128, 0, 0),
    ([130], 0, 164, 64, 0, 0), ([70, 3, 200], 5, 164, 100, 4, 0), ([70, 3, 200], 5, 96, 160, 3, 1), ([31, 300], 0, 255, 257, 0, 0),
    ([5, 4, 6, 3, 7, 2, 8, 0, 9], 0, 512, 384, 0, 0), ([256, 257, 255], 1, 256, 256, 8, 8), ([600], 0, 1000, 300, 0, 0), ([40, 600, 2], 9, 320, 520, 16, 0),
    ([1] * 40, 0, 1024, 128, 0, 0), ([4, 4], 0, 2048, 48, 0, 0), ([1, 3], 0, 3000, 17, 0, 0), ([700, 20, 513], 0, 72, 1030, 0, 0),
    ([1400, 0, 700, 5, 900], 3, 144, 3000, 0, 0), ([500, 64, 200, 3, 433], 2, 200, 2000, 8, 0)]


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("counts,nobody,wide,out,extra,at", SHAPES)
def test_product(api, typ, turned, counts, nobody, wide, out, extra, at):
    plan = plan_of(api, counts, nobody)
    slots, owned = sum(counts) + nobody, sum(counts)
    _, x = strided((slots, wide), typ, 1, extra, at)
    x[owned:] = float("nan")                                     # nobody's
    _, w = strided((len(counts), wide, out) if turned else (len(counts), out, wide), typ, 2, extra, at)
    for e, n in enumerate(counts):
        if n == 0:
            w[e] = float("nan")                                  # nobody asks them
    exact, size = exact_product(x.nan_to_num(0.0), plan, w.nan_to_num(0.0), turned)
    for result in {typ, "fp32"}:
        y_buf, y = strided((slots, out), result, 3, extra, at)
        assert api.fs_expert_matmul(x, plan, w, turned, out=y) is y
        close(y, exact, size, wide, result)
        assert bool((y[owned:] == 0).all()) and untouched(y_buf, y)
    again = api.fs_expert_matmul(x, plan, w, turned)
    assert again.dtype == x.dtype
    close(again, exact, size, wide, typ)
    close(api.fs_expert_matmul(x.contiguous(), plan, w.contiguous(), turned), exact, size, wide, typ)


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("counts,nobody,wide,out,extra,at", SHAPES + [([5000, 0, 1, 1200], 3, 48, 40, 0, 0), ([3000], 0, 130, 7, 0, 0)])
def test_gradient_of_the_weights(api, typ, counts, nobody, wide, out, extra, at):
    plan = plan_of(api, counts, nobody)
    slots, owned = sum(counts) + nobody, sum(counts)
    _, x = strided((slots, wide), typ, 1, extra, at)
    _, g = strided((slots, out), typ, 2, extra, at)
    x[owned:] = float("nan")
    g[owned:] = float("nan")
    exact, size = exact_weights(g, x, plan)
    for result in {typ, "fp32"}:
        d_buf, d = strided((len(counts), out, wide), result, 3, extra, at)
        before = d.double().clone()
        assert api.fs_expert_matmul_backward(g, x, plan, d_w=d) is d
        close(d, exact, size, max(counts), result)
        assert untouched(d_buf, d)
        d.copy_(before)
        api.fs_expert_matmul_backward(g, x, plan, d_w=d, accumulate=True)
        close(d, exact + before, size + before.abs(), max(counts) + 1, result)
        assert untouched(d_buf, d)
    d = api.fs_expert_matmul_backward(g, x, plan)
    assert d.shape == (len(counts), out, wide) and str(d.dtype) == "torch.float32"


@pytest.mark.parametrize("typ", list(HALF))
def test_gradients_against_differences(api, typ):
    """y is linear in x and in w: over a power of two, the difference of two results is the derivative up to the results' rounding."""
    import torch
    plan = plan_of(api, [5, 0, 9], 1)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)

    def whole(*shape):      # small whole numbers: every product and every sum is exact
        return torch.randint(-4, 5, shape, generator=gen, device="cuda").to(of(typ))

    x, w, g = whole(15, 24), whole(3, 16, 24), whole(15, 16)
    d_x = api.fs_expert_matmul(g, plan, w, turned=True, out=torch.empty(15, 24, device="cuda"))
    d_w = api.fs_expert_matmul_backward(g, x, plan)

    def loss(x_, w_):
        y = api.fs_expert_matmul(x_, plan, w_, out=torch.empty(15, 16, device="cuda"))
        return float((y.double() * g.double()).sum())

    for s, c in ((0, 0), (4, 23), (5, 7), (13, 1), (14, 3)):
        h = torch.zeros_like(x)
        h[s, c] = 1
        assert loss(x + h, w) - loss(x, w) == float(d_x[s, c])
    for e, o, c in ((0, 0, 0), (2, 15, 23), (2, 3, 4), (1, 2, 2)):
        h = torch.zeros_like(w)
        h[e, o, c] = 1
        assert loss(x, w + h) - loss(x, w) == float(d_w[e, o, c])


@pytest.mark.parametrize("typ", list(HALF))
def test_whole_numbers_are_exact_whatever_the_tile(api, typ):
    """Small whole numbers: any order gives the same sum, so that every element is in its place and counted once."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    for counts, wide, out in (([1, 2, 3], 512, 256), ([300, 5, 900], 192, 272), ([2048], 256, 512), ([37] * 30, 164, 64), ([100] * 8, 1024, 1024)):
        plan = plan_of(api, counts, 2)
        slots = sum(counts) + 2
        x = torch.randint(-2, 3, (slots, wide), generator=gen, device="cuda").to(of(typ))
        w = torch.randint(-2, 3, (len(counts), out, wide), generator=gen, device="cuda").to(of(typ))
        g = torch.randint(-2, 3, (slots, out), generator=gen, device="cuda").to(of(typ))
        y = torch.empty(slots, out, device="cuda")
        assert torch.equal(api.fs_expert_matmul(x, plan, w, out=y).double(), exact_product(x, plan, w, False)[0])
        turned = w.transpose(1, 2).contiguous()
        assert torch.equal(api.fs_expert_matmul(x, plan, turned, turned=True, out=y).double(), exact_product(x, plan, w, False)[0])
        assert torch.equal(api.fs_expert_matmul_backward(g, x, plan).double(), exact_weights(g, x, plan)[0])


@pytest.mark.parametrize("typ", list(HALF))
def test_long_sums_of_one_sign(api, typ):
    """What fp32 loses does not average out."""
    import torch
    plan = plan_of(api, [2, 20000], 0)
    x = torch.full((20002, 48), 0.7, device="cuda").to(of(typ))
    g = torch.full((20002, 40), 0.3, device="cuda").to(of(typ))
    d = api.fs_expert_matmul_backward(g, x, plan)
    each = float(x[0, 0].double() * g[0, 0].double())
    assert float((d[1].double() - each * 20000).abs().max()) <= 20001 * 2.0 ** -24 * each * 20000
    wide = torch.full((3, 65536), 0.7, device="cuda").to(of(typ))
    w = torch.full((2, 9, 65536), 0.3, device="cuda").to(of(typ))
    y = api.fs_expert_matmul(wide, plan_of(api, [1, 2]), w, out=torch.empty(3, 9, device="cuda"))
    assert float((y.double() - each * 65536).abs().max()) <= 65537 * 2.0 ** -24 * each * 65536


def test_infinities_and_nan_stay_in_their_rows_and_columns(api):
    import torch
    for typ in HALF:
        x = torch.randn(40, 64, device="cuda").to(of(typ))
        w = torch.randn(2, 48, 64, device="cuda").to(of(typ))
        x[3, 5], x[21, 0], w[1, 7, 9] = float("nan"), float("inf"), float("inf")
        y = api.fs_expert_matmul(x, plan_of(api, [20, 20]), w)
        bad = ~torch.isfinite(y)
        want = torch.zeros_like(bad)
        want[3], want[21], want[20:, 7] = True, True, True
        assert torch.equal(bad, want)


@pytest.mark.parametrize("typ", ["bf16", "fp32"])
def test_bounds_that_lead_outside_are_cut(api, typ):
    import torch
    x = torch.randn(20, 32, device="cuda").to(of(typ))
    w = torch.randn(3, 16, 32, device="cuda").to(of(typ))
    g = torch.randn(20, 16, device="cuda").to(of(typ))
    plan = api.ExpertPlan(torch.tensor([-5, 4, 1 << 30, 1 << 30], dtype=torch.int32, device="cuda"),
                          torch.empty(20, dtype=torch.int32, device="cuda"), torch.empty((20, 1), dtype=torch.int32, device="cuda"))
    y = api.fs_expert_matmul(x, plan, w, out=torch.empty(20, 16, device="cuda"))
    close(y, *exact_product(x, plan, w, False), 32, "fp32")
    d = api.fs_expert_matmul_backward(g, x, plan)
    close(d, *exact_weights(g, x, plan), 20, "fp32")
    wild = api.ExpertPlan(torch.tensor([19, -(1 << 31), (1 << 31) - 1, 3], dtype=torch.int32, device="cuda"), plan.order, plan.place)
    api.fs_expert_matmul(x, wild, w)                               # nothing is promised but that it stays inside
    api.fs_expert_matmul_backward(g, x, wild)
    torch.cuda.synchronize()


def test_bounds_that_descend_touch_nothing_else(api):
    # All experts claim all slots: as pieces of 128 rows they would be some 500 times as many as the slots have.
    import torch
    n, experts = 20000, 1024
    first = torch.tensor([0, n] * (experts // 2) + [n], dtype=torch.int32, device="cuda")
    plan = api.ExpertPlan(first, torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty((n, 1), dtype=torch.int32, device="cuda"))
    x, w = torch.ones(n, 64, device="cuda"), torch.ones(experts, 64, 64, device="cuda")
    around = torch.full((n + 2, 64), 7.0, device="cuda")
    api.fs_expert_matmul(x, plan, w, out=around[1:-1])
    api.fs_expert_matmul(x, plan, w, turned=True, out=around[1:-1])
    assert bool((around[0] == 7).all()) and bool((around[-1] == 7).all())
    grads = torch.full((experts + 2, 64, 64), 7.0, device="cuda")
    api.fs_expert_matmul_backward(x, x, plan, d_w=grads[1:-1])
    assert bool((grads[0] == 7).all()) and bool((grads[-1] == 7).all())


def test_weights_of_all_experts_in_one(api):
    import torch
    plan = plan_of(api, [9, 140, 3])
    x, w = torch.randn(152, 64, device="cuda"), torch.randn(1, 32, 64, device="cuda")
    y = api.fs_expert_matmul(x, plan, w.expand(3, 32, 64))
    assert torch.equal(y, api.fs_expert_matmul(x, plan, w.expand(3, 32, 64).contiguous()))


def test_no_slots(api):
    import torch
    plan = plan_of(api, [0, 0])
    x = torch.empty(0, 16, device="cuda")
    assert api.fs_expert_matmul(x, plan, torch.ones(2, 8, 16, device="cuda")).shape == (0, 8)
    assert bool((api.fs_expert_matmul_backward(torch.empty(0, 8, device="cuda"), x, plan) == 0).all())
    d = torch.ones(2, 8, 16, device="cuda")
    api.fs_expert_matmul_backward(torch.empty(0, 8, device="cuda"), x, plan, d_w=d, accumulate=True)
    assert bool((d == 1).all())


@pytest.mark.parametrize("typ", ["bf16", "fp32"])
def test_matrices_beyond_32_bit_offsets(api, typ):
    """Rows of more than 2^31 elements together; experts whose weights lie as far apart."""
    import torch
    wide = 8192
    slots = 262144 + 900
    plan = plan_of(api, [262144, 800], 100)
    x = torch.zeros(slots, wide, dtype=of(typ), device="cuda")
    x[::1000] = torch.randn(len(range(0, slots, 1000)), wide, device="cuda").to(of(typ))
    x[262144:] = torch.randn(900, wide, device="cuda").to(of(typ))
    store = torch.zeros((1 << 31) + 16 * wide, dtype=of(typ), device="cuda")
    w = store.as_strided((2, 16, wide), (1 << 31, wide, 1))
    w.copy_(torch.randn(2, 16, wide, device="cuda"))
    y = api.fs_expert_matmul(x, plan, w, out=torch.empty(slots, 16, device="cuda"))
    for s in (0, 1000, 261000, 262144, 262144 + 799):
        e = int(s >= 262144)
        exact, size = (w[e].double() * x[s].double()).sum(1), (w[e].double() * x[s].double()).abs().sum(1)
        assert bool(((y[s].double() - exact).abs() <= (wide + 1) * 2.0 ** -24 * size).all())
    assert bool((y[1] == 0).all()) and bool((y[-100:] == 0).all())
    g = torch.zeros(slots, 24, dtype=of(typ), device="cuda")
    g[262144:] = torch.randn(900, 24, device="cuda").to(of(typ))
    d = api.fs_expert_matmul_backward(g, x, plan)
    part = slice(262144, 262944)
    exact = g[part].double().t().contiguous() @ x[part].double()
    size = g[part].double().abs().t().contiguous() @ x[part].double().abs()
    close(d[1], exact, size, 800, "fp32")
    assert bool((d[0] == 0).all())


def test_other_streams_and_graphs(api):
    """Every replay has new inputs and new bounds, with eager work of the same tensors between them."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x = torch.randn(3000, 64, device="cuda", generator=gen).bfloat16()
    w = torch.randn(3, 48, 64, device="cuda", generator=gen).bfloat16()
    g = torch.randn(3000, 48, device="cuda", generator=gen).bfloat16()
    plan = plan_of(api, [1000, 1500, 400], 100)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y = api.fs_expert_matmul(x, plan, w, stream=s)
    d_x = api.fs_expert_matmul(g, plan, w, turned=True, stream=s)
    d_w = api.fs_expert_matmul_backward(g, x, plan, stream=s)
    s.synchronize()
    assert torch.equal(y, api.fs_expert_matmul(x, plan, w)) and torch.equal(d_w, api.fs_expert_matmul_backward(g, x, plan))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.fs_expert_matmul(x, plan, w, out=y)
        api.fs_expert_matmul(g, plan, w, turned=True, out=d_x)
        api.fs_expert_matmul_backward(g, x, plan, d_w=d_w)
    for counts in ([1000, 1500, 400], [0, 3000, 0], [2999, 0, 1], [1, 1, 1], [0, 0, 0]):
        plan.first.copy_(torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32))
        x.copy_(torch.randn(3000, 64, device="cuda", generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, api.fs_expert_matmul(x, plan, w))
        assert torch.equal(d_x, api.fs_expert_matmul(g, plan, w, turned=True))
        assert torch.equal(d_w, api.fs_expert_matmul_backward(g, x, plan))


def test_results_are_the_same_again(api):
    import torch
    plan = plan_of(api, [9000, 100, 5000], 50)
    x, g = torch.randn(14150, 96, device="cuda"), torch.randn(14150, 80, device="cuda")
    w = torch.randn(3, 80, 96, device="cuda")
    y, d = api.fs_expert_matmul(x, plan, w), api.fs_expert_matmul_backward(g, x, plan)
    for _ in range(3):
        assert torch.equal(y, api.fs_expert_matmul(x, plan, w)) and torch.equal(d, api.fs_expert_matmul_backward(g, x, plan))


def test_refusals_reach_the_caller(api):
    import torch
    plan = plan_of(api, [3, 5])
    x, w, g = torch.zeros(8, 16, device="cuda"), torch.zeros(2, 4, 16, device="cuda"), torch.zeros(8, 4, device="cuda")
    api.fs_expert_matmul(x, plan, w)
    for call in (lambda: api.fs_expert_matmul(x[:7], plan, w), lambda: api.fs_expert_matmul(x, plan, w[:1]), lambda: api.fs_expert_matmul(x, plan, w, turned=True),
                 lambda: api.fs_expert_matmul(x, plan, w.half()), lambda: api.fs_expert_matmul(x, plan, w.cpu()), lambda: api.fs_expert_matmul(x.cpu(), plan, w),
                 lambda: api.fs_expert_matmul(x, plan, w.transpose(1, 2)), lambda: api.fs_expert_matmul(x, plan, w, out=torch.zeros(8, 5, device="cuda")),
                 lambda: api.fs_expert_matmul(x, plan, w, out=torch.zeros(8, 4, device="cuda").half()), lambda: api.fs_expert_matmul(x.double(), plan, w.double()),
                 lambda: api.fs_expert_matmul(x.t(), plan, w), lambda: api.fs_expert_matmul_backward(g, x.half(), plan),
                 lambda: api.fs_expert_matmul_backward(g[:4], x, plan), lambda: api.fs_expert_matmul_backward(g, x, plan, accumulate=True),
                 lambda: api.fs_expert_matmul_backward(g, x, plan, d_w=torch.zeros(2, 16, 4, device="cuda")),
                 lambda: api.fs_expert_matmul_backward(g, x, plan, d_w=torch.zeros(1, 4, 16, device="cuda").expand(2, 4, 16))):
        with pytest.raises(api.FsError):
            call()
