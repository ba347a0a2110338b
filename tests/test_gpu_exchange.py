"""The expert plan, gather, combine and its gradient against the definition in 64 bits.

A sum of n products in fp32, whatever its order, is off by at most n * 2^-24 of the products' absolute sum (and the
smallest steps), the rounding to the output's type by half a step of the value."""
import numpy as np
import pytest

from oracle import mixture_oracle as MO

pytestmark = pytest.mark.gpu
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2201_00194_amd import api as A
    return A


def choices(seed, tokens, k, experts, missing=0.1, skew=0.0):
    rng = np.random.default_rng(seed)
    e = np.minimum((rng.random((tokens, k)) ** (1 + skew) * experts).astype(np.int32), experts - 1)
    e[rng.random((tokens, k)) < missing] = -1
    return e


def plan_of(api, expert, experts):
    import torch
    p = api.fs_expert_plan(torch.from_numpy(expert).cuda(), experts)
    torch.cuda.synchronize()
    return p


@pytest.mark.parametrize("tokens,k,experts", [(1, 1, 1), (1, 16, 8), (5, 2, 3), (63, 1, 30), (64, 1, 30), (65, 1, 31), (320, 2, 8), (1000, 4, 64),
                                              (2048, 1, 256), (4096, 1, 64), (4097, 1, 64), (5000, 3, 1024), (777, 8, 255), (40000, 4, 30),
                                              (131072, 2, 64), (60001, 8, 1000), (300000, 2, 127), (1200000, 4, 64)])
@pytest.mark.parametrize("missing,skew", [(0.0, 0.0), (0.2, 4.0)])
def test_plan(api, tokens, k, experts, missing, skew):
    e = choices(tokens + k, tokens, k, experts, missing, skew)
    p = plan_of(api, e, experts)
    first, order, place = MO.plan(e, experts)
    assert np.array_equal(p.first.cpu().numpy(), first)
    assert np.array_equal(p.order.cpu().numpy(), order)
    assert np.array_equal(p.place.cpu().numpy(), place)


@pytest.mark.parametrize("tokens", [1, 100, 70000])
def test_plans_of_one_expert_of_none_and_of_bad_numbers(api, tokens):
    for e in (np.full((tokens, 2), 5, np.int32), np.full((tokens, 2), -1, np.int32), np.full((tokens, 2), 1 << 30, np.int32),
              np.tile(np.array([[7, 8]], np.int32), (tokens, 1)), np.full((tokens, 2), -(1 << 31), np.int32)):
        p = plan_of(api, e, 8)
        first, order, place = MO.plan(e, 8)
        assert np.array_equal(p.first.cpu().numpy(), first) and np.array_equal(p.order.cpu().numpy(), order)
        assert np.array_equal(p.place.cpu().numpy(), place)


def test_plan_of_nothing(api):
    import torch
    p = api.fs_expert_plan(torch.zeros((0, 2), dtype=torch.int32, device="cuda"), 8)
    assert p.first.cpu().tolist() == [0] * 9 and p.order.numel() == 0


def strided(rng, rows, width, typ, extra, at=0):
    """A matrix of `typ` on the GPU, rows `width + extra` apart, starting `at` elements into memory, and its values."""
    import torch
    t = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[typ]
    stride = width + extra
    buf = torch.full((rows * stride + at + stride,), 5.0, dtype=t, device="cuda")
    view = buf[at: at + rows * stride].view(rows, stride)[:, :width]
    view.copy_(torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).to(t))
    return buf, view


def untouched(buf, view):
    """Nothing but the matrix was written."""
    mask = buf.clone()
    rows, width = view.shape
    at = view.storage_offset()
    m = mask[at: at + rows * view.stride(0)].view(rows, -1)
    m[:, :width] = 5.0
    return bool((mask == 5.0).all())


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("tokens,k,experts,width,extra,at", [
    (1, 1, 1, 1, 0, 0), (1, 8, 30, 164, 0, 0), (7, 2, 8, 1, 0, 0), (7, 2, 8, 1, 3, 1), (50, 4, 30, 3, 0, 0), (33, 3, 5, 16, 0, 0),
    (33, 3, 5, 16, 8, 0), (33, 3, 5, 16, 1, 0), (64, 2, 8, 17, 0, 1), (65, 4, 64, 64, 0, 0), (100, 16, 64, 65, 0, 0), (90, 2, 30, 164, 0, 0),
    (41, 5, 30, 164, 2, 3), (20, 8, 8, 255, 0, 0), (20, 8, 8, 256, 16, 8), (9, 4, 64, 1000, 0, 0), (9, 4, 64, 1024, 0, 0), (6, 3, 4, 2049, 0, 0),
    (5, 2, 4, 4096, 0, 0), (3000, 2, 64, 40, 0, 0), (2500, 1, 8, 2, 0, 0)])
def test_gather_combine_and_gradient(api, typ, tokens, k, experts, width, extra, at):
    import torch
    rng = np.random.default_rng(tokens + width)
    e = choices(tokens, tokens, k, experts, missing=0.15)
    p = plan_of(api, e, experts)
    _, order, place = MO.plan(e, experts)
    slots = tokens * k
    _, x = strided(rng, tokens, width, typ, extra, at)
    xs_buf, xs = strided(rng, slots, width, typ, extra, at)
    api.fs_expert_gather(x, p, xs)
    assert np.array_equal(xs.cpu().double().numpy(), MO.gather(x.cpu().double().numpy(), order, k))
    assert untouched(xs_buf, xs)

    _, y = strided(rng, slots, width, typ, extra, at)
    y[int(p.first[-1]):] = float("nan")                          # slots that nobody has
    w = torch.from_numpy(rng.standard_normal((tokens, k)).astype(np.float32)).cuda()
    w[torch.from_numpy(place < 0).cuda()] = float("nan")
    yn, wn = y.cpu().double().numpy(), w.cpu().double().numpy()
    tiny = 2.0 ** -25 if typ == "fp16" else 1e-36
    for weight in (w, None):
        o_buf, out = strided(rng, tokens, width, typ, extra, at)
        api.fs_expert_combine(y, p, weight, out)
        eo, size = MO.combine(yn, place, None if weight is None else wn)
        assert np.all(np.abs(out.cpu().double().numpy() - eo) <= k * 2.0 ** -24 * size + HALF[typ] * (np.abs(eo) + k * 2.0 ** -24 * size) + tiny)
        assert untouched(o_buf, out)

    _, g = strided(rng, tokens, width, typ, extra, at)
    dy_buf, d_y = strided(rng, slots, width, typ, extra, at)
    _, d_w = api.fs_expert_combine_backward(g, y, p, w, d_y)
    ey, ew, size = MO.combine_backward(g.cpu().double().numpy(), yn, place, wn)
    assert np.all(np.abs(d_y.cpu().double().numpy() - ey) <= (2.0 ** -24 + HALF[typ] * (1 + 2.0 ** -24)) * np.abs(ey) + tiny)
    assert untouched(dy_buf, d_y)
    assert np.all(np.abs(d_w.cpu().double().numpy() - ew) <= width * 2.0 ** -24 * size + 1e-36)


def test_gradient_of_the_combination_against_differences(api):
    """out is linear in y and in the weights: a difference over a power of two is the derivative up to rounding."""
    import torch
    rng = np.random.default_rng(1)
    e = choices(1, 12, 3, 5)
    p = plan_of(api, e, 5)
    y = torch.from_numpy(rng.standard_normal((36, 8)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.standard_normal((12, 3)).astype(np.float32)).cuda()
    g = torch.from_numpy(rng.standard_normal((12, 8)).astype(np.float32)).cuda()
    d_y, d_w = api.fs_expert_combine_backward(g, y, p, w)

    def loss(y_, w_):
        return float((api.fs_expert_combine(y_, p, w_).double() * g.double()).sum())

    for s, c in ((0, 0), (7, 3), (20, 7), (35, 1)):
        h = torch.zeros_like(y)
        h[s, c] = 0.5
        assert abs(loss(y + h, w) - loss(y - h, w) - float(d_y[s, c])) < 12 * 8 * 3 * 2.0 ** -21
    for t, j in ((0, 0), (5, 1), (11, 2)):
        h = torch.zeros_like(w)
        h[t, j] = 0.5
        assert abs(loss(y, w + h) - loss(y, w - h) - float(d_w[t, j])) < 12 * 8 * 3 * 2.0 ** -21


def test_a_plan_of_ones_own_stays_inside(api):
    """Places outside the slots are skipped, not followed."""
    import torch
    place = torch.tensor([[0, 99], [-5, 1], [2, 1 << 30]], dtype=torch.int32, device="cuda")
    p = api.ExpertPlan(torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda"), place)
    x = torch.arange(12, dtype=torch.float32, device="cuda").view(3, 4)
    xs = api.fs_expert_gather(x, p)
    assert torch.equal(xs[:3], x) and bool((xs[3:] == 0).all())
    out = api.fs_expert_combine(xs, p)
    assert torch.equal(out, x)
    d_y, d_w = api.fs_expert_combine_backward(x, xs, p, torch.ones(3, 2, device="cuda"))
    assert torch.equal(d_y[:3], x) and d_w.cpu()[0, 1] == 0 and d_w.cpu()[1, 0] == 0


def test_rows_beyond_32_bit_offsets(api):
    """Slots of more than 2^31 elements."""
    import torch
    tokens, k, width = 140000, 4, 4096
    e = torch.arange(tokens * k, device="cuda", dtype=torch.int32).view(tokens, k) % 3
    p = api.fs_expert_plan(e, 3)
    x = torch.randn(tokens, width, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    xs = api.fs_expert_gather(x, p)
    for s in (0, tokens, 524288 + 17, tokens * k - 1):
        assert torch.equal(xs[s], x[int(p.order[s]) // k])
    out = api.fs_expert_combine(xs, p, torch.full((tokens, k), 0.25, device="cuda"))
    assert torch.equal(out, x)                                    # four quarters, exact in fp32
    d_y, d_w = api.fs_expert_combine_backward(x, xs, p, torch.full((tokens, k), 2.0, device="cuda"))
    for s in (0, 524288 + 17, tokens * k - 1):
        assert torch.equal(d_y[s], (x[int(p.order[s]) // k].float() * 2).to(torch.bfloat16))
    sq = x[-1].double().square().sum()
    assert abs(float(d_w[-1, -1]) - float(sq)) <= float(sq) * width * 2.0 ** -24


def test_other_streams_and_graphs(api):
    import torch
    e = torch.from_numpy(choices(3, 500, 4, 30)).cuda()
    x = torch.randn(500, 164, device="cuda")
    w = torch.randn(500, 4, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    p = api.fs_expert_plan(e, 30, stream=s)
    xs = api.fs_expert_gather(x, p, stream=s)
    out = api.fs_expert_combine(xs, p, w, stream=s)
    d_y, d_w = api.fs_expert_combine_backward(x, xs, p, w, stream=s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.fs_expert_plan(e, 30, plan=p)
        api.fs_expert_gather(x, p, xs)
        api.fs_expert_combine(xs, p, w, out)
        api.fs_expert_combine_backward(x, xs, p, w, d_y, d_w)
    for seed in (4, 5, 6):
        e.copy_(torch.from_numpy(choices(seed, 500, 4, 30)))
        x.copy_(torch.randn(500, 164))
        g.replay()
        torch.cuda.synchronize()
        q = api.fs_expert_plan(e, 30)
        ys = api.fs_expert_gather(x, q)
        assert torch.equal(p.place, q.place) and torch.equal(p.order, q.order) and torch.equal(p.first, q.first)
        assert torch.equal(xs, ys) and torch.equal(out, api.fs_expert_combine(ys, q, w))
        a, b = api.fs_expert_combine_backward(x, ys, q, w)
        assert torch.equal(d_y, a) and torch.equal(d_w, b)


def test_refusals_reach_the_caller(api):
    import torch
    p = plan_of(api, choices(1, 4, 2, 8), 8)
    with pytest.raises(api.FsError):
        api.fs_expert_plan(torch.zeros(4, 2, device="cuda"), 8)
    with pytest.raises(api.FsError):
        api.fs_expert_plan(torch.zeros(4, 17, device="cuda", dtype=torch.int32), 8)
    with pytest.raises(api.FsError):
        api.fs_expert_gather(torch.zeros(5, 8, device="cuda"), p)
    with pytest.raises(api.FsError):
        api.fs_expert_combine(torch.zeros(7, 8, device="cuda"), p)
    with pytest.raises(api.FsError):
        api.fs_expert_combine(torch.zeros(8, 8, device="cuda"), p, torch.zeros(4, 3, device="cuda"))
    with pytest.raises(api.FsError):
        api.fs_expert_combine_backward(torch.zeros(4, 8, device="cuda"), torch.zeros(8, 8, device="cuda", dtype=torch.float16), p,
                                       torch.zeros(4, 2, device="cuda"))


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("k", [2, 7])
def test_weights_gradients_of_very_wide_rows(api, typ, k):
    """Products of one sign and size, so that what fp32 loses does not average out: a lane adds at most 256 of them one after the
    other, the lane's 64 such sums too, then 64 lanes meet; each product rounds once."""
    import torch
    tokens, width = 3, 1 << 20
    t = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[typ]
    p = plan_of(api, choices(9, tokens, k, 5, missing=0.2), 5)
    g = torch.linspace(0.1, 0.7, tokens, device="cuda")[:, None].expand(tokens, width).to(t).contiguous()
    y = torch.linspace(0.2, 0.9, tokens * k, device="cuda")[:, None].expand(tokens * k, width).to(t).contiguous()
    _, d_w = api.fs_expert_combine_backward(g, y, p, torch.ones(tokens, k, device="cuda"))
    there = p.place >= 0
    exp = torch.where(there, g[:, :1].double() * y[:, 0].double()[p.place.clamp(min=0).long()] * width, 0.0)
    assert bool(((d_w.double() - exp).abs() <= (256 + 64 + 6 + 2) * 2.0 ** -24 * exp).all()), float((d_w.double() / exp - 1)[there].abs().max())


def test_plans_and_arrays_of_another_shape_are_refused(api):
    """As many choices, but not the same tokens: lists written for the one would be read as the other's."""
    import torch
    p = plan_of(api, choices(1, 4, 3, 8), 8)
    kept = p.place.clone()
    for e, experts in ((choices(2, 6, 2, 8), 8), (choices(2, 12, 1, 8), 8), (choices(2, 4, 3, 7), 7)):
        with pytest.raises(api.FsError):
            api.fs_expert_plan(torch.from_numpy(e).cuda(), experts, plan=p)
    assert torch.equal(p.place, kept)
    e = torch.from_numpy(choices(3, 4, 3, 8)).cuda()
    assert api.fs_expert_plan(e, 8, plan=p) is p and torch.equal(p.place, api.fs_expert_plan(e, 8).place)
    x, y, w = torch.zeros(4, 5, device="cuda"), torch.zeros(12, 5, device="cuda"), torch.ones(4, 3, device="cuda")
    logits, params = torch.randn(4, 8, device="cuda"), api.route_params(8, 3)
    turned, turned_e = torch.ones(3, 4, device="cuda"), torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    for call in (lambda: api.fs_expert_combine(y, p, turned), lambda: api.fs_expert_combine_backward(x, y, p, turned),
                 lambda: api.fs_expert_combine_backward(x, y, p, w, d_weight=turned), lambda: api.fs_route(params, logits, expert=turned_e),
                 lambda: api.fs_route(params, logits, weight=turned), lambda: api.fs_route_backward(params, logits, turned_e, w),
                 lambda: api.fs_route_backward(params, logits, e, turned)):
        with pytest.raises(api.FsError):
            call()
    flat_e, flat_w = torch.empty(12, dtype=torch.int32, device="cuda"), torch.empty(12, device="cuda")
    e2, w2 = api.fs_route(params, logits)
    api.fs_route(params, logits, expert=flat_e, weight=flat_w)                     # the same memory, laid flat
    assert torch.equal(flat_e.view(4, 3), e2) and torch.equal(flat_w.view(4, 3), w2)
    assert torch.equal(api.fs_expert_combine(y + 1, p, flat_w), api.fs_expert_combine(y + 1, p, w2))
