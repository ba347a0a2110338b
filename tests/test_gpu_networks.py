"""Networks as experts, forwards, backwards, in 8 bits and taught, against the same steps in 64 bits on the host, from the library's own
choice of experts on (a tie cannot matter then).

Every product is off by at most (n + 2) * 2^-24 of its absolute sum in fp32; where one is the next one's input, the absolute sums are carried
through the same steps, so that their product with the sum of all the steps' shares bounds the end result."""
import numpy as np
import pytest

from oracle import experts_oracle as XO
from oracle import mixture_oracle as MO
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
    mix = NetworkMixture(api, features, experts, hidden, k, dtype, seed)
    return rng, off, torch.from_numpy(off).cuda(), rows, mix


def host(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("k,experts,features,hidden", [(1, 1, 20, 16), (2, 4, 164, 64), (3, 9, 65, 33), (4, 30, 164, 128)])
def test_scores_and_gradients(api, k, experts, features, hidden):
    import torch
    rng, off, o, rows, mix = study(api, k, experts, features, hidden, torch.float32)
    program, way = mix.forward(rows, o)
    d_program = torch.from_numpy(rng.standard_normal(off.size - 1).astype(np.float32)).cuda()
    d_gate, d_w, d_v = mix.gradients(way, d_program)

    expert = way["expert"].cpu().numpy()
    first, order, place = MO.plan(expert, experts)
    x, w, v, weight = MO.gather(host(rows), order, k), host(mix.w), host(mix.v), host(way["weight"])
    h, h_size = XO.matmul(x, first, w)
    h_off = (features + 2) * EPS * h_size
    # Clipping cuts where fp32 does: within h_off of 0 either is right.
    a_got, sure = host(way["a"]), np.abs(h) > h_off
    a = np.maximum(h, 0)
    assert np.all(np.abs(a_got - a) <= h_off) and np.all((a_got > 0)[sure] == (h > 0)[sure])
    open_ = a_got > 0
    y, _ = XO.matmul(a_got, first, v)
    y_size = XO.matmul(a_got, first, np.abs(v))[0]
    assert np.all(np.abs(host(way["y"]) - y) <= (hidden + 2) * EPS * y_size + 1e-30)
    row, row_size = MO.combine(host(way["y"]), place, weight)
    exp, size = np.zeros(off.size - 1), np.zeros(off.size - 1)
    for p in range(off.size - 1):
        exp[p], size[p] = row[off[p]:off[p + 1]].sum(), row_size[off[p]:off[p + 1]].sum()
    assert np.all(np.abs(host(program) - exp) <= (k + 12) * EPS * size + 1e-30)

    g = np.repeat(host(d_program), np.diff(off))[:, None]
    d_y, d_weight, dw_size = MO.combine_backward(g, host(way["y"]), place, weight)
    ev, sv = XO.matmul_backward(d_y, a_got, first, experts)
    assert np.all(np.abs(host(d_v) - ev) <= (order.size + 3) * EPS * sv + 1e-30)
    d_h = XO.matmul(d_y, first, np.swapaxes(v, 1, 2))[0] * open_
    ew, sw = XO.matmul_backward(d_h, x, first, experts)
    assert np.all(np.abs(host(d_w) - ew) <= (order.size + 6) * EPS * sw + 1e-30)
    dl, dl_size = MO.route_backward(host(way["logits"]), expert, d_weight)
    _, dl_size2 = MO.route_backward(host(way["logits"]), expert, dw_size)
    exp_gate = host(rows).T @ dl
    gate_size = np.abs(host(rows)).T @ (dl_size + dl_size2)
    assert np.all(np.abs(host(d_gate) - exp_gate) <= (rows.shape[0] + 256) * EPS * gate_size + 1e-30)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_sixteen_bits(api, dtype):
    """Scores of rounded hidden rows: every hidden value and every score rounds once more."""
    import torch
    half = torch.finfo(getattr(torch, dtype)).eps / 2
    _, off, o, rows, mix = study(api, 2, 8, 96, 64, getattr(torch, dtype))
    _, way = mix.forward(rows, o)
    first, order, _ = MO.plan(way["expert"].cpu().numpy(), 8)
    h, size = XO.matmul(MO.gather(host(rows), order, 2), first, host(mix.w))
    off_h = 98 * EPS * size
    assert np.all(np.abs(host(way["a"]) - np.maximum(h, 0)) <= off_h + half * (np.abs(h) + off_h) + 2.0 ** -25)
    y = XO.matmul(host(way["a"]), first, host(mix.v))[0]
    y_size = XO.matmul(host(way["a"]), first, np.abs(host(mix.v)))[0]
    assert np.all(np.abs(host(way["y"]) - y) <= 66 * EPS * y_size + 1e-30)


def test_serving_in_8_bits(api):
    """A product of two rows in 8 bits is off by half a step of each: at most scale_x / 2 * |w|_1 + scale_w / 2 * |x|_1 + n scale_x scale_w / 4."""
    import torch
    _, off, o, rows, mix = study(api, 2, 6, 164, 64, torch.float32)
    _, way = mix.forward(rows, o)
    mix.serve()
    (w, w_scale), _ = mix.served
    plan = way["plan"]
    q, scale = api.fs_expert_gather_i8(rows, plan)
    h = host(api.fs_expert_matmul_i8(q, scale, plan, w, w_scale))
    first, order, place = MO.plan(way["expert"].cpu().numpy(), 6)
    x, wn = MO.gather(host(rows), order, 2), host(mix.w)
    exact, size = XO.matmul(x, first, wn)
    sx, sw = host(scale), host(w_scale)
    for e in range(6):
        part = slice(first[e], first[e + 1])
        bound = (sx[part, None] / 2 * np.abs(wn[e]).sum(1) + sw[e] / 2 * np.abs(x[part]).sum(1)[:, None] + 164 / 4 * sx[part, None] * sw[e]) * (1 + 1e-6)
        assert np.all(np.abs(h[part] - exact[part]) <= bound + 1e-6 * size[part])
    got = mix.score_served(rows, o)
    assert got.shape == (off.size - 1,) and bool(torch.isfinite(got).all())
    assert torch.equal(got, mix.score_served(rows, o))


@pytest.mark.parametrize("k", [1, 3])
def test_a_router_that_is_taught(api, k):
    """One step's gradient against the oracle's; rows without a teacher teach nothing."""
    import torch
    rng, off, o, rows, mix = study(api, 2, 9, 40, 16, torch.float32)
    n = rows.shape[0]
    ids = torch.from_numpy(np.stack([rng.permutation(9)[:k] for _ in range(n)]).astype(np.int32)).cuda()
    ids[::5] = -1
    teacher = torch.from_numpy(rng.standard_normal((n, k)).astype(np.float32)).cuda()
    before, logits = mix.gate.clone(), host(rows.float() @ mix.gate)
    loss = mix.teach(rows, ids, teacher, rate=1.0, temperature=2.0)
    el, sl, eg, sg = XO.distill(logits, ids.cpu().numpy(), host(teacher), 2.0, 4.0, None, np.full(n, np.float32(1.0 / n)))
    assert abs(float(loss) - el.mean()) <= 300 * EPS * sl.mean()
    moved = host(before - mix.gate)
    exp, size = host(rows).T @ eg, np.abs(host(rows)).T @ sg
    assert np.all(np.abs(moved - exp) <= (n + 600) * EPS * size + 2 * EPS * np.abs(host(before)))
    assert np.all(eg[::5] == 0)


def test_training_runs(api):
    import torch
    _, off, o, rows, mix = study(api, 2, 5, 32, 24, torch.float32)
    target = torch.randn(off.size - 1, device="cuda")
    for _ in range(5):
        assert bool(torch.isfinite(mix.step(rows, o, target)))
    assert bool(torch.isfinite(mix.w).all()) and bool(torch.isfinite(mix.gate).all()) and mix.served is None


def test_the_products_in_one_graph(api):
    """The experts' part of a step, captured once and replayed with new rows and new bounds."""
    import torch
    _, off, o, rows, mix = study(api, 2, 6, 64, 32, torch.float32)
    _, way = mix.forward(rows, o)
    plan, x = way["plan"], way["x"]
    d_y = torch.randn(x.shape[0], 1, device="cuda")
    h, d_w, d_a = torch.empty(x.shape[0], 32, device="cuda"), torch.empty_like(mix.w), torch.empty(x.shape[0], 32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.fs_expert_plan(way["expert"], 6, plan=plan)
        api.fs_expert_gather(rows, plan, x)
        api.fs_expert_matmul(x, plan, mix.w, out=h)
        api.fs_expert_matmul(d_y, plan, mix.v, turned=True, out=d_a)
        api.fs_expert_matmul_backward(d_a, x, plan, d_w=d_w)
    for seed in range(4):
        gen = torch.Generator("cuda")
        gen.manual_seed(seed)
        rows.copy_(torch.randn(rows.shape, generator=gen, device="cuda"))
        way["expert"].copy_(torch.randint(-1, 6, way["expert"].shape, generator=gen, device="cuda", dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        p = api.fs_expert_plan(way["expert"], 6)
        xs = api.fs_expert_gather(rows, p)
        assert torch.equal(h, api.fs_expert_matmul(xs, p, mix.w))
        d = api.fs_expert_matmul(d_y, p, mix.v, turned=True)
        assert torch.equal(d_a, d) and torch.equal(d_w, api.fs_expert_matmul_backward(d, xs, p))


def test_no_rows_and_programs_without_rows(api):
    import torch
    from paper_2201_00194_amd.networks import NetworkMixture
    mix = NetworkMixture(api, 20, 3, hidden=16)
    none = torch.empty(0, 20, device="cuda")
    for off in ([0], [0, 0, 0]):
        off = torch.tensor(off, dtype=torch.int32, device="cuda")
        programs = off.shape[0] - 1
        score, way = mix.forward(none, off)
        assert score.tolist() == [0.0] * programs and mix.score_served(none, off).tolist() == [0.0] * programs
        assert all(bool((d == 0).all()) for d in mix.gradients(way, torch.ones(programs, device="cuda")))
        assert float(mix.step(none, off, torch.zeros(programs, device="cuda"))) == 0
    assert float(mix.teach(none, torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda"))) == 0
    rows = torch.randn(5, 20, device="cuda")
    score, _ = mix.forward(rows, torch.tensor([0, 0, 5, 5], dtype=torch.int32, device="cuda"))
    assert float(score[0]) == 0 and float(score[2]) == 0 and float(score[1]) != 0
