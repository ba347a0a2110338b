"""Rows in 8-bit integers, which are exact, and their products, whose sums are: only the multiplication with two scales (an integer to
fp32, two products: three roundings) and the rounding to the output's type are not."""
import numpy as np
import pytest

from oracle import experts_oracle as XO
from oracle import mixture_oracle as MO

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
    import torch
    first = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device="cuda")
    slots = int(sum(counts)) + nobody
    return api.ExpertPlan(first, torch.empty(slots, dtype=torch.int32, device="cuda"), torch.empty((slots, 1), dtype=torch.int32, device="cuda"))


def same(api, got, x):
    q, scale = XO.quantize(x.float().cpu().numpy())
    assert np.array_equal(got[1].cpu().numpy(), scale, equal_nan=True)
    assert np.array_equal(got[0].cpu().numpy(), q)


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("rows,width,extra,at", [(1, 1, 0, 0), (3, 1, 2, 1), (1, 1024, 0, 0), (7, 5, 0, 0), (64, 8, 0, 0), (65, 16, 0, 0), (33, 63, 0, 0),
                                                 (40, 64, 3, 0), (9, 164, 0, 0), (200, 255, 0, 1), (17, 512, 8, 8), (6, 1000, 0, 0), (5, 2048, 0, 0),
                                                 (3, 4097, 1, 0), (2, 20000, 0, 0), (1, 300001, 0, 0), (5000, 40, 0, 0)])
def test_rows(api, typ, rows, width, extra, at):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + width)
    buf = torch.randn(rows * (width + extra) + at, generator=gen, device="cuda").to(of(typ))
    x = buf[at:].view(rows, width + extra)[:, :width]
    same(api, api.fs_quantize_rows(x), x)
    room = torch.full((rows * (width + 5) + 3,), 77, dtype=torch.int8, device="cuda")
    q = room[3:].view(rows, width + 5)[:, :width]
    scale = torch.empty(rows, device="cuda")
    api.fs_quantize_rows(x, q, scale)
    same(api, (q, scale), x)
    assert bool((room[:3] == 77).all()) and bool((room[3:].view(rows, -1)[:, width:] == 77).all())


def test_quotients_on_and_beside_the_borders(api):
    """Values half a step from two integers, and the next floats on either side."""
    import torch
    rng = np.random.default_rng(5)
    rows = []
    for size in (127.0, 1.0, 3.7e-5, 1e30, 3.0e38, 2.0 ** -119, 2.0 ** -126, 1e-41, 2.0 ** -149, 0.0) + tuple(np.exp(rng.uniform(-40, 40, 50))):
        size = np.float32(size)
        scale = max(np.float32(np.float64(size) / 127), np.float32(2.0 ** -126))
        n = np.arange(-127, 127)
        mid = ((n + 0.5) * np.float64(scale)).astype(np.float32)
        v = np.concatenate((mid, np.nextafter(mid, np.float32(np.inf)), np.nextafter(mid, np.float32(-np.inf)), [size, -size, 0.0, -0.0]))
        rows.append(np.clip(v, -size, size).astype(np.float32))
    x = torch.from_numpy(np.stack(rows)).cuda()
    same(api, api.fs_quantize_rows(x), x)
    for t in (torch.bfloat16, torch.float16):
        y = x.to(t)
        y = torch.where(torch.isfinite(y), y, torch.zeros_like(y))
        same(api, api.fs_quantize_rows(y), y)
    whole = torch.arange(-254, 255, device="cuda").float()[None, :].expand(3, -1).contiguous()      # ties: quotients n + 1/2
    assert api.fs_quantize_rows(whole)[0][0].tolist() == [int(v) for v in np.rint(np.arange(-254, 255) / 2)]


@pytest.mark.parametrize("typ", list(HALF))
def test_rows_with_infinities_and_nan(api, typ):
    import torch
    x = torch.randn(6, 200, device="cuda").to(of(typ))
    x[1, 199], x[2, 0], x[4, 77], x[5] = float("inf"), float("-inf"), float("nan"), 0.0
    q, scale = api.fs_quantize_rows(x)
    same(api, (q, scale), x)
    assert torch.isnan(scale).tolist() == [False, True, True, False, True, False] and float(scale[5]) == 2.0 ** -126
    w = torch.ones(1, 32, 200, dtype=torch.int8, device="cuda")
    y = api.fs_expert_matmul_i8(q, scale, plan_of(api, [6]), w, torch.ones(1, 32, device="cuda"))
    assert torch.isnan(y).all(dim=1).tolist() == [False, True, True, False, True, False]
    assert torch.isnan(y).any(dim=1).tolist() == [False, True, True, False, True, False] and bool((y[5] == 0).all())


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("tokens,k,experts,width", [(1, 1, 1, 1), (1, 4, 30, 1024), (40, 3, 5, 17), (65, 2, 8, 164), (300, 8, 64, 64), (9, 16, 40, 3000), (2000, 2, 7, 40)])
def test_rows_to_their_slots(api, typ, tokens, k, experts, width):
    import torch
    rng = np.random.default_rng(tokens)
    expert = rng.integers(-1, experts, (tokens, k)).astype(np.int32)
    x = torch.randn(tokens, width, device="cuda").to(of(typ))
    x[tokens // 2, 0] = float("nan")
    plan = api.fs_expert_plan(torch.from_numpy(expert).cuda(), experts)
    q, scale = api.fs_expert_gather_i8(x, plan)
    first, order, _ = MO.plan(expert, experts)
    eq, es = XO.quantize(x.float().cpu().numpy())
    there = order >= 0
    token = np.where(there, order // k, 0)
    assert np.array_equal(q.cpu().numpy(), np.where(there[:, None], eq[token], 0))
    assert np.array_equal(scale.cpu().numpy(), np.where(there, es[token], 0), equal_nan=True)


def test_a_plan_of_ones_own_stays_inside(api):
    import torch
    place = torch.tensor([[0, 99], [-5, 1], [2, 1 << 30]], dtype=torch.int32, device="cuda")
    plan = api.ExpertPlan(torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda"), place)
    x = torch.randn(3, 40, device="cuda")
    q, scale = api.fs_expert_gather_i8(x, plan)
    eq, es = api.fs_quantize_rows(x)
    assert torch.equal(q[:3], eq) and torch.equal(scale[:3], es) and bool((q[3:] == 0).all()) and bool((scale[3:] == 0).all())


SHAPES = [([1], 0, 1, 1, 0, 0), ([3, 0, 5, 1], 2, 16, 24, 0, 0), ([2, 1], 1, 17, 3, 0, 0), ([0, 0], 4, 32, 32, 0, 0), ([15, 16, 17], 0, 40, 33, 3, 1),
          ([64, 65, 63, 1], 7, 63, 65, 0, 0), ([128, 127, 129, 0, 1], 3, 128, 128, 0, 0), ([70, 3, 200], 5, 164, 100, 12, 4), ([256, 257, 255], 1, 256, 256, 16, 16),
          ([600], 0, 1000, 300, 0, 0), ([1] * 40, 0, 1024, 128, 0, 0), ([4, 4], 0, 2048, 48, 0, 0), ([1, 3], 0, 3001, 17, 0, 0), ([700, 20, 513], 0, 72, 1030, 0, 0),
          ([300, 300], 1, 4096, 256, 0, 0), ([1400, 0, 700, 5, 900], 3, 144, 3000, 0, 0), ([500, 64, 200, 3, 433], 2, 208, 2000, 16, 16)]


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("counts,nobody,wide,out,extra,at", SHAPES)
def test_product(api, typ, counts, nobody, wide, out, extra, at):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(wide + out)
    plan = plan_of(api, counts, nobody)
    slots, owned, e = sum(counts) + nobody, sum(counts), len(counts)

    def whole(*shape):
        buf = torch.randint(-127, 128, (int(np.prod(shape[:-1])) * (shape[-1] + extra) + at,), generator=gen, device="cuda", dtype=torch.int8)
        return buf[at:].view(*shape[:-1], shape[-1] + extra)[..., :shape[-1]]

    q, w = whole(slots, wide), whole(e, out, wide)
    scale = torch.rand(slots, generator=gen, device="cuda") * 2.0 ** -9 + 1e-6
    scale[owned:] = float("nan")
    w_scale = torch.rand(e, out, generator=gen, device="cuda") * 2.0 ** -9 + 1e-6
    room = torch.full((slots, out + 3), 5.0, dtype=of(typ), device="cuda")
    y = room[:, :out]
    api.fs_expert_matmul_i8(q, scale, plan, w, w_scale, out=y)
    exact = torch.zeros(slots, out, dtype=torch.float64, device="cuda")
    for i, (a, b) in enumerate(XO.bounds(plan.first.tolist(), slots)[:-1]):
        exact[a:b] = (q[a:b].double() @ w[i].double().t().contiguous()) * scale[a:b, None].double() * w_scale[i].double()
    off = 3.01 * 2.0 ** -24 * exact.abs()
    assert bool(((y.double() - exact).abs() <= off + HALF[typ] * (exact.abs() + off) + LEAST[typ]).all())
    assert bool((room[:, out:] == 5.0).all()) and bool((y[owned:] == 0).all())
    assert torch.equal(api.fs_expert_matmul_i8(q, scale, plan, w, w_scale, dtype=of(typ)), y)


def test_the_longest_sum(api):
    import torch
    n = api.FS_MAX_I8_WIDTH
    q = torch.full((2, n), -127, dtype=torch.int8, device="cuda")
    q[1] = 127
    w = torch.full((1, 3, n), 127, dtype=torch.int8, device="cuda")
    y = api.fs_expert_matmul_i8(q, torch.ones(2, device="cuda"), plan_of(api, [2]), w, torch.ones(1, 3, device="cuda"))
    assert y.tolist() == [[float(np.float32(-127 * 127 * n))] * 3, [float(np.float32(127 * 127 * n))] * 3]
    with pytest.raises(api.FsError) as e:
        api.fs_expert_matmul_i8(torch.zeros(1, n + 1, dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda"), plan_of(api, [1]),
                                torch.zeros(1, 1, n + 1, dtype=torch.int8, device="cuda"), torch.ones(1, 1, device="cuda"))
    assert e.value.code == api.FS_EUNSUPPORTED


def test_other_streams_and_graphs(api):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    expert = torch.randint(-1, 6, (700, 3), generator=gen, device="cuda", dtype=torch.int32)
    x = torch.randn(700, 96, generator=gen, device="cuda")
    w = torch.randint(-127, 128, (6, 64, 96), generator=gen, device="cuda", dtype=torch.int8)
    w_scale = torch.rand(6, 64, generator=gen, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    plan = api.fs_expert_plan(expert, 6, stream=s)
    q, scale = api.fs_expert_gather_i8(x, plan, stream=s)
    y = api.fs_expert_matmul_i8(q, scale, plan, w, w_scale, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.fs_expert_plan(expert, 6, plan=plan)
        api.fs_expert_gather_i8(x, plan, q, scale)
        api.fs_expert_matmul_i8(q, scale, plan, w, w_scale, out=y)
    for _ in range(4):
        expert.copy_(torch.randint(-1, 6, (700, 3), generator=gen, device="cuda", dtype=torch.int32))
        x.copy_(torch.randn(700, 96, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        p2 = api.fs_expert_plan(expert, 6)
        q2, s2 = api.fs_expert_gather_i8(x, p2)
        assert torch.equal(q, q2) and torch.equal(scale, s2) and torch.equal(y, api.fs_expert_matmul_i8(q2, s2, p2, w, w_scale))


def test_refusals_reach_the_caller(api):
    import torch
    plan = plan_of(api, [3, 5])
    q, s = torch.zeros(8, 16, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda")
    w, ws = torch.zeros(2, 4, 16, dtype=torch.int8, device="cuda"), torch.ones(2, 4, device="cuda")
    api.fs_expert_matmul_i8(q, s, plan, w, ws)
    for call in (lambda: api.fs_expert_matmul_i8(q.float(), s, plan, w, ws), lambda: api.fs_expert_matmul_i8(q, s[:7], plan, w, ws),
                 lambda: api.fs_expert_matmul_i8(q, s, plan, w.float(), ws), lambda: api.fs_expert_matmul_i8(q, s, plan, w, ws.t().contiguous()),
                 lambda: api.fs_expert_matmul_i8(q, s, plan, w[:, :, :8], ws), lambda: api.fs_expert_matmul_i8(q, s, plan, w, ws, dtype=torch.float64),
                 lambda: api.fs_expert_matmul_i8(q, s.half(), plan, w, ws), lambda: api.fs_expert_matmul_i8(q.cpu(), s, plan, w, ws),
                 lambda: api.fs_quantize_rows(q), lambda: api.fs_quantize_rows(s), lambda: api.fs_quantize_rows(torch.ones(8, 16, device="cuda"), q=q[:, :8]),
                 lambda: api.fs_quantize_rows(torch.ones(8, 16, device="cuda"), scale=s[:4]), lambda: api.fs_expert_gather_i8(torch.ones(7, 16, device="cuda"), plan)):
        with pytest.raises(api.FsError):
            call()
