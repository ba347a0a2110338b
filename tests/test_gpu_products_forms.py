"""The forms that products by expert take with many slots, ragged or skewed lists, rows of any alignment and narrow results: small whole numbers,
whose sums are exact in any order, so that every element has to be in its place and counted once.  Nobody's rows and the weights of experts
without slots hold NaN (in 8 bits: scales that are NaN)."""
import numpy as np
import pytest

from oracle import experts_oracle as XO

pytestmark = pytest.mark.gpu
TYPES = ("fp32", "bf16", "fp16")


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2201_00194_amd import api as A
    return A


def of(typ):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "i8": torch.int8}[typ]


def plan_of(api, counts, nobody):
    import torch
    first = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device="cuda")
    slots = int(sum(counts)) + nobody
    return api.ExpertPlan(first, torch.empty(slots, dtype=torch.int32, device="cuda"), torch.empty((slots, 1), dtype=torch.int32, device="cuda"))


def whole(gen, typ, *shape, extra=0, at=0):
    """Whole numbers of -2 to 2, in rows that are `extra` elements further apart than they are wide, `at` elements into memory."""
    import torch
    n = int(np.prod(shape[:-1])) * (shape[-1] + extra)
    buf = torch.randint(-2, 3, (n + at,), generator=gen, device="cuda", dtype=torch.int8).to(of(typ))
    return buf[at:].view(*shape[:-1], shape[-1] + extra)[..., :shape[-1]]


def generator(seed):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def exact(plan, x, w):
    """Sums over the columns of x and of w[e], in 64 bits."""
    import torch
    y = torch.zeros(x.shape[0], w.shape[1], dtype=torch.float64, device="cuda")
    for e, (a, b) in enumerate(XO.bounds(plan.first.tolist(), x.shape[0])[:-1]):
        if b > a:
            y[a:b] = x[a:b].double() @ w[e].double().t().contiguous()
    return y


def product(api, typ, turned, counts, nobody, wide, out, extra=0, at=0):
    """A product of x and w, into results of the type and of 32 bits that have something beside them."""
    import torch
    gen = generator(wide + out + len(counts))
    plan, owned = plan_of(api, counts, nobody), sum(counts)
    slots = owned + nobody
    x = whole(gen, typ, slots, wide, extra=extra, at=at)
    w = whole(gen, typ, len(counts), out, wide, extra=0 if turned else extra, at=0 if turned else at)
    want = exact(plan, x, w)
    assert float(want.abs().max()) < 2.0 ** 24
    if typ == "i8":
        scale = torch.exp2(torch.randint(-3, 4, (slots,), generator=gen, device="cuda").float())
        w_scale = torch.exp2(torch.randint(-3, 4, (len(counts), out), generator=gen, device="cuda").float())
        for e, (a, b) in enumerate(XO.bounds(plan.first.tolist(), slots)[:-1]):
            want[a:b] *= scale[a:b, None].double() * w_scale[e].double()
        scale[owned:] = float("nan")
    else:
        x[owned:] = float("nan")
        for e, n in enumerate(counts):
            if n == 0:
                w[e] = float("nan")
        if turned:
            rows = torch.empty(len(counts) * wide * (out + extra) + at, dtype=of(typ), device="cuda")
            w = rows[at:].view(len(counts), wide, out + extra)[..., :out].copy_(w.transpose(1, 2))
    for result in (TYPES if typ == "i8" else {typ, "fp32"}):
        room = torch.full((slots, out + 8), 5.0, dtype=of(result), device="cuda")
        y = room[:, :out]
        if typ == "i8":
            api.fs_expert_matmul_i8(x, scale, plan, w, w_scale, out=y)
        else:
            api.fs_expert_matmul(x, plan, w, turned, out=y)
        expect = want.float().to(of(result))
        assert torch.equal(y, expect), (result, torch.nonzero(y != expect)[:5].tolist(), int((y != expect).sum()))
        assert bool((room[:, out:] == 5.0).all())


RAGGED = [9000, 0, 6500, 257, 4243]


@pytest.mark.parametrize("typ", ["bf16", "fp16", "i8"])
@pytest.mark.parametrize("wide,out", [(256, 2048), (208, 2040), (48, 2048), (1024, 1800), (64, 2304)])
def test_wide_tiles_one_after_the_other(api, typ, wide, out):
    """Tiles of 256 x 256, several a workgroup: 640 to 720 of them on 256 compute units, of one step of the sum and of many."""
    for turned in (False, True):
        if not (turned and typ == "i8"):
            product(api, typ, turned, RAGGED, 11, wide, out)


@pytest.mark.parametrize("typ", ["bf16", "fp16", "i8"])
def test_middle_tiles_one_after_the_other(api, typ):
    """Tiles of 128 x 128, 1200 and more of them, two a compute unit at a time."""
    counts = [100 + (e * 37) % 61 - 30 for e in range(200)]
    counts[7], counts[8] = 0, 300
    for turned in (False, True):
        if not (turned and typ == "i8"):
            product(api, typ, turned, counts, 5, 256, 768)
            product(api, typ, turned, counts, 0, 80, 760)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16", "i8"])
@pytest.mark.parametrize("wide,out", [(160, 64), (164, 64), (96, 48), (1024, 16)])
def test_narrow_tiles_one_after_the_other(api, typ, wide, out):
    """Tiles of 128 x 64, 1100 of them; 164 columns are whole chunks in fp32 alone, and come through registers otherwise."""
    product(api, typ, False, [1200 + (e * 131) % 400 for e in range(100)], 3, wide, out)
    if typ != "i8":
        product(api, typ, True, [1200 + (e * 131) % 400 for e in range(100)], 3, wide, out)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16", "i8"])
@pytest.mark.parametrize("wide,out,extra,at", [(101, 130, 0, 0), (101, 60, 2, 1), (64, 1, 1, 0), (1, 64, 0, 1), (3, 5, 0, 0), (7, 300, 1, 3), (257, 129, 0, 0),
                                               (128, 128, 1, 0), (164, 256, 3, 1), (33, 1030, 0, 0)])
def test_rows_of_any_alignment(api, typ, wide, out, extra, at):
    """Many rows an expert, whose operands are no whole aligned chunks: through registers, with last chunks that are moved, and rows too short for it."""
    for turned in (False, True):
        if not (turned and typ == "i8"):
            product(api, typ, turned, [3000, 0, 2500, 777, 1], 5, wide, out, extra, at)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "fp16", "i8"])
@pytest.mark.parametrize("wide,out", [(1024, 64), (1000, 33), (1601, 48)])
@pytest.mark.parametrize("mean,most", [(10, 0), (24, 0), (24, 500), (50, 0), (50, 1100)])
def test_few_rows_an_expert(api, typ, wide, out, mean, most):
    """One, two and four fragments of sixteen rows; one expert that has most of them."""
    experts = 30
    counts = [max(0, mean + (e * 7) % 11 - 5) for e in range(experts)]
    counts[3] = 0
    if most:
        counts = [most if e == 11 else (e % 3) * 10 for e in range(experts)]
    product(api, typ, False, counts, 4, wide, out)


@pytest.mark.parametrize("typ", ["bf16", "fp16", "fp32", "i8"])
@pytest.mark.parametrize("wide,out", [(256, 1024), (104, 72)])
def test_one_expert_has_nearly_all(api, typ, wide, out):
    """The form goes by the mean: whatever it is, the longest list is right."""
    for counts in ([1] * 20 + [30000] + [0] * 43, [5] * 500 + [6000] + [3] * 500):
        product(api, typ, False, counts, 2, wide, out)
        if typ != "i8":
            product(api, typ, True, counts, 2, wide, out)


def gradient(api, typ, counts, nobody, wide, out, extra=0, results=None):
    import torch
    gen = generator(wide * 3 + out)
    plan, owned = plan_of(api, counts, nobody), sum(counts)
    x, g = whole(gen, typ, owned + nobody, wide, extra=extra), whole(gen, typ, owned + nobody, out, extra=extra)
    x[owned:] = float("nan")
    g[owned:] = float("nan")
    want = torch.zeros(len(counts), out, wide, dtype=torch.float64, device="cuda")
    for e, (a, b) in enumerate(XO.bounds(plan.first.tolist(), owned)[:-1]):
        if b > a:
            want[e] = g[a:b].double().t().contiguous() @ x[a:b].double()
    for result in results or {typ, "fp32"}:
        before = whole(gen, result, len(counts), out, wide)
        for accumulate in (False, True):
            room = torch.full((len(counts), out, wide + 8), 5.0, dtype=of(result), device="cuda")
            d = room[:, :, :wide].copy_(before)
            api.fs_expert_matmul_backward(g, x, plan, d_w=d, accumulate=accumulate)
            expect = (want + before.double() if accumulate else want).float().to(of(result))
            assert torch.equal(d, expect), (result, accumulate, torch.nonzero(d != expect)[:5].tolist(), int((d != expect).sum()))
            assert bool((room[:, :, wide:] == 5.0).all())


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
@pytest.mark.parametrize("counts,wide,out", [([8000, 0, 2500, 1, 63, 64, 65, 1800, 1791, 1793, 1792, 700, 31, 2000, 100, 90], 1024, 1040),
                                             ([9000] + [2] * 14 + [0], 1024, 1032), ([300 + 40 * e for e in range(64)], 512, 520), ([33000, 7], 4096, 2056)])
def test_wide_tiles_of_the_weights_gradient(api, typ, counts, wide, out):
    """Tiles of 256 x 256, several a workgroup, of experts with one piece, none, and several whose sums are joined."""
    gradient(api, typ, counts, 9, wide, out)


@pytest.mark.parametrize("typ", ["bf16", "fp16"])
def test_wide_gradients_of_any_alignment(api, typ):
    gradient(api, typ, [4000, 0, 2500, 1, 63] + [500] * 11, 3, 1023, 1027, extra=1)


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("wide,out,extra", [(164, 256, 0), (164, 64, 0), (64, 1, 0), (1, 64, 0), (1, 1, 0), (130, 136, 0), (131, 133, 1)])
def test_gradients_of_narrow_weights(api, typ, wide, out, extra):
    """The widths of networks on feature rows, with an output layer of one column."""
    gradient(api, typ, [4000, 0, 9000, 1, 1200] + [700] * 25, 3, wide, out, extra=extra)


@pytest.mark.parametrize("typ", TYPES)
def test_gradients_of_as_many_experts_as_there_are(api, typ):
    """1024 lists, many of one length, most of them empty or in one piece."""
    counts = [(e * 37) % 19 for e in range(1024)]
    counts[0], counts[511], counts[1023] = 3000, 1700, 900
    gradient(api, typ, counts, 7, 40, 72)
    gradient(api, typ, [0] * 1023 + [5], 0, 136, 144)


@pytest.mark.parametrize("typ", ["fp32", "bf16", "i8"])
@pytest.mark.parametrize("pad", [0, 16])
def test_rows_far_apart(api, typ, pad):
    """Rows of x, of weights and of gradients 2^23 bytes and more apart: whole chunks, but beyond what a tile's loads reach from its first row."""
    import torch
    gen = generator(3)
    size = torch.empty(0, dtype=of(typ)).element_size()
    stride, wide, out, counts = (1 << 23) // size + pad, 64, 80, [150, 0, 145]
    plan, slots = plan_of(api, counts, 5), 300
    buf = torch.empty(slots * stride, dtype=of(typ), device="cuda")
    x = buf.as_strided((slots, wide), (stride, 1))
    x.copy_(whole(gen, typ, slots, wide))
    w = whole(gen, typ, 3, out, wide)
    want = exact(plan, x, w)
    if typ == "i8":
        one = torch.ones(slots, device="cuda")
        assert torch.equal(api.fs_expert_matmul_i8(x, one, plan, w, torch.ones(3, out, device="cuda")).double(), want)
        return
    y = torch.empty(slots, out, device="cuda")
    assert torch.equal(api.fs_expert_matmul(x, plan, w, out=y).double(), want)
    turned = buf[wide * 2:].as_strided((3, wide, out), (100 * stride, stride, 1))      # behind the rows of x, in the same memory
    turned.copy_(w.transpose(1, 2))
    assert torch.equal(api.fs_expert_matmul(x, plan, turned, turned=True, out=y).double(), want)
    g = whole(gen, typ, slots, out)
    d = torch.zeros(3, out, wide, dtype=torch.float64, device="cuda")
    for e, (a, b) in enumerate(XO.bounds(plan.first.tolist(), slots)[:-1]):
        d[e] = g[a:b].double().t().contiguous() @ x[a:b].double()
    assert torch.equal(api.fs_expert_matmul_backward(g, x, plan).double(), d)


@pytest.mark.parametrize("typ,step", [("fp16", -24), ("bf16", -133), ("fp32", -149)])
@pytest.mark.parametrize("counts,wide,out,at", [([3, 0, 5], 64, 48, 0), ([300, 200], 96, 144, 0), ([300, 200], 96, 144, 1), ([20000, 13], 256, 1024, 0), ([20000, 13], 255, 63, 0)])
def test_numbers_below_the_normal_ones(api, typ, step, counts, wide, out, at):
    """Operands of some of the type's smallest steps are not taken for 0, nor are such results."""
    import torch
    gen = generator(wide + at)
    plan, slots = plan_of(api, counts, 0), sum(counts)
    x, w = whole(gen, typ, slots, wide, extra=at, at=at), whole(gen, typ, len(counts), out, wide)
    want, d_want = exact(plan, x, w), torch.zeros(len(counts), out, wide, dtype=torch.float64, device="cuda")
    up = 0 if typ == "fp16" else 100
    small = x.double().mul(2.0 ** step).to(of(typ))
    assert float(small.abs().max()) == 2.0 ** (step + 1) and bool((small.double() == x.double() * 2.0 ** step).all())
    x.copy_(small)
    big = w * 2.0 ** up
    got = api.fs_expert_matmul(x, plan, big, out=torch.empty(slots, out, device="cuda"))
    assert torch.equal(got.double(), want * 2.0 ** (step + up))
    assert torch.equal(api.fs_expert_matmul(x, plan, big.transpose(1, 2).contiguous(), turned=True, out=got).double(), want * 2.0 ** (step + up))
    if typ == "fp16":                                    # results of the type, of some of its smallest steps
        assert torch.equal(api.fs_expert_matmul(x, plan, w).double(), want * 2.0 ** step)
    g = whole(gen, typ, slots, out)
    for e, (a, b) in enumerate(XO.bounds(plan.first.tolist(), slots)[:-1]):
        d_want[e] = g[a:b].double().t().contiguous() @ (x[a:b].double() * 2.0 ** up)
    assert torch.equal(api.fs_expert_matmul_backward(g * 2.0 ** up, x, plan).double(), d_want)
