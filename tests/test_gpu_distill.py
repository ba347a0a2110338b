"""Distillation from a teacher's largest logits and its gradient against the definition in 64 bits.

The kernel adds a row's exp(x - m) in fp32: each exponential is off by at most 2^-22 of itself (the difference, its product with
log2(e) / T, the hardware's exponential) plus 2^-23 for each unit of |x - m| in the exponent -- together less than
(4 + 100) * 2^-23 where it counts, as terms with x - m < -100 are nothing beside the largest -- and sums of n terms by n * 2^-24, of which
a thread adds at most n / 64.  The log of such a sum is off by as much absolutely, and everything else is added in 64 bits; so a loss is off by
at most that of the entries' sizes, and a gradient by that of what is added up in it and half a step of its type."""
import numpy as np
import pytest

from oracle import experts_oracle as XO

pytestmark = pytest.mark.gpu
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LEAST = {"fp32": 1e-37, "bf16": 1e-37, "fp16": 2.0 ** -25}


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2201_00194_amd import api as A
    return A


def of(typ):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[typ]


def study(seed, rows, classes, k, typ, spread=3.0, extra=0, at=0, temperature=1.0):
    """A student's logits (rows `extra` further apart, `at` into memory), a teacher's k largest and the log of its sum of all."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    buf = torch.full((rows * (classes + extra) + at,), 5.0, device="cuda", dtype=of(typ))
    x = buf[at:].view(rows, classes + extra)[:, :classes]
    x.copy_(torch.randn(rows, classes, generator=gen, device="cuda") * spread)
    full = x.float() + torch.randn(rows, classes, generator=gen, device="cuda")
    best = torch.topk(full, k, dim=1)
    total = torch.logsumexp(full.double() / temperature, dim=1).float()
    d_loss = torch.randn(rows, generator=gen, device="cuda")
    return x, best.indices, best.values, total, d_loss


def check(api, x, ids, teacher, d_loss, total=None, temperature=1.0, scale=1.0):
    import torch
    rows, classes = x.shape
    typ = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}[x.dtype]
    p = api.distill_params(classes, ids.shape[1], temperature, scale)
    room = torch.full((rows, classes + 3), 7.0, device="cuda", dtype=x.dtype)
    d = room[:, :classes]
    beside = torch.full((rows,), 9.0, device="cuda")
    loss = api.fs_distill(p, x, ids, teacher, total)
    assert api.fs_distill_backward(p, x, ids, teacher, d_loss, total, loss=beside, d_logits=d) is d
    assert torch.equal(api.fs_distill_backward(p, x, ids, teacher, d_loss, total), d.contiguous())
    assert bool((room[:, classes:] == 7.0).all())
    t32 = float(np.float32(temperature))
    el, sl, eg, sg = XO.distill(x.double().cpu().numpy(), ids.cpu().numpy(), teacher.double().cpu().numpy(), t32, float(np.float32(scale)),
                                None if total is None else total.double().cpu().numpy(), d_loss.double().cpu().numpy())
    share = (104 * 2 + classes / 64 + 64) * 2.0 ** -24
    for got in (loss, beside):
        off = np.abs(got.double().cpu().numpy() - el)
        assert np.all(off <= (share + 2.0 ** -23) * sl + 2.0 ** -24 * np.abs(el) + 1e-37), (np.argmax(off / (sl + 1e-30)), np.max(off / (sl + 1e-30)))
    off = np.abs(d.double().cpu().numpy() - eg)
    # The hardware's exponential has no results below 2^-126: where a class's is one, its gradient loses less than the row's factor
    # d_loss * scale / T times 2^-126 (a sum is 1 at least).
    lost = np.abs(d_loss.double().cpu().numpy() * scale / t32)[:, None] * 2.0 ** -126
    bound = (2 * share + 2.0 ** -22) * sg + HALF[typ] * (np.abs(eg) + (2 * share + 2.0 ** -22) * sg) + LEAST[typ] + lost
    assert np.all(off <= bound), (np.argwhere(off > bound)[:5], np.max(off / bound))


SIZES = [(1, 1, 1), (3, 2, 1), (5, 7, 3), (4, 30, 8), (64, 64, 8), (65, 63, 5), (7, 255, 16), (6, 256, 256), (9, 257, 20), (33, 1000, 64), (3, 1024, 1024), (3, 2049, 1000),
         (2, 4097, 64), (2, 32001, 20), (1, 100000, 33)]


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,classes,k", SIZES)
def test_losses_and_gradients(api, typ, rest, rows, classes, k):
    x, ids, teacher, total, d_loss = study(rows + classes, rows, classes, k, typ)
    check(api, x, ids, teacher, d_loss, total if rest else None)


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("temperature,scale,extra,at", [(2.0, 4.0, 0, 0), (0.5, 1.0, 3, 1), (0.1, -1.5, 8, 8), (37.0, 0.0, 1, 0), (1.0, 65536.0, 0, 3)])
def test_temperatures_scales_and_strides(api, typ, temperature, scale, extra, at):
    import torch
    x, ids, teacher, total, d_loss = study(3, 12, 515, 9, typ, extra=extra, at=at, temperature=temperature)
    for some in (None, total):
        check(api, x, ids, teacher, d_loss, some, temperature, scale)
        check(api, x, ids.int(), teacher.bfloat16(), d_loss, some, temperature, scale)
        check(api, x, ids.int(), teacher.half(), d_loss, some, temperature, scale)


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("temperature", [1e-20, 1e30])
@pytest.mark.parametrize("classes", [20, 5000, 140000])
def test_far_temperatures(api, typ, temperature, classes):
    x, ids, teacher, total, d_loss = study(5, 6, classes, 9, typ, temperature=temperature)
    for some in (None, total):
        check(api, x, ids, teacher, d_loss, some, temperature, temperature)


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("classes", [20, 700, 5000])
def test_masks_short_lists_and_bad_entries(api, typ, rest, classes):
    import torch
    x, ids, teacher, total, d_loss = study(classes, 24, classes, 6, typ)
    inf, nan = float("inf"), float("nan")
    x[0] = -inf                                         # no class at all
    x[1] = nan
    x[2, ::2] = -inf                                    # masks that take entries with them
    x[3, 1::2] = nan
    x[4].fill_(-inf).scatter_(0, ids[4], 1.5)           # nothing but the entries
    x[5] = -inf
    x[5, int(ids[5, 2])] = 0.25                         # one entry, and nothing else
    x[6].scatter_(0, ids[6], -inf)                      # no entry that the student may take
    ids[7] = -1                                         # no list
    ids[8, 2:] = -1
    ids[9, 1], ids[9, 4] = classes, 1 << 40
    teacher[10] = -inf
    teacher[11, 3], teacher[11, 0] = nan, -inf
    teacher[12, 1] = inf
    x[13, 5] = inf                                      # the largest float
    x[14, 0], x[14, 1] = inf, inf
    total[15], total[16], total[17] = nan, inf, -inf
    total[18] -= 3                                      # entries of more than all: no rest is left
    d_loss[19] = 0
    x[20] = torch.finfo(x.dtype).min                    # the type's lowest value everywhere
    x[21, ::3] = torch.finfo(x.dtype).min
    d_loss[[0, 1, 6, 7, 10]] = nan                      # of rows without a loss
    got = api.fs_distill_backward(api.distill_params(classes, 6), x, ids, teacher, d_loss, total if rest else None)
    assert bool((got[[0, 1, 6, 7, 10]] == 0).all()) and bool(torch.isfinite(got).all())
    d_loss = torch.nan_to_num(d_loss)
    check(api, x, ids, teacher, d_loss, total if rest else None)


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("rest", [False, True])
def test_a_class_named_more_than_once(api, typ, rest):
    x, ids, teacher, total, d_loss = study(8, 10, 90, 12, typ)
    ids[:, 7] = ids[:, 2]
    ids[3] = ids[3, 0]
    ids[4, 6:] = ids[4, :6]
    check(api, x, ids, teacher, d_loss, total + 1 if rest else None)


@pytest.mark.parametrize("typ", list(HALF))
def test_far_apart_and_near_one(api, typ):
    """Shares of the rest near 0 and near 1, logits hundreds apart, and students that have learned all."""
    import torch
    for spread in (0.01, 30.0, 300.0):
        x, ids, teacher, total, d_loss = study(6, 16, 600, 10, typ, spread=spread)
        check(api, x, ids, teacher, d_loss, total)
        check(api, x, ids, teacher, d_loss)
        own = torch.topk(x.float(), 10, dim=1)
        check(api, x, own.indices, own.values, d_loss, torch.logsumexp(x.double(), 1).float())
        check(api, x, own.indices, own.values, d_loss)


@pytest.mark.parametrize("rest", [False, True])
def test_gradient_against_differences(api, rest):
    """Central differences over h = 2^-4 of an oracle-free loss: its third derivative is below 2 in size, so they are off by h^2 / 3,
    and by the losses' own rounding over 2 h."""
    import torch
    x, ids, teacher, total, _ = study(2, 4, 40, 5, "fp32", spread=1.0)
    p = api.distill_params(40, 5, 1.0, 1.0)
    some = total if rest else None
    d = api.fs_distill_backward(p, x, ids, teacher, torch.ones(4, device="cuda"), some)
    h = 2.0 ** -4
    for c in list(range(0, 40, 7)) + ids[0].tolist():
        up, down = x.clone(), x.clone()
        up[:, c] += h
        down[:, c] -= h
        slope = (api.fs_distill(p, up, ids, teacher, some).double() - api.fs_distill(p, down, ids, teacher, some).double()) / (2 * h)
        assert bool(((slope - d[:, c].double()).abs() <= h * h / 3 + 64 * 2.0 ** -23 / h).all())


def test_a_routers_choice_as_the_teacher(api):
    """fs_route's choices, shorter lists among them, with the logits that they were made of."""
    import torch
    x, _, _, _, d_loss = study(5, 50, 24, 4, "fp32")
    teacher = torch.randn(50, 24, device="cuda")
    teacher[::3, 3:] = -float("inf")
    expert, _ = api.fs_route(api.route_params(24, 4), teacher)
    assert bool((expert < 0).any())
    check(api, x, expert, teacher.gather(1, expert.clamp(min=0).long()), d_loss)


def test_rows_beyond_32_bit_offsets(api):
    import torch
    rows, classes = 34000, 65536
    x = torch.zeros(rows, classes, dtype=torch.bfloat16, device="cuda")
    some = [0, 1, 32767, 32768, rows - 1]
    part, ids, teacher, total, d_loss = study(4, 5, classes, 8, "bf16")
    x[some] = part
    all_ids = torch.zeros(rows, 8, dtype=torch.int32, device="cuda")
    all_ids[some] = ids.int()
    all_t = torch.zeros(rows, 8, device="cuda")
    all_t[some] = teacher
    w = torch.zeros(rows, device="cuda")
    w[some] = d_loss
    p = api.distill_params(classes, 8)
    loss = torch.empty(rows, device="cuda")
    d = api.fs_distill_backward(p, x, all_ids, all_t, w, loss=loss)
    small = torch.empty(5, device="cuda")
    ds = api.fs_distill_backward(p, part, ids, teacher, d_loss, loss=small)
    share = (104 * 2 + classes / 64 + 64) * 2.0 ** -24 * 40          # two ways of adding the same row
    assert bool(((loss[some] - small).abs() <= share).all())
    assert bool(((d[some].float() - ds.float()).abs() <= (share + 2.0 ** -7) * ds.float().abs() + 1e-30).all()) and bool((d[100] == 0).all())


def test_the_most_classes(api):
    import torch
    n = api.FS_MAX_CLASSES
    for rest in (False, True):
        x, ids, teacher, total, d_loss = study(1, 1, n, 50, "bf16")
        check(api, x, ids, teacher, d_loss, total if rest else None)
    with pytest.raises(api.FsError) as e:
        api.fs_distill(api.distill_params(n + 1, 4), torch.zeros(1, n + 1, device="cuda"), torch.zeros(1, 4, device="cuda").int(), torch.zeros(1, 4, device="cuda"))
    assert e.value.code == api.FS_EUNSUPPORTED


def test_other_streams_and_graphs(api):
    """Captured calls of two graphs, replayed in turn with eager ones between them."""
    import torch
    sets = []
    for seed, rows, classes in ((1, 40, 300), (2, 3, 70000)):
        x, ids, teacher, total, d_loss = study(seed, rows, classes, 8, "bf16")
        p = api.distill_params(classes, 8)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        loss = api.fs_distill(p, x, ids, teacher, total, stream=s)
        d = api.fs_distill_backward(p, x, ids, teacher, d_loss, total, stream=s)
        s.synchronize()
        assert torch.equal(d, api.fs_distill_backward(p, x, ids, teacher, d_loss, total))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            api.fs_distill(p, x, ids, teacher, total, loss=loss)
            api.fs_distill_backward(p, x, ids, teacher, d_loss, total, d_logits=d)
        sets.append((graph, p, x, ids, teacher, total, d_loss, loss, d))
    for i in range(4):
        for graph, p, x, ids, teacher, total, d_loss, loss, d in sets:
            x.copy_(torch.randn(x.shape, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(loss, api.fs_distill(p, x, ids, teacher, total))
            assert torch.equal(d, api.fs_distill_backward(p, x, ids, teacher, d_loss, total))


def test_results_are_the_same_again(api):
    import torch
    for rows, classes in ((200, 1000), (2, 90000)):
        x, ids, teacher, total, d_loss = study(9, rows, classes, 30, "bf16")
        ids[:, 5] = ids[:, 9]
        p = api.distill_params(classes, 30)
        a, b = api.fs_distill(p, x, ids, teacher, total), api.fs_distill_backward(p, x, ids, teacher, d_loss, total)
        for _ in range(3):
            assert torch.equal(a, api.fs_distill(p, x, ids, teacher, total)) and torch.equal(b, api.fs_distill_backward(p, x, ids, teacher, d_loss, total))


def test_refusals_reach_the_caller(api):
    import torch
    p = api.distill_params(16, 4)
    x, ids, t, w = torch.zeros(8, 16, device="cuda"), torch.zeros(8, 4, device="cuda").int(), torch.zeros(8, 4, device="cuda"), torch.zeros(8, device="cuda")
    assert api.fs_distill(p, x[:0], ids[:0], t[:0]).shape == (0,)
    assert api.fs_distill_backward(p, x[:0], ids[:0], t[:0], w[:0]).shape == (0, 16)
    for call in (lambda: api.fs_distill(p, x[:, :15], ids, t), lambda: api.fs_distill(p, x, ids[:, :3], t), lambda: api.fs_distill(p, x, ids, t[:7]),
                 lambda: api.fs_distill(p, x, ids.float(), t), lambda: api.fs_distill(p, x, ids.short(), t), lambda: api.fs_distill(p, x, ids, t.double()),
                 lambda: api.fs_distill(p, x, ids, t, total=w[:4]), lambda: api.fs_distill(p, x, ids, t, loss=w.half()), lambda: api.fs_distill(p, x.cpu(), ids, t),
                 lambda: api.fs_distill(p, x, ids.cpu(), t), lambda: api.fs_distill(p, x.t().contiguous().t(), ids, t),
                 lambda: api.fs_distill_backward(p, x, ids, t, w[:4]), lambda: api.fs_distill_backward(p, x, ids, t, w, d_logits=x.half()),
                 lambda: api.fs_distill_backward(p, x, ids, t, None), lambda: api.fs_distill(api.distill_params(16, 4, temperature=0.0), x, ids, t)):
        with pytest.raises(api.FsError):
            call()
