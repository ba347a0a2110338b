"""Forms of the mixture's kernels that only large calls take: rows that leave past the caches, two tokens a lane, long sorts,
offsets of more than 32 bits.  Whole numbers where sums are compared bit for bit: fp32 holds all of them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2201_00194_amd import api as A
    return A


def torch_type(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


@pytest.mark.parametrize("typ,out_typ,rows,width,extra", [("fp32", "fp32", 1500003, 35, 0), ("fp32", "fp32", 60001, 877, 3), ("bf16", "bf16", 300002, 353, 1),
                                                          ("bf16", "fp32", 1000001, 53, 0), ("fp16", "fp16", 110001, 1001, 0), ("fp16", "fp32", 60002, 900, 8)])
def test_lookups_that_leave_past_the_caches(api, typ, out_typ, rows, width, extra):
    """200 MB of results and more.  One product, rounded as torch rounds it."""
    import torch
    gen = torch.Generator("cuda").manual_seed(rows)
    t = torch_type(out_typ)
    assert rows * width * t.itemsize >= 200 << 20
    table = torch.randn(3001, width + extra, device="cuda", generator=gen).to(torch_type(typ))[:, extra:]
    ids = torch.randint(-2, 3003, (rows,), device="cuda", generator=gen)
    buf = torch.full((rows, width + 2 * extra), 5.0, dtype=t, device="cuda")
    out = api.fs_embed(table, ids, scale=0.7, out=buf[:, extra:extra + width])
    there = (ids >= 0) & (ids < 3001)
    for a in range(0, rows, 200000):
        at = ids[a:a + 200000]
        want = (table[at.clamp(0, 3000)].float() * float(np.float32(0.7))).to(t)
        assert torch.equal(out[a:a + 200000], torch.where(there[a:a + 200000, None], want, 0))
    if extra:
        assert bool((buf[:, :extra] == 5).all()) and bool((buf[:, extra + width:] == 5).all())


@pytest.mark.parametrize("typ,tokens,k,width,extra", [("fp32", 500001, 3, 35, 0), ("fp16", 220001, 3, 164, 2), ("bf16", 130003, 4, 250, 0), ("fp32", 60001, 2, 501, 1),
                                                      ("bf16", 9001, 4, 1500, 0), ("fp32", 300001, 1, 175, 0)])
def test_exchanges_of_two_tokens_a_lane(api, typ, tokens, k, width, extra):
    """16 MB of results and more, an odd number of tokens, choices without a slot; all but one gather 200 MB and more too."""
    import torch
    gen = torch.Generator("cuda").manual_seed(tokens)
    t = torch_type(typ)
    assert tokens * width * t.itemsize >= 16 << 20
    expert = torch.randint(-1, 13, (tokens, k), device="cuda", generator=gen, dtype=torch.int32)
    expert[torch.rand(tokens, k, device="cuda", generator=gen) < 0.1] = 12
    p = api.fs_expert_plan(expert, 12)
    has = int(p.first[-1])
    there = (expert >= 0) & (expert < 12)
    assert has == int(there.sum())

    def rows(n):
        buf = torch.full((n, width + 2 * extra), 5.0, dtype=t, device="cuda")
        view = buf[:, extra:extra + width]
        view.copy_(torch.randn(n, width, device="cuda", generator=gen))
        return buf, view

    _, x = rows(tokens)
    buf, xs = rows(tokens * k)
    api.fs_expert_gather(x, p, xs)
    assert torch.equal(xs[:has], x[p.order[:has].long() // k]) and bool((xs[has:] == 0).all())
    assert not extra or (bool((buf[:, :extra] == 5).all()) and bool((buf[:, extra + width:] == 5).all()))

    _, y = rows(tokens * k)
    y[has:] = float("nan")
    w = torch.where(there, torch.randn(tokens, k, device="cuda", generator=gen), float("nan"))
    buf, out = rows(tokens)
    api.fs_expert_combine(y, p, w, out)
    _, g = rows(tokens)
    d_y, d_w = api.fs_expert_combine_backward(g, y, p, w)
    tiny = 2.0 ** -25 if typ == "fp16" else 1e-36
    for a in range(0, tokens, 50000):
        b = min(a + 50000, tokens)
        e, size = (torch.zeros(b - a, width, dtype=torch.float64, device="cuda") for _ in range(2))
        for j in range(k):
            on, at = there[a:b, j, None], p.place[a:b, j].clamp(min=0).long()
            v = torch.where(on, y[at].double() * w[a:b, j, None].double(), 0.0)
            e += v
            size += v.abs()
            gy = torch.where(on, g[a:b].double() * y[at].double(), 0.0)
            # a lane adds at most 256 products, then up to 64 lanes
            assert bool(((d_w[a:b, j].double() - gy.sum(dim=1)).abs() <= (256 + 8) * 2.0 ** -24 * gy.abs().sum(dim=1) + 1e-36).all())
            want = g[a:b].double() * w[a:b, j, None].double()
            assert bool(torch.where(on, (d_y[at].double() - want).abs() <= (2.0 ** -24 + HALF[typ] * (1 + 2.0 ** -24)) * want.abs() + tiny, True).all())
        off = k * 2.0 ** -24 * size
        assert bool(((out[a:b].double() - e).abs() <= off + HALF[typ] * (e.abs() + off) + tiny).all())
    assert bool((d_y[has:] == 0).all()) and bool((d_w[~there] == 0).all())
    assert not extra or (bool((buf[:, :extra] == 5).all()) and bool((buf[:, extra + width:] == 5).all()))


def whole_numbers(api, ids, g, vocab, accumulate=False, out_typ="fp32"):
    """The gradient of rows g of whole numbers, against index_add_ in 64 bits."""
    import torch
    rows, cols = ids.shape
    d = torch.full((vocab, g.shape[1]), 3.0, dtype=torch_type(out_typ), device="cuda")
    api.fs_embed_backward(g, ids if cols > 1 else ids[:, 0], vocab, scale=0.5, d_table=d, accumulate=accumulate)
    e = torch.zeros(vocab + 1, g.shape[1], dtype=torch.float64, device="cuda")
    at = torch.where((ids >= 0) & (ids < vocab), ids, vocab).long()
    for c in range(cols):
        e.index_add_(0, at[:, c], g.double())
    e = e[:vocab] * 0.5 + (3.0 if accumulate else 0.0)
    assert torch.equal(d.double(), e)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("rows,cols,vocab,width", [
    (8192, 1, 300000, 5),          # one workgroup sorts three digits
    (8192, 1, 600000, 9),          # and pairs of 64 bits
    (300, 27, 1 << 21, 3),
    (16384, 1, 700000, 64),        # 179 MB cleared beside it
    (9000, 1, 15624, 1024),        # just under and
    (9000, 1, 15625, 1024),        # as much as one workgroup's sort is worth it for
    (12001, 1, 250001, 64),
    (20000, 1, 1200000, 6),        # three passes over a long list
    (20000, 2, 1 << 20, 7),
    (70000, 3, 3000000, 2)])
def test_gradients_of_tables_with_many_rows(api, rows, cols, vocab, width, accumulate):
    import torch
    gen = torch.Generator("cuda").manual_seed(rows + vocab)
    ids = torch.randint(-1, vocab + 1, (rows, cols), device="cuda", generator=gen, dtype=torch.int32)
    ids[::3] = ids[0]                                                      # some tokens in many places
    ids[-1] = vocab - 1
    g = torch.randint(-8, 9, (rows, width), device="cuda", generator=gen).float()
    whole_numbers(api, ids, g, vocab, accumulate)


@pytest.mark.parametrize("typ,rows,cols,vocab,width", [("fp32", 20000, 1, 100, 20), ("fp32", 20000, 1, 600000, 20), ("fp32", 9000, 3, 50, 300),
                                                       ("bf16", 40000, 1, 77, 70), ("fp32", 200, 1, 50, 33), ("fp32", 20000, 90, 60, 130)])
def test_gradients_of_rows_far_apart(api, typ, rows, cols, vocab, width):
    """The rows of d_out reach past 4 GiB: their offsets need more than 32 bits."""
    import torch
    gen = torch.Generator("cuda").manual_seed(width)
    t = torch_type(typ)
    stride = (1 << 32) // t.itemsize // rows + 1000
    buf = torch.empty(rows * stride, dtype=t, device="cuda")
    g = buf.view(rows, stride)[:, 3:3 + width]
    g.copy_(torch.randint(-8, 9, (rows, width), device="cuda", generator=gen))
    ids = torch.randint(-1, vocab + 1, (rows, cols), device="cuda", generator=gen, dtype=torch.int32)
    assert (rows - 1) * stride * t.itemsize >= (1 << 32) - (1 << 30)
    whole_numbers(api, ids, g, vocab)


def test_gradient_of_few_wide_rows_that_many_ids_name(api):
    """Sorted by one workgroup, as so much is cleared beside it, and by bands, as the rows are wider together than a cache."""
    import torch
    gen = torch.Generator("cuda").manual_seed(5)
    ids = torch.randint(-1, 68, (200, 81), device="cuda", generator=gen, dtype=torch.int32)
    g = torch.randint(-8, 9, (200, 80000), device="cuda", generator=gen).to(torch.bfloat16)
    whole_numbers(api, ids, g, 67)
    whole_numbers(api, ids, g, 67, accumulate=True)
