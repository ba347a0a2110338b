"""fs_embed and fs_embed_backward against the definition in 64 bits.

A bag's sum of n fp32 values is off by at most n * 2^-24 of their absolute sum, the scale rounds once.  The table's gradient
adds at most 512 values one after the other in fp32, whatever a token's count, and the rest in 64 bits."""
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


def torch_type(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def matrix(rng, rows, width, typ, extra=0, at=0):
    import torch
    stride = width + extra
    buf = torch.full((rows * stride + at + stride,), 5.0, dtype=torch_type(typ), device="cuda")
    view = buf[at: at + rows * stride].view(rows, stride)[:, :width]
    view.copy_(torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).to(torch_type(typ)))
    return buf, view


def untouched(buf, view):
    mask = buf.clone()
    rows, width = view.shape
    mask[view.storage_offset(): view.storage_offset() + rows * view.stride(0)].view(rows, -1)[:, :width] = 5.0
    return bool((mask == 5.0).all())


def make_ids(rng, rows, cols, vocab, kind, bad=0.05):
    """(numpy ids, torch ids, base or None)"""
    import torch
    if kind == "leaf16":
        per = max(1, vocab // cols)
        ids = rng.integers(0, min(per + 2, 65536), (rows, cols))
        base = (np.arange(cols) * per).astype(np.int32)
        return ids, torch.from_numpy(ids.astype(np.uint16).view(np.int16)).cuda(), base
    ids = (rng.random((rows, cols)) ** 3 * vocab).astype(np.int64)
    out = rng.random((rows, cols)) < bad
    ids[out] = rng.choice([-1, -7, vocab, vocab + 3, 2147483647, -2147483648], out.sum())
    if kind == "int64":
        ids[rng.random((rows, cols)) < bad / 2] = (1 << 32) + 1        # not token 1
    t = torch.from_numpy(ids.astype(np.int32 if kind == "int32" else np.int64)).cuda()
    return ids, t, None


SHAPES = [(1, 1, 1, 1), (1, 1, 10, 64), (5, 1, 7, 3), (64, 1, 1000, 16), (300, 1, 50, 17), (200, 1, 3000, 256), (33, 1, 40, 1000), (20, 1, 65, 2048),
          (1, 100, 1270, 64), (1, 3, 9, 5), (37, 8, 100, 32), (320, 30, 930, 16), (130, 100, 6300, 64), (70, 7, 49, 33), (11, 300, 9000, 128),
          (3, 1000, 4000, 8)]


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("kind", ["int32", "int64", "leaf16"])
@pytest.mark.parametrize("rows,cols,vocab,width", SHAPES)
def test_lookup_and_bags(api, typ, kind, rows, cols, vocab, width):
    import torch
    rng = np.random.default_rng(rows + cols + width)
    ids, t, base = make_ids(rng, rows, cols, vocab, kind)
    where = MO.rows_of(ids, base, vocab)
    b = None if base is None else torch.from_numpy(base).cuda()
    for extra, at in ((0, 0), (3, 1), (8, 8)):
        _, table = matrix(rng, vocab, width, typ, extra, at)
        for out_typ in dict.fromkeys((typ, "fp32")):
            buf, out = matrix(rng, rows, width, out_typ, extra, at)
            api.fs_embed(table, t.view(-1) if cols == 1 else t, scale=0.7, col_base=b, out=out)
            scale = float(np.float32(0.7))
            exp, size = MO.embed(table.cpu().double().numpy(), where, scale)
            off = (cols + 1) * 2.0 ** -24 * size
            tiny = 2.0 ** -25 if out_typ == "fp16" else 1e-36
            assert np.all(np.abs(out.cpu().double().numpy() - exp) <= off + HALF[out_typ] * (np.abs(exp) + off) + tiny)
            assert untouched(buf, out)


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("kind", ["int32", "int64", "leaf16"])
@pytest.mark.parametrize("rows,cols,vocab,width", SHAPES + [(5000, 1, 5, 24), (3000, 4, 2, 8), (2000, 1, 200000, 4), (9000, 2, 1100, 40), (700, 30, 930, 65)])
def test_gradient(api, typ, kind, rows, cols, vocab, width):
    import torch
    rng = np.random.default_rng(rows + cols + width + 1)
    ids, t, base = make_ids(rng, rows, cols, vocab, kind)
    where = MO.rows_of(ids, base, vocab)
    b = None if base is None else torch.from_numpy(base).cuda()
    t = t.view(-1) if cols == 1 else t
    for extra, at in ((0, 0), (3, 1), (8, 8)):
        _, g = matrix(rng, rows, width, typ, extra, at)
        exp, size = MO.embed_backward(g.cpu().double().numpy(), where, vocab, float(np.float32(0.7)))
        off = 514 * 2.0 ** -24 * size
        for out_typ in dict.fromkeys((typ, "fp32")):
            tiny = 2.0 ** -25 if out_typ == "fp16" else 1e-36
            for accumulate in (False, True):
                buf, d = matrix(rng, vocab, width, out_typ, extra, at)
                before = d.cpu().double().numpy().copy() if accumulate else 0.0
                api.fs_embed_backward(g, t, vocab, scale=0.7, col_base=b, d_table=d, accumulate=accumulate)
                e = exp + before
                more = off + 2.0 ** -24 * (np.abs(exp) + np.abs(e))
                assert np.all(np.abs(d.cpu().double().numpy() - e) <= more + HALF[out_typ] * (np.abs(e) + more) + tiny)
                assert untouched(buf, d)


@pytest.mark.parametrize("rows,vocab", [(70000, 3), (100000, 1), (65537, 70000)])
def test_gradient_of_long_runs(api, rows, vocab):
    """One token nearly everywhere: its run is split, and the sum is the same from run to run."""
    import torch
    gen = torch.Generator("cuda").manual_seed(rows)
    ids = torch.zeros(rows, dtype=torch.int64, device="cuda")
    some = torch.rand(rows, device="cuda", generator=gen) < 0.1
    ids[some] = torch.randint(0, vocab, (int(some.sum()),), device="cuda", generator=gen)
    g = torch.randn(rows, 20, device="cuda", generator=gen)
    d = api.fs_embed_backward(g, ids, vocab, scale=0.5)
    exp = torch.zeros(vocab, 20, dtype=torch.float64, device="cuda").index_add_(0, ids, g.double()) * 0.5
    size = torch.zeros(vocab, 20, dtype=torch.float64, device="cuda").index_add_(0, ids, g.double().abs()) * 0.5
    assert bool(((d.double() - exp).abs() <= 516 * 2.0 ** -24 * size).all())
    assert torch.equal(d, api.fs_embed_backward(g, ids, vocab, scale=0.5))


@pytest.mark.parametrize("typ,rows,cols,vocab,width", [("fp32", 17000, 20, 700, 64), ("bf16", 70001, 7, 1500, 40), ("fp16", 41000, 9, 610, 65),
                                                       ("fp32", 4500, 100, 900, 256), ("fp32", 130000, 3, 60, 60)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_many_rows(api, typ, rows, cols, vocab, width, accumulate):
    """More rows than an XCD's L2 cache holds, each token named often: rows are taken in bands."""
    import torch
    gen = torch.Generator("cuda").manual_seed(rows)
    ids = torch.randint(-1, vocab + 1, (rows, cols), device="cuda", generator=gen, dtype=torch.int32)
    g = torch.randn(rows, width, device="cuda", generator=gen).to(torch_type(typ))
    there = (ids >= 0) & (ids < vocab)
    exp, size = (torch.zeros(vocab + 1, width, dtype=torch.float64, device="cuda") for _ in range(2))
    for c in range(cols):
        at = torch.where(there[:, c], ids[:, c], vocab).long()
        exp.index_add_(0, at, g.double())
        size.index_add_(0, at, g.double().abs())
    exp, size = exp[:vocab] * 0.5, size[:vocab] * 0.5
    for out_typ in dict.fromkeys((typ, "fp32")):
        d = torch.ones(vocab, width, dtype=torch_type(out_typ), device="cuda")
        api.fs_embed_backward(g, ids, vocab, scale=0.5, d_table=d, accumulate=accumulate)
        e = exp + 1 if accumulate else exp
        off = 520 * 2.0 ** -24 * size + 2.0 ** -23 * (e.abs() + exp.abs())
        assert bool(((d.double() - e).abs() <= off + HALF[out_typ] * (e.abs() + off)).all())
        again = torch.ones_like(d)
        api.fs_embed_backward(g, ids, vocab, scale=0.5, d_table=again, accumulate=accumulate)
        assert torch.equal(d, again)


@pytest.mark.parametrize("typ", list(HALF))
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 3), (64, 1), (65, 1), (85, 3), (255, 1), (256, 1), (257, 1), (1, 256), (128, 2)])
@pytest.mark.parametrize("vocab,width", [(1, 5), (3, 8), (40, 1), (300, 91), (9000, 12), (70, 1100)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_few_ids(api, typ, rows, cols, vocab, width, accumulate):
    """Few ids, every one of them once, or a token many times: at most 256 additions in fp32, a factor, a sum with what was there."""
    import torch
    gen = torch.Generator("cuda").manual_seed(rows * 1000 + vocab)
    ids = torch.randint(-1, vocab + 1, (rows, cols), device="cuda", generator=gen, dtype=torch.int32)
    g = torch.randn(rows, width + 1, device="cuda", generator=gen).to(torch_type(typ))[:, 1:]
    exp, size = (torch.zeros(vocab + 1, width, dtype=torch.float64, device="cuda") for _ in range(2))
    for c in range(cols):
        at = torch.where((ids[:, c] >= 0) & (ids[:, c] < vocab), ids[:, c], vocab).long()
        exp.index_add_(0, at, g.double())
        size.index_add_(0, at, g.double().abs())
    exp, size = exp[:vocab] * 0.5, size[:vocab] * 0.5
    for out_typ in dict.fromkeys((typ, "fp32")):
        buf = torch.ones(vocab, width + 3, dtype=torch_type(out_typ), device="cuda")
        d = api.fs_embed_backward(g, ids if cols > 1 else ids[:, 0], vocab, scale=0.5, d_table=buf[:, 1:width + 1], accumulate=accumulate)
        e = exp + 1 if accumulate else exp
        off = 258 * 2.0 ** -24 * size + 2.0 ** -23 * (e.abs() + exp.abs())
        tiny = 2.0 ** -25 if out_typ == "fp16" else 1e-36
        assert bool(((d.double() - e).abs() <= off + HALF[out_typ] * (e.abs() + off) + tiny).all())
        assert bool((buf[:, 0] == 1).all()) and bool((buf[:, width + 1:] == 1).all())


@pytest.mark.parametrize("rows,vocab,width", [(8192, 40000, 4), (8193, 40000, 4), (16384, 900, 33), (16384, 45001, 1024), (9001, 45001, 1024), (16385, 45001, 1024)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_at_the_borders_of_the_sorts(api, rows, vocab, width, accumulate):
    """One workgroup or several sort, and the table is cleared beside one kernel or in parts beside several."""
    import torch
    gen = torch.Generator("cuda").manual_seed(rows)
    ids = torch.randint(-1, vocab + 1, (rows,), device="cuda", generator=gen, dtype=torch.int64)
    g = torch.randn(rows, width, device="cuda", generator=gen)
    exp, size = (torch.zeros(vocab + 1, width, dtype=torch.float64, device="cuda") for _ in range(2))
    at = torch.where((ids >= 0) & (ids < vocab), ids, vocab)
    exp.index_add_(0, at, g.double())
    size.index_add_(0, at, g.double().abs())
    d = torch.full((vocab, width), 2.0, device="cuda")
    api.fs_embed_backward(g, ids, vocab, d_table=d, accumulate=accumulate)
    e = exp[:vocab] + (2 if accumulate else 0)
    assert bool(((d.double() - e).abs() <= 516 * 2.0 ** -24 * size[:vocab] + 2.0 ** -23 * e.abs()).all())


def test_few_ids_captured_into_a_graph(api):
    import torch
    ids = torch.randint(0, 90, (200,), device="cuda", dtype=torch.int64)
    g = torch.randn(200, 33, device="cuda")
    d = api.fs_embed_backward(g, ids, 90)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.fs_embed_backward(g, ids, 90, d_table=d)
    for _ in range(3):
        ids.copy_(torch.randint(0, 90, (200,)))
        g.copy_(torch.randn(200, 33))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(d, api.fs_embed_backward(g, ids, 90))


def test_gradient_against_differences(api):
    """out is linear in the table."""
    import torch
    rng = np.random.default_rng(2)
    ids = torch.from_numpy(rng.integers(0, 30, (25, 4)).astype(np.int32)).cuda()
    table = torch.from_numpy(rng.standard_normal((30, 6)).astype(np.float32)).cuda()
    g = torch.from_numpy(rng.standard_normal((25, 6)).astype(np.float32)).cuda()
    d = api.fs_embed_backward(g, ids, 30, scale=0.25)
    for v, c in ((0, 0), (13, 5), (29, 2)):
        h = torch.zeros_like(table)
        h[v, c] = 0.5
        up = (api.fs_embed(table + h, ids, scale=0.25).double() * g.double()).sum()
        down = (api.fs_embed(table - h, ids, scale=0.25).double() * g.double()).sum()
        assert abs(float(up - down) - float(d[v, c])) < 25 * 6 * 4 * 2.0 ** -21


def test_ids_of_a_scored_ensemble(api, oracle):
    """Leaf ids as fs_score_families writes them, tree offsets as fs_model_create takes them."""
    import torch
    from paper_2201_00194_amd import workloads as W
    f = W.make_small_family(seed=5, n_programs=60, stmts=(1, 9), n_trees=21, depth=5, early_leaf_q=0.2, k=4)
    dev = api.DeviceFamily(f, want_leaf_idx=True)
    api.fs_score_families([dev.family()])
    leaf = dev.leaf_idx.view(f.n_rows, f.model.n_trees)
    base = torch.from_numpy(np.ascontiguousarray(f.model.tree_off[:-1], dtype=np.int32)).cuda()
    n = int(f.model.tree_off[-1])
    value = torch.from_numpy(np.ascontiguousarray(f.model.value, dtype=np.float32)).cuda()
    sums = api.fs_embed(value.view(n, 1), leaf, col_base=base)           # leaf values for vectors: the rows' scores
    exp = oracle.row_scores(f.model, f.features) - np.float32(f.model.bias)
    np.testing.assert_allclose(sums.cpu().numpy()[:, 0], exp, atol=22 * 2.0 ** -24 * float(np.abs(f.model.value).max()) * 21 + 2.0 ** -23)


def test_infinities_and_nan_stay_where_they_are(api):
    import torch
    table = torch.randn(10, 12, device="cuda")
    table[3] = float("nan")
    table[4] = float("inf")
    ids = torch.tensor([[0, 1], [3, 1], [4, 0], [-1, -1], [11, 2]], dtype=torch.int32, device="cuda")
    out = api.fs_embed(table, ids)
    assert torch.equal(out[0], table[0] + table[1]) and bool(out[1].isnan().all()) and bool(out[2].isinf().all())
    assert bool((out[3] == 0).all()) and torch.equal(out[4], table[2])
    g = torch.randn(5, 12, device="cuda")
    g[3] = float("nan")                                            # a row of padding only
    d = api.fs_embed_backward(g, ids, 10)
    assert bool(d.isfinite().all()) and torch.equal(d[2], g[4]) and bool((d[5:] == 0).all())


def test_tables_beyond_32_bit_offsets(api):
    import torch
    vocab, width = 600000, 4096
    table = torch.zeros(vocab, width, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, 524288 + 5, vocab - 1, 17], dtype=torch.int64, device="cuda")
    table[ids] = torch.randn(4, width, device="cuda").to(torch.bfloat16)
    assert torch.equal(api.fs_embed(table, ids), table[ids])
    g = table[ids].clone()
    table.fill_(1.0)
    api.fs_embed_backward(g, ids, vocab, d_table=table)
    assert torch.equal(table[ids], g)
    assert int((table != 0).any(dim=1).sum()) == 4


def test_other_streams_and_graphs(api):
    import torch
    table = torch.randn(500, 64, device="cuda")
    ids = torch.randint(0, 500, (400, 9), device="cuda", dtype=torch.int32)
    g = torch.randn(400, 64, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = api.fs_embed(table, ids, stream=s)
    d = api.fs_embed_backward(g, ids, 500, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.fs_embed(table, ids, out=out)
        api.fs_embed_backward(g, ids, 500, d_table=d)
    for _ in range(3):
        ids.copy_(torch.randint(0, 500, (400, 9), dtype=torch.int32))
        g.copy_(torch.randn(400, 64))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, api.fs_embed(table, ids)) and torch.equal(d, api.fs_embed_backward(g, ids, 500))


def test_nothing_to_look_up(api):
    import torch
    table = torch.randn(6, 4, device="cuda")
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert api.fs_embed(table, none).shape == (0, 4)
    g = torch.zeros(0, 4, device="cuda")
    assert bool((api.fs_embed_backward(g, none, 6) == 0).all())
    d = table.clone()
    api.fs_embed_backward(g, none, 6, d_table=d, accumulate=True)
    assert torch.equal(d, table)


def test_refusals_reach_the_caller(api):
    import torch
    table, ids = torch.randn(6, 4, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for call in (lambda: api.fs_embed(table.double(), ids), lambda: api.fs_embed(table, ids.float()), lambda: api.fs_embed(table.t(), ids),
                 lambda: api.fs_embed(table, ids, scale=float("nan")), lambda: api.fs_embed(table, ids, out=torch.empty(3, 5, device="cuda")),
                 lambda: api.fs_embed(table, ids, out=torch.empty(3, 4, device="cuda", dtype=torch.float16)),
                 lambda: api.fs_embed(table, ids, col_base=torch.zeros(2, dtype=torch.int32, device="cuda")),
                 lambda: api.fs_embed_backward(table, ids, 6), lambda: api.fs_embed_backward(table[:3], ids, 0),
                 lambda: api.fs_embed_backward(table[:3], ids, 6, accumulate=True)):
        with pytest.raises(api.FsError):
            call()


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,width", [(1, 300001, 1), (2, 300000, 8), (3, 300000, 512), (1, 2000003, 512), (70, 100000, 130)])
def test_long_bags(api, typ, rows, cols, width):
    """Values of one sign, the same in every row of the table: what fp32 loses of them does not average out.  At most 256 are added in
    fp32 one after the other, then in 64 bits; joining up to 64 lanes' sums, the factor and the result round eight times more."""
    import torch
    gen = torch.Generator("cuda").manual_seed(cols + width)
    value = (torch.rand(width, device="cuda", generator=gen) + 0.1).to(torch_type(typ))
    table = value.expand(700, width).contiguous()
    ids = torch.randint(0, 703, (rows, cols), device="cuda", generator=gen, dtype=torch.int32)
    out = api.fs_embed(table, ids, scale=0.7, out=torch.empty(rows, width, device="cuda"))
    exp = (ids < 700).sum(dim=1, dtype=torch.float64)[:, None] * value.double() * float(np.float32(0.7))
    assert bool(((out.double() - exp).abs() <= (256 + 8) * 2.0 ** -24 * exp).all()), float((out.double() / exp - 1).abs().max())


@pytest.mark.parametrize("rows,cols", [(3, 1), (100, 2), (300, 3), (9000, 1), (20000, 2)])
def test_ids_and_bases_whose_sum_alone_fits(api, rows, cols):
    """The row is the column's base plus the id, also where the id by itself has more than 32 bits."""
    import torch
    vocab = 40
    base = torch.tensor([-2147483648, 2147483647, -5][:cols], dtype=torch.int32, device="cuda")
    row = torch.randint(-3, vocab + 3, (rows, cols), device="cuda")
    ids = row - base.long()
    far = torch.rand(rows, cols, device="cuda") < 0.2
    ids = torch.where(far & (row % 2 == 0), 9223372036854775807, torch.where(far, -9223372036854775807 - 1, ids))
    at = torch.where(far | (row < 0) | (row >= vocab), vocab, row)
    table = torch.randint(-9, 10, (vocab + 1, 12), device="cuda").float()
    table[vocab] = 0
    out = api.fs_embed(table[:vocab], ids, col_base=base)
    assert torch.equal(out, table[at].sum(dim=1))
    g = torch.randint(-9, 10, (rows, 12), device="cuda").float()          # sums of whole numbers are exact
    d = api.fs_embed_backward(g, ids, vocab, col_base=base)
    exp = torch.zeros(vocab + 1, 12, dtype=torch.float64, device="cuda")
    for c in range(cols):
        exp.index_add_(0, at[:, c], g.double())
    assert torch.equal(d.double(), exp[:vocab])


def test_the_longest_bag(api):
    """2^31 - 1 ids in one bag: the first, the last and those where its 64 parts meet are in the sum, and nothing behind them."""
    import torch
    n = 2147483647
    ids = torch.zeros(n + 1, dtype=torch.int16, device="cuda")
    per = (n + 63) // 64
    at = torch.tensor([0, 1, n - 1, n - 2] + [p * per + d for p in range(1, 64) for d in (-1, 0)], device="cuda")
    ids[at] = 1
    ids[n] = 2
    table = torch.tensor([[0.0], [1.0], [float("nan")]], device="cuda")
    assert float(api.fs_embed(table, ids[:n].view(1, n))) == at.numel()


def test_tables_of_more_rows_than_32_bits_hold_are_refused(api):
    """They would be taken for tables of the low 32 bits' rows."""
    import torch
    many = (1 << 32) + 5
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")
    for call in (lambda: api.fs_embed(torch.empty(many, 1, dtype=torch.bfloat16, device="cuda"), ids),
                 lambda: api.fs_embed_backward(torch.zeros(3, 1, device="cuda"), ids, many),
                 lambda: api.fs_expert_plan(torch.zeros(3, 1, dtype=torch.int32, device="cuda"), (1 << 32) + 8)):
        with pytest.raises(api.FsError):
            call()
    with pytest.raises(api.FsError):                        # no rows at all
        api.fs_expert_combine_backward(torch.zeros((), device="cuda"), torch.zeros(3, 1, device="cuda"),
                                       api.fs_expert_plan(torch.zeros(3, 1, dtype=torch.int32, device="cuda"), 2), torch.ones(3, 1, device="cuda"))
