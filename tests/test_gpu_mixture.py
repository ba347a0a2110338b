"""The mixture of family models against the same steps in 64 bits on the host, from the leaf ids and row scores of the scoring
oracle on.

Logits are products over `width` of sums over the map's trees, so they are off by (trees + width) * 2^-24 of their absolute sums
at most; where the reference's choices are further apart than that, the library's must be the same."""
import numpy as np
import pytest

from oracle import mixture_oracle as MO
from paper_2201_00194_amd import mixture as MX

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2201_00194_amd import api as A
    return A


@pytest.mark.parametrize("k", [1, 2, 4])
def test_scores_and_gradients_of_a_mixture(api, oracle, k):
    import torch
    map_model, models, X, off, member = MX.make_study(seed=3, families=4, programs=60, trees=12, depth=4)
    x, o, target = MX.targets_of(api, models, X, off, member)
    mix = MX.FamilyMixture(api, map_model, models, k=k, width=16, seed=1)
    program, way = mix.forward(x, o)
    d_program = torch.from_numpy(np.random.default_rng(5).standard_normal(member.size).astype(np.float32)).cuda()
    d_table, d_gate = mix.gradients(way, d_program)
    torch.cuda.synchronize()

    leaf = oracle.leaf_indices(map_model, X)
    assert np.array_equal(way["leaf"].cpu().numpy().view(np.uint16), leaf)
    table, gate = mix.table.cpu().double().numpy(), mix.gate.cpu().double().numpy()
    rows = MO.rows_of(leaf, map_model.tree_off[:-1], map_model.n_nodes)
    scale = float(np.float32(mix.leaf_scale))
    seen, seen_size = MO.embed(table, rows, scale)
    logits = seen @ gate
    off_logit = (map_model.n_trees + 16 + 4) * 2.0 ** -24 * (seen_size @ np.abs(gate))
    expert, weight = MO.route(logits, k, bias=np.zeros(4))
    sure = np.ones(X.shape[0], bool)
    ordered = np.sort(logits, axis=1)[:, ::-1]
    gaps = ordered[:, :-1] - ordered[:, 1:]
    sure = gaps[:, :min(k, 3)].min(axis=1) > 4 * off_logit.max(axis=1)
    assert sure.mean() > 0.99
    got = way["expert"].cpu().numpy()
    assert np.array_equal(got[sure], expert[sure])

    # From here on with the library's own choice, so that a tie cannot matter.
    _, order, place = MO.plan(got, 4)
    scores = np.stack([oracle.row_scores(m, X) for m in models]).astype(np.float64)
    y = np.where(order >= 0, scores[np.where(order >= 0, got.reshape(-1)[order], 0), order // k], 0.0)[:, None]
    assert np.array_equal(way["score"].cpu().numpy()[:, 0].astype(np.float64), y[:, 0])          # rows are scored bit for bit
    chosen = np.take_along_axis(logits, got.astype(np.int64), axis=1)
    w = np.exp(chosen - chosen.max(axis=1, keepdims=True))
    w /= w.sum(axis=1, keepdims=True)
    w_off = 4 * np.take_along_axis(off_logit, got.astype(np.int64), axis=1).max() + 120 * 2.0 ** -24
    assert np.all(np.abs(way["weight"].cpu().numpy() - w) <= w_off * w)
    row, row_size = MO.combine(y, place, w)
    exp = np.add.reduceat(row[:, 0], off[:-1])
    size = np.add.reduceat(row_size[:, 0], off[:-1])
    assert np.all(np.abs(program.cpu().numpy() - exp) <= (w_off + (k + 8) * 2.0 ** -24) * size + 1e-7)

    g = np.repeat(d_program.cpu().double().numpy(), np.diff(off))[:, None]
    _, dw, _ = MO.combine_backward(g, y, place, w)
    dl, dl_size = MO.route_backward(logits, got, dw)
    d_seen = dl @ gate.T
    exp_table, _ = MO.embed_backward(d_seen, rows, map_model.n_nodes, scale)
    _, table_size = MO.embed_backward(dl_size @ np.abs(gate).T, rows, map_model.n_nodes, scale)
    share = 8 * w_off + (16 + 4 + 514) * 2.0 ** -24
    assert np.all(np.abs(d_table.cpu().numpy() - exp_table) <= share * table_size + 1e-9)
    assert np.all(np.abs(d_gate.cpu().numpy() - seen.T @ dl) <= (share + X.shape[0] * 2.0 ** -24) * (seen_size.T @ dl_size) + 1e-9)


def test_training_sends_rows_to_their_families(api):
    import torch
    map_model, models, X, off, member = MX.make_study(seed=7, families=3, programs=150, trees=15, depth=4)
    x, o, target = MX.targets_of(api, models, X, off, member)
    mix = MX.FamilyMixture(api, map_model, models, k=2, width=32, seed=2)
    losses = [float(mix.step(x, o, target, rate=0.2, balance=1e-3)) for _ in range(40)]
    assert losses[-1] < losses[0]
    assert torch.isfinite(mix.table).all() and torch.isfinite(mix.gate).all()


def test_rows_that_cannot_be_laid_side_by_side_are_refused(api):
    from paper_2201_00194_amd import workloads as W
    f = W.make_small_family(seed=1, n_programs=4, stmts=(1, 2), n_trees=2, depth=2, n_features=6)
    with pytest.raises(ValueError):
        MX.FamilyMixture(api, f.model, [f.model])
