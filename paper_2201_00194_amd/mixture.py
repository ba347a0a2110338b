"""Candidates that no family owns: a learned mixture of the family models scores them.

The tuner finds a subgraph's family by static analysis (Section 4.1; find_family in Algorithm 1) and
lets that family's model estimate the candidates.  Candidates of a subgraph whose family is not known
have no such model.  Here every statement row is sent to the k family models that a router chooses,
and its score is the weighted sum of theirs.  The router sees a row by the leaves that it reaches in
one ensemble of its own (the *map*): the scaled sum of the leaves' learned vectors, times a gate, are the
logits.  Vectors and gate are trained on measured programs; a bias per family, moved by how often the
family was asked, balances the families and is in no weight.

The library does the work -- trees, embedding, routing, exchange and their gradients; this module only
puts the calls in order.  PyTorch multiplies by the gate and sums rows to programs.
"""
from __future__ import annotations

import math
from typing import Sequence

import numpy as np

from . import workloads as W


class FamilyMixture:
    """`map_model` and `models`: host `workloads.Model`s over the same features, whose number is a multiple of 4."""

    def __init__(self, api, map_model: W.Model, models: Sequence[W.Model], k: int = 2, width: int = 64, scale: float = 1.0,
                 seed: int = 0):
        import torch
        if map_model.n_features % 4 or any(m.n_features != map_model.n_features for m in models):
            raise ValueError("the models need the same number of features, a multiple of 4")
        self.api, self.torch = api, torch
        self.n_features, self.width = map_model.n_features, width
        self.map = api.fs_model.from_arrays(map_model)
        self.models = [api.fs_model.from_arrays(m) for m in models]
        self.leaf_base = torch.from_numpy(np.ascontiguousarray(map_model.tree_off[:-1], dtype=np.int32)).cuda()
        self.leaf_scale = 1.0 / math.sqrt(max(1, map_model.n_trees))
        self.params = api.route_params(len(models), k, renormalise=True, scale=scale)
        gen = torch.Generator("cuda")
        gen.manual_seed(seed)
        self.table = torch.randn(map_model.n_nodes, width, device="cuda", generator=gen)
        self.gate = torch.randn(width, len(models), device="cuda", generator=gen) / math.sqrt(width)
        self.bias = torch.zeros(len(models), device="cuda")

    def _one_row_programs(self, model, x, out, leaf=None):
        """Every row of x a program, whose scores go to `out`."""
        n_rows = x.shape[0]
        off = self.torch.arange(n_rows + 1, device="cuda", dtype=self.torch.int32)
        return self.api.Family(model, x, self.api.FS_ROWMAJOR, n_rows, off, out, leaf_idx=leaf)

    def forward(self, features, prog_off):
        """Scores of the programs of row-major device features [rows, n_features], and what `step` needs of the way there."""
        api, torch = self.api, self.torch
        n_rows = features.shape[0]
        leaf = torch.empty(n_rows, self.map.n_trees, dtype=torch.int16, device="cuda")
        api.fs_score_families([self._one_row_programs(self.map, features, torch.empty(n_rows, device="cuda"), leaf)])
        seen = api.fs_embed(self.table, leaf, scale=self.leaf_scale, col_base=self.leaf_base)
        logits = seen @ self.gate
        expert, weight = api.fs_route(self.params, logits, self.bias)
        plan = api.fs_expert_plan(expert, len(self.models))
        rows = api.fs_expert_gather(features, plan)
        first = plan.first.cpu().tolist()                 # the families' row counts: the library takes them from the host
        score = torch.zeros(n_rows * self.params.k, 1, device="cuda")
        fams = []
        for m, a, b in zip(self.models, first, first[1:]):
            if b > a:
                fams.append(self._one_row_programs(m, rows[a:b], score[a:b]))
        api.fs_score_families(fams)
        row_score = api.fs_expert_combine(score, plan, weight)
        lengths = (prog_off[1:] - prog_off[:-1]).long()
        program = torch.segment_reduce(row_score[:, 0], "sum", lengths=lengths, initial=0.0)
        return program, dict(leaf=leaf, seen=seen, logits=logits, expert=expert, weight=weight, plan=plan, score=score, lengths=lengths)

    def gradients(self, way, d_program):
        """(d_table, d_gate) of a loss whose gradient by the programs' scores is d_program."""
        api = self.api
        d_rows = d_program.repeat_interleave(way["lengths"], output_size=way["seen"].shape[0])[:, None].contiguous()
        _, d_weight = api.fs_expert_combine_backward(d_rows, way["score"], way["plan"], way["weight"])
        d_logits = api.fs_route_backward(self.params, way["logits"], way["expert"], d_weight)
        d_seen = d_logits @ self.gate.t()
        d_table = api.fs_embed_backward(d_seen, way["leaf"], self.table.shape[0], scale=self.leaf_scale, col_base=self.leaf_base)
        return d_table, way["seen"].t() @ d_logits

    def step(self, features, prog_off, target, rate: float = 0.1, balance: float = 0.0):
        """One step of gradient descent on the mean squared error against `target`; the loss before it, on the device."""
        torch = self.torch
        program, way = self.forward(features, prog_off)
        off = program - target
        d_table, d_gate = self.gradients(way, off * (2.0 / max(1, off.shape[0])))
        self.table -= rate * d_table
        self.gate -= rate * d_gate
        if balance:
            load = (way["plan"].first[1:] - way["plan"].first[:-1]).float()
            self.bias += balance * torch.sign(load.mean() - load)
        return (off * off).mean()


def make_study(seed: int = 0, families: int = 4, programs: int = 400, trees: int = 30, depth: int = 5):
    """(map model, family models, features, program offsets, family of each program): families differ in the level of a few
    columns."""
    rng = np.random.default_rng([seed, 4242])
    parts, models, member = [], [], []
    for f in range(families):
        fam = W.make_small_family(seed=seed * 100 + f, n_programs=programs, stmts=(1, 8), n_trees=trees, depth=depth)
        fam.features[:, 8 * f: 8 * f + 8] += 1.0
        parts.append(fam)
        models.append(fam.model)
        member.append(np.full(programs, f))
    features = np.concatenate([p.features for p in parts])
    lengths = np.concatenate([np.diff(p.prog_off) for p in parts])
    member = np.concatenate(member)
    order = rng.permutation(member.size)                         # programs of all families mixed
    starts = np.concatenate(([0], np.cumsum(lengths)))
    rows = np.concatenate([np.arange(starts[p], starts[p + 1]) for p in order])
    features, lengths, member = np.ascontiguousarray(features[rows]), lengths[order], member[order]
    off = np.concatenate(([0], np.cumsum(lengths))).astype(np.int32)
    map_model = W.draw_model(rng, features, 40, 4)
    return map_model, models, features, off, member


def targets_of(api, models, features, off, member):
    """Every program's score under its own family's model."""
    import torch
    x, o = torch.from_numpy(features).cuda(), torch.from_numpy(off).cuda()
    scores = []
    for m in models:
        out = torch.empty(off.size - 1, device="cuda")
        handle = api.fs_model.from_arrays(m)
        api.fs_score_families([api.Family(handle, x, api.FS_ROWMAJOR, features.shape[0], o, out)])
        torch.cuda.synchronize()
        scores.append(out)
    return x, o, torch.stack(scores)[torch.from_numpy(member).cuda(), torch.arange(off.size - 1, device="cuda")]


def main():
    import time

    import torch
    from . import api
    map_model, models, features, off, member = make_study()
    x, o, target = targets_of(api, models, features, off, member)
    mix = FamilyMixture(api, map_model, models, k=2, width=32)
    losses, t0 = [], 0.0
    for i in range(101):
        if i == 1:
            torch.cuda.synchronize()
            t0 = time.perf_counter()
        losses.append(mix.step(x, o, target, rate=0.2, balance=1e-3))
    torch.cuda.synchronize()
    print("%d programs, %d rows, %d families: %.0f us a step" % (member.size, x.shape[0], len(models), (time.perf_counter() - t0) * 1e4))
    for i in range(0, 101, 20):
        print("step %3d  mean squared error %.4f" % (i, float(losses[i])))
    score, _ = mix.forward(x, o)
    idx = torch.empty(16, dtype=torch.int32, device="cuda")
    api.fs_topk([api.TopkRequest(score, score.shape[0], 16, idx)])
    true = set(torch.topk(target, 16).indices.tolist())
    print("of the 16 best programs, %d are among the mixture's 16" % len(true & set(idx.tolist())))


if __name__ == "__main__":
    main()
