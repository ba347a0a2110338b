"""Candidates that no family owns, scored by small networks instead of tree ensembles.

As in `mixture`, a router gives every statement row to k experts and its score is the weighted sum of theirs.  An expert is a network of
one hidden layer here, score = v . max(W x, 0), so that router and experts are trained together by what programs measured.  The rows that an
expert gets differ in number from expert to expert: its products are fs_expert_matmul's, its weights' gradients
fs_expert_matmul_backward's.  Where the families of rows are known, the router learns from them directly
(fs_distill_backward, which gives the losses too); for serving, the weights are laid out once in 8-bit integers.

The library does the work; this module only puts the calls in order.  PyTorch multiplies by the gate, clips at 0 and sums rows to programs.
"""
from __future__ import annotations

import math

import numpy as np


class NetworkMixture:
    """`dtype`: of rows and weights (fp32, bf16 or fp16); the gate, gradients and scores are fp32.  Training keeps what of 16-bit weights their type
    does not hold, in fp32 beside them, so that steps smaller than the type's add up."""

    def __init__(self, api, n_features: int, n_experts: int, hidden: int = 64, k: int = 2, dtype=None, seed: int = 0):
        import torch
        self.api, self.torch = api, torch
        self.dtype = dtype or torch.float32
        self.n_experts, self.k = n_experts, k
        self.params = api.route_params(n_experts, k, renormalise=True)
        gen = torch.Generator("cuda")
        gen.manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(*shape, device="cuda", generator=gen) * scale

        self.gate = normal(n_features, n_experts, scale=1 / math.sqrt(n_features))
        self.w = normal(n_experts, hidden, n_features, scale=math.sqrt(2 / n_features)).to(self.dtype)
        self.v = normal(n_experts, 1, hidden, scale=1 / math.sqrt(hidden)).to(self.dtype)
        self.rests = None
        self.served = None

    def route(self, rows):
        logits = rows.float() @ self.gate
        expert, weight = self.api.fs_route(self.params, logits)
        return logits, expert, weight, self.api.fs_expert_plan(expert, self.n_experts)

    def _programs(self, row_score, prog_off):
        lengths = (prog_off[1:] - prog_off[:-1]).long()
        if row_score.shape[0] == 0 or lengths.shape[0] == 0:
            return row_score.new_zeros(lengths.shape[0]), lengths
        return self.torch.segment_reduce(row_score[:, 0], "sum", lengths=lengths, initial=0.0), lengths

    def forward(self, rows, prog_off):
        """Scores of the programs of device rows [rows, n_features] of `dtype`, and what `gradients` needs of the way there."""
        api, torch = self.api, self.torch
        logits, expert, weight, plan = self.route(rows)
        x = api.fs_expert_gather(rows, plan)
        a = torch.relu(api.fs_expert_matmul(x, plan, self.w))
        y = torch.empty(x.shape[0], 1, device="cuda")
        api.fs_expert_matmul(a, plan, self.v, out=y)
        program, lengths = self._programs(api.fs_expert_combine(y, plan, weight), prog_off)
        return program, dict(rows=rows, logits=logits, expert=expert, weight=weight, plan=plan, x=x, a=a, y=y, lengths=lengths)

    def gradients(self, way, d_program):
        """(d_gate, d_w, d_v), fp32, of a loss whose gradient by the programs' scores is d_program.  What passes through the networks on the way is
        of their type; fp16's numbers end at 2^-24 and 2^16, so that there the results' gradient is brought to 16 at most, which leaves room
        for output weights of up to some thousand, and the weights' gradients back."""
        api, torch, plan = self.api, self.torch, way["plan"]
        d_rows = d_program.repeat_interleave(way["lengths"], output_size=way["rows"].shape[0])[:, None].contiguous()
        d_y, d_weight = api.fs_expert_combine_backward(d_rows, way["y"], plan, way["weight"])
        scaled = self.dtype == torch.float16 and d_y.shape[0] > 0
        if scaled:
            size = d_y.abs().amax().clamp(min=2.0 ** -100) / 16
            d_y = d_y / size
        d_y = d_y.to(self.dtype)
        d_v = api.fs_expert_matmul_backward(d_y, way["a"], plan)
        d_a = api.fs_expert_matmul(d_y, plan, self.v, turned=True) * (way["a"] > 0)
        d_w = api.fs_expert_matmul_backward(d_a, way["x"], plan)
        if scaled:
            d_v, d_w = d_v * size, d_w * size
        d_logits = api.fs_route_backward(self.params, way["logits"], way["expert"], d_weight)
        return way["rows"].float().t() @ d_logits, d_w, d_v

    def _move(self, w, rest, by):
        """Takes `by` from 16-bit weights w that `rest` was rounded off, in place; what is rounded off now.  A rest that w cannot have been rounded
        from is of other weights, which were there before."""
        whole = w.float() + rest
        whole = self.torch.where(whole.to(w.dtype) == w, whole, w.float()) - by
        w.copy_(whole)
        return whole - w.float()

    def step(self, rows, prog_off, target, rate: float = 0.002):
        """One step of gradient descent on the mean squared error against `target`; the loss before it, on the device."""
        program, way = self.forward(rows, prog_off)
        off = program - target
        d_gate, d_w, d_v = self.gradients(way, off * (2.0 / max(1, off.shape[0])))
        self.gate -= rate * d_gate
        if self.dtype == self.torch.float32:
            self.w -= rate * d_w
            self.v -= rate * d_v
        else:
            rests = self.rests or (0.0, 0.0)
            self.rests = self._move(self.w, rests[0], rate * d_w), self._move(self.v, rests[1], rate * d_v)
        self.served = None
        return (off * off).sum() / max(1, off.shape[0])

    def teach(self, rows, ids, teacher, total=None, rate: float = 0.5, temperature: float = 1.0):
        """One step of the router towards a teacher's choice: for every row experts `ids` [rows, k] (-1: none) and their logits; the mean
        loss before it, on the device."""
        api, torch = self.api, self.torch
        n = rows.shape[0]
        logits = rows.float() @ self.gate
        params = api.distill_params(self.n_experts, ids.shape[1], temperature, temperature * temperature)
        loss = torch.empty(n, device="cuda")
        d_loss = torch.full((n,), 1.0 / max(1, n), device="cuda")
        d_logits = api.fs_distill_backward(params, logits, ids, teacher, d_loss, total=total, loss=loss)
        self.gate -= rate * (rows.float().t() @ d_logits)
        return loss.sum() / max(1, n)

    def serve(self):
        """Lays the weights out in 8-bit integers, a scale for every channel."""
        laid = []
        for w in (self.w, self.v):
            e, o, i = w.shape
            q, scale = self.api.fs_quantize_rows(w.reshape(e * o, i))
            laid.append((q.view(e, o, i), scale.view(e, o)))
        self.served = laid

    def score_served(self, rows, prog_off):
        """Scores of the programs by 8-bit products."""
        api, torch = self.api, self.torch
        if self.served is None:
            self.serve()
        (w, w_scale), (v, v_scale) = self.served
        _, _, weight, plan = self.route(rows)
        q, scale = api.fs_expert_gather_i8(rows, plan)
        a = torch.relu(api.fs_expert_matmul_i8(q, scale, plan, w, w_scale, dtype=self.dtype))
        q, scale = api.fs_quantize_rows(a)
        y = api.fs_expert_matmul_i8(q, scale, plan, v, v_scale)
        return self._programs(api.fs_expert_combine(y, plan, weight), prog_off)[0]


def main():
    import time

    import torch
    from . import api
    from .mixture import make_study, targets_of
    _, models, features, off, member = make_study()
    x, o, target = targets_of(api, models, features, off, member)
    x = (x - x.mean(0)) / (x.std(0) + 1e-6)
    target = (target - target.mean()) / target.std()
    family = torch.from_numpy(np.repeat(member, np.diff(off))).cuda().int()
    mix = NetworkMixture(api, x.shape[1], len(models))
    for i in range(51):
        loss = mix.teach(x, family[:, None].contiguous(), torch.zeros(x.shape[0], 1, device="cuda"))
        if i % 25 == 0:
            print("router's step %3d  loss %.4f" % (i, float(loss)))
    losses, t0 = [], 0.0
    for i in range(201):
        if i == 1:
            torch.cuda.synchronize()
            t0 = time.perf_counter()
        losses.append(mix.step(x, o, target))
    torch.cuda.synchronize()
    print("%d programs, %d rows, %d networks: %.0f us a step" % (member.size, x.shape[0], len(models), (time.perf_counter() - t0) * 5e3))
    for i in range(0, 201, 40):
        print("step %3d  mean squared error %.4f" % (i, float(losses[i])))
    full, served = mix.forward(x, o)[0], mix.score_served(x, o)
    print("8 bits: scores off by %.4f of their spread" % float((full - served).std() / full.std()))


if __name__ == "__main__":
    main()
