"""Work for the operators that let a learned router share statement rows out over the family models, for timing.

A search meets subgraphs whose family is not known.  A router then gives every statement row (a token) the k
family models (experts) that score it and their weights, from logits that are a product of the row's learned
embedding with a gate; the embedding is the scaled sum of learned vectors of the leaves that the row reaches in
an ensemble.  Rows travel to the experts' slots and their results come back, weighted.  Training sends gradients
the same way backwards.

Kinds of a case:
  route           logits to the k chosen experts and their weights
  route_train     that, and the logits' gradient from the weights'
  exchange        the plan of slots, rows to the slots, the experts' results back to the rows
  exchange_train  that, and the gradients of results, weights and rows
  embed           tokens to scaled vectors, or bags of tokens to scaled sums of vectors
  embed_grad      the gradient of the table
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2, "int32": 4, "int64": 8, "leaf16": 2}
_BIG = torch.finfo(torch.float32).max

# ---- the cases -----------------------------------------------------------------------------------

_ROUTE = {"kind": "route", "rows": 4096, "experts": 64, "k": 4, "type": "fp32", "score": "softmax", "renormalise": True,
          "bias": False, "groups": 1, "top_groups": 1, "group_best": 1, "scale": 1.0, "masked": 0.0}
_EXCHANGE = {"kind": "exchange", "rows": 32768, "experts": 30, "k": 2, "width": 164, "type": "fp32", "masked": 0.0}
_EMBED = {"kind": "embed", "rows": 4096, "bag": 1, "vocab": 50000, "width": 256, "type": "bf16", "ids": "int64",
          "scale": 1.0}


def listed():
    return [
        # one statement row asks thirty family models for their say: the latency of a call
        dict(_ROUTE, name="route_one", rows=1, experts=30),
        # the rows of a pool of 320 programs, 64 families, some of them without a model yet (masked)
        dict(_ROUTE, name="route_pool", rows=5120, experts=64, k=4, masked=0.2),
        # two million rows over 64 families in groups, balanced by a bias
        dict(_ROUTE, name="route_groups", rows=2000000, experts=64, k=8, type="bf16", score="sigmoid", bias=True, groups=8,
             top_groups=4, group_best=2, scale=2.5),
        # many experts, odd in number, as a router of fine-grained experts has them; training
        dict(_ROUTE, name="route_train_many", kind="route_train", rows=32768, experts=255, k=8, type="fp16", bias=True),
        # a training step's rows over 30 families, the weights not renormalised: a dense gradient
        dict(_ROUTE, name="route_train", kind="route_train", rows=262144, experts=30, k=4, renormalise=False),
        # the smallest exchange: a handful of rows
        dict(_EXCHANGE, name="exchange_few", rows=8, experts=8),
        # feature rows of a 4096-program population to their families and scores' vectors back
        dict(_EXCHANGE, name="exchange_rows", rows=32768, experts=30, k=4),
        # a training step on hidden rows of an ordinary width
        dict(_EXCHANGE, name="exchange_train", kind="exchange_train", rows=65536, experts=64, k=4, width=1024, type="bf16", masked=0.1),
        # the rows of one pool, leaves of a 100-tree ensemble of depth 6
        dict(_EMBED, name="embed_pool", rows=320, bag=100, vocab=12700, width=64, type="fp32", ids="leaf16", scale=0.1),
        # a long batch of single tokens, a wide table
        dict(_EMBED, name="embed_tokens", rows=131072, bag=1, vocab=65536, width=1024, scale=32.0),
        # the leaves' vectors of 32768 rows in a 100-tree ensemble
        dict(_EMBED, name="embed_grad_leaves", kind="embed_grad", rows=32768, bag=100, vocab=12700, width=64, type="fp32",
             ids="leaf16", scale=0.1),
        # a training step's tokens, a table of which most rows get nothing
        dict(_EMBED, name="embed_grad_tokens", kind="embed_grad", rows=16384, bag=1, vocab=65536, width=1024, scale=32.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("route", "route", "route_train", "exchange", "exchange_train", "embed", "embed", "embed_grad", "embed_grad"))
    typ = rng.choice(("fp32", "bf16", "fp16"))
    if kind.startswith("route"):
        rows = _log_int(rng, 1, 1000000)
        groups = rng.choice((1, 1, 2, 4, 8))
        per = _log_int(rng, 8 if groups == 1 else 4, 256 // groups)
        experts = groups * per
        while rows * experts > 64000000:
            rows //= 2
        top = groups if groups == 1 else rng.randint(1, groups)
        return dict(_ROUTE, kind=kind, rows=rows, experts=experts, k=rng.randint(1, min(8, top * per)), type=typ,
                    score=rng.choice(("softmax", "sigmoid")), renormalise=rng.random() < 0.6, bias=rng.random() < 0.5, groups=groups,
                    top_groups=top, group_best=rng.choice((1, 2)), scale=rng.choice((1.0, 2.5)), masked=rng.choice((0.0, 0.0, 0.3)))
    if kind.startswith("exchange"):
        rows, width, k = _log_int(rng, 1, 262144), _log_int(rng, 1, 2048), rng.randint(1, 8)
        while rows * k * width > 200000000:
            rows //= 2
        return dict(_EXCHANGE, kind=kind, rows=rows, experts=_log_int(rng, 8, 256), k=k, width=width, type=typ, masked=rng.choice((0.0, 0.2)))
    if rng.random() < 0.5:
        bag, depth = _log_int(rng, 8, 300), rng.randint(3, 8)
        rows, width = _log_int(rng, 1, 32768), _log_int(rng, 8, 128)
        while rows * bag * width > 200000000:
            rows //= 2
        return dict(_EMBED, kind=kind, rows=max(1, rows), bag=bag, vocab=bag * ((2 << depth) - 1), width=width, type=typ, ids="leaf16",
                    scale=round(1 / math.sqrt(bag), 4))
    rows, width, vocab = _log_int(rng, 1, 262144), _log_int(rng, 8, 2048), _log_int(rng, 1000, 131072)
    while rows * width > 100000000:
        rows //= 2
    while vocab * width > 100000000:
        vocab //= 2
    return dict(_EMBED, kind=kind, rows=rows, vocab=vocab, width=width, type=typ, ids=rng.choice(("int32", "int64")),
                scale=rng.choice((1.0, round(math.sqrt(width), 4))))


def _distinct(case):
    """How many rows of the table a call meets, as prepare() draws its tokens."""
    ids, vocab = case["rows"] * case["bag"], case["vocab"]
    if case["ids"] == "leaf16":
        return min(ids, case["bag"] * (vocab // case["bag"] // 2 + 1))
    rank = torch.arange(1, vocab + 1, dtype=torch.float64)
    return int((1 - torch.exp(-ids * torch.log1p(1 / rank) / math.log(vocab))).sum())


def work(case):
    b = _BYTES[case["type"]]
    if case["kind"].startswith("route"):
        n, slots = case["rows"] * case["experts"], case["rows"] * case["k"]
        w = {"bytes": n * b + slots * 8 + (4 * case["experts"] if case["bias"] else 0), "flops": 4 * n}
        if case["kind"] == "route_train":       # the weights' gradient in, the logits' out; the logits need not be read twice
            w = {"bytes": w["bytes"] + slots * 4 + n * b, "flops": w["flops"] + 4 * n}
        return w
    if case["kind"].startswith("exchange"):
        rows, slots = case["rows"] * case["width"], case["rows"] * case["k"] * case["width"]
        lists = case["rows"] * case["k"] * 4
        w = {"bytes": (2 * rows + 2 * slots) * b + 4 * lists + 4 * (case["experts"] + 1), "flops": 2 * slots}
        if case["kind"] == "exchange_train":    # out's gradient in, the results' and the weights' out; slots' rows in, the rows' out
            w = {"bytes": w["bytes"] + (2 * rows + 2 * slots) * b + lists, "flops": w["flops"] + 4 * slots}
        return w
    ids = case["rows"] * case["bag"]
    table = case["vocab"] if case["kind"] == "embed_grad" else _distinct(case)
    size = 4 if case["kind"] == "embed_grad" else b
    return {"bytes": ids * _BYTES[case["ids"]] + table * case["width"] * size + case["rows"] * case["width"] * b,
            "flops": 2 * ids * case["width"]}


# ---- what a program has in hand ------------------------------------------------------------------


def _popular(shape, vocab, gen, dev):
    """Tokens whose counts fall with their rank as in a text, the ranks scattered over the table."""
    rank = (torch.exp(torch.rand(shape, generator=gen, device=dev, dtype=torch.float64) * math.log(vocab)) - 1).long().clamp_(0, vocab - 1)
    return torch.randperm(vocab, generator=gen, device=dev)[rank]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 7919 + 17)
    t = _TYPES[case["type"]]
    s = {"case": case}
    rows = case["rows"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    if case["kind"].startswith("route"):
        e, k = case["experts"], case["k"]
        logits = normal(rows, e) * 1.5 + normal(e) * 0.5             # some experts are asked more often
        if case["masked"]:
            logits[:, torch.rand(e, generator=gen, device=dev) < case["masked"]] = -math.inf
            logits[torch.rand(rows, generator=gen, device=dev) < 0.01] = -math.inf     # rows that no expert may take
        s["logits"] = logits.to(t)
        s["bias"] = normal(e) * 0.05 if case["bias"] else None
        s["d_weight"] = normal(rows, k)
        s["groups"] = torch.arange(e, device=dev) // (e // case["groups"])
        if own:
            from paper_2201_00194_amd import api
            s["params"] = api.route_params(
                e, k, score=api.FS_SCORE_SIGMOID if case["score"] == "sigmoid" else api.FS_SCORE_SOFTMAX,
                renormalise=case["renormalise"], n_groups=case["groups"], top_groups=case["top_groups"],
                group_best=case["group_best"], scale=case["scale"])
    elif case["kind"].startswith("exchange"):
        e, k, d = case["experts"], case["k"], case["width"]
        wish = normal(rows, e) + normal(e) * 0.5
        s["expert"] = torch.sort(wish, dim=1, descending=True).indices[:, :k].to(torch.int32).contiguous()
        if case["masked"]:
            s["expert"][torch.rand(rows, generator=gen, device=dev) < case["masked"], k - 1] = -1   # fewer than k experts were to be had
        s["x"] = normal(rows, d).to(t)
        s["y"] = normal(rows * k, d).to(t)
        s["weight"] = torch.softmax(normal(rows, k), dim=1)
        s["d_out"] = normal(rows, d).to(t)
        s["d_xs"] = normal(rows * k, d).to(t)
    else:
        bag, vocab = case["bag"], case["vocab"]
        if case["ids"] == "leaf16":              # leaf ids of each tree, which count from the tree's own root
            per = vocab // bag
            leaf = (torch.rand(rows, bag, generator=gen, device=dev) ** 2 * (per // 2 + 1)).long() + (per // 2)
            s["ids"] = leaf.to(torch.int16)
            s["base"] = torch.arange(bag, device=dev, dtype=torch.int32) * per
        else:
            s["ids"] = _popular((rows,), vocab, gen, dev).to(torch.int32 if case["ids"] == "int32" else torch.int64)
            s["base"] = None
        if case["kind"] == "embed":
            s["table"] = normal(vocab, case["width"]).to(t)
        else:
            s["d_out"] = normal(rows, case["width"]).to(t)
    return s


# ---- one pass ------------------------------------------------------------------------------------


def run(state):
    kind = state["case"]["kind"]
    if kind.startswith("route"):
        return _own_route(state) if own else _plain_route(state)
    if kind.startswith("exchange"):
        return _own_exchange(state) if own else _plain_exchange(state)
    return _own_embed(state) if own else _plain_embed(state)


def _own_route(s):
    from paper_2201_00194_amd import api
    expert, weight = api.fs_route(s["params"], s["logits"], bias=s["bias"])
    if s["case"]["kind"] == "route":
        return {"expert": expert, "weight": weight}
    return {"expert": expert, "weight": weight, "d_logits": api.fs_route_backward(s["params"], s["logits"], expert, s["d_weight"])}


def _own_exchange(s):
    from paper_2201_00194_amd import api
    plan = api.fs_expert_plan(s["expert"], s["case"]["experts"])
    out = {"first": plan.first, "order": plan.order, "place": plan.place, "xs": api.fs_expert_gather(s["x"], plan),
           "out": api.fs_expert_combine(s["y"], plan, s["weight"])}
    if s["case"]["kind"] == "exchange_train":
        out["d_y"], out["d_weight"] = api.fs_expert_combine_backward(s["d_out"], s["y"], plan, s["weight"])
        out["d_x"] = api.fs_expert_combine(s["d_xs"], plan)
    return out


def _own_embed(s):
    from paper_2201_00194_amd import api
    c = s["case"]
    if c["kind"] == "embed":
        return api.fs_embed(s["table"], s["ids"], scale=c["scale"], col_base=s["base"])
    return api.fs_embed_backward(s["d_out"], s["ids"], c["vocab"], scale=c["scale"], col_base=s["base"])


def _plain_route(s):
    """Which experts: in 64 bits, since scores meet at the cut.  A masked expert's logit is -inf (or NaN)."""
    c, k = s["case"], s["case"]["k"]
    x = s["logits"].double()
    x = torch.where(torch.isnan(x), -math.inf, x).clamp(max=_BIG)
    top = x.max(dim=1, keepdim=True).values
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    if c["score"] == "softmax":
        log_score = x - top - torch.log(torch.exp(x - top).sum(dim=1, keepdim=True))
    else:
        log_score = torch.clamp(x, max=0) - torch.log1p(torch.exp(-torch.abs(x)))
    score = torch.where(torch.isneginf(x), 0.0, torch.exp(log_score))
    key = x if s["bias"] is None else torch.where(torch.isneginf(x), -math.inf, score + s["bias"].double())
    key = torch.where(torch.isnan(key), -math.inf, key)
    if c["groups"] > 1:
        of_group = torch.where(torch.isneginf(key), -math.inf, score if s["bias"] is None else key)
        best = torch.sort(of_group.view(c["rows"], c["groups"], -1), dim=2, descending=True).values[:, :, :c["group_best"]]
        none = torch.isneginf(best[:, :, 0])
        best = torch.where(none, -math.inf, torch.where(torch.isneginf(best), 0.0, best).sum(dim=2))
        rank = torch.sort(best, dim=1, descending=True, stable=True).indices
        taken = torch.zeros_like(none).scatter_(1, rank[:, :c["top_groups"]], True)
        key = torch.where(taken[:, s["groups"]], key, -math.inf)
    key, expert = torch.sort(key, dim=1, descending=True, stable=True)
    key, expert = key[:, :k], expert[:, :k]
    there = ~torch.isneginf(key)
    chosen = torch.where(there, log_score.gather(1, expert), -math.inf)
    if c["renormalise"]:
        high = chosen.max(dim=1, keepdim=True).values
        chosen = chosen - torch.where(torch.isinf(high), torch.zeros_like(high), high)
        total = torch.exp(chosen).sum(dim=1, keepdim=True)
        share = torch.exp(chosen) / torch.where(total > 0, total, torch.ones_like(total))
    else:
        share = torch.exp(chosen)
    out = {"expert": torch.where(there, expert, -1).to(torch.int32), "weight": (share * c["scale"]).float()}
    if c["kind"] == "route_train":
        share, dw = share.float(), torch.where(there, s["d_weight"], 0.0)
        if c["renormalise"]:
            g = share * (dw - (share * dw).sum(dim=1, keepdim=True))
            if c["score"] == "sigmoid":
                g = g * (1 - score).float().gather(1, expert)
            d = torch.zeros(x.shape, device=x.device).scatter_add_(1, expert, torch.where(there, g, 0.0))
        else:
            g = torch.zeros(x.shape, device=x.device).scatter_add_(1, expert, dw)
            p = score.float()
            d = p * (g - (p * g).sum(dim=1, keepdim=True)) if c["score"] == "softmax" else g * p * (1 - p)
        out["d_logits"] = (d * c["scale"]).to(s["logits"].dtype)
    return out


def _plain_exchange(s):
    c, expert = s["case"], s["expert"].reshape(-1).long()
    slots, k, e, t = expert.numel(), c["k"], c["experts"], s["x"].dtype
    there = expert >= 0
    order = torch.sort(torch.where(there, expert, e), stable=True).indices
    filled = there[order]
    place = torch.empty_like(order).scatter_(0, order, torch.arange(slots, device=order.device))
    first = torch.zeros(e + 1, dtype=torch.long, device=order.device)
    first[1:] = torch.cumsum((expert[:, None] == torch.arange(e, device=order.device)).sum(dim=0), 0)
    xs = torch.where(filled[:, None], s["x"][order // k], 0)

    def back(y, weight):
        y = torch.where(there[:, None], y[place].float(), 0.0).view(-1, k, c["width"])
        return (y if weight is None else y * weight[:, :, None]).sum(dim=1).to(t)

    out = {"first": first.to(torch.int32), "order": torch.where(filled, order, -1).to(torch.int32),
           "place": torch.where(there, place, -1).to(torch.int32).view(-1, k), "xs": xs, "out": back(s["y"], s["weight"])}
    if c["kind"] == "exchange_train":
        wide = s["d_out"].float()[:, None, :]
        dy = (wide * s["weight"][:, :, None]).view(slots, -1)
        out["d_y"] = torch.where(filled[:, None], dy[order], 0.0).to(t)
        dw = (wide * s["y"][place].float().view(-1, k, c["width"])).sum(dim=2)
        out["d_weight"] = torch.where(there.view(-1, k), dw, 0.0)
        out["d_x"] = back(s["d_xs"], None)
    return out


def _plain_ids(s):
    ids = s["ids"].long().view(s["case"]["rows"], -1)
    if s["base"] is None:
        return ids
    return (ids & 0xffff) + s["base"].long()


def _plain_embed(s):
    """The table's gradient is summed in 64 bits: a popular token's sum is long."""
    c, ids = s["case"], _plain_ids(s)
    if c["kind"] == "embed":
        return (s["table"].float()[ids].sum(dim=1) * c["scale"]).to(s["table"].dtype)
    each = s["d_out"].double()[:, None, :].expand(-1, ids.shape[1], -1).reshape(-1, c["width"])
    d = torch.zeros(c["vocab"], c["width"], dtype=torch.float64, device=ids.device)
    return (d.index_add_(0, ids.reshape(-1), each) * c["scale"]).float()


# ---- the definition, in 64 bits --------------------------------------------------------------------


def exact(case, seed):
    global own
    if _cost(case) > 400000000:
        return None
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["kind"].startswith("route"):
        return _exact_route(case, s)
    if case["kind"].startswith("exchange"):
        return _exact_exchange(case, s)
    return _exact_embed(case, s)


def _cost(case):
    if case["kind"].startswith("route"):
        return case["rows"] * case["experts"] * 2
    return case["rows"] * case.get("k", 1) * case["width"] * case.get("bag", 1)


def _exact_route(c, s):
    """Choices one after the other, each the largest key that is left."""
    x = torch.nan_to_num(s["logits"].double(), nan=-math.inf, posinf=_BIG, neginf=-math.inf)
    open_ = x > -math.inf
    if c["score"] == "softmax":
        log_score = torch.log_softmax(torch.where(open_.any(dim=1, keepdim=True), x, 0.0), dim=1)
    else:
        log_score = torch.nn.functional.logsigmoid(x)
    score = torch.where(open_, log_score.exp(), 0.0)
    key = x.clone() if s["bias"] is None else score + s["bias"].double()
    key[~open_] = -math.inf
    rows = torch.arange(c["rows"], device=x.device)
    if c["groups"] > 1:
        ranked = key if s["bias"] is not None else torch.where(open_, score, -math.inf)
        left = ranked.view(c["rows"], c["groups"], -1).clone()
        total = None
        for _ in range(c["group_best"]):
            v, i = left.max(dim=2)
            total = v if total is None else torch.where(torch.isneginf(v), total, total + v)
            left.scatter_(2, i[:, :, None], -math.inf)
            if left.shape[2] == 1:
                break
        keep = torch.zeros(c["rows"], c["groups"], dtype=torch.bool, device=x.device)
        for _ in range(c["top_groups"]):
            v = total.max(dim=1, keepdim=True).values
            first = ((total == v) & (v > -math.inf)).to(torch.int8).argmax(dim=1)
            keep[rows, first] |= (v > -math.inf)[:, 0]
            total[rows, first] = -math.inf
        key = torch.where(keep.repeat_interleave(c["experts"] // c["groups"], dim=1), key, -math.inf)
    expert, logs = [], []
    for _ in range(c["k"]):
        v = key.max(dim=1, keepdim=True).values
        first = (key == v).to(torch.int8).argmax(dim=1)
        there = v[:, 0] > -math.inf
        expert.append(torch.where(there, first, -1))
        logs.append(torch.where(there, log_score[rows, first], -math.inf))
        key[rows, first] = -math.inf
    expert, logs = torch.stack(expert, 1), torch.stack(logs, 1)
    some = (expert >= 0).any(dim=1, keepdim=True)
    q = torch.softmax(torch.where(some, logs, 0.0), dim=1) * some if c["renormalise"] else logs.exp()
    q = torch.where(expert >= 0, q, 0.0)
    out = {"expert": None, "weight": q * c["scale"]}
    if c["kind"] == "route_train":
        onto = torch.nn.functional.one_hot(expert.clamp(min=0), c["experts"]).double() * (expert >= 0)[:, :, None]
        dw = s["d_weight"].double() * c["scale"]
        if c["renormalise"]:       # weight_j = exp(a_j) / sum exp(a_i)
            da = torch.einsum("rke,rk->re", onto, q * (dw - (q * dw).sum(dim=1, keepdim=True)))
        else:                      # weight_j = exp(a_j)
            da = torch.einsum("rke,rk->re", onto, q * dw)
        if c["score"] == "softmax":   # a = l - log sum exp l
            d = da - score * da.sum(dim=1, keepdim=True)
        else:                         # a = log sigmoid(l)
            d = da * torch.sigmoid(-x)
        out["d_logits"] = torch.where(open_, d, 0.0)
    return out


def _exact_exchange(c, s):
    k, d = c["k"], c["width"]
    expert = s["expert"].long()
    slot = torch.full_like(expert, -1)
    at = 0
    owner = torch.full((expert.numel(),), -1, dtype=torch.long, device=expert.device)
    flat = torch.arange(expert.numel(), device=expert.device).view_as(expert)
    for e in range(c["experts"]):
        mine = expert == e
        n = int(mine.sum())
        slot[mine] = torch.arange(at, at + n, device=expert.device)
        owner[at:at + n] = flat[mine]
        at += n
    xs = torch.zeros(expert.numel(), d, dtype=torch.float64, device=expert.device)
    xs[:at] = s["x"].double()[owner[:at] // k]
    y, dout, w = s["y"].double(), s["d_out"].double(), s["weight"].double()
    res = torch.zeros(c["rows"], d, dtype=torch.float64, device=expert.device)
    dx, dw, dy = torch.zeros_like(res), torch.zeros_like(w), torch.zeros_like(xs)
    for j in range(k):
        has = (slot[:, j] >= 0)
        to = slot[has, j]
        res[has] += y[to] * w[has, j, None]
        dx[has] += s["d_xs"].double()[to]
        dw[has, j] = (dout[has] * y[to]).sum(dim=1)
        dy[to] = dout[has] * w[has, j, None]
    out = {"first": None, "order": None, "place": None, "xs": xs, "out": res}
    return dict(out, d_y=dy, d_weight=dw, d_x=dx) if c["kind"] == "exchange_train" else out


def _exact_embed(c, s):
    ids = s["ids"].long() % 65536 if s["base"] is not None else s["ids"].long()
    ids = ids.view(c["rows"], c["bag"]) + (0 if s["base"] is None else s["base"].long())
    if c["kind"] == "embed":
        out = torch.zeros(c["rows"], c["width"], dtype=torch.float64, device=ids.device)
        table = s["table"].double()
        for j in range(c["bag"]):
            out += table.index_select(0, ids[:, j])
        return out * c["scale"]
    d = torch.zeros(c["vocab"], c["width"], dtype=torch.float64, device=ids.device)
    d_out = s["d_out"].double()
    for j in range(c["bag"]):
        d.index_add_(0, ids[:, j], d_out)
    return d * c["scale"]
