"""Work for the operators that let networks be the experts of a mixture of family models, for timing.

A mixture sends statement rows (tokens) to the experts that a router chose.  Where the experts are small networks
instead of tree ensembles, rows in the experts' slots meet their expert's weights in a matrix product whose number of rows
differs from expert to expert.  Serving does the same in 8-bit integers, with a scale for every row and every channel of
the weights.  The router, and any other model that answers with logits, learns from a teacher of which only the largest logits are kept.

Kinds of a case:
  product         rows in slots times their experts' weights
  product_train   that, and the gradients of the rows and of the weights
  int8            tokens' rows in 8 bits to the slots, their products with 8-bit weights
  distill         every row's divergence from its teacher's largest logits
  distill_train   that, and the gradient of the logits
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
_BIG = torch.finfo(torch.float32).max

# ---- the cases -----------------------------------------------------------------------------------

_PRODUCT = {"kind": "product", "rows": 4096, "k": 4, "experts": 30, "in": 1024, "out": 1024, "type": "bf16", "missing": 0.0}
_DISTILL = {"kind": "distill", "rows": 4096, "classes": 64, "k": 8, "type": "fp32", "temperature": 1.0, "rest": False,
            "masked": 0.0}


def listed():
    return [
        # one statement row, scored by the networks of four families: the latency of a call, and of reading four weights
        dict(_PRODUCT, name="product_one", rows=1),
        # a small batch, a few rows for each of 64 families: reading all weights
        dict(_PRODUCT, name="product_few", rows=64, experts=64, **{"in": 2048}, type="fp16"),
        # feature rows of a 4096-program population to the first layer of their families' networks
        dict(_PRODUCT, name="product_rows", rows=32768, **{"in": 164, "out": 64}, type="fp32"),
        # hidden rows of an ordinary width into a wider layer, many of them
        dict(_PRODUCT, name="product_hidden", rows=65536, experts=64, out=2048, missing=0.05),
        # a training step on feature rows, 32 bits throughout
        dict(_PRODUCT, name="train_rows", kind="product_train", rows=16384, **{"in": 164, "out": 256}, type="fp32"),
        # a training step on hidden rows of an ordinary width
        dict(_PRODUCT, name="train_hidden", kind="product_train", rows=32768, experts=64, missing=0.1),
        # serving: a handful of rows, weights in 8 bits
        dict(_PRODUCT, name="int8_few", kind="int8", rows=8, k=2, **{"in": 2048, "out": 2048}),
        # serving: many hidden rows, weights in 8 bits
        dict(_PRODUCT, name="int8_hidden", kind="int8", rows=32768, out=4096, type="fp16"),
        # the router's rows of a pool, taught by the families' own eight best
        dict(_DISTILL, name="distill_router", rows=5120, masked=0.1),
        # one long row: the latency of a call
        dict(_DISTILL, name="distill_one", rows=1, classes=131072, k=64, type="bf16", rest=True),
        # a vocabulary of odd size, and what the teacher gives to classes outside its list
        dict(_DISTILL, name="distill_train_rest", kind="distill_train", rows=1000, classes=32001, k=20, type="fp16", rest=True, temperature=2.0),
        # a training step on a wide vocabulary
        dict(_DISTILL, name="distill_train_wide", kind="distill_train", rows=4096, classes=131072, k=64, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Most layers are a multiple of 32 wide, some are not."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.35 else max(32, (w + 16) // 32 * 32)


def draw(rng):
    kind = rng.choice(("product", "product", "product_train", "int8", "int8", "distill", "distill_train"))
    typ = rng.choice(("fp32", "bf16", "fp16"))
    if kind.startswith("distill"):
        rows, classes = _log_int(rng, 1, 65536), _log_int(rng, 16, 200000)
        while rows * classes > (134217728 if typ == "fp32" else 268435456):
            rows //= 2
        return dict(_DISTILL, kind=kind, rows=rows, classes=classes, k=min(_log_int(rng, 1, 128), classes // 2), type=typ,
                    rest=rng.random() < 0.4, temperature=rng.choice((1.0, 2.0, 0.5)), masked=rng.choice((0.0, 0.0, 0.2)))
    rows, k, experts = _log_int(rng, 1, 65536), rng.randint(1, 8), _log_int(rng, 1, 128)
    wide, out = _width(rng, 16, 4096), _width(rng, 16, 4096)
    while experts * wide * out > 200000000:
        experts //= 2
    most = {"product": 400000000000, "product_train": 130000000000, "int8": 500000000000}[kind]
    if typ == "fp32" and kind != "int8":
        most //= 8
    while rows * k * wide * out > most or rows * k * max(wide, out) > 400000000:
        rows //= 2
    return dict(_PRODUCT, kind=kind, rows=rows, k=min(k, experts), experts=experts, **{"in": wide, "out": out}, type=typ,
                missing=rng.choice((0.0, 0.1)))


def work(case):
    b = _BYTES[case["type"]]
    if case["kind"].startswith("distill"):
        n = case["rows"] * case["classes"]
        lists = case["rows"] * (case["k"] * 8 + 4 + (4 if case["rest"] else 0))
        if case["kind"] == "distill":
            return {"bytes": n * b + lists, "flops": 4 * n}
        return {"bytes": 2 * n * b + lists + 4 * case["rows"], "flops": 8 * n}
    slots, e, i, o = case["rows"] * case["k"], case["experts"], case["in"], case["out"]
    met = min(e, max(1, round(e * -math.expm1(-slots / e))))          # experts that have a row
    met = max(met, min(e, case["k"]))
    full = round(slots * (1 - case["missing"] / case["k"]))
    flops = 2 * full * i * o
    if case["kind"] == "int8":
        return {"bytes": case["rows"] * i * b + met * o * (i + 4) + slots * (o * b + 4), "flops": flops}
    w = {"bytes": full * i * b + met * i * o * b + slots * o * b, "flops": flops}
    if case["kind"] == "product_train":      # the results' gradient in; the rows' out, and the weights' in 32 bits
        w = {"bytes": w["bytes"] + full * o * b + slots * i * b + e * i * o * 4, "flops": 3 * flops}
    return w


# ---- what a program has in hand ------------------------------------------------------------------


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 6007 + 29)
    t = _TYPES[case["type"]]
    s = {"case": case}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    def rand(*shape):
        return torch.rand(shape, generator=gen, device=dev)

    rows, k = case["rows"], case["k"]
    if case["kind"].startswith("distill"):
        classes, temp = case["classes"], case["temperature"]
        common = normal(classes)                                        # some classes are likelier than others
        off = rand(classes) < case["masked"]
        s["logits"] = torch.empty(rows, classes, dtype=t, device=dev)
        s["ids"] = torch.empty(rows, k, dtype=torch.int32, device=dev)
        s["teacher"] = torch.empty(rows, k, device=dev)
        s["total"] = torch.empty(rows, device=dev) if case["rest"] else None
        step = max(1, 67108864 // classes)
        for a in range(0, rows, step):
            b = min(rows, a + step)
            x = normal(b - a, classes) * 2 + common
            full = x + normal(b - a, classes)                           # a teacher that knows more
            best = torch.topk(full, k, dim=1)
            s["ids"][a:b], s["teacher"][a:b] = best.indices.to(torch.int32), best.values
            if case["rest"]:
                s["total"][a:b] = torch.logsumexp(full / temp, dim=1)
            x[:, off] = -math.inf                                       # classes that the student may not take
            s["logits"][a:b] = x.to(t)
        s["ids"][:, k - 1:][rand(rows, 1) < 0.05] = -1                  # lists that are shorter
        s["ids"][rand(rows) < 0.01] = -1                                # rows without a teacher
        s["d_loss"] = (0.5 + rand(rows)) / rows * (65536.0 if t == torch.float16 else 1.0)      # in fp16, losses are scaled
        if own:
            from paper_2201_00194_amd import api
            s["params"] = api.distill_params(classes, k, temperature=temp, scale=temp * temp)
        return s

    e, i, o = case["experts"], case["in"], case["out"]
    wish = normal(rows, e) + normal(e) * 0.5                            # some experts are asked more often
    expert = torch.topk(wish, k, dim=1).indices.to(torch.int32).contiguous()
    expert[rand(rows) < case["missing"], k - 1] = -1                    # fewer than k experts were to be had
    if own:
        from paper_2201_00194_amd import api
        s["plan"] = api.fs_expert_plan(expert, e)
    flat = expert.reshape(-1).long()
    order = torch.sort(torch.where(flat < 0, e, flat), stable=True).indices
    s["order"] = torch.where(flat[order] >= 0, order, -1)
    s["first"] = torch.zeros(e + 1, dtype=torch.int32, device=dev)
    s["first"][1:] = torch.cumsum((flat[:, None] == torch.arange(e, device=dev)).sum(dim=0), 0)
    w = normal(e, o, i) / math.sqrt(i)
    if case["kind"] == "int8":
        s["w_scale"] = w.abs().amax(dim=2) / 127
        s["w"] = torch.round(w / s["w_scale"][:, :, None]).clamp(-127, 127).to(torch.int8)
        s["x"] = normal(rows, i).to(t)
        return s
    s["w"] = w.to(t)
    s["x"] = normal(rows * k, i).to(t)
    if case["kind"] == "product_train":
        s["d_y"] = normal(rows * k, o).to(t)
    return s


# ---- one pass ------------------------------------------------------------------------------------


def run(state):
    kind = state["case"]["kind"]
    if kind.startswith("distill"):
        return _own_distill(state) if own else _plain_distill(state)
    if kind == "int8":
        return _own_int8(state) if own else _plain_int8(state)
    return _own_product(state) if own else _plain_product(state)


def _own_product(s):
    from paper_2201_00194_amd import api
    y = api.fs_expert_matmul(s["x"], s["plan"], s["w"])
    if s["case"]["kind"] == "product":
        return y
    return {"y": y, "d_x": api.fs_expert_matmul(s["d_y"], s["plan"], s["w"], turned=True),
            "d_w": api.fs_expert_matmul_backward(s["d_y"], s["x"], s["plan"])}


def _own_int8(s):
    from paper_2201_00194_amd import api
    q, scale = api.fs_expert_gather_i8(s["x"], s["plan"])
    return {"y": api.fs_expert_matmul_i8(q, scale, s["plan"], s["w"], s["w_scale"], dtype=s["x"].dtype), "scale": scale}


def _own_distill(s):
    from paper_2201_00194_amd import api
    if s["case"]["kind"] == "distill":
        return api.fs_distill(s["params"], s["logits"], s["ids"], s["teacher"], total=s["total"])
    loss = torch.empty_like(s["d_loss"])
    d = api.fs_distill_backward(s["params"], s["logits"], s["ids"], s["teacher"], s["d_loss"], total=s["total"], loss=loss)
    return {"loss": loss, "d_logits": d}


def _ranges(s):
    first = s["first"].tolist()
    return [(e, a, b) for e, (a, b) in enumerate(zip(first, first[1:])) if b > a]


def _plain_product(s):
    c, x, w = s["case"], s["x"], s["w"]
    slots, t = x.shape[0], x.dtype
    y = torch.zeros(slots, c["out"], dtype=t, device=x.device)
    if c["kind"] == "product":
        for e, a, b in _ranges(s):
            y[a:b] = (x[a:b].float() @ w[e].float().t()).to(t)
        return y
    d_x = torch.zeros(slots, c["in"], dtype=t, device=x.device)
    d_w = torch.zeros(w.shape, device=x.device)
    for e, a, b in _ranges(s):
        rows, weights, g = x[a:b].float(), w[e].float(), s["d_y"][a:b].float()
        y[a:b] = (rows @ weights.t()).to(t)
        d_x[a:b] = (g @ weights).to(t)
        d_w[e] = g.t() @ rows
    return {"y": y, "d_x": d_x, "d_w": d_w}


def _plain_int8(s):
    """Scales and quotients in 64 bits, as quotients meet the borders between two integers."""
    c, x = s["case"], s["x"]
    size = x.float().abs().amax(dim=1)
    scale = (size.double() / 127).float().clamp(min=2.0 ** -126)
    q = torch.round(x.double() / scale.double()[:, None]).float()
    there = s["order"] >= 0
    token = torch.where(there, s["order"] // c["k"], 0)
    xs = q[token]
    slot_scale = torch.where(there, scale[token], 0.0)
    y = torch.zeros(token.shape[0], c["out"], dtype=x.dtype, device=x.device)
    for e, a, b in _ranges(s):
        y[a:b] = (xs[a:b] @ s["w"][e].float().t() * slot_scale[a:b, None] * s["w_scale"][e]).to(x.dtype)
    return {"y": y, "scale": slot_scale}


def _plain_distill(s):
    """Logarithms of sums and what is listed in 64 bits: shares of the rest are small differences."""
    c = s["case"]
    x, ids, temp = s["logits"].float() / c["temperature"], s["ids"].long(), c["temperature"]
    at = ids.clamp(min=0)
    listed_x = x.gather(1, at).double()
    there = (ids >= 0) & ~torch.isneginf(listed_x)
    none = ~there.any(dim=1, keepdim=True)
    t = torch.where(there, s["teacher"].double() / temp, -math.inf)

    def log_sum(v):
        high = v.max(dim=1, keepdim=True).values
        high = torch.where(torch.isinf(high), 0.0, high)
        return high.double() + torch.log(torch.exp(v - high).sum(dim=1, keepdim=True).double())

    all_x = log_sum(x)
    log_q = t - log_sum(t)
    if c["rest"]:
        unlisted = x.scatter(1, torch.where(there, at, at[:, :1]), -math.inf)      # rows that have none are left out below
        rest_x = log_sum(unlisted)
        some = ~torch.isneginf(rest_x)
        beside = torch.exp(torch.where(there & some, listed_x - rest_x, -math.inf)).sum(dim=1, keepdim=True)     # a list names a class once
        all_x = torch.where(some, rest_x + torch.log1p(beside), all_x)       # shares of the rest go by what is listed, however near to 1
        log_q = torch.where(some, t - s["total"][:, None], log_q)
        q_rest = torch.where(some, (1 - torch.exp(log_q).sum(dim=1, keepdim=True)).clamp(min=0), 0.0)
    q = torch.where(there, torch.exp(log_q), 0.0)
    log_q, listed_x = torch.where(there, log_q, 0.0), torch.where(there, listed_x, 0.0)
    loss = (q * (log_q - listed_x + all_x)).sum(dim=1, keepdim=True)
    if c["rest"]:
        loss = loss + torch.where(q_rest > 0, q_rest * (torch.log(q_rest) - rest_x + all_x), 0.0)
    scale = temp * temp
    loss = torch.where(none, 0.0, loss * scale)[:, 0].float()
    if c["kind"] == "distill":
        return loss
    high = x.max(dim=1, keepdim=True).values
    high = torch.where(torch.isinf(high), 0.0, high)
    d = torch.exp(x - high) * torch.exp(high - all_x).float()
    if c["rest"]:        # p - q_rest * p / p_rest, where it is not listed
        d = torch.where(torch.isneginf(unlisted), d, d * (1 - q_rest * torch.exp(all_x - rest_x)).float())
    d = d.scatter_add_(1, at, -q.float())
    d = torch.where(none | torch.isneginf(x), 0.0, d * (s["d_loss"][:, None] * (scale / temp)))
    return {"loss": loss, "d_logits": d.to(s["logits"].dtype)}


# ---- the definition, in 64 bits --------------------------------------------------------------------


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["kind"].startswith("distill"):
        return _exact_distill(case, s)
    return _exact_product(case, s)


def _exact_product(c, s):
    """Expert by expert, over the slots whose choice was that expert."""
    first, w, dev = s["first"].long(), s["w"].double(), s["w"].device
    slots = c["rows"] * c["k"]
    owner = torch.bucketize(torch.arange(slots, device=dev), first[1:], right=True)
    if c["kind"] == "int8":
        x = s["x"].double()
        scale = torch.clamp((x.abs().max(dim=1).values / 127).to(torch.float32), min=torch.finfo(torch.float32).tiny).double()
        token = s["order"].clamp(min=0) // c["k"]
        x, scale = torch.round(x / scale[:, None])[token], scale[token] * (s["order"] >= 0)
    else:
        x = s["x"].double()
    y = torch.zeros(slots, c["out"], dtype=torch.float64, device=dev)
    d_x, d_w = torch.zeros_like(x), torch.zeros_like(w)
    for e in range(c["experts"]):
        mine = torch.nonzero(owner == e)[:, 0]
        if not mine.numel():
            continue
        xe = x.index_select(0, mine)
        ye = torch.mm(xe, w[e].t().contiguous())
        if c["kind"] == "int8":
            ye = ye * scale.index_select(0, mine)[:, None] * s["w_scale"][e].double()
        y.index_copy_(0, mine, ye)
        if c["kind"] == "product_train":
            g = s["d_y"].index_select(0, mine).double()
            d_x.index_copy_(0, mine, torch.mm(g, w[e]))
            d_w[e] = torch.mm(g.t().contiguous(), xe)
    if c["kind"] == "int8":
        return {"y": y, "scale": scale}
    return y if c["kind"] == "product" else {"y": y, "d_x": d_x, "d_w": d_w}


def _exact_distill(c, s):
    """Some rows at a time: p and q as distributions over the classes, and one class of the rest."""
    rows, classes, temp = c["rows"], c["classes"], c["temperature"]
    loss = torch.zeros(rows, dtype=torch.float64, device=s["logits"].device)
    grad = torch.zeros(rows, classes, dtype=torch.float64, device=loss.device) if c["kind"] == "distill_train" else None
    step = max(1, 33554432 // classes)
    for a in range(0, rows, step):
        part = slice(a, min(rows, a + step))
        x = s["logits"][part].double() / temp
        ids = s["ids"][part].long()
        log_p = torch.log_softmax(x, dim=1)
        on = torch.zeros_like(x, dtype=torch.bool)
        value = torch.full_like(x, -math.inf)
        for j in range(c["k"]):
            has = torch.nonzero(ids[:, j] >= 0)[:, 0]
            on[has, ids[has, j]] = True
            value[has, ids[has, j]] = s["teacher"][part][has, j].double() / temp
        on &= x > -math.inf
        value = torch.where(on, value, -math.inf)
        taught = on.any(dim=1, keepdim=True)
        own_log = torch.log_softmax(torch.where(taught, value, 0.0), dim=1)
        q_rest = torch.zeros(x.shape[0], 1, dtype=torch.float64, device=x.device)
        beside = torch.where(on, -math.inf, x)
        if c["rest"]:
            open_ = (beside > -math.inf).any(dim=1, keepdim=True)
            own_log = torch.where(open_, value - s["total"][part].double()[:, None], own_log)
            q_rest = torch.where(open_, (1 - torch.where(on, own_log.exp(), 0.0).sum(dim=1, keepdim=True)).clamp(min=0), 0.0)
        q = torch.where(on, own_log.exp(), 0.0)
        total = torch.where(on, q * (own_log - log_p), 0.0).sum(dim=1)
        rest_p = torch.softmax(torch.where((beside > -math.inf).any(dim=1, keepdim=True), beside, 0.0), dim=1)
        if c["rest"]:
            log_rest = torch.logsumexp(torch.where(on, -math.inf, log_p), dim=1)
            total = total + torch.where(q_rest[:, 0] > 0, q_rest[:, 0] * (q_rest[:, 0].log() - log_rest), 0.0)
        loss[part] = torch.where(taught[:, 0], total * temp * temp, 0.0)
        if grad is not None:
            d = log_p.exp() - q - q_rest * torch.where(beside > -math.inf, rest_p, 0.0)
            d = torch.where(taught & (x > -math.inf), d, 0.0)
            grad[part] = d * (s["d_loss"][part].double()[:, None] * temp)
    return loss if grad is None else {"loss": loss, "d_logits": grad}
