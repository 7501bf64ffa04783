"""Measured cases of the operators on rows that name their network and of the distillation loss:
grouping rows by network, the products grouped by network with both gradients, and the loss
against a teacher's top logits with its gradient.

A pass makes the calls of one step of a user's program.  A program groups a batch's rows once and
then multiplies, so every pass of a product groups its rows first.  With `own` false the same
values come from elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _group(name, rows, per_row, networks):
    return {"name": name, "op": "group", "rows": rows, "per_row": per_row, "networks": networks}


def _product(name, op, rows, per_row, networks, inputs, outputs, dtype, act="none"):
    return {"name": name, "op": op, "rows": rows, "per_row": per_row, "networks": networks, "inputs": inputs,
            "outputs": outputs, "dtype": dtype, "act": act}


def _distill(name, op, rows, classes, top, dtype, labels):
    return {"name": name, "op": op, "rows": rows, "classes": classes, "top": top, "dtype": dtype, "labels": labels}


def listed():
    return [
        # a small batch of requests, each for two of 16 networks: one launch's latency
        _group("group_64x2_k16", 64, 2, 16),
        # an epoch's 60,000 rows, two of 256 child networks each (bench.py's largest K)
        _group("group_60000x2_k256", 60000, 2, 256),
        # one request through two of 64 child networks, first layer of 784-512-256-10
        _product("forward_1x2_k64_bf16", "forward", 1, 2, 64, 784, 512, "bf16", "relu"),
        # eight requests through wide networks: the weights that they name are read once
        _product("forward_8x2_k32_wide_bf16", "forward", 8, 2, 32, 2048, 4096, "bf16", "relu"),
        # one batch step of the widest workload, 256 child networks of 784-1024-10, rows by assignment
        _product("forward_32768_k256_fp32", "forward", 32768, 1, 256, 784, 1024, "fp32", "sigmoid"),
        # a large batch through wide layers, two networks a row
        _product("forward_32768x2_k32_bf16", "forward", 32768, 2, 32, 1024, 4096, "bf16", "relu"),
        # one batch step's backward of the bf16 workload: 64 child networks of 784-512-256-10
        _product("backward_4096_k64_bf16", "backward", 4096, 1, 64, 512, 256, "bf16", "relu"),
        # odd widths, few rows a network, fp32, two networks a row
        _product("backward_1501x2_k24_odd_fp32", "backward", 1501, 2, 24, 501, 203, "fp32"),
        # the backward of a large batch through wide layers
        _product("backward_16384x2_k16_bf16", "backward", 16384, 2, 16, 2048, 2048, "bf16"),
        # ten classes, the three that the teacher ranks first, an epoch's rows
        _distill("distill_60000x10_fp32", "distill", 60000, 10, 3, "fp32", True),
        # a step over many classes
        _distill("distill_4096x32000_bf16", "distill", 4096, 32000, 64, "bf16", True),
        # the loss alone, few rows and an odd number of classes
        _distill("loss_5x131071_fp32", "loss", 5, 131071, 20, "fp32", False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["group", "forward", "forward", "backward", "backward", "distill", "distill", "loss"])
    if op == "group":
        return dict(_group("", _log_int(rng, 1, 60000), rng.choice([1, 1, 2, 4]), _log_int(rng, 4, 256)), name="drawn")
    if op in ("forward", "backward"):
        while True:
            per_row = rng.choice([1, 1, 2, 4])
            networks = _log_int(rng, max(2, per_row), 256)
            rows, inputs, outputs = _log_int(rng, 1, 32768), _log_int(rng, 8, 2048), _log_int(rng, 8, 4096)
            if rng.random() < 0.6:  # most layers' widths are multiples of 8
                inputs, outputs = -(-inputs // 8) * 8, -(-outputs // 8) * 8
            dtype = rng.choice(["fp32", "bf16"])
            work = rows * per_row * inputs * outputs * (6 if dtype == "fp32" else 1)
            if work * (2 if op == "backward" else 1) <= 1.4e11 and networks * inputs * outputs <= 2.6e8:
                break
        act = rng.choice(["none", "relu", "sigmoid", "tanh"])
        if op == "backward" and per_row > 1:
            act = "none"
        return dict(_product("", op, rows, per_row, networks, inputs, outputs, dtype, act), name="drawn")
    while True:
        rows, classes = _log_int(rng, 1, 60000), _log_int(rng, 10, 131072)
        if rows * classes <= 1.3e8:
            break
    return dict(_distill("", op, rows, classes, min(classes, _log_int(rng, 1, 128)), rng.choice(["fp32", "bf16"]),
                         rng.random() < 0.5), name="drawn")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = dict(case)
    if case["op"] in ("distill", "loss"):
        n, v, k = case["rows"], case["classes"], case["top"]
        dtype = DTYPES[case["dtype"]]
        # a student that has learnt part of what the teacher answers
        teacher = normal(n, v) * 2
        s["z"] = (teacher * 0.7 + normal(n, v)).to(dtype)
        top = teacher.topk(k, dim=1)
        del teacher
        s["t"], s["idx"] = top.values.to(dtype), top.indices.to(torch.int32)
        # the last entries of some rows are padding: their teacher kept fewer
        keep = torch.randint(1, k + 1, (n, 1), generator=g, device="cuda")
        short = torch.rand(n, 1, generator=g, device="cuda") < 0.2
        s["idx"][(torch.arange(k, device="cuda") >= keep) & short] = -1
        s["y"] = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32) if case["labels"] else None
        s["temperature"], s["alpha"] = 2.0, (0.25 if case["labels"] else 0.0)
        s["g"] = torch.full((n,), 1.0 / n, device="cuda")
        return s
    n, per_row, networks = case["rows"], case["per_row"], case["networks"]
    # networks of unequal popularity, distinct ones within a row, one pair of a hundred dropped
    liking = 0.5 * normal(networks)
    gumbel = -torch.log(-torch.log(torch.rand(n, networks, generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
    ids = (gumbel + liking).topk(per_row, dim=1).indices.to(torch.int32)
    ids[torch.rand(n, per_row, generator=g, device="cuda") < 0.01] = -1
    s["ids"] = ids
    if case["op"] == "group":
        return s
    counts = torch.bincount((ids + 1).flatten().long(), minlength=networks + 1)[1:]
    s["largest"] = int(counts.max())  # the plain form's batched products are as tall as the largest group
    dtype, i, o = DTYPES[case["dtype"]], case["inputs"], case["outputs"]
    s["w"] = (normal(networks, o, i) * math.sqrt(2.0 / (i + o))).to(dtype)
    s["b"] = normal(networks, o) * 0.1
    # activations of the layer before, as its activation leaves them
    x = normal(n, i)
    x = {"relu": lambda v: torch.where(v < 0, -0.0, v), "sigmoid": torch.sigmoid, "tanh": torch.tanh, "none": lambda v: v}[case["act"]](x)
    s["x"] = x.to(dtype)
    if case["op"] == "backward":
        s["dy"] = (normal(n * per_row, o) * 0.01).to(dtype)
    return s


def run(s):
    return (_own if own else _plain)[s["op"]](s)


# ---- the framework's calls -----------------------------------------------------------------

def _own_group(s):
    from paper_2304_09590_amd import pnn
    groups = pnn.group_rows(s["ids"], s["networks"])
    return groups.offsets, groups.pairs


def _own_forward(s):
    from paper_2304_09590_amd import pnn
    groups = pnn.group_rows(s["ids"], s["networks"])
    return pnn.grouped_forward(groups, s["x"], s["w"], s["b"], act=_act_code(pnn, s["act"]))


def _own_backward(s):
    from paper_2304_09590_amd import pnn
    groups = pnn.group_rows(s["ids"], s["networks"])
    act = _act_code(pnn, s["act"])
    dx = pnn.grouped_backward_input(groups, s["dy"], s["w"], a=None if act is None else s["x"], act=act)
    dw, db = pnn.grouped_backward_weights(groups, s["dy"], s["x"])
    return dx, dw, db


def _own_loss(s):
    from paper_2304_09590_amd import pnn
    return pnn.distill_loss(s["z"], s["idx"], s["t"], y=s["y"], temperature=s["temperature"], alpha=s["alpha"])[0]


def _own_distill(s):
    from paper_2304_09590_amd import pnn
    loss, stats = pnn.distill_loss(s["z"], s["idx"], s["t"], y=s["y"], temperature=s["temperature"], alpha=s["alpha"])
    dz = pnn.distill_grad(s["z"], s["idx"], s["t"], stats, s["g"], y=s["y"], temperature=s["temperature"],
                          alpha=s["alpha"])
    return loss, dz


def _act_code(pnn, name):
    return {"none": None, "relu": pnn.RELU, "sigmoid": pnn.SIGMOID, "tanh": pnn.TANH}[name]


_own = {"group": _own_group, "forward": _own_forward, "backward": _own_backward, "loss": _own_loss,
        "distill": _own_distill}


# ---- plain forms ---------------------------------------------------------------------------

def _sorted_pairs(s):
    """Keys of the sorted pairs (networks = dropped), the pairs, the groups' first positions."""
    networks = s["networks"]
    ids = s["ids"].reshape(-1)
    key = torch.where((ids < 0) | (ids >= networks), networks, ids)
    key, order = torch.sort(key, stable=True)
    counts = torch.zeros(networks + 1, dtype=torch.int64, device=ids.device).scatter_add_(
        0, key.long(), torch.ones_like(key, dtype=torch.int64))
    return key.long(), order, counts.cumsum(0) - counts


def _plain_group(s):
    _, order, first = _sorted_pairs(s)
    return first.to(torch.int32), order.to(torch.int32)


def _act(name, z):
    if name == "relu":
        return torch.where(z < 0, z * 0, z)
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if name == "tanh":
        return 1 - 2 / (1 + torch.exp(2 * z))
    return z


def _slope(name, a):
    if name == "relu":
        return ((a > 0) | ((a == 0) & ~torch.signbit(a))).to(a.dtype)
    if name == "sigmoid":
        return a * (1 - a)
    if name == "tanh":
        return 1 - a * a
    return None


def _slots(s):
    """Each pair's place in batches of the largest group's height; the place after the last is the dropped pairs'."""
    key, order, first = _sorted_pairs(s)
    rank = torch.arange(key.numel(), device=key.device) - first[key]
    height = max(1, s["largest"])
    at = torch.where(key < s["networks"], key * height + rank, s["networks"] * height)
    return key, order, at, height


def _batched(rows, at, networks, height):
    b = torch.zeros(networks * height + 1, rows.shape[1], device=rows.device)
    b[at] = rows
    return b[:-1].view(networks, height, -1)


def _per_pair(batched, at, order):
    rows = torch.cat([batched.reshape(-1, batched.shape[-1]), torch.zeros(1, batched.shape[-1], device=at.device)])
    out = torch.empty(at.numel(), batched.shape[-1], device=at.device)
    out[order] = rows[at]
    return out


def _plain_forward(s):
    w, x, b, networks = s["w"], s["x"].float(), s["b"], s["networks"]
    ids = s["ids"].reshape(-1).long()
    if ids.numel() <= networks:  # few pairs: only the weights that they name
        kept = ((ids >= 0) & (ids < networks))[:, None]
        e = ids.clamp(0, networks - 1)
        z = torch.bmm(w[e].float(), x.repeat_interleave(s["per_row"], 0)[:, :, None])[:, :, 0] + b[e]
        return torch.where(kept, _act(s["act"], z), 0.0).to(w.dtype)
    _, order, at, height = _slots(s)
    xb = _batched(x[order // s["per_row"]], at, networks, height)
    z = torch.bmm(xb, w.float().transpose(1, 2)) + b[:, None, :]
    return _per_pair(_act(s["act"], z), at, order).to(w.dtype)


def _plain_backward(s):
    w, dy, x, networks, per_row = s["w"], s["dy"].float(), s["x"].float(), s["networks"], s["per_row"]
    _, order, at, height = _slots(s)
    dyb = _batched(dy[order], at, networks, height)
    dxp = _per_pair(torch.bmm(dyb, w.float()), at, order)
    dx = dxp.view(-1, per_row, dxp.shape[1]).sum(1)
    slope = _slope(s["act"], x)
    if slope is not None:
        dx = dx * slope
    xb = _batched(x[order // per_row], at, networks, height)
    return dx.to(w.dtype), torch.bmm(dyb.transpose(1, 2), xb), dyb.sum(1)


def _distill_parts(s):
    z, temperature, classes = s["z"].float(), s["temperature"], s["classes"]
    d = z - z.max(1, keepdim=True).values
    e = torch.exp(d / temperature)
    total = e.sum(1, keepdim=True)
    kept = (s["idx"] >= 0) & (s["idx"] < classes)
    at = torch.where(kept, s["idx"], 0).long()
    t = torch.where(kept, s["t"].float() / temperature, -math.inf)
    t = t - t.max(1, keepdim=True).values
    p = torch.exp(t)
    mass = p.sum(1, keepdim=True)
    p, log_p = p / mass, t - torch.log(mass)
    log_q = d.gather(1, at) / temperature - torch.log(total)
    kl = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    loss = (1 - s["alpha"]) * temperature * temperature * kl
    s_exp = None
    if s["y"] is not None:
        s_exp = torch.exp(d)
        s_total = s_exp.sum(1, keepdim=True)
        loss = loss + s["alpha"] * (torch.log(s_total) - d.gather(1, s["y"].long()[:, None]))[:, 0]
        s_exp = s_exp / s_total
    return loss, e / total, s_exp, at, p


def _plain_loss(s):
    return _distill_parts(s)[0]


def _plain_distill(s):
    loss, q, soft, at, p = _distill_parts(s)
    dz = (1 - s["alpha"]) * s["temperature"] * q.scatter_add(1, at, -p)
    if soft is not None:
        dz = dz + s["alpha"] * soft.scatter_add(1, s["y"].long()[:, None], -torch.ones_like(soft[:, :1]))
    return loss, (dz * s["g"][:, None]).to(s["z"].dtype)


_plain = {"group": _plain_group, "forward": _plain_forward, "backward": _plain_backward, "loss": _plain_loss,
          "distill": _plain_distill}


# ---- work and exact values -----------------------------------------------------------------

def work(case):
    if case["op"] in ("distill", "loss"):
        n, v, k = case["rows"], case["classes"], case["top"]
        size = 4 if case["dtype"] == "fp32" else 2
        moved = n * v * size + n * k * (4 + size) + 4 * n + (4 * n if case["labels"] else 0)
        if case["op"] == "distill":
            moved += n * v * size + 4 * n
        return {"bytes": moved, "flops": n * v * (12 if case["op"] == "distill" else 6)}
    n, per_row, networks = case["rows"], case["per_row"], case["networks"]
    pairs = n * per_row
    if case["op"] == "group":
        return {"bytes": 4 * pairs + 4 * pairs + 4 * (networks + 1), "flops": 0}
    size, i, o = (4 if case["dtype"] == "fp32" else 2), case["inputs"], case["outputs"]
    named = networks * (1 - (1 - 1 / networks) ** pairs)  # networks that some pair names
    weights = named * i * o
    moved = 4 * pairs + weights * size + n * i * size + pairs * o * size
    if case["op"] == "forward":
        return {"bytes": moved + 4 * named * o, "flops": 2 * pairs * i * o}
    moved += n * i * size + 4 * networks * o * (i + 1)
    return {"bytes": moved, "flops": 4 * pairs * i * o}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("distill", "loss"):
        return _exact_distill(s)
    networks, per_row = case["networks"], case["per_row"]
    ids = s["ids"].reshape(-1)
    members = [torch.nonzero(ids == e)[:, 0] for e in range(networks)]
    if case["op"] == "group":
        dropped = torch.nonzero((ids < 0) | (ids >= networks))[:, 0]
        first = [0]
        for m in members:
            first.append(first[-1] + m.numel())
        return (torch.tensor(first, dtype=torch.int32), torch.cat(members + [dropped]).to(torch.int32))
    i, o, act = case["inputs"], case["outputs"], case["act"]
    f64 = {"dtype": torch.float64, "device": "cuda"}
    if case["op"] == "forward":
        y = torch.zeros(ids.numel(), o, **f64)
        for e, m in enumerate(members):
            z = s["x"][m // per_row].double() @ s["w"][e].double().T + s["b"][e].double()
            y[m] = {"relu": lambda v: v.clamp(min=0), "sigmoid": torch.sigmoid, "tanh": torch.tanh,
                    "none": lambda v: v}[act](z)
        return y
    dx = torch.zeros(ids.numel(), i, **f64)
    dw, db = torch.zeros(networks, o, i, **f64), torch.zeros(networks, o, **f64)
    for e, m in enumerate(members):
        d, x = s["dy"][m].double(), s["x"][m // per_row].double()
        dx[m] = d @ s["w"][e].double()
        dw[e] = d.T @ x
        db[e] = d.sum(0)
    dx = dx.view(-1, per_row, i).sum(1)
    a = s["x"].double()
    if act == "relu":
        dx = dx * (a >= 0)  # the slope at 0 is 1, but -0 is a stored negative sum's
        dx = torch.where((a == 0) & torch.signbit(a), torch.zeros_like(dx), dx)
    elif act == "sigmoid":
        dx = dx * (a - a * a)
    elif act == "tanh":
        dx = dx * (1 - a) * (1 + a)
    return dx, dw, db


def _exact_distill(s):
    z, temperature, alpha = s["z"].double(), s["temperature"], s["alpha"]
    lq = torch.log_softmax(z / temperature, 1)
    target = torch.full_like(z[:, :1], 0).expand(z.shape[0], s["idx"].shape[1]).clone()
    kept = s["idx"] >= 0
    target[~kept] = -math.inf
    lp = torch.log_softmax(target + s["t"].double() / temperature, 1)
    p = torch.exp(lp)
    at = s["idx"].long().clamp(min=0)
    terms = torch.where(kept, p * (lp - lq.gather(1, at)), torch.zeros_like(p))
    loss = (1 - alpha) * temperature ** 2 * terms.sum(1)
    if s["y"] is not None:
        ls = torch.log_softmax(z, 1)
        loss = loss - alpha * ls.gather(1, s["y"].long()[:, None])[:, 0]
    if s["op"] == "loss":
        return loss
    dz = lq.exp_().scatter_add_(1, at, -p).mul_((1 - alpha) * temperature)
    if s["y"] is not None:
        soft = ls.exp_()
        soft[torch.arange(soft.shape[0], device=soft.device), s["y"].long()] -= 1
        dz += alpha * soft
    return loss, dz * s["g"].double()[:, None]
