"""What a pruned network in 4 bits is tuned and served with, as cases that can be timed: a teacher's top logits, the loss against them, low-rank adapters.

Six kinds of work, all through the public entry points:

* ``top``           the largest logits of each row with their classes, ``cprune_top_logits``: what an unpruned network leaves of its answers;
* ``loss``          distillation from those, forward, ``cprune_distill_loss``: a value a row, and what the backward call reads;
* ``loss_grad``     its gradient by the logits, ``cprune_distill_loss_backward``;
* ``step``          both in one pass where the rows' weights are known before, ``cprune_distill_step``: a training step's call;
* ``adapter``       ``cprune_adapter_linear``: low-rank adapters of several tuned variants beside one shared projection, each row with its own;
* ``adapter_grad``  its gradients by input and adapters, ``cprune_adapter_linear_backward``.

``own`` says whether ``run`` makes those calls or computes the same in elementary torch operations.  ``listed()`` gives fixed cases, ``draw(rng)`` more
of the same ranges, ``prepare(case, seed)`` what a program has in hand before the call, ``run(state)`` one pass, ``work(case)`` the bytes and operations
that the pass cannot do without and ``exact(case, seed)`` its result in 64 bits.

Top logits: descending, equal ones by their class; a logit of -infinity is a masked class and has -1 for its class.

Distillation, with p the softmax of a row's kept teacher logits over the temperature T (those with a class of -1 left out) and q_T the softmax of all of
the row's logits z over T:

    loss = (1 - hard) T^2 sum p (log p - log q_T) - hard log q_1[label]
    dz   = dloss ((1 - hard) T (q_T - p) + hard (q_1 - [label]))

A row whose list is empty, or that has no label (-1), goes without that term.  The statistics are a row's largest logit m and the logarithms of
sum exp((z - m) / T) and sum exp(z - m).

Adapters: hidden = scale_i (A_i x), y = act(base + B_i hidden) with i the row's adapter; a row of adapter -1 has no such term and a hidden of zeros.
Gradients, with g = scale_i (B_i^T dy): dx = dx_base + A_i^T g, dA_i = sum of g x^T and dB_i = sum of dy hidden^T over the rows of adapter i.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
ACTS = {"none": 0, "relu": 1, "relu6": 2, "silu": 3}


def _top(name, rows, classes, k, dtype, wide=0, masked=False):
    return {"name": name, "kind": "top", "rows": rows, "classes": classes, "k": k, "dtype": dtype, "wide": wide, "masked": masked}


def _loss(name, kind, rows, classes, k, dtype, temperature=2.0, hard=0.0, wide=0, masked=False):
    return {"name": name, "kind": kind, "rows": rows, "classes": classes, "k": k, "dtype": dtype, "temperature": temperature, "hard": hard, "wide": wide,
            "masked": masked}


def _adapter(name, kind, rows, k, c_out, rank, adapters, dtype, order="runs", base=True, act="none", hidden=False, wide=0):
    return {"name": name, "kind": kind, "rows": rows, "k": k, "c_out": c_out, "rank": rank, "adapters": adapters, "dtype": dtype, "order": order,
            "base": base, "act": act, "hidden": hidden, "wide": wide}


def listed():
    return [
        # the answers of a batch of 64 to ten classes: a call whose time is its launch
        _top("top_64x10_k4_f32", 64, 10, 4, "f32"),
        # a batch of long rows, an odd number of classes, some of them masked
        _top("top_2048x50257_k32_bf16", 2048, 50257, 32, "bf16", masked=True),
        # a training step of a 1000-class network at a batch of 256, with labels
        _loss("step_256x1000_k8_f32", "step", 256, 1000, 8, "f32", temperature=4.0, hard=0.1),
        # a teacher's list against long rows, the forward pass alone, the first classes of a padded row
        _loss("loss_4096x32768_k16_f16", "loss", 4096, 32768, 16, "f16", hard=0.5, wide=8),
        # two odd long rows: few rows for the device's units
        _loss("loss_grad_2x131071_k64_f32", "loss_grad", 2, 131071, 64, "f32", masked=True),
        # the largest step: two passes over a gigabyte are what it cannot do without
        _loss("step_4096x131072_k64_bf16", "step", 4096, 131072, 64, "bf16", temperature=1.0),
        # one row through one of eight variants
        _adapter("adapter_1x4096x4096_r16_n8_bf16", "adapter", 1, 4096, 4096, 16, 8, "bf16", order="mixed"),
        # a batch of single requests, each of its own variant
        _adapter("adapter_48x8192x8192_r16_n32_f16", "adapter", 48, 8192, 8192, 16, 32, "f16", order="mixed", act="silu"),
        # long requests behind each other
        _adapter("adapter_16384x4096x11008_r32_n8_bf16", "adapter", 16384, 4096, 11008, 32, 8, "bf16"),
        # a pruned 1x1 layer on a 56x56 map, odd numbers throughout, one adapter, what a training step keeps
        _adapter("adapter_3136x83x45_r5_f32", "adapter", 3136, 83, 45, 5, 1, "f32", order="one", hidden=True),
        # the 1x1 projection of a batch of 64 14x14 maps
        _adapter("adapter_grad_12544x576x96_r8_f16", "adapter_grad", 12544, 576, 96, 8, 1, "f16", order="one"),
        # variants trained beside each other, a wide rank
        _adapter("adapter_grad_8192x4096x4096_r64_n4_bf16", "adapter_grad", 8192, 4096, 4096, 64, 4, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["top", "loss", "loss_grad", "step", "adapter", "adapter", "adapter_grad", "adapter_grad"])
    dtype = rng.choice(sorted(TYPES))
    wide = rng.choice([0, 0, 0, 8, 13])
    if kind in ("top", "loss", "loss_grad", "step"):
        while True:
            rows, classes = _log_int(rng, 1, 16384), _log_int(rng, 10, 131072)
            if rng.random() < 0.5:
                classes = -(-classes // 8) * 8
            if rng.random() < 0.2:
                rows = rng.randint(1, 4)
            if rows * classes <= (2048 * 50257 if kind == "top" else 4096 * 131072) * 2 // SIZE[dtype]:
                break
        k = _log_int(rng, 1, min(128, classes))
        if kind == "top":
            case = _top("", rows, classes, k, dtype, wide, rng.random() < 0.5)
        else:
            case = _loss("", kind, rows, classes, k, dtype, rng.choice([1.0, 2.0, 4.0]), rng.choice([0.0, 0.1, 0.5]), wide, rng.random() < 0.5)
    else:
        while True:
            rows, k, c_out = _log_int(rng, 1, 16384), _log_int(rng, 16, 8192), _log_int(rng, 16, 11008)
            if rng.random() < 0.3:
                rows = rng.randint(1, 64)       # single requests
            if rng.random() < 0.5:
                k, c_out = -(-k // 8) * 8, -(-c_out // 8) * 8
            rank = rng.choice([4, 8, 16, 32, 64, rng.randint(1, 64)])
            order = rng.choice(["one", "runs", "mixed"])
            adapters = 1 if order == "one" else _log_int(rng, 1, 32)
            most = (16384 * (4096 + 11008) if kind == "adapter" else 8192 * (4096 + 4096)) * 2 // SIZE[dtype]
            if rows * (k + c_out) <= most and rows * (k + c_out) * rank <= most * 32 and adapters * rank <= 512:
                break
        case = _adapter("", kind, rows, k, c_out, rank, adapters, dtype, order, rng.random() < 0.8,
                        rng.choice(["none", "none", "relu", "silu"]) if kind == "adapter" else "none", kind == "adapter" and rng.random() < 0.4, wide)
    del case["name"]
    return case


# ---- what a program has in hand -------------------------------------------------------------------

def _logits(gen, case):
    """[rows, classes] of a classifier: rows of different sharpness; masked: classes that a row or all rows leave out; wide > 0: the first classes of wider
    rows."""
    rows, classes = case["rows"], case["classes"]
    z = torch.randn(rows, classes + case["wide"], generator=gen, device="cuda")
    z *= 1 + 2 * torch.rand(rows, 1, generator=gen, device="cuda")
    if case["masked"]:
        z.masked_fill_(torch.rand(classes + case["wide"], generator=gen, device="cuda") < 0.02, -math.inf)
        z[torch.arange(rows, device="cuda"), torch.randint(classes, (rows,), generator=gen, device="cuda")] = -math.inf
    return z.to(TYPES[case["dtype"]])[:, :classes]


def _prepare_loss(s, case, gen):
    rows, classes, k = case["rows"], case["classes"], case["k"]
    s["z"] = z = _logits(gen, case)
    t = 0.8 * z.float() + 0.8 * torch.randn(rows, classes, generator=gen, device="cuda")
    value, place = t.to(z.dtype).topk(k, dim=1)
    del t
    # lists of different lengths, some of them empty; a row's masked classes are in none
    length = torch.randint(1, 2 * k + 1, (rows, 1), generator=gen, device="cuda")
    length *= (torch.rand(rows, 1, generator=gen, device="cuda") >= 0.02).long() if rows > 8 else 1
    there = (torch.arange(k, device="cuda") < length) & (value > -math.inf)
    s["ids"] = torch.where(there, place, -1).int()
    s["teacher"] = torch.where(there, value, -math.inf)
    s["labels"] = None
    if case["hard"]:
        label = torch.randint(classes, (rows,), generator=gen, device="cuda")
        label = torch.where(z.gather(1, label[:, None])[:, 0] > -math.inf, label, -1)
        s["labels"] = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.05, -1, label).int()
    s["dloss"] = (0.5 + torch.rand(rows, generator=gen, device="cuda")) / rows
    if case["dtype"] == "f16":
        s["dloss"] *= rows      # (a loss scale, as such types are trained with)
    if case["kind"] == "loss_grad":
        # what the forward pass has left
        m = z.max(dim=1).values.float()
        far = z.double().sub_(m[:, None])
        s["stats"] = torch.stack([m, far.div(case["temperature"]).exp_().sum(dim=1).log_().float(), far.exp_().sum(dim=1).log_().float()])


def _rows(gen, rows, c, dtype, wide):
    x = torch.randn(rows, c + wide, generator=gen, device="cuda")
    x *= 0.5 + torch.rand(c + wide, generator=gen, device="cuda")
    return x.to(TYPES[dtype])[:, :c]


def _prepare_adapter(s, case, gen):
    rows, k, c_out, rank, n, dtype = (case[f] for f in ("rows", "k", "c_out", "rank", "adapters", "dtype"))
    s["x"] = _rows(gen, rows, k, dtype, case["wide"])
    s["a"] = (torch.randn(n, rank, k, generator=gen, device="cuda") / math.sqrt(k)).to(TYPES[dtype])
    s["b"] = (torch.randn(n, c_out, rank, generator=gen, device="cuda") * (0.3 / math.sqrt(rank))).to(TYPES[dtype])
    s["scale"] = 0.5 + 1.5 * torch.rand(n, generator=gen, device="cuda")
    if case["order"] == "one":
        s["which"] = None
    else:
        # one row in twenty, or one request, goes without
        if case["order"] == "mixed":
            which = torch.randint(n, (rows,), generator=gen, device="cuda")
            without = torch.rand(rows, generator=gen, device="cuda") < 0.05
            without[0] = False
            s["which"] = torch.where(without, -1, which).int()
        else:
            starts = torch.rand(2 * n, generator=gen, device="cuda").mul_(rows).long().sort().values
            of_run = torch.randperm(2 * n, generator=gen, device="cuda") % n
            of_run = torch.where((torch.arange(2 * n, device="cuda") == 0) & (starts[-1] > 0), -1, of_run)
            run = (torch.searchsorted(starts, torch.arange(rows, device="cuda"), right=True) - 1).clamp_(min=0)
            s["which"] = of_run[run].int()
    if case["kind"] == "adapter":
        s["base"] = _rows(gen, rows, c_out, dtype, case["wide"]) if case["base"] else None
        return
    s["dy"] = _rows(gen, rows, c_out, dtype, case["wide"])
    s["dx_base"] = _rows(gen, rows, k, dtype, 0) if case["base"] else None
    # what the forward pass has left
    s["hidden"] = _plain_hidden(s, s["x"], s["a"])
    if s["which"] is not None:
        s["hidden"] = s["hidden"].sum(dim=1)
    s["hidden"] = s["hidden"].reshape(rows, rank)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "top":
        s["z"] = _logits(gen, case)
    elif case["kind"] in ("loss", "loss_grad", "step"):
        _prepare_loss(s, case, gen)
    else:
        _prepare_adapter(s, case, gen)
    return s


# ---- the plain forms ------------------------------------------------------------------------------

def _plain_top(z, k):
    value, place = torch.sort(z, dim=1, descending=True, stable=True)
    value, place = value[:, :k], place[:, :k]
    return value.contiguous(), torch.where(value == -math.inf, -1, place).int()


def _plain_teacher(s, case):
    """-> (the list's probabilities, its classes with 0 in place of -1, what a row's first term counts)"""
    there = (s["ids"] >= 0) & (s["teacher"] > -math.inf)
    t = torch.where(there, s["teacher"].float() / case["temperature"], -math.inf)
    any_there = there.any(dim=1)
    p = torch.exp(t - torch.where(any_there, t.amax(dim=1), 0.0)[:, None])
    p = torch.where(there, p / p.sum(dim=1, keepdim=True), 0.0)
    return p, torch.where(there, s["ids"], 0).long(), any_there * (1 - case["hard"])


def _plain_stats(s, case):
    z = s["z"].float()
    m = z.amax(dim=1)
    far = z - m[:, None]
    if case["temperature"] == 1:
        one = torch.log(torch.exp(far).sum(dim=1))
        return far, torch.stack([m, one, one])
    return far, torch.stack([m, torch.log(torch.exp(far / case["temperature"]).sum(dim=1)), torch.log(torch.exp(far).sum(dim=1))])


def _plain_value(s, case, far, stats):
    T = case["temperature"]
    p, ids, soft = _plain_teacher(s, case)
    log_q = far.gather(1, ids) / T - stats[1][:, None]
    terms = torch.where(p > 0, p * (torch.log(torch.where(p > 0, p, 1.0)) - log_q), 0.0)
    loss = soft * T * T * terms.sum(dim=1)
    if s["labels"] is not None:
        label = s["labels"].long()
        one = stats[2] - far.gather(1, label.clamp(min=0)[:, None])[:, 0]
        loss = loss + case["hard"] * torch.where(label >= 0, one, 0.0)
    return loss


def _plain_slope(s, case, far, stats):
    T = case["temperature"]
    p, ids, soft = _plain_teacher(s, case)
    soft = (s["dloss"] * soft * T)[:, None]
    dz = torch.exp(far / T - stats[1][:, None]) * soft
    dz.scatter_add_(1, ids, -soft * p)
    if s["labels"] is not None:
        label = s["labels"].long()[:, None]
        w = torch.where(label >= 0, case["hard"] * s["dloss"][:, None], 0.0)
        dz += torch.exp(far - stats[2][:, None]) * w
        dz.scatter_add_(1, label.clamp(min=0), -w)
    return dz.to(s["z"].dtype)


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _plain_hidden(s, x, a):
    """scale (a x) of every adapter, zeros but for a row's own: fp32 [rows, adapters, rank]; a [adapters, rank, c]."""
    n, rank = a.shape[:2]
    h = (x.float() @ a.float().reshape(n * rank, -1).t()).reshape(-1, n, rank) * s["scale"][:, None]
    if s["which"] is None:
        return h
    return torch.where((s["which"][:, None] == torch.arange(n, device="cuda"))[..., None], h, 0.0)


def _plain_adapter(s, case):
    n, rank, c_out = case["adapters"], case["rank"], case["c_out"]
    h = _plain_hidden(s, s["x"], s["a"])
    y = h.reshape(-1, n * rank) @ s["b"].float().permute(0, 2, 1).reshape(n * rank, c_out)
    if s["base"] is not None:
        y = y + s["base"].float()
    y = _act(y, case["act"]).to(s["x"].dtype)
    return (y, h.sum(dim=1)) if case["hidden"] else y


def _plain_adapter_grad(s, case):
    n, rank, k, c_out = case["adapters"], case["rank"], case["k"], case["c_out"]
    dy, x = s["dy"].float(), s["x"].float()
    g = _plain_hidden(s, dy, s["b"].transpose(1, 2)).reshape(-1, n * rank)
    dx = g @ s["a"].float().reshape(n * rank, k)
    if s["dx_base"] is not None:
        dx = dx + s["dx_base"].float()
    own_row = s["hidden"][:, None, :].expand(-1, n, -1)
    if s["which"] is not None:
        own_row = torch.where((s["which"][:, None] == torch.arange(n, device="cuda"))[..., None], own_row, 0.0)
    db = dy.t() @ own_row.reshape(-1, n * rank)
    return dx.to(s["x"].dtype), (g.t() @ x).reshape(n, rank, k), db.reshape(c_out, n, rank).transpose(0, 1).contiguous()


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        if kind == "top":
            return _plain_top(s["z"], case["k"])
        if kind == "loss":
            far, stats = _plain_stats(s, case)
            return _plain_value(s, case, far, stats), stats
        if kind == "loss_grad":
            return _plain_slope(s, case, s["z"].float() - s["stats"][0][:, None], s["stats"])
        if kind == "step":
            far, stats = _plain_stats(s, case)
            return _plain_value(s, case, far, stats), _plain_slope(s, case, far, stats)
        return _plain_adapter(s, case) if kind == "adapter" else _plain_adapter_grad(s, case)
    from paper_2207_01260_amd import binding as B
    if kind == "top":
        return B.cprune_top_logits(s["z"], case["k"])
    if kind == "loss":
        return B.cprune_distill_loss(s["z"], s["ids"], s["teacher"], s["labels"], case["temperature"], case["hard"], want_stats=True)
    if kind == "loss_grad":
        return B.cprune_distill_loss_backward(s["dloss"], s["z"], s["ids"], s["teacher"], s["stats"], s["labels"], case["temperature"], case["hard"])
    if kind == "step":
        return B.cprune_distill_step(s["dloss"], s["z"], s["ids"], s["teacher"], s["labels"], case["temperature"], case["hard"])
    if kind == "adapter":
        return B.cprune_adapter_linear(s["x"], s["a"], s["b"], s["which"], s["scale"], s["base"], act=ACTS[case["act"]], want_hidden=case["hidden"])
    return B.cprune_adapter_linear_backward(s["dy"], s["x"], s["hidden"], s["a"], s["b"], s["which"], s["scale"], s["dx_base"])


def work(case):
    es, rows, k = SIZE[case["dtype"]], case["rows"], case["k"]
    if case["kind"] in ("top", "loss", "loss_grad", "step"):
        count, lists = rows * case["classes"], rows * k * (es + 4)
        if case["kind"] == "top":
            return {"bytes": es * count + lists, "flops": count}
        passes = 1 if case["kind"] == "loss" else 2
        each = {"loss": 16, "loss_grad": 16, "step": 8}[case["kind"]] + (4 if case["hard"] else 0)
        terms = 2 if case["hard"] and case["temperature"] != 1 else 1
        return {"bytes": passes * es * count + lists + each * rows, "flops": 4 * passes * terms * count}
    c_out, rank, used = case["c_out"], case["rank"], min(case["adapters"], rows)
    weights, which = used * rank * (k + c_out), 0 if case["order"] == "one" else 4 * rows
    if case["kind"] == "adapter":
        return {"bytes": es * (rows * (k + c_out + (c_out if case["base"] else 0)) + weights) + which + (4 * rows * rank if case["hidden"] else 0),
                "flops": 2 * rows * rank * (k + c_out)}
    every = case["adapters"] * rank * (k + c_out)
    return {"bytes": es * (rows * (2 * k + c_out + (k if case["base"] else 0)) + weights) + which + 4 * rows * rank + 4 * every,
            "flops": 4 * rows * rank * (k + c_out)}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_top(z, k):
    """Largest first, the lowest class of equal ones: one after another."""
    left, rows = z.double(), torch.arange(z.shape[0], device="cuda")
    places = torch.arange(z.shape[1], device="cuda")
    values, ids = [], []
    for _ in range(k):
        top = left.amax(dim=1)
        at = torch.where(left == top[:, None], places, z.shape[1]).amin(dim=1)
        at = at.clamp(max=z.shape[1] - 1)
        values.append(top)
        ids.append(torch.where(top == -math.inf, -1, at))
        left[rows, at] = -math.inf
    return torch.stack(values, dim=1), torch.stack(ids, dim=1).int()


def _exact_loss(s, case):
    """Some rows at a time: 64 bits of the largest case are four gigabytes."""
    z, T, hard, kind = s["z"], case["temperature"], case["hard"], case["kind"]
    rows, classes = z.shape
    at_a_time = max(1, (1 << 26) // classes)
    values, slopes, stats = [], [], []
    for lo in range(0, rows, at_a_time):
        part = slice(lo, min(rows, lo + at_a_time))
        zz = z[part].double()
        log_q = torch.log_softmax(zz / T, dim=1)
        t = s["teacher"][part].double() / T
        t[s["ids"][part] < 0] = -math.inf
        full = t.amax(dim=1) > -math.inf
        log_p = torch.log_softmax(t, dim=1)
        p = torch.where(full[:, None], log_p.exp(), 0.0)
        where = s["ids"][part].clamp(min=0).long()
        kept = torch.where(p > 0, p * (log_p - log_q.gather(1, where)), 0.0).sum(dim=1)
        value = (1 - hard) * T * T * kept
        if kind != "loss":
            q = torch.where(full[:, None], log_q.exp(), 0.0)
            slope = (1 - hard) * T * q.scatter_add(1, where, -p)
        if s["labels"] is not None:
            label = s["labels"][part].long()
            has = label >= 0
            log_1 = torch.log_softmax(zz, dim=1)
            value = value - hard * torch.where(has, log_1.gather(1, label.clamp(min=0)[:, None])[:, 0], 0.0)
            if kind != "loss":
                one = log_1.exp().scatter_add(1, label.clamp(min=0)[:, None], -torch.ones_like(zz[:, :1]))
                slope = slope + hard * torch.where(has[:, None], one, 0.0)
        values.append(value)
        if kind == "loss":
            m = zz.amax(dim=1)
            stats.append(torch.stack([m, torch.logsumexp(zz / T, dim=1) - m / T, torch.logsumexp(zz, dim=1) - m]))
        else:
            slopes.append((slope * s["dloss"][part, None].double()).float() if z.dtype != torch.float32 else slope * s["dloss"][part, None].double())
    if kind == "loss":
        return torch.cat(values), torch.cat(stats, dim=1)
    return torch.cat(slopes) if kind == "loss_grad" else (torch.cat(values), torch.cat(slopes))


def _rows_of(s, case, i):
    if s["which"] is None:
        return torch.arange(case["rows"], device="cuda")
    return (s["which"] == i).nonzero()[:, 0]


def _exact_adapter(s, case):
    y = torch.zeros(case["rows"], case["c_out"], dtype=torch.float64, device="cuda")
    hidden = torch.zeros(case["rows"], case["rank"], dtype=torch.float64, device="cuda")
    for i in range(case["adapters"]):
        at = _rows_of(s, case, i)
        hidden[at] = s["scale"][i].double() * (s["x"][at].double() @ s["a"][i].double().t())
        y[at] = hidden[at] @ s["b"][i].double().t()
    if s["base"] is not None:
        y += s["base"].double()
    if case["act"] == "relu":
        y.clamp_(min=0)
    elif case["act"] == "silu":
        y *= torch.sigmoid(y)
    return (y, hidden) if case["hidden"] else y


def _exact_adapter_grad(s, case):
    dx = torch.zeros(case["rows"], case["k"], dtype=torch.float64, device="cuda") if s["dx_base"] is None else s["dx_base"].double()
    da = torch.zeros(case["adapters"], case["rank"], case["k"], dtype=torch.float64, device="cuda")
    db = torch.zeros(case["adapters"], case["c_out"], case["rank"], dtype=torch.float64, device="cuda")
    for i in range(case["adapters"]):
        at = _rows_of(s, case, i)
        dy = s["dy"][at].double()
        g = s["scale"][i].double() * (dy @ s["b"][i].double())
        dx[at] += g @ s["a"][i].double()
        da[i] = g.t() @ s["x"][at].double()
        db[i] = dy.t() @ s["hidden"][at].double()
    return dx, da, db


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "top":
        return _exact_top(s["z"], case["k"])
    if case["kind"] in ("loss", "loss_grad", "step"):
        return _exact_loss(s, case)
    return _exact_adapter(s, case) if case["kind"] == "adapter" else _exact_adapter_grad(s, case)
