"""Operators of a student that learns from a trained model, at the sizes its users run.

A student of a sampled model answers from a node's own row, without its neighbours: gated
feed-forward blocks (``gated``: rows answered; ``train``: their step, forward and
backward).  It learns from the largest logits that the model gave each row (``top``), by
a loss against the student's logits and its gradient (``distill``).

``listed()`` names the fixed cases, ``draw(rng)`` gives more of the same ranges,
``prepare``/``run`` make and take one pass, ``work`` counts the bytes and
operations that a pass cannot do without, and ``exact`` is the result in
64 bits.
"""
from __future__ import annotations

import math

import torch

own = False   # True: run() calls the framework's kernels; False: the plain forms

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
IGNORE = -1


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one row answered by a wide block: every weight read once
        dict(name="gated-1", op="gated", m=1, d=1_024, f=4_096, out=1_024, dtype="bf16", act="silu"),
        # the rows of a large frontier answered by a narrow one, odd row count
        dict(name="gated-frontier", op="gated", m=99_603, d=128, f=512, out=64, dtype="bf16", act="silu"),
        # a small model's batch: launch latency
        dict(name="train-10k", op="train", m=256, d=64, f=256, out=16, dtype="f32", act="gelu", dx=True),
        # features that are not trained, of odd width, in the framework's training type
        dict(name="train-602", op="train", m=1_024, d=602, f=1_024, out=41, dtype="f32", act="silu", dx=False),
        # a frontier's rows, odd count, with the gradient that goes on to a trained table
        dict(name="train-frontier", op="train", m=65_537, d=256, f=1_024, out=256, dtype="bf16", act="relu", dx=True),
        # wide layers and many rows: the products dominate
        dict(name="train-wide", op="train", m=8_192, d=1_024, f=4_096, out=1_024, dtype="bf16", act="silu", dx=True),
        # one row of logits over every node
        dict(name="top-1", op="top", m=1, classes=169_000, k=64, dtype="f32"),
        # a frontier's rows over a few classes
        dict(name="top-41", op="top", m=99_603, classes=41, k=8, dtype="f32"),
        # a batch's logits over every node, kept for the student
        dict(name="top-169k", op="top", m=1_024, classes=169_000, k=32, dtype="bf16"),
        # a batch over a few classes, a part of it labelled: launch latency
        dict(name="distill-41", op="distill", m=1_024, classes=41, k=8, dtype="f32", temperature=2.0, alpha=0.7, pad=0.6),
        # an odd batch over many classes, some rows without a teacher, some with fewer logits, labels beside it
        dict(name="distill-10k", op="distill", m=4_093, classes=10_000, k=50, dtype="bf16", temperature=4.0, alpha=0.5, pad=0.2),
        # a batch over every node, from the teacher alone
        dict(name="distill-169k", op="distill", m=1_024, classes=169_000, k=64, dtype="f32", temperature=1.0, alpha=1.0, pad=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["gated", "gated", "train", "train", "train", "top", "top", "distill", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("gated", "train"):
        m = _log(rng, 1, 100_000)
        d = rng.choice([64, 100, 128, 256, 512, 602, 1_024, rng.randint(17, 700)])
        f = rng.choice([128, 256, 512, 1_024, 2_048, 4_096, rng.randint(40, 1_500)])
        out = rng.choice([16, 41, 64, 128, 256, 1_024, d, rng.randint(5, 600)])
        case = dict(op=op, m=m, d=d, f=f, out=out, dtype=dtype, act=rng.choice(["silu", "silu", "gelu", "relu"]))
        if op == "train":
            case["dx"] = rng.random() < 0.7
        most = 5e10 if dtype == "f32" else 3e11   # operations of a pass
        while work(case)["flops"] > most or case["m"] * f > 1e8:
            case["m"] = case["m"] // 2 + 1
        return case
    classes = rng.choice([_log(rng, 5, 170_000), _log(rng, 5, 170_000), 41, 10_000])
    m = _log(rng, 1, 100_000)
    while m * classes > 1.7e8:
        m = m // 2 + 1
    k = min(_log(rng, 1, 128), classes)
    case = dict(op=op, m=m, classes=classes, k=k, dtype=dtype)
    if op == "distill":
        case.update(temperature=rng.choice([1.0, 2.0, 4.0, 0.5]), alpha=rng.choice([1.0, 0.5, 0.9]), pad=rng.choice([0.0, 0.3]))
    return case


# ----------------------------------------------------------------- inputs
def _padded(rows, d, dtype, gen=None, std=1.0):
    """A [rows, d] view whose rows start on 16-byte boundaries (zeros without a generator)."""
    per = 16 // BYTES[dtype]
    t = torch.zeros((rows, (d + per - 1) // per * per), dtype=TORCH[dtype], device="cuda")
    if gen is not None:
        t.normal_(0.0, std, generator=gen)
    return t[:, :d]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dtype, m = case["op"], case["dtype"], case["m"]
    if op in ("gated", "train"):
        d, f, out = case["d"], case["f"], case["out"]
        s = dict(x=_padded(m, d, dtype, gen, 1.0), wg=_padded(d, f, dtype, gen, 1.0 / math.sqrt(d)),
                 wu=_padded(d, f, dtype, gen, 1.0 / math.sqrt(d)), wd=_padded(f, out, dtype, gen, 1.0 / math.sqrt(f)))
        if op == "train":
            s["dy"] = _padded(m, out, dtype, gen, 1.0 / m)
        return s
    v, k = case["classes"], case["k"]
    logits = _padded(m, v, dtype, gen, 2.0)
    if op == "top":
        return dict(logits=logits)
    # k distinct classes a row, the teacher's logits in falling order; the student leans towards them
    base = torch.randint(0, v, (m, 1), generator=gen, device="cuda")
    step = torch.randint(1, max(v // k, 1) + 1, (m, 1), generator=gen, device="cuda")
    j = torch.arange(k, device="cuda")
    ids = (base + j * step) % v
    teacher = torch.randn((m, k), generator=gen, device="cuda").mul_(2.0).add_(4.0).sort(dim=1, descending=True).values
    logits.scatter_add_(1, ids, (0.5 * teacher).to(TORCH[dtype]))
    # a part of the rows hold fewer logits than k, or none
    kept = torch.where(torch.rand((m, 1), generator=gen, device="cuda") < case["pad"],
                       torch.randint(0, k + 1, (m, 1), generator=gen, device="cuda"), k)
    ids = torch.where(j < kept, ids, -1).to(torch.int32)
    teacher = torch.where(j < kept, teacher, -math.inf)
    labels = None
    if case["alpha"] < 1.0:
        labels = torch.randint(0, v, (m,), generator=gen, device="cuda", dtype=torch.int32)
        labels[torch.rand(m, generator=gen, device="cuda") < case["pad"]] = IGNORE
    return dict(logits=logits, ids=ids, teacher=teacher, labels=labels)


def prepare(case, seed):
    """The inputs and, as a program keeps them, the output buffers and workspaces."""
    s = _inputs(case, seed)
    s.update(case)
    op, dtype, m = case["op"], case["dtype"], case["m"]
    if op in ("gated", "train"):
        d, f, out = case["d"], case["f"], case["out"]
        s["y"] = _padded(m, out, dtype)
        if op == "train":
            s["dx"] = _padded(m, d, dtype) if case["dx"] else None
            s["dwg"], s["dwu"], s["dwd"] = _padded(d, f, dtype), _padded(d, f, dtype), _padded(f, out, dtype)
    elif op == "top":
        s["values"] = torch.zeros((m, case["k"]), device="cuda")
        s["ids"] = torch.zeros((m, case["k"]), dtype=torch.int32, device="cuda")
    else:
        s["loss"], s["row_loss"] = torch.zeros(3, device="cuda"), torch.zeros(m, device="cuda")
        s["dlogits"] = _padded(m, case["classes"], dtype)
    if own:
        import paper_2404_09544_amd as G
        if op in ("gated", "train"):
            need = G.gated_ffn_workspace(m, d, f, out, dtype)
            if op == "train":
                need = max(need, G.gated_ffn_backward_workspace(m, d, f, out, dtype))
                s["saved"] = torch.empty(G.gated_ffn_saved(m, f, dtype), dtype=torch.uint8, device="cuda")
        elif op == "top":
            need = G.top_logits_workspace(m, case["classes"], case["k"], dtype)
        else:
            need = G.distill_workspace(m, case["classes"], case["k"], dtype)
        s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------- runs
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2404_09544_amd as G
    op = s["op"]
    if op == "gated":
        G.gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], s["y"], act=s["act"], workspace=s["workspace"])
        return s["y"]
    if op == "train":
        G.gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], s["y"], act=s["act"], saved=s["saved"], workspace=s["workspace"])
        G.gated_ffn_backward(s["x"], s["wg"], s["wu"], s["wd"], s["dy"], s["saved"], dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"],
                             dwd=s["dwd"], act=s["act"], workspace=s["workspace"])
        return {n: s[n] for n in ("y", "dx", "dwg", "dwu", "dwd")}
    if op == "top":
        G.top_logits(s["logits"], s["values"], s["ids"], workspace=s["workspace"])
        return dict(values=s["values"], ids=s["ids"])
    G.distill(s["logits"], s["ids"], s["teacher"], s["loss"], temperature=s["temperature"], alpha=s["alpha"],
              labels=s["labels"], ignore_label=IGNORE, row_loss=s["row_loss"], dlogits=s["dlogits"], workspace=s["workspace"])
    return {n: s[n] for n in ("loss", "row_loss", "dlogits")}


def _act(a, name):
    """The activation and its derivative."""
    if name == "silu":
        g = 1.0 / (1.0 + torch.exp(-a))
        return a * g, g * (1.0 + a * (1.0 - g))
    if name == "gelu":
        g = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
        return a * g, g + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    on = (a > 0).to(a.dtype)
    return a * on, on


def _run_plain(s):
    op, dt = s["op"], TORCH[s["dtype"]]
    if op in ("gated", "train"):
        x, wg, wu, wd = (s[n].float() for n in ("x", "wg", "wu", "wd"))
        a, b = x @ wg, x @ wu
        g, slope = _act(a, s["act"])
        h = g * b
        y = (h @ wd).to(dt)
        if op == "gated":
            return y
        dy = s["dy"].float()
        dh = dy @ wd.t()
        da, db = dh * b * slope, dh * g
        dx = (da @ wg.t() + db @ wu.t()).to(dt) if s["dx"] is not None else None
        return dict(y=y, dx=dx, dwg=(x.t() @ da).to(dt), dwu=(x.t() @ db).to(dt), dwd=(h.t() @ dy).to(dt))
    if op == "top":
        values, ids = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
        return dict(values=values[:, :s["k"]].contiguous(), ids=ids[:, :s["k"]].to(torch.int32))
    return _plain_distill(s, dt)


def _plain_distill(s, dt):
    t, alpha, z = s["temperature"], s["alpha"], s["logits"].float()
    rows = torch.arange(s["m"], device="cuda")
    top = z.amax(dim=1, keepdim=True)
    # the teacher's part: its kept logits as a distribution over their classes
    kept = (s["ids"] >= 0) & (s["teacher"] > -math.inf)
    has = kept.any(dim=1)
    n = has.sum().clamp(min=1)
    ids = torch.where(kept, s["ids"], 0).long()
    u = torch.where(kept, s["teacher"] / t, -math.inf)
    u = u - torch.where(has, u.amax(dim=1), 0.0)[:, None]
    q = torch.exp(u)
    total = torch.where(has, q.sum(dim=1), 1.0)[:, None]
    q = q / total
    log_q = torch.where(kept, u - torch.log(total), 0.0)
    e = torch.exp((z - top) / t)
    mass = e.sum(dim=1, keepdim=True)
    log_p = (z.gather(1, ids) - top) / t - torch.log(mass)
    kd = torch.where(has, t * t * (q * (log_q - log_p)).sum(dim=1), 0.0)
    dz = (e / mass).scatter_add_(1, ids, -q) * (has * (alpha * t / n))[:, None]
    first = kd.double().sum() / n
    row_loss, second = alpha * kd, torch.zeros_like(first)
    if s["labels"] is not None:
        counted = s["labels"] != IGNORE
        y, c = torch.where(counted, s["labels"], 0).long(), counted.sum().clamp(min=1)
        e = torch.exp(z - top)
        mass = e.sum(dim=1, keepdim=True)
        ce = torch.where(counted, torch.log(mass[:, 0]) - (z[rows, y] - top[:, 0]), 0.0)
        p = e / mass
        p[rows, y] -= 1.0
        dz += p * (counted * ((1.0 - alpha) / c))[:, None]
        row_loss = row_loss + (1.0 - alpha) * ce
        second = ce.double().sum() / c
    loss = torch.stack([alpha * first + (1.0 - alpha) * second, first, second]).float()
    return dict(loss=loss, row_loss=row_loss, dlogits=dz.to(dt))


# ------------------------------------------------------------------- work
def work(case):
    b, op, m = BYTES[case["dtype"]], case["op"], case["m"]
    if op in ("gated", "train"):
        d, f, out = case["d"], case["f"], case["out"]
        weights = f * (2 * d + out)
        if op == "gated":
            return dict(bytes=(m * (d + out) + weights) * b, flops=2 * m * weights)
        dx = 1 if case["dx"] else 0
        return dict(bytes=(m * (d + 2 * out + dx * d) + 2 * weights) * b,
                    flops=2 * m * weights + 2 * m * f * (2 * out + 2 * d + 2 * dx * d))
    v, k = case["classes"], case["k"]
    if op == "top":
        return dict(bytes=m * (v * b + 8 * k), flops=m * v)
    labels = case["alpha"] < 1.0
    return dict(bytes=m * (2 * v * b + 8 * k + 4 + (4 if labels else 0)) + 12, flops=m * v * (8 if labels else 5))


# ------------------------------------------------------------------ exact
def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("gated", "train"):
        return _exact_gated(case, s)
    if op == "top":
        # a logit's order as a whole number, with the index below it: no two are equal
        bits = s["logits"].float().view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
        key = order * 2 ** 20 - torch.arange(case["classes"], device="cuda")
        ids = torch.topk(key, case["k"], dim=1, sorted=True).indices
        return dict(values=torch.gather(s["logits"].double(), 1, ids), ids=ids.to(torch.int32))
    return _exact_distill(case, s)


def _exact_gated(case, s):
    """By groups of rows: every sum in 64 bits, the activation from its definition."""
    m, piece = case["m"], 16_384
    wg, wu, wd = s["wg"].double(), s["wu"].double(), s["wd"].double()
    train = case["op"] == "train"
    y, dx = [], []
    grads = [torch.zeros_like(w) for w in (wg, wu, wd)] if train else None
    for at in range(0, m, piece):
        x = s["x"][at:at + piece].double()
        a, b = torch.mm(x, wg), torch.mm(x, wu)
        if case["act"] == "silu":
            gate = torch.sigmoid(a)
            slope = gate + a * gate * torch.sigmoid(-a)
        elif case["act"] == "gelu":
            gate = 0.5 * torch.erfc(-a / math.sqrt(2.0))
            slope = gate + a * torch.exp(-a.square() / 2.0) / math.sqrt(2.0 * math.pi)
        else:
            gate = torch.heaviside(a, torch.zeros((), dtype=a.dtype, device="cuda"))
            slope = gate
        h = a * gate * b
        y.append(torch.mm(h, wd))
        if train:
            dy = s["dy"][at:at + piece].double()
            dh = torch.mm(dy, wd.t())
            da, db = dh * b * slope, dh * (a * gate)
            if case["dx"]:
                dx.append(torch.addmm(torch.mm(da, wg.t()), db, wu.t()))
            for total, left, right in zip(grads, (x, x, h), (da, db, dy)):
                total.addmm_(left.t(), right)
    if not train:
        return torch.cat(y)
    return dict(y=torch.cat(y), dx=torch.cat(dx) if case["dx"] else None, dwg=grads[0], dwu=grads[1], dwd=grads[2])


def _exact_distill(case, s):
    """By groups of rows: log-softmax of both sides, and the divergence as it is defined."""
    m, t, alpha, piece = case["m"], case["temperature"], case["alpha"], 1_024
    kept = s["ids"] >= 0
    has = kept.any(dim=1)
    n = max(1, int(has.sum()))
    labels = s["labels"]
    counted = labels != IGNORE if labels is not None else None
    c = max(1, int(counted.sum())) if labels is not None else 1
    kd, ce, dz = [], [], []
    for at in range(0, m, piece):
        rows = slice(at, at + piece)
        z, ids, on = s["logits"][rows].double(), s["ids"][rows].long(), kept[rows]
        log_p = torch.log_softmax(z / t, dim=1)
        log_q = torch.log_softmax(torch.where(on, s["teacher"][rows].double() / t, -math.inf), dim=1)
        log_q = torch.where(on, log_q, -math.inf)
        q = torch.exp(log_q)
        apart = torch.where(on, q * (log_q - torch.gather(log_p, 1, ids.clamp(min=0))), 0.0)
        kd.append(apart.sum(dim=1) * t ** 2)
        target = torch.zeros_like(z)
        target.scatter_add_(1, ids.clamp(min=0), q)
        grad = (torch.exp(log_p) - target) * (alpha * t / n)
        grad[~has[rows]] = 0.0
        if labels is not None:
            y, on = labels[rows].long().clamp(min=0), counted[rows]
            log_p = torch.log_softmax(z, dim=1)
            ce.append(torch.where(on, -torch.gather(log_p, 1, y[:, None])[:, 0], 0.0))
            p = torch.exp(log_p)
            p.scatter_add_(1, y[:, None], torch.full_like(z[:, :1], -1.0))
            p[~on] = 0.0
            grad = grad + p * ((1.0 - alpha) / c)
        dz.append(grad)
    kd = torch.cat(kd)
    row_loss = alpha * kd
    first, second = kd.sum() / n, torch.zeros((), dtype=torch.float64, device="cuda")
    if labels is not None:
        ce = torch.cat(ce)
        row_loss = row_loss + (1.0 - alpha) * ce
        second = ce.sum() / c
    return dict(loss=torch.stack([alpha * first + (1.0 - alpha) * second, first, second]), row_loss=row_loss, dlogits=torch.cat(dz))
