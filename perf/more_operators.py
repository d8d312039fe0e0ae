"""The operators of an attention layer over what the sampler returns, as cases that can be timed and whose results can be compared.

Three operators, through the functions of layer_binding.py:

  attend   attention of targets over their sampled events with a learned bias for the events' age, by buckets: outputs (keys and values in rows of the
           events or gathered from a table of nodes), and training (outputs and gradients)
  block    what stands between two layers: norm of a branch, its gate and scale, the sum with the residual, the norm before the next branch
  distill  the loss of a student's scores of all candidates against a teacher's highest ones, with its gradient

With `own` false the same results come from elementary torch operations in 32 bits; exact() computes them from the definitions in 64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = torch.device("cuda", 0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- the cases -----------------------------------------------------------------------------------

def _attend(mode, lists, lens, most, heads, kv_heads, head_dim, **kw):
    """`most`: the fan-out (lens "sampled") or the longest history there can be; `nodes`: rows of the table that keys and values are gathered from."""
    c = dict(op="attend", mode=mode, lists=lists, lens=lens, most=most, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype="f32", buckets=32, nodes=0, masked=0.0,
             times=True, newest_first=lens == "sampled")
    c.update(kw)
    return c


def _block(mode, rows, dim, **kw):
    c = dict(op="block", mode=mode, rows=rows, dim=dim, dtype="f32", gate=True, center=False)
    c.update(kw)
    return c


def _distill(rows, candidates, top, **kw):
    c = dict(op="distill", rows=rows, candidates=candidates, top=top, dtype="f32", rest=False, masked=0.0, temperature=2.0)
    c.update(kw)
    return c


def listed():
    return [
        # serving: one small batch of targets, keys and values of all nodes lie in a table; latency counts
        dict(_attend("run", 600, "sampled", 10, 2, 2, 50, nodes=1 << 18), name="attend serve 600"),
        # the same for a large batch of a stream, in 16 bits
        dict(_attend("run", 66_600, "sampled", 10, 4, 4, 32, dtype="bf16", nodes=1 << 19), name="attend serve 66k bf16"),
        # a training mini-batch: the ten newest events of 4000 roots
        dict(_attend("train", 4000, "sampled", 10, 2, 2, 50), name="attend train 4000 lists"),
        # a large batch in 16 bits, events without features are masked
        dict(_attend("train", 131_072, "sampled", 10, 2, 2, 64, dtype="bf16", masked=0.05), name="attend train 128k lists bf16"),
        # whole histories of nodes, power-law lengths, heads that share keys and values
        dict(_attend("train", 3001, "histories", 100_000, 8, 4, 32, buckets=64), name="attend train histories"),
        # few very long sequences, biased by position: the work has to be split along them
        dict(_attend("run", 7, "long", 120_000, 8, 4, 64, dtype="bf16", times=False), name="attend long bf16"),
        # between two layers, for one small batch that is served
        dict(_block("run", 600, 100), name="block serve 600"),
        # the neighbours of a large batch, in 16 bits, an odd multiple of a line
        dict(_block("train", 66_600, 172, dtype="bf16", center=True), name="block train 66k bf16"),
        # all events of a million
        dict(_block("train", 1_000_003, 128, gate=False), name="block train 1M"),
        # a mini-batch, each event ranked against a thousand nodes
        dict(_distill(600, 1000, 10), name="distill 600x1000"),
        # the candidates of a larger graph, teacher's mass outside its highest scores counted, some events masked
        dict(_distill(4000, 10_000, 50, dtype="bf16", rest=True, masked=0.05), name="distill 4000x10k bf16"),
        # every node of a large graph is a candidate
        dict(_distill(200, 500_009, 100, rest=True), name="distill 200x500k"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "block", "block", "distill", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    mode = rng.choice(["run", "train", "train"])
    if kind == "block":
        dim = rng.choice([32, 64, 100, 128, 172, 173, 256, 600])
        return _block(mode, _log_uniform(rng, 1, 100_000_000 // dim), dim, dtype=dtype, gate=rng.choice([True, False]), center=rng.choice([True, False]))
    if kind == "distill":
        v = _log_uniform(rng, 50, 500_000)
        return _distill(_log_uniform(rng, 1, min(80_000_000 // v, 50_000)), v, min(_log_uniform(rng, 1, 200), v // 2), dtype=dtype, rest=rng.choice([True, False]),
                        masked=rng.choice([0.0, 0.1]), temperature=rng.choice([1.0, 2.0, 4.0]))
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 1, 2, 3, 4])
    head_dim = rng.choice([8, 16, 32, 50, 64, 43, 128])
    lens = rng.choice(["sampled", "sampled", "histories", "long"])
    more = dict(dtype=dtype, buckets=rng.choice([8, 32, 33, 64]), masked=rng.choice([0.0, 0.2]), times=rng.choice([True, True, False]))
    room = 60_000_000 // (heads * head_dim)                      # rows
    if lens == "sampled":
        f = rng.choice([5, 10, 20, 64])
        return _attend(mode, _log_uniform(rng, 20, max(room // f, 40)), lens, f, heads, kv_heads, head_dim, nodes=rng.choice([0, 100_000]) if mode == "run" else 0, **more)
    if lens == "histories":
        return _attend(mode, _log_uniform(rng, 50, 500), lens, _log_uniform(rng, 1000, 20_000), heads, kv_heads, head_dim, **more)
    s = rng.randint(1, 20)
    return _attend(mode, s, lens, _log_uniform(rng, 100, max(room // s, 200)), heads, kv_heads, head_dim, **more)


# ---- inputs --------------------------------------------------------------------------------------

def _length_set(c):
    r = np.random.default_rng(17)
    if c["lens"] == "sampled":          # the fan-out, or fewer where a node has fewer neighbours in the window; some have none
        return np.minimum(c["most"], (r.exponential(4.0 * c["most"], c["lists"])).astype(np.int64))
    if c["lens"] == "histories":        # power law
        return np.minimum(c["most"], (r.pareto(0.8, c["lists"]) * 20).astype(np.int64))
    return np.maximum(c["most"] - r.integers(0, max(c["most"] // 8, 1), c["lists"]), 1)


def _prepare_attend(c, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    rand = lambda *s: torch.rand(s, generator=g, device=DEV)      # noqa: E731
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)    # noqa: E731
    h, kv, d, dt, n = c["heads"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]], c["lists"]
    lens = np.random.default_rng([18, seed]).permutation(_length_set(c))      # all inputs of a case have as many rows
    rows, rowptr = int(lens.sum()), torch.from_numpy(np.concatenate([[0], np.cumsum(lens)])).to(DEV)
    have = c["nodes"] or rows
    s = dict(op="attend", mode=c["mode"], rowptr=rowptr, newest_first=c["newest_first"], q=randn(n, h, d).to(dt), k=randn(have, kv, d).to(dt), v=randn(have, kv, d).to(dt),
             scale=d ** -0.5, table=0.5 * randn(c["buckets"], h), t=None, ts=None, index=None, mask=None, dout=None)
    # borders from half an event (times) or one place on up to the longest list, in equal ratios: fine among the newest events, coarser and coarser beyond
    near = 0.5 if c["times"] else 1.0
    s["edges"] = torch.tensor([near * (c["most"] / near) ** (i / (c["buckets"] - 2)) for i in range(c["buckets"] - 1)], device=DEV)
    if c["times"]:                      # times of a list fall (newest first) or rise by about 1 an event; the target's is a little later than all of them
        seq = torch.searchsorted(rowptr, torch.arange(rows, device=DEV), right=True) - 1
        at = (torch.arange(rows, device=DEV) - rowptr[seq]).float()
        length = (rowptr[1:] - rowptr[:-1]).float()
        s["ts"] = (length[seq] - at if c["newest_first"] else at) + rand(rows)
        s["t"] = length + 1 + rand(n)
    if c["nodes"]:
        s["index"] = torch.randint(0, c["nodes"], (rows,), generator=g, device=DEV, dtype=torch.int32)
        s["index"][rand(rows) < 0.01] = -1                        # neighbours that the table does not hold
    if c["masked"]:
        s["mask"] = rand(rows) >= c["masked"]
        s["mask"][int(rowptr[n // 2]): int(rowptr[n // 2 + 1])] = False      # one list has nothing left
        if not c["nodes"]:
            s["k"][~s["mask"]] = float("nan")                     # nothing was ever written there
            s["v"][~s["mask"]] = float("nan")
    if c["mode"] == "train":
        s["dout"] = randn(n, h, d).to(dt)
    return s


def _prepare_block(c, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    n, d, dt = c["rows"], c["dim"], DTYPES[c["dtype"]]
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)    # noqa: E731
    s = dict(op="block", mode=c["mode"], center=c["center"], eps=1e-6, x=randn(n, d).to(dt), branch=(0.3 + 2 * randn(n, d)).to(dt), gate=randn(n, d).to(dt) if c["gate"] else None,
             scale=0.5 + 0.1 * randn(d), post=1 + 0.1 * randn(d), pre=1 + 0.1 * randn(d), dout=None, dnext=None)
    if c["mode"] == "train":
        s["dout"], s["dnext"] = randn(n, d).to(dt), randn(n, d).to(dt)
    return s


def _prepare_distill(c, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    b, v, k, dt = c["rows"], c["candidates"], c["top"], DTYPES[c["dtype"]]
    rand = lambda *s: torch.rand(s, generator=g, device=DEV)      # noqa: E731
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)    # noqa: E731
    part = v // k                                                 # one of every part of the candidates, all distinct
    ids = torch.randint(0, v, (b, 1), generator=g, device=DEV) + torch.arange(k, device=DEV) * part + (rand(b, k) * part).long()
    ids = (ids % v)[:, torch.randperm(k, generator=g, device=DEV)]
    teacher = 5 - 3 * rand(b, k).sort(1).values
    logits = 1.5 * randn(b, v)
    logits.scatter_add_(1, ids, (teacher - 2).to(logits.dtype))   # the student has learned something already
    ids[rand(b, k) < 0.02] = -1                                   # fewer candidates than the list has room for
    s = dict(op="distill", logits=logits.to(dt), ids=ids.int(), teacher=teacher, lse=None, weight=None, temperature=c["temperature"], scale=1.0 / b)
    if c["rest"]:
        s["lse"] = torch.logsumexp(teacher / c["temperature"], 1) + 0.05 + 0.4 * rand(b)
    if c["masked"]:
        s["weight"] = (rand(b) >= c["masked"]).float() * (0.5 + rand(b))
        s["logits"][s["weight"] == 0] = float("nan")
    return s


def prepare(case, seed):
    return {"attend": _prepare_attend, "block": _prepare_block, "distill": _prepare_distill}[case["op"]](case, seed)


# ---- plain forms ---------------------------------------------------------------------------------

def _plain_attend(s):
    dt, rowptr = s["q"].dtype, s["rowptr"]
    n, h, d = s["q"].shape
    rows = s["mask"].shape[0] if s["mask"] is not None else s["index"].shape[0] if s["index"] is not None else s["k"].shape[0]
    kv = s["k"].shape[1]
    row = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(rowptr, row, right=True) - 1
    keep = torch.ones(rows, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"]
    if s["ts"] is not None:
        age = (s["t"][seq] - s["ts"]).clamp(min=0)
    else:
        age = (row - rowptr[seq] if s["newest_first"] else rowptr[seq + 1] - 1 - row).float()
    bucket = torch.searchsorted(s["edges"], age, right=True)
    k, v = s["k"], s["v"]
    if s["index"] is not None:
        keep = keep & (s["index"] >= 0)
        at = s["index"].clamp(min=0).long()
        k, v = k[at], v[at]
    k, v = (torch.where(keep[:, None, None], x.float(), 0.0) for x in (k, v))
    spread = lambda x: x.repeat_interleave(h // kv, 1)            # noqa: E731
    q = s["q"].float()[seq]
    score = s["scale"] * (q * spread(k)).sum(-1) + s["table"][bucket]
    score = torch.where(keep[:, None], score, -math.inf)
    top = torch.full((n, h), -math.inf, device=DEV).scatter_reduce_(0, seq[:, None].expand(-1, h), score, "amax")
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(score - top[seq])
    total = torch.zeros((n, h), device=DEV).index_add_(0, seq, e)
    p = e / torch.where(total == 0, 1.0, total)[seq]
    out = torch.zeros((n, h, d), device=DEV).index_add_(0, seq, p[:, :, None] * spread(v))
    result = dict(out=out.to(dt))
    if s["mode"] == "run":
        return result
    dout = s["dout"].float()
    delta = (dout * out).sum(-1)
    dout = dout[seq]
    ds = p * ((dout * spread(v)).sum(-1) - delta[seq])
    gather = lambda x: x.reshape(rows, kv, h // kv, d).sum(2)     # noqa: E731
    scaled = s["scale"] * ds[:, :, None]
    result.update(dq=torch.zeros((n, h, d), device=DEV).index_add_(0, seq, scaled * spread(k)).to(dt), dk=gather(scaled * q).to(dt), dv=gather(p[:, :, None] * dout).to(dt),
                  dtable=torch.zeros_like(s["table"]).index_add_(0, bucket, ds))
    return result


def _normed(v, center, eps):
    """The normed rows and one over their norm."""
    if center:
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + eps)
    return v * r, r


def _through_norm(g, y, r, center):
    """Gradient by a norm's input, given that by its output y."""
    g = g - y * (g * y).mean(1, keepdim=True)
    if center:
        g = g - g.mean(1, keepdim=True)
    return g * r


def _plain_block(s):
    dt = s["x"].dtype
    y, r = _normed(s["branch"].float(), s["center"], s["eps"])
    z = torch.sigmoid(s["gate"].float()) if s["gate"] is not None else 1.0
    factor = s["scale"] * s["post"]
    out = s["x"].float() + factor * z * y
    m, rm = _normed(out, s["center"], s["eps"])
    result = dict(out=out.to(dt), next=(s["pre"] * m).to(dt))
    if s["mode"] == "run":
        return result
    dnext = s["dnext"].float()
    g = s["dout"].float() + _through_norm(dnext * s["pre"], m, rm, s["center"])
    both = (g * z * y).sum(0)
    result.update(dx=g.to(dt), dbranch=_through_norm(g * factor * z, y, r, s["center"]).to(dt),
                  dgate=(g * factor * y * z * torch.sigmoid(-s["gate"].float())).to(dt) if s["gate"] is not None else None,
                  dscale=s["post"] * both, dpost=s["scale"] * both, dpre=(dnext * m).sum(0))
    return result


def _plain_distill(s):
    dt, tau = s["logits"].dtype, s["temperature"]
    b, v = s["logits"].shape
    w = s["weight"] if s["weight"] is not None else torch.ones(b, device=DEV)
    x = torch.where((w != 0)[:, None], s["logits"].float(), 0.0) / tau
    listed_ = s["ids"] >= 0
    ids = s["ids"].clamp(min=0).long()
    t = torch.where(listed_, s["teacher"] / tau, -math.inf)
    if s["lse"] is None:
        top = t.amax(1, keepdim=True)
        e = torch.exp(t - torch.where(top == -math.inf, 0.0, top))
        total = e.sum(1, keepdim=True)
        lse_t = torch.log(torch.where(total == 0, 1.0, total)) + torch.where(top == -math.inf, 0.0, top)
    else:
        lse_t = s["lse"][:, None]
    p = torch.exp(t - lse_t)
    some = p > 0
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    lse = torch.log(e.sum(1, keepdim=True)) + top
    q = torch.exp(x - lse)
    loss = torch.where(some, p * (t - lse_t - (x.gather(1, ids) - lse)), 0.0).sum(1)
    at, spread = torch.nonzero(listed_, as_tuple=True)[0], torch.zeros((b, v), device=DEV)
    where = (at, ids[listed_])
    grad = q * p.sum(1, keepdim=True)
    if s["lse"] is not None:
        rest = (1 - p.sum(1, keepdim=True)).clamp(min=0)
        member = spread.index_put(where, torch.ones((), device=DEV)) > 0
        outside = torch.where(member, 0.0, q)
        left = outside.sum(1, keepdim=True)
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(left)), 0.0)[:, 0]
        grad = q * (p.sum(1, keepdim=True) + rest) - outside * rest / left
    grad = grad - spread.index_put(where, p[listed_], accumulate=True)
    return dict(loss=s["scale"] * (w * loss).sum(), rows=torch.where(w != 0, w * loss, 0.0), dlogits=((s["scale"] / tau * w)[:, None] * grad).to(dt))


# ---- one pass ------------------------------------------------------------------------------------

def run(s):
    if not own:
        return {"attend": _plain_attend, "block": _plain_block, "distill": _plain_distill}[s["op"]](s)
    from paper_2311_17410_amd import layer_binding as L
    if s["op"] == "distill":
        return L.distill(s["logits"], s["ids"], s["teacher"], lse=s["lse"], weight=s["weight"], temperature=s["temperature"], scale=s["scale"])
    if s["op"] == "block":
        given = dict(gate=s["gate"], scale=s["scale"], post=s["post"], pre=s["pre"], eps=s["eps"], center=s["center"])
        out = L.block_run(s["x"], s["branch"], **given)
        if s["mode"] == "train":
            out.update(L.block_grad(s["x"], s["branch"], dout=s["dout"], dnext=s["dnext"], **given))
        return out
    given = dict(t=s["t"], ts=s["ts"], edges=s["edges"], table=s["table"], mask=s["mask"], scale=s["scale"], newest_first=s["newest_first"])
    if s["mode"] == "run":
        return dict(out=L.attend_run(s["rowptr"], s["q"], s["k"], s["v"], index=s["index"], **given)["out"])
    r = L.attend_run(s["rowptr"], s["q"], s["k"], s["v"], save=True, **given)
    return dict(out=r["out"], **L.attend_grad(s["rowptr"], s["q"], s["k"], s["v"], r["saved"], s["dout"], **given))


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    c = case
    w, train = {"f32": 4, "bf16": 2}[c["dtype"]], c.get("mode") == "train"
    if c["op"] == "block":
        n, gate = c["rows"] * c["dim"], bool(c["gate"])
        return {"bytes": n * w * (4 + gate + (4 + gate if train else 0)), "flops": n * (20 + (40 if train else 0))}
    if c["op"] == "distill":
        n = c["rows"] * c["candidates"]
        return {"bytes": 2 * n * w + c["rows"] * (8 * c["top"] + 8), "flops": 8 * n}
    rows, d, h, kv = int(_length_set(c).sum()), c["head_dim"], c["heads"], c["kv_heads"]
    per_row = (2 + 2 * train) * kv * d * w + 4 * bool(c["times"]) + 4 * bool(c["nodes"]) + bool(c["masked"])
    return {"bytes": rows * per_row + c["lists"] * ((2 + 2 * train) * h * d * w + 12), "flops": rows * h * d * (4 + 8 * train)}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _leaf(v):
    return None if v is None else v.double().requires_grad_()


def _exact_attend(c, s):
    lens = s["rowptr"][1:] - s["rowptr"][:-1]
    n, h, d = s["q"].shape
    rows = int(lens.sum())
    owner = torch.repeat_interleave(torch.arange(n, device=DEV), lens)
    place = torch.arange(rows, device=DEV) - torch.repeat_interleave(s["rowptr"][:-1], lens)
    age = place if s["newest_first"] else lens[owner] - 1 - place
    if s["ts"] is not None:             # (a difference of two times in 32 bits, rounded to 32, is what the borders are compared with)
        age = (s["t"][owner].double() - s["ts"].double()).float().clamp(min=0)
    bucket = sum((age >= edge).long() for edge in s["edges"])
    keep = torch.ones(rows, dtype=torch.bool, device=DEV)
    if s["mask"] is not None:
        keep &= s["mask"]
    if s["index"] is not None:
        keep &= s["index"] >= 0
    left = torch.nonzero(keep)[:, 0]    # the events that count
    of = s["index"][left].long() if s["index"] is not None else left
    own_, group = owner[left], h // c["kv_heads"]
    q, table, k, v = _leaf(s["q"]), _leaf(s["table"]), _leaf(s["k"][of]), _leaf(s["v"][of])
    counts = torch.bincount(own_, minlength=n)
    parts = []
    for i in range(h):                  # a head at a time
        score = s["scale"] * (q[own_, i] * k[:, i // group]).sum(1) + table[bucket[left], i]
        with torch.no_grad():
            top = torch.segment_reduce(score, "max", lengths=counts, initial=-1e300)
        e = torch.exp(score - top[own_])
        total = torch.zeros(n, dtype=torch.float64, device=DEV).index_add(0, own_, e)
        parts.append(torch.zeros((n, d), dtype=torch.float64, device=DEV).index_add(0, own_, (e / total[own_])[:, None] * v[:, i // group]))
        if s["dout"] is not None:       # (the heads' gradients add up; only one head's graph is alive at a time)
            parts[-1].backward(s["dout"][:, i].double())
            parts[-1] = parts[-1].detach()
    out = dict(out=torch.stack(parts, 1).detach())
    if s["dout"] is not None:
        full = lambda g: torch.zeros((rows,) + g.shape[1:], dtype=torch.float64, device=DEV).index_copy_(0, left, g)      # noqa: E731
        out.update(dq=q.grad, dk=full(k.grad), dv=full(v.grad), dtable=table.grad)
    return out


def _exact_block(s):
    x, b, gate, scale, post, pre = (_leaf(s[name]) for name in ("x", "branch", "gate", "scale", "post", "pre"))

    def norm(v):
        v = v - v.mean(1, keepdim=True) if s["center"] else v
        return v / torch.sqrt((v ** 2).sum(1, keepdim=True) / v.shape[1] + s["eps"])

    branch = norm(b) * post
    if gate is not None:
        branch = branch / (1 + torch.exp(-gate))
    out = x + scale * branch
    following = norm(out) * pre
    result = dict(out=out.detach(), next=following.detach())
    if s["dout"] is not None:
        ((out * s["dout"].double()).sum() + (following * s["dnext"].double()).sum()).backward()
        result.update(dx=x.grad, dbranch=b.grad, dgate=None if gate is None else gate.grad, dscale=scale.grad, dpost=post.grad, dpre=pre.grad)
    return result


def _exact_distill(c, s):
    b, v = s["logits"].shape
    w = torch.ones(b, dtype=torch.float64, device=DEV) if s["weight"] is None else s["weight"].double()
    parts, grads = [], []
    step = max(1, 4_000_000 // v)
    for lo in range(0, b, step):        # some rows at a time
        cut = slice(lo, lo + step)
        raw = s["logits"][cut].double()
        x = raw.masked_fill((w[cut] == 0)[:, None], 0.0).requires_grad_()
        logq = torch.log_softmax(x / c["temperature"], 1)
        ids, t = s["ids"][cut].long(), s["teacher"][cut].double() / c["temperature"]
        t = t.masked_fill(ids < 0, -math.inf)
        logp = t - (torch.logsumexp(t, 1, keepdim=True) if s["lse"] is None else s["lse"][cut].double()[:, None])
        logp = logp.masked_fill(ids < 0, -math.inf)               # (a row without entries)
        p = torch.exp(logp)
        at = torch.gather(logq, 1, ids.clamp(min=0))
        loss = (p * (logp - at).masked_fill(ids < 0, 0.0)).sum(1)
        if s["lse"] is not None:
            rest = 1 - p.sum(1)
            inside = torch.zeros((x.shape[0], v + 1), dtype=torch.bool, device=DEV)
            inside.scatter_(1, torch.where(ids < 0, v, ids), True)
            loss = loss + rest * (torch.log(rest) - torch.logsumexp(logq.masked_fill(inside[:, :v], -math.inf), 1))
        loss = w[cut] * loss
        (s["scale"] * loss.sum()).backward()
        parts.append(loss.detach())
        grads.append(x.grad)
    rows = torch.cat(parts)
    return dict(loss=s["scale"] * rows.sum(), rows=rows, dlogits=torch.cat(grads))


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_block(s) if s["op"] == "block" else (_exact_distill if s["op"] == "distill" else _exact_attend)(case, s)
