"""The operators of a training step on what the sampler returns, as cases that can be timed and whose results can be compared.

Three operators, through the functions of train_binding.py:

  recur   the gated recurrence over ragged lists of events: training (states and gradients), states alone, and the step that takes one event per node
  loss    the paired log-ratio loss of true links against sampled ones, with its gradients
  adamw   one optimizer step over all tensors of a model, states in 32 or in 8 bits

With `own` false the same results come from elementary torch operations in 32 bits; exact() computes them from the definitions in 64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = torch.device("cuda", 0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256                                  # weights that share the scale of an 8-bit state
GOLDEN = 0x9E3779B97F4A7C15                  # increment and multipliers of splitmix64
MIX1, MIX2 = 0xBF58476D1CE4E5B9, 0x94D049BB133111EB
WORD = (1 << 64) - 1


# ---- the cases -----------------------------------------------------------------------------------

def _recur(mode, seqs, lens, most, dim, **kw):
    """`most`: the fan-out (lens "sampled") or the longest history there can be."""
    c = dict(op="recur", mode=mode, seqs=seqs, lens=lens, most=most, dim=dim, dtype="f32", decay=True, newest_first=lens == "sampled", start=False, states=False)
    c.update(kw)
    return c


def _step(batch, nodes, dim, **kw):
    c = dict(op="recur", mode="step", batch=batch, nodes=nodes, dim=dim, dtype="f32", decay=True)
    c.update(kw)
    return c


def _loss(events, negatives, dim, **kw):
    c = dict(op="loss", events=events, negatives=negatives, dim=dim, dtype="f32", ref=False, masked=0.0, smoothing=0.0)
    c.update(kw)
    return c


def _adamw(nodes, dim, layers, **kw):
    c = dict(op="adamw", nodes=nodes, dim=dim, feat=172, layers=layers, bits=32, grad="f32", copy=False)
    c.update(kw)
    return c


def listed():
    return [
        # serving: the events of one small batch change the states of their nodes; latency counts
        dict(_step(600, 1 << 18, 100), name="step 600"),
        # the same for a large batch of a stream
        dict(_step(66_600, 1 << 19, 172, dtype="bf16"), name="step 66k bf16"),
        # a training mini-batch: the ten newest neighbours of 4000 roots, the last state of each list counts
        dict(_recur("train", 4000, "sampled", 10, 100), name="train 4000 lists"),
        # lists of a large batch, in 16 bits
        dict(_recur("train", 131_072, "sampled", 10, 128, dtype="bf16"), name="train 128k lists bf16"),
        # whole histories of nodes, power-law lengths, every state is used; a state is carried over from the batch before
        dict(_recur("train", 3001, "histories", 100_000, 172, start=True, states=True), name="train histories"),
        # few very long sequences: the work has to be split along them
        dict(_recur("train", 7, "long", 120_000, 256, dtype="bf16", start=True, states=True), name="train long bf16"),
        # states of one stream of a million events, no gradients
        dict(_recur("states", 1, "long", 1_000_003, 128, states=True), name="states 1M events"),
        # link prediction on a mini-batch: one sampled non-link for each event
        dict(_loss(600, 1, 100), name="loss 600x1"),
        # continued training against a frozen model, some sampled non-links turn out to be links and are masked
        dict(_loss(4000, 50, 172, dtype="bf16", ref=True, masked=0.05, smoothing=0.1), name="loss 4000x50 bf16"),
        # few events, each ranked against thousands of nodes
        dict(_loss(200, 10_000, 128, masked=0.01), name="loss 200x10k"),
        # weights of a small model: many small tensors, one of them odd
        dict(_adamw(0, 100, 4), name="adamw small"),
        # learned embeddings of a million nodes, states in 8 bits, weights trained in 16 bits from a copy in 32
        dict(_adamw(1_000_003, 128, 2, bits=8, grad="bf16", copy=True), name="adamw 1M nodes 8 bits"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["train", "train", "states", "step", "loss", "loss", "adamw"])
    dim = rng.choice([32, 64, 100, 128, 172, 173, 256])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "step":
        return _step(_log_uniform(rng, 1, 80_000), _log_uniform(rng, 1 << 17, 1 << 19), dim, dtype=dtype, decay=rng.choice([True, True, False]))
    if kind == "loss":
        k = _log_uniform(rng, 1, 4000)
        return _loss(min(_log_uniform(rng, 100, 100_000), max((1 << 27) // (dim * (k + 2)), 1)), k, dim, dtype=dtype, ref=rng.choice([False, True]),
                     masked=rng.choice([0.0, round(rng.uniform(0.01, 0.5), 3)]), smoothing=rng.choice([0.0, 0.05]))
    if kind == "adamw":
        return _adamw(_log_uniform(rng, 1, 900_000), rng.choice([32, 64, 100, 128]), rng.randint(1, 6), bits=rng.choice([8, 32]), grad=dtype, copy=dtype == "bf16")
    lens = rng.choice(["sampled", "sampled", "histories", "long"])
    more = dict(dtype=dtype, decay=rng.choice([True, True, False]), start=rng.choice([True, False]), states=kind == "states" or rng.choice([True, False]))
    room = 100_000_000 // dim                                    # rows
    if lens == "sampled":
        f = rng.choice([1, 5, 10, 20, 64])
        return _recur(kind, _log_uniform(rng, 200, room // f), lens, f, dim, **more)
    if lens == "histories":
        return _recur(kind, _log_uniform(rng, 50, 1500), lens, _log_uniform(rng, 1000, 60_000), dim, **more)
    s = rng.randint(1, 20)
    return _recur(kind, s, lens, _log_uniform(rng, 1000, room // s), dim, **more)


# ---- inputs --------------------------------------------------------------------------------------

def _lengths(c, seed):
    """How many events each list holds; `seed` puts them in order, so that all inputs of a case have as many rows."""
    return np.random.default_rng([18, seed]).permutation(_length_set(c))


def _length_set(c):
    r = np.random.default_rng(17)
    if c["lens"] == "sampled":          # the fan-out, or fewer where a node has fewer neighbours in the window; some have none
        return np.minimum(c["most"], (r.exponential(4.0 * c["most"], c["seqs"])).astype(np.int64))
    if c["lens"] == "histories":        # power law
        return np.minimum(c["most"], (r.pareto(0.8, c["seqs"]) * 20).astype(np.int64))
    return np.maximum(c["most"] - r.integers(0, max(c["most"] // 8, 1), c["seqs"]), 1)


def _prepare_recur(c, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    rand = lambda *s: torch.rand(s, generator=g, device=DEV)      # noqa: E731
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)    # noqa: E731
    d, dt = c["dim"], DTYPES[c["dtype"]]
    s = dict(op="recur", mode=c["mode"], decay=(0.5 * randn(d)).exp() if c["decay"] else None)
    if c["mode"] == "step":
        ids = torch.randperm(c["nodes"], generator=g, device=DEV)[: c["batch"]].int()
        ids[rand(c["batch"]) < 0.01] = -1                         # events of nodes that hold no state
        s.update(ids=ids, state=randn(c["nodes"], d), state_ts=rand(c["nodes"]), ts=1 + rand(c["batch"]))
        if not c["decay"]:
            s.update(ts=None, state_ts=None)
        rows = c["batch"]
    else:
        lens = _lengths(c, seed)
        rows, rowptr = int(lens.sum()), torch.from_numpy(np.concatenate([[0], np.cumsum(lens)])).to(DEV)
        s.update(rowptr=rowptr, longest=int(lens.max(initial=0)), newest_first=c["newest_first"], states=c["states"], ts=None, h0=None, t0=None)
        if c["decay"]:                  # times of a list fall (newest first) or rise by about 0.3 an event
            seq = torch.searchsorted(rowptr, torch.arange(rows, device=DEV), right=True) - 1
            at = (torch.arange(rows, device=DEV) - rowptr[seq]).float()
            s["ts"] = 0.3 * ((c["most"] - at if c["newest_first"] else at) + rand(rows))
        if c["start"]:
            s["h0"] = randn(c["seqs"], d)
            s["t0"] = -rand(c["seqs"]) if c["decay"] else None
        if c["mode"] == "train":
            s["dlast"] = randn(c["seqs"], d)
            s["dh"] = (0.1 * randn(rows, d)).to(dt) if c["states"] else None
    s["u"], s["x"] = (1.5 * randn(rows, d) - 1).to(dt), randn(rows, d).to(dt)
    return s


def _prepare_loss(c, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    b, k, d, dt = c["events"], c["negatives"], c["dim"], DTYPES[c["dtype"]]
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)    # noqa: E731
    anchor = randn(b, d)
    s = dict(op="loss", anchor=anchor.to(dt), pos=(0.1 * anchor + randn(b, d)).to(dt), neg=randn(b, k, d).to(dt), ref=randn(b, k) if c["ref"] else None, weight=None,
             beta=2.0 / math.sqrt(d), smoothing=c["smoothing"], scale=1.0 / (b * k))
    if c["masked"]:
        s["weight"] = (torch.rand((b, k), generator=g, device=DEV) >= c["masked"]).float()
        s["weight"][:: 97] = 0.0                                  # events that are masked altogether
        s["neg"][s["weight"] == 0] = float("nan")                 # nothing was ever written there
    return s


def _sizes(c):
    """Weights of each tensor: the embeddings, then matrices and vectors of the layers."""
    d = c["dim"]
    return ([c["nodes"] * d] if c["nodes"] else []) + c["layers"] * [c["feat"] * d, c["feat"] * d, d, d, d, d * d, d + 1]


def _prepare_adamw(c, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    sizes = _sizes(c)
    blocks = [-(-n // BLOCK) for n in sizes]
    first = np.concatenate([[0], np.cumsum(blocks)])
    total = int(first[-1]) * BLOCK                                # every tensor begins at a multiple of BLOCK in the flat buffers
    randn = lambda n: torch.randn(n, generator=g, device=DEV)     # noqa: E731
    real = torch.zeros(total, dtype=torch.bool, device=DEV)
    for n, f in zip(sizes, first):
        real[f * BLOCK: f * BLOCK + n] = True
    flat = dict(param=0.1 * randn(total) * real, grad=(0.02 * randn(total) * real).to(DTYPES[c["grad"]]))
    flat["copy"] = flat["param"].bfloat16() if c["copy"] else None
    if c["bits"] == 32:
        flat.update(m=0.01 * randn(total) * real, v=(0.02 * randn(total) * real).square())
    else:
        flat.update(m=(90 * randn(total) * real).clamp(-448, 448).to(torch.float8_e4m3fn), v=(90 * randn(total).abs() * real).clamp(max=448).to(torch.float8_e4m3fn),
                    m_scale=1e-4 * (1 + torch.rand(total // BLOCK, generator=g, device=DEV)), v_scale=2e-4 * (1 + torch.rand(total // BLOCK, generator=g, device=DEV)))
    decays = [0.01 if n > 4 * c["dim"] else 0.0 for n in sizes]   # vectors do not decay
    s = dict(op="adamw", bits=c["bits"], flat=flat, real=real, t=10, seed=seed, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, clip=torch.full((1,), 0.7, device=DEV),
             decay=torch.from_numpy(np.repeat(np.float32(decays), blocks)).to(DEV)[:, None])
    if own:                             # the optimizer that a program keeps
        from paper_2311_17410_amd import train_binding as T
        def parts(name, per=1):
            return None if flat.get(name) is None else [flat[name][f * BLOCK // per: f * BLOCK // per + -(-n // per)] for n, f in zip(sizes, first)]
        s["opt"] = T.AdamW(parts("param"), parts("grad"), copies=parts("copy"), bits=c["bits"], betas=s["betas"], eps=s["eps"], weight_decay=decays, seed=seed,
                           states=(parts("m"), parts("v"), parts("m_scale", BLOCK), parts("v_scale", BLOCK)))
    return s


def prepare(case, seed):
    return {"recur": _prepare_recur, "loss": _prepare_loss, "adamw": _prepare_adamw}[case["op"]](case, seed)


# ---- plain forms ---------------------------------------------------------------------------------

def _scan(a, b, longest):
    """h_i = a_i h_{i-1} + b_i over the rows, in log2(longest) rounds; a is 0 where a sequence begins."""
    by = 1
    while by < longest:
        b = torch.cat((b[:by], b[by:] + a[by:] * b[:-by]))
        a = torch.cat((a[:by], a[by:] * a[:-by]))
        by *= 2
    return b


def _plain_recur(s):
    dt, flip = s["u"].dtype, (lambda v: v.flip(0)) if s["newest_first"] else (lambda v: v)
    rowptr, n = s["rowptr"], s["u"].shape[0]
    seqs, d = rowptr.shape[0] - 1, s["u"].shape[1]
    u, x = flip(s["u"]).float(), flip(s["x"]).float()
    seq = flip(torch.searchsorted(rowptr, torch.arange(n, device=DEV), right=True) - 1)
    edge = torch.ones(1, dtype=torch.bool, device=DEV)
    begins, ends = torch.cat((edge, seq[1:] != seq[:-1])), torch.cat((seq[1:] != seq[:-1], edge))
    z, f = torch.sigmoid(u), torch.sigmoid(-u)
    if s["decay"] is not None:
        ts = flip(s["ts"])
        before = torch.cat((ts[:1], ts[:-1]))
        gap = (ts - torch.where(begins, s["t0"][seq] if s["t0"] is not None else ts, before)).clamp(min=0)[:, None]
        f = f * torch.exp(-s["decay"] * gap)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros((seqs, d), device=DEV)
    at0 = begins[:, None]
    h = _scan(torch.where(at0, 0.0, f), z * x + torch.where(at0, f * h0[seq], 0.0), s["longest"])
    last = h0.clone()
    last[seq[ends]] = h[ends]
    out = dict(h=flip(h).to(dt) if s["states"] else None, last=last)
    if s["mode"] == "states":
        return out
    before = torch.where(at0, h0[seq], torch.cat((h[:1], h[:-1])))
    grad = torch.where(ends[:, None], s["dlast"][seq], 0.0)
    if s["dh"] is not None:
        grad = grad + flip(s["dh"]).float()
    back = torch.where(ends[:, None], 0.0, torch.cat((f[1:], f[:1])))
    grad = _scan(back.flip(0), grad.flip(0), s["longest"]).flip(0)
    dh0 = s["dlast"].clone()
    dh0[seq[begins]] = (f * grad)[begins]
    out.update(dx=flip(z * grad).to(dt), du=flip(z * grad * (torch.sigmoid(-u) * x - f * before)).to(dt), dh0=dh0 if s["h0"] is not None else None,
               ddecay=-(gap * grad * f * before).sum(0) if s["decay"] is not None else None)
    return out


def _plain_step(s):
    held = s["ids"] >= 0
    ids, u, x = s["ids"][held].long(), s["u"][held].float(), s["x"][held].float()
    f = torch.sigmoid(-u)
    if s["decay"] is not None:
        ts = s["ts"][held]
        f = f * torch.exp(-s["decay"] * (ts - s["state_ts"][ids]).clamp(min=0)[:, None])
        s["state_ts"][ids] = ts
    h = f * s["state"][ids] + torch.sigmoid(u) * x
    s["state"][ids] = h
    out = torch.zeros_like(s["u"])
    out[held] = h.to(out.dtype)
    return dict(out=out, state=s["state"], state_ts=s["state_ts"])


def _plain_loss(s):
    dt = s["anchor"].dtype
    some = s["weight"] != 0 if s["weight"] is not None else torch.ones(s["neg"].shape[:2], dtype=torch.bool, device=DEV)
    w = s["weight"] if s["weight"] is not None else 1.0
    a, p, n = s["anchor"].float(), s["pos"].float(), torch.where(some[:, :, None], s["neg"].float(), 0.0)
    ratio = (a * p).sum(-1)[:, None] - (a[:, None] * n).sum(-1)
    margin = torch.where(some, s["beta"] * (ratio if s["ref"] is None else ratio - s["ref"]), 0.0)
    tail = torch.log1p(torch.exp(-margin.abs()))                  # softplus(-m) = tail + max(-m, 0)
    eps = s["smoothing"]
    loss = s["scale"] * (w * ((1 - eps) * (tail + (-margin).clamp(min=0)) + eps * (tail + margin.clamp(min=0)))).sum()
    c = torch.where(some, s["scale"] * s["beta"] * w * (eps - torch.sigmoid(-margin)), 0.0)
    csum = c.sum(1, keepdim=True)
    return dict(loss=loss, margin=margin, danchor=(csum * p - (c[:, :, None] * n).sum(1)).to(dt), dpos=(csum * a).to(dt), dneg=(-c[:, :, None] * a[:, None]).to(dt))


def _signed(v):
    return v - (1 << 64) if v >> 63 else v


def _random16(key, total):
    """Sixteen bits for each weight: the counter-based generator splitmix64, a word for every four weights."""
    z = torch.arange(1, total // 4 + 1, device=DEV) * _signed(GOLDEN) + _signed(key)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(MIX1)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(MIX2)
    z = z ^ ((z >> 31) & ((1 << 33) - 1))
    return torch.stack([(z >> by) & 0xFFFF for by in (0, 16, 32, 48)], 1).reshape(-1, BLOCK).int()


def _key(seed, t):
    z = (seed + GOLDEN * t) & WORD
    z = ((z ^ (z >> 30)) * MIX1) & WORD
    z = ((z ^ (z >> 27)) * MIX2) & WORD
    return z ^ (z >> 31)


def _to_8_bits(v, signed, random, real):
    """Rows of BLOCK values -> codes (e4m3, normal values only) and a scale for each row; rounded up or down at random, right on average."""
    top = v.abs().amax(1, keepdim=True)
    top = torch.where(top < 2.0 ** -100, 0.0, top)
    y = v * torch.where(top > 0, torch.full_like(top, 448.0) / top, 0.0)
    if not signed:
        y = torch.where(top > 0, y.clamp(min=2.0 ** -6), 0.0)
    bits = y.view(torch.int32)
    code = (((bits & 0x7FFFFFFF) + (random << 4)) >> 20) - (120 << 3)
    code = torch.where(real & (y.abs() >= 2.0 ** -6), code | ((bits >> 24) & 0x80), 0)
    return code.to(torch.uint8).view(torch.float8_e4m3fn).reshape(-1), (top * (1.0 / 448.0)).reshape(-1)


def _plain_adamw(s):
    f, t, (b1, b2) = s["flat"], s["t"], s["betas"]
    rows = lambda v: v.reshape(-1, BLOCK)                         # noqa: E731
    g = rows(f["grad"]).float() * s["clip"]
    if s["bits"] == 32:
        m, v = rows(f["m"]), rows(f["v"])
    else:
        m, v = rows(f["m"]).float() * f["m_scale"][:, None], (rows(f["v"]).float() * f["v_scale"][:, None]).square()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * (g * g)
    r = torch.sqrt(v)
    p = rows(f["param"]) * (1 - s["lr"] * s["decay"]) - (s["lr"] / (1 - b1 ** t)) * m / (r * (1 / math.sqrt(1 - b2 ** t)) + s["eps"])
    f["param"].copy_(p.reshape(-1))
    if f["copy"] is not None:
        f["copy"].copy_(f["param"])
    if s["bits"] == 32:
        f["m"].copy_(m.reshape(-1))
        f["v"].copy_(v.reshape(-1))
    else:
        random = _random16(_key(s["seed"], t), p.numel())
        for name, value in (("m", m), ("v", r)):
            code, scale = _to_8_bits(value, name == "m", random, rows(s["real"]))
            f[name].copy_(code)
            f[name + "_scale"].copy_(scale)
    return _written(f)


def _written(flat):
    return {name: v for name, v in flat.items() if name != "grad"}


# ---- one pass ------------------------------------------------------------------------------------

def run(s):
    if s["op"] == "adamw":
        s["t"] += 1
        if not own:
            return _plain_adamw(s)
        s["opt"].step(s["lr"], s["t"], s["clip"])
        return _written(s["flat"])
    if not own:
        return _plain_loss(s) if s["op"] == "loss" else _plain_step(s) if s["mode"] == "step" else _plain_recur(s)
    from paper_2311_17410_amd import train_binding as T
    if s["op"] == "loss":
        return T.pair_loss(s["anchor"], s["pos"], s["neg"], ref=s["ref"], weight=s["weight"], beta=s["beta"], smoothing=s["smoothing"], scale=s["scale"])
    if s["mode"] == "step":
        out = T.recur_step(s["ids"], s["u"], s["x"], s["state"], ts=s["ts"], decay=s["decay"], state_ts=s["state_ts"])
        return dict(out=out, state=s["state"], state_ts=s["state_ts"])
    given = dict(ts=s["ts"], decay=s["decay"], h0=s["h0"], t0=s["t0"], newest_first=s["newest_first"])
    r = T.recur_run(s["rowptr"], s["u"], s["x"], states=s["states"], save=s["mode"] == "train", **given)
    out = dict(h=r["h"], last=r["last"])
    if s["mode"] == "train":
        out.update(T.recur_grad(s["rowptr"], s["u"], s["x"], r["saved"], dh=s["dh"], dlast=s["dlast"], **given))
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    c, size = case, {"f32": 4, "bf16": 2}
    if c["op"] == "adamw":
        n = sum(_sizes(c))
        states = 16 if c["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (8 + size[c["grad"]] + states + (2 if c["copy"] else 0)), "flops": 15 * n}
    d, w = c["dim"], size[c["dtype"]]
    if c["op"] == "loss":
        b, k = c["events"], c["negatives"]
        read = b * k * (4 * bool(c["ref"]) + 4 * bool(c["masked"]))
        return {"bytes": 2 * (2 + k) * b * d * w + read + 4 * b * k, "flops": 6 * (k + 1) * b * d}
    if c["mode"] == "step":
        return {"bytes": c["batch"] * (d * (3 * w + 8) + 4 + 12 * bool(c["decay"])), "flops": 12 * c["batch"] * d}
    rows, seqs = int(_length_set(c).sum()), c["seqs"]
    states, train, start = bool(c["states"]), c["mode"] == "train", bool(c["start"])
    values = rows * d * (2 + states + (2 * 2 + states if train else 0))      # u, x, h; and u, x, dh, du, dx
    per_list = seqs * d * 4 * (1 + start + (1 + 2 * start if train else 0)) + 8 * seqs
    return {"bytes": values * w + per_list + 4 * rows * (1 + train) * bool(c["decay"]), "flops": rows * d * (12 + 25 * train)}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_scan(a, b):
    """h_i = a_i h_{i-1} + b_i row after row, for all pieces of the rows at once; then the pieces one after the other."""
    n, d = b.shape
    piece = max(1, int(math.sqrt(n)))
    pieces = -(-n // piece)
    pad = lambda v: torch.cat((v, v.new_zeros((pieces * piece - n, d)))).reshape(pieces, piece, d)      # noqa: E731
    a, b = pad(a), pad(b)
    for i in range(1, piece):
        b[:, i] += a[:, i] * b[:, i - 1]
        a[:, i] *= a[:, i - 1]
    carry = b.new_zeros(d)
    for k in range(pieces):
        b[k] += a[k] * carry
        carry = b[k, -1].clone()
    return b.reshape(-1, d)[:n]


def _exact_recur(c, s):
    n, seqs = s["u"].shape[0], c["seqs"]
    lens = (s["rowptr"][1:] - s["rowptr"][:-1])
    order = torch.arange(n, device=DEV)
    seq = torch.repeat_interleave(torch.arange(seqs, device=DEV), lens)
    if s["newest_first"]:               # row that is walked i-th: lists in their order, each from its last row to its first
        order = s["rowptr"][seq] + s["rowptr"][seq + 1] - 1 - order
    u, x = s["u"][order].double(), s["x"][order].double()
    first, final = s["rowptr"][:-1][lens > 0], s["rowptr"][1:][lens > 0] - 1
    z, q = 1 / (1 + torch.exp(-u)), 1 / (1 + torch.exp(u))
    f, gap = q.clone(), None
    if s["decay"] is not None:
        t = s["ts"][order].double()
        since = torch.zeros_like(t)
        since[1:] = t[1:] - t[:-1]
        since[first] = t[first] - s["t0"].double()[lens > 0] if s["t0"] is not None else 0.0
        gap = since.clamp(min=0)[:, None]
        f *= torch.exp(-gap * s["decay"].double())
    h0 = s["h0"].double() if s["h0"] is not None else torch.zeros((seqs, c["dim"]), dtype=torch.float64, device=DEV)
    a, b = f.clone(), z * x
    a[first] = 0
    b[first] += f[first] * h0[lens > 0]
    h = _exact_scan(a, b)
    del a, b
    last = h0.clone()
    last[lens > 0] = h[final]
    out = dict(h=torch.empty_like(h).index_copy_(0, order, h) if s["states"] else None, last=last)
    if c["mode"] == "states":
        return out
    g = torch.zeros_like(h) if s["dh"] is None else s["dh"][order].double()
    g[final] += s["dlast"].double()[lens > 0]
    a = torch.zeros_like(f)
    a[:-1] = f[1:]
    a[final] = 0
    g = _exact_scan(a.flip(0), g.flip(0)).flip(0)
    del a
    h = torch.roll(h, 1, 0)             # the state before each event
    h[first] = h0[lens > 0]
    back = lambda v: torch.empty_like(v).index_copy_(0, order, v)      # noqa: E731
    dh0 = s["dlast"].double()
    dh0[lens > 0] = f[first] * g[first]
    out.update(dx=back(z * g), du=back(z * q * x * g - z * f * h * g), dh0=dh0 if s["h0"] is not None else None,
               ddecay=-(gap * g * f * h).sum(0) if gap is not None else None)
    return out


def _exact_step(s):
    out, state = torch.zeros(s["u"].shape, dtype=torch.float64, device=DEV), s["state"].double()
    state_ts = None if s["state_ts"] is None else s["state_ts"].double()
    rows = torch.nonzero(s["ids"] >= 0)[:, 0]
    ids = s["ids"][rows].long()
    u, keep = s["u"][rows].double(), 1.0
    if state_ts is not None:
        keep = torch.exp(-torch.outer((s["ts"][rows].double() - state_ts[ids]).clamp(min=0), s["decay"].double()))
        state_ts[ids] = s["ts"][rows].double()
    state[ids] = out[rows] = (keep * state[ids] * torch.exp(-u) + s["x"][rows].double()) / (1 + torch.exp(-u))
    return dict(out=out, state=state, state_ts=state_ts)


def _exact_loss(s):
    a, p = s["anchor"].double(), s["pos"].double()
    b, k, d = s["neg"].shape
    w = (torch.ones((b, k), device=DEV) if s["weight"] is None else s["weight"]).double()
    ref = 0.0 if s["ref"] is None else s["ref"].double()
    diff = p[:, None] - s["neg"].double()
    diff[w == 0] = 0
    margin = (s["beta"] * (torch.matmul(diff, a[:, :, None])[:, :, 0] - ref)).masked_fill(w == 0, 0.0)
    eps = s["smoothing"]
    loss = s["scale"] * (w * (torch.logaddexp(torch.zeros_like(margin), -margin) + eps * margin)).sum()
    slope = s["scale"] * s["beta"] * w * (eps - 1 / (1 + torch.exp(margin)))
    return dict(loss=loss, margin=margin, danchor=(slope[:, :, None] * diff).sum(1), dpos=slope.sum(1)[:, None] * a, dneg=-slope[:, :, None] * a[:, None])


def _exact_adamw(s):
    f, t, (b1, b2) = s["flat"], s["t"] + 1, s["betas"]
    g = f["grad"].double() * s["clip"].double()
    m, v = f["m"].double(), f["v"].double()
    if s["bits"] == 8:
        m, v = m * f["m_scale"].double().repeat_interleave(BLOCK), (v * f["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m, v = m + (1 - b1) * (g - m), v + (1 - b2) * (g * g - v)
    decay = s["decay"].double().reshape(-1).repeat_interleave(BLOCK)
    p = f["param"].double()
    p = p - s["lr"] * decay * p - s["lr"] * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + s["eps"])
    copy = None if f["copy"] is None else p
    if s["bits"] == 32:
        return dict(param=p, copy=copy, m=m, v=v)
    tops = lambda v: v.reshape(-1, BLOCK).abs().amax(1) / 448      # noqa: E731
    return dict(param=p, copy=copy, m=None, v=None, m_scale=tops(m), v_scale=tops(v.sqrt()))      # codes are rounded at random


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "adamw":
        return _exact_adamw(s)
    return _exact_loss(s) if s["op"] == "loss" else _exact_step(s) if s["mode"] == "step" else _exact_recur(case, s)
