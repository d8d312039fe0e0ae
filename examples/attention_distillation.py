#!/usr/bin/env python3
"""Trains a small temporal attention model to rank all items as a teacher with a longer memory does, on one GPU.

A synthetic stream of (user, item, time) events in which users keep to the items of their kind.  For every event of a batch the model
attends from the user to the user's newest events, puts what it found behind norm, gate and residual, and scores every item; it learns the
teacher's highest scores.  The teacher has no weights: it averages the features of four times as many events.

  tns_run            the newest events of each user before its time (padding removed), for the model and for the teacher
  tns_cache_fetch    the feature rows of the neighbours
  products           queries, keys, values, gates and scores (torch)
  tns_attend_run     one output per user and head over its events, with a learned bias by the events' age
  tns_block_run      residual + scale sigmoid(gate) post norm(branch), and the norm before the scores
  tns_distill        loss and gradient of the scores against the teacher's highest ones and their mass
  tns_block_grad, tns_attend_grad   gradients; products give the weights'
  tns_adamw_step     one step over all weights

    python examples/attention_distillation.py [--steps 200]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for p in (ROOT, os.path.join(ROOT, "examples")):
    if p not in sys.path:
        sys.path.insert(0, p)

from link_training import stream  # noqa: E402
from paper_2311_17410_amd import binding as B  # noqa: E402
from paper_2311_17410_amd import cache_binding as KB  # noqa: E402
from paper_2311_17410_amd import layer_binding as L  # noqa: E402
from paper_2311_17410_amd import train_binding as T  # noqa: E402

TEMPERATURE = 0.5


class Model:
    """One attention layer over sampled events: its weights, their gradients and the optimizer that steps them."""

    def __init__(self, feat, heads, dim, buckets, seed, device):
        g = torch.Generator(device).manual_seed(seed)
        wide = heads * dim
        shapes = dict(own=(feat, wide), query=(feat, wide), key=(feat, wide), value=(feat, wide), gate=(feat, wide), item=(feat, wide), table=(buckets, heads), scale=(wide,),
                      post=(wide,), pre=(wide,))
        self.heads, self.dim = heads, dim
        self.w = {n: torch.randn(s, generator=g, device=device) / feat ** 0.5 if s[0] == feat else torch.zeros(s, device=device) for n, s in shapes.items()}
        for n in ("scale", "post", "pre"):
            self.w[n].fill_(1.0)
        self.g = {n: torch.zeros_like(v) for n, v in self.w.items()}
        self.edges = 0.05 * 2.0 ** torch.arange(buckets - 1, device=device)      # ages: a twentieth, a tenth, ... of the time that passes in all events
        self.opt = T.AdamW(list(self.w.values()), list(self.g.values()), weight_decay=[0.01 if s[0] == feat else 0.0 for s in shapes.values()])
        self.t = 0

    def forward(self, own, rowptr, events, t, ts, items):
        """Scores of all items for the owners of the lists, and what backward needs.  `events`: features of the lists' rows; `own`, `items`: of owners and items."""
        w, heads = self.w, (-1, self.heads, self.dim)
        x, z = own @ w["own"], own @ w["gate"]
        q, k, v = (own @ w["query"]).view(heads), (events @ w["key"]).view(heads), (events @ w["value"]).view(heads)
        lists = dict(t=t, ts=ts, edges=self.edges, table=w["table"], newest_first=True)
        a = L.attend_run(rowptr, q, k, v, save=True, **lists)
        branch = a["out"].view(x.shape)
        between = dict(gate=z, scale=w["scale"], post=w["post"], pre=w["pre"])
        b = L.block_run(x, branch, **between)
        embedded = items @ w["item"]
        return b["next"] @ embedded.t(), dict(own=own, rowptr=rowptr, events=events, items=items, x=x, qkv=(q, k, v), lists=lists, saved=a["saved"], branch=branch,
                                              between=between, next=b["next"], embedded=embedded)

    def backward(self, dscores, kept):
        """Gradients of all weights, given those by the scores."""
        g, c = self.g, kept
        d = L.block_grad(c["x"], c["branch"], dnext=dscores @ c["embedded"], **c["between"])
        a = L.attend_grad(c["rowptr"], *c["qkv"], c["saved"], d["dbranch"].view(-1, self.heads, self.dim), **c["lists"])
        for name, given, by in (("own", c["own"], d["dx"]), ("gate", c["own"], d["dgate"]), ("query", c["own"], a["dq"]), ("key", c["events"], a["dk"]), ("value", c["events"], a["dv"]),
                                ("item", c["items"], dscores.t() @ c["next"])):
            torch.matmul(given.t(), by.reshape(given.shape[0], -1), out=g[name])
        for name, by in (("table", a["dtable"]), ("scale", d["dscale"]), ("post", d["dpost"]), ("pre", d["dpre"])):
            g[name].copy_(by)

    def step(self, lr):
        norm = torch.cat([g.reshape(-1) for g in self.g.values()]).norm()
        self.t += 1
        self.opt.step(lr, self.t, (1.0 / norm.clamp(min=1.0)).reshape(1))


def teach(rowptr, events, items, top):
    """The teacher's highest scores of all items, and the logarithm of the sum over all: by the mean of the events' features."""
    n = rowptr.shape[0] - 1
    of = torch.repeat_interleave(torch.arange(n, device=events.device), rowptr[1:] - rowptr[:-1], output_size=events.shape[0])
    mean = torch.zeros((n, events.shape[1]), device=events.device).index_add_(0, of, events) / (rowptr[1:] - rowptr[:-1]).clamp(min=1)[:, None]
    scores = mean @ items.t()
    best, ids = scores.topk(top, 1)
    return ids.int(), best, torch.logsumexp(scores / TEMPERATURE, 1)


def train(steps=200, batch=500, heads=2, dim=32, feat=32, top=20, fanout=10, lr=1e-2, seed=0, users=1000, items=600, kinds=8, report=None, model=None):
    """Returns the losses, step by step, and the last step's model, scores and what led to them."""
    dev, nodes, warm = torch.device("cuda", 0), users + items, 20_000
    user, item, time = stream(users, items, kinds, warm + steps * batch, seed)
    plans = [B.Plan(nodes, f, B.TNS_POLICY_RECENT, flags=B.TNS_FLAG_DEVICE_INGEST) for f in (fanout, 4 * fanout)]
    d_user, d_item, d_time = (torch.from_numpy(v).to(dev) for v in (user, item, time))

    def ingest(lo, hi):
        a, b, t = d_user[lo:hi], d_item[lo:hi], d_time[lo:hi]
        for plan in plans:
            plan.add_edges_device(torch.cat((a, b)), torch.cat((b, a)), torch.cat((t, t)))

    gen = torch.Generator(dev).manual_seed(seed)
    features = 0.3 * torch.randn((nodes, feat), generator=gen, device=dev)
    kind = torch.arange(nodes, device=dev) % kinds
    kind[users:] = torch.arange(items, device=dev) % kinds
    features[:, :kinds] += torch.nn.functional.one_hot(kind, kinds).float()
    cache = KB.Cache(nodes, max(nodes // 5, 1), feat)
    model = model or Model(feat, heads, dim, 8, seed, dev)
    losses = []
    ingest(0, warm)
    for s in range(steps):
        lo, hi = warm + s * batch, warm + (s + 1) * batch
        roots, at = d_user[lo:hi], d_time[lo:hi]
        found = []
        for plan in plans:
            got = plan.run(roots, None, at)
            rows = int(got["rowptr"][-1])
            found.append((got["rowptr"], cache.fetch(got["cmp_nbr"][:rows], features)[0], got["cmp_ts"][:rows]))
        ids, best, lse = teach(found[1][0], found[1][1], features[users:], top)
        rowptr, events, ts = found[0]
        scores, kept = model.forward(features[roots.long()], rowptr, events, at.contiguous(), ts, features[users:])
        out = L.distill(scores, ids, best, lse=lse, temperature=TEMPERATURE, scale=1.0 / batch)
        model.backward(out["dlogits"], kept)
        model.step(lr)
        ingest(lo, hi)
        losses.append(out["loss"])
        if report and (s + 1) % report == 0:
            print(f"step {s + 1:5d}  loss {float(torch.stack(losses[-report:]).mean()):.4f}", flush=True)
    losses = torch.stack(losses).tolist()
    cache.close()
    for plan in plans:
        plan.close()
    return losses, model, dict(kept, scores=scores, ids=ids, best=best, lse=lse, batch=batch)


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=500)
    ap.add_argument("--heads", type=int, default=2)
    ap.add_argument("--dim", type=int, default=32)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    _, model, _ = train(a.steps, a.batch, a.heads, a.dim, seed=a.seed, report=20)
    model.opt.close()
    return 0


if __name__ == "__main__":
    sys.exit(main())
