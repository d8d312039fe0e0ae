#!/usr/bin/env python3
"""Trains a small temporal link model on what the sampler returns, on one GPU.

A synthetic stream of (user, item, time) events in which users keep to the items of their kind.  For every event of a batch the
model embeds the user, the item and a few other items at the event's time and is trained to score the true pair higher:

  tns_run            the newest events of each root before its time (padding removed)
  tns_cache_fetch    the feature rows of the neighbours
  two products       gate and candidate of every event (torch)
  tns_recur_run      one state per root over its events, oldest to newest, faded by the time between them
  tns_pair_loss      loss and gradients of the embeddings
  tns_recur_grad     gradients of gates, candidates and decay; two products give the weights' gradients
  tns_adamw_step     one step over all weights, states in 8 or 32 bits

    python examples/link_training.py [--steps 200] [--bits 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2311_17410_amd import binding as B  # noqa: E402
from paper_2311_17410_amd import cache_binding as KB  # noqa: E402
from paper_2311_17410_amd import train_binding as T  # noqa: E402


def stream(users, items, kinds, events, seed):
    """Events in time order; nine of ten go to an item of the user's kind (kind = id modulo kinds)."""
    rng = np.random.default_rng(seed)
    user = rng.integers(0, users, events)
    item = rng.integers(0, items // kinds, events) * kinds + np.where(rng.random(events) < 0.9, user % kinds, rng.integers(0, kinds, events))
    return user.astype(np.int32), (users + item).astype(np.int32), np.sort(rng.random(events).astype(np.float32)) * 100


class Model:
    """Weights, their gradients and the optimizer that steps them."""

    def __init__(self, feat, dim, bits, seed, device):
        g = torch.Generator(device).manual_seed(seed)
        shapes = dict(gate=(feat, dim), gate_bias=(dim,), value=(feat, dim), value_bias=(dim,), own=(feat, dim), decay=(dim,))
        self.w = {n: torch.randn(s, generator=g, device=device) / feat ** 0.5 if len(s) == 2 else torch.zeros(s, device=device) for n, s in shapes.items()}
        self.w["decay"].fill_(0.05)
        self.g = {n: torch.zeros_like(v) for n, v in self.w.items()}
        self.opt = T.AdamW(list(self.w.values()), list(self.g.values()), bits=bits, weight_decay=[0.01 if len(s) == 2 else 0.0 for s in shapes.values()], seed=seed)
        self.t = 0

    def step(self, lr):
        norm = torch.cat([g.reshape(-1) for g in self.g.values()]).norm()
        self.t += 1
        self.opt.step(lr, self.t, (1.0 / norm.clamp(min=1.0)).reshape(1))      # gradients clipped to a norm of 1
        self.w["decay"].clamp_(min=0.0)


def train(steps=200, batch=600, links=4, dim=64, feat=32, bits=8, lr=1e-2, seed=0, users=2000, items=1000, kinds=8, report=None):
    """Returns the losses and the shares of pairs in the right order, step by step."""
    dev = torch.device("cuda", 0)
    nodes = users + items
    warm = 20_000                                                # events before the first batch
    user, item, time = stream(users, items, kinds, warm + steps * batch, seed)
    plan = B.Plan(nodes, 10, B.TNS_POLICY_RECENT, flags=B.TNS_FLAG_DEVICE_INGEST)
    d_user, d_item, d_time = (torch.from_numpy(v).to(dev) for v in (user, item, time))

    def ingest(lo, hi):                                          # an event is an edge of both its nodes
        a, b, t = d_user[lo:hi], d_item[lo:hi], d_time[lo:hi]
        plan.add_edges_device(torch.cat((a, b)), torch.cat((b, a)), torch.cat((t, t)))

    gen = torch.Generator(dev).manual_seed(seed)
    features = torch.randn((nodes, feat), generator=gen, device=dev)
    kind = torch.arange(nodes, device=dev) % kinds
    kind[users:] = (torch.arange(items, device=dev)) % kinds
    features[:, :kinds] += torch.nn.functional.one_hot(kind, kinds).float()      # a weak hint of the kind
    cache = KB.Cache(nodes, max(nodes // 5, 1), feat)
    model, losses, right = Model(feat, dim, bits, seed, dev), [], []
    w, g = model.w, model.g
    ingest(0, warm)
    for s in range(steps):
        lo, hi = warm + s * batch, warm + (s + 1) * batch
        others = users + torch.randint(0, items, (batch * links,), generator=gen, device=dev, dtype=torch.int32)
        roots = torch.cat((d_user[lo:hi], d_item[lo:hi], others))
        at = torch.cat((d_time[lo:hi], d_time[lo:hi], d_time[lo:hi].repeat_interleave(links)))
        got = plan.run(roots, None, at)
        rows = int(got["rowptr"][-1])                            # how many neighbours there are in all
        nbr, ts = got["cmp_nbr"][:rows], got["cmp_ts"][:rows]
        feats, _ = cache.fetch(nbr, features)
        lists = dict(ts=ts, decay=w["decay"], newest_first=True)
        u, x = feats @ w["gate"] + w["gate_bias"], feats @ w["value"] + w["value_bias"]
        r = T.recur_run(got["rowptr"], u, x, states=False, save=True, **lists)
        emb = r["last"] + features[roots.long()] @ w["own"]
        # a negative that is the true item is masked
        weight = (others.view(batch, links) != d_item[lo:hi, None]).float()
        out = T.pair_loss(emb[:batch], emb[batch:2 * batch], emb[2 * batch:].view(batch, links, dim), weight=weight, beta=dim ** -0.5, scale=1.0 / (batch * links))
        demb = torch.cat((out["danchor"], out["dpos"], out["dneg"].view(-1, dim)))
        d = T.recur_grad(got["rowptr"], u, x, r["saved"], dlast=demb, **lists)
        torch.matmul(feats.t(), d["du"], out=g["gate"])
        torch.matmul(feats.t(), d["dx"], out=g["value"])
        torch.matmul(features[roots.long()].t(), demb, out=g["own"])
        torch.sum(d["du"], 0, out=g["gate_bias"])
        torch.sum(d["dx"], 0, out=g["value_bias"])
        g["decay"].copy_(d["ddecay"])
        model.step(lr)
        ingest(lo, hi)
        losses.append(out["loss"])
        right.append((out["margin"] > 0).float().mean())
        if report and (s + 1) % report == 0:
            print(f"step {s + 1:5d}  loss {float(torch.stack(losses[-report:]).mean()):.4f}  in order {float(torch.stack(right[-report:]).mean()):.3f}", flush=True)
    losses, right = torch.stack(losses).tolist(), torch.stack(right).tolist()
    model.opt.close()
    cache.close()
    plan.close()
    return losses, right


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=600)
    ap.add_argument("--links", type=int, default=4)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--bits", type=int, default=8, choices=[8, 32])
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    train(a.steps, a.batch, a.links, a.dim, bits=a.bits, seed=a.seed, report=20)
    return 0


if __name__ == "__main__":
    sys.exit(main())
