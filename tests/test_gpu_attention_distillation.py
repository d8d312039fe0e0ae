"""The example that runs sampler, cache, attention, block, distillation and optimizer together: it runs, and its gradients are those of its loss."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain_loss(w, c, model, temperature):
    """The loss of a step from elementary operations in 64 bits."""
    import torch
    own, events, items = (c[n].double() for n in ("own", "events", "items"))
    rowptr, lists = c["rowptr"].tolist(), c["lists"]
    heads = (-1, model.heads, model.dim)
    q, k, v = (own @ w["query"]).view(heads), (events @ w["key"]).view(heads), (events @ w["value"]).view(heads)
    outs = []
    for s in range(len(rowptr) - 1):
        lo, hi = rowptr[s], rowptr[s + 1]
        bucket = torch.searchsorted(lists["edges"], (lists["t"][s] - lists["ts"][lo:hi]).clamp(min=0), right=True)
        score = (q[s][None] * k[lo:hi]).sum(-1) * model.dim ** -0.5 + w["table"][bucket]
        outs.append((torch.softmax(score, 0)[:, :, None] * v[lo:hi]).sum(0))
    norm = lambda x: x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-6)      # noqa: E731
    out = own @ w["own"] + w["scale"] * torch.sigmoid(own @ w["gate"]) * w["post"] * norm(torch.stack(outs).flatten(1))
    scores = (w["pre"] * norm(out)) @ (items @ w["item"]).t()
    logq, ids = torch.log_softmax(scores / temperature, 1), c["ids"].long()
    logp = c["best"].double() / temperature - c["lse"].double()[:, None]
    p = torch.exp(logp)
    rest = 1 - p.sum(1)
    others = torch.logsumexp(logq.scatter(1, ids, float("-inf")), 1)
    return ((p * (logp - logq.gather(1, ids))).sum(1) + rest * (torch.log(rest) - others)).sum() / c["batch"], scores


def test_the_example_runs_and_its_gradients_are_its_loss_s():
    import attention_distillation as E
    import torch
    losses, model, c = E.train(steps=3, batch=60, users=200, items=150, seed=2)
    assert len(losses) == 3 and all(0 < x < 100 for x in losses)
    # the last step's weights have been stepped: its gradients once more, with the weights as they are
    w = {n: v.double().requires_grad_() for n, v in model.w.items()}
    scores, kept = model.forward(c["own"], c["rowptr"], c["events"], c["lists"]["t"], c["lists"]["ts"], c["items"])
    out = E.L.distill(scores, c["ids"], c["best"], lse=c["lse"], temperature=E.TEMPERATURE, scale=1.0 / c["batch"])
    model.backward(out["dlogits"], kept)
    want, exact = plain_loss(w, c, model, E.TEMPERATURE)
    want.backward()
    # chains of some ten sums of up to a few hundred products each: a thousand roundings of the largest value
    off = 1000 * 2.0 ** -24
    assert float((scores.double() - exact).abs().max()) < off * float(exact.abs().max())
    assert abs(float(out["loss"]) - float(want)) < off * (1 + float(want))
    for n, g in model.g.items():
        assert float((g.double() - w[n].grad).abs().max()) < off * float(w[n].grad.abs().max()) + 1e-9, n
    model.opt.close()
