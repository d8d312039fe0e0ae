"""Carries of the recurrence over many tiles and spans, with states that live for thousands of rows, against the oracle's scans in 64 bits (whose
sensitivity to a lost or repeated carry test_train_oracle.py shows): joins with one span a thread and with many, open and closed spans side by
side, tiles of 32 and of 64 rows, both orders of time, rows written past the caches."""
import numpy as np
import pytest

from oracle import train_oracle as O
from test_gpu_train import BF16, F32, close, T  # noqa: F401

pytestmark = pytest.mark.gpu

CUT = [19_000, 300, 1, 5, 700, 256, 14_000, 10, 5000, 512, 2, 511, 7000, 64, 32, 33, 3]


def mixed(rows):
    """Lists of CUT's lengths, over and over, with short ones between them."""
    lens, left = [], rows
    for i in range(1 << 20):
        for n in (CUT[i % len(CUT)], 1 + i % 7):
            lens.append(min(n, left))
            left -= lens[-1]
            if not left:
                return lens


@pytest.mark.parametrize("newest_first", [False, True])
@pytest.mark.parametrize("kind", ["one list", "many lists"], ids=["one", "many"])
@pytest.mark.parametrize("dtype, dim, rows", [(F32, 3, 50_000), (F32, 3, 70_001), (BF16, 66, 33_000), (BF16, 2, 60_000),      # tiles of 32 rows, two spans a thread or three
                                              (F32, 2, 600_000), (BF16, 130, 150_000),                                    # tiles of 64 rows: ten spans a thread, three
                                              (F32, 128, 300_000), (BF16, 128, 640_000)])                                 # and rows written past the caches
def test_recurrence_carries(T, dtype, dim, rows, kind, newest_first):      # noqa: F811
    import torch
    dt = torch.float32 if dtype == F32 else torch.bfloat16
    g = torch.Generator("cuda").manual_seed(rows + dim)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
    lens = [rows] if kind == "one list" else mixed(rows)
    S = len(lens)
    rowptr = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)])).cuda()
    u, x, dh = (randn(rows, dim) - 8).to(dt), randn(rows, dim).to(dt), randn(rows, dim).to(dt)
    time = torch.cumsum(2 * torch.rand(rows, generator=g, device="cuda", dtype=torch.float64), 0)
    ts = (time.flip(0) if newest_first else time).float()
    decay, h0, t0, dlast = 2e-4 * torch.rand(dim, generator=g, device="cuda"), randn(S, dim), torch.zeros(S, device="cuda"), randn(S, dim)
    t0[:] = ts[rowptr[1:] - 1 if newest_first else rowptr[:-1]] - 1
    lists = dict(ts=ts, decay=decay, h0=h0, t0=t0, newest_first=newest_first)
    r = T.recur_run(rowptr, u, x, save=True, **lists)
    got = dict(r, **T.recur_grad(rowptr, u, x, r["saved"], dh=dh, dlast=dlast, **lists))
    some = sorted({0, dim // 2, dim - 1})                            # channels have nothing to do with each other
    of = lambda v: v[:, some].float().cpu().numpy()                  # noqa: E731
    want = O.recurrence_scanned(rowptr.cpu().numpy(), of(u), of(x), ts.cpu().numpy(), decay.cpu().numpy()[some], of(h0), t0.cpu().numpy(), newest_first, of(dh), of(dlast))
    for k in ("h", "last", "du", "dx", "dh0"):
        close(k, got[k][:, some], want[k], want[k + "_off"], dtype if k in ("h", "du", "dx") else F32)
    close("ddecay", got["ddecay"][some], want["ddecay"], want["ddecay_off"])
