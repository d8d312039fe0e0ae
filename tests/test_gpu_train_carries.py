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


def test_recurrence_in_several_launches(T):      # noqa: F811
    """More than 2^30 rows of one channel: both passes take two launches.  Values around the rows where one ends, zeros between them (gates of a half: nothing
    gets through); both parts equal the oracle's."""
    import torch
    rows = (1 << 30) + 5000
    g = torch.Generator("cuda").manual_seed(22)
    rowptr = torch.tensor([0, 3000, (1 << 30) + 1000, rows], device="cuda")
    u, x, dh = (torch.zeros((rows, 1), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    near, far = slice(0, 12_000), slice((1 << 30) - 7000, rows)
    for part in (near, far):
        n = part.stop - part.start
        u[part] = (torch.randn((n, 1), generator=g, device="cuda") - 8).bfloat16()
        x[part], dh[part] = (torch.randn((n, 1), generator=g, device="cuda").bfloat16() for _ in range(2))
    h0, dlast = torch.randn((3, 1), generator=g, device="cuda"), torch.randn((3, 1), generator=g, device="cuda")
    for newest_first in (False, True):
        r = T.recur_run(rowptr, u, x, h0=h0, newest_first=newest_first, save=True)
        got = dict(r, **T.recur_grad(rowptr, u, x, r["saved"], h0=h0, newest_first=newest_first, dh=dh, dlast=dlast))
        for part, lens, there in ((near, [3000, 9000], [0, 1]), (far, [8000, 4000], [1, 2])):
            starts, ends = h0[there].cpu().numpy(), dlast[there].cpu().numpy()
            cut = there.index(1)                                     # the long list: its other end lies beyond the zeros
            (starts if (part is far) != newest_first else ends)[cut] = 0
            of = lambda v: v[part].float().cpu().numpy()             # noqa: E731
            want = O.recurrence_scanned(np.concatenate([[0], np.cumsum(lens)]), of(u), of(x), h0=starts, newest_first=newest_first, dh=of(dh), dlast=ends)
            for k in ("h", "du", "dx"):
                close(k, got[k][part], want[k], want[k + "_off"], BF16)
            whole = 1 - cut
            for k in ("last", "dh0"):
                close(k, got[k][there[whole]], want[k][whole], want[k + "_off"][whole])
        between = slice(near.stop + 1000, far.start - 1000)
        assert not got["dx"][between].any() and not got["h"][between].any()
