"""The training operators on the GPU against the oracle in 64 bits.  Tolerances are the oracle's running error bounds
(a result in bf16 lies between the roundings of the bound's two ends); states of the optimizer are compared bit for bit."""
import numpy as np
import pytest

from oracle import train_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = "f32", "bf16"


@pytest.fixture(scope="module")
def T():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2311_17410_amd import train_binding
    train_binding.lib()
    return train_binding


def torch_of(a, dtype=None):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda().to({None: None, F32: torch.float32, BF16: torch.bfloat16}[dtype] if dtype else torch.from_numpy(np.ascontiguousarray(a)).dtype)


def values(rng, shape, dtype, scale=1.0):
    """Normal values that the type holds exactly."""
    import torch
    v = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32))
    return (v.bfloat16().float() if dtype == BF16 else v).numpy()


def close(what, got, want, off, dtype=F32):
    """Every value within its bound; one in bf16 between the roundings of the bound's two ends."""
    import torch
    got = got.float().cpu().numpy().astype(np.float64) if hasattr(got, "cpu") else got
    low, high = want - off, want + off
    if dtype == BF16:
        low, high = (torch.from_numpy(np.asarray(v, np.float32)).bfloat16().double().numpy() for v in (low, high))
    bad = ~((got >= low - 1e-37) & (got <= high + 1e-37))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, first at {np.argwhere(bad)[0].tolist()}: {got[bad][0]!r} for {want[bad][0]!r}, bound {off[bad][0]:.3g}"


def the_lists(rng, lens, dim, dtype, decay, start):
    rp = np.concatenate([[0], np.cumsum(np.asarray(lens, np.int64))]).astype(np.int64)
    n, S = int(rp[-1]), len(lens)
    a = dict(rowptr=rp, u=values(rng, (n, dim), dtype, 1.5), x=values(rng, (n, dim), dtype), ts=None, decay=None, h0=None, t0=None)
    if decay:
        a.update(ts=rng.uniform(0, 2, n).astype(np.float32), decay=rng.uniform(0, 1, dim).astype(np.float32))
    if start:
        a.update(h0=values(rng, (S, dim), F32), t0=rng.uniform(0, 1, S).astype(np.float32) if decay else None)
    return a


def on_gpu(a, dtype):
    return {k: torch_of(v, dtype if k in ("u", "x") else None) for k, v in a.items()}


RAGGED = [3, 0, 10, 1, 0, 0, 7, 10, 10, 2] * 13
LISTS = {
    "no list": [], "none": [0], "one": [1], "empty ones": [0, 0, 0], "mixed": [1, 0, 3, 0, 0], "ragged": RAGGED, "wave": [64], "wave and one": [65],
    "around a wave": [63, 1, 64, 2, 127, 129], "holes": [5] + [0] * 300 + [70] + [0] * 64 + [1], "ones": [1] * 200, "long": [1000], "long and short": [5, 3000, 0, 2, 700],
    "sixteens": [16, 16, 32, 15, 17, 48], "very long": [9000, 1, 0, 4097],
}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("decay, start, newest_first", [(True, True, True), (True, False, False), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("lens", list(LISTS), ids=[k.replace(" ", "_") for k in LISTS])
def test_recurrence(T, lens, decay, start, newest_first, dtype):
    rng = np.random.default_rng(len(LISTS[lens]) + 7)
    dim = {"very long": 5, "long": 70, "long and short": 130, "ragged": 100}.get(lens, 33)
    a = the_lists(rng, LISTS[lens], dim, dtype, decay, start)
    n, S = a["u"].shape[0], len(LISTS[lens])
    dh, dlast = values(rng, (n, dim), dtype), values(rng, (S, dim), F32)
    want = O.recurrence(**a, newest_first=newest_first, dh=dh, dlast=dlast)
    g = on_gpu(a, dtype)
    r = T.recur_run(**g, newest_first=newest_first, save=True)
    close("h", r["h"], want["h"], want["h_off"], dtype)
    close("last", r["last"], want["last"], want["last_off"])
    got = T.recur_grad(**g, saved=r["saved"], newest_first=newest_first, dh=torch_of(dh, dtype), dlast=torch_of(dlast))
    for name in ("du", "dx"):
        close(name, got[name], want[name], want[name + "_off"], dtype)
    if start:
        close("dh0", got["dh0"], want["dh0"], want["dh0_off"])
    if decay:
        close("ddecay", got["ddecay"], want["ddecay"], want["ddecay_off"])
    assert (got["dh0"] is None) == (not start) and (got["ddecay"] is None) == (not decay)
    only = T.recur_run(**g, newest_first=newest_first, states=False)
    assert only["h"] is None and only["saved"] is None and bool((only["last"] == r["last"]).all())      # the same bits without the other outputs


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [1, 2, 3, 31, 64, 65, 128, 129, 172, 173, 256, 300, 1030])
def test_recurrence_channels(T, dim, dtype):
    rng = np.random.default_rng(dim)
    a = the_lists(rng, [4, 0, 30, 1, 9], dim, dtype, True, True)
    dh = values(rng, a["u"].shape, dtype)
    want = O.recurrence(**a, dh=dh)
    g = on_gpu(a, dtype)
    r = T.recur_run(**g, save=True)
    got = T.recur_grad(**g, saved=r["saved"], dh=torch_of(dh, dtype))
    close("h", r["h"], want["h"], want["h_off"], dtype)
    close("last", r["last"], want["last"], want["last_off"])
    for name in ("du", "dx"):
        close(name, got[name], want[name], want[name + "_off"], dtype)
    for name in ("ddecay", "dh0"):
        close(name, got[name], want[name], want[name + "_off"])


@pytest.mark.parametrize("newest_first", [False, True])
@pytest.mark.parametrize("dtype, dim, ld, skip", [(BF16, 32, 70, 1), (BF16, 32, 71, 0), (F32, 40, 43, 1), (BF16, 64, 64, 3), (BF16, 128, 130, 0)])
def test_recurrence_strides_and_rows_beyond_the_lists(T, dtype, dim, ld, skip, newest_first):
    """Rows that lie apart, at odd addresses; rows after the last list are not read (NaN) and not written."""
    import torch
    rng = np.random.default_rng(5)
    a = the_lists(rng, RAGGED, dim, dtype, True, False)
    n, more = a["u"].shape[0], 37
    dlast = values(rng, (len(RAGGED), dim), F32)
    want = O.recurrence(**a, newest_first=newest_first, dlast=dlast)
    g = on_gpu(a, dtype)
    for k in ("u", "x"):
        wide = torch.full(((n + more) * ld + skip,), float("nan"), dtype=g[k].dtype, device="cuda")
        view = wide[skip:].view(n + more, ld)[:, :dim] if ld * (n + more) + skip == wide.numel() else None
        view[:n] = g[k]
        g[k] = view
    g["ts"] = torch.cat((g["ts"], torch.full((more,), float("nan"), device="cuda")))
    r = T.recur_run(**g, newest_first=newest_first, save=True)
    close("h", r["h"][:n], want["h"], want["h_off"], dtype)
    close("last", r["last"], want["last"], want["last_off"])
    # outputs through the C interface, with strides and guards of their own
    desc = T._lists(g["rowptr"], g["u"], g["x"], g["ts"], g["decay"], None, None, newest_first)
    out = {k: torch.full(((n + more) * ld + skip,), 7.0, dtype=g["u"].dtype, device="cuda") for k in ("du", "dx", "h")}
    size = g["u"].element_size()
    _, ws, _ = T.tns_recur_workspace(desc)
    work, dd = torch.empty(ws, dtype=torch.uint8, device="cuda"), torch.empty(dim, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    T.tns_recur_grad(desc, r["saved"].data_ptr(), 0, dim, torch_of(dlast).data_ptr(), out["du"].data_ptr() + skip * size, ld, out["dx"].data_ptr() + skip * size, ld,
                     dd.data_ptr(), 0, work.data_ptr(), ws, stream)
    run_ws = torch.empty(T.tns_recur_workspace(desc)[0], dtype=torch.uint8, device="cuda")
    T.tns_recur_run(desc, out["h"].data_ptr() + skip * size, ld, 0, 0, run_ws.data_ptr(), run_ws.numel(), stream)
    for k, v in out.items():
        rows = v[skip:].view(n + more, ld)
        close(k, rows[:n, :dim], want[k], want[k + "_off"], dtype)
        assert bool((v[:skip] == 7).all()) and bool((rows[:, dim:] == 7).all()) and bool((rows[n:] == 7).all()), k
    close("ddecay", dd, want["ddecay"], want["ddecay_off"])


def test_recurrence_extreme_gates_and_times(T):
    """Gates from -200 to 200, times that are infinite, equal, falling; a NaN of one list stays in it."""
    rng = np.random.default_rng(6)
    a = the_lists(rng, [50, 40, 30], 20, F32, True, True)
    a["u"][:50] = rng.choice([-200.0, -88.5, -30, 0, 30, 88.5, 200], (50, 20)).astype(np.float32)
    a["ts"][:50] = rng.choice([-np.inf, 0, 1, 1e30, np.inf], 50).astype(np.float32)
    a["decay"][::2] = 0.0
    dh = values(rng, a["u"].shape, F32)
    want = O.recurrence(**a, dh=dh)
    g = on_gpu(a, F32)
    r = T.recur_run(**g, save=True)
    got = T.recur_grad(**g, saved=r["saved"], dh=torch_of(dh))
    close("h", r["h"], want["h"], want["h_off"])
    close("du", got["du"], want["du"], want["du_off"])
    close("dx", got["dx"], want["dx"], want["dx_off"])
    g["x"][60, 3] = float("nan")
    h = T.recur_run(**g)["h"].cpu().numpy()
    nan = np.isnan(h)
    assert nan[60:90, 3].all() and nan.sum() == 30
    g["x"][60, 3] = 0.0
    g["u"][60, 3] = float("nan")
    assert np.array_equal(np.isnan(T.recur_run(**g)["h"].cpu().numpy()), nan)


def test_recurrence_gradients_against_differences(T):
    """Slope along a direction: the gradients' product with it, and a central difference of the oracle."""
    rng = np.random.default_rng(8)
    a = the_lists(rng, [30, 0, 200, 7], 6, F32, True, True)
    dh, dlast = values(rng, a["u"].shape, F32), values(rng, (4, 6), F32)
    g = on_gpu(a, F32)
    r = T.recur_run(**g, save=True)
    got = T.recur_grad(**g, saved=r["saved"], dh=torch_of(dh), dlast=torch_of(dlast))
    for name in ("u", "x", "decay", "h0"):
        way = rng.standard_normal(a[name].shape)
        ends = []
        for by in (1e-5, -1e-5):
            o = O.recurrence(**dict(a, **{name: a[name].astype(np.float64) + by * way}))
            ends.append((o["h"] * dh).sum() + (o["last"] * dlast).sum())
        slope = (ends[0] - ends[1]) / 2e-5
        mine = (got["d" + name].cpu().numpy().astype(np.float64) * way)
        # a difference is off by its second order (1e-10 of the third derivative) and by the sums' rounding over 1e-5
        assert abs(mine.sum() - slope) < 1e-5 * np.abs(mine).sum() + 1e-6, name


def test_recurrence_same_bits_again_on_another_stream_and_in_a_graph(T):
    import torch
    rng = np.random.default_rng(9)
    lens = [5000, 3, 0, 800] + RAGGED
    a = the_lists(rng, lens, 100, BF16, True, True)
    g = on_gpu(a, BF16)
    dlast = torch_of(values(rng, (len(lens), 100), F32))

    def both():
        r = T.recur_run(**g, save=True)
        return {**{k: r[k] for k in ("h", "last")}, **T.recur_grad(**g, saved=r["saved"], dlast=dlast)}

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both()
    torch.cuda.current_stream().wait_stream(side)
    for k in first:
        assert torch.equal(first[k], again[k]), k
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = both()
    for _ in range(3):
        for v in kept.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k in first:
            assert torch.equal(first[k], kept[k]), k
        both()


def test_recurrence_offsets_beyond_32_bits(T):
    """rows * dim passes 2^32: the lists at the end equal the same lists alone."""
    import torch
    dim, n = 256, (1 << 24) + 5000
    tail = [4000, 0, 300, 7, 1]
    rng = np.random.default_rng(10)
    a = the_lists(rng, tail, dim, BF16, False, False)
    rows = n + sum(tail)
    g = on_gpu(a, BF16)
    u, x = (torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    u[n:], x[n:] = g["u"], g["x"]
    rowptr = torch.cat((torch.tensor([0, 10, n // 2]), n + torch.from_numpy(a["rowptr"]))).cuda()
    dlast = torch.zeros((len(tail) + 3, dim), device="cuda")
    dlast[3:] = torch_of(values(rng, (len(tail), dim), F32))
    want = O.recurrence(**a, dlast=dlast[3:].cpu().numpy())
    r = T.recur_run(rowptr, u, x, save=True)
    got = T.recur_grad(rowptr, u, x, saved=r["saved"], dlast=dlast)
    close("h", r["h"][n:], want["h"], want["h_off"], BF16)
    close("last", r["last"][3:], want["last"], want["last_off"])
    for name in ("du", "dx"):
        close(name, got[name][n:], want[name], want[name + "_off"], BF16)
        assert not got[name][:n].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch, dim, decay", [(1, 1, True), (1, 1030, True), (3, 64, False), (65, 100, True), (200, 172, True), (200, 173, False), (33, 128, True), (7, 300, True), (0, 16, True)])
def test_step(T, batch, dim, decay, dtype):
    rng = np.random.default_rng(batch + dim)
    nodes = 300
    ids = rng.permutation(nodes)[:batch].astype(np.int32)
    ids[4::9] = [-1, nodes, 1 << 30, -(1 << 31)][batch % 4]
    u, x, state = values(rng, (batch, dim), dtype, 2.0), values(rng, (batch, dim), dtype), values(rng, (nodes, dim), F32)
    ts, lam, sts = (rng.uniform(0, 2, batch).astype(np.float32), rng.uniform(0, 1, dim).astype(np.float32), rng.uniform(0, 2, nodes).astype(np.float32)) if decay else (None,) * 3
    out, off, after, after_off, after_ts = O.step(ids, u, x, state, ts, lam, sts)
    g_state, g_sts = torch_of(state), torch_of(sts)
    got = T.recur_step(torch_of(ids), torch_of(u, dtype), torch_of(x, dtype), g_state, torch_of(ts), torch_of(lam), g_sts)
    close("out", got, out, off, dtype)
    close("state", g_state, after, after_off)
    untouched = after_off.max(1) == 0
    assert np.array_equal(g_state.cpu().numpy()[untouched], state[untouched])
    if decay:
        assert np.array_equal(g_sts.cpu().numpy(), after_ts)


def test_step_equals_the_recurrence_event_by_event(T):
    """Fifty events of twenty nodes one at a time, and the twenty lists at once."""
    import torch
    rng = np.random.default_rng(11)
    a = the_lists(rng, [50] * 20, 96, F32, True, True)
    g = on_gpu(a, F32)
    last = T.recur_run(**g)["last"]
    state, state_ts, ids = g["h0"].clone(), g["t0"].clone(), torch.arange(20, dtype=torch.int32, device="cuda")
    for i in range(50):
        at = torch.arange(20, device="cuda") * 50 + i
        T.recur_step(ids, g["u"][at], g["x"][at], state, g["ts"][at], g["decay"], state_ts)
    want = O.recurrence(**a)
    close("state", state, want["last"], want["last_off"])
    close("last", last, want["last"], want["last_off"])


# ---- loss ------------------------------------------------------------------------------------------

PAIRS = [(1, 1, 1), (1, 0, 8), (0, 4, 8), (5, 1, 100), (3, 7, 128), (2, 300, 64), (1, 5000, 32), (600, 3, 172), (4, 9, 173), (3, 5, 260), (2, 70, 515), (2, 3, 1100),
         (1, 2, 2500), (40, 33, 20), (3, 4, 4)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("extras", [False, True], ids=["plain", "ref_weight_smoothing"])
@pytest.mark.parametrize("events, links, dim", PAIRS)
def test_pair_loss(T, events, links, dim, extras, dtype):
    rng = np.random.default_rng(events * 31 + links + dim)
    a, p, n = values(rng, (events, dim), dtype), values(rng, (events, dim), dtype), values(rng, (events, links, dim), dtype)
    kw = dict(beta=1.5 / np.sqrt(dim), scale=1.0 / max(events * links, 1))
    if extras:
        w = rng.choice([0.0, 0.0, 0.5, 1.0, 2.0], (events, links)).astype(np.float32)
        w[1::3] = 0.0                                  # events without a pair
        kw.update(ref=rng.standard_normal((events, links)).astype(np.float32), weight=w, smoothing=0.1)
        n[w == 0] = rng.choice([np.nan, np.inf, -np.inf, 3e38], (int((w == 0).sum()), 1))
        a[1::6], p[1::6], p[4::6] = np.nan, np.inf, np.nan
        kw["ref"][w == 0] = np.nan
    want = O.pair_loss(a, p, n, **kw)
    for k in ("ref", "weight"):
        kw[k] = torch_of(kw.get(k))
    got = T.pair_loss(torch_of(a, dtype), torch_of(p, dtype), torch_of(n, dtype), **kw)
    close("loss", got["loss"], np.float64(want["loss"]), want["loss_off"])
    close("margin", got["margin"], want["margin"], want["margin_off"])
    for k in ("danchor", "dpos", "dneg"):
        close(k, got[k], want[k], want[k + "_off"], dtype)
    only = T.pair_loss(torch_of(a, dtype), torch_of(p, dtype), torch_of(n, dtype), grads=False, **kw)
    assert only["dneg"] is None and bool((only["margin"] == got["margin"]).all()) and bool(only["loss"] == got["loss"])


@pytest.mark.parametrize("dtype, dim, ld, skip", [(F32, 100, 103, 1), (BF16, 100, 104, 2), (BF16, 100, 101, 1), (F32, 64, 68, 0), (F32, 6, 6, 2)])
def test_pair_loss_strides_and_addresses(T, dtype, dim, ld, skip):
    import torch
    rng = np.random.default_rng(dim + ld)
    a, p, n = values(rng, (9, dim), dtype), values(rng, (9, dim), dtype), values(rng, (9, 6, dim), dtype)
    want = O.pair_loss(a, p, n)

    def apart(v, ld):
        t = torch_of(v, dtype).reshape(-1, dim)
        wide = torch.full((t.shape[0] * ld + skip,), float("nan"), dtype=t.dtype, device="cuda")
        rows = wide[skip:].view(t.shape[0], ld)[:, :dim]
        rows.copy_(t)
        return rows

    got = T.pair_loss(apart(a, ld), apart(p, ld), apart(n, dim).view(9, 6, dim))
    for k in ("danchor", "dpos", "dneg"):
        close(k, got[k], want[k], want[k + "_off"], dtype)
    close("loss", got["loss"], np.float64(want["loss"]), want["loss_off"])


def test_pair_loss_far_margins_and_nan(T):
    """Margins of thousands: slopes of 0 and 1, loss linear; what is not a number and not masked reaches its own event alone."""
    rng = np.random.default_rng(12)
    a, p, n = values(rng, (6, 32), F32, 30.0), values(rng, (6, 32), F32, 30.0), values(rng, (6, 4, 32), F32, 30.0)
    want = O.pair_loss(a, p, n)
    got = T.pair_loss(torch_of(a), torch_of(p), torch_of(n))
    assert np.abs(want["margin"]).max() > 1000
    for k in ("loss", "danchor", "dpos", "dneg"):
        close(k, got[k], np.float64(want[k]), want[k + "_off"])
    n[2, 1, 5] = np.nan
    got = T.pair_loss(torch_of(a), torch_of(p), torch_of(n))
    assert np.isnan(float(got["loss"]))
    margin = np.isnan(got["margin"].cpu().numpy())
    assert margin[2, 1] and margin.sum() == 1
    assert np.array_equal(np.isnan(got["danchor"].cpu().numpy()).any(1), np.arange(6) == 2)


def test_pair_loss_gradients_against_differences(T):
    rng = np.random.default_rng(13)
    v = [values(rng, s, F32) for s in ((7, 40), (7, 40), (7, 5, 40))]
    got = T.pair_loss(*[torch_of(t) for t in v], beta=0.3, smoothing=0.05)
    for i, k in enumerate(("danchor", "dpos", "dneg")):
        way = rng.standard_normal(v[i].shape)
        ends = [O.pair_loss(*[t + by * way if j == i else t for j, t in enumerate(v)], beta=0.3, smoothing=0.05)["loss"] for by in (1e-5, -1e-5)]
        mine = got[k].cpu().numpy().astype(np.float64) * way
        assert abs(mine.sum() - (ends[0] - ends[1]) / 2e-5) < 1e-5 * np.abs(mine).sum() + 1e-6, k


def test_pair_loss_same_bits_again_and_in_a_graph(T):
    import torch
    rng = np.random.default_rng(14)
    v = [torch_of(values(rng, s, BF16), BF16) for s in ((3, 128), (3, 128), (3, 4001, 128))]
    first = T.pair_loss(*v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = T.pair_loss(*v)
    for _ in range(3):
        for t in kept.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        again = T.pair_loss(*v)
        for k in first:
            assert torch.equal(first[k], kept[k]) and torch.equal(first[k], again[k]), k


def test_pair_loss_offsets_beyond_32_bits(T):
    """events * links * dim passes 2^32: the last event equals itself alone."""
    import torch
    rng = np.random.default_rng(15)
    dim, links = 128, 1 << 16
    a, p, n = values(rng, (1, dim), BF16), values(rng, (1, dim), BF16), values(rng, (1, links, dim), BF16, 0.5)
    alone = T.pair_loss(torch_of(a, BF16), torch_of(p, BF16), torch_of(n, BF16))
    events = 520
    wide = torch.zeros((events, links, dim), dtype=torch.bfloat16, device="cuda")
    wide[-1] = torch_of(n, BF16)[0]
    big = [torch.zeros((events, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    big[0][-1], big[1][-1] = torch_of(a, BF16)[0], torch_of(p, BF16)[0]
    got = T.pair_loss(*big, wide)
    want = O.pair_loss(a, p, n)
    close("margin", got["margin"][-1:], want["margin"], want["margin_off"])
    for k in ("danchor", "dpos", "dneg"):
        close(k, got[k][-1:], want[k], want[k + "_off"], BF16)
        close(k, alone[k], want[k], want[k + "_off"], BF16)
    assert not got["dneg"][:-1].any() and not got["danchor"][:-1].any()


# ---- AdamW -----------------------------------------------------------------------------------------

SIZES = [1, 3, 4, 255, 256, 257, 1000, 4096, 4097, 0, 12345, 70001]


def the_weights(rng, sizes, bits, grad):
    made = []
    for n in sizes:
        w = dict(param=values(rng, n, F32, 0.1), grad=values(rng, n, grad, 0.02))
        if bits == 32:
            w["state"] = dict(m=values(rng, n, F32, 0.01), v=values(rng, n, F32, 0.02) ** 2)
        else:
            blocks = -(-n // 256)
            w["state"] = dict(m=rng.integers(0, 256, n).astype(np.uint8), v=rng.integers(0, 0x7F, n).astype(np.uint8),
                              m_scale=rng.uniform(0, 1e-4, blocks).astype(np.float32), v_scale=rng.uniform(0, 2e-4, blocks).astype(np.float32))
            w["state"]["m"][(w["state"]["m"] & 0x7F) == 0x7F] = 0
        made.append(w)
    return made


def optimizer(T, made, bits, grad, copies, skip=0, **kw):
    """AdamW over copies of the weights on the GPU; with `skip` every buffer begins that many elements after an aligned address."""
    import torch

    def place(v):
        t = torch_of(v)
        if not skip:
            return t
        wide = torch.zeros(t.numel() + skip, dtype=t.dtype, device="cuda")
        wide[skip:] = t
        return wide[skip:]

    states = [[place(w["state"][k]) for w in made] for k in made[0]["state"]]
    if bits == 8:
        states[:2] = [[t.view(torch.float8_e4m3fn) for t in part] for part in states[:2]]
    g = torch.bfloat16 if grad == BF16 else torch.float32
    return T.AdamW([place(w["param"]) for w in made], [place(w["grad"]).to(g) if not skip else place(w["grad"]) for w in made],
                   copies=[torch.zeros(len(w["param"]), dtype=torch.bfloat16, device="cuda") for w in made] if copies else None, bits=bits, states=states, **kw)


def check_adamw(opt, made, bits, t, decays, copies, **kw):
    first = 0
    for i, w in enumerate(made):
        new, off, state = O.adamw(w["param"], w["grad"], w["state"], t, first, weight_decay=decays[i], **kw)
        got = opt.params[i].cpu().numpy()
        close(f"param {i}", got.astype(np.float64), new, off)
        if copies:
            import torch
            assert torch.equal(opt.copies[i], opt.params[i].bfloat16()), i
        for k, v in state.items():
            mine = getattr(opt, k)[i]
            mine = (mine.view(__import__("torch").uint8) if bits == 8 and k in ("m", "v") else mine).cpu().numpy()
            assert np.array_equal(mine.view(np.uint8), v.view(np.uint8)), f"{k} of tensor {i}: {np.argwhere(mine != v)[:3].tolist()}"
        w.update(param=got, state=state)                # the next step goes on from what there is
        first += -(-len(w["param"]) // 256) * 256


@pytest.mark.parametrize("bits, grad, copies, skip", [(32, F32, False, 0), (32, BF16, True, 0), (8, F32, True, 0), (8, BF16, False, 0), (32, F32, False, 1), (8, F32, False, 3)])
def test_adamw_steps(T, bits, grad, copies, skip):
    rng = np.random.default_rng(bits + skip)
    made = the_weights(rng, SIZES, bits, grad)
    decays = [0.01 * (i % 3) for i in range(len(SIZES))]
    opt = optimizer(T, made, bits, grad, copies, skip, weight_decay=decays, seed=77)
    for t in (5, 6, 7):
        opt.step(2e-3, t, torch_of(np.float32([0.5])))
        check_adamw(opt, made, bits, t, decays, copies, lr=2e-3, seed=77, grad_scale=0.5)
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_zero_without_scale_and_left_out_steps(T, bits):
    import torch
    rng = np.random.default_rng(4)
    p, g = torch_of(values(rng, 1000, F32)), torch_of(values(rng, 1000, F32))
    g[300:700] = 0.0                                   # one block of 256 without a gradient, in part others
    opt = T.AdamW([p], [g], bits=bits, weight_decay=0.0)
    before = p.clone()
    for bad in (0.0, float("nan"), float("inf")):
        opt.step(1e-3, 1, torch_of(np.float32([bad])))
    assert torch.equal(p, before) and not opt.m[0].view(torch.uint8).any()
    opt.step(1e-3, 1)
    change = (p - before).cpu().numpy()
    sign = np.sign(g.cpu().numpy())
    # m / sqrt(v) = sign(g) after the first step; eps takes 1e-8 / |g| of it; p rounds to 2^-23 of its size
    assert (np.abs(change + 1e-3 * sign) < 1e-3 * (1e-8 / np.maximum(np.abs(g.cpu().numpy()), 1e-4) + 1e-6) + 2.0 ** -22 * np.abs(before.cpu().numpy())).all()
    if bits == 8:
        assert float(opt.m_scale[0][1]) != 0 and not opt.m[0].view(torch.uint8)[512:700].any()
    opt.close()


def test_adamw_not_finite(T):
    """In 32 bits an infinite gradient spoils its own weight, in 8 bits the state of its 256."""
    import torch
    rng = np.random.default_rng(5)
    for bits in (32, 8):
        p, g = torch_of(values(rng, 1024, F32)), torch_of(values(rng, 1024, F32))
        g[300] = float("inf")
        g[900] = float("nan")
        opt = T.AdamW([p], [g], bits=bits)
        opt.step(1e-3, 1)
        assert set(np.flatnonzero(~np.isfinite(p.cpu().numpy()))) == {300, 900}
        g[300] = g[900] = 0.1
        opt.step(1e-3, 2)
        bad = set(np.flatnonzero(~np.isfinite(p.cpu().numpy())))
        assert bad == ({300, 900} if bits == 32 else set(range(256, 512)) | set(range(768, 1024)))
        opt.close()


def test_adamw_many_tensors_and_a_graph(T):
    """Five hundred tensors in one launch; a captured step does the same again."""
    import torch
    rng = np.random.default_rng(6)
    made = the_weights(rng, list(rng.integers(1, 900, 500)), 8, F32)
    opt, twin = (optimizer(T, made, 8, F32, False, weight_decay=0.1, seed=3) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        twin.step(1e-3, 9)
    for _ in range(3):
        opt.step(1e-3, 9)
        graph.replay()
        torch.cuda.synchronize()
        for k in ("params", "m", "v", "m_scale", "v_scale"):
            for a, b in zip(getattr(opt, k), getattr(twin, k)):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), k
    opt.close()
    twin.close()


def test_adamw_eight_bits_follow_thirty_two(T):
    """A thousand steps towards a minimum: both get there, by about as much."""
    import torch
    gen = torch.Generator("cuda").manual_seed(0)
    goal = torch.randn(4096, device="cuda", generator=gen)
    left = {}
    for bits in (32, 8):
        p, g = torch.zeros(4096, device="cuda"), torch.zeros(4096, device="cuda")
        opt = T.AdamW([p], [g], bits=bits, weight_decay=0.0, seed=1)
        noise = torch.Generator("cuda").manual_seed(2)
        for t in range(1, 1001):
            g.copy_((p - goal) + 0.3 * torch.randn(4096, device="cuda", generator=noise))
            opt.step(1e-2 * (1 - t / 1001), t)
        left[bits] = float((p - goal).square().mean())
        opt.close()
    assert left[32] < 0.05 and left[8] < 2 * left[32] + 0.01, left


def test_refusals_of_tensors(T):
    import torch
    u = torch.zeros((4, 8), device="cuda")
    rp = torch.tensor([0, 4], device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: T.recur_run(rp.int(), u, u), lambda: T.recur_run(rp, u.half(), u.half()), lambda: T.recur_run(rp, u, u[:3]), lambda: T.recur_run(rp, u.t(), u.t()),
                 lambda: T.recur_run(rp, u, u, decay=torch.zeros(7, device="cuda"), ts=u[:, 0].contiguous()), lambda: T.recur_grad(rp, u, u, None),
                 lambda: T.recur_grad(rp, u, u, torch.zeros(4, dtype=torch.uint8, device="cuda")), lambda: T.recur_step(ids.long(), u, u, u),
                 lambda: T.recur_step(ids, u, u, u[:, :7]), lambda: T.pair_loss(u, u, u), lambda: T.pair_loss(u, u, torch.zeros((8, 2, 4), device="cuda").transpose(0, 2)),
                 lambda: T.AdamW([u], [u.half()]), lambda: T.AdamW([u], [u], bits=4), lambda: T.AdamW([u.t()], [u.t()]), lambda: T.AdamW([u], [u], weight_decay=[0.1, 0.2]),
                 lambda: T.AdamW([u], [u], copies=[u]), lambda: T.AdamW([], [])):
        with pytest.raises(ValueError):
            call()
    from paper_2311_17410_amd.binding import TnsError
    with pytest.raises(TnsError):
        T.recur_run(rp, u, u, ts=u[:, 0].contiguous())
    with pytest.raises(TnsError):
        T.recur_run(rp, u[:1].expand(4, 8), u)


def test_adamw_offsets_beyond_32_bits(T):
    """A tensor of more than 2^31 weights (2^33 bytes): its end equals the oracle's, the rest stays zero."""
    import torch
    n, tail = (1 << 31) + 1000, 4096 + 1000
    rng = np.random.default_rng(7)
    w = the_weights(rng, [tail], 8, BF16)[0]
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(-(-n // 256), device="cuda") for _ in range(2))
    scales = -(-tail // 256)
    p[-tail:], g[-tail:] = torch_of(w["param"]), torch_of(w["grad"], BF16)
    for to, k, size in ((m, "m", tail), (v, "v", tail), (ms, "m_scale", scales), (vs, "v_scale", scales)):
        to[-size:] = torch_of(w["state"][k])
    e4m3 = torch.float8_e4m3fn
    opt = T.AdamW([p], [g], bits=8, weight_decay=0.1, seed=3, states=([m.view(e4m3)], [v.view(e4m3)], [ms], [vs]))
    opt.step(1e-3, 4)
    new, off, state = O.adamw(w["param"], w["grad"], w["state"], 4, n - tail, weight_decay=0.1, seed=3)
    close("param", p[-tail:], new, off)
    for got, k, size in ((m, "m", tail), (v, "v", tail), (ms, "m_scale", scales), (vs, "v_scale", scales)):
        assert np.array_equal(got[-size:].cpu().numpy(), state[k]), k
    assert not p[:-tail].any() and not m[:-tail].any() and not v[:-tail].any()
    opt.close()


@pytest.mark.parametrize("dtype, dim", [(F32, 128), (BF16, 128)])
def test_recurrence_rows_written_past_the_caches(T, dtype, dim):
    """More rows than the last-level cache holds, of whole cache lines: the lists at the end equal the oracle's."""
    import torch
    n, tail = 600_000, [40, 0, 300, 7, 1]
    rng = np.random.default_rng(16)
    a = the_lists(rng, tail, dim, dtype, True, False)
    g = on_gpu(a, dtype)
    rows = n + sum(tail)
    u, x, dh = (torch.zeros((rows, dim), dtype=g["u"].dtype, device="cuda") for _ in range(3))
    assert 2 * u.numel() * u.element_size() > 1 << 28
    tail_dh = values(rng, (sum(tail), dim), dtype)
    u[n:], x[n:], dh[n:] = g["u"], g["x"], torch_of(tail_dh, dtype)
    ts = torch.cat((torch.zeros(n, device="cuda"), g["ts"]))
    rowptr = torch.cat((torch.arange(0, n, 100), n + torch.from_numpy(a["rowptr"]))).cuda()
    first = rowptr.shape[0] - 1 - len(tail)
    want = O.recurrence(**a, dh=tail_dh)
    r = T.recur_run(rowptr, u, x, ts=ts, decay=g["decay"], save=True)
    got = T.recur_grad(rowptr, u, x, saved=r["saved"], ts=ts, decay=g["decay"], dh=dh)
    close("h", r["h"][n:], want["h"], want["h_off"], dtype)
    close("last", r["last"][first:], want["last"], want["last_off"])
    for name in ("du", "dx"):
        close(name, got[name][n:], want[name], want[name + "_off"], dtype)
        assert not got[name][:n].any()
    close("ddecay", got["ddecay"], want["ddecay"], want["ddecay_off"])


@pytest.mark.parametrize("dtype, dim", [(F32, 64), (BF16, 33), (F32, 600), (BF16, 2500)])
@pytest.mark.parametrize("smoothing, sign", [(0.0, 1), (1.0, -1), (0.0, -1), (1.0, 1), (0.25, 1), (0.25, -1)])
def test_pair_loss_infinite_margins(T, smoothing, sign, dtype, dim):
    """A margin of infinity on the side whose factor is 0 adds nothing, on another side the loss is infinite; either way the gradients are the
    limit's, and the other pairs' are their own."""
    rng = np.random.default_rng(17)
    B, K = 5, 7
    a, p, n = values(rng, (B, dim), dtype), values(rng, (B, dim), dtype), values(rng, (B, K, dim), dtype)
    ref = rng.standard_normal((B, K)).astype(np.float32)
    far = rng.random((B, K)) < 0.3
    far[3] = True
    kw = dict(beta=1.0 / np.sqrt(dim), scale=1.0 / (B * K), smoothing=smoothing)
    got = T.pair_loss(torch_of(a, dtype), torch_of(p, dtype), torch_of(n, dtype), ref=torch_of(np.where(far, np.float32(-sign * np.inf), ref)), **kw)
    limit = O.pair_loss(a, p, n, ref=np.where(far, np.float32(-sign * 1e6), ref), **kw)      # (a margin of thousands: the slopes are 0 and 1)
    assert np.abs(limit["margin"][far]).min() > 1000
    for k in ("danchor", "dpos", "dneg"):
        close(k, got[k], limit[k], limit[k + "_off"], dtype)
    margin = got["margin"].cpu().numpy()
    assert (margin[far] == sign * np.inf).all()
    if smoothing == (0.0 if sign > 0 else 1.0):
        near = O.pair_loss(a, p, n, ref=ref, weight=np.where(far, 0.0, 1.0), **kw)
        close("loss", got["loss"], np.float64(near["loss"]), near["loss_off"])
    else:
        assert float(got["loss"]) == np.inf


@pytest.mark.parametrize("newest_first", [False, True])
@pytest.mark.parametrize("lens", [[], [0, 0], [3, 0, 10, 1], RAGGED], ids=["no_list", "empty_lists", "few", "ragged"])
@pytest.mark.parametrize("dtype, dim, more", [(F32, 33, 1), (F32, 100, 700), (BF16, 128, 64), (BF16, 70, 5000), (BF16, 300, 31)])
def test_recurrence_rows_of_no_list_are_zero(T, dtype, dim, more, lens, newest_first):
    """u and x with more rows than the lists hold: h, du and dx are zero there, whatever lay in their memory, and the products that make the
    gradients of weights can be taken over all rows."""
    import torch
    rng = np.random.default_rng(18)
    a = the_lists(rng, lens, dim, dtype, True, False)
    n = a["u"].shape[0]
    dlast, dh = values(rng, (len(lens), dim), F32), values(rng, (n + more, dim), dtype)
    want = O.recurrence(**a, newest_first=newest_first, dlast=dlast, dh=dh[:n])
    g = on_gpu(a, dtype)
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")      # noqa: E731
    for k in ("u", "x"):
        g[k] = torch.cat((g[k], nan(more, dim).to(g[k].dtype)))
    g["ts"] = torch.cat((g["ts"], nan(more)))
    stale = [nan(n + more, dim).to(g["u"].dtype) for _ in range(8)]      # memory that the outputs are likely to get
    del stale
    r = T.recur_run(**g, newest_first=newest_first, save=True)
    stale = [nan(n + more, dim).to(g["u"].dtype) for _ in range(8)]
    del stale
    got = T.recur_grad(**g, saved=r["saved"], newest_first=newest_first, dlast=torch_of(dlast), dh=torch_of(dh, dtype))
    for k, v in (("h", r["h"]), ("du", got["du"]), ("dx", got["dx"])):
        assert not v[n:].any(), k
        close(k, v[:n], want[k][:n], want[k + "_off"][:n], dtype)
        total, off = want[k].sum(0), want[k + "_off"].sum(0) + (n + 1) * 2.0 ** -24 * np.abs(want[k]).sum(0)
        if dtype == F32:
            close(f"sum of {k}", v.sum(0), total, off)
        else:
            assert bool(torch.isfinite(v.float().sum(0)).all())
    close("ddecay", got["ddecay"], want["ddecay"], want["ddecay_off"])
    # through the C interface, between guards
    desc = T._lists(g["rowptr"], g["u"], g["x"], g["ts"], g["decay"], None, None, newest_first)
    desc.flags |= T.TNS_ZERO_BEYOND
    ld, rows = dim + 3, n + more
    out = torch.full((rows * ld + 40,), 7.0, dtype=g["u"].dtype, device="cuda")
    work = torch.empty(T.tns_recur_workspace(desc)[0], dtype=torch.uint8, device="cuda")
    T.tns_recur_run(desc, out.data_ptr(), ld, 0, 0, work.data_ptr(), work.numel(), torch.cuda.current_stream().cuda_stream)
    inside = out[: rows * ld].view(rows, ld)
    assert not inside[n:, :dim].any() and bool((inside[:, dim:] == 7).all()) and bool((out[rows * ld:] == 7).all())
    close("h", inside[:n, :dim], want["h"][:n], want["h_off"][:n], dtype)


def test_within_autograd(T):
    """A Function of the caller's around the operators; what they change in place is noticed by a graph that kept it."""
    import torch
    rng = np.random.default_rng(19)
    a = the_lists(rng, [5, 0, 9], 12, F32, True, False)
    g = on_gpu(a, F32)

    class Last(torch.autograd.Function):
        @staticmethod
        def forward(ctx, u, x, decay):
            r = T.recur_run(g["rowptr"], u, x, ts=g["ts"], decay=decay, save=True)
            ctx.save_for_backward(u, x, decay, r["saved"])
            return r["last"]

        @staticmethod
        def backward(ctx, dlast):
            u, x, decay, saved = ctx.saved_tensors
            d = T.recur_grad(g["rowptr"], u, x, saved, ts=g["ts"], decay=decay, dlast=dlast.contiguous())
            return d["du"], d["dx"], d["ddecay"]

    leaves = [g[k].requires_grad_() for k in ("u", "x", "decay")]
    dlast = values(rng, (3, 12), F32)
    (Last.apply(*leaves) * torch_of(dlast)).sum().backward()
    want = O.recurrence(**a, dlast=dlast)
    for t, k in zip(leaves, ("du", "dx", "ddecay")):
        close(k, t.grad, want[k], want[k + "_off"])
    with pytest.raises(ValueError, match="autograd"):
        T.recur_run(g["rowptr"], *leaves[:2])

    ids, state, state_ts = torch.arange(3, dtype=torch.int32, device="cuda"), torch.zeros((3, 12), device="cuda"), torch.zeros(3, device="cuda")
    one, ts, x = torch.ones((3, 12), device="cuda"), torch.ones(3, device="cuda"), torch.ones((3, 12), device="cuda", requires_grad=True)
    kept = x * state
    versions = state._version, state_ts._version
    T.recur_step(ids, one, one, state, ts, torch.ones(12, device="cuda"), state_ts)
    assert state._version > versions[0] and state_ts._version > versions[1]
    with pytest.raises(RuntimeError, match="inplace"):
        kept.sum().backward()

    w = torch.ones(12, device="cuda", requires_grad=True)
    for bits in (32, 8):
        copy = torch.zeros(12, dtype=torch.bfloat16, device="cuda")
        opt = T.AdamW([w], [torch.ones(12, device="cuda")], copies=[copy], bits=bits)
        changed = [w, copy, opt.m[0], opt.v[0]] + ([opt.m_scale[0], opt.v_scale[0]] if bits == 8 else [])
        versions = [t._version for t in changed]
        kept = (x * w).sum()
        opt.step(1e-3, 1)
        assert all(t._version > v for t, v in zip(changed, versions))
        with pytest.raises(RuntimeError, match="inplace"):
            kept.backward()
        opt.close()


def test_gates_are_as_exact_as_stated(T):
    """z, 1 - z and the decay alone, from lists of one event (x = 1 without a state; x = 0 with a state of 1): the relative errors of the header,
    where the values are normal numbers."""
    import torch
    u = np.concatenate([np.linspace(-87, 87, 40_001), np.random.default_rng(23).normal(size=40_000)]).astype(np.float32)
    rowptr = torch.arange(len(u) + 1, device="cuda")
    g_u, one, none = torch_of(u)[:, None], torch.ones((len(u), 1), device="cuda"), torch.zeros((len(u), 1), device="cuda")
    bound = (1.5 * np.abs(u.astype(np.float64)) + 6) * O.U
    z, rest = O.sigmoid(u.astype(np.float64)), O.sigmoid(-u.astype(np.float64))
    for x, h0, want in ((one, None, z), (none, one, rest)):
        got = T.recur_run(rowptr, g_u, x, h0=h0)["h"][:, 0].cpu().numpy().astype(np.float64)
        normal = want >= 2.0 ** -126
        assert (np.abs(got - want) <= bound * want)[normal].all()
    # gates shut (1 - z = 1): the decay of a state of 1 over times that begin at 0
    for decay in (0.1, 1.0, 7.3):
        gap = np.linspace(0, 87 / decay, 40_001).astype(np.float32)
        shut, lam = torch.full((len(gap), 1), -200.0, device="cuda"), np.float32([decay])
        zero = torch.zeros((len(gap), 1), device="cuda")
        got = T.recur_run(torch.arange(len(gap) + 1, device="cuda"), shut, zero, ts=torch_of(gap), decay=torch_of(lam), h0=zero + 1, t0=zero[:, 0].contiguous())["h"][:, 0]
        v = lam.astype(np.float64) * gap
        want = np.exp(-v)
        # (and the product with 1 - z = 1)
        assert (np.abs(got.cpu().numpy() - want) <= (2.5 * v + 4) * O.U * want)[want >= 2.0 ** -126].all(), decay


@pytest.mark.parametrize("at", [0, 700])
def test_a_state_that_is_not_finite_stays_so(T, at):
    """An infinite value in a list of many tiles: from there on the list's states are infinite or NaN, before it and in other lists finite."""
    import torch
    rng = np.random.default_rng(24)
    a = the_lists(rng, [300, 3000, 50], 20, F32, True, True)
    a["x"][300 + at, 7] = np.inf
    h = T.recur_run(**on_gpu(a, F32))["h"].cpu().numpy()
    bad = ~np.isfinite(h)
    assert bad[300 + at: 3300, 7].all() and bad.sum() == 3000 - at
