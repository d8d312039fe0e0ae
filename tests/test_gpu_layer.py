"""The layer operators on the GPU against the oracle in 64 bits.  Tolerances are the oracle's running error bounds (a result in bf16 lies
between the roundings of the bound's two ends)."""
import numpy as np
import pytest

from oracle import layer_oracle as O
from test_gpu_train import BF16, F32, close, torch_of, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2311_17410_amd import layer_binding
    layer_binding.lib()
    return layer_binding


# ---- attention -----------------------------------------------------------------------------------

RAGGED = [3, 0, 10, 1, 0, 0, 7, 10, 10, 2] * 7
LISTS = {
    "no list": [], "none": [0], "one": [1], "empty ones": [0, 0, 0], "ragged": RAGGED, "wave": [64], "wave and one": [65], "around blocks": [63, 1, 64, 2, 127, 129, 128],
    "holes": [5] + [0] * 100 + [70] + [0] * 64 + [1], "ones": [1] * 70, "long": [1000], "long and short": [5, 900, 0, 2, 300, 64, 128, 191, 193], "several long": [40, 700, 450, 0, 600],
}


def the_events(rng, lens, heads, kv_heads, dim, dtype, buckets=8, times=True, masked=0.0, newest_first=True):
    rp = np.concatenate([[0], np.cumsum(np.asarray(lens, np.int64))]).astype(np.int64)
    n, S = int(rp[-1]), len(lens)
    a = dict(rowptr=rp, q=values(rng, (S, heads, dim), dtype), k=values(rng, (n, kv_heads, dim), dtype), v=values(rng, (n, kv_heads, dim), dtype), newest_first=newest_first)
    if buckets:
        a.update(table=values(rng, (buckets, heads), F32), edges=None if buckets == 1 else np.sort(rng.uniform(0, 5, buckets - 1)).astype(np.float32))
        if not times and buckets > 1:
            a["edges"] = np.float32(np.sort(rng.choice(40, buckets - 1, replace=buckets > 40)))      # whole numbers: places lie on them
    if times:
        a.update(t=rng.uniform(4, 5, S).astype(np.float32), ts=rng.uniform(0, 5, n).astype(np.float32))
    if masked:
        a["mask"] = rng.random(n) >= masked
        if S:
            a["mask"][rp[S // 2]: rp[S // 2 + 1]] = False
        a["k"][~a["mask"]] = np.nan
        a["v"][~a["mask"]] = np.nan
    return a


def on_gpu(a, dtype):
    return {k: v if isinstance(v, (bool, float)) else torch_of(v, dtype if k in ("q", "k", "v") else None) for k, v in a.items()}


def cleaned(a):
    """The oracle's arguments: rows that do not count are zero there."""
    o = dict(a)
    if a.get("mask") is not None and "index" not in a:
        for name in ("k", "v"):
            o[name] = np.where(a["mask"][:, None, None], a[name], 0)
    return o


def check_attend(L, a, dtype, dout=None, got=None):
    rng = np.random.default_rng(99)
    g = on_gpu(a, dtype)
    dout = values(rng, a["q"].shape, dtype) if dout is None else dout
    want = O.attend(**cleaned(a), dout=dout)
    r = L.attend_run(**g, save=True)
    close("out", r["out"], want["out"], want["out_off"], dtype)
    only = L.attend_run(**g)
    assert only["saved"] is None and bool((only["out"] == r["out"]).all())
    d = L.attend_grad(**g, saved=r["saved"], dout=torch_of(dout, dtype))
    n = int(a["rowptr"][-1])
    close("dq", d["dq"], want["dq"], want["dq_off"], dtype)
    for name in ("dk", "dv"):
        close(name, d[name][:n], want[name][:n], want[name + "_off"][:n], dtype)
        if a.get("mask") is not None:
            assert not d[name][:n][~g["mask"]].any()
    if "table" in a:
        close("dtable", d["dtable"], want["dtable"], want["dtable_off"])
    else:
        assert d["dtable"] is None
    return r, d


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads, kv_heads, buckets, times, masked, newest_first", [(2, 2, 8, True, 0.3, True), (4, 2, 9, False, 0.0, True), (3, 1, 33, False, 0.2, False), (1, 1, 0, False, 0.0, False)])
@pytest.mark.parametrize("lens", list(LISTS), ids=[k.replace(" ", "_") for k in LISTS])
def test_attend(L, lens, heads, kv_heads, buckets, times, masked, newest_first, dtype):
    rng = np.random.default_rng(len(LISTS[lens]) + heads)
    check_attend(L, the_events(rng, LISTS[lens], heads, kv_heads, 16, dtype, buckets, times, masked, newest_first), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [1, 2, 3, 4, 5, 8, 12, 30, 31, 43, 50, 64, 65, 100, 128, 129, 200, 254, 255, 256])
def test_attend_channels(L, dim, dtype):
    rng = np.random.default_rng(dim)
    check_attend(L, the_events(rng, [4, 0, 70, 1, 9, 140], 2, 1, dim, dtype, masked=0.2), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads, kv_heads, dim", [(3, 3, 50), (5, 5, 4), (8, 8, 64), (24, 24, 16), (6, 2, 8), (5, 1, 20), (7, 1, 64), (8, 1, 32), (16, 2, 33), (12, 3, 128), (40, 20, 2), (1024, 1024, 1)])
def test_attend_heads(L, heads, kv_heads, dim, dtype):
    rng = np.random.default_rng(heads + dim)
    check_attend(L, the_events(rng, [4, 0, 20, 1, 150], heads, kv_heads, dim, dtype, buckets=2, masked=0.1), dtype)


@pytest.mark.parametrize("buckets, heads", [(1, 2), (2, 2), (3, 1), (64, 2), (65, 4), (255, 2), (256, 8)])
def test_attend_buckets(L, buckets, heads):
    rng = np.random.default_rng(buckets)
    a = the_events(rng, [300, 20, 64], heads, heads, 8, F32, buckets)
    if buckets > 2:
        a["edges"][1] = a["edges"][0]                             # a bucket that nothing falls into
        a["ts"][:20] = a["t"][0] - a["edges"][0]                  # (rounded: beside the border or on it)
    check_attend(L, a, F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads, kv_heads", [(2, 2), (4, 1)])
def test_attend_ruled_out_buckets(L, heads, kv_heads, dtype):
    """A table entry of -infinity leaves its events out, head by head, whatever their rows hold."""
    rng = np.random.default_rng(4)
    lens = [1, 30, 0, 200, 4, 64]
    a = the_events(rng, lens, heads, kv_heads, 24, dtype, buckets=4, newest_first=True, times=False)
    a["edges"] = np.float32([1, 3, 100])
    a["table"][0, 0] = a["table"][2, 0] = a["table"][1, 1] = -np.inf
    check_attend(L, a, dtype)
    a["table"][0] = -np.inf                                       # the newest event of every list counts for no head: a list of one has nothing
    a["k"][a["rowptr"][:-1][np.array(lens) > 0]] = np.nan
    a["v"][a["rowptr"][:-1][np.array(lens) > 0]] = np.inf
    g = on_gpu(a, dtype)
    dout = values(rng, a["q"].shape, dtype)
    first = a["rowptr"][:-1][np.array(lens) > 0]
    o = dict(a, k=a["k"].copy(), v=a["v"].copy())
    o["k"][first] = o["v"][first] = 0
    want = O.attend(**o, dout=dout)
    r = L.attend_run(**g, save=True)
    close("out", r["out"], want["out"], want["out_off"], dtype)
    assert not r["out"][0].any() and not r["out"][2].any()
    d = L.attend_grad(**g, saved=r["saved"], dout=torch_of(dout, dtype))
    for name in ("dq", "dk", "dv"):
        close(name, d[name], want[name], want[name + "_off"], dtype)
    close("dtable", d["dtable"], want["dtable"], want["dtable_off"])
    if heads > 2:                       # rows that one head of a group leaves out hold numbers that are not finite; it stays as it was
        a = the_events(rng, [64, 10], heads, kv_heads, 24, dtype, buckets=2, newest_first=True, times=False)
        a["edges"] = np.float32([5])
        a["table"][0, 1] = -np.inf
        want = O.attend(**a, dout=dout[:2])
        a["v"][2] = np.nan
        a["k"][3] = np.nan
        g = on_gpu(a, dtype)
        r = L.attend_run(**g, save=True)
        d = L.attend_grad(**g, saved=r["saved"], dout=torch_of(dout[:2], dtype))
        for name, got in (("out", r["out"]), ("dq", d["dq"])):
            close(name, got[:, 1], want[name][:, 1], want[name + "_off"][:, 1], dtype)
            assert bool(got[0, 0].isnan().all()) and not bool(got[1].isnan().any())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads, kv_heads, dim", [(2, 2, 50), (4, 2, 32), (1, 1, 7)])
def test_attend_gathered(L, heads, kv_heads, dim, dtype):
    """Keys and values from a table of nodes; ids that it does not hold; the same id many times; a table without rows."""
    import torch
    rng = np.random.default_rng(dim)
    a = the_events(rng, RAGGED + [400, 3], heads, kv_heads, dim, dtype, masked=0.1)
    n, nodes = int(a["rowptr"][-1]), 50
    a["index"] = rng.integers(0, nodes, n).astype(np.int32)
    a["index"][rng.random(n) < 0.1] = rng.choice([-1, nodes, 2 ** 31 - 1, -2 ** 31])
    a["index"][:3] = [-1, nodes, -7]                              # the first list has none of its three
    a["index"][-3:] = 5
    a["k"], a["v"] = values(rng, (nodes, kv_heads, dim), dtype), values(rng, (nodes, kv_heads, dim), dtype)
    want = O.attend(**a)
    g = on_gpu(a, dtype)
    r = L.attend_run(**g)
    close("out", r["out"], want["out"], want["out_off"], dtype)
    assert not r["out"][0].any()
    g["k"], g["v"] = (torch.empty((0, kv_heads, dim), dtype=g["k"].dtype, device="cuda") for _ in range(2))
    assert not L.attend_run(**g)["out"].any()


def test_attend_ages_at_the_ends(L):
    """Times that are infinite, equal, later than the target's or no numbers."""
    rng = np.random.default_rng(6)
    a = the_events(rng, [60, 30, 10], 2, 2, 16, F32, buckets=5)
    a["edges"] = np.float32([0.0, 1.0, 1.0, 3e38])
    a["ts"][:60] = rng.choice([-np.inf, 0, 1, 4.5, 1e30, np.inf, np.nan], 60).astype(np.float32)
    a["t"][1] = np.inf
    a["t"][2] = np.nan
    check_attend(L, a, F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_far_scores_and_nan(L, dtype):
    """Scores of thousands: the largest alone counts; a NaN of one list stays in it."""
    rng = np.random.default_rng(7)
    a = the_events(rng, [70, 20, 30], 2, 2, 16, dtype)
    a["q"][0] *= 256
    a["k"][:70] *= 64
    want = O.attend(**a)
    g = on_gpu(a, dtype)
    out = L.attend_run(**g)["out"]
    # exponents of thousands: p is off by their size times 2^-24, which the bound has to first order
    close("out", out, want["out"], want["out_off"], dtype)
    g["v"][75, 0, 3] = float("nan")
    got = L.attend_run(**g)["out"]
    assert bool(got[1, 0, 3].isnan()) and int(got.isnan().sum()) == 1
    g["k"][75, 0, 3] = float("nan")
    got = L.attend_run(**g)["out"]
    assert bool(got[1, 0].isnan().all()) and int(got.isnan().sum()) == 16


@pytest.mark.parametrize("dtype, dim, skip, more", [(F32, 16, 0, 4), (F32, 16, 1, 3), (BF16, 32, 0, 8), (BF16, 32, 2, 4), (BF16, 32, 1, 5), (BF16, 20, 4, 2)])
def test_attend_strides_and_rows_beyond_the_lists(L, dtype, dim, skip, more):
    """Rows that lie apart, at odd addresses; rows after the last list are not read (NaN), their gradients zero, or through the C interface left."""
    import torch
    rng = np.random.default_rng(8)
    a = the_events(rng, RAGGED + [150], 4, 2, dim, dtype)
    n, beyond = int(a["rowptr"][-1]), 100
    g = on_gpu(a, dtype)

    def apart(t, rows):
        heads = t.shape[1]
        ld = heads * dim + more
        wide = torch.full(((rows + 1) * ld + skip,), float("nan"), dtype=t.dtype, device="cuda")
        view = wide[skip: skip + rows * ld].view(rows, ld)[:, : heads * dim].unflatten(1, (heads, dim))
        view[: t.shape[0]] = t
        return view

    g.update(q=apart(g["q"], len(RAGGED) + 1), k=apart(g["k"], n + beyond), v=apart(g["v"], n + beyond), ts=torch.cat((g["ts"], torch.full((beyond,), float("nan"), device="cuda"))))
    dout = values(rng, a["q"].shape, dtype)
    want = O.attend(**a, dout=dout)
    r = L.attend_run(**g, save=True)
    close("out", r["out"], want["out"], want["out_off"], dtype)
    d = L.attend_grad(**g, saved=r["saved"], dout=torch_of(dout, dtype))
    for name in ("dk", "dv"):
        close(name, d[name][:n], want[name], want[name + "_off"], dtype)
        assert not d[name][n:].any()
    close("dq", d["dq"], want["dq"], want["dq_off"], dtype)
    desc = L._described(g["rowptr"], g["q"], g["k"], g["v"], g["t"], g["ts"], g["edges"], g["table"], None, None, None, True)
    desc.flags &= ~L.TNS_ZERO_BEYOND
    size, need = 2 * dim, L.tns_attend_workspace(desc)[1]
    dk, dv = (torch.full(((n + beyond) * size + skip + 7,), 7.0, dtype=g["q"].dtype, device="cuda") for _ in range(2))
    dq, dtable, ws, dd = torch.empty_like(d["dq"]), torch.empty_like(d["dtable"]), torch.empty(need, dtype=torch.uint8, device="cuda"), torch_of(dout, dtype)
    at = skip * dk.element_size()
    L.tns_attend_grad(desc, r["saved"].data_ptr(), dd.data_ptr(), dq.data_ptr(), dk.data_ptr() + at, dv.data_ptr() + at, dtable.data_ptr(), ws.data_ptr(), need,
                      torch.cuda.current_stream().cuda_stream)
    for name, got in (("dk", dk), ("dv", dv)):
        assert bool((got[:skip] == 7).all()) and bool((got[skip + n * size:] == 7).all())
        close(name, got[skip: skip + n * size].view(n, 2, dim), want[name], want[name + "_off"], dtype)


def test_attend_gradients_against_differences(L):
    """Slope along a direction: the gradients' product with it, and a central difference of the oracle."""
    rng = np.random.default_rng(9)
    a = the_events(rng, [30, 0, 200, 7], 4, 2, 6, F32, masked=0.1)
    a = cleaned(a)
    dout = values(rng, a["q"].shape, F32)
    g = on_gpu(a, F32)
    r = L.attend_run(**g, save=True)
    d = L.attend_grad(**g, saved=r["saved"], dout=torch_of(dout))
    for name in ("q", "k", "v", "table"):
        way = rng.standard_normal(a[name].shape)
        ends = [(O.attend(**dict(a, **{name: a[name].astype(np.float64) + by * way}))["out"] * dout).sum() for by in (1e-5, -1e-5)]
        mine = d["d" + name].cpu().numpy().astype(np.float64) * way
        # a difference is off by its second order (1e-10 of the third derivative) and by the sums' rounding over 1e-5
        assert abs(mine.sum() - (ends[0] - ends[1]) / 2e-5) < 1e-5 * np.abs(mine).sum() + 1e-6, name


def replayed(both):
    """The same bits again, on another stream, and from a graph that is replayed with eager work between."""
    import torch
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


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_same_bits_again_on_another_stream_and_in_a_graph(L, dtype):
    rng = np.random.default_rng(10)
    a = the_events(rng, [5000, 3, 0, 800] + RAGGED, 4, 2, 20, dtype)
    g, dout = on_gpu(a, dtype), torch_of(values(rng, a["q"].shape, dtype), dtype)

    def both():
        r = L.attend_run(**g, save=True)
        return dict(out=r["out"], **L.attend_grad(**g, saved=r["saved"], dout=dout))

    replayed(both)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_many_long_lists(L, dtype):
    """Blocks of more than 64 rows, thousands of parts, several lists with several parts in each workgroup's share."""
    rng = np.random.default_rng(11)
    lens = [20000, 1, 0, 130000, 700, 64] + [300] * 1600
    a = the_events(rng, lens, 1, 1, 4, dtype, buckets=0, times=False)
    check_attend(L, a, dtype)


def test_attend_offsets_beyond_32_bits(L):
    """Rows of k and v, and of their gradients, beyond 2^32 bytes and values: the lists at the end equal the same lists alone."""
    import torch
    n, dim, tail = (1 << 23) + 5000, 256, [300, 0, 40, 7, 1]
    rng = np.random.default_rng(12)
    a = the_events(rng, tail, 2, 2, dim, BF16)
    rows = n + sum(tail)
    g = on_gpu(a, BF16)
    k, v = (torch.zeros((rows, 2, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[n:], v[n:] = g["k"], g["v"]
    zeros = lambda m: torch.zeros((m,), device="cuda")            # noqa: E731
    g.update(k=k, v=v, q=torch.cat((torch.zeros((3, 2, dim), dtype=torch.bfloat16, device="cuda"), g["q"])), ts=torch.cat((zeros(n), g["ts"])), t=torch.cat((zeros(3), g["t"])),
             rowptr=torch.cat((torch.tensor([0, 10, n // 2]), n + torch.from_numpy(a["rowptr"]))).cuda())
    dout = values(rng, a["q"].shape, BF16)
    want = O.attend(**a, dout=dout)
    r = L.attend_run(**g, save=True)
    close("out", r["out"][3:], want["out"], want["out_off"], BF16)
    d = L.attend_grad(**g, saved=r["saved"], dout=torch.cat((torch.zeros_like(g["q"][:3]), torch_of(dout, BF16))))
    for name in ("dk", "dv"):
        close(name, d[name][n:], want[name], want[name + "_off"], BF16)
        assert not d[name][:n].any()
    del d, r
    at = torch.arange(rows, device="cuda", dtype=torch.int32)[n:].contiguous()
    got = L.attend_run(torch.from_numpy(a["rowptr"]).cuda(), g["q"][3:], k, v, t=g["t"][3:], ts=g["ts"][n:], edges=g["edges"], table=g["table"], index=at, newest_first=True)["out"]
    close("gathered", got, want["out"], want["out_off"], BF16)


# ---- between two layers --------------------------------------------------------------------------

def the_block(rng, rows, dim, dtype, **without):
    a = dict(x=values(rng, (rows, dim), dtype), branch=values(rng, (rows, dim), dtype, 3.0) + np.float32(1), gate=values(rng, (rows, dim), dtype, 2.0), scale=values(rng, dim, F32),
             post=values(rng, dim, F32), pre=values(rng, dim, F32))
    if dtype == BF16:
        a["branch"] = values(rng, (rows, dim), dtype, 3.0)
    for name in without:
        a[name] = None
    return a


def block_on_gpu(a, dtype):
    return {k: torch_of(v, dtype if k in ("x", "branch", "gate") else None) for k, v in a.items()}


def check_block(L, a, dtype, dout, dnext, **kw):
    want = O.block(**a, dout=np.zeros_like(a["x"]) if dout is None else dout, dnext=dnext, **kw)
    g = block_on_gpu(a, dtype)
    r = L.block_run(**g, **kw)
    close("out", r["out"], want["out"], want["out_off"], dtype)
    if a["pre"] is not None:
        close("next", r["next"], want["next"], want["next_off"], dtype)
    else:
        assert r["next"] is None
    d = L.block_grad(**g, dout=torch_of(dout, dtype), dnext=torch_of(dnext, dtype), **kw)
    for name in ("dx", "dbranch", "dgate"):
        if name == "dgate" and a["gate"] is None:
            assert d[name] is None
        else:
            close(name, d[name], want[name], want[name + "_off"], dtype)
    for name in ("scale", "post", "pre"):
        if a[name] is None:
            assert d["d" + name] is None
        else:
            close("d" + name, d["d" + name], want["d" + name], want["d" + name + "_off"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("dim", [1, 2, 4, 7, 8, 31, 32, 33, 64, 100, 128, 172, 173, 256, 260, 511, 512, 513, 600, 1000, 1024, 2048, 2049, 4100, 8191, 8192])
def test_block_channels(L, dim, center, dtype):
    rng = np.random.default_rng(dim)
    rows = 37 if dim < 600 else 5
    a = the_block(rng, rows, dim, dtype)
    check_block(L, a, dtype, values(rng, (rows, dim), dtype), values(rng, (rows, dim), dtype), center=center, eps=1e-3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [0, 1, 3, 8, 9, 3000])
@pytest.mark.parametrize("without", [(), ("gate",), ("scale",), ("post",), ("pre",), ("gate", "scale", "post"), ("gate", "post", "pre", "scale")], ids=lambda w: "_".join(w) or "all")
def test_block_parts(L, without, rows, dtype):
    rng = np.random.default_rng(rows)
    a = the_block(rng, rows, 36, dtype, **dict.fromkeys(without))
    dnext = None if "pre" in without else values(rng, (rows, 36), dtype)
    check_block(L, a, dtype, values(rng, (rows, 36), dtype), dnext)
    check_block(L, a, dtype, None, dnext)
    check_block(L, a, dtype, values(rng, (rows, 36), dtype), None)


@pytest.mark.parametrize("dtype, dim, ld, skip", [(F32, 40, 43, 1), (F32, 40, 44, 0), (BF16, 40, 48, 4), (BF16, 40, 52, 2), (BF16, 64, 64, 8), (BF16, 40, 41, 1), (F32, 700, 704, 4)])
def test_block_strides_and_addresses(L, dtype, dim, ld, skip):
    import torch
    rng = np.random.default_rng(5)
    rows = 50
    a = the_block(rng, rows, dim, dtype)
    dout, dnext = values(rng, (rows, dim), dtype), values(rng, (rows, dim), dtype)
    want = O.block(**a, dout=dout, dnext=dnext)
    g = block_on_gpu(a, dtype)

    def apart(t):
        wide = torch.full((rows * ld + skip,), float("nan"), dtype=t.dtype, device="cuda")
        view = wide[skip:].view(rows, ld)[:, :dim]
        view.copy_(t)
        return view

    for name in ("x", "branch", "gate"):
        g[name] = apart(g[name])
    r = L.block_run(**g)
    d = L.block_grad(**g, dout=apart(torch_of(dout, dtype)), dnext=apart(torch_of(dnext, dtype)))
    for name, got in dict(r, dx=d["dx"], dbranch=d["dbranch"], dgate=d["dgate"]).items():
        close(name, got, want[name], want[name + "_off"], dtype)
    for name in ("dscale", "dpost", "dpre"):
        close(name, d[name], want[name], want[name + "_off"])
    # outputs at odd addresses, with guards
    desc = L._between(g["x"], g["branch"], g["gate"], g["scale"], g["post"], g["pre"], 1e-6, False)
    outs = {k: torch.full((rows * dim + 2 * skip + 8,), 7.0, dtype=g["x"].dtype, device="cuda") for k in ("out", "next")}
    at = skip * g["x"].element_size()
    L.tns_block_run(desc, outs["out"].data_ptr() + at, outs["next"].data_ptr() + at, torch.cuda.current_stream().cuda_stream)
    for name, got in outs.items():
        assert bool((got[:skip] == 7).all()) and bool((got[skip + rows * dim:] == 7).all())
        close(name, got[skip: skip + rows * dim].view(rows, dim), want[name], want[name + "_off"], dtype)


def test_block_far_gates_offsets_and_nan(L):
    """Gates from -200 to 200; rows far from zero with little spread; a NaN stays in its row and in the sums."""
    rng = np.random.default_rng(6)
    a = the_block(rng, 40, 100, F32)
    a["gate"][:20] = rng.choice([-200.0, -88.5, -30, 0, 30, 88.5, 200], (20, 100)).astype(np.float32)
    a["branch"][30:] += 1000
    check_block(L, a, F32, values(rng, (40, 100), F32), values(rng, (40, 100), F32), center=True)
    g = block_on_gpu(a, F32)
    g["branch"][7, 3] = float("nan")
    r = L.block_run(**g)
    for t in (r["out"], r["next"]):
        assert bool(t[7].isnan().all()) and int(t.isnan().sum()) == 100


def test_block_gradients_against_differences(L):
    rng = np.random.default_rng(7)
    a = the_block(rng, 6, 20, F32)
    dout, dnext = values(rng, (6, 20), F32), values(rng, (6, 20), F32)
    d = L.block_grad(**block_on_gpu(a, F32), dout=torch_of(dout), dnext=torch_of(dnext), center=True)
    for name in a:
        way = rng.standard_normal(a[name].shape)
        ends = []
        for by in (1e-5, -1e-5):
            o = O.block(**dict(a, **{name: a[name].astype(np.float64) + by * way}), center=True)
            ends.append((o["out"] * dout).sum() + (o["next"] * dnext).sum())
        mine = d["d" + name].cpu().numpy().astype(np.float64) * way
        assert abs(mine.sum() - (ends[0] - ends[1]) / 2e-5) < 1e-5 * np.abs(mine).sum() + 1e-6, name


@pytest.mark.parametrize("dtype, dim", [(F32, 100), (BF16, 172), (F32, 2000)])
def test_block_same_bits_again_on_another_stream_and_in_a_graph(L, dtype, dim):
    rng = np.random.default_rng(8)
    a = the_block(rng, 9001, dim, dtype) if dim < 2000 else the_block(rng, 2001, dim, dtype)
    g = block_on_gpu(a, dtype)
    dout, dnext = (torch_of(values(rng, a["x"].shape, dtype), dtype) for _ in range(2))
    replayed(lambda: dict(L.block_run(**g), **L.block_grad(**g, dout=dout, dnext=dnext)))


def test_block_offsets_beyond_32_bits(L):
    import torch
    rows, dim, tail = (1 << 23) + 100, 520, 40
    rng = np.random.default_rng(9)
    a = the_block(rng, tail, dim, BF16)
    dout, dnext = values(rng, (tail, dim), BF16), values(rng, (tail, dim), BF16)
    want = O.block(**a, dout=dout, dnext=dnext)
    g = block_on_gpu(a, BF16)
    behind = lambda t: torch.cat((torch.zeros((rows, dim), dtype=t.dtype, device="cuda"), t))      # noqa: E731
    for name in ("x", "branch", "gate"):
        g[name] = behind(g[name])
    r = L.block_run(**g)
    for name in ("out", "next"):
        close(name, r[name][rows:], want[name], want[name + "_off"], BF16)
    del r
    d = L.block_grad(**g, dout=behind(torch_of(dout, BF16)), dnext=behind(torch_of(dnext, BF16)))
    for name in ("dx", "dbranch", "dgate"):
        close(name, d[name][rows:], want[name], want[name + "_off"], BF16)
        assert not d[name][:rows].any()


# ---- distillation --------------------------------------------------------------------------------

def the_scores(rng, B, n, K, dtype, lse=False, weight=False):
    a = dict(logits=values(rng, (B, n), dtype, 2.0), ids=np.stack([rng.choice(n, K, replace=K > n) for _ in range(B)]).astype(np.int32) if B else np.zeros((0, K), np.int32),
             teacher=values(rng, (B, K), F32, 2.0), lse=None, weight=None)
    if lse:
        a["lse"] = (np.log(np.exp(a["teacher"].astype(np.float64) / 2).sum(1)) + rng.uniform(0.05, 1, B)).astype(np.float32)
    if weight:
        a["weight"] = (rng.random(B) > 0.4).astype(np.float32) * rng.uniform(0.5, 2, B).astype(np.float32)
        a["weight"][0] = 1.5
    return a


def check_distill(L, a, dtype, **kw):
    kw = dict(dict(temperature=2.0, scale=0.5), **kw)
    want = O.distill(**a, **kw)
    g = {k: torch_of(v, dtype if k == "logits" else None) for k, v in a.items()}
    if a["weight"] is not None:
        g["logits"][g["weight"] == 0] = float("nan")
    r = L.distill(**g, **kw)
    close("rows", r["rows"], want["rows"], want["rows_off"])
    close("loss", r["loss"].reshape(1), want["loss"].reshape(1), np.reshape(want["loss_off"], 1))
    close("dlogits", r["dlogits"], want["dlogits"], want["dlogits_off"], dtype)
    only = L.distill(**g, **kw, grad=False)
    assert only["dlogits"] is None and bool((only["rows"] == r["rows"]).all()) and float(only["loss"]) == float(r["loss"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lse, weight", [(False, False), (True, True)])
@pytest.mark.parametrize("n", [1, 2, 7, 64, 100, 508, 509, 1000, 1016, 1017, 2044, 2045, 4088, 4089, 8188, 8189, 16376, 16377, 16380, 16381, 32760, 32761, 70001])
def test_distill_candidates(L, n, lse, weight, dtype):
    rng = np.random.default_rng(n)
    check_distill(L, the_scores(rng, 5, n, min(20, n), dtype, lse and n > 1, weight), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B, n, K", [(0, 10, 3), (3, 10, 0), (1, 300, 1), (40, 300, 100), (3, 2000, 1000), (2, 5000, 1024), (2, 40000, 1024), (3000, 20, 4)])
@pytest.mark.parametrize("lse", [False, True])
def test_distill_rows_and_ids(L, B, n, K, lse, dtype):
    rng = np.random.default_rng(B + K)
    check_distill(L, the_scores(rng, B, n, K, dtype, lse), dtype, temperature=1.0 if not lse else 2.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lse", [False, True])
@pytest.mark.parametrize("n", [50, 3000, 40000])
def test_distill_ids_outside_twice_and_without_mass(L, n, lse, dtype):
    rng = np.random.default_rng(n)
    a = the_scores(rng, 6, n, 12, dtype, lse)
    a["ids"][0, 3:] = rng.choice([-1, n, 2 ** 31 - 1, -2 ** 31], 9)
    a["ids"][1] = -1                                              # no entry at all
    a["ids"][2] = [n - 1, 0, n - 1, 5, 5, 5, 0, n - 1, 7, 8, 9, 5]
    a["ids"][3] = n - 1
    a["teacher"][4, :5] = -np.inf
    a["teacher"][5] = -np.inf
    if lse:                                                       # (the sum over all stays above that over the list)
        a["lse"][:] = np.log(np.exp(np.maximum(a["teacher"].astype(np.float64), -1e30) / 2).sum(1) + 1.0).astype(np.float32)
    check_distill(L, a, dtype)


@pytest.mark.parametrize("dtype, n, ld, skip", [(F32, 1000, 1001, 1), (F32, 1000, 1004, 0), (BF16, 3001, 3001, 0), (BF16, 3001, 3007, 3), (F32, 40000, 40003, 2), (BF16, 70001, 70001, 5)])
def test_distill_strides_and_addresses(L, dtype, n, ld, skip):
    """Rows at every address; nothing before, between or behind them is read into a result or written."""
    import torch
    rng = np.random.default_rng(n)
    B = 9
    a = the_scores(rng, B, n, 30, dtype, True)
    want = O.distill(**a, temperature=2.0)
    g = {k: torch_of(v, dtype if k == "logits" else None) for k, v in a.items()}
    wide = torch.full((B * ld + skip,), float("nan"), dtype=g["logits"].dtype, device="cuda")
    view = wide[skip:].view(B, ld)[:, :n]
    view.copy_(g["logits"])
    g["logits"] = view
    r = L.distill(**g, temperature=2.0)
    close("rows", r["rows"], want["rows"], want["rows_off"])
    close("dlogits", r["dlogits"], want["dlogits"], want["dlogits_off"], dtype)
    out = torch.full((B * n + skip + 9,), 7.0, dtype=view.dtype, device="cuda")
    loss, need = torch.empty((), device="cuda"), L.tns_distill_workspace(B, n, 30)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    d = L.tns_distill_desc(B, n, 30, 0 if dtype == F32 else 1, view.data_ptr(), ld, g["ids"].data_ptr(), g["teacher"].data_ptr(), g["lse"].data_ptr(), None, 2.0, 1.0)
    L.tns_distill(d, loss.data_ptr(), 0, out.data_ptr() + skip * out.element_size(), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert bool((out[:skip] == 7).all()) and bool((out[skip + B * n:] == 7).all())
    assert torch.equal(out[skip: skip + B * n].view(B, n), r["dlogits"]) and float(loss) == float(r["loss"])


@pytest.mark.parametrize("n", [300, 40000])
def test_distill_ruled_out_far_and_nan_scores(L, n):
    """Candidates of score -infinity have q = 0; scores thousands apart; a NaN stays in its row."""
    import torch
    rng = np.random.default_rng(3)
    a = the_scores(rng, 4, n, 8, F32, True)
    a["logits"][1] *= 1000
    check_distill(L, a, F32)
    g = {k: torch_of(v) for k, v in a.items()}
    out = torch.ones(n, dtype=torch.bool, device="cuda")
    out[g["ids"][0].long()] = False
    out[: n // 2] = False
    g["logits"][0, out] = -float("inf")
    g["logits"][2, 17] = float("nan")
    r = L.distill(**g, temperature=2.0)
    clean = dict(a, logits=g["logits"].double().cpu().numpy())
    want = O.distill(**{k: None if v is None else v[:1] for k, v in clean.items()}, temperature=2.0)
    close("rows", r["rows"][:1], want["rows"], want["rows_off"])
    close("dlogits", r["dlogits"][:1], want["dlogits"], want["dlogits_off"])
    assert bool(r["rows"].isnan()[2]) and bool(r["dlogits"][2].isnan().all()) and int(r["dlogits"].isnan().sum()) == n and bool(r["loss"].isnan())
    # a candidate with mass that the student rules out: an infinite loss, a gradient of -p
    g["logits"][3, g["ids"][3, 0].long()] = -float("inf")
    r = L.distill(**g, temperature=2.0)
    assert float(r["rows"][3]) == float("inf") and bool(r["dlogits"][3].isfinite().all())


def test_distill_gradients_against_differences(L):
    rng = np.random.default_rng(4)
    for lse in (False, True):
        a = the_scores(rng, 5, 40, 6, F32, lse)
        d = L.distill(**{k: torch_of(v) for k, v in a.items()}, temperature=2.0)["dlogits"].cpu().numpy().astype(np.float64)
        way = rng.standard_normal(a["logits"].shape)
        ends = [float(O.distill(**dict(a, logits=a["logits"].astype(np.float64) + by * way), temperature=2.0)["loss"]) for by in (1e-5, -1e-5)]
        assert abs((d * way).sum() - (ends[0] - ends[1]) / 2e-5) < 1e-5 * np.abs(d * way).sum() + 1e-6


@pytest.mark.parametrize("dtype, n", [(F32, 500), (BF16, 9001), (F32, 50001)])
def test_distill_same_bits_again_on_another_stream_and_in_a_graph(L, dtype, n):
    rng = np.random.default_rng(5)
    a = the_scores(rng, 30, n, 50, dtype, True, True)
    a["ids"][:, 7] = a["ids"][:, 3] = a["ids"][:, 20]             # three of a kind
    g = {k: torch_of(v, dtype if k == "logits" else None) for k, v in a.items()}
    replayed(lambda: L.distill(**g))


@pytest.mark.parametrize("n", [1 << 20, 3000])
def test_distill_offsets_beyond_32_bits(L, n):
    import torch
    rng = np.random.default_rng(6)
    a = the_scores(rng, 2, n, 10, BF16, True)
    before = (1 << 32) // n + 1
    g = {k: torch_of(v, BF16 if k == "logits" else None) for k, v in a.items()}
    weight = torch.zeros(before + 2, device="cuda")
    weight[before:] = 1
    behind = lambda t: torch.cat((torch.zeros((before,) + t.shape[1:], dtype=t.dtype, device="cuda"), t))      # noqa: E731
    r = L.distill(behind(g["logits"]), behind(g["ids"]), behind(g["teacher"]), lse=behind(g["lse"]), weight=weight, temperature=2.0)
    want = O.distill(**a, temperature=2.0)
    close("rows", r["rows"][before:], want["rows"], want["rows_off"])
    close("dlogits", r["dlogits"][before:], want["dlogits"], want["dlogits_off"], BF16)
    assert not r["dlogits"][:before].any() and not r["rows"][:before].any()


# ---- what tensors may be -------------------------------------------------------------------------

def test_refusals_of_tensors(L):
    import torch
    from paper_2311_17410_amd.binding import TnsError
    q = torch.zeros((2, 2, 8), device="cuda")
    k = torch.zeros((4, 2, 8), device="cuda")
    rp = torch.tensor([0, 1, 4], device="cuda")
    x, w, ids = torch.zeros((4, 8), device="cuda"), torch.zeros(8, device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    table, edges = torch.zeros((3, 2), device="cuda"), torch.zeros(2, device="cuda")
    for call in (lambda: L.attend_run(rp.int(), q, k, k), lambda: L.attend_run(rp, q[:1], k, k), lambda: L.attend_run(rp, q, k, k[:3]), lambda: L.attend_run(rp, q.half(), k.half(), k.half()),
                 lambda: L.attend_run(rp, q, k.bfloat16(), k), lambda: L.attend_run(rp, q, k.transpose(1, 2), k), lambda: L.attend_run(rp, q, torch.zeros((2, 4, 8), device="cuda").transpose(0, 1), k),
                 lambda: L.attend_run(rp, q, k, k, edges=edges), lambda: L.attend_run(rp, q, k, k, table=table), lambda: L.attend_run(rp, q, k, k, table=table, edges=edges[:1]),
                 lambda: L.attend_run(rp, q, k, k, table=table[:, :1], edges=edges), lambda: L.attend_run(rp, q, k, k, mask=x[:, 0]), lambda: L.attend_run(rp, q, k, k, index=rp),
                 lambda: L.attend_run(rp, q, k, k.cpu()), lambda: L.attend_grad(rp, q, k, k, None, q), lambda: L.attend_grad(rp, q, k, k, torch.zeros(4, dtype=torch.uint8, device="cuda"), q),
                 lambda: L.attend_grad(rp, q, k, k, L.attend_run(rp, q, k, k, save=True)["saved"], q[:1]), lambda: L.block_run(x, x[:3]), lambda: L.block_run(x, x.bfloat16()),
                 lambda: L.block_run(x, x, post=w[:7]), lambda: L.block_run(x.t(), x.t()), lambda: L.block_grad(x, x, dout=x[:, :7]), lambda: L.distill(x, ids.long(), ids.float()),
                 lambda: L.distill(x, ids, ids.float()[:3]), lambda: L.distill(x.half(), ids, ids.float()), lambda: L.distill(x, ids, ids.float(), weight=w), lambda: L.distill(x.t(), ids, ids.float())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: L.attend_run(rp, q, k, k, t=edges), lambda: L.attend_run(rp, q, k[:1].expand(4, 2, 8), k), lambda: L.block_run(x[:1].expand(4, 8), x),
                 lambda: L.block_grad(x, x, dout=x, dnext=x), lambda: L.distill(x, ids, ids.float(), temperature=0.0), lambda: L.distill(x[:1].expand(4, 8), ids, ids.float())):
        with pytest.raises(TnsError):
            call()


def test_within_autograd(L):
    """Functions of the caller's around the operators, one behind the other: attention, block, scores, distillation."""
    import torch
    rng = np.random.default_rng(20)
    a = the_events(rng, [5, 0, 9, 70], 2, 2, 8, F32, buckets=4)
    g = on_gpu(a, F32)

    class Attend(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, table):
            r = L.attend_run(g["rowptr"], q, k, v, t=g["t"], ts=g["ts"], edges=g["edges"], table=table, newest_first=True, save=True)
            ctx.save_for_backward(q, k, v, table, r["saved"])
            return r["out"]

        @staticmethod
        def backward(ctx, dout):
            q, k, v, table, saved = ctx.saved_tensors
            d = L.attend_grad(g["rowptr"], q, k, v, saved, dout.contiguous(), t=g["t"], ts=g["ts"], edges=g["edges"], table=table, newest_first=True)
            return d["dq"], d["dk"], d["dv"], d["dtable"]

    class Block(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, branch, pre):
            ctx.save_for_backward(x, branch, pre)
            r = L.block_run(x, branch, pre=pre)
            return r["out"], r["next"]

        @staticmethod
        def backward(ctx, dout, dnext):
            x, branch, pre = ctx.saved_tensors
            d = L.block_grad(x, branch, dout=dout.contiguous(), dnext=dnext.contiguous(), pre=pre)
            return d["dx"], d["dbranch"], d["dpre"]

    class Distill(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, ids, teacher):
            r = L.distill(logits, ids, teacher)
            ctx.save_for_backward(r["dlogits"])
            return r["loss"]

        @staticmethod
        def backward(ctx, d):
            return ctx.saved_tensors[0] * d, None, None

    x, pre, nodes = values(rng, (4, 16), F32), values(rng, 16, F32), values(rng, (16, 30), F32)
    ids, teacher = torch_of(rng.integers(0, 30, (4, 5)).astype(np.int32)), torch_of(values(rng, (4, 5), F32))

    def loss_of(leaves, attend, block, distill):
        q, k, v, table, x, pre = leaves
        out, following = block(x, attend(q, k, v, table).reshape(4, 16), pre)
        return distill(following @ torch_of(nodes).to(q.dtype), ids, teacher) + out.square().sum()

    given = [torch_of(v) for v in (a["q"], a["k"], a["v"], a["table"], x, pre)]
    mine = [v.clone().requires_grad_() for v in given]
    loss = loss_of(mine, Attend.apply, Block.apply, Distill.apply)
    loss.backward()

    def plain_attend(q, k, v, table):
        outs = []
        for s in range(4):
            lo, hi = a["rowptr"][s], a["rowptr"][s + 1]
            age = (g["t"][s] - g["ts"][lo:hi]).clamp(min=0)
            score = torch.einsum("hd,nhd->nh", q[s], k[lo:hi]) * 8 ** -0.5 + table[torch.searchsorted(g["edges"], age, right=True)]
            outs.append((torch.softmax(score, 0)[:, :, None] * v[lo:hi]).sum(0))
        return torch.stack(outs)

    def plain_block(x, branch, pre):
        out = x + branch
        return out, pre * out / torch.sqrt(out.square().mean(1, keepdim=True) + 1e-6)

    def plain_distill(logits, ids, teacher):
        p = torch.softmax(teacher.double(), 1)
        return (p * (torch.log(p) - torch.log_softmax(logits, 1).gather(1, ids.long()))).sum()

    exact = [v.double().requires_grad_() for v in given]
    want = loss_of(exact, plain_attend, plain_block, plain_distill)
    want.backward()
    # chains of some hundred roundings of values around 1 (rows of 30 scores around 4, a gradient of their size): 2^-24 of 1e3 each
    assert abs(float(loss) - float(want)) < 1e3 * 2 ** -24 * float(want)
    for m, w in zip(mine, exact):
        assert float((m.grad.double() - w.grad).abs().max()) < 1e3 * 2 ** -24 * float(w.grad.abs().max())
    with pytest.raises(ValueError, match="autograd"):
        L.block_run(mine[4], mine[4])


# ---- many lists ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype, heads, kv_heads, dim, lists", [(F32, 1, 1, 256, 2500), (F32, 2, 2, 50, 4200), (BF16, 2, 2, 64, 8300), (BF16, 3, 3, 40, 4200), (F32, 4, 2, 7, 8300), (BF16, 8, 1, 60, 16500),
                                                                (F32, 1, 1, 15, 33000), (BF16, 40, 20, 32, 1100)])
@pytest.mark.parametrize("times, newest_first", [(True, True), (False, False)])
def test_attend_many_lists(L, dtype, heads, kv_heads, dim, lists, times, newest_first):
    """So many lists that brief ones are taken several a wave: some empty, some of 63 to 66 events, some far longer, the last wave's not full."""
    rng = np.random.default_rng(lists + heads)
    lens = np.minimum(rng.geometric(0.15, lists) - 1, 12)
    lens[rng.integers(0, lists, 12)] = [63, 64, 65, 66, 100, 300, 700, 31, 32, 33, 17, 16]
    lens[-1] = 40
    a = the_events(rng, lens, heads, kv_heads, dim, dtype, buckets=5, times=times, masked=0.2, newest_first=newest_first)
    check_attend(L, a, dtype)


@pytest.mark.parametrize("dtype, dim, lists", [(F32, 64, 4200), (BF16, 50, 8300)])
def test_attend_many_lists_gathered(L, dtype, dim, lists):
    rng = np.random.default_rng(lists)
    lens = np.minimum(rng.geometric(0.15, lists) - 1, 12)
    lens[rng.integers(0, lists, 4)] = [64, 65, 500, 33]
    a = the_events(rng, lens, 2, 2, dim, dtype, masked=0.1)
    n, nodes = int(a["rowptr"][-1]), 300
    a["index"] = rng.integers(-20, nodes + 20, n).astype(np.int32)
    a["k"], a["v"] = values(rng, (nodes, 2, dim), dtype), values(rng, (nodes, 2, dim), dtype)
    want = O.attend(**a)
    close("out", L.attend_run(**on_gpu(a, dtype))["out"], want["out"], want["out_off"], dtype)


def test_attend_many_lists_ruled_out_buckets_and_rows_beyond(L):
    """Brief lists several a wave: buckets that are ruled out for some heads of a group, rows that no list holds, the same bits again."""
    import torch
    rng = np.random.default_rng(31)
    lens = np.minimum(rng.geometric(0.2, 9000) - 1, 12)
    a = the_events(rng, lens, 4, 2, 16, F32, buckets=4, times=False)
    a["edges"] = np.float32([1, 2, 5])
    a["table"][0, 1] = a["table"][2, 2] = a["table"][3] = -np.inf
    dout = values(rng, a["q"].shape, F32)
    r, d = check_attend(L, a, F32, dout)
    g = on_gpu(a, F32)
    n = int(a["rowptr"][-1])
    for name in ("k", "v"):
        g[name] = torch.cat((g[name], torch.full((777, 2, 16), float("nan"), device="cuda")))
    again = L.attend_run(**g, save=True)
    assert torch.equal(again["out"], r["out"])
    back = L.attend_grad(**g, saved=again["saved"], dout=torch_of(dout))
    for name in ("dk", "dv"):
        assert torch.equal(back[name][:n], d[name]) and not back[name][n:].any()
    assert torch.equal(back["dq"], d["dq"])


def test_attend_rows_without_lists(L):
    """No list at all, and rows all the same: their gradients are zeros, the table's too."""
    import torch
    k = torch.full((200, 2, 8), float("nan"), device="cuda")
    q = torch.empty((0, 4, 8), device="cuda")
    table, edges = torch.ones((3, 4), device="cuda"), torch.tensor([1.0, 2.0], device="cuda")
    rp = torch.zeros(1, dtype=torch.int64, device="cuda")
    r = L.attend_run(rp, q, k, k, table=table, edges=edges, save=True)
    d = L.attend_grad(rp, q, k, k, r["saved"], q, table=table, edges=edges)
    assert r["out"].shape == q.shape and not d["dk"].any() and not d["dv"].any() and not d["dtable"].any()
    desc = L.tns_attend(0, 200, 0, 4, 2, 8, 0, 3, L.TNS_ZERO_BEYOND, None, None, k.data_ptr(), k.data_ptr(), 32, 16, 16, None, None, None, None, edges.data_ptr(), table.data_ptr(), 1.0)
    need = L.tns_attend_workspace(desc)[1]
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    d["dk"].fill_(1)
    L.tns_attend_grad(desc, 0, 0, 0, d["dk"].data_ptr(), d["dv"].data_ptr(), d["dtable"].data_ptr(), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert not d["dk"].any()


def test_first_calls_within_a_capture(L):
    """Kernels that have not run before in this process (sizes that no other test has) may be captured."""
    import torch
    rng = np.random.default_rng(40)
    a = the_events(rng, [9, 0, 70], 8, 1, 68, BF16, buckets=3)
    g, dout = on_gpu(a, BF16), torch_of(values(rng, a["q"].shape, BF16), BF16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = L.attend_run(**g, save=True)
        d = L.attend_grad(**g, saved=r["saved"], dout=dout)
    want = O.attend(**a, dout=dout.float().cpu().numpy())
    for _ in range(2):
        r["out"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        close("out", r["out"], want["out"], want["out_off"], BF16)
        for name in ("dq", "dk", "dv"):
            close(name, d[name], want[name], want[name + "_off"], BF16)
        close("dtable", d["dtable"], want["dtable"], want["dtable_off"])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_infinite_keys(L, dtype):
    """A key of minus infinity against a positive query: the event's score is minus infinity and its p zero, at whole and at odd head sizes."""
    rng = np.random.default_rng(41)
    for dim in (8, 13, 43, 64):
        a = the_events(rng, [5, 40], 2, 2, dim, dtype, buckets=0, times=False)
        a["q"][:, :, 0] = np.abs(a["q"][:, :, 0]) + 0.5
        g = on_gpu(a, dtype)
        a["q"] = g["q"].float().cpu().numpy()      # (as the type holds them)
        g["k"][2, :, 0] = -float("inf")
        g["k"][30, 1, 0] = -float("inf")
        got = L.attend_run(**g)["out"]
        assert bool(got.isfinite().all())
        # the same with these events left out
        a["k"][2, :, 0] = -1e4
        a["k"][30, 1, 0] = -1e4
        want = O.attend(**a)
        # p of exp(-5000 and less) is 0 in the oracle too
        close("out", got, want["out"], want["out_off"], dtype)


@pytest.mark.parametrize("dtype, kv_heads, dim, skip", [(F32, 1, 3, 1), (F32, 2, 16, 0), (BF16, 1, 7, 1), (BF16, 3, 5, 6), (BF16, 2, 32, 3)])
@pytest.mark.parametrize("rows, beyond", [(0, 1), (5, 700), (130, 63), (64, 64)])
def test_attend_zeros_beyond_at_any_address(L, rows, beyond, dtype, kv_heads, dim, skip):
    """Rows beyond the lists become zeros, and nothing beside them: at every address that the type allows."""
    import torch
    rng = np.random.default_rng(rows + dim)
    a = the_events(rng, [rows], kv_heads, kv_heads, dim, dtype, buckets=0, times=False)
    g = on_gpu(a, dtype)
    for name in ("k", "v"):
        g[name] = torch.cat((g[name], torch.full((beyond, kv_heads, dim), float("nan"), dtype=g[name].dtype, device="cuda")))
    r = L.attend_run(**g, save=True)
    dout = torch_of(values(rng, a["q"].shape, dtype), dtype)
    want = O.attend(**a, dout=dout.float().cpu().numpy())
    desc = L._described(g["rowptr"], g["q"], g["k"], g["v"], None, None, None, None, None, None, None, True)
    need, size, n = L.tns_attend_workspace(desc)[1], kv_heads * dim, rows + beyond
    out = [torch.full((n * size + skip + 9,), 7.0, dtype=dout.dtype, device="cuda") for _ in range(2)]
    dq, ws = torch.empty_like(g["q"]), torch.empty(need, dtype=torch.uint8, device="cuda")
    at = skip * dout.element_size()
    L.tns_attend_grad(desc, r["saved"].data_ptr(), dout.data_ptr(), dq.data_ptr(), out[0].data_ptr() + at, out[1].data_ptr() + at, 0, ws.data_ptr(), need,
                      torch.cuda.current_stream().cuda_stream)
    for name, got in zip(("dk", "dv"), out):
        assert bool((got[:skip] == 7).all()) and bool((got[skip + n * size:] == 7).all()) and not got[skip + rows * size: skip + n * size].any()
        close(name, got[skip: skip + rows * size].view(rows, kv_heads, dim), want[name], want[name + "_off"], dtype)
