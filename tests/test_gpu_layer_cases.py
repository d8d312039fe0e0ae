"""Calls of the layer operators at the ends of what their header allows, on the GPU against the oracle in 64 bits.  Tolerances as in test_gpu_layer.py."""
import numpy as np
import pytest

from oracle import layer_oracle as O
from test_gpu_layer import L, check_block, check_distill, on_gpu, the_block, the_events, the_scores      # noqa: F401
from test_gpu_train import BF16, F32, close, torch_of, values

pytestmark = pytest.mark.gpu


# ---- attention: lists of many parts, wherever they begin -------------------------------------------

def into_nan(L, a, g, dout, dtype):
    """Outputs and gradients through the C functions, written over NaN: what no kernel writes shows."""
    import torch
    desc = L._described(g["rowptr"], g["q"], g["k"], g["v"], g.get("t"), g.get("ts"), g.get("edges"), g.get("table"), None, g.get("mask"), None, a["newest_first"])
    run, grad, saved_bytes = L.tns_attend_workspace(desc)
    saved, ws = (torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (saved_bytes, max(run, grad)))
    nan = lambda t: torch.full_like(t, float("nan"))              # noqa: E731
    out = dict(out=nan(g["q"]), dq=nan(g["q"]), dk=nan(g["k"]), dv=nan(g["v"]))
    dtable = nan(g["table"]) if "table" in g else None
    stream = torch.cuda.current_stream().cuda_stream
    L.tns_attend_run(desc, out["out"].data_ptr(), saved.data_ptr(), ws.data_ptr(), ws.numel(), stream)
    ws.fill_(255)
    L.tns_attend_grad(desc, saved.data_ptr(), dout.data_ptr(), out["dq"].data_ptr(), out["dk"].data_ptr(), out["dv"].data_ptr(), 0 if dtable is None else dtable.data_ptr(),
                      ws.data_ptr(), ws.numel(), stream)
    want = O.attend(**a, dout=dout.float().cpu().numpy())
    for name, got in out.items():
        close(name, got, want[name], want[name + "_off"], dtype)
    if dtable is not None:
        close("dtable", dtable, want["dtable"], want["dtable_off"])


# (blocks have 16 rows up to 32768 rows of one turn, 32 up to 65536, then 64; every list here but the last has more than 256 parts)
MANY = {"five before 4097": [5, 4097], "one before 5000": [1, 5000], "five before 100000": [5, 100000], "one before 200000": [1, 200000],
        "in block 256": [4099, 6000], "at the end of block 255": [4095, 4500, 30], "at block 256": [4096, 4500, 30], "two": [3, 120000, 120000], "behind short ones": [7, 0, 300, 2, 70000, 1, 0, 90000, 64]}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads, kv_heads, dim, buckets", [(1, 1, 4, 0), (4, 2, 20, 5)])
@pytest.mark.parametrize("lens", list(MANY), ids=[k.replace(" ", "_") for k in MANY])
def test_attend_lists_of_many_parts_wherever_they_begin(L, lens, heads, kv_heads, dim, buckets, dtype):      # noqa: F811
    rng = np.random.default_rng(len(lens) + heads)
    a = the_events(rng, MANY[lens], heads, kv_heads, dim, dtype, buckets, times=buckets > 0)
    into_nan(L, a, on_gpu(a, dtype), torch_of(values(rng, a["q"].shape, dtype), dtype), dtype)


def test_attend_long_lists_in_blocks_of_512_rows(L):      # noqa: F811
    """Zeros give zeros: every output and gradient of lists that begin in the first block and go on beyond 256 blocks."""
    import torch
    lens = [10, 2_100_000, 0, 300, 2_200_000]
    rowptr = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)])).cuda()
    rows = sum(lens)
    zeros = lambda n: torch.zeros((n, 1, 4), device="cuda")       # noqa: E731
    q, k, v, dout = zeros(len(lens)), zeros(rows), zeros(rows), zeros(len(lens))
    desc = L._described(rowptr, q, k, v, None, None, None, None, None, None, None, True)
    run, grad, saved_bytes = L.tns_attend_workspace(desc)
    saved, ws = (torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (saved_bytes, max(run, grad)))
    out = [torch.full_like(t, float("nan")) for t in (q, q, k, v)]
    stream = torch.cuda.current_stream().cuda_stream
    L.tns_attend_run(desc, out[0].data_ptr(), saved.data_ptr(), ws.data_ptr(), ws.numel(), stream)
    L.tns_attend_grad(desc, saved.data_ptr(), dout.data_ptr(), *[t.data_ptr() for t in out[1:]], 0, ws.data_ptr(), ws.numel(), stream)
    for t in out:
        assert not t.any()                                        # (a NaN is true)


# ---- attention: table entries at the ends of fp32 --------------------------------------------------

LOWEST, LARGEST = float(np.finfo(np.float32).min), float(np.finfo(np.float32).max)
BF16_LOWEST = -float.fromhex("0x1.fep127")


def the_ends(rng, dtype, many, gathered=False):
    """Lists whose events have, by place, table entries of two ends of fp32; equal queries, so that the events of the higher entry have equal p."""
    lens = np.array([1, 30, 0, 700, 6000, 64, 2] + [5, 0, 12, 1, 9] * (1700 if many else 3))
    a = the_events(rng, lens, 2, 2, 16, dtype, buckets=2, times=False)
    a["edges"] = np.float32([3])                                  # three events of the first bucket, the others in the second
    a["q"][:] = 0
    if gathered:
        a["index"] = rng.permutation(int(a["rowptr"][-1])).astype(np.int32)
    return a, lens


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("many, gathered", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("first, second", [(LOWEST, LOWEST), (LOWEST, 0.0), (0.0, LOWEST), (LOWEST, -3e38), (LOWEST, BF16_LOWEST), (-2.4e38, -2.5e38), (-2.3e38, -2.4e38), (LARGEST, LARGEST), (LARGEST, 3e38),
                                           (1.0, LARGEST), (LOWEST, LARGEST), (-1e30, LOWEST), (LOWEST, float("-inf")), (float("-inf"), LARGEST), (-8.5e37, -8.6e37), (2.0 ** 126, 2.0 ** 126 * (1 - 2.0 ** -20))])
def test_attend_table_entries_at_the_ends(L, first, second, many, gathered, dtype):      # noqa: F811
    """The lowest finite number of a type is a number: events of nothing else have equal parts, and beside a higher one no part.  Only -infinity leaves out."""
    rng = np.random.default_rng(60)
    a, lens = the_ends(rng, dtype, many, gathered)
    a["table"] = np.float32([[first, first], [second, second]])
    out = L.attend_run(**on_gpu(a, dtype))["out"].float().cpu().numpy()
    v = a["v"].astype(np.float64) if not gathered else a["v"][a["index"]].astype(np.float64)
    for s in range(len(lens)):
        rows = v[a["rowptr"][s]: a["rowptr"][s + 1]]
        parts = [(entry, of) for entry, of in ((first, rows[:3]), (second, rows[3:])) if len(of) and entry != -np.inf]
        if not parts:
            assert not out[s].any()
            continue
        top = max(entry for entry, _ in parts)
        rows = np.concatenate([of for entry, of in parts if entry == top])
        mean = rows.mean(0)
        # every p is 1 before the sum and the sum a whole number; at most 128 additions one after the other (a slot takes 64 events, the joins the rest), a
        # reciprocal and a product
        off = (128 + 4) * 2.0 ** -24 * np.abs(rows).mean(0) + (2.0 ** -8 * np.abs(mean) if dtype == BF16 else 0)
        assert (np.abs(out[s] - mean) <= off).all(), s


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("entry", [100.0, -1e4, 1e4, -1e9, 1e9, -1e30, LOWEST, LARGEST])
def test_attend_gradients_of_lists_in_one_far_bucket(L, entry, many, dtype):      # noqa: F811
    """The softmax does not change where all scores have the same summand, and so do the gradients: those without a bias, whatever the entry."""
    rng = np.random.default_rng(61)
    a, lens = the_ends(rng, dtype, many)
    a["table"] = np.full((2, 2), entry, np.float32)
    dout = values(rng, a["q"].shape, dtype)
    want = O.attend(**dict(a, table=np.zeros((2, 2), np.float32)), dout=dout)      # (the queries are zero: the entry is the score, exactly)
    g = on_gpu(a, dtype)
    r = L.attend_run(**g, save=True)
    d = L.attend_grad(**g, saved=r["saved"], dout=torch_of(dout, dtype))
    for name, got in dict(d, out=r["out"]).items():
        close(name, got, want[name], want[name + "_off"], F32 if name == "dtable" else dtype)


@pytest.mark.parametrize("newest_first", [True, False])
def test_attend_places_beyond_24_bits(L, newest_first):      # noqa: F811
    """An event with 2^24 + 3 newer ones lies below the border 2^24 + 4, which fp32 holds and rounds the place to; the next one on it."""
    import torch
    n, border = (1 << 24) + 64, (1 << 24) + 4
    v = torch.zeros((n, 1, 1), device="cuda")
    q, rowptr, edges = torch.zeros((1, 1, 1), device="cuda"), torch.tensor([0, n], device="cuda"), torch.tensor([float(border)], device="cuda")
    row = lambda place: place if newest_first else n - 1 - place      # noqa: E731
    for place, counts in ((border - 2, True), (border - 1, True), (border, False), (border + 1, False), (n - 1, False)):
        mask = torch.zeros(n, dtype=torch.bool, device="cuda")
        mask[row(place)] = True
        v[row(place)] = 3.0
        r = L.attend_run(rowptr, q, v, v, edges=edges, table=torch.tensor([[0.0], [float("-inf")]], device="cuda"), mask=mask, newest_first=newest_first)
        assert float(r["out"]) == (3.0 if counts else 0.0), place
        v[row(place)] = 0.0


def test_attend_a_batch_without_events_from_a_table(L):      # noqa: F811
    """Targets that have no event at all, keys and values in a table of nodes: zeros."""
    import torch
    k, q, none = torch.full((50, 2, 8), float("nan"), device="cuda"), torch.ones((3, 4, 8), device="cuda"), torch.empty(0, device="cuda")
    rowptr, index, t = torch.zeros(4, dtype=torch.int64, device="cuda"), none.int(), torch.ones(3, device="cuda")
    table, edges = torch.ones((3, 4), device="cuda"), torch.tensor([1.0, 2.0], device="cuda")
    assert not L.attend_run(rowptr, q, k, k, index=index)["out"].any()
    assert not L.attend_run(rowptr, q, k, k, t=t, ts=none, edges=edges, table=table, index=index, mask=none.bool())["out"].any()
    assert L.attend_run(rowptr[:1], q[:0], k, k, index=index)["out"].shape == (0, 4, 8)


# ---- distillation: named candidates far above the others --------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [4, 50, 600, 3001, 9000, 40000])
@pytest.mark.parametrize("lead", [60.0, 90.0, 100.0, 128.0, 300.0, 1000.0, 4096.0])
def test_distill_named_far_above_the_others(L, lead, n, dtype):      # noqa: F811
    """A student that is sure of named candidates: the others' mass is compared in the logarithm, and their gradients stay numbers.  Of the named, one
    leads (rows 0, 1), all do (2), or the last of the row alone is unnamed and far below (3); an unnamed one leads in row 4."""
    rng = np.random.default_rng(n + int(lead))
    K = min(n - 1, 12)
    a = the_scores(rng, 5, n, K, dtype, True)
    for b in range(5):
        a["ids"][b] = rng.permutation(n - 1)[:K]
    for b in (0, 1):
        a["logits"][b, a["ids"][b, 0]] += lead
    a["logits"][2, a["ids"][2]] += lead
    a["logits"][3, n - 1] -= lead
    a["logits"][4, n - 1] += lead
    if dtype == BF16:
        a["logits"] = torch_of(a["logits"], BF16).float().cpu().numpy()
    check_distill(L, a, dtype, temperature=1.0)
    check_distill(L, a, dtype, temperature=0.5)
    for temperature in (1.0, 0.5):
        r = L.distill(**{k: torch_of(v, dtype if k == "logits" else None) for k, v in a.items()}, temperature=temperature)
        assert bool(r["rows"].isfinite().all()) and bool(r["dlogits"].isfinite().all())


def test_distill_a_sure_student_in_numbers(L):      # noqa: F811
    import torch
    logits = torch.tensor([[100.0, 0.0, 0.5, -1.0]], device="cuda")
    r = L.distill(logits, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([[0.7]], device="cuda").log(), lse=torch.zeros(1, device="cuda"))
    e = np.exp([0.0, 0.5, -1.0])
    # 0.7 log 0.7 + 0.3 (log 0.3 - log(1 + exp 0.5 + exp -1) + 100); the scores' difference and the logarithm are some ten roundings of values up to 100
    assert abs(float(r["loss"]) - (0.7 * np.log(0.7) + 0.3 * (np.log(0.3) - np.log(e.sum()) + 100))) < 10 * 2 ** -24 * 100
    assert np.allclose(r["dlogits"].cpu().numpy()[0], np.concatenate([[0.3], -0.3 * e / e.sum()]), rtol=0, atol=20 * 2 ** -24)


def test_distill_others_that_are_all_ruled_out(L):      # noqa: F811
    """Mass of others whose scores are all -infinity: an infinite loss as the header says, and no gradient by them."""
    import torch
    inf = float("inf")
    ids, teacher = torch.tensor([[0, 2]], dtype=torch.int32, device="cuda"), torch.tensor([[0.4, 0.4]], device="cuda").log()
    for n in (4, 40000):
        logits = torch.full((1, n), -inf, device="cuda")
        logits[0, 0], logits[0, 2] = 1.0, -3.0
        r = L.distill(logits, ids, teacher, lse=torch.zeros(1, device="cuda"))
        assert float(r["rows"][0]) == inf and not r["dlogits"][0, 3:].any() and bool(r["dlogits"].isfinite().all())


@pytest.mark.parametrize("dtype, n", [(F32, 1500), (F32, 9000), (BF16, 5000), (BF16, 20000), (F32, 40000), (BF16, 70000)])
def test_distill_same_bits_in_every_row_where_ids_come_twice(L, dtype, n):      # noqa: F811
    """Two thousand rows that are the same one: candidates that threads of different waves name come to the same sum, whichever thread is first."""
    import torch
    rng = np.random.default_rng(n)
    a = the_scores(rng, 1, n, 1024, dtype, True)
    for k in range(0, 1024, 128):
        a["ids"][0, k + 64: k + 128] = a["ids"][0, k: k + 64][::-1]      # twice, in the next wave
    a["ids"][0, 1000:] = a["ids"][0, 100:124]                     # and more often
    a["logits"][0, a["ids"][0]] += values(rng, 1024, dtype, 2.0)
    a["lse"][0] = np.log(np.exp(a["teacher"].astype(np.float64)).sum()) + 0.5
    g = {k: None if v is None else torch_of(np.repeat(v, 2000, 0), dtype if k == "logits" else None) for k, v in a.items()}
    r = L.distill(**g)
    assert bool((r["rows"] == r["rows"][0]).all()) and bool((r["dlogits"] == r["dlogits"][0]).all())
    a["logits"] = g["logits"][:1].float().cpu().numpy()
    check_distill(L, a, dtype, temperature=1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [40, 3000, 40000])
@pytest.mark.parametrize("temperature", [0.25, 1.0, 2.0])
def test_distill_teachers_far_from_zero(L, temperature, n, dtype):      # noqa: F811
    """The teacher's softmax does not change where all its scores have the same summand: far ones, and lists of nothing but a type's lowest or largest number."""
    rng = np.random.default_rng(n)
    a = the_scores(rng, 9, n, 10, dtype)
    a["teacher"][:7] = np.round(a["teacher"][:7] * 4) / 4         # (whole quarters, which the sums below hold)
    want = dict(a, teacher=a["teacher"].copy())
    for b, far in enumerate((1e4, -1e4, 2.0 ** 21, -(2.0 ** 21))):
        a["teacher"][b] += far
    a["teacher"][4], a["teacher"][5], a["teacher"][6] = -1e9, LOWEST, LARGEST
    want["teacher"][4:7] = 0
    a["teacher"][7, 3:] = LOWEST                                  # beside ordinary ones the lowest number has no part
    want["teacher"][7, 3:] = -np.inf
    want = O.distill(**want, temperature=temperature)
    r = L.distill(**{k: torch_of(v, dtype if k == "logits" else None) for k, v in a.items()}, temperature=temperature)
    close("rows", r["rows"], want["rows"], want["rows_off"])
    close("dlogits", r["dlogits"], want["dlogits"], want["dlogits_off"], dtype)


# ---- between two layers: values far from 1 ---------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [2.0 ** 54, 2.0 ** -54])
@pytest.mark.parametrize("without", [(), ("post",)])
@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("dim", [20, 8192])
def test_block_values_far_from_one(L, dim, center, without, size, dtype):      # noqa: F811
    """Rows of the sizes that the header names, without eps."""
    rng = np.random.default_rng(dim)
    a = the_block(rng, 6, dim, dtype, **dict.fromkeys(without))
    a["x"] *= np.float32(size)
    a["branch"] *= np.float32(size)
    check_block(L, a, dtype, values(rng, (6, dim), dtype), values(rng, (6, dim), dtype), center=center, eps=0.0)
