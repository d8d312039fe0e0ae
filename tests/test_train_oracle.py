"""The oracle of the training operators against closed forms, differences and counts; the interface and its refusals.  No GPU."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import train_oracle as O
from paper_2311_17410_amd import binding as B
from paper_2311_17410_amd import train_binding as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def lists(rng, lens, dim, decay=True, h0=True):
    rp = np.concatenate([[0], np.cumsum(lens)])
    n, S = int(rp[-1]), len(lens)
    a = dict(rowptr=rp, u=rng.normal(size=(n, dim)), x=rng.normal(size=(n, dim)))
    if decay:
        a.update(ts=rng.uniform(0, 3, n).astype(np.float32), decay=rng.uniform(0, 1, dim))
    if h0:
        a.update(h0=rng.normal(size=(S, dim)))
        if decay:
            a.update(t0=np.zeros(S, np.float32))
    return a


def test_recurrence_closed_forms():
    """Gates of one value: a geometric sum; one event: z x; gates shut: the state stays; wide open: the newest value."""
    n = 7
    q = 1 / (1 + np.exp(-0.3))
    r = O.recurrence([0, n], np.full((n, 1), 0.3), np.ones((n, 1)))
    assert np.allclose(r["h"][:, 0], 1 - (1 - q) ** np.arange(1, n + 1), rtol=1e-14)
    assert np.allclose(O.recurrence([0, 1], np.full((1, 1), 0.3), np.full((1, 1), 2.0))["last"], 2 * q)
    h0 = np.full((1, 1), 5.0)
    assert np.allclose(O.recurrence([0, n], np.full((n, 1), -800.0), np.ones((n, 1)), h0=h0)["last"], 5.0)
    assert np.allclose(O.recurrence([0, n], np.full((n, 1), 800.0), np.arange(n)[:, None], h0=h0)["last"], n - 1)
    # newest first is the same list turned round; a list without events keeps its state
    rng = np.random.default_rng(0)
    a = lists(rng, [4], 3)
    b = dict(a, u=a["u"][::-1], x=a["x"][::-1], ts=a["ts"][::-1])
    assert np.allclose(O.recurrence(**a)["h"], O.recurrence(**b, newest_first=True)["h"][::-1])
    assert np.array_equal(O.recurrence([0, 0], np.zeros((0, 1)), np.zeros((0, 1)), h0=h0)["last"], h0)
    # decay alone: exp(-lambda t)
    shut = np.full((2, 1), -800.0)
    r = O.recurrence([0, 2], shut, shut, ts=np.float32([1, 3]), decay=np.array([0.5]), h0=h0, t0=np.float32([0]))
    assert np.allclose(r["last"], 5 * np.exp(-1.5))


def test_gap():
    assert O.gap_of(3, 1) == 2 and O.gap_of(1, 3) == 0 and O.gap_of(np.nan, 0) == 0 and O.gap_of(np.inf, np.inf) == 0
    assert O.gap_of(np.inf, 0) == float(np.finfo(np.float32).max)


@pytest.mark.parametrize("newest_first", [False, True])
def test_recurrence_gradients_against_differences(newest_first):
    rng = np.random.default_rng(1)
    a = lists(rng, [3, 0, 1, 5], 2)
    n = len(a["u"])
    dh, dlast = rng.normal(size=(n, 2)), rng.normal(size=(4, 2))

    def scalar(b):
        r = O.recurrence(**b, newest_first=newest_first)
        return (r["h"] * dh).sum() + (r["last"] * dlast).sum()

    got = O.recurrence(**a, newest_first=newest_first, dh=dh, dlast=dlast)
    for name in ("u", "x", "decay", "h0"):
        d = np.zeros_like(a[name])
        for i in np.ndindex(d.shape):
            up, down = a[name].copy(), a[name].copy()
            up[i] += 1e-6
            down[i] -= 1e-6
            d[i] = (scalar(dict(a, **{name: up})) - scalar(dict(a, **{name: down}))) / 2e-6
        assert np.allclose(got["d" + name], d, rtol=1e-6, atol=1e-8), name


def test_pair_loss_closed_forms_and_differences():
    rng = np.random.default_rng(2)
    one = np.zeros((3, 2, 4))
    assert np.isclose(O.pair_loss(one[:, 0], one[:, 0], one)["loss"], 6 * np.log(2))
    a, p, n, r = rng.normal(size=(3, 4)), rng.normal(size=(3, 4)), rng.normal(size=(3, 2, 4)), rng.normal(size=(3, 2))
    w = np.array([[1.0, 0], [0, 0], [2, 0.5]])
    n[w == 0] = np.nan
    kw = dict(ref=r, weight=w, beta=0.75, smoothing=0.125, scale=0.5)
    got = O.pair_loss(a, p, n, **kw)
    assert not got["danchor"][1].any() and not got["dpos"][1].any() and not got["dneg"][w == 0].any() and np.isfinite(got["loss"])
    for name, i in (("danchor", 0), ("dpos", 1), ("dneg", 2)):
        v = [a, p, n]
        d = np.zeros_like(v[i])
        for at in np.ndindex(d.shape):
            loss = []
            for by in (1e-6, -1e-6):
                moved = list(v)
                moved[i] = v[i].copy()
                moved[i][at] += by
                loss.append(O.pair_loss(*moved, **kw)["loss"])
            d[at] = (loss[0] - loss[1]) / 2e-6
        assert np.allclose(got[name], d, rtol=1e-6, atol=1e-9), name


def test_adamw_first_step_and_codes():
    """After one step from zero the change is lr times the sign of the gradient; splitmix64's published outputs; e4m3's extremes."""
    g = np.float32([0.5, -2, 1e-3])
    new, _, st = O.adamw(np.zeros(3, np.float32), g, dict(m=np.zeros(3, np.float32), v=np.zeros(3, np.float32)), 1, weight_decay=0.0)
    assert np.allclose(new, -1e-3 * np.sign(g), rtol=1e-4)
    with np.errstate(over="ignore"):
        assert int(O.mix64(np.uint64((1234567 + O.GOLDEN) & O.MASK))) == 6457827717110365317      # first output for seed 1234567
    assert O.e4m3_value(0x7E) == 448 and O.e4m3_value(0x08) == 2.0 ** -6 and O.e4m3_value(0x81) == -(2.0 ** -9) and np.isnan(O.e4m3_value(0x7F))


def test_rounding_to_codes_is_right_on_average():
    """256 values, 4000 roundings: each mean within six standard errors of the value (a code is off by a sixteenth to an eighth at most)."""
    rng = np.random.default_rng(3)
    v = np.float32(rng.uniform(0.02, 1, 256) * rng.choice([-1, 1], 256))
    total = np.zeros(256)
    for t in range(4000):
        codes, scales = O.to_codes(v, True, O.random16(9, t + 1, 0, 256))
        total += O.e4m3_value(codes) * np.float64(scales[0])
    step = np.abs(v) / 8
    assert (np.abs(total / 4000 - v) < 6 * step / 2 / np.sqrt(4000) + 2.0 ** -16 * step).all()


def test_small_values_of_a_state():
    v = np.float32([1, 1e-6, 0] + [0.5] * 253)
    m, ms = O.to_codes(v, True, np.zeros(256, np.int64))
    r, rs = O.to_codes(v, False, np.zeros(256, np.int64))
    assert m[1] == m[2] == 0 and r[1] == r[2] == 8 and ms[0] == rs[0] == np.float32(1) * np.float32(1 / 448)
    m, ms = O.to_codes(np.zeros(300, np.float32), False, np.zeros(300, np.int64))
    assert not m.any() and not ms.any()


# ---- interface -----------------------------------------------------------------------------------

def test_every_declared_symbol_is_exported_and_bound():
    hdr = open(os.path.join(ROOT, "include", "tns_train.h")).read()
    declared = re.findall(r"TNS_API\s+[\w\s\*]+?\b(tns_\w+)\s*\(", hdr)
    assert sorted(declared) == sorted(T.EXPORTS)
    L = ctypes.CDLL(B.LIB_PATH)
    for name in declared:
        assert hasattr(L, name), name


def test_struct_sizes():
    assert [ctypes.sizeof(c) for c in (T.tns_recur, T.tns_pairs, T.tns_adamw_tensor, T.tns_adamw_config)] == [104, 104, 72, 48]


def recur(**kw):
    a = dict(S=2, rows=4, dim=8, dtype=0, flags=0, reserved=0, d_rowptr=256, d_u=256, d_x=256, ld_u=8, ld_x=8, d_ts=None, d_decay=None, d_h0=None, d_t0=None)
    a.update(kw)
    return T.tns_recur(*[a[n] for n, _ in T.tns_recur._fields_])


def refused(status, call, *args):
    with pytest.raises(B.TnsError) as e:
        call(*args)
    assert e.value.status == status, str(e.value)


@pytest.mark.parametrize("kw, status", [
    (dict(S=-1), B.TNS_EINVAL), (dict(rows=-1), B.TNS_EINVAL), (dict(S=1 << 31), B.TNS_ESIZE), (dict(rows=(1 << 40) + 1), B.TNS_ESIZE),
    (dict(dim=0), B.TNS_EINVAL), (dict(dim=65537), B.TNS_EINVAL), (dict(dtype=2), B.TNS_EINVAL), (dict(flags=2), B.TNS_EINVAL),
    (dict(reserved=1), B.TNS_EINVAL)])
def test_recurrence_refuses_descriptions(kw, status):
    refused(status, T.tns_recur_workspace, recur(**kw))


@pytest.mark.parametrize("kw", [dict(d_rowptr=None), dict(d_u=None), dict(d_x=None), dict(ld_u=7), dict(ld_x=0), dict(d_ts=256), dict(d_decay=256),
                                dict(d_t0=256)])
def test_recurrence_refuses_arrays(kw):
    r = recur(**kw)
    big = 1 << 40
    refused(B.TNS_EINVAL, T.tns_recur_run, r, 256, 8, 256, 256, 256, big)
    refused(B.TNS_EINVAL, T.tns_recur_grad, r, 256, 256, 8, 256, 256, 8, 256, 8, 0, 0, 256, big)


def test_recurrence_refuses_outputs():
    r, big = recur(), 1 << 40
    refused(B.TNS_EINVAL, T.tns_recur_run, r, 256, 7, 256, 256, 256, big)                                # rows of h overlap
    refused(B.TNS_EINVAL, T.tns_recur_run, r, 256, 8, 256, 260, 256, big)                                # saved states not aligned
    refused(B.TNS_EINVAL, T.tns_recur_run, r, 256, 8, 256, 256, 272, big)                                # workspace not aligned
    for bad in ((0, 256, 8, 0, 256, 8, 256, 8, 0), (256, 256, 8, 0, 0, 8, 256, 8, 0), (256, 256, 8, 0, 256, 8, 0, 8, 0), (256, 256, 7, 0, 256, 8, 256, 8, 0),
                (256, 256, 8, 0, 256, 7, 256, 8, 0), (256, 256, 8, 0, 256, 8, 256, 7, 0), (256, 256, 8, 0, 256, 8, 256, 8, 256), (264, 256, 8, 0, 256, 8, 256, 8, 0)):
        refused(B.TNS_EINVAL, T.tns_recur_grad, r, *bad, 0, 256, big)
    refused(B.TNS_EINVAL, T.tns_recur_grad, r, 256, 256, 8, 0, 256, 8, 256, 8, 0, 0, 0, big)             # no workspace
    refused(B.TNS_ESIZE, T.tns_recur_grad, r, 256, 256, 8, 0, 256, 8, 256, 8, 0, 0, 256, 0)


def test_step_refuses():
    ok = dict(B=2, num_ids=4, dim=8, dtype=0, d_ids=256, d_u=256, ld_u=8, d_x=256, ld_x=8, d_ts=256, d_decay=256, d_state=256, d_state_ts=256, d_out=256, ld_out=8)
    for kw, status in [(dict(B=-1), B.TNS_EINVAL), (dict(num_ids=-1), B.TNS_EINVAL), (dict(B=1 << 31), B.TNS_ESIZE), (dict(num_ids=1 << 31), B.TNS_ESIZE),
                       (dict(dim=0), B.TNS_EINVAL), (dict(dtype=-1), B.TNS_EINVAL), (dict(d_ids=None), B.TNS_EINVAL), (dict(d_u=None), B.TNS_EINVAL),
                       (dict(d_x=None), B.TNS_EINVAL), (dict(d_state=None), B.TNS_EINVAL), (dict(d_ts=None), B.TNS_EINVAL), (dict(d_decay=None), B.TNS_EINVAL),
                       (dict(d_state_ts=None), B.TNS_EINVAL), (dict(ld_u=7), B.TNS_EINVAL), (dict(ld_x=7), B.TNS_EINVAL), (dict(ld_out=7), B.TNS_EINVAL)]:
        refused(status, T.tns_recur_step, *dict(ok, **kw).values())


def test_pair_loss_refuses():
    ok = dict(B=2, K=3, dim=8, dtype=0, d_anchor=256, d_pos=256, d_neg=256, ld_anchor=8, ld_pos=8, d_ref=None, d_weight=None, beta=1.0, smoothing=0.0, scale=1.0)
    out = (256, 256, 256, 256, 256, 256, 1 << 40)
    for kw, status in [(dict(B=-1), B.TNS_EINVAL), (dict(K=-1), B.TNS_EINVAL), (dict(B=1 << 31), B.TNS_ESIZE), (dict(B=1 << 30, K=1 << 11), B.TNS_ESIZE),
                       (dict(dim=0), B.TNS_EINVAL), (dict(dim=1 << 17), B.TNS_EINVAL), (dict(dtype=3), B.TNS_EINVAL), (dict(d_anchor=None), B.TNS_EINVAL),
                       (dict(d_pos=None), B.TNS_EINVAL), (dict(d_neg=None), B.TNS_EINVAL), (dict(ld_anchor=7), B.TNS_EINVAL), (dict(ld_pos=7), B.TNS_EINVAL),
                       (dict(smoothing=-0.1), B.TNS_EINVAL), (dict(smoothing=1.1), B.TNS_EINVAL), (dict(smoothing=float("nan")), B.TNS_EINVAL)]:
        refused(status, T.tns_pair_loss, T.tns_pairs(*dict(ok, **kw).values()), *out)
    p = T.tns_pairs(*ok.values())
    for at, value, status in [(0, 0, B.TNS_EINVAL), (2, 0, B.TNS_EINVAL), (3, 0, B.TNS_EINVAL), (4, 0, B.TNS_EINVAL), (5, 0, B.TNS_EINVAL), (5, 264, B.TNS_EINVAL),
                              (6, 0, B.TNS_ESIZE)]:
        args = list(out)
        args[at] = value
        refused(status, T.tns_pair_loss, p, *args)
    refused(B.TNS_EINVAL, T.tns_pair_loss_workspace, -1, 1, 8)


def test_adamw_refuses():
    cfg = dict(beta1=0.9, beta2=0.999, eps=1e-8, seed=0, state_bits=8, grad_dtype=0, device=0, reserved=0)
    one = dict(n=5, d_param=256, d_copy=None, d_grad=256, d_m=256, d_v=256, d_m_scale=256, d_v_scale=256, weight_decay=0.0)
    for kw, status in [(dict(beta1=1.0), B.TNS_EINVAL), (dict(beta1=-0.1), B.TNS_EINVAL), (dict(beta2=float("nan")), B.TNS_EINVAL), (dict(eps=-1.0), B.TNS_EINVAL),
                       (dict(eps=float("inf")), B.TNS_EINVAL), (dict(state_bits=16), B.TNS_EINVAL), (dict(grad_dtype=2), B.TNS_EINVAL),
                       (dict(device=-1), B.TNS_EINVAL), (dict(reserved=1), B.TNS_EINVAL)]:
        refused(status, T.tns_adamw_create, T.tns_adamw_config(*dict(cfg, **kw).values()), [T.tns_adamw_tensor(*one.values())])
    for kw, status in [(dict(n=-1), B.TNS_EINVAL), (dict(n=(1 << 40) + 1), B.TNS_ESIZE), (dict(d_param=None), B.TNS_EINVAL), (dict(d_grad=None), B.TNS_EINVAL),
                       (dict(d_m=None), B.TNS_EINVAL), (dict(d_v=None), B.TNS_EINVAL), (dict(d_m_scale=None), B.TNS_EINVAL), (dict(d_v_scale=None), B.TNS_EINVAL),
                       (dict(weight_decay=float("inf")), B.TNS_EINVAL)]:
        refused(status, T.tns_adamw_create, T.tns_adamw_config(*cfg.values()), [T.tns_adamw_tensor(*dict(one, **kw).values())])
    refused(B.TNS_EINVAL, T.tns_adamw_step, None, 1e-3, 1)
    assert T.lib().tns_adamw_destroy(None) == B.TNS_OK


def test_tensors_off_the_gpu_are_refused():
    import torch
    v = torch.zeros(4, 8)
    for call in (lambda: T.recur_run(torch.zeros(2, dtype=torch.int64), v, v), lambda: T.recur_step(torch.zeros(4, dtype=torch.int32), v, v, v),
                 lambda: T.pair_loss(v, v, torch.zeros(4, 1, 8)), lambda: T.AdamW([v], [v])):
        with pytest.raises(ValueError):
            call()


def test_tensors_that_require_gradients_are_refused():
    """Results that autograd takes for constants are no results for a caller who relies on it (off the GPU: it is looked at first)."""
    import torch
    rp, ids = torch.zeros(2, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)
    v, g, d, t, many = torch.zeros(4, 8), torch.zeros(4, 8, requires_grad=True), torch.zeros(8, requires_grad=True), torch.zeros(4), torch.zeros(4, 1, 8)
    calls = [lambda: T.recur_run(rp, g, v), lambda: T.recur_run(rp, v, g), lambda: T.recur_run(rp, v, v, ts=t, decay=d), lambda: T.recur_run(rp, v, v, h0=g[:1]),
             lambda: T.recur_grad(rp, g, v, v), lambda: T.recur_grad(rp, v, v, v, dh=g), lambda: T.recur_step(ids, g, v, v), lambda: T.recur_step(ids, v, v, g),
             lambda: T.pair_loss(g, v, many), lambda: T.pair_loss(v, g, many), lambda: T.pair_loss(v, v, g[:, None]), lambda: T.pair_loss(v, v, many, weight=g[:, :1])]
    for call in calls:
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on the GPU"):
            call()


LONG = {"one": [900], "cut": [300, 1, 70, 2, 256, 40, 1, 1, 230]}


def slow(rng, lens, dim, decay=True, start=True):
    """Gates and decays that carry a state over thousands of rows."""
    a = lists(rng, lens, dim, decay, start)
    a["u"] = (a["u"] - 8).astype(np.float32)
    a["x"] = a["x"].astype(np.float32)
    if decay:
        a.update(decay=np.float32(rng.uniform(0, 2e-4, dim)), ts=np.float32(np.cumsum(rng.uniform(0, 2, len(a["u"])))))
    if start:
        a.update(h0=a["h0"].astype(np.float32))
    return a


@pytest.mark.parametrize("newest_first", [False, True])
@pytest.mark.parametrize("decay, start, both", [(True, True, True), (False, True, False), (True, False, True), (False, False, False)])
@pytest.mark.parametrize("lens", list(LONG))
def test_recurrence_by_scans_is_the_same(lens, decay, start, both, newest_first):
    rng = np.random.default_rng(20)
    a = slow(rng, LONG[lens], 3, decay, start)
    kw = dict(newest_first=newest_first, dh=rng.normal(size=a["u"].shape) if both else None, dlast=rng.normal(size=(len(LONG[lens]), 3)))
    want, got = O.recurrence(**a, **kw), O.recurrence_scanned(**a, **kw)
    for k, v in want.items():
        if (decay or not k.startswith("ddecay")) and (start or not k.startswith("dh0")):
            assert np.allclose(got[k], v, rtol=1e-9, atol=1e-12 * max(np.abs(v).max(), 1e-30)), k


@pytest.mark.parametrize("newest_first", [False, True])
@pytest.mark.parametrize("span, rows", [(256, 4000), (512, 9000)])
def test_a_lost_or_repeated_carry_is_far_outside_the_bounds(span, rows, newest_first):
    """Mistakes that a join of spans can make, in the factors of the 64-bit form: a carry lost at a border, a span's factor left out, one taken
    twice.  Each is seen in the states and in the rows' gradients (the decay's is a sum over all rows, in whose bound one span hardly counts)."""
    rng = np.random.default_rng(21)
    a = slow(rng, [rows], 2)
    kw = dict(newest_first=newest_first, dh=rng.normal(size=a["u"].shape), dlast=rng.normal(size=(1, 2)))
    want = O.recurrence_scanned(**a, **kw)
    at = rows // 2 // span * span

    def lost(f):
        f = f.copy()
        f[at] = 0
        return f

    def left_out(f):
        f = f.copy()
        f[at] /= f[at: at + span].prod(0)
        return f

    def twice(f):
        f = f.copy()
        f[at] *= f[at: at + span].prod(0)
        return f

    for mistake in (lost, left_out, twice):
        bad = O.recurrence_scanned(**a, **kw, change=mistake)
        for k in ("h", "dx", "du"):
            assert (np.abs(bad[k] - want[k]) > 4 * want[k + "_off"]).any(), (mistake.__name__, k)


@pytest.mark.parametrize("dim", [1, 64, 300])
def test_tiles_stay_as_they_are_however_many_rows_there_are(dim):
    """A tile's rows fit the lanes of a wave: what is kept for every tile grows with the rows."""
    one, two = (T.tns_recur_workspace(recur(S=2, rows=1 << k, dim=dim, ld_u=dim, ld_x=dim))[0] for k in (38, 39))
    assert one >= (1 << 38) // 64 * (8 * dim + 5) and two > 1.999 * one


def test_an_8_bit_second_moment_is_high_by_its_roundings_variance():
    """4000 steps of normal gradients: the root is right to a percent or two on average, its square high by some percent (as the header says)."""
    rng, n, v = np.random.default_rng(25), 256, np.zeros(256)
    state = dict(m=np.zeros(n, np.uint8), v=np.zeros(n, np.uint8), m_scale=np.zeros(1, np.float32), v_scale=np.zeros(1, np.float32))
    param, squares, roots = np.zeros(n, np.float32), [], []
    for t in range(1, 4001):
        g = (0.02 * rng.normal(size=n)).astype(np.float32)
        v = 0.999 * v + 0.001 * g.astype(np.float64) ** 2
        _, _, state = O.adamw(param, g, state, t, weight_decay=0.0, seed=5)
        if t > 2000 and t % 20 == 0:
            r = O.e4m3_value(state["v"]).astype(np.float64) * state["v_scale"][0]
            squares.append((r * r / v).mean())
            roots.append((r / np.sqrt(v)).mean())
    # single weights are off by 0.2, so their mean over 256 by 0.0125; four times that
    assert 1.0 < np.mean(squares) < 1.1 and abs(np.mean(roots) - 1.01) < 0.05, (np.mean(squares), np.mean(roots))


def test_tensors_with_tangents_are_refused():
    """Results without the tangents that they have would be constants to forward differentiation; a detached tensor has none, nor one within a Function."""
    import torch
    from torch.autograd import forward_ad
    rp, ids, many = torch.zeros(2, dtype=torch.int64), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 1, 8)

    def calls(v):
        return [lambda: T.recur_run(rp, v, v), lambda: T.recur_grad(rp, torch.zeros(4, 8), v, None), lambda: T.recur_step(ids, v, v, torch.zeros(4, 8)), lambda: T.pair_loss(v, v, many)]

    with forward_ad.dual_level():
        dual = forward_ad.make_dual(torch.zeros(4, 8), torch.ones(4, 8))
        for call in calls(dual):
            with pytest.raises(ValueError, match="tangents"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="tangents"):
                call()
        for call in calls(dual.detach()):
            with pytest.raises(ValueError, match="on the GPU"):
                call()

        class Once(torch.autograd.Function):
            @staticmethod
            def forward(x):
                for call in calls(x):
                    with pytest.raises(ValueError, match="on the GPU"):
                        call()
                return 2 * x

            @staticmethod
            def setup_context(ctx, inputs, output):
                pass

            @staticmethod
            def jvp(ctx, tangent):
                return 2 * tangent

        assert bool((forward_ad.unpack_dual(Once.apply(dual)).tangent == 2).all())
