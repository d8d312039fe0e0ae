"""The oracle of the layer operators against closed forms and differences; the interface and its refusals.  No GPU."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import layer_oracle as O
from paper_2311_17410_amd import binding as B
from paper_2311_17410_amd import layer_binding as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BIG = 1 << 40


def differences(f, a, name, by=1e-6):
    d = np.zeros_like(a[name])
    for i in np.ndindex(d.shape):
        ends = []
        for s in (by, -by):
            moved = a[name].copy()
            moved[i] += s
            ends.append(f(dict(a, **{name: moved})))
        d[i] = (ends[0] - ends[1]) / (2 * by)
    return d


def test_attend_closed_forms():
    """Equal scores: the mean; one event: its value; a far larger score: that event's value; nothing left: zero."""
    v = np.arange(12.0).reshape(4, 1, 3)
    q, k = np.zeros((1, 2, 3)), np.zeros((4, 1, 3))
    assert np.allclose(O.attend([0, 4], q, k, v)["out"][0], v.mean(0))
    assert np.allclose(O.attend([0, 1], q, k[:1], v[:1])["out"][0], v[0])
    table = np.array([[0.0, 0.0], [500.0, -np.inf]])
    r = O.attend([0, 4], q, k, v, edges=np.float32([3]), table=table, newest_first=True)["out"][0]      # places 0..3: the last has bucket 1
    assert np.allclose(r[0], v[3]) and np.allclose(r[1], v[:3].mean(0))
    r = O.attend([0, 4], q, k, v, edges=np.float32([3]), table=table)["out"][0]                         # the first row is the oldest, three events newer
    assert np.allclose(r[0], v[0]) and np.allclose(r[1], v[1:].mean(0))
    assert not O.attend([0, 4, 4], np.zeros((2, 2, 3)), k, v, mask=np.zeros(4, bool))["out"].any()
    r = O.attend([0, 4], q, k, v, index=np.int32([2, -1, 7, 2]))["out"][0]
    assert np.allclose(r, v[2])


def test_ages():
    assert list(O.gap_of(np.float32(3), np.float32([1, 3, 4, -np.inf, np.inf, np.nan]))) == [2, 0, 0, np.finfo(np.float32).max, 0, 0]
    # an age on a border belongs to the bucket above it
    v = np.float64([[[1.0]], [[0.0]]])
    table = np.array([[0.0], [300.0]])
    r = O.attend([0, 2], np.zeros((1, 1, 1)), v, v, t=np.float32([5]), ts=np.float32([3, 4]), edges=np.float32([2]), table=table)
    assert np.allclose(r["out"], 1)


@pytest.mark.parametrize("times", [True, False])
def test_attend_gradients_against_differences(times):
    rng = np.random.default_rng(1)
    lens = [3, 0, 1, 5]
    rp = np.concatenate([[0], np.cumsum(lens)])
    a = dict(q=rng.normal(size=(4, 4, 3)), k=rng.normal(size=(9, 2, 3)), v=rng.normal(size=(9, 2, 3)), table=rng.normal(size=(3, 4)))
    more = dict(edges=np.float32([1, 2]), mask=np.array([1, 1, 0, 1, 1, 1, 0, 1, 1], bool), newest_first=True)
    if times:
        more.update(t=np.float32([5, 5, 5, 6]), ts=rng.uniform(2, 5, 9).astype(np.float32))
    dout = rng.normal(size=a["q"].shape)
    got = O.attend(rp, **a, **more, dout=dout)
    for name in a:
        assert np.allclose(got["d" + name], differences(lambda b: (O.attend(rp, **b, **more)["out"] * dout).sum(), a, name), rtol=1e-6, atol=1e-8), name


@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("without", [(), ("gate",), ("post",), ("scale", "gate"), ("pre",)])
def test_block_gradients_against_differences(without, center):
    rng = np.random.default_rng(2)
    a = dict(x=rng.normal(size=(3, 5)), branch=rng.normal(size=(3, 5)), gate=rng.normal(size=(3, 5)), scale=rng.normal(size=5), post=rng.normal(size=5), pre=rng.normal(size=5))
    for name in without:
        a.pop(name)
    dout, dnext = rng.normal(size=(3, 5)), rng.normal(size=(3, 5)) if "pre" in a else None

    def scalar(b):
        r = O.block(**b, center=center)
        return (r["out"] * dout).sum() + ((r["next"] * dnext).sum() if dnext is not None else 0)

    got = O.block(**a, center=center, dout=dout, dnext=dnext)
    for name in a:
        assert np.allclose(got["d" + name], differences(scalar, a, name), rtol=1e-5, atol=1e-8), name


def test_block_closed_forms():
    """A constant row has no spread; a row of one sign and size is its own norm."""
    r = O.block(np.zeros((1, 4)), np.full((1, 4), 3.0), post=np.ones(4), pre=np.full(4, 2.0), eps=0.0)
    assert np.allclose(r["out"], 1) and np.allclose(r["next"], 2)
    assert np.allclose(O.block(np.ones((1, 4)), np.full((1, 4), 3.0), post=np.ones(4), center=True)["out"], 1)
    assert np.allclose(O.block(np.ones((1, 2)), np.full((1, 2), 4.0), gate=np.zeros((1, 2)), scale=np.full(2, 0.5))["out"], 2)


@pytest.mark.parametrize("rest", [False, True])
def test_distill_closed_forms_and_differences(rest):
    rng = np.random.default_rng(3)
    s, t = rng.normal(size=(4, 7)), rng.normal(size=(4, 3))
    ids = np.int32([[0, 3, 6], [2, -1, 9], [1, 1, 4], [5, 0, 2]])
    lse = np.log(np.exp(t / 2).sum(1)) + 0.3 if rest else None
    w = np.array([1.0, 0.5, 2.0, 0.0])
    kw = dict(lse=lse, weight=w, temperature=2.0, scale=0.25)
    got = O.distill(s, ids, t, **kw)
    d = differences(lambda a: O.distill(a["s"], ids, t, **kw)["loss"], dict(s=s), "s")
    assert np.allclose(got["dlogits"], d, rtol=1e-6, atol=1e-9) and not got["dlogits"][3].any() and got["rows"][3] == 0
    # a student that is the teacher: nothing to learn
    full = rng.normal(size=(1, 5))
    all_ = np.arange(5, dtype=np.int32)[None]
    r = O.distill(full, all_, full)
    assert abs(r["loss"]) < 1e-14 and np.abs(r["dlogits"]).max() < 1e-14
    some = O.distill(full, all_[:, :2], full[:, :2], lse=np.log(np.exp(full).sum(1)))
    assert abs(some["loss"]) < 1e-14 and np.abs(some["dlogits"]).max() < 1e-14
    # even scores, one certain candidate: the logarithm of their number
    assert np.isclose(O.distill(np.zeros((1, 8)), np.int32([[3]]), np.zeros((1, 1)))["loss"], np.log(8))
    assert O.distill(np.zeros((1, 8)), np.int32([[-1]]), np.zeros((1, 1)))["loss"] == 0


def test_distill_named_far_above_the_others():
    """One named candidate of score 100 and more above three others: the others' share of the loss is a sum in the logarithm."""
    for lead in (100.0, 1000.0):
        s = np.float64([[lead, 0.0, 0.5, -1.0]])
        r = O.distill(s, np.int32([[0]]), np.log([[0.7]]), lse=np.zeros(1))
        others = np.exp(s[0, 1:]) / np.exp(s[0, 1:]).sum()
        # log q of the named one is 0 but for exp(-99), that of the others together log of their sum minus the lead
        assert np.isclose(r["loss"], 0.7 * np.log(0.7) + 0.3 * (np.log(0.3) - (np.log(np.exp(s[0, 1:]).sum()) - lead)), rtol=1e-12)
        assert np.allclose(r["dlogits"][0], np.concatenate([[0.3], -0.3 * others]), rtol=1e-12) and np.isfinite(r["dlogits_off"]).all()


# ---- interface -----------------------------------------------------------------------------------

def test_every_declared_symbol_is_exported_and_bound():
    hdr = open(os.path.join(ROOT, "include", "tns_layer.h")).read()
    declared = re.findall(r"TNS_API\s+[\w\s\*]+?\b(tns_\w+)\s*\(", hdr)
    assert sorted(declared) == sorted(L.EXPORTS)
    lib = ctypes.CDLL(B.LIB_PATH)
    for name in declared:
        assert hasattr(lib, name), name


def test_struct_sizes():
    assert [ctypes.sizeof(c) for c in (L.tns_attend, L.tns_block, L.tns_distill_desc)] == [160, 104, 88]


def refused(status, call, *args):
    with pytest.raises(B.TnsError) as e:
        call(*args)
    assert e.value.status == status, str(e.value)


def attend(**kw):
    a = dict(S=2, rows=4, num=0, heads=4, kv_heads=2, head_dim=8, dtype=0, buckets=3, flags=0, d_rowptr=256, d_q=256, d_k=256, d_v=256, ld_q=32, ld_k=16, ld_v=16, d_index=None,
             d_mask=None, d_t=256, d_ts=256, d_edges=256, d_table=256, scale=1.0)
    a.update(kw)
    return L.tns_attend(*[a[n] for n, _ in L.tns_attend._fields_])


@pytest.mark.parametrize("kw, status", [
    (dict(S=-1), B.TNS_EINVAL), (dict(rows=-1), B.TNS_EINVAL), (dict(num=-1), B.TNS_EINVAL), (dict(S=1 << 31), B.TNS_ESIZE), (dict(num=1 << 31), B.TNS_ESIZE),
    (dict(rows=(1 << 40) + 1), B.TNS_ESIZE), (dict(heads=0), B.TNS_EINVAL), (dict(kv_heads=0), B.TNS_EINVAL), (dict(kv_heads=3), B.TNS_EINVAL), (dict(kv_heads=8), B.TNS_EINVAL),
    (dict(heads=18, kv_heads=2), B.TNS_EINVAL), (dict(heads=2048, kv_heads=1024), B.TNS_EINVAL), (dict(head_dim=0), B.TNS_EINVAL), (dict(head_dim=257), B.TNS_EINVAL),
    (dict(dtype=2), B.TNS_EINVAL), (dict(buckets=-1), B.TNS_EINVAL), (dict(buckets=257), B.TNS_EINVAL), (dict(heads=16, kv_heads=8, buckets=129), B.TNS_EINVAL),
    (dict(flags=2), B.TNS_EINVAL)])
def test_attend_refuses_descriptions(kw, status):
    refused(status, L.tns_attend_workspace, attend(**kw))


@pytest.mark.parametrize("kw", [dict(d_rowptr=None), dict(d_q=None), dict(d_k=None), dict(d_v=None), dict(ld_q=31), dict(ld_k=15), dict(ld_v=15), dict(num=4), dict(d_t=None),
                                dict(d_ts=None), dict(d_table=None), dict(d_edges=None), dict(buckets=0), dict(d_q=258), dict(d_k=257), dict(d_v=258)])
def test_attend_refuses_arrays(kw):
    a = attend(**kw)
    refused(B.TNS_EINVAL, L.tns_attend_run, a, 256, 256, 256, BIG)
    refused(B.TNS_EINVAL, L.tns_attend_grad, a, 256, 256, 256, 256, 256, 256, 256, BIG)


def test_attend_refuses_outputs():
    a = attend()
    for args, status in [((0, 0, 256, BIG), B.TNS_EINVAL), ((258, 0, 256, BIG), B.TNS_EINVAL), ((256, 264, 256, BIG), B.TNS_EINVAL), ((256, 0, 0, BIG), B.TNS_EINVAL),
                         ((256, 0, 264, BIG), B.TNS_EINVAL), ((256, 0, 256, 0), B.TNS_ESIZE)]:
        refused(status, L.tns_attend_run, a, *args)
    ok = [256, 256, 256, 256, 256, 256, 256, BIG]
    for at, value, status in [(0, 0, B.TNS_EINVAL), (0, 264, B.TNS_EINVAL), (1, 0, B.TNS_EINVAL), (1, 258, B.TNS_EINVAL), (2, 0, B.TNS_EINVAL), (3, 0, B.TNS_EINVAL),
                              (4, 0, B.TNS_EINVAL), (4, 257, B.TNS_EINVAL), (5, 0, B.TNS_EINVAL), (6, 0, B.TNS_EINVAL), (7, 0, B.TNS_ESIZE)]:
        refused(status, L.tns_attend_grad, a, *[value if i == at else v for i, v in enumerate(ok)])
    many = attend(rows=1 << 38)                                               # more blocks than a launch has workgroups for
    refused(B.TNS_ESIZE, L.tns_attend_run, many, 256, 256, 256, 1 << 62)
    refused(B.TNS_ESIZE, L.tns_attend_grad, many, *ok[:7], 1 << 62)
    refused(B.TNS_ESIZE, L.tns_attend_run, attend(ld_k=1 << 22), 256, 256, 256, BIG)
    refused(B.TNS_ESIZE, L.tns_attend_run, attend(ld_v=1 << 22), 256, 256, 256, BIG)
    refused(B.TNS_EINVAL, L.tns_attend_grad, attend(d_index=256, num=4), *ok)      # no gradients by gathered rows
    refused(B.TNS_EINVAL, L.tns_attend_grad, attend(buckets=0, d_table=None, d_edges=None), *ok)


def test_no_events_of_a_table_of_nodes():
    """Without a row, the index has no address: a table of nodes may be there all the same.  (Without lists nothing is launched.)"""
    L.tns_attend_run(attend(S=0, rows=0, num=4, d_index=None), 0, 0, 0, 0)
    refused(B.TNS_EINVAL, L.tns_attend_run, attend(S=0, rows=4, num=4, d_index=None), 0, 0, 256, BIG)


def block(**kw):
    a = dict(rows=4, dim=8, dtype=0, flags=0, reserved=0, d_x=256, d_branch=256, d_gate=256, ld_x=8, ld_branch=8, ld_gate=8, d_scale=256, d_post=256, d_pre=256, eps=1e-6)
    a.update(kw)
    return L.tns_block(*[a[n] for n, _ in L.tns_block._fields_])


@pytest.mark.parametrize("kw, status", [
    (dict(rows=-1), B.TNS_EINVAL), (dict(rows=(1 << 40) + 1), B.TNS_ESIZE), (dict(dim=0), B.TNS_EINVAL), (dict(dim=8193), B.TNS_EINVAL), (dict(dtype=2), B.TNS_EINVAL),
    (dict(flags=2), B.TNS_EINVAL), (dict(reserved=1), B.TNS_EINVAL), (dict(d_x=None), B.TNS_EINVAL), (dict(d_branch=None), B.TNS_EINVAL), (dict(ld_x=7), B.TNS_EINVAL),
    (dict(ld_branch=7), B.TNS_EINVAL), (dict(ld_gate=7), B.TNS_EINVAL), (dict(eps=-1.0), B.TNS_EINVAL), (dict(eps=float("nan")), B.TNS_EINVAL), (dict(eps=float("inf")), B.TNS_EINVAL),
    (dict(d_x=258), B.TNS_EINVAL), (dict(d_gate=257), B.TNS_EINVAL)])
def test_block_refuses(kw, status):
    b = block(**kw)
    refused(status, L.tns_block_run, b, 256, 256)
    refused(status, L.tns_block_grad, b, 256, 8, 256, 8, 256, 256, 256, 256, 256, 256, 256, BIG)


def test_block_refuses_outputs():
    for args in [(0, 256), (256, 0), (258, 256), (256, 257)]:
        refused(B.TNS_EINVAL, L.tns_block_run, block(), *args)
    refused(B.TNS_EINVAL, L.tns_block_run, block(d_pre=None), 256, 256)
    ok = [256, 8, 256, 8, 256, 256, 256, 256, 256, 256, 256, BIG]
    for at, value, status in [(0, 258, B.TNS_EINVAL), (1, 7, B.TNS_EINVAL), (3, 7, B.TNS_EINVAL), (4, 0, B.TNS_EINVAL), (5, 0, B.TNS_EINVAL), (6, 0, B.TNS_EINVAL), (6, 257, B.TNS_EINVAL),
                              (10, 0, B.TNS_EINVAL), (10, 264, B.TNS_EINVAL), (11, 0, B.TNS_ESIZE)]:
        refused(status, L.tns_block_grad, block(), *[value if i == at else v for i, v in enumerate(ok)])
    for kw in (dict(d_pre=None), dict(d_post=None), dict(d_scale=None), dict(d_gate=None)):
        refused(B.TNS_EINVAL, L.tns_block_grad, block(**kw), *ok)
    refused(B.TNS_EINVAL, L.tns_block_workspace, -1, 8)
    refused(B.TNS_EINVAL, L.tns_block_workspace, 1, 0)


def test_distill_refuses():
    ok = dict(B=2, V=8, K=3, dtype=0, d_logits=256, ld_logits=8, d_ids=256, d_teacher=256, d_lse=None, d_weight=None, temperature=1.0, scale=1.0)
    out = [256, 256, 256, 256, BIG]
    for kw, status in [(dict(B=-1), B.TNS_EINVAL), (dict(B=1 << 31), B.TNS_ESIZE), (dict(V=0), B.TNS_EINVAL), (dict(V=1 << 31, ld_logits=1 << 31), B.TNS_ESIZE), (dict(K=-1), B.TNS_EINVAL),
                       (dict(K=1025), B.TNS_EINVAL), (dict(dtype=2), B.TNS_EINVAL), (dict(d_logits=None), B.TNS_EINVAL), (dict(d_logits=258), B.TNS_EINVAL), (dict(ld_logits=7), B.TNS_EINVAL),
                       (dict(d_ids=None), B.TNS_EINVAL), (dict(d_teacher=None), B.TNS_EINVAL), (dict(temperature=0.0), B.TNS_EINVAL), (dict(temperature=-1.0), B.TNS_EINVAL),
                       (dict(temperature=float("nan")), B.TNS_EINVAL), (dict(temperature=float("inf")), B.TNS_EINVAL)]:
        refused(status, L.tns_distill, L.tns_distill_desc(*dict(ok, **kw).values()), *out)
    for at, value, status in [(0, 0, B.TNS_EINVAL), (2, 257, B.TNS_EINVAL), (3, 0, B.TNS_EINVAL), (3, 264, B.TNS_EINVAL), (4, 0, B.TNS_ESIZE)]:
        refused(status, L.tns_distill, L.tns_distill_desc(*ok.values()), *[value if i == at else v for i, v in enumerate(out)])
    refused(B.TNS_EINVAL, L.tns_distill_workspace, -1, 1, 1)


def calls(v, rp, ids):
    import torch
    h = v.view(4, 1, 8)
    return [lambda: L.attend_run(rp, h, h, h), lambda: L.attend_grad(rp, h, h, h, v, h), lambda: L.block_run(v, v), lambda: L.block_grad(v, v),
            lambda: L.distill(v, ids, torch.zeros(4, 2))]


def test_tensors_off_the_gpu_or_that_require_gradients_are_refused():
    import torch
    rp, ids = torch.tensor([0, 1, 2, 3, 4]), torch.zeros((4, 2), dtype=torch.int32)
    for call in calls(torch.zeros(4, 8), rp, ids):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
    for call in calls(torch.zeros((4, 8), requires_grad=True), rp, ids):
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on the GPU"):
            call()


def test_tensors_with_tangents_are_refused():
    """Results without the tangents that they have would be constants to forward differentiation; a detached tensor has none, nor one within a Function."""
    import torch
    from torch.autograd import forward_ad
    rp, ids = torch.tensor([0, 1, 2, 3, 4]), torch.zeros((4, 2), dtype=torch.int32)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(torch.zeros(4, 8), torch.ones(4, 8))
        for call in calls(dual, rp, ids):
            with pytest.raises(ValueError, match="tangents"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="tangents"):
                call()
        for call in calls(dual.detach(), rp, ids):
            with pytest.raises(ValueError, match="on the GPU"):
                call()

        class Once(torch.autograd.Function):
            @staticmethod
            def forward(x):
                for call in calls(x, rp, ids):
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
