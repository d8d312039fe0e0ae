"""Calls of the layer operators at the ends of what their header allows, on the GPU against the oracle in 64 bits.  Tolerances as in test_gpu_layer.py."""
import numpy as np
import pytest

from oracle import layer_oracle as O
from test_gpu_layer import L, on_gpu, the_events      # noqa: F401
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
