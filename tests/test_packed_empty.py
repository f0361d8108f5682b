"""Batches of empty sequences: every prompt of the batch was taken back.  Slots of sequences that start from zeros are set to zeros, those of
sequences that go on keep theirs, with tensors of no rows and with rows of padding alone."""
import ctypes

import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from paper_2411_19460_b200 import libssd
from tests.test_packed import make, make_conv, rows_shape


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


SLOTS, CARRY = [4, 0, -1, 2], [False, True, False, False]


def expected(state):
    want = state.clone()
    want[[4, 2]] = 0
    return want


@pytest.mark.gpu
@pytest.mark.parametrize("behind", [0, 1, 5])
@pytest.mark.parametrize("dtype,N", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
def test_scan(dtype, N, behind):
    t = make([0, 0, 0, 0], 4, 2, N, dtype, behind=behind, nslots=6)
    t["state"][5] = float("nan")
    t["state"][4] = float("nan")
    want = expected(t["state"])
    plan = libssd.PackedPlan(t["cu"], slots=SLOTS, carry=CARRY, nslots=6, heads=4)
    y = torch.full(t["x"].shape, 7.0, dtype=t["x"].dtype, device="cuda")
    args = [t[k] for k in ("x", "dt", "A", "Bm", "Cm", "D", "state")]
    ws = libssd.alloc_packed_workspace(plan, t["x"], t["Bm"])
    ws.fill_(255)
    assert libssd.ssd_packed_fwd(plan, *args, y=y, ws=ws) is y
    torch.cuda.synchronize()
    assert libssd.poll_status(ws) == libssd.SSD_OK
    assert torch.equal(t["state"].nan_to_num(9), want.nan_to_num(9)) and bool((y == 7).all())
    assert libssd.ssd_packed_fwd(plan, *args).shape == (behind, 4, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("behind", [0, 1, 5])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_convolution(dtype, behind):
    t = make_conv(behind, 24, dtype, 6, seed=3)
    t["state"][4] = float("nan")
    want = expected(t["state"])
    plan = libssd.PackedPlan([0] * 5, slots=SLOTS, carry=CARRY, nslots=6, heads=4)
    out = torch.full((behind, 24), 7.0, dtype=t["u"].dtype, device="cuda")
    libssd.ssd_conv_packed_fwd(plan, t["u"], t["w"], t["bias"], t["state"], out=out)
    assert torch.equal(t["state"], want) and bool((out == 7).all())
    assert libssd.ssd_conv_packed_fwd(plan, t["u"], t["w"], t["bias"], t["state"]).shape == (behind, 24)


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where no kernel can run on them")
def test_checks():
    """No rows pass the checks (and end at the missing device) where the plan has none, and are refused where it has some; rows need their tensors."""
    L, ok = libssd.lib(), ctypes.c_void_p(0x1000)
    empty, some = (libssd.PackedPlan(cu, nslots=8, heads=4, device="cpu") for cu in ([0, 0, 0], [0, 0, 2]))
    codes = {}
    for name, plan in (("empty", empty), ("some", some)):
        ph = ctypes.c_void_p(plan.host.data_ptr())
        for rows in (0, 2):
            s = rows_shape(rows=rows)
            assert (L.ssd_packed_workspace_bytes(ctypes.byref(s), ph) > 0) == (name == "empty" or rows == 2)
            codes[name, rows] = [L.ssd_packed_fwd(ctypes.byref(s), ph, ok, None, None, ok, None, None, ok, ok, None, ok, 1 << 30, None),
                                 L.ssd_conv_packed_fwd(ph, ok, rows, 16, 1, None, 0, ok, ok, ok, 8, 0, None, 0, None)]
    refused = [libssd.SSD_EINVAL] * 2
    assert all(c in (libssd.SSD_ECUDA, libssd.SSD_EDEVICE) for c in codes["empty", 0])
    assert codes["some", 0] == codes["some", 2] == codes["empty", 2] == refused
