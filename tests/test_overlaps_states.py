"""Outputs that share memory with dt or with the cache are refused, dt beside y in one wider tensor of fp32 is not: on the host, so on the CPU, through
the C ABI, as in tests/test_overlaps.py."""
import ctypes

import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from paper_2411_19460_b200 import libssd
from tests.test_overlaps import BASE, BIG, passed, vp
from tests.test_packed import rows_shape


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where no kernel can run on them")
X, FAR = BASE << 8, BASE << 12


def codes(s, dt, state, y):
    L = libssd.lib()
    plan = libssd.PackedPlan([0, 4, 10], slots=[0, 7], nslots=8, heads=4, device="cpu")
    x, b, c, ok = vp(X), vp(X << 4), vp(X << 6), vp(0x1000)
    return [L.ssd_packed_fwd(ctypes.byref(s), vp(plan.host.data_ptr()), ok, x, dt, ok, b, c, ok, state, y, ok, BIG, None),
            L.ssd_decode_slots(ctypes.byref(s), x, dt, ok, b, c, ok, state, ok, y, None)]


# fp32 rows of 512 elements: y 256 columns, dt 4 columns somewhere
@pytest.mark.parametrize("at,good", [(256, True), (508, True), (0, False), (252, False), (255, False), (512 * 9, False), (512 * 10, True), (-4, True), (-3, False)])
def test_dt_in_the_rows_of_y(at, good):
    s = rows_shape(dtype=0, y_rstride=512, dt_rstride=512)
    for rc in codes(s, vp(BASE + 4 * at), vp(FAR), vp(BASE)):
        assert passed(rc) if good else rc == libssd.SSD_EINVAL, rc


@pytest.mark.parametrize("dt_stride,good", [(4, False), (1024, False)])
def test_dt_of_another_stride_across_the_rows_of_y(dt_stride, good):
    s = rows_shape(dt_rstride=dt_stride)
    for rc in codes(s, vp(BASE + 512), vp(FAR), vp(BASE)):
        assert passed(rc) if good else rc == libssd.SSD_EINVAL, rc


SLOT = 4 * 64 * 128 * 4


@pytest.mark.parametrize("at,good", [(0, False), (8 * SLOT - 16, False), (8 * SLOT, True), (-10 * 512, True), (-10 * 512 + 16, False), (3 * SLOT, False)])
def test_y_in_the_states(at, good):
    for rc in codes(rows_shape(), vp(0x1000), vp(BASE), vp(BASE + at)):
        assert passed(rc) if good else rc == libssd.SSD_EINVAL, rc


@pytest.mark.parametrize("at,good", [(0, False), (8 * 96 - 16, False), (8 * 96, True), (-10 * 32, True), (-10 * 32 + 16, False)])
def test_out_in_the_cache_of_the_convolution(at, good):
    L, ok = libssd.lib(), vp(0x1000)
    plan = libssd.PackedPlan([0, 4, 10], slots=[0, 7], nslots=8, heads=4, device="cpu")
    u, state, out = vp(X), vp(BASE), vp(BASE + at)
    for rc in (L.ssd_conv_packed_fwd(vp(plan.host.data_ptr()), ok, 10, 16, 1, u, 0, ok, ok, state, 8, 0, out, 0, None),
               L.ssd_conv_step(10, 16, 1, u, 0, ok, ok, state, 8, 0, ok, out, 0, None)):
        assert passed(rc) if good else rc == libssd.SSD_EINVAL, rc
