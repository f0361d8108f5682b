"""Tiles of the packed convolution: 8, 16, 32 or 64 rows, by the rows of the batch.  Every tile length that a batch of that size has, full ones, whose rows
go round the ring of what is on its way more than once, and the ends of sequences in them.  Inputs, references and limits: tests/test_packed.py."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from paper_2411_19460_b200 import libssd
from tests.test_packed import check_conv, conv_reference, cumulative, f64, make_conv, td

# rows of a tile: lengths around one and two of them, filled up to the batch size
AROUND = {8: [7, 8, 9, 15, 16, 17, 1], 16: [12, 13, 15, 16, 17, 31, 32, 33, 3], 32: [29, 31, 32, 33, 47, 48, 63, 64, 65, 2], 64: [61, 63, 64, 65, 66, 127, 128, 129, 20]}
ROWS = {8: (3, 1024), 16: (1025, 4096), 32: (4097, 16384), 64: (16385, 20000)}


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


def lengths(tile, rows):
    lens = AROUND[tile] if sum(AROUND[tile]) < rows else []
    return [0] + lens + [rows - sum(lens), 0]


def tiles(plan):
    """(first row, rows, rows of the sequence in front, rows of the sequence) of each tile: behind the header of 64 bytes and the scan's units of 32."""
    raw = plan.host.numpy().tobytes()
    head = (ctypes.c_int32 * 16).from_buffer_copy(raw[:64])
    at = 64 + 32 * (head[4] + head[7])
    assert len(raw) == at + 32 * head[5]
    return np.frombuffer(raw[at:], dtype=np.int32).reshape(head[5], 8)[:, [0, 1, 4, 5]]


@pytest.mark.parametrize("tile,end", [(t, e) for t in ROWS for e in (0, 1)])
def test_rows_of_a_tile(tile, end):
    lens = lengths(tile, ROWS[tile][end])
    cu = cumulative(lens)
    got = tiles(libssd.PackedPlan(cu, heads=4, device="cpu"))
    want = [(cu[i] + r, min(tile, n - r), r, n) for i, n in enumerate(lens) for r in (range(0, n, tile) if n else [0])]
    assert [tuple(v) for v in got.tolist()] == want


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("C", [8, 520])
@pytest.mark.parametrize("tile,end", [(8, 1), (16, 0), (16, 1), (32, 0), (64, 0)])
def test_against_the_reference(tile, end, C, dtype):
    lens = lengths(tile, ROWS[tile][end])
    cu, n = cumulative(lens), len(lens)
    assert max(t[1] for t in tiles(libssd.PackedPlan(cu, heads=4, device="cpu"))) == tile
    slots = [n - i for i in range(n)]
    slots[3] = -1
    for parity in (0, 1):
        t = make_conv(cu[-1] + 9, C, dtype, n + 1, seed=70 + parity)
        t["u"][cu[-1]:] = float("nan")
        carry = [i % 2 == parity and i != 3 for i in range(n)]
        t["state"][[s for i, s in enumerate(slots) if not carry[i] and s >= 0]] = float("nan")
        before = t["state"].clone()
        plan = libssd.PackedPlan(cu, slots=slots, carry=carry, nslots=n + 1, heads=4)
        out = torch.full((cu[-1] + 9, C), 7.0, dtype=td(dtype), device="cuda")
        libssd.ssd_conv_packed_fwd(plan, t["u"], t["w"], t["bias"], t["state"], out=out)
        for i in range(n):
            past = f64(before[slots[i]]) if carry[i] else np.zeros((3, C))
            ref, size, last = conv_reference(f64(t["u"][cu[i]:cu[i + 1]]), f64(t["w"]), f64(t["bias"]), past)
            check_conv(out[cu[i]:cu[i + 1]], ref, size, dtype) if lens[i] else None
            if slots[i] >= 0:
                assert np.array_equal(f64(t["state"][slots[i]]), last)
        assert bool((out[cu[-1]:] == 7).all())
