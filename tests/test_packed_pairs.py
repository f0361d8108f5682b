"""The packed scan with two heads per CTA, as batches of many heads have it (bf16; more heads of sequences and ranges than SMs): both launches of cut
sequences, groups of an odd number of heads, whose last CTA has one, both state sizes, empty sequences and ones of a row, neighbours that are not finite.
References, limits and inputs are those of tests/test_packed.py and test_packed_rounding.py."""
import numpy as np
import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from paper_2411_19460_b200 import libssd
from tests import test_packed_rounding as rounding
from tests.test_packed import check, check_all, make, reference
from tests.test_packed_ranges import call, header, plan_of

SMS = 148
CUT = [(27, 3, 128, [2000, 1, 0, 129]), (33, 1, 64, [2500, 60, 2000]), (40, 8, 64, [2000, 1, 0, 129]), (40, 8, 128, [2000, 1, 0, 129]), (40, 1, 128, [3000, 50])]
WHOLE = [(65, 13, 64, [300, 129, 1, 0, 128, 37, 70, 33]), (65, 13, 128, [300, 129, 1, 0, 128, 37, 70, 33]), (48, 1, 64, [257, 2, 600, 0, 64]),
         (45, 5, 128, [257, 2, 600, 0, 64])]


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


def pairs(plan, heads, cut):
    units, sums = header(plan)
    assert units * heads > SMS and (sums > 0) == cut
    return plan


@pytest.mark.parametrize("cut,H,G,N,lens", [(True,) + c for c in CUT] + [(False,) + c for c in WHOLE])
def test_the_cases_are_of_two_heads_per_cta(cut, H, G, N, lens):
    pairs(libssd.PackedPlan([0] + list(np.cumsum(lens)), heads=H, device="cpu"), H, cut)


@pytest.mark.gpu
@pytest.mark.parametrize("strong", [False, True])
@pytest.mark.parametrize("cut,H,G,N,lens", [(True,) + c for c in CUT] + [(False,) + c for c in WHOLE])
def test_against_the_oracle(cut, H, G, N, lens, strong):
    n = len(lens)
    t = make(lens, H, G, N, "bf16", seed=61, behind=7, nslots=n + 2, strong=strong)
    slots = [n + 1 - i for i in range(n)]
    carry = [i % 2 == 0 for i in range(n)]
    if n > 3:
        slots[1], carry[1] = -1, False
    before = t["state"].clone()
    plan = pairs(plan_of(t, slots, carry), H, cut)
    ws = libssd.alloc_packed_workspace(plan, t["x"], t["Bm"])
    ws.fill_(255)
    y = torch.full(t["x"].shape, 7.0, dtype=torch.bfloat16, device="cuda")
    call(plan, t, y=y, ws=ws)
    torch.cuda.synchronize()
    assert libssd.poll_status(ws) == libssd.SSD_OK
    check_all(t, y, before, t["state"], slots, carry, "bf16")
    assert bool((y[t["cu"][-1]:] == 7).all())
    free = [s for s in range(n + 2) if s not in slots]
    assert torch.equal(t["state"][free], before[free])
    after = t["state"].clone()
    t["state"].copy_(before)
    assert torch.equal(call(plan, t, y=torch.full_like(y, 7.0)), y) and torch.equal(t["state"], after)


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,N,lens", [CUT[0], CUT[1], WHOLE[2]])
def test_products_are_rounded_with_the_result_only(H, G, N, lens):
    t = rounding.inputs(lens, H, G, N, 62, 1.0, False, False)
    carry = [i % 2 == 0 for i in range(len(lens))]
    before = t["state"].clone()
    y = call(plan_of(t, None, carry), t)
    rounding.check(t, y, carry, before)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("H,G,N,lens,bad", [(40, 8, 128, [2000, 500, 129], 1), (33, 1, 64, [2000, 500, 60], 0), (65, 13, 64, [70, 130, 33, 257, 64, 1], 3)])
def test_neighbours_that_are_not_finite(H, G, N, lens, bad, value):
    t = make(lens, H, G, N, "bf16", seed=63, behind=200)
    a, b = t["cu"][bad], t["cu"][bad + 1]
    for k in ("x", "Bm", "Cm", "dt"):
        t[k][a:b] = value
        t[k][t["cu"][-1]:] = value
    carry = [i % 2 == 0 for i in range(len(lens))]
    t["state"][[i for i in range(len(lens)) if not carry[i]]] = value
    before = t["state"].clone()
    y = torch.zeros(t["x"].shape, dtype=torch.bfloat16, device="cuda")
    call(plan_of(t, None, carry), t, y=y)
    check_all(t, y, before, t["state"], list(range(len(lens))), carry, "bf16", skip=[bad])
    assert not bool(torch.isfinite(y[a:b].float()).any()) and bool((y[t["cu"][-1]:] == 0).all())


@pytest.mark.gpu
def test_one_head_that_is_not_finite_leaves_the_other():
    """Of a pair: the first head's x is NaN from a row on, the second one's not, and the other way round."""
    for bad in (0, 1):
        t = make([700, 40], 150, 1, 128, "bf16", seed=64)
        t["x"][300:, bad] = float("nan")
        y = call(plan_of(t), t)
        good = [h for h in range(150) if h != bad]
        sub = dict(t, x=t["x"][:, good], dt=t["dt"][:, good], A=t["A"][good], D=t["D"][good])
        for i in range(2):
            ry, rh, ya, ha = reference(sub, t["cu"][i], t["cu"][i + 1], np.zeros((149, 64, 128)))
            check("y", y[t["cu"][i]:t["cu"][i + 1]][:, good], ry, ya, 11, "bf16")
            check("state", t["state"][i][good], rh, ha, 11, "fp32")
        assert not bool(torch.isfinite(y[300:, bad].float()).any())
