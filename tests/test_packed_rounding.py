"""What the packed scan may round in bf16, on inputs whose products count: no D x that they hide behind, and scores and states of the size of x.
The only rounding of half a step is the result's own.

Limits, element by element, for abs_ = the sum of the sizes of all terms and products = that without |D x| (tests/test_packed.py):
 2^-8 |y|          the result's rounding to bf16, half a step
 2^-16 products    the masked scores and the state in front of a block are operands of two bf16 parts each, a and b: a is off by half a step, 2^-8 of
                   the value, b holds that and is off by 2^-8 of it
 (64 + 2 chunks) 2^-24 abs_   sums, exponentials and decays, as there
With one part instead of two the second line would be 2^-8 products: more than the whole limit wherever the terms cancel to a fraction of their sizes."""
import numpy as np
import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from paper_2411_19460_b200 import libssd
from tests.test_packed import P, f64, make, reference


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


def inputs(lens, H, G, N, seed, size, D, strong):
    """B and C of `size`, made anew (those of make() are divided by sqrt(N))."""
    t = make(lens, H, G, N, "bf16", seed=seed, strong=strong)
    g = torch.Generator().manual_seed(seed + 1000)
    for k in ("Bm", "Cm"):
        t[k].copy_((torch.randn(t[k].shape, generator=g) * size).to(torch.bfloat16))
    if not D:
        t["D"].zero_()
    return t


def check(t, y, carry, before):
    cu = t["cu"]
    for i in range(len(cu) - 1):
        a, b = cu[i], cu[i + 1]
        h0 = f64(before[i]) if carry[i] else np.zeros(before.shape[1:])
        ref, _, (size, products), _ = reference(t, a, b, h0)
        off = np.abs(f64(y[a:b]) - ref)
        lim = 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * products + (64 + 2 * ((b - a + 63) // 64)) * 2.0 ** -24 * size
        assert np.all(off <= lim + 1e-30), (i, float(np.max(off / (lim + 1e-30))))


@pytest.mark.gpu
@pytest.mark.parametrize("strong", [False, True])
@pytest.mark.parametrize("size,D", [(1.0, False), (1.0, True), (0.1, False)])
@pytest.mark.parametrize("H,G,N,lens", [
    (3, 1, 128, [700, 129, 37]),           # a head per CTA
    (4, 2, 64, [700, 129, 37]),
    (60, 4, 128, [300, 129, 1, 37]),       # two heads per CTA, the last of a group alone
    (40, 1, 64, [200, 129, 1, 37]),
    (2, 1, 128, [5000]),                   # cut into ranges
])
def test_products_are_rounded_with_the_result_only(H, G, N, lens, size, D, strong):
    t = inputs(lens, H, G, N, 5, size, D, strong)
    carry = [i % 2 == 0 for i in range(len(lens))]
    before = t["state"].clone()
    plan = libssd.PackedPlan(t["cu"], carry=carry, heads=H)
    y = libssd.ssd_packed_fwd(plan, t["x"], t["dt"], t["A"], t["Bm"], t["Cm"], t["D"], t["state"])
    check(t, y, carry, before)


@pytest.mark.gpu
def test_error_is_that_of_one_rounding():
    """Root mean square of the error over all elements, D = 0, against that of the exact result rounded to bf16, the smallest that y can have (1.66e-3 of
    the result).  The terms of an element have either sign, so that the root of the sum of their squares is about the result's size: operands of two parts,
    off by 2^-16 at most, add 1e-5 of the result in quadrature, nothing; of one part, off by up to 2^-8 (1.66e-3 like the result's own), 40 %."""
    t = inputs([1500], 4, 1, 128, 7, 0.1, False, False)
    before = t["state"].clone()
    plan = libssd.PackedPlan(t["cu"], carry=[True], heads=4)
    y = f64(libssd.ssd_packed_fwd(plan, t["x"], t["dt"], t["A"], t["Bm"], t["Cm"], t["D"], t["state"]))
    ref = reference(t, 0, 1500, f64(before[0]))[0]
    own = f64(torch.from_numpy(ref).to(torch.bfloat16))
    assert y.shape == (1500, 4, P)
    assert np.sqrt(np.mean((y - ref) ** 2)) <= 1.01 * np.sqrt(np.mean((own - ref) ** 2))
