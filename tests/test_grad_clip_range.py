"""Clipping at the ends of fp32's range: norms above its largest value, factors below its smallest normal one.  References in 64 bits.

Limits: as in tests/test_grad_clip.py, 2^-21 of the result and half a step of its type, where results are normal numbers; a result below fp32's normal
numbers is off by half of its smallest one, 2^-150 (bf16: 2^-134)."""
import math

import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from paper_2411_19460_b200 import libssd


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


def norm_of(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def check(outs, grads, max_norm):
    scale = float(torch.tensor(max_norm, dtype=torch.float32)) / norm_of(grads)
    assert scale < 1
    for o, g in zip(outs, grads):
        exact = g.double() * scale
        bf16 = g.dtype == torch.bfloat16
        lim = exact.abs() * (2.0 ** -21 + (2.0 ** -8 if bf16 else 2.0 ** -24)) + 2.0 ** (-134 if bf16 else -150) * 1.001
        assert bool(((o.double() - exact).abs() <= lim).all()), float(((o.double() - exact).abs() / lim).max())


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("size,max_norm", [(3e38, 1.0), (3e38, 1e30), (2.5e38, 1e-3), (1e37, 1e-3), (1e37, 0.05), (3e38, 3.4e38), (1e10, 1e-30)])
def test_norms_and_factors_at_the_ends(size, max_norm, in_place):
    g = torch.Generator().manual_seed(1)
    grads = [((torch.rand(n, generator=g) * 2 - 1) * size).to(torch.bfloat16 if i % 2 else torch.float32).cuda() for i, n in enumerate([5000, 333, 7, 20001])]
    grads[0][:40] = torch.logspace(-30, 30, 40)
    before = [v.clone() for v in grads]
    outs = grads if in_place else [torch.full_like(v, 9.0) for v in grads]
    norm = float(libssd.ssd_grad_clip(grads, max_norm, out=None if in_place else outs))
    exact = norm_of(before)
    assert norm == math.inf if exact > 3.5e38 else abs(norm - exact) <= 2.0 ** -21 * exact
    check(outs, before, max_norm)


@pytest.mark.gpu
def test_a_norm_above_fp32_and_no_limit():
    grads = [torch.full((1000,), 3e38, device="cuda")]
    assert float(libssd.ssd_grad_clip(grads, math.inf)) == math.inf and bool((grads[0] == 3e38).all())
    assert float(libssd.ssd_grad_clip(grads, 0.0)) == math.inf and bool((grads[0] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_zeros_among_the_gradients(dtype):
    """Zeros of either sign, whole vectors and chunks of them, and next to squares that leave fp32: the same norm as without them."""
    g = torch.Generator().manual_seed(2)
    for scale in (1.0, 1e-25):
        v = (torch.randn(40000, generator=g) * scale).to(dtype)
        v[:9000] = 0
        v[20000:20016] = -0.0
        v[20024:20031] = 0
        v[30000:30007] = 0
        got = float(libssd.ssd_grad_clip([v.cuda(), torch.zeros(50000, dtype=dtype, device="cuda")], math.inf))
        assert abs(got - norm_of([v])) <= 2.0 ** -21 * norm_of([v])


@pytest.mark.gpu
def test_an_output_has_its_gradients_shape():
    g = torch.randn(6, 8, device="cuda")
    for shape in ((48,), (8, 6), (1, 6, 8)):
        with pytest.raises(ValueError):
            libssd.ssd_grad_clip([g], 1.0, out=[torch.empty(shape, device="cuda")])
