"""Infinities in the fp32 scan of packed prompts: parts of an infinity times parts of the other operand, which are of either sign, are NaN; the
formulas have infinities there, whose sign the inputs say.  What an infinity does not reach keeps its bits."""
import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from tests.test_packed import make
from tests.test_packed_ranges import call, header, plan_of

CHUNK = 64          # rows whose products are taken at once: from its row to the end of these an infinity of x or B is one term of a sum


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


def run(t, carry, state, **kw):
    t = dict(t, state=state.clone(), **kw)
    y = torch.full(t["x"].shape, 7.0, device="cuda")
    call(plan_of(t, None, carry), t, y=y)
    return y, t["state"]


def expect(got, signs, inf, what):
    assert torch.equal(got.double(), (torch.sign(signs) * inf).expand_as(got).double()), what


@pytest.mark.gpu
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("N,lens,at", [(64, [40, 300, 70], 200), (128, [40, 300, 70], 200), (128, [40, 5000, 70], 3000), (64, [40, 5000, 70], 3000)])
def test_infinities_come_out_as_infinities(N, lens, at, sign):
    t = make(lens, 3, 1, N, "fp32", seed=71)
    carry, state, inf = [True] * 3, t["state"].clone(), sign * float("inf")
    assert (header(plan_of(t, None, carry))[1] > 0) == (lens[1] > 1000)
    y0, s0 = run(t, carry, state)
    first, end, row, h, p, n = 40, 40 + lens[1], 40 + at, 1, 7, 9
    last = 40 + (at // CHUNK + 1) * CHUNK
    B, C = t["Bm"][:, 0].double(), t["Cm"][:, 0].double()
    others, keep, rest = [i for i in range(64) if i != p], [i for i in range(N) if i != n], list(range(first)) + list(range(end, sum(lens)))

    x = t["x"].clone()
    x[row, h, p] = inf
    y, s = run(t, carry, state, x=x)
    expect(y[row + 1:last, h, p], C[row + 1:last] @ B[row], inf, "x -> y")
    expect(s[1, h, p], B[row], inf, "x -> state")
    assert torch.equal(y[:, h, others], y0[:, h, others]) and torch.equal(y[:, [0, 2]], y0[:, [0, 2]]) and torch.equal(y[rest], y0[rest])
    assert torch.equal(y[first:last - CHUNK], y0[first:last - CHUNK])
    assert torch.equal(s[1, h, others], s0[1, h, others]) and torch.equal(s[[0, 2]], s0[[0, 2]]) and torch.equal(s[1, [0, 2]], s0[1, [0, 2]])

    Bm = t["Bm"].clone()
    Bm[row, 0, n] = inf
    y, s = run(t, carry, state, Bm=Bm)
    xr = t["x"][row].double()
    expect(y[row + 1:last], torch.sign(C[row + 1:last, n])[:, None, None] * torch.sign(xr)[None], inf, "B -> y")
    expect(s[1, :, :, n], xr, inf, "B -> state")
    assert torch.equal(s[1][:, :, keep], s0[1][:, :, keep]) and torch.equal(s[[0, 2]], s0[[0, 2]])
    assert torch.equal(y[first:last - CHUNK], y0[first:last - CHUNK]) and torch.equal(y[rest], y0[rest])

    Cm = t["Cm"].clone()
    Cm[row, 0, n] = inf                                  # its row alone, and no state
    y, s = run(t, carry, state, Cm=Cm)
    same = [i for i in range(sum(lens)) if i != row]
    assert torch.equal(y[same], y0[same]) and torch.equal(s, s0) and not bool(torch.isfinite(y[row]).any())

    carried = state.clone()
    carried[1, h, p, n] = inf
    y, s = run(t, carry, carried)
    expect(y[first:first + CHUNK, h, p], C[first:first + CHUNK, n], inf, "state -> y")
    assert s[1, h, p, n] == inf and torch.equal(s[1, h, p, keep], s0[1, h, p, keep])
    assert torch.equal(y[:, h, others], y0[:, h, others]) and torch.equal(y[:, [0, 2]], y0[:, [0, 2]]) and torch.equal(y[rest], y0[rest])


@pytest.mark.gpu
def test_nan_stays_nan():
    t = make([300, 70], 2, 1, 64, "fp32", seed=72)
    state = t["state"].clone()
    y0, s0 = run(t, [False, True], state)
    x = t["x"].clone()
    x[200, 1, 7] = float("nan")
    y, s = run(t, [False, True], state, x=x)
    assert bool(y[200:300, 1, 7].isnan().all()) and bool(s[0, 1, 7].isnan().all())
    assert torch.equal(y[:192], y0[:192]) and torch.equal(y[300:], y0[300:]) and torch.equal(y[:, 0], y0[:, 0]) and torch.equal(s[1], s0[1])
