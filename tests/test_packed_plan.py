"""Arguments of a plan."""
import numpy as np
import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from paper_2411_19460_b200 import libssd


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


@pytest.mark.parametrize("cu", [[0, 2.5, 4], torch.tensor([0.0, 3.7]), [0.0, float("nan")], np.array([0, 1.25])])
def test_rows_that_are_no_whole_numbers(cu):
    with pytest.raises(ValueError):
        libssd.PackedPlan(cu, heads=2, device="cpu")


@pytest.mark.parametrize("cu", [[0, 2, 4], torch.tensor([0, 2, 4], dtype=torch.int32), torch.tensor([0.0, 2.0, 4.0]), np.array([0, 2, 4]),
                                torch.tensor([0, 9, 2, 9, 4])[::2]])
def test_rows_of_any_type(cu):
    ref = libssd.PackedPlan([0, 2, 4], heads=2, device="cpu")
    assert torch.equal(libssd.PackedPlan(cu, heads=2, device="cpu").host, ref.host)
