"""Gradients whose rows share memory, as those of a mean over time or over sequences do: backward passes only read them."""
import pytest
import torch

from tests import test_gpu_operators_convolution as convolution
from tests import test_gpu_operators_scan as scan

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def spread(t):
    """One row for all steps, one sequence for all, one row for everything."""
    for row in (t[:, :1], t[:1], t[:1, :1]):
        yield row.contiguous().expand(t.shape)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("shape", [(3, 5, 7), (2, 70, 130)])
def test_convolution_takes_a_gradient_of_one_row(shape, kind):
    s = convolution.make(*shape, 4, kind)
    for rows in spread(s["dout"]):
        assert not rows.is_contiguous()
        shared, whole = (convolution.backward({**s, "dout": d}, True) for d in (rows, rows.contiguous()))
        assert all(torch.equal(a, b) for a, b in zip(shared, whole))
        space = torch.empty(1 << 22, dtype=torch.uint8, device="cuda:0")
        assert all(torch.equal(a, b) for a, b in zip(convolution.backward({**s, "dout": rows}, True, workspace=space), whole))


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("shape", [(3, 5, 7), (2, 70, 130)])
def test_scan_takes_a_gradient_of_one_row(shape, kind):
    s = scan.make(*shape, 16, kind)
    for rows in spread(s["dout"]):
        shared, whole = (scan.backward({**s, "dout": d}) for d in (rows, rows.contiguous()))
        assert all(torch.equal(shared[k], whole[k]) for k in whole)
