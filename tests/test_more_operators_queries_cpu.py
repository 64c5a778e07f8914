"""The workspace queries take what their passes take, and refuse what they refuse (CPU only)."""
import ctypes as C

import pytest

from paper_2010_16248_amd import binding as B
from tests.test_more_operators_cpu import convolution, lib, pointers, refused, scan  # noqa: F401  (lib is a fixture)


@pytest.mark.parametrize("change", [dict(out_step=0), dict(out_batch=0), dict(out_step=0, out_batch=0), dict(out_step=3)])
def test_convolution_workspace_of_a_gradient_whose_rows_share_memory(lib, change):  # noqa: F811
    """The backward pass reads grad_out: it goes as far as its workspace, and the query has to tell its size."""
    cfg, n = convolution(**change), C.c_size_t(0)
    refused(lib, lib.accordion_convolution_backward(C.byref(cfg), *pointers(12), 0, None), "workspace", B.ACC_ENOSPACE)
    assert lib.accordion_convolution_workspace_bytes(C.byref(cfg), C.byref(n)) == B.ACC_OK and n.value > 0
    m = C.c_size_t(0)
    assert lib.accordion_convolution_workspace_bytes(C.byref(convolution()), C.byref(m)) == B.ACC_OK and n.value == m.value


@pytest.mark.parametrize("change,word", [(dict(grad_x_step=-4), "stride"), (dict(grad_x_step=3), "overlap"), (dict(grad_x_batch=0), "overlap")])
def test_convolution_workspace_of_a_gradient_that_cannot_be_written(lib, change, word):  # noqa: F811
    cfg, n = convolution(**change), C.c_size_t(0)
    refused(lib, lib.accordion_convolution_backward(C.byref(cfg), *pointers(12), 1 << 40, None), word)
    refused(lib, lib.accordion_convolution_workspace_bytes(C.byref(cfg), C.byref(n)), word)


def test_scan_workspace_of_a_gradient_whose_rows_share_memory(lib):  # noqa: F811
    n = C.c_size_t(0)
    for change in (dict(out_step=0), dict(out_batch=0), dict(out_step=0, out_batch=0)):
        assert lib.accordion_scan_workspace_bytes(C.byref(scan(**change)), 1, C.byref(n)) == B.ACC_OK and n.value > 0
