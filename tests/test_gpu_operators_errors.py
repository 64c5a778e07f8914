"""What other HIP calls of the thread left behind as their error is not an operator's."""
import ctypes as C

import pytest
import torch

from paper_2010_16248_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _runtime():
    """The HIP runtime of this process."""
    with open("/proc/self/maps") as f:
        paths = {line.split()[-1] for line in f if "libamdhip64" in line}
    assert len(paths) == 1, paths
    return C.CDLL(paths.pop())


def test_an_older_error_of_the_thread_is_not_an_operators():
    torch.zeros(1, device=DEV)
    B.load_library()
    hip = _runtime()
    x, w, y = torch.randn(700, 40, device=DEV), torch.ones(40, device=DEV), torch.empty(700, 40, device=DEV)
    ids, table = torch.arange(700, device=DEV) % 30, torch.zeros(30, 40, device=DEV)
    workspace = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    weights, grads, state = [torch.ones(500, device=DEV)], [torch.ones(500, device=DEV)], B.adamw_state([500], 32, DEV)
    steps = x.view(7, 100, 40)
    torch.cuda.synchronize()
    failures = []
    for call in (lambda: B.layernorm_forward(x, w, None, y), lambda: B.embedding_forward(ids, table, y),
                 lambda: B.embedding_backward(ids, x, table, workspace=workspace, accumulate=True),
                 lambda: B.recurrence_forward(steps, steps, y.view(7, 100, 40), workspace=workspace),
                 lambda: B.adamw_step(weights, grads, state, 0.1, 1)):
        assert hip.hipSetDevice(9999) != 0            # no such device: an error that nobody has asked for yet
        try:
            call()
        except B.AccordionError as e:
            failures.append(str(e))
        hip.hipGetLastError()
    torch.cuda.synchronize()
    assert not failures
    assert weights[0].eq(weights[0][0]).all() and abs(float(weights[0][0]) - 0.9) < 1e-6
    ref = torch.zeros(30, 40, dtype=torch.float64).index_add_(0, ids.cpu(), x.double().cpu())
    assert (table.double().cpu() - ref).abs().max() < 1e-4
