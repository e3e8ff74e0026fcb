"""The windowed kernels under a budget of next to nothing: a wait that outlasts its polls may run out
anywhere, not at the first load alone. A call ends with its rows or with JET_ERR_TIMEOUT, never by
waiting, and the next call under the ordinary budget is the clean one's, bit for bit. (A poll
suspends by itself for longer than most waits take, so a call may well end with its rows.)"""
import pytest

from test_gpu_timeout import JET_ERR_TIMEOUT, JET_OK
from test_gpu_window import Prefill, Step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda(jet):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    yield jet
    jet.jet_set_wait_budget_ns(0)


def _hurried(cuda, call, budget_ns):
    old = cuda.jet_set_wait_budget_ns(budget_ns)
    try:
        call()
        return cuda.jet_device_status()
    finally:
        cuda.jet_set_wait_budget_ns(old)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_prefill_waits_that_run_out_anywhere(cuda, d):
    import torch
    p = Prefill(cuda, [3000, 70, 900], 16, 4, d, seed=3)
    ws = p.ws(700, 5)
    p.run(700, 5, ws=ws)
    first = p.o.clone()
    seen = [_hurried(cuda, lambda: cuda.jet_prefill_attend_window(
        p.dev, p.dims, 700, 5, p.q, p.k, p.v, p.o, ws), budget) for budget in (1, 1, 5000)]
    assert set(seen) <= {JET_OK, JET_ERR_TIMEOUT}
    p.o.fill_(7.0)
    p.run(700, 5, ws=ws)
    assert torch.equal(p.o, first)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_step_waits_that_run_out_anywhere(cuda, d):
    import torch
    s = Step(cuda, [3000] * 20 + [90], [2] * 21, [3, 2] * 21, 8, 2, d, True, seed=7)
    ws = s.ws(2000, 5)
    s.run(2000, 5, ws=ws)
    first = s.o.clone()
    seen = [_hurried(cuda, lambda: cuda.jet_prefix_attend_window(
        s.dev, s.dims, 2000, 5, s.q, s.k, s.v, s.kc, s.vc, s.o, ws), budget)
        for budget in (1, 1, 5000)]
    assert set(seen) <= {JET_OK, JET_ERR_TIMEOUT}
    s.o.fill_(7.0)
    s.run(2000, 5, ws=ws)
    assert torch.equal(s.o, first)
