"""Attention under a window where outputs come out NaN or infinite and are computed again from what
their rows see alone: in the step's chunks, beside keys that a row does not see, and under windows
long enough for the second computation to take its time."""
import pytest

from test_gpu_window import Step, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda(jet):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    yield jet
    jet.jet_set_wait_budget_ns(0)


@pytest.mark.parametrize("d,heads", [(64, (8, 8)), (128, (16, 2)), (256, (16, 2))])
def test_outputs_of_chunks_are_stored_once(cuda, d, heads):
    """Every row of a long window in chunks is computed again, as a key beside the first tokens is
    NaN: each output is the second computation's, call after call."""
    import torch
    P, window, sinks = 20000, 6000, 20
    s = Step(cuda, [P], [3], [5, 3, 9], *heads, d, True, seed=21)
    s.v[25] = s.k[25] = float("nan")   # seen by no row, loaded with the first ones
    ws = s.ws(window, sinks)
    s.run(window, sinks, ws=ws)
    s.check(window, sinks)
    first = s.o.clone()
    for _ in range(10):
        s.o.fill_(7.0)
        s.run(window, sinks, ws=ws)
        assert torch.equal(s.o, first)
