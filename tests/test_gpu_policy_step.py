"""The example step: its operators train, and its memory is what the estimate says."""
import importlib.util
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu


def example():
    path = Path(__file__).resolve().parents[1] / "examples" / "policy_step.py"
    spec = importlib.util.spec_from_file_location("policy_step", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("hidden,layers,vocab,tokens", [(256, 4, 1024, 512), (136, 2, 1021, 77)])
def test_step_trains_and_its_peak_is_estimated(hidden, layers, vocab, tokens):
    got = example().train(hidden, layers, vocab, tokens, steps=4)
    print(got, flush=True)
    # the first step's ratios are 1, its KL term 0: the loss is minus the mean advantage; then it falls
    assert got["loss"][-1] < got["loss"][0]
    assert got["gained"][0] > 0 > got["gained"][1]
    # every tensor of the step is in the trace; the device's allocator hands out blocks up to 1 MiB too large unsplit
    assert got["estimated"][0] <= got["measured"][0] <= 1.05 * got["estimated"][0] + 2**20
    assert got["estimated"][1] >= got["estimated"][0]
