"""A distillation step whose calls are marshalled by ctypes: the same bits as through the extension."""
import pytest
import torch

from paper_1911_05146_b200 import binding, build
from test_gpu_distillation_run import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_same_step_through_ctypes(dtype, monkeypatch):
    one, other = Step(dtype), Step(dtype)
    one.run()
    monkeypatch.setattr(binding, "_calls", None)
    monkeypatch.setattr(build, "calls", lambda force=False: None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other.run()
    assert isinstance(binding._calls, binding._CtypesCalls)
    torch.cuda.synchronize()
    assert torch.equal(one.params, other.params) and torch.equal(one.loss, other.loss) and torch.equal(one.ids, other.ids)
