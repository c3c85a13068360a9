"""A status call tells what the calls enqueued so far have left, on whichever stream they run."""
import pytest
import torch

import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("given_up", [False, True])
def test_linear_status_waits_for_a_stream_that_does_not_block(given_up):
    """A report that is still to be written (here by a fill, as a kernel's wait that gives up writes it) behind 0.2 s of work on such a stream."""
    scratch = torch.zeros(256, dtype=torch.uint8, device=DEV)
    value = torch.ones(1, dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    scratch[:1].copy_(value * 0)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(400_000_000)
        if given_up:
            scratch[:1].copy_(value)
    assert hpf.linear_status(scratch) is given_up
    assert s.query()


@pytest.mark.parametrize("given_up", [False, True])
def test_bnrelu_status_waits_for_a_stream_that_does_not_block(given_up):
    """The same of the BN+ReLU call, whose report is the third word of its scratch."""
    scratch = torch.zeros(256, dtype=torch.uint8, device=DEV)
    value = torch.ones(1, dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    scratch[8:9].copy_(value * 0)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(400_000_000)
        if given_up:
            scratch[8:9].copy_(value)
    assert hpf.bnrelu_status(scratch) is given_up
    assert s.query()
