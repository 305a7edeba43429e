"""The sampler and the distillation loss at the edges of what they take."""
import math

import numpy as np
import pytest
import torch

import test_gpu_distill as td
import test_gpu_sample as ts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ps():
    from paper_2603_19133_amd import binding
    return binding


def test_a_vocabulary_wider_than_the_view_is_refused(gpu, ps):
    """... by the forward call (the backward call, whose gradient has the view's columns, would be the first to notice)."""
    from paper_2603_19133_amd.training import distill_loss
    z = torch.zeros(4, 108, device="cuda")[:, :100]
    rec = ps.Compressed(torch.zeros(4, 5, dtype=torch.int32, device="cuda"), torch.ones(4, 5, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda"),
                        torch.ones(4, device="cuda"), torch.zeros(4, device="cuda"), 5)
    for call in (lambda v: distill_loss(z, rec, v, 1.0), lambda v: ps.distill(z, v, 1.0, rec), lambda v: ps.sample(z, v, torch.zeros(4, device="cuda"))):
        with pytest.raises(ps.PicoSpecError):
            call(101)
        call(100)
    torch.cuda.synchronize()
