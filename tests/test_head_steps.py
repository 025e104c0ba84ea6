"""A head's count of steps (CPU only: every update here is refused before a device call)."""
import pytest
import torch

import paper_2408_09697_amd as heta


def test_an_update_that_is_refused_is_no_step():
    head = heta.ClassifierHead(None, torch.zeros(4, 8), torch.zeros(8))
    with pytest.raises(RuntimeError):
        head.update()  # no gradients yet
    assert head.step == 0
    head.grads = {"W": torch.zeros(4, 8), "bias": torch.zeros(8)}
    with pytest.raises((heta.HetaError, TypeError, ValueError)):
        head.update()  # not on the device
    assert head.step == 0
