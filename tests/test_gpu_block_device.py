"""The recurrent block's operators refuse tensors of a GPU other than the current one: the call runs on
the current GPU's stream, and its kernels would read another GPU's memory."""
import pytest
import torch

import paper_1810_09958_amd as isam

pytestmark = pytest.mark.gpu


def test_tensors_of_another_gpu_are_refused(monkeypatch):
    x, W, D = torch.zeros((4, 8), device="cuda"), torch.zeros((16, 8), device="cuda"), torch.ones(8, device="cuda")
    gx = torch.zeros((4, 1, 16), device="cuda")
    states = torch.zeros((1, 1, 8), device="cuda")
    calls = [lambda: isam.linear_gru(gx), lambda: isam.linear_gru_backward(gx, None, states=states),
             lambda: isam.norm_residual(None, x, w_pre=D), lambda: isam.norm_residual_backward(None, x, x, w_pre=D),
             lambda: isam.gated_ffn(x, W), lambda: isam.gated_ffn_backward(x, W, x)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    here = torch.cuda.current_device()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: here + 1)
    monkeypatch.setattr(isam, "lib", lambda: pytest.fail("the library was called"))
    for call in calls:
        with pytest.raises(ValueError):
            call()
