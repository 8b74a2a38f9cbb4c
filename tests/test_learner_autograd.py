"""The operators record no gradient of their own: a tensor that asks for one is refused, not silently detached."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_1509_04210_b200 import learner


def _calls(x):
    """Calls with x in every place a matrix goes; on the CPU all of them are refused for one reason or another."""
    return [lambda: learner.mx4_quantize(x), lambda: learner.mx4_quantize(x, transpose=True), lambda: learner.act8_save(x),
            lambda: learner.act8_forward("gelu", x)]


def test_tensors_that_require_a_gradient_are_refused():
    for call in _calls(torch.zeros(4, 32, requires_grad=True)):
        with pytest.raises(ValueError, match="requires a gradient.*no_grad"):
            call()


def test_dual_tensors_are_refused():
    with fwd.dual_level():
        for call in _calls(fwd.make_dual(torch.zeros(4, 32), torch.ones(4, 32))):
            with pytest.raises(ValueError, match="requires a gradient|tangent"):
                call()


def test_they_are_taken_where_no_gradient_is_recorded():
    x = torch.zeros(4, 32, requires_grad=True)
    for wrap in (torch.no_grad, torch.inference_mode):
        with wrap():
            for call in _calls(x):
                with pytest.raises(ValueError, match="on the GPU is wanted"):      # the next thing that is checked
                    call()
    for call in _calls(x.detach()):
        with pytest.raises(ValueError, match="on the GPU is wanted"):
            call()


@pytest.mark.gpu
def test_every_matrix_on_the_gpu():
    x = torch.ones(40, 64, device="cuda")
    r = x.clone().requires_grad_()
    q, saved = learner.mx4_quantize(x), learner.act8_save(x)
    calls = [lambda t: learner.mx4_quantize(t), lambda t: learner.mx4_dequantize(q, out=t), lambda t: learner.mx4_matmul(t, q),
             lambda t: learner.mx4_matmul(t, q, out=torch.empty(40, 40, device="cuda")), lambda t: learner.act8_save(t),
             lambda t: learner.act8_values(saved, out=t), lambda t: learner.act8_forward("silu", t), lambda t: learner.act8_forward("swiglu", x, t),
             lambda t: learner.act8_forward("silu", x, out=t), lambda t: learner.act8_backward("silu", t, saved),
             lambda t: learner.act8_backward("silu", x, saved, out=t), lambda t: learner.act8_backward("swiglu", x, saved, saved, out_up=t),
             lambda t: learner.act8_weight_grad(t, saved)]
    for call in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            call(r)
        with torch.no_grad():
            call(r.clone())
        call(x.clone())
    learner.sync()
