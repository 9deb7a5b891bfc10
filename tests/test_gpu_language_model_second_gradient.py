"""A second gradient through an MLP that keeps 8 bits: an error, not the part of it that torch's products would give."""
import pytest

from test_gpu_language_model_8bit import lm  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("intervals", [32, 64])
def test_second_gradients_raise(lm, intervals):
    torch, module = lm
    torch.manual_seed(0)
    h = torch.randn(300, 1024, device="cuda").bfloat16().requires_grad_()
    weight = (torch.randn(256, 1024, device="cuda") / 32).bfloat16().requires_grad_()
    for dz in (torch.randn(300, 256, device="cuda").bfloat16(), torch.randn(300, 256, device="cuda").bfloat16().requires_grad_()):
        z = module._ActivatedLinear.apply(h, weight, intervals == 64)
        dh, dweight = torch.autograd.grad(z, (h, weight), dz, create_graph=True)
        for gradient in (dh, dweight):
            for of in (h, weight, dz):
                with pytest.raises(RuntimeError):
                    torch.autograd.grad(gradient.float().square().sum(), of, retain_graph=True)
        # the values are those of an ordinary step
        again = torch.autograd.grad(module._ActivatedLinear.apply(h, weight, intervals == 64), (h, weight), dz)
        assert torch.equal(dh.detach(), again[0]) and torch.equal(dweight.detach(), again[1])
