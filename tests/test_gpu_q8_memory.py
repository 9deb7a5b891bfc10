"""Outputs of calls on 8-bit integers beside what they read in one buffer, and over it."""
import pytest

from test_gpu_q8 import _codes, _scales, _x, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, inner, outer", [(2, 64, 64), (8, 512, 512), (300, 512, 512)])
@pytest.mark.parametrize("host", [True, False])
def test_one_buffer(gpu, monkeypatch, rows, inner, outer, host):
    torch, binding = gpu
    weight, weight_scales = _codes(torch, outer, inner, 1), _scales(torch, outer, 2)
    if not host:
        monkeypatch.setattr(binding, "_host", None)
    buffer = torch.zeros((rows, inner + outer), dtype=torch.bfloat16, device="cuda")
    x, out = buffer[:, :inner], buffer[:, inner:]
    x.copy_(_x(torch, rows, inner, torch.bfloat16, 3))
    kept = x.clone()
    want = binding.kq8_linear(kept, weight, weight_scales, activation="gelu")
    assert binding.kq8_linear(x, weight, weight_scales, activation="gelu", out=out).data_ptr() == out.data_ptr()
    assert torch.equal(out, want) and torch.equal(x, kept)
    codes, scales = binding.kq8_rows(x)
    bias, row_scales = kept.view(-1)[:2 * outer].view(torch.float32), kept.view(-1)[:2 * rows].view(torch.float32)
    for call in (lambda: binding.kq8_linear(kept, weight, weight_scales, out=kept), lambda: binding.kq8_linear(x, weight, weight_scales, out=buffer[:, inner - 1:-1]),
                 lambda: binding.kq8_linear(x, weight, weight_scales, bias, out=kept), lambda: binding.kq8_product(codes, row_scales, weight, weight_scales, out=kept),
                 lambda: binding.kq8_rows(kept, codes=kept.view(torch.int8)[:, :inner]), lambda: binding.kq8_rows(kept, scales=row_scales)):
        with pytest.raises(binding.KtanhError):
            call()
    assert torch.equal(x, kept)         # nothing was launched
