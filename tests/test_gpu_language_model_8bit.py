"""The example model on products in 8 bits, with activations kept in 8 bits and with sampled tokens: the operators together, each against its definition in the
model's own calls."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1909_07729_amd import language_model
    torch.cuda.set_device(0)
    return torch, language_model


def _prompts(torch, module, count, longest=90):
    tokens, offsets, _ = module.documents(torch.Generator().manual_seed(2), count, 64, longest)
    return [tokens[a:b] for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist())]


@pytest.mark.parametrize("intervals", [32, 64])
def test_gradients_with_activations_in_8_bits(lm, intervals):
    """The MLP's function by itself: its value is that of the one that keeps all, its gradients are the products' at the restored values."""
    torch, module = lm
    binding, autograd = module.binding, module.autograd
    torch.manual_seed(0)
    h = (torch.randn(300, 1024, device="cuda") * 2).bfloat16().requires_grad_()
    weight = (torch.randn(256, 1024, device="cuda") / 32).bfloat16().requires_grad_()
    dz = torch.randn(300, 256, device="cuda").bfloat16()
    z = module._ActivatedLinear.apply(h, weight, intervals == 64)
    assert torch.equal(z, torch.nn.functional.linear(autograd.kgelu(h, intervals=intervals), weight))
    dh, dweight = torch.autograd.grad(z, (h, weight), dz)
    keep = "kgelu64_keep8" if intervals == 64 else "kgelu_keep8"
    _, codes, scales = getattr(binding, keep)(h.detach())
    kept = (codes.float().view(-1, 128) * scales[:, None]).view(300, 1024).bfloat16()
    name = "kgelu64" if intervals == 64 else "kgelu"
    assert torch.equal(dh, getattr(binding, name + "_backward")((dz @ weight).detach().contiguous(), kept))
    assert torch.equal(dweight, dz.t() @ getattr(binding, name)(kept))


def test_a_step_with_activations_in_8_bits(lm):
    """All parameters get gradients, near those of the step that keeps all: the restored values are off by half a step, 1/254 of their group's largest, in a
    function and a slope that change by about as much as their argument; 0.1 of the norm is ten times that."""
    torch, module = lm
    batch = module.documents(torch.Generator().manual_seed(3), 8, 64, 100)
    grads = []
    for keep in (None, 8):
        torch.manual_seed(1)
        model = module.LanguageModel(keep=keep)
        logits = model(*batch)
        torch.nn.functional.cross_entropy(logits, batch[0].roll(-1)).backward()
        grads.append([p.grad for p in model.parameters()])
    for a, b in zip(*grads):
        assert b.isfinite().all() and (a - b).norm() <= 0.1 * a.norm()


def _defined(torch, binding):
    """``kq8_linear`` by its definition: the integers of kq8_rows, exact sums in 64 bits, its Float32 operations."""
    def linear(x, weight, weight_scales, bias=None, *, activation=None, out_dtype=torch.bfloat16, rows=binding.kq8_rows):
        codes, scales = rows(x, activation)
        sums = (codes.double() @ weight.double().t()).float()
        return (sums * scales[:, None] * weight_scales).to(out_dtype)
    return linear


@pytest.mark.parametrize("intervals", [32, 64])
def test_serving_with_weights_in_8_bits(lm, monkeypatch, intervals):
    """The same logits, bit for bit, with the product's definition in its place; and near those of the weights as they are: the integers are off by at most
    1/254 of the largest of a row, a few hundredths of the norm after ten products."""
    torch, module = lm
    torch.manual_seed(1)
    model = module.LanguageModel(intervals=intervals)
    prompts, weights = _prompts(torch, module, 5), module.Weights8(model)
    made, logits = module.generate(model, prompts, 9, weights=weights)
    plain = module.generate(model, prompts, 1)[1]
    assert (logits[:, 0] - plain[:, 0]).norm() < 0.1 * plain[:, 0].norm()
    linear = _defined(torch, module.binding)
    monkeypatch.setattr(module.binding, "kq8_linear", linear)
    rows64 = module.binding.kq8_rows64
    monkeypatch.setattr(module.binding, "kq8_linear64", lambda *args, **options: linear(*args, **options, rows=rows64))
    again, want = module.generate(model, prompts, 9, weights=weights)
    assert torch.equal(made, again) and torch.equal(logits, want)


def test_sampled_tokens(lm):
    """Each token is the one that the settings and the generator's numbers choose from the step's logits."""
    torch, module = lm
    torch.manual_seed(1)
    model, prompts = module.LanguageModel(), _prompts(torch, module, 6)
    sample = {"temperature": 0.9, "top_k": 20, "top_p": 0.95, "min_p": 0.01, "cap": 30.0}
    made, logits = module.generate(model, prompts, 7, sample=sample, generator=torch.Generator("cuda").manual_seed(4), weights=module.Weights8(model))
    numbers = torch.Generator("cuda").manual_seed(4)
    for i in range(7):
        assert torch.equal(made[:, i], module.binding.ksample(logits[:, i], torch.rand(6, generator=numbers, device="cuda"), **sample))
    greedy, logits = module.generate(model, prompts, 3, sample={"temperature": 0.0})
    assert torch.equal(greedy, logits.argmax(-1))


def test_the_command(lm, capsys):
    torch, module = lm
    module.main(["--steps", "3", "--keep", "8", "--weights", "8", "--temperature", "0.8", "--top-p", "0.9"])
    assert "generated tokens" in capsys.readouterr().out
