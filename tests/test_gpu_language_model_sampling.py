"""Tokens that the example model samples: through the model's own table."""
import pytest

from test_gpu_language_model_8bit import _prompts, lm  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("intervals", [32, 64])
def test_the_cap_goes_through_the_models_table(lm, monkeypatch, intervals):
    """A cap so low that the tables' values differ at most logits; only the model's own entry point is called."""
    torch, module = lm
    torch.manual_seed(1)
    model, prompts = module.LanguageModel(intervals=intervals), _prompts(torch, module, 6)
    sample = {"temperature": 0.2, "top_p": 0.95, "cap": 0.5}
    mine, other = (module.binding.ksample, "ksample64") if intervals == 32 else (module.binding.ksample64, "ksample")

    def refused(*args, **options):
        raise AssertionError("the other table's entry point")
    entry = module.binding.ksample                          # ksample64 calls it with its own name
    monkeypatch.setattr(module.binding, other, refused if other == "ksample64" else lambda *a, **o: entry(*a, **o) if "_entry" in o else refused())
    made, logits = module.generate(model, prompts, 7, sample=sample, generator=torch.Generator("cuda").manual_seed(4))
    numbers = torch.Generator("cuda").manual_seed(4)
    for i in range(7):
        assert torch.equal(made[:, i], mine(logits[:, i], torch.rand(6, generator=numbers, device="cuda"), **sample))


@pytest.mark.parametrize("weights", [False, True])
def test_logits_without_a_token(lm, weights):
    """``ksample`` answers -1, which an embedding would take as its last token."""
    torch, module = lm
    torch.manual_seed(1)
    model, prompts = module.LanguageModel(), _prompts(torch, module, 3)
    with torch.no_grad():
        model.head[5, 7] = float("nan")
    with pytest.raises(ValueError):
        module.generate(model, prompts, 4, sample={"temperature": 0.9, "top_k": 20}, weights=module.Weights8(model) if weights else None)
