"""The example model runs the operators together: it learns, and serving from the paged cache gives the training pass's logits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1909_07729_amd import language_model
    torch.cuda.set_device(0)
    return torch, language_model


def test_it_learns_to_repeat(lm):
    torch, module = lm
    torch.manual_seed(0)
    losses = module.train(module.LanguageModel(), 150)
    assert losses[0] > 3.5 and sum(losses[-5:]) / 5 < 0.5 * losses[0], (losses[0], losses[-5:])


@pytest.mark.parametrize("intervals", [32, 64])
def test_serving_gives_the_logits_of_the_training_pass(lm, intervals):
    """A prompt in pieces and then token by token, ragged, against one pass over prompt and continuation.  The two round at
    different places (weights of one token are not rounded to BFloat16), each by 2^-8 of BFloat16 values through two layers."""
    torch, module = lm
    torch.manual_seed(1)
    model = module.LanguageModel(intervals=intervals)
    tokens, offsets, _ = module.documents(torch.Generator().manual_seed(2), 5, 64, 90)
    prompts = [tokens[a:b] for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist())]
    made, logits = module.generate(model, prompts, 9)
    for prompt, new, served in zip(prompts, made, logits):
        text = torch.cat([prompt, new])
        at = torch.tensor([0, len(text)], dtype=torch.int32, device="cuda")
        with torch.no_grad():
            whole = model(text, at, torch.arange(len(text), device="cuda"))[len(prompt) - 1:-1]
        assert (whole - served).norm() / whole.norm() < 0.03
