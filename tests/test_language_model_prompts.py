"""Prompts that the example model refuses, on the host."""
import pytest
import torch

from paper_1909_07729_amd import language_model as lm


def test_prompts_without_tokens_are_refused():
    """Their logits would be memory that nothing has written."""
    model = lm.LanguageModel(vocabulary=16, width=32, layers=1, heads=2, kv_heads=1, dim=16, longest=64, device="cpu")
    some, none = torch.zeros(3, dtype=torch.long), torch.zeros(0, dtype=torch.long)
    for prompts in ([none], [some, none], [none, none]):
        with pytest.raises(ValueError):
            lm.generate(model, prompts, 5)
