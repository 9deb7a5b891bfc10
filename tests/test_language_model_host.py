"""What the example model checks and plans on the host: texts that its angles and its cache hold, and the columns of the page table that
a call needs.  The operators are replaced by stand-ins that run on the CPU."""
import pytest
import torch

from paper_1909_07729_amd import language_model as lm


@pytest.fixture
def model():
    torch.manual_seed(0)
    return lm.LanguageModel(vocabulary=16, width=32, layers=2, heads=2, kv_heads=1, dim=16, longest=64, device="cpu")


def test_texts_longer_than_the_angles_are_refused(model):
    with pytest.raises(ValueError):
        lm.train(model, 1, longest=65)
    with pytest.raises(ValueError):
        lm.generate(model, [torch.zeros(3, dtype=torch.long), torch.zeros(60, dtype=torch.long)], 5)


def test_calls_look_at_the_pages_that_the_longest_sequence_needs(model, monkeypatch):
    seen = []

    def paged(q, k_cache, v_cache, pages, lengths, offsets=None, *, cap):
        seen.append((pages.shape[1], int(lengths.max())))
        return q
    monkeypatch.setattr(lm.binding, "kcap_append", lambda q, *rest, **options: q)
    monkeypatch.setattr(lm.binding, "kcap_attention_paged", paged)
    monkeypatch.setattr(lm.autograd, "kgelu", lambda h, intervals: torch.nn.functional.gelu(h))
    cache = lm.PagedCache(2, 3, 60, 1, 16, page=8, device="cpu")
    assert cache.pages.shape == (3, 8) and sorted(cache.pages.flatten().tolist()) == list(range(24))
    model.serve(torch.zeros(20, dtype=torch.long), cache, torch.tensor([0, 4, 4, 20], dtype=torch.int32), longest=16)
    model.serve(torch.zeros(3, dtype=torch.long), cache)
    model.serve(torch.zeros(30, dtype=torch.long), cache, torch.tensor([0, 30, 30, 30], dtype=torch.int32))
    assert [s[0] for s in seen] == [2, 2, 3, 3, 6, 6]       # of 16, 17 and at most 47 keys
    assert all(longest <= columns * 8 for columns, longest in seen)
    with pytest.raises(ValueError):
        model.serve(torch.zeros(18, dtype=torch.long), cache, torch.tensor([0, 0, 0, 18], dtype=torch.int32), longest=18)
    assert cache.lengths.tolist() == [35, 1, 17]            # what is refused leaves the cache as it is
    model.serve(torch.zeros(18, dtype=torch.long), cache, torch.tensor([0, 6, 12, 18], dtype=torch.int32))
    assert cache.lengths.tolist() == [41, 7, 23] and seen[-1] == (8, 41)
