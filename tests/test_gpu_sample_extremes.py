"""The choice of the next token where its arithmetic could leave Float32, against the definition in 64 bits: equal tokens."""
import numpy as np
import pytest

from test_gpu_sample import _capped, _token, _uniform, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _narrow_rows(torch, vocabulary, spreads):
    """For each spread a row of zeros with a single value, one with as many as a sixth, and one of two values and a masked one.  Made on the host, which keeps
    subnormal numbers."""
    rng = np.random.default_rng(vocabulary)
    rows = np.zeros((len(spreads), 3, vocabulary), np.float32)
    for row, spread in zip(rows, np.array(spreads, np.float32)):
        row[0, vocabulary // 3] = spread
        row[1] = np.where(rng.random(vocabulary) < 1 / 6, spread, np.float32(0))
        row[2] = np.where(rng.random(vocabulary) < 0.5, -spread, np.float32(0))
        row[2, 1] = -np.inf
    assert (rows[:, 0].max(1) > 0).all()
    return torch.from_numpy(rows.reshape(-1, vocabulary))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocabulary", [3, 100, 8192, 9000, 32768, 40000])
@pytest.mark.parametrize("top_k", [2, 50, 256, 257])
def test_rows_of_tiny_spread(gpu, dtype, vocabulary, top_k):
    """From the smallest Float32 to spreads of which 1023 parts are ordinary numbers; the power of two at which bins of logits begin, from both sides.  Smaller
    temperatures tell the values apart: their quotients are exact enough in 64 bits that only a number within 2^-32 of a border could differ."""
    torch, binding = gpu
    spreads = [1e-45, 1e-40, 2.0 ** -126, 1e-38, 1e-37, 2e-36, 3e-36, 4e-36, 2.0 ** -110, 2.0 ** -109, 1e-30]
    logits = _narrow_rows(torch, vocabulary, spreads).to(getattr(torch, dtype)).cuda()
    rows = len(logits)
    z = logits.float().cpu().numpy()
    for i, settings in enumerate([dict(), dict(top_p=0.9), dict(min_p=0.3), dict(temperature=1e-37), dict(temperature=1e-36, top_p=0.7)]):
        u = _uniform(torch, rows, i)
        un = u.cpu().numpy()
        got = binding.ksample(logits, u, top_k=top_k, **settings).tolist()
        assert got == [_token(z[r], un[r], top_k=top_k, **settings) for r in range(rows)], settings


@pytest.mark.parametrize("vocabulary", [100, 9000, 32768])
def test_capped_rows_of_tiny_spread(gpu, oracle, vocabulary):
    torch, binding = gpu
    logits = _narrow_rows(torch, vocabulary, [1e-45, 1e-38, 1e-37, 3e-36, 1e-30]).cuda()
    z = _capped(oracle, logits.cpu().numpy(), 30.0, False)
    u = _uniform(torch, len(logits), 1)
    un = u.cpu().numpy()
    for top_k in (2, 50, 256):
        got = binding.ksample(logits, u, cap=30.0, top_k=top_k).tolist()
        assert got == [_token(z[r], un[r], top_k=top_k) for r in range(len(z))]


@pytest.mark.parametrize("vocabulary", [2, 300, 9000, 40000])
def test_temperatures_beyond_the_highest(gpu, vocabulary):
    """Rows' own temperatures above 3e38 are 3e38, at which logits of that size still differ: weights of 1 and e^-2."""
    torch, binding = gpu
    rng = np.random.default_rng(vocabulary)
    z = np.where(rng.random((6, vocabulary)) < 0.5, np.float32(3e38), np.float32(-3e38)).astype(np.float32)
    z[:, 0], z[:, -1] = 3e38, -3e38
    temperature = np.array([3e38, np.inf, 3.1e38, np.finfo(np.float32).max, np.inf, np.inf], np.float32)
    u = np.array([0.7, 0.7, 0.8, 0.9, 0.3, 0.95], np.float32)
    got = binding.ksample(torch.from_numpy(z).cuda(), torch.from_numpy(u).cuda(), temperature=torch.from_numpy(temperature).cuda()).tolist()
    assert got == [_token(z[r], u[r], temperature=3e38) for r in range(6)]
    assert vocabulary > 2 or got[:2] == [0, 0]
