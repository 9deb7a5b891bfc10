"""The 64-bit reference of capped attention held against itself: gradients against differences, K against its lines, joined pieces."""
import numpy as np
import pytest

from oracle import kcap_oracle


@pytest.mark.parametrize("mask", [dict(causal=True), dict(causal=False), dict(causal=True, window=2)])
def test_gradients_are_the_derivative_where_tanh_is(mask):
    """With TanH in K-TanH's place the formula is the derivative: central differences of step 1e-5 are off by 1e-10 and 1e-11 / 1e-5."""
    rng = np.random.default_rng(0)
    q, k, v, do = (rng.standard_normal(s) for s in ((5, 8), (7, 8), (7, 8), (5, 8)))
    options = dict(cap=2.0, scale=0.7, tanh=True, **mask)

    def loss(q, k, v):
        return (kcap_oracle.head(q, k, v, **options)["o"] * do).sum()
    grads = kcap_oracle.head(q, k, v, do=do, **options)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        differences = np.zeros_like(x)
        for at in np.ndindex(x.shape):
            held = x[at]
            x[at] = held + 1e-5
            up = loss(q, k, v)
            x[at] = held - 1e-5
            differences[at] = (up - loss(q, k, v)) / 2e-5
            x[at] = held
        assert np.abs(differences - grads[name]).max() < 1e-8, name


@pytest.mark.parametrize("intervals", [32, 64])
def test_k_is_a_line_on_each_interval(oracle, intervals):
    """K(x) = A x + B with A = 2^(E - E_i - r), B = 2^(E - 127) (1 - 2^-r + b/128), but for the bits that the shift drops."""
    rows = (oracle.table1() if intervals == 32 else oracle.fit_lut64()).as_tuples()
    each = intervals // 4
    for t, (E, r, b) in enumerate(rows):
        e_in = 125 + ((t // each - 125) & 3)
        first = 2.0 ** (e_in - 127) * (1 + (t % each) / each)
        x = (first + 2.0 ** (e_in - 127) / each * np.arange(64) / 64.3).astype(np.float32).astype(np.float64)
        line = 2.0 ** (E - e_in - r) * x + 2.0 ** (E - 127) * (1 - 2.0 ** -r + b / 128)
        k = kcap_oracle.k_of(x, intervals)
        assert (k <= line).all() and (line - k < 2.0 ** (E - 127 - 23)).all(), t


def test_masks():
    ok = kcap_oracle.seen(3, 5, True, 2)
    assert ok.astype(int).tolist() == [[0, 1, 1, 0, 0], [0, 0, 1, 1, 0], [0, 0, 0, 1, 1]]
    assert not kcap_oracle.seen(4, 2, True, 0)[:2].any()
    assert kcap_oracle.seen(2, 3, False, 0).all()


def test_a_nan_value_reaches_the_rows_that_see_it():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((4, 8)) for _ in range(3))
    v[2, 3] = np.nan
    v[1, 0] = np.inf
    o = kcap_oracle.head(q, k, v, cap=2.0, scale=1.0, tanh=True)["o"]
    assert np.isnan(o).sum() == 2 and np.isnan(o[2:, 3]).all()
    assert np.isinf(o).sum() == 3 and np.isinf(o[1:, 0]).all()
