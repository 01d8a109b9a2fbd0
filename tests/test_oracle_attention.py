"""CPU tests of the references of heads, attention and pages: gradients against
differences, known cases, and the pages' rule against what it has to keep."""

import numpy as np
import pytest

from oracle import attention as ref


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("batch", [None, 2])
def test_rotation_gradients_against_differences(interleaved, batch):
    rng = np.random.default_rng(1)
    lead = (5,) if batch is None else (batch, 5)
    x, dy = rng.standard_normal((2, *lead, 3, 12))
    w = rng.standard_normal((12,) if batch is None else (batch, 12))
    positions, freqs = rng.integers(-50, 50, lead[-1]), rng.standard_normal(4)
    f = lambda x, w: (ref.rotate_heads(x, w, positions, freqs, 1e-3, interleaved)[0] * dy).sum()  # noqa: E731
    dx, dw, _, _ = ref.rotate_heads_grads(dy, x, w, positions, freqs, 1e-3, interleaved)
    h = 1e-6
    for a, g, at in ((x, dx, 0), (w, dw, 1)):
        for _ in range(30):
            i = tuple(rng.integers(0, n) for n in a.shape)
            up, down = a.copy(), a.copy()
            up[i] += h
            down[i] -= h
            d = (f(up, w) - f(down, w) if at == 0 else f(x, up) - f(x, down)) / (2 * h)
            assert abs(d - g[i]) < 1e-7 * max(1, abs(d))  # h^2 of the third derivative, 1e-16 / h of rounding


def test_rotation_keeps_lengths_and_differences_of_positions():
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((2, 1, 1, 8))
    freqs = np.array([1.0, 0.1, 0.01, 0.0])
    at = lambda v, p: ref.turn(v, [p], freqs, False)  # noqa: E731
    assert np.allclose((at(x, 7) ** 2).sum(), (x ** 2).sum(), rtol=1e-14)
    assert np.allclose((at(x, 1007) * at(y, 1003)).sum(), (at(x, 4) * at(y, 0)).sum(), rtol=1e-12)


def test_attention_known_cases():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 2, 32)), rng.standard_normal((5, 1, 32)), rng.standard_normal((5, 1, 32))
    out, bound = ref.attend(q, k, v, 0.3, window=1)
    assert np.allclose(out, v[[2, 3, 4]]) and (bound < 1e-2).all()
    assert (ref.attend(q, k[:1], v[:1], 1.0)[0][:2] == 0).all()  # two queries before the first key
    assert np.allclose(ref.attend(0 * q, k, v, 1.0)[0][2], v.mean(0))


@pytest.mark.parametrize("seed", range(20))
def test_pages_rule(seed):
    rng = np.random.default_rng(seed)
    B, W, page, N = 7, 6, int(rng.choice([1, 3, 16])), 30
    tables, lengths, free = [[-1] * W for _ in range(B)], [0] * B, list(rng.permutation(N))
    for _ in range(30):
        counts = [int(c) for c in rng.integers(-1, 2 * page + 2, B)]
        before = (tables, lengths, free)
        tables, lengths, free, starts, positions, slots = ref.extend_pages(*before[:2], counts, free, page, 40)
        held = [p for t in tables for p in t if p >= 0]
        assert sorted(held + free) == list(range(N))  # no page is lost or given twice
        for b in range(B):
            got = starts[b + 1] - starts[b]
            assert got in (0, max(counts[b], 0)) and lengths[b] == before[1][b] + got
            assert sum(p >= 0 for p in tables[b]) == -(-lengths[b] // page)
        real = slots[:starts[-1]]
        assert len(set(real)) == len(real) and min(real, default=0) >= 0
        back = ref.truncate_pages(tables, lengths, before[1], free, page)
        assert back == before
        keep = [int(k) for k in rng.integers(-1, W * page, B)]
        tables, lengths, free = ref.truncate_pages(tables, lengths, keep, free, page)
