"""sc_paged_reserve for sequences that receive nothing, or little, at a window's edge inside a page that is not full: the page stays, and the next token goes there.

Here a place is needed as the header says: p R < base + new, and with a window p R < sinks or (p + 1) R > base + 1 - window, whether or not the rows at the page's end are there yet."""
import pytest
import torch

import test_gpu_reserve
from test_gpu_reserve import Both

pytestmark = pytest.mark.gpu


def needed(p, R, base, new, window, sinks):
    return p * R < base + new and (window == 0 or p * R < sinks or (p + 1) * R > base + 1 - window)


@pytest.fixture(autouse=True)
def by_the_header(monkeypatch):
    monkeypatch.setattr(test_gpu_reserve, "needed", needed)


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (1, 5), (20, 0)])
def test_a_page_that_is_not_full_stays_for_the_next_token(window, sinks):
    """Lengths on all sides of a page's end: filed, left alone for a step, then a token each, from the same page where it has room."""
    R = 16
    base = [10, 15, 16, 17, 20, 31, 32, 33, 1, 0]
    S = len(base)
    both = Both(S, 5, R, 5 * S, seed=window)
    assert both.step([0] * S, base, 40, window, sinks) == base
    assert both.step(base, [0] * S, 1, window, sinks) == base
    last = [both.table[s][base[s] // R] for s in range(S)]
    for s, n in enumerate(base):
        assert (last[s] >= 0) == (n % R > 0), n
    after = both.step(base, [1] * S, 1, window, sinks)
    assert after == [n + 1 for n in base]
    for s, n in enumerate(base):
        assert both.table[s][n // R] >= 0 and (n % R == 0 or both.table[s][n // R] == last[s])


@pytest.mark.parametrize("R,window,sinks", [(16, 1, 0), (16, 3, 20), (32, 20, 0), (16, 33, 1)])
def test_sequences_that_pause_now_and_then(R, window, sinks):
    gen = torch.Generator().manual_seed(R + window)
    S, P = 40, 12
    both = Both(S, P, R, S * P, seed=3)
    base = [0] * S
    for step in range(20):
        new = (torch.randint(0, 6, (S,), generator=gen) * (torch.rand(S, generator=gen) < 0.5)).tolist()
        assert both.step(base, new, 5, window, sinks, slots=step % 2 == 0) == [b + n for b, n in zip(base, new)]
        base = [b + n for b, n in zip(base, new)]
