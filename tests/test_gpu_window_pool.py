"""examples/window_serving.py where pages run out: a sequence that a step has no page for waits, and goes on once a request has ended."""
import os
import sys

import pytest
import torch

from test_gpu_reserve import reserve
from test_gpu_window_example import LENS

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
SMALL = dict(layers=2, width=128, Hkv=2, G=2)


@pytest.mark.parametrize("window,tokens", [(0, 70), (4096, 70), (100, 40)])
def test_the_pool_holds_all_that_the_sequences_need(window, tokens):
    import window_serving as ex
    seen = []
    pages, _, x = ex.serve(lens=LENS, tokens=tokens, window=window, sinks=4, watch=lambda pages, s: seen.append(pages.lens.tolist()), **SMALL)
    assert seen == [[n + s for n in LENS] for s in range(tokens + 1)] and torch.isfinite(x.float()).all()


@pytest.mark.parametrize("graph", [False, True])
def test_a_sequence_without_a_page_waits_and_goes_on(graph, monkeypatch):
    """The pool is what the prompts fill: the longest sequence and one behind it lack a page; the former ends, the latter goes on with its pages."""
    import window_serving as ex
    tokens, end = 40, 25
    pool = sum(-(-n // ex.R) for n in LENS)
    P = -(-(max(LENS) + tokens) // ex.R)
    # the pages in lists, sequence after sequence: which step serves whom
    table, stack, lens, want = [[-1] * P for _ in LENS], list(range(pool)), list(LENS), []
    reserve(table, ex.R, [0] * 4, lens, max(LENS), 0, 0, stack, pool)
    for s in range(tokens):
        new = [1] * 4
        if s >= end:
            new[1] = 0
        if s == end:
            lens[1] = 0
        after, _ = reserve(table, ex.R, lens, new, 1, 0, 0, stack, pool)
        lens = [b if n < 0 else n for b, n in zip(lens, after)]
        want.append((list(lens), [n < 0 for n in after]))
    assert [any(w[b] for _, w in want) for b in range(4)] == [False, True, True, False] and not any(want[-1][1]) and want[-1][0][2] > 64

    states = []
    attend = ex.sc.sc_paged8_decode_attn

    def attended(cache, Q, lens, **kw):
        O, lse = attend(cache, Q, lens, **kw)
        if not graph:
            states.append((lens.tolist(), O.clone()))
        return O, lse

    monkeypatch.setattr(ex.sc, "sc_paged8_decode_attn", attended)
    rows = []

    def watch(pages, s):
        rows.append((pages.lens.tolist(), pages.table.tolist(), pages.free[: int(pages.many)].tolist()))

    pages, model, x = ex.serve(lens=LENS, tokens=tokens, window=0, sinks=0, ends={end: 1}, graph=graph, watch=watch, pool=pool, **SMALL)
    assert [r[0] for r in rows[1:]] == [w[0] for w in want]
    assert rows[-1][1] == table and rows[-1][2] == stack
    assert torch.isfinite(x.float()).all()
    if not graph:      # a waiting sequence attends to nothing, the others to all their rows
        for s, (lens, waiting) in enumerate(want):
            for got, O in states[2 * s : 2 * s + 2]:
                assert got == [0 if w else n for n, w in zip(lens, waiting)]
                for b, n in enumerate(got):
                    assert torch.isfinite(O[b].float()).all() and bool((O[b] != 0).any()) == (n > 0)


def test_a_waiting_sequence_keeps_its_state():
    """The hidden state of a sequence that waits from some step on is that of the program stopped before it."""
    import window_serving as ex
    lens = (64, 40)      # full pages, and one with room for 24 rows
    kw = dict(lens=lens, window=0, sinks=0, pool=5, **SMALL)
    # the first sequence takes the fifth page with its first token and is full after 32, the second with its 25th lacks one
    (_, _, a), (pages, _, b) = (ex.serve(tokens=n, **kw) for n in (24, 30))
    assert pages.lens.tolist() == [94, 64]
    assert (a[1] == b[1]).all() and not (a[0] == b[0]).all()


def test_a_pool_without_room_for_the_prompts_is_refused():
    import window_serving as ex
    with pytest.raises(ValueError, match="pages"):
        ex.serve(lens=LENS, tokens=1, window=0, pool=sum(-(-n // ex.R) for n in LENS) - 1, **SMALL)
