"""sc_paged_reserve on the GPU against a program that keeps the pages in lists, one sequence and place after the other.  Everything is a whole number: equal."""
import pytest
import torch

from paper_2603_14303_amd import binding as sc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def needed(p, R, base, new, window, sinks):
    """By rows: place p holds a row that is not beyond the new ones, and that some token at `base` or behind it sees."""
    rows = range(p * R, min((p + 1) * R, base + new))
    return any(window == 0 or t < sinks or t >= base + 1 - window for t in rows)


def reserve(table, R, base, new, N, window, sinks, stack, pages):
    """Lists are changed in place -> lens, slots."""
    S, P = len(table), len(table[0])
    held = lambda x: 0 <= x < pages  # noqa: E731
    state = []
    for s in range(S):
        if base[s] < 0 or not 0 <= new[s] <= N or base[s] + new[s] > P * R:
            state.append(None)
            continue
        want = [needed(p, R, base[s], new[s], window, sinks) for p in range(P)]
        if any(want[p] and not held(table[s][p]) and p * R < base[s] for p in range(P)):
            state.append(None)
            continue
        state.append(want)
    back = [(s, p) for s in range(S) if state[s] for p in range(P) if held(table[s][p]) and not state[s][p]]
    given = [table[s][p] for s, p in back]
    available = len(stack) + len(given)
    lens, through, takes = [], 0, []
    for s in range(S):
        if state[s] is None:
            lens.append(-1)
            continue
        lack = [p for p in range(P) if state[s][p] and not held(table[s][p])]
        through += len(lack)
        ok = not lack or through <= available
        lens.append(base[s] + new[s] if ok else -1)
        takes += [(s, p) for p in lack] if ok else []
    for s, p in back:
        table[s][p] = -1
    source = given[: len(takes)]
    for _ in range(len(takes) - len(source)):
        source.append(stack.pop())
    stack.extend(reversed(given[len(takes) :]))
    for (s, p), page in zip(takes, source):
        table[s][p] = page
    slots = [[table[s][(base[s] + n) // R] * R + (base[s] + n) % R if lens[s] >= 0 and n < new[s] else -1 for n in range(N)] for s in range(S)]
    return lens, slots


class Both:
    def __init__(self, S, P, R, pages, seed=0, table_shape=None):
        gen = torch.Generator().manual_seed(seed)
        self.R, self.pages, self.shape = R, pages, table_shape or (S,)
        self.table = [[-1] * P for _ in range(S)]
        self.stack = torch.randperm(pages, generator=gen).tolist()
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        self.dtable = i32(self.table).reshape(*self.shape, P)
        self.dfree, self.dmany = i32(self.stack), i32([pages])
        self.ws = sc.paged_reserve_workspace(S, P, DEV)

    def step(self, base, new, N, window=0, sinks=0, slots=True):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV).reshape(self.shape)  # noqa: E731
        want_lens, want_slots = reserve(self.table, self.R, base, new, N, window, sinks, self.stack, self.pages)
        lens = torch.full(self.shape, -9, dtype=torch.int32, device=DEV)
        out = torch.full((*self.shape, N), -9, dtype=torch.int32, device=DEV) if slots else None
        sc.sc_paged_reserve(self.dtable, self.R, i32(base), lens, self.dfree, self.dmany, new_lens=i32(new), N=N, window=window, sinks=sinks, slots=out, workspace=self.ws)
        assert lens.flatten().tolist() == want_lens
        if slots:
            assert out.reshape(-1, N).tolist() == want_slots
        self.check()
        return want_lens

    def check(self):
        assert self.dtable.reshape(len(self.table), -1).tolist() == self.table
        assert int(self.dmany) == len(self.stack) and self.dfree.tolist()[: len(self.stack)] == self.stack


@pytest.mark.parametrize("S,P,R,window,sinks", [(1, 1, 16, 0, 0), (5, 40, 16, 0, 0), (7, 300, 16, 100, 20), (3, 600, 32, 64, 0), (300, 9, 64, 0, 0), (9, 20, 128, 200, 300), (4, 50, 16, 1, 1)])
def test_sequences_grow_step_by_step(S, P, R, window, sinks):
    gen = torch.Generator().manual_seed(S * P)
    both = Both(S, P, R, S * P, seed=1)
    base = [0] * S
    for step in range(12):
        most = max(1, P * R // 12)
        new = torch.randint(0, most + 1, (S,), generator=gen).tolist() if step % 3 == 0 else [1] * S
        new = [min(n, P * R - b) for n, b in zip(new, base)]
        lens = both.step(base, new, max(most, 1), window, sinks, slots=step % 2 == 0)
        assert lens == [b + n for b, n in zip(base, new)]
        base = lens
    both.step([0] * S, [0] * S, 1)
    assert len(both.stack) == S * P


def test_more_sequences_than_a_workgroup_adds_up():
    S = 2600
    gen = torch.Generator().manual_seed(8)
    both = Both(S, 3, 16, 3000, seed=8)
    base = [0] * S
    for step in range(4):      # growing, ending, some without room
        new = torch.randint(0, 17, (S,), generator=gen).tolist()
        gone = torch.rand(S, generator=gen) < 0.3
        base = [0 if g else b for b, g in zip(base, gone.tolist())]
        new = [min(n, 48 - b) for n, b in zip(new, base)]
        lens = both.step(base, new, 16, slots=step % 2 == 1)
        base = [b if n < 0 else n for b, n in zip(base, lens)]
        # (a sequence that was not served and has given back everything keeps its rows' pages: base says which)
    assert both.step([0] * S, [0] * S, 1) == [0] * S and len(both.stack) == 3000


def test_a_call_and_its_opposite_leave_the_stack_as_it_was():
    both = Both(6, 30, 16, 100, seed=2)
    base = [100, 0, 37, 64, 5, 63]
    both.step([0] * 6, base, 200)
    stack, table = list(both.stack), [list(x) for x in both.table]
    both.step(base, [60, 10, 0, 200, 1, 2], 200)
    both.step(base, [0] * 6, 200)
    assert both.stack == stack and both.table == table


def test_too_few_pages():
    both = Both(5, 20, 16, 30, seed=3)
    assert both.step([0] * 5, [160, 160, 176, 16, 160], 320) == [160, 160, -1, -1, -1]      # 10 + 10, then 11 do not fit, nor does anything behind
    assert both.step([160, 160, 0, 0, 0], [0, 0, 0, 16, 160], 320) == [160, 160, 0, 16, -1]
    # what one sequence gives back is there for the others in the same call
    assert both.step([0, 160, 0, 16, 0], [0, 0, 16, 0, 160], 320) == [0, 160, 16, 16, 160]


def test_lengths_that_are_not_possible_and_pages_that_are_missing():
    both = Both(6, 10, 16, 60, seed=4)
    both.step([0] * 6, [100, 100, 100, 100, 100, 100], 160)
    # negative, too many, more than asked for, beyond the table; the others go on
    assert both.step([-1, 100, 100, 100, 100, 100], [5, -2, 61, 40, 30, 0], 60) == [-1, -1, -1, 140, 130, 100]
    # behind a window the first pages go back, and a sequence that is cut back to where they were is refused
    assert both.step([100] * 6, [1] * 6, 1, window=20, sinks=4) == [101] * 6
    assert both.step([60, 101, 101, 79, 101, 100], [1] * 6, 1, window=20, sinks=4) == [-1, 102, 102, -1, 102, 101]
    big = 2**31 - 1
    assert both.step([big, 101, 101, 101, 101, 101], [big, 1, 1, 1, 1, 1], 1, window=big, sinks=big)[0] == -1


def test_a_table_of_pages_per_head_and_numbers_outside_the_pool():
    both = Both(6, 8, 32, 50, seed=5, table_shape=(2, 3))
    for row in both.table:
        row[5], row[6] = 50, -(2**31)
    both.dtable.copy_(torch.tensor(both.table, dtype=torch.int32).reshape(2, 3, 8))
    both.step([0] * 6, [1, 0, 33, 64, 200, 100], 200)
    both.step([1, 0, 33, 64, 200, 100], [0, 5, 0, 0, 0, 3], 5)


def test_counts_of_free_pages_that_are_not_possible():
    for many, want in ((-5, -1), (2**31 - 1, 16)):
        table = torch.full((1, 4), -1, dtype=torch.int32, device=DEV)
        lens, free, n = torch.zeros(1, dtype=torch.int32, device=DEV), torch.arange(6, dtype=torch.int32, device=DEV), torch.tensor([many], dtype=torch.int32, device=DEV)
        sc.sc_paged_reserve(table, 16, torch.zeros_like(lens), lens, free, n, N=16)
        assert lens.tolist() == [want] and int(n) == (0 if many < 0 else 5)


def test_a_page_that_is_named_twice_stays_inside_the_stack():
    table = torch.zeros((1, 8), dtype=torch.int32, device=DEV)
    fence = torch.full((12,), -7, dtype=torch.int32, device=DEV)
    free, lens, many = fence[:4], torch.zeros(1, dtype=torch.int32, device=DEV), torch.tensor([3], dtype=torch.int32, device=DEV)
    sc.sc_paged_reserve(table, 16, torch.zeros_like(lens), lens, free, many, N=0)
    assert int(many) == 4 and (fence[4:] == -7).all() and (table == -1).all()


def test_replayed_steps_and_two_graphs_with_one_workspace():
    """Tokens of a captured step take their pages from the stack as eager ones do."""
    S, P, R = 20, 12, 16
    both = Both(S, P, R, S * P, seed=6)
    base = torch.zeros(S, dtype=torch.int32, device=DEV)
    lens, slots = torch.zeros_like(base), torch.zeros((S, 3), dtype=torch.int32, device=DEV)
    new = torch.tensor([s % 4 for s in range(S)], dtype=torch.int32, device=DEV)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            sc.sc_paged_reserve(both.dtable, R, base, lens, both.dfree, both.dmany, new_lens=new, slots=slots, workspace=both.ws)
            base.copy_(lens)
    at = [0] * S
    for step in range(30):
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        at, want = reserve(both.table, R, at, [s % 4 for s in range(S)], 3, 0, 0, both.stack, both.pages)
        assert slots.tolist() == want and base.tolist() == at
        both.check()
        float(torch.rand(1000, device=DEV).sum())
