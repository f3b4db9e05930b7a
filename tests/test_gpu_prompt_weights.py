"""The weights of sc_prompt_attn in bf16 calls keep 16 bits, and nothing of them depends on what lies behind the last query.

Tolerances are those of test_gpu_prompt.py, with other numbers for a weight: it enters the second product as two bf16 numbers.  Of a weight of [1, 2) the first is off by 2^-8 at most (half
of bf16's 2^-7 there); what is left, below 2^-8, by half of that range's 2^-16: r = 2^-17.  Two products a key are n more roundings of a sum: u each.
"""
import math

import pytest
import torch

from paper_2603_14303_amd import binding as sc
from test_gpu_paged import BF, DEV, U, close, half_step
from test_gpu_prompt import reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,M,G,d,window,sinks", [
    (200, 200, 4, 128, 0, 0), (33, 700, 3, 64, 0, 0), (16, 4100, 4, 128, 0, 0), (150, 150, 1, 64, 40, 3), (300, 1100, 4, 128, 64, 16), (1030, 1030, 1, 64, 0, 0)])
def test_outputs_are_as_exact_as_their_type(N, M, G, d, window, sinks):
    """(Workgroups of 128 rows, with their keys in one piece and in splits, and of 256.)"""
    gen = torch.Generator().manual_seed(N + M)
    Q, K, V = (torch.randn((1, h, n, d), generator=gen).to(BF) for h, n in ((2 * G, N), (2, M), (2, M)))
    O, _ = sc.sc_prompt_attn(Q.to(DEV), K.to(DEV), V.to(DEV), window=window, sinks=sinks)
    for h in range(2 * G):
        wo, _, to, _ = reference(Q[0, h].double(), K[0, h // G].double(), V[0, h // G].double(), window, sinks, 1 / math.sqrt(d), 2.0**-17 + M * U)
        close(O[0, h], wo, to + half_step(BF) * wo.abs() * (1 + 2.0**-6) + 1e-30)


@pytest.mark.parametrize("N,d", [(300, 128), (1100, 64)])
def test_equal_weights_that_are_no_power_of_two(N, d):
    """All values of a head's elements are one number, and all keys but those of a first stretch have one logit: every weight is rounded alike, so nothing averages out, however many keys there are.

    The output before its rounding is off by less than 2^-17 + (2 n + 256) u < 2^-12 of the number.  Half a step of bf16 below 2 is 2^-8, more than 2^-9 of the numbers here: they are what comes out."""
    H = 32
    K = torch.zeros((1, H, N, d))
    for h in range(H):
        if h < 16:      # one first key that all others fall behind
            K[0, h, 0, 0] = 0.04 * (h + 1)
        else:           # a first tile that all others exceed, by less than the running maximum follows
            K[0, h, 64:, 0] = 0.3 * (h - 15)
    Q = torch.zeros((1, H, N, d))
    Q[..., 0] = 1
    numbers = torch.tensor([1.9921875, -1.75, 1.5078125, 1.2578125])
    V = numbers.repeat(d // 4).expand(1, H, N, d)
    O, _ = sc.sc_prompt_attn(*(x.to(BF).to(DEV) for x in (Q, K, V)), scale=1.0)
    assert (O.cpu().float() == V).all()


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("N,M,G", [(40, 600, 1), (330, 1200, 4)])
def test_rows_behind_the_last_query_change_nothing(dtype, N, M, G):
    """A wavefront has queries on both sides of the length: the same bits for those before it, whatever lies behind."""
    gen = torch.Generator().manual_seed(N)
    Q, K, V = (torch.randn((2, h, n, 128), generator=gen).to(dtype).to(DEV) for h, n in ((G, N), (1, M), (1, M)))
    junk = torch.randn(Q.shape, generator=gen).to(dtype).to(DEV)
    lens = (N - 20, N // 2 + 1)
    q_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    results = []
    for factor in (0.0, 1.0, 50.0, math.inf, math.nan):
        for b, n in enumerate(lens):
            Q[b, :, n:] = junk[b, :, n:] * factor
        O, L = sc.sc_prompt_attn(Q, K, V, q_lens=q_lens, O=torch.zeros_like(Q), lse=torch.zeros(Q.shape[:3], device=DEV))
        results.append((O, L))
    for O, L in results[1:]:
        assert (O == results[0][0]).all() and (L == results[0][1]).all()
