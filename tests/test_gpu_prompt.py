"""sc_prompt_attn on the GPU against a plain implementation in fp64.

Tolerances (u = 2^-24; r = 2^-8, the rounding of a probability to bf16, or 0 in fp32 calls):
  * a logit is a sum of d products in fp32, scaled: off by delta = (d + 16) u (sum_e |q_e k_e| |scale| + |logit|), so a weight by a factor exp(2 delta);
  * a weight enters the second product off by r of itself (bf16 has 7 bits behind the point: numbers of [1, 2) are 2^-7 apart,
    so a rounding is off by up to 2^-8 of 1, torch.finfo(bfloat16).eps / 2), while the denominator does not; sums over n keys: (n + 256) u.
    All that over sum_j w_j |v_j|, then the rounding of O;
  * lse: delta, the sum's own error, and a few roundings.
"""
import math

import pytest
import torch

from paper_2603_14303_amd import binding as sc
from test_gpu_paged import BF, DEV, F32, U, close, half_step

pytestmark = pytest.mark.gpu


def visible(n_q, n_k, window, sinks):
    pos = n_k - n_q + torch.arange(n_q)[:, None]
    j = torch.arange(n_k)[None]
    seen = j <= pos
    if window:
        seen &= (j > pos - window) | (j < sinks)
    return seen


def reference(q, k, v, window, sinks, scale, r):
    """One head in fp64 -> O, lse and how far they may be off (without O's own rounding)."""
    seen = visible(q.shape[0], k.shape[0], window, sinks)
    if q.shape[0] == 0 or k.shape[0] == 0:
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64), torch.zeros_like(q), torch.zeros(q.shape[0], dtype=torch.float64)
    z = (q @ k.T * scale).masked_fill(~seen, -math.inf)
    some = seen.any(1)
    size = (q.abs() @ k.abs().T * abs(scale)).masked_fill(~seen, 0).amax(1) + z.masked_fill(~seen, 0).abs().amax(1)
    delta = (q.shape[1] + 16) * U * size
    w = torch.softmax(z, 1).masked_fill(~seen, 0)
    lse = torch.logsumexp(z, 1)
    sums = (k.shape[0] + 256) * U
    o, tol = w @ v, (2 * delta + sums + r)[:, None] * (w @ v.abs())
    return torch.where(some[:, None], o, 0), lse, torch.where(some[:, None], tol, 0), delta + sums + 4 * U * lse.abs().nan_to_num(0, 0, 0)


def check(B, Hkv, G, N, M, d, dtype, q_lens=None, kv_lens=None, window=0, sinks=0, scale=0.0, fused=True, lse=True, seed=0, workspace=None, tweak=None):
    """Rows behind the lengths hold NaN and infinities on the way in, a mark on the way out."""
    gen = torch.Generator().manual_seed(seed)
    ql, kl = q_lens or [N] * B, kv_lens or [M] * B
    Q, K, V = (torch.randn((B, h, n, d), generator=gen).to(dtype) for h, n in ((Hkv * G, N), (Hkv, M), (Hkv, M)))
    if tweak:
        tweak(Q, K, V)
    for b in range(B):
        Q[b, :, ql[b]:], K[b, :, kl[b]:], V[b, :, kl[b]:] = math.nan, math.nan, math.inf
    dev = lambda x: (x.permute(0, 2, 1, 3).contiguous().to(DEV).permute(0, 2, 1, 3) if fused else x.to(DEV))  # noqa: E731
    O = torch.full((B, N, Hkv * G, d), 77.0, dtype=dtype, device=DEV).permute(0, 2, 1, 3) if fused else torch.full((B, Hkv * G, N, d), 77.0, dtype=dtype, device=DEV)
    L = torch.full((B, Hkv * G, N), 77.0, device=DEV) if lse else None
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    sc.sc_prompt_attn(dev(Q), dev(K), dev(V), q_lens=i32(q_lens), kv_lens=i32(kv_lens), window=window, sinks=sinks, scale=scale, O=O, lse=L, workspace=workspace)
    torch.cuda.synchronize()
    Oc, Lc = O.cpu(), None if L is None else L.cpu()
    for b in range(B):
        assert (Oc[b, :, ql[b]:] == 77).all() and (Lc is None or (Lc[b, :, ql[b]:] == 77).all())
        for h in range(Hkv * G):
            q, k, v = Q[b, h, : ql[b]].double(), K[b, h // G, : kl[b]].double(), V[b, h // G, : kl[b]].double()
            wo, wl, to, tl = reference(q, k, v, window, sinks, scale or 1 / math.sqrt(d), half_step(BF) if dtype == BF else 0.0)
            close(Oc[b, h, : ql[b]], wo, to + half_step(dtype) * wo.abs() * (1 + 2.0**-6) + 1e-30)
            if Lc is not None:
                close(Lc[b, h, : ql[b]], wl, tl)
    return Q, K, V, Oc, Lc


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 1), (128, 7), (64, 3), (128, 1), (64, 16)])
@pytest.mark.parametrize("N", [1, 2, 31, 33, 64, 65, 200])
def test_lengths_and_groups(dtype, d, G, N):
    check(2, 2, G, N, N, d, dtype, lse=N % 2 == 1, seed=N)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (32, 32), (64, 0), (64, 64), (63, 65), (100, 130), (1000, 4), (2**31 - 1, 2**31 - 1), (5, 2**31 - 1)])
def test_windows(dtype, window, sinks):
    check(1, 2, 2, 300, 300, 64, dtype, window=window, sinks=sinks, seed=window % 101)
    check(1, 1, 3, 70, 500, 128, dtype, window=window, sinks=sinks, seed=sinks % 101)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_ragged_batches(dtype):
    check(5, 2, 3, 150, 420, 128, dtype, q_lens=[0, 1, 150, 100, 37], kv_lens=[50, 1, 420, 100, 300])
    check(4, 1, 2, 90, 200, 64, dtype, q_lens=[90, 60, 10, 5], kv_lens=[30, 0, 9, 200], window=20, sinks=5)      # more queries than keys: the first ones see none
    check(3, 1, 5, 100, 260, 128, dtype, kv_lens=[260, 100, 130], window=70, sinks=65, fused=False)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_lengths_beyond_the_arrays_count_as_theirs(dtype):
    gen = torch.Generator().manual_seed(3)
    Q, K = torch.randn((2, 2, 40, 64), generator=gen).to(dtype).to(DEV), torch.randn((2, 1, 60, 64), generator=gen).to(dtype).to(DEV)
    lens = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    O, _ = sc.sc_prompt_attn(Q, K, K, q_lens=lens(41, -3), kv_lens=lens(2**31 - 1, 60), O=torch.zeros_like(Q))
    want, _ = sc.sc_prompt_attn(Q, K, K, O=torch.zeros_like(Q))
    assert (O[0] == want[0]).all() and (O[1] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,M", [(1, 5000), (16, 4100), (3, 700), (130, 3000)])
def test_few_queries_behind_a_long_context(dtype, N, M):
    """Keys in splits, whose partial results are joined; the same workspace for calls of other sizes."""
    ws = sc.prompt_attn_workspace(2, 8, 2, 130, 5000, 128, DEV)
    check(2, 2, 4, N, M, 128, dtype, kv_lens=[M, M // 3], workspace=ws)
    check(1, 2, 4, N, M, 128, dtype, window=900, sinks=10, workspace=ws, seed=1)


def test_many_tiles_of_rows():
    check(1, 4, 2, 4200, 4200, 128, BF, window=300, sinks=20)
    check(2, 4, 4, 2100, 2300, 64, BF, q_lens=[2100, 1999], kv_lens=[2300, 2000])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,M,G,window,sinks", [(257, 1025, 4, 0, 0), (300, 1100, 5, 64, 64), (1030, 1030, 1, 100, 130), (1024, 1089, 1, 1, 1), (130, 2500, 8, 700, 33), (600, 1026, 3, 0, 0)])
def test_256_rows_a_workgroup(d, N, M, G, window, sinks):
    """bf16 calls of at least 1024 rows a KV head over more than 1024 keys."""
    check(1, 2, G, N, M, d, BF, window=window, sinks=sinks, seed=M)
    check(3, 1, G, N, M, d, BF, q_lens=[N, 1, N - 100], kv_lens=[M, M - 70, N // 2], window=window, sinks=sinks, fused=False, seed=N)


@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 0), (90, 70)])
@pytest.mark.parametrize("N,M,G", [(600, 1090, 2), (150, 300, 2)])
def test_numbers_that_are_not_finite_in_workgroups_of_either_size(N, M, G, window, sinks):
    """Rows that do not see the number, and what is beside it in rows that see it in the values, are those of the formula, within the tolerance of any other call."""
    d, gen = 64, torch.Generator().manual_seed(M)
    Q, K, V = (torch.randn((1, h, n, d), generator=gen).to(BF) for h, n in ((G, N), (1, M), (1, M)))
    want = [reference(Q[0, h].double(), K[0, 0].double(), V[0, 0].double(), window, sinks, 1 / math.sqrt(d), half_step(BF)) for h in range(G)]
    seen = visible(N, M, window, sinks)
    others = torch.arange(d) != 5
    for which, value in (("V", math.nan), ("V", -math.inf), ("K", math.nan)):
        for j in (0, 63, 64, M - N, M - N + 1, M - N + 128, M - 65, M - 1):
            x = {"K": K.clone(), "V": V.clone()}
            x[which][0, 0, j, 5] = value
            O, _ = sc.sc_prompt_attn(Q.to(DEV), x["K"].to(DEV), x["V"].to(DEV), window=window, sinks=sinks)
            hit = seen[:, j]
            for h in range(G):
                o, (wo, _, to, _) = O[0, h].cpu(), want[h]
                tol = to + half_step(BF) * wo.abs() * (1 + 2.0**-6) + 1e-30
                close(o[~hit], wo[~hit], tol[~hit])
                if which == "V":
                    assert not o[hit][:, 5].isfinite().any()
                    close(o[hit][:, others], wo[hit][:, others], tol[hit][:, others])
                else:
                    assert o[hit].isnan().all()


@pytest.mark.parametrize("scale", [0.7, -0.3, 1e-3])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_scales(dtype, scale):
    check(1, 2, 2, 150, 150, 128, dtype, scale=scale)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logits_that_grow_along_the_keys(dtype):
    """The running maximum has to follow over and over; and keys that fall behind it by more than fp32 holds."""
    def rising(Q, K, V):
        Q.fill_(1.0)
        K.copy_((torch.arange(K.shape[2])[:, None] * 0.02).expand_as(K))
    check(1, 1, 2, 500, 500, 64, dtype, tweak=rising, scale=0.5)

    def falling(Q, K, V):
        Q.fill_(1.0)
        K.copy_((-torch.arange(K.shape[2])[:, None] * 0.05).expand_as(K))
    check(1, 1, 2, 500, 500, 64, dtype, tweak=falling, scale=1.0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 0), (40, 70)])
def test_numbers_that_are_not_finite_show_where_they_are_seen_and_nowhere_else(dtype, window, sinks):
    N, d, G = 260, 64, 2
    gen = torch.Generator().manual_seed(5)
    Q, K, V = (torch.randn((1, h, N, d), generator=gen).to(dtype) for h in (G, 1, 1))
    clean, _ = sc.sc_prompt_attn(Q.to(DEV), K.to(DEV), V.to(DEV), window=window, sinks=sinks)
    seen = visible(N, N, window, sinks)
    for which, value in (("V", math.nan), ("V", math.inf), ("V", -math.inf), ("K", math.nan), ("K", math.inf), ("Q", math.nan)):
        for j in (0, 63, 64, 100, 255):
            x = {"Q": Q.clone(), "K": K.clone(), "V": V.clone()}
            x[which][0, 0, j, 5] = value
            O, _ = sc.sc_prompt_attn(*(t.to(DEV) for t in x.values()), window=window, sinks=sinks)
            O = O.cpu()
            if which == "Q":
                assert O[0, 0, j].isnan().all()
                rest = torch.ones((G, N), dtype=torch.bool)
                rest[0, j] = False
                assert (O[0][rest] == clean.cpu()[0][rest]).all()
                continue
            hit = seen[:, j]
            assert O[0, :, ~hit].isfinite().all() and torch.allclose(O[0, :, ~hit].float(), clean.cpu()[0, :, ~hit].float(), rtol=2 * half_step(dtype) if dtype == BF else 1e-5, atol=1e-2 if dtype == BF else 1e-5)
            if which == "V":
                assert not O[0, :, hit, 5].isfinite().any()
                others = torch.arange(d) != 5
                assert O[0][:, hit][..., others].isfinite().all()
            elif math.isnan(value):
                assert O[0, :, hit].isnan().all()


def test_shared_rows_and_strides_of_zero():
    """Keys that all sequences share are one array, read through a stride of zero."""
    gen = torch.Generator().manual_seed(9)
    Q, K, V = torch.randn((3, 4, 50, 128), generator=gen).to(BF).to(DEV), torch.randn((1, 1, 50, 128), generator=gen).to(BF).to(DEV), torch.randn((1, 1, 50, 128), generator=gen).to(BF).to(DEV)
    got, _ = sc.sc_prompt_attn(Q, K.expand(3, 2, -1, -1), V.expand(3, 2, -1, -1))
    want, _ = sc.sc_prompt_attn(Q, K.expand(3, 2, -1, -1).contiguous(), V.expand(3, 2, -1, -1).contiguous())
    assert (got == want).all()


def test_replays_on_another_stream():
    gen = torch.Generator().manual_seed(11)
    Q, K, V = (torch.randn((1, h, 100, 128), generator=gen).to(BF).to(DEV) for h in (8, 2, 2))
    kv = torch.tensor([100], dtype=torch.int32, device=DEV)
    ws = sc.prompt_attn_workspace(1, 8, 2, 100, 100, 128, DEV)
    O = torch.zeros_like(Q)
    want, _ = sc.sc_prompt_attn(Q, K, V, kv_lens=kv)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sc.sc_prompt_attn(Q, K, V, kv_lens=kv, O=O, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert (O == want).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sc.sc_prompt_attn(Q, K, V, kv_lens=kv, O=O, workspace=ws)
    for _ in range(3):
        O.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert (O == want).all()
        Q.mul_(0.5)
        want, _ = sc.sc_prompt_attn(Q, K, V, kv_lens=kv)
