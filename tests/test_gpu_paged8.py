"""A cache held in pages of 8-bit codes, and windows over caches in pages, on the GPU: sc_paged8_append, sc_paged8_decode_attn and sc_paged_window_attn
against plain implementations.

Tolerances (u = 2^-24, a rounding of fp32):
  * codes and scales: equal to those of the formula's steps in fp32 (products, sums and reciprocals rounded one by one), which torch takes on the CPU;
    from the numbers themselves they are off by half a step: |x| 2^-4, at least scale 2^-10 (e4m3), scale / 2 (int8), and where a block has grown, by
    less than one final step more (the scales are powers of two: the errors of the steps before add up to half of it at most, twice);
  * attention: as for a cache that keeps its numbers, since codes are exact in bf16 and a scale is one factor of a logit, or of a weight, more: (d + 18) u.
"""
import math

import pytest
import torch

from paper_2603_14303_amd import binding as sc
from test_gpu_paged import BF, DEV, F32, U, Paged, attend, close, half_step

pytestmark = pytest.mark.gpu
E4, I8 = torch.float8_e4m3fn, torch.int8
LARGEST = {E4: 448.0, I8: 127.0}


# ------------------------------------------------------------------------------------------------ codes
def encode(code, x):
    """fp32 -> codes as their bytes."""
    if code == I8:
        return x.round().clamp(-127, 127).nan_to_num(0).to(I8).view(torch.uint8)
    return x.to(E4).view(torch.uint8)


def decode(code, b):
    return b.view(code).float()


def smallest_scale(code, largest):
    """From the numbers: 2^e with largest <= Q 2^e, e as small as possible but at least -126."""
    if not math.isfinite(largest):
        return math.nan
    e = -126
    while largest > LARGEST[code] * 2.0**e:
        e += 1
    return 2.0**e


class Paged8(Paged):
    """Pools of codes of any byte (no numbers among them) and scales that are no numbers, but for rows that the cache holds."""

    def __init__(self, B, Hkv, P, R, d, code, block, per_head_table=False, layout="phrd", counts=False, seed=0):
        super().__init__(B, Hkv, P, R, d, BF, per_head_table=per_head_table, counts=counts, seed=seed, junk=False)
        self.code, self.block = code, block
        shape = {"phrd": (self.n, self.heads, R, d), "prhd": (self.n, R, self.heads, d), "pkv": (self.n, 2, self.heads, R, d)}[layout]
        pools = [torch.randint(0, 256, shape, generator=self.gen, dtype=torch.uint8).to(DEV) for _ in range(1 if layout == "pkv" else 2)]
        pools = [pools[0][:, 0], pools[0][:, 1]] if layout == "pkv" else pools
        self.K, self.V = (x.permute(0, 2, 1, 3) if layout == "prhd" else x for x in pools)
        self.ks, self.vs = (torch.full((self.n, self.heads, R // block), math.nan, device=DEV) for _ in range(2))

    def cache(self, table=None):
        return sc.PagedCache8(self.K.view(self.code), self.V.view(self.code), self.ks, self.vs, (self.table if table is None else table).to(DEV), counts=self.counts)

    def fill(self, lens, seen=None):
        """Rows of (b, h) below lens[b][h] (those of seen(n) only) get codes and scales; returns their numbers in fp64."""
        out = {}
        K, V, ks, vs = (x.cpu() for x in (self.K, self.V, self.ks, self.vs))
        counts = None if self.counts is None else self.counts.cpu()
        for b in range(self.B):
            for h in range(self.H):
                t = torch.arange(int(lens[b][h]))
                t = t if seen is None else t[seen(len(t))]
                page, head, row = self.place(b, h, t)
                numbers = []
                for pool, scales in ((K, ks), (V, vs)):
                    codes = encode(self.code, torch.randn((len(t), self.d), generator=self.gen) * LARGEST[self.code] / 4.5)
                    codes = torch.where(decode(self.code, codes).isnan(), torch.zeros_like(codes), codes)
                    # of a block: a power of two, or any number that the caller has put there
                    unit = torch.exp2(torch.randint(-9, -5, scales.shape, generator=self.gen).float()) * (1 + 0.3 * torch.rand(scales.shape, generator=self.gen))
                    scales[page, head, row // self.block] = unit[page, head, row // self.block]
                    pool[page, head, row] = codes
                    numbers.append(decode(self.code, codes).double() * scales[page, head, row // self.block].double()[:, None])
                out[b, h] = (*numbers, None if counts is None else counts[page, head, row].double())
        for x, y in ((self.K, K), (self.V, V), (self.ks, ks), (self.vs, vs)):
            x.copy_(y)
        return out


def window_of(window, sinks):
    def seen(n):
        t = torch.arange(n)
        return t if window == 0 else t[(t >= n - window) | (t < sinks)]
    return seen


def check_windowed(pc, lens, G, qdt, window=0, sinks=0, per_head=True, scale=0.0, odt=None, workspace=None, hide=True, seed=1):
    """Rows that do not attend hold anything, pages without any that does have no number in the table."""
    B, H, d = pc.B, pc.H, pc.d
    seen = window_of(window, sinks)
    if isinstance(pc, Paged8):
        rows = pc.fill(lens, seen)
    else:
        rows = {}
        for key, (k, v, c) in Paged.fill(pc, lens).items():
            t = seen(k.shape[0])
            rows[key] = (k[t], v[t], None if c is None else c[t])
        K, V = pc.K.cpu(), pc.V.cpu()
        for b in range(B):
            for h in range(H):
                t = torch.ones(lens[b][h], dtype=torch.bool)
                t[seen(lens[b][h])] = False
                page, head, row = pc.place(b, h, t.nonzero()[:, 0])
                K[page, head, row] = math.nan
                V[page, head, row] = math.inf
        pc.K.copy_(K)
        pc.V.copy_(V)
    table = pc.table.clone()
    if hide:
        flat = table.reshape(-1, pc.P)
        for i in range(flat.shape[0]):
            n = max(lens[i]) if not pc.per_head_table else lens[i // H][i % H]
            if pc.per_head_table or len(set(lens[i])) == 1:
                used = torch.zeros(pc.P, dtype=torch.bool)
                used[seen(n) // pc.R] = True
                flat[i][~used] = torch.tensor([-1, 2**31 - 1, -(2**31), pc.n])[torch.arange(int((~used).sum())) % 4].to(torch.int32)
    Q = (1.5 * torch.randn((B, H * G, d), generator=torch.Generator().manual_seed(seed))).to(qdt)
    dl = torch.tensor(lens, dtype=torch.int32)
    dl = (dl if per_head else dl[:, 0].contiguous()).to(DEV)
    O = None if odt is None else torch.empty((B, H * G, d), dtype=odt, device=DEV)
    call = sc.sc_paged8_decode_attn if isinstance(pc, Paged8) else sc.sc_paged_window_attn
    O, lse = call(pc.cache(table), Q.to(DEV), dl, window=window, sinks=sinks, scale=scale, O=O, want_lse=True, workspace=workspace)
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(H):
            heads = slice(h * G, (h + 1) * G)
            wo, wl, to, tl = attend(Q[b, heads].double(), rows[b, h], scale or 1 / math.sqrt(d))
            close(O[b, heads], wo, to * (1 + 2 / d) + half_step(O.dtype) * wo.abs() * (1 + 2.0**-6) + 1e-30)
            close(lse[b, heads], wl, tl * (1 + 2 / d))
    return O, lse


# ------------------------------------------------------------------------------------------------ attention over codes
@pytest.mark.parametrize("code", [E4, I8])
@pytest.mark.parametrize("d,R,block,G,qdt", [(128, 64, 16, 4, BF), (128, 16, 16, 1, F32), (64, 32, 32, 7, BF), (64, 128, 128, 16, F32), (128, 256, 64, 3, BF)])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 33, 256, 257, 700])
def test_decode_lengths(code, d, R, block, G, qdt, n):
    pc = Paged8(2, 2, -(-n // R), R, d, code, block, seed=n)
    check_windowed(pc, [[n, n], [max(1, n // 2)] * 2], G, qdt, per_head=n % 2 == 0)


@pytest.mark.parametrize("code", [E4, I8])
@pytest.mark.parametrize("layout", ["phrd", "prhd", "pkv"])
def test_decode_layouts_and_empty_sequences(code, layout):
    pc = Paged8(3, 2, 6, 32, 128, code, 16, layout=layout, seed=3)
    O, lse = check_windowed(pc, [[0, 0], [100, 100], [192, 192]], 2, BF, per_head=False)
    assert (O[0] == 0).all() and (lse[0] == -math.inf).all()


@pytest.mark.parametrize("code,qdt,odt", [(E4, BF, F32), (I8, F32, BF), (E4, F32, F32)])
def test_decode_merged_rows_with_sizes(code, qdt, odt):
    pc = Paged8(2, 3, 20, 16, 128, code, 16, per_head_table=True, counts=True, seed=5)
    check_windowed(pc, [[300, 1, 17], [0, 250, 320]], 4, qdt, odt=odt)


@pytest.mark.parametrize("code", [E4, I8])
def test_decode_heads_split_over_workgroups(code):
    pc = Paged8(1, 2, 160, 64, 128, code, 32, seed=7)
    ws = sc.paged_workspace(1, 8, 2, 128, 160, DEV)
    for n in (10000, 5000, 10240):      # the same workspace again
        check_windowed(pc, [[n, n]], 4, BF, odt=F32, workspace=ws, scale=0.4)


def test_decode_more_heads_than_workgroups():
    pc = Paged8(40, 8, 20, 32, 64, E4, 16, seed=8)
    gen = torch.Generator().manual_seed(8)
    lens = [[n] * 8 for n in torch.randint(0, 641, (40,), generator=gen).tolist()]
    check_windowed(pc, lens, 2, BF, per_head=False)


# ------------------------------------------------------------------------------------------------ windows
@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3", "i8"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (17, 16), (100, 0), (100, 33), (250, 5), (1000, 4), (2**31 - 1, 2**31 - 1), (5, 2**31 - 1)])
def test_windows(kind, window, sinks):
    G, d, R = 3, 64, 16
    lens = [[n, n] for n in (1, 16, 31, 100, 133, 480)]
    if kind in ("bf16", "f32"):
        pc = Paged(6, 2, 30, R, d, BF if kind == "bf16" else F32, seed=window % 97 + sinks % 13)
    else:
        pc = Paged8(6, 2, 30, R, d, E4 if kind == "e4m3" else I8, 16, seed=window % 97 + sinks % 13)
    check_windowed(pc, lens, G, F32 if kind == "f32" else BF, window=window, sinks=sinks, per_head=False, odt=F32)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_windows_of_merged_rows_and_large_ones(kind):
    make = (lambda *a, **k: Paged(*a, BF, **k)) if kind == "bf16" else (lambda *a, **k: Paged8(*a, E4, 32, **k))
    check_windowed(make(2, 2, 30, 32, 128, per_head_table=True, counts=True, seed=11), [[900, 10], [321, 960]], 4, BF, window=200, sinks=40)
    check_windowed(make(2, 1, 150, 64, 128, seed=12), [[9600], [7000]], 8, F32, window=4000, sinks=100, odt=F32)


@pytest.mark.parametrize("code", [E4, I8])
def test_a_block_whose_scale_is_no_number_shows_where_it_attends(code):
    pc = Paged8(1, 1, 8, 16, 128, code, 16, seed=13)
    pc.fill([[128]])
    page, head, row = pc.place(0, 0, torch.tensor([40]))
    Q, lens = torch.randn((1, 2, 128), device=DEV).to(BF), torch.tensor([128], dtype=torch.int32, device=DEV)
    for which in (pc.ks, pc.vs):
        which[page, head, 0] = math.nan
    assert sc.sc_paged8_decode_attn(pc.cache(), Q, lens)[0].isnan().all()
    assert sc.sc_paged8_decode_attn(pc.cache(), Q, lens, window=80, sinks=32)[0].isfinite().all()      # rows 32 to 47 do not attend
    bad = pc.table.clone()
    bad[0, 7] = pc.n
    O, lse = sc.sc_paged8_decode_attn(pc.cache(bad), Q, lens, want_lse=True)
    assert O.isnan().all() and lse.isnan().all()


@pytest.mark.parametrize("code", [E4, I8])
def test_a_scale_that_is_no_number_does_not_show_where_no_row_of_its_block_has_weight(code):
    """Rows of size 0 or less weigh nothing, whatever is theirs; rows outside the window neither."""
    pc = Paged8(1, 1, 8, 32, 128, code, 16, per_head_table=True, counts=True, seed=15)
    pc.fill([[200]])
    t = torch.arange(48, 64)
    page, head, row = pc.place(0, 0, t)
    pc.counts[page, head, row] = torch.arange(16, dtype=torch.int32, device=DEV) % 3 - 2
    Q, lens = torch.randn((1, 3, 128), device=DEV).to(BF), torch.tensor([[200]], dtype=torch.int32, device=DEV)
    want = sc.sc_paged8_decode_attn(pc.cache(), Q, lens)[0]
    pc.ks[page, head, row // 16] = math.nan
    pc.vs[page, head, row // 16] = math.nan
    assert want.isfinite().all() and (sc.sc_paged8_decode_attn(pc.cache(), Q, lens)[0] == want).all()
    # a block whose last rows are behind the window, and the visible ones without weight
    want = sc.sc_paged8_decode_attn(pc.cache(), Q, lens, window=200 - 56, sinks=8)[0]
    pc.counts[page, head, row] = 1
    pc.counts[page[8:], head, row[8:]] = 0
    assert want.isfinite().all() and (sc.sc_paged8_decode_attn(pc.cache(), Q, lens, window=200 - 56, sinks=8)[0] == want).all()


# ------------------------------------------------------------------------------------------------ appending
def turned(x, cos, sin, rot, interleaved):
    """fp32, rounded product by product; x [N, d], cos and sin [N, rot / 2]."""
    a, b = (x[:, 0:rot:2], x[:, 1:rot:2]) if interleaved else (x[:, : rot // 2], x[:, rot // 2 : rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    t = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((t, x[:, rot:]), 1)


def appended(code, block, codes, scales, base, x):
    """One head's rows: codes [T, d] as bytes and scales [T / block] after x [n, d] fp32 has gone to rows base .. base + n."""
    codes, scales = codes.clone(), scales.clone()
    n = x.shape[0]
    for k in range(base // block, -(-(base + n) // block) if n else 0):
        t0, r0, r1 = k * block, max(base, k * block), min(base + n, (k + 1) * block)
        new = x[r0 - base : r1 - base]
        need = smallest_scale(code, float(new.abs().max()))
        old = float(scales[k])
        scale = need if r0 == t0 else (math.nan if math.isnan(need) or math.isnan(old) else max(need, old))
        if r0 > t0 and scale > old:
            ratio = torch.tensor(old) / torch.tensor(scale)
            codes[t0:r0] = encode(code, decode(code, codes[t0:r0]) * ratio)
        codes[r0:r1] = encode(code, new * (1 / torch.tensor(scale, dtype=torch.float32)))
        scales[k] = scale
    return codes, scales


def check_append(pc, base, new, N, dtype, rot=0, interleaved=False, per_head=False, G=0, seed=0, spread=True, sizes=False):
    B, H, d, R = pc.B, pc.H, pc.d, pc.R
    gen = torch.Generator().manual_seed(seed)
    pc.fill(base)
    K, V = (torch.randn((B, H, N, d), generator=gen) for _ in range(2))
    if spread:      # blocks whose scales grow, shrink and stay
        K, V = (x * torch.exp2(torch.randint(-12, 12, (B, H, N, 1), generator=gen).float()) for x in (K, V))
    K, V = K.to(dtype), V.to(dtype)
    before = [x.cpu().clone() for x in (pc.K, pc.V, pc.ks, pc.vs)]
    kw = {}
    if rot:
        a = torch.arange(4096, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
        cos_sin = torch.cat((a.cos(), a.sin()), 1).float()
        positions = torch.tensor([7 + 3 * b for b in range(B)], dtype=torch.int32)
        kw = dict(cos_sin=cos_sin.to(DEV), positions=positions.to(DEV), interleaved=interleaved)
        if G:
            kw["Q"] = torch.randn((B, H * G, N, d), generator=gen).to(BF).to(DEV)
    if sizes:
        kw["counts"] = torch.randint(1, 99, (B, H, N), generator=gen, dtype=torch.int32).to(DEV)
    lens32 = lambda x: (torch.tensor(x, dtype=torch.int32) if per_head else torch.tensor(x, dtype=torch.int32)[:, 0].contiguous()).to(DEV)  # noqa: E731
    lens = torch.full_like(lens32(base), -7)
    _, Qo = sc.sc_paged8_append(pc.cache(), K.to(DEV), V.to(DEV), lens32(base), lens, new_lens=lens32(new), **kw)
    torch.cuda.synchronize()
    want = [x.clone() for x in before]
    sized = None if pc.counts is None else pc.counts.cpu()
    for b in range(B):
        for h in range(H):
            o, n = base[b][h], new[b][h]
            t = torch.arange(min(-(-(o + n) // pc.block) * pc.block, pc.P * R))
            page, head, row = pc.place(b, h, t)
            for pool, scales, x in ((0, 2, K), (1, 3, V)):
                y = x[b, h, :n].float()
                if rot and pool == 0:
                    at = int(positions[b]) + torch.arange(n)
                    y = turned(y, cos_sin[at, : rot // 2], cos_sin[at, rot // 2 :], rot, interleaved)
                blocks = (page[:: pc.block], head, row[:: pc.block] // pc.block)
                codes, s = appended(pc.code, pc.block, before[pool][page, head, row], before[scales][blocks], o, y)
                want[pool][page, head, row], want[scales][blocks] = codes, s
                # how far the codes are from the numbers
                held, scale = decode(pc.code, codes[o : o + n]).double(), s.repeat_interleave(pc.block)[o : o + n, None].double()
                step = torch.maximum(y.double().abs() * 2.0**-4, scale * 2.0**-10) if pc.code == E4 else scale / 2
                if n:
                    assert ((held * scale - y.double()).abs() <= step * (1 + 2.0**-20)).all()
            if sizes:
                assert (sized[page[o : o + n], head, row[o : o + n]] == kw["counts"][b, h, :n].cpu()).all()
    for got, w in zip((pc.K, pc.V, pc.ks, pc.vs), want):
        got = got.cpu()
        assert ((got == w) | (got.isnan() & w.isnan() if got.is_floating_point() else torch.zeros_like(got, dtype=torch.bool))).all()
    assert lens.cpu().tolist() == (torch.tensor(base) + torch.tensor(new) if per_head else (torch.tensor(base) + torch.tensor(new))[:, 0]).tolist()
    return K, V, Qo


@pytest.mark.parametrize("code", [E4, I8])
@pytest.mark.parametrize("d,R,block,dtype", [(128, 64, 16, BF), (64, 16, 16, BF), (128, 64, 64, F32), (128, 128, 128, BF), (64, 128, 128, F32), (128, 32, 32, BF), (64, 64, 64, BF), (64, 32, 16, F32)])
@pytest.mark.parametrize("base,N", [(0, 1), (5, 1), (16, 1), (127, 1), (0, 200), (13, 60), (64, 64), (1, 15), (100, 129)])
def test_append(code, d, R, block, dtype, base, N):
    P = -(-(base + N) // R) + 1
    pc = Paged8(2, 2, P, R, d, code, block, seed=base + N)
    rot = (0, d, d // 2, 16)[(base + N) % 4]
    check_append(pc, [[base] * 2, [base // 2] * 2], [[N] * 2, [max(0, N - 3)] * 2], N, dtype, rot=rot, interleaved=base % 2 == 1, G=2 if rot else 0, seed=N)


@pytest.mark.parametrize("code", [E4, I8])
@pytest.mark.parametrize("layout", ["prhd", "pkv"])
def test_append_layouts(code, layout):
    check_append(Paged8(2, 3, 5, 32, 128, code, 32, layout=layout, seed=2), [[40] * 3, [0] * 3], [[70] * 3, [1] * 3], 70, BF, rot=128)


@pytest.mark.parametrize("code", [E4, I8])
def test_append_merged_rows(code):
    pc = Paged8(2, 3, 8, 16, 128, code, 16, per_head_table=True, counts=True, seed=4)
    check_append(pc, [[0, 3, 90], [17, 0, 16]], [[50, 0, 38], [1, 30, 16]], 50, BF, per_head=True, sizes=True)


@pytest.mark.parametrize("code", [E4, I8])
def test_tokens_appended_one_by_one_are_off_by_less_than_two_steps(code):
    """Numbers that grow from token to token: every token re-codes the block's rows."""
    pc = Paged8(1, 1, 2, 64, 64, code, 64, seed=6)
    gen = torch.Generator().manual_seed(6)
    x = torch.randn((64, 64), generator=gen) * torch.exp2(torch.arange(64) / 4.0 - 8)[:, None]
    cache, lens = pc.cache(), [torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2)]
    for t in range(64):
        sc.sc_paged8_append(cache, x[t].reshape(1, 1, 1, 64).to(DEV), -x[t].reshape(1, 1, 1, 64).to(DEV), lens[t % 2], lens[(t + 1) % 2])
    page = int(pc.table[0, 0])
    for pool, scales, want in ((pc.K, pc.ks, x), (pc.V, pc.vs, -x)):
        scale = float(scales[page, 0, 0])
        assert scale == smallest_scale(code, float(x.abs().max()))
        off = (decode(code, pool[page, 0].cpu()).double() * scale - want.double()).abs()
        # half a step at every rounding; halved from one to the next (int8), and for e4m3 exact but for its lowest range
        step = torch.maximum(want.abs().double() * 2.0**-4, torch.tensor(scale * 2.0**-9)) if code == E4 else torch.tensor(scale)
        assert (off <= step * (1 + 2.0**-20)).all()


@pytest.mark.parametrize("code", [E4, I8])
def test_numbers_that_are_not_finite_spoil_their_block_until_it_is_begun_again(code):
    pc = Paged8(1, 1, 3, 32, 64, code, 16, seed=9)
    cache = pc.cache()
    lens = [torch.tensor([n], dtype=torch.int32, device=DEV) for n in (0, 0)]
    for bad in (math.nan, math.inf, -math.inf):
        x = torch.randn((1, 1, 40, 64), device=DEV)
        y = x.clone()
        y[0, 0, 20, 3] = bad
        sc.sc_paged8_append(cache, x, y, lens[0], lens[1])
        page = pc.table[0].long()
        assert pc.ks[page[:1]].isfinite().all() and pc.ks[page[1], 0, 0].isfinite()
        assert pc.vs[page[0], 0, 0].isfinite() and pc.vs[page[0], 0, 1].isnan() and pc.vs[page[1], 0, 0].isfinite()
        Q = torch.randn((1, 1, 64), device=DEV)
        assert sc.sc_paged8_decode_attn(cache, Q, lens[1])[0].isnan().all()
        assert sc.sc_paged8_decode_attn(cache, Q, lens[1], window=8)[0].isfinite().all()
        # more rows behind it do not heal it; rows from the block's first one on do
        twenty = torch.tensor([24], dtype=torch.int32, device=DEV)
        sc.sc_paged8_append(cache, x[:, :, :4].contiguous(), x[:, :, :4].contiguous(), twenty, lens[1])
        assert pc.vs[page[0], 0, 1].isnan()
        sc.sc_paged8_append(cache, x[:, :, :4].contiguous(), x[:, :, :4].contiguous(), torch.tensor([16], dtype=torch.int32, device=DEV), lens[1])
        assert pc.vs[page[0], 0, 1].isfinite()


def test_append_extreme_numbers():
    for code in (E4, I8):
        pc = Paged8(1, 1, 1, 64, 64, code, 16, seed=1)
        x = torch.zeros((1, 1, 64, 64))
        x[0, 0, 16:32] = torch.finfo(torch.float32).max
        x[0, 0, 32:48] = torch.finfo(torch.float32).tiny / 4
        x[0, 0, 48, 0], x[0, 0, 49, 1] = LARGEST[code], -LARGEST[code] * (1 - 2.0**-23)
        lens = torch.zeros(1, dtype=torch.int32, device=DEV)
        sc.sc_paged8_append(pc.cache(), x.to(DEV), x.to(DEV), lens, lens.clone())
        page = int(pc.table[0, 0])
        assert pc.ks[page, 0].tolist() == [2.0**-126, smallest_scale(code, torch.finfo(torch.float32).max), 2.0**-126, 1.0]
        got = decode(code, pc.K[page, 0].cpu()).double()      # (256 * 2^120 is beyond fp32)
        assert (got[:16] == 0).all() and (got[48, 0] == LARGEST[code]) and (got[49, 1] == -LARGEST[code])
        assert ((got[16:32] * pc.ks[page, 0, 1].item() / torch.finfo(torch.float32).max - 1).abs() <= 2.0**-4).all()


@pytest.mark.parametrize("code", [E4, I8])
def test_append_reports_what_the_device_finds(code):
    """As sc_paged_append does: -1 and nothing written where the lengths are impossible; a bad page spoils only itself."""
    pc = Paged8(4, 1, 3, 16, 64, code, 16, seed=14)
    before = [x.clone() for x in (pc.K, pc.V, pc.ks, pc.vs)]
    base = torch.tensor([-1, 47, 5, 30], dtype=torch.int32, device=DEV)
    new = torch.tensor([1, 2, 6, 4], dtype=torch.int32, device=DEV)
    table = pc.table.clone()
    table[3, 2] = pc.n
    lens = torch.zeros(4, dtype=torch.int32, device=DEV)
    x = torch.randn((4, 1, 5, 64), device=DEV)
    sc.sc_paged8_append(pc.cache(table), x, x, base, lens, new_lens=new)
    assert lens.tolist() == [-1, -1, -1, -1]
    page = int(table[3, 1])
    for got, was in zip((pc.K, pc.V, pc.ks, pc.vs), before):
        changed = torch.ones(pc.n, dtype=torch.bool)
        changed[page] = False
        a, b = got.cpu()[changed], was.cpu()[changed]
        assert ((a == b) | ((a != a) & (b != b))).all()
    assert (pc.K[page, 0, 14:].cpu() != before[0][page, 0, 14:].cpu()).any()


def test_tensors_on_another_device_than_the_current_one_are_refused(monkeypatch):
    """(The current device is said to be another one.)  With and without outputs and workspaces of the caller's; nothing is changed."""
    pc, B, H, G, d = Paged8(2, 2, 3, 16, 64, E4, 16, seed=3), 2, 2, 2, 64
    lens, one = torch.tensor([20, 5], dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    Q, X, P = torch.randn((B, H * G, d), device=DEV), torch.randn((B, H, 1, d), device=DEV), torch.randn((B, H * G, 3, d), device=DEV)
    O, OP, out, slots = torch.full_like(Q, 7), torch.full_like(P, 7), torch.full_like(lens, 7), torch.full((2, 1), 7, dtype=torch.int32, device=DEV)
    plain = sc.PagedCache(torch.zeros((pc.n, H, 16, d), device=DEV), torch.zeros((pc.n, H, 16, d), device=DEV), pc.table.to(DEV))
    table, free = torch.full((2, 3), -1, dtype=torch.int32, device=DEV), torch.arange(4, dtype=torch.int32, device=DEV)
    ws, wr, wp = sc.paged_workspace(B, H * G, H, d, 3, DEV), sc.paged_reserve_workspace(2, 3, DEV), sc.prompt_attn_workspace(B, H * G, H, 3, 1, d, DEV)
    cache = pc.cache()
    kept = [t.clone() for t in (pc.K, pc.ks.view(torch.int32), table, free)]
    torch.cuda.synchronize()
    with monkeypatch.context() as m:
        m.setattr(torch._C, "_cuda_getDevice", lambda: 1)
        for call in (lambda: sc.sc_paged8_append(cache, X, X, lens, out), lambda: sc.sc_paged8_append(cache, X, X, lens, out, Q=X, cos_sin=torch.zeros((64, 64), device=DEV)),
                     lambda: sc.sc_paged8_decode_attn(cache, Q, lens, O=O, workspace=ws), lambda: sc.sc_paged8_decode_attn(cache, Q, lens, want_lse=True, workspace=ws),
                     lambda: sc.sc_paged_window_attn(plain, Q, lens, 4, O=O, workspace=ws), lambda: sc.sc_paged_window_attn(plain, Q, lens, 4, workspace=ws), lambda: sc.sc_paged_window_attn(plain, Q, lens, 4),
                     lambda: sc.sc_paged_reserve(table, 16, lens, out, free, one, slots=slots, workspace=wr), lambda: sc.sc_paged_reserve(table, 16, lens, out, free, one),
                     lambda: sc.sc_prompt_attn(P, X, X, O=OP, workspace=wp), lambda: sc.sc_prompt_attn(P, X, X)):
            with pytest.raises(sc.SemantiCacheError, match="current device"):
                call()
    torch.cuda.synchronize()
    assert all((t == 7).all() for t in (O, OP, out, slots)) and one.item() == 1
    assert all(torch.equal(a, b) for a, b in zip(kept, (pc.K, pc.ks.view(torch.int32), table, free)))
