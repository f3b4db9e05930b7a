"""examples/window_serving.py end to end: pages, prompts and every token's attention against plain evaluations over what the pages hold, and the captured
steps against eager ones."""
import math
import os
import sys

import pytest
import torch

from paper_2603_14303_amd import binding as sc
from test_gpu_paged8 import E4, decode

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
LENS = (130, 300, 64, 1)


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_every_step(code, monkeypatch):
    import window_serving as ex
    window, sinks, G = 40, 4, 3
    rows, calls = {}, []      # what each cache was given, in fp64: (cache, sequence, head) -> [n, d] keys and values
    append, attend, prompt = sc.sc_paged8_append, sc.sc_paged8_decode_attn, sc.sc_prompt_attn

    def appended(cache, K, V, base, lens, new_lens=None, Q=None, cos_sin=None):
        out = append(cache, K, V, base, lens, new_lens=new_lens, Q=Q, cos_sin=cos_sin)
        assert (lens == base + new_lens).all()
        k, v = K.cpu().double(), V.cpu().double()
        for b in range(k.shape[0]):
            o, n = int(base[b]), int(new_lens[b])
            if cos_sin is not None and n:      # one token, rotated by its position
                half = ex.D // 2
                c, s = cos_sin[o].cpu().double().split(half)
                a, e = k[b, :, :, :half].clone(), k[b, :, :, half:].clone()
                k[b] = torch.cat((a * c - e * s, e * c + a * s), -1)
            for h in range(k.shape[1]):
                was = rows.get((id(cache), b, h), (torch.zeros((0, ex.D), dtype=torch.float64),) * 2)
                rows[id(cache), b, h] = tuple(torch.cat((w[:o], x[b, h, :n])) for w, x in zip(was, (k, v)))
        return out

    def attended(cache, Q, lens, window=0, sinks=0, O=None, workspace=None):
        O, lse = attend(cache, Q, lens, window=window, sinks=sinks, O=O, workspace=workspace)
        K, V, table = (x.cpu() for x in (cache.K.view(torch.uint8), cache.V.view(torch.uint8), cache.table))
        ks, vs = cache.k_scale.cpu().double(), cache.v_scale.cpu().double()
        for b in range(Q.shape[0]):
            n = int(lens[b])
            if n == 0:
                assert (O[b] == 0).all()
                continue
            t = torch.arange(n)
            t = t[(t >= n - window) | (t < sinks)]
            page, row = table[b, t // ex.R].long(), t % ex.R
            assert (page >= 0).all()
            for h in range(cache.Hkv):
                k, v = ((decode(cache.K.dtype, pool[page, h, row]).double(), s[page, h, row // ex.E][:, None]) for pool, s in ((K, ks), (V, vs)))
                # codes: half a step off what was appended (bf16 numbers, rotated in fp32), and less than one more where a block has grown token by token
                for (c, s), want in zip((k, v), rows[id(cache), b, h]):
                    step = torch.maximum(want[t].abs() * 2.0**-4, s * 2.0**-9) if cache.K.dtype == E4 else s
                    assert ((c * s - want[t]).abs() <= step * (1 + 2.0**-20)).all()
                k, v = k[0] * k[1], v[0] * v[1]
                q = Q[b, h * G : (h + 1) * G].cpu().double()
                z = q @ k.T / math.sqrt(ex.D)
                w = torch.softmax(z, 1)
                # logits in fp32, weights of 16 bits and more, O rounded to bf16 (half a step: 2^-8)
                delta = (ex.D + 18) * 2.0**-24 * ((q.abs() @ k.abs().T / math.sqrt(ex.D)).amax(1) + z.abs().amax(1))
                want = w @ v
                tol = (2 * delta + 2.0**-17 + (n / 16 + 256) * 2.0**-24)[:, None] * (w @ v.abs()) + 2.0**-8 * want.abs()
                assert ((O[b, h * G : (h + 1) * G].cpu().double() - want).abs() <= tol).all()
        calls.append("token")
        return O, lse

    def prompted(Q, K, V, q_lens=None, kv_lens=None, window=0, sinks=0, O=None):
        prompt(Q, K, V, q_lens=q_lens, kv_lens=kv_lens, window=window, sinks=sinks, O=O)
        for b, n in enumerate(q_lens.tolist()):
            i, j = torch.arange(n)[:, None], torch.arange(n)[None]
            seen = (j <= i) & ((j > i - window) | (j < sinks))
            for h in range(Q.shape[1]):
                q, k, v = Q[b, h, :n].cpu().double(), K[b, h // G, :n].cpu().double(), V[b, h // G, :n].cpu().double()
                z = (q @ k.T / math.sqrt(ex.D)).masked_fill(~seen, -math.inf)
                w = torch.softmax(z, 1)
                delta = (ex.D + 16) * 2.0**-24 * ((q.abs() @ k.abs().T / math.sqrt(ex.D)).amax(1) + z.masked_fill(~seen, 0).abs().amax(1))
                want = w @ v
                tol = (2 * delta + 2.0**-8 + (n + 256) * 2.0**-24)[:, None] * (w @ v.abs()) + 2.0**-8 * want.abs() * (1 + 2.0**-6)      # (probabilities are bf16)
                assert ((O[b, h, :n].cpu().double() - want).abs() <= tol).all()
            assert (O[b, :, n:] == 0).all()
        calls.append("prompt")
        return O, None

    monkeypatch.setattr(ex.sc, "sc_paged8_append", appended)
    monkeypatch.setattr(ex.sc, "sc_paged8_decode_attn", attended)
    monkeypatch.setattr(ex.sc, "sc_prompt_attn", prompted)
    held = []

    def watch(pages, step):
        table = pages.table.cpu()
        mine = table[table >= 0].tolist() + pages.free[: int(pages.many)].tolist()
        assert sorted(mine) == list(range(pages.free.numel()))      # every page in one place
        held.append([int((row >= 0).sum()) for row in table])

    pages, model, x = ex.serve(layers=2, lens=LENS, tokens=5, window=window, sinks=sinks, code=code, ends={3: 2}, width=128, Hkv=2, G=G, graph=False, watch=watch)
    assert calls == ["prompt"] * 2 + ["token"] * 10 and torch.isfinite(x.float()).all()
    assert pages.lens.tolist() == [135, 305, 0, 6]
    assert held[0] == [-(-n // ex.R) for n in LENS]
    most = 1 + -(-window // ex.R) + 1
    assert all(n <= most for step in held[1:] for n in step) and held[-1][2] == 0


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_captured_steps_are_those_of_an_eager_program(code):
    import window_serving as ex
    kw = dict(layers=2, lens=LENS, tokens=40, window=33, sinks=3, code=code, ends={7: 1, 20: 0}, width=128, Hkv=2, G=2)
    states = []
    for graph in (False, True):
        pages, model, x = ex.serve(graph=graph, **kw)
        torch.cuda.synchronize()
        states.append((x, pages.table, pages.free[: int(pages.many)], pages.lens, *(t for layer in model for t in (layer.cache.K.view(torch.uint8), layer.cache.k_scale))))
    for a, b in zip(*states):
        assert a.shape == b.shape and (a == b).all()
