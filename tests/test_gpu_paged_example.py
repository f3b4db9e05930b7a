"""examples/paged_serving.py end to end: every step's attention against a plain evaluation over the rows that the pages hold."""
import math
import os
import sys

import pytest
import torch

from paper_2603_14303_amd import binding as sc

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("merge, keep", [(False, 0), (False, 7), (True, 0), (True, 5)])
def test_serving(merge, keep, monkeypatch):
    import paged_serving as ex
    print("serving", merge, keep, flush=True)
    seen = []
    attend = sc.sc_paged_decode_attn

    def checked(cache, Q, lens, sel=None, sel_lens=None, workspace=None):
        O, lse = attend(cache, Q, lens, sel=sel, sel_lens=sel_lens, workspace=workspace)
        B, Hq, d = Q.shape
        H, G = cache.Hkv, Hq // cache.Hkv
        K, V, table = cache.K.cpu().double(), cache.V.cpu().double(), cache.table.cpu().long()
        counts = None if cache.counts is None else cache.counts.cpu().double()
        n = lens.cpu() if lens.dim() == 2 else lens.cpu()[:, None].expand(-1, H)
        for b in range(B):
            for h in range(H):
                tab, head = (table[b, h], 0) if table.dim() == 3 else (table[b], h)
                t = torch.arange(int(n[b, h]))
                if sel is not None:
                    kept = sel[b, h, : int(sel_lens[b, h])].cpu().long()
                    assert len(kept) == min(keep, -(-int(n[b, h]) // ex.R)) and kept[0] == 0 and kept[-1] == (int(n[b, h]) - 1) // ex.R
                    t = t[torch.isin(t // ex.R, kept)]
                page, row = tab[t // ex.R], t % ex.R
                z = Q[b, h * G : (h + 1) * G].cpu().double() @ K[page, head, row].T / math.sqrt(d)
                if counts is not None:
                    assert (counts[page, head, row] >= 1).all()
                    z = z + counts[page, head, row].log()
                want = torch.softmax(z, 1) @ V[page, head, row]
                got = O[b, h * G : (h + 1) * G].cpu().double()
                # logits in fp32 (d + 16 roundings over sum |q k|), weights of 16 bits, O rounded to bf16 (half a step: 2^-8)
                delta = (d + 16) * 2.0**-24 * ((Q[b, h * G : (h + 1) * G].cpu().double().abs() @ K[page, head, row].abs().T / math.sqrt(d)).amax(1) + z.abs().amax(1))
                tol = (2 * delta + 2.0**-17 + (len(t) / 16 + 256) * 2.0**-24)[:, None] * (torch.softmax(z, 1) @ V[page, head, row].abs()) + 2.0**-8 * want.abs()
                assert ((got - want).abs() <= tol).all(), (b, h, float(((got - want).abs() / tol).max()))
        seen.append(1)
        return O, lse

    monkeypatch.setattr(ex.sc, "sc_paged_decode_attn", checked)
    lens = (130, 300, 64, 1)
    model, x = ex.serve(layers=2, lens=lens, tokens=3, keep=keep, merge=merge, width=128, Hkv=2, G=3)
    assert len(seen) == 6 and torch.isfinite(x.float()).all()
    for layer in model:
        rows = layer.lens.cpu()
        if merge:
            assert rows.shape == (4, 2) and (rows >= 4).all() and (rows <= torch.tensor(lens)[:, None] + 3).all() and (rows.sum(1) < 2 * torch.tensor(lens) + 6)[:3].all()
        else:
            assert rows.tolist() == [n + 3 for n in lens]
