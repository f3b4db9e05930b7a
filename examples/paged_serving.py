"""Serving from a cache held in pages: ragged prompts, then generated tokens, for several attention layers with random weights.

Every layer keeps its keys and values in pages of a pool that all sequences share.
  prompt   sc_paged_append takes the fused projection as it is, rotates keys and queries and files the rows; attention inside the prompt is not
           shown (any prefill kernel does it).
  token    sc_paged_append for the new token of every sequence, sc_paged_select keeps the pages that the query can attend to most, and
           sc_paged_decode_attn attends to those; or to all of them (--keep 0).
  merged   with --merge the prompt's cache is compressed first (sc_segment, sc_gsc_merge): every KV head of a sequence then has its own number of
           rows, with sizes, in pages of its own, and the tokens that follow are appended behind them with size 1.

    python examples/paged_serving.py --tokens 32 --keep 24
    python examples/paged_serving.py --tokens 32 --merge
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_14303_amd import binding as sc  # noqa: E402

R, D = 64, 128      # rows of a page, elements of a row


def angles(positions: int, rot: int, device) -> torch.Tensor:
    a = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    return torch.cat((a.cos(), a.sin()), 1).float().to(device)


class Layer:
    """Projections and the cache of one layer."""

    def __init__(self, width: int, Hkv: int, G: int, lens, room: int, merge_mask, tau: float, gen):
        dev = gen.device
        self.Hkv, self.G, self.merged = Hkv, G, merge_mask is not None
        self.qkv = torch.randn((width, (G + 2) * Hkv * D), generator=gen, device=dev).mul_(width**-0.5).to(torch.bfloat16)
        self.out = torch.randn((Hkv * G * D, width), generator=gen, device=dev).mul_((Hkv * G * D) ** -0.5).to(torch.bfloat16)
        self.mask, self.tau = merge_mask, tau
        B, P = len(lens), -(-(max(lens) + room) // R)
        tables, heads = (B * Hkv, 1) if self.merged else (B, Hkv)
        pool = torch.zeros((tables * P, 2, heads, R, D), dtype=torch.bfloat16, device=dev)
        table = torch.randperm(tables * P, generator=gen, device=dev).to(torch.int32).reshape((B, Hkv, P) if self.merged else (B, P))
        summaries = [torch.zeros((tables * P, heads, D), dtype=torch.bfloat16, device=dev) for _ in range(2)]
        counts = torch.zeros((tables * P, heads, R), dtype=torch.int32, device=dev) if self.merged else None
        self.cache = sc.PagedCache(pool[:, 0], pool[:, 1], table, counts=counts, k_min=summaries[0], k_max=summaries[1])
        self.ws = sc.paged_workspace(B, Hkv * G, Hkv, D, P, dev)
        self.lens = torch.zeros((B, Hkv) if self.merged else (B,), dtype=torch.int32, device=dev)
        self.fresh = torch.empty_like(self.lens)

    def split(self, x):
        """x [B, N, width] -> views [B, heads, N, D] of the fused projection."""
        y = (x @ self.qkv).unflatten(-1, (-1, D)).permute(0, 2, 1, 3)
        return y.split((self.G * self.Hkv, self.Hkv, self.Hkv), 1)

    def advance(self):
        self.lens, self.fresh = self.fresh, self.lens

    def prompt(self, x, prompt_lens, cos_sin):
        q, k, v = self.split(x)
        if not self.merged:
            sc.sc_paged_append(self.cache, k, v, self.lens, self.fresh, new_lens=prompt_lens, Q=q, cos_sin=cos_sin)
        else:
            # the compression works on rotated keys: file them in a dense array first (pages of that array's own rows)
            B, H, N, _ = k.shape
            pages = -(-N // R)
            dense = torch.zeros((2, B, H, pages * R, D), dtype=k.dtype, device=k.device)
            scratch = sc.PagedCache(*dense.unflatten(3, (pages, R)).reshape(2, B * H * pages, 1, R, D),
                                    torch.arange(B * H * pages, dtype=torch.int32, device=k.device).reshape(B, H, pages))
            sc.sc_paged_append(scratch, k, v, torch.zeros_like(prompt_lens), torch.empty_like(prompt_lens), new_lens=prompt_lens, cos_sin=cos_sin)
            K, V = (t[:, :, :N] for t in dense)
            offsets, chunks = sc.sc_segment(self.mask, prompt_lens)
            Kc, Vc, counts, rows, _ = sc.sc_gsc_merge(K, V, offsets, chunks, self.tau, seq_lens=prompt_lens)
            sc.sc_paged_append(self.cache, Kc, Vc, self.lens, self.fresh, new_lens=rows, counts=counts)
        self.advance()

    def token(self, x, positions, cos_sin, keep: int):
        """x [B, 1, width], positions int32 [B] -> attention output [B, 1, width]."""
        q, k, v = self.split(x)
        B = x.shape[0]
        counts = torch.ones((B, self.Hkv, 1), dtype=torch.int32, device=x.device) if self.merged else None
        _, q = sc.sc_paged_append(self.cache, k, v, self.lens, self.fresh, counts=counts, Q=q, cos_sin=cos_sin, positions=positions)
        self.advance()
        q = q.flatten(1).unflatten(1, (-1, D))
        chosen = {}
        if keep:
            chosen["sel"], chosen["sel_lens"] = sc.sc_paged_select(self.cache, q, self.lens, keep, first=1, recent=2, workspace=self.ws)
        O, _ = sc.sc_paged_decode_attn(self.cache, q, self.lens, workspace=self.ws, **chosen)
        return (O.flatten(1) @ self.out)[:, None]


def serve(layers: int = 2, lens=(900, 2000, 1400, 64), tokens: int = 16, keep: int = 12, merge: bool = False, width: int = 512, Hkv: int = 4, G: int = 4,
          tau: float = 0.3, seed: int = 0):
    """Prompts of the given lengths, then `tokens` steps for all sequences; returns the layers and the last hidden states."""
    dev = torch.device("cuda")
    gen = torch.Generator(dev).manual_seed(seed)
    B, N = len(lens), max(lens)
    prompt_lens = torch.tensor(lens, dtype=torch.int32, device=dev)
    mask = (torch.rand((B, N), generator=gen, device=dev) < 0.05).to(torch.uint8) if merge else None
    cos_sin = angles(N + tokens, D, dev)
    model = [Layer(width, Hkv, G, lens, tokens, mask, tau, gen) for _ in range(layers)]
    x = torch.randn((B, N, width), generator=gen, device=dev).to(torch.bfloat16)
    for layer in model:
        layer.prompt(x, prompt_lens, cos_sin)
    x = torch.randn((B, 1, width), generator=gen, device=dev).to(torch.bfloat16)
    for step in range(tokens):
        positions = prompt_lens + step
        for layer in model:
            y = x + layer.token(x, positions, cos_sin, keep)
            x = (y.float() * y.float().square().mean(-1, keepdim=True).rsqrt()).to(torch.bfloat16)
    return model, x


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--tokens", type=int, default=16)
    p.add_argument("--keep", type=int, default=12, help="pages that a query attends to (0: all)")
    p.add_argument("--merge", action="store_true", help="compress the prompts first")
    a = p.parse_args()
    model, x = serve(tokens=a.tokens, keep=a.keep, merge=a.merge)
    for i, layer in enumerate(model):
        print("layer %d: rows %s" % (i, layer.lens.tolist()))
    print("last hidden states: mean square %.4f" % x.float().square().mean().item())


if __name__ == "__main__":
    main()
