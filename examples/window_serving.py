"""Serving from caches that stay small: rows of 8 bits, a sliding window with first tokens that stay, pages handed out and taken back on the GPU.

Every layer attends to the newest `window` tokens and the first `sinks` ones, so a sequence holds a bounded number of pages however long it gets.
  pages    sc_paged_reserve gives every sequence the pages for the rows that arrive and takes back those that left its window; a request that ends
           gives back all of them.  A sequence that there is no page for waits with what it has, until a request ends.  One table serves all layers.
  prompt   sc_paged_append rotates keys and queries (filing the keys in an array of their own), sc_prompt_attn attends, and sc_paged8_append files the
           rows as 8-bit codes.
  token    sc_paged8_append and sc_paged8_decode_attn for the new token of every sequence.  The step is captured into a graph once: lengths, tables
           and the stack of free pages are on the GPU, so the host has nothing to decide between tokens.

    python examples/window_serving.py --tokens 64 --window 256 --code i8
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_14303_amd import binding as sc  # noqa: E402

R, E, D = 32, 16, 128      # rows of a page, rows of a scale, elements of a row
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}


def angles(positions: int, rot: int, device) -> torch.Tensor:
    a = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    return torch.cat((a.cos(), a.sin()), 1).float().to(device)


class Pages:
    """The table of all sequences and the stack of pages that none of them holds."""

    def __init__(self, B: int, most_rows: int, pages: int, window: int, sinks: int, device):
        P = -(-most_rows // R)
        self.window, self.sinks = window, sinks
        self.table = torch.full((B, P), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(pages, dtype=torch.int32, device=device)
        self.many = torch.full((1,), pages, dtype=torch.int32, device=device)
        self.lens = torch.zeros(B, dtype=torch.int32, device=device)       # rows that the cache holds
        self.next = torch.zeros_like(self.lens)                            # and will hold after the step; -1: there is no page for it
        self.ws = sc.paged_reserve_workspace(B, P, device)

    def reserve(self, new):
        sc.sc_paged_reserve(self.table, R, self.lens, self.next, self.free, self.many, new_lens=new, window=self.window, sinks=self.sinks, workspace=self.ws)

    def step(self, new):
        """Pages for the step's rows -> which sequences there are some for, and for the layers the rows that the cache holds and those that arrive: none of one that waits."""
        self.reserve(new)
        served = self.next >= 0
        return served, torch.where(served, self.lens, 0), torch.where(served, new, 0)

    def done(self, served):
        self.lens.copy_(torch.where(served, self.next, self.lens))

    def held(self) -> int:
        return int((self.table >= 0).sum())


class Layer:
    """Projections and the cache of one layer."""

    def __init__(self, width: int, Hkv: int, G: int, pages: Pages, code: str, gen):
        dev = gen.device
        self.Hkv, self.G, self.pages = Hkv, G, pages
        self.qkv = torch.randn((width, (G + 2) * Hkv * D), generator=gen, device=dev).mul_(width**-0.5).to(torch.bfloat16)
        self.out = torch.randn((Hkv * G * D, width), generator=gen, device=dev).mul_((Hkv * G * D) ** -0.5).to(torch.bfloat16)
        n, (B, P) = pages.free.numel(), pages.table.shape
        pool = torch.zeros((n, 2, Hkv, R, D), dtype=torch.uint8, device=dev).view(CODES[code])
        scales = [torch.zeros((n, Hkv, R // E), device=dev) for _ in range(2)]
        self.cache = sc.PagedCache8(pool[:, 0], pool[:, 1], *scales, pages.table)
        self.ws = sc.paged_workspace(B, Hkv * G, Hkv, D, P, dev)
        self.written = torch.zeros_like(pages.lens)
        self.O = torch.empty((B, Hkv * G, D), dtype=torch.bfloat16, device=dev)

    def split(self, x):
        """x [B, N, width] -> views [B, heads, N, D] of the fused projection."""
        y = (x @ self.qkv).unflatten(-1, (-1, D)).permute(0, 2, 1, 3)
        return y.split((self.G * self.Hkv, self.Hkv, self.Hkv), 1)

    def prompt(self, x, new, cos_sin):
        """Attention output of the prompts' rows; their keys and values are in the cache afterwards."""
        q, k, v = self.split(x)
        B, H, N, _ = k.shape
        many = -(-N // R)
        dense = torch.zeros((2, B, H, many * R, D), dtype=k.dtype, device=k.device)
        scratch = sc.PagedCache(*dense.unflatten(3, (many, R)).reshape(2, B * H * many, 1, R, D),
                                torch.arange(B * H * many, dtype=torch.int32, device=k.device).reshape(B, H, many))
        zero = torch.zeros_like(new)
        _, q = sc.sc_paged_append(scratch, k, v, zero, torch.empty_like(new), new_lens=new, Q=q, cos_sin=cos_sin)
        K, V = dense[0, :, :, :N], dense[1, :, :, :N]
        O = torch.zeros((B, N, self.G * H, D), dtype=q.dtype, device=q.device).permute(0, 2, 1, 3)
        sc.sc_prompt_attn(q, K, V, q_lens=new, kv_lens=new, window=self.pages.window, sinks=self.pages.sinks, O=O)
        sc.sc_paged8_append(self.cache, K, V, zero, self.written, new_lens=new)
        return O.permute(0, 2, 1, 3).flatten(2) @ self.out

    def token(self, x, base, new, cos_sin):
        """x [B, 1, width] -> attention output [B, 1, width] of a token behind base [B] rows; sequences with new = 0 are left alone."""
        q, k, v = self.split(x)
        _, q = sc.sc_paged8_append(self.cache, k, v, base, self.written, new_lens=new, Q=q, cos_sin=cos_sin)
        sc.sc_paged8_decode_attn(self.cache, q.flatten(1).unflatten(1, (-1, D)), self.written, window=self.pages.window, sinks=self.pages.sinks, O=self.O, workspace=self.ws)
        return (self.O.flatten(1) @ self.out)[:, None]


def normal(x):
    return (x.float() * x.float().square().mean(-1, keepdim=True).add(1e-6).rsqrt()).to(x.dtype)


def serve(layers: int = 2, lens=(900, 200, 400, 31), tokens: int = 16, window: int = 128, sinks: int = 4, code: str = "e4m3", ends=None, width: int = 512, Hkv: int = 4,
          G: int = 4, seed: int = 0, graph: bool = True, watch=None, pool=None):
    """Prompts of the given lengths, then `tokens` steps; `ends` {step: sequence}: that request ends before the step.  watch(pages, step) is called after
    the prompts (step -1) and every step.  pool: pages in all (None: as many as the sequences can need).  Returns pages, layers and the last hidden states."""
    dev = torch.device("cuda")
    gen = torch.Generator(dev).manual_seed(seed)
    B, N = len(lens), max(lens)
    # the prompts' pages are held until the first token; from then on all rows', or what the first tokens, a window and a page at its edge need
    prompts, ends_at = sum(-(-n // R) for n in lens), [-(-(n + tokens) // R) for n in lens]
    if pool is None:
        pool = max(prompts, sum(min(n, -(-sinks // R) - (-window // R) + 1) if window else n for n in ends_at))
    if pool < prompts:
        raise ValueError("the prompts fill %d pages, the pool has %d" % (prompts, pool))
    pages = Pages(B, N + tokens, pool, window, sinks, dev)
    cos_sin = angles(N + tokens, D, dev)
    model = [Layer(width, Hkv, G, pages, code, gen) for _ in range(layers)]
    new = torch.tensor(lens, dtype=torch.int32, device=dev)
    x = normal(torch.randn((B, N, width), generator=gen, device=dev).to(torch.bfloat16))
    pages.reserve(new)
    for layer in model:
        x = normal(x + layer.prompt(x, new, cos_sin))
    pages.lens.copy_(pages.next)
    if watch:
        watch(pages, -1)
    x = x[torch.arange(B, device=dev), new.long() - 1][:, None].contiguous()
    new.fill_(1)

    def step():
        served, base, rows = pages.step(new)
        y = x
        for layer in model:
            y = normal(y + layer.token(y, base, rows, cos_sin))
        x.copy_(torch.where(served[:, None, None], y, x))
        pages.done(served)

    captured = None
    for s in range(tokens):
        if ends and s in ends:      # its row of the table empties with the next reservation
            pages.lens[ends[s]] = 0
            new[ends[s]] = 0
        if not graph or s == 0:
            step()      # (the first one eagerly: libraries set themselves up)
        else:
            if captured is None:
                captured = torch.cuda.CUDAGraph()
                with torch.cuda.graph(captured):
                    step()
            captured.replay()
        if watch:
            watch(pages, s)
    return pages, model, x


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--tokens", type=int, default=64)
    p.add_argument("--window", type=int, default=256)
    p.add_argument("--sinks", type=int, default=4)
    p.add_argument("--code", choices=sorted(CODES), default="e4m3")
    a = p.parse_args()
    lens = (3000, 700, 1500, 64)
    told = []
    pages, model, x = serve(lens=lens, tokens=a.tokens, window=a.window, sinks=a.sinks, code=a.code, ends={a.tokens // 2: 1},
                            watch=lambda pages, s: told.append(pages.held()))
    print("rows of the sequences: %s" % pages.lens.tolist())
    print("pages held: %d after the prompts, %d after a token, %d at the end, of %d" % (told[0], told[1], told[-1], pages.free.numel()))
    print("last hidden states: mean square %.4f" % x.float().square().mean().item())


if __name__ == "__main__":
    main()
