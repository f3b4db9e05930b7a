"""Measured cases of serving from a cache of bounded size: pages handed out on the GPU, rows kept in 8 bits, a sliding window with first tokens that stay.

Kinds
  reserve   sc_paged_reserve: pages for the rows that arrive, pages that are not needed any more go back, and the slots of the new rows; then the same
            call without the new rows, which gives back what the first one took (a step that is taken back, or a request that ends).
  append8   sc_paged8_append: new keys and values go to pages of 8-bit codes with a scale for every block of rows and head, rotated on the way,
            with the queries of the same tokens.
  decode8   sc_paged8_decode_attn: attention of one new token of every sequence over such a cache, all of it or a window and the first rows.
  window    sc_paged_window_attn: the same with a window over a cache that keeps its numbers.
  prompt    sc_prompt_attn: attention of a prompt's rows, or of a chunk of them behind a context, causal, with or without window and first tokens.

A cache: pools [pages, heads, R, d] (heads: all KV heads, or 1 where every KV head has pages of its own) and a table of page numbers [B, P] or [B, Hkv, P].
Row t of a sequence (and head) is row t % R of page table[..., t // R].  A row t of n rows is visible to the last one if t >= n - window or t < sinks; a window of 0
is none.  Layers, heads and lengths are those of the workloads in paper_2603_14303_amd/workloads.py and of the tests.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
LARGEST = {"e4m3": 448.0, "i8": 127.0}
LAYER = {"B": 1, "Hkv": 8, "G": 4, "d": 128, "R": 64, "dtype": "bf16", "ragged": False, "merged": False, "window": 0, "sinks": 0}
MAX_POSITION = 1 << 17


def listed():
    reserve = {"kind": "reserve", "S": 64, "R": 64, "rows": 16384, "N": 1, "window": 0, "sinks": 0, "ragged": True}
    append = {**LAYER, "kind": "append8", "code": "e4m3", "block": 16, "N": 1, "base": 8000, "rot": 128, "interleaved": False}
    decode = {**LAYER, "kind": "decode8", "code": "e4m3", "block": 16, "q": "bf16", "lse": False}
    window = {**LAYER, "kind": "window", "q": "bf16", "lse": False, "window": 4096, "sinks": 16}
    prompt = {**LAYER, "kind": "prompt", "N": 8192, "context": 0, "lse": False}
    return [
        # one generated token of each of 64 sequences of up to 16k tokens: mostly nothing to hand out
        {"name": "reserve_tokens_64", **reserve},
        # prompts of up to 32k tokens for the heads of 64 sequences, every head pages of its own
        {"name": "reserve_prompts_512", **reserve, "S": 512, "rows": 0, "N": 32768},
        # one generated token of each of 64 sequences of different lengths
        {"name": "append8_tokens_64", **append, "B": 64, "ragged": True},
        # a 32k-token prompt of one layer, straight from the fused projection
        {"name": "append8_prompt_32k", **append, "N": 32768, "base": 0, "block": 64},
        # a short request
        {"name": "decode8_170", **decode, "rows": 170},
        # 32 contexts of 8k to 16k tokens with seven query heads per KV head
        {"name": "decode8_batch32", **decode, "B": 32, "Hkv": 4, "G": 7, "rows": 16384, "ragged": True},
        # the compressed caches of four 32k-token prompts in integers, sizes in the logits
        {"name": "decode8_merged_4", **decode, "B": 4, "rows": 8200, "ragged": True, "merged": True, "code": "i8", "block": 32, "lse": True},
        # 32 contexts of 8k to 16k tokens behind a window of 4096
        {"name": "window_batch32", **window, "B": 32, "rows": 16384, "ragged": True},
        # a small fp32 model
        {"name": "window_1k_f32", **window, "B": 3, "Hkv": 2, "G": 1, "d": 64, "R": 16, "dtype": "f32", "q": "f32", "rows": 1000, "ragged": True, "lse": True,
         "window": 200, "sinks": 4},
        # an 8k-token prompt of one layer, every token attends to all before it
        {"name": "prompt_8k", **prompt},
        # a 16k-token prompt behind a window of 4096
        {"name": "prompt_window_16k", **prompt, "N": 16384, "window": 4096, "sinks": 16},
        # the next 300 to 600 tokens of three sequences of a small fp32 model
        {"name": "prompt_chunk_f32", **prompt, "B": 3, "Hkv": 2, "G": 3, "d": 64, "dtype": "f32", "N": 600, "context": 1111, "ragged": True, "lse": True,
         "window": 500, "sinks": 4},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["reserve", "append8", "decode8", "window", "prompt", "prompt"])
    window, sinks = rng.choice([0, _log_int(rng, 16, 8192)]), rng.choice([0, 4, 16, _log_int(rng, 1, 100)])
    if kind == "reserve":
        c = {"kind": kind, "S": _log_int(rng, 1, 512), "R": rng.choice([16, 32, 64, 128, 256]), "window": window, "sinks": sinks if window else 0, "ragged": True}
        most = (16 << 20) // c["S"]
        c["rows"] = rng.choice([0, _log_int(rng, 1, min(131072, most))])
        c["N"] = 1 if c["rows"] and rng.random() < 0.6 else _log_int(rng, 2, max(2, min(32768, most)))
        return c
    c = dict(LAYER, kind=kind)
    c["dtype"], c["d"] = rng.choice([("bf16", 128)] * 5 + [("bf16", 64), ("f32", 128), ("f32", 64)])
    c["Hkv"], c["G"] = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 7, 8, 16])
    if kind == "prompt":
        c["window"], c["sinks"] = window, sinks if window else 0
        c["lse"] = rng.random() < 0.3
        c["B"] = _log_int(rng, 1, 16)
        c["ragged"] = c["B"] > 1
        c["context"] = rng.choice([0, 0, _log_int(rng, 1, 8192)])
        # at most the products of the largest listed case, a tenth of them in 32 bits
        most = 4 * 128 * 32 * 8192 * 8192 // 2 // (1 if c["dtype"] == "bf16" else 10) // (4 * c["d"] * c["B"] * c["Hkv"] * c["G"])
        c["N"] = max(1, min(16384, int(-c["context"] + math.sqrt(c["context"] ** 2 + 2 * most))))
        c["N"] = _log_int(rng, 1, c["N"])
        return c
    c["R"] = rng.choice([16, 32, 64, 64, 128, 256])
    c["B"] = _log_int(rng, 1, 64)
    c["ragged"] = c["B"] > 1
    if kind != "window":
        c["code"], c["block"] = rng.choice(["e4m3", "e4m3", "i8"]), rng.choice([x for x in (16, 32, 64, 128) if x <= c["R"]])
    if kind == "append8":
        c["merged"] = rng.random() < 0.25
        token = c["Hkv"] * c["d"] * (2 * (ES[c["dtype"]] + 1) + (0 if c["merged"] else 2 * c["G"] * ES[c["dtype"]]))
        most = (700 << 20) // (token * c["B"])
        c["N"] = 1 if rng.random() < 0.4 else _log_int(rng, 2, max(2, min(32768, most)))
        c["base"] = rng.choice([0, _log_int(rng, 1, max(1, min(16000, most)))])
        c["rot"] = 0 if c["merged"] else rng.choice([c["d"], c["d"], c["d"] // 2, 16])
        c["interleaved"] = rng.random() < 0.3
        return c
    c["q"] = c["dtype"] if rng.random() < 0.8 else rng.choice(["bf16", "f32"])
    c["lse"] = rng.random() < 0.3
    c["merged"] = rng.random() < 0.3
    c["window"], c["sinks"] = (window, sinks if window else 0) if kind == "decode8" else (window or 1000, sinks)
    most = (1 << 30) // (2 * c["Hkv"] * c["d"] * (1 if kind == "decode8" else ES[c["dtype"]]) * c["B"])
    c["rows"] = _log_int(rng, 1, max(1, min(131072, most)))
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _lens(shape, most, ragged, gen):
    """int32 on the GPU: `most`, or between half of it and all of it."""
    if not ragged or most < 2:
        return torch.full(shape, most, dtype=torch.int32, device="cuda")
    return torch.randint(most // 2, most + 1, shape, generator=gen, device="cuda", dtype=torch.int32)


def _randn(shape, dtype, gen):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)


def _codes(c, shape, gen):
    """Codes of a pool as appending leaves them: the largest of a block uses the upper half of the range."""
    x = _randn(shape, torch.float32, gen).mul_(LARGEST[c["code"]] / 5).clamp_(-LARGEST[c["code"]], LARGEST[c["code"]])
    return (x.round_() if c["code"] == "i8" else x).to(CODES[c["code"]])


def _pages(c, rows, gen):
    """Pools and table for `rows` rows of every sequence, pages in no order."""
    B, H, R, d = c["B"], c["Hkv"], c["R"], c["d"]
    P = -(-rows // R)
    tables = B * H if c["merged"] else B
    heads = 1 if c["merged"] else H
    n = tables * P + 3
    s = {}
    if c["kind"] == "window":
        s["K"], s["V"] = (_randn((n, heads, R, d), DTYPES[c["dtype"]], gen) for _ in range(2))
    else:
        s["K"], s["V"] = (_codes(c, (n, heads, R, d), gen) for _ in range(2))
        unit = 2.0 ** round(math.log2(5 / LARGEST[c["code"]]))      # numbers of about 1, with blocks of twice as large ones
        s["ks"], s["vs"] = ((torch.randint(0, 2, (n, heads, R // c["block"]), generator=gen, device="cuda") + 1).float() * unit for _ in range(2))
    order = torch.randperm(n, generator=gen, device="cuda")[: tables * P].to(torch.int32)
    s["table"] = order.reshape((B, H, P) if c["merged"] else (B, P))
    # sizes as the compression leaves them: a third of the rows are clusters of one
    size = torch.rand((n, heads, R), generator=gen, device="cuda")
    s["counts"] = torch.where(size < 0.36, 1, 2 + (-8.0 * torch.log1p(-(size - 0.36) / 0.6401)).to(torch.int32)).to(torch.int32) if c["merged"] else None
    return s


def _angles(rot):
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    a = torch.arange(MAX_POSITION, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-2.0 * i / rot)
    return torch.cat((a.cos(), a.sin()), 1).to(torch.float32)


def _kept(c, p, base, total):
    """Which places p of a table hold rows below `total` that a token from `base` on can see."""
    R = c["R"]
    seen = (p * R < total) & ((p * R < c["sinks"]) | ((p + 1) * R > base + 1 - c["window"]) if c["window"] else True)
    return seen


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator("cuda").manual_seed(seed)
    if c["kind"] == "reserve":
        S, R = c["S"], c["R"]
        P = -(-(c["rows"] + c["N"]) // R)
        pages = S * P
        s = {"c": c, "base": _lens((S,), c["rows"], c["ragged"], gen), "new": _lens((S,), c["N"], c["ragged"], gen)}
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        held = _kept(c, torch.arange(P, device="cuda"), s["base"][:, None], s["base"][:, None])
        s["table"] = torch.where(held, order.reshape(S, P), -1).contiguous()
        free = order.reshape(S, P)[~held]
        s["free"] = torch.zeros(pages, dtype=torch.int32, device="cuda")
        s["free"][: free.numel()] = free
        s["many"] = torch.full((1,), free.numel(), dtype=torch.int32, device="cuda")
        return s
    B, H, G, d, dt = c["B"], c["Hkv"], c["G"], c["d"], DTYPES[c["dtype"]]
    if c["kind"] == "prompt":
        N, M = c["N"], c["N"] + c["context"]
        # keys and values of context and chunk, with the queries of the chunk, as a fused projection leaves them
        qkv = _randn((B, M, (G + 2) * H, d), dt, gen).permute(0, 2, 1, 3)
        s = {"q": qkv[:, : G * H, M - N :], "k": qkv[:, G * H : (G + 1) * H], "v": qkv[:, (G + 1) * H :]}
        s["new"] = _lens((B,), N, c["ragged"], gen)
        s["lens"] = s["new"] + _lens((B,), c["context"], c["ragged"], gen)
        s["c"] = c
        return s
    per_head = (B, H) if c["merged"] else (B,)
    if c["kind"] == "append8":
        N = c["N"]
        s = _pages(c, c["base"] + N, gen)
        s["base"] = _lens(per_head, c["base"], c["ragged"], gen)
        s["new"] = _lens(per_head, N, c["ragged"], gen)
        if c["merged"]:
            s["k"], s["v"] = _randn((B, H, N, d), dt, gen), _randn((B, H, N, d), dt, gen)
            s["sizes"] = torch.randint(1, 40, (B, H, N), generator=gen, device="cuda", dtype=torch.int32)
        else:
            qkv = _randn((B, N, (G + 2) * H, d), dt, gen).permute(0, 2, 1, 3)
            s["q"], s["k"], s["v"] = qkv[:, : G * H], qkv[:, G * H : (G + 1) * H], qkv[:, (G + 1) * H :]
            s["cos_sin"] = _angles(c["rot"])
            s["positions"] = (s["base"] * 3).clamp(max=MAX_POSITION - N)      # what the cache holds may stand for more tokens than it has rows
        s["lens"] = torch.zeros_like(s["base"])
    else:
        s = _pages(c, c["rows"], gen)
        s["lens"] = _lens(per_head, c["rows"], c["ragged"], gen)
        s["q"] = _randn((B, H * G, d), DTYPES[c["q"]], gen).mul_(1.5)
    s["c"] = c
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _reserve(s, new):
    """One call: (lens, slots); table, free and many are changed."""
    c = s["c"]
    R, N = c["R"], c["N"]
    table, free, many = s["table"], s["free"], s["many"]
    base, total = s["base"].long()[:, None], (s["base"] + new).long()[:, None]
    p = torch.arange(table.shape[1], device="cuda")
    held, want = table >= 0, _kept(c, p, base, total)
    fine = ~(want & ~held & (p * R < base)).any(1, keepdim=True)
    back, take = held & ~want & fine, want & ~held & fine
    available = back.sum() + many.long()[0]
    through = take.sum(1).cumsum(0)[:, None]
    take &= through <= available
    fine &= (through <= available) | ~take.any(1, keepdim=True)
    # the k-th page taken is the k-th given back, then the top of the stack
    given, taken, taken_all = back.flatten().long().cumsum(0) - 1, take.flatten().long().cumsum(0) - 1, take.sum()
    returned = torch.zeros_like(free).scatter_(0, torch.where(back.flatten(), given, free.numel() - 1), torch.where(back.flatten(), table.flatten(), 0))
    returned = torch.where(torch.arange(free.numel(), device="cuda") < back.sum(), returned, 0)
    last = back.flatten().nonzero()
    if last.numel():
        returned[given[last[-1]]] = table.flatten()[last[-1]]
    k = taken.reshape(table.shape)
    fresh = torch.where(k < back.sum(), returned[k.clamp(0, free.numel() - 1)], free[(many.long()[0] - 1 - (k - back.sum())).clamp(0, free.numel() - 1)])
    left = given[back.flatten()][taken_all.clamp(max=back.sum()):] if last.numel() else given[:0]
    free[many.long()[0] + back.sum() - 1 - left] = returned[left]
    table.copy_(torch.where(take, fresh, torch.where(back, -1, table)))
    many.add_((back.sum() - taken_all).to(torch.int32))
    n = torch.arange(N, device="cuda")
    row = (base + n).clamp(max=table.shape[1] * R - 1)
    slots = torch.where((n < new.long()[:, None]) & fine, table.gather(1, row // R) * R + row % R, -1).to(torch.int32)
    return torch.where(fine, total, -1)[:, 0].to(torch.int32), slots


def _rotated(x, cos_sin, positions, rot, interleaved):
    """x [B, heads, N, d] in fp32 with its first `rot` elements turned by the angles of the rows' positions."""
    N = x.shape[2]
    p = positions[:, None].to(torch.int64) + torch.arange(N, device="cuda")
    cos, sin = cos_sin[p][:, None].split(rot // 2, -1)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., : rot // 2], x[..., rot // 2 : rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _places(c, table):
    """Page numbers [B, Hkv, P] and the head's place in its page, for indexing a pool."""
    H = c["Hkv"]
    at = (table if table.dim() == 3 else table[:, None, :].expand(-1, H, -1)).to(torch.int64)
    heads = torch.zeros((1, H, 1), dtype=torch.int64, device="cuda") if table.dim() == 3 else torch.arange(H, device="cuda")[None, :, None]
    return at, heads


def _smallest_scale(c, largest):
    """The smallest power of two that `largest` divided by it does not leave the codes' range, at least 2^-126."""
    m, e = torch.frexp(largest)      # m in [1/2, 1)
    top = 9 if c["code"] == "e4m3" else 7
    e = torch.where(largest > 0, e - top + (m > LARGEST[c["code"]] / 2.0**top), -126).clamp(min=-126)
    return torch.ldexp(torch.ones_like(largest), e)


def _encoded(c, x):
    return (x.round() if c["code"] == "i8" else x).to(CODES[c["code"]])


def _bytes(x):
    return x.view(torch.uint8)


def _append8(s):
    c = s["c"]
    H, R, N, E = c["Hkv"], c["R"], c["N"], c["block"]
    k, v, q = s["k"].float(), s["v"].float(), s.get("q")
    if c["rot"]:
        k = _rotated(k, s["cos_sin"], s["positions"], c["rot"], c["interleaved"])
        q = _rotated(q.float(), s["cos_sin"], s["positions"], c["rot"], c["interleaved"]).to(q.dtype)
    base, new = (x if x.dim() == 2 else x[:, None].expand(-1, H) for x in (s["base"].to(torch.int64), s["new"].to(torch.int64)))
    at, heads = _places(c, s["table"])
    # the blocks that the new rows touch, from the one that holds row `base` on
    first = base // E
    blocks = min((N + E - 2) // E + 1, at.shape[2] * R // E)
    block = first[..., None] + torch.arange(blocks, device="cuda")
    page = at.gather(2, (block * E // R).clamp(max=at.shape[2] - 1))
    spot = (page, heads, block % (R // E))
    t = block[..., None] * E + torch.arange(E, device="cuda")      # [B, H, blocks, E]
    held, fresh = t < base[..., None, None], (t >= base[..., None, None]) & (t < (base + new)[..., None, None])
    source = (t - base[..., None, None]).clamp(0, N - 1).flatten(2)
    row = (page[..., None], heads[..., None], t % R)
    touched = fresh.any(3)
    for pool, scales, x in ((s["K"], s["ks"], k), (s["V"], s["vs"], v)):
        x = x.gather(2, source[..., None].expand(-1, -1, -1, x.shape[3])).unflatten(2, (blocks, E))
        before = scales[spot]
        need = _smallest_scale(c, torch.where(fresh[..., None], x.abs(), 0).amax((3, 4)))
        scale = torch.where(held.any(3), torch.maximum(before, need), need)
        old = _bytes(pool)[row]
        again = _encoded(c, old.view(CODES[c["code"]]).float() * torch.where(held.any(3), before / scale, 1)[..., None, None])
        codes = _encoded(c, torch.where(fresh[..., None], x * (1 / scale)[..., None, None], 0))
        codes = torch.where(fresh[..., None], _bytes(codes), torch.where(held[..., None] & touched[..., None, None], _bytes(again), old))
        inside = (t < at.shape[2] * R).expand(-1, -1, -1, -1)
        where = tuple(i.expand(t.shape)[inside] for i in row)
        _bytes(pool).index_put_(where, codes[inside])
        whole = (block * E < at.shape[2] * R)
        scales.index_put_(tuple(i.expand(block.shape)[whole] for i in spot), torch.where(touched, scale, before)[whole])
    if s["counts"] is not None:
        n = torch.arange(N, device="cuda")
        place = ((at.gather(2, ((base[..., None] + n) // R).clamp(max=at.shape[2] - 1))), heads, (base[..., None] + n) % R)
        s["counts"].index_put_(place, torch.where(n < new[..., None], s["sizes"], s["counts"][place]))
    s["lens"].copy_(s["base"] + s["new"])
    return _appended(s, q)


def _appended(s, q):
    return {"K": s["K"], "V": s["V"], "ks": s["ks"], "vs": s["vs"], "counts": s["counts"], "lens": s["lens"], "q": q}


def _visible(c, row, n):
    return (row < n) & ((row >= n - c["window"]) | (row < c["sinks"]) if c["window"] else True)


def _attend(s):
    c = s["c"]
    B, H, G, d, R = c["B"], c["Hkv"], c["G"], c["d"], c["R"]
    at, heads = _places(c, s["table"])
    lens = s["lens"] if s["lens"].dim() == 2 else s["lens"][:, None].expand(-1, H)
    seen = _visible(c, torch.arange(at.shape[2] * R, device="cuda"), lens[..., None])
    if c["kind"] == "window":
        k, v = (s[x][at, heads].flatten(2, 3).float() for x in ("K", "V"))
    else:
        k, v = ((_bytes(s[x])[at, heads].view(CODES[c["code"]]).float().unflatten(3, (-1, c["block"])) * s[y][at, heads][..., None, None]).flatten(2, 4)
                for x, y in (("K", "ks"), ("V", "vs")))
    z = (s["q"].float().reshape(B, H, G, d) @ k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    if s["counts"] is not None:
        z = z + s["counts"][at, heads].flatten(2).float().log()[:, :, None]
    z = torch.where(seen[:, :, None], z, -math.inf)
    m = z.amax(3, keepdim=True)
    w = (z - m).exp()
    total = w.sum(3, keepdim=True)
    o = (w @ torch.where(seen[..., None], v, 0)) / total
    return {"O": o.reshape(B, H * G, d).to(s["q"].dtype), "lse": (m + total.log()).reshape(B, H * G) if c["lse"] else None}


def _prompt(s):
    c = s["c"]
    B, H, G, d, N = c["B"], c["Hkv"], c["G"], c["d"], c["N"]
    i, j = torch.arange(N, device="cuda"), torch.arange(s["k"].shape[2], device="cuda")
    real = i < s["new"][:, None]
    here = (s["lens"] - s["new"])[:, None] + i
    seen = _visible(c, j, here[..., None] + 1)[:, None, None]
    O, lse = [], []
    for h in range(H):      # the logits of all heads at once would not fit
        q, k, v = s["q"][:, h * G : (h + 1) * G].float(), s["k"][:, h : h + 1].float(), s["v"][:, h : h + 1].float()
        z = torch.where(seen[:, 0], (q @ k.transpose(2, 3)) * (1.0 / math.sqrt(d)), -math.inf)
        m = z.amax(3, keepdim=True)
        w = (z - m).exp_()
        total = w.sum(3, keepdim=True)
        O.append(((w @ v) / total).to(s["q"].dtype))
        lse.append((m + total.log())[..., 0])
    O, lse = torch.cat(O, 1), torch.cat(lse, 1)
    return {"O": torch.where(real[:, None, :, None], O, 0), "lse": torch.where(real[:, None], lse, 0) if c["lse"] else None}


# ------------------------------------------------------------------------------------------------ the framework's operators
def _own(s):
    """What a program makes once, when it sets its cache up: the description of the cache, a workspace, outputs to fill."""
    if "own" not in s:
        from paper_2603_14303_amd import binding as sc
        c = s["c"]
        o = {"sc": sc}
        if c["kind"] == "reserve":
            o["ws"] = sc.paged_reserve_workspace(c["S"], s["table"].shape[1], "cuda")
            o["lens"], o["back"] = torch.empty_like(s["base"]), torch.empty_like(s["base"])
            o["none"] = torch.zeros_like(s["base"])
            o["slots"] = torch.empty((c["S"], c["N"]), dtype=torch.int32, device="cuda")
        elif c["kind"] == "prompt":
            o["O"] = torch.zeros((c["B"], c["N"], c["Hkv"] * c["G"], c["d"]), dtype=s["q"].dtype, device="cuda").permute(0, 2, 1, 3)
            o["lse"] = torch.zeros((c["B"], c["Hkv"] * c["G"], c["N"]), dtype=torch.float32, device="cuda") if c["lse"] else None
            o["ws"] = sc.prompt_attn_workspace(c["B"], c["Hkv"] * c["G"], c["Hkv"], c["N"], c["N"] + c["context"], c["d"], "cuda")
        else:
            if c["kind"] == "window":
                o["cache"] = sc.PagedCache(s["K"], s["V"], s["table"], counts=s["counts"])
            else:
                o["cache"] = sc.PagedCache8(s["K"], s["V"], s["ks"], s["vs"], s["table"], counts=s["counts"])
            if c["kind"] == "append8":
                o["q"] = None if s.get("q") is None else torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
            else:
                o["ws"] = sc.paged_workspace(c["B"], c["Hkv"] * c["G"], c["Hkv"], c["d"], s["table"].shape[-1], "cuda")
                o["O"] = torch.empty_like(s["q"])
                o["lse"] = torch.empty((c["B"], c["Hkv"] * c["G"]), dtype=torch.float32, device="cuda") if c["lse"] else None
        s["own"] = o
    return s["own"]


def run(s):
    c = s["c"]
    if own:
        o = _own(s)
        sc = o["sc"]
        if c["kind"] == "reserve":
            sc.sc_paged_reserve(s["table"], c["R"], s["base"], o["lens"], s["free"], s["many"], new_lens=s["new"], window=c["window"], sinks=c["sinks"],
                                slots=o["slots"], workspace=o["ws"])
            sc.sc_paged_reserve(s["table"], c["R"], s["base"], o["back"], s["free"], s["many"], new_lens=o["none"], window=c["window"], sinks=c["sinks"],
                                workspace=o["ws"])
            return {"lens": o["lens"], "slots": o["slots"], "back": o["back"], "table": s["table"], "free": s["free"], "many": s["many"]}
        if c["kind"] == "append8":
            sc.sc_paged8_append(o["cache"], s["k"], s["v"], s["base"], s["lens"], new_lens=s["new"], counts=s.get("sizes"), Q=s.get("q"), Q_out=o["q"],
                                cos_sin=s.get("cos_sin"), positions=s.get("positions"), interleaved=c["interleaved"])
            return _appended(s, o["q"])
        if c["kind"] == "decode8":
            sc.sc_paged8_decode_attn(o["cache"], s["q"], s["lens"], window=c["window"], sinks=c["sinks"], O=o["O"], lse=o["lse"], workspace=o["ws"])
        elif c["kind"] == "window":
            sc.sc_paged_window_attn(o["cache"], s["q"], s["lens"], c["window"], sinks=c["sinks"], O=o["O"], lse=o["lse"], workspace=o["ws"])
        else:
            sc.sc_prompt_attn(s["q"], s["k"], s["v"], q_lens=s["new"], kv_lens=s["lens"], window=c["window"], sinks=c["sinks"], O=o["O"], lse=o["lse"],
                              workspace=o["ws"])
        return {"O": o["O"], "lse": o["lse"]}
    if c["kind"] == "reserve":
        lens, slots = _reserve(s, s["new"])
        back, _ = _reserve(s, torch.zeros_like(s["new"]))
        return {"lens": lens, "slots": slots, "back": back, "table": s["table"], "free": s["free"], "many": s["many"]}
    return _append8(s) if c["kind"] == "append8" else _prompt(s) if c["kind"] == "prompt" else _attend(s)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _pairs(N, context, window, sinks):
    """Visible (query, key) pairs of N queries behind `context` keys, about."""
    total = N * context + N * (N + 1) / 2
    if window:
        see = window + sinks
        a = min(max(see - context, 0), N)      # queries that see everything before them
        total = a * context + a * (a + 1) / 2 + (N - a) * see
    return total


def work(case):
    c = case
    share = 0.75 if c["ragged"] else 1.0      # lengths between half and all
    if c["kind"] == "reserve":
        S = c["S"]
        P = -(-(c["rows"] + c["N"]) // c["R"])
        taken = max(S * c["N"] * share, 1) / c["R"]
        return {"bytes": 2 * 4.0 * S * P + 4.0 * S * c["N"] + 4 * 4 * taken + 4 * 6.0 * S, "flops": 0.0}
    B, H, G, d, e = c["B"], c["Hkv"], c["G"], c["d"], ES[c["dtype"]]
    if c["kind"] == "prompt":
        N, M = max(1.0, c["N"] * share), max(1.0, (c["N"] + c["context"]) * share)
        return {"bytes": B * H * d * e * (2 * N * G + 2 * M) + (4 * B * H * G * N if c["lse"] else 0), "flops": 4.0 * d * B * H * G * _pairs(N, M - N, c["window"], c["sinks"])}
    if c["kind"] == "append8":
        n = max(1.0, B * c["N"] * share)
        rows = n * H
        bytes_ = rows * 2 * d * (e + 1) + 8 * max(rows / c["block"], B * H) + (rows * 8 if c["merged"] else 0)
        return {"bytes": bytes_ + (0 if c["merged"] else 2 * B * c["N"] * H * G * d * e + n * c["rot"] * 4), "flops": 3.0 * c["rot"] * (n * H + B * c["N"] * H * G) + 6.0 * rows * d}
    rows = max(1.0, c["rows"] * share)
    if c["window"]:
        rows = min(rows, c["window"] + c["sinks"])
    rows = B * H * rows
    row = 2 * d * e if c["kind"] == "window" else 2 * d + 8 / c["block"]
    io = B * H * G * (d * 2 * ES[c["q"]] + (4 if c["lse"] else 0))
    return {"bytes": rows * (row + (4 if c["merged"] else 0)) + io, "flops": 4.0 * d * G * rows}


# ------------------------------------------------------------------------------------------------ in 64 bits, one sequence and head at a time
def _nearest(code, x):
    """x rounded to the nearest number of the code's type, ties to even."""
    if code == "i8":
        return torch.round(x)
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0**-20))).clamp(min=-6)
    e = e + (x.abs() >= 2.0 ** (e + 1)).double() - (x.abs() < 2.0**e).double() * (e > -6)
    step = 2.0 ** (e - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "reserve":
        return None
    H, G = c["Hkv"], c["G"]
    length = lambda x, b, h: int(x[b, h] if x.dim() == 2 else x[b])  # noqa: E731
    if c["kind"] == "prompt":
        O = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device="cuda")
        for b in range(c["B"]):
            n, m = int(s["new"][b]), int(s["lens"][b])
            for h in range(H * G):
                q, k, v = s["q"][b, h, :n].double(), s["k"][b, h // G, :m].double(), s["v"][b, h // G, :m].double()
                for i0 in range(0, n, 4096):      # 4096 queries at a time
                    z = q[i0 : i0 + 4096] @ k.T / math.sqrt(c["d"])
                    behind = torch.arange(m - n + i0, m - n + i0 + z.shape[0], device="cuda")[:, None] - torch.arange(m, device="cuda")[None]
                    hidden = behind < 0
                    if c["window"]:
                        hidden |= (behind >= c["window"]) & (torch.arange(m, device="cuda") >= c["sinks"])
                    z = z.masked_fill(hidden, -math.inf)
                    O[b, h, i0 : i0 + z.shape[0]] = torch.softmax(z, 1) @ v
                    lse[b, h, i0 : i0 + z.shape[0]] = torch.logsumexp(z, 1)
        return {"O": O, "lse": lse if c["lse"] else None}
    R = c["R"]
    table = s["table"].tolist()

    def rows_of(b, h, n):
        """Page and row in its page of the first n rows of a sequence's head."""
        t = torch.arange(n, device="cuda")
        pages = torch.tensor(table[b][h] if c["merged"] else table[b], device="cuda")
        return pages[t // R], t % R

    if c["kind"] == "append8":
        def turned(x, b):
            x = x.double().clone()
            if not c["rot"]:
                return x
            half = c["rot"] // 2
            t = s["cos_sin"].double()[int(s["positions"][b]) : int(s["positions"][b]) + x.shape[-2]]
            z = torch.complex(t[:, :half], t[:, half:])
            i = slice(0, c["rot"], 2) if c["interleaved"] else slice(0, half)
            j = slice(1, c["rot"], 2) if c["interleaved"] else slice(half, c["rot"])
            z = torch.complex(x[..., i], x[..., j]) * z
            x[..., i], x[..., j] = z.real, z.imag
            return x

        E = c["block"]
        out = {x: s[x].double() for x in ("K", "V", "ks", "vs")}
        for b in range(c["B"]):
            for h in range(H):
                base, new = length(s["base"], b, h), length(s["new"], b, h)
                if new == 0:
                    continue
                head, first = 0 if c["merged"] else h, base // E * E
                page, row = (x[first:] for x in rows_of(b, h, base + new))
                group = torch.arange(base + new - first, device="cuda") // E
                for pool, scales, x in (("K", "ks", turned(s["k"][b, h], b)), ("V", "vs", s["v"][b, h].double())):
                    x = x[:new]
                    largest = torch.zeros(int(group[-1]) + 1, dtype=torch.float64, device="cuda").scatter_reduce(0, group[base - first :], x.abs().amax(1), "amax")
                    scale = 2.0 ** torch.ceil(torch.log2(largest.clamp(min=2.0**-130) / LARGEST[c["code"]]))
                    at = (page[::E], head, row[::E] // E)
                    if base > first:
                        before = out[scales][at][0].clone()
                        scale[0] = torch.maximum(scale[0], before)
                        old = (page[: base - first], head, row[: base - first])
                        out[pool][old] = _nearest(c["code"], out[pool][old] * before / scale[0])
                    out[scales][at] = scale
                    out[pool][page[base - first :], head, row[base - first :]] = _nearest(c["code"], x / scale[group[base - first :]][:, None])
        q = None if s.get("q") is None else torch.stack([turned(s["q"][b], b) for b in range(c["B"])])
        whole = c["code"] == "i8"      # its pools are compared as the whole numbers that they are
        return {"K": None if whole else out["K"], "V": None if whole else out["V"], "ks": out["ks"], "vs": out["vs"], "counts": None, "lens": None, "q": q}

    O = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        for h in range(H):
            n = length(s["lens"], b, h)
            mine = torch.arange(n, device="cuda")
            if c["window"]:
                mine = mine[(mine < c["sinks"]) | (n - mine <= c["window"])]
            page, row = (x[mine] for x in rows_of(b, h, n))
            head = 0 if c["merged"] else h
            k, v = s["K"][page, head, row].double(), s["V"][page, head, row].double()
            if c["kind"] == "decode8":
                k, v = k * s["ks"][page, head, row // c["block"]].double()[:, None], v * s["vs"][page, head, row // c["block"]].double()[:, None]
            z = k @ s["q"][b, h * G : (h + 1) * G].double().T / math.sqrt(c["d"])
            if c["merged"]:
                z = z + s["counts"][page, head, row].double().log()[:, None]
            O[b, h * G : (h + 1) * G] = torch.softmax(z, 0).T @ v
            lse[b, h * G : (h + 1) * G] = torch.logsumexp(z, 0)
    return {"O": O, "lse": lse if c["lse"] else None}
