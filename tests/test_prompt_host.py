"""Calls around prompts and pages that are handed out, without a GPU: refusals, workspaces, and the index arithmetic of csrc/sc_prompt.h and of the windows in
csrc/sc_paged_words.h against brute force."""
import ctypes
import os
import subprocess

import pytest

from paper_2603_14303_amd import binding as sc
from test_paged_host import ARG, FAKE, ROWS, UNSUPPORTED, WORKSPACE, lib  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CACHE8 = dict(K=FAKE, V=FAKE, k_scale=FAKE, v_scale=FAKE + (1 << 20), counts=None, table=FAKE, stride_page=4 * 32 * 128, stride_head=32 * 128, stride_row=128, code=0,
              block_rows=16, num_pages=100, page_heads=4, page_rows=32, table_len=20, table_per_head=0, B=2, Hkv=4, d=128)
BAD8 = [
    (dict(K=None), ARG), (dict(V=None), ARG), (dict(table=None), ARG), (dict(k_scale=None), ARG), (dict(v_scale=None), ARG), (dict(k_scale=FAKE + 2), ARG), (dict(K=FAKE + 8), ARG),
    (dict(B=0), ARG), (dict(Hkv=0), ARG), (dict(num_pages=0), ARG), (dict(table_len=0), ARG), (dict(page_rows=8), ARG), (dict(page_rows=48), ARG), (dict(page_rows=2048), ARG),
    (dict(page_heads=2), ARG), (dict(table_per_head=1), ARG), (dict(stride_row=64), ARG), (dict(stride_row=136), ARG), (dict(stride_head=128), ARG), (dict(stride_head=32 * 128 - 16), ARG),
    (dict(stride_page=3 * 32 * 128), ARG), (dict(block_rows=8), ARG), (dict(block_rows=24), ARG), (dict(block_rows=64), ARG), (dict(block_rows=0), ARG), (dict(block_rows=256, page_rows=256), ARG),
    (dict(v_scale=FAKE), ARG), (dict(v_scale=FAKE + 3196), ARG), (dict(code=2), UNSUPPORTED), (dict(code=-1), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(B=70000), UNSUPPORTED), (dict(table_len=2**27), UNSUPPORTED),
]


def test_append_to_codes_rejects_bad_arguments(lib):  # noqa: F811
    def call(cache=None, dtype=1, **kw):
        return lib.sc_paged8_append(ctypes.byref(sc._Paged8CacheStruct(**dict(CACHE8, **(cache or {})))), ctypes.byref(sc._PagedRowsStruct(**dict(ROWS, **kw))), dtype, None)
    for bad, want in BAD8:
        assert call(bad) == want, bad
    assert lib.sc_paged8_append(None, ctypes.byref(sc._PagedRowsStruct(**ROWS)), 1, None) == ARG
    assert lib.sc_paged8_append(ctypes.byref(sc._Paged8CacheStruct(**CACHE8)), None, 1, None) == ARG
    assert call(dtype=2) == UNSUPPORTED and call(dtype=-1) == UNSUPPORTED
    for name in ("K", "V", "base_lens", "lens", "Q", "Q_out"):
        assert call(**{name: None}) == ARG, name
    for name in ("K", "V", "Q", "Q_out", "cos_sin"):
        assert call(**{name: FAKE + 8}) == ARG, name
    assert call(N=0) == ARG and call(lens=FAKE) == ARG and call(new_lens=FAKE + 256) == ARG and call(rot=20) == ARG and call(rot=256) == ARG
    assert call(counts=FAKE) == ARG and call(dict(counts=FAKE)) == ARG
    assert call(k_stride_n=132) == ARG                      # (bf16 rows, whatever the codes)
    assert call(N=2**31 - 1) == UNSUPPORTED


def test_windowed_attention_rejects_bad_arguments(lib):  # noqa: F811
    from test_paged_host import BAD_CACHES, CACHE

    def attend(codes, cache=None, Q=FAKE, dtype=1, Hq=8, lens=FAKE, window=10, sinks=2, scale=0.0, O=FAKE, odt=1, lse=None, ws=FAKE, nbytes=1 << 30):
        if codes:
            c, f = sc._Paged8CacheStruct(**dict(CACHE8, **(cache or {}))), lib.sc_paged8_decode_attn
        else:
            c, f = sc._PagedCacheStruct(**dict(CACHE, **(cache or {}))), lib.sc_paged_window_attn
        return f(ctypes.byref(c), Q, dtype, Hq, lens, 0, window, sinks, scale, O, odt, lse, ws, nbytes, None)
    for bad, want in BAD8:
        assert attend(True, bad) == want, bad
    for bad, want in BAD_CACHES:
        assert attend(False, bad) == want, bad
    for codes in (True, False):
        for name in ("Q", "lens", "O"):
            assert attend(codes, **{name: None}) == ARG, name
        assert attend(codes, Q=FAKE + 8) == ARG and attend(codes, O=FAKE + 8) == ARG and attend(codes, lens=FAKE + 1) == ARG and attend(codes, lse=FAKE + 2) == ARG
        assert attend(codes, window=-1) == ARG and attend(codes, sinks=-1) == ARG and attend(codes, scale=float("nan")) == ARG
        assert attend(codes, Hq=9) == UNSUPPORTED and attend(codes, Hq=68) == UNSUPPORTED and attend(codes, dtype=3) == UNSUPPORTED and attend(codes, odt=3) == UNSUPPORTED
        assert attend(codes, ws=None) == WORKSPACE and attend(codes, ws=FAKE + 8) == WORKSPACE and attend(codes, nbytes=4096) == WORKSPACE
    assert lib.sc_paged8_decode_attn(None, FAKE, 1, 8, FAKE, 0, 0, 0, 0.0, FAKE, 1, None, FAKE, 1 << 30, None) == ARG


def test_reserve_rejects_bad_arguments(lib):  # noqa: F811
    good = dict(table=FAKE, sequences=10, table_len=20, num_pages=100, page_rows=32, base=FAKE + 4096, new=FAKE + 8192, N=5, window=0, sinks=0, free=FAKE + 12288, many=FAKE + 16384,
                lens=FAKE + 20480, slots=FAKE + 24576, ws=FAKE + 65536, nbytes=1 << 30)

    def call(**kw):
        return lib.sc_paged_reserve(*dict(good, **kw).values(), None)
    for name in ("table", "base", "free", "many", "lens"):
        assert call(**{name: None}) == ARG, name
    for name in ("table", "base", "new", "free", "many", "lens", "slots"):
        assert call(**{name: FAKE + 2}) == ARG, name
    for name in ("sequences", "table_len", "num_pages"):
        assert call(**{name: 0}) == ARG and call(**{name: -1}) == ARG, name
    for name in ("N", "window", "sinks"):
        assert call(**{name: -1}) == ARG, name
    assert call(page_rows=8) == ARG and call(page_rows=48) == ARG and call(page_rows=2048) == ARG
    assert call(lens=FAKE + 4096) == ARG and call(lens=FAKE + 8192) == ARG and call(lens=FAKE + 4096 + 36) == ARG
    for a, b in (("many", "free"), ("many", "table"), ("free", "table"), ("lens", "many"), ("slots", "lens"), ("slots", "free"), ("base", "table"), ("new", "slots"), ("base", "many")):
        assert call(**{a: good[b]}) == ARG, (a, b)
    assert call(sequences=(1 << 20) + 1) == UNSUPPORTED and call(sequences=1 << 20, table_len=1 << 9) == UNSUPPORTED
    assert call(table_len=1 << 26) == UNSUPPORTED and call(num_pages=1 << 26) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 8) == WORKSPACE and call(nbytes=1000) == WORKSPACE
    f = lib.sc_paged_reserve_workspace_bytes
    assert f(0, 5) == 0 and f(5, 0) == 0 and f(-1, 5) == 0 and f((1 << 20) + 1, 1) == 0 and f(1 << 20, 1 << 9) == 0
    assert f(10, 20) % 256 == 0 and f(512, 2048) >= 512 * 2048 * 4


PROMPT = dict(Q=FAKE, K=FAKE, V=FAKE, O=FAKE + (1 << 40), lse=None, q_lens=None, kv_lens=None, dtype=1, B=2, Hq=8, Hkv=2, N=10, M=30, d=128, window=0, sinks=0, scale=0.0,
              **{x + "_stride_" + y: s for x, n, h in (("q", 10, 8), ("k", 30, 2), ("v", 30, 2), ("o", 10, 8)) for y, s in (("b", h * n * 128), ("h", n * 128), ("n", 128))})


def test_prompt_rejects_bad_arguments(lib):  # noqa: F811
    def call(ws=FAKE, nbytes=1 << 30, **kw):
        return lib.sc_prompt_attn(ctypes.byref(sc._PromptStruct(**dict(PROMPT, **kw))), ws, nbytes, None)
    assert lib.sc_prompt_attn(None, FAKE, 1 << 30, None) == ARG
    for name in ("Q", "K", "V", "O"):
        assert call(**{name: None}) == ARG and call(**{name: FAKE + 8}) == ARG, name
    for name in ("q_lens", "kv_lens", "lse"):
        assert call(**{name: FAKE + 2}) == ARG, name
    for name in ("B", "Hq", "Hkv", "N", "M"):
        assert call(**{name: 0}) == ARG and call(**{name: -1}) == ARG, name
    assert call(window=-1) == ARG and call(sinks=-1) == ARG and call(scale=float("nan")) == ARG
    for x in "qkvo":
        for y in "bhn":
            assert call(**{x + "_stride_" + y: -128}) == ARG and call(**{x + "_stride_" + y: 132}) == ARG, (x, y)
    assert call(o_stride_n=64) == ARG and call(o_stride_h=0) == ARG and call(o_stride_h=128) == ARG      # rows of the output that meet
    assert call(d=96) == UNSUPPORTED and call(dtype=2) == UNSUPPORTED and call(Hq=9) == UNSUPPORTED and call(B=70000) == UNSUPPORTED and call(Hq=70000, Hkv=1) == UNSUPPORTED
    assert call(N=1 << 29) == UNSUPPORTED and call(M=(1 << 30) + 1) == UNSUPPORTED and call(k_stride_n=1 << 24) == UNSUPPORTED and call(v_stride_n=1 << 24) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 8) == WORKSPACE and call(nbytes=256) == WORKSPACE
    f = lib.sc_prompt_attn_workspace_bytes
    assert f(0, 8, 2, 10, 30, 128) == 0 and f(2, 9, 2, 10, 30, 128) == 0 and f(2, 8, 2, 10, 30, 96) == 0 and f(2, 8, 2, 0, 30, 128) == 0 and f(2, 8, 2, 10, 0, 128) == 0
    # a workspace for more queries, keys or sequences is large enough for fewer
    most = f(16, 64, 8, 4096, 65536, 128)
    for B in (1, 3, 16):
        for N in (1, 7, 64, 300, 4096):
            for M in (1, 64, 5000, 65536):
                assert 0 < f(B, 64, 8, N, M, 128) <= most and f(B, 64, 8, N, M, 64) <= f(B, 64, 8, N, M, 128)


WORDS = r"""
#include <stdio.h>
#include <stdlib.h>
#include <algorithm>
#include <vector>
#include "sc_paged_words.h"
#include "sc_prompt.h"
using namespace sc;
static long long checks = 0, wrong = 0;
#define CHECK(x) do { ++checks; if (!(x)) { ++wrong; printf("line %d: %s\n", __LINE__, #x); if (wrong > 20) exit(1); } } while (0)
static int any(int lo, int hi) { return lo + (int)((unsigned)rand() % (unsigned)(hi - lo + 1)); }
static int some(int most) { return any(0, 3) ? any(0, most) : any(0, 1) ? 0 : 2147483647; }

int main() {
    // ---- windows over pages: every visible row is visited once, rows of a step lie in one page, a step without visible rows looks nothing up
    for (int t = 0; t < 60000; ++t) {
        const int len = any(0, 400), window = some(450), sinks = some(450);
        const PagedGap gap = paged_gap(len, window, sinks);
        CHECK(gap.at >= 0 && gap.rows >= 0 && gap.at % 16 == 0 && gap.rows % 16 == 0 && gap.at + gap.rows <= len);
        std::vector<int> seen(len, 0);
        for (int r = 0; r < len - gap.rows; ++r) {
            const int row = r >= gap.at ? r + gap.rows : r;
            CHECK(row < len);
            if (row < len) seen[row]++;
            CHECK(row % 16 == r % 16);
        }
        for (int row = 0; row < len; ++row) {
            const bool sees = window <= 0 || (long long)row >= (long long)len - window || row < sinks;
            CHECK(paged_visible(row, len, window, sinks) == sees);
            CHECK(seen[row] <= 1 && (seen[row] == 1 || !sees));
        }
        CHECK(!paged_visible(len, len, window, sinks));
        for (int row = 0; row < len; row += 16) {
            bool some_seen = false;
            for (int i = row; i < std::min(row + 16, len); ++i) some_seen |= paged_visible(i, len, window, sinks);
            CHECK((paged_window_len(row, len, window, sinks) > 0) == some_seen);
            bool all_seen = true;
            for (int i = row; i < row + 16; ++i) all_seen &= paged_visible(i, len, window, sinks);
            CHECK(!paged_whole(row, len, window, sinks) || all_seen);
            CHECK(paged_whole(row, len, window, sinks) || !all_seen || (window > 0 && row < sinks && sinks < row + 16));
        }
        // steps that a launch reckons with
        if (window > 0) CHECK((long long)len - gap.rows <= (long long)window + sinks + 48);
    }
    // ---- places that a sequence needs
    for (int t = 0; t < 60000; ++t) {
        const int log2_R = any(4, 7), R = 1 << log2_R, base = any(0, 500), fresh = any(0, 200), window = some(300), sinks = some(300);
        for (int p = 0; p < 50; ++p) {
            bool want = false;
            for (int row = p * R; row < std::min((p + 1) * R, base + fresh); ++row) want |= window <= 0 || row < sinks || (long long)row >= (long long)base + 1 - window;
            // (a page whose rows end behind the window's edge is kept up to its last row, though none may be there yet)
            if (want) CHECK(paged_wants(p, log2_R, base, fresh, window, sinks));
            if (paged_wants(p, log2_R, base, fresh, window, sinks)) CHECK(p * R < base + fresh);
            if (!want && (p + 1) * R <= base + fresh) CHECK(!paged_wants(p, log2_R, base, fresh, window, sinks));
        }
    }
    CHECK(!paged_wants(0, 4, 0, 0, 0, 0) && paged_wants(134217727, 4, 2147483647, 2147483647, 2147483647, 0));
    // ---- prompts: the tiles that a span of queries visits hold every key that any of them sees, each once, and the two questions about a tile are answered rightly
    for (int t = 0; t < 40000; ++t) {
        const int KT = any(0, 1) ? 64 : 32, queries = any(1, 150), p0 = any(-200, 900), p1 = p0 + queries - 1, window = some(700), sinks = some(300);
        const PromptSpan s = prompt_span(p0, p1, window, sinks);
        const PromptTiles tiles = prompt_tiles(s, KT);
        CHECK(tiles.count >= 0 && tiles.sink_tiles >= 0 && tiles.start >= 0 && tiles.sink_tiles <= tiles.start);
        std::vector<int> visited((std::max(p1, 0) + KT) / KT + 1, 0);
        for (int k = 0; k < tiles.count; ++k) {
            const int tile = prompt_tile(tiles, k);
            CHECK(tile >= 0 && tile * KT <= p1 && (k == 0 || tile > prompt_tile(tiles, k - 1)));
            if (tile >= 0 && tile < (int)visited.size()) visited[tile]++;
        }
        for (int tile = 0; tile * KT <= std::max(p1, 0); ++tile) {
            bool sees_some = false, sees_all = true;
            for (int pos = p0; pos <= p1; ++pos)
                for (int key = tile * KT; key < (tile + 1) * KT; ++key) {
                    const bool sees = key <= pos && (window <= 0 || (long long)key > (long long)pos - window || key < sinks);
                    CHECK(prompt_sees(key, pos, prompt_edge(pos, window), sinks) == sees);
                    sees_some |= sees;
                    sees_all &= sees;
                }
            if (sees_some) CHECK(visited[tile] == 1);
            if (sees_some) CHECK(prompt_some(s, tile * KT, KT));
            CHECK(!prompt_all(s, tile * KT, KT) || sees_all);
            if (sees_all && sinks < 2147483647) CHECK(prompt_all(s, tile * KT, KT) || (tile * KT < sinks && (tile + 1) * KT > sinks));
        }
    }
    printf("%lld %lld\n", checks, wrong);
    return wrong != 0;
}
"""


def test_index_arithmetic_against_brute_force(tmp_path):
    src, exe = tmp_path / "words.cpp", tmp_path / "words"
    src.write_text(WORDS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-Wno-dangling-else", "-fsanitize=undefined,address", "-I",
                           os.path.join(ROOT, "paper_2603_14303_amd", "csrc"), "-o", str(exe), str(src)])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    checks, wrong = map(int, out.stdout.split())
    assert wrong == 0 and checks > 10**6


def test_the_wrappers_refuse_what_does_not_fit(monkeypatch):
    torch = pytest.importorskip("torch")
    cpu = torch.zeros((4, 2, 32, 64), dtype=torch.int8)
    scale, table = torch.zeros((4, 2, 2)), torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(sc.SemantiCacheError, match="GPU"):
        sc.PagedCache8(cpu, cpu, scale, scale, table)
    with pytest.raises(sc.SemantiCacheError, match="GPU"):
        sc.sc_paged_reserve(table, 16, table[:, 0].contiguous(), table[:, 1].contiguous(), table[0], torch.zeros(1, dtype=torch.int32))
    with pytest.raises(sc.SemantiCacheError, match="GPU"):
        sc.sc_prompt_attn(*(torch.zeros((1, 2, 5, 64)) for _ in range(3)))
    monkeypatch.setattr(sc, "_require_cuda", lambda *t: None)
    cache = sc.PagedCache8(cpu, cpu, scale, scale, table)
    with pytest.raises(sc.SemantiCacheError):
        cache.K = cpu
    for bad in (dict(K=cpu.float()), dict(V=cpu[:, :1]), dict(k_scale=scale[:, :, :1].double()), dict(v_scale=torch.zeros((4, 2, 3))), dict(k_scale=torch.zeros((4, 2, 5)), v_scale=torch.zeros((4, 2, 5))),
                dict(table=table.long()), dict(table=torch.zeros((2, 2, 3), dtype=torch.int32)), dict(counts=torch.zeros((4, 2, 31), dtype=torch.int32))):
        with pytest.raises(sc.SemantiCacheError):
            sc.PagedCache8(**dict(dict(K=cpu, V=cpu, k_scale=scale, v_scale=scale, table=table, counts=None), **bad))
    lens, Q = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 4, 64))
    plain = sc.PagedCache(cpu.float(), cpu.float(), table)
    with pytest.raises(sc.SemantiCacheError, match="calls of its own"):
        sc.sc_paged_decode_attn(cache, Q, lens)
    with pytest.raises(sc.SemantiCacheError, match="calls of its own"):
        sc.sc_paged_append(cache, Q, Q, lens, lens)
    with pytest.raises(sc.SemantiCacheError, match="calls of its own"):
        sc.sc_paged_select(cache, Q, lens, 4)
    with pytest.raises(sc.SemantiCacheError, match="PagedCache8"):
        sc.sc_paged8_append(plain, Q, Q, lens, lens)
    with pytest.raises(sc.SemantiCacheError, match="PagedCache8"):
        sc.sc_paged8_decode_attn(plain, Q, lens)
    with pytest.raises(sc.SemantiCacheError, match="PagedCache"):
        sc.sc_paged_window_attn(cache, Q, lens, 4)
    with pytest.raises(sc.SemantiCacheError, match="32-bit"):
        sc.sc_paged_window_attn(plain, Q, lens, 2**31)
    with pytest.raises(sc.SemantiCacheError, match="32-bit"):
        sc.sc_paged_reserve(table, 16, lens, lens.clone(), lens, lens[:1], window=2**40)
    for bad in (dict(table=table[0]), dict(base_lens=lens.long()), dict(lens=lens[:1]), dict(new_lens=lens[:1]), dict(free_pages=table), dict(num_free=lens), dict(slots=torch.zeros((2, 3)), N=3),
                dict(slots=torch.zeros((2, 3), dtype=torch.int32), N=4), dict(slots=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(sc.SemantiCacheError):
            sc.sc_paged_reserve(**dict(dict(table=table, page_rows=16, base_lens=lens, lens=lens.clone(), free_pages=lens, num_free=lens[:1]), **bad))
    X, K = torch.zeros((2, 4, 5, 64)), torch.zeros((2, 2, 7, 64))
    for bad in (dict(K=K[0]), dict(V=K[:, :, :6]), dict(K=K[:1], V=K[:1]), dict(V=K.bfloat16()), dict(q_lens=lens.long()), dict(kv_lens=lens[:1]), dict(O=X.bfloat16()), dict(lse=torch.zeros((2, 4, 6))),
                dict(Q=X.transpose(2, 3).contiguous().transpose(2, 3))):
        with pytest.raises(sc.SemantiCacheError):
            sc.sc_prompt_attn(**dict(dict(Q=X, K=K, V=K), **bad))


def test_streams_are_those_of_the_device_that_holds_the_tensors(monkeypatch):
    """Launches go to the current device: tensors anywhere else are refused (stand-ins, as there may be one device or none)."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device)

    class On:
        def __init__(self, device):
            self.device = device

        def get_device(self):
            return self.device
    assert sc._stream_of(On(1), None, On(1)) == 101
    for tensors in ((On(0),), (On(1), On(0)), (On(1), None, On(-1))):
        with pytest.raises(sc.SemantiCacheError, match="cuda:1"):
            sc._stream_of(*tensors)
