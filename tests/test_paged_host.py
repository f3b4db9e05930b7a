"""A cache held in pages, without a GPU: refusals of the sc_paged_* calls, and their index arithmetic (csrc/sc_paged_words.h) on good and bad
lengths, page numbers and selections."""
import ctypes
import os
import subprocess

import pytest

from paper_2603_14303_amd import binding as sc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # a 256-byte aligned non-null address; never dereferenced because validation fails first
ARG, UNSUPPORTED, CAPACITY, WORKSPACE = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sc.LIB_PATH):
        from paper_2603_14303_amd import build
        build.build(force=True)
    return sc.load_library()


CACHE = dict(K=FAKE, V=FAKE, counts=None, k_min=FAKE, k_max=FAKE, table=FAKE, stride_page=4 * 32 * 128, stride_head=32 * 128, stride_row=128, dtype=1,
             num_pages=100, page_heads=4, page_rows=32, table_len=20, table_per_head=0, B=2, Hkv=4, d=128)
ROWS = dict(K=FAKE, V=FAKE, k_stride_b=4 * 8 * 128, k_stride_h=8 * 128, k_stride_n=128, v_stride_b=4 * 8 * 128, v_stride_h=8 * 128, v_stride_n=128, N=8,
            base_lens=FAKE, new_lens=None, lens=FAKE + 256, cos_sin=FAKE, max_position=4096, rot=128, interleaved=0, Hq=8, positions=FAKE, Q=FAKE,
            Q_out=FAKE, q_stride_b=8 * 8 * 128, q_stride_h=8 * 128, q_stride_n=128, o_stride_b=8 * 8 * 128, o_stride_h=8 * 128, o_stride_n=128, q_dtype=1)

BAD_CACHES = [
    (dict(K=None), ARG), (dict(V=None), ARG), (dict(table=None), ARG), (dict(K=FAKE + 8), ARG), (dict(table=FAKE + 2), ARG), (dict(k_min=None), ARG),
    (dict(k_max=FAKE + 4), ARG), (dict(B=0), ARG), (dict(Hkv=0), ARG), (dict(num_pages=0), ARG), (dict(table_len=0), ARG), (dict(page_rows=8), ARG),
    (dict(page_rows=48), ARG), (dict(page_rows=2048), ARG), (dict(page_heads=2), ARG), (dict(table_per_head=1), ARG), (dict(page_heads=1), ARG),
    (dict(stride_row=64), ARG), (dict(stride_row=132), ARG), (dict(stride_row=2**30), ARG), (dict(stride_head=-128), ARG), (dict(stride_head=128), ARG),
    (dict(stride_head=32 * 128 - 8), ARG), (dict(stride_page=3 * 32 * 128), ARG), (dict(stride_page=4 * 32 * 128 + 4), ARG),
    (dict(d=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(B=70000), UNSUPPORTED), (dict(table_len=2**27), UNSUPPORTED),
    (dict(B=60000, Hkv=40, page_heads=40, stride_page=40 * 32 * 128), UNSUPPORTED),
]


def _status(call, cache=None, **kw):
    return call(sc._PagedCacheStruct(**dict(CACHE, **(cache or {}))), kw)


def test_append_rejects_bad_arguments(lib):
    def call(cache, kw):
        return lib.sc_paged_append(ctypes.byref(cache), ctypes.byref(sc._PagedRowsStruct(**dict(ROWS, **kw))), None)
    for bad, want in BAD_CACHES:
        assert _status(call, bad) == want, bad
    assert lib.sc_paged_append(None, ctypes.byref(sc._PagedRowsStruct(**ROWS)), None) == ARG
    assert lib.sc_paged_append(ctypes.byref(sc._PagedCacheStruct(**CACHE)), None, None) == ARG
    for name in ("K", "V", "base_lens", "lens", "Q", "Q_out"):
        assert _status(call, **{name: None}) == ARG, name
    for name in ("K", "V", "Q", "Q_out", "cos_sin"):
        assert _status(call, **{name: FAKE + 8}) == ARG, name
    for name in ("base_lens", "new_lens", "lens", "positions"):
        assert _status(call, **{name: FAKE + 514}) == ARG, name
    assert _status(call, N=0) == ARG and _status(call, N=-5) == ARG
    assert _status(call, lens=FAKE) == ARG                                    # read by some workgroups while another writes it
    assert _status(call, new_lens=FAKE + 256) == ARG
    assert _status(call, counts=FAKE) == ARG                                  # sizes without a place for them
    assert _status(call, dict(counts=FAKE)) == ARG                            # a place for sizes without any
    assert _status(call, dict(counts=FAKE + 4), counts=FAKE) == ARG
    assert _status(call, k_stride_n=132) == ARG and _status(call, v_stride_h=-8) == ARG and _status(call, q_stride_b=4) == ARG
    assert _status(call, o_stride_n=64) == ARG and _status(call, o_stride_h=0) == ARG      # two rows in one place
    for rot in (0, -16, 8, 24, 144):
        assert _status(call, rot=rot) == ARG, rot
    assert _status(call, max_position=0) == ARG
    assert _status(call, positions=None, per_head=1) == ARG                   # a token has one position
    assert _status(call, cos_sin=None, rot=0) == ARG                          # queries that nothing would turn
    assert _status(call, cos_sin=None, Q=None, Q_out=None) == ARG             # rot without angles
    assert _status(call, Hq=0) == ARG
    assert _status(call, q_dtype=7) == UNSUPPORTED and _status(call, Hq=70000) == UNSUPPORTED
    assert _status(call, dict(B=60000, Hkv=16, page_heads=16, page_rows=16, table_len=2**27 - 1, stride_page=16 * 32 * 128), N=2**31 - 1) == UNSUPPORTED      # grid


def test_append_refuses_lengths_that_are_read_while_they_are_written(lib):
    """positions, base_lens and new_lens are read by every workgroup; one of them writes lens.  B = 2 sequences, 4 heads."""
    arrays = dict(base_lens=FAKE + 1024, new_lens=FAKE + 5120, positions=FAKE + 4096)

    def status(lens, per_head=0):
        r = sc._PagedRowsStruct(**{**ROWS, **arrays, "lens": lens, "per_head": per_head})
        return lib.sc_paged_append(ctypes.byref(sc._PagedCacheStruct(**CACHE)), ctypes.byref(r), None)
    for name, at in arrays.items():
        assert status(at) == ARG and status(at + 4) == ARG and status(at - 4) == ARG, name
        # every head its own length: eight of them, and positions of the two sequences
        assert status(at, 1) == ARG and status(at + (4 if name == "positions" else 28), 1) == ARG and status(at - 28, 1) == ARG, name


def test_pools_of_any_order_and_none_that_overlap(lib):
    """Strides of pages, heads and rows (100 pages of 4 heads and 32 rows).  What passes is refused for its workspace."""
    def status(page, head, row, **kw):
        c = sc._PagedCacheStruct(**{**CACHE, "stride_page": page, "stride_head": head, "stride_row": row, **kw})
        return lib.sc_paged_decode_attn(ctypes.byref(c), FAKE, 1, 8, FAKE, 0, None, None, 0, 0.0, FAKE, 1, None, FAKE, 0, None)
    for s in ((16384, 4096, 128), (16384, 128, 512), (4096, 409600, 128), (128, 409600, 12800), (128, 12800, 51200), (512, 128, 51200), (20000, 4096, 128)):
        assert status(*s) == WORKSPACE, s
    for s in ((4088, 409600, 128), (4096, 409600 - 4096, 128), (128, 409600, 12792), (128, 128, 51200), (512, 128, 51192), (16384, 4096, 120), (2**61, 4096, 128), (16384, 0, 128), (16384, 4104, 128)):
        assert status(*s) == ARG, s
    # the stride of a dimension of one means nothing
    assert status(3, 4096, 128, num_pages=1) == WORKSPACE
    assert status(4096, 3, 128, page_heads=1, Hkv=8, table_per_head=1) == WORKSPACE


def test_append_refuses_queries_that_are_written_over_each_other(lib):
    """Q_out's rows [2, 8, 8, 128]: strides that are each as long as a row and still meet."""
    def status(b, h, n):
        r = sc._PagedRowsStruct(**{**ROWS, "new_lens": FAKE + 512, "o_stride_b": b, "o_stride_h": h, "o_stride_n": n})
        return lib.sc_paged_append(ctypes.byref(sc._PagedCacheStruct(**CACHE)), ctypes.byref(r), None)
    for strides in ((8192, 128, 128), (128, 1024, 128), (1024, 1024, 128), (8192, 1024, 136), (8184, 1024, 128), (8192 - 128, 128, 1024), (120, 128, 1024),
                    (2**62, 1024, 128)):
        assert status(*strides) == ARG, strides


def test_decode_rejects_bad_arguments(lib):
    need = lib.sc_paged_workspace_bytes(2, 8, 4, 128, 20)
    ok = dict(Q=FAKE, qdt=1, Hq=8, lens=FAKE, per_head=0, sel=FAKE, sel_lens=FAKE, keep=5, scale=0.0, O=FAKE, odt=1, lse=FAKE, ws=FAKE, wsb=need)

    def call(cache, kw):
        a = dict(ok, **kw)
        return lib.sc_paged_decode_attn(ctypes.byref(cache), a["Q"], a["qdt"], a["Hq"], a["lens"], a["per_head"], a["sel"], a["sel_lens"], a["keep"],
                                        a["scale"], a["O"], a["odt"], a["lse"], a["ws"], a["wsb"], None)
    for bad, want in BAD_CACHES:
        assert _status(call, bad) == want, bad
    for name in ("Q", "lens", "O", "sel", "sel_lens"):
        assert _status(call, **{name: None}) == ARG, name
    for name in ("Q", "O"):
        assert _status(call, **{name: FAKE + 8}) == ARG, name
    for name in ("lens", "sel", "sel_lens", "lse"):
        assert _status(call, **{name: FAKE + 2}) == ARG, name
    assert _status(call, Hq=0) == ARG and _status(call, Hq=9) == UNSUPPORTED and _status(call, Hq=68) == UNSUPPORTED      # 17 heads to a KV head
    assert _status(call, qdt=3) == UNSUPPORTED and _status(call, odt=-1) == UNSUPPORTED
    assert _status(call, scale=float("nan")) == ARG
    assert _status(call, keep=0) == CAPACITY and _status(call, keep=2**20 + 1) == UNSUPPORTED
    assert _status(call, ws=None) == WORKSPACE and _status(call, ws=FAKE + 8) == WORKSPACE and _status(call, wsb=4096) == WORKSPACE
    assert _status(call, dict(counts=FAKE + 4)) == ARG


def test_select_rejects_bad_arguments(lib):
    need = lib.sc_paged_workspace_bytes(2, 8, 4, 128, 20)
    ok = dict(Q=FAKE, qdt=1, Hq=8, lens=FAKE, per_head=0, keep=5, first=1, recent=2, sel=FAKE, sel_lens=FAKE, ws=FAKE, wsb=need)

    def call(cache, kw):
        a = dict(ok, **kw)
        return lib.sc_paged_select(ctypes.byref(cache), a["Q"], a["qdt"], a["Hq"], a["lens"], a["per_head"], a["keep"], a["first"], a["recent"], a["sel"],
                                   a["sel_lens"], a["ws"], a["wsb"], None)
    for bad, want in BAD_CACHES:
        assert _status(call, bad) == want, bad
    for name in ("Q", "lens", "sel", "sel_lens"):
        assert _status(call, **{name: None}) == ARG, name
    assert _status(call, dict(k_min=None, k_max=None)) == ARG                 # no summaries to go by
    assert _status(call, first=-1) == ARG and _status(call, recent=-1) == ARG
    assert _status(call, keep=0) == CAPACITY and _status(call, keep=2) == CAPACITY and _status(call, first=2**31 - 1) == CAPACITY
    assert _status(call, keep=2**20 + 1) == UNSUPPORTED and _status(call, Hq=9) == UNSUPPORTED and _status(call, qdt=3) == UNSUPPORTED
    assert _status(call, ws=None) == WORKSPACE and _status(call, ws=FAKE + 8) == WORKSPACE and _status(call, wsb=256) == WORKSPACE


def test_workspace(lib):
    f = lib.sc_paged_workspace_bytes
    assert f(0, 8, 4, 128, 20) == 0 and f(2, 9, 4, 128, 20) == 0 and f(2, 8, 4, 96, 20) == 0 and f(2, 8, 4, 128, 0) == 0
    assert f(2, 8, 4, 128, 20) % 256 == 0 and f(64, 64, 8, 128, 1 << 16) >= 64 * 8 * (1 << 16) * 8
    assert lib.sc_paged_init_workspace(None, 1 << 20, None) == WORKSPACE and lib.sc_paged_init_workspace(FAKE, 16, None) == WORKSPACE
    assert lib.sc_paged_init_workspace(FAKE + 8, 1 << 20, None) == WORKSPACE


WORDS = r"""
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <algorithm>
#include <vector>
#include "sc_paged_words.h"
using namespace sc;
static long long checks = 0, wrong = 0;
#define CHECK(x) do { ++checks; if (!(x)) { ++wrong; printf("line %d: %s\n", __LINE__, #x); if (wrong > 20) exit(1); } } while (0)
static int any(int lo, int hi) { return lo + rand() % (hi - lo + 1); }

// what a device array may hold where a number of [0, most) belongs
static int weird(int most) {
    switch (any(0, 9)) {
        case 0: return -1;
        case 1: return most;
        case 2: return -2147483647 - 1;
        case 3: return 2147483647;
        default: return any(0, most - 1);
    }
}

// 1 / y with an error of up to three roundings
static float inverse_of(int y) {
    float f = 1.0f / (float)y;
    for (int k = any(-3, 3); k; k += k > 0 ? -1 : 1) f = nextafterf(f, k > 0 ? 2.0f * f : 0.0f);
    return f;
}

// a table (a selection) that knows which of its entries may be read
struct Guarded {
    const std::vector<int> *v;
    int readable;
    int operator[](int i) const { CHECK(i >= 0 && i < (int)v->size() && i < readable); return (*v)[std::min(std::max(i, 0), (int)v->size() - 1)]; }
};

int main() {
    // ---- appended rows lie in the pages first .. last, and the slots of the launch reach them
    for (int t = 0; t < 300000; ++t) {
        const int log2_R = any(4, 10), R = 1 << log2_R, P = any(1, 6), N = any(1, 3 * R), turned = any(0, 1), most = any(1, 4 * R);
        const int base = any(0, 5) ? any(0, P * R) : weird(P * R), fresh = any(0, 5) ? any(0, N) : weird(N + 1);
        const long long pos0 = any(0, 5) ? any(0, most) : weird(most);
        const PagedAppendPlan a = paged_append_plan(base, fresh, N, P, log2_R, turned, pos0, most);
        const bool ok = base >= 0 && fresh >= 0 && fresh <= N && (long long)base + fresh <= (long long)P * R && (!turned || fresh == 0 || (pos0 >= 0 && pos0 + fresh <= most));
        CHECK(a.ok == ok);
        if (!ok || fresh == 0) { CHECK(a.last < a.first); continue; }
        CHECK(a.first == base / R && a.last == (base + fresh - 1) / R && a.last < P && a.last - a.first < paged_append_slots(N, R, P));
    }
    CHECK(!paged_append_plan(2147483647, 2147483647, 2147483647, 1 << 20, 10, false, 0, 0).ok);
    CHECK(paged_append_slots(2147483647, 16, 1 << 20) == 1 << 20 && paged_append_slots(1, 16, 9) == 1 && paged_append_slots(2, 16, 9) == 2 && paged_append_slots(17, 16, 9) == 2);
    CHECK(paged_append_slots(18, 16, 9) == 3);
    // ---- shares of items: every one has an id, those behind the last item are known by it; near shares are eight ids apart
    for (int t = 0; t < 2000; ++t) {
        const int items = any(1, 100), shares = any(1, 40), near = any(0, 1);
        std::vector<int> seen(items * shares, 0), chiplet(items, -1);
        const long long ids = paged_share_ids(items, shares, near);
        CHECK(ids < (long long)(items + 8) * shares);
        for (int id = 0; id < ids; ++id) {
            const PagedShare s = paged_share(id, shares, near);
            CHECK(s.share >= 0 && s.share < shares && s.item >= 0 && s.item < items + 8);
            if (s.item >= items) { CHECK(near); continue; }
            seen[s.item * shares + s.share]++;
            if (near) { CHECK(chiplet[s.item] < 0 || chiplet[s.item] == id % 8); chiplet[s.item] = id % 8; }
        }
        for (int x : seen) CHECK(x == 1);
    }
    // ---- stretches: every unit of every head belongs to one workgroup, its parts have places of their own, and the workgroups count themselves off
    for (int t = 0; t < 20000; ++t) {
        const int heads = any(1, 40), wgs = any(1, 64), unit = 16 * any(1, 12);
        std::vector<int> units;
        int total = 0;
        for (int h = 0; h < heads; ++h) {
            const int rows = any(0, 3) ? any(0, 400 * any(1, 20)) : any(0, 17);
            units.push_back(paged_units(rows, unit));
            CHECK((long long)units.back() * unit >= rows && units.back() >= 1 && (units.back() == 1 || (units.back() - 1) * unit < rows));
            total += units.back();
        }
        // equal shares, or heads rounded up to a multiple of a workgroup's units
        int per = (total + wgs - 1) / wgs, multiple = 1;
        if (any(0, 1)) {
            for (multiple = per;; ++multiple) {
                int parts = 0;
                for (int u : units) parts += paged_parts(u, multiple, inverse_of(multiple));
                if (parts <= wgs || multiple > 4 * per + 400) break;
            }
            int parts = 0;
            for (int &u : units) {
                const int n = paged_parts(u, multiple, inverse_of(multiple));
                CHECK(n * multiple >= u && (n - 1) * multiple < u);
                parts += n;
                u = n * multiple;
            }
            if (parts > wgs) continue;
            per = multiple;
            total = parts * multiple;
        }
        const float inverse = inverse_of(per);
        std::vector<int> covered(total, 0), places(2 * wgs, -1), left(heads, 0);
        for (int w = 0; w < wgs; ++w) {
            int pos = w * per;
            const int stop = std::min(pos + per, total);
            int h = 0, a = 0;
            while (h < heads && a + units[h] <= pos) a += units[h++];
            for (; pos < stop; a += units[h++]) {
                const int end = std::min(a + units[h], stop);
                for (int u = pos; u < end; ++u) covered[u]++;
                const int w0 = paged_first_wg(a, per, inverse), w1 = paged_last_wg(a, units[h], per, inverse);
                CHECK(w0 == a / per && w1 == (a + units[h] - 1) / per && w0 <= w && w <= w1);
                if (multiple > 1) CHECK(pos == w * per && end == stop);      // parts of one head only
                if (w0 == w1) CHECK(pos == a && end == a + units[h]);
                else {
                    const int place = paged_place(w, a, per);
                    CHECK(place >= 0 && place < 2 * wgs && places[place] == -1);
                    places[place] = h;
                    left[h]++;
                }
                pos = end;
            }
        }
        for (int u = 0; u < total; ++u) CHECK(covered[u] == 1);
        for (int h = 0, a = 0; h < heads; a += units[h++]) {
            const int w0 = paged_first_wg(a, per, inverse), w1 = paged_last_wg(a, units[h], per, inverse);
            CHECK(left[h] == (w1 > w0 ? w1 - w0 + 1 : 0));
            if (w1 > w0) for (int w = w0; w <= w1; ++w) CHECK(places[paged_place(w, a, per)] == h);
        }
    }
    // ---- quotients, from inverses that are off by some roundings
    for (int t = 0; t < 2000000; ++t) {
        const int y = any(0, 1) ? any(1, 300) : 1 + (int)((long long)rand() * rand() % (1 << 30)), most = (int)std::min<long long>(2147483647ll - 2 * y, (1ll << 20) * y);
        if (most <= 0) continue;
        int x = (int)(((long long)rand() << 20 ^ rand()) % most);
        if (any(0, 2) == 0) x = x / y * y;
        if (any(0, 2) == 0 && x >= y) x = x / y * y - 1;
        CHECK(paged_quotient(x, y, inverse_of(y)) == x / y);
    }
    // ---- groups of partial results: of one size, few enough to be joined in the shared memory of a workgroup
    for (int n = 1; n <= 256; ++n)
        for (int G = 1; G <= 16; ++G) {
            const int group = paged_group(n, G), groups = (n + group - 1) / group;
            int pad = 1;
            while (pad < G) pad *= 2;
            CHECK(group >= 1 && group <= n && group * pad <= 512 && groups * pad <= 512 && (groups == 1 || group == 16));
        }
    CHECK(paged_units(2147483647, 96) == 22369622 && paged_units(0, 96) == 1 && paged_units(-5, 96) == 1);
    // ---- a step's page: in the pool whatever the arrays hold, its rows those that the length leaves
    for (int t = 0; t < 300000; ++t) {
        const int log2_R = any(4, 8), R = 1 << log2_R, P = any(1, 9), pool = any(1, 30), len = any(0, P * R), keep = any(1, 9), selected = any(0, 1);
        std::vector<int> table(P), sel(keep);
        for (int &x : table) x = any(0, 3) ? any(0, pool - 1) : weird(pool);
        for (int &x : sel) x = any(0, 3) ? any(0, P - 1) : weird(P);
        const Guarded tab{&table, (len + R - 1) / R}, se{&sel, keep};
        const int row = 16 * any(0, (selected ? keep : P) * R / 16 - 1);
        const PagedStep s = paged_step(row, log2_R, len, P, pool, tab, selected, se);
        CHECK(s.page >= 0 && s.page < pool && s.left >= 0 && s.left <= 16);
        const int place = selected ? sel[row / R] : row / R;
        if (place < 0 || place >= P) { CHECK(s.bad && s.left == 0); continue; }
        const int want = std::min(std::max(len - (place * R + row % R), 0), 16);
        if (want == 0) CHECK(!s.bad && s.left == 0);
        else if (table[place] < 0 || table[place] >= pool) CHECK(s.bad && s.left == 0);
        else CHECK(!s.bad && s.left == want && s.page == table[place]);
    }
    printf("%lld %lld\n", checks, wrong);
    return wrong != 0;
}
"""


def test_index_arithmetic_stays_inside_whatever_the_arrays_hold(tmp_path):
    src, exe = tmp_path / "words.cpp", tmp_path / "words"
    src.write_text(WORDS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-Wno-dangling-else", "-fsanitize=undefined,address", "-I",
                           os.path.join(ROOT, "paper_2603_14303_amd", "csrc"), "-o", str(exe), str(src)])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    checks, wrong = map(int, out.stdout.split())
    assert wrong == 0 and checks > 10**6


def test_the_wrappers_refuse_what_does_not_fit():
    torch = pytest.importorskip("torch")
    K = torch.zeros((3, 2, 16, 64))
    table = torch.zeros((1, 2), dtype=torch.int32)
    with pytest.raises(sc.SemantiCacheError, match="GPU"):
        sc.PagedCache(K, K.clone(), table)
    with pytest.raises(sc.SemantiCacheError, match="identical"):
        sc.PagedCache(K, torch.zeros((3, 2, 32, 64)), table)
    with pytest.raises(sc.SemantiCacheError, match="table"):
        sc.PagedCache(K, K.clone(), table.to(torch.int64))
    with pytest.raises(sc.SemantiCacheError, match="one head"):
        sc.PagedCache(K, K.clone(), torch.zeros((1, 2, 4), dtype=torch.int32))
    with pytest.raises(sc.SemantiCacheError, match="counts"):
        sc.PagedCache(K, K.clone(), table, counts=torch.zeros((3, 2, 16)))
    with pytest.raises(sc.SemantiCacheError, match="together"):
        sc.PagedCache(K, K.clone(), table, k_min=torch.zeros((3, 2, 64)))
    with pytest.raises(sc.SemantiCacheError, match="dtype"):
        sc.PagedCache(K, K.clone(), table, k_min=torch.zeros((3, 2, 64)), k_max=torch.zeros((3, 2, 64), dtype=torch.bfloat16))


def test_the_tensors_of_a_cache_stay_the_same_ones(monkeypatch):
    """The library is given addresses: a tensor put in the place of another would not be seen, and the old one's memory would be used after it was freed."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(sc, "_require_cuda", lambda *a: None)
    K, table = torch.zeros((3, 2, 16, 64)), torch.zeros((1, 2), dtype=torch.int32)
    cache = sc.PagedCache(K, K.clone(), table)
    assert cache.struct.table == table.data_ptr() and cache.ptr == ctypes.addressof(cache.struct)
    for name, value in (("table", torch.zeros((1, 9), dtype=torch.int32)), ("K", K.clone()), ("counts", None), ("struct", None), ("ptr", 0), ("B", 2), ("other", 1)):
        with pytest.raises(sc.SemantiCacheError, match="new PagedCache"):
            setattr(cache, name, value)
    with pytest.raises(sc.SemantiCacheError, match="new PagedCache"):
        del cache.V
    assert cache.table is table and cache.struct.table == table.data_ptr()


def test_numbers_beyond_32_bits_are_refused(monkeypatch):
    """2^32 + 5 pages to keep are not five, and 2^32 + 3 rows (of stride zero) not three."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(sc, "_require_cuda", lambda *a: None)
    K, table, lens = torch.zeros((3, 2, 16, 64)), torch.zeros((1, 2), dtype=torch.int32), torch.zeros((1,), dtype=torch.int32)
    cache = sc.PagedCache(K, K.clone(), table)
    Q = torch.zeros((1, 2, 64))
    for kw in (dict(keep=2**32 + 5), dict(keep=5, first=2**32), dict(keep=5, recent=2**32 + 1)):
        with pytest.raises(sc.SemantiCacheError, match="32-bit"):
            sc.sc_paged_select(cache, Q, lens, **kw, sel=torch.zeros((1, 2, 5), dtype=torch.int32), workspace=object())
    rows = torch.zeros((1, 2, 1, 64)).expand(1, 2, 2**32 + 3, 64)
    with pytest.raises(sc.SemantiCacheError, match="32-bit"):
        sc.sc_paged_append(cache, rows, rows, lens, lens.clone())
