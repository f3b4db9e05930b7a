"""What sc_prompt_attn writes meets nothing else, without a GPU: the refusals, and the test for strided rows (csrc/sc_rows_meet.h) against sets of bytes."""
import ctypes
import os
import subprocess

from paper_2603_14303_amd import binding as sc
from test_paged_host import ARG, FAKE, lib  # noqa: F401
from test_prompt_host import PROMPT

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MB = 1 << 20
APART = dict(PROMPT, Q=FAKE, K=FAKE + MB, V=FAKE + 2 * MB, O=FAKE + 3 * MB, lse=FAKE + 4 * MB, q_lens=FAKE + 5 * MB, kv_lens=FAKE + 6 * MB)
ROW = 128 * 2      # bytes


def test_outputs_that_meet_something_are_refused(lib):  # noqa: F811
    def call(**kw):
        return lib.sc_prompt_attn(ctypes.byref(sc._PromptStruct(**dict(APART, **kw))), FAKE + 8 * MB, 1 << 30, None)
    q, kv, o = 2 * 8 * 10 * ROW, 2 * 2 * 30 * ROW, 2 * 8 * 10 * ROW
    for name, size in (("Q", q), ("K", kv), ("V", kv)):
        for at in (APART[name], APART[name] + size - ROW, APART[name] - o + ROW, APART[name] + size - 16):
            assert call(O=at) == ARG, (name, at)
    for name in ("q_lens", "kv_lens", "lse"):
        assert call(**{name: APART["O"]}) == ARG and call(**{name: APART["O"] + o - 4}) == ARG and call(**{name: APART["O"] - 4}) == ARG, name
    for name in ("Q", "K", "V", "O", "q_lens", "kv_lens"):
        assert call(lse=APART[name]) == ARG and call(lse=APART[name] - 2 * 8 * 10 * 4 + 4) == ARG, name
    # in one array [B, N, heads, d]: the output's heads among the queries, the keys, the values
    fused = dict(q_stride_b=10 * 30 * 128, q_stride_h=128, q_stride_n=30 * 128, o_stride_b=10 * 30 * 128, o_stride_h=128, o_stride_n=30 * 128, M=10,
                 k_stride_b=10 * 30 * 128, k_stride_h=128, k_stride_n=30 * 128, v_stride_b=10 * 30 * 128, v_stride_h=128, v_stride_n=30 * 128, Q=FAKE, K=FAKE + 8 * ROW, V=FAKE + 10 * ROW)
    for head in (0, 7, 8, 11):
        assert call(**fused, O=FAKE + head * ROW) == ARG, head


MEETING = r"""
#include <stdio.h>
#include <stdlib.h>
#include <set>
#include "sc_rows_meet.h"
using namespace sc;
static int any(int lo, int hi) { return lo + (int)((unsigned)rand() % (unsigned)(hi - lo + 1)); }
static std::set<long long> bytes_of(const RowsAt &r) {
    std::set<long long> s;
    for (int i = 0; i < r.size[0]; ++i)
        for (int j = 0; j < r.size[1]; ++j)
            for (int k = 0; k < r.size[2]; ++k) {
                long long at = (long long)r.at;
                const int n[3] = {i, j, k};
                for (int x = 0; x < 3; ++x) at += n[x] * (r.size[x] > 1 ? r.stride[x] : 0);
                for (int e = 0; e < r.bytes; ++e) s.insert(at + e);
            }
    return s;
}
int main() {
    long long wrong = 0, meet = 0, apart_inside = 0;
    for (int t = 0; t < 40000; ++t) {
        RowsAt a, b;
        const bool shared = any(0, 1);      // both views of one array: the same strides
        const int heads = any(2, 6), d = any(1, 3), n = any(1, 4), bs = any(1, 3);
        for (RowsAt *r : {&a, &b}) {
            r->at = 1000 + any(0, shared ? heads * d * n * bs : 60);
            if (shared) {
                r->bytes = any(1, d);
                const int64_t size[3] = {bs, any(1, heads), n}, nhd[3] = {(int64_t)n * heads * d, d, (int64_t)heads * d}, hnd[3] = {(int64_t)n * heads * d, (int64_t)n * d, d};
                const bool x = any(0, 3) != 0;
                for (int i = 0; i < 3; ++i) { r->size[i] = size[i]; r->stride[i] = x ? nhd[i] : hnd[i]; }
            } else {
                r->bytes = any(1, 5);
                for (int i = 0; i < 3; ++i) { r->size[i] = any(1, 4); r->stride[i] = any(0, 3) ? any(0, 40) : any(0, 3) * 7; }
            }
        }
        const auto x = bytes_of(a), y = bytes_of(b);
        bool common = false;
        for (long long e : x) common |= y.count(e) != 0;
        meet += common;
        apart_inside += !common && *x.begin() < *y.rbegin() && *y.begin() < *x.rbegin();
        if (rows_meet(a, b) != common || rows_meet(b, a) != common) ++wrong;
    }
    // large ones: a head of 2^30 rows beside another, and the same of one row more
    const int64_t N = 1 << 30, row = 256;
    const RowsAt big = {1 << 20, {3, 8, N}, {N * 16 * row, row, 16 * row}, row};
    RowsAt other = big;
    other.at += 8 * row;
    wrong += rows_meet(big, other) || rows_meet(other, big);
    other.size[1] = 9;      // its last head is the first of the next row
    wrong += !rows_meet(big, other) || !rows_meet(other, big);
    other = {(1 << 20) + 8 * row + (uint64_t)(N - 1) * 16 * row, {1, 1, 1}, {0, 0, 0}, 4};      // behind the last row's heads of the first
    wrong += rows_meet(big, other);
    other.at -= 4;
    wrong += !rows_meet(big, other);
    printf("%lld meet, %lld apart inside each other, %lld wrong\n", meet, apart_inside, wrong);
    return wrong || meet < 5000 || apart_inside < 2000;
}
"""


def test_strided_rows_against_sets_of_bytes(tmp_path):
    source, program = tmp_path / "meeting.cpp", str(tmp_path / "meeting")
    source.write_text(MEETING)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2603_14303_amd", "csrc"), str(source), "-o", program], check=True)
    out = subprocess.run([program], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
