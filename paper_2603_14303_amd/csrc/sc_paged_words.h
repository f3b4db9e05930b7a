// Index arithmetic of the calls on a cache held in pages: which rows a workgroup touches, whatever lengths, page numbers and selections the device
// arrays hold.  Plain functions, so that the host can try them.
#pragma once
#include <stdint.h>

namespace sc {

// ---- sc_paged_append: the rows that a sequence (and head) receives
struct PagedAppendPlan {
    bool ok;             // the lengths are possible; otherwise nothing is written
    int first, last;     // pages (places in the table) that receive rows; last < first: none
};
constexpr PagedAppendPlan paged_append_plan(int base, int fresh, int N, int P, int log2_R, bool turned, int64_t pos0, int max_position) {
    const bool ok = base >= 0 && fresh >= 0 && fresh <= N && (int64_t)base + fresh <= (int64_t)P << log2_R &&
                    (!turned || fresh == 0 || (pos0 >= 0 && pos0 + fresh <= max_position));
    return ok && fresh > 0 ? PagedAppendPlan{true, base >> log2_R, (base + fresh - 1) >> log2_R} : PagedAppendPlan{ok, 0, -1};
}
// places in the table that a call of N rows can touch: its last row may be the first of one more page
constexpr int paged_append_slots(int N, int R, int P) {
    const int64_t most = ((int64_t)N + R - 2) / R + 1;
    return most < P ? (int)most : P;
}

// `shares` workgroups (KV heads) for each of `items` (pages): workgroup id -> item and share.  The hardware hands ids to the 8 chiplets in turn; with `near`,
// all shares of an item are on one chiplet, whose cache then has the angles for them.
struct PagedShare {
    int item, share;
};
constexpr PagedShare paged_share(int id, int shares, bool near) {
    if (!near) return {id / shares, id % shares};
    const int k = id / 8;
    return {k / shares * 8 + id % 8, k % shares};
}
constexpr int64_t paged_share_ids(int64_t items, int shares, bool near) { return near ? (items + 7) / 8 * 8 * shares : items * shares; }

// ---- sc_paged_decode_attn
// x / y for x >= 0, y > 0 and quotients up to 2^20, given 1 / y up to a few roundings (the kernel's lengths are on the device, and a division there costs
// as much as a trip to the cache)
constexpr int paged_quotient(int x, int y, float inverse) {
    int q = (int)((float)x * inverse);
    const int rest = x - q * y;
    q += rest >= y ? 1 : 0;
    return rest < 0 ? q - 1 : q;
}
// Units of rows, laid end to end over all heads.  A head's units are rounded up to a multiple of what a workgroup takes (`multiple`; 1: not at all).
constexpr int paged_units(int rows, int unit) { return rows > unit ? (int)(((int64_t)rows + unit - 1) / unit) : 1; }
// workgroups of a head that take up to `per` units each and nothing of another head
constexpr int paged_parts(int units, int per, float inverse) { return paged_quotient(units + per - 1, per, inverse); }
// The head of units [a, a + units), in stretches of `per`: the workgroups that hold a part of it, and where workgroup w leaves its partial result.
// Every workgroup has two places: for the stretch at its start, and for one that begins later in it (only a head's first workgroup can have begun with
// another head).
constexpr int paged_first_wg(int a, int per, float inverse) { return paged_quotient(a, per, inverse); }
constexpr int paged_last_wg(int a, int units, int per, float inverse) { return paged_quotient(a + units - 1, per, inverse); }
constexpr int paged_place(int w, int a, int per) { return 2 * w + (a > w * per ? 1 : 0); }

// n partial results of G heads are joined at once, or in groups of this many first (64 of 8 heads, on four KV heads of 32768 rows: 20.5 us in groups, 22.6 at once; 32 of
// 16: 13.9 and 14.3; with 128 in place of 256 no difference)
constexpr int paged_group(int n, int G) { return n * G <= 256 || n <= 16 ? n : 16; }

// 16 rows of a head from row `row` (a multiple of 16) on, or from the same row of its selected pages: their page, and how many of them attend
struct PagedStep {
    int page, left;
    bool bad;        // a place outside the table, or a page number outside the pool: page is 0 then, and left is 0
};
template <typename Table, typename Selection>
constexpr PagedStep paged_step(int row, int log2_R, int len, int P, int num_pages, Table table, bool selected, Selection sel) {
    const int in_page = row & ((1 << log2_R) - 1);
    int place = row >> log2_R;
    if (selected) {
        place = sel[place];
        if (place < 0 || place >= P) return {0, 0, true};
    }
    const int64_t left = (int64_t)len - (((int64_t)place << log2_R) + in_page);
    if (left <= 0) return {0, 0, false};      // entries behind the length are not read
    const int page = table[place];
    if (page < 0 || page >= num_pages) return {0, 0, true};
    return {page, left < 16 ? (int)left : 16, false};
}

// ---- a window of `window` rows (0: none) and the first `sinks` rows
constexpr bool paged_visible(int row, int len, int window, int sinks) { return row < len && (window <= 0 || row >= len - window || row < sinks); }
// Rows that no step visits: `rows` of them from row `at` on, both multiples of 16 (a step of 16 rows that begins at a multiple of 16 stays in one page)
struct PagedGap {
    int at, rows;
};
constexpr PagedGap paged_gap(int len, int window, int sinks) {
    if (window <= 0 || len <= window) return {0, 0};
    const int64_t at = ((int64_t)(sinks < len ? sinks : len) + 15) / 16 * 16, next = (int64_t)(len - window) / 16 * 16;
    return at < next ? PagedGap{(int)at, (int)(next - at)} : PagedGap{0, 0};
}
// all 16 rows from `row` on attend
constexpr bool paged_whole(int row, int len, int window, int sinks) {
    return (int64_t)row + 16 <= len && (window <= 0 || row >= (int64_t)len - window || (int64_t)row + 16 <= sinks);
}
// `len`, or 0 if none of the 16 rows from `row` (a multiple of 16) on is visible: their page is not looked up then
constexpr int paged_window_len(int row, int len, int window, int sinks) {
    return window <= 0 || (int64_t)row + 16 > (int64_t)len - window || row < sinks ? len : 0;
}

// ---- sc_paged_reserve: does place `place` of a table hold rows below base + fresh that a token from `base` on sees, or rows that arrive
constexpr bool paged_wants(int place, int log2_R, int base, int fresh, int window, int sinks) {
    const int64_t row = (int64_t)place << log2_R, end = row + (1 << log2_R);
    return row < (int64_t)base + fresh && (window <= 0 || row < sinks || end > (int64_t)base + 1 - window);
}

}  // namespace sc
