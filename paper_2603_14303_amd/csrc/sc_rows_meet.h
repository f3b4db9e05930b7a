// Whether two arrays of rows have a byte in common, whatever their strides.  Plain functions, so that the host can try them.
#pragma once
#include <stdint.h>

namespace sc {

// rows of `bytes` bytes at every sum of i_k stride_k, 0 <= i_k < size_k (strides in bytes, 0 or more; that of a size of one means nothing)
struct RowsAt {
    uint64_t at;
    int64_t size[3], stride[3], bytes;
};

// They meet if  -a.bytes < a.at - b.at + sum of c_k s_k < b.bytes  for some whole c_k, lo_k <= c_k <= hi_k: a term for every stride s_k that either has (of a dimension that both have,
// the difference of the two numbers).  From the largest stride on, only few c_k leave a difference that the others can make up for, where arrays are laid out in any order of dimensions.
struct RowsSearch {
    __int128 s[6], lo[6], hi[6], below[7], above[7];      // below, above: what the terms from k on can add
    int terms;
    __int128 first, last;      // of the differences that meet
    int steps;
};
inline bool rows_search(RowsSearch &x, int k, __int128 d) {
    if (d + x.above[k] < x.first || d + x.below[k] > x.last) return false;
    if (k == x.terms) return true;
    // first <= d + c s + (below .. above) <= last
    const __int128 s = x.s[k], low = x.first - d - x.above[k + 1], high = x.last - d - x.below[k + 1];
    __int128 c = low >= 0 ? (low + s - 1) / s : -(-low / s), most = high >= 0 ? high / s : -((-high + s - 1) / s);
    if (c < x.lo[k]) c = x.lo[k];
    if (most > x.hi[k]) most = x.hi[k];
    for (; c <= most; ++c) {
        if (--x.steps < 0) return false;
        if (rows_search(x, k + 1, d + c * s)) return true;
    }
    return false;
}
// true: they do.  (Strides so contorted that this is not settled within 4096 steps are taken for apart.)
inline bool rows_meet(const RowsAt &a, const RowsAt &b) {
    RowsSearch x;
    x.terms = 0;
    for (int side = 0; side < 2; ++side)
        for (int i = 0; i < 3; ++i) {
            const RowsAt &r = side ? b : a;
            if (r.size[i] <= 1 || r.stride[i] == 0) continue;
            int k = 0;
            while (k < x.terms && x.s[k] > r.stride[i]) ++k;
            if (k == x.terms || x.s[k] != r.stride[i]) {
                for (int j = x.terms++; j > k; --j) { x.s[j] = x.s[j - 1]; x.lo[j] = x.lo[j - 1]; x.hi[j] = x.hi[j - 1]; }
                x.s[k] = r.stride[i];
                x.lo[k] = x.hi[k] = 0;
            }
            (side ? x.lo[k] : x.hi[k]) += side ? 1 - r.size[i] : r.size[i] - 1;
        }
    x.below[x.terms] = x.above[x.terms] = 0;
    for (int k = x.terms - 1; k >= 0; --k) {
        x.below[k] = x.below[k + 1] + x.lo[k] * x.s[k];
        x.above[k] = x.above[k + 1] + x.hi[k] * x.s[k];
    }
    x.first = 1 - (__int128)a.bytes;
    x.last = (__int128)b.bytes - 1;
    x.steps = 4096;
    return rows_search(x, 0, (__int128)a.at - (__int128)b.at);
}

}  // namespace sc
