// A cache held in pages as the kernels see it (internal; the public boundary is include/semanticache.h), and the launchers of its calls.
#pragma once
#include "sc_device.h"
#include "sc_host.h"
#include "sc_paged_words.h"

namespace sc {

struct PagedView {
    char *K, *V;
    int32_t *counts;
    char *k_min, *k_max;
    const int32_t *table;
    int64_t page_bytes, head_bytes;        // strides of the pools
    int row_bytes;
    int num_pages, page_heads;
    int R, log2_R;                         // rows of a page
    int P;                                 // entries of a table
    int table_per_head;
    int B, H, d;
    DType dtype;
};

__device__ __forceinline__ const int32_t *paged_table(const PagedView &c, int b, int h) {
    return c.table + (c.table_per_head ? (int64_t)b * c.H + h : (int64_t)b) * c.P;
}
// byte offset of a page's rows for head h, and its number among the pages' heads (counts, summaries)
__device__ __forceinline__ int64_t paged_offset(const PagedView &c, int page, int h) {
    return (int64_t)page * c.page_bytes + (c.page_heads == 1 ? 0 : (int64_t)h * c.head_bytes);
}
__device__ __forceinline__ int64_t paged_index(const PagedView &c, int page, int h) {
    return (int64_t)page * c.page_heads + (c.page_heads == 1 ? 0 : h);
}
__device__ __forceinline__ bool paged_bad(const PagedView &c, int page) { return (unsigned)page >= (unsigned)c.num_pages; }

// ---- across the lanes
// Sums over the lanes up to each one (DPP moves inside the rows of 16 lanes, then from row to row), and the maximum over all of them
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_rows(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_scan(int x) {
    x += dpp_rows<0x111, 0xf>(x);      // row_shr 1, 2, 4, 8
    x += dpp_rows<0x112, 0xf>(x);
    x += dpp_rows<0x114, 0xf>(x);
    x += dpp_rows<0x118, 0xf>(x);
    x += dpp_rows<0x142, 0xa>(x);      // row_bcast 15: lane 15 to the second row, lane 47 to the fourth
    x += dpp_rows<0x143, 0xc>(x);      // row_bcast 31: lane 31 to the upper half
    return x;
}
__device__ __forceinline__ int wave_max(int x) {      // x >= 0
    x = max(x, dpp_rows<0x111, 0xf>(x));
    x = max(x, dpp_rows<0x112, 0xf>(x));
    x = max(x, dpp_rows<0x114, 0xf>(x));
    x = max(x, dpp_rows<0x118, 0xf>(x));
    x = max(x, dpp_rows<0x142, 0xa>(x));
    x = max(x, dpp_rows<0x143, 0xc>(x));
    return __builtin_amdgcn_readlane(x, kWave - 1);
}

__device__ __forceinline__ float row_allreduce_max(float x) {      // over the 16 lanes of a row
    x = fmaxf(x, dpp<kDppQuadXor1>(x));
    x = fmaxf(x, dpp<kDppQuadXor2>(x));
    x = fmaxf(x, dpp<kDppHalfMirror>(x));
    return fmaxf(x, dpp<kDppMirror>(x));
}

// ---- sc_paged_append
struct PagedAppendArgs {
    PagedView c;
    const char *K, *V;
    int64_t k_b, k_h, k_n, v_b, v_h, v_n;   // bytes
    const int32_t *counts;
    int N, per_head;
    const int32_t *base_lens, *new_lens;
    int32_t *lens;
    const float *cos_sin;
    int max_position, rot, interleaved, Hq;
    const int32_t *positions;
    const char *Q;
    char *Q_out;
    int64_t q_b, q_h, q_n, o_b, o_h, o_n;   // bytes
    DType q_dtype;
};
// whether the call fits a grid: a workgroup per page and KV head, and per 16 tokens and query head at worst
inline bool paged_append_fits(int64_t B, int64_t H, int64_t R, int64_t N, int64_t Hq) {
    return (B * ((N + R - 2) / R + 1) + 7) * H + B * ((N + 15) / 16) * Hq <= INT32_MAX;
}
hipError_t launch_paged_append(const PagedAppendArgs &a, hipStream_t stream);

// ---- sc_paged_decode_attn
struct PagedDecodeArgs {
    PagedView c;
    const void *Q;
    DType q_dtype;
    int Hq;
    const int32_t *lens;
    int lens_per_head;
    const int32_t *sel, *sel_lens;
    int keep;
    float scale;
    void *O;
    DType o_dtype;
    float *lse;
    void *ws;
};
hipError_t launch_paged_decode(const PagedDecodeArgs &a, hipStream_t stream);

// ---- sc_paged_select
struct PagedSelectArgs {
    PagedView c;
    const void *Q;
    DType q_dtype;
    int Hq;
    const int32_t *lens;
    int lens_per_head;
    int keep, first, recent;
    int32_t *sel, *sel_lens;
    void *ws;
};
hipError_t launch_paged_select(const PagedSelectArgs &a, hipStream_t stream);

// ---- workspace: counters, then what the two calls need (they follow each other on a stream, so it is the same memory)
size_t paged_state_bytes();
size_t paged_decode_bytes(int G, int d);
size_t paged_select_bytes(int B, int H, int P);

}  // namespace sc
