// sc_paged_append: new rows of keys and values go to the pages of their sequences, rotated by their positions on the way, together with the queries
// of the same tokens; the pages' summaries (minimum and maximum of their keys) follow.
//
//     a' = a cos - b sin,  b' = b cos + a sin   for the pairs (a, b) of the first `rot` elements of a row, in fp32, rounded once.
//
// Bound by bytes: every row is read once and written once, and there are two operations a byte.  One to four wavefronts take one page of one KV head:
// all the rows that the call adds to that page, and, where summaries are kept, the keys that the page held before, so that no workgroup depends on
// another.  A lane holds two pieces of 16 bytes of a row, chosen so that the partners of a rotation are in the same lane.  The queries are rotated by workgroups of their own, which go over the heads of a group of tokens and read the angles once.
//
// Measured (d = 128, bf16): a prompt of 32768 tokens, 8 KV and 32 query heads: 152 us, 5.4 TB/s of rows read and written (a copy of that size: 5.2); one token
// 4.1 us, of which the launch is 1.8; 32 heads of 3000 to 6000 merged rows 36 us (4.2 TB/s; a copy of that size takes 32).
#include "sc_paged_rows.h"

namespace sc {

// a NaN stays
__device__ __forceinline__ float lower(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float higher(float a, float b) { return __builtin_elementwise_maximum(a, b); }
template <bool LOW> __device__ __forceinline__ float extreme(float a, float b) { return LOW ? lower(a, b) : higher(a, b); }

// The extremes over the lanes with the same pieces (lane % LPR).  Two values that are exchanged between the halves of the wavefront, and between its
// rows of 16 lanes, are reduced together, each in one half: lane (row r of 16 lanes, any place in it) ends up with values N / 4 r .. of the N.
template <int LPR, bool LOW, int N> __device__ __forceinline__ void gather_extremes(const float (&x)[N], float (&z)[N / 4]) {
    float y[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[i]), __float_as_uint(x[i + N / 2]), false, false);
        y[i] = extreme<LOW>(__uint_as_float(t[0]), __uint_as_float(t[1]));
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(y[i]), __float_as_uint(y[i + N / 4]), false, false);
        z[i] = extreme<LOW>(__uint_as_float(t[0]), __uint_as_float(t[1]));
        if constexpr (LPR <= 8) z[i] = extreme<LOW>(z[i], dpp<kDppRor8>(z[i]));
        if constexpr (LPR <= 4) z[i] = extreme<LOW>(z[i], dpp<kDppRor4>(z[i]));
    }
}

// ROT: with angles (without any, there are no queries either)
template <typename T, typename TQ, int D, bool ROT>
__global__ __launch_bounds__(kAppThreads) void paged_append_kernel(PagedAppendArgs p, AppendGrid g) {
    constexpr int WAVES = kAppThreads / kWave;
    constexpr int U = 2;                        // passes whose loads are on their way together
    const int tid = threadIdx.x;
    const PagedView &c = p.c;
    const int half = p.rot / 2;
    const bool interleaved = p.interleaved != 0;

    if (ROT && (int)blockIdx.x >= g.kv_blocks) {
        rotate_queries<TQ, D>(p, g, (int)blockIdx.x - g.kv_blocks);
        return;
    }

    // ---- keys and values: the wavefronts of the workgroup have one page of one KV head together, or several pages
    constexpr int E = Shape<T>::E, LPR = D / (2 * E);
    constexpr int RPW = kWave / LPR;            // rows of a wavefront's pass
    const int lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int j = lane % LPR;
    const Pieces at = pieces_of<E>(j, p.rot, interleaved);
    const PagedShare at_work = paged_share((int)blockIdx.x, c.H, g.kv_near != 0);
    const int h = at_work.share, group = at_work.item % g.page_groups, b = at_work.item / g.page_groups;
    if (b >= c.B) return;
    const int wpp = 1 << g.log2_waves, part = wave & (wpp - 1);
    const int li = p.per_head ? b * c.H + h : b;
    const int base = read_scalar(p.base_lens + li), new_len = read_scalar((p.new_lens ? p.new_lens : p.base_lens) + li);
    const int position = read_scalar(p.positions ? p.positions + b : p.base_lens + li);
    const int fresh = p.new_lens ? new_len : p.N;
    const int64_t pos0 = position;
    const PagedAppendPlan plan = paged_append_plan(base, fresh, p.N, c.P, c.log2_R, p.cos_sin != nullptr, pos0, p.max_position);
    const int32_t *table = paged_table(c, b, h);
    const int place = plan.first + group * (WAVES >> g.log2_waves) + (wave >> g.log2_waves);
    if (group == 0 && (p.per_head || h == 0)) {
        // the length of the sequence (and head): -1 if any page that it needs is not there
        int bad = 0;
        const int heads = (c.table_per_head && !p.per_head) ? c.H : 1;      // pages of their own, one length
        for (int k = 0; k < heads; ++k)
            for (int i = plan.first + tid; i <= plan.last; i += kAppThreads) bad |= paged_bad(c, table[(int64_t)k * c.P + i]);
        bad = __syncthreads_or(bad);
        if (tid == 0) p.lens[li] = (plan.ok && !bad) ? base + fresh : -1;
    }
    const int page = place <= plan.last ? read_scalar(table + place) : -1;
    const bool there = !paged_bad(c, page);
    const bool summary = c.k_min != nullptr;
    const int64_t row0 = (int64_t)place << c.log2_R;       // row of the sequence at the page's start
    const int r0 = (int)max((int64_t)base - row0, (int64_t)0), r1 = there ? (int)min((int64_t)base + fresh - row0, (int64_t)c.R) : 0;
    char *kp = c.K + (there ? paged_offset(c, page, h) : 0), *vp = c.V + (there ? paged_offset(c, page, h) : 0);
    const char *ks = p.K + b * p.k_b + h * p.k_h, *vs = p.V + b * p.v_b + h * p.v_h;
    const int32_t *sizes = p.counts + ((int64_t)b * c.H + h) * p.N;
    int32_t *counts = c.counts + (there ? paged_index(c, page, h) * c.R : 0);
    const int oa = at.ea * (int)sizeof(T), ob = at.eb * (int)sizeof(T);
    const int pass = RPW << g.log2_waves, from = summary ? 0 : r0;
    float lo[2 * E], hi[2 * E];
#pragma unroll
    for (int i = 0; i < 2 * E; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
    // rows t of the page: those below r0 are there already (and count in the summary), r0 .. r1 are new.  Lanes behind the last row read it again, so
    // that all loads of a pass are on their way at once.
    for (int t0 = from / pass * pass + part * RPW; t0 < r1; t0 += U * pass) {
        Raw<T> ka[U], kb[U], va[U], vb[U];
        float co[U][E], si[U][E];
        int size[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = min(max(t0 + u * pass + lane / LPR, from), r1 - 1);
            const int64_t n = row0 + max(t, r0) - base;      // row of the call
            const char *k = t < r0 ? kp + (int64_t)t * c.row_bytes : ks + n * p.k_n, *v = vs + n * p.v_n;
            ka[u].load(k + oa);
            kb[u].load(k + ob);
            va[u].load(v + oa);
            vb[u].load(v + ob);
            if constexpr (ROT) {
                const float *angles = p.cos_sin + (pos0 + n) * p.rot + (at.turned ? E * j : 0);
                load_angles(angles, co[u]);
                load_angles(angles + half, si[u]);
            }
            if (c.counts) size[u] = sizes[n];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * pass + lane / LPR;
            const bool is_new = t >= r0 && t < r1;
            if constexpr (ROT) {
                if (is_new && at.turned) {
                    float x[E], y[E];
                    ka[u].widen(x);
                    kb[u].widen(y);
                    turn(x, y, co[u], si[u], interleaved);
                    ka[u].round(x);
                    kb[u].round(y);
                }
            }
            if (is_new) {
                ka[u].store(kp + (int64_t)t * c.row_bytes + oa);
                kb[u].store(kp + (int64_t)t * c.row_bytes + ob);
                va[u].store(vp + (int64_t)t * c.row_bytes + oa);
                vb[u].store(vp + (int64_t)t * c.row_bytes + ob);
                if (c.counts && j == 0) counts[t] = size[u];
            }
            if (summary && t < r1) {      // of the keys as stored
                float x[E], y[E];
                ka[u].widen(x);
                kb[u].widen(y);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    lo[i] = lower(lo[i], x[i]);
                    hi[i] = higher(hi[i], x[i]);
                    lo[E + i] = lower(lo[E + i], y[i]);
                    hi[E + i] = higher(hi[E + i], y[i]);
                }
            }
        }
    }
    if (!summary) return;
    // ---- the lanes with the same pieces, then the page's wavefronts
    constexpr int M = E / 2;                // elements that a lane ends up with
    __shared__ __attribute__((aligned(16))) float s_lo[WAVES][D], s_hi[WAVES][D];
    float l[M], u[M];
    gather_extremes<LPR, true>(lo, l);
    gather_extremes<LPR, false>(hi, u);
    const int first = M * (lane / 16);
    const int el = first < E ? at.ea + first : at.eb + first - E;
    const bool writes = lane % 16 < LPR;
    if (wpp > 1) {
        if (writes) {
#pragma unroll
            for (int i = 0; i < M; ++i) {
                s_lo[wave][el + i] = l[i];
                s_hi[wave][el + i] = u[i];
            }
        }
        __syncthreads();
        if (part != 0) return;
        if (writes)
            for (int w = 1; w < wpp; ++w)
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    l[i] = lower(l[i], s_lo[wave + w][el + i]);
                    u[i] = higher(u[i], s_hi[wave + w][el + i]);
                }
    }
    if (writes && there) {
        const int64_t off = paged_index(c, page, h) * D + el;      // (exact: the values are of the type)
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint2 *>(c.k_min + 2 * off) = make_uint2(pack_bf16x2(l[0], l[1]), pack_bf16x2(l[2], l[3]));
            *reinterpret_cast<uint2 *>(c.k_max + 2 * off) = make_uint2(pack_bf16x2(u[0], u[1]), pack_bf16x2(u[2], u[3]));
        } else {
            *reinterpret_cast<float2 *>(c.k_min + 4 * off) = make_float2(l[0], l[1]);
            *reinterpret_cast<float2 *>(c.k_max + 4 * off) = make_float2(u[0], u[1]);
        }
    }
}

template <typename T, typename TQ, int D, bool ROT>
static hipError_t launch_append(const PagedAppendArgs &a, hipStream_t stream) {
    constexpr int WAVES = kAppThreads / kWave;
    constexpr int RPW = kWave / (D / (2 * Shape<T>::E));      // rows of a wavefront's pass
    AppendGrid g;
    // wavefronts of a page: two passes each, up to all four (32768 tokens in pages of 16 rows 153 us, with one pass each 160; merged rows in pages of 64 36.1 us, with four
    // 39.1; a token of 64 sequences in pages of 32 4.75 us, with four 4.5)
    g.log2_waves = 0;
    while (g.log2_waves < 2 && (2 * RPW << g.log2_waves) < a.c.R) ++g.log2_waves;
    const int pages = WAVES >> g.log2_waves, slots = paged_append_slots(a.N, a.c.R, a.c.P);
    g.page_groups = (slots + pages - 1) / pages;
    // Near: 32768 tokens 158 -> 152 us, merged rows 37.3 -> 35.8 (angles from one chiplet's cache, neighbouring rows of a projection read together); with
    // few pages there would be chiplets without work.  (The queries' workgroups too: 157.)
    const int64_t kv_items = (int64_t)a.c.B * g.page_groups;
    g.kv_near = kv_items >= kNearItems;
    g.kv_blocks = (int)paged_share_ids(kv_items, a.c.H, g.kv_near != 0);
    query_grid<TQ, D>(a, g);
    const unsigned blocks = (unsigned)g.kv_blocks + (unsigned)(a.c.B * g.q_tiles * g.q_groups);      // (paged_append_fits)
    hipLaunchKernelGGL((paged_append_kernel<T, TQ, D, ROT>), dim3(blocks), dim3(kAppThreads), 0, stream, a, g);
    return hipGetLastError();
}

template <typename T, int D> static hipError_t launch_append_q(const PagedAppendArgs &a, hipStream_t stream) {
    if (!a.cos_sin) return launch_append<T, T, D, false>(a, stream);
    return a.q_dtype == DType::BF16 ? launch_append<T, bf16_t, D, true>(a, stream) : launch_append<T, float, D, true>(a, stream);
}

hipError_t launch_paged_append(const PagedAppendArgs &a, hipStream_t stream) {
    if (a.c.dtype == DType::BF16) return a.c.d == 128 ? launch_append_q<bf16_t, 128>(a, stream) : launch_append_q<bf16_t, 64>(a, stream);
    return a.c.d == 128 ? launch_append_q<float, 128>(a, stream) : launch_append_q<float, 64>(a, stream);
}

}  // namespace sc
