// sc_paged_append: new rows of keys and values go to the pages of their sequences, rotated by their positions on the way, together with the queries
// of the same tokens; the pages' summaries (minimum and maximum of their keys) follow.
//
//     a' = a cos - b sin,  b' = b cos + a sin   for the pairs (a, b) of the first `rot` elements of a row, in fp32, rounded once.
//
// Bound by bytes: every row is read once and written once, and there are two operations a byte.  A workgroup takes one page of one KV head: all
// the rows that the call adds to that page, and, where summaries are kept, the keys that the page held before, so that no workgroup depends on
// another.  A lane holds two 16-byte (bf16) pieces of a row, chosen so that the partners of a rotation are in the same lane; 8 lanes make a row of
// 128 elements.  The queries are rotated by workgroups of their own, which go over the heads of a group of tokens and read the angles once.
#include "sc_paged.h"

namespace sc {

constexpr int kAppThreads = 256;

// Two pieces of 8 elements of a row, and the angles that turn them.
struct Pieces {
    int ea, eb;       // first elements
    bool turned;
};
template <int D> __device__ __forceinline__ Pieces pieces_of(int j, int rot, bool interleaved) {
    const bool turned = 16 * j < rot;
    const bool halves = turned && !interleaved;      // partners i and i + rot / 2; else neighbours, or elements that stay
    return {halves ? 8 * j : 16 * j, halves ? 8 * j + rot / 2 : 16 * j + 8, turned};
}
__device__ __forceinline__ void turn(float (&x)[8], float (&y)[8], const float (&c)[8], const float (&s)[8], bool interleaved) {
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1], e = y[2 * i], f = y[2 * i + 1];
            x[2 * i] = a * c[i] - b * s[i];
            x[2 * i + 1] = b * c[i] + a * s[i];
            y[2 * i] = e * c[4 + i] - f * s[4 + i];
            y[2 * i + 1] = f * c[4 + i] + e * s[4 + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = x[i], b = y[i];
            x[i] = a * c[i] - b * s[i];
            y[i] = b * c[i] + a * s[i];
        }
    }
}
// a NaN stays
__device__ __forceinline__ float lower(float a, float b) { return (b < a || b != b) ? b : a; }
__device__ __forceinline__ float higher(float a, float b) { return (b > a || b != b) ? b : a; }

template <typename T> __device__ __forceinline__ void rounded(float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const uint32_t u = pack_bf16x2(x[i], x[i + 1]);
            x[i] = bf16_lo(u);
            x[i + 1] = bf16_hi(u);
        }
    }
}

struct AppendGrid {
    int slots;            // pages that a sequence can touch
    int kv_blocks;
    int q_tiles, q_groups, q_heads;      // of tokens, of heads, heads of a group
};

template <typename T, typename TQ, int D>
__global__ __launch_bounds__(kAppThreads) void paged_append_kernel(PagedAppendArgs p, AppendGrid g) {
    constexpr int LPR = D / 16;
    constexpr int RPP = kAppThreads / LPR;      // rows of a pass
    const int tid = threadIdx.x;
    const int j = tid % LPR, r = tid / LPR;
    const PagedView &c = p.c;
    const Pieces at = pieces_of<D>(j, p.rot, p.interleaved != 0);
    const int half = p.rot / 2;

    if ((int)blockIdx.x >= g.kv_blocks) {
        // ---- queries: a tile of tokens, the heads of a group
        int id = (int)blockIdx.x - g.kv_blocks;
        const int group = id % g.q_groups;
        id /= g.q_groups;
        const int tile = id % g.q_tiles, b = id / g.q_tiles;
        const int n = tile * RPP + r;
        if (n >= p.N) return;
        const int64_t pos = (int64_t)(p.positions ? p.positions[b] : p.base_lens[b]) + n;
        const bool known = pos >= 0 && pos < p.max_position;
        float co[8], si[8];
        if (at.turned && known) {
            load8(p.cos_sin + pos * p.rot + 8 * j, co);
            load8(p.cos_sin + pos * p.rot + half + 8 * j, si);
        }
        const int h1 = min((group + 1) * g.q_heads, p.Hq);
        for (int h = group * g.q_heads; h < h1; ++h) {
            const TQ *src = reinterpret_cast<const TQ *>(p.Q + b * p.q_b + h * p.q_h + n * p.q_n);
            TQ *dst = reinterpret_cast<TQ *>(p.Q_out + b * p.o_b + h * p.o_h + n * p.o_n);
            float x[8], y[8];
            load8(src + at.ea, x);
            load8(src + at.eb, y);
            if (!known) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = y[i] = __builtin_nanf("");
            } else if (at.turned) {
                turn(x, y, co, si, p.interleaved != 0);
            }
            store8(dst + at.ea, x);
            store8(dst + at.eb, y);
        }
        return;
    }

    // ---- keys and values: one page of one KV head
    int id = (int)blockIdx.x;
    const int h = id % c.H;
    id /= c.H;
    const int slot = id % g.slots, b = id / g.slots;
    const int li = p.per_head ? b * c.H + h : b;
    const int base = p.base_lens[li];
    const int fresh = p.new_lens ? p.new_lens[li] : p.N;
    const int64_t pos0 = p.positions ? p.positions[b] : base;
    const PagedAppendPlan plan = paged_append_plan(base, fresh, p.N, c.P, c.log2_R, p.cos_sin != nullptr, pos0, p.max_position);
    const int32_t *table = paged_table(c, b, h);
    if (slot == 0 && (p.per_head || h == 0)) {
        // the length of the sequence (and head): -1 if any page that it needs is not there
        int bad = 0;
        const int heads = (c.table_per_head && !p.per_head) ? c.H : 1;      // pages of their own, one length
        for (int k = 0; k < heads; ++k)
            for (int i = plan.first + tid; i <= plan.last; i += kAppThreads) bad |= paged_bad(c, table[(int64_t)k * c.P + i]);
        bad = __syncthreads_or(bad);
        if (tid == 0) p.lens[li] = (plan.ok && !bad) ? base + fresh : -1;
    }
    const int place = plan.first + slot;
    if (place > plan.last) return;
    const int page = table[place];
    if (paged_bad(c, page)) return;
    const int64_t row0 = (int64_t)place << c.log2_R;       // row of the sequence at the page's start
    const int r0 = (int)max((int64_t)base - row0, (int64_t)0), r1 = (int)min((int64_t)base + fresh - row0, (int64_t)c.R);
    char *kp = c.K + paged_offset(c, page, h), *vp = c.V + paged_offset(c, page, h);
    const bool summary = c.k_min != nullptr;
    float lo[16], hi[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
    for (int row = (summary ? 0 : r0 / RPP * RPP) + r; row < r1; row += RPP) {
        T *kd = reinterpret_cast<T *>(kp + (int64_t)row * c.row_bytes);
        float x[8], y[8];
        if (row < r0) {
            if (!summary) continue;
            load8(kd + at.ea, x);
            load8(kd + at.eb, y);
        } else {
            const int64_t n = row0 + row - base;
            const T *ks = reinterpret_cast<const T *>(p.K + b * p.k_b + h * p.k_h + n * p.k_n);
            const T *vs = reinterpret_cast<const T *>(p.V + b * p.v_b + h * p.v_h + n * p.v_n);
            T *vd = reinterpret_cast<T *>(vp + (int64_t)row * c.row_bytes);
            float u[8], w[8];
            load8(ks + at.ea, x);
            load8(ks + at.eb, y);
            load8(vs + at.ea, u);
            load8(vs + at.eb, w);
            if (at.turned) {
                float co[8], si[8];
                load8(p.cos_sin + (pos0 + n) * p.rot + 8 * j, co);
                load8(p.cos_sin + (pos0 + n) * p.rot + half + 8 * j, si);
                turn(x, y, co, si, p.interleaved != 0);
            }
            store8(kd + at.ea, x);
            store8(kd + at.eb, y);
            store8(vd + at.ea, u);
            store8(vd + at.eb, w);
            if (c.counts && j == 0) c.counts[paged_index(c, page, h) * c.R + row] = p.counts[((int64_t)b * c.H + h) * p.N + n];
            if (summary) {      // of the keys as stored
                rounded<T>(x);
                rounded<T>(y);
            }
        }
        if (summary) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lo[i] = lower(lo[i], x[i]);
                hi[i] = higher(hi[i], x[i]);
                lo[8 + i] = lower(lo[8 + i], y[i]);
                hi[8 + i] = higher(hi[8 + i], y[i]);
            }
        }
    }
    if (!summary) return;
    // ---- the lanes with the same pieces, then the wavefronts
    __shared__ float s_lo[kAppThreads / kWave][D], s_hi[kAppThreads / kWave][D];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int off = LPR; off < kWave; off <<= 1) {
            lo[i] = lower(lo[i], __shfl_xor(lo[i], off, kWave));
            hi[i] = higher(hi[i], __shfl_xor(hi[i], off, kWave));
        }
    }
    if (tid % kWave < LPR) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = i < 8 ? at.ea + i : at.eb + i - 8;
            s_lo[tid / kWave][e] = lo[i];
            s_hi[tid / kWave][e] = hi[i];
        }
    }
    __syncthreads();
    if (tid < D) {
        float a = s_lo[0][tid], e = s_hi[0][tid];
#pragma unroll
        for (int w = 1; w < kAppThreads / kWave; ++w) {
            a = lower(a, s_lo[w][tid]);
            e = higher(e, s_hi[w][tid]);
        }
        const int64_t off = paged_index(c, page, h) * D + tid;
        if constexpr (sizeof(T) == 2) {      // exact: the values are bf16
            reinterpret_cast<uint16_t *>(c.k_min)[off] = (uint16_t)(__float_as_uint(a) >> 16);
            reinterpret_cast<uint16_t *>(c.k_max)[off] = (uint16_t)(__float_as_uint(e) >> 16);
        } else {
            reinterpret_cast<float *>(c.k_min)[off] = a;
            reinterpret_cast<float *>(c.k_max)[off] = e;
        }
    }
}

template <typename T, typename TQ, int D>
static hipError_t launch_append(const PagedAppendArgs &a, hipStream_t stream) {
    constexpr int RPP = kAppThreads / (D / 16);
    AppendGrid g;
    g.slots = paged_append_slots(a.N, a.c.R, a.c.P);
    g.kv_blocks = a.c.B * a.c.H * g.slots;
    g.q_tiles = (a.N + RPP - 1) / RPP;
    g.q_heads = 4;
    g.q_groups = a.Q ? (a.Hq + g.q_heads - 1) / g.q_heads : 0;
    const unsigned blocks = (unsigned)g.kv_blocks + (unsigned)(a.c.B * g.q_tiles * g.q_groups);      // (paged_append_fits)
    hipLaunchKernelGGL((paged_append_kernel<T, TQ, D>), dim3(blocks), dim3(kAppThreads), 0, stream, a, g);
    return hipGetLastError();
}

template <typename T, typename TQ> static hipError_t launch_append_d(const PagedAppendArgs &a, hipStream_t stream) {
    return a.c.d == 128 ? launch_append<T, TQ, 128>(a, stream) : launch_append<T, TQ, 64>(a, stream);
}

hipError_t launch_paged_append(const PagedAppendArgs &a, hipStream_t stream) {
    if (a.c.dtype == DType::BF16)
        return a.q_dtype == DType::BF16 ? launch_append_d<bf16_t, bf16_t>(a, stream) : launch_append_d<bf16_t, float>(a, stream);
    return a.q_dtype == DType::BF16 ? launch_append_d<float, bf16_t>(a, stream) : launch_append_d<float, float>(a, stream);
}

}  // namespace sc
