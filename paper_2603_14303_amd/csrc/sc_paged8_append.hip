// sc_paged8_append: new rows of keys and values go to pages of 8-bit codes, rotated by their positions on the way, together with the queries of the same tokens.
//
//     s = max(s_old, the smallest power of two with max |x| <= Q s)   over the new rows of a block of rows and head, s_old if it holds rows;  Q = 448 (e4m3), 127 (int8)
//     code = round(x / s),   codes that are there: round(code * (s_old / s)) where s has grown
//
// A scale that is a power of two costs int8 up to one bit and e4m3 nothing (its steps are relative), and it makes growing harmless: halving steps k times is off by less than
// one final step in all, however many appends it took, and e4m3 loses bits only at the lower end of its range.  Rounded once, from fp32, ties to even.
//
// Bound by bytes: a row is read once, in its own type, and written as one byte an element.  One to four wavefronts take one block of one KV head and keep its new rows in
// registers between the search for the largest number and the rounding.  No other workgroup touches the block, so nothing waits and nothing depends on an order.
//
// Measured (d = 128, from bf16): a prompt of 32768 tokens, 8 KV and 32 query heads: 145 to 153 us by card (5.2 to 4.9 TB/s; a copy of 4 GiB: 5.3 to 4.9); a token of each of 64 sequences 5.3 us, of which the launch is 1.8: lengths, page, scale and store
// follow each other.
#include "sc_paged_rows.h"

namespace sc {

struct Paged8Codes {
    float *k_scale, *v_scale;      // [page][head][R >> log2_block]
    int log2_block, e4m3;
};

// The formula is held to its roundings: a product that is fused with a sum moves numbers that lie next to a border between two codes.
template <int E> __device__ __forceinline__ void turn_rounded(float (&x)[E], float (&y)[E], const float (&c)[E], const float (&s)[E], bool interleaved) {
#pragma clang fp contract(off)
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1], e = y[2 * i], f = y[2 * i + 1];
            x[2 * i] = a * c[i] - b * s[i];
            x[2 * i + 1] = b * c[i] + a * s[i];
            y[2 * i] = e * c[E / 2 + i] - f * s[E / 2 + i];
            y[2 * i + 1] = f * c[E / 2 + i] + e * s[E / 2 + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float a = x[i], b = y[i];
            x[i] = a * c[i] - b * s[i];
            y[i] = b * c[i] + a * s[i];
        }
    }
}

// `bits` of the largest |x|: those of an infinity or more (a NaN) give NaN
__device__ __forceinline__ float smallest_scale(uint32_t bits, bool e4m3) {
    if (bits >= 0x7f800000u) return __builtin_nanf("");
    const int over = (bits & 0x7fffffu) > (e4m3 ? 0x600000u : 0x7e0000u) ? 1 : 0;      // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
    const int e = max((int)(bits >> 23) - (e4m3 ? 8 : 6) + over, 1);
    return __uint_as_float((uint32_t)e << 23);
}
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }      // a NaN stays

__device__ __forceinline__ uint32_t encode4(const float *x, float f, bool e4m3) {
    if (e4m3) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, lo, true);
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)(int)fminf(fmaxf(__builtin_rintf(x[i] * f), -127.f), 127.f);      // (beyond 127 only under a scale of the caller's)
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
}
__device__ __forceinline__ void decode4(uint32_t w, float *x, bool e4m3) {
    if (e4m3) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
    } else {
        x[0] = (float)(int8_t)w; x[1] = (float)(int8_t)(w >> 8); x[2] = (float)(int8_t)(w >> 16); x[3] = (float)((int32_t)w >> 24);
    }
}

// T: type of the rows that arrive.  RW: rows of a wavefront
template <typename T, int D, bool ROT, int RW>
__global__ __launch_bounds__(kAppThreads) void paged8_append_kernel(PagedAppendArgs p, AppendGrid g, Paged8Codes q) {
    constexpr int WAVES = kAppThreads / kWave;
    constexpr int E = Shape<T>::E, LPR = D / (2 * E), RPW = kWave / LPR, PASSES = RW / RPW;
    static_assert(PASSES >= 1, "a pass has no more rows than a wavefront");
    const PagedView &c = p.c;
    if (ROT && (int)blockIdx.x >= g.kv_blocks) {
        if (p.q_dtype == DType::BF16) rotate_queries<bf16_t, D>(p, g, (int)blockIdx.x - g.kv_blocks);
        else rotate_queries<float, D>(p, g, (int)blockIdx.x - g.kv_blocks);
        return;
    }
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int j = lane % LPR;
    const Pieces at = pieces_of<E>(j, p.rot, p.interleaved != 0);
    const PagedShare at_work = paged_share((int)blockIdx.x, c.H, g.kv_near != 0);
    const int h = at_work.share, group = at_work.item % g.page_groups, b = at_work.item / g.page_groups;
    if (b >= c.B) return;
    const int wpb = 1 << g.log2_waves, part = wave & (wpb - 1);      // wavefronts of a block
    const int li = p.per_head ? b * c.H + h : b;
    const int base = read_scalar(p.base_lens + li), new_len = read_scalar((p.new_lens ? p.new_lens : p.base_lens) + li);
    const int position = read_scalar(p.positions ? p.positions + b : p.base_lens + li);
    const int fresh = p.new_lens ? new_len : p.N;
    const int64_t pos0 = position;
    const int log2_E = q.log2_block, log2_bpp = c.log2_R - log2_E;      // rows of a block, blocks of a page
    const PagedAppendPlan plan = paged_append_plan(base, fresh, p.N, c.P << log2_bpp, log2_E, p.cos_sin != nullptr, pos0, p.max_position);
    const int32_t *table = paged_table(c, b, h);
    const int place = plan.first + group * (WAVES >> g.log2_waves) + (wave >> g.log2_waves);
    if (group == 0 && (p.per_head || h == 0)) {
        // the length of the sequence (and head): -1 if any page that it needs is not there
        int bad = 0;
        const int heads = (c.table_per_head && !p.per_head) ? c.H : 1;      // pages of their own, one length
        const int last = plan.last < plan.first ? -1 : plan.last >> log2_bpp;
        for (int k = 0; k < heads; ++k)
            for (int i = (plan.first >> log2_bpp) + tid; i <= last; i += kAppThreads) bad |= paged_bad(c, table[(int64_t)k * c.P + i]);
        bad = __syncthreads_or(bad);
        if (tid == 0) p.lens[li] = (plan.ok && !bad) ? base + fresh : -1;
    }
    const int page = place <= plan.last ? read_scalar(table + (place >> log2_bpp)) : -1;
    const bool there = !paged_bad(c, page);
    const int64_t row0 = (int64_t)place << log2_E;       // row of the sequence at the block's start
    const int in_page = (int)(row0 & (c.R - 1));
    const int r0 = (int)max((int64_t)base - row0, (int64_t)0), r1 = there ? (int)min((int64_t)base + fresh - row0, (int64_t)1 << log2_E) : 0;
    const bool work = r1 > r0;                           // of the block's rows [r0, r1) are new, those below r0 are held
    const int64_t off = there ? paged_offset(c, page, h) + (int64_t)in_page * c.row_bytes : 0;
    const int64_t scale_at = there ? (paged_index(c, page, h) << log2_bpp) + (in_page >> log2_E) : 0;
    const bool e4m3 = q.e4m3 != 0;

    // ---- the new rows.  Lanes behind the last one (before the first) read it again: all loads are on their way at once, and the largest number is not changed by it
    float x[PASSES][E], y[PASSES][E];      // keys, after the rotation
    Raw<T> va[PASSES], vb[PASSES];
    float k_old = 0.f, v_old = 0.f;
    uint32_t k_most = 0, v_most = 0;
    if (work) {
        Raw<T> ka[PASSES], kb[PASSES];
        const char *ks = p.K + b * p.k_b + h * p.k_h, *vs = p.V + b * p.v_b + h * p.v_h;
        if (r0 > 0) {
            k_old = q.k_scale[scale_at];
            v_old = q.v_scale[scale_at];
        }
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
            const int64_t n = row0 + min(max(part * RW + u * RPW + lane / LPR, r0), r1 - 1) - base;      // row of the call
            ka[u].load(ks + n * p.k_n + at.ea * (int)sizeof(T));
            kb[u].load(ks + n * p.k_n + at.eb * (int)sizeof(T));
            va[u].load(vs + n * p.v_n + at.ea * (int)sizeof(T));
            vb[u].load(vs + n * p.v_n + at.eb * (int)sizeof(T));
        }
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
            ka[u].widen(x[u]);
            kb[u].widen(y[u]);
            if constexpr (ROT) {
                if (at.turned) {
                    const int64_t n = row0 + min(max(part * RW + u * RPW + lane / LPR, r0), r1 - 1) - base;
                    const float *angles = p.cos_sin + (pos0 + n) * p.rot + E * j;
                    float co[E], si[E];
                    load_angles(angles, co);
                    load_angles(angles + p.rot / 2, si);
                    turn_rounded(x[u], y[u], co, si, p.interleaved != 0);
                }
            }
            float v[E], w[E];
            va[u].widen(v);
            vb[u].widen(w);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                k_most = max(k_most, max(__float_as_uint(x[u][i]) & 0x7fffffffu, __float_as_uint(y[u][i]) & 0x7fffffffu));
                v_most = max(v_most, max(__float_as_uint(v[i]) & 0x7fffffffu, __float_as_uint(w[i]) & 0x7fffffffu));
            }
        }
        k_most = (uint32_t)wave_max((int)k_most);
        v_most = (uint32_t)wave_max((int)v_most);
    }
    __shared__ uint32_t s_most[2][WAVES];
    if (wpb > 1) {
        if (lane == 0) {
            s_most[0][wave] = k_most;
            s_most[1][wave] = v_most;
        }
        __syncthreads();
        for (int w = wave - part; w < wave - part + wpb; ++w) {
            k_most = max(k_most, s_most[0][w]);
            v_most = max(v_most, s_most[1][w]);
        }
    }
    if (!work) return;
    float k_scale = smallest_scale(k_most, e4m3), v_scale = smallest_scale(v_most, e4m3);
    if (r0 > 0) {
        k_scale = larger(k_scale, k_old);
        v_scale = larger(v_scale, v_old);
    }
    char *kp = c.K + off, *vp = c.V + off;
    // ---- the rows that are there, in the new steps
    if (r0 > 0 && (k_scale > k_old || v_scale > v_old)) {
        const float kf = k_old / k_scale, vf = v_old / v_scale;      // (a factor of one changes nothing)
        for (int t = part * RPW + lane / LPR; t < r0; t += RPW << g.log2_waves) {
#pragma unroll
            for (int i = 0; i < 2 * E; i += 4) {
                const int64_t o = (int64_t)t * c.row_bytes + (i < E ? at.ea + i : at.eb + i - E);
                float z[4];
                if (k_scale > k_old) {
                    decode4(*reinterpret_cast<const uint32_t *>(kp + o), z, e4m3);
                    *reinterpret_cast<uint32_t *>(kp + o) = encode4(z, kf, e4m3);
                }
                if (v_scale > v_old) {
                    decode4(*reinterpret_cast<const uint32_t *>(vp + o), z, e4m3);
                    *reinterpret_cast<uint32_t *>(vp + o) = encode4(z, vf, e4m3);
                }
            }
        }
    }
    const float kf = 1.0f / k_scale, vf = 1.0f / v_scale;
    const int32_t *sizes = p.counts + ((int64_t)b * c.H + h) * p.N;
    int32_t *counts = c.counts + paged_index(c, page, h) * c.R + in_page;
#pragma unroll
    for (int u = 0; u < PASSES; ++u) {
        const int t = part * RW + u * RPW + lane / LPR;
        if (t >= r0 && t < r1) {
            float v[E], w[E];
            va[u].widen(v);
            vb[u].widen(w);
            const int64_t o = (int64_t)t * c.row_bytes;
            if constexpr (E == 8) {
                *reinterpret_cast<uint2 *>(kp + o + at.ea) = make_uint2(encode4(x[u], kf, e4m3), encode4(x[u] + 4, kf, e4m3));
                *reinterpret_cast<uint2 *>(kp + o + at.eb) = make_uint2(encode4(y[u], kf, e4m3), encode4(y[u] + 4, kf, e4m3));
                *reinterpret_cast<uint2 *>(vp + o + at.ea) = make_uint2(encode4(v, vf, e4m3), encode4(v + 4, vf, e4m3));
                *reinterpret_cast<uint2 *>(vp + o + at.eb) = make_uint2(encode4(w, vf, e4m3), encode4(w + 4, vf, e4m3));
            } else {
                *reinterpret_cast<uint32_t *>(kp + o + at.ea) = encode4(x[u], kf, e4m3);
                *reinterpret_cast<uint32_t *>(kp + o + at.eb) = encode4(y[u], kf, e4m3);
                *reinterpret_cast<uint32_t *>(vp + o + at.ea) = encode4(v, vf, e4m3);
                *reinterpret_cast<uint32_t *>(vp + o + at.eb) = encode4(w, vf, e4m3);
            }
            if (c.counts && j == 0) counts[t] = sizes[row0 + t - base];
        }
    }
    if (part == 0 && lane == 0) {
        q.k_scale[scale_at] = k_scale;
        q.v_scale[scale_at] = v_scale;
    }
}

template <typename T, int D, bool ROT, int RW>
static hipError_t launch_append8(const PagedAppendArgs &a, const Paged8Codes &q, hipStream_t stream) {
    constexpr int WAVES = kAppThreads / kWave;
    AppendGrid g;
    const int block = 1 << q.log2_block;
    g.log2_waves = block >= 64 ? 2 : block == 32 ? 1 : 0;
    const int blocks = WAVES >> g.log2_waves, slots = paged_append_slots(a.N, block, a.c.P << (a.c.log2_R - q.log2_block));
    g.page_groups = (slots + blocks - 1) / blocks;
    const int64_t kv_items = (int64_t)a.c.B * g.page_groups;
    g.kv_near = kv_items >= kNearItems;
    g.kv_blocks = (int)paged_share_ids(kv_items, a.c.H, g.kv_near != 0);
    if (a.q_dtype == DType::BF16) query_grid<bf16_t, D>(a, g);
    else query_grid<float, D>(a, g);
    const unsigned wgs = (unsigned)g.kv_blocks + (unsigned)(a.c.B * g.q_tiles * g.q_groups);      // (paged_append_fits)
    hipLaunchKernelGGL((paged8_append_kernel<T, D, ROT, RW>), dim3(wgs), dim3(kAppThreads), 0, stream, a, g, q);
    return hipGetLastError();
}
template <typename T, int D> static hipError_t launch_append8_d(const PagedAppendArgs &a, const Paged8Codes &q, hipStream_t stream) {
    if (q.log2_block <= 6) return a.cos_sin ? launch_append8<T, D, true, 16>(a, q, stream) : launch_append8<T, D, false, 16>(a, q, stream);
    return a.cos_sin ? launch_append8<T, D, true, 32>(a, q, stream) : launch_append8<T, D, false, 32>(a, q, stream);
}

hipError_t launch_paged8_append(const PagedAppendArgs &a, const Paged8View &v, hipStream_t stream) {
    const Paged8Codes q = {v.k_scale, v.v_scale, v.log2_block, v.code == 1};
    if (a.c.dtype == DType::BF16) return a.c.d == 128 ? launch_append8_d<bf16_t, 128>(a, q, stream) : launch_append8_d<bf16_t, 64>(a, q, stream);
    return a.c.d == 128 ? launch_append8_d<float, 128>(a, q, stream) : launch_append8_d<float, 64>(a, q, stream);
}

}  // namespace sc
