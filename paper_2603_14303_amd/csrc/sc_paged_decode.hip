// sc_paged_decode_attn: attention of one new token of every sequence over a cache held in pages.
//     O = softmax(q K^T scale + ln s) V   per (sequence, query head); the G <= 16 query heads of a KV head together, so that its rows are read once.
//
// Work.  Bound by bytes: 4 G operations for every 2 bytes of a row.  The rows of all (sequence, KV head) pairs are cut into units of kUnit rows and
// laid end to end; every workgroup takes an equal stretch of them, whatever lengths they come from (a ragged batch with a fixed number of splits
// per head waits for its longest sequence).  The lengths are on the device, so every workgroup adds them up by itself.  A head that lies within one
// workgroup's stretch is stored directly.  Otherwise every workgroup that holds a part of it leaves a partial result (running maximum, sum, fp32
// sums) in the workspace and counts itself off at the head's counter; the one that comes last joins the partial results.  Nobody waits.
//
// Step.  A wavefront takes 16 rows at a time, always of one page.  Keys are loaded as the first product wants them (lane (g, c) of the wavefront's
// 4 x 16 lanes: row c, 16 bytes at 64 ks + 16 g), values as the second one does (rows 4 g + i).  The scores leave the first product with lane (g, c)
// holding head c, rows 4 g + i: the second product's own layout, so the probabilities never move.  Softmax is online, in the exp2 domain.  bf16:
// v_mfma_f32_16x16x32_bf16 and v_mfma_f32_16x16x16_bf16, probabilities as two bf16 parts (a rounding of 2^-18; one part would put 2^-9 of each weight
// into the result, as much as its own rounding); fp32 queries over a bf16 cache as three parts, as are their probabilities; fp32 caches: v_mfma_f32_16x16x4_f32.
#include <type_traits>

#include "sc_paged.h"

namespace sc {

constexpr int kPagWaves = 6;
constexpr int kPagThreads = kPagWaves * kWave;
constexpr int kUnit = 16 * kPagWaves;        // rows of a unit: one step of every wavefront
constexpr int kMaxWgs = 512;                 // two workgroups of six wavefronts on each of the 256 compute units
constexpr int kPagPad = 4;                   // floats behind the sums of a partial result: maximum, sum, two unused
constexpr int kMaxHeadWgs = 64;              // workgroups per (sequence, KV head) at most, on average: each is a partial result to join
constexpr float kPagLog2e = 1.4426950408889634f;
constexpr float kPagLn2 = 0.6931471805599453f;

typedef float pag_f32x4 __attribute__((ext_vector_type(4)));
typedef short pag_short4 __attribute__((ext_vector_type(4)));
typedef __bf16 pag_bf16x8 __attribute__((ext_vector_type(8)));

struct PagDecParams {
    PagedView c;
    const void *Q;
    int q_is_bf16, G;
    const int32_t *lens;
    int lens_per_head;
    const int32_t *sel, *sel_lens;
    int keep;
    float scale_log2;
    void *O;
    int o_is_bf16;
    float *lse;
    int *counter;        // [B * H] workgroups that have left their part of a head
    float *part;         // [2 * kMaxWgs][G][D + kPagPad]: a workgroup's first stretch and its last one
    int wgs;             // workgroups of the launch
};

__device__ __forceinline__ float pag_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// rows of entry e: of sequence e, or of (sequence, KV head) e where lengths or a selection are per head
__device__ __forceinline__ int pag_rows(const PagDecParams &p, int e) {
    if (p.sel) return min(max(p.sel_lens[e], 0), p.keep) << p.c.log2_R;      // the rows of whole pages; those behind the length are masked
    return min(max(p.lens[e], 0), p.c.P << p.c.log2_R);
}
__device__ __forceinline__ int pag_units(int rows) { return paged_units(rows, kUnit); }

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) x += __shfl_xor(x, off, kWave);
    return x;
}

// x as NP bf16 parts whose sum it is (up to the last one's rounding)
template <int NP> __device__ __forceinline__ void split_bf16(float x0, float x1, uint32_t (&part)[NP]) {
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        part[k] = pack_bf16x2(x0, x1);
        x0 -= bf16_lo(part[k]);
        x1 -= bf16_hi(part[k]);
    }
}

// What a wavefront holds of 16 rows: KL pieces of 16 bytes a lane of keys; VL registers of values per row of the lane.
template <typename T, int D> struct Rows {
    static constexpr int KL = D * (int)sizeof(T) / 64;
    static constexpr int VW = D * (int)sizeof(T) / 64;      // dwords of a row of values that a lane holds: (4 of its rows) x (16 lanes a row)
    uint4 k[KL];
    uint32_t v[4][VW];
    int32_t n[4];
};

template <typename T, int D> __device__ __forceinline__ void load_keys(Rows<T, D> &x, const char *k, int row_bytes, int g, int c) {
    const char *at = k + (uint32_t)(c * row_bytes + 16 * g);
#pragma unroll
    for (int ks = 0; ks < Rows<T, D>::KL; ++ks) x.k[ks] = load16_stream(at + 64 * ks);
}
template <typename T, int D> __device__ __forceinline__ void load_values(Rows<T, D> &x, const char *v, int row_bytes, int g, int c) {
    constexpr int VW = Rows<T, D>::VW;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const char *at = v + (uint32_t)((4 * g + i) * row_bytes);
        if constexpr (VW == 2) {
            const uint2 t = *reinterpret_cast<const uint2 *>(at + 8 * c);
            x.v[i][0] = t.x;
            x.v[i][1] = t.y;
        } else {
#pragma unroll
            for (int q = 0; q < VW / 4; ++q) {
                const uint4 t = load16_stream(at + 256 * q + 16 * c);
                x.v[i][4 * q] = t.x;
                x.v[i][4 * q + 1] = t.y;
                x.v[i][4 * q + 2] = t.z;
                x.v[i][4 * q + 3] = t.w;
            }
        }
    }
}

// The accumulators of lane (g, c): acc[a][i] is head 4 g + i, element acc_element(a, c).
template <typename T, int D> struct Acc {
    static constexpr int N = D / 16;
    static __device__ __forceinline__ int element(int a, int c) {
        if constexpr (sizeof(T) == 2) return (D / 16) * c + a;      // 2 VW neighbouring elements
        else return 64 * (a / 4) + 4 * c + a % 4;
    }
};

// QP: parts of the queries (bf16 caches)
template <typename T, int D, int QP>
__global__ __launch_bounds__(kPagThreads) void paged_decode_kernel(PagDecParams p) {
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr int KL = Rows<T, D>::KL, VW = Rows<T, D>::VW, NA = Acc<T, D>::N;
    constexpr int PP = QP == 1 ? 2 : 3;       // parts of the probabilities (bf16)
    constexpr int kStride = D + kPagPad;
    const PagedView &cv = p.c;
    const int G = p.G;
    const int tid = threadIdx.x, lane = tid % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int g = lane / 16, c = lane % 16;
    const int wg = blockIdx.x;

    __shared__ __attribute__((aligned(16))) float s_acc[kPagWaves * 16 * D];
    __shared__ float s_m[kPagWaves][16], s_l[kPagWaves][16];
    __shared__ int s_last;

    // ---- my stretch of all units: every wavefront adds up the lengths, 64 at a time
    const bool per_head = p.sel != nullptr || p.lens_per_head != 0;
    const int entries = per_head ? cv.B * cv.H : cv.B, weight = per_head ? 1 : cv.H;
    int total = 0;
    for (int e0 = 0; e0 < entries; e0 += kWave) total += (e0 + lane < entries) ? pag_units(pag_rows(p, e0 + lane)) * weight : 0;
    total = wave_sum(total);
    const int per = (total + p.wgs - 1) / p.wgs;
    int pos = wg * per;
    const int stop = min(pos + per, total);
    if (pos >= total) return;
    int e = 0, cum = 0;      // entry that holds unit `pos`, and the units before it
    for (int e0 = 0;; e0 += kWave) {
        const int mine = (e0 + lane < entries) ? pag_units(pag_rows(p, e0 + lane)) * weight : 0;
        int incl = mine;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int t = __shfl_up(incl, off, kWave);
            incl += lane >= off ? t : 0;
        }
        const uint64_t beyond = ballot64(cum + incl > pos);
        if (beyond) {
            const int k = first_bit(beyond);
            e = e0 + k;
            cum += __shfl(incl - mine, k, kWave);
            break;
        }
        cum += __shfl(incl, kWave - 1, kWave);
    }
    e = __builtin_amdgcn_readfirstlane(e);
    cum = __builtin_amdgcn_readfirstlane(cum);
    int rows = pag_rows(p, e), units = pag_units(rows);
    int b, h;
    if (per_head) {
        b = e / cv.H;
        h = e - b * cv.H;
    } else {
        b = e;
        h = (pos - cum) / units;
    }
    int a = per_head ? cum : cum + h * units;       // unit at which the head starts

    while (true) {
        const int64_t bh = (int64_t)b * cv.H + h;
        const int end = min(a + units, stop);
        const int r0 = (pos - a) * kUnit, r1 = min((end - a) * kUnit, rows);
        const int32_t *table = paged_table(cv, b, h);
        const int32_t *sel = p.sel ? p.sel + bh * p.keep : nullptr;
        const int len = min(max(p.lens[p.lens_per_head ? bh : b], 0), cv.P << cv.log2_R);

        // ---- queries: lane (g, c) holds of head c what meets its pieces of a key; heads beyond the group are zero
        uint4 q[QP][KL];
        {
            const int64_t q0 = (((int64_t)b * cv.H + h) * G + c) * D;
#pragma unroll
            for (int ks = 0; ks < KL; ++ks) {
#pragma unroll
                for (int k = 0; k < QP; ++k) q[k][ks] = make_uint4(0u, 0u, 0u, 0u);
                if (c < G) {
                    if constexpr (kBf16 && QP == 1) {
                        q[0][ks] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const bf16_t *>(p.Q) + q0 + 32 * ks + 8 * g);
                    } else if constexpr (kBf16) {
                        float x[8];
                        load8(reinterpret_cast<const float *>(p.Q) + q0 + 32 * ks + 8 * g, x);
                        uint32_t w[4][QP];
#pragma unroll
                        for (int i = 0; i < 4; ++i) split_bf16<QP>(x[2 * i], x[2 * i + 1], w[i]);
#pragma unroll
                        for (int k = 0; k < QP; ++k) q[k][ks] = make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
                    } else if (p.q_is_bf16) {
                        const uint2 t = *reinterpret_cast<const uint2 *>(reinterpret_cast<const bf16_t *>(p.Q) + q0 + 16 * ks + 4 * g);
                        q[0][ks] = make_uint4(t.x << 16, t.x & 0xffff0000u, t.y << 16, t.y & 0xffff0000u);
                    } else {
                        q[0][ks] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const float *>(p.Q) + q0 + 16 * ks + 4 * g);
                    }
                }
            }
        }

        pag_f32x4 acc[NA];
#pragma unroll
        for (int i = 0; i < NA; ++i) acc[i] = pag_f32x4{0.f, 0.f, 0.f, 0.f};
        float m_run = -INFINITY, l_run = 0.f;
        bool bad = false;

        // ---- pages: lane i knows the page of the wavefront's step s0 + i and how many of the step's rows are there
        const int first = r0 + 16 * wave;
        const int steps = first < r1 ? (r1 - first + kUnit - 1) / kUnit : 0;
        int my_page = 0, my_left = 0;
        auto look_up = [&](int s0) {
            my_page = my_left = 0;
            if (s0 + lane < steps) {
                const PagedStep t = paged_step(first + (s0 + lane) * kUnit, cv.log2_R, len, cv.P, cv.num_pages, table, sel != nullptr, sel);
                my_page = t.page;
                my_left = t.left;
                bad |= t.bad;
            }
        };
        Rows<T, D> x;
        int left = 0, in_page = 0;
        int64_t off = 0, idx = 0;
        auto step_at = [&](int s) {
            if (s % kWave == 0) look_up(s);
            const int page = __builtin_amdgcn_readlane(my_page, s % kWave);
            left = __builtin_amdgcn_readlane(my_left, s % kWave);
            in_page = (first + s * kUnit) & (cv.R - 1);
            off = paged_offset(cv, page, h) + (int64_t)in_page * cv.row_bytes;
            idx = paged_index(cv, page, h) * cv.R + in_page;
        };
        auto load_sizes = [&]() {
            if (cv.counts) {
                const int4 t = *reinterpret_cast<const int4 *>(cv.counts + idx + 4 * g);
                x.n[0] = t.x; x.n[1] = t.y; x.n[2] = t.z; x.n[3] = t.w;
            }
        };
        if (steps > 0) {
            step_at(0);
            load_keys<T, D>(x, cv.K + off, cv.row_bytes, g, c);
            load_sizes();
            load_values<T, D>(x, cv.V + off, cv.row_bytes, g, c);
        }
        for (int s = 0; s < steps; ++s) {
            const int here = left;
            pag_f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KL; ++ks) {
                if constexpr (kBf16) {
#pragma unroll
                    for (int k = QP - 1; k >= 0; --k)      // the smallest part first
                        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pag_bf16x8, x.k[ks]), __builtin_bit_cast(pag_bf16x8, q[k][ks]), sc, 0, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(dword_of(x.k[ks], i)), __uint_as_float(dword_of(q[0][ks], i)), sc, 0, 0, 0);
                }
            }
            float sv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sv[i] = sc[i] * p.scale_log2;
                if (cv.counts) sv[i] = x.n[i] > 0 ? sv[i] + __log2f((float)x.n[i]) : -INFINITY;
                if (4 * g + i >= here) sv[i] = -INFINITY;
            }
            const bool more = s + 1 < steps;
            if (more) {
                step_at(s + 1);
                load_keys<T, D>(x, cv.K + off, cv.row_bytes, g, c);
                load_sizes();
            }
            float m_loc = m_run;
#pragma unroll
            for (int i = 0; i < 4; ++i) m_loc = fmaxf(m_loc, sv[i]);
            const float m_new = rows_allreduce_max(m_loc);
            const float m_safe = (m_new == -INFINITY) ? 0.f : m_new;
            const float alpha = pag_exp2(m_run - m_safe);
            float pi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) pi[i] = pag_exp2(sv[i] - m_safe);
            l_run = fmaf(l_run, alpha, (pi[0] + pi[1]) + (pi[2] + pi[3]));      // of the lane's own rows; added up behind the loop
            m_run = m_new;
            if (ballot64(alpha != 1.0f) != 0ull) {
                float al[4];      // the factor of head 4 g + i is in the lanes (.., 4 g + i)
#pragma unroll
                for (int i = 0; i < 4; ++i) al[i] = lane_gather(alpha, 20 * g + i);
#pragma unroll
                for (int k = 0; k < NA; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[k][i] *= al[i];
            }
            if (here < 16) {      // what lies behind the last row is not looked at (it may be anything, and 0 times a NaN is one)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int w = 0; w < VW; ++w) x.v[i][w] = 4 * g + i < here ? x.v[i][w] : 0u;
            }
            if constexpr (kBf16) {
                uint32_t p01[PP], p23[PP];
                split_bf16<PP>(pi[0], pi[1], p01);
                split_bf16<PP>(pi[2], pi[3], p23);
#pragma unroll
                for (int k = 0; k < NA; ++k) {
                    const uint32_t lo = (k & 1) ? pack_hi(x.v[0][k / 2], x.v[1][k / 2]) : pack_lo(x.v[0][k / 2], x.v[1][k / 2]);
                    const uint32_t hi = (k & 1) ? pack_hi(x.v[2][k / 2], x.v[3][k / 2]) : pack_lo(x.v[2][k / 2], x.v[3][k / 2]);
                    const pag_short4 bb = __builtin_bit_cast(pag_short4, make_uint2(lo, hi));
#pragma unroll
                    for (int t = PP - 1; t >= 0; --t)
                        acc[k] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(pag_short4, make_uint2(p01[t], p23[t])), bb, acc[k], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int k = 0; k < NA; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(pi[i], __uint_as_float(x.v[i][k]), acc[k], 0, 0, 0);
            }
            if (more) load_values<T, D>(x, cv.V + off, cv.row_bytes, g, c);
        }

        // ---- join the wavefronts
        float lw = rows_allreduce_sum(l_run);
        if (ballot64(bad) != 0ull) lw = __builtin_nanf("");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int hh = 4 * g + i;
            if (hh < G) {
#pragma unroll
                for (int k = 0; k < NA; ++k) s_acc[(wave * G + hh) * D + Acc<T, D>::element(k, c)] = acc[k][i];
            }
        }
        if (g == 0) { s_m[wave][c] = m_run; s_l[wave][c] = lw; }
        __syncthreads();
        const bool whole = pos == a && end == a + units;      // nobody else has a part of the head
        const int w0 = paged_first_wg(a, per), w1 = paged_last_wg(a, units, per);
        float *mine = p.part + (int64_t)paged_place(wg, a, per) * G * kStride;
        for (int i = tid; i < G * D; i += kPagThreads) {
            const int hh = i / D, el = i - hh * D;
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < kPagWaves; ++w) m = fmaxf(m, s_m[w][hh]);
            const float m_safe = (m == -INFINITY) ? 0.f : m;
            float o = 0.f, l = 0.f;
#pragma unroll
            for (int w = 0; w < kPagWaves; ++w) {
                const float f = pag_exp2(s_m[w][hh] - m_safe);
                o = fmaf(s_acc[(w * G + hh) * D + el], f, o);
                l = fmaf(s_l[w][hh], f, l);
            }
            if (whole) {
                const int64_t row = bh * G + hh;
                const float out = o * (l != 0.f ? 1.0f / l : 0.f);
                if (p.o_is_bf16) reinterpret_cast<uint16_t *>(p.O)[row * D + el] = (uint16_t)pack_bf16x2(out, out);
                else reinterpret_cast<float *>(p.O)[row * D + el] = out;
                if (el == 0 && p.lse) p.lse[row] = l != 0.f ? (m + __log2f(l)) * kPagLn2 : -INFINITY;
            } else {
                float *dst = mine + hh * kStride;
                __hip_atomic_store(dst + el, o, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (el == 0) {
                    __hip_atomic_store(dst + D, m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __hip_atomic_store(dst + D + 1, l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
            }
        }
        if (!whole) {
            // every wavefront's partial results are acknowledged by memory before the workgroup counts itself off
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) {
                const int before = __hip_atomic_fetch_add(p.counter + bh, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = before == w1 - w0;
            }
            __syncthreads();
            if (s_last) {
                if (tid == 0) __hip_atomic_store(p.counter + bh, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                for (int i = tid; i < G * D; i += kPagThreads) {
                    const int hh = i / D, el = i - hh * D;
                    float m = -INFINITY, o = 0.f, l = 0.f;
                    for (int w = w0; w <= w1; ++w) {
                        const float *src = p.part + ((int64_t)paged_place(w, a, per) * G + hh) * kStride;
                        const float ow = __hip_atomic_load(src + el, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        const float mw = __hip_atomic_load(src + D, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        const float lw2 = __hip_atomic_load(src + D + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        const float m2 = fmaxf(m, mw);
                        const float safe = (m2 == -INFINITY) ? 0.f : m2;
                        const float f0 = pag_exp2(m - safe), f1 = pag_exp2(mw - safe);
                        o = fmaf(ow, f1, o * f0);
                        l = fmaf(lw2, f1, l * f0);
                        m = m2;
                    }
                    const int64_t row = bh * G + hh;
                    const float out = o * (l != 0.f ? 1.0f / l : 0.f);
                    if (p.o_is_bf16) reinterpret_cast<uint16_t *>(p.O)[row * D + el] = (uint16_t)pack_bf16x2(out, out);
                    else reinterpret_cast<float *>(p.O)[row * D + el] = out;
                    if (el == 0 && p.lse) p.lse[row] = l != 0.f ? (m + __log2f(l)) * kPagLn2 : -INFINITY;
                }
            }
        }
        // ---- the next head of the stretch
        pos = end;
        if (pos >= stop) return;
        __syncthreads();      // the wavefronts' sums have been read
        a += units;
        ++h;
        if (h == cv.H) { h = 0; ++b; }
        if (per_head || h == 0) {
            ++e;
            rows = pag_rows(p, e);
            units = pag_units(rows);
        }
    }
}

// ------------------------------------------------------------------------------------------------
size_t paged_state_bytes(int B, int H) { return align_up((size_t)B * H * sizeof(int), 256); }
size_t paged_decode_bytes(int G, int d) { return align_up((size_t)2 * kMaxWgs * G * (d + kPagPad) * sizeof(float), 256); }

template <typename T, int D, int QP> static hipError_t launch_k(const PagDecParams &p, hipStream_t stream) {
    hipLaunchKernelGGL((paged_decode_kernel<T, D, QP>), dim3((unsigned)p.wgs), dim3(kPagThreads), 0, stream, p);
    return hipGetLastError();
}
template <typename T, int QP> static hipError_t launch_d(const PagDecParams &p, hipStream_t stream) {
    return p.c.d == 128 ? launch_k<T, 128, QP>(p, stream) : launch_k<T, 64, QP>(p, stream);
}

hipError_t launch_paged_decode(const PagedDecodeArgs &a, hipStream_t stream) {
    PagDecParams p;
    p.c = a.c;
    p.Q = a.Q; p.q_is_bf16 = a.q_dtype == DType::BF16; p.G = a.Hq / a.c.H;
    p.lens = a.lens; p.lens_per_head = a.lens_per_head;
    p.sel = a.sel; p.sel_lens = a.sel_lens; p.keep = a.keep;
    p.scale_log2 = a.scale * kPagLog2e;
    p.O = a.O; p.o_is_bf16 = a.o_dtype == DType::BF16; p.lse = a.lse;
    p.counter = reinterpret_cast<int *>(a.ws);
    p.part = reinterpret_cast<float *>(reinterpret_cast<char *>(a.ws) + paged_state_bytes(a.c.B, a.c.H));
    // never more workgroups than the tables (the selections) have units for, nor than a head's partial results are worth
    const int64_t heads = (int64_t)a.c.B * a.c.H;
    const int64_t most = ((int64_t)(a.sel ? a.keep : a.c.P) * a.c.R + kUnit - 1) / kUnit * heads;
    int64_t wgs = kMaxWgs < heads * kMaxHeadWgs ? kMaxWgs : heads * kMaxHeadWgs;
    if (wgs > most) wgs = most;
    p.wgs = (int)wgs;
    if (a.c.dtype == DType::BF16) return p.q_is_bf16 ? launch_d<bf16_t, 1>(p, stream) : launch_d<bf16_t, 3>(p, stream);
    return launch_d<float, 1>(p, stream);
}

}  // namespace sc
