// sc_paged_decode_attn: attention of one new token of every sequence over a cache held in pages.
//     O = softmax(q K^T scale + ln s) V   per (sequence, query head); the G <= 16 query heads of a KV head together, so that its rows are read once.
//
// Work.  Bound by bytes: 4 G operations for every 2 bytes of a row.  The rows of all (sequence, KV head) pairs are cut into units of a step's rows and
// laid end to end; every workgroup takes an equal stretch of them, whatever lengths they come from (a ragged batch with a fixed number of splits
// per head waits for its longest sequence).  The lengths are on the device, so every workgroup adds them up by itself.  A head that lies within one
// workgroup's stretch is stored directly.  Otherwise every workgroup that holds a part of it leaves a partial result (running maximum, sum, fp32
// sums) in the workspace and counts itself off; the one that comes last joins the partial results.  Nobody waits.
//
// Step.  A wavefront takes 16 rows at a time, always of one page.  Keys are loaded as the first product wants them (lane (g, c) of the wavefront's
// 4 x 16 lanes: row c, 16 bytes at 64 ks + 16 g), values as the second one does (rows 4 g + i).  The scores leave the first product with lane (g, c)
// holding head c, rows 4 g + i: the second product's own layout, so the probabilities never move.  Softmax is online, in the exp2 domain.  bf16:
// v_mfma_f32_16x16x32_bf16 and v_mfma_f32_16x16x16_bf16, probabilities as three bf16 parts, which hold all bits of fp32 (two parts, a rounding of 2^-18, are not
// faster: 8 heads x 32768 rows 27.9 us with either, 170 rows 6.6 and 6.5); fp32 queries over a bf16 cache as three parts, too; fp32 caches: v_mfma_f32_16x16x4_f32.
//
// Measured (d = 128, bf16): 8 heads x 32768 rows, G = 4: 27.4 us (4.9 TB/s; 18 us of it the rows, 7.4 TB/s); 128 heads of 8192 to 16384 rows, G = 7: 128 us
// from a graph (6.3 TB/s), 131 called one after another; 8 heads x 170 rows: 6.6 us, x 1 row 5.5, of which the launch is 1.8: arguments, lengths, page numbers, rows and the results' store follow each other.
// 8-bit codes, the same ragged heads (4 of 32 sequences), G = 7, pages of 64 rows: e4m3 74 us (5.5 TB/s), int8 78, with fp32 queries 82; bound by instructions as much as by bytes.  A window of 4096 of bf16 rows, 256 heads, G = 4: 85 us (6.3 TB/s).
#include <type_traits>

#include "sc_paged.h"

namespace sc {

constexpr int kPagWaves = 8;
constexpr int kPagThreads = kPagWaves * kWave;
// What a cache holds: T is float, bf16_t, or one of the 8-bit codes below.  A wavefront takes kSub times 16 rows a step: 8-bit rows are half as long as bf16's, and as
// many bytes have to be under way.
struct e4m3_t { uint8_t bits; };
struct i8_t { int8_t value; };
template <typename T> constexpr int kSub = sizeof(T) == 1 ? 2 : 1;
template <typename T> constexpr int kStep = 16 * kSub<T> * kPagWaves;        // rows of a step of all wavefronts: the unit of work
// steps up to which a head goes to one workgroup, if there is one for every head: 8 heads of 170 and 250 rows (two steps) 6.6 and 7.4 us, 8.2 and 8.3 split; of 400
// and 512 rows (four) 8.8 and 10.5 alone, 8.4 and 8.7 split
constexpr int kAlone = 2;
// steps beyond an equal share for which workgroups have parts of one head only: 64 heads of 3000 to 6000 rows 32.4 us, 33.0 with 0; but 24 of 9000 27.0 and 26.4, 128 of
// 1500 to 3000 33.6 and 32.9 (with 4 36.1)
constexpr int kMore = 2;
constexpr int kMaxWgs = 256;                 // one on each compute unit
constexpr int kMaxPairs = 512;              // (part, head) pairs that are joined at once, heads up to a power of two (paged_group)
constexpr int kPagPad = 4;                   // floats behind the sums of a partial result: maximum, sum, two unused
// workgroups per (sequence, KV head) at most, on average.  It only says something for up to three heads in all.  One head of 9000, 32768 and 131072 rows, G = 4: 11.5,
// 17.4 and 39 us; with 32 12.0, 22.6 and 64.  More workgroups would be faster yet (256: 11.0, 12.6 and 20), although each leaves a partial result to join.
constexpr int kMaxHeadWgs = 64;
constexpr float kPagLog2e = 1.4426950408889634f;
constexpr float kPagLn2 = 0.6931471805599453f;

typedef float pag_f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int pag_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int pag_u32x2 __attribute__((ext_vector_type(2)));
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
    int *counter;        // [2][2 * kMaxWgs] workgroups that have left their part of a head (of a group of parts), groups that have been joined; by the first one's place
    float *part;         // [2 * kMaxWgs][G][D + kPagPad]: a workgroup's first stretch and its last one
    int wgs;             // workgroups of the launch
    int window, sinks;   // (WIN) rows from len - window on and rows below `sinks` attend
    const float *k_scale, *v_scale;      // (8-bit codes) [page][head][R >> log2_block]
    int log2_block;
};

// a value that all lanes agree on, kept in a scalar register (what a division or a conversion gives is in a vector register otherwise, and every
// branch on it is one on lanes)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float readlane(float x, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane)); }
__device__ __forceinline__ float inverse_of(int y) { return __builtin_amdgcn_rcpf((float)y); }
__device__ __forceinline__ float pag_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// x as NP bf16 parts, the upper 8 bits of what is left each time: three hold all bits of fp32.  (Rounded parts would, too, but the first one of a number beyond
// bf16's largest is infinity.)
template <int NP> __device__ __forceinline__ void split_bf16(float x0, float x1, uint32_t (&part)[NP]) {
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        part[k] = pack_hi(__float_as_uint(x0), __float_as_uint(x1));
        x0 -= bf16_lo(part[k]);
        x1 -= bf16_hi(part[k]);
    }
}

// Two rounded parts, off by 2^-17 of x: for numbers that end in a bf16 result
__device__ __forceinline__ void split_bf16_rounded(float x0, float x1, uint32_t (&part)[2]) {
    part[0] = pack_bf16x2(x0, x1);
    part[1] = pack_bf16x2(x0 - bf16_lo(part[0]), x1 - bf16_hi(part[0]));
}

// What a wavefront holds of 16 rows: KL pieces of 16 bytes a lane of keys; VL registers of values per row of the lane.
template <typename T, int D> struct Rows {
    static constexpr int KL = D * (int)sizeof(T) / 64;
    static constexpr int VW = D * (int)sizeof(T) / 64;      // dwords of a row of values that a lane holds: (4 of its rows) x (16 lanes a row)
    uint4 k[KL];
    uint32_t v[4][VW];
    int32_t n[4];
};

// Rows come through buffer descriptors that begin at the step's first row and end behind the last one that attends: what lies behind reads as zeros
// (it may be anything in memory, and 0 times a NaN is one), a step without rows asks nothing of memory, and the lane's offsets are 32-bit and the same
// for every step.
typedef __amdgpu_buffer_rsrc_t pag_rsrc;
__device__ __forceinline__ pag_rsrc rows_at(const char *p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p), (short)0, bytes, 0x00020000); }
constexpr int kAuxNt = 2;          // buffer cache policy: read once by this launch
template <typename T, int D> __device__ __forceinline__ void load_keys(Rows<T, D> &x, pag_rsrc k, int lane_offset) {
#pragma unroll
    for (int ks = 0; ks < Rows<T, D>::KL; ++ks) {
        const pag_u32x4 t = __builtin_amdgcn_raw_buffer_load_b128(k, lane_offset + 64 * ks, 0, kAuxNt);
        x.k[ks] = make_uint4(t.x, t.y, t.z, t.w);
    }
}
template <typename T, int D> __device__ __forceinline__ void load_values(Rows<T, D> &x, pag_rsrc v, int lane_offset, int row_bytes) {
    constexpr int VW = Rows<T, D>::VW;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (VW == 1) {
            x.v[i][0] = __builtin_amdgcn_raw_buffer_load_b32(v, lane_offset + i * row_bytes, 0, kAuxNt);
        } else if constexpr (VW == 2) {
            const pag_u32x2 t = __builtin_amdgcn_raw_buffer_load_b64(v, lane_offset + i * row_bytes, 0, kAuxNt);
            x.v[i][0] = t.x;
            x.v[i][1] = t.y;
        } else {
#pragma unroll
            for (int q = 0; q < VW / 4; ++q) {
                const pag_u32x4 t = __builtin_amdgcn_raw_buffer_load_b128(v, lane_offset + i * row_bytes + 256 * q, 0, kAuxNt);
                x.v[i][4 * q] = t.x;
                x.v[i][4 * q + 1] = t.y;
                x.v[i][4 * q + 2] = t.z;
                x.v[i][4 * q + 3] = t.w;
            }
        }
    }
}

// ---- 8-bit codes as bf16, exactly (e4m3 has three bits behind the point, a whole number up to 128 seven): four codes of a dword in two dwords
template <typename T> __device__ __forceinline__ uint2 widen4(uint32_t w) {
    if constexpr (std::is_same_v<T, e4m3_t>) {
        return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
    } else {
        const float x0 = (float)(int8_t)w, x1 = (float)(int8_t)(w >> 8), x2 = (float)(int8_t)(w >> 16), x3 = (float)((int32_t)w >> 24);
        return make_uint2(pack_hi(__float_as_uint(x0), __float_as_uint(x1)), pack_hi(__float_as_uint(x2), __float_as_uint(x3)));
    }
}
// four dwords (rows) of four codes -> four dwords (columns) of the rows' codes
__device__ __forceinline__ void transpose4(const uint32_t (&r)[4], uint32_t (&c)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), b = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);      // rows 0, 1: columns 0 and 1, 2 and 3
    const uint32_t d = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), e = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
    c[0] = pack_lo(a, d); c[1] = pack_hi(a, d); c[2] = pack_lo(b, e); c[3] = pack_hi(b, e);
}

// The accumulators of lane (g, c): acc[a][i] is head 4 g + i, element acc_element(a, c).
template <typename T, int D> struct Acc {
    static constexpr int N = D / 16;
    static __device__ __forceinline__ int element(int a, int c) {
        if constexpr (sizeof(T) <= 2) return (D / 16) * c + a;      // neighbouring elements
        else return 64 * (a / 4) + 4 * c + a % 4;
    }
};

// ------------------------------------------------------------------------------------------------
// Partial results: [place][head][D + kPagPad] floats, written through to memory and read from there (the workgroups of a head run on chiplets whose
// L2s do not see each other's lines within a kernel).
constexpr int kAuxAgent = 16;      // buffer cache policy: device scope

struct Output {
    void *O;
    int o_is_bf16;
    float *lse;
};
__device__ __forceinline__ void store_result(const Output &p, int64_t row, int D, int e, const float4 &o, float m, float l) {
    const float f = l != 0.f ? 1.0f / l : 0.f;
    store_row4(p.O, p.o_is_bf16, row * D + e, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
    if (e == 0 && p.lse) p.lse[row] = l != 0.f ? (m + __log2f(l)) * kPagLn2 : -INFINITY;
}
template <int D> __device__ __forceinline__ void store_part(__amdgpu_buffer_rsrc_t rs, int at, int e, const float4 &o, float m, float l) {
    const pag_u32x4 t = {__float_as_uint(o.x), __float_as_uint(o.y), __float_as_uint(o.z), __float_as_uint(o.w)};
    __builtin_amdgcn_raw_buffer_store_b128(t, rs, (at + e) * 4, 0, kAuxAgent);
    if (e == 0) {
        const pag_u32x2 w = {__float_as_uint(m), __float_as_uint(l)};
        __builtin_amdgcn_raw_buffer_store_b64(w, rs, (at + D) * 4, 0, kAuxAgent);
    }
}

// Joins n partial results, whose places `place_of` gives, and hands each of the G D / 4 pieces of 16 bytes to `sink` with its head's maximum and sum.
// A thread owns one piece of one head and every NS-th part; all its loads of a pass are on their way before the first is used.
template <int D, typename PlaceOf, typename Sink>
__device__ __forceinline__ void join_parts(int G, __amdgpu_buffer_rsrc_t rs, int n, PlaceOf place_of, int tid, float *s_red, float (*s_weight)[kMaxPairs],
                                           float *s_total, Sink sink) {
    constexpr int QPR = D / 4, kStride = D + kPagPad, PASS = 8;
    constexpr int kNowhere = 0x7FFFFFF0;      // beyond the descriptor: zeros, and no memory traffic
    static_assert(16 * QPR <= kPagThreads, "a thread for every piece");
    const int lane = tid % kWave, wave = uniform(tid / kWave);
    const int log2_G = G > 1 ? 32 - __clz(G - 1) : 0;      // heads of a part, up to a power of two
    const int pieces = G * QPR;
    const float pieces_inverse = inverse_of(pieces);
    const int NS = min(uniform(paged_quotient(kPagThreads, pieces, pieces_inverse)), n);
    const int sg = paged_quotient(tid, pieces, pieces_inverse), piece = tid - sg * pieces;
    const bool worker = sg < NS;
    const int hh = piece / QPR, e = 4 * (piece - hh * QPR);
    float *s_m = s_weight[0], *s_l = s_weight[1];
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = 0; k0 < n; k0 += NS * PASS) {
        pag_u32x4 x[PASS];
#pragma unroll
        for (int t = 0; t < PASS; ++t)
            if (k0 + NS * t < n) {
                const int k = k0 + sg + NS * t;
                x[t] = __builtin_amdgcn_raw_buffer_load_b128(rs, worker && k < n ? ((place_of(k) * G + hh) * kStride + e) * 4 : kNowhere, 0, kAuxAgent);
            }
        if (k0 == 0) {      // the weights: a wavefront per head
            for (int i = tid; i < n << log2_G; i += kPagThreads) {
                const int k = i >> log2_G, h2 = i & ((1 << log2_G) - 1);
                const pag_u32x2 t = __builtin_amdgcn_raw_buffer_load_b64(rs, h2 < G ? ((place_of(k) * G + h2) * kStride + D) * 4 : kNowhere, 0, kAuxAgent);
                s_m[i] = __uint_as_float(t.x);
                s_l[i] = __uint_as_float(t.y);
            }
            __syncthreads();
            for (int h2 = wave; h2 < G; h2 += kPagWaves) {
                float m = -INFINITY;
                for (int k = lane; k < n; k += kWave) m = fmaxf(m, s_m[(k << log2_G) + h2]);
                m = rows_allreduce_max(row_allreduce_max(m));
                const float safe = m == -INFINITY ? 0.f : m;
                float l = 0.f;
                for (int k = lane; k < n; k += kWave) {
                    const float f = pag_exp2(s_m[(k << log2_G) + h2] - safe);
                    s_m[(k << log2_G) + h2] = f;
                    l = fmaf(s_l[(k << log2_G) + h2], f, l);
                }
                l = rows_allreduce_sum(row_allreduce_sum<16>(l));
                if (lane == 0) {
                    s_total[h2] = m;
                    s_total[16 + h2] = l;
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < PASS; ++t)
            if (k0 + NS * t < n) {
                const int k = k0 + sg + NS * t;
                const float f = worker && k < n ? s_m[(k << log2_G) + hh] : 0.f;
                o.x = fmaf(__uint_as_float(x[t].x), f, o.x);
                o.y = fmaf(__uint_as_float(x[t].y), f, o.y);
                o.z = fmaf(__uint_as_float(x[t].z), f, o.z);
                o.w = fmaf(__uint_as_float(x[t].w), f, o.w);
            }
    }
    if (NS > 1) {
        if (worker && sg > 0) *reinterpret_cast<float4 *>(s_red + 4 * tid) = o;
        __syncthreads();
        if (sg == 0) {
#pragma unroll 4
            for (int r = 1; r < NS; ++r) {
                const float4 t = *reinterpret_cast<const float4 *>(s_red + 4 * (r * pieces + piece));
                o.x += t.x; o.y += t.y; o.z += t.z; o.w += t.w;
            }
        }
    }
    if (sg == 0) sink(hh, e, o, s_total[hh], s_total[16 + hh]);
}

// a workgroup's results are on their way to memory: waits until they are there, counts the workgroup off, and tells the last of `n` (counter clear again)
__device__ __forceinline__ bool last_of(int *counter, int n, int tid, int *s_last) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // every wavefront: its own stores are acknowledged
    __syncthreads();
    if (tid == 0) {
        const int before = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_last = before == n - 1;
        if (before == n - 1) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return *s_last != 0;
}

// QP: parts of the queries (bf16 caches and codes).  WIN: a window and first rows that stay (p.window, p.sinks; codes always have it); p.sel is NULL then.  PP: parts of the probabilities (bf16 products)
template <typename T, int D, int QP, bool WIN, int PP>
__global__ __launch_bounds__(kPagThreads, 2) void paged_decode_kernel(PagDecParams p) {
    constexpr bool kBf16 = sizeof(T) <= 2;     // products in bf16
    constexpr bool kCodes = sizeof(T) == 1;
    constexpr int NS = kSub<T>, kStep = sc::kStep<T>;
    constexpr int NM = kBf16 ? D / 32 : Rows<T, D>::KL;               // first products a row, pieces of 16 bytes of a query
    constexpr int KL = Rows<T, D>::KL, VW = Rows<T, D>::VW, NA = Acc<T, D>::N;
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
    __shared__ float s_weight[2][kMaxPairs], s_total[32];

    // ---- my stretch of all units: every wavefront adds up the lengths, 64 at a time
    const bool per_head = p.sel != nullptr || p.lens_per_head != 0;
    const int entries = per_head ? cv.B * cv.H : cv.B, weight = per_head ? 1 : cv.H;
    int my_rows = 0, my_len = 0;      // of the lane's entry among the 64 at hand
    // WIN: rows that no step visits, `gap` of them from row `gap_at` on, both multiples of 16
    auto gap_of = [&](int len, int &gap_at) {
        const PagedGap x = paged_gap(len, p.window, p.sinks);
        gap_at = x.at;
        return x.rows;
    };
    auto entry = [&](int e) {
        my_rows = my_len = 0;
        if (e < entries) {
            my_len = min(max(p.lens[p.sel && !p.lens_per_head ? paged_quotient(e, cv.H, inverse_of(cv.H)) : e], 0), cv.P << cv.log2_R);
            my_rows = !WIN && p.sel ? min(max(p.sel_lens[e], 0), p.keep) << cv.log2_R : my_len;      // selected: the rows of whole pages; those behind the length are masked
            if constexpr (WIN) {
                int at;
                my_rows -= gap_of(my_len, at);
            }
        }
    };
    // Units of a head: its steps, rounded up to what a workgroup takes, so that no workgroup has parts of two heads (each costs it a start and a store,
    // as long as some two steps of a chip at work), if that gives no workgroup more than kMore steps beyond an equal share, or if all heads are short.
    // Otherwise every workgroup has its equal share, wherever heads begin in it.
    int total = 0, longest = 0;
    for (int e0 = 0; e0 < entries; e0 += kWave) {
        entry(e0 + lane);
        total += e0 + lane < entries ? paged_units(my_rows, kStep) * weight : 0;
        longest = max(longest, my_rows);
    }
    const int most = paged_units(wave_max(longest), kStep);
    int per, multiple;
    if (most <= kAlone / NS && cv.B * cv.H <= p.wgs) {
        per = multiple = most;
        total = cv.B * cv.H * most;
    } else {
        total = __builtin_amdgcn_readlane(wave_scan(total), kWave - 1);
        const int share = total <= p.wgs ? 1 : uniform((total + p.wgs - 1) / p.wgs);
        per = share;
        multiple = 1;
        for (int t = share; share > 1 && t <= share + kMore / NS; ++t) {
            const float inverse = inverse_of(t);
            int parts = 0;
            for (int e0 = 0; e0 < entries; e0 += kWave) {
                if (entries > kWave) entry(e0 + lane);
                parts += e0 + lane < entries ? paged_parts(paged_units(my_rows, kStep), t, inverse) * weight : 0;
            }
            parts = __builtin_amdgcn_readlane(wave_scan(parts), kWave - 1);
            if (parts <= p.wgs) {
                per = multiple = t;
                total = parts * t;
                break;
            }
        }
    }
    const float per_inverse = inverse_of(per), multiple_inverse = inverse_of(multiple);
    auto units_of = [&](int rows) { return multiple > 1 ? paged_parts(paged_units(rows, kStep), multiple, multiple_inverse) * multiple : paged_units(rows, kStep); };
    const int pos = wg * per;
    const int stop = min(pos + per, total);
    if (pos >= total) return;
    int e0 = 0, e = 0, cum = 0;      // entry that holds unit `pos`, and the units before it
    for (;; e0 += kWave) {
        if (entries > kWave) entry(e0 + lane);      // (else the lane has its entry still)
        const int mine = e0 + lane < entries ? units_of(my_rows) * weight : 0;
        const int incl = wave_scan(mine);
        const uint64_t beyond = ballot64(cum + incl > pos);
        if (beyond) {
            const int k = first_bit(beyond);
            e = e0 + k;
            cum += __builtin_amdgcn_readlane(incl - mine, k);
            break;
        }
        cum += __builtin_amdgcn_readlane(incl, kWave - 1);
    }
    int rows = __builtin_amdgcn_readlane(my_rows, e - e0), len = __builtin_amdgcn_readlane(my_len, e - e0), units = uniform(units_of(rows));
    const int b0 = per_head ? uniform(paged_quotient(e, cv.H, inverse_of(cv.H))) : e;
    int b = b0, h = per_head ? e - b0 * cv.H : uniform(paged_quotient(pos - cum, units, inverse_of(units)));
    int a = per_head ? cum : cum + h * units;       // unit at which the head starts

    // ---- a stretch within one head, and the wavefront's steps in it
    struct Stretch {
        int b, h, a, units, end;           // units [a, a + units) are the head's, the stretch goes to `end`
        int len, first, steps;             // rows of the sequence; the wavefront's first row, its steps (every kStep rows)
        int gap, gap_at;                   // (WIN)
        const int32_t *table, *sel;
    };
    auto stretch_at = [&](int pos) {
        Stretch t;
        t.b = uniform(b);
        t.h = uniform(h);
        t.a = uniform(a);
        t.units = uniform(units);
        t.end = uniform(min(a + units, stop));
        t.len = uniform(len);
        t.first = uniform((pos - a) * kStep + 16 * NS * wave);
        t.gap = t.gap_at = 0;
        if constexpr (WIN) {
            t.gap = uniform(gap_of(len, t.gap_at));
            t.gap_at = uniform(t.gap_at);
        }
        const int r1 = min((t.end - a) * kStep, rows);
        t.steps = uniform(t.first < r1 ? (r1 - t.first + kStep - 1) / kStep : 0);
        t.table = paged_table(cv, b, h);
        t.sel = !WIN && p.sel ? p.sel + ((int64_t)b * cv.H + h) * p.keep : nullptr;
        return t;
    };
    // Lane i knows the page of the i-th 16 rows from step s0 on, how many of them are there, and whether anything is wrong with it; of codes, their scales too
    struct Pages { int page, left, bad; float ks, vs; };
    auto row_of = [&](const Stretch &t, int s, int u) {      // of the sequence
        const int r = t.first + s * kStep + 16 * u;
        return WIN && r >= t.gap_at ? r + t.gap : r;
    };
    auto look_up = [&](const Stretch &t, int s0) {
        Pages x = {0, 0, 0, 0.f, 0.f};
        if (s0 + lane / NS < t.steps) {
            const int row = row_of(t, s0 + lane / NS, lane % NS);
            const PagedStep y = paged_step(row, cv.log2_R, WIN ? paged_window_len(row, t.len, p.window, p.sinks) : t.len, cv.P, cv.num_pages, t.table, !WIN && t.sel != nullptr, t.sel);
            x.page = y.page;
            x.left = y.left;
            x.bad = y.bad;
            if constexpr (kCodes) {
                if (y.left > 0) {
                    const int64_t at = (paged_index(cv, y.page, t.h) << (cv.log2_R - p.log2_block)) + ((row & (cv.R - 1)) >> p.log2_block);
                    x.ks = p.k_scale[at];
                    x.vs = p.v_scale[at];
                }
            }
        }
        return x;
    };
    // Queries: lane (g, c) holds of head c what meets its pieces of a key; heads beyond the group read as zeros
    uint4 q[QP][NM];
    auto load_queries = [&](const Stretch &t) {
        const int qs = p.q_is_bf16 ? 2 : 4;
        const pag_rsrc rows = rows_at(static_cast<const char *>(p.Q) + ((int64_t)t.b * cv.H + t.h) * G * D * qs, G * D * qs);
#pragma unroll
        for (int ks = 0; ks < NM; ++ks) {
            const int el = kCodes ? 64 * (ks / 2) + 16 * g + 8 * (ks % 2) : 32 * ks + 8 * g;      // the lane's elements of a key in this product (bf16)
            if constexpr (kBf16 && QP > 1) {
                const int at = (c * D + el) * 4;
                const pag_u32x4 y0 = __builtin_amdgcn_raw_buffer_load_b128(rows, at, 0, 0), y1 = __builtin_amdgcn_raw_buffer_load_b128(rows, at + 16, 0, 0);
                uint32_t w[4][QP];
                split_bf16<QP>(__uint_as_float(y0.x), __uint_as_float(y0.y), w[0]);
                split_bf16<QP>(__uint_as_float(y0.z), __uint_as_float(y0.w), w[1]);
                split_bf16<QP>(__uint_as_float(y1.x), __uint_as_float(y1.y), w[2]);
                split_bf16<QP>(__uint_as_float(y1.z), __uint_as_float(y1.w), w[3]);
#pragma unroll
                for (int k = 0; k < QP; ++k) q[k][ks] = make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
            } else if (!kBf16 && p.q_is_bf16) {
                const pag_u32x2 y = __builtin_amdgcn_raw_buffer_load_b64(rows, (c * D + 16 * ks + 4 * g) * 2, 0, 0);
                q[0][ks] = make_uint4(y.x << 16, y.x & 0xffff0000u, y.y << 16, y.y & 0xffff0000u);
            } else {
                const pag_u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(rows, kBf16 ? (c * D + el) * 2 : c * D * 4 + 64 * ks + 16 * g, 0, 0);
                q[0][ks] = make_uint4(y.x, y.y, y.z, y.w);
            }
        }
    };
    // The next step is on its way while one is worked on: the registers of the keys are requested anew as soon as the first product has used them, those of
    // the values behind the second, without asking whether there is another step (with a load that is issued or not, the compiler has the next step wait
    // for everything under way).  Two steps ahead were no faster anywhere, and 0.8 us slower with one or two steps (the requests beyond the last).
    Rows<T, D> x[NS];
    const char *values[NS];
    int left[NS];
    const int k_lane = c * cv.row_bytes + 16 * g, v_lane = 4 * g * cv.row_bytes + (VW <= 2 ? 4 * VW : 16) * c;
    const int size_bytes = cv.counts ? 64 : 0;
    auto request_keys = [&](const Stretch &t, Pages &pages, int s) {
        if (NS * s % kWave == 0 && s != 0) {
            const Pages y = look_up(t, s);
            pages = {y.page, y.left, pages.bad | y.bad, y.ks, y.vs};
        }
#pragma unroll
        for (int u = 0; u < NS; ++u) {
            const int page = __builtin_amdgcn_readlane(pages.page, (NS * s + u) % kWave), in_page = row_of(t, s, u) & (cv.R - 1);
            const int64_t off = paged_offset(cv, page, t.h) + (int64_t)in_page * cv.row_bytes;
            left[u] = __builtin_amdgcn_readlane(pages.left, (NS * s + u) % kWave);
            values[u] = cv.V + off;
            load_keys<T, D>(x[u], rows_at(cv.K + off, left[u] * cv.row_bytes), k_lane);
            const char *sizes = reinterpret_cast<const char *>(cv.counts) + (paged_index(cv, page, t.h) * cv.R + in_page) * (int64_t)sizeof(int32_t);
            const pag_u32x4 n = __builtin_amdgcn_raw_buffer_load_b128(rows_at(sizes, left[u] > 0 ? size_bytes : 0), 16 * g, 0, 0);
            x[u].n[0] = (int)n.x; x[u].n[1] = (int)n.y; x[u].n[2] = (int)n.z; x[u].n[3] = (int)n.w;
        }
    };
    auto request_values = [&]() {
#pragma unroll
        for (int u = 0; u < NS; ++u) load_values<T, D>(x[u], rows_at(values[u], left[u] * cv.row_bytes), v_lane, cv.row_bytes);
    };

    Stretch cur = stretch_at(pos);
    load_queries(cur);
    Pages pages = look_up(cur, 0);
    request_keys(cur, pages, 0);
    request_values();
    while (true) {
        const int64_t bh = (int64_t)cur.b * cv.H + cur.h;
        pag_f32x4 acc[NA];
#pragma unroll
        for (int i = 0; i < NA; ++i) acc[i] = pag_f32x4{0.f, 0.f, 0.f, 0.f};
        float m_run = -INFINITY, l_run = 0.f;
        for (int s = 0; s < cur.steps; ++s) {
            int here[NS];
            float sv[4 * NS], vs[NS];      // logits of the lane's rows: 4 g + i of every 16
            int nothing = 0;
#pragma unroll
            for (int u = 0; u < NS; ++u) {
                here[u] = left[u];
                float factor = p.scale_log2;
                vs[u] = 1.f;
                if constexpr (kCodes) {
                    factor *= readlane(pages.ks, (NS * s + u) % kWave);
                    vs[u] = readlane(pages.vs, (NS * s + u) % kWave);
                }
                pag_f32x4 sc = {0.f, 0.f, 0.f, 0.f};
                if constexpr (kBf16) {
                    pag_f32x4 rest = sc;      // of the queries' lower parts
#pragma unroll
                    for (int ks = 0; ks < NM; ++ks) {
                        uint4 key;
                        if constexpr (kCodes) {
                            const uint2 lo = widen4<T>(dword_of(x[u].k[ks / 2], 2 * (ks % 2))), hi = widen4<T>(dword_of(x[u].k[ks / 2], 2 * (ks % 2) + 1));
                            key = make_uint4(lo.x, lo.y, hi.x, hi.y);
                        } else {
                            key = x[u].k[ks];
                        }
                        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pag_bf16x8, key), __builtin_bit_cast(pag_bf16x8, q[0][ks]), sc, 0, 0, 0);
#pragma unroll
                        for (int k = QP - 1; k > 0; --k)
                            rest = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pag_bf16x8, key), __builtin_bit_cast(pag_bf16x8, q[k][ks]), rest, 0, 0, 0);
                    }
                    if constexpr (QP > 1) {      // a lower part that is zero meets an infinite key: the upper parts' sum is infinite, or no number, by itself then
#pragma unroll
                        for (int i = 0; i < 4; ++i) sc[i] += fabsf(rest[i]) < INFINITY ? rest[i] : 0.f;
                    }
                } else {
                    // four sums side by side: one over all d has twice the error (3 x 2 heads of 500 to 1000 rows take 9.0 us with either)
                    pag_f32x4 part[4] = {sc, sc, sc, sc};
#pragma unroll
                    for (int ks = 0; ks < KL; ++ks)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            part[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(dword_of(x[u].k[ks], i)), __uint_as_float(dword_of(q[0][ks], i)), part[i], 0, 0, 0);
                    sc = (part[0] + part[1]) + (part[2] + part[3]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float z = sc[i] * factor;
                    if (cv.counts) z = x[u].n[i] > 0 ? z + __log2f((float)x[u].n[i]) : -INFINITY;
                    if constexpr (!WIN) {
                        if (4 * g + i >= here[u]) z = -INFINITY;
                    }
                    sv[4 * u + i] = z;
                }
                if constexpr (WIN) {      // few steps have rows that do not attend
                    const int row = row_of(cur, s, u);
                    if (!paged_whole(row, cur.len, p.window, p.sinks)) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (4 * g + i >= here[u] || !paged_visible(row + 4 * g + i, cur.len, p.window, p.sinks)) {
                                sv[4 * u + i] = -INFINITY;
                                nothing |= 1 << (4 * u + i);
                            }
                    }
                }
                // rows without weight: their values may be anything, and 0 times a NaN is one
                if (cv.counts) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) nothing |= x[u].n[i] > 0 ? 0 : 1 << (4 * u + i);
                }
            }
            request_keys(cur, pages, s + 1);
            float m_loc = m_run;
#pragma unroll
            for (int i = 0; i < 4 * NS; ++i) m_loc = fmaxf(m_loc, sv[i]);
            const float m_new = rows_allreduce_max(m_loc);
            const float m_safe = (m_new == -INFINITY) ? 0.f : m_new;
            const float alpha = pag_exp2(m_run - m_safe);
            float pi[4 * NS], sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4 * NS; ++i) pi[i] = pag_exp2(sv[i] - m_safe);
#pragma unroll
            for (int u = 0; u < NS; ++u) sum = u == 0 ? (pi[0] + pi[1]) + (pi[2] + pi[3]) : sum + ((pi[4 * u] + pi[4 * u + 1]) + (pi[4 * u + 2] + pi[4 * u + 3]));
            l_run = fmaf(l_run, alpha, sum);      // of the lane's own rows; added up behind the loop
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
            // codes: with the values' scale, before they are split (a scale that is no number must not show where no row of its block attends)
            float pv[4 * NS];
#pragma unroll
            for (int i = 0; i < 4 * NS; ++i) pv[i] = kCodes ? pi[i] * vs[i / 4] : pi[i];
            if (ballot64(nothing != 0) != 0ull) {
                if constexpr (kCodes) {
#pragma unroll
                    for (int i = 0; i < 4 * NS; ++i) pv[i] = nothing >> i & 1 ? 0.f : pv[i];
                }
#pragma unroll
                for (int u = 0; u < NS; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int k = 0; k < VW; ++k) x[u].v[i][k] = nothing >> (4 * u + i) & 1 ? 0u : x[u].v[i][k];
            }
            if constexpr (kCodes) {
                // both 16 rows in one product: place 8 g + j of its inner dimension is row 4 g + j of the first 16, or 4 g + j - 4 of the second
                uint32_t part[4][PP];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (PP == 2) split_bf16_rounded(pv[2 * i], pv[2 * i + 1], part[i]);
                    else split_bf16<PP>(pv[2 * i], pv[2 * i + 1], part[i]);
                }
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    uint32_t col[NS][4];
#pragma unroll
                    for (int u = 0; u < NS; ++u) {
                        const uint32_t r[4] = {x[u].v[0][w], x[u].v[1][w], x[u].v[2][w], x[u].v[3][w]};
                        transpose4(r, col[u]);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint2 lo = widen4<T>(col[0][j]), hi = widen4<T>(col[NS - 1][j]);
                        const pag_bf16x8 bb = __builtin_bit_cast(pag_bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
#pragma unroll
                        for (int t = PP - 1; t >= 0; --t)
                            acc[4 * w + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pag_bf16x8, make_uint4(part[0][t], part[1][t], part[2][t], part[3][t])), bb,
                                                                                     acc[4 * w + j], 0, 0, 0);
                    }
                }
            } else if constexpr (kBf16) {
                uint32_t p01[PP], p23[PP];
                split_bf16<PP>(pi[0], pi[1], p01);
                split_bf16<PP>(pi[2], pi[3], p23);
#pragma unroll
                for (int k = 0; k < NA; ++k) {
                    const uint32_t lo = (k & 1) ? pack_hi(x[0].v[0][k / 2], x[0].v[1][k / 2]) : pack_lo(x[0].v[0][k / 2], x[0].v[1][k / 2]);
                    const uint32_t hi = (k & 1) ? pack_hi(x[0].v[2][k / 2], x[0].v[3][k / 2]) : pack_lo(x[0].v[2][k / 2], x[0].v[3][k / 2]);
                    const pag_short4 bb = __builtin_bit_cast(pag_short4, make_uint2(lo, hi));
#pragma unroll
                    for (int t = PP - 1; t >= 0; --t)
                        acc[k] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(pag_short4, make_uint2(p01[t], p23[t])), bb, acc[k], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int k = 0; k < NA; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(pi[i], __uint_as_float(x[0].v[i][k]), acc[k], 0, 0, 0);
            }
            request_values();
        }
        // ---- the next head of the workgroup's stretch, if any: its first rows are on their way while the results of this one are stored
        const bool more = cur.end < stop;
        Stretch nxt = cur;
        Pages nxt_pages = {0, 0, 0, 0.f, 0.f};
        if (more) {
            a += units;
            ++h;
            if (h == cv.H) { h = 0; ++b; }
            if (per_head || h == 0) {
                ++e;
                if (e - e0 == kWave) {
                    e0 = e;
                    entry(e0 + lane);
                }
                rows = __builtin_amdgcn_readlane(my_rows, e - e0);
                len = __builtin_amdgcn_readlane(my_len, e - e0);
                units = uniform(units_of(rows));
            }
            nxt = stretch_at(cur.end);
            nxt_pages = look_up(nxt, 0);
        }

        const bool bad = ballot64(pages.bad != 0) != 0ull;
        if (more) {
            load_queries(nxt);
            request_keys(nxt, nxt_pages, 0);
            request_values();
        }

        // What only follows is read from the kernel's arguments here, not kept in scalar registers (of which there are too few) from the start
        const auto *tail = (const __attribute__((address_space(4))) PagDecParams *)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(tail));
        const Output out = {tail->O, tail->o_is_bf16, tail->lse};
        const auto rs = __builtin_amdgcn_make_buffer_rsrc(tail->part, (short)0, 2 * kMaxWgs * G * kStride * 4, 0x00020000);
        // ---- join the wavefronts
        float lw = rows_allreduce_sum(l_run);
        if (bad) lw = __builtin_nanf("");
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
        const int w0 = uniform(paged_first_wg(cur.a, per, per_inverse)), w1 = uniform(paged_last_wg(cur.a, cur.units, per, per_inverse));
        const bool whole = w0 == w1;      // nobody else has a part of the head
        const int at = paged_place(wg, cur.a, per) * G * kStride;
        for (int i = tid; i < G * (D / 4); i += kPagThreads) {
            const int hh = i / (D / 4), el = 4 * (i - hh * (D / 4));
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < kPagWaves; ++w) m = fmaxf(m, s_m[w][hh]);
            const float m_safe = (m == -INFINITY) ? 0.f : m;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < kPagWaves; ++w) {
                const float f = pag_exp2(s_m[w][hh] - m_safe);
                const float4 t = *reinterpret_cast<const float4 *>(s_acc + (w * G + hh) * D + el);
                o.x = fmaf(t.x, f, o.x);
                o.y = fmaf(t.y, f, o.y);
                o.z = fmaf(t.z, f, o.z);
                o.w = fmaf(t.w, f, o.w);
                l = fmaf(s_l[w][hh], f, l);
            }
            if (whole) store_result(out, bh * G + hh, D, el, o, m, l);
            else store_part<D>(rs, at + hh * kStride, el, o, m, l);
        }
        if (!whole) {
            // ---- the last of the head's workgroups joins their results; of many, the last of every group first
            const int n = w1 - w0 + 1, group = paged_group(n, G);
            const int k0 = (wg - w0) / group * group, in_group = min(group, n - k0), groups = (n + group - 1) / group;
            auto place_of = [&](int w) { return paged_place(w, cur.a, per); };
            int *counter = tail->counter + place_of(w0 + k0);
            int parts = in_group, from = w0 + k0, by = 1;
            bool result = groups == 1;
            while (last_of(counter, parts, tid, &s_last)) {
                const int to = place_of(from) * G * kStride;
                join_parts<D>(G, rs, parts, [&](int k) { return place_of(from + k * by); }, tid, s_acc, s_weight, s_total, [&](int hh, int el, const float4 &o, float m, float l) {
                    if (result) store_result(out, bh * G + hh, D, el, o, m, l);
                    else store_part<D>(rs, to + hh * kStride, el, o, m, l);
                });
                if (result) break;
                counter = tail->counter + 2 * kMaxWgs + place_of(w0);
                parts = groups;
                from = w0;
                by = group;
                result = true;
            }
        }
        if (!more) return;
        __syncthreads();      // the wavefronts' sums have been read
        cur = nxt;
        pages = nxt_pages;
    }
}

// ------------------------------------------------------------------------------------------------
size_t paged_state_bytes() { return align_up((size_t)4 * kMaxWgs * sizeof(int), 256); }
size_t paged_decode_bytes(int G, int d) { return align_up((size_t)2 * kMaxWgs * G * (d + kPagPad) * sizeof(float), 256); }

template <typename T, int D, int QP, bool WIN> static hipError_t launch_k(const PagDecParams &p, hipStream_t stream) {
    // codes, bf16 results: two parts instead of three and masks only in steps that are not whole: 81 -> 77 us together for 32 x 4 heads of 8192 to 16384 rows, G = 7
    if constexpr (sizeof(T) == 1) {
        if (p.o_is_bf16) {
            hipLaunchKernelGGL((paged_decode_kernel<T, D, QP, WIN, 2>), dim3((unsigned)p.wgs), dim3(kPagThreads), 0, stream, p);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((paged_decode_kernel<T, D, QP, WIN, 3>), dim3((unsigned)p.wgs), dim3(kPagThreads), 0, stream, p);
    return hipGetLastError();
}
template <typename T, int QP, bool WIN> static hipError_t launch_d(const PagDecParams &p, hipStream_t stream) {
    return p.c.d == 128 ? launch_k<T, 128, QP, WIN>(p, stream) : launch_k<T, 64, QP, WIN>(p, stream);
}
template <typename T, bool WIN> static hipError_t launch_q(const PagDecParams &p, hipStream_t stream) {
    if constexpr (sizeof(T) > 2) return launch_d<T, 1, WIN>(p, stream);
    else return p.q_is_bf16 ? launch_d<T, 1, WIN>(p, stream) : launch_d<T, 3, WIN>(p, stream);
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
    p.part = reinterpret_cast<float *>(reinterpret_cast<char *>(a.ws) + paged_state_bytes());
    p.window = a.window; p.sinks = a.sinks;
    p.k_scale = a.k_scale; p.v_scale = a.v_scale; p.log2_block = a.log2_block;
    // never more workgroups than the tables (the selections, the windows) have units for, nor than a head's partial results are worth
    const int64_t heads = (int64_t)a.c.B * a.c.H, unit = a.code ? kStep<e4m3_t> : kStep<float>;
    int64_t rows = (int64_t)(a.sel ? a.keep : a.c.P) * a.c.R;
    if (a.window > 0 && (int64_t)a.window + a.sinks + 48 < rows) rows = (int64_t)a.window + a.sinks + 48;      // (paged_gap: the ends of both stretches are rounded to 16)
    const int64_t most = (rows + unit - 1) / unit * heads;
    int64_t wgs = kMaxWgs < heads * kMaxHeadWgs ? kMaxWgs : heads * kMaxHeadWgs;
    if (wgs > most) wgs = most;
    p.wgs = (int)wgs;
    if (a.code == 1) return launch_q<e4m3_t, true>(p, stream);
    if (a.code == 2) return launch_q<i8_t, true>(p, stream);
    if (a.window > 0) return a.c.dtype == DType::BF16 ? launch_q<bf16_t, true>(p, stream) : launch_q<float, true>(p, stream);
    return a.c.dtype == DType::BF16 ? launch_q<bf16_t, false>(p, stream) : launch_q<float, false>(p, stream);
}

}  // namespace sc
