// sc_paged_select: the pages of every (sequence, KV head) whose keys can come closest to its queries.
//     score(page) = max over the G heads of  sum_e max(q_e k_min_e, q_e k_max_e) = max over heads of (q+ . k_max + q- . k_min),  q+ = max(q, 0), q- = min(q, 0):
// no key between the page's bounds has a larger product with any of the queries.
//
// Two kernels.  The scores, bound by the summaries' bytes (2 d elements a page and head), are two products on the fp64 matrix cores (16 pages x 16 heads,
// v_mfma_f64_16x16x4_f64): the products of two bf16 numbers are exact in fp64 and their sums very nearly so, and the choice between two pages is
// that of exact arithmetic unless they are some 1e-13 apart.  (Sums in fp32 would choose another page than an exact evaluation in a few calls of a
// hundred, and which one would depend on the order of the sum.)  Then one workgroup per (sequence, KV head) finds the key of the last page to keep, eight bits at a time, and
// writes the places in order.
#include "sc_paged.h"

namespace sc {

typedef double sel_f64x4 __attribute__((ext_vector_type(4)));

struct PagSelParams {
    PagedView c;
    const void *Q;
    int G;
    const int32_t *lens;
    int lens_per_head;
    int keep, first, recent;
    int32_t *sel, *sel_lens;
    unsigned long long *keys;      // [B * H][P]
    int tiles;                     // workgroups per (sequence, KV head) of the scores
};

constexpr int kScoreThreads = 256;
constexpr int kScorePages = 16 * (kScoreThreads / kWave);
constexpr int kSelThreads = 1024;
// keys in the order of the scores: forced pages above what is not a number, above every number
constexpr unsigned long long kKeyForced = ~0ull, kKeyNaN = ~0ull - 1;

__device__ __forceinline__ unsigned long long score_key(double x) {
    if (x != x) return kKeyNaN;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, x + 0.0);      // (one zero)
    return (u >> 63) ? ~u : u | (1ull << 63);
}
__device__ __forceinline__ int held_pages(const PagSelParams &p, int64_t bh, int b) {
    const int len = min(max(p.lens[p.lens_per_head ? bh : b], 0), p.c.P << p.c.log2_R);
    return (len + p.c.R - 1) >> p.c.log2_R;
}
// 16 bytes as 8 (bf16) or 4 (fp32) numbers
__device__ __forceinline__ void widen(const uint4 &v, float (&x)[8]) {
    x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
    x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
}
__device__ __forceinline__ void widen(const uint4 &v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
}
template <int N> __device__ __forceinline__ void query_piece(const bf16_t *q, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __uint_as_float((uint32_t)q[i].bits << 16);
}
template <int N> __device__ __forceinline__ void query_piece(const float *q, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = q[i];
}

template <typename T, typename TQ, int D>
__global__ __launch_bounds__(kScoreThreads) void paged_score_kernel(PagSelParams p) {
    constexpr int E = 16 / (int)sizeof(T);            // elements of 16 bytes
    constexpr int KL = D / (4 * E);                   // pieces of a row per lane: 4 lanes share a row
    const PagedView &cv = p.c;
    const int64_t bh = blockIdx.x / p.tiles;
    const int tile = (int)(blockIdx.x - bh * p.tiles);
    const int b = (int)(bh / cv.H), h = (int)(bh - (int64_t)b * cv.H);
    const int lane = threadIdx.x % kWave, g = lane / 16, c = lane % 16;
    const int place = tile * kScorePages + 16 * (int)(threadIdx.x / kWave) + c;      // the lane's page: column c of the products
    const int pages = held_pages(p, bh, b);
    if (place - c >= pages) return;
    const int page = place < pages ? paged_table(cv, b, h)[place] : 0;
    const bool there = place < pages && !paged_bad(cv, page);
    const int64_t row = paged_index(cv, there ? page : 0, h) * D;
    uint4 lo[KL], hi[KL];
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) {
        lo[ks] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(cv.k_min) + row + E * (4 * ks + g));
        hi[ks] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(cv.k_max) + row + E * (4 * ks + g));
    }
    // rows of the products: query heads; those behind the group are its last one again and do not change the maximum
    const TQ *q = reinterpret_cast<const TQ *>(p.Q) + (bh * p.G + min(c, p.G - 1)) * D;
    sel_f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) {
        float x[E], l[E], u[E];
        query_piece<E>(q + E * (4 * ks + g), x);
        widen(lo[ks], l);
        widen(hi[ks], u);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            // (a NaN in a query goes through either product)
            acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(x[i] < 0.f ? 0.f : x[i]), (double)u[i], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(x[i] > 0.f ? 0.f : x[i]), (double)l[i], acc, 0, 0, 0);
        }
    }
    // the maximum over the heads: over the registers, and over the lanes that share the page (whatever row is where)
    double best = acc[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) best = (acc[i] > best || acc[i] != acc[i]) ? acc[i] : best;
#pragma unroll
    for (int off = 16; off < kWave; off <<= 1) {
        const double other = __shfl_xor(best, off, kWave);
        best = (other > best || other != other) ? other : best;
    }
    if (g == 0 && place < pages) {
        unsigned long long key = there ? score_key(best) : kKeyNaN;
        if (place < p.first || place >= pages - p.recent) key = kKeyForced;
        p.keys[bh * cv.P + place] = key;
    }
}

__global__ __launch_bounds__(kSelThreads) void paged_select_kernel(PagSelParams p) {
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / p.c.H);
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int n = held_pages(p, bh, b), keep = p.keep;
    int32_t *sel = p.sel + bh * keep;
    if (tid == 0) p.sel_lens[bh] = min(n, keep);
    if (n <= keep) {
        for (int i = tid; i < keep; i += kSelThreads) sel[i] = i < n ? i : -1;
        return;
    }
    const unsigned long long *keys = p.keys + bh * p.c.P;
    // ---- the key of rank keep, from the top eight bits down
    __shared__ int hist[256];
    __shared__ int s_digit, s_need;
    unsigned long long prefix = 0, mask = 0;
    int need = keep;      // of the keys that agree with the prefix
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kSelThreads) {
            const unsigned long long k = keys[i];
            if ((k & mask) == prefix) atomicAdd(&hist[(int)(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (wave == 0) {      // lane i: digits 255 - 4 i .. 252 - 4 i
            int v[4], sum = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) { v[t] = hist[255 - 4 * lane - t]; sum += v[t]; }
            int before = sum;
#pragma unroll
            for (int off = 1; off < kWave; off <<= 1) {
                const int t = __shfl_up(before, off, kWave);
                before += lane >= off ? t : 0;
            }
            before -= sum;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (before < need && before + v[t] >= need) { s_digit = 255 - 4 * lane - t; s_need = need - before; }
                before += v[t];
            }
        }
        __syncthreads();
        prefix |= (unsigned long long)s_digit << shift;
        mask |= 255ull << shift;
        need = s_need;
        __syncthreads();
    }
    // ---- the places, ascending: keys above it, and the first `need` of those equal to it
    __shared__ int s_above[kSelThreads / kWave], s_equal[kSelThreads / kWave];
    int above0 = 0, equal0 = 0;      // before this stretch of kSelThreads pages
    for (int i0 = 0; i0 < n; i0 += kSelThreads) {
        const unsigned long long k = i0 + tid < n ? keys[i0 + tid] : 0ull;
        const bool is_above = i0 + tid < n && k > prefix, is_equal = i0 + tid < n && k == prefix;
        const uint64_t ba = ballot64(is_above), be = ballot64(is_equal);
        if (lane == 0) { s_above[wave] = __popcll(ba); s_equal[wave] = __popcll(be); }
        __syncthreads();
        int above = above0, equal = equal0;
        for (int w = 0; w < kSelThreads / kWave; ++w) {
            above += w < wave ? s_above[w] : 0;
            equal += w < wave ? s_equal[w] : 0;
            above0 += s_above[w];
            equal0 += s_equal[w];
        }
        const uint64_t below = (1ull << lane) - 1;
        above += __popcll(ba & below);
        equal += __popcll(be & below);
        if (is_above || (is_equal && equal < need)) sel[above + min(equal, need)] = i0 + tid;
        __syncthreads();
    }
}

size_t paged_select_bytes(int B, int H, int P) { return align_up((size_t)B * H * P * sizeof(unsigned long long), 256); }

template <typename T, typename TQ, int D> static void launch_score(const PagSelParams &p, hipStream_t stream) {
    hipLaunchKernelGGL((paged_score_kernel<T, TQ, D>), dim3((unsigned)((int64_t)p.tiles * p.c.B * p.c.H)), dim3(kScoreThreads), 0, stream, p);
}
template <typename T, typename TQ> static void launch_score_d(const PagSelParams &p, hipStream_t stream) {
    if (p.c.d == 128) launch_score<T, TQ, 128>(p, stream);
    else launch_score<T, TQ, 64>(p, stream);
}

hipError_t launch_paged_select(const PagedSelectArgs &a, hipStream_t stream) {
    PagSelParams p;
    p.c = a.c;
    p.Q = a.Q; p.G = a.Hq / a.c.H;
    p.lens = a.lens; p.lens_per_head = a.lens_per_head;
    p.keep = a.keep; p.first = a.first; p.recent = a.recent;
    p.sel = a.sel; p.sel_lens = a.sel_lens;
    p.keys = reinterpret_cast<unsigned long long *>(reinterpret_cast<char *>(a.ws) + paged_state_bytes());
    p.tiles = (a.c.P + kScorePages - 1) / kScorePages;
    const bool qb = a.q_dtype == DType::BF16;
    if (a.c.dtype == DType::BF16) {
        if (qb) launch_score_d<bf16_t, bf16_t>(p, stream);
        else launch_score_d<bf16_t, float>(p, stream);
    } else {
        if (qb) launch_score_d<float, bf16_t>(p, stream);
        else launch_score_d<float, float>(p, stream);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_select_kernel, dim3((unsigned)(a.c.B * a.c.H)), dim3(kSelThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace sc
