// sc_paged_select: the pages of every (sequence, KV head) whose keys can come closest to its queries.
//     score(page) = max over the G heads of  sum_e max(q_e k_min_e, q_e k_max_e) = max over heads of (q+ . k_max + q- . k_min),  q+ = max(q, 0), q- = min(q, 0):
// no key between the page's bounds has a larger product with any of the queries.
//
// Two kernels.  The scores are two products on the fp64 matrix cores: the products of two bf16 numbers are exact in fp64 and their sums very nearly so,
// and the choice between two pages is that of exact arithmetic unless they are some 1e-13 apart.  (Sums in fp32 would choose another page than an
// exact evaluation in a few calls of a hundred, and which one would depend on the order of the sum.)  Then one workgroup per (sequence, KV head) finds
// the last page to keep and writes the places in order.  (As one kernel, in which the last workgroup of a head to have written its scores selects:
// 13.7 us with 256 threads and 15.0 with 1024 when these two took 4.9 + 6.5 for 2048 pages x 8 heads; now 4.4 + 5.8.)
#include "sc_paged.h"

namespace sc {

typedef double sel_f64x4 __attribute__((ext_vector_type(4)));

struct PagSelParams {
    PagedView c;
    const void *Q;
    int q_is_bf16, G;
    const int32_t *lens;
    int lens_per_head;
    int keep, first, recent;
    int32_t *sel, *sel_lens;
    unsigned long long *keys;      // [B * H][P]
    int tiles;                     // workgroups per (sequence, KV head) of the scores
};

constexpr int kScoreThreads = 256;
constexpr int kScorePages = 16 * (kScoreThreads / kWave);
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
// element i of 16 bytes of the type
template <typename T> __device__ __forceinline__ double element(const uint4 &v, int i) {
    if constexpr (sizeof(T) == 2) return (double)((i & 1) ? bf16_hi(dword_of(v, i / 2)) : bf16_lo(dword_of(v, i / 2)));
    else return (double)__uint_as_float(dword_of(v, i));
}

// A wavefront has 16 pages, the columns of its products; a lane holds of its page (lane % 16) every fourth piece of 16 bytes.  The heads are the rows, in
// fp64 in shared memory, their positive and their negative parts side by side.  NT: groups of four heads (v_mfma_f64_4x4x4_4b: four products of 4 heads x
// 4 pages), or 0: 16 heads (v_mfma_f64_16x16x4).  us for 2048 pages x 8 heads, G = 4; 1500 pages x 32 heads, G = 7; 2048 pages x 64 heads, G = 16 (d = 128,
// bf16): NT = 1 4.4; NT = 2 5.0 and 8.7; 16 heads 6.4, 12.1 and 24.7; NT = 4 27.0 for the last.  Vector instructions take two to three times as long, also
// with a query's element broadcast over a row of lanes on its way into the multiplication (51 for the last).  The first is a chain of trips to memory.
// The second has the matrix cores busy 30 % of its time and would take 4 us for the bytes, the third 60 %: every workgroup prepares all queries in fp64 for 64 pages,
// and a wavefront reads all of them from shared memory for 16.  With one query head a KV head it is the bytes: 131 MB of
// summaries in 24.6 us.  Products in fp32 with a bound on their error, and an evaluation in fp64 of the pages near the border by the second kernel,
// took 3.9, 6.2 and 14.3 us here and 3 to 5 more there: less in all only with more than eight query heads a KV head and many sequences.
template <typename T, int D, int NT>
__global__ __launch_bounds__(kScoreThreads) void paged_score_kernel(PagSelParams p) {
    constexpr int E = 16 / (int)sizeof(T);            // elements of 16 bytes
    constexpr int KL = D / (4 * E);                   // pieces of a row per lane: 4 lanes share a row
    constexpr int HEADS = NT ? 4 * NT : 16, STRIDE = HEADS + 1;
    // element e of a head: four rows of lanes read four neighbouring pieces at a time, and those lie in banks of their own if a piece is 16 banks more than a
    // multiple of 32 (pieces of four elements are: STRIDE is odd)
    constexpr int PAD = E == 8 ? 4 : 0;
    __shared__ double2 s_q[D * STRIDE + PAD * (D / E)];
    const auto q_place = [](int e, int head) { return e * STRIDE + PAD * (e / E) + head; };
    const PagedView &cv = p.c;
    const unsigned head_of = blockIdx.x / (unsigned)p.tiles;
    const int64_t bh = head_of;
    const int tile = (int)(blockIdx.x - head_of * (unsigned)p.tiles), b = (int)(head_of / (unsigned)cv.H), h = (int)(head_of - (unsigned)b * (unsigned)cv.H);
    const int lane = threadIdx.x % kWave, g = lane / 16, c = lane % 16;
    const int pages = held_pages(p, bh, b);
    if (pages <= p.keep || tile * kScorePages >= pages) return;
    const int place = tile * kScorePages + 16 * (int)(threadIdx.x / kWave) + c;      // the lane's page: column c of the products
    const int page = place < pages ? paged_table(cv, b, h)[place] : 0;
    const bool there = place < pages && !paged_bad(cv, page);
    // heads behind the group are its last one again and do not change the maximum; a thread has PER neighbouring elements of a head
    constexpr int PER = D * HEADS / kScoreThreads, TPH = kScoreThreads / HEADS;
    const int head = threadIdx.x / TPH, e0 = threadIdx.x % TPH * PER;
    const int64_t q_at = (bh * p.G + min(head, p.G - 1)) * D + e0;
    double x[PER];
    if (p.q_is_bf16) {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = load1_f64(reinterpret_cast<const bf16_t *>(p.Q) + q_at + i);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = load1_f64(reinterpret_cast<const float *>(p.Q) + q_at + i);
    }
    const int64_t row = paged_index(cv, there ? page : 0, h) * D;
    uint4 lo[KL], hi[KL];
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) {
        lo[ks] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(cv.k_min) + row + E * (4 * ks + g));
        hi[ks] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(cv.k_max) + row + E * (4 * ks + g));
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) s_q[q_place(e0 + i, head)] = make_double2(x[i] < 0.0 ? 0.0 * x[i] : x[i], x[i] > 0.0 ? 0.0 * x[i] : x[i]);      // (a NaN is in both, and beside infinity)
    __syncthreads();
    double best;
    // several sums side by side: a product takes four times as long as the next one that does not wait for it
    if constexpr (NT > 0) {
        double acc[NT][4] = {};
#pragma unroll
        for (int ks = 0; ks < KL; ++ks)
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const double u = element<T>(hi[ks], i), l = element<T>(lo[ks], i);
                const double2 *q = s_q + q_place(E * (4 * ks + g) + i, lane % 4);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const double2 y = q[4 * t];
                    acc[t][2 * (i % 2)] = __builtin_amdgcn_mfma_f64_4x4x4f64(y.x, u, acc[t][2 * (i % 2)], 0, 0, 0);
                    acc[t][2 * (i % 2) + 1] = __builtin_amdgcn_mfma_f64_4x4x4f64(y.y, l, acc[t][2 * (i % 2) + 1], 0, 0, 0);
                }
            }
        best = (acc[0][0] + acc[0][1]) + (acc[0][2] + acc[0][3]);
#pragma unroll
        for (int t = 1; t < NT; ++t) {
            const double sum = (acc[t][0] + acc[t][1]) + (acc[t][2] + acc[t][3]);
            best = (sum > best || sum != sum) ? sum : best;
        }
    } else {
        sel_f64x4 acc[2] = {{0.0, 0.0, 0.0, 0.0}, {0.0, 0.0, 0.0, 0.0}};
#pragma unroll
        for (int ks = 0; ks < KL; ++ks)
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const double2 y = s_q[q_place(E * (4 * ks + g) + i, c)];
                acc[0] = __builtin_amdgcn_mfma_f64_16x16x4f64(y.x, element<T>(hi[ks], i), acc[0], 0, 0, 0);
                acc[1] = __builtin_amdgcn_mfma_f64_16x16x4f64(y.y, element<T>(lo[ks], i), acc[1], 0, 0, 0);
            }
        acc[0] += acc[1];
        best = acc[0][0];
#pragma unroll
        for (int i = 1; i < 4; ++i) best = (acc[0][i] > best || acc[0][i] != acc[0][i]) ? acc[0][i] : best;
    }
    // the maximum over the heads: over the lanes that share the page (whatever head is where)
#pragma unroll
    for (int off = 16; off < kWave; off <<= 1) {
        const double other = __shfl_xor(best, off, kWave);
        best = (other > best || other != other) ? other : best;
    }
    // Where a bound or a query's element is infinite, the products above hold 0 x infinity, and their sum is no number; the larger product is one all the same
    // (unless an infinity meets a zero in it).  Pages without a number are worked out anew by the maximum, the four lanes of a page a piece of the row each.
    // (All lanes of the wavefront take part in the exchange, and the four of a page have the same sum and maximum.)
    if (ballot64(there && best != best) != 0ull) {
        double by_max = -INFINITY;
        for (int hh = 0; hh < p.G; ++hh) {
            double sum = 0.0;
            int64_t again = row;
            asm volatile("" : "+v"(again));      // (the bounds are read anew for every head: kept over the loop, in fp64, they would halve the workgroups of a compute unit)
#pragma unroll 1
            for (int ks = 0; ks < KL; ++ks) {
                const uint4 l = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(cv.k_min) + again + E * (4 * ks + g));
                const uint4 u = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(cv.k_max) + again + E * (4 * ks + g));
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const double2 y = s_q[q_place(E * (4 * ks + g) + i, hh)];
                    const double q = y.y != y.y ? y.x : y.x != y.x ? y.y : y.x + y.y, x = q * element<T>(l, i), z = q * element<T>(u, i);
                    sum += (x > z || x != x) ? x : z;      // (a NaN in either is the maximum)
                }
            }
#pragma unroll
            for (int off = 16; off < kWave; off <<= 1) sum += __shfl_xor(sum, off, kWave);
            by_max = (sum > by_max || sum != sum) ? sum : by_max;
        }
        if (best != best) best = by_max;
    }
    if (g == 0 && place < pages) {
        unsigned long long key = there ? score_key(best) : kKeyNaN;
        if (place < p.first || place >= pages - p.recent) key = kKeyForced;
        p.keys[bh * cv.P + place] = key;
    }
}

// One workgroup per (sequence, KV head).  The keys are spread over two buckets a thread, evenly between the smallest and the largest number, by one pass; the
// bucket that the last page to keep falls into holds a few of them, which are ranked against each other.  If they are more than fit (scores that are
// equal, or lie together far from a few others), the key is found eight bits at a time.
// One workgroup's wavefronts share four SIMDs, so the instructions, per key and per wavefront, are what bounds it: keys, numbers and buckets stay in registers
// (HELD a thread; MORE: those behind them are read again), stretches without keys are passed by, and few pages have few wavefronts.  2048 pages with 1024
// threads: 5.9 us (6.8 with the bucket found anew in every pass and four stretches counted whatever n is), of which loads 0.6, the range 0.8, the buckets 0.7,
// the rank's bucket 0.5, its keys 0.8, the places 0.9; 8192 pages: 9.6 us (13.7 with half of the keys in registers).
constexpr int kRanked = 256;

__device__ __forceinline__ int lanes_below(uint64_t m) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0)); }
__device__ __forceinline__ double key_score(unsigned long long k) { return __builtin_bit_cast(double, (k >> 63) ? k & ~(1ull << 63) : ~k); }

template <int THREADS, int HELD, bool MORE>
__global__ __launch_bounds__(THREADS) void paged_select_kernel(PagSelParams p) {
    const int64_t bh = blockIdx.x;
    const int b = (int)(blockIdx.x / (unsigned)p.c.H);
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int n = held_pages(p, bh, b), keep = p.keep;
    int32_t *sel = p.sel + bh * keep;
    if (tid == 0) p.sel_lens[bh] = min(n, keep);
    if (n <= keep) {
        for (int i = tid; i < keep; i += THREADS) sel[i] = i < n ? i : -1;
        return;
    }
    const unsigned long long *keys = p.keys + bh * p.c.P;
    constexpr int WAVES = THREADS / kWave, BUCKETS = 2 * THREADS;
    constexpr int LANES = kWave / WAVES, K = LANES < HELD ? LANES : HELD;      // stretches that a wavefront can count at a time, that it does
    static_assert(kRanked <= THREADS && HELD == (MORE ? 2 * K : K), "a thread for every ranked key, one or two rounds of counting");
    __shared__ int s_hist[BUCKETS];
    __shared__ float s_low[WAVES], s_high[WAVES];
    __shared__ int s_above[WAVES], s_count[kWave];
    __shared__ int s_bucket, s_need, s_ranked;
    __shared__ unsigned long long s_key[kRanked], s_border;
    __shared__ int s_place[kRanked], s_border_place;
    unsigned long long mine[HELD];
    float number[HELD];      // the scores in fp32 (the buckets only need an order), then, as integers, their buckets
#pragma unroll
    for (int k = 0; k < HELD; ++k) mine[k] = tid + k * THREADS < n ? keys[tid + k * THREADS] : 0ull;
    const auto number_of = [&](unsigned long long k) { return k < kKeyNaN ? (float)key_score(k) : INFINITY; };
    // ---- the smallest and the largest finite score
    float low = INFINITY, high = -INFINITY;
    const auto widen = [&](float x) {
        if (fabsf(x) < INFINITY) {
            low = fminf(low, x);
            high = fmaxf(high, x);
        }
    };
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        if (k * THREADS < n && tid + k * THREADS < n) {
            number[k] = number_of(mine[k]);
            widen(number[k]);
        }
    for (int i = tid + HELD * THREADS; MORE && i < n; i += THREADS) widen(number_of(keys[i]));
    low = -rows_allreduce_max(row_allreduce_max(-low));
    high = rows_allreduce_max(row_allreduce_max(high));
    if (lane == 0) { s_low[wave] = low; s_high[wave] = high; }
    for (int i = tid; i < BUCKETS; i += THREADS) s_hist[i] = 0;
    if (tid == 0) s_ranked = 0;
    __syncthreads();
    low = -row_allreduce_max(-s_low[lane % WAVES]);
    high = row_allreduce_max(s_high[lane % WAVES]);
    const float spread = high > low ? (float)(BUCKETS - 5) / (high - low) : 0.f;      // (0 too where high - low is not finite)
    const auto bucket_of = [&](unsigned long long k, float x) {      // never falls where the key grows
        const float at = fminf(fmaxf((x - low) * spread, 0.f), (float)(BUCKETS - 5));      // (no number where infinity is multiplied by zero: 0)
        return k >= kKeyNaN ? BUCKETS - 1 - (int)(k == kKeyNaN) : x >= INFINITY ? BUCKETS - 3 : x <= -INFINITY ? 0 : 1 + (int)at;
    };
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        if (k * THREADS < n && tid + k * THREADS < n) {
            const int to = bucket_of(mine[k], number[k]);
            number[k] = __int_as_float(to);
            atomicAdd(&s_hist[to], 1);
        }
    for (int i = tid + HELD * THREADS; MORE && i < n; i += THREADS) atomicAdd(&s_hist[bucket_of(keys[i], number_of(keys[i]))], 1);
    const auto each_of = [&](int bucket, auto f) {      // every key of a bucket, and its place
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (k * THREADS < n && tid + k * THREADS < n && __float_as_int(number[k]) == bucket) f(mine[k], tid + k * THREADS);
        for (int i = tid + HELD * THREADS; MORE && i < n; i += THREADS) {
            const unsigned long long k = keys[i];
            if (bucket_of(k, number_of(k)) == bucket) f(k, i);
        }
    };
    __syncthreads();
    // ---- the bucket of rank keep: thread t has buckets BUCKETS - 1 - 2 t and the one below
    {
        const int v0 = s_hist[BUCKETS - 1 - 2 * tid], v1 = s_hist[BUCKETS - 2 - 2 * tid];
        const int upto = wave_scan(v0 + v1);
        if (lane == kWave - 1) s_above[wave] = upto;
        __syncthreads();
        const int others = wave_scan(lane < WAVES ? s_above[lane % WAVES] : 0);
        int before = upto - v0 - v1 + (wave ? __builtin_amdgcn_readlane(others, wave - 1) : 0);
        if (before < keep && before + v0 >= keep) { s_bucket = BUCKETS - 1 - 2 * tid; s_need = keep - before; }
        before += v0;
        if (before < keep && before + v1 >= keep) { s_bucket = BUCKETS - 2 - 2 * tid; s_need = keep - before; }
    }
    __syncthreads();
    const int at = s_bucket;
    int need = s_need;      // of the keys that count as equal to the border's
    unsigned long long border = 0;
    int border_place = n;   // keys equal to the border's are kept up to this place
    if (s_hist[at] <= kRanked) {
        each_of(at, [&](unsigned long long k, int i) {
            const int r = atomicAdd(&s_ranked, 1);
            s_key[r] = k;
            s_place[r] = i;
        });
        __syncthreads();
        const int m = s_ranked;
        if (tid < m) {
            const unsigned long long k = s_key[tid];
            const int i = s_place[tid];
            int rank = 0;
            for (int r = 0; r < m; ++r) rank += s_key[r] > k || (s_key[r] == k && s_place[r] < i);
            if (rank == need - 1) { s_border = k; s_border_place = i; }
        }
        __syncthreads();
        border = s_border;
        border_place = s_border_place;
    } else {
        unsigned long long mask = 0;
        for (int shift = 56; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) s_hist[tid] = 0;
            __syncthreads();
            each_of(at, [&](unsigned long long k, int) {
                if ((k & mask) == border) atomicAdd(&s_hist[(int)(k >> shift) & 255], 1);
            });
            __syncthreads();
            if (wave == 0) {      // lane i: digits 255 - 4 i .. 252 - 4 i
                int v[4], sum = 0;
#pragma unroll
                for (int t = 0; t < 4; ++t) { v[t] = s_hist[255 - 4 * lane - t]; sum += v[t]; }
                int before = wave_scan(sum) - sum;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (before < need && before + v[t] >= need) { s_bucket = 255 - 4 * lane - t; s_need = need - before; }
                    before += v[t];
                }
            }
            __syncthreads();
            border |= (unsigned long long)s_bucket << shift;
            mask |= 255ull << shift;
            need = s_need;
        }
    }
    // ---- the places, ascending: keys above the border's, and of those equal to it the first ones (up to a place, or `need` of them); K stretches of
    // THREADS pages at a time, lane 16 k + w of every wavefront counting for stretch k and wavefront w
    const bool by_place = border_place < n;
    int above0 = 0, equal0 = 0;
    const auto put = [&](int i0, auto key_of) {
        uint64_t ba[K], be[K];
        int mine_of = 0;      // lane k: of stretch k
#pragma unroll
        for (int k = 0; k < K; ++k) {
            ba[k] = be[k] = 0;
            if (i0 + k * THREADS < n) {
                const int i = i0 + k * THREADS + tid;
                const unsigned long long x = key_of(k, i);      // (0 behind the last one)
                ba[k] = ballot64(x > border || (i <= border_place && x == border && by_place));
                if (!by_place) be[k] = ballot64(i < n && x == border);
                mine_of = lane == k ? __popcll(ba[k]) | __popcll(be[k]) << 16 : mine_of;
            }
        }
        if (i0 > 0) __syncthreads();
        if (lane < LANES) s_count[lane * WAVES + wave] = mine_of;
        __syncthreads();
        const int counts = s_count[lane], upto = wave_scan(counts);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (ba[k] | be[k]) {
                const int before = __builtin_amdgcn_readlane(upto - counts, k * WAVES + wave);
                const int above = above0 + (before & 0xffff) + lanes_below(ba[k]), equal = equal0 + (before >> 16) + lanes_below(be[k]);
                if (ba[k] >> lane & 1 || (be[k] >> lane & 1 && equal < need)) sel[above + min(equal, need)] = i0 + k * THREADS + tid;
            }
        const int all = __builtin_amdgcn_readlane(upto, kWave - 1);
        above0 += all & 0xffff;
        equal0 += all >> 16;
    };
    put(0, [&](int k, int) { return mine[k]; });
    if constexpr (MORE) {
        if (n > K * THREADS) put(K * THREADS, [&](int k, int) { return mine[K + k]; });
        for (int i0 = HELD * THREADS; i0 < n; i0 += K * THREADS) put(i0, [&](int, int i) { return i < n ? keys[i] : 0ull; });
    }
}

size_t paged_select_bytes(int B, int H, int P) { return align_up((size_t)B * H * P * sizeof(unsigned long long), 256); }

template <typename T, int D> static void launch_score(const PagSelParams &p, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)p.tiles * p.c.B * p.c.H)), threads(kScoreThreads);
    if (p.G <= 4) hipLaunchKernelGGL((paged_score_kernel<T, D, 1>), grid, threads, 0, stream, p);
    else if (p.G <= 8) hipLaunchKernelGGL((paged_score_kernel<T, D, 2>), grid, threads, 0, stream, p);
    else hipLaunchKernelGGL((paged_score_kernel<T, D, 0>), grid, threads, 0, stream, p);
}

template <int THREADS, int HELD, bool MORE> static void launch_choice(const PagSelParams &p, hipStream_t stream) {
    hipLaunchKernelGGL((paged_select_kernel<THREADS, HELD, MORE>), dim3((unsigned)(p.c.B * p.c.H)), dim3(THREADS), 0, stream, p);
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
    p.q_is_bf16 = a.q_dtype == DType::BF16;
    if (a.c.dtype == DType::BF16) {
        if (a.c.d == 128) launch_score<bf16_t, 128>(p, stream);
        else launch_score<bf16_t, 64>(p, stream);
    } else {
        if (a.c.d == 128) launch_score<float, 128>(p, stream);
        else launch_score<float, 64>(p, stream);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // both kernels, 64, 500, 1000, 1500, 2040 pages of 8 heads: 7.1, 7.8, 8.3, 8.8, 9.4 us with 512 threads, 8.2, 8.6, 8.8, 9.1, 9.5 with 1024; 256 threads take 7.0,
    // 8.1 and 9.2 for the first three; without the keys behind four stretches 1024 take 10.8 and 11.6 for 3000 and 4000, with them 10.9 and 11.7
    if (a.c.P <= 2048) launch_choice<512, 4, false>(p, stream);
    else launch_choice<1024, 8, true>(p, stream);
    return hipGetLastError();
}

}  // namespace sc
