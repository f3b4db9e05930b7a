// sc_paged_reserve: page tables and slot maps from the sequences' lengths.  Pages that a sequence needs for the rows that arrive are taken from a stack of free ones,
// pages that no row of it needs any more go back.
//
//     held(s, p) = table[s, p] is a page of the pool          want(s, p) = (paged_wants)   place p holds rows that are visible, or arrives
//     back = held and not want,   take = want and not held;   a sequence with a wanted place below base that is not held is refused, with nothing changed for it
//     the k-th page taken, in the order of (s, p), is the k-th given back in that order, then the stack's top; what is given back and not taken goes on the stack, the last one
//     first, so that a call that is followed by its opposite leaves the stack as it was.
//
// Two launches, bound by their chains of trips.  The first counts, a workgroup a sequence, and compacts what it gives back.  The second applies, a workgroup for 256 places of a sequence: it adds up the
// counts of the others by itself (of more than kResSelf sequences a launch between does, by one workgroup), knows the ranks of its places from them, and writes the slots of the rows that lie in them.  The stack is only
// read where more is taken than given back and only written where less is, so no workgroup waits for another.
//
// Measured: a token of 64 sequences 7.1 us (3.1 + 4.0), handed out and taken back one after the other 15; 512 sequences up to 32768 rows, with their slots, and all of them taken back 28 (3.4 + 16.8 with the slots, 67 MB of writes, and 4.9 + 5.0).  The workgroup that adds up more than 2048 sequences shows: a token handed out and taken back, 2048 sequences 26, 2049 33, 4096 48, 65536 604.  Added up by the last workgroup of the
// first launch, found by one counter for all, 512 sequences take 11.5 us there instead of 3.6.
#include "sc_paged.h"

namespace sc {

constexpr int kResThreads = 256;      // places of a chunk
constexpr int kResWaves = kResThreads / kWave;

constexpr int kResRows = 8;           // counts that a thread adds up
constexpr int kResSelf = kResThreads * kResRows;

// workspace: per sequence {taken, given back} (-1: refused) and, of many, their sums over the sequences before it; per chunk the same within the sequence; the call's totals (free pages at the start;
// of many also given back and taken); the pages given back by every sequence
struct ReserveSpace {
    int2 *count, *before, *chunk;
    int *total;
    int32_t *given;
};
static size_t reserve_layout(int S, int P, char *base, ReserveSpace &w) {
    const int64_t chunks = (P + kResThreads - 1) / kResThreads;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = align_up(at + bytes, 256);
        return base + here;
    };
    w.count = reinterpret_cast<int2 *>(take((size_t)S * sizeof(int2)));
    w.before = reinterpret_cast<int2 *>(take((size_t)S * sizeof(int2)));
    w.chunk = reinterpret_cast<int2 *>(take((size_t)S * chunks * sizeof(int2)));
    w.total = reinterpret_cast<int *>(take(4 * sizeof(int)));
    w.given = reinterpret_cast<int32_t *>(take((size_t)S * P * sizeof(int32_t)));
    return at;
}
size_t paged_reserve_bytes(int S, int P) {
    ReserveSpace w;
    return reserve_layout(S, P, nullptr, w);
}

struct ReserveParams {
    PagedReserveArgs a;
    ReserveSpace w;
    int log2_R, chunks;
};

struct Lengths {
    int base, fresh;
    bool ok;
};
__device__ __forceinline__ Lengths lengths_of(const PagedReserveArgs &a, int s, int log2_R) {
    const int base = a.base_lens[s], fresh = a.new_lens ? a.new_lens[s] : a.N;
    return {base, fresh, base >= 0 && fresh >= 0 && fresh <= a.N && (int64_t)base + fresh <= (int64_t)a.P << log2_R};
}

// Per thread a yes or no of two kinds: how many threads before this one say yes, and all of the workgroup
struct Ranks {
    int take, back, takes, backs;
};
__device__ __forceinline__ Ranks ranks(bool take, bool back, int lane, int wave, int2 *s_wave) {
    const uint64_t t = ballot64(take), k = ballot64(back), below = (1ull << lane) - 1;
    if (lane == 0) s_wave[wave] = make_int2(__popcll(t), __popcll(k));
    __syncthreads();
    Ranks r = {(int)__popcll(t & below), (int)__popcll(k & below), 0, 0};
#pragma unroll
    for (int w = 0; w < kResWaves; ++w) {
        const int2 n = s_wave[w];
        if (w < wave) { r.take += n.x; r.back += n.y; }
        r.takes += n.x;
        r.backs += n.y;
    }
    __syncthreads();
    return r;
}
// Sums over the threads before this one, and over all of the workgroup
struct Sums {
    int2 before, all;
};
__device__ __forceinline__ Sums sums(int2 x, int lane, int wave, int2 *s_wave) {
    const int2 incl = make_int2(wave_scan(x.x), wave_scan(x.y));
    if (lane == kWave - 1) s_wave[wave] = incl;
    __syncthreads();
    Sums r = {make_int2(incl.x - x.x, incl.y - x.y), make_int2(0, 0)};
#pragma unroll
    for (int w = 0; w < kResWaves; ++w) {
        const int2 n = s_wave[w];
        if (w < wave) { r.before.x += n.x; r.before.y += n.y; }
        r.all.x += n.x;
        r.all.y += n.y;
    }
    __syncthreads();
    return r;
}
__device__ __forceinline__ int wg_max(int x, int lane, int wave, int2 *s_wave) {      // x >= 0
    x = wave_max(x);
    if (lane == 0) s_wave[wave].x = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kResWaves; ++w) x = max(x, s_wave[w].x);
    __syncthreads();
    return x;
}

__global__ __launch_bounds__(kResThreads) void reserve_count_kernel(ReserveParams p) {
    const PagedReserveArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, s = blockIdx.x;
    __shared__ int2 s_wave[kResWaves];
    const int32_t *row = a.table + (int64_t)s * a.P;
    int page = tid < a.P ? row[tid] : -1;      // (with the lengths)
    const Lengths n = lengths_of(a, s, p.log2_R);
    if (s == 0 && tid == 0) p.w.total[0] = min(max(a.num_free[0], 0), a.num_pages);
    int takes = 0, backs = 0, missing = 0;
    for (int c = 0; n.ok && c < p.chunks; ++c) {
        const int place = c * kResThreads + tid;
        const int next = place + kResThreads < a.P ? row[place + kResThreads] : -1;
        const bool held = (unsigned)page < (unsigned)a.num_pages, want = place < a.P && paged_wants(place, p.log2_R, n.base, n.fresh, a.window, a.sinks);
        missing |= want && !held && ((int64_t)place << p.log2_R) < n.base;
        const Ranks r = ranks(want && !held, held && !want, lane, wave, s_wave);
        if (tid == 0) p.w.chunk[(int64_t)s * p.chunks + c] = make_int2(takes, backs);
        if (held && !want) p.w.given[(int64_t)s * a.P + backs + r.back] = page;
        takes += r.takes;
        backs += r.backs;
        page = next;
    }
    missing = __syncthreads_or(missing);
    if (tid == 0) p.w.count[s] = n.ok && !missing ? make_int2(takes, backs) : make_int2(-1, 0);
}

// more than kResSelf sequences: their places, by one workgroup
__global__ __launch_bounds__(kResThreads) void reserve_scan_kernel(ReserveParams p) {
    const PagedReserveArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    __shared__ int2 s_wave[kResWaves];
    int2 start = make_int2(0, 0);
    for (int s0 = 0; s0 < a.S; s0 += kResThreads) {
        const int s = s0 + tid;
        const int2 x = s < a.S ? p.w.count[s] : make_int2(0, 0);
        const Sums r = sums(make_int2(max(x.x, 0), x.y), lane, wave, s_wave);
        if (s < a.S) p.w.before[s] = make_int2(start.x + r.before.x, start.y + r.before.y);
        start.x += r.all.x;
        start.y += r.all.y;
    }
    const int available = p.w.total[0] + start.y;
    int taken = 0;
    for (int s = tid; s < a.S; s += kResThreads) {
        const int through = p.w.before[s].x + max(p.w.count[s].x, 0);      // (the thread's own)
        if (through <= available) taken = max(taken, through);
    }
    taken = wg_max(taken, lane, wave, s_wave);
    if (tid == 0) {
        p.w.total[1] = start.y;
        p.w.total[2] = taken;
    }
}

// SELF: the workgroup adds up the counts
template <bool SELF> __global__ __launch_bounds__(kResThreads) void reserve_apply_kernel(ReserveParams p) {
    const PagedReserveArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int s = blockIdx.x / p.chunks, c = blockIdx.x % p.chunks;
    __shared__ int2 s_wave[kResWaves], s_mine;
    __shared__ int32_t s_page[kResThreads];
    __shared__ int s_back[SELF ? kResSelf : 1];      // given back by the sequences before
    const int place = c * kResThreads + tid;
    int32_t *entry = a.table + (int64_t)s * a.P + place;
    const int page = place < a.P ? *entry : -1;
    const Lengths n = lengths_of(a, s, p.log2_R);
    const int2 count = p.w.count[s], chunk = p.w.chunk[(int64_t)s * p.chunks + c];
    const int free_pages = p.w.total[0];
    int2 before;
    int backs, taken;
    if constexpr (SELF) {
        int2 x[kResRows], mine = make_int2(0, 0);
#pragma unroll
        for (int i = 0; i < kResRows; ++i) {
            const int r = tid * kResRows + i;
            x[i] = r < a.S ? p.w.count[r] : make_int2(0, 0);
            x[i].x = max(x[i].x, 0);
            mine.x += x[i].x;
            mine.y += x[i].y;
        }
        const Sums r = sums(mine, lane, wave, s_wave);
        backs = r.all.y;
        int2 at = r.before;
        taken = 0;
#pragma unroll
        for (int i = 0; i < kResRows; ++i) {
            s_back[tid * kResRows + i] = at.y;
            if (tid * kResRows + i == s) s_mine = at;
            at.x += x[i].x;
            at.y += x[i].y;
            if (at.x <= free_pages + backs) taken = max(taken, at.x);
        }
        taken = wg_max(taken, lane, wave, s_wave);
        before = s_mine;
    } else {
        before = p.w.before[s];
        backs = p.w.total[1];
        taken = p.w.total[2];
    }
    // (pages go back all the same where there are none to take)
    const bool fine = count.x == 0 || (count.x > 0 && before.x + count.x <= free_pages + backs);
    int32_t now = page;
    if (count.x >= 0) {
        const bool held = (unsigned)page < (unsigned)a.num_pages, want = place < a.P && paged_wants(place, p.log2_R, n.base, n.fresh, a.window, a.sinks);
        const Ranks r = ranks(want && !held, held && !want, lane, wave, s_wave);
        if (want && !held && fine) {
            const int k = before.x + chunk.x + r.take;
            if (k < backs) {
                // the sequence that gives the k-th back: the last one whose first is not behind it
                auto first_of = [&](int q) { return SELF ? s_back[q] : p.w.before[q].y; };
                int lo = 0, hi = a.S - 1;
                while (lo < hi) {
                    const int mid = (lo + hi + 1) / 2;
                    if (first_of(mid) <= k) lo = mid;
                    else hi = mid - 1;
                }
                now = p.w.given[(int64_t)lo * a.P + (k - first_of(lo))];
            } else {
                now = a.free_pages[free_pages - 1 - (k - backs)];
            }
            *entry = now;
        } else if (held && !want) {
            const int k = before.y + chunk.y + r.back;
            const int64_t to = (int64_t)free_pages + backs - 1 - k;
            if (k >= taken && to < a.num_pages) a.free_pages[to] = page;      // (beyond the pool only if tables name a page twice)
            now = -1;
            *entry = -1;
        }
    }
    if (c == 0 && tid == 0) {
        a.lens[s] = fine ? n.base + n.fresh : -1;
        if (s == 0) a.num_free[0] = (int)min((int64_t)free_pages + backs - taken, (int64_t)a.num_pages);
    }
    if (!a.slots) return;
    s_page[tid] = now;
    __syncthreads();
    const int64_t first = (int64_t)c * kResThreads << p.log2_R, past = (int64_t)(c + 1) * kResThreads << p.log2_R;
    int32_t *slots = a.slots + (int64_t)s * a.N;
    if (fine) {
        const int t1 = (int)min((int64_t)n.base + n.fresh, past);
        for (int64_t t = max((int64_t)n.base, first) + tid; t < t1; t += kResThreads)
            slots[t - n.base] = (s_page[(t >> p.log2_R) - c * kResThreads] << p.log2_R) + (int)(t & ((1 << p.log2_R) - 1));
    }
    for (int64_t k = (fine ? n.fresh : 0) + (int64_t)c * kResThreads + tid; k < a.N; k += (int64_t)p.chunks * kResThreads) slots[k] = -1;
}

hipError_t launch_paged_reserve(const PagedReserveArgs &a, void *ws, hipStream_t stream) {
    ReserveParams p;
    p.a = a;
    reserve_layout(a.S, a.P, static_cast<char *>(ws), p.w);
    p.log2_R = __builtin_ctz((unsigned)a.R);
    p.chunks = (a.P + kResThreads - 1) / kResThreads;
    hipLaunchKernelGGL(reserve_count_kernel, dim3((unsigned)a.S), dim3(kResThreads), 0, stream, p);
    const dim3 wgs((unsigned)(a.S * p.chunks));      // (at most S P <= 2^28)
    if (a.S <= kResSelf) {
        hipLaunchKernelGGL(reserve_apply_kernel<true>, wgs, dim3(kResThreads), 0, stream, p);
    } else {
        hipLaunchKernelGGL(reserve_scan_kernel, dim3(1), dim3(kResThreads), 0, stream, p);
        hipLaunchKernelGGL(reserve_apply_kernel<false>, wgs, dim3(kResThreads), 0, stream, p);
    }
    return hipGetLastError();
}

}  // namespace sc
