// sc_paged_reserve: page tables and slot maps from the sequences' lengths.  Pages that a sequence needs for the rows that arrive are taken from a stack of free ones,
// pages that no row of it needs any more go back.
//
//     held(s, p) = table[s, p] is a page of the pool          want(s, p) = (paged_wants)   place p holds rows that are visible, or arrives
//     back = held and not want,   take = want and not held;   a sequence with a wanted place below base that is not held is refused, with nothing changed for it
//     the k-th page taken, in the order of (s, p), is the k-th given back in that order, then the stack's top; what is given back and not taken goes on the stack, the last one
//     first, so that a call that is followed by its opposite leaves the stack as it was.
//
// Two launches, bound by their chains of trips.  The first counts, a workgroup a sequence, and compacts what it gives back; the workgroup that ends last turns the counts into
// places of all sequences.  The second applies them, a workgroup for 256 places, and writes the slots of the rows that lie in them.  The stack is only read where more is taken than
// given back and only written where less is, so no workgroup waits for another.
#include "sc_paged.h"

namespace sc {

constexpr int kResThreads = 256;      // places of a chunk
constexpr int kResWaves = kResThreads / kWave;

// workspace, behind the counters: per sequence {taken, given back} and their sums over the sequences before it (negative: the sequence is refused), per chunk the same within the sequence, the
// pages given back by every sequence, and the call's totals
struct ReserveSpace {
    int *counter;
    int2 *count, *before, *chunk;
    int *total;      // free pages at the start, given back, taken
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
    w.counter = reinterpret_cast<int *>(take(paged_state_bytes()));
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
__device__ __forceinline__ int2 load_agent(const int2 *p) {
    const uint64_t x = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_int2((int)(uint32_t)x, (int)(uint32_t)(x >> 32));
}
__device__ __forceinline__ void store_agent(int2 *p, int2 x) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), (uint64_t)(uint32_t)x.y << 32 | (uint32_t)x.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__global__ __launch_bounds__(kResThreads) void reserve_count_kernel(ReserveParams p) {
    const PagedReserveArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, s = blockIdx.x;
    __shared__ int2 s_wave[kResWaves];
    __shared__ int s_last;
    const Lengths n = lengths_of(a, s, p.log2_R);
    const int32_t *row = a.table + (int64_t)s * a.P;
    int takes = 0, backs = 0, missing = 0;
    for (int c = 0; n.ok && c < p.chunks; ++c) {
        const int place = c * kResThreads + tid;
        const int page = place < a.P ? row[place] : -1;
        const bool held = (unsigned)page < (unsigned)a.num_pages, want = place < a.P && paged_wants(place, p.log2_R, n.base, n.fresh, a.window, a.sinks);
        missing |= want && !held && ((int64_t)place << p.log2_R) < n.base;
        const Ranks r = ranks(want && !held, held && !want, lane, wave, s_wave);
        if (tid == 0) p.w.chunk[(int64_t)s * p.chunks + c] = make_int2(takes, backs);
        if (held && !want) p.w.given[(int64_t)s * a.P + backs + r.back] = page;
        takes += r.takes;
        backs += r.backs;
    }
    missing = __syncthreads_or(missing);
    const bool fine = n.ok && !missing;
    if (tid == 0) store_agent(p.w.count + s, fine ? make_int2(takes, backs) : make_int2(-1, 0));
    // ---- the last workgroup: places of all sequences
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (its counts have arrived)
    __syncthreads();
    if (tid == 0) {
        const int before = __hip_atomic_fetch_add(p.w.counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = before == a.S - 1;
        if (s_last) __hip_atomic_store(p.w.counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
    __shared__ int2 s_sum[kResWaves];
    const int free_pages = min(max(a.num_free[0], 0), a.num_pages);
    int all_backs = 0;
    for (int s0 = 0; s0 < a.S; s0 += kResThreads) {
        const int2 x = s0 + tid < a.S ? load_agent(p.w.count + s0 + tid) : make_int2(0, 0);
        const int sum = __builtin_amdgcn_readlane(wave_scan(x.y), kWave - 1);
        if (lane == 0) s_sum[wave].y = sum;
        __syncthreads();
        for (int w = 0; w < kResWaves; ++w) all_backs += s_sum[w].y;
        __syncthreads();
    }
    const int available = (int)min((int64_t)free_pages + all_backs, (int64_t)INT32_MAX);
    int taken = 0, given = 0, served = 0;      // of the sequences before; taken by those that are served
    for (int s0 = 0; s0 < a.S; s0 += kResThreads) {
        const int2 x = s0 + tid < a.S ? load_agent(p.w.count + s0 + tid) : make_int2(-1, 0);
        const int mine = max(x.x, 0), t = wave_scan(mine), k = wave_scan(x.y);
        if (lane == kWave - 1) s_sum[wave] = make_int2(t, k);
        __syncthreads();
        int2 start = make_int2(taken, given);
        for (int w = 0; w < kResWaves; ++w) {
            const int2 y = s_sum[w];
            if (w < wave) { start.x += y.x; start.y += y.y; }
            taken += y.x;
            given += y.y;
        }
        const int through = start.x + t;
        const bool gets = x.x == 0 || (x.x > 0 && through <= available);
        if (gets && x.x > 0) served = max(served, through);
        if (s0 + tid < a.S) {
            const Lengths m = lengths_of(a, s0 + tid, p.log2_R);
            // (pages go back all the same where there are none to take)
            p.w.before[s0 + tid] = make_int2(x.x < 0 ? -1 : gets ? through - mine : -2, start.y + k - x.y);
            a.lens[s0 + tid] = gets ? m.base + m.fresh : -1;
        }
        __syncthreads();
    }
    served = wave_max(served);
    if (lane == 0) s_sum[wave].x = served;
    __syncthreads();
    if (tid == 0) {
        for (int w = 0; w < kResWaves; ++w) served = max(served, s_sum[w].x);
        p.w.total[0] = free_pages;
        p.w.total[1] = all_backs;
        p.w.total[2] = served;
        a.num_free[0] = min(available - served, a.num_pages);      // (more only if tables name a page twice)
    }
}

__global__ __launch_bounds__(kResThreads) void reserve_apply_kernel(ReserveParams p) {
    const PagedReserveArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int s = blockIdx.x / p.chunks, c = blockIdx.x % p.chunks;
    __shared__ int2 s_wave[kResWaves];
    __shared__ int32_t s_page[kResThreads];
    const Lengths n = lengths_of(a, s, p.log2_R);
    const int2 before = p.w.before[s], chunk = p.w.chunk[(int64_t)s * p.chunks + c];
    const int free_pages = p.w.total[0], backs = p.w.total[1], takes = p.w.total[2];
    const int place = c * kResThreads + tid;
    int32_t *entry = a.table + (int64_t)s * a.P + place;
    const int page = place < a.P ? *entry : -1;
    int32_t now = page;
    const bool fine = before.x >= 0;
    if (n.ok && before.x != -1) {
        const bool held = (unsigned)page < (unsigned)a.num_pages, want = place < a.P && paged_wants(place, p.log2_R, n.base, n.fresh, a.window, a.sinks);
        const Ranks r = ranks(want && !held, held && !want, lane, wave, s_wave);
        if (want && !held && fine) {
            const int k = before.x + chunk.x + r.take;
            if (k < backs) {
                // the sequence that gives the k-th back: the last one whose first is not behind it
                int lo = 0, hi = a.S - 1;
                while (lo < hi) {
                    const int mid = (lo + hi + 1) / 2;
                    if (p.w.before[mid].y <= k) lo = mid;
                    else hi = mid - 1;
                }
                now = p.w.given[(int64_t)lo * a.P + (k - p.w.before[lo].y)];
            } else {
                now = a.free_pages[free_pages - 1 - (k - backs)];
            }
            *entry = now;
        } else if (held && !want) {
            const int k = before.y + chunk.y + r.back;
            const int64_t to = (int64_t)free_pages + backs - 1 - k;
            if (k >= takes && to < a.num_pages) a.free_pages[to] = page;
            now = -1;
            *entry = -1;
        }
    }
    if (!a.slots) return;
    s_page[tid] = now;
    __syncthreads();
    const int total = fine && n.ok ? n.base + n.fresh : n.base;
    const int64_t first = (int64_t)c * kResThreads << p.log2_R, past = (int64_t)(c + 1) * kResThreads << p.log2_R;
    int32_t *slots = a.slots + (int64_t)s * a.N;
    if (fine && n.ok) {
        const int t1 = (int)min((int64_t)total, past);
        for (int64_t t = max((int64_t)n.base, first) + tid; t < t1; t += kResThreads)
            slots[t - n.base] = (s_page[(t >> p.log2_R) - c * kResThreads] << p.log2_R) + (int)(t & ((1 << p.log2_R) - 1));
    }
    for (int64_t k = (fine && n.ok ? n.fresh : 0) + (int64_t)c * kResThreads + tid; k < a.N; k += (int64_t)p.chunks * kResThreads) slots[k] = -1;
}

hipError_t launch_paged_reserve(const PagedReserveArgs &a, void *ws, hipStream_t stream) {
    ReserveParams p;
    p.a = a;
    reserve_layout(a.S, a.P, static_cast<char *>(ws), p.w);
    p.log2_R = __builtin_ctz((unsigned)a.R);
    p.chunks = (a.P + kResThreads - 1) / kResThreads;
    hipLaunchKernelGGL(reserve_count_kernel, dim3((unsigned)a.S), dim3(kResThreads), 0, stream, p);
    hipLaunchKernelGGL(reserve_apply_kernel, dim3((unsigned)(a.S * p.chunks)), dim3(kResThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace sc
