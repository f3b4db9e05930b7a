// sc_prompt_attn: attention of the rows of a prompt (or of a chunk of it behind a context), causal, with a window and first rows that stay.
//     O_i = softmax over the keys j that query i sees of (q_i . k_j scale) V,   pos = kv_len - q_len + i,   j <= pos and (no window, or j > pos - window, or j < sinks)
//
// Bound by the matrix cores: 4 d operations for every pair of a query and a key that it sees, for 4 d bytes of a row of keys and values that every tile of queries
// reads from the caches.
//
// Work.  The queries of the G heads that share a KV head are rows (token, head) of one matrix, so that a tile of rows spans few tokens (the diagonal and the
// window's edge cost little) and every tile of keys serves all of them.  A workgroup of eight wavefronts (four in small calls, and in fp32) takes 32 rows a wavefront and goes over the tiles of keys that any of its rows sees; only
// tiles that some row does not see whole are masked.  Products are S^T = K Q^T and O^T += V^T P^T in 32 x 32 tiles: a query row stays on one pair of lanes from the
// logits to the output, and the probabilities leave the first product in the layout of the second one's operand.  Keys and values go straight to shared
// memory (buffer_load .. lds), in three places (two in workgroups of four), the next tiles on their way; the 16-byte pieces of a row are exchanged so that reads across rows meet all banks, and values
// are read transposed (ds_read_b64_tr_b16).  The halves of a workgroup of eight take turns: one is at the matrix cores while the other forms probabilities, a barrier a phase.  Softmax is online, in the exp2 domain, its sums in fp32; probabilities enter the second product as two
// rounded bf16 parts, 2^-17 off, in fp32 calls as they are (v_mfma_f32_32x32x2_f32).  One part (the products take two thirds then, 8192 tokens 526 us instead of 705 on one card) would be 2^-8 off: that is a bf16 output's own rounding once more, 0.0020 of its norm instead of
// 0.0016, and where many keys have one weight, all of them are rounded the same way and the output is no mean of the values any more.
//
// Measured (d = 128, bf16, 8 KV and 32 query heads): 8192 tokens 690 to 730 us by card (1.13 to 1.20 PFLOP/s with the products of the second part; a library product of 8192^3 reaches 1.25 to 1.27), 16384 behind a window of 4096 1250 to 1310 (1.11 to 1.17): the matrix
// cores are busy 60 % of the cycles, and at that load the clock is at 1.9 GHz.  d = 64: 8192 tokens 450, 2048 59.  fp32, d = 64, 3 x 2 x 3 heads, up to 600 tokens: 33 to 36 us, 5 of it the second launch.
//
// Calls with few tiles of rows cut their keys into splits, whose partial results a second launch joins.
#include <type_traits>

#include "sc_device.h"
#include "sc_host.h"
#include "sc_prompt.h"

namespace sc {

constexpr float kProLog2e = 1.4426950408889634f;
constexpr float kProLn2 = 0.6931471805599453f;
// The running maximum follows once a logit exceeds it by this many powers of two: until then nothing needs rescaling, and weights up to 2^8 lose no bit
constexpr float kProSlack = 8.f;

typedef float pro_f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int pro_u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 pro_bf16x8 __attribute__((ext_vector_type(8)));
typedef short pro_s16x4 __attribute__((ext_vector_type(4)));

template <typename T> constexpr int kTileKeys = sizeof(T) == 2 ? 64 : 32;

struct ProParams {
    PromptArgs a;
    float scale_log2;
    uint32_t flip;         // sign of a negative scale, put on the queries
    int G, tiles;          // heads of a KV head; tiles of rows of a (sequence, KV head)
    int splits;
    float *part;           // [split][b, h][row][D + 4] sums, maximum, denominator
};

__device__ __forceinline__ float pro_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <typename T> __device__ __forceinline__ bool is_wild(uint32_t w) {      // an element of w is not finite
    return (w & 0x7f800000u) == 0x7f800000u || (sizeof(T) == 2 && (w & 0x7f80u) == 0x7f80u);
}
template <typename T> __device__ __forceinline__ uint32_t tamed(uint32_t w) {    // zero in its place
    if constexpr (sizeof(T) == 2) return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
    else return (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
}

// A tile of KT rows in shared memory, as it comes from memory without a register between (buffer_load .. lds: lane l of a wavefront writes the l-th 16 bytes from a common address on).  The 16-byte
// pieces of a row are exchanged by a function of the row, so that reads across rows meet all banks: the lanes ask for them in that order.
template <typename T, int D, int NW, bool VALUES> struct Tile {
    static constexpr int KT = kTileKeys<T>, RB = D * (int)sizeof(T), PIECES = RB / 16, BYTES = KT * RB;
    static constexpr int LOADS = BYTES / (1024 * NW);
    static_assert(LOADS * 1024 * NW == BYTES, "the same for every wavefront");
    static __device__ __forceinline__ int swap(int row) {
        if constexpr (sizeof(T) == 2 && VALUES) return D == 128 ? (row & 3) << 2 : (row >> 1 & 1) << 2;      // (read transposed: 4 rows x 64 bytes a half)
        else return row & (PIECES - 1);
    }
    int offset[LOADS];      // of the lane's pieces
    uint32_t stride;
    __device__ __forceinline__ void init(int64_t row_stride, int wave, int lane) {
        stride = (uint32_t)row_stride;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int c = (i * NW + wave) * kWave + lane, row = c / PIECES;
            offset[i] = row * (int)row_stride + ((c % PIECES) ^ swap(row)) * 16;
        }
    }
    // rows k0 .. of `rows`, up to `end`; nothing is read behind them
    __device__ __forceinline__ void load(char *lds, const char *rows, int k0, int end, int wave) const {
        const uint64_t at = (uint64_t)(uintptr_t)rows + (uint64_t)(uint32_t)k0 * stride;
        const int here = min(end - k0, KT);
        const pro_u32x4 rs = {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xffffu)),
                              (uint32_t)__builtin_amdgcn_readfirstlane(here > 0 ? (here - 1) * (int)stride + RB : 0), 0x00020000u};
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int m0 = __builtin_amdgcn_readfirstlane((int)(to + (i * NW + wave) * 1024));
            // (m0 is the compiler's to write; five wait states for a descriptor that v_readfirstlane has just written, which it does not count into the text)
            asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(m0), "v"(offset[i]), "s"(rs) : "memory");
        }
    }
    // The wavefront's own pieces, arrived: numbers that are not finite become zero.  Says whether there were any
    __device__ __forceinline__ bool tame(char *lds, int wave, int lane) const {
        bool any = false;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            auto *p = reinterpret_cast<pro_u32x4 *>(lds + (i * NW + wave) * 1024 + lane * 16);
            pro_u32x4 x = *p;
            bool wild = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) wild |= is_wild<T>(x[k]);
            if (wild) {
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = tamed<T>(x[k]);
                *p = x;
            }
            any |= wild;
        }
        return any;
    }
};

// four values of a row, elements e .. e + 3, as fp32
template <typename T> __device__ __forceinline__ float4 values4(const char *row, int e) {
    if constexpr (sizeof(T) == 2) {
        const uint2 w = *reinterpret_cast<const uint2 *>(row + 2 * e);
        return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
    } else {
        return *reinterpret_cast<const float4 *>(row + 4 * e);
    }
}
__device__ __forceinline__ float if_wild(float x) { return fabsf(x) < INFINITY ? 0.f : x; }

// NW wavefronts of 32 rows
template <typename T, int D, int NW>
__global__ __launch_bounds__(NW *kWave, NW / 4) void prompt_kernel(ProParams p) {
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr int KT = kTileKeys<T>, KB = KT / 32, DT = D / 32, ROWS = 32 * NW, kParts = kBf16 ? 2 : 1;
    using KTile = Tile<T, D, NW, false>;
    using VTile = Tile<T, D, NW, true>;
    constexpr bool kTurns = NW == 8;              // the halves of the workgroup take turns (below)
    constexpr int kPlaces = kTurns ? 3 : 2;
    __shared__ int s_wild[kPlaces][NW];
    __shared__ __attribute__((aligned(16))) char s_k[kPlaces][KTile::BYTES], s_v[kPlaces][VTile::BYTES];
    const PromptArgs &a = p.a;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int half = lane / 32, col = lane % 32;
    // ---- my tile of rows, the longest ones first
    const int heads = a.B * a.Hkv;
    const int id = blockIdx.x / p.splits, split = blockIdx.x % p.splits;
    const int bh = id % heads, b = bh / a.Hkv, h = bh % a.Hkv;
    const int first = (p.tiles - 1 - id / heads) * ROWS;
    const int q_len = a.q_lens ? min(max(a.q_lens[b], 0), a.N) : a.N, kv_len = a.kv_lens ? min(max(a.kv_lens[b], 0), a.M) : a.M;
    const int behind = kv_len - q_len;                 // position of the first query
    const int token0 = first / p.G, token1 = min((first + ROWS - 1) / p.G, q_len - 1);
    if (token0 >= q_len) return;
    const PromptSpan all = prompt_span((int64_t)behind + token0, (int64_t)behind + token1, a.window, a.sinks);
    const PromptTiles mine = prompt_tiles(all, KT);
    const int t0 = (int)((int64_t)mine.count * split / p.splits), t1 = (int)((int64_t)mine.count * (split + 1) / p.splits);
    // ... and my wavefront's
    const int row0 = first + 32 * wave;
    const int wt0 = row0 / p.G, wt1 = min((row0 + 31) / p.G, q_len - 1);
    const PromptSpan span = prompt_span((int64_t)behind + wt0, (int64_t)behind + wt1, a.window, a.sinks);

    const int token = (row0 + col) / p.G, head = h * p.G + (row0 + col) - token * p.G;
    const int pos = behind + token, edge = prompt_edge(pos, a.window);
    // ---- queries: bf16: lane (half, col) holds 8 half .. 8 half + 7 of every 16 elements of row `col`; fp32: elements (D / 2) half + ..
    constexpr int QL = kBf16 ? D / 16 : D / 8;
    pro_u32x4 q[QL];
    const char *src = a.Q + b * a.q_b + head * a.q_h + (int64_t)min(token, a.N - 1) * a.q_n;
#pragma unroll
    for (int i = 0; i < QL; ++i) {
        q[i] = *reinterpret_cast<const pro_u32x4 *>(src + (kBf16 ? (16 * i + 8 * half) * 2 : ((D / 2) * half + 4 * i) * 4));
        q[i] ^= kBf16 ? p.flip | p.flip >> 16 : p.flip;
        if (token >= q_len) q[i] = pro_u32x4{0, 0, 0, 0};      // (the maxima of all rows of a wavefront follow together: what lies behind the last query must not say when)
    }

    pro_f32x16 o[DT];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;

    // ---- a tile of keys for my rows: logits, probabilities, and their product with the values
    pro_f32x16 s[KB];                          // logits, then (fp32) probabilities
    pro_u32x4 w[kParts][kBf16 ? 2 * KB : 1];   // (bf16) probabilities, in two parts
    auto logits = [&](const char *lk) {
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[k][i] = 0.f;
        if constexpr (kBf16) {
#pragma unroll
            for (int e = 0; e < D / 16; ++e)
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    const int row = 32 * k + col;
                    const pro_u32x4 key = *reinterpret_cast<const pro_u32x4 *>(lk + row * KTile::RB + ((2 * e + half) ^ KTile::swap(row)) * 16);
                    s[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pro_bf16x8, key), __builtin_bit_cast(pro_bf16x8, q[e]), s[k], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int e = 0; e < D / 8; ++e) {
                const pro_u32x4 key = *reinterpret_cast<const pro_u32x4 *>(lk + col * KTile::RB + ((D / 8 * half + e) ^ KTile::swap(col)) * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(key[i]), __uint_as_float(q[e][i]), s[0], 0, 0, 0);
            }
        }
    };
    auto probabilities = [&](int k0, bool masked) {
        if (masked) {
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = k0 + 32 * k + 8 * (i / 4) + 4 * half + i % 4;
                    s[k][i] = prompt_sees(key, pos, edge, a.sinks) ? s[k][i] : -INFINITY;
                }
        }
        float mx = s[0][0];
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[k][i]);
        mx = halves_max(mx) * p.scale_log2;
        if (ballot64(mx > m_run + kProSlack) != 0ull) {
            const float m_new = fmaxf(m_run, mx);
            const float alpha = m_new == -INFINITY ? 1.f : pro_exp2(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
        }
        const float shift = m_run == -INFINITY ? 0.f : m_run;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[k][i] = pro_exp2(fmaf(s[k][i], p.scale_log2, -shift));
                sum[i % 2] += s[k][i];
            }
        l_run += sum[0] + sum[1];
        if constexpr (kBf16) {
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t hi = pack_bf16x2(s[k][2 * i], s[k][2 * i + 1]);
                    w[0][2 * k + i / 4][i % 4] = hi;
                    w[1][2 * k + i / 4][i % 4] = pack_bf16x2(s[k][2 * i] - bf16_lo(hi), s[k][2 * i + 1] - bf16_hi(hi));
                }
        }
    };
    auto add_values = [&](const char *lv) {
        // O^T += V^T P^T.  Place 8 half + j of the inner dimension is key 4 half + j of 16, or 8 + 4 half + j - 4
        if constexpr (kBf16) {
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        // 16 lanes read 4 keys x 16 elements, every lane four elements of a key, and get four keys of an element
                        const int lane16 = lane % 16, key = 32 * k + 16 * g + 4 * half + lane16 / 4;
                        const int at = 64 * d + 32 * (lane / 16 % 2) + 8 * (lane16 % 4);
                        uint2 v[2];
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            typedef __attribute__((address_space(3))) pro_s16x4 lds_s16x4;
                            const char *src = lv + (key + 8 * x) * VTile::RB + ((at / 16) ^ VTile::swap(key + 8 * x)) * 16 + at % 16;
                            v[x] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)src));
                        }
                        const pro_u32x4 val = {v[0].x, v[0].y, v[1].x, v[1].y};
#pragma unroll
                        for (int x = kParts - 1; x >= 0; --x)
                            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pro_bf16x8, val), __builtin_bit_cast(pro_bf16x8, w[x][2 * k + g]), o[d], 0, 0, 0);
                    }
                }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = 8 * (i / 4) + 4 * half + i % 4;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const float val = *reinterpret_cast<const float *>(lv + key * VTile::RB + ((8 * d + col / 4) ^ VTile::swap(key)) * 16 + col % 4 * 4);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(val, s[0][i], o[d], 0, 0, 0);
                }
            }
        }
    };
    // Values that are not finite, in a tile that some row of the workgroup does not see whole: 0 times such a number would be none.  They are zero in shared memory then, and added to
    // the rows that see them from where they lie
    auto attend_wild = [&](int k0, const char *rows, int here) {
        for (int key = 0; key < here; ++key)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 v = values4<T>(rows + (int64_t)key * a.v_n, 32 * d + 8 * i + 4 * half);
                    if (prompt_sees(k0 + key, pos, edge, a.sinks)) {
                        o[d][4 * i] += if_wild(v.x);
                        o[d][4 * i + 1] += if_wild(v.y);
                        o[d][4 * i + 2] += if_wild(v.z);
                        o[d][4 * i + 3] += if_wild(v.w);
                    }
                }
    };

    const char *kb = a.K + b * a.k_b + h * a.k_h, *vb = a.V + b * a.v_b + h * a.v_h;
    KTile kx;
    VTile vx;
    kx.init(a.k_n, wave, lane);
    vx.init(a.v_n, wave, lane);
    const int n = t1 - t0;
    auto key_of = [&](int t) { return prompt_tile(mine, t0 + t) * KT; };
    // Tile t is in place t % kPlaces of its buffers
    auto request_keys = [&](int t, int place) {
        if (t < n) kx.load(s_k[place], kb, key_of(t), kv_len, wave);
    };
    auto request_values = [&](int t, int place) {
        if (t < n) vx.load(s_v[place], vb, key_of(t), kv_len, wave);
    };
    auto settle = [&](int t, int place) {      // what the wavefront has requested is there; the values of tile t are fit for the product
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (t < n && !prompt_all(all, key_of(t), KT)) {
            const uint64_t any = ballot64(vx.tame(s_v[place], wave, lane));
            if (lane == 0) s_wild[place][wave] = any != 0;
        }
    };
    // ---- The two halves of the workgroup take turns: while one is at its products (values of a tile, logits of the next), the other forms probabilities, so that the matrix cores and the
    // vector units are at work together (wavefronts w and w + NW / 2 share a SIMD).  The second half runs one barrier behind the first.  Phase p lies between barriers p and p + 1:
    //     first half    logits 0 in phase 0, probabilities t in phase 2 t + 1, products t (values t, keys t + 1) in 2 t + 2
    //     second half   logits 0 in phase 1, probabilities t in phase 2 t + 2, products t in 2 t + 3
    // Keys t + 2 and values t + 1 are requested with probabilities t.  They take the places of keys t - 1 and values t - 2, which were last read in phase 2 t - 1, and are there by the end of phase
    // 2 t + 3: a half waits for what it has requested at the end of its phase of that number.
    // With four wavefronts, one on each SIMD, nobody takes turns: all are the first half, and keys t and values t - 1 make room.  With d = 64 a second workgroup fits beside them, in the other phase or not; with d = 128 the
    // compiler takes 290 registers (fp32: 348), and they are alone on a compute unit.
    const bool second = kTurns && wave >= NW / 2;
    auto meet = [&]() {      // (nothing of one phase is put off into the next one: the compiler would)
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };
    request_keys(0, 0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    meet();
    request_keys(1, 1);
    request_values(0, 0);
    if (second) meet();
    // (fp32: products of tiles that the wavefront's rows do not see are left out; bf16's are part of a fixed order of reads and products.  Chunks of a
    // small model 37.4 -> 35.5 us, 500 tokens of 2 x 2 heads 25.6 -> 23.8)
    auto sees = [&](int t) { return kBf16 || (t < n && prompt_some(span, key_of(t), KT)); };
    if (sees(0)) logits(s_k[0]);
    if (second) settle(0, 0);
    meet();
    int here = 0, next = 1, after = 2 % kPlaces;      // places of tiles t, t + 1, t + 2
    for (int t = 0; t < n; ++t) {
        const int k0 = key_of(t);
        const bool edges = !prompt_all(all, k0, KT);
        if (!second) settle(t, here);
        request_keys(t + 2, after);
        request_values(t + 1, next);
        const bool some = sees(t);
        if (some) probabilities(k0, !prompt_all(span, k0, KT));
        if constexpr (kBf16) {
#pragma unroll
            for (int i = 0; i < 2 * KB; ++i) asm volatile("" : "+v"(w[0][i]), "+v"(w[1][i]));
        }
        meet();
        __builtin_amdgcn_s_setprio(1);      // (who is at the products goes first: 8192 tokens 528 -> 522 us, with probabilities in one part)
        if (some) add_values(s_v[here]);
        if (sees(t + 1)) logits(s_k[next]);      // (bf16: behind the last tile of anything: nobody uses them)
        if constexpr (kBf16) {         // operands are read well ahead of the products that take them: a read takes as long as four products
            constexpr int kAhead = 8, PV = 2 * KB * DT, QK = KB * D / 16;
            __builtin_amdgcn_sched_group_barrier(0x100, 2 * kAhead, 0);
#pragma unroll
            for (int i = 0; i < PV - kAhead; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, kParts, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, kParts, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
#pragma unroll
            for (int i = 0; i < QK - kAhead; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (edges) {
            int wild = 0;
#pragma unroll
            for (int x = 0; x < NW; ++x) wild |= s_wild[here][x];
            if (some && __builtin_amdgcn_readfirstlane(wild)) attend_wild(k0, vb + (int64_t)k0 * a.v_n, min(kv_len - k0, KT));
        }
        if (second) settle(t + 1, next);
        meet();
        const int x = here;
        here = next;
        next = after;
        after = kTurns ? x : here;
    }
    if (kTurns && !second) meet();
    // ---- results
    if (token >= q_len) return;
    const float l = halves_sum(l_run);
    if (p.splits > 1) {
        float *part = p.part + (((int64_t)split * heads + bh) * ((int64_t)a.N * p.G) + row0 + col) * (D + 4);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4 *>(part + 32 * d + 8 * i + 4 * half) = make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
        if (half == 0) *reinterpret_cast<float2 *>(part + D) = make_float2(m_run, l);
        return;
    }
    const float f = l != 0.f ? 1.0f / l : 0.f;
    char *dst = a.O + b * a.o_b + head * a.o_h + (int64_t)token * a.o_n;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store_row4(dst, kBf16, 32 * d + 8 * i + 4 * half, make_float4(o[d][4 * i] * f, o[d][4 * i + 1] * f, o[d][4 * i + 2] * f, o[d][4 * i + 3] * f));
    if (a.lse && half == 0) a.lse[((int64_t)b * a.Hq + head) * a.N + token] = l != 0.f ? (m_run + __log2f(l)) * kProLn2 : -INFINITY;
}

// D / 4 threads a row, all partial results of it one after the other
template <int D>
__global__ __launch_bounds__(256) void prompt_join_kernel(ProParams p) {
    constexpr int TPR = D / 4;
    const PromptArgs &a = p.a;
    const int64_t rows = (int64_t)a.N * p.G, all = rows * a.B * a.Hkv;
    const int64_t i = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (i >= all) return;
    const int e = 4 * (threadIdx.x % TPR), bh = (int)(i / rows), b = bh / a.Hkv, h = bh % a.Hkv;
    const int r = (int)(i - (int64_t)bh * rows), token = r / p.G, head = h * p.G + r - token * p.G;
    if (token >= (a.q_lens ? min(max(a.q_lens[b], 0), a.N) : a.N)) return;
    const float *part = p.part + i * (D + 4);
    const int64_t next = all * (D + 4);
    constexpr int PASS = 8;      // partial results whose loads are on their way together (those behind the last one read it again, and count for nothing)
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    for (int s0 = 0; s0 < p.splits; s0 += PASS) {
        float2 ml[PASS];
        float4 x[PASS];
#pragma unroll
        for (int t = 0; t < PASS; ++t) {
            const float *from = part + min(s0 + t, p.splits - 1) * next;
            ml[t] = *reinterpret_cast<const float2 *>(from + D);
            x[t] = *reinterpret_cast<const float4 *>(from + e);
        }
        float m_new = m;
#pragma unroll
        for (int t = 0; t < PASS; ++t) m_new = fmaxf(m_new, ml[t].x);
        const float shift = m_new == -INFINITY ? 0.f : m_new, keep = pro_exp2(m - shift);
        o = make_float4(o.x * keep, o.y * keep, o.z * keep, o.w * keep);
        l *= keep;
        m = m_new;
#pragma unroll
        for (int t = 0; t < PASS; ++t) {
            const float f = s0 + t < p.splits ? pro_exp2(ml[t].x - shift) : 0.f;
            if (s0 + t >= p.splits) x[t] = make_float4(0.f, 0.f, 0.f, 0.f);
            l = fmaf(s0 + t < p.splits ? ml[t].y : 0.f, f, l);
            o.x = fmaf(x[t].x, f, o.x); o.y = fmaf(x[t].y, f, o.y); o.z = fmaf(x[t].z, f, o.z); o.w = fmaf(x[t].w, f, o.w);
        }
    }
    const float f = l != 0.f ? 1.0f / l : 0.f;
    store_row4(a.O + b * a.o_b + head * a.o_h + (int64_t)token * a.o_n, a.dtype == DType::BF16, e, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
    if (a.lse && e == 0) a.lse[((int64_t)b * a.Hq + head) * a.N + token] = l != 0.f ? (m + __log2f(l)) * kProLn2 : -INFINITY;
}

// ------------------------------------------------------------------------------------------------
struct ProShape {
    int rows, tiles, splits;      // rows of a workgroup, tiles of a (sequence, KV head), splits of the keys
};
static ProShape prompt_shape(int B, int Hq, int Hkv, int N, int M, int d, bool bf16) {
    const int64_t G = Hq / Hkv, rows = (int64_t)N * G, heads = (int64_t)B * Hkv;
    ProShape s;
    // Eight wavefronts take turns, four do not, and have a compute unit to themselves with d = 128.  512 tokens of 8 x 4 heads behind 16384 198 us with 256 rows, 282 with 128; 2048 tokens 77 and 83;
    // but 64 tokens 13.0 and 9.9, 16 behind 32768 52 and 49.  With few keys 128 rows are no slower as long as each compute unit has one workgroup at most: 512 and 1024 tokens of 8 x 4 heads 23.7 and
    // 40.6 us, 25.8 and 42.3 with 256; but 1024 behind 512 56 and 52, behind 2048 103 and 82 (three times 400 tokens, 312 workgroups, 23.5 with either)
    s.rows = bf16 && rows >= 1024 && (M > 1024 || (rows + 127) / 128 * heads > 256) ? 256 : 128;
    s.tiles = (int)((rows + s.rows - 1) / s.rows);
    // A workgroup for every compute unit with eight tiles of keys each at least; fp32, whose products take eight times as long, two of them with two tiles (500 tokens of 2 x 2 heads 24 us, 88 with
    // the former; with three or four chunks of a small model 40 to 43 us instead of 36; the former with twice the splits, when probabilities were in one part: 1024 tokens of 8 x 4 heads 45 us, 33)
    const int64_t wgs = s.tiles * heads, target = bf16 ? 256 : 512, most = bf16 ? (M + 511) / 512 : (M + 63) / 64;
    int64_t splits = wgs >= target * 3 / 4 ? 1 : target / wgs;
    if (splits > most) splits = most;
    if (splits > 64) splits = 64;
    s.splits = splits < 1 ? 1 : (int)splits;
    return s;
}
// Enough for every call of up to so many sequences, queries and keys: splits x workgroups are no more than prompt_shape's targets, 256 of 256 rows or 512 of 128
size_t prompt_workspace_bytes(int B, int Hq, int Hkv, int N, int M, int d) {
    (void)Hkv;
    const int64_t splits = (M + 63) / 64 < 64 ? (M + 63) / 64 : 64;
    int64_t rows = (int64_t)B * Hq * N;
    rows = rows < 65536 ? rows * splits : 65536;
    if (rows > 65536) rows = 65536;
    return align_up((size_t)rows * (d + 4) * sizeof(float), 256);
}
bool prompt_fits(int B, int Hq, int Hkv, int N, int M, int d, bool bf16) {
    const ProShape s = prompt_shape(B, Hq, Hkv, N, M, d, bf16);
    return (int64_t)s.tiles * B * Hkv * s.splits <= INT32_MAX && (int64_t)B * Hq * N <= ((int64_t)1 << 33);
}

template <typename T, int D, int NW> static hipError_t launch_prompt_k(const ProParams &p, hipStream_t stream) {
    const unsigned wgs = (unsigned)((int64_t)p.tiles * p.a.B * p.a.Hkv * p.splits);
    hipLaunchKernelGGL((prompt_kernel<T, D, NW>), dim3(wgs), dim3(NW * kWave), 0, stream, p);
    if (p.splits > 1) {
        const int64_t rows = (int64_t)p.a.N * p.a.Hq * p.a.B, per = 256 / (D / 4);
        hipLaunchKernelGGL((prompt_join_kernel<D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}
template <int D> static hipError_t launch_prompt_d(const ProParams &p, int rows, hipStream_t stream) {
    if (p.a.dtype != DType::BF16) return launch_prompt_k<float, D, 4>(p, stream);
    return rows == 256 ? launch_prompt_k<bf16_t, D, 8>(p, stream) : launch_prompt_k<bf16_t, D, 4>(p, stream);
}

hipError_t launch_prompt(const PromptArgs &a, hipStream_t stream) {
    const ProShape s = prompt_shape(a.B, a.Hq, a.Hkv, a.N, a.M, a.d, a.dtype == DType::BF16);
    ProParams p;
    p.a = a;
    p.scale_log2 = fabsf(a.scale) * kProLog2e;
    p.flip = a.scale < 0.f ? 0x80000000u : 0u;
    p.G = a.Hq / a.Hkv;
    p.tiles = s.tiles;
    p.splits = s.splits;
    p.part = static_cast<float *>(a.ws);
    return a.d == 128 ? launch_prompt_d<128>(p, s.rows, stream) : launch_prompt_d<64>(p, s.rows, stream);
}

}  // namespace sc
