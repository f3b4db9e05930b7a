// sc_prompt_attn: attention of the rows of a prompt (or of a chunk of it behind a context), causal, with a window and first rows that stay.
//     O_i = softmax over the keys j that query i sees of (q_i . k_j scale) V,   pos = kv_len - q_len + i,   j <= pos and (no window, or j > pos - window, or j < sinks)
//
// Bound by the matrix cores: 4 d operations for every pair of a query and a key that it sees, for 4 d bytes of a row of keys and values that every tile of queries
// reads from the caches.
//
// Work.  The queries of the G heads that share a KV head are rows (token, head) of one matrix, so that a tile of rows spans few tokens (the diagonal and the
// window's edge cost little) and every tile of keys serves all of them.  A workgroup of four wavefronts takes 32 QB rows a wavefront and goes over the tiles of keys that any of its rows sees; only
// tiles that some row does not see whole are masked.  Products are S^T = K Q^T and O^T += V^T P^T in 32 x 32 tiles: a query row stays on one pair of lanes from the
// logits to the output, and the probabilities leave the first product in the layout of the second one's operand.  Keys and values go through shared memory
// in two buffers, the next tile on its way in registers; rows are laid down with 16-byte pieces exchanged so that reads across rows meet all banks, and values
// are read transposed (ds_read_b64_tr_b16).  Softmax is online, in the exp2 domain, its sums in fp32; probabilities enter the second product as bf16 (each off by 2^-8 at
// most, as the bf16 output is by itself; errors of many keys average out), in fp32 calls as they are (v_mfma_f32_32x32x2_f32).
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

// A tile of keys (values) in shared memory: rows of RB bytes, 16-byte pieces of a row exchanged by `swap` (a function of the row)
template <typename T, int D, int THREADS, bool VALUES> struct Tile {
    static constexpr int KT = kTileKeys<T>, PIECES = D * (int)sizeof(T) / 16;
    static constexpr int RB = sizeof(T) == 2 ? 2 * D : 4 * D + 16;
    static constexpr int BYTES = KT * RB, LOADS = KT * PIECES / THREADS;
    static __device__ __forceinline__ int swap(int row) {
        if constexpr (sizeof(T) == 4) return 0;
        else if constexpr (!VALUES) return row & (PIECES - 1);
        else return D == 128 ? (row & 3) << 2 : (row >> 1 & 1) << 2;
    }
    // A thread's pieces: LOADS of them, of rows tid / PIECES + ...
    static __device__ __forceinline__ void load(pro_u32x4 (&x)[LOADS], const char *rows, int64_t stride, int here, int tid) {
        const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(rows), (short)0, here > 0 ? (int)((here - 1) * stride) + PIECES * 16 : 0, 0x00020000);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int c = tid + THREADS * i;
            x[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, (c / PIECES) * (int)stride + (c % PIECES) * 16, 0, 0);
        }
    }
    static __device__ __forceinline__ void store(const pro_u32x4 (&x)[LOADS], char *lds, int tid) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int c = tid + THREADS * i, row = c / PIECES;
            *reinterpret_cast<pro_u32x4 *>(lds + row * RB + ((c % PIECES) ^ swap(row)) * 16) = x[i];
        }
    }
    static __device__ __forceinline__ bool wild(const pro_u32x4 (&x)[LOADS]) {      // an element that is not finite
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (sizeof(T) == 2) any |= (uint32_t)((x[i][k] & 0x7f80u) == 0x7f80u) | (uint32_t)((x[i][k] & 0x7f800000u) == 0x7f800000u);
                else any |= (uint32_t)((x[i][k] & 0x7f800000u) == 0x7f800000u);
            }
        return any != 0;
    }
    static __device__ __forceinline__ void tame(pro_u32x4 (&x)[LOADS]) {            // zero in their place
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t w = x[i][k];
                if constexpr (sizeof(T) == 2) x[i][k] = ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
                else x[i][k] = (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
            }
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

// NW wavefronts of 32 QB rows
template <typename T, int D, int QB, int NW>
__global__ __launch_bounds__(NW *kWave, NW / 4) void prompt_kernel(ProParams p) {
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr int KT = kTileKeys<T>, KB = KT / 32, DT = D / 32, ROWS = 32 * QB * NW;
    using KTile = Tile<T, D, NW * kWave, false>;
    using VTile = Tile<T, D, NW * kWave, true>;
    __shared__ __attribute__((aligned(16))) char s_k[2][KTile::BYTES], s_v[2][VTile::BYTES];
    __shared__ int s_wild[2][NW];
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
    const int row0 = first + 32 * QB * wave;
    const int wt0 = row0 / p.G, wt1 = min((row0 + 32 * QB - 1) / p.G, q_len - 1);
    const bool idle = wt0 >= q_len;
    const PromptSpan span = prompt_span((int64_t)behind + wt0, (int64_t)behind + wt1, a.window, a.sinks);

    int token[QB], head[QB], pos[QB], edge[QB];
#pragma unroll
    for (int u = 0; u < QB; ++u) {
        const int r = row0 + 32 * u + col;
        token[u] = r / p.G;
        head[u] = h * p.G + r - token[u] * p.G;
        pos[u] = behind + token[u];
        edge[u] = prompt_edge(pos[u], a.window);
    }
    // ---- queries: bf16: lane (half, col) holds 8 half .. 8 half + 7 of every 16 elements of row `col`; fp32: elements (D / 2) half + ..
    constexpr int QL = kBf16 ? D / 16 : D / 8;
    pro_u32x4 q[QB][QL];
#pragma unroll
    for (int u = 0; u < QB; ++u) {
        const char *src = a.Q + b * a.q_b + head[u] * a.q_h + (int64_t)min(token[u], a.N - 1) * a.q_n;
#pragma unroll
        for (int i = 0; i < QL; ++i) {
            q[u][i] = *reinterpret_cast<const pro_u32x4 *>(src + (kBf16 ? (16 * i + 8 * half) * 2 : ((D / 2) * half + 4 * i) * 4));
            q[u][i] ^= kBf16 ? p.flip | p.flip >> 16 : p.flip;
        }
    }

    pro_f32x16 o[QB][DT];
    float m_run[QB], l_run[QB];
#pragma unroll
    for (int u = 0; u < QB; ++u) {
        m_run[u] = -INFINITY;
        l_run[u] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[u][t][i] = 0.f;
    }

    // ---- a tile of keys for my rows
    auto attend = [&](int k0, const char *lk, const char *lv) {
        pro_f32x16 s[QB][KB];
#pragma unroll
        for (int u = 0; u < QB; ++u)
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[u][k][i] = 0.f;
        if constexpr (kBf16) {
#pragma unroll
            for (int e = 0; e < D / 16; ++e)
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    const int row = 32 * k + col;
                    const pro_u32x4 key = *reinterpret_cast<const pro_u32x4 *>(lk + row * KTile::RB + ((2 * e + half) ^ KTile::swap(row)) * 16);
#pragma unroll
                    for (int u = 0; u < QB; ++u)
                        s[u][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pro_bf16x8, key), __builtin_bit_cast(pro_bf16x8, q[u][e]), s[u][k], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int e = 0; e < D / 8; ++e) {
                const pro_u32x4 key = *reinterpret_cast<const pro_u32x4 *>(lk + col * KTile::RB + ((D / 2) * half + 4 * e) * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int u = 0; u < QB; ++u)
                        s[u][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(key[i]), __uint_as_float(q[u][e][i]), s[u][0], 0, 0, 0);
            }
        }
        if (!prompt_all(span, k0, KT)) {
#pragma unroll
            for (int u = 0; u < QB; ++u)
#pragma unroll
                for (int k = 0; k < KB; ++k)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = k0 + 32 * k + 8 * (i / 4) + 4 * half + i % 4;
                        s[u][k][i] = prompt_sees(key, pos[u], edge[u], a.sinks) ? s[u][k][i] : -INFINITY;
                    }
        }
        // ---- softmax
#pragma unroll
        for (int u = 0; u < QB; ++u) {
            float mx = s[u][0][0];
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[u][k][i]);
            mx = halves_max(mx) * p.scale_log2;
            if (ballot64(mx > m_run[u] + kProSlack) != 0ull) {
                const float m_new = fmaxf(m_run[u], mx);
                const float alpha = m_new == -INFINITY ? 1.f : pro_exp2(m_run[u] - m_new);
                m_run[u] = m_new;
                l_run[u] *= alpha;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[u][d][i] *= alpha;
            }
            const float shift = m_run[u] == -INFINITY ? 0.f : m_run[u];
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[u][k][i] = pro_exp2(fmaf(s[u][k][i], p.scale_log2, -shift));
                    sum[i % 2] += s[u][k][i];
                }
            l_run[u] += sum[0] + sum[1];
        }
        // ---- O^T += V^T P^T.  Place 8 half + j of the inner dimension is key 4 half + j of 16, or 8 + 4 half + j - 4
        if constexpr (kBf16) {
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    pro_u32x4 w[QB];
#pragma unroll
                    for (int u = 0; u < QB; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[u][i] = pack_bf16x2(s[u][k][8 * g + 2 * i], s[u][k][8 * g + 2 * i + 1]);
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
                        for (int u = 0; u < QB; ++u)
                            o[u][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pro_bf16x8, val), __builtin_bit_cast(pro_bf16x8, w[u]), o[u][d], 0, 0, 0);
                    }
                }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = 8 * (i / 4) + 4 * half + i % 4;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const float val = *reinterpret_cast<const float *>(lv + key * VTile::RB + (32 * d + col) * 4);
#pragma unroll
                    for (int u = 0; u < QB; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(val, s[u][0][i], o[u][d], 0, 0, 0);
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
#pragma unroll
                    for (int u = 0; u < QB; ++u)
                        if (prompt_sees(k0 + key, pos[u], edge[u], a.sinks)) {
                            o[u][d][4 * i] += if_wild(v.x);
                            o[u][d][4 * i + 1] += if_wild(v.y);
                            o[u][d][4 * i + 2] += if_wild(v.z);
                            o[u][d][4 * i + 3] += if_wild(v.w);
                        }
                }
    };

    const char *kb = a.K + b * a.k_b + h * a.k_h, *vb = a.V + b * a.v_b + h * a.v_h;
    pro_u32x4 kx[KTile::LOADS], vx[VTile::LOADS];
    auto request = [&](int t) {
        const int k0 = prompt_tile(mine, t) * KT;
        KTile::load(kx, kb + (int64_t)k0 * a.k_n, a.k_n, min(kv_len - k0, KT), tid);
        VTile::load(vx, vb + (int64_t)k0 * a.v_n, a.v_n, min(kv_len - k0, KT), tid);
    };
    auto lay_down = [&](int t, int buf) {
        if (!prompt_all(all, prompt_tile(mine, t) * KT, KT)) {
            const bool wild = VTile::wild(vx);
            const uint64_t any = ballot64(wild);
            if (lane == 0) s_wild[buf][wave] = any != 0;
            if (wild) VTile::tame(vx);
        }
        KTile::store(kx, s_k[buf], tid);
        VTile::store(vx, s_v[buf], tid);
    };
    if (t0 < t1) {
        request(t0);
        lay_down(t0, 0);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1, k0 = prompt_tile(mine, t) * KT;
        if (t + 1 < t1) request(t + 1);
        if (!idle && prompt_some(span, k0, KT)) {
            attend(k0, s_k[buf], s_v[buf]);
            if (!prompt_all(all, k0, KT)) {
                int wild = 0;
#pragma unroll
                for (int w = 0; w < NW; ++w) wild |= s_wild[buf][w];
                if (__builtin_amdgcn_readfirstlane(wild)) attend_wild(k0, vb + (int64_t)k0 * a.v_n, min(kv_len - k0, KT));
            }
        }
        if (t + 1 < t1) lay_down(t + 1, buf ^ 1);
        __syncthreads();
    }
    // ---- results
#pragma unroll
    for (int u = 0; u < QB; ++u) {
        if (token[u] >= q_len) continue;
        const float l = halves_sum(l_run[u]);
        if (p.splits > 1) {
            float *part = p.part + (((int64_t)split * heads + bh) * ((int64_t)a.N * p.G) + row0 + 32 * u + col) * (D + 4);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4 *>(part + 32 * d + 8 * i + 4 * half) = make_float4(o[u][d][4 * i], o[u][d][4 * i + 1], o[u][d][4 * i + 2], o[u][d][4 * i + 3]);
            if (half == 0) *reinterpret_cast<float2 *>(part + D) = make_float2(m_run[u], l);
            continue;
        }
        const float f = l != 0.f ? 1.0f / l : 0.f;
        char *dst = a.O + b * a.o_b + head[u] * a.o_h + (int64_t)token[u] * a.o_n;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store_row4(dst, kBf16, 32 * d + 8 * i + 4 * half, make_float4(o[u][d][4 * i] * f, o[u][d][4 * i + 1] * f, o[u][d][4 * i + 2] * f, o[u][d][4 * i + 3] * f));
        if (a.lse && half == 0) a.lse[((int64_t)b * a.Hq + head[u]) * a.N + token[u]] = l != 0.f ? (m_run[u] + __log2f(l)) * kProLn2 : -INFINITY;
    }
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
    float m = -INFINITY;
    for (int s = 0; s < p.splits; ++s) m = fmaxf(m, part[s * next + D]);
    const float shift = m == -INFINITY ? 0.f : m;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
    for (int s = 0; s < p.splits; ++s) {
        const float2 ml = *reinterpret_cast<const float2 *>(part + s * next + D);
        const float4 x = *reinterpret_cast<const float4 *>(part + s * next + e);
        const float f = pro_exp2(ml.x - shift);
        l = fmaf(ml.y, f, l);
        o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
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
    s.rows = bf16 && rows * heads >= 128 * 256 ? 256 : 128;
    s.tiles = (int)((rows + s.rows - 1) / s.rows);
    // a workgroup for every compute unit, with eight tiles of keys each at least
    const int64_t wgs = s.tiles * heads, most = (M + 511) / 512;
    int64_t splits = wgs >= 192 ? 1 : 256 / wgs;
    if (splits > most) splits = most;
    if (splits > 64) splits = 64;
    s.splits = splits < 1 ? 1 : (int)splits;
    return s;
}
size_t prompt_workspace_bytes(int B, int Hq, int Hkv, int N, int M, int d) {
    size_t most = 0;
    for (int bf16 = 0; bf16 < 2; ++bf16) {
        const ProShape s = prompt_shape(B, Hq, Hkv, N, M, d, bf16 != 0);
        const size_t bytes = s.splits > 1 ? (size_t)s.splits * B * Hq * N * (d + 4) * sizeof(float) : 0;
        if (bytes > most) most = bytes;
    }
    return align_up(most + 256, 256);
}
bool prompt_fits(int B, int Hq, int Hkv, int N, int M, int d, bool bf16) {
    const ProShape s = prompt_shape(B, Hq, Hkv, N, M, d, bf16);
    return (int64_t)s.tiles * B * Hkv * s.splits <= INT32_MAX && (int64_t)B * Hq * N <= ((int64_t)1 << 33);
}

#ifndef PRO_QB
#define PRO_QB 1
#define PRO_NW 8
#endif
template <typename T, int D, int QB, int NW> static hipError_t launch_prompt_k(const ProParams &p, hipStream_t stream) {
    const unsigned wgs = (unsigned)((int64_t)p.tiles * p.a.B * p.a.Hkv * p.splits);
    hipLaunchKernelGGL((prompt_kernel<T, D, QB, NW>), dim3(wgs), dim3(NW * kWave), 0, stream, p);
    if (p.splits > 1) {
        const int64_t rows = (int64_t)p.a.N * p.a.Hq * p.a.B, per = 256 / (D / 4);
        hipLaunchKernelGGL((prompt_join_kernel<D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}
template <int D> static hipError_t launch_prompt_d(const ProParams &p, int rows, hipStream_t stream) {
    if (p.a.dtype != DType::BF16) return launch_prompt_k<float, D, 1, 4>(p, stream);
    return rows == 256 ? launch_prompt_k<bf16_t, D, PRO_QB, PRO_NW>(p, stream) : launch_prompt_k<bf16_t, D, 1, 4>(p, stream);
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
