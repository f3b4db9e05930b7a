// What the appending kernels have in common: the pieces of a row that a lane holds, the rotation of positions, and the workgroups that rotate queries.
#pragma once
#include "sc_paged.h"

namespace sc {

constexpr int kAppThreads = 256;
// groups of pages from which the heads of one are kept on a chiplet: eight for each of them.  Prompts of 4096 and 8192 tokens (64 and 128 groups) 23.9 and 44.2 us, 24.2
// and 45.4 otherwise; below, chiplets would be left without work: 256 tokens (four groups) 4.8 us, 5.1 near; a token each of 16 and 32 sequences 4.4 and 4.5, 4.6 near
constexpr int kNearItems = 64;

// A lane's two pieces of 16 bytes of a row (of E elements each), chosen so that the partners of a rotation are in the same lane
template <typename T> struct Shape {
    static constexpr int E = 16 / (int)sizeof(T);
};
struct Pieces {
    int ea, eb;       // first elements
    bool turned;
};
template <int E> __device__ __forceinline__ Pieces pieces_of(int j, int rot, bool interleaved) {
    const bool turned = 2 * E * j < rot;
    const bool halves = turned && !interleaved;      // partners i and i + rot / 2; else neighbours, or elements that stay
    return {halves ? E * j : 2 * E * j, halves ? E * j + rot / 2 : 2 * E * j + E, turned};
}
// the angles of both are the E from E j on
template <int E> __device__ __forceinline__ void turn(float (&x)[E], float (&y)[E], const float (&c)[E], const float (&s)[E], bool interleaved) {
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
template <int E> __device__ __forceinline__ void load_angles(const float *p, float (&x)[E]) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
        const float4 t = *reinterpret_cast<const float4 *>(p + i);
        x[i] = t.x; x[i + 1] = t.y; x[i + 2] = t.z; x[i + 3] = t.w;
    }
}
// 16 bytes as they lie in memory
typedef unsigned int raw_u32x4 __attribute__((ext_vector_type(4)));      // (HIP's own uint4 would be copied through memory)
template <typename T> struct Raw {
    static constexpr int E = Shape<T>::E;
    raw_u32x4 w;
    __device__ __forceinline__ void load(const char *p) { w = *reinterpret_cast<const raw_u32x4 *>(p); }
    __device__ __forceinline__ void store(char *p) const { *reinterpret_cast<raw_u32x4 *>(p) = w; }
    __device__ __forceinline__ void widen(float (&x)[E]) const {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (sizeof(T) == 2) x[i] = (i & 1) ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
            else x[i] = __uint_as_float(w[i]);
        }
    }
    __device__ __forceinline__ void round(const float (&x)[E]) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (sizeof(T) == 2) w[i / 2] = pack_bf16x2(x[i & ~1], x[i | 1]);
            else w[i] = __float_as_uint(x[i]);
        }
    }
};

// A number that the whole wavefront reads, and that nobody writes meanwhile: through the scalar cache
__device__ __forceinline__ int read_scalar(const int32_t *p) { return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p; }

struct AppendGrid {
    int kv_blocks, page_groups;             // workgroups of the keys and values; of a sequence and head
    int log2_waves;                         // wavefronts of a page
    int kv_near;                            // the heads of a page on one chiplet (paged_share)
    int log2_tokens, q_tiles;               // tokens that a workgroup of the queries holds at a time; tiles of so many
    int q_heads, q_groups;                  // heads that it goes over; groups of so many
};

// Queries (workgroup id0 of theirs): a tile of tokens, several heads at a time (of few tokens, all heads that there is room for)
template <typename TQ, int D>
__device__ __forceinline__ void rotate_queries(const PagedAppendArgs &p, const AppendGrid &g, int id0) {
    constexpr int WAVES = kAppThreads / kWave, U = 2;      // passes whose loads are on their way together
    constexpr int E = Shape<TQ>::E, LPR = D / (2 * E), RPW = kWave / LPR;
    const int tid = threadIdx.x, half = p.rot / 2;
    const bool interleaved = p.interleaved != 0;
    const int j = tid % LPR;
    const Pieces at = pieces_of<E>(j, p.rot, interleaved);
    int id = id0;
    const int group = id % g.q_groups;
    id /= g.q_groups;
    const int tile = id % g.q_tiles, b = id / g.q_tiles;
    const int r = tid / LPR;
    const int n = (tile << g.log2_tokens) + (r & ((1 << g.log2_tokens) - 1));
    if (n >= p.N) return;
    const int64_t pos = (int64_t)read_scalar((p.positions ? p.positions : p.base_lens) + b) + n;
    const bool known = pos >= 0 && pos < p.max_position;
    float co[E], si[E];
    if (at.turned && known) {
        load_angles(p.cos_sin + pos * p.rot + E * j, co);
        load_angles(p.cos_sin + pos * p.rot + half + E * j, si);
    }
    const int step = (WAVES * RPW) >> g.log2_tokens;
    const int h1 = min((group + 1) * g.q_heads, p.Hq);
    const char *src = p.Q + b * p.q_b + n * p.q_n;
    char *dst = p.Q_out + b * p.o_b + n * p.o_n;
    for (int h = group * g.q_heads + (r >> g.log2_tokens); h < h1; h += U * step) {
        Raw<TQ> a[U], e[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (h + u * step < h1) {
                a[u].load(src + (h + u * step) * p.q_h + at.ea * (int)sizeof(TQ));
                e[u].load(src + (h + u * step) * p.q_h + at.eb * (int)sizeof(TQ));
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (h + u * step < h1) {
                if (!known || at.turned) {
                    float x[E], y[E];
                    a[u].widen(x);
                    e[u].widen(y);
                    if (known) turn(x, y, co, si, interleaved);
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        x[i] = known ? x[i] : __builtin_nanf("");
                        y[i] = known ? y[i] : __builtin_nanf("");
                    }
                    a[u].round(x);
                    e[u].round(y);
                }
                a[u].store(dst + (h + u * step) * p.o_h + at.ea * (int)sizeof(TQ));
                e[u].store(dst + (h + u * step) * p.o_h + at.eb * (int)sizeof(TQ));
            }
    }
}

// the queries' share of a grid (kv_blocks, page_groups, log2_waves and kv_near are the caller's)
template <typename TQ, int D> inline void query_grid(const PagedAppendArgs &a, AppendGrid &g) {
    constexpr int WAVES = kAppThreads / kWave, QRPW = kWave / (D / (2 * Shape<TQ>::E));
    g.log2_tokens = 0;
    while ((1 << g.log2_tokens) < a.N && (1 << g.log2_tokens) < WAVES * QRPW) ++g.log2_tokens;
    g.q_tiles = (a.N + (1 << g.log2_tokens) - 1) >> g.log2_tokens;
    g.q_heads = WAVES * QRPW >> g.log2_tokens;      // (32768 tokens, 8 + 32 heads: 2 heads 159 us, 4 161, 8 163, 16 169)
    if (g.q_heads < 2) g.q_heads = 2;
    g.q_groups = a.Q ? (a.Hq + g.q_heads - 1) / g.q_heads : 0;
}

}  // namespace sc
