// sc_prompt_attn as its launcher sees it (internal; the public boundary is include/semanticache.h), and which keys a tile of queries visits.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace sc {

// ---- plain functions, so that the host can try them.  Positions and keys are below 2^30, a position may be negative.
// a query at `pos` sees the keys up to itself that lie behind `edge`, or before `sinks`
constexpr int prompt_edge(int64_t pos, int window) { return window > 0 && pos - window > -1 ? (int)(pos - window) : -1; }
constexpr bool prompt_sees(int key, int pos, int edge, int sinks) { return key <= pos && (key > edge || key < sinks); }
// queries at positions p0 .. p1: their first and last one, and the edges of their windows
struct PromptSpan {
    int p0, p1, edge0, edge1, sinks;
};
constexpr PromptSpan prompt_span(int64_t p0, int64_t p1, int window, int sinks) { return {(int)p0, (int)p1, prompt_edge(p0, window), prompt_edge(p1, window), sinks}; }
// keys [k0, k0 + KT): does any of the queries see any of them (it may say yes for none), do all see all
constexpr bool prompt_some(const PromptSpan &s, int k0, int KT) { return k0 <= s.p1 && (k0 + KT - 1 > s.edge0 || k0 < s.sinks); }
constexpr bool prompt_all(const PromptSpan &s, int k0, int KT) { return k0 + KT - 1 <= s.p0 && (k0 > s.edge1 || k0 + KT - 1 < s.sinks); }
// Tiles of KT keys that the queries visit: the first `sink_tiles` ones, then those from `start` on, `count` in all
struct PromptTiles {
    int sink_tiles, start, count;
};
constexpr PromptTiles prompt_tiles(const PromptSpan &s, int KT) {
    if (s.p1 < 0) return {0, 0, 0};
    const int lo = s.edge0 + 1;                                       // the first key of any window
    const int stay = s.sinks <= s.p1 ? s.sinks : s.p1 + 1;
    int front = lo > 0 ? (stay + KT - 1) / KT : 0, start = lo / KT;
    if (front >= start) {
        if (front > 0) start = 0;
        front = 0;
    }
    return {front, start, front + s.p1 / KT + 1 - start};
}
constexpr int prompt_tile(const PromptTiles &t, int k) { return k < t.sink_tiles ? k : t.start + k - t.sink_tiles; }

}  // namespace sc
