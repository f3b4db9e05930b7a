// sc_prompt_attn as its launcher sees it (internal; the public boundary is include/semanticache.h), and which keys a tile of queries visits.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace sc {

// ---- plain functions, so that the host can try them
// Tiles of `KT` keys that queries at positions p0 .. p1 visit: the first `sink_tiles` ones, then those from `start` on, `count` in all
struct PromptTiles {
    int sink_tiles, start, count;
};
constexpr PromptTiles prompt_tiles(int64_t p0, int64_t p1, int64_t window, int64_t sinks, int KT) {
    if (p1 < 0) return {0, 0, 0};
    const int64_t lo = window > 0 && p0 - window + 1 > 0 ? p0 - window + 1 : 0;      // the first key of any window
    const int64_t stay = sinks < p1 + 1 ? sinks : p1 + 1;
    int64_t front = lo > 0 ? (stay + KT - 1) / KT : 0, start = lo / KT;
    if (front >= start) {
        front = 0;
        if (lo > 0 && stay > 0) start = 0;
    }
    return {(int)front, (int)start, (int)(front + p1 / KT + 1 - start)};
}
constexpr int prompt_tile(const PromptTiles &t, int k) { return k < t.sink_tiles ? k : t.start + k - t.sink_tiles; }
// keys [k0, k0 + KT): does any of the queries at p0 .. p1 see any of them (it may say yes for none), do all see all
constexpr bool prompt_some(int64_t k0, int64_t p0, int64_t p1, int64_t window, int64_t sinks, int KT) {
    return k0 <= p1 && (window <= 0 || k0 + KT - 1 > p0 - window || k0 < sinks);
}
constexpr bool prompt_all(int64_t k0, int64_t p0, int64_t p1, int64_t window, int64_t sinks, int KT) {
    return k0 + KT - 1 <= p0 && (window <= 0 || k0 > p1 - window || k0 + KT <= sinks);
}
constexpr bool prompt_sees(int64_t pos, int64_t key, int64_t window, int64_t sinks) { return key <= pos && (window <= 0 || key > pos - window || key < sinks); }

}  // namespace sc
