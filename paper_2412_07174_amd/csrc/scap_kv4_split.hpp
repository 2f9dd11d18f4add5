// How an attention call over the 4-bit cache cuts the key axis: the arithmetic that every workgroup does on the device, in plain C++, so that it
// can be checked on the host at the ends of its ranges.
//
// A row block is worth its sequence's range of tokens.  Chunks are at least 1 / places of all work, places being the workgroups of a head that run at
// once.  Only blocks longer than a chunk are cut, so fewer than `places` of them are, into at most 2 * places pieces: the room for partial
// results and arrival counters (2 * (places + 2) and places + 2 a head) rests on that, and so does the grid (blocks + places + 2 a
// head).  The additional two cover the rounding of sums of 2^20 sequences in fp32.
#pragma once

#include <cstdint>

namespace scap {

constexpr int kKv4MaxRange = 1 << 30;  // tokens of a sequence, at most

// Tokens of a chunk where `left` of them are to take `total`.  No less than the longest sequence where it is bounded from above: a smaller bound
// would cut more blocks than there are places.
constexpr int kv4_chunk(float total, int left, int min_chunk) {
    const float c = total / (float)left + 1.f;
    const int n = c < (float)kKv4MaxRange ? (int)c : kKv4MaxRange;
    return n > min_chunk ? n : min_chunk;
}

// Chunks of a sequence's row blocks.  One where its rows exceed what a slot of the workspace holds, or with one place, which has no slots.
// inv: 1 / chunk.
constexpr int kv4_cut(int range, int rows, int chunk, float inv, int places, int slot_rows) {
    if (places <= 1 || rows > slot_rows) return 1;
    int c = (int)((float)range * inv);
    c += (int64_t)c * chunk < range;
    c -= (int64_t)(c - 1) * chunk >= range;
    return c > 1 ? c : 1;
}

// Chunks of c tokens make at most total / c + n workgroups of every head, and n / 2 fewer as a rule.  As many as run at once are wanted, and not a
// few more, which would run alone behind them: the shortest chunk of three that keeps to that.  items(chunk, 1 / chunk): workgroups of a head.
template <typename F>
constexpr int kv4_choose_chunk(float total, int n, int places, int min_chunk, float& inv, F items) {
    int chunk = 0;
    for (int spare = 0; spare < 3; ++spare) {
        const int left = places - n * spare / 2;
        if (spare > 0 && left <= 0) break;  // more rows' blocks than places: several rounds in any case
        chunk = kv4_chunk(total, left, min_chunk);
        inv = 1.f / (float)chunk;
        if (items(chunk, inv) <= places) break;
    }
    return chunk;
}

}  // namespace scap
