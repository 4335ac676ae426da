// Which kernel attends over the 4-bit cache, and in which order it adds a row's keys (host code alone).
#pragma once
#include <algorithm>
#include <cstdint>

// Waves that share pairs (1: the kernel for prompts, whose waves have pairs of their own), key chunks and their length in tiles
struct Kv4Order { int kw, chunks, chunk_tiles; };
// `pairs` (row, head) pairs of a KV head, a bound or what stands for it; fixed: the order must not depend on the rows of a call, only
// on these numbers.  A compute unit holds eight waves, two a SIMD, of these registers:
//   more than 64 pairs, and waves with 32 of their own fill the chip: nothing is shared (kw 1; us of 4 prompts of up to 2048 rows, 12 heads, 106, with kw
//     2 119; of 16 of 400 25 | 35).  The four waves of such a workgroup decode tiles for each other, so three of them at least have to have
//     pairs (512 x 2 KV heads over 700 tokens, 66 pairs: 72 us, with kw 2 91; 96: 75 | 90; but 54: 73 | 54, and 256 x 8, 64 pairs: 130 | 91, 20: 115 |
//     53, 4: 89, with kw 4 43)
//   up to 16 pairs: eight waves a workgroup where that is not more than fill the chip (one sequence of 700 tokens, 9 / 3 heads: 6.9, with four
//     8.5; 64 of 2300, 12 / 2: 15.3 | 17.6), else four (256 of 700, 16 / 2: 14.1, with eight 18.4, with two 18.1)
//   else two, and key chunks until the waves fill the chip.  (Few sequences pay for that with a second launch: one of 768 tokens, 9 / 3 heads of 64, 15
//     pairs 7.2 us, 18 pairs 11.8, 27 11.6; 64 of them 7.6 | 14.9; one of 8192, 16 / 2 of 128, 16 pairs 14.7, 24 15.1)
inline Kv4Order kv4_order(int64_t batch, int kv_heads, int64_t pairs, int64_t max_kv, int most_chunks, bool fixed) {
    constexpr int64_t kWaves = 2048;                        // two a SIMD
    const int64_t heads = batch * kv_heads, tiles = (max_kv + 31) / 32;
    Kv4Order o{2, 1, 1 << 26};
    const int64_t row_waves = (pairs + 31) / 32;
    if (!fixed && pairs > 64 && row_waves * heads >= kWaves) {
        o.kw = 1;
        return o;
    }
    if (!fixed && pairs <= 16) o.kw = heads * 8 <= kWaves ? 8 : 4;
    const int64_t want = std::clamp<int64_t>((kWaves + heads * row_waves * o.kw - 1) / (heads * row_waves * o.kw), 1, most_chunks);
    const int64_t per = std::max<int64_t>((tiles + want - 1) / want, 4 * o.kw);      // four tiles a wave at least
    if (tiles > per) {
        o.chunks = (int)((tiles + per - 1) / per);
        o.chunk_tiles = (int)per;
    }
    return o;
}
