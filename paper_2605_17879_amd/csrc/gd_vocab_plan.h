// Which tiles, pieces and parts the cross entropy over a vocabulary is worked out in: host arithmetic on sizes alone,
// without HIP, so that a test can compile it by itself.
#ifndef GD_VOCAB_PLAN_H_
#define GD_VOCAB_PLAN_H_

#include <stdint.h>

namespace vocab_plan {

constexpr uint32_t BK = 64;                       // elements of k staged at a time
constexpr uint64_t PIECE = 1ull << 28;            // the most elements of a piece of G
constexpr uint64_t PACK = 1ull << 27;             // the most elements of a packed piece of W
constexpr uint64_t MOST_TILES = 1ull << 23;       // of a launch: HIP takes less than 2^32 threads in a dimension

inline uint64_t up_to(uint64_t v, uint64_t unit) { return (v + unit - 1) / unit * unit; }

// Which tiles.  Large ones move half as much per product but come one to a CU, small ones two, and a launch ends with
// its last round: what a choice costs is rounds x (blocks of k + what a tile takes before and behind them) x the
// time of a block of all CUs at once (measured with long k: 1.5 us for 256 large tiles, 1.1 for 512 small ones).
constexpr uint64_t CUS = 256;
constexpr double LARGE_BLOCK = 1.5, SMALL_BLOCK = 1.1, AROUND = 7.0;
inline double large_cost(uint64_t tiles, double blocks) { return (double)((tiles + CUS - 1) / CUS) * (blocks + AROUND) * LARGE_BLOCK; }
inline double small_cost(uint64_t tiles, double blocks) { return (double)((tiles + 2 * CUS - 1) / (2 * CUS)) * (blocks + AROUND) * SMALL_BLOCK; }

// How many of `cols` go to large tiles where `rows` stand against them (a multiple of 256, or all of them): full rounds of
// large tiles, the rest in small ones, or one kind alone.
inline uint64_t large_part(uint64_t cols, uint64_t rows, uint64_t k) {
    const double blocks = (double)up_to(k, BK) / BK;
    const uint64_t across = up_to(rows, 256) / 256, all = up_to(cols, 256) / 256, small = up_to(rows, 128) / 128;
    uint64_t best = 0;
    double least = small_cost(small * (up_to(cols, 128) / 128), blocks);
    const double whole = large_cost(across * all, blocks);
    if (whole < least) { least = whole; best = cols; }
    const uint64_t full = across * all / CUS * CUS / across;     // tiles across `cols` in full rounds
    if (full > 0 && full < all) {
        const double both = large_cost(across * full, blocks) + small_cost(small * (up_to(cols - full * 256, 128) / 128), blocks) + 3.0;
        if (both < least) best = full * 256;
    }
    return best;
}

// The product with a long k and few tiles: parts of k, a slab of sums each, that the CUs have work alike.
struct split_plan {
    bool large;
    uint32_t splits;
};
inline split_plan split_for(uint64_t m, uint64_t n, uint64_t k) {
    const uint64_t blocks = up_to(k, BK) / BK;
    const uint64_t large = up_to(m, 256) / 256 * (up_to(n, 256) / 256), small = up_to(m, 128) / 128 * (up_to(n, 128) / 128);
    split_plan best{false, 1};
    double least = 1e30;
    for (uint32_t s = 1; s <= 64; ++s) {
        const double per = (double)((blocks + s - 1) / s);
        if (s > 1 && per < 8) break;
        const double sums = s * (double)m * (double)n * 8 / 4.9e6;       // a slab written and read
        const double l = large_cost(large * s, per) + sums, t = small_cost(small * s, per) + sums;
        if (l < least) { least = l; best = split_plan{true, s}; }
        if (t < least) { least = t; best = split_plan{false, s}; }
    }
    return best;
}

// Where rows and words make too few tiles for the chip, the waves' blocks of k in turn win: while tiles of 64 rows and
// 128 words are at most half as many as CUs (us, tiles of 128 x 128 / in turn, width 2 048: 128 rows x 8 000 words
// 37.9 / 33.4, x 16 000 43.1 / 58.2, 256 x 4 000 31.8 / 32.8, 512 x 2 000 32.1 / 32.6; width 4 096: 64 x 16 384
// 70.4 / 58.6, 4 x 32 768 77.1 / 76.1).
inline bool few_tiles(uint64_t n, uint64_t vocab) { return up_to(n, 64) / 64 * (up_to(vocab, 128) / 128) <= CUS / 2; }

// The words of a launch of the logits' sums: at most `want` of them and `most_tiles` tiles of 128 x 128, and whole large
// tiles where more words follow.
inline uint32_t words_at_once(uint64_t n, uint64_t vocab, uint64_t want, uint64_t most_tiles = MOST_TILES) {
    uint64_t words = most_tiles / (up_to(n, 128) / 128) / 2 * 256;
    if (words < 256) words = 256;
    if (want < words) words = want;
    return (uint32_t)(words < vocab ? words : vocab);
}

// Parts of the vocabulary that each row's sums come in, a tile each.
inline uint32_t parts_of_words(uint64_t words, uint64_t n, uint64_t k, bool few) {
    if (few) return (uint32_t)(up_to(words, 32) / 32);
    const uint64_t large = large_part(words, n, k);
    return (uint32_t)(up_to(large, 256) / 256 + (large < words ? up_to(words - large, 128) / 128 : 0));
}

}  // namespace vocab_plan

#endif  // GD_VOCAB_PLAN_H_
