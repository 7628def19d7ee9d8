// How a launch of the attention over the paged cache is cut.  On its own so that the host can check it.
#pragma once

#define PG_MAX_SPLIT 16

struct PagedChoice {
    int rows;       // query rows per CTA: 32, 64, 128 or 256
    int splits;     // of the keys: CTAs of a cluster
};

// blocks: query blocks of all (sequence, head) pairs; tiles: of the longest sequence, with the tree's; cap[s]: CTAs that run at once in clusters of s.
inline int paged_splits(int blocks, int sm_count, int tiles, const int* cap) {
    if (blocks > sm_count && tiles <= 128) return 1;
    int best = 1;
    long best_cost = 0;
    for (int s = 1; s <= PG_MAX_SPLIT && s <= tiles; ++s) {
        if (s > 1 && cap[s] <= 0) continue;
        const long ctas = (long)blocks * s, at_once = cap[s] > 0 ? cap[s] : sm_count;
        const long waves = (ctas + at_once - 1) / at_once;
        const long cost = waves * (2 * ((tiles + s - 1) / s) + 20 + (s > 1 ? 8 : 0));
        if (s == 1 || cost < best_cost) { best_cost = cost; best = s; }
    }
    return best;
}

// pairs: (sequence, kv head); rows: query rows of one pair.
// (Times back to back, inputs rotating.)
// Few rows: a block of 32 or 64 holds them four times or twice over, each copy a part of a tile's columns.  Tokens without drafts (four rows), 32 sequences of 1024 to 8192:
// 80 us in blocks of 32, 93 in blocks of 64, 106 of 128; one token behind 512: 7.9, 8.1, 9.5.  Trees of 16 (64 rows) behind 2048 tokens, 32 sequences: 58 us in blocks of 64, 65 of 128;
// one: 12.2 and 13.2.
// More than 128 rows: a CTA of 256 converts a tile of values once for both halves and takes 1.7 times (short prefixes) to 2 times (long ones) as long as one of 128,
// so it is taken where blocks of 128 need twice the rounds of the machine.  64 heads over 8, trees of 62, 4096 tokens: 8 sequences 102 us against 110, 4 sequences 99 against 58;
// 32 heads over 8, trees of 60, 2048 tokens: 16 sequences 61 against 67, 8 sequences 58 against 36.
// Splits: one token behind 32768 takes 42 us with 8 CTAs a head, 58 with 11 and 49 with 16 (which do not all fit at once); a tree of 60 behind 2048 tokens 17.0 with 6 and 19.0 with 4;
// single tokens behind 1000 to 4000, 8 sequences, 26 with 2 and 39 with 1.
inline PagedChoice paged_choice(int pairs, int rows, int sm_count, int tiles, const int* cap) {
    PagedChoice c;
    auto rounds = [&](int r) { return (pairs * ((rows + r - 1) / r) + sm_count - 1) / sm_count; };
    c.rows = rows <= 32 ? 32 : rows <= 64 ? 64 : rows > 128 && rounds(128) >= 2 * rounds(256) ? 256 : 128;
    c.splits = paged_splits(pairs * ((rows + c.rows - 1) / c.rows), sm_count, tiles, cap);
    return c;
}
