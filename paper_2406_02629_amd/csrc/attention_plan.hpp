// Which kernels of attention_kernels.hip take a call and how it is cut up.  Plain C++, so that the rules can be checked without a GPU.
// SS_NLIMB: limbs of a field element (8, or 6 over the 45-bit prime).
#pragma once
#include <algorithm>
#include <stddef.h>

namespace SS_NS {

inline unsigned blocks_of(size_t a, size_t b) { return (unsigned)((a + b - 1) / b); }
inline size_t whole_256(size_t b) { return (b + 255) & ~(size_t)255; }

// ------------------------------------------------------------------ rotary positions

// What a rotation reads and writes, from which on it goes past the caches: heads of 128 turned whole, us, past / by way of them: 151 MB 25.7 / 22.2,
// 185 MB 28.8 / 31.7, 302 MB 44.7 / 48.8, 369 MB 53 / 66, 738 MB 106 / 125.
constexpr size_t STREAM_BYTES = (size_t)256 << 20;
// (messages and results past the caches where they are more than these hold)
inline bool rotary_streams(int n, int t, int tokens, int heads, int dim, int rot)
{
    return (size_t)tokens * heads * ((size_t)rot * (t + 1 + n) + (size_t)dim * 2 * n) * 8 > STREAM_BYTES;
}

// two elements at a time, 16 bytes to a load; aligned: the tensors to 16 bytes.  (us, so / one pair of a head to a thread.  Interleaved, 321 tokens
// of 12 heads of 80: n = 5 10.0 / 11.3, n = 3 7.4 / 8.3.  Halves, whose threads take two pairs: 512 tokens of 32 heads of 128, n = 3 27.3 / 27.9, n = 5
// 45.5 / 42.8; 256 15.1 / 15.9, 22.1 / 23.9; of 12 heads of 80, 640 11.8 / 10.4, 17.0 / 14.5, 321 8.5 / 7.9, 12.1 / 10.8, 64 5.2 / 5.1, 6.8 / 5.5: below
// about 600000 elements the pair to a thread would be the faster one there.  2048 tokens 93 / 118.)
inline bool wide_rotary(int dim, int rot, int interleaved, size_t ld, bool aligned)
{
    return (interleaved || rot / 2 % 2 == 0) && dim % 2 == 0 && ld % 2 == 0 && aligned;
}

// ------------------------------------------------------------------ appending to the cache

// Elements of the new keys from which on the kernel for many tokens takes them: tokens of 8 heads of 128, us, it / one thread per pair: n = 5, 128
// tokens 14.3 / 13.8, 256 20.9 / 25.6; n = 3 11.2 / 10.1, 13.8 / 16.3.  Those are one run of places; several runs leave whole cells only as far as the first
// one's phase holds, but the rest costs no more than there: 16 runs of 64 n = 5 87 / 143, n = 3 57 / 58, runs of 333, 700 and 1015 189 / 277, 127 / 189.
// Single tokens of many sequences, bytes on either side: 256 51.5 / 49.6, 31.4 / 30.4, 2048 1058 / 929, 640 / 571.
constexpr size_t WIDE_APPEND = (size_t)3 << 16;
inline bool wide_append(int tokens, int kv, int dim, int rot, size_t ld_k, bool aligned)
{
    return (size_t)tokens * kv * dim >= WIDE_APPEND && tokens >= 16 && rot / 2 % 4 == 0 && ld_k % 2 == 0 && aligned;
}

// ------------------------------------------------------------------ attention

constexpr size_t MAX_GROUPS = ((size_t)1 << 24) - 1;   // workgroups of 256 threads in a launch: less than 2^32 threads (the runtime cuts more off)
// Keys up to which one workgroup takes the softmax of a row, as many as its registers hold (the whole attention, us, so / in blocks of 1024 keys: 32
// rows of 1100 keys, n = 5, 36.3 / 43.3, of 4096 87.5 / 91.1, n = 3 52.2 / 56.6; 512 rows of 2048, n = 5, 115 / 127, of 4096 222 / 242; 2048 rows 734 / 790).
constexpr size_t SHORT_ROW = 4096;
constexpr int MAX_RUN = 16320;      // keys that the 32-bit sums of the values can take, in blocks of 64: 8 * 16383 * 2^14 < 2^31
constexpr int SHORT_KEYS = 256;     // that softmax and values in one launch hold

// how a call over `tokens` tokens is cut up: into slabs of tokens whose messages fit the room it has; the contraction of the values
// into `splits` runs of `run` keys, with a plane of their own each where there are several
struct attention_plan {
    int row_tiles;                // of 16 rows to a workgroup
    int slab;                     // tokens, 0: the room is too small
    int splits, run;
    int key_block;                // keys of a workgroup of the scores
    int dblocks;                  // workgroups to a head in the values, 64 elements each
    bool finish;                  // softmax and values in one launch
    size_t keys;                  // of a row in the messages: the longest context in whole blocks of 64
    size_t rows, bytes;           // of a slab
    bool split_rows;              // the softmax of a row in several workgroups
    size_t query_bytes;           // of LDS for the digits of a tile's queries
};

// most tiles of `rows` rows that the sequences of a call can have
inline size_t tile_bound(size_t tokens, size_t seqs, size_t group, size_t rows)
{
    const size_t one = tokens * blocks_of(group, rows), all = tokens * group / rows + seqs;
    return one < all ? one : all;
}

inline attention_plan plan_attention(int n, int t, int tokens, int seqs, int heads, int kv, int dim, int max_length, size_t room)
{
    attention_plan p = {};
    const size_t group = heads / kv, nr = 2 * t + 1;
    p.keys = ((size_t)max_length + 63) & ~(size_t)63;
    p.dblocks = blocks_of(dim, 64);
    // (a run of tokens is planned as a call of as many: a single token always fits into what a call of one needs)
    for (p.slab = tokens;; p.slab = (p.slab + 1) / 2) {
        // Larger tiles and blocks read less, but leave fewer waves to a SIMD and fewer workgroups.  The whole attention, us, tiles of 32 / of 16 rows
        // (by the workgroups of the scores with 32), chunks of 64 to 512 tokens of 16 heads over 4 of 128: n = 5, (320) 126 / 106, (720) 210 / 210,
        // (1280) 368 / 368, (1920) 520 / 536, (2560) 673 / 699, (7680) 1980 / 2065, (10400) 2572 / 2693; n = 3 (432) 155 / 142, (1152) 330 / 320, (1536) 398 / 398,
        // (4608) 1192 / 1209, over the 45-bit prime 137 / 122, 269 / 271, 336 / 333, 1000 / 1042; chunks of 17 to 121 over 121 to 777, heads of 80, n = 5
        // (1160) 174 / 154; 230 tokens over 700 to 1024, n = 3, 45-bit prime (480) 88 / 74.  Keys to a workgroup, 128 / 256 / 512 / 1024: single tokens over 32768
        // 333 / 335 / 342 / 343, over 500 to 2001 189 / 193 / 204 / 203; 512 tokens over 4096 2757 / 2638 / 2577 / 2577, the last two 162 / 155 / 154 / 154 and
        // 74.5 / 72.2 / 74.5 / 76.8 (there 1024 leaves 384 workgroups for 768 places).
        const size_t sequence_rows = blocks_of(p.slab, seqs) * group;
        auto tiles = [&](size_t rows) { return tile_bound(p.slab, seqs, group, rows); };
        auto workgroups = [&](size_t rows, size_t block) { return tiles(rows) * blocks_of(p.keys, block) * kv * nr; };
        p.row_tiles = sequence_rows > 16 && workgroups(32, 512) >= 2048 ? 2 : 1;
        p.key_block = sequence_rows > 16 ? 1024 : 128;
        while (p.key_block > 256 && workgroups(16 * p.row_tiles, p.key_block) < (p.row_tiles == 2 ? 4096 : 768)) p.key_block /= 2;
        // one launch for softmax and values while each of its workgroups has a CU to itself (us, one launch / two): single tokens of 32 heads of
        // 128 over 64 keys, n = 5, one sequence 15.9 / 17.8, 4 16.9 / 19.9, 16 (800 workgroups) 33.1 / 33.5, 64 103 / 97; over 256 keys, one
        // 21.8 / 22.4
        p.finish = p.row_tiles == 1 && p.keys <= SHORT_KEYS && tiles(16) * kv * n <= 256;
        // single tokens read the values once, which several rounds of workgroups spread best over the memory (us, 2048 / 1024 workgroups wanted:
        // 87 / 98); chunks multiply, and a round of 384 that needs no sum is as good as three runs (20.4 / 19.5 + 5.2 for the sum)
        const size_t wanted = blocks_of(sequence_rows <= 16 ? 2048 : 384, tiles(16 * p.row_tiles) * p.dblocks * kv * n);
        p.run = (int)((blocks_of(p.keys, wanted) + 63) & ~63u);
        if (p.run > MAX_RUN) p.run = MAX_RUN;
        if (p.run < 256) p.run = 256;
        p.splits = p.finish ? 1 : (int)blocks_of(p.keys, p.run);
        p.rows = (size_t)p.slab * heads;
        p.split_rows = p.keys > SHORT_ROW;
        p.query_bytes = (size_t)p.row_tiles * p.dblocks * SS_NLIMB * 1024;
        const size_t blocks = p.split_rows ? blocks_of(p.keys, 1024) : 0;
        p.bytes = whole_256(nr * p.rows * p.keys * 8) + (blocks ? whole_256(p.rows * (p.keys + 2 * blocks) * 8) : 0) +
                  (p.finish ? 0 : whole_256((size_t)n * p.rows * p.keys * SS_NLIMB)) + (p.splits > 1 ? whole_256((size_t)p.splits * n * p.rows * dim * 8) : 0);
        const size_t most = std::max(std::max(workgroups(16 * p.row_tiles, p.key_block), tiles(16 * p.row_tiles) * kv * n * p.splits * p.dblocks),
                                     std::max(p.rows * std::max(blocks, (size_t)1), (size_t)blocks_of(p.rows * dim, 256 / (p.splits > 8 ? 4 : 1)) * n));
        if (p.bytes <= room && most <= MAX_GROUPS) return p;
        if (p.slab == 1) break;
    }
    p.slab = 0;
    return p;
}

}  // namespace SS_NS
