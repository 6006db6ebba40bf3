// How the calls of adapter_kernels.hip and sample_kernels.hip are cut up.  Plain C++, so that the rules can be checked without a GPU.
// SS_NLIMB: limbs of a field element (8, or 6 over the 45-bit prime).
#pragma once
#include <algorithm>
#include <stddef.h>

namespace SS_NS {

inline size_t div_up(size_t a, size_t b) { return (a + b - 1) / b; }

// ------------------------------------------------------------------ low-rank adapters

// An adapter lies in memory as the digits of its two matrices:
//   down [2t+1][K / 64][limb][4][rank][16] int8: byte b of quarter q is element k = 64 block + 8 (b / 2) + 2 q + b % 2 of the contraction, so
//     that four lanes find 8 elements of a row of x in 64 bytes; past K zeros
//   up [n][N / 32][2][limb R / 16][16][16] int8: column 32 block + 2 c + h is number c of half h, whose 16 bytes of a chunk are consecutive digits
//     in the order limb, rank (R: 8, or the rank in whole sixteens, zeros behind it); past N zeros
inline size_t padded_rank(size_t rank) { return rank <= 8 ? 8 : (rank + 15) & ~(size_t)15; }
inline size_t up_steps(size_t rank) { return div_up(SS_NLIMB * padded_rank(rank), 64); }   // products that the digits of a column take
inline size_t down_party_bytes(int K, int rank) { return div_up(K, 64) * SS_NLIMB * 64 * rank; }
inline size_t up_party_bytes(int rank, int N) { return div_up(N, 32) * 2 * SS_NLIMB * padded_rank(rank) * 16; }

constexpr size_t MAX_SERVING_GROUPS = ((size_t)1 << 24) - 1;   // workgroups of 256 threads in a launch: less than 2^32 threads
// Tensors that the caches do not hold: read and written past them (second product, us, past / by way of them: 2048 tokens by 4096 columns, n = 5, 671 MB, rank 16
// 156 / 158, rank 64 300 / 310; n = 3, 403 MB, 86.8 / 93.6; 134 MB 62.2 / 60.8, 49 MB 23.8 / 22.8)
constexpr size_t STREAMED_BYTES = (size_t)256 << 20;
constexpr int MAX_PLANES = 8;                                  // partial sums of the first product, which the reduction adds

constexpr int DOWN_ROWS = 16, UP_ROWS = 16, UP_TILE_ROWS = 64;   // tokens to a tile of the first product, of the second by either kernel

struct adapter_plan {
    bool grouped;                 // tiles of tokens that share an adapter, whichever requests they belong to
    bool apart;                   // every wave of the first product has a tile of its own
    bool diagonals;               // the second product over limbs and rank together
    int splits, run;              // contraction of the first product: in `splits` runs of `run` blocks of 64
    bool streams;                 // the second product's tensors go past the caches
    int col_groups;               // workgroups that share the columns of a tile of the second product
    size_t messages, planes, z;   // bytes: of the reduction's messages, of the first product's planes, of its reduced result
    size_t down_tiles, up_tiles;  // most that there can be
    size_t down_groups, up_groups, bytes;
};

// most tiles of `rows` tokens that requests can have
inline size_t request_tiles(size_t tokens, size_t requests, size_t rows, bool grouped)
{
    return grouped ? tokens : std::min(tokens, tokens / rows + requests);
}

inline adapter_plan plan_adapters(int n, int t, int tokens, int requests, int K, int rank, int N)
{
    adapter_plan p = {};
    const size_t nr = 2 * t + 1, k = t + 1, count = (size_t)tokens * rank, blocks = div_up(K, 64);
    // Tokens by their adapters, although every workgroup goes through the requests then, and those of tokens that are in another's tile for nothing (first and
    // second product, us, so / request by request: 128 requests of a token with 27 adapters between them, n = 3, 23 + 61 / 35 + 103, with an adapter each
    // 44 + 140 / 43 + 139; 64 with 8, n = 5, 24 + 23 / 28 + 30; 400 with 8 72 + 94 / 124 + 89; 8 with 8 10.0 + 7.9 / 9.2 + 7.7.  Of two tokens each, 64 with 27,
    // n = 3, 23 + 75 / 30 + 66; of four each, 32 with 4, n = 5, 48 + 66 / 23 + 26).  It goes by the whole call, so that one long request leaves single tokens with a
    // tile each (8 adapters, rank 16, n = 5, whole calls: 512 tokens 81, 64 single ones 53, together in a call 113).  Beyond 1024 requests the searches cost what the
    // fewer reads save (single tokens with 8 adapters, whole calls: 1024 519, 1025 526).
    p.grouped = requests > 1 && requests <= 1024 && tokens <= 2 * requests;
    // Limbs and rank together, or diagonals apart (second product, us: 2048 tokens by 4096 columns, n = 5, rank 8 135 / 265, 16 157 / 274, 32 241 / 278; 1000
    // by 1024, n = 3, rank 32 22.8 / 23.7).  Beyond rank 32 two sums no longer fit 32 bits.  The rule does not tell the primes apart, though over the 45-bit
    // one the form that it takes for ranks 17 to 32 is the slower where it was measured (37 to 333 tokens by 2560, rank 32, 35.6 / 28.0).
    p.diagonals = rank <= 32;
    p.down_tiles = request_tiles(tokens, requests, DOWN_ROWS, p.grouped);
    // A block of 64 elements takes a CU so long, a workgroup half a microsecond beside its blocks, the reduction 0.3 for each plane.  First product, us, by runs:
    // 64 tokens of 4096, rank 16, n = 5, 1 19, 2 13, 4 9.9, 6 9.6, 8 10.7 (reduction 4.0 to 6.2); 128 tokens, rank 32, 1 30, 2 23, 4 27; 2048 tokens, rank
    // 16, 1 112, 2 101, 3 103; 37 to 333 tokens, rank 64, 45-bit prime, 1 19, 2 12.5, 4 11.8; 668 tokens, rank 128, 1 133, 2 114, 3 124, 4 110, 5 99.
    const double block = rank <= 16 ? 0.25 : rank <= 32 ? 0.5 : rank <= 64 ? 1.0 : 2.0;
    auto cost = [&](size_t s, int own) { return div_up(div_up(p.down_tiles, own) * nr * s, 256) * (own * block * div_up(blocks, s) + 0.5) + 0.3 * s; };
    p.splits = 1;
    for (size_t s = 2; s <= MAX_PLANES && s * 6 <= blocks; s++)
        if (cost(s, 1) < cost(p.splits, 1)) p.splits = (int)s;
    // Where there are many tiles each wave has its own, goes through all the blocks of its run, and adds its sums to nobody's (us, so / four waves to a tile: 2048
    // tokens of 4096, n = 5, 3 runs 89 / 103, 2 117, 4 110; 1000 47 / 53; 16384 of 64 25 / 71; 8192 of 256 33 / 44; 5000 of 512, n = 3, 22 / 25; 512 of
    // 4096, whose cost is more, 36 / 28).
    const double together = cost(p.splits, 1);
    for (size_t s = 1; rank <= 16 && !p.grouped && s <= MAX_PLANES && (s == 1 || s * 6 <= blocks); s++)
        if (cost(s, 4) < (p.apart ? cost(p.splits, 4) : together)) p.splits = (int)s, p.apart = true;
    p.down_tiles = request_tiles(tokens, requests + 1, DOWN_ROWS, p.grouped);   // with those of tokens that no request has
    p.run = (int)div_up(blocks, p.splits);
    p.splits = (int)div_up(blocks, p.run);
    p.down_groups = div_up(p.down_tiles, p.apart ? 4 : 1) * nr * p.splits;
    p.up_tiles = request_tiles(tokens, requests, p.diagonals ? UP_ROWS : UP_TILE_ROWS, p.grouped);
    const size_t units = div_up(N, p.diagonals ? 128 : 32), per_tile = p.diagonals ? div_up(units, 4) : units;
    // Workgroups with the diagonals apart stage their tile's digits for some 10 us and take 3 for 32 columns; two of them fit a CU.  What fills the chip once
    // is best while each of them has few columns (us, 37 to 333 tokens, 2560 columns, rank 64, 45-bit prime, by workgroups to a tile: 8 46.8, 16 30.4, 20 42.1,
    // 40 41.0; 100 to 401 tokens, 1024 columns, rank 128: 4 52.8, 8 43.3, 16 53.4); long ones are as good in several rounds (2048 tokens,
    // 4096 columns, rank 64, n = 5: 4 336, 8 298, 20 306, 64 362).
    const double full = n * ((double)tokens / UP_TILE_ROWS + requests * 0.5);   // tiles, about
    size_t wanted = (size_t)(512 / full);
    if (p.diagonals || wanted < 1 || units > 16 * wanted) wanted = div_up(2048, p.up_tiles * n);
    p.col_groups = (int)std::max<size_t>(1, std::min(wanted, per_tile));
    p.up_groups = p.up_tiles * n * p.col_groups;
    p.streams = (size_t)n * tokens * N * 16 > STREAMED_BYTES;
    auto whole = [](size_t b) { return (b + 255) & ~(size_t)255; };
    p.messages = whole((nr * k + k * n + k + n) * count * 8);
    // (room for as many as any number of tokens asks for, so that the room of a larger call holds a smaller one; a call that takes one run leaves up to seven
    // parts of eight unused)
    p.planes = whole(std::max<size_t>(1, std::min<size_t>(MAX_PLANES, blocks / 6)) * nr * count * 8);
    p.z = whole((size_t)n * count * 8);
    p.bytes = p.messages + p.planes + p.z;
    return p;
}

// ------------------------------------------------------------------ sampling

constexpr int SMALL_VOCAB = 8192;             // tokens whose logits one workgroup holds,
constexpr int MEDIUM_VOCAB = 32768;           // alone on its CU
constexpr int SAMPLE_BIN_BITS = 11, SAMPLE_BINS = 1 << SAMPLE_BIN_BITS;
constexpr int SAMPLE_OPEN = 1024;             // tokens to a workgroup that opens (us at 512, 1024, 2048: 1 row of 32000 3.5, 4.2, 5.5;
                                              // 256 of them 31.8, 32.7, 37.6; 64 of 200003 64.6, 60.2, 63.7)
constexpr int SAMPLE_CHUNK = 512;             // to a wave that counts or collects: 2^20 tokens are 2048 chunks
constexpr int SAMPLE_LIST = 4096;             // tokens near a cut that are listed (more are found among all, by one workgroup: 1 row of 2^20 tokens, normal logits of
                                              // deviation 2.5, top_p 0.99 746 us, top_k 50, whose list has room, 32; 2^18 tokens, top_p 0.99 33)
constexpr int SAMPLE_PLAN = 64;                // bytes for where the cuts of a row lie
constexpr size_t SAMPLE_ROOM = (size_t)512 << 20;

struct sample_plan {
    bool small;                   // one launch, a workgroup to a row
    int slab;                     // rows at a time, 0: the room is too small
    int opens, groups;            // workgroups of a row that open, that count
    int chunks, key_ld;           // of a row; its keys with what fills the last 16 bytes
    size_t bytes;
};

inline sample_plan plan_sample(int rows, int vocab, size_t room)
{
    sample_plan p = {};
    // One launch or four, us: 1 row of 4096 tokens 13.5 / 25.2, of 8192 17.6 / 26.7, 256 rows of 2048 16.1 / 32.5, of 8192 24.6 / 38.4, 1000 68 / 102.  Beyond, a
    // workgroup has a CU to itself and a row of 32000 takes it 58 us: 1 row of 16384 25.0 / 24.9, of 32000 38.2 / 25.0; 32 rows 32.3 / 30.0 and 57.6 / 32.1; 128
    // 34.1 / 36.8 and 58.6 / 49.6; 256 of 32000 62.6 / 75.1, 300 106 / 88.
    p.small = vocab <= SMALL_VOCAB || (vocab <= MEDIUM_VOCAB && div_up(rows, 256) * (10.0 + vocab / 640.0) < 22.0 + rows * (vocab / 150000.0));
    p.slab = rows;
    if (vocab <= SMALL_VOCAB) return p;
    p.opens = (int)div_up(vocab, SAMPLE_OPEN);
    p.chunks = (int)div_up(vocab, SAMPLE_CHUNK);
    p.groups = (int)std::min(div_up(p.chunks, 16), div_up(512, rows));
    p.key_ld = (vocab + 3) & ~3;
    const size_t row = (size_t)SAMPLE_BINS * 12 + (size_t)((p.chunks + 1) & ~1) * 8 + (size_t)SAMPLE_LIST * 8 + (size_t)p.key_ld * 4 + (size_t)p.opens * 4 +
                       SAMPLE_PLAN + 4;
    const size_t most = std::max<size_t>(1, std::min(room, SAMPLE_ROOM) / row);
    p.slab = (int)std::min<size_t>(std::min<size_t>(rows, most), MAX_SERVING_GROUPS / p.opens / 4);
    p.bytes = p.slab * row;
    if (p.small)                                  // (which needs no room; less rows may)
        p.slab = rows;
    else if (p.bytes > room)
        p.slab = 0;
    return p;
}

}  // namespace SS_NS
