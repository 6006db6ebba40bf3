// Low-rank adapters of many requests beside a projection that they share, on shares.  A request's tokens x take its adapter (A [K][rank],
// B [rank][N]):
//   1. parties i = 1..2t+1: Z_i = x_i A_i mod p (degree 2t, 2 f fraction bits), the contraction cut into runs with a plane of sums each
//   2. degree reduction and truncation of Z (the reduction's own kernel, which adds the planes) -> z, degree t, f fraction bits
//   3. every party: y_i = base_i + z_i B_i mod p (degree 2t), base being the shared projection's product
// Products run on int8 MFMA over balanced 8-bit digits, as in a dense layer.
#include "kernels.hpp"
#include "digits.hpp"
#include "diagonals.hpp"
#include "truncation.hpp"
#include "lanes.hpp"

namespace SS_NS {

namespace {

constexpr int BLOCK = 256;

typedef const int __attribute__((address_space(4))) *constant_ints;
__device__ __forceinline__ int fixed_at(const int *p, size_t i) { return ((constant_ints)(uintptr_t)p)[i]; }

// ------------------------------------------------------------------ laying an adapter out

// 16 elements of a column of A to a thread (down, see serving_plan.hpp).  a [.][K][given] of each party; given <= rank, the rest is zero.
__global__ __launch_bounds__(BLOCK) void pack_down_kernel(const u64 *a, signed char *down, int K, int given, int rank, unsigned items, size_t party_bytes)
{
    const unsigned i = blockIdx.x * BLOCK + threadIdx.x;
    if (i >= items) return;
    const int party = blockIdx.y, r = (int)(i % (unsigned)rank), q = (int)(i / (unsigned)rank & 3), kb = (int)(i / (unsigned)rank >> 2);
    u64 y[4][4];
#pragma unroll
    for (int b = 0; b < 16; b++) {
        const int k = 64 * kb + 8 * (b >> 1) + 2 * q + (b & 1);
        y[b >> 2][b & 3] = balanced_digits(k < K && r < given ? a[((size_t)party * K + k) * given + r] : 0);
    }
    signed char *dst = down + party * party_bytes + ((size_t)kb * SS_NLIMB * 4 + q) * rank * 16 + (size_t)r * 16;
#pragma unroll
    for (int l = 0; l < SS_NLIMB; l++)
        *reinterpret_cast<v4i *>(dst + (size_t)l * 4 * rank * 16) =
            (v4i){(int)limb_dword(y[0], l), (int)limb_dword(y[1], l), (int)limb_dword(y[2], l), (int)limb_dword(y[3], l)};
}

// 16 digits of a column of B to a thread (up).  b [n][given][N]; padded: the rank in whole eights.  Every element is read and split once for each limb, which
// happens when an adapter is loaded, not when it is used (4096 by 4096, n = 5, both matrices: rank 16 10.7 us, rank 64 26; 960 by 2560, rank 64,
// n = 3, 45-bit prime 10.7).
__global__ __launch_bounds__(BLOCK) void pack_up_kernel(const u64 *b, signed char *up, int given, int padded, int N, unsigned items, size_t party_bytes)
{
    const unsigned i = blockIdx.x * BLOCK + threadIdx.x;
    if (i >= items) return;
    const unsigned chunks = (unsigned)(SS_NLIMB * padded / 16);
    const int party = blockIdx.y, c = (int)(i & 15), chunk = (int)(i / 16 % chunks), half = (int)(i / 16 / chunks);
    const int col = 32 * (half >> 1) + 2 * c + (half & 1);
    u32 d[4] = {0, 0, 0, 0};
    for (int e = 0; e < 16; e++) {
        const int at = chunk * 16 + e, limb = at / padded, r = at - limb * padded;
        const u64 x = r < given && col < N ? b[((size_t)party * given + r) * N + col] : 0;
        d[e >> 2] |= ((u32)(balanced_digits(x) >> (8 * limb)) & 255) << (8 * (e & 3));
    }
    *reinterpret_cast<v4i *>(up + party * party_bytes + (size_t)i * 16) = (v4i){(int)d[0], (int)d[1], (int)d[2], (int)d[3]};
}

// ------------------------------------------------------------------ products

struct adapter_args {
    const int *start, *adapter;     // [requests + 1], [requests]
    int requests, tokens, adapters, grouped;
    int K, rank, padded, N;
    const signed char *down, *up;
    size_t down_party, up_party, down_bytes, up_bytes;   // of a party, of an adapter
    const u64 *x, *base;
    size_t ld_x, ld_base, ld_y;
    u64 *planes, *y;                // planes [splits][2t+1][tokens][rank]
    const u64 *z;                   // [n][tokens][rank]
    int nr, n, run, col_groups;
    unsigned tiles;                 // that there can be
    fdiv dTiles;
    size_t plane;                   // 2t+1 shares
};

// the tokens of a tile, all with one adapter
struct row_tile {
    int count, adapter;             // adapter: -1 if they have none
};

// Tile number -> its tokens, `most` at most, to rows in LDS (the wave's own, or everyone's after the next barrier).  False: no such tile.
// Tiles follow one another request by request, or (grouped) tile i is that of token i, which has the tokens behind it with the same adapter too, whichever requests
// they belong to, if the number of those in front of it is a multiple of `most`, and is none otherwise: requests of single tokens read an adapter that they
// share once.
// OUTSIDE: tokens that no request has (in front of the first, behind the last) have tiles too, without an adapter, behind the others.
template <bool OUTSIDE>
__device__ __forceinline__ bool find_rows(const adapter_args &g, int tile, int most, int *rows, row_tile &r)
{
    const int lane = threadIdx.x & 63;
    auto request = [&](int b, int &first, int &count, int &adapter) {
        first = count = 0, adapter = -1;
        if (b >= g.requests) return;
        first = min(max(g.start[b], 0), g.tokens);
        count = max(0, min(g.start[b + 1], g.tokens) - first);
        adapter = g.adapter[b];
        if (adapter < 0 || adapter >= g.adapters) adapter = -1;
    };
    auto keep = [&](int first, int count, int adapter) {
        r = {__builtin_amdgcn_readfirstlane(min(most, count)), __builtin_amdgcn_readfirstlane(adapter)};
        if (lane < r.count) rows[lane] = first + lane;
        return true;
    };
    auto outside = [&](int number) {
        const int begin = min(max(fixed_at(g.start, 0), 0), g.tokens), inside = max(0, min(fixed_at(g.start, g.requests), g.tokens) - begin);
        const int at = number * most, left = g.tokens - inside - at;
        if (!OUTSIDE || left <= 0) return false;
        r = {min(most, left), -1};
        if (lane < r.count) rows[lane] = at + lane < begin ? at + lane : at + lane + inside;
        return true;
    };
    int first, count, adapter;
    if (g.requests == 1) {                       // without a search
        first = min(max(fixed_at(g.start, 0), 0), g.tokens), count = min(fixed_at(g.start, 1), g.tokens) - first;
        adapter = fixed_at(g.adapter, 0);
        if (tile * most >= count) return outside(tile - (max(count, 0) + most - 1) / most);
        return keep(first + tile * most, count - tile * most, adapter < 0 || adapter >= g.adapters ? -1 : adapter);
    }
    if (!g.grouped) {
        int base = 0;
        for (int b0 = 0; b0 < g.requests; b0 += 64) {
            request(b0 + lane, first, count, adapter);
            const int mine = (count + most - 1) / most, upto = (int)wave_upto((u32)mine);
            const unsigned long long past = __ballot(base + upto > tile);
            if (past) {
                const int l = __ffsll((long long)past) - 1, at = (tile - base - __builtin_amdgcn_readlane(upto - mine, l)) * most;
                return keep(__builtin_amdgcn_readlane(first, l) + at, __builtin_amdgcn_readlane(count, l) - at, __builtin_amdgcn_readlane(adapter, l));
            }
            base += __builtin_amdgcn_readlane(upto, 63);
        }
        return outside(tile - base);
    }
    int owner = -1, wanted = -1, place = 0;
    for (int b0 = 0; b0 < g.requests && owner < 0; b0 += 64) {
        request(b0 + lane, first, count, adapter);
        const unsigned long long mine = __ballot(tile >= first && tile < first + count);
        if (!mine) continue;
        const int l = __ffsll((long long)mine) - 1;
        owner = b0 + l, wanted = __builtin_amdgcn_readlane(adapter, l), place = tile - __builtin_amdgcn_readlane(first, l);
    }
    if (owner < 0 && !OUTSIDE) return false;
    if (wanted < 0) return keep(tile, 1, -1);
    int behind = 0;                              // tokens listed so far
    for (int b0 = 0; b0 < g.requests; b0 += 64) {
        request(b0 + lane, first, count, adapter);
        if (adapter != wanted) count = 0;
        const bool before = b0 + lane < owner;
        place += (int)wave_sum((u32)(before ? count : 0));
        if (b0 + 64 <= owner) continue;
        if (before) count = 0;
        if (b0 + lane == owner) count -= tile - first, first = tile;
        if (b0 <= owner && place % most) return false;
        const int upto = (int)wave_upto((u32)count), at = behind + upto - count;
        for (int i = 0; i < count && at + i < most; i++) rows[at + i] = first + i;
        behind += __builtin_amdgcn_readlane(upto, 63);
        if (behind >= most) break;
    }
    r = {min(behind, most), wanted};
    return true;
}

// Step 1: one workgroup per (tile of 16 tokens, party and run of the contraction).  Its four waves share the columns of A between CW and the blocks of
// 64 elements between 4 / CW; a wave takes CT times 16 columns.  APART: four tiles, a wave has one to itself.  Elements become digits where they are
// loaded: those that several waves need go through LDS, each wave bringing a part.  The next block's elements and digits of A are on their way while those at
// hand are multiplied.
// Bound by products and the making of digits, which loads overlap only in part, and by how evenly the workgroups fill 256 CUs.  2048 tokens of 4096, rank 16,
// n = 5: 89 us (336 MB, 53 at a copy's rate; 86 G operations, 25; four waves to a tile 103, of which without the loads 51, without those of x 61, of A
// 87).  1001 tokens of 4096, rank 128, n = 3: 99 us, 2.0 of 3.5 POP/s.  8 tokens with an adapter each, K = 4096, rank 16, n = 5: 9.6 us, 22 MB (eight waves to
// a workgroup 10.0 to 12).
template <int CW, int CT, bool WIDE, bool APART = false>
__global__ __launch_bounds__(BLOCK, 2) void down_kernel(adapter_args g)
{
    constexpr int KW = APART ? 1 : 4 / CW, PAIRS = 8 / CW, WORDS = 4 / CW;
    static_assert(!APART || CW == 1, "a wave with its own tile has all the columns");
    __shared__ v4i xd[CW > 1 ? 2 : 1][CW > 1 ? KW * TILE : 1];
    __shared__ int sums[KW > 1 ? CW : 1][KW > 1 ? ND : 1][BLOCK];
    __shared__ int tile_rows[APART ? 4 : 1][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned slot = g.grouped ? blockIdx.x : xcd_slot(blockIdx.x, gridDim.x), run = fd_div(slot, g.dTiles);
    const int cw = wave % CW, kw = APART ? 0 : wave / CW, split = (int)(run / (unsigned)g.nr), party = (int)run - split * g.nr, q = lane >> 4, c16 = lane & 15;
    int *rows = tile_rows[APART ? wave : 0];
    row_tile r;
    if (!find_rows<true>(g, (int)(slot - run * g.tiles) * (APART ? 4 : 1) + (APART ? wave : 0), 16, rows, r)) return;
    u64 *out = g.planes + split * g.plane + (size_t)party * g.tokens * g.rank;
    if constexpr (APART) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (other lanes' rows: the barrier alone orders no memory; LDS is in order, so no instruction)
        __builtin_amdgcn_wave_barrier();
    } else
        __syncthreads();
    if (r.adapter < 0) {                             // (zeros: the reduction sends what is left here, also for tokens of no request)
        for (int i = APART ? lane : tid; i < r.count * g.rank; i += APART ? 64 : BLOCK) out[(size_t)rows[i / g.rank] * g.rank + i % g.rank] = 0;
        return;
    }
    if constexpr (KW > 1) {
        for (int i = tid; i < CW * ND * BLOCK; i += BLOCK) (&sums[0][0][0])[i] = 0;
    }
    const int begin = split * g.run, end = min(begin + g.run, (g.K + 63) >> 6), turns = (end - begin + KW - 1) / KW;
    const u64 *row = g.x + ((size_t)party * g.tokens + rows[min(c16, r.count - 1)]) * g.ld_x;
    const size_t limb = (size_t)g.rank * 64;
    const signed char *a = g.down + r.adapter * g.down_bytes + party * g.down_party + (size_t)q * g.rank * 16;
    size_t column[CT];
#pragma unroll
    for (int c = 0; c < CT; c++) column[c] = (size_t)min((cw * CT + c) * 16 + c16, g.rank - 1) * 16;
    // this wave's part of a lane's 16 elements of block kb; past the row's end anything (A is zero there)
    auto load_x = [&](int kb, u64 (&v)[2 * PAIRS]) {
#pragma unroll
        for (int j = 0; j < PAIRS; j++) {
            const int k = 64 * kb + 2 * q + 8 * (cw * PAIRS + j);
            if constexpr (WIDE) {
                pack_t<2> p;
                p.load_streaming(row + (k < g.K ? k : 0));
                v[2 * j] = p.v[0], v[2 * j + 1] = p.v[1];
            } else {
                v[2 * j] = row[k < g.K ? k : 0];
                v[2 * j + 1] = row[k + 1 < g.K ? k + 1 : 0];
            }
        }
    };
    auto load_a = [&](int kb, int c, v4i (&w)[NL]) {
#pragma unroll
        for (int l = 0; l < NL; l++) w[l] = *reinterpret_cast<const v4i *>(a + (size_t)kb * NL * limb + l * limb + column[c]);
    };
    v4i acc[CT][ND], w[NL], next[NL];
    u64 v[2 * PAIRS];
#pragma unroll
    for (int c = 0; c < CT; c++)
#pragma unroll
        for (int s = 0; s < ND; s++) acc[c][s] = (v4i){0, 0, 0, 0};
    int kb = begin + kw;
    load_x(min(kb, end - 1), v);
    load_a(min(kb, end - 1), 0, w);
    for (int turn = 0; turn < turns; turn++) {
        const bool live = kb < end;
        const int kb_next = kb + KW;
        u32 d[WORDS][8];
#pragma unroll
        for (int b = 0; b < WORDS; b++) {
            const u64 y[4] = {balanced_digits(v[4 * b]), balanced_digits(v[4 * b + 1]), balanced_digits(v[4 * b + 2]), balanced_digits(v[4 * b + 3])};
            limb_dwords(y, d[b]);
        }
        const v4i *tile = nullptr;
        if constexpr (CW > 1) {
            tile = &xd[turn & 1][kw * TILE + lane];
#pragma unroll
            for (int l = 0; l < NL; l++)
#pragma unroll
                for (int b = 0; b < WORDS; b++) reinterpret_cast<u32 *>(&xd[turn & 1][kw * TILE + l * 64 + lane])[cw * WORDS + b] = d[b][l];
        }
        load_x(min(kb_next, end - 1), v);
        if constexpr (CW > 1) __syncthreads();
#pragma unroll
        for (int c = 0; c < CT; c++) {
            load_a(min(c + 1 < CT ? kb : kb_next, end - 1), c + 1 < CT ? c + 1 : 0, next);
            __builtin_amdgcn_sched_barrier(0);       // the loads leave before the products
            if (live) {
#pragma unroll
                for (int i = 0; i < NL; i++) {
                    v4i x;
                    if constexpr (CW > 1)
                        x = tile[i * 64];
                    else
                        x = (v4i){(int)d[0][i], (int)d[1][i], (int)d[2][i], (int)d[3][i]};
#pragma unroll
                    for (int j = 0; j < NL; j++) acc[c][i + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, w[j], acc[c][i + j], 0, 0, 0);
                }
            }
#pragma unroll
            for (int l = 0; l < NL; l++) w[l] = next[l];
        }
        kb = kb_next;
    }
    if constexpr (KW > 1) {                          // the sums of several waves, as whole numbers
        __syncthreads();
#pragma unroll
        for (int s = 0; s < ND; s++)
#pragma unroll
            for (int i = 0; i < 4; i++) atomicAdd(&sums[cw][s][(4 * q + i) * 16 + c16], acc[0][s][i]);
        __syncthreads();
        const int token = tid >> 4;
#pragma unroll
        for (int c = 0; c < CW; c++) {
            const int col = c * 16 + (tid & 15);
            if (token >= r.count || col >= g.rank) continue;
            v4i total[ND];
#pragma unroll
            for (int s = 0; s < ND; s++) total[s][0] = sums[c][s][tid];
            out[(size_t)rows[token] * g.rank + col] = fold_diagonals(total, 0);
        }
    } else {
#pragma unroll
        for (int c = 0; c < CT; c++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int token = 4 * q + i, col = (cw * CT + c) * 16 + c16;
                if (token < r.count && col < g.rank) out[(size_t)rows[token] * g.rank + col] = fold_diagonals(acc[c], i);
            }
    }
}

// Words that four rows of 16 lanes hold of four items, one part of each: afterwards row q has the four parts of item q.
__device__ __forceinline__ void exchange(int (&v)[4])
{
    const auto a = __builtin_amdgcn_permlane32_swap((u32)v[0], (u32)v[2], false, false);   // parts 0 and 1 of items 0 and 2, parts 2 and 3
    const auto b = __builtin_amdgcn_permlane32_swap((u32)v[1], (u32)v[3], false, false);
    const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    v[0] = (int)lo[0], v[1] = (int)lo[1], v[2] = (int)hi[0], v[3] = (int)hi[1];
}

// Four items' diagonal sums 4 q .. 4 q + 3 of a column in row q -> in row q item q's field element plus `more`.  The sums lie below 2^22 (a rank of at
// most 32: 8 * 32 * 2^14), so that two of them fit 32 bits.
__device__ __forceinline__ u64 fold_items(const v4i (&acc)[4], u64 more)
{
    int lo[4], hi[4];
    long long g[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        lo[i] = acc[i][0] + (int)((u32)acc[i][1] << 8);
        hi[i] = acc[i][2] + (int)((u32)acc[i][3] << 8);
    }
    exchange(lo), exchange(hi);
#pragma unroll
    for (int q = 0; q < 4; q++) g[q] = mad_i64(hi[q], 1 << 16, (long long)lo[q]);
#if defined(SS_FIELD_P45)
    return fold_words((u64)(g[0] + WORD_OFFSET), (u64)(g[1] + WORD_OFFSET), (u64)(g[2] + WORD_OFFSET), more);
#else
    return fold_words(g[0], g[1], g[2], g[3], more);
#endif
}

// y = 0 in the rows of all requests, where there is no base, which the second product then adds to: y is written twice and read once (2048 tokens of 4096 by 4096,
// rank 16, n = 5, whole calls: 285 us, with a base 245)
__global__ __launch_bounds__(BLOCK) void clear_kernel(adapter_args g)
{
    const int first = min(max(fixed_at(g.start, 0), 0), g.tokens), last = min(fixed_at(g.start, g.requests), g.tokens);
    for (int t = first + (int)blockIdx.x; t < last; t += gridDim.x)
        for (int c = threadIdx.x; c < g.N; c += BLOCK) g.y[((size_t)blockIdx.y * g.tokens + t) * g.ld_y + c] = 0;
}

// y = base of tokens without an adapter; rows: in LDS, behind a barrier
__device__ __forceinline__ void pass_through(const adapter_args &g, const row_tile &r, const int *rows, const u64 *base, u64 *y, int part)
{
    if (base == y) return;
    for (int t = 0; t < r.count; t++)
        for (int c = part * BLOCK + threadIdx.x; c < g.N; c += g.col_groups * BLOCK) y[rows[t] * g.ld_y + c] = base[rows[t] * g.ld_base + c];
}

// How a tensor is read and written: element by element, two neighbours in 16 bytes, or these past the caches
enum access { NARROW, PAIRS, STREAM_PAIRS };

// columns col and col + 1 of a row of N (NARROW: at most the first may exist)
template <access MODE>
__device__ __forceinline__ pack_t<2> load_pair(const u64 *row, int col, int N)
{
    pack_t<2> v = {{0, 0}};
    if (col < N) {
        if constexpr (MODE == STREAM_PAIRS)
            v.load_streaming(row + col);
        else if constexpr (MODE == PAIRS)
            v.load(row + col);
        else {
            v.v[0] = row[col];
            if (col + 1 < N) v.v[1] = row[col + 1];
        }
    }
    return v;
}

template <access MODE>
__device__ __forceinline__ void store_pair(u64 *row, int col, int N, const pack_t<2> &v)
{
    if (col >= N) return;
    if constexpr (MODE != NARROW)
        v.template send<MODE == STREAM_PAIRS>(row + col);
    else {
        row[col] = v.v[0];
        if (col + 1 < N) row[col + 1] = v.v[1];
    }
}

// Step 3 over limbs and rank together: D[s][c] = sum over (j, r) of z_{s-j}[r] B_j[r][c] is diagonal sum s of column c, which makes one MFMA of 16
// diagonals by 16 columns for 64 digits of a column, and one accumulator.  A's rows are the digits of z, in LDS with their limbs falling
// and zeros around them, read from a place that moves up by the rank with every diagonal: limb l of element i of a token lies at (15 - l) R + i.
__device__ __forceinline__ int diagonals_stride(int R, int steps) { return 15 * R + 64 * steps; }

__device__ __forceinline__ void stage_diagonals(const adapter_args &g, signed char *zd, int places, int stride, int party, const row_tile &r, const int *rows)
{
    const int tid = threadIdx.x;
    for (int i = tid * 4; i < places * stride; i += BLOCK * 4) *reinterpret_cast<int *>(zd + i) = 0;
    __syncthreads();
    for (int i = tid; i < r.count * g.rank; i += BLOCK) {
        const int t = i / g.rank, e = i - t * g.rank;
        const u64 d = balanced_digits(g.z[((size_t)party * g.tokens + rows[t]) * g.rank + e]);
#pragma unroll
        for (int l = 0; l < NL; l++) zd[t * stride + (15 - l) * g.padded + e] = (signed char)(d >> (8 * l));
    }
    __syncthreads();
}

// 64 digits, step m, of the 16 diagonals of a token (8-byte alignment)
__device__ __forceinline__ v4i diagonals_at(const signed char *zd, int R, int m)
{
    const int lane = threadIdx.x & 63;
    const int2 *p = reinterpret_cast<const int2 *>(zd + (15 - (lane & 15)) * R + (lane >> 4) * 16 + m * 64);
    const int2 a = p[0], b = p[1];
    return (v4i){a.x, a.y, b.x, b.y};
}

// Tiles of UP_ROWS tokens of a request whose rank takes M products.  A wave keeps the digits of 128 columns of B in registers and takes the tokens one
// after the other, each a result of 1 KB in a row; the next token's digits and the base of those after it are on their way.
// Bound by memory, and by exchanging and folding the diagonals beside it: 2048 tokens by 4096 columns, n = 5, rank 16 150 us, 671 MB at 4.5 TB/s (copying
// in the same order 122 to 141; without memory 115 to 126); rank 8 133, rank 32 240 (products).  128 tokens with 27 adapters, rank 32, 8192 columns, n = 3:
// 61 us, 220 MB, of which B is 170.  64 columns to a wave for rank 32: 282 instead of 238.
template <int M, access MODE>
__global__ __launch_bounds__(BLOCK, 2) void up_diagonals_kernel(adapter_args g)
{
    extern __shared__ signed char zd[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = blockIdx.y / g.n, party = blockIdx.y - part * g.n;
    __shared__ int rows[UP_ROWS];
    row_tile r;
    // (of grouped tiles those that there are stand in front: they are spread over the XCDs)
    if (!find_rows<false>(g, g.grouped ? (int)blockIdx.x : (int)xcd_slot(blockIdx.x, gridDim.x), UP_ROWS, rows, r)) return;
    const u64 *base = g.base + (size_t)party * g.tokens * g.ld_base;
    u64 *y = g.y + (size_t)party * g.tokens * g.ld_y;
    __syncthreads();
    if (r.adapter < 0) {
        pass_through(g, r, rows, base, y, part);
        return;
    }
    const int own_row = rows[min(lane & (UP_ROWS - 1), r.count - 1)];   // of the token with the lane's number
    const int R = g.padded, chunks = NL * R / 16, stride = diagonals_stride(R, M), q = lane >> 4, c16 = lane & 15;
    const int blocks = (g.N + 31) >> 5, units = (blocks + 3) >> 2, step = g.col_groups * 4;
    const signed char *b = g.up + r.adapter * g.up_bytes + party * g.up_party;
    v4i w[2][4][M];
    auto load_b = [&](int unit) {
#pragma unroll
        for (int i = 0; i < 4; i++)              // (behind the last block of 32 columns, it again)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const signed char *at = b + (size_t)(2 * min(4 * unit + i, blocks - 1) + h) * chunks * 256;
#pragma unroll
                for (int m = 0; m < M; m++)
                    w[h][i][m] = *reinterpret_cast<const v4i *>(at + min(4 * m + q, chunks - 1) * 256 + c16 * 16);
            }
    };
    constexpr int AHEAD = 4;
    pack_t<2> more[AHEAD];
    int unit = part * 4 + wave;
    auto load_base = [&](int t, int u) {
        return load_pair<MODE>(base + (size_t)__builtin_amdgcn_readlane(own_row, min(t, r.count - 1)) * g.ld_base, 128 * u + 32 * q + 2 * c16, g.N);
    };
    if (unit < units) {
        load_b(unit);
#pragma unroll
        for (int i = 0; i < AHEAD; i++) more[i] = load_base(i, unit);
    }
    stage_diagonals(g, zd, UP_ROWS + 1, stride, party, r, rows);
    auto digits = [&](int t, v4i (&a)[M]) {
#pragma unroll
        for (int m = 0; m < M; m++) {
            a[m] = diagonals_at(zd + t * stride, R, m);
            if (NL != 8 && 4 * m + q >= chunks) a[m] = (v4i){0, 0, 0, 0};   // (of the last product's chunks those that do not exist)
        }
    };
    for (; unit < units; unit += step) {
        const int col = 128 * unit + 32 * q + 2 * c16;
        v4i a[2][M];
        digits(0, a[0]);
        for (int t0 = 0; t0 < r.count; t0 += AHEAD) {
#pragma unroll
            for (int i = 0; i < AHEAD; i++) {
                const int t = t0 + i;
                if (t >= r.count) break;
                digits(t + 1, a[(i + 1) & 1]);           // (there is a place behind the last token)
                pack_t<2> o;
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    v4i acc[4];
#pragma unroll
                    for (int m = 0; m < M; m++)
#pragma unroll
                        for (int k = 0; k < 4; k++)
                            acc[k] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i & 1][m], w[h][k][m], m ? acc[k] : (v4i){0, 0, 0, 0}, 0, 0, 0);
                    o.v[h] = fold_items(acc, more[i].v[h]);
                }
                more[i] = load_base(t + AHEAD, unit);
                store_pair<MODE>(y + (size_t)__builtin_amdgcn_readlane(own_row, t) * g.ld_y, col, g.N, o);
            }
        }
        if (unit + step < units) {
            load_b(unit + step);
#pragma unroll
            for (int i = 0; i < AHEAD; i++) more[i] = load_base(i, unit + step);
        }
    }
}

// Tiles of 64 tokens of a request with a larger rank: diagonal sums apart, as in a dense layer; the digits of z in LDS in MFMA order, a wave takes
// 16 tokens and 32 columns of B at a time.  The waves share the columns as above.
// Bound by staging and rounds of workgroups in small calls, by reading B for every 16 tokens in large ones: 1001 tokens by 1024 columns, rank 128, n = 3, 43 us
// (1.2 POP/s); 555 by 2560, rank 64, 45-bit prime, 30 us; 2048 by 4096, rank 64, n = 5, 300 us (671 MB, 1.1 POP/s).
template <access MODE>
__global__ __launch_bounds__(BLOCK, 2) void up_tile_kernel(adapter_args g)
{
    extern __shared__ v4i zt[];                  // [token / 16][rank / 64][limb][64 lanes]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = blockIdx.y / g.n, party = blockIdx.y - part * g.n;
    int *rows = reinterpret_cast<int *>(zt);     // (until the digits are written)
    row_tile r;
    if (!find_rows<false>(g, blockIdx.x, 64, rows, r)) return;
    const u64 *base = g.base + (size_t)party * g.tokens * g.ld_base;
    u64 *y = g.y + (size_t)party * g.tokens * g.ld_y;
    __syncthreads();
    if (r.adapter < 0) {
        pass_through(g, r, rows, base, y, part);
        return;
    }
    const int per_limb = g.padded / 16, chunks = NL * per_limb, blocks = (g.rank + 63) >> 6, q = lane >> 4, c16 = lane & 15;
    const u64 *z = g.z + (size_t)party * g.tokens * g.rank;
    const int log = r.count > 32 ? 2 : r.count > 16 ? 1 : 0, first = (wave & ((1 << log) - 1)) * 16;   // 2^log waves to the tokens, the others to the columns
    const int row = tid & ((16 << log) - 1), own_row = rows[min(row, r.count - 1)];   // a thread stages parts of one row
    int to[4];
#pragma unroll
    for (int c = 0; c < 4; c++) to[c] = rows[min(first + 4 * q + c, r.count - 1)];
    __syncthreads();
    for (int i = tid; i < (16 << log) * blocks * 16; i += BLOCK) {      // four elements of it
        const int e = (i >> (4 + log)) * 4;
        u64 v[4];
#pragma unroll
        for (int c = 0; c < 4; c++) v[c] = balanced_digits(row < r.count && e + c < g.rank ? z[(size_t)own_row * g.rank + e + c] : 0);
        u32 *dst = reinterpret_cast<u32 *>(zt + ((row >> 4) * blocks + (e >> 6)) * TILE + (row & 15) + 16 * ((e & 63) >> 4)) + ((e & 15) >> 2);
#pragma unroll
        for (int l = 0; l < NL; l++) dst[l * 256] = limb_dword(v, l);
    }
    __syncthreads();
    const signed char *b = g.up + r.adapter * g.up_bytes + party * g.up_party + c16 * 16;
    const int units = (g.N + 31) >> 5;
    const v4i *mine = zt + (first >> 4) * blocks * TILE + lane;
    int u = part * (4 >> log) + (wave >> log);
    const int step = g.col_groups * (4 >> log);
    // 16 columns (half h of 32) by 64 ranks; behind the rank the digits of z are 0
    auto load = [&](int unit, int kb, int h, v4i (&w)[NL]) {
        const signed char *src = b + ((size_t)(2 * unit + h) * chunks + min(4 * kb + q, per_limb - 1)) * 256;
#pragma unroll
        for (int j = 0; j < NL; j++) w[j] = *reinterpret_cast<const v4i *>(src + (size_t)j * per_limb * 256);
    };
    v4i w[2][NL];
    if (u < units) load(u, 0, 0, w[0]);
    for (; u < units; u += step) {
        v4i acc[2][ND];
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int s = 0; s < ND; s++) acc[h][s] = (v4i){0, 0, 0, 0};
        const int col = 32 * u + 2 * c16;
        pack_t<2> more[4];
#pragma unroll
        for (int c = 0; c < 4; c++) more[c] = load_pair<MODE>(base + (size_t)to[c] * g.ld_base, col, g.N);
        for (int kb = 0; kb < blocks; kb++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                // the next 16 columns on their way (behind the last, some again)
                load(h == 0 || kb + 1 < blocks ? u : min(u + step, units - 1), h == 0 ? kb : kb + 1 < blocks ? kb + 1 : 0, 1 - h, w[1 - h]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < NL; i++) {
                    const v4i x = mine[kb * TILE + i * 64];
#pragma unroll
                    for (int j = 0; j < NL; j++) acc[h][i + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, w[h][j], acc[h][i + j], 0, 0, 0);
                }
            }
#pragma unroll
        for (int c = 0; c < 4; c++) {
            if (first + 4 * q + c >= r.count) continue;
            pack_t<2> o;
            o.v[0] = fold_diagonals(acc[0], c, more[c].v[0]);
            o.v[1] = fold_diagonals(acc[1], c, more[c].v[1]);
            store_pair<MODE>(y + (size_t)to[c] * g.ld_y, col, g.N, o);
        }
    }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

hipError_t ss_launch_pack_adapter(const ss_adapters &s, int index, const u64 *a, const u64 *b, int given, int n, int t, hipStream_t stream)
{
    const int padded = (int)padded_rank(s.rank), nr = 2 * t + 1;
    const size_t down = down_party_bytes(s.K, s.rank), up = up_party_bytes(s.rank, s.N);
    const unsigned down_items = (unsigned)(down / SS_NLIMB / 16), up_items = (unsigned)(up / 16);
    hipLaunchKernelGGL(pack_down_kernel, dim3((unsigned)div_up(down_items, BLOCK), nr), dim3(BLOCK), 0, stream, a, s.down + (size_t)index * nr * down, s.K, given,
                       s.rank, down_items, down);
    hipLaunchKernelGGL(pack_up_kernel, dim3((unsigned)div_up(up_items, BLOCK), n), dim3(BLOCK), 0, stream, b, s.up + (size_t)index * n * up, given, padded, s.N,
                       up_items, up);
    return hipGetLastError();
}

hipError_t ss_launch_adapters_down(const adapter_plan &plan, const ss_adapters &s, const ss_requests &req, const u64 *x, size_t ld_x, u64 *planes, int n, int t,
                                   hipStream_t stream)
{
    adapter_args g = {};
    g.start = req.start, g.adapter = req.adapter, g.requests = req.requests, g.tokens = req.tokens, g.grouped = plan.grouped;
    g.adapters = s.adapters, g.K = s.K, g.rank = s.rank;
    g.down = s.down, g.nr = 2 * t + 1, g.n = n;
    g.down_party = down_party_bytes(s.K, s.rank), g.down_bytes = g.nr * g.down_party;
    g.x = x, g.ld_x = ld_x, g.planes = planes, g.plane = (size_t)g.nr * req.tokens * s.rank;
    g.run = plan.run;
    g.tiles = (unsigned)(plan.apart ? div_up(plan.down_tiles, 4) : plan.down_tiles);
    g.dTiles = make_fdiv(g.tiles);
    const dim3 grid((unsigned)plan.down_groups);
    const bool wide = s.K % 2 == 0 && ld_x % 2 == 0 && aligned16(x);
#define SS_DOWN(CW, CT) hipLaunchKernelGGL((wide ? down_kernel<CW, CT, true> : down_kernel<CW, CT, false>), grid, dim3(BLOCK), 0, stream, g)
    if (plan.apart)
        hipLaunchKernelGGL((wide ? down_kernel<1, 1, true, true> : down_kernel<1, 1, false, true>), grid, dim3(BLOCK), 0, stream, g);
    else if (s.rank <= 16)
        SS_DOWN(1, 1);
    else if (s.rank <= 32)
        SS_DOWN(2, 1);
    else if (s.rank <= 64)
        SS_DOWN(4, 1);
    else
        SS_DOWN(4, 2);
#undef SS_DOWN
    return hipGetLastError();
}

hipError_t ss_launch_adapters_up(const adapter_plan &plan, const ss_adapters &s, const ss_requests &req, const u64 *z, const u64 *base, size_t ld_base, u64 *y,
                                 size_t ld_y, int n, int t, hipStream_t stream)
{
    (void)t;
    adapter_args g = {};
    g.start = req.start, g.adapter = req.adapter, g.requests = req.requests, g.tokens = req.tokens, g.grouped = plan.grouped;
    g.adapters = s.adapters, g.rank = s.rank, g.padded = (int)padded_rank(s.rank), g.N = s.N;
    g.up = s.up, g.n = n;
    g.up_party = up_party_bytes(s.rank, s.N), g.up_bytes = n * g.up_party;
    g.z = z, g.base = base, g.ld_base = ld_base, g.y = y, g.ld_y = ld_y;
    g.col_groups = plan.col_groups;
    const int steps = (int)up_steps(s.rank);
    const size_t lds = plan.diagonals ? (UP_ROWS + 1) * (15 * g.padded + 64 * steps) : 4 * div_up(s.rank, 64) * TILE * 16;
    const dim3 grid((unsigned)plan.up_tiles, n * plan.col_groups);
    const bool pairs = s.N % 2 == 0 && ld_y % 2 == 0 && aligned16(y) && (!base || (ld_base % 2 == 0 && aligned16(base)));
    if (!base) {
        hipLaunchKernelGGL(clear_kernel, dim3((unsigned)std::min(req.tokens, 4096), n), dim3(BLOCK), 0, stream, g);
        g.base = y, g.ld_base = ld_y;
    }
    const access mode = !pairs ? NARROW : plan.streams ? STREAM_PAIRS : PAIRS;
#define SS_MODE(KERNEL, ...)                                                                                                              \
    hipLaunchKernelGGL((mode == NARROW ? KERNEL<__VA_ARGS__ NARROW> : mode == PAIRS ? KERNEL<__VA_ARGS__ PAIRS> : KERNEL<__VA_ARGS__ STREAM_PAIRS>), grid, \
                       dim3(BLOCK), lds, stream, g)
#define SS_COMMA ,
    if (!plan.diagonals)
        SS_MODE(up_tile_kernel, );
    else if (steps == 1)
        SS_MODE(up_diagonals_kernel, 1 SS_COMMA);
    else if (steps == 2)
        SS_MODE(up_diagonals_kernel, 2 SS_COMMA);
    else
        SS_MODE(up_diagonals_kernel, SS_NLIMB / 2 SS_COMMA);                   // a rank of 17 to 32
#undef SS_COMMA
#undef SS_MODE
    return hipGetLastError();
}

}  // namespace SS_NS
