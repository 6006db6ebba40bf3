// The next token of every row from shares of its logits: REC, then a draw in whole numbers from the softmax of the row, cut by top-k, top-p and
// min-p.  The tokens that may be drawn are the first ones in the order of falling logits, equal ones by their number, so a cut is a distance from
// the row's largest logit and how many of the tokens at that distance are kept.  A histogram of distances, with how many tokens each bin has and
// what they weigh, says in which bin a cut lies; the tokens of that bin alone are looked at further.
//
// Up to SMALL_VOCAB tokens, and up to MEDIUM_VOCAB where there are about as many rows as CUs, one workgroup takes a row in one launch.  Other rows go
// through four, so that many workgroups share a row:
//   open     REC, and the largest logit of every 1024
//   count    the histogram
//   collect  what the tokens weigh that stay whatever the cut is, for every 512; the tokens of the bins with a cut, in a list
//   pick     the cut, the weights of the list's tokens that stay, and the draw
#include "kernels.hpp"
#include "power2.hpp"
#include "truncation.hpp"
#include "lanes.hpp"

namespace SS_NS {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = SAMPLE_BINS, CHUNK = SAMPLE_CHUNK;
constexpr int OPEN_THREADS = 256;
constexpr int NOT_ALLOWED = -2147483647 - 1;

// Distances lo .. lo + span - 1 among which a cut lies, and what comes before them
struct cut_range {
    u32 lo, span;                   // span 0: no such cut
    u64 left;                       // tokens (top_k) or weight (top_p) to take from the range
    u64 before;                     // weight of the tokens in front
};

struct row_plan {
    u32 sure;                       // distances below stay
    cut_range few, part;            // part.left only where few.span is 0: it depends on what few leaves
};

struct sample_args {
    const u64 *logits;              // [n][rows][ld]
    size_t ld;
    int rows, vocab, f;
    const int4 *params;             // scale, top_k, top_p, min_p
    const long long *random;
    const u32 *allowed;             // a bit to a token, or nullptr
    size_t ld_allowed;
    long long *tokens;
    int *shown;                     // probability of the token, 30 fraction bits
    // of the rows of this launch, row0 the first
    int row0, opens, groups, chunks, key_ld;
    fdiv dOpens, dGroups;
    int *keys;                      // [.][key_ld]: logits in units of 2^-min(f, 16)
    int *tops;                      // [.][opens]
    u32 *count;                     // [.][BINS]
    u64 *sum;                       // [.][BINS]
    u64 *sure;                      // [.][chunks]
    u32 *listed;                    // [.]
    row_plan *plans;                // [.]
    u64 *list;                      // [.][SAMPLE_LIST]: distance 2^20 + token
};

// the opened logit in units of 2^-min(f, 16), the far ones as the last that 32 bits hold
__device__ __forceinline__ int logit_of(u64 v, int f)
{
    const long long s = (v <= (SS_P - 1) / 2 ? (long long)v : (long long)v - (long long)SS_P) >> (f - min(f, 16));
    return (int)min(max(s, -2147483647ll), 2147483647ll);
}

// what a row asks for, and the weight of a distance
struct row_rule {
    u32 scale, least, few, part;    // least: smallest weight that is kept; few: top_k or 0; part: top_p, 2^30 for none
    int shift, bits;
    u32 reach;                      // distances from here on have no weight
    __device__ __forceinline__ bool cuts() const { return few || part < 1u << 30; }
    // Bins of the histogram: distances below 2^(bits + 1) have one each, others share one with those that have the same `bits` + 1 first digits, so
    // that whatever the temperature is a bin is narrow beside its distance
    __device__ __forceinline__ u32 bin_of(u32 d) const
    {
        const int s = max(0, 31 - bits - __clz((int)d));
        return ((u32)s << bits) + (d >> s);
    }
    __device__ __forceinline__ u32 first_of(u32 bin) const   // the next bin's, less one, is its last
    {
        const int s = max(0, (int)(bin >> bits) - 1);
        return (bin - ((u32)s << bits)) << s;
    }
    __device__ __forceinline__ u32 weight(u32 distance) const { return power2((u64)distance * scale >> shift); }
    // what tokens that weigh `of` have to be cut to, see top_p
    __device__ __forceinline__ u64 need(u64 of) const
    {
        const u64 lo = of * part, hi = __umul64hi(of, part), up = (hi << 34 | lo >> 30) + ((lo & ((1u << 30) - 1)) != 0);
        return up ? up : 1;
    }
};

__device__ __forceinline__ row_rule rule_of(const int4 &p, int f)
{
    row_rule r;
    r.scale = p.x <= 0 ? 0x7FFFFFFFu : (u32)max(p.x, 1 << 14);   // (of the largest logit alone the weight does not depend on it)
    r.least = (u32)min(max(p.w, 1), 1 << 30);
    r.few = p.x <= 0 ? 1 : (u32)max(p.y, 0);
    r.part = (u32)min(max(p.z, 0), 1 << 30);
    r.shift = min(f, 16) + 8;
    r.reach = (u32)(((31ull << (16 + r.shift)) + r.scale - 1) / r.scale);   // <= 31 2^26
    r.bits = r.reach <= 1u << 22 ? 7 : 6;        // (digits of a distance + 1 - bits) 2^bits bins: up to 22 digits 2048, up to 31 1664
    return r;
}

__device__ __forceinline__ int wave_max(int v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = max(v, __shfl_xor(v, d));
    return v;
}

// sum over the threads up to one's own, and over all of them; lds: one for each wave
template <typename T>
__device__ __forceinline__ T block_upto(T v, T *lds, T &all)
{
    static_assert(WAVES == 16, "a row of lanes adds up the waves");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    v = wave_upto(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[wave] = v;
    __syncthreads();
    const T waves = row_upto(lds[threadIdx.x & 15]);
    all = read_lane(waves, 15);
    return wave ? v + read_lane(waves, wave - 1) : v;
}

struct row_state {
    u32 count[BINS];                // of the tokens in a bin, then of those at the cut in a chunk
    u64 sum[BINS];                  // what they weigh, then what stays of a chunk
    u64 red64[WAVES], found_sum;
    u32 red32[WAVES], found_count;
    int bin[3];
};

// From the histogram in s: where the cuts lie.
__device__ __forceinline__ row_plan plan_row(row_state &s, const row_rule &rule)
{
    const int tid = threadIdx.x;
    const u32 c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1];
    const u64 s0 = s.sum[2 * tid], s1 = s.sum[2 * tid + 1];
    u32 all_count;
    u64 all_sum;
    const u32 c = block_upto(c0 + c1, s.red32, all_count);
    const u64 w = block_upto(s0 + s1, s.red64, all_sum);
    if (tid < 3) s.bin[tid] = BINS;
    __syncthreads();
    row_plan p = {rule.reach, {0, 0, 0, 0}, {0, 0, 0, 0}};
    u64 least = all_sum, most = all_sum;         // what top_k leaves weighs so much
    if (rule.few && all_count >= rule.few) {     // (uniform)
        if (c >= rule.few && c - c0 - c1 < rule.few) {
            const bool second = c - c1 < rule.few;
            s.bin[0] = 2 * tid + second;
            s.found_count = second ? c - c1 : c - c1 - c0;
            s.found_sum = second ? w - s1 : w - s1 - s0;
            s.red64[0] = second ? s1 : s0;       // (what the block sums left there is no longer needed)
        }
        __syncthreads();
        const u32 lo = rule.first_of((u32)s.bin[0]);
        p.few = {lo, rule.first_of((u32)s.bin[0] + 1) - lo, rule.few - s.found_count, s.found_sum};
        p.sure = p.few.lo;
        least = s.found_sum;
        most = s.found_sum + s.red64[0];
    }
    if (rule.part < 1u << 30) {
        const u64 low = rule.need(least), high = rule.need(most);
        __syncthreads();
        auto look = [&](u64 need, int which) {   // the first bin up to which the tokens weigh so much
            if (w >= need && w - s0 - s1 < need) {
                const bool second = w - s1 < need;
                s.bin[which] = 2 * tid + second;
                if (which == 1) s.found_sum = second ? w - s1 : w - s1 - s0;
            }
        };
        look(low, 1), look(high, 2);
        __syncthreads();
        const u32 lo = rule.first_of((u32)s.bin[1]);
        p.part = {lo, rule.first_of((u32)s.bin[2] + 1) - lo, high - s.found_sum, s.found_sum};
        p.sure = p.part.lo;
    }
    return p;
}

struct cut_place {
    u32 distance, ties;             // tokens below the distance stay, and so many of those at it
    u64 before;                     // weight of the former
};

// The distance in a range at which the tokens up to it are as many as is left to take (BY_SUM: weigh as much).  each(f) calls f(distance, token) for all tokens
// of the range at least.
template <bool BY_SUM, typename E>
__device__ __forceinline__ cut_place find_cut(row_state &s, const row_rule &rule, cut_range r, E &&each)
{
    const int tid = threadIdx.x;
    for (;;) {
        const int shift = max(0, 32 - __clz((int)(r.span - 1)) - SAMPLE_BIN_BITS);
        __syncthreads();
        for (int i = tid; i < BINS; i += THREADS) s.count[i] = 0, s.sum[i] = 0;
        __syncthreads();
        each([&](u32 d, int) {
            if (d < r.lo || d - r.lo >= r.span) return;
            atomicAdd(&s.count[(d - r.lo) >> shift], 1u);
            atomicAdd((unsigned long long *)&s.sum[(d - r.lo) >> shift], (unsigned long long)rule.weight(d));
        });
        __syncthreads();
        const u32 c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1];
        const u64 s0 = s.sum[2 * tid], s1 = s.sum[2 * tid + 1];
        u32 all_count;
        u64 all_sum;
        const u32 c = block_upto(c0 + c1, s.red32, all_count);
        const u64 w = block_upto(s0 + s1, s.red64, all_sum);
        const u64 to = BY_SUM ? w : c, before = to - (BY_SUM ? s0 + s1 : c0 + c1);
        if (to >= r.left && before < r.left) {
            const bool second = to - (BY_SUM ? s1 : c1) < r.left;
            s.bin[0] = 2 * tid + second;
            s.found_count = second ? c - c1 : c - c1 - c0;
            s.found_sum = second ? w - s1 : w - s1 - s0;
        }
        __syncthreads();
        r.left -= BY_SUM ? s.found_sum : s.found_count;
        r.before += s.found_sum;
        r.lo += (u32)s.bin[0] << shift;
        r.span = 1u << shift;
        if (shift == 0) break;
    }
    const u32 w = rule.weight(r.lo);
    return {r.lo, (u32)(BY_SUM ? (r.left + w - 1) / w : r.left), r.before};
}

// The cuts of a row, then, with what is sure of every chunk in sure(c), the draw.  each: as in find_cut, of the tokens in the ranges of the plan;
// key(j): that of token j.
template <typename E, typename S, typename K>
__device__ __forceinline__ void draw_token(const sample_args &g, int row, row_state &s, const row_rule &rule, const row_plan &plan, int top, E &&each, S &&sure,
                                           K &&key)
{
    const int tid = threadIdx.x;
    cut_place cut = {rule.reach, 0, 0};
    cut_range part = plan.part;
    if (plan.few.span) {
        cut = find_cut<false>(s, rule, plan.few, each);
        if (part.span) part.left = rule.need(cut.before + (u64)cut.ties * rule.weight(cut.distance)) - part.before;
    }
    if (part.span) cut = find_cut<true>(s, rule, part, each);
    const u32 at_cut = cut.distance < rule.reach ? rule.weight(cut.distance) : 0;
    const int chunks = (g.vocab + CHUNK - 1) / CHUNK;
    __syncthreads();
    for (int c = tid; c < 2 * THREADS; c += THREADS) {
        s.count[c] = 0;
        s.sum[c] = c < chunks ? sure(c) : 0;
    }
    __syncthreads();
    each([&](u32 d, int j) {
        if (d < plan.sure || d > cut.distance) return;
        const u32 w = rule.weight(d);
        if (w < rule.least) return;
        if (d == cut.distance)
            atomicAdd(&s.count[j / CHUNK], 1u);
        else
            atomicAdd((unsigned long long *)&s.sum[j / CHUNK], (unsigned long long)w);
    });
    __syncthreads();
    const u32 t0 = s.count[2 * tid], t1 = s.count[2 * tid + 1];
    u32 all_ties;
    u64 sum;
    const u32 before0 = block_upto(t0 + t1, s.red32, all_ties) - t0 - t1, before1 = before0 + t0;
    auto kept = [&](u32 mine, u32 before) { return cut.ties > before ? min(mine, cut.ties - before) : 0; };
    const u64 w0 = s.sum[2 * tid] + (u64)at_cut * kept(t0, before0), w1 = s.sum[2 * tid + 1] + (u64)at_cut * kept(t1, before1);
    const u64 upto = block_upto(w0 + w1, s.red64, sum);
    const u64 target = __umul64hi((u64)g.random[row] << 2, sum);
    if (upto > target && upto - w0 - w1 <= target) {
        const bool second = upto - w1 <= target;
        s.bin[0] = 2 * tid + second;
        s.found_count = second ? before1 : before0;
        s.found_sum = second ? upto - w1 : upto - w1 - w0;
    }
    __syncthreads();
    const int j = s.bin[0] * CHUNK + tid, k = tid < CHUNK && j < g.vocab ? key(j) : NOT_ALLOWED;
    const u32 d = (u32)top - (u32)k, v = k != NOT_ALLOWED && d < rule.reach && d <= cut.distance ? rule.weight(d) : 0;
    const bool tie = v >= rule.least && d == cut.distance;
    const u32 rank = s.found_count + block_upto((u32)tie, s.red32, all_ties);
    const u64 before = s.found_sum, w = v < rule.least || (tie && rank > cut.ties) ? 0 : v;
    u64 chunk;
    const u64 to = before + block_upto(w, s.red64, chunk);
    if (to - w <= target && target < to) {
        g.tokens[row] = j;
        g.shown[row] = (int)(((w << 30) + sum / 2) / sum);
    }
}

__device__ __forceinline__ int key_of(const sample_args &g, const ss_rec_params &rp, int row, int j, u64 opened)
{
    const u64 v = rp.dinv == 1 ? opened : ss_mul(opened, rp.dinv);
    const bool allowed = !g.allowed || (g.allowed[(size_t)row * g.ld_allowed + (j >> 5)] >> (j & 31) & 1);
    return allowed ? logit_of(v, g.f) : NOT_ALLOWED;
}

// ------------------------------------------------------------------ a workgroup to a row

// The row's logits stay in LDS.  Bound by the row's way through one CU: its shares, two atomics of LDS to a token for the histogram, one for the draw to the
// word of its chunk, which all 64 lanes of a wave have in common, and three to five times over the keys.  256 rows of 2048 16 us, of 8192 25, of 32000 63
// (m = 2: 131 MB).
template <int MOST>
__global__ __launch_bounds__(THREADS) void sample_kernel(sample_args g, ss_rec_params rp)
{
    __shared__ row_state s;
    __shared__ int keys[MOST];
    constexpr int FLIGHT = 4;                    // loads of a share on their way
    const int tid = threadIdx.x, row = blockIdx.x;
    const row_rule rule = rule_of(g.params[row], g.f);
    int top = NOT_ALLOWED;
    for (int j0 = tid; j0 < g.vocab; j0 += FLIGHT * THREADS) {
        ss_sacc2 acc[FLIGHT];
#pragma unroll
        for (int i = 0; i < FLIGHT; i++) acc[i].clear();
        for (int q = 0; q < rp.m; q++) {
            const u64 *x = g.logits + ((size_t)rp.plane[q] * g.rows + row) * g.ld;
            u64 v[FLIGHT];
#pragma unroll
            for (int i = 0; i < FLIGHT; i++) v[i] = x[min(j0 + i * THREADS, g.vocab - 1)];
#pragma unroll
            for (int i = 0; i < FLIGHT; i++) {
                SS_SPLIT31(v[i], w0, w1);
                acc[i].mac(w0, w1, rp.ilambda[q]);
            }
        }
#pragma unroll
        for (int i = 0; i < FLIGHT; i++) {
            const int j = j0 + i * THREADS;
            if (j >= g.vocab) continue;
            const int key = key_of(g, rp, row, j, acc[i].value());
            keys[j] = key;
            top = max(top, key);
        }
    }
    top = wave_max(top);
    if ((tid & 63) == 0) s.red32[tid >> 6] = (u32)top;
    for (int i = tid; i < BINS; i += THREADS) s.count[i] = 0, s.sum[i] = 0;
    __syncthreads();
    for (int w = 0; w < WAVES; w++) top = max(top, (int)s.red32[w]);
    __syncthreads();
    if (top == NOT_ALLOWED) {
        if (tid == 0) g.tokens[row] = -1, g.shown[row] = 0;
        return;
    }
    auto each = [&](auto &&f) {
        for (int j = tid; j < g.vocab; j += THREADS) {
            const u32 d = (u32)top - (u32)keys[j];
            if (keys[j] != NOT_ALLOWED && d < rule.reach) f(d, j);
        }
    };
    each([&](u32 d, int) {
        atomicAdd(&s.count[rule.bin_of(d)], 1u);
        atomicAdd((unsigned long long *)&s.sum[rule.bin_of(d)], (unsigned long long)rule.weight(d));
    });
    __syncthreads();
    row_plan plan = plan_row(s, rule);
    plan.sure = 0;                               // (all tokens are looked at again)
    draw_token(g, row, s, rule, plan, top, each, [](int) { return 0ull; }, [&](int j) { return keys[j]; });
}

// ------------------------------------------------------------------ many workgroups to a row

// REC.  Bound by reading the shares: 64 rows of 200003, m = 3, 60 us, 5.1 TB/s with the keys written; 256 of 32000, m = 2, 32; one row 4.2, a launch and a
// load.
template <bool WIDE, bool STREAM>
__global__ __launch_bounds__(OPEN_THREADS) void open_kernel(sample_args g, ss_rec_params rp)
{
    __shared__ int red[OPEN_THREADS / 64];
    const int tid = threadIdx.x;
    const u32 at = fd_div(blockIdx.x, g.dOpens), block = blockIdx.x - at * g.opens;
    const int row = g.row0 + (int)at;
    for (u32 i = block * OPEN_THREADS + tid; i < (u32)BINS; i += g.opens * OPEN_THREADS) g.count[(size_t)at * BINS + i] = 0, g.sum[(size_t)at * BINS + i] = 0;
    if (block == 0 && tid == 0) g.listed[at] = 0;
    // four tokens to a thread: neighbours two by two (WIDE), or one by one
    constexpr int PER = SAMPLE_OPEN / OPEN_THREADS;
    ss_sacc2 acc[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) acc[i].clear();
    const int j0 = (int)block * SAMPLE_OPEN + (WIDE ? 2 * tid : tid);
    auto place = [&](int i) { return WIDE ? j0 + (i >> 1) * 2 * OPEN_THREADS + (i & 1) : j0 + i * OPEN_THREADS; };
    for (int q = 0; q < rp.m; q++) {
        const u64 *x = g.logits + ((size_t)rp.plane[q] * g.rows + row) * g.ld;
        u64 v[PER];
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < PER; i += 2) {
                const int j = place(i);
                pack_t<2> p = {{0, 0}};
                if (j + 1 < g.vocab)
                    STREAM ? p.load_streaming(x + j) : p.load(x + j);
                else if (j < g.vocab)
                    p.v[0] = x[j];
                v[i] = p.v[0], v[i + 1] = p.v[1];
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const u64 *from = x + min(place(i), g.vocab - 1);
                v[i] = STREAM ? __builtin_nontemporal_load(from) : *from;
            }
        }
#pragma unroll
        for (int i = 0; i < PER; i++) {
            SS_SPLIT31(v[i], w0, w1);
            acc[i].mac(w0, w1, rp.ilambda[q]);
        }
    }
    int top = NOT_ALLOWED, *keys = g.keys + (size_t)at * g.key_ld;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int j = place(i), k = j < g.vocab ? key_of(g, rp, row, j, acc[i].value()) : NOT_ALLOWED;
        if (j < g.key_ld) keys[j] = k;
        top = max(top, k);
    }
    top = wave_max(top);
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < OPEN_THREADS / 64; w++) top = max(top, red[w]);
        g.tops[(size_t)at * g.opens + block] = top;
    }
}

// the largest logit of a row
__device__ __forceinline__ int top_of(const sample_args &g, u32 at, u32 *lds)
{
    int top = NOT_ALLOWED;
    for (int i = threadIdx.x; i < g.opens; i += THREADS) top = max(top, g.tops[(size_t)at * g.opens + i]);
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = (u32)top;
    __syncthreads();
    for (int w = 0; w < WAVES; w++) top = max(top, (int)lds[w]);
    __syncthreads();
    return top;
}

// Eight keys of a lane: its wave takes the 512 of a chunk.  (Behind the row's end: not allowed.)
__device__ __forceinline__ void load_keys(const sample_args &g, u32 at, int chunk, int (&k)[8])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int j = chunk * CHUNK + i * 256 + lane * 4;
        int4 v = {NOT_ALLOWED, NOT_ALLOWED, NOT_ALLOWED, NOT_ALLOWED};
        if (j < g.key_ld) v = *reinterpret_cast<const int4 *>(g.keys + (size_t)at * g.key_ld + j);
        k[4 * i] = v.x, k[4 * i + 1] = v.y, k[4 * i + 2] = v.z, k[4 * i + 3] = v.w;
    }
}

// The histogram of a part of a row, in LDS first.  Bound by the weights' multiplications and two atomics of LDS to a token; rows without a cut only start and end.
// 1 row of 32000 5.2 us, 8 rows of 128000 6.2, 64 rows of 200003 without cuts 4.6.
__global__ __launch_bounds__(THREADS) void count_kernel(sample_args g)
{
    __shared__ u32 count[BINS];
    __shared__ u64 sum[BINS];
    __shared__ u32 red[WAVES];
    const int tid = threadIdx.x;
    const u32 at = fd_div(blockIdx.x, g.dGroups), group = blockIdx.x - at * g.groups;
    const row_rule rule = rule_of(g.params[g.row0 + at], g.f);
    if (!rule.cuts()) return;
    int chunk = (int)group * WAVES + (tid >> 6), k[8];
    load_keys(g, at, chunk, k);
    for (int i = tid; i < BINS; i += THREADS) count[i] = 0, sum[i] = 0;
    const int top = top_of(g, at, red);
    while (chunk < g.chunks) {
        int next[8];
        load_keys(g, at, chunk += g.groups * WAVES, next);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const u32 d = (u32)top - (u32)k[i];
            if (k[i] != NOT_ALLOWED && d < rule.reach) {
                atomicAdd(&count[rule.bin_of(d)], 1u);
                atomicAdd((unsigned long long *)&sum[rule.bin_of(d)], (unsigned long long)rule.weight(d));
            }
            k[i] = next[i];
        }
    }
    __syncthreads();
    for (int i = tid; i < BINS; i += THREADS)
        if (count[i]) {
            atomicAdd(g.count + (size_t)at * BINS + i, count[i]);
            atomicAdd((unsigned long long *)(g.sum + (size_t)at * BINS + i), (unsigned long long)sum[i]);
        }
}

// the plan of a row from its histogram in memory
__device__ __forceinline__ row_plan load_plan(const sample_args &g, u32 at, row_state &s, const row_rule &rule)
{
    if (!rule.cuts()) return {rule.reach, {0, 0, 0, 0}, {0, 0, 0, 0}};
    for (int i = threadIdx.x; i < BINS; i += THREADS) s.count[i] = g.count[(size_t)at * BINS + i], s.sum[i] = g.sum[(size_t)at * BINS + i];
    __syncthreads();
    return plan_row(s, rule);
}

__device__ __forceinline__ bool in_ranges(const row_plan &p, u32 d) { return d - p.few.lo < p.few.span || d - p.part.lo < p.part.span; }

// What a wave does with a chunk once the plan is known: what is sure of it, its tokens near the cuts to the list
__device__ __forceinline__ void collect_chunk(const sample_args &g, u32 at, int chunk, const int (&k)[8], int top, const row_rule &rule, const row_plan &plan)
{
    const int lane = threadIdx.x & 63;
    u64 sum = 0;
    unsigned long long near[8];                  // lanes whose token is near a cut
    u32 listed = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const u32 d = (u32)top - (u32)k[i];
        const bool live = k[i] != NOT_ALLOWED && d < rule.reach;
        if (live && d < plan.sure) {
            const u32 w = rule.weight(d);
            if (w >= rule.least) sum += w;
        }
        near[i] = __ballot(live && in_ranges(plan, d));
        listed += (u32)__popcll(near[i]);
    }
    if (listed) {                                // (one place in the list for all of them: the wave waits for it once)
        u32 first = 0;
        if (lane == 0) first = atomicAdd(g.listed + at, listed);
        first = (u32)__builtin_amdgcn_readfirstlane((int)first);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const u32 place = first + (u32)__popcll(near[i] & ((1ull << lane) - 1));
            if ((near[i] >> lane & 1) && place < (u32)SAMPLE_LIST)
                g.list[(size_t)at * SAMPLE_LIST + place] = (u64)((u32)top - (u32)k[i]) << 20 | (u32)(chunk * CHUNK + (i >> 2) * 256 + lane * 4 + (i & 3));
            first += (u32)__popcll(near[i]);
        }
    }
    sum = wave_sum(sum);
    if (lane == 0) g.sure[(size_t)at * g.chunks + chunk] = sum;
}

// Bound by loading the histogram and its block sums (5 us), then by the weights' 32-bit multiplications, at a quarter of the rate.  1 row of 32000 7.5 us,
// 8 of 128000 10, 64 of 200003 19.
__global__ __launch_bounds__(THREADS) void collect_kernel(sample_args g)
{
    __shared__ row_state s;
    const u32 at = fd_div(blockIdx.x, g.dGroups), group = blockIdx.x - at * g.groups;
    const row_rule rule = rule_of(g.params[g.row0 + at], g.f);
    int chunk = (int)group * WAVES + (threadIdx.x >> 6), k[8];
    load_keys(g, at, chunk, k);
    const int top = top_of(g, at, s.red32);
    const row_plan plan = load_plan(g, at, s, rule);
    if (group == 0 && threadIdx.x == 0) g.plans[at] = plan;
    while (chunk < g.chunks) {
        int next[8];
        load_keys(g, at, chunk + g.groups * WAVES, next);
        collect_chunk(g, at, chunk, k, top, rule, plan);
        chunk += g.groups * WAVES;
#pragma unroll
        for (int i = 0; i < 8; i++) k[i] = next[i];
    }
}

// One workgroup to a row, bound by its chain of block sums and loads: 7 us without a cut, 8 to 10 with them.
__global__ __launch_bounds__(THREADS) void pick_kernel(sample_args g)
{
    __shared__ row_state s;
    const int row = g.row0 + blockIdx.x;
    const u32 at = blockIdx.x;
    const row_rule rule = rule_of(g.params[row], g.f);
    const int top = top_of(g, at, s.red32);
    if (top == NOT_ALLOWED) {
        if (threadIdx.x == 0) g.tokens[row] = -1, g.shown[row] = 0;
        return;
    }
    const row_plan plan = g.plans[at];
    const int *keys = g.keys + (size_t)at * g.key_ld;
    const u64 *list = g.list + (size_t)at * SAMPLE_LIST;
    const u32 listed = g.listed[at];
    auto each = [&](auto &&f) {
        if (listed <= (u32)SAMPLE_LIST) {
            for (u32 i = threadIdx.x; i < listed; i += THREADS) f((u32)(list[i] >> 20), (int)(list[i] & 0xFFFFF));
            return;
        }
        for (int j = threadIdx.x; j < g.vocab; j += THREADS) {   // many equal logits
            const u32 d = (u32)top - (u32)keys[j];
            if (keys[j] != NOT_ALLOWED && d < rule.reach && in_ranges(plan, d)) f(d, j);
        }
    };
    draw_token(g, row, s, rule, plan, top, each, [&](int c) { return g.sure[(size_t)at * g.chunks + c]; }, [&](int j) { return keys[j]; });
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

hipError_t ss_launch_sample(const sample_plan &plan, const ss_sampling &q, const u64 *logits, size_t ld, int rows, int vocab, int f, const ss_rec_params &rp,
                            void *room, long long *tokens, int *shown, hipStream_t stream)
{
    sample_args g = {};
    g.logits = logits, g.ld = ld, g.rows = rows, g.vocab = vocab, g.f = f;
    g.params = q.params, g.random = q.random, g.allowed = q.allowed, g.ld_allowed = q.ld_allowed, g.tokens = tokens, g.shown = shown;
    if (plan.small) {
        hipLaunchKernelGGL((vocab <= SMALL_VOCAB ? sample_kernel<SMALL_VOCAB> : sample_kernel<MEDIUM_VOCAB>), dim3(rows), dim3(THREADS), 0, stream, g, rp);
        return hipGetLastError();
    }
    g.opens = plan.opens, g.groups = plan.groups, g.chunks = plan.chunks, g.key_ld = plan.key_ld;
    g.dOpens = make_fdiv((u32)plan.opens), g.dGroups = make_fdiv((u32)plan.groups);
    char *at = (char *)room;
    g.sum = (u64 *)at, at += (size_t)plan.slab * BINS * 8;
    g.sure = (u64 *)at, at += (size_t)plan.slab * ((plan.chunks + 1) & ~1) * 8;
    g.list = (u64 *)at, at += (size_t)plan.slab * SAMPLE_LIST * 8;
    g.plans = (row_plan *)at, at += (size_t)plan.slab * SAMPLE_PLAN;
    g.keys = (int *)at, at += (size_t)plan.slab * plan.key_ld * 4;
    g.count = (u32 *)at, at += (size_t)plan.slab * BINS * 4;
    g.tops = (int *)at, at += (size_t)plan.slab * plan.opens * 4;
    g.listed = (u32 *)at;
    static_assert(sizeof(row_plan) <= SAMPLE_PLAN && alignof(row_plan) <= 16, "a row's plan has its room");
    const bool wide = ld % 2 == 0 && aligned16(logits);
    const bool streams = (size_t)rp.m * rows * vocab * 8 > STREAMED_BYTES;
    const auto open = wide ? streams ? open_kernel<true, true> : open_kernel<true, false> : streams ? open_kernel<false, true> : open_kernel<false, false>;
    for (g.row0 = 0; g.row0 < rows; g.row0 += plan.slab) {
        const unsigned now = (unsigned)std::min(plan.slab, rows - g.row0);
        hipLaunchKernelGGL(open, dim3(now * plan.opens), dim3(OPEN_THREADS), 0, stream, g, rp);
        hipLaunchKernelGGL(count_kernel, dim3(now * plan.groups), dim3(THREADS), 0, stream, g);
        hipLaunchKernelGGL(collect_kernel, dim3(now * plan.groups), dim3(THREADS), 0, stream, g);
        hipLaunchKernelGGL(pick_kernel, dim3(now), dim3(THREADS), 0, stream, g);
    }
    return hipGetLastError();
}

}  // namespace SS_NS
