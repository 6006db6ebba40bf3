// The next token of every row from shares of its logits: REC, then a draw in whole numbers from the softmax of the row, cut by top-k, top-p and
// min-p.  The tokens that may be drawn are the first ones in the order of falling logits, equal ones by their number, so a cut is a distance from
// the row's largest logit and how many of the tokens at that distance are kept; it is found by histograms of distances, digit by digit.
#include "kernels.hpp"
#include "power2.hpp"

namespace SS_NS {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = 2048, BIN_BITS = 11;
constexpr int NOT_ALLOWED = -2147483647 - 1;

struct sample_args {
    const u64 *logits;              // [n][rows][ld]
    size_t ld;
    int rows, vocab, f;
    const int4 *params;             // scale, top_k, top_p, min_p
    const long long *random;
    const u32 *allowed;             // a bit to a token, or nullptr
    size_t ld_allowed;
    int *keys;                      // [rows][vocab]: logits in units of 2^-min(f, 16)
    long long *tokens;
    int *shown;                     // probability of the token, 30 fraction bits
};

// the opened logit in units of 2^-min(f, 16), the far ones as the last that 32 bits hold
__device__ __forceinline__ int logit_of(u64 v, int f)
{
    const long long s = (v <= (SS_P - 1) / 2 ? (long long)v : (long long)v - (long long)SS_P) >> (f - min(f, 16));
    return (int)min(max(s, -2147483647ll), 2147483647ll);
}

// what a row asks for, and the weight of a distance
struct row_rule {
    u32 scale, least;               // smallest weight that is kept
    int shift;
    u64 reach;                      // distances from here on have no weight
    __device__ __forceinline__ u32 weight(u32 distance) const { return power2((u64)distance * scale >> shift); }
};

template <typename T>
__device__ __forceinline__ T wave_upto(T v)      // sum of the lanes up to one's own
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T x = __shfl_up(v, d);
        if (lane >= d) v += x;
    }
    return v;
}

template <typename T>
__device__ __forceinline__ T wave_sum(T v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// sum over the threads up to one's own, and over all of them; lds: one for each wave
template <typename T>
__device__ __forceinline__ T block_upto(T v, T *lds, T &all)
{
    const int wave = threadIdx.x >> 6;
    v = wave_upto(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[wave] = v;
    __syncthreads();
    T before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; w++) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    return v + before;
}

// tokens at a distance below `distance` and at it; of the latter the first `ties` are kept
struct cut_place {
    u32 distance;
    u32 ties;
    u64 before;                     // weight of the former
};

struct row_state {
    u32 count[BINS];
    u64 sum[BINS];
    u64 red64[WAVES];
    u32 red32[WAVES];
    int bin;
    u64 before_sum;
    u32 before_count, at;
};

// The first distance at which the tokens up to it are `few` (BY_SUM: weigh `need`), or no place if they are less altogether.  total: weight of all
// tokens, set by the first histogram; need_of(total) gives what is needed.
template <bool BY_SUM, typename F>
__device__ __forceinline__ bool find_cut(const int *keys, int vocab, int top, const row_rule &rule, row_state &s, u32 few, F &&need_of, u64 &total, cut_place &cut)
{
    const int tid = threadIdx.x;
    int shift = 0;
    while ((rule.reach - 1) >> shift >= BINS) shift++;
    u64 lo = 0, need = 0, before_sum = 0;
    u32 before_count = 0;
    for (bool first = true;; first = false) {
        for (int i = tid; i < BINS; i += THREADS) s.count[i] = 0, s.sum[i] = 0;
        if (tid == 0) s.bin = BINS;
        __syncthreads();
        for (int j = tid; j < vocab; j += THREADS) {
            const int key = keys[j];
            const u32 d = (u32)top - (u32)key;
            if (key == NOT_ALLOWED || d >= rule.reach || d < lo) continue;
            const u64 bin = (d - lo) >> shift;
            if (bin >= BINS) continue;
            atomicAdd(&s.count[bin], 1u);
            atomicAdd((unsigned long long *)&s.sum[bin], (unsigned long long)rule.weight(d));
        }
        __syncthreads();
        const u32 c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1];
        const u64 s0 = s.sum[2 * tid], s1 = s.sum[2 * tid + 1];
        u32 all_count;
        u64 all_sum;
        const u32 c = before_count + block_upto(c0 + c1, s.red32, all_count);
        const u64 w = before_sum + block_upto(s0 + s1, s.red64, all_sum);
        if (first) {
            total = all_sum;
            need = BY_SUM ? need_of(total) : 0;
            if (!BY_SUM && all_count < few) return false;
        }
        const bool past0 = BY_SUM ? w - s1 >= need : c - c1 >= few, past1 = BY_SUM ? w >= need : c >= few;
        if (past1) atomicMin(&s.bin, past0 ? 2 * tid : 2 * tid + 1);
        __syncthreads();
        if (s.bin >> 1 == tid) {
            const bool second = s.bin & 1;
            s.before_count = second ? c - c1 : c - c1 - c0;
            s.before_sum = second ? w - s1 : w - s1 - s0;
            s.at = second ? c1 : c0;
        }
        __syncthreads();
        before_count = s.before_count;
        before_sum = s.before_sum;
        lo += (u64)s.bin << shift;
        if (shift == 0) break;
        shift = max(0, shift - BIN_BITS);
        __syncthreads();
    }
    cut.distance = (u32)lo;
    cut.before = before_sum;
    if constexpr (BY_SUM) {
        const u32 w = rule.weight(cut.distance);
        cut.ties = (u32)((need - before_sum + w - 1) / w);
    } else {
        cut.ties = few - before_count;
    }
    __syncthreads();
    return true;
}

// One workgroup to a row.
__global__ __launch_bounds__(THREADS) void sample_kernel(sample_args g, ss_rec_params rp)
{
    __shared__ row_state s;
    const int tid = threadIdx.x, row = blockIdx.x;
    int *keys = g.keys + (size_t)row * g.vocab;
    const int4 p = g.params[row];
    int top = NOT_ALLOWED;
    for (int j = tid; j < g.vocab; j += THREADS) {
        ss_sacc acc;
        acc.clear();
        for (int i = 0; i < rp.m; i++) acc.mac(g.logits[((size_t)rp.plane[i] * g.rows + row) * g.ld + j], rp.ilambda[i]);
        const u64 v = rp.dinv == 1 ? acc.value() : ss_mul(acc.value(), rp.dinv);
        const bool allowed = !g.allowed || (g.allowed[row * g.ld_allowed + (j >> 5)] >> (j & 31) & 1);
        const int key = allowed ? logit_of(v, g.f) : NOT_ALLOWED;
        keys[j] = key;
        top = max(top, key);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) top = max(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) s.red32[tid >> 6] = (u32)top;
    __syncthreads();
    for (int w = 0; w < WAVES; w++) top = max(top, (int)s.red32[w]);
    __syncthreads();
    if (top == NOT_ALLOWED) {
        if (tid == 0) g.tokens[row] = -1, g.shown[row] = 0;
        return;
    }
    row_rule rule;
    rule.scale = (u32)max(p.x, 1 << 14);
    rule.least = (u32)min(max(p.w, 1), 1 << 30);
    rule.shift = min(g.f, 16) + 8;
    rule.reach = ((31ull << (16 + rule.shift)) + rule.scale - 1) / rule.scale;   // <= 31 2^26
    cut_place cut = {(u32)rule.reach, 0, 0};
    u64 total = 0;
    const u32 few = p.x <= 0 ? 1 : p.y <= 0 ? 0 : (u32)p.y;
    bool limited = few && find_cut<false>(keys, g.vocab, top, rule, s, few, [](u64) { return 0ull; }, total, cut);
    if (p.z < 1 << 30) {
        const u64 within = limited ? cut.before + (u64)cut.ties * rule.weight(cut.distance) : 0;
        const u32 part = (u32)max(p.z, 0);
        find_cut<true>(keys, g.vocab, top, rule, s, 0, [&](u64 all) {
            const u64 of = limited ? within : all, lo = of * part, hi = __umul64hi(of, part);
            return max(1ull, (unsigned long long)((hi << 34 | lo >> 30) + ((lo & ((1 << 30) - 1)) != 0)));
        }, total, cut);
    }
    // weights of chunks of 1024 tokens in their own order, tokens at the cut apart
    const u32 at_cut = cut.distance < rule.reach ? rule.weight(cut.distance) : 0;
    const int lane = tid & 63, chunks = (g.vocab + THREADS - 1) / THREADS;
    for (int c = tid >> 6; c < chunks; c += WAVES) {
        u64 sum = 0;
        u32 ties = 0;
        for (int i = 0; i < THREADS; i += 64) {
            const int j = c * THREADS + i + lane;
            if (j >= g.vocab) continue;
            const int key = keys[j];
            const u32 d = (u32)top - (u32)key;
            if (key == NOT_ALLOWED || d > cut.distance) continue;
            const u32 w = d < rule.reach ? rule.weight(d) : 0;
            if (w < rule.least) continue;
            if (d == cut.distance) ties++; else sum += w;
        }
        sum = wave_sum(sum), ties = wave_sum(ties);
        if (lane == 0) s.sum[c] = sum, s.count[c] = ties;
    }
    __syncthreads();
    const u32 mine = tid < chunks ? s.count[tid] : 0;
    u32 all_ties;
    u64 sum;
    const u32 ties_before = block_upto(mine, s.red32, all_ties) - mine;
    const u64 weight = (tid < chunks ? s.sum[tid] : 0) + (u64)at_cut * min(mine, cut.ties > ties_before ? cut.ties - ties_before : 0);
    const u64 upto = block_upto(weight, s.red64, sum);
    const u64 target = __umul64hi((u64)g.random[row] << 2, sum);
    if (upto - weight <= target && target < upto) {
        s.bin = tid;
        s.before_count = ties_before;
        s.before_sum = upto - weight;
    }
    __syncthreads();
    const int j = s.bin * THREADS + tid;
    const int key = j < g.vocab ? keys[j] : NOT_ALLOWED;
    const u32 d = (u32)top - (u32)key, w0 = key != NOT_ALLOWED && d < rule.reach && d <= cut.distance ? rule.weight(d) : 0;
    const bool tie = w0 >= rule.least && d == cut.distance;
    const u32 rank = s.before_count + block_upto((u32)tie, s.red32, all_ties);
    const u64 before = s.before_sum;
    const u64 w = w0 < rule.least || (tie && rank > cut.ties) ? 0 : w0;
    u64 chunk;
    const u64 to = before + block_upto(w, s.red64, chunk);
    if (to - w <= target && target < to) {
        g.tokens[row] = j;
        g.shown[row] = (int)(((w << 30) + sum / 2) / sum);
    }
}

}  // namespace

hipError_t ss_launch_sample(const ss_sampling &q, const u64 *logits, size_t ld, int rows, int vocab, int f, const ss_rec_params &rp, void *room, long long *tokens,
                            int *shown, hipStream_t stream)
{
    const sample_args g = {logits, ld, rows, vocab, f, q.params, q.random, q.allowed, q.ld_allowed, (int *)room, tokens, shown};
    hipLaunchKernelGGL(sample_kernel, dim3(rows), dim3(THREADS), 0, stream, g, rp);
    return hipGetLastError();
}

}  // namespace SS_NS
