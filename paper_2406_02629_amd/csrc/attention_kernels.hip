// What a transformer block needs beside its dense layers, on shares: rotary positions, a paged cache of keys and values, and the
// attention of new tokens over it.
//
// Attention of a row (token, head) over the keys j < limit, all parties holding degree-t shares:
//   1. party i = 1..2t+1: score S_i[j] = q_i . k_i[j] mod p (degree 2t, 2 f fraction bits), plus its share of a mask that is the same for
//      all keys of the row, shared afresh with degree 2t for every key                            -> msg[i][row][j]
//      (of keys that the row does not see nothing is sent: the mask would not hide their differences from the others)
//   2. the elite party reconstructs s[j] + mask, takes the softmax of the row, which no constant added to it changes, as whole
//      numbers (softmax_weight below), and shares the weights (degree t); every party's share of a key beyond the limit is 0
//   3. every party i = 1..n: O_i = sum_j P_i[j] v_i[j] mod p (degree 2t)
// Products run on int8 MFMA over balanced 8-bit digits, as in a dense layer.
//
// Every message lies in memory, as the protocol has it: a row of L keys costs 8 (2t+1) L bytes of scores and NL n L of weights, each written
// and read once, beside the cache itself.  So three kernels, not one: a workgroup that took all steps for its rows would
// take 2t+1 parties' keys and n parties' values one after the other (single tokens of 32 heads of 128 over 64 keys, n = 5: 24 to 46 us for one
// sequence to four, against 16 to 19.5).  Only softmax and values go together, over short contexts.
// Figures of the kernels below are those of MI355X, where a copy moves 6.3 TB/s, a sum reads 6.1 and int8 MFMA reaches 3.6 POP/s on random
// digits.
#include "kernels.hpp"
#include "eval.hpp"
#include "digits.hpp"
#include "diagonals.hpp"
#include "truncation.hpp"

namespace SS_NS {

namespace {

constexpr int BLOCK = 256;

inline unsigned ceil_div(size_t a, size_t b) { return (unsigned)((a + b - 1) / b); }

// what describes the call does not change while it runs: read by way of the scalar cache wherever the index is the same for a wave
typedef const int __attribute__((address_space(4))) *constant_ints;
__device__ __forceinline__ int fixed_at(const int *p, size_t i) { return ((constant_ints)(uintptr_t)p)[i]; }
typedef const long long __attribute__((address_space(4))) *constant_longs;
__device__ __forceinline__ long long fixed_at(const long long *p, size_t i) { return ((constant_longs)(uintptr_t)p)[i]; }

// ------------------------------------------------------------------ rotary positions

// a c - b s as any word of the right residue below 2^63; a, b canonical, |c|, |s| <= 2^31
__device__ __forceinline__ u64 turn(u64 a, int c, u64 b, long long s)
{
    const long long lo = (long long)(a & 0x7FFFFFFF) * c - (long long)(b & 0x7FFFFFFF) * s;   // two terms below 2^62 each
    const long long hi = (long long)(a >> 31) * c - (long long)(b >> 31) * s;
#if defined(SS_FIELD_P45)
    const u64 l = ((u64)lo & SS_PMASK) + (u64)(lo >> 45) * SS_PC + SS_P;   // > 0, < 2^47
    const u64 h = (u64)(hi + (long long)(SS_P << 2));                      // |hi| < 2^46
    return l + SS_PC * (h >> 14) + ((h & 0x3FFFull) << 31);                // h 2^31, h = a 2^14 + b: 55 a + b 2^31
#else
    const u64 l = ((u64)lo & SS_P) + (u64)(lo >> 61) + SS_P;               // > 0, < 2^62 + 4
    const u64 h = ((u64)hi & SS_P) + (u64)(hi >> 61) + SS_P;
    return l + ((h & 0x3FFFFFFFull) << 31) + (h >> 30);
#endif
}

// SSS-Truncation of VEC neighbours from element e on whose shares of the parties 1..k are xq (any residue below 2^63): the new shares in o[],
// the messages of both steps to u [k][count] and wsh [n][count]
template <int N, int T, int VEC, bool STREAM>
__device__ __forceinline__ void truncate_elements(const u64 (&xq)[VEC][T + 1], size_t e, size_t count, u64 *__restrict__ u, u64 *__restrict__ wsh,
                                                  const ss_tr_params &tp, pack_t<VEC> (&o)[MAXP<N>])
{
    constexpr int K = T + 1;
    const int n = N ? N : tp.n;
    pack_t<VEC> um[K], w[MAXP<N>];
#pragma unroll
    for (int c = 0; c < VEC; c++) {
        const u64 counter = ss_counter(e + c);
        u64 alpha, a[T], b[T];
        const u64 ev = mask_of<T>(tp, e + c, alpha);
#pragma unroll
        for (int j = 0; j < T; j++) a[j] = ss_draw_lazy_at(tp.alpha_key[j], counter);
        ss_sacc2 acc;
        acc.clear();
        eval_points<T, K>(alpha, a, [&](int q, u64 v) {
            const u64 m = ss_reduce(xq[c][q] + v);
            um[q].v[c] = m;
            SS_SPLIT31(m, w0, w1);
            acc.mac(w0, w1, tp.ilambda[q]);
        });
        // the elite party's quotient, shared; the mask off
        const u64 quotient = shift_signed(acc.value(), tp.f);
#pragma unroll
        for (int j = 0; j < T; j++) {
            a[j] = ss_draw_lazy_at(tp.gen_key[j], counter);
            b[j] = ss_fold(a[j] + ss_draw_lazy_at(tp.alphat_key[j], counter));
        }
        eval_points<T, MAXP<N>>(quotient, a, [&](int m, u64 v) { w[m].v[c] = v; }, n);
        eval_points<T, MAXP<N>>(ss_canon(quotient + SS_P - ev), b, [&](int m, u64 v) { o[m].v[c] = v; }, n);
    }
#pragma unroll
    for (int q = 0; q < K; q++) um[q].template send<STREAM>(u + (size_t)q * count + e);
#pragma unroll
    for (int m = 0; m < MAXP<N>; m++)
        if (N != 0 || m < n) w[m].template send<STREAM>(wsh + (size_t)m * count + e);
}

// how a tensor of heads is dealt to threads: `width` threads to each head, of which `pairs` turn pairs
struct rotary_shape {
    int tokens, heads, dim, width, pairs;
    fdiv dWidth, dHeads;
};

// cosine and sine of pair j of a token
__device__ __forceinline__ int2 angle_of(const ss_rope &rope, int token, int j)
{
    return rope.table[(size_t)min(max(rope.pos[token], 0), rope.positions - 1) * (rope.rot >> 1) + j];
}

// pair j of (token, head), elements a and b, rotated and truncated: shares of both
template <int N, int T>
__device__ __forceinline__ void rotate_pair(const u64 *x, size_t ld, const rotary_shape &g, int token, int head, int j, u64 *__restrict__ u,
                                            u64 *__restrict__ wsh, const ss_rope &rope, const ss_tr_params &tp, int &a, int &b,
                                            pack_t<1> (&oa)[MAXP<N>], pack_t<1> (&ob)[MAXP<N>])
{
    constexpr int K = T + 1;
    const int half = rope.rot >> 1;
    a = rope.interleaved ? 2 * j : j;
    b = rope.interleaved ? 2 * j + 1 : j + half;
    const u64 *row = x + (size_t)token * ld + (size_t)head * g.dim;
    const size_t party = (size_t)g.tokens * ld, count = (size_t)g.tokens * g.heads * rope.rot;
    const int2 cs = angle_of(rope, token, j);
    u64 ra[1][K], rb[1][K];
#pragma unroll
    for (int q = 0; q < K; q++) {
        const u64 xa = row[q * party + a], xb = row[q * party + b];
        ra[0][q] = turn(xa, cs.x, xb, cs.y);
        rb[0][q] = turn(xb, cs.x, xa, -(long long)cs.y);
    }
    const size_t e = ((size_t)token * g.heads + head) * rope.rot;
    truncate_elements<N, T, 1, false>(ra, e + a, count, u, wsh, tp, oa);
    truncate_elements<N, T, 1, false>(rb, e + b, count, u, wsh, tp, ob);
}

// One thread per pair, or element that passes through, of a head: for whatever the kernel below cannot load 16 bytes at a time.
template <int N, int T>
__global__ __launch_bounds__(BLOCK) void rotary_kernel(const u64 *x, size_t ld, u64 *__restrict__ u, u64 *__restrict__ wsh, u64 *out,
                                                       rotary_shape g, ss_rope rope, ss_tr_params tp)
{
    const u32 i = blockIdx.x * BLOCK + threadIdx.x;
    if (i >= (u32)(g.tokens * g.heads * g.width)) return;
    const u32 th = fd_div(i, g.dWidth), token = fd_div(th, g.dHeads), head = th - token * g.heads;
    const int j = (int)(i - th * g.width), n = N ? N : tp.n;
    const size_t count = (size_t)g.tokens * g.heads * g.dim;
    u64 *dst = out + (size_t)th * g.dim;
    if (j >= g.pairs) {
        const int d = j + g.pairs;
#pragma unroll
        for (int m = 0; m < MAXP<N>; m++)
            if (N != 0 || m < n) dst[m * count + d] = x[((size_t)m * g.tokens + token) * ld + (size_t)head * g.dim + d];
        return;
    }
    int a, b;
    pack_t<1> oa[MAXP<N>], ob[MAXP<N>];
    rotate_pair<N, T>(x, ld, g, (int)token, (int)head, j, u, wsh, rope, tp, a, b, oa, ob);
#pragma unroll
    for (int m = 0; m < MAXP<N>; m++)
        if (N != 0 || m < n) {
            oa[m].store(dst + m * count + a);
            ob[m].store(dst + m * count + b);
        }
}

// Neighbouring elements two at a time, 16 bytes to a load and a store: interleaved pair t, or pairs 2 t and 2 t + 1 of two halves, rotated and
// truncated; emit(element of the head, shares of it and of the next), once or twice.  src: the head in share 1, `party` elements to the next
// share, e: its number among the turned elements.  (Everything 16-byte aligned, strides and halves even.)
template <int N, int T, bool INTERLEAVED, bool STREAM, typename F>
__device__ __forceinline__ void rotate_two(const u64 *src, size_t party, size_t e, size_t count, int token, int t, u64 *__restrict__ u,
                                           u64 *__restrict__ wsh, const ss_rope &rope, const ss_tr_params &tp, F &&emit)
{
    constexpr int K = T + 1;
    pack_t<2> o[MAXP<N>];
    u64 r[2][K];
    if constexpr (INTERLEAVED) {
        const int2 cs = angle_of(rope, token, t);
#pragma unroll
        for (int q = 0; q < K; q++) {
            pack_t<2> v;
            v.load(src + q * party + 2 * t);
            r[0][q] = turn(v.v[0], cs.x, v.v[1], cs.y);
            r[1][q] = turn(v.v[1], cs.x, v.v[0], -(long long)cs.y);
        }
        truncate_elements<N, T, 2, STREAM>(r, e + 2 * t, count, u, wsh, tp, o);
        emit(2 * t, o);
    } else {
        const int half = rope.rot >> 1, j = 2 * t;
        const int2 c0 = angle_of(rope, token, j), c1 = angle_of(rope, token, j + 1);
        u64 rb[2][K];
#pragma unroll
        for (int q = 0; q < K; q++) {
            pack_t<2> a, b;
            a.load(src + q * party + j);
            b.load(src + q * party + j + half);
            r[0][q] = turn(a.v[0], c0.x, b.v[0], c0.y);
            r[1][q] = turn(a.v[1], c1.x, b.v[1], c1.y);
            rb[0][q] = turn(b.v[0], c0.x, a.v[0], -(long long)c0.y);
            rb[1][q] = turn(b.v[1], c1.x, a.v[1], -(long long)c1.y);
        }
        truncate_elements<N, T, 2, STREAM>(r, e + j, count, u, wsh, tp, o);
        emit(j, o);
        truncate_elements<N, T, 2, STREAM>(rb, e + j + half, count, u, wsh, tp, o);
        emit(j + half, o);
    }
}

// The rotation of a head in such steps, or two elements that pass through, to a thread.  The random polynomials of the truncation are drawn
// where they are used, so that memory bounds it: shares in and out, t + 1 + n words of messages per element.  2048 tokens, 32 heads of
// 128, half of each turned, n = 3: 93 us, 537 MB at 5.8 TB/s (one thread per pair: 118).  8 tokens, n = 5: 7 us, a launch and one element's
// chain of draws.  STREAM: messages and results past the caches.
template <int N, int T, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(BLOCK) void rotary_wide_kernel(const u64 *x, size_t ld, u64 *__restrict__ u, u64 *__restrict__ wsh, u64 *out,
                                                            rotary_shape g, ss_rope rope, ss_tr_params tp)
{
    const u32 i = blockIdx.x * BLOCK + threadIdx.x;
    if (i >= (u32)(g.tokens * g.heads * g.width)) return;
    const u32 th = fd_div(i, g.dWidth), token = fd_div(th, g.dHeads), head = th - token * g.heads;
    const int t = (int)(i - th * g.width), n = N ? N : tp.n;
    const size_t plane = (size_t)g.tokens * g.heads * g.dim, party = (size_t)g.tokens * ld, count = (size_t)g.tokens * g.heads * rope.rot;
    const u64 *src = x + (size_t)token * ld + (size_t)head * g.dim;
    u64 *dst = out + (size_t)th * g.dim;
    if (t >= g.pairs) {
        const int d = rope.rot + 2 * (t - g.pairs);
#pragma unroll
        for (int m = 0; m < MAXP<N>; m++)
            if (N != 0 || m < n) {
                pack_t<2> v;
                v.load(src + m * party + d);
                v.template send<STREAM>(dst + m * plane + d);
            }
        return;
    }
    rotate_two<N, T, INTERLEAVED, STREAM>(src, party, (size_t)th * rope.rot, count, (int)token, t, u, wsh, rope, tp,
                                          [&](int d, const pack_t<2> (&o)[MAXP<N>]) {
#pragma unroll
                                              for (int m = 0; m < MAXP<N>; m++)
                                                  if (N != 0 || m < n) o[m].template send<STREAM>(dst + m * plane + d);
                                          });
}

// ------------------------------------------------------------------ appending to the cache

struct append_shape {
    rotary_shape r;
    const long long *slots;
    signed char *keys, *values;
    size_t party, head, page;          // strides in bytes
    unsigned capacity, page_size;      // keys of the cache, of a page
    int steps, step_blocks;            // many tokens: threads to a key, in blocks of 16
    int value_blocks;                  // workgroups to 16 tokens of the values
    fdiv dPage;
};

// of the token's place in the cache: its cell in head 0 of party 0, and the key inside the cell
__device__ __forceinline__ bool place_of(const append_shape &s, int token, size_t &cell, int &key)
{
    const long long slot = fixed_at(s.slots, token);
    if (slot < 0 || slot >= (long long)s.capacity) return false;
    const u32 page = fd_div((u32)slot, s.dPage), in = (u32)slot - page * s.page_size;
    key = (int)(in & 15);
    cell = page * s.page + (size_t)(in >> 4) * (SS_NLIMB * 16) * s.r.dim;
    return true;
}

template <int N>
__device__ __forceinline__ void put_key(const append_shape &s, size_t cell, int key, int head, int d, const pack_t<1> (&v)[MAXP<N>], int n)
{
#pragma unroll
    for (int m = 0; m < MAXP<N>; m++)
        if (N != 0 || m < n) {
            const u64 dig = balanced_digits(v[m].v[0]);
            signed char *c = s.keys + cell + m * s.party + head * s.head + (d >> 4) * 256 + key * 16 + (d & 15);
#pragma unroll
            for (int l = 0; l < SS_NLIMB; l++) c[(size_t)l * s.r.dim * 16] = (signed char)(dig >> (8 * l));
        }
}

// A few tokens: one thread per pair (or element that passes through) of a key, then one per element of a value; digits go out as bytes.  A
// launch and one element's chain of draws bound it: 8 tokens of 8 heads of 128, n = 5, 6.1 us.
template <int N, int T>
__global__ __launch_bounds__(BLOCK) void append_kernel(const u64 *k, size_t ld_k, const u64 *v, size_t ld_v, u64 *__restrict__ u,
                                                       u64 *__restrict__ wsh, append_shape s, ss_rope rope, ss_tr_params tp, u32 key_blocks)
{
    const int n = N ? N : tp.n;
    const rotary_shape &g = s.r;
    pack_t<1> o[MAXP<N>];
    size_t cell;
    int key;
    if (blockIdx.x >= key_blocks) {
        const u32 i = (blockIdx.x - key_blocks) * BLOCK + threadIdx.x;
        if (i >= (u32)(g.tokens * g.heads * g.dim)) return;
        const u32 per = (u32)(g.heads * g.dim), token = i / per, rest = i - token * per, head = rest / g.dim, d = rest - head * g.dim;
        if (!place_of(s, (int)token, cell, key)) return;
#pragma unroll
        for (int m = 0; m < MAXP<N>; m++)
            if (N != 0 || m < n) {
                const u64 dig = balanced_digits(v[((size_t)m * g.tokens + token) * ld_v + rest]);
                signed char *c = s.values + cell + m * s.party + head * s.head + d * 16 + key;
#pragma unroll
                for (int l = 0; l < SS_NLIMB; l++) c[(size_t)l * g.dim * 16] = (signed char)(dig >> (8 * l));
            }
        return;
    }
    const u32 i = blockIdx.x * BLOCK + threadIdx.x;
    if (i >= (u32)(g.tokens * g.heads * g.width)) return;
    const u32 th = fd_div(i, g.dWidth), token = fd_div(th, g.dHeads), head = th - token * g.heads;
    const int j = (int)(i - th * g.width);
    const bool placed = place_of(s, (int)token, cell, key);
    if (j >= g.pairs) {
        if (!placed) return;
        const int d = j + g.pairs;
#pragma unroll
        for (int m = 0; m < MAXP<N>; m++)
            if (N != 0 || m < n) o[m].load(k + ((size_t)m * g.tokens + token) * ld_k + (size_t)head * g.dim + d);
        put_key<N>(s, cell, key, (int)head, d, o, n);
        return;
    }
    int a, b;
    pack_t<1> ob[MAXP<N>];
    rotate_pair<N, T>(k, ld_k, g, (int)token, (int)head, j, u, wsh, rope, tp, a, b, o, ob);
    if (!placed) return;
    put_key<N>(s, cell, key, (int)head, a, o, n);
    put_key<N>(s, cell, key, (int)head, b, ob, n);
}

// Many tokens go in blocks of 16 that end with a cell if the tokens follow one another in the cache: the first block lacks as many as there
// are keys in front of the first token.
__device__ __forceinline__ int first_of_block(const append_shape &s, int block)
{
    const long long slot = fixed_at(s.slots, 0);
    return block * 16 - (slot < 0 ? 0 : (int)(slot & 15));
}

// Elements d and d + 1 of a key, from each of two neighbouring lanes, which have four in a row between them: each lane stores the dwords of half
// of the limbs.
template <int N, typename F>
__device__ __forceinline__ void put_key_four(const append_shape &s, size_t cell, int key, int head, int d, int n, F &&value)
{
    constexpr int HALF = SS_NLIMB / 2;
    const bool odd = threadIdx.x & 1;
    signed char *c = s.keys + cell + head * s.head + (d >> 4) * 256 + key * 16 + (d & 12) + (odd ? (size_t)HALF * s.r.dim * 16 : 0);
#pragma unroll
    for (int m = 0; m < MAXP<N>; m++)
        if (N != 0 || m < n) {
            u32 y[4];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const u64 dig = balanced_digits(value(m, i));
                const u32 low = (u32)dig, high = (u32)(dig >> (8 * HALF)), keep = odd ? high : low, give = odd ? low : high;
                const u32 got = (u32)__builtin_amdgcn_update_dpp(0, (int)give, 0xB1, 0xF, 0xF, true);   // the other lane of the two
                y[i] = odd ? got : keep;
                y[2 + i] = odd ? keep : got;
            }
#pragma unroll
            for (int l = 0; l < HALF; l++) {
                const u32 sel = (u32)l | ((u32)(4 + l) << 8) | 0x0c0c0000u;
                *reinterpret_cast<u32 *>(c + m * s.party + (size_t)l * s.r.dim * 16) =
                    __builtin_amdgcn_perm(__builtin_amdgcn_perm(y[3], y[2], sel), __builtin_amdgcn_perm(y[1], y[0], sel), 0x05040100u);
            }
        }
}

// Many tokens, keys: eight lanes take 16 elements (or twice 16) of a token two (or two and two) at a time, a wave eight tokens, so that where
// the tokens follow one another in the cache its dwords of a limb lie in a row, 128 bytes of a cell.  (Halves of a head in multiples of
// four, 16-byte alignment.)
template <int N, int T, bool INTERLEAVED>
__device__ __forceinline__ void append_keys(const u64 *k, size_t ld, u64 *__restrict__ u, u64 *__restrict__ wsh, const append_shape &s,
                                            const ss_rope &rope, const ss_tr_params &tp, int group, int step_block, int head)
{
    const int n = N ? N : tp.n, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const rotary_shape &g = s.r;
    const int step = step_block * 16 + (wave >> 1) * 8 + (lane & 7);
    const int token = first_of_block(s, group) + (wave & 1) * 8 + (lane >> 3);
    if (token < 0 || token >= g.tokens || step >= s.steps) return;   // (never one of two lanes alone: steps are even)
    size_t cell;
    int key;
    const bool placed = place_of(s, token, cell, key);
    const size_t party = (size_t)g.tokens * ld;
    const u64 *src = k + (size_t)token * ld + (size_t)head * g.dim;
    const int turning = INTERLEAVED ? g.pairs : g.pairs >> 1;
    if (step >= turning) {
        if (!placed) return;
        const int d = rope.rot + (step - turning) * 2;
        put_key_four<N>(s, cell, key, head, d, n, [&](int m, int i) { return src[m * party + d + i]; });
        return;
    }
    const size_t count = (size_t)g.tokens * g.heads * rope.rot, e = ((size_t)token * g.heads + head) * rope.rot;
    rotate_two<N, T, INTERLEAVED, false>(src, party, e, count, token, step, u, wsh, rope, tp, [&](int d, const pack_t<2> (&o)[MAXP<N>]) {
        if (placed) put_key_four<N>(s, cell, key, head, d, n, [&](int m, int i) { return o[m].v[i]; });
    });
}

// Many tokens, values: a thread takes one element of 16 tokens of one party.  Where they are the 16 keys of a cell, in order, it stores 16
// bytes of every limb and a wave 1 KB in a row; otherwise (ends of a run of tokens) bytes.
__device__ __forceinline__ void append_values(const u64 *v, size_t ld, const append_shape &s, int group, int m, int d, int head)
{
    const rotary_shape &g = s.r;
    const int t0 = first_of_block(s, group);
    const u64 *src = v + (size_t)m * g.tokens * ld + (size_t)head * g.dim + d;
    u64 y[4][4];
#pragma unroll
    for (int i = 0; i < 16; i++) y[i >> 2][i & 3] = src[(size_t)min(max(t0 + i, 0), g.tokens - 1) * ld];
    size_t cell;
    int key;
    bool run = t0 >= 0 && t0 + 16 <= g.tokens && place_of(s, t0, cell, key) && key == 0;   // uniform
    if (run) {
        const long long slot = fixed_at(s.slots, t0);
#pragma unroll
        for (int i = 1; i < 16; i++) run &= fixed_at(s.slots, t0 + i) == slot + i;
    }
#pragma unroll
    for (int i = 0; i < 16; i++) y[i >> 2][i & 3] = balanced_digits(y[i >> 2][i & 3]);
    signed char *dst = s.values + m * s.party + head * s.head + d * 16;
    const size_t limb = (size_t)g.dim * 16;
    if (run) {
#pragma unroll
        for (int l = 0; l < SS_NLIMB; l++)
            *reinterpret_cast<v4i *>(dst + cell + l * limb) =
                (v4i){(int)limb_dword(y[0], l), (int)limb_dword(y[1], l), (int)limb_dword(y[2], l), (int)limb_dword(y[3], l)};
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; i++)
        if (t0 + i >= 0 && t0 + i < g.tokens && place_of(s, t0 + i, cell, key)) {
#pragma unroll
            for (int l = 0; l < SS_NLIMB; l++) dst[cell + l * limb + key] = (signed char)(y[i >> 2][i & 3] >> (8 * l));
        }
}

// Both in one launch, bound by memory: keys, values and their digits, t + 1 + n words of messages per element of a key.  2048 tokens of 8 heads of
// 128, n = 5, one run of places: 98 us, 436 MB at 4.4 TB/s (the kernel for a few tokens, whose bytes go out one by one: 269).
// Grid.x: blocks of 16 tokens by blocks of 16 steps of the keys, then by blocks of 256 elements and parties of the values; grid.y: heads.
template <int N, int T, bool INTERLEAVED>
__global__ __launch_bounds__(BLOCK) void append_many_kernel(const u64 *k, size_t ld_k, const u64 *v, size_t ld_v, u64 *__restrict__ u,
                                                            u64 *__restrict__ wsh, append_shape s, ss_rope rope, ss_tr_params tp, int key_blocks,
                                                            fdiv dDim)
{
    const int n = N ? N : tp.n, head = blockIdx.y;
    if ((int)blockIdx.x < key_blocks) {
        const int group = (int)blockIdx.x / s.step_blocks;
        append_keys<N, T, INTERLEAVED>(k, ld_k, u, wsh, s, rope, tp, group, (int)blockIdx.x - group * s.step_blocks, head);
        return;
    }
    const int at = (int)blockIdx.x - key_blocks, group = at / s.value_blocks;
    const u32 i = (u32)(at - group * s.value_blocks) * BLOCK + threadIdx.x, m = fd_div(i, dDim);
    if ((int)m < n) append_values(v, ld_v, s, group, (int)m, (int)(i - m * s.r.dim), head);
}

// ------------------------------------------------------------------ attention

struct attn_args {
    ss_paged c;
    ss_sequences s;
    size_t cell, head_bytes, party_bytes, page_bytes;
    int heads, group, causal;
    int tok0, tok1;                 // the slab
    fdiv dGroup, dCells, dHeads, dScores, dValues;   // Scores, Values: by heads x parties
    const u64 *q;
    size_t ld_q;
    u64 *msg;                       // [2t+1][rows][keys]
    u64 *opened, *tops, *sums;      // of long rows: [rows][keys], [rows][keys / 1024]
    signed char *weights;           // [n][rows][keys / 64][limb][64]
    u64 *out, *parts;               // parts [splits][n][rows][dim]
    size_t rows, keys;
    int splits, run, tile_rows, key_block, dblocks;
    u32 rows_now;                   // of this slab: the last may be smaller
};

// a sequence's share of the slab: first token, tokens, and the limit of its first token there
struct seq_span {
    int first, count, limit, step;  // limit of token first + i: limit + i * step, at least 0
};

__device__ __forceinline__ seq_span span_of(const attn_args &g, int b)
{
    const int s0 = fixed_at(g.s.start, b), s1 = fixed_at(g.s.start, b + 1);
    const int first = max(s0, g.tok0), last = min(s1, g.tok1);
    int len = min(fixed_at(g.s.length, b), g.s.max_length);
    len = max(0, (int)min((long long)len, (long long)g.s.max_pages * g.c.page_cells * 16));
    return {first, max(0, last - first), g.causal ? len - (s1 - first) + 1 : len, g.causal ? 1 : 0};
}
__device__ __forceinline__ int limit_at(const seq_span &s, int i) { return max(0, s.limit + i * s.step); }

// tile number -> sequence and first row of the tile (rows of a sequence and kv head: token-major, then the heads of the group);
// every lane of the wave calls.  -1: no such tile (of a single sequence it may also be one without rows).
__device__ __forceinline__ int find_tile(const attn_args &g, int tile, int &row0)
{
    if (g.s.seqs == 1) {
        row0 = tile * g.tile_rows;
        return 0;
    }
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0; b0 < g.s.seqs; b0 += 64) {
        const int b = b0 + lane;
        int mine = 0;
        if (b < g.s.seqs) {
            const int first = max(fixed_at(g.s.start, b), g.tok0), last = min(fixed_at(g.s.start, b + 1), g.tok1);
            mine = (max(0, last - first) * g.group + g.tile_rows - 1) / g.tile_rows;
        }
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        const unsigned long long past = __ballot(base + upto > tile);
        if (past) {
            const int l = __ffsll((long long)past) - 1;
            row0 = (tile - base - __shfl(upto - mine, l)) * g.tile_rows;
            return b0 + l;
        }
        base += __shfl(upto, 63);
    }
    return -1;
}

// byte offset of a cell of the context of sequence b in head 0 of party 0 (cells past the table's end and pages outside the cache: some
// cell of the cache, whose products have weight 0)
__device__ __forceinline__ size_t cell_at(const attn_args &g, int b, int cell)
{
    const int slot = (int)fd_div((u32)cell, g.dCells), in = cell - slot * g.c.page_cells;
    const int page = fixed_at(g.s.table, (size_t)b * g.s.max_pages + min(slot, g.s.max_pages - 1));
    return (size_t)min(max(page, 0), g.c.pages - 1) * g.page_bytes + (size_t)in * g.cell;
}

template <int NLn>
__device__ __forceinline__ void clear(v4i (&acc)[NLn])
{
#pragma unroll
    for (int s = 0; s < NLn; s++) acc[s] = (v4i){0, 0, 0, 0};
}

// 64 contraction indices of MT blocks of 16 rows, whose digits lie at a in LDS, `stride` apart, times the 16 columns of k.  FIRST: the
// sums start here.
template <int MT, bool FIRST>
__device__ __forceinline__ void multiply(const v4i *a, int stride, const v4i (&k)[NL], v4i (&acc)[MT][ND])
{
#pragma unroll
    for (int i = 0; i < NL; i++)
#pragma unroll
        for (int m = 0; m < MT; m++) {
            const v4i x = a[m * stride + i * 64];
#pragma unroll
            for (int j = 0; j < NL; j++)
                acc[m][i + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, k[j], FIRST && (i == 0 || j == NL - 1) ? (v4i){0, 0, 0, 0} : acc[m][i + j], 0, 0, 0);
        }
    // two reads ahead of the products (left to itself the compiler waits for every read where registers are few)
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
    for (int q = 0; q < MT * NL; q++) {
        __builtin_amdgcn_sched_group_barrier(0x008, NL, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
}

// A party's shares of the masks of four rows for one key, below 2^62 (2^47): those of parties 1..2t are drawn (own_key), those of party 2t+1 are what
// makes them open to the mask, its own multiplier being 1.  One set of shares for the whole row would leave the differences of a party's messages
// plain products of its queries and keys.  mask, counter: of the rows; step: the key's part of the counter.  (Four rows together, so that
// a key of the generator is waited for once.  acc: at most six terms.)
__device__ __forceinline__ void mask_shares(const ss_softmax_params &sp, const u64 *mask, const u64 *counter, u64 step, bool last, u64 own_key, u64 (&v)[4])
{
    if (!last) {
#pragma unroll
        for (int r = 0; r < 4; r++) v[r] = ss_draw_lazy_at(own_key, counter[r] + step);
        return;
    }
    ss_sacc2 acc[4];
#pragma unroll
    for (int r = 0; r < 4; r++) acc[r].clear();
    for (int i = 0; i < 2 * sp.t; i++) {
        const u64 k = sp.maskgen_key[i];
        const int c = -sp.ilambda[i];
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const u64 x = ss_draw_lazy_at(k, counter[r] + step);
            SS_SPLIT31(x, w0, w1);
            acc[r].mac(w0, w1, c);
        }
    }
#pragma unroll
    for (int r = 0; r < 4; r++) v[r] = mask[r] + acc[r].lazy();
}

// Digits of the queries to LDS, qd [row / 16][dim / 64][limb][64 lanes]: item `it` is four consecutive elements of a row; 16 items take 64
// elements, so that a wave reads 512 consecutive bytes of a row.  (What lies in the places of rows that do not exist reaches their
// results alone.)
__device__ __forceinline__ void stage_query(const attn_args &g, v4i *qd, const size_t *rowat, int party, int kb_n, int it)
{
    const int rk = it >> 4, kb = kb_n > 1 ? rk % kb_n : 0, r = kb_n > 1 ? rk / kb_n : rk, d = kb * 64 + (it & 15) * 4;
    u64 y[4] = {0, 0, 0, 0};
    if (d < g.c.dim) {
        const u64 *src = g.q + (size_t)party * g.s.tokens * g.ld_q + rowat[r] + d;
#pragma unroll
        for (int c = 0; c < 4; c++) y[c] = balanced_digits(src[c]);
    }
    u32 *dst = reinterpret_cast<u32 *>(qd + (size_t)((r >> 4) * kb_n + kb) * TILE + (r & 15) + 16 * ((d & 63) >> 4)) + ((d & 15) >> 2);
#pragma unroll
    for (int l = 0; l < NL; l++) dst[l * 256] = limb_dword(y, l);
}

// Step 1: one workgroup per (tile of 16 MT rows, block of g.key_block keys, kv head and party).  The digits of the queries lie in LDS in
// MFMA order; a wave takes a cell of 16 keys at a time straight from the cache, the next 64 elements of a cell (or the next cell's first)
// on their way while those at hand are multiplied.  A cell is a wave's own (no other has a use for it) and its digits are in MFMA order as
// they lie, so they need no LDS.
// Single tokens are bound by reading the keys once: 32 heads over 8 of 128, n = 5, eight contexts of 500 to 2001, 410 MB in 86 to 92 us (4.4 to
// 4.8 TB/s); n = 3, one of 32768, 805 MB in 155 to 163 (4.9 to 5.2).  Chunks by the matrix cores and by what stands between the products: 512 tokens
// of 16 heads over 4096 keys, n = 5, 1150 to 1240 us, 2.1 to 2.3 POP/s, at the 1.8 GHz that this work leaves the card: products 57 % of the cycles, beside
// them the folds of 15 sums (MT = 2: 8 for 256 products) and the masks (one draw to a score, 2t at party 2t+1: 200 of the us).
template <int MT>
__global__ __launch_bounds__(256, 2) void scores_kernel(attn_args g, ss_softmax_params sp)
{
    extern __shared__ v4i qd[];                  // [MT][dim / 64][limb][64 lanes]
    __shared__ u64 mask[16 * MT], counter[16 * MT];   // of the row, and of its draws for key 0
    __shared__ int rowid[16 * MT], seen[16 * MT];     // keys that the row sees: none where there is no row
    __shared__ size_t rowat[16 * MT];            // of the row's query in a share of q
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = (int)fd_div(blockIdx.x, g.dScores), hp = (int)blockIdx.x - tile * g.c.kv * (2 * sp.t + 1);
    const int head = hp / (2 * sp.t + 1), party = hp - head * (2 * sp.t + 1);
    int row0 = 0;
    const int b = __builtin_amdgcn_readfirstlane(find_tile(g, tile, row0));
    if (b < 0) return;
    row0 = __builtin_amdgcn_readfirstlane(row0);
    const seq_span s = span_of(g, b);
    const int nrows = min(16 * MT, s.count * g.group - row0);
    if (nrows <= 0) return;
    const int last = (int)fd_div((u32)(row0 + nrows - 1), g.dGroup), lim = limit_at(s, last);
    const int key0 = blockIdx.y * g.key_block;
    if (key0 >= lim) return;
    const int kb_n = (g.c.dim + 63) / 64, groups = g.c.dim >> 4;
    const int cell_end = min(key0 + g.key_block, lim + 15) >> 4;
    int cell = (key0 >> 4) + wave;
    // (elements past the head's end: those of its last 16 again, the queries' digits are 0 there)
    const signed char *base = g.c.keys + party * g.party_bytes + head * g.head_bytes + (lane & 15) * 16;
    auto load = [&](size_t at, int kb, v4i (&k)[NL]) {
        const signed char *src = base + at + (size_t)min(kb * 4 + (lane >> 4), groups - 1) * 256;
#pragma unroll
        for (int l = 0; l < NL; l++) k[l] = *reinterpret_cast<const v4i *>(src + (size_t)(l * groups) * 256);
    };
    v4i k[NL], next[NL];
    size_t at = 0;
    if (cell < cell_end) {
        at = cell_at(g, b, cell);
        load(at, 0, k);
    }
    if (tid < 16 * MT) {
        seen[tid] = 0;
        if (tid < nrows) {
            const int i = (int)fd_div((u32)(row0 + tid), g.dGroup), h = head * g.group + row0 + tid - i * g.group;
            rowid[tid] = (s.first + i - g.tok0) * g.heads + h;
            seen[tid] = limit_at(s, i);
            rowat[tid] = (size_t)(s.first + i) * g.ld_q + (size_t)h * g.c.dim;
            const u64 row = (u64)(s.first + i) * g.heads + h;
            mask[tid] = ss_draw_field(sp.mask_key, row);
            counter[tid] = ss_counter(row << 32);
        }
    }
    __syncthreads();
    for (int it = tid; it < nrows * kb_n * 16; it += 256) stage_query(g, qd, rowat, party, kb_n, it);
    __syncthreads();
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): the first digits are there, the loop's waits are for its own loads alone
    const bool last_party = party == 2 * sp.t;
    const u64 own_key = sp.maskgen_key[last_party ? 0 : party];
    for (; cell < cell_end; cell += 4) {
        const size_t at_next = cell_at(g, b, min(cell + 4, cell_end - 1));
        v4i acc[MT][ND];
        for (int kb = 0; kb < kb_n; kb++) {
            // (always: a load that may not have been sent would be waited for at once.  Behind the last cell, its own first elements again)
            const bool same = kb + 1 < kb_n;
            load(same ? at : at_next, same ? kb + 1 : 0, next);
            __builtin_amdgcn_sched_barrier(0);   // the loads leave before the products
            const v4i *a = qd + kb * TILE + lane;
            if (kb == 0)
                multiply<MT, true>(a, kb_n * TILE, k, acc);
            else
                multiply<MT, false>(a, kb_n * TILE, k, acc);
#pragma unroll
            for (int l = 0; l < NL; l++) k[l] = next[l];
        }
        at = at_next;
#pragma unroll
        for (int m = 0; m < MT; m++) {
            const int row = m * 16 + 4 * (lane >> 4), key = cell * 16 + (lane & 15);
            u64 share[4];
            mask_shares(sp, mask + row, counter + row, (u64)key * SS_GAMMA, last_party, own_key, share);
#pragma unroll
            for (int r = 0; r < 4; r++)
                if (key < seen[row + r]) g.msg[((size_t)party * g.rows + rowid[row + r]) * g.keys + key] = fold_diagonals(acc[m], r, share[r]);
        }
    }
}

__device__ __forceinline__ long long lift(u64 v) { return v <= (SS_P - 1) / 2 ? (long long)v : (long long)v - (long long)SS_P; }

// floor(2^30 2^-x) for the distance `below` >= 0 of a score (2 f fraction bits) from the row's maximum, x in octaves with 16 fraction
// bits: 2^-x for x in [0, 1) by a polynomial of degree 5 that takes the value 1 at 0 and is off by 2.2e-7 at most, Horner's scheme
// in 30 fraction bits, each product cut to them
__device__ __forceinline__ u32 softmax_weight(long long below, const ss_softmax_params &sp)
{
    const int h = min(2 * sp.f, 24);
    const u64 d = min((u64)below >> (2 * sp.f - h), (u64)1 << 37), u = (d * sp.scale) >> (h + 8);
    const u32 r = (u32)u << 16;                  // the fraction, 32 bits
    u32 w = 1077640u;
    w = 10033292u - __umulhi(w, r);
    w = 59494488u - __umulhi(w, r);
    w = 257928559u - __umulhi(w, r);
    w = 744260865u - __umulhi(w, r);
    w = 1073741824u - __umulhi(w, r);
    const u64 octaves = u >> 16;
    return octaves < 31 ? w >> octaves : 0;
}

template <int THREADS = BLOCK, typename T, typename F>
__device__ __forceinline__ T block_reduce(T v, T *lds, F &&op)   // lds: one for each wave
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = op(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; w++) v = op(v, lds[w]);
    return v;
}

__device__ __forceinline__ int sequence_of(const attn_args &g, int token)
{
    int lo = 0, hi = g.s.seqs;       // the last b with start[b] <= token
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (fixed_at(g.s.start, mid) <= token) lo = mid; else hi = mid;
    }
    return lo;
}

// where a row stands: its place in the slab, its token and head, the keys it sees, and those that the products read of its tile
struct row_place {
    int id, token, head, limit, covered;
};

__device__ __forceinline__ bool row_at(const attn_args &g, int id, row_place &r)
{
    const int i = (int)fd_div((u32)id, g.dHeads), token = g.tok0 + i, b = sequence_of(g, token), head = id - i * g.heads;
    const seq_span s = span_of(g, b);
    if (token < s.first || token >= s.first + s.count) return false;
    const int at = token - s.first, in_group = head - (int)fd_div((u32)head, g.dGroup) * g.group;
    const int row = at * g.group + in_group, end = min((row | (g.tile_rows - 1)) + 1, s.count * g.group);
    r = {id, token, head, limit_at(s, at), (limit_at(s, (int)fd_div((u32)(end - 1), g.dGroup)) + 63) & ~63};
    return true;
}

// Step 2, what the elite party reconstructs: four scores of a row from those of the parties 1..2t+1 (keys from j on, all loads in flight
// together; places beyond the limit hold anything)
template <int T>
__device__ __forceinline__ void open_scores(const attn_args &g, const ss_softmax_params &sp, const row_place &r, int j, u64 (&v)[4])
{
    constexpr int NR = 2 * T + 1;
    const size_t plane = g.rows * g.keys;
    const u64 *msg = g.msg + (size_t)r.id * g.keys + j;
    u64 m[NR][4];
#pragma unroll
    for (int i = 0; i < NR; i++)
#pragma unroll
        for (int c = 0; c < 4; c++) m[i][c] = msg[i * plane + c];
#pragma unroll
    for (int c = 0; c < 4; c++) {
        ss_sacc2 acc;
        acc.clear();
#pragma unroll
        for (int i = 0; i < NR; i++) {
            SS_SPLIT31(m[i][c], w0, w1);
            acc.mac(w0, w1, sp.ilambda[i]);
        }
        v[c] = acc.value();
    }
}

struct row_norm {
    u64 recip;      // reciprocal of the sum of the weights
    int drop;       // bits that the sum is shifted by
};

__device__ __forceinline__ u64 wave_value(u64 v)   // that all lanes have
{
    return (u64)(u32)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (u32)__builtin_amdgcn_readfirstlane((int)v);
}

// A row belongs to a wave or a workgroup: both words are kept in scalar registers.  The shifts by `drop` need it: a 64-bit shift whose amount
// lies in the last vector register that the wave has can read v0 in its place here, which the compiler does not avoid.
__device__ __forceinline__ row_norm norm_of(u64 of)
{
    const u64 sum = wave_value(of);
    if (!sum) return {0, 0};
    const int drop = max(0, 32 - __clzll((long long)sum));
    // floor(2^62 / x), 2^30 <= x < 2^32, by way of a quotient in 53 bits that is off by one at most
    const u64 x = sum >> drop;
    u64 q = (u64)(4611686018427387904.0 / (double)x);
    const long long rest = (long long)((1ull << 62) - q * x);
    q = rest < 0 ? q - 1 : rest >= (long long)x ? q + 1 : q;
    return {wave_value(q), drop};
}

// the weight of a key, w / sum, with sp.bits fraction bits
__device__ __forceinline__ u64 weight_of(u32 w, const row_norm &nm, const ss_softmax_params &sp)
{
    return ((((u64)w * nm.recip) >> 16) + (1ull << (45 - sp.bits + nm.drop))) >> (46 - sp.bits + nm.drop);
}

// The weights of four keys (w, 30 fraction bits, 0 beyond the limit; `seen` of them are keys that the row sees), shared, as digits.  The shares
// need not be below p for that: any word of the residue has digits that the sums of the values hold.
template <int N, int T>
__device__ __forceinline__ void share_weights(const attn_args &g, const ss_softmax_params &sp, const row_place &r, int j, const u32 (&w)[4], int seen,
                                              const row_norm &nm)
{
    const int n = N ? N : sp.n;
    u64 y[MAXP<N>][4];
    const u64 counter = ss_counter(((u64)r.token * g.heads + r.head) << 32 | (u32)j);
#pragma unroll
    for (int c = 0; c < 4; c++) {
        u64 a[T];
#pragma unroll
        for (int x = 0; x < T; x++) a[x] = c < seen ? ss_draw_lazy_at(sp.gen_key[x], counter + c * SS_GAMMA) : 0;
        eval_points<T, MAXP<N>, LAZY>(weight_of(w[c], nm, sp), a, [&](int m, u64 v) { y[m][c] = balanced_digits(v); }, n);
    }
    signed char *dst = g.weights + (size_t)r.id * g.keys * NL + (size_t)(j >> 6) * (64 * NL) + (j & 63);
#pragma unroll
    for (int m = 0; m < MAXP<N>; m++)
        if (N != 0 || m < n) {
            u32 d[8];
            limb_dwords(y[m], d);
#pragma unroll
            for (int l = 0; l < NL; l++) *reinterpret_cast<u32 *>(dst + m * g.rows * g.keys * NL + l * 64) = d[l];
        }
}

// Step 2 for rows of up to 4 THREADS RUNS keys, one workgroup each: opened once, maximum, weights and sum in registers.  Many rows are
// bound by their arithmetic (210 vector instructions to a key at n = 5, a seventh of them products) and, next to it, by the messages in and the weights
// out: 8192 of 3585 to 4096 keys, n = 5, 490 us for 2.5 GB, 5.1 TB/s (past the caches 90 to 130 more: the weights are read again at once).
// 256 rows of 2001 keys 13 to 14 us, the chain from load to load of one row.
template <int N, int T, int RUNS, int THREADS>
__global__ __launch_bounds__(THREADS) void softmax_kernel(attn_args g, ss_softmax_params sp)
{
    __shared__ long long red[THREADS / 64];
    row_place r;
    if (!row_at(g, blockIdx.x, r)) return;
    const int tid = threadIdx.x;
    __shared__ u64 first;
    u64 v[RUNS][4];
    long long top = -(1ll << 62);
    u32 w[RUNS][4];
#pragma unroll
    for (int u = 0; u < RUNS; u++) {
        const int j = (u * THREADS + tid) * 4;
        if (j < r.limit) open_scores<T>(g, sp, r, j, v[u]);
    }
    if (tid == 0) first = v[0][0];
    __syncthreads();
    const u64 ref = first;                       // differences of a row are small, whatever its mask is
#pragma unroll
    for (int u = 0; u < RUNS; u++) {
        const int j = (u * THREADS + tid) * 4;
#pragma unroll
        for (int c = 0; c < 4; c++)
            if (j + c < r.limit) {
                const long long d = lift(ss_sub(v[u][c], ref));
                v[u][c] = (u64)d;
                top = max(top, d);
            }
    }
    top = block_reduce<THREADS>(top, red, [](long long x, long long y) { return max(x, y); });
    long long sum = 0;
#pragma unroll
    for (int u = 0; u < RUNS; u++) {
        const int j = (u * THREADS + tid) * 4;
#pragma unroll
        for (int c = 0; c < 4; c++) {
            w[u][c] = j + c < r.limit ? softmax_weight(top - (long long)v[u][c], sp) : 0;
            sum += w[u][c];
        }
    }
    sum = block_reduce<THREADS>(sum, red, [](long long x, long long y) { return x + y; });
    const row_norm nm = norm_of((u64)sum);
#pragma unroll
    for (int u = 0; u < RUNS; u++) {
        const int j = (u * THREADS + tid) * 4;
        if (j >= r.covered) break;
        share_weights<N, T>(g, sp, r, j, w[u], r.limit - j, nm);
    }
}

// ... for longer rows, which several workgroups take in blocks of 1024 keys (32 rows of 32768, n = 3: 10 + 7.4 + 12.5 us; in one workgroup to a row
// they would leave seven CUs of eight idle): opened, with the largest score of each block,
template <int T>
__global__ __launch_bounds__(BLOCK) void open_kernel(attn_args g, ss_softmax_params sp)
{
    __shared__ long long red[4];
    __shared__ u64 first;
    row_place r;
    const int j = (blockIdx.y * BLOCK + threadIdx.x) * 4;
    if (!row_at(g, blockIdx.x, r) || (int)blockIdx.y * 1024 >= r.limit) return;
    u64 v[4];
    if (j < r.limit) {
        open_scores<T>(g, sp, r, j, v);
        u64 *opened = g.opened + (size_t)r.id * g.keys + j;
#pragma unroll
        for (int c = 0; c < 4; c++) opened[c] = v[c];
    }
    if (threadIdx.x == 0) first = v[0];
    __syncthreads();
    long long top = -(1ll << 62);
    if (j < r.limit) {
#pragma unroll
        for (int c = 0; c < 4; c++)
            if (j + c < r.limit) top = max(top, lift(ss_sub(v[c], first)));
    }
    top = block_reduce(top, red, [](long long x, long long y) { return max(x, y); });
    if (threadIdx.x == 0) g.tops[(size_t)r.id * gridDim.y + blockIdx.y] = ss_add(first, top < 0 ? SS_P - (u64)(-top) : (u64)top);
}

// the largest score of a row
__device__ __forceinline__ u64 top_of(const attn_args &g, const row_place &r, long long *red)
{
    const u64 *tops = g.tops + (size_t)r.id * gridDim.y, ref = tops[0];
    long long top = 0;
    for (int k = threadIdx.x; k * 1024 < r.limit; k += BLOCK) top = max(top, lift(ss_sub(tops[k], ref)));
    top = block_reduce(top, red, [](long long x, long long y) { return max(x, y); });
    return ss_add(ref, (u64)top);
}

// the sum of the weights of each block,
__global__ __launch_bounds__(BLOCK) void sum_kernel(attn_args g, ss_softmax_params sp)
{
    __shared__ long long red[4];
    row_place r;
    const int j = (blockIdx.y * BLOCK + threadIdx.x) * 4;
    if (!row_at(g, blockIdx.x, r) || (int)blockIdx.y * 1024 >= r.limit) return;
    const u64 top = top_of(g, r, red);
    long long sum = 0;
#pragma unroll
    for (int c = 0; c < 4; c++)
        if (j + c < r.limit) sum += softmax_weight(lift(ss_sub(top, g.opened[(size_t)r.id * g.keys + j + c])), sp);
    sum = block_reduce(sum, red, [](long long x, long long y) { return x + y; });
    if (threadIdx.x == 0) g.sums[(size_t)r.id * gridDim.y + blockIdx.y] = (u64)sum;
}

// and the weights.
template <int N, int T>
__global__ __launch_bounds__(BLOCK) void weights_kernel(attn_args g, ss_softmax_params sp)
{
    __shared__ long long red[4];
    row_place r;
    const int j = (blockIdx.y * BLOCK + threadIdx.x) * 4;
    if (!row_at(g, blockIdx.x, r) || (int)blockIdx.y * 1024 >= r.covered) return;
    u32 w[4] = {0, 0, 0, 0};
    row_norm nm = {0, 0};
    if (r.limit) {
        const u64 top = top_of(g, r, red);
        long long sum = 0;
        for (int k = threadIdx.x; k * 1024 < r.limit; k += BLOCK) sum += (long long)g.sums[(size_t)r.id * gridDim.y + k];
        nm = norm_of((u64)block_reduce(sum, red, [](long long x, long long y) { return x + y; }));
#pragma unroll
        for (int c = 0; c < 4; c++)
            if (j + c < r.limit) w[c] = softmax_weight(lift(ss_sub(top, g.opened[(size_t)r.id * g.keys + j + c])), sp);
    }
    if (j < r.covered) share_weights<N, T>(g, sp, r, j, w, r.limit - j, nm);
}

// Step 3: one workgroup per (tile of 16 MT rows, run of keys and up to 64 elements of the head, kv head and party); a wave takes 16
// elements.  The digits of 64 weights of every row go through LDS to all waves, those of the values to a wave's registers; the next
// 64 keys are on their way while those at hand are multiplied.  (The weights too by way of registers: behind copies straight into LDS the
// compiler waits before the next read of any LDS.)  Long rows of few tokens are cut into runs, which join_kernel adds up.
// Single tokens are bound by reading the values once: the sizes at scores_kernel 84 to 88 and 144 to 150 us, 4.7 to 5.6 TB/s.  Chunks by the
// matrix cores: 915 to 1000 us there, 2.6 to 2.8 POP/s, products 79 % of the cycles.  A workgroup of eight waves that takes 128 elements
// saves half of the weights' reads but leaves one workgroup to a CU: 1020 against 935 us; waves by the head's size (5 for 80 elements) 64
// against 54.
template <int MT>
__global__ __launch_bounds__(256, 2) void values_kernel(attn_args g, int n)
{
    __shared__ v4i wd[2][MT * TILE];
    __shared__ size_t cells[MAX_RUN / 16 + 4];
    __shared__ int rowid[16 * MT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = (int)fd_div(blockIdx.x, g.dValues), hp = (int)blockIdx.x - tile * g.c.kv * n;
    const int head = hp / n, party = hp - head * n;
    const int split = blockIdx.y / g.dblocks, dt = (blockIdx.y - split * g.dblocks) * 4 + wave;   // 16 elements each
    int row0 = 0;
    const int b = __builtin_amdgcn_readfirstlane(find_tile(g, tile, row0));
    if (b < 0) return;
    row0 = __builtin_amdgcn_readfirstlane(row0);
    const seq_span s = span_of(g, b);
    const int nrows = min(16 * MT, s.count * g.group - row0);
    if (nrows <= 0) return;
    const int lim = limit_at(s, (int)fd_div((u32)(row0 + nrows - 1), g.dGroup));
    const int k0 = split * g.run, k1 = min(k0 + g.run, lim), units = (k1 - k0 + 63) >> 6;
    if (split && k0 >= lim) return;              // (the first run writes the zeros of rows that see nothing)
    for (int c = tid; c < units * 4; c += 256) cells[c] = cell_at(g, b, k0 / 16 + c);
    if (tid < 16 * MT) {
        const int r = min(tid, nrows - 1), i = (int)fd_div((u32)(row0 + r), g.dGroup);
        rowid[tid] = (s.first + i - g.tok0) * g.heads + head * g.group + row0 + r - i * g.group;
    }
    __syncthreads();
    const bool live = dt * 16 < g.c.dim;         // (others only bring weights)
    const size_t limb = (size_t)g.c.dim * 16;
    const signed char *base = g.c.values + party * g.party_bytes + head * g.head_bytes + (min(dt, (g.c.dim >> 4) - 1) * 16 + (lane & 15)) * 16;
    const signed char *wrow[MT];
    v4i acc[MT][ND];
#pragma unroll
    for (int m = 0; m < MT; m++) {
        clear(acc[m]);
        wrow[m] = g.weights + ((size_t)party * g.rows + rowid[m * 16 + (lane & 15)]) * g.keys * NL + (lane >> 4) * 16 + (size_t)k0 * NL;
    }
    // limb slices of the weights that this wave brings to LDS: numbers wave, wave + 4, ... of MT NL
    constexpr int SLICES = MT * NL, MOST = (SLICES + 3) / 4;
    v4i slice[MOST];
    auto load_weights = [&](int unit) {
#pragma unroll
        for (int k = 0; k < MOST; k++) {
            const int q = min(wave + 4 * k, SLICES - 1);   // (twice the last where they do not come out even)
            slice[k] = *reinterpret_cast<const v4i *>((MT == 1 || q < NL ? wrow[0] : wrow[MT - 1]) + (size_t)unit * (64 * NL) + (q < NL ? q : q - NL) * 64);
        }
    };
    auto keep_weights = [&](int stage) {
#pragma unroll
        for (int k = 0; k < MOST; k++) wd[stage][min(wave + 4 * k, SLICES - 1) * 64 + lane] = slice[k];
    };
    auto load_values = [&](int unit, v4i (&v)[NL]) {
        const signed char *src = base + cells[unit * 4 + (lane >> 4)];
#pragma unroll
        for (int l = 0; l < NL; l++) v[l] = *reinterpret_cast<const v4i *>(src + l * limb);
    };
    v4i v[NL], next[NL];
    if (units) {
        load_weights(0);
        load_values(0, v);
        keep_weights(0);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): the loop's waits are for its own loads alone
    for (int u = 0; u < units; u++) {
        __syncthreads();                         // everyone's weights are in LDS, and nobody reads the other stage any more
        const int ahead = min(u + 1, units - 1); // (the last again behind the last: nobody reads it)
        load_values(ahead, next);
        load_weights(ahead);
        __builtin_amdgcn_sched_barrier(0);       // the loads leave before the products
        if (live) multiply<MT, false>(&wd[u & 1][lane], TILE, v, acc);
        __builtin_amdgcn_sched_barrier(0);
        keep_weights((u + 1) & 1);
#pragma unroll
        for (int l = 0; l < NL; l++) v[l] = next[l];
    }
    if (!live) return;
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int row = m * 16 + 4 * (lane >> 4) + r;
            if (row >= nrows) continue;
            const size_t id = rowid[row], d = dt * 16 + (lane & 15);
            const u64 o = fold_diagonals(acc[m], r);
            if (g.splits == 1)
                g.out[((size_t)party * g.s.tokens * g.heads + (size_t)g.tok0 * g.heads + id) * g.c.dim + d] = o;
            else
                g.parts[(((size_t)split * n + party) * g.rows + id) * g.c.dim + d] = o;
        }
}

// Steps 2 and 3 in one launch for contexts of up to 256 keys: one workgroup of eight waves per (tile of 16 rows, kv head and party) takes the
// softmax of the rows, a wave to a row and four keys to a lane, keeps its own party's shares of the weights in LDS and multiplies, a
// wave to 16 elements of the head.  All parties' workgroups take the same softmax, which costs less than a launch.  Bound by its chain of
// loads: 4 heads of 64 over 33 keys, n = 3, 6.0 to 6.9 us beside 5.4 to 5.9 of the scores (three launches: 19 for all).
template <int T>
__global__ __launch_bounds__(512) void finish_kernel(attn_args g, ss_softmax_params sp)
{
    constexpr int WAVES = 8;
    __shared__ v4i wd[SHORT_KEYS / 64 * TILE];   // [key / 64][limb][64 lanes]
    __shared__ int rowid[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int head = blockIdx.y / sp.n, party = blockIdx.y - head * sp.n;
    int row0 = 0;
    const int b = __builtin_amdgcn_readfirstlane(find_tile(g, blockIdx.x, row0));
    if (b < 0) return;
    row0 = __builtin_amdgcn_readfirstlane(row0);
    const seq_span s = span_of(g, b);
    const int nrows = min(16, s.count * g.group - row0);
    if (nrows <= 0) return;
    const int lim = limit_at(s, (int)fd_div((u32)(row0 + nrows - 1), g.dGroup)), blocks = (lim + 63) >> 6, groups = g.c.dim >> 4;
    const signed char *values = g.c.values + party * g.party_bytes + head * g.head_bytes + (lane & 15) * 16;
    const size_t limb = (size_t)g.c.dim * 16;
    auto load = [&](int dt, int blk, v4i (&v)[NL]) {
        const signed char *src = values + cell_at(g, b, blk * 4 + (lane >> 4)) + dt * 256;
#pragma unroll
        for (int l = 0; l < NL; l++) v[l] = *reinterpret_cast<const v4i *>(src + l * limb);
    };
    v4i v[NL], next[NL];
    if (blocks && wave < groups) load(wave, 0, v);
    for (int row = wave; row < nrows; row += WAVES) {
        const int i = (int)fd_div((u32)(row0 + row), g.dGroup), h = head * g.group + row0 + row - i * g.group, j = lane * 4;
        const row_place r = {(s.first + i - g.tok0) * g.heads + h, s.first + i, h, limit_at(s, i), blocks * 64};
        if (lane == 0) rowid[row] = r.id;
        u64 o[4] = {0, 0, 0, 0}, y[4];
        u32 w[4];
        if (j < r.limit) open_scores<T>(g, sp, r, j, o);
        const u64 ref = __shfl(o[0], 0);
        long long top = -(1ll << 62), sum = 0;
#pragma unroll
        for (int c = 0; c < 4; c++)
            if (j + c < r.limit) top = max(top, lift(ss_sub(o[c], ref)));
#pragma unroll
        for (int d = 32; d; d >>= 1) top = max(top, __shfl_xor(top, d));
#pragma unroll
        for (int c = 0; c < 4; c++) {
            w[c] = j + c < r.limit ? softmax_weight(top - lift(ss_sub(o[c], ref)), sp) : 0;
            sum += w[c];
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        const row_norm nm = norm_of((u64)sum);
#pragma unroll
        for (int c = 0; c < 4; c++) {
            const u64 counter = ss_counter(((u64)r.token * g.heads + h) << 32 | (u32)(j + c));
            u64 a[T];
#pragma unroll
            for (int x = 0; x < T; x++) a[x] = ss_draw_field_at(sp.gen_key[x], counter);
            const u64 share = ss_poly_eval<T>(weight_of(w[c], nm, sp), a, T, party + 1);
            y[c] = j + c < r.limit ? balanced_digits(share) : 0;
        }
        if (j < r.covered) {
            u32 *dst = reinterpret_cast<u32 *>(wd + (j >> 6) * TILE + row + (j & 48)) + ((j & 15) >> 2);
#pragma unroll
            for (int l = 0; l < NL; l++) dst[l * 256] = limb_dword(y, l);
        }
    }
    __syncthreads();
    for (int dt = wave; dt < groups; dt += WAVES) {
        v4i acc[1][ND];
        clear(acc[0]);
        for (int blk = 0; blk < blocks; blk++) {
            // (behind the last, its own again)
            const bool same = blk + 1 < blocks, more = dt + WAVES < groups;
            load(same || !more ? dt : dt + WAVES, same ? blk + 1 : 0, next);
            multiply<1, false>(wd + blk * TILE + lane, 0, v, acc);
#pragma unroll
            for (int l = 0; l < NL; l++) v[l] = next[l];
        }
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int row = 4 * (lane >> 4) + r;
            if (row < nrows)
                g.out[((size_t)party * g.s.tokens * g.heads + (size_t)g.tok0 * g.heads + rowid[row]) * g.c.dim + dt * 16 + (lane & 15)] =
                    fold_diagonals(acc[0], r);
        }
    }
}

// The runs of a row added up, WAYS waves to a result, each every WAYS-th run.  (us, one wave / four: 43 runs of 4096 results of three parties
// 10.4 / 5.8; 3 runs of 117760 of three 5.0 / 7.9.)
template <int WAYS>
__global__ __launch_bounds__(BLOCK) void join_kernel(attn_args g, int n, fdiv dDim)
{
    constexpr int RESULTS = BLOCK / WAYS, FLIGHT = 8 / WAYS < 4 ? 4 : 8 / WAYS;   // loads in flight
    __shared__ u64 sums[WAYS][RESULTS];
    const int at = threadIdx.x & (RESULTS - 1), way = threadIdx.x / RESULTS;
    const u32 i = blockIdx.x * RESULTS + at, id = fd_div(i, dDim), party = blockIdx.y;
    row_place r;
    const bool live = id < g.rows_now && row_at(g, (int)id, r);
    const int runs = live ? (r.limit + g.run - 1) / g.run : 0;
    const size_t plane = (size_t)n * g.rows * g.c.dim;
    const u64 *p = g.parts + (size_t)party * g.rows * g.c.dim + i;
    u64 o = 0;
    for (int s0 = way; s0 < runs; s0 += FLIGHT * WAYS) {
        u64 x[FLIGHT];
#pragma unroll
        for (int s = 0; s < FLIGHT; s++) x[s] = p[min(s0 + WAYS * s, runs - 1) * plane];
#pragma unroll
        for (int s = 0; s < FLIGHT; s++) o = s0 + WAYS * s < runs ? ss_add(o, x[s]) : o;
    }
    if constexpr (WAYS > 1) {
        sums[way][at] = o;
        __syncthreads();
        if (way) return;
#pragma unroll
        for (int w = 1; w < WAYS; w++) o = ss_add(o, sums[w][at]);
    }
    if (live) g.out[((size_t)party * g.s.tokens + g.tok0) * g.heads * g.c.dim + i] = o;
}

rotary_shape make_shape(int tokens, int heads, int dim, int pairs, int width)
{
    return {tokens, heads, dim, width, pairs, make_fdiv((u32)width), make_fdiv((u32)heads)};
}

size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

hipError_t ss_launch_rotary(const u64 *x, size_t ld, u64 *u, u64 *wsh, u64 *out, int tokens, int heads, int dim, const ss_rope &rope,
                            const ss_tr_params &tp, hipStream_t stream)
{
    const int half = rope.rot / 2;
    const bool wide = wide_rotary(dim, rope.rot, rope.interleaved, ld, aligned16(x) && aligned16(out));
    const int pairs = !wide ? half : rope.interleaved ? half : half / 2, width = wide ? pairs + (dim - rope.rot) / 2 : dim - half;
    const rotary_shape g = make_shape(tokens, heads, dim, pairs, width);
    const dim3 grid(ceil_div((size_t)tokens * heads * width, BLOCK));
    const bool streams = rotary_streams(tp.n, tp.t, tokens, heads, dim, rope.rot);
#define SS_WIDE(NC, TC, I)                                                                                                       \
    hipLaunchKernelGGL((streams ? rotary_wide_kernel<NC, TC, I, true> : rotary_wide_kernel<NC, TC, I, false>), grid, dim3(BLOCK), 0, \
                       stream, x, ld, u, wsh, out, g, rope, tp)
#define SS_LAUNCH(NC, TC)                                                                                              \
    do {                                                                                                               \
        if (!wide)                                                                                                     \
            hipLaunchKernelGGL((rotary_kernel<NC, TC>), grid, dim3(BLOCK), 0, stream, x, ld, u, wsh, out, g, rope, tp); \
        else if (rope.interleaved)                                                                                     \
            SS_WIDE(NC, TC, true);                                                                                     \
        else                                                                                                           \
            SS_WIDE(NC, TC, false);                                                                                    \
    } while (0)
    SS_SCHEME(tp.n, tp.t, SS_LAUNCH);
#undef SS_LAUNCH
#undef SS_WIDE
    return hipGetLastError();
}

hipError_t ss_launch_append(const ss_paged &c, const u64 *k, size_t ld_k, const u64 *v, size_t ld_v, int tokens, const long long *slots,
                            u64 *u, u64 *wsh, const ss_rope &rope, const ss_tr_params &tp, hipStream_t stream)
{
    const int half = rope.rot / 2;
    append_shape s = {};
    s.r = make_shape(tokens, c.kv, c.dim, half, c.dim - half);
    s.slots = slots;
    s.keys = c.keys;
    s.values = c.values;
    s.head = (size_t)c.page_cells * (SS_NLIMB * 16) * c.dim;
    s.party = s.head * c.kv;
    s.page = s.party * tp.n;
    s.page_size = (unsigned)c.page_cells * 16;
    s.capacity = s.page_size * (unsigned)c.pages;
    s.dPage = make_fdiv(s.page_size);
    if (wide_append(tokens, c.kv, c.dim, rope.rot, ld_k, aligned16(k))) {
        s.steps = (rope.interleaved ? half : half / 2) + (c.dim - rope.rot) / 2;
        s.step_blocks = (int)ceil_div(s.steps, 16);
        s.value_blocks = (int)ceil_div((size_t)tp.n * c.dim, BLOCK);
        const unsigned groups = ceil_div((size_t)tokens + 15, 16);
        const int keys = (int)groups * s.step_blocks;
        const dim3 grid(keys + groups * s.value_blocks, c.kv);
#define SS_LAUNCH(NC, TC)                                                                                                  \
    hipLaunchKernelGGL((rope.interleaved ? append_many_kernel<NC, TC, true> : append_many_kernel<NC, TC, false>), grid, dim3(BLOCK), 0, \
                       stream, k, ld_k, v, ld_v, u, wsh, s, rope, tp, keys, make_fdiv((u32)c.dim))
        SS_SCHEME(tp.n, tp.t, SS_LAUNCH);
#undef SS_LAUNCH
        return hipGetLastError();
    }
    const unsigned key_blocks = ceil_div((size_t)tokens * c.kv * s.r.width, BLOCK);
    const dim3 grid(key_blocks + ceil_div((size_t)tokens * c.kv * c.dim, BLOCK));
#define SS_LAUNCH(NC, TC) \
    hipLaunchKernelGGL((append_kernel<NC, TC>), grid, dim3(BLOCK), 0, stream, k, ld_k, v, ld_v, u, wsh, s, rope, tp, key_blocks)
    SS_SCHEME(tp.n, tp.t, SS_LAUNCH);
#undef SS_LAUNCH
    return hipGetLastError();
}

hipError_t ss_launch_attention(const attention_plan &plan, const ss_paged &cache, const ss_sequences &seqs, const u64 *q, size_t ld_q, int heads,
                               int causal, const ss_softmax_params &sp, void *room, u64 *out, hipStream_t stream)
{
    attn_args g = {};
    g.c = cache;
    g.s = seqs;
    g.cell = (size_t)NL * 16 * cache.dim;
    g.head_bytes = g.cell * cache.page_cells;
    g.party_bytes = g.head_bytes * cache.kv;
    g.page_bytes = g.party_bytes * sp.n;
    g.heads = heads;
    g.group = heads / cache.kv;
    g.causal = causal;
    g.dGroup = make_fdiv((u32)g.group);
    g.dCells = make_fdiv((u32)cache.page_cells);
    g.dHeads = make_fdiv((u32)heads);
    g.dScores = make_fdiv((u32)cache.kv * (2 * sp.t + 1));
    g.dValues = make_fdiv((u32)cache.kv * sp.n);
    g.q = q;
    g.ld_q = ld_q;
    g.rows = plan.rows;
    g.keys = plan.keys;
    g.splits = plan.splits;
    g.run = plan.run;
    g.tile_rows = 16 * plan.row_tiles;
    g.key_block = plan.key_block;
    g.dblocks = plan.dblocks;
    const int nr = 2 * sp.t + 1, n = sp.n;
    const unsigned blocks = ceil_div(plan.keys, 1024);
    char *at = (char *)room;
    g.msg = (u64 *)at;
    at += align256((size_t)nr * g.rows * g.keys * 8);
    if (plan.split_rows) {
        g.opened = (u64 *)at;
        g.tops = g.opened + g.rows * g.keys;
        g.sums = g.tops + g.rows * blocks;
        at += align256(g.rows * (g.keys + 2 * blocks) * 8);
    }
    g.weights = (signed char *)at;
    at += plan.finish ? 0 : align256((size_t)n * g.rows * g.keys * NL);
    g.parts = (u64 *)at;
    g.out = out;
    const size_t lds = plan.query_bytes;
    if (lds > 48 * 1024) {
        const void *scores = plan.row_tiles == 1 ? (const void *)scores_kernel<1> : (const void *)scores_kernel<2>;
        if (hipError_t e = hipFuncSetAttribute(scores, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds); e != hipSuccess) return e;
    }
    for (int tok = 0; tok < seqs.tokens; tok += plan.slab) {
        g.tok0 = tok;
        g.tok1 = min(seqs.tokens, tok + plan.slab);
        g.rows_now = (u32)(g.tok1 - tok) * heads;
        // heads and parties run fastest over the workgroups, which are dealt to the XCDs in turn: every head and party has the same work,
        // whatever the lengths of the sequences, and the tiles of one read the same keys and values
        const unsigned tiles = (unsigned)tile_bound(g.tok1 - tok, seqs.seqs, g.group, g.tile_rows);
        const dim3 sgrid(tiles * cache.kv * nr, ceil_div(plan.keys, plan.key_block)), vgrid(tiles * cache.kv * n, plan.splits * plan.dblocks);
        const dim3 rgrid(g.rows_now), wgrid(g.rows_now, blocks), block(BLOCK);
        if (plan.row_tiles == 1)
            hipLaunchKernelGGL((scores_kernel<1>), sgrid, dim3(256), lds, stream, g, sp);
        else
            hipLaunchKernelGGL((scores_kernel<2>), sgrid, dim3(256), lds, stream, g, sp);
        if (plan.finish) {
            const dim3 fgrid(tiles, cache.kv * n);
            if (sp.t == 1)
                hipLaunchKernelGGL(finish_kernel<1>, fgrid, dim3(512), 0, stream, g, sp);
            else if (sp.t == 2)
                hipLaunchKernelGGL(finish_kernel<2>, fgrid, dim3(512), 0, stream, g, sp);
            else
                hipLaunchKernelGGL(finish_kernel<3>, fgrid, dim3(512), 0, stream, g, sp);
            if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            continue;
        }
        // rows of 1024 to 4096 keys: four runs of 256 threads where they fill the card, 1024 threads otherwise (the whole attention, us, four runs /
        // 1024 threads: n = 3, 2048 rows of 2000 keys 209 / 220, 8192 of 1100 408 / 454, of 4096 1576 / 1574; n = 5, 992 rows of 4096 399 / 401, 512 228.8 / 227.5,
        // 32 of 1100 37.1 / 36.3, of 4096 90.0 / 88.6)
#define SS_LAUNCH(NC, TC)                                                                               \
    do {                                                                                                \
        if (plan.split_rows) {                                                                          \
            hipLaunchKernelGGL((open_kernel<TC>), wgrid, block, 0, stream, g, sp);                      \
            hipLaunchKernelGGL(sum_kernel, wgrid, block, 0, stream, g, sp);                             \
            hipLaunchKernelGGL((weights_kernel<NC, TC>), wgrid, block, 0, stream, g, sp);               \
        } else if (blocks == 1)                                                                         \
            hipLaunchKernelGGL((softmax_kernel<NC, TC, 1, 256>), rgrid, block, 0, stream, g, sp);       \
        else if (g.rows_now < 1024)                                                                     \
            hipLaunchKernelGGL((softmax_kernel<NC, TC, 1, 1024>), rgrid, dim3(1024), 0, stream, g, sp); \
        else                                                                                            \
            hipLaunchKernelGGL((softmax_kernel<NC, TC, 4, 256>), rgrid, block, 0, stream, g, sp);       \
    } while (0)
        SS_SCHEME(sp.n, sp.t, SS_LAUNCH);
#undef SS_LAUNCH
        if (plan.row_tiles == 1)
            hipLaunchKernelGGL((values_kernel<1>), vgrid, dim3(256), 0, stream, g, n);
        else
            hipLaunchKernelGGL((values_kernel<2>), vgrid, dim3(256), 0, stream, g, n);
        const size_t results = (size_t)g.rows_now * cache.dim;
        if (plan.splits > 8)
            hipLaunchKernelGGL(join_kernel<4>, dim3(ceil_div(results, BLOCK / 4), n), block, 0, stream, g, n, make_fdiv((u32)cache.dim));
        else if (plan.splits > 1)
            hipLaunchKernelGGL(join_kernel<1>, dim3(ceil_div(results, BLOCK), n), block, 0, stream, g, n, make_fdiv((u32)cache.dim));
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace SS_NS
