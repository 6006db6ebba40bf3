// Masked truncation (Sec. VI-B) of the element a thread owns, shared by the kernels that truncate: the mask, what the elite party
// does with the opened value, and the sharing and unmasking of the quotient.
#pragma once
#include "kernels.hpp"
#include "eval.hpp"

namespace SS_NS {

template <int VEC>
struct pack_t;
template <>
struct pack_t<1> {
    u64 v[1];
    __device__ __forceinline__ void load(const u64 *p) { v[0] = *p; }
    __device__ __forceinline__ void load_streaming(const u64 *p) { v[0] = __builtin_nontemporal_load(p); }
    __device__ __forceinline__ void store(u64 *p) const { *p = v[0]; }
    __device__ __forceinline__ void store_streaming(u64 *p) const { __builtin_nontemporal_store(v[0], p); }
    template <bool STREAM>
    __device__ __forceinline__ void send(u64 *p) const { STREAM ? store_streaming(p) : store(p); }
};
template <>
struct pack_t<2> {
    u64 v[2];
    __device__ __forceinline__ void load(const u64 *p)
    {
        const ulonglong2 q = *reinterpret_cast<const ulonglong2 *>(p);
        v[0] = q.x;
        v[1] = q.y;
    }
    __device__ __forceinline__ void load_streaming(const u64 *p)
    {
        typedef unsigned long long v2u __attribute__((ext_vector_type(2)));
        const v2u q = __builtin_nontemporal_load(reinterpret_cast<const v2u *>(p));
        v[0] = q.x;
        v[1] = q.y;
    }
    __device__ __forceinline__ void store(u64 *p) const
    {
        ulonglong2 q;
        q.x = v[0];
        q.y = v[1];
        *reinterpret_cast<ulonglong2 *>(p) = q;
    }
    // for output that nothing in the same launch reads again
    __device__ __forceinline__ void store_streaming(u64 *p) const
    {
        typedef unsigned long long v2u __attribute__((ext_vector_type(2)));
        v2u q = {v[0], v[1]};
        __builtin_nontemporal_store(q, reinterpret_cast<v2u *>(p));
    }
    template <bool STREAM>
    __device__ __forceinline__ void send(u64 *p) const { STREAM ? store_streaming(p) : store(p); }
};

// A message that nothing in the launch reads again.  STREAM: past the caches, see streams_messages.
template <bool STREAM>
__device__ __forceinline__ void send(u64 *p, u64 v)
{
    if constexpr (STREAM)
        __builtin_nontemporal_store(v, p);
    else
        *p = v;
}

// e of the truncation mask alpha = e * 2^f: uniform in [1, 2^(32-f)]
__device__ __forceinline__ u64 mask_e(u64 key, u64 e, int f)
{
    return 1 + ((ss_draw(key, e) >> 3) & ((1ULL << (32 - f)) - 1));
}

// the same before a division by kh*kw: the sample space of e shrinks to [1, floor(2^(32-f) / kdiv)], which keeps
// alpha = e * 2^f * kdiv within (0, 2^32] (Sec. VII-B); range = 2^(32-f) gives mask_e
__device__ __forceinline__ u64 mask_e_below(u64 key, u64 e, unsigned range)
{
    return 1 + (ss_draw(key, e) >> 3) % range;
}

// what the elite party does with the reconstructed x + alpha: floor division of the signed value by 2^f
__device__ __forceinline__ u64 shift_signed(u64 v, int f)
{
    const int64_t sv = (v <= (SS_P - 1) / 2) ? (int64_t)v : (int64_t)v - (int64_t)SS_P;
    const int64_t qv = sv >> f;
    return qv >= 0 ? (u64)qv : SS_P - (u64)(-qv);
}

// The same followed by the rounding division that average pooling moves into the truncation (Sec. VI-C):
// [q / kdiv] = floor((q + floor(kdiv/2)) / kdiv) on the signed quotient q, so that a remainder of
// ceil(kdiv/2) or more goes up (the worst case of App. C) and [(q + e*kdiv) / kdiv] = [q / kdiv] + e.
__device__ __forceinline__ u64 shift_round_div(u64 v, int f, int kdiv)
{
    const int64_t sv = (v <= (SS_P - 1) / 2) ? (int64_t)v : (int64_t)v - (int64_t)SS_P;
    const int64_t a = (sv >> f) + kdiv / 2;
    const u64 d = (u64)kdiv;
    return a >= 0 ? (u64)a / d : SS_P - ((u64)(-a) + d - 1) / d;
}

// sum of v * c over at most 8 terms, v canonical given as v = w0 + w1 2^31 (w0 < 2^31), |c| < 2^26
struct ss_sacc2 {
    long long lo, hi;
    __device__ __forceinline__ void clear() { lo = 0; hi = 0; }
    __device__ __forceinline__ void mac(u32 w0, u32 w1, int c)
    {
        lo += (long long)(int)w0 * c;   // |sum| < 8 * 2^31 * 2^26 = 2^60
        hi += (long long)(int)w1 * c;
    }
    // the sum, below 2^61 + 2^3 (2^45 + 2^25)
    __device__ __forceinline__ u64 lazy() const
    {
#if defined(SS_FIELD_P45)
        // here |hi| < 2^43 (w1 < 2^14).  Offsets that are multiples of p make both words positive;
        // h 2^31 with h = a 2^14 + b: a 2^45 + b 2^31 = 55 a + b 2^31
        const u64 l = (u64)(lo + (long long)(SS_P << 16)), h = (u64)(hi + (long long)SS_P);   // < 2^62, < 2^46
        return ss_fold(l + SS_PC * (h >> 14) + ((h & 0x3FFFull) << 31));
#else
        const u64 l = (u64)(lo + (long long)SS_P), h = (u64)(hi + (long long)SS_P);   // in (2^60, 2^62)
        // h 2^31 with 2^61 = 1: low 30 bits of h shifted, the rest wraps to weight 1
        return ss_fold(l + ((h & 0x3FFFFFFFull) << 31) + (h >> 30));
#endif
    }
    __device__ __forceinline__ u64 value() const { return ss_canon(lazy()); }
};
#define SS_SPLIT31(v, w0, w1) const u32 w0 = (u32)(v)&0x7FFFFFFFu, w1 = (u32)((v) >> 31)


template <int N>
constexpr int MAXP = N ? N : SS_MAXN;

template <int T>
__device__ __forceinline__ u64 mask_of(const ss_tr_params &tp, size_t e, u64 &alpha)
{
    const u64 ev = tp.kdiv > 1 ? mask_e_below(tp.e_key, e, tp.e_range) : mask_e(tp.e_key, e, tp.f);
    alpha = tp.kdiv > 1 ? (ev * (u64)tp.kdiv) << tp.f : ev << tp.f;   // <= 2^32
    return ev;
}

// truncation steps 2 and 3 from the opened x + alpha (canonical): the new shares in o[], their secret in `secret`; the
// messages of step 2 go to wsh unless it is nullptr
template <int N, int T, bool STREAM>
__device__ __forceinline__ void shift_and_unmask(u64 opened, u64 ev, u64 counter, size_t em, size_t mcount,
                                                 u64 *__restrict__ wsh, const ss_tr_params &tp, int n, u64 (&o)[MAXP<N>],
                                                 u64 &secret)
{
    const u64 w = tp.kdiv > 1 ? shift_round_div(opened, tp.f, tp.kdiv) : shift_signed(opened, tp.f);
    u64 cw[T], co[T];
#pragma unroll
    for (int j = 0; j < T; j++) {
        cw[j] = ss_draw_lazy_at(tp.gen_key[j], counter);
        co[j] = ss_fold(cw[j] + ss_draw_lazy_at(tp.alphat_key[j], counter));
    }
    if (wsh) eval_points<T, MAXP<N>>(w, cw, [&](int m, u64 v) { send<STREAM>(wsh + (size_t)m * mcount + em, v); }, n);
    secret = ss_canon(w + SS_P - ev);
    eval_points<T, MAXP<N>>(secret, co, [&](int m, u64 v) { o[m] = v; }, n);
}

}  // namespace SS_NS

// (3,1) and (5,2), and the two counts of t = 3, have their party count fixed at compile time; the other counts of t = 1 and
// 2 take theirs at run time.  SS_SCHEME(n, t, LAUNCH) runs LAUNCH(N, T).
#define SS_SCHEME(n_, t_, LAUNCH)               \
    do {                                        \
        if ((n_) == 5 && (t_) == 2) LAUNCH(5, 2); \
        else if ((n_) == 3 && (t_) == 1) LAUNCH(3, 1); \
        else if ((t_) == 1) LAUNCH(0, 1);       \
        else if ((t_) == 2) LAUNCH(0, 2);       \
        else if ((n_) == 7) LAUNCH(7, 3);       \
        else LAUNCH(8, 3);                      \
    } while (0)
