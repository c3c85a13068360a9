// What a classifier's logits are read for beyond the mean loss: the log-probability of a given label with the entropy and
// the likeliest classes (hpf_logprobs_*), and the loss against a teacher's largest logits (hpf_distill_*), with gradients.
//
// Mathematics.  With s = logits / T, M = max s and S = sum exp(s - M):  lse = M + ln S, log p_c = s_c - lse,
// entropy H = ln S - (sum exp(s - M) (s - M)) / S.  A thread runs over its share of a row once and keeps (M, S, the weighted
// sum); a larger maximum scales what is there.  Shares are joined within a warp, a CTA and, for few rows, a cluster of CTAs
// over distributed shared memory, always in the same order: results do not depend on timing.  All sums are fp32 over at most
// a few hundred terms per thread, exponents in base 2 (ex2.approx, 2^-22).
//
// Layout.  Rows of at most 1024 classes: a warp per row, the row in registers.  Longer rows: a CTA per row of 16-byte
// loads, four in flight per thread; a row that starts off a 16-byte boundary has its first and last few classes read one by one.
// Fewer rows than SMs: the row is cut into up to 8 parts, one per CTA of a cluster.
#pragma once
#include "../../include/hpf.h"
#include "hpf_kernels.h"
#include "pairs.cuh"

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <initializer_list>
#include <math.h>

namespace cg = cooperative_groups;

namespace hpf {
namespace {

constexpr int kWarpRow = 1024;     // classes up to which a warp holds a row
constexpr int kMaxParts = 8;       // CTAs a row is cut into (portable cluster size)
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFloor = -1e30f;   // stands for less where a class at it weighs nothing (see LogprobsGrad::far)
constexpr float kGone = -200.f;    // 2 to this is 0 in fp32

__device__ __forceinline__ float ninf() { return __int_as_float(0xff800000); }
// The first step of every kernel: where it is launched as a programmatic dependent (see launch_rows), it waits here for its predecessor's results.
__device__ __forceinline__ void enter()
{
    pdl_launch_dependents();
    pdl_wait();
}

// ---- element types ---------------------------------------------------------------------------------------------------
template <typename T> struct Io;
template <> struct Io<float> {
    static constexpr int V = 4;
    static constexpr uint32_t kMinusInf = 0xff800000u;
    static constexpr float kLowest = -3.4028235e38f, kBound = kFloor;      // the type's lowest value; what bounded() leaves at least
    static __device__ __forceinline__ void unpack(const uint4& r, float* f)
    {
        f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* f)
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
    // of two pieces, value by value (a NaN loses); the largest value of a piece; -inf replaced by the type's lowest value; nothing below
    // -10^30 (the lowest value of fp16 is above that).  A NaN stays.
    static __device__ __forceinline__ uint4 larger(const uint4& a, const uint4& b)
    {
        return make_uint4(one(a.x, b.x), one(a.y, b.y), one(a.z, b.z), one(a.w, b.w));
    }
    static __device__ __forceinline__ uint32_t one(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
    static __device__ __forceinline__ float largest(const uint4& a) { return fmaxf(fmaxf(__uint_as_float(a.x), __uint_as_float(a.y)), fmaxf(__uint_as_float(a.z), __uint_as_float(a.w))); }
    static __device__ __forceinline__ uint4 finite(const uint4& a)
    {
        return make_uint4(low(a.x), low(a.y), low(a.z), low(a.w));
    }
    static __device__ __forceinline__ uint32_t low(uint32_t v) { return v == 0xff800000u ? 0xff7fffffu : v; }
    static __device__ __forceinline__ uint4 bounded(const uint4& a) { return make_uint4(above(a.x), above(a.y), above(a.z), above(a.w)); }
    static __device__ __forceinline__ uint32_t above(uint32_t v) { return __uint_as_float(v) < kFloor ? __float_as_uint(kFloor) : v; }
};
template <typename T, typename T2, uint32_t LOWEST, uint32_t FLOOR>
struct Packed16 {
    static __device__ __forceinline__ uint32_t one(uint32_t a, uint32_t b)
    {
        const T2 m = __hmax2(*reinterpret_cast<const T2*>(&a), *reinterpret_cast<const T2*>(&b));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ uint4 larger(const uint4& a, const uint4& b) { return make_uint4(one(a.x, b.x), one(a.y, b.y), one(a.z, b.z), one(a.w, b.w)); }
    template <uint32_t BOUND>
    static __device__ __forceinline__ uint32_t above(uint32_t a)
    {
        const uint32_t bound = BOUND;
        const T2 m = __hmax2_nan(*reinterpret_cast<const T2*>(&a), *reinterpret_cast<const T2*>(&bound));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ uint4 finite(const uint4& a) { return make_uint4(above<LOWEST>(a.x), above<LOWEST>(a.y), above<LOWEST>(a.z), above<LOWEST>(a.w)); }
    static __device__ __forceinline__ uint4 bounded(const uint4& a) { return make_uint4(above<FLOOR>(a.x), above<FLOOR>(a.y), above<FLOOR>(a.z), above<FLOOR>(a.w)); }
};
template <> struct Io<__nv_bfloat16> : Packed16<__nv_bfloat16, __nv_bfloat162, 0xff7fff7fu, 0xf14af14au> {
    static constexpr int V = 8;
    static constexpr uint32_t kMinusInf = 0xff80ff80u;
    static constexpr float kLowest = -3.3895314e38f, kBound = kFloor;
    static __device__ __forceinline__ void two(uint32_t w, float* f)
    {
        f[0] = __uint_as_float(w << 16);
        f[1] = __uint_as_float(w & 0xffff0000u);
    }
    static __device__ __forceinline__ void unpack(const uint4& r, float* f) { two(r.x, f); two(r.y, f + 2); two(r.z, f + 4); two(r.w, f + 6); }
    static __device__ __forceinline__ uint32_t join(float a, float b)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) { return make_uint4(join(f[0], f[1]), join(f[2], f[3]), join(f[4], f[5]), join(f[6], f[7])); }
    static __device__ __forceinline__ float largest(const uint4& a)
    {
        float f[2];
        two(one(one(a.x, a.y), one(a.z, a.w)), f);
        return fmaxf(f[0], f[1]);
    }
    static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Io<__half> : Packed16<__half, __half2, 0xfbfffbffu, 0xfbfffbffu> {
    static constexpr int V = 8;
    static constexpr uint32_t kMinusInf = 0xfc00fc00u;
    static constexpr float kLowest = -65504.f, kBound = -65504.f;
    static __device__ __forceinline__ void two(uint32_t w, float* f)
    {
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
        f[0] = v.x; f[1] = v.y;
    }
    static __device__ __forceinline__ void unpack(const uint4& r, float* f) { two(r.x, f); two(r.y, f + 2); two(r.z, f + 4); two(r.w, f + 6); }
    static __device__ __forceinline__ uint32_t join(float a, float b)
    {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) { return make_uint4(join(f[0], f[1]), join(f[2], f[3]), join(f[4], f[5]), join(f[6], f[7])); }
    static __device__ __forceinline__ float largest(const uint4& a)
    {
        float f[2];
        two(one(one(a.x, a.y), one(a.z, a.w)), f);
        return fmaxf(f[0], f[1]);
    }
    static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};

// The share of one row that a CTA runs over: whole 16-byte pieces [c0, c1), the first of them `lead` classes into the row,
// and the classes before the first boundary and behind the last one, which the row's first and last part take.
template <typename T>
struct Share {
    const T* row;
    int n, lead, c0, c1, tail;
    bool first, last;
    __device__ __forceinline__ Share(const T* r, int classes, int part, int parts) : row(r), n(classes)
    {
        constexpr int V = Io<T>::V;
        lead = (int)(((16 - (reinterpret_cast<uintptr_t>(r) & 15)) & 15) / sizeof(T));
        if (lead > n) lead = n;
        const int chunks = (n - lead) / V;
        tail = lead + chunks * V;
        c0 = (int)((long long)chunks * part / parts);
        c1 = (int)((long long)chunks * (part + 1) / parts);
        first = part == 0;
        last = part == parts - 1;
    }
    __device__ __forceinline__ const uint4* pieces() const { return reinterpret_cast<const uint4*>(row + lead); }
    __device__ __forceinline__ uint4 load(int c) const { return *(reinterpret_cast<const uint4*>(row + lead) + c); }
    // the last reading of a piece: it goes first when L2 needs room
    __device__ __forceinline__ uint4 load_last(int c) const { return __ldcs(reinterpret_cast<const uint4*>(row + lead) + c); }
    // the class that this thread reads by itself, or -1: V - 1 at most at either end of the row
    __device__ __forceinline__ int edge(int tid) const
    {
        if (tid < 8) return first && tid < lead ? tid : -1;
        if (tid < 16) return last && tail + tid - 8 < n ? tail + tid - 8 : -1;
        return -1;
    }
    __device__ __forceinline__ bool mine(int c) const     // does class c belong to this share?
    {
        if (c < 0 || c >= n) return false;
        if (c < lead) return first;
        if (c >= tail) return last;
        const int k = (c - lead) / Io<T>::V;
        return k >= c0 && k < c1;
    }
};

// ---- running sums ----------------------------------------------------------------------------------------------------
// m: largest logit, s = sum 2^((v - m) c), w = sum 2^((v - m) c) (v - m), h = the sum of s at temperature 1
struct Sums {
    float m, s, w, h;
};
template <bool ENTROPY, bool HARD>
__device__ __forceinline__ void rescale(Sums& a, float m, float c)
{
    if (a.m == m) return;
    const float u = a.m - m, r = ex2(u * c);                      // -inf where a.m is: what weighs nothing is left out, not multiplied
    if (ENTROPY) a.w = r == 0.f ? 0.f : r * fmaf(u, a.s, a.w);
    a.s *= r;
    if (HARD) a.h *= ex2(u * kLog2e);
    a.m = m;
}
// The maximum is subtracted before anything is scaled: a row of the type's lowest value stays finite, and large logits lose nothing.
template <bool ENTROPY, bool HARD>
__device__ __forceinline__ void add_value(Sums& a, float v, float c, float base)
{
    const float u = v - base;
    const float e = ex2(u * c);
    a.s += e;
    if (ENTROPY) a.w = e == 0.f ? a.w : fmaf(e, u, a.w);          // u may be -inf; a NaN passes
    if (HARD) a.h += ex2(u * kLog2e);
}
__device__ __forceinline__ float base_of(float m) { return m == ninf() ? 0.f : m; }

// Where a thread leaves the largest logit of each stretch of its strip (for the list of the largest classes).
struct Stretches {
    float* at;           // [count][threads]
    int count, iters;    // stretches, and the rounds of the loop below that one takes
};

// How the sum at temperature 1 is formed: from an exponential of its own, or, where the temperature is a small whole number, as a power of
// the one at hand.  A second exponential a class makes the loop as long as the special-function unit takes for it (4096 x 128000
// bf16: 279 us instead of 190).
constexpr int kNoHard = -1, kOwnExp = 0;

// One thread's share of the row.  ENTROPY: -inf is replaced by the type's lowest value (0 (-inf) would be NaN in the weighted sum) as long as
// that is so far below the largest logit that it weighs 0 too; else (a strip of nothing but such masks, or a temperature of hundreds
// in fp16), or where v - m could overflow, each class is looked at by itself.
// between(): what else has to come from memory, asked for while the first pieces are under way.
template <typename T, int NT, bool ENTROPY, int POWER, typename F>
__device__ __forceinline__ Sums run_over(const Share<T>& sh, float c, int tid, const Stretches* st, F&& between)
{
    constexpr int V = Io<T>::V, U = 4;
    constexpr bool HARD = POWER != kNoHard;
    const uint4 none = make_uint4(Io<T>::kMinusInf, Io<T>::kMinusInf, Io<T>::kMinusInf, Io<T>::kMinusInf);
    Sums a{ninf(), 0.f, 0.f, 0.f};
    f2 s2 = 0, w2 = 0, h2 = 0;
    const f2 c2 = pair(c, c), one2 = pair(kLog2e, kLog2e);
    f2 base2 = 0;                                             // -m, twice
    const auto near = [&](float m) { return ENTROPY && !((Io<T>::kLowest - m) * c < kGone && m < 1e30f); };
    bool careful = near(0.f);
    int slot = 0, left = st ? st->iters : 0;
    float stretch = ninf();
    // one round: U pieces, of which the first `there` hold classes
    const auto round = [&](const uint4 (&raw)[U], int there) {
        const float top = Io<T>::largest(Io<T>::larger(Io<T>::larger(raw[0], raw[1]), Io<T>::larger(raw[2], raw[3])));
        if (st) {
            stretch = fmaxf(stretch, top);
            if (--left == 0) {
                st->at[slot * NT + tid] = stretch;
                ++slot;
                left = st->iters;
                stretch = ninf();
            }
        }
        if (top > a.m) {
            const float u = a.m - top, r = ex2(u * c);            // as in rescale
            const f2 r2 = pair(r, r);
            if (ENTROPY) w2 = r == 0.f ? 0 : mul2(r2, fma2(pair(u, u), s2, w2));
            s2 = mul2(r2, s2);
            if (POWER == kOwnExp || POWER > 1) {
                const float q = ex2(u * kLog2e);
                h2 = mul2(pair(q, q), h2);
            }
            a.m = top;
            base2 = pair(-top, -top);
            careful = near(top);
        }
        if (ENTROPY && careful) {
            Sums b{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < there) {
                    float f[V];
                    Io<T>::unpack(raw[u], f);
#pragma unroll
                    for (int j = 0; j < V; ++j) add_value<true, false>(b, f[j], c, base_of(a.m));
                }
            s2 = add2(s2, pair(b.s, 0.f));
            w2 = add2(w2, pair(b.w, 0.f));
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < there) {
                float f[V];
                Io<T>::unpack(ENTROPY ? Io<T>::finite(raw[u]) : raw[u], f);
#pragma unroll
                for (int j = 0; j < V; j += 2) {
                    const f2 d = add2(pair(f[j], f[j + 1]), base2);
                    const f2 e = ex2_2(mul2(d, c2));
                    s2 = add2(s2, e);
                    if (ENTROPY) w2 = fma2(e, d, w2);
                    if (POWER == kOwnExp) h2 = add2(h2, ex2_2(mul2(d, one2)));
                    if (POWER == 2) h2 = fma2(e, e, h2);
                    if (POWER == 3) h2 = fma2(mul2(e, e), e, h2);
                    if (POWER == 4) { const f2 q = mul2(e, e); h2 = fma2(q, q, h2); }
                }
            }
    };
    // whole rounds without a question, the next one's pieces under way; then what is left
    const int full = (sh.c1 - sh.c0) / (U * NT), rest = sh.c0 + full * U * NT + tid;
    int there = 0;
    const uint4* at = sh.pieces() + sh.c0 + tid;
    uint4 raw[U], next[U];
    const auto load_rest = [&](uint4 (&to)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = rest + u * NT < sh.c1;
            to[u] = in ? sh.load(rest + u * NT) : none;
            there += in;
        }
    };
    if (full > 0) {
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = at[u * NT];
    } else {
        load_rest(raw);
    }
    between();
#pragma unroll 2
    for (int r = 0; r < full; ++r) {
        at += U * NT;
        if (r + 1 < full) {
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = at[u * NT];
        } else {
            load_rest(next);
        }
        round(raw, U);
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = next[u];
    }
    if (there) round(raw, there);
    if (st)
        for (; slot < st->count; ++slot) {
            st->at[slot * NT + tid] = stretch;
            stretch = ninf();
        }
    float x, y;
    split(s2, &x, &y); a.s = x + y;
    split(w2, &x, &y); a.w = x + y;
    split(h2, &x, &y); a.h = POWER == 1 ? a.s : x + y;
    const int e = sh.edge(tid);
    if (e >= 0) {
        const float v = Io<T>::get(sh.row[e]);
        if (v > a.m) rescale<ENTROPY, HARD>(a, v, c);
        add_value<ENTROPY, HARD>(a, v, c, base_of(a.m));
    }
    return a;
}
template <typename T, int NT, bool HARD, typename F>
__device__ __forceinline__ Sums run_over_power(const Share<T>& sh, float c, int tid, int power, F&& between)
{
    if constexpr (!HARD) return run_over<T, NT, false, kNoHard>(sh, c, tid, nullptr, between);
    if (power == 1) return run_over<T, NT, false, 1>(sh, c, tid, nullptr, between);
    if (power == 2) return run_over<T, NT, false, 2>(sh, c, tid, nullptr, between);
    if (power == 3) return run_over<T, NT, false, 3>(sh, c, tid, nullptr, between);
    if (power == 4) return run_over<T, NT, false, 4>(sh, c, tid, nullptr, between);
    return run_over<T, NT, false, kOwnExp>(sh, c, tid, nullptr, between);
}

template <bool ENTROPY, bool HARD>
__device__ __forceinline__ Sums warp_sums(Sums a, float c)
{
    float m = a.m;
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    rescale<ENTROPY, HARD>(a, m, c);
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
        if (ENTROPY) a.w += __shfl_xor_sync(0xffffffffu, a.w, d);
        if (HARD) a.h += __shfl_xor_sync(0xffffffffu, a.h, d);
    }
    return a;
}
// of `count` <= 32 partial results, one per lane
template <bool ENTROPY, bool HARD>
__device__ __forceinline__ Sums join_sums(const Sums* part, int count, int lane, float c)
{
    Sums a = lane < count ? part[lane] : Sums{ninf(), 0.f, 0.f, 0.f};
    return warp_sums<ENTROPY, HARD>(a, c);
}
// the same value for every thread of the CTA
template <int NT, bool ENTROPY, bool HARD>
__device__ __forceinline__ Sums block_sums(Sums a, float c, Sums* s_part)
{
    a = warp_sums<ENTROPY, HARD>(a, c);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = a;
    __syncthreads();
    return join_sums<ENTROPY, HARD>(s_part, NT / 32, threadIdx.x & 31, c);
}
// Another CTA's shared memory may be written once that CTA runs: every thread says so early (cluster_here) and waits for the others before the
// first write (cluster_all_here), by when they long have.
__device__ __forceinline__ void cluster_here() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_all_here() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// The same value for every CTA of a row: each puts its sums into the shared memory of all (into, not out of: nobody has to stay for others
// to read).  s_parts: one place per part.  After cluster_here().
template <bool HARD>
__device__ __forceinline__ Sums cluster_sums(Sums a, float c, int part, int parts, Sums* s_parts)
{
    cg::cluster_group cl = cg::this_cluster();
    cluster_all_here();
    if ((int)threadIdx.x < parts) *cl.map_shared_rank(&s_parts[part], threadIdx.x) = a;
    cl.sync();
    return join_sums<false, HARD>(s_parts, parts, threadIdx.x & 31, c);
}

constexpr float kLseExact = 128.f;   // an lse below this is off by 128 2^-24 = 7.6e-6 at most

// ---- gradients -------------------------------------------------------------------------------------------------------
// Writes g(two logits) for every two classes of the share.  `out` may be the logits themselves: a thread writes what it has read.
// BOUNDED: nothing below Io<T>::kBound comes.  AGAIN: the row has been gone over just now; it is read from its end to its start, what is in L2
// since last first (4096 x 128000 bf16: 487 -> 452 us).
template <typename T, int NT, bool BOUNDED, bool AGAIN, typename F>
__device__ __forceinline__ void write_row(const Share<T>& sh, T* out, int tid, F&& g)
{
    constexpr int V = Io<T>::V, U = 4;
    const bool wide = ((reinterpret_cast<uintptr_t>(out + sh.lead)) & 15) == 0;
    const int full = (sh.c1 - sh.c0) / (U * NT), rest = sh.c0 + full * U * NT + tid;
    const auto put = [&](int c, const uint4& raw) {
        float f[V];
        Io<T>::unpack(BOUNDED ? Io<T>::bounded(raw) : raw, f);
#pragma unroll
        for (int j = 0; j < V; j += 2) split(g(pair(f[j], f[j + 1])), &f[j], &f[j + 1]);
        T* to = out + sh.lead + c * V;
        if (wide) __stcs(reinterpret_cast<uint4*>(to), Io<T>::pack(f));
        else
#pragma unroll
            for (int j = 0; j < V; ++j) to[j] = Io<T>::put(f[j]);
    };
    const auto put_rest = [&]() {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (rest + u * NT < sh.c1) raw[u] = AGAIN ? sh.load_last(rest + u * NT) : sh.load(rest + u * NT);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (rest + u * NT < sh.c1) put(rest + u * NT, raw[u]);
    };
    if (AGAIN) put_rest();
    if constexpr (AGAIN) {
        uint4 raw[U], next[U];
        int i = sh.c0 + (full - 1) * U * NT + tid;
        if (full > 0) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = sh.load_last(i + u * NT);
        }
#pragma unroll 2
        for (int k = full; k > 0; --k, i -= U * NT) {
            if (k > 1) {
#pragma unroll
                for (int u = 0; u < U; ++u) next[u] = sh.load_last(i + (u - U) * NT);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) put(i + u * NT, raw[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = next[u];
        }
    } else {
        for (int k = 0; k < full; ++k) {
            const int i = sh.c0 + k * U * NT + tid;
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = sh.load(i + u * NT);
#pragma unroll
            for (int u = 0; u < U; ++u) put(i + u * NT, raw[u]);
        }
    }
    if (!AGAIN) put_rest();
    const int e = sh.edge(tid);
    if (e >= 0) {
        const float v = Io<T>::get(sh.row[e]);
        float a, b;
        split(g(pair(BOUNDED && v < Io<T>::kBound ? Io<T>::kBound : v, 0.f)), &a, &b);
        out[e] = Io<T>::put(a);
    }
}

// ---- launches --------------------------------------------------------------------------------------------------------
int sm_count()
{
    static PerDevice<int> sms;
    int n = 0;
    if (sms.get(&n, [](int dev, int* v) { return cudaDeviceGetAttribute(v, cudaDevAttrMultiProcessorCount, dev); }) != cudaSuccess) return 148;
    return n;
}
// Parts of a row: while the CTAs (of 512 threads) still fit the SMs one each and every part keeps 8 KB.
int parts_of(int64_t rows, int n, size_t elem)
{
    int parts = 1;
    while (parts < kMaxParts && rows * parts * 2 <= sm_count() && (size_t)n * elem / (2 * parts) >= 8192) parts *= 2;
    return parts;
}
// As a programmatic dependent a kernel is scheduled while its predecessor in the stream drains.  That saves 0.5 us of a small call and 2 of a large
// one, but CTAs that fill up what a predecessor of one wave leaves free share the SMs unevenly (777 x 32003 fp16, loss and gradient: 23 -> 28 us):
// it is done below 2 MB of logits and from three waves on.
template <typename K, typename A>
cudaError_t launch_rows(K* kernel, int64_t rows, int parts, int threads, cudaStream_t st, const A& args, size_t bytes)
{
    const bool dependent = bytes < (2u << 20) || rows * parts * threads >= (int64_t)3 * 1024 * sm_count();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * parts));
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (dependent) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (parts > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)parts;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, args);
}
// Rows per SM from which CTAs of 128 threads take them: eight rows at different steps hide each other's waits better than four (4096 x 50021
// bf16 with 8 listed classes: 94 -> 82 us; 100 rows: 8.7 -> 11 us).
constexpr int kManyRows = 4;

template <typename K, typename A>
cudaError_t launch_warps(K* kernel, int64_t rows, cudaStream_t st, const A& args, size_t bytes)
{
    return launch_rows(kernel, (rows + 3) / 4, 1, 128, st, args, bytes);
}

// ---- checks ----------------------------------------------------------------------------------------------------------
int element(int32_t dtype) { return dtype == HPF_FP32 ? 4 : 2; }
bool on(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
int check_rows(const void* logits, int64_t rows, int32_t classes, int64_t ld, int32_t dtype)
{
    if (dtype != HPF_FP32 && dtype != HPF_BF16 && dtype != HPF_FP16) return api_fail(HPF_ERR_INVALID, "dtype must be HPF_FP32, HPF_BF16 or HPF_FP16");
    if (rows < 0 || classes < 1 || ld < classes) return api_fail(HPF_ERR_INVALID, "rows < 0, classes < 1 or a row stride below the class count");
    if (rows > 0x7fffffff / kMaxParts || classes > (1 << 30)) return api_fail(HPF_ERR_UNSUPPORTED, "more than 2^28 rows or 2^30 classes");
    if (rows && (!logits || !on(logits, element(dtype)))) return api_fail(HPF_ERR_INVALID, "logits: null or not aligned to their type");
    return HPF_OK;
}
// Labels, lists and statistics are int32 and fp32 (null where a call has none).
int check_words(std::initializer_list<const void*> all)
{
    for (const void* p : all)
        if (!on(p, 4)) return api_fail(HPF_ERR_INVALID, "labels, lists or statistics not aligned to their type");
    return HPF_OK;
}
// A gradient may take the logits' own place, row by row: then its rows are theirs.
int check_gradient(const void* logits, const void* out, int64_t rows, int64_t ld, int64_t ld_d, int32_t dtype)
{
    if (!out || !on(out, element(dtype))) return api_fail(HPF_ERR_INVALID, "gradient: null or not aligned to its type");
    if (out == logits && rows > 1 && ld_d != ld) return api_fail(HPF_ERR_INVALID, "a gradient in the logits' place needs their row stride");
    return HPF_OK;
}

}  // namespace
}  // namespace hpf
