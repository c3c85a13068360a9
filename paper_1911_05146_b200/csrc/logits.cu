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
#include "../../include/hpf.h"
#include "hpf_kernels.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <math.h>

namespace cg = cooperative_groups;

namespace hpf {
namespace {

constexpr int kMaxTop = 64;        // classes logprobs_fwd lists per row
constexpr int kMaxTeacher = 256;   // entries of a teacher's list per row
constexpr int kWarpRow = 1024;     // classes up to which a warp holds a row
constexpr int kMaxParts = 8;       // CTAs a row is cut into (portable cluster size)
constexpr int kGroups = 128;       // groups of threads whose maxima bound the k-th largest class
constexpr int kCandidates = 512;   // classes at or above that bound that are ranked by counting
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFloor = -1e30f;   // stands for -inf where it meets a weight of 0

__device__ __forceinline__ float ninf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- element types ---------------------------------------------------------------------------------------------------
template <typename T> struct Io;
template <> struct Io<float> {
    static constexpr int V = 4;
    static constexpr uint32_t kMinusInf = 0xff800000u;
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
// Two values in one instruction: the loops below are bound by what an SM issues, not by its arithmetic.
typedef unsigned long long f2;
__device__ __forceinline__ f2 pair(float a, float b) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void split(f2 v, float* a, float* b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f2 ex2_2(f2 v)
{
    float a, b;
    split(v, &a, &b);
    return pair(ex2(a), ex2(b));
}

// m: largest logit, s = sum 2^((v - m) c), w = sum 2^((v - m) c) (v - m), h = the sum of s at temperature 1
struct Sums {
    float m, s, w, h;
};
template <bool ENTROPY, bool HARD>
__device__ __forceinline__ void rescale(Sums& a, float m, float c)
{
    if (a.m == m) return;
    const float u = fmaxf(a.m - m, kFloor), r = ex2(u * c);       // a.m may be -inf: everything it weighs is 0
    if (ENTROPY) a.w = r * fmaf(u, a.s, a.w);
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
    if (ENTROPY) a.w = fmaf(e, fmaxf(u, kFloor), a.w);
    if (HARD) a.h += ex2(u * kLog2e);
}
__device__ __forceinline__ float base_of(float m) { return m == ninf() ? 0.f : m; }

// The upper half of a logit's place among the floats: in their order, equal where the upper 16 bits are.
__device__ __forceinline__ uint32_t order16(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    return (b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) >> 16;
}
// Where a thread leaves the largest logit of each stretch of its strip (for the list of the largest classes).
struct Stretches {
    float* at;           // [count][threads]
    int count, iters;    // stretches, and the rounds of the loop below that one takes
};

// How the sum at temperature 1 is formed: from an exponential of its own, or, where the temperature is a small whole number, as a power of
// the one at hand.  A second exponential a class makes the loop as long as the special-function unit takes for it (4096 x 128000
// bf16: 279 us instead of 190).
constexpr int kNoHard = -1, kOwnExp = 0;

// One thread's share of the row.  ENTROPY: -inf is replaced by the type's lowest value ahead of the weighted sum (0 (-inf) would be NaN);
// v - m overflows only where m > 10^30, where every class but the largest weighs nothing: see write_stats.
template <typename T, int NT, bool ENTROPY, int POWER>
__device__ __forceinline__ Sums run_over(const Share<T>& sh, float c, int tid, const Stretches* st)
{
    constexpr int V = Io<T>::V, U = 4;
    constexpr bool HARD = POWER != kNoHard;
    const uint4 none = make_uint4(Io<T>::kMinusInf, Io<T>::kMinusInf, Io<T>::kMinusInf, Io<T>::kMinusInf);
    Sums a{ninf(), 0.f, 0.f, 0.f};
    f2 s2 = 0, w2 = 0, h2 = 0;
    const f2 c2 = pair(c, c), one2 = pair(kLog2e, kLog2e);
    f2 base2 = 0;                                             // -m, twice
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
            const float u = fmaxf(a.m - top, kFloor), r = ex2(u * c);
            const f2 r2 = pair(r, r);
            if (ENTROPY) w2 = mul2(r2, fma2(pair(u, u), s2, w2));
            s2 = mul2(r2, s2);
            if (POWER == kOwnExp || POWER > 1) {
                const float q = ex2(u * kLog2e);
                h2 = mul2(pair(q, q), h2);
            }
            a.m = top;
            base2 = pair(-top, -top);
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
template <typename T, int NT, bool HARD>
__device__ __forceinline__ Sums run_over_power(const Share<T>& sh, float c, int tid, int power)
{
    if constexpr (!HARD) return run_over<T, NT, false, kNoHard>(sh, c, tid, nullptr);
    if (power == 1) return run_over<T, NT, false, 1>(sh, c, tid, nullptr);
    if (power == 2) return run_over<T, NT, false, 2>(sh, c, tid, nullptr);
    if (power == 3) return run_over<T, NT, false, 3>(sh, c, tid, nullptr);
    if (power == 4) return run_over<T, NT, false, 4>(sh, c, tid, nullptr);
    return run_over<T, NT, false, kOwnExp>(sh, c, tid, nullptr);
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
// The same value for every CTA of a row: each puts its sums into the shared memory of all (into, not out of: nobody has to stay for others
// to read).  s_parts: one place per part.
template <bool HARD>
__device__ __forceinline__ Sums cluster_sums(Sums a, float c, int part, int parts, Sums* s_parts)
{
    cg::cluster_group cl = cg::this_cluster();
    if ((int)threadIdx.x < parts) *cl.map_shared_rank(&s_parts[part], threadIdx.x) = a;
    cl.sync();
    return join_sums<false, HARD>(s_parts, parts, threadIdx.x & 31, c);
}

// ---- the k largest classes -------------------------------------------------------------------------------------------
// Unique keys in the order of the list: the value's order (both zeros alike), then the lower class first.  0 = not a class
// that can be listed (masked, or not a number).
__device__ __forceinline__ unsigned long long class_key(float v, int cls)
{
    if (!(v > ninf())) return 0ull;
    const uint32_t b = __float_as_uint(v + 0.0f);
    const uint32_t o = b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
    return ((unsigned long long)o << 32) | (uint32_t)(0x7fffffff - cls);
}
__device__ __forceinline__ float key_value(unsigned long long key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int key_class(unsigned long long key) { return 0x7fffffff - (int)(uint32_t)(key & 0xffffffffu); }

template <int NT>
struct TopShared {
    static constexpr int kStretches = (NT == 512 ? 8 : 16) * NT;
    float maxima[NT];
    float stretch[kStretches];
    unsigned long long cand[kCandidates];
    int rank[kCandidates];
    unsigned short list[kStretches];
    int count, listed;
    float bound;
};

// Calls f(value, class) for every class at or above the bound in the listed stretches, which are spread over the CTA piece by piece, and in
// the row's ends.
template <typename T, int NT, typename F>
__device__ __forceinline__ void over_stretches(const Share<T>& sh, const TopShared<NT>& sm, int listed, float bound, int iters, F&& f)
{
    constexpr int V = Io<T>::V, U = 4;
    const unsigned per = (unsigned)(iters * U);                    // pieces of a stretch
    for (unsigned w = threadIdx.x; w < (unsigned)listed * per; w += NT) {
        const unsigned at = iters == 1 ? w / U : w / per, piece = w - at * per, entry = sm.list[at];
        const int c = sh.c0 + (int)(entry % NT) + (int)((entry / NT) * per + piece) * NT;
        if (c < sh.c1) {
            float v[V];
            Io<T>::unpack(sh.load(c), v);
            uint32_t which = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) which |= (v[j] >= bound && v[j] > ninf() ? 1u : 0u) << j;
            for (; which; which &= which - 1) {
                const int j = __ffs(which) - 1;
                float x = v[0];
#pragma unroll
                for (int i = 1; i < V; ++i) x = i == j ? v[i] : x;
                f(x, sh.lead + c * V + j);
            }
        }
    }
    const int e = sh.edge(threadIdx.x);
    if (e >= 0) {
        const float x = Io<T>::get(sh.row[e]);
        if (x >= bound && x > ninf()) f(x, e);
    }
}

// One warp: the k-th largest of the maxima of 32 groups of threads (a lane's group: threads lane, lane + 32, ...), by a bitonic sort.
constexpr int kFewTop = 16;
template <int NT>
__device__ __forceinline__ float kth_of_32(const float* maxima, int k, int lane)
{
    float v = ninf();
#pragma unroll
    for (int t = 0; t < NT; t += 32) v = fmaxf(v, maxima[t + lane]);
#pragma unroll
    for (int size = 2; size <= 32; size *= 2)
#pragma unroll
        for (int d = size / 2; d; d /= 2) {
            const float o = __shfl_xor_sync(0xffffffffu, v, d);
            const bool larger = ((lane & d) == 0) == ((lane & size) == 0);       // largest first, over all 32 in the end
            v = larger ? fmaxf(v, o) : fminf(v, o);
        }
    return __shfl_sync(0xffffffffu, v, k - 1);
}
// The same of 128 groups (threads t, t + 128, ...), to the upper 16 bits: four keys a lane, the bound found bit by bit.
template <int NT>
__device__ __forceinline__ float kth_of_128(const float* maxima, int k, int lane)
{
    uint32_t key[kGroups / 32];
#pragma unroll
    for (int i = 0; i < kGroups / 32; ++i) {
        float v = ninf();
#pragma unroll
        for (int t = 0; t < NT; t += kGroups) v = fmaxf(v, maxima[t + i * 32 + lane]);
        key[i] = order16(v);
    }
    // the bits that all keys share are the bound's too
    const uint32_t most = __reduce_max_sync(0xffffffffu, max(max(key[0], key[1]), max(key[2], key[3])));
    const uint32_t least = __reduce_min_sync(0xffffffffu, min(min(key[0], key[1]), min(key[2], key[3])));
    uint32_t bit = most == least ? 0u : 0x80000000u >> __clz(most ^ least), bound = bit ? most & ~(2 * bit - 1) : most;
    for (; bit; bit >>= 1) {
        int count = 0;
#pragma unroll
        for (int i = 0; i < kGroups / 32; ++i) count += __popc(__ballot_sync(0xffffffffu, key[i] >= (bound | bit)));
        if (count >= k) bound |= bit;
    }
    const uint32_t o = bound << 16;
    return bound ? __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)) : ninf();
}

// The k largest classes of this CTA's share are among the sm.cand[0 .. the result); sm.rank has their places.  Every thread knows the largest logit of each stretch of its strip
// (sm.stretch) and of all of it (my_max).  The k-th largest of G group maxima is a lower bound of the k-th largest class, so only stretches
// whose maximum reaches it are read again (from L2): about G ln(G / (G - k)) classes pass for unordered rows.  G is 32 up to k = 16, 128
// above; a group's threads lie apart, so that a row sorted by frequency does not put its head into one group.  Where too many pass
// (long runs of equal logits), a bisection over the unique keys raises the bound until they fit.
template <typename T, int NT>
__device__ __forceinline__ int select_top(const Share<T>& sh, float my_max, int k, int iters, TopShared<NT>& sm)
{
    const int tid = threadIdx.x;
    sm.maxima[tid] = my_max;
    if (tid == 0) { sm.count = 0; sm.listed = 0; }
    for (int i = tid; i < kCandidates; i += NT) sm.rank[i] = 0;
    __syncthreads();
    if (tid < 32) {
        const float bound = k <= kFewTop ? kth_of_32<NT>(sm.maxima, k, tid) : kth_of_128<NT>(sm.maxima, k, tid);
        if (tid == 0) sm.bound = bound;
    }
    __syncthreads();
    const float bound = sm.bound;
    if (my_max >= bound && my_max > ninf()) {
#pragma unroll
        for (int s = 0; s < TopShared<NT>::kStretches / NT; ++s) {
            const float v = sm.stretch[s * NT + tid];
            if (v >= bound && v > ninf()) sm.list[atomicAdd(&sm.listed, 1)] = (unsigned short)(s * NT + tid);
        }
    }
    __syncthreads();
    const int listed = sm.listed;
    over_stretches<T, NT>(sh, sm, listed, bound, iters, [&](float v, int cls) {
        const int at = atomicAdd(&sm.count, 1);
        if (at < kCandidates) sm.cand[at] = class_key(v, cls);
    });
    __syncthreads();
    int count = sm.count;
    if (count > kCandidates) {
        // at least k keys are >= lo, fewer than k are >= hi
        unsigned long long lo = class_key(bound, 0x7fffffff), hi = ~0ull;
        if (lo == 0ull) lo = 1ull;
        while (count > kCandidates) {
            const unsigned long long mid = lo + (hi - lo) / 2;
            __syncthreads();
            if (tid == 0) sm.count = 0;
            __syncthreads();
            over_stretches<T, NT>(sh, sm, listed, bound, iters, [&](float v, int cls) {
                const unsigned long long key = class_key(v, cls);
                if (key >= mid) {
                    const int at = atomicAdd(&sm.count, 1);
                    if (at < kCandidates) sm.cand[at] = key;
                }
            });
            __syncthreads();
            const int above = sm.count;
            if (above >= k) { lo = mid; count = above; }
            else hi = mid;
        }
        __syncthreads();
    }
    // a class's place is the number of larger keys; several threads count for one where there are enough
    int share = NT;
    while (share >= 2 * count && share > 32) share /= 2;
    for (int i = tid % share; i < count; i += share) {
        const unsigned long long mine = sm.cand[i];
        int rank = 0;
#pragma unroll 4
        for (int j = tid / share; j < count; j += NT / share) rank += sm.cand[j] > mine;
        if (share == NT) sm.rank[i] = rank;
        else atomicAdd(&sm.rank[i], rank);
    }
    __syncthreads();
    return count;
}

struct LogprobsArgs {
    const void* logits;
    const int32_t* labels;
    float *logprob, *entropy, *lse;
    int32_t* top_ids;
    float* top_logprobs;
    int64_t rows, ld;
    int n, k, parts;
    float inv_t;
};

__device__ __forceinline__ void write_top(const LogprobsArgs& p, int64_t row, int rank, unsigned long long key, float m, float ln_s)
{
    p.top_ids[row * p.k + rank] = key ? key_class(key) : -1;
    p.top_logprobs[row * p.k + rank] = key ? (key_value(key) - m) * p.inv_t - ln_s : ninf();
}
template <typename T>
__device__ __forceinline__ void write_stats(const LogprobsArgs& p, int64_t row, const Sums& a)
{
    // a row without a finite logit has no distribution: a.m = -inf, a.s = 0
    const bool none = a.m == ninf() && a.s == 0.f;
    const float ln_s = logf(a.s);
    // above 10^30 every class but the largest ones weighs nothing (and may have overflowed in the weighted sum)
    const float w = a.m > 1e30f && a.m < __int_as_float(0x7f800000) ? 0.f : a.w;
    if (p.lse) p.lse[row] = none ? ninf() : fmaf(a.m, p.inv_t, ln_s);
    if (p.entropy) p.entropy[row] = none ? 0.f : fmaf(-p.inv_t, w / a.s, ln_s);
    if (p.logprob) {
        const int label = p.labels[row];
        float lp = 0.f;
        if (label >= 0 && label < p.n) {
            const float v = Io<T>::get(reinterpret_cast<const T*>(p.logits)[row * p.ld + label]);
            lp = none || v == ninf() ? ninf() : (v - a.m) * p.inv_t - ln_s;
            if (a.s != a.s) lp = a.s;
        }
        p.logprob[row] = lp;
    }
}

template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT, 1024 / NT) logprobs_fwd_kernel(const __grid_constant__ LogprobsArgs p)
{
    constexpr bool PARTS = NT == 512;                   // a row is cut into parts only where few rows leave the CTAs large
    __shared__ Sums s_part[32];
    __shared__ Sums s_parts[kMaxParts];
    __shared__ __align__(16) unsigned char s_top[TOP ? sizeof(TopShared<NT>) : 16];
    __shared__ unsigned long long s_all[TOP && PARTS ? kMaxParts * kMaxTop : 1];
    const int part = PARTS ? (int)(blockIdx.x % (unsigned)p.parts) : 0;
    const int64_t row = PARTS ? blockIdx.x / (unsigned)p.parts : blockIdx.x;
    const float c = p.inv_t * kLog2e;
    const Share<T> sh(reinterpret_cast<const T*>(p.logits) + row * p.ld, p.n, part, PARTS ? p.parts : 1);
    TopShared<NT>& sm = *reinterpret_cast<TopShared<NT>*>(s_top);
    Stretches st{nullptr, 0, 0};
    if (TOP) {
        const int rounds = (sh.c1 - sh.c0 + 4 * NT - 1) / (4 * NT);
        st.at = sm.stretch;
        st.count = TopShared<NT>::kStretches / NT;
        st.iters = (rounds + st.count - 1) / st.count;
    }
    Sums a = run_over<T, NT, true, kNoHard>(sh, c, threadIdx.x, TOP ? &st : nullptr);
    const float my_max = a.m;
    a = block_sums<NT, true, false>(a, c, s_part);
    // the strips' maxima leave the row's ends out: they are always looked at again
    int count = 0;
    if constexpr (TOP) count = select_top<T, NT>(sh, my_max, p.k, st.iters, sm);
    if (!PARTS || p.parts == 1) {
        if (threadIdx.x == 0) write_stats<T>(p, row, a);
        if constexpr (TOP) {
            const float ln_s = logf(a.s);
            for (int i = threadIdx.x; i < count; i += NT)
                if (sm.rank[i] < p.k) write_top(p, row, sm.rank[i], sm.cand[i], a.m, ln_s);
            for (int i = count + threadIdx.x; i < p.k; i += NT) write_top(p, row, i, 0ull, a.m, ln_s);
        }
        return;
    }
    if constexpr (PARTS) {
        // sums and lists go to the row's first CTA
        cg::cluster_group cl = cg::this_cluster();
        if (threadIdx.x == 0) *cl.map_shared_rank(&s_parts[part], 0) = a;
        if constexpr (TOP) {
            unsigned long long* there = cl.map_shared_rank(s_all + part * p.k, 0);
            for (int i = threadIdx.x; i < count; i += NT)
                if (sm.rank[i] < p.k) there[sm.rank[i]] = sm.cand[i];
            for (int i = count + threadIdx.x; i < p.k; i += NT) there[i] = 0ull;
        }
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        if (part) return;
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        a = join_sums<true, false>(s_parts, p.parts, threadIdx.x & 31, c);
        if (threadIdx.x == 0) write_stats<T>(p, row, a);
        if constexpr (TOP) {
            const float ln_s = logf(a.s);
            const int total = p.parts * p.k;
            for (int i = threadIdx.x; i < total; i += NT) {
                // the parts' lists are in order: a class's place is the number of larger keys in each
                const unsigned long long mine = s_all[i];
                int rank = 0;
                for (int q = 0; q < p.parts; ++q) {
                    const unsigned long long* list = s_all + q * p.k;
                    int lo = 0;                              // keys before lo are larger
#pragma unroll
                    for (int step = kMaxTop; step; step >>= 1)
                        if (lo + step <= p.k && list[lo + step - 1] > mine) lo += step;
                    rank += lo;
                }
                if (mine && rank < p.k) write_top(p, row, rank, mine, a.m, ln_s);
            }
            // fewer classes than places
            int listed = 0;
            for (int i = threadIdx.x & 31; i < total; i += 32) listed += s_all[i] != 0ull;
            listed = __reduce_add_sync(0xffffffffu, listed);
            for (int i = listed + threadIdx.x; i < p.k; i += NT) write_top(p, row, i, 0ull, a.m, ln_s);
        }
    }
}

// A warp per row of at most 32 J classes, all in registers; the list is taken one class at a time.
template <typename T, int J>
__global__ void __launch_bounds__(128) logprobs_fwd_warp_kernel(const __grid_constant__ LogprobsArgs p)
{
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    const float c = p.inv_t * kLog2e;
    float v[J];
    Sums a{ninf(), 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
        v[j] = lane + 32 * j < p.n ? Io<T>::get(x[lane + 32 * j]) : ninf();
        a.m = fmaxf(a.m, v[j]);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(0xffffffffu, a.m, d));
    const float base = base_of(a.m);
#pragma unroll
    for (int j = 0; j < J; ++j) add_value<true, false>(a, v[j], c, base);
    a = warp_sums<true, false>(a, c);
    if (lane == 0) write_stats<T>(p, row, a);
    if (p.k == 0) return;
    const float ln_s = logf(a.s);
    uint32_t o[J];
#pragma unroll
    for (int j = 0; j < J; ++j) o[j] = (uint32_t)(class_key(v[j], 0) >> 32);
    for (int r = 0; r < p.k; ++r) {
        uint32_t mine = 0;
        int at = 0x7fffffff;
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (o[j] > mine) { mine = o[j]; at = lane + 32 * j; }
        const uint32_t top = __reduce_max_sync(0xffffffffu, mine);
        const int cls = __reduce_min_sync(0xffffffffu, mine == top ? at : 0x7fffffff);
        if (lane == 0) write_top(p, row, r, top ? ((unsigned long long)top << 32) | (uint32_t)(0x7fffffff - cls) : 0ull, a.m, ln_s);
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (lane + 32 * j == cls) o[j] = 0;
    }
}

// ---- gradients -------------------------------------------------------------------------------------------------------
// Writes g(two logits) for every two classes of the share.  `out` may be the logits themselves: a thread writes what it has read.
// BOUNDED: nothing below -10^30 comes.  AGAIN: the row has been gone over just now; it is read from its end to its start, what is in L2
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
        split(g(pair(BOUNDED && v < kFloor ? kFloor : v, 0.f)), &a, &b);
        out[e] = Io<T>::put(a);
    }
}

struct LogprobsGradArgs {
    const void* logits;
    const int32_t* labels;
    const float *lse, *entropy, *d_logprob, *d_entropy;
    void* d_logits;
    int64_t rows, ld, ld_d;
    int n, parts;
    float inv_t;
};
// p of a class = 2^((v - m) c) inv_s.  From a saved log-sum-exp: m = T lse, inv_s = 1.  In fp32 that number carries ln S only while it is small
// itself; where it is not (logits in the hundreds, a row of the type's lowest value, nothing but -inf) m and S are formed again.
struct RowScale {
    float m, s;                      // S = s (1 from a saved lse)
    bool none;                       // no finite logit: no distribution
};
constexpr float kLseExact = 128.f;   // an lse below this is off by 128 2^-24 = 7.6e-6 at most
__device__ __forceinline__ RowScale scale_of(const Sums& a) { return RowScale{base_of(a.m), a.s, a.m == ninf() && a.s == 0.f}; }

struct LogprobsGrad {                // of one row: a class gets p (a + b (v - m)), the label g on top
    float c, m, a, b, g_lp, g_h, h, inv_t;
    int label;
    bool dead;                       // nothing flows back: zeros, whatever the logits hold
    bool far;                        // scales at which a class at -10^30 would weigh something, or its product with b overflow
    __device__ __forceinline__ LogprobsGrad(const LogprobsGradArgs& p, int64_t row)
    {
        label = p.labels ? p.labels[row] : -1;
        if (label >= p.n) label = -1;
        g_lp = label >= 0 && p.d_logprob ? p.d_logprob[row] : 0.f;
        g_h = p.d_entropy ? p.d_entropy[row] : 0.f;
        h = p.d_entropy ? p.entropy[row] : 0.f;
        dead = g_lp == 0.f && g_h == 0.f;
        c = p.inv_t * kLog2e;
        inv_t = p.inv_t;
    }
    __device__ __forceinline__ void scale(const RowScale& s)
    {
        if (s.none) dead = true;
        m = s.m;
        // ln p = (v - m) / T - ln S:  -(g_lp + g_h (ln p + H)) / T
        const float w = inv_t / s.s;
        a = -w * (g_lp + g_h * (h - logf(s.s)));
        b = -w * g_h * inv_t;
        far = !(fabsf(m) < 1e29f) || !(fabsf(b) < 1e6f) || !(c > 1e-20f);
    }
    __device__ __forceinline__ float slow(float v) const
    {
        const float u = v - m, e = ex2(u * c);
        return e * (e == 0.f ? a : fmaf(b, u, a));           // (a NaN, of a row without a finite sum, passes)
    }
    __device__ __forceinline__ f2 operator()(f2 v) const
    {
        const f2 u = add2(v, pair(-m, -m));
        return mul2(ex2_2(mul2(u, pair(c, c))), fma2(pair(b, b), u, pair(a, a)));
    }
    __device__ __forceinline__ float label_value(float v) const { return slow(v) + g_lp * inv_t; }
};
template <typename T, int NT>
__global__ void __launch_bounds__(NT) logprobs_bwd_kernel(const __grid_constant__ LogprobsGradArgs p)
{
    __shared__ Sums s_part[32];
    __shared__ Sums s_parts[kMaxParts];
    const int part = (int)(blockIdx.x % (unsigned)p.parts);
    const int64_t row = blockIdx.x / (unsigned)p.parts;
    const Share<T> sh(reinterpret_cast<const T*>(p.logits) + row * p.ld, p.n, part, p.parts);
    T* out = reinterpret_cast<T*>(p.d_logits) + row * p.ld_d;
    LogprobsGrad g(p, row);
    const float label_v = g.label >= 0 ? Io<T>::get(sh.row[g.label]) : 0.f;
    const float lse = p.lse[row];
    RowScale s{lse / p.inv_t, 1.f, false};
    if (!g.dead && !(fabsf(lse) < kLseExact)) {              // the same for every part of a row
        Sums a = block_sums<NT, false, false>(run_over<T, NT, false, kNoHard>(sh, g.c, threadIdx.x, nullptr), g.c, s_part);
        if (p.parts > 1) a = cluster_sums<false>(a, g.c, part, p.parts, s_parts);
        s = scale_of(a);
    }
    g.scale(s);
    __syncthreads();                                         // the label's logit has been read (the gradient may be written in its place)
    if (g.dead) write_row<T, NT, false, false>(sh, out, threadIdx.x, [](f2) { return (f2)0; });
    else if (g.far)
        write_row<T, NT, false, false>(sh, out, threadIdx.x, [&](f2 v) {
            float x, y;
            split(v, &x, &y);
            return pair(g.slow(x), g.slow(y));
        });
    else write_row<T, NT, true, false>(sh, out, threadIdx.x, g);
    if (!g.dead && sh.mine(g.label)) {
        __syncthreads();
        if (threadIdx.x == 0) out[g.label] = Io<T>::put(g.label_value(label_v));
    }
}
// the sums of a row that a warp goes over by itself
template <typename T, bool HARD>
__device__ __forceinline__ Sums warp_run_over(const T* x, int n, float c, int lane)
{
    Sums a{ninf(), 0.f, 0.f, 0.f};
    for (int i = lane; i < n; i += 32) a.m = fmaxf(a.m, Io<T>::get(x[i]));
    const float base = base_of(a.m);
    for (int i = lane; i < n; i += 32) add_value<false, HARD>(a, Io<T>::get(x[i]), c, base);
    return warp_sums<false, HARD>(a, c);
}
template <typename T>
__global__ void __launch_bounds__(128) logprobs_bwd_warp_kernel(const __grid_constant__ LogprobsGradArgs p)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    const int lane = threadIdx.x & 31;
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    T* out = reinterpret_cast<T*>(p.d_logits) + row * p.ld_d;
    LogprobsGrad g(p, row);
    const float lse = p.lse[row];
    RowScale s{lse / p.inv_t, 1.f, false};
    if (!g.dead && !(fabsf(lse) < kLseExact)) s = scale_of(warp_run_over<T, false>(x, p.n, g.c, lane));
    g.scale(s);
    for (int i = lane; i < p.n; i += 32) {
        const float v = Io<T>::get(x[i]);
        out[i] = Io<T>::put(g.dead ? 0.f : i == g.label ? g.label_value(v) : g.slow(v));
    }
}

// ---- distillation ----------------------------------------------------------------------------------------------------
struct DistillArgs {
    const void* logits;
    const int32_t *labels, *ids;
    const float* teacher;
    float *loss, *stats;             // stats [rows][2]: log-sum-exp at the temperature and at 1
    const float* d_loss;
    void* d_logits;
    int64_t rows, ld, ld_d;
    int n, k, parts;
    float temp, inv_t, alpha;
    int power;                       // the temperature where it is 1, 2, 3 or 4, else 0
};
struct Teacher {                     // of one row, in shared memory
    float q[kMaxTeacher], ln_q[kMaxTeacher], v[kMaxTeacher];
    int id[kMaxTeacher];
};
struct Entry {                       // one entry of the list, with the student's logit at its class
    int id;
    float t, v;
    __device__ __forceinline__ bool holds() const { return id >= 0 && !(t == ninf()); }
};
template <typename T>
__device__ __forceinline__ Entry read_entry(const DistillArgs& p, const T* x, int64_t row, int j)
{
    const int id = p.ids[row * p.k + j];
    const float t = p.teacher[row * p.k + j];
    const bool there = id >= 0 && id < p.n;
    return Entry{there ? id : -1, there ? t : ninf(), there ? Io<T>::get(x[id]) : 0.f};
}
__device__ __forceinline__ void put_entry(Teacher& t, int j, const Entry& e)
{
    t.id[j] = e.id;
    t.ln_q[j] = e.t;
    t.v[j] = e.v;
}
// One warp: the distribution over the list, from its logits.
__device__ __forceinline__ void list_distribution(const DistillArgs& p, Teacher& t, int lane)
{
    float m = ninf();
    for (int j = lane; j < p.k; j += 32) m = fmaxf(m, t.ln_q[j]);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    const float base = base_of(m);
    float s = 0.f;
    for (int j = lane; j < p.k; j += 32) {
        const float u = (t.ln_q[j] - base) * p.inv_t;
        t.ln_q[j] = u;
        t.q[j] = ex2(u * kLog2e);
        s += t.q[j];
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    const bool none = s == 0.f;
    const float inv = none ? 0.f : 1.f / s, ln_s = none ? 0.f : logf(s);
    for (int j = lane; j < p.k; j += 32) {
        t.q[j] *= inv;
        t.ln_q[j] -= ln_s;
    }
    __syncwarp();
}
// p_T of a class = 2^((v - m) c) / s, p = 2^((v - m1) log2 e) / h
struct RowStats {
    float m, s, m1, h;
    bool none;
};
// One warp: the row's loss.
__device__ __forceinline__ float distill_loss(const DistillArgs& p, const Teacher& t, float label_v, bool label_there, const RowStats& st, int lane)
{
    if (st.none) return 0.f;
    const float ln_s = logf(st.s);
    float a = 0.f;
    for (int j = lane; j < p.k; j += 32)
        if (!(t.q[j] == 0.f)) a += t.q[j] * (t.ln_q[j] - ((t.v[j] - st.m) * p.inv_t - ln_s));
#pragma unroll
    for (int d = 16; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
    float loss = p.alpha > 0.f ? p.alpha * p.temp * p.temp * a : 0.f;
    if (p.alpha < 1.f && label_there) loss -= (1.f - p.alpha) * ((label_v - st.m1) - logf(st.h));
    return loss;
}
__device__ __forceinline__ RowStats stats_of(const Sums& a) { return RowStats{base_of(a.m), a.s, base_of(a.m), a.h, a.m == ninf() && a.s == 0.f}; }
template <bool HARD>
__device__ __forceinline__ void write_loss(const DistillArgs& p, int64_t row, const RowStats& st, float loss)
{
    p.loss[row] = loss;
    if (p.stats) {
        p.stats[2 * row] = st.none ? ninf() : fmaf(st.m, p.inv_t, logf(st.s));
        p.stats[2 * row + 1] = st.none ? ninf() : HARD ? st.m1 + logf(st.h) : 0.f;
    }
}
// saved statistics, and whether they say enough (see RowScale)
__device__ __forceinline__ RowStats read_stats(const DistillArgs& p, int64_t row, bool* enough)
{
    const float a = p.stats[2 * row], b = p.stats[2 * row + 1];
    *enough = fabsf(a) < kLseExact && fabsf(b) < kLseExact;
    return RowStats{a * p.temp, 1.f, b, 1.f, false};
}
struct DistillGrad {                 // of one row: what every class gets, and what the listed ones get on top
    float c, m, m1, soft, hard, power_hard, w, label;
    bool dead;                       // no distribution, or a weight of 0: zeros, whatever the logits hold
    __device__ __forceinline__ DistillGrad(const DistillArgs& p, const RowStats& st, float d_loss, bool list_there, bool label_there)
    {
        w = d_loss;
        dead = st.none || d_loss == 0.f;
        c = p.inv_t * kLog2e;
        m = st.m;
        m1 = st.m1;
        label = label_there ? (1.f - p.alpha) * w : 0.f;
        soft = list_there ? p.alpha * p.temp * w / st.s : 0.f;
        hard = label / st.h;
        // p = (2^((v - m) c))^T 2^((m - m1) log2 e) / h; with a saved lse m - m1 is below (T - 1) ln n
        power_hard = hard * ex2((m - m1) * kLog2e);
    }
    template <bool HARD>
    __device__ __forceinline__ float value(float v) const
    {
        float g = soft * ex2((v - m) * c);
        if (HARD) g = fmaf(hard, ex2((v - m1) * kLog2e), g);
        return g;
    }
    template <int POWER>
    __device__ __forceinline__ f2 two(f2 v) const
    {
        const f2 e = ex2_2(mul2(add2(v, pair(-m, -m)), pair(c, c)));
        const f2 a = pair(soft, soft), b = POWER == kOwnExp ? pair(hard, hard) : pair(power_hard, power_hard);
        if (POWER == kNoHard) return mul2(a, e);
        if (POWER == 1) return mul2(add2(a, b), e);
        if (POWER == 2) return mul2(fma2(b, e, a), e);
        if (POWER == 3) return mul2(fma2(b, mul2(e, e), a), e);
        if (POWER == 4) return mul2(fma2(b, mul2(mul2(e, e), e), a), e);
        return fma2(b, ex2_2(mul2(add2(v, pair(-m1, -m1)), pair(kLog2e, kLog2e))), mul2(a, e));
    }
};
// Classes of the list and the label, written again with what they get on top.  A class listed twice gets both weights: every one of its
// entries writes the same sum.
template <typename T, bool HARD, typename Mine>
__device__ __forceinline__ void write_listed(const DistillArgs& p, const Teacher& t, const DistillGrad& g, int label, float label_v, T* out, int tid, int threads, Mine&& mine)
{
    const float per_q = p.alpha * p.temp * g.w;
    for (int j = tid; j < p.k; j += threads) {
        const int id = t.id[j];
        if (id < 0 || !mine(id)) continue;
        float q = 0.f;
#pragma unroll 8
        for (int i = 0; i < p.k; ++i) q += t.id[i] == id ? t.q[i] : 0.f;
        float v = g.value<HARD>(t.v[j]) - per_q * q;
        if (HARD && id == label) v -= g.label;
        out[id] = Io<T>::put(v);
    }
    if (HARD && tid == threads - 1 && label >= 0 && mine(label)) {
        float q = 0.f;
#pragma unroll 8
        for (int i = 0; i < p.k; ++i) q += t.id[i] == label ? t.q[i] : 0.f;
        out[label] = Io<T>::put(g.value<HARD>(label_v) - per_q * q - g.label);
    }
}

// FWD: the statistics are formed here (and the loss written); BWD: the gradient is written.  Both: the second reading of the row comes
// from L2.
template <typename T, int NT, bool HARD, bool FWD, bool BWD>
__global__ void __launch_bounds__(NT, 1024 / NT) distill_kernel(const __grid_constant__ DistillArgs p)
{
    __shared__ Sums s_part[32];
    __shared__ Sums s_parts[kMaxParts];
    __shared__ Teacher s_teacher;
    const int part = (int)(blockIdx.x % (unsigned)p.parts);
    const int64_t row = blockIdx.x / (unsigned)p.parts;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    const Share<T> sh(x, p.n, part, p.parts);
    const float c = p.inv_t * kLog2e;
    // the list and the student's logits at its classes come in while the row is gone over
    constexpr int ENTRIES = (kMaxTeacher + NT - 1) / NT;
    Entry entry[ENTRIES];
    bool holds = false;
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i) {
        entry[i] = Entry{-1, ninf(), 0.f};
        if ((int)threadIdx.x + i * NT < p.k) entry[i] = read_entry<T>(p, x, row, threadIdx.x + i * NT);
    }
    const int label = HARD ? p.labels[row] : -1;
    const bool there = HARD && label >= 0 && label < p.n;
    const float label_v = there ? Io<T>::get(x[label]) : 0.f;
    const float d_loss = BWD ? p.d_loss[row] : 0.f;
    RowStats st;
    bool form = FWD;                         // the same for every part of a row
    if constexpr (!FWD) {
        bool enough;
        st = read_stats(p, row, &enough);
        form = !enough;
    }
    Sums a{ninf(), 0.f, 0.f, 0.f};
    if (form) a = run_over_power<T, NT, HARD>(sh, c, threadIdx.x, p.power);
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i) {
        if ((int)threadIdx.x + i * NT < p.k) put_entry(s_teacher, threadIdx.x + i * NT, entry[i]);
        holds = holds || entry[i].holds();
    }
    const bool list_there = __syncthreads_or(holds);
    if (form) {
        a = block_sums<NT, false, HARD>(a, c, s_part);
        if (p.parts > 1) a = cluster_sums<HARD>(a, c, part, p.parts, s_parts);
        st = stats_of(a);
    }
    if (warp == 0) {
        list_distribution(p, s_teacher, lane);
        if (FWD && part == 0) {
            const float loss = distill_loss(p, s_teacher, label_v, there, st, lane);
            if (lane == 0) write_loss<HARD>(p, row, st, loss);
        }
    }
    if constexpr (BWD) {
        const DistillGrad g(p, st, d_loss, list_there, there);
        T* out = reinterpret_cast<T*>(p.d_logits) + row * p.ld_d;
        if (g.dead) write_row<T, NT, false, FWD>(sh, out, threadIdx.x, [](f2) { return (f2)0; });
        else if (!HARD) write_row<T, NT, false, FWD>(sh, out, threadIdx.x, [&](f2 v) { return g.two<kNoHard>(v); });
        else if (p.power == 1) write_row<T, NT, false, FWD>(sh, out, threadIdx.x, [&](f2 v) { return g.two<1>(v); });
        else if (p.power == 2) write_row<T, NT, false, FWD>(sh, out, threadIdx.x, [&](f2 v) { return g.two<2>(v); });
        else if (p.power == 3) write_row<T, NT, false, FWD>(sh, out, threadIdx.x, [&](f2 v) { return g.two<3>(v); });
        else if (p.power == 4) write_row<T, NT, false, FWD>(sh, out, threadIdx.x, [&](f2 v) { return g.two<4>(v); });
        else write_row<T, NT, false, FWD>(sh, out, threadIdx.x, [&](f2 v) { return g.two<kOwnExp>(v); });
        __syncthreads();
        if (!g.dead)
            write_listed<T, HARD>(p, s_teacher, g, there ? label : -1, label_v, out, threadIdx.x, NT, [&](int cls) { return sh.mine(cls); });
    }
}

// A warp per row of at most 32 J classes.
template <typename T, int J, bool HARD, bool FWD, bool BWD>
__global__ void __launch_bounds__(128) distill_warp_kernel(const __grid_constant__ DistillArgs p)
{
    __shared__ Teacher s_teacher[4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = (int64_t)blockIdx.x * 4 + warp;
    if (row >= p.rows) return;
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    const int label = HARD ? p.labels[row] : -1;
    const bool there = HARD && label >= 0 && label < p.n;
    const float label_v = there ? Io<T>::get(x[label]) : 0.f;
    float v[J];
    float m = ninf();
#pragma unroll
    for (int j = 0; j < J; ++j) {
        v[j] = lane + 32 * j < p.n ? Io<T>::get(x[lane + 32 * j]) : ninf();
        m = fmaxf(m, v[j]);
    }
    bool holds = false;
    for (int j = lane; j < p.k; j += 32) {
        const Entry e = read_entry<T>(p, x, row, j);
        put_entry(s_teacher[warp], j, e);
        holds = holds || e.holds();
    }
    const bool list_there = __any_sync(0xffffffffu, holds);
    list_distribution(p, s_teacher[warp], lane);
    const float c = p.inv_t * kLog2e;
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    RowStats st;
    bool enough = false;
    if constexpr (!FWD) st = read_stats(p, row, &enough);
    if (!enough) {
        Sums a{m, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < J; ++j) add_value<false, HARD>(a, v[j], c, base_of(m));
        st = stats_of(warp_sums<false, HARD>(a, c));
    }
    if constexpr (FWD) {
        const float loss = distill_loss(p, s_teacher[warp], label_v, there, st, lane);
        if (lane == 0) write_loss<HARD>(p, row, st, loss);
    }
    if constexpr (BWD) {
        const DistillGrad g(p, st, p.d_loss[row], list_there, there);
        T* out = reinterpret_cast<T*>(p.d_logits) + row * p.ld_d;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (lane + 32 * j < p.n) out[lane + 32 * j] = Io<T>::put(g.dead ? 0.f : g.value<HARD>(v[j]));
        __syncwarp();
        if (!g.dead) write_listed<T, HARD>(p, s_teacher[warp], g, there ? label : -1, label_v, out, lane, 32, [](int) { return true; });
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
template <typename K, typename A>
cudaError_t launch_rows(K* kernel, int64_t rows, int parts, int threads, cudaStream_t st, const A& args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * parts));
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args);
}
// Rows per SM from which CTAs of 128 threads take them: eight rows at different steps hide each other's waits better than four (4096 x 50021
// bf16 with 8 listed classes: 94 -> 82 us; 100 rows: 8.7 -> 11 us).
constexpr int kManyRows = 4;

template <typename K, typename A>
cudaError_t launch_warps(K* kernel, int64_t rows, cudaStream_t st, const A& args)
{
    kernel<<<(unsigned)((rows + 3) / 4), 128, 0, st>>>(args);
    return cudaGetLastError();
}

template <typename T>
cudaError_t logprobs_fwd(LogprobsArgs& a, cudaStream_t st)
{
    if (a.n <= 32) return launch_warps(logprobs_fwd_warp_kernel<T, 1>, a.rows, st, a);
    if (a.n <= 256) return launch_warps(logprobs_fwd_warp_kernel<T, 8>, a.rows, st, a);
    if (a.n <= kWarpRow) return launch_warps(logprobs_fwd_warp_kernel<T, 32>, a.rows, st, a);
    a.parts = parts_of(a.rows, a.n, sizeof(T));
    if (a.parts > 1) {
        if (a.k) return launch_rows(logprobs_fwd_kernel<T, 512, true>, a.rows, a.parts, 512, st, a);
        return launch_rows(logprobs_fwd_kernel<T, 512, false>, a.rows, a.parts, 512, st, a);
    }
    // (longer rows would have stretches of more than one round, 1.06 of the time with 256 threads at 256 KB)
    if (a.rows >= kManyRows * sm_count() && (size_t)a.n * sizeof(T) <= TopShared<128>::kStretches * 64) {
        if (a.k) return launch_rows(logprobs_fwd_kernel<T, 128, true>, a.rows, 1, 128, st, a);
        return launch_rows(logprobs_fwd_kernel<T, 128, false>, a.rows, 1, 128, st, a);
    }
    if (a.k) return launch_rows(logprobs_fwd_kernel<T, 256, true>, a.rows, 1, 256, st, a);
    return launch_rows(logprobs_fwd_kernel<T, 256, false>, a.rows, 1, 256, st, a);
}
template <typename T>
cudaError_t logprobs_bwd(LogprobsGradArgs& a, cudaStream_t st)
{
    if (a.n <= kWarpRow) return launch_warps(logprobs_bwd_warp_kernel<T>, a.rows, st, a);
    a.parts = parts_of(a.rows, a.n, sizeof(T));
    return launch_rows(logprobs_bwd_kernel<T, 256>, a.rows, a.parts, 256, st, a);
}
template <typename T, int NT, bool HARD, bool FWD, bool BWD>
cudaError_t distill_rows(DistillArgs& a, cudaStream_t st)
{
    auto* kernel = distill_kernel<T, NT, HARD, FWD, BWD>;
    return launch_rows(kernel, a.rows, a.parts, NT, st, a);
}
template <typename T, bool HARD, bool FWD, bool BWD>
cudaError_t distill_one(DistillArgs& a, cudaStream_t st)
{
    if (a.n <= 32) return launch_warps(distill_warp_kernel<T, 1, HARD, FWD, BWD>, a.rows, st, a);
    if (a.n <= 256) return launch_warps(distill_warp_kernel<T, 8, HARD, FWD, BWD>, a.rows, st, a);
    if (a.n <= kWarpRow) return launch_warps(distill_warp_kernel<T, 32, HARD, FWD, BWD>, a.rows, st, a);
    a.parts = parts_of(a.rows, a.n, sizeof(T));
    // Loss and gradient at once read a row twice, so the rows in work should fit L2: half as many of long ones (4096 rows of 256 KB: 445 us
    // with CTAs of 256, 412 with 512; of 100 KB: 165 and 200, 184 with 128; of 128 KB: 108 and 106; of 40 KB: 92 and 81 with 128).
    if (a.parts > 1 || (FWD && BWD && (size_t)a.n * sizeof(T) > 120 * 1024)) return distill_rows<T, 512, HARD, FWD, BWD>(a, st);
    if (a.rows >= kManyRows * sm_count() && (!BWD || (size_t)a.n * sizeof(T) <= 64 * 1024)) return distill_rows<T, 128, HARD, FWD, BWD>(a, st);
    return distill_rows<T, 256, HARD, FWD, BWD>(a, st);
}
template <typename T, bool FWD, bool BWD>
cudaError_t distill(DistillArgs& a, cudaStream_t st)
{
    return a.alpha < 1.f ? distill_one<T, true, FWD, BWD>(a, st) : distill_one<T, false, FWD, BWD>(a, st);
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
int power_of(float temperature) { return temperature == 1.f ? 1 : temperature == 2.f ? 2 : temperature == 3.f ? 3 : temperature == 4.f ? 4 : 0; }
int check_distill(const void* logits, const int32_t* labels, const int32_t* ids, const float* teacher, int64_t rows, int32_t classes, int64_t ld,
                  int32_t k, float temperature, float alpha, int32_t dtype)
{
    const int bad = check_rows(logits, rows, classes, ld, dtype);
    if (bad != HPF_OK) return bad;
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.f / temperature)) return api_fail(HPF_ERR_INVALID, "the temperature must be positive");
    if (!(alpha >= 0.f && alpha <= 1.f)) return api_fail(HPF_ERR_INVALID, "alpha must lie in [0, 1]");
    if (k < 0 || k > kMaxTeacher) return api_fail(HPF_ERR_UNSUPPORTED, "a teacher's list has at most 256 entries per row");
    if (rows && ((k && (!ids || !teacher)) || (alpha < 1.f && !labels))) return api_fail(HPF_ERR_INVALID, "null list, or null labels with alpha < 1");
    return HPF_OK;
}
template <bool FWD, bool BWD>
int distill_call(DistillArgs& a, int32_t dtype, void* stream)
{
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == HPF_FP32   ? distill<float, FWD, BWD>(a, st)
                          : dtype == HPF_BF16 ? distill<__nv_bfloat16, FWD, BWD>(a, st)
                                              : distill<__half, FWD, BWD>(a, st);
    return e == cudaSuccess ? HPF_OK : api_cuda_fail(e, "distillation kernel");
}

}  // namespace
}  // namespace hpf

using namespace hpf;

extern "C" int hpf_logprobs_fwd(const void* d_logits, const int32_t* d_labels, float* d_logprob, float* d_entropy, float* d_lse,
                                int32_t* d_top_ids, float* d_top_logprobs, int64_t rows, int32_t classes, int64_t ld, int32_t k,
                                float temperature, int32_t dtype, void* stream)
{
    const int bad = check_rows(d_logits, rows, classes, ld, dtype);
    if (bad != HPF_OK) return bad;
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.f / temperature)) return api_fail(HPF_ERR_INVALID, "the temperature must be positive");
    if (k < 0 || k > kMaxTop) return api_fail(HPF_ERR_UNSUPPORTED, "at most 64 classes are listed per row");
    if (rows == 0) return HPF_OK;
    if ((d_logprob && !d_labels) || (k && (!d_top_ids || !d_top_logprobs))) return api_fail(HPF_ERR_INVALID, "null labels, or k > 0 with a null list");
    LogprobsArgs a{d_logits, d_labels, d_logprob, d_entropy, d_lse, d_top_ids, d_top_logprobs, rows, ld, classes, k, 1, 1.f / temperature};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == HPF_FP32 ? logprobs_fwd<float>(a, st) : dtype == HPF_BF16 ? logprobs_fwd<__nv_bfloat16>(a, st) : logprobs_fwd<__half>(a, st);
    return e == cudaSuccess ? HPF_OK : api_cuda_fail(e, "hpf_logprobs_fwd");
}

extern "C" int hpf_logprobs_bwd(const void* d_logits, const int32_t* d_labels, const float* d_lse, const float* d_entropy,
                                const float* d_dlogprob, const float* d_dentropy, void* d_dlogits, int64_t rows, int32_t classes,
                                int64_t ld, int64_t ld_d, float temperature, int32_t dtype, void* stream)
{
    const int bad = check_rows(d_logits, rows, classes, ld, dtype);
    if (bad != HPF_OK) return bad;
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.f / temperature)) return api_fail(HPF_ERR_INVALID, "the temperature must be positive");
    if (ld_d < classes) return api_fail(HPF_ERR_INVALID, "a row stride below the class count");
    if (rows == 0) return HPF_OK;
    if (!d_lse || !d_dlogits || !on(d_dlogits, element(dtype)) || (d_dlogprob && !d_labels) || (d_dentropy && !d_entropy))
        return api_fail(HPF_ERR_INVALID, "null argument");
    LogprobsGradArgs a{d_logits, d_labels, d_lse, d_entropy, d_dlogprob, d_dentropy, d_dlogits, rows, ld, ld_d, classes, 1, 1.f / temperature};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == HPF_FP32 ? logprobs_bwd<float>(a, st) : dtype == HPF_BF16 ? logprobs_bwd<__nv_bfloat16>(a, st) : logprobs_bwd<__half>(a, st);
    return e == cudaSuccess ? HPF_OK : api_cuda_fail(e, "hpf_logprobs_bwd");
}

extern "C" int hpf_distill_fwd(const void* d_logits, const int32_t* d_labels, const int32_t* d_teacher_ids, const float* d_teacher_logits,
                               float* d_loss, float* d_stats, int64_t rows, int32_t classes, int64_t ld, int32_t k, float temperature,
                               float alpha, int32_t dtype, void* stream)
{
    const int bad = check_distill(d_logits, d_labels, d_teacher_ids, d_teacher_logits, rows, classes, ld, k, temperature, alpha, dtype);
    if (bad != HPF_OK) return bad;
    if (rows == 0) return HPF_OK;
    if (!d_loss) return api_fail(HPF_ERR_INVALID, "null argument");
    DistillArgs a{d_logits, d_labels, d_teacher_ids, d_teacher_logits, d_loss, d_stats, nullptr, nullptr, rows, ld, 0, classes, k, 1, temperature, 1.f / temperature, alpha, power_of(temperature)};
    return distill_call<true, false>(a, dtype, stream);
}

extern "C" int hpf_distill_bwd(const void* d_logits, const int32_t* d_labels, const int32_t* d_teacher_ids, const float* d_teacher_logits,
                               const float* d_stats, const float* d_dloss, void* d_dlogits, int64_t rows, int32_t classes, int64_t ld,
                               int64_t ld_d, int32_t k, float temperature, float alpha, int32_t dtype, void* stream)
{
    const int bad = check_distill(d_logits, d_labels, d_teacher_ids, d_teacher_logits, rows, classes, ld, k, temperature, alpha, dtype);
    if (bad != HPF_OK) return bad;
    if (ld_d < classes) return api_fail(HPF_ERR_INVALID, "a row stride below the class count");
    if (rows == 0) return HPF_OK;
    if (!d_stats || !d_dloss || !d_dlogits || !on(d_dlogits, element(dtype))) return api_fail(HPF_ERR_INVALID, "null argument");
    DistillArgs a{d_logits, d_labels, d_teacher_ids, d_teacher_logits, nullptr, const_cast<float*>(d_stats), d_dloss, d_dlogits, rows, ld, ld_d, classes, k, 1, temperature, 1.f / temperature, alpha, power_of(temperature)};
    return distill_call<false, true>(a, dtype, stream);
}

extern "C" int hpf_distill_fwd_bwd(const void* d_logits, const int32_t* d_labels, const int32_t* d_teacher_ids, const float* d_teacher_logits,
                                   const float* d_dloss, float* d_loss, void* d_dlogits, int64_t rows, int32_t classes, int64_t ld,
                                   int64_t ld_d, int32_t k, float temperature, float alpha, int32_t dtype, void* stream)
{
    const int bad = check_distill(d_logits, d_labels, d_teacher_ids, d_teacher_logits, rows, classes, ld, k, temperature, alpha, dtype);
    if (bad != HPF_OK) return bad;
    if (ld_d < classes) return api_fail(HPF_ERR_INVALID, "a row stride below the class count");
    if (rows == 0) return HPF_OK;
    if (!d_loss || !d_dloss || !d_dlogits || !on(d_dlogits, element(dtype))) return api_fail(HPF_ERR_INVALID, "null argument");
    DistillArgs a{d_logits, d_labels, d_teacher_ids, d_teacher_logits, d_loss, nullptr, d_dloss, d_dlogits, rows, ld, ld_d, classes, k, 1, temperature, 1.f / temperature, alpha, power_of(temperature)};
    return distill_call<true, true>(a, dtype, stream);
}
