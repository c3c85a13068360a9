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
constexpr int kCandidates = 1024;  // classes at or above that bound that are ranked by counting
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
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
};
template <> struct Io<__nv_bfloat16> {
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
    static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Io<__half> {
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
    __device__ __forceinline__ uint4 load(int c) const { return *(reinterpret_cast<const uint4*>(row + lead) + c); }
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
// m: largest logit, s = sum 2^((v - m) c), w = sum 2^((v - m) c) (v - m) c, h = the sum of s at temperature 1
struct Sums {
    float m, s, w, h;
};
template <bool ENTROPY, bool HARD>
__device__ __forceinline__ void rescale(Sums& a, float m, float c)
{
    if (a.m == m) return;
    const float d = fmaxf((a.m - m) * c, kFloor);        // a.m may be -inf: everything it weighs is 0
    const float r = ex2(d);
    if (ENTROPY) a.w = r * fmaf(d, a.s, a.w);
    a.s *= r;
    if (HARD) a.h *= ex2(fmaxf((a.m - m) * kLog2e, kFloor));
    a.m = m;
}
// The maximum is subtracted before anything is scaled: a row of the type's lowest value stays finite, and large logits lose nothing.
template <bool ENTROPY, bool HARD>
__device__ __forceinline__ void add_value(Sums& a, float v, float c, float base)
{
    const float u = v - base;
    const float d = u * c;
    const float e = ex2(d);
    a.s += e;
    if (ENTROPY) a.w = fmaf(e, fmaxf(d, kFloor), a.w);
    if (HARD) a.h += ex2(u * kLog2e);
}
__device__ __forceinline__ float base_of(float m) { return m == ninf() ? 0.f : m; }

template <typename T, int NT, bool ENTROPY, bool HARD>
__device__ __forceinline__ Sums run_over(const Share<T>& sh, float c, int tid)
{
    constexpr int V = Io<T>::V, U = 4;
    Sums a{ninf(), 0.f, 0.f, 0.f};
    float base = 0.f;
    for (int i = sh.c0 + tid; i < sh.c1; i += U * NT) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            raw[u] = i + u * NT < sh.c1 ? sh.load(i + u * NT) : make_uint4(Io<T>::kMinusInf, Io<T>::kMinusInf, Io<T>::kMinusInf, Io<T>::kMinusInf);
        float top = ninf();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[V];
            Io<T>::unpack(raw[u], f);
#pragma unroll
            for (int j = 0; j < V; ++j) top = fmaxf(top, f[j]);
        }
        if (top > a.m) {
            rescale<ENTROPY, HARD>(a, top, c);
            base = top;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * NT < sh.c1) {
                float f[V];
                Io<T>::unpack(raw[u], f);
#pragma unroll
                for (int j = 0; j < V; ++j) add_value<ENTROPY, HARD>(a, f[j], c, base);
            }
    }
    const int e = sh.edge(tid);
    if (e >= 0) {
        const float v = Io<T>::get(sh.row[e]);
        if (v > a.m) rescale<ENTROPY, HARD>(a, v, c);
        add_value<ENTROPY, HARD>(a, v, c, base_of(a.m));
    }
    return a;
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

// the same value for every thread of the CTA, and of the cluster where a row has several parts
template <int NT, bool ENTROPY, bool HARD>
__device__ __forceinline__ Sums block_sums(Sums a, float c, int parts, Sums* s_part, Sums* s_mine)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    a = warp_sums<ENTROPY, HARD>(a, c);
    if (lane == 0) s_part[warp] = a;
    __syncthreads();
    a = join_sums<ENTROPY, HARD>(s_part, NT / 32, lane, c);
    if (parts > 1) {
        cg::cluster_group cl = cg::this_cluster();
        if (threadIdx.x == 0) *s_mine = a;
        cl.sync();
        Sums b{ninf(), 0.f, 0.f, 0.f};
        if (lane < parts) b = *cl.map_shared_rank(s_mine, lane);
        a = warp_sums<ENTROPY, HARD>(b, c);
    }
    return a;
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

struct TopShared {
    float group[kGroups];
    float maxima[1024];
    int threads[1024];
    unsigned long long cand[kCandidates];
    unsigned long long best[kMaxTop];
    int count, listed;
    float bound;
};

// Calls f(value, class) for every class of the strips of the threads in `list`, spread over the CTA, and of the row's ends.
template <typename T, int NT, typename F>
__device__ __forceinline__ void over_strips(const Share<T>& sh, const int* list, int listed, F&& f)
{
    constexpr int V = Io<T>::V;
    const int per = (sh.c1 - sh.c0 + NT - 1) / NT;                 // pieces of a strip
    for (int w = threadIdx.x; w < listed * per; w += NT) {
        const int c = sh.c0 + list[w / per] + (w % per) * NT;
        if (c < sh.c1) {
            float v[V];
            Io<T>::unpack(sh.load(c), v);
#pragma unroll
            for (int j = 0; j < V; ++j) f(v[j], sh.lead + c * V + j);
        }
    }
    const int e = sh.edge(threadIdx.x);
    if (e >= 0) f(Io<T>::get(sh.row[e]), e);
}

// The k largest classes of this CTA's share, best first, into sm.best.  Every thread knows the largest logit of its strip.
// The k-th largest of 128 group maxima is a lower bound of the k-th largest class, so only strips whose maximum reaches it are read
// again (from L2): about 128 ln(128 / (128 - k)) classes pass for unordered rows.  Threads t, t + 128, ... form a group, so that a row sorted
// by frequency does not put its head into one group.  Where too many pass (long runs of equal logits), a bisection over the unique
// keys raises the bound until they fit.
template <typename T, int NT>
__device__ __forceinline__ void select_top(const Share<T>& sh, float my_max, int k, TopShared& sm)
{
    const int tid = threadIdx.x;
    sm.maxima[tid] = my_max;
    if (tid == 0) { sm.count = 0; sm.listed = 0; }
    if (tid < kMaxTop) sm.best[tid] = 0ull;
    __syncthreads();
    float g = ninf();
    if (tid < kGroups) {
        for (int t = tid; t < NT; t += kGroups) g = fmaxf(g, sm.maxima[t]);
        sm.group[tid] = g;
    }
    __syncthreads();
    if (tid < kGroups) {
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < kGroups; j += 4) {
            const float4 o = *reinterpret_cast<const float4*>(&sm.group[j]);
            rank += (o.x > g || (o.x == g && j < tid)) + (o.y > g || (o.y == g && j + 1 < tid)) +
                    (o.z > g || (o.z == g && j + 2 < tid)) + (o.w > g || (o.w == g && j + 3 < tid));
        }
        if (rank == k - 1) sm.bound = g;
    }
    __syncthreads();
    const float bound = sm.bound;
    if (my_max >= bound && my_max > ninf()) sm.threads[atomicAdd(&sm.listed, 1)] = tid;
    __syncthreads();
    const int listed = sm.listed;
    over_strips<T, NT>(sh, sm.threads, listed, [&](float v, int cls) {
        if (v >= bound && v > ninf()) {
            const int at = atomicAdd(&sm.count, 1);
            if (at < kCandidates) sm.cand[at] = class_key(v, cls);
        }
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
            over_strips<T, NT>(sh, sm.threads, listed, [&](float v, int cls) {
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
    }
    __syncthreads();
    for (int i = tid; i < count; i += NT) {
        const unsigned long long mine = sm.cand[i];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += sm.cand[j] > mine;
        if (rank < k) sm.best[rank] = mine;
    }
    __syncthreads();
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
    if (p.lse) p.lse[row] = none ? ninf() : fmaf(a.m, p.inv_t, ln_s);
    if (p.entropy) p.entropy[row] = none ? 0.f : fmaf(-kLn2, a.w / a.s, ln_s);
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
__global__ void __launch_bounds__(NT, NT == 256 ? 5 : 1) logprobs_fwd_kernel(const __grid_constant__ LogprobsArgs p)
{
    __shared__ Sums s_part[32];
    __shared__ Sums s_mine;
    __shared__ __align__(16) unsigned char s_top[TOP ? sizeof(TopShared) : 16];
    __shared__ unsigned long long s_all[TOP && NT == 1024 ? kMaxParts * kMaxTop : 1];
    const int part = (int)(blockIdx.x % (unsigned)p.parts);
    const int64_t row = blockIdx.x / (unsigned)p.parts;
    const float c = p.inv_t * kLog2e;
    const Share<T> sh(reinterpret_cast<const T*>(p.logits) + row * p.ld, p.n, part, p.parts);
    Sums a = run_over<T, NT, true, false>(sh, c, threadIdx.x);
    const float my_max = a.m;
    a = block_sums<NT, true, false>(a, c, p.parts, s_part, &s_mine);
    if (part == 0 && threadIdx.x == 0) write_stats<T>(p, row, a);
    if constexpr (TOP) {
        TopShared& sm = *reinterpret_cast<TopShared*>(s_top);
        // the strips' maxima leave the row's ends out: they are always looked at again
        select_top<T, NT>(sh, my_max, p.k, sm);
        const float ln_s = logf(a.s);
        if (p.parts == 1) {
            if ((int)threadIdx.x < p.k) write_top(p, row, threadIdx.x, sm.best[threadIdx.x], a.m, ln_s);
        } else if constexpr (NT == 1024) {
            cg::cluster_group cl = cg::this_cluster();
            cl.sync();
            if (part == 0) {
                const int total = p.parts * p.k;
                for (int i = threadIdx.x; i < total; i += NT) s_all[i] = cl.map_shared_rank(&sm, i / p.k)->best[i % p.k];
                __syncthreads();
                for (int i = threadIdx.x; i < total; i += NT) {
                    const unsigned long long mine = s_all[i];
                    int rank = 0;
                    for (int j = 0; j < total; ++j) rank += s_all[j] > mine || (s_all[j] == mine && j < i);   // only zeros repeat
                    if (rank < p.k) write_top(p, row, rank, mine, a.m, ln_s);
                }
            }
        }
    }
    if (p.parts > 1) cg::this_cluster().sync();          // nobody leaves while its shared memory is read
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
// Writes g(logit, class) for every class of the share.  `out` may be the logits themselves: a thread writes what it has read.
template <typename T, int NT, typename F>
__device__ __forceinline__ void write_row(const Share<T>& sh, T* out, int tid, F&& g)
{
    constexpr int V = Io<T>::V, U = 2;
    const bool wide = ((reinterpret_cast<uintptr_t>(out + sh.lead)) & 15) == 0;
    for (int i = sh.c0 + tid; i < sh.c1; i += U * NT) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * NT < sh.c1) raw[u] = *(reinterpret_cast<const uint4*>(sh.row + sh.lead) + i + u * NT);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * NT < sh.c1) {
                float f[V];
                Io<T>::unpack(raw[u], f);
                const int at = sh.lead + (i + u * NT) * V;
#pragma unroll
                for (int j = 0; j < V; ++j) f[j] = g(f[j], at + j);
                if (wide) __stcs(reinterpret_cast<uint4*>(out + at), Io<T>::pack(f));
                else
#pragma unroll
                    for (int j = 0; j < V; ++j) out[at + j] = Io<T>::put(f[j]);
            }
    }
    const int e = sh.edge(tid);
    if (e >= 0) out[e] = Io<T>::put(g(Io<T>::get(sh.row[e]), e));
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
// log2 p of a class = (v - m) c - l2s.  From a saved log-sum-exp: m = 0.  In fp32 that number carries ln S only while it is small
// itself; where it is not (logits in the hundreds, a row of the type's lowest value, nothing but -inf) m and S are formed again.
struct RowScale {
    float m, l2s;
    bool none;                       // no finite logit: no distribution
};
constexpr float kLseExact = 128.f;   // an lse below this is off by 128 2^-24 = 7.6e-6 at most
__device__ __forceinline__ RowScale scale_of(const Sums& a) { return RowScale{base_of(a.m), log2f(a.s), a.m == ninf() && a.s == 0.f}; }

struct LogprobsGrad {                // of one row
    float c, m, l2s, g_lp, g_h, h, inv_t;
    int label;
    bool dead;                       // nothing flows back: zeros, whatever the logits hold
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
        m = s.m;
        l2s = s.l2s;
        if (s.none) dead = true;
    }
    __device__ __forceinline__ float operator()(float v, int cls) const
    {
        if (dead) return 0.f;
        const float d = fmaf(v - m, c, -l2s);                     // log2 p
        float g = -ex2(d) * fmaf(g_h, fmaf(fmaxf(d, kFloor), kLn2, h), g_lp);
        if (cls == label) g += g_lp;
        return g * inv_t;
    }
};
template <typename T, int NT>
__global__ void __launch_bounds__(NT) logprobs_bwd_kernel(const __grid_constant__ LogprobsGradArgs p)
{
    __shared__ Sums s_part[32];
    __shared__ Sums s_mine;
    const int part = (int)(blockIdx.x % (unsigned)p.parts);
    const int64_t row = blockIdx.x / (unsigned)p.parts;
    const Share<T> sh(reinterpret_cast<const T*>(p.logits) + row * p.ld, p.n, part, p.parts);
    LogprobsGrad g(p, row);
    bool again = false;              // the same for every part of a row
    const float lse = p.lse[row];
    RowScale s{0.f, lse * kLog2e, false};
    if (!g.dead && !(fabsf(lse) < kLseExact)) {
        again = true;
        s = scale_of(block_sums<NT, false, false>(run_over<T, NT, false, false>(sh, g.c, threadIdx.x), g.c, p.parts, s_part, &s_mine));
    }
    g.scale(s);
    write_row<T, NT>(sh, reinterpret_cast<T*>(p.d_logits) + row * p.ld_d, threadIdx.x, g);
    if (again && p.parts > 1) cg::this_cluster().sync();
}
// the sums of a row that a warp goes over by itself
template <typename T, bool HARD>
__device__ __forceinline__ Sums warp_run_over(const T* x, int n, float c, int lane)
{
    Sums a{ninf(), 0.f, 0.f, 0.f};
    for (int i = lane; i < n; i += 32) a.m = fmaxf(a.m, Io<T>::get(x[i]));
    for (int i = lane; i < n; i += 32) add_value<false, HARD>(a, Io<T>::get(x[i]), c, base_of(a.m));
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
    RowScale s{0.f, lse * kLog2e, false};
    if (!g.dead && !(fabsf(lse) < kLseExact)) s = scale_of(warp_run_over<T, false>(x, p.n, g.c, lane));
    g.scale(s);
    for (int i = lane; i < p.n; i += 32) out[i] = Io<T>::put(g(Io<T>::get(x[i]), i));
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
};
struct Teacher {                     // of one row, in shared memory
    float q[kMaxTeacher], ln_q[kMaxTeacher], v[kMaxTeacher];
    int id[kMaxTeacher];
};
// One warp: the list's distribution and the student's logits at its classes (read before anything is written in place).
// Returns the list's mass: 1, or 0 where it holds nothing.
template <typename T>
__device__ __forceinline__ float read_teacher(const DistillArgs& p, int64_t row, Teacher& t, int lane)
{
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    float m = ninf();
    for (int j = lane; j < p.k; j += 32) {
        const int id = p.ids[row * p.k + j];
        const bool there = id >= 0 && id < p.n;
        const float v = there ? p.teacher[row * p.k + j] : ninf();
        t.id[j] = there ? id : -1;
        t.ln_q[j] = v;
        t.v[j] = there ? Io<T>::get(x[id]) : 0.f;
        m = v > m ? v : m;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    const float base = m == ninf() ? 0.f : m;
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
    return none ? 0.f : 1.f;
}
struct RowStats {
    float m, l2s, l2h;               // log2-sum-exp around m at the temperature and at 1
    bool none;
};
// One warp: the row's loss.
__device__ __forceinline__ float distill_loss(const DistillArgs& p, const Teacher& t, float label_v, bool label_there, const RowStats& st, int lane)
{
    if (st.none) return 0.f;
    const float ln_s = st.l2s * kLn2;
    float a = 0.f;
    for (int j = lane; j < p.k; j += 32)
        if (!(t.q[j] == 0.f)) a += t.q[j] * (t.ln_q[j] - ((t.v[j] - st.m) * p.inv_t - ln_s));
#pragma unroll
    for (int d = 16; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
    float loss = p.alpha > 0.f ? p.alpha * p.temp * p.temp * a : 0.f;
    if (p.alpha < 1.f && label_there) loss -= (1.f - p.alpha) * ((label_v - st.m) - st.l2h * kLn2);
    return loss;
}
template <bool HARD>
__device__ __forceinline__ RowStats stats_of(const Sums& a)
{
    return RowStats{base_of(a.m), log2f(a.s), HARD ? log2f(a.h) : 0.f, a.m == ninf() && a.s == 0.f};
}
template <bool HARD>
__device__ __forceinline__ void write_loss(const DistillArgs& p, int64_t row, const RowStats& st, float loss)
{
    p.loss[row] = loss;
    if (p.stats) {
        p.stats[2 * row] = st.none ? ninf() : fmaf(st.m, p.inv_t, st.l2s * kLn2);
        p.stats[2 * row + 1] = st.none ? ninf() : HARD ? fmaf(st.l2h, kLn2, st.m) : 0.f;
    }
}
// saved statistics, and whether they say enough (see RowScale)
__device__ __forceinline__ RowStats read_stats(const DistillArgs& p, int64_t row, bool* enough)
{
    const float a = p.stats[2 * row], b = p.stats[2 * row + 1];
    *enough = fabsf(a) < kLseExact && fabsf(b) < kLseExact;
    return RowStats{0.f, a * kLog2e, b * kLog2e, false};
}
struct DistillGrad {                 // of one row: what every class gets, and what the listed ones get on top
    float c, m, l2s, l2h, soft, hard, w;
    bool dead;                       // no distribution, or a weight of 0: zeros, whatever the logits hold
    __device__ __forceinline__ DistillGrad(const DistillArgs& p, const RowStats& st, float d_loss, float mass, bool label_there)
    {
        w = d_loss;
        dead = st.none || d_loss == 0.f;
        c = p.inv_t * kLog2e;
        m = st.m;
        l2s = st.l2s;
        l2h = st.l2h;
        soft = p.alpha * p.temp * mass * w;
        hard = label_there ? (1.f - p.alpha) * w : 0.f;
    }
    template <bool HARD>
    __device__ __forceinline__ float value(float v) const
    {
        const float u = v - m;
        float g = soft * ex2(fmaf(u, c, -l2s));
        if (HARD) g = fmaf(hard, ex2(fmaf(u, kLog2e, -l2h)), g);
        return g;
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
        for (int i = 0; i < p.k; ++i) q += t.id[i] == id ? t.q[i] : 0.f;
        float v = g.value<HARD>(t.v[j]) - per_q * q;
        if (HARD && id == label) v -= g.hard;
        out[id] = Io<T>::put(v);
    }
    if (HARD && tid == 0 && label >= 0 && mine(label)) {
        float q = 0.f;
        for (int i = 0; i < p.k; ++i) q += t.id[i] == label ? t.q[i] : 0.f;
        out[label] = Io<T>::put(g.value<HARD>(label_v) - per_q * q - g.hard);
    }
}

// FWD: the statistics are formed here (and the loss written); BWD: the gradient is written.  Both: the second reading of
// the row comes from L2, which holds the rows in work (one per CTA).
template <typename T, int NT, bool HARD, bool FWD, bool BWD>
__global__ void __launch_bounds__(NT, NT == 256 ? 4 : 1) distill_kernel(const __grid_constant__ DistillArgs p)
{
    __shared__ Sums s_part[32];
    __shared__ Sums s_mine;
    __shared__ Teacher s_teacher;
    __shared__ float s_mass;
    const int part = (int)(blockIdx.x % (unsigned)p.parts);
    const int64_t row = blockIdx.x / (unsigned)p.parts;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    const Share<T> sh(x, p.n, part, p.parts);
    const int label = HARD ? p.labels[row] : -1;
    const bool there = HARD && label >= 0 && label < p.n;
    const float label_v = there ? Io<T>::get(x[label]) : 0.f;
    if (warp == 0) {
        const float mass = read_teacher<T>(p, row, s_teacher, lane);
        if (lane == 0) s_mass = mass;
    }
    const float c = p.inv_t * kLog2e;
    RowStats st;
    bool again = FWD;
    if constexpr (FWD) {
        st = stats_of<HARD>(block_sums<NT, false, HARD>(run_over<T, NT, false, HARD>(sh, c, threadIdx.x), c, p.parts, s_part, &s_mine));
        if (part == 0 && warp == 0) {
            const float loss = distill_loss(p, s_teacher, label_v, there, st, lane);
            if (lane == 0) write_loss<HARD>(p, row, st, loss);
        }
    } else {
        bool enough;                 // the same for every part of a row
        st = read_stats(p, row, &enough);
        again = !enough;
        if (again) st = stats_of<HARD>(block_sums<NT, false, HARD>(run_over<T, NT, false, HARD>(sh, c, threadIdx.x), c, p.parts, s_part, &s_mine));
    }
    if constexpr (BWD) {
        __syncthreads();
        const DistillGrad g(p, st, p.d_loss[row], s_mass, there);
        T* out = reinterpret_cast<T*>(p.d_logits) + row * p.ld_d;
        write_row<T, NT>(sh, out, threadIdx.x, [&](float v, int) { return g.dead ? 0.f : g.value<HARD>(v); });
        __syncthreads();
        if (!g.dead)
            write_listed<T, HARD>(p, s_teacher, g, there ? label : -1, label_v, out, threadIdx.x, NT, [&](int cls) { return sh.mine(cls); });
    }
    if (again && p.parts > 1) cg::this_cluster().sync();
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
    const float mass = read_teacher<T>(p, row, s_teacher[warp], lane);
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
        st = stats_of<HARD>(warp_sums<false, HARD>(a, c));
    }
    if constexpr (FWD) {
        const float loss = distill_loss(p, s_teacher[warp], label_v, there, st, lane);
        if (lane == 0) write_loss<HARD>(p, row, st, loss);
    }
    if constexpr (BWD) {
        const DistillGrad g(p, st, p.d_loss[row], mass, there);
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
// Parts of a row: while there are fewer CTAs than SMs and every part keeps 8 KB.
int parts_of(int64_t rows, int n, size_t elem)
{
    int parts = 1;
    while (parts < kMaxParts && rows * parts < sm_count() && (size_t)n * elem / (2 * parts) >= 8192) parts *= 2;
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
        if (a.k) return launch_rows(logprobs_fwd_kernel<T, 1024, true>, a.rows, a.parts, 1024, st, a);
        return launch_rows(logprobs_fwd_kernel<T, 1024, false>, a.rows, a.parts, 1024, st, a);
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
template <typename T, bool HARD, bool FWD, bool BWD>
cudaError_t distill_one(DistillArgs& a, cudaStream_t st)
{
    if (a.n <= 32) return launch_warps(distill_warp_kernel<T, 1, HARD, FWD, BWD>, a.rows, st, a);
    if (a.n <= 256) return launch_warps(distill_warp_kernel<T, 8, HARD, FWD, BWD>, a.rows, st, a);
    if (a.n <= kWarpRow) return launch_warps(distill_warp_kernel<T, 32, HARD, FWD, BWD>, a.rows, st, a);
    a.parts = parts_of(a.rows, a.n, sizeof(T));
    if (a.parts > 1) return launch_rows(distill_kernel<T, 1024, HARD, FWD, BWD>, a.rows, a.parts, 1024, st, a);
    return launch_rows(distill_kernel<T, 256, HARD, FWD, BWD>, a.rows, 1, 256, st, a);
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
    DistillArgs a{d_logits, d_labels, d_teacher_ids, d_teacher_logits, d_loss, d_stats, nullptr, nullptr, rows, ld, 0, classes, k, 1, temperature, 1.f / temperature, alpha};
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
    DistillArgs a{d_logits, d_labels, d_teacher_ids, d_teacher_logits, nullptr, const_cast<float*>(d_stats), d_dloss, d_dlogits, rows, ld, ld_d, classes, k, 1, temperature, 1.f / temperature, alpha};
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
    DistillArgs a{d_logits, d_labels, d_teacher_ids, d_teacher_logits, d_loss, nullptr, d_dloss, d_dlogits, rows, ld, ld_d, classes, k, 1, temperature, 1.f / temperature, alpha};
    return distill_call<true, true>(a, dtype, stream);
}
