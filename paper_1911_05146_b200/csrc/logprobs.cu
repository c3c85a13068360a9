// Log-probabilities of given labels with entropy and the likeliest classes, and their gradient (hpf_logprobs_fwd, hpf_logprobs_bwd).
// The running sums and the way a row is shared out are in logits.cuh.
#include "logits.cuh"

namespace hpf {
namespace {

constexpr int kMaxTop = 64;        // classes listed per row
constexpr int kGroups = 128;       // groups of threads whose maxima bound the k-th largest class
constexpr int kCandidates = 512;   // classes at or above that bound that are ranked by counting
constexpr int kWarpCandidates = 192;

// The upper half of a logit's place among the floats: in their order, equal where the upper 16 bits are.
__device__ __forceinline__ uint32_t order16(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    return (b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) >> 16;
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

// One warp: the k-th largest of its lanes' values, by a bitonic sort; of the maxima of 32 groups of threads (a lane's: lane, lane + 32, ...).
constexpr int kFewTop = 16;
__device__ __forceinline__ float kth_of_warp(float v, int k, int lane)
{
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
template <int NT>
__device__ __forceinline__ float kth_of_32(const float* maxima, int k, int lane)
{
    float v = ninf();
#pragma unroll
    for (int t = 0; t < NT; t += 32) v = fmaxf(v, maxima[t + lane]);
    return kth_of_warp(v, k, lane);
}
// The k-th largest of 128 values, four a lane, to the upper 16 bits: found bit by bit.
__device__ __forceinline__ float kth_of_four(const float (&value)[4], int k)
{
    uint32_t key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = order16(value[i]);
    // the bits that all keys share are the bound's too
    const uint32_t most = __reduce_max_sync(0xffffffffu, max(max(key[0], key[1]), max(key[2], key[3])));
    const uint32_t least = __reduce_min_sync(0xffffffffu, min(min(key[0], key[1]), min(key[2], key[3])));
    uint32_t bit = most == least ? 0u : 0x80000000u >> __clz(most ^ least), bound = bit ? most & ~(2 * bit - 1) : most;
    for (; bit; bit >>= 1) {
        int count = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) count += __popc(__ballot_sync(0xffffffffu, key[i] >= (bound | bit)));
        if (count >= k) bound |= bit;
    }
    const uint32_t o = bound << 16;
    // (fewer than k values above -inf: cut to 16 bits, the key of -inf would be read back as a NaN, which nothing reaches)
    return bound > order16(ninf()) ? __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)) : ninf();
}

// Of 128 groups of threads (t, t + 128, ...).
template <int NT>
__device__ __forceinline__ float kth_of_128(const float* maxima, int k, int lane)
{
    static_assert(kGroups == 128, "four groups a lane");
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = ninf();
#pragma unroll
        for (int t = 0; t < NT; t += kGroups) v[i] = fmaxf(v[i], maxima[t + i * 32 + lane]);
    }
    return kth_of_four(v, k);
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
// The label's logit, if it is wanted and there is a label (else `there` is false).
template <typename T>
__device__ __forceinline__ float label_logit(const LogprobsArgs& p, int64_t row, int label, bool* there)
{
    *there = label >= 0 && label < p.n;
    return *there ? Io<T>::get(reinterpret_cast<const T*>(p.logits)[row * p.ld + label]) : 0.f;
}
__device__ __forceinline__ void write_stats(const LogprobsArgs& p, int64_t row, const Sums& a, float label_v, bool label_there)
{
    // a row without a finite logit has no distribution: a.m = -inf, a.s = 0
    const bool none = a.m == ninf() && a.s == 0.f;
    const float ln_s = logf(a.s);
    if (p.lse) p.lse[row] = none ? ninf() : fmaf(a.m, p.inv_t, ln_s);
    if (p.entropy) p.entropy[row] = none ? 0.f : fmaf(-p.inv_t, a.w / a.s, ln_s);
    if (p.logprob) {
        float lp = 0.f;
        if (label_there) {
            lp = none || label_v == ninf() ? ninf() : (label_v - a.m) * p.inv_t - ln_s;
            if (a.s != a.s) lp = a.s;
        }
        p.logprob[row] = lp;
    }
}

template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT, 1024 / NT) logprobs_fwd_kernel(const __grid_constant__ LogprobsArgs p)
{
    enter();
    constexpr bool PARTS = NT == 512;                   // a row is cut into parts only where few rows leave the CTAs large
    __shared__ Sums s_part[32];
    __shared__ Sums s_parts[kMaxParts];
    __shared__ __align__(16) unsigned char s_top[TOP ? sizeof(TopShared<NT>) : 16];
    __shared__ unsigned long long s_all[TOP && PARTS ? kMaxParts * kMaxTop : 1];
    if (PARTS && p.parts > 1) cluster_here();
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
    // (the label's logit would be two waits at the row's end, while everybody else has left)
    const int label = p.logprob && threadIdx.x == 0 ? p.labels[row] : -1;
    bool label_there = false;
    float label_v = 0.f;
    Sums a = run_over<T, NT, true, kNoHard>(sh, c, threadIdx.x, TOP ? &st : nullptr, [&]() { label_v = label_logit<T>(p, row, label, &label_there); });
    const float my_max = a.m;
    a = block_sums<NT, true, false>(a, c, s_part);
    // the strips' maxima leave the row's ends out: they are always looked at again
    int count = 0;
    if constexpr (TOP) count = select_top<T, NT>(sh, my_max, p.k, st.iters, sm);
    if (!PARTS || p.parts == 1) {
        if (threadIdx.x == 0) write_stats(p, row, a, label_v, label_there);
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
        cluster_all_here();
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
        if (threadIdx.x == 0) write_stats(p, row, a, label_v, label_there);
        if constexpr (TOP) {
            const float ln_s = logf(a.s);
            const int total = p.parts * p.k;
            for (int i = threadIdx.x; i < total; i += NT) {
                const unsigned long long mine = s_all[i];
                int rank = 0;
                if (total <= 256) {
#pragma unroll 8
                    for (int j = 0; j < total; ++j) rank += s_all[j] > mine;
                }
                // the parts' lists are in order: a class's place is the number of larger keys in each
                for (int q = 0; total > 256 && q < p.parts; ++q) {
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

// A warp per row of at most 32 J classes, all in registers.
template <typename T, int J>
__global__ void __launch_bounds__(128) logprobs_fwd_warp_kernel(const __grid_constant__ LogprobsArgs p)
{
    enter();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    const float c = p.inv_t * kLog2e;
    float v[J];
    Sums a{ninf(), 0.f, 0.f, 0.f};
    const int label = p.logprob && lane == 0 ? p.labels[row] : -1;
#pragma unroll
    for (int j = 0; j < J; ++j) v[j] = lane + 32 * j < p.n ? Io<T>::get(x[lane + 32 * j]) : ninf();
    bool label_there;
    const float label_v = label_logit<T>(p, row, label, &label_there);
#pragma unroll
    for (int j = 0; j < J; ++j) a.m = fmaxf(a.m, v[j]);
#pragma unroll
    for (int d = 16; d; d >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(0xffffffffu, a.m, d));
    const float base = base_of(a.m);
#pragma unroll
    for (int j = 0; j < J; ++j) add_value<true, false>(a, v[j], c, base);
    a = warp_sums<true, false>(a, c);
    if (lane == 0) write_stats(p, row, a, label_v, label_there);
    if (p.k == 0) return;
    const float ln_s = logf(a.s);
    if constexpr (J > 1) {
        // as in select_top: classes at or above the k-th largest maximum (of the lanes, or of four groups a lane) are candidates, ranked by counting
        __shared__ unsigned long long s_cand[4][kWarpCandidates];
        unsigned long long* cand = s_cand[threadIdx.x >> 5];
        float top[4] = {ninf(), ninf(), ninf(), ninf()};
#pragma unroll
        for (int j = 0; j < J; ++j) top[j & 3] = fmaxf(top[j & 3], v[j]);
        const float bound = p.k <= kFewTop ? kth_of_warp(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), p.k, lane) : kth_of_four(top, p.k);
        int count = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const bool in = v[j] >= bound && v[j] > ninf();
            const uint32_t which = __ballot_sync(0xffffffffu, in);
            const int at = count + __popc(which & ((1u << lane) - 1));
            if (in && at < kWarpCandidates) cand[at] = class_key(v[j], lane + 32 * j);
            count += __popc(which);
        }
        if (count <= kWarpCandidates) {                       // (long runs of equal logits go on below)
            __syncwarp();
            for (int i = lane; i < count; i += 32) {
                const unsigned long long mine = cand[i];
                int rank = 0;
#pragma unroll 8
                for (int j = 0; j < count; ++j) rank += cand[j] > mine;
                if (rank < p.k) write_top(p, row, rank, mine, a.m, ln_s);
            }
            for (int i = count + lane; i < p.k; i += 32) write_top(p, row, i, 0ull, a.m, ln_s);
            return;
        }
    }
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
__device__ __forceinline__ RowScale scale_of(const Sums& a) { return RowScale{base_of(a.m), a.s, a.m == ninf() && a.s == 0.f}; }

struct LogprobsGrad {                // of one row: a class gets p (a + b k (v - m)), the label g on top
    float c, m, a, b, k, g_lp, g_h, h, inv_t;
    int label;
    bool dead;                       // nothing flows back: zeros, whatever the logits hold
    bool far;                        // scales at which a class at `bound` (what stands for less) would weigh something, or its product with b overflow; `k` other than 1
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
    __device__ __forceinline__ void scale(const RowScale& s, float bound)
    {
        if (s.none) dead = true;
        m = s.m;
        // ln p = (v - m) / T - ln S:  -(g_lp + g_h (ln p + H)) / T.  b k = -w g_h / T; where 1 / T^2 comes near fp32's ends, k takes 1 / T.
        const float w = inv_t / s.s;
        const bool apart = !(inv_t > 1e-15f && inv_t < 1e15f);
        a = -w * (g_lp + g_h * (h - logf(s.s)));
        b = apart ? -w * g_h : -w * g_h * inv_t;
        k = apart ? inv_t : 1.f;
        far = apart || !(fabsf(m) < 1e29f) || !(fabsf(b) < 1e6f) || !((bound - m) * c < kGone);
    }
    __device__ __forceinline__ float slow(float v) const
    {
        const float u = v - m, e = ex2(u * c);
        return e * (e == 0.f ? a : fmaf(b, u * k, a));           // (a NaN, of a row without a finite sum, passes)
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
    enter();
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
        if (p.parts > 1) cluster_here();
        Sums a = block_sums<NT, false, false>(run_over<T, NT, false, kNoHard>(sh, g.c, threadIdx.x, nullptr, []() {}), g.c, s_part);
        if (p.parts > 1) a = cluster_sums<false>(a, g.c, part, p.parts, s_parts);
        s = scale_of(a);
    }
    g.scale(s, Io<T>::kBound);
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
    enter();
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    const int lane = threadIdx.x & 31;
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
    T* out = reinterpret_cast<T*>(p.d_logits) + row * p.ld_d;
    LogprobsGrad g(p, row);
    const float lse = p.lse[row];
    RowScale s{lse / p.inv_t, 1.f, false};
    if (!g.dead && !(fabsf(lse) < kLseExact)) s = scale_of(warp_run_over<T, false>(x, p.n, g.c, lane));
    g.scale(s, Io<T>::kBound);
    for (int i0 = lane; i0 < p.n; i0 += 256) {               // eight loads under way (`out` may be x: they cannot pass the stores)
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i0 + 32 * j < p.n) v[j] = Io<T>::get(x[i0 + 32 * j]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + 32 * j;
            if (i < p.n) out[i] = Io<T>::put(g.dead ? 0.f : i == g.label ? g.label_value(v[j]) : g.slow(v[j]));
        }
    }
}

template <typename T>
cudaError_t logprobs_fwd(LogprobsArgs& a, cudaStream_t st)
{
    if (a.n <= 32) return launch_warps(logprobs_fwd_warp_kernel<T, 1>, a.rows, st, a, (size_t)a.rows * a.n * sizeof(T));
    if (a.n <= 256) return launch_warps(logprobs_fwd_warp_kernel<T, 8>, a.rows, st, a, (size_t)a.rows * a.n * sizeof(T));
    if (a.n <= kWarpRow) return launch_warps(logprobs_fwd_warp_kernel<T, 32>, a.rows, st, a, (size_t)a.rows * a.n * sizeof(T));
    a.parts = parts_of(a.rows, a.n, sizeof(T));
    if (a.parts > 1) {
        if (a.k) return launch_rows(logprobs_fwd_kernel<T, 512, true>, a.rows, a.parts, 512, st, a, (size_t)a.rows * a.n * sizeof(T));
        return launch_rows(logprobs_fwd_kernel<T, 512, false>, a.rows, a.parts, 512, st, a, (size_t)a.rows * a.n * sizeof(T));
    }
    // (longer rows would have stretches of more than one round, 1.06 of the time with 256 threads at 256 KB)
    if (a.rows >= kManyRows * sm_count() && (size_t)a.n * sizeof(T) <= TopShared<128>::kStretches * 64) {
        if (a.k) return launch_rows(logprobs_fwd_kernel<T, 128, true>, a.rows, 1, 128, st, a, (size_t)a.rows * a.n * sizeof(T));
        return launch_rows(logprobs_fwd_kernel<T, 128, false>, a.rows, 1, 128, st, a, (size_t)a.rows * a.n * sizeof(T));
    }
    if (a.k) return launch_rows(logprobs_fwd_kernel<T, 256, true>, a.rows, 1, 256, st, a, (size_t)a.rows * a.n * sizeof(T));
    return launch_rows(logprobs_fwd_kernel<T, 256, false>, a.rows, 1, 256, st, a, (size_t)a.rows * a.n * sizeof(T));
}
template <typename T>
cudaError_t logprobs_bwd(LogprobsGradArgs& a, cudaStream_t st)
{
    if (a.n <= kWarpRow) return launch_warps(logprobs_bwd_warp_kernel<T>, a.rows, st, a, (size_t)a.rows * a.n * sizeof(T));
    a.parts = parts_of(a.rows, a.n, sizeof(T));
    return launch_rows(logprobs_bwd_kernel<T, 256>, a.rows, a.parts, 256, st, a, (size_t)a.rows * a.n * sizeof(T));
}

// 1 / T stays away from the ends of fp32
bool temperature_ok(float t) { return t >= 1e-30f && t <= 1e30f; }

}  // namespace
}  // namespace hpf

using namespace hpf;

extern "C" int hpf_logprobs_fwd(const void* d_logits, const int32_t* d_labels, float* d_logprob, float* d_entropy, float* d_lse,
                                int32_t* d_top_ids, float* d_top_logprobs, int64_t rows, int32_t classes, int64_t ld, int32_t k,
                                float temperature, int32_t dtype, void* stream)
{
    const int bad = check_rows(d_logits, rows, classes, ld, dtype);
    if (bad != HPF_OK) return bad;
    if (!temperature_ok(temperature)) return api_fail(HPF_ERR_INVALID, "the temperature must lie in [1e-30, 1e30]");
    if (k < 0 || k > kMaxTop) return api_fail(HPF_ERR_UNSUPPORTED, "at most 64 classes are listed per row");
    if (rows == 0) return HPF_OK;
    if ((d_logprob && !d_labels) || (k && (!d_top_ids || !d_top_logprobs))) return api_fail(HPF_ERR_INVALID, "null labels, or k > 0 with a null list");
    const int words = check_words({d_labels, d_logprob, d_entropy, d_lse, d_top_ids, d_top_logprobs});
    if (words != HPF_OK) return words;
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
    if (!temperature_ok(temperature)) return api_fail(HPF_ERR_INVALID, "the temperature must lie in [1e-30, 1e30]");
    if (ld_d < classes) return api_fail(HPF_ERR_INVALID, "a row stride below the class count");
    if (rows == 0) return HPF_OK;
    if (!d_lse || (d_dlogprob && !d_labels) || (d_dentropy && !d_entropy)) return api_fail(HPF_ERR_INVALID, "null argument");
    const int words = check_words({d_labels, d_lse, d_entropy, d_dlogprob, d_dentropy});
    if (words != HPF_OK) return words;
    const int out = check_gradient(d_logits, d_dlogits, rows, ld, ld_d, dtype);
    if (out != HPF_OK) return out;
    LogprobsGradArgs a{d_logits, d_labels, d_lse, d_entropy, d_dlogprob, d_dentropy, d_dlogits, rows, ld, ld_d, classes, 1, 1.f / temperature};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == HPF_FP32 ? logprobs_bwd<float>(a, st) : dtype == HPF_BF16 ? logprobs_bwd<__nv_bfloat16>(a, st) : logprobs_bwd<__half>(a, st);
    return e == cudaSuccess ? HPF_OK : api_cuda_fail(e, "hpf_logprobs_bwd");
}

