// The loss against a teacher's largest logits, mixed with cross-entropy on the labels, and its gradient (hpf_distill_fwd, hpf_distill_bwd,
// hpf_distill_fwd_bwd).  The running sums and the way a row is shared out are in logits.cuh.
#include "logits.cuh"

namespace hpf {
namespace {

constexpr int kMaxTeacher = 256;   // entries of a teacher's list per row

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
// In two steps, the second of which needs what the first has fetched.
__device__ __forceinline__ void fetch_entry(const DistillArgs& p, int64_t row, int j, Entry* e)
{
    e->id = p.ids[row * p.k + j];
    e->t = p.teacher[row * p.k + j];
}
template <typename T>
__device__ __forceinline__ void finish_entry(const DistillArgs& p, const T* x, Entry* e)
{
    const bool there = e->id >= 0 && e->id < p.n;
    e->v = there ? Io<T>::get(x[e->id]) : 0.f;
    if (!there) *e = Entry{-1, ninf(), 0.f};
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
        // T (ln q - ln p_T): the logit's distance is not divided by T, which leaves fp32 for the type's lowest value
        if (!(t.q[j] == 0.f)) a += t.q[j] * fmaf(p.temp, t.ln_q[j] + ln_s, st.m - t.v[j]);
#pragma unroll
    for (int d = 16; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
    float loss = p.alpha > 0.f ? p.alpha * p.temp * a : 0.f;
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
    enter();
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
        if ((int)threadIdx.x + i * NT < p.k) fetch_entry(p, row, threadIdx.x + i * NT, &entry[i]);
    }
    const int label = HARD ? p.labels[row] : -1;
    const bool there = HARD && label >= 0 && label < p.n;
    float label_v = 0.f;
    const float d_loss = BWD ? p.d_loss[row] : 0.f;
    const auto gather = [&]() {
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i)
            if ((int)threadIdx.x + i * NT < p.k) finish_entry<T>(p, x, &entry[i]);
        if (there) label_v = Io<T>::get(x[label]);
    };
    RowStats st;
    bool form = FWD;                         // the same for every part of a row
    if constexpr (!FWD) {
        bool enough;
        st = read_stats(p, row, &enough);
        form = !enough;
    }
    Sums a{ninf(), 0.f, 0.f, 0.f};
    if (form && p.parts > 1) cluster_here();
    if (form) a = run_over_power<T, NT, HARD>(sh, c, threadIdx.x, p.power, gather);
    else gather();
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
    enter();
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
        Entry e;
        fetch_entry(p, row, j, &e);
        finish_entry<T>(p, x, &e);
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

template <typename T, int NT, bool HARD, bool FWD, bool BWD>
cudaError_t distill_rows(DistillArgs& a, cudaStream_t st)
{
    auto* kernel = distill_kernel<T, NT, HARD, FWD, BWD>;
    return launch_rows(kernel, a.rows, a.parts, NT, st, a, (size_t)a.rows * a.n * sizeof(T));
}
template <typename T, bool HARD, bool FWD, bool BWD>
cudaError_t distill_one(DistillArgs& a, cudaStream_t st)
{
    if (a.n <= 32) return launch_warps(distill_warp_kernel<T, 1, HARD, FWD, BWD>, a.rows, st, a, (size_t)a.rows * a.n * sizeof(T));
    if (a.n <= 256) return launch_warps(distill_warp_kernel<T, 8, HARD, FWD, BWD>, a.rows, st, a, (size_t)a.rows * a.n * sizeof(T));
    if (a.n <= kWarpRow) return launch_warps(distill_warp_kernel<T, 32, HARD, FWD, BWD>, a.rows, st, a, (size_t)a.rows * a.n * sizeof(T));
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

int power_of(float temperature) { return temperature == 1.f ? 1 : temperature == 2.f ? 2 : temperature == 3.f ? 3 : temperature == 4.f ? 4 : 0; }
int check_distill(const void* logits, const int32_t* labels, const int32_t* ids, const float* teacher, int64_t rows, int32_t classes, int64_t ld,
                  int32_t k, float temperature, float alpha, int32_t dtype)
{
    const int bad = check_rows(logits, rows, classes, ld, dtype);
    if (bad != HPF_OK) return bad;
    // the loss is a difference of logarithms, good to 1e-6, times T^2: beyond 100 that is as large as the loss of a list of all classes, and T^2 overflows in the end
    if (!(temperature >= 1e-3f && temperature <= 100.f)) return api_fail(HPF_ERR_INVALID, "the temperature of a distillation must lie in [0.001, 100]");
    if (!(alpha >= 0.f && alpha <= 1.f)) return api_fail(HPF_ERR_INVALID, "alpha must lie in [0, 1]");
    if (k < 0 || k > kMaxTeacher) return api_fail(HPF_ERR_UNSUPPORTED, "a teacher's list has at most 256 entries per row");
    if (rows && ((k && (!ids || !teacher)) || (alpha < 1.f && !labels))) return api_fail(HPF_ERR_INVALID, "null list, or null labels with alpha < 1");
    return check_words({labels, ids, teacher});
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

extern "C" int hpf_distill_fwd(const void* d_logits, const int32_t* d_labels, const int32_t* d_teacher_ids, const float* d_teacher_logits,
                               float* d_loss, float* d_stats, int64_t rows, int32_t classes, int64_t ld, int32_t k, float temperature,
                               float alpha, int32_t dtype, void* stream)
{
    const int bad = check_distill(d_logits, d_labels, d_teacher_ids, d_teacher_logits, rows, classes, ld, k, temperature, alpha, dtype);
    if (bad != HPF_OK) return bad;
    if (rows == 0) return HPF_OK;
    if (!d_loss) return api_fail(HPF_ERR_INVALID, "null argument");
    const int words = check_words({d_loss, d_stats});
    if (words != HPF_OK) return words;
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
    if (!d_stats || !d_dloss) return api_fail(HPF_ERR_INVALID, "null argument");
    const int words = check_words({d_stats, d_dloss});
    if (words != HPF_OK) return words;
    const int out = check_gradient(d_logits, d_dlogits, rows, ld, ld_d, dtype);
    if (out != HPF_OK) return out;
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
    if (!d_loss || !d_dloss) return api_fail(HPF_ERR_INVALID, "null argument");
    const int words = check_words({d_loss, d_dloss});
    if (words != HPF_OK) return words;
    const int out = check_gradient(d_logits, d_dlogits, rows, ld, ld_d, dtype);
    if (out != HPF_OK) return out;
    DistillArgs a{d_logits, d_labels, d_teacher_ids, d_teacher_logits, d_loss, nullptr, d_dloss, d_dlogits, rows, ld, ld_d, classes, k, 1, temperature, 1.f / temperature, alpha, power_of(temperature)};
    return distill_call<true, true>(a, dtype, stream);
}
