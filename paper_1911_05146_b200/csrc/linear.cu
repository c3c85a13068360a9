// The linear layer: y = act(x W^T + b) + residual, and its gradients (hpf_linear_fwd, hpf_linear_bwd).
//
// Three matrix products share one kernel, out[M][N] = sum_k A(m, k) B(n, k), because an operand may be read either way round:
//   forward  out = y [rows][out]   A = x  (k contiguous)           B = W (k contiguous)
//   dx       out = dx [rows][in]   A = dz (k = out contiguous)     B = W (n = in contiguous)
//   dW       out = dW [out][in]    A = dz (m = out contiguous)     B = x (n = in contiguous)
// dz = dy * act'(z) and db = sum_rows dz come from a kernel of their own ahead of the two, since both products read dz.
//
// One CTA per SM: a TMA producer, one thread issuing tcgen05.mma into TMEM (two accumulators, so that the write-out of a tile runs
// under the next one's products) and eight write-out warps.  A tile is 128 x BN; a stage of the ring is 128 bytes of k.
// 16-bit operands: one MMA per 16 k, fp32 accumulators.  fp32 operands: x = hi + lo with hi the bits a TF32 operand keeps; four more
// warps write lo beside each stage and three MMAs form hi hi + lo hi + hi lo.  What is left out of a product (lo lo, and the bits of a lo
// that TF32 drops) is below 3 2^-20 of it, about 2^-21 on average.
// The accumulator truncates each addition, an error that grows with the number of additions and always points to zero: where the
// result is fp32, sums are taken out of TMEM every few stages and added up in registers, rounded to nearest; where it has 16 bits, every 64
// stages of a long sum.
//
// Few tiles (few rows, small layers): the k loop is split over a cluster of up to 8 CTAs.  Each leaves its fp32 partial tile in
// its own shared memory; the CTAs then add the partial tiles up over distributed shared memory, always in rank order.
#include "../../include/hpf.h"
#include "conv_tc.h"
#include "hpf_kernels.h"
#include "pairs.cuh"
#include "tc_ptx.cuh"

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <initializer_list>
#include <math.h>

namespace cg = cooperative_groups;

namespace hpf {
namespace {

constexpr int kRow = 128;                      // bytes of k (or of m / n) in a row of a stage: the swizzle's width
constexpr int kRing = 192 * 1024;              // bytes of the ring of stages
constexpr int kBlock = 4096;                   // a 32 x 32 block of fp32 on its way out
constexpr int kOutWarps = 8;
constexpr int kSmem = kRing + kOutWarps * (kBlock + 128) + 1024;
constexpr int kMaxStages = 8;
constexpr int kMaxSplit = 8;

struct GemmArgs {
    CUtensorMap ta, tb, t_out, t_z;            // the last two where `copy_out`
    int rows, cols;                            // of out
    int k_blocks, tiles_m, tiles_n, split;
    int swap;                                  // few rows: a tile's 128 lanes are columns of out, its BN columns rows of out
    int a_mn, b_mn;                            // operand has m / n contiguous (else k)
    int a_box, b_box;                          // rows of m / n that a k-contiguous stage is filled with (the rest is never looked at)
    uint32_t idesc;
    int act, wide;                             // wide: every output and the residual take 16-byte accesses
    int copy_out;                              // tiles leave by tensor copies (wide, whole k in one CTA, rows of out in the lanes) of so many columns
    int by_slab;                               // by these, or column by column through the same blocks; else row by row (finish_rows)
    void *out, *z;
    const void *bias, *residual;
    int64_t ld;                                // of out, z and residual
    DeviceStatus* status;
};

// ---- PTX this kernel adds ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void umma_f16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
        "}\n" ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 32 lanes x 32 consecutive 32-bit columns, arrived: thread i of the warp receives lane (base lane + i)
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v)
{
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
        "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
// Back to where tmem_ld32 has them, 16 columns; read again after tmem_st_wait()
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* v)
{
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// A wait that does not look at the abort flag: for copies in flight after another wait gave up.
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity)
{
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity) && clock64() - t0 < kWaitLimit) {}
}
// Operand with m / n contiguous, 16-bit: rows of 64 values (128 bytes, 128-byte swizzle), 8 rows of k 1024 bytes apart, the next
// 64 values of m / n `block_bytes` further on.
__device__ __forceinline__ uint64_t desc_mn16(uint32_t addr, uint32_t block_bytes) { return smem_desc(addr, block_bytes, 1024, 128); }

// ---- element types ----------------------------------------------------------------------------------------------------
template <typename T> struct Pack;
__device__ __forceinline__ uint16_t shared_u16(uint32_t addr)
{
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t shared_u32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
template <> struct Pack<float> {
    static constexpr int V = 4;
    using Word = uint32_t;
    static __device__ __forceinline__ Word shared_word(uint32_t at) { return shared_u32(at); }
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
template <> struct Pack<__nv_bfloat16> {
    static constexpr int V = 8;
    using Word = uint16_t;
    static __device__ __forceinline__ Word shared_word(uint32_t at) { return shared_u16(at); }
    static __device__ __forceinline__ void unpack(const uint4& r, float* f)
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ uint32_t two(float a, float b)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) { return make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7])); }
    static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Pack<__half> {
    static constexpr int V = 8;
    using Word = uint16_t;
    static __device__ __forceinline__ Word shared_word(uint32_t at) { return shared_u16(at); }
    static __device__ __forceinline__ void unpack(const uint4& r, float* f)
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = v.x; f[2 * i + 1] = v.y;
        }
    }
    static __device__ __forceinline__ uint32_t two(float a, float b)
    {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) { return make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7])); }
    static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};

__device__ __forceinline__ float reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ f2 both(float v) { return pair(v, v); }
// gelu is z Phi(z), its slope Phi(z) + z phi(z).  Phi(-|z|) = Q(t) e^(-z^2 / 2) with t = 1 / (1 + P |z|): Q, half the scaled complementary error function,
// is smooth in t and was fitted with the least largest relative error over |z| <= 14.5, where e^(-z^2 / 2) leaves fp32.  So the small values of the
// negative side are as exact as the large ones.  Seven terms: 1.5e-6; nine, for fp32: 6.4e-8 (a layer of 8192 x 64 -> 16384 bf16, all write-out: 143 us with nine,
// 136 with seven, 134 with five, which get 5.6e-5).  e^(-z^2 / 2) is what phi needs too: 2 special-function results a value where erff and expf took about 60
// instructions (the dz kernel of 8192 x 16384 bf16: 354 us with those).
template <typename T> struct Tail {
    static constexpr int N = 7;
    static constexpr float P = 0.353553391f;
    static __device__ __forceinline__ float term(int i)
    {
        const float c[N] = {0.141161801f, 0.138845259f, 0.14046068f, 0.0197253018f, 0.193506594f, -0.17757707f, 0.043876714f};
        return c[i];
    }
};
template <> struct Tail<float> {
    static constexpr int N = 9;
    static constexpr float P = 0.282842712f;
    static __device__ __forceinline__ float term(int i)
    {
        const float c[N] = {0.112818819f, 0.11319271f, 0.101148179f, 0.0959035988f, 0.0417257859f, 0.0413279856f, 0.0442964147f, -0.0712659048f, 0.0208524438f};
        return c[i];
    }
};
// Gives Phi and e^(-z^2 / 2).
template <typename T>
__device__ __forceinline__ void gauss(f2 z, f2* cdf, f2* e)
{
    constexpr int N = Tail<T>::N;
    float z0, z1, d0, d1;
    split(z, &z0, &z1);
    split(fma2(pair(fabsf(z0), fabsf(z1)), both(Tail<T>::P), both(1.f)), &d0, &d1);
    const f2 t = pair(reciprocal(d0), reciprocal(d1));
    *e = ex2_2(mul2(mul2(z, z), both(-0.72134752044f)));
    f2 q = both(Tail<T>::term(N - 1));
#pragma unroll
    for (int i = N - 2; i >= 0; --i) q = fma2(t, q, both(Tail<T>::term(i)));
    const f2 tail = mul2(mul2(t, q), *e);
    float t0, t1, u0, u1;
    split(tail, &t0, &t1);
    split(fma2(tail, both(-1.f), both(1.f)), &u0, &u1);
    *cdf = pair(z0 > 0.f ? u0 : t0, z1 > 0.f ? u1 : t1);
}
__device__ __forceinline__ f2 sigmoid(f2 z)
{
    float a, b;
    split(add2(ex2_2(mul2(z, both(-1.44269504089f))), both(1.f)), &a, &b);
    return pair(reciprocal(a), reciprocal(b));
}
template <typename T, int V>
__device__ __forceinline__ void activate(float* v, int act)
{
    static_assert(V % 2 == 0, "values in pairs");
    if (act == HPF_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = v[j] < 0.f ? 0.f : v[j];          // a NaN stays
    } else if (act == HPF_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const f2 z = pair(v[j], v[j + 1]);
            f2 cdf, e;
            gauss<T>(z, &cdf, &e);
            split(mul2(z, cdf), &v[j], &v[j + 1]);
        }
    } else if (act == HPF_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const f2 z = pair(v[j], v[j + 1]);
            split(mul2(z, sigmoid(z)), &v[j], &v[j + 1]);
        }
    }
}
// g *= act'(z)
template <typename T, int V>
__device__ __forceinline__ void apply_slope(float* g, const float* z, int act)
{
    if (act == HPF_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] = z[j] > 0.f ? g[j] : z[j] != z[j] ? z[j] : 0.f;
        return;
    }
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        const f2 zz = pair(z[j], z[j + 1]);
        f2 s;
        if (act == HPF_ACT_GELU) {
            f2 e;
            gauss<T>(zz, &s, &e);
            s = fma2(mul2(zz, both(0.39894228040f)), e, s);
        } else {
            s = sigmoid(zz);                                                 // s (1 + z (1 - s))
            s = mul2(s, fma2(zz, fma2(s, both(-1.f), both(1.f)), both(1.f)));
        }
        split(mul2(pair(g[j], g[j + 1]), s), &g[j], &g[j + 1]);
    }
}

// ---- the product ------------------------------------------------------------------------------------------------------
struct Tile {
    int m, n;
};
// Tiles in groups of 16 rows of tiles, so that CTAs working at the same time share operands in L2.
__device__ __forceinline__ Tile tile_at(int t, int tiles_m, int tiles_n)
{
    constexpr int G = 16;
    const int group = t / (G * tiles_n), first = group * G;
    const int rows = min(tiles_m - first, G), in = t - group * G * tiles_n;
    return Tile{first + in % rows, in / rows};
}
// Where 16-byte unit u of row r of a 32 x 32 block lies: units of a row are spread so that both the writers (a row per lane) and the
// readers (a few rows at a time) touch all banks.
__device__ __forceinline__ uint32_t unit_at(uint32_t block, int r, int u) { return block + r * 128 + ((u ^ (r & 7)) << 4); }
__device__ __forceinline__ float4 shared_get4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ float shared_get(uint32_t addr)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr));
    return v;
}
// A lane's 32 values as row `lane` of the block, or (swapped) as column `lane`.
__device__ __forceinline__ void block_put(uint32_t block, int lane, const float* v, int swap)
{
    if (!swap) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(unit_at(block, lane, u)), "f"(v[4 * u]), "f"(v[4 * u + 1]), "f"(v[4 * u + 2]), "f"(v[4 * u + 3])
                         : "memory");
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) asm volatile("st.shared.f32 [%0], %1;" ::"r"(unit_at(block, j, lane >> 2) + (lane & 3) * 4), "f"(v[j]) : "memory");
    }
}
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, int rank)
{
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
    return there;
}
// Towards the CTAs of a cluster: a tile's quarter blocks (8 rows x 32 columns, 1 KB) are dealt out to the ranks; the owner gets the `split`
// versions of a quarter side by side, by bulk copies that its barrier counts.  (Stores to the owners took 3.6 us for a 128 x 128 tile of four,
// loads from the others 5.)
__device__ __forceinline__ void send_quarter(uint32_t src, uint32_t dst, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], 1024, [%2];" ::"r"(dst), "r"(src), "r"(bar) : "memory");
}

__device__ __forceinline__ void tma_store_2d(const void* tmap, uint32_t src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tmap), "r"(src), "r"(c0), "r"(c1) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// all but the last N copies out have read their shared memory
template <int N>
__device__ __forceinline__ void tma_store_wait()
{
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
// A 32 x 32 block on its way out by a tensor copy: a lane holds row `lane`; 16-byte units are spread as the copy's swizzle has them.
template <typename T>
struct Slab {
    static constexpr int kBytes = 32 * 32 * sizeof(T), kSlabs = kBlock / kBytes;
    static __device__ __forceinline__ void put(uint32_t slab, int lane, const float* v)
    {
        constexpr int V = Pack<T>::V;
#pragma unroll
        for (int u = 0; u < 32 / V; ++u) {
            const uint32_t at = sizeof(T) == 2 ? slab + lane * 64 + ((u ^ ((lane >> 1) & 3)) << 4) : slab + lane * 128 + ((u ^ (lane & 7)) << 4);
            const uint4 w = Pack<T>::pack(v + u * V);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
        }
    }
};
// One warp sends the block of out at (row0, col0) off, `n` counting its copies.  Rows and columns beyond out are cut off by the copy.
template <typename T>
__device__ __forceinline__ void send_slab(const CUtensorMap* map, uint32_t slabs, int* n, const float* v, int row0, int col0, int lane)
{
    const uint32_t slab = slabs + (*n % Slab<T>::kSlabs) * Slab<T>::kBytes;
    ++*n;
    if (lane == 0) tma_store_wait<Slab<T>::kSlabs - 1>();
    __syncwarp();
    Slab<T>::put(slab, lane, v);
    fence_async_smem();
    __syncwarp();
    if (lane == 0) tma_store_2d(map, slab, col0, row0);
}
// Two blocks side by side as one copy of 64 columns of a 16-bit type, the left one first: what a copy out takes goes with its rows (about 7 clocks of
// the copy engine each), not with their length.  (4096 x 4096 gradients of 128 rows: 12.5 us with copies of 32 columns.)
template <typename T>
__device__ __forceinline__ void send_half(const CUtensorMap* map, uint32_t slab, const float* v, int row0, int col0, int cols, int lane)
{
    if constexpr (sizeof(T) == 2) {
        const int half = (col0 >> 5) & 1;
        if (!half) {
            if (lane == 0) tma_store_wait<0>();
            __syncwarp();
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint4 w = Pack<T>::pack(v + u * 8);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(unit_at(slab, lane, half * 4 + u)), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
        }
        if (half || col0 + 32 >= cols) {                       // (the right half may lie behind the last column)
            fence_async_smem();
            __syncwarp();
            if (lane == 0) tma_store_2d(map, slab, col0 - half * 32, row0);
        }
    }
}
// The same where rows of out are off 16-byte boundaries: a row at a time, a column per lane.
template <typename T>
__device__ __forceinline__ void store_slab(void* out, const GemmArgs& p, uint32_t slab, const float* v, int row0, int col0, int lane)
{
    using Word = typename Pack<T>::Word;
    constexpr int UNIT = 16 / (int)sizeof(T), PITCH = 32 * (int)sizeof(T);
    __syncwarp();
    Slab<T>::put(slab, lane, v);
    __syncwarp();
    if (col0 + lane >= p.cols) return;
    uint32_t at[8];                                          // of the lane's value in rows 0 .. 7; the pattern repeats
#pragma unroll
    for (int i = 0; i < 8; ++i) at[i] = slab + i * PITCH + (((lane / UNIT) ^ (sizeof(T) == 2 ? (i >> 1) & 3 : i)) << 4) + (lane % UNIT) * (int)sizeof(T);
    Word* q = reinterpret_cast<Word*>(out) + (int64_t)row0 * p.ld + col0 + lane;
    const int rows = min(32, p.rows - row0);
#pragma unroll 1
    for (int g = 0; g < rows; g += 8) {
        Word w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = Pack<T>::shared_word(at[i] + g * PITCH);
        if (g + 8 <= rows) {
#pragma unroll
            for (int i = 0; i < 8; ++i, q += p.ld) *q = w[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i, q += p.ld)
                if (g + i < rows) *q = w[i];
        }
    }
}
// One warp finishes the block of out at (row0, col0), a row per lane: bias, activation, residual (where rows lie on 16-byte boundaries), one
// rounding.
template <typename T>
__device__ __forceinline__ void send_block(const GemmArgs& p, uint32_t slabs, uint32_t s_bias, int* n, float* v, int row0, int col0, int lane)
{
    constexpr int V = Pack<T>::V;
    if (row0 >= p.rows || col0 >= p.cols) return;
    const T* r = reinterpret_cast<const T*>(p.residual) + (int64_t)(row0 + lane) * p.ld + col0;
    const auto residual = [&](int u) {                       // 16 bytes of it; a last piece of fewer than V columns is read one by one
        if (row0 + lane >= p.rows || col0 + u * V >= p.cols) return make_uint4(0, 0, 0, 0);
        if (col0 + (u + 1) * V <= p.cols) return *reinterpret_cast<const uint4*>(r + u * V);
        float f[V];
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = col0 + u * V + j < p.cols ? Pack<T>::get(r[u * V + j]) : 0.f;
        return Pack<T>::pack(f);
    };
    constexpr int AHEAD = sizeof(T) == 2 ? 32 / V : 1;       // fetched before the rest is done, where registers allow
    uint4 res[AHEAD];
    if (AHEAD > 1 && p.residual) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) res[u] = residual(u);
    }
    if (p.bias) {
        const float b = col0 + lane < p.cols ? Pack<T>::get(reinterpret_cast<const T*>(p.bias)[col0 + lane]) : 0.f;
        __syncwarp();
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(s_bias + lane * 4), "f"(b) : "memory");
        __syncwarp();
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float4 s = shared_get4(s_bias + u * 16);
            v[4 * u] += s.x; v[4 * u + 1] += s.y; v[4 * u + 2] += s.z; v[4 * u + 3] += s.w;
        }
    }
    if (p.z) {
        if (p.copy_out) send_slab<T>(&p.t_z, slabs, n, v, row0, col0, lane);
        else store_slab<T>(p.z, p, slabs, v, row0, col0, lane);
    }
    if (p.act != HPF_ACT_NONE) activate<T, 32>(v, p.act);
    if (p.residual) {
#pragma unroll
        for (int u = 0; u < 32 / V; ++u) {
            float f[V];
            Pack<T>::unpack(AHEAD > 1 ? res[u % AHEAD] : residual(u), f);
#pragma unroll
            for (int j = 0; j < V; ++j) v[u * V + j] += f[j];
        }
    }
    if (p.copy_out == 64) send_half<T>(&p.t_out, slabs, v, row0, col0, p.cols, lane);
    else if (p.copy_out) send_slab<T>(&p.t_out, slabs, n, v, row0, col0, lane);
    else store_slab<T>(p.out, p, slabs, v, row0, col0, lane);
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// One warp finishes ROWS_IN rows of out from (row0, col0) on, 32 columns wide, whose fp32 sums lie in shared memory: bias, activation,
// residual, one rounding.  `split` versions of the sums, 1 KB apart, are added up in order.  16 bytes of a row per lane where rows lie on
// 16-byte boundaries, else a column per lane: either way an access is whole sectors.  Four (eight) accesses of each kind are under
// way together; not more, since code unrolled further no longer fitted the instruction caches.
template <typename T, int ROWS_IN>
__device__ __forceinline__ void finish_rows(const GemmArgs& p, uint32_t block, int split, int row0, int col0, int lane)
{
    constexpr int V = Pack<T>::V, PER_ROW = 32 / V, ROWS = 32 / PER_ROW;
    const int rows = min(ROWS_IN, p.rows - row0);
    if (rows <= 0 || col0 >= p.cols) return;
    if (p.wide && col0 + 32 <= p.cols) {
        constexpr int PASSES = ROWS_IN / ROWS, B = PASSES < 4 ? PASSES : 4;
        const int c = lane % PER_ROW, col = col0 + c * V;
        float bias[V];
#pragma unroll
        for (int j = 0; j < V; ++j) bias[j] = 0.f;
        if (p.bias) {
#pragma unroll
            for (int j = 0; j < V; ++j) bias[j] = Pack<T>::get(reinterpret_cast<const T*>(p.bias)[col + j]);
        }
#pragma unroll 1
        for (int g = 0; g < PASSES; g += B) {
            float v[B * V];
            uint4 res[B];
            const int r0 = g * ROWS + lane / PER_ROW;
            const int64_t at = (int64_t)(row0 + r0) * p.ld + col, step = ROWS * p.ld;
            if (p.residual) {
#pragma unroll
                for (int i = 0; i < B; ++i)
                    if (r0 + i * ROWS < rows) res[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.residual) + at + i * step);
            }
#pragma unroll
            for (int i = 0; i < B; ++i)
#pragma unroll
                for (int h = 0; h < V / 4; ++h) {
                    const float4 s = shared_get4(unit_at(block, r0 + i * ROWS, c * (V / 4) + h));
                    float* f = v + i * V + h * 4;
                    f[0] = s.x; f[1] = s.y; f[2] = s.z; f[3] = s.w;
                }
            for (int k = 1; k < split; ++k) {
#pragma unroll
                for (int i = 0; i < B; ++i)
#pragma unroll
                    for (int h = 0; h < V / 4; ++h) {
                        const float4 s = shared_get4(unit_at(block + k * 1024, r0 + i * ROWS, c * (V / 4) + h));
                        float* f = v + i * V + h * 4;
                        f[0] += s.x; f[1] += s.y; f[2] += s.z; f[3] += s.w;
                    }
            }
#pragma unroll
            for (int i = 0; i < B * V; ++i) v[i] += bias[i % V];
            if (p.z) {
#pragma unroll
                for (int i = 0; i < B; ++i)
                    if (r0 + i * ROWS < rows) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.z) + at + i * step) = Pack<T>::pack(v + i * V);
            }
            if (p.act != HPF_ACT_NONE) activate<T, B * V>(v, p.act);
            if (p.residual) {
#pragma unroll
                for (int i = 0; i < B; ++i) {
                    float f[V];
                    Pack<T>::unpack(res[i], f);
#pragma unroll
                    for (int j = 0; j < V; ++j) v[i * V + j] += f[j];
                }
            }
#pragma unroll
            for (int i = 0; i < B; ++i)
                if (r0 + i * ROWS < rows) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.out) + at + i * step) = Pack<T>::pack(v + i * V);
        }
    } else if (col0 + lane < p.cols) {
        const int col = col0 + lane;
        const float bias = p.bias ? Pack<T>::get(reinterpret_cast<const T*>(p.bias)[col]) : 0.f;
#pragma unroll 1
        for (int g = 0; g < rows; g += 8) {
            float v[8], res[8];
            const int64_t at = (int64_t)(row0 + g) * p.ld + col;
            if (p.residual) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (g + i < rows) res[i] = Pack<T>::get(reinterpret_cast<const T*>(p.residual)[at + i * p.ld]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = shared_get(unit_at(block, g + i, lane >> 2) + (lane & 3) * 4);
            for (int k = 1; k < split; ++k) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += shared_get(unit_at(block + k * 1024, g + i, lane >> 2) + (lane & 3) * 4);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += bias;
            if (p.z) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (g + i < rows) reinterpret_cast<T*>(p.z)[at + i * p.ld] = Pack<T>::put(v[i]);
            }
            if (p.act != HPF_ACT_NONE) activate<T, 8>(v, p.act);
            if (p.residual) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += res[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (g + i < rows) reinterpret_cast<T*>(p.out)[at + i * p.ld] = Pack<T>::put(v[i]);
        }
    }
}

// E: bytes of an operand value (2: fp16 / bf16, 4: fp32 as three TF32 products).  PROMOTE: sums leave TMEM every few stages.
template <int E, int BN>
struct Shape {
    static constexpr int kA = kTileM * kRow, kB = BN * kRow;
    static constexpr int kStage = (kA + kB) * (E == 4 ? 2 : 1);
    static constexpr int kStages = kRing / kStage < kMaxStages ? kRing / kStage : kMaxStages;
    static constexpr int kThreads = (4 + kOutWarps + (E == 4 ? 4 : 0)) * 32;
    static constexpr int kInner = kRow / E;              // values in a row of a stage
};
// Stages whose products are added up in TMEM where sums leave it on the way (PROMOTE).  fp32 results: 12 or 16 truncating additions.  (fp32
// operands: with 4 stages, 48 additions, a product of K = 2048 was 1.2e-6 off, with 1 stage it is as far off as one summed in fp32 FMAs.)
// 16-bit results of long sums: 256 additions, each up to a step short and as much inside: at most 2^-14 of the sum, 1 / 8 of half a step of fp16.
template <int E, typename T>
constexpr int kChunkStages = E == 4 ? 1 : sizeof(T) == 4 ? 4 : 64;
// Stages up to which a CTA's sums for 16-bit results stay in TMEM: 512 additions, at most 2^-13 short.  (With no such limit sums of
// 2^20 products of one sign, 8192 additions a CTA, came out 1.25e-3 too small: 2.5 half steps of fp16.  Taking them out costs nothing that can be
// measured: 8192 x 16384 -> 4096 bf16 759 us either way.)
constexpr int kLongSum = 128;

template <int E, typename T, int BN, bool PROMOTE>
__global__ void __launch_bounds__(Shape<E, BN>::kThreads, 1) linear_gemm_kernel(const __grid_constant__ GemmArgs p)
{
    using S = Shape<E, BN>;
    constexpr int STAGES = S::kStages, CHUNK = kChunkStages<E, T>;
    constexpr bool LONG = PROMOTE && sizeof(T) == 2;        // long sums of 16-bit results: back in TMEM for the write-out
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long s_bars[3 * kMaxStages + 5];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t staging = ring + kRing;
    const uint32_t full = smem_u32(s_bars), empty = full + 8 * kMaxStages, ready = empty + 8 * kMaxStages, acc_full = ready + 8 * kMaxStages, acc_empty = acc_full + 16, joined = acc_empty + 16;
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int split = p.split;
    const int rank = split > 1 ? (int)(blockIdx.x % (unsigned)split) : 0;
    const int tiles = p.tiles_m * p.tiles_n;
    const int first = (int)(blockIdx.x / (unsigned)split), step = split > 1 ? tiles : (int)gridDim.x;      // a cluster has one tile
    const int kb0 = (int)((long long)p.k_blocks * rank / split), kb1 = (int)((long long)p.k_blocks * (rank + 1) / split);

    if (threadIdx.x == 32) {
        prefetch_tmap(&p.ta);
        prefetch_tmap(&p.tb);
    }
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
            mbar_init(ready + 8 * i, 4);
        }
        mbar_init(joined, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, kOutWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_alloc(smem_u32(&s_tmem), 2 * BN);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_launch_dependents();
    pdl_wait();
    volatile int* abort_flag = &s_abort;

    if (warp == 0) {
        if (elect_one()) {
            const uint32_t bytes = (p.a_mn ? S::kA : p.a_box * kRow) + (p.b_mn ? S::kB : p.b_box * kRow);
            int it = 0;
            bool live = true;
            for (int t = first; live && t < tiles; t += step) {
                const Tile tile = tile_at(t, p.tiles_m, p.tiles_n);
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int s = it % STAGES;
                    if (!mbar_wait(empty + 8 * s, ((it / STAGES) & 1) ^ 1, abort_flag)) { report(p.status, 40); live = false; break; }
                    const uint32_t a = ring + s * S::kStage, b = a + S::kA, bar = full + 8 * s;
                    mbar_expect_tx(bar, bytes);
                    const int k = kb * S::kInner;
                    if (p.a_mn) {
#pragma unroll
                        for (int i = 0; i < kTileM / S::kInner; ++i) tma_load_2d(a + i * S::kInner * kRow, &p.ta, bar, tile.m * kTileM + i * S::kInner, k);
                    } else {
                        tma_load_2d(a, &p.ta, bar, k, tile.m * kTileM);
                    }
                    if (p.b_mn) {                              // (never with BN = 32: few rows are k-contiguous)
#pragma unroll
                        for (int i = 0; i < BN / S::kInner; ++i) tma_load_2d(b + i * S::kInner * kRow, &p.tb, bar, tile.n * BN + i * S::kInner, k);
                    } else {
                        tma_load_2d(b, &p.tb, bar, k, tile.n * BN);
                    }
                }
            }
            // nothing leaves while a copy is in flight: the last copies into each stage have landed when its full barrier has turned
            for (int i = it > STAGES ? it - STAGES : 0; i < it; ++i) mbar_drain(full + 8 * (i % STAGES), (i / STAGES) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            const uint64_t layout_step_a = p.a_mn ? (E == 4 ? 1024 >> 4 : 2048 >> 4) : 2;
            const uint64_t layout_step_b = p.b_mn ? (E == 4 ? 1024 >> 4 : 2048 >> 4) : 2;
            int it = 0, chunk = 0;
            bool live = true;
            for (int t = first; live && t < tiles; t += step) {
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int in_chunk = PROMOTE ? (kb - kb0) % CHUNK : kb - kb0;
                    const int buf = chunk & 1;
                    if (in_chunk == 0) {
                        if (!mbar_wait(acc_empty + 8 * buf, ((chunk >> 1) & 1) ^ 1, abort_flag)) { report(p.status, 41); live = false; break; }
                        tc_fence_after();
                    }
                    const int s = it % STAGES;
                    if (!mbar_wait((E == 4 ? ready : full) + 8 * s, (it / STAGES) & 1, abort_flag)) { report(p.status, 42); live = false; break; }
                    tc_fence_after();
                    const uint32_t a = ring + s * S::kStage, b = a + S::kA;
                    uint64_t da, db;
                    if (E == 4) {
                        da = p.a_mn ? smem_desc_mn(a, S::kInner * kRow) : smem_desc(a, 16, 1024, 128);
                        db = p.b_mn ? smem_desc_mn(b, S::kInner * kRow) : smem_desc(b, 16, 1024, 128);
                    } else {
                        da = p.a_mn ? desc_mn16(a, S::kInner * kRow) : smem_desc(a, 16, 1024, 128);
                        db = p.b_mn ? desc_mn16(b, S::kInner * kRow) : smem_desc(b, 16, 1024, 128);
                    }
                    const uint32_t d = tmem + buf * BN;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint64_t ak = da + k * layout_step_a, bk = db + k * layout_step_b;
                        const uint32_t more = in_chunk > 0 || k > 0;
                        if constexpr (E == 4) {
                            constexpr uint64_t lo = (uint64_t)(S::kA + S::kB) >> 4;
                            umma_tf32(d, ak + lo, bk, p.idesc, more);
                            umma_tf32(d, ak, bk + lo, p.idesc, 1);
                            umma_tf32(d, ak, bk, p.idesc, 1);
                        } else {
                            umma_f16(d, ak, bk, p.idesc, more);
                        }
                    }
                    umma_commit(empty + 8 * s);
                    if (kb + 1 == kb1 || (PROMOTE && in_chunk + 1 == CHUNK)) {
                        umma_commit(acc_full + 8 * buf);
                        ++chunk;
                    }
                }
            }
            // the products issued have read their stages when the last commits of these have arrived
            for (int i = it > STAGES ? it - STAGES : 0; i < it; ++i) mbar_drain(empty + 8 * (i % STAGES), (i / STAGES) & 1);
        }
        __syncwarp();
    } else if (warp >= 4 && warp < 4 + kOutWarps) {
        constexpr int BLOCKS = BN / 64 > 0 ? BN / 64 : 1;     // blocks of 32 columns of this warp (BN = 32: of the first four warps)
        const int quad = warp & 3, half = (warp - 4) >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t mine = staging + (warp - 4) * kBlock;
        const uint32_t bias = staging + kOutWarps * kBlock + (warp - 4) * 128;
        float acc[PROMOTE ? BLOCKS : 1][32];
        int chunk = 0, sent = 0, held = 0;                    // held: the accumulator that has the finished sums
        bool live = true;
        for (int t = first; live && t < tiles; t += step) {
            const Tile tile = tile_at(t, p.tiles_m, p.tiles_n);
            // block c of the tile, once its sums are in the warp's registers
            const auto hand_over = [&](int c, float* v) {
                const int at_m = tile.m * kTileM + quad * 32, at_n = tile.n * BN + c * 32;
                const int row0 = p.swap ? at_n : at_m, col0 = p.swap ? at_m : at_n;
                if (p.by_slab) {
                    send_block<T>(p, mine, bias, &sent, v, at_m, at_n, lane);
                    return;
                }
                block_put(mine, lane, v, p.swap);
                __syncwarp();
                finish_rows<T, 32>(p, mine, 1, row0, col0, lane);
                __syncwarp();
            };
            if constexpr (PROMOTE && !LONG) {
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int j = 0; j < 32; ++j) acc[b][j] = 0.f;
                for (int kb = kb0; live && kb < kb1; kb += CHUNK, ++chunk) {
                    const int buf = chunk & 1;
                    live = mbar_wait(acc_full + 8 * buf, (chunk >> 1) & 1, abort_flag);
                    live = __all_sync(0xffffffffu, live);
                    if (!live) { report(p.status, 43); break; }
                    tc_fence_after();
                    if (BN > 32 || half == 0) {
#pragma unroll
                        for (int b = 0; b < BLOCKS; ++b) {
                            float v[32];
                            tmem_ld32(tmem + lanes + buf * BN + (half * BLOCKS + b) * 32, v);
#pragma unroll
                            for (int j = 0; j < 32; ++j) acc[b][j] += v[j];
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acc_empty + 8 * buf);
                }
                if (!live) break;
                if (split == 1 && (BN > 32 || half == 0)) {
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) hand_over(half * BLOCKS + b, acc[b]);
                }
            } else {
                if constexpr (LONG) {
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                        for (int j = 0; j < 32; ++j) acc[b][j] = 0.f;
                }
                for (int kb = kb0;; kb += CHUNK) {
                    held = chunk & 1;
                    live = mbar_wait(acc_full + 8 * held, (chunk >> 1) & 1, abort_flag);
                    live = __all_sync(0xffffffffu, live);
                    if (!live) { report(p.status, 43); break; }
                    tc_fence_after();
                    ++chunk;
                    if constexpr (!LONG) break;
                    if (BN > 32 || half == 0) {
#pragma unroll
                        for (int i = 0; i < 2 * BLOCKS; ++i) {
                            float v[16], *sums = acc[i >> 1] + (i & 1) * 16;
                            tmem_ld16(tmem + lanes + held * BN + half * BLOCKS * 32 + i * 16, v);
#pragma unroll
                            for (int j = 0; j < 16; ++j) sums[j] += v[j];
                        }
                    }
                    if (kb + CHUNK >= kb1) break;
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acc_empty + 8 * held);
                }
                if (!live) break;
                if constexpr (LONG) {
                    if (BN > 32 || half == 0) {
#pragma unroll
                        for (int i = 0; i < 2 * BLOCKS; ++i) tmem_st16(tmem + lanes + held * BN + half * BLOCKS * 32 + i * 16, acc[i >> 1] + (i & 1) * 16);
                    }
                    tmem_st_wait();
                }
                if (split > 1) break;                          // the sums are fetched once the whole cluster is done
#pragma unroll 1
                for (int b = 0; b < BLOCKS; ++b) {
                    const int c = half * BLOCKS + b;
                    float v[32];
                    if (BN > 32 || half == 0) tmem_ld32(tmem + lanes + held * BN + c * 32, v);
                    if (b == BLOCKS - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(acc_empty + 8 * held);
                    }
                    if (BN > 32 || half == 0) hand_over(c, v);
                }
            }
        }
        if (p.copy_out && lane == 0) tma_store_wait<0>();
        if (split > 1) {
            const Tile tile = tile_at(first, p.tiles_m, p.tiles_n);
            const uint32_t slots = ring + kRing / 2;           // versions of the quarters that this CTA adds up
            const bool mine_too = live && (BN > 32 || half == 0);
            // the first row of out of quarter i of the tile
            const auto row_of = [&](int i) { return (p.swap ? tile.n * BN + (i >> 4) * 32 : tile.m * kTileM + ((i >> 2) & 3) * 32) + (i & 3) * 8; };
            if (mine_too) {
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    const int c = half * BLOCKS + b;
                    float v[32];
                    if constexpr (!PROMOTE || LONG) tmem_ld32(tmem + lanes + held * BN + c * 32, v);
                    const float* sums = v;
                    if constexpr (PROMOTE && !LONG) sums = acc[b];
                    block_put(ring + (c * 4 + quad) * kBlock, lane, sums, p.swap);
                }
                fence_async_smem();
            }
            __syncwarp();
            cluster_arrive();
            cluster_wait();                                    // every product of the cluster is done: the rings are free
            if (warp == 4 && lane == 0) {
                int expected = 0;
                for (int i = rank; i < BN / 32 * 16; i += split) expected += row_of(i) < p.rows;
                mbar_expect_tx(joined, (uint32_t)(expected * split * 1024));
            }
            if (mine_too && lane < 4 * BLOCKS) {
                const int i = ((half * BLOCKS + (lane >> 2)) * 4 + quad) * 4 + (lane & 3), owner = i & (split - 1);
                if (row_of(i) < p.rows) send_quarter(ring + i * 1024, at_rank(slots + ((i & -split) + rank) * 1024, owner), at_rank(joined, owner));
            }
            __syncwarp();
            live = mbar_wait(joined, 0, abort_flag) && live;
            live = __all_sync(0xffffffffu, live);
            if (!live) report(p.status, 45);
            cluster_arrive();                                  // what was sent to this CTA has left its senders
            if (live) {
                for (int i = warp - 4; i * split + rank < BN / 32 * 16; i += kOutWarps) {
                    const int item = i * split + rank;
                    const int col0 = p.swap ? tile.m * kTileM + ((item >> 2) & 3) * 32 : tile.n * BN + (item >> 4) * 32;
                    finish_rows<T, 8>(p, slots + i * split * 1024, split, row_of(item), col0, lane);
                }
            }
            __syncwarp();
            cluster_wait();
        }
    } else if (E == 4 && warp >= 4 + kOutWarps) {
        // lo parts: what a TF32 operand drops of each value, beside the stage, in the same places
        const int tid = threadIdx.x - (4 + kOutWarps) * 32;
        constexpr int UNITS = (S::kA + S::kB) / 16;
        int it = 0;
        bool live = true;
        for (int t = first; live && t < tiles; t += step) {
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const int s = it % STAGES;
                live = mbar_wait(full + 8 * s, (it / STAGES) & 1, abort_flag);
                live = __all_sync(0xffffffffu, live);
                if (!live) { report(p.status, 44); break; }
                const uint32_t raw = ring + s * S::kStage + tid * 16, lo = raw + S::kA + S::kB;
#pragma unroll
                for (int u = 0; u < UNITS / 128; u += 4) {
                    float4 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (u + i < UNITS / 128) v[i] = shared_get4(raw + (u + i) * 2048);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (u + i < UNITS / 128)
                            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(lo + (u + i) * 2048), "f"(v[i].x - tf32_hi(v[i].x)), "f"(v[i].y - tf32_hi(v[i].y)),
                                     "f"(v[i].z - tf32_hi(v[i].z)), "f"(v[i].w - tf32_hi(v[i].w))
                                     : "memory");
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(ready + 8 * s);
            }
        }
    }

    if (split > 1 && !(warp >= 4 && warp < 4 + kOutWarps)) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 2) tmem_dealloc(tmem, 2 * BN);
}

// ---- dz and its column sums --------------------------------------------------------------------------------------------
struct DzArgs {
    const void *dy, *z;
    void *dz, *db;                   // dz: null where dy itself is read by the products; db may be null
    int64_t rows, ld, ld_dz;
    int n, parts, act, db_fp32;
};
// 16 bytes from anywhere: the two aligned pieces that hold them, and their bits shifted into place.  Rows off 16-byte boundaries are read in
// whole pieces too.
template <bool SHIFT>
struct Piece {
    uint4 a, b;
    __device__ __forceinline__ void load(const char* at)
    {
        const char* piece = SHIFT ? at - (reinterpret_cast<uintptr_t>(at) & 15) : at;
        a = *reinterpret_cast<const uint4*>(piece);
        if (SHIFT) b = *(reinterpret_cast<const uint4*>(piece) + 1);
    }
    __device__ __forceinline__ uint4 get(const char* at) const
    {
        if (!SHIFT) return a;
        const uint32_t s = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15);
        uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = s & 8 ? w[i + 2] : w[i];
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = s & 4 ? w[i + 1] : w[i];
        const uint32_t bits = (s & 3) * 8;
        return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
    }
};

// A CTA goes down 128 bytes of columns, 32 rows at a time; `parts` CTAs of a cluster share the rows and add their sums up in rank order.
// The loads of U rows a thread are issued before the first is used.
// LONG: blocks of 64 rows a thread are added up by themselves, since a sum of equal values drifts with the additions in a row (2^20 rows of 0.1 came
// out 3.9e-5 off).  Its registers cost a kernel with an activation 14 %: it is for threads of more than kLongColumn rows.
constexpr int kLongColumn = 512;
template <typename T, bool SHIFT, bool ACT, bool LONG>
__global__ void __launch_bounds__(256, SHIFT ? 3 : 4) linear_dz_kernel(const __grid_constant__ DzArgs p)
{
    constexpr int COLS = 128 / sizeof(T), V = Pack<T>::V, ROWS = 32, U = ACT || SHIFT ? 2 : 4;
    constexpr int BLOCK = 64 / U;                            // rounds of a block
    __shared__ float s_sum[8][COLS];
    __shared__ float s_total[COLS];
    __shared__ float s_block[LONG ? V : 1][LONG ? 256 : 1];  // of the blocks before
    const int part = (int)(blockIdx.x % (unsigned)p.parts);
    const int c0 = (int)(blockIdx.x / (unsigned)p.parts) * COLS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = (threadIdx.x & 7) * V;
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.f;
    const T *dy = reinterpret_cast<const T*>(p.dy) + c0 + col, *z = reinterpret_cast<const T*>(p.z) + c0 + col;
    T* dz = reinterpret_cast<T*>(p.dz) + c0 + col;
    const int step = p.parts * ROWS;
    const int there = p.n - c0 - col;                        // columns from here on
    pdl_launch_dependents();
    pdl_wait();
    const int64_t first = (int64_t)part * ROWS + (threadIdx.x >> 3);
    dy += first * p.ld;
    z += first * p.ld;
    dz += first * p.ld_dz;
    int rounds = 0;
    for (int64_t r0 = first; r0 < p.rows; r0 += U * step) {
        if (LONG && rounds++ % BLOCK == 0 && rounds > 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float& block = s_block[LONG ? j : 0][LONG ? threadIdx.x : 0];
                block = rounds > BLOCK + 1 ? block + sum[j] : sum[j];
                sum[j] = 0.f;
            }
        }
        Piece<SHIFT> gp[U], zp[ACT ? U : 1];
        uint32_t whole = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // a shifted piece reaches up to 15 bytes to either side: never out of the first row's start nor of the last row's end
            const int64_t r = r0 + u * step;
            bool in = r < p.rows && there >= V;
            if (SHIFT && ((r == 0 && c0 + col < V) || (r == p.rows - 1 && there < 2 * V))) in = false;
            if (in) {
                whole |= 1u << u;
                gp[u].load(reinterpret_cast<const char*>(dy + u * step * p.ld));
                if (ACT) zp[ACT ? u : 0].load(reinterpret_cast<const char*>(z + u * step * p.ld));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r0 + u * step >= p.rows) break;
            const T *g_at = dy + u * step * p.ld, *z_at = z + u * step * p.ld;
            float g[V], zv[V];
            if (whole >> u & 1) {
                Pack<T>::unpack(gp[u].get(reinterpret_cast<const char*>(g_at)), g);
                if (ACT) Pack<T>::unpack(zp[ACT ? u : 0].get(reinterpret_cast<const char*>(z_at)), zv);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    g[j] = j < there ? Pack<T>::get(g_at[j]) : 0.f;
                    zv[j] = ACT && j < there ? Pack<T>::get(z_at[j]) : 0.f;
                }
            }
            if (ACT) apply_slope<T, V>(g, zv, p.act);
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += g[j];
            // dz is rounded to the operands' type: the tensor cores take it in that type only.  Its rows are whole numbers of 128 bytes long.
            if (p.dz && there > 0) *reinterpret_cast<uint4*>(dz + u * step * p.ld_dz) = Pack<T>::pack(g);
        }
        dy += U * step * p.ld;
        z += U * step * p.ld;
        dz += U * step * p.ld_dz;
    }
    if (!p.db) return;
    if (LONG && rounds > BLOCK) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += s_block[LONG ? j : 0][LONG ? threadIdx.x : 0];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 8);
        sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 16);
        if (lane < 8) s_sum[warp][col + j] = sum[j];
    }
    __syncthreads();
    if (threadIdx.x < COLS) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += s_sum[w][threadIdx.x];
        s_total[threadIdx.x] = t;
    }
    if (p.parts > 1) cg::this_cluster().sync();
    if (part == 0 && threadIdx.x < COLS && c0 + (int)threadIdx.x < p.n) {
        float t = s_total[threadIdx.x];
        for (int k = 1; k < p.parts; ++k) t += *cg::this_cluster().map_shared_rank(&s_total[threadIdx.x], k);
        if (p.db_fp32) reinterpret_cast<float*>(p.db)[c0 + threadIdx.x] = t;
        else reinterpret_cast<T*>(p.db)[c0 + threadIdx.x] = Pack<T>::put(t);
    }
    if (p.parts > 1) cg::this_cluster().sync();
}

// Rows that a tensor copy cannot address (start or stride off 16 bytes), laid out again at a stride that it can: 16 bytes a thread, `across`
// threads along a row.
template <typename T>
__global__ void __launch_bounds__(256) linear_repack_kernel(const T* in, T* out, int64_t rows, int n, int64_t ld, int64_t ld_out, int across)
{
    constexpr int V = 16 / (int)sizeof(T);
    const int col = (int)(blockIdx.x * across + threadIdx.x % across) * V, down = 256 / across;
    pdl_launch_dependents();
    pdl_wait();
    if (col >= n) return;
    const int64_t step = (int64_t)gridDim.y * down;
#pragma unroll 4
    for (int64_t r = (int64_t)blockIdx.y * down + threadIdx.x / across; r < rows; r += step) {
        const T* at = in + r * ld + col;
        uint4 v;
        // pieces reach up to 15 bytes to either side: never out of the first row's start nor of the last row's end
        if (col + V <= n && !(r == 0 && col < V) && !(r == rows - 1 && col + 2 * V > n)) {
            Piece<true> p;
            p.load(reinterpret_cast<const char*>(at));
            v = p.get(reinterpret_cast<const char*>(at));
        } else {
            T w[V];
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = col + j < n ? at[j] : T(0);
            memcpy(&v, w, 16);
        }
        *reinterpret_cast<uint4*>(out + r * ld_out + col) = v;
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------
size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }
// rows of what is laid out in scratch: whole 128-byte lines (a row of a stage that straddles two took the copies 1.5 times as long)
int64_t padded(int64_t n, int e) { return (n * e + 127) / 128 * 128 / e; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int sm_count()
{
    static PerDevice<int> sms;
    int n = 0;
    if (sms.get(&n, [](int dev, int* v) { return cudaDeviceGetAttribute(v, cudaDevAttrMultiProcessorCount, dev); }) != cudaSuccess) return 148;
    return n;
}

// Every kernel of this file is launched as a programmatic dependent: it may be scheduled while its predecessor in the stream drains, sets
// itself up, and waits for the predecessor's results before its first access to global memory.  (A backward pass is three kernels, 2 us of
// launch and set-up each otherwise.)
template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, const Args&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

struct Operand {
    const void* p;
    int64_t rows, cols, ld;          // as it lies in memory: cols contiguous
    bool mn;                         // the contiguous dimension is m / n
};

// A two-dimensional tensor map.  A host thread that has made no call of the runtime yet has no current context, which the driver's encoder wants:
// cudaSetDevice makes the device's primary context current (and changes nothing where it is).
cudaError_t encode_2d(CUtensorMap* tm, CUtensorMapDataType type, void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
                      CUtensorMapSwizzle swizzle, CUtensorMapL2promotion promotion)
{
    const cuuint32_t ones[2] = {1, 1};
    for (int attempt = 0;; ++attempt) {
        if (g_encode(tm, type, 2, base, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS)
            return cudaSuccess;
        if (attempt) return cudaErrorInvalidValue;
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e == cudaSuccess) e = cudaSetDevice(dev);
        if (e != cudaSuccess) return e;
    }
}
// box: rows of m / n of a k-contiguous stage
template <int E>
cudaError_t make_map(CUtensorMap* tm, const Operand& o, int32_t dtype, int box_rows)
{
    constexpr int inner = kRow / E;
    const cuuint64_t dims[2] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(o.ld * E)};
    const cuuint32_t box[2] = {(cuuint32_t)inner, (cuuint32_t)(o.mn ? inner : box_rows)};
    const CUtensorMapDataType type = dtype == HPF_FP32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == HPF_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return encode_2d(tm, type, const_cast<void*>(o.p), dims, strides, box, E == 4 && o.mn ? CU_TENSOR_MAP_SWIZZLE_128B_ATOM_32B : CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

// map of an output: copies of 32 rows x 32 or 64 columns
template <typename T>
cudaError_t make_out_map(CUtensorMap* tm, void* out, int64_t rows, int64_t cols, int64_t ld, int32_t dtype, int width)
{
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(ld * sizeof(T))};
    const cuuint32_t box[2] = {(cuuint32_t)width, 32};
    const CUtensorMapDataType type = sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == HPF_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return encode_2d(tm, type, out, dims, strides, box, width * sizeof(T) == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE);
}

template <int E, typename T, int BN, bool PROMOTE>
cudaError_t launch_gemm(GemmArgs& g, cudaStream_t st)
{
    auto* kernel = linear_gemm_kernel<E, T, BN, PROMOTE>;
    static PerDevice<bool> attributes;
    bool set = false;
    cudaError_t e = attributes.get(&set, [&](int, bool* v) { *v = true; return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); });
    if (e != cudaSuccess) return e;
    const int tiles = g.tiles_m * g.tiles_n;
    const unsigned grid = g.split > 1 ? (unsigned)(tiles * g.split) : (unsigned)(tiles < sm_count() ? tiles : sm_count());
    return launch(kernel, grid, Shape<E, BN>::kThreads, kSmem, g.split, st, g);
}

// Clusters of 1, 2, 4 and 8 CTAs of this kernel's shape that the device holds at a time (one CTA per SM; a cluster stays within a GPC,
// so of the larger ones fewer fit than the SMs would make: with twice 8 more CTAs than fit, products took 16 us longer).
struct Fit {
    int clusters[4];
};
cudaError_t how_many_fit(Fit* fit)
{
    static PerDevice<Fit> known;
    return known.get(fit, [](int, Fit* f) {
        auto* kernel = linear_gemm_kernel<2, __nv_bfloat16, 128, false>;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        for (int i = 0; i < 4 && e == cudaSuccess; ++i) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(1u << i);
            cfg.blockDim = dim3(Shape<2, 128>::kThreads);
            cfg.dynamicSmemBytes = kSmem;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = 1u << i;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&f->clusters[i], kernel, &cfg);
            if (i == 0 && f->clusters[0] < 1) f->clusters[0] = 1;           // (a size of which none fits is not chosen)
        }
        return e;
    });
}
struct Plan {
    int bn, split;
};
// Tile width and split of k by a modelled time in clocks: waves of CTAs x (stages a CTA runs through x clocks of a stage + what a tile
// costs besides).  A stage takes its MMAs (M = 128: 39 clocks at N = 32, 48 at 64, 64 at 128, 128 at 256), its copies, reckoned at 48 bytes a
// clock, or, with fp32 operands, what goes through shared memory at 128 bytes a clock (copied in, lo parts formed, three products read: 768
// bytes a row of a stage), whichever is longest.  (The rate of copies is on the low side: SMs got 74 bytes a clock in 509 x 50021 -> 1024 with 128
// columns, 77 in 4096 x 4096 -> 8192 with 256.  At 76 of them, 95 of 100 drawn sizes get the same plan.)
Plan choose(int64_t lanes, int64_t cols, int k_blocks, int narrowest, int widest, bool fp32, const Fit& fit)
{
    Plan best{widest, 1};
    double least = 1e300;
    for (int bn = widest; bn >= narrowest; bn /= 2) {
        const int64_t tiles = ((lanes + kTileM - 1) / kTileM) * ((cols + bn - 1) / bn);
        const double products = (fp32 ? 12 : 4) * (bn == 256 ? 128.0 : bn == 128 ? 64.0 : bn == 64 ? 48.0 : 39.0), copies = (kTileM + bn) * kRow / 48.0;
        const double shared = fp32 ? (kTileM + bn) * 6.0 : 0.0;
        const double stage = products > copies ? (products > shared ? products : shared) : copies > shared ? copies : shared;
        for (int i = 0, split = 1; split <= kMaxSplit; ++i, split *= 2) {
            if (split > 1 && (bn == 256 || k_blocks < 2 * split || tiles > 2 * fit.clusters[i])) break;      // (two versions of 256 columns do not fit the ring)
            const int64_t waves = (tiles + fit.clusters[i] - 1) / fit.clusters[i];
            const double t = waves * (((k_blocks + split - 1) / split) * stage + 6.0 * bn) + 2500.0 + (split > 1 ? 1500.0 : 0.0);
            if (t < least) { least = t; best = Plan{bn, split}; }
        }
    }
    return best;
}

template <int E, typename T, bool PROMOTE>
cudaError_t launch_width(GemmArgs& g, int bn, int32_t dtype, cudaStream_t st)
{
    // 64 columns where one warp has two blocks side by side and its staging is needed for one output only.  A copy writes whole 16-byte units, also past
    // the last column: rows that end inside one leave row by row.
    g.copy_out = !g.wide || g.split > 1 || g.swap || g.cols * sizeof(T) % 16 ? 0 : sizeof(T) == 2 && bn >= 128 && !g.z ? 64 : 32;
    g.by_slab = g.copy_out || (!g.wide && !g.swap && !g.residual);
    if (g.copy_out) {
        cudaError_t e = make_out_map<T>(&g.t_out, g.out, g.rows, g.cols, g.ld, dtype, g.copy_out);
        if (e == cudaSuccess && g.z) e = make_out_map<T>(&g.t_z, g.z, g.rows, g.cols, g.ld, dtype, g.copy_out);
        if (e != cudaSuccess) return e;
    }
    if constexpr (sizeof(T) == 2) {
        if (bn == 256) return launch_gemm<E, T, 256, PROMOTE>(g, st);
    }
    return bn == 128 ? launch_gemm<E, T, 128, PROMOTE>(g, st) : bn == 64 ? launch_gemm<E, T, 64, PROMOTE>(g, st) : launch_gemm<E, T, 32, PROMOTE>(g, st);
}

constexpr int kFewRows = 64;       // up to here the rows of out are the narrow side of a tile

// out[rows][cols] = sum_k a(row, k) b(col, k); out_fp32: the result is fp32 whatever the operands' type is
template <int E>
cudaError_t gemm(GemmArgs& g, Operand a, Operand b, int64_t rows, int64_t cols, int64_t K, int32_t dtype, bool out_fp32, cudaStream_t st)
{
    const bool promote = dtype == HPF_FP32 || out_fp32;
    Fit fit;
    cudaError_t e = how_many_fit(&fit);
    if (e != cudaSuccess) return e;
    const size_t oe = promote ? 4 : 2;
    g.rows = (int)rows;
    g.cols = (int)cols;
    g.wide = aligned16(g.out) && (g.ld * oe) % 16 == 0 && (!g.z || aligned16(g.z)) && (!g.residual || aligned16(g.residual));
    g.swap = rows <= kFewRows && !a.mn;
    int64_t lanes = rows, across = cols;
    if (g.swap) {
        const Operand o = a; a = b; b = o;
        lanes = cols;
        across = rows;
    }
    g.k_blocks = (int)((K * E + kRow - 1) / kRow);
    const Plan plan = choose(lanes, across, g.k_blocks, g.swap ? 32 : 64, g.swap ? (across <= 32 ? 32 : 64) : promote ? 128 : 256, E == 4, fit);
    g.split = plan.split;
    g.tiles_m = (int)((lanes + kTileM - 1) / kTileM);
    g.tiles_n = (int)((across + plan.bn - 1) / plan.bn);
    g.a_mn = a.mn; g.b_mn = b.mn;
    g.a_box = (int)(lanes < kTileM ? (lanes + 7) / 8 * 8 : kTileM);
    g.b_box = (int)(across < plan.bn ? (across + 7) / 8 * 8 : plan.bn);
    const uint32_t fmt = dtype == HPF_FP32 ? 2u : dtype == HPF_BF16 ? 1u : 0u;
    g.idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((a.mn ? 1u : 0u) << 15) | ((b.mn ? 1u : 0u) << 16) | ((uint32_t)(plan.bn >> 3) << 17) | ((uint32_t)(kTileM >> 4) << 24);
    e = make_map<E>(&g.ta, a, dtype, g.a_box);
    if (e == cudaSuccess) e = make_map<E>(&g.tb, b, dtype, g.b_box);
    if (e != cudaSuccess) return e;
    if constexpr (E == 4) {
        return launch_width<4, float, true>(g, plan.bn, dtype, st);
    } else {
        if (out_fp32) return launch_width<2, float, true>(g, plan.bn, dtype, st);
        if ((g.k_blocks + g.split - 1) / g.split > kLongSum)
            return dtype == HPF_BF16 ? launch_width<2, __nv_bfloat16, true>(g, plan.bn, dtype, st) : launch_width<2, __half, true>(g, plan.bn, dtype, st);
        return dtype == HPF_BF16 ? launch_width<2, __nv_bfloat16, false>(g, plan.bn, dtype, st) : launch_width<2, __half, false>(g, plan.bn, dtype, st);
    }
}
cudaError_t gemm_any(GemmArgs& g, const Operand& a, const Operand& b, int64_t rows, int64_t cols, int64_t K, int32_t dtype, bool out_fp32, cudaStream_t st)
{
    return dtype == HPF_FP32 ? gemm<4>(g, a, b, rows, cols, K, dtype, out_fp32, st) : gemm<2>(g, a, b, rows, cols, K, dtype, out_fp32, st);
}

cudaError_t repack(const void* in, void* out, int64_t rows, int n, int64_t ld, int64_t ld_out, int e, cudaStream_t st)
{
    const int pieces = (int)(((int64_t)n * e + 15) / 16);
    int across = 256;
    while (across > 8 && across / 2 >= pieces) across /= 2;
    const int64_t wide = (pieces + across - 1) / across, high = (rows + 256 / across - 1) / (256 / across);
    // (a few rows a thread where there are more than the GPU holds at a time)
    const int64_t most = (16 * sm_count() + wide - 1) / wide;
    const dim3 grid((unsigned)wide, (unsigned)(high < most ? high : most < 65535 ? most : 65535));
    if (e == 4) return launch(linear_repack_kernel<uint32_t>, grid, 256, 0, 1, st, static_cast<const uint32_t*>(in), static_cast<uint32_t*>(out), rows, n, ld, ld_out, across);
    return launch(linear_repack_kernel<uint16_t>, grid, 256, 0, 1, st, static_cast<const uint16_t*>(in), static_cast<uint16_t*>(out), rows, n, ld, ld_out, across);
}

template <typename T>
cudaError_t launch_dz(DzArgs& a, cudaStream_t st)
{
    const int cols = 128 / sizeof(T);
    // one CTA goes down up to 256 rows by itself: joining a cluster's sums takes longer than that
    const int64_t want = (a.rows + 255) / 256;
    a.parts = (int)(want > 8 ? 8 : want);
    const bool wide = aligned16(a.dy) && (a.ld * sizeof(T)) % 16 == 0 && (a.act == HPF_ACT_NONE || aligned16(a.z));
    const bool longer = a.db && a.rows > (int64_t)a.parts * 32 * kLongColumn;
    auto* kernel = longer ? (a.act == HPF_ACT_NONE ? (wide ? linear_dz_kernel<T, false, false, true> : linear_dz_kernel<T, true, false, true>)
                                                   : (wide ? linear_dz_kernel<T, false, true, true> : linear_dz_kernel<T, true, true, true>))
                          : (a.act == HPF_ACT_NONE ? (wide ? linear_dz_kernel<T, false, false, false> : linear_dz_kernel<T, true, false, false>)
                                                   : (wide ? linear_dz_kernel<T, false, true, false> : linear_dz_kernel<T, true, true, false>));
    return launch(kernel, (unsigned)((a.n + cols - 1) / cols * a.parts), 256, 0, a.parts, st, a);
}

// ---- scratch: status word | dz | x laid out again | W laid out again ----------------------------------------------------
struct Scratch {
    size_t dz, x, w, total;
};
// x_ok, w_ok, dy_ok: a tensor copy can address the rows as they lie
Scratch scratch_of(int64_t rows, int n_in, int n_out, int e, bool x_ok, bool w_ok, bool dy_ok, int act, bool bwd)
{
    Scratch s;
    s.dz = 256;
    s.x = s.dz + (bwd && (act != HPF_ACT_NONE || !dy_ok) ? up((size_t)rows * padded(n_out, e) * e, 256) : 0);
    s.w = s.x + (x_ok ? 0 : up((size_t)rows * padded(n_in, e) * e, 256));
    s.total = s.w + (w_ok ? 0 : up((size_t)n_out * padded(n_in, e) * e, 256));
    return s;
}
int check(int64_t rows, int32_t n_in, int32_t n_out, int64_t ld_x, int64_t ld_y, int32_t dtype, int32_t act)
{
    if (dtype != HPF_FP32 && dtype != HPF_BF16 && dtype != HPF_FP16) return api_fail(HPF_ERR_INVALID, "dtype must be HPF_FP32, HPF_BF16 or HPF_FP16");
    if (act < HPF_ACT_NONE || act > HPF_ACT_SILU) return api_fail(HPF_ERR_INVALID, "unknown activation");
    if (rows < 0 || n_in < 1 || n_out < 1 || ld_x < n_in || ld_y < n_out) return api_fail(HPF_ERR_INVALID, "rows < 0, an empty side, or a row stride below the row's length");
    if (rows > (1 << 30) || n_in > (1 << 30) || n_out > (1 << 30)) return api_fail(HPF_ERR_UNSUPPORTED, "more than 2^30 rows, inputs or outputs");
    // a tensor copy's strides end at 2^40 bytes, a launch at 2^31 tiles
    if (ld_x > (1ll << 36) || ld_y > (1ll << 36)) return api_fail(HPF_ERR_UNSUPPORTED, "a row stride above 2^36");
    const int64_t tm = (rows + kTileM - 1) / kTileM, ti = (n_in + 63) / 64, to = (n_out + 63) / 64;
    if (tm * ti > 0x3fffffff || tm * to > 0x3fffffff || (to + 1) * ti > 0x3fffffff) return api_fail(HPF_ERR_UNSUPPORTED, "more than 2^30 tiles");
    return HPF_OK;
}
bool value_aligned(const void* p, int e) { return (reinterpret_cast<uintptr_t>(p) & (e - 1)) == 0; }
bool any_of(const void* p, std::initializer_list<const void*> others)
{
    for (const void* o : others)
        if (p && p == o) return true;
    return false;
}
bool row_ok(const void* p, int64_t ld, int e) { return aligned16(p) && (ld * e) % 16 == 0; }

}  // namespace
}  // namespace hpf

using namespace hpf;

extern "C" int hpf_linear_scratch_bytes(int64_t rows, int32_t n_in, int32_t n_out, int64_t ld_x, int64_t ld_y, int32_t dtype, int32_t act, int32_t aligned, size_t* bytes)
{
    if (!bytes) return api_fail(HPF_ERR_INVALID, "null argument");
    const int bad = check(rows, n_in, n_out, ld_x, ld_y, dtype, act);
    if (bad != HPF_OK) return bad;
    const int e = dtype == HPF_FP32 ? 4 : 2;
    *bytes = scratch_of(rows, n_in, n_out, e, aligned && (ld_x * e) % 16 == 0, aligned && ((int64_t)n_in * e) % 16 == 0, aligned && (ld_y * e) % 16 == 0, act, true).total;
    return HPF_OK;
}

extern "C" int hpf_linear_fwd(const void* d_x, const void* d_w, const void* d_bias, const void* d_residual, void* d_y, void* d_z, int64_t rows,
                              int32_t n_in, int32_t n_out, int64_t ld_x, int64_t ld_y, int32_t dtype, int32_t act, void* d_scratch,
                              size_t scratch_bytes, void* stream)
{
    const int bad = check(rows, n_in, n_out, ld_x, ld_y, dtype, act);
    if (bad != HPF_OK) return bad;
    if (rows == 0) return HPF_OK;
    const int e = dtype == HPF_FP32 ? 4 : 2;
    if (!d_x || !d_w || !d_y || !d_scratch) return api_fail(HPF_ERR_INVALID, "null argument");
    for (const void* p : {d_x, d_w, d_bias, d_residual, static_cast<const void*>(d_y), static_cast<const void*>(d_z)})
        if (!value_aligned(p, e)) return api_fail(HPF_ERR_INVALID, "a tensor is not aligned to its type");
    const bool x_ok = row_ok(d_x, ld_x, e), w_ok = row_ok(d_w, n_in, e);
    const Scratch s = scratch_of(rows, n_in, n_out, e, x_ok, w_ok, true, act, false);
    if (!aligned16(d_scratch) || scratch_bytes < s.total) return api_fail(HPF_ERR_WORKSPACE, "scratch too small or misaligned (hpf_linear_scratch_bytes)");
    if (any_of(d_y, {d_x, d_w, d_bias}) || any_of(d_z, {d_x, d_w, d_bias, d_residual, d_y})) return api_fail(HPF_ERR_INVALID, "an output in an input's place");
    cudaError_t ce = conv_tc_init();
    if (ce != cudaSuccess) return api_cuda_fail(ce, "hpf_linear_fwd: set-up");
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    char* base = static_cast<char*>(d_scratch);
    Operand x{d_x, rows, n_in, ld_x, false}, w{d_w, n_out, n_in, n_in, false};
    if (!x_ok) { ce = repack(d_x, base + s.x, rows, n_in, ld_x, padded(n_in, e), e, st); x.p = base + s.x; x.ld = padded(n_in, e); }
    if (ce == cudaSuccess && !w_ok) { ce = repack(d_w, base + s.w, n_out, n_in, n_in, padded(n_in, e), e, st); w.p = base + s.w; w.ld = padded(n_in, e); }
    if (ce != cudaSuccess) return api_cuda_fail(ce, "hpf_linear_fwd: layout");
    GemmArgs g = {};
    g.act = act; g.out = d_y; g.z = d_z; g.bias = d_bias; g.residual = d_residual; g.ld = ld_y;
    g.status = reinterpret_cast<DeviceStatus*>(d_scratch);
    ce = gemm_any(g, x, w, rows, n_out, n_in, dtype, false, st);
    return ce == cudaSuccess ? HPF_OK : api_cuda_fail(ce, "hpf_linear_fwd");
}

extern "C" int hpf_linear_bwd(const void* d_dy, const void* d_z, const void* d_x, const void* d_w, void* d_dx, void* d_dw, void* d_dbias, int64_t rows,
                              int32_t n_in, int32_t n_out, int64_t ld_x, int64_t ld_y, int32_t dtype, int32_t act, int32_t grad_type,
                              void* d_scratch, size_t scratch_bytes, void* stream)
{
    const int bad = check(rows, n_in, n_out, ld_x, ld_y, dtype, act);
    if (bad != HPF_OK) return bad;
    if (grad_type != dtype && grad_type != HPF_FP32) return api_fail(HPF_ERR_INVALID, "grad_type must be dtype or HPF_FP32");
    const int e = dtype == HPF_FP32 ? 4 : 2, ge = grad_type == HPF_FP32 ? 4 : 2;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (!value_aligned(d_dw, ge) || !value_aligned(d_dbias, ge)) return api_fail(HPF_ERR_INVALID, "a tensor is not aligned to its type");
    if (rows == 0) {
        // an empty batch: sums of nothing
        cudaError_t ce = d_dw ? cudaMemsetAsync(d_dw, 0, (size_t)n_out * n_in * ge, st) : cudaSuccess;
        if (ce == cudaSuccess && d_dbias) ce = cudaMemsetAsync(d_dbias, 0, (size_t)n_out * ge, st);
        return ce == cudaSuccess ? HPF_OK : api_cuda_fail(ce, "hpf_linear_bwd: empty batch");
    }
    if (!d_dy || (d_dx && !d_w) || (d_dw && !d_x) || (act != HPF_ACT_NONE && !d_z) || !d_scratch) return api_fail(HPF_ERR_INVALID, "null argument");
    for (const void* p : {d_dy, d_z, d_x, d_w, static_cast<const void*>(d_dx)})
        if (!value_aligned(p, e)) return api_fail(HPF_ERR_INVALID, "a tensor is not aligned to its type");
    const bool x_ok = !d_dw || row_ok(d_x, ld_x, e), w_ok = !d_dx || row_ok(d_w, n_in, e), dy_ok = row_ok(d_dy, ld_y, e);
    const bool products = d_dx || d_dw;
    const Scratch s = scratch_of(rows, n_in, n_out, e, x_ok, w_ok, dy_ok || !products, products ? act : HPF_ACT_NONE, true);
    if (!aligned16(d_scratch) || scratch_bytes < s.total) return api_fail(HPF_ERR_WORKSPACE, "scratch too small or misaligned (hpf_linear_scratch_bytes)");
    if (any_of(d_dx, {d_dy, d_z, d_x, d_w, d_dw, d_dbias}) || any_of(d_dw, {d_dy, d_z, d_x, d_w, d_dbias}) || any_of(d_dbias, {d_dy, d_z, d_x, d_w}))
        return api_fail(HPF_ERR_INVALID, "an output in an input's place");
    cudaError_t ce = conv_tc_init();
    if (ce != cudaSuccess) return api_cuda_fail(ce, "hpf_linear_bwd: set-up");
    char* base = static_cast<char*>(d_scratch);
    DzArgs d = {};
    const bool own_dz = products && (act != HPF_ACT_NONE || !dy_ok);
    d.dy = d_dy; d.z = d_z; d.dz = own_dz ? base + s.dz : nullptr; d.db = d_dbias;
    d.rows = rows; d.ld = ld_y; d.ld_dz = padded(n_out, e); d.n = n_out; d.act = act; d.db_fp32 = grad_type == HPF_FP32;
    if (own_dz || d_dbias) {
        ce = dtype == HPF_FP32 ? launch_dz<float>(d, st) : dtype == HPF_BF16 ? launch_dz<__nv_bfloat16>(d, st) : launch_dz<__half>(d, st);
        if (ce != cudaSuccess) return api_cuda_fail(ce, "hpf_linear_bwd: dz");
    }
    const void* dz = own_dz ? base + s.dz : d_dy;
    const int64_t ld_dz = own_dz ? d.ld_dz : ld_y;
    GemmArgs g = {};
    g.status = reinterpret_cast<DeviceStatus*>(d_scratch);
    if (d_dx) {
        Operand a{dz, rows, n_out, ld_dz, false}, w{d_w, n_out, n_in, n_in, true};
        if (!w_ok) { ce = repack(d_w, base + s.w, n_out, n_in, n_in, padded(n_in, e), e, st); w.p = base + s.w; w.ld = padded(n_in, e); }
        g.out = d_dx; g.ld = ld_x;
        if (ce == cudaSuccess) ce = gemm_any(g, a, w, rows, n_in, n_out, dtype, false, st);
        if (ce != cudaSuccess) return api_cuda_fail(ce, "hpf_linear_bwd: dx");
    }
    if (d_dw) {
        Operand a{dz, rows, n_out, ld_dz, true}, x{d_x, rows, n_in, ld_x, true};
        if (!x_ok) { ce = repack(d_x, base + s.x, rows, n_in, ld_x, padded(n_in, e), e, st); x.p = base + s.x; x.ld = padded(n_in, e); }
        g.out = d_dw; g.ld = n_in;
        if (ce == cudaSuccess) ce = gemm_any(g, a, x, n_out, n_in, rows, dtype, grad_type == HPF_FP32, st);
        if (ce != cudaSuccess) return api_cuda_fail(ce, "hpf_linear_bwd: dW");
    }
    return HPF_OK;
}

extern "C" int hpf_linear_status(const void* d_scratch, int32_t* h_gave_up)
{
    if (!d_scratch || !h_gave_up) return api_fail(HPF_ERR_INVALID, "null argument");
    DeviceStatus s = {};
    const cudaError_t e = read_when_idle(&s, d_scratch, sizeof(s));
    if (e != cudaSuccess) return api_cuda_fail(e, "hpf_linear_status");
    *h_gave_up = s.code != 0;
    return HPF_OK;
}
