// What the kernels that take a row (a row pair) by a CTA or a cluster of them and need no other launch share: exponentials,
// softmax sums and how they are merged, the launch.
//
// A softmax sum is (m, s) with s = sum 2^(x c - m), c = log2(e) / tau: m is a whole number near the largest x c, so that sums are merged by exact
// powers of two, and fma(x, c, -m) carries one rounding of a small number.  m is a reference, not the maximum: the exponent
// of the largest term, or of a larger one.  Rows whose largest |x c| lies beyond 4 million -- nothing but a mask of -1e9 or of the type's lowest
// value, a temperature next to zero -- are FAR: they are evaluated once more with the difference in front, 2^((x - m) c), m a logit, which holds for
// finite logits of any size and costs an addition per two logits more.
#pragma once
#include "bebop_chunk.cuh"

namespace bebop {

namespace {

constexpr int kRowsMaxCluster = 16;
constexpr int kRowsSmem = 232448 - 12288;     // dynamic shared memory of a CTA, at most (the rest: static tables)
constexpr uint32_t kRowsSpin = 1u << 22;

// log2(e) / tau, finite whatever tau, so that 0 * c is 0: to double precision (d), as the nearest float (c), and as a sum of floats hi + lo with lo
// above 0, so that a masked logit's -inf stays -inf in both products.
struct RScale { double d; float c, hi, lo; };
__device__ __forceinline__ RScale rows_scale(float tau) {
    RScale r;
    r.d = fmin(1.4426950408889634 / (tau_ok(tau) ? (double)tau : 1.0), 3e38);
    r.c = (float)r.d;
    r.hi = __int_as_float(__float_as_int(__double2float_rd(r.d)) - 1);
    r.lo = fmaxf((float)(r.d - (double)r.hi), 1e-45f);
    return r;
}

struct __align__(16) RSum { double s; float m; int bad; };      // bad: bit 0 a NaN or +inf, bit 1 a wait that gave up
__device__ __forceinline__ RSum no_sum() { RSum r; r.s = 0.0; r.m = -INFINITY; r.bad = 0; return r; }

constexpr float kRowsFar = (float)kFarExp;     // (where chunk_exponent ends)
__device__ __forceinline__ bool sum_far(float m) { return fabsf(m) >= kRowsFar && m > -INFINITY; }
// the factor that takes a sum around a to the reference b >= a; 0 where a is -inf
template <bool FAR> __device__ __forceinline__ double ref_factor(float a, float b, const RScale& c) {
    if (FAR) return a == -INFINITY ? 0.0 : exp2(fmax(((double)a - (double)b) * c.d, -1100.0));
    return pow2d((int)fmaxf(a - b, -1100.f));                // (also: -inf, and -inf - -inf, which max takes as -1100)
}
// the exponent of logit x around reference m
template <bool FAR> __device__ __forceinline__ double row_arg(float x, float m, const RScale& c) { return FAR ? ((double)x - (double)m) * c.d : fma((double)x, c.d, -(double)m); }

// The slice of a row: vectors [v0, v0 + nv) of it, where the caller has them.
struct Slice { const unsigned char* p; int v0, nv, V; };

// vector vi of a slice; what lies beyond the slice or the vocabulary reads as -inf
template <int DT>
__device__ __forceinline__ uint4 row_vec(const Slice& s, int vi) {
    constexpr int VEC = Elem<DT>::VEC;
    uint4 x = neg_inf_vec<DT>();
    if (vi < s.nv) {
        x = ldg16_stream(s.p + (size_t)vi * 16);
        const int left = s.V - (s.v0 + vi) * VEC;
        if (left < VEC) mask_tail<DT>(x, left);
    }
    return x;
}

// The exponentials of a vector's logits around reference m, two at a time; LOW: with the low part of c.
template <int DT, bool LOW, bool FAR>
__device__ __forceinline__ void row_exp(const uint4& raw, float m, const RScale& c, float* e) {
    constexpr int VEC = Elem<DT>::VEC;
    float f[VEC];
    unpack<DT>(raw, f);
    const float ch = LOW ? c.hi : c.c;
    const float2 m2 = make_float2(-m, -m), c2 = make_float2(ch, ch), l2 = make_float2(c.lo, c.lo);
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
        float2 x = make_float2(f[i], f[i + 1]), t;
        if (FAR) { x = __fadd2_rn(x, m2); t = __fmul2_rn(x, c2); } else t = __ffma2_rn(x, c2, m2);
        if (LOW) t = __ffma2_rn(x, l2, t);
        e[i] = ex2f(t.x);
        e[i + 1] = ex2f(t.y);
    }
}

__device__ __forceinline__ float2 minus2(float2 a, float2 b) { return __ffma2_rn(b, make_float2(-1.f, -1.f), a); }
__device__ __forceinline__ float series_least(float m, const RScale& c) { return (m - 120.f) / c.hi; }
// 2^(x c - m) of two logits in fp32, `down` = m, by the series of 2^f, |f| <= 1/2, to the seventh power (the next term is 5e-9 at most, 6e-10 in the mean): unlike ex2.approx's, its errors
// are roundings without a mean that would stay in a sum of thousands.  Logits below `least` count as that: next to nothing.
__device__ __forceinline__ float2 series_exp2(float2 x, const RScale& c, float least, int down) {
    // x c = n + f first, f exactly but for 2^-26: the exponent loses nothing to the size of x c - m
    const float2 magic = make_float2(12582912.f, 12582912.f), hi = make_float2(c.hi, c.hi), lo = make_float2(c.lo, c.lo);
    x.x = fmaxf(x.x, least); x.y = fmaxf(x.y, least);
    const float2 r = __ffma2_rn(x, hi, magic), f = __ffma2_rn(x, lo, __ffma2_rn(x, hi, minus2(magic, r)));
    const auto k = [](float a) { return make_float2(a, a); };
    float2 p = __ffma2_rn(f, k(1.5252734e-5f), k(1.5403530e-4f));      // ln2^7 / 7!, ln2^6 / 6!, ...
    p = __ffma2_rn(f, p, k(1.3333558e-3f));
    p = __ffma2_rn(f, p, k(9.6181291e-3f));
    p = __ffma2_rn(f, p, k(5.5504109e-2f));
    p = __ffma2_rn(f, p, k(2.4022651e-1f));
    p = __ffma2_rn(f, p, k(6.9314718e-1f));
    p = __ffma2_rn(f, p, k(1.f));
    return make_float2(__int_as_float(__float_as_int(p.x) + ((__float_as_int(r.x) - down) << 23)), __int_as_float(__float_as_int(p.y) + ((__float_as_int(r.y) - down) << 23)));
}
constexpr float kHeavy = 0.0078125f;           // terms from here on are taken in double beside the series

// Sum over a warp of numbers >= 0 (the same bits in every lane), exact to 2^-24 of each and 2^-40 of the largest: a power of two takes the largest into [1, 2),
// then they are added as integers.  A tenth of the latency of five steps of double shuffles and additions.
__device__ __forceinline__ double warp_sum_pos(double s) {
    const float f = (float)s;
    const int top = redux_max(__float_as_int(f)) & 0x7f800000;
    const float scale = __int_as_float(0x7f000000 - max(top, 0x00800000));      // 2^(127 - e)
    return warp_sum_fixed(f * scale) * __hiloint2double((1023 - 127 + (max(top, 0x00800000) >> 23)) << 20, 0);
}

// Sums of the lanes merged over a warp (the same bits in every lane).
template <bool FAR> __device__ __forceinline__ RSum warp_merge(RSum r, const RScale& c) {
    RSum o;
    o.m = ord2f(redux_max(f2ord(r.m)));
    o.bad = __reduce_or_sync(0xffffffffu, r.bad);
    o.s = warp_sum_pos(r.s * ref_factor<FAR>(r.m, o.m, c));
    return o;
}

// A warp's sum of vectors [a, b) of a slice around its largest logit (FAR), in double, from memory; but for the tokens that `skip`, the bits of a vector, names.
template <int DT, typename F> __device__ __noinline__ RSum far_sum(const Slice& sl, int a, int b, const RScale& c, F skip) {
    constexpr int VEC = Elem<DT>::VEC;
    const int lane = threadIdx.x & 31;
    float top = -INFINITY;
    RSum r = no_sum();
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
        for (int v = a + lane; v < b; v += 32) {
            const uint32_t e = skip(v);
            float f[VEC];
            unpack<DT>(row_vec<DT>(sl, v), f);
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (!(e >> i & 1)) { if (pass == 0) top = fmaxf(top, f[i]); else r.s += q_exp2(row_arg<true>(f[i], r.m, c), g_pow2_64); }
        }
        if (pass == 0) r.m = ord2f(redux_max(f2ord(top)));
        if (r.m == -INFINITY) break;
    }
    r.s = warp_sum(r.s);
    return r;
}

__device__ __forceinline__ int sum_status(const RSum& r) {
    if (r.bad & 2) return ST_WAIT;
    if (r.bad & 1) return ST_NONFINITE;
    return r.m == -INFINITY ? ST_EMPTY : 0;
}

// gradient vector `vi` of a row (in its own type) from floats
template <int DT> __device__ __forceinline__ void store_whole(unsigned char* row, int vi, const float* f) {
    const uint4 x = pack<DT>(f);
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" :: "l"(row + (size_t)vi * 16), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
// ... that may end beyond the vocabulary: by its elements
template <int DT>
__device__ __forceinline__ void store_vec(unsigned char* row, int vi, int V, const float* f) {
    constexpr int VEC = Elem<DT>::VEC;
    const int left = V - vi * VEC;
    if (left >= VEC) { store_whole<DT>(row, vi, f); return; }
#pragma unroll
    for (int i = 0; i < VEC; ++i) if (i < left) {
        if (DT == 0) reinterpret_cast<float*>(row)[(size_t)vi * VEC + i] = f[i];
        else reinterpret_cast<unsigned short*>(row)[(size_t)vi * VEC + i] = (unsigned short)(pack_bf16x2(f[i], 0.f) & 0xffffu);
    }
}

// ------------------------------------------------------------------ host
int rows_sms() {
    static int cached[64] = {0};
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64 && cached[dev]) return cached[dev];
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return 0; }
    if (dev >= 0 && dev < 64) cached[dev] = n;
    return n;
}
template <auto kernel> cudaError_t rows_ready() {
    static bool done[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64 && done[dev]) return cudaSuccess;
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsSmem)) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) done[dev] = true;
    return cudaSuccess;
}
// `clusters` clusters of C CTAs
template <auto kernel, typename A> cudaError_t rows_launch(const A& args, int clusters, int C, int threads, int bytes, cudaStream_t stream) {
    cudaError_t e = rows_ready<kernel>();
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)clusters * (unsigned)C); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = bytes; cfg.stream = stream;
    cfg.attrs = C == 1 ? attr + 1 : attr; cfg.numAttrs = C == 1 ? 1 : 2;      // (a plain grid starts sooner than one of clusters)
    return cudaLaunchKernelEx(&cfg, kernel, args);
}

}  // namespace

}  // namespace bebop
