// bebop_tv_grad: the TV loss of row pairs with its gradient in the draft logits.
//
//   p, q = softmax(target / tau), softmax(draft / tau);  tv = sum max(0, p - q) = 1/2 sum |p - q|;  S = sum q 1[q <= p]
//   gradient of g tv in draft logit v:  -(g / tau) q_v (1[q_v <= p_v] - S)                              (Eq. tv_grad)
//
// The gradient jumps by q_v g / tau where q_v = p_v, so the comparison is made on logits: q_v <= p_v where
// z_p - z_q >= theta = (lse_p - lse_q) tau.  The difference of two logits is (almost) exact; what carries an error is
// theta, by the fp32 exponentials in the two sums.  A row pair that has a logit difference within the bound of that error is
// evaluated again with sums in double, so that every comparison is the one that 64 bits give.
//
// A CTA (a cluster of them, where there are fewer row pairs than SMs or rows are long) takes a row pair three times: the first time from DRAM, then out of L2.
//   pass 1  the rows' softmax sums
//   pass 2  sum |p - q|, S, the smallest |z_p - z_q - theta|
//   again   where that smallest distance is below the bound: the sums more exactly (33 us of the CTA's time at 151,936 tokens), by which the tokens that were open are decided
//   pass 3  the gradient
// 768 row pairs of 151,936 bf16: 264 us (0.41 of the copy rate; 241 where no comparison is open, 289 with three), 512 of 262,144: 281 to 341, 12 of 1,024 fp32: 5.6.  Some 36 instructions a pair of logits and its
// five exponentials bound it, with the meetings between passes; DRAM is busy in the first and the last pass.
#include "bebop_kernels.h"
#include "bebop_ring.cuh"

namespace bebop {

namespace {

struct TvGradArgs {
    RowArgs r;
    const float* grad_tv;
    float *tv, *s_aux;
    int32_t* row_status;
    unsigned char* grad;
    int64_t g_row_bytes;
    RingShape s;
    int expire;               // test hook: a wait counts as run out
};

// What passes 2 and 3 need of a row pair.
struct PairRef {
    float mp, mq;             // references
    float rho;                // S_p / S_q
    float theta;              // q <= p where z_p - z_q >= theta
    float near;               // distances below it are not certain
    double theta_d;           // theta
};

constexpr int kTvSlots = 2;
template <int DT> using TvRing = Ring<DT, 2, kTvSlots>;
struct __align__(16) TvSums { RSum p, q; };

// How far theta may be off, in units of tau.  Sums in fp32: every term carries an error of the order of 2^-24 (ex2.approx's bound is 2^-22) and of either sign, so
// that a sum is off by 2^-24 sqrt(sum p^2), where sum p^2 <= 1 / s as no term is above 1, and by what the exponents' roundings have in common.  kNearKappa times that and kNearFloor: on 73,728 row
// pairs (1,024 to 151,936 tokens, N(0, 1) to N(0, 6^2), three temperatures, both types) the largest error is 0.57 of it.
constexpr float kNearKappa = 3.6f, kNearFloor = 5e-8f;
__device__ __forceinline__ float near_fp32(const TvSums& t) { return kNearFloor + kNearKappa * 5.9604644775390625e-08f * (rsqrtf((float)t.p.s) + rsqrtf((float)t.q.s)); }
constexpr float kNearDouble = 1e-12f;                         // sums in double: 2.4e-15

// FAR: the references are logits.
template <bool FAR> __device__ __forceinline__ PairRef pair_ref(const RSum& p, const RSum& q, float tau, float near) {
    PairRef o;
    o.mp = p.m; o.mq = q.m;
    const double rho = p.s / q.s, unit = (double)tau * 0.6931471805599453;      // a logit's power of two
    o.rho = (float)rho;
    o.theta_d = (FAR ? 0.0 : ((double)p.m - (double)q.m) * unit) + log2(rho) * unit;      // (lse_p - lse_q) tau (FAR: less the references)
    o.theta = (float)o.theta_d;
    // the float difference of the logits and theta are off by half a step of theta each
    o.near = near * tau + (float)(2.384185791015625e-07 * fabs(o.theta_d));
    return o;
}

__device__ __forceinline__ float min3_abs(float a, float b, float c) {      // of the magnitudes (NaN counts for nothing)
    float d; asm("min.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d;
}
__device__ __forceinline__ float sign_of(float u) { return __uint_as_float(0x3f800000u | (__float_as_uint(u) & 0x80000000u)); }      // 1 or -1

// z_p - z_q - theta of two tokens (NaN: masked in both rows, q = 0).  EXACT: distances below `near` in double; FAR: all of them, and each logit less its row's
// largest first, as their difference may have no room for theta.
template <bool FAR> __device__ __forceinline__ float exact_above(float u, float p, float q, const PairRef& R) {
    if ((!FAR && fabsf(u) > R.near) || (p == -INFINITY && q == -INFINITY)) return u;
    const double d = FAR ? ((double)p - (double)R.mp) - ((double)q - (double)R.mq) - R.theta_d : (double)p - (double)q - R.theta_d;
    return d >= 0.0 ? fmaxf((float)d, 0.f) : fminf((float)d, -1e-45f);
}
template <bool FAR, bool EXACT> __device__ __forceinline__ float2 above(float p0, float p1, float q0, float q1, const PairRef& R) {
    float2 u = __fadd2_rn(minus2(make_float2(p0, p1), make_float2(q0, q1)), make_float2(-R.theta, -R.theta));
    if (EXACT) { u.x = exact_above<FAR>(u.x, p0, q0, R); u.y = exact_above<FAR>(u.y, p1, q1, R); }
    return u;
}
// Pass 2 of one vector pair: sum |p - q| S_p, the q that are not above p less the others, (EXACT) all q, the smallest distance.
struct PairAcc { float2 ab, ss, qs; float nearest; };
__device__ __forceinline__ PairAcc no_acc() { PairAcc A; A.ab = make_float2(0.f, 0.f); A.ss = A.qs = A.ab; A.nearest = INFINITY; return A; }
template <int DT, bool FAR, bool EXACT>
__device__ __forceinline__ void pair_vec(const uint4& xp, const uint4& xq, const PairRef& R, const RScale& c, PairAcc& A) {
    constexpr int VEC = Elem<DT>::VEC;
    float ep[VEC], eq[VEC], fp[VEC], fq[VEC];
    row_exp<DT, DT == 0, FAR>(xp, R.mp, c, ep);
    row_exp<DT, DT == 0, FAR>(xq, R.mq, c, eq);
    unpack<DT>(xp, fp); unpack<DT>(xq, fq);
    const float2 rh = make_float2(-R.rho, -R.rho);
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
        const float2 q = make_float2(eq[i], eq[i + 1]), u = above<FAR, EXACT>(fp[i], fp[i + 1], fq[i], fq[i + 1], R);
        A.nearest = min3_abs(u.x, u.y, A.nearest);
        const float2 r = __ffma2_rn(rh, q, make_float2(ep[i], ep[i + 1])), s = make_float2(sign_of(u.x), sign_of(u.y));
        A.ab = __ffma2_rn(r, s, A.ab);                       // (r has u's sign, but for roundings of its own size)
        A.ss = __ffma2_rn(q, s, A.ss);
        if (EXACT) A.qs = __fadd2_rn(A.qs, q);
    }
}
// Pass 3 of one vector pair: q times `below` where it is not above p, times `over` where it is.
template <int DT, bool FAR, bool EXACT>
__device__ __forceinline__ void grad_vec(const uint4& xp, const uint4& xq, const PairRef& R, const RScale& c, float below, float over, float* g) {
    constexpr int VEC = Elem<DT>::VEC;
    float eq[VEC], fp[VEC], fq[VEC];
    row_exp<DT, DT == 0, FAR>(xq, R.mq, c, eq);
    unpack<DT>(xp, fp); unpack<DT>(xq, fq);
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
        const float2 u = above<FAR, EXACT>(fp[i], fp[i + 1], fq[i], fq[i + 1], R);
        const float2 o = __fmul2_rn(make_float2(eq[i], eq[i + 1]), make_float2(u.x >= 0.f ? below : over, u.y >= 0.f ? below : over));
        g[i] = o.x; g[i + 1] = o.y;
    }
}

struct __align__(16) TvMass { double ab, ss, q; int near, pad; };
struct __align__(16) TvTwo { double a, b; };
constexpr int kTvOpen = 192;
struct TvOpen { float p, q, e, s; };                         // a token's logits, its exponential of the draft's, the sign it was given
struct TvGradShared {
    TvSums sum[kRingWarps], cta_sum[kRowsMaxCluster];
    TvMass mass[4][kRingWarps], cta_mass[4][kRowsMaxCluster];        // (pass 2, and three times more)
    TvTwo max[kRingWarps], cta_max[kRowsMaxCluster], exact[2][kRingWarps], cta_exact[2][kRowsMaxCluster];
    TvTwo finer[kRingWarps], cta_finer[kRowsMaxCluster];
    unsigned long long bar[kRingWarps][kTvSlots];
    int opens;                                               // tokens whose comparison is open: how many, the first of them,
    unsigned long long open_mass;                            // what they weigh (2^-44), the smallest and the largest difference of their logits (ordered)
    long long open_least, open_most;
    TvOpen open[kTvOpen];
};

__device__ __forceinline__ RSum merge_sum(RSum r, const RScale& c) {      // (in double: theta hangs on it)
    RSum o;
    o.m = ord2f(redux_max(f2ord(r.m)));
    o.bad = __reduce_or_sync(0xffffffffu, r.bad);
    o.s = warp_sum(r.s * ref_factor<false>(r.m, o.m, c));
    return o;
}
__device__ __forceinline__ TvMass merge_mass(const TvMass* s, int n) {
    const int lane = threadIdx.x & 31;
    TvMass m = {0.0, 0.0, 0.0, 0, 0};
    if (lane < n) m = s[lane];
    m.ab = warp_sum(m.ab); m.ss = warp_sum(m.ss); m.q = warp_sum(m.q);
    m.near = __any_sync(0xffffffffu, m.near);
    return m;
}


// The sums of a row pair whose comparisons are open, more exactly: the terms from 2^-7 of the largest on in double, the others (most, and light) by the series above,
// whose errors have no mean: of near_finer's bound, five to ten times below near_fp32's, the largest error on the row pairs above is 0.40.  A fifth of tv_exact's time.
template <int DT> __device__ __noinline__ void tv_finer(TvRing<DT>& held, TvGradShared& S, int left0, const RScale& scale, int rank, int C, TvSums& tot) {
    constexpr int VEC = Elem<DT>::VEC;
    const int lane = threadIdx.x & 31;
    TvRing<DT> ring = held;
    const RScale c = scale;
    const int down[2] = {(int)tot.p.m, (int)tot.q.m};
    const float least[2] = {series_least(tot.p.m, c), series_least(tot.q.m, c)};
    const float m[2] = {tot.p.m, tot.q.m};
    double d[2] = {0.0, 0.0};
    ring.chunks_of(false, nullptr, [&](const unsigned char* at, int from, int, bool) {
        const int rem = ring.bytes - from, left = left0 - (from >> 4) * VEC;
#pragma unroll 1
        for (int j = 0; j < kRingVecs && j * 512 < rem; ++j) {
            unsigned heavy = 0;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float f[VEC];
                unpack<DT>(TvRing<DT>::edge_vec(at, w, j, rem, left), f);
                float2 s = make_float2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < VEC; i += 2) {
                    float2 e = series_exp2(make_float2(f[i], f[i + 1]), c, least[w], down[w]);
                    if (e.x >= kHeavy) { heavy |= 1u << (w * VEC + i); e.x = 0.f; }
                    if (e.y >= kHeavy) { heavy |= 2u << (w * VEC + i); e.y = 0.f; }
                    s = __fadd2_rn(s, e);
                }
                d[w] += (double)(s.x + s.y);
            }
#pragma unroll 1
            for (; heavy; heavy &= heavy - 1) {
                const int i = __ffs(heavy) - 1, w = i / VEC;
                const unsigned char* const z = at + w * TvRing<DT>::PART + j * 512 + (i % VEC) * (16 / VEC);
                const float f = DT == 0 ? *reinterpret_cast<const float*>(z) : __uint_as_float((unsigned)*reinterpret_cast<const unsigned short*>(z) << 16);
                const double e = q_exp2(row_arg<false>(f, w ? m[1] : m[0], c), g_pow2_64);
                if (w) d[1] += e; else d[0] += e;
            }
        }
    });
    held = ring;
    const TvTwo s = meet(S.finer, S.cta_finer, TvTwo{warp_sum(d[0]), warp_sum(d[1])}, C, rank, [&](const TvTwo* s, int n) {
        return TvTwo{warp_sum(lane < n ? s[lane].a : 0.0), warp_sum(lane < n ? s[lane].b : 0.0)};
    });
    tot.p.s = s.a; tot.q.s = s.b;
}
// (4 2^-24 sqrt(sum p^2) over the light terms, none of which is above 2^-7)
__device__ __forceinline__ float near_finer(const TvSums& t) { return 6e-9f + 2.1073424255e-08f * (rsqrtf((float)t.p.s) + rsqrtf((float)t.q.s)); }

// ... and all of them in double.  FAR: around the rows' largest logits, which are found first.
template <int DT, bool FAR> __device__ __noinline__ void tv_exact(TvRing<DT>& ring, TvGradShared& S, int left0, const RScale& c, int rank, int C, TvSums& tot) {
    constexpr int VEC = Elem<DT>::VEC;
    const int lane = threadIdx.x & 31;
    if (FAR) {
        float mp = -INFINITY, mq = -INFINITY;
        ring.pass_small(left0, false, nullptr, [&](int, const uint4* x, auto) { mp = fmaxf(mp, vec_max<DT>(x[0])); mq = fmaxf(mq, vec_max<DT>(x[1])); }, NoHook());
        mp = ord2f(redux_max(f2ord(mp))); mq = ord2f(redux_max(f2ord(mq)));
        const TvTwo m = meet(S.max, S.cta_max, TvTwo{(double)mp, (double)mq}, C, rank, [&](const TvTwo* s, int n) {
            const float a = lane < n ? (float)s[lane].a : -INFINITY, b = lane < n ? (float)s[lane].b : -INFINITY;
            return TvTwo{(double)ord2f(redux_max(f2ord(a))), (double)ord2f(redux_max(f2ord(b)))};
        });
        tot.p.m = (float)m.a; tot.q.m = (float)m.b;
    }
    double d[2] = {0.0, 0.0};
    ring.pass_small(left0, false, nullptr, [&](int, const uint4* x, auto) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const float m = w ? tot.q.m : tot.p.m;
            float f[VEC];
            unpack<DT>(x[w], f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) d[w] += q_exp2(row_arg<FAR>(f[i], m, c), g_pow2_64);
        }
    }, NoHook());
    constexpr int k = FAR ? 1 : 0;
    const TvTwo s = meet(S.exact[k], S.cta_exact[k], TvTwo{warp_sum(d[0]), warp_sum(d[1])}, C, rank, [&](const TvTwo* s, int n) {
        return TvTwo{warp_sum(lane < n ? s[lane].a : 0.0), warp_sum(lane < n ? s[lane].b : 0.0)};
    });
    tot.p.s = s.a; tot.q.s = s.b;
}

// order-preserving whole number of a double that is a number
__device__ __forceinline__ long long dord(double x) { const long long b = __double_as_longlong(x); return b ^ ((b >> 63) & 0x7fffffffffffffffLL); }

// The tokens of a chunk whose comparison is open.
template <int DT> __device__ __noinline__ void tv_collect(TvGradShared& S, const unsigned char* b, int rem, int left, const PairRef& R, const RScale& c) {
    constexpr int VEC = Elem<DT>::VEC;
    for (int j = 0; j < kRingVecs && j * 512 < rem; ++j) {
        const uint4 xp = TvRing<DT>::edge_vec(b, 0, j, rem, left), xq = TvRing<DT>::edge_vec(b, 1, j, rem, left);
        float eq[VEC], fp[VEC], fq[VEC];
        row_exp<DT, DT == 0, false>(xq, R.mq, c, eq);
        unpack<DT>(xp, fp); unpack<DT>(xq, fq);
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
            const float2 u = above<false, false>(fp[i], fp[i + 1], fq[i], fq[i + 1], R);
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (fabsf(k ? u.y : u.x) <= R.near) {
                    const int at = atomicAdd(&S.opens, 1);
                    if (at < kTvOpen) S.open[at] = {fp[i + k], fq[i + k], eq[i + k], sign_of(k ? u.y : u.x)};
                    const long long d = dord((double)fp[i + k] - (double)fq[i + k]);
                    atomicMin(&S.open_least, d); atomicMax(&S.open_most, d);
                    atomicAdd(&S.open_mass, (unsigned long long)((double)eq[i + k] * 0x1p44));
                }
        }
    }
}

}  // namespace

template <int DT>
__global__ void __launch_bounds__(32 * kRingWarps, 1) k_tv_grad(const __grid_constant__ TvGradArgs a) {
    constexpr int VEC = Elem<DT>::VEC;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ TvGradShared S;
    const RowArgs& R = a.r;
    const int C = a.s.C, sv = a.s.sv;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    const int rank = (int)cluster_rank(), clusters = a.s.clusters;
    const int v0 = rank * sv, nv = max(min(sv, R.nvec - v0), 0), per = run_length(nv, nw), wa = min(warp * per, nv), len = min(per, nv - wa);
    const int left0 = R.V - (v0 + wa) * VEC;                // tokens from the warp's first vector on
    TvRing<DT> ring;
    ring.init(smem + (size_t)warp * TvRing<DT>::BYTES, S.bar[warp], len, left0);
    // (programmatic dependent launch: nothing of the caller's memory is touched until the grid before this one is through)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const auto run_at = [&](int unit, const unsigned char** at) {
        at[0] = reinterpret_cast<const unsigned char*>(row_ptr(R, unit, 0)) + (int64_t)(v0 + wa) * 16;
        at[1] = reinterpret_cast<const unsigned char*>(row_ptr(R, unit, R.K + 1)) + (int64_t)(v0 + wa) * 16;
    };
    int u = (int)(blockIdx.x / (unsigned)C);
    float next_tau = tau_of(R, u), next_g = a.grad_tv ? a.grad_tv[u] : 1.f;
    run_at(u, ring.at);
    ring.first();
    if (C > 1) cluster_sync();                              // every CTA of the cluster has started
#pragma unroll 1
    for (; u < R.B; u += clusters) {
        const float tau = next_tau, g = next_g;
        const RScale c = rows_scale(tau);
        const bool more = u + clusters < R.B;
        if (more) { next_tau = tau_of(R, u + clusters); if (a.grad_tv) next_g = a.grad_tv[u + clusters]; }      // (asked for a row pair ahead)
        unsigned char* const grow = a.grad + (int64_t)u * a.g_row_bytes + (int64_t)(v0 + wa) * 16;      // the warp's run of the gradient
        const bool first = rank == 0 && threadIdx.x == 0;
        // ---- pass 1
        typename TvRing<DT>::Sum rs[2];
        ring.template sums<DT == 0>(left0, false, nullptr, c, rs, NoHook());
        TvSums tot;
        tot.p.s = warp_sum(rs[0].s); tot.q.s = warp_sum(rs[1].s);
        tot.p.m = rs[0].e == E_EMPTY ? -INFINITY : (float)rs[0].e; tot.q.m = rs[1].e == E_EMPTY ? -INFINITY : (float)rs[1].e;
        tot.p.bad = (rs[0].bad ? 1 : 0) | (a.expire || ring.failed ? 2 : 0); tot.q.bad = rs[1].bad ? 1 : 0;
        if (threadIdx.x == 0) { S.opens = 0; S.open_mass = 0; S.open_least = LLONG_MAX; S.open_most = LLONG_MIN; }                    // (nobody looks at the last unit's any more: a meeting lies behind)
        tot = meet(S.sum, S.cta_sum, tot, C, rank, [&](const TvSums* s, int n) {
            TvSums o, x;
            x.p = x.q = no_sum();
            if (lane < n) x = s[lane];
            o.p = merge_sum(x.p, c); o.q = merge_sum(x.q, c);
            return o;
        });
        int st = sum_status(tot.p) | sum_status(tot.q);
        if (st & ST_WAIT) st = ST_WAIT;
        else if (!tau_ok(tau)) st = ST_BAD_TEMP;
        const unsigned char* next_at[2] = {nullptr, nullptr};
        if (more) run_at(u + clusters, next_at);
        PairRef ref = pair_ref<false>(tot.p, tot.q, tau, near_fp32(tot));
        double tv = 0.0, s_aux = 0.0, scale = 0.0;
        const bool far = !st && (far_exponent((int)tot.p.m) || far_exponent((int)tot.q.m));
        bool again = far, wide = false;
        if (st) ring.pass_small(left0, false, nullptr, [](int, const uint4*, auto) {}, NoHook());       // (the same in every CTA)
        else {
            // ---- pass 2
            PairAcc A = no_acc();
            double s_ab = 0.0, s_ss = 0.0, s_qs = 0.0;
            int n = 0, open = 0;
            const auto spill = [&] {
                s_ab += (double)(A.ab.x + A.ab.y); s_ss += (double)(A.ss.x + A.ss.y); s_qs += (double)(A.qs.x + A.qs.y);
                A = no_acc();
                n = 0;
            };
            const auto part = [&] {
                TvMass m;
                m.ab = warp_sum(s_ab); m.ss = warp_sum(s_ss); m.q = wide ? warp_sum(s_qs) : 0.0; m.pad = 0;
                m.near = open;
                return m;
            };
            ring.pass(left0, false, nullptr, [&](int, const uint4* x, auto) { pair_vec<DT, false, false>(x[0], x[1], ref, c, A); }, [&](const unsigned char* b, int from) {
                if (__any_sync(0xffffffffu, A.nearest <= ref.near)) {
                    tv_collect<DT>(S, b, ring.bytes - from, left0 - (from >> 4) * VEC, ref, c);
                    open = 1;
                    A.nearest = INFINITY;
                }
                if (++n == 4) spill();
            });
            spill();
            TvMass mass = meet(S.mass[0], S.cta_mass[0], part(), C, rank, merge_mass);
            // ---- and again where a comparison is not certain, or a row FAR: the sums in double, by which the comparisons that were open are decided ...
            again = far || mass.near;
            int wide_too = far;
            if (again && !far) {
                const float near = ref.near;
                for (int level = 0; level < 2; ++level) {
                    TvRing<DT> r2 = ring;                  // (by a copy, so that the ring itself stays in registers)
                    TvSums exact = tot;
                    if (level == 0) tv_finer<DT>(r2, S, left0, c, rank, C, exact); else tv_exact<DT, false>(r2, S, left0, c, rank, C, exact);
                    ring = r2;
                    ref = pair_ref<false>(exact.p, exact.q, tau, 0.f);
                    ref.near = near;
                    const double still = (double)(level == 0 ? near_finer(exact) : kNearDouble) * (double)tau;
                    TvMass m = {0.0, 0.0, 0.0, 0, 0};
                    const int opens = S.opens;
                    long long moved = 0;                    // (whole numbers: the tokens' order in the list does not matter)
                    // (more than the list holds: on a grid of bf16 logits all at one difference, and decided alike)
                    const bool alike = opens > kTvOpen && S.open_least == S.open_most;
                    m.near = opens > kTvOpen && !alike;
                    for (int i = threadIdx.x; i < (alike ? 1 : min(opens, kTvOpen)); i += blockDim.x) {
                        const TvOpen o = S.open[i];
                        const double d = (double)o.p - (double)o.q - ref.theta_d;
                        if (fabs(d) <= still) m.near = 1;
                        const long long e = alike ? (long long)S.open_mass : (long long)((double)o.e * 0x1p44);
                        if ((d >= 0.0) != (o.s > 0.f)) moved += d >= 0.0 ? e : -e;
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) moved += __shfl_xor_sync(0xffffffffu, moved, o);
                    m.ss = (double)moved * 0x1p-43; m.near = __any_sync(0xffffffffu, m.near);
                    m = meet(S.mass[1 + level], S.cta_mass[1 + level], m, C, rank, merge_mass);
                    wide_too = m.near;
                    if (!m.near || level == 1) { mass.ss += m.ss; break; }
                }
            }
            // ... and, where even that leaves it open (equal rows, rows of one token, many ties), or FAR: around the rows' largest logits, pass 2 too.
            if (wide_too) {
                wide = true;
                TvRing<DT> r2 = ring;
                tv_exact<DT, true>(r2, S, left0, c, rank, C, tot);
                ring = r2;
                ref = pair_ref<true>(tot.p, tot.q, tau, 0.f);
                s_ab = s_ss = s_qs = 0.0;
                ring.pass_small(left0, false, nullptr, [&](int, const uint4* x, auto) { pair_vec<DT, true, true>(x[0], x[1], ref, c, A); }, [&](const unsigned char*, int) { spill(); });
                open = 0;
                mass = meet(S.mass[3], S.cta_mass[3], part(), C, rank, merge_mass);
            }
            const double q = wide ? mass.q : tot.q.s;       // (wide: by the same terms' sum, so that S is 1 where no q is above p)
            tv = fmin(fmax(0.5 * mass.ab / tot.p.s, 0.0), 1.0);
            s_aux = fmin(fmax(0.5 * (mass.ss + q) / q, 0.0), 1.0);
            scale = (double)g / ((double)tau * q);
        }
        if (first) {
            if (a.tv) a.tv[u] = (float)tv;
            if (a.s_aux) a.s_aux[u] = (float)s_aux;
            if (a.row_status) a.row_status[u] = st;
        }
        // ---- pass 3
        const float below = (float)(-scale * (1.0 - s_aux)), over = (float)(scale * s_aux);
        const auto put = [&](int at, const float* o, auto whole) {
            if (decltype(whole)::value) store_whole<DT>(grow + at, 0, o);
            else if (at < ring.bytes) store_vec<DT>(grow, at >> 4, left0, o);
        };
        const unsigned char* const* const next = more ? next_at : nullptr;
        if (st) ring.pass_small(left0, true, next, [&](int at, const uint4*, auto whole) {
            float o[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) o[i] = 0.f;
            put(at, o, whole);
        }, NoHook());
        else if (wide) ring.pass_small(left0, true, next, [&](int at, const uint4* x, auto whole) { float o[VEC]; grad_vec<DT, true, true>(x[0], x[1], ref, c, below, over, o); put(at, o, whole); }, NoHook());
        else if (again) ring.pass_small(left0, true, next, [&](int at, const uint4* x, auto whole) { float o[VEC]; grad_vec<DT, false, true>(x[0], x[1], ref, c, below, over, o); put(at, o, whole); }, NoHook());
        else ring.pass(left0, true, next, [&](int at, const uint4* x, auto whole) { float o[VEC]; grad_vec<DT, false, false>(x[0], x[1], ref, c, below, over, o); put(at, o, whole); }, NoHook());
    }
    if (C > 1) cluster_sync();                              // (nobody stores into a CTA that has left)
}

cudaError_t tv_grad(const RowArgs& r, const float* grad_tv, float* tv, float* s_aux, int32_t* row_status, void* grad, int64_t ld_grad,
                    cudaStream_t stream) {
    TvGradArgs a;
    a.r = r; a.grad_tv = grad_tv; a.tv = tv; a.s_aux = s_aux; a.row_status = row_status;
    a.grad = static_cast<unsigned char*>(grad);
    a.g_row_bytes = ld_grad * (r.dt == 0 ? 4 : 2);
    a.expire = take_expire_wait() ? 1 : 0;
    const auto none = [](int) { return 0; };
    cudaError_t e = r.dt == 0 ? ring_shape<k_tv_grad<0>>(r.B, 2, r.nvec, TvRing<0>::BYTES, 0, none, a.s) : ring_shape<k_tv_grad<1>>(r.B, 2, r.nvec, TvRing<1>::BYTES, 0, none, a.s);
    if (e != cudaSuccess) return e;
    return r.dt == 0 ? ring_launch<k_tv_grad<0>>(a, a.s, stream) : ring_launch<k_tv_grad<1>>(a, a.s, stream);
}

}  // namespace bebop
