// bebop_tv_grad: the TV loss of row pairs with its gradient in the draft logits, one cluster of CTAs per row pair.
//
//   p, q = softmax(target / tau), softmax(draft / tau);  tv = sum max(0, p - q) = 1/2 sum |p - q|;  S = sum q 1[q <= p]
//   gradient of g tv in draft logit v:  -(g / tau) q_v (1[q_v <= p_v] - S)                              (Eq. tv_grad)
//
// The gradient jumps by q_v g / tau where q_v = p_v, so the comparison is made on logits: q_v <= p_v where
// z_p - z_q >= theta = (lse_p - lse_q) tau.  The difference of two logits is (almost) exact; what carries an error is
// theta, by the fp32 exponentials in the two sums.  A row pair that has a logit difference within the bound of that error is
// evaluated again with sums in double, so that every comparison is the one that 64 bits give.
//
//   pass 1  the rows' softmax sums; the CTAs exchange theirs
//   pass 2  sum |p - q|, S, the smallest |z_p - z_q - theta|; in place of the two logits their q with the comparison as its sign
//           (a vector of each row gives 32 bytes: eight floats for bf16, in place of the draft's alone for fp32); exchange
//   again   where that smallest distance is below the bound: sums in double from memory, and pass 2 once more
//   pass 3  the gradient
#include "bebop_kernels.h"
#include "bebop_rows.cuh"

namespace bebop {

namespace {

struct TvMass { double absum, signed_q, q; };        // sum |e_p - rho e_q|, sum of the signed and of the plain e_q

struct TvGradArgs {
    RowArgs r;
    const float* grad_tv;
    float *tv, *s_aux;
    int32_t* row_status;
    unsigned char* grad;
    int64_t g_row_bytes;
    RowsShape s;
    int expire;               // test hook: the wait for the rows counts as run out
};

struct TvGradShared {
    RSum warp[2][kRowsMaxWarps], cta[2][kRowsMaxCluster];
    double mass[3][kRowsMaxWarps], cta_mass[3][kRowsMaxCluster];
    double wsum[2][kRowsMaxWarps], cta_sum[2][kRowsMaxCluster];
    int near[kRowsMaxWarps], cta_near[kRowsMaxCluster];
    unsigned long long bar[kRowsMaxWarps];
    double tab[64];
    int failed;
};

// What passes 2 and 3 need of a row pair.
struct PairRef {
    float mp, mq;             // references
    float rho_hi, rho_lo;     // S_p / S_q
    float theta;              // q <= p where z_p - z_q >= theta
    float near;               // distances below this are not certain
    double theta_d;           // theta
};

__device__ __forceinline__ PairRef pair_ref(const RSum& p, const RSum& q, const RScale& c, float tau) {
    PairRef o;
    o.mp = p.m; o.mq = q.m;
    const double rho = p.s / q.s;
    o.rho_hi = (float)rho; o.rho_lo = (float)(rho - (double)o.rho_hi);
    const double off = log2(rho) / c.d;                          // (lse_p - lse_q) tau - (mp - mq)
    o.theta_d = ((double)p.m - (double)q.m) + off;
    o.theta = (float)o.theta_d;
    // the sums' relative error, taken as 2^-22 each (ex2.approx's bound for every term; the sums' own is a tenth of it), moves theta by tau
    // times that; the float difference of the logits and theta are off by half a step of theta each.  Beyond a float's range: always in double.
    o.near = fabs(o.theta_d) < 1e38 ? (float)(4.76837158203125e-07 / (c.d * 0.6931471805599453) + 2.384185791015625e-07 * fabs(o.theta_d)) : INFINITY;
    return o;
}

// One vector pair: signed q (its sign: whether q > p), and the sums.  `exact`: distances below `near` are decided in double.
template <int DT>
__device__ __forceinline__ void pair_vec(const uint4& xp, const uint4& xq, const PairRef& R, const RScale& c, bool exact, float* sq,
                                         float& absum, float& ssum, float& qsum, float& nearest) {
    constexpr int VEC = Elem<DT>::VEC;
    float fp[VEC], fq[VEC], ep[VEC], eq[VEC];
    unpack<DT>(xp, fp); unpack<DT>(xq, fq);
    row_exp<DT, DT == 0>(xp, R.mp, c, ep);
    row_exp<DT, DT == 0>(xq, R.mq, c, eq);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        float u = (fp[i] - fq[i]) - R.theta;                        // (NaN: masked in both rows, q = 0)
        if (exact && !(fabsf(u) > R.near)) u = (double)fp[i] - (double)fq[i] >= R.theta_d ? 1.f : -1.f;
        nearest = fminf(nearest, fabsf(u));
        const float r = fmaf(-R.rho_lo, eq[i], fmaf(-R.rho_hi, eq[i], ep[i]));
        absum += fabsf(r);
        sq[i] = u >= 0.f ? eq[i] : -eq[i];
        ssum += sq[i];
        qsum += eq[i];
    }
}

template <int DT> __device__ __forceinline__ void grad_vec(const float* sq, float below, float above, float* g) {
#pragma unroll
    for (int i = 0; i < Elem<DT>::VEC; ++i) g[i] = __float_as_int(sq[i]) >= 0 ? sq[i] * below : sq[i] * above;
}

}  // namespace

template <int DT, bool RES>
__global__ void __launch_bounds__(256, 2) k_tv_grad(const __grid_constant__ TvGradArgs a) {
    constexpr int VEC = Elem<DT>::VEC;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ TvGradShared S;
    const RowArgs& R = a.r;
    const int C = a.s.C, sv = a.s.sv;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = blockDim.x >> 5;
    const int rank = (int)cluster_rank(), b = (int)(blockIdx.x / (unsigned)C);
    cluster_arrive();                                       // (waited for before the first store into another CTA)
    if (lane == 0) { mbar_init(&S.bar[warp], 1); asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
    if (tid < 64) S.tab[tid] = g_pow2_64[tid];
    if (tid == 0) S.failed = a.expire;
    __syncthreads();
    // (programmatic dependent launch: nothing of the caller's memory is touched until the grid before this one is through)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const float tau = tau_of(R, b);
    const RScale c = rows_scale(tau);
    const int v0 = rank * sv, nv = max(min(sv, R.nvec - v0), 0);
    const unsigned char* const gp = reinterpret_cast<const unsigned char*>(row_ptr(R, b, 0)) + (int64_t)v0 * 16;
    const unsigned char* const gq = reinterpret_cast<const unsigned char*>(row_ptr(R, b, R.K + 1)) + (int64_t)v0 * 16;
    const Slice mp{gp, v0, nv, R.V}, mq{gq, v0, nv, R.V};   // in memory
    const Slice sp{RES ? smem : gp, v0, nv, R.V}, sq{RES ? smem + (size_t)sv * 16 : gq, v0, nv, R.V};
    const int per = ((nv + nw - 1) / nw + 7) & ~7, wa = min(warp * per, nv), wb = min(wa + per, nv);      // the warp's vectors
    if (RES && lane == 0 && wb > wa) {
        const uint32_t bytes = (uint32_t)(wb - wa) * 16u;
        mbar_arrive_expect(&S.bar[warp], 2 * bytes);
        bulk_load(smem_u32(smem + (size_t)wa * 16), gp + (size_t)wa * 16, bytes, &S.bar[warp]);
        bulk_load(smem_u32(smem + (size_t)(sv + wa) * 16), gq + (size_t)wa * 16, bytes, &S.bar[warp]);
    }
    // ---- pass 1
    if (RES && wb > wa && !rows_wait(&S.bar[warp], 0)) S.failed = 1;
    for (int w = 0; w < 2; ++w) {
        const RSum r = warp_total(warp_row_sum<DT, RES, true>(w ? sq : sp, wa, wb, c));
        if (lane == 0) S.warp[w][warp] = r;
    }
    cluster_wait();                                         // every CTA of the cluster has started
    __syncthreads();
    if (warp < 2) {
        RSum r = lane < nw ? S.warp[warp][lane] : no_sum();
        r = warp_merge(r, c.d);
        if (S.failed) r.bad |= 2;
        if (lane < C) send_sum(&S.cta[warp][rank], r, lane);
    }
    cluster_sync();
    const RSum tp = warp_merge(lane < C ? S.cta[0][lane] : no_sum(), c.d), tq = warp_merge(lane < C ? S.cta[1][lane] : no_sum(), c.d);
    int st = sum_status(tp) | sum_status(tq);
    if (st & ST_WAIT) st = ST_WAIT;
    else if (!tau_ok(tau)) st = ST_BAD_TEMP;
    const float g = a.grad_tv ? a.grad_tv[b] : 1.f;
    unsigned char* const grow = a.grad + (int64_t)b * a.g_row_bytes;
    if (st) {                                               // (the same in every CTA)
        float z[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[i] = 0.f;
        for (int v = tid; v < nv; v += blockDim.x) store_vec<DT>(grow, v0 + v, R.V, z);
        if (rank == 0 && tid == 0) {
            if (a.tv) a.tv[b] = 0.f;
            if (a.s_aux) a.s_aux[b] = 0.f;
            if (a.row_status) a.row_status[b] = st;
        }
        return;
    }
    PairRef ref = pair_ref(tp, tq, c, tau);
    // ---- pass 2, and again where a comparison is not certain
    bool again = false;
    for (;;) {
        TvMass m = {0.0, 0.0, 0.0};
        float nearest = INFINITY;
        for (int v = wa + lane; v < wb; v += 32) {
            float sv8[VEC];
            float ab = 0.f, ss = 0.f, qs = 0.f;
            if (!again) pair_vec<DT>(row_vec<DT, RES>(sp, v), row_vec<DT, RES>(sq, v), ref, c, false, sv8, ab, ss, qs, nearest);
            else pair_vec<DT>(row_vec<DT, false>(mp, v), row_vec<DT, false>(mq, v), ref, c, true, sv8, ab, ss, qs, nearest);
            m.absum += (double)ab; m.signed_q += (double)ss; m.q += (double)qs;
            if (RES) {
                if (DT == 1) *reinterpret_cast<float4*>(smem + (size_t)v * 16) = make_float4(sv8[0], sv8[1], sv8[2], sv8[3]);
                *reinterpret_cast<float4*>(smem + (size_t)(sv + v) * 16) = make_float4(sv8[VEC - 4], sv8[VEC - 3], sv8[VEC - 2], sv8[VEC - 1]);
            }
        }
        m.absum = warp_sum(m.absum); m.signed_q = warp_sum(m.signed_q); m.q = warp_sum(m.q);
        const int near = __any_sync(0xffffffffu, nearest <= ref.near);
        if (lane == 0) { S.mass[0][warp] = m.absum; S.mass[1][warp] = m.signed_q; S.mass[2][warp] = m.q; S.near[warp] = near; }
        __syncthreads();
        if (warp == 0) {
            const int n = __any_sync(0xffffffffu, lane < nw && S.near[lane]);
            double s[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) s[i] = warp_sum(lane < nw ? S.mass[i][lane] : 0.0);
            if (lane < C) {
#pragma unroll
                for (int i = 0; i < 3; ++i) st_remote(at_rank(&S.cta_mass[i][rank], lane), s[i]);
                st_remote(at_rank(&S.cta_near[rank], lane), n);
            }
        }
        cluster_sync();
        if (again || !__any_sync(0xffffffffu, lane < C && S.cta_near[lane])) break;
        // ---- the sums in double, around the same references
        double ds[2] = {0.0, 0.0};
        for (int w = 0; w < 2; ++w)
            for (int v = wa + lane; v < wb; v += 32) {
                float f[VEC];
                unpack<DT>(row_vec<DT, false>(w ? mq : mp, v), f);
                const double m0 = (double)(w ? ref.mq : ref.mp);
#pragma unroll
                for (int i = 0; i < VEC; ++i) ds[w] += q_exp2(((double)f[i] - m0) * c.d, S.tab);
            }
        for (int w = 0; w < 2; ++w) { const double x = warp_sum(ds[w]); if (lane == 0) S.wsum[w][warp] = x; }
        __syncthreads();
        if (warp < 2) {
            const double x = warp_sum(lane < nw ? S.wsum[warp][lane] : 0.0);
            if (lane < C) st_remote(at_rank(&S.cta_sum[warp][rank], lane), x);
        }
        cluster_sync();
        RSum xp = tp, xq = tq;
        xp.s = warp_sum(lane < C ? S.cta_sum[0][lane] : 0.0);
        xq.s = warp_sum(lane < C ? S.cta_sum[1][lane] : 0.0);
        ref = pair_ref(xp, xq, c, tau);
        again = true;
    }
    double absum = lane < C ? S.cta_mass[0][lane] : 0.0, signed_q = lane < C ? S.cta_mass[1][lane] : 0.0, q = lane < C ? S.cta_mass[2][lane] : 0.0;
    absum = warp_sum(absum); signed_q = warp_sum(signed_q); q = warp_sum(q);
    const double sum_p = tp.s, s_aux = fmin(fmax(0.5 * (signed_q + q) / q, 0.0), 1.0);      // (by the same terms' sum: 1 where no q is above p)
    if (rank == 0 && tid == 0) {
        if (a.tv) a.tv[b] = (float)fmin(fmax(0.5 * absum / sum_p, 0.0), 1.0);
        if (a.s_aux) a.s_aux[b] = (float)s_aux;
        if (a.row_status) a.row_status[b] = 0;
    }
    // ---- pass 3
    const double scale = (double)g / ((double)tau * q);
    const float below = (float)(-scale * (1.0 - s_aux)), above = (float)(-scale * s_aux);       // (times |q|; a negative q brings its own sign)
    float nearest = 0.f;
    for (int v = wa + lane; v < wb; v += 32) {
        float s8[VEC], o[VEC];
        if (RES) {
            if (DT == 1) { const float4 x = *reinterpret_cast<const float4*>(smem + (size_t)v * 16); s8[0] = x.x; s8[1] = x.y; s8[2] = x.z; s8[3] = x.w; }
            const float4 y = *reinterpret_cast<const float4*>(smem + (size_t)(sv + v) * 16);
            s8[VEC - 4] = y.x; s8[VEC - 3] = y.y; s8[VEC - 2] = y.z; s8[VEC - 1] = y.w;
        } else {
            float ab = 0.f, ss = 0.f, qs = 0.f;
            pair_vec<DT>(row_vec<DT, false>(mp, v), row_vec<DT, false>(mq, v), ref, c, again, s8, ab, ss, qs, nearest);
        }
        grad_vec<DT>(s8, below, above, o);
        store_vec<DT>(grow, v0 + v, R.V, o);
    }
}

cudaError_t tv_grad(const RowArgs& r, const float* grad_tv, float* tv, float* s_aux, int32_t* row_status, void* grad, int64_t ld_grad,
                    bool stream_rows, cudaStream_t stream) {
    TvGradArgs a;
    a.r = r; a.grad_tv = grad_tv; a.tv = tv; a.s_aux = s_aux; a.row_status = row_status;
    a.grad = static_cast<unsigned char*>(grad);
    a.g_row_bytes = ld_grad * (r.dt == 0 ? 4 : 2);
    a.s = rows_shape(r.B, 2, r.nvec, stream_rows);
    a.expire = take_expire_wait() ? 1 : 0;
    if (a.s.res) return r.dt == 0 ? rows_launch<k_tv_grad<0, true>>(a, r.B, a.s, stream) : rows_launch<k_tv_grad<1, true>>(a, r.B, a.s, stream);
    return r.dt == 0 ? rows_launch<k_tv_grad<0, false>>(a, r.B, a.s, stream) : rows_launch<k_tv_grad<1, false>>(a, r.B, a.s, stream);
}

}  // namespace bebop
