// bebop_distill: KL divergence of a student's rows from a teacher's top logits, and its gradient, one cluster of CTAs per row.
//
//   q = softmax(z / tau) over the whole vocabulary; entries i = (id, t_i), p_i = k exp((t_i - t_max) / tau):
//   without the teacher's logsumexp k makes sum p_i = 1; with it k = exp(t_max / tau - lse), and the mass r = 1 - P, P = sum p_i,
//   that the entries leave out meets the student's mass s outside the entries as one more token.
//   loss = sum p_i (log p_i - log q_i) + r log(r / s)
//   gradient of g loss: (g / tau) ((P + r) q_v - p_v) for an entry, (g / tau) (P + r - r / s) q_v elsewhere
//
// A warp owns a run of the row's vectors and the entries that fall into it.  Once its vectors are in shared memory it takes the
// entries' logits out (they become -inf, their values go into a table by entry), so that its sum is the mass outside the entries,
// without the cancellation of 1 - sum q_i; the entries' sums, in double, travel beside it.  After one exchange every CTA
// has all the row's numbers.  The gradient of the entries is written behind the vectors that hold them.
#include "bebop_kernels.h"
#include "bebop_rows.cuh"

namespace bebop {

namespace {

struct DistillArgs {
    RowArgs r;                // (draft only)
    const int32_t* ids;       // [N, T]
    const void* top;          // [N, T]
    const float* lse;         // [N] or nullptr
    const float* grad_loss;   // [N] or nullptr
    float* loss;
    int32_t* row_status;
    unsigned char* grad;      // or nullptr
    int64_t g_row_bytes;
    int T, top_dt;
    int o_z, o_w, o_bits;     // offsets in shared memory: entries' logits and weights, a bit for every token of the slice that is an entry
    RowsShape s;
    int expire;
};

// What a warp, a CTA and the cluster know of a row: the sum outside the entries, the entries' sum, W = sum w, A = sum w (t - t_max) / tau,
// B = sum w (z - top_m) / tau, with w = exp((t - t_max) / tau).
struct __align__(16) DSum { double s, top_s, W, A, B; float m, top_m; int bad, pad; };      // bad: 1 NaN or +inf, 2 wait, 4 bad id

__device__ __forceinline__ DSum no_dsum() {
    DSum d; d.s = d.top_s = d.W = d.A = d.B = 0.0; d.m = d.top_m = -INFINITY; d.bad = d.pad = 0;
    return d;
}
// W (a - b) / tau, also where nothing (W = 0) hangs on a
__device__ __forceinline__ double moved(double W, float a, float b, double inv_tau) { return W > 0.0 && a != b ? W * (((double)a - (double)b) * inv_tau) : 0.0; }

// sums of the lanes merged over a warp (the same bits in every lane)
__device__ __forceinline__ DSum warp_merge(DSum d, double c, double inv_tau) {
    DSum o;
    o.m = ord2f(redux_max(f2ord(d.m)));
    o.top_m = ord2f(redux_max(f2ord(d.top_m)));
    o.bad = __reduce_or_sync(0xffffffffu, d.bad);
    o.pad = 0;
    o.s = warp_sum(d.s * ref_factor(d.m, o.m, c));
    o.top_s = warp_sum(d.top_s * ref_factor(d.top_m, o.top_m, c));
    o.W = warp_sum(d.W);
    o.A = warp_sum(d.A);
    o.B = warp_sum(d.B + moved(d.W, d.top_m, o.top_m, inv_tau));
    return o;
}

struct DistillShared {
    DSum warp[kRowsMaxWarps], cta[kRowsMaxCluster];
    unsigned long long bar[kRowsMaxWarps];
};

// the bits of vector vi's tokens
template <int DT> __device__ __forceinline__ uint32_t entry_bits(const uint32_t* bits, int vi) {
    constexpr int VEC = Elem<DT>::VEC;
    return (bits[(vi * VEC) >> 5] >> ((vi * VEC) & 31)) & ((1u << VEC) - 1u);
}
// Rows read from memory: entries are masked by their bits.
template <int DT> __device__ __forceinline__ uint4 without_entries(uint4 x, uint32_t b) {
    if (b == 0) return x;
    constexpr int VEC = Elem<DT>::VEC;
    float f[VEC];
    unpack<DT>(x, f);
#pragma unroll
    for (int i = 0; i < VEC; ++i) if (b >> i & 1) f[i] = -INFINITY;
    return pack<DT>(f);
}

}  // namespace

template <int DT, bool RES>
__global__ void __launch_bounds__(256, 2) k_distill(const __grid_constant__ DistillArgs a) {
    constexpr int VEC = Elem<DT>::VEC;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ DistillShared S;
    const RowArgs& R = a.r;
    const int C = a.s.C, sv = a.s.sv, T = a.T;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = blockDim.x >> 5;
    const int rank = (int)cluster_rank(), b = (int)(blockIdx.x / (unsigned)C);
    float* const ez = reinterpret_cast<float*>(smem + a.o_z);
    double* const ew = reinterpret_cast<double*>(smem + a.o_w);
    uint32_t* const bits = reinterpret_cast<uint32_t*>(smem + a.o_bits);
    cluster_arrive();                                       // (waited for before the first store into another CTA)
    const int v0 = rank * sv, nv = max(min(sv, R.nvec - v0), 0);
    // the warp's vectors; a multiple of eight, so that no two warps share a word of the entries' bits
    const int per = ((nv + nw - 1) / nw + 7) & ~7, wa = min(warp * per, nv), wb = min(wa + per, nv);
    if (lane == 0) { mbar_init(&S.bar[warp], 1); asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
    for (int i = wa * VEC / 32 + lane; i < (wb * VEC + 31) / 32; i += 32) bits[i] = 0u;
    __syncwarp();
    // (programmatic dependent launch: nothing of the caller's memory is touched until the grid before this one is through)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const float tau = tau_of(R, b);
    const RScale c = rows_scale(tau);
    const double inv_tau = 1.0 / (double)tau;
    const unsigned char* const gz = reinterpret_cast<const unsigned char*>(row_ptr(R, b, R.K + 1)) + (int64_t)v0 * 16;
    const Slice sl{RES ? smem : gz, v0, nv, R.V};
    if (RES && lane == 0 && wb > wa) {
        const uint32_t bytes = (uint32_t)(wb - wa) * 16u;
        mbar_arrive_expect(&S.bar[warp], bytes);
        bulk_load(smem_u32(smem + (size_t)wa * 16), gz + (size_t)wa * 16, bytes, &S.bar[warp]);
    }
    // ---- the teacher's entries: every warp looks them all over, for their largest logit
    const int32_t* const ids = a.ids + (int64_t)b * T;
    auto teacher = [&](int i) { return a.top_dt == 0 ? static_cast<const float*>(a.top)[(int64_t)b * T + i] : load_one<1>(static_cast<const char*>(a.top) + (int64_t)b * T * 2, i); };
    int bad = 0, valid = 0;
    float tmax = -INFINITY;
    for (int i = lane; i < T; i += 32) {
        const int id = ids[i];
        if (id == -1) continue;
        const float t = teacher(i);
        valid = 1;
        if (id < 0 || id >= R.V) bad |= 4;
        if (!(t < INFINITY)) bad |= 1;
        else tmax = fmaxf(tmax, t);
    }
    tmax = ord2f(redux_max(f2ord(tmax)));
    valid = __any_sync(0xffffffffu, valid);
    const float lse = a.lse ? a.lse[b] : 0.f;
    if (!(fabsf(lse) < INFINITY)) bad |= 1;
    // ---- the entries of the warp's own vectors leave the row
    if (RES && wb > wa && !rows_wait(&S.bar[warp], 0)) bad |= 2;
    if (a.expire) bad |= 2;
    DSum d = no_dsum();
    const int t0 = (v0 + wa) * VEC, t1 = min((v0 + wb) * VEC, R.V);      // the warp's tokens
    for (int i = lane; i < T; i += 32) {
        const int id = ids[i];
        if (id < t0 || id >= t1) continue;
        const int at = id - v0 * VEC;
        if (atomicOr(&bits[at >> 5], 1u << (at & 31)) >> (at & 31) & 1) { bad |= 4; continue; }      // (given twice)
        const float z = load_one<DT>(reinterpret_cast<const char*>(sl.p), at), t = teacher(i);
        if (!(z < INFINITY)) bad |= 1;
        d.top_m = max_nan(d.top_m, z);
        ez[i] = z;
        ew[i] = t > -INFINITY ? q_exp2(((double)t - (double)tmax) * c.d, g_pow2_64) : 0.0;
        if (RES) {
            if (DT == 0) reinterpret_cast<float*>(smem)[at] = -INFINITY;
            else reinterpret_cast<unsigned short*>(smem)[at] = 0xff80u;
        }
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
    d.top_m = ord2f(redux_max(f2ord(d.top_m)));
    if (!(bad & 5))
        for (int i = lane; i < T; i += 32) {
            const int id = ids[i];
            if (id < t0 || id >= t1) continue;
            const float z = ez[i];
            const double w = ew[i], x = ((double)z - (double)d.top_m) * inv_tau;
            if (z > -INFINITY) d.top_s += q_exp2(((double)z - (double)d.top_m) * c.d, g_pow2_64);
            if (w > 0.0) {
                d.W += w;
                d.A += w * (((double)teacher(i) - (double)tmax) * inv_tau);
                d.B += z > -INFINITY ? w * x : -INFINITY;
            }
        }
    __syncwarp();
    // ---- pass 1: the sum of what is left
    if (RES) {
        const RSum r = warp_row_sum<DT, true, true>(sl, wa, wb, c);
        d.s = r.s; d.m = r.m; bad |= r.bad;
    } else {
        RSum r = no_sum();
        for (int v = wa; v < wb; v += 32) {
            const int vi = v + lane;
            const uint4 x = vi < wb ? without_entries<DT>(row_vec<DT, false>(sl, vi), entry_bits<DT>(bits, vi)) : neg_inf_vec<DT>();
            const float wm = ord2f(redux_max(f2ord(max_nan(vec_max<DT>(x), -INFINITY))));
            if (!(wm < INFINITY)) { r.bad = 1; continue; }
            if (wm == -INFINITY) continue;
            if (!(wm <= r.m + c.slack)) { r.s *= ref_factor(r.m, wm, c.d); r.m = wm; }
            float e[VEC];
            row_exp<DT, true>(x, r.m, c, e);
            r.s += (double)sum_fixed<VEC>(e);
        }
        d.s = r.s; d.m = r.m; bad |= r.bad;
    }
    d.bad = bad;
    d = warp_merge(d, c.d, inv_tau);
    if (lane == 0) S.warp[warp] = d;
    cluster_wait();                                         // every CTA of the cluster has started
    __syncthreads();
    if (warp == 0) {
        d = warp_merge(lane < nw ? S.warp[lane] : no_dsum(), c.d, inv_tau);
        if (lane < C) {
            const uint32_t to = at_rank(&S.cta[rank], lane);
            st_remote(to, d.s); st_remote(to + 8, d.top_s); st_remote(to + 16, d.W); st_remote(to + 24, d.A); st_remote(to + 32, d.B);
            st_remote(to + 40, __float_as_int(d.m)); st_remote(to + 44, __float_as_int(d.top_m)); st_remote(to + 48, d.bad);
        }
    }
    cluster_sync();
    d = warp_merge(lane < C ? S.cta[lane] : no_dsum(), c.d, inv_tau);
    const float M = fmaxf(d.m, d.top_m);
    const double tail = d.s * ref_factor(d.m, M, c.d), top = d.top_s * ref_factor(d.top_m, M, c.d), total = tail + top;
    int st = 0;
    if (d.bad & 2) st = ST_WAIT;
    else if (!tau_ok(tau)) st = ST_BAD_TEMP;
    else if (d.bad & 4) st = ST_BAD_TOKEN;
    else if (valid) st = (d.bad & 1) || !(total == total) ? ST_NONFINITE : M == -INFINITY || (!a.lse && !(d.W > 0.0)) ? ST_EMPTY : 0;
    const bool nothing = st != 0 || !valid;                 // (the same in every CTA)
    // ---- the loss
    const double logk = a.lse ? (double)tmax * inv_tau - (double)lse : -log(d.W), k = a.lse ? (d.W > 0.0 ? exp(logk) : 0.0) : 1.0 / d.W;
    const double P = a.lse ? k * d.W : 1.0, r = a.lse ? fmax(1.0 - P, 0.0) : 0.0;
    if (rank == 0 && tid == 0) {
        double loss = 0.0;
        if (!nothing) {
            const double logS = log(total);
            if (d.W > 0.0) loss = k * d.A + P * logk - (k * (d.B + moved(d.W, d.top_m, M, inv_tau)) - P * logS);
            if (r > 0.0) loss += r * (log(r) - log(tail) + logS);
        }
        a.loss[b] = (float)loss;
        if (a.row_status) a.row_status[b] = st;
    }
    if (!a.grad) return;
    // ---- the gradient
    unsigned char* const grow = a.grad + (int64_t)b * a.g_row_bytes;
    const double G = nothing ? 0.0 : (a.grad_loss ? (double)a.grad_loss[b] : 1.0) * inv_tau, Gq = nothing ? 0.0 : G / total;
    const float other = nothing || !(tail > 0.0) ? 0.f : (float)(Gq * (P + r - (r > 0.0 ? r * total / tail : 0.0)));
    const float mref = nothing ? 0.f : M;
    for (int v = wa + lane; v < wb; v += 32) {
        float e[VEC];
        if (nothing) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) e[i] = 0.f;
        } else {
            uint4 x = row_vec<DT, RES>(sl, v);
            if (!RES) x = without_entries<DT>(x, entry_bits<DT>(bits, v));
            row_exp<DT, DT == 0>(x, mref, c, e);
#pragma unroll
            for (int i = 0; i < VEC; ++i) e[i] *= other;
        }
        store_vec<DT>(grow, v0 + v, R.V, e);
    }
    if (nothing) return;
    __syncwarp();                                           // (the warp's entries, behind the vectors that hold them)
    for (int i = lane; i < T; i += 32) {
        const int id = ids[i];
        if (id < t0 || id >= t1) continue;
        const double q = ez[i] > -INFINITY ? q_exp2(((double)ez[i] - (double)M) * c.d, g_pow2_64) : 0.0;
        const float x = (float)(Gq * (P + r) * q - G * k * ew[i]);
        if (DT == 0) reinterpret_cast<float*>(grow)[id] = x;
        else reinterpret_cast<unsigned short*>(grow)[id] = (unsigned short)(pack_bf16x2(x, 0.f) & 0xffffu);
    }
}

cudaError_t distill(const RowArgs& r, const int32_t* ids, const void* top, int top_dt, int T, const float* lse, const float* grad_loss, float* loss,
                    int32_t* row_status, void* grad, int64_t ld_grad, bool stream_rows, cudaStream_t stream) {
    DistillArgs a;
    a.r = r; a.ids = ids; a.top = top; a.top_dt = top_dt; a.T = T; a.lse = lse; a.grad_loss = grad_loss; a.loss = loss; a.row_status = row_status;
    a.grad = static_cast<unsigned char*>(grad);
    a.g_row_bytes = ld_grad * (r.dt == 0 ? 4 : 2);
    a.expire = take_expire_wait() ? 1 : 0;
    // beside the slice: 12 bytes an entry, a bit a token
    const int vec = r.dt == 0 ? 4 : 8;
    a.s = rows_shape(r.B, 1, r.nvec, stream_rows, 12 * T + 64, vec);
    const int bits = ((a.s.sv * vec + 31) / 32 + 1) * 4;
    a.o_w = a.s.bytes; a.o_z = a.o_w + 8 * T; a.o_bits = (a.o_z + 4 * T + 15) & ~15;
    a.s.bytes = a.o_bits + bits;
    if (a.s.res) return r.dt == 0 ? rows_launch<k_distill<0, true>>(a, r.B, a.s, stream) : rows_launch<k_distill<1, true>>(a, r.B, a.s, stream);
    return r.dt == 0 ? rows_launch<k_distill<0, false>>(a, r.B, a.s, stream) : rows_launch<k_distill<1, false>>(a, r.B, a.s, stream);
}

}  // namespace bebop
