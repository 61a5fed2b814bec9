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

// What a warp knows of a row: the sum outside the entries, around m; of the entries the sum, around top_m (a logit), W = sum w, A = sum w (t_max - t) / tau,
// B = sum w (top_m - z) / tau, with w = exp((t - t_max) / tau).
struct __align__(16) DSum { double s, top_s, W, A, B; float m, top_m; int bad, pad; };      // bad: 1 NaN or +inf, 2 wait, 4 bad id, 8 an entry with weight that the draft masks

__device__ __forceinline__ DSum no_dsum() {
    DSum d; d.s = d.top_s = d.W = d.A = d.B = 0.0; d.m = d.top_m = -INFINITY; d.bad = d.pad = 0;
    return d;
}
// 2^((a - b) c) of two logits, 0 where a is -inf
__device__ __forceinline__ double logit_factor(float a, float b, const RScale& c) { return a == -INFINITY ? 0.0 : a == b ? 1.0 : q_exp2(((double)a - (double)b) * c.d, g_pow2_64); }
// the entries' sums of `x` around the reference of `o`
__device__ __forceinline__ void entries_into(DSum& o, const DSum& x, const RScale& c, double inv_tau) {
    if (x.top_m == -INFINITY) { o.W += x.W; o.A += x.A; return; }
    o.top_s += x.top_s * logit_factor(x.top_m, o.top_m, c);
    o.W += x.W; o.A += x.A;
    o.B += x.B + x.W * (((double)o.top_m - (double)x.top_m) * inv_tau);
}
// n warps' sums merged (the same bits in every lane)
template <bool FAR> __device__ __forceinline__ DSum warp_merge(const DSum* s, int n, const RScale& c, double inv_tau) {
    const int lane = threadIdx.x & 31;
    float m = -INFINITY, tm = -INFINITY;
    int bad = 0;
    for (int i = lane; i < n; i += 32) { m = fmaxf(m, s[i].m); tm = fmaxf(tm, s[i].top_m); bad |= s[i].bad; }
    DSum o = no_dsum();
    o.m = ord2f(redux_max(f2ord(m)));
    o.top_m = ord2f(redux_max(f2ord(tm)));
    for (int i = lane; i < n; i += 32) {
        o.s += s[i].s * ref_factor<FAR>(s[i].m, o.m, c);
        if (s[i].W > 0.0 || s[i].top_m > -INFINITY) entries_into(o, s[i], c, inv_tau);
    }
    o.bad = __reduce_or_sync(0xffffffffu, bad);
    o.s = warp_sum_pos(o.s);
    o.top_s = warp_sum(o.top_s); o.W = warp_sum(o.W); o.A = warp_sum(o.A); o.B = warp_sum(o.B);      // (in double: 1 - P is what matters of W, and B may be as large as a logit)
    return o;
}

// What the gradient needs: (g / tau) / sum q (P + r), (g / tau) k, the factor outside the entries, the reference; the row has none; it is to be done again as FAR.
struct DistillGrad { double q, w; float other, M; int nothing, far; };

struct DistillShared {
    DSum sum[kRowsMaxParts];  // the warps' sums of all CTAs, by rank and warp
    DistillGrad grad;
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

// What a warp brings to the passes over the row.
struct DistillRow {
    Slice sl;
    uint32_t* bits;
    float* ez;
    double* ew;
    const int32_t* ids;
    RScale c;
    double inv_tau;
    float tau, lse;
    DSum d;                   // the entries' sums
    int bad, valid, rank, b, wa, wb, v0, t0, t1;
    float tmax;
};

// The row's numbers from the merged sums.
struct DistillNumbers { float M; double up, tail, total, logk, k, P, r; int st, nothing, far; };
template <bool FAR> __device__ __forceinline__ DistillNumbers numbers(const DistillArgs& a, const DistillRow& w, const DSum& d) {
    const RScale& c = w.c;
    DistillNumbers o;
    o.far = !FAR && !(d.bad & 7) && w.valid && tau_ok(w.tau) && (sum_far(d.m) || (fabs((double)d.top_m * c.d) >= (double)kRowsFar && d.top_m > -INFINITY));
    // both sums around M
    o.M = fmaxf(d.m, FAR ? d.top_m : (float)((double)d.top_m * c.d));
    o.up = d.top_m == -INFINITY ? 0.0 : row_arg<FAR>(d.top_m, o.M, c);      // the entries' reference above M, as a power of two
    o.tail = d.m == -INFINITY ? 0.0 : d.s * q_exp2(FAR ? ((double)d.m - (double)o.M) * c.d : (double)d.m - (double)o.M, g_pow2_64);
    o.total = o.tail + (d.top_m == -INFINITY ? 0.0 : d.top_s * q_exp2(o.up, g_pow2_64));
    o.st = 0;
    if (d.bad & 2) o.st = ST_WAIT;
    else if (!tau_ok(w.tau)) o.st = ST_BAD_TEMP;
    else if (d.bad & 4) o.st = ST_BAD_TOKEN;
    else if (w.valid) o.st = d.bad & 1 ? ST_NONFINITE : o.M == -INFINITY || (!a.lse && !(d.W > 0.0)) ? ST_EMPTY : 0;
    o.nothing = o.st != 0 || !w.valid;
    o.logk = a.lse ? (double)w.tmax * w.inv_tau - (double)w.lse : 0.0;
    o.k = a.lse ? (d.W > 0.0 ? q_exp2(fmin(o.logk * 1.4426950408889634, 1000.0), g_pow2_64) : 0.0) : 1.0 / d.W;
    o.P = a.lse ? o.k * d.W : 1.0;
    o.r = a.lse ? fmax(1.0 - o.P, 0.0) : 0.0;
    return o;
}
// KL: sum p (log p - log q) + r log(r / s).  (Of rank 0, behind the gradient: its logarithms are on nobody's way there.)
__device__ __forceinline__ double kl(const DistillArgs& a, const DSum& d, const DistillNumbers& o) {
    // the entries' logits lie B / W below top_m in the mean, which lies `up` above M
    const double logS = log(o.total), logk = a.lse ? o.logk : -log(d.W);
    double loss = 0.0;
    if (d.W > 0.0) loss = o.P * (logk + logS) - o.k * (d.A - d.B + d.W * (o.up * 0.6931471805599453));
    if (o.r > 0.0) loss += o.r * (log(o.r) - log(o.tail) + logS);
    return d.bad & 8 ? INFINITY : loss;
}

template <int DT, bool RES, bool FAR> __device__ __forceinline__ void gradient(const DistillArgs& a, const DistillRow& w, const DistillGrad& g) {
    constexpr int VEC = Elem<DT>::VEC;
    const RowArgs& R = a.r;
    const RScale& c = w.c;
    const int lane = threadIdx.x & 31;
    unsigned char* const grow = a.grad + (int64_t)w.b * a.g_row_bytes;
    if (g.nothing) {
        float z[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[i] = 0.f;
        for (int v = w.wa + lane; v < w.wb; v += 32) store_vec<DT>(grow, w.v0 + v, R.V, z);
        return;
    }
    int v = w.wa + lane;
    if (RES && !FAR) {
        const int full = min(w.wb, R.V / VEC - w.v0);
#pragma unroll 2
        for (; v < full; v += 32) {
            float e[VEC];
            row_exp<DT, DT == 0, FAR>(*reinterpret_cast<const uint4*>(w.sl.p + (size_t)v * 16), g.M, c, e);
#pragma unroll
            for (int i = 0; i < VEC; ++i) e[i] *= g.other;
            store_whole<DT>(grow, w.v0 + v, e);
        }
    }
    for (; v < w.wb; v += 32) {
        float e[VEC];
        uint4 x = row_vec<DT, RES>(w.sl, v);
        if (!RES) x = without_entries<DT>(x, entry_bits<DT>(w.bits, v));
        row_exp<DT, DT == 0, FAR>(x, g.M, c, e);
#pragma unroll
        for (int i = 0; i < VEC; ++i) e[i] *= g.other;
        store_vec<DT>(grow, w.v0 + v, R.V, e);
    }
    __syncwarp();                                           // (the warp's entries, behind the vectors that hold them)
    for (int i = lane; i < a.T; i += 32) {
        const int id = w.ids[i];
        if (id < w.t0 || id >= w.t1) continue;
        const double q = w.ez[i] > -INFINITY ? q_exp2(row_arg<FAR>(w.ez[i], g.M, c), g_pow2_64) : 0.0;
        const float x = (float)(g.q * q - g.w * w.ew[i]);
        if (DT == 0) reinterpret_cast<float*>(grow)[id] = x;
        else reinterpret_cast<unsigned short*>(grow)[id] = (unsigned short)(pack_bf16x2(x, 0.f) & 0xffffu);
    }
}
// The sum outside the entries, the exchange, the loss and the gradient.  True: the row is FAR, and nothing has been written.
template <int DT, bool RES, bool FAR>
__device__ __forceinline__ bool distill_rest(const DistillArgs& a, DistillShared& S, const DistillRow& w, bool first) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5, C = a.s.C;
    const RScale& c = w.c;
    const double inv_tau = w.inv_tau;
    DSum d = w.d;
    d.bad = w.bad;
    // ---- pass 1
    if (RES) {
        const RSum r = warp_row_sum<DT, true, true, FAR>(w.sl, w.wa, w.wb, c);
        d.s = r.s; d.m = r.m; d.bad |= r.bad;
    } else {
        RSum r = no_sum();
        for (int v = w.wa; v < w.wb; v += RCV) {
            uint4 x[RV];
#pragma unroll
            for (int j = 0; j < RV; ++j) {
                const int vi = v + j * 32 + lane;
                x[j] = vi < w.wb ? without_entries<DT>(row_vec<DT, false>(w.sl, vi), entry_bits<DT>(w.bits, vi)) : neg_inf_vec<DT>();
            }
            chunk_into<DT, true, FAR>(r, x, c);
        }
        d.s = r.s; d.m = r.m; d.bad |= r.bad;
    }
    d.s = warp_sum_pos(d.s);
    if (first) cluster_wait();                              // every CTA of the cluster has started
    if (lane < C) {
        const uint32_t to = at_rank(&S.sum[w.rank * nw + warp], lane);
        st_remote(to, d.s); st_remote(to + 8, d.top_s); st_remote(to + 16, d.W); st_remote(to + 24, d.A); st_remote(to + 32, d.B);
        st_remote(to + 40, __float_as_int(d.m)); st_remote(to + 44, __float_as_int(d.top_m)); st_remote(to + 48, d.bad);
    }
    cluster_sync();
    if (warp == 0) {
        d = warp_merge<FAR>(S.sum, C * nw, c, inv_tau);
        const DistillNumbers o = numbers<FAR>(a, w, d);
        if (lane == 0) {
            DistillGrad g;
            const double G = (a.grad_loss ? (double)a.grad_loss[w.b] : 1.0) * inv_tau, Gq = G / o.total;
            g.q = Gq * (o.P + o.r); g.w = G * o.k; g.M = o.M; g.nothing = o.nothing; g.far = o.far;
            g.other = o.tail > 0.0 ? (float)(Gq * (o.P + o.r - (o.r > 0.0 ? o.r * o.total / o.tail : 0.0))) : 0.f;
            S.grad = g;
        }
    }
    __syncthreads();
    const DistillGrad g = S.grad;                           // (the same in every CTA)
    if (g.far) return true;
    if (a.grad) gradient<DT, RES, FAR>(a, w, g);
    if (warp == 0 && w.rank == 0) {
        d = warp_merge<FAR>(S.sum, C * nw, c, inv_tau);
        const DistillNumbers o = numbers<FAR>(a, w, d);
        if (lane == 0) {
            a.loss[w.b] = o.nothing ? 0.f : (float)kl(a, d, o);
            if (a.row_status) a.row_status[w.b] = o.st;
        }
    }
    return false;
}
template <int DT, bool RES> __device__ __noinline__ void distill_far(const DistillArgs& a, DistillShared& S, const DistillRow& w) {
    cluster_sync();                                         // (every CTA has read the sums that are written again now)
    distill_rest<DT, RES, true>(a, S, w, false);
}

}  // namespace

template <int DT, bool RES>
__global__ void __launch_bounds__(256, 3) k_distill(const __grid_constant__ DistillArgs a) {
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
    int mine = 0;
    const int t0 = (v0 + wa) * VEC, t1 = min((v0 + wb) * VEC, R.V);      // the warp's tokens
    for (int i = lane; i < T; i += 32) {
        const int id = ids[i];
        if (id < t0 || id >= t1) continue;
        mine = 1;
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
    mine = __any_sync(0xffffffffu, mine);
    d.top_m = ord2f(redux_max(f2ord(d.top_m)));
    if (mine && !(bad & 5)) {
        for (int i = lane; i < T; i += 32) {
            const int id = ids[i];
            if (id < t0 || id >= t1) continue;
            const float z = ez[i];
            const double w = ew[i], below = (double)d.top_m - (double)z;
            if (z > -INFINITY) d.top_s += q_exp2(-below * c.d, g_pow2_64);
            if (w > 0.0) {
                d.W += w;
                d.A += w * (((double)tmax - (double)teacher(i)) * inv_tau);
                if (z > -INFINITY) d.B += w * (below * inv_tau); else bad |= 8;
            }
        }
        d.top_s = warp_sum(d.top_s); d.W = warp_sum(d.W); d.A = warp_sum(d.A); d.B = warp_sum(d.B);
        bad = __reduce_or_sync(0xffffffffu, bad);
    }
    __syncwarp();
    const DistillRow row{sl, reinterpret_cast<uint32_t*>(bits), ez, ew, ids, c, inv_tau, tau, lse, d, bad, valid, rank, b, wa, wb, v0, t0, t1, tmax};
    if (RES) {
        if (distill_rest<DT, RES, false>(a, S, row, true)) distill_far<DT, RES>(a, S, row);
    } else distill_rest<DT, RES, true>(a, S, row, true);
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
