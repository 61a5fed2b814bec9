// bebop_distill: KL divergence of a student's rows from a teacher's top logits, and its gradient.
//
//   q = softmax(z / tau) over the whole vocabulary; entries i = (id, t_i), p_i = k exp((t_i - t_max) / tau):
//   without the teacher's logsumexp k makes sum p_i = 1; with it k = exp(t_max / tau - lse), and the mass r = 1 - P, P = sum p_i,
//   that the entries leave out meets the student's mass s outside the entries as one more token.
//   loss = sum p_i (log p_i - log q_i) + r log(r / s)
//   gradient of g loss: (g / tau) ((P + r) q_v - p_v) for an entry, (g / tau) (P + r - r / s) q_v elsewhere
//
// A CTA (a cluster of them, where there are fewer rows than SMs or rows are long) takes a row twice, the second time out of L2.
//   pass 1  the sum outside the entries, without the cancellation of 1 - sum q_i: a bit for every token of the row says which are
//           entries, and a lane masks those in its vectors once they are in shared memory.  The entries' own sums, in double, travel beside it.
//   pass 2  the gradient, as of a row without entries; the entries' own is written behind it.
// The entries are one warp's work, the keeper's, beside the readers': while they are in pass 1 of a row it gathers and sums that row's entries and sets the next
// row's bits; between the passes it has the row's numbers; behind pass 2 it writes the entries' gradient.  The readers wait for it once a row.
// 768 rows of 151,936 bf16, 64 entries: 118 us (0.61 of the copy rate; 134 with the entries spread over all warps), the loss alone 73; 100 rows of 49,999 fp32: 14.6, 12 of 1,024: 6.3.  The passes of a row lie one
// after the other (DRAM reads, then writes), 14 instructions a logit at half the issue rate.
#include "bebop_kernels.h"
#include "bebop_ring.cuh"

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
    // offsets in shared memory: two rows' entries; for two rows a bit for every token of the slice that is an entry, so many words, and a byte for every 32 vectors that hold one (the next row's
    // `second` bytes behind: 0 where both do not fit, and a cluster takes one row)
    int o_tab, o_bits, words, marks, second;
    RingShape s;
    int expire;
};

constexpr int kDistillSlots = 2;
template <int DT> using DistillRing = Ring<DT, 1, kDistillSlots>;
// What a warp knows of a row: the sum outside the entries, around m; of the entries the largest logits of teacher (t_m) and student (z_m), the student's sum around
// z_m, W = sum w, A = sum w (t_m - t) / tau, B = sum w (z_m - z) / tau, with w = exp((t - t_m) / tau).
struct __align__(16) DSum { double s, top_s, W, A, B; float m, z_m, t_m; int bad, pad[2]; };
enum { D_NONFINITE = 1, D_WAIT = 2, D_ID = 4, D_MASKED = 8, D_ANY = 16 };      // (D_MASKED: an entry with weight that the draft masks; D_ANY: the row has an entry)

// 2^((a - b) c) of two logits, 0 where a is -inf
__device__ __forceinline__ double logit_factor(float a, float b, const RScale& c) { return a == -INFINITY ? 0.0 : a == b ? 1.0 : q_exp2(((double)a - (double)b) * c.d, g_pow2_64); }
__device__ __forceinline__ float warp_max(float x) { return ord2f(redux_max(f2ord(x))); }
// n <= 32 records merged by a warp (the same bits in every lane).  In double: 1 - P is what matters of W, and B may be as large as a logit.
template <bool FAR> __device__ __forceinline__ DSum merge(const DSum* s, int n, const RScale& c, double inv_tau) {
    const int lane = threadIdx.x & 31;
    DSum x;
    x.s = x.top_s = x.W = x.A = x.B = 0.0; x.m = x.z_m = x.t_m = -INFINITY; x.bad = 0;
    if (lane < n) x = s[lane];
    DSum o;
    o.m = warp_max(x.m); o.z_m = warp_max(x.z_m); o.t_m = warp_max(x.t_m);
    o.bad = __reduce_or_sync(0xffffffffu, x.bad);
    o.s = warp_sum_pos(x.s * ref_factor<FAR>(x.m, o.m, c));
    o.top_s = warp_sum(x.top_s * logit_factor(x.z_m, o.z_m, c));
    const double f = logit_factor(x.t_m, o.t_m, c), W = x.W * f;
    o.W = warp_sum(W);
    o.A = warp_sum(W > 0.0 ? x.A * f + W * (((double)o.t_m - (double)x.t_m) * inv_tau) : 0.0);
    o.B = warp_sum(W > 0.0 && x.z_m > -INFINITY ? x.B * f + W * (((double)o.z_m - (double)x.z_m) * inv_tau) : 0.0);
    o.pad[0] = o.pad[1] = 0;
    return o;
}

// The numbers of a row's entries: log k, k, P, r.
struct EntryNumbers { double logk, k, P, r; };
__device__ __forceinline__ EntryNumbers entry_numbers(const DSum& d, double inv_tau, bool has_lse, float lse) {
    EntryNumbers o;
    o.logk = has_lse ? (double)d.t_m * inv_tau - (double)lse : 0.0;
    o.k = has_lse ? (d.W > 0.0 ? q_exp2(fmin(o.logk * 1.4426950408889634, 1000.0), g_pow2_64) : 0.0) : 1.0 / d.W;
    o.P = has_lse ? o.k * d.W : 1.0;
    o.r = has_lse ? fmax(1.0 - o.P, 0.0) : 0.0;
    return o;
}
// What pass 2 needs: the factor outside the entries, the reference; nothing: the gradient is 0; far: the sums are to be done again as FAR.
struct __align__(16) DistillRow { float other, M; int nothing, far; };
// The keeper's numbers of a row: sums around M (all, outside the entries), the entries' reference above M as a power of two, and for their gradient (g / tau) / sum q (P + r), (g / tau) k.
struct RowNumbers { DistillRow row; double total, tail, up, q, w; int st; };
template <bool FAR> __device__ __forceinline__ RowNumbers numbers(const DSum& d, const EntryNumbers& e, const RScale& c, float tau, double inv_tau, bool has_lse, float g) {
    const bool any = d.bad & D_ANY;
    RowNumbers o;
    o.row.far = !FAR && !(d.bad & 7) && any && tau_ok(tau) && (sum_far(d.m) || (fabs((double)d.z_m * c.d) >= (double)kRowsFar && d.z_m > -INFINITY));
    const float M = fmaxf(d.m, FAR ? d.z_m : (float)((double)d.z_m * c.d));
    o.row.M = M;
    o.up = d.z_m == -INFINITY ? 0.0 : row_arg<FAR>(d.z_m, M, c);
    o.tail = d.m == -INFINITY ? 0.0 : d.s * (FAR ? q_exp2(((double)d.m - (double)M) * c.d, g_pow2_64) : q_exp2((double)d.m - (double)M, g_pow2_64));
    o.total = o.tail + (d.z_m == -INFINITY ? 0.0 : d.top_s * q_exp2(o.up, g_pow2_64));
    o.st = 0;
    if (d.bad & D_WAIT) o.st = ST_WAIT;
    else if (!tau_ok(tau)) o.st = ST_BAD_TEMP;
    else if (d.bad & D_ID) o.st = ST_BAD_TOKEN;
    else if (any) o.st = d.bad & D_NONFINITE ? ST_NONFINITE : M == -INFINITY || (!has_lse && !(d.W > 0.0)) ? ST_EMPTY : 0;
    o.row.nothing = o.st != 0 || !any;
    const double G = (double)g * inv_tau;
    o.q = G / o.total * (e.P + e.r);
    o.w = G * e.k;
    o.row.other = o.tail > 0.0 ? (float)(o.q - (e.r > 0.0 ? G * e.r / o.tail : 0.0)) : 0.f;
    return o;
}
// KL: sum p (log p - log q) + r log(r / s), by a warp: four logarithms side by side.
__device__ __forceinline__ double kl(const DSum& d, const EntryNumbers& e, const RowNumbers& o, bool has_lse) {
    const int lane = threadIdx.x & 31;
    const double l = log(lane == 0 ? o.total : lane == 1 ? d.W : lane == 2 ? e.r : o.tail);
    const double logS = __shfl_sync(0xffffffffu, l, 0), logW = __shfl_sync(0xffffffffu, l, 1), logr = __shfl_sync(0xffffffffu, l, 2), logs = __shfl_sync(0xffffffffu, l, 3);
    // the entries' logits lie B / W below z_m in the mean, which lies `up` above M
    double loss = 0.0;
    if (d.W > 0.0) loss = e.P * ((has_lse ? e.logk : -logW) + logS) - e.k * (d.A - d.B + d.W * (o.up * 0.6931471805599453));
    if (e.r > 0.0) loss += e.r * (logr - logs + logS);
    return d.bad & D_MASKED ? INFINITY : loss;
}

struct DistillShared {
    RSum sum[kRingWarps];
    DSum cta_sum[3][kRowsMaxCluster];      // (two rows' in turn; a FAR row's second sums)
    DistillRow row;
    unsigned long long bar[kRingWarps][kDistillSlots];
};
enum { BAR_SUMS = 1, BAR_ROW, BAR_WRITTEN };                  // the readers' sums are there; the row's numbers are; the readers have written its gradient

// the bits of vector vi's tokens
template <int DT> __device__ __forceinline__ uint32_t entry_bits(const unsigned char* bits, int vi) { return DT == 0 ? (bits[vi >> 1] >> ((vi & 1) * 4)) & 15u : bits[vi]; }

// What a CTA works on.
template <int DT> struct DistillCta {
    const DistillArgs& a;
    DistillShared& S;
    unsigned char* bits[2];                                 // of this row and the next, in turn
    int* tab;
    int rank, nw, v0, nv;                                   // (nw readers)

    __device__ __forceinline__ const unsigned char* draft(int u) const { return reinterpret_cast<const unsigned char*>(row_ptr(a.r, u, a.r.K + 1)); }
    __device__ __forceinline__ int threads() const { return 32 * (nw + 1); }
    // A reader's sum to the keeper ...
    __device__ __forceinline__ void give(const RSum& mine) const {
        if ((threadIdx.x & 31) == 0) S.sum[threadIdx.x >> 5] = mine;
        bar_arrive(BAR_SUMS, threads());
        if (a.s.C > 1) cluster_sync();
        bar_sync(BAR_ROW, threads());
    }
    // ... which joins them to its record, and the records of the cluster's CTAs
    template <bool FAR> __device__ __forceinline__ DSum gather(DSum d, DSum* ctas, const RScale& c, double inv_tau) const {
        const int lane = threadIdx.x & 31, C = a.s.C;
        __syncwarp();
        bar_sync(BAR_SUMS, threads());
        const RSum r = warp_merge<FAR>(lane < nw ? S.sum[lane] : no_sum(), c);
        d.s = r.s; d.m = r.m; d.bad |= r.bad;
        if (C == 1) return d;
        if (lane < C) {
            const uint32_t to = at_rank(&ctas[rank], lane);
            const int* const v = reinterpret_cast<const int*>(&d);
#pragma unroll
            for (int i = 0; i < (int)sizeof(DSum) / 4; ++i) st_remote(to + 4 * i, v[i]);
        }
        cluster_sync();
        return merge<FAR>(ctas, C, c, inv_tau);
    }
    static __device__ __forceinline__ void bar_arrive(int id, int n) { asm volatile("barrier.cta.arrive %0, %1;" :: "r"(id), "r"(n) : "memory"); }
    static __device__ __forceinline__ void bar_sync(int id, int n) { asm volatile("barrier.cta.sync %0, %1;" :: "r"(id), "r"(n) : "memory"); }

    __device__ __forceinline__ void readers(unsigned char* smem);
    __device__ __forceinline__ void keeper();
};

template <int DT> __device__ __forceinline__ void DistillCta<DT>::readers(unsigned char* smem) {
    constexpr int VEC = Elem<DT>::VEC;
    using Rows = DistillRing<DT>;
    const RowArgs& R = a.r;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = run_length(nv, nw), wa = min(warp * per, nv), len = min(per, nv - wa);
    const int left0 = R.V - (v0 + wa) * VEC;                // tokens from the warp's first vector on
    const int clusters = a.s.clusters;
    int u = (int)(blockIdx.x / (unsigned)a.s.C);
    Rows ring;
    ring.init(smem + (size_t)warp * Rows::BYTES, S.bar[warp], len, left0);
    ring.at[0] = draft(u) + (int64_t)(v0 + wa) * 16;
    ring.first();
    float tau = tau_of(R, u);
    float tau_c = tau;
    RScale c = rows_scale(tau);
    __syncthreads();                                        // (the first row's bits)
    if (a.s.C > 1) cluster_sync();                          // every CTA of the cluster has started
    int k = 0;
#pragma unroll 1
    for (; u < R.B; u += clusters, k ^= 1) {
        const bool more = u + clusters < R.B;
        const unsigned char* next_at[1] = {nullptr};
        if (more) next_at[0] = draft(u + clusters) + (int64_t)(v0 + wa) * 16;
        const unsigned char* const* const next = more ? next_at : nullptr;
        if (tau != tau_c) { c = rows_scale(tau); tau_c = tau; }
        if (more) tau = tau_of(R, u + clusters);            // (asked for a row ahead)
        // ---- pass 1
        const unsigned char* const my_bits = bits[k];
        const unsigned char* const my_rows = my_bits + 4 * a.words;
        typename Rows::Sum rs[1];
        ring.template sums<true>(left0, !a.grad, next, c, rs, [&](const unsigned char* b, int from) {
            const int vi = wa + (from >> 4) + lane;
            uint32_t held = __ballot_sync(0xffffffffu, lane < kRingVecs && my_rows[(vi - lane) / 32 + lane]);      // the rows of 32 vectors that have entries
            if (held) {
#pragma unroll 1
                for (; held; held &= held - 1) {
                    const int j = __ffs(held) - 1;
                    for (uint32_t e = entry_bits<DT>(my_bits, vi + j * 32); e; e &= e - 1) {
                        unsigned char* const z = const_cast<unsigned char*>(b) + j * 512 + (__ffs(e) - 1) * (16 / VEC);
                        if (DT == 0) *reinterpret_cast<float*>(z) = -INFINITY; else *reinterpret_cast<unsigned short*>(z) = 0xff80u;
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (before the slot's next copy)
            }
        });
        RSum mine;
        mine.s = warp_sum_pos(rs[0].s);
        mine.m = rs[0].e == E_EMPTY ? -INFINITY : (float)rs[0].e;
        mine.bad = (rs[0].bad ? D_NONFINITE : 0) | (ring.failed ? D_WAIT : 0);
        give(mine);
        const bool far = S.row.far;                         // (the same in every CTA)
        if (far) {
            mine = far_sum<DT>(Slice{draft(u) + (int64_t)v0 * 16, v0, nv, R.V}, wa, wa + len, c, [=](int v) { return entry_bits<DT>(my_bits, v); });
            give(mine);
        }
        if (!a.grad) continue;
        // ---- pass 2
        const float M = S.row.M, other = S.row.other;
        const bool nothing = S.row.nothing;
        unsigned char* const run = a.grad + (int64_t)u * a.g_row_bytes + (int64_t)(v0 + wa) * 16;
        const auto put = [&](int at, const float* o, auto whole) {
            if (decltype(whole)::value) store_whole<DT>(run + at, 0, o);
            else if (at < ring.bytes) store_vec<DT>(run, at >> 4, left0, o);
        };
        if (nothing || far) ring.pass_small(left0, true, next, [&](int at, const uint4* x, auto whole) {
            float o[VEC];
            row_exp<DT, DT == 0, true>(x[0], M, c, o);
#pragma unroll
            for (int i = 0; i < VEC; ++i) o[i] = nothing ? 0.f : o[i] * other;
            put(at, o, whole);
        }, NoHook());
        else ring.pass(left0, true, next, [&](int at, const uint4* x, auto whole) {
            float o[VEC];
            row_exp<DT, DT == 0, false>(x[0], M, c, o);
            const float2 f = make_float2(other, other);
#pragma unroll
            for (int i = 0; i < VEC; i += 2) { const float2 y = __fmul2_rn(make_float2(o[i], o[i + 1]), f); o[i] = y.x; o[i + 1] = y.y; }
            put(at, o, whole);
        }, NoHook());
        bar_arrive(BAR_WRITTEN, threads());
    }
}

template <int DT> __device__ __forceinline__ void DistillCta<DT>::keeper() {
    const RowArgs& R = a.r;
    const int T = a.T, clusters = a.s.clusters, lane = threadIdx.x & 31;
    const int t0 = v0 * Elem<DT>::VEC, t1 = min((v0 + nv) * Elem<DT>::VEC, R.V);      // the CTA's tokens
    // the entries of this row and the next, every one its lane's own: id (-1: none, or another CTA's), teacher's logit, student's
    const auto id_at = [&](int k, int i) -> int& { return tab[k * 3 * T + i]; };
    const auto t_at = [&](int k, int i) -> float& { return reinterpret_cast<float*>(tab)[(k * 3 + 1) * T + i]; };
    const auto z_at = [&](int k, int i) -> float& { return reinterpret_cast<float*>(tab)[(k * 3 + 2) * T + i]; };
    constexpr int kAhead = 8;                               // entries of a lane asked for at a time
    // row u's entries into the table and the bits; what is wrong with them
    const auto take = [&](int k, int u) {
        int bad = 0;
        const int32_t* const ids = a.ids + (int64_t)u * T;
        const char* const top = static_cast<const char*>(a.top) + (int64_t)u * T * (a.top_dt == 0 ? 4 : 2);
        for (int i0 = lane; i0 < T; i0 += 32 * kAhead) {
            int id[kAhead];
            float t[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int i = i0 + 32 * j;
                id[j] = i < T ? ids[i] : -1;
                t[j] = i >= T ? 0.f : a.top_dt == 0 ? reinterpret_cast<const float*>(top)[i] : load_one<1>(top, i);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int i = i0 + 32 * j;
                if (id[j] != -1) {
                    bad |= D_ANY;
                    if (id[j] < 0 || id[j] >= R.V) { bad |= D_ID; id[j] = -1; }
                    else if (id[j] < t0 || id[j] >= t1) id[j] = -1;
                }
                if (id[j] >= 0) {
                    const int at = id[j] - t0;
                    if (atomicOr(reinterpret_cast<uint32_t*>(bits[k]) + (at >> 5), 1u << (at & 31)) >> (at & 31) & 1) bad |= D_ID;      // (given twice)
                    bits[k][4 * a.words + at / (32 * Elem<DT>::VEC)] = 1;
                    if (!(t[j] < INFINITY)) bad |= D_NONFINITE;
                }
                if (i < T) { id_at(k, i) = id[j]; t_at(k, i) = t[j]; }
            }
        }
        return bad;
    };
    // ... their sums (`bad`: the lane's)
    const auto sums = [&](int k, int u, int bad, float lse, const RScale& c, double inv_tau) {
        DSum d;
        float tm = -INFINITY, zm = -INFINITY;
        const char* const row = reinterpret_cast<const char*>(draft(u));
        for (int i0 = lane; i0 < T; i0 += 32 * kAhead) {
            float z[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int i = i0 + 32 * j, id = i < T ? id_at(k, i) : -1;
                z[j] = id < 0 ? -INFINITY : load_one<DT>(row, id);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int i = i0 + 32 * j;
                if (!(z[j] < INFINITY)) bad |= D_NONFINITE;
                if (i < T) {
                    if (id_at(k, i) >= 0) tm = max_nan(tm, t_at(k, i));
                    zm = max_nan(zm, z[j]);
                    z_at(k, i) = z[j];
                }
            }
        }
        if (!(fabsf(lse) < INFINITY)) bad |= D_NONFINITE;
        bad |= a.expire ? D_WAIT : 0;
        d.bad = __reduce_or_sync(0xffffffffu, bad);
        d.t_m = warp_max(tm); d.z_m = warp_max(zm);
        d.s = d.top_s = d.W = d.A = d.B = 0.0; d.m = -INFINITY; d.pad[0] = d.pad[1] = 0;
        if (d.bad & (D_NONFINITE | D_ID)) { d.t_m = d.z_m = -INFINITY; return d; }
        if (d.t_m == -INFINITY && d.z_m == -INFINITY) return d;
        for (int i = lane; i < T; i += 32) {
            if (id_at(k, i) < 0) continue;
            const float t = t_at(k, i), z = z_at(k, i);
            const double above = (double)d.t_m - (double)t, below = (double)d.z_m - (double)z, w = t > -INFINITY ? q_exp2(-above * c.d, g_pow2_64) : 0.0;
            if (z > -INFINITY) d.top_s += q_exp2(-below * c.d, g_pow2_64);
            if (w > 0.0) {
                d.W += w;
                d.A += w * (above * inv_tau);
                if (z > -INFINITY) d.B += w * (below * inv_tau); else d.bad |= D_MASKED;
            }
        }
        d.top_s = warp_sum(d.top_s); d.W = warp_sum(d.W); d.A = warp_sum(d.A); d.B = warp_sum(d.B);
        d.bad = __reduce_or_sync(0xffffffffu, d.bad);
        return d;
    };
    int u = (int)(blockIdx.x / (unsigned)a.s.C), k = 0;
    int bad = take(0, u);
    __syncthreads();
    if (a.s.C > 1) cluster_sync();
#pragma unroll 1
    for (; u < R.B; u += clusters, k ^= 1) {
        const float tau = tau_of(R, u), lse = a.lse ? a.lse[u] : 0.f, g = a.grad_loss ? a.grad_loss[u] : 1.f;
        const RScale c = rows_scale(tau);
        const double inv_tau = 1.0 / (double)tau;
        const DSum mine = sums(k, u, bad, lse, c, inv_tau);
        bad = u + clusters < R.B ? take(k ^ 1, u + clusters) : 0;
        EntryNumbers e = entry_numbers(mine, inv_tau, a.lse, lse);
        DSum tot;
        RowNumbers n;
        const auto settle = [&](DSum* ctas, auto far) {
            tot = gather<decltype(far)::value != 0>(mine, ctas, c, inv_tau);
            if (a.s.C > 1) e = entry_numbers(tot, inv_tau, a.lse, lse);
            n = numbers<decltype(far)::value != 0>(tot, e, c, tau, inv_tau, a.lse, g);
            if (lane == 0) S.row = n.row;
            __syncwarp();
            bar_sync(BAR_ROW, threads());
        };
        settle(S.cta_sum[k], Count<0>());
        const bool far = n.row.far;
        if (far) settle(S.cta_sum[2], Count<1>());
        for (int i = lane; i < T; i += 32) { const int id = id_at(k, i); if (id >= 0) { reinterpret_cast<uint32_t*>(bits[k])[(id - t0) >> 5] = 0u; bits[k][4 * a.words + (id - t0) / (32 * Elem<DT>::VEC)] = 0; } }
        __syncwarp();                                       // (before the bits of the row after next)
        const bool nothing = n.row.nothing;
        if (rank == 0) {
            const double loss = kl(tot, e, n, a.lse);
            if (lane == 0) {
                a.loss[u] = nothing ? 0.f : (float)loss;
                if (a.row_status) a.row_status[u] = n.st;
            }
        }
        if (!a.grad) continue;
        // ---- the entries' gradient, behind the vectors that hold them
        unsigned char* const grow = a.grad + (int64_t)u * a.g_row_bytes;
        bar_sync(BAR_WRITTEN, threads());
        if (nothing) continue;
        for (int i = lane; i < T; i += 32) {
            const int id = id_at(k, i);
            if (id < 0) continue;
            const float z = z_at(k, i), t = t_at(k, i);
            const double q = z > -INFINITY ? q_exp2(far ? row_arg<true>(z, n.row.M, c) : row_arg<false>(z, n.row.M, c), g_pow2_64) : 0.0;
            const double w = t > -INFINITY ? q_exp2(((double)t - (double)tot.t_m) * c.d, g_pow2_64) : 0.0;
            const float x = (float)(n.q * q - n.w * w);
            if (DT == 0) reinterpret_cast<float*>(grow)[id] = x;
            else reinterpret_cast<unsigned short*>(grow)[id] = (unsigned short)(pack_bf16x2(x, 0.f) & 0xffffu);
        }
    }
}

}  // namespace

template <int DT>
__global__ void __launch_bounds__(32 * kRingWarps, 1) k_distill(const __grid_constant__ DistillArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ DistillShared S;
    const int rank = (int)cluster_rank(), nw = (blockDim.x >> 5) - 1, v0 = rank * a.s.sv;
    DistillCta<DT> cta{a, S, {smem + a.o_bits, smem + a.o_bits + a.second}, reinterpret_cast<int*>(smem + a.o_tab), rank, nw, v0, max(min(a.s.sv, a.r.nvec - v0), 0)};
    for (int i = threadIdx.x; i < (a.marks + a.second) / 4; i += blockDim.x) reinterpret_cast<uint32_t*>(smem + a.o_bits)[i] = 0u;
    // (programmatic dependent launch: nothing of the caller's memory is touched until the grid before this one is through)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __syncthreads();
    if ((int)(threadIdx.x >> 5) < nw) cta.readers(smem); else cta.keeper();
    if (a.s.C > 1) cluster_sync();                          // (nobody stores into a CTA that has left)
}

cudaError_t distill(const RowArgs& r, const int32_t* ids, const void* top, int top_dt, int T, const float* lse, const float* grad_loss, float* loss,
                    int32_t* row_status, void* grad, int64_t ld_grad, cudaStream_t stream) {
    DistillArgs a;
    a.r = r; a.ids = ids; a.top = top; a.top_dt = top_dt; a.T = T; a.lse = lse; a.grad_loss = grad_loss; a.loss = loss; a.row_status = row_status;
    a.grad = static_cast<unsigned char*>(grad);
    a.g_row_bytes = ld_grad * (r.dt == 0 ? 4 : 2);
    a.expire = take_expire_wait() ? 1 : 0;
    const int vec = r.dt == 0 ? 4 : 8;
    // (a bit a token, of whole chunks beyond the slice: a lane looks at all of its chunk's vectors)
    const auto words = [=](int sv) { return ((sv + kRingChunk) * vec + 31) / 32; };
    const auto marks = [=](int sv) { return (4 * words(sv) + sv / 32 + kRingVecs + 16) & ~15; };
    const int ring = DistillRing<0>::BYTES;
    const auto shape = [&](int rows) {
        const auto extra = [=](int sv) { return 24 * T + 32 + rows * marks(sv); };
        return r.dt == 0 ? ring_shape<k_distill<0>>(r.B, 1, r.nvec, ring, 1, extra, a.s) : ring_shape<k_distill<1>>(r.B, 1, r.nvec, ring, 1, extra, a.s);
    };
    cudaError_t e = shape(2);
    const bool both = e == cudaSuccess;
    if (e == cudaErrorInvalidConfiguration && (e = shape(1)) == cudaSuccess) a.s.clusters = r.B;      // (vocabularies beyond 10 million)
    if (e != cudaSuccess) return e;
    a.o_tab = (a.s.threads / 32 - 1) * ring; a.o_bits = (a.o_tab + 24 * T + 15) & ~15; a.words = words(a.s.sv); a.marks = marks(a.s.sv); a.second = both ? a.marks : 0;
    return r.dt == 0 ? ring_launch<k_distill<0>>(a, a.s, stream) : ring_launch<k_distill<1>>(a, a.s, stream);
}

}  // namespace bebop
