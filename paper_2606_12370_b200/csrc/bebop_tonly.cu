// bebop_target_only_verify: drafts without a distribution against the target's probabilities, one cluster of CTAs per sequence.
//
//   p_k = softmax(target[k] / tau); accept x_k while u_k < p_k(x_k) (Sec. 2.2, target-only sampling); at a reject at position n
//   draw from p_n without x_n, else from the row behind the last draft: y = min{v : C(v) >= u_final C(V - 1)}
//
// The CTAs take the rows one after the other and stop where the sequence does; a row behind the stop is not read, but for the chunks that are on their way when
// the row before it is rejected.  The hardware hands out the sequences.
// A warp owns a run of a row's vectors, in the order of the tokens, and leaves its sum, so that the draw goes from the CTAs' sums to the warps' and from there, over
// the owner's run once more, to the tokens.  It is made with the fp32 exponentials of the sums; where their error could change the token, once more by the series of 2^f with what is heavy in
// double (2 % of the draws below come to it), and in double (0.3 %).  (The lanes' sums of every chunk kept for the draw, so that it reads one chunk again and not a run: 262 us for the 237 below, as the passes
// pay for it.)
// 1,024 sequences of up to five rows of 151,936 bf16: 237 us (0.45 of the copy rate; 170 without draws), 256 of four: 101 to 114, one: 13 to 18.  Sequences of different lengths and the draws that are left open bound
// it; a step of the draw costs 25 to 80 us of its CTA's time.
#include "bebop_kernels.h"
#include "bebop_ring.cuh"

namespace bebop {

namespace {

struct TonlyArgs {
    RowArgs r;                // (target only)
    const int32_t* draft_tokens;
    const float* u_accept;
    const float* u_final;
    int32_t* accept_len;
    int32_t* out_tokens;
    float* p_draft;           // or nullptr
    int32_t* row_status;      // or nullptr
    RingShape s;
    int expire;
};

constexpr int kTonlyWarps = 16, kTonlySlots = 2, kTonlyGrains = 256;
template <int DT> using TonlyRing = Ring<DT, 1, kTonlySlots>;
struct __align__(16) TonlyVerdict { int ok, y, none, pad; };
struct TonlyShared {
    RSum sum[2][kTonlyWarps], cta_sum[2][kRowsMaxCluster];  // by the parity of the row: a CTA may be one row ahead
    TonlyVerdict verdict[kTonlyWarps], cta_verdict[3][kRowsMaxCluster];
    double wmass[kTonlyWarps], cmass[3][kRowsMaxCluster], grain[kTonlyGrains];
    unsigned long long bar[kTonlyWarps][kTonlySlots];
    double tab[64];
};

// How far a prefix of a row's masses, of sum S around its largest's power of two, may be off, in S.  ex2.approx: the errors are independent and below 2^-22 each, 2^-22 sqrt(sum p^2) in
// the mean at most, and sum p^2 <= 1 / S; a chunk's tokens are added up in fp32 by the lane, a random error of less than 2^-23 of each of `parts` such sums.  The series, with what
// is heavy in double: 4 2^-24 sqrt(sum p^2) of the rest, none of which is above 2^-7; the parts are vectors.
__device__ __forceinline__ double draw_error(double S, int nvec, int level) {
    return level == 0 ? 1.1920928955078125e-07 / sqrt(S) + 5.9604644775390625e-08 / sqrt((double)max(nvec / kRingVecs, 1))
                      : 1.0536712127723509e-08 / sqrt(S) + 5.9604644775390625e-08 / sqrt((double)nvec);
}

// A stopped sequence's row, for the draw.
struct TonlyRow {
    Slice sl;                 // the CTA's slice, where the caller has it
    RScale c;
    RSum tot;
    int x;                    // the rejected draft (-1: none)
    int rank, C, per, nvec, V;      // (per: vectors of a warp's run)
    double uf;
};

// The masses of vector vi's tokens, the rejected draft's 0: by LEVEL 0 ex2.approx, 1 the series, what is heavy in double, 2 double, 3 double around a logit (FAR).
template <int DT, int LEVEL> __device__ __forceinline__ double vec_mass(const uint4& v, int vi, const TonlyRow& r, const double* tab, double* m) {
    constexpr int VEC = Elem<DT>::VEC;
    float f[VEC], e[VEC];
    unpack<DT>(v, f);
    const int xi = r.x - (r.sl.v0 + vi) * VEC;
    double big = 0.0;
    if (LEVEL >= 2) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            m[i] = i == xi ? 0.0 : q_exp2(row_arg<LEVEL == 3>(f[i], r.tot.m, r.c), tab);
            big += m[i];
        }
        return big;
    }
    if (LEVEL == 0) row_exp<DT, true, false>(v, r.tot.m, r.c, e);
    else {
        const float least = series_least(r.tot.m, r.c);
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
            const float2 y = series_exp2(make_float2(f[i], f[i + 1]), r.c, least, (int)r.tot.m);
            e[i] = y.x; e[i + 1] = y.y;
        }
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        if (i == xi || f[i] == -INFINITY) e[i] = 0.f;
        m[i] = (double)e[i];
    }
    if (LEVEL == 1) {
        unsigned heavy = 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) heavy |= e[i] >= kHeavy ? 1u << i : 0u;
#pragma unroll 1
        for (; heavy; heavy &= heavy - 1) {                 // (few lanes have one)
            const int k = __ffs(heavy) - 1;
            float z = 0.f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) if (i == k) { z = f[i]; e[i] = 0.f; }
            const double y = q_exp2(row_arg<false>(z, r.tot.m, r.c), tab);
            big += y;
#pragma unroll
            for (int i = 0; i < VEC; ++i) if (i == k) m[i] = y;
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) s += e[i];
    return big + (double)s;
}
// vectors [a, b) of the slice through the warp's ring: f(the lane's vector, where it is in the slice, the first lane's)
template <int DT, typename F> __device__ __forceinline__ void vectors(TonlyRing<DT>& ring, const TonlyRow& r, int a, int b, F&& f) {
    const int left = r.V - (r.sl.v0 + a) * Elem<DT>::VEC;
    ring.aim(r.sl.p + (size_t)a * 16, max(b - a, 0), left);
    ring.pass_small(left, true, nullptr, [&](int at, const uint4* x, auto) { f(x[0], a + (at >> 4), a + ((at & ~511) >> 4)); }, NoHook());
}

// The draw: the owner of t = u_final Z among the CTAs, the warps' runs, the run's grains of vectors, its vectors, its tokens.  `mass`: the warp's (LEVEL 0; else it is taken here).  The same in every
// warp of the cluster: whether a token was drawn for certain, and in one of them the token (y); none: nothing is left to draw from.
template <int DT, int LEVEL> __device__ __forceinline__ TonlyVerdict draw(TonlyShared& S, TonlyRing<DT>& ring, const TonlyRow& r, double mass) {
    constexpr int VEC = Elem<DT>::VEC;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5, C = r.C;
    double m[VEC];
    if (LEVEL > 0) {
        const int a = min(warp * r.per, r.sl.nv);
        mass = 0.0;
        vectors<DT>(ring, r, a, min(a + r.per, r.sl.nv), [&](const uint4& x, int vi, int) { mass += vec_mass<DT, LEVEL>(x, vi, r, S.tab, m); });
        mass = warp_sum(mass);
    }
    __syncthreads();                                        // (the last level's masses have been read)
    if (lane == 0) S.wmass[warp] = mass;
    __syncthreads();
    const double cta = warp_sum(lane < nw ? S.wmass[lane] : 0.0);
    double cm = lane == 0 ? cta : 0.0;
    constexpr int turn = LEVEL < 2 ? LEVEL : 2;
    if (C > 1) {
        if (warp == 0 && lane < C) st_remote(at_rank(&S.cmass[turn][r.rank], lane), cta);
        cluster_sync();
        cm = lane < C ? S.cmass[turn][lane] : 0.0;
    }
    const double Z = warp_sum(cm), t = r.uf * Z, error = LEVEL < 2 ? draw_error(r.tot.s, r.nvec, LEVEL) * r.tot.s : 0.0;
    double base = 0.0, total;
    bool hit;
    TonlyVerdict o = {0, -1, 0, 0};
    o.none = LEVEL >= 2 && !(Z > 0.0);
    if (Z > error && pick_lane(cm, 0.0, t, &base, &total, &hit) == r.rank) {
        double below = base;
        const int w = pick_lane(lane < nw ? S.wmass[lane] : 0.0, below, t, &base, &total, &hit);
        below = base;
        const int a0 = min(w * r.per, r.sl.nv), a1 = min(a0 + r.per, r.sl.nv);
        const int grain = max((a1 - a0 + 32 * kTonlyGrains - 1) / (32 * kTonlyGrains), 1) * 32, grains = (a1 - a0 + grain - 1) / grain;
        // (every warp a part of them, in turn, one vector a lane and grain)
        const int some = ((grains + nw - 1) / nw), g0 = min(warp * some, grains), g1 = min(g0 + some, grains);
        double in = 0.0;
        int next = a0 + (g0 + 1) * grain, g = g0;
        vectors<DT>(ring, r, a0 + g0 * grain, min(a0 + g1 * grain, a1), [&](const uint4& x, int vi, int v) {
            in += vec_mass<DT, LEVEL>(x, vi, r, S.tab, m);
            if (v + 32 >= next || v + 32 >= a1) {
                const double s = warp_sum(in);
                if (lane == 0) S.grain[g] = s;
                ++g; next += grain; in = 0.0;
            }
        });
        __syncthreads();
        if (warp == 0) {
            // the grain that t lies in (or the last with mass), the vector, the token
            int at = -1;
            double lo = below;
            for (int i = 0; i < grains; i += 32) {
                const int src = pick_lane(i + lane < grains ? S.grain[i + lane] : 0.0, below, t, &base, &total, &hit);
                if (src >= 0) { at = i + src; lo = base; }
                if (hit) break;
                below = total;
            }
            if (at >= 0) {
                const int b0 = a0 + at * grain, b1 = min(b0 + grain, a1);
                below = lo;
                // (the last vector with mass up to t: its lane has the tokens')
                double mine[VEC];
                int vi = -1;
#pragma unroll 1
                for (int v = b0; v < b1; v += 32) {
                    const double s = vec_mass<DT, LEVEL>(v + lane < b1 ? row_vec<DT>(r.sl, v + lane) : neg_inf_vec<DT>(), v + lane, r, S.tab, m);
                    const int src = pick_lane(s, below, t, &base, &total, &hit);
                    if (src >= 0) {
                        vi = v + src; lo = base;
#pragma unroll
                        for (int i = 0; i < VEC; ++i) mine[i] = __shfl_sync(0xffffffffu, m[i], src);
                    }
                    if (hit) break;
                    below = total;
                }
                if (vi >= 0) {
                    bool done = false, sure = false;
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (mine[i] > 0.0 && !done) {
                            o.y = (r.sl.v0 + vi) * VEC + i;
                            const double hi = lo + mine[i];
                            done = hi >= t;
                            sure = t - lo > error && hi - t > error;
                            lo = hi;
                        }
                    o.ok = LEVEL >= 2 || (done && sure);
                }
            }
        }
    }
    if (LEVEL >= 2) { o.ok = o.y >= 0; return o; }
    return meet(S.verdict, S.cta_verdict[turn], o, C, r.rank, [&](const TonlyVerdict* s, int k) {
        TonlyVerdict v = o;
        v.ok = __any_sync(0xffffffffu, lane < k && s[lane].ok);
        return v;
    });
}
template <int DT, int LEVEL> __device__ __noinline__ TonlyVerdict draw_again(TonlyShared& S, TonlyRing<DT>& held, const TonlyRow& r) {
    TonlyRing<DT> ring = held;
    const TonlyRow row = r;
    const TonlyVerdict o = draw<DT, LEVEL>(S, ring, row, 0.0);
    held = ring;
    return o;
}

}  // namespace

template <int DT>
__global__ void __launch_bounds__(32 * kTonlyWarps, 1) k_target_only(const __grid_constant__ TonlyArgs a) {
    constexpr int VEC = Elem<DT>::VEC;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ TonlyShared S;
    const RowArgs& R = a.r;
    const int C = a.s.C, sv = a.s.sv, K = R.K;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = blockDim.x >> 5;
    const int rank = (int)cluster_rank(), b = (int)(blockIdx.x / (unsigned)C);
    const int v0 = rank * sv, nv = max(min(sv, R.nvec - v0), 0);
    const int per = run_length(nv, nw), wa = min(warp * per, nv), wb = min(wa + per, nv);      // the warp's vectors
    const int left0 = R.V - (v0 + wa) * VEC;
    if (C > 1) cluster_arrive();                            // (waited for before the first store into another CTA)
    TonlyRing<DT> ring;
    ring.init(smem + (size_t)warp * TonlyRing<DT>::BYTES, S.bar[warp], wb - wa, left0);
    if (tid < 64) S.tab[tid] = g_pow2_64[tid];
    // (programmatic dependent launch: nothing of the caller's memory is touched until the grid before this one is through)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    ring.at[0] = reinterpret_cast<const unsigned char*>(row_ptr(R, b, 0)) + (int64_t)(v0 + wa) * 16;
    ring.first();
    const int L = len_of(R, b);
    const float tau = tau_of(R, b), uf = a.u_final[b];
    const RScale c = rows_scale(tau);
    // every warp knows the drafts: lane k position k
    int tk = 0; float u = 0.f;
    if (lane < L) { tk = a.draft_tokens[(int64_t)b * K + lane]; u = a.u_accept[(int64_t)b * K + lane]; }
    int st = tau_ok(tau) ? 0 : ST_BAD_TEMP;
    if (!st && __any_sync(0xffffffffu, lane < L && (tk < 0 || tk >= R.V))) st = ST_BAD_TOKEN;
    __syncthreads();                                        // (the table)
    if (C > 1) cluster_wait();                              // every CTA of the cluster has started
    double px = 0.0;                                        // lane k: p_k(x_k), of the rows read
    int n = 0, x = -1;                                      // the row at hand; its draft
    float zx = 0.f;
    Slice sl{nullptr, v0, nv, R.V};
    RSum tot = no_sum(), mine;                              // the row's sum, the warp's
    bool far = false;
    auto arg = [&](float z) { return far ? row_arg<true>(z, tot.m, c) : row_arg<false>(z, tot.m, c); };
    int asked = 1;                                          // rows asked for that have not been read
    for (; !st; ++n) {
        const unsigned char* const g = reinterpret_cast<const unsigned char*>(row_ptr(R, b, n)) + (int64_t)v0 * 16;
        x = n < L ? __shfl_sync(0xffffffffu, tk, n) : -1;
        zx = n < L ? load_one<DT>(row_ptr(R, b, n), x) : 0.f;
        const unsigned char* next_at[1] = {nullptr};
        if (n < L) next_at[0] = reinterpret_cast<const unsigned char*>(row_ptr(R, b, n + 1)) + (int64_t)(v0 + wa) * 16;
        typename TonlyRing<DT>::Sum rs[1];
        ring.template sums<true>(left0, true, n < L ? next_at : nullptr, c, rs, NoHook());
        asked = n < L;
        mine.s = warp_sum_pos(rs[0].s);
        mine.m = rs[0].e == E_EMPTY ? -INFINITY : (float)rs[0].e;
        mine.bad = (rs[0].bad ? 1 : 0) | (a.expire || ring.failed ? 2 : 0);
        tot = meet(S.sum[n & 1], S.cta_sum[n & 1], mine, C, rank, [&](const RSum* s, int k) { return warp_merge<false>(lane < k ? s[lane] : no_sum(), c); });
        sl.p = g;
        if (!tot.bad && sum_far(tot.m)) {
            far = true;
            const RSum r = far_sum<DT>(sl, wa, wb, c, [](int) { return 0u; });
            __syncthreads();                                // (every warp has read the sums that are written again now)
            if (C > 1) cluster_sync();
            tot = meet(S.sum[n & 1], S.cta_sum[n & 1], r, C, rank, [&](const RSum* s, int k) { return warp_merge<true>(lane < k ? s[lane] : no_sum(), c); });
        } else far = false;
        st = sum_status(tot);
        if (st || n == L) break;
        const double p = fmin(q_exp2(arg(zx), S.tab) / tot.s, 1.0);
        if (lane == n) px = p;
        if (!((double)__shfl_sync(0xffffffffu, u, n) < p)) break;
    }
    if (asked) ring.drain();
    const int nn = st ? 0 : n;
    if (rank == 0 && warp == 0) {
        int32_t* const out = a.out_tokens + (int64_t)b * (K + 1);
        for (int q = lane; q <= K; q += 32) if (st || q != nn) out[q] = !st && q < nn ? tk : -1;      // (q < nn <= 32: q == lane)
        if (lane < K && a.p_draft) a.p_draft[(int64_t)b * K + lane] = st ? 0.f : (float)px;
        if (lane == 0) { a.accept_len[b] = nn; if (a.row_status) a.row_status[b] = st; }
    }
    if (st) return;                                         // (the same in every CTA: the last meeting lies behind, and nobody stores into a CTA any more)
    // ---- the draw, with the exponentials of the sums; where a token is not certain, with the series'; in double
    TonlyRow row{sl, c, tot, n == L ? -1 : x, rank, C, per, R.nvec, R.V, (double)uf};
    TonlyVerdict o = {0, -1, 0, 0};
    if (!far) {
        double mass = mine.s * ref_factor<false>(mine.m, tot.m, c);
        const int xv = row.x / VEC - v0;                    // the rejected draft's vector
        if (row.x >= 0 && xv >= wa && xv < wb) {            // (the warp's)
            float e[VEC];
            row_exp<DT, true, false>(row_vec<DT>(sl, xv), tot.m, c, e);
#pragma unroll
            for (int i = 0; i < VEC; ++i) if ((v0 + xv) * VEC + i == row.x) mass = fmax(mass - (double)e[i], 0.0);
        }
        o = draw<DT, 0>(S, ring, row, mass);
        if (!o.ok) o = draw_again<DT, 1>(S, ring, row);
        if (!o.ok) o = draw_again<DT, 2>(S, ring, row);
    } else o = draw_again<DT, 3>(S, ring, row);
    if (ring.failed && lane == 0 && a.row_status) a.row_status[b] = ST_WAIT;
    if (warp == 0 && lane == 0) {
        int32_t* const out = a.out_tokens + (int64_t)b * (K + 1) + nn;
        if (o.y >= 0 && o.ok) *out = o.y;
        else if (o.none && rank == 0) {                     // nothing is left beside the rejected draft: drawn from p, which is the draft
            *out = row.x;
            if (a.row_status) a.row_status[b] = ST_ZERO_RESID;
        }
    }
}

cudaError_t target_only(const RowArgs& r, const int32_t* draft_tokens, const float* u_accept, const float* u_final, int32_t* accept_len, int32_t* out_tokens,
                        float* p_draft, int32_t* row_status, cudaStream_t stream) {
    TonlyArgs a;
    a.r = r; a.draft_tokens = draft_tokens; a.u_accept = u_accept; a.u_final = u_final;
    a.accept_len = accept_len; a.out_tokens = out_tokens; a.p_draft = p_draft; a.row_status = row_status;
    a.expire = take_expire_wait() ? 1 : 0;
    const int sms = rows_sms() > 0 ? rows_sms() : 148;
    RingShape& s = a.s;
    s.C = 1;
    // (256 sequences of up to four rows of 151,936: 103 us with a CTA each, 110 with two; one sequence: 24 us with one, 12 with sixteen)
    while (s.C < kRowsMaxCluster && (long long)r.B * (s.C + 1) <= sms && r.nvec > s.C * 1024) ++s.C;
    for (;; --s.C) {
        s.sv = (r.nvec + s.C - 1) / s.C;
        int warps = (s.sv + 31) / 32;                       // a row of 32 vectors each at least: the smallest calls wait for the longest run
        warps = warps < 2 ? 2 : warps > kTonlyWarps ? kTonlyWarps : warps;
        s.threads = 32 * warps; s.bytes = warps * TonlyRing<0>::BYTES; s.clusters = r.B;
        // (no larger clusters than the device holds at a time)
        if (s.C == 1 || (r.dt == 0 ? ring_resident<k_target_only<0>>(s.C, s.threads, s.bytes) : ring_resident<k_target_only<1>>(s.C, s.threads, s.bytes)) >= r.B) break;
    }
    return r.dt == 0 ? ring_launch<k_target_only<0>>(a, s, stream) : ring_launch<k_target_only<1>>(a, s, stream);
}

}  // namespace bebop
