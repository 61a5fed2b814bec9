// bebop_target_only_verify: drafts without a distribution against the target's probabilities, one cluster of CTAs per sequence.
//
//   p_k = softmax(target[k] / tau); accept x_k while u_k < p_k(x_k) (Sec. 2.2, target-only sampling); at a reject at position n
//   draw from p_n without x_n, else from the row behind the last draft: y = min{v : C(v) >= u_final C(V - 1)}
//
// The cluster takes the rows one after the other and stops where the sequence does: rows behind the stop are never read.  A row's
// slices lie in the CTAs' shared memory; a warp owns a run of its vectors, in the order of the tokens, and leaves its sum, so
// that the draw goes from the CTAs' sums to the warps' to the tokens'.
#include "bebop_kernels.h"
#include "bebop_rows.cuh"

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
    RowsShape s;
    int expire;
};

struct TonlyShared {
    RSum sum[2][kRowsMaxParts];                             // the warps' sums of all CTAs, by rank and warp; by the parity of the row: a CTA may be one row ahead
    double wmass[kRowsMaxWarps], cmass[kRowsMaxCluster];
    unsigned long long bar[kRowsMaxWarps];
    double tab[64];
};

}  // namespace

template <int DT, bool RES>
__global__ void __launch_bounds__(256, 3) k_target_only(const __grid_constant__ TonlyArgs a) {
    constexpr int VEC = Elem<DT>::VEC;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ TonlyShared S;
    const RowArgs& R = a.r;
    const int C = a.s.C, sv = a.s.sv, K = R.K;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = blockDim.x >> 5;
    const int rank = (int)cluster_rank(), b = (int)(blockIdx.x / (unsigned)C);
    cluster_arrive();                                       // (waited for before the first store into another CTA)
    if (lane == 0) { mbar_init(&S.bar[warp], 1); asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
    if (tid < 64) S.tab[tid] = g_pow2_64[tid];
    __syncthreads();
    // (programmatic dependent launch: nothing of the caller's memory is touched until the grid before this one is through)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int L = len_of(R, b);
    const float tau = tau_of(R, b), uf = a.u_final[b];
    const RScale c = rows_scale(tau);
    const int v0 = rank * sv, nv = max(min(sv, R.nvec - v0), 0);
    const int per = (nv + nw - 1) / nw, wa = min(warp * per, nv), wb = min(wa + per, nv);      // the warp's vectors
    // every warp knows the drafts: lane k position k
    int tk = 0; float u = 0.f;
    if (lane < L) { tk = a.draft_tokens[(int64_t)b * K + lane]; u = a.u_accept[(int64_t)b * K + lane]; }
    int st = tau_ok(tau) ? 0 : ST_BAD_TEMP;
    if (!st && __any_sync(0xffffffffu, lane < L && (tk < 0 || tk >= R.V))) st = ST_BAD_TOKEN;
    double px = 0.0;                                        // lane k: p_k(x_k), of the rows read
    int n = 0, x = -1;                                      // the row at hand; its draft
    Slice sl{smem, v0, nv, R.V};
    RSum tot = no_sum();
    bool far = false;
    auto arg = [&](float z) { return far ? row_arg<true>(z, tot.m, c) : row_arg<false>(z, tot.m, c); };
    auto merge = [&](const RSum* s) { return far ? warp_merge<true>(lane_share<true>(s, C * nw, c), c) : warp_merge<false>(lane_share<false>(s, C * nw, c), c); };
    for (; !st; ++n) {
        const unsigned char* const g = reinterpret_cast<const unsigned char*>(row_ptr(R, b, n)) + (int64_t)v0 * 16;
        int bad = a.expire ? 2 : 0;
        if (RES) {
            if (wb > wa) {
                if (lane == 0) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (the warp has read the row before this one)
                    mbar_arrive_expect(&S.bar[warp], (uint32_t)(wb - wa) * 16u);
                    bulk_load(smem_u32(smem + (size_t)wa * 16), g + (size_t)wa * 16, (uint32_t)(wb - wa) * 16u, &S.bar[warp]);
                }
                if (!rows_wait(&S.bar[warp], n & 1)) bad |= 2;
            }
        } else sl.p = g;
        x = n < L ? __shfl_sync(0xffffffffu, tk, n) : -1;
        const float zx = n < L ? load_one<DT>(row_ptr(R, b, n), x) : 0.f;
        far = !RES;
        for (;;) {
            RSum r = warp_total(far ? warp_row_sum<DT, RES, true, true>(sl, wa, wb, c) : warp_row_sum<DT, RES, true, false>(sl, wa, wb, c));
            r.bad |= bad;
            if (n == 0 && !(RES && far)) cluster_wait();    // every CTA of the cluster has started
            if (lane < C) send_sum(&S.sum[n & 1][rank * nw + warp], r, lane);
            cluster_sync();
            tot = merge(S.sum[n & 1]);
            if (far || tot.bad || !sum_far(tot.m)) break;
            far = true;
            cluster_sync();                                 // (every CTA has read the sums that are written again now)
        }
        st = sum_status(tot);
        if (st || n == L) break;
        const double p = fmin(q_exp2(arg(zx), S.tab) / tot.s, 1.0);
        if (lane == n) px = p;
        if (!((double)__shfl_sync(0xffffffffu, u, n) < p)) break;
    }
    if (st == ST_BAD_TEMP || st == ST_BAD_TOKEN) cluster_wait();
    const int nn = st ? 0 : n;
    if (rank == 0 && warp == 0) {
        int32_t* const out = a.out_tokens + (int64_t)b * (K + 1);
        for (int q = lane; q <= K; q += 32) if (st || q != nn) out[q] = !st && q < nn ? tk : -1;      // (q < nn <= 32: q == lane)
        if (lane < K && a.p_draft) a.p_draft[(int64_t)b * K + lane] = st ? 0.f : (float)px;
        if (lane == 0) { a.accept_len[b] = nn; if (a.row_status) a.row_status[b] = st; }
    }
    if (st) return;                                         // (the same in every CTA)
    // ---- the draw, in double: the warps' masses, the CTAs', the owner's
    if (n == L) x = -1;
    int32_t* const out = a.out_tokens + (int64_t)b * (K + 1) + nn;
    auto masses = [&](int vi, double* m) {                  // of vector vi's tokens, the rejected draft's 0
        float f[VEC];
        unpack<DT>(row_vec<DT, RES>(sl, vi), f);
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            m[i] = (v0 + vi) * VEC + i == x ? 0.0 : q_exp2(arg(f[i]), S.tab);
            s += m[i];
        }
        return s;
    };
    double ws = 0.0, m[VEC];
    for (int v = wa + lane; v < wb; v += 32) ws += masses(v, m);
    ws = warp_sum(ws);
    if (lane == 0) S.wmass[warp] = ws;
    __syncthreads();
    if (warp == 0) {
        ws = warp_sum(lane < nw ? S.wmass[lane] : 0.0);
        if (lane < C) st_remote(at_rank(&S.cmass[rank], lane), ws);
    }
    cluster_sync();
    if (warp != 0) return;
    const double cm = lane < C ? S.cmass[lane] : 0.0, Z = warp_sum(cm);
    if (!(Z > 0.0)) {
        // nothing is left beside the rejected draft: drawn from p, which is the draft
        if (rank == 0 && lane == 0) { *out = x; if (a.row_status) a.row_status[b] = ST_ZERO_RESID; }
        return;
    }
    const double t = (double)uf * Z;
    double base, total;
    bool hit;
    if (pick_lane(cm, 0.0, t, &base, &total, &hit) != rank) return;
    double below = base;
    const int w = pick_lane(lane < nw ? S.wmass[lane] : 0.0, below, t, &base, &total, &hit);
    const int a0 = min(w * per, nv), a1 = min(a0 + per, nv);
    // the run's vectors, 32 at a time, for the last of them whose sum is needed; then its tokens
    below = base;
    int g0 = a0;
    for (int v = a0; v < a1; v += 32) {
        const double s = v + lane < a1 ? masses(v + lane, m) : 0.0;
        const int src = pick_lane(s, below, t, &base, &total, &hit);
        if (src >= 0) { g0 = v + src; ws = base; }
        if (hit) break;
        below = total;
    }
    if (lane == 0) {
        masses(g0, m);
        double run = ws;
        int y = -1;
        bool done = false;
#pragma unroll
        for (int i = 0; i < VEC; ++i) if (m[i] > 0.0 && !done) { y = (v0 + g0) * VEC + i; run += m[i]; done = run >= t; }
        *out = y;
    }
}

cudaError_t target_only(const RowArgs& r, const int32_t* draft_tokens, const float* u_accept, const float* u_final, int32_t* accept_len, int32_t* out_tokens,
                        float* p_draft, int32_t* row_status, bool stream_rows, cudaStream_t stream) {
    TonlyArgs a;
    a.r = r; a.draft_tokens = draft_tokens; a.u_accept = u_accept; a.u_final = u_final;
    a.accept_len = accept_len; a.out_tokens = out_tokens; a.p_draft = p_draft; a.row_status = row_status;
    a.expire = take_expire_wait() ? 1 : 0;
    a.s = rows_shape(r.B, 1, r.nvec, stream_rows);
    if (a.s.res) return r.dt == 0 ? rows_launch<k_target_only<0, true>>(a, r.B, a.s, stream) : rows_launch<k_target_only<1, true>>(a, r.B, a.s, stream);
    return r.dt == 0 ? rows_launch<k_target_only<0, false>>(a, r.B, a.s, stream) : rows_launch<k_target_only<1, false>>(a, r.B, a.s, stream);
}

}  // namespace bebop
