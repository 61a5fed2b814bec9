// Rows that go through a CTA several times: what the kernels that take them so share.
//
// A unit (a row, a row pair) belongs to one CTA, or to a cluster of them where there are fewer units than SMs.  A warp owns a run of the unit's vectors and goes
// through it once for every pass, in chunks of kRingChunk vectors of each row: the first time from DRAM, then out of L2.  The chunks arrive in the warp's own ring
// in shared memory by bulk copies that its first lane asks for, one ring's length ahead, over the ends of passes and units; so what a pass has to wait for
// is the meeting of the warps between two passes, a fraction of a microsecond against the tens that a pass over a long row takes.
#pragma once
#include "bebop_rows.cuh"

namespace bebop {

namespace {

constexpr int kRingWarps = 16, kRingVecs = 6, kRingChunk = 32 * kRingVecs;      // warps of a CTA, at most; vectors per lane and row of a chunk; vectors of a chunk

template <int N> struct Count { static constexpr int value = N; };

__device__ __noinline__ bool ring_wait_long(uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < kRowsSpin; ++i) { if (mbar_try(bar, parity)) return true; __nanosleep(32); }
    return false;
}

// ROWS rows side by side; SLOTS slots of a chunk of each (fewer where a run has fewer chunks).
template <int DT, int ROWS, int SLOTS> struct Ring {
    static constexpr int VEC = Elem<DT>::VEC, PART = kRingChunk * 16, SLOT = ROWS * PART, BYTES = SLOTS * SLOT;      // bytes of a chunk of a row, of a slot, of a warp's ring
    const unsigned char* buf;                 // the lane's place in it
    uint32_t smem, bar;                       // the ring and its slots' barriers
    const unsigned char* at[ROWS];            // the warp's runs of the unit that is being asked for
    int bytes, off;                           // of a run; where the next chunk to ask for begins
    uint32_t slots, ask_slot, take_slot, phase;      // (phase: a bit for every slot)
    int full;                                 // rows of 32 vectors, one a lane, that lie inside the run and the vocabulary: all but the last, perhaps
    bool failed;
    unsigned long long stays, gone;           // L2 policies

    __device__ __forceinline__ void shape(int len, int left0) {
        bytes = len * 16; off = 0; slots = max(1, min(SLOTS, (len + kRingChunk - 1) / kRingChunk)); ask_slot = take_slot = 0;
        full = (left0 < len * VEC ? len - 1 : len) / 32;
    }
    // another run, once nothing is on its way any more
    __device__ __forceinline__ void aim(const unsigned char* run, int len, int left0) {
        shape(len, left0);
        at[0] = run;
        first();
    }
    __device__ __forceinline__ void init(unsigned char* b, unsigned long long* s, int len, int left0) {
        buf = b + (threadIdx.x & 31) * 16; smem = smem_u32(b); bar = smem_u32(s);
        phase = 0; failed = false;
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(stays));
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(gone));
        shape(len, left0);
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) mbar_init(&s[i], 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    }
    // asks for the next chunk of the unit at `at`.  `leave`: for the last time, so that its lines leave L2 first (768 row pairs of 151,936 bf16, 90 MB of them under way: 284 us
    // without, 279 with; in clusters of two, half as many, 297 and 271).
    __device__ __forceinline__ void ask(bool leave = false) {
        const int n = min(PART, bytes - off);
        if ((threadIdx.x & 31) == 0) {
            const uint32_t b = bar + 8 * ask_slot, to = smem + ask_slot * SLOT;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(b), "r"(ROWS * n) : "memory");
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                             :: "r"(to + r * PART), "l"(at[r] + off), "r"(n), "r"(b), "l"(leave ? gone : stays) : "memory");
        }
        if (++ask_slot == slots) ask_slot = 0;
        off = off + PART >= bytes ? 0 : off + PART;
    }
    __device__ __forceinline__ void first() { if (bytes > 0) for (uint32_t i = 0; i < slots; ++i) ask(); }
    // Waits for the chunks that nobody takes any more (asked for by a pass with `next`).
    __device__ __forceinline__ void drain() {
        if (bytes > 0)
            for (uint32_t i = 0; i < slots; ++i) {
                const uint32_t b = bar + 8 * take_slot;
                const uint32_t parity = phase >> take_slot & 1u;
                if (!mbar_try(b, parity)) ring_wait_long(b, parity);
                phase ^= 1u << take_slot;
                if (++take_slot == slots) take_slot = 0;
            }
    }
    // One pass, by whole warps: f(the lane's first vector of a chunk, in shared memory; its bytes from the run's start; how many full rows it has, and whether another, in part).  `next`: where the next unit's run lies, if this is the unit's last pass (and there is one), else null.
    template <typename F> __device__ __forceinline__ void chunks_of(bool last, const unsigned char* const* next, F&& f) {
#pragma unroll 1
        for (int rem = bytes; rem > 0; rem -= PART) {
            const uint32_t b = bar + 8 * take_slot;
            const uint32_t parity = phase >> take_slot & 1u;
            if (!mbar_try(b, parity) && !ring_wait_long(b, parity)) failed = true;
            const int from = bytes - rem, n = min(kRingVecs, full - from / 512);
            f(buf + take_slot * SLOT, from, n, n < kRingVecs && rem > n * 512);
            phase ^= 1u << take_slot;
            if (++take_slot == slots) take_slot = 0;
            __syncwarp();
            // the slot is free: the chunk one ring's length ahead, of this unit or, behind its last pass, of the next
            if (!last || rem > (int)slots * PART) ask(last);
            else if (next) {
                if (off == 0)
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) at[r] = next[r];
                ask();
            }
        }
    }
    // vector j of a lane's chunk; beyond the run (`rem` bytes from the chunk's start on) or the vocabulary (`left` tokens) masked
    static __device__ __forceinline__ uint4 edge_vec(const unsigned char* b, int r, int j, int rem, int left) {
        const int vi = j * 32 + (threadIdx.x & 31), l = left - vi * VEC;
        uint4 x = neg_inf_vec<DT>();
        if (vi * 16 < rem) x = *reinterpret_cast<const uint4*>(b + r * PART + j * 512);
        if (l < VEC) mask_tail<DT>(x, max(l, 0));
        return x;
    }
    static __device__ __forceinline__ uint4 whole_vec(const unsigned char* b, int r, int j) { return *reinterpret_cast<const uint4*>(b + r * PART + j * 512); }
    // ... vector by vector: f(its bytes from the run's start, the vectors of the rows, whether it lies inside the run and the vocabulary), and g(the lane's place in a chunk, its bytes from the run's start) behind every chunk.
    // `left0`: tokens of the vocabulary from the run's first on.
    template <typename F, typename G> __device__ __forceinline__ void pass(int left0, bool last, const unsigned char* const* next, F&& f, G&& g) {
        const int lane = threadIdx.x & 31;
        chunks_of(last, next, [&](const unsigned char* b, int from, int n, bool part) {
            const auto row = [&](int j) {
                uint4 x[ROWS];
#pragma unroll
                for (int r = 0; r < ROWS; ++r) x[r] = whole_vec(b, r, j);
                f(from + (j * 32 + lane) * 16, x, Count<1>());
            };
            if (n == kRingVecs) {
#pragma unroll
                for (int j = 0; j < kRingVecs; ++j) row(j);
            } else {
#pragma unroll 2
                for (int j = 0; j < n; ++j) row(j);
                if (part) {
                    uint4 x[ROWS];
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) x[r] = edge_vec(b, r, n, bytes - from, left0 - (from >> 4) * VEC);
                    f(from + (n * 32 + lane) * 16, x, Count<0>());
                }
            }
            g(b, from);
        });
    }
    // ... the same for what is seldom called: a small loop (its instructions come from memory first, by the 128 bytes; six vectors' worth of them cost 25 us, this 2)
    template <typename F, typename G> __device__ __forceinline__ void pass_small(int left0, bool last, const unsigned char* const* next, F&& f, G&& g) {
        const int lane = threadIdx.x & 31;
        chunks_of(last, next, [&](const unsigned char* b, int from, int, bool) {
            const int rem = bytes - from, left = left0 - (from >> 4) * VEC;
#pragma unroll 1
            for (int j = 0; j < kRingVecs && j * 512 < rem; ++j) {
                uint4 x[ROWS];
#pragma unroll
                for (int r = 0; r < ROWS; ++r) x[r] = edge_vec(b, r, j, rem, left);
                f(from + (j * 32 + lane) * 16, x, Count<0>());
            }
            g(b, from);
        });
    }
    // A pass for the rows' softmax sums: around the exponent of the warp's largest logit so far, a chunk's (at the end of a run a vector's) tokens in fp32, those in double.
    struct Sum { double s; int e; float ef, top; bool bad; };
    // h(the lane's place in a chunk, its bytes from the run's start) sees every chunk first, and may change the lane's own vectors of it.
    template <bool LOW, typename H> __device__ __forceinline__ void sums(int left0, bool last, const unsigned char* const* next, const RScale& c, Sum* o, H&& h) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) { o[r].s = 0.0; o[r].e = E_EMPTY; o[r].ef = 0.f; o[r].top = -INFINITY; o[r].bad = false; }
        const auto into = [&](Sum& a, const uint4* x, auto count) {
            constexpr int N = decltype(count)::value;
            const float m = vecs_max<DT, N>(x);
            if (!__all_sync(0xffffffffu, m <= a.top)) {       // (also a NaN; hardly ever after the first chunks)
                const QExp E = chunk_exponent(m, c.c);
                if (E.e == E_BAD) a.bad = true;
                else if (E.e > a.e) {
                    a.s *= a.e == E_EMPTY ? 0.0 : pow2d(max(a.e - E.e, -500));
                    a.e = E.e; a.ef = E.ef;
                    a.top = (E.ef - 0.0625f) / c.c;           // (a margin beyond every rounding: what is not above it has x c <= e)
                }
            }
            float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float e[VEC];
                row_exp<DT, LOW, false>(x[j], a.ef, c, e);
#pragma unroll
                for (int q = 0; q < VEC; q += 4) { s0 = __fadd2_rn(s0, make_float2(e[q], e[q + 1])); s1 = __fadd2_rn(s1, make_float2(e[q + 2], e[q + 3])); }
            }
            a.s += (double)((s0.x + s0.y) + (s1.x + s1.y));
        };
        chunks_of(last, next, [&](const unsigned char* b, int from, int n, bool part) {
            h(b, from);
            const auto rows = [&](int j0, auto count) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    uint4 x[decltype(count)::value];
#pragma unroll
                    for (int j = 0; j < decltype(count)::value; ++j) x[j] = whole_vec(b, r, j0 + j);
                    into(o[r], x, count);
                }
            };
            if (n == kRingVecs) rows(0, Count<kRingVecs>());
            else {
                int j = 0;
#pragma unroll 1
                for (; j + 2 <= n; j += 2) rows(j, Count<2>());
                if (j < n) rows(j, Count<1>());
                if (part)
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) { const uint4 x = edge_vec(b, r, n, bytes - from, left0 - (from >> 4) * VEC); into(o[r], &x, Count<1>()); }
            }
        });
    }
};
// the run of warp `warp` of nw, of nv vectors: whole rows of 32
__device__ __forceinline__ int run_length(int nv, int nw) { return ((nv + 31) / 32 + nw - 1) / nw * 32; }

// The warps' records, merged by a warp over its lanes (merge(records, n)), over the CTA and, through distributed shared memory, the cluster: the same in every
// warp.  `warps` and `ctas` must not be in use any more; a second meeting takes others.
template <typename R, typename F> __device__ __forceinline__ R meet(R* warps, R* ctas, const R& mine, int C, int rank, F&& merge) {
    static_assert(sizeof(R) % 16 == 0, "records are sent in words");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    if (lane == 0) warps[warp] = mine;
    __syncthreads();
    if (C == 1) return merge(warps, nw);
    if (warp == 0) {
        const R r = merge(warps, nw);
        if (lane < C) {
            const uint32_t d = at_rank(&ctas[rank], lane);
            const int* const v = reinterpret_cast<const int*>(&r);
#pragma unroll
            for (int i = 0; i < (int)sizeof(R) / 4; ++i) st_remote(d + 4 * i, v[i]);
        }
    }
    cluster_sync();
    return merge(ctas, C);
}

// ... into the first warp alone.  (Nothing else of the cluster meets between two of these: `ctas` are taken in turn.)
template <typename R, typename F> __device__ __forceinline__ R meet_first(R* warps, R* ctas, const R& mine, int C, int rank, F&& merge) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    R r = mine;
    if (lane == 0) warps[warp] = mine;
    __syncthreads();
    if (warp == 0) r = merge(warps, nw);
    if (C == 1) return r;
    if (warp == 0 && lane < C) {
        const uint32_t d = at_rank(&ctas[rank], lane);
        const int* const v = reinterpret_cast<const int*>(&r);
#pragma unroll
        for (int i = 0; i < (int)sizeof(R) / 4; ++i) st_remote(d + 4 * i, v[i]);
    }
    cluster_sync();
    if (warp == 0) r = merge(ctas, C);
    return r;
}
struct NoHook { __device__ __forceinline__ void operator()(const unsigned char*, int) const {} };

struct RingShape { int C, sv, threads, clusters, bytes; };      // CTAs per unit, vectors per slice, threads, clusters of the grid, dynamic shared memory

// How many clusters of a kernel's CTAs the device holds at a time (asked once per device, cut and use of shared memory; 0: not known).
template <auto kernel> int ring_resident(int C, int threads, int bytes) {
    struct Held { int n, bytes; };
    static Held cached[64][kRowsMaxCluster + 1][kRingWarps + 1] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); return 0; }
    Held& held = cached[dev][C][threads / 32];
    const Held now = held;
    if (now.n && now.bytes == bytes) return now.n > 0 ? now.n : 0;
    int got = 0;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)C); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = bytes; cfg.attrs = attr; cfg.numAttrs = 1;
    if (rows_ready<kernel>() != cudaSuccess || cudaOccupancyMaxActiveClusters(&got, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); got = 0; }
    held = Held{got > 0 ? got : -1, bytes};
    return got > 0 ? got : 0;
}

// The cut of a call of `units` units of `held` rows of nvec vectors; `others`: warps of a CTA beside those with a ring; `extra`: shared memory of a CTA beside the rings, for a slice of sv vectors.
template <auto kernel, typename E> cudaError_t ring_shape(int units, int held, int nvec, int ring_bytes, int others, E&& extra, RingShape& s) {
    const cudaError_t e = rows_ready<kernel>();
    if (e != cudaSuccess) return e;
    const int sms = rows_sms() > 0 ? rows_sms() : 148;
    s.C = 1;
    while (s.C < kRowsMaxCluster && (long long)units * (s.C + 1) <= sms && nvec > s.C * 1024) ++s.C;
    // The units under way at a time stay in L2 between their passes (90 MB of row pairs, read three times, came from DRAM 1.9 times).  Where a unit to an SM is more than that, two CTAs share
    // an SM, one's passes under the other's meetings, and a unit has as many as keeps them below (512 row pairs of 262,144 bf16: 326 us with four of 8 warps, 375 with two of 16, 415 with one).
    const double mb = nvec * 16e-6 * held;
    const bool two = sms / s.C * mb > 80.0;
    while (two && s.C < kRowsMaxCluster && 2.0 * sms / s.C * mb > 95.0) ++s.C;
    const int most = (two ? kRingWarps / 2 : kRingWarps) - others;
    for (;; --s.C) {
        s.sv = (nvec + s.C - 1) / s.C;
        // Where there are more units than SMs, warps with seven chunks each at least: short rows then share an SM, one's passes under another's meetings (1,024 rows of
        // 32,000 bf16 logits, loss alone: 39 us with 3 warps each, 58 with 15).  Else a warp for every chunk (100 rows of 49,999 fp32 logits: 15 us with 15, 38 with 3).
        const int chunks = (long long)units * s.C > sms && !two ? 7 : 1;
        int warps = (s.sv + chunks * kRingChunk - 1) / (chunks * kRingChunk);
        warps = warps < 2 ? 2 : warps > most ? most : warps;
        for (;; --warps) {
            s.threads = 32 * (warps + others);
            s.bytes = warps * ring_bytes + extra(s.sv);
            if (s.bytes <= kRowsSmem || warps == 1) break;
        }
        if (s.bytes > kRowsSmem) return cudaErrorInvalidConfiguration;
        s.clusters = ring_resident<kernel>(s.C, s.threads, s.bytes);
        // (few units: no larger clusters than the device holds at a time -- seven of sixteen, nine of fifteen)
        if (s.clusters >= units || (long long)units * s.C > sms || s.C == 1) break;
    }
    if (s.clusters <= 0) s.clusters = 1;
    if (s.clusters > units) s.clusters = units;
    return cudaSuccess;
}
template <auto kernel, typename A> cudaError_t ring_launch(const A& args, const RingShape& s, cudaStream_t stream) {
    return rows_launch<kernel>(args, s.clusters, s.C, s.threads, s.bytes, stream);
}

}  // namespace

}  // namespace bebop
