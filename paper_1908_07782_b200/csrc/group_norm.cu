// Group norm with an activation, channels last, for samples of many workers; forward and backward.
//
//   x [B][L][C], C = groups * Cg;  mean, rstd over the L * Cg values of a (sample, group)
//   h = (x - mean) * rstd,  z = h * gamma_w + beta_w,  y = act(z)                       w = the sample's worker
//   dz = dy * act'(z),  dgamma_w = sum dz * h,  dbeta_w = sum dz,  t = dz * gamma_w
//   dx = rstd * (t - mean(t) - h * mean(t * h))
//
// Bound by HBM: forward 1 read and 1 write of x, backward 2 reads and 1 write.  To read everything once, the unit of
// work is a (sample, block of whole groups): its L x CB slab is brought into shared memory, reduced and written out
// from there.  A cluster of up to 8 CTAs shares the slab along L and exchanges its sums through distributed shared
// memory.  Every thread works on the vectors it loaded itself (thread = (row, column)).  Slabs that 8 CTAs cannot hold are read again from global memory (L2)
// in place of shared memory (RES = false).
//
// Forward statistics: each thread takes mean and M2 (sum of squared deviations from its own mean) of its positions,
// for each run of channels of its vector that lie in one group, and these are merged by counts: sum of n_i * mean_i for the mean, M2_i + n_i (mean_i - mean)^2 for M2.
// Nothing is cancelled, whatever the size of the mean.
//
// z is formed in the roundings of the formula as written (no FMA), in both directions alike: a value that the forward
// pass clipped at zero is a value whose gradient the backward pass drops.
#include "host_common.h"
#include "step_common.cuh"

namespace {

using combo_step::add2;
using combo_step::Elem;
using combo_step::f32x2;
using combo_step::fma2;
using combo_step::hi_of;
using combo_step::lo_of;
using combo_step::mul2;
using combo_step::neg2;
using combo_step::pair;
using combo_step::warp_sum;

constexpr int kThreads = 128;
constexpr int kCtasPerSm = 4;           // that many slabs are in flight on an SM
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;          // portable cluster size

struct NormParams {
    const unsigned char* x;
    const unsigned char* dy;            // backward only
    unsigned char* y;                   // y, or dx
    const unsigned char* gamma;
    const unsigned char* beta;
    const int64_t* begin;               // [N + 1], or NULL: one worker
    float* mean;                        // [B][G]
    float* rstd;
    float2* partial;                    // backward: [B][C] sums of dz * h and dz of a CTA's samples of one worker, at the first of them
    long long x_pitch, y_pitch, dy_pitch, par_pitch;
    long long B;
    int L, C, G, Cg, GB, nblk, CS, Lc, N, ns, par_bytes, sub;
    float eps;
    // sub: channels of a vector that surely share a group, the largest power of two up to V that divides Cg
    int cb_max;                         // channels of a full block of groups, rounded up to a multiple of 4
    unsigned stat_off, par_off, grp_off, slab_off, slab_bytes;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
// only tells the peers that this CTA has read what it wanted of theirs
__device__ __forceinline__ void cluster_done() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// positions of the slab that the cluster's CTA `rank` holds
__device__ __forceinline__ int rank_len(const NormParams& p, int rank) { return max(0, min(p.Lc, p.L - rank * p.Lc)); }
// float2 at the same shared-memory place of the cluster's CTA `rank`
__device__ __forceinline__ float2 peer_float2(const float2* p, uint32_t rank) {
    uint32_t a = smem_u32(p), r;
    float2 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(r) : "memory");
    return v;
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ float load_par(const unsigned char* p, long long i, int bytes) {
    return bytes == 4 ? Elem<4>::get(p + i * 4) : Elem<2>::get(p + i * 2);
}

// the worker that sample b belongs to: the last one whose first sample is at or before b; the whole block
__device__ __forceinline__ int worker_of(const NormParams& p, long long b) {
    if (!p.begin) return 0;
    int c = 0;
    for (int base = 0; base < p.N; base += kThreads) {
        const int i = base + (int)threadIdx.x;
        const int got = __syncthreads_count(i < p.N && p.begin[i] <= b);
        c += got;
        if (got < kThreads) break;
    }
    return max(c - 1, 0);
}

// z in the formula's own roundings: (x - mean) * rstd, times gamma, plus beta
__device__ __forceinline__ f32x2 normed(f32x2 x, f32x2 neg_mean, f32x2 rstd) { return mul2(add2(x, neg_mean), rstd); }
__device__ __forceinline__ f32x2 affine(f32x2 h, f32x2 gamma, f32x2 beta) { return add2(mul2(h, gamma), beta); }
// ReLU keeps NaN.  SiLU: the fast exponential and division are within a few units of binary32's last place over the
// range where the result is not lost in rounding (the accurate ones took the kernel from memory to issue bound).
template <int ACT> __device__ __forceinline__ float activate(float z) {
    if (ACT == COMBO_ACT_RELU) {
        float r;
        asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(z));
        return r;
    }
    if (ACT == COMBO_ACT_SILU) return __fdividef(z, 1.0f + __expf(-z));
    return z;
}
// dy * act'(z); a gradient where ReLU clipped is dropped, whatever its value
template <int ACT> __device__ __forceinline__ float back_activate(float dy, float z) {
    if (ACT == COMBO_ACT_RELU) return z > 0.0f ? dy : 0.0f;
    if (ACT == COMBO_ACT_SILU) {
        const float s = __fdividef(1.0f, 1.0f + __expf(-z));
        return dy * (s * fmaf(z, 1.0f - s, 1.0f));
    }
    return dy;
}

// One slab: `nl` positions of `nv` vectors, thread = (row, column).  A vector is 16 bytes, V elements in V / 2 pairs;
// or (VEC = false) one element, twice in a pair whose upper half is ignored.
template <int EB, bool VEC> struct Lane {
    static constexpr int V = VEC ? Elem<EB>::V : 1;
    static constexpr int VB = V * EB;
    static constexpr int P = VEC ? V / 2 : 1;
    __device__ static __forceinline__ void unpack(uint32_t shared, f32x2 (&x)[P]) {
        if constexpr (VEC) {
            uint4 v;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(shared));
            widen(v, x);
        } else if constexpr (EB == 4) {
            float v;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(shared));
            x[0] = pair(v, v);
        } else {
            unsigned short v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(shared));
            const float f = __uint_as_float((uint32_t)v << 16);
            x[0] = pair(f, f);
        }
    }
    __device__ static __forceinline__ void unpack(const unsigned char* q, f32x2 (&x)[P]) {
        if constexpr (VEC) {
            widen(*reinterpret_cast<const uint4*>(q), x);
        } else {
            const float v = Elem<EB>::get(q);
            x[0] = pair(v, v);
        }
    }
    __device__ static __forceinline__ void widen(const uint4& v, f32x2 (&x)[P]) {
        if constexpr (VEC) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if constexpr (EB == 2) x[i] = pair(combo_step::widen_lo(w[i]), combo_step::widen_hi(w[i]));
                else x[i] = pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            }
        }
    }
    __device__ static __forceinline__ void store(void* q, const f32x2 (&x)[P]) {
        if constexpr (!VEC) Elem<EB>::put(q, lo_of(x[0]));
        else if constexpr (EB == 2)
            __stcs(static_cast<uint4*>(q), make_uint4(combo_step::pack_bf16(lo_of(x[0]), hi_of(x[0])), combo_step::pack_bf16(lo_of(x[1]), hi_of(x[1])),
                                                      combo_step::pack_bf16(lo_of(x[2]), hi_of(x[2])), combo_step::pack_bf16(lo_of(x[3]), hi_of(x[3]))));
        else __stcs(static_cast<ulonglong2*>(q), make_ulonglong2(x[0], x[1]));
    }
    // a vector's V floats of a table in shared memory
    __device__ static __forceinline__ void table(const float* t, f32x2 (&x)[P]) {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < P; ++i) x[i] = *reinterpret_cast<const f32x2*>(t + 2 * i);
        } else {
            x[0] = pair(t[0], t[0]);
        }
    }
    // Channels come in runs of `sub` that belong to one group: sums over each run, in every pair of the run.
    __device__ static __forceinline__ void fold(f32x2 (&x)[P], int sub) {
        if constexpr (VEC) {
            if (sub >= 2)
#pragma unroll
                for (int i = 0; i < P; ++i) { const float s = lo_of(x[i]) + hi_of(x[i]); x[i] = pair(s, s); }
            if (sub >= 4)
#pragma unroll
                for (int i = 0; i + 1 < P; i += 2) x[i] = x[i + 1] = add2(x[i], x[i + 1]);
            if constexpr (P == 4)
                if (sub >= 8) { x[0] = add2(x[0], x[2]); x[1] = x[2] = x[3] = x[0]; }
        }
    }
    // brings n vectors of one column, `step` bytes apart, into shared memory, `to_step` bytes apart
    __device__ static __forceinline__ void fetch(uint32_t to, uint32_t to_step, const unsigned char* q, long long step, int n) {
        if constexpr (VEC) {
#pragma unroll 4
            for (int k = 0; k < n; ++k, q += step, to += to_step)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(q) : "memory");
        } else if constexpr (EB == 4) {
#pragma unroll 4
            for (int k = 0; k < n; ++k, q += step, to += to_step)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(q) : "memory");
        } else {
            for (int k = 0; k < n; k += 8, q += 8 * step, to += 8 * to_step) {
                unsigned short v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + j < n) v[j] = *reinterpret_cast<const unsigned short*>(q + j * step);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + j < n) asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + j * to_step), "h"(v[j]) : "memory");
            }
        }
    }
};

// A thread's vectors of one column, one after another: in shared memory, or where they came from.
template <bool RES> struct Walk;
template <> struct Walk<true> {
    uint32_t q, step;
    __device__ __forceinline__ Walk(uint32_t slab, int vb, int nv, int rows, int trow, int col, const unsigned char*, long long)
        : q(slab + (uint32_t)((trow * nv + col) * vb)), step((uint32_t)(rows * nv * vb)) {}
    __device__ __forceinline__ void next() { q += step; }
};
template <> struct Walk<false> {
    const unsigned char* q;
    long long step;
    __device__ __forceinline__ Walk(uint32_t, int vb, int, int rows, int trow, int col, const unsigned char* g, long long pitch)
        : q(g + trow * pitch + col * vb), step(rows * pitch) {}
    __device__ __forceinline__ void next() { q += step; }
};

// What a CTA works on, the same in both directions.
template <int V> struct Place {
    int rank, g0, ng, c0, cb, nv, nl, l0, rows, cstep, trow, tcol, sub, base, extra;
    long long unit;
    __device__ __forceinline__ Place(const NormParams& p) {
        const int tid = threadIdx.x;
        rank = p.CS > 1 ? (int)cluster_rank() : 0;
        const unsigned u = blockIdx.x / (unsigned)p.CS;
        unit = u / (unsigned)p.nblk;
        g0 = (int)(u % (unsigned)p.nblk) * p.GB;
        ng = min(p.GB, p.G - g0);
        c0 = g0 * p.Cg;
        cb = ng * p.Cg;
        nv = cb / V;
        l0 = rank * p.Lc;
        nl = rank_len(p, rank);
        rows = nv < kThreads ? kThreads / nv : 1;
        cstep = nv < kThreads ? nv : kThreads;
        trow = tid / cstep;
        tcol = trow < rows ? tid - trow * cstep : nv;
        sub = p.sub;
        base = nl / rows;
        extra = nl - base * rows;
    }
    __device__ __forceinline__ int positions(int row) const { return base + (row < extra ? 1 : 0); }
};

// gamma and beta of the block's channels, for worker w
__device__ __forceinline__ void load_params(const NormParams& p, int w, int c0, int cb, float* ga, float* be) {
    for (int c = threadIdx.x; c < cb; c += kThreads) {
        ga[c] = p.gamma ? load_par(p.gamma, w * p.par_pitch + c0 + c, p.par_bytes) : 1.0f;
        be[c] = p.gamma ? load_par(p.beta, w * p.par_pitch + c0 + c, p.par_bytes) : 0.0f;
    }
}

// mean (negated) and rstd of a vector's channels, which begin at channel c of the block
template <typename Ln> __device__ __forceinline__ void group_pairs(const float2* fin, int c, int Cg, int sub, f32x2 (&m)[Ln::P], f32x2 (&rs)[Ln::P]) {
    if (sub == Ln::V) {                          // the whole vector in one group
        const float2 f = fin[c / Cg];
#pragma unroll
        for (int i = 0; i < Ln::P; ++i) { m[i] = pair(-f.x, -f.x); rs[i] = pair(f.y, f.y); }
    } else {
#pragma unroll
        for (int i = 0; i < Ln::P; ++i) {
            const float2 f = fin[(c + 2 * i) / Cg], e = fin[(c + 2 * i + 1) / Cg];
            m[i] = pair(-f.x, -e.x);
            rs[i] = pair(f.y, e.y);
        }
    }
}

template <int EB, bool VEC, bool RES, int ACT> __global__ void __launch_bounds__(kThreads, kCtasPerSm) k_norm(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB, P = Ln::P;
    extern __shared__ __align__(128) unsigned char smem[];
    float2* stat = reinterpret_cast<float2*>(smem + p.stat_off);       // [rows][cb / sub] mean, M2 of a thread's runs
    float* ga_s = reinterpret_cast<float*>(smem + p.par_off);          // [cb]
    float* be_s = ga_s + p.cb_max;                                     // [cb]
    float2* grp = reinterpret_cast<float2*>(smem + p.grp_off);         // [GB] this CTA's mean and M2, read by the cluster
    float2* fin = grp + p.GB;                                          // [GB] mean and rstd
    const uint32_t slab = smem_u32(smem + p.slab_off);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Place<V> at(p);
    const int nl = at.nl, nv = at.nv, rows = at.rows;
    const long long b = at.unit;
    const long long xp = p.x_pitch * EB, yp = p.y_pitch * EB;
    const unsigned char* x = p.x + (b * p.L + at.l0) * xp + (long long)at.c0 * EB;
    unsigned char* y = p.y + (b * p.L + at.l0) * yp + (long long)at.c0 * EB;
    const int n = at.positions(at.trow);        // of this thread
    const auto walk = [&](int col) { return Walk<RES>(slab, VB, nv, rows, at.trow, col, x, xp); };
    if (RES)
        for (int col = at.tcol; col < nv; col += at.cstep) {
            const Walk<true> to(slab, VB, nv, rows, at.trow, col, x, xp);
            Ln::fetch(to.q, to.step, x + at.trow * xp + col * VB, rows * xp, n);
        }
    load_params(p, worker_of(p, b), at.c0, at.cb, ga_s, be_s);
    if (RES) cp_async_wait();

    const int runs = at.cb / at.sub;
    const float inv = 1.0f / (float)max(n * at.sub, 1);
    for (int col = at.tcol; col < nv; col += at.cstep) {
        f32x2 m[P], q[P];
#pragma unroll
        for (int i = 0; i < P; ++i) m[i] = q[i] = 0;
        auto at_v = walk(col);
#pragma unroll 4
        for (int k = 0; k < n; ++k, at_v.next()) {
            f32x2 v[P];
            Ln::unpack(at_v.q, v);
#pragma unroll
            for (int i = 0; i < P; ++i) m[i] = add2(m[i], v[i]);
        }
        Ln::fold(m, at.sub);
#pragma unroll
        for (int i = 0; i < P; ++i) m[i] = neg2(mul2(m[i], pair(inv, inv)));
        at_v = walk(col);
#pragma unroll 4
        for (int k = 0; k < n; ++k, at_v.next()) {
            f32x2 v[P];
            Ln::unpack(at_v.q, v);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const f32x2 d = add2(v[i], m[i]);
                q[i] = fma2(d, d, q[i]);
            }
        }
        Ln::fold(q, at.sub);
        float2* mine = stat + at.trow * runs + col * V / at.sub;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (2 * i % at.sub == 0) mine[2 * i / at.sub] = make_float2(-lo_of(m[i]), lo_of(q[i]));
            if (VEC && at.sub == 1) mine[2 * i + 1] = make_float2(-hi_of(m[i]), hi_of(q[i]));
        }
    }
    __syncthreads();
    // a warp per group: merge of rows * (Cg / sub) entries, each with the count of its row
    const int per = p.Cg / at.sub;
    for (int g = warp; g < at.ng; g += kWarps) {
        const int entries = rows * per;
        float s = 0.0f, q = 0.0f;
        for (int i = lane; i < entries; i += 32) {
            const int r = per == 1 ? i : i / per;
            s = fmaf((float)(at.positions(r) * at.sub), stat[r * runs + g * per + i - r * per].x, s);
        }
        const float m = nl > 0 ? warp_sum(s) / (float)((long long)nl * p.Cg) : 0.0f;
        for (int i = lane; i < entries; i += 32) {
            const int r = per == 1 ? i : i / per;
            const float2 e = stat[r * runs + g * per + i - r * per];
            const float d = e.x - m;
            q += fmaf((float)(at.positions(r) * at.sub) * d, d, e.y);
        }
        q = warp_sum(q);
        if (lane == 0) grp[g] = make_float2(m, q);
    }
    if (p.CS > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
    for (int g = tid; g < at.ng; g += kThreads) {
        const float total = (float)((long long)p.L * p.Cg);
        float m = grp[g].x, q = grp[g].y;
        if (p.CS > 1) {
            float2 e[kMaxCluster];
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r)
                if (r < p.CS) e[r] = peer_float2(grp + g, r);
            float s = 0.0f;
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r)
                if (r < p.CS) s = fmaf((float)((long long)rank_len(p, r) * p.Cg), e[r].x, s);
            m = s / total;
            q = 0.0f;
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r)
                if (r < p.CS) {
                    const float d = e[r].x - m;
                    q += fmaf((float)((long long)rank_len(p, r) * p.Cg) * d, d, e[r].y);
                }
        }
        const float rs = 1.0f / sqrtf(q / total + p.eps);
        fin[g] = make_float2(m, rs);
        if (at.rank == 0) {
            if (p.mean) p.mean[b * p.G + at.g0 + g] = m;
            if (p.rstd) p.rstd[b * p.G + at.g0 + g] = rs;
        }
    }
    __syncthreads();
    if (p.CS > 1) cluster_done();               // peers' sums are read; waited for before this CTA leaves
    for (int col = at.tcol; col < nv; col += at.cstep) {
        f32x2 m[P], rs[P], ga[P], be[P];
        group_pairs<Ln>(fin, col * V, p.Cg, at.sub, m, rs);
        Ln::table(ga_s + col * V, ga);
        Ln::table(be_s + col * V, be);
        auto at_v = walk(col);
        unsigned char* to = y + at.trow * yp + col * VB;
#pragma unroll 4
        for (int k = 0; k < n; ++k, at_v.next(), to += rows * yp) {
            f32x2 v[P];
            Ln::unpack(at_v.q, v);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const f32x2 z = affine(normed(v[i], m[i], rs[i]), ga[i], be[i]);
                v[i] = pair(activate<ACT>(lo_of(z)), activate<ACT>(hi_of(z)));
            }
            Ln::store(to, v);
        }
    }
    if (p.CS > 1) cluster_wait();
}

template <int EB, bool VEC, bool RES, int ACT> __global__ void __launch_bounds__(kThreads, kCtasPerSm) k_norm_back(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB, P = Ln::P;
    extern __shared__ __align__(128) unsigned char smem[];
    float4* stat = reinterpret_cast<float4*>(smem + p.stat_off);       // [P][rows][nv] a thread's sums of dz * h and of dz, by pairs of channels
    float* ga_s = reinterpret_cast<float*>(smem + p.par_off);          // [cb]
    float* be_s = ga_s + p.cb_max;                                     // [cb]
    float2* grp = reinterpret_cast<float2*>(smem + p.grp_off);         // [GB] sums of t and t * h of this CTA
    float2* fin = grp + p.GB;                                          // [GB] their means over the whole slab
    float2* norm = fin + p.GB;                                         // [GB] mean and rstd
    float2* chan = norm + p.GB;                                        // [cb] this CTA's sums per channel
    float2* acc = chan + p.cb_max;                                     // [cb] the same over the worker's samples
    const uint32_t slab = smem_u32(smem + p.slab_off);
    combo_step::pdl_release();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Place<V> at(p);
    const int nl = at.nl, nv = at.nv, rows = at.rows, cb = at.cb;
    const long long xp = p.x_pitch * EB, yp = p.y_pitch * EB, dp = p.dy_pitch * EB;
    const long long b0 = at.unit * p.ns, b1 = min(b0 + p.ns, p.B);
    const float inv = 1.0f / (float)((long long)p.L * p.Cg);
    const int n = at.positions(at.trow);        // of this thread
    // rows of the table of sums are added in `parts` lots side by side, then the lots
    const int pairs = nv * P, parts = min(max(kThreads / pairs, 1), rows);
    const auto add_channel = [&](int c, float2 s) {
        chan[c] = s;
        if (p.CS == 1) acc[c] = make_float2(acc[c].x + s.x, acc[c].y + s.y);
    };
    int w = -1;
    long long wb = b0;                          // the worker's first sample here
    for (long long b = b0; b < b1; ++b) {
        const long long first = b * p.L + at.l0;
        const unsigned char* x = p.x + first * xp + (long long)at.c0 * EB;
        const unsigned char* dy = p.dy + first * dp + (long long)at.c0 * EB;
        unsigned char* dx = p.y + first * yp + (long long)at.c0 * EB;
        if (RES) {
            for (int col = at.tcol; col < nv; col += at.cstep) {
                const Walk<true> to(slab, VB, nv, rows, at.trow, col, x, xp);
                Ln::fetch(to.q, to.step, x + at.trow * xp + col * VB, rows * xp, n);
                Ln::fetch(to.q + p.slab_bytes, to.step, dy + at.trow * dp + col * VB, rows * dp, n);
            }
        }
        const int owner = worker_of(p, b);
        if (owner != w) {                       // (behind worker_of's or the loop's barrier) the channels' sums of the worker before leave for its slot
            for (int c = tid; c < cb; c += kThreads) {
                if (w >= 0) p.partial[wb * p.C + at.c0 + c] = acc[c];
                acc[c] = make_float2(0.0f, 0.0f);
            }
            load_params(p, owner, at.c0, cb, ga_s, be_s);
            w = owner;
            wb = b;
        }
        for (int g = tid; g < at.ng; g += kThreads) norm[g] = make_float2(p.mean[b * p.G + at.g0 + g], p.rstd[b * p.G + at.g0 + g]);
        __syncthreads();
        if (RES) cp_async_wait();
        const auto walk = [&](int col) { return Walk<RES>(slab, VB, nv, rows, at.trow, col, x, xp); };
        const auto dwalk = [&](int col) { return Walk<RES>(slab + p.slab_bytes, VB, nv, rows, at.trow, col, dy, dp); };
        for (int col = at.tcol; col < nv; col += at.cstep) {
            f32x2 m[P], rs[P], ga[P], be[P], s1[P], s2[P];
            group_pairs<Ln>(norm, col * V, p.Cg, at.sub, m, rs);
            Ln::table(ga_s + col * V, ga);
            Ln::table(be_s + col * V, be);
#pragma unroll
            for (int i = 0; i < P; ++i) s1[i] = s2[i] = 0;
            auto at_v = walk(col);
            auto at_d = dwalk(col);
#pragma unroll 2
            for (int k = 0; k < n; ++k, at_v.next(), at_d.next()) {
                f32x2 v[P], d[P];
                Ln::unpack(at_v.q, v);
                Ln::unpack(at_d.q, d);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const f32x2 h = normed(v[i], m[i], rs[i]), z = affine(h, ga[i], be[i]);
                    const f32x2 dz = pair(back_activate<ACT>(lo_of(d[i]), lo_of(z)), back_activate<ACT>(hi_of(d[i]), hi_of(z)));
                    s1[i] = fma2(dz, h, s1[i]);
                    s2[i] = add2(s2[i], dz);
                }
            }
#pragma unroll
            for (int i = 0; i < P; ++i)
                stat[(i * rows + at.trow) * nv + col] = make_float4(lo_of(s1[i]), hi_of(s1[i]), lo_of(s2[i]), hi_of(s2[i]));
        }
        __syncthreads();
        if (parts > 1) {                         // pair k = (i, col): its rows lie nv entries apart
            const int part = tid / pairs, k = tid - part * pairs, i = k / nv;
            float4* mine = stat + i * (rows - 1) * nv + k;
            if (part < parts) {
                float4 s = mine[part * nv];
                for (int r = part + parts; r < rows; r += parts) {
                    const float4 e = mine[r * nv];
                    s.x += e.x; s.y += e.y; s.z += e.z; s.w += e.w;
                }
                mine[part * nv] = s;             // row `part` is read by this thread alone
            }
            __syncthreads();
        }
        for (int k = tid; k < pairs; k += kThreads) {
            const int i = k / nv, col = k - i * nv;
            const float4* mine = stat + i * rows * nv + col;
            float4 s = mine[0];
            for (int r = 1; r < parts; ++r) {
                const float4 e = mine[r * nv];
                s.x += e.x; s.y += e.y; s.z += e.z; s.w += e.w;
            }
            const int c = col * V + 2 * i;
            add_channel(c, make_float2(s.x, s.z));
            if (VEC) add_channel(c + 1, make_float2(s.y, s.w));
        }
        __syncthreads();
        for (int g = warp; g < at.ng; g += kWarps) {
            float t = 0.0f, th = 0.0f;
            for (int c = g * p.Cg + lane; c < (g + 1) * p.Cg; c += 32) {
                const float2 s = chan[c];
                th = fmaf(ga_s[c], s.x, th);
                t = fmaf(ga_s[c], s.y, t);
            }
            t = warp_sum(t);
            th = warp_sum(th);
            if (lane == 0) grp[g] = make_float2(t, th);
        }
        if (p.CS > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
        for (int g = tid; g < at.ng; g += kThreads) {
            float2 s = p.CS > 1 ? make_float2(0.0f, 0.0f) : grp[g];
            for (int r = 0; p.CS > 1 && r < p.CS; ++r) {
                const float2 e = peer_float2(grp + g, r);
                s.x += e.x;
                s.y += e.y;
            }
            fin[g] = make_float2(s.x * inv, s.y * inv);
        }
        if (p.CS > 1) {                          // the cluster's CTAs share the channels among them
            for (int c = tid * p.CS + at.rank; c < cb; c += kThreads * p.CS) {
                float2 s = make_float2(0.0f, 0.0f);
                for (int r = 0; r < p.CS; ++r) {
                    const float2 e = peer_float2(chan + c, r);
                    s.x += e.x;
                    s.y += e.y;
                }
                p.partial[b * p.C + at.c0 + c] = s;
            }
        }
        __syncthreads();
        if (p.CS > 1) cluster_done();
        for (int col = at.tcol; col < nv; col += at.cstep) {
            f32x2 m[P], rs[P], ga[P], be[P], m1[P], m2[P];
            group_pairs<Ln>(norm, col * V, p.Cg, at.sub, m, rs);
            group_pairs<Ln>(fin, col * V, p.Cg, at.sub, m1, m2);
            Ln::table(ga_s + col * V, ga);
            Ln::table(be_s + col * V, be);
            auto at_v = walk(col);
            auto at_d = dwalk(col);
            unsigned char* to = dx + at.trow * yp + col * VB;
#pragma unroll 2
            for (int k = 0; k < n; ++k, at_v.next(), at_d.next(), to += rows * yp) {
                f32x2 v[P], d[P];
                Ln::unpack(at_v.q, v);
                Ln::unpack(at_d.q, d);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const f32x2 h = normed(v[i], m[i], rs[i]), z = affine(h, ga[i], be[i]);
                    const f32x2 dz = pair(back_activate<ACT>(lo_of(d[i]), lo_of(z)), back_activate<ACT>(hi_of(d[i]), hi_of(z)));
                    v[i] = mul2(rs[i], fma2(neg2(h), m2[i], fma2(dz, ga[i], m1[i])));    // m1 comes negated
                }
                Ln::store(to, v);
            }
        }
        if (p.CS > 1) cluster_wait();            // ns is 1 here: the last thing this CTA does
        else __syncthreads();                    // the tables are free for the next sample
    }
    if (p.CS == 1)                               // the loop's last barrier has made acc whole
        for (int c = tid; c < cb; c += kThreads) p.partial[wb * p.C + at.c0 + c] = acc[c];
}

// dgamma and dbeta of worker blockIdx.y: what each CTA left at its first sample of the worker, added in a fixed order.
constexpr int kSumRows = 8;
__global__ void __launch_bounds__(32 * kSumRows) k_norm_params(const NormParams p, float* dgamma, float* dbeta, long long pitch) {
    __shared__ float2 sh[kSumRows][32];
    combo_step::pdl_wait();
    const int w = blockIdx.y, lane = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    const long long s0 = p.begin ? max((long long)p.begin[w], 0LL) : 0;
    const long long s1 = p.begin ? min((long long)p.begin[w + 1], p.B) : p.B;
    float2 s = make_float2(0.0f, 0.0f);
    if (c < p.C && s0 < s1) {
        const long long k0 = s0 / p.ns, k1 = (s1 - 1) / p.ns;
#pragma unroll 4
        for (long long k = k0 + row; k <= k1; k += kSumRows) {
            const float2 e = p.partial[max(k * p.ns, s0) * p.C + c];
            s.x += e.x;
            s.y += e.y;
        }
    }
    sh[row][lane] = s;
    __syncthreads();
    if (row == 0 && c < p.C) {
        s = sh[0][lane];
#pragma unroll
        for (int r = 1; r < kSumRows; ++r) { s.x += sh[r][lane].x; s.y += sh[r][lane].y; }
        dgamma[w * pitch + c] = s.x;
        dbeta[w * pitch + c] = s.y;
    }
}

// ---------------------------------------------------------------- host
constexpr unsigned kSlabTarget = 50 * 1024;     // shared memory of a CTA's slab aimed at: four CTAs on an SM
constexpr int kRowBytes = 128;                  // least bytes of a position that a block of groups takes
constexpr int kMaxChannels = COMBO_NORM_MAX_CHANNELS;   // of a block of groups: bounds the tables in shared memory (40 bytes each)
constexpr int kShortSample = 32;                // positions under which a CTA of the backward pass takes several samples

struct Plan {
    bool vec, res;
    size_t smem;
    long long grid;
};

int samples_per_cta(int L) { return L >= kShortSample ? 1 : (kShortSample + L - 1) / L; }

combo_status plan_norm(NormParams& p, Plan& plan, int eb, bool vec, bool back, int sms, int smem_optin) {
    const int V = vec ? 16 / eb : 1, arrays = back ? 2 : 1;
    // whole groups, at least kRowBytes of a position, whole vectors
    int GB = 1;
    while (GB < p.G && (GB * p.Cg * eb < kRowBytes || GB * p.Cg % V != 0)) ++GB;
    if (vec && (long long)GB * p.Cg > kMaxChannels) return plan_norm(p, plan, eb, false, back, sms, smem_optin);
    p.GB = GB;
    p.nblk = (p.G + GB - 1) / GB;
    p.ns = back ? samples_per_cta(p.L) : 1;
    const long long cb = (long long)GB * p.Cg;
    p.cb_max = (int)(cb + 3) / 4 * 4;
    const long long chunks = (p.B + p.ns - 1) / p.ns, units = chunks * p.nblk;
    const long long nv = cb / V, rows = nv < kThreads ? kThreads / nv : 1;
    p.sub = 1;
    while (p.sub < V && p.Cg % (2 * p.sub) == 0) p.sub *= 2;
    // forward: rows * cb / sub entries of 8 bytes, backward: 16 bytes for every pair of channels; the last block of
    // groups may be narrower and have more rows, but never more than kThreads vectors
    const long long vecs = nv > kThreads ? nv : kThreads;
    const unsigned long long stat = (unsigned long long)vecs * (back ? (V > 1 ? V / 2 : 1) * 16 : V / p.sub * 8), grp = (3ull * GB + (back ? 2 * p.cb_max : 0)) * 8;
    const auto round = [](unsigned long long v) { return (v + 127) / 128 * 128; };
    const unsigned long long par = 8ull * p.cb_max, fixed = round(stat) + round(par) + round(grp);
    const unsigned long long room = (unsigned long long)smem_optin - fixed;
    int CS = 1;
    const auto slab = [&](int cs) { return round((unsigned long long)((p.L + cs - 1) / cs) * cb * eb); };
    // small slabs let several CTAs share an SM (one loads while others store); and no SM is left idle
    while (CS < kMaxCluster && (arrays * slab(CS) > kSlabTarget || (units * CS * 2 <= sms && p.L >= 2 * CS * rows))) CS *= 2;
    plan.res = arrays * slab(CS) <= room;
    p.CS = CS;
    if (CS > 1) p.ns = 1;
    p.Lc = (p.L + CS - 1) / CS;
    p.stat_off = 0;
    p.par_off = (unsigned)round(stat);
    p.grp_off = (unsigned)(round(stat) + round(par));
    p.slab_off = (unsigned)fixed;
    p.slab_bytes = (unsigned)(plan.res ? slab(CS) : 0);
    plan.vec = vec;
    plan.smem = fixed + (plan.res ? arrays * slab(CS) : 0);
    plan.grid = (p.B + p.ns - 1) / p.ns * p.nblk * CS;
    return plan.grid > 0x7fffffffLL ? COMBO_ERR_INVALID_ARG : COMBO_OK;
}

// `which`: a number of its own for every kernel
cudaError_t launch_norm(void (*kern)(NormParams), int which, const NormParams& p, const Plan& plan, int smem_optin, cudaStream_t st) {
    static uint64_t allowed[48];
    cudaError_t e = combo_host::allow_smem(kern, smem_optin, &allowed[which]);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)plan.grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = plan.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.CS;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.CS > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

typedef void (*NormKernel)(NormParams);
template <int EB, bool VEC, bool RES> NormKernel pick_act(bool back, int act) {
    switch (act) {
        case COMBO_ACT_RELU: return back ? k_norm_back<EB, VEC, RES, COMBO_ACT_RELU> : k_norm<EB, VEC, RES, COMBO_ACT_RELU>;
        case COMBO_ACT_SILU: return back ? k_norm_back<EB, VEC, RES, COMBO_ACT_SILU> : k_norm<EB, VEC, RES, COMBO_ACT_SILU>;
        default: return back ? k_norm_back<EB, VEC, RES, COMBO_ACT_NONE> : k_norm<EB, VEC, RES, COMBO_ACT_NONE>;
    }
}
template <int EB> NormKernel pick(bool back, bool vec, bool res, int act) {
    if (vec) return res ? pick_act<EB, true, true>(back, act) : pick_act<EB, true, false>(back, act);
    return res ? pick_act<EB, false, true>(back, act) : pick_act<EB, false, false>(back, act);
}

int number_of(int eb, bool back, const Plan& plan, int act) {
    return (((eb == 4 ? 1 : 0) * 2 + back) * 2 + plan.vec) * 2 * 3 + plan.res * 3 + act;
}

// What forward and backward ask alike.
combo_status check_shape(int elem_bytes, int param_bytes, const void* gamma, const void* beta, int64_t param_pitch,
                         const int64_t* begin, int N, int64_t B, int64_t L, int64_t C, int groups, int act) {
    if (elem_bytes != 4 && elem_bytes != 2) return COMBO_ERR_INVALID_ARG;
    if (N < 1 || N > COMBO_MAX_WORKERS || B < 0 || L < 1 || C < 1 || groups < 1 || groups > C || C % groups != 0)
        return COMBO_ERR_INVALID_ARG;
    if (C / groups > kMaxChannels) return COMBO_ERR_INVALID_ARG;
    if (L > (1 << 28) || C > (1 << 20) || B > (1LL << 40) / L / C) return COMBO_ERR_INVALID_ARG;
    if (act < COMBO_ACT_NONE || act > COMBO_ACT_SILU) return COMBO_ERR_INVALID_ARG;
    if ((gamma == nullptr) != (beta == nullptr) || (!begin && N != 1)) return COMBO_ERR_INVALID_ARG;
    if (gamma && ((param_bytes != 4 && param_bytes != 2) || (N > 1 && param_pitch < C) ||
                  !combo_host::aligned_to(gamma, param_bytes) || !combo_host::aligned_to(beta, param_bytes)))
        return COMBO_ERR_INVALID_ARG;
    if (!combo_host::aligned_to(begin, 8)) return COMBO_ERR_INVALID_ARG;
    return COMBO_OK;
}

bool array_ok(const void* p, int64_t pitch, int64_t C, int eb) {
    return p && combo_host::aligned_to(p, eb) && pitch >= C && pitch <= (1LL << 40) / C;
}
size_t extent(int64_t B, int64_t L, int64_t C, int64_t pitch, int eb) { return B < 1 ? 0 : (size_t)((B * L - 1) * pitch + C) * eb; }
bool vec_ok(const void* p, int64_t pitch, int eb) { return combo_host::aligned_to(p, 16) && pitch * eb % 16 == 0; }
// an output may be an input, element for element; it may not overlap it in any other way
bool clash(const void* out, int64_t out_pitch, size_t out_n, const void* in, int64_t in_pitch, size_t in_n) {
    return combo_host::overlap(out, out_n, in, in_n) && !(out == in && out_pitch == in_pitch);
}

}  // namespace

extern "C" {

size_t combo_group_norm_scratch_bytes(int64_t B, int64_t L, int64_t C) {
    if (B < 0 || L < 1 || C < 1 || L > (1 << 28) || C > (1 << 20) || B > (1LL << 40) / L / C)
        return 0;
    return (size_t)(B < 1 ? 1 : B) * (size_t)C * sizeof(float2);
}

combo_status combo_group_norm(const void* x, int64_t x_pitch, void* y, int64_t y_pitch, int elem_bytes, const void* gamma,
                              const void* beta, int param_bytes, int64_t param_pitch, const int64_t* d_begin, int N,
                              int64_t B, int64_t L, int64_t C, int groups, float eps, int act, float* mean_out,
                              float* rstd_out, void* stream) {
    combo_status rc = check_shape(elem_bytes, param_bytes, gamma, beta, param_pitch, d_begin, N, B, L, C, groups, act);
    if (rc != COMBO_OK) return rc;
    if (!(eps >= 0.0f)) return COMBO_ERR_INVALID_ARG;
    if (B == 0) return COMBO_OK;
    if (!array_ok(x, x_pitch, C, elem_bytes) || !array_ok(y, y_pitch, C, elem_bytes)) return COMBO_ERR_INVALID_ARG;
    if (!combo_host::aligned_to(mean_out, 4) || !combo_host::aligned_to(rstd_out, 4)) return COMBO_ERR_INVALID_ARG;
    if (clash(y, y_pitch, extent(B, L, C, y_pitch, elem_bytes), x, x_pitch, extent(B, L, C, x_pitch, elem_bytes)))
        return COMBO_ERR_ALIAS;
    int sms = 0, smem = 0;
    if ((rc = combo_host::device(&sms, &smem)) != COMBO_OK) return rc;
    NormParams p = {};
    p.x = static_cast<const unsigned char*>(x);
    p.y = static_cast<unsigned char*>(y);
    p.gamma = static_cast<const unsigned char*>(gamma);
    p.beta = static_cast<const unsigned char*>(beta);
    p.begin = d_begin;
    p.mean = mean_out;
    p.rstd = rstd_out;
    p.x_pitch = x_pitch;
    p.y_pitch = y_pitch;
    p.par_pitch = N > 1 ? param_pitch : 0;
    p.par_bytes = param_bytes;
    p.B = B;
    p.L = (int)L;
    p.C = (int)C;
    p.G = groups;
    p.Cg = (int)(C / groups);
    p.N = N;
    p.eps = eps;
    const bool vec = C * elem_bytes % 16 == 0 && vec_ok(x, x_pitch, elem_bytes) && vec_ok(y, y_pitch, elem_bytes);
    Plan plan;
    if ((rc = plan_norm(p, plan, elem_bytes, vec, false, sms, smem)) != COMBO_OK) return rc;
    auto kern = elem_bytes == 4 ? pick<4>(false, plan.vec, plan.res, act) : pick<2>(false, plan.vec, plan.res, act);
    cudaError_t e = launch_norm(kern, number_of(elem_bytes, false, plan, act), p, plan, smem, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "group norm launch");
}

combo_status combo_group_norm_backward(const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch, void* dx,
                                       int64_t dx_pitch, int elem_bytes, const void* gamma, const void* beta,
                                       int param_bytes, int64_t param_pitch, const int64_t* d_begin, int N, int64_t B,
                                       int64_t L, int64_t C, int groups, int act, const float* mean, const float* rstd,
                                       float* dgamma, float* dbeta, int64_t grad_pitch, void* scratch,
                                       size_t scratch_bytes, void* stream) {
    combo_status rc = check_shape(elem_bytes, param_bytes, gamma, beta, param_pitch, d_begin, N, B, L, C, groups, act);
    if (rc != COMBO_OK) return rc;
    if ((dgamma == nullptr) != (dbeta == nullptr) || (dgamma && N > 1 && grad_pitch < C)) return COMBO_ERR_INVALID_ARG;
    if (!combo_host::aligned_to(dgamma, 4) || !combo_host::aligned_to(dbeta, 4)) return COMBO_ERR_INVALID_ARG;
    if (!scratch || !combo_host::aligned_to(scratch, 8) || scratch_bytes < combo_group_norm_scratch_bytes(B, L, C))
        return COMBO_ERR_INVALID_ARG;
    int sms = 0, smem = 0;
    NormParams p = {};
    p.begin = d_begin;
    p.partial = static_cast<float2*>(scratch);
    p.B = B;
    p.C = (int)C;
    p.N = N;
    p.ns = 1;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (B > 0) {
        if (!array_ok(x, x_pitch, C, elem_bytes) || !array_ok(dy, dy_pitch, C, elem_bytes) ||
            !array_ok(dx, dx_pitch, C, elem_bytes) || !mean || !rstd)
            return COMBO_ERR_INVALID_ARG;
        if (!combo_host::aligned_to(mean, 4) || !combo_host::aligned_to(rstd, 4)) return COMBO_ERR_INVALID_ARG;
        const size_t n = extent(B, L, C, dx_pitch, elem_bytes);
        if (clash(dx, dx_pitch, n, x, x_pitch, extent(B, L, C, x_pitch, elem_bytes)) ||
            clash(dx, dx_pitch, n, dy, dy_pitch, extent(B, L, C, dy_pitch, elem_bytes)))
            return COMBO_ERR_ALIAS;
    }
    if ((rc = combo_host::device(&sms, &smem)) != COMBO_OK) return rc;
    if (B > 0) {
        p.x = static_cast<const unsigned char*>(x);
        p.dy = static_cast<const unsigned char*>(dy);
        p.y = static_cast<unsigned char*>(dx);
        p.gamma = static_cast<const unsigned char*>(gamma);
        p.beta = static_cast<const unsigned char*>(beta);
        p.mean = const_cast<float*>(mean);
        p.rstd = const_cast<float*>(rstd);
        p.x_pitch = x_pitch;
        p.y_pitch = dx_pitch;
        p.dy_pitch = dy_pitch;
        p.par_pitch = N > 1 ? param_pitch : 0;
        p.par_bytes = param_bytes;
        p.L = (int)L;
        p.G = groups;
        p.Cg = (int)(C / groups);
        const bool vec = C * elem_bytes % 16 == 0 && vec_ok(x, x_pitch, elem_bytes) && vec_ok(dx, dx_pitch, elem_bytes) &&
                         vec_ok(dy, dy_pitch, elem_bytes);
        Plan plan;
        if ((rc = plan_norm(p, plan, elem_bytes, vec, true, sms, smem)) != COMBO_OK) return rc;
        auto kern = elem_bytes == 4 ? pick<4>(true, plan.vec, plan.res, act) : pick<2>(true, plan.vec, plan.res, act);
        if ((e = launch_norm(kern, number_of(elem_bytes, true, plan, act), p, plan, smem, st)) != cudaSuccess) return combo_host::fail(e, "group norm backward launch");
    }
    if (dgamma) {
        const dim3 grid((unsigned)((C + 31) / 32), (unsigned)N);
        e = combo_host::launch_after(k_norm_params, grid, dim3(32 * kSumRows), 0, st, p, dgamma, dbeta, (long long)(N > 1 ? grad_pitch : 0));
        if (e != cudaSuccess) return combo_host::fail(e, "group norm parameter gradient launch");
    }
    return COMBO_OK;
}

}  // extern "C"
