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
// memory.  Every thread works on the vectors it loaded itself (thread = column + row, rows apart), so no barrier
// stands between loading and the first pass.  Slabs that 8 CTAs cannot hold are read again from global memory (L2)
// in place of shared memory (RES = false).
//
// Forward statistics: each thread takes mean and M2 (sum of squared deviations from its own mean) per channel of its
// positions, and these are merged by counts: sum of n_i * mean_i for the mean, M2_i + n_i (mean_i - mean)^2 for M2.
// Nothing is cancelled, whatever the size of the mean.
//
// z is formed in the roundings of the formula as written (no FMA), in both directions alike: a value that the forward
// pass clipped at zero is a value whose gradient the backward pass drops.
#include "host_common.h"
#include "step_common.cuh"

namespace {

using combo_step::Elem;
using combo_step::warp_sum;

constexpr int kThreads = 256;
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
    int L, C, G, Cg, GB, nblk, CS, Lc, N, act, ns, par_bytes;
    float eps;
    unsigned stat_off, grp_off, slab_off, slab_bytes;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
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
__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
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

__device__ __forceinline__ float normed(float x, float mean, float rstd) { return __fmul_rn(__fsub_rn(x, mean), rstd); }
__device__ __forceinline__ float affine(float h, float gamma, float beta) { return __fadd_rn(__fmul_rn(h, gamma), beta); }
// ReLU keeps NaN.  SiLU: the fast exponential and division are within a few units of binary32's last place over the
// range where the result is not lost in rounding (the accurate ones took the kernel from memory to issue bound).
__device__ __forceinline__ float activate(float z, int act) {
    if (act == COMBO_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (act == COMBO_ACT_SILU) return __fdividef(z, 1.0f + __expf(-z));
    return z;
}
// dy * act'(z); a gradient where ReLU clipped is dropped, whatever its value
__device__ __forceinline__ float back_activate(float dy, float z, int act) {
    if (act == COMBO_ACT_RELU) return z > 0.0f ? dy : 0.0f;
    if (act == COMBO_ACT_SILU) {
        const float s = __fdividef(1.0f, 1.0f + __expf(-z));
        return dy * (s * fmaf(z, 1.0f - s, 1.0f));
    }
    return dy;
}

// One slab: `nl` positions of `nv` vectors (V elements each), thread = (row, column).
template <int EB, bool VEC> struct Lane {
    static constexpr int V = VEC ? Elem<EB>::V : 1;
    static constexpr int VB = V * EB;
    __device__ static __forceinline__ void unpack(const void* q, float (&x)[V]) {
        if constexpr (VEC) Elem<EB>::unpack(*static_cast<const uint4*>(q), x);
        else x[0] = Elem<EB>::get(q);
    }
    __device__ static __forceinline__ void store(void* q, const float (&x)[V]) {
        if constexpr (VEC) __stcs(static_cast<uint4*>(q), Elem<EB>::pack(x));
        else Elem<EB>::put(q, x[0]);
    }
    // brings a thread's share of the slab into shared memory
    __device__ static __forceinline__ void fetch(unsigned char* slab, const unsigned char* src, long long pitch_bytes, int nl,
                                                 int nv, int rows, int trow, int tcol, int cstep) {
        for (int col = tcol; col < nv; col += cstep) {
            if constexpr (VEC) {
                for (int l = trow; l < nl; l += rows) cp_async16(slab + ((long long)l * nv + col) * VB, src + l * pitch_bytes + col * VB);
            } else {
                typedef typename Elem<EB>::type T;
                for (int l = trow; l < nl; l += 8 * rows) {
                    T v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (l + j * rows < nl) v[j] = *reinterpret_cast<const T*>(src + (l + j * rows) * pitch_bytes + col * VB);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (l + j * rows < nl) *reinterpret_cast<T*>(slab + ((long long)(l + j * rows) * nv + col) * VB) = v[j];
                }
            }
        }
    }
};

template <int EB, bool VEC, bool RES> __global__ void __launch_bounds__(kThreads) k_norm(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB;
    extern __shared__ __align__(128) unsigned char smem[];
    float2* stat = reinterpret_cast<float2*>(smem + p.stat_off);       // [rows][cb] mean, M2 of a thread's channels
    float2* grp = reinterpret_cast<float2*>(smem + p.grp_off);         // [GB] this CTA's mean and M2, read by the cluster
    float2* fin = grp + p.GB;                                          // [GB] mean and rstd
    unsigned char* slab = smem + p.slab_off;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = p.CS > 1 ? (int)cluster_rank() : 0;
    const long long unit = blockIdx.x / p.CS;
    const long long b = unit / p.nblk;
    const int g0 = (int)(unit % p.nblk) * p.GB, ng = min(p.GB, p.G - g0);
    const int c0 = g0 * p.Cg, cb = ng * p.Cg, nv = cb / V;
    const int l0 = rank * p.Lc, nl = rank_len(p, rank);
    const int rows = nv < kThreads ? kThreads / nv : 1;
    const int cstep = nv < kThreads ? nv : kThreads;
    const int trow = tid / cstep, tcol = trow < rows ? tid % cstep : nv;
    const long long xp = p.x_pitch * EB, yp = p.y_pitch * EB;
    const unsigned char* x = p.x + (b * p.L + l0) * xp + (long long)c0 * EB;
    unsigned char* y = p.y + (b * p.L + l0) * yp + (long long)c0 * EB;
    if (RES) Ln::fetch(slab, x, xp, nl, nv, rows, trow, tcol, cstep);
    const int w = worker_of(p, b);
    if (RES) cp_async_wait();
    const unsigned char* src = RES ? slab : x;
    const long long sp = RES ? (long long)nv * VB : xp;

    const int mine = nl > trow ? (nl - trow + rows - 1) / rows : 0;     // positions of this thread
    for (int col = tcol; col < nv; col += cstep) {
        float m[V], q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) m[i] = q[i] = 0.0f;
#pragma unroll 4
        for (int l = trow; l < nl; l += rows) {
            float v[V];
            Ln::unpack(src + l * sp + col * VB, v);
#pragma unroll
            for (int i = 0; i < V; ++i) m[i] += v[i];
        }
        const float inv = mine ? 1.0f / (float)mine : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) m[i] *= inv;
#pragma unroll 4
        for (int l = trow; l < nl; l += rows) {
            float v[V];
            Ln::unpack(src + l * sp + col * VB, v);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = v[i] - m[i];
                q[i] = fmaf(d, d, q[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) stat[trow * cb + col * V + i] = make_float2(m[i], q[i]);
    }
    __syncthreads();
    // a warp per group: merge of rows * Cg entries, entry (r, c) with the count of row r
    for (int g = warp; g < ng; g += kWarps) {
        const int n = rows * p.Cg;
        float s = 0.0f, q = 0.0f;
        for (int i = lane; i < n; i += 32) {
            const int r = i / p.Cg, c = i - r * p.Cg;
            const int cnt = nl > r ? (nl - r + rows - 1) / rows : 0;
            s = fmaf((float)cnt, stat[r * cb + g * p.Cg + c].x, s);
        }
        const float m = nl > 0 ? warp_sum(s) / (float)((long long)nl * p.Cg) : 0.0f;
        for (int i = lane; i < n; i += 32) {
            const int r = i / p.Cg, c = i - r * p.Cg;
            const int cnt = nl > r ? (nl - r + rows - 1) / rows : 0;
            const float2 e = stat[r * cb + g * p.Cg + c];
            const float d = e.x - m;
            q += fmaf((float)cnt * d, d, e.y);
        }
        q = warp_sum(q);
        if (lane == 0) grp[g] = make_float2(m, q);
    }
    if (p.CS > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
    for (int g = tid; g < ng; g += kThreads) {
        const float total = (float)((long long)p.L * p.Cg);
        float m, q;
        if (p.CS > 1) {
            float s = 0.0f;
            q = 0.0f;
            for (int r = 0; r < p.CS; ++r) s = fmaf((float)((long long)rank_len(p, r) * p.Cg), peer_float2(grp + g, r).x, s);
            m = s / total;
            for (int r = 0; r < p.CS; ++r) {
                const float2 e = peer_float2(grp + g, r);
                const float d = e.x - m;
                q += fmaf((float)((long long)rank_len(p, r) * p.Cg) * d, d, e.y);
            }
        } else {
            m = grp[g].x;
            q = grp[g].y;
        }
        const float rs = 1.0f / sqrtf(q / total + p.eps);
        fin[g] = make_float2(m, rs);
        if (rank == 0) {
            if (p.mean) p.mean[b * p.G + g0 + g] = m;
            if (p.rstd) p.rstd[b * p.G + g0 + g] = rs;
        }
    }
    __syncthreads();
    if (p.CS > 1) cluster_arrive();             // peers' sums are read; waited for before this CTA leaves
    for (int col = tcol; col < nv; col += cstep) {
        float m[V], rs[V], ga[V], be[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = col * V + i;
            const float2 f = fin[c / p.Cg];
            m[i] = f.x;
            rs[i] = f.y;
            ga[i] = p.gamma ? load_par(p.gamma, w * p.par_pitch + c0 + c, p.par_bytes) : 1.0f;
            be[i] = p.gamma ? load_par(p.beta, w * p.par_pitch + c0 + c, p.par_bytes) : 0.0f;
        }
#pragma unroll 4
        for (int l = trow; l < nl; l += rows) {
            float v[V];
            Ln::unpack(src + l * sp + col * VB, v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activate(affine(normed(v[i], m[i], rs[i]), ga[i], be[i]), p.act);
            Ln::store(y + l * yp + col * VB, v);
        }
    }
    if (p.CS > 1) cluster_wait();
}

template <int EB, bool VEC, bool RES> __global__ void __launch_bounds__(kThreads) k_norm_back(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB;
    extern __shared__ __align__(128) unsigned char smem[];
    float2* stat = reinterpret_cast<float2*>(smem + p.stat_off);       // [rows][cb] sums of dz * h and dz of a thread's channels
    float2* grp = reinterpret_cast<float2*>(smem + p.grp_off);         // [GB] sums of t and t * h of this CTA
    float2* fin = grp + p.GB;                                          // [GB] their means over the whole slab
    float2* chan = fin + p.GB;                                         // [GB * Cg] this CTA's sums per channel
    float2* acc = chan + p.GB * p.Cg;                                  // [GB * Cg] the same over the worker's samples
    unsigned char* slab = smem + p.slab_off;
    combo_step::pdl_release();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = p.CS > 1 ? (int)cluster_rank() : 0;
    const long long unit = blockIdx.x / p.CS;
    const long long chunk = unit / p.nblk;
    const int g0 = (int)(unit % p.nblk) * p.GB, ng = min(p.GB, p.G - g0);
    const int c0 = g0 * p.Cg, cb = ng * p.Cg, nv = cb / V;
    const int l0 = rank * p.Lc, nl = rank_len(p, rank);
    const int rows = nv < kThreads ? kThreads / nv : 1;
    const int cstep = nv < kThreads ? nv : kThreads;
    const int trow = tid / cstep, tcol = trow < rows ? tid % cstep : nv;
    const long long xp = p.x_pitch * EB, yp = p.y_pitch * EB, dp = p.dy_pitch * EB;
    const long long b0 = chunk * p.ns, b1 = min(b0 + p.ns, p.B);
    const float inv = 1.0f / (float)((long long)p.L * p.Cg);
    int w = -1;
    long long wb = b0;                          // the worker's first sample here
    for (long long b = b0; b < b1; ++b) {
        const unsigned char* x = p.x + (b * p.L + l0) * xp + (long long)c0 * EB;
        const unsigned char* dy = p.dy + (b * p.L + l0) * dp + (long long)c0 * EB;
        unsigned char* dx = p.y + (b * p.L + l0) * yp + (long long)c0 * EB;
        if (RES) {
            Ln::fetch(slab, x, xp, nl, nv, rows, trow, tcol, cstep);
            Ln::fetch(slab + p.slab_bytes, dy, dp, nl, nv, rows, trow, tcol, cstep);
        }
        const int owner = worker_of(p, b);
        if (owner != w) {                       // the channels' sums of the worker before leave for its slot
            for (int c = tid; c < cb; c += kThreads) {
                if (w >= 0) p.partial[wb * p.C + c0 + c] = acc[c];
                acc[c] = make_float2(0.0f, 0.0f);
            }
            w = owner;
            wb = b;
        }
        if (RES) cp_async_wait();
        const unsigned char* src = RES ? slab : x;
        const unsigned char* dsrc = RES ? slab + p.slab_bytes : dy;
        const long long sp = RES ? (long long)nv * VB : xp, dsp = RES ? (long long)nv * VB : dp;
        for (int col = tcol; col < nv; col += cstep) {
            float m[V], rs[V], ga[V], be[V], s1[V], s2[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = col * V + i;
                const long long g = b * p.G + g0 + c / p.Cg;
                m[i] = p.mean[g];
                rs[i] = p.rstd[g];
                ga[i] = p.gamma ? load_par(p.gamma, w * p.par_pitch + c0 + c, p.par_bytes) : 1.0f;
                be[i] = p.gamma ? load_par(p.beta, w * p.par_pitch + c0 + c, p.par_bytes) : 0.0f;
                s1[i] = s2[i] = 0.0f;
            }
#pragma unroll 2
            for (int l = trow; l < nl; l += rows) {
                float v[V], d[V];
                Ln::unpack(src + l * sp + col * VB, v);
                Ln::unpack(dsrc + l * dsp + col * VB, d);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float h = normed(v[i], m[i], rs[i]);
                    const float dz = back_activate(d[i], affine(h, ga[i], be[i]), p.act);
                    s1[i] = fmaf(dz, h, s1[i]);
                    s2[i] += dz;
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) stat[trow * cb + col * V + i] = make_float2(s1[i], s2[i]);
        }
        __syncthreads();
        for (int c = tid; c < cb; c += kThreads) {
            float2 s = make_float2(0.0f, 0.0f);
            for (int r = 0; r < rows; ++r) {
                const float2 e = stat[r * cb + c];
                s.x += e.x;
                s.y += e.y;
            }
            chan[c] = s;
            if (p.CS == 1) acc[c] = make_float2(acc[c].x + s.x, acc[c].y + s.y);
        }
        __syncthreads();
        for (int g = warp; g < ng; g += kWarps) {
            float t = 0.0f, th = 0.0f;
            for (int c = lane; c < p.Cg; c += 32) {
                const float2 s = chan[g * p.Cg + c];
                const float ga = p.gamma ? load_par(p.gamma, w * p.par_pitch + c0 + g * p.Cg + c, p.par_bytes) : 1.0f;
                th = fmaf(ga, s.x, th);
                t = fmaf(ga, s.y, t);
            }
            t = warp_sum(t);
            th = warp_sum(th);
            if (lane == 0) grp[g] = make_float2(t, th);
        }
        if (p.CS > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
        for (int g = tid; g < ng; g += kThreads) {
            float2 s = p.CS > 1 ? make_float2(0.0f, 0.0f) : grp[g];
            for (int r = 0; p.CS > 1 && r < p.CS; ++r) {
                const float2 e = peer_float2(grp + g, r);
                s.x += e.x;
                s.y += e.y;
            }
            fin[g] = make_float2(s.x * inv, s.y * inv);
        }
        if (p.CS > 1) {                          // the cluster's CTAs share the channels among them
            for (int c = tid; c < cb; c += kThreads) {
                if (c % p.CS != rank) continue;
                float2 s = make_float2(0.0f, 0.0f);
                for (int r = 0; r < p.CS; ++r) {
                    const float2 e = peer_float2(chan + c, r);
                    s.x += e.x;
                    s.y += e.y;
                }
                p.partial[b * p.C + c0 + c] = s;
            }
        }
        __syncthreads();
        if (p.CS > 1) cluster_arrive();
        for (int col = tcol; col < nv; col += cstep) {
            float m[V], rs[V], ga[V], be[V], m1[V], m2[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = col * V + i;
                const long long g = b * p.G + g0 + c / p.Cg;
                const float2 f = fin[c / p.Cg];
                m[i] = p.mean[g];
                rs[i] = p.rstd[g];
                ga[i] = p.gamma ? load_par(p.gamma, w * p.par_pitch + c0 + c, p.par_bytes) : 1.0f;
                be[i] = p.gamma ? load_par(p.beta, w * p.par_pitch + c0 + c, p.par_bytes) : 0.0f;
                m1[i] = f.x;
                m2[i] = f.y;
            }
#pragma unroll 2
            for (int l = trow; l < nl; l += rows) {
                float v[V], d[V];
                Ln::unpack(src + l * sp + col * VB, v);
                Ln::unpack(dsrc + l * dsp + col * VB, d);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float h = normed(v[i], m[i], rs[i]);
                    const float dz = back_activate(d[i], affine(h, ga[i], be[i]), p.act);
                    v[i] = rs[i] * (fmaf(dz, ga[i], -m1[i]) - h * m2[i]);
                }
                Ln::store(dx + l * yp + col * VB, v);
            }
        }
        if (p.CS > 1) cluster_wait();            // ns is 1 here: the last thing this CTA does
        else __syncthreads();                    // stat, chan and fin are free for the next sample
    }
    if (p.CS == 1)
        for (int c = tid; c < cb; c += kThreads) p.partial[wb * p.C + c0 + c] = acc[c];
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
constexpr int kMaxChannels = COMBO_NORM_MAX_CHANNELS;   // of a block of groups: bounds the tables in shared memory (24 bytes each)
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
    const long long chunks = (p.B + p.ns - 1) / p.ns, units = chunks * p.nblk;
    const long long nv = cb / V, rows = nv < kThreads ? kThreads / nv : 1;
    // rows * cb entries; the last block of groups may be narrower and have more rows, kThreads * V entries at most
    const unsigned long long stat = (unsigned long long)(cb > kThreads * V ? cb : kThreads * V) * 8, grp = (2ull * GB + (back ? 2 * cb : 0)) * 8;
    const auto round = [](unsigned long long v) { return (v + 127) / 128 * 128; };
    const unsigned long long fixed = round(stat) + round(grp);
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
    p.grp_off = (unsigned)round(stat);
    p.slab_off = (unsigned)fixed;
    p.slab_bytes = (unsigned)(plan.res ? slab(CS) : 0);
    plan.vec = vec;
    plan.smem = fixed + (plan.res ? arrays * slab(CS) : 0);
    plan.grid = (p.B + p.ns - 1) / p.ns * p.nblk * CS;
    return plan.grid > 0x7fffffffLL ? COMBO_ERR_INVALID_ARG : COMBO_OK;
}

cudaError_t launch_norm(void (*kern)(NormParams), const NormParams& p, const Plan& plan, cudaStream_t st) {
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plan.smem);
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

template <int EB> void (*pick(bool back, bool vec, bool res))(NormParams) {
    if (back) {
        if (vec) return res ? k_norm_back<EB, true, true> : k_norm_back<EB, true, false>;
        return res ? k_norm_back<EB, false, true> : k_norm_back<EB, false, false>;
    }
    if (vec) return res ? k_norm<EB, true, true> : k_norm<EB, true, false>;
    return res ? k_norm<EB, false, true> : k_norm<EB, false, false>;
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
    p.act = act;
    p.eps = eps;
    const bool vec = C * elem_bytes % 16 == 0 && vec_ok(x, x_pitch, elem_bytes) && vec_ok(y, y_pitch, elem_bytes);
    Plan plan;
    if ((rc = plan_norm(p, plan, elem_bytes, vec, false, sms, smem)) != COMBO_OK) return rc;
    auto kern = elem_bytes == 4 ? pick<4>(false, plan.vec, plan.res) : pick<2>(false, plan.vec, plan.res);
    cudaError_t e = launch_norm(kern, p, plan, static_cast<cudaStream_t>(stream));
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
        p.act = act;
        const bool vec = C * elem_bytes % 16 == 0 && vec_ok(x, x_pitch, elem_bytes) && vec_ok(dx, dx_pitch, elem_bytes) &&
                         vec_ok(dy, dy_pitch, elem_bytes);
        Plan plan;
        if ((rc = plan_norm(p, plan, elem_bytes, vec, true, sms, smem)) != COMBO_OK) return rc;
        auto kern = elem_bytes == 4 ? pick<4>(true, plan.vec, plan.res) : pick<2>(true, plan.vec, plan.res);
        if ((e = launch_norm(kern, p, plan, st)) != cudaSuccess) return combo_host::fail(e, "group norm backward launch");
    }
    if (dgamma) {
        const dim3 grid((unsigned)((C + 31) / 32), (unsigned)N);
        e = combo_host::launch_after(k_norm_params, grid, dim3(32 * kSumRows), 0, st, p, dgamma, dbeta, (long long)(N > 1 ? grad_pitch : 0));
        if (e != cudaSuccess) return combo_host::fail(e, "group norm parameter gradient launch");
    }
    return COMBO_OK;
}

}  // extern "C"
