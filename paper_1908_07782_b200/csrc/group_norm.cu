// Group norm with an activation, channels last, for samples of many workers; forward and backward.
//
//   x [B][L][C], C = groups * Cg;  mean, rstd over the L * Cg values of a (sample, group)
//   h = (x - mean) * rstd,  z = h * gamma_w + beta_w,  y = act(z)                       w = the sample's worker
//   dz = dy * act'(z),  dgamma_w = sum dz * h,  dbeta_w = sum dz,  t = dz * gamma_w
//   dx = rstd * (t - mean(t) - h * mean(t * h))
//
// Bound by HBM: forward 1 read and 1 write of x, backward 2 reads and 1 write.  Two ways, by a rule on sizes (resident()):
//
//   resident   small inputs and short samples, one launch: a CTA brings the slab of a (sample, block of whole groups) into
//              shared memory, reduces it and writes the result from there.  Every thread works on the vectors it loaded
//              itself (thread = (row, column)).
//   streamed   k_*_sums takes chunks of a sample straight from global memory into registers and leaves each chunk's sums
//              in scratch; k_*_apply merges them and reads its chunk again, from L2 (126 MB) if that still holds it -- chunks
//              are taken from the last one back.  A CTA has no phases in which its SM's memory pipe idles, which is worth
//              more than the second read costs.
//
// Measured: forward 37 x 3136 x 256 bfloat16, ReLU, 33 us (18 at the copy rate), backward 98 x 784 x 128 floats, SiLU, 42 us (18)
// and 123 x 196 x 1024 bfloat16, ReLU, 61 us (23; its three arrays outgrow L2), one sample of 8 workers, 49 x 512, 5 us.  Far
// from the copy rate: samples of one or a few positions, backward (1386 x 1 x 256 floats 29 us for 4 MB).
//
// Forward statistics: each thread takes mean and M2 (sum of squared deviations from its own mean) of its positions,
// for each run of channels of its vector that lie in one group, and these are merged by counts: sum of n_i * mean_i for
// the mean, M2_i + n_i (mean_i - mean)^2 for M2.  No large squares are subtracted: a large mean costs what its own
// rounding to binary32 does, two or three units of its last place.  (Resident: two passes.  Streamed: one pass about a pivot
// that follows the mean, so that a first position, or a first chunk, far from all others costs nothing either.)
//
// z is formed in the roundings of the formula as written (no FMA), in both directions alike: a value that the forward
// pass clipped at zero is a value whose gradient the backward pass drops.
#include <type_traits>

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
constexpr int kCtasPerSm = 4;           // resident: that many slabs are in flight on an SM
constexpr int kStreamCtas = 3;          // streamed: with 160 registers a thread and two batches of loads under way; four and six were slower
constexpr int kWarps = kThreads / 32;

struct NormParams {
    const unsigned char* x;
    const unsigned char* dy;            // backward only
    unsigned char* y;                   // y, or dx
    const unsigned char* gamma;
    const unsigned char* beta;
    const int64_t* begin;               // [N + 1], or NULL: one worker
    float* mean;                        // [B][G]
    float* rstd;
    float2* chan;                       // backward: sums of dz * h and dz per channel; streamed [B][chunks][C]; resident [B][C],
                                        // of a CTA's samples of one worker, at the first of them
    float2* part;                       // streamed: [B][chunks][G] a chunk's mean and M2, or its sums of t and t * h
    long long x_pitch, y_pitch, dy_pitch, par_pitch;
    long long B;
    int L, C, G, Cg, GB, nblk, chunks, Lc, N, ns, par_bytes, sub;
    float eps;
    // sub: channels of a vector that surely share a group, the largest power of two up to V that divides Cg
    int cb_max;                         // channels of a full block of groups, rounded up to a multiple of 4
    float* dgamma;                      // backward
    float* dbeta;
    long long grad_pitch;
    int param_ctas;                     // CTAs that add the parameters' gradients
    unsigned stat_off, par_off, grp_off, slab_off, slab_bytes;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
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
// ReLU keeps NaN.  SiLU of floats goes through e = exp(-|z|) <= 1, so that nothing overflows and the quotient's denominator
// lies in 1 to 2, where the fast division errs by two units of the last place: with the exponential's one or two and three
// roundings within six such units, whatever z is.  For bfloat16 arrays (EB = 2) the fast exponential: 2 + 1.2 |z| units,
// 2e-6 at z = -20 and 1e-5 at -80, of what is rounded to 2^-9 behind it (dgamma and dbeta, which are not, take it over, at
// normed values of a few units), and 0 where z < -87.  Measured (fast / accurate): backward 98 x 784 x 128 floats 39.4 / 41.6
// us; bfloat16 forward 40 x 3136 x 256 41.7 / 48.9, backward 128 x 196 x 1024 69 / 85.
template <int ACT, int EB> __device__ __forceinline__ float activate(float z) {
    if (ACT == COMBO_ACT_RELU) {
        float r;
        asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(z));
        return r;
    }
    if (ACT == COMBO_ACT_SILU) {
        if (EB == 2) return __fdividef(z, 1.0f + __expf(-z));
        const float e = expf(-fabsf(z));
        return __fdividef(z >= 0.0f ? z : z * e, 1.0f + e);
    }
    return z;
}
// dy * act'(z); a gradient where ReLU clipped is dropped, whatever its value
template <int ACT, int EB> __device__ __forceinline__ float back_activate(float dy, float z) {
    if (ACT == COMBO_ACT_RELU) return z > 0.0f ? dy : 0.0f;
    if (ACT == COMBO_ACT_SILU) {
        if (EB == 2) {
            const float s = __fdividef(1.0f, 1.0f + __expf(-z));
            return dy * (s * fmaf(z, 1.0f - s, 1.0f));
        }
        // the sigmoid and what it lacks of 1, either as exact as the other
        const float e = expf(-fabsf(z)), r = __fdividef(1.0f, 1.0f + e), er = e * r;
        const float s = z >= 0.0f ? r : er, lack = z >= 0.0f ? er : r;
        return dy * (s * fmaf(z, lack, 1.0f));
    }
    return dy;
}

// One slab: `nl` positions of `nv` vectors, thread = (row, column).  A vector is 16 bytes, V elements in V / 2 pairs;
// or (VEC = false) one element, twice in a pair whose upper half is ignored.
template <int EB, bool VEC> struct Lane {
    static constexpr int kBytes = EB;
    static constexpr int V = VEC ? Elem<EB>::V : 1;
    static constexpr int VB = V * EB;
    static constexpr int P = VEC ? V / 2 : 1;
    typedef typename std::conditional<VEC, uint4, typename std::conditional<EB == 4, float, unsigned short>::type>::type Raw;
    __device__ static __forceinline__ void unpack(uint32_t shared, f32x2 (&x)[P]) {
        if constexpr (VEC) {
            uint4 v;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(shared));
            widen(v, x);
        } else if constexpr (EB == 4) {
            float v;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(shared));
            widen(v, x);
        } else {
            unsigned short v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(shared));
            widen(v, x);
        }
    }
    __device__ static __forceinline__ void widen(const Raw& v, f32x2 (&x)[P]) {
        if constexpr (VEC) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if constexpr (EB == 2) x[i] = pair(combo_step::widen_lo(w[i]), combo_step::widen_hi(w[i]));
                else x[i] = pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            }
        } else if constexpr (EB == 4) {
            x[0] = pair(v, v);
        } else {
            const float f = __uint_as_float((uint32_t)v << 16);
            x[0] = pair(f, f);
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
    // Means m and M2 q of n values each, channel by channel, merged over each run, in every pair of the run.
    __device__ static __forceinline__ void merge(f32x2 (&m)[P], f32x2 (&q)[P], int sub, float n) {
        if constexpr (VEC) {
            if (sub >= 2)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float d = lo_of(m[i]) - hi_of(m[i]), a = 0.5f * (lo_of(m[i]) + hi_of(m[i]));
                    const float v = fmaf(0.5f * n * d, d, lo_of(q[i]) + hi_of(q[i]));
                    m[i] = pair(a, a);
                    q[i] = pair(v, v);
                }
            if (sub >= 4)
#pragma unroll
                for (int i = 0; i + 1 < P; i += 2) merge2(m[i], q[i], m[i + 1], q[i + 1], n);
            if constexpr (P == 4)
                if (sub >= 8) {
                    merge2(m[0], q[0], m[2], q[2], 2.0f * n);
                    m[1] = m[3] = m[0];
                    q[1] = q[3] = q[0];
                }
        }
    }
    // two such pairs of 2 n values each, merged in both
    __device__ static __forceinline__ void merge2(f32x2& m0, f32x2& q0, f32x2& m1, f32x2& q1, float n) {
        const f32x2 d = add2(m0, neg2(m1)), half = pair(0.5f, 0.5f);
        q0 = q1 = fma2(mul2(d, pair(n, n)), d, add2(q0, q1));
        m0 = m1 = mul2(add2(m0, m1), half);
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

// A thread's vectors of one column of a slab in shared memory, one after another.
struct Walk {
    uint32_t q, step;
    __device__ __forceinline__ Walk(uint32_t slab, int vb, int nv, int rows, int trow, int col)
        : q(slab + (uint32_t)((trow * nv + col) * vb)), step((uint32_t)(rows * nv * vb)) {}
    __device__ __forceinline__ void next() { q += step; }
};

// What a CTA works on: a chunk of positions of a block of groups of a sample (resident: of a lot of p.ns samples).
template <int V> struct Place {
    int chunk, g0, ng, c0, cb, nv, nl, l0, rows, cstep, trow, tcol, sub, base, extra;
    long long lot;
    __device__ __forceinline__ Place(const NormParams& p, unsigned unit) {
        const int tid = threadIdx.x;
        unsigned u = unit / (unsigned)p.chunks;
        chunk = (int)(unit - u * p.chunks);
        lot = u / (unsigned)p.nblk;
        g0 = (int)(u % (unsigned)p.nblk) * p.GB;
        ng = min(p.GB, p.G - g0);
        c0 = g0 * p.Cg;
        cb = ng * p.Cg;
        nv = cb / V;
        l0 = chunk * p.Lc;
        nl = min(p.Lc, p.L - l0);
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

// Lanes that share a group, out of a warp: as many as it has entries, a power of two.
__device__ __forceinline__ int lanes_for(int entries) {
    int n = 1;
    while (n < entries && n < 32) n *= 2;
    return n;
}
// sum over neighbouring lots of n lanes
__device__ __forceinline__ float lot_sum(float v, int n) {
    for (int o = n / 2; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Merges a block's entries (mean, M2) of runs, [rows][cb / sub], each with the count of its row, to one pair for each group,
// which one lane passes on.
template <typename At, typename F> __device__ __forceinline__ void merge_groups(const NormParams& p, const At& at, const float2* stat, F out) {
    const int per = p.Cg / at.sub, runs = at.cb / at.sub, entries = at.rows * per;
    const int n = lanes_for(entries), lane = threadIdx.x & (n - 1), lots = kThreads / n;
    const float inv = 1.0f / (float)((long long)at.nl * p.Cg);
    for (int g0 = 0; g0 < at.ng; g0 += lots) {
        const int g = g0 + (int)threadIdx.x / n;
        const bool mine = g < at.ng;
        float s = 0.0f, q = 0.0f;
        for (int i = lane; mine && i < entries; i += n) {
            const int r = per == 1 ? i : i / per;
            s = fmaf((float)(at.positions(r) * at.sub), stat[r * runs + g * per + i - r * per].x, s);
        }
        const float m = lot_sum(s, n) * inv;
        for (int i = lane; mine && i < entries; i += n) {
            const int r = per == 1 ? i : i / per;
            const float2 e = stat[r * runs + g * per + i - r * per];
            const float d = e.x - m;
            q += fmaf((float)(at.positions(r) * at.sub) * d, d, e.y);
        }
        q = lot_sum(q, n);
        if (mine && lane == 0) out(g, m, q);
    }
}
// A thread's entries for merge_groups: (negated) means and M2 of a vector's runs.
template <typename Ln> __device__ __forceinline__ void store_runs(float2* mine, int sub, const f32x2 (&neg_m)[Ln::P], const f32x2 (&q)[Ln::P]) {
#pragma unroll
    for (int i = 0; i < Ln::P; ++i) {
        if (2 * i % sub == 0) mine[2 * i / sub] = make_float2(-lo_of(neg_m[i]), lo_of(q[i]));
        if (Ln::V > 1 && sub == 1) mine[2 * i + 1] = make_float2(-hi_of(neg_m[i]), hi_of(q[i]));
    }
}
template <typename Ln, int ACT>
__device__ __forceinline__ void forward_vector(f32x2 (&v)[Ln::P], const f32x2 (&m)[Ln::P], const f32x2 (&rs)[Ln::P], const f32x2 (&ga)[Ln::P],
                                               const f32x2 (&be)[Ln::P]) {
#pragma unroll
    for (int i = 0; i < Ln::P; ++i) {
        const f32x2 z = affine(normed(v[i], m[i], rs[i]), ga[i], be[i]);
        v[i] = pair(activate<ACT, Ln::kBytes>(lo_of(z)), activate<ACT, Ln::kBytes>(hi_of(z)));
    }
}
// h and dz of a pair of values
template <int ACT, int EB>
__device__ __forceinline__ void back_pair(f32x2 x, f32x2 d, f32x2 m, f32x2 rs, f32x2 ga, f32x2 be, f32x2& h, f32x2& dz) {
    h = normed(x, m, rs);
    const f32x2 z = affine(h, ga, be);
    dz = pair(back_activate<ACT, EB>(lo_of(d), lo_of(z)), back_activate<ACT, EB>(hi_of(d), hi_of(z)));
}
template <typename Ln, int ACT>
__device__ __forceinline__ void back_vector(f32x2 (&v)[Ln::P], const f32x2 (&d)[Ln::P], const f32x2 (&m)[Ln::P], const f32x2 (&rs)[Ln::P],
                                            const f32x2 (&ga)[Ln::P], const f32x2 (&be)[Ln::P], const f32x2 (&neg_m1)[Ln::P], const f32x2 (&m2)[Ln::P]) {
#pragma unroll
    for (int i = 0; i < Ln::P; ++i) {
        f32x2 h, dz;
        back_pair<ACT, Ln::kBytes>(v[i], d[i], m[i], rs[i], ga[i], be[i], h, dz);
        v[i] = mul2(rs[i], fma2(neg2(h), m2[i], fma2(dz, ga[i], neg_m1[i])));
    }
}

// Adds the block's table of sums, [P][rows][nv] of (dz * h, dz) for pairs of channels, over the rows: out(channel, sums).
// Rows are added in lots side by side, then the lots.  The block; the table is overwritten.
template <typename Ln, typename At, typename F> __device__ __forceinline__ void add_rows(const At& at, float4* stat, F out) {
    const int tid = threadIdx.x, nv = at.nv, rows = at.rows;
    const int pairs = nv * Ln::P, parts = min(max(kThreads / pairs, 1), rows);
    if (parts > 1) {                             // pair k = (i, col): its rows lie nv entries apart
        const int part = tid / pairs, k = tid - part * pairs, i = k / nv;
        float4* mine = stat + i * (rows - 1) * nv + k;
        if (part < parts) {
            float4 s = mine[part * nv];
            for (int r = part + parts; r < rows; r += parts) {
                const float4 e = mine[r * nv];
                s.x += e.x; s.y += e.y; s.z += e.z; s.w += e.w;
            }
            mine[part * nv] = s;                 // row `part` is read by this thread alone
        }
        __syncthreads();
    }
    for (int k = tid; k < pairs; k += kThreads) {
        const int i = k / nv, col = k - i * nv;
        const float4* mine = stat + i * rows * nv + col;
        float4 s = mine[0];
        const int n = parts > 1 ? parts : rows;
        for (int r = 1; r < n; ++r) {
            const float4 e = mine[r * nv];
            s.x += e.x; s.y += e.y; s.z += e.z; s.w += e.w;
        }
        const int c = col * Ln::V + 2 * i;
        out(c, make_float2(s.x, s.z));
        if (Ln::V > 1) out(c + 1, make_float2(s.y, s.w));
    }
}
// Sums of t = dz * gamma and of t * h over each group's channels, which one lane passes on.
template <typename At, typename F>
__device__ __forceinline__ void add_groups(const NormParams& p, const At& at, const float2* chan, const float* ga_s, F out) {
    const int n = lanes_for(p.Cg), lane = threadIdx.x & (n - 1), lots = kThreads / n;
    for (int g0 = 0; g0 < at.ng; g0 += lots) {
        const int g = g0 + (int)threadIdx.x / n;
        const bool mine = g < at.ng;
        float t = 0.0f, th = 0.0f;
        for (int c = g * p.Cg + lane; mine && c < (g + 1) * p.Cg; c += n) {
            const float2 s = chan[c];
            th = fmaf(ga_s[c], s.x, th);
            t = fmaf(ga_s[c], s.y, t);
        }
        t = lot_sum(t, n);
        th = lot_sum(th, n);
        if (mine && lane == 0) out(g, t, th);
    }
}

// ---------------------------------------------------------------- resident
template <int EB, bool VEC, int ACT> __global__ void __launch_bounds__(kThreads, kCtasPerSm) k_norm(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB, P = Ln::P;
    extern __shared__ __align__(128) unsigned char smem[];
    float2* stat = reinterpret_cast<float2*>(smem + p.stat_off);       // [rows][cb / sub] mean, M2 of a thread's runs
    float* ga_s = reinterpret_cast<float*>(smem + p.par_off);          // [cb]
    float* be_s = ga_s + p.cb_max;                                     // [cb]
    float2* fin = reinterpret_cast<float2*>(smem + p.grp_off);         // [GB] mean and rstd
    const uint32_t slab = smem_u32(smem + p.slab_off);
    const Place<V> at(p, blockIdx.x);
    const int nv = at.nv, rows = at.rows;
    const long long b = at.lot;
    const long long xp = p.x_pitch * EB, yp = p.y_pitch * EB;
    const unsigned char* x = p.x + b * p.L * xp + (long long)at.c0 * EB;
    unsigned char* y = p.y + b * p.L * yp + (long long)at.c0 * EB;
    const int n = at.positions(at.trow);        // of this thread
    for (int col = at.tcol; col < nv; col += at.cstep) {
        const Walk to(slab, VB, nv, rows, at.trow, col);
        Ln::fetch(to.q, to.step, x + at.trow * xp + col * VB, rows * xp, n);
    }
    load_params(p, worker_of(p, b), at.c0, at.cb, ga_s, be_s);
    cp_async_wait();

    const int runs = at.cb / at.sub;
    const float inv = 1.0f / (float)max(n * at.sub, 1);
    for (int col = at.tcol; col < nv; col += at.cstep) {
        f32x2 m[P], q[P];
#pragma unroll
        for (int i = 0; i < P; ++i) m[i] = q[i] = 0;
        Walk at_v(slab, VB, nv, rows, at.trow, col);
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
        at_v = Walk(slab, VB, nv, rows, at.trow, col);
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
        store_runs<Ln>(stat + at.trow * runs + col * V / at.sub, at.sub, m, q);
    }
    __syncthreads();
    merge_groups(p, at, stat, [&](int g, float m, float q) {
        const float rs = 1.0f / sqrtf(q / (float)((long long)p.L * p.Cg) + p.eps);
        fin[g] = make_float2(m, rs);
        if (p.mean) p.mean[b * p.G + at.g0 + g] = m;
        if (p.rstd) p.rstd[b * p.G + at.g0 + g] = rs;
    });
    __syncthreads();
    for (int col = at.tcol; col < nv; col += at.cstep) {
        f32x2 m[P], rs[P], ga[P], be[P];
        group_pairs<Ln>(fin, col * V, p.Cg, at.sub, m, rs);
        Ln::table(ga_s + col * V, ga);
        Ln::table(be_s + col * V, be);
        Walk at_v(slab, VB, nv, rows, at.trow, col);
        unsigned char* to = y + at.trow * yp + col * VB;
#pragma unroll 4
        for (int k = 0; k < n; ++k, at_v.next(), to += rows * yp) {
            f32x2 v[P];
            Ln::unpack(at_v.q, v);
            forward_vector<Ln, ACT>(v, m, rs, ga, be);
            Ln::store(to, v);
        }
    }
}

template <int EB, bool VEC, int ACT> __global__ void __launch_bounds__(kThreads, kCtasPerSm) k_norm_back(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB, P = Ln::P;
    extern __shared__ __align__(128) unsigned char smem[];
    float4* stat = reinterpret_cast<float4*>(smem + p.stat_off);       // [P][rows][nv] a thread's sums of dz * h and of dz, by pairs of channels
    float* ga_s = reinterpret_cast<float*>(smem + p.par_off);          // [cb]
    float* be_s = ga_s + p.cb_max;                                     // [cb]
    float2* fin = reinterpret_cast<float2*>(smem + p.grp_off);         // [GB] means of t and t * h
    float2* norm = fin + p.GB;                                         // [GB] mean and rstd
    float2* chan = norm + p.GB;                                        // [cb] sums per channel
    float2* acc = chan + p.cb_max;                                     // [cb] the same over the worker's samples
    const uint32_t slab = smem_u32(smem + p.slab_off);
    combo_step::pdl_release();
    const int tid = threadIdx.x;
    const Place<V> at(p, blockIdx.x);
    const int nv = at.nv, rows = at.rows, cb = at.cb;
    const long long xp = p.x_pitch * EB, yp = p.y_pitch * EB, dp = p.dy_pitch * EB;
    const long long b0 = at.lot * p.ns, b1 = min(b0 + p.ns, p.B);
    const float inv = 1.0f / (float)((long long)p.L * p.Cg);
    const int n = at.positions(at.trow);        // of this thread
    int w = -1;
    long long wb = b0;                          // the worker's first sample here
    for (long long b = b0; b < b1; ++b) {
        const unsigned char* x = p.x + b * p.L * xp + (long long)at.c0 * EB;
        const unsigned char* dy = p.dy + b * p.L * dp + (long long)at.c0 * EB;
        unsigned char* dx = p.y + b * p.L * yp + (long long)at.c0 * EB;
        for (int col = at.tcol; col < nv; col += at.cstep) {
            const Walk to(slab, VB, nv, rows, at.trow, col);
            Ln::fetch(to.q, to.step, x + at.trow * xp + col * VB, rows * xp, n);
            Ln::fetch(to.q + p.slab_bytes, to.step, dy + at.trow * dp + col * VB, rows * dp, n);
        }
        const int owner = worker_of(p, b);
        if (owner != w) {                       // (behind the loop's barrier) the sums of the worker before leave for their slot
            for (int c = tid; c < cb; c += kThreads) {
                if (w >= 0) p.chan[wb * p.C + at.c0 + c] = acc[c];
                acc[c] = make_float2(0.0f, 0.0f);
            }
            load_params(p, owner, at.c0, cb, ga_s, be_s);
            w = owner;
            wb = b;
        }
        for (int g = tid; g < at.ng; g += kThreads) norm[g] = make_float2(p.mean[b * p.G + at.g0 + g], p.rstd[b * p.G + at.g0 + g]);
        __syncthreads();
        cp_async_wait();
        for (int col = at.tcol; col < nv; col += at.cstep) {
            f32x2 m[P], rs[P], ga[P], be[P], s1[P], s2[P];
            group_pairs<Ln>(norm, col * V, p.Cg, at.sub, m, rs);
            Ln::table(ga_s + col * V, ga);
            Ln::table(be_s + col * V, be);
#pragma unroll
            for (int i = 0; i < P; ++i) s1[i] = s2[i] = 0;
            Walk at_v(slab, VB, nv, rows, at.trow, col);
#pragma unroll 2
            for (int k = 0; k < n; ++k, at_v.next()) {
                f32x2 v[P], d[P];
                Ln::unpack(at_v.q, v);
                Ln::unpack(at_v.q + p.slab_bytes, d);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    f32x2 h, dz;
                    back_pair<ACT, EB>(v[i], d[i], m[i], rs[i], ga[i], be[i], h, dz);
                    s1[i] = fma2(dz, h, s1[i]);
                    s2[i] = add2(s2[i], dz);
                }
            }
#pragma unroll
            for (int i = 0; i < P; ++i)
                stat[(i * rows + at.trow) * nv + col] = make_float4(lo_of(s1[i]), hi_of(s1[i]), lo_of(s2[i]), hi_of(s2[i]));
        }
        __syncthreads();
        add_rows<Ln>(at, stat, [&](int c, float2 s) {
            chan[c] = s;
            acc[c] = make_float2(acc[c].x + s.x, acc[c].y + s.y);
        });
        __syncthreads();
        add_groups(p, at, chan, ga_s, [&](int g, float t, float th) { fin[g] = make_float2(t * inv, th * inv); });
        __syncthreads();
        for (int col = at.tcol; col < nv; col += at.cstep) {
            f32x2 m[P], rs[P], ga[P], be[P], m1[P], m2[P];
            group_pairs<Ln>(norm, col * V, p.Cg, at.sub, m, rs);
            group_pairs<Ln>(fin, col * V, p.Cg, at.sub, m1, m2);
            Ln::table(ga_s + col * V, ga);
            Ln::table(be_s + col * V, be);
            Walk at_v(slab, VB, nv, rows, at.trow, col);
            unsigned char* to = dx + at.trow * yp + col * VB;
#pragma unroll 2
            for (int k = 0; k < n; ++k, at_v.next(), to += rows * yp) {
                f32x2 v[P], d[P];
                Ln::unpack(at_v.q, v);
                Ln::unpack(at_v.q + p.slab_bytes, d);
                back_vector<Ln, ACT>(v, d, m, rs, ga, be, m1, m2);
                Ln::store(to, v);
            }
        }
        __syncthreads();                         // the tables are free for the next sample
    }
    for (int c = tid; c < cb; c += kThreads) p.chan[wb * p.C + at.c0 + c] = acc[c];
}

// ---------------------------------------------------------------- streamed
// A thread's vectors of one column in global memory, N at a time in registers.
template <int EB, bool VEC, int N> struct Batch {
    using Ln = Lane<EB, VEC>;
    typename Ln::Raw raw[N];
    // the first n of them
    __device__ __forceinline__ void load(const unsigned char* q, long long step, int n) {
        if (n >= N) {
#pragma unroll
            for (int j = 0; j < N; ++j, q += step) raw[j] = *reinterpret_cast<const typename Ln::Raw*>(q);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < n) raw[j] = *reinterpret_cast<const typename Ln::Raw*>(q + j * step);
        }
    }
};
constexpr int kBatch = 8, kPair = 4;     // vectors a thread asks for at once, of one array and of each of two

template <int EB, bool VEC> __global__ void __launch_bounds__(kThreads, kStreamCtas) k_norm_sums(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB, P = Ln::P;
    extern __shared__ __align__(128) unsigned char smem[];
    float2* stat = reinterpret_cast<float2*>(smem + p.stat_off);
    combo_step::pdl_release();
    const Place<V> at(p, blockIdx.x);
    const long long b = at.lot, xp = p.x_pitch * EB, step = at.rows * xp;
    const unsigned char* x = p.x + (b * p.L + at.l0 + at.trow) * xp + (long long)at.c0 * EB;
    const int n = at.positions(at.trow);
    for (int col = at.tcol; col < at.nv; col += at.cstep) {
        // sums of the distances from a pivot and of their squares, one pass; the pivot is a channel's first value, and the mean
        // of all positions so far each time their number has doubled.  Those behind a pivot are then never more than those
        // it is the mean of, and s * s / count takes at most half of q away (7/8 of the first batch's)
        f32x2 pivot[P], s[P], q[P];              // the pivot negated
        const unsigned char* from = x + col * VB;
        if (n > 0) Ln::widen(*reinterpret_cast<const typename Ln::Raw*>(from), pivot);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            pivot[i] = n > 0 ? neg2(pivot[i]) : 0;
            s[i] = q[i] = 0;
        }
        const auto take = [&](const typename Ln::Raw& raw) {
            f32x2 e[P];
            Ln::widen(raw, e);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const f32x2 d = add2(e[i], pivot[i]);
                s[i] = add2(s[i], d);
                q[i] = fma2(d, d, q[i]);
            }
        };
        // the pivot becomes the mean of the first `count` positions, q their M2
        const auto move = [&](int count) {
            const float inv = 1.0f / (float)max(count, 1);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const f32x2 off = mul2(s[i], pair(inv, inv));
                q[i] = fma2(neg2(s[i]), off, q[i]);
                pivot[i] = add2(pivot[i], neg2(off));
                s[i] = 0;
            }
        };
        Batch<EB, VEC, kBatch> v, next;          // the next ones are under way while these are added
        next.load(from, step, n);
        int mark = kBatch;
        for (int k = 0; k < n; k += kBatch) {
            v = next;
            from += kBatch * step;
            next.load(from, step, n - k - kBatch);
            if (n - k >= kBatch) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) take(v.raw[j]);
                if (k + kBatch == mark) {
                    move(mark);
                    mark *= 2;
                }
            } else {
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (j < n - k) take(v.raw[j]);
            }
        }
        // mean and M2 of each channel, then of each run: equal counts merge as means and half squared distances
        move(n);
        f32x2(&m)[P] = pivot;
        Ln::merge(m, q, at.sub, (float)n);
        store_runs<Ln>(stat + at.trow * (at.cb / at.sub) + col * V / at.sub, at.sub, m, q);
    }
    __syncthreads();
    merge_groups(p, at, stat, [&](int g, float m, float q) {
        p.part[(b * p.chunks + at.chunk) * p.G + at.g0 + g] = make_float2(m, q);
    });
}

// What the sample's chunks left for each of the block's groups, groups side by side and a group's chunks in lots; the block.
// Backward: their sums, done(group, sums).
template <typename At, typename D>
__device__ __forceinline__ void gather_chunks(const NormParams& p, const At& at, float2* lots, D done) {
    const int parts = max(kThreads / at.ng, 1), part = (int)threadIdx.x / at.ng;
    const float2* e = p.part + at.lot * p.chunks * p.G + at.g0;
    if (part < parts)
        for (int g = (int)threadIdx.x - part * at.ng; g < at.ng; g += kThreads) {
            float2 acc = make_float2(0.0f, 0.0f);
#pragma unroll 8
            for (int k = part; k < p.chunks; k += parts) {
                const float2 v = e[(long long)k * p.G + g];
                acc.x += v.x;
                acc.y += v.y;
            }
            if (parts == 1) done(g, acc);
            else lots[part * at.ng + g] = acc;
        }
    if (parts == 1) return;
    __syncthreads();
    for (int g = threadIdx.x; g < at.ng; g += kThreads) {
        float2 s = lots[g];
        for (int r = 1; r < parts; ++r) { s.x += lots[r * at.ng + g].x; s.y += lots[r * at.ng + g].y; }
        done(g, s);
    }
}
// Forward: their means and M2 merged by counts, done(group, mean, M2).  A lot is taken as k_norm_sums takes positions, about a
// pivot that moves to the mean each time the lot's chunks have doubled; then the lots about the mean of all.
template <typename At, typename D>
__device__ __forceinline__ void merge_chunks(const NormParams& p, const At& at, float2* lots, D done) {
    const int parts = min(max(kThreads / at.ng, 1), p.chunks), part = (int)threadIdx.x / at.ng;
    const float2* e = p.part + at.lot * p.chunks * p.G + at.g0;
    const float whole = (float)((long long)p.Lc * p.Cg), last = (float)((long long)(p.L - (p.chunks - 1) * p.Lc) * p.Cg);
    const auto count = [&](int r) {              // values in lot r
        const int n = (p.chunks - 1 - r) / parts + 1;
        return (p.chunks - 1 - r) % parts == 0 ? fmaf((float)(n - 1), whole, last) : (float)n * whole;
    };
    if (part < parts)
        for (int g = (int)threadIdx.x - part * at.ng; g < at.ng; g += kThreads) {
            float pivot = 0.0f, s = 0.0f, q = 0.0f, values = 0.0f;
            const auto move = [&]() {
                const float off = s / values;
                q = fmaf(-s, off, q);
                pivot += off;
                s = 0.0f;
            };
            int mark = 8;
            for (int k = part, taken = 0; k < p.chunks; k += 8 * parts) {
                float2 v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + j * parts < p.chunks) v[j] = e[(long long)(k + j * parts) * p.G + g];
                if (taken == 0) pivot = v[0].x;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + j * parts < p.chunks) {
                        const float n = k + j * parts == p.chunks - 1 ? last : whole, d = v[j].x - pivot;
                        s = fmaf(n, d, s);
                        q += fmaf(n * d, d, v[j].y);
                        values += n;
                    }
                taken += 8;
                if (taken == mark) {
                    move();
                    mark *= 2;
                }
            }
            move();
            if (parts == 1) done(g, pivot, q);
            else lots[part * at.ng + g] = make_float2(pivot, q);
        }
    if (parts == 1) return;
    __syncthreads();
    const float total = (float)((long long)p.L * p.Cg);
    for (int g = threadIdx.x; g < at.ng; g += kThreads) {
        const float first = lots[g].x;
        float s = 0.0f, q = 0.0f;
        for (int r = 1; r < parts; ++r) s = fmaf(count(r), lots[r * at.ng + g].x - first, s);
        const float m = first + s / total;
        for (int r = 0; r < parts; ++r) {
            const float2 v = lots[r * at.ng + g];
            const float d = v.x - m;
            q += fmaf(count(r) * d, d, v.y);
        }
        done(g, m, q);
    }
}

template <int EB, bool VEC, int ACT> __global__ void __launch_bounds__(kThreads, kStreamCtas) k_norm_apply(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB, P = Ln::P;
    extern __shared__ __align__(128) unsigned char smem[];
    float* ga_s = reinterpret_cast<float*>(smem + p.par_off);
    float* be_s = ga_s + p.cb_max;
    float2* fin = reinterpret_cast<float2*>(smem + p.grp_off);
    float2* lots = reinterpret_cast<float2*>(smem + p.stat_off);
    const Place<V> at(p, gridDim.x - 1 - blockIdx.x);
    const long long b = at.lot, xp = p.x_pitch * EB, yp = p.y_pitch * EB, step = at.rows * xp;
    const unsigned char* x = p.x + (b * p.L + at.l0 + at.trow) * xp + (long long)at.c0 * EB;
    unsigned char* y = p.y + (b * p.L + at.l0 + at.trow) * yp + (long long)at.c0 * EB;
    const int n = at.positions(at.trow);
    Batch<EB, VEC, kBatch> r, next;              // the next ones are under way while these are taken
    if (at.tcol < at.nv) next.load(x + at.tcol * VB, step, n);
    load_params(p, worker_of(p, b), at.c0, at.cb, ga_s, be_s);
    combo_step::pdl_wait();
    merge_chunks(p, at, lots, [&](int g, float m, float q) {
        const float rs = 1.0f / sqrtf((q < 0.0f ? 0.0f : q) / (float)((long long)p.L * p.Cg) + p.eps);     // below zero by rounding alone
        fin[g] = make_float2(m, rs);
        if (at.chunk == 0) {
            if (p.mean) p.mean[b * p.G + at.g0 + g] = m;
            if (p.rstd) p.rstd[b * p.G + at.g0 + g] = rs;
        }
    });
    __syncthreads();
    for (int col = at.tcol; col < at.nv; col += at.cstep) {
        f32x2 m[P], rs[P], ga[P], be[P];
        group_pairs<Ln>(fin, col * V, p.Cg, at.sub, m, rs);
        Ln::table(ga_s + col * V, ga);
        Ln::table(be_s + col * V, be);
        const unsigned char* from = x + col * VB;
        unsigned char* to = y + col * VB;
        if (col != at.tcol) next.load(from, step, n);
        for (int k = 0; k < n; k += kBatch) {
            r = next;
            from += kBatch * step;
            next.load(from, step, n - k - kBatch);
            const auto give = [&](int j) {
                f32x2 v[P];
                Ln::widen(r.raw[j], v);
                forward_vector<Ln, ACT>(v, m, rs, ga, be);
                Ln::store(to, v);
                to += at.rows * yp;
            };
            if (n - k >= kBatch) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) give(j);
            } else {
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (j < n - k) give(j);
            }
        }
    }
}

template <int EB, bool VEC, int ACT> __global__ void __launch_bounds__(kThreads, kStreamCtas) k_back_sums(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB, P = Ln::P;
    extern __shared__ __align__(128) unsigned char smem[];
    float4* stat = reinterpret_cast<float4*>(smem + p.stat_off);
    float* ga_s = reinterpret_cast<float*>(smem + p.par_off);
    float* be_s = ga_s + p.cb_max;
    float2* norm = reinterpret_cast<float2*>(smem + p.grp_off);        // [GB] mean and rstd
    float2* chan = norm + p.GB;                                        // [cb]
    combo_step::pdl_release();
    const Place<V> at(p, blockIdx.x);
    const long long b = at.lot, xp = p.x_pitch * EB, dp = p.dy_pitch * EB;
    const long long first = b * p.L + at.l0 + at.trow;
    const unsigned char* x = p.x + first * xp + (long long)at.c0 * EB;
    const unsigned char* dy = p.dy + first * dp + (long long)at.c0 * EB;
    const int n = at.positions(at.trow);
    Batch<EB, VEC, kPair> rx, rd, nx, nd;        // the next ones are under way while these are taken
    if (at.tcol < at.nv) {
        nx.load(x + at.tcol * VB, at.rows * xp, n);
        nd.load(dy + at.tcol * VB, at.rows * dp, n);
    }
    for (int g = threadIdx.x; g < at.ng; g += kThreads) norm[g] = make_float2(p.mean[b * p.G + at.g0 + g], p.rstd[b * p.G + at.g0 + g]);
    load_params(p, worker_of(p, b), at.c0, at.cb, ga_s, be_s);
    __syncthreads();
    for (int col = at.tcol; col < at.nv; col += at.cstep) {
        f32x2 m[P], rs[P], ga[P], be[P], s1[P], s2[P];
        group_pairs<Ln>(norm, col * V, p.Cg, at.sub, m, rs);
        Ln::table(ga_s + col * V, ga);
        Ln::table(be_s + col * V, be);
#pragma unroll
        for (int i = 0; i < P; ++i) s1[i] = s2[i] = 0;
        const unsigned char *from = x + col * VB, *dfrom = dy + col * VB;
        if (col != at.tcol) {
            nx.load(from, at.rows * xp, n);
            nd.load(dfrom, at.rows * dp, n);
        }
        for (int k = 0; k < n; k += kPair) {
            rx = nx;
            rd = nd;
            from += kPair * at.rows * xp;
            dfrom += kPair * at.rows * dp;
            nx.load(from, at.rows * xp, n - k - kPair);
            nd.load(dfrom, at.rows * dp, n - k - kPair);
            const auto take = [&](int j) {
                f32x2 v[P], d[P];
                Ln::widen(rx.raw[j], v);
                Ln::widen(rd.raw[j], d);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    f32x2 h, dz;
                    back_pair<ACT, EB>(v[i], d[i], m[i], rs[i], ga[i], be[i], h, dz);
                    s1[i] = fma2(dz, h, s1[i]);
                    s2[i] = add2(s2[i], dz);
                }
            };
            if (n - k >= kPair) {
#pragma unroll
                for (int j = 0; j < kPair; ++j) take(j);
            } else {
#pragma unroll
                for (int j = 0; j < kPair; ++j)
                    if (j < n - k) take(j);
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i)
            stat[(i * at.rows + at.trow) * at.nv + col] = make_float4(lo_of(s1[i]), hi_of(s1[i]), lo_of(s2[i]), hi_of(s2[i]));
    }
    __syncthreads();
    const long long slot = b * p.chunks + at.chunk;
    add_rows<Ln>(at, stat, [&](int c, float2 s) {
        chan[c] = s;
        p.chan[slot * p.C + at.c0 + c] = s;
    });
    __syncthreads();
    add_groups(p, at, chan, ga_s, [&](int g, float t, float th) { p.part[slot * p.G + at.g0 + g] = make_float2(t, th); });
}

// dgamma and dbeta of 32 channels of a worker: what the CTAs left of its samples, added in a fixed order; the block.
__device__ __forceinline__ void add_params(const NormParams& p, unsigned unit, float2 (*sh)[32]) {
    const int blocks = (p.C + 31) / 32;
    const int w = (int)(unit / blocks), lane = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int c = (int)(unit - (unsigned)w * blocks) * 32 + lane;
    const long long s0 = p.begin ? max((long long)p.begin[w], 0LL) : 0;
    const long long s1 = p.begin ? min((long long)p.begin[w + 1], p.B) : p.B;
    float2 s = make_float2(0.0f, 0.0f);
    if (c < p.C && s0 < s1) {
        // resident: a slot for each CTA's samples, the first one's; streamed: for each chunk
        const bool lots = p.chunks == 1;
        const long long k0 = lots ? s0 / p.ns : s0 * p.chunks, k1 = lots ? (s1 - 1) / p.ns : s1 * p.chunks - 1;
#pragma unroll 8
        for (long long k = k0 + row; k <= k1; k += kWarps) {
            const float2 e = p.chan[(lots ? max(k * p.ns, s0) : k) * p.C + c];
            s.x += e.x;
            s.y += e.y;
        }
    }
    sh[row][lane] = s;
    __syncthreads();
    if (row == 0 && c < p.C) {
        s = sh[0][lane];
#pragma unroll
        for (int r = 1; r < kWarps; ++r) { s.x += sh[r][lane].x; s.y += sh[r][lane].y; }
        p.dgamma[w * p.grad_pitch + c] = s.x;
        p.dbeta[w * p.grad_pitch + c] = s.y;
    }
}
__global__ void __launch_bounds__(kThreads) k_norm_params(const NormParams p) {
    __shared__ float2 sh[kWarps][32];
    combo_step::pdl_wait();
    add_params(p, blockIdx.x, sh);
}

template <int EB, bool VEC, int ACT> __global__ void __launch_bounds__(kThreads, kStreamCtas) k_back_apply(const NormParams p) {
    using Ln = Lane<EB, VEC>;
    constexpr int V = Ln::V, VB = Ln::VB, P = Ln::P;
    extern __shared__ __align__(128) unsigned char smem[];
    float* ga_s = reinterpret_cast<float*>(smem + p.par_off);
    float* be_s = ga_s + p.cb_max;
    float2* norm = reinterpret_cast<float2*>(smem + p.grp_off);        // [GB] mean and rstd
    float2* fin = norm + p.GB;                                         // [GB] means of t and t * h
    if (blockIdx.x < (unsigned)p.param_ctas) {       // the parameters' gradients need the same sums
        combo_step::pdl_wait();
        add_params(p, blockIdx.x, reinterpret_cast<float2(*)[32]>(smem + p.stat_off));
        return;
    }
    float2* lots = reinterpret_cast<float2*>(smem + p.stat_off);
    const Place<V> at(p, gridDim.x - 1 - blockIdx.x);
    const long long b = at.lot, xp = p.x_pitch * EB, yp = p.y_pitch * EB, dp = p.dy_pitch * EB;
    const long long first = b * p.L + at.l0 + at.trow;
    const unsigned char* x = p.x + first * xp + (long long)at.c0 * EB;
    const unsigned char* dy = p.dy + first * dp + (long long)at.c0 * EB;
    unsigned char* dx = p.y + first * yp + (long long)at.c0 * EB;
    const int n = at.positions(at.trow);
    Batch<EB, VEC, kPair> rx, rd, nx, nd;        // the next ones are under way while these are taken
    if (at.tcol < at.nv) {
        nx.load(x + at.tcol * VB, at.rows * xp, n);
        nd.load(dy + at.tcol * VB, at.rows * dp, n);
    }
    for (int g = threadIdx.x; g < at.ng; g += kThreads) norm[g] = make_float2(p.mean[b * p.G + at.g0 + g], p.rstd[b * p.G + at.g0 + g]);
    load_params(p, worker_of(p, b), at.c0, at.cb, ga_s, be_s);
    combo_step::pdl_wait();
    const float inv = 1.0f / (float)((long long)p.L * p.Cg);
    gather_chunks(p, at, lots, [&](int g, float2 s) { fin[g] = make_float2(s.x * inv, s.y * inv); });
    __syncthreads();
    for (int col = at.tcol; col < at.nv; col += at.cstep) {
        f32x2 m[P], rs[P], ga[P], be[P], m1[P], m2[P];
        group_pairs<Ln>(norm, col * V, p.Cg, at.sub, m, rs);
        group_pairs<Ln>(fin, col * V, p.Cg, at.sub, m1, m2);
        Ln::table(ga_s + col * V, ga);
        Ln::table(be_s + col * V, be);
        const unsigned char *from = x + col * VB, *dfrom = dy + col * VB;
        unsigned char* to = dx + col * VB;
        if (col != at.tcol) {
            nx.load(from, at.rows * xp, n);
            nd.load(dfrom, at.rows * dp, n);
        }
        for (int k = 0; k < n; k += kPair) {
            rx = nx;
            rd = nd;
            from += kPair * at.rows * xp;
            dfrom += kPair * at.rows * dp;
            nx.load(from, at.rows * xp, n - k - kPair);
            nd.load(dfrom, at.rows * dp, n - k - kPair);
            const auto give = [&](int j) {
                f32x2 v[P], d[P];
                Ln::widen(rx.raw[j], v);
                Ln::widen(rd.raw[j], d);
                back_vector<Ln, ACT>(v, d, m, rs, ga, be, m1, m2);
                Ln::store(to, v);
                to += at.rows * yp;
            };
            if (n - k >= kPair) {
#pragma unroll
                for (int j = 0; j < kPair; ++j) give(j);
            } else {
#pragma unroll
                for (int j = 0; j < kPair; ++j)
                    if (j < n - k) give(j);
            }
        }
    }
}

// ---------------------------------------------------------------- host
constexpr int kRowBytes = 128;                  // resident: least bytes of a position that a block of groups takes,
constexpr int kSlabBytes = 8 * 1024;            // and of a slab
constexpr long long kChunk = 8 * 1024;   // streamed: least elements of a chunk
// Where the resident way is taken; measured at resident().
constexpr long long kResidentBytes = 8ll << 20;
constexpr long long kShortBytes = 32 * 1024;
constexpr long long kManySamples = 180;         // for each that a CTA takes
constexpr long long kSamplesPerWorker = 64;
constexpr int kWorkersAdding = 5;
constexpr unsigned long long kMostSlab = 112 * 1024;   // 784 positions of 128 channels, bfloat16, two slabs of 100 KB: 13.6 / 9.4 us at 1 MB
constexpr int kMostCtas = 512;                  // streamed: most chunks of all samples together, where there are more than samples
constexpr int kMaxChannels = COMBO_NORM_MAX_CHANNELS;   // of a block of groups: bounds the tables in shared memory (40 bytes each)
constexpr int kShortSample = 32;                // positions under which a CTA of the backward pass takes several samples

struct Plan {
    bool vec, res;
    size_t smem;
    long long grid;
};

int samples_per_cta(int L) { return L >= kShortSample ? 1 : (kShortSample + L - 1) / L; }
// Most chunks of a sample: of kChunk elements at least, a position at least, and no more in all than a device runs at once (444
// CTAs on 148 SMs), which bounds the scratch memory by the samples and channels, whatever the length.
int chunks_of(int64_t B, int64_t L, int64_t C) {
    int64_t n = (L * C + kChunk - 1) / kChunk;
    if (n > L) n = L;
    if (n > kMostCtas / B) n = kMostCtas / B;
    return (int)(n < 1 ? 1 : n);
}

// Tables and blocks of groups for one way; false where its shared memory does not suffice.
bool layout(NormParams& p, Plan& plan, int eb, bool vec, bool res, bool back, int smem_optin, int sms) {
    const int V = vec ? 16 / eb : 1, arrays = back ? 2 : 1;
    // whole groups and whole vectors; resident: as few as fill kRowBytes and kSlabBytes; streamed: as many as there are threads for
    int GB = 1;
    if (res) {
        while (GB < p.G && ((long long)GB * p.Cg * eb < kRowBytes || (long long)p.L * GB * p.Cg * eb < kSlabBytes || GB * p.Cg % V != 0)) ++GB;
    } else {
        for (int n = p.G; n > 1; --n)
            if (n * p.Cg % V == 0 && n * p.Cg / V <= kThreads) { GB = n; break; }
        while (GB < p.G && GB * p.Cg % V != 0) ++GB;
    }
    if (GB > 1 && GB * p.Cg > kMaxChannels) {
        if (vec) return false;                   // groups that only together make whole vectors
        GB = kMaxChannels / p.Cg;
    }
    p.GB = GB;
    p.nblk = (p.G + GB - 1) / GB;
    const long long cb = (long long)GB * p.Cg, nv = cb / V;
    p.cb_max = (int)(cb + 3) / 4 * 4;
    p.ns = res && back ? samples_per_cta(p.L) : 1;
    p.chunks = 1;
    if (!res) {                                  // as many as have all CTAs on the device at once, where that is enough of them
        const long long slots = (long long)sms * kStreamCtas / (p.B * p.nblk), most = chunks_of(p.B, p.L, p.C);
        p.chunks = (int)(slots < 1 ? 1 : slots < most ? slots : most);
    }
    p.Lc = (p.L + p.chunks - 1) / p.chunks;
    p.chunks = (p.L + p.Lc - 1) / p.Lc;          // none of them empty
    p.sub = 1;
    while (p.sub < V && p.Cg % (2 * p.sub) == 0) p.sub *= 2;
    // forward: rows * cb / sub entries of 8 bytes, backward: 16 bytes for every pair of channels; the last block of
    // groups may be narrower and have more rows, but never more than kThreads vectors
    const long long vecs = nv > kThreads ? nv : kThreads;
    const auto round = [](unsigned long long v) { return (v + 127) / 128 * 128; };
    const unsigned long long stat = round((unsigned long long)vecs * (back ? (V > 1 ? V / 2 : 1) * 16 : V / p.sub * 8));   // at least kThreads pairs, as gather_chunks wants
    const unsigned long long par = round(8ull * p.cb_max), grp = round((2ull * GB + (back ? 2 * p.cb_max : 0)) * 8);
    const unsigned long long slab = res ? round((unsigned long long)p.L * cb * eb) : 0;
    p.stat_off = 0;
    p.par_off = (unsigned)stat;
    p.grp_off = (unsigned)(stat + par);
    p.slab_off = (unsigned)(stat + par + grp);
    p.slab_bytes = (unsigned)slab;
    if (arrays * slab > kMostSlab || stat + par + grp + arrays * slab > (unsigned long long)smem_optin) return false;
    plan.vec = vec;
    plan.res = res;
    plan.smem = stat + par + grp + arrays * slab;
    plan.grid = (p.B + p.ns - 1) / p.ns * p.nblk * p.chunks;
    return true;
}

// Whether the resident layout in `p` and `plan` is the faster way.  Measured, resident / streamed in us, bfloat16 unless said, 8
// workers:
//   forward, samples of up to 32 KB: always (1 position of 1024 channels, 4096 samples 27 / 60; 49 of 64, 1337 19 / 43).
//   forward, longer ones: while the CTAs are no more than 1.6 times what the device holds at once, up to 8 MB: 49 of 512
//     channels in 32 groups, 4 MB (0.85 of it) 6.6 / 8.5, 8 MB (1.7) 11.4 / 9.9, floats 8 MB (1.56) 8.4 / 8.9; 49 of 2048, 8 MB
//     (1.14) 7.3 / 10.3; 196 of 256, 8 MB (0.57) 6.4 / 10.0.
//   backward, several samples to a CTA (they go through it one after another, 3 to 5 us each): where there are so many that the
//     streamed way's CTA for each costs more: 1 position of 256 channels, 512 samples 94 / 16, 2048 96 / 41, 8192 102 / 145;
//     4 of 256, 512 samples 29 / 16, 2048 34 / 41; 8 of 1024, 256 samples 21 / 15, 1024 35 / 42.
//   backward, others: while the CTAs fit the device at once, up to 8 MB, and the parameters' gradients, which the streamed way
//     adds beside its second pass, are sums over few samples: 49 of 1024, 8 MB (0.57) 10.3 / 14.9; 49 of 256, 16 MB (1.7)
//     18.6 / 14.2; for one worker instead of 8: 49 of 256, 42 samples 9.4 / 8.4, 167 18.0 / 13.9.  Samples of up to 16 KB, x and
//     dy: always where five workers or more share the adding (49 of 64, 1337 samples for 8 workers 27 / 32, for one 78 / 38).
bool resident(const NormParams& p, const Plan& plan, bool back, long long sample_bytes, int smem_optin, int sms) {
    if (p.ns > 1) return p.B > kManySamples * p.ns;
    if (!back && sample_bytes <= kShortBytes) return true;
    if (back && sample_bytes <= kShortBytes / 2 && p.N >= kWorkersAdding) return true;
    if (sample_bytes * p.B > kResidentBytes) return false;
    const long long fit = (smem_optin + 1024) / (long long)(plan.smem + 1024), at_once = sms * (fit < kCtasPerSm ? fit : kCtasPerSm);
    return back ? plan.grid <= at_once && p.B <= kSamplesPerWorker * p.N : plan.grid * 5 <= at_once * 8;
}

combo_status choose(NormParams& p, Plan& plan, int eb, bool vec, bool back, int smem_optin, int sms) {
    const long long sample_bytes = (long long)p.L * p.C * eb * (back ? 2 : 1);
    for (int v = vec ? 1 : 0; v >= 0; --v) {
        if (layout(p, plan, eb, v != 0, true, back, smem_optin, sms) && resident(p, plan, back, sample_bytes, smem_optin, sms)) break;
        if (layout(p, plan, eb, v != 0, false, back, smem_optin, sms)) break;
        if (v == 0) return COMBO_ERR_INVALID_ARG;
    }
    return plan.grid > 0x7fffffffLL ? COMBO_ERR_INVALID_ARG : COMBO_OK;
}

typedef void (*NormKernel)(NormParams);
// The kernels of one call: resident one, streamed two, and a number for each kernel of the library.
struct Kernels {
    NormKernel first, second;
    int number;
};
template <int EB, bool VEC, int ACT> Kernels pick_way(bool back, bool res) {
    if (res) return {back ? k_norm_back<EB, VEC, ACT> : k_norm<EB, VEC, ACT>, nullptr, 0};
    return {back ? k_back_sums<EB, VEC, ACT> : k_norm_sums<EB, VEC>, back ? k_back_apply<EB, VEC, ACT> : k_norm_apply<EB, VEC, ACT>, 0};
}
template <int EB, bool VEC> Kernels pick_act(bool back, bool res, int act) {
    return act == COMBO_ACT_RELU ? pick_way<EB, VEC, COMBO_ACT_RELU>(back, res)
           : act == COMBO_ACT_SILU ? pick_way<EB, VEC, COMBO_ACT_SILU>(back, res) : pick_way<EB, VEC, COMBO_ACT_NONE>(back, res);
}
Kernels pick(int eb, bool back, const Plan& plan, int act) {
    Kernels k = eb == 4 ? (plan.vec ? pick_act<4, true>(back, plan.res, act) : pick_act<4, false>(back, plan.res, act))
                        : (plan.vec ? pick_act<2, true>(back, plan.res, act) : pick_act<2, false>(back, plan.res, act));
    k.number = ((((eb == 4) * 2 + back) * 2 + plan.vec) * 2 + plan.res) * 3 + act;
    return k;
}

cudaError_t launch(const NormParams& p, const Plan& plan, int eb, bool back, int act, int smem_optin, cudaStream_t st) {
    static uint64_t allowed[2][48];
    const Kernels k = pick(eb, back, plan, act);
    combo_host::set_step_path(plan.res ? combo_host::kPathResident : combo_host::kPathStreamed);
    cudaError_t e = combo_host::allow_smem(k.first, smem_optin, &allowed[0][k.number]);
    if (e != cudaSuccess) return e;
    k.first<<<(unsigned)plan.grid, kThreads, plan.smem, st>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess || !k.second) return e;
    if ((e = combo_host::allow_smem(k.second, smem_optin, &allowed[1][k.number])) != cudaSuccess) return e;
    return combo_host::launch_after(k.second, dim3((unsigned)plan.grid + p.param_ctas), dim3(kThreads), plan.smem, st, p);
}

// Scratch: sums per chunk and group, then (backward) per chunk and channel
size_t part_bytes(int64_t B, int64_t L, int64_t C, int groups) { return ((size_t)B * chunks_of(B, L, C) * groups * 8 + 127) / 128 * 128; }

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
bool vec_ok(const void* p, int64_t pitch, int eb) { return combo_host::aligned_to(p, 16) && pitch * eb % 16 == 0; }
// an output may be an input, element for element; it may not overlap it in any other way
bool clash(const void* out, int64_t out_pitch, const void* in, int64_t in_pitch, int64_t positions, int64_t C, int eb) {
    if (out == in && (out_pitch == in_pitch || positions == 1)) return false;
    const size_t width = (size_t)C * eb;
    return combo_host::overlap(combo_host::Rows{out, positions, width, (size_t)out_pitch * eb}, combo_host::Rows{in, positions, width, (size_t)in_pitch * eb});
}

bool scratch_ok(const void* scratch, size_t bytes, int64_t B, int64_t L, int64_t C, int groups) {
    return scratch && combo_host::aligned_to(scratch, 16) && bytes >= combo_group_norm_scratch_bytes(B, L, C, groups);
}

}  // namespace

extern "C" {

size_t combo_group_norm_scratch_bytes(int64_t B, int64_t L, int64_t C, int groups) {
    if (B < 0 || L < 1 || C < 1 || L > (1 << 28) || C > (1 << 20) || B > (1LL << 40) / L / C || groups < 1 || groups > C)
        return 0;
    const int64_t n = B < 1 ? 1 : B;
    return part_bytes(n, L, C, groups) + (size_t)n * chunks_of(n, L, C) * C * sizeof(float2);
}

combo_status combo_group_norm(const void* x, int64_t x_pitch, void* y, int64_t y_pitch, int elem_bytes, const void* gamma,
                              const void* beta, int param_bytes, int64_t param_pitch, const int64_t* d_begin, int N,
                              int64_t B, int64_t L, int64_t C, int groups, float eps, int act, float* mean_out,
                              float* rstd_out, void* scratch, size_t scratch_bytes, void* stream) {
    combo_status rc = check_shape(elem_bytes, param_bytes, gamma, beta, param_pitch, d_begin, N, B, L, C, groups, act);
    if (rc != COMBO_OK) return rc;
    if (!(eps >= 0.0f) || !scratch_ok(scratch, scratch_bytes, B, L, C, groups)) return COMBO_ERR_INVALID_ARG;
    if (B == 0) return COMBO_OK;
    if (!array_ok(x, x_pitch, C, elem_bytes) || !array_ok(y, y_pitch, C, elem_bytes)) return COMBO_ERR_INVALID_ARG;
    if (!combo_host::aligned_to(mean_out, 4) || !combo_host::aligned_to(rstd_out, 4)) return COMBO_ERR_INVALID_ARG;
    if (clash(y, y_pitch, x, x_pitch, B * L, C, elem_bytes)) return COMBO_ERR_ALIAS;
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
    p.part = static_cast<float2*>(scratch);
    Plan plan;
    if ((rc = choose(p, plan, elem_bytes, vec, false, smem, sms)) != COMBO_OK) return rc;
    cudaError_t e = launch(p, plan, elem_bytes, false, act, smem, static_cast<cudaStream_t>(stream));
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
    if (!scratch_ok(scratch, scratch_bytes, B, L, C, groups)) return COMBO_ERR_INVALID_ARG;
    int sms = 0, smem = 0;
    NormParams p = {};
    p.begin = d_begin;
    p.part = static_cast<float2*>(scratch);
    p.chan = reinterpret_cast<float2*>(static_cast<unsigned char*>(scratch) + part_bytes(B < 1 ? 1 : B, L, C, groups));
    p.chunks = 1;
    p.dgamma = dgamma;
    p.dbeta = dbeta;
    p.grad_pitch = N > 1 ? grad_pitch : 0;
    p.param_ctas = dgamma ? (int)((C + 31) / 32 * N) : 0;
    Plan plan = {};
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
        if (clash(dx, dx_pitch, x, x_pitch, B * L, C, elem_bytes) || clash(dx, dx_pitch, dy, dy_pitch, B * L, C, elem_bytes))
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
        if ((rc = choose(p, plan, elem_bytes, vec, true, smem, sms)) != COMBO_OK) return rc;
        if ((e = launch(p, plan, elem_bytes, true, act, smem, st)) != cudaSuccess) return combo_host::fail(e, "group norm backward launch");
    }
    if (p.param_ctas > 0 && (B == 0 || plan.res)) {
        e = combo_host::launch_after(k_norm_params, dim3((unsigned)p.param_ctas), dim3(kThreads), 0, st, p);
        if (e != cudaSuccess) return combo_host::fail(e, "group norm parameter gradient launch");
    }
    return COMBO_OK;
}

}  // extern "C"
