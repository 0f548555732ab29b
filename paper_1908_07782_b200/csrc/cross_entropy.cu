// Softmax cross entropy of a linear classifier, grouped by worker; the logits are never kept.
//
//   z_mv = x_m . W_w,v      lse_m = log sum_v exp z_mv      loss_m = lse_m - z_m,label        m in worker w's rows, v a class
//   d_mv = (exp(z_mv - lse_m) - [v = label_m]) g_m          dx_m = sum_v d_mv W_w,v           dW_w,v = sum_m d_mv x_m
//
// Large calls pack the labelled rows and go through the tensor cores (cross_entropy_tensor.cuh), which bound them: forward 8 x 817
// rows, 1024 -> 30001 bfloat16 365 to 388 us, gradients 4 x 1995 rows, 768 -> 32000 into floats 1725 to 1970; one row a worker, 16 x
// 1024 -> 32000, 190 us, bound by its 1.05 GB of weights.  Small ones are bound by latency and take one launch, or two, of
// multiply-adds: loss of 8 x 1 row, 256 -> 10, 8.4 us, gradients of 8 x 167 rows 18.
#include <cuda_fp16.h>
#include <string.h>

#include "host_common.h"
#include "step_common.cuh"
#include "cross_entropy_tensor.cuh"

namespace {

using combo_step::Elem;

struct Loss {
    const unsigned char *x, *w;
    const int64_t *labels, *begin;
    const float *row_grad, *lse_in;
    unsigned char *dx, *dw;
    float *loss, *lse;
    float *d;                     // [M][V] of scratch
    long long x_pitch, w_pitch, w_stride, dx_pitch, dw_pitch, dw_stride;      // elements
    long long M;
    int N, K, V;
};

__device__ __forceinline__ void rows_of(const Loss& p, int w, long long& r0, long long& r1) {
    r0 = min(max((long long)p.begin[w], 0LL), p.M);
    r1 = min(max((long long)p.begin[w + 1], r0), p.M);
}

// ---------------------------------------------------------------- few multiply-adds: a CTA takes eight rows of a worker
constexpr int kThreads = 256, kWarps = kThreads / 32, kR = 8, kU = 4, kFewClasses = 256;

// The worker and first row of lot `block` of kR rows; false behind the last.  A thread counts the lots of its neighbouring workers, and
// the one whose they are looks among them.  2000 workers of one row, 256 -> 10, 46 us (one by one 371).
__device__ __forceinline__ bool find_rows(const Loss& p, long long block, int& w, long long& i0, long long& i1) {
    __shared__ long long sums[kWarps], first;
    __shared__ int owner;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, per = (p.N + kThreads - 1) / kThreads;
    const auto lots = [&](int k) {
        rows_of(p, k, i0, i1);
        return (i1 - i0 + kR - 1) / kR;
    };
    if (t == 0) owner = -1;
    const int w0 = min(t * per, p.N), w1 = min(w0 + per, p.N);
    long long mine = 0;
#pragma unroll 8
    for (int k = w0; k < w1; ++k) mine += lots(k);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    long long at = upto - mine;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) at += k < warp ? sums[k] : 0;
    if (block >= at && block < at + mine) {
        int k = w0;
        for (long long n = lots(k); block >= at + n; n = lots(k)) {
            at += n;
            ++k;
        }
        owner = k;
        first = i0 + (block - at) * kR;
    }
    __syncthreads();
    w = owner;
    if (w < 0) return false;
    rows_of(p, w, i0, i1);
    i0 = first;
    return true;
}

// A lane's share of a line of K elements, step `c` of ceil(K / (32 E)): E neighbours in 16 bytes, or elements 32 apart.
template <int EB, bool VEC> __device__ __forceinline__ void load_share(const unsigned char* line, int c, int lane, int K, float (&v)[Elem<EB>::V]) {
    constexpr int E = Elem<EB>::V;
    if (VEC) {
        const int k = (c * 32 + lane) * E;
        if (K % E == 0 || k + E <= K) {
            uint4 q = make_uint4(0, 0, 0, 0);
            if (k < K) q = *reinterpret_cast<const uint4*>(line + (long long)k * EB);
            Elem<EB>::unpack(q, v);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = k + e < K ? Elem<EB>::get(line + (long long)(k + e) * EB) : 0.0f;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int k = (c * E + e) * 32 + lane;
            v[e] = k < K ? Elem<EB>::get(line + (long long)k * EB) : 0.0f;
        }
    }
}
// The index of element e of that share.
template <int EB, bool VEC> __device__ __forceinline__ int share_index(int c, int lane, int e) {
    return VEC ? (c * 32 + lane) * Elem<EB>::V + e : (c * Elem<EB>::V + e) * 32 + lane;
}

// 32 sums over the warp's lanes at once: lane l gets that of v[l].
__device__ __forceinline__ float sums_of_32(float (&v)[32], int lane) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int k = 0; k < o; ++k) {
            const float keep = up ? v[k + o] : v[k], give = up ? v[k] : v[k + o];
            v[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    return v[0];
}

// Logits of kU classes from v0 for kR rows: lane l gets class v0 + l / kR, row l % kR.
template <int EB, bool VEC>
__device__ __forceinline__ float logits(const Loss& p, const unsigned char* x0, int rows, const unsigned char* w0, int v0, int lane) {
    constexpr int E = Elem<EB>::V;
    float acc[kU * kR];
#pragma unroll
    for (int i = 0; i < kU * kR; ++i) acc[i] = 0.0f;
    for (int c = 0; c * 32 * E < p.K; ++c) {
        float wv[kU][E];
#pragma unroll
        for (int u = 0; u < kU; ++u) load_share<EB, VEC>(w0 + (long long)min(v0 + u, p.V - 1) * p.w_pitch * EB, c, lane, p.K, wv[u]);
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            if (r < rows) {
                float xv[E];
                load_share<EB, VEC>(x0 + r * p.x_pitch * EB, c, lane, p.K, xv);
#pragma unroll
                for (int u = 0; u < kU; ++u)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[u * kR + r] = fmaf(xv[e], wv[u][e], acc[u * kR + r]);
            }
        }
    }
    return sums_of_32(acc, lane);
}

// (m, s) stands for s exp(m); joins two.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
    const float most = fmaxf(m, m2);
    if (m2 != m2 || m != m) {
        m = s = __int_as_float(0x7fffffff);
    } else if (most != -INFINITY) {
        s = s * expf(m - most) + s2 * expf(m2 - most);
        m = most;
    }
}

template <int EB, bool VEC> __global__ void __launch_bounds__(kThreads) k_few_loss(const Loss p) {
    int w;
    long long i0, i1;
    combo_step::pdl_release();
    combo_step::pdl_wait();
    if (!find_rows(p, blockIdx.x, w, i0, i1)) return;
    const int rows = (int)min(i1 - i0, (long long)kR), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = lane % kR;
    const unsigned char *x0 = p.x + i0 * p.x_pitch * EB, *w0 = p.w + w * p.w_stride * EB;
    const int64_t label = row < rows ? p.labels[i0 + row] : -1;
    float m = -INFINITY, s = 0.0f, mine = 0.0f;
    bool found = false;
    for (int v0 = warp * kU; v0 < p.V; v0 += kWarps * kU) {
        const float z = logits<EB, VEC>(p, x0, rows, w0, v0, lane);
        const int v = v0 + lane / kR;
        if (v < p.V) {
            join(m, s, z, 1.0f);
            if (v == label) { mine = z; found = true; }
        }
    }
    __shared__ float sm[3][kWarps][32];
    __shared__ int where[kR];
    if (threadIdx.x < kR) where[threadIdx.x] = -1;
    __syncthreads();
    sm[0][warp][lane] = m;
    sm[1][warp][lane] = s;
    if (found) where[row] = warp * 32 + lane;
    sm[2][warp][lane] = mine;
    __syncthreads();
    if (threadIdx.x < rows) {
        const int r = threadIdx.x;
        m = -INFINITY;
        s = 0.0f;
        for (int k = 0; k < kWarps; ++k)
            for (int u = 0; u < kU; ++u) join(m, s, sm[0][k][u * kR + r], sm[1][k][u * kR + r]);
        const float rest = logf(s);                            // s is at least 1
        p.lse[i0 + r] = where[r] >= 0 ? m + rest : 0.0f;
        p.loss[i0 + r] = where[r] >= 0 ? m - (&sm[2][0][0])[where[r]] + rest : 0.0f;
    }
}

// What the warps hold for `lines` x (32 E) results, acc[line][e] a lane, added up in the warps' order and given to put(line, k, sum).
constexpr int kSumWarps = 16;
template <int EB, bool VEC, typename F>
__device__ __forceinline__ void join_warps(const float (&acc)[kR][Elem<EB>::V], int c, int lane, int warp, F put) {
    constexpr int E = Elem<EB>::V;
    __shared__ float sm[kSumWarps][2][32 * E + 1];
#pragma unroll
    for (int h = 0; h < kR; h += 2) {
        __syncthreads();
#pragma unroll
        for (int l = 0; l < 2; ++l)
#pragma unroll
            for (int e = 0; e < E; ++e) sm[warp][l][e * 32 + lane] = acc[h + l][e];
        __syncthreads();
        for (int o = threadIdx.x; o < 2 * 32 * E; o += kSumWarps * 32) {
            const int l = o / (32 * E), at = o % (32 * E);
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kSumWarps; ++k) sum += sm[k][l][VEC ? at % E * 32 + at / E : at];
            put(h + l, c * 32 * E + at, sum);
        }
    }
}

template <int EB, bool VEC> __global__ void __launch_bounds__(kThreads) k_few_back(const Loss p) {
    int w;
    long long i0, i1;
    combo_step::pdl_release();
    combo_step::pdl_wait();
    if (!find_rows(p, blockIdx.x, w, i0, i1)) return;
    const int rows = (int)min(i1 - i0, (long long)kR), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = lane % kR;
    const unsigned char *x0 = p.x + i0 * p.x_pitch * EB, *w0 = p.w + w * p.w_stride * EB;
    const int64_t label = row < rows ? p.labels[i0 + row] : -1;
    const bool has = label >= 0 && label < p.V;
    float g = 0.0f;
    if (p.row_grad) {
        if (has) g = p.row_grad[i0 + row];
    } else {
        // the worker's labelled rows
        long long a, b;
        rows_of(p, w, a, b);
        int count = 0;
        for (long long i = a + threadIdx.x; i - threadIdx.x < b; i += kThreads)
            count += __syncthreads_count(i < b && p.labels[i] >= 0 && p.labels[i] < p.V);
        if (has) g = 1.0f / (float)count;
    }
    const float lse = has ? p.lse_in[i0 + row] : 0.0f;
    __shared__ __align__(16) float d[kFewClasses][kR];
    for (int v0 = warp * kU; v0 < p.V; v0 += kWarps * kU) {
        const float z = logits<EB, VEC>(p, x0, rows, w0, v0, lane);
        const int v = v0 + lane / kR;
        if (v < p.V) {
            const float f = has ? (expf(z - lse) - (v == label ? 1.0f : 0.0f)) * g : 0.0f;
            d[v][row] = f;
            if (row < rows) p.d[(i0 + row) * p.V + v] = f;
        }
    }
    __syncthreads();
    const unsigned some = __ballot_sync(0xffffffffu, has && lane < kR);          // rows with a label
    // dx: threads side by side along the inputs, as many groups over the classes as there is room for, joined in their order
    __shared__ float part[kThreads][kR + 1];
    int side = 32;
    while (side < kThreads && side < p.K) side *= 2;
    const int group = threadIdx.x / side, groups = kThreads / side;
    for (int k0 = 0; k0 < p.K; k0 += side) {
        const int k = k0 + threadIdx.x % side;
        float acc[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) acc[r] = 0.0f;
        if (k < p.K) {
#pragma unroll 8
            for (int v = group; v < p.V; v += groups) {
                const float wv = Elem<EB>::get(w0 + ((long long)v * p.w_pitch + k) * EB);
#pragma unroll
                for (int r = 0; r < kR; ++r) acc[r] = fmaf(d[v][r], wv, acc[r]);
            }
        }
        if (groups > 1) {
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kR; ++r) part[threadIdx.x][r] = acc[r];
            __syncthreads();
            if (group == 0) {
                for (int g2 = 1; g2 < groups; ++g2)
#pragma unroll
                    for (int r = 0; r < kR; ++r) acc[r] += part[threadIdx.x + g2 * side][r];
            }
        }
        if (group == 0 && k < p.K) {
#pragma unroll
            for (int r = 0; r < kR; ++r)
                if (r < rows) Elem<EB>::put(p.dx + ((i0 + r) * p.dx_pitch + k) * EB, some >> r & 1u ? acc[r] : 0.0f);
        }
    }
}

// Eight classes' gradients of one worker by 32 E columns; warps share out the rows.
template <int EB, int OB, bool VEC> __global__ void __launch_bounds__(kSumWarps * 32) k_few_weights(const Loss p) {
    constexpr int E = Elem<EB>::V;
    const int w = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x;
    long long i0, i1;
    combo_step::pdl_release();
    combo_step::pdl_wait();
    rows_of(p, w, i0, i1);
    for (int v0 = blockIdx.y * kR; v0 < p.V; v0 += gridDim.y * kR) {
        float acc[kR][E];
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[r][e] = 0.0f;
        // several rows' loads at once; a row without a label may hold anything (its d is 0)
#pragma unroll 4
        for (long long i = i0 + warp; i < i1; i += kSumWarps) {
            const int64_t label = p.labels[i];
            const bool has = label >= 0 && label < p.V;
            float xv[E], f[kR];
            load_share<EB, VEC>(p.x + i * p.x_pitch * EB, c, lane, p.K, xv);
#pragma unroll
            for (int r = 0; r < kR; ++r) f[r] = p.d[i * p.V + min(v0 + r, p.V - 1)];
#pragma unroll
            for (int e = 0; e < E; ++e) xv[e] = has ? xv[e] : 0.0f;
#pragma unroll
            for (int r = 0; r < kR; ++r)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[r][e] = fmaf(f[r], xv[e], acc[r][e]);
        }
        join_warps<EB, VEC>(acc, c, lane, warp, [&](int r, int k, float sum) {
            if (v0 + r < p.V && k < p.K) Elem<OB>::put(p.dw + (w * p.dw_stride + (v0 + r) * p.dw_pitch + k) * OB, sum);
        });
    }
}

template <int EB, bool VEC> cudaError_t launch_few(const Loss& p, int grad_bytes, cudaStream_t st) {
    const long long lots = p.M / kR + (p.N < p.M ? p.N : p.M);
    const unsigned grid = (unsigned)(lots < 1 ? 1 : lots);
    if (!grad_bytes) return combo_host::launch_after(k_few_loss<EB, VEC>, dim3(grid), dim3(kThreads), 0, st, p);
    cudaError_t e = cudaSuccess;
    if (p.M > 0) e = combo_host::launch_after(k_few_back<EB, VEC>, dim3(grid), dim3(kThreads), 0, st, p);
    if (e != cudaSuccess) return e;
    const unsigned classes = (unsigned)((p.V + kR - 1) / kR);
    const dim3 g((unsigned)((p.K + 32 * Elem<EB>::V - 1) / (32 * Elem<EB>::V)), classes < 65535 ? classes : 65535, (unsigned)p.N);
    return grad_bytes == 4 ? combo_host::launch_after(k_few_weights<EB, 4, VEC>, g, dim3(kSumWarps * 32), 0, st, p)
                           : combo_host::launch_after(k_few_weights<EB, 2, VEC>, g, dim3(kSumWarps * 32), 0, st, p);
}

// ---------------------------------------------------------------- packing of rows and weights for the tensor cores
using namespace combo_loss;

// Where things lie in scratch.
struct Packed {
    int *count, *list, *pos, *row0, *tiles, *src, *label;      // [N]; [M]; [M]; [N + 1]; [N + 2]; [cap]: forward the row, backward the worker; [cap]
    float *lse, *g, *own;                                      // [cap]
    unsigned short *xh, *wh;                                   // forward, floats: planes of float16, as x and w
    float *x_unit, *w_unit;                                    // [cap], [N][piece]: what their numbers count in
    unsigned short *x, *w, *d;                                 // planes of [cap][kp]; of [N][classes there are][kp]; of [piece / 8][cap][8]
    float2* part;
    float* dx;
    long long cap;
    int kp, height;                                            // inputs, up to a multiple of 64; rows of a tile
};

constexpr int kCountThreads = 1024, kCountRows = 8;

// A worker's labelled rows, in order: how many, and which.  The others' results are zeros.
__global__ void __launch_bounds__(kCountThreads) k_count(const Loss p, const Packed s) {
    __shared__ int sums[33];
    const int w = blockIdx.x, t = threadIdx.x, lane = t & 31;
    combo_step::pdl_release();
    combo_step::pdl_wait();
    long long r0, r1;
    rows_of(p, w, r0, r1);
    int before = 0;
    for (long long i0 = r0; i0 < r1; i0 += kCountThreads * kCountRows) {
        const long long i = i0 + t * kCountRows;
        unsigned has = 0;
#pragma unroll
        for (int e = 0; e < kCountRows; ++e) {
            const int64_t label = i + e < r1 ? p.labels[i + e] : -1;
            has |= (unsigned)(label >= 0 && label < p.V) << e;
        }
        const int mine = __popc(has);
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) sums[t >> 5] = upto;
        __syncthreads();
        if (t < 32) {
            const int v = sums[t];
            int u = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int k = __shfl_up_sync(0xffffffffu, u, o);
                if (lane >= o) u += k;
            }
            sums[t] = u - v;
            if (t == 31) sums[32] = u;
        }
        __syncthreads();
        int at = before + sums[t >> 5] + upto - mine;
#pragma unroll
        for (int e = 0; e < kCountRows; ++e) {
            if (has >> e & 1u) {
                s.list[r0 + at++] = (int)(i + e);
            } else if (i + e < r1) {
                if (p.loss) p.loss[i + e] = p.lse[i + e] = 0.0f;
                else s.pos[i + e] = -1;
            }
        }
        before += sums[32];
        __syncthreads();
    }
    if (t == 0) s.count[w] = before;
}

// Eight neighbours of a line of `left` elements, zeros behind.  Off 16-byte boundaries the aligned 16 bytes that hold some of them
// are read whole and shifted.
template <int EB> __device__ __forceinline__ void load8(const unsigned char* q, int left, bool vec, float (&v)[8]) {
    constexpr int W = 2 * EB;                    // words of eight elements
    uint32_t w[W + 4];
    const int some = min(max(left, 0), 8);
    if (vec && left >= 8) {
#pragma unroll
        for (int h = 0; h < EB / 2; ++h) {
            const uint4 f = reinterpret_cast<const uint4*>(q)[h];
            w[4 * h] = f.x; w[4 * h + 1] = f.y; w[4 * h + 2] = f.z; w[4 * h + 3] = f.w;
        }
    } else {
        const int off = (int)(reinterpret_cast<uintptr_t>(q) & 15u);
        const uint4* from = reinterpret_cast<const uint4*>(q - off);
#pragma unroll
        for (int h = 0; h <= EB / 2; ++h) {
            uint4 f = make_uint4(0, 0, 0, 0);
            if (some > 0 && h * 16 < off + some * EB) f = from[h];
            w[4 * h] = f.x; w[4 * h + 1] = f.y; w[4 * h + 2] = f.z; w[4 * h + 3] = f.w;
        }
        if (off & 8) {
#pragma unroll
            for (int i = 0; i < W + 2; ++i) w[i] = w[i + 2];
        }
        if (off & 4) {
#pragma unroll
            for (int i = 0; i < W + 1; ++i) w[i] = w[i + 1];
        }
        if (EB == 2 && (off & 2)) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float f = EB == 4 ? __uint_as_float(w[e]) : e & 1 ? combo_step::widen_hi(w[e / 2]) : combo_step::widen_lo(w[e / 2]);
        v[e] = e < some ? f : 0.0f;
    }
}
// Writes them as bfloat16 planes: each holds what the ones before leave, rounded; towards zero where rounding would overflow.
template <int PLANES> __device__ __forceinline__ void store_planes(unsigned short* to, long long plane, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < PLANES; ++k) {
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[e] = combo_step::pack_bf16(v[2 * e], v[2 * e + 1]);
            if (PLANES > 1) {
                if (fabsf(v[2 * e]) > 3.3895314e38f && fabsf(v[2 * e]) <= 3.4028235e38f) o[e] = (o[e] & 0xffff0000u) | __float_as_uint(v[2 * e]) >> 16;
                if (fabsf(v[2 * e + 1]) > 3.3895314e38f && fabsf(v[2 * e + 1]) <= 3.4028235e38f) o[e] = (o[e] & 0xffffu) | (__float_as_uint(v[2 * e + 1]) & 0xffff0000u);
                v[2 * e] -= combo_step::widen_lo(o[e]);
                v[2 * e + 1] -= combo_step::widen_hi(o[e]);
            }
        }
        *reinterpret_cast<uint4*>(to + k * plane) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// Two planes of float16 of v in units of `unit`.
__device__ __forceinline__ void store_halves(unsigned short* to, long long plane, const float (&v)[8], float per_unit) {
    uint32_t o[2][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 f = make_float2(v[2 * e] * per_unit, v[2 * e + 1] * per_unit);
        const __half2 hi = __floats2half2_rn(f.x, f.y);
        const __half2 lo = __floats2half2_rn(f.x - __low2float(hi), f.y - __high2float(hi));
        o[0][e] = *reinterpret_cast<const uint32_t*>(&hi);
        o[1][e] = *reinterpret_cast<const uint32_t*>(&lo);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) *reinterpret_cast<uint4*>(to + k * plane) = make_uint4(o[k][0], o[k][1], o[k][2], o[k][3]);
}
// The power of two that takes the largest of a warp's finite magnitudes to 2^14 .. 2^15, and its inverse.
__device__ __forceinline__ float unit_of(float most, float& per_unit) {
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 16));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 8));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 4));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
    const int e = most > 0.0f ? max((int)(__float_as_uint(most) >> 23) - 127, -100) : 14;
    per_unit = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
    return __uint_as_float((uint32_t)(127 - 14 + e) << 23);
}
__device__ __forceinline__ float most_of(const float (&v)[8]) {
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[e]) <= 3.4028235e38f ? fabsf(v[e]) : 0.0f);
    return most;
}
// A line of K floats by a warp, kp values and zeros: as halves (what they count in is returned), or as three planes of bfloat16.
__device__ __forceinline__ float store_line(const unsigned char* line, int K, int kp, int vec, int lane, bool halves, unsigned short* to, long long plane) {
    float most = 0.0f, per_unit = 1.0f, unit = 1.0f;
    if (halves) {
        for (int k = lane * 8; k < K; k += 256) {
            float v[8];
            load8<4>(line + (long long)k * 4, K - k, vec, v);
            most = fmaxf(most, most_of(v));
        }
        unit = unit_of(most, per_unit);
    }
    for (int k = lane * 8; k < kp; k += 256) {
        float v[8];
        load8<4>(line + (long long)k * 4, K - k, vec, v);
        if (halves) store_halves(to + k, plane, v, per_unit);
        else store_planes<3>(to + k, plane, v);
    }
    return unit;
}

// Packs the labelled rows, `lot` to a warp, whose places its lanes look up at once; the first CTA leaves the tables of where the workers' rows lie.
template <int EB> __global__ void __launch_bounds__(kThreads) k_pack(const Loss p, const Packed s, int vec, int lot, const Splits splits) {
    extern __shared__ int begins[];                            // packed rows [N + 1]
    __shared__ int sums[kWarps];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    combo_step::pdl_release();
    combo_step::pdl_wait();
    const int per = (p.N + kThreads - 1) / kThreads;
    const auto scan = [&](int unit, int* to, int scale) {      // ascending sums of ceil(count / unit) * scale
        int mine = 0;
        for (int w = t * per; w < min((t + 1) * per, p.N); ++w) mine += (s.count[w] + unit - 1) / unit;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        __syncthreads();
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
        int at = upto - mine;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) at += k < warp ? sums[k] : 0;
        for (int w = t * per; w < min((t + 1) * per, p.N); ++w) {
            to[w] = at * scale;
            at += (s.count[w] + unit - 1) / unit;
        }
        if (t == kThreads - 1) to[p.N] = at * scale;
        __syncthreads();
    };
    scan(kStep, begins, kStep);
    if (blockIdx.x == 0) {
        for (int w = t; w <= p.N; w += kThreads) s.row0[w] = begins[w];
        scan(s.height, s.tiles, 1);
        if (t == 0) s.tiles[p.N + 1] = splits_of(splits, s.tiles[p.N]);
    }
    const int total = begins[p.N];
    const int j0 = (blockIdx.x * kWarps + warp) * lot, rows = min(lot, total - j0);
    int place = -1;                                            // of the lane's row
    if (lane < rows) {
        const int j = j0 + lane;
        int lo = 0, hi = p.N - 1;                              // the last w with begins[w] <= j
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (begins[mid] <= j) lo = mid;
            else hi = mid - 1;
        }
        long long r0, r1;
        rows_of(p, lo, r0, r1);
        const int rank = j - begins[lo], count = s.count[lo];
        if (rank < count) place = s.list[r0 + rank];
        s.src[j] = p.loss ? place : lo;
        s.label[j] = place >= 0 ? (int)p.labels[place] : -1;
        if (!p.loss && place >= 0) {
            s.pos[place] = j;
            s.lse[j] = p.lse_in[place];
            s.g[j] = p.row_grad ? p.row_grad[place] : 1.0f / (float)count;
        }
    }
    for (int i = 0; i < rows; ++i) {
        const int j = j0 + i, from = __shfl_sync(0xffffffffu, place, i);
        if (EB == 4) {
            const float unit = store_line(p.x + from * p.x_pitch * EB, from >= 0 ? p.K : 0, s.kp, vec, lane, p.loss != nullptr,
                                          (p.loss ? s.xh : s.x) + (long long)j * s.kp, s.cap * s.kp);
            if (lane == 0) s.x_unit[j] = unit;
        } else {
            unsigned short* to = s.x + (long long)j * s.kp;
#pragma unroll 4
            for (int k = lane * 8; k < s.kp; k += 256) {
                float v[8];
                load8<EB>(p.x + (from * p.x_pitch + k) * EB, from >= 0 ? p.K - k : 0, vec, v);
                store_planes<1>(to + k, 0, v);
            }
        }
    }
}

// The weights of `classes` classes from v0 on as planes, zeros where there are none: a warp a class where it looks for the largest
// (forward, floats; a piece's units lie `piece` apart), else threads side by side along all of them.
template <int EB> __global__ void __launch_bounds__(kThreads) k_planes(const Loss p, const Packed s, int v0, int classes, int piece, int vec) {
    combo_step::pdl_release();
    combo_step::pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long lines = (long long)p.N * classes, plane = lines * s.kp;
    if (EB == 4 && p.loss) {
        for (long long line = blockIdx.x * (long long)kWarps + (threadIdx.x >> 5); line < lines; line += (long long)gridDim.x * kWarps) {
            const int w = (int)(line / classes), v = v0 + (int)(line - (long long)w * classes);
            const float unit = store_line(p.w + (w * p.w_stride + v * p.w_pitch) * EB, v < p.V ? p.K : 0, s.kp, vec, lane, true, s.wh + line * s.kp, plane);
            if (lane == 0) s.w_unit[(long long)w * piece + (v - v0)] = unit;
        }
        return;
    }
    const unsigned lots = (unsigned)s.kp / 8;
    const long long all = lines * lots;
#pragma unroll 4
    for (long long o = blockIdx.x * (long long)kThreads + threadIdx.x; o < all; o += (long long)gridDim.x * kThreads) {
        const long long line = all < (1LL << 32) ? (unsigned)o / lots : o / lots;
        const int k = (int)(o - line * lots) * 8, w = (int)((unsigned)line / (unsigned)classes), v = v0 + (int)(line - (long long)w * classes);
        float f[8];
        load8<EB>(p.w + (w * p.w_stride + v * p.w_pitch + k) * EB, v < p.V ? p.K - k : 0, vec, f);
        store_planes<EB == 4 ? 3 : 1>(s.w + o * 8, plane, f);
    }
}

// A row's log-sum-exp from its pieces, 32 rows to a CTA, and its loss: a thread takes eight pieces at a time, so that their loads
// and exponentials do not wait for one another.
constexpr int kFinishWarps = 32;
__global__ void __launch_bounds__(kFinishWarps * 32) k_finish(const Loss p, const Packed s, int pieces) {
    __shared__ float sm[2][kFinishWarps][32];
    combo_step::pdl_release();
    combo_step::pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, j = blockIdx.x * 32 + lane;
    if (blockIdx.x * 32 >= s.row0[p.N]) return;
    const int from = s.src[j];
    float m = -INFINITY, sum = 0.0f;
    if (from >= 0) {
        for (int i0 = warp; i0 < pieces; i0 += 8 * warps) {
            float2 v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = i0 + e * warps < pieces ? s.part[(i0 + e * warps) * s.cap + j] : make_float2(-INFINITY, 0.0f);
            float most = m;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, v[e].x);
            const float zero = most == -INFINITY ? 0.0f : most;
            sum *= exp2_fast((m - zero) * kLog2E);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v[e].y * exp2_fast((v[e].x - zero) * kLog2E);
            m = most;
        }
    }
    sm[0][warp][lane] = m;
    sm[1][warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && from >= 0) {
        float most = -INFINITY;
#pragma unroll 8
        for (int k = 0; k < warps; ++k) most = fmaxf(most, sm[0][k][lane]);
        const float zero = most == -INFINITY ? 0.0f : most;
        sum = 0.0f;
#pragma unroll 8
        for (int k = 0; k < warps; ++k) sum += sm[1][k][lane] * exp2_fast((sm[0][k][lane] - zero) * kLog2E);
        // the sum is at least 1: a loss is not below 0, and small ones do not come out of a difference of large logits
        const float rest = logf(sum);
        p.lse[from] = zero + rest;
        p.loss[from] = zero - s.own[j] + rest;
    }
}

// 32 bytes.  An ordinary load that stays behind the wait for the preceding kernel: it may still be writing them while this one starts,
// which the read-only path does not allow for.
__device__ __forceinline__ void load32(const void* from, uint32_t (&v)[8]) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "l"(from)
                 : "memory");
}

// The rows' gradients to their places, a warp `lot` rows whose places its lanes look up at once: the parts of the sums added up,
// zeros for rows without a label.
template <int EB> __global__ void __launch_bounds__(kThreads) k_rows_out(const Loss p, const Packed s, const Pass q, int vec, int w_vec, int lot) {
    combo_step::pdl_release();
    combo_step::pdl_wait();
    const int lane = threadIdx.x & 31, splits = q.tiles[q.N + 1];
    const long long total = q.row0[q.N], a = min(max((long long)p.begin[0], 0LL), p.M), b = min(max((long long)p.begin[p.N], a), p.M);
    const long long m0 = a + (blockIdx.x * (long long)kWarps + (threadIdx.x >> 5)) * lot;
    const int rows = (int)min((long long)lot, b - m0);
    if (rows <= 0) return;
    // of the lane's row
    const int place = lane < rows ? s.pos[m0 + lane] : -1;
    float rest = 0.0f, factor = 1.0f;
    long long weights = 0;
    if (place >= 0) {
        if (!q.scaled) factor = s.g[place];
        if (EB == 2) {
            rest = s.own[place];
            weights = s.src[place] * p.w_stride + s.label[place] * p.w_pitch;
        }
    }
    for (int i0 = 0; i0 < rows; ++i0) {
        const long long m = m0 + i0;
        const int j = __shfl_sync(0xffffffffu, place, i0);
        const float own = __shfl_sync(0xffffffffu, rest, i0), g = __shfl_sync(0xffffffffu, factor, i0);
        const unsigned char* w = p.w + __shfl_sync(0xffffffffu, weights, i0) * EB;
#pragma unroll 1
        for (int k = lane * 8; k < p.K; k += 256) {
            const int left = p.K - k;
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = 0.0f;
            if (j >= 0) {
                for (int i = 0; i < splits; i += 4) {
                    uint32_t v[4][8];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[h][e] = 0u;
                        if (i + h < splits) load32(q.dx + ((i + h) * total + j) * q.dx_pitch + k, v[h]);
                    }
#pragma unroll
                    for (int h = 0; h < 4; ++h)
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] += __uint_as_float(v[h][e]);
                }
                if (EB == 2) {
                    // d of a row's label is most of its gradient: what the plane's rounding left of it comes here
                    float v[8];
                    load8<EB>(w + (long long)k * EB, left, w_vec, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = fmaf(own, v[e], f[e]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] *= g;
            }
            unsigned char* to = p.dx + (m * p.dx_pitch + k) * EB;
            if (vec && left >= 8) {
                if constexpr (EB == 2) {
                    *reinterpret_cast<uint4*>(to) = Elem<2>::pack(f);
                } else {
                    reinterpret_cast<float4*>(to)[0] = make_float4(f[0], f[1], f[2], f[3]);
                    reinterpret_cast<float4*>(to)[1] = make_float4(f[4], f[5], f[6], f[7]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < left) Elem<EB>::put(to + e * EB, f[e]);
            }
        }
    }
}

// ---------------------------------------------------------------- host
bool sizes_ok(int N, int64_t M, int64_t n_in, int64_t n_out, int elem_bytes, int grad_bytes) {
    return (elem_bytes == 2 || elem_bytes == 4) && (grad_bytes == 0 || grad_bytes == 4 || (grad_bytes == 2 && elem_bytes == 2)) && N >= 1 &&
           N <= COMBO_MAX_WORKERS && M >= 0 && M <= COMBO_LINEAR_MAX_ROWS && n_in >= 1 && n_out >= 1 && n_in <= COMBO_LINEAR_MAX_WIDTH &&
           n_out <= COMBO_LINEAR_MAX_WIDTH;
}

constexpr int kSms = 148;
// Aimed at for a piece of classes: d, and the weights' planes.  Pieces that stay in L2 cost more by their launches and by adding
// to dx than reading d from memory does; beyond some 600 MB little is gained.  Measured with 128 / 256 / 384 / 512 MB / 1 GB more than the
// least: gradients of 8 x 326 of 2186 rows, 1024 -> 30001 917 / 721 / 681 / 598 / 599 us, of 4 x 1995, 768 -> 32000 2608 / 1950 / 1867 /
// 1868 / 1932, of 8 x 1000 floats, 256 -> 20000 1803 / 1536 / 1527 / 1350 / 1456; of 2 x 2000, 512 -> 60000 into floats 1401 (640 MB) and
// 1222 (1 GB).  A caller who would rather have the memory gives less.
constexpr size_t kPieceBytes = (size_t)640 << 20;
// Asked for of that for copies of bfloat16 weights, which calls on 16-byte boundaries do not make: forward 8 x 1000 rows, 1023 ->
// 30001 722 us (128 MB), 641 (256 MB), 601 (all, 491 MB).
constexpr size_t kCopyBytes = (size_t)1 << 28;

// How a call is computed, by its sizes alone.
struct Plan {
    bool few;
    int cg, halves, planes, d_planes, kp;        // planes of x and w, float16 and bfloat16; of d
    int out_warps;                               // of the logits' kernels, that take results
    int v_width, k_width, unit;                  // tiles along the classes, along the inputs; pieces are multiples of `unit`
    long long cap;
    long long dx_rows;                           // of the sums for dx, all splits
    size_t x, part, dx, region;                  // places in scratch
    size_t room, least, total;                   // bytes of the region for pieces; of scratch, at least and as it pays
};

size_t up(size_t n, size_t unit) { return (n + unit - 1) / unit * unit; }

int even_width(int64_t n, int most, int unit) {
    const int64_t tiles = (n + most - 1) / most;
    return (int)up((size_t)((n + tiles - 1) / tiles), unit);
}

// Classes whose weights a piece has planes of.
size_t lines_of(size_t piece, size_t V) { return piece < up(V, 8) ? piece : up(V, 8); }

// Bytes of a piece of so many classes: of d, and of the weights' planes.
size_t d_bytes(const Plan& a, size_t piece) { return up(piece * a.cap * a.d_planes * 2, 256); }
size_t planes_bytes(const Plan& a, int N, size_t V, size_t piece) {
    return up((size_t)N * (lines_of(piece, V) * a.kp * (a.planes + a.halves) * 2 + (a.halves ? piece * 4 : 0)), 256);
}
size_t piece_bytes(const Plan& a, int N, size_t V, size_t piece, bool back, bool direct) {
    return (back ? d_bytes(a, piece) : 0) + (direct ? 0 : planes_bytes(a, N, V, piece));
}

Plan plan_of(int N, int64_t M, int64_t K, int64_t V, int elem_bytes, int grad_bytes) {
    Plan a = {};
    const bool back = grad_bytes != 0;
    // Few multiply-adds: one launch, or two, against four and seven.  Measured, 8 workers, few / tensor cores: loss of 1336 rows, 256 ->
    // 64, floats 11.9 / 23.9 us, 512 -> 256 54 / 41; bfloat16 11.3 / 17.0, 47 / 20; gradients 28.6 / 53.5, 147 / 82 and 36 / 38,
    // 160 / 45; of 8000 rows, 256 -> 10, 86 / 84 and 113 / 46; many classes of few inputs take a warp many turns (16 -> 1000: 75 to 300).
    a.few = M == 0 || (M <= 2048 && V <= kFewClasses && V * K <= (elem_bytes == 4 ? 1 << 15 : 1 << 14));
    if (a.few) {
        a.total = a.least = 256 + (back ? (size_t)M * V * 4 : 0);
        return a;
    }
    // Pairs of CTAs halve what a product takes from L2, single ones waste less of ragged rows.  Measured (pairs / single): loss of 8 x
    // 300 rows, 128 -> 8000, floats 66 / 61 us, bfloat16 36 / 33; of 8 x 817, 1024 -> 30001, 359 / 414; gradients of 8 x 250, 256 ->
    // 1000, floats 91 / 74, bfloat16 46 / 43; of 8 x 1000, 256 -> 8000 622 / 696 and 174 / 183.
    a.cg = M / N > 128 && (back ? V * K > (1 << 19) : K > 512) ? 2 : 1;
    // Sixteen warps for the results hide each other's waits where a tile's products take less time than they do; eight keep more in
    // registers.  Measured (16 / 8): loss of 8 x 1000 rows, 40 -> 20000, floats 203 / 243 us, 512 -> 8000 258 / 280, bfloat16
    // 1024 -> 30001 373 / 359; gradients of 8 x 1000 rows, bfloat16 40 -> 20000 281 / 298, of 8 x 326, 1024 -> 30001 640 / 629; with
    // three planes of d to write, 4 x 1995 rows, 768 -> 32000 1777 / 1887, 5 x 1000, 1216 -> 9213 529 / 525.
    a.out_warps = K <= (elem_bytes == 2 && grad_bytes == 4 ? 1024 : 512) ? 16 : 8;
    a.halves = elem_bytes == 4 && !back ? 2 : 0;
    a.planes = elem_bytes == 2 ? 1 : back ? 3 : 0;
    // A bfloat16 dW of few rows takes two planes: sums of a row or two do not average the rounding of d, which came on top of their own
    // (off by up to 3.8e-3 of their size, now by 1.7e-3 as bfloat16 is; of many rows 2.4e-3).  Measured (two / one): 16 x 1 row, 1024 ->
    // 32000 637 / 626 us, 16 x 120 821 / 782, 43 x 37, 128 -> 22408 302 / 273; of many rows it is one more of three products.
    a.d_planes = grad_bytes == 4 ? 3 : grad_bytes == 2 && M <= 128LL * N ? 2 : 1;
    a.kp = (int)up(K, 64);
    const int most = elem_bytes == 4 && back && a.cg == 1 ? 128 : 256;       // two stages in shared memory
    a.v_width = even_width(V, most, 128);
    a.k_width = even_width(K, most, 128);
    if (V > 1024) a.v_width = most;
    a.unit = a.v_width;
    a.cap = (long long)up(M + 63 * (N < M ? N : M), 64);
    const size_t cap = (size_t)a.cap;
    size_t at = up((size_t)N * 4, 256) + 2 * up((size_t)M * 4, 256) + 2 * up((size_t)(N + 2) * 4, 256) + 6 * up(cap * 4, 256);
    a.x = at;
    at += up(cap * a.kp * (a.planes + a.halves) * 2, 256);
    a.part = at;
    if (!back) {
        at += up(a.out_warps / 4 * up(V, a.v_width) / a.v_width * cap * 8, 256);
    } else {
        const size_t wt = up(K, a.k_width) / a.k_width, split_rows = (size_t)kMaxTurns * (kSms / a.cg) / wt * 128 * a.cg;
        a.dx = at;
        a.dx_rows = (long long)(cap > split_rows ? cap : split_rows);
        at += up((size_t)a.dx_rows * wt * a.k_width * 4, 256);
    }
    a.region = at;
    const size_t all = up(V, a.unit), copy = planes_bytes(a, N, V, all), least = piece_bytes(a, N, V, a.unit, back, false);
    a.room = (back ? d_bytes(a, all) : 0) + (elem_bytes == 4 || copy < kCopyBytes ? copy : kCopyBytes);
    if (a.room > kPieceBytes) a.room = kPieceBytes;
    if (a.room < least) a.room = least;
    a.total = at + a.room;
    a.least = at + least;
    return a;
}

// Tensor map of elements of eb bytes; boxes of 128 bytes, swizzled, by `rows`, or of `plain` elements without a swizzle.
bool map_of(CUtensorMap* map, void* base, int eb, int rank, const long long* dims, const long long* strides, int rows, int plain = 0) {
    cuuint64_t d[4], s[3];
    const cuuint32_t box[4] = {plain ? (cuuint32_t)plain : 128u / eb, (cuuint32_t)rows, 1, 1}, ones[4] = {1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) d[i] = (cuuint64_t)dims[i];
    for (int i = 0; i + 1 < rank; ++i) s[i] = (cuuint64_t)strides[i] * eb;
    const CUtensorMapDataType type = eb == 8 ? CU_TENSOR_MAP_DATA_TYPE_UINT64 : eb == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return combo_host::encode_tiled(map, type, rank, base, d, s, box, ones, plain ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int CG, int MODE, int PA, int PB, int OB, int kOutWarps = 8> cudaError_t launch_loss(Pass q, const Maps& maps, long long tiles, int sms, int smem_optin, cudaStream_t st) {
    static uint64_t allowed;
    auto kern = k_loss<CG, MODE, PA, PB, OB, kOutWarps>;
    const int turn = MODE == kWeights && !q.vec ? kOutWarps * kTurn : MODE == kRows || MODE == kWeights ? kOutWarps * kPut : 0, most = smem_optin - kStaticSmem;
    q.stage_bytes = (PA * 2 + PB * (q.width / CG / 64)) * kBlock;
    q.stages = (most - 1024 - turn) / q.stage_bytes;
    if (q.stages > kMaxStages) q.stages = kMaxStages;
    cudaError_t e = combo_host::allow_smem(kern, most, &allowed);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles < sms / CG ? tiles : sms / CG) * CG);
    cfg.blockDim = dim3(out_threads(kOutWarps));
    cfg.dynamicSmemBytes = 1024 + (size_t)q.stages * q.stage_bytes + turn;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, q, maps);
}

// EB: bytes of the inputs; GB: of dW (0: forward); D: planes of d.
template <int CG, int EB, int GB, int D> cudaError_t run_tensor(const Plan& a, const Loss& p, unsigned char* scratch, int sms, int smem_optin, cudaStream_t st) {
    constexpr bool kBack = GB != 0;
    constexpr int P = EB == 4 ? 3 : 1, L = EB == 2 ? 1 : kBack ? 3 : 2;      // planes: of the gradients' products, of the logits'
    const auto vec_ok = [](const void* b, long long pitch, long long stride, int eb) {
        return combo_host::aligned_to(b, 16) && pitch * eb % 16 == 0 && stride * eb % 16 == 0;
    };
    Packed s = {};
    s.cap = a.cap;
    s.kp = a.kp;
    s.height = 128 * CG;
    size_t at = 0;
    const auto take = [&](size_t bytes) { unsigned char* r = scratch + at; at += up(bytes, 256); return r; };
    const size_t cap = (size_t)a.cap;
    s.count = reinterpret_cast<int*>(take((size_t)p.N * 4));
    s.list = reinterpret_cast<int*>(take((size_t)p.M * 4));
    s.pos = reinterpret_cast<int*>(take((size_t)p.M * 4));
    s.row0 = reinterpret_cast<int*>(take((size_t)(p.N + 2) * 4));
    s.tiles = reinterpret_cast<int*>(take((size_t)(p.N + 2) * 4));
    s.src = reinterpret_cast<int*>(take(cap * 4));
    s.label = reinterpret_cast<int*>(take(cap * 4));
    s.lse = reinterpret_cast<float*>(take(cap * 4));
    s.g = reinterpret_cast<float*>(take(cap * 4));
    s.own = reinterpret_cast<float*>(take(cap * 4));
    s.x_unit = reinterpret_cast<float*>(take(cap * 4));
    s.xh = reinterpret_cast<unsigned short*>(scratch + a.x);
    s.x = s.xh + cap * a.kp * a.halves;
    s.part = reinterpret_cast<float2*>(scratch + a.part);
    s.dx = reinterpret_cast<float*>(scratch + a.dx);

    // bfloat16 weights on 16-byte boundaries are read where they lie
    const bool w_vec = vec_ok(p.w, p.w_pitch, p.w_stride, EB), direct = EB == 2 && w_vec && p.w_pitch < (1LL << 36) && p.w_stride < (1LL << 36);
    int piece = (int)up(p.V, a.unit);
    for (int n = 2; piece > a.unit && !(direct && !kBack) && piece_bytes(a, p.N, p.V, piece, kBack, direct) > a.room; ++n)
        piece = (int)up((p.V + n - 1) / n, a.unit);
    const int there = (int)lines_of(piece, p.V);               // classes whose weights have planes
    s.d = reinterpret_cast<unsigned short*>(scratch + a.region);
    s.w_unit = reinterpret_cast<float*>(s.d + (kBack ? d_bytes(a, piece) / 2 : 0));
    s.wh = reinterpret_cast<unsigned short*>(s.w_unit + (a.halves ? (size_t)piece * p.N : 0));
    s.w = s.wh + (size_t)there * p.N * a.kp * a.halves;

    cudaError_t e = combo_host::launch_after(k_count, dim3(p.N), dim3(kCountThreads), 0, st, p, s);
    if (e != cudaSuccess) return e;
    // a part's sums: 128 KB a CTA, at 5 TB/s each way, against 0.29 us a stage (floats six times)
    const int kt = (p.K + a.k_width - 1) / a.k_width, whole = (int)(piece < (long long)up(p.V, 64) ? piece : up(p.V, 64)) / kStep;
    const Splits splits = {kSms / CG, kt, whole, 0.125f * CG / (EB == 4 ? 6 : 1)};
    const long long pack_per = a.cap / (sms * 64);
    const int pack_lot = pack_per < 1 ? 1 : pack_per > 8 ? 8 : (int)pack_per;
    e = combo_host::launch_after(k_pack<EB>, dim3((unsigned)((a.cap + pack_lot * kWarps - 1) / (pack_lot * kWarps))), dim3(kThreads), (size_t)(p.N + 1) * 4, st, p,
                                 s, (int)vec_ok(p.x, p.x_pitch, 0, EB), pack_lot, splits);
    if (e != cudaSuccess) return e;

    // bfloat16 or floats by whole boxes where 16-byte boundaries allow
    const bool dw_vec = kBack && vec_ok(p.dw, p.dw_pitch, p.dw_stride, kBack ? GB : 4) && p.dw_pitch < (1LL << 36) && p.dw_stride < (1LL << 36);
    const long long dx_pitch = kt * a.k_width;
    CUtensorMap mx = {}, mw = {}, mxh = {}, mwh = {}, md = {}, mdw = {}, out_dx = {}, out_dw = {};
    const long long lines = (long long)there * a.kp, flat = a.cap * a.kp;
    const long long xd[3] = {a.kp, a.cap, P}, hd[3] = {a.kp, a.cap, L}, xs[2] = {a.kp, flat};
    const long long wd[4] = {direct ? p.K : a.kp, direct ? p.V : there, p.N, direct ? 1 : P}, vd[4] = {a.kp, there, p.N, L};
    const long long ws[3] = {direct ? p.w_pitch : a.kp, direct ? (p.N > 1 ? p.w_stride : 8) : lines, direct ? 8 : lines * p.N};
    // d: eight classes of a row in 16 bytes, rows side by side, so that a warp that writes and a box that is read run along memory;
    // in 64-bit units, of which a box may have 256
    const long long dd[3] = {2 * a.cap, piece / 8, D}, ds[2] = {a.cap * 2, a.cap * 2 * (piece / 8)};
    bool fine = (EB == 4 && !kBack) || (map_of(&mx, s.x, 2, 3, xd, xs, 64) &&
                                        map_of(&mw, direct ? const_cast<unsigned char*>(p.w) : reinterpret_cast<unsigned char*>(s.w), 2, 4, wd, ws, 64));
    if (L == 2 && fine) fine = map_of(&mxh, s.xh, 2, 3, hd, xs, 64) && map_of(&mwh, s.wh, 2, 4, vd, ws, 64);
    if (kBack && fine) {
        const long long rd[3] = {dx_pitch, a.dx_rows, 1}, rs[2] = {dx_pitch, 8};
        const long long gd[3] = {p.K, p.V, p.N}, gs[2] = {p.dw_pitch, p.N > 1 ? p.dw_stride : 8};
        fine = map_of(&md, s.d, 8, 3, dd, ds, 8, 256) && map_of(&mdw, s.d, 8, 3, dd, ds, 16, 128) && map_of(&out_dx, s.dx, 4, 3, rd, rs, 32) &&
               (!dw_vec || map_of(&out_dw, p.dw, kBack ? GB : 4, 3, gd, gs, 32));
    }
    if (!fine) return cudaErrorInvalidValue;

    Pass q = {};
    q.row0 = s.row0;
    q.tiles = s.tiles;
    q.N = p.N;
    q.V = p.V;
    q.K = p.K;
    q.row_cap = a.cap;
    q.count = s.count;
    q.x_unit = s.x_unit;
    q.w_unit = s.w_unit;
    q.piece = piece;
    q.d = reinterpret_cast<unsigned char*>(s.d);
    q.d_blocks = piece / 8;
    q.scaled = p.row_grad != nullptr;
    q.label = s.label;
    q.lse = s.lse;
    q.g = s.g;
    q.part = s.part;
    q.own = s.own;
    q.dx = s.dx;
    q.dw = p.dw;
    q.dw_pitch = p.dw_pitch;
    q.dw_stride = p.dw_stride;
    q.dx_pitch = dx_pitch;
    // Where classes are few, exponentials near 1 hand the logits' errors on, and shorter parts cost little, the classes' tile being one.
    // Gradients of the weights off by, and time (shorter / as of more classes): floats, 13 x 1800 rows, 128 -> 18, 2.5e-7, 98 us /
    // 1.4e-6, 91; floats of bfloat16, 3 x 1200, 1408 -> 14, 5.6e-7, 111 / 1.7e-6, 109.  Of many classes: floats, 8 x 250, 512 -> 10000,
    // 539 / 498 us, floats of bfloat16, 4 x 1995, 768 -> 32000, 2092 / 1770, both off by less than 1e-6 as they are.
    const bool few_classes = p.V <= kFewClasses;
    const long long row_tiles = p.M / s.height + (p.N < p.M ? p.N : p.M);          // at most
    for (int v0 = 0; v0 < p.V; v0 += piece) {
        const int classes = p.V - v0 < piece ? p.V - v0 : piece;
        if (!direct) {
            const long long grid = ((long long)p.N * there + kWarps - 1) / kWarps;
            e = combo_host::launch_after(k_planes<EB>, dim3((unsigned)(grid < sms * 16 ? grid : sms * 16)), dim3(kThreads), 0, st, p, s, v0, there, piece, (int)w_vec);
            if (e != cudaSuccess) return e;
        }
        q.v0 = v0;
        q.v_end = v0 + classes;
        q.w_row = direct ? v0 : 0;
        q.width = a.v_width;
        q.wt = (classes + a.v_width - 1) / a.v_width;
        q.steps = a.kp / kStep;
        q.part_steps = EB == 4 ? kBack && few_classes ? 1 : 2 : GB == 4 && few_classes ? 4 : 16;
        const Maps logits_of = L == 2 ? Maps{mxh, mwh, mwh} : Maps{mx, mw, mw};
        constexpr int kMode = kBack ? kGrad : kStats, kOut = kBack ? D : 1;
        constexpr int kMost = CG == 2 && !kBack ? 8 : 16;              // forward, pairs take more than 512 inputs
        e = a.out_warps == kMost ? launch_loss<CG, kMode, L, L, kOut, kMost>(q, logits_of, row_tiles * q.wt, sms, smem_optin, st)
                                 : launch_loss<CG, kMode, L, L, kOut, 8>(q, logits_of, row_tiles * q.wt, sms, smem_optin, st);
        if (e != cudaSuccess) return e;
        if constexpr (kBack) {
            q.width = a.k_width;
            q.wt = kt;
            q.steps = (classes + kStep - 1) / kStep;
            q.add = v0 > 0;
            if (EB == 2) q.part_steps = 16;
            // bfloat16 rows take the first plane of d: the others are below their rounding
            e = launch_loss<CG, kRows, EB == 4 ? 3 : 1, P, 1>(q, Maps{md, mw, out_dx}, row_tiles * kt * kMaxSplits, sms, smem_optin, st);
            if (e != cudaSuccess) return e;
            q.ht = (classes + s.height - 1) / s.height;
            // Floats of bfloat16 take d to 24 bits, in three planes, and are summed in shorter parts: off by 6e-7 of their size (4 x
            // 1995 rows; 1.1e-6 in parts of 512, for a hundredth of the time; 2.5e-6 with two planes, for a quarter).
            if (EB == 2 && GB == 4) q.part_steps = few_classes ? 2 : 4;
            q.vec = dw_vec;
            e = launch_loss<CG, kWeights, D, P, GB>(q, Maps{mdw, mx, out_dw}, (long long)p.N * kt * q.ht, sms, smem_optin, st);
            if (e != cudaSuccess) return e;
        }
    }
    if (!kBack) {
        const int pieces = a.out_warps / 4 * ((p.V + a.v_width - 1) / a.v_width), warps = pieces >= 8 * kFinishWarps ? kFinishWarps : pieces / 8 < 4 ? 4 : pieces / 8;
        return combo_host::launch_after(k_finish, dim3((unsigned)((cap + 31) / 32)), dim3(warps * 32), 0, st, p, s, pieces);
    }
    // several rows to a warp where there are many: one search for all, but rows wait for one another
    const long long per = p.M / (sms * 128);
    const int lot = per < 1 ? 1 : per > 8 ? 8 : (int)per;
    return combo_host::launch_after(k_rows_out<EB>, dim3((unsigned)((p.M + lot * kWarps - 1) / (lot * kWarps))), dim3(kThreads), 0, st, p, s, q,
                                    (int)vec_ok(p.dx, p.dx_pitch, 0, EB), (int)w_vec, lot);
}

template <int CG> cudaError_t launch_tensor(const Plan& a, const Loss& p, int elem_bytes, int grad_bytes, void* scratch, int sms, int smem_optin, cudaStream_t st) {
    unsigned char* b = static_cast<unsigned char*>(scratch);
    if (elem_bytes == 4) return grad_bytes ? run_tensor<CG, 4, 4, 3>(a, p, b, sms, smem_optin, st) : run_tensor<CG, 4, 0, 1>(a, p, b, sms, smem_optin, st);
    if (grad_bytes == 4) return run_tensor<CG, 2, 4, 3>(a, p, b, sms, smem_optin, st);
    if (grad_bytes == 0) return run_tensor<CG, 2, 0, 1>(a, p, b, sms, smem_optin, st);
    if constexpr (CG == 1) {                         // pairs have more rows a worker
        if (a.d_planes == 2) return run_tensor<1, 2, 2, 2>(a, p, b, sms, smem_optin, st);
    }
    return run_tensor<CG, 2, 2, 1>(a, p, b, sms, smem_optin, st);
}

combo_status cross_entropy(Loss p, int elem_bytes, int grad_bytes, int64_t n_in, int64_t n_out, void* scratch, size_t scratch_bytes, void* stream) {
    if (!sizes_ok(p.N, p.M, n_in, n_out, elem_bytes, grad_bytes)) return COMBO_ERR_INVALID_ARG;
    const bool back = grad_bytes != 0;
    if (!p.begin || !combo_host::aligned_to(p.begin, 8)) return COMBO_ERR_INVALID_ARG;
    if (!scratch || !combo_host::aligned_to(scratch, 256) || scratch_bytes < plan_of(p.N, p.M, n_in, n_out, elem_bytes, grad_bytes).least)
        return COMBO_ERR_INVALID_ARG;
    if (p.M > 0) {
        if (!p.x || !p.labels || p.x_pitch < n_in || p.x_pitch > (1LL << 40) / p.M) return COMBO_ERR_INVALID_ARG;
        if (!combo_host::aligned_to(p.x, elem_bytes) || !combo_host::aligned_to(p.labels, 8)) return COMBO_ERR_INVALID_ARG;
        if (back ? !p.lse_in || !p.dx || p.dx_pitch < n_in || p.dx_pitch > (1LL << 40) / p.M : !p.loss || !p.lse) return COMBO_ERR_INVALID_ARG;
        if (!combo_host::aligned_to(p.loss, 4) || !combo_host::aligned_to(p.lse, 4) || !combo_host::aligned_to(p.lse_in, 4) ||
            !combo_host::aligned_to(p.row_grad, 4) || !combo_host::aligned_to(p.dx, elem_bytes))
            return COMBO_ERR_INVALID_ARG;
    }
    const auto weights_ok = [&](const void* w, int64_t pitch, int64_t stride, int eb) {
        return w && combo_host::aligned_to(w, eb) && pitch >= n_in && pitch <= (1LL << 40) / n_out &&
               (p.N == 1 || (stride >= (n_out - 1) * pitch + n_in && stride <= (1LL << 44) / p.N));
    };
    if (!weights_ok(p.w, p.w_pitch, p.w_stride, elem_bytes) || (back && !weights_ok(p.dw, p.dw_pitch, p.dw_stride, grad_bytes))) return COMBO_ERR_INVALID_ARG;
    if (p.N == 1) p.w_stride = p.dw_stride = 0;
    // what is written must not overlap what is read, nor another output
    const auto bytes_of = [&](int64_t pitch, int64_t stride, int eb) { return ((size_t)(p.N - 1) * stride + (n_out - 1) * pitch + n_in) * eb; };
    const size_t m = (size_t)p.M;
    const combo_host::Rows x = {p.x, p.M, (size_t)n_in * elem_bytes, (size_t)p.x_pitch * elem_bytes};
    const combo_host::Rows dx = {p.dx, back ? p.M : 0, (size_t)n_in * elem_bytes, (size_t)p.dx_pitch * elem_bytes};
    struct Span { const void* p; size_t n; };
    const Span in[] = {{p.x, x.extent()}, {p.w, bytes_of(p.w_pitch, p.w_stride, elem_bytes)}, {p.labels, m * 8}, {p.begin, ((size_t)p.N + 1) * 8},
                       {p.lse_in, p.lse_in ? m * 4 : 0}, {p.row_grad, p.row_grad ? m * 4 : 0}};
    const Span out[] = {{p.dx, dx.extent()}, {p.dw, back ? bytes_of(p.dw_pitch, p.dw_stride, grad_bytes) : 0}, {p.loss, back ? 0 : m * 4},
                        {p.lse, back ? 0 : m * 4}, {scratch, scratch_bytes}};
    for (int i = 0; i < 5; ++i) {
        for (int k = 0; k < 6; ++k)
            if (combo_host::overlap(out[i].p, out[i].n, in[k].p, in[k].n) && !(i == 0 && k == 0 && !combo_host::overlap(dx, x))) return COMBO_ERR_ALIAS;
        for (int k = 0; k < i; ++k)
            if (combo_host::overlap(out[i].p, out[i].n, out[k].p, out[k].n)) return COMBO_ERR_ALIAS;
    }
    int sms = 0, smem = 0;
    const combo_status rc = combo_host::device(&sms, &smem);
    if (rc != COMBO_OK) return rc;
    if (p.M == 0 && !back) return COMBO_OK;
    p.K = (int)n_in;
    p.V = (int)n_out;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    Plan plan = plan_of(p.N, p.M, n_in, n_out, elem_bytes, grad_bytes);
    // what there is, up to what pays
    const size_t given = scratch_bytes - plan.region, pays = plan.room > kPieceBytes ? plan.room : kPieceBytes;
    plan.room = given < pays ? given : pays;
    combo_host::set_step_path(plan.few ? combo_host::kPathMultiplyAdd : plan.cg == 2 ? combo_host::kPathTensorPairs : combo_host::kPathTensor);
    if (!plan.few) {
        e = plan.cg == 2 ? launch_tensor<2>(plan, p, elem_bytes, grad_bytes, scratch, sms, smem, st)
                         : launch_tensor<1>(plan, p, elem_bytes, grad_bytes, scratch, sms, smem, st);
        return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "cross entropy launch");
    }
    p.d = static_cast<float*>(scratch);
    const auto vec_ok = [&](const void* a, int64_t pitch, int64_t stride) {
        return combo_host::aligned_to(a, 16) && pitch * elem_bytes % 16 == 0 && stride * elem_bytes % 16 == 0;
    };
    const bool vec = vec_ok(p.x, p.x_pitch, 0) && vec_ok(p.w, p.w_pitch, p.w_stride);
    if (elem_bytes == 4) e = vec ? launch_few<4, true>(p, grad_bytes, st) : launch_few<4, false>(p, grad_bytes, st);
    else e = vec ? launch_few<2, true>(p, grad_bytes, st) : launch_few<2, false>(p, grad_bytes, st);
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "cross entropy launch");
}

}  // namespace

namespace combo_host {

cudaError_t cross_entropy_status(int* code) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(code, combo_loss::g_loss_status, sizeof(int));
    if (e == cudaSuccess && *code != 0) e = cudaMemcpyToSymbol(combo_loss::g_loss_status, &zero, sizeof(int));
    return e;
}

}  // namespace combo_host

extern "C" {

size_t combo_grouped_cross_entropy_scratch_bytes(int N, int64_t M, int64_t n_in, int64_t n_out, int elem_bytes, int grad_bytes) {
    return sizes_ok(N, M, n_in, n_out, elem_bytes, grad_bytes) ? plan_of(N, M, n_in, n_out, elem_bytes, grad_bytes).total : 0;
}

size_t combo_grouped_cross_entropy_least_scratch_bytes(int N, int64_t M, int64_t n_in, int64_t n_out, int elem_bytes, int grad_bytes) {
    return sizes_ok(N, M, n_in, n_out, elem_bytes, grad_bytes) ? plan_of(N, M, n_in, n_out, elem_bytes, grad_bytes).least : 0;
}

combo_status combo_grouped_cross_entropy(const void* x, int64_t x_pitch, const void* w, int64_t w_pitch, int64_t w_stride, int elem_bytes,
                                         const int64_t* d_labels, const int64_t* d_begin, int N, int64_t M, int64_t n_in, int64_t n_out,
                                         float* loss_out, float* lse_out, void* scratch, size_t scratch_bytes, void* stream) {
    Loss p = {};
    p.x = static_cast<const unsigned char*>(x);
    p.x_pitch = x_pitch;
    p.w = static_cast<const unsigned char*>(w);
    p.w_pitch = w_pitch;
    p.w_stride = w_stride;
    p.labels = d_labels;
    p.begin = d_begin;
    p.N = N;
    p.M = M;
    p.loss = loss_out;
    p.lse = lse_out;
    return cross_entropy(p, elem_bytes, 0, n_in, n_out, scratch, scratch_bytes, stream);
}

combo_status combo_grouped_cross_entropy_backward(const void* x, int64_t x_pitch, const void* w, int64_t w_pitch, int64_t w_stride,
                                                  int elem_bytes, const int64_t* d_labels, const float* lse, const float* row_grad, void* dx,
                                                  int64_t dx_pitch, void* dw, int64_t dw_pitch, int64_t dw_stride, int grad_bytes,
                                                  const int64_t* d_begin, int N, int64_t M, int64_t n_in, int64_t n_out, void* scratch,
                                                  size_t scratch_bytes, void* stream) {
    if (grad_bytes == 0) return COMBO_ERR_INVALID_ARG;
    Loss p = {};
    p.x = static_cast<const unsigned char*>(x);
    p.x_pitch = x_pitch;
    p.w = static_cast<const unsigned char*>(w);
    p.w_pitch = w_pitch;
    p.w_stride = w_stride;
    p.labels = d_labels;
    p.lse_in = lse;
    p.row_grad = row_grad;
    p.dx = static_cast<unsigned char*>(dx);
    p.dx_pitch = dx_pitch;
    p.dw = static_cast<unsigned char*>(dw);
    p.dw_pitch = dw_pitch;
    p.dw_stride = dw_stride;
    p.begin = d_begin;
    p.N = N;
    p.M = M;
    return cross_entropy(p, elem_bytes, grad_bytes, n_in, n_out, scratch, scratch_bytes, stream);
}

}  // extern "C"
