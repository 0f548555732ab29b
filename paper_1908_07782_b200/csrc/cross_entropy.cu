// Softmax cross entropy of a linear classifier, grouped by worker; the logits are never kept.
//
//   z_mv = x_m . W_w,v      lse_m = log sum_v exp z_mv      loss_m = lse_m - z_m,label        m in worker w's rows, v a class
//   d_mv = (exp(z_mv - lse_m) - [v = label_m]) g_m          dx_m = sum_v d_mv W_w,v           dW_w,v = sum_m d_mv x_m
#include <string.h>

#include "host_common.h"
#include "step_common.cuh"

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
constexpr int kThreads = 256, kWarps = kThreads / 32, kR = 8, kU = 4;

// The worker and first row of lot `block` of kR rows, workers counted through kThreads at a time; false behind the last.
__device__ __forceinline__ bool find_rows(const Loss& p, long long block, int& w, long long& i0, long long& i1) {
    __shared__ int lots[kThreads];
    long long before = 0;
    const int t = threadIdx.x;
    for (int w0 = 0; w0 < p.N; w0 += kThreads) {
        long long a = 0, b = 0;
        if (w0 + t < p.N) rows_of(p, w0 + t, a, b);
        lots[t] = (int)((b - a + kR - 1) / kR);
        __syncthreads();
        for (int k = 0; k < kThreads && w0 + k < p.N; ++k) {
            if (block < before + lots[k]) {
                w = w0 + k;
                rows_of(p, w, i0, i1);
                i0 += (block - before) * kR;
                return true;
            }
            before += lots[k];
        }
        __syncthreads();
    }
    return false;
}

// A lane's share of a line of K elements, step `c` of ceil(K / (32 E)): E neighbours in 16 bytes, or elements 32 apart.
template <int EB, bool VEC> __device__ __forceinline__ void load_share(const unsigned char* line, int c, int lane, int K, float (&v)[Elem<EB>::V]) {
    constexpr int E = Elem<EB>::V;
    if (VEC) {
        const int k = (c * 32 + lane) * E;
        if (k + E <= K) {
            Elem<EB>::unpack(*reinterpret_cast<const uint4*>(line + (long long)k * EB), v);
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
        const float lse = m + logf(s);
        p.lse[i0 + r] = where[r] >= 0 ? lse : 0.0f;
        p.loss[i0 + r] = where[r] >= 0 ? lse - (&sm[2][0][0])[where[r]] : 0.0f;
    }
}

// What the warps hold for `lines` x (32 E) results, acc[line][e] a lane, added up in the warps' order and given to put(line, k, sum).
template <int EB, bool VEC, typename F>
__device__ __forceinline__ void join_warps(const float (&acc)[kR][Elem<EB>::V], int c, int lane, int warp, F put) {
    constexpr int E = Elem<EB>::V;
    __shared__ float sm[kWarps][2][32 * E + 1];
#pragma unroll
    for (int h = 0; h < kR; h += 2) {
        __syncthreads();
#pragma unroll
        for (int l = 0; l < 2; ++l)
#pragma unroll
            for (int e = 0; e < E; ++e) sm[warp][l][e * 32 + lane] = acc[h + l][e];
        __syncthreads();
        for (int o = threadIdx.x; o < 2 * 32 * E; o += kThreads) {
            const int l = o / (32 * E), at = o % (32 * E);
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) sum += sm[k][l][VEC ? at % E * 32 + at / E : at];
            put(h + l, c * 32 * E + at, sum);
        }
    }
}

template <int EB, bool VEC> __global__ void __launch_bounds__(kThreads) k_few_back(const Loss p) {
    constexpr int E = Elem<EB>::V;
    int w;
    long long i0, i1;
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
    for (int v0 = warp * kU; v0 < p.V; v0 += kWarps * kU) {
        const float z = logits<EB, VEC>(p, x0, rows, w0, v0, lane);
        const int v = v0 + lane / kR;
        if (v < p.V && row < rows) p.d[(i0 + row) * p.V + v] = has ? (expf(z - lse) - (v == label ? 1.0f : 0.0f)) * g : 0.0f;
    }
    __syncthreads();
    const float* d = p.d + i0 * p.V;
    const unsigned some = __ballot_sync(0xffffffffu, has && lane < kR);
    for (int c = 0; c * 32 * E < p.K; ++c) {
        float acc[kR][E];
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[r][e] = 0.0f;
        for (int v = warp; v < p.V; v += kWarps) {
            float wv[E];
            load_share<EB, VEC>(w0 + (long long)v * p.w_pitch * EB, c, lane, p.K, wv);
#pragma unroll
            for (int r = 0; r < kR; ++r) {
                if (some >> r & 1u) {
                    const float f = d[(long long)r * p.V + v];
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[r][e] = fmaf(f, wv[e], acc[r][e]);
                }
            }
        }
        join_warps<EB, VEC>(acc, c, lane, warp, [&](int r, int k, float sum) {
            if (r < rows && k < p.K) Elem<EB>::put(p.dx + ((i0 + r) * p.dx_pitch + k) * EB, sum);
        });
    }
}

// Eight classes' gradients of one worker by 32 E columns; warps share out the rows.
template <int EB, int OB, bool VEC> __global__ void __launch_bounds__(kThreads) k_few_weights(const Loss p) {
    constexpr int E = Elem<EB>::V;
    const int w = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x;
    long long i0, i1;
    rows_of(p, w, i0, i1);
    for (int v0 = blockIdx.y * kR; v0 < p.V; v0 += gridDim.y * kR) {
        float acc[kR][E];
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[r][e] = 0.0f;
        for (long long i = i0 + warp; i < i1; i += kWarps) {
            const int64_t label = p.labels[i];
            if (label < 0 || label >= p.V) continue;
            float xv[E];
            load_share<EB, VEC>(p.x + i * p.x_pitch * EB, c, lane, p.K, xv);
#pragma unroll
            for (int r = 0; r < kR; ++r) {
                const float f = p.d[i * p.V + min(v0 + r, p.V - 1)];
#pragma unroll
                for (int e = 0; e < E; ++e) acc[r][e] = fmaf(f, xv[e], acc[r][e]);
            }
        }
        join_warps<EB, VEC>(acc, c, lane, warp, [&](int r, int k, float sum) {
            if (v0 + r < p.V && k < p.K) Elem<OB>::put(p.dw + (w * p.dw_stride + (v0 + r) * p.dw_pitch + k) * OB, sum);
        });
    }
}

template <int EB, bool VEC> cudaError_t launch_few(const Loss& p, int grad_bytes, cudaStream_t st) {
    const long long lots = p.M / kR + (p.N < p.M ? p.N : p.M);
    const unsigned grid = (unsigned)(lots < 1 ? 1 : lots);
    if (!grad_bytes) {
        if (p.M > 0) k_few_loss<EB, VEC><<<grid, kThreads, 0, st>>>(p);
        return cudaGetLastError();
    }
    if (p.M > 0) k_few_back<EB, VEC><<<grid, kThreads, 0, st>>>(p);
    const unsigned classes = (unsigned)((p.V + kR - 1) / kR);
    const dim3 g((unsigned)((p.K + 32 * Elem<EB>::V - 1) / (32 * Elem<EB>::V)), classes < 65535 ? classes : 65535, (unsigned)p.N);
    if (grad_bytes == 4) k_few_weights<EB, 4, VEC><<<g, kThreads, 0, st>>>(p);
    else k_few_weights<EB, 2, VEC><<<g, kThreads, 0, st>>>(p);
    return cudaGetLastError();
}

// ---------------------------------------------------------------- host
bool sizes_ok(int N, int64_t M, int64_t n_in, int64_t n_out, int elem_bytes, int grad_bytes) {
    return (elem_bytes == 2 || elem_bytes == 4) && (grad_bytes == 0 || grad_bytes == 4 || (grad_bytes == 2 && elem_bytes == 2)) && N >= 1 &&
           N <= COMBO_MAX_WORKERS && M >= 0 && M <= COMBO_LINEAR_MAX_ROWS && n_in >= 1 && n_out >= 1 && n_in <= COMBO_LINEAR_MAX_WIDTH &&
           n_out <= COMBO_LINEAR_MAX_WIDTH;
}

size_t scratch_needed(int N, int64_t M, int64_t n_in, int64_t n_out, int elem_bytes, int grad_bytes) {
    (void)N; (void)n_in; (void)elem_bytes;
    return 256 + (grad_bytes ? (size_t)M * n_out * 4 : 0);
}

combo_status cross_entropy(Loss p, int elem_bytes, int grad_bytes, int64_t n_in, int64_t n_out, void* scratch, size_t scratch_bytes, void* stream) {
    if (!sizes_ok(p.N, p.M, n_in, n_out, elem_bytes, grad_bytes)) return COMBO_ERR_INVALID_ARG;
    const bool back = grad_bytes != 0;
    if (!p.begin || !combo_host::aligned_to(p.begin, 8)) return COMBO_ERR_INVALID_ARG;
    if (!scratch || !combo_host::aligned_to(scratch, 256) || scratch_bytes < scratch_needed(p.N, p.M, n_in, n_out, elem_bytes, grad_bytes))
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
    p.d = static_cast<float*>(scratch);
    const auto vec_ok = [&](const void* a, int64_t pitch, int64_t stride) {
        return combo_host::aligned_to(a, 16) && pitch * elem_bytes % 16 == 0 && stride * elem_bytes % 16 == 0;
    };
    const bool vec = vec_ok(p.x, p.x_pitch, 0) && vec_ok(p.w, p.w_pitch, p.w_stride);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (elem_bytes == 4) e = vec ? launch_few<4, true>(p, grad_bytes, st) : launch_few<4, false>(p, grad_bytes, st);
    else e = vec ? launch_few<2, true>(p, grad_bytes, st) : launch_few<2, false>(p, grad_bytes, st);
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "cross entropy launch");
}

}  // namespace

extern "C" {

size_t combo_grouped_cross_entropy_scratch_bytes(int N, int64_t M, int64_t n_in, int64_t n_out, int elem_bytes, int grad_bytes) {
    return sizes_ok(N, M, n_in, n_out, elem_bytes, grad_bytes) ? scratch_needed(N, M, n_in, n_out, elem_bytes, grad_bytes) : 0;
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
