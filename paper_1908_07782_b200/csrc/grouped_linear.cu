// Products grouped by worker: every worker's rows (samples) times its own weights.
//
//   forward          Y[m][n]   = sum_k X[m][k]  W_w[n][k]      m in worker w's rows
//   gradient, rows   dX[m][k]  = sum_n dY[m][n] W_w[n][k]
//   gradient, weights dW_w[n][k] = sum_m dY[m][n] X[m][k]      over worker w's rows
//
// all of the form C(i, j) = sum_r A(i, r) B(j, r), with either index of an operand contiguous in memory:
//
//                     i            j           r
//   forward           m (ragged)   n           k        both operands contiguous along r
//   gradient, rows    m (ragged)   k           n        A along r, B along j
//   gradient, weights n            k           m (ragged)   both along i / j
#include "host_common.h"
#include "step_common.cuh"

namespace {

using combo_step::Elem;
using combo_step::f32x2;
using combo_step::fma2;
using combo_step::hi_of;
using combo_step::lo_of;
using combo_step::pair;

enum Mode { kForward = 0, kGradInput = 1, kGradWeight = 2 };

struct Product {
    const unsigned char* a;       // rows' operand: X, dY, dY
    const unsigned char* b;       // W, W, X
    unsigned char* c;             // Y, dX, dW
    const int64_t* begin;         // [N + 1]
    long long a_pitch, b_pitch, c_pitch;      // elements between rows
    long long stride;             // elements between workers, of W or dW
    long long M;                  // rows in all
    int N, I, J, R;               // extents of i, j, r; the ragged one is M
    int a_vec, b_vec, c_vec;      // whether 16-byte vectors can be read (written) along the contiguous index
};

__device__ __forceinline__ void rows_of(const Product& p, int w, long long& r0, long long& r1) {
    r0 = min(max((long long)p.begin[w], 0LL), p.M);
    r1 = min(max((long long)p.begin[w + 1], r0), p.M);
}

// ---------------------------------------------------------------- binary32 multiply-adds
// 128 x 128 outputs for a block of 256 threads, 8 x 8 each, 16 values of r at a time through two shared-memory stages;
// the next stage's loads are in registers while this one's products are formed.  Takes every type, pitch and alignment.
constexpr int kFT = 128, kFK = 16, kFThreads = 256;
constexpr int kFPad = 4;

// Eight neighbouring elements of one line; those at or beyond `left` are zero.
template <int EB> __device__ __forceinline__ void load8(const unsigned char* q, int left, bool vec, float (&v)[8]) {
    if (vec && left >= 8) {
        if constexpr (EB == 4) {
            const uint4 a = *reinterpret_cast<const uint4*>(q), b = *reinterpret_cast<const uint4*>(q + 16);
            float x[4], y[4];
            Elem<4>::unpack(a, x);
            Elem<4>::unpack(b, y);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = x[i]; v[4 + i] = y[i]; }
        } else {
            Elem<2>::unpack(*reinterpret_cast<const uint4*>(q), v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? Elem<EB>::get(q + i * EB) : 0.0f;
    }
}

// A thread's share of a 128 x 16 operand tile.  ALONG_R: r is contiguous; else the tile index is.
template <int EB, bool ALONG_R>
__device__ __forceinline__ void load_part(const unsigned char* base, long long pitch, long long i0, long long i_end, long long r0,
                                          long long r_end, bool vec, float (&v)[8]) {
    const int t = threadIdx.x;
    const long long i = i0 + (ALONG_R ? t >> 1 : (t & 15) * 8), r = r0 + (ALONG_R ? (t & 1) * 8 : t >> 4);
    const long long left = ALONG_R ? (i < i_end ? r_end - r : 0) : (r < r_end ? i_end - i : 0);
    const int n = (int)min(max(left, 0LL), 8LL);
    load8<EB>(base + (ALONG_R ? i * pitch + r : r * pitch + i) * EB, n, vec, v);
}

template <bool ALONG_R> __device__ __forceinline__ void store_part(float (*s)[kFT + kFPad], const float (&v)[8]) {
    const int t = threadIdx.x;
    if (ALONG_R) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s[(t & 1) * 8 + k][t >> 1] = v[k];
    } else {
        float4* d = reinterpret_cast<float4*>(&s[t >> 4][(t & 15) * 8]);
        d[0] = make_float4(v[0], v[1], v[2], v[3]);
        d[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

template <int EB, int OB, int MODE> __global__ void __launch_bounds__(kFThreads, 2) k_fma(const Product p) {
    constexpr bool A_R = MODE != kGradWeight, B_R = MODE == kForward;
    __shared__ __align__(16) float sa[2][kFK][kFT + kFPad];
    __shared__ __align__(16) float sb[2][kFK][kFT + kFPad];
    const int t = threadIdx.x;
    int w = 0;
    long long i0, i1, r0 = 0, r1 = p.R;
    const long long j0 = (long long)blockIdx.x * kFT;
    if (MODE == kGradWeight) {
        w = blockIdx.z;
        i0 = (long long)blockIdx.y * kFT;
        i1 = p.I;
        rows_of(p, w, r0, r1);
    } else {
        // the tile of rows that block y of the grid stands for: counted through the workers, 256 at a time
        long long before = 0;
        bool found = false;
        for (int w0 = 0; w0 < p.N && !found; w0 += kFThreads) {
            __shared__ int tiles[kFThreads];
            long long a = 0, b = 0;
            if (w0 + t < p.N) rows_of(p, w0 + t, a, b);
            tiles[t] = (int)((b - a + kFT - 1) / kFT);
            __syncthreads();
            for (int k = 0; k < kFThreads && w0 + k < p.N; ++k) {
                if (blockIdx.y < before + tiles[k]) { w = w0 + k; found = true; break; }
                before += tiles[k];
            }
            __syncthreads();
        }
        if (!found) return;
        rows_of(p, w, i0, i1);
        i0 += ((long long)blockIdx.y - before) * kFT;
    }
    const unsigned char* a = p.a;
    const unsigned char* b = MODE == kGradWeight ? p.b : p.b + w * p.stride * EB;
    f32x2 acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0;
    const int ti = t >> 4, tj = t & 15;
    float va[8], vb[8];
    int s = 0;
    if (r0 < r1) {
        load_part<EB, A_R>(a, p.a_pitch, i0, i1, r0, r1, p.a_vec, va);
        load_part<EB, B_R>(b, p.b_pitch, j0, p.J, r0, r1, p.b_vec, vb);
        store_part<A_R>(sa[0], va);
        store_part<B_R>(sb[0], vb);
    }
    __syncthreads();
    for (long long r = r0; r < r1; r += kFK) {
        const bool more = r + kFK < r1;
        if (more) {
            load_part<EB, A_R>(a, p.a_pitch, i0, i1, r + kFK, r1, p.a_vec, va);
            load_part<EB, B_R>(b, p.b_pitch, j0, p.J, r + kFK, r1, p.b_vec, vb);
        }
#pragma unroll
        for (int k = 0; k < kFK; ++k) {
            const float4 x0 = *reinterpret_cast<const float4*>(&sa[s][k][ti * 4]);
            const float4 x1 = *reinterpret_cast<const float4*>(&sa[s][k][64 + ti * 4]);
            const ulonglong2 y0 = *reinterpret_cast<const ulonglong2*>(&sb[s][k][tj * 4]);
            const ulonglong2 y1 = *reinterpret_cast<const ulonglong2*>(&sb[s][k][64 + tj * 4]);
            const float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
            const f32x2 y[4] = {y0.x, y0.y, y1.x, y1.y};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x2 xx = pair(x[i], x[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fma2(xx, y[j], acc[i][j]);
            }
        }
        if (more) {
            store_part<A_R>(sa[s ^ 1], va);
            store_part<B_R>(sb[s ^ 1], vb);
        }
        __syncthreads();
        s ^= 1;
    }
    unsigned char* c = MODE == kGradWeight ? p.c + w * p.stride * OB : p.c;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const long long row = i0 + (i >> 2) * 64 + ti * 4 + (i & 3);
        if (row >= i1) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long long col = j0 + h * 64 + tj * 4;
            unsigned char* q = c + (row * p.c_pitch + col) * OB;
            const float v[4] = {lo_of(acc[i][2 * h]), hi_of(acc[i][2 * h]), lo_of(acc[i][2 * h + 1]), hi_of(acc[i][2 * h + 1])};
            if (p.c_vec && col + 4 <= p.J) {
                if constexpr (OB == 4) *reinterpret_cast<float4*>(q) = make_float4(v[0], v[1], v[2], v[3]);
                else *reinterpret_cast<uint2*>(q) = make_uint2(combo_step::pack_bf16(v[0], v[1]), combo_step::pack_bf16(v[2], v[3]));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (col + k < p.J) Elem<OB>::put(q + k * OB, v[k]);
            }
        }
    }
}

// ---------------------------------------------------------------- host
template <int EB, int OB> cudaError_t launch_fma(const Product& p, int mode, cudaStream_t st) {
    const unsigned cols = (unsigned)((p.J + kFT - 1) / kFT);
    if (mode == kGradWeight) {
        const dim3 grid(cols, (unsigned)((p.I + kFT - 1) / kFT), (unsigned)p.N);
        k_fma<EB, OB, kGradWeight><<<grid, kFThreads, 0, st>>>(p);
    } else {
        // every worker adds less than one tile to those its rows fill
        const long long tiles = p.M / kFT + (p.N < p.M ? p.N : p.M);
        const dim3 grid(cols, (unsigned)(tiles < 1 ? 1 : tiles));
        if (mode == kForward) k_fma<EB, OB, kForward><<<grid, kFThreads, 0, st>>>(p);
        else k_fma<EB, OB, kGradInput><<<grid, kFThreads, 0, st>>>(p);
    }
    return cudaGetLastError();
}

bool vec_ok(const void* p, int64_t pitch, int64_t stride, int eb) {
    return combo_host::aligned_to(p, 16) && pitch * eb % 16 == 0 && stride * eb % 16 == 0;
}

// rows, each `width` elements, `pitch` apart
size_t extent(int64_t rows, int64_t width, int64_t pitch, int eb) { return rows < 1 ? 0 : (size_t)((rows - 1) * pitch + width) * eb; }

// Checks and launches one of the three.
combo_status product(int mode, const void* rows1, int64_t pitch1, const void* rows2, int64_t pitch2, const void* weights,
                     int64_t w_pitch, int64_t w_stride, int elem_bytes, int out_bytes, const int64_t* begin, int N, int64_t M,
                     int64_t n_in, int64_t n_out, void* stream) {
    if (!((elem_bytes == 4 && out_bytes == 4) || (elem_bytes == 2 && (out_bytes == 2 || out_bytes == 4)))) return COMBO_ERR_INVALID_ARG;
    if (N < 1 || N > COMBO_MAX_WORKERS || M < 0 || M > COMBO_LINEAR_MAX_ROWS || n_in < 1 || n_out < 1 ||
        n_in > COMBO_LINEAR_MAX_WIDTH || n_out > COMBO_LINEAR_MAX_WIDTH)
        return COMBO_ERR_INVALID_ARG;
    if (!begin || !combo_host::aligned_to(begin, 8)) return COMBO_ERR_INVALID_ARG;
    // rows1: X (forward), dY; rows2: Y, dX (outputs) or X
    const int64_t width1 = mode == kForward ? n_in : n_out, width2 = mode == kForward ? n_out : n_in;
    const int eb2 = mode == kGradWeight ? elem_bytes : out_bytes, ebw = mode == kGradWeight ? out_bytes : elem_bytes;
    if (M > 0) {
        if (!rows1 || !rows2 || pitch1 < width1 || pitch2 < width2) return COMBO_ERR_INVALID_ARG;
        if (pitch1 > (1LL << 40) / M || pitch2 > (1LL << 40) / M) return COMBO_ERR_INVALID_ARG;
        if (!combo_host::aligned_to(rows1, elem_bytes) || !combo_host::aligned_to(rows2, eb2)) return COMBO_ERR_INVALID_ARG;
    }
    if (!weights || !combo_host::aligned_to(weights, ebw) || w_pitch < n_in || w_pitch > (1LL << 40) / n_out)
        return COMBO_ERR_INVALID_ARG;
    if (N > 1 && (w_stride < (n_out - 1) * w_pitch + n_in || w_stride > (1LL << 44) / N)) return COMBO_ERR_INVALID_ARG;
    if (N == 1) w_stride = 0;
    const size_t n1 = extent(M, width1, pitch1, elem_bytes), n2 = extent(M, width2, pitch2, eb2);
    const size_t nw = ((size_t)(N - 1) * w_stride + (n_out - 1) * w_pitch + n_in) * ebw;
    const void* out = mode == kGradWeight ? weights : rows2;
    const size_t nout = mode == kGradWeight ? nw : n2;
    if (combo_host::overlap(out, nout, rows1, n1) ||
        combo_host::overlap(out, nout, mode == kGradWeight ? rows2 : weights, mode == kGradWeight ? n2 : nw))
        return COMBO_ERR_ALIAS;
    int sms = 0, smem = 0;
    combo_status rc = combo_host::device(&sms, &smem);
    if (rc != COMBO_OK) return rc;
    if (mode != kGradWeight && M == 0) return COMBO_OK;

    Product p = {};
    p.a = static_cast<const unsigned char*>(rows1);
    p.a_pitch = pitch1;
    p.a_vec = vec_ok(rows1, pitch1, 0, elem_bytes);
    p.begin = begin;
    p.stride = w_stride;
    p.M = M;
    p.N = N;
    if (mode == kGradWeight) {
        p.b = static_cast<const unsigned char*>(rows2);
        p.b_pitch = pitch2;
        p.c = static_cast<unsigned char*>(const_cast<void*>(weights));
        p.c_pitch = w_pitch;
        p.b_vec = vec_ok(rows2, pitch2, 0, elem_bytes);
        p.c_vec = vec_ok(weights, w_pitch, w_stride, out_bytes);
        p.I = (int)n_out;
        p.J = (int)n_in;
    } else {
        p.b = static_cast<const unsigned char*>(weights);
        p.b_pitch = w_pitch;
        p.c = static_cast<unsigned char*>(const_cast<void*>(rows2));
        p.c_pitch = pitch2;
        p.b_vec = vec_ok(weights, w_pitch, w_stride, elem_bytes);
        p.c_vec = vec_ok(rows2, pitch2, 0, out_bytes);
        p.J = (int)width2;
        p.R = (int)width1;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (elem_bytes == 4) e = launch_fma<4, 4>(p, mode, st);
    else if (out_bytes == 2) e = launch_fma<2, 2>(p, mode, st);
    else e = launch_fma<2, 4>(p, mode, st);
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "grouped product launch");
}

}  // namespace

extern "C" {

combo_status combo_grouped_linear(const void* x, int64_t x_pitch, const void* w, int64_t w_pitch, int64_t w_stride, void* y,
                                  int64_t y_pitch, int elem_bytes, int out_bytes, const int64_t* d_begin, int N, int64_t M,
                                  int64_t n_in, int64_t n_out, void* stream) {
    return product(kForward, x, x_pitch, y, y_pitch, w, w_pitch, w_stride, elem_bytes, out_bytes, d_begin, N, M, n_in, n_out, stream);
}

combo_status combo_grouped_linear_grad_input(const void* dy, int64_t dy_pitch, const void* w, int64_t w_pitch,
                                             int64_t w_stride, void* dx, int64_t dx_pitch, int elem_bytes, int out_bytes,
                                             const int64_t* d_begin, int N, int64_t M, int64_t n_in, int64_t n_out,
                                             void* stream) {
    return product(kGradInput, dy, dy_pitch, dx, dx_pitch, w, w_pitch, w_stride, elem_bytes, out_bytes, d_begin, N, M, n_in, n_out,
                   stream);
}

combo_status combo_grouped_linear_grad_weight(const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch, void* dw,
                                              int64_t dw_pitch, int64_t dw_stride, int elem_bytes, int out_bytes,
                                              const int64_t* d_begin, int N, int64_t M, int64_t n_in, int64_t n_out,
                                              void* stream) {
    return product(kGradWeight, dy, dy_pitch, x, x_pitch, dw, dw_pitch, dw_stride, elem_bytes, out_bytes, d_begin, N, M, n_in, n_out,
                   stream);
}

}  // extern "C"
