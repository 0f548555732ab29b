// Gradient norms of all workers over many tensors, and clipping.
//
//   norm_w = sqrt( sum over worker w's tensors of g^2 ),  c_w = min(1, max_norm / (norm_w + 1e-6)),  out = c_w * g
//
// A worker's gradient is a list of tensors; all lists, one after another, form one sequence of `total` elements
// (begin[t] = position of tensor t, first[w] = first tensor of worker w).  Every CTA takes one contiguous piece of the
// sequence, so that it meets few workers (one or two when there are fewer workers than CTAs) and one search at
// its start finds its place.  Inside a piece the warps take units of 4 KB in turn (smaller ones where there are too few of
// those for all warps); 4 KB are 8 vectors of 16 bytes per lane, all in flight at once, with ragged ends and unaligned tensors peeled element by element.
//
//   k_grad_norm    sums of squares: per (CTA, worker) one binary64 partial sum in scratch.  CTA b and worker w meet in
//                  slot b + w: along the sequence b and w never decrease and one of them grows from one meeting to
//                  the next, so no two meetings share a slot and `grid + N` slots are enough.
//   k_grad_scale   the same walk from the back (what k_grad_norm read last is still in L2), scaled and stored
//   k_grad_finish  norms alone, where nothing is to be scaled
//
// Bound by HBM: 2 reads and 1 write of the gradient, less what L2 (126 MB) still holds on the second read.
// Measured: 32 x 11.7 M floats 722 us (6.2 TB/s over the three passes; 456 us were one read and one write), 16 x 23.5 M
// bfloat16 in rows off 16-byte boundaries 390 us; 8 x 1 M floats 26 us, bound by the two launches' latencies.
// The partial sums are added in a fixed order, so results do not change from run to run.
#include "host_common.h"
#include "step_common.cuh"

namespace {

using combo_step::Elem;
using combo_step::warp_sum;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnitBytes = 4096;
constexpr int kVecs = kUnitBytes / 16 / 32;     // vectors per lane and unit
constexpr int kCtasPerSm = 3;                   // 256 x 3 against 512 x 2 (64 registers a thread, spilled): 722 us against 798
constexpr int kMaxGrid = 1024;                  // bound of the scratch size

struct Table {
    const unsigned char* const* src;
    unsigned char* const* dst;
    const int64_t* begin;     // [n_tensors + 1]
    const int32_t* first;     // [N + 1]
    int n_tensors, N, grid;
    int unit;                 // elements
    long long total;          // elements
    long long piece;          // elements of one CTA's piece, a multiple of the unit
    float max_norm;
    float* norm;
    float* coef;
    double* partial;          // [grid + N]
};

__device__ __forceinline__ long long owner_end(const Table& p, int w) {
    const int t = min(max(p.first[w], 0), p.n_tensors);
    return min(max((long long)p.begin[t], 0LL), p.total);
}

// The tensor that holds position `pos`, the last one that begins at or before it, and its worker, the last one whose
// first tensor is at or before that: the whole block counts, both tables' loads under way together.
__device__ __forceinline__ void locate(const Table& p, long long pos, int& t, int& w) {
    const int i = (int)threadIdx.x;
    const int f0 = i < p.N ? p.first[i] : 0x7fffffff;
    int c = 0;
    for (int base = 0; base < p.n_tensors; base += kThreads) {
        const int got = __syncthreads_count(base + i < p.n_tensors && (long long)p.begin[base + i] <= pos);
        c += got;
        if (got < kThreads) break;
    }
    t = max(c - 1, 0);
    c = __syncthreads_count(f0 <= t);
    for (int base = kThreads; base < p.N && c == base; base += kThreads)
        c += __syncthreads_count(base + i < p.N && p.first[base + i] <= t);
    w = max(c - 1, 0);
}

// One warp's place in the sequence: the tensor that holds position `pos`, found forwards or backwards.
struct Cursor {
    int t;
    long long lo, hi;         // positions of the tensor's first element and behind its last
    __device__ __forceinline__ void set(const Table& p, int tt) {
        t = tt;
        lo = p.begin[t];
        hi = p.begin[t + 1];
    }
    __device__ __forceinline__ void seek(const Table& p, long long pos, int lane) {
        if (pos >= lo && pos < hi) return;
        int tt = t;
        if (pos >= hi) {      // 32 tensors at a time: count those that begin at or before pos
            while (tt + 1 < p.n_tensors) {
                const int i = tt + 1 + lane;
                const unsigned m = __ballot_sync(0xffffffffu, i < p.n_tensors && (long long)p.begin[i] <= pos);
                tt += __popc(m);
                if (m != 0xffffffffu) break;
            }
        } else {              // the last one at or before t that begins at or before pos
            while (tt > 0) {
                const int i = tt - 1 - lane;
                const unsigned m = __ballot_sync(0xffffffffu, i >= 0 && (long long)p.begin[i] <= pos);
                if (m) { tt = tt - 1 - (__ffs(m) - 1); break; }
                tt = max(tt - 32, 0);
            }
        }
        set(p, tt);
    }
};

// Sum of squares of n values of one lane: binary32 over the run, then one addition in binary64.  A run whose
// squares leave the comfortable range of binary32 (or that is all zero, infinite or NaN) is taken in binary64.
template <int N_> __device__ __forceinline__ double run_squares(const float (&x)[N_]) {
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int i = 0; i < N_; i += 2) {
        s0 = fmaf(x[i], x[i], s0);
        s1 = fmaf(x[i + 1], x[i + 1], s1);
    }
    const float s = s0 + s1;
    if (s >= 1e-30f && s <= 1e38f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < N_; ++i) d = fma((double)x[i], (double)x[i], d);
    return d;
}

// Part of a unit that lies in one tensor, as vectors and ragged ends.
template <int EB> struct Span {
    const unsigned char* p;   // first element
    int n;                    // elements
    int head;                 // elements before the first 16-byte boundary
    int nv;                   // whole vectors
    __device__ __forceinline__ Span(const unsigned char* base, long long off, int count) {
        constexpr int V = Elem<EB>::V;
        p = base + off * EB;
        n = count;
        head = min((int)((16u - (unsigned)(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / EB, n);
        nv = (n - head) / V;
    }
};

template <int EB> __device__ __forceinline__ double span_squares(const Span<EB>& s, int lane) {
    constexpr int V = Elem<EB>::V;
    double acc = 0.0;
    const uint4* body = reinterpret_cast<const uint4*>(s.p + s.head * EB);
    uint4 v[kVecs];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
        const int i = j * 32 + lane;
        v[j] = i < s.nv ? __ldg(body + i) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < kVecs; j += 2) {
        if (j * 32 >= s.nv) break;
        float x[2 * V], a[V], b[V];
        Elem<EB>::unpack(v[j], a);
        Elem<EB>::unpack(v[j + 1], b);
#pragma unroll
        for (int i = 0; i < V; ++i) { x[i] = a[i]; x[V + i] = b[i]; }
        acc += run_squares(x);
    }
    const int tail = s.n - s.head - s.nv * V;
    if (s.head + tail > 0) {                     // at most 2 (V - 1) elements: one lane each
        float x[2] = {0.0f, 0.0f};
        if (lane < s.head) x[0] = Elem<EB>::get(s.p + lane * EB);
        if (lane < tail) x[1] = Elem<EB>::get(s.p + (s.head + s.nv * V + lane) * EB);
        if (lane < max(s.head, tail)) acc += run_squares(x);
    }
    return acc;
}

template <int EB>
__device__ __forceinline__ void span_scale(const Span<EB>& s, unsigned char* out, float c, int lane) {
    constexpr int V = Elem<EB>::V;
    const bool same_phase = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(s.p)) & 15u) == 0;
    if (same_phase) {
        const uint4* body = reinterpret_cast<const uint4*>(s.p + s.head * EB);
        uint4* dst = reinterpret_cast<uint4*>(out + s.head * EB);
        uint4 v[kVecs];
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = j * 32 + lane;
            if (i < s.nv) v[j] = __ldcs(body + i);
        }
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = j * 32 + lane;
            if (i < s.nv) {
                float x[V];
                Elem<EB>::unpack(v[j], x);
#pragma unroll
                for (int k = 0; k < V; ++k) x[k] *= c;
                __stcs(dst + i, Elem<EB>::pack(x));
            }
        }
        const int tail0 = s.head + s.nv * V, tail = s.n - tail0;
        if (lane < s.head) Elem<EB>::put(out + lane * EB, Elem<EB>::get(s.p + lane * EB) * c);
        if (lane < tail) Elem<EB>::put(out + (tail0 + lane) * EB, Elem<EB>::get(s.p + (tail0 + lane) * EB) * c);
    } else {                                     // source and destination differ in their 16-byte phase
        for (int i = lane; i < s.n; i += 256) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i + j * 32 < s.n) x[j] = Elem<EB>::get(s.p + (i + j * 32) * EB);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i + j * 32 < s.n) Elem<EB>::put(out + (i + j * 32) * EB, x[j] * c);
        }
    }
}

// A block's sum of one binary64 value per thread, in a fixed order, in every thread.
__device__ __forceinline__ double block_sum(double v, double* sh) {
    v = warp_sum(v);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) sh[warp] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) s += sh[i];
    __syncthreads();
    return s;
}

template <int EB> __global__ void __launch_bounds__(kThreads, kCtasPerSm) k_grad_norm(const Table p) {
    const int U = p.unit;
    __shared__ double sh[kWarps];
    combo_step::pdl_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long r0 = p.piece * blockIdx.x, r1 = min(r0 + p.piece, p.total);
    if (r0 >= r1) return;
    int w, t;
    locate(p, r0, t, w);
    Cursor cur;
    cur.set(p, t);
    long long lo = r0;
    while (lo < r1 && w < p.N) {
        const long long hi = min(owner_end(p, w + 1), r1);
        double acc = 0.0;
        for (long long u = lo + (long long)warp * U; u < hi; u += (long long)kWarps * U) {
            const long long ue = min(u + U, hi);
            long long at = u;
            while (at < ue) {
                cur.seek(p, at, lane);
                const long long e = min(ue, cur.hi);
                if (e <= at || at < cur.lo) break;   // a table that is not ascending
                acc += span_squares<EB>(Span<EB>(p.src[cur.t], at - cur.lo, (int)(e - at)), lane);
                at = e;
            }
        }
        if (hi > lo) {
            const double s = block_sum(acc, sh);
            if (threadIdx.x == 0) p.partial[blockIdx.x + w] = s;
            lo = hi;
        }
        ++w;
    }
}

// Norm and coefficient of worker w from the partial sums of the CTAs that met it; the whole block.
__device__ __forceinline__ float owner_coef(const Table& p, int w, long long lo, long long hi, double* sh, float* norm) {
    double s = 0.0;
    if (hi > lo) {
        const int b0 = (int)(lo / p.piece), b1 = (int)((hi - 1) / p.piece);
        for (int b = b0 + (int)threadIdx.x; b <= b1; b += kThreads) s += p.partial[b + w];
    }
    s = block_sum(s, sh);
    const float n = (float)sqrt(s);
    const float r = p.max_norm / (n + 1e-6f);
    *norm = n;
    return r >= 1.0f ? 1.0f : r;                 // a NaN norm gives a NaN coefficient
}

__device__ __forceinline__ void write_norm(const Table& p, int w, float norm, float coef) {
    if (threadIdx.x == 0) {
        if (p.norm) p.norm[w] = norm;
        if (p.coef) p.coef[w] = coef;
    }
}

__global__ void __launch_bounds__(kThreads) k_grad_finish(const Table p) {
    __shared__ double sh[kWarps];
    combo_step::pdl_wait();
    for (int w = blockIdx.x; w < p.N; w += gridDim.x) {
        float norm;
        const float c = owner_coef(p, w, owner_end(p, w), owner_end(p, w + 1), sh, &norm);
        write_norm(p, w, norm, c);
    }
}

template <int EB> __global__ void __launch_bounds__(kThreads, kCtasPerSm) k_grad_scale(const Table p) {
    const int U = p.unit;
    __shared__ double sh[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long r0 = min(p.piece * blockIdx.x, p.total), r1 = min(r0 + p.piece, p.total);
    int w, t;                                    // of the last element before r1
    locate(p, r1 - 1, t, w);
    Cursor cur;
    cur.set(p, t);
    combo_step::pdl_wait();
    if (blockIdx.x == 0) {                       // workers without an element
        for (int i = threadIdx.x; i < p.N; i += kThreads)
            if (owner_end(p, i) >= owner_end(p, i + 1)) {
                if (p.norm) p.norm[i] = 0.0f;
                if (p.coef) p.coef[i] = p.max_norm / 1e-6f >= 1.0f ? 1.0f : p.max_norm / 1e-6f;
            }
    }
    long long hi = r1;
    while (hi > r0 && w >= 0) {
        const long long w_lo = owner_end(p, w), w_hi = owner_end(p, w + 1);
        const long long lo = max(w_lo, r0);
        if (lo < hi) {
            float norm;
            const float c = owner_coef(p, w, w_lo, w_hi, sh, &norm);
            if (w_lo >= r0) write_norm(p, w, norm, c);
            const long long n_units = (hi - lo + U - 1) / U;
            for (long long k = n_units - 1 - warp; k >= 0; k -= kWarps) {
                const long long u = lo + k * U, ue = min(u + U, hi);
                long long at = u;
                while (at < ue) {
                    cur.seek(p, at, lane);
                    const long long e = min(ue, cur.hi);
                    if (e <= at || at < cur.lo) break;
                    const Span<EB> s(p.src[cur.t], at - cur.lo, (int)(e - at));
                    unsigned char* out = p.dst[cur.t] + (at - cur.lo) * EB;
                    // gradients that stay as they are where they are need no pass
                    if (c != 1.0f || out != s.p) span_scale<EB>(s, out, c, lane);
                    at = e;
                }
            }
            hi = lo;
        }
        --w;
    }
}

__global__ void k_check_tensors(const Table p, int eb, int32_t* flag) {
    const int n = max(p.n_tensors, p.N);
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i <= n; i += gridDim.x * blockDim.x) {
        if (i <= p.n_tensors) {
            const long long b = p.begin[i];
            bool bad = b < 0 || b > p.total || (i == 0 && b != 0) || (i == p.n_tensors && b != p.total);
            if (i < p.n_tensors) {
                const long long e = p.begin[i + 1];
                const uintptr_t a = reinterpret_cast<uintptr_t>(p.src[i]);
                bad |= e < b || (e > b && (a == 0 || a % eb != 0));
            }
            if (bad) atomicMax(flag, 1 + i);
        }
        if (i <= p.N) {
            const int f = p.first[i];
            bool bad = f < 0 || f > p.n_tensors || (i == 0 && f != 0) || (i == p.N && f != p.n_tensors);
            if (i < p.N) bad |= p.first[i + 1] < f;
            if (bad) atomicMax(flag, 1 + p.n_tensors + i);
        }
    }
}

combo_status check_table(const void* const* tensors, const int64_t* begin, const int32_t* first, int n_tensors, int N,
                         int64_t total, int elem_bytes) {
    if (elem_bytes != 4 && elem_bytes != 2) return COMBO_ERR_INVALID_ARG;
    if (N < 1 || N > COMBO_MAX_WORKERS || n_tensors < 0 || total < 0 || total > (1LL << 46)) return COMBO_ERR_INVALID_ARG;
    if (!begin || !first || (n_tensors > 0 && !tensors) || (total > 0 && n_tensors == 0)) return COMBO_ERR_INVALID_ARG;
    if (!combo_host::aligned_to(tensors, 8) || !combo_host::aligned_to(begin, 8) || !combo_host::aligned_to(first, 4))
        return COMBO_ERR_INVALID_ARG;
    return COMBO_OK;
}

combo_status norm_impl(const void* const* tensors, void* const* out, const int64_t* begin, const int32_t* first,
                       int n_tensors, int N, int64_t total, int elem_bytes, float max_norm, float* norm_out,
                       float* coef_out, void* scratch, size_t scratch_bytes, void* stream, bool scale) {
    combo_status rc = check_table(tensors, begin, first, n_tensors, N, total, elem_bytes);
    if (rc != COMBO_OK) return rc;
    if (!(max_norm >= 0.0f)) return COMBO_ERR_INVALID_ARG;
    if (scale && n_tensors > 0 && (!out || !combo_host::aligned_to(out, 8))) return COMBO_ERR_INVALID_ARG;
    if (!scale && !norm_out && !coef_out) return COMBO_ERR_INVALID_ARG;
    if (!combo_host::aligned_to(norm_out, 4) || !combo_host::aligned_to(coef_out, 4)) return COMBO_ERR_INVALID_ARG;
    if (!scratch || !combo_host::aligned_to(scratch, 8) || scratch_bytes < combo_grad_scratch_bytes(N))
        return COMBO_ERR_INVALID_ARG;
    int sms = 0, smem = 0;
    if ((rc = combo_host::device(&sms, &smem)) != COMBO_OK) return rc;
    Table p = {};
    p.src = reinterpret_cast<const unsigned char* const*>(tensors);
    p.dst = reinterpret_cast<unsigned char* const*>(out);
    p.begin = begin;
    p.first = first;
    p.n_tensors = n_tensors;
    p.N = N;
    p.total = total;
    p.max_norm = max_norm;
    p.norm = norm_out;
    p.coef = coef_out;
    p.partial = static_cast<double*>(scratch);
    // one unit for each warp, the larger the unit the better, until every SM holds its CTAs; then longer pieces.
    // Units of 512 bytes keep a warp to few tensors where there are many small ones.
    const long long most = (long long)sms * kCtasPerSm < kMaxGrid ? (long long)sms * kCtasPerSm : kMaxGrid;
    long long unit = 512 / elem_bytes;
    while (unit * elem_bytes < kUnitBytes && total > unit * kWarps * most) unit *= 2;
    p.unit = (int)unit;
    const long long units = (total + unit - 1) / unit;
    long long grid = (units + kWarps - 1) / kWarps;
    if (grid > most) grid = most;
    if (grid < 1) grid = 1;
    p.piece = (units + grid - 1) / grid * unit;
    if (p.piece < unit) p.piece = unit;
    p.grid = (int)grid;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (total > 0) {
        if (elem_bytes == 4) k_grad_norm<4><<<p.grid, kThreads, 0, st>>>(p);
        else k_grad_norm<2><<<p.grid, kThreads, 0, st>>>(p);
        if ((e = cudaGetLastError()) != cudaSuccess) return combo_host::fail(e, "gradient norm launch");
    }
    if (scale && total > 0) {
        e = elem_bytes == 4 ? combo_host::launch_after(k_grad_scale<4>, dim3(p.grid), dim3(kThreads), 0, st, p)
                            : combo_host::launch_after(k_grad_scale<2>, dim3(p.grid), dim3(kThreads), 0, st, p);
    } else {
        e = combo_host::launch_after(k_grad_finish, dim3(N < sms * 2 ? N : sms * 2), dim3(kThreads), 0, st, p);
    }
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "gradient clipping launch");
}

}  // namespace

extern "C" {

size_t combo_grad_scratch_bytes(int N) {
    return N < 1 || N > COMBO_MAX_WORKERS ? 0 : (size_t)(kMaxGrid + N) * sizeof(double);
}

combo_status combo_grad_norm(const void* const* d_tensors, const int64_t* d_begin, const int32_t* d_first, int n_tensors,
                             int N, int64_t total, int elem_bytes, float max_norm, float* norm_out, float* coef_out,
                             void* scratch, size_t scratch_bytes, void* stream) {
    return norm_impl(d_tensors, nullptr, d_begin, d_first, n_tensors, N, total, elem_bytes, max_norm, norm_out, coef_out,
                     scratch, scratch_bytes, stream, false);
}

combo_status combo_grad_clip(const void* const* d_tensors, void* const* d_out, const int64_t* d_begin,
                             const int32_t* d_first, int n_tensors, int N, int64_t total, int elem_bytes, float max_norm,
                             float* norm_out, float* coef_out, void* scratch, size_t scratch_bytes, void* stream) {
    return norm_impl(d_tensors, d_out, d_begin, d_first, n_tensors, N, total, elem_bytes, max_norm, norm_out, coef_out,
                     scratch, scratch_bytes, stream, true);
}

combo_status combo_check_tensors(const void* const* d_tensors, const int64_t* d_begin, const int32_t* d_first,
                                 int n_tensors, int N, int64_t total, int elem_bytes, void* stream, int32_t* dev_flag) {
    combo_status rc = check_table(d_tensors, d_begin, d_first, n_tensors, N, total, elem_bytes);
    if (rc != COMBO_OK) return rc;
    if (!dev_flag) return COMBO_ERR_INVALID_ARG;
    int sms = 0, smem = 0;
    if ((rc = combo_host::device(&sms, &smem)) != COMBO_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaMemsetAsync(dev_flag, 0, sizeof(int32_t), st);
    if (e != cudaSuccess) return combo_host::fail(e, "cudaMemsetAsync");
    Table p = {};
    p.src = reinterpret_cast<const unsigned char* const*>(d_tensors);
    p.begin = d_begin;
    p.first = d_first;
    p.n_tensors = n_tensors;
    p.N = N;
    p.total = total;
    const int n = n_tensors > N ? n_tensors : N;
    k_check_tensors<<<n / 256 + 1 < 1024 ? n / 256 + 1 : 1024, 256, 0, st>>>(p, elem_bytes, dev_flag);
    e = cudaGetLastError();
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "tensor table check launch");
}

}  // extern "C"
