// Dropout whose mask is a function of counters and is never stored.
//
//   y = residual + keep * x * scale,   keep = (bits of the element >= T),   T = p in 1/65536,   scale = 65536 / (65536 - T)
//
// The bits come from the generator that draws the peers (splitmix64, Steele, Lea, Flood 2014), each step starting from the output
// before xor the next word: seed, round | worker, site, place; one draw of 64 bits serves four neighbours of a row.  A place counts
// within the worker's own rows, so a worker's mask does not depend on the other workers or on which GPU holds it.
//
// Bound by HBM: two passes over the data (three with a residual).  A vector of 16 bytes costs two draws of about 30 instructions
// for bfloat16, one for float, and as many again for the elements: half of what can be issued while its bytes pass.
#include "host_common.h"
#include "step_common.cuh"

namespace {

using combo_step::Elem;

struct Dropout {
    const unsigned char *x, *residual;
    unsigned char* y;
    long long x_pitch, r_pitch, y_pitch;         // elements
    const int64_t* begin;                        // [N + 1]; null: one worker with all rows
    long long M, n;
    uint64_t first;                              // the generator's state behind the seed
    uint32_t round, site, worker0, threshold;    // threshold << 16 of the bits; none_left: nothing is kept
    float scale;
    int N, none_left, lanes, pieces;             // lanes for a row, pieces of a row (a warp's units are 32 / lanes rows by one piece)
};

__host__ __device__ __forceinline__ uint64_t splitmix_step(uint64_t z) {
    z += 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// The worker that row m belongs to, or -1.
__device__ __forceinline__ int owner(const int64_t* begin, int N, long long m) {
    if (!begin) return 0;
    int lo = 0, hi = N;                          // the last w with begin[w] <= m
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (__ldg(reinterpret_cast<const long long*>(begin) + mid) <= m) lo = mid;
        else hi = mid - 1;
    }
    return lo < N && __ldg(reinterpret_cast<const long long*>(begin) + lo) <= m ? lo : -1;
}

constexpr int kThreads = 256, kUnroll = 4;

// EB bytes an element.  VEC: a lane's lot is 16 aligned bytes; else four elements, one at a time.
template <int EB, bool VEC, bool RES> __global__ void __launch_bounds__(kThreads) k_dropout(const Dropout p) {
    constexpr int V = VEC ? 16 / EB : 4, H = V / 4;
    combo_step::pdl_release();
    const int lane = threadIdx.x & 31;
    const long long lots = (p.n + 3) / 4, width = (p.n + V - 1) / V;       // draws and lots of a row
    const int per_warp = 32 / p.lanes;
    const long long units = (p.M + per_warp - 1) / per_warp * p.pieces;
    combo_step::pdl_wait();
    for (long long u = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); u < units; u += (long long)gridDim.x * (kThreads / 32)) {
        const long long rows = p.pieces == 1 ? u : u / p.pieces;
        const long long m = rows * per_warp + lane / p.lanes, v0 = (u - rows * p.pieces) * (kUnroll * 32) + lane % p.lanes;
        if (m >= p.M) continue;
        const unsigned char* x = p.x + m * p.x_pitch * EB;
        const unsigned char* r = RES ? p.residual + m * p.r_pitch * EB : nullptr;
        unsigned char* y = p.y + m * p.y_pitch * EB;
        const int w = owner(p.begin, p.N, m);
        if (w < 0) continue;
        const uint64_t key = splitmix_step(splitmix_step(p.first ^ ((uint64_t)p.round << 32 | (uint32_t)(p.worker0 + w))) ^
                                           (0x8000000000000000ull | p.site));
        const uint64_t place = (uint64_t)(m - (p.begin ? __ldg(reinterpret_cast<const long long*>(p.begin) + w) : 0)) * lots;
        uint4 a[kUnroll], b[kUnroll];
        if (VEC) {
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const long long v = v0 + k * p.lanes;
                if ((v + 1) * V <= p.n) {
                    a[k] = *reinterpret_cast<const uint4*>(x + v * 16);
                    if (RES) b[k] = *reinterpret_cast<const uint4*>(r + v * 16);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const long long v = v0 + k * p.lanes;
            if (v >= width) break;
            const bool whole = VEC && (v + 1) * V <= p.n;
            const int some = (int)min(p.n - v * V, (long long)V);
            float f[V], g[V];
            if (whole) {
                if constexpr (VEC) {
                    Elem<EB>::unpack(a[k], f);
                    if (RES) Elem<EB>::unpack(b[k], g);
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    f[e] = e < some ? Elem<EB>::get(x + (v * V + e) * EB) : 0.0f;
                    if (RES) g[e] = e < some ? Elem<EB>::get(r + (v * V + e) * EB) : 0.0f;
                }
            }
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const uint64_t z = splitmix_step(key ^ (place + v * H + h));
                const uint32_t half[2] = {(uint32_t)z, (uint32_t)(z >> 32)};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t bits = e & 1 ? half[e >> 1] : half[e >> 1] << 16;      // the element's 16 bits in front
                    const float t = bits >= p.threshold && !p.none_left ? f[h * 4 + e] * p.scale : 0.0f;
                    f[h * 4 + e] = RES ? t + g[h * 4 + e] : t;
                }
            }
            if (whole) {
                if constexpr (VEC) *reinterpret_cast<uint4*>(y + v * 16) = Elem<EB>::pack(f);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e < some) Elem<EB>::put(y + (v * V + e) * EB, f[e]);
            }
        }
    }
}

template <int EB> cudaError_t launch(Dropout p, int sms, bool vec, cudaStream_t st) {
    const int V = vec ? 16 / EB : 4;
    const long long width = (p.n + V - 1) / V;
    // Lanes to a row: the fewest that take it in one piece.
    p.lanes = 1;
    while (p.lanes < 32 && p.lanes * kUnroll < width) p.lanes *= 2;
    p.pieces = (int)((width + p.lanes * kUnroll - 1) / (p.lanes * kUnroll));
    const long long per_warp = 32 / p.lanes, units = (p.M + per_warp - 1) / per_warp * p.pieces;
    long long grid = (units + kThreads / 32 - 1) / (kThreads / 32);
    if (grid > (1 << 30)) grid = 1 << 30;
    (void)sms;
    const dim3 g((unsigned)grid), b(kThreads);
    if (p.residual) return vec ? combo_host::launch_after(k_dropout<EB, true, true>, g, b, 0, st, p) : combo_host::launch_after(k_dropout<EB, false, true>, g, b, 0, st, p);
    return vec ? combo_host::launch_after(k_dropout<EB, true, false>, g, b, 0, st, p) : combo_host::launch_after(k_dropout<EB, false, false>, g, b, 0, st, p);
}

}  // namespace

extern "C" combo_status combo_dropout(const void* x, int64_t x_pitch, const void* residual, int64_t residual_pitch, void* y, int64_t y_pitch,
                                      int elem_bytes, const int64_t* d_begin, int N, int64_t M, int64_t n, float p, uint64_t seed,
                                      uint32_t round, uint32_t site, int first_worker, void* stream) {
    if ((elem_bytes != 4 && elem_bytes != 2) || N < 1 || N > COMBO_MAX_WORKERS || M < 0 || n < 1 || !(p >= 0.0f && p <= 1.0f)) return COMBO_ERR_INVALID_ARG;
    if (first_worker < 0 || first_worker > COMBO_MAX_WORKERS - N) return COMBO_ERR_INVALID_ARG;
    if (n > (1LL << 32) || M > (1LL << 40) / n) return COMBO_ERR_INVALID_ARG;
    if ((!d_begin && N != 1) || !combo_host::aligned_to(d_begin, 8)) return COMBO_ERR_INVALID_ARG;
    if (M > 0) {
        if (!x || !y || x_pitch < n || y_pitch < n || (residual && residual_pitch < n)) return COMBO_ERR_INVALID_ARG;
        if (x_pitch > (1LL << 44) / M || y_pitch > (1LL << 44) / M || (residual && residual_pitch > (1LL << 44) / M)) return COMBO_ERR_INVALID_ARG;
        const size_t eb = (size_t)elem_bytes;
        if (!combo_host::aligned_to(x, eb) || !combo_host::aligned_to(y, eb) || !combo_host::aligned_to(residual, eb)) return COMBO_ERR_INVALID_ARG;
        const combo_host::Rows rx = {x, M, (size_t)n * eb, (size_t)x_pitch * eb}, ry = {y, M, (size_t)n * eb, (size_t)y_pitch * eb};
        const combo_host::Rows rr = {residual, M, (size_t)n * eb, (size_t)residual_pitch * eb};
        if (!(x == y && (x_pitch == y_pitch || M == 1)) && combo_host::overlap(rx, ry)) return COMBO_ERR_ALIAS;
        if (residual && !(residual == y && (residual_pitch == y_pitch || M == 1)) && combo_host::overlap(rr, ry)) return COMBO_ERR_ALIAS;
    }
    int sms = 0, smem = 0;
    const combo_status rc = combo_host::device(&sms, &smem);
    if (rc != COMBO_OK) return rc;
    if (M == 0) return COMBO_OK;
    const uint32_t T = (uint32_t)(p * 65536.0 + 0.5);
    Dropout q = {};
    q.x = static_cast<const unsigned char*>(x);
    q.residual = static_cast<const unsigned char*>(residual);
    q.y = static_cast<unsigned char*>(y);
    q.x_pitch = x_pitch;
    q.r_pitch = residual_pitch;
    q.y_pitch = y_pitch;
    q.begin = d_begin;
    q.M = M;
    q.n = n;
    q.first = splitmix_step(seed);
    q.round = round;
    q.site = site;
    q.worker0 = (uint32_t)first_worker;
    q.threshold = T << 16;
    q.none_left = T == 65536;
    q.scale = q.none_left ? 0.0f : (float)(65536.0 / (65536 - T));
    q.N = N;
    const auto fits = [&](const void* a, int64_t pitch) { return combo_host::aligned_to(a, 16) && (M == 1 || pitch * elem_bytes % 16 == 0); };
    const bool vec = fits(x, x_pitch) && fits(y, y_pitch) && (!residual || fits(residual, residual_pitch));
    const cudaError_t e = elem_bytes == 4 ? launch<4>(q, sms, vec, static_cast<cudaStream_t>(stream)) : launch<2>(q, sms, vec, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "dropout launch");
}
