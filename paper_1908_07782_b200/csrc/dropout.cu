// Dropout whose mask is a function of counters and is never stored.
//
//   y = residual + keep * x * scale,   keep = (bits of the element >= T),   T = p in 1/65536,   scale = 65536 / (65536 - T)
//
// The bits come from the generator that draws the peers (splitmix64, Steele, Lea, Flood 2014), each step starting from the output
// before xor the next word: seed, round | worker, site, place; one draw of 64 bits serves four neighbours of a row.  A place counts
// within the worker's own rows, so a worker's mask does not depend on the other workers or on which GPU holds it.
//
// Bound by HBM: two passes over the data (three with a residual).  A draw takes some 25 instructions and an element five, which is
// most of what can be issued while its bytes pass; so a warp takes several rows for one search of their worker and one key, and
// places within a row are counted in 32 bits.
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
    int N, none_left, lanes, rounds;             // lanes for a row; rounds of loads that they need for it
    int lots, width;                             // draws of a row; 16 bytes (or four elements) of it
    long long share;                             // rounds of a warp
};

__host__ __device__ __forceinline__ uint64_t splitmix_step(uint64_t z) {
    z += 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// Rows of one worker: first and end; the key of its draws.  A row of no worker is in a range without a key.
struct Owner {
    long long first, end;
    uint64_t key;
    bool some;
};
// The whole warp asks for rows m of its lanes, the first lane's being the least: 32 borders at a time lead to that lane's worker,
// and lanes beyond it go on by halves.
__device__ __forceinline__ Owner owner_of(const Dropout& p, long long m) {
    Owner o;
    int w = 0;
    o.first = 0;
    o.end = p.M;
    o.some = true;
    if (p.begin) {
        // (ordinary loads: a preceding kernel may have written the table while this one started)
        const long long* begin = reinterpret_cast<const long long*>(p.begin);
        const long long m0 = __shfl_sync(0xffffffffu, m, 0);
        int lo = -1, hi = p.N;                   // the last w with begin[w] <= m; -1: none
        while (lo < hi) {
            const int step = (hi - lo + 31) / 32, at = lo + 1 + (threadIdx.x & 31) * step;
            const unsigned below = __ballot_sync(0xffffffffu, at <= hi && begin[min(at, p.N)] <= m0);
            if (below == 0u) break;
            const int k = 31 - __clz(below);
            hi = min(hi, lo + (k + 1) * step);
            lo = lo + 1 + k * step;
        }
        hi = p.N;
        if (lo < p.N && begin[lo + 1] > m) hi = lo;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (begin[mid] <= m) lo = mid;
            else hi = mid - 1;
        }
        w = lo;
        o.some = lo >= 0 && lo < p.N;
        if (o.some) o.first = begin[lo];
        if (lo < p.N) o.end = begin[lo + 1];
    }
    o.key = splitmix_step(splitmix_step(p.first ^ ((uint64_t)p.round << 32 | (uint32_t)(p.worker0 + w))) ^ (0x8000000000000000ull | p.site));
    return o;
}

constexpr int kThreads = 256, kCtas = 4;     // CTAs on an SM
// Loads under way of a lane: with a residual twice as many bytes to a load.  Measured (4 / 2): 15001 x 4096 bfloat16 49 / 55 us
// (5.0 TB/s), with a residual 35395 x 1024 44 / 41 (5.3 TB/s).
__host__ __device__ constexpr int unroll(bool res) { return res ? 2 : 4; }

// Keeps and drops the elements of a lot of V from draw `place` on; f becomes residual + kept.
template <int V, bool RES> __device__ __forceinline__ void drop(float (&f)[V], const float (&g)[V], const Dropout& p, uint64_t key, uint64_t place) {
#pragma unroll
    for (int e = 0; e < V; e += 2) {
        const combo_step::f32x2 t = combo_step::mul2(combo_step::pair(f[e], f[e + 1]), combo_step::pair(p.scale, p.scale));
        f[e] = combo_step::lo_of(t);
        f[e + 1] = combo_step::hi_of(t);
    }
#pragma unroll
    for (int h = 0; h < V / 4; ++h) {
        const uint64_t z = splitmix_step(key ^ (place + h));
        const uint32_t half[2] = {(uint32_t)z, (uint32_t)(z >> 32)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t bits = e & 1 ? half[e >> 1] : half[e >> 1] << 16;      // the element's 16 bits in front
            const float t = bits >= p.threshold && !p.none_left ? f[h * 4 + e] : 0.0f;
            f[h * 4 + e] = RES ? t + g[h * 4 + e] : t;
        }
    }
}

// EB bytes an element.  VEC: a lane's lot is 16 aligned bytes; else four elements, one at a time.
template <int EB, bool VEC, bool RES> __global__ void __launch_bounds__(kThreads, kCtas) k_dropout(const Dropout p) {
    constexpr int V = VEC ? 16 / EB : 4, H = V / 4, U = unroll(RES);
    combo_step::pdl_release();
    const int lane = threadIdx.x & 31, side = 32 / p.lanes;      // rows side by side in a warp
    // a warp's rounds: several rows' or a part of one's
    const long long all = (p.M + side - 1) / side * p.rounds, from = ((long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * p.share;
    const long long to = min(from + p.share, all);
    combo_step::pdl_wait();
    if (from >= to) return;
    long long m = from / p.rounds * side + lane / p.lanes;
    int round = (int)(from % p.rounds);
    Owner o = {0, -1, 0, false};
    for (long long t = from; t < to; ++t) {
        const unsigned char* x = p.x + m * p.x_pitch * EB;
        const unsigned char* r = RES ? p.residual + m * p.r_pitch * EB : nullptr;
        unsigned char* y = p.y + m * p.y_pitch * EB;
        const int v0 = round * U * p.lanes + lane % p.lanes;
        uint4 a[U], b[U];
        const bool whole = VEC && m < p.M && (long long)(v0 + (U - 1) * p.lanes + 1) * V <= p.n;
        if (whole) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                a[k] = *reinterpret_cast<const uint4*>(x + (uint32_t)(v0 + k * p.lanes) * 16ull);
                if (RES) b[k] = *reinterpret_cast<const uint4*>(r + (uint32_t)(v0 + k * p.lanes) * 16ull);
            }
        }
        // the loads are under way while the worker is looked for
        if (__any_sync(0xffffffffu, m >= o.end && m < p.M)) o = owner_of(p, m);
        if (o.some && m < p.M) {
            const uint64_t place = (uint64_t)(m - o.first) * (uint32_t)p.lots;
            if (whole) {
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    if constexpr (VEC) {
                        float f[V], g[V];
                        Elem<EB>::unpack(a[k], f);
                        if (RES) Elem<EB>::unpack(b[k], g);
                        drop<V, RES>(f, g, p, o.key, place + (uint32_t)(v0 + k * p.lanes) * H);
                        *reinterpret_cast<uint4*>(y + (uint32_t)(v0 + k * p.lanes) * 16ull) = Elem<EB>::pack(f);
                    }
                }
            } else {
                // the end of a row, or rows off 16-byte boundaries
                for (int k = 0; k < U; ++k) {
                    const int v = v0 + k * p.lanes;
                    if (v >= p.width) break;
                    const long long at = (long long)v * V;
                    const int some = (int)min(p.n - at, (long long)V);
                    float f[V], g[V];
                    if (VEC && some == V) {
                        if constexpr (VEC) {
                            Elem<EB>::unpack(*reinterpret_cast<const uint4*>(x + at * EB), f);
                            if (RES) Elem<EB>::unpack(*reinterpret_cast<const uint4*>(r + at * EB), g);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            f[e] = e < some ? Elem<EB>::get(x + (at + e) * EB) : 0.0f;
                            g[e] = RES && e < some ? Elem<EB>::get(r + (at + e) * EB) : 0.0f;
                        }
                    }
                    drop<V, RES>(f, g, p, o.key, place + (uint32_t)v * H);
                    if (VEC && some == V) {
                        if constexpr (VEC) *reinterpret_cast<uint4*>(y + at * EB) = Elem<EB>::pack(f);
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            if (e < some) Elem<EB>::put(y + (at + e) * EB, f[e]);
                    }
                }
            }
        }
        if (++round == p.rounds) {
            round = 0;
            m += side;
        }
    }
}

template <int EB> cudaError_t launch(Dropout p, int sms, bool vec, cudaStream_t st) {
    const int V = vec ? 16 / EB : 4;
    p.lots = (int)((p.n + 3) / 4);
    p.width = (int)((p.n + V - 1) / V);
    const int U = unroll(p.residual != nullptr);
    // Lanes to a row: the fewest that take it in one round of loads.  The rounds are shared out evenly to as many warps as are
    // on the device at once.
    p.lanes = 1;
    while (p.lanes < 32 && p.lanes * U < p.width) p.lanes *= 2;
    p.rounds = (p.width + p.lanes * U - 1) / (p.lanes * U);
    const long long side = 32 / p.lanes, all = (p.M + side - 1) / side * p.rounds, warps = (long long)sms * kCtas * (kThreads / 32);
    p.share = (all + warps - 1) / warps;
    const long long grid = ((all + p.share - 1) / p.share + kThreads / 32 - 1) / (kThreads / 32);
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
        if (d_begin && combo_host::overlap(y, ry.extent(), d_begin, ((size_t)N + 1) * 8)) return COMBO_ERR_ALIAS;
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
