// The cross entropy's products on the tensor cores.
//
// Labelled rows are first packed: worker after worker, each from a multiple of 64 on, zeros behind a worker's last.  bfloat16 as
// it is; floats as planes that add up to them: forward two of float16, scaled by a power of two to each row's and class's largest
// (22 bits, or 2^-39 of the largest if that is more), backward three of bfloat16 (24 bits, whatever the range: d reaches over many
// orders, and planes of both kinds for the logits and for the gradients cost more than they save).  Then, for a piece of the classes at a time,
//
//                height (128 a CTA)      width                  summed r          results
//   logits       rows                    classes                inputs            forward: (max, sum of exponentials) of a row's 64 or 128
//                                                                                 classes; backward: d, as bfloat16 planes in scratch
//   rows'        rows                    inputs                 classes           dx, added up in scratch over the pieces
//   weights'     classes                 inputs                 rows              dW
//
// A lane of TMEM is a row of results, so the softmax needs no exchange between threads: a thread holds 64 or 128 logits of one row.
// Floats are products of planes: x0 w0 + (x0 w1 + x1 w0), and for three x0 w2 + x1 w1 + x2 w0; what is left out of a product is
// 2^-24 of it on average, or below that.  (Forward by three planes: 254 against 185 us for 32 x 1056 rows, 512 -> 1000.)
// The tensor cores truncate at every addition of 16 products, so only `part_steps` stages of 64 are summed there (floats: two, with the
// small products first), and the parts are added with rounding in the registers of the warps that take the results.
#pragma once
#include "tensor_core.cuh"

namespace combo_loss {

using namespace combo_tc;
using combo_step::add2;
using combo_step::f32x2;
using combo_step::hi_of;
using combo_step::lo_of;
using combo_step::mul2;
using combo_step::neg2;
using combo_step::pair;

enum Mode { kStats = 0, kGrad = 1, kRows = 2, kWeights = 3 };

constexpr int kStep = 64;                    // values of r in a stage
constexpr int kBlock = 64 * kStep * 2;       // bytes of a block of 64 x 64
constexpr int kFirstOutWarp = 4;
constexpr int out_threads(int warps) { return 32 * (kFirstOutWarp + warps); }
constexpr int kMaxStages = 8;
constexpr int kTurn = 32 * 33 * 4;           // weights': bytes in which a warp turns 32 x 32 results
constexpr int kPut = 32 * 128;               // bytes that a warp hands to TMA: 32 rows of 128
constexpr int kTmemColumns = 512;
constexpr int kStaticSmem = 1024;
constexpr float kLog2E = 1.4426950408889634f;

__device__ int g_loss_status;                // 0, or the site of the first wait that gave up
__device__ __forceinline__ bool give_up(int site) {
    atomicCAS(&g_loss_status, 0, site);
    return false;
}

// Where the packed rows of the workers lie: `row0` [N + 1] first packed row (multiples of 64), `tiles` [N + 2] tiles of rows before, and the
// number of parts of dx's sums.
struct Pass {
    const int *row0, *tiles;
    int N, V, K;
    int width, wt, ht;                       // of a tile; tiles along the width; along the height (weights')
    int steps, part_steps;                   // stages of r of a tile (weights': by the worker); summed by the tensor cores
    int stages, stage_bytes;
    int v0, w_row;                           // the piece's first class, and where the map of the weights has it
    int v_end;                               // weights': behind the piece's last class
    int add, vec;                            // rows': whether sums are there already; weights': whether TMA may store them
    int scaled;                              // whether d holds the rows' factors g; else the weights' gradients are divided by `count`
    long long row_cap;
    unsigned char* d;                        // [planes][d_blocks][row_cap] of eight classes in 16 bytes
    int d_blocks;
    long long dx_pitch;
    const int* label;                        // of packed rows; -1 behind a worker's last
    const float *lse, *g;
    const int* count;                        // labelled rows of a worker
    const float *x_unit, *w_unit;            // forward, floats: what a packed row's, and a class's of the piece, numbers count in
    int piece;                               // classes of a piece
    float2* part;                            // [pieces of a thread's columns][row_cap]
    float* own;                              // a row's logit of its label; kGrad: what the first plane of d leaves of its d
    float* dx;                               // [splits][rows][dx_pitch]
    unsigned char* dw;
    long long dw_pitch, dw_stride;
};
struct alignas(64) Maps {
    CUtensorMap a, b, out;                   // out: of dx or dW, 32 rows of 128 bytes to a box
};

// Into how many parts the sums over a piece's classes are cut, to have work for all CTAs where rows are few: the number with the
// least time, in tiles of the whole sum: turns of the CTAs by parts of a tile, and what a part's sums cost in memory (written, read
// and added up: `cost` for as many tiles as stages).
constexpr int kMaxSplits = 16, kMaxTurns = 4;
struct Splits {
    int clusters, wt, steps;                 // that run at once; tiles along the inputs; a whole piece's stages
    float cost;
};
__device__ __forceinline__ int splits_of(const Splits& q, int tiles) {
    const int total = tiles * q.wt;
    const float each = q.cost * total / q.steps;
    int best = 1;
    float least = 1e30f;
    for (int s = 1; s <= kMaxSplits && (s == 1 || (s * 8 <= q.steps && total * s <= kMaxTurns * q.clusters)); ++s) {
        const float time = (float)((total * s + q.clusters - 1) / q.clusters) / s + s * each;
        if (time < 0.95f * least) { least = time; best = s; }
    }
    return best;
}

struct Tile {
    int w, row, row_end;                     // worker; first packed row (rows', logits) or all that are summed
    int split, h0, c0;                       // first of the height (weights') and of the width
    int step0, steps;
};

// Walks the tiles t, t + stride, ...; the whole warp.  Lanes find 32 tiles at once: the search and the divisions take more than a
// thousand cycles, during which nothing is loaded (tiles of 16 stages: 621 cycles a stage with them before every tile, 597 so).
template <int CG, int MODE> struct Walk {
    const Pass& q;
    int t, stride, lane, at, splits;
    int w, row, rows, code, high;            // the lane's tile; w < 0: none
    __device__ __forceinline__ Walk(const Pass& q_, int first, int stride_) : q(q_), t(first), stride(stride_) {
        lane = threadIdx.x & 31;
        splits = MODE == kRows ? q.tiles[q.N + 1] : 1;
        at = 32;
    }
    __device__ __forceinline__ void find() {
        const int mine = t + lane * stride;
        w = -1;
        row = rows = code = high = 0;
        if (MODE == kWeights) {
            const int per = q.wt * q.ht;
            if (mine < per * q.N) {
                w = mine / per;
                const int k = mine - w * per;
                high = k / q.wt;
                code = k - high * q.wt;
                row = q.row0[w];
                rows = q.row0[w + 1] - row;
            }
        } else {
            const int mult = q.wt * splits;
            int lo = 0, hi = q.N;            // the last w with so many tiles before it
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (q.tiles[mid] * mult <= mine) lo = mid;
                else hi = mid - 1;
            }
            if (lo < q.N) {
                w = lo;
                const int before = q.tiles[w], tiles = q.tiles[w + 1] - before, k = mine - before * mult, rest = k / tiles;
                row = (k - rest * tiles) * 128 * CG;
                rows = q.row0[w + 1] - q.row0[w] - row;
                row += q.row0[w];
                code = rest;
            }
        }
        t += 32 * stride;
        at = 0;
    }
    __device__ __forceinline__ bool next(Tile& x) {
        if (at == 32) find();
        x.w = __shfl_sync(0xffffffffu, w, at);
        if (x.w < 0) return false;
        x.row = __shfl_sync(0xffffffffu, row, at);
        const int n = __shfl_sync(0xffffffffu, rows, at), c = __shfl_sync(0xffffffffu, code, at);
        x.row_end = x.row + n;
        x.h0 = x.split = x.step0 = 0;
        x.steps = q.steps;
        if (MODE == kWeights) {
            x.h0 = __shfl_sync(0xffffffffu, high, at) * 128 * CG;
            x.c0 = c * q.width;
            x.steps = n / kStep;
        } else if (MODE == kRows) {
            x.split = c / q.wt;
            x.c0 = (c - x.split * q.wt) * q.width;
            const int per = (q.steps + splits - 1) / splits;
            x.step0 = min(x.split * per, q.steps);
            x.steps = min(per, q.steps - x.step0);
        } else {
            x.c0 = c * q.width;
        }
        ++at;
        return true;
    }
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// A warp's columns c .. of acc, 128 bytes of a lane's row, into shared memory in TMA's order (16 bytes of a row at their number xor
// the row's), and on from there by `hand`, which one thread calls.
template <int EB, int kCols, typename F> __device__ __forceinline__ void put_box(uint32_t put, const f32x2 (&acc)[kCols], int c, int lane, F hand) {
    if (elect()) tma_store_wait_read();
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x2 v = acc[(EB == 4 ? (c + k * 4 + e) / 2 : (c + k * 8) / 2 + e) % kCols];
            o[e] = EB == 4 ? __float_as_uint(e & 1 ? hi_of(v) : lo_of(v)) : combo_step::pack_bf16(lo_of(v), hi_of(v));
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(put + lane * 128 + ((k ^ (lane & 7)) << 4)), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3])
                     : "memory");
    }
    fence_async();
    __syncwarp();
    if (elect()) hand();
    __syncwarp();
}

// PA, PB: planes of the height's and the width's operand.  OB: weights': bytes of a result; kGrad: planes of d.
template <int CG, int MODE, int PA, int PB, int OB, int kOutWarps>
__global__ void __launch_bounds__(out_threads(kOutWarps), 1) k_loss(const Pass q, const __grid_constant__ Maps maps) {
    constexpr bool A_R = MODE != kWeights, B_R = MODE == kStats || MODE == kGrad;
    constexpr int kPlanes = PA > PB ? PA : PB, kCols = 1024 / kOutWarps;
    constexpr bool kHalf = MODE == kStats && PA == 2;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 4];
    __shared__ uint32_t tmem_at;
    __shared__ int dead;                     // a wait of this CTA gave up: every role leaves its loop
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = CG == 1 ? 0 : (int)(blockIdx.x & 1);
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int s) { return bar0 + 8 * s; };
    const auto empty = [&](int s) { return bar0 + 8 * (kMaxStages + s); };
    const auto acc_full = [&](int b) { return bar0 + 8 * (2 * kMaxStages + b); };
    const auto acc_empty = [&](int b) { return bar0 + 8 * (2 * kMaxStages + 2 + b); };
    if (threadIdx.x == 0) {
        for (int s = 0; s < q.stages; ++s) {
            mbar_init(full(s), 2);           // one arrival for either operand, and the bytes of all CTAs
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), kOutWarps * CG);
        }
        mbar_init_fence();
        dead = 0;
        prefetch_map(&maps.a);
        prefetch_map(&maps.b);
    }
    if (warp == 1) tmem_alloc<CG>(smem_u32(&tmem_at), kTmemColumns);
    combo_step::pdl_release();
    combo_step::pdl_wait();
    tc_fence_before();
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    volatile int* dead_v = &dead;
    const int first = (int)blockIdx.x / CG, stride = (int)gridDim.x / CG;
    const int blocks_b = q.width / CG / 64;  // of 64 along the width, of this CTA
    Tile x;

    if (warp == 0 || warp == 2) {
        // ------------------------------------------------------------ loads: warp 0 the height's operand, warp 2 the width's
        const int op = warp >> 1;
        const CUtensorMap* map = op == 0 ? &maps.a : &maps.b;
        const int planes = op == 0 ? PA : PB, blocks = op == 0 ? 2 : blocks_b;
        const uint32_t bytes = (uint32_t)(planes * blocks) * kBlock, offset = op == 0 ? 0u : (uint32_t)PA * 2 * kBlock;
        const uint32_t bar_leader = CG == 1 ? full(0) : at_leader(full(0));
        Walk<CG, MODE> walk(q, first, stride);
        uint32_t done = 0;
        bool ok = true;
        while (walk.next(x)) {
            uint32_t s = done % q.stages, ph = done / q.stages & 1u;
            if (elect()) {
                // along the operand's own index; a step goes along r
                const int own = op == 0 ? (MODE == kWeights ? x.h0 : x.row) + rank * 128 : x.c0 + rank * blocks_b * 64;
                for (int k = 0; k < x.steps; ++k) {
                    if (!mbar_wait(empty(s), ph ^ 1u, dead_v)) { ok = give_up(50); break; }
                    if (rank == 0) mbar_arrive_expect(full(s), bytes * CG);
                    uint32_t to = smem + s * q.stage_bytes + offset;
                    const int r = (x.step0 + k) * kStep, bar = bar_leader + 8 * s;
                    for (int p = 0; p < planes; ++p) {
                        if (op == 0 && (MODE == kRows || MODE == kWeights)) {
                            // d: both blocks at once
                            if (MODE == kRows) tma_3d<CG>(to, map, 2 * own, r / 8, p, bar);
                            else tma_3d<CG>(to, map, 2 * (x.row + r), own / 8, p, bar);
                            to += 2 * kBlock;
                            continue;
                        }
                        for (int b = 0; b < blocks; ++b, to += kBlock) {
                            const int i = own + b * 64;
                            if (op == 0) tma_3d<CG>(to, map, r, i, p, bar);
                            else if (MODE == kRows) tma_4d<CG>(to, map, i, q.w_row + r, x.w, p, bar);
                            else if (MODE == kWeights) tma_3d<CG>(to, map, i, x.row + r, p, bar);
                            else tma_4d<CG>(to, map, r, q.w_row + i, x.w, p, bar);
                        }
                    }
                    if (++s == (uint32_t)q.stages) { s = 0; ph ^= 1u; }
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            done += x.steps;
        }
        if (!ok) {
            // after a wait that gave up nothing tells when the copies under way have landed: far longer than they take
            *dead_v = 1;
            for (int k = 0; k < 2000; ++k) __nanosleep(1000);
        }
        // No copy may be under way when the CTA leaves: the products have freed the last stages.
        for (uint32_t k = 1; k <= done && k <= (uint32_t)q.stages && ok; ++k)
            ok = mbar_wait(empty((done - k) % q.stages), (done - k) / q.stages & 1u, dead_v) || give_up(51);
    } else if (warp == 1) {
        // ------------------------------------------------------------ products, by one thread of the leader
        if (rank == 0) {
            Walk<CG, MODE> walk(q, first, stride);
            uint32_t done = 0, turn = 0;     // stages; parts, which take the two accumulators in turn
            bool ok = true;
            const uint32_t kind = kHalf ? product_kind_half(128 * CG, q.width, A_R, B_R) : product_kind(128 * CG, q.width, A_R, B_R);
            while (walk.next(x)) {
                const int parts = (x.steps + q.part_steps - 1) / q.part_steps;
                if (elect()) {
                    uint32_t s = done % q.stages, ph = done / q.stages & 1u;
                    for (int part = 0; part < parts && ok; ++part) {
                        const uint32_t n = turn + part, buf = n & 1u, d = tmem + buf * 256;
                        if (!mbar_wait(acc_empty(buf), (n >> 1 & 1u) ^ 1u, dead_v)) { ok = give_up(52); break; }
                        tc_fence_after();
                        const int k1 = min((part + 1) * q.part_steps, x.steps);
                        for (int k = part * q.part_steps; k < k1; ++k) {
                            if (!mbar_wait(full(s), ph, dead_v)) { ok = give_up(53); break; }
                            tc_fence_after();
                            const uint32_t a0 = smem + s * q.stage_bytes, b0 = a0 + PA * 2 * kBlock;
                            bool add = k > part * q.part_steps;
#pragma unroll
                            for (int sum = kPlanes - 1; sum >= 0; --sum)
#pragma unroll
                                for (int pa = 0; pa <= sum; ++pa) {
                                    const int pb = sum - pa;
                                    if (pa >= PA || pb >= PB) continue;
                                    const uint32_t a = a0 + pa * 2 * kBlock;
                                    const uint64_t da = MODE == kRows ? operand_plain(a, 128 * 16, 128) : MODE == kWeights ? operand_plain(a, 128, 64 * 16) : operand(a, true, 0);
                                    const uint64_t db = operand(b0 + pb * blocks_b * kBlock, B_R, kBlock);
                                    constexpr uint32_t kStepA = MODE == kRows ? 2 * 128 * 16 : MODE == kWeights ? 2 * 128 : step16(true);
#pragma unroll
                                    for (int c = 0; c < kStep / 16; ++c) {
                                        mma<CG>(d, da + (uint64_t)(c * kStepA >> 4), db + (uint64_t)(c * step16(B_R) >> 4), kind, add);
                                        add = true;
                                    }
                                }
                            mma_commit<CG>(empty(s));
                            if (++s == (uint32_t)q.stages) { s = 0; ph ^= 1u; }
                        }
                        if (ok) mma_commit<CG>(acc_full(buf));
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                done += x.steps;
                turn += parts;
            }
            if (!ok) *dead_v = 1;
        }
    } else if (warp >= kFirstOutWarp) {
        // ------------------------------------------------------------ results: a warp's quarter of the rows by its part of the columns
        Walk<CG, MODE> walk(q, first, stride);
        const int quarter = warp & 3, share = (warp - kFirstOutWarp) >> 2, columns = q.width / (kOutWarps / 4);
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + share * columns;
        uint32_t turn = 0;
        const uint32_t put = smem + q.stages * q.stage_bytes + (warp - kFirstOutWarp) * kPut;
        bool ok = true;
        while (walk.next(x)) {
            const int parts = (x.steps + q.part_steps - 1) / q.part_steps;
            const int col = x.c0 + share * columns;      // the first of the thread's columns
            const int j = x.row + rank * 128 + quarter * 32 + lane;          // the packed row (weights': none)
            // workers' rows begin at multiples of 64: a warp's are all this worker's, or another's or nobody's
            const bool mine = MODE != kWeights && j < x.row_end;
            f32x2 acc[kCols / 2];                        // pairs of columns
#pragma unroll
            for (int e = 0; e < kCols / 2; ++e) acc[e] = 0;
            for (int part = 0; part < parts; ++part) {
                const uint32_t n = turn + part, buf = n & 1u;
                ok = mbar_wait(acc_full(buf), n >> 1 & 1u, dead_v) || give_up(54);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < kCols; c += 16) {
                    if (c < columns) {
                        uint32_t v[16];
                        tmem_load16(lanes + buf * 256 + c, v);
                        tmem_load_wait(v);
#pragma unroll
                        for (int e = 0; e < 8; ++e) acc[c / 2 + e] = add2(acc[c / 2 + e], pair(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])));
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(CG == 1 ? acc_empty(buf) : at_leader(acc_empty(buf)));
            }
            if (!ok) break;
            turn += parts;
            if constexpr (MODE == kWeights) {
                if (!q.scaled) {
                    const float scale = parts > 0 ? 1.0f / (float)q.count[x.w] : 0.0f;
#pragma unroll
                    for (int e = 0; e < kCols / 2; ++e) acc[e] = mul2(acc[e], pair(scale, scale));
                }
                const int v = q.v0 + x.h0 + rank * 128 + quarter * 32;
                if (v >= q.v_end) continue;
                const int lines = min(q.v_end - v, 32);
                if (q.vec) {
                    // TMA writes whole 16 bytes: the box in which a line ends inside them is left to the lanes, a class each
                    const bool whole = q.K * OB % 16 == 0;
#pragma unroll
                    for (int c = 0; c < kCols; c += 128 / OB) {
                        if (c < columns && col + c < q.K) {
                            if (whole || col + c + 128 / OB <= q.K) {
                                put_box<OB, kCols / 2>(put, acc, c, lane, [&] { tma_store_3d(&maps.out, put, col + c, v, x.w); });
                            } else if (lane < lines) {
                                unsigned char* to = q.dw + (x.w * q.dw_stride + (v + lane) * q.dw_pitch + col + c) * OB;
#pragma unroll
                                for (int e = 0; e < 128 / OB; ++e)
                                    if (col + c + e < q.K) combo_step::Elem<OB>::put(to + e * OB, e & 1 ? hi_of(acc[(c + e) / 2 % (kCols / 2)]) : lo_of(acc[(c + e) / 2 % (kCols / 2)]));
                            }
                        }
                    }
                } else {
                    // off 16-byte boundaries: lots of 32 x 32 are turned and stored a line at a time
                    float* turned = reinterpret_cast<float*>(smem_raw + (smem - smem_u32(smem_raw)) + q.stages * q.stage_bytes + (warp - kFirstOutWarp) * kTurn);
#pragma unroll
                    for (int c = 0; c < kCols; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                turned[lane * 33 + 2 * e] = lo_of(acc[c / 2 + e]);
                                turned[lane * 33 + 2 * e + 1] = hi_of(acc[c / 2 + e]);
                            }
                            __syncwarp();
                            if (c + lane < columns && col + c + lane < q.K)
                                for (int line = 0; line < lines; ++line)
                                    combo_step::Elem<OB>::put(q.dw + (x.w * q.dw_stride + (v + line) * q.dw_pitch + col + c + lane) * OB, turned[line * 33 + lane]);
                            __syncwarp();
                        }
                    }
                }
            } else {
                if (!mine) continue;
                if constexpr (kHalf) {
                    const float unit = q.x_unit[j];
                    const float4* units = reinterpret_cast<const float4*>(q.w_unit + (long long)x.w * q.piece + col);
#pragma unroll
                    for (int c = 0; c < kCols; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = c; e < c + 32; e += 4) {
                                const float4 u = units[e / 4];
                                acc[e / 2] = mul2(mul2(acc[e / 2], pair(unit, unit)), pair(u.x, u.y));
                                acc[e / 2 + 1] = mul2(mul2(acc[e / 2 + 1], pair(unit, unit)), pair(u.z, u.w));
                            }
                        }
                    }
                }
                if constexpr (MODE == kStats) {
                    // classes that are not there
                    const int left = q.V - (q.v0 + col);
                    if (left < columns) {
#pragma unroll
                        for (int e = 0; e < kCols; e += 2)
                            acc[e / 2] = pair(e < left ? lo_of(acc[e / 2]) : -INFINITY, e + 1 < left ? hi_of(acc[e / 2]) : -INFINITY);
                    }
                    float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < kCols; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) most[e & 3] = fmaxf(most[e & 3], fmaxf(lo_of(acc[c / 2 + e]), hi_of(acc[c / 2 + e])));
                        }
                    }
                    // differences to the largest first, so that a row's sum holds a 1 and no rounding of large logits
                    const float m = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])), zero = m == -INFINITY ? 0.0f : -m;
                    f32x2 sum[2] = {0, 0};
#pragma unroll
                    for (int c = 0; c < kCols; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const f32x2 x2 = mul2(add2(acc[c / 2 + e], pair(zero, zero)), pair(kLog2E, kLog2E));
                                sum[e & 1] = add2(sum[e & 1], pair(exp2_fast(lo_of(x2)), exp2_fast(hi_of(x2))));
                            }
                        }
                    }
                    sum[0] = add2(sum[0], sum[1]);
                    q.part[((q.v0 + col) / columns) * q.row_cap + j] = make_float2(m, lo_of(sum[0]) + hi_of(sum[0]));
                    const int at = q.label[j] - q.v0 - col;
                    if (__any_sync(0xffffffffu, at >= 0 && at < columns)) {
                        float z = 0.0f;
#pragma unroll
                        for (int e = 0; e < kCols; ++e)
                            if (e == at) z = e & 1 ? hi_of(acc[e / 2]) : lo_of(acc[e / 2]);
                        if (at >= 0 && at < columns) q.own[j] = z;
                    }
                } else if constexpr (MODE == kGrad) {
                    const int left = q.v_end - (q.v0 + col), label = q.label[j];
                    const float lse = label >= 0 ? -q.lse[j] : 0.0f;
                    const int at = label - q.v0 - col;
                    const bool here = label >= 0 && at >= 0 && at < columns;
                    const bool any = __any_sync(0xffffffffu, here), all = __all_sync(0xffffffffu, label >= 0) && left >= columns;
                    float g = 1.0f;
                    if (q.scaled) g = label >= 0 ? q.g[j] : 0.0f;
                    unsigned char* to = q.d + ((long long)(col / 8) * q.row_cap + j) * 16;
                    float own = 0.0f;                // d of the row's label
                    // 32 classes at a time, from the logits to their places in scratch: 16 bytes a lane, a warp's side by side
#pragma unroll
                    for (int c = 0; c < kCols; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = c / 2; e < c / 2 + 16; ++e) {
                                // the difference first: a product would be rounded at the size of the logits
                                const f32x2 x2 = mul2(add2(acc[e], pair(lse, lse)), pair(kLog2E, kLog2E));
                                acc[e] = pair(exp2_fast(lo_of(x2)), exp2_fast(hi_of(x2)));
                            }
                            if (any) {
#pragma unroll
                                for (int e = c; e < c + 32; e += 2)
                                    acc[e / 2] = add2(acc[e / 2], pair(e == at ? -1.0f : 0.0f, e + 1 == at ? -1.0f : 0.0f));
                            }
                            if (q.scaled) {
#pragma unroll
                                for (int e = c / 2; e < c / 2 + 16; ++e) acc[e] = mul2(acc[e], pair(g, g));
                            }
                            if (!all) {
                                // rows without a label and classes that are not there: 0, whatever the product is
#pragma unroll
                                for (int e = c; e < c + 32; e += 2)
                                    acc[e / 2] = pair(label >= 0 && e < left ? lo_of(acc[e / 2]) : 0.0f, label >= 0 && e + 1 < left ? hi_of(acc[e / 2]) : 0.0f);
                            }
                            if (any) {
#pragma unroll
                                for (int e = c; e < c + 32; ++e)
                                    if (e == at) own = e & 1 ? hi_of(acc[e / 2]) : lo_of(acc[e / 2]);
                            }
#pragma unroll
                            for (int p = 0; p < OB; ++p) {
#pragma unroll
                                for (int k = c; k < c + 32; k += 8) {
                                    uint32_t o[4];
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        f32x2& v = acc[k / 2 + e];
                                        o[e] = combo_step::pack_bf16(lo_of(v), hi_of(v));
                                        if (p + 1 < OB) v = add2(v, neg2(pair(combo_step::widen_lo(o[e]), combo_step::widen_hi(o[e]))));
                                    }
                                    *reinterpret_cast<uint4*>(to + ((long long)p * q.d_blocks + k / 8) * q.row_cap * 16) = make_uint4(o[0], o[1], o[2], o[3]);
                                }
                            }
                        }
                    }
                    if (here) q.own[j] = own - combo_step::widen_lo(combo_step::pack_bf16(own, 0.0f));
                } else {
                    const int y = x.split * q.row0[q.N] + j - lane;
                    if (!q.add || x.steps > 0) {
#pragma unroll
                        for (int c = 0; c < kCols; c += 32)
                            if (c < columns) put_box<4, kCols / 2>(put, acc, c, lane, [&] { q.add ? tma_add_3d(&maps.out, put, col + c, y, 0) : tma_store_3d(&maps.out, put, col + c, y, 0); });
                    }
                }
            }
        }
        if (MODE == kRows || MODE == kWeights) tma_store_wait();
        if (!ok) *dead_v = 1;
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    tc_fence_after();
    if (warp == 1) tmem_release<CG>(tmem, kTmemColumns);
}

}  // namespace combo_loss
