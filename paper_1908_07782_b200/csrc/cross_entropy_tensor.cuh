// The cross entropy's products on the tensor cores.
//
// Labelled rows are first packed: worker after worker, each from a multiple of 64 on, as bfloat16 planes (floats: three, which hold
// all 24 bits: x = x0 + x1 + x2), zeros behind a worker's last.  Then, for a piece of the classes at a time,
//
//                height (128 a CTA)      width                  summed r          results
//   logits       rows                    classes                inputs            forward: (max, sum of exponentials) of a row's 128
//                                                                                 classes; backward: d, as bfloat16 planes in scratch
//   rows'        rows                    inputs                 classes           dx, added up in scratch over the pieces
//   weights'     classes                 inputs                 rows              dW
//
// A lane of TMEM is a row of results, so the softmax needs no exchange between threads: a thread holds 128 logits of one row.
// Floats are products of planes: x0 w0 + (x0 w1 + x1 w0) + (x0 w2 + x1 w1 + x2 w0); what is left out is below 2^-24 of a product.
// The tensor cores truncate at every addition of 16 products, so only `part_steps` stages of 64 are summed there (floats: one, with the
// small products first), and the parts are added with rounding in the registers of the warps that take the results.
#pragma once
#include "tensor_core.cuh"

namespace combo_loss {

using namespace combo_tc;

enum Mode { kStats = 0, kGrad = 1, kRows = 2, kWeights = 3 };

constexpr int kStep = 64;                    // values of r in a stage
constexpr int kBlock = 64 * kStep * 2;       // bytes of a block of 64 x 64
constexpr int kOutWarps = 8, kFirstOutWarp = 4, kTcThreads = 32 * (kFirstOutWarp + kOutWarps);
constexpr int kMaxStages = 8;
constexpr int kTurn = 32 * 33 * 4;           // weights': bytes in which a warp turns 32 x 32 results
constexpr int kPut = 32 * 128;               // kGrad: bytes that a warp hands to TMA, 32 rows of 64 values; two such places
constexpr int kTmemColumns = 512;
constexpr int kStaticSmem = 1024;
constexpr float kLog2E = 1.4426950408889634f;

__device__ int g_loss_status;                // 0, or the site of the first wait that gave up
__device__ __forceinline__ bool give_up(int site) {
    atomicCAS(&g_loss_status, 0, site);
    return false;
}

// Where the packed rows of the workers lie: `row0` [N + 1] first packed row (multiples of 64), `tiles` [N + 1] tiles of rows before.
struct Pass {
    const int *row0, *tiles;
    int N, V, K;
    int width, wt, ht;                       // of a tile; tiles along the width; along the height (weights')
    int steps, part_steps;                   // stages of r of a tile (weights': by the worker); summed by the tensor cores
    int stages, stage_bytes;
    int v0, w_row;                           // the piece's first class, and where the map of the weights has it
    int v_end;                               // weights': behind the piece's last class
    int clusters, split_steps;               // rows': that run at once; a whole piece's stages
    int add, vec;                            // rows': whether sums are there already; weights': bytes that a store may take at once
    int scaled;                              // whether d holds the rows' factors g; else the weights' gradients are divided by `count`
    long long row_cap, dx_pitch;
    const int* label;                        // of packed rows; -1 behind a worker's last
    const float *lse, *g;
    const int* count;                        // labelled rows of a worker
    float2* part;                            // [2 tiles of classes][row_cap]
    float* own;                              // a row's logit of its label; kGrad: what the first plane of d leaves of its d
    float* dx;                               // [splits][rows][dx_pitch]
    unsigned char* dw;
    long long dw_pitch, dw_stride;
};
struct alignas(64) Maps {
    CUtensorMap a, b, d;                     // d: kGrad's results, [planes][row_cap][piece], 32 rows to a box
};

// Into how many parts the sums over a piece's classes are cut, to have work for all CTAs where rows are few: the number with the
// fewest turns for the whole, a turn being a part of a tile; of at least eight stages, and in four turns at most.
constexpr int kMaxSplits = 16, kMaxTurns = 4;
__device__ __forceinline__ int splits_of(const Pass& q) {
    const int total = q.tiles[q.N] * q.wt;
    int best = 1;
    float least = 1e30f;
    for (int s = 1; s <= kMaxSplits && (s == 1 || (s * 8 <= q.split_steps && total * s <= kMaxTurns * q.clusters)); ++s) {
        const float turns = (float)((total * s + q.clusters - 1) / q.clusters) / s;
        if (turns < 0.95f * least) { least = turns; best = s; }
    }
    return best;
}

struct Tile {
    int w, row, row_end;                     // worker; first packed row (rows', logits) or all that are summed
    int split, h0, c0;                       // first of the height (weights') and of the width
    int step0, steps;
};

// Walks the tiles t, t + stride, ...; the whole warp.
template <int CG, int MODE> struct Walk {
    const Pass& q;
    int t, lane, w0, mult, splits, upto;     // upto: tiles up to the lane's worker, that one with it
    __device__ __forceinline__ Walk(const Pass& q_, int first) : q(q_), t(first) {
        lane = threadIdx.x & 31;
        splits = MODE == kRows ? splits_of(q) : 1;
        mult = q.wt * splits;
        w0 = 0;
        if (MODE != kWeights) lot();
    }
    __device__ __forceinline__ void lot() { upto = q.tiles[min(w0 + lane + 1, q.N)] * mult; }
    __device__ __forceinline__ bool next(Tile& x, int stride) {
        if (MODE == kWeights) {
            const int per = q.wt * q.ht;
            if (t >= per * q.N) return false;
            x.w = t / per;
            const int k = t - x.w * per;
            x.c0 = k % q.wt * q.width;
            x.h0 = k / q.wt * 128 * CG;
            x.row = q.row0[x.w];
            x.row_end = q.row0[x.w + 1];
            x.split = x.step0 = 0;
            x.steps = (x.row_end - x.row) / kStep;
        } else {
            unsigned m;
            while (!(m = __ballot_sync(0xffffffffu, upto > t))) {
                w0 += 32;
                if (w0 >= q.N) return false;
                lot();
            }
            x.w = w0 + __ffs(m) - 1;
            const int before = q.tiles[x.w], mine = q.tiles[x.w + 1] - before, at = t - before * mult, rest = at / mine;
            x.split = rest / q.wt;
            x.c0 = (rest - x.split * q.wt) * q.width;
            x.h0 = 0;
            x.row = q.row0[x.w] + (at - rest * mine) * 128 * CG;
            x.row_end = q.row0[x.w + 1];
            const int per = MODE == kRows ? (q.steps + splits - 1) / splits : q.steps;
            x.step0 = min(x.split * per, q.steps);
            x.steps = min(per, q.steps - x.step0);
        }
        t += stride;
        return true;
    }
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void store32(void* to, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ void load32(const void* from, uint32_t (&v)[8]) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "l"(from)
                 : "memory");
}

// PA, PB: planes of the height's and the width's operand.  OB: weights': bytes of a result; kGrad: planes of d.
template <int CG, int MODE, int PA, int PB, int OB>
__global__ void __launch_bounds__(kTcThreads, 1) k_loss(const Pass q, const __grid_constant__ Maps maps) {
    constexpr bool A_R = MODE != kWeights, B_R = MODE == kStats || MODE == kGrad;
    constexpr int kPlanes = PA > PB ? PA : PB;
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
        Walk<CG, MODE> walk(q, first);
        uint32_t done = 0;
        bool ok = true;
        while (walk.next(x, stride)) {
            uint32_t s = done % q.stages, ph = done / q.stages & 1u;
            if (elect()) {
                // along the operand's own index; a step goes along r
                const int own = op == 0 ? (MODE == kWeights ? x.h0 : x.row) + rank * 128 : x.c0 + rank * blocks_b * 64;
                for (int k = 0; k < x.steps; ++k) {
                    if (!mbar_wait(empty(s), ph ^ 1u, dead_v)) { ok = give_up(50); break; }
                    if (rank == 0) mbar_arrive_expect(full(s), bytes * CG);
                    uint32_t to = smem + s * q.stage_bytes + offset;
                    const int r = (x.step0 + k) * kStep, bar = bar_leader + 8 * s;
                    for (int p = 0; p < planes; ++p)
                        for (int b = 0; b < blocks; ++b, to += kBlock) {
                            const int i = own + b * 64;
                            if (MODE == kStats || MODE == kGrad) {
                                if (op == 0) tma_3d<CG>(to, map, r, i, p, bar);
                                else tma_4d<CG>(to, map, r, q.w_row + i, x.w, p, bar);
                            } else if (MODE == kRows) {
                                if (op == 0) tma_3d<CG>(to, map, r, i, p, bar);
                                else tma_4d<CG>(to, map, i, q.w_row + r, x.w, p, bar);
                            } else {
                                tma_3d<CG>(to, map, i, x.row + r, p, bar);
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
            Walk<CG, MODE> walk(q, first);
            uint32_t done = 0, turn = 0;     // stages; parts, which take the two accumulators in turn
            bool ok = true;
            const uint32_t kind = product_kind(128 * CG, q.width, A_R, B_R);
            while (walk.next(x, stride)) {
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
                                    const uint64_t da = operand(a0 + pa * 2 * kBlock, A_R, kBlock), db = operand(b0 + pb * blocks_b * kBlock, B_R, kBlock);
#pragma unroll
                                    for (int c = 0; c < kStep / 16; ++c) {
                                        mma<CG>(d, da + (uint64_t)(c * step16(A_R) >> 4), db + (uint64_t)(c * step16(B_R) >> 4), kind, add);
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
        // ------------------------------------------------------------ results: four warps for either half of the columns
        Walk<CG, MODE> walk(q, first);
        const int quarter = warp & 3, half = (warp - kFirstOutWarp) >> 2, columns = q.width / 2;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + half * columns;
        uint32_t turn = 0, puts = 0;
        const uint32_t put = smem + q.stages * q.stage_bytes + (warp - kFirstOutWarp) * 2 * kPut;
        bool ok = true;
        while (walk.next(x, stride)) {
            const int parts = (x.steps + q.part_steps - 1) / q.part_steps;
            const int col = x.c0 + half * columns;       // the first of the thread's columns
            const int j = x.row + rank * 128 + quarter * 32 + lane;          // the packed row (weights': none)
            // workers' rows begin at multiples of 64: a warp's are all this worker's, or another's or nobody's
            const bool mine = MODE != kWeights && j < x.row_end;
            float acc[128];
#pragma unroll
            for (int e = 0; e < 128; ++e) acc[e] = 0.0f;
            if (MODE == kRows && q.add && mine && x.steps > 0) {
                const float* from = q.dx + ((long long)x.split * q.row0[q.N] + j) * q.dx_pitch + col;
#pragma unroll
                for (int c = 0; c < 128; c += 8) {
                    if (c < columns) {
                        uint32_t o[8];
                        load32(from + c, o);
#pragma unroll
                        for (int e = 0; e < 8; ++e) acc[c + e] = __uint_as_float(o[e]);
                    }
                }
            }
            for (int part = 0; part < parts; ++part) {
                const uint32_t n = turn + part, buf = n & 1u;
                ok = mbar_wait(acc_full(buf), n >> 1 & 1u, dead_v) || give_up(54);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < 128; c += 16) {
                    if (c < columns) {
                        uint32_t v[16];
                        tmem_load16(lanes + buf * 256 + c, v);
                        tmem_load_wait(v);
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[c + e] += __uint_as_float(v[e]);
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
                    for (int e = 0; e < 128; ++e) acc[e] *= scale;
                }
                const int v = q.v0 + x.h0 + rank * 128 + quarter * 32 + lane;
                if (q.vec) {
                    if (v < q.v_end) {
                        unsigned char* to = q.dw + (x.w * q.dw_stride + v * q.dw_pitch + col) * OB;
                        constexpr int kLane = 32 / OB;   // 32 bytes a store, or 16
#pragma unroll
                        for (int c = 0; c < 128; c += kLane) {
                            if (c < columns) {
                                uint32_t o[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    o[e] = OB == 4 ? __float_as_uint(acc[c + (OB == 4 ? e : 0)]) : combo_step::pack_bf16(acc[c + (OB == 4 ? 0 : 2 * e)], acc[c + (OB == 4 ? 0 : 2 * e + 1)]);
                                if (col + c + kLane <= q.K && q.vec == 32) {
                                    store32(to + c * OB, o);
                                } else if (col + c < q.K) {
                                    // K is a multiple of what 16 bytes hold
                                    *reinterpret_cast<uint4*>(to + c * OB) = make_uint4(o[0], o[1], o[2], o[3]);
                                    if (col + c + kLane / 2 < q.K) *reinterpret_cast<uint4*>(to + c * OB + 16) = make_uint4(o[4], o[5], o[6], o[7]);
                                }
                            }
                        }
                    }
                } else {
                    // off 16-byte boundaries: lots of 32 x 32 are turned and stored a line at a time
                    float* turned = reinterpret_cast<float*>(smem_raw + (smem - smem_u32(smem_raw)) + q.stages * q.stage_bytes + (warp - kFirstOutWarp) * kTurn);
                    const int base = q.v0 + x.h0 + rank * 128 + quarter * 32, lines = min(q.v_end - base, 32);
#pragma unroll
                    for (int c = 0; c < 128; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) turned[lane * 33 + e] = acc[c + e];
                            __syncwarp();
                            if (col + c + lane < q.K)
                                for (int line = 0; line < lines; ++line)
                                    combo_step::Elem<OB>::put(q.dw + (x.w * q.dw_stride + (base + line) * q.dw_pitch + col + c + lane) * OB, turned[line * 33 + lane]);
                            __syncwarp();
                        }
                    }
                }
            } else {
                if (!mine) continue;
                if constexpr (MODE == kStats) {
                    // classes that are not there
                    const int left = q.V - (q.v0 + col);
                    if (left < columns) {
#pragma unroll
                        for (int e = 0; e < 128; ++e)
                            if (e >= left) acc[e] = -INFINITY;
                    }
                    float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 128; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) most[e & 3] = fmaxf(most[e & 3], acc[c + e]);
                        }
                    }
                    const float m = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])), zero = m == -INFINITY ? 0.0f : m;
                    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int c = 0; c < 128; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) sum[e & 3] += exp2_fast((acc[c + e] - zero) * kLog2E);
                        }
                    }
                    q.part[((q.v0 + col) / columns) * q.row_cap + j] = make_float2(m, (sum[0] + sum[1]) + (sum[2] + sum[3]));
                    const int at = q.label[j] - q.v0 - col;
                    if (__any_sync(0xffffffffu, at >= 0 && at < columns)) {
                        float z = 0.0f;
#pragma unroll
                        for (int e = 0; e < 128; ++e)
                            if (e == at) z = acc[e];
                        if (at >= 0 && at < columns) q.own[j] = z;
                    }
                } else if constexpr (MODE == kGrad) {
                    const int left = q.v_end - (q.v0 + col), label = q.label[j];
                    const float lse = label >= 0 ? q.lse[j] : 0.0f;
                    const int at = label - q.v0 - col;
#pragma unroll
                    for (int c = 0; c < 128; c += 32) {
                        if (c < columns) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) acc[c + e] = exp2_fast((acc[c + e] - lse) * kLog2E);
                        }
                    }
                    const bool here = label >= 0 && at >= 0 && at < columns;
                    const bool any = __any_sync(0xffffffffu, here);
                    if (any) {
#pragma unroll
                        for (int e = 0; e < 128; ++e)
                            if (e == at) acc[e] -= 1.0f;
                    }
                    if (q.scaled) {
                        const float g = label >= 0 ? q.g[j] : 0.0f;
#pragma unroll
                        for (int e = 0; e < 128; ++e) acc[e] *= g;
                    }
                    // rows without a label and classes that are not there: 0, whatever the product is
                    if (left < columns) {
#pragma unroll
                        for (int e = 0; e < 128; ++e)
                            if (e >= left) acc[e] = 0.0f;
                    }
                    if (!__all_sync(0xffffffffu, label >= 0)) {
#pragma unroll
                        for (int e = 0; e < 128; ++e) acc[e] = label >= 0 ? acc[e] : 0.0f;
                    }
                    if (any) {
                        float rest = 0.0f;
#pragma unroll
                        for (int e = 0; e < 128; ++e)
                            if (e == at) rest = acc[e] - combo_step::widen_lo(combo_step::pack_bf16(acc[e], 0.0f));
                        if (here) q.own[j] = rest;
                    }
                    // 64 columns of a plane at a time, in TMA's order: 16 bytes of a row at (their number xor the row's) of its 128
#pragma unroll
                    for (int p = 0; p < OB; ++p) {
#pragma unroll
                        for (int c = 0; c < 128; c += 64) {
                            if (c < columns) {
                                const uint32_t place = put + (puts & 1u) * kPut;
                                if (elect()) tma_store_wait_read<1>();
                                __syncwarp();
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    uint32_t o[4];
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        float &lo = acc[c + k * 8 + 2 * e], &hi = acc[c + k * 8 + 2 * e + 1];
                                        o[e] = combo_step::pack_bf16(lo, hi);
                                        if (p + 1 < OB) {
                                            lo -= combo_step::widen_lo(o[e]);
                                            hi -= combo_step::widen_hi(o[e]);
                                        }
                                    }
                                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place + lane * 128 + ((k ^ (lane & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                                                 "r"(o[2]), "r"(o[3])
                                                 : "memory");
                                }
                                fence_async();
                                __syncwarp();
                                if (elect()) tma_store_3d(&maps.d, place, col + c, j - lane, p);
                                __syncwarp();
                                ++puts;
                            }
                        }
                    }
                } else {
                    float* to = q.dx + ((long long)x.split * q.row0[q.N] + j) * q.dx_pitch + col;
                    if (!q.add || x.steps > 0) {
#pragma unroll
                        for (int c = 0; c < 128; c += 8) {
                            if (c < columns) {
                                uint32_t o[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(acc[c + e]);
                                store32(to + c, o);
                            }
                        }
                    }
                }
            }
        }
        if (MODE == kGrad) tma_store_wait();
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
