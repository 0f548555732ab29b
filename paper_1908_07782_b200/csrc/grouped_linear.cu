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
//
// Measured (bfloat16 on 16-byte boundaries unless said): forward 16 x 1065 rows, 1024 -> 4096: 116 to 122 us in the first hundred
// calls (1200 TFLOP/s of a measured 1675), 136 to 144 in calls that go on (1020 of 1385), when the power limit has the clock
// at 1.22 to 1.33 GHz instead of 1.97; gradient of the weights 16 x 924 rows, 4096 -> 1024, into floats: 112 to 118 us (1050),
// then 130 to 139 (900); of the rows 32 x 168, 2048 -> 1000: 45 to 68 us, by where the arrays lie, bound by its 131 MB of weights;
// one row a worker, 16 x 1024 -> 1024: 8.7 us for 33 MB.  Off 16-byte boundaries 100 to 180 TFLOP/s; floats 46 TFLOP/s, bound by
// the multiply-add pipe.
#include <string.h>

#include "host_common.h"
#include "step_common.cuh"
#include "tensor_core.cuh"

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
// float operands: FT x FT outputs for a block of 256 threads, 128 with 8 x 8 each or 64 with 4 x 4, 16 values of r at a time
// through two shared-memory stages; the next stage's loads are in registers while this one's products are formed.  Any
// pitch and alignment.
constexpr int kFK = 16, kFThreads = 256;
constexpr int kFPad = 4;

// N neighbouring elements of one line; those at or beyond `left` are zero.
template <int N> __device__ __forceinline__ void load_some(const unsigned char* q, int left, bool vec, float (&v)[N]) {
    if (vec && left >= N) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            float x[4];
            Elem<4>::unpack(*reinterpret_cast<const uint4*>(q + i * 4), x);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i + k] = x[k];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < left ? Elem<4>::get(q + i * 4) : 0.0f;
    }
}

// A thread's share, N = FT / 16 neighbours, of an FT x 16 operand tile.  ALONG_R: r is contiguous; else the tile index is.
template <bool ALONG_R, int N>
__device__ __forceinline__ void load_part(const unsigned char* base, long long pitch, long long i0, long long i_end, long long r0,
                                          long long r_end, bool vec, float (&v)[N]) {
    constexpr int kLine = 16 / N;                // threads for a line along r
    const int t = threadIdx.x;
    const long long i = i0 + (ALONG_R ? t / kLine : (t & 15) * N), r = r0 + (ALONG_R ? t % kLine * N : t >> 4);
    const long long left = ALONG_R ? (i < i_end ? r_end - r : 0) : (r < r_end ? i_end - i : 0);
    load_some<N>(base + (ALONG_R ? i * pitch + r : r * pitch + i) * 4, (int)min(max(left, 0LL), (long long)N), vec, v);
}

template <bool ALONG_R, int N> __device__ __forceinline__ void store_part(float (*s)[N * 16 + kFPad], const float (&v)[N]) {
    constexpr int kLine = 16 / N;
    const int t = threadIdx.x;
    if (ALONG_R) {
#pragma unroll
        for (int k = 0; k < N; ++k) s[t % kLine * N + k][t / kLine] = v[k];
    } else {
        float4* d = reinterpret_cast<float4*>(&s[t >> 4][(t & 15) * N]);
#pragma unroll
        for (int k = 0; k < N / 4; ++k) d[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    }
}

template <int MODE, int FT> __global__ void __launch_bounds__(kFThreads, 2) k_fma(const Product p) {
    constexpr int N = FT / 16, H = FT / 64;      // of a thread: elements of an operand tile; lots of 4 rows and of 4 columns
    constexpr bool A_R = MODE != kGradWeight, B_R = MODE == kForward;
    __shared__ __align__(16) float sa[2][kFK][FT + kFPad];
    __shared__ __align__(16) float sb[2][kFK][FT + kFPad];
    const int t = threadIdx.x;
    int w = 0;
    long long i0, i1, r0 = 0, r1 = p.R;
    const long long j0 = (long long)blockIdx.x * FT;
    if (MODE == kGradWeight) {
        w = blockIdx.z;
        i0 = (long long)blockIdx.y * FT;
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
            tiles[t] = (int)((b - a + FT - 1) / FT);
            __syncthreads();
            for (int k = 0; k < kFThreads && w0 + k < p.N; ++k) {
                if (blockIdx.y < before + tiles[k]) { w = w0 + k; found = true; break; }
                before += tiles[k];
            }
            __syncthreads();
        }
        if (!found) return;
        rows_of(p, w, i0, i1);
        i0 += ((long long)blockIdx.y - before) * FT;
    }
    const unsigned char* a = p.a;
    const unsigned char* b = MODE == kGradWeight ? p.b : p.b + w * p.stride * 4;
    f32x2 acc[4 * H][2 * H];
#pragma unroll
    for (int i = 0; i < 4 * H; ++i)
#pragma unroll
        for (int j = 0; j < 2 * H; ++j) acc[i][j] = 0;
    const int ti = t >> 4, tj = t & 15;
    float va[N], vb[N];
    int s = 0;
    if (r0 < r1) {
        load_part<A_R>(a, p.a_pitch, i0, i1, r0, r1, p.a_vec, va);
        load_part<B_R>(b, p.b_pitch, j0, p.J, r0, r1, p.b_vec, vb);
        store_part<A_R>(sa[0], va);
        store_part<B_R>(sb[0], vb);
    }
    __syncthreads();
    for (long long r = r0; r < r1; r += kFK) {
        const bool more = r + kFK < r1;
        if (more) {
            load_part<A_R>(a, p.a_pitch, i0, i1, r + kFK, r1, p.a_vec, va);
            load_part<B_R>(b, p.b_pitch, j0, p.J, r + kFK, r1, p.b_vec, vb);
        }
#pragma unroll
        for (int k = 0; k < kFK; ++k) {
            float xs[4 * H];
            f32x2 ys[2 * H];
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const float4 x = *reinterpret_cast<const float4*>(&sa[s][k][h * 64 + ti * 4]);
                const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(&sb[s][k][h * 64 + tj * 4]);
                xs[4 * h] = x.x; xs[4 * h + 1] = x.y; xs[4 * h + 2] = x.z; xs[4 * h + 3] = x.w;
                ys[2 * h] = y.x; ys[2 * h + 1] = y.y;
            }
#pragma unroll
            for (int i = 0; i < 4 * H; ++i) {
                const f32x2 xx = pair(xs[i], xs[i]);
#pragma unroll
                for (int j = 0; j < 2 * H; ++j) acc[i][j] = fma2(xx, ys[j], acc[i][j]);
            }
        }
        if (more) {
            store_part<A_R>(sa[s ^ 1], va);
            store_part<B_R>(sb[s ^ 1], vb);
        }
        __syncthreads();
        s ^= 1;
    }
    unsigned char* c = MODE == kGradWeight ? p.c + w * p.stride * 4 : p.c;
#pragma unroll
    for (int i = 0; i < 4 * H; ++i) {
        const long long row = i0 + (i >> 2) * 64 + ti * 4 + (i & 3);
        if (row >= i1) continue;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const long long col = j0 + h * 64 + tj * 4;
            unsigned char* q = c + (row * p.c_pitch + col) * 4;
            const float v[4] = {lo_of(acc[i][2 * h]), hi_of(acc[i][2 * h]), lo_of(acc[i][2 * h + 1]), hi_of(acc[i][2 * h + 1])};
            if (p.c_vec && col + 4 <= p.J) {
                *reinterpret_cast<float4*>(q) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (col + k < p.J) Elem<4>::put(q + k * 4, v[k]);
            }
        }
    }
}

// ---------------------------------------------------------------- tensor cores
// bfloat16 operands.  The weights' index is the height of the product (128 CG outputs), the
// ragged rows its width: a worker's rows are cut evenly into tiles of at most p.width, and the width of a product can
// be any multiple of 16 CG, so that ragged rows cost at most 16 CG - 1 idle columns a worker, not half a tile.
//
//              height i                       width j                    summed r
//   forward    n: W, along r                  rows: X, along r           k
//   grad rows  k: W, along i                  rows: dY, along r          n
//   grad w.    n: dY, along i                 k: X, along j              rows (ragged)
//
// Persistent CTAs; two warps that issue TMA loads, one for either operand, into a ring of stages of 64 values of r, a
// warp that issues the products, four warps that take finished accumulators out of TMEM (two of them there, 256 columns
// each, so that the next tile's products run meanwhile), turn them through shared memory and store them.  The last rows
// of a worker in the gradient of the weights: what the load brought beyond them is zeroed in shared memory before the
// products see it, by a warp of its own in a stage of its own (another worker's NaN would not vanish by being multiplied with zero).
//
// The tensor cores truncate each addition of 16 products to the accumulator, towards zero: over terms of one sign the
// error grows faster than their number, 8e-7 of the sum after 1000 terms, 8e-6 after 4096, 3e-4 after 65536.  A sum of more
// than kPartSteps stages is therefore cut into parts of that many, formed one after another in the first accumulator and
// added with rounding, by the warps that take results, to the second one, which such a tile has to itself: 8e-6 whatever the
// length.  Measured (whole / in parts): gradient of the weights 1024 x 1024 into floats, 4 x 16384 rows 135 / 138 us, 16 x 5000
// 138 / 156; forward 16 x 500 rows, 8192 -> 1024: 139 / 148.  Parts of 2048 would leave 2e-6 and catch sums of 4096.
using namespace combo_tc;

__device__ int g_linear_status;              // 0, or the site of the first wait that gave up
__device__ __forceinline__ bool give_up(int site) {
    atomicCAS(&g_linear_status, 0, site);
    return false;
}

constexpr int kOutWarps = 4;                 // one for each quarter of TMEM's lanes (eight were no faster)
constexpr int kFirstOutWarp = 4;
constexpr int kLoadWarps = 16;               // where threads load: warps behind those, two sets of eight
constexpr int tc_threads(bool by_threads) { return 32 * (kFirstOutWarp + kOutWarps + (by_threads ? kLoadWarps : 0)); }
constexpr int kStep = 64;                    // values of r in a stage
constexpr int kOperandA = 128 * kStep * 2;   // bytes of the height's operand in a stage
constexpr int kRowBoxes = 4;                 // boxes of 32, 64, 128 or 256 rows of X or dY
constexpr int kMaxStages = 8;
constexpr int kPartSteps = 64;               // stages of r that the tensor cores sum by themselves: 4096 values
constexpr int kTurn = 32 * 33 * 4;           // bytes in which an epilogue warp turns 32 x 32 outputs
constexpr int kTmemColumns = 512;
constexpr int kStaticSmem = 1024;           // room for the kernel's barriers

struct TcParams {
    Product p;
    int width;                               // widest tile along j
    int stages, stage_bytes;
    int a_blocks, b_blocks;                  // whether an operand along i or j comes by a map of blocks of 64, in one copy; else a copy a block
};
// Tensor maps: the height's operand; the width's, by the rows of a box (one map in the gradient of the weights)
struct alignas(64) TcMaps {
    CUtensorMap a, b[kRowBoxes];
};

// One tile of the grid's work, and how far the ring has gone.
struct Tile {
    int w;                                   // worker
    long long row0, row1;                    // its rows: of the tile (forward, rows' gradient), or all that are summed
    int i0, j0, n;                           // outputs; n = the product's width
    int steps;                               // stages of r
};

// Walks the tiles t, t + stride, ... in order, workers 32 at a time.  The whole warp.
template <int CG, int MODE> struct Tiles {
    const TcParams& q;
    int t, lane, w0, mt, jt;
    int incl, total, before;                 // tiles of the lane's worker and those before it in the lot; of the lot; before the lot
    __device__ __forceinline__ Tiles(const TcParams& q_, int first) : q(q_), t(first) {
        lane = threadIdx.x & 31;
        mt = (q.p.I + 128 * CG - 1) / (128 * CG);
        jt = (q.p.J + q.width - 1) / q.width;
        w0 = before = total = incl = 0;
        if (MODE != kGradWeight) lot();
    }
    __device__ __forceinline__ void lot() {
        long long a = 0, b = 0;
        if (w0 + lane < q.p.N) rows_of(q.p, w0 + lane, a, b);
        incl = (int)((b - a + q.width - 1) / q.width) * mt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        total = __shfl_sync(0xffffffffu, incl, 31);
    }
    __device__ __forceinline__ bool next(Tile& x, int stride) {
        if (MODE == kGradWeight) {
            const int per = mt * jt;
            if (t >= per * q.p.N) return false;
            x.w = t / per;
            const int k = t - x.w * per;
            x.i0 = (k % mt) * 128 * CG;
            x.j0 = (k / mt) * q.width;
            x.n = q.width;
            rows_of(q.p, x.w, x.row0, x.row1);
            x.steps = (int)((x.row1 - x.row0 + kStep - 1) / kStep);
        } else {
            while (t >= before + total) {
                before += total;
                w0 += 32;
                if (w0 >= q.p.N) return false;
                lot();
            }
            const unsigned m = __ballot_sync(0xffffffffu, incl > t - before);
            const int k = __ffs(m) - 1;
            const int end = __shfl_sync(0xffffffffu, incl, k), prev = __shfl_sync(0xffffffffu, incl, k > 0 ? k - 1 : 0);
            const int start = k > 0 ? prev : 0, at = t - before - start, tiles = (end - start) / mt;
            x.w = w0 + k;
            long long a, b;
            rows_of(q.p, x.w, a, b);
            const int even = (int)((b - a + tiles - 1) / tiles);
            x.n = (even + 16 * CG - 1) / (16 * CG) * (16 * CG);
            x.i0 = (at % mt) * 128 * CG;
            x.j0 = (at / mt) * x.n;
            x.row0 = a + x.j0;
            x.row1 = min(x.row0 + x.n, b);
            x.steps = (q.p.R + kStep - 1) / kStep;
        }
        t += stride;
        return true;
    }
};

// Whose turn it is of the two accumulators, alike in the warp that issues products and in those that take results.  Tiles take
// them in turn; one whose sum is cut into parts takes both, and the tile behind it waits for the first.
struct Turns {
    uint32_t buf = 0, uses = 0;              // the tile's accumulator (its first); bit b: whether that of accumulator b is odd
    // parts of the tile's sum (none where no row is summed)
    __device__ __forceinline__ int begin(const Tile& x) {
        if (x.steps > kPartSteps) buf = 0;
        return (x.steps + kPartSteps - 1) / kPartSteps;
    }
    __device__ __forceinline__ uint32_t parity(int part) const { return (uses >> buf ^ (uint32_t)part) & 1u; }
    __device__ __forceinline__ void end(int parts) {
        uses ^= (uint32_t)(parts & 1) << buf;
        buf = parts == 0 ? buf : parts == 1 ? buf ^ 1u : 0u;
    }
};

// Zeroes lines [left, next multiple of 16) of `blocks` blocks of 64 lines of 128 bytes; a warp.
__device__ __forceinline__ void zero_tail(uint32_t at, int blocks, int left, int lane) {
    const int words = ((left + 15) / 16 * 16 - left) * 8;
    for (int block = 0; block < blocks; ++block)
        for (int o = lane; o < words; o += 32)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + block * 64 * kStep * 2 + left * 128 + o * 16), "r"(0u) : "memory");
    fence_async();
    __syncwarp();
}

// Loads by threads, for operands that TMA cannot take (bases, pitches or strides that are no multiples of 16 bytes).  A
// warp brings lines of 64 values, a 32-bit word a lane; where a line begins in the middle of a word, each lane joins
// halves of its own and its neighbour's.  (A word that the line's first or last value shares is read whole: 2 bytes of
// the same aligned word.)  Lines and values that are not the operand's are zero, so nothing is left to be zeroed after.
// A set of eight warps takes a lot of three blocks of 64 lines at once, so that a whole stage is under way together.  (One
// set that asked for its next lot before storing the one at hand was slower: what bounds is the issue of the joining.)
struct Lot {
    uint32_t w[24];              // a warp's words: line u * 8 + wl of block gi in w[gi * 8 + u]
    uint32_t odd, end;           // lines that begin in the middle of a word; of lane e, the value behind line e's last whole word
    int valid[3], lines[3];      // values of a line, lines of a warp
};
// blocks g0 .. g0 + 2 of stage k: two of the height's operand, then the width's
template <int MODE> __device__ __forceinline__ void load_lot(Lot& t, const Product& p, const Tile& x, int k, int g0, int blocks, int wl, int lane) {
    constexpr bool A_R = MODE == kForward, B_R = MODE != kGradWeight;
    const unsigned char* wa = MODE == kGradWeight ? p.a : p.b + x.w * p.stride * 2;
    const unsigned char* wb = MODE == kGradWeight ? p.b : p.a;
    const long long pa = MODE == kGradWeight ? p.a_pitch : p.b_pitch, pb = MODE == kGradWeight ? p.b_pitch : p.a_pitch;
    // first value of the stage along r and the end of r; an operand along r has its lines along its own index
    const long long r0 = MODE == kGradWeight ? x.row0 + (long long)k * kStep : (long long)k * kStep;
    const long long r_end = MODE == kGradWeight ? x.row1 : p.R;
    t.odd = t.end = 0;
#pragma unroll
    for (int gi = 0; gi < 3; ++gi) {
        const int g = g0 + gi;
        const bool height = g < 2;
        const int block = height ? g : g - 2;
        const bool along_r = height ? A_R : B_R;
        const long long index0 = height ? x.i0 : MODE == kGradWeight ? x.j0 : x.row0;        // of the operand's own index
        const long long index_end = height ? p.I : MODE == kGradWeight ? p.J : x.row1;
        const long long line0 = along_r ? index0 + block * 64 + wl : r0 + wl, line_end = along_r ? index_end : r_end;
        const long long col0 = along_r ? r0 : index0 + block * 64, col_end = along_r ? r_end : index_end;
        const int valid = g < blocks ? (int)min(max(col_end - col0, 0LL), 64LL) : 0;
        const int lines = (int)min(max((line_end - line0 + 7) / 8, 0LL), 8LL);
        t.valid[gi] = valid;
        t.lines[gi] = lines;
        const long long step = (height ? pa : pb) * 16;
        const unsigned char* q = (height ? wa : wb) + line0 * (step / 8) + col0 * 2;
        if (lane >> 3 == gi && valid == 64 && (lane & 7) < lines) {
            const unsigned char* mine = q + (lane & 7) * step;
            if (reinterpret_cast<uintptr_t>(mine) & 2u) t.end = __ldg(reinterpret_cast<const unsigned short*>(mine + 126));
        }
#pragma unroll
        for (int u = 0; u < 8; ++u, q += step) {
            const int e = gi * 8 + u, half = (int)(reinterpret_cast<uintptr_t>(q) >> 1 & 1u);
            const uint32_t* word = reinterpret_cast<const uint32_t*>(q - 2 * half) + lane;
            t.w[e] = u < lines && 2 * lane - half < valid && valid > 0 ? __ldg(word) : 0u;
            t.odd |= (uint32_t)half << e;
        }
    }
}
template <int MODE> __device__ __forceinline__ void store_lot(const Lot& t, const Tile& x, int g0, int blocks, uint32_t stage, int wl, int lane) {
    constexpr bool B_R = MODE != kGradWeight;
#pragma unroll
    for (int gi = 0; gi < 3; ++gi) {
        const int g = g0 + gi;
        if (g >= blocks) break;
        const uint32_t to = stage + (g < 2 ? g * 64 * kStep * 2 : kOperandA + (g - 2) * 64 * kStep * 2) + wl * 128 + ((lane * 4) ^ (wl << 4));
        const uint32_t keep = (2 * lane < t.valid[gi] ? 0xffffu : 0u) | (2 * lane + 1 < t.valid[gi] ? 0xffff0000u : 0u);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int e = gi * 8 + u;
            uint32_t v = t.w[e];
            if (t.odd >> e & 1u) {               // the same for the whole warp
                uint32_t next = __shfl_down_sync(0xffffffffu, v, 1);
                const uint32_t behind = __shfl_sync(0xffffffffu, t.end, e);
                if (lane == 31) next = behind;
                v = __funnelshift_r(v, next, 16);
            }
            v &= u < t.lines[gi] ? keep : 0u;
            // the width's operand along r has x.n lines
            if (g < 2 || !B_R || (g - 2) * 64 + wl + u * 8 < x.n)
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + u * 1024), "r"(v) : "memory");
        }
    }
}

template <int CG, int MODE, int OB, bool THREADS>
__global__ void __launch_bounds__(tc_threads(THREADS), 1) k_tc(const TcParams q, const __grid_constant__ TcMaps maps) {
    constexpr bool A_R = MODE == kForward, B_R = MODE != kGradWeight;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 7];
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
    // the stage behind the ring, for the rows of a tile's end (gradient of the weights): loaded, zeroed, free
    const uint32_t tail_full = bar0 + 8 * (2 * kMaxStages + 4), tail_ready = tail_full + 8, tail_empty = tail_full + 16;
    const uint32_t tail_at = smem + q.stages * q.stage_bytes;
    if (threadIdx.x == 0) {
        for (int s = 0; s < q.stages; ++s) {
            // one arrival for either operand, and the bytes of all CTAs; or one for each warp that loads
            mbar_init(full(s), THREADS ? kLoadWarps : 2);
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), kOutWarps * CG);
        }
        mbar_init(tail_full, 2);             // of this CTA alone
        mbar_init(tail_ready, CG);           // the leader's: from either CTA
        mbar_init(tail_empty, 1);
        mbar_init_fence();
        dead = 0;
        if (!THREADS) prefetch_map(&maps.a);
    }
    if (warp == 1) tmem_alloc<CG>(smem_u32(&tmem_at), kTmemColumns);
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
    Tile x;

    if (THREADS && warp >= kFirstOutWarp + kOutWarps) {
        // ------------------------------------------------------------ loads by threads
        Tiles<CG, MODE> tiles(q, first);
        // two sets of three blocks: six, the most there are
        const int set = (warp - kFirstOutWarp - kOutWarps) >> 3, wl = (warp - kFirstOutWarp - kOutWarps) & 7;
        uint32_t s = 0, ph = 0;
        bool ok = true;
        while (ok && tiles.next(x, stride)) {
            const int blocks = 2 + (x.n + 63) / 64;
            for (int k = 0; k < x.steps && ok; ++k) {
                Lot t;
                load_lot<MODE>(t, q.p, x, k, set * 3, blocks, wl, lane);
                ok = mbar_wait(empty(s), ph ^ 1u, dead_v) || give_up(49);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                store_lot<MODE>(t, x, set * 3, blocks, smem + s * q.stage_bytes, wl, lane);
                fence_async();
                __syncwarp();
                if (elect()) mbar_arrive(full(s));
                __syncwarp();
                if (++s == (uint32_t)q.stages) { s = 0; ph ^= 1u; }
            }
        }
        if (!ok) *dead_v = 1;
    } else if (!THREADS && (warp == 0 || warp == 2)) {
        // ------------------------------------------------------------ loads: warp 0 the height's operand, warp 2 the width's
        const int operand = warp == 0 ? 0 : 1;
        Tiles<CG, MODE> tiles(q, first);
        uint32_t done = 0, tails = 0;        // stages of the ring issued; tiles with an end of their own
        const uint32_t bar_leader = CG == 1 ? full(0) : at_leader(full(0));
        bool ok = true;
        while (tiles.next(x, stride)) {
            const int half = x.n / CG;       // of the width: this CTA's share
            int bytes = kOperandA;           // of a stage
            const CUtensorMap* map = &maps.a;
            const bool blocks = operand == 0 ? q.a_blocks : q.b_blocks;
            if (operand == 1 && MODE == kGradWeight) {
                bytes = half * kStep * 2;
                map = &maps.b[0];
            } else if (operand == 1) {
                const int m = half <= 32 ? 0 : half <= 64 ? 1 : half <= 128 ? 2 : 3;
                bytes = (32 << m) * kStep * 2;
                map = &maps.b[m];
            }
            const int at = operand == 0 ? x.i0 + rank * 128 : MODE == kGradWeight ? x.j0 + rank * half : (int)x.row0 + rank * half;
            // the last rows, if some of a 16 are another's: they go to a stage of their own, where a warp zeroes the others,
            // and are asked for as soon as that stage is sure to be free, when the ring has come round to this tile
            const int rest = MODE == kGradWeight ? (int)((x.row1 - x.row0) % kStep) : 0;
            const int plain = rest % 16 != 0 ? x.steps - 1 : x.steps;
            const int ahead = plain < x.steps ? min(plain, q.stages) : -1;
            uint32_t s = done % q.stages, ph = done / q.stages & 1u;
            const auto load = [&](int k, uint32_t to, uint32_t bar) {
                const int r = MODE == kGradWeight ? (int)x.row0 + k * kStep : k * kStep;
                to += operand * kOperandA;
                if (operand == 0 && MODE == kForward) tma_3d<CG>(to, map, r, at, x.w, bar);
                else if (operand == 1 && MODE != kGradWeight) tma_2d<CG>(to, map, r, at, bar);
                else if (blocks && MODE == kGradInput) tma_4d<CG>(to, map, 0, r, at / 64, x.w, bar);
                else if (blocks) tma_3d<CG>(to, map, 0, r, at / 64, bar);
                else
                    for (int c = 0; c * 64 * kStep * 2 < bytes; ++c) {
                        if (MODE == kGradInput) tma_3d<CG>(to + c * 64 * kStep * 2, map, at + c * 64, r, x.w, bar);
                        else tma_2d<CG>(to + c * 64 * kStep * 2, map, at + c * 64, r, bar);
                    }
            };
            if (elect()) {
                for (int k = 0; k <= plain; ++k) {
                    if (MODE == kGradWeight && k == ahead) {
                        if (!mbar_wait(tail_empty, tails & 1u ^ 1u, dead_v)) { ok = give_up(42); break; }
                        mbar_arrive_expect(tail_full, bytes);
                        load(plain, tail_at, tail_full);
                    }
                    if (k == plain) break;
                    if (!mbar_wait(empty(s), ph ^ 1u, dead_v)) { ok = give_up(40); break; }
                    // the leader expects the bytes of both CTAs; the other one's may come before
                    if (rank == 0) mbar_arrive_expect(full(s), bytes * CG);
                    load(k, smem + s * q.stage_bytes, bar_leader + 8 * s);
                    if (++s == q.stages) { s = 0; ph ^= 1u; }
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            done += plain;
            if (plain < x.steps) ++tails;
        }
        if (!ok) {
            // after a wait that gave up nothing tells when the copies under way have landed: far longer than they take
            *dead_v = 1;
            for (int k = 0; k < 2000; ++k) __nanosleep(1000);
        }
        // No copy may be under way when the CTA leaves: the products have freed the last stages.
        for (uint32_t k = 1; k <= done && k <= (uint32_t)q.stages && ok; ++k)
            ok = mbar_wait(empty((done - k) % q.stages), (done - k) / q.stages & 1u, dead_v) || give_up(43);
        if (ok && tails > 0 && !mbar_wait(tail_empty, (tails - 1) & 1u, dead_v)) {
            give_up(48);
            *dead_v = 1;
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ products, by one thread of the leader
        if (rank == 0) {
            Tiles<CG, MODE> tiles(q, first);
            uint32_t done = 0, tails = 0;
            Turns turns;
            bool ok = true;
            while (tiles.next(x, stride)) {
                if (x.steps == 0) continue;
                const int parts = turns.begin(x);
                const uint32_t buf = turns.buf;
                const int rest = MODE == kGradWeight ? (int)((x.row1 - x.row0) % kStep) : 0;
                const int plain = !THREADS && rest % 16 != 0 ? x.steps - 1 : x.steps;
                if (elect()) {
                    const uint32_t d = tmem + buf * 256, kind = product_kind(128 * CG, x.n, A_R, B_R);
                    uint32_t s = done % q.stages, ph = done / q.stages & 1u;
                    const auto issue = [&](uint32_t a, int n16, bool add) {
                        const uint64_t da = operand(a, A_R, 64 * kStep * 2), db = operand(a + kOperandA, B_R, 64 * kStep * 2);
#pragma unroll
                        for (int c = 0; c < kStep / 16; ++c)
                            if (MODE != kGradWeight || c < n16)
                                mma<CG>(d, da + (uint64_t)(c * step16(A_R) >> 4), db + (uint64_t)(c * step16(B_R) >> 4), kind, add || c > 0);
                    };
                    for (int part = 0; part < parts && ok; ++part) {
                        const int k0 = part * kPartSteps, k1 = min(k0 + kPartSteps, x.steps);
                        if (!mbar_wait(acc_empty(buf), turns.parity(part) ^ 1u, dead_v)) { ok = give_up(44); break; }
                        tc_fence_after();
                        for (int k = k0; k < min(k1, plain); ++k) {
                            if (!mbar_wait(full(s), ph, dead_v)) { ok = give_up(45); break; }
                            tc_fence_after();
                            issue(smem + s * q.stage_bytes, k + 1 == x.steps && rest ? (rest + 15) / 16 : kStep / 16, k > k0);
                            mma_commit<CG>(empty(s));
                            if (++s == q.stages) { s = 0; ph ^= 1u; }
                        }
                        if (MODE == kGradWeight && plain < k1 && ok) {
                            // zeros that threads of both CTAs have written
                            if (CG == 1 ? mbar_wait(tail_ready, tails & 1u, dead_v) : mbar_wait_cluster(tail_ready, tails & 1u, dead_v)) {
                                tc_fence_after();
                                issue(tail_at, (rest + 15) / 16, plain > k0);
                                mma_commit<CG>(tail_empty);
                            } else {
                                ok = give_up(46);
                            }
                        }
                        if (ok) mma_commit<CG>(acc_full(buf));
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                done += plain;
                if (plain < x.steps) ++tails;
                turns.end(parts);
            }
            if (!ok) *dead_v = 1;
        }
    } else if (warp == 3) {
        // ------------------------------------------------------------ rows of others, zeroed
        if (MODE == kGradWeight && !THREADS) {
            Tiles<CG, MODE> tiles(q, first);
            uint32_t tails = 0;
            bool ok = true;
            while (tiles.next(x, stride)) {
                const int rest = (int)((x.row1 - x.row0) % kStep);
                if (rest % 16 == 0) continue;
                ok = mbar_wait(tail_full, tails & 1u, dead_v) || give_up(41);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                ++tails;
                zero_tail(tail_at, 2 + x.n / CG / 64, rest, lane);
                if (elect()) {
                    if (rank == 0) mbar_arrive(tail_ready);
                    else mbar_arrive_release(at_leader(tail_ready));
                }
                __syncwarp();
            }
            if (!ok) *dead_v = 1;
        }
    } else if (warp >= kFirstOutWarp && warp < kFirstOutWarp + kOutWarps) {
        // ------------------------------------------------------------ results
        Tiles<CG, MODE> tiles(q, first);
        const int quarter = warp & 3;        // a warp reads the 32 lanes of TMEM that its number allows
        float* turn = reinterpret_cast<float*>(smem_raw + (smem - smem_u32(smem_raw)) + (q.stages + (MODE == kGradWeight && !THREADS ? 1 : 0)) * q.stage_bytes + quarter * kTurn);
        Turns turns;
        bool ok = true;
        while (tiles.next(x, stride)) {
            const int i = x.i0 + rank * 128 + quarter * 32;
            const bool any = x.steps > 0;
            const int parts = turns.begin(x);
            const uint32_t buf = turns.buf, lanes = tmem + ((uint32_t)(quarter * 32) << 16);
            const int columns = i < q.p.I ? MODE == kGradWeight ? min(x.n, q.p.J - x.j0) : (int)(x.row1 - x.row0) : 0;
            const auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(CG == 1 ? acc_empty(buf) : at_leader(acc_empty(buf)));
            };
            for (int part = 0; part < parts; ++part) {
                ok = mbar_wait(acc_full(buf), turns.parity(part), dead_v) || give_up(47);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_fence_after();
                if (parts == 1) break;
                for (int c0 = 0; c0 < columns; c0 += 16) tmem_fold16(lanes + c0, lanes + 256 + c0, part > 0);
                tmem_store_wait();
                // the last part's accumulator goes with the sums, which the next tile but one may overwrite
                if (part + 1 < parts) release();
            }
            if (!ok) break;
            unsigned char* c = MODE == kGradWeight ? q.p.c + x.w * q.p.stride * OB : q.p.c;
            if (columns > 0) {
                // lots of 32 columns; the next lot's load is under way while this one is stored
                const uint32_t acc = lanes + (parts > 1 ? 256 : buf * 256);
                uint32_t next[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) next[e] = 0u;
                if (any) tmem_load32(acc, next);
                for (int c0 = 0; c0 < columns; c0 += 32) {
                    uint32_t v[32];
                    if (any) tmem_load_wait(next);
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = next[e];
                    if (any && c0 + 32 < columns) tmem_load32(acc + c0 + 32, next);
                    // 33 floats to a line: neither the writes nor the reads meet on a bank
#pragma unroll
                    for (int e = 0; e < 32; ++e) turn[MODE == kGradWeight ? lane * 33 + e : e * 33 + lane] = __uint_as_float(v[e]);
                    __syncwarp();
                    // out(line, col) is the result at (row0 + line, col0 + col)
                    const long long row0 = MODE == kGradWeight ? (long long)i : x.row0 + c0, row_end = MODE == kGradWeight ? (long long)q.p.I : x.row1;
                    const int col0 = MODE == kGradWeight ? x.j0 + c0 : i, col_end = MODE == kGradWeight ? q.p.J : q.p.I;
                    if (q.p.c_vec && col0 + 32 <= col_end) {
                        // a lane stores 16 bytes, neighbours what lies beside it
                        constexpr int kLane = 16 / OB, kPerLine = 32 / kLane;
#pragma unroll
                        for (int e = 0; e < kPerLine; ++e) {
                            const int line = e * (32 / kPerLine) + lane / kPerLine, col = lane % kPerLine * kLane;
                            float o[kLane];
#pragma unroll
                            for (int f = 0; f < kLane; ++f) o[f] = turn[line * 33 + col + f];
                            if (row0 + line < row_end)
                                *reinterpret_cast<uint4*>(c + ((row0 + line) * q.p.c_pitch + col0 + col) * OB) = Elem<OB>::pack(o);
                        }
                    } else if (col0 + lane < col_end) {
                        // off 16-byte boundaries, or at the end of the lines: a line a store
                        unsigned char* to = c + (row0 * q.p.c_pitch + col0 + lane) * OB;
                        const int lines = (int)min(row_end - row0, 32LL);
#pragma unroll 8
                        for (int line = 0; line < lines; ++line, to += q.p.c_pitch * OB) Elem<OB>::put(to, turn[line * 33 + lane]);
                    }
                    __syncwarp();
                }
            }
            if (any) release();
            turns.end(parts);
        }
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

// ---------------------------------------------------------------- host
template <int FT> cudaError_t launch_fma(const Product& p, int mode, cudaStream_t st) {
    combo_host::set_step_path(combo_host::kPathMultiplyAdd);
    const unsigned cols = (unsigned)((p.J + FT - 1) / FT);
    if (mode == kGradWeight) {
        const dim3 grid(cols, (unsigned)((p.I + FT - 1) / FT), (unsigned)p.N);
        k_fma<kGradWeight, FT><<<grid, kFThreads, 0, st>>>(p);
    } else {
        // every worker adds less than one tile to those its rows fill
        const long long tiles = p.M / FT + (p.N < p.M ? p.N : p.M);
        const dim3 grid(cols, (unsigned)(tiles < 1 ? 1 : tiles));
        if (mode == kForward) k_fma<kForward, FT><<<grid, kFThreads, 0, st>>>(p);
        else k_fma<kGradInput, FT><<<grid, kFThreads, 0, st>>>(p);
    }
    return cudaGetLastError();
}

// Tensor map of bfloat16 rows, `pitch` apart, in `layers` lots `stride` apart (0: none); boxes of 64 elements by `rows_box`
// rows.  blocks > 0: boxes of that many times 64 elements, laid out block after block (width a multiple of 64).
bool encode(CUtensorMap* map, const void* base, long long width, long long rows, long long pitch, int layers, long long stride,
            int rows_box, int blocks) {
    cuuint64_t dims[4], strides[3];
    cuuint32_t box[4], ones[4] = {1, 1, 1, 1};
    int n = 0;
    const auto add = [&](long long dim, long long step, int b) {
        dims[n] = (cuuint64_t)dim;
        if (n > 0) strides[n - 1] = (cuuint64_t)step * 2;
        box[n++] = (cuuint32_t)b;
    };
    add(blocks ? kStep : width, 1, kStep);
    add(rows, pitch, rows_box);
    if (blocks) add(width / kStep, kStep, blocks);
    if (layers) add(layers, stride ? stride : 8, 1);
    return combo_host::encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, n, const_cast<void*>(base), dims, strides, box, ones,
                                    CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int CG, int MODE, int OB, bool THREADS> cudaError_t launch_tc_inst(const TcParams& q, const TcMaps& maps, int smem_most, int grid, cudaStream_t st) {
    static uint64_t allowed;
    auto kern = k_tc<CG, MODE, OB, THREADS>;
    const size_t smem = 1024 + (size_t)(q.stages + (MODE == kGradWeight && !THREADS ? 1 : 0)) * q.stage_bytes + kOutWarps * kTurn;
    cudaError_t e = combo_host::allow_smem(kern, smem_most, &allowed);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(tc_threads(THREADS));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CG;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, q, maps);
}

template <int CG, bool THREADS> combo_status launch_tc(const Product& p, int mode, int out_bytes, int sms, int smem_optin, cudaStream_t st) {
    TcParams q = {p, 256, 0, 0, 0, 0};
    combo_host::set_step_path(THREADS ? combo_host::kPathTensorThreads : CG == 2 ? combo_host::kPathTensorPairs : combo_host::kPathTensor);
    // the height is W's (forward: n_out, rows' gradient: n_in) or n_out; see the table above
    const long long mt = (p.I + 128 * CG - 1) / (128 * CG);
    long long tiles;
    if (mode == kGradWeight) {
        const int least = 64 * CG;
        while (q.width > least && (q.width / 2 >= p.J || mt * ((p.J + q.width - 1) / q.width) * p.N * CG < sms)) q.width /= 2;
        tiles = mt * ((p.J + q.width - 1) / q.width) * p.N;
    } else {
        // the host knows the workers' rows on average only
        const long long mean = (p.M + p.N - 1) / p.N;
        const auto count = [&](int width) { return mt * p.N * ((mean + width - 1) / width); };
        while (q.width > 32 * CG && (q.width >= 4 * mean || count(q.width) * CG < sms)) q.width /= 2;
        tiles = mt * (p.M / q.width + (p.N < p.M ? p.N : p.M));
    }
    if (tiles > 0x40000000LL) return COMBO_ERR_INVALID_ARG;
    const int half = q.width / CG;
    q.stage_bytes = kOperandA + half * kStep * 2;
    q.stages = (smem_optin - kStaticSmem - 1024 - kOutWarps * kTurn) / q.stage_bytes;
    if (mode == kGradWeight && !THREADS) --q.stages;     // one behind the ring
    if (q.stages > kMaxStages) q.stages = kMaxStages;
    int grid = sms / CG * CG;
    if (tiles * CG < grid) grid = (int)tiles * CG;
    if (grid < CG) grid = CG;
    TcMaps maps;
    memset(&maps, 0, sizeof(maps));
    bool fine = true;                            // threads load by the addresses alone
    // p.a: the rows' operand of the first kind (X, dY, dY), p.b: W, W, X.  An operand along i or j comes in blocks of 64: in
    // one copy where its width is a multiple of that, else (a block would run into the next row) in one copy a block
    if (THREADS) {
    } else if (mode == kForward) {
        fine = encode(&maps.a, p.b, p.R, p.I, p.b_pitch, p.N, p.stride, 128, 0);
    } else if (mode == kGradInput) {
        q.a_blocks = p.I % kStep == 0;
        fine = encode(&maps.a, p.b, p.I, p.R, p.b_pitch, p.N, p.stride, kStep, q.a_blocks ? 2 : 0);
    } else {
        q.a_blocks = p.I % kStep == 0;
        q.b_blocks = p.J % kStep == 0;
        fine = encode(&maps.a, p.a, p.I, p.M, p.a_pitch, 0, 0, kStep, q.a_blocks ? 2 : 0) &&
               encode(&maps.b[0], p.b, p.J, p.M, p.b_pitch, 0, 0, kStep, q.b_blocks ? half / kStep : 0);
    }
    for (int m = 0; !THREADS && mode != kGradWeight && m < kRowBoxes && (32 << m) <= half && fine; ++m)
        fine = encode(&maps.b[m], p.a, p.R, p.M, p.a_pitch, 0, 0, 32 << m, 0);
    if (!fine) return COMBO_ERR_CUDA;
    cudaError_t e;
    const int most = smem_optin - kStaticSmem;
    if (mode == kForward) e = out_bytes == 2 ? launch_tc_inst<CG, kForward, 2, THREADS>(q, maps, most, grid, st) : launch_tc_inst<CG, kForward, 4, THREADS>(q, maps, most, grid, st);
    else if (mode == kGradInput) e = out_bytes == 2 ? launch_tc_inst<CG, kGradInput, 2, THREADS>(q, maps, most, grid, st) : launch_tc_inst<CG, kGradInput, 4, THREADS>(q, maps, most, grid, st);
    else e = out_bytes == 2 ? launch_tc_inst<CG, kGradWeight, 2, THREADS>(q, maps, most, grid, st) : launch_tc_inst<CG, kGradWeight, 4, THREADS>(q, maps, most, grid, st);
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "grouped product launch");
}

bool vec_ok(const void* p, int64_t pitch, int64_t stride, int eb) {
    return combo_host::aligned_to(p, 16) && pitch * eb % 16 == 0 && stride * eb % 16 == 0;
}

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
    const combo_host::Rows r1 = {rows1, M, (size_t)width1 * elem_bytes, (size_t)pitch1 * elem_bytes};
    const combo_host::Rows r2 = {rows2, M, (size_t)width2 * eb2, (size_t)pitch2 * eb2};
    const size_t nw = ((size_t)(N - 1) * w_stride + (n_out - 1) * w_pitch + n_in) * ebw;
    const auto in_weights = [&](const combo_host::Rows& r) { return combo_host::overlap(weights, nw, r.p, r.extent()); };
    if (mode == kGradWeight ? in_weights(r1) || in_weights(r2) : combo_host::overlap(r2, r1) || in_weights(r2)) return COMBO_ERR_ALIAS;
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
    if (elem_bytes == 2) {
        Product t = p;
        if (mode != kGradWeight) t.I = p.J;      // the weights' index is the height there
        // TMA wants 16-byte bases, pitches and strides (and a row at least)
        if (!p.a_vec || !p.b_vec || M == 0) return launch_tc<1, true>(t, mode, out_bytes, sms, smem, st);
        // Pairs of CTAs halve what the tensor cores and L2 deliver for a product; a single one wastes less where there are
        // too few tiles of 256 outputs for all pairs.  Measured: 16 x 1065 rows, 1024 -> 4096: 118 us against 131; 16 rows,
        // 1024 -> 1024: no difference.
        const long long heights = (t.I + 255) / 256, widths = mode == kGradWeight ? (t.J + 255) / 256 : 1;
        if (heights * widths * N >= sms / 2) return launch_tc<2, false>(t, mode, out_bytes, sms, smem, st);
        return launch_tc<1, false>(t, mode, out_bytes, sms, smem, st);
    }
    // Tiles of 128 read shared memory half as often; those of 64 serve where 128 leave SMs idle or most of their rows.
    // Measured (128 / 64): 14 tiles of 128 (7 x 94 rows, 305 -> 144) 44 / 21 us, 64 (8 x 200, 512 -> 512) 58 / 43, 128 whole
    // ones (gradient of the weights, 512 x 512) 25 / 31, 2304 (32 x 1046, 512 -> 1000) 778 / 1106; 16 x 1 row 107 / 77.
    const long long mean = mode == kGradWeight ? p.I : (M + N - 1) / N;
    const bool narrow = (mean + 127) / 128 * ((p.J + 127) / 128) * N * 2 <= sms || mean <= 64;
    const cudaError_t e = narrow && M <= (1 << 21) ? launch_fma<64>(p, mode, st) : launch_fma<128>(p, mode, st);
    return e == cudaSuccess ? COMBO_OK : combo_host::fail(e, "grouped product launch");
}

}  // namespace

namespace combo_host {

cudaError_t grouped_linear_status(int* code) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(code, g_linear_status, sizeof(int));
    if (e == cudaSuccess && *code != 0) e = cudaMemcpyToSymbol(g_linear_status, &zero, sizeof(int));
    return e;
}

}  // namespace combo_host

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
