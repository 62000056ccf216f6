// The gated feed-forward block, forward and backward.
//
//   forward   a = x Wg^T,  b = x Wu^T,  h = act(a) b,  y = h Wd^T
//   backward  dh = dy Wd,  da = dh b act'(a),  db = dh act(a),
//             dx = da Wg + db Wu,  dWg = da^T x,  dWu = db^T x,  dWd = dy^T h
//
// Five matrix products, bound by the tensor cores for more than a few hundred tokens: forward 6 T d f
// operations, backward 12 T d f.  What is not a product is fused into the products' ends: both
// projections of a tile are accumulated side by side and meet as act(a) b before anything is
// written; dh never leaves the chip, da and db do; the three weight gradients are one launch.
//
// One kernel template serves all five.  A pair of CTAs (cta_group::2) owns a tile of 256 rows and BN
// columns, each CTA 128 of the rows; warp 0 brings 64-deep slices of both operands in by TMA, warp 1 of
// the pair's first CTA issues tcgen05.mma, eight warps bring the accumulators out of TMEM, apply
// the epilogue and store, while the next tile's products run into the other accumulator.  The
// grid is persistent: one pair for every two SMs, tiles dealt out in turn.  Transposed operands
// (Wd, Wg, Wu in the backward pass, everything in the weight gradients) are read as they lie, as
// MN-major operands; nothing is transposed in memory.
//
// B200, bfloat16, 8192 x 1600 x 6400, in a loop at the power cap: forward 400 us, with the outputs for the backward pass 429
// (1170 TFLOP/s), backward 902 (1115); the library's products alone take 415 and 897.  In short bursts 343, 368 and 756.
//
// hidden, da and db are held in the 16-bit type between the products: they are operands of the next ones, which take 16-bit
// numbers (hidden is the caller's tensor besides).  Each is rounded once, from fp32; the outputs after them are 1.4 times as far from the
// 64-bit result as with fp32 in between (bfloat16 0.0023 in place of 0.0017, float16 0.00029 in place of 0.00021, as 2-norms).
//
// Rows whose address or stride is not a multiple of 16 bytes cannot be read by TMA; they are first
// copied to padded rows in the workspace.
#include "a2sgd_tcgen05.cuh"
#include "a2sgd_train.cuh"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

using namespace a2sgd_train;
using namespace a2sgd_tc;

namespace {

constexpr int kBM = 256;                  // rows of a tile, 128 a CTA
constexpr int kBK = 64;                   // depth of a slice: 128 bytes a row
constexpr int kEpilogueWarps = 8;
constexpr int kFirstEpilogueWarp = 3; // after A's loads, the products and B's loads
constexpr int kThreads = 32 * (kFirstEpilogueWarp + kEpilogueWarps);
constexpr uint32_t kABytes = 128 * kBK * 2;  // A's slice in one CTA
constexpr uint32_t kChunk = 64 * kBK * 2;    // 64 columns of an MN-major slice
constexpr uint32_t kTmemColumns = 512;
constexpr uint32_t kStaging = 32 * 128;      // 32 rows of 64 columns on their way out: two for each epilogue warp
constexpr uint32_t kSmem = 227 * 1024;
constexpr int kMostStages = 8;
// Room for the slices: 160 KB, five stages of the widest tile.
constexpr uint32_t kOperands = (kSmem - 1024 - 512 - kEpilogueWarps * 2 * kStaging) / 1024 * 1024;

enum Epilogue { kStore = 0, kGate = 1, kGateGrad = 2 };

// CTAs whose bounded wait ran out, since the library was loaded: only ever counted up, so that no reader takes the news
// from another.  a2sgd_gated_ffn_status compares it with what was last seen from a stream.
__device__ unsigned int g_waits_run_out = 0;

// 16-bit rows that the epilogue writes, by TMA where `map` could be made, else element by element; or reads.
struct Rows {
    CUtensorMap map; // boxes of 32 rows and 64 columns
    void *p;
    int64_t ld;
    int tma;
};

struct Problem {
    int m, n;           // rows and columns of the output
    int tiles_m, tiles_n, first; // tiles down and across, and this problem's first tile
    int seg;            // operand pairs that are added up: a[seg], b[seg], ...
    int k_blocks;       // slices of all its pairs together
};

struct GemmArgs {
    CUtensorMap a[3], b[3];
    Rows out[3];        // by problem; kGate: h; kGateGrad: da
    Rows out2;          // kGate: a second copy of h, when p is set; kGateGrad: db
    Rows gate, up;      // kGate: written when p is set; kGateGrad: read
    int operands;       // pairs in use
    int seg_blocks[3];  // slices of an operand pair
    Problem problem[3];
    int problems;
    int bn;             // columns of a tile
    int box;            // B's rows in one box (K-major B)
    int stages;
    uint32_t stage_bytes;
    // Work: `whole` tiles, then the remaining ones in `splits` parts of their depth each
    int whole, items, splits;
    float *partials;    // [items - whole][bn / 4][256][4]
    // Rows that the next launch will read, brought into L2 once this one's own loads are on their way (rows 0: none)
    const void *ahead[2];
    int64_t ahead_ld;
    int ahead_rows, ahead_bytes;
};

// ------------------------------------------------------------------ activations
// value and slope of two preactivations, through p = the sigmoid of z: silu(a) = a p(a); gelu in its tanh form is
// a p(2 k (a + c a^3)).  Both saturate without a special case: exp2 overflows to infinity, whose reciprocal is 0.
// Packed arithmetic throughout, 2 special functions an element: the ends of the tiles would else take
// longer than their products (17500 clocks a tile of 256 columns when each element was computed alone,
// with the choice of the activation inside, against 14600 for 25 slices).
__device__ __forceinline__ f32x2 sigmoid_of_minus(f32x2 z_log2) // 1 / (1 + 2^z)
{
    float a, b, x, y;
    unpair(z_log2, a, b);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(a));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(b));
    unpair(add2(pair(x, y), pair(1.0f)), a, b);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(a));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(b));
    return pair(x, y);
}
template <int ACT>
__device__ __forceinline__ void activation2(f32x2 a, f32x2 &value, f32x2 &slope)
{
    constexpr float kLog2e = 1.4426950408889634f;
    if constexpr (ACT == A2SGD_ACT_SILU) {
        const f32x2 p = sigmoid_of_minus(mul2(a, pair(-kLog2e)));
        value = mul2(a, p);
        slope = fma2(value, fma2(p, pair(-1.0f), pair(1.0f)), p);
    } else {
        constexpr float k2 = 1.5957691216057308f, c = 0.044715f;
        float x, y;
        unpair(mul2(a, a), x, y);
        const f32x2 square = pair(fminf(x, 1e20f), fminf(y, 1e20f)); // beyond, p is 0 or 1 and the slope's last term 0 times this
        const f32x2 p = sigmoid_of_minus(mul2(mul2(a, pair(-k2 * kLog2e)), fma2(square, pair(c), pair(1.0f))));
        value = mul2(a, p);
        slope = fma2(mul2(value, fma2(p, pair(-1.0f), pair(1.0f))), fma2(square, pair(3.0f * c * k2), pair(k2)), p);
    }
}
template <int ACT>
__device__ __forceinline__ void gate_columns(float (&a)[32], const float (&b)[32]) // a <- act(a) b
{
#pragma unroll
    for (int k = 0; k < 32; k += 2) {
        f32x2 value, slope;
        activation2<ACT>(pair(a[k], a[k + 1]), value, slope);
        unpair(mul2(value, pair(b[k], b[k + 1])), a[k], a[k + 1]);
    }
}
template <int ACT>
__device__ __forceinline__ void gate_gradient(const float *dh, float (&a)[8], float (&b)[8]) // a <- dh b act'(a), b <- dh act(a)
{
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        f32x2 value, slope;
        activation2<ACT>(pair(a[k], a[k + 1]), value, slope);
        const f32x2 g = pair(dh[k], dh[k + 1]);
        unpair(mul2(mul2(g, pair(b[k], b[k + 1])), slope), a[k], a[k + 1]);
        unpair(mul2(g, value), b[k], b[k + 1]);
    }
}

// ------------------------------------------------------------------ staged rows
// A warp's 32 rows of 64 columns, 128 bytes a row, the 16-byte pieces of a row permuted by the row's number
// as the TMA's 128-byte swizzle does: lanes that hold a row each meet no bank twice.
__device__ __forceinline__ uint32_t piece(uint32_t buf, uint32_t row, uint32_t i) { return buf + row * 128 + ((i ^ (row & 7)) << 4); }

template <typename T>
__device__ __forceinline__ uint4 pack8(const float *v)
{
    return make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()), pack2(v[6], v[7], T()));
}
template <typename T>
__device__ __forceinline__ void unpack8(uint4 q, float (&v)[8])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = lo_f32(w[j], T());
        v[2 * j + 1] = hi_f32(w[j], T());
    }
}

// Staged rows out: one TMA store, or any alignment, 32 consecutive elements of a row at a time.  The whole warp.
__device__ __forceinline__ void rows_out(const Rows &o, uint32_t buf, int row0, int col0, int m, int n, uint32_t lane)
{
    if (o.tma) {
        fence_async();
        __syncwarp();
        if (lane == 0) {
            tma_store(&o.map, col0, row0, buf);
            tma_store_commit();
        }
    } else {
        __syncwarp();
        const int rows = min(32, m - row0), cols = min(64, n - col0), c0 = lane, c1 = lane + 32;
        uint16_t *p = static_cast<uint16_t *>(o.p) + (int64_t)row0 * o.ld + col0;
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 8) { // eight rows' reads before their writes
            uint16_t v[8][2];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                v[r][0] = ld_shared16(piece(buf, r0 + r, c0 >> 3) + (c0 & 7) * 2);
                v[r][1] = ld_shared16(piece(buf, r0 + r, c1 >> 3) + (c1 & 7) * 2);
            }
#pragma unroll
            for (int r = 0; r < 8; ++r, p += o.ld) {
                if (r0 + r < rows && c0 < cols) p[c0] = v[r][0];
                if (r0 + r < rows && c1 < cols) p[c1] = v[r][1];
            }
        }
        __syncwarp();
    }
}

// ------------------------------------------------------------------ the product
// One piece of work: a tile, all of its depth or a part of it.
struct Item {
    int p, tm, tn;      // problem, tile
    int k0, k1;         // slices
    int cols;           // columns of the product, a multiple of 32, the tile's or less at the edge
    int slot;           // of the partial sums; -1: the whole depth
};

// a / b and its remainder for a < 2^24 and quotients below 2^20: by the approximate reciprocal, put right by one.  Every
// role works out every tile, which counts where tiles are a slice or two deep (64 tokens backward 68 -> 66 us).
__device__ __forceinline__ int quick_div(int a, int b, int &rest)
{
    int q = __float2int_rz(__fdividef((float)a, (float)b));
    rest = a - q * b;
    if (rest < 0) --q, rest += b;
    if (rest >= b) ++q, rest -= b;
    return q;
}

// Tiles are walked in groups of 8 tiles down, so that the pairs at work share slices of both operands in L2.
__device__ __forceinline__ Item item_at(const GemmArgs &g, int i)
{
    Item t;
    int tile = i, part = 0;
    t.slot = -1;
    if (i >= g.whole) {
        t.slot = i - g.whole;
        tile = g.whole + quick_div(t.slot, g.splits, part);
    }
    t.p = 0;
    if (g.problems > 1 && tile >= g.problem[1].first) t.p = g.problems > 2 && tile >= g.problem[2].first ? 2 : 1;
    const Problem &q = g.problem[t.p];
    tile -= q.first;
    int rest, row;
    const int group = quick_div(tile, 8 * q.tiles_n, rest);
    t.tn = quick_div(rest, min(8, q.tiles_m - group * 8), row);
    t.tm = group * 8 + row;
    t.k0 = 0;
    t.k1 = q.k_blocks;
    if (t.slot >= 0) {
        int unused;
        t.k0 = quick_div(q.k_blocks * part, g.splits, unused);
        t.k1 = quick_div(q.k_blocks * (part + 1), g.splits, unused);
    }
    t.cols = min(g.bn, (q.n - t.tn * g.bn + 31) / 32 * 32);
    return t;
}

template <typename T, int EPI, bool A_MN, bool B_MN, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) k_gemm(const __grid_constant__ GemmArgs g)
{
    extern __shared__ char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t staging = base + kOperands;
    __shared__ __align__(8) uint64_t bars[2 * kMostStages + 4];
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int s) { return bar0 + 8u * s; };
    const auto empty = [&](int s) { return bar0 + 8u * (kMostStages + s); };
    const auto acc_full = [&](int i) { return bar0 + 8u * (2 * kMostStages + i); };
    const auto acc_empty = [&](int i) { return bar0 + 8u * (2 * kMostStages + 2 + i); };
    __shared__ uint32_t tmem_at;
    __shared__ volatile int gave_up;

    const uint32_t rank = cluster_rank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMostStages; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(acc_full(i), 1);
            bar_init(acc_empty(i), 2 * kEpilogueWarps);
        }
        gave_up = 0;
        bar_init_fence();
    }
    if (threadIdx.x >= 64 && threadIdx.x < 64 + 6) { // the maps are parameters: no need to wait for the launch before
        const int i = (threadIdx.x - 64) % 3;
        if (threadIdx.x < 67 && i < g.operands) tma_prefetch_map(&g.a[i]);
        if (threadIdx.x >= 67 && i < (EPI == kGate ? 2 : g.operands)) tma_prefetch_map(&g.b[i]);
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&tmem_at), kTmemColumns);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = tmem_at;
    wait_prior_grid();
    release_next_grid();

    if (warp == 0 || warp == 2) {
        // ---------------------------------------------------------- operands in: warp 0 A's, warp 2 B's
        // The warp walks the slices together, so that addresses stay in uniform registers; one thread issues.
        const bool chosen = elect_one();
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        const uint32_t leader = map_to(full(0), 0), stage_bytes = g.stage_bytes;
        const int stages = g.stages;
        for (int i = pair; ok && i < g.items; i += pairs) {
            const Item t = item_at(g, i);
            const Problem &q = g.problem[t.p];
            const int mine = EPI == kGate ? 128 : t.cols / 2; // columns of B in this CTA
            const int loads = B_MN && mine > 64 ? 2 : 1;
            const uint32_t load_bytes = B_MN ? kChunk : g.box * 128u;
            const uint32_t bytes = 2 * (kABytes + (uint32_t)loads * load_bytes); // of both CTAs
            const int row = t.tm * kBM + (int)rank * 128;
            const int col = EPI == kGate ? t.tn * 128 : t.tn * g.bn + (int)rank * mine;
            int k = t.k0, before = 0; // slices of the operand pairs before this one
            for (int seg = q.seg; ok && k < t.k1; before += g.seg_blocks[seg++]) {
                const int last = min(t.k1, before + g.seg_blocks[seg]);
                const CUtensorMap *ma = &g.a[seg], *mb = EPI == kGate ? &g.b[rank] : &g.b[seg];
                for (; k < last; ++k) {
                    ok = bar_wait(empty(stage), phase ^ 1u, &gave_up);
                    if (!ok) break;
                    const uint32_t bar = leader + 8u * stage;
                    const uint32_t sa = base + stage * stage_bytes, sb = sa + kABytes;
                    const int depth = (k - before) * kBK;
                    if (chosen) {
                        if (warp == 0) {
                            if (rank == 0) bar_expect(full(stage), bytes);
                            if constexpr (A_MN) {
                                tma_load_pair(sa, ma, row, depth, bar);
                                tma_load_pair(sa + kChunk, ma, row + 64, depth, bar);
                            } else {
                                tma_load_pair(sa, ma, depth, row, bar);
                            }
                        } else {
                            if constexpr (B_MN) {
                                tma_load_pair(sb, mb, col, depth, bar);
                                if (loads == 2) tma_load_pair(sb + kChunk, mb, col + 64, depth, bar);
                            } else {
                                tma_load_pair(sb, mb, depth, col, bar);
                            }
                        }
                    }
                    __syncwarp();
                    if (++stage == stages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
        if (warp == 2 && chosen) {
            for (int r = blockIdx.x; r < g.ahead_rows; r += gridDim.x) {
                const int64_t at = r * g.ahead_ld * 2;
                l2_prefetch(static_cast<const char *>(g.ahead[0]) + at, g.ahead_bytes);
                if (g.ahead[1]) l2_prefetch(static_cast<const char *>(g.ahead[1]) + at, g.ahead_bytes);
            }
        }
        // every slice has been consumed: nothing is in flight towards this CTA any more
        for (int s = 0; ok && s < stages; ++s) {
            ok = bar_wait(empty(stage), phase ^ 1u, &gave_up);
            if (++stage == stages) {
                stage = 0;
                phase ^= 1u;
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ---------------------------------------------------------- products
        constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
        constexpr uint32_t kStepA = A_MN ? 16 * 128 : 32, kStepB = B_MN ? 16 * 128 : 32; // 16 of k further
        const bool chosen = elect_one();
        int stage = 0, turn = 0;
        uint32_t phase = 0;
        bool ok = true;
        const uint32_t stage_bytes = g.stage_bytes;
        const int stages = g.stages;
        for (int i = pair; ok && i < g.items; i += pairs, ++turn) {
            const Item t = item_at(g, i);
            const int acc = turn & 1;
            ok = bar_wait(acc_empty(acc), ((turn >> 1) & 1) ^ 1, &gave_up);
            if (!ok) break;
            fence_after();
            const uint32_t desc = EPI == kGate ? instruction_desc(kType, A_MN, B_MN, kBM, 256)
                                               : instruction_desc(kType, A_MN, B_MN, kBM, 0) | (uint32_t)(t.cols >> 3) << 17;
            const uint32_t d = tmem + acc * 256;
            for (int k = t.k0; k < t.k1; ++k) {
                ok = bar_wait(full(stage), phase, &gave_up);
                if (!ok) break;
                fence_after();
                if (chosen) {
                    const uint32_t sa = base + stage * stage_bytes;
                    const uint64_t da = operand_desc(sa, A_MN ? kChunk : 16), db = operand_desc(sa + kABytes, B_MN ? kChunk : 16);
#pragma unroll
                    for (int j = 0; j < kBK / 16; ++j)
                        mma_pair(d, da + j * (kStepA >> 4), db + j * (kStepB >> 4), desc, k > t.k0 || j > 0);
                    commit_pair(empty(stage));
                    if (k + 1 == t.k1) commit_pair(acc_full(acc));
                }
                __syncwarp();
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
    } else if (warp >= kFirstEpilogueWarp) {
        // ---------------------------------------------------------- accumulators out
        const uint32_t quarter = warp & 3, half = (warp - kFirstEpilogueWarp) >> 2; // a warp reads the TMEM lanes of its quarter
        const uint32_t buf0 = staging + (warp - kFirstEpilogueWarp) * 2 * kStaging, buf1 = buf0 + kStaging;
        int turn = 0;
        for (int i = pair; i < g.items; i += pairs, ++turn) {
            const Item t = item_at(g, i);
            const Problem &q = g.problem[t.p];
            const int acc = turn & 1;
            const int row0 = t.tm * kBM + (int)rank * 128 + quarter * 32; // this warp's 32 rows
            const bool live = row0 < q.m;
            const uint32_t d = tmem + acc * 256 + (quarter * 32u << 16);
            if constexpr (EPI == kGate) {
                if (!bar_wait(acc_full(acc), (turn >> 1) & 1, &gave_up)) break;
                fence_after();
                const int c = half * 64, col0 = t.tn * 128 + c;
                if (lane == 0) tma_store_read<0>();
                __syncwarp();
                uint4 h[8];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float a[32], b[32];
                    tmem_ld32(d + c + 32 * j, a);
                    tmem_ld32(d + 128 + c + 32 * j, b);
                    tmem_wait_ld();
                    if (g.gate.p) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            st_shared(piece(buf0, lane, 4 * j + k), pack8<T>(a + 8 * k));
                            st_shared(piece(buf1, lane, 4 * j + k), pack8<T>(b + 8 * k));
                        }
                    }
                    gate_columns<ACT>(a, b);
#pragma unroll
                    for (int k = 0; k < 4; ++k) h[4 * j + k] = pack8<T>(a + 8 * k);
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(map_to(acc_empty(acc), 0));
                if (live && col0 < q.n) {
                    if (g.gate.p) {
                        rows_out(g.gate, buf0, row0, col0, q.m, q.n, lane);
                        rows_out(g.up, buf1, row0, col0, q.m, q.n, lane);
                        if (lane == 0) tma_store_read<0>();
                        __syncwarp();
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) st_shared(piece(buf0, lane, k), h[k]);
                    rows_out(g.out[0], buf0, row0, col0, q.m, q.n, lane);
                    if (g.out2.p) rows_out(g.out2, buf0, row0, col0, q.m, q.n, lane);
                }
            } else if constexpr (EPI == kGateGrad) {
                // Blocks of 32 columns, two in turn: one is brought in while another is worked on, and da and db leave from
                // where a and b arrived, by cp.async and plain stores, 64 consecutive bytes a row (TMA boxes with a
                // barrier a block measured the same).
                const int count = (min(t.cols, q.n - t.tn * g.bn) + 31) / 32, rounds = live ? (count - (int)half + 1) / 2 : 0;
                const int first = t.tn * g.bn + half * 32;       // this warp's blocks: every second one
                const int copy_row = lane >> 2, copy_piece = lane & 3; // rows copy_row + 8 i, 16 bytes of each
                const auto place = [&](int k, uint32_t row, uint32_t e) {
                    return buf0 + (k & 1) * kStaging + row * 64 + ((e ^ (row >> 1 & 3)) << 4); // swizzled; b 2 KB on
                };
                const auto bring = [&](int k) {
                    const int col = first + 64 * k + copy_piece * 8;
                    const uint32_t bytes = max(0, min(8, q.n - col)) * 2;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = copy_row + 8 * i, row = row0 + r;
                        const bool there = k < rounds && row < q.m && bytes;
                        const int64_t at_gate = there ? (int64_t)row * g.gate.ld + col : 0, at_up = there ? (int64_t)row * g.up.ld + col : 0;
                        async_copy16(place(k, r, copy_piece), static_cast<const T *>(g.gate.p) + at_gate, there ? bytes : 0);
                        async_copy16(place(k, r, copy_piece) + kStaging / 2, static_cast<const T *>(g.up.p) + at_up, there ? bytes : 0);
                    }
                    async_commit();
                };
                if (row0 + (int)lane < q.m) { // the later blocks into L2: a row's 128 bytes for both halves' warps
                    const Rows &o = half ? g.up : g.gate;
                    for (int k = 2; k < rounds; ++k) l2_prefetch_line(static_cast<const T *>(o.p) + (int64_t)(row0 + lane) * o.ld + t.tn * g.bn + 64 * k);
                }
                bring(0);
                bring(1);
                if (!bar_wait(acc_full(acc), (turn >> 1) & 1, &gave_up)) break;
                fence_after();
                for (int k = 0; k < rounds; ++k) {
                    float dh[32];
                    tmem_ld32(d + half * 32 + 64 * k, dh);
                    async_wait<1>();
                    __syncwarp();
                    tmem_wait_ld();
                    if (k + 1 == rounds) { // all that this warp reads has been read
                        fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive_cluster(map_to(acc_empty(acc), 0));
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t pa = place(k, lane, e), pb = pa + kStaging / 2;
                        float a[8], b[8];
                        unpack8<T>(ld_shared(pa), a);
                        unpack8<T>(ld_shared(pb), b);
                        gate_gradient<ACT>(dh + 8 * e, a, b);
                        st_shared(pa, pack8<T>(a));
                        st_shared(pb, pack8<T>(b));
                    }
                    __syncwarp();
                    const int col = first + 64 * k + copy_piece * 8;
#pragma unroll
                    for (int i = 0; i < 4; ++i) { // da and db have padded rows: whole pieces
                        const int r = copy_row + 8 * i, row = row0 + r;
                        const uint4 va = ld_shared(place(k, r, copy_piece)), vb = ld_shared(place(k, r, copy_piece) + kStaging / 2);
                        if (row < q.m && col < q.n) {
                            *reinterpret_cast<uint4 *>(static_cast<T *>(g.out[0].p) + (int64_t)row * g.out[0].ld + col) = va;
                            *reinterpret_cast<uint4 *>(static_cast<T *>(g.out2.p) + (int64_t)row * g.out2.ld + col) = vb;
                        }
                    }
                    __syncwarp();
                    bring(k + 2);
                }
                if (rounds == 0) {
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_cluster(map_to(acc_empty(acc), 0));
                }
                async_wait<0>();
                __syncwarp();
            } else {
                if (!bar_wait(acc_full(acc), (turn >> 1) & 1, &gave_up)) break;
                fence_after();
                const int subs = (min(t.cols, q.n - t.tn * g.bn) + 63) / 64;
                if (t.slot < 0) { // the last tile's stores have been read out of the buffers
                    if (lane == 0) tma_store_read<0>();
                    __syncwarp();
                }
#pragma unroll
                for (int turn2 = 0; turn2 < 2; ++turn2) { // a warp has two blocks of 64 columns at most
                    const int sub = half + 2 * turn2;
                    if (!live || sub >= subs) break;
                    float v[64];
                    tmem_ld32(d + sub * 64, reinterpret_cast<float(&)[32]>(v));
                    tmem_ld32(d + sub * 64 + 32, reinterpret_cast<float(&)[32]>(v[32]));
                    tmem_wait_ld();
                    if (t.slot < 0) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) st_shared(piece(turn2 ? buf1 : buf0, lane, k), pack8<T>(v + 8 * k));
                    } else {
                        // rows side by side: 512 consecutive bytes a warp and store
                        float4 *part = reinterpret_cast<float4 *>(g.partials) +
                                       ((int64_t)t.slot * (g.bn / 4) + sub * 16) * kBM + rank * 128 + quarter * 32 + lane;
#pragma unroll
                        for (int k = 0; k < 16; ++k) part[k * kBM] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                    }
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(map_to(acc_empty(acc), 0));
                if (t.slot < 0 && live) {
                    const int col0 = t.tn * g.bn + half * 64;
                    if ((int)half < subs) rows_out(g.out[t.p], buf0, row0, col0, q.m, q.n, lane);
                    if ((int)half + 2 < subs) rows_out(g.out[t.p], buf1, row0, col0 + 128, q.m, q.n, lane);
                }
            }
        }
        if (lane == 0) tma_store_done();
    }
    __syncwarp();
    __syncthreads();
    if (gave_up) {
        // leave the copies and products in flight a bounded time to end, and say so
        if (threadIdx.x == 0) atomicAdd(&g_waits_run_out, 1u);
        const uint64_t begin = now_ns();
        while (now_ns() - begin < 5000000ull) __nanosleep(1000);
    }
    cluster_sync();
    if (warp == 1) tmem_free_pair(tmem, kTmemColumns);
}

// The parts of the tiles that were split, added up in order.  A CTA takes 32 rows of 32 columns: its warps read 32 rows
// of 4 columns each, 512 bytes in a row, and write rows of 32 columns.
constexpr int kJoinCols = 32;
template <typename T>
__global__ void __launch_bounds__(256) k_join(const __grid_constant__ GemmArgs g)
{
    __shared__ T sums[32][kJoinCols + 2];
    wait_prior_grid();
    release_next_grid();
    const Item t = item_at(g, g.whole + (int)blockIdx.x * g.splits);
    const Problem &q = g.problem[t.p];
    const int row0 = t.tm * kBM + blockIdx.z * 32, col0 = t.tn * g.bn + blockIdx.y * kJoinCols;
    if (row0 >= q.m || col0 >= q.n) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t next = (int64_t)(g.bn / 4) * kBM;
    float v[4] = {};
    if (col0 + warp * 4 < q.n) { // rows past the end were not written: not stored below
        const float4 *part = reinterpret_cast<const float4 *>(g.partials) + (int64_t)t.slot * next +
                             (blockIdx.y * (kJoinCols / 4) + warp) * kBM + blockIdx.z * 32 + lane;
#pragma unroll 8
        for (int s = 0; s < g.splits; ++s) {
            const float4 x = __ldcg(part + s * next);
            v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[lane][warp * 4 + i] = from_f32<T>(v[i]);
    __syncthreads();
    const int rows = min(32, q.m - row0);
    T *out = static_cast<T *>(g.out[t.p].p) + (int64_t)row0 * g.out[t.p].ld + col0;
    for (int r = warp; r < rows; r += 8) {
        if (col0 + lane < q.n) out[(int64_t)r * g.out[t.p].ld + lane] = sums[r][lane];
    }
}

// ------------------------------------------------------------------ rows that TMA cannot read
struct PackJob {
    const uint16_t *src;
    uint16_t *dst;
    int64_t ld_src, ld_dst;
    int64_t rows;
    int cols;
};
struct PackArgs {
    PackJob job[8];
};
__global__ void __launch_bounds__(256) k_pack(const __grid_constant__ PackArgs a)
{
    wait_prior_grid();
    release_next_grid();
    const PackJob &j = a.job[blockIdx.y];
    const int pieces = (j.cols + 7) / 8; // 16 bytes of a padded row each
    const int64_t all = j.rows * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces;
        const int c = (int)(i - r * pieces) * 8;
        const uint16_t *s = j.src + r * j.ld_src + c;
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (c + k < j.cols) w[k / 2] |= (uint32_t)s[k] << (16 * (k & 1));
        }
        *reinterpret_cast<uint4 *>(j.dst + r * j.ld_dst + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ------------------------------------------------------------------ few tokens
// Up to 16 tokens the block is bound by the weights' bytes, and tiles of 256 rows would be nearly empty.  Here
// the weights are the left operand of mma.sync (m16n8k16), 16 of their rows a CTA.  A lane copies 16 bytes, 8 consecutive
// k of one row, into a place of shared memory that it alone reads, several steps ahead (cp.async: no registers held, no
// barrier); since the order of k within a product is free as long as both operands share it, those 8 are the lane's part
// of two products, and the tokens' 8 k lie the same way.  Eight warps, and the CTAs of a cluster, share the depth; their
// sums meet in shared memory, in order, where the gate, the activation and the product are applied.
// One call, its weights from memory, this form against the tiles above: aligned matrices, 16 tokens, 512 x 1408 13.1 and 15.7 us, 1024 x 4096
// 20.5 and 21.3, 1600 x 6400 18.5 and 30.9, 4096 x 11008 58.4 and 78.8; with four blocks of 8 tokens, at 17 to 32, 13.1 and 15.7, 26 and 21.4,
// 27 and 28.8, 78 and 79.4 (another set of kernels for a tenth at most: left out).
constexpr int kFewTokens = 16;
// Rows that are not aligned come in element by element, here for every token block, in the tiles' way once into padded copies:
// this form wins for small matrices.  8 tokens: 512 x 1408 12.3 and 19.3 us, 777 x 2051 23.2 and 23.9, 1024 x 4096 35.3 and 34.3, 1600 x 6400
// 67.5 and 56.8, 4096 x 11008 337 and 201; 1 token: 777 x 2051 20.6 and 24.0, 1024 x 4096 30.9 and 35.6, 1600 x 6400 61.5 and 59.9; 16 tokens:
// 512 x 1408 12.5 and 19.6, 777 x 2051 26.8 and 23.9.
inline bool few_elements(int64_t tokens, int d, int f) { return (int64_t)d * f * (tokens + 7) <= 1 << 25; }
constexpr int kFewWarps = 8;
constexpr uint32_t kFewPiece = 32 * 16; // what a warp copies at once
// Steps of 32 k on their way: as many as leave room for three CTAs an SM.  One token, 1600 x 6400, weights from memory, in a
// graph: 14.5 us (4.2 TB/s; 4096 x 11008: 50 us, 5.4 TB/s); 15.1 and 60 us with four warps, 20 us with two CTAs an SM.
__host__ __device__ constexpr int few_steps_ahead(bool dual, int nt) { return 70 * 1024 / (kFewWarps * ((dual ? 4 : 2) + nt) * (int)kFewPiece) < 12 ? 70 * 1024 / (kFewWarps * ((dual ? 4 : 2) + nt) * (int)kFewPiece) : 12; }

struct FewArgs {
    const void *w0, *w1; // w1: the second projection, side by side with w0
    const void *x;
    int64_t ld0, ld1, ldx;
    int rows, depth, tokens; // rows of the weights = columns of the output
    int act;
    void *out, *gate, *up;
    int64_t ldo, ld_gate, ld_up;
    int parts; // CTAs of a cluster
};

template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 8 elements of a row from k on into a lane's own place; zeros past the row's end and where the row does not exist.
template <bool VEC>
__device__ __forceinline__ void few_copy(uint32_t place, const uint16_t *row, int k, int depth, bool live)
{
    const int there = live && k < depth ? min(8, depth - k) : 0;
    if constexpr (VEC) {
        async_copy16(place, there ? row + k : row, 2 * there);
    } else {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i < there) w[i / 2] |= (uint32_t)row[k + i] << (16 * (i & 1));
        }
        st_shared(place, make_uint4(w[0], w[1], w[2], w[3]));
    }
}
template <typename T, bool DUAL, int NT, bool VEC>
__global__ void __launch_bounds__(32 * kFewWarps) k_few(const __grid_constant__ FewArgs g)
{
    constexpr int kSides = DUAL ? 2 : 1, kCols = 8 * NT, kAhead = few_steps_ahead(DUAL, NT), kPieces = 2 * kSides + NT;
    extern __shared__ __align__(16) char ring[]; // [warps][kAhead][kPieces][32 lanes][16 bytes]
    __shared__ float sums[kFewWarps][kSides][16][kCols + 1];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, c = lane & 3;
    const int part = blockIdx.x % g.parts, row0 = blockIdx.x / g.parts * 16;
    const int steps = (g.depth + 31) / 32, share = part * kFewWarps + warp, shares = g.parts * kFewWarps;
    const int s0 = (int)((int64_t)steps * share / shares), s1 = (int)((int64_t)steps * (share + 1) / shares);
    const uint32_t mine = smem_u32(ring) + warp * kAhead * kPieces * kFewPiece + lane * 16;
    const auto place = [&](int slot, int p) { return mine + (uint32_t)(slot * kPieces + p) * kFewPiece; };

    // rows that do not exist are not read: their copies have no bytes, from the matrix's first row
    const bool live[2] = {row0 + (int)quad < g.rows, row0 + 8 + (int)quad < g.rows};
    const uint16_t *w[kSides][2], *x[NT];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        w[0][r] = static_cast<const uint16_t *>(g.w0) + (live[r] ? (int64_t)(row0 + 8 * r + quad) * g.ld0 : 0);
        if constexpr (DUAL) w[1][r] = static_cast<const uint16_t *>(g.w1) + (live[r] ? (int64_t)(row0 + 8 * r + quad) * g.ld1 : 0);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n] = static_cast<const uint16_t *>(g.x) + (n * 8 + (int)quad < g.tokens ? (int64_t)(n * 8 + quad) * g.ldx : 0);
    const auto copy_weights = [&](int s, int slot) {
#pragma unroll
        for (int e = 0; e < kSides; ++e) {
#pragma unroll
            for (int r = 0; r < 2; ++r) few_copy<VEC>(place(slot, 2 * e + r), w[e][r], s * 32 + (int)c * 8, g.depth, live[r]);
        }
    };
    const auto copy_tokens = [&](int s, int slot) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            few_copy<VEC>(place(slot, 2 * kSides + n), x[n], s * 32 + (int)c * 8, g.depth, n * 8 + (int)quad < g.tokens);
    };
    // The second launch of a call may start on its weights at once: the one before it, which wrote its tokens, does not
    // write them, and had itself waited for what was before the call.
    if constexpr (DUAL) {
        wait_prior_grid();
        release_next_grid();
    }
    for (int s = s0; s < min(s1, s0 + kAhead); ++s) copy_weights(s, s - s0);
    if constexpr (!DUAL) {
        wait_prior_grid();
        release_next_grid();
    }
    for (int s = s0; s < s0 + kAhead; ++s) {
        if (s < s1) copy_tokens(s, s - s0);
        async_commit();
    }
    float acc[kSides][NT][4] = {};
    for (int s = s0, slot = 0; s < s1; ++s, slot = slot + 1 == kAhead ? 0 : slot + 1) {
        async_wait<kAhead - 1>();
        uint4 a[kSides][2], b[NT];
#pragma unroll
        for (int e = 0; e < kSides; ++e) {
#pragma unroll
            for (int r = 0; r < 2; ++r) a[e][r] = ld_shared(place(slot, 2 * e + r));
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) b[n] = ld_shared(place(slot, 2 * kSides + n));
#pragma unroll
        for (int e = 0; e < kSides; ++e) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                mma_16816<T>(acc[e][n], a[e][0].x, a[e][1].x, a[e][0].y, a[e][1].y, b[n].x, b[n].y);
                mma_16816<T>(acc[e][n], a[e][0].z, a[e][1].z, a[e][0].w, a[e][1].w, b[n].z, b[n].w);
            }
        }
        if (s + kAhead < s1) {
            copy_weights(s + kAhead, slot);
            copy_tokens(s + kAhead, slot);
        }
        async_commit();
    }
#pragma unroll
    for (int e = 0; e < kSides; ++e) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[warp][e][quad + 8 * (i >> 1)][n * 8 + 2 * c + (i & 1)] = acc[e][n][i];
        }
    }
    __syncthreads();
    // this CTA's sums into its first warp's places
    for (int i = threadIdx.x; i < kSides * 16 * kCols; i += 32 * kFewWarps) {
        const int e = i / (16 * kCols), r = i / kCols % 16, n = i % kCols;
        float v = sums[0][e][r][n];
#pragma unroll
        for (int k = 1; k < kFewWarps; ++k) v += sums[k][e][r][n];
        sums[0][e][r][n] = v;
    }
    if (g.parts > 1) cluster_sync();
    else __syncthreads();
    // every CTA of the cluster finishes its share of the outputs
    for (int i = part * 32 * kFewWarps + threadIdx.x; i < 16 * kCols; i += g.parts * 32 * kFewWarps) {
        const int r = i % 16, n = i / 16;
        if (n >= g.tokens || row0 + r >= g.rows) continue;
        float v[kSides];
#pragma unroll
        for (int e = 0; e < kSides; ++e) {
            v[e] = 0.0f;
            const uint32_t at = smem_u32(&sums[0][e][r][n]);
            for (int p = 0; p < g.parts; ++p) {
                float y;
                if (g.parts > 1) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(y) : "r"(map_to(at, p)) : "memory");
                else y = sums[0][e][r][n];
                v[e] += y;
            }
        }
        const int col = row0 + r;
        if constexpr (DUAL) {
            f32x2 value, slope;
            if (g.act == A2SGD_ACT_SILU) activation2<A2SGD_ACT_SILU>(pair(v[0], 0.0f), value, slope);
            else activation2<A2SGD_ACT_GELU_TANH>(pair(v[0], 0.0f), value, slope);
            float h, other;
            unpair(value, h, other);
            static_cast<T *>(g.out)[(int64_t)n * g.ldo + col] = from_f32<T>(h * v[1]);
            if (g.gate) {
                static_cast<T *>(g.gate)[(int64_t)n * g.ld_gate + col] = from_f32<T>(v[0]);
                static_cast<T *>(g.up)[(int64_t)n * g.ld_up + col] = from_f32<T>(v[1]);
            }
        } else {
            static_cast<T *>(g.out)[(int64_t)n * g.ldo + col] = from_f32<T>(v[0]);
        }
    }
    __syncwarp(); // lanes past the last token have left the loop's body early, and the barrier wants whole warps
    if (g.parts > 1) cluster_sync(); // no CTA leaves while another reads its sums
}

// ------------------------------------------------------------------ host
// A matrix of 16-bit elements as the kernels see it.
struct Matrix {
    const void *p = nullptr;
    int64_t ld = 0, rows = 0;
    int cols = 0;
};

inline int64_t padded(int64_t cols) { return (cols + 7) / 8 * 8; }

// Tiles of `box_rows` rows and 64 columns, 128 bytes a row, swizzled.
bool make_map(CUtensorMap *map, const Matrix &m, int dtype, int box_rows)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(m.rows > 1 ? m.ld : padded(m.cols)) * 2}; // one row: any stride is right
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, steps[2] = {1, 1};
    return encode(map, dtype == A2SGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                  const_cast<void *>(m.p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline bool tma_ok(const Matrix &m) { return aligned(m.p, 16) && (m.rows <= 1 || m.ld % 8 == 0); }
inline uint64_t room(int64_t rows, int64_t cols) { return ((uint64_t)rows * padded(cols) * 2 + 255) / 256 * 256; }
inline int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// What the epilogue writes: by TMA where rows allow it.  A TMA store leaves out what lies past the end of a row in pieces
// of 16 bytes only, so that rows of other lengths are written element by element.
bool set_rows(Rows &r, const Matrix &m, int dtype)
{
    r.p = const_cast<void *>(m.p);
    r.ld = m.ld;
    r.tma = m.p && tma_ok(m) && m.cols % 8 == 0;
    return !r.tma || make_map(&r.map, m, dtype, 32);
}

// Rows that are read or written without TMA.
void set_plain(Rows &r, const Matrix &m)
{
    r.p = const_cast<void *>(m.p);
    r.ld = m.ld;
}

// Rows of the workspace with their padding, which may be written.
Matrix whole_rows(Matrix m)
{
    m.cols = (int)m.ld;
    return m;
}

// ---- the shape of a launch ---------------------------------------------------------------------------
// What a slice of a tile costs, in clocks: the tensor cores take 2 a column, the way from L2 about 56 bytes a clock
// and SM.  With [8192, 6400] x [1600, 6400]^T a round of tiles took 27, 33 and 37 us at 128, 192 and 256
// columns: 459, 559, 624 clocks a slice against 439, 512 and 585 by this rule.
inline double slice_clocks(int bn) { return std::max(2.0 * bn, (16384.0 + 64.0 * bn) / 56.0); }

constexpr int kMostPairs = 80;  // pairs that take part in splitting: bounds the workspace
constexpr int kLeastSlices = 4; // of a part of a tile

struct Shape {
    int bn = 256, splits = 1;
    double cost = 1e30;
};

// Tiles that do not fill a last round over the pairs of SMs are split in depth, as evenly as the pairs allow.
inline int splits_of(int64_t tiles, int pairs, int k_blocks)
{
    const int64_t rest = tiles % pairs;
    if (rest == 0) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(pairs, kMostPairs) / rest, k_blocks / kLeastSlices));
}

// Products with plain outputs, all of the same depth: the width and the splitting with the least cost.
struct Extent {
    int64_t m;
    int n;
};
Shape choose(const Extent *outs, int count, int k_blocks, bool b_mn, int pairs)
{
    Shape best;
    int widest = 0;
    for (int i = 0; i < count; ++i) widest = std::max(widest, outs[i].n);
    for (int bn : {64, 128, 192, 256}) {             // whole staged blocks of 64 columns
        if (b_mn && bn != 128 && bn != 256) continue; // whole chunks of 64 columns in either CTA
        if (bn > 128 && bn - 64 >= widest) continue;
        int64_t tiles = 0;
        for (int i = 0; i < count; ++i) tiles += (int64_t)ceil_div(outs[i].m, kBM) * ceil_div(outs[i].n, bn);
        for (int splits : {1, splits_of(tiles, pairs, k_blocks)}) {
            const double rounds = (double)(tiles / pairs) + (tiles % pairs ? 1.0 / splits : 0.0);
            // and the last tile's way out, and joining the parts: a launch, and their bytes through L2
            const double join = splits > 1 ? 6000.0 + (double)(tiles % pairs) * splits * 2.0 * kBM * bn * 4 / (2 * pairs * 40.0) : 0.0;
            const double cost = rounds * k_blocks * slice_clocks(bn) + 12.0 * bn + join;
            if (cost < best.cost) {
                best.bn = bn;
                best.splits = splits;
                best.cost = cost;
            }
        }
    }
    return best;
}

inline uint64_t partial_bytes(int64_t slots, int bn) { return (uint64_t)slots * kBM * bn * sizeof(float); }

template <typename T, int EPI, bool A_MN, bool B_MN, int ACT = 0>
int launch_gemm(GemmArgs &g, int tiles, int sms, cudaStream_t s)
{
    const void *fn = reinterpret_cast<const void *>(&k_gemm<T, EPI, A_MN, B_MN, ACT>);
    A2_TRAIN_CUDA(allow_smem(fn, kSmem - 1024));
    const int pairs = sms / 2;
    g.whole = g.splits > 1 ? tiles / pairs * pairs : tiles;
    g.items = g.whole + (tiles - g.whole) * g.splits;
    g.stage_bytes = kABytes + (EPI == kGate ? 128u : (uint32_t)g.bn / 2) * 128u;
    g.stages = (int)std::min<uint32_t>(kMostStages, kOperands / g.stage_bytes);
    void *params[] = {&g};
    A2_TRAIN_CUDA(launch(fn, dim3(2 * (unsigned)std::min(g.items, pairs)), kThreads, kSmem - 1024, params, s));
    if (EPI == kStore && g.splits > 1)
        A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_join<T>),
                             dim3((unsigned)(tiles - g.whole), (unsigned)(g.bn / kJoinCols), kBM / 32), 256, 0, params, s));
    return A2SGD_OK;
}

// The weights of the next product, for launches of no more than two rounds of tiles: their ends and the next launch's
// start would leave the memory idle.  Rows that bulk copies can read (the pointers are TMA operands': 16-byte rows).
void bring_ahead(GemmArgs &g, int tiles, int sms, const Matrix &w0, const Matrix *w1)
{
    if (tiles > 2 * (sms / 2) || (w1 && w1->ld != w0.ld)) return;
    g.ahead[0] = w0.p;
    g.ahead[1] = w1 ? w1->p : nullptr;
    g.ahead_ld = w0.ld;
    g.ahead_bytes = w0.cols / 8 * 16;
    g.ahead_rows = g.ahead_bytes ? (int)w0.rows : 0;
}

// The maps of one operand pair.  An operand that is not transposed lies as [rows, k], a transposed one as [k, rows].
template <bool A_MN, bool B_MN>
bool add_operands(GemmArgs &g, int i, const Matrix &a, const Matrix &b, int dtype)
{
    return make_map(&g.a[i], a, dtype, A_MN ? kBK : 128) && make_map(&g.b[i], b, dtype, B_MN ? kBK : g.box);
}

// Adds a product of `segs` operand pairs, each `k` deep, from pair `seg` on.
int add_problem(GemmArgs &g, int64_t m, int n, int tile_n, int seg, int segs, int64_t k, int tiles)
{
    Problem &q = g.problem[g.problems++];
    q.m = (int)m;
    q.n = n;
    q.tiles_m = ceil_div(m, kBM);
    q.tiles_n = ceil_div(n, tile_n);
    q.first = tiles;
    q.seg = seg;
    q.k_blocks = segs * ceil_div(k, kBK);
    for (int i = seg; i < seg + segs; ++i) g.seg_blocks[i] = ceil_div(k, kBK);
    g.operands = seg + segs;
    return tiles + q.tiles_m * q.tiles_n;
}

void set_shape(GemmArgs &g, const Shape &shape, float *partials)
{
    g.bn = shape.bn;
    g.box = shape.bn / 2;
    g.splits = shape.splits;
    g.partials = partials;
}

struct Packer {
    PackArgs args{};
    int jobs = 0;
    int64_t most_pieces = 0;
    char *begin, *at;
    explicit Packer(void *workspace) : begin(static_cast<char *>(workspace)), at(begin) {}
    void *take(int64_t rows, int64_t cols)
    {
        void *p = at;
        at += room(rows, cols);
        return p;
    }
    // The matrix itself, or where its padded copy will be.
    Matrix usable(const Matrix &m)
    {
        if (tma_ok(m)) return m;
        Matrix c = m;
        c.ld = padded(m.cols);
        c.p = take(m.rows, m.cols);
        args.job[jobs++] = PackJob{static_cast<const uint16_t *>(m.p), static_cast<uint16_t *>(const_cast<void *>(c.p)), m.ld, c.ld,
                                   m.rows, m.cols};
        most_pieces = std::max(most_pieces, m.rows * (padded(m.cols) / 8));
        return c;
    }
    uint64_t used() const { return (uint64_t)(at - begin); }
    bool fits(uint64_t bytes) const { return used() == 0 || (begin && used() <= bytes); }
    // The shape, without its splitting where the rest of the workspace has no room for the partial sums.
    Shape fit(Shape shape, uint64_t bytes) const
    {
        if (shape.splits > 1 && (!begin || used() + partial_bytes(kMostPairs, shape.bn) > bytes)) shape.splits = 1;
        return shape;
    }
    int run(int sms, cudaStream_t s)
    {
        if (!jobs) return A2SGD_OK;
        void *params[] = {&args};
        A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_pack),
                             dim3((unsigned)std::min<int64_t>((most_pieces + 255) / 256, (int64_t)sms * 8), jobs), 256, 0, params, s));
        return A2SGD_OK;
    }
};

int check(const Matrix &m, bool needed)
{
    if (!m.p) return needed ? A2SGD_ERR_ARG : A2SGD_OK;
    if (m.rows > 1 && m.ld < m.cols) return A2SGD_ERR_ARG;
    return aligned(m.p, 2) ? A2SGD_OK : A2SGD_ERR_ALIGN;
}

int check_sizes(uint64_t tokens, uint32_t d, uint32_t f, int dtype, int act)
{
    if ((dtype != A2SGD_BF16 && dtype != A2SGD_F16) || (act != A2SGD_ACT_SILU && act != A2SGD_ACT_GELU_TANH)) return A2SGD_ERR_ARG;
    if (d == 0 || f == 0) return A2SGD_ERR_ARG;
    if (tokens >= (1ull << 30) || d >= (1u << 24) || f >= (1u << 24)) return A2SGD_ERR_TOO_LARGE;
    // tiles and slices are counted in 24 bits, what a tile's place in them is worked out from
    constexpr uint64_t kMost = 1ull << 24;
    const uint64_t wide = std::max(d, f) / 64 + 1;
    if ((tokens / kBM + 1) * wide >= kMost || 3 * ((uint64_t)d / 64 + 1) * ((uint64_t)f / 64 + 1) >= kMost ||
        std::max<uint64_t>(tokens, 2 * std::max(d, f)) / kBK * kMostPairs >= kMost)
        return A2SGD_ERR_TOO_LARGE;
    return A2SGD_OK;
}

template <typename T, bool DUAL, bool VEC>
const void *pick_few(int tokens)
{
    return tokens <= 8 ? reinterpret_cast<const void *>(&k_few<T, DUAL, 1, VEC>) : reinterpret_cast<const void *>(&k_few<T, DUAL, 2, VEC>);
}

template <typename T, bool DUAL>
int launch_few(FewArgs &g, bool vec, int sms, cudaStream_t s)
{
    const void *fn = vec ? pick_few<T, DUAL, true>(g.tokens) : pick_few<T, DUAL, false>(g.tokens);
    const int nt = g.tokens <= 8 ? 1 : 2;
    const size_t smem = (size_t)kFewWarps * few_steps_ahead(DUAL, nt) * ((DUAL ? 4 : 2) + nt) * kFewPiece;
    A2_TRAIN_CUDA(allow_smem(fn, smem));
    // the depth is shared out over a cluster until there are two CTAs an SM, as long as a warp keeps two steps
    const int groups = ceil_div(g.rows, 16), steps = ceil_div(g.depth, 32);
    g.parts = 1;
    while (g.parts < 8 && groups * g.parts < 2 * sms && steps >= g.parts * 2 * kFewWarps * 2) g.parts *= 2;
    void *params[] = {&g};
    A2_TRAIN_CUDA(launch(fn, dim3((unsigned)(groups * g.parts)), 32 * kFewWarps, smem, params, s, (unsigned)g.parts));
    return A2SGD_OK;
}

template <typename T>
int forward_few(const Matrix &x, const Matrix &wg, const Matrix &wu, const Matrix &wd, const Matrix &y, const Matrix &h,
                const Matrix &gate, const Matrix &up, int act, int sms, cudaStream_t s)
{
    FewArgs g{};
    g.w0 = wg.p, g.ld0 = wg.ld;
    g.w1 = wu.p, g.ld1 = wu.ld;
    g.x = x.p, g.ldx = x.ld;
    g.rows = h.cols;
    g.depth = x.cols;
    g.tokens = (int)x.rows;
    g.act = act;
    g.out = const_cast<void *>(h.p), g.ldo = h.ld;
    g.gate = const_cast<void *>(gate.p), g.ld_gate = gate.ld;
    g.up = const_cast<void *>(up.p), g.ld_up = up.ld;
    const int rc = launch_few<T, true>(g, tma_ok(wg) && tma_ok(wu) && tma_ok(x), sms, s);
    if (rc != A2SGD_OK) return rc;
    g = FewArgs{};
    g.w0 = wd.p, g.ld0 = wd.ld;
    g.x = h.p, g.ldx = h.ld;
    g.rows = y.cols;
    g.depth = h.cols;
    g.tokens = (int)x.rows;
    g.out = const_cast<void *>(y.p), g.ldo = y.ld;
    return launch_few<T, false>(g, tma_ok(wd) && tma_ok(h), sms, s);
}

template <typename T>
int forward(const Matrix &x, const Matrix &wg, const Matrix &wu, const Matrix &wd, Matrix y, Matrix h, Matrix gate, Matrix up, int act,
            int dtype, void *workspace, uint64_t workspace_bytes, int sms, cudaStream_t s)
{
    const int64_t t = x.rows;
    const int d = x.cols, f = h.cols;
    Packer pack(workspace);
    const Matrix px = pack.usable(x), pg = pack.usable(wg), pu = pack.usable(wu), pd = pack.usable(wd);
    Matrix ph = h; // what the second product reads
    if (!tma_ok(h)) {
        ph.ld = padded(h.cols);
        ph.p = pack.take(h.rows, h.cols);
    }
    const Extent out{t, d};
    const Shape shape = pack.fit(choose(&out, 1, ceil_div(f, kBK), false, sms / 2), workspace_bytes);
    if (!pack.fits(workspace_bytes)) return A2SGD_ERR_ARG; // for few tokens too, so that what is refused does not go by their number
    const bool whole = tma_ok(x) && tma_ok(wg) && tma_ok(wu) && tma_ok(wd) && tma_ok(h);
    if (t <= kFewTokens && (whole || few_elements(t, d, f))) return forward_few<T>(x, wg, wu, wd, y, h, gate, up, act, sms, s);
    int rc = pack.run(sms, s);
    if (rc != A2SGD_OK) return rc;

    GemmArgs g{};
    g.bn = 256;
    g.box = 128;
    g.splits = 1;
    if (!add_operands<false, false>(g, 0, px, pg, dtype) || !make_map(&g.b[1], pu, dtype, 128) || !set_rows(g.out[0], h, dtype) ||
        (ph.p != h.p && !set_rows(g.out2, whole_rows(ph), dtype)) || !set_rows(g.gate, gate, dtype) || !set_rows(g.up, up, dtype))
        return A2SGD_ERR_CUDA;
    const int tiles = add_problem(g, t, f, 128, 0, 1, d, 0);
    bring_ahead(g, tiles, sms, pd, nullptr);
    rc = act == A2SGD_ACT_SILU ? launch_gemm<T, kGate, false, false, A2SGD_ACT_SILU>(g, tiles, sms, s)
                               : launch_gemm<T, kGate, false, false, A2SGD_ACT_GELU_TANH>(g, tiles, sms, s);
    if (rc != A2SGD_OK) return rc;

    g = GemmArgs{};
    set_shape(g, shape, reinterpret_cast<float *>(pack.at));
    if (!add_operands<false, false>(g, 0, ph, pd, dtype) || !set_rows(g.out[0], y, dtype)) return A2SGD_ERR_CUDA;
    return launch_gemm<T, kStore, false, false>(g, add_problem(g, t, d, g.bn, 0, 1, f, 0), sms, s);
}

template <typename T>
int backward(const Matrix &dy, const Matrix &x, const Matrix &wg, const Matrix &wu, const Matrix &wd, const Matrix &h,
             const Matrix &gate, const Matrix &up, const Matrix &dx, const Matrix &dwg, const Matrix &dwu, const Matrix &dwd, int act,
             int dtype, void *workspace, uint64_t workspace_bytes, int sms, cudaStream_t s)
{
    const int64_t t = x.rows;
    const int d = x.cols, f = h.cols;
    const bool inner = dx.p || dwg.p || dwu.p; // da and db are needed
    Packer pack(workspace);
    Matrix da, db, pdy, pwd, pwg, pwu, px, ph, pgate, pup;
    pdy = pack.usable(dy);
    if (inner) {
        pwd = pack.usable(wd);
        pgate = pack.usable(gate);
        pup = pack.usable(up);
        da.rows = db.rows = t;
        da.cols = db.cols = f;
        da.ld = db.ld = padded(f);
        da.p = pack.take(t, f);
        db.p = pack.take(t, f);
    }
    if (dx.p) {
        pwg = pack.usable(wg);
        pwu = pack.usable(wu);
    }
    if (dwg.p || dwu.p) px = pack.usable(x);
    if (dwd.p) ph = pack.usable(h);
    const Extent out{t, d};
    const Shape shape = dx.p ? pack.fit(choose(&out, 1, 2 * ceil_div(f, kBK), true, sms / 2), workspace_bytes) : Shape();
    Extent weights[3];
    int weight_count = 0;
    for (const Matrix *w : {&dwg, &dwu, &dwd}) {
        if (w->p) weights[weight_count++] = Extent{w->rows, w->cols};
    }
    const Shape weight_shape =
        weight_count ? pack.fit(choose(weights, weight_count, ceil_div(t, kBK), true, sms / 2), workspace_bytes) : Shape();
    if (!pack.fits(workspace_bytes)) return A2SGD_ERR_ARG;
    int rc = pack.run(sms, s);
    if (rc != A2SGD_OK) return rc;

    if (inner) {
        GemmArgs g{};
        Shape narrow; // half the columns where that still makes one round of tiles: twice the SMs bring in Wd
        if ((int64_t)ceil_div(t, kBM) * ceil_div(f, 128) <= sms / 2) narrow.bn = 128;
        set_shape(g, narrow, nullptr);
        if (!add_operands<false, true>(g, 0, pdy, pwd, dtype)) return A2SGD_ERR_CUDA;
        set_plain(g.out[0], da);
        set_plain(g.out2, db);
        set_plain(g.gate, pgate);
        set_plain(g.up, pup);
        const int tiles = add_problem(g, t, f, g.bn, 0, 1, d, 0);
        if (dx.p) bring_ahead(g, tiles, sms, pwg, &pwu);
        rc = act == A2SGD_ACT_SILU ? launch_gemm<T, kGateGrad, false, true, A2SGD_ACT_SILU>(g, tiles, sms, s)
                                   : launch_gemm<T, kGateGrad, false, true, A2SGD_ACT_GELU_TANH>(g, tiles, sms, s);
        if (rc != A2SGD_OK) return rc;
    }
    if (dx.p) {
        GemmArgs g{};
        set_shape(g, shape, reinterpret_cast<float *>(pack.at));
        if (!add_operands<false, true>(g, 0, da, pwg, dtype) || !add_operands<false, true>(g, 1, db, pwu, dtype) ||
            !set_rows(g.out[0], dx, dtype))
            return A2SGD_ERR_CUDA;
        rc = launch_gemm<T, kStore, false, true>(g, add_problem(g, t, d, g.bn, 0, 2, f, 0), sms, s);
        if (rc != A2SGD_OK) return rc;
    }
    if (weight_count) {
        GemmArgs g{};
        set_shape(g, weight_shape, reinterpret_cast<float *>(pack.at));
        int i = 0, tiles = 0;
        const auto add = [&](const Matrix &a, const Matrix &b, const Matrix &out) {
            if (!out.p) return true;
            if (!add_operands<true, true>(g, i, a, b, dtype) || !set_rows(g.out[i], out, dtype)) return false;
            tiles = add_problem(g, out.rows, out.cols, g.bn, i, 1, t, tiles);
            ++i;
            return true;
        };
        if (!add(da, px, dwg) || !add(db, px, dwu) || !add(pdy, ph, dwd)) return A2SGD_ERR_CUDA;
        rc = launch_gemm<T, kStore, true, true>(g, tiles, sms, s);
    }
    return rc;
}

int clear_rows(const Matrix &m, cudaStream_t s)
{
    if (m.p) A2_TRAIN_CUDA(cudaMemset2DAsync(const_cast<void *>(m.p), (size_t)(m.rows > 1 ? m.ld : m.cols) * 2, 0, (size_t)m.cols * 2, (size_t)m.rows, s));
    return A2SGD_OK;
}

} // namespace

extern "C" uint64_t a2sgd_gated_ffn_workspace(uint64_t tokens, uint32_t d, uint32_t f, uint32_t flags)
{
    const int64_t t = (int64_t)std::min<uint64_t>(tokens, 1ull << 30);
    uint64_t bytes = flags & A2SGD_FFN_BACKWARD ? 2 * room(t, f) : 0;
    if (!(flags & A2SGD_FFN_ALIGNED)) {
        bytes += 2 * room(f, d) + room(d, f) + room(t, f) + room(t, d); // Wg, Wu, Wd, h, x
        if (flags & A2SGD_FFN_BACKWARD) bytes += room(t, d) + 2 * room(t, f); // dy, gate, up
    }
    if (tokens) bytes += partial_bytes(kMostPairs, 256); // partial sums of tiles that are split, at the widest
    return bytes;
}

extern "C" int a2sgd_gated_ffn_forward(const void *x, int64_t x_stride, const void *w_gate, int64_t w_gate_stride,
                                       const void *w_up, int64_t w_up_stride, const void *w_down, int64_t w_down_stride,
                                       void *y, int64_t y_stride, void *hidden, int64_t hidden_stride, void *gate,
                                       int64_t gate_stride, void *up, int64_t up_stride, int dtype, int activation,
                                       uint64_t tokens, uint32_t d, uint32_t f, void *workspace, uint64_t workspace_bytes,
                                       int device, void *stream)
{
    int rc = check_sizes(tokens, d, f, dtype, activation);
    if (rc != A2SGD_OK || tokens == 0) return rc;
    const int64_t t = (int64_t)tokens;
    const Matrix mx{x, x_stride, t, (int)d}, mg{w_gate, w_gate_stride, f, (int)d}, mu{w_up, w_up_stride, f, (int)d},
        md{w_down, w_down_stride, d, (int)f}, my{y, y_stride, t, (int)d}, mh{hidden, hidden_stride, t, (int)f},
        ma{gate, gate_stride, t, (int)f}, mb{up, up_stride, t, (int)f};
    if (!gate != !up) return A2SGD_ERR_ARG;
    for (const Matrix *m : {&mx, &mg, &mu, &md, &my, &mh, &ma, &mb}) {
        rc = check(*m, m != &ma && m != &mb);
        if (rc != A2SGD_OK) return rc;
    }
    if (!aligned(workspace, 256)) return A2SGD_ERR_ALIGN;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms < 2) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == A2SGD_BF16
               ? forward<__nv_bfloat16>(mx, mg, mu, md, my, mh, ma, mb, activation, dtype, workspace, workspace_bytes, sms, s)
               : forward<__half>(mx, mg, mu, md, my, mh, ma, mb, activation, dtype, workspace, workspace_bytes, sms, s);
}

extern "C" int a2sgd_gated_ffn_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *w_gate,
                                        int64_t w_gate_stride, const void *w_up, int64_t w_up_stride, const void *w_down,
                                        int64_t w_down_stride, const void *hidden, int64_t hidden_stride, const void *gate,
                                        int64_t gate_stride, const void *up, int64_t up_stride, void *dx, int64_t dx_stride,
                                        void *dw_gate, int64_t dw_gate_stride, void *dw_up, int64_t dw_up_stride,
                                        void *dw_down, int64_t dw_down_stride, int dtype, int activation, uint64_t tokens,
                                        uint32_t d, uint32_t f, void *workspace, uint64_t workspace_bytes, int device,
                                        void *stream)
{
    int rc = check_sizes(tokens, d, f, dtype, activation);
    if (rc != A2SGD_OK) return rc;
    const int64_t t = (int64_t)tokens;
    const Matrix mdy{dy, dy_stride, t, (int)d}, mx{x, x_stride, t, (int)d}, mg{w_gate, w_gate_stride, f, (int)d},
        mu{w_up, w_up_stride, f, (int)d}, md{w_down, w_down_stride, d, (int)f}, mh{hidden, hidden_stride, t, (int)f},
        ma{gate, gate_stride, t, (int)f}, mb{up, up_stride, t, (int)f}, odx{dx, dx_stride, t, (int)d},
        odg{dw_gate, dw_gate_stride, f, (int)d}, odu{dw_up, dw_up_stride, f, (int)d}, odd{dw_down, dw_down_stride, d, (int)f};
    for (const Matrix *m : {&mdy, &mx, &mg, &mu, &md, &mh, &ma, &mb}) {
        rc = check(*m, tokens != 0);
        if (rc != A2SGD_OK) return rc;
    }
    for (const Matrix *m : {&odx, &odg, &odu, &odd}) {
        rc = check(*m, false);
        if (rc != A2SGD_OK) return rc;
    }
    if (!aligned(workspace, 256)) return A2SGD_ERR_ALIGN;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms < 2) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (tokens == 0) { // no tokens: the weights' gradients are zero
        for (const Matrix *m : {&odg, &odu, &odd}) {
            rc = clear_rows(*m, s);
            if (rc != A2SGD_OK) return rc;
        }
        return A2SGD_OK;
    }
    return dtype == A2SGD_BF16 ? backward<__nv_bfloat16>(mdy, mx, mg, mu, md, mh, ma, mb, odx, odg, odu, odd, activation, dtype,
                                                         workspace, workspace_bytes, sms, s)
                               : backward<__half>(mdy, mx, mg, mu, md, mh, ma, mb, odx, odg, odu, odd, activation, dtype,
                                                  workspace, workspace_bytes, sms, s);
}

extern "C" int a2sgd_gated_ffn_status(int device, int *device_status, void *stream)
{
    if (!device_status) return A2SGD_ERR_ARG;
    DeviceGuard guard(device);
    if (!guard.ok) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    unsigned int count = 0;
    A2_TRAIN_CUDA(cudaMemcpyFromSymbolAsync(&count, g_waits_run_out, sizeof count, 0, cudaMemcpyDeviceToHost, s));
    A2_TRAIN_CUDA(cudaStreamSynchronize(s));
    *device_status = count_moved(device, s, count, &g_waits_run_out) ? A2SGD_ERR_TIMEOUT : A2SGD_OK;
    return A2SGD_OK;
}
