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
// Rows whose address or stride is not a multiple of 16 bytes cannot be read by TMA; they are first
// copied to padded rows in the workspace.
#include "a2sgd_tcgen05.cuh"
#include "a2sgd_train.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <type_traits>

using namespace a2sgd_train;
using namespace a2sgd_tc;

namespace {

constexpr int kBM = 256;                  // rows of a tile, 128 a CTA
constexpr int kBK = 64;                   // depth of a slice: 128 bytes a row
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
constexpr uint32_t kABytes = 128 * kBK * 2; // A's slice in one CTA
constexpr uint32_t kTmemColumns = 512;

enum Epilogue { kStore = 0, kGate = 1, kGateGrad = 2 };

// Latched when a kernel's bounded wait ran out; read and cleared by a2sgd_gated_ffn_status.
__device__ int g_status = 0;

struct Problem {
    int m, n;          // rows and columns of the output
    int tiles_m, first; // tiles down, and this problem's first tile
    int seg, segs;     // operand pairs that are added up: a[seg], b[seg], ...
    void *out;
    int64_t ldo;
};

struct GemmArgs {
    CUtensorMap a[3], b[3];
    int k_blocks[3];
    Problem problem[3];
    int problems, tiles;
    int act;
    // kGate: out is h; these are optional.  kGateGrad: out is da, out2 db, gate and up are read.
    void *out2;       // kGate: a second copy of h (padded rows)
    int64_t ldo2;
    void *gate, *up;
    int64_t ld_gate, ld_up;
};

template <int BN>
struct Shape {
    static constexpr uint32_t kBBytes = (BN / 2) * kBK * 2;
    static constexpr uint32_t kStage = kABytes + kBBytes;
    static constexpr int kStages = BN == 256 ? 6 : 8;
    static constexpr uint32_t kBarriers = kStage * kStages;
    static constexpr uint32_t kSmem = kBarriers + 256 + 1024; // and the alignment of the first stage
};

// ------------------------------------------------------------------ activations
// value and slope share p = the sigmoid: silu(a) = a s(a); gelu in its tanh form is a s(2 k (a + c a^3)).
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
__device__ __forceinline__ void activation(int act, float a, float &value, float &slope)
{
    if (act == A2SGD_ACT_SILU) {
        const float p = sigmoid(a);
        value = a * p;
        slope = p * (1.0f + a * (1.0f - p));
    } else {
        constexpr float k2 = 1.5957691216057308f, c = 0.044715f;
        const float p = sigmoid(k2 * (a + c * a * a * a));
        value = a * p;
        const float pq = p * (1.0f - p);
        slope = pq == 0.0f ? p : p + a * pq * (k2 * (1.0f + 3.0f * c * a * a));
    }
}

// ------------------------------------------------------------------ global rows, 32 columns at a time
template <typename T>
__device__ __forceinline__ void store32(T *row, int column, int n, const float (&v)[32], bool vec)
{
    if (vec && column + 32 <= n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<uint4 *>(row + column + 8 * i) =
                make_uint4(pack2(v[8 * i], v[8 * i + 1], T()), pack2(v[8 * i + 2], v[8 * i + 3], T()),
                           pack2(v[8 * i + 4], v[8 * i + 5], T()), pack2(v[8 * i + 6], v[8 * i + 7], T()));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (column + i < n) row[column + i] = from_f32<T>(v[i]);
        }
    }
}
template <typename T>
__device__ __forceinline__ void load32(const T *row, int column, int n, float (&v)[32], bool vec)
{
    if (vec && column + 32 <= n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 q = *reinterpret_cast<const uint4 *>(row + column + 8 * i);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[8 * i + 2 * j] = lo_f32(w[j], T());
                v[8 * i + 2 * j + 1] = hi_f32(w[j], T());
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = column + i < n ? to_f32(row[column + i]) : 0.0f;
    }
}
__device__ __forceinline__ bool rows_vector(const void *p, int64_t ld) { return ((uintptr_t)p & 15u) == 0 && ld % 8 == 0; }

// ------------------------------------------------------------------ the product
template <typename T, int EPI, bool A_MN, bool B_MN, int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) k_gemm(const __grid_constant__ GemmArgs g)
{
    using S = Shape<BN>;
    extern __shared__ char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bars = base + S::kBarriers;
    const auto full = [&](int s) { return bars + 8u * s; };
    const auto empty = [&](int s) { return bars + 8u * (S::kStages + s); };
    const auto acc_full = [&](int i) { return bars + 8u * (2 * S::kStages + i); };
    const auto acc_empty = [&](int i) { return bars + 8u * (2 * S::kStages + 2 + i); };
    __shared__ uint32_t tmem_at;
    __shared__ volatile int gave_up;

    const uint32_t rank = cluster_rank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(acc_full(i), 1);
            bar_init(acc_empty(i), 2 * kEpilogueWarps);
        }
        gave_up = 0;
        bar_init_fence();
        for (int i = 0; i < 3; ++i) {
            tma_prefetch_map(&g.a[i]);
            tma_prefetch_map(&g.b[i]);
        }
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&tmem_at), kTmemColumns);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = tmem_at;
    wait_prior_grid();
    release_next_grid();

    const auto problem_of = [&](int tile) {
        int p = 0;
        while (p + 1 < g.problems && tile >= g.problem[p + 1].first) ++p;
        return p;
    };

    if (warp == 0 && lane == 0) {
        // ---------------------------------------------------------- operands in
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int tile = pair; ok && tile < g.tiles; tile += pairs) {
            const Problem &q = g.problem[problem_of(tile)];
            const int local = tile - q.first, tm = local % q.tiles_m, tn = local / q.tiles_m;
            const int row = tm * kBM + (int)rank * 128;
            const int col = EPI == kGate ? tn * 128 : tn * BN + (int)rank * (BN / 2);
            for (int seg = q.seg; ok && seg < q.seg + q.segs; ++seg) {
                const CUtensorMap *ma = &g.a[seg], *mb = EPI == kGate ? &g.b[rank] : &g.b[seg];
                for (int kb = 0; kb < g.k_blocks[seg]; ++kb) {
                    ok = bar_wait(empty(stage), phase ^ 1u, &gave_up);
                    if (!ok) break;
                    if (rank == 0) bar_expect(full(stage), 2 * S::kStage);
                    const uint32_t bar = map_to(full(stage), 0);
                    const uint32_t sa = base + stage * S::kStage, sb = sa + kABytes;
                    if constexpr (A_MN) {
                        tma_load_pair(sa, ma, row, kb * kBK, bar);
                        tma_load_pair(sa + 64 * kBK * 2, ma, row + 64, kb * kBK, bar);
                    } else {
                        tma_load_pair(sa, ma, kb * kBK, row, bar);
                    }
                    if constexpr (B_MN) {
#pragma unroll
                        for (int j = 0; j < BN / 128; ++j) tma_load_pair(sb + j * 64 * kBK * 2, mb, col + 64 * j, kb * kBK, bar);
                    } else {
                        tma_load_pair(sb, mb, kb * kBK, col, bar);
                    }
                    if (++stage == S::kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
        // every slice has been consumed: nothing is in flight towards this CTA any more
        for (int s = 0; ok && s < S::kStages; ++s) {
            ok = bar_wait(empty(stage), phase ^ 1u, &gave_up);
            if (++stage == S::kStages) {
                stage = 0;
                phase ^= 1u;
            }
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---------------------------------------------------------- products
        constexpr uint32_t kType = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
        constexpr uint32_t kDesc = instruction_desc(kType, A_MN, B_MN, kBM, BN);
        constexpr uint32_t kStepA = A_MN ? 16 * 128 : 32, kStepB = B_MN ? 16 * 128 : 32; // 16 of k further
        int stage = 0, turn = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int tile = pair; ok && tile < g.tiles; tile += pairs, ++turn) {
            const Problem &q = g.problem[problem_of(tile)];
            const int acc = turn & 1;
            ok = bar_wait(acc_empty(acc), ((turn >> 1) & 1) ^ 1, &gave_up);
            if (!ok) break;
            fence_after();
            const uint32_t d = tmem + acc * 256;
            bool add = false;
            for (int seg = q.seg; ok && seg < q.seg + q.segs; ++seg) {
                for (int kb = 0; kb < g.k_blocks[seg]; ++kb) {
                    ok = bar_wait(full(stage), phase, &gave_up);
                    if (!ok) break;
                    fence_after();
                    const uint32_t sa = base + stage * S::kStage, sb = sa + kABytes;
#pragma unroll
                    for (int k = 0; k < kBK / 16; ++k) {
                        mma_pair(d, operand_desc(sa + k * kStepA, A_MN ? 64 * kBK * 2 : 16),
                                 operand_desc(sb + k * kStepB, B_MN ? 64 * kBK * 2 : 16), kDesc, add);
                        add = true;
                    }
                    commit_pair(empty(stage));
                    if (++stage == S::kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
            commit_pair(acc_full(acc));
        }
    } else if (warp >= 2) {
        // ---------------------------------------------------------- accumulators out
        const uint32_t quarter = warp & 3, half = (warp - 2) >> 2; // a warp reads the TMEM lanes of its quarter
        int turn = 0;
        for (int tile = pair; tile < g.tiles; tile += pairs, ++turn) {
            const Problem &q = g.problem[problem_of(tile)];
            const int local = tile - q.first, tm = local % q.tiles_m, tn = local / q.tiles_m;
            const int acc = turn & 1;
            const int row = tm * kBM + (int)rank * 128 + quarter * 32 + lane;
            const bool live = row < q.m;
            if (!bar_wait(acc_full(acc), (turn >> 1) & 1, &gave_up)) break;
            fence_after();
            const uint32_t d = tmem + acc * 256 + (quarter * 32u << 16);
            if constexpr (EPI == kGate) {
                T *h = static_cast<T *>(q.out) + (int64_t)row * q.ldo;
                T *h2 = static_cast<T *>(g.out2) + (int64_t)row * g.ldo2;
                T *ga = static_cast<T *>(g.gate) + (int64_t)row * g.ld_gate;
                T *up = static_cast<T *>(g.up) + (int64_t)row * g.ld_up;
                const bool vh = rows_vector(q.out, q.ldo), vg = rows_vector(g.gate, g.ld_gate), vu = rows_vector(g.up, g.ld_up);
#pragma unroll 1
                for (int c = half * 64; c < (int)half * 64 + 64; c += 32) {
                    float a[32], b[32];
                    tmem_ld32(d + c, a);
                    tmem_ld32(d + 128 + c, b);
                    tmem_wait_ld();
                    const int column = tn * 128 + c;
                    if (live && g.gate) {
                        store32(ga, column, q.n, a, vg);
                        store32(up, column, q.n, b, vu);
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float value, slope;
                        activation(g.act, a[i], value, slope);
                        a[i] = value * b[i];
                    }
                    if (live) {
                        if (q.out) store32(h, column, q.n, a, vh);
                        if (g.out2) store32(h2, column, q.n, a, true);
                    }
                }
            } else if constexpr (EPI == kGateGrad) {
                T *da = static_cast<T *>(q.out) + (int64_t)row * q.ldo;
                T *db = static_cast<T *>(g.out2) + (int64_t)row * g.ldo2;
                const T *ga = static_cast<const T *>(g.gate) + (int64_t)row * g.ld_gate;
                const T *up = static_cast<const T *>(g.up) + (int64_t)row * g.ld_up;
                const bool vg = rows_vector(g.gate, g.ld_gate), vu = rows_vector(g.up, g.ld_up);
#pragma unroll 1
                for (int c = half * (BN / 2); c < (int)(half + 1) * (BN / 2); c += 32) {
                    float dh[32], a[32], b[32];
                    const int column = tn * BN + c;
                    tmem_ld32(d + c, dh);
                    if (live) {
                        load32(ga, column, q.n, a, vg);
                        load32(up, column, q.n, b, vu);
                    }
                    tmem_wait_ld();
                    if (live) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            float value, slope;
                            activation(g.act, a[i], value, slope);
                            a[i] = dh[i] * b[i] * slope;
                            b[i] = dh[i] * value;
                        }
                        store32(da, column, q.n, a, true);
                        store32(db, column, q.n, b, true);
                    }
                }
            } else {
                T *out = static_cast<T *>(q.out) + (int64_t)row * q.ldo;
                const bool vo = rows_vector(q.out, q.ldo);
#pragma unroll 1
                for (int c = half * (BN / 2); c < (int)(half + 1) * (BN / 2); c += 32) {
                    float v[32];
                    tmem_ld32(d + c, v);
                    tmem_wait_ld();
                    if (live) store32(out, tn * BN + c, q.n, v, vo);
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive_cluster(map_to(acc_empty(acc), 0));
        }
    }
    __syncwarp();
    __syncthreads();
    if (gave_up) {
        // leave the copies and products in flight a bounded time to end, and say so
        if (threadIdx.x == 0) atomicExch(&g_status, A2SGD_ERR_TIMEOUT);
        const uint64_t begin = now_ns();
        while (now_ns() - begin < 5000000ull) __nanosleep(1000);
    }
    cluster_sync();
    if (warp == 1) tmem_free_pair(tmem, kTmemColumns);
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
    PackJob job[6];
};
__global__ void __launch_bounds__(256) k_pack(const __grid_constant__ PackArgs a)
{
    wait_prior_grid();
    release_next_grid();
    const PackJob &j = a.job[blockIdx.y];
    for (int64_t r = blockIdx.x; r < j.rows; r += gridDim.x) {
        const uint16_t *s = j.src + r * j.ld_src;
        uint16_t *d = j.dst + r * j.ld_dst;
        for (int c = threadIdx.x; c < j.cols; c += 256) d[c] = s[c];
    }
}

// ------------------------------------------------------------------ host
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

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

template <typename T, int EPI, bool A_MN, bool B_MN, int BN>
int launch_gemm(GemmArgs &g, int sms, cudaStream_t s)
{
    const void *fn = reinterpret_cast<const void *>(&k_gemm<T, EPI, A_MN, B_MN, BN>);
    static std::atomic<uint64_t> allowed{0}; // devices on which this kernel may use its shared memory
    int device = 0;
    A2_TRAIN_CUDA(cudaGetDevice(&device));
    const uint64_t bit = 1ull << (device & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        A2_TRAIN_CUDA(cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<BN>::kSmem));
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    const unsigned pairs = (unsigned)std::min(g.tiles, sms / 2);
    void *params[] = {&g};
    A2_TRAIN_CUDA(launch(fn, dim3(2 * pairs), kThreads, Shape<BN>::kSmem, params, s));
    return A2SGD_OK;
}

// The maps of one operand pair.  An operand that is not transposed lies as [rows, k], a transposed one as [k, rows].
template <bool A_MN, bool B_MN, int BN>
bool add_operands(GemmArgs &g, int i, const Matrix &a, const Matrix &b, int64_t k, int dtype)
{
    g.k_blocks[i] = ceil_div(k, kBK);
    return make_map(&g.a[i], a, dtype, A_MN ? kBK : 128) && make_map(&g.b[i], b, dtype, B_MN ? kBK : BN / 2);
}

void add_problem(GemmArgs &g, int64_t m, int n, int tile_n, int seg, int segs, void *out, int64_t ldo)
{
    Problem &q = g.problem[g.problems++];
    q.m = (int)m;
    q.n = n;
    q.tiles_m = ceil_div(m, kBM);
    q.first = g.tiles;
    q.seg = seg;
    q.segs = segs;
    q.out = out;
    q.ldo = ldo;
    g.tiles += q.tiles_m * ceil_div(n, tile_n);
}

// Columns of a tile of a plain product: the width that leaves the tensor cores least idle, counting whole
// rounds of tiles over the pairs of SMs.
int tile_columns(int64_t m, int n, int sms)
{
    const int pairs = std::max(1, sms / 2);
    const int64_t rows = ceil_div(m, kBM);
    const int64_t wide = (rows * ceil_div(n, 256) + pairs - 1) / pairs * 256;
    const int64_t narrow = (rows * ceil_div(n, 128) + pairs - 1) / pairs * 128;
    return narrow < wide ? 128 : 256;
}

struct Packer {
    PackArgs args{};
    int jobs = 0;
    int64_t most_rows = 0;
    char *at;
    explicit Packer(void *workspace) : at(static_cast<char *>(workspace)) {}
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
        most_rows = std::max(most_rows, m.rows);
        return c;
    }
    int run(int sms, cudaStream_t s)
    {
        if (!jobs) return A2SGD_OK;
        void *params[] = {&args};
        A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_pack),
                             dim3((unsigned)std::min<int64_t>(most_rows, (int64_t)sms * 8), jobs), 256, 0, params, s));
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
    // tiles are counted in 32 bits
    if ((tokens / kBM + 1) * (std::max(d, f) / 128 + 1) >= (1ull << 30) || ((uint64_t)d / 128 + 1) * (f / 128 + 1) >= (1ull << 28))
        return A2SGD_ERR_TOO_LARGE;
    return A2SGD_OK;
}

template <typename T>
int forward(const Matrix &x, const Matrix &wg, const Matrix &wu, const Matrix &wd, Matrix y, Matrix h, Matrix gate, Matrix up, int act,
            int dtype, void *workspace, uint64_t workspace_bytes, int sms, cudaStream_t s)
{
    Packer pack(workspace);
    const Matrix px = pack.usable(x), pg = pack.usable(wg), pu = pack.usable(wu), pd = pack.usable(wd);
    Matrix ph = h; // what the second product reads
    if (!tma_ok(h)) {
        ph.ld = padded(h.cols);
        ph.p = pack.take(h.rows, h.cols);
    }
    const uint64_t need = (uint64_t)(pack.at - static_cast<char *>(workspace));
    if (need && (!workspace || workspace_bytes < need)) return A2SGD_ERR_ARG;
    int rc = pack.run(sms, s);
    if (rc != A2SGD_OK) return rc;
    const int64_t t = x.rows;
    const int d = x.cols, f = h.cols;

    GemmArgs g{};
    g.act = act;
    if (!add_operands<false, false, 256>(g, 0, px, pg, d, dtype) || !make_map(&g.b[1], pu, dtype, 128)) return A2SGD_ERR_CUDA;
    add_problem(g, t, f, 128, 0, 1, const_cast<void *>(h.p), h.ld);
    if (ph.p != h.p) {
        g.out2 = const_cast<void *>(ph.p);
        g.ldo2 = ph.ld;
    }
    g.gate = const_cast<void *>(gate.p);
    g.ld_gate = gate.ld;
    g.up = const_cast<void *>(up.p);
    g.ld_up = up.ld;
    rc = launch_gemm<T, kGate, false, false, 256>(g, sms, s);
    if (rc != A2SGD_OK) return rc;

    g = GemmArgs{};
    if (tile_columns(t, d, sms) == 256) {
        if (!add_operands<false, false, 256>(g, 0, ph, pd, f, dtype)) return A2SGD_ERR_CUDA;
        add_problem(g, t, d, 256, 0, 1, const_cast<void *>(y.p), y.ld);
        return launch_gemm<T, kStore, false, false, 256>(g, sms, s);
    }
    if (!add_operands<false, false, 128>(g, 0, ph, pd, f, dtype)) return A2SGD_ERR_CUDA;
    add_problem(g, t, d, 128, 0, 1, const_cast<void *>(y.p), y.ld);
    return launch_gemm<T, kStore, false, false, 128>(g, sms, s);
}

template <typename T, int BN>
int input_gradient(const Matrix &da, const Matrix &db, const Matrix &wg, const Matrix &wu, const Matrix &dx, int dtype, int sms,
                   cudaStream_t s)
{
    GemmArgs g{};
    if (!add_operands<false, true, BN>(g, 0, da, wg, da.cols, dtype) || !add_operands<false, true, BN>(g, 1, db, wu, db.cols, dtype))
        return A2SGD_ERR_CUDA;
    add_problem(g, dx.rows, dx.cols, BN, 0, 2, const_cast<void *>(dx.p), dx.ld);
    return launch_gemm<T, kStore, false, true, BN>(g, sms, s);
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
    Matrix da, db, pdy, pwd, pwg, pwu, px, ph;
    pdy = pack.usable(dy);
    if (inner) {
        pwd = pack.usable(wd);
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
    const uint64_t need = (uint64_t)(pack.at - static_cast<char *>(workspace));
    if (need && (!workspace || workspace_bytes < need)) return A2SGD_ERR_ARG;
    int rc = pack.run(sms, s);
    if (rc != A2SGD_OK) return rc;

    if (inner) {
        GemmArgs g{};
        g.act = act;
        if (!add_operands<false, true, 256>(g, 0, pdy, pwd, d, dtype)) return A2SGD_ERR_CUDA;
        add_problem(g, t, f, 256, 0, 1, const_cast<void *>(da.p), da.ld);
        g.out2 = const_cast<void *>(db.p);
        g.ldo2 = db.ld;
        g.gate = const_cast<void *>(gate.p);
        g.ld_gate = gate.ld;
        g.up = const_cast<void *>(up.p);
        g.ld_up = up.ld;
        rc = launch_gemm<T, kGateGrad, false, true, 256>(g, sms, s);
        if (rc != A2SGD_OK) return rc;
    }
    if (dx.p) {
        rc = tile_columns(t, d, sms) == 256 ? input_gradient<T, 256>(da, db, pwg, pwu, dx, dtype, sms, s)
                                            : input_gradient<T, 128>(da, db, pwg, pwu, dx, dtype, sms, s);
        if (rc != A2SGD_OK) return rc;
    }
    if (dwg.p || dwu.p || dwd.p) {
        GemmArgs g{};
        int i = 0;
        const auto add = [&](const Matrix &a, const Matrix &b, const Matrix &out) {
            if (!out.p) return true;
            if (!add_operands<true, true, 256>(g, i, a, b, t, dtype)) return false;
            add_problem(g, out.rows, out.cols, 256, i, 1, const_cast<void *>(out.p), out.ld);
            ++i;
            return true;
        };
        if (!add(da, px, dwg) || !add(db, px, dwu) || !add(pdy, ph, dwd)) return A2SGD_ERR_CUDA;
        rc = launch_gemm<T, kStore, true, true, 256>(g, sms, s);
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
        if (flags & A2SGD_FFN_BACKWARD) bytes += room(t, d);            // dy
    }
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
    if (sms == 0) return A2SGD_ERR_CUDA;
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
    if (sms == 0) return A2SGD_ERR_CUDA;
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
    const int zero = 0;
    A2_TRAIN_CUDA(cudaStreamSynchronize(s));
    A2_TRAIN_CUDA(cudaMemcpyFromSymbol(device_status, g_status, sizeof(int)));
    A2_TRAIN_CUDA(cudaMemcpyToSymbol(g_status, &zero, sizeof(int)));
    return A2SGD_OK;
}
