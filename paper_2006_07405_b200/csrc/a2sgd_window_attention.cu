// Attention with a sliding window and first tokens that stay visible, forward and backward.
//
//   forward    S = scale Q K^T where a query sees a key,  P = exp(S - lse),  lse = log sum exp S,  O = P V
//   backward   delta = sum_c dO O,  dP = dO V^T,  dS = P (dP - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// Three kernels: tiles of 128 queries on the tensor cores (k_forward), a few queries over a long cache (k_few), and the backward pass, twice the
// same template (k_backward).  S, dP, sums, references and outputs are fp32.  P and dS are rounded once to the 16-bit type, since they are operands
// of products of 16-bit values; the sum that divides P is taken before that rounding, so that a row's error is P's alone (half a step of each term).
// Scores are kept in units of log 2: one fused multiply-add and one exp2 an element.
//
// Every wait on an mbarrier ends after two seconds at most; the kernel then says so (a2sgd_window_attention_status) and leaves.
#include "a2sgd_tcgen05.cuh"
#include "a2sgd_train.cuh"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

using namespace a2sgd_train;
using namespace a2sgd_tc;

namespace {

struct Heads {
    void *p;
    int64_t seq, row, head;
};

struct Range {
    int first, count;
};
__device__ __forceinline__ Range range_of(const int32_t *ranges, int b, int rows)
{
    if (!ranges) return {0, rows};
    const int first = min(max(ranges[2 * b], 0), rows);
    return {first, min(max(ranges[2 * b + 1], 0), rows - first)};
}
template <typename T>
__device__ __forceinline__ T *at(const Heads &h, int b, int64_t row, int head)
{
    return static_cast<T *>(h.p) + (int64_t)b * h.seq + row * h.row + (int64_t)head * h.head;
}
// CTAs whose bounded wait ran out, since the library was loaded: only ever counted up.
__device__ unsigned int g_waits_run_out = 0;

constexpr float kLn2 = 0.6931471805599453f;
// log sum exp of a row that sees some key, from the sum about 2^ref.  No sum: every score was -infinity, and the softmax of that is not a number.
__device__ __forceinline__ float lse_from(float ref, float sum) { return sum > 0.0f ? (ref + log2f(sum)) * kLn2 : NAN; }

// ------------------------------------------------------------------ forward
// Persistent CTAs, two an SM, deal out the tiles of 128 queries of one head, the longest first.  For each tile a CTA walks the blocks of 64
// keys that any of its queries sees: the first tokens' blocks, then those of the window.  Warp 4 brings tiles, queries and keys in by TMA, warp 7 the
// values, warp 5 issues S = Q K^T, warp 6 O += P V, warps 0 to 3 hold the softmax, a thread a query.
//   S goes into TMEM;  a thread reads its row, forms P and writes it over S in 16 bits;  P is read from TMEM by its product with V.
// Three buffers of S (two where O has 128 columns): the next block's, be it the next tile's, is formed while the present one's P is.
// P is taken about a reference that is moved, and O and the sum with it, only where P would grow beyond a limit (Probabilities): nearly no
// block touches O, and blocks without a mask need no maximum.
//
// Bound, for heads of 64, by the softmax' warps: 16 exponentials a clock and SM are 164 us of 8 x 4096 queries, 25 heads of 64, window 1024 (737 M
// pairs), and with the loads from and stores to TMEM, the sums and the rounding to 16 bits a block takes a warp twice that; the products alone are
// 116 us.  B200: 349 us (541 TFLOP/s, tensor pipe 30 % busy); 20011 packed rows, 16 heads of 128, window 4096, float16: 234 us (838 TFLOP/s,
// 53 %); among other work 381 and 267.  One CTA an SM with 16 softmax warps, and every second exponential as a polynomial on the multiply-add pipe,
// measured the same; one loading warp for keys and values 6 % more, 16-byte stores 1 to 2 %.
struct ForwardArgs {
    CUtensorMap q, k, v;
    Heads o, values; // values: what v is read from
    float *lse;
    const int32_t *q_ranges, *k_ranges;
    int q_heads, group, d, q_rows, k_rows, window, sinks;
    int packed_q, q_planes, k_planes, v_planes; // planes: more than one: by sequence
    int sequences, tiles;                       // tiles of a sequence, or of all packed ones
    int items, lanes, together;                 // tiles of all heads; heads, times sequences that are not packed; of them at a time
    int wide_o;                                 // bytes of a store
    float scale_log2;
};

constexpr int kBlock = 64; // keys: of 128, two buffers of S and an O of 64 columns leave no second CTA on the SM
template <int D>
struct ForwardShape {
    static constexpr int kThreads = 256, kCtas = 2, kStages = D == 64 ? 4 : 2; // of keys, and of values
    static constexpr uint32_t kTile = (D / 64) * 16384u, kSlice = (D / 64) * 8192u; // 128 rows, 64 rows
    static constexpr uint32_t kSmem = kTile + 2 * kStages * kSlice + 1024;
    static constexpr int kBuffers = D == 64 ? 3 : 2; // of S
    static constexpr uint32_t kColumns = 256, kO = 64 * kBuffers;
};

// The sequence and the tile of `unit` rows that a CTA has among packed sequences; count 0: none.  One warp.
__device__ __forceinline__ void locate(const int32_t *ranges, int sequences, int rows, int unit, int target, int &seq, int &tile)
{
    const int lane = threadIdx.x & 31;
    seq = -1, tile = 0;
    for (int b0 = 0; b0 < sequences; b0 += 32) {
        const int b = b0 + lane;
        const int mine = b < sequences ? (range_of(ranges, b, rows).count + unit - 1) / unit : 0;
        int sum = mine;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, s);
            if (lane >= s) sum += v;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, sum > target);
        if (hit) {
            const int who = __ffs(hit) - 1;
            seq = b0 + who;
            tile = target - __shfl_sync(0xffffffffu, sum - mine, who);
            return;
        }
        target -= __shfl_sync(0xffffffffu, sum, 31);
    }
}

// The blocks of keys that a run of queries at places p0 to p1 (its last) sees, in order: sink_blocks first ones, then from first_block on.
struct Blocks {
    int sink_blocks, first_block, count;
    Blocks() = default;
    __device__ __forceinline__ Blocks(int p0, int p1, int window, int sinks, int block)
    {
        const int end = p1 < 0 ? 0 : p1 / block + 1, lo = max(0, p0 - window + 1);
        first_block = min(lo / block, end);
        sink_blocks = sinks > 0 ? min((sinks - 1) / block + 1, first_block) : 0;
        count = sink_blocks + end - first_block;
    }
    __device__ __forceinline__ int operator[](int n) const { return n < sink_blocks ? n : first_block + n - sink_blocks; }
};

__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Rows `valid` on of a tile of `rows` rows in shared memory are cleared: what lies behind a sequence may be anything, and zero times that
// is not zero.  The whole warp.
__device__ __forceinline__ void clear_rows(uint32_t tile, int chunks, int rows, int valid)
{
    for (int c = 0; c < chunks; ++c)
        for (int i = valid * 8 + (int)(threadIdx.x & 31); i < rows * 8; i += 32)
            st_shared(tile + (uint32_t)(c * rows * 128 + i * 16), make_uint4(0, 0, 0, 0));
    fence_async();
    __syncwarp();
}

// A hidden pair's P (or dS) is 0, and 0 times infinity is not a number: an operand that is not finite reaches rows that do not see it.  So a tile
// with an output that is not finite is done once more, with care: blocks that not every row sees are looked through before their product with P, what is
// not finite in them is put to 0, and the rows that do see it are given it by mend_row.  A tile without such an output pays for the question: 8 x 4096,
// 25 heads of 64, forward 345 -> 349 us, backward 1140 -> 1152, 5003 packed rows 3 us (looked through at once: 366, 1183 and 11 us).  With a first
// token's value, and 67 queries' gradients, not finite in every sequence: 1.2 ms and 2.8 ms.
constexpr int kAgain = 64;
struct Again { // in shared memory: the tiles to be done again, in turn
    int last;  // of those that have been put down, the tile's number among the CTA's
    volatile int count, items[kAgain];
    // One lane of each warp that has found something; a CTA's warps are never a tile apart.
    __device__ __forceinline__ void put(int tile, int item)
    {
        if (atomicMax(&last, tile) >= tile) return;
        items[count % kAgain] = item;
        __threadfence_block();
        count = count + 1;
    }
    // By the loading warp: whether the next tile is to be one of these, `done` of which have been taken; as long as there are others, not before half a list.
    __device__ __forceinline__ bool due(int done, bool others)
    {
        const int waiting = __shfl_sync(0xffffffffu, count, 0) - done;
        return waiting > 0 && (!others || waiting >= kAgain / 2);
    }
};
// Not a number where some element of v, of `count` that matter, is not finite.
__device__ __forceinline__ float judge(const float (&v)[32], int count)
{
    f32x2 z[2] = {};
    if (count >= 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 4) z[0] = fma2(pair(v[i], v[i + 1]), pair(0.0f), z[0]), z[1] = fma2(pair(v[i + 2], v[i + 3]), pair(0.0f), z[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 32; i += 2) z[0] = fma2(pair(i < count ? v[i] : 0.0f, i + 1 < count ? v[i + 1] : 0.0f), pair(0.0f), z[0]);
    }
    return sum2(add2(z[0], z[1]));
}
template <typename T>
__host__ __device__ constexpr uint32_t infinity_bits() { return std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u; }
__device__ __forceinline__ uint32_t larger_halves(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ void add_size(uint32_t &top, const uint4 &w)
{
    top = larger_halves(larger_halves(larger_halves(top, w.x & 0x7fff7fffu), w.y & 0x7fff7fffu), larger_halves(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
}
template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t sizes) { return (sizes & 0x7fffu) >= infinity_bits<T>() || (sizes >> 16 & 0x7fffu) >= infinity_bits<T>(); }
template <typename T>
__device__ __forceinline__ uint32_t finite_halves(uint32_t w)
{
    const uint32_t low = (w & 0x7fffu) >= infinity_bits<T>() ? 0u : w & 0xffffu, high = (w >> 16 & 0x7fffu) >= infinity_bits<T>() ? 0u : w & 0xffff0000u;
    return low | high;
}
// Of `pieces` times 16 bytes of shared memory.  The whole warp.
template <typename T>
__device__ __forceinline__ bool some_not_finite(uint32_t tile, int pieces)
{
    uint32_t top = 0;
#pragma unroll 8
    for (int i = threadIdx.x & 31; i < pieces; i += 32) add_size(top, ld_shared(tile + 16u * i));
    return __any_sync(0xffffffffu, not_finite<T>(top));
}
// Puts what is not finite in the 64 rows of a block, `chunks` times 128 bytes each, to 0; returns the rows that had some.  The whole warp.
template <typename T>
__device__ __forceinline__ uint64_t clear_not_finite(uint32_t tile, int chunks)
{
    uint32_t low = 0, high = 0;
#pragma unroll 1
    for (int i = threadIdx.x & 31; i < chunks * 512; i += 32) {
        const uint4 w = ld_shared(tile + 16u * i), f = make_uint4(finite_halves<T>(w.x), finite_halves<T>(w.y), finite_halves<T>(w.z), finite_halves<T>(w.w));
        if (f.x != w.x || f.y != w.y || f.z != w.z || f.w != w.w) {
            st_shared(tile + 16u * i, f);
            const int row = i >> 3 & 63;
            (row < 32 ? low : high) |= 1u << (row & 31);
        }
    }
    fence_async();
    low = __reduce_or_sync(0xffffffffu, low), high = __reduce_or_sync(0xffffffffu, high);
    return (uint64_t)high << 32 | low;
}
// The rows that were put to 0, of a tile's blocks, in shared memory: for who sees them.
constexpr int kMarred = 32;
struct Marred {
    int count; // beyond kMarred: all rows of all blocks may be
    int block[kMarred];
    uint64_t rows[kMarred];
    __device__ __forceinline__ void put(int n, int b, uint64_t r)
    {
        if (n < kMarred) block[n] = b, rows[n] = r;
    }
};
// Columns first to last (first a multiple of 8) of an output that this thread wrote, and of a row that it sees, in a tensor that TMA can read: what is not
// finite there is not finite here.  As a product with 0 < P: plus itself; with dS, whose sign may be any: not a number.  Returns whether no column
// is finite any more.
template <bool SIGNED, typename T, typename O>
__device__ __forceinline__ bool add_not_finite(O *out, const T *row, int first, int last)
{
    bool none = true;
    for (int c = first; c < last; c += 8) {
        if (c + 8 <= last) {
            uint32_t top = 0;
            add_size(top, *reinterpret_cast<const uint4 *>(row + c));
            if (!not_finite<T>(top)) {
                none = false;
                continue;
            }
        }
        for (int i = c; i < min(c + 8, last); ++i) {
            const float v = to_f32(row[i]), sum = isfinite(v) ? 0.0f : SIGNED ? to_f32(out[i]) + v : NAN;
            if (!isfinite(v)) out[i] = from_f32<O>(sum);
            none = none && !isfinite(v);
        }
    }
    return none;
}

// Up to 32 elements of a row: 32 or 16 bytes at a time (a thread's own sectors: 16-byte stores half fill them), or one element.
template <typename T>
__device__ __forceinline__ void store_row(T *p, const float *v, int count, int bytes)
{
    if (bytes == 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 16) {
            if (i >= count) break;
            uint32_t w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = pack2(v[i + 2 * k], v[i + 2 * k + 1], T());
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + i), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                         "r"(w[5]), "r"(w[6]), "r"(w[7])
                         : "memory");
        }
    } else if (bytes == 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (8 * i < count)
                *reinterpret_cast<uint4 *>(p + 8 * i) = make_uint4(pack2(v[8 * i], v[8 * i + 1], T()), pack2(v[8 * i + 2], v[8 * i + 3], T()),
                                                                   pack2(v[8 * i + 4], v[8 * i + 5], T()), pack2(v[8 * i + 6], v[8 * i + 7], T()));
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i < count) p[i] = from_f32<T>(v[i]);
    }
}

// The powers of 2 between which P is held: a reference is put so that its row's largest P is 2^(kFirst - 1) to 2^kFirst, and moved when one is above
// 2^kMost, or the sum over a block of 64 without a mask above 2^kSum (kMost + 6 at least, so that a block of equal scores does not ask for what does not
// come).  bfloat16 has fp32's range.  float16 loses what is below 2^-25, while the row's sum keeps it: P is lifted, so that this is 2^-31 of the
// largest, and 2^17 far keys take no more than 2^-14 from an output.  (Few queries: the maximum is known in every run of keys.)
template <typename T>
struct Probabilities {
    static constexpr float kFirst = 0.0f, kMost = 8.0f, kSum = 8192.0f, kMostFew = 8.0f;
};
template <>
struct Probabilities<__half> {
    static constexpr float kFirst = 7.0f, kMost = 9.0f, kSum = 32768.0f, kMostFew = 15.0f;
};

template <typename T>
__host__ __device__ constexpr uint32_t type_bits() { return std::is_same<T, __nv_bfloat16>::value ? 1u : 0u; }

// The largest of N numbers; those that are not numbers do not count.
template <int N>
__device__ __forceinline__ float most_of(const float *x)
{
    float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int i = 4; i < N; i += 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (i + j + 4 < N) asm("max.f32 %0, %0, %1, %2;" : "+f"(top[j]) : "f"(x[i + j]), "f"(x[i + j + 4]));
            else top[j] = fmaxf(top[j], x[i + j]);
        }
    }
    return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}
__device__ __forceinline__ void hide(float (&x)[32], uint32_t seen)
{
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = seen >> i & 1u ? x[i] : -INFINITY;
}
// 2^(x c + off) packed in 16 bits; returns their sum.
template <typename T>
__device__ __forceinline__ float exponentials(const float (&x)[32], float c, float off, uint32_t (&p)[16])
{
    const f32x2 c2 = pair(c), off2 = pair(off);
    f32x2 sums[4] = {};
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float x0, x1;
        unpair(fma2(pair(x[i], x[i + 1]), c2, off2), x0, x1);
        x0 = exp2_approx(x0), x1 = exp2_approx(x1);
        sums[i / 2 & 3] = add2(sums[i / 2 & 3], pair(x0, x1));
        p[i / 2] = pack2(x0, x1, T());
    }
    return sum2(add2(add2(sums[0], sums[1]), add2(sums[2], sums[3])));
}

// A tile: whose it is, its queries and the blocks of keys that they see.  The loading warp works them out and leaves them in shared memory.
struct Tile {
    int seq, head, p0, rows;     // place of the first query; queries, at least 1
    int q_row, k_row, k_count;   // rows of the plane, keys
    int item, careful;
    Blocks blocks;
    // Whether every query sees every key of the 64 from k0 on.
    __device__ __forceinline__ bool all_seen(int k0, int window, int sinks) const { return k0 + kBlock - 1 <= p0 && (k0 > p0 + rows - 1 - window || k0 + kBlock <= sinks); }
};
constexpr int kTiles = 8; // kept in shared memory, in turn (fewer than half of kAgain: as many may be put down while the loading warp does not look)
// The whole warp (packed sequences are searched through by its lanes).  False where there are no queries.
__device__ __forceinline__ bool find_tile(const ForwardArgs &a, int item, Tile &t)
{
    const int part = item / (a.together * a.tiles), rest = item - part * a.together * a.tiles;
    const int wide = min(a.together, a.lanes - part * a.together), lane = part * a.together + rest % wide;
    int tile = a.tiles - 1 - rest / wide;
    t.head = lane % a.q_heads;
    if (a.packed_q) {
        locate(a.q_ranges, a.sequences, a.q_rows, 128, tile, t.seq, tile);
        if (t.seq < 0) return false;
    } else {
        t.seq = lane / a.q_heads;
    }
    const Range qr = range_of(a.q_ranges, t.seq, a.q_rows), kr = range_of(a.k_ranges, t.seq, a.k_rows);
    t.rows = min(128, qr.count - tile * 128);
    if (t.rows <= 0) return false;
    t.p0 = tile * 128 + kr.count - qr.count;
    t.q_row = qr.first + tile * 128;
    t.k_row = kr.first;
    t.k_count = kr.count;
    t.blocks = Blocks(t.p0, t.p0 + t.rows - 1, a.window, a.sinks, kBlock);
    return true;
}
__device__ __forceinline__ int64_t lse_of(const ForwardArgs &a, const Tile &t, int row)
{
    return ((int64_t)(a.packed_q ? 0 : t.seq) * a.q_heads + t.head) * a.q_rows + t.q_row + row;
}

// What a query sees that is not finite, in blocks that not all of its tile's see.
template <typename T>
__device__ __noinline__ void mend_row(T *out, const ForwardArgs &a, const Tile &tile, int place, const Marred &marred)
{
    const T *values = at<T>(a.values, tile.seq, tile.k_row, tile.head / a.group);
    const bool listed = marred.count <= kMarred;
    for (int i = 0; i < (listed ? marred.count : tile.blocks.count); ++i) {
        const int k0 = tile.blocks[listed ? marred.block[i] : i] * kBlock;
        if (tile.all_seen(k0, a.window, a.sinks)) continue;
        for (uint64_t rows = listed ? marred.rows[i] : ~0ull; rows; rows &= rows - 1) {
            const int key = k0 + __ffsll((long long)rows) - 1;
            if (!(key <= place && (key > place - a.window || key < a.sinks))) continue;
            if (add_not_finite<true>(out, values + (int64_t)key * a.values.row, 0, a.d)) return;
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(ForwardShape<D>::kThreads, ForwardShape<D>::kCtas) k_forward(const __grid_constant__ ForwardArgs a)
{
    using Shape = ForwardShape<D>;
    constexpr int kStages = Shape::kStages, kChunks = D / 64, kBuffers = Shape::kBuffers;
    constexpr uint32_t kSlice = Shape::kSlice;
    extern __shared__ char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = base + Shape::kTile;
    __shared__ __align__(8) uint64_t bars[4 * kStages + 2 * kTiles + 5 + 3 * kBuffers];
    __shared__ Tile tiles[kTiles];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int gave_up;
    __shared__ Marred marred;
    __shared__ Again again;
    const uint32_t bar0 = smem_u32(bars);
    // keys' stages, then values'
    const auto full = [&](int s) { return bar0 + 8u * s; };
    const auto empty = [&](int s) { return bar0 + 8u * (2 * kStages + s); };
    const uint32_t tile0 = bar0 + 32u * kStages, more0 = tile0 + 16u * kTiles;
    const auto tile_full = [&](int t) { return tile0 + 8u * (t % kTiles); };
    const auto tile_empty = [&](int t) { return tile0 + 8u * (kTiles + t % kTiles); };
    const uint32_t q_full = more0, q_empty = more0 + 8, tail = more0 + 16, o_full = more0 + 24, o_empty = more0 + 32;
    const auto s_full = [&](int g) { return more0 + 40 + 8u * (g % kBuffers); };
    const auto p_full = [&](int g) { return more0 + 40 + 8u * (kBuffers + g % kBuffers); };
    const auto pv_done = [&](int g) { return more0 + 40 + 8u * (2 * kBuffers + g % kBuffers); };

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < 4 * kStages; ++s) bar_init(bar0 + 8u * s, 1);
        for (int t = 0; t < kTiles; ++t) {
            bar_init(tile_full(t), 1);
            bar_init(tile_empty(t), 6);
        }
        for (uint32_t b : {q_full, q_empty, tail}) bar_init(b, 1);
        bar_init(o_full, 2); // the products, and what is to be known about them
        bar_init(o_empty, 4);
        for (int i = 0; i < kBuffers; ++i) {
            bar_init(s_full(i), 1);
            bar_init(p_full(i), 4);
            bar_init(pv_done(i), 1);
        }
        gave_up = 0;
        again.last = -1, again.count = 0;
        bar_init_fence();
    }
    if (warp == 5) tmem_alloc(smem_u32(&tmem_at), Shape::kColumns);
    const int beyond = (int)threadIdx.x - 128;
    if (beyond >= 0 && beyond < 3 && a.k_rows > 0) tma_prefetch_map(beyond == 0 ? &a.q : beyond == 1 ? &a.k : &a.v); // parameters: no need to wait for the launch before
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_at;
    wait_prior_grid();
    release_next_grid(); // not before this CTA has its TMEM: the next kernel's CTAs may want some, and wait for this one's end

    if (warp == 4) {
        // ---------------------------------------------------------- tiles, queries and keys in
        const bool chosen = elect_one();
        int t = -1, g = 0, done_again = 0; // tiles and blocks so far
        bool ok = true, judged = false;
        for (int item = blockIdx.x; ok;) {
            Tile k;
            k.rows = k.blocks.count = 0;
            const bool others = item < a.items;
            if (!others && !judged) { // what the last tiles came out as
                for (int u = max(0, t - kTiles + 1); ok && u <= t; ++u) ok = bar_wait_cta(tile_empty(u), u / kTiles & 1, &gave_up);
                if (!ok) break;
                judged = true;
            }
            k.careful = again.due(done_again, others);
            const bool end = !others && !k.careful;
            k.item = k.careful ? again.items[done_again++ % kAgain] : item;
            if (!k.careful) item += gridDim.x;
            if (!end && !find_tile(a, k.item, k)) continue;
            if (!end && k.blocks.count == 0) { // queries that see nothing
                for (int r = 0; r < k.rows; ++r) {
                    T *o = at<T>(a.o, k.seq, k.q_row + r, k.head);
                    for (int c = lane; c < a.d; c += 32) o[c] = from_f32<T>(0.0f);
                    if (a.lse && lane == 0) a.lse[lse_of(a, k, r)] = -INFINITY;
                }
                continue;
            }
            ++t;
            ok = bar_wait_cta(tile_empty(t), (t / kTiles & 1) ^ 1, &gave_up);
            if (!ok) break;
            if (lane == 0) tiles[t % kTiles] = k;
            __syncwarp();
            if (chosen) bar_arrive(tile_full(t));
            __syncwarp();
            if (end) break;
            ok = bar_wait_cta(q_empty, (t & 1) ^ 1, &gave_up); // the last tile's queries have been read
            if (ok && chosen) {
                bar_expect(q_full, Shape::kTile);
                for (int c = 0; c < kChunks; ++c) tma_load4(base + c * 16384u, &a.q, 64 * c, k.q_row, k.head, a.q_planes > 1 ? k.seq : 0, q_full);
            }
            __syncwarp();
            const int head = k.head / a.group, plane = a.k_planes > 1 ? k.seq : 0;
            for (int n = 0; ok && n < k.blocks.count; ++n, ++g) {
                const int stage = g % kStages;
                ok = bar_wait_cta(empty(stage), (g / kStages & 1) ^ 1, &gave_up);
                if (ok && chosen) {
                    bar_expect(full(stage), kSlice);
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) tma_load4(ring + stage * kSlice + c * 8192u, &a.k, 64 * c, k.k_row + k.blocks[n] * kBlock, head, plane, full(stage));
                }
                __syncwarp();
            }
        }
        // every tile has been consumed: nothing is in flight towards this CTA any more
        for (int s = 0; ok && s < kStages; ++s) ok = bar_wait_cta(empty((g + s) % kStages), ((g + s) / kStages & 1) ^ 1, &gave_up);
    } else if (warp == 7) {
        // ---------------------------------------------------------- values in
        const bool chosen = elect_one();
        int g = 0;
        uint32_t tails = 0;
        bool ok = true;
        for (int t = 0; ok; ++t) {
            ok = bar_wait_cta(tile_full(t), t / kTiles & 1, &gave_up);
            if (!ok) break;
            const Tile v = tiles[t % kTiles];
            __syncwarp();
            if (chosen) bar_arrive(tile_empty(t));
            __syncwarp();
            if (v.rows == 0) break;
            const int head = v.head / a.group, plane = a.v_planes > 1 ? v.seq : 0;
            for (int n = 0; ok && n < v.blocks.count; ++n, ++g) {
                const int stage = kStages + g % kStages;
                const int block = v.blocks[n], valid = v.k_count - block * kBlock;
                const bool clear = a.k_ranges && valid < kBlock;
                const uint32_t dst = ring + stage * kSlice, bar = clear ? tail : full(stage);
                ok = bar_wait_cta(empty(stage), (g / kStages & 1) ^ 1, &gave_up);
                if (!ok) break;
                if (chosen) {
                    bar_expect(bar, kSlice);
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) tma_load4(dst + c * 8192u, &a.v, 64 * c, v.k_row + block * kBlock, head, plane, bar);
                }
                __syncwarp();
                if (clear) {
                    ok = bar_wait_cta(tail, tails & 1u, &gave_up);
                    ++tails;
                    if (!ok) break;
                    clear_rows(dst, kChunks, kBlock, valid);
                    if (chosen) bar_arrive(full(stage));
                    __syncwarp();
                }
            }
        }
        for (int s = 0; ok && s < kStages; ++s) ok = bar_wait_cta(empty(kStages + (g + s) % kStages), ((g + s) / kStages & 1) ^ 1, &gave_up);
    } else if (warp == 5) {
        // ---------------------------------------------------------- S = Q K^T, as far ahead as there are buffers
        const bool chosen = elect_one();
        const int steps = (a.d + 15) / 16; // of 16 elements of the head
        const uint32_t desc = instruction_desc(type_bits<T>(), false, false, 128, kBlock);
        const uint64_t dq = operand_desc(base, 16);
        int g = 0;
        bool ok = true;
        for (int t = 0; ok; ++t) {
            ok = bar_wait_cta(tile_full(t), t / kTiles & 1, &gave_up);
            const int count = ok ? tiles[t % kTiles].blocks.count : 0;
            if (count == 0) break;
            ok = bar_wait_cta(q_full, t & 1, &gave_up);
            for (int n = 0; ok && n < count; ++n, ++g) {
                const int stage = g % kStages;
                ok = bar_wait_cta(full(stage), g / kStages & 1, &gave_up);
                if (g >= kBuffers) ok = ok && bar_wait_cta(pv_done(g), (g / kBuffers + 1) & 1, &gave_up); // P has been read where S goes
                if (!ok) break;
                fence_after();
                if (chosen) {
                    const uint64_t dk = operand_desc(ring + stage * kSlice, 16);
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) // 64 elements a chunk
                        if (j < steps)
                            mma_ss(tmem + 64 * (g % kBuffers), dq + (((j >> 2) * 16384u + (j & 3) * 32u) >> 4), dk + (((j >> 2) * 8192u + (j & 3) * 32u) >> 4), desc, j > 0);
                    commit(s_full(g));
                    commit(empty(stage));
                    if (n + 1 == count) commit(q_empty);
                }
                __syncwarp();
            }
        }
    } else if (warp == 6) {
        // ---------------------------------------------------------- O += P V
        const bool chosen = elect_one();
        const uint32_t desc = instruction_desc(type_bits<T>(), false, true, 128, 0) | (uint32_t)(2 * ((a.d + 15) / 16)) << 17;
        int g = 0;
        bool ok = true;
        for (int t = 0; ok; ++t) {
            ok = bar_wait_cta(tile_full(t), t / kTiles & 1, &gave_up);
            const int count = ok ? tiles[t % kTiles].blocks.count : 0;
            if (count == 0) break;
            ok = bar_wait_cta(o_empty, (t & 1) ^ 1, &gave_up); // the last tile's output has been read
            const Tile &tile = tiles[t % kTiles];
            const bool careful = tile.careful;
            int bad = 0;
            for (int n = 0; ok && n < count; ++n, ++g) {
                const int stage = kStages + g % kStages;
                ok = bar_wait_cta(full(stage), g / kStages & 1, &gave_up);
                if (!ok) break;
                if (careful && !tile.all_seen(tile.blocks[n] * kBlock, a.window, a.sinks) && some_not_finite<T>(ring + stage * kSlice, (int)(kSlice / 16))) { // while P is formed
                    const uint64_t rows = clear_not_finite<T>(ring + stage * kSlice, kChunks);
                    if (chosen) marred.put(bad, n, rows);
                    ++bad;
                }
                ok = bar_wait_cta(p_full(g), g / kBuffers & 1, &gave_up);
                if (!ok) break;
                fence_after();
                if (chosen) {
                    const uint64_t dv = operand_desc(ring + stage * kSlice, 8192);
#pragma unroll
                    for (int j = 0; j < kBlock / 16; ++j)
                        mma_ts(tmem + Shape::kO, tmem + 64 * (g % kBuffers) + 8 * j, dv + j * (2048 >> 4), desc, n > 0 || j > 0);
                    commit(pv_done(g));
                    commit(empty(stage));
                    if (n + 1 == count) {
                        marred.count = bad;
                        bar_arrive(o_full);
                        commit(o_full);
                        bar_arrive(tile_empty(t));
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp < 4) {
        // ---------------------------------------------------------- softmax, a thread a query
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16), to = lanes + Shape::kO;
        const float c = a.scale_log2;
        int g = 0; // blocks so far
        for (int vt = 0;; ++vt) {
            bar_pass_cta(tile_full(vt), vt / kTiles & 1, &gave_up);
            if (__any_sync(0xffffffffu, gave_up)) break;
            const Tile tile = tiles[vt % kTiles];
            if (tile.rows == 0) break;
            const int row = warp * 32 + lane, place = tile.p0 + row;
            const int w0 = tile.p0 + warp * 32, w1 = w0 + 31; // the warp's places
            const bool live = row < tile.rows;
            // P = 2^(c s - ref); a row's reference is a whole number, so that what was summed about one is taken to another exactly
            float ref = live ? -INFINITY : 0.0f, total = 0.0f;
            bool ready = false; // every row of the warp has a reference
            const auto some_seen = [&](int g0) { return g0 <= w1 && (g0 + 31 > w0 - a.window || g0 < a.sinks); }; // of 32 keys, by the warp
            const auto seen_by = [&](int g0) { return below(place + 1 - g0) & (~below(place - a.window + 1 - g0) | below(a.sinks - g0)); };
            for (int n = 0; n < tile.blocks.count; ++n, ++g) {
                const int k0 = tile.blocks[n] * kBlock;
                const uint32_t ts = lanes + 64 * (g % kBuffers); // S, and P over it
                const bool inside = k0 + 63 <= w0 && (k0 > w1 - a.window || k0 + 63 < a.sinks); // every row sees all 64
                bar_pass_cta(s_full(g), g / kBuffers & 1, &gave_up);
                fence_after();
                bool done = false;
                if (inside && ready) {
                    // No maximum is taken: too large a sum says that the row has risen too far above its reference.
                    uint32_t p[32];
                    float x[32], y[32];
                    tmem_ld32(ts, x);
                    tmem_ld32(ts + 32, y);
                    tmem_wait_ld();
                    const float sum = exponentials<T>(x, c, -ref, reinterpret_cast<uint32_t(&)[16]>(p[0])) +
                                      exponentials<T>(y, c, -ref, reinterpret_cast<uint32_t(&)[16]>(p[16]));
                    done = !__any_sync(0xffffffffu, live && sum > Probabilities<T>::kSum);
                    if (done) {
                        tmem_st32(ts, p);
                        total += sum;
                    }
                }
                if (!done) {
                    // 32 keys at a time, read twice: for the maximum, and for P, which lies over scores that have been read
                    float top = -INFINITY;
#pragma unroll 1
                    for (int e = 0; e < 64; e += 32) {
                        if (!some_seen(k0 + e)) continue;
                        float x[32];
                        tmem_ld32(ts + e, x);
                        tmem_wait_ld();
                        hide(x, seen_by(k0 + e));
                        top = fmaxf(top, most_of<32>(x));
                    }
                    const float next = live && top * c > ref + Probabilities<T>::kMost ? ceilf(top * c) - Probabilities<T>::kFirst : ref;
                    const bool moves = next > ref;
                    if (__any_sync(0xffffffffu, moves)) {
                        const float shrink = moves ? exp2_approx(ref - next) : 1.0f; // 0 from -infinity
                        ref = next;
                        total *= shrink;
                        if (n > 0) {
                            bar_pass_cta(pv_done(g - 1), (g - 1) / kBuffers & 1, &gave_up); // O is at rest
                            fence_after();
#pragma unroll 1
                            for (int e = 0; 16 * e < a.d; ++e) {
                                uint32_t r[16];
                                tmem_ld16(to + 16 * e, r);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * shrink);
                                tmem_st16(to + 16 * e, r);
                            }
                        }
                    }
                    ready = __all_sync(0xffffffffu, ref != -INFINITY);
                    const float off = ref == -INFINITY ? 0.0f : -ref;
#pragma unroll 1
                    for (int e = 0; e < 64; e += 32) {
                        uint32_t p[16] = {};
                        if (some_seen(k0 + e)) {
                            float x[32];
                            tmem_ld32(ts + e, x);
                            tmem_wait_ld();
                            hide(x, seen_by(k0 + e));
                            total += exponentials<T>(x, c, off, p);
                        }
                        tmem_st16(ts + e / 2, p);
                    }
                }
                tmem_wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full(g));
            }
            const bool some = place >= 0; // the row sees a key: that at its own place, at least
            const float inverse = 1.0f / total; // not a number: neither is the output
            T *p = live ? at<T>(a.o, tile.seq, tile.q_row + row, tile.head) : nullptr;
            if (live && a.lse) a.lse[lse_of(a, tile, row)] = some ? lse_from(ref, total) : -INFINITY;
            bar_pass_cta(o_full, vt & 1, &gave_up);
            fence_after();
            const bool mend = tile.careful && marred.count;
            float sound = 0.0f;
#pragma unroll 1
            for (int e = 0; 32 * e < a.d; ++e) {
                float o[32];
                tmem_ld32(to + 32 * e, o);
                tmem_wait_ld();
                if (32 * e + 32 >= a.d) { // all of it has been read
                    fence_before();
                    __syncwarp();
                    if (lane == 0 && !mend) bar_arrive(o_empty);
                }
                sound += judge(o, a.d - 32 * e);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = some ? o[i] * inverse : 0.0f;
                if (live) store_row(p + 32 * e, o, a.d - 32 * e, a.wide_o);
            }
            if (mend) { // the next tile's list may not be begun before this one has been read
                if (live) mend_row(p, a, tiles[vt % kTiles], place, marred);
                __syncwarp();
                if (lane == 0) bar_arrive(o_empty);
            }
            if (__any_sync(0xffffffffu, live && sound != sound && total < INFINITY && !tile.careful) && lane == 0) again.put(vt, tile.item);
            __syncwarp();
            if (lane == 0) bar_arrive(tile_empty(vt));
        }
    }
    __syncwarp();
    __syncthreads();
    if (gave_up) {
        // leave the copies and products in flight a bounded time to end, and say so
        if (threadIdx.x == 0) atomicAdd(&g_waits_run_out, 1u);
        const uint64_t begin = now_ns();
        while (now_ns() - begin < 5000000ull) __nanosleep(1000);
    }
    if (warp == 5) tmem_free(tmem, Shape::kColumns);
}

// ------------------------------------------------------------------ few queries
// A query or a few over a long cache are bound by the cache's bytes.  A CTA takes up to 16 rows, the queries of all heads of one key
// head, and a share of the keys that they see; its warps take 16 keys at a time, each a run of its own, with mma.sync (m16n8k16): the
// scores leave a warp's registers as the left operand of P V.  Keys come by cp.async into places that the lane alone reads: the order of a head's elements is
// free as long as q has the same.  Values come in rows, and through ldmatrix.trans.  Every warp has its own maximum, sum and output; they meet in shared
// memory, and those of a row's CTAs in that of a cluster's CTA, or beyond eight CTAs in memory and a second launch.
//
// B200: 64 sequences, 32 heads of 128, 8 key heads, 4112 of 8192 keys visible, 1079 MB: 171 us (6.3 TB/s, 96 % of a copy's), among other work 182.
// 4 sequences, 25 heads of 64, 1028 keys, 26 MB: 10.8 us on the device, 11 to 13.5 a call: 2 until the first keys are asked for, 5 until the last are
// used, 1.2 and 0.9 for the two joins (with threads of eight columns each, and a cluster's CTAs reading one another, 13.0 us); the call itself is 10.5
// us on the host.
// 1 sequence, 32 heads of 128, 8 key heads: 8192 keys (34 MB) 14.4 us, 131072 keys (537 MB) 77 us (7.0 TB/s: part of it stays in L2).
constexpr int kFewRows = 16, kFewKeys = 16, kFewCluster = 8, kMostShares = 320; // the last: CTAs of a call whose rows are shared out beyond a cluster
template <int D>
struct FewShape {
    static constexpr int kWarps = D == 64 ? 8 : 4, kStages = 3;
    static constexpr int kRow = D + 2, kPartial = kFewRows * kRow; // floats of a row's share: outputs, reference (log 2), sum
    static constexpr uint32_t kKeys = kFewKeys * D * 2, kStage = 2 * kKeys, kRing = kWarps * kStages * kStage;
    static constexpr uint32_t kSmem = kRing + (kFewRows + kFewCluster - 1) * kRow * 4; // with a cluster's shares of this CTA's rows
};
struct FewArgs {
    Heads q, k, v, o;
    float *lse, *partials;
    const int32_t *q_ranges, *k_ranges;
    int q_heads, kv_heads, group, d, q_rows, k_rows, window, sinks;
    int tiles, shares, cluster; // of 16 rows; of a row's keys, which are a cluster's CTAs
    float scale_log2;
};

template <typename T>
__device__ __forceinline__ void mma_rows(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
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
__device__ __forceinline__ void load_transposed(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}

// Column c of a row's shares, sums about different references, joined: at(k, i) is float i of the row in share k of `n`.
struct Joined {
    float out, ref, sum;
};
template <int D, typename At>
__device__ __forceinline__ Joined join(const At &at_share, int n, int c)
{
    Joined x{0.0f, -INFINITY, 0.0f};
#pragma unroll 8
    for (int k = 0; k < n; ++k) x.ref = fmaxf(x.ref, at_share(k, D));
#pragma unroll 8
    for (int k = 0; k < n; ++k) {
        const float ref = at_share(k, D), f = exp2_approx(ref - x.ref), sum = at_share(k, D + 1), out = at_share(k, c);
        if (ref != -INFINITY || sum != 0.0f) { // else it has seen nothing; scores that are not numbers leave no reference, but a sum
            x.sum = fmaf(f, sum, x.sum);
            x.out = fmaf(f, out, x.out);
        }
    }
    return x;
}
template <typename T>
__device__ __forceinline__ void put_joined(const FewArgs &a, const Range &qr, int ahead, int seq, int kv, int tile, int r, int c, const Joined &x)
{
    const int row = tile * kFewRows + r, t = row / a.group, head = kv * a.group + row - t * a.group;
    const bool some = t + ahead >= 0; // the key at its own place, at least
    if (c < a.d) at<T>(a.o, seq, qr.first + t, head)[c] = from_f32<T>(some ? x.out / x.sum : 0.0f);
    if (a.lse && c == 0) a.lse[((int64_t)seq * a.q_heads + head) * a.q_rows + qr.first + t] = some ? lse_from(x.ref, x.sum) : -INFINITY;
}

template <typename T, int D>
__global__ void __launch_bounds__(32 * FewShape<D>::kWarps) k_few(const __grid_constant__ FewArgs a)
{
    using Shape = FewShape<D>;
    constexpr int kSteps = D / 32, kPieces = D / 8;
    extern __shared__ __align__(128) char smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, c = lane & 3;
    const int tile = blockIdx.x / a.shares, share = blockIdx.x - tile * a.shares, kv = blockIdx.y, seq = blockIdx.z;
    if (a.cluster) cluster_arrive(); // has begun: its memory may be written to
    wait_prior_grid();
    release_next_grid();
    const Range qr = range_of(a.q_ranges, seq, a.q_rows), kr = range_of(a.k_ranges, seq, a.k_rows);
    const int rows = min(kFewRows, qr.count * a.group - tile * kFewRows), ahead = kr.count - qr.count;
    // what some row sees: the first tokens up to `first`, and the keys from lo to end
    const int t0 = tile * kFewRows / a.group, t1 = rows > 0 ? (tile * kFewRows + rows - 1) / a.group : t0;
    int lo = max(0, t0 + ahead - a.window + 1), first = min(a.sinks, lo);
    const int end = rows > 0 ? max(0, t1 + ahead + 1) : 0;
    if (first == lo) lo = first = 0; // one run
    first = min(first, end);
    const int units0 = (first + kFewKeys - 1) / kFewKeys, units = units0 + (max(0, end - lo) + kFewKeys - 1) / kFewKeys;
    const int worker = share * Shape::kWarps + warp, workers = a.shares * Shape::kWarps;
    const int each = units / workers, rest = units - each * workers, u0 = each * worker + min(worker, rest), u1 = u0 + each + (worker < rest);

    const uint32_t mine = smem_u32(smem_raw) + warp * Shape::kStages * Shape::kStage;
    // a lane's pieces of a run: keys quad and quad + 8, elements 8 c and every 32 on; values: elements 8 e of every (32 / kPieces)th row
    const int e = lane % kPieces, r0 = lane / kPieces;
    const T *keys = at<T>(a.k, seq, kr.first, kv), *values = at<T>(a.v, seq, kr.first, kv);
    const T *lane_keys = keys + (int64_t)quad * a.k.row + 8 * c, *lane_values = values + (int64_t)r0 * a.v.row + 8 * e;
    const int64_t keys8 = 8 * a.k.row, values_step = (32 / kPieces) * a.v.row;
    const int value_bytes = 2 * max(0, min(8, a.d - 8 * e));
    const auto bring = [&](int u, int stage) {
        if (u < u1) {
            const int k0 = u < units0 ? u * kFewKeys : lo + (u - units0) * kFewKeys, left = (u < units0 ? first : end) - k0;
            const uint32_t place = mine + stage * Shape::kStage + lane * 16, value_place = mine + stage * Shape::kStage + Shape::kKeys;
            const T *k = lane_keys + (int64_t)k0 * a.k.row, *v = lane_values + (int64_t)k0 * a.v.row;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const bool in = quad + 8 * n < left;
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int there = in ? 2 * max(0, min(8, a.d - 32 * s - 8 * c)) : 0;
                    async_copy16(place + (n * kSteps + s) * 512, there ? k + n * keys8 + 32 * s : keys, there);
                }
            }
#pragma unroll
            for (int i = 0; i < kPieces / 2; ++i) {
                const int r = i * (32 / kPieces) + r0, there = r < left ? value_bytes : 0;
                async_copy16(value_place + r * (D * 2) + ((e ^ (r & 7)) << 4), there ? v + i * values_step : values, there);
            }
        }
        async_commit();
    };
#pragma unroll
    for (int i = 0; i < Shape::kStages - 1; ++i) bring(u0 + i, i); // the long way is memory's: q comes meanwhile

    // q: rows quad and quad + 8, elements 32 s + 8 c on
    uint32_t q[kSteps][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = tile * kFewRows + quad + 8 * h, t = r / a.group;
        const bool live = quad + 8 * h < rows;
        const uint16_t *p = live ? at<uint16_t>(a.q, seq, qr.first + t, kv * a.group + r - t * a.group) : nullptr;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            uint32_t w[4] = {0, 0, 0, 0};
            const int at0 = 32 * s + 8 * c;
            if (live && at0 + 8 <= a.d) {
                const uint4 x = *reinterpret_cast<const uint4 *>(p + at0);
                w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
            } else if (live) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (at0 + i < a.d) w[i / 2] |= (uint32_t)p[at0 + i] << (16 * (i & 1));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) q[s][2 * i + h] = w[i];
        }
    }
    float o[kPieces][4] = {}, ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};
    const int place0 = (tile * kFewRows + quad) / a.group + ahead, place1 = (tile * kFewRows + quad + 8) / a.group + ahead;
    const float cl = a.scale_log2;
    int stage = 0;
    for (int u = u0; u < u1; ++u) {
        async_wait<Shape::kStages - 2>();
        __syncwarp();
        const uint32_t place = mine + stage * Shape::kStage;
        {
            const int ahead_stage = stage == 0 ? Shape::kStages - 1 : stage - 1; // the one before: read by all lanes
            bring(u + Shape::kStages - 1, ahead_stage);
        }
        float s[2][4] = {};
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int x = 0; x < kSteps; ++x) {
                const uint4 b = ld_shared(place + ((n * kSteps + x) * 32 + lane) * 16);
                mma_rows<T>(s[n], q[x][0], q[x][1], q[x][2], q[x][3], b.x, b.y);
                mma_rows<T>(s[n], q[x][4], q[x][5], q[x][6], q[x][7], b.z, b.w);
            }
        }
        const int k0 = u < units0 ? u * kFewKeys : lo + (u - units0) * kFewKeys, stop = u < units0 ? first : end;
        const bool all = k0 + kFewKeys <= stop && k0 + kFewKeys - 1 <= t0 + ahead && (k0 > t1 + ahead - a.window || k0 + kFewKeys <= a.sinks);
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!all) {
                    const int key = k0 + 8 * n + 2 * c + (i & 1), at_place = i < 2 ? place0 : place1;
                    if (key >= stop || !(key <= at_place && (key > at_place - a.window || key < a.sinks))) s[n][i] = -INFINITY;
                }
                top[i >> 1] = fmaxf(top[i >> 1], s[n][i]);
            }
        float shrink[2];
        bool moves = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
            top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2)) * cl;
            shrink[h] = 1.0f;
            if (top[h] > ref[h] + Probabilities<T>::kMostFew) { // from -infinity, too
                const float next = top[h] - Probabilities<T>::kFirst;
                shrink[h] = exp2_approx(ref[h] - next);
                ref[h] = next;
                moves = true;
            }
        }
        if (__any_sync(0xffffffffu, moves)) {
            sum[0] *= shrink[0], sum[1] *= shrink[1];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) o[j][0] *= shrink[0], o[j][1] *= shrink[0], o[j][2] *= shrink[1], o[j][3] *= shrink[1];
        }
        const float off0 = ref[0] == -INFINITY ? 0.0f : -ref[0], off1 = ref[1] == -INFINITY ? 0.0f : -ref[1];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[n][i] = exp2_approx(fmaf(s[n][i], cl, i < 2 ? off0 : off1));
            sum[0] += s[n][0] + s[n][1];
            sum[1] += s[n][2] + s[n][3];
        }
        if (!all) { // as in the kernel for many queries
            const uint32_t values_at = place + Shape::kKeys;
            uint32_t sizes = 0;
#pragma unroll
            for (int i = 0; i < kPieces / 2; ++i) {
                const int r = i * (32 / kPieces) + r0;
                add_size(sizes, ld_shared(values_at + r * (D * 2) + ((e ^ (r & 7)) << 4)));
            }
            if (__any_sync(0xffffffffu, not_finite<T>(sizes))) {
#pragma unroll 1
                for (int r = 0; r < kFewKeys && k0 + r < stop; ++r) {
                    const int key = k0 + r;
                    const bool sees0 = key <= place0 && (key > place0 - a.window || key < a.sinks), sees1 = key <= place1 && (key > place1 - a.window || key < a.sinks);
#pragma unroll
                    for (int j = 0; j < kPieces; ++j) {
                        const uint32_t w = ld_shared32(values_at + r * (D * 2) + ((j ^ (r & 7)) << 4) + 4 * c);
                        const float x = lo_f32(w, T()), y = hi_f32(w, T());
                        if (!isfinite(x)) o[j][0] += sees0 ? x : 0.0f, o[j][2] += sees1 ? x : 0.0f;
                        if (!isfinite(y)) o[j][1] += sees0 ? y : 0.0f, o[j][3] += sees1 ? y : 0.0f;
                    }
                }
                __syncwarp();
#pragma unroll 1
                for (int i = 0; i < kPieces / 2; ++i) {
                    const int r = i * (32 / kPieces) + r0;
                    const uint32_t piece = values_at + r * (D * 2) + ((e ^ (r & 7)) << 4);
                    const uint4 w = ld_shared(piece);
                    st_shared(piece, make_uint4(finite_halves<T>(w.x), finite_halves<T>(w.y), finite_halves<T>(w.z), finite_halves<T>(w.w)));
                }
                __syncwarp();
            }
        }
        const uint32_t a0 = pack2(s[0][0], s[0][1], T()), a1 = pack2(s[0][2], s[0][3], T()), a2 = pack2(s[1][0], s[1][1], T()), a3 = pack2(s[1][2], s[1][3], T());
        const int r = lane & 15; // the row whose address this lane gives: keys 0 to 15, twice
#pragma unroll
        for (int j = 0; j < kPieces; j += 2) {
            uint32_t b[4];
            load_transposed(place + Shape::kKeys + r * (D * 2) + (((j + (lane >> 4)) ^ (r & 7)) << 4), b);
            mma_rows<T>(o[j], a0, a1, a2, a3, b[0], b[1]);
            mma_rows<T>(o[j + 1], a0, a1, a2, a3, b[2], b[3]);
        }
        __syncwarp();
        if (++stage == Shape::kStages) stage = 0;
    }
    async_wait<0>();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
    }
    __syncthreads(); // the keys' places are free
    float *parts = reinterpret_cast<float *>(smem_raw), *own = parts + warp * Shape::kPartial;
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) *reinterpret_cast<float2 *>(own + (quad + 8 * h) * Shape::kRow + 8 * j + 2 * c) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
    if (c == 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) *reinterpret_cast<float2 *>(own + (quad + 8 * h) * Shape::kRow + D) = make_float2(ref[h], sum[h]);
    }
    __syncthreads();
    // the warps' sums are joined, a thread a column of a row; then, if other CTAs have shares of the row, they go to the CTA of the cluster that
    // joins this row, or to memory
    const int slots = (kFewRows + a.shares - 1) / a.shares; // rows that a CTA of a cluster joins
    const uint32_t got = smem_u32(smem_raw) + Shape::kRing;
    if (a.cluster) cluster_wait();
    for (int i = threadIdx.x; i < rows * D; i += 32 * Shape::kWarps) {
        const int r = i / D, col = i % D;
        const Joined x = join<D>([&](int k, int f) { return parts[k * Shape::kPartial + r * Shape::kRow + f]; }, Shape::kWarps, col);
        if (a.shares == 1) {
            put_joined<T>(a, qr, ahead, seq, kv, tile, r, col, x);
        } else if (a.cluster) {
            const int slot = r / a.shares;
            const uint32_t to = map_to(got + 4u * ((share * slots + slot) * Shape::kRow), r - slot * a.shares);
            st_cluster(to + 4u * col, x.out);
            if (col == 0) {
                st_cluster(to + 4u * D, x.ref);
                st_cluster(to + 4u * (D + 1), x.sum);
            }
        } else {
            float *to = a.partials + (((int64_t)seq * a.kv_heads + kv) * gridDim.x + blockIdx.x) * Shape::kPartial + r * Shape::kRow;
            to[col] = x.out;
            if (col == 0) to[D] = x.ref, to[D + 1] = x.sum;
        }
    }
    if (!a.cluster) return;
    __syncwarp();
    cluster_sync();
    const float *shares = reinterpret_cast<const float *>(smem_raw + Shape::kRing);
    for (int i = threadIdx.x; i < slots * D; i += 32 * Shape::kWarps) {
        const int slot = i / D, r = slot * a.shares + share;
        if (r >= rows) break;
        put_joined<T>(a, qr, ahead, seq, kv, tile, r, i % D, join<D>([&](int k, int f) { return shares[(k * slots + slot) * Shape::kRow + f]; }, a.shares, i % D));
    }
}
// The shares of a row that are more than a cluster's: a CTA a row, a thread a column, the shares' factors in shared memory.
constexpr int kJoinThreads = 128;
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) k_few_join(const __grid_constant__ FewArgs a)
{
    using Shape = FewShape<D>;
    constexpr int kWarps = kJoinThreads / 32;
    __shared__ float refs[kMostShares], factors[kMostShares], tops[kWarps], sums[kWarps];
    wait_prior_grid();
    release_next_grid();
    const int tile = blockIdx.x / kFewRows, r = blockIdx.x % kFewRows, kv = blockIdx.y, seq = blockIdx.z, n = a.shares;
    const Range qr = range_of(a.q_ranges, seq, a.q_rows);
    if (r >= qr.count * a.group - tile * kFewRows) return;
    const float *parts = a.partials + (((int64_t)seq * a.kv_heads + kv) * a.tiles + tile) * n * Shape::kPartial + r * Shape::kRow;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Joined x{0.0f, -INFINITY, 0.0f};
    for (int k = threadIdx.x; k < n; k += kJoinThreads) {
        refs[k] = parts[k * Shape::kPartial + D];
        x.ref = fmaxf(x.ref, refs[k]);
    }
#pragma unroll
    for (int m = 16; m; m >>= 1) x.ref = fmaxf(x.ref, __shfl_xor_sync(0xffffffffu, x.ref, m));
    if (lane == 0) tops[warp] = x.ref;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) x.ref = fmaxf(x.ref, tops[w]);
    for (int k = threadIdx.x; k < n; k += kJoinThreads) {
        const float sum = parts[k * Shape::kPartial + D + 1];
        const bool some = refs[k] != -INFINITY || sum != 0.0f; // as in join
        factors[k] = some ? exp2_approx(refs[k] - x.ref) : -1.0f;
        if (some) x.sum = fmaf(factors[k], sum, x.sum);
    }
#pragma unroll
    for (int m = 16; m; m >>= 1) x.sum += __shfl_xor_sync(0xffffffffu, x.sum, m);
    if (lane == 0) sums[warp] = x.sum;
    __syncthreads();
    x.sum = sums[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) x.sum += sums[w];
    if (threadIdx.x >= D) return;
#pragma unroll 16
    for (int k = 0; k < n; ++k) {
        const float out = parts[k * Shape::kPartial + (int)threadIdx.x];
        if (!(factors[k] < 0.0f)) x.out = fmaf(factors[k], out, x.out);
    }
    put_joined<T>(a, qr, range_of(a.k_ranges, seq, a.k_rows).count - qr.count, seq, kv, tile, r, threadIdx.x, x);
}

struct DeltaArgs {
    Heads o, dout;
    const float *lse;
    float *lse2, *delta;
    int64_t rows;
    unsigned int *next; // two, cleared
    int blocks, heads, d, wide; // CTAs of a plane
    // packed queries whose first tokens' passes are cut into parts (see PartsList)
    const int32_t *q_ranges, *k_ranges;
    int *list;
    int sequences, k_rows, group, part_blocks, more, listed;
};

// ------------------------------------------------------------------ backward
// Two launches of one template, so that each output is added up by one CTA, in order, and the same call gives the same bits.  (S and dP are formed twice:
// 14 D operations a pair in place of 10, and two exponentials in place of one.  One launch would have to keep dq's parts and join them in order.)
//   KEYS false: 128 queries stay, blocks of 64 keys pass:        dQ += dS K
//   KEYS true:  128 keys stay, blocks of 64 queries pass, of all query heads of the key head:   dK += dS^T Q,  dV += P^T dO
// In either, with A, A' the tiles that stay and B, B' those that pass:  S = A B^T, dP = A' B'^T into TMEM; a thread reads its row, forms
// P = exp(scale S - lse) and dS = P (dP - delta) and writes them over S and dP in 16 bits; then out += dS B, out' += P B'.
// Roles and tiles as in the forward pass, one CTA an SM, with three buffers of S and dP (two where dK and dV of 128 elements leave no more) and
// two groups of four warps, each with half of a block.
// The first tokens' keys are seen by every query: their tiles' passes are cut into parts, whose sums are joined in order by k_fold_keys.  Sequences of packed
// queries are cut by their own lengths, which the device knows: see PartsList.
//
// Bound by the softmax' warps and what lies between them and the products: S and dP come out of TMEM, P and dS go back, 1100 to 1400 clocks a block of
// 64, in which the products take 611 and the exponentials 560.  B200, 8 x 4096 queries, 25 heads of 64, window 1024: 1152 us (409 TFLOP/s of the 10 D
// operations a pair), among other work 1230; by themselves, cold, dk and dv 653, dq 500, delta 55, the fold 5.  5003 packed rows, 12 heads of 80: 77
// us.  CTAs take their tiles from a counter, and dq's begin where dk and dv's end (tiles dealt out by number, dq first: 113 us for the packed rows, 1 %
// more for the others; one launch after the other 118, and 3 %).  Which
// CTA has a tile changes nothing in its result.  Measured and not taken: blocks of 128 with places of their own for P and dS (1240 us: one buffer
// only), 16 softmax warps, two CTAs an SM, exponentials by polynomials (no change).
struct BackwardArgs {
    CUtensorMap stay0, stay1, pass0, pass1;
    Heads out0, out1; // dq; or dk, dv
    Heads passing;    // what k, or dout, is read from
    int wide0, wide1;
    const float *lse2, *delta; // [q_heads][q_rows] a plane: log2 e times lse, delta
    float *partials;           // rows of dk and of dv, [2][D] each: see partial_row
    const int32_t *q_ranges, *k_ranges;
    int q_heads, kv_heads, group, d, q_rows, k_rows, window, sinks;
    int packed_q, packed_k, sequences; // packed_q: one plane of lse2 and delta
    int stay0_planes, stay1_planes, pass0_planes, pass1_planes;
    int tiles, lanes, items, together;
    int parts, part_blocks, sink_tiles, sink_rows, extra; // parts of a first tokens' tile, blocks of each; tiles and keys; items of a lane beyond its tiles
    const int *list;   // packed queries: PartsList, and then `extra` are a key head's and come before all others
    int listed, slots; // room in it; parts of a key head that it can have
    unsigned int *next; // items taken beyond every CTA's first one
    int beside;         // dq: the launch before is that of dk and dv, whose CTAs have all waited for what this one reads: it waits for its end only
    float scale, scale_log2;
};
template <int D, bool KEYS>
struct BackwardShape {
    static constexpr int kBuffers = KEYS && D == 128 ? 2 : 3, kGroups = 2, kThreads = 128 * kGroups + 128;
    static constexpr int kStages = D == 64 ? 8 : 4, kStay = D == 64 ? 2 : 1; // kStay: the next tile's come while this one's are read
    static constexpr uint32_t kTile = (D / 64) * 16384u, kSlice = (D / 64) * 8192u, kStage = 2 * kSlice; // 128 rows, 64 rows, both tensors' 64
    static constexpr uint32_t kSmem = kStay * 2 * kTile + kStages * kStage + 1024;
    static constexpr uint32_t kColumns = 512, kOut = kBuffers * 128; // of dK or dQ; dV's behind
};

// Sequences of packed queries whose first tokens' passes have more than one part, in order: their number, the sequences, and for each how many parts
// beyond a first one the sequences before it have (and, last, all have); and for the fold their queries, and their keys' first row and number.  Every
// query is in one sequence, so that the parts of all together are bound by the rows (`more` beyond the first ones); a sequence beyond that bound, as
// overlapping ranges could have it, keeps one part.
struct PartsList {
    const int *p;
    int room; // sequences; read through L1: thousands of warps of the fold ask for the same few lines
    __device__ __forceinline__ int count() const { return p[0]; }
    __device__ __forceinline__ int sequence(int m) const { return p[1 + m]; }
    __device__ __forceinline__ int before(int m) const { return p[1 + room + m]; }
    struct Entry {
        int m, seq, before, next; // m -1: there is none; next: `before` of the entry behind
    };
    // The first entry whose sequence is at least x, or (parts) the one that has the x-th of the parts beyond first ones.  The whole warp; what it reads
    // is asked for at once.
    __device__ __forceinline__ Entry find(int x, bool parts) const
    {
        const int n = count(), lane = threadIdx.x & 31;
        for (int i0 = 0; i0 < room; i0 += 32) {
            const int i = min(i0 + lane, room - 1), seq = sequence(i), first = before(i), next = before(i + 1);
            if (i0 >= n) break;
            const unsigned hit = __ballot_sync(0xffffffffu, i0 + lane < n && (parts ? next > x : seq >= x));
            if (hit) {
                const int who = __ffs(hit) - 1;
                return {i0 + who, __shfl_sync(0xffffffffu, seq, who), __shfl_sync(0xffffffffu, first, who), __shfl_sync(0xffffffffu, next, who)};
            }
        }
        return {-1, -1, 0, 0};
    }
    __device__ __forceinline__ int fact(int which, int m) const { return p[2 + (2 + which) * room + m]; } // queries, first key, keys
    static uint64_t bytes(int64_t room) { return (uint64_t)(5 * room + 2) * 4; }
};
// Its making, by one CTA of 256 threads.
__device__ __forceinline__ void list_parts(const DeltaArgs &a)
{
    __shared__ int64_t sums[8];
    __shared__ int ranks[8], count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int64_t sum_before = 0;
    int rank_before = 0;
    if (tid == 0) count = 0, a.list[1 + a.listed] = 0;
    for (int b0 = 0; b0 < a.sequences; b0 += 256) {
        const int b = b0 + tid;
        const int64_t blocks = b < a.sequences ? (int64_t)((range_of(a.q_ranges, b, (int)a.rows).count + 63) / 64) * a.group : 0;
        const int64_t mine = blocks ? (blocks - 1) / a.part_blocks : 0;
        int64_t sum = mine;
        int rank = mine > 0;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, sum, s);
            const int r = __shfl_up_sync(0xffffffffu, rank, s);
            if (lane >= s) sum += v, rank += r;
        }
        __syncthreads();
        if (lane == 31) sums[warp] = sum, ranks[warp] = rank;
        __syncthreads();
        for (int w = 0; w < 8; ++w) {
            if (w < warp) sum += sums[w], rank += ranks[w];
        }
        if (mine > 0 && sum_before + sum <= a.more) { // and so rank_before + rank, at least one each, is not more either
            const int m = rank_before + rank - 1;
            a.list[1 + m] = b;
            a.list[2 + a.listed + m] = (int)(sum_before + sum);
            const Range kr = range_of(a.k_ranges, b, a.k_rows);
            int *fact = a.list + 2 + 2 * a.listed + m;
            fact[0] = range_of(a.q_ranges, b, (int)a.rows).count, fact[a.listed] = kr.first, fact[2 * a.listed] = kr.count;
            atomicMax(&count, m + 1);
        }
        for (int w = 0; w < 8; ++w) sum_before += sums[w], rank_before += ranks[w];
    }
    __syncthreads();
    if (tid == 0) a.list[0] = count;
}

struct BackwardTile {
    int seq, head;         // KEYS: key head
    int row, rows, place0; // in the plane, number; KEYS: first key, else place of the first query
    int q_row, q_count, k_row, k_count;
    int first, count;      // KEYS: first query of the first block; blocks (times heads) of this part
    int part, begin;       // KEYS: part, and its first block
    int parts, slot;       // KEYS: parts that the tile may have; with a list, the sequence's first place among the parts of all
    int item, careful;
    Blocks blocks;         // of keys
    // Whether every row that stays sees, or is seen by, every row of the 64 that pass from o0 on.
    template <bool KEYS>
    __device__ __forceinline__ bool all_seen(int o0, int window, int sinks) const
    {
        if (!KEYS) return o0 + kBlock - 1 <= place0 && (o0 > place0 + rows - 1 - window || o0 + kBlock <= sinks);
        const int ahead = k_count - q_count, last_key = place0 + rows - 1;
        return o0 + ahead >= last_key && (min(o0 + kBlock, q_count) - 1 + ahead - window < place0 || last_key < sinks);
    }
};

// KEYS: the blocks of queries, times heads, that see the keys kb to kb + 127 (within the range), from query `first` on.
__device__ __forceinline__ int query_blocks(int kb, int q_count, int k_count, int window, int sinks, int group, int &first)
{
    const int ahead = k_count - q_count, last_key = min(kb + 127, k_count - 1);
    first = max(0, kb - ahead);
    const int end = kb < sinks ? q_count : (int)min((int64_t)q_count, (int64_t)last_key + window - ahead);
    return end > first ? (end - first + 63) / 64 * group : 0;
}

template <bool KEYS>
__device__ __forceinline__ bool find_tile(const BackwardArgs &a, int item, BackwardTile &t)
{
    const int heads = KEYS ? a.kv_heads : a.q_heads;
    int tile;
    t.part = 0, t.parts = KEYS ? a.parts : 1, t.slot = 0;
    const int listed = KEYS && a.list ? a.extra * heads : 0; // of all key heads together, first
    const PartsList list{a.list, a.listed};
    if (KEYS && item < listed) {
        t.head = item % heads;
        tile = item / heads % a.sink_tiles;
        const int x = item / heads / a.sink_tiles;
        const PartsList::Entry its = list.find(x, true);
        if (its.m < 0) return false;
        t.seq = its.seq, t.part = 1 + x - its.before, t.parts = 1 + its.next - its.before, t.slot = its.before + its.m;
    } else {
        item -= listed;
        const int each = a.tiles + (KEYS && !a.list ? a.extra : 0);
        const int group = item / (a.together * each), rest = item - group * a.together * each;
        const int wide = min(a.together, a.lanes - group * a.together), lane = group * a.together + rest % wide;
        tile = rest / wide;
        t.head = lane % heads;
        t.seq = lane / heads;
        if (KEYS && !a.list && tile < a.extra) {
            const int more = a.parts - 1;
            t.part = 1 + tile % more;
            tile /= more;
            if (a.packed_k) t.seq = tile / a.sink_tiles, tile %= a.sink_tiles;
        } else {
            tile = KEYS ? tile - (a.list ? 0 : a.extra) : a.tiles - 1 - tile;
            if (KEYS ? a.packed_k : a.packed_q) locate(KEYS ? a.k_ranges : a.q_ranges, a.sequences, KEYS ? a.k_rows : a.q_rows, 128, tile, t.seq, tile);
            if (t.seq < 0) return false;
            if (KEYS && a.list) {
                t.parts = 1;
                if (tile < a.sink_tiles) {
                    const PartsList::Entry its = list.find(t.seq, false);
                    if (its.seq == t.seq) t.parts += its.next - its.before, t.slot = its.before + its.m;
                }
            }
        }
    }
    const Range qr = range_of(a.q_ranges, t.seq, a.q_rows), kr = range_of(a.k_ranges, t.seq, a.k_rows);
    t.q_row = qr.first, t.q_count = qr.count, t.k_row = kr.first, t.k_count = kr.count;
    t.rows = min(128, (KEYS ? kr.count : qr.count) - tile * 128);
    if (t.rows <= 0) return false;
    t.row = (KEYS ? kr.first : qr.first) + tile * 128;
    t.begin = 0;
    if (KEYS) {
        t.place0 = tile * 128;
        const int all = query_blocks(tile * 128, qr.count, kr.count, a.window, a.sinks, a.group, t.first);
        t.begin = t.part * a.part_blocks;
        t.count = min(all - t.begin, t.parts > 1 ? a.part_blocks : all);
        if (t.part && t.count <= 0) return false;
        t.count = max(t.count, 0);
    } else {
        t.place0 = tile * 128 + kr.count - qr.count;
        t.blocks = Blocks(t.place0, t.place0 + t.rows - 1, a.window, a.sinks, kBlock);
        t.count = t.blocks.count;
    }
    return true;
}

// Where a key's row of partial sums of a part begins, of dk; dv's are behind.  slot: with a list, the sequence's.
template <int D>
__device__ __forceinline__ float *partial_row(const BackwardArgs &a, int seq, int slot, int head, int key, int part)
{
    const int64_t row = a.list ? ((int64_t)head * a.slots + slot + part) * a.sink_rows + key : ((int64_t)(seq * a.kv_heads + head) * a.sink_rows + key) * a.parts + part;
    return a.partials + row * 2 * D;
}

// As in the forward pass: dq from the keys, dv from the outputs' gradients (what is not finite of a query is in its lse, and so in P and dk already).
// `row`, at `place`, is the thread's, of the tile's; so are `columns` of it on, 32 in `step`.
template <typename T, int D, bool KEYS>
__device__ __noinline__ void mend_row(const BackwardArgs &a, const BackwardTile &tile, int place, int row, int columns, int step, bool partial, const Marred &marred)
{
    if (!partial && tile.part) return;
    const int ahead = tile.k_count - tile.q_count;
    float *sums = partial ? partial_row<D>(a, tile.seq, tile.slot, tile.head, place, tile.part) + D : nullptr;
    T *out = partial ? nullptr : at<T>(KEYS ? a.out1 : a.out0, tile.seq, tile.row + row, tile.head);
    const bool listed = marred.count <= kMarred;
    for (int i = 0; i < (listed ? marred.count : tile.count); ++i) {
        const int n = listed ? marred.block[i] : i, at_block = tile.begin + n, o0 = KEYS ? tile.first + at_block / a.group * 64 : tile.blocks[n] * kBlock;
        if (tile.template all_seen<KEYS>(o0, a.window, a.sinks)) continue;
        const int head = KEYS ? tile.head * a.group + at_block % a.group : tile.head / a.group, end = KEYS ? tile.q_count : tile.k_count;
        const T *passing = at<T>(a.passing, tile.seq, KEYS ? tile.q_row : tile.k_row, head);
        for (uint64_t rows = listed ? marred.rows[i] : ~0ull; rows; rows &= rows - 1) {
            const int o = o0 + __ffsll((long long)rows) - 1, q_place = KEYS ? o + ahead : place, key = KEYS ? place : o;
            if (!(o < end && key <= q_place && (key > q_place - a.window || key < a.sinks))) continue;
            bool none = true;
            for (int c = columns; c < a.d; c += step) {
                const T *from = passing + (int64_t)o * a.passing.row;
                none = (partial ? add_not_finite<KEYS>(sums, from, c, min(c + 32, a.d)) : add_not_finite<KEYS>(out, from, c, min(c + 32, a.d))) && none;
            }
            if (none) return;
        }
    }
}

template <typename T, int D, bool KEYS>
__global__ void __launch_bounds__(BackwardShape<D, KEYS>::kThreads, 1) k_backward(const __grid_constant__ BackwardArgs a)
{
    using Shape = BackwardShape<D, KEYS>;
    constexpr int kStages = Shape::kStages, kChunks = D / 64, kBuffers = Shape::kBuffers, kGroups = Shape::kGroups, kStay = Shape::kStay, kLoad = 4 * kGroups, kForm = kLoad + 1, kAdd = kLoad + 2;
    constexpr uint32_t kSlice = Shape::kSlice, kTile = Shape::kTile;
    extern __shared__ char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = base + kStay * 2 * kTile;
    __shared__ __align__(8) uint64_t bars[2 * kStages + 2 * kTiles + 4 + 2 * kStay + 3 * kBuffers];
    __shared__ BackwardTile tiles[kTiles];
    __shared__ __align__(16) float columns[KEYS ? kStages : 1][2][64]; // KEYS: -lse2 and -delta of the queries that pass
    __shared__ uint32_t tmem_at;
    __shared__ volatile int gave_up;
    __shared__ Marred marred;
    __shared__ Again again;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int s) { return bar0 + 8u * s; };
    const auto empty = [&](int s) { return bar0 + 8u * (kStages + s); };
    const uint32_t tile0 = bar0 + 16u * kStages, more0 = tile0 + 16u * kTiles;
    const auto tile_full = [&](int t) { return tile0 + 8u * (t % kTiles); };
    const auto tile_empty = [&](int t) { return tile0 + 8u * (kTiles + t % kTiles); };
    const uint32_t out_full = more0, out_empty = more0 + 8;
    const auto tail = [&](int i) { return more0 + 16 + 8u * i; };
    const auto stay_full = [&](int t) { return more0 + 32 + 8u * (t % kStay); };
    const auto stay_empty = [&](int t) { return more0 + 32 + 8u * (kStay + t % kStay); };
    const uint32_t more1 = more0 + 32 + 16u * kStay;
    const auto s_full = [&](int g) { return more1 + 8u * (g % kBuffers); };
    const auto p_full = [&](int g) { return more1 + 8u * (kBuffers + g % kBuffers); };
    const auto out_done = [&](int g) { return more1 + 8u * (2 * kBuffers + g % kBuffers); };

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < 2 * kStages; ++s) bar_init(bar0 + 8u * s, 1);
        for (int t = 0; t < kTiles; ++t) {
            bar_init(tile_full(t), 1);
            bar_init(tile_empty(t), 4 * kGroups + 2);
        }
        for (uint32_t b : {tail(0), tail(1)}) bar_init(b, 1);
        bar_init(out_full, 2); // the products, and what is to be known about them
        for (int i = 0; i < kStay; ++i) {
            bar_init(stay_full(i), 1);
            bar_init(stay_empty(i), 1);
        }
        bar_init(out_empty, 4 * kGroups);
        for (int i = 0; i < kBuffers; ++i) {
            bar_init(s_full(i), 1);
            bar_init(p_full(i), 4 * kGroups);
            bar_init(out_done(i), 1);
        }
        gave_up = 0;
        again.last = -1, again.count = 0;
        bar_init_fence();
    }
    if (warp == kForm) tmem_alloc(smem_u32(&tmem_at), Shape::kColumns);
    const int beyond = (int)threadIdx.x - 32 * kLoad;
    if (beyond >= 0 && beyond < 4 && a.q_rows > 0 && a.k_rows > 0) tma_prefetch_map(beyond == 0 ? &a.stay0 : beyond == 1 ? &a.stay1 : beyond == 2 ? &a.pass0 : &a.pass1);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_at;
    if (!a.beside) wait_prior_grid();
    release_next_grid(); // as in the forward pass

    // Blocks come by two warps, every second one each: what a warp does for a block takes as long as its products.  `g`: blocks before this tile.
    const auto bring_blocks = [&](const BackwardTile &t, int g, int which, uint32_t tail_bar, uint32_t &tails, bool chosen) {
        const int first = (g ^ which) & 1, begin = t.begin + first;
        int member = KEYS ? begin % a.group : 0, block = KEYS ? begin / a.group : 0; // KEYS: of the key head's query heads; of queries
        const int plane0 = a.pass0_planes > 1 ? t.seq : 0, plane1 = a.pass1_planes > 1 ? t.seq : 0, count = KEYS ? t.q_count : t.k_count;
        const int64_t lines = KEYS ? ((int64_t)(a.packed_q ? 0 : t.seq) * a.q_heads + t.head * a.group) * a.q_rows + t.q_row + lane : 0;
        for (int n = first; n < t.count; n += 2) {
            const int stage = (g + n) % kStages;
            const int head = KEYS ? t.head * a.group + member : t.head / a.group;
            const int at_row = KEYS ? t.first + block * 64 : t.blocks[n] * kBlock; // in the sequence
            const int row = (KEYS ? t.q_row : t.k_row) + at_row, valid = count - at_row;
            const uint32_t dst = ring + stage * Shape::kStage;
            const bool clear = (KEYS ? a.q_ranges : a.k_ranges) && valid < kBlock;
            float lse0 = -INFINITY, lse1 = -INFINITY, delta0 = 0.0f, delta1 = 0.0f; // on their way while the stage is waited for
            if (KEYS) {
                const int64_t line = lines + (int64_t)member * a.q_rows + at_row;
                if (lane < valid) lse0 = -__ldcg(a.lse2 + line), delta0 = -__ldcg(a.delta + line);
                if (lane + 32 < valid) lse1 = -__ldcg(a.lse2 + line + 32), delta1 = -__ldcg(a.delta + line + 32);
                for (member += 2; member >= a.group; member -= a.group) ++block;
            }
            if (!bar_wait_cta(empty(stage), ((g + n) / kStages & 1) ^ 1, &gave_up)) return false;
            if (KEYS) {
                columns[stage][0][lane] = lse0, columns[stage][0][32 + lane] = lse1;
                columns[stage][1][lane] = delta0, columns[stage][1][32 + lane] = delta1;
                __syncwarp();
            }
            const uint32_t bar = clear ? tail_bar : full(stage);
            if (chosen) {
                bar_expect(bar, Shape::kStage);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    tma_load4(dst + c * 8192u, &a.pass0, 64 * c, row, head, plane0, bar);
                    tma_load4(dst + kSlice + c * 8192u, &a.pass1, 64 * c, row, head, plane1, bar);
                }
            }
            __syncwarp();
            if (clear) {
                if (!bar_wait_cta(tail_bar, tails & 1u, &gave_up)) return false;
                ++tails;
                clear_rows(dst, 2 * kChunks, kBlock, valid);
                if (chosen) bar_arrive(full(stage));
                __syncwarp();
            }
        }
        return true;
    };
    if (warp == kLoad) {
        // ---------------------------------------------------------- tiles in
        const bool chosen = elect_one();
        int kt = -1, g = 0, done_again = 0;
        uint32_t tails = 0;
        bool ok = true, judged = false;
        const auto take = [&] {
            unsigned int n = lane == 0 ? atomicAdd(a.next, 1u) : 0;
            return (int)(gridDim.x + __shfl_sync(0xffffffffu, n, 0));
        };
        bool taken = true;
        for (int item = blockIdx.x; ok;) { // as in the forward pass
            if (!taken) item = take(); // not before the last tile's blocks are on their way
            taken = true;
            BackwardTile t;
            t.rows = t.count = 0;
            const bool others = item < a.items;
            if (!others && !judged) {
                for (int u = max(0, kt - kTiles + 1); ok && u <= kt; ++u) ok = bar_wait_cta(tile_empty(u), u / kTiles & 1, &gave_up);
                if (!ok) break;
                judged = true;
            }
            t.careful = again.due(done_again, others);
            const bool end = !others && !t.careful;
            t.item = t.careful ? again.items[done_again++ % kAgain] : item;
            if (!t.careful && others) taken = false;
            if (!end && !find_tile<KEYS>(a, t.item, t)) continue;
            if (!end && t.count == 0) { // rows that nothing sees, or that see nothing
                for (int r = 0; r < t.rows; ++r) {
                    for (int o = 0; o < (KEYS ? 2 : 1); ++o) {
                        const Heads &h = o ? a.out1 : a.out0;
                        if (!h.p) continue;
                        T *p = at<T>(h, t.seq, t.row + r, t.head);
                        for (int c = lane; c < a.d; c += 32) p[c] = from_f32<T>(0.0f);
                    }
                }
                continue;
            }
            ++kt;
            ok = bar_wait_cta(tile_empty(kt), (kt / kTiles & 1) ^ 1, &gave_up);
            if (!ok) break;
            if (lane == 0) tiles[kt % kTiles] = t;
            __syncwarp();
            if (chosen) bar_arrive(tile_full(kt));
            __syncwarp();
            if (end) break;
            ok = bar_wait_cta(stay_empty(kt), (kt / kStay & 1) ^ 1, &gave_up); // those that were there have been read
            if (!ok) break;
            if (chosen) {
                const int head = t.head, plane0 = a.stay0_planes > 1 ? t.seq : 0, plane1 = a.stay1_planes > 1 ? t.seq : 0;
                const uint32_t stay = base + (kt % kStay) * 2 * kTile;
                bar_expect(stay_full(kt), 2 * kTile);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    tma_load4(stay + c * 16384u, &a.stay0, 64 * c, t.row, head, plane0, stay_full(kt));
                    tma_load4(stay + kTile + c * 16384u, &a.stay1, 64 * c, t.row, head, plane1, stay_full(kt));
                }
            }
            __syncwarp();
            ok = bring_blocks(t, g, 0, tail(0), tails, chosen);
            g += t.count;
        }
        // every tile has been consumed: nothing is in flight towards this CTA any more
        for (int s = 0; ok && s < kStages; ++s) ok = bar_wait_cta(empty((g + s) % kStages), ((g + s) / kStages & 1) ^ 1, &gave_up);
    } else if (warp == kLoad + 3) {
        const bool chosen = elect_one();
        int g = 0;
        uint32_t tails = 0;
        for (int vt = 0;; ++vt) {
            if (!bar_wait_cta(tile_full(vt), vt / kTiles & 1, &gave_up)) break;
            const BackwardTile t = tiles[vt % kTiles];
            __syncwarp();
            if (chosen) bar_arrive(tile_empty(vt));
            __syncwarp();
            if (t.rows == 0 || !bring_blocks(t, g, 1, tail(1), tails, chosen)) break;
            g += t.count;
        }
    } else if (warp == kForm) {
        // ---------------------------------------------------------- S and dP, as far ahead as there are buffers
        const bool chosen = elect_one();
        const int steps = (a.d + 15) / 16;
        const uint32_t desc = instruction_desc(type_bits<T>(), false, false, 128, kBlock);
        const bool with0 = a.out0.p != nullptr;
        int g = 0;
        bool ok = true;
        for (int t = 0; ok; ++t) {
            ok = bar_wait_cta(tile_full(t), t / kTiles & 1, &gave_up);
            const int count = ok ? tiles[t % kTiles].count : 0;
            if (count == 0) break;
            ok = bar_wait_cta(stay_full(t), t / kStay & 1, &gave_up);
            const uint32_t stay = base + (t % kStay) * 2 * kTile;
            const uint64_t d0 = operand_desc(stay, 16), d1 = operand_desc(stay + kTile, 16);
            for (int n = 0; ok && n < count; ++n, ++g) {
                const int stage = g % kStages;
                ok = bar_wait_cta(full(stage), g / kStages & 1, &gave_up);
                if (g >= kBuffers) ok = ok && bar_wait_cta(out_done(g), (g / kBuffers + 1) & 1, &gave_up); // P and dS have been read where S and dP go
                if (!ok) break;
                fence_after();
                if (chosen) {
                    const uint32_t s = tmem + 128 * (g % kBuffers);
                    const uint64_t b0 = operand_desc(ring + stage * Shape::kStage, 16), b1 = operand_desc(ring + stage * Shape::kStage + kSlice, 16);
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) { // 64 elements a chunk
                        const uint32_t oa = ((j >> 2) * 16384u + (j & 3) * 32u) >> 4, ob = ((j >> 2) * 8192u + (j & 3) * 32u) >> 4;
                        if (j < steps) mma_ss(s, d0 + oa, b0 + ob, desc, j > 0);
                    }
                    if (with0) {
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) {
                            const uint32_t oa = ((j >> 2) * 16384u + (j & 3) * 32u) >> 4, ob = ((j >> 2) * 8192u + (j & 3) * 32u) >> 4;
                            if (j < steps) mma_ss(s + 64, d1 + oa, b1 + ob, desc, j > 0);
                        }
                    }
                    commit(s_full(g));
                    if (n + 1 == count) commit(stay_empty(t));
                }
                __syncwarp();
            }
        }
    } else if (warp == kAdd) {
        // ---------------------------------------------------------- the outputs
        const bool chosen = elect_one();
        const uint32_t desc = instruction_desc(type_bits<T>(), false, true, 128, 0) | (uint32_t)(2 * ((a.d + 15) / 16)) << 17;
        const bool with0 = a.out0.p != nullptr, with1 = KEYS && a.out1.p != nullptr;
        int g = 0;
        bool ok = true;
        for (int t = 0; ok; ++t) {
            ok = bar_wait_cta(tile_full(t), t / kTiles & 1, &gave_up);
            const int count = ok ? tiles[t % kTiles].count : 0;
            if (count == 0) break;
            ok = bar_wait_cta(out_empty, (t & 1) ^ 1, &gave_up); // the last tile's outputs have been read
            const BackwardTile &tile = tiles[t % kTiles];
            const bool careful = tile.careful;
            int bad = 0;
            for (int n = 0; ok && n < count; ++n, ++g) {
                const int stage = g % kStages;
                // as in the forward pass; S and dP are formed of what is there
                bool clear = false;
                constexpr int kPieces = (int)((KEYS ? Shape::kStage : kSlice) / 16);
                if (careful && !tile.template all_seen<KEYS>(KEYS ? tile.first + (tile.begin + n) / a.group * 64 : tile.blocks[n] * kBlock, a.window, a.sinks)) {
                    ok = bar_wait_cta(full(stage), g / kStages & 1, &gave_up);
                    if (!ok) break;
                    clear = some_not_finite<T>(ring + stage * Shape::kStage, kPieces); // while P is formed
                }
                ok = bar_wait_cta(p_full(g), g / kBuffers & 1, &gave_up);
                if (!ok) break;
                if (clear) {
                    uint64_t rows = clear_not_finite<T>(ring + stage * Shape::kStage, kChunks);
                    if (KEYS) rows = clear_not_finite<T>(ring + stage * Shape::kStage + kSlice, kChunks);
                    if (chosen) marred.put(bad, n, rows);
                    ++bad;
                }
                fence_after();
                if (chosen) {
                    const uint32_t s = tmem + 128 * (g % kBuffers), ds = KEYS ? s + 64 : s;
                    const uint64_t b0 = operand_desc(ring + stage * Shape::kStage, 8192), b1 = operand_desc(ring + stage * Shape::kStage + kSlice, 8192);
                    if (with1) {
#pragma unroll
                        for (int j = 0; j < kBlock / 16; ++j) mma_ts(tmem + Shape::kOut + D, s + 32 * (j >> 1) + 8 * (j & 1), b1 + j * (2048 >> 4), desc, n > 0 || j > 0);
                    }
                    if (with0) {
#pragma unroll
                        for (int j = 0; j < kBlock / 16; ++j) mma_ts(tmem + Shape::kOut, ds + 32 * (j >> 1) + 8 * (j & 1), b0 + j * (2048 >> 4), desc, n > 0 || j > 0);
                    }
                    commit(out_done(g));
                    commit(empty(stage)); // S and dP, which had read it, too, are done: P came of them
                    if (n + 1 == count) {
                        marred.count = bad;
                        bar_arrive(out_full);
                        commit(out_full);
                        bar_arrive(tile_empty(t));
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp < kLoad) {
        // ---------------------------------------------------------- P and dS, a thread a row
        const int group = warp >> 2, quarter = warp & 3;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        const float c = a.scale_log2;
        int buffer = 0, stage = 0;
        uint32_t phase = 0, stage_phase = 0;
        for (int vt = 0;; ++vt) {
            bar_pass_cta(tile_full(vt), vt / kTiles & 1, &gave_up);
            if (__any_sync(0xffffffffu, gave_up)) break;
            const BackwardTile tile = tiles[vt % kTiles];
            if (tile.rows == 0) break;
            const int row = quarter * 32 + lane, place = tile.place0 + row; // KEYS: the key
            const int w0 = tile.place0 + quarter * 32, w1 = w0 + 31;
            const bool live = row < tile.rows;
            const int ahead = tile.k_count - tile.q_count;
            float minus_lse = -INFINITY, minus_delta = 0.0f;
            if (!KEYS && live) {
                const int64_t line = ((int64_t)(a.packed_q ? 0 : tile.seq) * a.q_heads + tile.head) * a.q_rows + tile.row + row;
                minus_lse = -__ldcg(a.lse2 + line);
                minus_delta = -__ldcg(a.delta + line);
            }
            int member = KEYS ? tile.begin % a.group : 0, block = KEYS ? tile.begin / a.group : 0;
            for (int n = 0; n < tile.count; ++n) {
                const uint32_t ts = lanes + 128 * buffer + 32 * group;
                const int o0 = (KEYS ? tile.first + block * 64 : tile.blocks[n] * kBlock) + 32 * group, o1 = o0 + 31; // this group's queries (KEYS) or keys
                if (KEYS && ++member == a.group) member = 0, ++block;
                bool some, all;
                if (KEYS) { // queries at places o0 + ahead on
                    some = o1 + ahead >= w0 && o0 < tile.q_count && (o0 + ahead - a.window < w1 || w0 < a.sinks);
                    all = o0 + ahead >= w1 && o1 < tile.q_count && (o1 + ahead - a.window < w0 || w1 < a.sinks);
                } else {
                    some = o0 <= w1 && (o1 > w0 - a.window || o0 < a.sinks);
                    all = o1 <= w0 && (o0 > w1 - a.window || o1 < a.sinks);
                }
                uint32_t p[16], ds[16];
                if (KEYS) bar_pass_cta(full(stage), stage_phase, &gave_up);
                bar_pass_cta(s_full(buffer), phase, &gave_up);
                fence_after();
                if (some) {
                    float x[32], y[32];
                    tmem_ld32(ts, x);
                    tmem_ld32(ts + 64, y);
                    tmem_wait_ld();
                    const f32x2 c2 = pair(c);
                    const float4 *l4 = reinterpret_cast<const float4 *>(&columns[KEYS ? stage : 0][0][KEYS ? 32 * group : 0]);
                    const float4 *d4 = reinterpret_cast<const float4 *>(&columns[KEYS ? stage : 0][1][KEYS ? 32 * group : 0]);
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        float4 l = make_float4(minus_lse, minus_lse, minus_lse, minus_lse), dl = make_float4(minus_delta, minus_delta, minus_delta, minus_delta);
                        if (KEYS) l = l4[i / 4], dl = d4[i / 4];
                        unpair(fma2(pair(x[i], x[i + 1]), c2, pair(l.x, l.y)), x[i], x[i + 1]);
                        unpair(fma2(pair(x[i + 2], x[i + 3]), c2, pair(l.z, l.w)), x[i + 2], x[i + 3]);
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[i + k] = exp2_approx(x[i + k]);
                        unpair(mul2(pair(x[i], x[i + 1]), add2(pair(y[i], y[i + 1]), pair(dl.x, dl.y))), y[i], y[i + 1]);
                        unpair(mul2(pair(x[i + 2], x[i + 3]), add2(pair(y[i + 2], y[i + 3]), pair(dl.z, dl.w))), y[i + 2], y[i + 3]);
                    }
                    if (!all) {
                        uint32_t seen;
                        if (KEYS) seen = ~below(place - ahead - o0) & below(tile.q_count - o0) & (place < a.sinks ? ~0u : below(place + a.window - ahead - o0));
                        else seen = below(place + 1 - o0) & (~below(place - a.window + 1 - o0) | below(a.sinks - o0));
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            if (KEYS) x[i] = seen >> i & 1u ? x[i] : 0.0f;
                            y[i] = seen >> i & 1u ? y[i] : 0.0f;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (KEYS) p[i] = pack2(x[2 * i], x[2 * i + 1], T());
                        ds[i] = pack2(y[2 * i], y[2 * i + 1], T());
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) p[i] = ds[i] = 0;
                }
                // over scores that this thread has read
                if (KEYS) tmem_st16(ts, p);
                tmem_st16(KEYS ? ts + 64 : ts, ds);
                tmem_wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full(buffer));
                if (++buffer == kBuffers) buffer = 0, phase ^= 1u;
                if (++stage == kStages) stage = 0, stage_phase ^= 1u;
            }
            bar_pass_cta(out_full, vt & 1, &gave_up);
            fence_after();
            const bool mend = tile.careful && marred.count;
            float sound = 0.0f;
            // the outputs, 32 columns of each a group of warps in turn
            const uint32_t to = lanes + Shape::kOut;
            const bool partial = KEYS && tile.parts > 1 && live && place < a.sinks; // another part of this tile has some, too
#pragma unroll 1
            for (int i = group; i < (KEYS ? 2 : 1) * (D / 32); i += kGroups) {
                const int o = i / (D / 32), cc = i % (D / 32) * 32;
                const Heads &h = o ? a.out1 : a.out0;
                if (!h.p || cc >= a.d) continue;
                const float factor = o ? 1.0f : a.scale;
                float v[32];
                tmem_ld32(to + D * o + cc, v);
                tmem_wait_ld();
                sound += judge(v, a.d - cc);
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] *= factor;
                if (partial) {
                    float *q = partial_row<D>(a, tile.seq, tile.slot, tile.head, place, tile.part) + o * D + cc;
#pragma unroll
                    for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4 *>(q + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
                } else if (live && tile.part == 0) {
                    store_row(at<T>(h, tile.seq, tile.row + row, tile.head) + cc, v, a.d - cc, o ? a.wide1 : a.wide0);
                }
            }
            fence_before();
            __syncwarp();
            if (mend && live && (!KEYS || a.out1.p)) mend_row<T, D, KEYS>(a, tiles[vt % kTiles], place, row, 32 * group, 32 * kGroups, partial, marred);
            __syncwarp();
            if (lane == 0) bar_arrive(out_empty);
            if (__any_sync(0xffffffffu, live && sound != sound && minus_lse == minus_lse && !tile.careful) && lane == 0) again.put(vt, tile.item);
            __syncwarp();
            if (lane == 0) bar_arrive(tile_empty(vt));
        }
    }
    __syncwarp();
    __syncthreads();
    if (gave_up) {
        // leave the copies and products in flight a bounded time to end, and say so
        if (threadIdx.x == 0) atomicAdd(&g_waits_run_out, 1u);
        const uint64_t begin = now_ns();
        while (now_ns() - begin < 5000000ull) __nanosleep(1000);
    }
    if (warp == kForm) tmem_free(tmem, Shape::kColumns);
    if (a.beside) wait_prior_grid(); // who waits for this launch waits for dq, too
}

// The parts' sums of the first tokens' keys, in order.  A warp 32 columns of one output of a key and key head.
template <typename T, int D>
__global__ void __launch_bounds__(256) k_fold_keys(const __grid_constant__ BackwardArgs a)
{
    wait_prior_grid();
    release_next_grid();
    constexpr int kPieces = 2 * (D / 32);
    // 32 bits hold a key, a head and a sequence: each has a row of partial sums
    const uint32_t warp = blockIdx.x * 8 + (threadIdx.x >> 5), item = warp / kPieces;
    const int piece = (int)(warp % kPieces), o = piece / (D / 32), c = piece % (D / 32) * 32 + (threadIdx.x & 31);
    const int key = (int)(item % a.sink_rows), lane = (int)(item / a.sink_rows), head = lane % a.kv_heads;
    int seq = lane / a.kv_heads, slot = 0, q_count;
    if (seq >= (a.list ? a.listed : a.sequences)) return;
    Range kr;
    if (a.list) {
        const PartsList list{a.list, a.listed};
        const int m = seq, n = list.count();
        seq = list.sequence(m), slot = list.before(m) + m;
        q_count = list.fact(0, m), kr = {list.fact(1, m), list.fact(2, m)};
        if (m >= n) return;
    } else {
        q_count = range_of(a.q_ranges, seq, a.q_rows).count, kr = range_of(a.k_ranges, seq, a.k_rows);
    }
    if (key >= kr.count) return;
    int first;
    const int all = query_blocks(key / 128 * 128, q_count, kr.count, a.window, a.sinks, a.group, first);
    const int parts = (all + a.part_blocks - 1) / a.part_blocks;
    if (parts == 0) return; // cleared where the tile was found
    const Heads &h = o ? a.out1 : a.out0;
    if (!h.p || c >= a.d) return;
    const float *p = partial_row<D>(a, seq, slot, head, key, 0) + o * D + c;
    const int64_t step = (a.list ? a.sink_rows : 1) * 2 * D;
    float sum = 0.0f;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) sum += p[k * step];
    at<T>(h, seq, kr.first + key, head)[c] = from_f32<T>(sum);
}

// lse in units of log 2 and delta of every query: eight or sixteen lanes a query and head; a CTA takes 16 rows of a plane.
constexpr int kDeltaRows = 16;
template <typename T, int LANES>
__global__ void __launch_bounds__(256) k_delta(const __grid_constant__ DeltaArgs a)
{
    wait_prior_grid();
    release_next_grid();
    if (blockIdx.x == 0 && threadIdx.x < 2) a.next[threadIdx.x] = 0;
    if (a.list && blockIdx.x == gridDim.x - 1) { // a CTA for it alone
        list_parts(a);
        return;
    }
    constexpr int kEach = 256 / LANES, kAhead = 4; // queries at a time, whose reads come before their sums
    const int lane = threadIdx.x % LANES, plane = blockIdx.x / a.blocks;
    const int64_t row0 = (int64_t)(blockIdx.x % a.blocks) * kDeltaRows;
    const int count = (int)min((int64_t)kDeltaRows, a.rows - row0) * a.heads;
    for (int i0 = threadIdx.x / LANES; i0 - (int)threadIdx.x / LANES < count; i0 += kEach * kAhead) {
        Raw8<T> x[kAhead], y[kAhead];
        float sum[kAhead] = {};
        int64_t line[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int i = min(i0 + e * kEach, count - 1), r = i / a.heads, head = i - r * a.heads;
            const int64_t row = row0 + r;
            const T *o = static_cast<const T *>(a.o.p) + plane * a.o.seq + row * a.o.row + (int64_t)head * a.o.head;
            const T *g = static_cast<const T *>(a.dout.p) + plane * a.dout.seq + row * a.dout.row + (int64_t)head * a.dout.head;
            line[e] = ((int64_t)plane * a.heads + head) * a.rows + row;
            if (a.wide) {
                if (lane * 8 < a.d) x[e].load(o + lane * 8), y[e].load(g + lane * 8);
                else x[e].zero(), y[e].zero();
            } else {
                for (int c = lane; c < a.d; c += LANES) sum[e] = fmaf(to_f32(o[c]), to_f32(g[c]), sum[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (a.wide) {
                float u[8], v[8];
                x[e].unpack(u);
                y[e].unpack(v);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[e] = fmaf(u[k], v[k], sum[e]);
            }
#pragma unroll
            for (int s = LANES / 2; s; s >>= 1) sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], s);
            if (lane == 0 && i0 + e * kEach < count) {
                const float l = a.lse[line[e]];
                a.lse2[line[e]] = l == -INFINITY ? INFINITY : l * 1.4426950408889634f;
                a.delta[line[e]] = sum[e];
            }
        }
    }
}

// ------------------------------------------------------------------ tensors that TMA cannot read
struct PackJob {
    Heads src;
    uint16_t *dst;
    int64_t rows; // of all planes
    int plane_rows, heads;
};
struct PackArgs {
    PackJob job[4];
    int d, padded;
};
__global__ void __launch_bounds__(256) k_pack_heads(const __grid_constant__ PackArgs a)
{
    wait_prior_grid();
    release_next_grid();
    const PackJob &j = a.job[blockIdx.y];
    const int pieces = a.padded / 8; // 16 bytes of a padded head each
    const int64_t all = j.rows * j.heads * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t head_row = i / pieces, row = head_row / j.heads, plane = row / j.plane_rows;
        const int c = (int)(i - head_row * pieces) * 8, head = (int)(head_row - row * j.heads);
        const uint16_t *s = static_cast<const uint16_t *>(j.src.p) + plane * j.src.seq + (row - plane * j.plane_rows) * j.src.row + (int64_t)head * j.src.head + c;
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < a.d) w[k / 2] |= (uint32_t)s[k] << (16 * (k & 1));
        *reinterpret_cast<uint4 *>(j.dst + i * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ------------------------------------------------------------------ host
int check_shape(const a2sgd_attention *s)
{
    if (!s || (s->dtype != A2SGD_BF16 && s->dtype != A2SGD_F16)) return A2SGD_ERR_ARG;
    if (s->kv_heads == 0 || s->q_heads == 0 || s->q_heads % s->kv_heads || s->head_dim == 0) return A2SGD_ERR_ARG;
    // as the kernels have it: 0 times a hidden score's -infinity, or infinity times a score of 0, is not a number
    const float scale = (float)s->scale, scale_log2 = (float)(s->scale * 1.4426950408889634);
    if (s->window == 0 || !(scale > 0.0f) || !(scale_log2 > 0.0f) || !std::isfinite(scale_log2)) return A2SGD_ERR_ARG;
    if (s->head_dim > A2SGD_ATTENTION_MAX_HEAD_DIM || s->q_heads > 65535u || s->sequences > 65535u || s->q_rows >= (1ull << 30) ||
        s->k_rows >= (1ull << 30))
        return A2SGD_ERR_TOO_LARGE;
    return A2SGD_OK;
}

// A tensor of `heads` heads and `rows` rows a sequence.  like: it is written, as the tensor `like` is read: no two elements may share a place, and it
// is packed where that is.
int check_heads(const a2sgd_attention *s, const a2sgd_heads *h, uint32_t heads, uint64_t rows, const int32_t *ranges, bool needed,
                const a2sgd_heads *like)
{
    if (!h || !h->p) return needed && rows ? A2SGD_ERR_ARG : A2SGD_OK;
    if (h->sequence_stride < 0 || h->row_stride < 0 || h->head_stride < 0) return A2SGD_ERR_ARG;
    if (like) {
        const bool packed = ranges && (!like->p || like->sequence_stride == 0);
        if ((s->sequences > 1 && (h->sequence_stride == 0) != packed) || (h->row_stride == 0 && rows > 1) || (h->head_stride == 0 && heads > 1))
            return A2SGD_ERR_ARG;
    }
    return aligned(h->p, 2) ? A2SGD_OK : A2SGD_ERR_ALIGN;
}

Heads heads_of(const a2sgd_heads *h)
{
    return h && h->p ? Heads{h->p, h->sequence_stride, h->row_stride, h->head_stride} : Heads{nullptr, 0, 0, 0};
}

// A tensor of heads with its extents; planes: 1 where all sequences lie in one, or read the same.
struct Tensor {
    Heads h;
    int64_t rows;
    int heads, d, planes;
};
inline int padded(int d) { return (d + 7) / 8 * 8; }
inline uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }
inline uint64_t room(int64_t planes, int64_t rows, int heads, int d) { return up256((uint64_t)planes * rows * heads * padded(d) * 2); }

Tensor tensor_of(const a2sgd_attention *s, const a2sgd_heads *h, bool keys)
{
    Tensor t;
    t.h = heads_of(h);
    t.rows = (int64_t)(keys ? s->k_rows : s->q_rows);
    t.heads = (int)(keys ? s->kv_heads : s->q_heads);
    t.d = (int)s->head_dim;
    t.planes = t.h.seq == 0 ? 1 : (int)s->sequences;
    return t;
}
bool tma_ok(const Tensor &t)
{
    const auto step = [](int64_t extent, int64_t stride) { return extent <= 1 || (stride > 0 && stride % 8 == 0); };
    return aligned(t.h.p, 16) && step(t.rows, t.h.row) && step(t.heads, t.h.head) && step(t.planes, t.h.seq);
}
// Tiles of `box` rows and 64 elements of one head, 128 bytes a row, swizzled.
bool make_map(CUtensorMap *map, const Tensor &t, int dtype, int box)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const auto step = [](int64_t extent, int64_t stride) { return (cuuint64_t)(extent > 1 ? stride : 8) * 2; }; // one: any stride is right
    const cuuint64_t dims[4] = {(cuuint64_t)t.d, (cuuint64_t)t.rows, (cuuint64_t)t.heads, (cuuint64_t)t.planes};
    const cuuint64_t strides[3] = {step(t.rows, t.h.row), step(t.heads, t.h.head), step(t.planes, t.h.seq)};
    const cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1}, steps[4] = {1, 1, 1, 1};
    return encode(map, dtype == A2SGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, t.h.p, dims, strides,
                  boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// 16-byte accesses to whole rows of heads
bool wide(const Tensor &t) { return t.d % 8 == 0 && tma_ok(t); }
// The widest stores to them, in bytes.
int store_bytes(const Tensor &t)
{
    const auto step = [](int64_t extent, int64_t stride) { return extent <= 1 || stride % 16 == 0; };
    if (!t.h.p || !wide(t)) return 2;
    return t.d % 16 == 0 && aligned(t.h.p, 32) && step(t.rows, t.h.row) && step(t.heads, t.h.head) && step(t.planes, t.h.seq) ? 32 : 16;
}

struct Packer {
    PackArgs args{};
    int jobs = 0;
    int64_t most = 0;
    char *begin, *at;
    explicit Packer(void *workspace) : begin(static_cast<char *>(workspace)), at(begin) {}
    void *take(uint64_t bytes)
    {
        void *p = at;
        at += up256(bytes);
        return p;
    }
    // The tensor itself, or where its padded copy will be.
    Tensor usable(const Tensor &t)
    {
        if (t.rows == 0 || tma_ok(t)) return t;
        Tensor c = t;
        const int p = padded(t.d);
        c.h.head = p;
        c.h.row = (int64_t)t.heads * p;
        c.h.seq = t.planes > 1 ? t.rows * c.h.row : 0;
        c.h.p = take(room(t.planes, t.rows, t.heads, t.d));
        args.job[jobs++] = PackJob{t.h, static_cast<uint16_t *>(c.h.p), t.planes * t.rows, (int)t.rows, t.heads};
        args.d = t.d, args.padded = p;
        most = std::max(most, t.planes * t.rows * t.heads * (p / 8));
        return c;
    }
    bool fits(uint64_t bytes) const { return at == begin || (begin && (uint64_t)(at - begin) <= bytes); }
    int run(int sms, cudaStream_t s)
    {
        if (!jobs) return A2SGD_OK;
        void *params[] = {&args};
        A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_pack_heads),
                             dim3((unsigned)std::min<int64_t>((most + 255) / 256, (int64_t)sms * 16), (unsigned)jobs), 256, 0, params, s));
        return A2SGD_OK;
    }
};

// Queries that are few enough: the rows of a key head's queries, in sequences that are not packed (whose lengths the host does not know).  64 sequences,
// 32 heads of 128, 8 key heads, 4112 keys: 32 rows 304 us here and 48 rows 452, where tiles of 128 queries take 533; 64 rows 539 and 488.
constexpr int kFewMost = 48;
inline bool few(const a2sgd_attention *s, bool packed_q) { return !packed_q && s->q_rows * (s->q_heads / s->kv_heads) <= kFewMost; }
inline uint64_t share_bytes(const a2sgd_attention *s) { return (uint64_t)kMostShares * kFewRows * ((s->head_dim <= 64 ? 64 : 128) + 2) * 4; }

template <typename T, int D>
int launch_few(FewArgs &f, int sequences, float *partials, int sms, cudaStream_t s)
{
    using Shape = FewShape<D>;
    f.tiles = (f.q_rows * f.group + kFewRows - 1) / kFewRows;
    if (f.kv_heads > 65535 || sequences > 65535) return A2SGD_ERR_TOO_LARGE;
    const int64_t items = (int64_t)f.tiles * f.kv_heads * sequences;
    // a row's keys are shared out until there are two CTAs an SM, as long as a warp keeps four runs of 16 keys (4 sequences, 25 heads of 64, 1028 keys:
    // two CTAs a row 11.8 us, one 14.5)
    const int64_t seen = std::min<int64_t>(f.k_rows, (int64_t)std::min(f.window, 1 << 29) + f.sinks), units = (seen + kFewKeys - 1) / kFewKeys;
    int64_t shares = 1;
    if (items < 2 * sms) shares = std::max<int64_t>(1, std::min<int64_t>(std::min(2 * sms, kMostShares) / items, units / (Shape::kWarps * 4)));
    // Beyond a cluster there is a second launch: only where the warps of a cluster's CTAs would have more than twelve runs each.  One sequence, 32
    // heads of 128, 8 key heads: 4096 keys (8 runs) 14.3 us with 16 CTAs a row and 13.0 with eight, 8192 keys 14.4 (32 CTAs) and 18.8,
    // 131072 keys 76.7 (37) and 198; 4 heads of 64: 8192 keys (8 runs) 13.5 and 11.4, 32768 14.2 and 22.7.
    if (!partials || units <= 12 * kFewCluster * Shape::kWarps) shares = std::min<int64_t>(shares, kFewCluster);
    f.shares = (int)shares;
    f.cluster = shares > 1 && shares <= kFewCluster;
    f.partials = partials;
    void *params[] = {&f};
    const void *fn = reinterpret_cast<const void *>(&k_few<T, D>);
    A2_TRAIN_CUDA(allow_smem(fn, Shape::kSmem));
    const dim3 rows((unsigned)f.tiles, (unsigned)f.kv_heads, (unsigned)sequences);
    A2_TRAIN_CUDA(launch(fn, dim3(rows.x * (unsigned)f.shares, rows.y, rows.z), 32 * Shape::kWarps, Shape::kSmem, params, s, f.cluster ? (unsigned)f.shares : 1));
    if (f.shares > 1 && !f.cluster) A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_few_join<T, D>), dim3(rows.x * kFewRows, rows.y, rows.z), kJoinThreads, 0, params, s));
    return A2SGD_OK;
}

template <typename T, int D>
int launch_forward(ForwardArgs &f, int64_t rows, int sms, cudaStream_t s)
{
    using Shape = ForwardShape<D>;
    f.tiles = (int)(f.packed_q ? rows / 128 + f.sequences : (rows + 127) / 128);
    const int64_t lanes = (int64_t)f.q_heads * (f.packed_q ? 1 : f.sequences), items = lanes * f.tiles;
    if (items > 0x3fffffff) return A2SGD_ERR_TOO_LARGE;
    f.lanes = (int)lanes;
    // Heads that are worked on side by side: as many as their keys and values fit into L2 with (48 MB of 126), those that some tile of a wave
    // sees.  8 x 4096, 25 heads of 128, no window: 862 us, all 200 at once 971.
    const int64_t live = std::min<int64_t>(f.k_rows, (int64_t)f.window + 2048);
    f.together = (int)std::min<int64_t>(lanes, std::max<int64_t>(8, (48ll << 20) * f.group / std::max<int64_t>(1, live * D * 4)));
    f.items = (int)items;
    const void *fn = reinterpret_cast<const void *>(&k_forward<T, D>);
    A2_TRAIN_CUDA(allow_smem(fn, Shape::kSmem));
    void *params[] = {&f};
    A2_TRAIN_CUDA(launch(fn, dim3((unsigned)std::min<int64_t>(items, (int64_t)sms * Shape::kCtas)), Shape::kThreads, Shape::kSmem, params, s));
    return A2SGD_OK;
}

template <typename T>
int forward(const a2sgd_attention *shape, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &o, float *lse, void *workspace,
            uint64_t workspace_bytes, int sms, cudaStream_t s)
{
    Packer pack(workspace);
    const Tensor pq = pack.usable(q), pk = pack.usable(k), pv = pack.usable(v);
    if (!pack.fits(workspace_bytes)) return A2SGD_ERR_ARG;
    const int rc = pack.run(sms, s);
    if (rc != A2SGD_OK) return rc;
    if (few(shape, shape->q_ranges && q.h.seq == 0)) {
        FewArgs f{};
        f.q = pq.h, f.k = pk.h, f.v = pv.h, f.o = o.h;
        f.lse = lse;
        f.q_ranges = shape->q_ranges, f.k_ranges = shape->k_ranges;
        f.q_heads = q.heads, f.kv_heads = k.heads, f.group = q.heads / k.heads, f.d = q.d;
        f.q_rows = (int)q.rows, f.k_rows = (int)k.rows;
        f.window = (int)std::min<uint64_t>(shape->window, 1u << 30);
        f.sinks = (int)std::min<uint64_t>(shape->sinks, 1u << 30);
        f.scale_log2 = (float)(shape->scale * 1.4426950408889634);
        const bool room_for_shares = pack.begin && (uint64_t)(pack.at - pack.begin) + share_bytes(shape) <= workspace_bytes;
        float *partials = room_for_shares ? reinterpret_cast<float *>(pack.at) : nullptr;
        return q.d <= 64 ? launch_few<T, 64>(f, (int)shape->sequences, partials, sms, s) : launch_few<T, 128>(f, (int)shape->sequences, partials, sms, s);
    }
    ForwardArgs f{};
    if (!make_map(&f.q, pq, shape->dtype, 128)) return A2SGD_ERR_CUDA;
    if (k.rows && (!make_map(&f.k, pk, shape->dtype, kBlock) || !make_map(&f.v, pv, shape->dtype, kBlock))) return A2SGD_ERR_CUDA;
    f.o = o.h, f.values = pv.h;
    f.lse = lse;
    f.q_ranges = shape->q_ranges, f.k_ranges = shape->k_ranges;
    f.q_heads = q.heads, f.group = q.heads / k.heads, f.d = q.d;
    f.q_rows = (int)q.rows, f.k_rows = (int)k.rows;
    f.window = (int)std::min<uint64_t>(shape->window, 1u << 30);
    f.sinks = (int)std::min<uint64_t>(shape->sinks, 1u << 30);
    f.packed_q = shape->q_ranges && q.h.seq == 0;
    f.q_planes = pq.planes, f.k_planes = pk.planes, f.v_planes = pv.planes;
    f.sequences = (int)shape->sequences;
    f.wide_o = store_bytes(o);
    f.scale_log2 = (float)(shape->scale * 1.4426950408889634);
    return q.d <= 64 ? launch_forward<T, 64>(f, q.rows, sms, s) : launch_forward<T, 128>(f, q.rows, sms, s);
}

// How the first tokens' tiles are cut: the blocks of an ordinary tile's pass each, or 32 at least.
struct Parts {
    int parts = 1, blocks = 0, sink_tiles = 0, sink_rows = 0;
    int more = 0, listed = 0; // packed queries: parts of all sequences beyond a first one each; sequences that have some
};
Parts parts_of(const a2sgd_attention *s, bool packed_q)
{
    Parts p;
    const int64_t group = s->q_heads / s->kv_heads, q_rows = (int64_t)s->q_rows, k_rows = (int64_t)s->k_rows;
    const int64_t sinks = std::min<int64_t>(s->sinks, k_rows), window = (int64_t)std::min<uint64_t>(s->window, 1u << 30);
    if (sinks == 0 || window >= q_rows) return p;
    const int64_t ordinary = ((127 + window + 63) / 64 + 1) * group, each = std::max<int64_t>(ordinary, 32), all = (q_rows + 63) / 64 * group;
    if (all <= each) return p;
    p.parts = (int)((all + each - 1) / each);
    p.blocks = (int)each;
    p.sink_tiles = (int)((sinks + 127) / 128);
    p.sink_rows = (int)sinks;
    if (packed_q) {
        // A sequence with a second part has more than `each` >= 3 group blocks times heads, so four blocks of 64 or more and 193 rows at least: there are
        // at most q_rows / 193 of them, with q_rows / 64 blocks and one for each that is not full.
        p.more = (int)(((q_rows + 63) / 64 + std::min<int64_t>(s->sequences, q_rows / 193)) * group / each);
        p.listed = (int)std::min<int64_t>(s->sequences, p.more);
    }
    return p;
}
constexpr uint64_t kCounters = 256; // bytes: of items taken, by dk and dv, and by dq
uint64_t partial_bytes(const a2sgd_attention *s, bool packed_q)
{
    const Parts p = parts_of(s, packed_q);
    if (p.parts == 1) return 0;
    const uint64_t rows = (packed_q ? (uint64_t)(p.more + p.listed) : (uint64_t)s->sequences * p.parts) * s->kv_heads * p.sink_rows;
    return up256(rows * 2 * (s->head_dim <= 64 ? 64 : 128) * 4) + (packed_q ? up256(PartsList::bytes(p.listed)) : 0);
}

template <typename T, int D, bool KEYS>
int launch_backward(BackwardArgs &b, int64_t rows, int sms, cudaStream_t s)
{
    using Shape = BackwardShape<D, KEYS>;
    const bool packed = KEYS ? b.packed_k : b.packed_q;
    b.tiles = (int)(packed ? rows / 128 + b.sequences : (rows + 127) / 128);
    const int64_t lanes = (int64_t)(KEYS ? b.kv_heads : b.q_heads) * (packed ? 1 : b.sequences);
    // with a list, of a key head; else of a lane
    const int64_t extra = !KEYS ? 0 : b.list ? (int64_t)b.sink_tiles * (b.slots - b.listed) : (int64_t)b.sink_tiles * (b.parts - 1) * (packed ? b.sequences : 1);
    const int64_t items = lanes * b.tiles + (KEYS && b.list ? b.kv_heads : lanes) * extra;
    if (items > 0x3fffffff) return A2SGD_ERR_TOO_LARGE;
    b.lanes = (int)lanes;
    b.extra = (int)extra;
    b.items = (int)items;
    // as in the forward pass: what the tiles of a wave read at the same time stays in L2
    const int64_t live = std::min<int64_t>(KEYS ? b.q_rows : b.k_rows, (int64_t)b.window + 2048);
    b.together = (int)std::min<int64_t>(lanes, std::max<int64_t>(8, (48ll << 20) * (KEYS ? 1 : b.group) / std::max<int64_t>(1, live * D * 4 * (KEYS ? b.group : 1))));
    const void *fn = reinterpret_cast<const void *>(&k_backward<T, D, KEYS>);
    A2_TRAIN_CUDA(allow_smem(fn, Shape::kSmem));
    void *params[] = {&b};
    A2_TRAIN_CUDA(launch(fn, dim3((unsigned)std::min<int64_t>(items, sms)), Shape::kThreads, Shape::kSmem, params, s));
    return A2SGD_OK;
}

template <typename T, int D>
int run_backward(BackwardArgs &b, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &dout, const Tensor &dq, const Tensor &dk,
                 const Tensor &dv, int dtype, int sms, cudaStream_t s)
{
    int rc = A2SGD_OK;
    const bool keys = (dk.h.p || dv.h.p) && k.rows;
    if (keys) {
        const auto maps = [&] {
            return make_map(&b.stay0, k, dtype, 128) && make_map(&b.stay1, v, dtype, 128) &&
                   (q.rows == 0 || (make_map(&b.pass0, q, dtype, kBlock) && make_map(&b.pass1, dout, dtype, kBlock)));
        };
        if (!maps()) return A2SGD_ERR_CUDA;
        b.stay0_planes = k.planes, b.stay1_planes = v.planes, b.pass0_planes = q.planes, b.pass1_planes = dout.planes;
        b.out0 = dk.h, b.out1 = dv.h;
        b.passing = dout.h;
        b.wide0 = store_bytes(dk), b.wide1 = store_bytes(dv);
        rc = launch_backward<T, D, true>(b, k.rows, sms, s);
        if (rc != A2SGD_OK) return rc;
    }
    if (dq.h.p && q.rows) {
        BackwardArgs c = b;
        const auto maps = [&] {
            return make_map(&c.stay0, q, dtype, 128) && make_map(&c.stay1, dout, dtype, 128) &&
                   (k.rows == 0 || (make_map(&c.pass0, k, dtype, kBlock) && make_map(&c.pass1, v, dtype, kBlock)));
        };
        if (!maps()) return A2SGD_ERR_CUDA;
        c.stay0_planes = q.planes, c.stay1_planes = dout.planes, c.pass0_planes = k.planes, c.pass1_planes = v.planes;
        c.out0 = dq.h, c.out1 = Heads{nullptr, 0, 0, 0};
        c.passing = k.h;
        c.wide0 = store_bytes(dq);
        c.next = b.next + 1;
        c.beside = keys;
        rc = launch_backward<T, D, false>(c, q.rows, sms, s);
        if (rc != A2SGD_OK) return rc;
    }
    if (keys && b.parts > 1) {
        const int64_t rows = (int64_t)(b.list ? b.listed : b.sequences) * b.kv_heads * b.sink_rows; // far below a grid's limit: their partial sums fit the workspace
        void *params[] = {&b};
        A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_fold_keys<T, D>), dim3((unsigned)(rows * 2 * (D / 32) / 8 + 1)), 256, 0, params, s));
    }
    return rc;
}

template <typename T>
int backward(const a2sgd_attention *shape, const Tensor &dout, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &o, const float *lse,
             const Tensor &dq, const Tensor &dk, const Tensor &dv, void *workspace, uint64_t workspace_bytes, int sms, cudaStream_t s)
{
    Packer pack(workspace);
    const bool packed_q = shape->q_ranges && q.h.seq == 0, packed_k = shape->k_ranges && k.h.seq == 0;
    const uint64_t lines = (uint64_t)(packed_q ? 1 : shape->sequences) * shape->q_heads * shape->q_rows;
    BackwardArgs b{};
    float *lse2 = static_cast<float *>(pack.take(lines * 4)), *delta = static_cast<float *>(pack.take(lines * 4));
    b.lse2 = lse2, b.delta = delta;
    b.next = static_cast<unsigned int *>(pack.take(kCounters));
    const Parts parts = parts_of(shape, packed_q);
    const uint64_t for_parts = partial_bytes(shape, packed_q), for_list = parts.listed ? up256(PartsList::bytes(parts.listed)) : 0;
    int *list = for_list ? static_cast<int *>(pack.take(for_list)) : nullptr;
    b.partials = static_cast<float *>(pack.take(for_parts - for_list));
    const Tensor pq = pack.usable(q), pk = pack.usable(k), pv = pack.usable(v), pdout = pack.usable(dout);
    if (!pack.fits(workspace_bytes)) return A2SGD_ERR_ARG;
    int rc = pack.run(sms, s);
    if (rc != A2SGD_OK) return rc;
    if (lines) {
        DeltaArgs d{};
        d.o = o.h, d.dout = dout.h;
        d.lse = lse;
        d.lse2 = lse2, d.delta = delta, d.next = b.next;
        d.rows = q.rows;
        const int64_t planes = packed_q ? 1 : (int64_t)shape->sequences, blocks = (q.rows + kDeltaRows - 1) / kDeltaRows;
        if (planes * blocks >= 0x7fffffff) return A2SGD_ERR_TOO_LARGE;
        d.blocks = (int)blocks;
        d.heads = q.heads, d.d = q.d;
        d.wide = wide(o) && wide(dout);
        if (dk.h.p || dv.h.p) {
            d.list = list, d.q_ranges = shape->q_ranges, d.k_ranges = shape->k_ranges;
            d.sequences = (int)shape->sequences, d.k_rows = (int)k.rows, d.group = q.heads / k.heads;
            d.part_blocks = parts.blocks, d.more = parts.more, d.listed = parts.listed;
        }
        void *params[] = {&d};
        const void *fn = q.d <= 64 ? reinterpret_cast<const void *>(&k_delta<T, 8>) : reinterpret_cast<const void *>(&k_delta<T, 16>);
        A2_TRAIN_CUDA(launch(fn, dim3((unsigned)(planes * blocks) + (d.list != nullptr)), 256, 0, params, s));
    } else {
        A2_TRAIN_CUDA(cudaMemsetAsync(b.next, 0, kCounters, s));
    }
    b.q_ranges = shape->q_ranges, b.k_ranges = shape->k_ranges;
    b.q_heads = q.heads, b.kv_heads = k.heads, b.group = q.heads / k.heads, b.d = q.d;
    b.q_rows = (int)q.rows, b.k_rows = (int)k.rows;
    b.window = (int)std::min<uint64_t>(shape->window, 1u << 30);
    b.sinks = (int)std::min<uint64_t>(shape->sinks, 1u << 30);
    b.packed_q = packed_q, b.packed_k = packed_k;
    b.sequences = (int)shape->sequences;
    b.parts = parts.parts, b.part_blocks = parts.blocks, b.sink_tiles = parts.sink_tiles, b.sink_rows = parts.sink_rows;
    b.list = list, b.listed = parts.listed, b.slots = parts.more + parts.listed;
    b.scale = (float)shape->scale;
    b.scale_log2 = (float)(shape->scale * 1.4426950408889634);
    return q.d <= 64 ? run_backward<T, 64>(b, pq, pk, pv, pdout, dq, dk, dv, shape->dtype, sms, s)
                     : run_backward<T, 128>(b, pq, pk, pv, pdout, dq, dk, dv, shape->dtype, sms, s);
}

} // namespace

extern "C" uint64_t a2sgd_window_attention_workspace(const a2sgd_attention *shape, uint32_t flags)
{
    if (!shape || shape->head_dim > A2SGD_ATTENTION_MAX_HEAD_DIM) return 0;
    const int64_t q_planes = flags & A2SGD_ATTENTION_PACKED_Q ? 1 : shape->sequences, k_planes = flags & A2SGD_ATTENTION_PACKED_K ? 1 : shape->sequences;
    const int d = (int)shape->head_dim;
    uint64_t bytes = 0;
    if (shape->kv_heads == 0) return 0;
    if (flags & A2SGD_ATTENTION_BACKWARD) bytes += 2 * up256((uint64_t)q_planes * shape->q_heads * shape->q_rows * 4) + kCounters +
                                                  (flags & A2SGD_ATTENTION_PACKED_Q ? partial_bytes(shape, true) : std::max(partial_bytes(shape, false), partial_bytes(shape, true)));
    else if (few(shape, flags & A2SGD_ATTENTION_PACKED_Q)) bytes += share_bytes(shape);
    if (!(flags & A2SGD_ATTENTION_ALIGNED))
        bytes += (flags & A2SGD_ATTENTION_BACKWARD ? 2 : 1) * room(q_planes, (int64_t)shape->q_rows, (int)shape->q_heads, d) +
                 2 * room(k_planes, (int64_t)shape->k_rows, (int)shape->kv_heads, d);
    return bytes;
}

extern "C" int a2sgd_window_attention_forward(const a2sgd_attention *shape, const a2sgd_heads *q, const a2sgd_heads *k,
                                              const a2sgd_heads *v, const a2sgd_heads *o, float *lse, void *workspace,
                                              uint64_t workspace_bytes, int device, void *stream)
{
    int rc = check_shape(shape);
    if (rc != A2SGD_OK || shape->sequences == 0 || shape->q_rows == 0) return rc;
    if ((rc = check_heads(shape, q, shape->q_heads, shape->q_rows, shape->q_ranges, true, nullptr)) != A2SGD_OK ||
        (rc = check_heads(shape, k, shape->kv_heads, shape->k_rows, shape->k_ranges, true, nullptr)) != A2SGD_OK ||
        (rc = check_heads(shape, v, shape->kv_heads, shape->k_rows, shape->k_ranges, true, nullptr)) != A2SGD_OK ||
        (rc = check_heads(shape, o, shape->q_heads, shape->q_rows, shape->q_ranges, true, q)) != A2SGD_OK)
        return rc;
    if (!aligned(workspace, 256) || !aligned(lse, 4)) return A2SGD_ERR_ALIGN;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms < 1) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Tensor tq = tensor_of(shape, q, false), tk = tensor_of(shape, k, true), tv = tensor_of(shape, v, true), to = tensor_of(shape, o, false);
    return shape->dtype == A2SGD_BF16 ? forward<__nv_bfloat16>(shape, tq, tk, tv, to, lse, workspace, workspace_bytes, sms, s)
                                      : forward<__half>(shape, tq, tk, tv, to, lse, workspace, workspace_bytes, sms, s);
}

extern "C" int a2sgd_window_attention_backward(const a2sgd_attention *shape, const a2sgd_heads *dout, const a2sgd_heads *q,
                                               const a2sgd_heads *k, const a2sgd_heads *v, const a2sgd_heads *o, const float *lse,
                                               const a2sgd_heads *dq, const a2sgd_heads *dk, const a2sgd_heads *dv, void *workspace,
                                               uint64_t workspace_bytes, int device, void *stream)
{
    int rc = check_shape(shape);
    if (rc != A2SGD_OK || shape->sequences == 0) return rc;
    for (const a2sgd_heads *h : {q, dout, o}) {
        if ((rc = check_heads(shape, h, shape->q_heads, shape->q_rows, shape->q_ranges, true, nullptr)) != A2SGD_OK) return rc;
        // what belongs to packed queries lies as they do
        if (shape->sequences > 1 && shape->q_ranges && shape->q_rows && q->sequence_stride == 0 && h->sequence_stride != 0) return A2SGD_ERR_ARG;
    }
    for (const a2sgd_heads *h : {k, v})
        if ((rc = check_heads(shape, h, shape->kv_heads, shape->k_rows, shape->k_ranges, true, nullptr)) != A2SGD_OK) return rc;
    for (const a2sgd_heads *h : {dk, dv})
        if ((rc = check_heads(shape, h, shape->kv_heads, shape->k_rows, shape->k_ranges, false, k)) != A2SGD_OK) return rc;
    if ((rc = check_heads(shape, dq, shape->q_heads, shape->q_rows, shape->q_ranges, false, q)) != A2SGD_OK) return rc;
    if (!lse && shape->q_rows) return A2SGD_ERR_ARG;
    if (!aligned(workspace, 256) || !aligned(lse, 4)) return A2SGD_ERR_ALIGN;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms < 1) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Tensor tdo = tensor_of(shape, dout, false), tq = tensor_of(shape, q, false), tk = tensor_of(shape, k, true), tv = tensor_of(shape, v, true),
                 to = tensor_of(shape, o, false), tdq = tensor_of(shape, dq, false), tdk = tensor_of(shape, dk, true), tdv = tensor_of(shape, dv, true);
    return shape->dtype == A2SGD_BF16 ? backward<__nv_bfloat16>(shape, tdo, tq, tk, tv, to, lse, tdq, tdk, tdv, workspace, workspace_bytes, sms, s)
                                      : backward<__half>(shape, tdo, tq, tk, tv, to, lse, tdq, tdk, tdv, workspace, workspace_bytes, sms, s);
}

extern "C" int a2sgd_window_attention_status(int device, int *device_status, void *stream)
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
