// Layer norm, forward and backward, with the gradients of its weight and bias.
//
//   forward   mean = sum_c x / d,  rstd = 1 / sqrt(sum_c (x - mean)^2 / d + eps),  y = (x - mean) rstd w + b
//   backward  xhat = (x - mean) rstd,  g = dy w,
//             dx = rstd (g - sum_c g / d - xhat sum_c (g xhat) / d),
//             dw = sum_rows dy xhat,  db = sum_rows dy
//
// Bound by HBM: x once and y once forward, x and dy once and dx once backward.  A group of TPR
// threads owns the columns of a row, each thread the same columns of every row it meets, so that the
// weight and the bias, and backward the two column sums, stay in its registers over all rows.  R rows
// are in flight together: their loads are issued before any is used, and the threads of a group meet
// at one barrier for the R rows' sums.  The squared deviations are summed in a second reduction over
// the registers, not from a sum of squares, which cancels when the mean is large against the spread.
// All sums are fp32, in runs of at most kRun terms a thread (the columns of a long row, the rows of a column), the runs one after
// another, and trees or short chains over the threads, groups and CTAs; every order is fixed.
//
// B200, 65536 x 1600 bfloat16: forward 79 us (5.3 TB/s), a warp a row; backward 134 us (4.7 TB/s), two rows in flight: the wait at a
// row pair's barrier, with two CTAs an SM to hide it and 53 % of the issue slots in use (one row at a time 277 us; four do not fit
// the registers).
//
// Rows too long for registers (over kMostCols) take k_ln_*_long, which walk the row again instead, an element an access: 4096 x
// 12288 bfloat16 forward 152 us, backward 295 us.
#include "a2sgd_train.cuh"

#include <algorithm>
#include <cmath>
#include <cstdint>

using namespace a2sgd_train;

namespace {

constexpr int kMaxThreads = 1024;                       // of the long forms and the fold
constexpr int kRowThreads = 512;                        // of the register forms: 128 registers each
constexpr uint32_t kMostCols = kRowThreads * 16;        // 8192: at most 16 columns a thread
constexpr uint32_t kFoldCols = 32;                   // columns of one CTA of the fold
// Terms of a running sum.  7812 equal terms in one chain were off by 1.2e-4 of their sum, in runs of 512 by 7e-7; a chain
// of n fp32 additions may be off by n 2^-24.
constexpr uint32_t kRun = 512;

struct LnArgs {
    const void *x, *dy, *w, *b;
    void *y; // forward: y; backward: dx
    float *mean, *rstd;
    int64_t x_stride, dy_stride, y_stride;
    uint64_t rows;
    uint32_t d;
    uint32_t tpr;    // threads of a row
    uint32_t groups; // rows at a time / R
    float inv_d, eps;
    float *partials; // backward: [grid][2][d]
    void *dw, *db;
    uint32_t parts;
    bool add; // to the partial sums of the rows before
};

__device__ __forceinline__ void keep_partial(const LnArgs &a, float *at, float v) { *at = a.add ? __ldcg(at) + v : v; }

// N sums (a power of two) over the threads of a group, the same in each of them.  A group of up to 32 threads
// (a power of two) is part of a warp; a larger one is a whole number of warps and takes one barrier of the CTA.
// Within a warp the values are folded across lanes, half of them going each way, until a lane holds one: N = 8
// takes 9 shuffles in place of 40.  Two buffers in turn: a warp that runs ahead writes the other one, and meets the
// barrier before it comes back to the first.
template <int N>
struct GroupSum {
    float *sh; // [2][warps of the CTA][N]
    uint32_t tpr, warps, in_group, group;
    int turn = 0;
    // v <- finish(sums).  With a whole warp or more, a lane holds sum number lane % N (or lane / (32 / N)) before they
    // are handed round, and `finish` is applied to that one only.
    template <typename F>
    __device__ __forceinline__ void operator()(float (&v)[N], F finish)
    {
        const uint32_t lane = threadIdx.x & 31;
        if (tpr < 32) {
            for (uint32_t o = tpr / 2; o; o >>= 1) {
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = finish(v[i]);
            return;
        }
        int o = 16;
#pragma unroll
        for (int n = N / 2; n; n >>= 1, o >>= 1) {
            const bool upper = lane & o;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float send = upper ? v[i] : v[n + i];
                v[i] = (upper ? v[n + i] : v[i]) + __shfl_xor_sync(0xffffffffu, send, o);
            }
        }
        float x = v[0];
#pragma unroll
        for (; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        // x: sum number lane / (32 / N)
        if (tpr == 32) {
            x = finish(x);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, x, i * (32 / N));
            return;
        }
        float *slot = sh + ((uint32_t)turn * (kRowThreads / 32) + group * warps) * N;
        turn ^= 1;
        if (lane % (32 / N) == 0) slot[(in_group >> 5) * N + lane / (32 / N)] = x;
        __syncthreads();
        x = lane < warps * N ? slot[lane] : 0.0f;
        for (uint32_t k = lane + 32; k < warps * N; k += 32) x += slot[k];
#pragma unroll
        for (int q = N; q < 32; q <<= 1) x += __shfl_xor_sync(0xffffffffu, x, q);
        x = finish(x);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, x, i);
    }
};

// The columns of a thread.  VEC: eight consecutive ones at a time, from (k tpr + t) 8 on; else every tpr-th one from t on.
template <int NC, bool VEC>
__device__ __forceinline__ uint32_t column(int i, uint32_t t, uint32_t tpr)
{
    return VEC ? ((i / 8) * tpr + t) * 8 + (i & 7) : i * tpr + t;
}

// A thread's columns of one row; `row` points at its first one, `left` is the number of columns from there on.
template <typename T, int NC, bool VEC>
struct RowPart {
    Raw8<T> raw[VEC ? NC / 8 : 1];
    T one[VEC ? 1 : NC];
    __device__ __forceinline__ void load(const T *row, int left, uint32_t tpr, bool live)
    {
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < NC / 8; ++k) {
                if (live && (int)(k * tpr * 8) < left) raw[k].load(row + k * tpr * 8);
                else raw[k].zero();
            }
        } else {
#pragma unroll
            for (int k = 0; k < NC; ++k) one[k] = live && (int)(k * tpr) < left ? row[k * tpr] : from_f32<T>(0.0f);
        }
    }
    __device__ __forceinline__ void unpack(f32x2 (&p)[NC / 2]) const
    {
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < NC / 8; ++k) {
                float e[8];
                raw[k].unpack(e);
#pragma unroll
                for (int i = 0; i < 4; ++i) p[k * 4 + i] = pair(e[2 * i], e[2 * i + 1]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < NC / 2; ++k) p[k] = pair(to_f32(one[2 * k]), to_f32(one[2 * k + 1]));
        }
    }
};

template <typename T, int NC, bool VEC>
__device__ __forceinline__ void store_part(T *row, int left, uint32_t tpr, const f32x2 (&p)[NC / 2])
{
    float f[NC];
#pragma unroll
    for (int i = 0; i < NC / 2; ++i) unpair(p[i], f[2 * i], f[2 * i + 1]);
    if constexpr (VEC) {
#pragma unroll
        for (int k = 0; k < NC / 8; ++k) {
            if ((int)(k * tpr * 8) < left) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = f[k * 8 + i];
                store8(row + k * tpr * 8, e);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            if ((int)(k * tpr) < left) row[k * tpr] = from_f32<T>(f[k]);
        }
    }
}

__device__ __forceinline__ float half_of(f32x2 p, int which)
{
    float lo, hi;
    unpair(p, lo, hi);
    return which ? hi : lo;
}

// Rows of a group from `row` on, at most r.
__device__ __forceinline__ int rows_left(uint64_t row, int r, uint64_t rows)
{
    return row + r <= rows ? r : row < rows ? (int)(rows - row) : 0;
}

// Columns of a vector of W, or the value that stands for a missing vector.
template <typename W, int NC, bool VEC>
__device__ __forceinline__ void load_vector(const void *v, float missing, uint32_t t, uint32_t tpr, uint32_t d, f32x2 (&out)[NC / 2])
{
    float f[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const uint32_t c = column<NC, VEC>(i, t, tpr);
        f[i] = c < d && v ? to_f32(static_cast<const W *>(v)[c]) : missing;
    }
#pragma unroll
    for (int i = 0; i < NC / 2; ++i) out[i] = pair(f[2 * i], f[2 * i + 1]);
}

template <typename T, typename W, int NC, int R, bool VEC>
__global__ void __launch_bounds__(kRowThreads) k_ln_forward(const __grid_constant__ LnArgs a)
{
    constexpr int kPairs = NC / 2;
    extern __shared__ float sh[];
    const uint32_t group = threadIdx.x / a.tpr, t = threadIdx.x - group * a.tpr;
    const int left = (int)a.d - (int)(VEC ? t * 8 : t); // columns from this thread's first one on
    GroupSum<R> sum{sh, a.tpr, a.tpr >> 5, t, group};
    wait_prior_grid();
    release_next_grid();
    f32x2 w[kPairs], b[kPairs];
    load_vector<W, NC, VEC>(a.w, 1.0f, t, a.tpr, a.d, w);
    load_vector<W, NC, VEC>(a.b, 0.0f, t, a.tpr, a.d, b);
    const uint64_t at_once = (uint64_t)a.groups * R, step = gridDim.x * at_once;
    uint64_t row = blockIdx.x * at_once + group * R;
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.x_stride + (VEC ? t * 8 : t);
    T *y = static_cast<T *>(a.y) + (int64_t)row * a.y_stride + (VEC ? t * 8 : t);
    RowPart<T, NC, VEC> next[R]; // the loads of the next rows are on their way while these are worked on
    int rows = rows_left(row, R, a.rows);
#pragma unroll
    for (int r = 0; r < R; ++r) next[r].load(x + r * a.x_stride, left, a.tpr, r < rows);
    for (uint64_t r0 = blockIdx.x * at_once; r0 < a.rows; r0 += step) {
        f32x2 v[R][kPairs];
#pragma unroll
        for (int r = 0; r < R; ++r) next[r].unpack(v[r]);
        x += step * a.x_stride;
        const int next_rows = rows_left(row + step, R, a.rows);
#pragma unroll
        for (int r = 0; r < R; ++r) next[r].load(x + r * a.x_stride, left, a.tpr, r < next_rows);
        float mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2 s = v[r][0];
#pragma unroll
            for (int i = 1; i < kPairs; ++i) s = add2(s, v[r][i]);
            mean[r] = sum2(s);
        }
        sum(mean, [&](float s) { return s * a.inv_d; });
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const f32x2 m = pair(-mean[r]);
            rstd[r] = 0.0f;
#pragma unroll
            for (int k = 0; k < (VEC ? NC / 8 : 1); ++k) { // pieces that are there as a whole, or not at all
                f32x2 s = pair(0.0f);
#pragma unroll
                for (int i = k * 4; i < (VEC ? k * 4 + 4 : kPairs); ++i) {
                    v[r][i] = add2(v[r][i], m);
                    f32x2 q = v[r][i];
                    if (!VEC) // each column for itself
                        q = mul2(q, pair((int)(2 * i * a.tpr) < left ? 1.0f : 0.0f, (int)((2 * i + 1) * a.tpr) < left ? 1.0f : 0.0f));
                    s = fma2(q, q, s);
                }
                rstd[r] += !VEC || (int)(k * a.tpr * 8) < left ? sum2(s) : 0.0f;
            }
        }
        sum(rstd, [&](float s) { return 1.0f / sqrtf(fmaf(s, a.inv_d, a.eps)); });
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const f32x2 p = pair(rstd[r]);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) v[r][i] = fma2(mul2(v[r][i], p), w[i], b[i]);
            if (r < rows) {
                store_part<T, NC, VEC>(y + r * a.y_stride, left, a.tpr, v[r]);
                if (t == 0) {
                    if (a.mean) a.mean[row + r] = mean[r];
                    if (a.rstd) a.rstd[row + r] = rstd[r];
                }
            }
        }
        row += step;
        y += step * a.y_stride;
        rows = next_rows;
    }
}

template <typename T, typename W, int NC, int R, bool VEC>
__global__ void __launch_bounds__(kRowThreads) k_ln_backward(const __grid_constant__ LnArgs a)
{
    constexpr int kPairs = NC / 2;
    extern __shared__ float sh[];
    const uint32_t group = threadIdx.x / a.tpr, t = threadIdx.x - group * a.tpr;
    const int left = (int)a.d - (int)(VEC ? t * 8 : t);
    GroupSum<2 * R> sum{sh, a.tpr, a.tpr >> 5, t, group};
    wait_prior_grid();
    release_next_grid();
    f32x2 w[kPairs], dw[kPairs], db[kPairs];
    load_vector<W, NC, VEC>(a.w, 1.0f, t, a.tpr, a.d, w);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) dw[i] = db[i] = pair(0.0f);
    const uint64_t at_once = (uint64_t)a.groups * R, step = gridDim.x * at_once;
    uint64_t row = blockIdx.x * at_once + group * R;
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.x_stride + (VEC ? t * 8 : t);
    const T *dy = static_cast<const T *>(a.dy) + (int64_t)row * a.dy_stride + (VEC ? t * 8 : t);
    T *dx = static_cast<T *>(a.y) + (int64_t)row * a.y_stride + (VEC ? t * 8 : t);
    RowPart<T, NC, VEC> px[R], pg[R], nx[R], ng[R];
    float mean[R], rstd[R], next_mean[R], next_rstd[R];
    int rows = rows_left(row, R, a.rows);
    const auto fetch = [&](uint64_t first, int count) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            nx[r].load(x + r * a.x_stride, left, a.tpr, r < count);
            ng[r].load(dy + r * a.dy_stride, left, a.tpr, r < count);
            next_mean[r] = r < count ? __ldcg(a.mean + first + r) : 0.0f;
            next_rstd[r] = r < count ? __ldcg(a.rstd + first + r) : 0.0f;
        }
    };
    fetch(row, rows);
    for (uint64_t r0 = blockIdx.x * at_once; r0 < a.rows; r0 += step) {
        float s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            px[r] = nx[r];
            pg[r] = ng[r];
            mean[r] = -next_mean[r];
            rstd[r] = next_rstd[r];
        }
        x += step * a.x_stride;
        dy += step * a.dy_stride;
        const int next_rows = rows_left(row + step, R, a.rows);
        fetch(row + step, next_rows);
        // columns past d and rows past the end hold dy = 0 and drop out of all four sums
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2 v[kPairs], g[kPairs];
            px[r].unpack(v);
            pg[r].unpack(g);
            const f32x2 m = pair(mean[r]), p = pair(rstd[r]);
            f32x2 s1 = pair(0.0f), s2 = pair(0.0f);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                const f32x2 xhat = mul2(add2(v[i], m), p), u = mul2(g[i], w[i]);
                db[i] = add2(db[i], g[i]);
                dw[i] = fma2(g[i], xhat, dw[i]);
                s1 = add2(s1, u);
                s2 = fma2(u, xhat, s2);
            }
            s[2 * r] = sum2(s1);
            s[2 * r + 1] = sum2(s2);
        }
        sum(s, [&](float q) { return -q * a.inv_d; });
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!a.y || r >= rows) break;
            f32x2 v[kPairs], g[kPairs];
            px[r].unpack(v);
            pg[r].unpack(g);
            const f32x2 m = pair(mean[r]), p = pair(rstd[r]), c1 = pair(s[2 * r]), c2 = pair(s[2 * r + 1]);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) g[i] = mul2(p, fma2(mul2(add2(v[i], m), p), c2, fma2(g[i], w[i], c1)));
            store_part<T, NC, VEC>(dx + r * a.y_stride, left, a.tpr, g);
        }
        row += step;
        dx += step * a.y_stride;
        rows = next_rows;
    }
    if (!a.partials) return;
    // the groups' column sums, in order, through shared memory: [groups][2][d]
    if (a.groups > 1) {
        __syncthreads();
        float *mine = sh + (size_t)group * 2 * a.d;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const uint32_t c = column<NC, VEC>(i, t, a.tpr);
            if (c < a.d) {
                mine[c] = half_of(dw[i / 2], i & 1);
                mine[a.d + c] = half_of(db[i / 2], i & 1);
            }
        }
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < 2 * a.d; c += blockDim.x) {
            float v = 0.0f;
            for (uint32_t g = 0; g < a.groups; ++g) v += sh[(size_t)g * 2 * a.d + c];
            keep_partial(a, a.partials + (size_t)blockIdx.x * 2 * a.d + c, v);
        }
        return;
    }
    float *out = a.partials + (size_t)blockIdx.x * 2 * a.d;
    if (VEC && a.add) { // beforehand, all reads side by side (element forms have no registers left for it)
#pragma unroll
        for (int i = 0; i < NC; i += 2) {
            const uint32_t c = column<NC, VEC>(i, t, a.tpr), e = column<NC, VEC>(i + 1, t, a.tpr);
            dw[i / 2] = add2(dw[i / 2], pair(c < a.d ? __ldcg(out + c) : 0.0f, e < a.d ? __ldcg(out + e) : 0.0f));
            db[i / 2] = add2(db[i / 2], pair(c < a.d ? __ldcg(out + a.d + c) : 0.0f, e < a.d ? __ldcg(out + a.d + e) : 0.0f));
        }
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const uint32_t c = column<NC, VEC>(i, t, a.tpr);
        if (c < a.d) {
            if (VEC) {
                out[c] = half_of(dw[i / 2], i & 1);
                out[a.d + c] = half_of(db[i / 2], i & 1);
            } else {
                keep_partial(a, out + c, half_of(dw[i / 2], i & 1));
                keep_partial(a, out + a.d + c, half_of(db[i / 2], i & 1));
            }
        }
    }
}

// ------------------------------------------------------------------ a warp a row
// Rows of up to 2048 columns that vector accesses can read: a lane holds K pieces of 8 columns, 256 columns apart, and
// a row's sums need five shuffles and no barrier.  The weight and the bias wait in shared memory as fp32.
constexpr int kWarpThreads = 128;
constexpr uint32_t kWarpCols = 2048;

template <typename W>
__device__ __forceinline__ void vector_to_shared(float *sh, const void *v, float missing, uint32_t d, uint32_t cols)
{
    for (uint32_t c = threadIdx.x; c < cols; c += kWarpThreads) sh[c] = c < d && v ? to_f32(static_cast<const W *>(v)[c]) : missing;
}
__device__ __forceinline__ void shared8(const float *sh, f32x2 (&p)[4])
{
    const float4 a = reinterpret_cast<const float4 *>(sh)[0], b = reinterpret_cast<const float4 *>(sh)[1];
    p[0] = pair(a.x, a.y), p[1] = pair(a.z, a.w), p[2] = pair(b.x, b.y), p[3] = pair(b.z, b.w);
}
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T> &raw, f32x2 (&p)[4])
{
    float f[8];
    raw.unpack(f);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pair(f[2 * i], f[2 * i + 1]);
}
template <typename T>
__device__ __forceinline__ void store8(T *at, const f32x2 (&p)[4])
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpair(p[i], f[2 * i], f[2 * i + 1]);
    a2sgd_train::store8(at, f);
}
__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

template <typename T, typename W, int K>
__global__ void __launch_bounds__(kWarpThreads) k_ln_forward_warp(const __grid_constant__ LnArgs a)
{
    __shared__ __align__(16) float w[256 * K], b[256 * K];
    const uint32_t lane = threadIdx.x & 31;
    wait_prior_grid();
    release_next_grid();
    const bool last = (K - 1) * 256 + lane * 8 < a.d; // of the pieces only the last one may not exist
    const uint64_t step = (uint64_t)gridDim.x * (kWarpThreads / 32);
    uint64_t row = blockIdx.x * (kWarpThreads / 32) + (threadIdx.x >> 5);
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.x_stride + lane * 8;
    T *y = static_cast<T *>(a.y) + (int64_t)row * a.y_stride + lane * 8;
    Raw8<T> next[K];
    const auto fetch = [&](bool live) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (live && (k < K - 1 || last)) next[k].load(x + k * 256);
            else next[k].zero();
        }
    };
    fetch(row < a.rows);
    vector_to_shared<W>(w, a.w, 1.0f, a.d, 256 * K);
    vector_to_shared<W>(b, a.b, 0.0f, a.d, 256 * K);
    __syncthreads();
    while (row < a.rows) {
        f32x2 v[K][4];
#pragma unroll
        for (int k = 0; k < K; ++k) unpack8(next[k], v[k]);
        x += step * a.x_stride;
        fetch(row + step < a.rows); // on its way while this row is worked on
        f32x2 s = pair(0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s = add2(s, v[k][i]);
        }
        const float mean = warp_sum(sum2(s)) * a.inv_d;
        const f32x2 m = pair(-mean);
        float var = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            s = pair(0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[k][i] = add2(v[k][i], m);
                s = fma2(v[k][i], v[k][i], s);
            }
            var += k < K - 1 || last ? sum2(s) : 0.0f;
        }
        const float rstd = 1.0f / sqrtf(fmaf(warp_sum(var), a.inv_d, a.eps));
        const f32x2 p = pair(rstd);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            f32x2 wk[4], bk[4];
            shared8(w + k * 256 + lane * 8, wk);
            shared8(b + k * 256 + lane * 8, bk);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k][i] = fma2(mul2(v[k][i], p), wk[i], bk[i]);
            if (k < K - 1 || last) store8(y + k * 256, v[k]);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        row += step;
        y += step * a.y_stride;
    }
}

// The CTAs' column sums, added up in order: 32 columns a CTA, 32 slices of the CTAs side by side.
template <typename W>
__global__ void __launch_bounds__(kMaxThreads) k_ln_fold(const __grid_constant__ LnArgs a)
{
    __shared__ float sh[kMaxThreads / kFoldCols][kFoldCols + 1];
    wait_prior_grid();
    release_next_grid();
    const uint32_t lane = threadIdx.x % kFoldCols, slice = threadIdx.x / kFoldCols;
    const uint32_t c = blockIdx.x * kFoldCols + lane; // of the 2 d columns dw | db
    float v = 0.0f;
    if (c < 2 * a.d) {
#pragma unroll 4
        for (uint32_t p = slice; p < a.parts; p += kMaxThreads / kFoldCols) v += __ldcg(a.partials + (size_t)p * 2 * a.d + c);
    }
    sh[slice][lane] = v;
    __syncthreads();
    if (slice == 0 && c < 2 * a.d) {
        v = 0.0f;
        for (uint32_t k = 0; k < kMaxThreads / kFoldCols; ++k) v += sh[k][lane];
        W *out = static_cast<W *>(c < a.d ? a.dw : a.db);
        if (out) out[c < a.d ? c : c - a.d] = from_f32<W>(v);
    }
}

// ------------------------------------------------------------------ rows of any length
__device__ __forceinline__ float block_sum(float v, float *sh)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads(); // the last sum has been read
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0f;
    for (uint32_t k = 0; k < blockDim.x / 32; ++k) v += sh[k];
    return v;
}

// N sums over a thread's columns of a row, in runs of kRun terms: term(c, run) adds a column's.  Unrolled as measured: at
// 4096 x 12288 bf16 forward 152 and 175 us by four and by two, backward 361 and 295 (registers: 44 and 32 a thread).
template <int N, typename F>
__device__ __forceinline__ void strided_sums(uint32_t d, float (&total)[N], F term)
{
#pragma unroll
    for (int i = 0; i < N; ++i) total[i] = 0.0f;
    uint32_t c = threadIdx.x;
    do {
        const uint32_t end = min(d, c + kRun * kMaxThreads);
        float run[N] = {};
#pragma unroll (N == 1 ? 4 : 2)
        for (; c < end; c += kMaxThreads) term(c, run);
#pragma unroll
        for (int i = 0; i < N; ++i) total[i] += run[i];
    } while (c < d);
}

template <typename T, typename W>
__global__ void __launch_bounds__(kMaxThreads) k_ln_forward_long(const __grid_constant__ LnArgs a)
{
    __shared__ float sh[kMaxThreads / 32];
    wait_prior_grid();
    release_next_grid();
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.x_stride;
        T *y = static_cast<T *>(a.y) + (int64_t)row * a.y_stride;
        float sum[1];
        strided_sums(a.d, sum, [&](uint32_t c, float (&v)[1]) { v[0] += to_f32(x[c]); });
        const float mean = block_sum(sum[0], sh) * a.inv_d;
        strided_sums(a.d, sum, [&](uint32_t c, float (&v)[1]) {
            const float e = to_f32(x[c]) - mean;
            v[0] = fmaf(e, e, v[0]);
        });
        const float rstd = 1.0f / sqrtf(fmaf(block_sum(sum[0], sh), a.inv_d, a.eps));
        for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
            const float w = a.w ? to_f32(static_cast<const W *>(a.w)[c]) : 1.0f;
            const float b = a.b ? to_f32(static_cast<const W *>(a.b)[c]) : 0.0f;
            y[c] = from_f32<T>(fmaf((to_f32(x[c]) - mean) * rstd, w, b));
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Column sums of a slice of the rows: one thread a column.
template <typename T>
__global__ void __launch_bounds__(256) k_ln_columns_long(const __grid_constant__ LnArgs a)
{
    wait_prior_grid();
    release_next_grid();
    const uint32_t c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.d) return;
    float dw = 0.0f, db = 0.0f;
    for (uint64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float g = to_f32((static_cast<const T *>(a.dy) + (int64_t)row * a.dy_stride)[c]);
        const float x = to_f32((static_cast<const T *>(a.x) + (int64_t)row * a.x_stride)[c]);
        db += g;
        dw = fmaf(g, (x - a.mean[row]) * a.rstd[row], dw);
    }
    keep_partial(a, a.partials + (size_t)blockIdx.y * 2 * a.d + c, dw);
    keep_partial(a, a.partials + (size_t)blockIdx.y * 2 * a.d + a.d + c, db);
}

template <typename T, typename W>
__global__ void __launch_bounds__(kMaxThreads) k_ln_backward_long(const __grid_constant__ LnArgs a)
{
    __shared__ float sh[kMaxThreads / 32];
    wait_prior_grid();
    release_next_grid();
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.x_stride;
        const T *dy = static_cast<const T *>(a.dy) + (int64_t)row * a.dy_stride;
        T *dx = static_cast<T *>(a.y) + (int64_t)row * a.y_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s[2];
        strided_sums(a.d, s, [&](uint32_t c, float (&v)[2]) {
            const float u = to_f32(dy[c]) * (a.w ? to_f32(static_cast<const W *>(a.w)[c]) : 1.0f);
            v[0] += u;
            v[1] = fmaf(u, (to_f32(x[c]) - mean) * rstd, v[1]);
        });
        const float c1 = block_sum(s[0], sh) * a.inv_d, c2 = block_sum(s[1], sh) * a.inv_d;
        for (uint32_t c = threadIdx.x; c < a.d; c += blockDim.x) {
            const float w = a.w ? to_f32(static_cast<const W *>(a.w)[c]) : 1.0f;
            const float xhat = (to_f32(x[c]) - mean) * rstd;
            dx[c] = from_f32<T>(rstd * (fmaf(to_f32(dy[c]), w, -c1) - xhat * c2));
        }
    }
}

// ------------------------------------------------------------------ host
struct Plan {
    const void *fn = nullptr;
    bool long_row = false;
    uint32_t tpr = 0, groups = 0;
    int nc = 0, r = 0;
    unsigned threads = 0, grid = 0;
    size_t smem = 0;
};

template <typename T, typename W>
const void *pick_warp(int k)
{
#define A2_LNW(K) \
    if (k == K) return reinterpret_cast<const void *>(&k_ln_forward_warp<T, W, K>);
    A2_LNW(2) A2_LNW(3) A2_LNW(4) A2_LNW(5) A2_LNW(6) A2_LNW(7) A2_LNW(8)
#undef A2_LNW
    return nullptr;
}

// Rows in flight of a group (and as many being worked on), where there are rows enough: the backward pass has twice
// the registers of a row to hold, rows without vector accesses hold an element a register.
template <bool BWD, bool VEC>
constexpr int kRows = VEC && !BWD ? 4 : 2;

template <typename T, typename W, bool BWD, int NC, int R, bool VEC>
const void *row_kernel()
{
    if constexpr (BWD) return reinterpret_cast<const void *>(&k_ln_backward<T, W, NC, R, VEC>);
    else return reinterpret_cast<const void *>(&k_ln_forward<T, W, NC, R, VEC>);
}
template <typename T, typename W, bool BWD, bool VEC>
const void *pick_rows(int nc, int r)
{
    if (nc == 16) return row_kernel<T, W, BWD, 16, 1, VEC>();
    return r == 1 ? row_kernel<T, W, BWD, 8, 1, VEC>() : row_kernel<T, W, BWD, 8, kRows<BWD, VEC>, VEC>();
}
template <typename T, typename W, bool BWD>
const void *pick(int nc, int r, bool vec)
{
    return vec ? pick_rows<T, W, BWD, true>(nc, r) : pick_rows<T, W, BWD, false>(nc, r);
}

template <bool BWD>
const void *pick_types(int dtype, int param, int nc, int r, bool vec)
{
    if (dtype == A2SGD_F32) return pick<float, float, BWD>(nc, r, vec);
    if (dtype == A2SGD_BF16)
        return param == A2SGD_F32 ? pick<__nv_bfloat16, float, BWD>(nc, r, vec)
                                  : pick<__nv_bfloat16, __nv_bfloat16, BWD>(nc, r, vec);
    return param == A2SGD_F32 ? pick<__half, float, BWD>(nc, r, vec) : pick<__half, __half, BWD>(nc, r, vec);
}
const void *pick_warp_types(int dtype, int param, int k)
{
    if (dtype == A2SGD_F32) return pick_warp<float, float>(k);
    if (dtype == A2SGD_BF16) return param == A2SGD_F32 ? pick_warp<__nv_bfloat16, float>(k) : pick_warp<__nv_bfloat16, __nv_bfloat16>(k);
    return param == A2SGD_F32 ? pick_warp<__half, float>(k) : pick_warp<__half, __half>(k);
}

#define A2_LN_LONG(name)                                                                                         \
    const void *name##_of(int dtype, int param)                                                                  \
    {                                                                                                            \
        if (dtype == A2SGD_F32) return reinterpret_cast<const void *>(&name<float, float>);                      \
        if (dtype == A2SGD_BF16)                                                                                 \
            return param == A2SGD_F32 ? reinterpret_cast<const void *>(&name<__nv_bfloat16, float>)              \
                                      : reinterpret_cast<const void *>(&name<__nv_bfloat16, __nv_bfloat16>);     \
        return param == A2SGD_F32 ? reinterpret_cast<const void *>(&name<__half, float>)                         \
                                  : reinterpret_cast<const void *>(&name<__half, __half>);                       \
    }
A2_LN_LONG(k_ln_forward_long)
A2_LN_LONG(k_ln_backward_long)
#undef A2_LN_LONG

// Column slices of the long form's column sums.
inline uint32_t long_parts(uint64_t rows) { return (uint32_t)std::min<uint64_t>(64, std::max<uint64_t>(1, rows / 16)); }

constexpr int kCtasPerSm = 4; // at most: the partial sums of the backward pass are sized by it

Plan make_plan(uint64_t rows, uint32_t d, bool vec, bool backward, int sms, int device, int dtype, int param)
{
    Plan p;
    if (d > kMostCols) {
        p.long_row = true;
        p.threads = kMaxThreads;
        p.grid = (unsigned)std::min<uint64_t>(rows, (uint64_t)sms * 2);
        p.fn = backward ? k_ln_backward_long_of(dtype, param) : k_ln_forward_long_of(dtype, param);
        return p;
    }
    if (vec && !backward && d > 256 && d <= kWarpCols && (dtype == A2SGD_F32 || d % 256)) {
        // A warp a row wins by its few instructions once a warp has rows enough to hide its start, ten or more here, and
        // where a row's threads of 8 columns each would not be whole warps, or read fp32.  This form against the other, us: bf16, 1600
        // columns, 65536 rows (37 a warp) 75 and 82, 32768 42 and 43, 16384 25.5 and 23.2, 8192 (5 a warp) 17.1 and 13.0; 264 columns, 65536
        // and 32768 rows 20.0 and 23.5, 11.5 and 12.9; fp32, 65536 rows, 512, 1024 and 2048 columns 51 and 57, 101 and 106, 200 and 210, 8192
        // rows 10.2 and 10.0, 18.5 and 18.1, 36 and 29.  Whole warps in 16 bits, 65536 rows, 512, 1024 and 2048 columns: 27.0
        // and 25.9, 48.9 and 48.2, 93.3 and 92.5, and worse for fewer: the other form.
        const void *fn = pick_warp_types(dtype, param, (int)(d + 255) / 256);
        const uint64_t resident = (uint64_t)sms * resident_ctas(fn, kWarpThreads, 0, device);
        if (rows >= resident * (kWarpThreads / 32) * 10) {
            p.threads = kWarpThreads;
            p.fn = fn;
            p.grid = (unsigned)resident;
            return p;
        }
    }
    p.nc = d <= (uint32_t)kRowThreads * 8 ? 8 : 16;
    const uint32_t need = (d + p.nc - 1) / p.nc; // threads that have columns
    if (need <= 32) {
        p.tpr = 1;
        while (p.tpr < need) p.tpr *= 2;
    } else {
        p.tpr = (need + 31) / 32 * 32;
    }
    // short rows share a CTA of up to 256 threads
    p.groups = p.tpr <= 128 ? 256 / p.tpr : 1;
    p.groups = std::max(1u, std::min<uint32_t>(p.groups, 64));
    if ((uint64_t)p.groups > rows) p.groups = (uint32_t)std::max<uint64_t>(1, rows);
    // whole warps
    while (p.tpr * p.groups % 32) ++p.groups;
    p.threads = p.tpr * p.groups;
    // several rows in flight where there are enough to keep every SM busy with them
    const bool several = p.nc == 8 && rows >= (uint64_t)sms * p.groups * 8;
    p.r = !several ? 1 : backward ? (vec ? kRows<true, true> : kRows<true, false>) : vec ? kRows<false, true> : kRows<false, false>;
    const size_t sums = sizeof(float) * 2 * (kRowThreads / 32) * (backward ? 2 : 1) * p.r;
    p.smem = std::max(sums, backward && p.groups > 1 ? sizeof(float) * 2 * d * p.groups : (size_t)0);
    p.fn = backward ? pick_types<true>(dtype, param, p.nc, p.r, vec) : pick_types<false>(dtype, param, p.nc, p.r, vec);
    // every CTA resident at once: the rows are dealt out evenly
    const uint64_t trips = (rows + (uint64_t)p.groups * p.r - 1) / ((uint64_t)p.groups * p.r);
    const uint64_t slots = (uint64_t)sms * std::min(kCtasPerSm, resident_ctas(p.fn, p.threads, p.smem, device));
    p.grid = (unsigned)std::min<uint64_t>(trips, slots);
    return p;
}

int check(const void *x, int64_t x_stride, int dtype, int param, uint64_t rows, uint32_t d)
{
    if (!known(dtype) || (param != A2SGD_F32 && param != dtype) || d == 0 || d >= (1u << 30) || rows >= (1ull << 40))
        return A2SGD_ERR_ARG;
    if (rows == 0) return A2SGD_OK;
    if (!x || (rows > 1 && x_stride < (int64_t)d)) return A2SGD_ERR_ARG;
    return aligned(x, size_of(dtype)) ? A2SGD_OK : A2SGD_ERR_ALIGN;
}

inline bool rows_vector(const void *p, int64_t stride, uint64_t rows, int dtype)
{
    return aligned(p, 16) && (rows <= 1 || (size_t)stride * size_of(dtype) % 16 == 0);
}

int run(const Plan &p, LnArgs &a, cudaStream_t s)
{
    void *params[] = {&a};
    A2_TRAIN_CUDA(launch(p.fn, dim3(p.grid), p.threads, p.smem, params, s));
    return A2SGD_OK;
}

} // namespace

extern "C" int a2sgd_layer_norm_forward(const void *x, int64_t x_stride, int dtype, const void *weight, const void *bias,
                                        int param_dtype, void *y, int64_t y_stride, float *mean, float *rstd,
                                        uint64_t rows, uint32_t d, double eps, int device, void *stream)
{
    int rc = check(x, x_stride, dtype, param_dtype, rows, d);
    if (rc == A2SGD_OK && rows) rc = check(y, y_stride, dtype, param_dtype, rows, d);
    if (rc != A2SGD_OK) return rc;
    if (!std::isfinite(eps) || !(eps >= 0.0)) return A2SGD_ERR_ARG;
    if (!aligned(weight, size_of(param_dtype)) || !aligned(bias, size_of(param_dtype)) || !aligned(mean, 4) || !aligned(rstd, 4))
        return A2SGD_ERR_ALIGN;
    if (rows == 0) return A2SGD_OK;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms == 0) return A2SGD_ERR_CUDA;
    const bool vec = d % 8 == 0 && rows_vector(x, x_stride, rows, dtype) && rows_vector(y, y_stride, rows, dtype);
    const Plan p = make_plan(rows, d, vec, false, sms, device, dtype, param_dtype);
    LnArgs a{};
    a.x = x;
    a.w = weight;
    a.b = bias;
    a.y = y;
    a.mean = mean;
    a.rstd = rstd;
    a.x_stride = x_stride;
    a.y_stride = y_stride;
    a.rows = rows;
    a.d = d;
    a.tpr = p.tpr;
    a.groups = p.groups;
    a.inv_d = 1.0f / (float)d;
    a.eps = (float)eps;
    return run(p, a, static_cast<cudaStream_t>(stream));
}

extern "C" uint64_t a2sgd_layer_norm_workspace(uint64_t rows, uint32_t d, int device)
{
    (void)rows;
    const int sms = sm_count(device);
    // the partial sums of dw and db: one pair of rows a CTA (or a slice, for long rows)
    return sizeof(float) * 2 * (uint64_t)d * (uint64_t)(d > kMostCols ? 64 : std::max(1, sms) * kCtasPerSm);
}

extern "C" int a2sgd_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int dtype,
                                         const void *weight, int param_dtype, const float *mean, const float *rstd,
                                         void *dx, int64_t dx_stride, void *dweight, void *dbias, uint64_t rows, uint32_t d,
                                         void *workspace, uint64_t workspace_bytes, int device, void *stream)
{
    int rc = check(x, x_stride, dtype, param_dtype, rows, d);
    if (rc == A2SGD_OK && rows) rc = check(dy, dy_stride, dtype, param_dtype, rows, d);
    if (rc == A2SGD_OK && rows && dx) rc = check(dx, dx_stride, dtype, param_dtype, rows, d);
    if (rc != A2SGD_OK) return rc;
    if (rows && (!mean || !rstd)) return A2SGD_ERR_ARG;
    const size_t pe = size_of(param_dtype);
    if (!aligned(weight, pe) || !aligned(dweight, pe) || !aligned(dbias, pe) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(workspace, 4))
        return A2SGD_ERR_ALIGN;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms == 0) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (rows == 0) { // no rows: the sums are zero
        if (dweight) A2_TRAIN_CUDA(cudaMemsetAsync(dweight, 0, pe * d, s));
        if (dbias) A2_TRAIN_CUDA(cudaMemsetAsync(dbias, 0, pe * d, s));
        return A2SGD_OK;
    }
    const bool columns = dweight || dbias;
    if (!columns && !dx) return A2SGD_OK;
    const bool vec = d % 8 == 0 && rows_vector(x, x_stride, rows, dtype) && rows_vector(dy, dy_stride, rows, dtype) &&
                     (!dx || rows_vector(dx, dx_stride, rows, dtype));
    const Plan p = make_plan(rows, d, vec, true, sms, device, dtype, param_dtype);
    LnArgs a{};
    a.x = x;
    a.dy = dy;
    a.w = weight;
    a.y = dx;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.x_stride = x_stride;
    a.dy_stride = dy_stride;
    a.y_stride = dx_stride;
    a.rows = rows;
    a.d = d;
    a.tpr = p.tpr;
    a.groups = p.groups;
    a.inv_d = 1.0f / (float)d;
    a.dw = dweight;
    a.db = dbias;
    a.parts = p.long_row ? long_parts(rows) : p.grid;
    a.partials = columns ? static_cast<float *>(workspace) : nullptr;
    if (columns && (!workspace || workspace_bytes < sizeof(float) * 2 * (uint64_t)d * a.parts)) return A2SGD_ERR_ARG;
    // Rows whose column sums take more than kRun terms a thread are taken in as many launches as that makes runs.
    const auto launch_runs = [&](uint64_t most, auto &&go) {
        if (rows <= most) {
            rc = go();
            return;
        }
        const LnArgs whole = a;
        for (uint64_t first = 0; rc == A2SGD_OK && first < rows; first += most) {
            a.rows = std::min(most, rows - first);
            a.x = static_cast<const char *>(x) + (int64_t)first * x_stride * (int64_t)size_of(dtype);
            a.dy = static_cast<const char *>(dy) + (int64_t)first * dy_stride * (int64_t)size_of(dtype);
            if (dx) a.y = static_cast<char *>(dx) + (int64_t)first * dx_stride * (int64_t)size_of(dtype);
            a.mean = whole.mean + first;
            a.rstd = whole.rstd + first;
            a.add = first != 0;
            rc = go();
        }
        a = whole;
    };
    if (p.long_row) {
        if (columns) { // before dx, which may take the place of x or dy
            const void *fn = dtype == A2SGD_F32    ? reinterpret_cast<const void *>(&k_ln_columns_long<float>)
                             : dtype == A2SGD_BF16 ? reinterpret_cast<const void *>(&k_ln_columns_long<__nv_bfloat16>)
                                                   : reinterpret_cast<const void *>(&k_ln_columns_long<__half>);
            launch_runs((uint64_t)kRun * a.parts, [&]() -> int {
                void *params[] = {&a};
                A2_TRAIN_CUDA(launch(fn, dim3((d + 255) / 256, a.parts), 256, 0, params, s));
                return A2SGD_OK;
            });
        }
        if (rc == A2SGD_OK && dx) rc = run(p, a, s);
    } else {
        launch_runs(columns ? (uint64_t)kRun * p.grid * p.groups : rows, [&] { return run(p, a, s); });
    }
    if (rc != A2SGD_OK || !columns) return rc;
    const void *fold = param_dtype == A2SGD_F32    ? reinterpret_cast<const void *>(&k_ln_fold<float>)
                       : param_dtype == A2SGD_BF16 ? reinterpret_cast<const void *>(&k_ln_fold<__nv_bfloat16>)
                                                   : reinterpret_cast<const void *>(&k_ln_fold<__half>);
    void *params[] = {&a};
    A2_TRAIN_CUDA(launch(fold, dim3((2 * d + kFoldCols - 1) / kFoldCols), kMaxThreads, 0, params, s));
    return A2SGD_OK;
}
