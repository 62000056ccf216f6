// The residual connection of a block with its gate, its scale, the norm after the block and the norm before the next one.
//
//   forward   n = norm(y) w1 + b1,  z = x + alpha gate n,  u = norm(z) w2 + b2
//   backward  t = dz + back(du w2; z),  dx = t,  dn = alpha gate t,  dy = back(dn w1; y),  and the columns' sums
//
// Bound by memory: forward reads x, y and writes z, u; backward reads dz, du, y, z and writes dx, dy.  A CTA takes a run of
// consecutive rows, one after another, a row's elements in its threads' registers, the parameters in shared memory; the next row's are on
// their way while the present one is worked on.  Each norm costs one barrier: a warp forms its own mean and sum of squares about it by shuffles, and
// the warps' are joined from shared memory (Chan's formula), so that no element is squared about anything but a mean near its own.
//
// The columns' sums: t hat1 and t (from which the gate's, the post weight's and the post bias' gradients follow, a gate at a time), du hat2
// and du.  A CTA adds its rows up in registers or shared memory, leaves one partial sum a column, and a second kernel adds the CTAs' in order.  No chain
// of additions has more than 512 terms: after 512 rows, or at a gate's end, a sum goes to memory, after 512 of those to the next place.
//
// Statistics, sums and z before its rounding are fp32; z and u (dx and dy) are rounded once, as they are written.
//
// B200, 65536 x 1600, bfloat16: forward with an fp32 residual stream 256 us (4.9 TB/s, 75 % of a copy's; 280 among other work), four CTAs of 224 threads an SM: a row's two
// barriers and the little that is on its way meanwhile bound it (two rows on their way take the registers of a CTA: 306 us; parameters read from
// memory for each row 761).  Backward of a layer norm 361 us (3.5 TB/s), of which the fold is 15: three CTAs an SM (80 registers, beyond which 8 bytes a
// thread spill; with an fp32 stream 40, all in fp32 136, one element an access 184 to 216, and above 4096 columns 108 to 132 there; two CTAs 405
// us).  16 rows: 7.0 us on the device, 11 a call.  A gate of few rows costs its sums' way to memory: 64 rows a gate 878 us.
#include "a2sgd_train.cuh"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

using namespace a2sgd_train;

namespace {

constexpr int kMostThreads = 512;
constexpr int kSums = 4; // t hat1, t, du hat2, du
constexpr int kStrips = 32;
constexpr int kRun = 512; // terms of a running sum (7812 equal terms in one chain were off by 1.2e-4 of their sum)

struct Rows {
    void *p;
    int64_t ld;
};
struct Args {
    Rows x, y, z, u, dz, du, dx, dy;
    const void *w1, *b1, *gate, *w2, *b2;
    float *mean1, *rstd1, *mean2, *rstd2;
    int64_t rows, gate_rows, run; // rows of a CTA
    int d, param, rms, post;
    float alpha, eps;
    // backward
    void *dw1, *db1, *dgate, *dw2, *db2;
    float *partials;      // [CTAs][4][d]: dw1, db1, dw2, db2
    float *runs;          // [CTAs][4][d]: up to kRun terms of those each; NULL where every CTA puts its sums down but once
    float *gate_partials; // [CTAs][2][d]
    int ctas;
};

__device__ __forceinline__ float param_at(const void *p, int type, int64_t i)
{
    if (type == A2SGD_F32) return static_cast<const float *>(p)[i];
    if (type == A2SGD_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(static_cast<const __half *>(p)[i]);
}
__device__ __forceinline__ void param_put(void *p, int type, int64_t i, float v)
{
    if (type == A2SGD_F32) static_cast<float *>(p)[i] = v;
    else if (type == A2SGD_BF16) static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half *>(p)[i] = __float2half_rn(v);
}

// Eight elements of a thread: consecutive ones, or ones a CTA's threads apart (any alignment).
template <typename T, int VEC>
struct Eight;
template <typename T>
struct Eight<T, 8> {
    Raw8<T> raw;
    __device__ __forceinline__ void load(const T *row, int chunk, int d)
    {
        const int c = (chunk * (int)blockDim.x + (int)threadIdx.x) * 8;
        if (c < d) raw.load(row + c);
        else raw.zero();
    }
    __device__ __forceinline__ void unpack(float (&f)[8]) const { raw.unpack(f); }
    __device__ static __forceinline__ void store(T *row, int chunk, int d, const float (&f)[8])
    {
        const int c = (chunk * (int)blockDim.x + (int)threadIdx.x) * 8;
        if (c < d) store8(row + c, f);
    }
};
template <typename T>
struct Eight<T, 1> {
    T v[8];
    __device__ __forceinline__ void load(const T *row, int chunk, int d)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = (chunk * 8 + i) * (int)blockDim.x + (int)threadIdx.x;
            v[i] = c < d ? row[c] : from_f32<T>(0.0f);
        }
    }
    __device__ __forceinline__ void unpack(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = to_f32(v[i]);
    }
    __device__ static __forceinline__ void store(T *row, int chunk, int d, const float (&f)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = (chunk * 8 + i) * (int)blockDim.x + (int)threadIdx.x;
            if (c < d) row[c] = from_f32<T>(f[i]);
        }
    }
};
template <int VEC>
__device__ __forceinline__ int column(int chunk, int i)
{
    return VEC == 8 ? (chunk * (int)blockDim.x + (int)threadIdx.x) * 8 + i : (chunk * 8 + i) * (int)blockDim.x + (int)threadIdx.x;
}
// Parameters as the rows need them, in fp32, in shared memory: vector k of a CTA's columns, zeros past the end.  Eight columns of a thread lie
// together where its elements do, so that they come in two 128-bit accesses; the parameters' own accesses are a CTA's start, or a gate's.
template <int VEC, int C>
struct Columns {
    float *p;
    __device__ __forceinline__ int span() const { return C * 8 * (int)blockDim.x; }
    template <typename F>
    __device__ __forceinline__ void fill(int k, int d, F value) const
    {
        for (int c = threadIdx.x; c < span(); c += blockDim.x) // VEC 8: the first four of each eight columns, then the second four: no bank twice
            p[k * span() + (VEC == 8 ? (c >> 2 & 1) * (span() / 2) + (c >> 3) * 4 + (c & 3) : c)] = c < d ? value(c) : 0.0f;
    }
    __device__ __forceinline__ void read(int k, int chunk, f32x2 (&f)[4]) const
    {
        if constexpr (VEC == 8) {
            const ulonglong2 *q = reinterpret_cast<const ulonglong2 *>(p + k * span() + column<8>(chunk, 0) / 2);
            const ulonglong2 x = q[0], y = q[span() / 8];
            f[0] = x.x, f[1] = x.y, f[2] = y.x, f[3] = y.y;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = pair(p[k * span() + column<1>(chunk, 2 * i)], p[k * span() + column<1>(chunk, 2 * i + 1)]);
        }
    }
};

// Eight numbers as four pairs.
__device__ __forceinline__ void pairs8(f32x2 (&p)[4], const float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pair(f[2 * i], f[2 * i + 1]);
}
__device__ __forceinline__ void singles8(float (&f)[8], const f32x2 (&p)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) unpair(p[i], f[2 * i], f[2 * i + 1]);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    return v;
}

// Two sums over the CTA's threads, in a fixed order.  slot: [2][warps] floats, not in use since the barrier before the last.
__device__ __forceinline__ void cta_sums(float &a, float &b, float *slot)
{
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
    a = warp_sum(a);
    b = warp_sum(b);
    if (warps > 1) {
        if ((threadIdx.x & 31) == 0) {
            slot[warp] = a;
            slot[16 + warp] = b;
        }
        __syncthreads();
        a = b = 0.0f;
        for (int w = 0; w < warps; ++w) {
            a += slot[w];
            b += slot[16 + w];
        }
    }
}

// The mean (0 for RMS) and 1 / sqrt(variance or mean square + eps) of a row whose elements the threads hold, zeros past its end.
template <int VEC, int C>
__device__ __forceinline__ void moments(const f32x2 (&v)[C][4], const Args &a, float *slot, float &mean, float &rstd)
{
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
    f32x2 pairs = pair(0.0f);
    float sum = 0.0f, square;
    if (a.rms) {
#pragma unroll
        for (int k = 0; k < C; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) pairs = fma2(v[k][i], v[k][i], pairs);
        square = sum2(pairs);
        cta_sums(sum, square, slot);
        mean = 0.0f;
        rstd = 1.0f / sqrtf(square / (float)a.d + a.eps);
        return;
    }
    int count = 0;
#pragma unroll
    for (int k = 0; k < C; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) pairs = add2(pairs, v[k][i]);
        if (VEC == 8) {
            count += column<VEC>(k, 0) < a.d ? 8 : 0;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) count += column<VEC>(k, i) < a.d;
        }
    }
    sum = warp_sum(sum2(pairs));
    const float n = (float)__reduce_add_sync(0xffffffffu, count), own = n > 0.0f ? sum / n : 0.0f;
    const f32x2 minus = pair(-own);
    pairs = pair(0.0f);
#pragma unroll
    for (int k = 0; k < C; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x2 e = add2(v[k][i], minus);
            if (VEC == 8 ? column<VEC>(k, 0) >= a.d : column<VEC>(k, 2 * i + 1) >= a.d) { // past the end
                float x, y;
                unpair(e, x, y);
                e = pair(column<VEC>(k, 2 * i) < a.d ? x : 0.0f, 0.0f);
            }
            pairs = fma2(e, e, pairs);
        }
    square = warp_sum(sum2(pairs));
    mean = own;
    if (warps > 1) {
        if ((threadIdx.x & 31) == 0) {
            slot[warp] = sum;
            slot[16 + warp] = square;
            slot[32 + warp] = n;
        }
        __syncthreads();
        sum = square = 0.0f;
        for (int w = 0; w < warps; ++w) sum += slot[w];
        mean = sum / (float)a.d;
        for (int w = 0; w < warps; ++w) {
            const float m = slot[32 + w], off = m > 0.0f ? slot[w] / m - mean : 0.0f;
            square += slot[16 + w] + m * off * off;
        }
    }
    rstd = 1.0f / sqrtf(square / (float)a.d + a.eps);
}

template <typename T, typename R, int VEC, int C, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 4 : C == 1 ? 2 : 1) k_forward(const __grid_constant__ Args a)
{
    extern __shared__ __align__(16) float columns[]; // alpha gate w1, alpha gate b1, w2, b2
    __shared__ float slots[2][48]; // in turn: one barrier a norm leaves no time to empty them
    int turn = 0;
    wait_prior_grid();
    release_next_grid();
    const int64_t row0 = (int64_t)blockIdx.x * a.run, end = min(a.rows, row0 + a.run);
    if (row0 >= end) return;
    const Columns<VEC, C> cols{columns};
    cols.fill(2, a.d, [&](int c) { return a.w2 ? param_at(a.w2, a.param, c) : 1.0f; });
    cols.fill(3, a.d, [&](int c) { return a.b2 ? param_at(a.b2, a.param, c) : 0.0f; });
    Eight<T, VEC> y[C];
    Eight<R, VEC> x[C];
    const auto bring = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            y[k].load(static_cast<const T *>(a.y.p) + r * a.y.ld, k, a.d);
            x[k].load(static_cast<const R *>(a.x.p) + r * a.x.ld, k, a.d);
        }
    };
    bring(row0);
    int64_t gate_end = row0; // rows from here on have another gate
    for (int64_t r = row0; r < end; ++r) {
        f32x2 n[C][4], z[C][4];
#pragma unroll
        for (int k = 0; k < C; ++k) {
            float f[8];
            y[k].unpack(f);
            pairs8(n[k], f);
            x[k].unpack(f);
            pairs8(z[k], f);
        }
        if (r + 1 < end) bring(r + 1);
        if (r == gate_end) {
            const int64_t group = a.gate ? r / a.gate_rows : 0;
            gate_end = a.gate ? min(end, (group + 1) * a.gate_rows) : end;
            __syncthreads();
            const auto gate = [&](int c) { return a.gate ? a.alpha * param_at(a.gate, a.param, group * a.d + c) : a.alpha; };
            cols.fill(0, a.d, [&](int c) { return gate(c) * (a.post && a.w1 ? param_at(a.w1, a.param, c) : 1.0f); });
            cols.fill(1, a.d, [&](int c) { return a.post && a.b1 ? gate(c) * param_at(a.b1, a.param, c) : 0.0f; });
            __syncthreads();
        }
        float mean = 0.0f, rstd = 1.0f;
        if (a.post) {
            moments<VEC, C>(n, a, slots[turn ^= 1], mean, rstd);
            if (threadIdx.x == 0) {
                if (a.mean1) a.mean1[r] = mean;
                if (a.rstd1) a.rstd1[r] = rstd;
            }
        }
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const f32x2 by = pair(rstd);
            f32x2 w[4], b[4];
            cols.read(0, k, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[k][i] = fma2(a.rms ? mul2(n[k][i], by) : mul2(add2(n[k][i], pair(-mean)), by), w[i], z[k][i]); // past the end: w is 0
            if (a.post && a.b1) {
                cols.read(1, k, b);
#pragma unroll
                for (int i = 0; i < 4; ++i) z[k][i] = add2(z[k][i], b[i]);
            }
            float f[8];
            singles8(f, z[k]);
            Eight<R, VEC>::store(static_cast<R *>(a.z.p) + r * a.z.ld, k, a.d, f);
        }
        moments<VEC, C>(z, a, slots[turn ^= 1], mean, rstd);
        if (threadIdx.x == 0) {
            if (a.mean2) a.mean2[r] = mean;
            if (a.rstd2) a.rstd2[r] = rstd;
        }
#pragma unroll
        for (int k = 0; k < C; ++k) {
            f32x2 w[4], b[4] = {};
            float u[8];
            cols.read(2, k, w);
            if (a.b2) cols.read(3, k, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = fma2(mul2(add2(z[k][i], pair(-mean)), pair(rstd)), w[i], b[i]);
            singles8(u, w);
            Eight<T, VEC>::store(static_cast<T *>(a.u.p) + r * a.u.ld, k, a.d, u);
        }
    }
}

template <typename T, typename R, int VEC, int C, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : 1) k_backward(const __grid_constant__ Args a)
{
    extern __shared__ __align__(16) float columns[]; // w2, alpha gate w1 (alpha gate without a norm), and the four sums: for C == 1 on their way out
    __shared__ float slots[2][48]; // in turn: one barrier a norm leaves no time to empty them
    int turn = 0;
    wait_prior_grid();
    release_next_grid();
    const int64_t row0 = (int64_t)blockIdx.x * a.run, end = min(a.rows, row0 + a.run);
    if (row0 >= end) return;
    const Columns<VEC, C> cols{columns};
    float *sums = columns + 2 * cols.span();
    const bool want = a.partials != nullptr;
    f32x2 acc[kSums][4] = {};
    const auto sum_at = [&](int s, int k, int i) -> float & { return sums[s * cols.span() + (k * 8 + i) * (int)blockDim.x + (int)threadIdx.x]; };
    if constexpr (C > 1) {
        for (int s = 0; s < kSums; ++s)
            for (int k = 0; k < C; ++k)
                for (int i = 0; i < 8; ++i) sum_at(s, k, i) = 0.0f;
    }
    cols.fill(0, a.d, [&](int c) { return a.w2 ? param_at(a.w2, a.param, c) : 1.0f; });
    Eight<T, VEC> y[C], du[C];
    Eight<R, VEC> z[C], dz[C];
    // what the next row starts with is asked for as soon as its place is free
    const auto bring_pre = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            du[k].load(static_cast<const T *>(a.du.p) + r * a.du.ld, k, a.d);
            z[k].load(static_cast<const R *>(a.z.p) + r * a.z.ld, k, a.d);
        }
    };
    const auto bring_post = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            y[k].load(static_cast<const T *>(a.y.p) + r * a.y.ld, k, a.d);
            if (a.dz.p) dz[k].load(static_cast<const R *>(a.dz.p) + r * a.dz.ld, k, a.d);
        }
    };
    float next_mean1 = 0.0f, next_rstd1 = 1.0f, next_mean2 = 0.0f, next_rstd2;
    const auto bring_stats = [&](int64_t r) {
        next_rstd2 = a.rstd2[r];
        if (!a.rms) next_mean2 = a.mean2[r];
        if (a.post) next_rstd1 = a.rstd1[r];
        if (a.post && !a.rms) next_mean1 = a.mean1[r];
    };
    bring_stats(row0);
    bring_pre(row0);
    bring_post(row0);
    int64_t gate_end = row0, group = 0; // rows from here on have another gate
    int puts = 0; // how often the sums of t were put down; those of du are after every kRun-th row
    const float per = 1.0f / (float)a.d;
    for (int64_t r = row0; r < end; ++r) {
        const float mean1 = next_mean1, rstd1 = next_rstd1, mean2 = next_mean2, rstd2 = next_rstd2;
        if (r + 1 < end) bring_stats(r + 1);
        if (r == gate_end) {
            group = a.gate ? r / a.gate_rows : 0;
            gate_end = a.gate ? min(end, (group + 1) * a.gate_rows) : end;
            __syncthreads();
            cols.fill(1, a.d, [&](int c) {
                const float g = a.gate ? a.alpha * param_at(a.gate, a.param, group * a.d + c) : a.alpha;
                return g * (a.post && a.w1 ? param_at(a.w1, a.param, c) : 1.0f);
            });
            __syncthreads();
        }
        // the norm before the next block: hat = norm(z), g = du w2
        f32x2 hat[C][4], t[C][4], s0s = pair(0.0f), s1s = pair(0.0f);
        const auto add_up = [&](int which, int k, int i, f32x2 v, f32x2 h) { // v h and v
            if constexpr (C == 1) {
                acc[which][i] = fma2(v, h, acc[which][i]);
                acc[which + 1][i] = add2(acc[which + 1][i], v);
            } else {
                float x, y, m, n;
                unpair(v, x, y);
                unpair(h, m, n);
                sum_at(which, k, 2 * i) += x * m;
                sum_at(which, k, 2 * i + 1) += y * n;
                sum_at(which + 1, k, 2 * i) += x;
                sum_at(which + 1, k, 2 * i + 1) += y;
            }
        };
#pragma unroll
        for (int k = 0; k < C; ++k) {
            f32x2 w[4];
            float f[8];
            cols.read(0, k, w);
            z[k].unpack(f);
            pairs8(hat[k], f);
            du[k].unpack(f);
            pairs8(t[k], f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hat[k][i] = mul2(add2(hat[k][i], pair(-mean2)), pair(rstd2)); // past the end t is 0
                if (want) add_up(2, k, i, t[k][i], hat[k][i]);
                t[k][i] = mul2(t[k][i], w[i]);
                s0s = add2(s0s, t[k][i]);
                s1s = fma2(t[k][i], hat[k][i], s1s);
            }
        }
        float s0 = sum2(s0s), s1 = sum2(s1s);
        if (r + 1 < end) bring_pre(r + 1);
        cta_sums(s0, s1, slots[turn ^= 1]);
        s0 = a.rms ? 0.0f : s0 * per;
        s1 *= per;
        // t, dx, and the norm after the block
        f32x2 p0s = pair(0.0f), p1s = pair(0.0f);
#pragma unroll
        for (int k = 0; k < C; ++k) {
            f32x2 w[4], e[4] = {};
            float f[8];
            if (a.dz.p) {
                dz[k].unpack(f);
                pairs8(e, f);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) t[k][i] = fma2(fma2(hat[k][i], pair(-s1), add2(t[k][i], pair(-s0))), pair(rstd2), e[i]);
            if (a.dx.p) {
                singles8(f, t[k]);
                Eight<R, VEC>::store(static_cast<R *>(a.dx.p) + r * a.dx.ld, k, a.d, f);
            }
            y[k].unpack(f);
            pairs8(hat[k], f);
            cols.read(1, k, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hat[k][i] = mul2(add2(hat[k][i], pair(-mean1)), pair(rstd1));
                if (want) add_up(0, k, i, t[k][i], hat[k][i]);
                t[k][i] = mul2(t[k][i], w[i]); // past the end w is 0
                p0s = add2(p0s, t[k][i]);
                p1s = fma2(t[k][i], hat[k][i], p1s);
            }
        }
        float p0 = sum2(p0s), p1 = sum2(p1s);
        if (r + 1 < end) bring_post(r + 1);
        if (a.post) {
            cta_sums(p0, p1, slots[turn ^= 1]);
            p0 = a.rms ? 0.0f : p0 * per;
            p1 *= per;
        }
        if (a.dy.p) {
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (a.post) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[k][i] = mul2(fma2(hat[k][i], pair(-p1), add2(t[k][i], pair(-p0))), pair(rstd1));
                }
                float f[8];
                singles8(f, t[k]);
                Eight<T, VEC>::store(static_cast<T *>(a.dy.p) + r * a.dy.ld, k, a.d, f);
            }
        }
        // what the rows since the last time give to the gate, the post weight and the post bias, and to the pre weight and bias
        if (want && ((r + 1 - row0) % kRun == 0 || r + 1 == gate_end)) {
            const int64_t runs = (r - row0) / kRun; // before this one
            const bool last = r + 1 == end, gate_over = r + 1 == gate_end, begun = runs * kRun + row0 > max(row0, group * a.gate_rows); // some of the gate's rows have been
            const bool du_due = last || (r + 1 - row0) % kRun == 0;
            const bool whole = a.gate && group * a.gate_rows >= row0 && min(a.rows, (group + 1) * a.gate_rows) <= end;
            const int slot = a.gate && group != row0 / a.gate_rows;
            const int64_t mine = (int64_t)blockIdx.x * kSums * a.d;
            const auto put = [&](int s, int c, int64_t n, float v) { // the n-th of a sum's runs
                float *sum = a.partials + mine + s * a.d + c, *run = a.runs + mine + s * a.d + c;
                const int place = (int)(n % kRun);
                if (place) v += *run;
                if (last || place == kRun - 1) *sum = n >= kRun ? *sum + v : v;
                else *run = v;
            };
            if constexpr (C == 1) { // through shared memory: a column at a time takes few registers
#pragma unroll
                for (int q = 0; q < kSums; ++q)
                    if (q < 2 || du_due) {
                        float f[8];
                        singles8(f, acc[q]);
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum_at(q, 0, i) = f[i];
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[q][i] = pair(0.0f);
                    }
            }
#pragma unroll 1
            for (int k = 0; k < C; ++k) {
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    const int c = column<VEC>(k, i);
                    if (c >= a.d) continue;
                    const auto take = [&](int q) {
                        const float v = sum_at(q, k, i);
                        if (C > 1) sum_at(q, k, i) = 0.0f;
                        return v;
                    };
                    const float one_hat = take(0), one = take(1);
                    if (a.dgate) {
                        const float w1 = a.post && a.w1 ? param_at(a.w1, a.param, c) : 1.0f, b1 = a.post && a.b1 ? param_at(a.b1, a.param, c) : 0.0f;
                        float *part = a.gate_partials + ((int64_t)blockIdx.x * 2 + slot) * a.d + c, v = a.alpha * fmaf(w1, one_hat, b1 * one);
                        if (begun) v += *part;
                        if (whole && gate_over) param_put(a.dgate, a.param, group * a.d + c, v);
                        else *part = v; // a whole gate's place is free: a first gate that has rows before this CTA, or a last one behind it, is another
                    }
                    const float f = a.gate ? a.alpha * param_at(a.gate, a.param, group * a.d + c) : a.alpha;
                    put(0, c, puts, f * one_hat);
                    put(1, c, puts, f * one);
                    if (du_due) {
                        put(2, c, runs, take(2));
                        put(3, c, runs, take(3));
                    }
                }
            }
            ++puts;
        }
    }
}

// The CTAs' sums, added up in order: blocks of 32 columns, 32 strips of CTAs each.  blockIdx.y: dw1, db1, dw2, db2, then the gates.
__global__ void __launch_bounds__(1024) k_fold(const __grid_constant__ Args a)
{
    __shared__ float part[kStrips][32];
    wait_prior_grid();
    release_next_grid();
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), strip = threadIdx.x >> 5;
    const int64_t groups = a.gate ? (a.rows + a.gate_rows - 1) / a.gate_rows : 0;
    for (int64_t job = blockIdx.y; job < kSums + groups; job += gridDim.y) {
        void *out;
        int64_t at = c;
        int first = 0, last = a.ctas - 1;
        if (job < kSums) {
            out = job == 0 ? a.dw1 : job == 1 ? a.db1 : job == 2 ? a.dw2 : a.db2;
        } else {
            const int64_t g = job - kSums;
            out = a.dgate;
            at += g * a.d;
            first = (int)(g * a.gate_rows / a.run);
            last = (int)((min(a.rows, (g + 1) * a.gate_rows) - 1) / a.run);
            if (first == last) out = nullptr; // written by the one CTA that had all of its rows
        }
        if (!out) continue;
        float sum = 0.0f;
        if (c < a.d) {
            const int count = last - first + 1, lo = first + count * strip / kStrips, hi = first + count * (strip + 1) / kStrips;
            const bool gate = job >= kSums;
            const float *p = (gate ? a.gate_partials : a.partials + job * a.d) + c;
            const int64_t step = (int64_t)(gate ? 2 : kSums) * a.d;
            // of a gate's CTAs only the first may have begun with another gate's rows, and then this gate's sums are its second ones
            const bool second = gate && first * a.run < (job - kSums) * a.gate_rows;
#pragma unroll 8
            for (int k = lo; k < hi; ++k) sum += __ldcg(p + k * step + (second && k == first ? a.d : 0));
        }
        part[strip][threadIdx.x & 31] = sum;
        __syncthreads();
        if (strip == 0 && c < a.d) {
            for (int k = 1; k < kStrips; ++k) sum += part[k][threadIdx.x];
            param_put(out, a.param, at, sum);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ host
struct Plan {
    int threads, chunks, vec, most; // threads that the kernel is compiled for
};
Plan plan_of(uint32_t d, bool vec)
{
    Plan p;
    p.vec = vec ? 8 : 1;
    p.chunks = d > 8u * kMostThreads ? 2 : 1;
    const int pieces = (int)(d + 8 * p.chunks - 1) / (8 * p.chunks);
    p.threads = (pieces + 31) / 32 * 32;
    p.most = p.threads <= 256 ? 256 : 512;
    return p;
}

template <typename T, typename R>
const void *pick(const Plan &p, bool backward)
{
#define A2_PICK(V, K, N)                                                                                         \
    if (p.vec == V && p.chunks == K && p.most == N)                                                              \
        return backward ? reinterpret_cast<const void *>(&k_backward<T, R, V, K, N>) : reinterpret_cast<const void *>(&k_forward<T, R, V, K, N>);
    A2_PICK(8, 1, 256)
    A2_PICK(8, 1, 512)
    A2_PICK(8, 2, 512)
    A2_PICK(1, 1, 256)
    A2_PICK(1, 1, 512)
    A2_PICK(1, 2, 512)
#undef A2_PICK
    return nullptr;
}
const void *pick_types(int dtype, int residual, const Plan &p, bool backward)
{
    if (dtype == A2SGD_F32) return pick<float, float>(p, backward);
    if (dtype == A2SGD_BF16) return residual == A2SGD_F32 ? pick<__nv_bfloat16, float>(p, backward) : pick<__nv_bfloat16, __nv_bfloat16>(p, backward);
    return residual == A2SGD_F32 ? pick<__half, float>(p, backward) : pick<__half, __half>(p, backward);
}
size_t smem_of(const Plan &p, bool backward)
{
    return (size_t)(backward ? 2 + kSums : 4) * p.chunks * 8 * p.threads * 4;
}

int check_shape(const a2sgd_residual *s)
{
    if (!s || !known(s->dtype) || (s->residual_dtype != A2SGD_F32 && s->residual_dtype != s->dtype) ||
        (s->param_dtype != A2SGD_F32 && s->param_dtype != s->dtype) || s->d == 0 || (s->flags & ~3u) || !std::isfinite((float)s->alpha) ||
        (s->gate && s->gate_rows == 0))
        return A2SGD_ERR_ARG;
    if (s->d > A2SGD_RESIDUAL_MAX_COLUMNS || s->rows >= (1ull << 40) || s->gate_rows >= (1ull << 62)) return A2SGD_ERR_TOO_LARGE;
    for (const void *p : {s->post_weight, s->post_bias, s->gate, s->pre_weight, s->pre_bias})
        if (!aligned(p, size_of(s->param_dtype))) return A2SGD_ERR_ALIGN;
    for (const float *p : {s->post_mean, s->post_rstd, s->pre_mean, s->pre_rstd})
        if (!aligned(p, 4)) return A2SGD_ERR_ALIGN;
    return A2SGD_OK;
}
int check_rows(const a2sgd_rows *r, const a2sgd_residual *s, int dtype, bool needed)
{
    if (!r || !r->p) return needed ? A2SGD_ERR_ARG : A2SGD_OK;
    if (s->rows > 1 && r->stride < (int64_t)s->d) return A2SGD_ERR_ARG;
    return aligned(r->p, size_of(dtype)) ? A2SGD_OK : A2SGD_ERR_ALIGN;
}
Rows rows_of(const a2sgd_rows *r) { return r && r->p ? Rows{r->p, r->stride} : Rows{nullptr, 0}; }
bool wide(const a2sgd_rows *r, const a2sgd_residual *s, int dtype)
{
    if (!r || !r->p) return true;
    return aligned(r->p, 16) && (s->rows <= 1 || r->stride * (int64_t)size_of(dtype) % 16 == 0);
}

Args common(const a2sgd_residual *s)
{
    Args a{};
    a.w1 = s->post_weight, a.b1 = s->post_bias, a.gate = s->gate, a.w2 = s->pre_weight, a.b2 = s->pre_bias;
    a.mean1 = s->post_mean, a.rstd1 = s->post_rstd, a.mean2 = s->pre_mean, a.rstd2 = s->pre_rstd;
    a.rows = (int64_t)s->rows;
    a.gate_rows = s->gate ? (int64_t)s->gate_rows : 1;
    a.d = (int)s->d;
    a.param = s->param_dtype;
    a.rms = (s->flags & A2SGD_RESIDUAL_RMS) != 0;
    a.post = (s->flags & A2SGD_RESIDUAL_POST_NORM) != 0;
    a.alpha = (float)s->alpha;
    a.eps = (float)s->eps;
    return a;
}

constexpr int kMostCtas = 1024; // that leave partial sums
// CTAs of the backward pass on a device, by the kernel that fits it most often; without a device, all that may be.
int64_t most_ctas(uint64_t rows, uint32_t d, int device)
{
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms < 1 || d == 0 || d > A2SGD_RESIDUAL_MAX_COLUMNS) return std::min<int64_t>((int64_t)rows, kMostCtas);
    int most = 1;
    for (int dtype : {A2SGD_F32, A2SGD_BF16, A2SGD_F16})
        for (int residual : {(int)A2SGD_F32, dtype})
            for (bool vec : {false, true}) {
                const Plan p = plan_of(d, vec);
                const void *fn = pick_types(dtype, residual, p, true);
                const size_t smem = smem_of(p, true);
                if (allow_smem(fn, smem) != cudaSuccess) (void)cudaGetLastError();
                most = std::max(most, resident_ctas(fn, (unsigned)p.threads, smem, device));
            }
    return std::min<int64_t>((int64_t)rows, std::min<int64_t>((int64_t)sms * most, kMostCtas));
}
// Whether a CTA may put its sums down more than once: with several gates, or where rows are many on any number of CTAs from one an SM on.
bool several_puts(uint64_t rows, uint64_t gate_rows, int device)
{
    const int sms = sm_count(device);
    return (gate_rows && gate_rows < rows) || sms < 1 || rows > (uint64_t)std::min(sms, kMostCtas) * kRun;
}
inline uint64_t sums_bytes(int64_t ctas, uint32_t d, bool several, bool gate) { return (uint64_t)ctas * ((several ? 2 : 1) * kSums + (gate ? 2 : 0)) * d * 4; }

} // namespace

extern "C" int a2sgd_residual_norm_forward(const a2sgd_residual *shape, const a2sgd_rows *x, const a2sgd_rows *y, const a2sgd_rows *z,
                                           const a2sgd_rows *u, int device, void *stream)
{
    int rc = check_shape(shape);
    if (rc != A2SGD_OK) return rc;
    if (!std::isfinite((float)shape->eps) || shape->eps < 0.0) return A2SGD_ERR_ARG;
    if (shape->rows == 0) return A2SGD_OK;
    const int t = shape->dtype, r = shape->residual_dtype;
    if ((rc = check_rows(x, shape, r, true)) != A2SGD_OK || (rc = check_rows(y, shape, t, true)) != A2SGD_OK ||
        (rc = check_rows(z, shape, r, true)) != A2SGD_OK || (rc = check_rows(u, shape, t, true)) != A2SGD_OK)
        return rc;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms < 1) return A2SGD_ERR_CUDA;
    Args a = common(shape);
    a.x = rows_of(x), a.y = rows_of(y), a.z = rows_of(z), a.u = rows_of(u);
    const Plan p = plan_of(shape->d, shape->d % 8 == 0 && wide(x, shape, r) && wide(y, shape, t) && wide(z, shape, r) && wide(u, shape, t));
    const void *fn = pick_types(t, r, p, false);
    const size_t smem = smem_of(p, false);
    A2_TRAIN_CUDA(allow_smem(fn, smem));
    const int64_t most = (int64_t)sms * resident_ctas(fn, (unsigned)p.threads, smem, device);
    a.run = (a.rows + most - 1) / most;
    void *params[] = {&a};
    A2_TRAIN_CUDA(launch(fn, dim3((unsigned)((a.rows + a.run - 1) / a.run)), (unsigned)p.threads, smem, params, static_cast<cudaStream_t>(stream)));
    return A2SGD_OK;
}

extern "C" uint64_t a2sgd_residual_norm_workspace(uint64_t rows, uint32_t d, uint64_t gate_rows, int device)
{
    return sums_bytes(most_ctas(rows, d, device), d, several_puts(rows, gate_rows, device), gate_rows != 0);
}

extern "C" int a2sgd_residual_norm_backward(const a2sgd_residual *shape, const a2sgd_rows *dz, const a2sgd_rows *du, const a2sgd_rows *y,
                                            const a2sgd_rows *z, const a2sgd_rows *dx, const a2sgd_rows *dy,
                                            const a2sgd_residual_sums *sums, void *workspace, uint64_t workspace_bytes, int device,
                                            void *stream)
{
    int rc = check_shape(shape);
    if (rc != A2SGD_OK) return rc;
    const int t = shape->dtype, r = shape->residual_dtype;
    const bool rms = shape->flags & A2SGD_RESIDUAL_RMS, post = shape->flags & A2SGD_RESIDUAL_POST_NORM, some = shape->rows != 0;
    if ((rc = check_rows(dz, shape, r, false)) != A2SGD_OK || (rc = check_rows(du, shape, t, some)) != A2SGD_OK ||
        (rc = check_rows(y, shape, t, some)) != A2SGD_OK || (rc = check_rows(z, shape, r, some)) != A2SGD_OK ||
        (rc = check_rows(dx, shape, r, false)) != A2SGD_OK || (rc = check_rows(dy, shape, t, false)) != A2SGD_OK)
        return rc;
    if (some && (!shape->pre_rstd || (!rms && !shape->pre_mean) || (post && (!shape->post_rstd || (!rms && !shape->post_mean)))))
        return A2SGD_ERR_ARG;
    const a2sgd_residual_sums none{};
    if (!sums) sums = &none;
    const void *outs[] = {sums->dpost_weight, sums->dpost_bias, sums->dgate, sums->dpre_weight, sums->dpre_bias};
    bool want = false;
    for (const void *p : outs) {
        if (!aligned(p, size_of(shape->param_dtype))) return A2SGD_ERR_ALIGN;
        want = want || p;
    }
    if ((sums->dgate && !shape->gate) || (!post && (sums->dpost_weight || sums->dpost_bias))) return A2SGD_ERR_ARG;
    if (!aligned(workspace, 256)) return A2SGD_ERR_ALIGN;
    if (want && some && (!workspace || workspace_bytes < sums_bytes(1, shape->d, false, shape->gate))) return A2SGD_ERR_ARG;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms < 1) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (!some) {
        for (const void *p : outs)
            if (p && p != sums->dgate) A2_TRAIN_CUDA(cudaMemsetAsync(const_cast<void *>(p), 0, (size_t)shape->d * size_of(shape->param_dtype), s));
        return A2SGD_OK;
    }
    Args a = common(shape);
    a.dz = rows_of(dz), a.du = rows_of(du), a.y = rows_of(y), a.z = rows_of(z), a.dx = rows_of(dx), a.dy = rows_of(dy);
    a.dw1 = sums->dpost_weight, a.db1 = sums->dpost_bias, a.dgate = sums->dgate, a.dw2 = sums->dpre_weight, a.db2 = sums->dpre_bias;
    bool vec = shape->d % 8 == 0;
    for (const a2sgd_rows *m : {dz, z, dx}) vec = vec && wide(m, shape, r);
    for (const a2sgd_rows *m : {du, y, dy}) vec = vec && wide(m, shape, t);
    const Plan p = plan_of(shape->d, vec);
    const void *fn = pick_types(t, r, p, true);
    const size_t smem = smem_of(p, true);
    A2_TRAIN_CUDA(allow_smem(fn, smem));
    const int64_t most = std::min<int64_t>((int64_t)sms * resident_ctas(fn, (unsigned)p.threads, smem, device), kMostCtas);
    a.run = (a.rows + most - 1) / most;
    a.ctas = (int)((a.rows + a.run - 1) / a.run);
    if (want) {
        const int64_t each = (int64_t)a.ctas * kSums * a.d;
        const bool several = several_puts(shape->rows, shape->gate ? shape->gate_rows : 0, device);
        if (workspace_bytes < sums_bytes(a.ctas, shape->d, several, shape->gate)) return A2SGD_ERR_ARG; // no more than a2sgd_residual_norm_workspace
        a.partials = static_cast<float *>(workspace);
        a.runs = several ? a.partials + each : nullptr;
        a.gate_partials = a.partials + (several ? 2 : 1) * each;
    }
    void *params[] = {&a};
    A2_TRAIN_CUDA(launch(fn, dim3((unsigned)a.ctas), (unsigned)p.threads, smem, params, s));
    if (want) {
        const int64_t groups = a.dgate ? (a.rows + a.gate_rows - 1) / a.gate_rows : 0;
        A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_fold), dim3((unsigned)(a.d + 31) / 32, (unsigned)std::min<int64_t>(kSums + groups, 1024)),
                             32 * kStrips, 0, params, s));
    }
    return A2SGD_OK;
}
