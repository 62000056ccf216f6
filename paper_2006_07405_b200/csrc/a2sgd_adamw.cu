// AdamW over a list of tensors, with its state in 32 or in 8 bits, and the clip factor from the
// global norm of the gradients.  The formulas and the formats are documented in include/a2sgd.h.
//
// 28 bytes an element with fp32 gradients and 32-bit states, which HBM bounds (B200, 1.56 G elements with their norm 7352 us, 6.8 TB/s);
// 16 with 8-bit ones (14 with 16-bit gradients), which instruction issue bounds (79 % of the slots, 3.9 TB/s over 30 M).  One CTA takes a tile of 8 blocks of 256 elements of one tensor,
// one warp a block, one lane 8 consecutive elements, all loads of a lane in flight together; the
// hardware's CTA scheduler evens out SMs that stream at different speeds.  A table entry of 32
// bytes a tile holds the tile's addresses, so that one dependent read stands before the loads.
//
// Every operation is a single IEEE rounding in the order the header gives (no contraction to a
// fused multiply-add), so that a step is defined to the bit, and with it the 8-bit codes.
#include "a2sgd_adamw_arith.cuh"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

using namespace a2sgd_train;

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kStateBlock = A2SGD_ADAMW_BLOCK; // one warp, 8 elements a lane
constexpr uint32_t kTile = kThreads * 8;            // 8 blocks
static_assert(kStateBlock == 256, "a block of the 8-bit states is one warp of 8 elements a lane");
constexpr int kNormCtas = 2048; // partial sums of the norm at most
// Blocks whose largest state is below 2^-100 are held as zeros: the gain 127^2 / scale stays finite.
constexpr float kSmallestScale = 7.888609052210118e-31f;
constexpr float kPerM = 1.0f / 16129.0f, kPerV = 1.0f / 65025.0f; // rounded once, then factors

struct __align__(32) Tile {
    float *w;
    const void *grad;
    void *w16;
    uint32_t block;  // first block of the state
    uint16_t count;  // elements, 1..kTile
    uint16_t vector; // every address allows the widest accesses
};

struct StepArgs {
    const Tile *tiles;
    float *m, *v;                      // 32-bit states
    int8_t *mq;                        // 8-bit states
    uint8_t *vq;
    float *m_scale, *v_scale;
    const float *grad_scale;           // nullptr: 1
    float beta1, one_minus_beta1, beta2, one_minus_beta2, decay, rate, root, eps;
    uint32_t dither;
    uint32_t least_plain; // of v, for plain_range
};

// Two 12-bit numbers from the element's place in the state and the step: a counter (Weyl sequence,
// golden-ratio increment) through two multiply-xorshift rounds.
__device__ __forceinline__ uint32_t dither_bits(uint32_t place, uint32_t step_key)
{
    uint32_t h = place * 0x9E3779B1u + step_key;
    h ^= h >> 16;
    h *= 0x7FEB3525u;
    h ^= h >> 15;
    h *= 0x94D049BBu;
    h ^= h >> 16;
    return h;
}

// Bytes become floats and floats bytes without the conversion unit, which issues a quarter as often as the adder:
// a byte is the low mantissa of 2^23.

// 12 bits of the dither as 1 + u: bits 31..20 for m's code, bits 19..8 for v's.
__device__ __forceinline__ uint32_t dither_m(uint32_t h) { return 0x3F800000u | (h >> 9 & 0x007FF800u); }
__device__ __forceinline__ uint32_t dither_v(uint32_t h) { return 0x3F800000u | (h << 3 & 0x007FF800u); }

// Codes to bytes: a whole number plus 1.5 * 2^23 has its two's complement in the low byte.
__device__ __forceinline__ uint32_t bytes4(float a, float b, float c, float d)
{
    float x, y, z, w;
    unpair(add2(pair(a, b), pair(12582912.0f)), x, y);
    unpair(add2(pair(c, d), pair(12582912.0f)), z, w);
    const uint32_t lo = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(z), __float_as_uint(w), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
}
// Bytes to the values they stand for, two at a time: m = q |q| cm from two's complement with the top bit flipped
// (q + 128), and sqrt(v) = q^2 cr.
__device__ __forceinline__ f32x2 m_of(uint32_t flipped, int byte, f32x2 cm)
{
    const f32x2 q = add2(pair(__uint_as_float(__byte_perm(flipped, 0x4B000000u, 0x7540u | byte)),
                              __uint_as_float(__byte_perm(flipped, 0x4B000000u, 0x7541u + byte))), pair(-8388736.0f));
    float a, b;
    unpair(q, a, b);
    return mul2(mul2(q, pair(fabsf(a), fabsf(b))), cm);
}
__device__ __forceinline__ f32x2 root_of(uint32_t word, int byte, f32x2 cr)
{
    const f32x2 q = add2(pair(__uint_as_float(__byte_perm(word, 0x4B000000u, 0x7540u | byte)),
                              __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7541u + byte))), pair(-8388608.0f));
    return mul2(mul2(q, q), cr);
}

struct Gain {
    float scale, gain;
};
__device__ __forceinline__ Gain gain_of(uint32_t largest_bits, float top_squared)
{
    Gain r;
    r.scale = __uint_as_float(largest_bits);
    if (r.scale < kSmallestScale) r.scale = 0.0f; // false for NaN, which stays and shows
    r.gain = r.scale == 0.0f ? 0.0f : __fmul_rn(__frcp_rn(r.scale), top_squared);
    return r;
}

// GT: gradient type.  CT: type of the 16-bit copy of the weights, float when there is none.
// EIGHT: 8-bit states.
template <typename GT, typename CT, bool EIGHT>
__global__ void __launch_bounds__(kThreads, 5) k_adamw(const __grid_constant__ StepArgs a)
{
    constexpr bool kCopy = sizeof(CT) == 2;
    const Tile *entry = a.tiles + blockIdx.x; // the plan's own table, written before any step
    const uint4 e0 = __ldg(reinterpret_cast<const uint4 *>(entry));
    const uint4 e1 = __ldg(reinterpret_cast<const uint4 *>(entry) + 1);
    wait_prior_grid();
    release_next_grid();
    Tile t;
    *reinterpret_cast<uint4 *>(&t) = e0;
    *(reinterpret_cast<uint4 *>(&t) + 1) = e1;

    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t first = warp * kStateBlock; // of this warp's block inside the tile
    if (first >= t.count) return;
    const float scale = a.grad_scale ? __ldcg(a.grad_scale) : 1.0f;
    if (!isfinite(scale)) return; // a norm that was not finite: the step changes nothing
    const uint64_t block = (uint64_t)t.block + warp;
    const uint32_t live = min((uint32_t)t.count - first, kStateBlock);
    const bool vector = t.vector && live == kStateBlock;
    const uint32_t base = lane * 8; // a lane's 8 consecutive places inside the block

    __align__(16) float w[8], g[8];
    float m[8], v[8];
    float *wp = t.w + first;
    const GT *gp = static_cast<const GT *>(t.grad) + first;
    const uint64_t at = block * kStateBlock + base;

    uint2 mw = make_uint2(0, 0), vw = make_uint2(0, 0);
    float ms = 0.f, vs = 0.f;
    if constexpr (EIGHT) {
        ms = __ldcg(a.m_scale + block);
        vs = __ldcg(a.v_scale + block);
        mw = *reinterpret_cast<const uint2 *>(a.mq + at);
        vw = *reinterpret_cast<const uint2 *>(a.vq + at);
    } else {
        ld256(a.m + at, m);
        ld256(a.v + at, v);
    }
    // Tensors that wide accesses cannot read, and their last blocks, go through shared memory: every 32nd element of
    // the block a lane in memory, 8 consecutive ones in the arithmetic.
    __shared__ __align__(16) float turn[kThreads / 32][2][kStateBlock];
    float(*mine)[kStateBlock] = turn[warp];
    if (vector) {
        Raw8<GT> graw;
        ld256(wp + base, w);
        graw.load(gp + base);
        graw.unpack(g);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t p = lane + i * 32;
            w[i] = p < live ? wp[p] : 0.0f;
            g[i] = p < live ? to_f32(gp[p]) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            mine[0][lane + i * 32] = w[i];
            mine[1][lane + i * 32] = g[i];
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            *reinterpret_cast<float4 *>(w + i) = *reinterpret_cast<const float4 *>(&mine[0][base + i]);
            *reinterpret_cast<float4 *>(g + i) = *reinterpret_cast<const float4 *>(&mine[1][base + i]);
        }
    }
    // m, v and sqrt(v) after the step
    f32x2 m2[4], v2[4], r2[4];
    if constexpr (EIGHT) {
        const f32x2 cm = pair(__fmul_rn(ms, kPerM)), cr = pair(__fmul_rn(vs, kPerV));
        mw.x ^= 0x80808080u, mw.y ^= 0x80808080u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m2[i] = m_of(i < 2 ? mw.x : mw.y, 2 * (i & 1), cm);
            const f32x2 root = root_of(i < 2 ? vw.x : vw.y, 2 * (i & 1), cr);
            v2[i] = mul2(root, root);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m2[i] = pair(m[2 * i], m[2 * i + 1]);
            v2[i] = pair(v[2 * i], v[2 * i + 1]);
        }
    }
    uint32_t big_m = 0, big_v = 0, least_v = 0xffffffffu; // bit patterns order like the values, NaN above infinity
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 gi = mul2(pair(g[2 * i], g[2 * i + 1]), pair(scale));
        m2[i] = add2_of_products(mul2(m2[i], pair(a.beta1)), mul2(gi, pair(a.one_minus_beta1)));
        v2[i] = add2_of_products(mul2(v2[i], pair(a.beta2)), mul2(mul2(gi, gi), pair(a.one_minus_beta2)));
        unpair(m2[i], m[2 * i], m[2 * i + 1]);
        unpair(v2[i], v[2 * i], v[2 * i + 1]);
#pragma unroll
        for (int k = 2 * i; k < 2 * i + 2; ++k) {
            big_m = max(big_m, __float_as_uint(m[k]) & 0x7fffffffu);
            big_v = max(big_v, __float_as_uint(v[k]));
            least_v = min(least_v, __float_as_uint(v[k]));
        }
    }
    if (plain_range(least_v, a.least_plain, big_v, big_m)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r2[i] = root2(v2[i]);
            const f32x2 q = quotient2(m2[i], add2_of_products(mul2(r2[i], pair(a.root)), pair(a.eps)));
            unpair(add2_of_products(mul2(pair(w[2 * i], w[2 * i + 1]), pair(a.decay)), mul2(q, pair(-a.rate))), w[2 * i], w[2 * i + 1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float r[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int e = 2 * i + k;
                r[k] = __fsqrt_rn(v[e]);
                const float q = __fdiv_rn(m[e], __fadd_rn(__fmul_rn(r[k], a.root), a.eps));
                w[e] = __fsub_rn(__fmul_rn(w[e], a.decay), __fmul_rn(q, a.rate));
            }
            r2[i] = pair(r[0], r[1]);
        }
    }

    if (vector) {
        st256(wp + base, w);
        if constexpr (kCopy) store8(static_cast<CT *>(t.w16) + first + base, w);
    } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; i += 4) *reinterpret_cast<float4 *>(&mine[0][base + i]) = *reinterpret_cast<const float4 *>(w + i);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t p = lane + i * 32;
            if (p < live) {
                const float x = mine[0][p];
                wp[p] = x;
                if constexpr (kCopy) static_cast<CT *>(t.w16)[first + p] = from_f32<CT>(x);
            }
        }
    }
    if constexpr (!EIGHT) {
        st256(a.m + at, m);
        st256(a.v + at, v);
    } else {
        // the largest root is the root of the largest v: a correctly rounded root is monotonic
        const float top_v = __uint_as_float(__reduce_max_sync(0xffffffffu, big_v));
        const Gain gr = gain_of(__float_as_uint(__fsqrt_rn(top_v)), 65025.0f);
        const Gain gm = gain_of(__reduce_max_sync(0xffffffffu, big_m), 16129.0f);
        float qm[8], qr[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t h0 = dither_bits((uint32_t)at + 2 * i, a.dither);
            const uint32_t h1 = dither_bits((uint32_t)at + 2 * i + 1, a.dither);
            const float m0 = m[2 * i], m1 = m[2 * i + 1];
            encode2(mul2(pair(fabsf(m0), fabsf(m1)), pair(gm.gain)), dither_m(h0), dither_m(h1), 127.0f, 0.0f, qm[2 * i], qm[2 * i + 1]);
            encode2(mul2(r2[i], pair(gr.gain)), dither_v(h0), dither_v(h1), 255.0f, 2.0f, qr[2 * i], qr[2 * i + 1]);
            qm[2 * i] = copysignf(qm[2 * i], m0);
            qm[2 * i + 1] = copysignf(qm[2 * i + 1], m1);
        }
        const uint2 mo = make_uint2(bytes4(qm[0], qm[1], qm[2], qm[3]), bytes4(qm[4], qm[5], qm[6], qm[7]));
        const uint2 vo = make_uint2(bytes4(qr[0], qr[1], qr[2], qr[3]), bytes4(qr[4], qr[5], qr[6], qr[7]));
        *reinterpret_cast<uint2 *>(a.mq + at) = mo;
        *reinterpret_cast<uint2 *>(a.vq + at) = vo;
        if (lane == 0) {
            a.m_scale[block] = gm.scale;
            a.v_scale[block] = gr.scale;
        }
    }
}

// ------------------------------------------------------------------ global norm of the gradients
// Squares are added in fp64 (an fp32 square overflows from 2e19 up and vanishes below 1e-23), each
// CTA over its tiles, the CTA that draws the last ticket over the CTAs in order: no floating-point
// atomics, the same bits every time.
template <typename GT>
__global__ void __launch_bounds__(kThreads) k_grad_norm(const Tile *tiles, uint64_t n_tiles, double *partials,
                                                        unsigned int *ticket, float max_norm, float *out)
{
    wait_prior_grid();
    release_next_grid();
    double sum = 0.0;
    for (uint64_t k = blockIdx.x; k < n_tiles; k += gridDim.x) {
        const GT *gp = static_cast<const GT *>(tiles[k].grad);
        const uint32_t count = tiles[k].count;
        if (tiles[k].vector && count == kTile) {
            Raw8<GT> raw;
            float g[8];
            raw.load(gp + threadIdx.x * 8);
            raw.unpack(g);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fma((double)g[i], (double)g[i], sum);
        } else {
            for (uint32_t p = threadIdx.x; p < count; p += kThreads) {
                const double g = to_f32(gp[p]);
                sum = fma(g, g, sum);
            }
        }
    }
    __shared__ double sh[kThreads / 32];
    __shared__ bool last;
    const auto block_sum = [&](double x) {
#pragma unroll
        for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
        __syncthreads();
        x = 0.0;
        for (int i = 0; i < kThreads / 32; ++i) x += sh[i];
        __syncthreads();
        return x;
    };
    sum = block_sum(sum);
    if (threadIdx.x == 0) {
        partials[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kThreads) sum += __ldcg(partials + i);
    sum = block_sum(sum);
    if (threadIdx.x == 0) {
        *ticket = 0; // for the next call on this plan
        const double norm = sqrt(sum);
        out[0] = (float)norm;
        // a factor that is not finite makes a step skip itself
        out[1] = isfinite((float)norm) ? (float)((double)max_norm / fmax(norm, (double)max_norm)) : nanf("");
    }
}

// ------------------------------------------------------------------ 8-bit state <-> 32-bit values
__global__ void __launch_bounds__(kThreads) k_read_state(const int8_t *mq, const uint8_t *vq, const float *m_scale,
                                                         const float *v_scale, uint64_t blocks, float *m_out, float *v_out)
{
    wait_prior_grid();
    release_next_grid();
    const uint64_t block = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (block >= blocks) return;
    const uint64_t at = block * kStateBlock + (threadIdx.x & 31) * 8;
    const uint2 mw = *reinterpret_cast<const uint2 *>(mq + at), vw = *reinterpret_cast<const uint2 *>(vq + at);
    const f32x2 cm = pair(__fmul_rn(m_scale[block], kPerM)), cr = pair(__fmul_rn(v_scale[block], kPerV));
    const uint32_t flipped[2] = {mw.x ^ 0x80808080u, mw.y ^ 0x80808080u}, word[2] = {vw.x, vw.y};
    float m[8], v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unpair(m_of(flipped[i / 2], 2 * (i & 1), cm), m[2 * i], m[2 * i + 1]);
        const f32x2 root = root_of(word[i / 2], 2 * (i & 1), cr);
        unpair(mul2(root, root), v[2 * i], v[2 * i + 1]);
    }
    if (m_out) st256(m_out + at, m);
    if (v_out) st256(v_out + at, v);
}

__global__ void __launch_bounds__(kThreads) k_write_state(const float *m_in, const float *v_in, uint64_t blocks,
                                                          int8_t *mq, uint8_t *vq, float *m_scale, float *v_scale)
{
    wait_prior_grid();
    release_next_grid();
    const uint64_t block = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (block >= blocks) return;
    const uint64_t at = block * kStateBlock + (threadIdx.x & 31) * 8;
    float m[8], r[8];
    ld256(m_in + at, m);
    ld256(v_in + at, r);
    uint32_t big_m = 0, big_r = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        r[i] = __fsqrt_rn(r[i]);
        big_m = max(big_m, __float_as_uint(m[i]) & 0x7fffffffu);
        big_r = max(big_r, __float_as_uint(r[i]) & 0x7fffffffu);
    }
    const Gain gm = gain_of(__reduce_max_sync(0xffffffffu, big_m), 16129.0f);
    const Gain gr = gain_of(__reduce_max_sync(0xffffffffu, big_r), 65025.0f);
    constexpr uint32_t kHalf = 0x3FC00000u; // u = 1/2: to the nearer square
    float qm[8], qr[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        encode2(mul2(pair(fabsf(m[i]), fabsf(m[i + 1])), pair(gm.gain)), kHalf, kHalf, 127.0f, 0.0f, qm[i], qm[i + 1]);
        encode2(mul2(pair(r[i], r[i + 1]), pair(gr.gain)), kHalf, kHalf, 255.0f, 2.0f, qr[i], qr[i + 1]);
        qm[i] = copysignf(qm[i], m[i]);
        qm[i + 1] = copysignf(qm[i + 1], m[i + 1]);
    }
    *reinterpret_cast<uint2 *>(mq + at) = make_uint2(bytes4(qm[0], qm[1], qm[2], qm[3]), bytes4(qm[4], qm[5], qm[6], qm[7]));
    *reinterpret_cast<uint2 *>(vq + at) = make_uint2(bytes4(qr[0], qr[1], qr[2], qr[3]), bytes4(qr[4], qr[5], qr[6], qr[7]));
    if ((threadIdx.x & 31) == 0) {
        m_scale[block] = gm.scale;
        v_scale[block] = gr.scale;
    }
}

template <typename GT, bool EIGHT>
const void *pick_copy(int copy)
{
    switch (copy) {
    case A2SGD_BF16: return reinterpret_cast<const void *>(&k_adamw<GT, __nv_bfloat16, EIGHT>);
    case A2SGD_F16: return reinterpret_cast<const void *>(&k_adamw<GT, __half, EIGHT>);
    default: return reinterpret_cast<const void *>(&k_adamw<GT, float, EIGHT>);
    }
}
template <bool EIGHT>
const void *pick_step(int grad, int copy)
{
    switch (grad) {
    case A2SGD_BF16: return pick_copy<__nv_bfloat16, EIGHT>(copy);
    case A2SGD_F16: return pick_copy<__half, EIGHT>(copy);
    default: return pick_copy<float, EIGHT>(copy);
    }
}

} // namespace

struct a2sgd_adamw {
    int device = 0;
    bool eight = false;
    int grad_dtype = A2SGD_F32;
    int w16_dtype = A2SGD_F32; // A2SGD_F32: no copy
    uint64_t n_tiles = 0, blocks = 0;
    void *m = nullptr, *v = nullptr; // the caller's
    float *m_scale = nullptr, *v_scale = nullptr;
    // owned
    Tile *tiles = nullptr;
    double *partials = nullptr;
    unsigned int *ticket = nullptr;
};

extern "C" uint64_t a2sgd_adamw_state_elements(uint32_t S, const uint64_t *numel)
{
    if (!numel) return 0;
    uint64_t n = 0;
    for (uint32_t s = 0; s < S; ++s) n += (numel[s] + kStateBlock - 1) / kStateBlock * kStateBlock;
    return n;
}

extern "C" int a2sgd_adamw_create(a2sgd_adamw **out, uint32_t S, const uint64_t *numel, float *const *w,
                                  const void *const *grad, int grad_dtype, void *const *w16, int w16_dtype,
                                  int state_bits, void *m, void *v, float *m_scale, float *v_scale, int device)
{
    if (!out) return A2SGD_ERR_ARG;
    *out = nullptr;
    if (S == 0 || !numel || !w || !grad || !m || !v || !known(grad_dtype)) return A2SGD_ERR_ARG;
    if (state_bits != 8 && state_bits != 32) return A2SGD_ERR_ARG;
    if (state_bits == 8 ? (!m_scale || !v_scale) : (m_scale || v_scale)) return A2SGD_ERR_ARG;
    if (w16 && w16_dtype != A2SGD_BF16 && w16_dtype != A2SGD_F16) return A2SGD_ERR_ARG;
    if (!aligned(m, 32) || !aligned(v, 32) || !aligned(m_scale, 4) || !aligned(v_scale, 4)) return A2SGD_ERR_ALIGN;
    uint64_t total = 0;
    for (uint32_t s = 0; s < S; ++s) {
        if (numel[s] == 0 || numel[s] >= (1ull << 40) || !w[s] || !grad[s] || (w16 && !w16[s])) return A2SGD_ERR_ARG;
        if (!aligned(w[s], 4) || !aligned(grad[s], size_of(grad_dtype)) || (w16 && !aligned(w16[s], 2))) return A2SGD_ERR_ALIGN;
        total += (numel[s] + kStateBlock - 1) / kStateBlock;
    }
    if (total >= (1ull << 32)) return A2SGD_ERR_TOO_LARGE; // blocks are counted in 32 bits: 2^40 elements
    DeviceGuard guard(device);
    if (!guard.ok) return A2SGD_ERR_CUDA;

    std::vector<Tile> tiles;
    a2sgd_adamw *p = nullptr;
    try {
        uint64_t block = 0;
        for (uint32_t s = 0; s < S; ++s) {
            const bool vec = aligned(w[s], 32) && aligned(grad[s], 16) && (!w16 || aligned(w16[s], 16));
            for (uint64_t off = 0; off < numel[s]; off += kTile) {
                Tile t;
                t.w = w[s] + off;
                t.grad = static_cast<const char *>(grad[s]) + off * size_of(grad_dtype);
                t.w16 = w16 ? static_cast<char *>(w16[s]) + off * 2 : nullptr;
                t.block = (uint32_t)(block + off / kStateBlock);
                t.count = (uint16_t)std::min<uint64_t>(kTile, numel[s] - off);
                t.vector = vec;
                tiles.push_back(t);
            }
            block += (numel[s] + kStateBlock - 1) / kStateBlock;
        }
        p = new a2sgd_adamw();
    } catch (const std::bad_alloc &) {
        return A2SGD_ERR_NOMEM;
    }
    if (tiles.size() > 0x7fffffffull) {
        delete p;
        return A2SGD_ERR_TOO_LARGE;
    }
    p->device = device;
    p->eight = state_bits == 8;
    p->grad_dtype = grad_dtype;
    p->w16_dtype = w16 ? w16_dtype : A2SGD_F32;
    p->n_tiles = tiles.size();
    p->blocks = total;
    p->m = m;
    p->v = v;
    p->m_scale = m_scale;
    p->v_scale = v_scale;
    bool ok = cudaMalloc(&p->tiles, sizeof(Tile) * tiles.size()) == cudaSuccess;
    ok = ok && cudaMalloc(&p->partials, sizeof(double) * kNormCtas) == cudaSuccess;
    ok = ok && cudaMalloc(&p->ticket, sizeof(unsigned int)) == cudaSuccess;
    ok = ok && cudaMemset(p->ticket, 0, sizeof(unsigned int)) == cudaSuccess;
    ok = ok && cudaMemcpy(p->tiles, tiles.data(), sizeof(Tile) * tiles.size(), cudaMemcpyHostToDevice) == cudaSuccess;
    ok = ok && cudaStreamSynchronize(nullptr) == cudaSuccess; // the table is there before a step on any stream
    if (!ok) {
        (void)cudaGetLastError();
        a2sgd_adamw_destroy(p);
        return A2SGD_ERR_NOMEM;
    }
    *out = p;
    return A2SGD_OK;
}

extern "C" int a2sgd_adamw_destroy(a2sgd_adamw *p)
{
    if (!p) return A2SGD_OK;
    DeviceGuard guard(p->device);
    cudaFree(p->tiles);
    cudaFree(p->partials);
    cudaFree(p->ticket);
    (void)cudaGetLastError();
    delete p;
    return A2SGD_OK;
}

extern "C" int a2sgd_adamw_grad_norm(a2sgd_adamw *p, float max_norm, float *norm_and_scale, void *stream)
{
    if (!p || !norm_and_scale || !(max_norm > 0.0f) || !std::isfinite(max_norm)) return A2SGD_ERR_ARG;
    if (!aligned(norm_and_scale, 4)) return A2SGD_ERR_ALIGN;
    DeviceGuard guard(p->device);
    const int sms = guard.ok ? sm_count(p->device) : 0;
    if (sms == 0) return A2SGD_ERR_CUDA;
    const void *fn = p->grad_dtype == A2SGD_BF16  ? reinterpret_cast<const void *>(&k_grad_norm<__nv_bfloat16>)
                     : p->grad_dtype == A2SGD_F16 ? reinterpret_cast<const void *>(&k_grad_norm<__half>)
                                                  : reinterpret_cast<const void *>(&k_grad_norm<float>);
    const unsigned grid = (unsigned)std::min<uint64_t>(p->n_tiles, std::min(kNormCtas, sms * 8));
    void *params[] = {&p->tiles, &p->n_tiles, &p->partials, &p->ticket, &max_norm, &norm_and_scale};
    A2_TRAIN_CUDA(launch(fn, dim3(grid), kThreads, 0, params, static_cast<cudaStream_t>(stream)));
    return A2SGD_OK;
}

extern "C" int a2sgd_adamw_step(a2sgd_adamw *p, double lr, double beta1, double beta2, double eps, double weight_decay,
                                uint64_t step, const float *grad_scale, void *stream)
{
    if (!p || step == 0) return A2SGD_ERR_ARG;
    if (!std::isfinite(lr) || !(lr >= 0.0) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
        !(eps <= FLT_MAX) || !((float)eps > 0.0f) || !std::isfinite(weight_decay) || !(weight_decay >= 0.0))
        return A2SGD_ERR_ARG;
    const double decay = 1.0 - lr * weight_decay, rate = lr / (1.0 - std::pow(beta1, (double)step));
    if (!(std::fabs(decay) <= FLT_MAX) || !(rate <= FLT_MAX)) return A2SGD_ERR_ARG; // not finite as fp32
    if (!aligned(grad_scale, 4)) return A2SGD_ERR_ALIGN;
    DeviceGuard guard(p->device);
    if (!guard.ok) return A2SGD_ERR_CUDA;
    StepArgs a{};
    a.tiles = p->tiles;
    if (p->eight) {
        a.mq = static_cast<int8_t *>(p->m);
        a.vq = static_cast<uint8_t *>(p->v);
        a.m_scale = p->m_scale;
        a.v_scale = p->v_scale;
    } else {
        a.m = static_cast<float *>(p->m);
        a.v = static_cast<float *>(p->v);
    }
    a.grad_scale = grad_scale;
    a.beta1 = (float)beta1;
    a.one_minus_beta1 = (float)(1.0 - beta1);
    a.beta2 = (float)beta2;
    a.one_minus_beta2 = (float)(1.0 - beta2);
    a.decay = (float)decay;
    a.rate = (float)rate;
    a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    a.eps = (float)eps;
    a.dither = (uint32_t)step * 0x85A308D3u + 0x243F6A89u;
    a.least_plain = eps <= kMostPlainEps ? kLeastPlain : 0xffffffffu; // no v passes: the library path
    const void *fn = p->eight ? pick_step<true>(p->grad_dtype, p->w16_dtype) : pick_step<false>(p->grad_dtype, p->w16_dtype);
    void *params[] = {&a};
    A2_TRAIN_CUDA(launch(fn, dim3((unsigned)p->n_tiles), kThreads, 0, params, static_cast<cudaStream_t>(stream)));
    return A2SGD_OK;
}

extern "C" int a2sgd_adamw_read_state(a2sgd_adamw *p, float *m_out, float *v_out, void *stream)
{
    if (!p || (!m_out && !v_out)) return A2SGD_ERR_ARG;
    if (!aligned(m_out, 32) || !aligned(v_out, 32)) return A2SGD_ERR_ALIGN;
    DeviceGuard guard(p->device);
    if (!guard.ok) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (!p->eight) {
        const size_t bytes = p->blocks * kStateBlock * sizeof(float);
        if (m_out) A2_TRAIN_CUDA(cudaMemcpyAsync(m_out, p->m, bytes, cudaMemcpyDeviceToDevice, s));
        if (v_out) A2_TRAIN_CUDA(cudaMemcpyAsync(v_out, p->v, bytes, cudaMemcpyDeviceToDevice, s));
        return A2SGD_OK;
    }
    const unsigned grid = (unsigned)((p->blocks + kThreads / 32 - 1) / (kThreads / 32));
    void *params[] = {&p->m, &p->v, &p->m_scale, &p->v_scale, &p->blocks, &m_out, &v_out};
    A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_read_state), dim3(grid), kThreads, 0, params, s));
    return A2SGD_OK;
}

extern "C" int a2sgd_adamw_write_state(a2sgd_adamw *p, const float *m_in, const float *v_in, void *stream)
{
    if (!p || !m_in || !v_in) return A2SGD_ERR_ARG;
    if (!aligned(m_in, 32) || !aligned(v_in, 32)) return A2SGD_ERR_ALIGN;
    DeviceGuard guard(p->device);
    if (!guard.ok) return A2SGD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (!p->eight) {
        const size_t bytes = p->blocks * kStateBlock * sizeof(float);
        A2_TRAIN_CUDA(cudaMemcpyAsync(p->m, m_in, bytes, cudaMemcpyDeviceToDevice, s));
        A2_TRAIN_CUDA(cudaMemcpyAsync(p->v, v_in, bytes, cudaMemcpyDeviceToDevice, s));
        return A2SGD_OK;
    }
    const unsigned grid = (unsigned)((p->blocks + kThreads / 32 - 1) / (kThreads / 32));
    void *params[] = {&m_in, &v_in, &p->blocks, &p->m, &p->v, &p->m_scale, &p->v_scale};
    A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_write_state), dim3(grid), kThreads, 0, params, s));
    return A2SGD_OK;
}
