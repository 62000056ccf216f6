// Rotary positions with several axes: pairs of a head's elements turned by angles that grow with the token's places.
//
//   (u, v) <- (u cos - v sin, u sin + v cos),   angle = positions[axis of the pair][token] * omega_pair
//
// Bound by memory: every element of q and k is read and written once.  A thread takes eight pairs of one token (one where addresses, strides or
// pairs do not allow 128-bit accesses), works out their sines and cosines once, and walks the heads with them; few tokens share their heads out
// among threads, until the SMs are full.  B200, 65531 tokens, 32 and 8 heads of 128: 215 us (6.2 TB/s, 95 % of a copy's; fp32 464); 4097 tokens, 13 and 13 heads
// of 80 in fp32, odd rows: 20.5 us (3.3 TB/s: a single element an access); 16 tokens: 2.8 us on the device, 9.7 a call.
//
// An angle is a 64-bit fraction of a turn, the product of the position and the frequency in turns modulo 2^64: whole turns fall
// off by themselves, so that a position of 2^30 is turned as exactly as one of 1.  (In fp32 the product alone would be off by
// position * 2^-24 radians.)  The upper bits say the quarter of a turn; what is left, at most an eighth either way, is rounded
// to fp32, at most 2^-28 of a turn off, and goes through sincospif, whose error is two units in the last place.
#include "a2sgd_train.cuh"

#include <algorithm>
#include <cmath>
#include <cstdint>

using namespace a2sgd_train;

namespace {

constexpr int kMostPairs = A2SGD_ROTARY_MAX_HEAD_DIM / 2;
constexpr int kThreads = 256;

struct Side {
    const void *in;
    void *out;
    int64_t in_row, in_head, out_row, out_head;
    int heads;
};
struct Args {
    Side q, k;
    const int32_t *positions;
    uint64_t turn[kMostPairs]; // of each pair: turns a step, as a fraction of 2^64
    uint8_t axis[kMostPairs];
    int64_t tokens;
    int pairs, d, interleaved, inverse;
    int units, tail_units; // of a head: groups of pairs, and of elements past them
    int split, heads_each; // threads that share a token's heads, and heads of each
};

// VEC consecutive elements as they are in memory
template <typename T, int VEC>
struct Piece {
    Raw8<T> raw;
    __device__ __forceinline__ void load(const T *p) { raw.load(p); }
    __device__ __forceinline__ void unpack(float (&f)[8]) const { raw.unpack(f); }
    __device__ static __forceinline__ void store(T *p, const float (&f)[8]) { store8(p, f); }
};
template <typename T>
struct Piece<T, 1> {
    T raw;
    __device__ __forceinline__ void load(const T *p) { raw = *p; }
    __device__ __forceinline__ void unpack(float (&f)[1]) const { f[0] = to_f32(raw); }
    __device__ static __forceinline__ void store(T *p, const float (&f)[1]) { *p = from_f32<T>(f[0]); }
};

template <typename T, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) k_rotary(const __grid_constant__ Args a)
{
    wait_prior_grid();
    release_next_grid();
    const int per_token = (a.units + a.tail_units) * a.split;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, token = i / per_token;
    if (token >= a.tokens) return;
    const int rest = (int)(i - token * per_token), part = rest / (a.units + a.tail_units), unit = rest - part * (a.units + a.tail_units);
    const int first = part * a.heads_each, last = min(first + a.heads_each, a.q.heads + a.k.heads);
    const bool turns = unit < a.units;
    float c[VEC], s[VEC];
    int at0, at1; // the elements of the unit: interleaved, 2 VEC consecutive ones; a tail, VEC
    if (turns) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int pair = unit * VEC + e;
            const uint64_t angle = (uint64_t)(int64_t)a.positions[a.axis[pair] * a.tokens + token] * a.turn[pair];
            const uint32_t quarter = (uint32_t)((angle + (1ull << 61)) >> 62);
            const int32_t left = (int32_t)((angle - ((uint64_t)quarter << 62)) >> 32); // of a turn, times 2^32
            float sn, cs;
            sincospif((float)left * 0x1p-31f, &sn, &cs);
            if (quarter & 1) {
                const float t = sn;
                sn = cs;
                cs = -t;
            }
            if (quarter & 2) sn = -sn, cs = -cs;
            c[e] = cs;
            s[e] = a.inverse ? -sn : sn;
        }
        at0 = INTERLEAVED ? 2 * unit * VEC : unit * VEC;
        at1 = INTERLEAVED ? at0 + VEC : at0 + a.pairs;
    } else {
        at0 = at1 = 2 * a.pairs + (unit - a.units) * VEC;
    }
    const auto source = [&](int h) {
        const Side &x = h < a.q.heads ? a.q : a.k;
        return static_cast<const T *>(x.in) + token * x.in_row + (int64_t)(h < a.q.heads ? h : h - a.q.heads) * x.in_head;
    };
    const auto target = [&](int h) {
        const Side &x = h < a.q.heads ? a.q : a.k;
        return static_cast<T *>(x.out) + token * x.out_row + (int64_t)(h < a.q.heads ? h : h - a.q.heads) * x.out_head;
    };
    constexpr int kAhead = VEC == 8 ? 4 : 8; // heads whose reads come before their writes
    for (int h0 = first; h0 < last; h0 += kAhead) {
        Piece<T, VEC> u[kAhead], v[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (h0 + e >= last) break;
            const T *p = source(h0 + e);
            u[e].load(p + at0);
            if (turns) v[e].load(p + at1);
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (h0 + e >= last) break;
            T *p = target(h0 + e);
            float m[VEC], n[VEC], x[VEC], y[VEC];
            u[e].unpack(m);
            if (turns) {
                v[e].unpack(n);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    if constexpr (INTERLEAVED && VEC > 1) {
                        // pair j of the unit is elements 2 j and 2 j + 1 of u and v one after another
                        const float f = j < VEC / 2 ? m[(2 * j) % VEC] : n[(2 * j) % VEC], g = j < VEC / 2 ? m[(2 * j + 1) % VEC] : n[(2 * j + 1) % VEC];
                        (j < VEC / 2 ? x : y)[(2 * j) % VEC] = f * c[j] - g * s[j];
                        (j < VEC / 2 ? x : y)[(2 * j + 1) % VEC] = f * s[j] + g * c[j];
                    } else {
                        x[j] = m[j] * c[j] - n[j] * s[j];
                        y[j] = m[j] * s[j] + n[j] * c[j];
                    }
                }
                Piece<T, VEC>::store(p + at0, x);
                Piece<T, VEC>::store(p + at1, y);
            } else {
                Piece<T, VEC>::store(p + at0, m);
            }
        }
    }
}

// ------------------------------------------------------------------ host
int check(const a2sgd_heads *h, uint32_t heads, uint64_t tokens, int dtype, bool written)
{
    if (!h || !h->p) return A2SGD_ERR_ARG;
    if (h->row_stride < 0 || h->head_stride < 0) return A2SGD_ERR_ARG;
    if (written && ((h->row_stride == 0 && tokens > 1) || (h->head_stride == 0 && heads > 1))) return A2SGD_ERR_ARG;
    return aligned(h->p, size_of(dtype)) ? A2SGD_OK : A2SGD_ERR_ALIGN;
}
bool wide(const a2sgd_heads *h, int dtype)
{
    const int64_t whole = 16 / (int64_t)size_of(dtype);
    return aligned(h->p, 16) && h->row_stride % whole == 0 && h->head_stride % whole == 0;
}

template <typename T>
const void *pick(bool vec, bool interleaved)
{
    if (vec) return interleaved ? reinterpret_cast<const void *>(&k_rotary<T, 8, true>) : reinterpret_cast<const void *>(&k_rotary<T, 8, false>);
    return interleaved ? reinterpret_cast<const void *>(&k_rotary<T, 1, true>) : reinterpret_cast<const void *>(&k_rotary<T, 1, false>);
}

} // namespace

extern "C" int a2sgd_rotary(const a2sgd_heads *q, const a2sgd_heads *k, const a2sgd_heads *q_out, const a2sgd_heads *k_out,
                            const int32_t *positions, uint32_t axes, const uint32_t *sections, double base, uint32_t flags,
                            uint64_t tokens, uint32_t q_heads, uint32_t k_heads, uint32_t head_dim, int dtype, int device, void *stream)
{
    if (!known(dtype) || axes == 0 || axes > A2SGD_ROTARY_MAX_AXES || !sections || !std::isfinite(base) || !(base > 0.0) || head_dim == 0 ||
        q_heads == 0 || (flags & ~7u))
        return A2SGD_ERR_ARG;
    if (head_dim > A2SGD_ROTARY_MAX_HEAD_DIM || tokens >= (1ull << 31) || q_heads > 65535u || k_heads > 65535u) return A2SGD_ERR_TOO_LARGE;
    uint64_t pairs = 0;
    for (uint32_t i = 0; i < axes; ++i) {
        if (sections[i] == 0) return A2SGD_ERR_ARG;
        pairs += sections[i];
    }
    if (2 * pairs > head_dim) return A2SGD_ERR_ARG;
    if (tokens == 0) return A2SGD_OK;
    if (!positions) return A2SGD_ERR_ARG;
    if (!aligned(positions, 4)) return A2SGD_ERR_ALIGN;
    Args a;
    a.k = Side{};
    bool vec = pairs % 8 == 0 && (head_dim - 2 * pairs) % 8 == 0;
    const auto side = [&](Side &s, const a2sgd_heads *in, const a2sgd_heads *out, uint32_t heads) {
        int rc = check(in, heads, tokens, dtype, false);
        if (rc == A2SGD_OK) rc = check(out, heads, tokens, dtype, true);
        if (rc != A2SGD_OK) return rc;
        s = Side{in->p, out->p, in->row_stride, in->head_stride, out->row_stride, out->head_stride, (int)heads};
        vec = vec && wide(in, dtype) && wide(out, dtype);
        return (int)A2SGD_OK;
    };
    int rc = side(a.q, q, q_out, q_heads);
    if (rc == A2SGD_OK && k_heads) rc = side(a.k, k, k_out, k_heads);
    if (rc != A2SGD_OK) return rc;
    // omega_j in turns, modulo a whole one: powers by repeated products in 64 bits of mantissa
    const long double kTurn = 6.283185307179586476925286766559005768L;
    long double omega = 1.0L, ratio = powl((long double)base, -1.0L / (long double)pairs);
    for (uint32_t i = 0, j = 0; i < axes; ++i) {
        if (flags & A2SGD_ROTARY_LADDER_PER_AXIS) {
            omega = 1.0L;
            ratio = powl((long double)base, -1.0L / (long double)sections[i]);
        }
        for (uint32_t l = 0; l < sections[i]; ++l, ++j, omega *= ratio) {
            const long double t = omega / kTurn, part = t < 1.0L ? t : t - floorl(t);
            a.turn[j] = part >= 1.0L ? 0 : (uint64_t)(part * 18446744073709551616.0L);
            a.axis[j] = (uint8_t)i;
        }
    }
    a.positions = positions;
    a.tokens = (int64_t)tokens;
    a.pairs = (int)pairs;
    a.d = (int)head_dim;
    a.interleaved = (flags & A2SGD_ROTARY_INTERLEAVED) != 0;
    a.inverse = (flags & A2SGD_ROTARY_INVERSE) != 0;
    const int step = vec ? 8 : 1;
    a.units = (int)pairs / step;
    const bool in_place = q->p == q_out->p && q->row_stride == q_out->row_stride && q->head_stride == q_out->head_stride &&
                          (k_heads == 0 || (k->p == k_out->p && k->row_stride == k_out->row_stride && k->head_stride == k_out->head_stride));
    a.tail_units = in_place ? 0 : (int)(head_dim - 2 * pairs) / step;
    DeviceGuard guard(device);
    const int sms = guard.ok ? sm_count(device) : 0;
    if (sms < 1) return A2SGD_ERR_CUDA;
    // a token's heads are shared out until the SMs are full
    const int heads = (int)(q_heads + k_heads);
    const int64_t threads = (int64_t)tokens * (a.units + a.tail_units);
    a.split = (int)std::max<int64_t>(1, std::min<int64_t>(heads, (int64_t)sms * 2048 / threads));
    a.heads_each = (heads + a.split - 1) / a.split;
    a.split = (heads + a.heads_each - 1) / a.heads_each;
    const int64_t blocks = (threads * a.split + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff) return A2SGD_ERR_TOO_LARGE;
    const void *fn = dtype == A2SGD_F32    ? pick<float>(vec, a.interleaved)
                     : dtype == A2SGD_BF16 ? pick<__nv_bfloat16>(vec, a.interleaved)
                                           : pick<__half>(vec, a.interleaved);
    void *params[] = {&a};
    A2_TRAIN_CUDA(launch(fn, dim3((unsigned)blocks), kThreads, 0, params, static_cast<cudaStream_t>(stream)));
    return A2SGD_OK;
}
