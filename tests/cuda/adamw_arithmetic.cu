// Roots, quotients and codes of AdamW's step (csrc/a2sgd_adamw_arith.cuh) against the single operations of CUDA: every
// mantissa for the roots; for the quotients every divisor mantissa with the numerators whose quotients lie nearest the middle between two
// numbers, and hashed ones over the whole range; for the codes the neighbourhood of every square with every dither.
// Prints a line for each with the number of differences.
#include "a2sgd_adamw_arith.cuh"

#include <cstdio>

using namespace a2sgd_train;

__device__ unsigned long long differences;
__device__ unsigned int example[2];

__device__ void differ(float a, float b)
{
    if (atomicAdd(&differences, 1ull) == 0) {
        example[0] = __float_as_uint(a);
        example[1] = __float_as_uint(b);
    }
}
__device__ bool same(float a, float b) { return __float_as_uint(a) == __float_as_uint(b); }

// bits of 2^exponent and of 2^(exponent + 1) with every mantissa
__global__ void roots(int exponent)
{
    const uint32_t i = blockIdx.x * 256 + threadIdx.x; // 2^23: a pair holds the two binades of one mantissa
    const float a = __uint_as_float((uint32_t)(exponent + 127) << 23 | i), b = __uint_as_float((uint32_t)(exponent + 128) << 23 | i);
    float x, y;
    unpair(root2(pair(a, b)), x, y);
    if (!same(x, __fsqrt_rn(a))) differ(a, x);
    if (!same(y, __fsqrt_rn(b))) differ(b, y);
}

__device__ void quotient(float m, float d)
{
    float x, y;
    unpair(quotient2(pair(m, -m), pair(d)), x, y);
    if (!same(x, __fdiv_rn(m, d))) differ(m, d);
    if (!same(y, __fdiv_rn(-m, d))) differ(-m, d);
}

// d = D 2^j with D odd.  N 2^s = d (2 Q + 1) + c says that N / d is c / (2 d) of a unit away from the middle between two numbers
// (s = 24 where N >= d, 25 where N < d): with c = c' 2^j, N = c' / 2^(s - j) mod D.
__global__ void quotients_near_the_middle(int scale_m, int scale_d)
{
    const uint32_t d = (1u << 23) + blockIdx.x * 256 + threadIdx.x;
    const int j = __ffs(d) - 1;
    const uint32_t odd = d >> j;
    if (odd == 1) return;
    for (int s = 24; s <= 25; ++s) {
        const uint32_t lo = s == 24 ? d : 1u << 23, hi = s == 24 ? 1u << 24 : d; // N in [lo, hi)
        for (int c = -4; c <= 4; ++c) {
            if (c == 0) continue;
            uint32_t n = (uint32_t)((c + 8ll * odd) % odd);
            for (int k = j; k < s; ++k) n = n & 1 ? (n + odd) / 2 : n / 2;
            uint32_t at = n + (lo > n ? (lo - n + odd - 1) / odd * odd : 0);
            for (int tries = 0; tries < 6 && at < hi; ++tries, at += odd) quotient(ldexpf((float)at, scale_m - 23), ldexpf((float)d, scale_d - 23));
        }
    }
}

__device__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16, x *= 0x7feb352du, x ^= x >> 15, x *= 0x846ca68bu;
    return x ^ x >> 16;
}
// d from 2^-40 to 2^68, |m| from 2^-100 to 2^80, quotients in the normal range
__global__ void quotients_hashed(uint32_t seed)
{
    for (int k = 0; k < 64; ++k) {
        const uint32_t a = mix(seed + 64 * (blockIdx.x * 256 + threadIdx.x) + k), b = mix(a + 0x9e3779b9u), c = mix(b + seed);
        const int ed = -40 + (int)(c % 108), em = -100 + (int)((c >> 8) % 180);
        if (em - ed <= -125) continue;
        quotient(__uint_as_float((uint32_t)(em + 127) << 23 | a >> 9), __uint_as_float((uint32_t)(ed + 127) << 23 | b >> 9));
    }
}

// The rule in single operations: q = floor(sqrt(s)), one more where s - q^2 > u (2 q + 1).
__device__ float code(float s, float u, float top, float least)
{
    float q = floorf(__fsqrt_rn(s));
    if (__fsub_rn(s, q * q) > u * (2.0f * q + 1.0f)) q += 1.0f;
    return fmaxf(fminf(q, top), least);
}
// Block: a square; thread: 16 of the 4096 dithers; 257 numbers around the square and as many spread up to the next.
__global__ void codes(float top, float least)
{
    const float square = (float)(blockIdx.x * blockIdx.x);
    for (uint32_t k = threadIdx.x * 16; k < threadIdx.x * 16 + 16; ++k) {
        const uint32_t bits = 0x3f800000u | k << 11;
        const float u = (float)k * (1.0f / 4096.0f);
        for (int i = -128; i <= 128; ++i) {
            const int32_t at = (int32_t)__float_as_uint(square) + i;
            if (at < 0) continue;
            const float near = __uint_as_float((uint32_t)at), far = square + (2.0f * blockIdx.x + 1.0f) * (float)(i + 128) * (1.0f / 257.0f);
            float x, y;
            encode2(pair(near, far), bits, bits, top, least, x, y);
            if (!same(x, code(near, u, top, least))) differ(near, u);
            if (!same(y, code(far, u, top, least))) differ(far, u);
        }
    }
}

static bool report(const char *what)
{
    unsigned long long n = 0, zero = 0;
    unsigned int e[2] = {0, 0};
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&n, differences, sizeof n) != cudaSuccess ||
        cudaMemcpyFromSymbol(e, example, sizeof e) != cudaSuccess || cudaMemcpyToSymbol(differences, &zero, sizeof zero) != cudaSuccess) {
        std::printf("%s: %s\n", what, cudaGetErrorString(cudaGetLastError()));
        return false;
    }
    std::printf("%s: %llu differences", what, n);
    if (n) std::printf(", first %08x %08x", e[0], e[1]);
    std::printf("\n");
    return n == 0;
}

int main()
{
    bool good = true;
    for (int e = -80; e < 80; e += 2) roots<<<1 << 15, 256>>>(e);
    good &= report("roots");
    const int scales[][2] = {{0, 0}, {79, -40}, {-57, 67}, {79, 67}, {-99, -40}, {-99, 20}, {1, 0}, {0, 1}};
    for (const auto &s : scales) quotients_near_the_middle<<<1 << 15, 256>>>(s[0], s[1]);
    good &= report("quotients near the middle of two numbers");
    for (uint32_t k = 0; k < 8; ++k) quotients_hashed<<<1 << 16, 256>>>(k << 28 | k);
    good &= report("hashed quotients");
    codes<<<128, 256>>>(127.0f, 0.0f);
    codes<<<256, 256>>>(255.0f, 2.0f);
    good &= report("codes");
    return good ? 0 : 1;
}
