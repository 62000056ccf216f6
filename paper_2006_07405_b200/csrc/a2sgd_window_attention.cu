// Attention with a sliding window and first tokens that stay visible, forward and backward.
#include "a2sgd_train.cuh"

#include <algorithm>
#include <cmath>
#include <cstdint>

using namespace a2sgd_train;

namespace {

struct Heads {
    void *p;
    int64_t seq, row, head;
};

struct Args {
    Heads q, k, v, o, dout, dq, dk, dv;
    float *lse, *delta;
    const int32_t *q_ranges, *k_ranges;
    int sequences, q_heads, kv_heads, d, group;
    int q_rows, k_rows, window, sinks;
    int packed_q; // one lse plane
    float scale;
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
__device__ __forceinline__ int64_t lse_at(const Args &a, int b, int head, int64_t row)
{
    return ((int64_t)(a.packed_q ? 0 : b) * a.q_heads + head) * a.q_rows + row;
}
__device__ __forceinline__ bool sees(int place, int key, int window, int sinks)
{
    return key <= place && (key > place - window || key < sinks);
}

// A warp a query: 32 keys at a time, a lane each, then the lanes share out the head's elements.
template <typename T, bool BACKWARD>
__global__ void __launch_bounds__(128) k_query(const __grid_constant__ Args a)
{
    wait_prior_grid();
    release_next_grid();
    const int lane = threadIdx.x & 31, head = blockIdx.y, b = blockIdx.z, i = blockIdx.x * 4 + (threadIdx.x >> 5);
    const Range qr = range_of(a.q_ranges, b, a.q_rows), kr = range_of(a.k_ranges, b, a.k_rows);
    if (i >= qr.count) return;
    const int64_t row = qr.first + i;
    const int place = i + kr.count - qr.count;
    const T *q = at<T>(a.q, b, row, head), *g = BACKWARD ? at<T>(a.dout, b, row, head) : nullptr;
    const T *o = BACKWARD ? at<T>(a.o, b, row, head) : nullptr;
    float delta = 0.0f, lse = 0.0f;
    if (BACKWARD) {
        for (int c = lane; c < a.d; c += 32) delta += to_f32(g[c]) * to_f32(o[c]);
        for (int s = 16; s; s >>= 1) delta += __shfl_xor_sync(0xffffffffu, delta, s);
        lse = a.lse[lse_at(a, b, head, row)];
        if (lane == 0) a.delta[lse_at(a, b, head, row)] = delta;
    }
    float acc[4] = {}, top = -INFINITY, total = 0.0f;
    const int lo = max(0, place - a.window + 1), end = min(place + 1, kr.count);
    for (int j0 = 0; j0 < end; j0 += 32) {
        if (j0 + 32 <= lo && j0 >= a.sinks) {
            j0 = lo / 32 * 32 - 32;
            continue;
        }
        const int j = j0 + lane;
        const bool on = j < end && sees(place, j, a.window, a.sinks);
        float s = -INFINITY, dp = 0.0f;
        if (on) {
            const T *k = at<T>(a.k, b, kr.first + j, head / a.group), *v = at<T>(a.v, b, kr.first + j, head / a.group);
            s = 0.0f;
            for (int c = 0; c < a.d; ++c) {
                s += to_f32(q[c]) * to_f32(k[c]);
                if (BACKWARD) dp += to_f32(g[c]) * to_f32(v[c]);
            }
            s *= a.scale;
        }
        float p;
        if (BACKWARD) {
            p = on ? expf(s - lse) * (dp - delta) * a.scale : 0.0f;
        } else {
            float most = s;
            for (int x = 16; x; x >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
            const float next = fmaxf(top, most), base = next == -INFINITY ? 0.0f : next, shrink = expf(top - base);
            p = expf(s - base);
            total *= shrink;
            for (float &x : acc) x *= shrink;
            top = next;
            float sum = p;
            for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
            total += sum;
        }
        for (int r = 0; r < 32 && j0 + r < end; ++r) {
            const float w = __shfl_sync(0xffffffffu, p, r);
            if (!sees(place, j0 + r, a.window, a.sinks)) continue;
            const T *x = at<T>(BACKWARD ? a.k : a.v, b, kr.first + j0 + r, head / a.group);
            for (int e = 0; e < 4; ++e)
                if (lane + 32 * e < a.d) acc[e] += w * to_f32(x[lane + 32 * e]);
        }
    }
    if (BACKWARD && !a.dq.p) return;
    T *out = at<T>(BACKWARD ? a.dq : a.o, b, row, head);
    for (int e = 0; e < 4; ++e)
        if (lane + 32 * e < a.d) out[lane + 32 * e] = from_f32<T>(BACKWARD ? acc[e] : total > 0.0f ? acc[e] / total : 0.0f);
    if (!BACKWARD && a.lse && lane == 0) a.lse[lse_at(a, b, head, row)] = top + logf(total);
}

// A warp a key and key head: the queries that see it, 32 at a time.
template <typename T>
__global__ void __launch_bounds__(128) k_key(const __grid_constant__ Args a)
{
    wait_prior_grid();
    release_next_grid();
    const int lane = threadIdx.x & 31, kv = blockIdx.y, b = blockIdx.z, j = blockIdx.x * 4 + (threadIdx.x >> 5);
    const Range qr = range_of(a.q_ranges, b, a.q_rows), kr = range_of(a.k_ranges, b, a.k_rows);
    if (j >= kr.count) return;
    const T *k = at<T>(a.k, b, kr.first + j, kv), *v = at<T>(a.v, b, kr.first + j, kv);
    const int ahead = kr.count - qr.count;
    const int first = max(0, j - ahead);
    const int end = j < a.sinks ? qr.count : (int)min((int64_t)qr.count, (int64_t)j - ahead + a.window);
    float dk[4] = {}, dv[4] = {};
    for (int head = kv * a.group; head < (kv + 1) * a.group; ++head) {
        for (int i0 = first; i0 < end; i0 += 32) {
            const int i = i0 + lane;
            float p = 0.0f, ds = 0.0f;
            if (i < end) {
                const T *q = at<T>(a.q, b, qr.first + i, head), *g = at<T>(a.dout, b, qr.first + i, head);
                float s = 0.0f, dp = 0.0f;
                for (int c = 0; c < a.d; ++c) {
                    s += to_f32(q[c]) * to_f32(k[c]);
                    dp += to_f32(g[c]) * to_f32(v[c]);
                }
                const int64_t at_row = lse_at(a, b, head, qr.first + i);
                p = expf(s * a.scale - a.lse[at_row]);
                ds = p * (dp - a.delta[at_row]) * a.scale;
            }
            for (int r = 0; r < 32 && i0 + r < end; ++r) {
                const float wp = __shfl_sync(0xffffffffu, p, r), ws = __shfl_sync(0xffffffffu, ds, r);
                const T *q = at<T>(a.q, b, qr.first + i0 + r, head), *g = at<T>(a.dout, b, qr.first + i0 + r, head);
                for (int e = 0; e < 4; ++e) {
                    if (lane + 32 * e >= a.d) break;
                    dk[e] += ws * to_f32(q[lane + 32 * e]);
                    dv[e] += wp * to_f32(g[lane + 32 * e]);
                }
            }
        }
    }
    for (int e = 0; e < 4; ++e) {
        if (lane + 32 * e >= a.d) break;
        if (a.dk.p) at<T>(a.dk, b, kr.first + j, kv)[lane + 32 * e] = from_f32<T>(dk[e]);
        if (a.dv.p) at<T>(a.dv, b, kr.first + j, kv)[lane + 32 * e] = from_f32<T>(dv[e]);
    }
}

// ------------------------------------------------------------------ host
int check_shape(const a2sgd_attention *s)
{
    if (!s || (s->dtype != A2SGD_BF16 && s->dtype != A2SGD_F16)) return A2SGD_ERR_ARG;
    if (s->kv_heads == 0 || s->q_heads == 0 || s->q_heads % s->kv_heads || s->head_dim == 0) return A2SGD_ERR_ARG;
    if (s->window == 0 || !std::isfinite(s->scale) || !(s->scale > 0.0)) return A2SGD_ERR_ARG;
    if (s->head_dim > A2SGD_ATTENTION_MAX_HEAD_DIM || s->q_heads > 65535u || s->sequences > 65535u || s->q_rows >= (1ull << 30) ||
        s->k_rows >= (1ull << 30))
        return A2SGD_ERR_TOO_LARGE;
    return A2SGD_OK;
}

// A tensor of `heads` heads and `rows` rows a sequence.  written: no two elements may share a place.
int check_heads(const a2sgd_attention *s, const a2sgd_heads *h, uint32_t heads, uint64_t rows, const int32_t *ranges, bool needed,
                bool written)
{
    if (!h || !h->p) return needed && rows ? A2SGD_ERR_ARG : A2SGD_OK;
    if (h->sequence_stride < 0 || h->row_stride < 0 || h->head_stride < 0) return A2SGD_ERR_ARG;
    if (written && ((h->sequence_stride == 0 && s->sequences > 1 && !ranges) || (h->row_stride == 0 && rows > 1) ||
                    (h->head_stride == 0 && heads > 1)))
        return A2SGD_ERR_ARG;
    return aligned(h->p, 2) ? A2SGD_OK : A2SGD_ERR_ALIGN;
}

Heads heads_of(const a2sgd_heads *h)
{
    return h && h->p ? Heads{h->p, h->sequence_stride, h->row_stride, h->head_stride} : Heads{nullptr, 0, 0, 0};
}

Args common(const a2sgd_attention *s, const a2sgd_heads *q, const a2sgd_heads *k, const a2sgd_heads *v, const a2sgd_heads *o)
{
    Args a{};
    a.q = heads_of(q), a.k = heads_of(k), a.v = heads_of(v), a.o = heads_of(o);
    a.q_ranges = s->q_ranges, a.k_ranges = s->k_ranges;
    a.sequences = (int)s->sequences, a.q_heads = (int)s->q_heads, a.kv_heads = (int)s->kv_heads, a.d = (int)s->head_dim;
    a.group = a.q_heads / a.kv_heads;
    a.q_rows = (int)s->q_rows, a.k_rows = (int)s->k_rows;
    a.window = (int)std::min<uint64_t>(s->window, 1u << 30);
    a.sinks = (int)std::min<uint64_t>(s->sinks, 1u << 30);
    a.packed_q = s->q_ranges && q->sequence_stride == 0;
    a.scale = (float)s->scale;
    return a;
}

template <typename T>
int forward(Args &a, cudaStream_t s)
{
    void *params[] = {&a};
    A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_query<T, false>),
                         dim3((unsigned)(a.q_rows + 3) / 4, (unsigned)a.q_heads, (unsigned)a.sequences), 128, 0, params, s));
    return A2SGD_OK;
}

template <typename T>
int backward(Args &a, cudaStream_t s)
{
    void *params[] = {&a};
    if (a.q_rows)
        A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_query<T, true>),
                             dim3((unsigned)(a.q_rows + 3) / 4, (unsigned)a.q_heads, (unsigned)a.sequences), 128, 0, params, s));
    if (a.k_rows && (a.dk.p || a.dv.p))
        A2_TRAIN_CUDA(launch(reinterpret_cast<const void *>(&k_key<T>),
                             dim3((unsigned)(a.k_rows + 3) / 4, (unsigned)a.kv_heads, (unsigned)a.sequences), 128, 0, params, s));
    return A2SGD_OK;
}

} // namespace

extern "C" uint64_t a2sgd_window_attention_workspace(const a2sgd_attention *shape, uint32_t flags)
{
    if (!shape || !(flags & A2SGD_ATTENTION_BACKWARD)) return 0;
    return (uint64_t)shape->sequences * shape->q_heads * shape->q_rows * 4;
}

extern "C" int a2sgd_window_attention_forward(const a2sgd_attention *shape, const a2sgd_heads *q, const a2sgd_heads *k,
                                              const a2sgd_heads *v, const a2sgd_heads *o, float *lse, void *workspace,
                                              uint64_t workspace_bytes, int device, void *stream)
{
    int rc = check_shape(shape);
    if (rc != A2SGD_OK || shape->sequences == 0 || shape->q_rows == 0) return rc;
    if ((rc = check_heads(shape, q, shape->q_heads, shape->q_rows, shape->q_ranges, true, false)) != A2SGD_OK ||
        (rc = check_heads(shape, k, shape->kv_heads, shape->k_rows, shape->k_ranges, true, false)) != A2SGD_OK ||
        (rc = check_heads(shape, v, shape->kv_heads, shape->k_rows, shape->k_ranges, true, false)) != A2SGD_OK ||
        (rc = check_heads(shape, o, shape->q_heads, shape->q_rows, shape->q_ranges, true, true)) != A2SGD_OK)
        return rc;
    if (!aligned(workspace, 256) || !aligned(lse, 4)) return A2SGD_ERR_ALIGN;
    (void)workspace_bytes;
    DeviceGuard guard(device);
    if (!guard.ok) return A2SGD_ERR_CUDA;
    Args a = common(shape, q, k, v, o);
    a.lse = lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return shape->dtype == A2SGD_BF16 ? forward<__nv_bfloat16>(a, s) : forward<__half>(a, s);
}

extern "C" int a2sgd_window_attention_backward(const a2sgd_attention *shape, const a2sgd_heads *dout, const a2sgd_heads *q,
                                               const a2sgd_heads *k, const a2sgd_heads *v, const a2sgd_heads *o, const float *lse,
                                               const a2sgd_heads *dq, const a2sgd_heads *dk, const a2sgd_heads *dv, void *workspace,
                                               uint64_t workspace_bytes, int device, void *stream)
{
    int rc = check_shape(shape);
    if (rc != A2SGD_OK || shape->sequences == 0) return rc;
    for (const a2sgd_heads *h : {dout, q, o})
        if ((rc = check_heads(shape, h, shape->q_heads, shape->q_rows, shape->q_ranges, true, false)) != A2SGD_OK) return rc;
    for (const a2sgd_heads *h : {k, v})
        if ((rc = check_heads(shape, h, shape->kv_heads, shape->k_rows, shape->k_ranges, true, false)) != A2SGD_OK) return rc;
    for (const a2sgd_heads *h : {dk, dv})
        if ((rc = check_heads(shape, h, shape->kv_heads, shape->k_rows, shape->k_ranges, false, true)) != A2SGD_OK) return rc;
    if ((rc = check_heads(shape, dq, shape->q_heads, shape->q_rows, shape->q_ranges, false, true)) != A2SGD_OK) return rc;
    if (!lse && shape->q_rows) return A2SGD_ERR_ARG;
    if (!aligned(workspace, 256) || !aligned(lse, 4)) return A2SGD_ERR_ALIGN;
    if (workspace_bytes < a2sgd_window_attention_workspace(shape, A2SGD_ATTENTION_BACKWARD | A2SGD_ATTENTION_ALIGNED))
        return A2SGD_ERR_ARG;
    DeviceGuard guard(device);
    if (!guard.ok) return A2SGD_ERR_CUDA;
    Args a = common(shape, q, k, v, o);
    a.dout = heads_of(dout), a.dq = heads_of(dq), a.dk = heads_of(dk), a.dv = heads_of(dv);
    a.lse = const_cast<float *>(lse);
    a.delta = static_cast<float *>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return shape->dtype == A2SGD_BF16 ? backward<__nv_bfloat16>(a, s) : backward<__half>(a, s);
}

extern "C" int a2sgd_window_attention_status(int device, int *device_status, void *stream)
{
    if (!device_status) return A2SGD_ERR_ARG;
    DeviceGuard guard(device);
    if (!guard.ok) return A2SGD_ERR_CUDA;
    A2_TRAIN_CUDA(cudaStreamSynchronize(static_cast<cudaStream_t>(stream)));
    *device_status = A2SGD_OK;
    return A2SGD_OK;
}
