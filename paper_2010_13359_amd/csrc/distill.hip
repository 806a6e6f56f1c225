// Distillation from a teacher's top logits: the loss of student logits against
// softmax(val / T) over the entries that the teacher sent, and its gradient.
#include "layers.hpp"

namespace dq {
namespace {

constexpr int kMostEntries = 1024;
constexpr int kThreads = 512, kWaves = kThreads / 64;

struct DistillArgs {
    const float *val;
    const uint32_t *idx;
    const float *weight;  // or NULL
    int64_t V, ld;
    int k;
    float T, inv_T;
};

constexpr float kNone = -INFINITY;

// exp((z - largest) / T).  The exponent's product with log2(e) is carried with
// what its rounding lost where the result is kept in 32 bits: exp2's own
// argument has an ulp of 2^-17 at 2^6, which would be 5e-6 of the result; a
// 16-bit result has no use for it.
template <bool FINE>
__device__ __forceinline__ float exp_of(float z, float largest, float inv_T) {
    constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596299e-8f;
    const float x = (z - largest) * inv_T;
    const float hi = x * kLog2e;
    float e = __builtin_amdgcn_exp2f(hi);
    if (FINE) {
        const float lo = fmaf(x, kLog2eRest, fmaf(x, kLog2e, -hi));
        if (e > 0.0f) e = fmaf(e, lo * 0.693147182f, e);
    }
    return e;
}

// The reference of the exponents: 0 while no logit above -inf is known, so
// that -inf - reference is -inf and not NaN.
__device__ __forceinline__ float reference(float largest) { return largest == kNone ? 0.0f : largest; }

// Running maximum and sum of a softmax.  A sum that knows no logit above -inf
// is 0 (or NaN), and its factor exp(-inf - reference) is 0 too.
struct Softmax {
    float largest, total;
};

// The teacher's distribution of one token into LDS: t[j], log t[j], and whether
// entry j counts.  Every thread of the workgroup calls it; returns whether any
// entry counts.
__device__ bool teacher(const DistillArgs &a, int64_t row, float *t, float *logt, uint32_t *idx, float (*slots)[kWaves]) {
    const float *val = a.val + row * a.k;
    const uint32_t *from = a.idx + row * a.k;
    float top = kNone;
    bool any = false;
    for (int j = threadIdx.x; j < a.k; j += kThreads) {
        const uint32_t i = from[j];
        const float v = val[j];
        const bool counts = i < a.V && v != kNone;
        idx[j] = counts ? i : UINT32_MAX;
        t[j] = v;
        any |= counts;
        if (counts) top = fmaxf(top, v);
    }
    any = __syncthreads_or(any);
    top = group_max<kWaves>(top, slots[0]);
    float sum = 0.0f;
    for (int j = threadIdx.x; j < a.k; j += kThreads) {
        if (idx[j] == UINT32_MAX) continue;
        logt[j] = (t[j] - top) * a.inv_T;
        t[j] = expf(logt[j]);
        sum += t[j];
    }
    sum = group_sum<kWaves>(sum, slots[1]);
    const float log_sum = logf(sum);
    for (int j = threadIdx.x; j < a.k; j += kThreads) {
        if (idx[j] == UINT32_MAX) continue;
        logt[j] -= log_sum;
        t[j] /= sum;
    }
    __syncthreads();
    return any;
}

// One workgroup per token.  LOSS: the statistics and the loss; GRAD: dz, from
// the statistics just made or (LOSS not) from `stats`.
template <typename T, bool LOSS, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_distill(const T *z, DistillArgs a, float *loss, float *stats, T *dz) {
    constexpr bool FINE = sizeof(T) == 4;
    __shared__ float t[kMostEntries], logt[kMostEntries];
    __shared__ uint32_t idx[kMostEntries];
    __shared__ float slots[6][kWaves];
    const int64_t row = blockIdx.x;
    const T *from = z + row * a.ld;
    T *to = dz + row * a.ld;
    const float weight = a.weight ? a.weight[row] : 1.0f;
    bool takes_part = weight != 0.0f;
    if (takes_part) takes_part = teacher(a, row, t, logt, idx, slots);
    Softmax s{kNone, 0.0f};
    if (takes_part) {
        if (LOSS) {
            for (int64_t c = 8 * threadIdx.x; c < a.V; c += 8 * kThreads) {
                const f32x8 f = load8(from + c, a.V - c, kNone);
                float top = s.largest;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, f[i]);
                if (top > s.largest) {
                    s.total *= exp_of<FINE>(s.largest, top, a.inv_T);
                    s.largest = top;
                }
                const float ref = reference(s.largest);
#pragma unroll
                for (int i = 0; i < 8; ++i) s.total += exp_of<FINE>(f[i], ref, a.inv_T);
            }
            const float mine = s.largest;
            s.largest = group_max<kWaves>(mine, slots[2]);
            s.total = group_sum<kWaves>(s.total * exp_of<FINE>(mine, reference(s.largest), a.inv_T), slots[3]);
            takes_part = !(s.largest == kNone && s.total == 0.0f);
        } else {
            s.largest = stats[2 * row];
            s.total = stats[2 * row + 1];
            takes_part = s.total != 0.0f;
        }
    }
    if (LOSS) {
        float sum = 0.0f;
        if (takes_part) {
            const float log_total = logf(s.total);
            for (int j = threadIdx.x; j < a.k; j += kThreads) {
                if (idx[j] == UINT32_MAX || t[j] == 0.0f) continue;
                const float logs = (static_cast<float>(from[idx[j]]) - s.largest) * a.inv_T - log_total;
                sum = fmaf(t[j], logt[j] - logs, sum);
            }
        }
        sum = group_sum<kWaves>(sum, slots[4]);
        if (threadIdx.x == 0) {
            loss[row] = takes_part ? weight * a.T * a.T * sum : 0.0f;
            if (stats) {
                stats[2 * row] = takes_part ? s.largest : 0.0f;
                stats[2 * row + 1] = takes_part ? s.total : 0.0f;
            }
        }
    }
    if (GRAD) {
        if (!takes_part) {
            for (int64_t c = 8 * threadIdx.x; c < a.ld; c += 8 * kThreads) store8(to + c, a.ld - c, f32x8(0.0f));
            return;
        }
        const float coef = weight * a.T, over = coef / s.total;
        // the teacher's entries first, for dz may be z
        for (int j = threadIdx.x; j < a.k; j += kThreads) {
            if (idx[j] == UINT32_MAX) continue;
            float sum = 0.0f;  // an index named more than once: the same sum for each
            for (int o = 0; o < a.k; ++o) sum += idx[o] == idx[j] ? t[o] : 0.0f;
            logt[j] = (exp_of<FINE>(static_cast<float>(from[idx[j]]), s.largest, a.inv_T) / s.total - sum) * coef;
        }
        __syncthreads();
        for (int64_t c = 8 * threadIdx.x; c < a.ld; c += 8 * kThreads) {
            f32x8 f = load8(from + c, a.V - c, kNone);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = c + i < a.V ? exp_of<FINE>(f[i], s.largest, a.inv_T) * over : 0.0f;
            store8(to + c, a.ld - c, f);
        }
        __syncthreads();
        for (int j = threadIdx.x; j < a.k; j += kThreads)
            if (idx[j] != UINT32_MAX) to[idx[j]] = static_cast<T>(logt[j]);
    }
}

dqgan_status check(dqgan_plan P, const dqgan_distill_desc *d) {
    if (!P || !d) return DQGAN_EINVAL;
    if (d->vocab < 1 || d->ld < d->vocab || d->ld > INT32_MAX || d->k < 1 || d->k > kMostEntries) return DQGAN_EINVAL;
    if (!(d->temperature >= 0x1p-10f && d->temperature <= 0x1p10f)) return DQGAN_EINVAL;
    if (!tokens_ok(P, d->tokens) || !type_ok(d->type) || d->reserved != 0) return DQGAN_EINVAL;
    return DQGAN_OK;
}

dqgan_status check_inputs(const dqgan_distill_desc *d, const void *z, const float *val, const uint32_t *idx,
                          const float *weight) {
    const bool any = d->tokens > 0;
    DQ_TRY(check_ptr(z, any));
    DQ_TRY(check_ptr(val, any));
    DQ_TRY(check_ptr(idx, any));
    return check_ptr(weight, false);
}

template <bool LOSS, bool GRAD>
dqgan_status run(dqgan_plan P, const dqgan_distill_desc *d, const void *z, const float *val, const uint32_t *idx,
                 const float *weight, float *loss, float *stats, void *dz, hipStream_t st) {
    const DistillArgs a{val, idx, weight, d->vocab, d->ld, d->k, d->temperature, 1.0f / d->temperature};
    const int64_t rows = d->tokens * P->desc.M;
    // a launch has fewer than 2^32 threads
    constexpr int64_t kMost = int64_t(1) << 22;
    for (int64_t r = 0; r < rows; r += kMost) {
        const uint32_t n = static_cast<uint32_t>(rows - r < kMost ? rows - r : kMost);
        DistillArgs b = a;
        b.val += r * a.k;
        b.idx += r * a.k;
        if (b.weight) b.weight += r;
        with_type(d->type, [&](auto t) {
            using T = decltype(t);
            k_distill<T, LOSS, GRAD><<<n, kThreads, 0, st>>>(static_cast<const T *>(z) + r * a.ld, b, loss ? loss + r : loss,
                                                             stats ? stats + 2 * r : stats,
                                                             static_cast<T *>(dz) + (GRAD ? r * a.ld : 0));
        });
    }
    return launched();
}

}  // namespace
}  // namespace dq

using namespace dq;

extern "C" {

dqgan_status dqgan_distill_forward(dqgan_plan P, const dqgan_distill_desc *d, const void *z, const float *val,
                                   const uint32_t *idx, const float *weight, float *loss, float *stats, void *workspace,
                                   void *stream) {
    DQ_TRY(check(P, d));
    const bool any = d->tokens > 0;
    DQ_TRY(check_inputs(d, z, val, idx, weight));
    DQ_TRY(check_ptr(loss, any));
    DQ_TRY(check_ptr(stats, any));
    DQ_TRY(check_ptr(workspace, false));
    DQ_TRY(check_device(P));
    if (!any) return DQGAN_OK;
    return run<true, false>(P, d, z, val, idx, weight, loss, stats, nullptr, static_cast<hipStream_t>(stream));
}

dqgan_status dqgan_distill_backward(dqgan_plan P, const dqgan_distill_desc *d, const void *z, const float *val,
                                    const uint32_t *idx, const float *weight, const float *stats, void *dz,
                                    void *stream) {
    DQ_TRY(check(P, d));
    const bool any = d->tokens > 0;
    DQ_TRY(check_inputs(d, z, val, idx, weight));
    DQ_TRY(check_ptr(stats, any));
    DQ_TRY(check_ptr(dz, any));
    DQ_TRY(check_device(P));
    if (!any) return DQGAN_OK;
    return run<false, true>(P, d, z, val, idx, weight, nullptr, const_cast<float *>(stats), dz,
                            static_cast<hipStream_t>(stream));
}

dqgan_status dqgan_distill_fused(dqgan_plan P, const dqgan_distill_desc *d, const void *z, const float *val,
                                 const uint32_t *idx, const float *weight, float *loss, void *dz, void *workspace,
                                 void *stream) {
    DQ_TRY(check(P, d));
    const bool any = d->tokens > 0;
    DQ_TRY(check_inputs(d, z, val, idx, weight));
    DQ_TRY(check_ptr(loss, any));
    DQ_TRY(check_ptr(dz, any));
    DQ_TRY(check_ptr(workspace, false));
    DQ_TRY(check_device(P));
    if (!any) return DQGAN_OK;
    return run<true, true>(P, d, z, val, idx, weight, loss, nullptr, dz, static_cast<hipStream_t>(stream));
}

dqgan_status dqgan_distill_bytes(dqgan_plan P, const dqgan_distill_desc *d, size_t *bytes) {
    DQ_TRY(check(P, d));
    if (!bytes) return DQGAN_EINVAL;
    *bytes = 0;
    return DQGAN_OK;
}

}  // extern "C"
