// Distillation from a teacher's top logits: the loss of student logits against
// softmax(val / T) over the entries that the teacher sent, and its gradient.
#include "layers.hpp"

namespace dq {
namespace {

constexpr int kMostEntries = 1024;

struct DistillArgs {
    const float *val;
    const uint32_t *idx;
    const float *weight;  // or NULL
    int64_t V, ld;
    int k;
    float T, inv_T, log2e_T;  // 1 / T, log2(e) / T
};

constexpr float kNone = -INFINITY;

// exp((z - largest) / T) as a power of two.  A 32-bit result carries along what
// the rounding of the exponent's product with log2(e) lost: at an exponent of
// 2^6 that is up to 3e-6 of the result.  A 16-bit result has no use for it.
template <bool FINE>
__device__ __forceinline__ float exp_of(const DistillArgs &a, float z, float largest) {
    if (!FINE) return __builtin_amdgcn_exp2f((z - largest) * a.log2e_T);
    constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596299e-8f;
    const float x = (z - largest) * a.inv_T, hi = x * kLog2e;
    const float e = __builtin_amdgcn_exp2f(hi);
    const float lo = fmaf(x, kLog2eRest, fmaf(x, kLog2e, -hi));
    return e > 0.0f ? fmaf(e, lo * 0.693147182f, e) : e;
}

// The reference of the exponents: 0 while no logit above -inf is known, so
// that -inf - reference is -inf and not NaN.
__device__ __forceinline__ float reference(float largest) { return largest == kNone ? 0.0f : largest; }

// Running maximum and sum of a softmax.  A sum that knows no logit above -inf
// is 0 (or NaN), and its factor exp(-inf - reference) is 0 too.
struct Softmax {
    float largest, total;
};

// One token's message in LDS: its entries' indices (UINT32_MAX: does not count),
// the student's logits there, and t and log t.
struct Message {
    uint32_t idx[kMostEntries];
    float z[kMostEntries], t[kMostEntries], logt[kMostEntries];
    float slots[4][16];
};

// Reads a message and the student's logits at its entries, and makes t and
// log t.  Every thread of the workgroup calls it.  Returns 0 if no entry counts,
// 1 if their indices ascend (so that none comes twice), else 2.
template <typename T, int W>
__device__ int teacher(const DistillArgs &a, int64_t row, const T *z, Message &s) {
    const float *val = a.val + row * a.k;
    const uint32_t *from = a.idx + row * a.k;
    float top = kNone;
    int have = 0;  // 1: an entry counts; 2: the indices do not ascend
    for (int j = threadIdx.x; j < a.k; j += 64 * W) {
        const uint32_t i = from[j];
        const float v = val[j];
        const bool counts = i < a.V && v != kNone;
        if (i < a.V && j > 0 && from[j - 1] >= i) have |= 2;
        s.idx[j] = counts ? i : UINT32_MAX;
        s.t[j] = v;
        if (!counts) continue;
        have |= 1;
        top = fmaxf(top, v);
        s.z[j] = static_cast<float>(z[i]);
    }
    have = (__syncthreads_or(have & 1) ? 1 : 0) | (__syncthreads_or(have & 2) ? 2 : 0);
    top = group_max<W>(top, s.slots[0]);
    float sum = 0.0f;
    for (int j = threadIdx.x; j < a.k; j += 64 * W) {
        if (s.idx[j] == UINT32_MAX) continue;
        s.logt[j] = (s.t[j] - top) * a.inv_T;
        s.t[j] = expf(s.logt[j]);
        sum += s.t[j];
    }
    sum = group_sum<W>(sum, s.slots[1]);
    const float log_sum = logf(sum);
    for (int j = threadIdx.x; j < a.k; j += 64 * W) {
        if (s.idx[j] == UINT32_MAX) continue;
        s.logt[j] -= log_sum;
        s.t[j] /= sum;
    }
    __syncthreads();
    return (have & 1) == 0 ? 0 : (have & 2) ? 2 : 1;
}

// The loss of a token that takes part.  Every thread calls it.
template <int W>
__device__ float loss_of(const DistillArgs &a, const Message &s, Softmax x, float *slot) {
    const float log_total = logf(x.total);
    float sum = 0.0f;
    for (int j = threadIdx.x; j < a.k; j += 64 * W) {
        if (s.idx[j] == UINT32_MAX || s.t[j] == 0.0f) continue;
        sum = fmaf(s.t[j], s.logt[j] - ((s.z[j] - x.largest) * a.inv_T - log_total), sum);
    }
    return group_sum<W>(sum, slot);
}

// dz at entry j's index.  An index named more than once gets the same value from
// each of its entries.
template <bool FINE>
__device__ float entry_gradient(const DistillArgs &a, const Message &s, int have, Softmax x, float coef, int j) {
    float sum = s.t[j];
    if (have == 2) {
        sum = 0.0f;
        for (int o = 0; o < a.k; ++o) sum += s.idx[o] == s.idx[j] ? s.t[o] : 0.0f;
    }
    return (exp_of<FINE>(a, s.z[j], x.largest) / x.total - sum) * coef;
}

// Keeps the compiler from holding a row's logits converted to 32 bits between
// two passes over them, which takes twice the registers.
template <typename V>
__device__ __forceinline__ void forget(V &raw) {
    typedef uint32_t Words __attribute__((ext_vector_type(sizeof(V) / 4)));
    Words w = __builtin_bit_cast(Words, raw);
#pragma unroll
    for (unsigned i = 0; i < sizeof(V) / 4; ++i) asm("" : "+v"(w[i]));
    raw = __builtin_bit_cast(V, w);
}

// One workgroup per token, whose logits stay in registers between the
// statistics and the gradient: NV vectors of eight per lane, and the last
// V % 8 one each in the first lanes.  LOSS: the statistics and the loss; GRAD:
// dz, from the statistics just made or (LOSS not) from `stats`.
template <typename T, int W, int NV, bool LOSS, bool GRAD>
__global__ __launch_bounds__(64 * W) void k_distill_row(const T *z, DistillArgs a, float *loss, float *stats, T *dz) {
    constexpr bool FINE = sizeof(T) == 4;
    typedef typename Vec8<T>::type Raw;
    typedef typename Vec8<T>::packed Packed;
    __shared__ Message s;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const T *from = z + row * a.ld;
    T *to = dz + row * a.ld;
    const float weight = a.weight ? a.weight[row] : 1.0f;
    const int vectors = static_cast<int>(a.V >> 3), rest = static_cast<int>(a.V & 7);
    int have = 0;
    Softmax x{0.0f, 0.0f};
    Raw raw[NV];
    float last = kNone;
    if (weight != 0.0f) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int q = tid + 64 * W * v;
            if (q < vectors)
                raw[v] = reinterpret_cast<const Packed *>(from)[q];
            else
                raw[v] = static_cast<T>(kNone);
        }
        if (tid < rest) last = static_cast<float>(from[8 * vectors + tid]);
        have = teacher<T, W>(a, row, from, s);
    }
    if (have != 0) {
        if (LOSS) {
            float top = last;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const f32x8 f = __builtin_convertvector(raw[v], f32x8);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, f[i]);
            }
            x.largest = group_max<W>(top, s.slots[2]);
            const float ref = reference(x.largest);
            float sum = exp_of<FINE>(a, last, ref);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                forget(raw[v]);
                const f32x8 f = __builtin_convertvector(raw[v], f32x8);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += exp_of<FINE>(a, f[i], ref);
            }
            x.total = group_sum<W>(sum, s.slots[3]);
            if (x.largest == kNone && x.total == 0.0f) have = 0;
        } else {
            x.largest = stats[2 * row];
            x.total = stats[2 * row + 1];
            if (x.total == 0.0f) have = 0;
        }
    }
    if (LOSS) {
        float value = 0.0f;
        if (have != 0) value = weight * a.T * a.T * loss_of<W>(a, s, x, s.slots[0]);
        if (tid == 0) {
            loss[row] = value;
            if (stats) {
                stats[2 * row] = have ? x.largest : 0.0f;
                stats[2 * row + 1] = have ? x.total : 0.0f;
            }
        }
    }
    if (GRAD) {
        if (have == 0) {
            for (int64_t c = 8 * tid; c < a.ld; c += 8 * 64 * W) store8(to + c, a.ld - c, f32x8(0.0f));
            return;
        }
        const float coef = weight * a.T, over = coef / x.total;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int q = tid + 64 * W * v;
            forget(raw[v]);
            f32x8 f = __builtin_convertvector(raw[v], f32x8);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = exp_of<FINE>(a, f[i], x.largest) * over;
            if (q < vectors) reinterpret_cast<Packed *>(to)[q] = __builtin_convertvector(f, Raw);
        }
        if (tid < rest) to[8 * vectors + tid] = static_cast<T>(exp_of<FINE>(a, last, x.largest) * over);
        for (int64_t c = a.V + tid; c < a.ld; c += 64 * W) to[c] = static_cast<T>(0.0f);
        __syncthreads();
        for (int j = tid; j < a.k; j += 64 * W)
            if (s.idx[j] != UINT32_MAX) to[s.idx[j]] = static_cast<T>(entry_gradient<FINE>(a, s, have, x, coef, j));
    }
}

// Rows that do not fit the registers: read twice.
template <typename T, bool LOSS, bool GRAD>
__global__ __launch_bounds__(1024) void k_distill_long(const T *z, DistillArgs a, float *loss, float *stats, T *dz) {
    constexpr bool FINE = sizeof(T) == 4;
    constexpr int W = 16;
    __shared__ Message s;
    const int64_t row = blockIdx.x;
    const T *from = z + row * a.ld;
    T *to = dz + row * a.ld;
    const float weight = a.weight ? a.weight[row] : 1.0f;
    int have = 0;
    Softmax x{kNone, 0.0f};
    if (weight != 0.0f) have = teacher<T, W>(a, row, from, s);
    if (have != 0) {
        if (LOSS) {
            for (int64_t c = 8 * threadIdx.x; c < a.V; c += 8 * 64 * W) {
                const f32x8 f = load8(from + c, a.V - c, kNone);
                float top = x.largest;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, f[i]);
                if (top > x.largest) {
                    x.total *= exp_of<FINE>(a, x.largest, top);
                    x.largest = top;
                }
                const float ref = reference(x.largest);
#pragma unroll
                for (int i = 0; i < 8; ++i) x.total += exp_of<FINE>(a, f[i], ref);
            }
            const float mine = x.largest;
            x.largest = group_max<W>(mine, s.slots[2]);
            x.total = group_sum<W>(x.total * exp_of<FINE>(a, mine, reference(x.largest)), s.slots[3]);
            if (x.largest == kNone && x.total == 0.0f) have = 0;
        } else {
            x.largest = stats[2 * row];
            x.total = stats[2 * row + 1];
            if (x.total == 0.0f) have = 0;
        }
    }
    if (LOSS) {
        float value = 0.0f;
        if (have != 0) value = weight * a.T * a.T * loss_of<W>(a, s, x, s.slots[0]);
        if (threadIdx.x == 0) {
            loss[row] = value;
            if (stats) {
                stats[2 * row] = have ? x.largest : 0.0f;
                stats[2 * row + 1] = have ? x.total : 0.0f;
            }
        }
    }
    if (GRAD) {
        const float coef = weight * a.T, over = coef / x.total;
        for (int64_t c = 8 * threadIdx.x; c < a.ld; c += 8 * 64 * W) {
            f32x8 f = 0.0f;
            if (have != 0) {
                f = load8(from + c, a.V - c, kNone);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = c + i < a.V ? exp_of<FINE>(a, f[i], x.largest) * over : 0.0f;
            }
            store8(to + c, a.ld - c, f);
        }
        if (have == 0) return;
        __syncthreads();
        for (int j = threadIdx.x; j < a.k; j += 64 * W)
            if (s.idx[j] != UINT32_MAX) to[s.idx[j]] = static_cast<T>(entry_gradient<FINE>(a, s, have, x, coef, j));
    }
}

// f(W, NV) with the smallest row shape that holds V, or (0, 0).  A lane keeps
// up to 64 registers of logits.
template <typename T, typename F>
void with_shape(int64_t V, F &&f) {
    using std::integral_constant;
    constexpr int MOST = sizeof(T) == 4 ? 8 : 16;
    if (V <= 2048)
        f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (V <= 4096)
        f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    else if (V <= 8192)
        f(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    else if (V <= 512 * 4 * MOST)
        f(integral_constant<int, 4>{}, integral_constant<int, MOST>{});
    else if (V <= 512 * 8 * MOST)
        f(integral_constant<int, 8>{}, integral_constant<int, MOST>{});
    else if (V <= 512 * 16 * MOST)
        f(integral_constant<int, 16>{}, integral_constant<int, MOST>{});
    else
        f(integral_constant<int, 0>{}, integral_constant<int, 0>{});
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
    const DistillArgs a{val, idx, weight, d->vocab, d->ld, d->k, d->temperature, 1.0f / d->temperature,
                        static_cast<float>(1.4426950408889634 / d->temperature)};
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
            const T *from = static_cast<const T *>(z) + r * a.ld;
            T *to = static_cast<T *>(dz) + (GRAD ? r * a.ld : 0);
            float *l = loss ? loss + r : loss, *x = stats ? stats + 2 * r : stats;
            with_shape<T>(a.V, [&](auto w, auto nv) {
                constexpr int W = decltype(w)::value, NV = decltype(nv)::value;
                if constexpr (W == 0)
                    k_distill_long<T, LOSS, GRAD><<<n, 1024, 0, st>>>(from, b, l, x, to);
                else
                    k_distill_row<T, W, NV, LOSS, GRAD><<<n, 64 * W, 0, st>>>(from, b, l, x, to);
            });
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
