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

// exp(x), x = (z - largest) / T, as a power of two.  Of 32-bit logits it carries along
// what the rounding of the exponent's product with log2(e) lost: at an exponent of 2^6
// that is up to 3e-6 of the result.  Of 16-bit logits it does not: the constant and the
// product are off by 2 |x| 2^-24 of the result.  dz has 16 bits and no use for more.  The
// statistics and the loss have 32: their sum is off by the softmax's mean of that, at
// most 2 ln(V) 2^-24 (the mean of |x| is the softmax's entropy less the logarithm of the
// sum, which is 1 or more), 1.4e-6 for 128000 logits that were themselves rounded to
// 2^-12 or 2^-9.
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
    float z[kMostEntries];
    union {
        struct {
            float t[kMostEntries], logt[kMostEntries];
        };
        uint32_t seen[2 * kMostEntries];  // before them: the indices by their hash
    };
    float slots[4][16];
};

// Whether an index comes twice among the message's.  Every thread calls it.
template <int W>
__device__ bool repeats(int k, Message &s) {
    const int bits = 33 - __builtin_clz(k - 1 | 1);  // at least twice k places
    const uint32_t last = (1u << bits) - 1;
    for (uint32_t i = threadIdx.x; i <= last; i += 64 * W) s.seen[i] = UINT32_MAX;
    __syncthreads();
    bool twice = false;
    for (int j = threadIdx.x; j < k; j += 64 * W) {
        const uint32_t i = s.idx[j];
        if (i == UINT32_MAX) continue;
        for (uint32_t h = i * 2654435769u >> (32 - bits);; h = (h + 1) & last) {
            const uint32_t there = atomicCAS(&s.seen[h], UINT32_MAX, i);
            twice |= there == i;
            if (there == i || there == UINT32_MAX) break;
        }
    }
    return __syncthreads_or(twice) != 0;
}

// Reads a message and the student's logits at its entries (those that lie in
// columns [begin, end), or all of them from `gathered`), and makes t and log t.
// Every thread of the workgroup calls it.  Returns 0 if no entry counts, 2 if an
// index may come twice (of interest for GRAD), else 1: at once if they ascend,
// otherwise by their hash.  Loss and gradient of 4096 x 2000 bf16 logits with
// messages in no order, of 16 entries 15.5 us where each entry looks at all
// others and 16.4 with a hash; of 64 19.9 and 17.0, of 256 49 and 20.8, of 1024
// 551 and 35.6.
constexpr int kLookAtAll = 32;
template <typename T, int W, bool GRAD>
__device__ int teacher(const DistillArgs &a, int64_t row, const T *z, const float *gathered, int64_t begin, int64_t end,
                       Message &s) {
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
        if (gathered)
            s.z[j] = gathered[j];
        else if (i >= begin && i < end)
            s.z[j] = static_cast<float>(z[i]);
    }
    have = (__syncthreads_or(have & 1) ? 1 : 0) | (__syncthreads_or(have & 2) ? 2 : 0);
    bool twice = have == 3;
    if (GRAD && twice && a.k > kLookAtAll) {
        twice = repeats<W>(a.k, s);
        for (int j = threadIdx.x; j < a.k; j += 64 * W) s.t[j] = val[j];
    }
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
    return (have & 1) == 0 ? 0 : twice ? 2 : 1;
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

// NV vectors of 16 bytes per lane of a row's columns [0, V) in registers, NL more in
// LDS (`held`, kHeld of all lanes together, each used by its own lane only), and the
// last V % kPer columns one each in the first lanes.  Vectors beyond the row are -inf.
constexpr int kHeld = 4032;
template <typename T, int W, int NV, int NL, bool STREAM>
struct Logits {
    typedef typename Vec16<T>::type Raw;
    typedef typename Vec16<T>::packed Packed;
    typedef typename Vec16<T>::wide Wide;
    static constexpr int kPer = Vec16<T>::kPer;
    static constexpr bool FINE = sizeof(T) == 4;
    Raw raw[NV];
    float last;

    static __device__ __forceinline__ int at(int v) { return static_cast<int>(threadIdx.x) + 64 * W * v; }
    template <int FROM, int UPTO>
    __device__ __forceinline__ void load_part(const T *from, int vectors, Raw *to) {
#pragma unroll
        for (int v = FROM; v < UPTO; ++v) {
            if (at(v) < vectors) {
                const Packed *p = reinterpret_cast<const Packed *>(from) + at(v);
                to[v - FROM] = STREAM ? __builtin_nontemporal_load(p) : *p;
            } else {
                to[v - FROM] = static_cast<T>(kNone);
            }
        }
    }
    __device__ __forceinline__ void load(const T *from, int vectors, int rest, Raw *held) {
        if constexpr (NL == 0) {
            load_part<0, NV>(from, vectors, raw);
        } else {
            // as many as fit at a time: the first ones go to LDS as soon as they are here
            Raw first[NL];
            load_part<NV, NV + NL>(from, vectors, first);
            load_part<0, NV - NL>(from, vectors, raw);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int v = 0; v < NL; ++v)
                if (at(NV + v) < vectors) held[at(v)] = first[v];
            __builtin_amdgcn_sched_barrier(0);
            load_part<NV - NL, NV>(from, vectors, raw + NV - NL);
        }
        last = static_cast<int>(threadIdx.x) < rest ? static_cast<float>(from[kPer * vectors + threadIdx.x]) : kNone;
    }
    __device__ __forceinline__ static float most(Raw r, float top) {
        const Wide f = __builtin_convertvector(r, Wide);
#pragma unroll
        for (int i = 0; i < kPer; ++i) top = fmaxf(top, f[i]);
        return top;
    }
    __device__ __forceinline__ float largest(int vectors, const Raw *held) const {
        float top = last;
#pragma unroll
        for (int v = 0; v < NV; ++v) top = most(raw[v], top);
#pragma unroll
        for (int v = 0; v < NL; ++v)
            if (at(NV + v) < vectors) top = most(held[at(v)], top);
        return top;
    }
    __device__ __forceinline__ static float add(const DistillArgs &a, Raw r, float ref, float sum) {
        const Wide f = __builtin_convertvector(r, Wide);
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += exp_of<FINE>(a, f[i], ref);
        return sum;
    }
    __device__ __forceinline__ float sum(const DistillArgs &a, float ref, int vectors, const Raw *held) {
        float sum = exp_of<FINE>(a, last, ref);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            forget(raw[v]);
            sum = add(a, raw[v], ref, sum);
        }
#pragma unroll
        for (int v = 0; v < NL; ++v)
            if (at(NV + v) < vectors) sum = add(a, held[at(v)], ref, sum);
        return sum;
    }
    // s * over
    __device__ __forceinline__ static void put(const DistillArgs &a, Raw r, float largest, float over, T *to, int q) {
        Wide f = __builtin_convertvector(r, Wide);
#pragma unroll
        for (int i = 0; i < kPer; ++i) f[i] = exp_of<FINE>(a, f[i], largest) * over;
        Packed *p = reinterpret_cast<Packed *>(to) + q;
        r = __builtin_convertvector(f, Raw);
        if (STREAM)
            __builtin_nontemporal_store(r, p);
        else
            *p = r;
    }
    __device__ __forceinline__ void gradient(const DistillArgs &a, float largest, float over, T *to, int vectors, int rest,
                                             const Raw *held) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            forget(raw[v]);
            if (at(v) < vectors) put(a, raw[v], largest, over, to, at(v));
        }
#pragma unroll
        for (int v = 0; v < NL; ++v)
            if (at(NV + v) < vectors) put(a, held[at(v)], largest, over, to, at(NV + v));
        if (static_cast<int>(threadIdx.x) < rest)
            to[kPer * vectors + threadIdx.x] = static_cast<T>(exp_of<FINE>(a, last, largest) * over);
    }
};

// Zeros of columns [begin, end) of a row.
template <typename T, int W>
__device__ void clear(T *to, int64_t begin, int64_t end) {
    for (int64_t c = begin + 8 * threadIdx.x; c < end; c += 8 * 64 * W) store8(to + c, end - c, f32x8(0.0f));
}

// Vectors per lane of a 16-wave workgroup that leave room for a second one on its
// CU, at 64 registers a lane (loss and gradient of 4096 x 80000 bf16 logits 233 us,
// 333 with one of 16 vectors; the loss 130 and 228), and how many more fit half a
// CU's LDS beside the message (4096 x 128000: 380 us, 429 with one workgroup of 16
// vectors; the loss 182 and 250).
constexpr int kTwoVectors = 12, kTwoHeld = 4;

// One workgroup per token, whose logits stay in registers between the
// statistics and the gradient, so that z is read once: largest logit, sum of the
// exponentials, then dz from the same registers; the message's entries are written
// over it last.  LOSS: the statistics and the loss; GRAD: dz, from the statistics
// just made or (LOSS not) from `stats`.  Bound by memory: loss and gradient of 4096
// x 32000 bf16 logits (528 MB) 102 us, 5.2 TB/s; of 8192 x 128000 (4.2 GB) 823, 5.1;
// the gradient of 3108 x 30011 f16 72 us.  What keeps it from a copy's 6.1 is that a
// workgroup first only reads, then computes, then only writes, and what overlaps is
// the others on its CU; one workgroup a CU that asks for the next row meanwhile was
// slower than two that do not.
template <typename T, int W, int NV, int NL, bool LOSS, bool GRAD, bool STREAM>
__global__ __launch_bounds__(64 * W, NV == kTwoVectors ? 8 : 1) void k_distill_row(const T *z, DistillArgs a, float *loss,
                                                                                   float *stats, T *dz) {
    constexpr bool FINE = sizeof(T) == 4;
    constexpr int kPer = Vec16<T>::kPer;
    __shared__ Message s;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const T *from = z + row * a.ld;
    T *to = dz + row * a.ld;
    const float weight = a.weight ? a.weight[row] : 1.0f;
    const int vectors = static_cast<int>(a.V / kPer), rest = static_cast<int>(a.V % kPer);
    int have = 0;
    Softmax x{0.0f, 0.0f};
    Logits<T, W, NV, NL, STREAM> l;
    __shared__ typename Vec16<T>::type held[NL > 0 ? kHeld : 1];
    if (weight != 0.0f) {
        l.load(from, vectors, rest, held);
        have = teacher<T, W, GRAD>(a, row, from, nullptr, 0, a.V, s);
    }
    if (have != 0) {
        if (LOSS) {
            x.largest = group_max<W>(l.largest(vectors, held), s.slots[2]);
            x.total = group_sum<W>(l.sum(a, reference(x.largest), vectors, held), s.slots[3]);
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
            clear<T, W>(to, 0, a.ld);
            return;
        }
        const float coef = weight * a.T, over = coef / x.total;
        l.gradient(a, x.largest, over, to, vectors, rest, held);
        clear<T, W>(to, a.V, a.ld);
        // Entries come after their vectors, streamed ones too: stores of a workgroup's
        // waves to one address stay in the order that a barrier gives them, as they
        // leave through one compute unit's cache.
        __syncthreads();
        for (int j = tid; j < a.k; j += 64 * W)
            if (s.idx[j] != UINT32_MAX) to[s.idx[j]] = static_cast<T>(entry_gradient<FINE>(a, s, have, x, coef, j));
    }
}

// Few tokens or very long rows: a row's columns are shared out in slices of kSlice
// elements, one workgroup each, first for the statistics, then for loss and dz.
constexpr int kSliceVectors = 4;
template <typename T>
constexpr int kSlice = 64 * 4 * kSliceVectors * Vec16<T>::kPer;

// Statistics of one slice, and the student's logits at the message's entries
// (before dz, which may be z, is written).
template <typename T>
__global__ __launch_bounds__(256) void k_distill_part(const T *z, DistillArgs a, Softmax *part, float *gathered) {
    __shared__ float slots[2][4];
    const int64_t row = blockIdx.y, begin = static_cast<int64_t>(blockIdx.x) * kSlice<T>;
    if (a.weight && a.weight[row] == 0.0f) return;
    const int64_t n = a.V - begin < kSlice<T> ? a.V - begin : kSlice<T>;
    const T *from = z + row * a.ld;
    Logits<T, 4, kSliceVectors, 0, false> l;
    l.load(from + begin, static_cast<int>(n / Vec16<T>::kPer), static_cast<int>(n % Vec16<T>::kPer), nullptr);
    for (int64_t j = blockIdx.x * 256 + threadIdx.x; j < a.k; j += 256 * gridDim.x) {
        const uint32_t i = a.idx[row * a.k + j];
        if (i < a.V) gathered[row * a.k + j] = static_cast<float>(from[i]);
    }
    const float largest = group_max<4>(l.largest(0, nullptr), slots[0]);
    const float total = group_sum<4>(l.sum(a, reference(largest), 0, nullptr), slots[1]);
    if (threadIdx.x == 0) part[row * gridDim.x + blockIdx.x] = Softmax{largest, total};
}

// LOSS: joins the slices' statistics; the first slice's workgroup writes them
// and the loss.  GRAD: dz of one slice.
template <typename T, bool LOSS, bool GRAD>
__global__ __launch_bounds__(256) void k_distill_slice(const T *z, DistillArgs a, int slices, const Softmax *part,
                                                       const float *gathered, float *loss, float *stats, T *dz) {
    constexpr bool FINE = sizeof(T) == 4;
    __shared__ Message s;
    const int64_t row = blockIdx.y, begin = static_cast<int64_t>(blockIdx.x) * kSlice<T>;
    const int64_t n = a.V - begin < kSlice<T> ? a.V - begin : kSlice<T>;
    const int vectors = static_cast<int>(n / Vec16<T>::kPer), rest = static_cast<int>(n % Vec16<T>::kPer);
    const int tid = threadIdx.x;
    const T *from = z + row * a.ld;
    T *to = dz + row * a.ld;
    const float weight = a.weight ? a.weight[row] : 1.0f;
    int have = 0;
    Softmax x{0.0f, 0.0f};
    Logits<T, 4, kSliceVectors, 0, false> l;
    if (weight != 0.0f) {
        if (GRAD) l.load(from + begin, vectors, rest, nullptr);
        have = teacher<T, 4, GRAD>(a, row, from, LOSS ? gathered + row * a.k : nullptr, begin, begin + n, s);
    }
    if (have != 0) {
        if (LOSS) {
            const Softmax *p = part + row * slices;
            float top = kNone, sum = 0.0f;
            for (int i = tid; i < slices; i += 256) top = fmaxf(top, p[i].largest);
            x.largest = group_max<4>(top, s.slots[2]);
            for (int i = tid; i < slices; i += 256)
                sum += p[i].total * exp_of<FINE>(a, p[i].largest, reference(x.largest));
            x.total = group_sum<4>(sum, s.slots[3]);
            if (x.largest == kNone && x.total == 0.0f) have = 0;
        } else {
            x.largest = stats[2 * row];
            x.total = stats[2 * row + 1];
            if (x.total == 0.0f) have = 0;
        }
    }
    if (LOSS && blockIdx.x == 0) {
        float value = 0.0f;
        if (have != 0) value = weight * a.T * a.T * loss_of<4>(a, s, x, s.slots[0]);
        if (tid == 0) {
            loss[row] = value;
            if (stats) {
                stats[2 * row] = have ? x.largest : 0.0f;
                stats[2 * row + 1] = have ? x.total : 0.0f;
            }
        }
    }
    if (GRAD) {
        if (begin + n == a.V) clear<T, 4>(to, a.V, a.ld);
        if (have == 0) {
            clear<T, 4>(to, begin, begin + n);
            return;
        }
        const float coef = weight * a.T, over = coef / x.total;
        l.gradient(a, x.largest, over, to + begin, vectors, rest, nullptr);
        __syncthreads();
        for (int j = tid; j < a.k; j += 256) {
            const uint32_t i = s.idx[j];
            if (i != UINT32_MAX && i >= begin && i < begin + n)
                to[i] = static_cast<T>(entry_gradient<FINE>(a, s, have, x, coef, j));
        }
    }
}

// f(W, NV, NL) with the smallest row shape that holds `bytes` (up to kRowMost).  A
// lane keeps up to 64 registers of logits.
constexpr int64_t kTwoRows = 16 * 64 * 16 * kTwoVectors, kRowMost = kTwoRows + 16 * kHeld, kRowFewer = 131072, kFewRows = 128;
template <int N>
using Int = std::integral_constant<int, N>;
template <typename F>
void with_shape(int64_t bytes, F &&f) {
    if (bytes <= 4096)
        f(Int<4>{}, Int<1>{}, Int<0>{});
    else if (bytes <= 8192)
        f(Int<4>{}, Int<2>{}, Int<0>{});
    else if (bytes <= 16384)
        f(Int<4>{}, Int<4>{}, Int<0>{});
    else if (bytes <= 32768)
        f(Int<4>{}, Int<8>{}, Int<0>{});
    else if (bytes <= 65536)
        f(Int<4>{}, Int<16>{}, Int<0>{});
    else if (bytes <= 131072)
        f(Int<8>{}, Int<16>{}, Int<0>{});
    else if (bytes <= kTwoRows)
        f(Int<16>{}, Int<kTwoVectors>{}, Int<0>{});
    else
        f(Int<16>{}, Int<kTwoVectors>{}, Int<kTwoHeld>{});
}

// Rows are shared out in slices
//  - where a row does not fit a workgroup's registers;
//  - where it takes half a CU or more and there are so few that most CUs would have
//    none: loss and gradient of 64 rows of 128000 bf16 logits 15 us in slices and
//    21 by rows, of 128 rows of 80000 16 and 18, of 256 26 and 22.
// The rule does not ask whether the gradient is wanted too, so that the loss has the
// same bits with it and without.
bool split(int64_t rows, int64_t bytes) { return bytes > kRowMost || (bytes > kRowFewer && rows <= kFewRows); }
int64_t slices_of(int64_t bytes) { return ceil_div(bytes, 64 * 4 * kSliceVectors * 16); }

// Whether long rows (12 or 16 vectors a lane) pass by the caches: loss and gradient
// of 60 MB of bf16 logits, read and written, the same; of 120 MB, rows of 32000 29.8
// us so and 35.6 not, of 128000 31.5 and 37.3; 1 GB 195 / 213 and 201 / 218.  Beyond,
// rows of more than 64 KB that begin at lines of 128 bytes gain (128000: 2 GB 373 /
// 399, 4 GB 751 / 764), others lose (98000: 2 GB 420 / 413, 4 GB 844 / 797; 32000: 2 GB
// 416 / 411).  Entries are written into the row once more: not if there are as
// many as lines (526 MB of 32000, 256 entries 117 / 137, 1024 233 / 170).
constexpr double kStreamFrom = 64e6, kStreamUpTo = 1.4e9;
bool streams(int64_t rows, const dqgan_distill_desc *d, int64_t bytes) {
    if (d->k > bytes / 128) return false;
    const bool lines = bytes > 65536 && d->ld * (bytes / d->vocab) % 128 == 0;
    const double total = 2.0 * static_cast<double>(rows) * static_cast<double>(bytes);
    return total >= kStreamFrom && (lines || total <= kStreamUpTo);
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

size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

// Slices' statistics, then the student's logits at the entries.
size_t part_bytes(int64_t rows, int64_t row_bytes) {
    return round256(sizeof(Softmax) * static_cast<size_t>(rows * slices_of(row_bytes)));
}
int64_t row_bytes_of(const dqgan_distill_desc *d) { return d->vocab * (d->type == DQGAN_F32 ? 4 : 2); }

DistillArgs from_row(DistillArgs a, int64_t r) {
    a.val += r * a.k;
    a.idx += r * a.k;
    if (a.weight) a.weight += r;
    return a;
}

template <bool LOSS, bool GRAD>
dqgan_status run(dqgan_plan P, const dqgan_distill_desc *d, const void *z, const float *val, const uint32_t *idx,
                 const float *weight, float *loss, float *stats, void *dz, void *workspace, hipStream_t st) {
    const DistillArgs a{val, idx, weight, d->vocab, d->ld, d->k, d->temperature, 1.0f / d->temperature,
                        static_cast<float>(1.4426950408889634 / d->temperature)};
    const int64_t rows = d->tokens * P->desc.M, bytes = row_bytes_of(d);
    if (split(rows, bytes)) {
        const uint32_t slices = static_cast<uint32_t>(slices_of(bytes));
        Softmax *part = static_cast<Softmax *>(workspace);
        float *gathered = reinterpret_cast<float *>(static_cast<char *>(workspace) + part_bytes(rows, bytes));
        for (int64_t r = 0; r < rows; r += 65535) {  // a launch's most in the second dimension
            const uint32_t n = static_cast<uint32_t>(rows - r < 65535 ? rows - r : 65535);
            const DistillArgs b = from_row(a, r);
            with_type(d->type, [&](auto t) {
                using T = decltype(t);
                const T *from = static_cast<const T *>(z) + r * a.ld;
                if (LOSS) k_distill_part<T><<<dim3(slices, n), 256, 0, st>>>(from, b, part + r * slices, gathered + r * a.k);
                k_distill_slice<T, LOSS, GRAD><<<dim3(GRAD ? slices : 1, n), 256, 0, st>>>(
                    from, b, static_cast<int>(slices), part + r * slices, gathered + r * a.k, LOSS ? loss + r : nullptr,
                    stats ? stats + 2 * r : stats, static_cast<T *>(dz) + (GRAD ? r * a.ld : 0));
            });
        }
        return launched();
    }
    // a launch has fewer than 2^32 threads
    constexpr int64_t kMost = int64_t(1) << 21;
    for (int64_t r = 0; r < rows; r += kMost) {
        const uint32_t n = static_cast<uint32_t>(rows - r < kMost ? rows - r : kMost);
        const DistillArgs b = from_row(a, r);
        with_type(d->type, [&](auto t) {
            using T = decltype(t);
            const T *from = static_cast<const T *>(z) + r * a.ld;
            T *to = static_cast<T *>(dz) + (GRAD ? r * a.ld : 0);
            float *l = loss ? loss + r : loss, *x = stats ? stats + 2 * r : stats;
            with_shape(bytes, [&](auto w, auto nv, auto nl) {
                constexpr int W = decltype(w)::value, NV = decltype(nv)::value, NL = decltype(nl)::value;
                if (GRAD && NV >= kTwoVectors && streams(rows, d, bytes))
                    k_distill_row<T, W, NV, NL, LOSS, GRAD, GRAD && NV >= kTwoVectors><<<n, 64 * W, 0, st>>>(from, b, l, x, to);
                else
                    k_distill_row<T, W, NV, NL, LOSS, GRAD, false><<<n, 64 * W, 0, st>>>(from, b, l, x, to);
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
    DQ_TRY(check_ptr(workspace, any && split(d->tokens * P->desc.M, row_bytes_of(d))));
    DQ_TRY(check_device(P));
    if (!any) return DQGAN_OK;
    return run<true, false>(P, d, z, val, idx, weight, loss, stats, nullptr, workspace,
                            static_cast<hipStream_t>(stream));
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
    return run<false, true>(P, d, z, val, idx, weight, nullptr, const_cast<float *>(stats), dz, nullptr,
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
    DQ_TRY(check_ptr(workspace, any && split(d->tokens * P->desc.M, row_bytes_of(d))));
    DQ_TRY(check_device(P));
    if (!any) return DQGAN_OK;
    return run<true, true>(P, d, z, val, idx, weight, loss, nullptr, dz, workspace,
                           static_cast<hipStream_t>(stream));
}

dqgan_status dqgan_distill_bytes(dqgan_plan P, const dqgan_distill_desc *d, size_t *bytes) {
    DQ_TRY(check(P, d));
    if (!bytes) return DQGAN_EINVAL;
    const int64_t rows = d->tokens * P->desc.M, row = row_bytes_of(d);
    *bytes = rows > 0 && split(rows, row) ? part_bytes(rows, row) + sizeof(float) * static_cast<size_t>(rows * d->k) : 0;
    return DQGAN_OK;
}

}  // extern "C"
