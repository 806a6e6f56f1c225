// Layer norm of M workers, each with its own weight and bias in its row of P,
// and its gradients, those of weight and bias in the worker's row of G.
#include "layers.hpp"

namespace dq {
namespace {

// Row shapes: L lanes of a wave, or W whole waves, and NV vectors of 16 bytes per
// lane, so that a row stays in registers between the statistics and their use.
// Elements beyond the last whole vector, and beyond NV vectors a lane, lie one each
// in the row's first lanes.
template <int L, int W, int NV>
struct Shape {
    static constexpr int kLanes = W == 1 ? L : 64 * W, kThreads = W < 4 ? 256 : 64 * W, kRows = kThreads / kLanes;
    // Backward: workgroups of all workers together, and the least rows of one where
    // there are many, so that the partial sums are a fraction of what is read.  With
    // 2048, 1024 and 512 workgroups rows of 64 bf16 elements (206 MB) take 55, 57 and
    // 81 us, of 2048 (806 MB) 172, 173 and 188, of 4096 (806 MB) 175, 167 and 155.
    static constexpr int kGroups = W == 1 ? 2048 : W * NV <= 4 ? 1024 : 512, kLeast = W == 1 ? 32 : 8;
    // A row's vectors, and whether the rest fits one element a lane.
    template <typename T>
    static __host__ __device__ __forceinline__ int vectors(int64_t D) {
        return static_cast<int>(D / Vec16<T>::kPer < kLanes * NV ? D / Vec16<T>::kPer : kLanes * NV);
    }
    template <typename T>
    static bool holds(int64_t D) {
        return D <= static_cast<int64_t>(kLanes) * (NV * Vec16<T>::kPer + 1);
    }
    static constexpr int kVectors = NV, kPerWave = W == 1 ? 64 / L : 1;  // rows a wave holds
    // The first row of this wave's, in a scalar register: a loop over it keeps one
    // set of sums.
    static __device__ __forceinline__ int64_t first_row() {
        return static_cast<int64_t>(blockIdx.x) * kRows +
               (W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kPerWave : 0);
    }
    // Whether any lane of this wave has a vector v of a row; the same for the wave.
    static __device__ __forceinline__ bool any(int v, int vectors) {
        return (W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 64) + kLanes * v < vectors;
    }
    static __device__ __forceinline__ int row_of_wave() { return kPerWave == 1 ? 0 : (threadIdx.x & 63) / L; }
    // sums over a row's lanes; `slot`: W floats of LDS per value
    static __device__ __forceinline__ float sum(float x, float *slot) {
        if (W > 1) return group_sum<W>(x, slot);
        return L == 16 ? lanes_sum<16>(x) : wave_sum(x);
    }
    static __device__ __forceinline__ float2 sums(float x, float y, float *slot) {
        if (W == 1) return make_float2(sum(x, slot), sum(y, slot));
        x = wave_sum(x);
        y = wave_sum(y);
        if ((threadIdx.x & 63) == 0) {
            slot[threadIdx.x >> 6] = x;
            slot[W + (threadIdx.x >> 6)] = y;
        }
        __syncthreads();
        return make_float2(lanes_sum<W>(slot[threadIdx.x & (W - 1)]), lanes_sum<W>(slot[W + (threadIdx.x & (W - 1))]));
    }
};

struct NormArgs {
    const float *P;
    int64_t ldp;
    int64_t gamma, beta;  // -1: none
    int64_t D, N;
    float eps;
};

// Element i of a row whose start is the same in every lane: an address of a
// scalar and a 32-bit part.
template <typename T>
__device__ __forceinline__ T *at(T *row, int i) {
    return (T *)((const char *)row + static_cast<uint32_t>(i) * static_cast<uint32_t>(sizeof(T)));
}

// A lane's elements of a row, as they lie in memory; beyond the row its last ones
// once more, so that loads need no branch.
template <typename T, typename S, bool STREAM>
struct Row {
    typename Vec16<T>::type raw[S::kVectors];
    typename Bits<T>::type last;
    __device__ __forceinline__ void load(const T *p, int lane, int vectors, int rest) {
        if (vectors > 0) {
#pragma unroll
            for (int v = 0; v < S::kVectors; ++v) {
                if (!S::any(v, vectors)) break;
                const int q = lane + S::kLanes * v;
                raw[v] = load16<T, STREAM>(at(p, Vec16<T>::kPer * (q < vectors ? q : vectors - 1)));
            }
        }
        if (rest > 0) last = load_bits(at(p, Vec16<T>::kPer * vectors + (lane < rest ? lane : 0)));
    }
};
// ... and of a parameter's row.
template <typename T, typename S>
struct Params {
    typename Vec16<T>::wide of[S::kVectors];
    float last;
    __device__ __forceinline__ void load(const float *p, float none, bool there, int lane, int vectors, int rest) {
        last = none;
#pragma unroll
        for (int v = 0; v < S::kVectors; ++v) of[v] = none;
        if (!there) return;
#pragma unroll
        for (int v = 0; v < S::kVectors; ++v)
            if (lane + S::kLanes * v < vectors) of[v] = load_floats<T>(p + Vec16<T>::kPer * (lane + S::kLanes * v));
        if (lane < rest) last = p[Vec16<T>::kPer * vectors + lane];
    }
};

// What y is made of.  The mean in binary32 is off by some units of its last place,
// which matters to rows that lie far from zero for their deviation: of 1000 elements
// about 10^4 with a deviation of 0.01 the variance would be off by 0.3 % and y by
// 0.05.  Such rows (the mean above eight deviations) take the mean r of x - mean too,
// and y and the variance about mean + r: off by 1e-7 and 3e-7.  Of the others y is off
// by at most 8 (depth of the sum) 2^-24 for it, and they cost one comparison (8 x 4000
// rows of 9000 bf16 262 us; without r 254, with r for all rows 279; 32 x 16384 of 64
// with one row in a hundred far 29, 28 and 31, with none 26.9 and 26.1).
constexpr float kFar = 64.0f;  // the square of eight
struct Centre {
    float var, rstd, r = 0.0f, shift = 0.0f;
    bool far;
    __device__ __forceinline__ Centre(float mean, float squares, float eps)
        : var(squares), rstd(1.0f / sqrtf(squares + eps)), far(mean * mean > kFar * (squares + eps)) {}
    __device__ __forceinline__ void correct(float rest, float eps) {
        r = rest;
        const float v = fmaf(-r, r, var);
        rstd = 1.0f / sqrtf((v < 0.0f ? 0.0f : v) + eps);  // just below 0: equal elements
        shift = -r * rstd;
    }
    // of an element from which the computed mean has been taken
    __device__ __forceinline__ float normal(float f) const { return fmaf(f, rstd, shift); }
};

// Two passes over the registers: the mean, then the mean square of what is
// left.  Bound by memory: 8 x
// 8192 rows of 2048 bf16 (537 MB) 95 us, 5.7 TB/s of the 6.1 of a large copy; few
// rows are one launch and two sums over a wave, 2.7 us.
template <typename T, typename S, bool STREAM>
__global__ __launch_bounds__(S::kThreads) void k_norm_fwd(const T *x, NormArgs a, T *y, float *stats) {
    constexpr int kPer = Vec16<T>::kPer, NV = S::kVectors;
    typedef typename Vec16<T>::wide Wide;
    __shared__ float slots[3][16];
    const int lane = threadIdx.x % S::kLanes;
    const int64_t m = blockIdx.y, D = a.D;
    const int vectors = S::template vectors<T>(D), rest = static_cast<int>(D) - kPer * vectors;
    Params<T, S> g, b;
    g.load(a.P + m * a.ldp + a.gamma, 1.0f, a.gamma >= 0, lane, vectors, rest);
    b.load(a.P + m * a.ldp + a.beta, 0.0f, a.beta >= 0, lane, vectors, rest);
    const float inv = 1.0f / static_cast<float>(D);
    const int64_t step = static_cast<int64_t>(gridDim.x) * S::kRows;
    for (int64_t first = S::first_row(); first < a.N; first += step) {
        const bool in = first + S::row_of_wave() < a.N;
        const int64_t n = in ? first + S::row_of_wave() : a.N - 1;
        Row<T, S, false> row;
        row.load(x + (m * a.N + n) * D, lane, vectors, rest);
        Wide f[NV];
        float last = lane < rest ? widen_bits<T>(row.last) : 0.0f, s = last;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!S::any(v, vectors)) break;
            f[v] = widen<T>(row.raw[v]);
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) part += f[v][i];
            s += lane + S::kLanes * v < vectors ? part : 0.0f;
        }
        const float mean = S::sum(s, slots[0]) * inv;
        last -= mean;
        s = lane < rest ? last * last : 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!S::any(v, vectors)) break;
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                f[v][i] -= mean;
                part = fmaf(f[v][i], f[v][i], part);
            }
            s += lane + S::kLanes * v < vectors ? part : 0.0f;
        }
        Centre centre(mean, S::sum(s, slots[1]) * inv, a.eps);
        if (__any(centre.far)) {  // of one row for all waves, or of this wave's rows
            s = lane < rest ? last : 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!S::any(v, vectors)) break;
                float part = 0.0f;
#pragma unroll
                for (int i = 0; i < kPer; ++i) part += f[v][i];
                s += lane + S::kLanes * v < vectors ? part : 0.0f;
            }
            const float r = S::sum(s, slots[2]) * inv;
            if (centre.far) centre.correct(r, a.eps);
        }
        T *out = y + (m * a.N + n) * D;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!S::any(v, vectors)) break;
            const int q = lane + S::kLanes * v;
#pragma unroll
            for (int i = 0; i < kPer; ++i) f[v][i] = fmaf(centre.normal(f[v][i]), g.of[v][i], b.of[v][i]);
            if (q < vectors && in) store16<T, STREAM>(at(out, kPer * q), narrow<T>(f[v]));
        }
        if (lane < rest && in) *at(out, kPer * vectors + lane) = static_cast<T>(fmaf(centre.normal(last), g.last, b.last));
        if (stats && lane == 0 && in) {
            stats[2 * (m * a.N + n)] = mean + centre.r;
            stats[2 * (m * a.N + n) + 1] = centre.rstd;
        }
    }
}

// Rows that do not fit the registers: read three times, four if far from zero.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_fwd_long(const T *x, NormArgs a, T *y, float *stats) {
    __shared__ float slots[3][16];
    const int64_t m = blockIdx.y, D = a.D;
    const float inv = 1.0f / static_cast<float>(D);
    for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
        const T *row = x + (m * a.N + n) * D;
        float s = 0.0f;
        for (int64_t c = 8 * threadIdx.x; c < D; c += 8192) {
            const f32x8 f = load8(row + c, D - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += f[i];
        }
        const float mean = group_sum<16>(s, slots[0]) * inv;
        s = 0.0f;
        for (int64_t c = 8 * threadIdx.x; c < D; c += 8192) {
            const f32x8 f = load8(row + c, D - c, mean);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(f[i] - mean, f[i] - mean, s);
        }
        Centre centre(mean, group_sum<16>(s, slots[1]) * inv, a.eps);
        if (centre.far) {  // the same for all waves
            s = 0.0f;
            for (int64_t c = 8 * threadIdx.x; c < D; c += 8192) {
                const f32x8 f = load8(row + c, D - c, mean);
#pragma unroll
                for (int i = 0; i < 8; ++i) s += f[i] - mean;
            }
            centre.correct(group_sum<16>(s, slots[2]) * inv, a.eps);
        }
        T *out = y + (m * a.N + n) * D;
        for (int64_t c = 8 * threadIdx.x; c < D; c += 8192) {
            f32x8 f = load8(row + c, D - c), g = 1.0f, b = 0.0f;
            if (a.gamma >= 0) g = load8(a.P + m * a.ldp + a.gamma + c, D - c);
            if (a.beta >= 0) b = load8(a.P + m * a.ldp + a.beta + c, D - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = fmaf(centre.normal(f[i] - mean), g[i], b[i]);
            store8(out + c, D - c, f);
        }
        if (stats && threadIdx.x == 0) {
            stats[2 * (m * a.N + n)] = mean + centre.r;
            stats[2 * (m * a.N + n) + 1] = centre.rstd;
        }
    }
}

// Where the columns' sums go: to part[m][share][2][D], or, of one workgroup per
// worker, to G.  Neither: not wanted.
struct Sums {
    float *part, *G;
    int64_t ld;
    bool add;
};

// One workgroup takes every gridDim.x-th group of rows of its worker and keeps
// its columns' sums of dy and dy * xh in registers meanwhile: x and dy are read once
// for all three results.  8 x
// 2048 rows of 1024 bf16 (101 MB) 20.8 us, and k_norm_params 3.9; 3 x 1111 rows of
// 4801 f16 (96 MB, and 16 MB of sums written and read) 27.5 and 5.1: a row's two sums over the
// workgroup come between its loads and its stores, and loads of the next row ahead
// of them were no faster.
template <typename T, typename S, int STREAM>
__global__ __launch_bounds__(S::kThreads, S::kVectors < 3 || S::kThreads > 256 ? 4 : 2) void k_norm_bwd(
    const T *x, const T *dy, NormArgs a, const float *stats, T *dx, Sums out) {
    constexpr int kPer = Vec16<T>::kPer, NV = S::kVectors;
    typedef typename Vec16<T>::wide Wide;
    __shared__ float slots[2][2 * 16];
    const int lane = threadIdx.x % S::kLanes;
    const int64_t m = blockIdx.y, D = a.D;
    const int vectors = S::template vectors<T>(D), rest = static_cast<int>(D) - kPer * vectors;
    Params<T, S> g;
    g.load(a.P + m * a.ldp + a.gamma, 1.0f, a.gamma >= 0, lane, vectors, rest);
    Wide sg[NV], sb[NV];
    float last_sg = 0.0f, last_sb = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        sg[v] = 0.0f;
        sb[v] = 0.0f;
    }
    const float inv = 1.0f / static_cast<float>(D);
    const int64_t step = static_cast<int64_t>(gridDim.x) * S::kRows;
    int turn = 0;
    for (int64_t first = S::first_row(); first < a.N; first += step, turn ^= 1) {
        const bool in = first + S::row_of_wave() < a.N;
        const int64_t n = in ? first + S::row_of_wave() : a.N - 1;
        const float2 st = reinterpret_cast<const float2 *>(stats)[m * a.N + n];
        Row<T, S, (STREAM > 1)> rx, ry;
        rx.load(x + (m * a.N + n) * D, lane, vectors, rest);
        ry.load(dy + (m * a.N + n) * D, lane, vectors, rest);
        const float mean = st.x, rstd = st.y;
        const float last_xh = lane < rest ? (widen_bits<T>(rx.last) - mean) * rstd : 0.0f;
        float last_u = lane < rest && in ? widen_bits<T>(ry.last) : 0.0f;
        last_sg = fmaf(last_u, last_xh, last_sg);
        last_sb += last_u;
        last_u *= g.last;
        float s1 = last_u, s2 = last_u * last_xh;
#pragma unroll
        for (int v = 0; v < NV; ++v) {  // sg and sb of lanes beyond the row are not stored
            if (!S::any(v, vectors)) break;
            const Wide xv = widen<T>(rx.raw[v]);
            Wide yv = widen<T>(ry.raw[v]);
            if (S::kPerWave > 1 && !in) yv = 0.0f;
            float p1 = 0.0f, p2 = 0.0f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const float xh = (xv[i] - mean) * rstd, u = yv[i] * g.of[v][i];
                sg[v][i] = fmaf(yv[i], xh, sg[v][i]);
                sb[v][i] += yv[i];
                p1 += u;
                p2 = fmaf(u, xh, p2);
            }
            s1 += lane + S::kLanes * v < vectors ? p1 : 0.0f;
            s2 += lane + S::kLanes * v < vectors ? p2 : 0.0f;
            settle(sg[v]);  // one vector's temporaries at a time
            settle(sb[v]);
            asm volatile("" : "+v"(s1), "+v"(s2));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (dx) {
            const float2 c = S::sums(s1, s2, slots[turn]);
            const float c1 = c.x * inv, c2 = c.y * inv;
            T *out = dx + (m * a.N + n) * D;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!S::any(v, vectors)) break;
                const int q = lane + S::kLanes * v;
                forget(rx.raw[v]);
                forget(ry.raw[v]);
                const Wide xv = widen<T>(rx.raw[v]), yv = widen<T>(ry.raw[v]);
                Wide d;
#pragma unroll
                for (int i = 0; i < kPer; ++i) d[i] = rstd * (yv[i] * g.of[v][i] - c1 - (xv[i] - mean) * rstd * c2);
                if (q < vectors && in) store16<T, (STREAM > 0)>(at(out, kPer * q), narrow<T>(d));
                __builtin_amdgcn_sched_barrier(0);
            }
            if (lane < rest && in) *at(out, kPer * vectors + lane) = static_cast<T>(rstd * (last_u - c1 - last_xh * c2));
        }
    }
    // the workgroup's rows hold the same columns; summed in their order
    constexpr int R = S::kRows, kWidth = S::kLanes * NV * kPer;
    __shared__ float sums[R > 1 ? R : 1][R > 1 ? kWidth : 1], tails[R > 1 ? R : 1][R > 1 ? S::kLanes : 1];
    for (int k = 0; k < 2; ++k) {
        const int64_t base = k == 0 ? a.gamma : a.beta;
        if (!out.part && (!out.G || base < 0)) continue;
        float *to = out.part ? out.part + ((m * gridDim.x + blockIdx.x) * 2 + k) * D : out.G + m * out.ld + base;
        const bool add = !out.part && out.add;
        if (R == 1) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (lane + S::kLanes * v >= vectors) continue;
                float *at = to + kPer * (lane + S::kLanes * v);
                Wide s = k == 0 ? sg[v] : sb[v];
                if (add) s += load_floats<T>(at);
                store_floats<T>(at, s);
            }
            if (lane < rest) {
                float *at = to + kPer * vectors + lane;
                *at = (k == 0 ? last_sg : last_sb) + (add ? *at : 0.0f);
            }
            continue;
        }
        const int r = threadIdx.x / S::kLanes;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < kPer; ++i) sums[r][kPer * (lane + S::kLanes * v) + i] = k == 0 ? sg[v][i] : sb[v][i];
        tails[r][lane] = k == 0 ? last_sg : last_sb;
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += S::kThreads) {
            const bool tail = c >= kPer * vectors;
            float s = 0.0f;
#pragma unroll
            for (int q = 0; q < R; ++q) s += tail ? tails[q][c - kPer * vectors] : sums[q][c];
            to[c] = add ? to[c] + s : s;
        }
    }
}

// Rows that do not fit the registers: read twice.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_bwd_long(const T *x, const T *dy, NormArgs a, const float *stats, T *dx) {
    __shared__ float slots[2][2][16];
    const int64_t m = blockIdx.y, D = a.D;
    const float inv = 1.0f / static_cast<float>(D);
    int turn = 0;
    for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x, turn ^= 1) {
        const int64_t at = (m * a.N + n) * D;
        const float mean = stats[2 * (m * a.N + n)], rstd = stats[2 * (m * a.N + n) + 1];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t c = 8 * threadIdx.x; c < D; c += 8192) {
            const f32x8 f = load8(x + at + c, D - c, mean), d = load8(dy + at + c, D - c);
            f32x8 g = 1.0f;
            if (a.gamma >= 0) g = load8(a.P + m * a.ldp + a.gamma + c, D - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = d[i] * g[i];
                s1 += u;
                s2 = fmaf(u, (f[i] - mean) * rstd, s2);
            }
        }
        const float c1 = group_sum<16>(s1, slots[turn][0]) * inv, c2 = group_sum<16>(s2, slots[turn][1]) * inv;
        for (int64_t c = 8 * threadIdx.x; c < D; c += 8192) {
            const f32x8 f = load8(x + at + c, D - c, mean);
            f32x8 d = load8(dy + at + c, D - c), g = 1.0f;
            if (a.gamma >= 0) g = load8(a.P + m * a.ldp + a.gamma + c, D - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = rstd * (d[i] * g[i] - c1 - (f[i] - mean) * rstd * c2);
            store8(dx + at + c, D - c, d);
        }
    }
}
// ... and their columns' sums, one lane per eight columns of one share of the rows.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_sums_long(const T *x, const T *dy, NormArgs a, const float *stats,
                                                        int shares, float *part) {
    const int64_t m = blockIdx.z, D = a.D, c = 8 * (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x);
    if (c >= D) return;
    f32x8 sg = 0.0f, sb = 0.0f;
    for (int64_t n = blockIdx.y; n < a.N; n += shares) {
        const int64_t at = (m * a.N + n) * D + c;
        const float mean = stats[2 * (m * a.N + n)], rstd = stats[2 * (m * a.N + n) + 1];
        const f32x8 f = load8(x + at, D - c, mean), d = load8(dy + at, D - c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sg[i] = fmaf(d[i], (f[i] - mean) * rstd, sg[i]);
            sb[i] += d[i];
        }
    }
    float *to = part + (m * shares + blockIdx.y) * 2 * D + c;
    store8(to, D - c, sg);
    store8(to + D, D - c, sb);
}

// G's weight and bias from the shares' sums: 64 columns per workgroup, its waves
// taking every 16th share, eight of them on their way at a time.
__global__ __launch_bounds__(1024) void k_norm_params(const float *part, int shares, NormArgs a, int64_t ld, float *G,
                                                      bool add) {
    constexpr int kWaves = 16, kBatch = 8;
    __shared__ float sums[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m = blockIdx.y, D = a.D, col = static_cast<int64_t>(blockIdx.x) * 64 + lane;
    const float *p = part + m * shares * 2 * D + (col < 2 * D ? col : 2 * D - 1);
    float s = 0.0f;
    for (int b = wave; b < shares; b += kWaves * kBatch) {
        float f[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) f[u] = p[static_cast<int64_t>(b + kWaves * u < shares ? b + kWaves * u : b) * 2 * D];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (b + kWaves * u < shares) s += f[u];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave > 0 || col >= 2 * D) return;
    for (int w = 1; w < kWaves; ++w) s += sums[w][lane];
    const int64_t base = col < D ? a.gamma : a.beta;
    if (base < 0) return;
    float *to = G + m * ld + base + (col < D ? col : col - D);
    *to = add ? *to + s : s;
}

// ---------------------------------------------------------------------------

// Widest rows that stay in registers; forward, of f32 they are those of up to 17408,
// which 16 waves of four vectors hold.
constexpr int kForwardMost = 32768, kBackwardMost = 16384;

// Workgroups per worker of the forward pass: 8192 in all, and 2048 of wide rows,
// whose weight and bias are as much to read as a row (8192 and 2048: rows of 2048
// bf16 elements, 537 MB, 95.6 and 103 us, of 16384 127 and 106).
int64_t forward_groups(int64_t M, int64_t N, int rows_per_group, int threads) {
    const int64_t most = ceil_div(N, rows_per_group), want = ceil_div(threads > 256 ? 2048 : 8192, M);
    return most < want ? most : want;
}
// Shares of a worker's rows whose columns' sums are kept apart.  One where a
// workgroup comes through all rows in up to 8 turns, and adds its sums to G itself,
// as the second launch is 3 us of the host's time: 128 rows of 64 bf16 9.2 us and 12.5,
// 32 of 512 9.0 and 12.3, 8 of 5000 13.3 and 15.8; with 16 turns 64 rows of 1024 would
// take 18 where shares take 12, 16 of 5000 24 and 16.
constexpr int64_t kAlone = 8;
// Otherwise 8 rows at least (16 where a workgroup takes as many at a time), and 4 of
// those that take a workgroup each while there are CUs for all (1000 rows of 4096 f16
// 14.7 us and 18.2, 500 of 12288 19.7 and 26.2; 2 x 1000 of 12288 52 and 43).
int shares_of(int64_t M, int64_t N, int groups, int least, int rows, int threads) {
    if (ceil_div(N, rows) <= kAlone) return 1;
    const int few = rows > 8 ? rows : 8;
    const bool short_ones = rows == 1 && M * ceil_div(N, 4) <= (threads > 256 ? 256 : 512);
    const int64_t want = ceil_div(groups, M), most = ceil_div(N, short_ones ? 4 : M * N < 8192 ? few : least);
    const int64_t s = most < want ? most : want;
    return static_cast<int>(s < 1 ? 1 : s);
}

// How the rows pass by the caches, by the bytes of all of them.  Forward: whether what
// is written does; 8192 rows of 2048 bf16 for each of 8 workers (537 MB): 95.6 us
// written so, 107.5 not; 66 MB the same.  Backward: 0 not, 1 what is written, 2 what is
// read too.  Rows of 1024 bf16, us with 0, 1 and 2: 50 MB 15.8 15.9 18.1, 90 MB 23.4
// 21.7 24.1, 130 MB 32.6 28.9 30.4, 220 MB 55.8 54.4 51.8, 800 MB 158.6 156.9 143.9; of
// f32 22.8 20.5 22.6 with 90 MB and 48.5 47.4 44.9 with 220; rows of 512 to 9000 in the
// same order (9000 bf16: all three within 2 % from 130 MB on; 180 MB of 1024: 2 by 4 %).
bool forward_streams(double bytes) { return bytes > 100e6; }
int backward_streams(double bytes) { return bytes > 200e6 ? 2 : bytes > 80e6 ? 1 : 0; }
template <typename F>
void with_streams(int streams, F &&f) {
    if (streams == 0)
        f(std::integral_constant<int, 0>{});
    else if (streams == 1)
        f(std::integral_constant<int, 1>{});
    else
        f(std::integral_constant<int, 2>{});
}

dqgan_status check(dqgan_plan P, const dqgan_norm_desc *d, int64_t ldp) {
    if (!P || !d) return DQGAN_EINVAL;
    const int64_t n = P->desc.d;
    if (d->width < 1 || d->width > kMaxWidth || !tokens_ok(P, d->tokens) || !type_ok(d->type) || d->reserved != 0)
        return DQGAN_EINVAL;
    if (!(d->eps >= 0.0f) || !isfinite(d->eps) || !ldp_ok(P, ldp)) return DQGAN_EINVAL;
    for (int64_t at : {d->gamma, d->beta})
        if (at < -1 || (at >= 0 && (d->width > n || at > n - d->width))) return DQGAN_EINVAL;
    if (d->gamma >= 0 && d->beta >= 0 && d->gamma < d->beta + d->width && d->beta < d->gamma + d->width)
        return DQGAN_EINVAL;
    return DQGAN_OK;
}

NormArgs args(const dqgan_norm_desc *d, const float *P, int64_t ldp) {
    return NormArgs{P, ldp, d->gamma, d->beta, d->width, d->tokens, d->eps};
}

// f(Shape{}) with the smallest row shape that holds D elements of T; returns
// false, f not called, if D is above MOST.  16 waves of four vectors have 128
// registers a lane, too few for the backward pass of 16-bit types.
template <typename S, typename T, typename F>
bool if_holds(int64_t D, F &f) {
    if (!S::template holds<T>(D)) return false;
    f(S{});
    return true;
}
template <typename T, int MOST, typename F>
bool with_shape(int64_t D, F &&f) {
    if (D > MOST) return false;
    if (if_holds<Shape<16, 1, 1>, T>(D, f) || if_holds<Shape<16, 1, 2>, T>(D, f) || if_holds<Shape<64, 1, 1>, T>(D, f) ||
        if_holds<Shape<64, 1, 2>, T>(D, f) || if_holds<Shape<64, 1, 3>, T>(D, f) || if_holds<Shape<64, 4, 1>, T>(D, f) || if_holds<Shape<64, 4, 2>, T>(D, f) ||
        if_holds<Shape<64, 4, 3>, T>(D, f) || if_holds<Shape<64, 4, 4>, T>(D, f) || if_holds<Shape<64, 16, 2>, T>(D, f))
        return true;
    if constexpr (MOST / Vec16<T>::kPer > 2048) return if_holds<Shape<64, 16, 4>, T>(D, f);
    return false;
}

// Shares of a call's rows, and whether they are one workgroup's that needs no workspace.
struct Shares {
    int count;
    bool alone;
};
Shares backward_shares(int64_t M, const dqgan_norm_desc *d) {
    Shares shares{shares_of(M, d->tokens, 512, 8, 1, 1024), false};
    with_type(d->type, [&](auto t) {
        with_shape<decltype(t), kBackwardMost>(d->width, [&](auto s) {
            using S = decltype(s);
            shares.count = shares_of(M, d->tokens, S::kGroups, S::kLeast, S::kRows, S::kThreads);
            shares.alone = shares.count == 1;
        });
    });
    return shares;
}

}  // namespace
}  // namespace dq

using namespace dq;

extern "C" {

dqgan_status dqgan_norm_forward(dqgan_plan P, const dqgan_norm_desc *d, const void *x, const float *params, int64_t ldp,
                                void *y, float *stats, void *stream) {
    DQ_TRY(check(P, d, ldp));
    const bool any = d->tokens > 0;
    DQ_TRY(check_ptr(x, any));
    DQ_TRY(check_ptr(y, any));
    DQ_TRY(check_ptr(stats, false));
    DQ_TRY(check_ptr(params, any && (d->gamma >= 0 || d->beta >= 0)));
    DQ_TRY(check_device(P));
    if (!any) return DQGAN_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const NormArgs a = args(d, params, ldp);
    const int64_t M = P->desc.M;
    with_type(d->type, [&](auto t) {
        using T = decltype(t);
        const T *from = static_cast<const T *>(x);
        T *to = static_cast<T *>(y);
        const uint32_t my = static_cast<uint32_t>(M);
        if (!with_shape<T, kForwardMost>(d->width, [&](auto s) {
                using S = decltype(s);
                const dim3 grid(static_cast<uint32_t>(forward_groups(M, d->tokens, S::kRows, S::kThreads)), my);
                if (forward_streams(2.0 * sizeof(T) * M * d->tokens * d->width))
                    k_norm_fwd<T, S, true><<<grid, S::kThreads, 0, st>>>(from, a, to, stats);
                else
                    k_norm_fwd<T, S, false><<<grid, S::kThreads, 0, st>>>(from, a, to, stats);
            }))
            k_norm_fwd_long<T><<<dim3(static_cast<uint32_t>(forward_groups(M, d->tokens, 1, 1024)), my), 1024, 0, st>>>(
                from, a, to, stats);
    });
    return launched();
}

dqgan_status dqgan_norm_bytes(dqgan_plan P, const dqgan_norm_desc *d, size_t *bytes) {
    DQ_TRY(check(P, d, 0));
    if (!bytes) return DQGAN_EINVAL;
    const bool sums = d->tokens > 0 && (d->gamma >= 0 || d->beta >= 0);
    const Shares shares = backward_shares(P->desc.M, d);
    *bytes = sums && !shares.alone ? sizeof(float) * 2 * static_cast<size_t>(d->width) * P->desc.M * shares.count : 0;
    return DQGAN_OK;
}

dqgan_status dqgan_norm_backward(dqgan_plan P, const dqgan_norm_desc *d, const void *x, const void *dy,
                                 const float *params, int64_t ldp, const float *stats, void *dx, float *G, int32_t add,
                                 void *workspace, void *stream) {
    DQ_TRY(check(P, d, ldp));
    const bool any = d->tokens > 0, sums = d->gamma >= 0 || d->beta >= 0;
    DQ_TRY(check_ptr(x, any));
    DQ_TRY(check_ptr(dy, any));
    DQ_TRY(check_ptr(stats, any));
    DQ_TRY(check_ptr(dx, false));
    DQ_TRY(check_ptr(params, any && d->gamma >= 0));
    DQ_TRY(check_ptr(G, sums));
    const Shares shares = any ? backward_shares(P->desc.M, d) : Shares{0, false};
    DQ_TRY(check_ptr(workspace, any && sums && !shares.alone));
    DQ_TRY(check_device(P));
    hipStream_t st = static_cast<hipStream_t>(stream);
    NormArgs a = args(d, params, ldp);
    const int64_t M = P->desc.M, D = d->width;
    const bool alone = sums && shares.alone;
    float *part = sums && !alone ? static_cast<float *>(workspace) : nullptr;
    const Sums out{part, alone ? G : nullptr, P->desc.ld, add != 0};
    if (any && (dx || sums)) {
        with_type(d->type, [&](auto t) {
            using T = decltype(t);
            const T *xt = static_cast<const T *>(x), *dyt = static_cast<const T *>(dy);
            T *dxt = static_cast<T *>(dx);
            const uint32_t my = static_cast<uint32_t>(M), of = static_cast<uint32_t>(shares.count);
            if (with_shape<T, kBackwardMost>(D, [&](auto s) {
                    using S = decltype(s);
                    with_streams(backward_streams(3.0 * sizeof(T) * M * d->tokens * D), [&](auto streams) {
                        k_norm_bwd<T, S, decltype(streams)::value><<<dim3(of, my), S::kThreads, 0, st>>>(
                            xt, dyt, a, stats, dxt, out);
                    });
                }))
                return;
            if (sums)  // first: dx may be dy
                k_norm_sums_long<T><<<dim3(static_cast<uint32_t>(ceil_div(D, 2048)), of, my), 256, 0, st>>>(
                    xt, dyt, a, stats, shares.count, part);
            if (dx)
                k_norm_bwd_long<T><<<dim3(static_cast<uint32_t>(forward_groups(M, d->tokens, 1, 1024)), my), 1024, 0, st>>>(
                    xt, dyt, a, stats, dxt);
        });
    }
    if (sums && !alone && (any || !add)) {
        const dim3 grid(static_cast<uint32_t>(ceil_div(2 * D, 64)), static_cast<uint32_t>(M));
        k_norm_params<<<grid, 1024, 0, st>>>(part, shares.count, a, P->desc.ld, G, add != 0);
    }
    return launched();
}

}  // extern "C"
