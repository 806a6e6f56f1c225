// Layer norm of M workers, each with its own weight and bias in its row of P,
// and its gradients, those of weight and bias in the worker's row of G.
#include "layers.hpp"

namespace dq {
namespace {

// Row shapes: W waves per row, NV vectors of eight elements per lane, so that
// a row of up to 512 W NV elements stays in registers between the statistics
// and their use.
template <int W>
constexpr int kThreads = W < 4 ? 256 : 64 * W;
template <int W>
constexpr int kRowsPerGroup = W < 4 ? 4 / W : 1;

struct NormArgs {
    const float *P;
    int64_t ldp;
    int64_t gamma, beta;  // -1: none
    int64_t D, N;
    float eps;
};

// Two passes over the registers: the mean, then the mean square of what is
// left, so that a large mean costs the variance no digits.
template <typename T, int W, int NV>
__global__ __launch_bounds__(kThreads<W>) void k_norm_fwd(const T *x, NormArgs a, T *y, float *stats) {
    __shared__ float slots[2][W];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t m = blockIdx.y, D = a.D;
    f32x8 g[NV], b[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int64_t c = 8 * (lane + 64 * W * v);
        g[v] = 1.0f;
        b[v] = 0.0f;
        if (a.gamma >= 0 && c < D) g[v] = load8(a.P + m * a.ldp + a.gamma + c, D - c);
        if (a.beta >= 0 && c < D) b[v] = load8(a.P + m * a.ldp + a.beta + c, D - c);
    }
    const float inv = 1.0f / static_cast<float>(D);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRowsPerGroup<W>;
    for (int64_t n = static_cast<int64_t>(blockIdx.x) * kRowsPerGroup<W> + (W == 1 ? threadIdx.x >> 6 : 0); n < a.N;
         n += step) {
        const T *row = x + (m * a.N + n) * D;
        f32x8 f[NV];
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = 8 * (lane + 64 * W * v);
            f[v] = load8(row + c, D - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += f[v][i];
        }
        const float mean = group_sum<W>(s, slots[0]) * inv;
        s = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = 8 * (lane + 64 * W * v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[v][i] = c + i < D ? f[v][i] - mean : 0.0f;
                s = fmaf(f[v][i], f[v][i], s);
            }
        }
        const float rstd = 1.0f / sqrtf(group_sum<W>(s, slots[1]) * inv + a.eps);
        T *out = y + (m * a.N + n) * D;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = 8 * (lane + 64 * W * v);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[v][i] = fmaf(f[v][i] * rstd, g[v][i], b[v][i]);
            store8(out + c, D - c, f[v]);
        }
        if (stats && lane == 0) {
            stats[2 * (m * a.N + n)] = mean;
            stats[2 * (m * a.N + n) + 1] = rstd;
        }
    }
}

// Rows that do not fit the registers: read three times.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_fwd_long(const T *x, NormArgs a, T *y, float *stats) {
    __shared__ float slots[2][16];
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
        const float rstd = 1.0f / sqrtf(group_sum<16>(s, slots[1]) * inv + a.eps);
        T *out = y + (m * a.N + n) * D;
        for (int64_t c = 8 * threadIdx.x; c < D; c += 8192) {
            f32x8 f = load8(row + c, D - c), g = 1.0f, b = 0.0f;
            if (a.gamma >= 0) g = load8(a.P + m * a.ldp + a.gamma + c, D - c);
            if (a.beta >= 0) b = load8(a.P + m * a.ldp + a.beta + c, D - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = fmaf((f[i] - mean) * rstd, g[i], b[i]);
            store8(out + c, D - c, f);
        }
        if (stats && threadIdx.x == 0) {
            stats[2 * (m * a.N + n)] = mean;
            stats[2 * (m * a.N + n) + 1] = rstd;
        }
    }
}

// One workgroup takes every gridDim.x-th group of rows of its worker, keeps
// its columns' sums of dy and dy * xh in registers meanwhile and leaves them in
// part[m][blockIdx.x][2][D].
template <typename T, int W, int NV>
__global__ __launch_bounds__(kThreads<W>) void k_norm_bwd(const T *x, const T *dy, NormArgs a, const float *stats,
                                                          T *dx, float *part) {
    __shared__ float slots[2][2][W];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t m = blockIdx.y, D = a.D;
    f32x8 g[NV], sg[NV], sb[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int64_t c = 8 * (lane + 64 * W * v);
        g[v] = 1.0f;
        if (a.gamma >= 0 && c < D) g[v] = load8(a.P + m * a.ldp + a.gamma + c, D - c);
        sg[v] = 0.0f;
        sb[v] = 0.0f;
    }
    const float inv = 1.0f / static_cast<float>(D);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRowsPerGroup<W>;
    int turn = 0;
    for (int64_t n = static_cast<int64_t>(blockIdx.x) * kRowsPerGroup<W> + (W == 1 ? threadIdx.x >> 6 : 0); n < a.N;
         n += step, turn ^= 1) {
        const int64_t at = (m * a.N + n) * D;
        const float mean = stats[2 * (m * a.N + n)], rstd = stats[2 * (m * a.N + n) + 1];
        f32x8 xh[NV], u[NV];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = 8 * (lane + 64 * W * v);
            xh[v] = load8(x + at + c, D - c, mean);
            u[v] = load8(dy + at + c, D - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                xh[v][i] = (xh[v][i] - mean) * rstd;
                sg[v][i] = fmaf(u[v][i], xh[v][i], sg[v][i]);
                sb[v][i] += u[v][i];
                u[v][i] *= g[v][i];
                s1 += u[v][i];
                s2 = fmaf(u[v][i], xh[v][i], s2);
            }
        }
        if (!dx) continue;
        const float c1 = group_sum<W>(s1, slots[turn][0]) * inv, c2 = group_sum<W>(s2, slots[turn][1]) * inv;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = 8 * (lane + 64 * W * v);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[v][i] = rstd * (u[v][i] - c1 - xh[v][i] * c2);
            store8(dx + at + c, D - c, u[v]);
        }
    }
    if (!part) return;
    constexpr int R = kRowsPerGroup<W>;
    __shared__ float sums[R > 1 ? R - 1 : 1][R > 1 ? 64 : 1][8];
    float *to = part + (m * gridDim.x + blockIdx.x) * 2 * D;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t c = 8 * (lane + 64 * W * v);
            f32x8 s = k == 0 ? sg[v] : sb[v];
            if (R > 1) {  // the group's waves hold the same columns
                const int w = threadIdx.x >> 6;
                __syncthreads();
                if (w > 0) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) sums[w - 1][lane][i] = s[i];
                }
                __syncthreads();
                if (w == 0) {
#pragma unroll
                    for (int r = 0; r < R - 1; ++r)
#pragma unroll
                        for (int i = 0; i < 8; ++i) s[i] += sums[r][lane][i];
                }
            }
            if (R == 1 || threadIdx.x < 64) store8(to + k * D + c, D - c, s);
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

// G's weight and bias from the shares' sums: 64 columns per workgroup, four
// quarters of the shares side by side.
__global__ __launch_bounds__(256) void k_norm_params(const float *part, int shares, NormArgs a, int64_t ld, float *G,
                                                     bool add) {
    __shared__ float quarter[3][64];
    const int64_t m = blockIdx.y, D = a.D, col = static_cast<int64_t>(blockIdx.x) * 64 + (threadIdx.x & 63);
    const int q = threadIdx.x >> 6;
    float s = 0.0f;
    if (col < 2 * D) {
        const float *p = part + m * shares * 2 * D + col;
        for (int b = q; b < shares; b += 4) s += p[static_cast<int64_t>(b) * 2 * D];
    }
    if (q > 0) quarter[q - 1][threadIdx.x & 63] = s;
    __syncthreads();
    if (q > 0 || col >= 2 * D) return;
    s = ((s + quarter[0][threadIdx.x]) + quarter[1][threadIdx.x]) + quarter[2][threadIdx.x];
    const int64_t base = col < D ? a.gamma : a.beta;
    if (base < 0) return;
    float *to = G + m * ld + base + (col < D ? col : col - D);
    *to = add ? *to + s : s;
}

// ---------------------------------------------------------------------------

constexpr int64_t kGroups = 2048;    // workgroups that fill the card several times over
constexpr int64_t kWidest = 32768;   // 16 waves, four vectors a lane

// Workgroups per worker of the kernels that loop over rows.
int64_t forward_groups(int64_t M, int64_t N, int rows_per_group) {
    const int64_t most = ceil_div(N, rows_per_group), want = ceil_div(kGroups, M);
    return most < want ? most : want;
}
// Shares of the rows whose columns' sums are kept apart: enough to fill the
// card, and at least 16 rows each, so that their partial sums are a fraction
// of what is read.
int backward_shares(int64_t M, int64_t N) {
    const int64_t want = ceil_div(1024, M), most = ceil_div(N, 16);
    const int64_t s = most < want ? most : want;
    return static_cast<int>(s < 1 ? 1 : s);
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

// f(W, NV) with the smallest row shape that holds D.
template <typename F>
void with_shape(int64_t D, F &&f) {
    using std::integral_constant;
    if (D <= 512)
        f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    else if (D <= 1024)
        f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    else if (D <= 2048)
        f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (D <= 4096)
        f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    else if (D <= 8192)
        f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (D <= 16384)
        f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
    else
        f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
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
        if (d->width > kWidest) {
            const dim3 grid(static_cast<uint32_t>(forward_groups(M, d->tokens, 1)), static_cast<uint32_t>(M));
            k_norm_fwd_long<T><<<grid, 1024, 0, st>>>(static_cast<const T *>(x), a, static_cast<T *>(y), stats);
            return;
        }
        with_shape(d->width, [&](auto w, auto nv) {
            constexpr int W = decltype(w)::value, NV = decltype(nv)::value;
            const dim3 grid(static_cast<uint32_t>(forward_groups(M, d->tokens, kRowsPerGroup<W>)),
                            static_cast<uint32_t>(M));
            k_norm_fwd<T, W, NV><<<grid, kThreads<W>, 0, st>>>(static_cast<const T *>(x), a, static_cast<T *>(y), stats);
        });
    });
    return launched();
}

dqgan_status dqgan_norm_bytes(dqgan_plan P, const dqgan_norm_desc *d, size_t *bytes) {
    DQ_TRY(check(P, d, 0));
    if (!bytes) return DQGAN_EINVAL;
    const bool sums = d->tokens > 0 && (d->gamma >= 0 || d->beta >= 0);
    *bytes = sums ? sizeof(float) * 2 * static_cast<size_t>(d->width) * P->desc.M * backward_shares(P->desc.M, d->tokens)
                  : 0;
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
    DQ_TRY(check_ptr(workspace, any && sums));
    DQ_TRY(check_device(P));
    hipStream_t st = static_cast<hipStream_t>(stream);
    NormArgs a = args(d, params, ldp);
    const int64_t M = P->desc.M, D = d->width;
    const int shares = any ? backward_shares(M, d->tokens) : 0;
    float *part = sums ? static_cast<float *>(workspace) : nullptr;
    if (any && (dx || sums)) {
        with_type(d->type, [&](auto t) {
            using T = decltype(t);
            const T *xt = static_cast<const T *>(x), *dyt = static_cast<const T *>(dy);
            T *dxt = static_cast<T *>(dx);
            if (D > kWidest) {
                if (sums) {  // first: dx may be dy
                    const dim3 grid(static_cast<uint32_t>(ceil_div(D, 2048)), static_cast<uint32_t>(shares),
                                    static_cast<uint32_t>(M));
                    k_norm_sums_long<T><<<grid, 256, 0, st>>>(xt, dyt, a, stats, shares, part);
                }
                if (dx) {
                    const dim3 grid(static_cast<uint32_t>(forward_groups(M, d->tokens, 1)), static_cast<uint32_t>(M));
                    k_norm_bwd_long<T><<<grid, 1024, 0, st>>>(xt, dyt, a, stats, dxt);
                }
                return;
            }
            with_shape(D, [&](auto w, auto nv) {
                constexpr int W = decltype(w)::value, NV = decltype(nv)::value;
                const dim3 grid(static_cast<uint32_t>(shares), static_cast<uint32_t>(M));
                k_norm_bwd<T, W, NV><<<grid, kThreads<W>, 0, st>>>(xt, dyt, a, stats, dxt, part);
            });
        });
    }
    if (sums && (any || !add)) {
        const dim3 grid(static_cast<uint32_t>(ceil_div(2 * D, 64)), static_cast<uint32_t>(M));
        k_norm_params<<<grid, 256, 0, st>>>(part, shares, a, P->desc.ld, G, add != 0);
    }
    return launched();
}

}  // extern "C"
