// Embedding lookup of M workers, each from its own table in its row of P, and
// its gradient, summed over sorted tokens into the worker's row of G.
//
// The gradient's launches:
//   k_embed_sort   one workgroup per worker sorts its tokens (stable, so that
//                  equal ones stay in their order); the other workgroups of the
//                  launch write the table's part of G as 0 meanwhile;
//   k_embed_sum    chunks of kChunk sorted places, one wave per chunk and 512
//                  channels.  A token whose places lie within a chunk has its row
//                  written; one that runs across chunks leaves a partial sum in
//                  each, so that a frequent token is as much work as a rare one;
//   k_embed_join   sums those.
#include "layers.hpp"

namespace dq {
namespace {

constexpr int kChunk = 32;           // sorted places per wave of k_embed_sum
constexpr int kSlab = 512;           // channels per wave
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kDigitMost = 9;        // bits of a sort digit: 512 counters for each of 16 waves
constexpr int64_t kFillFloats = 16384;  // of G per workgroup

struct EmbedArgs {
    int64_t offset, V, D, N, ld;
    float scale;
};

// `lanes` (a power of two) consecutive threads per token.
template <typename T, typename I>
__global__ __launch_bounds__(256) void k_embed_fwd(const I *tok, const float *P, int64_t ldp, EmbedArgs a, int shift,
                                                   T *out) {
    const int64_t m = blockIdx.y;
    const int lanes = 1 << shift, per = 256 >> shift, lane = threadIdx.x & (lanes - 1);
    for (int64_t n = static_cast<int64_t>(blockIdx.x) * per + (threadIdx.x >> shift); n < a.N;
         n += static_cast<int64_t>(gridDim.x) * per) {
        const I t = tok[m * a.N + n];
        const bool there = t >= 0 && static_cast<int64_t>(t) < a.V;
        const float *row = P + m * ldp + a.offset + (there ? static_cast<int64_t>(t) : 0) * a.D;
        T *to = out + (m * a.N + n) * a.D;
        for (int64_t c = 8 * lane; c < a.D; c += 8 * lanes) {
            f32x8 f = 0.0f;
            if (there) {
                f = load8(row + c, a.D - c);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= a.scale;
            }
            store8(to + c, a.D - c, f);
        }
    }
}

// The sorted lists of one worker: token and place, with padded places as token V
// behind all others.
struct Lists {
    uint32_t *key[2], *at[2];  // [M][N]: the passes go from one pair to the other
};

template <typename I>
__device__ __forceinline__ uint32_t key_of(const I *tok, int64_t i, int64_t V) {
    const I t = tok[i];
    return t >= 0 && static_cast<int64_t>(t) < V ? static_cast<uint32_t>(t) : static_cast<uint32_t>(V);
}

// Stable sort by digits from the lowest up.  A wave owns a contiguous run of
// places and, of the counters [digit][wave], its own column.
template <typename I>
__device__ void sort_tokens(const I *tok, int64_t V, int64_t N, uint32_t *const key[2], uint32_t *const at[2], int bits,
                            int passes) {
    __shared__ uint32_t count[kSortWaves << kDigitMost];
    __shared__ uint32_t total[kSortWaves];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t run = (N + kSortThreads - 1) / kSortThreads * 64;
    const int64_t begin = wave * run < N ? wave * run : N, end = begin + run < N ? begin + run : N;
    const int counters = kSortWaves << bits;
    for (int p = 0; p < passes; ++p) {
        const uint32_t *from_key = key[(p + 1) & 1], *from_at = at[(p + 1) & 1];
        uint32_t *to_key = key[p & 1], *to_at = at[p & 1];
        const int shift = p * bits;
        const uint32_t mask = (1u << bits) - 1;
        for (int i = tid; i < counters; i += kSortThreads) count[i] = 0;
        __syncthreads();
        for (int64_t i = begin + lane; i < end; i += 64) {
            const uint32_t k = p == 0 ? key_of(tok, i, V) : from_key[i];
            atomicAdd(&count[((k >> shift & mask) * kSortWaves) + wave], 1u);
        }
        __syncthreads();
        // exclusive sums over [digit][wave]
        const int each = counters / kSortThreads;
        uint32_t sum = 0;
        for (int i = 0; i < each; ++i) sum += count[tid * each + i];
        uint32_t upto = sum;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t other = __shfl_up(upto, o);
            if (lane >= o) upto += other;
        }
        if (lane == 63) total[wave] = upto;
        __syncthreads();
        uint32_t base = upto - sum;
        for (int w = 0; w < wave; ++w) base += total[w];
        for (int i = 0; i < each; ++i) {
            const uint32_t c = count[tid * each + i];
            count[tid * each + i] = base;
            base += c;
        }
        __syncthreads();
        for (int64_t i0 = begin; i0 < end; i0 += 64) {
            const int64_t i = i0 + lane;
            const bool in = i < end;
            const uint32_t k = !in ? 0 : p == 0 ? key_of(tok, i, V) : from_key[i];
            const uint32_t where = p == 0 || !in ? static_cast<uint32_t>(i) : from_at[i];
            const uint32_t digit = k >> shift & mask;
            uint64_t same = __ballot(in);
            for (int b = 0; b < bits; ++b) {
                const uint64_t set = __ballot(digit >> b & 1);
                same &= (digit >> b & 1) ? set : ~set;
            }
            if (in) {
                uint32_t *slot = &count[digit * kSortWaves + wave];
                const uint32_t first = *reinterpret_cast<volatile uint32_t *>(slot);
                const int before = __popcll(same & ((uint64_t(1) << lane) - 1));
                if (before == 0) *reinterpret_cast<volatile uint32_t *>(slot) = first + __popcll(same);
                to_key[first + before] = k;
                to_at[first + before] = where;
            }
        }
        __syncthreads();
    }
}

template <typename I>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(const I *tok, EmbedArgs a, int M, Lists l, int bits,
                                                             int passes, int fills, float *G) {
    if (static_cast<int>(blockIdx.x) < M) {
        const int64_t at = static_cast<int64_t>(blockIdx.x) * a.N;
        uint32_t *const keys[2] = {l.key[0] + at, l.key[1] + at}, *const ats[2] = {l.at[0] + at, l.at[1] + at};
        sort_tokens(tok + at, a.V, a.N, keys, ats, bits, passes);
        return;
    }
    // the table's part of G, from a 16-byte boundary on in vectors
    const int64_t b = blockIdx.x - M, m = b / fills, len = a.V * a.D;
    float *to = G + m * a.ld + a.offset;
    const int64_t head = len < ((4 - (a.offset & 3)) & 3) ? len : ((4 - (a.offset & 3)) & 3);
    const int64_t quads = (len - head) / 4, each = (quads + fills - 1) / fills;
    const int64_t first = (b % fills) * each, last = first + each < quads ? first + each : quads;
    f32x4 *v = reinterpret_cast<f32x4 *>(to + head);
    for (int64_t q = first + threadIdx.x; q < last; q += kSortThreads) v[q] = 0.0f;
    if (b % fills == 0) {
        if (threadIdx.x < head) to[threadIdx.x] = 0.0f;
        if (threadIdx.x < ((len - head) & 3)) to[head + 4 * quads + threadIdx.x] = 0.0f;
    }
}

__device__ __forceinline__ void put_row(float *to, int64_t n, f32x8 s, float scale, bool add) {
    if (n <= 0) return;
    f32x8 f = 0.0f;
    if (add) f = load8(to, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = add ? f[i] + s[i] * scale : s[i] * scale;
    store8(to, n, f);
}

template <typename T>
__global__ __launch_bounds__(256) void k_embed_sum(const uint32_t *key, const uint32_t *at, const T *dout, EmbedArgs a,
                                                   int64_t chunks, int slabs, float *part, float *G, bool add) {
    const int64_t m = blockIdx.y, task = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (task >= chunks * slabs) return;
    const int64_t chunk = task / slabs, c = (task % slabs) * kSlab + 8 * (threadIdx.x & 63), rest = a.D - c;
    const int64_t e0 = chunk * kChunk, e1 = e0 + kChunk < a.N ? e0 + kChunk : a.N;
    const int n = static_cast<int>(e1 - e0);
    key += m * a.N;
    at += m * a.N;
    dout += m * a.N * a.D;
    G += m * a.ld + a.offset;
    part += (m * chunks + chunk) * 2 * a.D;
    const uint32_t V = static_cast<uint32_t>(a.V);
    const uint32_t before = e0 > 0 ? key[e0 - 1] : V, after = e1 < a.N ? key[e1] : V;
    f32x8 s = 0.0f;
    int from = 0;
    for (int e = 0; e < n; ++e) {
        const uint32_t k = key[e0 + e];
        if (k == V) break;
        if (rest > 0) {
            const f32x8 f = load8(dout + static_cast<int64_t>(at[e0 + e]) * a.D + c, rest);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += f[i];
        }
        const uint32_t next = e + 1 < n ? key[e0 + e + 1] : after;
        if (e + 1 < n && next == k) continue;
        const bool began = from == 0 && before == k, goes_on = e + 1 == n && next == k;
        if (!began && !goes_on)
            put_row(G + static_cast<int64_t>(k) * a.D + c, rest, s, a.scale, add);
        else
            store8(part + (began ? 0 : a.D) + c, rest, s);
        s = 0.0f;
        from = e + 1;
    }
}

// A token that runs on beyond the chunk it begins in: that chunk's second
// partial sum and the first ones of those that follow.
template <int W>
__global__ __launch_bounds__(64 * W) void k_embed_join(const uint32_t *key, EmbedArgs a, int64_t chunks, int slabs,
                                                       const float *part, float *G, bool add) {
    __shared__ float sums[W > 1 ? W - 1 : 1][64][8];
    const int64_t m = blockIdx.y, chunk = static_cast<int64_t>(blockIdx.x) / slabs;
    key += m * a.N;
    const uint32_t V = static_cast<uint32_t>(a.V);
    const int64_t e0 = chunk * kChunk, e1 = e0 + kChunk;
    if (e1 >= a.N) return;
    const uint32_t k = key[e1 - 1];
    if (k == V || key[e1] != k) return;
    if (e0 > 0 && key[e0 - 1] == k) return;
    int64_t lo = e1, hi = a.N;  // key[lo] == k, the first other key is at or below hi
    while (hi - lo > 1) {
        const int64_t mid = lo + (hi - lo) / 2;
        if (key[mid] == k)
            lo = mid;
        else
            hi = mid;
    }
    const int64_t last = lo / kChunk;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t c = (blockIdx.x % slabs) * kSlab + 8 * lane, rest = a.D - c;
    part += m * chunks * 2 * a.D + c;
    // each wave a contiguous share of the partial sums
    const int64_t each = (last - chunk + W - 1) / W, first = chunk + 1 + wave * each;
    const int64_t upto = first + each < last + 1 ? first + each : last + 1;
    f32x8 s = 0.0f;
    if (wave == 0) s = load8(part + (2 * chunk + 1) * a.D, rest);
    for (int64_t b = first; b < upto; ++b) {
        const f32x8 f = load8(part + 2 * b * a.D, rest);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += f[i];
    }
    if (W > 1) {
        if (wave > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[wave - 1][lane][i] = s[i];
        }
        __syncthreads();
        if (wave > 0) return;
        for (int w = 0; w < W - 1; ++w)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += sums[w][lane][i];
    }
    put_row(G + m * a.ld + a.offset + static_cast<int64_t>(k) * a.D + c, rest, s, a.scale, add);
}

// ---------------------------------------------------------------------------

constexpr int64_t kMostGroups = int64_t(1) << 24;  // of 256 threads in a launch's first dimension: below 2^32 threads

int64_t chunks_of(int64_t N) { return ceil_div(N, kChunk); }
int slabs_of(int64_t D) { return static_cast<int>(ceil_div(D, kSlab)); }

dqgan_status check(dqgan_plan P, const dqgan_embed_desc *d) {
    if (!P || !d) return DQGAN_EINVAL;
    const int64_t n = P->desc.d;
    if (d->vocab < 1 || d->vocab > INT32_MAX - 1 || d->width < 1 || d->width > kMaxWidth) return DQGAN_EINVAL;
    if (d->offset < 0 || d->offset >= n || d->vocab > (n - d->offset) / d->width) return DQGAN_EINVAL;
    if (!tokens_ok(P, d->tokens) || !type_ok(d->type) || d->reserved != 0 || !isfinite(d->scale)) return DQGAN_EINVAL;
    if (d->index_type != DQGAN_I32 && d->index_type != DQGAN_I64) return DQGAN_EINVAL;
    if (chunks_of(d->tokens) * slabs_of(d->width) > kMostGroups) return DQGAN_EINVAL;
    return DQGAN_OK;
}

EmbedArgs args(dqgan_plan P, const dqgan_embed_desc *d) {
    return EmbedArgs{d->offset, d->vocab, d->width, d->tokens, P->desc.ld, d->scale};
}

template <typename F>
void with_index(int32_t type, F &&f) {
    if (type == DQGAN_I32)
        f(int32_t{});
    else
        f(int64_t{});
}

size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

// The workspace: two pairs of lists, then the partial sums.
size_t list_bytes(int64_t M, int64_t N) { return round256(sizeof(uint32_t) * static_cast<size_t>(M * N)); }

}  // namespace
}  // namespace dq

using namespace dq;

extern "C" {

dqgan_status dqgan_embed_forward(dqgan_plan P, const dqgan_embed_desc *d, const void *tok, const float *params,
                                 int64_t ldp, void *out, void *stream) {
    DQ_TRY(check(P, d));
    if (!ldp_ok(P, ldp)) return DQGAN_EINVAL;
    const bool any = d->tokens > 0;
    DQ_TRY(check_ptr(tok, any));
    DQ_TRY(check_ptr(params, any));
    DQ_TRY(check_ptr(out, any));
    DQ_TRY(check_device(P));
    if (!any) return DQGAN_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const EmbedArgs a = args(P, d);
    int shift = 0;
    while (shift < 8 && (int64_t(8) << shift) < a.D) ++shift;
    const int64_t groups = ceil_div(a.N, 256 >> shift);
    const dim3 grid(static_cast<uint32_t>(groups < 65536 ? groups : 65536), static_cast<uint32_t>(P->desc.M));
    with_type(d->type, [&](auto t) {
        with_index(d->index_type, [&](auto i) {
            using T = decltype(t);
            using I = decltype(i);
            k_embed_fwd<T, I><<<grid, 256, 0, st>>>(static_cast<const I *>(tok), params, ldp, a, shift,
                                                    static_cast<T *>(out));
        });
    });
    return launched();
}

dqgan_status dqgan_embed_bytes(dqgan_plan P, const dqgan_embed_desc *d, size_t *bytes) {
    DQ_TRY(check(P, d));
    if (!bytes) return DQGAN_EINVAL;
    const int64_t M = P->desc.M;
    *bytes = d->tokens == 0 ? 0
                            : 4 * list_bytes(M, d->tokens) + sizeof(float) * 2 *
                                                                 static_cast<size_t>(M * chunks_of(d->tokens)) * d->width;
    return DQGAN_OK;
}

dqgan_status dqgan_embed_backward(dqgan_plan P, const dqgan_embed_desc *d, const void *tok, const void *dout, float *G,
                                  int32_t add, void *workspace, void *stream) {
    DQ_TRY(check(P, d));
    const bool any = d->tokens > 0;
    DQ_TRY(check_ptr(tok, any));
    DQ_TRY(check_ptr(dout, any));
    DQ_TRY(check_ptr(G));
    DQ_TRY(check_ptr(workspace, any));
    DQ_TRY(check_device(P));
    hipStream_t st = static_cast<hipStream_t>(stream);
    const EmbedArgs a = args(P, d);
    const int64_t M = P->desc.M;
    Lists l{};
    if (any)
        for (int i = 0; i < 2; ++i) {
            l.key[i] = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + (2 * i) * list_bytes(M, a.N));
            l.at[i] = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + (2 * i + 1) * list_bytes(M, a.N));
        }
    float *part = reinterpret_cast<float *>(static_cast<char *>(workspace) + 4 * list_bytes(M, a.N));
    int bits = 1;  // of the largest key, V
    while ((a.V >> bits) != 0) ++bits;
    const int passes = (bits + kDigitMost - 1) / kDigitMost;
    int digit = (bits + passes - 1) / passes;
    if (digit < 6) digit = 6;  // 1024 counters at least: one per thread
    const int64_t want = ceil_div(a.V * a.D, kFillFloats), most = kMostGroups / 8 / M;
    const int fills = add ? 0 : static_cast<int>(want < most ? want : most);
    const int sorts = any ? static_cast<int>(M) : 0;
    const uint32_t groups = static_cast<uint32_t>(sorts + M * fills);
    if (groups == 0) return DQGAN_OK;
    with_index(d->index_type, [&](auto i) {
        using I = decltype(i);
        k_embed_sort<I><<<groups, kSortThreads, 0, st>>>(static_cast<const I *>(tok), a, sorts, l, digit, passes, fills, G);
    });
    if (!any) return launched();
    const uint32_t *key = l.key[(passes - 1) & 1], *at = l.at[(passes - 1) & 1];
    const int64_t chunks = chunks_of(a.N);
    const int slabs = slabs_of(a.D);
    const dim3 grid(static_cast<uint32_t>(ceil_div(chunks * slabs, 4)), static_cast<uint32_t>(M));
    with_type(d->type, [&](auto t) {
        using T = decltype(t);
        k_embed_sum<T><<<grid, 256, 0, st>>>(key, at, static_cast<const T *>(dout), a, chunks, slabs, part, G, add != 0);
    });
    if (chunks > 1)
        k_embed_join<4><<<dim3(static_cast<uint32_t>(chunks * slabs), static_cast<uint32_t>(M)), 256, 0, st>>>(
            key, a, chunks, slabs, part, G, add != 0);
    return launched();
}

}  // extern "C"
