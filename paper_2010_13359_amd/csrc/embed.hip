// Embedding lookup of M workers, each from its own table in its row of P, and
// its gradient, summed over sorted tokens into the worker's row of G.
//
// The gradient of up to kFew tokens is one launch, k_embed_few: a workgroup owns
// some rows of the table, writes 0 to them and then the sums of those that are
// tokens; each wave has all tokens in its lanes.
//
// The launches of more:
//   k_embed_sort   sorts runs of kRun tokens, one workgroup each (stable, so that
//                  equal ones stay in their order); the other workgroups of the
//                  launch write the table's part of G as 0 meanwhile;
//   k_embed_merge  joins kFan sorted runs to one, as often as there is more than
//                  one run: each token counts the smaller ones in the other runs;
//   k_embed_sum    chunks of 8 or 32 sorted places, one wave per chunk and 1 KB of
//                  dout's rows, or several chunks per wave where the rows are
//                  narrow.  It writes the rows of the tokens that begin in its
//                  chunk and end there or in the next.  One that runs on leaves a
//                  partial sum in each of its chunks, so that a frequent token is
//                  as much work as a rare one;
//   k_embed_join   sums those.
// No sum uses atomics: its order goes by the tokens alone, and the same call gives
// the same bits.  For 8 x 4096 tokens, tables of 32000 x 1024 and bf16, the launch that
// writes 1.05 GB of zeros beside the sort takes 164 us, bound by memory (6.4 TB/s, a
// plain fill 6.9); the sums 44 (2.8 TB/s: 4 waves a CU that wait for their own loads)
// and the join 5.
#include "layers.hpp"

namespace dq {
namespace {

constexpr int kRun = 4096;                 // tokens per workgroup of k_embed_sort
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kEach = kRun / kSortThreads;
constexpr int kDigitMost = 9;              // bits of a sort digit: 512 counters for each of 16 waves
constexpr int kFan = 4;
constexpr int64_t kFillFloats = 32768;     // of G per workgroup

struct EmbedArgs {
    int64_t offset, V, D, N, ld;
    float scale;
};

// 1 << shift consecutive threads per token, four channels each, forward_rows
// tokens at a time: their rows are asked for before the first is used (8 x 8192
// tokens, rows of 1024, to bf16: 47 us, one at a time 74.6; 402 MB at most, if no
// token came twice, are 8.5 TB/s, as frequent rows stay in the caches).  A padded
// place reads the table's first row and writes 0.
template <typename T>
constexpr int forward_rows = sizeof(T) == 4 ? 2 : 4;
template <typename T, typename I, bool STREAM>
__global__ __launch_bounds__(256) void k_embed_fwd(const I *tok, const float *P, int64_t ldp, EmbedArgs a, int shift,
                                                   int64_t vectors, T *out) {
    constexpr int kRows = forward_rows<T>;
    typedef T Four __attribute__((ext_vector_type(4)));
    typedef T FourAnywhere __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const int64_t m = blockIdx.y;
    const int lanes = 1 << shift, per = 256 >> shift, lane = threadIdx.x & (lanes - 1);
    const float *table = P + m * ldp + a.offset;
    tok += m * a.N;
    out += m * a.N * a.D;
    for (int64_t n = (static_cast<int64_t>(blockIdx.x) * per * kRows) + (threadIdx.x >> shift); n < a.N;
         n += static_cast<int64_t>(gridDim.x) * per * kRows) {
        const float *row[kRows];
        bool there[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int64_t i = n + u * per < a.N ? n + u * per : n;
            const I t = tok[i];
            there[u] = t >= 0 && static_cast<int64_t>(t) < a.V;
            row[u] = table + (there[u] ? static_cast<int64_t>(t) : 0) * a.D;
        }
        for (int64_t q = lane; q < vectors; q += lanes) {
            f32x4 f[kRows];
#pragma unroll
            for (int u = 0; u < kRows; ++u) f[u] = load_floats<float>(row[u] + 4 * q);
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                if (n + u * per >= a.N) break;
                f[u] = there[u] ? f[u] * a.scale : f32x4(0.0f);
                FourAnywhere *to = reinterpret_cast<FourAnywhere *>(out + (n + u * per) * a.D + 4 * q);
                const Four v = __builtin_convertvector(f[u], Four);
                if (STREAM)
                    __builtin_nontemporal_store(v, to);
                else
                    *to = v;
            }
        }
        const int64_t c = 4 * vectors + lane;
        if (c < a.D) {
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                if (n + u * per < a.N)
                    out[(n + u * per) * a.D + c] = static_cast<T>(there[u] ? row[u][c] * a.scale : 0.0f);
        }
    }
}

// Zeros to n floats from `to` on, in vectors from a 16-byte boundary on; thread
// `tid` of `threads`.
__device__ __forceinline__ void fill(float *to, int64_t n, int64_t tid, int64_t threads) {
    const int64_t ahead = (16 - (reinterpret_cast<uintptr_t>(to) & 15)) / 4 & 3, head = ahead < n ? ahead : n;
    const int64_t quads = (n - head) / 4;
    f32x4 *v = reinterpret_cast<f32x4 *>(to + head);
    for (int64_t q = tid; q < quads; q += threads) v[q] = 0.0f;
    if (tid < head) to[tid] = 0.0f;
    if (tid < n - head - 4 * quads) to[head + 4 * quads + tid] = 0.0f;
}

// A worker's tokens to sort: padded places count as token V, behind all others.
template <typename I>
__device__ __forceinline__ uint32_t key_of(const I *tok, int64_t i, int64_t V) {
    const I t = tok[i];
    return t >= 0 && static_cast<int64_t>(t) < V ? static_cast<uint32_t>(t) : static_cast<uint32_t>(V);
}

// Stable sort of one run by digits from the lowest up, in registers and LDS.  A
// wave owns 256 consecutive places and, of the counters [digit][wave], its own
// column; a lane finds the lanes of its wave with its digit by one ballot a bit.
// 4096 tokens of 15 bits, two passes: 8.5 us, of 16 runs at a time 11.3; each
// pass is five waits for the whole workgroup.
template <typename I>
__device__ void sort_run(const I *tok, int64_t begin, int64_t N, int64_t V, int bits, int passes, uint32_t *key,
                         uint32_t *at) {
    __shared__ __align__(16) uint16_t count[kSortWaves << kDigitMost];
    __shared__ uint32_t keys[kRun];
    __shared__ uint16_t places[kRun];
    __shared__ uint32_t total[kSortWaves];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, mine = wave * 64 * kEach + lane;
    const int each = (kSortWaves << bits) / kSortThreads;  // counters per thread
    uint32_t k[kEach], rank[kEach];
    uint16_t place[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = mine + 64 * j;
        k[j] = begin + i < N ? key_of(tok, begin + i, V) : static_cast<uint32_t>(V);
        place[j] = static_cast<uint16_t>(i);
    }
    for (int p = 0; p < passes; ++p) {
        const int shift = p * bits;
        for (int i = tid; i < (kSortWaves << bits) / 2; i += kSortThreads) reinterpret_cast<uint32_t *>(count)[i] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const uint32_t digit = k[j] >> shift & ((1u << bits) - 1);
            uint64_t same = ~uint64_t(0);
            for (int b = 0; b < bits; ++b) {
                const bool set = digit >> b & 1;
                const uint64_t with = __ballot(set);
                same &= set ? with : ~with;
            }
            volatile uint16_t *slot = &count[digit * kSortWaves + wave];
            const uint32_t first = *slot;
            const int before = __popcll(same & ((uint64_t(1) << lane) - 1));
            if (before == 0) *slot = static_cast<uint16_t>(first + __popcll(same));
            rank[j] = first + before;
        }
        __syncthreads();
        // exclusive sums over [digit][wave]
        uint32_t sum = 0;
        for (int i = 0; i < each; ++i) sum += count[tid * each + i];
        const uint32_t upto = wave_prefix(sum);
        if (lane == 63) total[wave] = upto;
        __syncthreads();
        const uint32_t totals = row_prefix(total[lane & (kSortWaves - 1)]);
        uint32_t base = upto - sum + (wave > 0 ? __builtin_amdgcn_readlane(totals, wave > 0 ? wave - 1 : 0) : 0);
        for (int i = 0; i < each; ++i) {
            const uint32_t c = count[tid * each + i];
            count[tid * each + i] = static_cast<uint16_t>(base);
            base += c;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const uint32_t to = count[(k[j] >> shift & ((1u << bits) - 1)) * kSortWaves + wave] + rank[j];
            keys[to] = k[j];
            places[to] = place[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            k[j] = keys[mine + 64 * j];
            place[j] = places[mine + 64 * j];
        }
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int64_t i = begin + mine + 64 * j;  // what lies beyond N came last and stays there
        if (i < N) {
            key[i] = k[j];
            at[i] = static_cast<uint32_t>(begin + place[j]);
        }
    }
}

template <typename I>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(const I *tok, EmbedArgs a, int runs, int sorts, int bits,
                                                             int passes, uint32_t *key, uint32_t *at, int fills, float *G) {
    if (static_cast<int>(blockIdx.x) < sorts) {
        const int64_t first = static_cast<int64_t>(blockIdx.x / runs) * a.N;
        sort_run(tok + first, static_cast<int64_t>(blockIdx.x % runs) * kRun, a.N, a.V, bits, passes, key + first,
                 at + first);
        return;
    }
    // an equal part of a table's part of G, in whole quads
    const int64_t b = blockIdx.x - sorts, m = b / fills, len = a.V * a.D, each = ((len + fills - 1) / fills + 3) & ~int64_t(3);
    const int64_t first = (b % fills) * each;
    if (first < len)
        fill(G + m * a.ld + a.offset + first, len - first < each ? len - first : each, threadIdx.x, kSortThreads);
}

// Runs of `len` places (at least a workgroup's 256) to runs of kFan * len: a
// token's new place is its place in its run plus, for each other run, how many of
// its tokens come before.  A wave holds 64 neighbours of a sorted run: first its
// lanes search for its first and its last token, 16 lanes a run, each of which
// looks at one of the 16 places that cut what is left in 17; the other tokens'
// counts lie between those two, most often some 64 places apart.  Every step waits
// for memory, so searches go side by side.  65536 tokens: two launches of 7.5 us,
// of 16 workers 23 us each; one launch that joins 16 runs 17.8 and 73.
__global__ __launch_bounds__(256) void k_embed_merge(const uint32_t *key, const uint32_t *at, int N, int len,
                                                     uint32_t *to_key, uint32_t *to_at) {
    constexpr int kCuts = 64 / kFan;  // lanes a run
    constexpr uint64_t kEachRun = ~uint64_t(0) / ((uint64_t(1) << kFan) - 1);  // every kFan-th bit
    const int first = static_cast<int>(blockIdx.x) * 256, i = first + threadIdx.x, lane = threadIdx.x & 63;
    const int64_t m = blockIdx.y;
    key += m * N;
    at += m * N;
    const int run = first / len, group = run / kFan * kFan;
    const bool in = i < N;
    const uint32_t k = key[in ? i : N - 1], where = at[in ? i : N - 1];
    uint32_t ends[2] = {0, 0};  // counts of the wave's first and last token in run group + lane % kFan
    {
        const int r = lane % kFan, j = lane / kFan;
        const int64_t begin = static_cast<int64_t>(group + r) * len;
        const uint32_t here = begin >= N || group + r == run ? 0 : static_cast<uint32_t>(N - begin < len ? N - begin : len);
        const uint32_t mine[2] = {static_cast<uint32_t>(__builtin_amdgcn_readlane(k, 0)) + (group + r < run),
                                  static_cast<uint32_t>(__builtin_amdgcn_readlane(k, 63)) + (group + r < run)};
        uint32_t left[2] = {here, here};  // the count is in [ends, ends + left]
        while (__ballot((left[0] | left[1]) != 0) != 0) {
            bool before[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t cut = ends[e] + static_cast<uint32_t>(uint64_t(j + 1) * (left[e] + 1) / (kCuts + 1));
                before[e] = cut <= ends[e] || key[begin + cut - 1] < mine[e];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int yes = __popcll(__ballot(before[e]) >> r & kEachRun);  // of this run's lanes
                const uint32_t n = left[e], low = ends[e];
                if (yes > 0) ends[e] = low + static_cast<uint32_t>(uint64_t(yes) * (n + 1) / (kCuts + 1));
                const uint32_t high = yes < kCuts ? low + static_cast<uint32_t>(uint64_t(yes + 1) * (n + 1) / (kCuts + 1)) - 1 : low + n;
                left[e] = high - ends[e];
            }
        }
    }
    uint32_t less[kFan], most[kFan], width = 0;
#pragma unroll
    for (int r = 0; r < kFan; ++r) {
        less[r] = __builtin_amdgcn_readlane(ends[0], r);
        most[r] = __builtin_amdgcn_readlane(ends[1], r);
        width = most[r] - less[r] > width ? most[r] - less[r] : width;
    }
    for (int step = width == 0 ? 0 : 1 << (31 - __builtin_clz(width)); step > 0; step >>= 1) {
#pragma unroll
        for (int r = 0; r < kFan; ++r) {
            const uint32_t upto = less[r] + step;
            // equal tokens of earlier runs come before, of later ones behind
            if (upto <= most[r] && key[static_cast<int64_t>(group + r) * len + upto - 1] < k + (group + r < run))
                less[r] = upto;
        }
    }
    int64_t to = static_cast<int64_t>(group) * len + (i - run * len);
#pragma unroll
    for (int r = 0; r < kFan; ++r) to += less[r];
    if (!in) return;
    to_key[m * N + to] = k;
    to_at[m * N + to] = where;
}

// A lane's channels: sixteen bytes of dout (`whole`), and one of the last D % kPer
// in the first lanes of the last slab (`tail`).  `from` and `from_tail` are places
// within the row for the lanes without any too, so that loads need no branch.
template <typename T>
struct Channels {
    typedef typename Vec16<T>::wide Wide;
    static constexpr int kPer = Vec16<T>::kPer;
    int64_t c, ct, from, from_tail;  // first channel, tail channel
    bool whole, tail, some_whole, some_tail;
    __device__ __forceinline__ Channels(int64_t D, int slab, int slabs, int width, int lane) {
        const int64_t vectors = D / kPer, q = static_cast<int64_t>(slab) * width + lane;
        whole = lane < width && q < vectors;
        c = kPer * q;
        ct = kPer * vectors + lane;
        tail = slab == slabs - 1 && ct < D;
        some_whole = vectors > 0;
        some_tail = slab == slabs - 1 && kPer * vectors < D;
        from = whole ? c : 0;
        from_tail = tail ? ct : D - 1;
    }
    __device__ __forceinline__ void put(float *to, Wide s, float t, float scale, bool add) const {
        if (whole) {
            Wide f = s * scale;
            if (add) f += load_floats<T>(to + c);
            store_floats<T>(to + c, f);
        }
        if (tail) to[ct] = add ? to[ct] + t * scale : t * scale;
    }
    __device__ __forceinline__ void leave(float *to, Wide s, float t) const {
        if (whole) store_floats<T>(to + c, s);
        if (tail) to[ct] = t;
    }
};

constexpr int kBatch = 8;
// Workgroups of all workers' first rows come first: tokens of low number are the
// frequent ones in most vocabularies, and their sums take longest (16 workers, 192
// tokens, 30000 x 64 29.8 us so and 39 worker by worker).  Against the launches of
// more, 192 tokens for each of M workers' tables of V x D (bf16): 1 x 1000 x 1024
// 8.4 and 16.7 us, 1 x 32000 x 1024 26.9 and 34.3, 8 x 150 x 64 13.8 and 16.0, 26 x
// 53776 x 77 85 and 92, 16 x 30000 x 64 29.8 and 34.3.  A token that comes
// N times is N rows one after the other, so that more are not better off here.
constexpr int kFewRounds = 3, kFew = 64 * kFewRounds, kFewWaves = 8, kFewBatch = 4;
template <typename T, typename I>
__global__ __launch_bounds__(64 * kFewWaves) void k_embed_few(const I *tok, const T *dout, EmbedArgs a, uint32_t workers,
                                                              int64_t rows, int slabs, int width, float *G, bool add) {
    const int64_t m = blockIdx.x % workers, row0 = static_cast<int64_t>(blockIdx.x / workers) * rows;
    const int64_t mine = a.V - row0 < rows ? a.V - row0 : rows;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    dout += m * a.N * a.D;
    G += m * a.ld + a.offset + row0 * a.D;
    uint32_t row[kFewRounds];
    uint64_t todo[kFewRounds], any = 0;
#pragma unroll
    for (int j = 0; j < kFewRounds; ++j) {
        const int i = 64 * j + lane;
        const int64_t t = i < a.N ? static_cast<int64_t>(tok[m * a.N + i]) : -1;
        const bool hit = t >= row0 && t < row0 + mine;
        row[j] = hit ? static_cast<uint32_t>(t - row0) : UINT32_MAX;
        todo[j] = __ballot(hit);
        any |= todo[j];
    }
    if (!add) fill(G, mine * a.D, tid, 64 * kFewWaves);
    if (any == 0) return;
    __syncthreads();  // the zeros come before the sums
    int task = 0;
#pragma unroll
    for (int j = 0; j < kFewRounds; ++j) {
        while (todo[j] != 0) {
            const uint32_t r = __builtin_amdgcn_readlane(row[j], __ffsll(static_cast<long long>(todo[j])) - 1);
            uint64_t of_row[kFewRounds];
#pragma unroll
            for (int i = 0; i < kFewRounds; ++i) {
                of_row[i] = i < j ? 0 : __ballot(row[i] == r);
                todo[i] &= ~of_row[i];
            }
            for (int slab = 0; slab < slabs; ++slab, ++task) {
                if (task % kFewWaves != wave) continue;
                const Channels<T> ch(a.D, slab, slabs, width, lane);
                typename Vec16<T>::wide s = 0.0f;
                float last_s = 0.0f;
#pragma unroll
                for (int i = 0; i < kFewRounds; ++i) {
                    for (uint64_t same = of_row[i]; same != 0;) {
                        const T *from[kFewBatch];
                        int count = 0;
#pragma unroll
                        for (int u = 0; u < kFewBatch; ++u) {
                            if (same != 0) {
                                from[u] = dout + (64 * i + __ffsll(static_cast<long long>(same)) - 1) * a.D;
                                same &= same - 1;
                                ++count;
                            } else {
                                from[u] = from[0];
                            }
                        }
                        typename Vec16<T>::type raw[kFewBatch];
                        typename Bits<T>::type last[kFewBatch];
                        if (ch.some_whole) {
#pragma unroll
                            for (int u = 0; u < kFewBatch; ++u) raw[u] = load16(from[u] + ch.from);
                        }
                        if (ch.some_tail) {
#pragma unroll
                            for (int u = 0; u < kFewBatch; ++u) last[u] = load_bits(from[u] + ch.from_tail);
                        }
#pragma unroll
                        for (int u = 0; u < kFewBatch; ++u) {
                            if (u >= count) break;
                            if (ch.some_whole) s += widen<T>(raw[u]);
                            if (ch.some_tail) last_s += widen_bits<T>(last[u]);
                        }
                    }
                }
                ch.put(G + static_cast<int64_t>(r) * a.D, s, last_s, a.scale, add);
            }
        }
    }
}

// A task is CHUNK sorted places and one slab of the row, done by L lanes.
template <typename T, int L, int CHUNK, bool STREAM>
__global__ __launch_bounds__(256) void k_embed_sum(const uint32_t *key, const uint32_t *at, const T *dout, EmbedArgs a,
                                                   int64_t chunks, int slabs, int width, float *part, float *G, bool add) {
    constexpr int kSeen = 2 * CHUNK, kGroups = 256 / L;  // places of a chunk and the next
    constexpr bool kWave = L == 64;
    static_assert(kSeen <= 64 && (kWave || kSeen % L == 0), "a bit for each place");
    __shared__ uint32_t keys[kWave ? 1 : kGroups][kWave ? 1 : kSeen], places[kWave ? 1 : kGroups][kWave ? 1 : kSeen];
    const int64_t m = blockIdx.y, task = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / L;
    if (task >= chunks * slabs) return;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int64_t chunk = task / slabs;
    const Channels<T> ch(a.D, static_cast<int>(task % slabs), slabs, width, lane);
    const int64_t e0 = chunk * CHUNK;
    key += m * a.N;
    at += m * a.N;
    dout += m * a.N * a.D;
    G += m * a.ld + a.offset;
    part += (m * chunks + chunk) * 2 * a.D;
    const uint32_t V = static_cast<uint32_t>(a.V);
    const uint32_t before = e0 > 0 ? key[e0 - 1] : V;
    const uint32_t earlier = e0 > CHUNK ? key[e0 - CHUNK - 1] : V;  // the last place before the chunk before
    const uint32_t behind = e0 + kSeen < a.N ? key[e0 + kSeen] : V;
    // bit i: the token at place e0 + i ends there; is none (padded places come last)
    uint64_t ends = 0, none = 0;
    uint32_t k = V, where = 0;
    if constexpr (kWave) {  // lane i: place e0 + i
        k = e0 + lane < a.N ? key[e0 + lane] : V;
        where = e0 + lane < a.N ? at[e0 + lane] : 0;
        uint32_t next = __shfl_down(k, 1);
        if (lane == kSeen - 1) next = behind;
        ends = __ballot(k != next);
        none = __ballot(k == V);
    } else {
        constexpr int kEach = kSeen / L;
        uint32_t mine[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int64_t e = e0 + L * j + lane;
            mine[j] = e < a.N ? key[e] : V;
            places[group][L * j + lane] = e < a.N ? at[e] : 0;
            keys[group][L * j + lane] = mine[j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // a group lies in one wave
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const uint32_t across = j + 1 < kEach ? __shfl(mine[j + 1 < kEach ? j + 1 : j], 0, L) : behind;
            uint32_t next = __shfl_down(mine[j], 1, L);
            if (lane == L - 1) next = across;
            const int base = (threadIdx.x & 63) / L * L;
            ends |= (__ballot(mine[j] != next) >> base & ((uint64_t(1) << L) - 1)) << (L * j);
            none |= (__ballot(mine[j] == V) >> base & ((uint64_t(1) << L) - 1)) << (L * j);
        }
    }
    if constexpr (kSeen < 64) {
        ends &= (uint64_t(1) << kSeen) - 1;
        none |= ~uint64_t(0) << kSeen;
    }
    const auto key_at = [&](int e) {
        return kWave ? static_cast<uint32_t>(__builtin_amdgcn_readlane(k, e)) : keys[kWave ? 0 : group][kWave ? 0 : e];
    };
    const auto place_at = [&](int e) {
        return kWave ? static_cast<uint32_t>(__builtin_amdgcn_readlane(where, e)) : places[kWave ? 0 : group][kWave ? 0 : e];
    };
    const int valid = __popcll(~none);
    const uint32_t head = key_at(0);
    // places of the token that began in an earlier chunk, and whether it was that chunk's to finish
    const int led = head != V && head == before ? (ends != 0 ? __ffsll(static_cast<long long>(ends)) : 65) : 0;
    const bool finished = led <= CHUNK && earlier != head;
    int first = led > 0 && finished ? led : 0;
    bool leading = led > 0 && !finished;  // its partial sum comes first
    // to the end of the last token that begins here, if that is in sight
    int n = valid < CHUNK ? valid : CHUNK;
    if (n == CHUNK && !(ends >> (CHUNK - 1) & 1)) {
        const bool mine = !(leading && led > CHUNK);  // it begins here
        const uint64_t later = ends >> CHUNK;
        if (mine && later != 0) n = CHUNK + __ffsll(static_cast<long long>(later));
    }
    typename Vec16<T>::wide s = 0.0f;
    float t = 0.0f;
    for (int b = first; b < n; b += kBatch) {
        const T *row[kBatch];
        typename Vec16<T>::type raw[kBatch];
        typename Bits<T>::type last[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)  // beyond n: this batch's first row once more
            row[u] = dout + static_cast<int64_t>(place_at(b + u < n ? b + u : b)) * a.D;
        if (ch.some_whole) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) raw[u] = load16<T, STREAM>(row[u] + ch.from);
        }
        if (ch.some_tail) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) last[u] = load_bits(row[u] + ch.from_tail);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (b + u >= n) break;
            if (ch.some_whole) s += widen<T>(raw[u]);
            if (ch.some_tail) t += widen_bits<T>(last[u]);
            const bool end = ends >> (b + u) & 1;
            if (!end && b + u + 1 < n) continue;
            if (!leading && end)
                ch.put(G + static_cast<int64_t>(key_at(b + u)) * a.D, s, t, a.scale, add);
            else
                ch.leave(part + (leading ? 0 : a.D), s, t);
            s = 0.0f;
            t = 0.0f;
            leading = false;
        }
    }
}

// Tokens that run on beyond the chunk after the one they begin in: that chunk's
// second partial sum and the first ones of those that follow, in this order.  One
// workgroup per kJoinChunks chunks and slab: its waves look at one chunk's border
// each and how far the token there goes; then its groups of L lanes take one such
// token each, and one of many chunks is shared out among them (a million places of
// one token, rows of 64 bf16: the whole gradient 208 us, and 846 when a wave took
// all its lanes for one partial sum and the token's chunks were counted 64 by 64).
constexpr int kJoinWaves = 8, kJoinChunks = kJoinWaves, kMany = 2 * kBatch;
template <typename T, int L, int CHUNK>
__global__ __launch_bounds__(64 * kJoinWaves) void k_embed_join(const uint32_t *key, EmbedArgs a, int64_t chunks, int slabs,
                                                                   int width, const float *part, float *G, bool add) {
    constexpr int kGroups = 64 * kJoinWaves / L, kPer = Vec16<T>::kPer, kAhead = (L == 64 ? 32 : 16) / kPer;
    static_assert(kJoinChunks <= kGroups, "a group for each token");
    __shared__ float sums[kGroups][L][kPer + 1], tails[kGroups][L];
    __shared__ int counts[kJoinChunks];  // chunks that begin with the token; 0: no such token
    __shared__ uint32_t tokens[kJoinChunks];
    typedef typename Vec16<T>::wide Wide;
    const int64_t m = blockIdx.y, from = static_cast<int64_t>(blockIdx.x / slabs) * kJoinChunks;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    key += m * a.N;
    G += m * a.ld + a.offset;
    part += m * chunks * 2 * a.D;
    const uint32_t V = static_cast<uint32_t>(a.V);
    {
        const int wave = threadIdx.x >> 6, probe = threadIdx.x & 63;
        const int64_t chunk = from + wave, e0 = chunk * CHUNK, e1 = e0 + CHUNK;
        int n = 0;
        uint32_t token = V;
        if (e1 + CHUNK < a.N) {
            token = key[e1 - 1];
            if (token != V && key[e1 + CHUNK] == token && !(e0 > 0 && key[e0 - 1] == token)) {
                // the first chunk that does not begin with it: 64 looked at in one go, apart
                // by steps that grow till one is past the token's end and then shrink
                int64_t last = chunk + 2;  // the one before begins with it
                for (int64_t step = 1;;) {
                    const int64_t e = (last + probe * step) * CHUNK;
                    const uint64_t others = ~__ballot(e < a.N && key[e < a.N ? e : 0] == token);
                    if (others == 0) {
                        last += 63 * step + 1;
                        step *= 64;
                        continue;
                    }
                    const int p = __ffsll(static_cast<long long>(others)) - 1;
                    if (step == 1 || p == 0) {
                        last += p;
                        break;
                    }
                    last += (p - 1) * step + 1;
                    step /= 64;
                }
                n = static_cast<int>(last - chunk - 1);
            }
        }
        if (probe == 0) {
            counts[wave] = n;
            tokens[wave] = token;
        }
    }
    __syncthreads();
    const Channels<T> ch(a.D, static_cast<int>(blockIdx.x % slabs), slabs, width, lane);
    Wide s = 0.0f;
    float t = 0.0f;
    // the second partial sum of chunk c and the first ones of chunks [first, upto)
    const auto begin = [&](int64_t c) {
        const float *p = part + (2 * c + 1) * a.D;
        if (ch.whole) s = load_floats<T>(p + ch.c);
        if (ch.tail) t = p[ch.ct];
    };
    const auto go_on = [&](int64_t first, int64_t upto) {
        for (int64_t b = first; b < upto; b += kAhead) {
            const float *p = part + 2 * b * a.D;
            if (ch.some_whole) {
                Wide f[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) f[u] = load_floats<T>(p + (b + u < upto ? 2 * u * a.D : 0) + ch.from);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (b + u < upto) s += f[u];
            }
            if (ch.some_tail) {
                float f[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) f[u] = p[(b + u < upto ? 2 * u * a.D : 0) + ch.from_tail];
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (b + u < upto) t += f[u];
            }
        }
    };
    if (group < kJoinChunks && counts[group] > 0 && counts[group] <= kMany) {
        const int64_t chunk = from + group;
        begin(chunk);
        go_on(chunk + 1, chunk + 1 + counts[group]);
        ch.put(G + static_cast<int64_t>(tokens[group]) * a.D, s, t, a.scale, add);
    }
    for (int i = 0; i < kJoinChunks; ++i) {
        const int n = counts[i];
        if (n <= kMany) continue;
        const int64_t chunk = from + i, each = (n + kGroups - 1) / kGroups, first = chunk + 1 + group * each;
        const int64_t end = chunk + 1 + n;
        s = 0.0f;
        t = 0.0f;
        if (group == 0) begin(chunk);
        go_on(first, first + each < end ? first + each : end);
        __syncthreads();  // the one before has been read
#pragma unroll
        for (int c = 0; c < kPer; ++c) sums[group][lane][c] = s[c];
        tails[group][lane] = t;
        __syncthreads();
        if (group != 0) continue;
        for (int g = 1; g < kGroups; ++g) {
#pragma unroll
            for (int c = 0; c < kPer; ++c) s[c] += sums[g][lane][c];
            t += tails[g][lane];
        }
        ch.put(G + static_cast<int64_t>(tokens[i]) * a.D, s, t, a.scale, add);
    }
}

// ---------------------------------------------------------------------------

constexpr int64_t kMostGroups = int64_t(1) << 24;  // bound of a launch's workgroups of 256 threads: 2^32 threads

// The vectors of a row in equal shares of up to 64, one per wave.
int slabs_of(int64_t D, int per) {
    const int64_t s = ceil_div(D / per, 64);
    return static_cast<int>(s < 1 ? 1 : s);
}
int width_of(int64_t D, int per) { return static_cast<int>(ceil_div(D / per, slabs_of(D, per))); }

constexpr int kChunkLong = 32, kChunkShort = 8;
// Sorted places per wave of k_embed_sum: few where its waves would be up to four
// per CU.  Whole gradients (bf16, M x N tokens, V x D), us with 32 and with 8:
// 1 x 256, 3000 x 64 22.2 / 16.3; 1 x 2048, 3000 x 768 28.3 / 20.9; 8 x 2048,
// 3000 x 512 33.5 / 28.4; 1 x 16384, 3000 x 768 43.0 / 39.3; behind the bound 2 x
// 20000, 1000 x 1024 51.3 / 57.4, 32 x 4096, 1000 x 64 36.9 / 50.9.
int chunk_of(int64_t M, const dqgan_embed_desc *d) {
    const int64_t waves = M * ceil_div(d->tokens, kChunkLong) * slabs_of(d->width, d->type == DQGAN_F32 ? 4 : 8);
    return waves <= 1024 ? kChunkShort : kChunkLong;
}
// f(L, CHUNK): of rows of up to 256 bytes a wave sums several chunks.  16 x 65536
// tokens, 3000 x 128 bf16 204 us a wave a chunk and 180 so, of 3000 x 64 196 and
// 152; 32 lanes a chunk of 512 byte rows made no difference.
template <typename F>
void with_task(int chunk, int width, F &&f) {
    using std::integral_constant;
    if (chunk == kChunkShort)
        f(integral_constant<int, 64>{}, integral_constant<int, kChunkShort>{});
    else if (width <= 8)
        f(integral_constant<int, 8>{}, integral_constant<int, kChunkLong>{});
    else if (width <= 16)
        f(integral_constant<int, 16>{}, integral_constant<int, kChunkLong>{});
    else
        f(integral_constant<int, 64>{}, integral_constant<int, kChunkLong>{});
}

// Rows of a workgroup of k_embed_few: 8 to 128 KB of G, to fill the card, and up
// to 64, as the tokens among them are added one wave each (192 tokens, bf16: 16 x
// 30000 x 64 29.8 us so and 34.5 with 512, 26 x 53776 x 77 84.6 and 93.7).
constexpr int64_t kFewRowsMost = 64, kFewGroupsMost = int64_t(1) << 22;
int64_t few_rows(int64_t M, int64_t V, int64_t D) {
    int64_t floats = M * V * D / 4096;
    if (floats < 2048) floats = 2048;
    if (floats > kFillFloats) floats = kFillFloats;
    int64_t rows = floats / D;
    if (rows < 1) rows = 1;
    if (rows > kFewRowsMost) rows = kFewRowsMost;
    const int64_t least = ceil_div(M * V, kFewGroupsMost);  // a launch has fewer than 2^32 threads
    return rows < least ? least : rows;
}

dqgan_status check(dqgan_plan P, const dqgan_embed_desc *d) {
    if (!P || !d) return DQGAN_EINVAL;
    const int64_t n = P->desc.d;
    if (d->vocab < 1 || d->vocab > INT32_MAX - 1 || d->width < 1 || d->width > kMaxWidth) return DQGAN_EINVAL;
    if (d->offset < 0 || d->offset >= n || d->vocab > (n - d->offset) / d->width) return DQGAN_EINVAL;
    if (!tokens_ok(P, d->tokens) || !type_ok(d->type) || d->reserved != 0 || !isfinite(d->scale)) return DQGAN_EINVAL;
    if (d->index_type != DQGAN_I32 && d->index_type != DQGAN_I64) return DQGAN_EINVAL;
    // k_embed_join's workgroups of 512 threads, and with them k_embed_sum's of 256
    const int64_t slabs = slabs_of(d->width, d->type == DQGAN_F32 ? 4 : 8);
    if (ceil_div(ceil_div(d->tokens, kChunkLong), kJoinChunks) * slabs >= kMostGroups / 2) return DQGAN_EINVAL;
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

// Whether `out` passes by the caches.  Rows of whole vectors from 30 MB on: 134 MB of
// 1024 bf16 47 us so and 53 not, 40 MB 14.4 and 15.5, of 64 11.9 and 12.5; 20 MB the
// same.  The lines of other rows come in pieces, from vectors and single channels:
// from 60 MB on (40 MB of 138 bf16 20.2 and 17.8, 60 MB 26.9 and 29.2, of 203 f32 14.3
// and 13.5, 19.2 and 21.3) if they have 256 bytes (800 MB: 138 bf16 363 and 366, 71 f32
// 338 and 341, but 57 f32 430 and 298, 71 bf16 542 and 479), or from 65 to 160 MB, about
// what the Infinity Cache takes, if they have 140 (71 bf16: 60 MB 37 and 34, 80 MB 47
// and 54, 150 MB 95 and 102, 220 MB 159 and 143; 117: 70 MB 32 and 36).
bool forward_streams(double bytes, int64_t D, int64_t size) {
    if (D % 4 == 0) return bytes > 30e6;
    return D * size >= 256 ? bytes > 60e6 : D * size >= 140 && bytes > 65e6 && bytes < 160e6;
}
// Whether dout passes by the caches: 268 MB 148 us (the whole gradient) so and 181
// not, 134 MB 356 and 365, 33 MB 118 and 114.
bool backward_streams(double bytes) { return bytes > 100e6; }

size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

// The workspace: lists of tokens and of their places (two pairs where runs are
// merged), then the partial sums.
size_t list_bytes(int64_t M, int64_t N) { return round256(sizeof(uint32_t) * static_cast<size_t>(M * N)); }
int pairs_of(int64_t N) { return N > kRun ? 2 : 1; }

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
    // At least the four lanes of the last D % 4 channels; from 32 lanes on, one more
    // channel for up to half of them: 11 x 50469 tokens, rows of 561 to bf16 233 us, 275
    // with 256 lanes for 140 vectors; rows of 138 105 and 119.  With one more for all of
    // them rows of 1280 lose (83 us and 73), with 16 lanes those of 71 (162 and 146).
    const auto reach = [](int64_t lanes) { return 4 * lanes + (lanes >= 32 ? lanes / 2 : 0); };
    int shift = 2;
    while (shift < 8 && reach(int64_t(1) << shift) < a.D) ++shift;
    const int64_t lanes = int64_t(1) << shift, vectors = a.D <= reach(lanes) && a.D > 4 * lanes ? lanes : a.D >> 2;
    with_type(d->type, [&](auto t) {
        with_index(d->index_type, [&](auto i) {
            using T = decltype(t);
            using I = decltype(i);
            const int64_t groups = ceil_div(a.N, forward_rows<T> * (256 >> shift));
            const dim3 grid(static_cast<uint32_t>(groups < 65536 ? groups : 65536), static_cast<uint32_t>(P->desc.M));
            if (forward_streams(static_cast<double>(sizeof(T)) * P->desc.M * a.N * a.D, a.D, sizeof(T)))
                k_embed_fwd<T, I, true><<<grid, 256, 0, st>>>(static_cast<const I *>(tok), params, ldp, a, shift, vectors,
                                                              static_cast<T *>(out));
            else
                k_embed_fwd<T, I, false><<<grid, 256, 0, st>>>(static_cast<const I *>(tok), params, ldp, a, shift, vectors,
                                                               static_cast<T *>(out));
        });
    });
    return launched();
}

dqgan_status dqgan_embed_bytes(dqgan_plan P, const dqgan_embed_desc *d, size_t *bytes) {
    DQ_TRY(check(P, d));
    if (!bytes) return DQGAN_EINVAL;
    const int64_t M = P->desc.M;
    *bytes = d->tokens <= kFew ? 0
                            : 2 * pairs_of(d->tokens) * list_bytes(M, d->tokens) +
                                  sizeof(float) * 2 * static_cast<size_t>(M * ceil_div(d->tokens, chunk_of(M, d))) * d->width;
    return DQGAN_OK;
}

dqgan_status dqgan_embed_backward(dqgan_plan P, const dqgan_embed_desc *d, const void *tok, const void *dout, float *G,
                                  int32_t add, void *workspace, void *stream) {
    DQ_TRY(check(P, d));
    const bool any = d->tokens > 0;
    DQ_TRY(check_ptr(tok, any));
    DQ_TRY(check_ptr(dout, any));
    DQ_TRY(check_ptr(G));
    DQ_TRY(check_ptr(workspace, d->tokens > kFew));
    DQ_TRY(check_device(P));
    hipStream_t st = static_cast<hipStream_t>(stream);
    const EmbedArgs a = args(P, d);
    const int64_t M = P->desc.M;
    if (a.N <= kFew) {
        if (!any && add) return DQGAN_OK;
        const int64_t rows = few_rows(M, a.V, a.D);
        with_type(d->type, [&](auto t) {
            with_index(d->index_type, [&](auto i) {
                using T = decltype(t);
                using I = decltype(i);
                k_embed_few<T, I><<<static_cast<uint32_t>(M * ceil_div(a.V, rows)), 64 * kFewWaves, 0, st>>>(
                    static_cast<const I *>(tok), static_cast<const T *>(dout), a, static_cast<uint32_t>(M), rows,
                    slabs_of(a.D, Vec16<T>::kPer), width_of(a.D, Vec16<T>::kPer), G, add != 0);
            });
        });
        return launched();
    }
    const size_t list = list_bytes(M, a.N);
    uint32_t *key[2], *at[2];
    for (int i = 0; i < 2; ++i) {
        key[i] = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + 2 * i * list);
        at[i] = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + (2 * i + 1) * list);
    }
    float *part = reinterpret_cast<float *>(static_cast<char *>(workspace) + 2 * pairs_of(a.N) * list);
    int bits = 1;  // of the largest key, V
    while ((a.V >> bits) != 0) ++bits;
    const int passes = (bits + kDigitMost - 1) / kDigitMost;
    int digit = (bits + passes - 1) / passes;
    if (digit < 6) digit = 6;  // 1024 counters at least: one per thread
    const int64_t want = ceil_div(a.V * a.D, kFillFloats), most = kMostGroups / 8 / M;
    const int fills = add ? 0 : static_cast<int>(want < most ? want : most);
    const int runs = static_cast<int>(ceil_div(a.N, kRun)), sorts = static_cast<int>(M * runs);
    const int64_t groups = sorts + M * fills;
    with_index(d->index_type, [&](auto i) {
        using I = decltype(i);
        k_embed_sort<I><<<static_cast<uint32_t>(groups), kSortThreads, 0, st>>>(
            static_cast<const I *>(tok), a, runs, sorts, digit, passes, key[0], at[0], fills, G);
    });
    int now = 0;
    for (int64_t len = kRun; len < a.N; len *= kFan, now ^= 1)
        k_embed_merge<<<dim3(static_cast<uint32_t>(ceil_div(a.N, 256)), static_cast<uint32_t>(M)), 256, 0, st>>>(
            key[now], at[now], static_cast<int>(a.N), static_cast<int>(len), key[now ^ 1], at[now ^ 1]);
    const int chunk = chunk_of(M, d);
    const int64_t chunks = ceil_div(a.N, chunk);
    with_type(d->type, [&](auto t) {
        using T = decltype(t);
        const int slabs = slabs_of(a.D, Vec16<T>::kPer), width = width_of(a.D, Vec16<T>::kPer);
        const uint32_t my = static_cast<uint32_t>(M);
        with_task(chunk, width, [&](auto l, auto c) {
            constexpr int L = decltype(l)::value, C = decltype(c)::value;
            const dim3 grid(static_cast<uint32_t>(ceil_div(chunks * slabs, 256 / L)), my);
            with_stream(backward_streams(static_cast<double>(sizeof(T)) * M * a.N * a.D), [&](auto streams) {
                // short chunks are of 34 MB of dout at most
                k_embed_sum<T, L, C, decltype(streams)::value && C == kChunkLong><<<grid, 256, 0, st>>>(
                    key[now], at[now], static_cast<const T *>(dout), a, chunks, slabs, width, part, G, add != 0);
            });
            if (chunks > 2)
                k_embed_join<T, L, C><<<dim3(static_cast<uint32_t>(ceil_div(chunks, kJoinChunks) * slabs), my), 64 * kJoinWaves, 0,
                                     st>>>(key[now], a, chunks, slabs, width, part, G, add != 0);
        });
    });
    return launched();
}

}  // extern "C"
