// Shared parts of the layer operators (include/dqgan_layers.h): argument
// checks, access to activations of any type at any alignment, reductions over
// a wave and a workgroup.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/dqgan_layers.h"
#include "device.hpp"
#include "plan.hpp"

namespace dq {

// ---------------------------------------------------------------------------
// host: argument checks and dispatch

#define DQ_TRY(expr)                   \
    do {                               \
        dqgan_status s_ = (expr);      \
        if (s_ != DQGAN_OK) return s_; \
    } while (0)

constexpr int64_t kMaxRows = INT32_MAX;          // tokens of all workers together
constexpr int64_t kMaxTokens = int64_t(1) << 30;
constexpr int64_t kMaxWidth = int64_t(1) << 24;

// A device pointer that the call uses if `used`.
inline dqgan_status check_ptr(const void *p, bool used = true) {
    if (!p) return used ? DQGAN_EINVAL : DQGAN_OK;
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 ? DQGAN_OK : DQGAN_EALIGN;
}
inline dqgan_status check_device(const dqgan_plan_s *P) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return DQGAN_EHIP;
    return dev == P->device ? DQGAN_OK : DQGAN_EINVAL;
}
inline bool tokens_ok(const dqgan_plan_s *P, int64_t tokens) {
    return tokens >= 0 && tokens <= kMaxTokens && tokens * P->desc.M <= kMaxRows;
}
inline bool ldp_ok(const dqgan_plan_s *P, int64_t ldp) { return ldp == 0 || ldp == P->desc.ld; }
inline bool type_ok(int32_t t) { return t == DQGAN_F32 || t == DQGAN_BF16 || t == DQGAN_F16; }

// f(T{}) with T the C++ type of a dqgan_type.
template <typename F>
void with_type(int32_t type, F &&f) {
    if (type == DQGAN_F32)
        f(float{});
    else if (type == DQGAN_BF16)
        f(__bf16{});
    else
        f(_Float16{});
}

inline dqgan_status launched() { return hipGetLastError() == hipSuccess ? DQGAN_OK : DQGAN_EHIP; }

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------
// device: eight elements of a row per lane.  A row starts wherever an odd
// width or offset puts it, so vectors are aligned to their element only; the
// hardware loads and stores those in one instruction too.

typedef float f32x8 __attribute__((ext_vector_type(8)));
template <typename T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(8)));
    typedef T packed __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

// Sixteen bytes of a row: kPer elements.
template <typename T>
struct Vec16 {
    static constexpr int kPer = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef T packed __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    typedef float wide __attribute__((ext_vector_type(16 / sizeof(T))));
};

// Keeps the compiler from holding a row converted to 32 bits between two passes
// over it, which takes twice the registers.
template <typename V>
__device__ __forceinline__ void forget(V &raw) {
    typedef uint32_t Words __attribute__((ext_vector_type(sizeof(V) / 4)));
    Words w = __builtin_bit_cast(Words, raw);
#pragma unroll
    for (unsigned i = 0; i < sizeof(V) / 4; ++i) asm("" : "+v"(w[i]));
    raw = __builtin_bit_cast(V, w);
}

// The values are made here, and not where they are next used.
template <typename V>
__device__ __forceinline__ void settle(V &x) {
#pragma unroll
    for (unsigned i = 0; i < sizeof(V) / 4; ++i) {
        float f = x[i];
        asm volatile("" : "+v"(f));
        x[i] = f;
    }
}

// An element's bits: a load that is not converted where it is issued.
template <typename T>
struct Bits {
    typedef uint16_t type;
};
template <>
struct Bits<float> {
    typedef uint32_t type;
};
template <typename T>
__device__ __forceinline__ typename Bits<T>::type load_bits(const T *p) {
    return *reinterpret_cast<const typename Bits<T>::type *>(p);
}
template <typename T>
__device__ __forceinline__ float widen_bits(typename Bits<T>::type b) {
    return static_cast<float>(__builtin_bit_cast(T, b));
}

template <typename T, bool STREAM = false>
__device__ __forceinline__ typename Vec16<T>::type load16(const T *p) {
    const typename Vec16<T>::packed *v = reinterpret_cast<const typename Vec16<T>::packed *>(p);
    return STREAM ? __builtin_nontemporal_load(v) : *v;
}
template <typename T, bool STREAM = false>
__device__ __forceinline__ void store16(T *p, typename Vec16<T>::type v) {
    if (STREAM)
        __builtin_nontemporal_store(v, reinterpret_cast<typename Vec16<T>::packed *>(p));
    else
        *reinterpret_cast<typename Vec16<T>::packed *>(p) = v;
}
template <typename T>
__device__ __forceinline__ typename Vec16<T>::type narrow(typename Vec16<T>::wide v) {
    return __builtin_convertvector(v, typename Vec16<T>::type);
}
template <typename T>
__device__ __forceinline__ typename Vec16<T>::wide widen(typename Vec16<T>::type v) {
    return __builtin_convertvector(v, typename Vec16<T>::wide);
}
// As many floats of a parameter's row (a lane's channels of Vec16<T>).
template <typename T>
__device__ __forceinline__ typename Vec16<T>::wide load_floats(const float *p) {
    typedef float packed __attribute__((ext_vector_type(16 / sizeof(T)), aligned(4)));
    return *reinterpret_cast<const packed *>(p);
}
template <typename T>
__device__ __forceinline__ void store_floats(float *p, typename Vec16<T>::wide v) {
    typedef float packed __attribute__((ext_vector_type(16 / sizeof(T)), aligned(4)));
    *reinterpret_cast<packed *>(p) = v;
}

// p[0..8), of which n are there; the others come as `fill`.
template <typename T>
__device__ __forceinline__ f32x8 load8(const T *p, int64_t n, float fill = 0.0f) {
    if (n >= 8) {
        const typename Vec8<T>::type v = *reinterpret_cast<const typename Vec8<T>::packed *>(p);
        return __builtin_convertvector(v, f32x8);
    }
    f32x8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? static_cast<float>(p[i]) : fill;
    return f;
}
template <typename T>
__device__ __forceinline__ void store8(T *p, int64_t n, f32x8 f) {
    if (n >= 8) {
        const typename Vec8<T>::type v = __builtin_convertvector(f, typename Vec8<T>::type);
        *reinterpret_cast<typename Vec8<T>::packed *>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = static_cast<T>(f[i]);
}

// Sum and maximum over the 64 lanes, in every lane (DPP: within quads, rows of
// 16, then across rows).  The order of the sum is fixed.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_or(float old, float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, x),
                                                                 CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float lane63(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp_or<0xB1, 0xF>(0.0f, x);   // lane ^ 1
    x += dpp_or<0x4E, 0xF>(0.0f, x);   // lane ^ 2
    x += dpp_or<0x141, 0xF>(0.0f, x);  // half row mirrored
    x += dpp_or<0x140, 0xF>(0.0f, x);  // row mirrored: every lane has its row's sum
    x += dpp_or<0x142, 0xA>(0.0f, x);  // row 0 into row 1, row 2 into row 3
    x += dpp_or<0x143, 0xC>(0.0f, x);  // rows 0 and 1 into rows 2 and 3
    return lane63(x);
}
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, dpp_or<0xB1, 0xF>(x, x));
    x = fmaxf(x, dpp_or<0x4E, 0xF>(x, x));
    x = fmaxf(x, dpp_or<0x141, 0xF>(x, x));
    x = fmaxf(x, dpp_or<0x140, 0xF>(x, x));
    x = fmaxf(x, dpp_or<0x142, 0xA>(x, x));
    x = fmaxf(x, dpp_or<0x143, 0xC>(x, x));
    return lane63(x);
}

// Sum over this lane and those before it in its row of 16, and in the wave.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_zero(uint32_t x) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ uint32_t row_prefix(uint32_t x) {
    x += dpp_zero<0x111, 0xF>(x);
    x += dpp_zero<0x112, 0xF>(x);
    x += dpp_zero<0x114, 0xF>(x);
    x += dpp_zero<0x118, 0xF>(x);
    return x;
}
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x) {
    x = row_prefix(x);
    x += dpp_zero<0x142, 0xA>(x);
    x += dpp_zero<0x143, 0xC>(x);
    return x;
}

// Sum and maximum over groups of W consecutive lanes (4, 8 or 16), in each.
template <int W>
__device__ __forceinline__ float lanes_sum(float x) {
    x += dpp_or<0xB1, 0xF>(0.0f, x);
    x += dpp_or<0x4E, 0xF>(0.0f, x);
    if (W > 4) x += dpp_or<0x141, 0xF>(0.0f, x);
    if (W > 8) x += dpp_or<0x140, 0xF>(0.0f, x);
    return x;
}
template <int W>
__device__ __forceinline__ float lanes_max(float x) {
    x = fmaxf(x, dpp_or<0xB1, 0xF>(x, x));
    x = fmaxf(x, dpp_or<0x4E, 0xF>(x, x));
    if (W > 4) x = fmaxf(x, dpp_or<0x141, 0xF>(x, x));
    if (W > 8) x = fmaxf(x, dpp_or<0x140, 0xF>(x, x));
    return x;
}

// Sum over the W waves of a workgroup, in every lane: each wave reads the W
// sums side by side in its lanes and adds them up again.  `slot` is W floats of
// LDS that the next call does not use again (two slots in turn).
template <int W>
__device__ __forceinline__ float group_sum(float x, float *slot) {
    x = wave_sum(x);
    if (W == 1) return x;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = x;
    __syncthreads();
    return lanes_sum<W>(slot[threadIdx.x & (W - 1)]);
}
template <int W>
__device__ __forceinline__ float group_max(float x, float *slot) {
    x = wave_max(x);
    if (W == 1) return x;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = x;
    __syncthreads();
    return lanes_max<W>(slot[threadIdx.x & (W - 1)]);
}

}  // namespace dq
