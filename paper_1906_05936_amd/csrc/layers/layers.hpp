// What the layer operators share: argument checks without host allocations,
// under-aligned vector accesses, the 8-bit format.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../lsgd_host.hpp"
#include "../lsgd_kernels.hpp"
#include "../../../include/layers/lsgd_layers.h"

#pragma clang fp contract(off)

namespace lsgd {
namespace layers {

constexpr int64_t kMaxDim = 0x7fffffff;

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ------------------------------------------------------------------ host checks

inline lsgd_status check_dtype(lsgd_dtype t, const char* what) {
    return t == LSGD_F32 || t == LSGD_BF16 ? LSGD_OK : fail(LSGD_ERR_DTYPE, "%s=%d", what, static_cast<int>(t));
}
inline lsgd_status check_size(int64_t n, const char* what) {
    return n >= 0 && n <= kMaxDim ? LSGD_OK
                                  : fail(LSGD_ERR_SIZE, "%s=%lld outside [0, 2^31)", what, static_cast<long long>(n));
}
// A matrix of at most 2^46 elements: byte counts and offsets stay within 64 bits.
inline lsgd_status check_matrix(int64_t rows, int64_t cols, const char* what) {
    return rows == 0 || cols <= (int64_t{1} << 46) / rows
               ? LSGD_OK
               : fail(LSGD_ERR_SIZE, "%s of %lld x %lld elements", what, static_cast<long long>(rows),
                      static_cast<long long>(cols));
}
inline lsgd_status check_buffer(const void* p, uintptr_t align, const char* what) {
    if (!p) return fail(LSGD_ERR_NULL, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(p) & (align - 1))
        return fail(LSGD_ERR_ALIGN, "%s is not %d-byte aligned", what, static_cast<int>(align));
    return LSGD_OK;
}
inline int64_t elem_size(lsgd_dtype t) { return t == LSGD_F32 ? 4 : 2; }

// LSGD_ERR_ALIAS if one of the `written` ranges overlaps another range. In the order
// of their addresses a range overlaps one before it if the furthest end so far lies
// behind its begin. (128 copies and 128 transposed ones: 9 us of host time; all
// pairs took 255.)
template <int N>
struct Ranges {
    Range r[N];
    int n = 0;
    void add(const void* p, int64_t bytes, bool written, const char* what) {
        const uintptr_t b = reinterpret_cast<uintptr_t>(p);
        if (bytes > 0) r[n++] = Range{b, b + static_cast<uintptr_t>(bytes), written, what};
    }
    lsgd_status check() {
        std::sort(r, r + n, [](const Range& x, const Range& y) { return x.begin < y.begin; });
        const Range *furthest = nullptr, *furthest_written = nullptr;
        for (const Range* i = r; i != r + n; ++i) {
            const Range* before = i->written ? furthest : furthest_written;
            if (before && i->begin < before->end)
                return fail(LSGD_ERR_ALIAS, "written buffer %s overlaps %s", i->written ? i->what : before->what,
                            i->written ? before->what : i->what);
            if (!furthest || furthest->end < i->end) furthest = i;
            if (i->written && (!furthest_written || furthest_written->end < i->end)) furthest_written = i;
        }
        return LSGD_OK;
    }
};

// 8-bit matrices: bytes from row to row, and of the whole buffers.
__host__ __device__ inline int64_t pitch8(int64_t cols) { return ceil_div(cols, 128) * 128; }
__host__ __device__ inline int64_t scale_pitch8(int64_t cols) { return ceil_div(ceil_div(cols, 128), 4) * 4; }
inline int64_t codes_bytes(int64_t rows, int64_t cols) { return rows * pitch8(cols); }
inline int64_t scales_bytes(int64_t rows, int64_t cols, int64_t block) {
    return ceil_div(rows, block) * scale_pitch8(cols);
}

#define LSGD_TRY(expr)                                 \
    do {                                               \
        const lsgd_status st_ = (expr);                \
        if (st_ != LSGD_OK) return st_;                \
    } while (0)


// ------------------------------------------------------------------ device side

// Rows of an odd length start anywhere: these types carry the alignment of one
// element, and gfx950 loads and stores them with one 128-bit instruction.
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_u2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_u2 __attribute__((ext_vector_type(2), aligned(2)));

__device__ __forceinline__ float bf16_to_f32(uint32_t h) { return __builtin_bit_cast(float, h << 16); }

// Nearest-even (one instruction for two numbers); a NaN stays one.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t f32_to_bf16x2(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
__device__ __forceinline__ uint32_t f32_to_bf16(float f) { return f32_to_bf16x2(f, 0.0f) & 0xffffu; }

// Elements [0, k) of the 8 at p (k in [0, 8]; those behind stay 0).
__device__ __forceinline__ void load8(const float* p, int k, float (&x)[8]) {
    if (k >= 8) {
        const f32x4_u a = *reinterpret_cast<const f32x4_u*>(p), b = *reinterpret_cast<const f32x4_u*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < k ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void load8(const uint16_t* p, int k, float (&x)[8]) {
    if (k >= 8) {
        const u32x4_u2 a = *reinterpret_cast<const u32x4_u2*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[2 * i] = bf16_to_f32(a[i] & 0xffffu), x[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < k ? bf16_to_f32(p[i]) : 0.0f;
    }
}
// The same for what is read once only: it does not stay in the caches.
__device__ __forceinline__ void load8_once(const uint16_t* p, int k, float (&x)[8]) {
    if (k < 8) return load8(p, k, x);
    const u32x4_u2 a = __builtin_nontemporal_load(reinterpret_cast<const u32x4_u2*>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x[2 * i] = bf16_to_f32(a[i] & 0xffffu), x[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
}
__device__ __forceinline__ void store8(uint16_t* p, int k, const float (&x)[8]) {
    if (k >= 8) {
        u32x4_u2 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = f32_to_bf16x2(x[2 * i], x[2 * i + 1]);
        *reinterpret_cast<u32x4_u2*>(p) = a;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < k) p[i] = static_cast<uint16_t>(f32_to_bf16(x[i]));
    }
}

// A wave's 512 columns from `col` on, in two halves of 256 with 4 neighbours per
// lane each (col: the lane's first), so that every instruction of a wave covers
// whole cache lines; elements past `dim` read as 0 and are not written. (8
// neighbours per lane leave two binary32 stores of 16 bytes with gaps of 16, which
// wrote at 4.3 TB/s instead of 6.)
__device__ __forceinline__ int64_t slab_column(int64_t slab, uint32_t lane) { return slab * 512 + lane * 4; }

__device__ __forceinline__ void load4(const float* p, int k, float* x) {
    if (k >= 4) {
        const f32x4_u a = *reinterpret_cast<const f32x4_u*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < k ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void load4(const uint16_t* p, int k, float* x) {
    if (k >= 4) {
        const u32x2_u2 a = *reinterpret_cast<const u32x2_u2*>(p);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            x[2 * i] = bf16_to_f32(a[i] & 0xffffu), x[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < k ? bf16_to_f32(p[i]) : 0.0f;
    }
}
// The first k of four neighbours.
__device__ __forceinline__ void store4(float* p, int k, f32x4 v) {
    if (k >= 4) {
        *reinterpret_cast<f32x4_u*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < k) p[i] = v[i];
    }
}
__device__ __forceinline__ void store4(uint16_t* p, int k, f32x4 v) {
    if (k >= 4) {
        *reinterpret_cast<u32x2_u2*>(p) = u32x2_u2{f32_to_bf16x2(v[0], v[1]), f32_to_bf16x2(v[2], v[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < k) p[i] = static_cast<uint16_t>(f32_to_bf16(v[i]));
    }
}
// row: the row's first element.
template <typename T>
__device__ __forceinline__ void load_slab(const T* row, int64_t col, int64_t dim, float (&x)[8]) {
    const int64_t left = dim - col;
    load4(row + col, static_cast<int>(min(left, static_cast<int64_t>(4))), x);
    load4(row + col + 256, static_cast<int>(min(left - 256, static_cast<int64_t>(4))), x + 4);
}
// The same for a row that is read once only.
__device__ __forceinline__ void load4_once(const float* p, int k, float* x) {
    if (k < 4) return load4(p, k, x);
    const f32x4_u a = __builtin_nontemporal_load(reinterpret_cast<const f32x4_u*>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i];
}
__device__ __forceinline__ void load4_once(const uint16_t* p, int k, float* x) {
    if (k < 4) return load4(p, k, x);
    const u32x2_u2 a = __builtin_nontemporal_load(reinterpret_cast<const u32x2_u2*>(p));
#pragma unroll
    for (int i = 0; i < 2; ++i)
        x[2 * i] = bf16_to_f32(a[i] & 0xffffu), x[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
}
template <typename T>
__device__ __forceinline__ void load_slab_once(const T* row, int64_t col, int64_t dim, float (&x)[8]) {
    const int64_t left = dim - col;
    load4_once(row + col, static_cast<int>(min(left, static_cast<int64_t>(4))), x);
    load4_once(row + col + 256, static_cast<int>(min(left - 256, static_cast<int64_t>(4))), x + 4);
}
template <typename T>
__device__ __forceinline__ void store_slab(T* row, int64_t col, int64_t dim, const float (&x)[8]) {
    const int64_t left = dim - col;
    store4(row + col, static_cast<int>(min(left, static_cast<int64_t>(4))), f32x4{x[0], x[1], x[2], x[3]});
    store4(row + col + 256, static_cast<int>(min(left - 256, static_cast<int64_t>(4))), f32x4{x[4], x[5], x[6], x[7]});
}

// |x| where x is finite, else 0.
__device__ __forceinline__ float finite_abs(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
    return u < 0x7f800000u ? __builtin_bit_cast(float, u) : 0.0f;
}

// The scale byte of a block whose largest finite magnitude is `a`: exponent e
// + 127 with the smallest e in [-126, 127] for which a <= 448 * 2^e = 1.75 *
// 2^(e+8). For a = 1.f * 2^E that is E - 8, one more where 1.f > 1.75. A
// subnormal a (E field 0) lies far below 448 * 2^-126, the least scale's range.
__device__ __forceinline__ uint32_t scale_byte(float a) {
    const uint32_t u = __builtin_bit_cast(uint32_t, a);
    if (u == 0) return 127u;
    const int e = static_cast<int>(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return static_cast<uint32_t>(e < 1 ? 1 : e);
}
// 2^-(e) for the byte e + 127 in [1, 247]: exact, normal.
__device__ __forceinline__ float inverse_scale(uint32_t byte) {
    return __builtin_bit_cast(float, (254u - byte) << 23);
}

// Four codes (nearest-even; every |x| <= 448, or NaN or infinity, which become NaN).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}

}  // namespace layers
}  // namespace lsgd
