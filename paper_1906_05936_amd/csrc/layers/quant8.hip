// Activations and parameters in 8 bits (lsgd_layers.h): codes, and a
// power-of-two scale for each block.
#include <type_traits>

#include "layers.hpp"

namespace lsgd {
namespace layers {
namespace {

// The largest of the 16 lanes of a row, in all of them.
__device__ __forceinline__ float max_of_16(float a) {
    const auto turned = [](float x, auto by) {   // by lanes, within the row
        constexpr int ctrl = 0x120 + decltype(by)::value;
        return __builtin_bit_cast(
            float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xf, 0xf, true));
    };
    a = fmaxf(a, turned(a, std::integral_constant<int, 8>{}));
    a = fmaxf(a, turned(a, std::integral_constant<int, 4>{}));
    a = fmaxf(a, turned(a, std::integral_constant<int, 2>{}));
    return fmaxf(a, turned(a, std::integral_constant<int, 1>{}));
}

// Block 1. A wave takes 512 columns of a row, a lane 8 of them: 16 lanes hold a
// block of 128, whose largest magnitude goes round by lane exchanges; the four
// scales leave as one word. Bound by the bytes of x read and codes written, as
// long as it takes few instructions: fmaxf passes NaNs over, and only where an
// infinity is left are the magnitudes looked at again. 16384 x 4096 bfloat16: 35 us,
// 5.8 TB/s; with x kept in the caches, or a wave for every 512 columns, 39 to 42.
// For binary32 a lane has 4 columns in either half of the block, so that an
// instruction reads whole lines, and neighbouring workgroups take the same rows, a
// wave for every 512 columns: 16384 x 4096 53 us, 6.4 TB/s, with 8 neighbours a lane and
// neighbouring workgroups along the rows, as for bfloat16, 75; 16384 x 4095 62 and 71,
// 8192 x 8191 60 and 69, 333 x 1999 3.2 and 3.4, 5000 x 129 3.9 and 3.6. For bfloat16
// the order of the workgroups makes 34 of 35 us at 16384 x 4096, but 43 of 38 at 8192 x
// 8191 and 24 of 21 at 4096 x 8191.
template <typename T>
__global__ __launch_bounds__(kBlock) void quant_rows_kernel(const T* __restrict__ x, int64_t rows, int64_t cols,
                                                            int64_t pitch, int64_t spitch, uint32_t groups,
                                                            uint8_t* __restrict__ codes,
                                                            uint8_t* __restrict__ scales) {
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr bool kHalves = sizeof(T) == 4;
    const uint32_t at = kHalves ? blockIdx.y : blockIdx.x, of = kHalves ? gridDim.y : gridDim.x;
    const uint32_t first = kHalves ? blockIdx.x : blockIdx.y, step = kHalves ? gridDim.x : gridDim.y;
    for (int64_t r = static_cast<int64_t>(at) * (kBlock / 64) + wave; r < rows; r += static_cast<int64_t>(of) * (kBlock / 64)) {
        for (uint32_t g = first; g < groups; g += step) {
            const int64_t c = static_cast<int64_t>(g) * 512 + (kHalves ? lane / 16 * 128 + lane % 16 * 4 : lane * 8);
            const auto inside = [&](int64_t from, int64_t most) {
                return static_cast<int>(max(static_cast<int64_t>(0), min(cols - from, most)));
            };
            float v[8];
            if constexpr (kHalves) {
                load4_once(x + r * cols + c, inside(c, 4), v);
                load4_once(x + r * cols + c + 64, inside(c + 64, 4), v + 4);
            } else {
                load8_once(x + r * cols + c, inside(c, 8), v);
            }
            float a = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(v[i]));
            if (__ballot(a == __builtin_inff())) {
                a = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) a = fmaxf(a, finite_abs(v[i]));
            }
            const uint32_t byte = scale_byte(max_of_16(a));
            const float inv = inverse_scale(byte);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= inv;
            const uint32_t lo = codes4(v[0], v[1], v[2], v[3]), hi = codes4(v[4], v[5], v[6], v[7]);
            if (c < pitch) {
                uint8_t* q = codes + r * pitch + c;
                if constexpr (kHalves) {
                    *reinterpret_cast<uint32_t*>(q) = lo;
                    *reinterpret_cast<uint32_t*>(q + 64) = hi;
                } else {
                    *reinterpret_cast<u32x2*>(q) = u32x2{lo, hi};
                }
            }
            const uint32_t word = __builtin_amdgcn_readlane(byte, 0) | __builtin_amdgcn_readlane(byte, 16) << 8 |
                                  __builtin_amdgcn_readlane(byte, 32) << 16 |
                                  static_cast<uint32_t>(__builtin_amdgcn_readlane(byte, 48)) << 24;
            if (lane == 0) *reinterpret_cast<uint32_t*>(scales + r * spitch + g * 4) = word;
        }
    }
}

// Block 128. A workgroup holds a tile of 128 x 128 parameters in registers (a
// lane: 4 rows by 4 columns), agrees on its largest magnitude, and brings the codes
// into LDS as they are and transposed, from where every copy is written in rows
// of 128 bytes. The transpose of each 4 x 4 happens in registers. Bound by the
// parameters read and the copies written (8192 x 2048, four copies and four
// transposed: 32 us, 6.3 TB/s; with stores through the caches 47; one copy and one
// transposed of 4096 x 4096, past the caches / through them: 22.2 / 23.4 us, with a product
// of 16 rows behind it 29.2 / 29.4, of 512 rows 57 / 53), and where the
// tiles are few by the way from load to store (1000 x 777: 4.9 us; with four 4 x 4 to
// each of a quarter of the lanes 7.3, and 33 for the large one). Up to kCopies copies
// a launch keep their pointers in the kernel's arguments; up to kLaunchTiles tiles
// side by side fit a launch, the next one starts at first_col.
constexpr int kTileThreads = 1024;
constexpr int64_t kLaunchTiles = 0xffffffffLL / kTileThreads;   // a dispatch holds at most 2^32 - 1 work-items along x
constexpr int kCopies = 32;
constexpr int kRowWords = 33;    // LDS words per row of 128 codes: rows start in different banks

struct Copies {
    uint8_t* codes[kCopies];
    uint8_t* scales[kCopies];
};

__device__ __forceinline__ void put_tile(const uint32_t (&tile)[128][kRowWords], uint32_t byte, const Copies& to,
                                         int n, int64_t rows, int64_t cols, int64_t r0, int64_t c0) {
    const int64_t pitch = pitch8(cols), spitch = scale_pitch8(cols);
    const int64_t blocks = pitch / 128, cb = c0 / 128;
    const int row = threadIdx.x / 8, w = threadIdx.x % 8 * 4;
    if (r0 + row < rows) {
        const u32x4 v{tile[row][w], tile[row][w + 1], tile[row][w + 2], tile[row][w + 3]};
        for (int k = 0; k < n; ++k)
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(to.codes[k] + (r0 + row) * pitch + c0 + w * 4));
    }
    // the scale, and behind the last block of columns the row's padding
    const int64_t end = cb == blocks - 1 ? spitch : cb + 1;
    for (int k = threadIdx.x; k < n; k += kTileThreads)
        for (int64_t s = cb; s < end; ++s)
            to.scales[k][r0 / 128 * spitch + s] = static_cast<uint8_t>(s == cb ? byte : 127u);
}

__global__ __launch_bounds__(kTileThreads) void quant_blocks_kernel(const float* __restrict__ p, int64_t rows,
                                                                    int64_t cols, int64_t first_col, Copies plain,
                                                                    int n_plain, Copies transposed, int n_transposed) {
    __shared__ uint32_t tile[128][kRowWords];
    __shared__ float wave_max[kTileThreads / 64];
    const int64_t c0 = first_col + static_cast<int64_t>(blockIdx.x) * 128, r0 = static_cast<int64_t>(blockIdx.y) * 128;
    const int tr = threadIdx.x / 32 * 4, tc = threadIdx.x % 32 * 4;
    const int k = static_cast<int>(max(static_cast<int64_t>(0), min(cols - c0 - tc, static_cast<int64_t>(4))));
    float v[4][4];
#pragma unroll
    for (int b = 0; b < 4; ++b) load4(p + (r0 + tr + b) * cols + c0 + tc, r0 + tr + b < rows ? k : 0, v[b]);
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, finite_abs((&v[0][0])[i]));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileThreads / 64; ++i) m = fmaxf(m, wave_max[i]);
    const uint32_t byte = scale_byte(m);
    const float inv = inverse_scale(byte);
    uint32_t q[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) q[b] = codes4(v[b][0] * inv, v[b][1] * inv, v[b][2] * inv, v[b][3] * inv);
    if (n_plain > 0) {
#pragma unroll
        for (int b = 0; b < 4; ++b) tile[tr + b][tc / 4] = q[b];
        __syncthreads();
        put_tile(tile, byte, plain, n_plain, rows, cols, r0, c0);
        __syncthreads();
    }
    if (n_transposed > 0) {
        // bytes of (row b, column j) -> (column j, row b)
        const uint32_t x0 = __builtin_amdgcn_perm(q[1], q[0], 0x05010400u);
        const uint32_t x1 = __builtin_amdgcn_perm(q[1], q[0], 0x07030602u);
        const uint32_t y0 = __builtin_amdgcn_perm(q[3], q[2], 0x05010400u);
        const uint32_t y1 = __builtin_amdgcn_perm(q[3], q[2], 0x07030602u);
        tile[tc][tr / 4] = __builtin_amdgcn_perm(y0, x0, 0x05040100u);
        tile[tc + 1][tr / 4] = __builtin_amdgcn_perm(y0, x0, 0x07060302u);
        tile[tc + 2][tr / 4] = __builtin_amdgcn_perm(y1, x1, 0x05040100u);
        tile[tc + 3][tr / 4] = __builtin_amdgcn_perm(y1, x1, 0x07060302u);
        __syncthreads();
        put_tile(tile, byte, transposed, n_transposed, cols, rows, c0, r0);
    }
}

}  // namespace
}  // namespace layers
}  // namespace lsgd

using namespace lsgd;
using namespace lsgd::layers;

extern "C" {

LSGD_API int64_t lsgd_pitch8(int64_t cols) { return pitch8(cols); }
LSGD_API int64_t lsgd_scale_pitch8(int64_t cols) { return scale_pitch8(cols); }

LSGD_API lsgd_status lsgd_quant8(const void* x, lsgd_dtype xdt, int64_t rows, int64_t cols, void* codes, void* scales,
                                 void* stream) {
    LSGD_TRY(check_dtype(xdt, "x dtype"));
    LSGD_TRY(check_size(rows, "rows"));
    LSGD_TRY(check_size(cols, "cols"));
    LSGD_TRY(check_matrix(rows, cols, "x"));
    if (rows == 0 || cols == 0) return LSGD_OK;
    LSGD_TRY(check_buffer(x, 16, "x"));
    LSGD_TRY(check_buffer(codes, 16, "codes"));
    LSGD_TRY(check_buffer(scales, 16, "scales"));
    Ranges<3> ranges;
    ranges.add(x, rows * cols * elem_size(xdt), false, "x");
    ranges.add(codes, codes_bytes(rows, cols), true, "codes");
    ranges.add(scales, scales_bytes(rows, cols, 1), true, "scales");
    LSGD_TRY(ranges.check());
    // bfloat16: a wave per 512 columns while that does not fill the card four times, then one for four
    const int64_t groups = ceil_div(cols, 512), full = 4 * 32 * static_cast<int64_t>(device_cus());
    const int64_t of_rows = ceil_div(rows, kBlock / 64);
    const int64_t across = std::min<int64_t>(1024, xdt == LSGD_F32 || rows * groups <= full ? groups : ceil_div(groups, 4));
    const dim3 grid = xdt == LSGD_F32
                          ? dim3(static_cast<unsigned>(across), static_cast<unsigned>(std::min<int64_t>(65535, of_rows)))
                          : dim3(static_cast<unsigned>(std::min<int64_t>(kMaxGridBlocks / across, of_rows)),
                                 static_cast<unsigned>(across));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (xdt == LSGD_F32)
        hipLaunchKernelGGL((quant_rows_kernel<float>), grid, dim3(kBlock), 0, s, static_cast<const float*>(x), rows,
                           cols, pitch8(cols), scale_pitch8(cols), static_cast<uint32_t>(groups),
                           static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales));
    else
        hipLaunchKernelGGL((quant_rows_kernel<uint16_t>), grid, dim3(kBlock), 0, s, static_cast<const uint16_t*>(x),
                           rows, cols, pitch8(cols), scale_pitch8(cols), static_cast<uint32_t>(groups),
                           static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales));
    return check_launch("lsgd_quant8");
}

LSGD_API lsgd_status lsgd_copy_out8(const float* params, int64_t rows, int64_t cols, void* const* codes,
                                    void* const* scales, int32_t n_replicas, void* const* codes_t,
                                    void* const* scales_t, int32_t n_transposed, void* stream) {
    if (n_replicas < 0 || n_replicas > LSGD_MAX_REPLICAS || n_transposed < 0 || n_transposed > LSGD_MAX_REPLICAS)
        return fail(LSGD_ERR_SIZE, "n_replicas=%d or n_transposed=%d outside [0, %d]", n_replicas, n_transposed,
                    LSGD_MAX_REPLICAS);
    LSGD_TRY(check_size(rows, "rows"));
    LSGD_TRY(check_size(cols, "cols"));
    LSGD_TRY(check_matrix(rows, cols, "params"));
    if (ceil_div(rows, 128) > 65535)
        return fail(LSGD_ERR_SIZE, "rows=%lld above 65535 * 128", static_cast<long long>(rows));
    if (rows == 0 || cols == 0 || n_replicas + n_transposed == 0) return LSGD_OK;
    LSGD_TRY(check_buffer(params, 16, "params"));
    if ((n_replicas && (!codes || !scales)) || (n_transposed && (!codes_t || !scales_t)))
        return fail(LSGD_ERR_NULL, "an array of copies is NULL");
    Ranges<4 * LSGD_MAX_REPLICAS + 1> ranges;
    ranges.add(params, rows * cols * 4, false, "params");
    for (int32_t i = 0; i < n_replicas; ++i) {
        LSGD_TRY(check_buffer(codes[i], 16, "a replica's codes"));
        LSGD_TRY(check_buffer(scales[i], 16, "a replica's scales"));
        ranges.add(codes[i], codes_bytes(rows, cols), true, "a replica's codes");
        ranges.add(scales[i], scales_bytes(rows, cols, 128), true, "a replica's scales");
    }
    for (int32_t i = 0; i < n_transposed; ++i) {
        LSGD_TRY(check_buffer(codes_t[i], 16, "a transposed replica's codes"));
        LSGD_TRY(check_buffer(scales_t[i], 16, "a transposed replica's scales"));
        ranges.add(codes_t[i], codes_bytes(cols, rows), true, "a transposed replica's codes");
        ranges.add(scales_t[i], scales_bytes(cols, rows, 128), true, "a transposed replica's scales");
    }
    LSGD_TRY(ranges.check());
    const int64_t tiles = ceil_div(cols, 128);
    for (int32_t at = 0; at < n_replicas || at < n_transposed; at += kCopies) {
        Copies a{}, b{};
        const int na = std::max(0, std::min(kCopies, n_replicas - at));
        const int nb = std::max(0, std::min(kCopies, n_transposed - at));
        for (int i = 0; i < na; ++i)
            a.codes[i] = static_cast<uint8_t*>(codes[at + i]), a.scales[i] = static_cast<uint8_t*>(scales[at + i]);
        for (int i = 0; i < nb; ++i)
            b.codes[i] = static_cast<uint8_t*>(codes_t[at + i]), b.scales[i] = static_cast<uint8_t*>(scales_t[at + i]);
        for (int64_t tile = 0; tile < tiles; tile += kLaunchTiles) {
            const dim3 grid(static_cast<unsigned>(std::min(kLaunchTiles, tiles - tile)),
                            static_cast<unsigned>(ceil_div(rows, 128)));
            hipLaunchKernelGGL(quant_blocks_kernel, grid, dim3(kTileThreads), 0, static_cast<hipStream_t>(stream), params,
                               rows, cols, tile * 128, a, na, b, nb);
            LSGD_TRY(check_launch("lsgd_copy_out8"));
        }
    }
    return LSGD_OK;
}

}  // extern "C"
