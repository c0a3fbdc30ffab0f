// A linear layer's parameter gradient from its activations in 8 bits
// (lsgd_layers.h).
#include "mfma.hpp"

namespace lsgd {
namespace layers {
namespace {

constexpr int kStep = 64;                   // rows of grad and x a step adds up
constexpr int kTile = 128;                  // outputs of a workgroup, each way; one block of x's scales
constexpr int kRowBytes = kTile * 2;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Byte offset of columns [16 p, 16 p + 16) of a row in an LDS tile: the 32-byte
// pieces of a row are exchanged so that the four rows (and two of the four
// lane groups) of a transposing read meet different banks.
__device__ __forceinline__ int piece_at(int row, int p) {
    return row * kRowBytes + ((p ^ ((row & 3) | (row >> 1 & 4))) << 5);
}

// Both operands lie with the summed axis as their rows, while the matrix
// instruction wants 8 neighbours along it in a lane: LDS holds 64 rows of 128
// columns of both in bfloat16, and ds_read_b64_tr_b16 hands each lane four
// rows of its column. The codes become bfloat16 on their way into LDS. The next
// step's global loads run during the products. With gridDim.z > 1 a workgroup
// sums its share of the rows into its part of the workspace.
template <typename OT>
__global__ __launch_bounds__(256) void weight_grad8_kernel(const uint16_t* __restrict__ grad,
                                                           const uint8_t* __restrict__ x,
                                                           const uint8_t* __restrict__ scales, int64_t m, int64_t n,
                                                           int64_t k, int64_t pitch, int64_t spitch, int64_t share,
                                                           OT* __restrict__ out, float* __restrict__ parts,
                                                           bool accumulate) {
    __shared__ __align__(16) uint8_t lds[2][2][kStep * kRowBytes];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t k0 = static_cast<int64_t>(blockIdx.x) * kTile, n0 = static_cast<int64_t>(blockIdx.y) * kTile;
    const int64_t begin = blockIdx.z * share, end = min(begin + share, m);
    const int wk = wave % 2 * 64, wn = wave / 2 * 64;

    // this lane's part of a step: 8 columns of grad in 4 rows, 16 of x in 2
    u32x4 g[4], c[2];
    uint32_t s[2];
    const int gc = t % 16 * 8;
    const int gk = static_cast<int>(max(static_cast<int64_t>(0), min(n - n0 - gc, static_cast<int64_t>(8))));
    auto fetch = [&](int64_t row0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = row0 + i * 16 + t / 16;
            const uint16_t* p = grad + r * n + n0 + gc;
            if (r < end && gk == 8) {
                const u32x4_u2 v = *reinterpret_cast<const u32x4_u2*>(p);
                g[i] = u32x4{v[0], v[1], v[2], v[3]};
            } else {
                const int kk = r < end ? gk : 0;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    g[i][j] = (2 * j < kk ? p[2 * j] : 0u) | (2 * j + 1 < kk ? static_cast<uint32_t>(p[2 * j + 1]) << 16 : 0u);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t r = row0 + i * 32 + t / 8;
            c[i] = u32x4{0, 0, 0, 0};
            s[i] = 127;
            if (r < end) {
                c[i] = *reinterpret_cast<const u32x4*>(x + r * pitch + k0 + t % 8 * 16);
                s[i] = scales[r * spitch + blockIdx.x];
            }
        }
    };
    auto keep = [&](int stage) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = i * 16 + t / 16;
            *reinterpret_cast<u32x4*>(&lds[stage][0][piece_at(row, t % 16 / 2) + t % 2 * 16]) = g[i];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = i * 32 + t / 8;
            const float f = scale_value(s[i]);
            const u32x2 a = widen4(c[i][0], f), b = widen4(c[i][1], f), d = widen4(c[i][2], f), e = widen4(c[i][3], f);
            u32x4* to = reinterpret_cast<u32x4*>(&lds[stage][1][piece_at(row, t % 8)]);
            to[0] = u32x4{a[0], a[1], b[0], b[1]};
            to[1] = u32x4{d[0], d[1], e[0], e[1]};
        }
    };

    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    if (begin < end) {
        fetch(begin);
        keep(0);
    }
    __syncthreads();
    int stage = 0;
    for (int64_t row0 = begin; row0 < end; row0 += kStep, stage ^= 1) {
        const bool more = row0 + kStep < end;
        if (more) fetch(row0 + kStep);
        // 8 rows along the sum for column 16 p + lane % 16
        auto fragment = [&](const uint8_t* tile, int half, int p) {
            const int row = half * 32 + lane / 16 * 8 + lane % 16 / 4;
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + piece_at(row, p) + lane % 4 * 8));
            const s16x4 b =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + piece_at(row + 4, p) + lane % 4 * 8));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        };
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            bf16x8 fx[4], fg[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) fx[j] = fragment(lds[stage][1], half, wk / 16 + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) fg[i] = fragment(lds[stage][0], half, wn / 16 + i);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[j], fg[i], acc[i][j], 0, 0, 0);
        }
        if (more) keep(stage ^ 1);
        __syncthreads();
    }
    float* part = gridDim.z > 1 ? parts + static_cast<int64_t>(blockIdx.z) * n * k : nullptr;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = n0 + wn + i * 16 + lane % 16;
        if (row >= n) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t col = k0 + wk + j * 16 + lane / 16 * 4;
            const int left = static_cast<int>(min(k - col, static_cast<int64_t>(4)));
            if (left <= 0) continue;
            if (part) {
                store4(part + row * k + col, left, acc[i][j]);
            } else {
                OT* o = out + row * k + col;
                f32x4 v = acc[i][j];
                if (accumulate)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (u < left) v[u] += value_of(o[u]);
                store4(o, left, v);
            }
        }
    }
}

// out (+)= the sum of the parts, in order.
template <typename OT>
__global__ __launch_bounds__(kBlock) void add_parts_kernel(const float* __restrict__ parts, int64_t n, int count,
                                                           OT* __restrict__ out, bool accumulate) {
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * 4;
    if (i >= n) return;
    const int left = static_cast<int>(min(n - i, static_cast<int64_t>(4)));
    f32x4 v{0, 0, 0, 0};
    for (int c = 0; c < count; ++c) {
        const float* p = parts + c * n + i;
        if (left == 4) {
            v += *reinterpret_cast<const f32x4_u*>(p);
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] += u < left ? p[u] : 0.0f;
        }
    }
    if (accumulate)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (u < left) v[u] += value_of(out[i + u]);
    store4(out + i, left, v);
}

// Shares of the summed rows: as many as give every compute unit two workgroups,
// of 256 rows at least.
struct Split {
    int64_t share;
    int count;
};
Split split_of(int64_t m, int64_t n, int64_t k) {
    const int64_t tiles = ceil_div(n, kTile) * ceil_div(k, kTile);
    const int64_t want = std::max<int64_t>(1, std::min(ceil_div(m, 256), 512 / tiles));
    const int64_t share = ceil_div(ceil_div(m, want), kStep) * kStep;
    return Split{share, static_cast<int>(std::max<int64_t>(1, ceil_div(m, share)))};
}

template <typename OT>
lsgd_status launch(const void* grad, const void* x, const void* scales, int64_t m, int64_t n, int64_t k, void* out,
                   bool accumulate, void* workspace, hipStream_t s) {
    const Split sp = m > 0 ? split_of(m, n, k) : Split{kStep, 1};
    float* parts = static_cast<float*>(workspace);
    const dim3 grid(static_cast<unsigned>(ceil_div(k, kTile)), static_cast<unsigned>(ceil_div(n, kTile)),
                    static_cast<unsigned>(sp.count));
    hipLaunchKernelGGL((weight_grad8_kernel<OT>), grid, dim3(256), 0, s, static_cast<const uint16_t*>(grad),
                       static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(scales), m, n, k, pitch8(k),
                       scale_pitch8(k), sp.share, static_cast<OT*>(out), parts, accumulate);
    LSGD_TRY(check_launch("lsgd_weight_grad8"));
    if (sp.count > 1) {
        hipLaunchKernelGGL((add_parts_kernel<OT>), dim3(static_cast<unsigned>(ceil_div(n * k, 4 * kBlock))),
                           dim3(kBlock), 0, s, parts, n * k, sp.count, static_cast<OT*>(out), accumulate);
        LSGD_TRY(check_launch("lsgd_weight_grad8"));
    }
    return LSGD_OK;
}

lsgd_status check_sizes(int64_t m, int64_t n, int64_t k) {
    LSGD_TRY(check_size(m, "m"));
    LSGD_TRY(check_size(n, "n"));
    LSGD_TRY(check_size(k, "k"));
    LSGD_TRY(check_matrix(m, n, "grad"));
    LSGD_TRY(check_matrix(m, k, "x"));
    LSGD_TRY(check_matrix(n, k, "out"));
    return ceil_div(n, kTile) <= 65535
               ? LSGD_OK
               : fail(LSGD_ERR_SIZE, "n=%lld above 65535 * 128", static_cast<long long>(n));
}

size_t workspace_bytes_of(int64_t m, int64_t n, int64_t k) {
    if (m == 0 || n == 0 || k == 0) return 0;
    const Split sp = split_of(m, n, k);
    return sp.count > 1 ? static_cast<size_t>(sp.count) * n * k * 4 : 0;
}

}  // namespace
}  // namespace layers
}  // namespace lsgd

using namespace lsgd;
using namespace lsgd::layers;

extern "C" {

LSGD_API lsgd_status lsgd_weight_grad8_workspace_size(int64_t m, int64_t n, int64_t k, size_t* bytes) {
    LSGD_TRY(check_sizes(m, n, k));
    if (!bytes) return fail(LSGD_ERR_NULL, "bytes is NULL");
    *bytes = workspace_bytes_of(m, n, k);
    return LSGD_OK;
}

LSGD_API lsgd_status lsgd_weight_grad8(const void* grad, const void* x, const void* x_scales, int64_t m, int64_t n,
                                       int64_t k, void* out, lsgd_dtype odt, int32_t accumulate, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    LSGD_TRY(check_dtype(odt, "out dtype"));
    LSGD_TRY(check_sizes(m, n, k));
    if (n == 0 || k == 0 || (m == 0 && accumulate)) return LSGD_OK;
    LSGD_TRY(check_buffer(out, 16, "out"));
    const size_t need = workspace_bytes_of(m, n, k);
    if (m > 0) {
        LSGD_TRY(check_buffer(grad, 16, "grad"));
        LSGD_TRY(check_buffer(x, 16, "x"));
        LSGD_TRY(check_buffer(x_scales, 16, "x_scales"));
        Ranges<5> ranges;
        ranges.add(grad, m * n * 2, false, "grad");
        ranges.add(x, codes_bytes(m, k), false, "x");
        ranges.add(x_scales, scales_bytes(m, k, 1), false, "x_scales");
        ranges.add(out, n * k * elem_size(odt), true, "out");
        if (need > 0) {
            LSGD_TRY(check_buffer(workspace, 256, "workspace"));
            if (workspace_bytes < need)
                return fail(LSGD_ERR_SIZE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
            ranges.add(workspace, static_cast<int64_t>(need), true, "workspace");
        }
        LSGD_TRY(ranges.check());
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    return odt == LSGD_F32 ? launch<float>(grad, x, x_scales, m, n, k, out, accumulate != 0, workspace, s)
                           : launch<uint16_t>(grad, x, x_scales, m, n, k, out, accumulate != 0, workspace, s);
}

}  // extern "C"
