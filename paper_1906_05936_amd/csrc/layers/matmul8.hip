// The product of two 8-bit matrices over their columns (lsgd_layers.h).
#include "mfma.hpp"

namespace lsgd {
namespace layers {
namespace {

// One operand: codes, scales and how its rows share them.
struct Operand {
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t rows;
    int shift;   // log2(block): the scale row of row r is r >> shift
};

// A workgroup of WM x WN waves computes a tile of (WM * TM * 16) x (WN * TN *
// 16) outputs, 128 columns of a and b at a time, which the next step's loads
// (straight into LDS, no registers) overlap. LDS rows are 128 bytes, their
// 16-byte chunks exchanged by row % 8, so that the 8 rows of a fragment read
// meet all banks. b is the matrix instruction's first operand: a lane then holds
// 4 neighbouring columns of one output row.
template <int TM, int TN, int WM, int WN, bool Exact, typename OT>
__global__ __launch_bounds__(WM * WN * 64) void matmul8_kernel(Operand A, Operand B, int64_t pitch, int64_t spitch,
                                                               OT* __restrict__ out) {
    constexpr int kWaves = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16;
    __shared__ __align__(16) uint8_t lds[2][(BM + BN) * 128];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = static_cast<int64_t>(blockIdx.y) * BM, n0 = static_cast<int64_t>(blockIdx.x) * BN;
    const int wm = wave % WM * (TM * 16), wn = wave / WM * (TN * 16);
    const int steps = static_cast<int>(pitch / 128);

    // rows past the end repeat the last one; their outputs are not stored
    auto fetch = [&](int stage, int step) {
        constexpr int kLoads = (BM + BN) / 8;   // of 8 rows each
#pragma unroll
        for (int i = 0; i < kLoads / kWaves; ++i) {
            const int first = (i * kWaves + wave) * 8;
            const int row = first + lane / 8, chunk = (lane % 8) ^ (row % 8);
            const bool a = first < BM;
            const int64_t r = a ? min(m0 + row, A.rows - 1) : min(n0 + row - BM, B.rows - 1);
            load_lds16((a ? A.codes : B.codes) + r * pitch + step * 128 + chunk * 16, &lds[stage][first * 128]);
        }
    };
    const uint8_t* sa[TM];
    const uint8_t* sb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
        sa[i] = A.scales + (min(m0 + wm + i * 16 + lane % 16, A.rows - 1) >> A.shift) * spitch;
#pragma unroll
    for (int j = 0; j < TN; ++j)
        sb[j] = B.scales + (min(n0 + wn + j * 16 + lane % 16, B.rows - 1) >> B.shift) * spitch;

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    uint32_t wa[TM], wb[TN];
    fetch(0, 0);
    for (int base = 0; base < steps; base += 4) {
#pragma unroll
        for (int i = 0; i < TM; ++i) wa[i] = *reinterpret_cast<const uint32_t*>(sa[i] + base);
#pragma unroll
        for (int j = 0; j < TN; ++j) wb[j] = *reinterpret_cast<const uint32_t*>(sb[j] + base);
        unrolled<4>([&](auto ic) {
            constexpr int u = decltype(ic)::value;
            const int step = base + u;
            if (step >= steps) return;
            loads_done();
            if (step + 1 < steps) fetch((u + 1) & 1, step + 1);
            const uint8_t* t = lds[u & 1];
            auto fragment = [&](int row) {
                row += lane % 16;
                const int g = lane / 16;
                Codes32 f;
                f.half[0] = *reinterpret_cast<const u32x4*>(t + row * 128 + (g ^ (row % 8)) * 16);
                f.half[1] = *reinterpret_cast<const u32x4*>(t + row * 128 + ((g + 4) ^ (row % 8)) * 16);
                return f;
            };
            using Frag = typename Product<Exact>::Fragment;
            Frag fb[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = Product<Exact>::template prepare<u>(fragment(BM + wn + j * 16), wb[j]);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const Frag fa = Product<Exact>::template prepare<u>(fragment(wm + i * 16), wa[i]);
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = Product<Exact>::template multiply<u>(fb[j], wb[j], fa, wa[i], acc[i][j]);
            }
        });
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm + i * 16 + lane % 16;
        if (m >= A.rows) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + wn + j * 16 + lane / 16 * 4;
            const int64_t left = B.rows - n;
            if (left > 0) store4(out + m * B.rows + n, static_cast<int>(min(left, static_cast<int64_t>(4))), acc[i][j]);
        }
    }
}

template <typename OT>
__global__ __launch_bounds__(kBlock) void zero_kernel(OT* __restrict__ out, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kBlock)
        out[i] = 0;
}

template <bool Exact, typename OT>
lsgd_status launch(const Operand& a, const Operand& b, int64_t k, void* out, hipStream_t s) {
    if (k == 0) {
        const int64_t n = a.rows * b.rows;
        hipLaunchKernelGGL((zero_kernel<OT>), dim3(static_cast<unsigned>(std::min<int64_t>(4096, ceil_div(n, kBlock)))),
                           dim3(kBlock), 0, s, static_cast<OT*>(out), n);
        return check_launch("lsgd_matmul8");
    }
    const dim3 grid(static_cast<unsigned>(ceil_div(b.rows, 128)), static_cast<unsigned>(ceil_div(a.rows, 128)));
    hipLaunchKernelGGL((matmul8_kernel<4, 4, 2, 2, Exact, OT>), grid, dim3(256), 0, s, a, b, pitch8(k), scale_pitch8(k),
                       static_cast<OT*>(out));
    return check_launch("lsgd_matmul8");
}

}  // namespace
}  // namespace layers
}  // namespace lsgd

using namespace lsgd;
using namespace lsgd::layers;

extern "C" {

LSGD_API lsgd_status lsgd_matmul8(const void* a, const void* a_scales, int32_t a_block, int64_t m, const void* b,
                                  const void* b_scales, int32_t b_block, int64_t n, int64_t k, void* out,
                                  lsgd_dtype odt, void* stream) {
    LSGD_TRY(check_dtype(odt, "out dtype"));
    if ((a_block != 1 && a_block != 128) || (b_block != 1 && b_block != 128))
        return fail(LSGD_ERR_UNSUPPORTED, "blocks of %d and %d rows; 1 or 128 are supported", a_block, b_block);
    LSGD_TRY(check_size(m, "m"));
    LSGD_TRY(check_size(n, "n"));
    LSGD_TRY(check_size(k, "k"));
    LSGD_TRY(check_matrix(m, k, "a"));
    LSGD_TRY(check_matrix(n, k, "b"));
    LSGD_TRY(check_matrix(m, n, "out"));
    if (ceil_div(m, 128) > 65535) return fail(LSGD_ERR_SIZE, "m=%lld above 65535 * 128", static_cast<long long>(m));
    if (m == 0 || n == 0) return LSGD_OK;
    LSGD_TRY(check_buffer(out, 16, "out"));
    Ranges<5> ranges;
    ranges.add(out, m * n * elem_size(odt), true, "out");
    if (k > 0) {
        LSGD_TRY(check_buffer(a, 16, "a"));
        LSGD_TRY(check_buffer(a_scales, 16, "a_scales"));
        LSGD_TRY(check_buffer(b, 16, "b"));
        LSGD_TRY(check_buffer(b_scales, 16, "b_scales"));
        ranges.add(a, codes_bytes(m, k), false, "a");
        ranges.add(a_scales, scales_bytes(m, k, a_block), false, "a_scales");
        ranges.add(b, codes_bytes(n, k), false, "b");
        ranges.add(b_scales, scales_bytes(n, k, b_block), false, "b_scales");
        LSGD_TRY(ranges.check());
    }
    const Operand A{static_cast<const uint8_t*>(a), static_cast<const uint8_t*>(a_scales), m, a_block == 1 ? 0 : 7};
    const Operand B{static_cast<const uint8_t*>(b), static_cast<const uint8_t*>(b_scales), n, b_block == 1 ? 0 : 7};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return odt == LSGD_F32 ? launch<true, float>(A, B, k, out, s) : launch<false, uint16_t>(A, B, k, out, s);
}

}  // extern "C"
