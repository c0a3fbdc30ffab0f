// A linear layer's parameter gradient from its activations in 8 bits
// (lsgd_layers.h).
#include "mfma.hpp"

namespace lsgd {
namespace layers {
namespace {

// Four neighbours of the gradient, or of a part of it.
template <typename OT>
__device__ __forceinline__ void put4(float* part, OT* out, int64_t at, int left, f32x4 v, bool accumulate) {
    if (part) return store4(part + at, left, v);
    if (accumulate) {
        float before[4];
        load4(out + at, left, before);
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] += before[u];
    }
    store4(out + at, left, v);
}

constexpr int kStep = 64;      // rows of grad and x a stage adds up

typedef short s16x4 __attribute__((ext_vector_type(4)));

// 8 neighbours along the rows of the lane's column: the instruction hands each of 16
// lanes four rows of its column.
__device__ __forceinline__ bf16x8 read_transposed(const uint8_t* p, int four_rows) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + four_rows));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Rows [row0, row0 + 64) of both operands as far as they lie below `end` (at most
// m), from a tile's first column on. What lies behind counts as 0; columns past
// the tile's own matrix hold anything and meet outputs that are not stored. A
// buffer gives 0 for a word that is not wholly inside, and for an odd n the last
// element of a row begins one: there it reaches into the next row, but behind row
// m - 1 there is none, and add_last adds what that element gives.
struct Rows {
    Buffer grad, x, scales;
    __device__ __forceinline__ Rows(const uint16_t* g, const uint8_t* codes, const uint8_t* s, int64_t row0, int64_t end,
                                    int64_t m, int64_t n, int64_t n0, uint32_t pitch, uint32_t spitch, int64_t k0)
        : Rows(g, codes, s, row0, static_cast<uint32_t>(max(static_cast<int64_t>(0), min(end - row0, static_cast<int64_t>(kStep)))),
               n, n0, pitch, spitch, k0, end < m || row0 + kStep < m ? static_cast<uint32_t>(n) % 2 * 2 : 0) {}

private:
    static __device__ __forceinline__ uint32_t bytes(uint32_t rows, uint32_t row, uint32_t first, uint32_t more) {
        return rows ? rows * row - first + more : 0;
    }
    __device__ __forceinline__ Rows(const uint16_t* g, const uint8_t* codes, const uint8_t* s, int64_t row0, uint32_t rows,
                                    int64_t n, int64_t n0, uint32_t pitch, uint32_t spitch, int64_t k0, uint32_t more)
        : grad(g + row0 * n + n0, bytes(rows, static_cast<uint32_t>(n) * 2, static_cast<uint32_t>(n0) * 2, more)),
          x(codes + row0 * pitch + k0, bytes(rows, pitch, static_cast<uint32_t>(k0), 0)),
          scales(s + row0 * spitch + k0 / 128, bytes(rows, spitch, static_cast<uint32_t>(k0 / 128), 0)) {}
};

// v, at [n - 1][col..] for an odd n, plus grad[m - 1][n - 1] * x[m - 1][col..]; col is a multiple of 4.
__device__ __forceinline__ void add_last(f32x4& v, const uint16_t* grad, const uint8_t* x, const uint8_t* scales,
                                         int64_t m, int64_t n, uint32_t pitch, uint32_t spitch, int64_t col) {
    const float g = bf16_to_f32(grad[m * n - 1]);
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(x + (m - 1) * pitch + col);
    const u32x2 w = widen4(codes, scale_value(scales[(m - 1) * spitch + col / 128]));
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] += g * bf16_to_f32(u % 2 ? w[u / 2] >> 16 : w[u / 2] & 0xffffu);
}

// Both operands lie with the summed axis as their rows, while the matrix
// instruction wants 8 neighbours along it in a lane: LDS holds 64 rows of T
// columns of both in bfloat16, read with a transposing instruction. The codes
// become bfloat16 on their way into LDS; a stage's loads into registers run two
// stages ahead. T x T outputs in four waves. With gridDim.y > 1 a workgroup sums its
// share of the rows into its part of the workspace.
template <int T, typename OT>
__global__ __launch_bounds__(256) void weight_grad8_kernel(const uint16_t* __restrict__ grad,
                                                           const uint8_t* __restrict__ x,
                                                           const uint8_t* __restrict__ scales, int64_t m, int64_t n,
                                                           int64_t k, uint32_t pitch, uint32_t spitch, int64_t share,
                                                           TileOrder order, OT* __restrict__ out,
                                                           float* __restrict__ parts, bool accumulate) {
    constexpr int kRow = T * 2, kOperand = kStep * kRow, kStage = 2 * kOperand, F = T / 32;   // F: fragments of a wave, each way
    constexpr int kGrad = T / 32, kX = T / 64;   // 16-byte loads of a lane
    __shared__ __align__(16) uint8_t lds[2 * kStage];
    uint32_t tn, tk;
    if (!order.tile(blockIdx.x, tn, tk)) return;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t n0 = static_cast<int64_t>(tn) * T, k0 = static_cast<int64_t>(tk) * T;
    const int64_t begin = blockIdx.y * share, end = min(begin + share, m);
    const int wk = wave % 2 * F, wn = wave / 2 * F;   // in pieces of 16 columns
    const int stages = static_cast<int>((end - begin + kStep - 1) / kStep);

    // LDS rows in pieces of 32 bytes, exchanged by row so that the four rows of a
    // transposing read (and with 8 pieces two of its lane groups) meet different banks
    auto piece_at = [](int row, int p) { return row * kRow + ((p ^ (T == 64 ? row & 3 : (row & 3) | (row >> 1 & 4))) << 5); };
    uint32_t grad_at[kGrad], x_at[kX], scale_at[kX];
#pragma unroll
    for (int i = 0; i < kGrad; ++i)
        grad_at[i] = (i * (2048 / T) + t / (T / 8)) * static_cast<uint32_t>(n) * 2 + t % (T / 8) * 16;
#pragma unroll
    for (int i = 0; i < kX; ++i) {
        const uint32_t row = i * (4096 / T) + t / (T / 16);
        x_at[i] = row * pitch + t % (T / 16) * 16;
        scale_at[i] = row * spitch;
    }
    struct Staged {
        u32x4 g[kGrad], c[kX];
        uint32_t s[kX];
    } one, two;   // even and odd stages
    auto fetch = [&](Staged& to, int stage) {
        const Rows rows(grad, x, scales, begin + stage * static_cast<int64_t>(kStep), end, m, n, n0, pitch, spitch, k0);
#pragma unroll
        for (int i = 0; i < kX; ++i) to.s[i] = rows.scales.load1(scale_at[i]);
#pragma unroll
        for (int i = 0; i < kX; ++i) to.c[i] = rows.x.load16(x_at[i]);
#pragma unroll
        for (int i = 0; i < kGrad; ++i) to.g[i] = rows.grad.load16(grad_at[i]);
    };
    auto keep = [&](const Staged& from, int stage) {
        uint8_t* to = lds + (stage & 1) * kStage;
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const float f = scale_value(from.s[i]);
            const u32x4& c = from.c[i];
            const u32x2 a = widen4(c[0], f), b = widen4(c[1], f), d = widen4(c[2], f), e = widen4(c[3], f);
            u32x4* p = reinterpret_cast<u32x4*>(to + kOperand + piece_at(i * (4096 / T) + t / (T / 16), t % (T / 16)));
            p[0] = u32x4{a[0], a[1], b[0], b[1]};
            p[1] = u32x4{d[0], d[1], e[0], e[1]};
        }
#pragma unroll
        for (int i = 0; i < kGrad; ++i)
            *reinterpret_cast<u32x4*>(to + piece_at(i * (2048 / T) + t / (T / 8), t % (T / 8) / 2) + t % 2 * 16) = from.g[i];
    };
    f32x4 acc[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    auto multiply = [&](int stage) {
        const uint8_t* at = lds + (stage & 1) * kStage;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            // lane l: column l % 16 of a piece, 8 rows from (l / 16) * 8 on
            const int row = half * 32 + lane / 16 * 8 + lane % 16 / 4;
            auto fragment = [&](const uint8_t* tile, int p) {
                const int first = piece_at(row, p), next = piece_at(row + 4, p);
                return read_transposed(tile + first + lane % 4 * 8, next - first);
            };
            bf16x8 fx[F], fg[F];
#pragma unroll
            for (int j = 0; j < F; ++j) fx[j] = fragment(at + kOperand, wk + j);
#pragma unroll
            for (int i = 0; i < F; ++i) fg[i] = fragment(at, wn + i);
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int j = 0; j < F; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[j], fg[i], acc[i][j], 0, 0, 0);
        }
    };
    fetch(one, 0);
    fetch(two, 1);
    keep(one, 0);
    __syncthreads();
    // (a stage behind the last one holds zeros)
#pragma unroll 1
    for (int stage = 0; stage < stages; stage += 2) {
        fetch(one, stage + 2);
        multiply(stage);
        keep(two, stage + 1);
        lds_done();
        fetch(two, stage + 3);
        multiply(stage + 1);
        keep(one, stage + 2);
        lds_done();
    }
    float* part = gridDim.y > 1 ? parts + static_cast<int64_t>(blockIdx.y) * n * k : nullptr;
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const int64_t row = n0 + (wn + i) * 16 + lane % 16;
        if (row >= n) continue;
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const int64_t col = k0 + (wk + j) * 16 + lane / 16 * 4;
            const int left = static_cast<int>(min(k - col, static_cast<int64_t>(4)));
            if (left <= 0) continue;
            f32x4 v = acc[i][j];
            if (n % 2 && m > 0 && row == n - 1 && end == m) add_last(v, grad, x, scales, m, n, pitch, spitch, col);
            put4(part, out, row * k + col, left, v, accumulate);
        }
    }
}

// The kernel for large gradients: 256 x 256 outputs in four waves of 128 x 128, one
// on each SIMD. A stage is 64 rows of both operands in LDS, and a wave reads
// the fragments of 16 rows (for instructions of 32 x 32 x 16) while the products of
// the 16 before them run. Before the products of a stage's last 16 rows the waves
// meet: the next stage has arrived, and this one's LDS is free for the stage
// after that, which was loaded into registers a stage earlier; the codes become
// bfloat16 on their way from there. (Loads straight into LDS have to have arrived
// before the next transposing read, which took a third longer.) Needs 256 rows and
// columns. The last tile of a row or column of tiles lies inside the matrix too and
// stores what no other tile does. (So a row of the last tile ends with a whole word,
// also for an odd n, and add_last has nothing to add.)
constexpr int kWideTile = 256;

template <typename OT>
__global__ __launch_bounds__(256) void weight_grad8_wide_kernel(const uint16_t* __restrict__ grad,
                                                                const uint8_t* __restrict__ x,
                                                                const uint8_t* __restrict__ scales, int64_t m,
                                                                int64_t n, int64_t k, uint32_t pitch, uint32_t spitch,
                                                                int64_t share, TileOrder order, OT* __restrict__ out,
                                                                float* __restrict__ parts, bool accumulate) {
    constexpr int kRow = kWideTile * 2, kOperand = kStep * kRow, kStage = 2 * kOperand;   // bytes
    __shared__ __align__(16) uint8_t lds[2 * kStage];
    uint32_t tn, tk;
    if (!order.tile(blockIdx.x, tn, tk)) return;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t n0 = min(static_cast<int64_t>(tn) * kWideTile, n - kWideTile);
    const int64_t k0 = min(static_cast<int64_t>(tk) * kWideTile, static_cast<int64_t>(pitch) - kWideTile);
    const int64_t begin = blockIdx.y * share, end = min(begin + share, m);
    const int wn = wave % 2 * 128, wk = wave / 2 * 128;
    const int stages = static_cast<int>((end - begin + kStep - 1) / kStep);

    // LDS: rows of 512 bytes in pieces of 32 (16 columns), exchanged by row % 4, so
    // that the four rows of two neighbouring pieces that 32 lanes read together
    // lie in different banks. Rows past the end are outside the buffers: nothing
    // is read there, and what they would hold counts as 0.
    uint32_t grad_at[8], x_at[4], scale_at[4];   // a lane's 8 columns of 8 rows of grad, 16 of 4 rows of x
#pragma unroll
    for (int i = 0; i < 8; ++i) grad_at[i] = (i * 8 + t / 32) * static_cast<uint32_t>(n) * 2 + t % 32 * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x_at[i] = (i * 16 + t / 16) * pitch + t % 16 * 16;
        scale_at[i] = (i * 16 + t / 16) * spitch + t % 16 / 8;
    }
    struct Staged {
        u32x4 g[8], c[4];
        uint32_t s[4];
    } one, two;   // even and odd stages
    Rows rows(grad, x, scales, begin, end, m, n, n0, pitch, spitch, k0);   // of the stage that is loaded next
    // the q-th of a stage's 16 loads
    auto fetch = [&](Staged& to, auto q) {
        if constexpr (q < 4) to.s[q] = rows.scales.load1(scale_at[q]);
        else if constexpr (q < 8) to.c[q - 4] = rows.x.load16(x_at[q - 4]);
        else to.g[q - 8] = rows.grad.load16(grad_at[q - 8]);
    };
    // an eighth of a stage's way into LDS: 8 columns of x of one of a lane's rows, and of grad
    auto keep = [&](const Staged& from, int stage, auto q) {
        uint8_t* to = lds + (stage & 1) * kStage;
        constexpr int i = q / 2, part = q % 2;
        const int row = i * 16 + t / 16, g_row = q * 8 + t / 32;
        const float f = scale_value(from.s[i]);
        const u32x2 a = widen4(from.c[i][2 * part], f), b = widen4(from.c[i][2 * part + 1], f);
        *reinterpret_cast<u32x4*>(to + kOperand + row * kRow + ((t % 16) ^ (row % 4 * 2)) * 32 + part * 16) =
            u32x4{a[0], a[1], b[0], b[1]};
        *reinterpret_cast<u32x4*>(to + g_row * kRow + ((t % 32 / 2) ^ (g_row % 4 * 2)) * 32 + t % 2 * 16) = from.g[q];
    };

    struct Fragments {
        bf16x8 g[4], x[4];
    } even, odd;
    // lane l: column l % 32 of a tile of 32, 8 rows from (l / 32) * 8 on; the instruction
    // transposes 4 rows of 16 columns in 16 lanes
    const int row_of = lane / 32 * 8 + lane % 16 / 4;
    int piece[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        piece[j] = row_of * kRow + ((j * 2 + lane / 16 % 2) ^ (lane % 16 / 4 * 2)) * 32 + lane % 4 * 8;
    // the q-th of 8 fragments of a stage's 16 rows number `chunk`
    auto read = [&](Fragments& f, int stage, int chunk, auto q) {
        const uint8_t* at = lds + (stage & 1) * kStage + chunk * 16 * kRow;
        if constexpr (q < 4) f.x[q] = read_transposed(at + kOperand + wk * 2 + piece[q], 4 * kRow);
        else f.g[q - 4] = read_transposed(at + wn * 2 + piece[q - 4], 4 * kRow);
    };
    f32x16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    auto multiply = [&](const Fragments& f, auto q) {
        constexpr int i = q / 4, j = q % 4;
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.x[j], f.g[i], acc[i][j], 0, 0, 0);
    };
    auto next_rows = [&](int stage) {
        rows = Rows(grad, x, scales, begin + stage * static_cast<int64_t>(kStep), end, m, n, n0, pitch, spitch, k0);
    };
    unrolled<16>([&](auto q) { fetch(one, q); });
    next_rows(1);
    unrolled<16>([&](auto q) { fetch(two, q); });
    unrolled<8>([&](auto q) { keep(one, 0, q); });
    __syncthreads();
    unrolled<8>([&](auto q) { keep(two, 1, q); });
    unrolled<8>([&](auto q) { read(even, 0, 0, q); });
    __builtin_amdgcn_sched_barrier(0);
    next_rows(2);
    unrolled<16>([&](auto q) { fetch(one, q); });
    next_rows(3);
    // The order is the source's, a load behind every third product (left to the compiler,
    // two behind each of the first eight: 496 us instead of 448, as the loads' addresses
    // take the compute unit as long as a product).
    auto run = [&](const Staged& mine, Staged& other, int stage) {
        unrolled<3>([&](auto c) {
            const Fragments& now = c % 2 ? odd : even;
            Fragments& then = c % 2 ? even : odd;
            unrolled<16>([&](auto q) {
                multiply(now, q);
                if constexpr (q % 2 == 0) read(then, stage, c + 1, std::integral_constant<int, q / 2>{});
                constexpr int at = c * 16 + q;
                if constexpr (at % 3 == 1) fetch(other, std::integral_constant<int, at / 3>{});
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        lds_done();
        unrolled<16>([&](auto q) {
            multiply(odd, q);
            if constexpr (q < 8) keep(mine, stage + 2, q);
            else read(even, stage + 1, 0, std::integral_constant<int, q - 8>{});
            if constexpr (q == 12) next_rows(stage + 4);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // (a stage behind the last one holds zeros)
#pragma unroll 1
    for (int stage = 0; stage < stages; stage += 2) {
        run(one, two, stage);
        run(two, one, stage + 1);
    }
    lds_done();

    // 32 rows of a wave's outputs at a time pass through LDS (16-byte chunks
    // exchanged by row), so that rows leave in runs of 512 bytes
    float* part = gridDim.y > 1 ? parts + static_cast<int64_t>(blockIdx.y) * n * k : nullptr;
    uint8_t* mine = lds + wave * 16384;
    const int64_t first_n = static_cast<int64_t>(tn) * kWideTile, first_k = static_cast<int64_t>(tk) * kWideTile;
    const int64_t col = k0 + wk + lane % 32 * 4;
    const int left = col < first_k ? 0 : static_cast<int>(max(static_cast<int64_t>(0), min(k - col, static_cast<int64_t>(4))));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            asm volatile("" : "+a"(acc[i][j]));   // read from its accumulation registers here, not earlier
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int chunk = j * 8 + r * 2 + lane / 32;
                *reinterpret_cast<f32x4*>(mine + lane % 32 * 512 + (chunk ^ (lane % 32)) * 16) =
                    f32x4{acc[i][j][r * 4], acc[i][j][r * 4 + 1], acc[i][j][r * 4 + 2], acc[i][j][r * 4 + 3]};
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll 4
        for (int q = 0; q < 16; ++q) {
            const int r = q * 2 + lane / 32;
            const int64_t row = n0 + wn + i * 32 + r;
            const f32x4 v = *reinterpret_cast<const f32x4*>(mine + r * 512 + ((lane % 32) ^ r) * 16);
            if (row < first_n || left <= 0) continue;
            put4(part, out, row * k + col, left, v, accumulate);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// out (+)= the sum of the parts: a workgroup's four waves add up a quarter of the parts
// each, in order, for 256 outputs, then these in order.
template <typename OT>
__global__ __launch_bounds__(kBlock) void add_parts_kernel(const float* __restrict__ parts, int64_t n, int count,
                                                           OT* __restrict__ out, bool accumulate) {
    __shared__ f32x4 sums[kBlock / 64 - 1][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 64 + lane) * 4;
    const int left = static_cast<int>(max(static_cast<int64_t>(0), min(n - i, static_cast<int64_t>(4))));
    const int each = (count + 3) / 4, from = min(wave * each, count), to = min(from + each, count);
    f32x4 v{0, 0, 0, 0};
#pragma unroll 4
    for (int c = from; c < to; ++c) {
        float x[4];
        load4(parts + c * n + i, left, x);
        v += f32x4{x[0], x[1], x[2], x[3]};
    }
    if (wave > 0) sums[wave - 1][lane] = v;
    __syncthreads();
    if (wave > 0 || left == 0) return;
#pragma unroll
    for (int w = 0; w < kBlock / 64 - 1; ++w) v += sums[w][lane];
    put4(nullptr, out, i, left, v, accumulate);
}

// How a call is done: tiles of 256, 128 or 64 outputs each way, and the summed rows
// in `count` shares whose parts, where there are several, are added at the end.
constexpr int64_t kMaxSplit = int64_t{1} << 30;   // outputs: add_parts_kernel's threads stay within a dispatch
struct Way {
    int tile, count;
    int64_t share;
    size_t parts_bytes(int64_t n, int64_t k) const { return count > 1 ? static_cast<size_t>(count) * n * k * 4 : 0; }
};

// The way with the least estimated time. A stage of 64 rows takes 1.7 us of a compute
// unit with 256 x 256 outputs (one workgroup), 0.84 or 1.2 with 128 x 128 (one or two), and
// 0.45 to 1.2 with 64 x 64 (one to four); a workgroup's start and end 8, 4 and 3 us; parts
// are written and read again at 5 bytes a ns, and each takes 0.1 us. Measured, us, with
// tiles of 256 / 128 / 64 only (m x n x k): 16384x4096x4096 438 / 604 / 970, 4096x4096x4096
// 120 / 160 / 254, 3000x5000x2000 78 / 92 / 128, 8192x2048x2048 88 / 91 / 130,
// 2048x4096x1024 56 / 31 / 39, 1024x1024x1024 33 / 18 / 10, 4099x300x515 26 / 15 / 13. With
// parts at 1.5 bytes a ns they were too few (6000x1000x1000 41 instead of 30).
Way way_of(int64_t m, int64_t n, int64_t k) {
    if (m == 0) return Way{128, 1, kStep};
    Way best{};
    double least = 0;
    const int64_t stages = ceil_div(m, kStep);
    for (int tile = 256; tile >= 64; tile /= 2) {
        if (tile == 256 && (n < 256 || pitch8(k) < 256)) continue;
        const int64_t tiles = ceil_div(n, tile) * ceil_div(k, tile), cus = device_cus(), most_of_cu = tile == 256 ? 1 : tile == 128 ? 2 : 4;
        const double fixed_us = tile == 256 ? 8 : tile == 128 ? 4 : 3;
        const auto stage_us = [&](int64_t of_cu) {   // with so many workgroups on a compute unit
            return tile == 256 ? 1.7 : tile == 128 ? 0.48 + 0.36 * of_cu : 0.2 + 0.25 * of_cu;
        };
        const int64_t most = n * k > kMaxSplit ? 1 : std::min<int64_t>(stages, 64);
        for (int64_t count = 1; count <= most; ++count) {
            const double join_us = count > 1 ? 3 + count * (0.1 + n * k / 0.6e6) : 0;
            if (best.count > 0 && join_us >= least) break;   // and so for more of them
            const int64_t each = ceil_div(stages, count);
            if (count > 1 && ceil_div(stages, each) != count) continue;
            const int64_t rounds = tiles * count / (cus * most_of_cu), rest = tiles * count - rounds * cus * most_of_cu;
            const double us = rounds * (each * stage_us(most_of_cu) + fixed_us) +
                              (rest > 0 ? each * stage_us(ceil_div(rest, cus)) + fixed_us : 0) + join_us;
            if (best.count == 0 || us < least) least = us, best = Way{tile, static_cast<int>(count), each * kStep};
        }
    }
    return best;
}

template <int T, typename OT>
lsgd_status launch_tiles(const Way& w, const void* grad, const void* x, const void* scales, int64_t m, int64_t n, int64_t k,
                         void* out, bool accumulate, float* parts, hipStream_t s) {
    const TileOrder order(ceil_div(n, T), ceil_div(k, T));
    if (order.blocks() * w.count > kMaxGridBlocks)
        return fail(LSGD_ERR_SIZE, "%lld tiles", static_cast<long long>(order.blocks() * w.count));
    const dim3 grid(static_cast<unsigned>(order.blocks()), static_cast<unsigned>(w.count));
    const uint16_t* g = static_cast<const uint16_t*>(grad);
    const uint8_t *c = static_cast<const uint8_t*>(x), *sc = static_cast<const uint8_t*>(scales);
    const uint32_t pitch = static_cast<uint32_t>(pitch8(k)), spitch = static_cast<uint32_t>(scale_pitch8(k));
    if constexpr (T == kWideTile)
        hipLaunchKernelGGL((weight_grad8_wide_kernel<OT>), grid, dim3(256), 0, s, g, c, sc, m, n, k, pitch, spitch, w.share,
                           order, static_cast<OT*>(out), parts, accumulate);
    else
        hipLaunchKernelGGL((weight_grad8_kernel<T, OT>), grid, dim3(256), 0, s, g, c, sc, m, n, k, pitch, spitch, w.share,
                           order, static_cast<OT*>(out), parts, accumulate);
    return check_launch("lsgd_weight_grad8");
}

template <typename OT>
lsgd_status launch(const Way& w, const void* grad, const void* x, const void* scales, int64_t m, int64_t n, int64_t k,
                   void* out, bool accumulate, void* workspace, hipStream_t s) {
    float* parts = static_cast<float*>(workspace);
    if (w.tile == 256) LSGD_TRY((launch_tiles<256, OT>(w, grad, x, scales, m, n, k, out, accumulate, parts, s)));
    else if (w.tile == 128) LSGD_TRY((launch_tiles<128, OT>(w, grad, x, scales, m, n, k, out, accumulate, parts, s)));
    else LSGD_TRY((launch_tiles<64, OT>(w, grad, x, scales, m, n, k, out, accumulate, parts, s)));
    if (w.count > 1) {
        hipLaunchKernelGGL((add_parts_kernel<OT>), dim3(static_cast<unsigned>(ceil_div(n * k, 256))),
                           dim3(kBlock), 0, s, parts, n * k, w.count, static_cast<OT*>(out), accumulate);
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
    // 64 rows lie within 32-bit offsets
    if (n > (1 << 24) || k > (1 << 24))
        return fail(LSGD_ERR_SIZE, "n=%lld or k=%lld above 2^24", static_cast<long long>(n), static_cast<long long>(k));
    return LSGD_OK;
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
    *bytes = n > 0 && k > 0 ? way_of(m, n, k).parts_bytes(n, k) : 0;
    return LSGD_OK;
}

LSGD_API lsgd_status lsgd_weight_grad8(const void* grad, const void* x, const void* x_scales, int64_t m, int64_t n,
                                       int64_t k, void* out, lsgd_dtype odt, int32_t accumulate, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    LSGD_TRY(check_dtype(odt, "out dtype"));
    LSGD_TRY(check_sizes(m, n, k));
    if (n == 0 || k == 0 || (m == 0 && accumulate)) return LSGD_OK;
    LSGD_TRY(check_buffer(out, 16, "out"));
    const Way w = way_of(m, n, k);
    const size_t need = w.parts_bytes(n, k);
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
    return odt == LSGD_F32 ? launch<float>(w, grad, x, x_scales, m, n, k, out, accumulate != 0, workspace, s)
                           : launch<uint16_t>(w, grad, x, x_scales, m, n, k, out, accumulate != 0, workspace, s);
}

}  // extern "C"
