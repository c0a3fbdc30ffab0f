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
// 16-byte chunks exchanged by row / 2 % 8, so that the same chunk of 16 rows lies in
// all 64 banks (by row % 8 two rows of 16 met in each bank). b is the matrix
// instruction's first operand: a lane then holds 4 neighbouring columns of one output
// row. Offsets inside a tile are 32-bit.
template <int TM, int TN, int WM, int WN, typename OT>
__global__ __launch_bounds__(WM * WN * 64) void matmul8_kernel(Operand A, Operand B, uint32_t pitch, uint32_t spitch,
                                                               TileOrder order, OT* __restrict__ out) {
    constexpr int kWaves = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16, kStage = (BM + BN) * 128;
    constexpr int kLoadsA = BM / 8 / kWaves, kLoads = (BM + BN) / 8 / kWaves;   // of 8 rows each, per wave
    static_assert(kLoadsA * 8 * kWaves == BM && kLoads * 8 * kWaves == BM + BN, "every wave loads as many rows");
    static_assert(kWaves % 2 == 0, "row / 2 % 8 of a loaded row");
    __shared__ __align__(16) uint8_t lds[2 * kStage];
    uint32_t tm, tn;
    if (!order.tile(blockIdx.x, tm, tn)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = static_cast<int64_t>(tm) * BM, n0 = static_cast<int64_t>(tn) * BN;
    const int wm = wave % WM * (TM * 16), wn = wave / WM * (TN * 16);
    const int steps = static_cast<int>(pitch / 128);
    // rows past the end repeat the last one; their outputs are not stored
    const uint32_t last_a = static_cast<uint32_t>(min(A.rows - m0, static_cast<int64_t>(BM))) - 1;
    const uint32_t last_b = static_cast<uint32_t>(min(B.rows - n0, static_cast<int64_t>(BN))) - 1;
    const uint8_t* codes_a = A.codes + m0 * pitch;
    const uint8_t* codes_b = B.codes + n0 * pitch;
    uint32_t from[kLoads];   // a lane's 16 bytes of the rows it loads
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const uint32_t row = ((i < kLoadsA ? i : i - kLoadsA) * kWaves + wave) * 8 + lane / 8;
        from[i] = min(row, i < kLoadsA ? last_a : last_b) * pitch + ((lane % 8) ^ (wave % 2 * 4 + lane / 16)) * 16;
    }
    auto fetch = [&](uint8_t* stage) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            load_lds16((i < kLoadsA ? codes_a : codes_b) + from[i], stage + (i * kWaves + wave) * 1024);
        codes_a += 128;
        codes_b += 128;
    };
    // scale words: a row's offset from the tile's first scale row
    const uint8_t* scales_a = A.scales + (m0 >> A.shift) * spitch;
    const uint8_t* scales_b = B.scales + (n0 >> B.shift) * spitch;
    const uint32_t part_a = static_cast<uint32_t>(m0) & ((1u << A.shift) - 1);
    const uint32_t part_b = static_cast<uint32_t>(n0) & ((1u << B.shift) - 1);

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    uint32_t wa[TM], wb[TN];
    // fragment rows: lane % 16, whose row / 2 exchanges the chunks
    const int at = lane % 16 * 128 + ((lane / 16) ^ (lane / 2 % 8)) * 16;
    const int at_a = wm * 128 + at, at_b = (BM + wn) * 128 + at;
    fetch(lds);
    for (int base = 0; base < steps; base += 4) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
            wa[i] = *reinterpret_cast<const uint32_t*>(
                scales_a + ((part_a + min(static_cast<uint32_t>(wm + i * 16 + lane % 16), last_a)) >> A.shift) * spitch + base);
#pragma unroll
        for (int j = 0; j < TN; ++j)
            wb[j] = *reinterpret_cast<const uint32_t*>(
                scales_b + ((part_b + min(static_cast<uint32_t>(wn + j * 16 + lane % 16), last_b)) >> B.shift) * spitch + base);
        unrolled<4>([&](auto ic) {
            constexpr int u = decltype(ic)::value;
            if (base + u >= steps) return;
            loads_done();
            if (base + u + 1 < steps) fetch(lds + ((u + 1) & 1) * kStage);
            const uint8_t* t = lds + (u & 1) * kStage;
            auto fragment = [&](int off) {
                Codes32 f;
                f.half[0] = *reinterpret_cast<const u32x4*>(t + off);
                f.half[1] = *reinterpret_cast<const u32x4*>(t + (off ^ 64));
                return f;
            };
            Widened32 fb[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = widen32<u>(fragment(at_b + j * 2048), wb[j]);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const Widened32 fa = widen32<u>(fragment(at_a + i * 2048), wa[i]);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = multiply(fb[j], fa, acc[i][j]);
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

// The kernel for many tiles: 256 x 256 outputs in four waves of 128 x 128, one on
// each SIMD, so that a wave's fragments (64 columns of a and b at a time) are read
// while the products of the ones before them run, and widened by quarters (for
// instructions of 32 x 32 x 16), one while the one before it is multiplied: all live
// in registers, beside the 256 of the outputs. A stage (128 columns of a and b) is in
// LDS for the fragment reads while the next one arrives. A workgroup goes through
// several tiles, and its loads run two stages ahead, across the end of a tile: the
// next one's first stages arrive while this one's outputs leave. 8192 x 8192 x 4096:
// 349 us to bfloat16, 1.58 PFLOP/s, 367 to binary32 (with 128 x 128 outputs 456, 471):
// as fast as a large library product of bfloat16, so bound by the matrix units.
constexpr int kWideTile = 256;

// The stage that a workgroup loads next: tile, place in it, addresses. The last
// tile of a row or column of tiles lies inside the matrix too, over a part of
// the one before it: both compute the same bits there.
struct WideLoads {
    static constexpr int kLoads = 8;          // of 8 rows each, per wave and operand
    static constexpr int kStage = 2 * kWideTile * 128;
    uint32_t row_a[2], row_b[2];              // scale rows of two of a wave's fragments each
    Buffer codes_a, codes_b, scales_a, scales_b;
    uint32_t stage;

    static __device__ __forceinline__ int64_t origin(uint32_t tile, int64_t rows) {
        return min(static_cast<int64_t>(tile) * kWideTile, rows - kWideTile);
    }
    __device__ __forceinline__ WideLoads() : codes_a(nullptr, 0), codes_b(nullptr, 0), scales_a(nullptr, 0), scales_b(nullptr, 0) {}
    __device__ __forceinline__ void set(const Operand& A, const Operand& B, uint32_t tm, uint32_t tn, uint32_t pitch,
                                        uint32_t spitch, int wave, int lane) {
        const int64_t m0 = origin(tm, A.rows), n0 = origin(tn, B.rows);
        codes_a = Buffer(A.codes + m0 * pitch, kWideTile * pitch);
        codes_b = Buffer(B.codes + n0 * pitch, kWideTile * pitch);
        const uint32_t part_a = static_cast<uint32_t>(m0) & ((1u << A.shift) - 1);
        const uint32_t part_b = static_cast<uint32_t>(n0) & ((1u << B.shift) - 1);
        scales_a = Buffer(A.scales + (m0 >> A.shift) * spitch, (((part_a + kWideTile - 1) >> A.shift) + 1) * spitch);
        scales_b = Buffer(B.scales + (n0 >> B.shift) * spitch, (((part_b + kWideTile - 1) >> B.shift) + 1) * spitch);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            row_a[i] = ((part_a + wave % 2 * 128 + i * 64 + lane) >> A.shift) * spitch;
            row_b[i] = ((part_b + wave / 2 * 128 + i * 64 + lane) >> B.shift) * spitch;
        }
        stage = 0;
    }
    // The q-th of a stage's 2 kLoads loads; `from`: a lane's 16 bytes of the wave's first 8 rows.
    __device__ __forceinline__ void fetch(int q, uint8_t* to, uint32_t from, uint32_t pitch, int wave) const {
        (q < kLoads ? codes_a : codes_b).load_lds16(from, stage * 128 + q % kLoads * 32 * pitch, to + (q * 4 + wave) * 1024);
    }
    // A word holds a row's scales of four stages. It is loaded for the first of them;
    // for the others the offsets lie outside the buffer, which costs no access.
    __device__ __forceinline__ bool first_of_four() const { return stage % 4 == 0; }
    __device__ __forceinline__ void fetch_scales(int i, uint32_t (&words)[4]) const {
        words[i] = (i < 2 ? scales_a : scales_b).load4((i < 2 ? row_a[i] : row_b[i - 2]) | (first_of_four() ? 0 : 0x80000000u), stage);
    }
    __device__ __forceinline__ void fetch_all(uint8_t* to, uint32_t from, uint32_t pitch, int wave, uint32_t (&words)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) fetch_scales(i, words);
#pragma unroll
        for (int q = 0; q < 2 * kLoads; ++q) fetch(q, to, from, pitch, wave);
    }
};

template <typename OT>
__global__ __launch_bounds__(256) void matmul8_wide_kernel(Operand A, Operand B, uint32_t pitch, uint32_t spitch,
                                                           TileOrder order, OT* __restrict__ out) {
    constexpr int kStage = WideLoads::kStage;
    __shared__ __align__(16) uint8_t lds[2 * kStage + 4 * 8192];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % 2 * 128, wn = wave / 2 * 128;
    const uint32_t stages = pitch / 128;
    uint32_t tm, tn, next_tm, next_tn, block = blockIdx.x;
    if (!order.tile(block, tm, tn)) return;
    const uint32_t from = (wave * 8 + lane / 8) * pitch + ((lane % 8) ^ (wave % 2 * 4 + lane / 16)) * 16;
    WideLoads loads;
    loads.set(A, B, tm, tn, pitch, spitch, wave, lane);
    uint32_t scales[8], words[4];   // of this stage (a's fragments, then b's), as loaded for the next
    // the words of 64 rows: those of 32 rows in both halves of the wave
    auto spread = [](uint32_t word, uint32_t& low, uint32_t& high) {
        const auto w = __builtin_amdgcn_permlane32_swap(word, word, false, false);
        low = w[0];
        high = w[1];
    };
    struct Fragments {
        Codes32 a[4], b[4];
    } even, odd;   // columns [0, 64) and [64, 128) of a stage
    // a lane reads chunks 4 h + lane / 32 and the second behind it of row lane % 32
    const uint32_t at = lane % 32 * 128 + ((lane / 32) ^ (lane / 2 % 8)) * 16;
    // the q-th of a half stage's 16 reads
    auto read = [&](Fragments& f, uint32_t stage, int h, auto q) {
        constexpr int i = q % 4, part = q / 8;
        const uint8_t* x = lds + stage + (at ^ (h * 64 + part * 32));
        if constexpr (q % 8 < 4) f.b[i].half[part] = *reinterpret_cast<const u32x4*>(x + (kWideTile + wn + i * 32) * 128);
        else f.a[i].half[part] = *reinterpret_cast<const u32x4*>(x + (wm + i * 32) * 128);
    };
    loads.fetch_all(lds, from, pitch, wave, words);
    loads_done();
#pragma unroll
    for (int i = 0; i < 4; ++i) spread(words[i], scales[2 * i], scales[2 * i + 1]);
    loads.stage = 1;
    loads.fetch_all(lds + kStage, from, pitch, wave, words);
    unrolled<16>([&](auto q) { read(even, 0, 0, q); });
    // a quarter of a half stage in bfloat16 (a lane's 8 columns of every row), and
    // the next one, whose e-th of 32 steps this is
    struct Widened {
        uint32_t a[4][4], b[4][4];
    } quarter[2];
    auto widen = [&](const Fragments& f, const uint32_t (&s)[8], auto g, auto e) {
        constexpr int i = e / 8, word = g * 2 + e % 4 / 2;
        const float sa = scale_value(s[i] & 0xffu), sb = scale_value(s[4 + i] & 0xffu);
        if constexpr (e % 8 < 4) quarter[g % 2].a[i][e % 4] = widen2<e % 2>(f.a[i].word[word], sa);
        else quarter[g % 2].b[i][e % 4] = widen2<e % 2>(f.b[i].word[word], sb);
    };
    unrolled<32>([&](auto e) { widen(even, scales, std::integral_constant<int, 0>{}, e); });
    uint32_t here = 0;
    bool four = false;   // whether `words` holds four stages' scales, and not nothing
    for (;;) {
        f32x16 acc[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
        // a half stage, 64 products of 32 x 32 x 16. Meanwhile the next half is read
        // and, by quarters, widened (`then`: its scales).
        auto half = [&](const Fragments& f, Fragments& next, uint32_t stage, int h, const uint32_t (&then)[8], auto fetch) {
            unrolled<4>([&](auto g) {
                unrolled<16>([&](auto q) {
                    constexpr int i = q / 4, j = q % 4, at = g * 16 + q;
                    const auto eight = [](const uint32_t (&x)[4]) {
                        return __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], x[2], x[3]});
                    };
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eight(quarter[g % 2].b[j]), eight(quarter[g % 2].a[i]),
                                                                        acc[i][j], 0, 0, 0);
                    unrolled<2>([&](auto u) {
                        using E = std::integral_constant<int, q * 2 + u>;
                        if constexpr (g < 3) widen(f, scales, std::integral_constant<int, g + 1>{}, E{});
                        else widen(next, then, std::integral_constant<int, 0>{}, E{});
                    });
                    if constexpr (at % 4 == 0) read(next, stage, h, std::integral_constant<int, at / 4>{});
                    if constexpr (at % 4 == 2) fetch(std::integral_constant<int, at / 4>{});
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        };
        block += gridDim.x;
        const bool more = order.tile(block, next_tm, next_tn);
#pragma unroll 1
        for (int last_two = 0; last_two < 2; ++last_two) {
            // while this tile's last two stages are multiplied, the next one's first
            // two arrive (behind the last tile its own again, which nothing reads)
            if (last_two) {
                if (more) loads.set(A, B, next_tm, next_tn, pitch, spitch, wave, lane);
                loads.stage = ~0u;
            }
#pragma unroll 1
            for (uint32_t t = last_two ? stages - 2 : 0; t < (last_two ? stages : stages - 2); ++t) {
                // The order is the source's: a product, then a part of the next quarter's
                // widening, a read or a load. (The compiler puts the loads in one burst, and
                // moves of scales behind it, which wait for them.)
                half(even, odd, here, 1, scales, [](auto) {});
                loads_done();   // this stage is in every wave's registers, and the next has arrived
                uint32_t then[8];   // the next stage's scales
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    spread(words[i], then[2 * i], then[2 * i + 1]);
                    then[2 * i] = four ? then[2 * i] : scales[2 * i] >> 8;
                    then[2 * i + 1] = four ? then[2 * i + 1] : scales[2 * i + 1] >> 8;
                    asm volatile("" : "+v"(then[2 * i]), "+v"(then[2 * i + 1]));   // done here, not behind the loads
                }
                ++loads.stage;
                four = loads.first_of_four();
                half(odd, even, here ^ kStage, 0, then, [&](auto q) {
                    loads.fetch(q, lds + here, from, pitch, wave);
                    if constexpr (q < 4) loads.fetch_scales(q, words);
                });
#pragma unroll
                for (int i = 0; i < 8; ++i) scales[i] = then[i];
                here ^= kStage;
            }
        }
        // 32 rows of the wave's outputs, 256 bytes of each, at a time pass through LDS
        // (16-byte chunks exchanged by row), so that rows leave in runs, past the caches
        // (2304 x 4096 x 512 14.8 us, through them 16.2, with lsgd_quant8 of the outputs
        // behind it 22.9 and 23.5; 4096 x 4096 x 4096 90 and 92, 102 and 101)
        uint32_t l = lane;
        asm volatile("" : "+v"(l));   // the addresses below are not worth registers during the products
        constexpr int kPart = 256 / (32 * sizeof(OT));   // fragments of 32 columns in 256 bytes
        const uint64_t row_bytes = static_cast<uint64_t>(B.rows) * sizeof(OT);
        uint8_t* o = reinterpret_cast<uint8_t*>(out + (WideLoads::origin(tm, A.rows) + wm) * B.rows +
                                                WideLoads::origin(tn, B.rows) + wn) + l / 16 * row_bytes + l % 16 * 16;
        uint8_t* mine = lds + 2 * kStage + wave * 8192;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int p = 0; p < 4 / kPart; ++p) {
#pragma unroll
                for (int u = 0; u < kPart; ++u) {
                    f32x16& v = acc[i][p * kPart + u];
                    asm volatile("" : "+a"(v));   // read from its accumulation registers here, not earlier
                    uint8_t* row = mine + l % 32 * 256;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if constexpr (sizeof(OT) == 4)
                            *reinterpret_cast<f32x4*>(row + ((u * 8 + r * 2 + l / 32) ^ (l % 16)) * 16) =
                                f32x4{v[r * 4], v[r * 4 + 1], v[r * 4 + 2], v[r * 4 + 3]};
                        else
                            *reinterpret_cast<u32x2*>(row + ((u * 4 + r) ^ (l % 16)) * 16 + l / 32 * 8) =
                                u32x2{f32_to_bf16x2(v[r * 4], v[r * 4 + 1]), f32_to_bf16x2(v[r * 4 + 2], v[r * 4 + 3])};
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_wave_barrier();
                uint8_t* to = o + p * 256;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const uint32_t row = q * 4 + l / 16;
                    const u32x4 v = *reinterpret_cast<const u32x4*>(mine + row * 256 + ((l % 16) ^ (row % 16)) * 16);
                    __builtin_nontemporal_store(u32x4_u2{v[0], v[1], v[2], v[3]}, reinterpret_cast<u32x4_u2*>(to));
                    to += 4 * row_bytes;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            o += 32 * row_bytes;
        }
        if (!more) break;
        tm = next_tm;
        tn = next_tn;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load into LDS outlives the workgroup
}

// The kernel for few tiles: a workgroup's W waves share one small tile of outputs
// and divide its columns of a and b, so that a wave has K / (128 W) stages to
// go through instead of K / 128. Each wave loads its stages into a ring of
// D slots of LDS that are its own (in rows of 128 bytes, as the larger kernels
// do; loads straight into registers, 64 bytes of a row each, were slower by half),
// so nothing waits for another wave until the sums meet in LDS, added in wave
// order. Bound by latency: the ring holds the first D stages at once, but behind
// them hardly a load overlaps another, as the waits for the scales' registers, loaded in
// between, take in the codes of the slot behind as well (16 x 4096 x 4096, whose
// waves have four stages: 5.3 us for 17 MB).
template <int TM, int TN, int W, int D, typename OT>
__global__ __launch_bounds__(W * 64) void matmul8_narrow_kernel(Operand A, Operand B, uint32_t pitch, uint32_t spitch,
                                                                TileOrder order, OT* __restrict__ out) {
    constexpr int kSlot = (TM + TN) * 2048, kLoads = (TM + TN) * 2;   // loads of 8 rows each
    constexpr int kRing = W * D * kSlot, kSums = W * TM * TN * 1024;
    __shared__ __align__(16) uint8_t lds[kRing > kSums ? kRing : kSums];
    uint32_t tm, tn;
    if (!order.tile(blockIdx.x, tm, tn)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = static_cast<int64_t>(tm) * (TM * 16), n0 = static_cast<int64_t>(tn) * (TN * 16);
    const uint32_t stages = pitch / 128;
    // rows past the end repeat the last one; their outputs are not stored
    const uint8_t* from[kLoads];
    const uint8_t *sa[TM], *sb[TN];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const bool a = i < TM * 2;
        const int64_t r = a ? min(m0 + i * 8 + lane / 8, A.rows - 1) : min(n0 + (i - TM * 2) * 8 + lane / 8, B.rows - 1);
        from[i] = (a ? A.codes : B.codes) + r * pitch + ((lane % 8) ^ (i % 2 * 4 + lane / 16)) * 16;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = A.scales + (min(m0 + i * 16 + lane % 16, A.rows - 1) >> A.shift) * spitch;
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = B.scales + (min(n0 + j * 16 + lane % 16, B.rows - 1) >> B.shift) * spitch;
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    uint8_t* ring = lds + wave * (D * kSlot);
    uint32_t wa[D][TM], wb[D][TN];
    const uint32_t each = (stages + W - 1) / W, begin = wave * each, end = min(begin + each, stages);
    if (begin < end) {
        // stages past the end repeat the last one, into slots that nothing reads any more
        auto fetch = [&](uint32_t s, int d) {
            s = min(s, end - 1);
#pragma unroll
            for (int i = 0; i < TM; ++i) wa[d][i] = sa[i][s];
#pragma unroll
            for (int j = 0; j < TN; ++j) wb[d][j] = sb[j][s];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load_lds16(from[i] + s * 128, ring + d * kSlot + i * 1024);
        };
        unrolled<D>([&](auto d) { fetch(begin + decltype(d)::value, decltype(d)::value); });
        const int at = lane % 16 * 128 + ((lane / 16) ^ (lane / 2 % 8)) * 16;
        for (uint32_t base = begin; base < end; base += D)
            unrolled<D>([&](auto dc) {
                constexpr int d = decltype(dc)::value;
                if (base + d >= end) return;
                // This stage has arrived: at least (D - 1) * kLoads loads were issued after it
                // (and the scales of the stages behind it, which the count leaves out, so that
                // some of these have to arrive too).
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * kLoads) : "memory");
                auto fragment = [&](int off) {
                    Codes32 f;
                    f.half[0] = *reinterpret_cast<const u32x4*>(ring + d * kSlot + off);
                    f.half[1] = *reinterpret_cast<const u32x4*>(ring + d * kSlot + (off ^ 64));
                    return f;
                };
                Codes32 ra[TM], rb[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) rb[j] = fragment((TM + j) * 2048 + at);
#pragma unroll
                for (int i = 0; i < TM; ++i) ra[i] = fragment(i * 2048 + at);
                uint32_t va[TM], vb[TN];
#pragma unroll
                for (int i = 0; i < TM; ++i) va[i] = wa[d][i];
#pragma unroll
                for (int j = 0; j < TN; ++j) vb[j] = wb[d][j];
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the slot is loaded again
                fetch(base + d + D, d);
                Widened32 fb[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[j] = widen32<0>(rb[j], vb[j]);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const Widened32 fa = widen32<0>(ra[i], va[i]);
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = multiply(fb[j], fa, acc[i][j]);
                }
            });
    }
    loads_done();   // the rings are free
    f32x4* sums = reinterpret_cast<f32x4*>(lds);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) sums[(wave * TM * TN + i * TN + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int q = wave; q < TM * TN; q += W) {
        f32x4 v = sums[q * 64 + lane];
        for (uint32_t w = 1; w < W && w * each < stages; ++w) v += sums[(w * TM * TN + q) * 64 + lane];
        const int64_t m = m0 + q / TN * 16 + lane % 16, n = n0 + q % TN * 16 + lane / 16 * 4, left = B.rows - n;
        if (m < A.rows && left > 0) store4(out + m * B.rows + n, static_cast<int>(min(left, static_cast<int64_t>(4))), v);
    }
}

template <typename OT>
__global__ __launch_bounds__(kBlock) void zero_kernel(OT* __restrict__ out, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kBlock)
        out[i] = 0;
}

template <int TM, int TN, int WM, int WN, typename OT>
lsgd_status launch_tiles(const Operand& a, const Operand& b, int64_t k, void* out, hipStream_t s) {
    const TileOrder order(ceil_div(a.rows, WM * TM * 16), ceil_div(b.rows, WN * TN * 16));
    if (order.blocks() > kMaxGridBlocks) return fail(LSGD_ERR_SIZE, "%lld tiles", static_cast<long long>(order.blocks()));
    hipLaunchKernelGGL((matmul8_kernel<TM, TN, WM, WN, OT>), dim3(static_cast<unsigned>(order.blocks())),
                       dim3(WM * WN * 64), 0, s, a, b, static_cast<uint32_t>(pitch8(k)),
                       static_cast<uint32_t>(scale_pitch8(k)), order, static_cast<OT*>(out));
    return check_launch("lsgd_matmul8");
}

template <int TM, int TN, int W, int D, typename OT>
lsgd_status launch_narrow(const Operand& a, const Operand& b, int64_t k, void* out, hipStream_t s) {
    const TileOrder order(ceil_div(a.rows, TM * 16), ceil_div(b.rows, TN * 16));
    hipLaunchKernelGGL((matmul8_narrow_kernel<TM, TN, W, D, OT>), dim3(static_cast<unsigned>(order.blocks())), dim3(W * 64),
                       0, s, a, b, static_cast<uint32_t>(pitch8(k)), static_cast<uint32_t>(scale_pitch8(k)), order,
                       static_cast<OT*>(out));
    return check_launch("lsgd_matmul8");
}

template <typename OT>
lsgd_status launch(const Operand& a, const Operand& b, int64_t k, void* out, hipStream_t s) {
    if (k == 0) {
        const int64_t n = a.rows * b.rows;
        hipLaunchKernelGGL((zero_kernel<OT>), dim3(static_cast<unsigned>(std::min<int64_t>(4096, ceil_div(n, kBlock)))),
                           dim3(kBlock), 0, s, static_cast<OT*>(out), n);
        return check_launch("lsgd_matmul8");
    }
    // The smallest tile of which every compute unit gets at most one: with one
    // round of workgroups the time is a wave's loads one after another. us to bfloat16, at
    // m x n x k, 16x16 / 32x16 / 32x32 / 64x32 / 64x64 / 128x128 outputs:
    // 16x4096x4096 5.3 / 6.3 / 7.1 / 8.7 / 12.8 / 35, 256x512x4096 8.3 / 7.5 / 8.3 /
    // 11.7 / 15.0 / 40, 512x512x512 5.2 / 5.2 / 4.0 / 4.5 / 6.3 / 8.3, 256x2048x2048
    // 15.9 / 15.6 / 10.0 / 7.0 / 9.7 / 21, 1024x1024x4096 46 / 49 / 29 / 22 / 16 / 41
    // (about 4 of each is the call; to binary32 the same).
    const int64_t cus = device_cus();
    const auto fits = [&](int64_t rows, int64_t cols) {
        return ceil_div(a.rows, rows) * ceil_div(b.rows, cols) <= cus;
    };
    if (fits(16, 16)) return launch_narrow<1, 1, 8, 2, OT>(a, b, k, out, s);
    if (fits(32, 16)) return launch_narrow<2, 1, 8, 2, OT>(a, b, k, out, s);
    if (fits(32, 32)) return launch_narrow<2, 2, 8, 2, OT>(a, b, k, out, s);
    if (fits(64, 32)) return launch_narrow<4, 2, 8, 1, OT>(a, b, k, out, s);
    // Two rounds of 64 x 64 outputs are faster than one of 128 x 128 where many columns
    // are summed: us, 64 x 64 / 128 x 128: 1792x848x2804 23 / 28, 166x6658x2723 22 / 27,
    // 1402x951x1610 18 / 19, 794x1835x724 13 / 12.
    const bool two_rounds = k > 2048 && ceil_div(a.rows, 64) * ceil_div(b.rows, 64) <= 2 * cus;
    if (fits(64, 64) || two_rounds) return launch_narrow<4, 4, 4, 2, OT>(a, b, k, out, s);
    // A round of 256 x 256 tiles takes about as long as one of two 128 x 128 tiles per
    // compute unit, which hold half of it: k = 4096, us to bfloat16, wide / 128 x 128:
    // 2048x4096 67 / 62, 2304x4096 69 / 91, 4096x4096 90 / 118, 4608x4096 151 / 143,
    // 6144x4096 152 / 174, 8192x8192 349 / 456 (to binary32 69 / 63, 70 / 91, 98 / 120,
    // 156 / 145, 157 / 176, 367 / 471).
    const TileOrder wide(ceil_div(a.rows, 256), ceil_div(b.rows, 256));
    const int64_t tiles = ceil_div(a.rows, 128) * ceil_div(b.rows, 128);
    if (a.rows >= kWideTile && b.rows >= kWideTile && k > 128 && ceil_div(wide.tiles(), cus) < ceil_div(tiles, 2 * cus)) {
        const dim3 grid(static_cast<unsigned>(std::min<int64_t>(wide.blocks(), cus / 8 * 8)));
        hipLaunchKernelGGL((matmul8_wide_kernel<OT>), grid, dim3(256), 0, s, a, b, static_cast<uint32_t>(pitch8(k)),
                           static_cast<uint32_t>(scale_pitch8(k)), wide, static_cast<OT*>(out));
        return check_launch("lsgd_matmul8");
    }
    return launch_tiles<4, 4, 2, 2, OT>(a, b, k, out, s);
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
    // 256 rows of a tile lie within 32-bit offsets
    if (k < 0 || k > (1 << 23)) return fail(LSGD_ERR_SIZE, "k=%lld outside [0, 2^23]", static_cast<long long>(k));
    LSGD_TRY(check_matrix(m, k, "a"));
    LSGD_TRY(check_matrix(n, k, "b"));
    LSGD_TRY(check_matrix(m, n, "out"));
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
    return odt == LSGD_F32 ? launch<float>(A, B, k, out, s) : launch<uint16_t>(A, B, k, out, s);
}

}  // extern "C"
