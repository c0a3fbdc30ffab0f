// Token table: rows looked up, and the table's gradient by sorted tokens
// (lsgd_layers.h).
#include "layers.hpp"

namespace lsgd {
namespace layers {
namespace {

// ---------------------------------------------------------------- lookup

template <typename I>
__device__ __forceinline__ int64_t token_row(const I* tokens, int64_t i, int64_t rows) {
    const int64_t t = static_cast<int64_t>(tokens[i]);
    return t >= 0 && t < rows ? t : -1;
}

// 16 bytes of a row of out from the same elements of a row of the table.
template <typename TT>
__device__ __forceinline__ void scaled_copy(const TT* t, float scale, float* o, int k) {
    float x[4] = {0, 0, 0, 0};
    if (t) load4(t, k, x);
    const f32x4 v = f32x4{x[0], x[1], x[2], x[3]} * scale;
    if (k < 4) return store4(o, k, v);
    __builtin_nontemporal_store(f32x4_u{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_u*>(o));
}
template <typename TT>
__device__ __forceinline__ void scaled_copy(const TT* t, float scale, uint16_t* o, int k) {
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (t) load8(t, k, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= scale;
    if (k < 8) return store8(o, k, x);
    u32x4_u2 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = f32_to_bf16x2(x[2 * i], x[2 * i + 1]);
    __builtin_nontemporal_store(a, reinterpret_cast<u32x4_u2*>(o));
}

// A copy of rows: bound by the bytes of the rows read and written. A lane moves
// 16 bytes of out; `lanes` (a power of two) of them walk one row, so that a
// workgroup holds 256 / lanes short rows or a part of a long one. 16384 rows of
// 4096 bfloat16: 33 us, 8.2 TB/s counting every row read (frequent rows come from
// the caches); with stores through the caches 43. Those keep out of the caches what is
// read next: with lsgd_quant8 of the rows behind the lookup (evenly spread tokens) the two
// take, past the caches / through them, 4.7 / 4.4 us for 256 rows of 1024, 13.9 / 13.3 for
// 2048 of 4096, 80 / 77 for 16384 (the lookup alone 2.3 / 2.3, 6.8 / 7.8, 39 / 45), and to
// binary32 6.6 / 6.4, 19.5 / 19.1 and, 8192 rows, 72 / 61 (alone 3.0 / 3.1, 9.5 / 13.0, 31 / 42).
template <typename TT, typename OT, typename I>
__global__ __launch_bounds__(kBlock) void embed_lookup_kernel(const TT* __restrict__ table, int64_t rows, int64_t dim,
                                                              const I* __restrict__ tokens, int64_t n_tokens,
                                                              float scale, OT* __restrict__ out, int lanes) {
    constexpr int kVec = 16 / sizeof(OT);
    const int per = kBlock / lanes;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * per + threadIdx.x / lanes; i < n_tokens;
         i += static_cast<int64_t>(gridDim.x) * per) {
        const int64_t t = token_row(tokens, i, rows);
        const float f = t >= 0 ? scale : 0.0f;
        for (int64_t c = threadIdx.x % lanes * kVec; c < dim; c += lanes * kVec)
            scaled_copy(t >= 0 ? table + t * dim + c : nullptr, f, out + i * dim + c,
                        static_cast<int>(min(dim - c, static_cast<int64_t>(kVec))));
    }
}

template <typename TT, typename OT>
void launch_lookup(const void* table, int64_t rows, int64_t dim, const void* tokens, lsgd_index_type it, int64_t n,
                   float scale, void* out, hipStream_t s) {
    int lanes = 1;
    while (lanes < kBlock && lanes * static_cast<int64_t>(16 / sizeof(OT)) < dim) lanes *= 2;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(kMaxGridBlocks, ceil_div(n, kBlock / lanes))));
    if (it == LSGD_I32)
        hipLaunchKernelGGL((embed_lookup_kernel<TT, OT, int32_t>), grid, dim3(kBlock), 0, s,
                           static_cast<const TT*>(table), rows, dim, static_cast<const int32_t*>(tokens), n, scale,
                           static_cast<OT*>(out), lanes);
    else
        hipLaunchKernelGGL((embed_lookup_kernel<TT, OT, int64_t>), grid, dim3(kBlock), 0, s,
                           static_cast<const TT*>(table), rows, dim, static_cast<const int64_t*>(tokens), n, scale,
                           static_cast<OT*>(out), lanes);
}

// ---------------------------------------------------------------- gradient
//
// The E = n_workers * n_tokens entries (entry e: worker e / n_tokens, position
// e % n_tokens) are sorted by token, equal tokens by entry. The sorted order is
// cut into pieces, and a wave sums a piece's gradients run by run of equal
// tokens. A row of no more entries than a piece has belongs to the wave in whose
// piece it starts, which writes it at once; of a longer one every piece's part
// goes to a slot, and a last kernel adds these. So the work is divided by
// entries, whatever the tokens' frequencies (a wave per row took 670 us where
// one row had a tenth of all entries). Rows without entries are written by the
// same launch. Bound by the gradients read and the table written; the sort
// moves a few bytes per token.

constexpr int kSortThreads = 512, kSortRounds = 8;
constexpr int kSortTile = kSortThreads * kSortRounds;   // entries a workgroup of the radix sort holds
constexpr int kDigitBits = 9;              // two passes for tables of up to 2^18 - 1 rows
constexpr int kBins = 1 << kDigitBits;
constexpr int kOwnSums = 256;              // up to so many workgroups each add up the counts before its own
constexpr int kDirectThreads = 1024, kDirectMax = 512;   // entries that need no sort of their own
constexpr int kRankBits = 13, kRankMax = 1 << kRankBits;   // entries that are sorted by counting smaller ones
// Sorted entries in a piece, which a wave's lanes hold: where the pieces are few,
// latency counts and a wave takes 8 (509 entries of 203 binary32: 22 us, with 16 24,
// with 32 30), else 32, as the slots cost bytes (131072 of 2048 bfloat16: 413 us,
// with 16 432).
constexpr int kFewPiece = 8, kManyPiece = 32;
constexpr int64_t kFewWaves = 1 << 14;
int piece_of(int64_t E, int64_t dim) { return E * ceil_div(dim, 512) <= kFewWaves * kFewPiece ? kFewPiece : kManyPiece; }
constexpr int64_t kMaxGradDim = 1 << 24;
constexpr int64_t kMaxEntries = 1 << 28;   // grids over pieces stay within a dispatch

struct Workers {
    const void* grads[kMaxWorkers];
    const void* tokens[kMaxWorkers];
};

struct Sorted {
    uint32_t* key;     // [E] row, or `rows` for tokens outside the table
    uint32_t* entry;   // [E]
    uint32_t* last;    // many entries only: [rows] end of the row's entries, 0 for a row without
    uint32_t* starts;  // [pieces] whether a row of several pieces starts in it
};

template <typename I>
__device__ __forceinline__ uint32_t key_of(const Workers& w, uint32_t e, uint32_t n_tokens, uint32_t rows) {
    const uint32_t k = e / n_tokens;
    const I* t = static_cast<const I*>(w.tokens[k]);
    const int64_t v = static_cast<int64_t>(t[e - k * n_tokens]);
    return v >= 0 && v < static_cast<int64_t>(rows) ? static_cast<uint32_t>(v) : rows;
}

// p[0..n) = 0, by `count` workgroups of which this is number `block`.
__device__ __forceinline__ void clear(uint32_t* p, uint32_t n, uint32_t block, uint32_t count) {
    for (uint64_t i = static_cast<uint64_t>(block) * blockDim.x + threadIdx.x; i < n;
         i += static_cast<uint64_t>(count) * blockDim.x)
        p[i] = 0;
}

// Zeros into the rows v0 + r, r < n <= 64, whose bit in `rows` is set: a workgroup of
// `waves` waves, 512 columns of a row at a time each.
template <typename OT>
__device__ __forceinline__ void zero_rows(OT* out, uint64_t v0, uint64_t rows, uint32_t n, int64_t dim, uint32_t slabs,
                                          uint32_t wave, uint32_t waves, uint32_t lane) {
    const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (uint32_t item = wave; item < n * slabs; item += waves)
        if (rows >> (item / slabs) & 1)
            store_slab(out + static_cast<int64_t>(v0 + item / slabs) * dim, slab_column(item % slabs, lane), dim, zero);
}

// Few entries. Key and entry in one number of type K; the rank of an entry is how many
// are smaller: each of the first ceil(E / 64) workgroups ranks 64, its 16 waves
// counting over a sixteenth of all entries each; E^2 comparisons in one launch,
// against five for the radix sort (which takes over where E^2 shows). The other
// workgroups write zeros into the rows without entries, 64 rows each, which they
// find among the tokens themselves.
template <typename K, typename I, typename OT>
__global__ __launch_bounds__(1024) void rank_kernel(Workers w, uint32_t n_tokens, uint32_t E, uint32_t rows, Sorted s,
                                                    OT* __restrict__ out, int64_t dim, uint32_t slabs) {
    __shared__ __align__(16) K keys[kRankMax];
    __shared__ uint32_t part[16][64];
    __shared__ uint32_t has[2];   // a bit for each of 64 rows
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t ranking = (E + 63) / 64;
    if (blockIdx.x >= ranking) {
        for (uint64_t v0 = static_cast<uint64_t>(blockIdx.x - ranking) * 64; v0 < rows;
             v0 += static_cast<uint64_t>(gridDim.x - ranking) * 64) {
            if (threadIdx.x < 2) has[threadIdx.x] = 0;
            __syncthreads();
            for (uint32_t e = threadIdx.x; e < E; e += 1024) {
                const uint64_t r = key_of<I>(w, e, n_tokens, rows) - v0;
                if (r < 64) atomicOr(&has[r / 32], 1u << (r % 32));
            }
            __syncthreads();
            const uint64_t empty = ~(static_cast<uint64_t>(has[1]) << 32 | has[0]);
            zero_rows(out, v0, empty, static_cast<uint32_t>(min(static_cast<uint64_t>(64), rows - v0)), dim, slabs, wave, 16,
                      lane);
            __syncthreads();
        }
        return;
    }
    const uint32_t span = (E + 63) / 64 * 4;   // of a wave, filled up with numbers that are smaller than none
    for (uint32_t e = threadIdx.x; e < 16 * span; e += 1024)
        keys[e] = e < E ? static_cast<K>(key_of<I>(w, e, n_tokens, rows)) << kRankBits | e : ~K{0};
    __syncthreads();
    const uint32_t e = blockIdx.x * 64 + lane;
    const K mine = keys[min(e, E - 1)];
    uint32_t smaller = 0;
#pragma unroll 4
    for (uint32_t j = wave * span; j < (wave + 1) * span; j += 4)
#pragma unroll
        for (int u = 0; u < 4; ++u) smaller += keys[j + u] < mine;
    part[wave][lane] = smaller;
    __syncthreads();
    if (wave == 0 && e < E) {
        uint32_t rank = 0;
        for (int i = 0; i < 16; ++i) rank += part[i][lane];
        s.key[rank] = static_cast<uint32_t>(mine >> kRankBits);
        s.entry[rank] = e;
    }
}

// Radix sort, least significant digit first; two launches a pass: each
// workgroup's counts per digit, and the entries in their new places, in order.
template <typename I, bool First>
__device__ __forceinline__ uint32_t sort_key(const Workers& w, const uint32_t* key, uint32_t p, uint32_t n_tokens,
                                             uint32_t rows) {
    if constexpr (First) return key_of<I>(w, p, n_tokens, rows);
    return key[p];
}

// counts[block][digit]; the workgroups behind the `blocks` that count clear `last`.
template <typename I, bool First>
__global__ __launch_bounds__(kSortThreads) void digit_count_kernel(Workers w, const uint32_t* __restrict__ key,
                                                                   uint32_t n_tokens, uint32_t E, uint32_t rows,
                                                                   int shift, uint32_t blocks,
                                                                   uint32_t* __restrict__ counts,
                                                                   uint32_t* __restrict__ last) {
    __shared__ uint32_t c[kBins];
    if (blockIdx.x >= blocks) return clear(last, rows, blockIdx.x - blocks, gridDim.x - blocks);
    for (int i = threadIdx.x; i < kBins; i += kSortThreads) c[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortRounds; ++i) {
        const uint32_t p = blockIdx.x * kSortTile + i * kSortThreads + threadIdx.x;
        if (p < E) atomicAdd(&c[sort_key<I, First>(w, key, p, n_tokens, rows) >> shift & (kBins - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kSortThreads) counts[static_cast<size_t>(blockIdx.x) * kBins + i] = c[i];
}

// For many workgroups: counts[b][d] = the entries of digit d in the workgroups
// before b, totals[d] = those of all. One workgroup per 64 digits, its waves
// adding an eighth of the workgroups each, twice.
__global__ __launch_bounds__(512) void block_sums_kernel(uint32_t* __restrict__ counts, uint32_t blocks,
                                                         uint32_t* __restrict__ totals) {
    __shared__ uint32_t part[8][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * 64 + lane;
    const uint32_t each = (blocks + 7) / 8, b0 = min(wave * each, blocks), b1 = min(b0 + each, blocks);
    uint32_t sum = 0;
#pragma unroll 8
    for (uint32_t b = b0; b < b1; ++b) sum += counts[static_cast<size_t>(b) * kBins + d];
    part[wave][lane] = sum;
    __syncthreads();
    uint32_t at = 0;
    for (uint32_t v = 0; v < wave; ++v) at += part[v][lane];
    for (uint32_t b = b0; b < b1; ++b) {
        const uint32_t n = counts[static_cast<size_t>(b) * kBins + d];
        counts[static_cast<size_t>(b) * kBins + d] = at;
        at += n;
    }
    if (wave == 7) totals[d] = at;
}

template <typename I, bool First>
__global__ __launch_bounds__(kSortThreads) void digit_place_kernel(Workers w, const uint32_t* __restrict__ key,
                                                                   const uint32_t* __restrict__ entry,
                                                                   uint32_t n_tokens, uint32_t E, uint32_t rows,
                                                                   int shift, const uint32_t* __restrict__ counts,
                                                                   const uint32_t* __restrict__ totals,
                                                                   uint32_t* __restrict__ key_out,
                                                                   uint32_t* __restrict__ entry_out) {
    constexpr int kWaves = kSortThreads / 64;
    static_assert(kSortThreads == kBins, "a lane adds up the counts of one digit");
    __shared__ uint32_t c[kWaves][kBins];
    __shared__ uint32_t wave_sum[kWaves];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t k[kSortRounds], e[kSortRounds], rank[kSortRounds];
    const uint32_t p0 = blockIdx.x * kSortTile + wave * (kSortRounds * 64) + lane;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const uint32_t p = min(p0 + r * 64, E - 1);
        k[r] = sort_key<I, First>(w, key, p, n_tokens, rows);
        e[r] = First ? p : entry[p];
    }
    // this lane's digit: its entries in the workgroups before this one, and in all
    uint32_t before = 0, all = 0;
    if (totals) {
        before = counts[static_cast<size_t>(blockIdx.x) * kBins + threadIdx.x];
        all = totals[threadIdx.x];
    } else {
#pragma unroll 16
        for (uint32_t b = 0; b < gridDim.x; ++b) {
            const uint32_t n = counts[static_cast<size_t>(b) * kBins + threadIdx.x];
            before += b < blockIdx.x ? n : 0;
            all += n;
        }
    }
    for (int i = threadIdx.x; i < kWaves * kBins; i += kSortThreads) (&c[0][0])[i] = 0;
    __syncthreads();
    // A wave's 512 entries in order, 64 at a time: an entry's rank among its
    // wave's entries of the same digit is the count so far plus the lanes before it.
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const bool in = p0 + r * 64 < E;
        const uint32_t d = k[r] >> shift & (kBins - 1);
        uint64_t same = __ballot(in);
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {
            const uint64_t v = __ballot(d >> b & 1);
            same &= (d >> b & 1) ? v : ~v;
        }
        const uint32_t ahead = __popcll(same & ((1ull << lane) - 1));
        if (in) {
            const uint32_t seen = c[wave][d];
            rank[r] = seen + ahead;
            __builtin_amdgcn_wave_barrier();
            if (ahead == 0) c[wave][d] = seen + static_cast<uint32_t>(__popcll(same));
        }
        __builtin_amdgcn_wave_barrier();
    }
    // where the digit starts: a running sum of the totals
    uint32_t sum = all;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(sum, d);
        if (lane >= static_cast<uint32_t>(d)) sum += o;
    }
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    uint32_t at = sum - all + before;
    for (uint32_t v = 0; v < wave; ++v) at += wave_sum[v];
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
        const uint32_t n = c[v][threadIdx.x];
        c[v][threadIdx.x] = at;
        at += n;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const uint32_t p = p0 + r * 64;
        if (p < E) {
            const uint32_t to = c[wave][k[r] >> shift & (kBins - 1)] + rank[r];
            key_out[to] = k[r];
            entry_out[to] = e[r];
        }
    }
}

__global__ __launch_bounds__(kBlock) void row_ends_kernel(Sorted s, uint32_t E, uint32_t rows) {
    const uint32_t p = blockIdx.x * kBlock + threadIdx.x;
    if (p >= E) return;
    const uint32_t k = s.key[p];
    if (k < rows && (p + 1 == E || s.key[p + 1] != k)) s.last[k] = p + 1;
}

// scale * acc (+ out) into a row, from the lane's column on.
template <typename OT>
__device__ __forceinline__ void put_row(OT* row, int64_t col, int64_t dim, float scale, bool accumulate,
                                        const float (&acc)[8]) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = acc[i] * scale;
    if (accumulate) {
        float x[8];
        load_slab(row, col, dim, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += x[i];
    }
    store_slab(row, col, dim, y);
}

// Workgroups below `piece_blocks`: a wave sums one piece, 512 columns. The
// others write zeros into the rows without entries, kZeroRows at a time.
constexpr uint32_t kZeroRows = 16;

template <int kPiece, typename GT, typename OT>
__global__ __launch_bounds__(kBlock) void sum_pieces_kernel(Workers w, Sorted s, uint32_t n_tokens, uint32_t E,
                                                            uint32_t rows, int64_t dim, uint32_t slabs, float scale,
                                                            uint32_t piece_blocks, float* __restrict__ slots,
                                                            OT* __restrict__ out, bool accumulate) {
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x >= piece_blocks) {
        const uint32_t stride = (gridDim.x - piece_blocks) * kZeroRows;
        for (uint64_t v0 = static_cast<uint64_t>(blockIdx.x - piece_blocks) * kZeroRows; v0 < rows; v0 += stride) {
            const uint32_t n = min(kZeroRows, static_cast<uint32_t>(rows - v0));
            const uint64_t empty = __ballot(lane < n && (E == 0 || s.last[v0 + min(lane, n - 1)] == 0));
            zero_rows(out, v0, empty, n, dim, slabs, wave, kBlock / 64, lane);
        }
        return;
    }
    const uint32_t item = blockIdx.x * (kBlock / 64) + wave, c = item / slabs, p = c * kPiece;
    if (p >= E) return;
    const int64_t col = slab_column(item % slabs, lane);
    // lanes: entries [p, p + 2 kPiece); keys past the end match none
    constexpr uint32_t kP = kPiece;
    const bool in = lane < 2 * kP && p + lane < E;
    const uint32_t key = in ? s.key[p + lane] : ~0u, e = in ? s.entry[p + lane] : 0, wk = e / n_tokens;
    const uint32_t ahead = lane < kP && p + lane >= kP ? s.key[p + lane - kP] : ~0u;   // of the kPiece entries before
    const uint64_t at = reinterpret_cast<uint64_t>(w.grads[wk]) +
                        static_cast<uint64_t>(e - wk * n_tokens) * static_cast<uint64_t>(dim) * sizeof(GT);
    const uint32_t lo = static_cast<uint32_t>(at), hi = static_cast<uint32_t>(at >> 32);
    const uint32_t n = min(kP, E - p);
    const uint32_t k_first = __builtin_amdgcn_readlane(key, 0), k_last = __builtin_amdgcn_readlane(key, n - 1);
    const uint32_t before = __popcll(__ballot(ahead == k_first)), with = __popcll(__ballot(key == k_first));
    const uint32_t of_last = __popcll(__ballot(key == k_last));
    // [from, to): the entries to add; first: they begin with a part of a longer row
    // that began before; leaves: they end with a part of one that goes on
    const bool first = before > 0 && before + with > kP;
    const uint32_t from = before > 0 && !first ? with : 0;
    const bool leaves = k_last < rows && !(k_last == k_first && before > 0) && of_last > kP;
    const uint64_t mine = __ballot(in && key < rows);   // tokens outside the table come last
    uint32_t to = n;
    if (!leaves && !(k_last == k_first && before > 0))
        to = max(n, 64 - static_cast<uint32_t>(__clzll(static_cast<long long>(__ballot(key == k_last)))));
    to = min(to, static_cast<uint32_t>(__popcll(mine)));
    if (item % slabs == 0 && lane == 0) s.starts[c] = leaves;
    const uint32_t next = __shfl_down(key, 1);
    uint64_t ends = __ballot(lane == 63 || next != key);
    if (to > 0) ends |= 1ull << (to - 1);
    auto row = [&](uint32_t j) {
        // readlane gives a signed int: its low half must not be sign-extended
        const uint32_t l = __builtin_amdgcn_readlane(lo, j), h = __builtin_amdgcn_readlane(hi, j);
        return reinterpret_cast<const GT*>(static_cast<uint64_t>(h) << 32 | l);
    };
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    // rows whose loads are under way (131072 entries of 2048: 4 360 us, 8 367, without once-only loads 373 and 413)
    constexpr int kAhead = 4;
    bool slot_first = first;
    for (uint32_t j = from; j < to; j += kAhead) {
        float x[kAhead][8];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) load_slab_once(row(min(j + u, to - 1)), col, dim, x[u]);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (j + u >= to) break;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += x[u][i];
            if (ends >> (j + u) & 1) {
                const bool slot_last = leaves && j + u == to - 1;
                if (slot_first || slot_last)
                    store_slab(slots + (2 * static_cast<int64_t>(c) + (slot_first ? 0 : 1)) * dim, col, dim, acc);
                else
                    put_row(out + static_cast<int64_t>(__builtin_amdgcn_readlane(key, j + u)) * dim, col, dim, scale,
                            accumulate, acc);
                slot_first = false;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
            }
        }
    }
}

// How many pieces behind piece c begin with row v, which fills the first of them.
template <int kPiece>
__device__ __forceinline__ uint32_t pieces_behind(const uint32_t* key, uint32_t c, uint32_t pieces, uint32_t v) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t step = 1, lo = c + 1, hi = pieces;   // piece lo begins with v; the 64 from it on, then all others
    for (;;) {
        const uint64_t at = lo + static_cast<uint64_t>(lane) * step;
        const uint32_t n = __popcll(__ballot(at < hi && key[min(at, static_cast<uint64_t>(hi - 1)) * kPiece] == v));
        lo += (n - 1) * step;
        if (step == 1 && (n < 64 || lo + 1 >= hi)) return lo - c;
        if (step > 1) hi = min(hi, lo + step);
        step = max(1u, (hi - lo + 63) / 64);
    }
}

// Rows of several pieces: a workgroup adds the slot 2c + 1 of the piece c in which
// the row starts and the following pieces' slots 2c, divided over its waves in
// order, then the waves' sums in order. It looks at a few pieces, 512 columns. A
// frequent row takes as long as a wave has slots to add, so with small pieces twice the
// waves look at half the pieces (118000 entries of 40, a tenth in one row: 88 us
// instead of 102; with large ones, 131072 of 2048, 370 instead of 362).
constexpr uint32_t join_pieces(int piece) { return piece == kFewPiece ? 4 : 8; }
constexpr int join_threads(int piece) { return piece == kFewPiece ? 1024 : 512; }

template <int kPiece, typename OT>
__global__ __launch_bounds__(join_threads(kPiece)) void join_pieces_kernel(Sorted s, uint32_t pieces, int64_t dim, uint32_t slabs,
                                                             float scale, const float* __restrict__ slots,
                                                             OT* __restrict__ out, bool accumulate) {
    constexpr uint32_t kWaves = join_threads(kPiece) / 64, kJoin = join_pieces(kPiece);
    __shared__ float sums[kWaves - 1][512];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t c0 = blockIdx.x / slabs * kJoin;
    const int64_t col = slab_column(blockIdx.x % slabs, lane);
    const uint32_t c_mine = c0 + lane;
    const bool start = lane < kJoin && c_mine < pieces && s.starts[c_mine] != 0;
    const uint32_t v_mine = start ? s.key[static_cast<size_t>(c_mine) * kPiece + kPiece - 1] : 0;
    const uint32_t last_mine = start && s.last ? s.last[v_mine] : 0;
    for (uint64_t todo = __ballot(start); todo; todo &= todo - 1) {
        const uint32_t at_lane = static_cast<uint32_t>(__ffsll(static_cast<unsigned long long>(todo))) - 1, c = c0 + at_lane;
        const uint32_t v = __builtin_amdgcn_readlane(v_mine, at_lane), last = __builtin_amdgcn_readlane(last_mine, at_lane);
        const uint32_t n = s.last ? (last - 1) / kPiece - c + 1 : 1 + pieces_behind<kPiece>(s.key, c, pieces, v), each = (n + kWaves - 1) / kWaves;
        const uint32_t from = min(wave * each, n), to = min(from + each, n);
        const float* slot = slots + 2 * static_cast<int64_t>(c) * dim;
        float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        uint32_t i = from;
        if (i == 0) {
            load_slab(slot + dim, col, dim, acc);
            i = 1;
        }
        for (; i + 8 <= to; i += 8) {
            float x[8][8];
#pragma unroll
            for (int u = 0; u < 8; ++u) load_slab(slot + 2 * static_cast<int64_t>(i + u) * dim, col, dim, x[u]);
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += x[u][j];
        }
        for (; i < to; ++i) {
            float x[8];
            load_slab(slot + 2 * static_cast<int64_t>(i) * dim, col, dim, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += x[j];
        }
        if (wave > 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[wave - 1][lane + j * 64] = acc[j];
        __syncthreads();
        if (wave == 0) {
            for (uint32_t u = 1; u < kWaves; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += sums[u - 1][lane + j * 64];
            put_row(out + static_cast<int64_t>(v) * dim, col, dim, scale, accumulate, acc);
        }
        __syncthreads();
    }
}

// The fewest entries: no sort, no workspace, one launch. A workgroup takes 64 rows of
// the table, 512 columns. It puts the entries of its rows in order (a stable
// counting sort by row in LDS), each of its 16 waves sums a sixteenth of them run by
// run, and runs that reach over several waves meet in LDS, in order.
template <typename I, typename GT, typename OT>
__global__ __launch_bounds__(kDirectThreads) void direct_kernel(Workers w, uint32_t n_tokens, uint32_t E, uint32_t rows,
                                                            int64_t dim, float scale, OT* __restrict__ out,
                                                            bool accumulate) {
    constexpr uint32_t kWaves = kDirectThreads / 64;
    __shared__ float parts[kWaves][2][512];   // of a wave's first run and its last, where they are not whole
    __shared__ uint32_t before[kWaves][64];   // entries of a row in the waves before
    __shared__ uint32_t entry[kDirectMax], row_of[kDirectMax];
    __shared__ uint32_t row_start[65];
    __shared__ uint32_t joins[kWaves + 1];    // bit 0: a wave's first run began before, 1: it is the wave's only one
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t col = slab_column(blockIdx.y, lane);
    const uint32_t key = threadIdx.x < E ? key_of<I>(w, threadIdx.x, n_tokens, rows) : rows;
    const uint32_t v0 = blockIdx.x * 64;
    const uint32_t d = key - v0;
    const bool in = key < rows && key >= v0 && d < 64;
    before[wave][lane] = 0;
    __builtin_amdgcn_wave_barrier();
    uint64_t same = __ballot(in);
#pragma unroll
    for (int b = 0; b < 6; ++b) {
        const uint64_t v = __ballot(d >> b & 1);
        same &= (d >> b & 1) ? v : ~v;
    }
    const uint32_t ahead = __popcll(same & ((1ull << lane) - 1));
    if (in && ahead == 0) before[wave][d] = static_cast<uint32_t>(__popcll(same));
    __syncthreads();
    if (wave == 0) {
        uint32_t n = 0;
#pragma unroll
        for (uint32_t v = 0; v < kWaves; ++v) {
            const uint32_t c = before[v][lane];
            before[v][lane] = n;
            n += c;
        }
        uint32_t sum = n;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const uint32_t o = __shfl_up(sum, step);
            if (lane >= static_cast<uint32_t>(step)) sum += o;
        }
        row_start[lane + 1] = sum;
        if (lane == 0) row_start[0] = 0, joins[kWaves] = 0;
    }
    __syncthreads();
    const uint32_t n = row_start[64];
    if (in) {
        const uint32_t at = row_start[d] + before[wave][d] + ahead;
        entry[at] = threadIdx.x;
        row_of[at] = d;
    }
    __syncthreads();
    const uint32_t each = (n + kWaves - 1) / kWaves, p = min(wave * each, n), q = min(p + each, n);
    bool first = false, leaves = false, whole = false;
    if (p < q) {
        const uint32_t mine = min(p + lane, q - 1), e = entry[mine], r = row_of[mine], wk = e / n_tokens;
        const uint64_t at = reinterpret_cast<uint64_t>(w.grads[wk]) +
                            static_cast<uint64_t>(e - wk * n_tokens) * static_cast<uint64_t>(dim) * sizeof(GT);
        const uint32_t lo = static_cast<uint32_t>(at), hi = static_cast<uint32_t>(at >> 32), len = q - p;
        const uint32_t r_first = __builtin_amdgcn_readlane(r, 0), r_last = __builtin_amdgcn_readlane(r, len - 1);
        first = p > 0 && row_of[p - 1] == r_first;
        leaves = q < n && row_of[q] == r_last;
        whole = r_first == r_last;
        const uint32_t next = __shfl_down(r, 1);
        const uint64_t ends = __ballot(lane == len - 1 || (lane < len && next != r));
        auto row = [&](uint32_t j) {
            // readlane gives a signed int: its low half must not be sign-extended
            const uint32_t l = __builtin_amdgcn_readlane(lo, j), h = __builtin_amdgcn_readlane(hi, j);
            return reinterpret_cast<const GT*>(static_cast<uint64_t>(h) << 32 | l);
        };
        float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        bool part = first;
        constexpr int kAhead = 4;
        for (uint32_t j = 0; j < len; j += kAhead) {
            float x[kAhead][8];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) load_slab_once(row(min(j + u, len - 1)), col, dim, x[u]);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (j + u >= len) break;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] += x[u][i];
                if (ends >> (j + u) & 1) {
                    if (part || (leaves && j + u == len - 1)) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) parts[wave][part ? 0 : 1][lane + i * 64] = acc[i];
                    } else {
                        put_row(out + static_cast<int64_t>(v0 + __builtin_amdgcn_readlane(r, j + u)) * dim, col, dim,
                                scale, accumulate, acc);
                    }
                    part = false;
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
                }
            }
        }
    }
    if (lane == 0) joins[wave] = (first ? 1u : 0u) | (whole ? 2u : 0u);
    if (!accumulate) {
        const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const uint32_t here = min(64u, rows - v0);
        for (uint32_t r = wave; r < here; r += kWaves)
            if (row_start[r] == row_start[r + 1]) store_slab(out + static_cast<int64_t>(v0 + r) * dim, col, dim, zero);
    }
    __syncthreads();
    if (leaves && !(first && whole)) {   // this wave's last run began in it and goes on
        float acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = parts[wave][1][lane + i * 64];
        for (uint32_t v = wave + 1;; ++v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += parts[v][0][lane + i * 64];
            if (!(joins[v] & 2) || !(joins[v + 1] & 1)) break;
        }
        put_row(out + static_cast<int64_t>(v0 + row_of[q - 1]) * dim, col, dim, scale, accumulate, acc);
    }
}

// ---------------------------------------------------------------- host side

struct Layout {
    size_t key[2], entry[2], last, starts, counts, totals, slots, bytes;
};

int64_t sort_blocks(int64_t E) { return ceil_div(E, kSortTile); }

// Whether direct_kernel does it: up to 512 entries while its workgroups fit the card
// at once. us, direct / sorted (rows x columns, entries): 5003 x 203, 509 14 / 21;
// 100 x 4096, 250 13 / 20; 32000 x 1024, 510 47 / 43; 131072 x 2048, 250 128 / 112;
// 2 x 256, 500 13 to 22 / 20, 1024 43 / 20.
bool direct(int64_t E, int64_t rows, int64_t dim) {
    return E <= kDirectMax && ceil_div(rows, 64) * ceil_div(dim, 512) <= 2 * device_cus();
}

Layout layout_of(int64_t E, int64_t rows, int64_t dim) {
    Layout l{};
    if (direct(E, rows, dim)) return l;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    const bool radix = E > kRankMax;
    l.key[0] = take(4 * E);
    l.entry[0] = take(4 * E);
    l.key[1] = radix ? take(4 * E) : 0;
    l.entry[1] = radix ? take(4 * E) : 0;
    l.last = radix ? take(4 * rows) : 0;
    l.counts = radix ? take(4 * kBins * sort_blocks(E)) : 0;
    l.totals = radix ? take(4 * kBins) : 0;
    const int64_t pieces = ceil_div(E, piece_of(E, dim));
    l.starts = take(4 * pieces);
    l.slots = pieces > 1 ? take(static_cast<size_t>(2 * pieces) * dim * 4) : 0;
    l.bytes = at;
    return l;
}

// Sorts the entries; few of them: fills out's rows without entries as well, unless
// `out` is null.
template <typename I, typename OT>
lsgd_status sort_tokens(const Workers& w, uint32_t n_tokens, uint32_t E, uint32_t rows, int64_t dim, const Layout& l,
                        char* ws, Sorted& s, OT* out, hipStream_t st) {
    auto u32 = [&](size_t off) { return reinterpret_cast<uint32_t*>(ws + off); };
    s.starts = u32(l.starts);
    if (E <= kRankMax) {
        s.key = u32(l.key[0]);
        s.entry = u32(l.entry[0]);
        const int64_t zeros = out ? std::min<int64_t>(4096, ceil_div(rows, 64)) : 0;
        const dim3 grid(static_cast<unsigned>((E + 63) / 64 + zeros));
        const uint32_t slabs = static_cast<uint32_t>(ceil_div(dim, 512));
        if (rows < 1u << (32 - kRankBits))   // keys reach `rows`
            hipLaunchKernelGGL((rank_kernel<uint32_t, I, OT>), grid, dim3(1024), 0, st, w, n_tokens, E, rows, s, out, dim,
                               slabs);
        else
            hipLaunchKernelGGL((rank_kernel<uint64_t, I, OT>), grid, dim3(1024), 0, st, w, n_tokens, E, rows, s, out, dim,
                               slabs);
        return check_launch("lsgd_embed_grad");
    }
    s.last = u32(l.last);
    const unsigned clears = static_cast<unsigned>(std::min<int64_t>(1024, ceil_div(rows, 4 * kBlock)));
    const unsigned blocks = static_cast<unsigned>(sort_blocks(E));
    uint32_t *counts = u32(l.counts), *totals = blocks > kOwnSums ? u32(l.totals) : nullptr;
    int from = 0;
    for (int shift = 0; shift == 0 || (shift < 32 && rows >> shift); shift += kDigitBits) {   // keys reach `rows`
        const uint32_t *key = u32(l.key[from]), *entry = u32(l.entry[from]);
        uint32_t *key_out = u32(l.key[1 - from]), *entry_out = u32(l.entry[1 - from]);
        if (shift == 0)
            hipLaunchKernelGGL((digit_count_kernel<I, true>), dim3(blocks + clears), dim3(kSortThreads), 0, st, w, key,
                               n_tokens, E, rows, shift, blocks, counts, s.last);
        else
            hipLaunchKernelGGL((digit_count_kernel<I, false>), dim3(blocks), dim3(kSortThreads), 0, st, w, key, n_tokens,
                               E, rows, shift, blocks, counts, s.last);
        if (totals)
            hipLaunchKernelGGL(block_sums_kernel, dim3(kBins / 64), dim3(512), 0, st, counts, blocks, totals);
        if (shift == 0)
            hipLaunchKernelGGL((digit_place_kernel<I, true>), dim3(blocks), dim3(kSortThreads), 0, st, w, key, entry,
                               n_tokens, E, rows, shift, counts, totals, key_out, entry_out);
        else
            hipLaunchKernelGGL((digit_place_kernel<I, false>), dim3(blocks), dim3(kSortThreads), 0, st, w, key, entry,
                               n_tokens, E, rows, shift, counts, totals, key_out, entry_out);
        LSGD_TRY(check_launch("lsgd_embed_grad"));
        from = 1 - from;
    }
    s.key = u32(l.key[from]);
    s.entry = u32(l.entry[from]);
    hipLaunchKernelGGL(row_ends_kernel, dim3((E + kBlock - 1) / kBlock), dim3(kBlock), 0, st, s, E, rows);
    return check_launch("lsgd_embed_grad");
}

template <int kPiece, typename GT, typename OT>
lsgd_status sum_rows_of(const Workers& w, const Sorted& s, uint32_t n_tokens, uint32_t E, uint32_t rows, int64_t dim,
                        float scale, float* slots, OT* out, bool accumulate, hipStream_t st) {
    const int64_t slabs = ceil_div(dim, 512), pieces = ceil_div(E, kPiece);
    const int64_t piece_blocks = ceil_div(pieces * slabs, kBlock / 64);
    const bool zeroed = E > 0 && E <= kRankMax;   // by the launch that sorted
    const int64_t zero_blocks = accumulate || zeroed ? 0 : std::min<int64_t>(1 << 20, ceil_div(rows, kZeroRows));
    hipLaunchKernelGGL((sum_pieces_kernel<kPiece, GT, OT>), dim3(static_cast<unsigned>(piece_blocks + zero_blocks)),
                       dim3(kBlock), 0, st, w, s, n_tokens, E, rows, dim, static_cast<uint32_t>(slabs), scale,
                       static_cast<uint32_t>(piece_blocks), slots, out, accumulate);
    LSGD_TRY(check_launch("lsgd_embed_grad"));
    if (pieces > 1) {
        hipLaunchKernelGGL((join_pieces_kernel<kPiece, OT>), dim3(static_cast<unsigned>(ceil_div(pieces, join_pieces(kPiece)) * slabs)),
                           dim3(join_threads(kPiece)), 0, st, s, static_cast<uint32_t>(pieces), dim, static_cast<uint32_t>(slabs), scale,
                           slots, out, accumulate);
        LSGD_TRY(check_launch("lsgd_embed_grad"));
    }
    return LSGD_OK;
}

template <typename GT, typename OT>
lsgd_status sum_rows(const Workers& w, const Sorted& s, uint32_t n_tokens, uint32_t E, uint32_t rows, int64_t dim,
                     float scale, float* slots, OT* out, bool accumulate, hipStream_t st) {
    return piece_of(E, dim) == kManyPiece
               ? sum_rows_of<kManyPiece, GT>(w, s, n_tokens, E, rows, dim, scale, slots, out, accumulate, st)
               : sum_rows_of<kFewPiece, GT>(w, s, n_tokens, E, rows, dim, scale, slots, out, accumulate, st);
}

template <typename I, typename GT, typename OT>
lsgd_status launch_direct(const Workers& w, uint32_t n_tokens, uint32_t E, uint32_t rows, int64_t dim, float scale, OT* out,
                          bool accumulate, hipStream_t st) {
    const int64_t slabs = ceil_div(dim, 512);
    const dim3 grid(static_cast<unsigned>(ceil_div(rows, 64)), static_cast<unsigned>(slabs));
    hipLaunchKernelGGL((direct_kernel<I, GT, OT>), grid, dim3(kDirectThreads), 0, st, w, n_tokens, E, rows, dim, scale, out,
                       accumulate);
    return check_launch("lsgd_embed_grad");
}

lsgd_status check_index_type(lsgd_index_type it) {
    return it == LSGD_I32 || it == LSGD_I64 ? LSGD_OK
                                            : fail(LSGD_ERR_DTYPE, "index type %d", static_cast<int>(it));
}

lsgd_status check_grad_sizes(int32_t n_workers, int64_t n_tokens, int64_t rows, int64_t dim) {
    if (n_workers < 1 || n_workers > LSGD_MAX_WORKERS)
        return fail(LSGD_ERR_SIZE, "n_workers=%d outside [1, %d]", n_workers, LSGD_MAX_WORKERS);
    LSGD_TRY(check_size(n_tokens, "n_tokens"));
    if (n_tokens * n_workers > kMaxEntries)
        return fail(LSGD_ERR_SIZE, "n_workers * n_tokens=%lld above 2^28", static_cast<long long>(n_tokens * n_workers));
    LSGD_TRY(check_size(rows, "rows"));
    if (dim < 0 || dim > kMaxGradDim)
        return fail(LSGD_ERR_SIZE, "dim=%lld outside [0, 2^24]", static_cast<long long>(dim));
    LSGD_TRY(check_matrix(n_tokens * n_workers, dim, "gradients"));
    return check_matrix(rows, dim, "out");
}

}  // namespace
}  // namespace layers
}  // namespace lsgd

using namespace lsgd;
using namespace lsgd::layers;

extern "C" {

LSGD_API lsgd_status lsgd_embed_lookup(const void* table, lsgd_dtype tdt, int64_t rows, int64_t dim,
                                       const void* tokens, lsgd_index_type it, int64_t n_tokens, float scale,
                                       void* out, lsgd_dtype odt, void* stream) {
    LSGD_TRY(check_dtype(tdt, "table dtype"));
    LSGD_TRY(check_dtype(odt, "out dtype"));
    LSGD_TRY(check_index_type(it));
    LSGD_TRY(check_size(rows, "rows"));
    LSGD_TRY(check_size(dim, "dim"));
    LSGD_TRY(check_size(n_tokens, "n_tokens"));
    LSGD_TRY(check_matrix(rows, dim, "table"));
    LSGD_TRY(check_matrix(n_tokens, dim, "out"));
    if (n_tokens == 0 || dim == 0) return LSGD_OK;
    if (rows > 0) LSGD_TRY(check_buffer(table, 16, "table"));
    const int64_t isz = it == LSGD_I32 ? 4 : 8;
    LSGD_TRY(check_buffer(tokens, isz, "tokens"));
    LSGD_TRY(check_buffer(out, 16, "out"));
    Ranges<3> ranges;
    ranges.add(table, rows * dim * elem_size(tdt), false, "table");
    ranges.add(tokens, n_tokens * isz, false, "tokens");
    ranges.add(out, n_tokens * dim * elem_size(odt), true, "out");
    LSGD_TRY(ranges.check());
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (tdt == LSGD_F32 && odt == LSGD_F32)
        launch_lookup<float, float>(table, rows, dim, tokens, it, n_tokens, scale, out, s);
    else if (tdt == LSGD_F32)
        launch_lookup<float, uint16_t>(table, rows, dim, tokens, it, n_tokens, scale, out, s);
    else if (odt == LSGD_F32)
        launch_lookup<uint16_t, float>(table, rows, dim, tokens, it, n_tokens, scale, out, s);
    else
        launch_lookup<uint16_t, uint16_t>(table, rows, dim, tokens, it, n_tokens, scale, out, s);
    return check_launch("lsgd_embed_lookup");
}

LSGD_API lsgd_status lsgd_embed_grad_workspace_size(int32_t n_workers, int64_t n_tokens, int64_t rows, int64_t dim,
                                                    size_t* bytes) {
    LSGD_TRY(check_grad_sizes(n_workers, n_tokens, rows, dim));
    if (!bytes) return fail(LSGD_ERR_NULL, "bytes is NULL");
    const int64_t E = n_tokens * n_workers;
    *bytes = E > 0 && rows > 0 && dim > 0 ? layout_of(E, rows, dim).bytes : 0;
    return LSGD_OK;
}

LSGD_API lsgd_status lsgd_embed_grad(const void* const* grads, lsgd_dtype gdt, const void* const* tokens,
                                     lsgd_index_type it, int32_t n_workers, int64_t n_tokens, int64_t rows,
                                     int64_t dim, float scale, void* out, lsgd_dtype odt, int32_t accumulate,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    LSGD_TRY(check_dtype(gdt, "gradient dtype"));
    LSGD_TRY(check_dtype(odt, "out dtype"));
    LSGD_TRY(check_index_type(it));
    LSGD_TRY(check_grad_sizes(n_workers, n_tokens, rows, dim));
    const int64_t E = n_tokens * n_workers;
    if (rows == 0 || dim == 0 || (E == 0 && accumulate)) return LSGD_OK;
    LSGD_TRY(check_buffer(out, 16, "out"));
    Layout l{};
    Workers w{};
    if (E > 0) {
        if (!grads || !tokens) return fail(LSGD_ERR_NULL, "grads or tokens is NULL");
        l = layout_of(E, rows, dim);
        if (l.bytes > 0) LSGD_TRY(check_buffer(workspace, 256, "workspace"));
        if (workspace_bytes < l.bytes)
            return fail(LSGD_ERR_SIZE, "workspace of %zu bytes, %zu needed", workspace_bytes, l.bytes);
        const int64_t isz = it == LSGD_I32 ? 4 : 8;
        Ranges<2 * LSGD_MAX_WORKERS + 2> ranges;
        ranges.add(out, rows * dim * elem_size(odt), true, "out");
        ranges.add(workspace, static_cast<int64_t>(l.bytes), true, "workspace");
        for (int32_t i = 0; i < n_workers; ++i) {
            LSGD_TRY(check_buffer(grads[i], 16, "a gradient"));
            LSGD_TRY(check_buffer(tokens[i], isz, "an array of tokens"));
            ranges.add(grads[i], n_tokens * dim * elem_size(gdt), false, "a gradient");
            ranges.add(tokens[i], n_tokens * isz, false, "an array of tokens");
            w.grads[i] = grads[i];
            w.tokens[i] = tokens[i];
        }
        LSGD_TRY(ranges.check());
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    Sorted s{};
    const uint32_t nt = static_cast<uint32_t>(n_tokens), e32 = static_cast<uint32_t>(E), r32 = static_cast<uint32_t>(rows);
    float* slots = reinterpret_cast<float*>(ws + l.slots);
    const bool acc = accumulate != 0;
    const auto run = [&](auto grad_type, auto* o) -> lsgd_status {
        using GT = decltype(grad_type);
        if (E > 0 && direct(E, rows, dim))
            return it == LSGD_I32 ? launch_direct<int32_t, GT>(w, nt, e32, r32, dim, scale, o, acc, st)
                                  : launch_direct<int64_t, GT>(w, nt, e32, r32, dim, scale, o, acc, st);
        if (E > 0) {
            auto* zeroed = acc ? nullptr : o;
            if (it == LSGD_I32) LSGD_TRY(sort_tokens<int32_t>(w, nt, e32, r32, dim, l, ws, s, zeroed, st));
            else LSGD_TRY(sort_tokens<int64_t>(w, nt, e32, r32, dim, l, ws, s, zeroed, st));
        }
        return sum_rows<GT>(w, s, nt, e32, r32, dim, scale, slots, o, acc, st);
    };
    float* o32 = static_cast<float*>(out);
    uint16_t* o16 = static_cast<uint16_t*>(out);
    if (gdt == LSGD_F32) return odt == LSGD_F32 ? run(float{}, o32) : run(float{}, o16);
    return odt == LSGD_F32 ? run(uint16_t{}, o32) : run(uint16_t{}, o16);
}

}  // extern "C"
