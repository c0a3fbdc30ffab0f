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

// A copy of rows: bound by the bytes of the rows read and written. A lane moves
// 8 elements; `lanes` (a power of two) of them walk one row, so that a
// workgroup holds 256 / lanes short rows or a part of a long one.
template <typename TT, typename OT, typename I>
__global__ __launch_bounds__(kBlock) void embed_lookup_kernel(const TT* __restrict__ table, int64_t rows, int64_t dim,
                                                              const I* __restrict__ tokens, int64_t n_tokens,
                                                              float scale, OT* __restrict__ out, int lanes) {
    const int per = kBlock / lanes;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * per + threadIdx.x / lanes; i < n_tokens;
         i += static_cast<int64_t>(gridDim.x) * per) {
        const int64_t t = token_row(tokens, i, rows);
        for (int64_t c = threadIdx.x % lanes * 8; c < dim; c += lanes * 8) {
            const int k = static_cast<int>(dim - c < 8 ? dim - c : 8);
            float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (t >= 0) {
                load8(table + t * dim + c, k, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= scale;
            }
            store8(out + i * dim + c, k, x);
        }
    }
}

template <typename TT, typename OT>
void launch_lookup(const void* table, int64_t rows, int64_t dim, const void* tokens, lsgd_index_type it, int64_t n,
                   float scale, void* out, hipStream_t s) {
    int lanes = 1;
    while (lanes < kBlock && lanes * 8 < dim) lanes *= 2;
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
// e % n_tokens) are sorted by token, equal tokens by entry; `first` and `last`
// bound each row's entries in the sorted order. Then every row of the gradient
// is written once by the wave that sums its entries; a row of many entries
// (frequent tokens hold up to a tenth of a text) is summed in pieces first, so
// that no wave has a long list to itself. Bound by the gradients read and the
// table written; the sort moves a few bytes per token.

constexpr int kSortTile = 2048;       // entries a workgroup of the radix sort holds
constexpr int kDigitBits = 9;         // two passes for tables of up to 2^18 - 1 rows
constexpr int kBins = 1 << kDigitBits;
constexpr int kRankMax = 4096;        // entries that are sorted by counting smaller ones
constexpr int kPiece = 64;            // sorted entries in a piece

struct Workers {
    const void* grads[kMaxWorkers];
    const void* tokens[kMaxWorkers];
};

struct Sorted {
    uint32_t* key;     // [E] row, or `rows` for tokens outside the table
    uint32_t* entry;   // [E]
    uint32_t* first;   // [rows]
    uint32_t* last;    // [rows]
};

template <typename I>
__device__ __forceinline__ uint32_t key_of(const Workers& w, uint32_t e, uint32_t n_tokens, uint32_t rows) {
    const uint32_t k = e / n_tokens;
    const I* t = static_cast<const I*>(w.tokens[k]);
    const int64_t v = static_cast<int64_t>(t[e - k * n_tokens]);
    return v >= 0 && v < static_cast<int64_t>(rows) ? static_cast<uint32_t>(v) : rows;
}

__global__ __launch_bounds__(kBlock) void clear_bounds_kernel(uint32_t* __restrict__ p, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kBlock)
        p[i] = 0;
}

// Rank of an entry = entries with a smaller key + earlier entries with the same
// one. A workgroup ranks 64 entries, its 16 waves counting over a sixteenth of
// all entries each; E^2 comparisons in one launch, against six for the radix
// sort (which takes over where E^2 shows).
template <typename I>
__global__ __launch_bounds__(1024) void rank_kernel(Workers w, uint32_t n_tokens, uint32_t E, uint32_t rows, Sorted s) {
    __shared__ uint32_t keys[kRankMax];
    __shared__ uint32_t part[3][16][64];
    for (uint32_t e = threadIdx.x; e < E; e += 1024) keys[e] = key_of<I>(w, e, n_tokens, rows);
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t e0 = blockIdx.x * 64, e = e0 + lane;
    const uint32_t k = e < E ? keys[e] : 0;
    const uint32_t span = (E + 15) / 16, j0 = min(wave * span, E), j1 = min(j0 + span, E);
    uint32_t lt = 0, eq = 0, before = 0;
    for (uint32_t j = j0; j < j1; ++j) {
        const uint32_t q = keys[j];
        lt += q < k;
        eq += q == k;
        before += q == k && j < e;
    }
    part[0][wave][lane] = lt;
    part[1][wave][lane] = eq;
    part[2][wave][lane] = before;
    __syncthreads();
    if (wave == 0 && e < E) {
        lt = eq = before = 0;
        for (int i = 0; i < 16; ++i) lt += part[0][i][lane], eq += part[1][i][lane], before += part[2][i][lane];
        s.key[lt + before] = k;
        s.entry[lt + before] = e;
        if (k < rows && before == 0) s.first[k] = lt, s.last[k] = lt + eq;
    }
}

// Radix sort, least significant digit first; three launches a pass: each
// workgroup's counts per digit, their running sum over (digit, workgroup), and
// the entries in their new places, in order.
template <typename I, bool First>
__device__ __forceinline__ uint32_t sort_key(const Workers& w, const uint32_t* key, uint32_t p, uint32_t n_tokens,
                                             uint32_t rows) {
    if constexpr (First) return key_of<I>(w, p, n_tokens, rows);
    return key[p];
}

template <typename I, bool First>
__global__ __launch_bounds__(kBlock) void digit_count_kernel(Workers w, const uint32_t* __restrict__ key,
                                                             uint32_t n_tokens, uint32_t E, uint32_t rows, int shift,
                                                             uint32_t* __restrict__ counts) {
    __shared__ uint32_t c[kBins];
    for (int i = threadIdx.x; i < kBins; i += kBlock) c[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortTile / kBlock; ++i) {
        const uint32_t p = blockIdx.x * kSortTile + i * kBlock + threadIdx.x;
        if (p < E) atomicAdd(&c[sort_key<I, First>(w, key, p, n_tokens, rows) >> shift & (kBins - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kBlock) counts[static_cast<size_t>(i) * gridDim.x + blockIdx.x] = c[i];
}

// counts[0..n) = sum of the counts before each; one workgroup.
__global__ __launch_bounds__(1024) void running_sum_kernel(uint32_t* __restrict__ counts, uint32_t n) {
    __shared__ uint32_t wave_sum[16];
    uint32_t carry = 0;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (uint32_t base = 0; base < n; base += 4096) {
        const uint32_t i = base + threadIdx.x * 4;
        uint32_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = i + j < n ? counts[i + j] : 0;
        const uint32_t mine = v[0] + v[1] + v[2] + v[3];
        uint32_t sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t o = __shfl_up(sum, d);
            if (lane >= static_cast<uint32_t>(d)) sum += o;
        }
        if (lane == 63) wave_sum[wave] = sum;
        __syncthreads();
        uint32_t before = carry, all = 0;
#pragma unroll
        for (uint32_t k = 0; k < 16; ++k) {
            const uint32_t x = wave_sum[k];
            before += k < wave ? x : 0;
            all += x;
        }
        carry += all;
        uint32_t at = before + sum - mine;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (i + j < n) counts[i + j] = at;
            at += v[j];
        }
        __syncthreads();
    }
}

template <typename I, bool First>
__global__ __launch_bounds__(kBlock) void digit_place_kernel(Workers w, const uint32_t* __restrict__ key,
                                                             const uint32_t* __restrict__ entry, uint32_t n_tokens,
                                                             uint32_t E, uint32_t rows, int shift,
                                                             const uint32_t* __restrict__ counts,
                                                             uint32_t* __restrict__ key_out,
                                                             uint32_t* __restrict__ entry_out) {
    constexpr int kWaves = kBlock / 64, kRounds = kSortTile / kBlock;
    __shared__ uint32_t c[kWaves][kBins];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < kWaves * kBins; i += kBlock) (&c[0][0])[i] = 0;
    __syncthreads();
    // A wave's 512 entries in order, 64 at a time: an entry's rank among its
    // wave's entries of the same digit is the count so far plus the lanes
    // before it.
    uint32_t k[kRounds], rank[kRounds];
    const uint32_t p0 = blockIdx.x * kSortTile + wave * (kRounds * 64) + lane;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const uint32_t p = p0 + r * 64;
        const bool in = p < E;
        k[r] = in ? sort_key<I, First>(w, key, p, n_tokens, rows) : 0;
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
    __syncthreads();
    for (int d = threadIdx.x; d < kBins; d += kBlock) {
        uint32_t at = counts[static_cast<size_t>(d) * gridDim.x + blockIdx.x];
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            const uint32_t n = c[v][d];
            c[v][d] = at;
            at += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const uint32_t p = p0 + r * 64;
        if (p < E) {
            const uint32_t to = c[wave][k[r] >> shift & (kBins - 1)] + rank[r];
            key_out[to] = k[r];
            entry_out[to] = First ? p : entry[p];
        }
    }
}

__global__ __launch_bounds__(kBlock) void row_bounds_kernel(Sorted s, uint32_t E, uint32_t rows) {
    const uint32_t p = blockIdx.x * kBlock + threadIdx.x;
    if (p >= E) return;
    const uint32_t k = s.key[p];
    if (k >= rows) return;
    if (p == 0 || s.key[p - 1] != k) s.first[k] = p;
    if (p + 1 == E || s.key[p + 1] != k) s.last[k] = p + 1;
}

// acc += the gradients of sorted entries [p, q), columns c.. of the lane, in order.
template <typename GT>
__device__ __forceinline__ void sum_entries(const Workers& w, const uint32_t* entry, uint32_t p, uint32_t q,
                                            uint32_t n_tokens, int64_t dim, int64_t c, int k, float (&acc)[8]) {
    for (; p < q; p += 64) {
        const uint32_t lane = threadIdx.x & 63, n = min(q - p, 64u);
        const uint32_t e = lane < n ? entry[p + lane] : 0;
        const uint32_t wk = e / n_tokens;
        const uint64_t at = reinterpret_cast<uint64_t>(w.grads[wk]) +
                            static_cast<uint64_t>(e - wk * n_tokens) * static_cast<uint64_t>(dim) * sizeof(GT);
        const uint32_t lo = static_cast<uint32_t>(at), hi = static_cast<uint32_t>(at >> 32);
        auto row = [&](uint32_t j) {
            // readlane gives a signed int: its low half must not be sign-extended
            const uint32_t l = __builtin_amdgcn_readlane(lo, j), h = __builtin_amdgcn_readlane(hi, j);
            return reinterpret_cast<const GT*>(static_cast<uint64_t>(h) << 32 | l) + c;
        };
        uint32_t j = 0;
        for (; j + 4 <= n; j += 4) {
            float x[4][8];
#pragma unroll
            for (int u = 0; u < 4; ++u) load8(row(j + u), k, x[u]);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] += x[u][i];
        }
        for (; j < n; ++j) {
            float x[8];
            load8(row(j), k, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += x[i];
        }
    }
}

// Partial sums of the rows with more than kPiece entries: a wave sums the
// entries of one aligned piece [64 c, 64 c + 64) of the sorted order that belong
// to the row of its first entry (slot 2c) or, if that is another, of its last
// (slot 2c + 1). No third row of a piece has that many entries.
template <typename GT>
__global__ __launch_bounds__(kBlock) void piece_sums_kernel(Workers w, Sorted s, uint32_t n_tokens, uint32_t E,
                                                            uint32_t rows, int64_t dim, uint32_t slabs,
                                                            float* __restrict__ slots) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t item = static_cast<uint64_t>(blockIdx.x) * (kBlock / 64) + (threadIdx.x >> 6);
    const uint32_t c = static_cast<uint32_t>(item / slabs), slab = static_cast<uint32_t>(item % slabs);
    const uint64_t p0 = static_cast<uint64_t>(c) * kPiece;
    if (p0 >= E) return;
    const uint32_t p = static_cast<uint32_t>(p0), q = min(p + kPiece, E);
    const int64_t col = static_cast<int64_t>(slab) * 512 + lane * 8;
    const int k = static_cast<int>(max(static_cast<int64_t>(0), min(dim - col, static_cast<int64_t>(8))));
    const uint32_t k0 = __builtin_amdgcn_readfirstlane(s.key[p]), k1 = __builtin_amdgcn_readfirstlane(s.key[q - 1]);
    for (int side = 0; side < 2; ++side) {
        const uint32_t v = side ? k1 : k0;
        if ((side && k1 == k0) || v >= rows) continue;
        const uint32_t a = __builtin_amdgcn_readfirstlane(s.first[v]), b = __builtin_amdgcn_readfirstlane(s.last[v]);
        if (b - a <= kPiece) continue;
        float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        sum_entries<GT>(w, s.entry, max(a, p), min(b, q), n_tokens, dim, col, k, acc);
        store8(slots + (2 * static_cast<int64_t>(c) + side) * dim + col, k, acc);
    }
}

// Every row: its entries' sum, or that of its pieces, times scale. A workgroup
// takes 16 rows; a wave one row's slab of 512 columns at a time.
constexpr int kRowsPerBlock = 16;

template <typename GT, typename OT>
__global__ __launch_bounds__(kBlock) void row_sums_kernel(Workers w, Sorted s, uint32_t n_tokens, uint32_t rows,
                                                          int64_t dim, uint32_t slabs, float scale,
                                                          const float* __restrict__ slots, OT* __restrict__ out,
                                                          bool accumulate) {
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (uint32_t v0 = blockIdx.x * kRowsPerBlock; v0 < rows; v0 += gridDim.x * kRowsPerBlock) {
        const uint32_t nv = min(static_cast<uint32_t>(kRowsPerBlock), rows - v0);
        const uint32_t mine = v0 + min(lane, nv - 1);
        const uint32_t firsts = s.first ? s.first[mine] : 0, lasts = s.first ? s.last[mine] : 0;
        for (uint32_t item = wave; item < nv * slabs; item += kBlock / 64) {
            const uint32_t r = item / slabs, slab = item % slabs;
            const uint32_t a = __builtin_amdgcn_readlane(firsts, r), b = __builtin_amdgcn_readlane(lasts, r);
            if (accumulate && a == b) continue;
            const int64_t col = static_cast<int64_t>(slab) * 512 + lane * 8;
            const int k = static_cast<int>(max(static_cast<int64_t>(0), min(dim - col, static_cast<int64_t>(8))));
            float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (b - a <= kPiece) {
                sum_entries<GT>(w, s.entry, a, b, n_tokens, dim, col, k, acc);
            } else {
                // a piece's slot 2c is the row of its first entry, so only the piece
                // in which the row starts, if not at its first entry, has it in 2c + 1
                for (uint32_t c = a / kPiece; c <= (b - 1) / kPiece; ++c) {
                    const bool starts = c == a / kPiece && s.key[static_cast<size_t>(c) * kPiece] != v0 + r;
                    float x[8];
                    load8(slots + (2 * static_cast<int64_t>(c) + starts) * dim + col, k, x);
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i] += x[i];
                }
            }
            OT* o = out + static_cast<int64_t>(v0 + r) * dim + col;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] *= scale;
            if (accumulate) {
                float x[8];
                load8(o, k, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] += x[i];
            }
            store8(o, k, acc);
        }
    }
}

// ---------------------------------------------------------------- host side

struct Layout {
    size_t key[2], entry[2], bounds, counts, slots, bytes;
};

int64_t sort_blocks(int64_t E) { return ceil_div(E, kSortTile); }

Layout layout_of(int64_t E, int64_t rows, int64_t dim) {
    Layout l{};
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
    l.bounds = take(8 * rows);
    l.counts = radix ? take(4 * kBins * sort_blocks(E)) : 0;
    l.slots = E > kPiece ? take(static_cast<size_t>(2 * ceil_div(E, kPiece)) * dim * 4) : 0;
    l.bytes = at;
    return l;
}

template <typename I>
lsgd_status sort_tokens(const Workers& w, uint32_t n_tokens, uint32_t E, uint32_t rows, const Layout& l, char* ws,
                        Sorted& s, hipStream_t st) {
    auto u32 = [&](size_t off) { return reinterpret_cast<uint32_t*>(ws + off); };
    s.first = u32(l.bounds);
    s.last = s.first + rows;
    const int64_t n = 2ll * rows;
    hipLaunchKernelGGL(clear_bounds_kernel, dim3(static_cast<unsigned>(std::min<int64_t>(2048, ceil_div(n, kBlock)))),
                       dim3(kBlock), 0, st, s.first, n);
    LSGD_TRY(check_launch("lsgd_embed_grad"));
    if (E <= kRankMax) {
        s.key = u32(l.key[0]);
        s.entry = u32(l.entry[0]);
        hipLaunchKernelGGL((rank_kernel<I>), dim3((E + 63) / 64), dim3(1024), 0, st, w, n_tokens, E, rows, s);
        return check_launch("lsgd_embed_grad");
    }
    const unsigned blocks = static_cast<unsigned>(sort_blocks(E));
    uint32_t* counts = u32(l.counts);
    int from = 0;
    for (int shift = 0; shift == 0 || rows >> shift; shift += kDigitBits) {   // keys reach `rows`
        const uint32_t *key = u32(l.key[from]), *entry = u32(l.entry[from]);
        uint32_t *key_out = u32(l.key[1 - from]), *entry_out = u32(l.entry[1 - from]);
        if (shift == 0)
            hipLaunchKernelGGL((digit_count_kernel<I, true>), dim3(blocks), dim3(kBlock), 0, st, w, key, n_tokens, E,
                               rows, shift, counts);
        else
            hipLaunchKernelGGL((digit_count_kernel<I, false>), dim3(blocks), dim3(kBlock), 0, st, w, key, n_tokens, E,
                               rows, shift, counts);
        hipLaunchKernelGGL(running_sum_kernel, dim3(1), dim3(1024), 0, st, counts, kBins * blocks);
        if (shift == 0)
            hipLaunchKernelGGL((digit_place_kernel<I, true>), dim3(blocks), dim3(kBlock), 0, st, w, key, entry,
                               n_tokens, E, rows, shift, counts, key_out, entry_out);
        else
            hipLaunchKernelGGL((digit_place_kernel<I, false>), dim3(blocks), dim3(kBlock), 0, st, w, key, entry,
                               n_tokens, E, rows, shift, counts, key_out, entry_out);
        LSGD_TRY(check_launch("lsgd_embed_grad"));
        from = 1 - from;
    }
    s.key = u32(l.key[from]);
    s.entry = u32(l.entry[from]);
    hipLaunchKernelGGL(row_bounds_kernel, dim3((E + kBlock - 1) / kBlock), dim3(kBlock), 0, st, s, E, rows);
    return check_launch("lsgd_embed_grad");
}

template <typename GT, typename OT>
lsgd_status sum_rows(const Workers& w, const Sorted& s, uint32_t n_tokens, uint32_t E, uint32_t rows, int64_t dim,
                     float scale, float* slots, void* out, bool accumulate, hipStream_t st) {
    const uint32_t slabs = static_cast<uint32_t>(ceil_div(dim, 512));
    if (E > kPiece) {
        const int64_t items = ceil_div(E, kPiece) * slabs;
        hipLaunchKernelGGL((piece_sums_kernel<GT>), dim3(static_cast<unsigned>(ceil_div(items, kBlock / 64))),
                           dim3(kBlock), 0, st, w, s, n_tokens, E, rows, dim, slabs, slots);
        LSGD_TRY(check_launch("lsgd_embed_grad"));
    }
    hipLaunchKernelGGL((row_sums_kernel<GT, OT>), dim3(static_cast<unsigned>(std::min<int64_t>(kMaxGridBlocks, ceil_div(rows, kRowsPerBlock)))),
                       dim3(kBlock), 0, st, w, s, n_tokens, rows, dim, slabs, scale, slots, static_cast<OT*>(out),
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
    LSGD_TRY(check_size(n_tokens * n_workers, "n_workers * n_tokens"));
    LSGD_TRY(check_size(rows, "rows"));
    LSGD_TRY(check_size(dim, "dim"));
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
        LSGD_TRY(check_buffer(workspace, 256, "workspace"));
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
    if (E > 0) {
        if (it == LSGD_I32) LSGD_TRY(sort_tokens<int32_t>(w, nt, e32, r32, l, ws, s, st));
        else LSGD_TRY(sort_tokens<int64_t>(w, nt, e32, r32, l, ws, s, st));
    }
    float* slots = reinterpret_cast<float*>(ws + l.slots);
    const bool acc = accumulate != 0;
    if (gdt == LSGD_F32 && odt == LSGD_F32)
        return sum_rows<float, float>(w, s, nt, e32, r32, dim, scale, slots, out, acc, st);
    if (gdt == LSGD_F32) return sum_rows<float, uint16_t>(w, s, nt, e32, r32, dim, scale, slots, out, acc, st);
    if (odt == LSGD_F32) return sum_rows<uint16_t, float>(w, s, nt, e32, r32, dim, scale, slots, out, acc, st);
    return sum_rows<uint16_t, uint16_t>(w, s, nt, e32, r32, dim, scale, slots, out, acc, st);
}

}  // extern "C"
