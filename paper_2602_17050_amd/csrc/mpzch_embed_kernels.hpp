// Typed lookup of embedding rows with scaling and dropout, its gradient by sorted slots, and the optimizer step of the rows
// that a batch touched.
//
// With s_i the slot of position i, row(s) = s mod num_rows, f = scale * 65536 / (65536 - T):
//   lookup     out[i, j] = f * rows[row(s_i), j] where (i, j) is kept, else 0; s_i < 0 is padding, a row of zeros
//   gradient   G[r, j]   = f * sum of grad[i, j] over the kept (i, j) with row(s_i) = r, for every r that is named
//   step       w[r] -= lr G[r]  or  state[r] += mean_j G[r, j]^2, w[r] -= lr G[r] / (sqrt(state[r]) + eps)
// Whether (i, j) is kept is computed wherever it is needed and stored nowhere: word(i, j) = output i * ceil(dim / 4) + j / 4
// of the SplitMix64 generator that starts at the seed holds the 16-bit draws of four neighbouring elements, and an element is
// dropped where its draw is below T.  16 bits because a word of 64 costs two 64-bit products, six quarter-rate instructions.
#pragma once
#include "mpzch_common.hpp"

#include <type_traits>

namespace mpzch {

// V neighbouring elements as they lie in memory; aligned to their size, to 16 bytes at most
template <typename E, int V>
struct PackOf {
    typedef E type __attribute__((ext_vector_type(V), aligned(V * sizeof(E) < 16 ? V * sizeof(E) : 16)));
};
template <typename E, int V>
using Pack = typename PackOf<E, V>::type;
template <int V>
using Floats = float __attribute__((ext_vector_type(V)));

template <typename E, int V>
__device__ __forceinline__ Floats<V> load_floats(const char *at)
{
    return __builtin_convertvector(*reinterpret_cast<const Pack<E, V> *>(at), Floats<V>);
}
// (rounded once, to nearest, ties to even)
template <typename E, int V>
__device__ __forceinline__ void store_floats(char *at, Floats<V> v)
{
    typedef E to __attribute__((ext_vector_type(V)));
    *reinterpret_cast<Pack<E, V> *>(at) = __builtin_convertvector(v, to);
}

// the element types of the C ABI
constexpr int kF32 = 0, kBf16 = 1, kF16 = 2;

template <int V>
__device__ __forceinline__ Floats<V> load_typed(int type, const char *base, int64_t element)
{
    if (type == kF32) return load_floats<float, V>(base + element * 4);
    if (type == kBf16) return load_floats<__bf16, V>(base + element * 2);
    return load_floats<_Float16, V>(base + element * 2);
}
template <int V>
__device__ __forceinline__ void store_typed(int type, char *base, int64_t element, Floats<V> v)
{
    if (type == kF32) store_floats<float, V>(base + element * 4, v);
    else if (type == kBf16) store_floats<__bf16, V>(base + element * 2, v);
    else store_floats<_Float16, V>(base + element * 2, v);
}

// ------------------------------------------------------------------ the mask
constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

struct Mask {
    const uint64_t *seed;
    uint32_t threshold;          // T; 0: no dropout
    int32_t words;               // ceil(dim / 4)
};

// v with the dropped ones of the elements j0 .. j0 + V of position i at zero (j0 a multiple of V)
template <int V>
__device__ __forceinline__ Floats<V> masked(Floats<V> v, uint64_t seed, const Mask &m, int64_t i, int32_t j0)
{
    const uint64_t word = (uint64_t)i * (uint64_t)m.words + (uint32_t)(j0 >> 2);
#pragma unroll
    for (int w = 0; w < (V + 3) / 4; ++w) {
        uint64_t draws = mix64(seed + (word + w) * kGolden);
        if constexpr (V < 4) draws >>= 16 * (j0 & 3);
#pragma unroll
        for (int e = 0; e < (V < 4 ? V : 4); ++e)
            if ((uint32_t)(draws >> (16 * e) & 0xFFFF) < m.threshold) v[4 * w + e] = 0.f;
    }
    return v;
}

// ------------------------------------------------------------------ lookup
// x = q * d + r without a division: the quotient by floor((2^32 - 1) / d) is the exact one or one less
struct Div32 {
    uint32_t d, inverse;
};
__host__ __device__ inline Div32 div32(uint32_t d) { return Div32{d, ~0u / d}; }
__device__ __forceinline__ uint32_t divided(const Div32 &by, uint32_t x, uint32_t *rest)
{
    uint32_t q = __umulhi(x, by.inverse), r = x - q * by.d;
    if (r >= by.d) {
        r -= by.d;
        ++q;
    }
    *rest = r;
    return q;
}

// One lane per piece of V elements; a workgroup takes kEmbedPieces * kBlock neighbouring pieces of the output in a turn.
constexpr int kEmbedPieces = 4;
struct EmbedArgs {
    const int64_t *slots;
    int64_t n;
    const char *rows;
    RowMod mod;
    int64_t row_stride;
    char *out;
    int64_t out_stride;
    Div32 pieces;                // of a row
    float factor;
    Mask mask;
};

template <typename TI, typename TO, int V, bool DROP>
__global__ __launch_bounds__(kBlock) void k_embed(EmbedArgs a)
{
    const int64_t total = a.n * a.pieces.d;
    const uint32_t turn = gridDim.x * (uint32_t)(kBlock * kEmbedPieces);
    uint32_t c0, dc;
    int64_t k0 = divided(a.pieces, blockIdx.x * (uint32_t)(kBlock * kEmbedPieces), &c0);
    const uint32_t dk = divided(a.pieces, turn, &dc);
    const uint64_t seed = DROP ? *a.mask.seed : 0;
    for (int64_t i = (int64_t)blockIdx.x * kBlock * kEmbedPieces + threadIdx.x; i - threadIdx.x < total; i += turn) {
        int64_t k[kEmbedPieces], slot[kEmbedPieces];
        uint32_t c[kEmbedPieces];
        Floats<V> v[kEmbedPieces];
#pragma unroll
        for (int u = 0; u < kEmbedPieces; ++u) {
            k[u] = k0 + divided(a.pieces, c0 + u * kBlock + threadIdx.x, &c[u]);
            slot[u] = i + u * kBlock < total ? a.slots[k[u]] : -1;
        }
#pragma unroll
        for (int u = 0; u < kEmbedPieces; ++u) {
            v[u] = Floats<V>(0.f);
            if (slot[u] >= 0)
                v[u] = load_floats<TI, V>(a.rows + row_of(a.mod, slot[u]) * a.row_stride + (int64_t)c[u] * (V * sizeof(TI)));
        }
#pragma unroll
        for (int u = 0; u < kEmbedPieces; ++u) {
            if (i + u * kBlock >= total) continue;
            Floats<V> x = v[u] * a.factor;
            if constexpr (DROP) x = masked<V>(x, seed, a.mask, k[u], (int32_t)(c[u] * V));
            if (slot[u] < 0) x = Floats<V>(0.f);
            store_floats<TO, V>(a.out + k[u] * a.out_stride + (int64_t)c[u] * (V * sizeof(TO)), x);
        }
        k0 += dk;
        c0 += dc;
        if (c0 >= a.pieces.d) {
            c0 -= a.pieces.d;
            ++k0;
        }
    }
}

// ------------------------------------------------------------------ sort
// Entries {row << 32 | position} in ascending order: a radix sort by digits of 8 bits, least significant first, each pass
// stable, so that the positions of a row stay ascending.  Padding has the row num_rows and ends up behind everything.
constexpr int kDigits = 256, kDigitBits = 8;
constexpr int kSortItems = 16;
constexpr int kSortTile = kBlock * kSortItems;         // entries of a workgroup, 1 024 neighbouring ones for each wavefront

struct SortSource {
    const int64_t *slots;        // first pass: entries are made from them
    const uint64_t *entries;     // later ones
    RowMod mod;
    int64_t n;
    int32_t shift;               // of the digit inside an entry
};
template <bool FIRST>
__device__ __forceinline__ uint64_t sort_entry(const SortSource &s, int64_t i)
{
    if constexpr (FIRST) {
        const int64_t slot = s.slots[i];
        const uint64_t row = slot < 0 ? (uint64_t)s.mod.num_rows : (uint64_t)row_of(s.mod, slot);
        return row << 32 | (uint64_t)i;
    } else {
        return s.entries[i];
    }
}

// hist[digit * tiles + tile]: how many entries of the tile have the digit
template <bool FIRST>
__global__ __launch_bounds__(kBlock) void k_sort_hist(SortSource s, uint32_t *hist)
{
    __shared__ uint32_t count[kDigits];
    count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortTile;
#pragma unroll
    for (int u = 0; u < kSortItems; ++u) {
        const int64_t i = first + u * kBlock + threadIdx.x;
        if (i < s.n) atomicAdd(&count[(uint32_t)(sort_entry<FIRST>(s, i) >> s.shift) & (kDigits - 1)], 1u);
    }
    __syncthreads();
    hist[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = count[threadIdx.x];
}

// exclusive prefix over the lanes of a workgroup, and the sum; `sums` holds one word per wavefront
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t *sums, uint32_t *total)
{
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const uint32_t y = __shfl_up(x, d);
        if (lane_id() >= d) x += y;
    }
    if (lane_id() == kWave - 1) sums[threadIdx.x / kWave] = x;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int w = 0; w < (int)blockDim.x / kWave; ++w) {
        if (w < (int)threadIdx.x / kWave) before += sums[w];
        all += sums[w];
    }
    __syncthreads();
    *total = all;
    return before + x - v;
}

// in place: how many entries of earlier tiles have the digit; totals[digit]: of all tiles.  One workgroup per digit.
__global__ __launch_bounds__(kBlock) void k_sort_scan(uint32_t *hist, uint32_t *totals, int32_t tiles)
{
    __shared__ uint32_t sums[kWavesPerBlock];
    uint32_t *row = hist + (int64_t)blockIdx.x * tiles;
    uint32_t carry = 0;
    for (int32_t t0 = 0; t0 < tiles; t0 += kBlock) {
        const int32_t t = t0 + (int32_t)threadIdx.x;
        const uint32_t v = t < tiles ? row[t] : 0;
        uint32_t total;
        const uint32_t before = block_prefix(v, sums, &total);
        if (t < tiles) row[t] = carry + before;
        carry += total;
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

// Every wavefront ranks its entries 64 at a time: the lanes with the same digit find each other by ballots over the digit's
// bits, the first of them adds their number to the wavefront's count in LDS.  The entries then go to LDS in their new order,
// so that neighbouring lanes store neighbouring entries.
template <bool FIRST>
__global__ __launch_bounds__(kBlock) void k_sort_scatter(SortSource s, const uint32_t *hist, const uint32_t *totals, uint64_t *out)
{
    __shared__ uint32_t count[kWavesPerBlock][kDigits];
    __shared__ uint32_t local[kDigits], global[kDigits], sums[kWavesPerBlock];
    __shared__ uint64_t sorted[kSortTile];
    const int wave = threadIdx.x / kWave, lane = lane_id();
#pragma unroll
    for (int w = 0; w < kWavesPerBlock; ++w) count[w][threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortTile;
    const int64_t left = s.n - first;
    const int mine = (int)(left < kSortTile ? left : kSortTile);
    uint64_t entry[kSortItems];
    uint32_t rank[kSortItems];
#pragma unroll
    for (int u = 0; u < kSortItems; ++u) {
        const int at = wave * (kWave * kSortItems) + u * kWave + lane;
        entry[u] = at < mine ? sort_entry<FIRST>(s, first + at) : 0;
    }
#pragma unroll
    for (int u = 0; u < kSortItems; ++u) {
        const bool there = wave * (kWave * kSortItems) + u * kWave + lane < mine;
        const uint32_t digit = (uint32_t)(entry[u] >> s.shift) & (kDigits - 1);
        uint64_t same = __ballot(there);
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {
            const uint64_t set = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
        uint32_t before = 0;
        const int leader = there ? __ffsll((unsigned long long)same) - 1 : lane;
        if (there && lane == leader) before = atomicAdd(&count[wave][digit], (uint32_t)__popcll(same));
        before = __shfl(before, leader);
        rank[u] = before + (uint32_t)__popcll(same & ((1ull << lane) - 1));
    }
    __syncthreads();
    {
        const uint32_t d = threadIdx.x;
        uint32_t sum = 0, of_digit;
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w) {
            const uint32_t c = count[w][d];
            count[w][d] = sum;
            sum += c;
        }
        local[d] = block_prefix(sum, sums, &of_digit);
        global[d] = block_prefix(totals[d], sums, &of_digit) + hist[(int64_t)d * gridDim.x + blockIdx.x];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortItems; ++u) {
        if (wave * (kWave * kSortItems) + u * kWave + lane >= mine) continue;
        const uint32_t digit = (uint32_t)(entry[u] >> s.shift) & (kDigits - 1);
        sorted[local[digit] + count[wave][digit] + rank[u]] = entry[u];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortItems; ++u) {
        const int at = u * kBlock + threadIdx.x;
        if (at >= mine) continue;
        const uint64_t e = sorted[at];
        const uint32_t digit = (uint32_t)(e >> s.shift) & (kDigits - 1);
        out[(int64_t)global[digit] + (at - (int)local[digit])] = e;
    }
}

// ------------------------------------------------------------------ sums over the sorted entries
// A run is the entries of one row.  A workgroup has a tile of neighbouring entries, a group of lanes in it (a power of two of
// them, V * NP elements of the row for each) a part of the tile.  What a group knows of a run:
//   it begins and ends in the part   the group emits its sum
//   it began before                  the part's share goes to LDS, and whether the run goes on behind the part
//   it goes on behind                the group in whose part it begins adds the following groups' shares, in their order
// and the same again for the tiles, whose shares go to memory and are added by k_join.  All sums are in 32 bits, in an order
// that n, dim and the types alone determine.
constexpr int kReduceTile = 2048;
constexpr uint32_t kNoRow = ~0u;
constexpr uint32_t kHeadShare = 1, kThrough = 2, kTailShare = 4;      // flags of a part or a tile

struct ReduceArgs {
    const uint64_t *entries;
    int64_t n;
    uint32_t num_rows;
    int32_t tile;                // entries of a workgroup, a multiple of its groups
    int32_t lanes;               // of a group
    int32_t col_blocks;          // workgroups that share out the columns of a tile
    const char *grad;
    int64_t grad_stride;
    int32_t dim;
    float factor;
    Mask mask;
    // shares of the tiles
    uint32_t *flags;
    uint32_t *tail_index;        // of the run that leaves the tile
    float *head, *tail;          // tiles x dim
    const uint32_t *heads;       // runs that begin in a tile, or (scanned) in all tiles before
    int32_t scanned;
    // gradient
    int64_t *out_slots, *out_count;
    char *out_rows;
    int64_t cap;
    // step
    char *rows;
    int64_t row_stride;          // elements
    float *state;
    const float *lr;
    float eps;
    int32_t type;                // of out_rows or rows
};

// runs that begin in each tile
__global__ __launch_bounds__(kBlock) void k_count_heads(const uint64_t *entries, int64_t n, uint32_t num_rows, int32_t tile,
                                                         uint32_t *heads)
{
    __shared__ uint32_t sums[kWavesPerBlock];
    const int64_t first = (int64_t)blockIdx.x * tile;
    uint32_t mine = 0;
    for (int k = threadIdx.x; k < tile; k += kBlock) {
        const int64_t i = first + k;
        if (i >= n) break;
        const uint32_t row = (uint32_t)(entries[i] >> 32);
        mine += row != num_rows && (i == 0 || (uint32_t)(entries[i - 1] >> 32) != row);
    }
    uint32_t total;
    block_prefix(mine, sums, &total);
    if (threadIdx.x == 0) heads[blockIdx.x] = total;
}
// heads of tiles -> heads of all tiles before, in place; one workgroup
__global__ __launch_bounds__(kBlock) void k_scan_heads(uint32_t *heads, int32_t tiles)
{
    __shared__ uint32_t sums[kWavesPerBlock];
    uint32_t carry = 0;
    for (int32_t t0 = 0; t0 < tiles; t0 += kBlock) {
        const int32_t t = t0 + (int32_t)threadIdx.x;
        const uint32_t v = t < tiles ? heads[t] : 0;
        uint32_t total;
        const uint32_t before = block_prefix(v, sums, &total);
        if (t < tiles) heads[t] = carry + before;
        carry += total;
    }
}

template <typename TG, int V, int NP, bool STEP>
__global__ __launch_bounds__(kBlock) void k_reduce(ReduceArgs a)
{
    __shared__ uint32_t row_of_entry[kReduceTile + 2], position[kReduceTile];
    __shared__ uint32_t sums[kWavesPerBlock], part_heads[kBlock], part_flags[kBlock];
    __shared__ Floats<V> shares[NP][kBlock];

    const int32_t tile_index = (int32_t)(blockIdx.x / (uint32_t)a.col_blocks), block_col = (int32_t)(blockIdx.x % (uint32_t)a.col_blocks);
    const int64_t first = (int64_t)tile_index * a.tile;
    const int64_t left = a.n - first;
    const int m = (int)(left < a.tile ? left : a.tile);
    const int groups = kBlock / a.lanes, per = a.tile / groups;
    const int group = threadIdx.x / a.lanes, lane = threadIdx.x % a.lanes;

    // the tile's entries, and the rows before and behind it
    for (int k = threadIdx.x; k < m; k += kBlock) {
        const uint64_t e = a.entries[first + k];
        row_of_entry[k + 1] = (uint32_t)(e >> 32);
        position[k] = (uint32_t)e;
    }
    if (threadIdx.x == 0) {
        row_of_entry[0] = first > 0 ? (uint32_t)(a.entries[first - 1] >> 32) : kNoRow;
        row_of_entry[m + 1] = first + m < a.n ? (uint32_t)(a.entries[first + m] >> 32) : kNoRow;
    }
    // runs before the tile
    uint32_t index = 0;
    if constexpr (!STEP) {
        if (a.scanned) index = a.heads[tile_index];
        else {
            uint32_t mine = 0;
            for (int t = threadIdx.x; t < tile_index; t += kBlock) mine += a.heads[t];
            block_prefix(mine, sums, &index);
        }
    }
    part_heads[threadIdx.x] = 0;
    __syncthreads();
    const int begin = group * per < m ? group * per : m, end = begin + per < m ? begin + per : m;
    if constexpr (!STEP) {
        uint32_t mine = 0;
        for (int k = begin + lane; k < end; k += a.lanes)
            mine += row_of_entry[k + 1] != a.num_rows && row_of_entry[k + 1] != row_of_entry[k];
        for (int d = 1; d < a.lanes; d <<= 1) mine += __shfl_xor(mine, d);
        if (lane == 0) part_heads[group] = mine;
        __syncthreads();
        uint32_t all;
        const uint32_t before = block_prefix(part_heads[threadIdx.x], sums, &all);
        part_heads[threadIdx.x] = before;
        __syncthreads();
        if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *a.out_count = (int64_t)index + all;
        index += part_heads[group];
    }

    int32_t column[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) column[p] = ((block_col * NP + p) * a.lanes + lane) * V;
    const uint64_t seed = a.mask.threshold ? *a.mask.seed : 0;
    Floats<V> sum[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) sum[p] = Floats<V>(0.f);

    // a finished sum
    auto emit = [&](uint32_t row, uint32_t at) {
        if constexpr (STEP) {
            const float lr = *a.lr;
            float rate = lr;
            if (a.state) {
                float squares = 0.f;
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float g = sum[p][e] * a.factor;
                        if (column[p] < a.dim) squares += g * g;
                    }
                for (int d = 1; d < a.lanes; d <<= 1) squares += __shfl_xor(squares, d);
                const float state = a.state[row] + squares / (float)a.dim;
                if (lane == 0) a.state[row] = state;
                rate = lr / (sqrtf(state) + a.eps);
            }
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                if (column[p] >= a.dim) continue;
                const int64_t element = (int64_t)row * a.row_stride + column[p];
                const Floats<V> w = load_typed<V>(a.type, a.rows, element);
                store_typed<V>(a.type, a.rows, element, w - sum[p] * a.factor * rate);
            }
        } else {
            if ((int64_t)at >= a.cap) return;
            if (block_col == 0 && lane == 0) a.out_slots[at] = row;
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (column[p] < a.dim) store_typed<V>(a.type, a.out_rows, (int64_t)at * a.dim + column[p], sum[p] * a.factor);
        }
    };

    constexpr int kAhead = NP * V >= 16 ? 2 : 4;
    uint32_t flags = 0;
    bool from_before = begin < end && row_of_entry[begin] == row_of_entry[begin + 1];
    for (int k0 = begin; k0 < end; k0 += kAhead) {
        Floats<V> g[kAhead][NP];
        uint32_t at[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int k = k0 + u < end ? k0 + u : end - 1;
            at[u] = position[k];
            const bool wanted = k0 + u < end && row_of_entry[k + 1] != a.num_rows;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                g[u][p] = Floats<V>(0.f);
                if (wanted && column[p] < a.dim)
                    g[u][p] = load_floats<TG, V>(a.grad + (int64_t)at[u] * a.grad_stride + (int64_t)column[p] * sizeof(TG));
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int k = k0 + u;
            if (k >= end) break;
            const uint32_t row = row_of_entry[k + 1];
            if (row == a.num_rows) { from_before = false; continue; }
            if (row_of_entry[k] != row) ++index;
#pragma unroll
            for (int p = 0; p < NP; ++p)
                sum[p] += a.mask.threshold ? masked<V>(g[u][p], seed, a.mask, at[u], column[p]) : g[u][p];
            if (row_of_entry[k + 2] == row && k + 1 < end) continue;
            const bool goes_on = row_of_entry[k + 2] == row;
            if (from_before) {
                flags |= kHeadShare | (goes_on ? kThrough : 0);
#pragma unroll
                for (int p = 0; p < NP; ++p) shares[p][threadIdx.x] = sum[p];
            } else if (goes_on) {
                flags |= kTailShare;
            } else {
                emit(row, index - 1);
            }
            from_before = false;
            if (!goes_on) {
#pragma unroll
                for (int p = 0; p < NP; ++p) sum[p] = Floats<V>(0.f);
            }
        }
    }
    if (lane == 0) part_flags[group] = flags;
    __syncthreads();

    // shares of the parts from g on, as far as the run goes; whether it leaves the tile
    auto add_following = [&](int g) {
        for (; g < groups; ++g) {
            const uint32_t f = part_flags[g];
#pragma unroll
            for (int p = 0; p < NP; ++p) sum[p] += shares[p][g * a.lanes + lane];
            if (!(f & kThrough)) return false;
        }
        return true;
    };
    auto keep = [&](float *to) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            if (column[p] >= a.dim) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) to[(int64_t)tile_index * a.dim + column[p] + e] = sum[p][e];
        }
    };
    if (flags & kTailShare) {
        if (!add_following(group + 1)) {
            emit(row_of_entry[end], index - 1);
        } else {
            keep(a.tail);
            if (lane == 0 && block_col == 0) a.tail_index[tile_index] = index - 1;
        }
    }
    if (group == 0) {
        const bool head = part_flags[0] & kHeadShare;
        bool through = false;
        if (head) {
#pragma unroll
            for (int p = 0; p < NP; ++p) sum[p] = Floats<V>(0.f);
            through = add_following(0);
            keep(a.head);
        }
        if (block_col == 0 && lane == 0) {
            const bool leaves = row_of_entry[m] == row_of_entry[m + 1] && row_of_entry[m] != a.num_rows;
            a.flags[tile_index] = (head ? kHeadShare : 0) | (through ? kThrough : 0) | (leaves && !through ? kTailShare : 0);
        }
    }
}

// The runs that leave the tile in which they begin: a workgroup each, whose lanes share out the columns (a power of two of
// them, `lanes`) and, where there are fewer columns than lanes, the tiles.
constexpr int kJoinColumns = 4;              // of a lane: a step has the whole row in one workgroup
template <bool STEP>
__global__ __launch_bounds__(kBlock) void k_join(ReduceArgs a, int32_t tiles)
{
    __shared__ int32_t last_tile;
    __shared__ float part[kBlock];
    const int32_t tile_index = (int32_t)(blockIdx.x / (uint32_t)a.col_blocks), block_col = (int32_t)(blockIdx.x % (uint32_t)a.col_blocks);
    if (!(a.flags[tile_index] & kTailShare)) return;
    // the tile in which the run ends: the first one behind this that it does not go through
    if (threadIdx.x == 0) last_tile = tiles - 1;
    __syncthreads();
    for (int32_t t0 = tile_index + 1; t0 < tiles; t0 += kBlock) {
        const int32_t t = t0 + (int32_t)threadIdx.x;
        if (t < tiles && !(a.flags[t] & kThrough)) atomicMin(&last_tile, t);
        __syncthreads();
        const bool found = last_tile < t0 + kBlock;
        __syncthreads();
        if (found) break;
    }
    const int32_t last = last_tile;
    const uint32_t row = (uint32_t)(a.entries[(int64_t)(tile_index + 1) * a.tile] >> 32);
    const int sharers = kBlock / a.lanes, sharer = threadIdx.x / a.lanes, lane = threadIdx.x % a.lanes;
    float sum[kJoinColumns];
    float squares = 0.f;
#pragma unroll
    for (int p = 0; p < kJoinColumns; ++p) {
        const int32_t c = (block_col * kJoinColumns + p) * a.lanes + lane;
        sum[p] = 0.f;
        if (c < a.dim) {
            if (sharer == 0) sum[p] = a.tail[(int64_t)tile_index * a.dim + c];
#pragma unroll 4
            for (int32_t t = tile_index + 1 + sharer; t <= last; t += sharers) sum[p] += a.head[(int64_t)t * a.dim + c];
        }
        if (sharers > 1) {
            part[threadIdx.x] = sum[p];
            __syncthreads();
            if (sharer == 0)
                for (int g = 1; g < sharers; ++g) sum[p] += part[g * a.lanes + lane];
            __syncthreads();
        }
        sum[p] *= a.factor;
        if (c < a.dim && sharer == 0) squares += sum[p] * sum[p];
    }
    if constexpr (STEP) {
        const float lr = *a.lr;
        float rate = lr;
        if (a.state) {
            part[threadIdx.x] = squares;
            __syncthreads();
            for (int d = kBlock / 2; d > 0; d >>= 1) {
                if ((int)threadIdx.x < d) part[threadIdx.x] += part[threadIdx.x + d];
                __syncthreads();
            }
            const float state = a.state[row] + part[0] / (float)a.dim;
            __syncthreads();                  // (all have read it)
            if (threadIdx.x == 0) a.state[row] = state;
            rate = lr / (sqrtf(state) + a.eps);
        }
        if (sharer != 0) return;
#pragma unroll
        for (int p = 0; p < kJoinColumns; ++p) {
            const int32_t c = p * a.lanes + lane;
            if (c >= a.dim) continue;
            const int64_t element = (int64_t)row * a.row_stride + c;
            store_typed<1>(a.type, a.rows, element, load_typed<1>(a.type, a.rows, element) - sum[p] * rate);
        }
    } else {
        const int64_t at = a.tail_index[tile_index];
        if (sharer != 0 || at >= a.cap) return;
        if (block_col == 0 && lane == 0) a.out_slots[at] = row;
#pragma unroll
        for (int p = 0; p < kJoinColumns; ++p) {
            const int32_t c = (block_col * kJoinColumns + p) * a.lanes + lane;
            if (c < a.dim) store_typed<1>(a.type, a.out_rows, at * a.dim + c, Floats<1>(sum[p]));
        }
    }
}

}  // namespace mpzch
