// Sort of a batch's slots by row.
#pragma once
#include "mpzch_embed_kernels.hpp"

namespace mpzch {

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / kWave;

// Entries {row << 32 | position} in ascending order.  Padding has the row num_rows and ends up behind everything.
struct SortSource {
    const int64_t *slots;        // first pass: entries are made from them
    const uint64_t *entries;     // later ones
    RowMod mod;
    int64_t n;
    int32_t shift, bits;         // of the digit inside an entry
};
__device__ __forceinline__ uint32_t sort_row(const RowMod &mod, int64_t slot)
{
    return slot < 0 ? (uint32_t)mod.num_rows : (uint32_t)row_of(mod, slot);
}
template <bool FIRST>
__device__ __forceinline__ uint64_t sort_entry(const SortSource &s, int64_t i)
{
    if constexpr (FIRST) return (uint64_t)sort_row(s.mod, s.slots[i]) << 32 | (uint64_t)i;
    else return s.entries[i];
}

// Short batches: an entry's place is the number of entries before it.  A workgroup counts for 16 entries, an entry in four lanes of each
// of its 16 wavefronts, which have a 64th of the batch each.  n^2 comparisons, but one launch, and all compute units share them:
// with the sums, gradients of 1 024 positions 10.8 us, 4 000 18, 8 000 28, where passes over digits take 29; 10 000 38 and 30.
constexpr int kRankMax = 8192;
constexpr int kRanked = 16, kRankParts = kSortBlock / kRanked;
__global__ __launch_bounds__(kSortBlock) void k_sort_rank(const int64_t *slots, RowMod mod, int32_t n, uint64_t *out)
{
    __shared__ __align__(16) uint32_t rows[kRankMax];
    __shared__ uint32_t place[kRanked];
    const int32_t whole = (n + 3) / 4 * 4;
    for (int32_t i = threadIdx.x; i < whole; i += kSortBlock) rows[i] = i < n ? sort_row(mod, slots[i]) : ~0u;
    if (threadIdx.x < kRanked) place[threadIdx.x] = 0;
    __syncthreads();
    const int32_t block = (int32_t)blockIdx.x * kRanked, mine = block + (int32_t)threadIdx.x % kRanked;
    const uint32_t row = rows[mine < n ? mine : n - 1];
    const int32_t part = threadIdx.x / kRanked, share = (whole / 4 + kRankParts - 1) / kRankParts * 4;
    const int32_t begin = part * share < whole ? part * share : whole, end = begin + share < whole ? begin + share : whole;
    uint32_t before = 0;
    auto upto = [&](int32_t at) { return at < begin ? begin : at > end ? end : at; };
    // entries before the 16 of this workgroup, among them, behind them (all borders are multiples of four)
    const int32_t first = upto(block), last = upto(block + kRanked);
#pragma unroll 4
    for (int32_t j = begin; j < first; j += 4) {
        const u32x4 r = *reinterpret_cast<const u32x4 *>(rows + j);
        before += (r[0] <= row) + (r[1] <= row) + (r[2] <= row) + (r[3] <= row);
    }
#pragma unroll 4
    for (int32_t j = first; j < last; j += 4) {
        const u32x4 r = *reinterpret_cast<const u32x4 *>(rows + j);
#pragma unroll
        for (int k = 0; k < 4; ++k) before += r[k] < row || (r[k] == row && j + k < mine);
    }
#pragma unroll 4
    for (int32_t j = last; j < end; j += 4) {
        const u32x4 r = *reinterpret_cast<const u32x4 *>(rows + j);
        before += (r[0] < row) + (r[1] < row) + (r[2] < row) + (r[3] < row);
    }
    atomicAdd(&place[threadIdx.x % kRanked], before);
    __syncthreads();
    if (threadIdx.x < kRanked && mine < n) out[place[threadIdx.x]] = (uint64_t)row << 32 | (uint32_t)mine;
}

// Longer ones: a radix sort, least significant digit first, each pass stable, so that the positions of a row stay ascending.
// A pass counts the digits of every tile (k_sort_hist), adds up what earlier tiles hold (k_sort_scan; where there are few
// tiles, k_sort_scatter itself) and moves the entries (k_sort_scatter).  The last of these could count the next pass's digits as
// it goes, with atomics on the counts of the tiles that it moves entries to, and save a launch: a step of 65 536 positions
// 40 -> 57 us, of 1 M 174 -> 383.
// Digits of up to kWideBits bits where passes are few launches after all, of kNarrowBits where there are many entries to move: the
// more digits, the shorter the stretches that a tile stores side by side.
constexpr int kWideBits = 11, kNarrowBits = 9, kLeastBits = 6;
constexpr int kScanDigits = 16;

// hist[tile][digit]: how many entries of the tile have the digit, 16 bits each
template <bool FIRST, int ITEMS, int BITS>
__global__ __launch_bounds__(kSortBlock) void k_sort_hist(SortSource s, uint32_t *hist)
{
    __shared__ uint32_t count[1 << BITS];
    const uint32_t digits = 1u << s.bits;
    for (uint32_t d = threadIdx.x; d < digits; d += kSortBlock) count[d] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * (kSortBlock * ITEMS);
    uint64_t entry[ITEMS];
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        const int64_t i = first + u * kSortBlock + threadIdx.x;
        entry[u] = i < s.n ? sort_entry<FIRST>(s, i) : 0;
    }
    // (entries of a frequent row lie side by side behind the first pass: a wavefront with one digit adds it once)
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        const uint32_t digit = (uint32_t)(entry[u] >> s.shift) & (digits - 1);
        const bool there = first + u * kSortBlock + threadIdx.x < s.n;
        const uint64_t same = __ballot(there && digit == (uint32_t)__builtin_amdgcn_readfirstlane((int)digit));
        if (same == __ballot(there)) {
            if (there && lane_id() == 0) atomicAdd(&count[digit], (uint32_t)__popcll(same));
        } else if (there) {
            atomicAdd(&count[digit], 1u);
        }
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits / 2; d += kSortBlock)
        hist[(int64_t)blockIdx.x * (digits / 2) + d] = count[2 * d] | count[2 * d + 1] << 16;
}

// before[tile][digit]: entries of earlier tiles with the digit; behind the last tile the entries of all.  A workgroup has 16 digits,
// each lane two of them and a 128th of the tiles; lanes with the same digits are 8 apart.
__global__ __launch_bounds__(kSortBlock) void k_sort_scan(const uint32_t *hist, uint32_t *before, int32_t tiles, int32_t bits)
{
    constexpr int kPairs = kScanDigits / 2, kParts = kSortBlock / kPairs;
    __shared__ uint32_t sums[2][kSortWaves][kPairs];
    const int32_t pairs = 1 << (bits - 1);
    const int32_t mine = threadIdx.x % kPairs, pair = (int32_t)blockIdx.x * kPairs + mine, part = threadIdx.x / kPairs;
    const int32_t per = (tiles + kParts - 1) / kParts, begin = part * per < tiles ? part * per : tiles, end = begin + per < tiles ? begin + per : tiles;
    uint32_t a = 0, b = 0;
#pragma unroll 8
    for (int32_t t = begin; t < end; ++t) {
        const uint32_t v = hist[(int64_t)t * pairs + pair];
        a += v & 0xFFFF;
        b += v >> 16;
    }
    uint32_t low = a, high = b;
#pragma unroll
    for (int d = kPairs; d < kWave; d <<= 1) {
        const uint32_t x = __shfl_up(low, d), y = __shfl_up(high, d);
        if (lane_id() >= d) {
            low += x;
            high += y;
        }
    }
    const int wave = threadIdx.x / kWave;
    if (lane_id() >= kWave - kPairs) {
        sums[0][wave][mine] = low;
        sums[1][wave][mine] = high;
    }
    __syncthreads();
    low -= a;
    high -= b;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w)
        if (w < wave) {
            low += sums[0][w][mine];
            high += sums[1][w][mine];
        }
    for (int32_t t = begin; t < end; ++t) {
        uint32_t *to = before + ((int64_t)t * pairs + pair) * 2;
        to[0] = low;
        to[1] = high;
        const uint32_t v = hist[(int64_t)t * pairs + pair];
        low += v & 0xFFFF;
        high += v >> 16;
    }
    if (part == kParts - 1) {                    // (its part ends with the last tile, if it is not empty behind it)
        uint32_t *to = before + ((int64_t)tiles * pairs + pair) * 2;
        to[0] = low;
        to[1] = high;
    }
}

// Every wavefront ranks its entries 64 at a time: the lanes with the same digit find each other by ballots over the digit's
// bits, the first of them adds their number to the wavefront's count in LDS (its own, so the order of its accesses is that of
// the program).  The entries then go to LDS in their new order, so that neighbouring lanes store neighbouring entries.
template <bool FIRST, int ITEMS, int BITS>
__global__ __launch_bounds__(kSortBlock) void k_sort_scatter(SortSource s, const uint32_t *hist, const uint32_t *before, int32_t tiles,
                                                              uint64_t *out)
{
    constexpr int kTile = kSortBlock * ITEMS;
    // the counts of the wavefronts, 16 bits each, and then the entries
    constexpr int kCountBytes = kSortWaves * (2 << BITS), kEntryBytes = kTile * 8;
    __shared__ __align__(16) unsigned char area[kCountBytes > kEntryBytes ? kCountBytes : kEntryBytes];
    __shared__ uint32_t earlier[1 << BITS], all[1 << BITS], sums[2][kSortWaves];
    uint32_t *const global = earlier, *const local = all;
    uint16_t *const count = reinterpret_cast<uint16_t *>(area);
    uint64_t *const sorted = reinterpret_cast<uint64_t *>(area);
    const uint32_t digits = 1u << s.bits, pairs = digits / 2;
    const int wave = threadIdx.x / kWave, lane = lane_id();
    for (uint32_t k = threadIdx.x; k < kSortWaves * pairs / 4; k += kSortBlock) reinterpret_cast<u32x4 *>(area)[k] = u32x4(0);
    if (!before)
        for (uint32_t d = threadIdx.x; d < digits; d += kSortBlock) earlier[d] = all[d] = 0;
    const int64_t first = (int64_t)blockIdx.x * kTile;
    const int64_t left = s.n - first;
    const int mine = (int)(left < kTile ? left : kTile);
    uint64_t entry[ITEMS];
    uint32_t place[ITEMS];
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        const int at = wave * (kWave * ITEMS) + u * kWave + lane;
        entry[u] = at < mine ? sort_entry<FIRST>(s, first + at) : 0;
    }
    // what earlier tiles hold of two digits, and all tiles; where the tiles are added up here, by all lanes, a part of the tiles each
    if (before) {
        if (threadIdx.x < pairs) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                earlier[2 * threadIdx.x + k] = before[((int64_t)blockIdx.x * pairs + threadIdx.x) * 2 + k];
                all[2 * threadIdx.x + k] = before[((int64_t)tiles * pairs + threadIdx.x) * 2 + k];
            }
        }
    } else {
        const int parts = kSortBlock / pairs, pair = threadIdx.x % pairs;
        uint32_t e[2] = {0, 0}, x[2] = {0, 0};
        for (int32_t t0 = threadIdx.x / pairs; t0 < tiles; t0 += 8 * parts) {
            uint32_t v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int32_t t = t0 + u * parts;
                v[u] = hist[(int64_t)(t < tiles ? t : t0) * pairs + pair];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int32_t t = t0 + u * parts;
                const uint32_t counted = t < tiles ? v[u] : 0, early = t < (int32_t)blockIdx.x ? v[u] : 0;
                e[0] += early & 0xFFFF;
                e[1] += early >> 16;
                x[0] += counted & 0xFFFF;
                x[1] += counted >> 16;
            }
        }
        __syncthreads();                         // (the sums are empty)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            atomicAdd(&earlier[2 * pair + k], e[k]);
            atomicAdd(&all[2 * pair + k], x[k]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        const bool there = wave * (kWave * ITEMS) + u * kWave + lane < mine;
        const uint32_t digit = (uint32_t)(entry[u] >> s.shift) & (digits - 1);
        const uint64_t all_there = __ballot(there);
        uint32_t low = (uint32_t)all_there, high = (uint32_t)(all_there >> 32);
        for (int b = 0; b < s.bits; ++b) {
            const int32_t bit = (int32_t)(digit << (31 - b)) >> 31;        // all ones or zeros
            const uint64_t set = __ballot(bit != 0);
            low &= ~((uint32_t)set ^ (uint32_t)bit);
            high &= ~((uint32_t)(set >> 32) ^ (uint32_t)bit);
        }
        const uint64_t same = (uint64_t)high << 32 | low;
        const uint32_t at = (uint32_t)wave * digits + digit;
        const uint32_t so_far = count[at];
        place[u] = so_far + (uint32_t)__popcll(same & ((1ull << lane) - 1));
        // (no instruction: the hardware does a wavefront's accesses in order, the compiler is kept from moving any across)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (there && (same >> lane) == 1) count[at] = (uint16_t)(place[u] + 1);       // the last of them
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    {
        // counts of earlier wavefronts, two digits in a word (no carry: a tile has less than 2^16 entries)
        uint32_t sum = 0;
        if (threadIdx.x < pairs) {
            uint32_t c[kSortWaves];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) c[w] = reinterpret_cast<uint32_t *>(area)[w * pairs + threadIdx.x];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                reinterpret_cast<uint32_t *>(area)[w * pairs + threadIdx.x] = sum;
                sum += c[w];
            }
        }
        // exclusive prefixes over the digits, of this tile's counts and of all tiles'
        uint32_t e[2] = {0, 0}, x[2] = {0, 0};
        if (threadIdx.x < pairs) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                e[k] = earlier[2 * threadIdx.x + k];
                x[k] = all[2 * threadIdx.x + k];
            }
        }
        const uint32_t own = (sum & 0xFFFF) + (sum >> 16), every = x[0] + x[1];
        uint32_t here = own, there = every;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const uint32_t y = __shfl_up(here, d), z = __shfl_up(there, d);
            if (lane >= d) {
                here += y;
                there += z;
            }
        }
        if (lane == kWave - 1) {
            sums[0][wave] = here;
            sums[1][wave] = there;
        }
        __syncthreads();
        here -= own;
        there -= every;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w)
            if (w < wave) {
                here += sums[0][w];
                there += sums[1][w];
            }
        if (threadIdx.x < pairs) {
            local[2 * threadIdx.x] = here;
            local[2 * threadIdx.x + 1] = here + (sum & 0xFFFF);
            global[2 * threadIdx.x] = there + e[0] - here;
            global[2 * threadIdx.x + 1] = there + x[0] + e[1] - here - (sum & 0xFFFF);
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        const uint32_t digit = (uint32_t)(entry[u] >> s.shift) & (digits - 1);
        place[u] += local[digit] + count[(uint32_t)wave * digits + digit];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < ITEMS; ++u)
        if (wave * (kWave * ITEMS) + u * kWave + lane < mine) sorted[place[u]] = entry[u];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        const int at = u * kSortBlock + threadIdx.x;
        if (at >= mine) continue;
        const uint64_t e = sorted[at];
        out[global[(uint32_t)(e >> s.shift) & (digits - 1)] + (uint32_t)at] = e;       // (the sum is below n; the parts may wrap)
    }
}

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
        const uint32_t row = row_at(entries, i);
        mine += row != num_rows && (i == 0 || row_at(entries, i - 1) != row);
    }
    uint32_t total;
    block_prefix(mine, sums, &total);
    if (threadIdx.x == 0) heads[blockIdx.x] = total;
}
// heads of tiles -> heads of all tiles before, in place; one workgroup
__global__ __launch_bounds__(kSortBlock) void k_scan_heads(uint32_t *heads, int32_t tiles)
{
    __shared__ uint32_t sums[kSortWaves];
    uint32_t carry = 0;
    for (int32_t t0 = 0; t0 < tiles; t0 += kSortBlock) {
        const int32_t t = t0 + (int32_t)threadIdx.x;
        const uint32_t v = t < tiles ? heads[t] : 0;
        uint32_t total;
        const uint32_t before = block_prefix(v, sums, &total);
        if (t < tiles) heads[t] = carry + before;
        carry += total;
    }
}

}  // namespace mpzch
