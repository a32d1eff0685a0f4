// Host side of the embedding operators of include/mpzch.h: argument checks, the scratch of the gradients, launches.
#include "../../include/mpzch.h"
#include "mpzch_reduce.hpp"
#include "mpzch_sort.hpp"
#include "mpzch_host.hpp"

#include <cmath>
#include <cstring>
#include <new>

using namespace mpzch;

struct mpzch_embed_s {
    char *base = nullptr;
    int device = -1;             // that the scratch is on
    int64_t cap_n = 0, cap_dim = 0;
};

namespace {

static_assert(kF32 == MPZCH_F32 && kBf16 == MPZCH_BF16 && kF16 == MPZCH_F16, "the element types of the header");

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int pow2_at_least(int64_t x)
{
    int p = 1;
    while (p < x) p *= 2;
    return p;
}
int64_t element_bytes(int32_t type) { return type == MPZCH_F32 ? 4 : 2; }
bool type_ok(int32_t type) { return type == MPZCH_F32 || type == MPZCH_BF16 || type == MPZCH_F16; }

// A 2-D tensor with dense rows, aligned to its elements.
struct Rows {
    const void *at;
    int32_t type;
    int64_t dim, stride;         // elements, bytes
    bool ok() const
    {
        const int64_t e = element_bytes(type);
        return at && type_ok(type) && stride >= dim * e && stride % e == 0 && (uintptr_t)at % e == 0;
    }
};

// elements of a piece: 16 bytes of the wider of two tensors, or what a short row has
int piece_width(int64_t dim, int32_t type, int32_t other)
{
    int width = type == MPZCH_F32 || other == MPZCH_F32 ? 4 : 8;
    while (width > dim) width /= 2;
    return width;
}

// Results of this many bytes are stored past the caches.  Together with a kernel behind that reads them and writes as much, us, through /
// past: lookups of 33 MB 23.7 / 23.2, 77 MB 44.2 / 43.8, 179 MB 110 / 118 (the memory-side cache would have held them for the
// reader), 512 MB 336 / 327; of 8 MB, through the caches, 12.0.
constexpr int64_t kPastCaches = (int64_t)1 << 24;
// Gradients of this many bytes are read past the caches, of which the rest of the program keeps more that way: half of the memory-side
// one, since what a backward pass has just written may still be there.  us, through / past: sums of 512 MB 290.5 / 280, a step from
// 256 MB 171.7 / 164.5; of 33 and 38 MB, which the cache did hold, 37.2 / 38.5 and 59.2 / 62.3.
constexpr int64_t kReadPastCaches = (int64_t)1 << 27;

// scale and dropout of a call
bool make_mask(float scale, double drop_p, const int64_t *seed, int64_t dim, float *factor, Mask *mask)
{
    if (!std::isfinite(scale) || !(drop_p >= 0.0 && drop_p <= 1.0)) return false;
    const uint32_t t = (uint32_t)std::floor(drop_p * 65536.0 + 0.5);
    if (t && !seed) return false;
    mask->seed = (const uint64_t *)seed;
    mask->threshold = t;
    mask->row_step = (uint64_t)((dim + 3) / 4) * kGolden;
    mask->ragged = dim % 4 != 0;
    *factor = t == 65536 ? 0.f : (float)((double)scale * 65536.0 / (65536.0 - t));
    return std::isfinite(*factor);               // (0 * infinity: NaN where kept terms sum to zero)
}

// ---- lookup ---------------------------------------------------------------------------------
template <typename TI, typename TO, int V>
mpzch_status_t launch_embed(const EmbedArgs &a, int grid, hipStream_t s)
{
    return a.mask.threshold ? launch(k_embed<TI, TO, V, true>, grid, kBlock, s, a) : launch(k_embed<TI, TO, V, false>, grid, kBlock, s, a);
}
template <typename TI, typename TO>
mpzch_status_t launch_embed(const EmbedArgs &a, int width, int grid, hipStream_t s)
{
    switch (width) {
    case 8:
        if constexpr (sizeof(TI) == 2 && sizeof(TO) == 2) return launch_embed<TI, TO, 8>(a, grid, s);
        return MPZCH_ERR_UNSUPPORTED;
    case 4: return launch_embed<TI, TO, 4>(a, grid, s);
    case 2: return launch_embed<TI, TO, 2>(a, grid, s);
    default: return launch_embed<TI, TO, 1>(a, grid, s);
    }
}
template <typename TI>
mpzch_status_t launch_embed(const EmbedArgs &a, int32_t out_type, int width, int grid, hipStream_t s)
{
    switch (out_type) {
    case MPZCH_F32: return launch_embed<TI, float>(a, width, grid, s);
    case MPZCH_BF16: return launch_embed<TI, __bf16>(a, width, grid, s);
    default: return launch_embed<TI, _Float16>(a, width, grid, s);
    }
}

// ---- gradient -------------------------------------------------------------------------------
// How the sums are shared out: kReduceWaves wavefronts or more, but no part of a tile shorter than kPartMin entries (or, where
// the groups are many, no tile shorter than kTileMin) and no tile longer than kReduceTile.  us by wavefronts (2 048, 4 096,
// 8 192): gradient of 300 007 positions 67 62 68, steps of 1 M 176 175 182, of 16 384 positions of 1 024 elements 37.3 36.9 36.7;
// by the shortest part (2, 4, 8): a step of 65 536 39.1 39.2 44.8, of 16 384 50 42 37 (with four entries under way there; with
// two 36.9); without kTileMin / with it: steps of 1 024 and 4 000 positions of 16 elements 11.1 / 10.5 and 16.7 / 15.9, of 20 000 of
// 64 34.0 / 31.6, a gradient of 20 011 of 50 33.2 / 31.1.
constexpr int64_t kReduceWaves = 4096;
constexpr int kPartMin = 4, kTileMin = 128;
constexpr int64_t kTilesAdded = 2048;        // up to which a workgroup itself adds up the heads of the tiles before its own

struct ReducePlan {
    int lanes, pieces, col_blocks, tile, tiles;      // pieces: of a lane, as compiled
};
ReducePlan reduce_plan(int64_t n, int64_t dim, int width)
{
    ReducePlan p;
    const int64_t pieces = ceil_div(dim, width);
    p.lanes = pieces < kWave ? pow2_at_least(pieces) : kWave;
    p.pieces = pieces <= kWave ? 1 : 16 / width;
    p.col_blocks = (int)ceil_div(pieces, (int64_t)p.lanes * p.pieces);
    const int groups = kReduceBlock / p.lanes;
    int64_t per = ceil_div(n * p.lanes * p.col_blocks, kWave * kReduceWaves);
    const int least = groups * kPartMin <= kTileMin ? kPartMin : groups < kTileMin ? kTileMin / groups : 1;
    if (per < least) per = least;
    if (per > kReduceTile / groups) per = kReduceTile / groups;
    p.tile = (int)per * groups;
    p.tiles = n > 0 ? (int)ceil_div(n, p.tile) : 1;
    return p;
}
// most tiles, and most columns' blocks, of any batch of up to n positions and rows of up to dim elements: the parts are as
// short as the number of wavefronts allows (kReduceWaves wavefronts in all), or the tiles as long as can be
int64_t most_tiles(int64_t n)
{
    const int64_t waves = kReduceBlock / kWave;
    const int64_t some = ceil_div(n, waves * kPartMin) < kReduceWaves / waves ? ceil_div(n, waves * kPartMin) : kReduceWaves / waves;
    const int64_t full = ceil_div(n, kReduceTile);
    return 1 + (some > full ? some : full);
}
int64_t most_col_blocks(int64_t dim) { return ceil_div(dim, kWave * 16); }

// How a batch is sorted beyond kRankMax.  Few tiles leave compute units idle, many take the workgroups long to add up; passes are
// launches.  us, whole calls, by entries of a lane (1, 2, 4): a step of 65 536 39.3 39.4 43.1, gradients of 20 011 31.1 33.1 37.3 and
// of 300 007 79 67 72, steps of 1 M - 190 184, gradients of 2 M - 330 307 (and 8: 309).
constexpr int64_t kWideMost = 65536;         // digits of kWideBits: two passes for a million rows (39.3 us instead of 41.3)
constexpr int64_t kTwoMost = 524288;         // two entries a lane up to here, four beyond
constexpr int kFewTiles = 256;               // added up by every workgroup; beyond, by a launch (147 tiles 67 and 76 us, 489 346 and 306)
struct SortPlan {
    int passes, bits, tiles;
};
SortPlan sort_plan(int64_t n, int64_t num_rows)
{
    int bits = 0;
    while (num_rows >> bits) ++bits;             // (padding has the row num_rows)
    SortPlan p;
    p.passes = (int)ceil_div(bits, n <= kWideMost ? kWideBits : kNarrowBits);
    p.bits = (int)ceil_div(bits, p.passes);
    if (p.bits < kLeastBits) p.bits = kLeastBits;
    p.tiles = (int)ceil_div(n, kSortBlock * (n <= kWideMost ? 1 : n <= kTwoMost ? 2 : 4));
    return p;
}
// words of the histograms (and twice that, and a tile more, of their scan) that any batch of up to n positions needs
int64_t hist_words(int64_t n)
{
    const int64_t wide = kWideMost / kSortBlock << (kWideBits - 1);
    const int64_t two = ceil_div(n < kTwoMost ? n : kTwoMost, 2 * kSortBlock), four = ceil_div(n, 4 * kSortBlock);
    const int64_t narrow = (two > four ? two : four) << (kNarrowBits - 1);
    return wide > narrow ? wide : narrow;
}

struct Areas {
    uint64_t *entries[2];
    uint32_t *hist, *before, *heads, *tail_index, *arrived;
    float *head, *tail;
};
size_t arrived_bytes(int64_t n, int64_t dim) { return 4 * (size_t)most_tiles(n) * (size_t)most_col_blocks(dim); }
size_t lay_out(int64_t n, int64_t dim, char *base, Areas *out)
{
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = base + at;
        at += (bytes + 255) & ~(size_t)255;
        return p;
    };
    const int64_t tiles = most_tiles(n);
    out->entries[0] = (uint64_t *)take(8 * (size_t)n);
    out->entries[1] = (uint64_t *)take(8 * (size_t)n);
    out->hist = (uint32_t *)take(4 * (size_t)hist_words(n));
    out->before = (uint32_t *)take(8 * ((size_t)hist_words(n) + (1 << (kNarrowBits - 1))));
    out->heads = (uint32_t *)take(4 * (size_t)tiles);
    out->tail_index = (uint32_t *)take(4 * (size_t)tiles);
    out->arrived = (uint32_t *)take(arrived_bytes(n, dim));
    out->head = (float *)take(4 * (size_t)tiles * (size_t)dim);
    out->tail = (float *)take(4 * (size_t)tiles * (size_t)dim);
    return at;
}

mpzch_status_t ensure(mpzch_embed_t *h, int64_t n, int64_t dim)
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return MPZCH_ERR_HIP;
    if (h->base && h->device != dev) return MPZCH_ERR_INVALID_ARG;
    if (h->base && n <= h->cap_n && dim <= h->cap_dim) return MPZCH_OK;
    if (n < 1024) n = 1024;
    if (dim < 64) dim = 64;
    if (n < h->cap_n) n = h->cap_n;
    if (dim < h->cap_dim) dim = h->cap_dim;
    if (h->base) {
        if (hipDeviceSynchronize() != hipSuccess) return MPZCH_ERR_HIP;
        (void)hipFree(h->base);
        h->base = nullptr;
        h->cap_n = h->cap_dim = 0;
    }
    Areas areas;
    char *base = nullptr;
    if (hipMalloc((void **)&base, lay_out(n, dim, nullptr, &areas)) != hipSuccess) {
        (void)hipGetLastError();
        return MPZCH_ERR_ALLOC;
    }
    lay_out(n, dim, base, &areas);
    // the counters are zero between the calls; this is the only clear
    if (hipMemset(areas.arrived, 0, arrived_bytes(n, dim)) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
        (void)hipFree(base);
        return MPZCH_ERR_HIP;
    }
    h->base = base;
    h->device = dev;
    h->cap_n = n;
    h->cap_dim = dim;
    return MPZCH_OK;
}

template <bool FIRST, int ITEMS, int BITS>
mpzch_status_t sort_pass(const Areas &w, const SortPlan &p, const SortSource &src, uint64_t *to, hipStream_t s)
{
    TRY(launch(k_sort_hist<FIRST, ITEMS, BITS>, p.tiles, kSortBlock, s, src, w.hist));
    const uint32_t *before = nullptr;
    if (p.tiles > kFewTiles) {
        before = w.before;
        TRY(launch(k_sort_scan, (1 << p.bits) / kScanDigits, kSortBlock, s, (const uint32_t *)w.hist, w.before, p.tiles, p.bits));
    }
    return launch(k_sort_scatter<FIRST, ITEMS, BITS>, p.tiles, kSortBlock, s, src, (const uint32_t *)w.hist, before, p.tiles, to);
}
template <bool FIRST>
mpzch_status_t sort_pass(const Areas &w, const SortPlan &p, const SortSource &src, uint64_t *to, hipStream_t s)
{
    if (src.n <= kWideMost) return sort_pass<FIRST, 1, kWideBits>(w, p, src, to, s);
    if (src.n <= kTwoMost) return sort_pass<FIRST, 2, kNarrowBits>(w, p, src, to, s);
    return sort_pass<FIRST, 4, kNarrowBits>(w, p, src, to, s);
}

// entries in ascending order; *out: where they are
mpzch_status_t sort_slots(const Areas &w, const int64_t *slots, int64_t n, int64_t num_rows, const uint64_t **out, hipStream_t s)
{
    SortSource src{slots, nullptr, row_mod(num_rows), n, 32, 0};
    if (n <= kRankMax) {
        *out = w.entries[0];
        return launch(k_sort_rank, (int)ceil_div(n, kRanked), kSortBlock, s, slots, src.mod, (int32_t)n, w.entries[0]);
    }
    const SortPlan p = sort_plan(n, num_rows);
    src.bits = p.bits;
    for (int k = 0; k < p.passes; ++k, src.shift += p.bits) {
        uint64_t *to = w.entries[k & 1];
        if (k == 0) TRY(sort_pass<true>(w, p, src, to, s));
        else TRY(sort_pass<false>(w, p, src, to, s));
        src.entries = to;
    }
    *out = src.entries;
    return MPZCH_OK;
}

// Everything behind the argument checks.  `a` holds what the caller gave.
template <bool STEP>
mpzch_status_t run_gradient(mpzch_embed_t *h, const int64_t *slots, int64_t n, int64_t num_rows, const Rows &grad, ReduceArgs a,
                            hipStream_t s)
{
    TRY(ensure(h, n, grad.dim));
    Areas w;
    lay_out(h->cap_n, h->cap_dim, h->base, &w);
    if (n > 0) TRY(sort_slots(w, slots, n, num_rows, &a.entries, s));
    else a.entries = w.entries[0];

    const int width = piece_width(grad.dim, grad.type, grad.type);
    const ReducePlan p = reduce_plan(n, grad.dim, width);
    a.n = n;
    a.num_rows = (uint32_t)num_rows;
    a.dim = (int32_t)grad.dim;
    a.tiles = p.tiles;
    a.tile = p.tile;
    a.lanes = p.lanes;
    a.col_blocks = p.col_blocks;
    a.grad = (const char *)grad.at;
    a.grad_stride = (uint32_t)grad.stride;
    a.read_past_caches = n * grad.dim * element_bytes(grad.type) >= kReadPastCaches;
    a.tail_index = w.tail_index;
    a.arrived = w.arrived;
    a.head = w.head;
    a.tail = w.tail;
    a.heads = w.heads;
    const int grid = p.tiles * p.col_blocks;
    if constexpr (STEP) {
        return a.type == MPZCH_F32 ? launch_reduce_4(a, grad.type, width, p.pieces, grid, s) : launch_reduce_2(a, grad.type, width, p.pieces, grid, s);
    } else {
        a.heads_are = n <= kRankMax ? kCountHere : p.tiles <= kTilesAdded ? kOfTile : kBeforeTile;
        if (a.heads_are != kCountHere) TRY(launch(k_count_heads, p.tiles, kBlock, s, a.entries, n, a.num_rows, a.tile, w.heads));
        if (a.heads_are == kBeforeTile) TRY(launch(k_scan_heads, 1, kSortBlock, s, w.heads, p.tiles));
        return launch_reduce_0(a, grad.type, width, p.pieces, grid, s);
    }
}

constexpr int64_t kMaxGradRows = ((int64_t)1 << 32) - 2;     // rows and the padding behind them in 32 bits, one value to spare
constexpr int64_t kMaxStride = ((int64_t)1 << 32) - 1;

}  // namespace

extern "C" {

mpzch_status_t mpzch_embed(const int64_t *slots, int64_t n, const void *rows, int32_t rows_type, int64_t num_rows, int64_t dim,
                           int64_t row_stride_bytes, float scale, double drop_p, const int64_t *seed,
                           void *out, int32_t out_type, int64_t out_stride_bytes, void *stream)
{
    if (n < 0 || n > MPZCH_MAX_BATCH || num_rows < 1 || dim < 1 || dim > MPZCH_MAX_DIM) return MPZCH_ERR_INVALID_ARG;
    const Rows in{rows, rows_type, dim, row_stride_bytes}, to{out, out_type, dim, out_stride_bytes};
    EmbedArgs a;
    if (!make_mask(scale, drop_p, seed, dim, &a.factor, &a.mask)) return MPZCH_ERR_INVALID_ARG;
    if (n == 0 && type_ok(rows_type) && type_ok(out_type)) return MPZCH_OK;
    if (!slots || !in.ok() || !to.ok()) return MPZCH_ERR_INVALID_ARG;
    const int width = piece_width(dim, rows_type, out_type);
    a.slots = slots;
    a.n = n;
    a.rows = (const char *)rows;
    a.mod = row_mod(num_rows);
    a.row_stride = row_stride_bytes;
    a.out = (char *)out;
    a.out_stride = out_stride_bytes;
    a.dim = (int32_t)dim;
    a.pieces = div32((uint32_t)ceil_div(dim, width));
    a.past_caches = n * dim * element_bytes(out_type) >= kPastCaches;
    hipStream_t s = (hipStream_t)stream;
    const int64_t blocks = ceil_div(n * a.pieces.d, kBlock * kEmbedPieces);
    const int grid = (int)(blocks < kEmbedBlocks ? blocks : kEmbedBlocks);
    switch (rows_type) {
    case MPZCH_F32: return launch_embed<float>(a, out_type, width, grid, s);
    case MPZCH_BF16: return launch_embed<__bf16>(a, out_type, width, grid, s);
    default: return launch_embed<_Float16>(a, out_type, width, grid, s);
    }
}

mpzch_status_t mpzch_embed_create(mpzch_embed_t **out)
{
    if (!out) return MPZCH_ERR_INVALID_ARG;
    *out = new (std::nothrow) mpzch_embed_s();
    return *out ? MPZCH_OK : MPZCH_ERR_ALLOC;
}

mpzch_status_t mpzch_embed_destroy(mpzch_embed_t *h)
{
    if (!h) return MPZCH_OK;
    if (h->base) {
        (void)hipDeviceSynchronize();
        (void)hipFree(h->base);
    }
    delete h;
    return MPZCH_OK;
}

mpzch_status_t mpzch_embed_reserve(mpzch_embed_t *h, int64_t max_n, int64_t max_dim)
{
    if (!h || max_n < 0 || max_n > MPZCH_MAX_BATCH || max_dim < 0 || max_dim > MPZCH_MAX_DIM) return MPZCH_ERR_INVALID_ARG;
    return ensure(h, max_n, max_dim);
}

mpzch_status_t mpzch_embed_grad(mpzch_embed_t *h, const int64_t *slots, int64_t n, int64_t num_rows,
                                const void *grad, int32_t grad_type, int64_t dim, int64_t grad_stride_bytes,
                                float scale, double drop_p, const int64_t *seed,
                                int64_t *out_slots, void *out_rows, int32_t out_type, int64_t out_cap, int64_t *out_count,
                                void *stream)
{
    if (!h || n < 0 || n > MPZCH_MAX_BATCH || num_rows < 1 || dim < 1 || dim > MPZCH_MAX_DIM || out_cap < 0 || !out_count)
        return MPZCH_ERR_INVALID_ARG;
    if (!type_ok(grad_type) || !type_ok(out_type)) return MPZCH_ERR_INVALID_ARG;
    if (num_rows > kMaxGradRows || grad_stride_bytes > kMaxStride) return MPZCH_ERR_UNSUPPORTED;
    ReduceArgs a;
    std::memset(&a, 0, sizeof a);
    if (!make_mask(scale, drop_p, seed, dim, &a.factor, &a.mask)) return MPZCH_ERR_INVALID_ARG;
    const Rows g{grad, grad_type, dim, grad_stride_bytes};
    const Rows to{out_rows, out_type, dim, dim * element_bytes(out_type)};
    if (n > 0 && (!slots || !g.ok())) return MPZCH_ERR_INVALID_ARG;
    if (out_cap > 0 && (!out_slots || !to.ok())) return MPZCH_ERR_INVALID_ARG;
    a.out_slots = out_slots;
    a.out_count = out_count;
    a.out_rows = (char *)out_rows;
    a.cap = out_cap;
    a.past_caches = (n < out_cap ? n : out_cap) * dim * element_bytes(out_type) >= kPastCaches;
    a.type = out_type;
    return run_gradient<false>(h, slots, n, num_rows, g, a, (hipStream_t)stream);
}

mpzch_status_t mpzch_embed_step(mpzch_embed_t *h, const int64_t *slots, int64_t n,
                                const void *grad, int32_t grad_type, int64_t dim, int64_t grad_stride_bytes,
                                float scale, double drop_p, const int64_t *seed,
                                void *rows, int32_t rows_type, int64_t num_rows, int64_t row_stride_bytes,
                                float *state, const float *lr, float eps, void *stream)
{
    if (!h || n < 0 || n > MPZCH_MAX_BATCH || num_rows < 1 || dim < 1 || !lr) return MPZCH_ERR_INVALID_ARG;
    if (!type_ok(grad_type) || !type_ok(rows_type)) return MPZCH_ERR_INVALID_ARG;
    if (num_rows > kMaxGradRows || dim > MPZCH_MAX_STEP_DIM || grad_stride_bytes > kMaxStride || row_stride_bytes > kMaxStride)
        return MPZCH_ERR_UNSUPPORTED;
    if (state && !(std::isfinite(eps) && eps > 0.f)) return MPZCH_ERR_INVALID_ARG;
    ReduceArgs a;
    std::memset(&a, 0, sizeof a);
    if (!make_mask(scale, drop_p, seed, dim, &a.factor, &a.mask)) return MPZCH_ERR_INVALID_ARG;
    const Rows g{grad, grad_type, dim, grad_stride_bytes}, w{rows, rows_type, dim, row_stride_bytes};
    if (n > 0 && (!slots || !g.ok())) return MPZCH_ERR_INVALID_ARG;
    if (!w.ok()) return MPZCH_ERR_INVALID_ARG;
    if (n == 0) return MPZCH_OK;
    a.rows = (char *)rows;
    a.row_stride = (uint32_t)row_stride_bytes;
    // (one more rounding of the mean than a division by dim, half a step, where dim is no power of two: the sum has dim of them)
    a.per_element = 1.f / (float)dim;
    a.type = rows_type;
    a.state = state;
    a.lr = lr;
    a.eps = eps;
    return run_gradient<true>(h, slots, n, num_rows, g, a, (hipStream_t)stream);
}

}  // extern "C"
