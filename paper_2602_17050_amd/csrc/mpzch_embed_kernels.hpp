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

// V neighbouring elements as they lie in memory, aligned as one element: rows of any length and tensors that begin anywhere are
// read with the same wide loads.  (The last piece of a row whose length is no multiple of V is moved back to the row's last V
// elements: what two lanes have of it is the same.)
template <typename E, int V>
struct PackOf {
    typedef E type __attribute__((ext_vector_type(V), aligned(sizeof(E))));
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
// Rounded once, to nearest, ties to even.  past_caches: non-temporally, so that large results do not drive out of the caches what
// is read again.  Of three tables in turn, us, through / past: lookup of 2 M rows of 256 bytes 164 / 157.4 (and with non-temporal loads
// of the table's rows 179), of 33 MB 10.6 / 9.8, gradient of 2 M rows (271 MB of sums) 288.5 / 280.
template <typename E, int V>
__device__ __forceinline__ void store_floats(char *at, Floats<V> v, bool past_caches = false)
{
    typedef E to __attribute__((ext_vector_type(V)));
    const Pack<E, V> x = __builtin_convertvector(v, to);
    if (past_caches) {
        asm volatile("" ::: "memory");           // (or the compiler makes one plain store of the two)
        __builtin_nontemporal_store(x, reinterpret_cast<Pack<E, V> *>(at));
        asm volatile("" ::: "memory");
    } else {
        *reinterpret_cast<Pack<E, V> *>(at) = x;
    }
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
__device__ __forceinline__ void store_typed(int type, char *base, int64_t element, Floats<V> v, bool past_caches = false)
{
    if (type == kF32) store_floats<float, V>(base + element * 4, v, past_caches);
    else if (type == kBf16) store_floats<__bf16, V>(base + element * 2, v, past_caches);
    else store_floats<_Float16, V>(base + element * 2, v, past_caches);
}

// V elements as they lie in memory, 16 or 32 bits each: converted where they are used, so that many loads can be under way
template <int BYTES, int V>
struct Raw {
    typedef std::conditional_t<BYTES == 4, float, uint16_t> E;
    Pack<E, V> v;
    __device__ __forceinline__ void load(const char *rows, int64_t element) { v = *reinterpret_cast<const Pack<E, V> *>(rows + element * BYTES); }
    __device__ __forceinline__ void load_past_caches(const char *rows, int64_t element)
    {
        v = __builtin_nontemporal_load(reinterpret_cast<const Pack<E, V> *>(rows + element * BYTES));
    }
    __device__ __forceinline__ Floats<V> floats(int type) const
    {
        if constexpr (BYTES == 4) {
            return __builtin_convertvector(v, Floats<V>);
        } else {
            typedef uint16_t u16v __attribute__((ext_vector_type(V)));
            typedef __bf16 bf16v __attribute__((ext_vector_type(V)));
            typedef _Float16 f16v __attribute__((ext_vector_type(V)));
            const u16v bits = v;
            return type == kBf16 ? __builtin_convertvector(__builtin_bit_cast(bf16v, bits), Floats<V>)
                                 : __builtin_convertvector(__builtin_bit_cast(f16v, bits), Floats<V>);
        }
    }
};

// ------------------------------------------------------------------ the mask
constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

struct Mask {
    const uint64_t *seed;
    uint32_t threshold;          // T; 0: no dropout
    uint64_t row_step;           // from one position's words to the next one's, in the generator: ceil(dim / 4) * kGolden
    int32_t ragged;              // whether pieces may begin inside a word: dim is no multiple of 4
};

// the generator's state before the word of element j0 of position 0
__device__ __forceinline__ uint64_t mask_column(uint64_t seed, int32_t j0) { return seed + (uint64_t)(uint32_t)(j0 >> 2) * kGolden; }
// v with the dropped ones of the elements j0 .. j0 + V of position i at zero; at_column = mask_column(seed, j0)
template <int V>
__device__ __forceinline__ Floats<V> masked(Floats<V> v, uint64_t at_column, const Mask &m, uint32_t i, int32_t j0)
{
    const uint64_t first = at_column + (uint64_t)i * m.row_step;
    constexpr int kWords = (V + 3) / 4;
    uint64_t draws[kWords];
#pragma unroll
    for (int w = 0; w < kWords; ++w) draws[w] = mix64(first + w * kGolden);
    if (m.ragged) {
        const int shift = 16 * (j0 & 3);
        if (shift) {                             // the piece goes on in the next word
            uint64_t next = 0;
            if (shift + 16 * V > 64 * kWords) next = mix64(first + kWords * kGolden);
#pragma unroll
            for (int w = 0; w < kWords; ++w)
                draws[w] = draws[w] >> shift | (w + 1 < kWords ? draws[w + 1 < kWords ? w + 1 : 0] : next) << (64 - shift);
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if ((uint32_t)(draws[e / 4] >> (16 * (e % 4)) & 0xFFFF) < m.threshold) v[e] = 0.f;
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

// One lane per piece of V elements; a workgroup takes kEmbedPieces * kBlock neighbouring pieces of the output in a turn.  Bound by
// memory: slots, rows (random, each a few lines) and output.  2 M positions of 128 bf16 elements out of 25 M, 661 MB to move, by
// pieces of a lane (2, 4, 8): 179 165 167 us; with 8, 32 and any number of workgroups for a compute unit 172 165 159.5;
// with loads that no lane leaves out 157.5 (4.2 TB/s).
constexpr int kEmbedPieces = 4;
constexpr int64_t kEmbedBlocks = (int64_t)1 << 21;     // so that a turn's pieces fit 32 bits
struct EmbedArgs {
    const int64_t *slots;
    int64_t n;
    const char *rows;
    RowMod mod;
    int64_t row_stride;
    char *out;
    int64_t out_stride;
    int32_t dim;
    Div32 pieces;                // of a row
    float factor;
    Mask mask;
    bool past_caches;            // the output is stored non-temporally
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
        int32_t column[kEmbedPieces];
        Raw<sizeof(TI), V> v[kEmbedPieces];
#pragma unroll
        for (int u = 0; u < kEmbedPieces; ++u) {
            uint32_t c;
            k[u] = k0 + divided(a.pieces, c0 + u * kBlock + threadIdx.x, &c);
            column[u] = (int32_t)c * V < a.dim - V ? (int32_t)c * V : a.dim - V;
            slot[u] = a.slots[k[u] < a.n ? k[u] : a.n - 1];      // (lanes behind the last piece store nothing)
        }
#pragma unroll
        for (int u = 0; u < kEmbedPieces; ++u) {
            // (padding: the first row, in the caches)
            const int64_t row = slot[u] >= 0 ? row_of(a.mod, slot[u]) : 0;
            v[u].load(a.rows + row * a.row_stride, column[u]);
        }
#pragma unroll
        for (int u = 0; u < kEmbedPieces; ++u) {
            if (i + u * kBlock >= total) continue;
            Floats<V> x = v[u].floats(std::is_same_v<TI, __bf16> ? kBf16 : kF16) * a.factor;
            if constexpr (DROP) x = masked<V>(x, mask_column(seed, column[u]), a.mask, (uint32_t)k[u], column[u]);
            if (slot[u] < 0) x = Floats<V>(0.f);
            store_floats<TO, V>(a.out + k[u] * a.out_stride + (int64_t)column[u] * sizeof(TO), x, a.past_caches);
        }
        k0 += dk;
        c0 += dc;
        if (c0 >= a.pieces.d) {
            c0 -= a.pieces.d;
            ++k0;
        }
    }
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

}  // namespace mpzch
