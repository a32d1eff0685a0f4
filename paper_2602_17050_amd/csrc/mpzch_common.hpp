// What the device code of the remap and of the embedding operators share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mpzch {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x3 __attribute__((ext_vector_type(3)));

constexpr int kWave = 64;
constexpr int kBlock = 256;
constexpr int kWavesPerBlock = kBlock / kWave;

__device__ __forceinline__ int lane_id() { return threadIdx.x & (kWave - 1); }

// Output 0 of the SplitMix64 generator that starts at x; output k is mix64(x + k * golden).
__device__ __forceinline__ uint64_t mix64(uint64_t x)
{
    uint64_t z = x + 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// slot mod num_rows without a division: the quotient by the reciprocal floor((2^64 - 1) / num_rows) is the exact one or
// one less for slots below 2^63.
struct RowMod {
    int64_t num_rows;
    uint64_t inverse;
};
__host__ __device__ inline RowMod row_mod(int64_t num_rows) { return RowMod{num_rows, ~0ull / (uint64_t)num_rows}; }
__device__ __forceinline__ int64_t row_of(const RowMod &m, int64_t slot)
{
    if (slot < m.num_rows) return slot;
    const int64_t r = slot - (int64_t)(__umul64hi((uint64_t)slot, m.inverse) * (uint64_t)m.num_rows);
    return r >= m.num_rows ? r - m.num_rows : r;
}

}  // namespace mpzch
