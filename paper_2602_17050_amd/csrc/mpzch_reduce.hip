// Sums over the sorted entries of a batch, for the gradient (MPZCH_TABLE_BYTES 0) or the step of a table whose elements have that
// many bytes.
#include "mpzch_host.hpp"
#include "mpzch_reduce.hpp"

namespace mpzch {

namespace {

// A run is the entries of one row.  A workgroup has a tile of neighbouring entries, a group of lanes in it (a power of two of
// them, V * NP elements of the row for each) a part of the tile.  What a group knows of a run:
//   it begins and ends in the part   the group emits its sum
//   it began before                  the part has a share of it; it may go through the part
//   it goes on behind                the group in whose part it begins adds the shares of the parts that it goes through
// A run that goes on behind the tile for kBehind entries at most is finished there, by all groups of the workgroup in which it
// is, and the following tiles leave it out.  A longer one has a share in memory for every tile; which workgroup is the last to
// write one is found with a counter, and that one adds them up.  All sums are in 32 bits, in an order that n, dim, the types and
// the run's place alone determine: who is last does not change it.  (Against 64 bits they are off by 4e-8 to 5e-8 of the gradient's
// size; sums in 64 bits, rounded to 32 at the end, by 2e-8 to 3e-8: twice the registers for about one bit.)
//
// Bound by memory where batches are long: every gradient row is read once, 256 bytes and more at a random place.  2 M positions
// of 128 bf16 elements (799 MB to move) take this kernel 202 us (4.0 TB/s; a copy 4.8), a step of 1 M (394 MB) 109, and the vector
// units are busy for nearly half of that.  By round trips where they are short: entries, gradients and weights, shares.  65 536
// positions with a step (20 MB) 16 us, 1 024 7 to 8.
constexpr int kBehind = 128;
constexpr uint32_t kNoRow = ~0u;
constexpr uint32_t kHeadShare = 1, kThrough = 2, kTailShare = 4;      // flags of a part

// Shares are read by a workgroup that may run on another die, with an L2 of its own: they are stored and loaded as atomics of the
// whole device, which go past the L2s one by one.  (A fence of the device instead writes the whole L2 back, the other workgroups'
// outputs with it: gradient of 2 M positions 336 -> 535 us.)
template <typename T>
__device__ __forceinline__ void store_shared(T *to, T v) { __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T>
__device__ __forceinline__ T load_shared(const T *at) { return __hip_atomic_load(const_cast<T *>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// this lane's stores have reached the memory that all dies see
__device__ __forceinline__ void wait_for_stores() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// the sum over the lanes of a group (a power of two of them, the same for the wavefront), in every lane
template <int CONTROL>
__device__ __forceinline__ float from_lane(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CONTROL, 0xF, 0xF, true));
}
__device__ __forceinline__ float group_sum(float x, int lanes)
{
    if (lanes > 1) x += from_lane<0xB1>(x);          // lanes 1 0 3 2
    if (lanes > 2) x += from_lane<0x4E>(x);          // lanes 2 3 0 1
    if (lanes > 4) x += from_lane<0x141>(x);         // the other four of eight, mirrored: they have one sum
    if (lanes > 8) x += from_lane<0x140>(x);         // the other eight of sixteen
    if (lanes > 16) x += __shfl_xor(x, 16);
    if (lanes > 32) x += __shfl_xor(x, 32);
    return x;
}

[[maybe_unused]] __device__ __forceinline__ uint32_t wave_sum(uint32_t x)
{
    x += (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true);
    x += (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true);
    x += (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true);
    x += (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, true);
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// how many of x(0) .. x(count - 1), ascending, are below v (or, with EQUAL, not above it): a wavefront looks at 64 of them at a time
template <bool EQUAL, typename X>
__device__ __forceinline__ int32_t wave_search(int32_t count, uint32_t v, X x)
{
    int32_t low = 0, high = count;               // the answer is in [low, high]
    while (low < high) {
        const int32_t step = (high - low + kWave - 1) / kWave;
        const int32_t at = low + lane_id() * step;
        bool below = false;
        if (at < high) below = EQUAL ? x(at) <= v : x(at) < v;
        const int yes = __popcll(__ballot(below));      // ascending: the first `yes` lanes
        if (yes == 0) return low;
        const int32_t last = low + (yes - 1) * step;
        high = last + step < high ? last + step : high;
        low = last + 1;
    }
    return low;
}

// lr / (sqrt(state) + eps) need not fit 32 bits where its product with a sum G does: an eps below lr / 2^128 on a state of zero would
// give infinity, and NaN for a sum of zero.  A quotient that is no ordinary number is divided by a power of two, with which G is
// multiplied first.  True if there is one.  (Step of 1 M positions 162.7 -> 164.6 us; with the power for every quotient 167.)
__device__ __forceinline__ bool adagrad_rate(float lr, float state, float eps, float &rate, float &power)
{
    const float root = sqrtf(state) + eps;
    rate = lr / root;
    constexpr int kInfinite = 0x204, kSubnormal = 0x90, kZero = 0x60;
    if (__builtin_expect(!__builtin_amdgcn_classf(rate, kInfinite | kSubnormal | kZero), 1)) return false;
    // (root is at least 2^-149, and lr beyond 2^-21 where the quotient is infinite: finite for all lr below 2^78)
    const float up = fabsf(rate) > 1.f ? 0x1p50f : root > 0x1p-60f ? 0x1p-50f : 1.f;
    power = up * up;
    rate = lr / up / (root * up);
    return true;
}

// The sum of a run whose shares lie in the tiles owner .. last, by a whole workgroup: `lanes` lanes (a power of two) for the
// columns of this block, and the rest of it for every sharers-th tile.
constexpr int kJoinColumns = 2;              // of a lane at a time; a step has the whole row at once
template <bool STEP>
__device__ __forceinline__ void join_run(const ReduceArgs &a, float *part, uint32_t row, int32_t owner, int32_t last, int32_t col_first,
                                         int32_t col_end)
{
    constexpr int kColumns = kJoinColumns;
    constexpr int kJoinAhead = 16;
    static_assert(!STEP || kColumns * kReduceBlock >= MPZCH_MAX_STEP_DIM);
    int32_t lanes = kWave;
    while (lanes < kReduceBlock && lanes < col_end - col_first) lanes *= 2;
    const int sharers = kReduceBlock / lanes, sharer = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    const int64_t index = STEP ? 0 : load_shared(a.tail_index + owner);
    for (int32_t c0 = col_first; c0 < col_end; c0 += kColumns * lanes) {
        __syncthreads();                         // (`part` is free)
        float sum[kColumns];
        float squares = 0.f;
        float weight[kColumns], state = 0.f, lr = 0.f;
        if constexpr (STEP) {                    // (under way with the shares)
            lr = *a.lr;
            if (a.state) state = a.state[row];
#pragma unroll
            for (int p = 0; p < kColumns; ++p) {
                const int32_t c = c0 + p * lanes + lane;
                weight[p] = load_typed<1>(a.type, a.rows + (uint64_t)row * a.row_stride, c < col_end ? c : 0)[0];
            }
        }
#pragma unroll
        for (int p = 0; p < kColumns; ++p) {
            const int32_t c = c0 + p * lanes + lane;
            sum[p] = sharer == 0 && c < col_end ? load_shared(a.tail + (int64_t)owner * a.dim + c) : 0.f;
        }
        for (int32_t t0 = owner + 1 + sharer; t0 <= last; t0 += kJoinAhead * sharers) {
            float v[kJoinAhead][kColumns];
#pragma unroll
            for (int u = 0; u < kJoinAhead; ++u) {
                const int32_t t = t0 + u * sharers <= last ? t0 + u * sharers : last;
#pragma unroll
                for (int p = 0; p < kColumns; ++p) {
                    const int32_t c = c0 + p * lanes + lane;
                    v[u][p] = load_shared(a.head + (int64_t)t * a.dim + (c < col_end ? c : col_first));
                }
            }
#pragma unroll
            for (int u = 0; u < kJoinAhead; ++u)
#pragma unroll
                for (int p = 0; p < kColumns; ++p) sum[p] += t0 + u * sharers <= last ? v[u][p] : 0.f;
        }
        if (sharers > 1) {
#pragma unroll
            for (int p = 0; p < kColumns; ++p) part[p * kReduceBlock + threadIdx.x] = sum[p];
            __syncthreads();
            if (sharer == 0) {
#pragma unroll
                for (int g = 1; g < kReduceBlock / kWave; ++g)
#pragma unroll
                    for (int p = 0; p < kColumns; ++p) sum[p] += g < sharers ? part[p * kReduceBlock + (g < sharers ? g : 0) * lanes + lane] : 0.f;
            }
        }
#pragma unroll
        for (int p = 0; p < kColumns; ++p) {
            const int32_t c = c0 + p * lanes + lane;
            sum[p] *= a.factor;
            if (c < col_end && sharer == 0) squares += sum[p] * sum[p];
        }
        if constexpr (STEP) {
            float rate = lr;
            if (a.state) {
                __syncthreads();                  // (the shares have been read)
                const float of_wave = group_sum(squares, kWave);
                if (lane_id() == 0) part[threadIdx.x / kWave] = of_wave;
                __syncthreads();
                float all = 0.f;
#pragma unroll
                for (int w = 0; w < kReduceBlock / kWave; ++w) all += part[w];
                state += all * a.per_element;
                if (threadIdx.x == 0) a.state[row] = state;
                float power;
                if (adagrad_rate(lr, state, a.eps, rate, power)) {
#pragma unroll
                    for (int p = 0; p < kColumns; ++p) sum[p] *= power;
                }
            }
#pragma unroll
            for (int p = 0; p < kColumns; ++p) {
                const int32_t c = c0 + p * lanes + lane;
                if (c >= col_end || sharer != 0) continue;
                store_typed<1>(a.type, a.rows + (uint64_t)row * a.row_stride, c, Floats<1>(weight[p] - sum[p] * rate));
            }
        } else if (sharer == 0 && index < a.cap) {
            if (c0 == 0 && lane == 0) a.out_slots[index] = row;
#pragma unroll
            for (int p = 0; p < kColumns; ++p) {
                const int32_t c = c0 + p * lanes + lane;
                if (c < col_end) store_typed<1>(a.type, a.out_rows, index * a.dim + c, Floats<1>(sum[p]));
            }
        }
    }
}

// WB: bytes of an element of the table, for a step; 0: the gradient
template <typename TG, int V, int NP, int WB>
__global__ __launch_bounds__(kReduceBlock) void k_reduce(ReduceArgs a)
{
    constexpr bool STEP = WB != 0;
    constexpr int kWaves = kReduceBlock / kWave;
    __shared__ uint32_t row_of_entry[kReduceTile + kBehind + 2], position[kReduceTile + kBehind];
    __shared__ uint32_t heads_before[kWaves], wave_through[kWaves], joins;
    __shared__ uint64_t run_begins[(kReduceTile + kBehind) / kWave];
    __shared__ Floats<V> shares[NP][kReduceBlock];
    __shared__ float join_part[kJoinColumns * kReduceBlock];

    const int32_t tile_index = (int32_t)(blockIdx.x / (uint32_t)a.col_blocks), block_col = (int32_t)(blockIdx.x % (uint32_t)a.col_blocks);
    const int64_t first = (int64_t)tile_index * a.tile;
    const int64_t left = a.n - first;
    const int m = (int)(left < a.tile ? left : a.tile);
    const int behind = (int)(left - m < kBehind ? left - m : kBehind);
    const int groups = kReduceBlock / a.lanes, per = a.tile / groups;
    const int group = threadIdx.x / a.lanes, lane = threadIdx.x % a.lanes, wave = threadIdx.x / kWave;

    // the tile's entries and the next ones, the row before them and the one behind; for a gradient, where runs begin, 64 entries a word
    for (int k = threadIdx.x; k < m + behind; k += kReduceBlock) {
        const uint64_t e = a.entries[first + k];
        const uint32_t row = (uint32_t)(e >> 32);
        if constexpr (!STEP) {
            const uint32_t before = first + k > 0 ? row_at(a.entries, first + k - 1) : kNoRow;
            const uint64_t begins = __ballot(k < m && row != a.num_rows && row != before);
            if (lane_id() == 0) run_begins[k / kWave] = begins;
        }
        row_of_entry[k + 1] = row;
        position[k] = (uint32_t)e;
    }
    if (threadIdx.x == 0) {
        row_of_entry[0] = first > 0 ? row_at(a.entries, first - 1) : kNoRow;
        row_of_entry[m + behind + 1] = first + m + behind < a.n ? row_at(a.entries, first + m + behind) : kNoRow;
    }
    uint32_t earlier = 0;                        // runs that begin in the tiles before this: a lane's share of them
    if constexpr (!STEP) {
        if (a.heads_are == kOfTile) {
            for (int t = threadIdx.x; t < tile_index; t += kReduceBlock) earlier += a.heads[t];
        } else if (a.heads_are == kCountHere) {
#pragma unroll 4
            for (int64_t i = threadIdx.x; i < first; i += kReduceBlock) {
                const uint32_t row = row_at(a.entries, i);
                earlier += row != a.num_rows && (i == 0 || row_at(a.entries, i - 1) != row);
            }
        } else if (threadIdx.x == 0) {
            earlier = a.heads[tile_index];
        }
    }
    if constexpr (!STEP) {
        earlier = wave_sum(earlier);
        if (lane_id() == 0) heads_before[wave] = earlier;
    }
    __syncthreads();
    const int begin = group * per < m ? group * per : m, end = begin + per < m ? begin + per : m;
    // `index`: runs that begin before the part
    uint32_t index = 0;
    if constexpr (!STEP) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) index += heads_before[w];
        const bool counts = blockIdx.x == gridDim.x - 1 && threadIdx.x == 0;
        if (counts) {
            uint32_t all = 0;
            for (int k = 0; k < m; k += kWave) all += (uint32_t)__popcll(run_begins[k / kWave]);
            *a.out_count = (int64_t)index + all;
        }
#pragma unroll 4
        for (int k = 0; k < begin / kWave; ++k) index += (uint32_t)__popcll(run_begins[k]);
        if (begin % kWave) index += (uint32_t)__popcll(run_begins[begin / kWave] & ((1ull << begin % kWave) - 1));
    }
    // what is left out: padding, and the rest of a run that an earlier tile has finished
    const uint32_t tile_end_row = m > 0 ? row_of_entry[m] : kNoRow;
    const bool begins_inside = m > 0 && row_of_entry[0] == row_of_entry[1];
    // (the entry kBehind behind the tile's begin; it is in LDS, for the tile and kBehind more are)
    const bool finished = begins_inside && row_of_entry[1 + (kBehind < m + behind ? kBehind : m + behind)] != row_of_entry[1];
    const uint32_t skipped = finished ? row_of_entry[1] : a.num_rows;
    const bool leaves = m > 0 && row_of_entry[m + 1] == tile_end_row && tile_end_row != a.num_rows && tile_end_row != skipped;
    const bool long_run = leaves && row_of_entry[m + behind + 1] == tile_end_row;      // further than kBehind behind the tile

    // where a piece would begin, and where it does (a.dim: none)
    const auto piece_of = [&](int p) { return ((block_col * NP + p) * a.lanes + lane) * V; };
    int32_t column[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int32_t piece = piece_of(p);
        column[p] = piece < a.dim ? (piece < a.dim - V ? piece : a.dim - V) : a.dim;
    }
    const uint64_t seed = a.mask.threshold ? *a.mask.seed : 0;
    uint64_t mask_at[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) mask_at[p] = mask_column(seed, column[p]);
    const float lr = STEP ? *a.lr : 0.f;
    Floats<V> sum[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) sum[p] = Floats<V>(0.f);

    typedef Raw<STEP ? WB : 4, V> Weights;
    auto load_weights = [&](uint32_t row, Weights (&w)[NP], float &state) {
        state = a.state ? a.state[row] : 0.f;
#pragma unroll
        for (int p = 0; p < NP; ++p) w[p].load(a.rows + (uint64_t)row * a.row_stride, column[p] < a.dim ? column[p] : 0);
    };
    // a finished sum (which nothing looks at behind this)
    auto emit_step = [&](uint32_t row, const Weights (&w)[NP], float state) {
        float rate = lr;
#pragma unroll
        for (int p = 0; p < NP; ++p) sum[p] *= a.factor;
        if (a.state) {
            float squares = 0.f;
            if (a.dim % V == 0) {
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (column[p] < a.dim) squares += sum[p][e] * sum[p][e];
            } else {                             // (elements that another lane has, too, count once)
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (column[p] < a.dim && column[p] + e >= piece_of(p)) squares += sum[p][e] * sum[p][e];
            }
            squares = group_sum(squares, a.lanes);
            state += squares * a.per_element;
            if (lane == 0) a.state[row] = state;
            float power;
            if (adagrad_rate(lr, state, a.eps, rate, power)) {
#pragma unroll
                for (int p = 0; p < NP; ++p) sum[p] *= power;
            }
        }
#pragma unroll
        for (int p = 0; p < NP; ++p)
            if (column[p] < a.dim)
                store_typed<V>(a.type, a.rows + (uint64_t)row * a.row_stride, column[p], w[p].floats(a.type) - sum[p] * rate);
    };
    auto emit_grad = [&](uint32_t row, uint32_t at) {
        if ((int64_t)at >= a.cap) return;
        if (block_col == 0 && lane == 0) a.out_slots[at] = row;
#pragma unroll
        for (int p = 0; p < NP; ++p)
            if (column[p] < a.dim) store_typed<V>(a.type, a.out_rows, (int64_t)((uint64_t)at * (uint32_t)a.dim) + column[p], sum[p] * a.factor, a.past_caches);
    };
    // (unconditional loads, so that all that are asked for are under way at a time: where nothing is wanted, of a row that is in the
    // caches anyway; a lane without columns has the first one)
    typedef Raw<sizeof(TG), V> Gradient;
    constexpr int kGradType = std::is_same_v<TG, float> ? kF32 : std::is_same_v<TG, __bf16> ? kBf16 : kF16;
    auto load_grad = [&](uint32_t at, Gradient (&g)[NP]) {
#pragma unroll
        for (int p = 0; p < NP; ++p) g[p].load(a.grad + (uint64_t)at * a.grad_stride, column[p] < a.dim ? column[p] : 0);
    };
    auto add = [&](const Gradient (&g)[NP], uint32_t at) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const Floats<V> v = g[p].floats(kGradType);
            sum[p] += a.mask.threshold ? masked<V>(v, mask_at[p], a.mask, at, column[p]) : v;
        }
    };

    // entries under way at a time: with 8 a step of 1 M positions took 247 instead of 182 us, with 2 192 (registers, wavefronts)
    constexpr int kAhead = NP > 1 ? 2 : 4;
    uint32_t flags = 0;
    bool from_before = begin < end && row_of_entry[begin] == row_of_entry[begin + 1];
    for (int k0 = begin; k0 < end; k0 += kAhead) {
        Gradient g[kAhead][NP];
        Weights w[kAhead][NP];
        float state[kAhead];
        uint32_t at[kAhead], row[kAhead + 2];    // the entries' rows, and those before and behind them
        bool counts[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead + 2; ++u) row[u] = row_of_entry[k0 + u];       // (behind the part: not looked at)
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            counts[u] = k0 + u < end && row[u + 1] != a.num_rows && row[u + 1] != skipped;
            at[u] = position[counts[u] ? k0 + u : 0];
        }
        if (a.read_past_caches) {
            asm volatile("" ::: "memory");       // (or the compiler makes plain loads of both)
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int p = 0; p < NP; ++p)
                    g[u][p].load_past_caches(a.grad + (uint64_t)at[u] * a.grad_stride, column[p] < a.dim ? column[p] : 0);
            asm volatile("" ::: "memory");
        } else {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) load_grad(at[u], g[u]);
        }
        if constexpr (STEP) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) load_weights(counts[u] && row[u + 2] != row[u + 1] ? row[u + 1] : 0, w[u], state[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (!counts[u]) {
                from_before = false;
                continue;
            }
            if (row[u] != row[u + 1]) ++index;
            add(g[u], at[u]);
            const bool goes_on = row[u + 2] == row[u + 1];
            if (goes_on && k0 + u + 1 < end) continue;
            if (from_before) {
                flags |= kHeadShare | (goes_on ? kThrough : 0);
#pragma unroll
                for (int p = 0; p < NP; ++p) shares[p][threadIdx.x] = sum[p];
            } else if (goes_on) {
                flags |= kTailShare;
            } else if constexpr (STEP) {
                emit_step(row[u + 1], w[u], state[u]);
            } else {
                emit_grad(row[u + 1], index - 1);
            }
            from_before = false;
            if (!goes_on) {
#pragma unroll
                for (int p = 0; p < NP; ++p) sum[p] = Floats<V>(0.f);
            }
        }
    }

    // A chain is the shares of following parts as far as a run goes: first inside every wavefront, from each of its parts to its
    // end, by doubling; the chains from the wavefronts' first parts then go to LDS.
    const bool had_tail = flags & kTailShare;
    Weights tail_weights[NP];                    // (of the run that goes on: under way meanwhile)
    float tail_state = 0.f;
    if constexpr (STEP) load_weights(had_tail ? row_of_entry[end] : 0, tail_weights, tail_state);
    const int in_wave = kWave / a.lanes, place = group % in_wave;
    Floats<V> chain[NP];
    bool through = flags & kThrough;
#pragma unroll
    for (int p = 0; p < NP; ++p) chain[p] = flags & kHeadShare ? shares[p][threadIdx.x] : Floats<V>(0.f);
    for (int d = 1; d < in_wave; d <<= 1) {
        const bool next = __shfl_down((int)through, d * a.lanes);
        const bool adds = through && place + d < in_wave;
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float x = __shfl_down(chain[p][e], d * a.lanes);
                if (adds) chain[p][e] += x;
            }
        if (adds) through = next;
    }
    if (place == 0) {
#pragma unroll
        for (int p = 0; p < NP; ++p) shares[p][threadIdx.x] = chain[p];
        if (lane == 0) wave_through[wave] = through;
    }
    // the run that the part leaves unfinished goes on with the next part's chain
    bool unfinished = had_tail;
    {
        const bool next = __shfl_down((int)through, a.lanes);
        const bool adds = had_tail && place + 1 < in_wave;
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float x = __shfl_down(chain[p][e], a.lanes);
                if (adds) sum[p][e] += x;
            }
        if (adds) unfinished = next;
    }
    __syncthreads();
    auto emit_tail = [&]() {
        if constexpr (STEP) emit_step(row_of_entry[end], tail_weights, tail_state);
        else emit_grad(row_of_entry[end], index - 1);
    };
    auto follow = [&](Floats<V> (&to)[NP], int w) {      // ... and with those of the wavefronts from w on; whether it leaves the tile
        int until = w;
        while (until < kWaves && wave_through[until]) ++until;
        const int last = until < kWaves ? until : kWaves - 1;
#pragma unroll 2
        for (int i = w; i <= last; ++i)
#pragma unroll
            for (int p = 0; p < NP; ++p) to[p] += shares[p][i * kWave + lane];
        return until == kWaves;
    };
    if (unfinished) unfinished = follow(sum, wave + 1);
    if (had_tail && !unfinished) emit_tail();
    // the run that came from the tile before
    const bool has_head = group == 0 && (flags & kHeadShare);
    const bool head_goes_on = has_head && through && follow(chain, 1);

    const bool finishes = leaves && !long_run;   // (the same for the whole workgroup)
    if (finishes) {                              // the entries behind the tile, a part of them for every group
        const int share = (kBehind + groups - 1) / groups;
        const int from = m + group * share, to = from + share < m + behind ? from + share : m + behind;
        Floats<V> kept[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            kept[p] = sum[p];
            sum[p] = Floats<V>(0.f);
        }
        for (int k0 = from; k0 < to && row_of_entry[k0 + 1] == tile_end_row; k0 += kAhead) {
            Gradient v[kAhead][NP];
            uint32_t at[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                at[u] = position[k0 + u < to ? k0 + u : from];
                load_grad(at[u], v[u]);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (k0 + u < to && row_of_entry[k0 + u + 1] == tile_end_row) add(v[u], at[u]);
        }
        for (int d = a.lanes; d < kWave; d <<= 1)
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[p][e] += __shfl_xor(sum[p][e], d);
        __syncthreads();                         // (the chains have been read)
        if (place == 0) {
#pragma unroll
            for (int p = 0; p < NP; ++p) shares[p][threadIdx.x] = sum[p];
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) sum[p] = kept[p];
        __syncthreads();
        if (unfinished || head_goes_on) {
#pragma unroll 2
            for (int w = 0; w < kWaves; ++w)
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const Floats<V> x = shares[p][w * kWave + lane];
                    if (unfinished) sum[p] += x;
                    else chain[p] += x;
                }
        }
        if (unfinished) emit_tail();
        unfinished = false;
    }
    // Shares go to memory by way of LDS, so that neighbouring lanes store neighbouring elements (past the L2s every store is a
    // transaction of its own).  They are there before the counter says so, and the last workgroup of a run reads them behind it.
    const bool head_share = begins_inside && !finished && row_of_entry[1] != a.num_rows;
    const bool tail_share = long_run && !(begins_inside && tile_end_row == row_of_entry[1]);
    if (!head_share && !tail_share) return;
    const int32_t col_first = block_col * NP * V * a.lanes;
    const int32_t columns = NP * V * a.lanes < a.dim - col_first ? NP * V * a.lanes : a.dim - col_first;
    float *const part = reinterpret_cast<float *>(&shares[0][0]);        // (room for eight groups' sums)
    __syncthreads();
    auto keep = [&](float *to, const Floats<V> (&v)[NP]) {
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (column[p] < a.dim && column[p] + e >= piece_of(p)) to[column[p] + e - col_first] = v[p][e];
    };
    if (unfinished) {
        keep(part, sum);
        // by the workgroup of every block of columns, the same value: arrivals are counted for each block by itself, so the last one
        // of a block sees what its own owner stored before it arrived, and nothing of another block's
        if (lane == 0) store_shared(a.tail_index + tile_index, index - 1);
    }
    if (has_head) keep(part + NP * V * a.lanes, chain);
    __syncthreads();
    for (int32_t c = threadIdx.x; c < columns; c += kReduceBlock) {
        if (tail_share) store_shared(a.tail + (int64_t)tile_index * a.dim + col_first + c, part[c]);
        if (head_share) store_shared(a.head + (int64_t)tile_index * a.dim + col_first + c, part[NP * V * a.lanes + c]);
    }
    // (meanwhile) the tile in which a run begins, and the last one that it goes into by more than kBehind entries: most of them are
    // among the 63 tiles on either side, at which a wavefront looks at once
    auto extent = [&](bool head, uint32_t row, int32_t &owner, int32_t &last) {
        const auto begin_row = [&](int32_t t) { return row_at(a.entries, (int64_t)t * a.tile); };
        const auto behind_row = [&](int32_t t) {
            const int64_t i = (int64_t)t * a.tile + kBehind;
            return i < a.n ? row_at(a.entries, i) : kNoRow;
        };
        const int32_t before = tile_index - lane_id(), after = tile_index + lane_id();
        const bool inside = head && before > 0 && begin_row(before) == row && row_at(a.entries, (int64_t)before * a.tile - 1) == row;
        const bool goes_into = after < a.tiles && behind_row(after) <= row;
        const uint64_t runs_into = __ballot(inside), reaches = __ballot(goes_into);
        owner = tile_index - (int32_t)__popcll(runs_into);
        if (~runs_into == 0) {
            owner = wave_search<false>(a.tiles, row, begin_row);
            if (owner > 0 && row_at(a.entries, (int64_t)owner * a.tile - 1) == row) --owner;       // (it begins at a tile's begin, or inside one)
        }
        last = tile_index + (int32_t)__popcll(reaches) - 1;
        if (~reaches == 0) last = wave_search<true>(a.tiles, row, behind_row) - 1;
    };
    int32_t head_owner = 0, head_last = 0, tail_owner = 0, tail_last = 0;
    if (head_share) extent(true, row_of_entry[1], head_owner, head_last);
    if (tail_share) extent(false, tile_end_row, tail_owner, tail_last);
    wait_for_stores();
    __syncthreads();
    for (int which = 0; which < 2; ++which) {
        const bool head = which == 0;
        if (!(head ? head_share : tail_share)) continue;
        const uint32_t row = head ? row_of_entry[1] : tile_end_row;
        const int32_t owner = head ? head_owner : tail_owner, last = head ? head_last : tail_last;
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t *counter = a.arrived + (int64_t)owner * a.col_blocks + block_col;
            const bool is_last = atomicAdd(counter, 1u) == (uint32_t)(last - owner);
            if (is_last) store_shared(counter, 0u);
            joins = is_last;
        }
        __syncthreads();
        if (!joins) continue;
        join_run<STEP>(a, join_part, row, owner, last, col_first, col_first + columns);
        __syncthreads();
    }
}

template <typename TG, int WB>
mpzch_status_t launch_reduce(const ReduceArgs &a, int width, int pieces, int grid, hipStream_t s)
{
    switch (width) {
    case 8:
        if constexpr (sizeof(TG) == 2)
            return pieces == 1 ? launch(k_reduce<TG, 8, 1, WB>, grid, kReduceBlock, s, a) : launch(k_reduce<TG, 8, 2, WB>, grid, kReduceBlock, s, a);
        return MPZCH_ERR_UNSUPPORTED;
    case 4:
        if constexpr (sizeof(TG) == 4)           // (16 bits: rows of four to seven elements)
            if (pieces != 1) return launch(k_reduce<TG, 4, 4, WB>, grid, kReduceBlock, s, a);
        return launch(k_reduce<TG, 4, 1, WB>, grid, kReduceBlock, s, a);
    case 2: return launch(k_reduce<TG, 2, 1, WB>, grid, kReduceBlock, s, a);       // (rows of three elements, or two)
    default: return launch(k_reduce<TG, 1, 1, WB>, grid, kReduceBlock, s, a);
    }
}
template <int WB>
mpzch_status_t launch_reduce(const ReduceArgs &a, int32_t grad_type, int width, int pieces, int grid, hipStream_t s)
{
    switch (grad_type) {
    case MPZCH_F32: return launch_reduce<float, WB>(a, width, pieces, grid, s);
    case MPZCH_BF16: return launch_reduce<__bf16, WB>(a, width, pieces, grid, s);
    default: return launch_reduce<_Float16, WB>(a, width, pieces, grid, s);
    }
}

}  // namespace

#define MPZCH_DEFINE(bytes) MPZCH_LAUNCH_REDUCE(bytes) { return launch_reduce<bytes>(a, grad_type, width, pieces, grid, s); }
#define MPZCH_DEFINE_FOR(bytes) MPZCH_DEFINE(bytes)
MPZCH_DEFINE_FOR(MPZCH_TABLE_BYTES)

}  // namespace mpzch
