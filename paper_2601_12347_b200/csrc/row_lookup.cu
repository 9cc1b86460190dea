// Rows looked up by id, and the gradient of the table they came from:
//   out_i = scale table[ids_i],      dtable[r] = scale * sum of dy_i over the i with ids_i = r, in the order of i.
// The gradient sorts (id, i) by id and sums runs of one id.  Every 32 places of the sorted list are a warp's, however the ids are
// distributed: a run that lies within them is finished there; what a run has in them that goes on beyond is a partial sum.  The partial sums of a
// block's eight warps are such a list again, for one of its warps, and those of all blocks, a 128th as many as entries, for the same kernel.
// No atomics on sums, so every call gives the same bits.
//
// What bounds it.  300 007 rows of 256 bf16, 50 000 of them in the table, some named by thousands: lookup 34 us (154 MB written, 4.5 TB/s), the sort 43 (two passes of
// three launches of 4 to 10 us: latency), rows 44 (154 MB gathered in pieces of 512 bytes, 3.5 TB/s), lists 19.  20 011 fp32 rows of 602 into a table of 232 965: zeros beside
// the sort 101 us (561 MB, 5.6 TB/s), lookup 25 and rows 24 (rows that 16 bytes do not divide).
#include "row_vectors.cuh"

#include <algorithm>
#include <cstring>
#include <utility>

namespace rp {

// ---- lookup --------------------------------------------------------------------------------------------------------
struct LookupParams {
    int rows, width, lanes;      // lanes: threads of a row, a power of two
    const void* table;
    int64_t ld_table, table_rows;
    const int32_t* ids;
    void* out;
    int64_t ld_out;
    float scale;
    uint32_t scale_pair;         // LK_PAIRS: the scale in the rows' type, twice
};

constexpr int LK_BLOCK = 256;

constexpr int LK_ROWS = 4;       // rows of a thread that are on their way together

// How rows are scaled.  LK_COPY: not at all.  LK_PAIRS: 16-bit rows by a scale of their own type, two elements per instruction, whose product is rounded
// once.  LK_FLOAT: by way of fp32, rounded there and to the result's type.  (300 007 rows of 256 bf16: 48 us by way of fp32, 34 in pairs.)
enum { LK_FLOAT, LK_PAIRS, LK_COPY };

template <typename T> __device__ __forceinline__ uint32_t times_pair(uint32_t a, uint32_t b) {
    uint32_t d;
    if constexpr (std::is_same<T, __half>::value) asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

template <typename T, typename TO, int V, int HOW>
__global__ void __launch_bounds__(LK_BLOCK) k_lookup_rows(const __grid_constant__ LookupParams p) {
    pdl_enter();
    const int t = threadIdx.x & (p.lanes - 1), per_block = LK_BLOCK / p.lanes;
    for (int64_t row0 = (int64_t)blockIdx.x * per_block * LK_ROWS + threadIdx.x / p.lanes; row0 < p.rows; row0 += (int64_t)gridDim.x * per_block * LK_ROWS) {
        int id[LK_ROWS];
        const T* from[LK_ROWS];
        bool real[LK_ROWS], in[LK_ROWS];
#pragma unroll
        for (int u = 0; u < LK_ROWS; ++u) in[u] = row0 + u * per_block < p.rows, id[u] = in[u] ? p.ids[row0 + u * per_block] : -1;
#pragma unroll
        for (int u = 0; u < LK_ROWS; ++u) {
            real[u] = id[u] >= 0 && id[u] < p.table_rows;
            from[u] = static_cast<const T*>(p.table) + max(id[u], 0) * p.ld_table;
        }
        TO* const to = static_cast<TO*>(p.out) + row0 * p.ld_out;
        for (int c = t * V; c < p.width; c += p.lanes * V) {
            Piece<T, V> v[LK_ROWS];
#pragma unroll
            for (int u = 0; u < LK_ROWS; ++u) {
#pragma unroll
                for (int e = 0; e < V; ++e) v[u].v[e] = from_f32<T>(0.f);
                if (real[u]) v[u] = *reinterpret_cast<const Piece<T, V>*>(from[u] + c);
            }
#pragma unroll
            for (int u = 0; u < LK_ROWS; ++u) {
                if (!in[u]) continue;
                Piece<TO, V> y;
                if constexpr (HOW == LK_PAIRS) {
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) reinterpret_cast<uint32_t*>(&y)[e] = real[u] ? times_pair<T>(reinterpret_cast<const uint32_t*>(&v[u])[e], p.scale_pair) : 0u;
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        if constexpr (HOW == LK_COPY && std::is_same<T, TO>::value) y.v[e] = v[u].v[e];
                        else y.v[e] = from_f32<TO>(real[u] ? to_f32(v[u].v[e]) * p.scale : 0.f);      // (zeros stay zeros whatever the scale)
                    }
                }
                *reinterpret_cast<Piece<TO, V>*>(to + u * per_block * p.ld_out + c) = y;
            }
        }
    }
}

template <typename T, typename TO, int V, int HOW>
static cudaError_t launch_lookup(LookupParams p, void* stream) {
    p.lanes = 1;
    while (p.lanes < LK_BLOCK && p.lanes * V < p.width) p.lanes *= 2;
    const int64_t blocks = ((int64_t)p.rows * p.lanes + LK_BLOCK * LK_ROWS - 1) / (LK_BLOCK * LK_ROWS);
    return launch(k_lookup_rows<T, TO, V, HOW>, dim3((unsigned)std::min<int64_t>(blocks, (int64_t)sm_count() * 32)), LK_BLOCK, 0, stream, p);
}
template <typename T, typename TO, int V>
static cudaError_t launch_lookup(LookupParams p, void* stream) {
    if constexpr (std::is_same<T, TO>::value) {
        if (p.scale == 1.f) return launch_lookup<T, TO, V, LK_COPY>(p, stream);
        if constexpr (sizeof(T) == 2 && V > 1) {
            const T s = std::is_same<T, __half>::value ? T(__float2half_rn(p.scale)) : T(__float2bfloat16_rn(p.scale));
            uint16_t bits;
            std::memcpy(&bits, &s, 2);
            if ((float)s == p.scale) {
                p.scale_pair = (uint32_t)bits << 16 | bits;
                return launch_lookup<T, TO, V, LK_PAIRS>(p, stream);
            }
        }
    }
    return launch_lookup<T, TO, V, LK_FLOAT>(p, stream);
}

template <typename T, typename TO>
static cudaError_t launch_lookup(const LookupParams& p, int v, void* stream) {
    constexpr int WIDE = 16 / sizeof(T);
    if (v >= WIDE) return launch_lookup<T, TO, WIDE>(p, stream);
    if (v >= 2) return launch_lookup<T, TO, 2>(p, stream);
    return launch_lookup<T, TO, 1>(p, stream);
}

// ---- rows of a step ----------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(LK_BLOCK) k_live_rows(const __grid_constant__ ripple_live_rows_args p) {
    pdl_enter();
    for (int64_t i = (int64_t)blockIdx.x * LK_BLOCK + threadIdx.x; i < p.rows; i += (int64_t)gridDim.x * LK_BLOCK) {
        const int id = p.ids[i], label = p.labels[i];
        const bool live = id >= 0 && id < p.table_rows && label >= 0 && label < p.classes;
        if (p.live_ids) p.live_ids[i] = live ? id : -1;
        if (p.live_rows) p.live_rows[i] = live ? (int)i : -1;
        if (p.live_labels) p.live_labels[i] = live ? label : -1;
    }
}

// ---- zeros ---------------------------------------------------------------------------------------------------------
// The gradient's table is mostly zeros where ids are few; they are written by blocks behind those of the kernels that sort, which by themselves
// would leave the memory idle (20 011 ids of a table of 232 965 rows, 602 fp32 columns: 272 us for lookup and gradient with the zeros first, 152 so).
struct ZeroParams {
    uint8_t* at;
    int64_t units, row_bytes, pitch;       // rows; a table without gaps counts as rows of ZERO_PIECE bytes, the last one shorter
    int64_t last_bytes;
};
constexpr int64_t ZERO_PIECE = 32 * 1024;

static ZeroParams zeros_of(void* p, int64_t rows, int64_t width, int64_t ld, int size) {
    if (rows == 0) return {};
    if (ld > width) return {static_cast<uint8_t*>(p), rows, width * size, ld * size, width * size};
    const int64_t bytes = rows * width * size, units = (bytes + ZERO_PIECE - 1) / ZERO_PIECE;
    return {static_cast<uint8_t*>(p), units, ZERO_PIECE, ZERO_PIECE, bytes - (units - 1) * ZERO_PIECE};
}
// share `part` of `parts`
static ZeroParams share_of(const ZeroParams& z, int part, int parts) {
    const int64_t first = z.units * part / parts, end = z.units * (part + 1) / parts;
    return {z.at + first * z.pitch, end - first, z.row_bytes, z.pitch, end == z.units ? z.last_bytes : z.row_bytes};
}
__device__ __forceinline__ void write_zeros(const ZeroParams& z, int block, int blocks) {
    for (int64_t u = block; u < z.units; u += blocks) {
        uint8_t* const begin = z.at + u * z.pitch;
        uint8_t* const end = begin + (u == z.units - 1 ? z.last_bytes : z.row_bytes);
        uint8_t* const from = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(begin) + 15) & ~(uintptr_t)15);
        uint8_t* const to = reinterpret_cast<uint8_t*>(reinterpret_cast<uintptr_t>(end) & ~(uintptr_t)15);
        if (from >= to) {                  // (elements have 2 bytes at least, and lie at multiples of 2)
            for (uint8_t* p = begin + 2 * threadIdx.x; p < end; p += 2 * blockDim.x) *reinterpret_cast<uint16_t*>(p) = 0;
            continue;
        }
        if (begin + 2 * threadIdx.x < from) *reinterpret_cast<uint16_t*>(begin + 2 * threadIdx.x) = 0;
        if (to + 2 * threadIdx.x < end) *reinterpret_cast<uint16_t*>(to + 2 * threadIdx.x) = 0;
#pragma unroll 4
        for (uint8_t* p = from + 16 * threadIdx.x; p < to; p += 16 * blockDim.x) *reinterpret_cast<uint4*>(p) = make_uint4(0, 0, 0, 0);
    }
}
__global__ void __launch_bounds__(256) k_zeros(const __grid_constant__ ZeroParams z) {
    pdl_enter();
    write_zeros(z, blockIdx.x, gridDim.x);
}
constexpr int ZERO_BLOCKS = 8;             // per SM

// ---- (id, place) in the order of ids -----------------------------------------------------------------------------------
// From the lowest digit up; a pass counts the digits of every tile, adds the counts up, and moves the entries; entries of one digit
// stay in order.  Ids outside the table become `table_rows` and come last.
constexpr int SR_WARPS = 8, SR_BITS = 11;
// Entries of a tile: few where that gives every SM a tile or two at most, for a tile takes as long as its warps have rounds.
constexpr int SR_TILE_FINE = 1024, SR_TILE = 4096, SR_FINE = 1 << 19;
constexpr int SR_SMALL = 4096, SR_SMALL_BITS = 8;      // entries that one block sorts in shared memory, digits of 8 bits

struct SortParams {
    int n, tile, tiles;          // entries of a tile
    ZeroParams zeros;            // for the blocks behind those that sort
    int shift, digits;           // of this pass
    uint32_t table_rows;
    const int32_t* ids;          // first pass; else null
    const uint32_t* keys;
    const int32_t* places;
    uint32_t* keys_out;
    int32_t* places_out;
    int32_t* counts;             // digits x tiles, then their exclusive sums along the tiles
    int32_t* totals;             // digits
};

__device__ __forceinline__ uint32_t key_of(int id, uint32_t table_rows) { return min((uint32_t)id, table_rows); }    // (negative ids are large)
__device__ __forceinline__ uint32_t sort_key(const SortParams& p, int i) { return p.ids ? key_of(p.ids[i], p.table_rows) : p.keys[i]; }

__global__ void __launch_bounds__(32 * SR_WARPS) k_sort_count(const __grid_constant__ SortParams p) {
    pdl_enter();
    if ((int)blockIdx.x >= p.tiles) return write_zeros(p.zeros, blockIdx.x - p.tiles, gridDim.x - p.tiles);
    __shared__ int32_t count[1 << SR_BITS];
    for (int d = threadIdx.x; d < p.digits; d += blockDim.x) count[d] = 0;
    __syncthreads();
    const int first = blockIdx.x * p.tile;
#pragma unroll 4
    for (int e = threadIdx.x; e < p.tile; e += blockDim.x) {
        const int i = first + e;
        const bool in = i < p.n;
        const int d = in ? (int)(sort_key(p, i) >> p.shift & (uint32_t)(p.digits - 1)) : -1;
        // (equal digits of a warp at once: popular ids would queue up at one place)
        const uint32_t same = __match_any_sync(FULL, d);
        if (in && (same & ((1u << lane_id()) - 1)) == 0) atomicAdd(&count[d], __popc(same));
    }
    __syncthreads();
    for (int d = threadIdx.x; d < p.digits; d += blockDim.x) p.counts[(int64_t)d * p.tiles + blockIdx.x] = count[d];
}

// a warp per digit
__global__ void __launch_bounds__(256) k_sort_scan(const __grid_constant__ SortParams p) {
    pdl_enter();
    const int blocks = (p.digits + 7) / 8;
    if ((int)blockIdx.x >= blocks) return write_zeros(p.zeros, blockIdx.x - blocks, gridDim.x - blocks);
    const int d = blockIdx.x * 8 + (threadIdx.x >> 5), lane = lane_id();
    if (d >= p.digits) return;
    int32_t* const row = p.counts + (int64_t)d * p.tiles;
    int sum = 0;
    for (int t = 0; t < p.tiles; t += 32) {
        const int v = t + lane < p.tiles ? row[t + lane] : 0, up_to = warp_inclusive_scan(v);
        if (t + lane < p.tiles) row[t + lane] = sum + up_to - v;
        sum += __shfl_sync(FULL, up_to, 31);
    }
    if (lane == 0) p.totals[d] = sum;
}

// Places of a tile's entries, warp by warp in contiguous parts: at[warp][digit] is where the warp's next entry of that digit goes.
// entry(e): the digit of the tile's entry e, negative beyond its end; move(e, to): its new place.
template <int WARPS, typename E, typename M, typename B>
__device__ __forceinline__ void move_tile(int32_t* at, int digits, int entries, E entry, M move, B base) {
    const int warp = threadIdx.x >> 5, lane = lane_id();
    const int part = (entries + 32 * WARPS - 1) / (32 * WARPS) * 32, begin = warp * part;
    for (int d = threadIdx.x; d < digits * WARPS; d += 32 * WARPS) at[d] = 0;
    __syncthreads();
    const uint32_t before = (1u << lane) - 1;
    for (int e = begin; e < begin + part; e += 32) {
        const int d = entry(e + lane);
        const uint32_t same = __match_any_sync(FULL, d);
        if (d >= 0 && (same & before) == 0) at[warp * digits + d] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    base();                      // counts of the warps become places: at[w][d] = start of d + entries of the warps before
    __syncthreads();
    for (int e = begin; e < begin + part; e += 32) {
        const int d = entry(e + lane);
        const uint32_t same = __match_any_sync(FULL, d);
        const int start = d >= 0 ? at[warp * digits + d] : 0;
        __syncwarp();
        if (d >= 0) {
            move(e + lane, start + __popc(same & before));
            if ((same & before) == 0) at[warp * digits + d] = start + __popc(same);
        }
        __syncwarp();
    }
    __syncthreads();
}

// ROUNDS: 32 entries each, of a warp.  A warp counts its entries of every digit, and with that knows each one's rank among its own; the counts of the
// warps before, of the tiles before and of the digits before are added.
template <int ROUNDS>
__global__ void __launch_bounds__(32 * SR_WARPS) k_sort_move(const __grid_constant__ SortParams p) {
    pdl_enter();
    if ((int)blockIdx.x >= p.tiles) return write_zeros(p.zeros, blockIdx.x - p.tiles, gridDim.x - p.tiles);
    extern __shared__ int32_t at[];            // warps x digits, and behind them the digits' starts
    __shared__ int32_t scratch[33];
    int32_t* const start = at + SR_WARPS * p.digits;
    const int warp = threadIdx.x >> 5, lane = lane_id(), first = blockIdx.x * p.tile + warp * (32 * ROUNDS);
    uint32_t key[ROUNDS];
    int32_t place[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = first + 32 * r + lane;
        key[r] = i < p.n ? sort_key(p, i) : 0xffffffffu, place[r] = p.ids || i >= p.n ? i : p.places[i];
    }
    for (int d = threadIdx.x; d < p.digits * SR_WARPS; d += blockDim.x) at[d] = 0;
    // starts of the digits: sums of the totals before them
    const int per = (p.digits + blockDim.x - 1) / blockDim.x, d0 = threadIdx.x * per;
    int mine = 0, all;
    for (int d = d0; d < min(d0 + per, p.digits); ++d) mine += p.totals[d];
    int sum = block_exclusive_scan(mine, scratch, all);          // (and a barrier behind the zeros)
    for (int d = d0; d < min(d0 + per, p.digits); ++d) {
        start[d] = sum + p.counts[(int64_t)d * p.tiles + blockIdx.x];
        sum += p.totals[d];
    }
    int32_t* const own = at + warp * p.digits;
    const uint32_t before = (1u << lane) - 1;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const bool in = first + 32 * r + lane < p.n;
        const int d = in ? (int)(key[r] >> p.shift & (uint32_t)(p.digits - 1)) : -1;
        const uint32_t same = __match_any_sync(FULL, d);
        const int had = in ? own[d] : 0;
        __syncwarp();
        rank[r] = had + __popc(same & before);
        if (in && (same & before) == 0) own[d] = had + __popc(same);
        __syncwarp();
    }
    __syncthreads();
    for (int d = threadIdx.x; d < p.digits; d += blockDim.x) {
        int sum = start[d];
        for (int w = 0; w < SR_WARPS; ++w) {
            const int c = at[w * p.digits + d];
            at[w * p.digits + d] = sum;
            sum += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        if (first + 32 * r + lane >= p.n) continue;
        const int to = own[key[r] >> p.shift & (uint32_t)(p.digits - 1)] + rank[r];
        p.keys_out[to] = key[r], p.places_out[to] = place[r];
    }
}

// All passes of up to SR_SMALL entries by one block.
constexpr int SS_WARPS = 16;
struct SmallSort {
    uint32_t key[2][SR_SMALL];
    uint16_t place[2][SR_SMALL];
    int32_t at[SS_WARPS << SR_SMALL_BITS];
    int32_t scratch[33];
};
__global__ void __launch_bounds__(32 * SS_WARPS) k_sort_small(const __grid_constant__ SortParams p, int bits) {
    pdl_enter();
    if (blockIdx.x > 0) return write_zeros(p.zeros, blockIdx.x - 1, gridDim.x - 1);
    extern __shared__ __align__(16) uint8_t raw[];
    SmallSort& s = *reinterpret_cast<SmallSort*>(raw);
    constexpr int DIGITS = 1 << SR_SMALL_BITS;
    for (int i = threadIdx.x; i < p.n; i += blockDim.x) s.key[0][i] = key_of(p.ids[i], p.table_rows), s.place[0][i] = (uint16_t)i;
    __syncthreads();
    int b = 0;
    for (int shift = 0; shift < bits; shift += SR_SMALL_BITS, b ^= 1) {
        auto entry = [&](int e) { return e < p.n ? (int)(s.key[b][e] >> shift & (DIGITS - 1)) : -1; };
        auto move = [&](int e, int to) { s.key[b ^ 1][to] = s.key[b][e], s.place[b ^ 1][to] = s.place[b][e]; };
        auto base = [&]() {
            const int d = threadIdx.x;
            int mine = 0, all;
            if (d < DIGITS) for (int w = 0; w < SS_WARPS; ++w) mine += s.at[w * DIGITS + d];
            int sum = block_exclusive_scan(mine, s.scratch, all);
            if (d < DIGITS) {
                for (int w = 0; w < SS_WARPS; ++w) {
                    const int c = s.at[w * DIGITS + d];
                    s.at[w * DIGITS + d] = sum;
                    sum += c;
                }
            }
        };
        move_tile<SS_WARPS>(s.at, DIGITS, p.n, entry, move, base);
    }
    for (int i = threadIdx.x; i < p.n; i += blockDim.x) p.keys_out[i] = s.key[b][i], p.places_out[i] = s.place[b][i];
}
static_assert(32 * SS_WARPS >= 1 << SR_SMALL_BITS, "a thread per digit");

// ---- sums of runs --------------------------------------------------------------------------------------------------
// An entry of a list of partial sums: the key, with EMPTY where the run only goes on through this place.
constexpr uint32_t EMPTY = 0x80000000u, NO_KEY = 0xffffffffu;

struct RunParams {
    int n, width, slices;        // entries; parts of the columns, a block each
    uint32_t table_rows;
    const uint32_t* keys;        // n, ascending (without EMPTY), NO_KEY anywhere
    const int32_t* places;       // row of src of every entry; null: the entry's own
    const void* src;
    int64_t ld_src;
    uint32_t* next_keys;         // two for every block's entries: partial sums of runs that go on beyond them
    float* next;
    int ld_next;
    void* out;
    int64_t ld_out;
    float scale;
    int accumulate;
};

constexpr int RS_WARPS = 8, RS_CHUNK = 32 * RS_WARPS;      // entries of a block, 32 of a warp

__device__ __forceinline__ uint32_t bare(uint32_t key) { return key & ~EMPTY; }

// V neighbouring elements as they lie in memory, 32 bits at a time: as elements the compiler would widen all of them as soon as they are there, into
// registers that there are not (300 007 rows of 256 bf16: 121 us in place of 58).
template <typename T, int V> struct Raw {
    static constexpr int WORDS = V * (int)sizeof(T) < 4 ? 1 : V * (int)sizeof(T) / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void read(const T* from) {
        if constexpr (V * sizeof(T) == 2) w[0] = *reinterpret_cast<const uint16_t*>(from);
        else *reinterpret_cast<Piece<uint32_t, WORDS>*>(w) = *reinterpret_cast<const Piece<uint32_t, WORDS>*>(from);
    }
    __device__ __forceinline__ float at(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
        else return __half2float(__ushort_as_half((unsigned short)(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu)));
    }
};

// Runs of the same key among entries in order.  begin(k): the next run; add(piece): an entry of it; finish: the last one.  A run that lies within the entries is `complete`, the
// one that comes from before them and the one that goes on behind them are partial sums.
template <typename TO, int V, int NP>
struct Runs {
    const RunParams& p;
    const int c0;                // this lane's columns: c0 + 32 V j
    float* head;                 // where this lane's part of the partial sums goes
    float* tail;
    uint32_t run, head_key = NO_KEY, tail_key = NO_KEY;
    bool from_before;
    float sum[NP][V];
    __device__ __forceinline__ Runs(const RunParams& p_, int c, uint32_t first, uint32_t before, float* h, float* t) : p(p_), c0(c), head(h), tail(t), run(bare(first)), from_before(bare(first) == before) { clear(); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < NP; ++j) {
#pragma unroll
            for (int e = 0; e < V; ++e) sum[j][e] = 0.f;
        }
    }
    template <typename F> __device__ __forceinline__ void each(F f) {
#pragma unroll
        for (int j = 0; j < NP; ++j) if (c0 + j * 32 * V < p.width) f(j, j * 32 * V);
    }
    __device__ __forceinline__ void finish(bool goes_on) {
        if (run < p.table_rows) {
            if (from_before || goes_on) {
                float* const to = from_before ? head : tail;
                each([&](int j, int c) {
                    Piece<float, V> y;
#pragma unroll
                    for (int e = 0; e < V; ++e) y.v[e] = sum[j][e];
                    *reinterpret_cast<Piece<float, V>*>(to + c) = y;
                });
                if (from_before) head_key = run;
                if (goes_on) tail_key = from_before ? run | EMPTY : run;
            } else {
                TO* const to = static_cast<TO*>(p.out) + (int64_t)run * p.ld_out + c0;
                each([&](int j, int c) {
                    Piece<TO, V> y;
                    if (p.accumulate) y = *reinterpret_cast<const Piece<TO, V>*>(to + c);
#pragma unroll
                    for (int e = 0; e < V; ++e) y.v[e] = from_f32<TO>(sum[j][e] * p.scale + (p.accumulate ? to_f32(y.v[e]) : 0.f));
                    *reinterpret_cast<Piece<TO, V>*>(to + c) = y;
                });
            }
            clear();
        }
    }
    __device__ __forceinline__ void begin(uint32_t key) {
        finish(false);
        run = bare(key), from_before = false;
    }
    template <typename F> __device__ __forceinline__ void add(F piece) {
        each([&](int j, int) {
            const auto& v = piece(j);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[j][e] += v.at(e);
        });
    }
};

constexpr int RS_GROUPS = 2;       // of four rows of a warp, on their way at once
// Rows travel as asynchronous copies into places of shared memory that a lane alone reads: what is on its way takes no registers (300 007 rows of 256 bf16:
// four rows of a warp in registers 58 us, eight as copies 44; sixteen, which leave room for two blocks of an SM, 53).
template <typename T, int V> constexpr int rs_ring_bytes(int np) { return V * (int)sizeof(T) >= 16 ? RS_WARPS * 4 * RS_GROUPS * 32 * V * np * (int)sizeof(T) : 0; }
template <typename T, typename TO, int V, int NP>
__global__ void __launch_bounds__(32 * RS_WARPS) k_sum_runs(const __grid_constant__ RunParams p) {
    pdl_enter();
    constexpr bool RING = V * sizeof(T) >= 16;
    constexpr int COLS = 32 * V * NP;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ __align__(16) float part[2 * RS_WARPS][COLS];
    __shared__ uint32_t part_key[2 * RS_WARPS];
    const int warp = threadIdx.x >> 5, lane = lane_id(), block = blockIdx.x / p.slices, slice = blockIdx.x - block * p.slices;
    const int c0 = slice * COLS + lane * V, first = block * RS_CHUNK, last = min(p.n, first + RS_CHUNK);
    auto key_at = [&](int i) { return i >= 0 && i < p.n ? bare(p.keys[i]) : bare(NO_KEY); };
    uint32_t head_key = NO_KEY, tail_key = NO_KEY;
    const int begin = first + 32 * warp, count = min(32, last - begin);
    if (count > 0) {
        const uint32_t before = key_at(begin - 1), after = key_at(begin + count);
        const int i = begin + min(lane, count - 1);
        const uint32_t key = p.keys[i];
        const int place = p.places ? p.places[i] : i;
        Runs<TO, V, NP> runs(p, c0, __shfl_sync(FULL, key, 0), before, &part[2 * warp][lane * V], &part[2 * warp + 1][lane * V]);
        // where runs begin, and what is read (not: padding, EMPTY, nothing at all): a bit for every entry, so that an entry costs no comparison
        const uint32_t key_before = __shfl_up_sync(FULL, bare(key), 1);
        const uint32_t begins = __ballot_sync(FULL, lane > 0 && lane < count && bare(key) != key_before);
        const uint32_t reads = __ballot_sync(FULL, lane < count && key < p.table_rows);
        const T* const src = static_cast<const T*>(p.src) + c0;
        if constexpr (RING) {
            // four rows to a group of copies, RS_GROUPS groups on their way
            constexpr int ROW = COLS * (int)sizeof(T);
            uint8_t* const mine = ring + warp * (4 * RS_GROUPS * ROW) + lane * V * (int)sizeof(T);
            auto request = [&](int e0) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const T* const from = src + (int64_t)__shfl_sync(FULL, place, (e0 + u) & 31) * p.ld_src;
                    const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine + ((e0 + u) & (4 * RS_GROUPS - 1)) * ROW);
                    if (e0 < 32 && (reads >> ((e0 + u) & 31) & 1)) runs.each([&](int, int c) { copy_async<V * (int)sizeof(T)>(to + c * (int)sizeof(T), from + c); });
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
#pragma unroll
            for (int g = 0; g < RS_GROUPS; ++g) request(4 * g);
#pragma unroll 1
            for (int e0 = 0; e0 < count; e0 += 4) {
                asm volatile("cp.async.wait_group %0;" ::"n"(RS_GROUPS - 1) : "memory");
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (begins >> (e0 + u) & 1) runs.begin(__shfl_sync(FULL, key, e0 + u));
                    const T* const from = reinterpret_cast<const T*>(mine + ((e0 + u) & (4 * RS_GROUPS - 1)) * ROW);
                    if (reads >> (e0 + u) & 1) {
                        runs.add([&](int j) {
                            Raw<T, V> r;
                            r.read(from + j * 32 * V);
                            return r;
                        });
                    }
                }
                request(e0 + 4 * RS_GROUPS);
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        } else {
            // (narrower accesses through registers: 20 011 rows of 602 fp32, 24 us, as copies of 8 bytes 29)
            constexpr int AHEAD = 4;
            Raw<T, V> v[AHEAD][NP];
#pragma unroll 1
            for (int e0 = 0; e0 < count; e0 += AHEAD) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const T* const from = src + (int64_t)__shfl_sync(FULL, place, e0 + u) * p.ld_src;
                    if (reads >> (e0 + u) & 1) runs.each([&](int j, int c) { v[u][j].read(from + c); });
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (begins >> (e0 + u) & 1) runs.begin(__shfl_sync(FULL, key, e0 + u));
                    if (reads >> (e0 + u) & 1) runs.add([&](int j) -> const Raw<T, V>& { return v[u][j]; });
                }
            }
        }
        runs.finish(runs.run == after);
        head_key = runs.head_key, tail_key = runs.tail_key;
    }
    if (lane < 2) part_key[2 * warp + lane] = lane ? tail_key : head_key;
    const bool any = __syncthreads_or(head_key != NO_KEY || tail_key != NO_KEY);
    if (warp > 0) return;
    // the warps' partial sums, in the same way
    head_key = tail_key = NO_KEY;
    if (any) {
        const int64_t at = 2ll * block * p.ld_next + c0;
        Runs<TO, V, NP> runs(p, c0, part_key[0], key_at(first - 1), p.next + at, p.next + at + p.ld_next);
        for (int e = 0; e < 2 * RS_WARPS; ++e) {
            const uint32_t k = part_key[e];
            if (bare(k) != runs.run) runs.begin(k);
            if (k < p.table_rows) {
                runs.add([&](int j) {
                    Raw<float, V> r;
                    r.read(&part[e][lane * V + j * 32 * V]);
                    return r;
                });
            }
        }
        runs.finish(runs.run == key_at(last));
        head_key = runs.head_key, tail_key = runs.tail_key;
    }
    if (p.next_keys && slice == 0 && lane < 2) p.next_keys[2 * block + lane] = lane ? tail_key : head_key;
}

template <typename T, typename TO, int V, int NP>
static cudaError_t launch_runs(RunParams p, void* stream) {
    p.slices = (p.width + 32 * V * NP - 1) / (32 * V * NP);
    const int64_t blocks = (int64_t)((p.n + RS_CHUNK - 1) / RS_CHUNK) * p.slices;
    constexpr int bytes = rs_ring_bytes<T, V>(NP);
    static bool ready[64];
    const cudaError_t e = allow_shared(k_sum_runs<T, TO, V, NP>, bytes, ready);
    if (e != cudaSuccess) return e;
    return launch(k_sum_runs<T, TO, V, NP>, dim3((unsigned)blocks), 32 * RS_WARPS, bytes, stream, p);
}

// ---- few rows ------------------------------------------------------------------------------------------------------
// Up to FW_ROWS rows: a block for each.  The block of an id's first row finds the others and sums them; one launch in place of a sort.
constexpr int FW_ROWS = 256;
template <typename T, typename TO, int V>
__global__ void __launch_bounds__(FW_ROWS) k_lookup_grad_few(const __grid_constant__ RunParams p, const int32_t* ids) {
    pdl_enter();
    __shared__ int32_t rows[FW_ROWS];
    __shared__ int32_t before[FW_ROWS / 32 + 1];
    const int me = blockIdx.x, t = threadIdx.x, id = ids[me];
    if (id < 0 || (uint32_t)id >= p.table_rows) return;
    const bool same = t < p.n && ids[t] == id;
    if (__syncthreads_or(same && t < me)) return;
    // the rows of this id, in order
    const uint32_t all = __ballot_sync(FULL, same);
    if (lane_id() == 0) before[t >> 5] = __popc(all);
    __syncthreads();
    int count = 0, at = 0;
    for (int w = 0; w < FW_ROWS / 32; ++w) {
        if (w == t >> 5) at = count;
        count += before[w];
    }
    if (same) rows[at + __popc(all & ((1u << lane_id()) - 1))] = t;
    __syncthreads();
    const Vec<V> scale = all_of<V>(p.scale);
    TO* const to = static_cast<TO*>(p.out) + (int64_t)id * p.ld_out;
    for (int c = t * V; c < p.width; c += FW_ROWS * V) {
        Vec<V> sum = all_of<V>(0.f);
#pragma unroll 8
        for (int i = 0; i < count; ++i) plus<V>(sum, load<T, V>(static_cast<const T*>(p.src) + (int64_t)rows[i] * p.ld_src + c));
        times<V>(sum, scale);
        if (p.accumulate) plus<V>(sum, load<TO, V>(to + c));
        store<TO, V>(to + c, sum);
    }
}

// The same for a table that is small as well: a block for each row of it writes it, zeros included, and no other launch.
constexpr int64_t FW_TABLE = 4 << 20, FW_TABLE_ROWS = 8192;      // bytes; rows: four rounds of blocks, which for narrow rows are what it takes
template <typename T, typename TO, int V>
__global__ void __launch_bounds__(128) k_lookup_grad_table(const __grid_constant__ RunParams p, const int32_t* ids) {
    pdl_enter();
    __shared__ int32_t rows[FW_ROWS];
    __shared__ int32_t before[FW_ROWS / 32];
    const int t = threadIdx.x;
    uint32_t all[FW_ROWS / 128];
    bool same[FW_ROWS / 128];
#pragma unroll
    for (int h = 0; h < FW_ROWS / 128; ++h) {
        same[h] = t + 128 * h < p.n && ids[t + 128 * h] == (int)blockIdx.x;
        all[h] = __ballot_sync(FULL, same[h]);
        if (lane_id() == 0) before[(t + 128 * h) >> 5] = __popc(all[h]);
    }
    __syncthreads();
    int count = 0;
#pragma unroll
    for (int w = 0; w < FW_ROWS / 32; ++w) {
#pragma unroll
        for (int h = 0; h < FW_ROWS / 128; ++h)
            if (w == (t + 128 * h) >> 5 && same[h]) rows[count + __popc(all[h] & ((1u << lane_id()) - 1))] = t + 128 * h;
        count += before[w];
    }
    __syncthreads();
    if (count == 0 && p.accumulate) return;
    const Vec<V> scale = all_of<V>(p.scale);
    TO* const to = static_cast<TO*>(p.out) + blockIdx.x * p.ld_out;
    for (int c = t * V; c < p.width; c += 128 * V) {
        Vec<V> sum = all_of<V>(0.f);
#pragma unroll 8
        for (int i = 0; i < count; ++i) plus<V>(sum, load<T, V>(static_cast<const T*>(p.src) + (int64_t)rows[i] * p.ld_src + c));
        if (count > 0) times<V>(sum, scale);
        if (p.accumulate) plus<V>(sum, load<TO, V>(to + c));
        store<TO, V>(to + c, sum);
    }
}

// ---- the call ------------------------------------------------------------------------------------------------------
static int64_t up128(int64_t x) { return (x + 127) / 128 * 128; }

// What a call keeps where in its workspace (bytes).
struct GradPlan {
    int n, bits, tile, tiles, passes, digit_bits;
    int64_t keys[2], places[2], counts, totals;
    int levels;                  // lists of partial sums
    int64_t list_keys[12], list[12];
    int list_n[12], ld;
    int64_t bytes;
};
static GradPlan plan_grad(int64_t rows, int64_t table_rows, int width) {
    GradPlan g = {};
    g.n = (int)rows;
    if (rows <= FW_ROWS || table_rows == 0) return g;
    while (g.bits < 32 && (uint64_t)table_rows >> g.bits) ++g.bits;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up128(bytes);
        return here;
    };
    g.passes = (g.bits + SR_BITS - 1) / SR_BITS;
    g.digit_bits = (g.bits + g.passes - 1) / g.passes;
    g.tile = rows <= SR_FINE ? SR_TILE_FINE : SR_TILE;
    g.tiles = (int)((rows + g.tile - 1) / g.tile);
    const bool small = rows <= SR_SMALL;
    for (int b = 0; b < (small ? 1 : 2); ++b) g.keys[b] = take(rows * 4), g.places[b] = take(rows * 4);
    if (!small) g.counts = take(((int64_t)g.tiles << g.digit_bits) * 4), g.totals = take((int64_t)4 << g.digit_bits);
    g.ld = (width + 7) / 8 * 8;
    int64_t n = rows;
    while (n > RS_CHUNK) {
        n = (n + RS_CHUNK - 1) / RS_CHUNK * 2;
        g.list_n[g.levels] = (int)n;
        g.list_keys[g.levels] = take(n * 4);
        g.list[g.levels++] = take(n * g.ld * 4);
    }
    g.bytes = at;
    return g;
}

template <typename T, typename TO, int V>
static cudaError_t launch_lookup_grad(const ripple_lookup_rows_grad_args& a, void* stream) {
    const GradPlan g = plan_grad(a.rows, a.out_rows, a.width);
    cudaError_t e = cudaSuccess;
    RunParams r = {};
    r.n = g.n, r.width = a.width, r.table_rows = (uint32_t)a.out_rows, r.scale = a.scale, r.accumulate = a.accumulate;
    r.src = a.dy, r.ld_src = a.ld_dy, r.out = a.out, r.ld_out = a.ld_out;
    uint8_t* const work = static_cast<uint8_t*>(a.workspace);
    const ZeroParams zeros = a.accumulate ? ZeroParams{} : zeros_of(a.out, a.out_rows, a.width, a.ld_out, sizeof(TO));
    const unsigned zero_blocks = (unsigned)std::min<int64_t>(zeros.units, (int64_t)ZERO_BLOCKS * sm_count());
    if (a.rows <= FW_ROWS) {
        if (a.out_rows <= FW_TABLE_ROWS && a.out_rows * a.width * (int64_t)sizeof(TO) <= FW_TABLE)
            return launch(k_lookup_grad_table<T, TO, V>, dim3((unsigned)a.out_rows), 128, 0, stream, r, a.ids);
        if (zeros.units > 0) e = launch(k_zeros, dim3(zero_blocks), 256, 0, stream, zeros);
        if (e != cudaSuccess || a.rows == 0) return e;
        return launch(k_lookup_grad_few<T, TO, V>, dim3((unsigned)a.rows), FW_ROWS, 0, stream, r, a.ids);
    }
    SortParams s = {};
    s.n = g.n, s.tile = g.tile, s.tiles = g.tiles, s.table_rows = (uint32_t)a.out_rows, s.ids = a.ids;
    auto keys = [&](int b) { return reinterpret_cast<uint32_t*>(work + g.keys[b]); };
    auto places = [&](int b) { return reinterpret_cast<int32_t*>(work + g.places[b]); };
    int b = 0;                   // where the sorted list is
    if (a.rows <= SR_SMALL) {
        static bool ready[64];
        if ((e = allow_shared(k_sort_small, (int)sizeof(SmallSort), ready)) != cudaSuccess) return e;
        s.keys_out = keys(0), s.places_out = places(0), s.zeros = zeros;
        e = launch(k_sort_small, dim3(1 + zero_blocks), 32 * SS_WARPS, sizeof(SmallSort), stream, s, g.bits);
    } else {
        static bool ready[64], ready_fine[64];
        auto* const move = g.tile == SR_TILE ? k_sort_move<SR_TILE / (32 * SR_WARPS)> : k_sort_move<SR_TILE_FINE / (32 * SR_WARPS)>;
        if ((e = allow_shared(k_sort_move<SR_TILE / (32 * SR_WARPS)>, (SR_WARPS + 1) << (SR_BITS + 2), ready)) != cudaSuccess) return e;
        if ((e = allow_shared(k_sort_move<SR_TILE_FINE / (32 * SR_WARPS)>, (SR_WARPS + 1) << (SR_BITS + 2), ready_fine)) != cudaSuccess) return e;
        s.counts = reinterpret_cast<int32_t*>(work + g.counts), s.totals = reinterpret_cast<int32_t*>(work + g.totals);
        s.digits = 1 << g.digit_bits;
        int share = 0;
        auto next_share = [&]() { s.zeros = share_of(zeros, share, 3 * g.passes), ++share; };
        for (int pass = 0; pass < g.passes && e == cudaSuccess; ++pass) {
            s.shift = pass * g.digit_bits;
            if (pass > 0) s.ids = nullptr, s.keys = keys(b), s.places = places(b), b ^= 1;
            s.keys_out = keys(b), s.places_out = places(b);
            next_share();
            e = launch(k_sort_count, dim3((unsigned)g.tiles + zero_blocks), 32 * SR_WARPS, 0, stream, s);
            next_share();
            if (e == cudaSuccess) e = launch(k_sort_scan, dim3((unsigned)(s.digits + 7) / 8 + zero_blocks), 256, 0, stream, s);
            next_share();
            if (e == cudaSuccess) e = launch(move, dim3((unsigned)g.tiles + zero_blocks), 32 * SR_WARPS, (size_t)(SR_WARPS + 1) * s.digits * 4, stream, s);
        }
    }
    if (e != cudaSuccess) return e;
    r.keys = keys(b), r.places = places(b), r.ld_next = g.ld;
    for (int l = 0; l <= g.levels && e == cudaSuccess; ++l) {
        const bool more = l < g.levels;
        r.next_keys = more ? reinterpret_cast<uint32_t*>(work + g.list_keys[l]) : nullptr;
        r.next = more ? reinterpret_cast<float*>(work + g.list[l]) : nullptr;
        if (l == 0) e = launch_runs<T, TO, V, (V * (int)sizeof(T) == 16 ? 1 : 4 / V)>(r, stream);
        else e = launch_runs<float, TO, V, (V >= 4 ? 1 : 4 / V)>(r, stream);
        if (more) r.keys = r.next_keys, r.places = nullptr, r.src = r.next, r.ld_src = g.ld, r.n = g.list_n[l];
    }
    return e;
}

template <typename T, typename TO>
static cudaError_t launch_lookup_grad(const ripple_lookup_rows_grad_args& a, int v) {
    constexpr int WIDE = 16 / sizeof(T);
    if (v >= WIDE) return launch_lookup_grad<T, TO, WIDE>(a, a.cuda_stream);
    if (v >= 2) return launch_lookup_grad<T, TO, 2>(a, a.cuda_stream);
    return launch_lookup_grad<T, TO, 1>(a, a.cuda_stream);
}

// The widest access, up to 16 bytes of the first type, that matrices of `width` columns allow.
struct Access {
    int v;
    Access(int width, int size) : v(16 / size) { while (width % v) v >>= 1; }
    void fits(const void* ptr, int64_t ld, int size) {
        while (v > 1 && (ld % v || reinterpret_cast<uintptr_t>(ptr) % (v * size < 16 ? v * size : 16))) v >>= 1;
    }
};

}  // namespace rp

using namespace rp;

#define REFUSE(...)                      \
    do {                                 \
        note_error(WHAT ": " __VA_ARGS__); \
        return RIPPLE_ERR_INVALID_ARG;   \
    } while (0)

#define WHAT "lookup_rows"
extern "C" ripple_status ripple_lookup_rows(const ripple_lookup_rows_args* a) {
    if (!a) REFUSE("null arguments");
    if (a->rows < 0 || a->rows > INT32_MAX) REFUSE("rows out of range");
    if (a->width < 1 || a->width > 16384) REFUSE("width must be 1 to 16384");
    if (!type_ok(a->type) || !type_ok(a->out_type) || (a->out_type != a->type && a->type != RIPPLE_TYPE_F32))
        REFUSE("unknown type, or another type of out than a 16-bit table's");
    if (a->table_rows < 0) REFUSE("negative number of table rows");
    if (a->rows > 0 && ((!a->table && a->table_rows > 0) || !a->ids || !a->out)) REFUSE("null table, ids or out");
    if (a->ld_table < 0 || a->ld_out < a->width) REFUSE("leading dimension negative, or of out below its width");
    const int ts = type_size(a->type), os = type_size(a->out_type);
    for (auto [ptr, size] : {std::pair<const void*, int>{a->table, ts}, {a->out, os}, {a->ids, 4}})
        if (reinterpret_cast<uintptr_t>(ptr) % size) REFUSE("misaligned pointer");
    const Extent table{a->table, a->table_rows, a->ld_table, a->width, ts}, out{a->out, a->rows, a->ld_out, a->width, os}, ids{a->ids, a->rows, 1, 1, 4};
    if (extents_meet(out, table) || extents_meet(out, ids)) REFUSE("out overlaps an input");
    if (a->rows == 0) return RIPPLE_OK;
    Access v(a->width, ts);
    v.fits(a->table, a->ld_table, ts), v.fits(a->out, a->ld_out, os);
    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    LookupParams p = {};
    p.rows = (int)a->rows, p.width = a->width, p.table = a->table, p.ld_table = a->ld_table, p.table_rows = a->table_rows, p.ids = a->ids;
    p.out = a->out, p.ld_out = a->ld_out, p.scale = a->scale;
    cudaError_t e;
    switch (a->type * 4 + a->out_type) {
        case RIPPLE_TYPE_F32 * 4 + RIPPLE_TYPE_F32: e = launch_lookup<float, float>(p, v.v, a->cuda_stream); break;
        case RIPPLE_TYPE_F32 * 4 + RIPPLE_TYPE_BF16: e = launch_lookup<float, __nv_bfloat16>(p, v.v, a->cuda_stream); break;
        case RIPPLE_TYPE_F32 * 4 + RIPPLE_TYPE_F16: e = launch_lookup<float, __half>(p, v.v, a->cuda_stream); break;
        case RIPPLE_TYPE_BF16 * 4 + RIPPLE_TYPE_BF16: e = launch_lookup<__nv_bfloat16, __nv_bfloat16>(p, v.v, a->cuda_stream); break;
        default: e = launch_lookup<__half, __half>(p, v.v, a->cuda_stream); break;
    }
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("lookup_rows launch", e);
}
#undef WHAT

#define WHAT "live_rows"
extern "C" ripple_status ripple_live_rows(const ripple_live_rows_args* a) {
    if (!a) REFUSE("null arguments");
    if (a->rows < 0 || a->rows > INT32_MAX || a->table_rows < 0) REFUSE("rows or rows of the table out of range");
    if (a->classes < 1 || a->classes > RIPPLE_MAX_CLASSES) REFUSE("classes out of range");
    if (!a->live_ids && !a->live_rows && !a->live_labels) REFUSE("no output");
    if (a->rows > 0 && (!a->ids || !a->labels)) REFUSE("null ids or labels");
    const int32_t* const all[] = {a->ids, a->labels, a->live_ids, a->live_rows, a->live_labels};
    for (const int32_t* ptr : all)
        if (reinterpret_cast<uintptr_t>(ptr) % 4) REFUSE("misaligned pointer");
    for (int o = 2; o < 5; ++o)
        for (int i = 0; i < o; ++i)
            if (extents_meet({all[o], a->rows, 1, 1, 4}, {all[i], a->rows, 1, 1, 4})) REFUSE("an output overlaps another argument");
    if (a->rows == 0) return RIPPLE_OK;
    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    const int64_t blocks = std::min<int64_t>((a->rows + LK_BLOCK - 1) / LK_BLOCK, (int64_t)sm_count() * 8);
    const cudaError_t e = launch(k_live_rows, dim3((unsigned)blocks), LK_BLOCK, 0, a->cuda_stream, *a);
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("live_rows launch", e);
}
#undef WHAT

static bool lookup_grad_sizes_ok(const ripple_lookup_rows_grad_args* a) {
    return a->rows >= 0 && a->rows <= INT32_MAX - SR_TILE && a->width >= 1 && a->width <= 16384 && a->out_rows >= 0 && a->out_rows < INT32_MAX;
}

extern "C" int64_t ripple_lookup_rows_grad_workspace_bytes(const ripple_lookup_rows_grad_args* a) {
    return a && lookup_grad_sizes_ok(a) ? plan_grad(a->rows, a->out_rows, a->width).bytes : -1;
}

#define WHAT "lookup_rows_grad"
extern "C" ripple_status ripple_lookup_rows_grad(const ripple_lookup_rows_grad_args* a) {
    if (!a) REFUSE("null arguments");
    if (!lookup_grad_sizes_ok(a)) REFUSE("rows, width (1 to 16384) or rows of out out of range");
    if (!type_ok(a->type) || !type_ok(a->out_type) || (a->out_type != a->type && a->out_type != RIPPLE_TYPE_F32))
        REFUSE("unknown type, or a type of out that is neither dy's nor fp32");
    if (a->accumulate < 0 || a->accumulate > 1) REFUSE("accumulate must be 0 or 1");
    if ((a->rows > 0 && (!a->dy || !a->ids)) || (a->out_rows > 0 && !a->out)) REFUSE("null dy, ids or out");
    if (a->ld_dy < 0 || a->ld_out < a->width) REFUSE("leading dimension negative, or of out below its width");
    const int ts = type_size(a->type), os = type_size(a->out_type);
    for (auto [ptr, size] : {std::pair<const void*, int>{a->dy, ts}, {a->out, os}, {a->ids, 4}})
        if (reinterpret_cast<uintptr_t>(ptr) % size) REFUSE("misaligned pointer");
    const int64_t need = plan_grad(a->rows, a->out_rows, a->width).bytes;
    if (a->workspace_bytes < need || (need > 0 && !a->workspace)) REFUSE("workspace too small");
    if (reinterpret_cast<uintptr_t>(a->workspace) & 127) REFUSE("misaligned workspace");
    const Extent dy{a->dy, a->rows, a->ld_dy, a->width, ts}, out{a->out, a->out_rows, a->ld_out, a->width, os}, ids{a->ids, a->rows, 1, 1, 4},
        work{need > 0 ? a->workspace : nullptr, 1, 1, need, 1};
    for (const Extent* o : {&out, &work})
        for (const Extent* in : {&dy, &ids})
            if (extents_meet(*o, *in)) REFUSE("out or the workspace overlaps an input");
    if (extents_meet(out, work)) REFUSE("out overlaps the workspace");
    if (a->out_rows == 0) return RIPPLE_OK;
    Access v(a->width, ts);
    v.fits(a->dy, a->ld_dy, ts), v.fits(a->out, a->ld_out, os);
    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    cudaError_t e;
    const bool wide = a->out_type != a->type;
    switch (a->type) {
        case RIPPLE_TYPE_F32: e = launch_lookup_grad<float, float>(*a, v.v); break;
        case RIPPLE_TYPE_BF16: e = wide ? launch_lookup_grad<__nv_bfloat16, float>(*a, v.v) : launch_lookup_grad<__nv_bfloat16, __nv_bfloat16>(*a, v.v); break;
        default: e = wide ? launch_lookup_grad<__half, float>(*a, v.v) : launch_lookup_grad<__half, __half>(*a, v.v); break;
    }
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("lookup_rows_grad launch", e);
}
