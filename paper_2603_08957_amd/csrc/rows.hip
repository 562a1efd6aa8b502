// Rows of a table by token, and the table's gradient.
//
// A lookup is the join of a list of tokens with a table keyed by token,
//   out[t] = scale * E[id[t]],
// and its gradient the GROUP BY sum of the same join,
//   dE[v] = scale * sum over t with id[t] = v of g[t].
// Both move rows and compute next to nothing: memory bounds them.
#include "mx.h"
#include "tre_internal.h"

#include <type_traits>

namespace tre {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// A lane moves E consecutive elements of a row with one access of 16 bytes in
// the wider of the two types (eight where both sides have 16 bits, else four):
// with eight fp32 values, two stores of 16 bytes 32 apart, 65,536 rows of
// gradients took 25 us longer.  Rows of an odd number of elements begin
// anywhere; a wide access off its alignment still costs less than narrow ones.
template <typename TI, typename TO>
constexpr int lane_elems() { return sizeof(TI) == 4 || sizeof(TO) == 4 ? 4 : 8; }

typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_4 __attribute__((ext_vector_type(4), aligned(4)));

template <int E>
__device__ inline void load_all(const float* p, float (&v)[E]) {
#pragma unroll
    for (int h = 0; h < E; h += 4) {
        const f32x4_4 a = *reinterpret_cast<const f32x4_4*>(p + h);
#pragma unroll
        for (int i = 0; i < 4; i++) v[h + i] = a[i];
    }
}
template <int E>
__device__ inline void load_all(const uint16_t* p, float (&v)[E]) {
    uint32_t a[E / 2];
    if constexpr (E == 8) {
        const u32x4_2 x = *reinterpret_cast<const u32x4_2*>(p);
#pragma unroll
        for (int i = 0; i < 4; i++) a[i] = x[i];
    } else {
        const u32x2_2 x = *reinterpret_cast<const u32x2_2*>(p);
        a[0] = x[0];
        a[1] = x[1];
    }
#pragma unroll
    for (int i = 0; i < E / 2; i++) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}
// (ONCE: not kept in L2, where rows that are read again have their place)
template <bool ONCE, typename V>
__device__ inline void store_as(void* p, V v) {
    if constexpr (ONCE) __builtin_nontemporal_store(v, static_cast<V*>(p));
    else *static_cast<V*>(p) = v;
}
template <bool ONCE, int E>
__device__ inline void store_all(float* p, const float (&v)[E]) {
#pragma unroll
    for (int h = 0; h < E; h += 4) store_as<ONCE>(p + h, f32x4_4{v[h], v[h + 1], v[h + 2], v[h + 3]});
}
template <bool ONCE, int E>
__device__ inline void store_all(uint16_t* p, const float (&v)[E]) {
    uint32_t a[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; i++)
        a[i] = uint32_t(f32_to_bf16_rne(v[2 * i])) | (uint32_t(f32_to_bf16_rne(v[2 * i + 1])) << 16);
    if constexpr (E == 8) store_as<ONCE>(p, u32x4_2{a[0], a[1], a[2], a[3]});
    else store_as<ONCE>(p, u32x2_2{a[0], a[1]});
}
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
__device__ inline void store1(float* p, float v) { *p = v; }
__device__ inline void store1(uint16_t* p, float v) { *p = f32_to_bf16_rne(v); }

// The up to E elements of a row from element e on.
template <int E, typename T>
__device__ inline void load_run(const T* row, int64_t e, int64_t n, float (&v)[E]) {
    if (e + E <= n) {
        load_all(row + e, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < E; i++) v[i] = e + i < n ? load1(row + e + i) : 0.f;
}
template <bool ONCE = false, int E, typename T>
__device__ inline void store_run(T* row, int64_t e, int64_t n, const float (&v)[E]) {
    if (e + E <= n) {
        store_all<ONCE>(row + e, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < E; i++)
        if (e + i < n) store1(row + e + i, v[i]);
}

// Token t of a list of 4- or 8-byte integers.
__device__ inline int64_t token(const void* ids, int id_bytes, int64_t t) {
    return id_bytes == 8 ? static_cast<const int64_t*>(ids)[t] : int64_t(static_cast<const int32_t*>(ids)[t]);
}

// How threads lie on rows: `lanes` (a power of two, at most a wavefront) side by
// side on a row, each with some consecutive elements, `slices` such strips to a
// row; a row of few elements then shares its wavefront with others.
struct Strip {
    int32_t shift;   // lanes = 1 << shift
    int64_t slices;
};
Strip strip(int64_t elems, int per_lane) {
    Strip p{0, 1};
    while (p.shift < 6 && (int64_t(per_lane) << p.shift) < elems) p.shift++;
    const int64_t w = int64_t(per_lane) << p.shift;
    p.slices = (elems + w - 1) / w;
    return p;
}

// ----------------------------------------------------------------- lookup

struct LookupArgs {
    const void* table;
    const void* ids;
    void* out;
    int64_t* status;
    int64_t n_rows, elems, n_ids;
    int64_t groups;              // of kStrips strips or rows
    Strip strip;
    int64_t tile_rows, blocks;   // 4-bit tiles: rows of a tile, blocks of a row
    int64_t tile_bytes;
    float scale;
    int32_t id_bytes;
};

struct Mx4 {};

// Strips of a row (WIDE), or rows, that a thread has in flight together: a
// wavefront that moves one strip lives too short for its launch (131,072 rows
// of 4,096 bf16 values 406 us).
constexpr int kStrips = 4;

template <typename TI, int E>
__device__ inline void lookup_load(const LookupArgs& g, int64_t id, int64_t e, float (&v)[E]) {
    if constexpr (std::is_same_v<TI, Mx4>) {
        const int64_t tile = id / g.tile_rows;
        const uint8_t* at = static_cast<const uint8_t*>(g.table) + tile * g.tile_bytes;
        const uint32_t b = mx_block_of(uint32_t(g.tile_rows), mx_group(g.blocks), uint32_t(id - tile * g.tile_rows),
                                       uint32_t(e / kMxBlock));
        const uint8_t* codes = at + int64_t(b) * 16 + e % kMxBlock / 2;
        const int sb = at[g.tile_rows * g.blocks * 16 + b];
        if constexpr (E == 8) {
            mx_values(*reinterpret_cast<const uint32_t*>(codes), sb, v);
        } else {
            float w[8];
            mx_values(*reinterpret_cast<const uint16_t*>(codes), sb, w);
#pragma unroll
            for (int i = 0; i < E; i++) v[i] = w[i];
        }
    } else {
        load_run(static_cast<const TI*>(g.table) + id * g.elems, e, g.elems, v);
    }
}

template <typename TI, typename TO, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_lookup(LookupArgs g) {
    constexpr int E = lane_elems<TI, TO>();
    const int64_t x = block_index() * kThreads + threadIdx.x;
    const int lane = int(x & ((1 << g.strip.shift) - 1));
    int64_t t[kStrips], e[kStrips];
    float v[kStrips][E], scale[kStrips];  // 0 for no token: its row is zero under any scale
    if constexpr (WIDE) {
        // (a wavefront's row is the same for its lanes)
        const int64_t w = block_index() * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t row = w / g.groups, s0 = (w - row * g.groups) * kStrips;
        if (row >= g.n_ids) return;
        const int64_t id = token(g.ids, g.id_bytes, row);
        const bool in = id >= 0 && id < g.n_rows;
        if (g.status && id >= g.n_rows && s0 == 0 && lane == 0) *g.status = TRE_E_KEYRANGE;
#pragma unroll
        for (int i = 0; i < kStrips; i++) {
            t[i] = row;
            e[i] = ((s0 + i) * 64 + lane) * E;
            scale[i] = in ? g.scale : 0.f;
#pragma unroll
            for (int j = 0; j < E; j++) v[i][j] = 0.f;
            if (in && e[i] < g.elems) lookup_load<TI>(g, id, e[i], v[i]);
        }
    } else {
        int64_t id[kStrips];
        const int64_t r0 = (x >> g.strip.shift) * kStrips;
#pragma unroll
        for (int i = 0; i < kStrips; i++) {
            t[i] = r0 + i;
            e[i] = t[i] < g.n_ids ? lane * E : g.elems;
            id[i] = t[i] < g.n_ids ? token(g.ids, g.id_bytes, t[i]) : -1;
            if (g.status && id[i] >= g.n_rows && lane == 0) *g.status = TRE_E_KEYRANGE;
        }
#pragma unroll
        for (int i = 0; i < kStrips; i++) {
#pragma unroll
            for (int j = 0; j < E; j++) v[i][j] = 0.f;
            const bool in = id[i] >= 0 && id[i] < g.n_rows;
            scale[i] = in ? g.scale : 0.f;
            if (in && e[i] < g.elems) lookup_load<TI>(g, id[i], e[i], v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kStrips; i++) {
        if (e[i] >= g.elems) continue;
#pragma unroll
        for (int j = 0; j < E; j++) v[i][j] *= scale[i];
        store_run<true>(static_cast<TO*>(g.out) + t[i] * g.elems, e[i], g.elems, v[i]);
    }
}

// --------------------------------------------------------------- gradient

// The tokens are sorted (stably, so those of a row stay in their order) and
// cut into chunks, each summed by its own wavefronts; a token whose run crosses
// a chunk's border leaves partial sums that further launches add in chunk
// order.  The order of every sum follows from the tokens alone.
//
// Chunks are short where there are few of them to fill the chip.
constexpr int64_t kShortChunks = 16384;  // up to so many tokens
inline int chunk_of(int64_t n) { return n <= kShortChunks ? 8 : 32; }
// Rows in flight together.
constexpr int kBatch = 4;
// Wavefronts that zero rows: so many if there are four rows for each.  (With
// half as many 46,492 rows of 1,024 fp32 zeros take 38 us, not 35, and the
// gradient of 65,536 rows, which has other work to hide them, 306, not 313.)
constexpr int64_t kZeroWaves = 4096;
// Elements of a row that a wavefront zeroes.
constexpr int64_t kZeroSlice = 8192;

struct GradArgs {
    const uint32_t* keys;   // sorted; n_rows: no row
    const uint32_t* pos;
    const void* grad;
    void* out;
    float* part;            // [chunk][2][elems]: the sums of its first and last token
    int64_t n_ids, n_rows, elems, chunks;
    int64_t zero_waves;     // the first wavefronts zero rows
    Strip strip;
    int64_t zero_slices;
    float scale;
    int32_t accumulate, chunk, zero_rows;
};

__device__ inline uint32_t token_key(const void* ids, int id_bytes, int64_t t, int64_t n_rows, int64_t* status) {
    const int64_t id = token(ids, id_bytes, t);
    if (status && id >= n_rows) *status = TRE_E_KEYRANGE;
    return uint32_t(id >= 0 && id < n_rows ? id : n_rows);
}

__global__ __launch_bounds__(kThreads) void k_grad_keys(const void* __restrict__ ids, int id_bytes, int64_t n,
                                                        int64_t n_rows, uint32_t* __restrict__ keys,
                                                        uint32_t* __restrict__ pos, int64_t* __restrict__ status) {
    const int64_t t = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (t >= n) return;
    keys[t] = token_key(ids, id_bytes, t, n_rows, status);
    pos[t] = uint32_t(t);
}

// Few tokens are sorted in one launch: a workgroup counts, for its 16, the
// tokens that go before them, 16 threads to a part of the list.  (Four
// wavefronts for 64 tokens took 30 us for 6,300 of them, sixteen 13; with 16
// tokens to a workgroup a gradient of 5,900 takes 38.5 us in all, with 32 39.4,
// with 64 41, and one of 8,192 54, 56 and 58.)
constexpr int kRankMax = 8192, kRankThreads = 1024, kRankTokens = 16, kRankParts = kRankThreads / kRankTokens;

__global__ __launch_bounds__(kRankThreads) void k_grad_rank(const void* __restrict__ ids, int id_bytes, int n, int64_t n_rows,
                                                        uint32_t* __restrict__ keys, uint32_t* __restrict__ pos,
                                                        int64_t* __restrict__ status) {
    __shared__ uint4 all[kRankMax / 4];
    __shared__ int32_t part[kRankParts][kRankTokens];
    uint32_t* flat = reinterpret_cast<uint32_t*>(all);
    const int padded = (n + 4 * kRankParts - 1) / (4 * kRankParts) * (4 * kRankParts);  // (after every token)
#pragma unroll 4
    for (int t = threadIdx.x; t < padded; t += kRankThreads)
        flat[t] = t < n ? token_key(ids, id_bytes, t, n_rows, blockIdx.x == 0 ? status : nullptr) : 0xffffffffu;
    __syncthreads();
    const int own = threadIdx.x % kRankTokens, p = threadIdx.x / kRankTokens, i0 = blockIdx.x * kRankTokens, i = i0 + own;
    const uint32_t key = i < n ? flat[i] : 0u;
    const int q0 = padded / 4 / kRankParts * p, q1 = q0 + padded / 4 / kRankParts;
    int before = 0;
    // quads before the workgroup's tokens (equal ones go before), its own, those after
    const int a = min(max(i0 / 4, q0), q1), b = min(max((i0 + kRankTokens) / 4, q0), q1);
#pragma unroll 4
    for (int q = q0; q < a; q++) {
        const uint4 k = all[q];
        before += (k.x <= key) + (k.y <= key) + (k.z <= key) + (k.w <= key);
    }
    for (int q = a; q < b; q++) {
        const uint4 k = all[q];
        before += (k.x < key || (k.x == key && 4 * q < i)) + (k.y < key || (k.y == key && 4 * q + 1 < i)) +
                  (k.z < key || (k.z == key && 4 * q + 2 < i)) + (k.w < key || (k.w == key && 4 * q + 3 < i));
    }
#pragma unroll 4
    for (int q = b; q < q1; q++) {
        const uint4 k = all[q];
        before += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
    }
    part[p][own] = before;
    __syncthreads();
    if (p == 0 && i < n) {
        int at = 0;
#pragma unroll
        for (int j = 0; j < kRankParts; j++) at += part[j][own];
        keys[at] = key;
        pos[at] = uint32_t(i);
    }
}

template <typename TO, int N>
__device__ inline void put_row(const GradArgs& g, int64_t row, int64_t e, const float (&acc)[N]) {
    TO* at = static_cast<TO*>(g.out) + row * g.elems;
    float v[N];
    if (g.accumulate) {
        load_run(at, e, g.elems, v);
#pragma unroll
        for (int i = 0; i < N; i++) v[i] += g.scale * acc[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = g.scale * acc[i];
    }
    store_run<true>(at, e, g.elems, v);
}

// Zeroes elements begin to end of the output: whole 128-byte lines but for the
// first and last.  (A strip of each row for itself leaves a broken line at every
// strip's end where rows are not of whole lines: 46,492 rows of 998 fp32 values
// took 56 us, of 1,001 bf16 values 33; with one token's gradient they take 36 and
// 19 now.)
template <typename TO>
__device__ inline void zero_span(TO* out, int64_t begin, int64_t end) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int E = 16 / sizeof(TO), kLine = 128 / sizeof(TO);
    for (int64_t x = begin / kLine * kLine + (threadIdx.x & 63) * E; x < end; x += 64 * E) {
        if (x >= begin && x + E <= end) {
            __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4*>(out + x));
            continue;
        }
#pragma unroll
        for (int i = 0; i < E; i++)
            if (x + i >= begin && x + i < end) store1(out + x + i, 0.f);
    }
}

// Zeroes a slice of g.zero_rows rows (at most 64), but for rows that a token
// has: every lane looks one row up in the sorted keys.
template <typename TO>
__device__ inline void zero_rows(const GradArgs& g, int64_t w) {
    const int lane = threadIdx.x & 63;
    const int64_t r0 = w / g.zero_slices * g.zero_rows, e0 = w % g.zero_slices * kZeroSlice;
    const int64_t row = r0 + lane;
    int64_t lo = 0, hi = g.n_ids;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (int64_t(g.keys[mid]) < row) lo = mid + 1;
        else hi = mid;
    }
    const bool absent = lane < g.zero_rows && row < g.n_rows && (lo == g.n_ids || int64_t(g.keys[lo]) != row);
    TO* out = static_cast<TO*>(g.out);
    for (uint64_t m = __ballot(absent); m;) {
        const int at = __ffsll((unsigned long long)m) - 1;
        // rows of one slice that follow each other are one span
        const uint64_t after = ~(m >> at);
        const int rows = g.zero_slices > 1 ? 1 : after ? __ffsll((unsigned long long)after) - 1 : 64;
        const int64_t begin = (r0 + at) * g.elems + e0;
        zero_span(out, begin, g.zero_slices > 1 ? begin + min(g.elems - e0, kZeroSlice) : begin + rows * g.elems);
        m &= ~((rows < 64 ? (uint64_t(1) << rows) - 1 : ~uint64_t(0)) << at);
    }
}

// Rows of zeros, unless the sums are added to what is there; then a strip of a
// chunk.  WIDE: a wavefront to a strip.
template <typename TI, typename TO, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_grad_sum(GradArgs g) {
    constexpr int E = lane_elems<TI, TO>();
    int64_t w = block_index() * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w < g.zero_waves) {
        zero_rows<TO>(g, w);
        return;
    }
    w -= g.zero_waves;
    const int64_t x = WIDE ? w : (w * 64 + (threadIdx.x & 63)) >> g.strip.shift;
    const int64_t c = x / g.strip.slices;
    const int lane = threadIdx.x & ((1 << g.strip.shift) - 1);
    const int64_t e = (((x - c * g.strip.slices) << g.strip.shift) + lane) * E;
    if (c >= g.chunks || e >= g.elems) return;
    const int64_t i0 = c * g.chunk, i1 = min(i0 + g.chunk, g.n_ids);
    const int64_t none = g.n_rows;
    uint32_t key = g.keys[i0];
    if (int64_t(key) >= none) return;
    float acc[E];
#pragma unroll
    for (int h = 0; h < E; h++) acc[h] = 0.f;
    bool first = i0 > 0 && g.keys[i0 - 1] == key;  // the run began in an earlier chunk
    for (int64_t ib = i0; ib < i1; ib += kBatch) {
        uint32_t k[kBatch];
        float v[kBatch][E];
#pragma unroll
        for (int j = 0; j < kBatch; j++) {
            const int64_t i = min(ib + j, i1 - 1);
            k[j] = g.keys[i];
            // (the row of a token that is none is there to be read too)
            load_run(static_cast<const TI*>(g.grad) + int64_t(g.pos[i]) * g.elems, e, g.elems, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kBatch; j++) {
            if (ib + j >= i1) break;
            if (k[j] != key) {
                if (first) store_run(g.part + 2 * c * g.elems, e, g.elems, acc);
                else put_row<TO>(g, key, e, acc);
                first = false;
#pragma unroll
                for (int h = 0; h < E; h++) acc[h] = 0.f;
                key = k[j];
                if (int64_t(key) >= none) return;
            }
#pragma unroll
            for (int h = 0; h < E; h++) acc[h] += v[j][h];
        }
    }
    if (first) store_run(g.part + 2 * c * g.elems, e, g.elems, acc);
    else if (i1 < g.n_ids && g.keys[i1] == key) store_run(g.part + (2 * c + 1) * g.elems, e, g.elems, acc);
    else put_row<TO>(g, key, e, acc);
}

// The up to two elements of a row from e on (past its end, its last one again).
__device__ inline void load_pair(const float* row, int64_t e, int64_t n, float (&v)[2]) {
#pragma unroll
    for (int i = 0; i < 2; i++) v[i] = row[min(e + i, n - 1)];
}
__device__ inline void store_pair(float* row, int64_t e, int64_t n, const float (&v)[2]) {
#pragma unroll
    for (int i = 0; i < 2; i++)
        if (e + i < n) row[e + i] = v[i];
}
template <typename TO>
__device__ inline void put_pair(const GradArgs& g, int64_t row, int64_t e, const float (&v)[2]) {
    TO* at = static_cast<TO*>(g.out) + row * g.elems + e;
#pragma unroll
    for (int i = 0; i < 2; i++)
        if (e + i < g.elems) store1(at + i, g.accumulate ? load1(at + i) + g.scale * v[i] : g.scale * v[i]);
}

// The partial sums of kFan neighbouring chunks: those of a run that ends among
// them are added to its row, the others to the two that the group leaves for
// the next level, until one group holds all.  (One thread adding the partial
// sums of a run to its end took 51 us for 65,536 tokens of which one is a
// twentieth, and would take 15 times that if they were all alike.)
//
// A wavefront to a group and a strip of its rows.  Each lane looks at one
// chunk's borders, and only the partial sums that are there are read.
// Up to 64 chunks are joined at once.
constexpr int kFan = 16, kFanLast = 64, kJoinBatch = 16, kJoinLane = 2;
inline int fan_of(int64_t chunks) { return chunks <= kFanLast ? kFanLast : kFan; }

struct JoinArgs {
    const float* in;   // [chunk][2][elems]
    float* out;        // [group][2][elems]
    int64_t span;      // tokens of a chunk
    int64_t chunks, groups, slices;
    int32_t fan;
};

template <typename TO>
__global__ __launch_bounds__(kThreads) void k_grad_join(GradArgs g, JoinArgs a) {
    const int64_t w = block_index() * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t group = w / a.slices;
    if (group >= a.groups) return;
    const int lane = threadIdx.x & 63;
    const int64_t e = ((w - group * a.slices) * 64 + lane) * kJoinLane;
    const int64_t c0 = group * a.fan, c = c0 + lane;
    const int count = int(min(int64_t(a.fan), a.chunks - c0));
    bool cont = false, more = false, whole = false;
    uint32_t key = 0;
    if (lane < count) {
        const int64_t p0 = c * a.span, p1 = min(p0 + a.span, g.n_ids);
        key = g.keys[p0];
        const uint32_t before = g.keys[p0 > 0 ? p0 - 1 : 0], last = g.keys[p1 - 1], next = g.keys[p1 < g.n_ids ? p1 : p1 - 1];
        cont = p0 > 0 && before == key && int64_t(key) < g.n_rows;            // its first run began earlier
        more = p1 < g.n_ids && last == next && int64_t(last) < g.n_rows;      // its last run goes on
        whole = cont && key == last;                                          // and is its first
    }
    const uint64_t conts = __ballot(cont), goes = __ballot(more), wholes = __ballot(whole);
    // (Lanes past the row's end stay: the keys that they hold are read below.)
    float acc[kJoinLane] = {0.f, 0.f};
    bool first = conts & 1;  // the run at hand began in an earlier group
    for (uint64_t todo = conts | (goes & ~wholes); todo;) {
        int at[kJoinBatch];
        float v[kJoinBatch][2][kJoinLane];
#pragma unroll
        for (int j = 0; j < kJoinBatch; j++) {
            at[j] = todo ? __ffsll((unsigned long long)todo) - 1 : -1;
            todo &= todo - 1;
            if (at[j] < 0) continue;
            if (conts >> at[j] & 1) load_pair(a.in + 2 * (c0 + at[j]) * g.elems, e, g.elems, v[j][0]);
            if ((goes & ~wholes) >> at[j] & 1) load_pair(a.in + (2 * (c0 + at[j]) + 1) * g.elems, e, g.elems, v[j][1]);
        }
#pragma unroll
        for (int j = 0; j < kJoinBatch; j++) {
            if (at[j] < 0) break;
            const bool on = goes >> at[j] & 1, all = wholes >> at[j] & 1;
            if (conts >> at[j] & 1) {
#pragma unroll
                for (int h = 0; h < kJoinLane; h++) acc[h] += v[j][0][h];
                if (!(on && all)) {
                    if (first) store_pair(a.out + 2 * group * g.elems, e, g.elems, acc);
                    else put_pair<TO>(g, __builtin_amdgcn_readlane(key, at[j]), e, acc);
                    first = false;
                }
            }
            if (on && !all) {
#pragma unroll
                for (int h = 0; h < kJoinLane; h++) acc[h] = v[j][1][h];
            }
        }
    }
    if (goes >> (count - 1) & 1) store_pair(a.out + (2 * group + (first ? 0 : 1)) * g.elems, e, g.elems, acc);
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

int key_bits(int64_t n_rows) {
    int b = 1;
    while ((int64_t(1) << b) <= n_rows) b++;
    return b;
}

struct GradLayout {
    size_t keys, keys_alt, pos, pos_alt, hist, tmp, part, total;
};

GradLayout grad_layout(int64_t n, int64_t elems) {
    GradLayout L{};
    size_t off = 0;
    auto take = [&](size_t b) {
        const size_t o = off;
        off += align256(b);
        return o;
    };
    const size_t m = size_t(std::max<int64_t>(n, 1)), c = size_t(chunk_of(n));
    size_t chunks = 0;
    L.keys = take(4 * m);
    L.pos = take(4 * m);
    const size_t radix = n > kRankMax ? m : 0;
    L.keys_alt = take(4 * radix);
    L.pos_alt = take(4 * radix);
    const int64_t h = radix_u32_hist_elems(int64_t(m));
    L.hist = take(radix ? 4 * size_t(h) : 0);
    L.tmp = take(radix ? 4 * scan_tmp_elems(h) : 0);
    // two partial sums of a row for each chunk, of every level
    for (size_t k = (m + c - 1) / c; k > 0; k = k > 1 ? (k + size_t(fan_of(int64_t(k))) - 1) / size_t(fan_of(int64_t(k))) : 0)
        chunks += k;
    L.part = take(8 * chunks * size_t(elems));
    L.total = off;
    return L;
}

dim3 wave_grid(int64_t waves) { return grid_of((waves + kWaves - 1) / kWaves); }

template <typename TI, typename TO>
hipError_t lookup(LookupArgs g, hipStream_t s) {
    constexpr int E = lane_elems<TI, TO>();
    g.strip = strip(g.elems, E);
    if (g.elems > 64 * E) {
        g.groups = (g.strip.slices + kStrips - 1) / kStrips;
        const int64_t waves = g.n_ids * g.groups;
        k_lookup<TI, TO, true><<<wave_grid(waves), kThreads, 0, s>>>(g);
    } else {
        const int64_t threads = ((g.n_ids + kStrips - 1) / kStrips) << g.strip.shift;
        k_lookup<TI, TO, false><<<wave_grid((threads + 63) / 64), kThreads, 0, s>>>(g);
    }
    return hipGetLastError();
}

template <typename TI, typename TO>
hipError_t grad_sum(GradArgs g, hipStream_t s) {
    constexpr int E = lane_elems<TI, TO>();
    g.strip = strip(g.elems, E);
    g.zero_slices = (g.elems + kZeroSlice - 1) / kZeroSlice;
    g.zero_rows = 64;
    while (g.zero_rows > 4 && g.n_rows / g.zero_rows * g.zero_slices < kZeroWaves) g.zero_rows /= 2;
    g.zero_waves = g.accumulate ? 0 : (g.n_rows + g.zero_rows - 1) / g.zero_rows * g.zero_slices;
    const int64_t waves = g.zero_waves + ((g.chunks * g.strip.slices << g.strip.shift) + 63) / 64;
    if (waves == 0) return hipSuccess;
    const dim3 grid = wave_grid(waves);
    if (g.strip.shift == 6) k_grad_sum<TI, TO, true><<<grid, kThreads, 0, s>>>(g);
    else k_grad_sum<TI, TO, false><<<grid, kThreads, 0, s>>>(g);
    return hipGetLastError();
}

}  // namespace

size_t lookup_grad_ws_bytes(int64_t n, int64_t n_rows, int64_t elems) {
    (void)n_rows;
    return grad_layout(n, elems).total;
}

hipError_t launch_lookup(const void* table, int table_dtype, int64_t n_rows, int64_t elems, int64_t tile_rows,
                         const void* ids, int id_bytes, int64_t n_ids, float scale, void* out, int out_dtype,
                         int64_t* status, hipStream_t s) {
    LookupArgs g{};
    g.table = table;
    g.ids = ids;
    g.out = out;
    g.status = status;
    g.n_rows = n_rows;
    g.elems = elems;
    g.n_ids = n_ids;
    g.tile_rows = tile_rows;
    g.blocks = mx_row_blocks(elems);
    g.tile_bytes = mx_tile_bytes(tile_rows, elems);
    g.scale = scale;
    g.id_bytes = id_bytes;
    const bool half = out_dtype == TRE_BF16;
    if (table_dtype == TRE_MXFP4) return half ? lookup<Mx4, uint16_t>(g, s) : lookup<Mx4, float>(g, s);
    if (table_dtype == TRE_BF16) return half ? lookup<uint16_t, uint16_t>(g, s) : lookup<uint16_t, float>(g, s);
    return half ? lookup<float, uint16_t>(g, s) : lookup<float, float>(g, s);
}

hipError_t launch_lookup_grad(const void* grad, int grad_dtype, const void* ids, int id_bytes, int64_t n_ids, float scale,
                              void* out, int out_dtype, int64_t n_rows, int64_t elems, bool accumulate, int64_t* status,
                              char* ws, hipStream_t s) {
    const GradLayout L = grad_layout(n_ids, elems);
    uint32_t* keys = reinterpret_cast<uint32_t*>(ws + L.keys);
    uint32_t* pos = reinterpret_cast<uint32_t*>(ws + L.pos);
    hipError_t e;
    if (n_ids > kRankMax) {
        uint32_t* keys2 = reinterpret_cast<uint32_t*>(ws + L.keys_alt);
        uint32_t* pos2 = reinterpret_cast<uint32_t*>(ws + L.pos_alt);
        const int kb = key_bits(n_rows);
        k_grad_keys<<<unsigned((n_ids + kThreads - 1) / kThreads), kThreads, 0, s>>>(ids, id_bytes, n_ids, n_rows, keys, pos,
                                                                                     status);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if ((e = radix_sort_u32(keys, pos, keys2, pos2, n_ids, kb, reinterpret_cast<int32_t*>(ws + L.hist),
                                reinterpret_cast<int32_t*>(ws + L.tmp), s)) != hipSuccess)
            return e;
        if (radix_result_in_alt(n_ids, kb)) {
            keys = keys2;
            pos = pos2;
        }
    } else if (n_ids > 0) {
        const unsigned grid = unsigned((n_ids + kRankTokens - 1) / kRankTokens);
        k_grad_rank<<<grid, kRankThreads, 0, s>>>(ids, id_bytes, int(n_ids), n_rows, keys, pos, status);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    GradArgs g{};
    g.keys = keys;
    g.pos = pos;
    g.grad = grad;
    g.out = out;
    g.part = reinterpret_cast<float*>(ws + L.part);
    g.n_ids = n_ids;
    g.n_rows = n_rows;
    g.elems = elems;
    g.chunk = chunk_of(n_ids);
    g.chunks = (n_ids + g.chunk - 1) / g.chunk;
    g.scale = scale;
    g.accumulate = accumulate;
    const bool half = out_dtype == TRE_BF16;
    if (grad_dtype == TRE_BF16) e = half ? grad_sum<uint16_t, uint16_t>(g, s) : grad_sum<uint16_t, float>(g, s);
    else e = half ? grad_sum<float, uint16_t>(g, s) : grad_sum<float, float>(g, s);
    if (e != hipSuccess) return e;
    JoinArgs a{};
    a.in = g.part;
    a.span = g.chunk;
    a.slices = (elems + 64 * kJoinLane - 1) / (64 * kJoinLane);
    for (a.chunks = g.chunks; a.chunks > 1; a.chunks = a.groups) {
        a.fan = fan_of(a.chunks);
        a.groups = (a.chunks + a.fan - 1) / a.fan;
        float* out = const_cast<float*>(a.in) + 2 * a.chunks * elems;
        a.out = out;
        const int64_t waves = a.groups * a.slices;
        if (half) k_grad_join<uint16_t><<<wave_grid(waves), kThreads, 0, s>>>(g, a);
        else k_grad_join<float><<<wave_grid(waves), kThreads, 0, s>>>(g, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        a.in = out;
        a.span *= a.fan;
    }
    return hipSuccess;
}

}  // namespace tre
