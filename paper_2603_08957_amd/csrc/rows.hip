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
constexpr int kLane = 8;              // elements of a row to a lane
constexpr int kSlice = 64 * kLane;    // elements of a row to a wavefront

// 16 bytes on any element boundary: rows of an odd number of elements begin
// anywhere, and the wide access still costs less than one per element.
typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ inline void load8(const float* p, float (&v)[kLane]) {
    const f32x4_4 a = *reinterpret_cast<const f32x4_4*>(p), b = *reinterpret_cast<const f32x4_4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        v[i] = a[i];
        v[4 + i] = b[i];
    }
}
__device__ inline void load8(const uint16_t* p, float (&v)[kLane]) {
    const u32x4_2 a = *reinterpret_cast<const u32x4_2*>(p);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}
__device__ inline void store8(float* p, const float (&v)[kLane]) {
    *reinterpret_cast<f32x4_4*>(p) = f32x4_4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_4*>(p + 4) = f32x4_4{v[4], v[5], v[6], v[7]};
}
__device__ inline void store8(uint16_t* p, const float (&v)[kLane]) {
    u32x4_2 a;
#pragma unroll
    for (int i = 0; i < 4; i++)
        a[i] = uint32_t(f32_to_bf16_rne(v[2 * i])) | (uint32_t(f32_to_bf16_rne(v[2 * i + 1])) << 16);
    *reinterpret_cast<u32x4_2*>(p) = a;
}
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
__device__ inline void store1(float* p, float v) { *p = v; }
__device__ inline void store1(uint16_t* p, float v) { *p = f32_to_bf16_rne(v); }

// The up to eight elements of a row from element e on.
template <typename T>
__device__ inline void load_run(const T* row, int64_t e, int64_t n, float (&v)[kLane]) {
    if (e + kLane <= n) {
        load8(row + e, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kLane; i++) v[i] = e + i < n ? load1(row + e + i) : 0.f;
}
template <typename T>
__device__ inline void store_run(T* row, int64_t e, int64_t n, const float (&v)[kLane]) {
    if (e + kLane <= n) {
        store8(row + e, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kLane; i++)
        if (e + i < n) store1(row + e + i, v[i]);
}

// Token t of a list of 4- or 8-byte integers.
__device__ inline int64_t token(const void* ids, int id_bytes, int64_t t) {
    return id_bytes == 8 ? static_cast<const int64_t*>(ids)[t] : int64_t(static_cast<const int32_t*>(ids)[t]);
}

// ----------------------------------------------------------------- lookup

struct LookupArgs {
    const void* table;
    const void* ids;
    void* out;
    int64_t* status;
    int64_t n_rows, elems, n_ids;
    int64_t slices;              // of a row
    int64_t tile_rows, blocks;   // 4-bit tiles: rows of a tile, blocks of a row
    int64_t tile_bytes;
    float scale;
    int32_t id_bytes;
};

struct Mx4 {};

// A wavefront per row and slice.
template <typename TI, typename TO>
__global__ __launch_bounds__(kThreads) void k_lookup(LookupArgs g) {
    const int64_t x = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int64_t t = x / g.slices;
    if (t >= g.n_ids) return;
    const int64_t e = (x - t * g.slices) * kSlice + (threadIdx.x & 63) * kLane;
    const int64_t id = token(g.ids, g.id_bytes, t);
    if (g.status && id >= g.n_rows && e == 0) *g.status = TRE_E_KEYRANGE;
    if (e >= g.elems) return;
    float v[kLane] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (id >= 0 && id < g.n_rows) {
        if constexpr (std::is_same_v<TI, Mx4>) {
            const int64_t tile = id / g.tile_rows, row = (id - tile * g.tile_rows) * g.blocks;
            const uint8_t* at = static_cast<const uint8_t*>(g.table) + tile * g.tile_bytes;
            const uint32_t q = *reinterpret_cast<const uint32_t*>(at + row * 16 + e / 2);
            mx_values(q, at[g.tile_rows * g.blocks * 16 + row + e / kMxBlock], v);
        } else {
            load_run(static_cast<const TI*>(g.table) + id * g.elems, e, g.elems, v);
        }
#pragma unroll
        for (int i = 0; i < kLane; i++) v[i] *= g.scale;
    }
    store_run(static_cast<TO*>(g.out) + t * g.elems, e, g.elems, v);
}

// --------------------------------------------------------------- gradient

// The tokens are sorted (stably, so those of a row stay in their order) and
// cut into chunks of kChunk, each summed by its own workgroups; a token whose
// run crosses a chunk's border leaves partial sums that a second launch adds
// in chunk order.  The order of every sum follows from the tokens alone.
constexpr int kChunk = 32;

struct GradArgs {
    const uint32_t* keys;   // sorted; n_rows: no row
    const uint32_t* pos;
    const uint32_t* bits;   // rows that occur
    const void* grad;
    void* out;
    float* part;            // [chunk][2][elems]: the sums of its first and last token
    int64_t n_ids, n_rows, elems, slices, chunks;
    float scale;
    int32_t accumulate;
};

__global__ __launch_bounds__(kThreads) void k_grad_keys(const void* __restrict__ ids, int id_bytes, int64_t n,
                                                        int64_t n_rows, uint32_t* __restrict__ keys,
                                                        uint32_t* __restrict__ pos, uint32_t* __restrict__ bits,
                                                        int64_t* __restrict__ status) {
    const int64_t t = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (t >= n) return;
    const int64_t id = token(ids, id_bytes, t);
    const bool ok = id >= 0 && id < n_rows;
    if (status && id >= n_rows) *status = TRE_E_KEYRANGE;
    keys[t] = uint32_t(ok ? id : n_rows);
    pos[t] = uint32_t(t);
    if (ok && bits) atomicOr(&bits[id >> 5], 1u << (id & 31));
}

template <typename TO>
__device__ inline void put_row(const GradArgs& g, int64_t row, int64_t e, const float (&acc)[kLane]) {
    TO* at = static_cast<TO*>(g.out) + row * g.elems;
    float v[kLane];
    if (g.accumulate) {
        load_run(at, e, g.elems, v);
#pragma unroll
        for (int i = 0; i < kLane; i++) v[i] += g.scale * acc[i];
    } else {
#pragma unroll
        for (int i = 0; i < kLane; i++) v[i] = g.scale * acc[i];
    }
    store_run(at, e, g.elems, v);
}

// A wavefront per chunk and slice, then (not accumulating) one per row and
// slice that zeroes the rows no token has.
template <typename TI, typename TO>
__global__ __launch_bounds__(kThreads) void k_grad_sum(GradArgs g) {
    const int64_t x = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int64_t c = x / g.slices;
    const int64_t e = (x - c * g.slices) * kSlice + (threadIdx.x & 63) * kLane;
    if (e >= g.elems) return;
    float acc[kLane] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c >= g.chunks) {
        const int64_t row = c - g.chunks;
        if (g.accumulate || row >= g.n_rows || (g.bits[row >> 5] >> (row & 31)) & 1) return;
        store_run(static_cast<TO*>(g.out) + row * g.elems, e, g.elems, acc);
        return;
    }
    const int64_t i0 = c * kChunk, i1 = min(i0 + kChunk, g.n_ids);
    uint32_t key = g.keys[i0];
    if (int64_t(key) >= g.n_rows) return;
    bool first = i0 > 0 && g.keys[i0 - 1] == key;  // the run began in an earlier chunk
    for (int64_t i = i0; i < i1; i++) {
        const uint32_t k = g.keys[i];
        if (k != key) {
            if (first) store_run(g.part + 2 * c * g.elems, e, g.elems, acc);
            else put_row<TO>(g, key, e, acc);
            first = false;
#pragma unroll
            for (int j = 0; j < kLane; j++) acc[j] = 0.f;
            key = k;
            if (int64_t(key) >= g.n_rows) return;
        }
        float v[kLane];
        load_run(static_cast<const TI*>(g.grad) + int64_t(g.pos[i]) * g.elems, e, g.elems, v);
#pragma unroll
        for (int j = 0; j < kLane; j++) acc[j] += v[j];
    }
    if (first) store_run(g.part + 2 * c * g.elems, e, g.elems, acc);
    else if (i1 < g.n_ids && g.keys[i1] == key) store_run(g.part + (2 * c + 1) * g.elems, e, g.elems, acc);
    else put_row<TO>(g, key, e, acc);
}

// A wavefront per chunk and slice: the run that begins in the chunk and goes
// on past it.
template <typename TO>
__global__ __launch_bounds__(kThreads) void k_grad_join(GradArgs g) {
    const int64_t x = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int64_t c = x / g.slices;
    const int64_t e = (x - c * g.slices) * kSlice + (threadIdx.x & 63) * kLane;
    const int64_t i0 = c * kChunk, i1 = i0 + kChunk;
    if (i1 >= g.n_ids || e >= g.elems) return;
    const uint32_t key = g.keys[i1 - 1];
    if (int64_t(key) >= g.n_rows || g.keys[i1] != key) return;
    if (g.keys[i0] == key && i0 > 0 && g.keys[i0 - 1] == key) return;  // it began earlier
    float acc[kLane], v[kLane];
    load_run(g.part + (2 * c + 1) * g.elems, e, g.elems, acc);
    for (int64_t d = c + 1; d < g.chunks && g.keys[d * kChunk] == key; d++) {
        load_run(g.part + 2 * d * g.elems, e, g.elems, v);
#pragma unroll
        for (int j = 0; j < kLane; j++) acc[j] += v[j];
    }
    put_row<TO>(g, key, e, acc);
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

int key_bits(int64_t n_rows) {
    int b = 1;
    while ((int64_t(1) << b) <= n_rows) b++;
    return b;
}

struct GradLayout {
    size_t keys, keys_alt, pos, pos_alt, hist, tmp, bits, part, total;
};

GradLayout grad_layout(int64_t n, int64_t n_rows, int64_t elems) {
    GradLayout L{};
    size_t off = 0;
    auto take = [&](size_t b) {
        const size_t o = off;
        off += align256(b);
        return o;
    };
    const size_t m = size_t(std::max<int64_t>(n, 1));
    L.keys = take(4 * m);
    L.keys_alt = take(4 * m);
    L.pos = take(4 * m);
    L.pos_alt = take(4 * m);
    const int64_t h = radix_hist_elems(int64_t(m));
    L.hist = take(4 * size_t(h));
    L.tmp = take(4 * scan_tmp_elems(h));
    L.bits = take(4 * size_t((n_rows + 31) / 32));
    L.part = take(8 * size_t((m + kChunk - 1) / kChunk) * size_t(elems));
    L.total = off;
    return L;
}

unsigned wave_grid(int64_t waves) { return unsigned((waves + kWaves - 1) / kWaves); }

}  // namespace

size_t lookup_grad_ws_bytes(int64_t n, int64_t n_rows, int64_t elems) { return grad_layout(n, n_rows, elems).total; }

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
    g.slices = (elems + kSlice - 1) / kSlice;
    g.tile_rows = tile_rows;
    g.blocks = mx_row_blocks(elems);
    g.tile_bytes = mx_tile_bytes(tile_rows, elems);
    g.scale = scale;
    g.id_bytes = id_bytes;
    const int64_t waves = n_ids * g.slices;
    if (waves / kWaves >= int64_t(0x7fffffff)) return hipErrorInvalidConfiguration;
    const unsigned grid = wave_grid(waves);
    const bool half = out_dtype == TRE_BF16;
    if (table_dtype == TRE_MXFP4) {
        if (half) k_lookup<Mx4, uint16_t><<<grid, kThreads, 0, s>>>(g);
        else k_lookup<Mx4, float><<<grid, kThreads, 0, s>>>(g);
    } else if (table_dtype == TRE_BF16) {
        if (half) k_lookup<uint16_t, uint16_t><<<grid, kThreads, 0, s>>>(g);
        else k_lookup<uint16_t, float><<<grid, kThreads, 0, s>>>(g);
    } else {
        if (half) k_lookup<float, uint16_t><<<grid, kThreads, 0, s>>>(g);
        else k_lookup<float, float><<<grid, kThreads, 0, s>>>(g);
    }
    return hipGetLastError();
}

hipError_t launch_lookup_grad(const void* grad, int grad_dtype, const void* ids, int id_bytes, int64_t n_ids, float scale,
                              void* out, int out_dtype, int64_t n_rows, int64_t elems, bool accumulate, int64_t* status,
                              char* ws, hipStream_t s) {
    const GradLayout L = grad_layout(n_ids, n_rows, elems);
    uint32_t* keys = reinterpret_cast<uint32_t*>(ws + L.keys);
    uint32_t* pos = reinterpret_cast<uint32_t*>(ws + L.pos);
    uint32_t* keys2 = reinterpret_cast<uint32_t*>(ws + L.keys_alt);
    uint32_t* pos2 = reinterpret_cast<uint32_t*>(ws + L.pos_alt);
    uint32_t* bits = reinterpret_cast<uint32_t*>(ws + L.bits);
    hipError_t e;
    if (!accumulate && (e = launch_fill_zero(bits, 4 * size_t((n_rows + 31) / 32), s)) != hipSuccess) return e;
    const int kb = key_bits(n_rows);
    if (n_ids > 0) {
        k_grad_keys<<<unsigned((n_ids + kThreads - 1) / kThreads), kThreads, 0, s>>>(ids, id_bytes, n_ids, n_rows, keys, pos,
                                                                                     accumulate ? nullptr : bits, status);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if ((e = radix_sort_u32(keys, pos, keys2, pos2, n_ids, kb, reinterpret_cast<int32_t*>(ws + L.hist),
                                reinterpret_cast<int32_t*>(ws + L.tmp), s)) != hipSuccess)
            return e;
    }
    const bool alt = radix_result_in_alt(n_ids, kb);
    GradArgs g{};
    g.keys = alt ? keys2 : keys;
    g.pos = alt ? pos2 : pos;
    g.bits = bits;
    g.grad = grad;
    g.out = out;
    g.part = reinterpret_cast<float*>(ws + L.part);
    g.n_ids = n_ids;
    g.n_rows = n_rows;
    g.elems = elems;
    g.slices = (elems + kSlice - 1) / kSlice;
    g.chunks = (n_ids + kChunk - 1) / kChunk;
    g.scale = scale;
    g.accumulate = accumulate;
    const int64_t waves = (g.chunks + (accumulate ? 0 : n_rows)) * g.slices;
    if (waves == 0) return hipSuccess;
    if (waves / kWaves >= int64_t(0x7fffffff)) return hipErrorInvalidConfiguration;
    const unsigned grid = wave_grid(waves);
    const bool half = out_dtype == TRE_BF16;
    if (grad_dtype == TRE_BF16) {
        if (half) k_grad_sum<uint16_t, uint16_t><<<grid, kThreads, 0, s>>>(g);
        else k_grad_sum<uint16_t, float><<<grid, kThreads, 0, s>>>(g);
    } else {
        if (half) k_grad_sum<float, uint16_t><<<grid, kThreads, 0, s>>>(g);
        else k_grad_sum<float, float><<<grid, kThreads, 0, s>>>(g);
    }
    if ((e = hipGetLastError()) != hipSuccess || g.chunks <= 1) return e;
    const unsigned joins = wave_grid(g.chunks * g.slices);
    if (half) k_grad_join<uint16_t><<<joins, kThreads, 0, s>>>(g);
    else k_grad_join<float><<<joins, kThreads, 0, s>>>(g);
    return hipGetLastError();
}

}  // namespace tre
