// Tiles in microscaled 4-bit floating point: quantisation, reading back and
// the contraction of matched pairs on the scaled MFMA.
//
// A block is 32 values of the contracted index.  With m its largest magnitude,
//   e = floor(log2 m) - 2 (at least -127),  q = round(x / 2^e) to E2M1,
// and W[m,n] += sum over blocks of 2^(eA + eB) sum_k qA qB, which
// v_mfma_scale_f32_16x16x128_f8f6f4 does for four blocks at a time: lane l
// holds the 32 codes (16 bytes) and the scale byte of row l % 16, block l / 16,
// of either operand, and element (4 (l / 16) + i, l % 16) of the sums.
#include "lds_copy.h"
#include "mx.h"
#include "tre_internal.h"

#include <atomic>
#include <cmath>

namespace tre {

namespace {

constexpr int kThreads = 256;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ inline float as_f32(const float* p) { return *p; }
__device__ inline float as_f32(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }

__device__ inline void put(float* p, float v) { *p = v; }
// (a value of a block has two significant bits: its upper half is the value)
__device__ inline void put(uint16_t* p, float v) { *p = uint16_t(__float_as_uint(v) >> 16); }

// Element offset of index x inside a tile (Dims in kernel arguments: few, mostly one).
__device__ inline int64_t offset_of(const Dims& d, int64_t x) {
    int64_t o = 0;
    for (int i = d.n - 1; i > 0; i--) {
        const int64_t q = x / d.size[i];
        o += (x - q * d.size[i]) * d.stride[i];
        x = q;
    }
    return d.n ? o + x * d.stride[0] : 0;
}

// Division of x < 2^31 by d: with 2^(s - 1) < d <= 2^s and m = ceil(2^(31 + s) / d),
// x m / 2^(31 + s) lies above x / d by less than x 2^-(31 + s) < 1 / d.
struct Divisor {
    uint32_t d = 1, m = 0, s = 0;
    Divisor() = default;
    explicit Divisor(int64_t by) : d(uint32_t(by)) {
        while ((int64_t(1) << s) < by) s++;
        if (s) m = uint32_t(((uint64_t(1) << (31 + s)) + d - 1) / d);
    }
    __device__ uint32_t of(uint32_t x) const { return s ? __umulhi(x, m) >> (s - 1) : x; }
};

// An operand's tiles before and after.
struct MxTiles {
    Dims row, k;
    Divisor tile, line;  // eights of a tile, of a row
    int64_t elems;      // of an unquantised tile
    int64_t rows, K;
    int64_t blocks;     // of a row
    int group;          // blocks of a group
    int lanes;          // rows kernels: log2 of the lanes side by side on a row
    int64_t bytes;      // of a 4-bit tile
    int64_t n;          // tiles
};

// The scale byte of a block whose largest magnitude has these bits: exponent
// field - 2, which is the bias of 127 and the 2 of E2M1's largest exponent in
// one.
__device__ inline int scale_byte(uint32_t max_bits) {
    return max_bits >= 0x7f800000u ? kMxNanScale : max(int(max_bits >> 23) - 2, 0);
}

// The codes of eight values under a scale byte.  (The conversion takes its
// scale from the exponent field alone: a byte of 0 is 2^-127.)
__device__ inline uint32_t codes8(const float* v, int sb) {
    const float s = __uint_as_float(uint32_t(sb) << 23);
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], s, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], s, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], s, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], s, 3);
    return sb == kMxNanScale ? 0u : q;
}

// Block b's scale byte of a tile, and after the last one the bytes that pad the
// tile.
__device__ inline void put_scale(const MxTiles& g, uint8_t* tile, uint32_t b, int sb) {
    const int64_t blocks = g.rows * g.blocks;
    tile[blocks * 16 + b] = uint8_t(sb);
    if (b == uint32_t(blocks) - 1)
        for (int64_t i = blocks * 17; i < g.bytes; i++) tile[i] = 0;
}

// ---- any layout: a thread per block, its values found one by one (134 M bf16
// values whose contracted labels are not side by side 380 us to quantise and 650
// to read back; the kernels below take 67 and 53)

template <typename T>
__global__ __launch_bounds__(kThreads) void k_mx_quantize(MxTiles g, const T* __restrict__ src, uint8_t* __restrict__ dst) {
    const int64_t b = block_index() * kThreads + threadIdx.x;
    const int64_t per = g.rows * g.blocks;
    if (b >= g.n * per) return;
    const int64_t t = b / per, x = b - t * per, r = x / g.blocks, k0 = (x - r * g.blocks) * kMxBlock;
    const T* at = src + t * g.elems + offset_of(g.row, r);
    float v[kMxBlock];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kMxBlock; i++) {
        v[i] = k0 + i < g.K ? as_f32(at + offset_of(g.k, k0 + i)) : 0.f;
        m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    }
    const int sb = scale_byte(m);
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; i++) q[i] = codes8(v + 8 * i, sb);
    uint8_t* out = dst + t * g.bytes;
    const uint32_t at_block = mx_block_of(uint32_t(g.rows), g.group, uint32_t(r), uint32_t(x - r * g.blocks));
    *reinterpret_cast<uint4*>(out + int64_t(at_block) * 16) = make_uint4(q[0], q[1], q[2], q[3]);
    put_scale(g, out, at_block, sb);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize(MxTiles g, const uint8_t* __restrict__ src, T* __restrict__ dst) {
    const int64_t b = block_index() * kThreads + threadIdx.x;
    const int64_t per = g.rows * g.blocks;
    if (b >= g.n * per) return;
    const int64_t t = b / per, x = b - t * per, r = x / g.blocks, k0 = (x - r * g.blocks) * kMxBlock;
    const uint8_t* in = src + t * g.bytes;
    const uint32_t from = mx_block_of(uint32_t(g.rows), g.group, uint32_t(r), uint32_t(x - r * g.blocks));
    const uint4 c = *reinterpret_cast<const uint4*>(in + int64_t(from) * 16);
    const uint32_t q[4] = {c.x, c.y, c.z, c.w};
    const int sb = in[per * 16 + from];
    T* at = dst + t * g.elems + offset_of(g.row, r);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        float v[8];
        mx_values(q[i], sb, v);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int64_t k = k0 + 8 * i + j;
            if (k < g.K) put(at + offset_of(g.k, k), v[j]);
        }
    }
}

// ---- the contracted index consecutive in the tile: a lane per eight values,
// four to a block, so a wavefront's loads and stores are whole runs of the
// row.  (A thread per block reads 64 bytes apart: 134 M bf16 values took 294 us
// to quantise and 588 to read back.)

constexpr int kRun = 4;  // eights of a thread, a workgroup's width apart, in flight together

// Eight values of a row as they are loaded: rows begin on any element.
typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

template <typename T>
struct Eight;

template <>
struct Eight<uint16_t> {
    uint32_t v[4];
    __device__ void load(const uint16_t* p, int64_t n) {
        if (n >= 8) {
            const u32x4_2 a = *reinterpret_cast<const u32x4_2*>(p);
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = a[i];
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
            v[i] = (2 * i < n ? uint32_t(p[2 * i]) : 0u) | (2 * i + 1 < n ? uint32_t(p[2 * i + 1]) << 16 : 0u);
    }
    // the eight from k on of a row of K, a multiple of eight; zeros past it
    __device__ void load_or_zero(const uint16_t* row, uint32_t k, uint32_t K) {
        load(row + min(k, K - 8), 8);
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = k < K ? v[i] : 0u;
    }
    // bits of the largest magnitude, as fp32
    __device__ uint32_t top() const {
        u16x2 m = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
        return uint32_t(max(m[0], m[1])) << 16;
    }
    __device__ uint32_t codes(int sb) const {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const float s = __uint_as_float(uint32_t(sb) << 23);
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2, v[0]), s, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2, v[1]), s, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2, v[2]), s, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(bf16x2, v[3]), s, 3);
        return sb == kMxNanScale ? 0u : q;
    }
};

template <>
struct Eight<float> {
    float v[8];
    __device__ void load(const float* p, int64_t n) {
        if (n >= 8) {
            const u32x4_4 a = *reinterpret_cast<const u32x4_4*>(p), b = *reinterpret_cast<const u32x4_4*>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                v[i] = __uint_as_float(a[i]);
                v[4 + i] = __uint_as_float(b[i]);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < n ? p[i] : 0.f;
    }
    __device__ void load_or_zero(const float* row, uint32_t k, uint32_t K) {
        load(row + min(k, K - 8), 8);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = k < K ? v[i] : 0.f;
    }
    __device__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
        return m;
    }
    __device__ uint32_t codes(int sb) const { return codes8(v, sb); }
};

// the maximum over the four lanes of a quad
__device__ inline uint32_t quad_max(uint32_t m) {
    m = max(m, uint32_t(__builtin_amdgcn_mov_dpp(int(m), 0xB1, 0xf, 0xf, true)));  // lanes 1 0 3 2
    return max(m, uint32_t(__builtin_amdgcn_mov_dpp(int(m), 0x4E, 0xf, 0xf, true)));  // lanes 2 3 0 1
}

// The eights of a workgroup: kRun * kWaves strips, a wavefront's each, of
// consecutive rows (over all tiles) and the same 1 << g.lanes eights of them, so
// that rows which lie side by side in a group are written together.  g.line:
// strips' eights of a row, g.tile: rows of a tile.
constexpr int kWaves = kThreads / 64;

struct RunPos {
    int64_t t;       // tile
    uint32_t r, e;   // row in it, eight of the row
    bool in;
};
// (the workgroup's first row is found in 64 bits, the others from it in 32)
__device__ inline RunPos run_pos(const MxTiles& g, int64_t t0, uint32_t r0, uint32_t e0, int i) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t row = r0 + ((i * kWaves + w) << (6 - g.lanes)) + (lane >> g.lanes), dt = g.tile.of(row);
    RunPos p;
    p.t = t0 + dt;
    p.r = row - dt * g.tile.d;
    p.e = e0 + (lane & ((1 << g.lanes) - 1));
    p.in = p.t < g.n;
    return p;
}
__device__ inline void run_start(const MxTiles& g, int64_t& t0, uint32_t& r0, uint32_t& e0) {
    const int64_t b = block_index(), rows = b / g.line.d;  // (strips of a row vary first)
    e0 = uint32_t(b - rows * g.line.d) << g.lanes;
    const int64_t row = rows * (int64_t(kRun * kWaves) << (6 - g.lanes));
    t0 = row / g.tile.d;
    r0 = uint32_t(row - t0 * g.tile.d);
}

// How a row's eights lie in the unquantised tile: all of them, all but blocks
// of zeros at the end, the last cut.
enum RunKind { RUN_FULL, RUN_WHOLE, RUN_CUT };

template <typename T, RunKind KIND>
__global__ __launch_bounds__(kThreads) void k_mx_quantize_rows(MxTiles g, const T* __restrict__ src, uint8_t* __restrict__ dst) {
    int64_t t0;
    uint32_t r0, e0;
    run_start(g, t0, r0, e0);
    const uint32_t eights = uint32_t(g.blocks * 4), rows = uint32_t(g.rows);
    Eight<T> v[kRun];
#pragma unroll
    for (int i = 0; i < kRun; i++) {
        // (past the last row or eight: a place that is there, not written)
        RunPos p = run_pos(g, t0, r0, e0, i);
        if (!p.in) p.t = p.r = 0;
        const uint32_t k = min(p.e, eights - 1) * 8;
        const T* at = src + p.t * g.elems + (g.row.n <= 1 ? int64_t(p.r) * g.row.stride[0] : offset_of(g.row, p.r));
        if constexpr (KIND == RUN_FULL) v[i].load(at + k, 8);
        else if constexpr (KIND == RUN_WHOLE) v[i].load_or_zero(at, k, uint32_t(g.K));
        else v[i].load(at + k, g.K - k);
    }
#pragma unroll
    for (int i = 0; i < kRun; i++) {
        const RunPos p = run_pos(g, t0, r0, e0, i);
        const int sb = scale_byte(quad_max(v[i].top()));
        if (!p.in || p.e >= eights) continue;
        uint8_t* out = dst + p.t * g.bytes;
        const uint32_t b = mx_block_of(rows, g.group, p.r, p.e / 4);
        *reinterpret_cast<uint32_t*>(out + int64_t(b) * 16 + (p.e & 3) * 4) = v[i].codes(sb);
        if ((p.e & 3) == 0) put_scale(g, out, b, sb);
    }
}

// (eights past K are not read)
template <typename T, bool CUT>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize_rows(MxTiles g, const uint8_t* __restrict__ src, T* __restrict__ dst) {
    int64_t t0;
    uint32_t r0, e0;
    run_start(g, t0, r0, e0);
    const uint32_t eights = uint32_t((g.K + 7) / 8), rows = uint32_t(g.rows);
    uint32_t q[kRun];
    int sb[kRun];
#pragma unroll
    for (int i = 0; i < kRun; i++) {
        RunPos p = run_pos(g, t0, r0, e0, i);
        if (!p.in) p.t = p.r = 0;
        const uint32_t e = min(p.e, eights - 1), b = mx_block_of(rows, g.group, p.r, e / 4);
        const uint8_t* at = src + p.t * g.bytes;
        q[i] = *reinterpret_cast<const uint32_t*>(at + int64_t(b) * 16 + (e & 3) * 4);
        sb[i] = at[g.rows * g.blocks * 16 + b];
    }
#pragma unroll
    for (int i = 0; i < kRun; i++) {
        const RunPos p = run_pos(g, t0, r0, e0, i);
        if (!p.in || p.e >= eights) continue;
        const int64_t k = 8 * int64_t(p.e);
        T* out = dst + p.t * g.elems + (g.row.n <= 1 ? int64_t(p.r) * g.row.stride[0] : offset_of(g.row, p.r)) + k;
        float v[8];
        mx_values(q[i], sb[i], v);
        if (!CUT || g.K - k >= 8) {
            if constexpr (sizeof(T) == 2) {
                u32x4_2 a;
#pragma unroll
                for (int j = 0; j < 4; j++) a[j] = __builtin_amdgcn_perm(__float_as_uint(v[2 * j + 1]), __float_as_uint(v[2 * j]), 0x07060302u);
                *reinterpret_cast<u32x4_2*>(out) = a;
            } else {
                u32x4_4 a, b;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    a[j] = __float_as_uint(v[j]);
                    b[j] = __float_as_uint(v[4 + j]);
                }
                *reinterpret_cast<u32x4_4*>(out) = a;
                *reinterpret_cast<u32x4_4*>(out + 4) = b;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (k + j < g.K) put(out + j, v[j]);
        }
    }
}

// ---- the rows consecutive in the tile (two or more: of one row the contracted
// index is consecutive): a thread per block of one fp32 row or two bf16 rows,
// so that lanes side by side read consecutive rows of one k.  The last of an
// odd number of bf16 rows goes with the row before it once more.

// A thread's tile, block and first row: the lanes of a wavefront take
// consecutive lines (of R rows) of a group, its wavefronts the group's blocks.
// g.line: lines of a tile, g.tile: lines and groups.
struct ColPos {
    int64_t t;
    uint32_t kb, r;
};
template <int R>
__device__ inline ColPos col_pos(const MxTiles& g) {
    const int w = threadIdx.x >> 6, sets = kWaves / g.group;  // wavefronts of different lines
    const int64_t x0 = block_index() * (64 * sets), t0 = x0 / g.tile.d;
    const uint32_t x = uint32_t(x0 - t0 * g.tile.d) + (w / g.group) * 64 + (threadIdx.x & 63), dt = g.tile.of(x), y = x - dt * g.tile.d;
    const uint32_t group = g.line.of(y);
    ColPos p;
    p.t = t0 + dt;
    p.kb = group * g.group + w % g.group;
    p.r = min((y - group * g.line.d) * R, uint32_t(g.rows) - R);
    return p;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_mx_quantize_cols(MxTiles g, const T* __restrict__ src, uint8_t* __restrict__ dst) {
    constexpr int R = sizeof(T) == 2 ? 2 : 1;
    typedef uint32_t u32_2 __attribute__((aligned(2)));
    const ColPos p = col_pos<R>(g);
    if (p.t >= g.n) return;
    const int left = int(min(g.K - int64_t(p.kb) * kMxBlock, int64_t(kMxBlock)));  // below 1: a block of zeros
    const int64_t sk = g.k.stride[0];
    // k past the last reads the last (of a block past K: the tile's first) and counts as zero
    const T* at = src + p.t * g.elems + (left > 0 ? int64_t(p.kb) * kMxBlock * sk : 0) + p.r;
    uint32_t v[kMxBlock];  // bf16: both rows of a k
#pragma unroll
    for (int i = 0; i < kMxBlock; i++) {
        v[i] = *reinterpret_cast<const u32_2*>(at);
        if (i + 1 < left) at += sk;
    }
#pragma unroll
    for (int i = 0; i < kMxBlock; i++) v[i] = i < left ? v[i] : 0u;
    uint8_t* out = dst + p.t * g.bytes;
    const int64_t b0 = mx_block_of(uint32_t(g.rows), g.group, p.r, p.kb);
    if constexpr (R == 1) {
        uint32_t m = 0;
        float f[kMxBlock];
#pragma unroll
        for (int i = 0; i < kMxBlock; i++) {
            m = max(m, v[i] & 0x7fffffffu);
            f[i] = __uint_as_float(v[i]);
        }
        const int sb = scale_byte(m);
        *reinterpret_cast<uint4*>(out + b0 * 16) =
            make_uint4(codes8(f, sb), codes8(f + 8, sb), codes8(f + 16, sb), codes8(f + 24, sb));
        put_scale(g, out, uint32_t(b0), sb);
    } else {
        u16x2 m = {0, 0};
#pragma unroll
        for (int i = 0; i < kMxBlock; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
#pragma unroll
        for (int h = 0; h < R; h++) {
            const int sb = scale_byte(uint32_t(m[h]) << 16);
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                Eight<uint16_t> e;
#pragma unroll
                for (int j = 0; j < 4; j++)  // the row's half of two k
                    e.v[j] = __builtin_amdgcn_perm(v[8 * i + 2 * j + 1], v[8 * i + 2 * j], h ? 0x07060302u : 0x05040100u);
                q[i] = e.codes(sb);
            }
            *reinterpret_cast<uint4*>(out + (b0 + h * g.group) * 16) = make_uint4(q[0], q[1], q[2], q[3]);
            put_scale(g, out, uint32_t(b0 + h * g.group), sb);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize_cols(MxTiles g, const uint8_t* __restrict__ src, T* __restrict__ dst) {
    constexpr int R = sizeof(T) == 2 ? 2 : 1;
    typedef uint32_t u32_2 __attribute__((aligned(2)));
    const ColPos p = col_pos<R>(g);
    const int left = int(min(g.K - int64_t(p.kb) * kMxBlock, int64_t(kMxBlock)));
    if (p.t >= g.n || left <= 0) return;
    const int64_t sk = g.k.stride[0];
    T* at = dst + p.t * g.elems + int64_t(p.kb) * kMxBlock * sk + p.r;
    const uint8_t* in = src + p.t * g.bytes;
    const int64_t b0 = mx_block_of(uint32_t(g.rows), g.group, p.r, p.kb), scales = g.rows * g.blocks * 16;
    uint4 c[R];
    int sb[R];
#pragma unroll
    for (int h = 0; h < R; h++) {
        c[h] = *reinterpret_cast<const uint4*>(in + (b0 + h * g.group) * 16);
        sb[h] = in[scales + b0 + h * g.group];
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        float v[R][8];
#pragma unroll
        for (int h = 0; h < R; h++) {
            const uint32_t q[4] = {c[h].x, c[h].y, c[h].z, c[h].w};
            mx_values(q[i], sb[h], v[h]);
        }
#pragma unroll
        for (int j = 0; j < 8; j++) {
            if (8 * i + j >= left) return;
            if constexpr (R == 1) put(at, v[0][j]);
            else *reinterpret_cast<u32_2*>(at) = __builtin_amdgcn_perm(__float_as_uint(v[R - 1][j]), __float_as_uint(v[0][j]), 0x07060302u);
            at += sk;
        }
    }
}

MxTiles mx_tiles(const Plan& p, int op, int64_t n) {
    MxTiles g{};
    g.row = p.mx_row[op];
    g.k = p.mx_k[op];
    g.elems = p.tile_elems[op];
    g.rows = p.mx_rows[op];
    g.K = p.nK;
    g.blocks = p.mx_blocks;
    g.group = mx_group(g.blocks);
    g.bytes = p.mx_bytes[op];
    g.n = n;
    return g;
}

// ------------------------------------------------------------ contraction

// acc += A B for four blocks of 16 rows each (see above)
__device__ inline f32x4 mx_mfma(const i32x4& a, const i32x4& b, const f32x4& acc, uint32_t sa, uint32_t sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(i32x8{a[0], a[1], a[2], a[3], 0, 0, 0, 0},
                                                            i32x8{b[0], b[1], b[2], b[3], 0, 0, 0, 0}, acc, 4, 4, 0, int(sa),
                                                            0, int(sb));
}

// The same for two blocks of 32 rows each, their scales in byte SB of sa and sb.
template <int SB>
__device__ inline f32x16 mx_mfma32(const i32x4& a, const i32x4& b, const f32x16& acc, uint32_t sa, uint32_t sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(i32x8{a[0], a[1], a[2], a[3], 0, 0, 0, 0},
                                                           i32x8{b[0], b[1], b[2], b[3], 0, 0, 0, 0}, acc, 4, 4, SB, int(sa),
                                                           SB, int(sb));
}

struct MxArgs {
    const uint8_t *A, *B;
    const int32_t *pa, *pb;
    int64_t a_bytes, b_bytes;    // of a tile
    int32_t a_scales, b_scales;  // where a tile's scales begin
    int32_t M, N, blocks;        // rows of A and B to a batch index, blocks of a row
    int32_t a_rows, b_rows;      // of a tile
    int32_t m_blocks, n_blocks, wg_blocks;
    int32_t w_affine, w_bf16, batched;
    int32_t waves_n;             // k_mx: wavefronts of a workgroup side by side along N
    int64_t w_sm, w_sn, w_elems; // affine: W(m, n) at m w_sm + n w_sn
    const int32_t *tWM, *tWN, *tWB;
    const Unit* units;
    const int32_t* seg_start;    // not null: a unit to a key, its pairs from here
    const WsHeader* hdr;
    float* W;
    float* partials;
};

// (Keys out of order, which an asynchronous call reports in its counts, can
// leave segments that end before they begin or reach over others: none of them
// is a unit.)
__device__ inline bool mx_unit(const MxArgs& g, int64_t unit, Unit& u) {
    const int32_t err = g.hdr->err_u | g.hdr->err_v;
    const int64_t n_w = g.hdr->n_w, n_units = g.hdr->n_units;
    if (unit >= (g.seg_start ? err ? 0 : n_w : n_units)) return false;
    u = g.seg_start ? Unit{int32_t(unit), g.seg_start[unit], g.seg_start[unit + 1], -1} : g.units[unit];
    return u.p1 > u.p0;
}

// The sums of a wavefront's TM x TN tiles of S x S, whose first is at (m0, n0), to
// the output or partial tile.  The products are taken with B's rows as the
// instruction's first operand, so that a lane has four consecutive n of one row
// m at a time, and one store for them: sums 4 q .. 4 q + 3 are
// (lane % S, 4 lane / S + 256 q / S ..) of their tile.  (A store for each sum
// made the end of a 128 x 256 block take as long as 19 of its stages.)
template <int S, int TM, int TN, typename V>
__device__ inline void mx_store(const MxArgs& g, const Unit& u, int b, int m0, int n0, const V (&acc)[TM][TN]) {
    typedef uint32_t u32x2_2 __attribute__((ext_vector_type(2), aligned(2)));
    typedef float f32x4_4 __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int Q = S * S / 256;
    const int lane = threadIdx.x & 63;
    const int64_t base = (u.slot >= 0 ? int64_t(u.slot) : int64_t(u.seg)) * g.w_elems + (g.batched ? g.tWB[b] : 0);
    const bool half = g.w_bf16 && u.slot < 0;
    float* out = u.slot >= 0 ? g.partials : g.W;
#pragma unroll
    for (int i = 0; i < TM; i++) {
        const int m = m0 + S * i + (lane & (S - 1));
        if (m >= g.M) continue;
        const int64_t row = base + (g.w_affine ? m * g.w_sm : int64_t(g.tWM[m]));
        float* at = out + row;
        uint16_t* at16 = reinterpret_cast<uint16_t*>(out) + row;
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int q = 0; q < Q; q++) {
                const int n = n0 + S * j + 256 / S * q + lane / S * 4;
                const f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (g.w_affine && g.w_sn == 1 && n + 4 <= g.N) {
                    if (half)
                        *reinterpret_cast<u32x2_2*>(at16 + n) =
                            u32x2_2{uint32_t(f32_to_bf16_rne(v[0])) | uint32_t(f32_to_bf16_rne(v[1])) << 16,
                                    uint32_t(f32_to_bf16_rne(v[2])) | uint32_t(f32_to_bf16_rne(v[3])) << 16};
                    else
                        *reinterpret_cast<f32x4_4*>(at + n) = f32x4_4{v[0], v[1], v[2], v[3]};
                    continue;
                }
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    if (n + e >= g.N) continue;
                    const int64_t c = g.w_affine ? (n + e) * g.w_sn : int64_t(g.tWN[n + e]);
                    if (half) at16[c] = f32_to_bf16_rne(v[e]);
                    else at[c] = v[e];
                }
            }
    }
}

// An index list read by scalar loads: the compiler would take vector loads for
// one that the copies' assembly might write, and wait for the copies with them.
__device__ inline int32_t pair_index(const int32_t* list, int64_t i) {
    typedef const __attribute__((address_space(4))) int32_t* constant;
    return reinterpret_cast<constant>(reinterpret_cast<uintptr_t>(list))[i];
}

// Few rows on one side (M), or rows of one or two blocks: a wavefront has TM x TN
// tiles of 16 x 16 and reads its fragments from memory, a batch of steps (of
// four blocks) ahead of the one it multiplies.  g.waves_n wavefronts of a
// workgroup lie side by side along N; the others take every other step of the
// same tiles, and the first of them adds their sums in order.
//
// What bounds it is how much is on its way: one token against 32,768 rows of
// 4,096 values (71 MB) took 36 us a step at a time and takes 15 (4.6 TB/s) with
// batches of four in two tiles of 16 rows; of eight, or in one tile, 17 to 19.
//
// SHORT: rows of one or two blocks; a step is then the rows of four or two
// pairs, each lane's its own.  (5% dense blocks of 64 in 8,192 x 8,192 times 512
// columns: 14 us; of 32 in 4,096 x 4,096: 6.7.)
template <int TM, int TN, int U, bool SHORT>
__global__ __launch_bounds__(kThreads) void k_mx(MxArgs g) {
    __shared__ f32x4 sums[kWaves][TM * TN][64];
    const uint32_t wg = uint32_t(block_index()), unit = wg / uint32_t(g.wg_blocks);
    Unit u;
    if (!mx_unit(g, unit, u)) return;
    int x = int(wg - unit * g.wg_blocks);
    const int nb = x % g.n_blocks;
    x /= g.n_blocks;
    const int mb = x % g.m_blocks, b = x / g.m_blocks;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, gr = lane >> 4;
    const int wn = w % g.waves_n, wk = w / g.waves_n, deep = kWaves / g.waves_n;
    const int m0 = mb * 16 * TM, n0 = (nb * g.waves_n + wn) * 16 * TN;
    // a lane's rows: past the last they are the last (their sums are not written)
    const int per_row = SHORT ? g.blocks : 4;
    uint32_t ra[TM], rb[TN];
#pragma unroll
    for (int i = 0; i < TM; i++) ra[i] = uint32_t(b * g.M + min(m0 + 16 * i + r, g.M - 1)) * per_row + (SHORT ? gr & (per_row - 1) : gr);
#pragma unroll
    for (int j = 0; j < TN; j++) rb[j] = uint32_t(b * g.N + min(n0 + 16 * j + r, g.N - 1)) * per_row + (SHORT ? gr & (per_row - 1) : gr);
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int n_pairs = u.p1 - u.p0;
    const int steps = SHORT ? 1 : g.blocks / 4;                 // of a pair
    const int shift = SHORT ? 2 - (g.blocks >> 1) : 0;          // pairs of a step: 1 << shift
    const int64_t total = SHORT ? (int64_t(n_pairs) + (1 << shift) - 1) >> shift : int64_t(n_pairs) * steps;
    struct Batch {
        i32x4 a[U][TM], b[U][TN];
        uint32_t sa[U][TM], sb[U][TN];
    };
    // The batch's steps s, s + deep, ...: past the last one, the last again.
    auto load = [&](Batch& v, int64_t s) {
        int64_t ia[U], ib[U];
        int kk[U];
#pragma unroll
        for (int i = 0; i < U; i++) {
            const int64_t at = min(s + int64_t(i) * deep, total - 1);
            if constexpr (SHORT) {
                const int64_t p = u.p0 + min((at << shift) + (gr >> (2 - shift)), int64_t(n_pairs) - 1);
                ia[i] = g.pa[p];
                ib[i] = g.pb[p];
                kk[i] = 0;
            } else {
                const int p = int(at / steps);
                ia[i] = pair_index(g.pa, u.p0 + p);
                ib[i] = pair_index(g.pb, u.p0 + p);
                kk[i] = int(at - int64_t(p) * steps);
            }
        }
#pragma unroll
        for (int i = 0; i < U; i++) {
            const uint8_t* at = g.A + ia[i] * g.a_bytes + int64_t(kk[i]) * g.a_rows * 64;
            const uint8_t* bt = g.B + ib[i] * g.b_bytes + int64_t(kk[i]) * g.b_rows * 64;
            const uint8_t* as = g.A + ia[i] * g.a_bytes + g.a_scales + int64_t(kk[i]) * g.a_rows * 4;
            const uint8_t* bs = g.B + ib[i] * g.b_bytes + g.b_scales + int64_t(kk[i]) * g.b_rows * 4;
#pragma unroll
            for (int h = 0; h < TM; h++) {
                v.a[i][h] = *reinterpret_cast<const i32x4*>(at + ra[h] * 16);
                v.sa[i][h] = as[ra[h]];
            }
#pragma unroll
            for (int h = 0; h < TN; h++) {
                v.b[i][h] = *reinterpret_cast<const i32x4*>(bt + rb[h] * 16);
                v.sb[i][h] = bs[rb[h]];
            }
        }
    };
    auto multiply = [&](Batch& v, int64_t s) {
#pragma unroll
        for (int i = 0; i < U; i++) {
            const int64_t at = s + int64_t(i) * deep;
            if (at >= total) break;
            if constexpr (SHORT) {
                // (a pair past the last: zeros under a scale that is a number)
                const bool in = (at << shift) + (gr >> (2 - shift)) < n_pairs;
#pragma unroll
                for (int h = 0; h < TM; h++) {
                    v.a[i][h] = in ? v.a[i][h] : i32x4{0, 0, 0, 0};
                    v.sa[i][h] = in ? v.sa[i][h] : 0;
                }
#pragma unroll
                for (int h = 0; h < TN; h++) v.sb[i][h] = in ? v.sb[i][h] : 0;
            }
#pragma unroll
            for (int h = 0; h < TM; h++)
#pragma unroll
                for (int j = 0; j < TN; j++) acc[h][j] = mx_mfma(v.b[i][j], v.a[i][h], acc[h][j], v.sb[i][j], v.sa[i][h]);
        }
    };
    if (n0 < g.N) {
        Batch x0, x1;
        const int64_t stride = int64_t(U) * deep;
        int64_t s = wk;
        if (s < total) load(x0, s);
        for (; s < total; s += 2 * stride) {
            if (s + stride < total) load(x1, s + stride);
            multiply(x0, s);
            if (s + 2 * stride < total) load(x0, s + 2 * stride);
            if (s + stride < total) multiply(x1, s + stride);
        }
    }
    if (deep > 1) {
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++) sums[w][i * TN + j][lane] = acc[i][j];
        __syncthreads();
        if (wk > 0) return;
        for (int d = 1; d < deep; d++)
#pragma unroll
            for (int i = 0; i < TM; i++)
#pragma unroll
                for (int j = 0; j < TN; j++) acc[i][j] += sums[d * g.waves_n + wn][i * TN + j][lane];
    }
    if (n0 < g.N) mx_store<16>(g, u, b, m0, n0, acc);
}

// Rows of four blocks or more: 2 x 2 wavefronts, each with TM x TN tiles of
// 32 x 32 (v_mfma_scale_f32_32x32x64_f8f6f4: lane l holds block l / 32 of two of
// row l % 32, and sums (8 (i / 4) + 4 (l / 32) + i % 4, l % 32)), read their
// fragments from LDS.  A stage is one group of four blocks of every row of one
// pair, copied straight into LDS two stages ahead.
//
// A stage's codes are [row][4 blocks of 16 bytes], block k of row r in slot
// k ^ ((r >> 2) & 3): the lanes that read together then meet every bank
// once.  A row's four scale bytes are one dword; those of a lane's TM (TN) rows,
// which lie 32 rows apart, are side by side.
//
// A call of an 8192^3 product took, with its rows' quantisation and the join
// (60 us of it, then 50):
//   256 x 256 for the only workgroup of a CU, 16 x 16 tiles        533 us
//   128 x 256, two workgroups per CU: one's products cover what the
//   other waits for                                                503
//   tiles in groups of four blocks: a third of the L2's requests   385
//   all reads of a stage on their way before its first product     377
//   four sums to a store                                           340
//   no unit table                                                  325
// The kernel is then at 299 to 308 us, 3.57 to 3.68 PFLOP/s, at a clock of 1.86
// GHz (in traces whose launches follow each other up to 348 in the median; a
// stage 0.99 us for two workgroups, their starts and ends 12 us each).  With no copies in the loop
// 16 x 16 tiles took 240; registers alone do 6.6 PFLOP/s of random codes (power;
// 8.7 of zeros), so the wavefronts' waits for LDS and each other bound it.  A
// raised priority around the products, the copies issued after the reads, and
// other slots (the bank conflicts' third of the LDS time) changed it by 2% or
// less.
constexpr int kStages = 3;

__device__ inline int mx_slot(int r, int k) { return k ^ ((r >> 2) & 3); }

template <int TM, int TN>
constexpr int mx_stage_bytes() { return (64 * TM + 64 * TN) * 68; }

// Wavefronts of a SIMD that the sums leave room for.
template <int TM, int TN>
constexpr int mx_waves() { return TM * TN >= 8 ? 2 : TM * TN >= 4 ? 3 : 4; }

template <int TM, int TN>
__global__ __launch_bounds__(kThreads, (mx_waves<TM, TN>())) void k_mx_lds(MxArgs g) {
    extern __shared__ __align__(16) char lds[];
    constexpr int BM = 64 * TM, BN = 64 * TN, ROWS = BM + BN, kStage = mx_stage_bytes<TM, TN>();
    const uint32_t wg = uint32_t(block_index()), unit = wg / uint32_t(g.wg_blocks);
    Unit u;
    if (!mx_unit(g, unit, u)) return;
    int x = int(wg - unit * g.wg_blocks);
    const int nb = x % g.n_blocks;
    x /= g.n_blocks;
    const int mb = x % g.m_blocks, b = x / g.m_blocks;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, half = lane >> 5;
    const int wm = w >> 1, wn = w & 1;

    // this wavefront's copies of a stage: codes 16 rows at a time (64 of A to
    // the workgroup, then of B), scales 64 rows at a time.  Rows past the last
    // copy the last.
    constexpr int NC = ROWS / 64, NS = (ROWS / 64 + 3) / 4;
    auto row_of = [&](int row) {
        return row < BM ? b * g.M + min(mb * BM + row, g.M - 1) : b * g.N + min(nb * BN + row - BM, g.N - 1);
    };
    uint32_t voff[NC], vsc[NS];
#pragma unroll
    for (int i = 0; i < NC; i++) {
        const int row = i * 64 + w * 16 + (lane >> 2);
        voff[i] = uint32_t(row_of(row) * 4 + mx_slot(row, lane & 3)) * 16u;
    }
#pragma unroll
    for (int i = 0; i < NS; i++) {
        // position (half, r, tile) holds row 32 (tiles half + tile) + r
        const int p = min((w + 4 * i) * 64, ROWS - 64) + lane;
        const bool a = p < BM;
        const int T = a ? TM : TN, q = a ? p : p - BM, hf = q / (32 * T), rr = q % (32 * T) / T, t = q % T;
        vsc[i] = uint32_t(row_of((a ? 0 : BM) + (hf * T + t) * 32 + rr)) * 4u;
    }
    const uint32_t lds0 = lds_address(lds);
    const int steps = g.blocks / 4;  // stages of a pair
    const int64_t a_step = int64_t(g.a_rows) * 64, b_step = int64_t(g.b_rows) * 64;
    const int64_t total = int64_t(u.p1 - u.p0) * steps;
    // the next stage to copy: its codes and scales; the pair after its own is known
    const uint8_t *at, *bt, *as, *bs;
    auto set_pair = [&](int32_t a, int32_t bx) {
        at = g.A + a * g.a_bytes;
        bt = g.B + bx * g.b_bytes;
        as = at + g.a_scales;
        bs = bt + g.b_scales;
    };
    set_pair(pair_index(g.pa, u.p0), pair_index(g.pb, u.p0));
    int32_t after = min(u.p0 + 1, u.p1 - 1), left = steps;
    int32_t a_next = pair_index(g.pa, after), b_next = pair_index(g.pb, after);
    auto copy = [&](uint32_t l) {
#pragma unroll
        for (int i = 0; i < NC; i++) lds_copy16<false>(l + i * 4096 + w * 1024, i < TM ? at : bt, voff[i]);
#pragma unroll
        for (int i = 0; i < NS; i++) {
            const int p = (w + 4 * i) * 64;
            if (p < ROWS) lds_copy4(l + ROWS * 64 + p * 4, p < BM ? as : bs, vsc[i]);
        }
        at += a_step;
        bt += b_step;
        as += a_step / 16;
        bs += b_step / 16;
        if (--left == 0) {
            left = steps;
            set_pair(a_next, b_next);
            after = min(after + 1, u.p1 - 1);
            a_next = pair_index(g.pa, after);
            b_next = pair_index(g.pb, after);
        }
    };
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.f;
    copy(lds0);
    if (total > 1) copy(lds0 + kStage);
    // stage `now` is read while `then`, two on, is copied
    uint32_t now = 0, then = 2 * kStage;
    for (int64_t s = 0; s < total; s++) {
        // this stage's copies have landed once every wavefront has waited for
        // its own (the next stage's may be in flight); the barrier also says
        // that the stage before, whose place the copies below take, is read
        if (s + 1 < total) {
            if (ROWS / 64 == 4 * NS || w < ROWS / 64 % 4) lds_copy_wait<NC + NS>();
            else lds_copy_wait<NC + NS - 1>();
        } else {
            lds_copy_wait<0>();
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // no read of LDS moves up past it
        if (s + 2 < total) copy(lds0 + then);
        const char* l = lds + now;
        now = now == 2 * kStage ? 0 : now + kStage;
        then = then == 2 * kStage ? 0 : then + kStage;
        i32x4 fa[TM][2], fb[TN][2];
        uint32_t sa[TM], sb[TN];
#pragma unroll
        for (int i = 0; i < TM; i++) sa[i] = reinterpret_cast<const uint32_t*>(l + ROWS * 64)[wm * 32 * TM + r * TM + i];
#pragma unroll
        for (int j = 0; j < TN; j++) sb[j] = reinterpret_cast<const uint32_t*>(l + ROWS * 64)[BM + wn * 32 * TN + r * TN + j];
        // blocks half and 2 + half of the group
        const int sl[2] = {mx_slot(r, half) * 16, mx_slot(r, 2 + half) * 16};
#pragma unroll
        for (int k = 0; k < 2; k++) {
#pragma unroll
            for (int i = 0; i < TM; i++) fa[i][k] = *reinterpret_cast<const i32x4*>(l + ((wm * TM + i) * 32 + r) * 64 + sl[k]);
#pragma unroll
            for (int j = 0; j < TN; j++) fb[j][k] = *reinterpret_cast<const i32x4*>(l + (BM + (wn * TN + j) * 32 + r) * 64 + sl[k]);
        }
        // All reads are on their way before the first product: the compiler
        // would put each of B's in front of its products and wait for it there.
        // (An empty statement that uses a value and might touch memory: reads
        // stay in front of it.)
#pragma unroll
        for (int i = 0; i < TM; i++) {
            asm volatile("" : "+v"(sa[i])::"memory");
            sa[i] >>= 8 * half;  // bytes 0 and 2: the scales of the lane's two blocks
        }
#pragma unroll
        for (int j = 0; j < TN; j++) {
            asm volatile("" : "+v"(sb[j])::"memory");
            sb[j] >>= 8 * half;
        }
#pragma unroll
        for (int k = 0; k < 2; k++) {
#pragma unroll
            for (int i = 0; i < TM; i++) asm volatile("" : "+v"(fa[i][k])::"memory");
#pragma unroll
            for (int j = 0; j < TN; j++) {
                asm volatile("" : "+v"(fb[j][k])::"memory");
#pragma unroll
                for (int i = 0; i < TM; i++)
                    acc[i][j] = k ? mx_mfma32<2>(fb[j][k], fa[i][k], acc[i][j], sb[j], sa[i])
                                  : mx_mfma32<0>(fb[j][k], fa[i][k], acc[i][j], sb[j], sa[i]);
            }
        }
        lds_read_wait();
    }
    mx_store<32>(g, u, b, mb * BM + wm * 32 * TM, nb * BN + wn * 32 * TN, acc);
}

// How a plan's tiles are cut among workgroups.
struct MxShape {
    int64_t M, N;
    bool lds;
    int tm, tn;  // tiles of a wavefront, 32 x 32 from LDS, else 16 x 16
    int64_t m_blocks, n_blocks;
    bool turned = false;   // k_mx: A and B exchanged
    int waves_n = 1;
};

// The blocks that k_mx_lds is built for and what they take, in microseconds:
// `step` for a stage with every place on the chip taken, and `ends` for a
// workgroup's start and stores, from 8192 x 8192 outputs of 16 and 64 stages.
// (64 x 128 took 1.24 a stage, more than the same turned: not built.)  Of short
// keys that is too little: 128 keys of 128 x 1024 outputs and seven stages on
// average are 19 us by it, and 26 to 28 measured.
struct MxKind {
    int tm, tn, slots;
    double step, ends;
};
constexpr MxKind kMxKinds[] = {
    {2, 4, 512, 0.99, 11.8}, {2, 2, 768, 0.77, 8.9}, {2, 1, 1024, 0.73, 4.9}, {1, 4, 512, 0.67, 7.5}, {1, 1, 1536, 0.67, 3.3},
};
// A stage is taken to be no shorter than kMxStep, however few workgroups there
// are (of 64 x 64 outputs it measures 0.25 us with up to 64 of them on the chip,
// 0.34 with 512).
constexpr double kMxStep = 0.4, kMxAlone = 60;

double mx_rounds(double groups, int slots, double steps, double step, double ends) {
    const double whole = std::floor(groups / slots), rest = groups / slots - whole;
    return whole * (steps * step + ends) + (rest > 0 ? steps * std::max(kMxStep, step * rest) + ends : 0);
}

// The cut for `units` units of `steps` steps each, and its time.
MxShape mx_shape(const Plan& p, double units, double steps, double* time = nullptr) {
    MxShape h;
    h.M = p.swap ? p.nN : p.nM;
    h.N = p.swap ? p.nM : p.nN;
    h.lds = p.mx_blocks >= 4 && h.M > 32 && h.N > 32;
    double best = 0;
    if (h.lds) {
        for (const MxKind& k : kMxKinds) {
            const int64_t mb = (h.M + 64 * k.tm - 1) / (64 * k.tm), nb = (h.N + 64 * k.tn - 1) / (64 * k.tn);
            const double t = mx_rounds(units * double(p.nB * mb * nb), k.slots, steps, k.step, k.ends);
            if (best > 0 && t >= best) continue;
            best = t;
            h.tm = k.tm;
            h.tn = k.tn;
            h.m_blocks = mb;
            h.n_blocks = nb;
        }
        if (time) *time = best;
        return h;
    }
    // the longer side along N
    h.turned = h.M > h.N;
    if (h.turned) std::swap(h.M, h.N);
    h.tm = h.M > 16 ? 2 : 1;
    h.tn = h.N > 16 ? 2 : 1;
    h.waves_n = h.N > 32 * h.tn ? 4 : h.N > 16 * h.tn ? 2 : 1;
    h.m_blocks = (h.M + 16 * h.tm - 1) / (16 * h.tm);
    h.n_blocks = (h.N + 16 * h.tn * h.waves_n - 1) / (16 * h.tn * h.waves_n);
    // (a step of a wavefront about 0.4 us, a workgroup's start and end 5)
    if (time) *time = mx_rounds(units * double(p.nB * h.m_blocks * h.n_blocks), 512, std::ceil(steps * h.waves_n / kWaves), 0.4, 5.0);
    return h;
}

// Matrix instructions that a pair takes along its contracted index.
double mx_steps(const Plan& p) { return double(p.mx_blocks) / 4; }

template <int TM, int TN>
hipError_t run_lds(const MxArgs& g, dim3 grid, hipStream_t s) {
    constexpr int bytes = kStages * mx_stage_bytes<TM, TN>();
    // above 64 KB a kernel has to be allowed it, once per device
    if (bytes > 65536) {
        static std::atomic<uint64_t> allowed{0};
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
        if (!(allowed.load(std::memory_order_relaxed) & bit)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_mx_lds<TM, TN>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                    bytes);
            if (e != hipSuccess) return e;
            allowed.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    return launch_k(k_mx_lds<TM, TN>, grid, dim3{unsigned(kThreads)}, size_t(bytes), s, g);
}

template <int TM, int TN, int U>
hipError_t run_mx(bool few, const MxArgs& g, dim3 grid, hipStream_t s) {
    return few ? launch_k(k_mx<TM, TN, U / 2, true>, grid, dim3{unsigned(kThreads)}, 0, s, g)
               : launch_k(k_mx<TM, TN, U, false>, grid, dim3{unsigned(kThreads)}, 0, s, g);
}

template <int TM>
hipError_t run_lds_n(int tn, const MxArgs& g, dim3 grid, hipStream_t s) {
    if constexpr (TM == 2)
        if (tn == 2) return run_lds<TM, 2>(g, grid, s);
    return tn == 4 ? run_lds<TM, 4>(g, grid, s) : run_lds<TM, 1>(g, grid, s);
}

}  // namespace

namespace {

// How a tile is read or written: along its rows, across them, or element by element.
enum MxWay { MX_ROWS, MX_COLS, MX_ANY };
MxWay mx_way(const MxTiles& g) {
    if (g.k.n == 0 || (g.k.n == 1 && g.k.stride[0] == 1)) return MX_ROWS;
    if (g.k.n == 1 && g.row.n == 1 && g.row.stride[0] == 1) return MX_COLS;
    return MX_ANY;
}

// Workgroups for `items` of `per` to a workgroup.
dim3 mx_grid(int64_t items, int64_t per) { return grid_of((items + per - 1) / per); }

// The launch along rows of `eights` eights each.
dim3 rows_grid(MxTiles& g, int64_t eights) {
    g.lanes = 0;
    while (g.lanes < 6 && (1 << g.lanes) < eights) g.lanes++;
    // (a block's four eights are a quad of lanes)
    g.lanes = std::max(g.lanes, 2);
    g.line = Divisor((eights + (1 << g.lanes) - 1) >> g.lanes);
    g.tile = Divisor(g.rows);
    const int64_t rows = int64_t(kRun * kWaves) << (6 - g.lanes);
    return mx_grid((g.n * g.rows + rows - 1) / rows * g.line.d, 1);
}

// The launch across rows.
template <typename T>
dim3 cols_grid(MxTiles& g) {
    constexpr int R = sizeof(T) == 2 ? 2 : 1;
    const int64_t lines = (g.rows + R - 1) / R, groups = g.blocks / g.group;
    g.line = Divisor(lines);
    g.tile = Divisor(lines * groups);
    return mx_grid(g.n * lines * groups, 64 * (kWaves / g.group));
}

template <typename T>
hipError_t quantize(MxTiles g, const T* src, uint8_t* dst, hipStream_t s) {
    const MxWay way = mx_way(g);
    const dim3 grid = way == MX_ROWS   ? rows_grid(g, g.blocks * 4)
                          : way == MX_COLS ? cols_grid<T>(g)
                                           : mx_grid(g.n * g.rows * g.blocks, kThreads);
    if (way == MX_COLS) k_mx_quantize_cols<<<grid, kThreads, 0, s>>>(g, src, dst);
    else if (way == MX_ANY) k_mx_quantize<<<grid, kThreads, 0, s>>>(g, src, dst);
    else if (g.K == g.blocks * kMxBlock) k_mx_quantize_rows<T, RUN_FULL><<<grid, kThreads, 0, s>>>(g, src, dst);
    else if (g.K % 8 == 0) k_mx_quantize_rows<T, RUN_WHOLE><<<grid, kThreads, 0, s>>>(g, src, dst);
    else k_mx_quantize_rows<T, RUN_CUT><<<grid, kThreads, 0, s>>>(g, src, dst);
    return hipGetLastError();
}

template <typename T>
hipError_t dequantize(MxTiles g, const uint8_t* src, T* dst, hipStream_t s) {
    const MxWay way = mx_way(g);
    const dim3 grid = way == MX_ROWS   ? rows_grid(g, (g.K + 7) / 8)
                          : way == MX_COLS ? cols_grid<T>(g)
                                           : mx_grid(g.n * g.rows * g.blocks, kThreads);
    if (way == MX_COLS) k_mx_dequantize_cols<<<grid, kThreads, 0, s>>>(g, src, dst);
    else if (way == MX_ANY) k_mx_dequantize<<<grid, kThreads, 0, s>>>(g, src, dst);
    else if (g.K % 8 == 0) k_mx_dequantize_rows<T, false><<<grid, kThreads, 0, s>>>(g, src, dst);
    else k_mx_dequantize_rows<T, true><<<grid, kThreads, 0, s>>>(g, src, dst);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const Plan& p, int op, const void* tiles, int src_dtype, int64_t n, void* mx, hipStream_t s) {
    const MxTiles g = mx_tiles(p, op, n);
    uint8_t* out = static_cast<uint8_t*>(mx);
    return src_dtype == TRE_BF16 ? quantize(g, static_cast<const uint16_t*>(tiles), out, s)
                                 : quantize(g, static_cast<const float*>(tiles), out, s);
}

hipError_t launch_mx_dequantize(const Plan& p, int op, const void* mx, int64_t n, void* tiles, int dst_dtype, hipStream_t s) {
    const MxTiles g = mx_tiles(p, op, n);
    const uint8_t* in = static_cast<const uint8_t*>(mx);
    return dst_dtype == TRE_BF16 ? dequantize(g, in, static_cast<uint16_t*>(tiles), s)
                                 : dequantize(g, in, static_cast<float*>(tiles), s);
}

// Unit length: keys are cut where that shortens the launch by more than the
// partial tiles cost (written and read once, at about 4 TB/s, and a launch).
int64_t mx_unit_pairs(const Plan& p, int64_t n_pairs, int64_t n_w) {
    const double len = double(n_pairs) / double(std::max<int64_t>(n_w, 1));
    int64_t unit = std::max<int64_t>(n_pairs, 1);
    double best = 0;
    for (int c = 1; c <= 64 && c <= len; c++) {
        const double pairs = std::ceil(len / c);
        double t;
        mx_shape(p, double(n_w) * c, std::ceil(pairs * mx_steps(p)), &t);
        if (c > 1) t += 6.0 + double(n_w) * c * double(p.tile_elems[2]) * 8.0 / 4e6;
        if (c > 1 && t >= 0.95 * best) continue;
        best = t;
        if (c > 1) {
            unit = int64_t(pairs);
            continue;
        }
        // One key far longer than the others would be alone at the end: where
        // the labels allow one of more than kMxAlone, units end there (or at
        // the launch's own time, or twice the average).  Below that the unit
        // table and the partial sums' look in the outputs cost more (10 us)
        // than they save in most launches.
        const double step = kMxStep * mx_steps(p), most = std::max(kMxAlone, t);
        if (double(p.key_pairs_max) * step > most) unit = std::min(unit, int64_t(std::ceil(std::max(most / step, 2 * len))));
    }
    return unit;
}

// Whether a launch of one unit per key reads the join's segments instead of a
// unit table, which takes a launch of 8 us to write: that one gives the longest
// keys first, which keys of one length, or work of few rounds, do not need
// (128 keys of 5 to 13 pairs of 128 x 1024 outputs: 52 us without, 62 with).
constexpr double kMxTable = 100;
bool mx_whole_keys(const Plan& p, int64_t n_pairs, int64_t n_w) {
    if (p.n_join == 0 || n_pairs <= n_w) return true;
    double t;
    mx_shape(p, double(n_w), std::ceil(double(n_pairs) / double(std::max<int64_t>(n_w, 1)) * mx_steps(p)), &t);
    return t <= kMxTable;
}

namespace {

MxShape launch_shape(const Plan& p, int64_t n_pairs, int64_t unit_bound) {
    return mx_shape(p, double(unit_bound), std::ceil(double(n_pairs) / double(unit_bound) * mx_steps(p)));
}

}  // namespace

int32_t mx_block(const Plan& p, int64_t n_pairs, int64_t unit_bound) {
    const MxShape h = launch_shape(p, n_pairs, unit_bound);
    const int rows = h.lds ? 64 * h.tm : 16 * h.tm, cols = h.lds ? 64 * h.tn : 16 * h.tn * h.waves_n;
    return rows << 16 | cols;
}

hipError_t launch_mx(const Plan& p, const Layout& L, char* ws, const void* u_tiles, const void* v_tiles, float* w_tiles,
                     int64_t n_pairs, int64_t unit_bound, bool whole_keys, hipStream_t s) {
    const MxShape h = launch_shape(p, n_pairs, unit_bound);
    const int a = p.swap != h.turned ? 1 : 0, b = 1 - a;
    const int32_t* tb = reinterpret_cast<const int32_t*>(ws + L.tables);
    const int32_t* pairs[2] = {reinterpret_cast<const int32_t*>(ws + L.pu), reinterpret_cast<const int32_t*>(ws + L.pv)};
    const void* tiles[2] = {u_tiles, v_tiles};
    MxArgs g{};
    g.A = static_cast<const uint8_t*>(tiles[a]);
    g.B = static_cast<const uint8_t*>(tiles[b]);
    g.pa = pairs[a];
    g.pb = pairs[b];
    g.a_bytes = p.mx_bytes[a];
    g.b_bytes = p.mx_bytes[b];
    g.blocks = int32_t(p.mx_blocks);
    g.a_rows = int32_t(p.mx_rows[a]);
    g.b_rows = int32_t(p.mx_rows[b]);
    g.a_scales = int32_t(p.mx_rows[a] * p.mx_blocks * 16);
    g.b_scales = int32_t(p.mx_rows[b] * p.mx_blocks * 16);
    g.M = int32_t(h.M);
    g.N = int32_t(h.N);
    g.m_blocks = int32_t(h.m_blocks);
    g.n_blocks = int32_t(h.n_blocks);
    const int64_t wg = p.nB * h.m_blocks * h.n_blocks;
    if (wg > int64_t(0x7fffffff) || wg * unit_bound > int64_t(0x7fffffff)) return hipErrorInvalidConfiguration;
    g.wg_blocks = int32_t(wg);
    g.w_affine = p.tile_w_affine;
    g.w_sm = h.turned ? 1 : p.tile_w_sm;
    g.w_sn = h.turned ? p.tile_w_sm : 1;
    g.waves_n = h.waves_n;
    g.w_bf16 = p.opt.w_bf16;
    g.batched = p.nB > 1;
    g.w_elems = p.tile_elems[2];
    g.tWM = tb + p.table_off[h.turned ? T_WN : T_WM];
    g.tWN = tb + p.table_off[h.turned ? T_WM : T_WN];
    g.tWB = tb + p.table_off[T_WB];
    g.units = reinterpret_cast<const Unit*>(ws + L.unit_desc);
    g.seg_start = whole_keys ? reinterpret_cast<const int32_t*>(ws + L.seg_start) : nullptr;
    g.hdr = reinterpret_cast<const WsHeader*>(ws + L.hdr);
    g.W = w_tiles;
    g.partials = reinterpret_cast<float*>(ws + L.partials);
    const dim3 grid = grid_of(wg * unit_bound);
    if (h.lds)
        return h.tm == 2 ? run_lds_n<2>(h.tn, g, grid, s) : run_lds_n<1>(h.tn, g, grid, s);
    const bool few = p.mx_blocks < 4;
    // (of two rows of tiles there are two columns too: the longer side is N)
    if (h.tm == 2) return run_mx<2, 2, 4>(few, g, grid, s);
    return h.tn == 2 ? run_mx<1, 2, 4>(few, g, grid, s) : run_mx<1, 1, 4>(few, g, grid, s);
}

}  // namespace tre
