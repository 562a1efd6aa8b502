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

namespace tre {

namespace {

constexpr int kThreads = 256;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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

// ---- any layout: a thread per block

template <typename T>
__global__ __launch_bounds__(kThreads) void k_mx_quantize(MxTiles g, const T* __restrict__ src, uint8_t* __restrict__ dst) {
    const int64_t b = int64_t(blockIdx.x) * kThreads + threadIdx.x;
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
    *reinterpret_cast<uint4*>(out + x * 16) = make_uint4(q[0], q[1], q[2], q[3]);
    out[per * 16 + x] = uint8_t(sb);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize(MxTiles g, const uint8_t* __restrict__ src, T* __restrict__ dst) {
    const int64_t b = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t per = g.rows * g.blocks;
    if (b >= g.n * per) return;
    const int64_t t = b / per, x = b - t * per, r = x / g.blocks, k0 = (x - r * g.blocks) * kMxBlock;
    const uint8_t* in = src + t * g.bytes;
    const uint4 c = *reinterpret_cast<const uint4*>(in + x * 16);
    const uint32_t q[4] = {c.x, c.y, c.z, c.w};
    const int sb = in[per * 16 + x];
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

// The eights of a workgroup: kRun * kThreads consecutive ones, g.line to a row
// and g.tile to a tile, the first found in 64 bits and the others from it in 32.
struct RunPos {
    int64_t t0;
    uint32_t w0;
};
__device__ inline RunPos run_pos(const MxTiles& g) {
    const int64_t q = int64_t(blockIdx.x) * (kRun * kThreads), t = q / g.tile.d;
    return RunPos{t, uint32_t(q - t * g.tile.d)};
}

// How a row's eights lie in the unquantised tile: one after the other through
// the whole tile; whole, but rows begin anywhere or end in zeros; the last cut.
enum RunKind { RUN_LINEAR, RUN_WHOLE, RUN_CUT };

template <typename T, RunKind KIND>
__global__ __launch_bounds__(kThreads) void k_mx_quantize_rows(MxTiles g, const T* __restrict__ src, uint8_t* __restrict__ dst) {
    const RunPos p = run_pos(g);
    const int64_t scales = g.rows * g.blocks * 16;
    Eight<T> v[kRun];
    uint32_t dt[kRun], w[kRun];  // tile after the first, eight in the tile
    bool in[kRun];
#pragma unroll
    for (int i = 0; i < kRun; i++) {
        const uint32_t x = p.w0 + i * kThreads + threadIdx.x;
        dt[i] = g.tile.of(x);
        w[i] = x - dt[i] * g.tile.d;
        in[i] = p.t0 + dt[i] < g.n;
        // (past the last tile: the first tile again, not written)
        const T* at = src + (p.t0 + (in[i] ? dt[i] : 0)) * g.elems;
        if constexpr (KIND == RUN_LINEAR) {
            v[i].load(at + uint64_t(w[i]) * 8, 8);
        } else {
            const uint32_t r = g.line.of(w[i]), k = (w[i] - r * g.line.d) * 8;
            at += g.row.n <= 1 ? int64_t(r) * g.row.stride[0] : offset_of(g.row, r);
            if constexpr (KIND == RUN_WHOLE) v[i].load_or_zero(at, k, uint32_t(g.K));
            else v[i].load(at + k, g.K - k);
        }
    }
#pragma unroll
    for (int i = 0; i < kRun; i++) {
        const int sb = scale_byte(quad_max(v[i].top()));
        if (!in[i]) continue;
        uint8_t* out = dst + (p.t0 + dt[i]) * g.bytes;
        *reinterpret_cast<uint32_t*>(out + uint64_t(w[i]) * 4) = v[i].codes(sb);
        if ((w[i] & 3) == 0) out[scales + w[i] / 4] = uint8_t(sb);
    }
}

// (g.line: the eights of a row that reach into K; blocks past it are not read)
template <typename T, bool CUT>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize_rows(MxTiles g, const uint8_t* __restrict__ src, T* __restrict__ dst) {
    const RunPos p = run_pos(g);
    const int64_t scales = g.rows * g.blocks * 16;
    uint32_t q[kRun], dt[kRun], r[kRun], k[kRun];
    int sb[kRun];
    bool in[kRun];
#pragma unroll
    for (int i = 0; i < kRun; i++) {
        const uint32_t x = p.w0 + i * kThreads + threadIdx.x;
        dt[i] = g.tile.of(x);
        const uint32_t w = x - dt[i] * g.tile.d;
        in[i] = p.t0 + dt[i] < g.n;
        r[i] = g.line.of(w);
        k[i] = (w - r[i] * g.line.d) * 8;
        const uint8_t* at = src + (p.t0 + (in[i] ? dt[i] : 0)) * g.bytes;
        const uint32_t b = r[i] * uint32_t(g.blocks) + k[i] / kMxBlock;
        q[i] = *reinterpret_cast<const uint32_t*>(at + uint64_t(b) * 16 + (k[i] % kMxBlock) / 2);
        sb[i] = at[scales + b];
    }
#pragma unroll
    for (int i = 0; i < kRun; i++) {
        if (!in[i]) continue;
        T* out = dst + (p.t0 + dt[i]) * g.elems + (g.row.n <= 1 ? int64_t(r[i]) * g.row.stride[0] : offset_of(g.row, r[i])) + k[i];
        float v[8];
        mx_values(q[i], sb[i], v);
        if (!CUT || g.K - k[i] >= 8) {
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
                if (k[i] + j < g.K) put(out + j, v[j]);
        }
    }
}

// ---- the rows consecutive in the tile (two or more: of one row the contracted
// index is consecutive): a thread per block of one fp32 row or two bf16 rows,
// so that lanes side by side read consecutive rows of one k.  The last of an
// odd number of bf16 rows goes with the row before it once more.

// A thread's tile, block and first row; g.line: lines (of R rows) of a tile,
// g.tile: lines and blocks.
struct ColPos {
    int64_t t;
    uint32_t kb, r;
};
template <int R>
__device__ inline ColPos col_pos(const MxTiles& g) {
    const int64_t x0 = int64_t(blockIdx.x) * kThreads, t0 = x0 / g.tile.d;
    const uint32_t x = uint32_t(x0 - t0 * g.tile.d) + threadIdx.x, dt = g.tile.of(x), w = x - dt * g.tile.d;
    ColPos p;
    p.t = t0 + dt;
    p.kb = g.line.of(w);
    p.r = min((w - p.kb * g.line.d) * R, uint32_t(g.rows) - R);
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
    const int64_t b0 = int64_t(p.r) * g.blocks + p.kb, scales = g.rows * g.blocks * 16;
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
        out[scales + b0] = uint8_t(sb);
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
            *reinterpret_cast<uint4*>(out + (b0 + h * g.blocks) * 16) = make_uint4(q[0], q[1], q[2], q[3]);
            out[scales + b0 + h * g.blocks] = uint8_t(sb);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize_cols(MxTiles g, const uint8_t* __restrict__ src, T* __restrict__ dst) {
    constexpr int R = sizeof(T) == 2 ? 2 : 1;
    typedef uint32_t u32_2 __attribute__((aligned(2)));
    const ColPos p = col_pos<R>(g);
    if (p.t >= g.n) return;
    const int left = int(min(g.K - int64_t(p.kb) * kMxBlock, int64_t(kMxBlock)));
    const int64_t sk = g.k.stride[0];
    T* at = dst + p.t * g.elems + int64_t(p.kb) * kMxBlock * sk + p.r;
    const uint8_t* in = src + p.t * g.bytes;
    const int64_t b0 = int64_t(p.r) * g.blocks + p.kb, scales = g.rows * g.blocks * 16;
    uint4 c[R];
    int sb[R];
#pragma unroll
    for (int h = 0; h < R; h++) {
        c[h] = *reinterpret_cast<const uint4*>(in + (b0 + h * g.blocks) * 16);
        sb[h] = in[scales + b0 + h * g.blocks];
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
    g.bytes = p.mx_bytes[op];
    g.n = n;
    return g;
}

// ------------------------------------------------------------ contraction

struct MxArgs {
    const uint8_t *A, *B;
    const int32_t *pa, *pb;
    int64_t a_bytes, b_bytes;    // of a tile
    int32_t a_scales, b_scales;  // where a tile's scales begin
    int32_t M, N, blocks;        // rows of A and B to a batch index, blocks of a row
    int32_t m_blocks, n_blocks, wg_blocks;
    int32_t w_affine, w_bf16, batched;
    int64_t w_sm, w_elems;
    const int32_t *tWM, *tWN, *tWB;
    const Unit* units;
    const WsHeader* hdr;
    float* W;
    float* partials;
};

// The sums of a wavefront's TM x TN tiles, whose first is at (m0, n0), to the
// output or partial tile.
template <int TM, int TN>
__device__ inline void mx_store(const MxArgs& g, const Unit& u, int b, int m0, int n0, const f32x4 (&acc)[TM][TN]) {
    const int lane = threadIdx.x & 63, r = lane & 15, gr = lane >> 4;
    const int64_t base = (u.slot >= 0 ? int64_t(u.slot) : int64_t(u.seg)) * g.w_elems + (g.batched ? g.tWB[b] : 0);
    const bool half = g.w_bf16 && u.slot < 0;
    float* out = u.slot >= 0 ? g.partials : g.W;
    int32_t col[TN];
    bool in[TN];
#pragma unroll
    for (int j = 0; j < TN; j++) {
        const int n = n0 + 16 * j + r;
        in[j] = n < g.N;
        col[j] = g.w_affine || !in[j] ? n : g.tWN[n];
    }
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int m = m0 + 16 * i + 4 * gr + e;
            if (m >= g.M) continue;
            const int64_t row = base + (g.w_affine ? m * g.w_sm : int64_t(g.tWM[m]));
            if (half) {
                uint16_t* at = reinterpret_cast<uint16_t*>(out) + row;
#pragma unroll
                for (int j = 0; j < TN; j++)
                    if (in[j]) at[col[j]] = f32_to_bf16_rne(acc[i][j][e]);
            } else {
                float* at = out + row;
#pragma unroll
                for (int j = 0; j < TN; j++)
                    if (in[j]) at[col[j]] = acc[i][j][e];
            }
        }
}

// Four wavefronts side by side along N, each with TM x TN tiles of 16 x 16.
template <int TM, int TN>
__global__ __launch_bounds__(kThreads) void k_mx(MxArgs g) {
    const int64_t unit = blockIdx.x / g.wg_blocks;
    if (unit >= g.hdr->n_units) return;
    const Unit u = g.units[unit];
    int x = int(blockIdx.x - unit * g.wg_blocks);
    const int nb = x % g.n_blocks;
    x /= g.n_blocks;
    const int mb = x % g.m_blocks, b = x / g.m_blocks;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, gr = lane >> 4;
    const int m0 = mb * 16 * TM, n0 = (nb * 4 + w) * 16 * TN;
    if (n0 >= g.N) return;
    // rows past the last read the last (their sums are not written)
    int32_t ra[TM], rb[TN];
#pragma unroll
    for (int i = 0; i < TM; i++) ra[i] = (b * g.M + min(m0 + 16 * i + r, g.M - 1)) * g.blocks;
#pragma unroll
    for (int j = 0; j < TN; j++) rb[j] = (b * g.N + min(n0 + 16 * j + r, g.N - 1)) * g.blocks;
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // the unit's blocks one pair after the other, four to an instruction
    const int64_t total = int64_t(u.p1 - u.p0) * g.blocks;
    for (int64_t q0 = 0; q0 < total; q0 += 4) {
        const int64_t q = q0 + gr;
        const bool in = q < total;
        const int64_t pair = in ? q / g.blocks : 0;
        const int kb = in ? int(q - pair * g.blocks) : 0;
        const uint8_t* at = g.A + g.pa[u.p0 + pair] * g.a_bytes;
        const uint8_t* bt = g.B + g.pb[u.p0 + pair] * g.b_bytes;
        i32x8 fa[TM], fb[TN];
        int sa[TM], sb[TN];
#pragma unroll
        for (int i = 0; i < TM; i++) {
            const uint4 c = *reinterpret_cast<const uint4*>(at + int64_t(ra[i] + kb) * 16);
            fa[i] = in ? i32x8{int(c.x), int(c.y), int(c.z), int(c.w), 0, 0, 0, 0} : i32x8{};
            sa[i] = in ? at[g.a_scales + ra[i] + kb] : 0;
        }
#pragma unroll
        for (int j = 0; j < TN; j++) {
            const uint4 c = *reinterpret_cast<const uint4*>(bt + int64_t(rb[j] + kb) * 16);
            fb[j] = in ? i32x8{int(c.x), int(c.y), int(c.z), int(c.w), 0, 0, 0, 0} : i32x8{};
            sb[j] = in ? bt[g.b_scales + rb[j] + kb] : 0;
        }
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[i], fb[j], acc[i][j], 4, 4, 0, sa[i], 0, sb[j]);
    }
    mx_store(g, u, b, m0, n0, acc);
}

// Rows of four blocks or more: 2 x 2 wavefronts, each with TM x TN tiles, read
// their fragments from LDS.  A stage is four blocks of every row of one pair,
// copied straight into LDS two stages ahead.
//
// A stage's codes are [row][4 blocks of 16 bytes], block k of row r in slot
// k ^ ((r >> 1 ^ r >> 3) & 3): the eight or sixteen lanes that read together
// then meet every bank once.  A row's four scale bytes are one dword; those of
// a lane's TM (TN) rows, which lie 16 rows apart, are side by side.
constexpr int kStages = 3;

// An index list read by scalar loads: the compiler would take vector loads for
// one that the copies' assembly might write, and wait for the copies with them.
__device__ inline int32_t pair_index(const int32_t* list, int64_t i) {
    typedef const __attribute__((address_space(4))) int32_t* constant;
    return reinterpret_cast<constant>(reinterpret_cast<uintptr_t>(list))[i];
}

__device__ inline int mx_slot(int r, int k) { return k ^ ((r >> 1 ^ r >> 3) & 3); }

template <int TM, int TN>
constexpr int mx_stage_bytes() { return (32 * TM + 32 * TN) * 68; }

template <int TM, int TN>
__global__ __launch_bounds__(kThreads) void k_mx_lds(MxArgs g) {
    extern __shared__ __align__(16) char lds[];
    constexpr int BM = 32 * TM, BN = 32 * TN, ROWS = BM + BN, kStage = mx_stage_bytes<TM, TN>();
    const int64_t unit = blockIdx.x / g.wg_blocks;
    if (unit >= g.hdr->n_units) return;
    const Unit u = g.units[unit];
    int x = int(blockIdx.x - unit * g.wg_blocks);
    const int nb = x % g.n_blocks;
    x /= g.n_blocks;
    const int mb = x % g.m_blocks, b = x / g.m_blocks;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, gr = lane >> 4;
    const int wm = w >> 1, wn = w & 1;
    const int steps = g.blocks / 4;  // stages of a pair

    // this wavefront's copies of a stage: codes 16 rows at a time (A's rows,
    // then B's), scales 64 at a time.  Rows past the last copy the last.
    constexpr int NC = ROWS / 16 / 4, NS = (ROWS / 64 + 3) / 4;
    static_assert(ROWS % 64 == 0, "a wavefront copies whole groups of rows");
    auto row_of = [&](int row) {
        return row < BM ? b * g.M + min(mb * BM + row, g.M - 1) : b * g.N + min(nb * BN + row - BM, g.N - 1);
    };
    uint32_t voff[NC], vsc[NS];
#pragma unroll
    for (int i = 0; i < NC; i++) {
        const int row = (w + 4 * i) * 16 + (lane >> 2);
        voff[i] = uint32_t(row_of(row) * g.blocks + mx_slot(row & 15, lane & 3)) * 16u;
    }
#pragma unroll
    for (int i = 0; i < NS; i++) {
        // position (half, r, tile) holds row 16 (tiles half + tile) + r
        const int p = min((w + 4 * i) * 64, ROWS - 64) + lane;
        const bool a = p < BM;
        const int T = a ? TM : TN, q = a ? p : p - BM, half = q / (16 * T), rr = q % (16 * T) / T, t = q % T;
        vsc[i] = uint32_t(row_of((a ? 0 : BM) + (half * T + t) * 16 + rr) * g.blocks);
    }
    const uint32_t lds0 = lds_address(lds);
    const int64_t total = int64_t(u.p1 - u.p0) * steps;
    // where the next stage to copy begins; the pair after its own is known
    int64_t pair = u.p0;
    int step = 0;
    const uint8_t *at = g.A + pair_index(g.pa, pair) * g.a_bytes, *bt = g.B + pair_index(g.pb, pair) * g.b_bytes;
    int64_t after = min(pair + 1, int64_t(u.p1) - 1);
    int32_t a_next = pair_index(g.pa, after), b_next = pair_index(g.pb, after);
    auto copy = [&](int slot) {
        const uint32_t l = lds0 + uint32_t(slot) * kStage;
#pragma unroll
        for (int i = 0; i < NC; i++) {
            const int rows = (w + 4 * i) * 16;
            lds_copy16<false>(l + rows * 64, (rows < BM ? at : bt) + step * 64, voff[i]);
        }
#pragma unroll
        for (int i = 0; i < NS; i++) {
            const int p = (w + 4 * i) * 64;
            if (p < ROWS) lds_copy4(l + ROWS * 64 + p * 4, (p < BM ? at + g.a_scales : bt + g.b_scales) + step * 4, vsc[i]);
        }
        if (++step == steps) {
            step = 0;
            at = g.A + a_next * g.a_bytes;
            bt = g.B + b_next * g.b_bytes;
            after = min(after + 1, int64_t(u.p1) - 1);
            a_next = pair_index(g.pa, after);
            b_next = pair_index(g.pb, after);
        }
    };
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    copy(0);
    if (total > 1) copy(1);
    int now = 0;
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
        const int then = now >= 1 ? now - 1 : now + 2;  // (now + 2) % 3
        if (s + 2 < total) copy(then);
        const char* l = lds + now * kStage;
        now = now == 2 ? 0 : now + 1;
        i32x8 fa[TM], fb[TN];
        uint32_t sa[TM], sb[TN];
        const int sl = mx_slot(r, gr) * 16;
#pragma unroll
        for (int i = 0; i < TM; i++) {
            const uint4 c = *reinterpret_cast<const uint4*>(l + ((wm * TM + i) * 16 + r) * 64 + sl);
            fa[i] = i32x8{int(c.x), int(c.y), int(c.z), int(c.w), 0, 0, 0, 0};
            sa[i] = reinterpret_cast<const uint32_t*>(l + ROWS * 64)[wm * 16 * TM + r * TM + i] >> (8 * gr);
        }
#pragma unroll
        for (int j = 0; j < TN; j++) {
            const uint4 c = *reinterpret_cast<const uint4*>(l + (BM + (wn * TN + j) * 16 + r) * 64 + sl);
            fb[j] = i32x8{int(c.x), int(c.y), int(c.z), int(c.w), 0, 0, 0, 0};
            sb[j] = reinterpret_cast<const uint32_t*>(l + ROWS * 64)[BM + wn * 16 * TN + r * TN + j] >> (8 * gr);
        }
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int i = 0; i < TM; i++)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[i], fb[j], acc[i][j], 4, 4, 0, int(sa[i]), 0,
                                                                             int(sb[j]));
        lds_read_wait();
    }
    mx_store(g, u, b, mb * BM + wm * 16 * TM, nb * BN + wn * 16 * TN, acc);
}

// How a plan's tiles are cut among workgroups.
struct MxShape {
    int64_t M, N;
    bool lds;
    int tm, tn;  // 16 x 16 tiles of a wavefront
    int64_t m_blocks, n_blocks;
};

MxShape mx_shape(const Plan& p) {
    MxShape h;
    h.M = p.swap ? p.nN : p.nM;
    h.N = p.swap ? p.nM : p.nN;
    h.lds = p.mx_blocks >= 4 && h.M > 32 && h.N > 32;
    if (h.lds) {
        // of 256, 128 or 64 rows the one that leaves the fewest places empty, the larger of two alike
        auto cut = [](int64_t n) {
            int best = 8;
            for (int t : {4, 2})
                if ((n + 32 * t - 1) / (32 * t) * t < (n + 32 * best - 1) / (32 * best) * best) best = t;
            return best;
        };
        h.tm = cut(h.M);
        h.tn = cut(h.N);
        h.m_blocks = (h.M + 32 * h.tm - 1) / (32 * h.tm);
        h.n_blocks = (h.N + 32 * h.tn - 1) / (32 * h.tn);
        return h;
    }
    h.tm = h.M > 32 ? 4 : h.M > 16 ? 2 : 1;
    h.tn = h.N > 64 ? 2 : 1;
    h.m_blocks = (h.M + 16 * h.tm - 1) / (16 * h.tm);
    h.n_blocks = (h.N + 64 * h.tn - 1) / (64 * h.tn);
    return h;
}

template <int TM, int TN>
hipError_t run_lds(const MxArgs& g, dim3 grid, hipStream_t s) {
    constexpr int bytes = kStages * mx_stage_bytes<TM, TN>();
    // above 64 KB the kernel has to be told once per device (here: per call, a host-side note)
    if (bytes > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_mx_lds<TM, TN>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    return launch_k(k_mx_lds<TM, TN>, grid, dim3{unsigned(kThreads)}, size_t(bytes), s, g);
}

template <int TM>
hipError_t run_lds_n(int tn, const MxArgs& g, dim3 grid, hipStream_t s) {
    return tn == 8 ? run_lds<TM, 8>(g, grid, s) : tn == 4 ? run_lds<TM, 4>(g, grid, s) : run_lds<TM, 2>(g, grid, s);
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

// Workgroups for `items` of `per` to a workgroup, 0 if they are too many.
unsigned mx_grid(int64_t items, int64_t per) {
    const int64_t b = (items + per - 1) / per;
    return b > int64_t(0x7fffffff) ? 0u : unsigned(b);
}

// Threads to a tile across its rows, and where they stand.
template <typename T>
int64_t col_threads(MxTiles& g, int64_t blocks) {
    constexpr int R = sizeof(T) == 2 ? 2 : 1;
    const int64_t lines = (g.rows + R - 1) / R;
    g.line = Divisor(lines);
    g.tile = Divisor(lines * blocks);
    return lines * blocks;
}

template <typename T>
hipError_t quantize(MxTiles g, const T* src, uint8_t* dst, hipStream_t s) {
    const MxWay way = mx_way(g);
    if (way == MX_ROWS) {
        g.line = Divisor(g.blocks * 4);
        g.tile = Divisor(g.rows * g.blocks * 4);
        const unsigned grid = mx_grid(g.n * g.rows * g.blocks * 4, kRun * kThreads);
        if (!grid) return hipErrorInvalidConfiguration;
        const bool side_by_side = g.row.n == 0 || (g.row.n == 1 && g.row.stride[0] == g.K);
        if (side_by_side && g.K == g.blocks * kMxBlock) k_mx_quantize_rows<T, RUN_LINEAR><<<grid, kThreads, 0, s>>>(g, src, dst);
        else if (g.K % 8 == 0) k_mx_quantize_rows<T, RUN_WHOLE><<<grid, kThreads, 0, s>>>(g, src, dst);
        else k_mx_quantize_rows<T, RUN_CUT><<<grid, kThreads, 0, s>>>(g, src, dst);
    } else {
        const unsigned grid = mx_grid(g.n * (way == MX_COLS ? col_threads<T>(g, g.blocks) : g.rows * g.blocks), kThreads);
        if (!grid) return hipErrorInvalidConfiguration;
        if (way == MX_COLS) k_mx_quantize_cols<<<grid, kThreads, 0, s>>>(g, src, dst);
        else k_mx_quantize<<<grid, kThreads, 0, s>>>(g, src, dst);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t dequantize(MxTiles g, const uint8_t* src, T* dst, hipStream_t s) {
    const MxWay way = mx_way(g);
    if (way == MX_ROWS) {
        const int64_t line = (g.K + 7) / 8;
        g.line = Divisor(line);
        g.tile = Divisor(g.rows * line);
        const unsigned grid = mx_grid(g.n * g.rows * line, kRun * kThreads);
        if (!grid) return hipErrorInvalidConfiguration;
        if (g.K % 8 == 0) k_mx_dequantize_rows<T, false><<<grid, kThreads, 0, s>>>(g, src, dst);
        else k_mx_dequantize_rows<T, true><<<grid, kThreads, 0, s>>>(g, src, dst);
    } else {
        const unsigned grid = mx_grid(
            g.n * (way == MX_COLS ? col_threads<T>(g, (g.K + kMxBlock - 1) / kMxBlock) : g.rows * g.blocks), kThreads);
        if (!grid) return hipErrorInvalidConfiguration;
        if (way == MX_COLS) k_mx_dequantize_cols<<<grid, kThreads, 0, s>>>(g, src, dst);
        else k_mx_dequantize<<<grid, kThreads, 0, s>>>(g, src, dst);
    }
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

int64_t mx_blocks_per_unit(const Plan& p) {
    const MxShape h = mx_shape(p);
    return p.nB * h.m_blocks * h.n_blocks;
}

hipError_t launch_mx(const Plan& p, const Layout& L, char* ws, const void* u_tiles, const void* v_tiles, float* w_tiles,
                     int64_t n_pairs, int64_t unit_bound, hipStream_t s) {
    (void)n_pairs;
    const MxShape h = mx_shape(p);
    const int a = p.swap ? 1 : 0, b = 1 - a;
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
    g.w_sm = p.tile_w_sm;
    g.w_bf16 = p.opt.w_bf16;
    g.batched = p.nB > 1;
    g.w_elems = p.tile_elems[2];
    g.tWM = tb + p.table_off[T_WM];
    g.tWN = tb + p.table_off[T_WN];
    g.tWB = tb + p.table_off[T_WB];
    g.units = reinterpret_cast<const Unit*>(ws + L.unit_desc);
    g.hdr = reinterpret_cast<const WsHeader*>(ws + L.hdr);
    g.W = w_tiles;
    g.partials = reinterpret_cast<float*>(ws + L.partials);
    const dim3 grid{unsigned(wg * unit_bound)}, block{unsigned(kThreads)};
    if (h.lds)
        return h.tm == 8 ? run_lds_n<8>(h.tn, g, grid, s) : h.tm == 4 ? run_lds_n<4>(h.tn, g, grid, s) : run_lds_n<2>(h.tn, g, grid, s);
    if (h.tm == 4)
        return h.tn == 2 ? launch_k(k_mx<4, 2>, grid, block, 0, s, g) : launch_k(k_mx<4, 1>, grid, block, 0, s, g);
    if (h.tm == 2)
        return h.tn == 2 ? launch_k(k_mx<2, 2>, grid, block, 0, s, g) : launch_k(k_mx<2, 1>, grid, block, 0, s, g);
    return h.tn == 2 ? launch_k(k_mx<1, 2>, grid, block, 0, s, g) : launch_k(k_mx<1, 1>, grid, block, 0, s, g);
}

}  // namespace tre
