// Tiles in microscaled 4-bit floating point: quantisation, reading back and
// the contraction of matched pairs on the scaled MFMA.
//
// A block is 32 values of the contracted index.  With m its largest magnitude,
//   e = floor(log2 m) - 2 (at least -127),  q = round(x / 2^e) to E2M1,
// and W[m,n] += sum over blocks of 2^(eA + eB) sum_k qA qB, which
// v_mfma_scale_f32_16x16x128_f8f6f4 does for four blocks at a time: lane l
// holds the 32 codes (16 bytes) and the scale byte of row l % 16, block l / 16,
// of either operand, and element (4 (l / 16) + i, l % 16) of the sums.
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

// An operand's tiles before and after.
struct MxTiles {
    Dims row, k;
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

// A thread per block.
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
    // (the conversion takes its scale from the exponent field alone: 0 is 2^-127)
    const float s = __uint_as_float(uint32_t(sb) << 23);
    uint32_t q[4] = {0, 0, 0, 0};
    if (sb != kMxNanScale) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[i], v[8 * i], v[8 * i + 1], s, 0);
            q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[i], v[8 * i + 2], v[8 * i + 3], s, 1);
            q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[i], v[8 * i + 4], v[8 * i + 5], s, 2);
            q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[i], v[8 * i + 6], v[8 * i + 7], s, 3);
        }
    }
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
    const int64_t base = (u.slot >= 0 ? int64_t(u.slot) : int64_t(u.seg)) * g.w_elems + (g.batched ? g.tWB[b] : 0);
    const bool half = g.w_bf16 && u.slot < 0;
    float* out = u.slot >= 0 ? g.partials : g.W;
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int m = m0 + 16 * i + 4 * gr + e;
            if (m >= g.M) continue;
            const int64_t row = base + (g.w_affine ? m * g.w_sm : int64_t(g.tWM[m]));
#pragma unroll
            for (int j = 0; j < TN; j++) {
                const int n = n0 + 16 * j + r;
                if (n >= g.N) continue;
                const int64_t o = row + (g.w_affine ? n : g.tWN[n]);
                if (half) reinterpret_cast<uint16_t*>(out)[o] = f32_to_bf16_rne(acc[i][j][e]);
                else out[o] = acc[i][j][e];
            }
        }
}

struct MxShape {
    int64_t M, N;
    int tm, tn;
    int64_t m_blocks, n_blocks;
};

MxShape mx_shape(const Plan& p) {
    MxShape h;
    h.M = p.swap ? p.nN : p.nM;
    h.N = p.swap ? p.nM : p.nN;
    h.tm = h.M > 32 ? 4 : h.M > 16 ? 2 : 1;
    h.tn = h.N > 64 ? 2 : 1;
    h.m_blocks = (h.M + 16 * h.tm - 1) / (16 * h.tm);
    h.n_blocks = (h.N + 64 * h.tn - 1) / (64 * h.tn);
    return h;
}

}  // namespace

hipError_t launch_mx_quantize(const Plan& p, int op, const void* tiles, int src_dtype, int64_t n, void* mx, hipStream_t s) {
    const MxTiles g = mx_tiles(p, op, n);
    const int64_t grid = (n * g.rows * g.blocks + kThreads - 1) / kThreads;
    if (grid > int64_t(0x7fffffff)) return hipErrorInvalidConfiguration;
    uint8_t* out = static_cast<uint8_t*>(mx);
    if (src_dtype == TRE_BF16)
        k_mx_quantize<<<unsigned(grid), kThreads, 0, s>>>(g, static_cast<const uint16_t*>(tiles), out);
    else
        k_mx_quantize<<<unsigned(grid), kThreads, 0, s>>>(g, static_cast<const float*>(tiles), out);
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(const Plan& p, int op, const void* mx, int64_t n, void* tiles, int dst_dtype, hipStream_t s) {
    const MxTiles g = mx_tiles(p, op, n);
    const int64_t grid = (n * g.rows * g.blocks + kThreads - 1) / kThreads;
    if (grid > int64_t(0x7fffffff)) return hipErrorInvalidConfiguration;
    const uint8_t* in = static_cast<const uint8_t*>(mx);
    if (dst_dtype == TRE_BF16)
        k_mx_dequantize<<<unsigned(grid), kThreads, 0, s>>>(g, in, static_cast<uint16_t*>(tiles));
    else
        k_mx_dequantize<<<unsigned(grid), kThreads, 0, s>>>(g, in, static_cast<float*>(tiles));
    return hipGetLastError();
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
    if (h.tm == 4)
        return h.tn == 2 ? launch_k(k_mx<4, 2>, grid, block, 0, s, g) : launch_k(k_mx<4, 1>, grid, block, 0, s, g);
    if (h.tm == 2)
        return h.tn == 2 ? launch_k(k_mx<2, 2>, grid, block, 0, s, g) : launch_k(k_mx<2, 1>, grid, block, 0, s, g);
    return h.tn == 2 ? launch_k(k_mx<1, 2>, grid, block, 0, s, g) : launch_k(k_mx<1, 1>, grid, block, 0, s, g);
}

}  // namespace tre
