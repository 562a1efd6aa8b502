// What many tensors do together at the end of a training step: the norm of their
// gradients, and an AdamW step of their weights with moments in 32 or 8 bits.
//
// Tensors of all sizes share a launch: its arguments hold their places and the
// number of the first workgroup of each, so that nothing is kept on the device
// between calls and a captured call holds what it was given.  Memory bounds both:
// 134 M fp32 weights, gradients and moments take 675 us (5.6 TB/s), 67 M weights in
// fp32 with bf16 gradients and 8-bit moments 182 (5.2), the norm of 400 M bf16
// gradients 143 (5.6).  Rounded by chance, 67 M weights in bf16 take 174 us and more,
// of which the vector units work 130 (73 operations an element, 15 of them the hash).
#include "codes.h"
#include "tre_internal.h"
#include "values.h"

#include <cmath>

namespace tre {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// The tensor of a workgroup: the last whose first workgroup is it or one before.
template <int N>
__device__ inline int tensor_of(const uint32_t (&first)[N], int count, uint32_t block) {
    const int lane = threadIdx.x & 63;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; i += 64) n += __popcll(__ballot(i + lane < count && first[min(i + lane, N - 1)] <= block));
    return __builtin_amdgcn_readfirstlane(n - 1);
}

// ----------------------------------------------------------------- norm

constexpr int kNormRuns = 8;

// Tensors of a launch, whose arguments stay below 4 KB.
constexpr int kNormMany = 190;

struct NormArgs {
    const void* x[kNormMany];
    int64_t size[kNormMany];
    uint32_t first[kNormMany];  // workgroup
    uint8_t half[kNormMany];    // whether in bf16
    int32_t count;
    double* part;       // of the launch's workgroups
    int64_t per;        // elements of a workgroup
};
static_assert(sizeof(NormArgs) <= 4096, "a launch's arguments");

template <typename T>
__device__ inline double squares(const T* x, int64_t n) {
    constexpr int E = 16 / sizeof(T);
    constexpr int64_t kStep = int64_t(kThreads) * E;
    double s[2] = {0., 0.};
    int64_t b = 0;
    for (; b + kNormRuns * kStep <= n; b += kNormRuns * kStep) {
        float v[kNormRuns][E];
#pragma unroll
        for (int j = 0; j < kNormRuns; j++) load_all(x + b + j * kStep + threadIdx.x * E, v[j]);
#pragma unroll
        for (int j = 0; j < kNormRuns; j++)
#pragma unroll
            for (int i = 0; i < E; i++) s[i & 1] = __builtin_fma(double(v[j][i]), double(v[j][i]), s[i & 1]);
    }
    for (b += threadIdx.x * E; b < n; b += kStep) {
        float v[E];
        load_run(x, b, n, v);
#pragma unroll
        for (int i = 0; i < E; i++) s[i & 1] = __builtin_fma(double(v[i]), double(v[i]), s[i & 1]);
    }
    return s[0] + s[1];
}

// The sum over a workgroup of one value each, in thread 0.
__device__ inline double sum_all(double s) {
    __shared__ double part[16];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.;
    for (int w = 0; w < int(blockDim.x) >> 6; w++) s += part[w];
    return s;
}

// Squares are summed in 64 bits: no fp32 value's overflows, and the sum's error
// does not grow with the model.  Memory is still what bounds it: an element takes
// a conversion and one fused product.
__global__ __launch_bounds__(kThreads) void k_squares(NormArgs a) {
    const uint32_t block = uint32_t(block_index());
    const int i = tensor_of(a.first, a.count, block);
    const int64_t at = int64_t(block - a.first[i]) * a.per, n = min(a.per, a.size[i] - at);
    if (n <= 0) return;  // (a workgroup that only the grid's shape has)
    const double s = sum_all(a.half[i] ? squares(static_cast<const uint16_t*>(a.x[i]) + at, n)
                                       : squares(static_cast<const float*>(a.x[i]) + at, n));
    if (threadIdx.x == 0) a.part[block] = s;
}

constexpr int kFinishThreads = 1024;

__global__ __launch_bounds__(kFinishThreads) void k_norm(const double* __restrict__ part, int64_t n, float max_norm,
                                                         float* __restrict__ out) {
    double s = 0.;
    for (int64_t i = threadIdx.x; i < n; i += kFinishThreads) s += part[i];
    s = sum_all(s);
    if (threadIdx.x) return;
    const double norm = sqrt(s);
    const bool finite = norm <= double(__FLT_MAX__);
    out[0] = float(norm);
    out[1] = !finite ? __builtin_nanf("") : max_norm < 0.f ? 1.f : float(fmin(double(max_norm) / (norm + 1e-6), 1.));
}

// Elements of a workgroup, so that some thousand workgroups' sums are left to one
// workgroup: 400 M bf16 elements take 137 us (5.8 TB/s) and 4.5 for the sums, with
// twice as many parts 137 and 6.4, with half 143 and 4.
constexpr int64_t kNormParts = 8192, kNormLeast = 4096;
int64_t norm_per(int n, const int64_t* sizes) {
    int64_t total = 0, per = kNormLeast;
    for (int i = 0; i < n; i++) total += sizes[i];
    while (per * kNormParts < total) per *= 2;
    return per;
}

// ---------------------------------------------------------------- AdamW
//
//   m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Moments in 8 bits.  32 consecutive elements share a power of two, the one that
// brings the largest magnitude into [128, 256); times it a value is a small
// floating point number: a first moment's a sign, 4 bits of exponent (bias 7) and
// 3 of fraction, a second moment's 5 (bias 23) and 3.  A power of two loses
// nothing where values have exponents of their own, and scaling by it is exact.
// The second moment's range is twice the first's as exponents go, which the root
// halves again.  One that is not zero takes the least code at least: a zero would
// leave a first moment that is not zero over eps alone.
//
// Rounding to nearest loses steps that are below half a code's: a second moment
// with b2 = 0.999 moves by a thousandth where codes are an eighth apart.  So with
// a seed it is by chance, up with the probability that a value's place between two
// codes has, which is right on average; weights in bf16 then too.

// Tensors of a launch, whose arguments stay below 4 KB: weights, gradients, elements
// (the upper bits in `kind`), where the moments begin (in blocks of 32) and the first
// workgroup.
constexpr int kAdamMany = 134;

struct AdamArgs {
    void* p[kAdamMany];
    const void* g[kAdamMany];
    uint32_t size[kAdamMany], at32[kAdamMany], first[kAdamMany];
    uint8_t kind[kAdamMany];  // 1: weights in bf16, 2: gradients in bf16; the rest: size >> 32
    int32_t count;
    void* state;
    int64_t total;
    const float *lr_dev, *scale_dev;
    const int64_t* step_dev;
    int64_t per;            // elements of a workgroup
    double log_beta1, log_beta2;
    bool small_roots;       // whether roots below 2^-63 count beside eps
    float b1, nb1, b2, nb2, c1, c2, lr, decay, weight_decay, eps, scale;
    uint32_t seed0, seed1, step;
};

static_assert(sizeof(AdamArgs) <= 4096, "a launch's arguments");

struct Rates {
    float c1, c2, lr, decay, scale;
    uint32_t k0;
};

// 1 / (1 - b^t) from the logarithm of b: 1 - e^x for x = t log b < 0, near 0 by its
// series (to 2^-24 of itself for x > -1/2, whose next term is x^8 / 9!).
__device__ inline float correction(double log_b, int64_t t) {
    const float x = float(log_b * double(t));
    float s = 1.f / 40320.f;
#pragma unroll
    for (int k = 7; k >= 1; k--) {
        constexpr float kInverse[8] = {0.f, 1.f, 1.f / 2.f, 1.f / 6.f, 1.f / 24.f, 1.f / 120.f, 1.f / 720.f, 1.f / 5040.f};
        s = s * x + kInverse[k];
    }
    return 1.f / (x > -0.5f ? -x * s : 1.f - __builtin_amdgcn_exp2f(x * 1.4426950408889634f));
}

__device__ inline Rates rates_of(const AdamArgs& a) {
    Rates r{a.c1, a.c2, a.lr, a.decay, a.scale, 0};
    uint32_t step = a.step;
    if (a.scale_dev) r.scale = *a.scale_dev;
    if (a.lr_dev) {
        r.lr = *a.lr_dev;
        r.decay = 1.f - r.lr * a.weight_decay;
    }
    if (a.step_dev) {
        const int64_t t = max(*a.step_dev, int64_t(1));
        r.c1 = correction(a.log_beta1, t);
        r.c2 = correction(a.log_beta2, t);
        step = uint32_t(t);
    }
    r.k0 = a.seed0 + step * 0x9E3779B1u;
    return r;
}

// Random bits of an element: a hash of (seed, step, element) by shifts and products
// with the leading bits of the golden ratio and of the roots of 2, 3 and 5.  low:
// the element's number; k1: the seed's upper half and what the number's adds.
struct Chance {
    uint32_t h, y;  // the upper 20 bits are the first and the second moment's
    __device__ uint32_t weight() const { return (h ^ (y << 4)) & 0xffffu; }
};
__device__ inline Chance chance_of(uint32_t low, uint32_t k0, uint32_t k1) {
    uint32_t h = (low ^ k0) * 0x6A09E667u;
    h ^= h >> 15;
    h = (h + k1) * 0xBB67AE85u;
    h ^= h >> 13;
    uint32_t y = h * 0x3C6EF373u;
    y ^= y >> 16;
    return {h, y};
}
__device__ inline uint32_t chance_key(uint32_t k1, int64_t element) { return k1 + uint32_t(element >> 32) * 0xBB67AE85u; }

// A first moment's codes are those of the instructions for 8-bit floats (4 bits of
// exponent, bias 7), which stay below 480, their NaN's: two of four codes.
template <bool UPPER>
__device__ inline void first_pair(uint32_t codes, uint32_t byte, float& x, float& y) {
    const auto v = __builtin_amdgcn_cvt_pk_f32_fp8(codes, UPPER);
    x = ldexpf(v[0], int(byte) - 127);
    y = ldexpf(v[1], int(byte) - 127);
}
// A second moment's code as the upper bits of a float of exponent E less 127 (a
// denormal for E = 0) is 2^(bias - 127) of its value.
__device__ inline float second_moment(uint32_t codes, int i, uint32_t byte) {
    return ldexpf(__uint_as_float((codes >> (8 * i) & 255u) << 20), int(byte) - kBias2);
}

// Codes of first moments times the block's power of two.  By chance the
// instruction adds a word's upper 20 bits below the last bit that stays.
template <bool CHANCE, typename C>
__device__ inline uint32_t first_codes(const float (&y)[4], const C& c) {
    int q = 0;
    if constexpr (CHANCE) {
        q = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], c[0].h, q, 0);
        q = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], c[1].h, q, 1);
        q = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], c[2].h, q, 2);
        q = __builtin_amdgcn_cvt_sr_fp8_f32(y[3], c[3].h, q, 3);
    } else {
        q = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], q, false);
        q = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], q, true);
    }
    return uint32_t(q);
}
// The exponent (of a float's bits) of a block's largest magnitude, 7 at least; 8
// lanes to a block.  255: a NaN or an infinity.
__device__ inline uint32_t block_exponent(uint32_t bits) {
    bits = max(bits, uint32_t(__builtin_amdgcn_update_dpp(0, bits, 0xB1, 0xf, 0xf, true)));
    bits = max(bits, uint32_t(__builtin_amdgcn_update_dpp(0, bits, 0x4E, 0xf, 0xf, true)));
    bits = max(bits, uint32_t(__builtin_amdgcn_update_dpp(0, bits, 0x141, 0xf, 0xf, true)));
    return max(bits >> 23, 7u);
}
__device__ inline uint8_t block_byte(uint32_t exponent) { return uint8_t(exponent == 255u ? 255u : exponent - 7u); }
// 2^(127 - byte)
__device__ inline float block_scale(uint32_t exponent) { return __uint_as_float((261u - exponent) << 23); }

// A lane takes 4 elements at once (16 bytes in fp32), a wavefront a run of 256; the
// next run's are loaded before this one's are used.
constexpr int kLane = 4;
constexpr int64_t kRun = 64 * kLane;

template <typename T>
__device__ inline void store4(T* at, const float (&v)[kLane], bool cut) {
    if constexpr (sizeof(T) == 2) {
        if (cut) {  // (bf16 values already)
            u32x2_2 w;
            w[0] = __float_as_uint(v[0]) >> 16 | (__float_as_uint(v[1]) & 0xffff0000u);
            w[1] = __float_as_uint(v[2]) >> 16 | (__float_as_uint(v[3]) & 0xffff0000u);
            __builtin_nontemporal_store(w, reinterpret_cast<u32x2_2*>(at));
            return;
        }
    }
    store_all<true>(at, v);
}

// The square roots of v c, c >= 1.  The instruction takes what is below 2^-126 for 0,
// so small ones are brought up by 2^24 first: a root below 2^-63 would be lost, which
// is less than half a unit of an eps of 2^-39 or more, and only below that is it
// looked for (four operations more of an element's 73).
__device__ inline void roots_of(const float (&v)[kLane], float c, bool small, float (&root)[kLane]) {
    if (!small) {
#pragma unroll
        for (int i = 0; i < kLane; i++) root[i] = __builtin_amdgcn_sqrtf(v[i] * c);
        return;
    }
#pragma unroll
    for (int i = 0; i < kLane; i++) {
        const bool low = v[i] < 0x1p-100f;
        root[i] = __builtin_amdgcn_sqrtf((low ? v[i] * 0x1p24f : v[i]) * c) * (low ? 0x1p-12f : 1.f);
    }
}

// 4 elements as they come.
template <int BITS, typename TP, typename TG>
struct Held {
    uint32_t p[sizeof(TP)], g[sizeof(TG)], m[BITS / 8], v[BITS / 8];  // (4 elements of so many bytes each, in words)
    uint32_t mb, vb;
};
template <typename T>
__device__ inline void load4(const T* at, uint32_t (&w)[sizeof(T)]) {
    if constexpr (sizeof(T) == 4) {
        const f32x4_4 x = *reinterpret_cast<const f32x4_4*>(at);
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = __float_as_uint(x[i]);
    } else {
        const u32x2_2 x = *reinterpret_cast<const u32x2_2*>(at);
        w[0] = x[0];
        w[1] = x[1];
    }
}
template <typename T>
__device__ inline void load_upto4(const T* at, int64_t n, uint32_t (&w)[sizeof(T)]) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T)); i++) w[i] = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (i >= n) break;
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(at[i]);
        else w[i / 2] |= uint32_t(at[i]) << (16 * (i & 1));
    }
}
template <int N>
__device__ inline float value4(const uint32_t (&w)[N], int i) {
    if constexpr (N == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}

// A tensor's part that a wavefront steps.
template <int BITS, bool CHANCE, typename TP, typename TG>
struct Part {
    using H = Held<BITS, TP, TG>;
    const AdamArgs& a;
    const Rates& r;
    TP* p;
    const TG* g;
    int64_t at, n;   // the tensor's first element among all, its elements
    uint32_t lane;

    // The run from element e on (a scalar; the lanes' offsets from it are 32 bits).
    template <bool WHOLE>
    __device__ H load(int64_t e) const {
        H h;
        const uint32_t o = lane * kLane;
        if constexpr (WHOLE) {
            load4(p + e + o, h.p);
            load4(g + e + o, h.g);
        } else {
            load_upto4(p + e + o, n - e - o, h.p);
            load_upto4(g + e + o, n - e - o, h.g);
        }
        if constexpr (BITS == 32) {
            const float* m = static_cast<const float*>(a.state) + at + e;
            load4(m + o, h.m);
            load4(m + a.total + o, h.v);
        } else {
            const uint8_t* m = static_cast<const uint8_t*>(a.state) + at + e;
            const uint8_t* b = static_cast<const uint8_t*>(a.state) + 2 * a.total + (at + e) / 32;
            h.m[0] = *reinterpret_cast<const uint32_t*>(m + o);
            h.v[0] = *reinterpret_cast<const uint32_t*>(m + a.total + o);
            h.mb = b[o / 32];
            h.vb = b[a.total / 32 + o / 32];
        }
        return h;
    }

    template <bool WHOLE>
    __device__ void step(int64_t e, const H& h) const {
        const uint32_t o = lane * kLane;
        float pv[kLane], mv[kLane], vv[kLane];
        Chance c[kLane];
        uint32_t m_top = 0, v_top = 0;
        float b1 = a.b1, b2 = a.b2;
        if constexpr (BITS == 8) {  // a block that holds NaN
            b1 = h.mb == 255u ? __builtin_nanf("") : b1;
            b2 = h.vb == 255u ? __builtin_nanf("") : b2;
        }
        const float rate = -r.lr * r.c1;
        // (the element's number may pass 2^32 in a run)
        const uint32_t low0 = uint32_t(at + e), low = low0 + o;
        const uint32_t k = low < low0 ? chance_key(a.seed1, at + e + kRun) : chance_key(a.seed1, at + e);
        if constexpr (BITS == 8) {
            first_pair<false>(h.m[0], h.mb, mv[0], mv[1]);
            first_pair<true>(h.m[0], h.mb, mv[2], mv[3]);
        }
#pragma unroll
        for (int i = 0; i < kLane; i++) {
            if constexpr (BITS == 8) {
                vv[i] = second_moment(h.v[0], i, h.vb);
            } else {
                mv[i] = value4(h.m, i);
                vv[i] = value4(h.v, i);
            }
            if constexpr (CHANCE && (BITS == 8 || sizeof(TP) == 2)) c[i] = chance_of(low + i, r.k0, k);
            {
                // (each product and sum rounded for itself, so that a moment next to a border between two codes is the same
                // whoever computes it)
#pragma clang fp contract(off)
                const float gi = value4(h.g, i) * r.scale;
                mv[i] = mv[i] * b1 + gi * a.nb1;
                vv[i] = vv[i] * b2 + gi * gi * a.nb2;
            }
        }
        float root[kLane];
        roots_of(vv, r.c2, a.small_roots, root);
#pragma unroll
        for (int i = 0; i < kLane; i++) {
            pv[i] = value4(h.p, i) * r.decay + rate * mv[i] * __builtin_amdgcn_rcpf(root[i] + a.eps);
            if constexpr (CHANCE && sizeof(TP) == 2) {
                const float up = __uint_as_float((__float_as_uint(pv[i]) + c[i].weight()) & 0xffff0000u);
                pv[i] = pv[i] == pv[i] ? up : __builtin_nanf("");
            }
            if constexpr (BITS == 8) {
                m_top = max(m_top, __float_as_uint(mv[i]) & 0x7fffffffu);
                v_top = max(v_top, __float_as_uint(vv[i]) & 0x7fffffffu);
            }
        }
        if constexpr (WHOLE) store4(p + e + o, pv, CHANCE);
        else store_run<true>(p, e + o, n, pv);
        if constexpr (BITS == 32) {
            float* m = static_cast<float*>(a.state) + at + e;
            store_all<true>(m + o, mv);
            store_all<true>(m + a.total + o, vv);
        } else {
            const uint32_t em = block_exponent(m_top), ev = block_exponent(v_top);
            const float sm = block_scale(em), sv = block_scale(ev);
            const float y[kLane] = {mv[0] * sm, mv[1] * sm, mv[2] * sm, mv[3] * sm};
            const uint32_t mq = first_codes<CHANCE>(y, c);
            uint32_t vq = 0;
#pragma unroll
            for (int i = 0; i < kLane; i++) {  // (at least 1 where it is not zero)
                const uint32_t w = second_code<CHANCE>(vv[i] * sv, c[i].y);
                vq |= max(w, min(__float_as_uint(vv[i]), 1u)) << (8 * i);
            }
            uint8_t* m = static_cast<uint8_t*>(a.state) + at + e;
            uint8_t* b = static_cast<uint8_t*>(a.state) + 2 * a.total + (at + e) / 32;
            *reinterpret_cast<uint32_t*>(m + o) = em == 255u ? 0u : mq;
            *reinterpret_cast<uint32_t*>(m + a.total + o) = ev == 255u ? 0u : vq;
            if ((lane & 7) == 0) {
                b[o / 32] = block_byte(em);
                b[a.total / 32 + o / 32] = block_byte(ev);
            }
        }
    }

    // The runs from e on, kRun * kWaves apart, that end at `end` or before; what is left of the tensor's last one.
    __device__ void all(int64_t e, int64_t end) const {
        constexpr int64_t kNext = kRun * kWaves;
        if (e + kRun <= end) {
            H h = load<true>(e);
#pragma unroll 1
            for (; e + kNext + kRun <= end; e += kNext) {
                const H next = load<true>(e + kNext);
                step<true>(e, h);
                h = next;
            }
            step<true>(e, h);
            e += kNext;
        }
        // (the moments have whole blocks)
        if (e < end && end == n && e + lane * kLane / 32 * 32 < n) step<false>(e, load<false>(e));
    }
};

template <int BITS, bool CHANCE, typename TP, typename TG>
__device__ inline void adam_block(const AdamArgs& a, const Rates& r, int i, int64_t e) {
    const Part<BITS, CHANCE, TP, TG> part{a, r, static_cast<TP*>(a.p[i]), static_cast<const TG*>(a.g[i]), int64_t(a.at32[i]) * 32,
                                          int64_t(a.kind[i] >> 2) << 32 | a.size[i], threadIdx.x & 63};
    part.all(e + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kRun, min(part.n, e + a.per));
}

template <int BITS, bool CHANCE>
__global__ __launch_bounds__(kThreads) void k_adam(AdamArgs a) {
    const uint32_t block = uint32_t(block_index());
    const int i = tensor_of(a.first, a.count, block);
    const Rates r = rates_of(a);
    if (r.scale != r.scale) return;  // (a norm that is not finite: no step)
    const int64_t e0 = int64_t(block - a.first[i]) * a.per;
    switch (a.kind[i] & 3) {
        case 0: adam_block<BITS, CHANCE, float, float>(a, r, i, e0); break;
        case 1: adam_block<BITS, CHANCE, uint16_t, float>(a, r, i, e0); break;
        case 2: adam_block<BITS, CHANCE, float, uint16_t>(a, r, i, e0); break;
        default: adam_block<BITS, CHANCE, uint16_t, uint16_t>(a, r, i, e0); break;
    }
}

// 8-bit moments read back.
template <typename TO>
__global__ __launch_bounds__(kThreads) void k_moments(const uint8_t* __restrict__ state, int64_t total, TO* __restrict__ m,
                                                      TO* __restrict__ v) {
    const int64_t e = (block_index() * kThreads + threadIdx.x) * 8;
    if (e >= total) return;
    const uint2 mc = *reinterpret_cast<const uint2*>(state + e), vc = *reinterpret_cast<const uint2*>(state + total + e);
    const uint32_t mb = state[2 * total + e / 32], vb = state[2 * total + total / 32 + e / 32];
    float mv[8], vv[8];
    first_pair<false>(mc.x, mb, mv[0], mv[1]);
    first_pair<true>(mc.x, mb, mv[2], mv[3]);
    first_pair<false>(mc.y, mb, mv[4], mv[5]);
    first_pair<true>(mc.y, mb, mv[6], mv[7]);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        vv[i] = vb == 255u ? __builtin_nanf("") : second_moment(i < 4 ? vc.x : vc.y, i & 3, vb);
        if (mb == 255u) mv[i] = __builtin_nanf("");
    }
    store_all<true>(m + e, mv);
    store_all<true>(v + e, vv);
}

// Elements of a workgroup: a run for each wavefront, or four of the shorter 8-bit
// ones.  (134 M elements in 32 bits: 671 us with one, 695 with two, 715 with four;
// 67 M in 8 bits, rounded by chance: 233, 207, 176, and 180 with eight.)
int64_t adam_per(int bits) { return kRun * kWaves * (bits == 32 ? 1 : 4); }

int64_t room_of(int64_t n) { return (n + 31) / 32 * 32; }

template <int BITS>
hipError_t adam(const AdamArgs& a, bool chance, int64_t blocks, hipStream_t s) {
    if (chance) k_adam<BITS, true><<<grid_of(blocks), kThreads, 0, s>>>(a);
    else k_adam<BITS, false><<<grid_of(blocks), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t grad_norm_ws_bytes(int n, const int64_t* sizes) {
    const int64_t per = norm_per(n, sizes);
    int64_t parts = 1;
    for (int i = 0; i < n; i++) parts += (sizes[i] + per - 1) / per;
    return (size_t(parts) * 8 + 255) / 256 * 256;
}

hipError_t launch_grad_norm(int n, const void* const* tensors, const int32_t* types, const int64_t* sizes, float max_norm,
                            float* out, char* ws, hipStream_t s) {
    NormArgs a{};
    a.per = norm_per(n, sizes);
    a.part = reinterpret_cast<double*>(ws);
    int64_t parts = 0, blocks = 0;
    for (int i = 0; i < n; i++) {
        if (sizes[i] > 0) {
            const int k = a.count++;
            a.x[k] = tensors[i];
            a.size[k] = sizes[i];
            a.first[k] = uint32_t(blocks);
            a.half[k] = types[i] == TRE_BF16;
            blocks += (sizes[i] + a.per - 1) / a.per;
        }
        if (a.count == kNormMany || (i == n - 1 && a.count)) {
            k_squares<<<grid_of(blocks), kThreads, 0, s>>>(a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            a.part += blocks;
            parts += blocks;
            blocks = 0;
            a.count = 0;
        }
    }
    k_norm<<<1, kFinishThreads, 0, s>>>(reinterpret_cast<const double*>(ws), parts, max_norm, out);
    return hipGetLastError();
}

int64_t adamw_room(int n, const int64_t* sizes) {
    int64_t total = 0;
    for (int i = 0; i < n; i++) total += room_of(sizes[i]);
    return total;
}

hipError_t launch_adamw(int n, void* const* params, const int32_t* param_types, const void* const* grads,
                        const int32_t* grad_types, const int64_t* sizes, void* state, const tre_adamw_options& o, hipStream_t s) {
    AdamArgs a{};
    a.per = adam_per(o.bits);
    a.state = state;
    a.total = adamw_room(n, sizes);
    a.lr_dev = o.lr_dev;
    a.scale_dev = o.grad_scale_dev;
    a.step_dev = o.step_dev;
    a.log_beta1 = std::log(o.beta1);  // (-inf for 0)
    a.log_beta2 = std::log(o.beta2);
    a.b1 = float(o.beta1);
    a.nb1 = float(1. - o.beta1);
    a.b2 = float(o.beta2);
    a.nb2 = float(1. - o.beta2);
    if (!o.step_dev) {
        a.c1 = float(1. / (1. - std::pow(o.beta1, double(o.step))));
        a.c2 = float(1. / (1. - std::pow(o.beta2, double(o.step))));
        a.step = uint32_t(o.step);
    }
    a.lr = float(o.lr);
    a.decay = float(1. - o.lr * o.weight_decay);
    a.weight_decay = float(o.weight_decay);
    a.eps = float(o.eps);
    a.small_roots = a.eps < 0x1p-39f;
    a.scale = float(o.grad_scale);
    a.seed0 = uint32_t(o.seed);
    a.seed1 = uint32_t(o.seed >> 32);
    int64_t blocks = 0, at = 0;
    for (int i = 0; i < n; i++) {
        if (sizes[i] > 0) {
            const int k = a.count++;
            a.p[k] = params[i];
            a.g[k] = grads[i];
            a.size[k] = uint32_t(sizes[i]);
            a.at32[k] = uint32_t(at / 32);
            a.first[k] = uint32_t(blocks);
            a.kind[k] = uint8_t((param_types[i] == TRE_BF16) | (grad_types[i] == TRE_BF16) << 1 | (sizes[i] >> 32) << 2);
            blocks += (sizes[i] + a.per - 1) / a.per;
            at += room_of(sizes[i]);
        }
        if (a.count == kAdamMany || (i == n - 1 && a.count)) {
            const hipError_t e = o.bits == 8 ? adam<8>(a, o.stochastic != 0, blocks, s) : adam<32>(a, o.stochastic != 0, blocks, s);
            if (e != hipSuccess) return e;
            blocks = 0;
            a.count = 0;
        }
    }
    return hipSuccess;
}

hipError_t launch_adamw_moments(const void* state, int64_t total, void* m, void* v, int dtype, hipStream_t s) {
    const dim3 grid = grid_of((total / 8 + kThreads - 1) / kThreads);
    const uint8_t* x = static_cast<const uint8_t*>(state);
    if (dtype == TRE_BF16) k_moments<<<grid, kThreads, 0, s>>>(x, total, static_cast<uint16_t*>(m), static_cast<uint16_t*>(v));
    else k_moments<<<grid, kThreads, 0, s>>>(x, total, static_cast<float*>(m), static_cast<float*>(v));
    return hipGetLastError();
}

}  // namespace tre
