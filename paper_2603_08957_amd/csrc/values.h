// Runs of consecutive fp32 or bf16 values in a lane's registers, and tokens.
#pragma once
#include "tre_internal.h"

namespace tre {

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

}  // namespace tre
