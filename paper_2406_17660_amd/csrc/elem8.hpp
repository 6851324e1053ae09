// Eight consecutive elements of an fp32 or bf16 array in any position: one or two 16-byte accesses
// on the elements' own alignment (the memory system takes them on any), or single elements where
// a row ends inside the eight.  Used by the norms and by AdamW.
#pragma once
#include "common.hpp"

namespace grass {
namespace {

typedef uint32_t raw4_t __attribute__((ext_vector_type(4)));
typedef raw4_t raw4_on2_t __attribute__((aligned(2)));
typedef raw4_t raw4_on4_t __attribute__((aligned(4)));

// Nearest even, NaN stays NaN; two values per instruction.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const f32x2_t x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t));
}

// The eight as they lie in memory.  `once`: the streaming hint, for what is not read again soon.
template <typename T>
struct Raw8;
template <>
struct Raw8<uint16_t> {
    raw4_t a;
    __device__ __forceinline__ void load(const uint16_t* p) { a = *reinterpret_cast<const raw4_on2_t*>(p); }
    __device__ __forceinline__ void load_once(const uint16_t* p) {
        a = __builtin_nontemporal_load(reinterpret_cast<const raw4_on2_t*>(p));
    }
    __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<raw4_on2_t*>(p) = a; }
    __device__ __forceinline__ void store_once(uint16_t* p) const {
        __builtin_nontemporal_store(a, reinterpret_cast<raw4_on2_t*>(p));
    }
    __device__ __forceinline__ void zero() { a = raw4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ float get(int i) const {
        return __uint_as_float((i & 1) ? a[i / 2] & 0xFFFF0000u : a[i / 2] << 16);
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void load_some(const uint16_t* p, int count) {
        zero();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) a[i / 2] |= static_cast<uint32_t>(p[i]) << (16 * (i & 1));
    }
    __device__ __forceinline__ void store_some(uint16_t* p, int count) const {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = static_cast<uint16_t>(a[i / 2] >> (16 * (i & 1)));
    }
};
template <>
struct Raw8<float> {
    raw4_t a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const raw4_on4_t*>(p);
        b = *reinterpret_cast<const raw4_on4_t*>(p + 4);
    }
    __device__ __forceinline__ void load_once(const float* p) {
        a = __builtin_nontemporal_load(reinterpret_cast<const raw4_on4_t*>(p));
        b = __builtin_nontemporal_load(reinterpret_cast<const raw4_on4_t*>(p + 4));
    }
    __device__ __forceinline__ void store(float* p) const {
        *reinterpret_cast<raw4_on4_t*>(p) = a;
        *reinterpret_cast<raw4_on4_t*>(p + 4) = b;
    }
    __device__ __forceinline__ void store_once(float* p) const {
        __builtin_nontemporal_store(a, reinterpret_cast<raw4_on4_t*>(p));
        __builtin_nontemporal_store(b, reinterpret_cast<raw4_on4_t*>(p + 4));
    }
    __device__ __forceinline__ void zero() { a = b = raw4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i < 4 ? a[i & 3] : b[i & 3]); }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = __float_as_uint(x[i]);
            b[i] = __float_as_uint(x[4 + i]);
        }
    }
    __device__ __forceinline__ void load_some(const float* p, int count) {
        zero();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) (i < 4 ? a : b)[i & 3] = __float_as_uint(p[i]);
    }
    __device__ __forceinline__ void store_some(float* p, int count) const {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = get(i);
    }
};

}  // namespace
}  // namespace grass
