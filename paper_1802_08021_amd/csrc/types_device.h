// Device helpers for values held in fp32, bf16 or fp16: vector loads and
// stores that need no alignment beyond the element's, and a wave's maximum.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sparcml {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// Storage type of an element type id (kF32, kBf16, kF16).
template <int TYPE>
struct Elem;
template <>
struct Elem<kF32> {
    typedef float type;
    typedef f32x4 vec4;
};
template <>
struct Elem<kBf16> {
    typedef __bf16 type;
    typedef bf16x4 vec4;
};
template <>
struct Elem<kF16> {
    typedef _Float16 type;
    typedef f16x4 vec4;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A pointer known to be to global memory (one read from a table would be taken
// for a generic one, whose accesses wait for LDS too).
#define SPARCML_GLOBAL __attribute__((address_space(1)))
template <class T>
__device__ __forceinline__ SPARCML_GLOBAL T* as_global(T* p)
{
    return (SPARCML_GLOBAL T*)p;
}

// Element i of 16 bytes of a type, as fp32.
template <int TYPE>
__device__ __forceinline__ float unpack(u32x4 w, int i)
{
    if (TYPE == kF32) return __uint_as_float(w[i & 3]);
    if (TYPE == kBf16) return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w[i >> 1] >> 16 : w[i >> 1]));
}

// A vector from p on, at any element-aligned address (one access: gfx950 takes
// unaligned vector accesses to global memory); streamed, marked nontemporal,
// unless it is read once more soon (KEEP).
template <class V, bool KEEP = false, class E>
__device__ __forceinline__ V load_vec(const E* p)
{
    typedef V U __attribute__((aligned(sizeof(E))));
    const SPARCML_GLOBAL U* q = (const SPARCML_GLOBAL U*)p;
    return KEEP ? *q : __builtin_nontemporal_load(q);
}
template <class V, class E>
__device__ __forceinline__ void store_vec(E* p, V v)
{
    typedef V U __attribute__((aligned(sizeof(E))));
    __builtin_nontemporal_store(v, (SPARCML_GLOBAL U*)p);
}

// Sum and maximum of the 64 lanes' values, in every lane: shifts within rows
// of 16 lanes, then the row broadcasts (lanes that a step has no source for
// add zero or keep their own).
template <int CTRL, int ROWS, bool SUM>
__device__ __forceinline__ float wave_step(float x)
{
    const int v = __float_as_int(x);
    const float y = __int_as_float(__builtin_amdgcn_update_dpp(SUM ? 0 : v, v, CTRL, ROWS, 0xF, false));
    return SUM ? x + y : fmaxf(x, y);
}
template <bool SUM>
__device__ __forceinline__ float wave_join(float x)
{
    x = wave_step<0x111, 0xF, SUM>(x);  // row_shr:1
    x = wave_step<0x112, 0xF, SUM>(x);  // row_shr:2
    x = wave_step<0x114, 0xF, SUM>(x);  // row_shr:4
    x = wave_step<0x118, 0xF, SUM>(x);  // row_shr:8
    x = wave_step<0x142, 0xA, SUM>(x);  // row_bcast:15
    x = wave_step<0x143, 0xC, SUM>(x);  // row_bcast:31
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// Largest of the 64 lanes' values, in every lane: shifts within rows of 16
// lanes, then the row broadcasts.
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    auto mx = [](uint32_t a, int b) { return a > (uint32_t)b ? a : (uint32_t)b; };
    v = mx(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true));   // row_shr:1
    v = mx(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true));   // row_shr:2
    v = mx(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true));   // row_shr:4
    v = mx(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true));   // row_shr:8
    v = mx(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false));  // row_bcast:15
    v = mx(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false));  // row_bcast:31
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

}  // namespace sparcml
