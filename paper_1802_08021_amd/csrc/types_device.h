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

// Four consecutive elements from p on, at any element-aligned address (one
// access: gfx950 takes unaligned vector accesses to global memory).
template <class V, class E>
__device__ __forceinline__ V load4(const E* p)
{
    typedef V U __attribute__((aligned(sizeof(E))));
    return *reinterpret_cast<const U*>(p);
}
template <class V, class E>
__device__ __forceinline__ void store4(E* p, V v)
{
    typedef V U __attribute__((aligned(sizeof(E))));
    *reinterpret_cast<U*>(p) = v;
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
