// What the kernels that read rows of logits share: pieces of 16 bytes, sums over a wavefront.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace zf {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <typename ElemT> struct Piece;       // 16 bytes at any multiple of an element: the memory system takes them there
template <> struct Piece<uint32_t> { typedef u32x4 type __attribute__((aligned(4))); };
template <> struct Piece<uint16_t> { typedef u32x4 type __attribute__((aligned(2))); };

static const float LOG2_E = 1.44269504088896340736f, LN_2 = 0.69314718055994530942f;

__device__ __forceinline__ float of_bits(uint32_t x) { return __uint_as_float(x); }
__device__ __forceinline__ float of_bits(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
// Over a wavefront, to all lanes, by moves between lanes of 1, 2, 4, 8, 16 and 32; sums in this order, whatever the timing.
template <int CTRL, int ROWS = 0xF> __device__ __forceinline__ uint32_t moved(uint32_t none, uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, CTRL, ROWS, 0xF, false); }
template <class F>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, uint32_t none, F f) {
    x = f(x, moved<0x111>(none, x));           // the lane one below, of the same sixteen
    x = f(x, moved<0x112>(none, x));
    x = f(x, moved<0x114>(none, x));
    x = f(x, moved<0x118>(none, x));
    x = f(x, moved<0x142, 0xA>(none, x));      // lane 15 of each sixteen to the next
    x = f(x, moved<0x143, 0xC>(none, x));      // lane 31 to the upper half
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ float wave_max(float x) {
    return __uint_as_float(over_wave(__float_as_uint(x), 0xFF800000u, [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ float wave_sum(float x) {
    return __uint_as_float(over_wave(__float_as_uint(x), 0u, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ float two_to(float x) { return __builtin_amdgcn_exp2f(x); }   // below 2^-126 nothing

}  // namespace
}  // namespace zf
