// Device and host helpers shared by the operators of lsm_block.h.
#pragma once
#include "../../include/lsm_block.h"
#include "lsm_internal.h"

namespace lsm {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// After each launch that others of a call follow: they take addresses from what it writes.
inline bool launched() { return hipGetLastError() == hipSuccess; }

constexpr int64_t kAxisThreads = 0xffffffff;  // most threads of a launch along an axis

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {  // round to nearest even
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

// The elements of one 16-byte piece as floats, and back: 8 of bf16 (TIO = uint16_t) or 4 of fp32.
template <typename TIO> constexpr int kPiece = 16 / int(sizeof(TIO));
__device__ __forceinline__ void unpack(const u32x4& v, float (&x)[8]) {
    _Pragma("unroll") for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(v[i]); x[2 * i + 1] = bf16_hi(v[i]); }
}
__device__ __forceinline__ void unpack(const u32x4& v, float (&x)[4]) {
    _Pragma("unroll") for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
}
__device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
    return u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
}
__device__ __forceinline__ u32x4 pack(const float (&x)[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

// lanes set in a ballot (HIP's own returns an unsigned number)
__device__ __forceinline__ int lanes(unsigned long long mask) { return __builtin_popcountll(mask); }

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(int(__float_as_uint(x)), CTRL, 0xf, 0xf, true));
}
// sum over aligned groups of N lanes (8, 16, 32 or 64), in every lane; the same order in all of them
template <int N>
__device__ __forceinline__ float group_sum(float x) {
    x += dpp<0xB1>(x);   // lane ^ 1
    x += dpp<0x4E>(x);   // lane ^ 2
    x += dpp<0x141>(x);  // the other four of eight
    if (N >= 16) x += dpp<0x140>(x);  // the other eight of sixteen
    if (N >= 32) x += __shfl_xor(x, 16, 64);
    if (N >= 64) x += __shfl_xor(x, 32, 64);
    return x;
}

}  // namespace
}  // namespace lsm
