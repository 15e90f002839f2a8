// Exchanges between the lanes of a wavefront, and conversions between bf16 and fp32 bits, that the kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace resq {

// value of lane (l ^ MASK): data-parallel-primitive moves inside a row of 16
// lanes where the pattern has one (quad permutes for 1 and 2, a rotation by 8),
// the swizzle unit inside 32 lanes, a general shuffle across the two halves
template <int MASK>
__device__ __forceinline__ float lane_xor(float x) {
    const int xi = __float_as_int(x);
    int r;
    if constexpr (MASK == 1) r = __builtin_amdgcn_update_dpp(xi, xi, 0xB1, 0xF, 0xF, false);       // quad_perm [1,0,3,2]
    else if constexpr (MASK == 2) r = __builtin_amdgcn_update_dpp(xi, xi, 0x4E, 0xF, 0xF, false);  // quad_perm [2,3,0,1]
    else if constexpr (MASK == 8) r = __builtin_amdgcn_update_dpp(xi, xi, 0x128, 0xF, 0xF, false); // row_ror:8
    else if constexpr (MASK == 4) r = __builtin_amdgcn_ds_swizzle(xi, 0x101F);                     // xor 4 within 32
    else if constexpr (MASK == 16) r = __builtin_amdgcn_ds_swizzle(xi, 0x401F);                    // xor 16 within 32
    else r = __float_as_int(__shfl_xor(x, MASK));
    return __int_as_float(r);
}

__device__ __forceinline__ float bf16_bits_to_f32(uint32_t b) { return __uint_as_float(b << 16); }

// Butterfly reductions over the 64 lanes of a wavefront; the lane exchanges are
// the cheap ones of the transform kernel (DPP moves, swizzles) where they exist.
// G = 16, 32 or 64: the reduction runs inside aligned groups of G lanes.
template <int G = 64>
__device__ __forceinline__ float wave_max(float a) {
    a = fmaxf(a, lane_xor<1>(a));
    a = fmaxf(a, lane_xor<2>(a));
    a = fmaxf(a, lane_xor<4>(a));
    a = fmaxf(a, lane_xor<8>(a));
    if constexpr (G > 16) a = fmaxf(a, lane_xor<16>(a));
    if constexpr (G > 32) a = fmaxf(a, lane_xor<32>(a));
    return a;
}
template <int G = 64>
__device__ __forceinline__ int wave_sum(int v) {
    v += __float_as_int(lane_xor<1>(__int_as_float(v)));
    v += __float_as_int(lane_xor<2>(__int_as_float(v)));
    v += __float_as_int(lane_xor<4>(__int_as_float(v)));
    v += __float_as_int(lane_xor<8>(__int_as_float(v)));
    if constexpr (G > 16) v += __float_as_int(lane_xor<16>(__int_as_float(v)));
    if constexpr (G > 32) v += __float_as_int(lane_xor<32>(__int_as_float(v)));
    return v;
}

// inclusive sums over the lanes of a wavefront
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // row_bcast:15
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // row_bcast:31
    return x;
}
// sum and maximum over a row of 16 lanes (quad permutes, then mirrors: what they exchange is alike in the halves by then)
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float row_sum16(float x) {
    x += dpp<0xB1>(x);
    x += dpp<0x4E>(x);
    x += dpp<0x141>(x);
    return x + dpp<0x140>(x);
}
__device__ __forceinline__ float row_max16(float x) {
    x = fmaxf(x, dpp<0xB1>(x));
    x = fmaxf(x, dpp<0x4E>(x));
    x = fmaxf(x, dpp<0x141>(x));
    return fmaxf(x, dpp<0x140>(x));
}
// with lane l ^ 32
__device__ __forceinline__ float halves_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ float halves_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
// sum over the four lanes l % 16 + 16 k: swaps of rows of 16 lanes and of halves
__device__ __forceinline__ float rows_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// and maximum over the wavefront of what is a row's alone
__device__ __forceinline__ float rows_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return halves_max(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
}

// cap * tanh(x / cap): by the exponential, or near 0, where that would cancel, by the series (its sixth term is below 2^-24)
__device__ __forceinline__ float soft_cap(float x, float cap, float inv_cap) {
    const float y = x * inv_cap, y2 = y * y;
    const float big = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * 2.88539008177792681472f) + 1.0f);
    const float small = y * fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
    return cap * (y2 < 0.0625f ? small : big);
}

__device__ __forceinline__ void unpack8_bf16(const uint4& w, float (&v)[8]) {
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        v[j] = __uint_as_float((j & 1) ? (ww[j >> 1] & 0xFFFF0000u) : (ww[j >> 1] << 16));
}

// low bytes of four registers -> one dword
__device__ __forceinline__ uint32_t pack_low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(b, a, 0x0c0c0400u) | __builtin_amdgcn_perm(d, c, 0x04000c0cu);
}

typedef float v2f_had __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf_had __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16_pair(float lo, float hi) {
    const v2bf_had r = __builtin_convertvector((v2f_had){lo, hi}, v2bf_had);   // round to nearest even
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Division of numbers below 2^31 by one that the host knows: by a product with 2^(31 + s) / d, rounded up, s the bits of d - 1
// (its error, below 2^-31 of the quotient's unit times the dividend, never reaches the next quotient).
struct FastDiv {
    uint32_t d, mul, shift;
    __host__ FastDiv() = default;
    __host__ explicit FastDiv(uint32_t n) : d(n) {
        uint32_t s = 0;
        while ((1u << s) < n && s < 31) ++s;
        shift = 31 + s;
        mul = (uint32_t)(((uint64_t)1 << shift) / n + 1);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return (uint32_t)((uint64_t)x * mul >> shift); }
};

}  // namespace resq
