// Compact K/V cache rows (Section 5.1 and Appendix C: the cache is quantized per
// head with the asymmetric quantizer of Eq. 1, an eighth of the channels in 8
// bits).  One row per head of a token, no padding:
//   r bytes: the 8-bit codes, 0..255 | (d - r) / 2 bytes: the 4-bit codes, 0..15,
//   channel r + 2j in bits 0..3, r + 2j + 1 in bits 4..7 | fp32 s_hi, z_hi, s_lo, z_lo
// with x ~ code * s + z per group: r + (d - r) / 2 + 16 bytes for 2 d bytes of bf16.
// G lanes hold a row, eight channels each: no LDS, no barrier.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_lanes.hip.h"

namespace resq {

// a row's numbers at any even address (a row of paged K/V whose r is an odd multiple of four has 4 k + 2 bytes)
struct __attribute__((packed, aligned(2))) EvenDword { uint32_t v; };
struct __attribute__((packed, aligned(2))) EvenFloat { float v; };

// One row: v holds channels [C gl, C gl + C) of it in lane gl of the G lanes (all lanes of a wavefront call this: exchanges
// and votes), row is where its bytes go, null for none.  C = 8, or 4 where r is not a multiple of eight: a lane's are of one group.
template <int G, int C = 8>
__device__ __forceinline__ void quantize_kv_row(const uint4 v, int gl, int d, int r, uint8_t* __restrict__ row) {
    const int nunits = d / C, hi_units = r / C;
    const bool live = gl < nunits, high = gl < hi_units;
    const float inf = __builtin_huge_valf();
    float mx = -inf, nmn = -inf;
    if (live) {
        float f[8];
        unpack8_bf16(v, f);
        if constexpr (C == 8) {
            mx = fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7])));
            nmn = -fminf(fminf(fminf(f[0], f[1]), fminf(f[2], f[3])), fminf(fminf(f[4], f[5]), fminf(f[6], f[7])));
        } else {
            mx = fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3]));
            nmn = -fminf(fminf(f[0], f[1]), fminf(f[2], f[3]));
        }
    }
    const float mx_h = wave_max<G>(high ? mx : -inf), nmn_h = wave_max<G>(high ? nmn : -inf);
    const float mx_l = wave_max<G>(live && !high ? mx : -inf);
    const float nmn_l = wave_max<G>(live && !high ? nmn : -inf);
    // A lane's columns are all of one group: it needs one scale, one reciprocal and one pass of the
    // quantizer, with the constants of its own group (run for both groups on all lanes and
    // selected afterwards, which the votes across the wavefront suggest, it took 6.7 instead of 5.0 us
    // for 32768 rows of 128 columns at r = 16, and 30.4 instead of 22.4, 4.0 TB/s, for 262144; by events at the
    // kernel's start and end, a kernel trace says 0.7 us more).
    const float levels = high ? 255.0f : 15.0f;
    const float zero = live ? -(high ? nmn_h : nmn_l) : 0.0f;
    const float range = live ? (high ? mx_h : mx_l) - zero : 0.0f;
    const float scale = range == 0.0f ? 1.0f : range / levels;  // asym_scale
    const float inv = 1.0f / scale;
    constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: quant8_asym, with the codes themselves
    const float tie = 0.5f - (levels + 1.0f) * 9.5367431640625e-07f;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float ds[C];
    uint32_t u[C];
    bool near_tie[C], any_tie = false;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        ds[j] = __uint_as_float((j & 1) ? (w[j >> 1] & 0xFFFF0000u) : (w[j >> 1] << 16)) - zero;
        const float t = ds[j] * inv;
        const float uf = t + kMagic;
        near_tie[j] = !(fabsf(t - (uf - kMagic)) <= tie);
        any_tie |= near_tie[j];
        u[j] = __float_as_uint(uf);
    }
    if (__builtin_amdgcn_ballot_w64(any_tie) != 0) {  // wave-uniform, then per element slot
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (__builtin_amdgcn_ballot_w64(near_tie[j]) != 0)
                u[j] = (uint32_t)(int)fminf(fmaxf(rintf(ds[j] / scale), 0.0f), levels);
    }
    if (!row || !live) return;
    if constexpr (C == 4) {
        if (high) reinterpret_cast<EvenDword*>(row + gl * 4)->v = pack_low_bytes(u[0], u[1], u[2], u[3]);
        else
            *reinterpret_cast<uint16_t*>(row + r + (gl - hi_units) * 2) =
                (uint16_t)((u[0] & 0xFu) | (u[1] & 0xFu) << 4 | (u[2] & 0xFu) << 8 | (u[3] & 0xFu) << 12);
        if (gl == 0 || gl == hi_units) {   // (both groups are there: r is no multiple of eight, d is)
            EvenFloat* p = reinterpret_cast<EvenFloat*>(row + r + (d - r) / 2) + (high ? 0 : 2);
            p[0].v = scale;
            p[1].v = zero;
        }
        return;
    }
    float* par = reinterpret_cast<float*>(row + r + (d - r) / 2);
    if (high) {
        uint32_t* dst = reinterpret_cast<uint32_t*>(row + gl * 8);   // rows are 4-byte aligned
        dst[0] = pack_low_bytes(u[0], u[1], u[2], u[3]);
        dst[1] = pack_low_bytes(u[4], u[5], u[6], u[7]);
    } else {
        uint32_t by[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) by[k] = (u[2 * k + 1] << 4) | (u[2 * k] & 0xFu);
        *reinterpret_cast<uint32_t*>(row + r + (gl - hi_units) * 4) = pack_low_bytes(by[0], by[1], by[2], by[3]);
    }
    // The first lane of a group writes its constants.  A row of one group: all four in one store by the first
    // lane, scale 1 and zero-point 0 for the absent group (the present one's two and the absent one's apart:
    // 262144 rows of 128 columns 24.4 / 21.1 us at r = 0, 24.8 / 22.1 at r = 128).
    if (hi_units == 0 || hi_units == nunits) {
        if (gl == 0) {
            par[0] = high ? scale : 1.0f;
            par[1] = high ? zero : 0.0f;
            par[2] = high ? 1.0f : scale;
            par[3] = high ? 0.0f : zero;
        }
    } else if (gl == 0 || gl == hi_units) {
        par[high ? 0 : 2] = scale;
        par[high ? 1 : 3] = zero;
    }
}

// The reader of rows with C = 4: channels [4 gl, 4 gl + 4).
__device__ __forceinline__ uint2 dequantize_kv_half_piece(const uint8_t* __restrict__ row, int gl, int d, int r) {
    const bool high = 4 * gl < r;
    const EvenFloat* par = reinterpret_cast<const EvenFloat*>(row + r + (d - r) / 2) + (high ? 0 : 2);
    const uint32_t c = high ? reinterpret_cast<const EvenDword*>(row + gl * 4)->v
                            : *reinterpret_cast<const uint16_t*>(row + r + (gl - (r >> 2)) * 2);
    const float s = par[0].v, z = par[1].v;
    float f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = fmaf((float)(high ? (c >> (8 * k)) & 0xFFu : (c >> (4 * k)) & 0xFu), s, z);
    return make_uint2(pack_bf16_pair(f[0], f[1]), pack_bf16_pair(f[2], f[3]));
}

// The reader of such rows: channels [8 gl, 8 gl + 8) of x[m, k] = bf16(code * s + z) (Eq. 1).
__device__ __forceinline__ uint4 dequantize_kv_piece(const uint8_t* __restrict__ row, int gl, int d, int r) {
    const int hi_units = r >> 3;
    const float* par = reinterpret_cast<const float*>(row + r + (d - r) / 2);
    float f[8];
    if (gl < hi_units) {
        const uint32_t* src = reinterpret_cast<const uint32_t*>(row + gl * 8);
        const uint32_t c0 = src[0], c1 = src[1];
        const float s = par[0], z = par[1];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = fmaf((float)(((k < 4 ? c0 : c1) >> (8 * (k & 3))) & 0xFFu), s, z);
    } else {
        const uint32_t c = *reinterpret_cast<const uint32_t*>(row + r + (gl - hi_units) * 4);
        const float s = par[2], z = par[3];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = fmaf((float)((c >> (4 * k)) & 0xFu), s, z);
    }
    uint4 o;
    o.x = pack_bf16_pair(f[0], f[1]);
    o.y = pack_bf16_pair(f[2], f[3]);
    o.z = pack_bf16_pair(f[4], f[5]);
    o.w = pack_bf16_pair(f[6], f[7]);
    return o;
}

}  // namespace resq
