// What stands between two blocks of a layer, in one pass over each token's row:
//   a  = y, or y * rsqrt(mean(y^2) + eps) * (offset + w_post)        the norm behind the block
//   h' = h + alpha * gate * a                                         gate, residual scale, residual sum
//   x  = h' * rsqrt(mean(h'^2) + eps) * (offset + w_pre)              the norm in front of the next block
// all of it in fp32 with one rounding of each output (x from h' as it was before its rounding).  A row stays in the registers of T
// threads, 8 P channels each: everything is read once, at once, and the two sums of squares are the only exchanges.  (P = 4, above 16384
// channels: 104 bytes of each thread go through scratch memory; 2048 x 32768 in bf16 177 us, 3.0 TB/s.)
// Bound by HBM.  Measured on MI355X: 8192 x 8192, fp32 residual stream, gate 172 us, 5.5 TB/s; 3001 x 8192 in bf16 with both norms 40 us, 4.9
// TB/s (a copy of 1 GiB reaches 5.1, a plain kernel with the first call's reads and writes 5.25, with the second's 5.2); one token of 4096 7 us, 2.3 of them the kernel, the rest the host's call.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_lanes.hip.h"
#include "resq_layout.h"

namespace resq {

constexpr int kNormMaxWidth = 32768;

struct NormArgs {
    const uint16_t* y;      // null: no block, h' = h
    int64_t ldy;
    const uint16_t* gate;   // null: 1
    int64_t ldg;
    const void* h;
    int64_t ldh;
    const uint16_t *w_post, *w_pre;   // null: no norm
    float offset, eps, alpha;
    void* h_out;            // null: not written
    int64_t ldho;
    uint16_t* x;            // null: not written
    int64_t ldx;
    int64_t tokens;
    int width;
};

struct __attribute__((packed, aligned(4))) Floats4 { float v[4]; };

// channels [c, c + 8) of a row, zeros behind its last one
__device__ __forceinline__ void norm_load(const uint16_t* row, int c, int width, float (&v)[8]) {
    if (c + 8 <= width) {
        const Piece16 p = *reinterpret_cast<const Piece16*>(row + c);
        unpack8_bf16(make_uint4(p.x, p.y, p.z, p.w), v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < width ? bf16_bits_to_f32(row[c + i]) : 0.0f;
    }
}
__device__ __forceinline__ void norm_load(const float* row, int c, int width, float (&v)[8]) {
    if (c + 8 <= width) {
        const Floats4 p = *reinterpret_cast<const Floats4*>(row + c), q = *reinterpret_cast<const Floats4*>(row + c + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = p.v[i];
            v[4 + i] = q.v[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < width ? row[c + i] : 0.0f;
    }
}
__device__ __forceinline__ void norm_store(uint16_t* row, int c, int width, const float (&v)[8]) {
    uint32_t p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pack_bf16_pair(v[2 * i], v[2 * i + 1]);
    if (c + 8 <= width) {
        *reinterpret_cast<Piece16*>(row + c) = Piece16{p[0], p[1], p[2], p[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < width) row[c + i] = (uint16_t)(p[i >> 1] >> (16 * (i & 1)));
    }
}
__device__ __forceinline__ void norm_store(float* row, int c, int width, const float (&v)[8]) {
    if (c + 8 <= width) {
        Floats4 p, q;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p.v[i] = v[i];
            q.v[i] = v[4 + i];
        }
        *reinterpret_cast<Floats4*>(row + c) = p;
        *reinterpret_cast<Floats4*>(row + c + 4) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < width) row[c + i] = v[i];
    }
}

// T threads to a row, in workgroups of at least 256, P pieces of 8 channels to a thread; H: the type of h
template <int T, int P, typename H>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_residual_kernel(const NormArgs a) {
    constexpr int kThreads = T < 256 ? 256 : T, kWaves = T / 64;
    __shared__ float part[2][kThreads / 64];
    const int t = threadIdx.x % T, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * (kThreads / T) + threadIdx.x / T;
    const bool live = token < a.tokens;
    const int width = live ? a.width : 0;
    const int64_t at = live ? token : 0;

    auto squares = [&](const float (&v)[P][8], int which) {   // rsqrt of the row's mean square
        float s = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(v[p][i], v[p][i], s);
        s = rows_sum(row_sum16(s));
        if constexpr (kWaves > 1) {
            if (lane == 0) part[which][wave] = s;
            __syncthreads();
            s = 0.0f;
            const int first = wave / kWaves * kWaves;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s += part[which][first + w];
        }
        // (the instruction takes what is below the normal numbers for 0)
        s = s / (float)a.width + a.eps;
        const bool tiny = s < 1.17549435e-38f;
        return __builtin_amdgcn_rsqf(tiny ? s * 4294967296.0f : s) * (tiny ? 65536.0f : 1.0f);
    };

    float y[P][8], h[P][8];
    const H* h_row = static_cast<const H*>(a.h) + at * a.ldh;
#pragma unroll
    for (int p = 0; p < P; ++p) norm_load(h_row, 8 * (t + p * T), width, h[p]);
    if (a.y) {
        float g[P][8], w[P][8];
#pragma unroll
        for (int p = 0; p < P; ++p) norm_load(a.y + at * a.ldy, 8 * (t + p * T), width, y[p]);
        if (a.gate) {
#pragma unroll
            for (int p = 0; p < P; ++p) norm_load(a.gate + at * a.ldg, 8 * (t + p * T), width, g[p]);
        }
        if (a.w_post) {
#pragma unroll
            for (int p = 0; p < P; ++p) norm_load(a.w_post, 8 * (t + p * T), width, w[p]);
            const float f = squares(y, 0);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[p][i] *= f * (a.offset + w[p][i]);
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) h[p][i] = fmaf(a.alpha, a.gate ? y[p][i] * g[p][i] : y[p][i], h[p][i]);
    }
    if (a.h_out) {
        H* row = static_cast<H*>(a.h_out) + at * a.ldho;
#pragma unroll
        for (int p = 0; p < P; ++p) norm_store(row, 8 * (t + p * T), width, h[p]);
    }
    if (a.x) {
        float w[P][8];
#pragma unroll
        for (int p = 0; p < P; ++p) norm_load(a.w_pre, 8 * (t + p * T), width, w[p]);
        const float f = squares(h, 1);
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[p][i] = h[p][i] * (f * (a.offset + w[p][i]));
            norm_store(a.x + at * a.ldx, 8 * (t + p * T), width, w[p]);
        }
    }
}

}  // namespace resq
