// The position embedding of query and key heads (in front of the projection onto the cache basis, Section 4.3), with the norm of
// each head in the same pass where a model has one:
//   n = x * rsqrt(mean(x^2) + eps) * w                                (fp32, not rounded in between; or n = x)
//   (a, b) -> m * (a cos - b sin, b cos + a sin),  angle = position * freq[i] for pair i
// and one rounding to bf16 at the end.  The angle is reduced modulo a turn in fp64, so that far positions lose nothing.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_lanes.hip.h"

namespace resq {

constexpr int kRopeMaxHead = 512;

struct RopeArgs {
    const uint16_t* x;
    int64_t ldx, ldxh;
    int64_t tokens;
    int heads, heads_q, d;
    const uint16_t* w_q;
    const uint16_t* w_k;
    float eps;
    const int32_t* positions;
    const double* freq;
    int rot, interleaved;
    float mscale;
    uint16_t* y;
    int64_t ldy, ldyh;
};

// cos and sin of position * freq radians
__device__ __forceinline__ void rope_angle(int position, double freq, float& c, float& s) {
    constexpr double kTurn = 0.15915494309189533577;   // 1 / (2 pi)
    const double turns = (double)position * (freq * kTurn);
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
}

// one wavefront to a head of a token
__global__ __launch_bounds__(256) void rope_heads_kernel(const RopeArgs a) {
    __shared__ float rows[4][kRopeMaxHead];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m = (int64_t)blockIdx.x * 4 + wave;
    const bool live = m < a.tokens * a.heads;
    const int64_t token = live ? m / a.heads : 0;
    const int head = live ? (int)(m - token * a.heads) : 0;
    const uint16_t* x = a.x + token * a.ldx + head * a.ldxh;
    const uint16_t* w = head < a.heads_q ? a.w_q : a.w_k;
    float* row = rows[wave];
    float sum = 0.0f;
    for (int c = lane; c < a.d; c += 64) {
        const float v = bf16_bits_to_f32(x[c]);
        row[c] = v;
        sum += v * v;
    }
    if (w) {
        for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
        const float inv = 1.0f / sqrtf(sum / (float)a.d + a.eps);
        for (int c = lane; c < a.d; c += 64) row[c] = row[c] * inv * bf16_bits_to_f32(w[c]);
    }
    __syncthreads();
    if (!live) return;
    uint16_t* y = a.y + token * a.ldy + head * a.ldyh;
    const int half = a.rot >> 1;
    for (int i = lane; i < half; i += 64) {
        const int ca = a.interleaved ? 2 * i : i, cb = a.interleaved ? 2 * i + 1 : i + half;
        float c, s;
        rope_angle(a.positions[token], a.freq[i], c, s);
        c *= a.mscale;
        s *= a.mscale;
        const float va = row[ca], vb = row[cb];
        const uint32_t o = pack_bf16_pair(va * c - vb * s, vb * c + va * s);
        y[ca] = (uint16_t)o;
        y[cb] = (uint16_t)(o >> 16);
    }
    for (int c = a.rot + lane; c < a.d; c += 64) y[c] = (uint16_t)pack_bf16_pair(row[c], 0.0f);
}

}  // namespace resq
