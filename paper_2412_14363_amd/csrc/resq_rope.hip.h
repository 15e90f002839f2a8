// The position embedding of query and key heads (in front of the projection onto the cache basis, Section 4.3), with the norm of
// each head in the same pass where a model has one:
//   n = x * rsqrt(mean(x^2) + eps) * w                                (fp32, not rounded in between; or n = x)
//   (a, b) -> m * (a cos - b sin, b cos + a sin),  angle = position * freq[i] for pair i
// and one rounding to bf16 at the end.  The angle is reduced modulo a turn in fp64, so that far positions lose nothing.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_lanes.hip.h"
#include "resq_layout.h"

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

// Rows of whole 16-byte pieces, two of them to a lane, LG lanes to a head: the two pieces that a pair's halves are in, or two in
// a row.  The lanes of a workgroup are dealt to TB tokens (a power of two), each head group of which takes every so many heads
// of its token; the tokens' cosines and sines are taken once per workgroup, into LDS and from there into registers.
// Bound by HBM from a few thousand rows on (4 bytes per channel: 8192 tokens of 40 heads of 128 26.7 us, 6.3 TB/s, part of it from
// the caches), by the launch at a step's sizes (one token 2.7 us).
template <int LG>
__global__ __launch_bounds__(256) void rope_pieces_kernel(const RopeArgs a, int tb_log2, int heads_per_block) {
    constexpr int kGroups = 256 / LG;
    extern __shared__ float2 turns[];   // [TB][rot / 2]
    const int gl = threadIdx.x & (LG - 1), group = threadIdx.x / LG;
    const int gt = kGroups >> tb_log2;   // groups of a token
    const int64_t token0 = (int64_t)blockIdx.x << tb_log2;
    const int mine = group / gt;
    const int64_t token = token0 + mine;
    const int h_end = min(a.heads, (int)(blockIdx.y + 1) * heads_per_block);
    int head = blockIdx.y * heads_per_block + (group - mine * gt);
    const bool live = token < a.tokens;
    const int half = a.rot >> 1, pieces = a.d >> 3;

    // the lane's pieces: halves of eight pairs, or neighbours
    int pa, pb;
    if (!a.interleaved && gl < a.rot >> 4) {
        pa = gl;
        pb = gl + (a.rot >> 4);
    } else {
        pa = 2 * gl;   // (half layout: in front of them rot / 16 lanes with two pieces each)
        pb = pa + 1;
    }
    const bool has_a = pa < pieces, has_b = pb < pieces;
    const uint16_t* xrow = a.x + (live ? token : 0) * a.ldx;
    auto load = [&](int h, uint4 (&v)[2]) {
        v[0] = v[1] = make_uint4(0u, 0u, 0u, 0u);
        if (live && h < h_end) {
            const uint4* p = reinterpret_cast<const uint4*>(xrow + h * a.ldxh);
            if (has_a) v[0] = p[pa];
            if (has_b) v[1] = p[pb];
        }
    };
    uint4 v[2], next[2];
    load(head, v);

    for (int e = threadIdx.x; e < half << tb_log2; e += 256) {
        const int tok = e / half, i = e - tok * half;
        if (token0 + tok < a.tokens) {
            float c, s;
            rope_angle(a.positions[token0 + tok], a.freq[i], c, s);
            turns[e] = make_float2(c * a.mscale, s * a.mscale);
        }
    }
    // the norms' weights of the lane's pieces, for queries and for keys
    uint4 w[2][2];
    if (a.w_q || a.w_k) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint16_t* wp = k ? a.w_k : a.w_q;
            w[k][0] = w[k][1] = make_uint4(0u, 0u, 0u, 0u);
            if (!wp) continue;
            if (has_a) {
                const Piece16 p = reinterpret_cast<const Piece16*>(wp)[pa];
                w[k][0] = make_uint4(p.x, p.y, p.z, p.w);
            }
            if (has_b) {
                const Piece16 p = reinterpret_cast<const Piece16*>(wp)[pb];
                w[k][1] = make_uint4(p.x, p.y, p.z, p.w);
            }
        }
    }
    __syncthreads();
    // pair j of the lane: half layout, channels j of both pieces; interleaved, four pairs of each piece
    float2 cs[8];
    const bool turn_a = 8 * pa < a.rot, turn_b = 8 * pb < a.rot;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int i = a.interleaved ? 4 * (j < 4 ? pa : pb) + (j & 3) : 8 * pa + j;
        const bool turn = a.interleaved && j >= 4 ? turn_b : turn_a;
        cs[j] = turn ? turns[mine * half + i] : make_float2(1.0f, 0.0f);
    }
    const bool pair_halves = !a.interleaved && turn_a;
    uint16_t* yrow = a.y + (live ? token : 0) * a.ldy;

    while (head - (group - mine * gt) < h_end) {   // (all lanes together: the norm's exchanges)
        load(head + gt, next);
        float f[2][8];
        unpack8_bf16(v[0], f[0]);
        unpack8_bf16(v[1], f[1]);
        if (a.w_q || a.w_k) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(f[0][j], f[0][j], fmaf(f[1][j], f[1][j], sum));
            if constexpr (LG > 1) sum += lane_xor<1>(sum);
            if constexpr (LG > 2) sum += lane_xor<2>(sum);
            if constexpr (LG > 4) sum += lane_xor<4>(sum);
            if constexpr (LG > 8) sum += lane_xor<8>(sum);
            if constexpr (LG > 16) sum += lane_xor<16>(sum);
            const float inv = 1.0f / sqrtf(sum / (float)a.d + a.eps);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float g[8];
                unpack8_bf16(head < a.heads_q ? w[0][k] : w[1][k], g);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[k][j] = f[k][j] * inv * g[j];
            }
        }
        if (live && head < h_end) {
            if (pair_halves) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float p = f[0][j], q = f[1][j];
                    f[0][j] = p * cs[j].x - q * cs[j].y;
                    f[1][j] = q * cs[j].x + p * cs[j].y;
                }
            } else if (a.interleaved) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float p = f[k][2 * j], q = f[k][2 * j + 1];
                        const float2 t = cs[4 * k + j];
                        f[k][2 * j] = p * t.x - q * t.y;
                        f[k][2 * j + 1] = q * t.x + p * t.y;
                    }
            }
            uint4* dst = reinterpret_cast<uint4*>(yrow + head * a.ldyh);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint4 o = make_uint4(pack_bf16_pair(f[k][0], f[k][1]), pack_bf16_pair(f[k][2], f[k][3]),
                                           pack_bf16_pair(f[k][4], f[k][5]), pack_bf16_pair(f[k][6], f[k][7]));
                if (k == 0 ? has_a : has_b) dst[k == 0 ? pa : pb] = o;
            }
        }
        v[0] = next[0];
        v[1] = next[1];
        head += gt;
    }
}

// Any other rows, element by element: a workgroup to a token, whose cosines and sines it takes once, a wavefront to every fourth
// head; the next head's elements are asked for before this one's are turned.
__global__ __launch_bounds__(256) void rope_heads_kernel(const RopeArgs a, int heads_per_block) {
    constexpr int kEach = kRopeMaxHead / 64;   // elements of a lane at most
    __shared__ float rows[4][kRopeMaxHead];
    __shared__ float2 turns[kRopeMaxHead / 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = a.rot >> 1;
    const int64_t token = blockIdx.x;
    const int h_begin = blockIdx.y * heads_per_block, h_end = min(a.heads, h_begin + heads_per_block);
    const uint16_t* x = a.x + token * a.ldx;
    uint32_t v[kEach] = {};
    auto load = [&](int head) {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (64 * k < a.d && 64 * k + lane < a.d) v[k] = x[head * a.ldxh + 64 * k + lane];
    };
    int head = h_begin + wave;
    if (head < h_end) load(head);
    for (int i = threadIdx.x; i < half; i += 256) {
        float c, s;
        rope_angle(a.positions[token], a.freq[i], c, s);
        turns[i] = make_float2(c * a.mscale, s * a.mscale);
    }
    __syncthreads();
    float* row = rows[wave];
    for (; head < h_end; head += 4) {
        float f[kEach], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            f[k] = 64 * k + lane < a.d ? bf16_bits_to_f32(v[k]) : 0.0f;
            sum = fmaf(f[k], f[k], sum);
        }
        if (head + 4 < h_end) load(head + 4);
        const uint16_t* w = head < a.heads_q ? a.w_q : a.w_k;
        float inv = 1.0f;
        if (w) {
            for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
            inv = 1.0f / sqrtf(sum / (float)a.d + a.eps);
        }
        uint16_t* y = a.y + token * a.ldy + head * a.ldyh;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int c = 64 * k + lane;
            if (64 * k < a.d && c < a.d) {
                const float g = w ? f[k] * inv * bf16_bits_to_f32(w[c]) : f[k];
                if (c < a.rot) row[c] = g;
                else y[c] = (uint16_t)pack_bf16_pair(g, 0.0f);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        for (int i = lane; i < half; i += 64) {
            const int ca = a.interleaved ? 2 * i : i, cb = a.interleaved ? 2 * i + 1 : i + half;
            const float2 cs = turns[i];
            const float va = row[ca], vb = row[cb];
            const uint32_t o = pack_bf16_pair(va * cs.x - vb * cs.y, vb * cs.x + va * cs.y);
            y[ca] = (uint16_t)o;
            y[cb] = (uint16_t)(o >> 16);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace resq
