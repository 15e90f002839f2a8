// The position embedding of query and key heads (in front of the projection onto the cache basis, Section 4.3), with the norm of
// each head in the same pass where a model has one:
//   n = x * rsqrt(mean(x^2) + eps) * w                                (fp32, not rounded in between; or n = x)
//   (a, b) -> m * (a cos - b sin, b cos + a sin),  angle = position * freq[i] for pair i
// and one rounding to bf16 at the end.  The angle is reduced modulo a turn in pairs of fp64 numbers, so that far positions lose nothing.
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

// cos and sin of position * freq radians.  Both products are held as a double and its error, so that what is left of whole turns is
// right to the last of its fp32 bits (a double alone is 3e-7 radians off at position 2^31, more than fp32 is).
__device__ __forceinline__ void rope_angle(int position, double freq, float& c, float& s) {
#pragma clang fp contract(off)   // (turns - rint(turns) as a product and a difference in one would hold `rest` already)
    constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;   // 1 / (2 pi)
    const double p = position, f = freq * kTurn, f_rest = fma(freq, kTurnRest, fma(freq, kTurn, -f));
    const double turns = p * f, rest = fma(p, f_rest, fma(p, f, -turns));
    sincospif(2.0f * (float)((turns - rint(turns)) + rest), &s, &c);
}

// n of a row's elements in a piece of eight, from any address on (ANY), or eight or none at a multiple of 16 bytes
template <bool ANY>
__device__ __forceinline__ void load_piece(const uint16_t* p, int n, uint4& v) {
    if constexpr (ANY) {
        if (n >= 8) {
            const Piece16 o = *reinterpret_cast<const Piece16*>(p);
            v = make_uint4(o.x, o.y, o.z, o.w);
        } else if (n > 0) {
            uint32_t w[8] = {};
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < n) w[j] = p[j];
            v = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6]);
        }
    } else if (n > 0) {
        v = *reinterpret_cast<const uint4*>(p);
    }
}
template <bool ANY>
__device__ __forceinline__ void store_piece(uint16_t* p, int n, const uint4& v) {
    if constexpr (ANY) {
        if (n >= 8) {
            *reinterpret_cast<Piece16*>(p) = Piece16{v.x, v.y, v.z, v.w};
        } else if (n > 0) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < n) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
        }
    } else if (n > 0) {
        *reinterpret_cast<uint4*>(p) = v;
    }
}

// Two 16-byte pieces to a lane, LG lanes to a head: the two pieces that a pair's halves are in, or two in a row.  The lanes of a
// workgroup are dealt to TB tokens (a power of two), each head group of which takes every so many heads of its token; the tokens'
// cosines and sines are taken once per workgroup, into LDS and from there into registers.
// ANY: rows whose pieces begin anywhere.  2048 tokens of 40 heads of 128, 54 channels turned, 14.0 us (a wavefront to a head, element by
// element, 24.7), with all turned, the norm, and rows 130 apart 12.5 (32); whole pieces of the same size 8.1 (in a captured graph,
// on one set of inputs; on three sets in turn 9.0).
// Bound by HBM from a few thousand rows on (4 bytes per channel: 8192 tokens of 40 heads of 128 26.3 us, 6.4 TB/s, part of it from
// the caches), by the launch at a step's sizes (one token 2.6 us).
template <int LG, bool ANY>
__global__ __launch_bounds__(256) void rope_pieces_kernel(const RopeArgs a, int tb_log2, int heads_per_block) {
    constexpr int kGroups = 256 / LG;
    extern __shared__ float2 turns[];   // [TB][rot / 2], one at least
    const int gl = threadIdx.x & (LG - 1), group = threadIdx.x / LG;
    const int gt = kGroups >> tb_log2;   // groups of a token
    const int64_t token0 = (int64_t)blockIdx.x << tb_log2;
    const int mine = group / gt;
    const int64_t token = token0 + mine;
    const int h_end = min(a.heads, (int)(blockIdx.y + 1) * heads_per_block);
    int head = blockIdx.y * heads_per_block + (group - mine * gt);
    const bool live = token < a.tokens;
    const int half = a.rot >> 1;

    // the lane's pieces, first channels and widths: halves of eight pairs, or neighbours.  The last piece of a stretch of channels is
    // its last eight, what it has in common with the one before done twice (and counted once).
    int ca, cb, na, nb, skip_a = 0, skip_b = 0;
    const int pair_lanes = a.interleaved ? 0 : ANY ? (half + 7) >> 3 : a.rot >> 4;   // half layout: in front of the others
    const bool pair_halves = gl < pair_lanes;
    const int begin = pair_halves ? 0 : a.interleaved ? 0 : a.rot, end = pair_halves ? half : a.d;
    ca = begin + (pair_halves ? 8 : 16) * (gl - (pair_halves ? 0 : pair_lanes));
    cb = pair_halves ? ca : ca + 8;
    na = min(8, end - ca);
    nb = min(8, end - cb);
    if (ANY && end - begin >= 8) {
        if (na > 0 && na < 8) {
            skip_a = 8 - na;
            ca = end - (na = 8);
        }
        if (nb > 0 && nb < 8) {
            skip_b = 8 - nb;
            cb = end - (nb = 8);
        }
    }
    if (pair_halves) cb += half;
    const uint16_t* xrow = a.x + (live ? token : 0) * a.ldx;
    auto load = [&](int h, uint4 (&v)[2]) {
        v[0] = v[1] = make_uint4(0u, 0u, 0u, 0u);
        if (live && h < h_end) {
            const uint16_t* p = xrow + h * a.ldxh;
            load_piece<ANY>(p + ca, na, v[0]);
            load_piece<ANY>(p + cb, nb, v[1]);
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
            load_piece<true>(wp + ca, na, w[k][0]);
            load_piece<true>(wp + cb, nb, w[k][1]);
        }
    }
    __syncthreads();
    // pair j of the lane: half layout, channels j of both pieces; interleaved, four pairs of each piece; those there are to turn
    float2 cs[8];
    uint32_t turn = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int i = a.interleaved ? ((j < 4 ? ca : cb) >> 1) + (j & 3) : ca + j;
        const bool there = (a.interleaved || pair_halves) && i < half;
        cs[j] = turns[mine * half + (there ? i : 0)];
        turn |= (uint32_t)there << j;
    }
    uint16_t* yrow = a.y + (live ? token : 0) * a.ldy;

    while (head - (group - mine * gt) < h_end) {   // (all lanes together: the norm's exchanges)
        load(head + gt, next);
        float f[2][8];
        unpack8_bf16(v[0], f[0]);
        unpack8_bf16(v[1], f[1]);
        if (a.w_q || a.w_k) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = !ANY || j >= skip_a ? f[0][j] : 0.0f, q = !ANY || j >= skip_b ? f[1][j] : 0.0f;
                sum = fmaf(p, p, fmaf(q, q, sum));
            }
            if constexpr (LG > 1) sum += lane_xor<1>(sum);
            if constexpr (LG > 2) sum += lane_xor<2>(sum);
            if constexpr (LG > 4) sum += lane_xor<4>(sum);
            if constexpr (LG > 8) sum += lane_xor<8>(sum);
            if constexpr (LG > 16) sum += lane_xor<16>(sum);
            if constexpr (LG > 32) sum += lane_xor<32>(sum);
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
                        const bool turned = turn >> (4 * k + j) & 1;   // (not by a factor of 0: the other may be infinite)
                        f[k][2 * j] = turned ? p * t.x - q * t.y : p;
                        f[k][2 * j + 1] = turned ? q * t.x + p * t.y : q;
                    }
            }
            uint16_t* dst = yrow + head * a.ldyh;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint4 o = make_uint4(pack_bf16_pair(f[k][0], f[k][1]), pack_bf16_pair(f[k][2], f[k][3]),
                                           pack_bf16_pair(f[k][4], f[k][5]), pack_bf16_pair(f[k][6], f[k][7]));
                store_piece<ANY>(dst + (k == 0 ? ca : cb), k == 0 ? na : nb, o);
            }
        }
        v[0] = next[0];
        v[1] = next[1];
        head += gt;
    }
}

}  // namespace resq
