// Attention of one new token of each sequence over a prefix that all sequences of the batch share, in pages of compact K/V rows
// (resq_kv_row.hip.h): for each K/V head the queries of all sequences are rows of one product, so that the prefix is read and made into
// numbers once for 128 of them and not once for each sequence.  The sequences' own tokens are resq_attend.hip.h's; a last kernel joins both.
//   k_t = code * s + z of each group, x = scale * q . k_t, capped or not; out = sum e^(x - lse) v, as there
//
// A workgroup makes a tile of 64 rows into fp16 numbers in LDS and has 128 queries attend to it (resq_flash.hip.h).  fp16 holds
// code * s + z to 2^-12 of itself, an eighth of what bf16 loses, which would add as much again to the error of a bf16 result; its range is
// made up for by powers of two: of a query (its largest channel becomes 2^13), of the keys of 16 tokens, and of the values of all tokens so
// far.  What is below 2^-27 of the largest number of its 16 tokens loses bits, down to 2^-38 of it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_flash.hip.h"

namespace resq {

constexpr int kPrefixThreads = 256;
constexpr int kPrefixWaves = kPrefixThreads / 64;
constexpr int kPrefixRows = kFlashRows * kPrefixWaves;   // of a workgroup
constexpr int kPrefixKeys = 64;
constexpr int kPrefixLeast = 512 / kPrefixKeys;          // tiles of a part at least

struct PrefixArgs {
    const uint16_t* q;
    int64_t ldq, ldqh;
    int B, heads_k, d, r, row_bytes;
    FastDiv share, parts, heads;
    const int32_t* prefix_len;
    const int32_t* prefix_table;
    int max_prefix;        // tokens that the prefix's table can name
    const int32_t* lens;   // own tokens of each sequence, below 0: the sequence is not there
    const uint8_t* pages[2];
    int num_pages;
    FastDiv page_size;
    int64_t page_stride, head_stride, row_stride;
    float scale, softcap;
    int window;            // 2^30: none
    const float* own_out;  // [B][heads_q][d], [B][heads_q]: the own tokens' results (workspace)
    const float* own_lse;
    uint16_t* out;
    int64_t ldo, ldoh;
    float* lse;
    float* part_ml;        // [tile, head, part][128][2]: maximum (times log2 e) and sum (workspace)
    float* part_acc;       // [tile, head, part][128][d]: weighted sums (workspace)
};

// The tokens of the prefix that some row may see, [begin, end) with begin a multiple of a tile, and the parts they are cut into.
struct PrefixKeys {
    int begin, end, per, parts;
};
__device__ __forceinline__ PrefixKeys prefix_keys(const PrefixArgs& a) {
    PrefixKeys k;
    k.end = min(max(a.prefix_len[0], 0), a.max_prefix);
    k.begin = max(k.end - a.window, 0) / kPrefixKeys * kPrefixKeys;   // (own tokens leave fewer)
    const int tiles = (k.end - k.begin + kPrefixKeys - 1) / kPrefixKeys;
    const int parts = min((int)a.parts.d, max(tiles / kPrefixLeast, 1));
    k.per = (tiles + parts - 1) / parts;
    k.parts = k.per ? (tiles + k.per - 1) / k.per : 0;
    return k;
}

// 2^e of exponent bits e, and 2^13 over it, which makes numbers below 2^(e + 1) ones below 2^14
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)e << 23); }
__device__ __forceinline__ int exponent_of(float x) { return max((int)(__float_as_uint(x) >> 23), 27); }   // x >= 0; bits, 127 is 2^0
__device__ __forceinline__ float to_half_range(int e) { return two_to(267 - e); }

template <int W, int OCC, bool CAP>
__global__ __launch_bounds__(kPrefixThreads, OCC) void attend_prefix_kernel(const PrefixArgs a) {
    using Tile = FlashTile<W>;
    constexpr int KEYS = kPrefixKeys, kTileBytes = KEYS * Tile::kPitch;
    constexpr int kLanes = kPrefixThreads / KEYS;       // threads of a token
    constexpr int kUnits = Tile::kPieces / kLanes;      // pieces of 8 channels of a thread
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // two tiles of keys, two of values
    struct Group { int key, value, there, pad; };       // of 16 tokens: exponents of keys and values, and which of them there are
    __shared__ __attribute__((aligned(16))) Group groups[2][KEYS / 16];

    const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int unit = (int)a.heads(blockIdx.x), hk = (int)blockIdx.x - unit * a.heads_k;
    const int tile = (int)a.parts(unit), piece = unit - tile * (int)a.parts.d;
    const PrefixKeys keys = prefix_keys(a);
    if (piece >= keys.parts) return;
    const int begin = keys.begin + piece * keys.per * KEYS, end = min(keys.end, begin + keys.per * KEYS);

    // ---- the own row ----
    const int rows = a.B * (int)a.share.d, row = tile * kPrefixRows + wave * kFlashRows + (lane & 31);
    const bool live = row < rows;
    const int b = (int)a.share(live ? row : 0), head = hk * (int)a.share.d + (live ? row : 0) - b * (int)a.share.d;
    const int own = a.lens[b];
    // the first token that the row sees: own tokens count for the window too
    const int low = live && own >= 0 ? (int)max((int64_t)keys.end + own - a.window, (int64_t)0) : 0x7FFFFFFF;
    FlashRow<W, true> r;
    r.clear();
    float qf;   // what a score's product is multiplied with for the query's part
    {
        const uint16_t* src = a.q + b * a.ldq + head * a.ldqh;
        float top = 0.0f;
#pragma unroll
        for (int s = 0; s < Tile::kSteps; ++s) {
            const int ch = 16 * s + 8 * half;
            Piece16 p{0u, 0u, 0u, 0u};
            if (live && ch < a.d) p = *reinterpret_cast<const Piece16*>(src + ch);
            r.q[s] = (v4u_flash){p.x, p.y, p.z, p.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top = fmaxf(top, fmaxf(__uint_as_float(r.q[s][e] << 16 & 0x7FFF0000u), __uint_as_float(r.q[s][e] & 0x7FFF0000u)));
        }
        const int e = exponent_of(halves_max(top));
        const float f = to_half_range(e);
#pragma unroll
        for (int s = 0; s < Tile::kSteps; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r.q[s][i] = flash_pack<true>(__uint_as_float(r.q[s][i] << 16) * f, __uint_as_float(r.q[s][i] & 0xFFFF0000u) * f);
        qf = a.scale * two_to(e - 13);
        if (!CAP) qf *= 1.44269504088896340736f;
    }
    const bool looks = __builtin_amdgcn_ballot_w64(low < end) != 0;   // some row of the wavefront sees something
    const int low_there = low == 0x7FFFFFFF ? 0 : low;                // of a row that is there

    // ---- rows of a tile: read two tiles ahead, made into numbers one ahead ----
    const int my_token = t / kLanes, my_unit = t % kLanes;
    const int64_t head_off = hk * a.head_stride;
    int page_next = -1;
    bool there = false;
    uint2 code[2][kUnits];
    float par[2][4];
    auto load_page = [&](int key0) {
        const int tok = key0 + my_token;
        page_next = -1;
        if (tok < end) page_next = a.prefix_table[a.page_size((uint32_t)tok)];
    };
    auto load = [&](int key0) {
        const int tok = key0 + my_token;
        there = (unsigned)page_next < (unsigned)a.num_pages;
        if (there) {
            const int64_t off = page_next * a.page_stride + (tok - (int)a.page_size((uint32_t)tok) * (int)a.page_size.d) * a.row_stride + head_off;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const uint8_t* src = a.pages[kv] + off;
                const Piece16 p = *reinterpret_cast<const Piece16*>(src + a.row_bytes - 16);
                par[kv][0] = __uint_as_float(p.x);
                par[kv][1] = __uint_as_float(p.y);
                par[kv][2] = __uint_as_float(p.z);
                par[kv][3] = __uint_as_float(p.w);
#pragma unroll
                for (int u = 0; u < kUnits; ++u) {
                    const int ch = 8 * (my_unit + u * kLanes);   // of the 8-bit group, of the 4-bit one, or half and half
                    code[kv][u] = make_uint2(0u, 0u);
                    if (ch + 8 <= a.r) {
                        const Piece8 c = *reinterpret_cast<const Piece8*>(src + ch);
                        code[kv][u] = make_uint2(c.x, c.y);
                    } else if (ch >= a.r) {
                        if (ch < a.d) code[kv][u].x = reinterpret_cast<const Piece4*>(src + a.r + ((ch - a.r) >> 1))->x;
                    } else {
                        code[kv][u].x = reinterpret_cast<const Piece4*>(src + ch)->x;
                        code[kv][u].y = *reinterpret_cast<const uint16_t*>(src + a.r);
                    }
                }
            }
        } else {
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
                for (int i = 0; i < 4; ++i) par[kv][i] = 0.0f;
#pragma unroll
                for (int u = 0; u < kUnits; ++u) code[kv][u] = make_uint2(0u, 0u);
            }
        }
    };
    const float inf = __builtin_huge_valf();
    // value_e: the exponent that values are counted in so far
    auto store = [&](int buffer, int value_e) {
        uint8_t* dst[2] = {lds + buffer * kTileBytes, lds + (2 + buffer) * kTileBytes};
        int e[2];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            float top = 0.0f;
            if (a.r > 0) top = fmaxf(fabsf(par[kv][1]), fabsf(fmaf(255.0f, par[kv][0], par[kv][1])));
            if (a.r < a.d) top = fmaxf(top, fmaxf(fabsf(par[kv][3]), fabsf(fmaf(15.0f, par[kv][2], par[kv][3]))));
            e[kv] = exponent_of(rows_max(row_max16(top < inf ? top : 0.0f)));   // a wavefront has 16 tokens
            if (kv == 1) e[1] = max(e[1], value_e);
            const float f = to_half_range(e[kv]);
            const float sh = par[kv][0] * f, zh = par[kv][1] * f, sl = par[kv][2] * f, zl = par[kv][3] * f;
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                const int piece = my_unit + u * kLanes, ch = 8 * piece;
                const uint2 c = code[kv][u];
                float v[8];
                if (ch >= a.r) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = fmaf((float)(c.x >> (4 * i) & 15u), sl, zl);
                } else {
                    const bool mixed = ch + 8 > a.r;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[i] = fmaf((float)(c.x >> (8 * i) & 255u), sh, zh);
                        v[4 + i] = mixed ? fmaf((float)(c.y >> (4 * i) & 15u), sl, zl) : fmaf((float)(c.y >> (8 * i) & 255u), sh, zh);
                    }
                }
                const v4u_flash o = {flash_pack<true>(v[0], v[1]), flash_pack<true>(v[2], v[3]), flash_pack<true>(v[4], v[5]), flash_pack<true>(v[6], v[7])};
                *reinterpret_cast<v4u_flash*>(dst[kv] + (kv ? Tile::value_at(my_token, piece) : Tile::key_at(my_token, piece))) = o;
            }
        }
        const uint64_t some = __builtin_amdgcn_ballot_w64(there);
        if (lane == 0) {
            int mask = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) mask |= (int)(some >> (kLanes * i) & 1) << i;
            groups[buffer][wave] = Group{e[0], e[1], mask, 0};
        }
    };
    static_assert(KEYS == 16 * kPrefixWaves);
    const float inv_cap = CAP ? 1.0f / a.softcap : 0.0f;

    int value_e = 27;   // (the exponent of the tile that is attended to, and of all before)
    load_page(begin);
    load(begin);
    load_page(begin + KEYS);
    store(0, value_e);
    load(begin + KEYS);
    load_page(begin + 2 * KEYS);
    __syncthreads();
    int buffer = 0;
    for (int key0 = begin; key0 < end; key0 += KEYS, buffer ^= 1) {
        // ---- what this tile is counted in ----
        float f[KEYS / 16], up[KEYS / 16];
        int ve[KEYS / 16], e_new = value_e;
        uint64_t mask = 0;
#pragma unroll
        for (int g = 0; g < KEYS / 16; ++g) {
            const Group gr = groups[buffer][g];
            f[g] = qf * two_to(__builtin_amdgcn_readfirstlane(gr.key) - 13);
            ve[g] = __builtin_amdgcn_readfirstlane(gr.value);
            e_new = max(e_new, ve[g]);
            mask |= (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(gr.there) << (16 * g);
        }
        bool scaled = false;
#pragma unroll
        for (int g = 0; g < KEYS / 16; ++g) {
            up[g] = two_to(max(127 + ve[g] - e_new, 0));
            scaled |= ve[g] != e_new;
        }
        if (e_new != value_e) {
            const float back = two_to(max(127 + value_e - e_new, 0));
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) r.acc[c] *= back;
            value_e = e_new;
        }
        if (key0 + KEYS < end) {
            store(buffer ^ 1, value_e);
            if (key0 + 2 * KEYS < end) {
                load(key0 + 2 * KEYS);
                load_page(key0 + 3 * KEYS);
            }
        }
        if (looks) {
            const uint8_t *kt = lds + buffer * kTileBytes, *vt = lds + (2 + buffer) * kTileBytes;
            const bool partly = mask != ~0ull || __builtin_amdgcn_ballot_w64(low_there > key0) != 0;
            const int from = low - key0;
            auto sees = [&](int key) { return (mask >> key & 1) != 0 && key >= from; };
            const float* by = scaled ? up : nullptr;
            if (partly) r.template step<KEYS, CAP, false, true>(kt, vt, f, by, a.softcap, inv_cap, sees);
            else r.template step<KEYS, CAP, false, false>(kt, vt, f, by, a.softcap, inv_cap, sees);
        }
        __syncthreads();
    }

    // ---- this part of the result ----
    const float sum = halves_sum(r.l) * two_to(127 - (int)kFlashHalfBias);
    if (!live) return;
    const float f = two_to(max(value_e - 13 - (int)kFlashHalfBias, 0));
    const int64_t slot = ((int64_t)tile * a.heads_k + hk) * a.parts.d + piece;
    const int at = wave * kFlashRows + (lane & 31);
    float* dst = a.part_acc + (slot * kPrefixRows + at) * a.d;
#pragma unroll
    for (int c = 0; c < Tile::kBlocks; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int ch = 32 * c + 8 * (i >> 2) + 4 * half;
            if (ch < a.d)
                *reinterpret_cast<float4*>(dst + ch) = make_float4(r.acc[c][i] * f, r.acc[c][i + 1] * f, r.acc[c][i + 2] * f, r.acc[c][i + 3] * f);
        }
    if (half == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * kPrefixRows + at) * 2) = make_float2(r.m, sum);
}

// Joins the parts of the prefix and the own tokens' result, whose maximum is its log-sum-exp and whose sum is 1; four channels to a thread.
__global__ __launch_bounds__(kPrefixThreads) void attend_prefix_join_kernel(const PrefixArgs a) {
    const int fours = a.d >> 2, heads_q = a.heads_k * (int)a.share.d;
    const int64_t e = (int64_t)blockIdx.x * kPrefixThreads + threadIdx.x, line = e / fours;
    if (line >= (int64_t)a.B * heads_q) return;
    const int ch = 4 * (int)(e - line * fours), b = (int)(line / heads_q), head = (int)(line - (int64_t)b * heads_q);
    const int hk = (int)a.share(head), row = b * (int)a.share.d + head - hk * (int)a.share.d;
    const int parts = prefix_keys(a).parts;
    const bool live = a.lens[b] >= 0;
    const float inf = __builtin_huge_valf();
    const int64_t slot = ((int64_t)(row / kPrefixRows) * a.heads_k + hk) * a.parts.d;
    const float* ml = a.part_ml + (slot * kPrefixRows + row % kPrefixRows) * 2;
    const float* acc = a.part_acc + (slot * kPrefixRows + row % kPrefixRows) * a.d + ch;
    const float own = live ? a.own_lse[line] * 1.44269504088896340736f : -inf;
    float top = own == -inf ? kFlashNone : own, sum = own == -inf ? 0.0f : 1.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (sum != 0.0f) o = *reinterpret_cast<const float4*>(a.own_out + line * a.d + ch);
    const float own_top = top;
    if (live) {
        for (int i = 0; i < parts; ++i) top = fmaxf(top, ml[(int64_t)i * kPrefixRows * 2]);
        const float f0 = __builtin_amdgcn_exp2f(own_top - top);
        if (!(f0 == 0.0f)) {
            sum *= f0;
            o.x *= f0;
            o.y *= f0;
            o.z *= f0;
            o.w *= f0;
        } else {
            sum = o.x = o.y = o.z = o.w = 0.0f;
        }
        for (int i = 0; i < parts; ++i) {
            const float2 part = *reinterpret_cast<const float2*>(ml + (int64_t)i * kPrefixRows * 2);
            const float4 v = *reinterpret_cast<const float4*>(acc + (int64_t)i * kPrefixRows * a.d);
            const float f = __builtin_amdgcn_exp2f(part.x - top);
            if (f == 0.0f && part.y == part.y) continue;   // a part whose keys the row does not see, or that weigh nothing
            sum = fmaf(f, part.y, sum);
            o.x = fmaf(f, v.x, o.x);
            o.y = fmaf(f, v.y, o.y);
            o.z = fmaf(f, v.z, o.z);
            o.w = fmaf(f, v.w, o.w);
        }
    }
    const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
    *reinterpret_cast<Piece8*>(a.out + b * a.ldo + head * a.ldoh + ch) = Piece8{pack_bf16_pair(o.x * f, o.y * f), pack_bf16_pair(o.z * f, o.w * f)};
    if (ch == 0 && a.lse) a.lse[line] = sum == 0.0f ? -inf : top * 0.69314718055994530942f + logf(sum);
}

}  // namespace resq
