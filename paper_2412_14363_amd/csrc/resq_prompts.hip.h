// Attention over whole prompts: causal, sequences packed one after the other, grouped heads, on top of cached tokens or not.
//   x_ij = scale * q_i . k_j, capped to cap * tanh(x / cap) where there is a cap
//   out_i = sum_j e^(x_ij - lse_i) v_j, lse_i = ln sum_j e^(x_ij)
// over the keys j of the sequence with own(i) - window < j <= own(i), own(i) = i + nk - nq a query's own place among its sequence's keys.
//
// A workgroup has 128 rows, 32 to a wavefront (resq_flash.hip.h); a row is a query and one of the heads that share a K/V head, so that
// a tile of keys and values in LDS serves all of them, and tiles on the diagonal are few (with four heads to a K/V head 128 rows are
// 32 queries).  Keys and values come to LDS in tiles of 64, a tile ahead.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_flash.hip.h"

namespace resq {

constexpr int kPromptThreads = 256;
constexpr int kPromptWaves = kPromptThreads / 64;
constexpr int kPromptRows = kFlashRows * kPromptWaves;   // of a workgroup

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t ldq, ldqh, ldk, ldkh, ldv, ldvh;
    const int32_t *cu_q, *cu_k;
    int B, tokens_q, tokens_k, heads_k, d;
    FastDiv share;       // query heads to a K/V head
    FastDiv heads, parts;
    float scale, softcap;
    int window;          // 2^30: none
    int least;           // tiles of keys of a part at least
    int fold, units;     // from unit `fold` on the order is turned round, see the launch
    uint16_t* out;
    int64_t ldo, ldoh;
    float* lse;
    float* part_ml;      // [tile, head, part][128][2]: maximum (times log2 e) and sum (workspace)
    float* part_acc;     // [tile, head, part][128][d]: weighted sums (workspace)
};

// A workgroup's rows: tile `tile` of a sequence's.
struct PromptTile {
    int q0, nq, k0, nk;  // the sequence's first query and key, and how many there are
    int row0, rows;      // the first row of the tile among the sequence's (queries x share), and the sequence's rows
};

// The tile with the number `at` among all sequences' tiles, counted from the last one (later rows see more keys: the longest work
// comes first).  False where there are not so many.
__device__ __forceinline__ bool prompt_tile(const PromptArgs& a, int at, PromptTile& tile) {
    __shared__ int part[kPromptWaves], found[5];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    auto first = [&](const int32_t* cu, int b, int most) { return min(max(cu[b], 0), most); };
    auto tiles = [&](int b) {
        const int q0 = first(a.cu_q, b, a.tokens_q), q1 = first(a.cu_q, b + 1, a.tokens_q);
        return (int)(((int64_t)max(q1 - q0, 0) * a.share.d + kPromptRows - 1) / kPromptRows);
    };
    const int per = (a.B + kPromptThreads - 1) / kPromptThreads;
    const int b0 = min(t * per, a.B), b1 = min(b0 + per, a.B);
    int mine = 0;
    for (int b = b0; b < b1; ++b) mine += tiles(b);
    const int upto = wave_scan(mine);
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    int total = 0, before = 0;
#pragma unroll
    for (int w = 0; w < kPromptWaves; ++w) {
        if (w == wave) before = total;
        total += part[w];
    }
    if (at >= total) return false;
    at = total - 1 - at;
    int start = before + upto - mine;
    if (start <= at && at < start + mine) {
        for (int b = b0; b < b1; ++b) {
            const int n = tiles(b);
            if (at < start + n) {
                found[0] = first(a.cu_q, b, a.tokens_q);
                found[1] = first(a.cu_q, b + 1, a.tokens_q);
                found[2] = first(a.cu_k, b, a.tokens_k);
                found[3] = first(a.cu_k, b + 1, a.tokens_k);
                found[4] = at - start;
                break;
            }
            start += n;
        }
    }
    __syncthreads();
    tile.q0 = __builtin_amdgcn_readfirstlane(found[0]);
    tile.nq = __builtin_amdgcn_readfirstlane(found[1]) - tile.q0;
    tile.k0 = __builtin_amdgcn_readfirstlane(found[2]);
    tile.nk = max(__builtin_amdgcn_readfirstlane(found[3]) - tile.k0, 0);
    tile.row0 = __builtin_amdgcn_readfirstlane(found[4]) * kPromptRows;
    tile.rows = tile.nq * (int)a.share.d;
    return true;
}

// Keys that a tile's rows see, [begin, end) with begin a multiple of a tile of keys, cut into parts of so many tiles.
struct PromptKeys {
    int begin, end, per, parts;
};
template <int KEYS>
__device__ __forceinline__ PromptKeys prompt_keys(const PromptArgs& a, const PromptTile& t) {
    PromptKeys k;
    const int last = min(t.row0 + kPromptRows, t.rows) - 1, shift = t.nk - t.nq;
    const int own0 = (int)a.share(t.row0) + shift, own1 = (int)a.share(last) + shift;
    k.end = max(own1 + 1, 0);   // at most nk
    k.begin = min(max(own0 - (a.window - 1), 0), k.end) / KEYS * KEYS;
    const int tiles = (k.end - k.begin + KEYS - 1) / KEYS;
    const int parts = min((int)a.parts.d, max(tiles / a.least, 1));
    k.per = (tiles + parts - 1) / parts;
    k.parts = k.per ? (tiles + k.per - 1) / k.per : 1;
    return k;
}

template <int W, int KEYS, int OCC, bool CAP>
__global__ __launch_bounds__(kPromptThreads, OCC) void attend_prompts_kernel(const PromptArgs a) {
    using Tile = FlashTile<W>;
    constexpr int kTileBytes = KEYS * Tile::kPitch;
    constexpr int kMoves = kTileBytes / 1024 / kPromptWaves;   // of 1024 bytes of a tile's keys (values) that a wavefront fetches
    constexpr int kRowsAMove = 64 / Tile::kPieces;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // two tiles of keys, two of values

    const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    // heads are neighbours in the grid: with 8 of them (or a multiple) each die has a head's keys and values in its own L2
    int unit = (int)a.heads(blockIdx.x);
    const int hk = (int)blockIdx.x - unit * (int)a.heads.d;
    if (unit >= a.fold) unit = a.fold + a.units - 1 - unit;
    const int order = (int)a.parts(unit), piece = unit - order * (int)a.parts.d;
    PromptTile tile;
    if (!prompt_tile(a, order, tile)) return;
    const PromptKeys keys = prompt_keys<KEYS>(a, tile);
    if (piece >= keys.parts) return;
    const int begin = keys.begin + piece * keys.per * KEYS, end = min(keys.end, begin + keys.per * KEYS);

    // ---- tiles of keys and values, straight to LDS: a wavefront's move is some whole rows, a lane's place in it is given, so what is
    // fetched there is the piece that belongs there ----
    const uint8_t* k_src = reinterpret_cast<const uint8_t*>(a.k + tile.k0 * a.ldk + hk * a.ldkh);
    const uint8_t* v_src = reinterpret_cast<const uint8_t*>(a.v + tile.k0 * a.ldv + hk * a.ldvh);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int my_row = wave * (kMoves * kRowsAMove) + lane / Tile::kPieces;   // of the first move
    auto fetch = [&](int key0, int buffer) {
        const uint8_t *k = k_src + key0 * (2 * a.ldk), *v = v_src + key0 * (2 * a.ldv);
#pragma unroll
        for (int i = 0; i < kMoves; ++i) {
            const int row = my_row + i * kRowsAMove;
            const int pk = min((Tile::key_at(row, lane % Tile::kPieces) - row * Tile::kPitch) >> 4, (a.d >> 3) - 1);   // (channels behind
            const int pv = min((Tile::value_at(row, lane % Tile::kPieces) - row * Tile::kPitch) >> 4, (a.d >> 3) - 1);   // the head's: any)
            const uint32_t from = (uint32_t)min(row, end - 1 - key0);   // (keys behind the last: any that is there)
            const uint32_t to = lds0 + buffer * kTileBytes + (wave * kMoves + i) * 1024;
            flash_fetch(to, k, from * (uint32_t)(2 * a.ldk) + 16 * pk);
            flash_fetch(to + 2 * kTileBytes, v, from * (uint32_t)(2 * a.ldv) + 16 * pv);
        }
    };

    // ---- which tiles all rows see whole: those come first, then the ones in front of them and behind ----
    const int last_row = min(tile.row0 + kPromptRows, tile.rows) - 1, shift = tile.nk - tile.nq;
    const int own0 = (int)a.share(tile.row0) + shift, own1 = (int)a.share(last_row) + shift;
    const int end_floor = end / KEYS * KEYS;   // (begin is a multiple of KEYS)
    const int whole0 = min(max((max(own1 - (a.window - 1), 0) + KEYS - 1) / KEYS * KEYS, begin), end_floor);
    const int whole1 = max(min((own0 + 1) / KEYS * KEYS, end_floor), whole0);
    const int n_whole = (whole1 - whole0) / KEYS, n_front = (whole0 - begin) / KEYS;
    const int n_all = (end - begin + KEYS - 1) / KEYS;
    auto key_of = [&](int n) {
        const int m = n - n_whole;
        return m < 0 ? whole0 + n * KEYS : m < n_front ? begin + m * KEYS : whole1 + (m - n_front) * KEYS;
    };
    if (n_all > 0) fetch(key_of(0), 0);

    // ---- the own row ----
    const int row = tile.row0 + wave * kFlashRows + (lane & 31);
    const bool live = row < tile.rows;
    const int token = (int)a.share(live ? row : 0), head = hk * (int)a.share.d + (live ? row : 0) - token * (int)a.share.d;
    const int own = live ? token + shift : -1;   // a row that is not there sees nothing
    FlashRow<W, false> r;
    {
        const uint16_t* src = a.q + (tile.q0 + token) * a.ldq + head * a.ldqh;
#pragma unroll
        for (int s = 0; s < Tile::kSteps; ++s) {
            const int ch = 16 * s + 8 * half;
            Piece16 p{0u, 0u, 0u, 0u};
            if (live && ch < a.d) p = *reinterpret_cast<const Piece16*>(src + ch);
            r.q[s] = (v4u_flash){p.x, p.y, p.z, p.w};
        }
    }
    r.clear();
    const float inv_cap = CAP ? 1.0f / a.softcap : 0.0f;
    const float inf = __builtin_huge_valf();
    float f[KEYS / 16];
    f[0] = CAP ? a.scale : a.scale * 1.44269504088896340736f;

    flash_landed();
    int n = 0, buffer = 0;
    for (; n < n_whole; ++n, buffer ^= 1) {
        if (n + 1 < n_all) fetch(key_of(n + 1), buffer ^ 1);
        r.template step<KEYS, CAP, true, false>(lds + buffer * kTileBytes, lds + (2 + buffer) * kTileBytes, f, nullptr, a.softcap, inv_cap,
                                                [](int, int) { return true; });
        flash_landed();
    }
    for (; n < n_all; ++n, buffer ^= 1) {
        const int key0 = key_of(n);
        if (n + 1 < n_all) fetch(key_of(n + 1), buffer ^ 1);
        const int behind = own - key0 - 4 * half;   // keys from the lane's first one to the row's own
        // (a wavefront whose rows see nothing of the tile goes on to the next)
        if (__builtin_amdgcn_ballot_w64(own >= key0 && own - key0 < a.window + KEYS - 1) != 0)
            r.template step<KEYS, CAP, true, true>(lds + buffer * kTileBytes, lds + (2 + buffer) * kTileBytes, f, nullptr, a.softcap, inv_cap,
                                                   [&](int kb, int i) {
                                                       const int c = 32 * kb + 8 * (i >> 2) + (i & 3);
                                                       return behind >= c && behind - c < a.window;
                                                   });
        flash_landed();
    }

    // ---- the result, or this part of it ----
    const float sum = halves_sum(r.l);
    if (!live) return;
    if (keys.parts == 1) {
        const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
        uint16_t* dst = a.out + (tile.q0 + token) * a.ldo + head * a.ldoh;
#pragma unroll
        for (int c = 0; c < Tile::kBlocks; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int ch = 32 * c + 8 * (i >> 2) + 4 * half;
                if (ch < a.d)
                    *reinterpret_cast<Piece8*>(dst + ch) = Piece8{pack_bf16_pair(r.acc[c][i] * f, r.acc[c][i + 1] * f),
                                                                  pack_bf16_pair(r.acc[c][i + 2] * f, r.acc[c][i + 3] * f)};
            }
        if (a.lse && half == 0)
            a.lse[(int64_t)(tile.q0 + token) * (a.heads.d * a.share.d) + head] = sum == 0.0f ? -inf : r.m * 0.69314718055994530942f + logf(sum);
        return;
    }
    const int64_t slot = ((int64_t)order * a.heads.d + hk) * a.parts.d + piece;
    const int at = wave * kFlashRows + (lane & 31);
    float* dst = a.part_acc + (slot * kPromptRows + at) * a.d;
#pragma unroll
    for (int c = 0; c < Tile::kBlocks; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int ch = 32 * c + 8 * (i >> 2) + 4 * half;
            if (ch < a.d) *reinterpret_cast<float4*>(dst + ch) = make_float4(r.acc[c][i], r.acc[c][i + 1], r.acc[c][i + 2], r.acc[c][i + 3]);
        }
    if (half == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * kPromptRows + at) * 2) = make_float2(r.m, sum);
}

// Joins the parts of tiles that have several: m = max m_i, f_i = 2^(m_i - m), out = sum f_i acc_i / sum f_i l_i, lse = m ln 2 + ln sum f_i l_i
template <int KEYS>
__global__ __launch_bounds__(kPromptThreads) void attend_prompts_join_kernel(const PromptArgs a) {
    const int order = (int)a.heads(blockIdx.x), hk = (int)blockIdx.x - order * (int)a.heads.d;
    PromptTile tile;
    if (!prompt_tile(a, order, tile)) return;
    const PromptKeys keys = prompt_keys<KEYS>(a, tile);
    if (keys.parts == 1) return;
    const int fours = a.d >> 2, rows = min(kPromptRows, tile.rows - tile.row0);
    const int64_t slot = ((int64_t)order * a.heads.d + hk) * a.parts.d;
    for (int e = threadIdx.x + blockIdx.y * kPromptThreads; e < rows * fours; e += kPromptThreads * gridDim.y) {
        const int row = e / fours, ch = 4 * (e - row * fours);
        const float* ml = a.part_ml + (slot * kPromptRows + row) * 2;
        const float* acc = a.part_acc + (slot * kPromptRows + row) * a.d + ch;
        float top = kFlashNone, sum = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int i = 0; i < keys.parts; ++i) top = fmaxf(top, ml[(int64_t)i * kPromptRows * 2]);
        for (int i = 0; i < keys.parts; ++i) {
            const float2 part = *reinterpret_cast<const float2*>(ml + (int64_t)i * kPromptRows * 2);
            const float4 v = *reinterpret_cast<const float4*>(acc + (int64_t)i * kPromptRows * a.d);
            const float f = __builtin_amdgcn_exp2f(part.x - top);
            if (f == 0.0f && part.y == part.y) continue;   // a part whose keys the row does not see, or that weigh nothing
            sum = fmaf(f, part.y, sum);
            o.x = fmaf(f, v.x, o.x);
            o.y = fmaf(f, v.y, o.y);
            o.z = fmaf(f, v.z, o.z);
            o.w = fmaf(f, v.w, o.w);
        }
        const int r = tile.row0 + row, token = (int)a.share(r), head = hk * (int)a.share.d + r - token * (int)a.share.d;
        const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<Piece8*>(a.out + (tile.q0 + token) * a.ldo + head * a.ldoh + ch) =
            Piece8{pack_bf16_pair(o.x * f, o.y * f), pack_bf16_pair(o.z * f, o.w * f)};
        if (ch == 0 && a.lse)
            a.lse[(int64_t)(tile.q0 + token) * (a.heads.d * a.share.d) + head] =
                sum == 0.0f ? -__builtin_huge_valf() : top * 0.69314718055994530942f + logf(sum);
    }
}

}  // namespace resq
