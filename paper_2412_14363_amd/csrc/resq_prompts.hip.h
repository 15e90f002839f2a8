// Attention over whole prompts: causal, sequences packed one after the other, grouped heads, on top of cached tokens or not.
//   x_ij = scale * q_i . k_j, capped to cap * tanh(x / cap) where there is a cap
//   out_i = sum_j e^(x_ij - lse_i) v_j, lse_i = ln sum_j e^(x_ij)
// over the keys j of the sequence with own(i) - window < j <= own(i), own(i) = i + nk - nq a query's own place among its sequence's keys.
//
// A workgroup has 256 rows, 32 to each of eight wavefronts (resq_flash.hip.h); a row is a query and one of the heads that share a K/V head, so
// that a tile of keys and values in LDS serves all of them, and tiles on the diagonal are few (with four heads to a K/V head 256 rows are
// 64 queries).  Keys and values come straight to LDS in tiles of 64 (32 for heads above 128), two tiles ahead, three of each in LDS.  The
// wavefronts are two groups half a tile apart: while one has the matrix cores, which a tile's products keep busy for 1024 cycles of a
// wavefront, the other makes weights of its scores and asks for tiles (1000 cycles).  Heads of 64 and less take four wavefronts and
// three workgroups to a compute unit, which find each other's gaps by themselves.
//
// Weights are rounded to bf16 for the second product, which takes the values as they are: a result, rounded to bf16 itself, is then off by 1.7 10^-3 of
// its size where its own rounding alone leaves 1.5.  In two numbers the second product would be twice as long, at the matrix cores' turn, which
// bounds the kernel; in masked tiles alone short prompts gained that bit, 17 tokens in 9.9 us for 9.4, longer ones none (24 ragged ones 203 for 198).
//
// Tiles that all rows see whole come first, in a loop without masks; what the diagonal, the window and the ends leave follows.  Values
// that are infinite or NaN are left out of the masked tiles' products (0 times them is NaN) and given to the rows that see them, one by one,
// at the end.  Where there are fewer workgroups than compute units the keys are cut into parts, and a second kernel joins them.
//
// What bounds it: the matrix turn, 2020 cycles where its products are 1024, that is LDS, 48 reads of a wavefront in each turn; and on
// large calls the power limit (products of random numbers alone run at 1.6 GHz).  Measured on MI355X: 8192 tokens, 32 heads on 8 of 128
// 528-550 us, 1.0 PFLOP/s of the pairs that are seen, where a plain product of 8192 x 8192 x 8192 reaches 1.3; the matrix cores are busy
// 46 % of all cycles, LDS banks never in conflict.  2048 tokens 66 us: the last workgroup has all 32 tiles of keys, at 2 us each, when half of
// the compute units are idle; cut in two 91, for a workgroup's way to its first product is 7 us and results of parts take another pass.
// On the way, at 8192 tokens: tiles through registers and masks everywhere 1649 us; tiles straight to LDS, whole ones in a loop without
// masks, maxima that rise only when they must 585; the two groups 528-550.  24 ragged prompts of heads of 64 with window and cap 189-192
// us, three chunks of up to 300 tokens behind up to 30000 316, of which the join is 11 (28 with one part's loads at a time).  Heads of 192 238 for 4096
// tokens of 16 heads on 8, 430 TFLOP/s; of 256, for which registers do not suffice, 689, 200.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_flash.hip.h"

namespace resq {

constexpr int kPromptWaves = 8;   // of a workgroup at most
constexpr int kPromptMost = (1 << 25) - 1;   // tiles that a thread counts, of which a call has 2^24 + 65535 at most
constexpr __host__ __device__ int prompt_rows(int waves) { return kFlashRows * waves; }   // of a workgroup

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
    uint16_t* out;
    int64_t ldo, ldoh;
    float* lse;
    float* part_ml;      // [tile, head, part][rows][2]: maximum (times log2 e) and sum (workspace)
    float* part_acc;     // [tile, head, part][rows][d]: weighted sums (workspace)
};

// A workgroup's rows: tile `tile` of a sequence's.
struct PromptTile {
    int q0, nq, k0, nk;  // the sequence's first query and key, and how many there are
    int row0, rows;      // the first row of the tile among the sequence's (queries x share), and the sequence's rows
};

// The tile with the number `at` among all sequences' tiles, counted from the last one (later rows see more keys: the longest work
// comes first).  False where there are not so many.
template <int WAVES>
__device__ __forceinline__ bool prompt_tile(const PromptArgs& a, int at, PromptTile& tile) {
    constexpr int kPromptThreads = 64 * WAVES, kPromptRows = prompt_rows(WAVES);
    __shared__ uint32_t part[kPromptWaves];
    __shared__ int found[5];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    auto first = [&](const int32_t* cu, int b, int most) { return min(max(cu[b], 0), most); };
    auto tiles = [&](int b) {
        const int q0 = first(a.cu_q, b, a.tokens_q), q1 = first(a.cu_q, b + 1, a.tokens_q);
        return (int)(((int64_t)max(q1 - q0, 0) * a.share.d + kPromptRows - 1) / kPromptRows);
    };
    const int per = (a.B + kPromptThreads - 1) / kPromptThreads;
    const int b0 = min(t * per, a.B), b1 = min(b0 + per, a.B);
    // (lengths that decrease name rows again and again: their counts stop at what 32 bits hold, so that one thread still finds each tile)
    int mine = 0;
    for (int b = b0; b < b1; ++b) mine = min(mine + tiles(b), kPromptMost);
    const uint32_t upto = (uint32_t)wave_scan(mine);
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    uint32_t total = 0, before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w == wave) before = total;
        total = min(total + part[w], 64u * kPromptMost);
    }
    if ((uint32_t)at >= total) return false;
    const uint32_t mirror = total - 1 - (uint32_t)at;
    uint32_t start = before + upto - (uint32_t)mine;
    if (start <= mirror && mirror < start + (uint32_t)mine) {
        for (int b = b0; b < b1; ++b) {
            const uint32_t n = (uint32_t)tiles(b);
            if (mirror < start + n) {
                found[0] = first(a.cu_q, b, a.tokens_q);
                found[1] = first(a.cu_q, b + 1, a.tokens_q);
                found[2] = first(a.cu_k, b, a.tokens_k);
                found[3] = first(a.cu_k, b + 1, a.tokens_k);
                found[4] = (int)(mirror - start);
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
template <int WAVES, int KEYS>
__device__ __forceinline__ PromptKeys prompt_keys(const PromptArgs& a, const PromptTile& t) {
    PromptKeys k;
    const int last = min(t.row0 + prompt_rows(WAVES), t.rows) - 1, shift = t.nk - t.nq;
    const int own0 = (int)a.share(t.row0) + shift, own1 = (int)a.share(last) + shift;
    k.end = max(own1 + 1, 0);   // at most nk
    k.begin = min(max(own0 - (a.window - 1), 0), k.end) / KEYS * KEYS;
    const int tiles = (k.end - k.begin + KEYS - 1) / KEYS;
    const int parts = min((int)a.parts.d, max(tiles / a.least, 1));
    k.per = (tiles + parts - 1) / parts;
    k.parts = k.per ? (tiles + k.per - 1) / k.per : 1;
    return k;
}

// WAVES: 8, in two groups half a tile apart, or 4; OCC: wavefronts to a SIMD
template <int W, int KEYS, int WAVES, int OCC, bool CAP>
__global__ __launch_bounds__(64 * WAVES, OCC) void attend_prompts_kernel(const PromptArgs a) {
    using Tile = FlashTile<W>;
    constexpr bool kPair = WAVES == 8;
    constexpr int kTileBytes = KEYS * Tile::kPitch, kPromptRows = prompt_rows(WAVES);
    constexpr int kMoves = kTileBytes / 1024 / 4;   // of 1024 bytes of a tile that a wavefront fetches
    constexpr int kRowsAMove = 64 / Tile::kPieces;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // three tiles of keys, three of values

    const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6), group = kPair ? wave >> 2 : 0;
    // heads are neighbours in the grid: with 8 of them (or a multiple) each die has a head's keys and values in its own L2
    const int unit = (int)a.heads(blockIdx.x), hk = (int)blockIdx.x - unit * (int)a.heads.d;
    const int order = (int)a.parts(unit), piece = unit - order * (int)a.parts.d;
    PromptTile tile;
    if (!prompt_tile<WAVES>(a, order, tile)) return;
    const PromptKeys keys = prompt_keys<WAVES, KEYS>(a, tile);
    if (piece >= keys.parts) return;
    const int begin = keys.begin + piece * keys.per * KEYS, end = min(keys.end, begin + keys.per * KEYS);
    const int n_all = (end - begin + KEYS - 1) / KEYS;

    // ---- tiles straight to LDS, keys by the first group and values by the second: a wavefront's move is some whole rows, a lane's place
    // in it is given, so what is fetched there is the piece that belongs there ----
    const uint8_t* k_src = reinterpret_cast<const uint8_t*>(a.k + tile.k0 * a.ldk + hk * a.ldkh);
    const uint8_t* v_src = reinterpret_cast<const uint8_t*>(a.v + tile.k0 * a.ldv + hk * a.ldvh);
    const int my_row = (wave & 3) * (kMoves * kRowsAMove) + lane / Tile::kPieces;   // of the first move
    // tiles that all rows see whole come first, then the ones in front of them and behind
    const int shift = tile.nk - tile.nq;
    const int own0 = (int)a.share(tile.row0) + shift, own1 = (int)a.share(min(tile.row0 + kPromptRows, tile.rows) - 1) + shift;
    const int end_floor = end / KEYS * KEYS;   // (begin is a multiple of KEYS)
    const int whole0 = min(max((max(own1 - (a.window - 1), 0) + KEYS - 1) / KEYS * KEYS, begin), end_floor);
    const int whole1 = max(min((own0 + 1) / KEYS * KEYS, end_floor), whole0);
    const int n_whole = (whole1 - whole0) / KEYS, n_front = (whole0 - begin) / KEYS;
    auto key_of = [&](int n) {
        const int m = n - n_whole;
        return m < 0 ? whole0 + n * KEYS : m < n_front ? begin + m * KEYS : whole1 + (m - n_front) * KEYS;
    };
    auto fetch_one = [&](int n, bool vals) __attribute__((always_inline)) {
        const int key0 = key_of(n), last = end - 1 - key0;
        const int64_t ld2 = 2 * (vals ? a.ldv : a.ldk);
        const uint8_t* from = (vals ? v_src : k_src) + key0 * ld2;
        const uint32_t to = flash_lds(lds) + (3 * vals + n % 3) * kTileBytes + (wave & 3) * kMoves * 1024;
#pragma unroll
        for (int i = 0; i < kMoves; ++i) {
            const int row = my_row + i * kRowsAMove, place = vals ? Tile::value_at(row, lane % Tile::kPieces) : Tile::key_at(row, lane % Tile::kPieces);
            const int piece = min((place % Tile::kPitch) >> 4, (a.d >> 3) - 1);   // (channels behind the head's: any)
            flash_fetch(to + i * 1024, from, (uint32_t)min(row, last) * (uint32_t)ld2 + 16 * piece);   // (keys behind the last: any that is there)
        }
    };
    auto fetch = [&](int n) __attribute__((always_inline)) {
        if constexpr (kPair) {
            fetch_one(n, group != 0);
        } else {
            fetch_one(n, false);
            fetch_one(n, true);
        }
    };
    constexpr int kFetch = kPair ? kMoves : 2 * kMoves;   // of a wavefront for a tile
    if (n_all > 0) fetch(0);
    if (n_all > 1) fetch(1);

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
    const float inf = __builtin_huge_valf();
    const float factor = a.scale * 1.44269504088896340736f;
    const FlashCap<true> cap(CAP ? a.softcap : 1.0f, factor);

    // ---- Two groups of wavefronts, one of each to a SIMD, half a tile apart: while one is at the matrix cores the other is at the vector ALU. ----
    constexpr int kAhead = W <= 64 || W > 128 ? 0 : CAP ? 2 : KEYS / 16;   // (capped scores need the registers)
    FlashTurn<W, KEYS, kAhead> s;
    auto keys_in = [&](int n) { return lds + n % 3 * kTileBytes; };
    auto values_in = [&](int n) { return lds + (3 + n % 3) * kTileBytes; };
    flash_landed();
    if (kPair && group) flash_after_products();
    uint64_t odd = 0;   // tiles with values that are not finite, of those behind the whole ones (at most 512 / KEYS + 4)
    int n = 0;
    if (n_whole > 0) {
        auto softmax = [&]() __attribute__((always_inline)) {
            flash_after_products();
            if (n + 2 < n_all) fetch(n + 2);
            r.ask_ahead(s, values_in(n));
            r.template softmax<KEYS, CAP, false>(s, {factor}, cap);
            if (n + 2 < n_all) flash_after_softmax<kFetch>();
            else flash_after_softmax<0>();
            ++n;
        };
        r.template products<KEYS, false, false>(s, keys_in(0), nullptr);
        softmax();
        // (where the loop begins in a line of 64 bytes of the instruction cache costs up to 2 %: 8 bytes behind its start 528 us for 8192 tokens, at 0,
        // 16, 24, 32 or 56 538 to 541; 8 bytes are what these 14 instructions of 4 and what the compiler puts behind them come to)
        if constexpr (W == 128 && !CAP) asm volatile(".p2align 6\n\t.fill 14, 4, 0xBF800000");   // s_nop 0
        while (n < n_whole) {
            r.template products<KEYS, true, false>(s, keys_in(n), values_in(n + 2));
            softmax();
        }
        r.weigh_rest(s, values_in(n + 2));
    }
    for (; n < n_all; ++n) {
        r.template products<KEYS, false, false>(s, keys_in(n), nullptr);
        flash_after_products();
        if (n + 2 < n_all) fetch(n + 2);
        const int behind = own - key_of(n) - 4 * half;   // keys from the lane's first one to the row's own
        r.mask(s, [&](int key) { return (unsigned)(behind - key) < (unsigned)a.window; });
        r.template softmax<KEYS, CAP, true>(s, {factor}, cap);
        odd |= (uint64_t)r.template weigh_finite<KEYS>(s.p, values_in(n)) << (n - n_whole);
        if (n + 2 < n_all) flash_after_softmax<kFetch>();
        else flash_after_softmax<0>();
    }
    if (kPair && !group) flash_after_products();   // as many barriers as the other group

    // ---- what infinities and NaN among the values make of the rows that see them, one after the other ----
    for (; odd != 0; odd &= odd - 1) {
        const int key0 = key_of(n_whole + __builtin_ctzll(odd));
#pragma unroll 1
        for (int key = key0; key < min(key0 + KEYS, end); ++key) {
            const uint16_t *k = a.k + (tile.k0 + key) * a.ldk + hk * a.ldkh, *v = a.v + (tile.k0 + key) * a.ldv + hk * a.ldvh;
            float x = 0.0f;
            int d = a.d;   // (compared where it is needed, not in front of everything)
            asm volatile("" : "+s"(d));
#pragma unroll
            for (int s = 0; s < Tile::kSteps; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int ch = 16 * s + 8 * half + e;
                    const float of_q = bf16_bits_to_f32(r.q[s][e >> 1] >> (16 * (e & 1)) & 0xFFFFu);
                    if (ch < d) x = fmaf(of_q, bf16_bits_to_f32(k[ch]), x);
                }
            x = halves_sum(x);
            x = CAP ? cap(x) : x * factor;
            if ((unsigned)(own - key) >= (unsigned)a.window) continue;
            const float w = __builtin_amdgcn_exp2f(x - r.m);
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int ch = 32 * c + 8 * (i >> 2) + 4 * half + (i & 3);
                    if (ch < d) {
                        const float o = r.odd_value(v[ch]);
                        r.acc[c][i] = o == 0.0f ? r.acc[c][i] : fmaf(w, o, r.acc[c][i]);
                    }
                }
        }
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
template <int KEYS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void attend_prompts_join_kernel(const PromptArgs a) {
    constexpr int kPromptThreads = 64 * WAVES, kPromptRows = prompt_rows(WAVES);
    const int order = (int)a.heads(blockIdx.x), hk = (int)blockIdx.x - order * (int)a.heads.d;
    PromptTile tile;
    if (!prompt_tile<WAVES>(a, order, tile)) return;
    const PromptKeys keys = prompt_keys<WAVES, KEYS>(a, tile);
    if (keys.parts == 1) return;
    const int fours = a.d >> 2, rows = min(kPromptRows, tile.rows - tile.row0);
    const int64_t slot = ((int64_t)order * a.heads.d + hk) * a.parts.d;
    for (int e = threadIdx.x + blockIdx.y * kPromptThreads; e < rows * fours; e += kPromptThreads * gridDim.y) {
        const int row = e / fours, ch = 4 * (e - row * fours);
        const float* ml = a.part_ml + (slot * kPromptRows + row) * 2;
        const float* acc = a.part_acc + (slot * kPromptRows + row) * a.d + ch;
        float top = kFlashNone, sum = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        // four parts' loads at a time, none behind a branch
        auto part_of = [&](int i) { return (int64_t)min(i, keys.parts - 1) * kPromptRows; };
        for (int i = 0; i < keys.parts; i += 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) top = fmaxf(top, ml[part_of(i + k) * 2]);
        }
        for (int i = 0; i < keys.parts; i += 4) {
            float2 part[4];
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                part[k] = *reinterpret_cast<const float2*>(ml + part_of(i + k) * 2);
                v[k] = *reinterpret_cast<const float4*>(acc + part_of(i + k) * a.d);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // (a part whose keys the row does not see has sums of 0; one whose keys weigh nothing may have NaN, which stays)
                const float f = __builtin_amdgcn_exp2f(part[k].x - top);
                const bool none = i + k >= keys.parts;
                sum = none ? sum : fmaf(f, part[k].y, sum);
                o.x = none ? o.x : fmaf(f, v[k].x, o.x);
                o.y = none ? o.y : fmaf(f, v[k].y, o.y);
                o.z = none ? o.z : fmaf(f, v[k].z, o.z);
                o.w = none ? o.w : fmaf(f, v[k].w, o.w);
            }
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
