// Attention of one new token of each sequence over the paged cache of compact K/V rows (resq_kv_row.hip.h, resq_kv.hip.h).
//   x_t = scale * q . k_t, k_t = code * s + z (not rounded), capped to cap * tanh(x_t / cap) where there is a cap
//   out = sum_t exp(x_t - m) v_t / sum_t exp(x_t - m), lse = m + log(sum)
// over the tokens t < len of the sequence (the last `window` of them where there is a window) whose page exists.
//
// One pass with the running maximum and sum of the softmax, products on the bf16 matrix cores (16x16x32), codes as operands:
// a code has at most 8 significant bits, so that bf16 holds it exactly, and scales and zero-points, which are a token's, stay
// out of the sums:
//   q . k_t = s_h (q_h . c_h) + z_h sum(q_h) + s_l (q_l . c_l) + z_l sum(q_l)
//   sum_t p_t v_t = sum_t (p_t s_t) c_t + sum_t p_t z_t, for each group of channels
// A wavefront takes 32 tokens of one K/V head at a time:
//   S (queries x tokens) = Q x K codes^T: with up to 8 queries (Q = 8) both halves of the 16 rows hold them, the upper for the
//   first 16 tokens and the lower for the others, so that a lane ends with one token and four queries, and the softmax works
//   on no empty lane where queries are 8; with up to 16 (Q = 16) a lane has two tokens
//   O (channels x queries) += V codes^T x P: the weights P go through LDS to where this product wants them, as two bf16
//   numbers each, the nearest one and the one nearest to what it leaves: with up to 8 queries in the two halves of the columns,
//   else in two products.  What both leave, at most 2^-17 of the weight, meets the middle of its operands (135.5, 127.5) in fp32 beside the
//   zero-points, so that an output is off by at most 2^-17 of half its values' range: 256 x 512 tokens 55.9 us, with two truncations
//   and nothing made of the rest 54.9 (a hundred times the error), with a third bf16 number, and a product more, 56.8 (no error)
// A 4-bit code becomes a bf16 number by being put under the leading bits of 16 (keys) or 128 (values): one shift and one
// and-or for two codes.  The constants leave again with the zero-points, once per token; for values every second token has
// the code's complement and the opposite sign, c + 128 and c - 143, so that the sums stay small.
// The maximum is looked at again only when a score is 2^8 times what it allows: sums of weights up to 2^8 lose nothing.
//
// The work is cut into units of 128 tokens of one head (four wavefronts, 32 tokens each); all units of the call in a row are
// dealt to the workgroups in runs of equal cost, whatever the sequences' lengths are (they are read on the GPU).  A head
// that ends up with several workgroups is joined by a second kernel from their maxima, sums and partial outputs.  (Joined by the
// workgroup that is done last, a sequence of 131072 tokens took half as long again: 64 parts read by one workgroup.)
//
// Times here and at the dispatch are of whole calls, both kernels, in a captured graph over three sets of inputs in turn (those of
// more than some 90 MB come from HBM), medians; "N x T" is N sequences of T tokens, 8 K/V heads of 128 with 32 queries, r = 16 and pages
// of 16 rows unless it says otherwise.
// Bound where runs are long: HBM, 2 row bytes per token and K/V head, with the vector ALU (400 instructions a tile) close behind.  This
// kernel alone, by a trace: 48 ragged sequences up to 8192 tokens 57 us, 4.6 TB/s, one of 131072 with 64 queries 41 us, 4.5 TB/s (a plain read
// of as much 6.3).  Short runs: the way to the first tile (lengths, then pages, then rows, each a read of its own) and out again, about
// 5 us of the 8.1 that one sequence of 777 tokens takes.  Few queries to a K/V head: the vector ALU, because a lane does the softmax
// of four queries whether they are there or not (24 sequences, heads of 64 with one query each, window 1500: 566 instructions a
// tile, some 10 us of 19.4).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_kv_row.hip.h"
#include "resq_lanes.hip.h"
#include "resq_layout.h"

namespace resq {

constexpr int kAttendThreads = 256;
constexpr int kAttendWaves = kAttendThreads / 64;
constexpr int kAttendMaxHead = 256;
constexpr int kAttendTile = 32;                              // tokens of a wavefront's step
constexpr int kAttendUnit = kAttendTile * kAttendWaves;      // tokens of a unit
// what it costs to begin and to end a head, in units: 48 ragged sequences 80.1 us at 0, 63.8 at 2, 62.3 at 3, 62.1 at 4; behind a
// window of 1500 24.1, 25.2, 22.8, 25.6; equal lengths lose by it: 32 x 4096 45.0 at 0, 46.9 at 3, 256 x 512 55.8 and 56.5
constexpr int kAttendHeadCost = 3;
constexpr int kAttendMaxGrid = 3 * 256;                      // workgroups: three to a compute unit at most
constexpr int kAttendRows = 16;                              // queries of a workgroup at most
constexpr int kAttendJoinFew = 8;                            // partial results that a thread reads at once
constexpr int kAttendJoinSplit = 1024;                       // heads from which a workgroup joins all of a head's queries, see there
constexpr int kAttendPRow = 80;                              // bytes of a row of weights in LDS: 32 in bf16, and what keeps rows on other banks
constexpr float kAttendNone = -3.0e38f;                      // the maximum of no scores: finite, so that differences stay numbers
constexpr float kAttendSlack = 8.0f;                         // of the running maximum, in powers of two
constexpr int kAttendLdsPad = 512;                           // reads of whole pieces go this far behind the last row at most

typedef float v4f_att __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_att __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf_att __attribute__((ext_vector_type(8)));

struct AttendArgs {
    const uint16_t* q;
    int64_t ldq, ldqh;
    int B, heads_k, share, qtiles, d, r, row_bytes;
    const int32_t* lens;
    const int32_t* table;
    int64_t ld_table;
    const uint8_t* pages[2];
    int num_pages;
    FastDiv page_size;
    int64_t page_stride, head_stride, row_stride;
    int max_len;      // tokens that a table row can name
    int window;       // 0: none
    float scale, softcap;
    uint16_t* out;
    int64_t ldo, ldoh;
    float* lse;
    int32_t* joins;    // [B][heads][2]: a head's first partial result, and the workgroup that has its last one (workspace)
    float* part_ml;    // [2 grid][16][2]: maximum (times log2 e) and sum of a partial result's queries (workspace)
    float* part_acc;   // [2 grid][rows][d]: and its weighted sums (workspace)
    int rows;          // queries of a partial result
    int blocks16;      // page_size is a multiple of 16, and 16 rows' offsets fit 32 bits
    int fours_magic;   // e * fours_magic >> 16 is e / (d / 4) for e < 1024
    int lds_red;       // bytes in front of the maxima and sums in LDS
};

// first token of a sequence that is seen, and units from the tile it is in
__device__ __forceinline__ int attend_first(const AttendArgs& a, int len) {
    return a.window && len > a.window ? len - a.window : 0;
}
__device__ __forceinline__ int attend_len(const AttendArgs& a, int b) { return min(max(a.lens[b], 0), a.max_len); }
__device__ __forceinline__ int attend_units(const AttendArgs& a, int len) {
    const int from = attend_first(a, len) & ~(kAttendTile - 1);
    return (len - from + kAttendUnit - 1) / kAttendUnit;
}
// what a head of so many units costs, counted in units
__device__ __forceinline__ int attend_cost(int units) { return units == 0 ? 0 : units + kAttendHeadCost; }

__device__ __forceinline__ v4f_att attend_mfma(const v4u_att& x, const v4u_att& y, const v4f_att& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf_att, x), __builtin_bit_cast(v8bf_att, y), c, 0, 0, 0);
}
// upper halves of two fp32 numbers: their truncations to bf16
__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// Constants of (x & mask) | bits, which is one instruction if one of the two comes from a scalar register and the other from a
// vector register: left to itself the compiler writes both into two instructions.
struct CodeBits {
    uint32_t mask, bits;
    __device__ __forceinline__ CodeBits(uint32_t m, uint32_t b) : mask(m), bits(b) { asm volatile("" : "+s"(mask), "+v"(bits)); }
    __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return (x & mask) | bits; }
};
// sum over the four lanes l % 16 + 16 k: swaps of rows of 16 lanes and of halves
__device__ __forceinline__ float rows_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// cap * tanh(x / cap): by the exponential, or near 0, where that would cancel, by the series (its sixth term is below 2^-24)
__device__ __forceinline__ float soft_cap(float x, float cap, float inv_cap) {
    const float y = x * inv_cap, y2 = y * y;
    const float big = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * 2.88539008177792681472f) + 1.0f);
    const float small = y * fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
    return cap * (y2 < 0.0625f ? small : big);
}

// 16 bytes of a row in pages, at any even address
__device__ __forceinline__ uint4 piece_at(const uint8_t* p) {
    const Piece16 o = *reinterpret_cast<const Piece16*>(p);
    return make_uint4(o.x, o.y, o.z, o.w);
}

// A row comes to LDS in pieces of 16 bytes: its codes (the last of their pieces may hold a part of what follows them, or be
// there in vain: codes of some kind, which meet zeros or are not written out), and the 16 bytes of its scales and zero-points.
// The pitch of rows in LDS is a constant, so that every address is a lane's base and a constant, with the constants last, and
// 16 more than a multiple of 32, so that 16 rows, and rows 4 apart, spread over all banks (32 x 4096: 47 us,
// the same at 96 bytes in place of 112, 64.5 at 128).
__host__ __device__ constexpr int attend_pieces(int NL, int HT) { return HT * 16 + NL * 8 < 256 ? (HT * 16 + NL * 8) / 16 + 1 : 17; }
__host__ __device__ constexpr int attend_pitch(int NL, int HT) { return (attend_pieces(NL, HT) | 1) * 16; }
__host__ __device__ constexpr int attend_tiles_bytes(int NL, int HT) {
    return kAttendWaves * 2 * kAttendTile * attend_pitch(NL, HT) + kAttendLdsPad;
}
__host__ __device__ constexpr int attend_weights_bytes(int Q) { return 2 * 2 * Q * kAttendPRow; }   // of a wavefront
__device__ __forceinline__ int64_t lane_of64(int64_t x, int lane) {
    return ((int64_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
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
// NL: 4-bit channels of a lane in the second product (16 NL channels in all), HT: 16-channel tiles of the 8-bit group,
// Q: queries that fit, 8 or 16, BLOCKS: pages of a multiple of 16 rows, so that 16 tokens in a row from a multiple of 16 on are one
// page's and two scalar offsets serve a tile instead of one per row (32 x 4096 without an 8-bit group 44.9
// us against 46.9, 256 channels in 8 bits 132 against 175, 256 x 512 56.5 against 58.9), OCC: workgroups to a compute unit
template <int NL, int HT, int Q, bool BLOCKS, int OCC>
__global__ __launch_bounds__(kAttendThreads, OCC) void attend_kv_cache_kernel(const AttendArgs a) {
    constexpr int LS = NL / 2, HS = (HT + 1) / 2;   // steps of 32 channels of the first product
    constexpr int P = attend_pitch(NL, HT);
    constexpr int NT = Q / 8;                       // tokens of a lane in the softmax
    constexpr int PL = attend_pieces(NL, HT);
    constexpr int KU = (kAttendTile * PL + 63) / 64;     // pieces of a tile's keys (values) that a lane moves
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ int part[kAttendWaves], found[3];

    const int t = threadIdx.x, lane = t & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int heads = a.heads_k * a.qtiles;   // heads' query tiles of a sequence

    // ---- the run of units that is this workgroup's ----
    const int per = (a.B + kAttendThreads - 1) / kAttendThreads;   // sequences of a thread, in a row
    const int b0 = min(t * per, a.B), b1 = min(b0 + per, a.B);
    int mine = 0, len_b = 0;
    for (int b = b0; b < b1; ++b) {
        len_b = attend_len(a, b);
        mine += attend_cost(attend_units(a, len_b)) * heads;
    }
    int upto = wave_scan(mine);
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    int total = 0, before = 0;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) {
        if (w == wave) before = total;
        total += part[w];
    }
    total = __builtin_amdgcn_readfirstlane(total);
    // Workgroups go to the eight dies in turn; runs that follow one another, whose heads lie side by side in token-major pages (and
    // whose queries share a K/V head's rows where they are more than 16), stay on one die and meet in its L2 (32 x 4096 in
    // token-major pages 57.0 us, dealt in turn 75.6).
    const int W = min(total, (int)gridDim.x), per_die = (W + 7) >> 3;
    const int w0 = (blockIdx.x & 7) * per_die + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per_die || w0 >= W) return;
    const int share = total / W, rest = total - share * W;   // the first `rest` runs are a unit longer
    int u = w0 * share + min(w0, rest);
    const int u_end = u + share + (w0 < rest);
    int start = before + upto - mine;   // of this thread's first sequence
    if (start <= u && u < start + mine) {
        for (int b = b0; b < b1; ++b) {
            if (per > 1) len_b = attend_len(a, b);
            const int cost = attend_cost(attend_units(a, len_b)) * heads;
            if (u < start + cost) {
                found[0] = b;
                found[1] = start;
                found[2] = len_b;
                break;
            }
            start += cost;
        }
    }
    __syncthreads();
    int b = __builtin_amdgcn_readfirstlane(found[0]), seq_start = __builtin_amdgcn_readfirstlane(found[1]);
    int len = __builtin_amdgcn_readfirstlane(found[2]);

    const int RB = a.row_bytes, low = a.d - a.r;
    uint8_t* kt = lds + wave * (2 * kAttendTile * P);
    uint8_t* vt = kt + kAttendTile * P;
    uint8_t* pt = lds + attend_tiles_bytes(NL, HT) + wave * attend_weights_bytes(Q);   // weights: 8-bit group's, 4-bit group's
    const float inv_cap = a.softcap > 0.0f ? 1.0f / a.softcap : 0.0f;
    const float kLog2e = 1.44269504088896340736f;
    const float sc2 = a.softcap > 0.0f ? kLog2e : a.scale * kLog2e;
    const float inf = __builtin_huge_valf();

    const CodeBits key_bits(0x00780078u, 0x41804180u), value_bits(0x000F000Fu, 0xC3004300u);

    bool first_head = true;
    while (u < u_end) {
        // ---- the next head in the run ----
        const int units = attend_units(a, len), cost = attend_cost(units);
        if (u >= seq_start + cost * heads) {
            seq_start += cost * heads;
            // the next sequence that has tokens, looked for 64 at a time: a padded batch may have many without in a row (200 tokens
            // and 120000 with 998 empty sequences between them 26 us, with 65533 344; one after the other 156 and 9060)
            uint64_t some = 0;
            for (++b; b < a.B; b += 64) {
                len_b = b + lane < a.B ? attend_len(a, b + lane) : 0;
                some = __builtin_amdgcn_ballot_w64(len_b > 0);
                if (some) break;
            }
            if (!some) break;   // (there is one as long as nobody writes the lengths meanwhile)
            const int skip = __builtin_ctzll(some);
            b += skip;
            len = __builtin_amdgcn_readlane(len_b, skip);
            continue;
        }
        const int head = (u - seq_start) / cost, begin = (u - seq_start) - head * cost;
        const int end = min(cost, begin + (u_end - u));
        u += end - begin;
        const int first_unit = max(begin - kAttendHeadCost, 0), n_units = end - kAttendHeadCost - first_unit;
        if (n_units <= 0) continue;   // this run ends where the head begins
        const int hk = head / a.qtiles, qt = head - hk * a.qtiles;
        const int t_low = attend_first(a, len), from = t_low & ~(kAttendTile - 1);
        const int t_begin = from + first_unit * kAttendUnit;
        const int t_end = min(len, t_begin + n_units * kAttendUnit);
        const int64_t head_off = hk * a.head_stride;
        const int32_t* table = a.table + b * a.ld_table;

        // ---- rows of a tile to LDS, by way of registers, a tile ahead ----
        int tile0 = t_begin + wave * kAttendTile;
        // BLOCKS: lane l has the offset of block l % 2 of the wavefront's tile l / 2, counted from tile0.  Else it has the page of
        // row l % 32 of the tile that is loaded next.
        int64_t entry = 0;
        bool entry_ok = false;
        int page = -1;
        auto load_entries = [&](int tile) {
            const int tok = tile + (lane >> 1) * kAttendUnit + (lane & 1) * 16;
            page = -1;
            if (tok < t_end) page = table[a.page_size((uint32_t)tok)];
        };
        auto set_entries = [&](int tile) {
            const int tok = tile + (lane >> 1) * kAttendUnit + (lane & 1) * 16;
            entry_ok = (unsigned)page < (unsigned)a.num_pages;
            entry = entry_ok ? page * a.page_stride + (tok - (int)a.page_size((uint32_t)tok) * (int)a.page_size.d) * a.row_stride + head_off : 0;
        };
        auto load_page = [&](int tile) {
            const int tok = tile + (lane & 31);
            page = -1;
            if (tok >= t_low && tok < t_end) page = table[a.page_size((uint32_t)tok)];
        };
        // the pages of the first tile are asked for before anything else
        if constexpr (BLOCKS) load_entries(tile0);
        else load_page(tile0);
        __builtin_amdgcn_sched_barrier(0);
        v4f_att acch[HT], accl[NL ? NL : 1];
#pragma unroll
        for (int j = 0; j < HT; ++j) acch[j] = (v4f_att){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NL; ++j) accl[j] = (v4f_att){0.0f, 0.0f, 0.0f, 0.0f};
        // of the own four queries: running maximum times log2 e, sum of weights, and weighted sums of zero-points (with what the
        // codes' offsets and the weights' rests come to), the last three over the own tokens
        float m2[4], l[4], zero_h[4], zero_l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m2[i] = kAttendNone;
            l[i] = zero_h[i] = zero_l[i] = 0.0f;
        }

        uint4 kreg[KU], vreg[KU];   // (where a row is not there they keep what they had: codes of some kind)
#pragma unroll
        for (int i = 0; i < KU; ++i) kreg[i] = vreg[i] = make_uint4(0u, 0u, 0u, 0u);
        // a lane's pieces: the row, what is in front of it in the row, and where it goes
        int piece_row[KU], piece_off[KU], piece_to[KU];
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int k = i * 64 + lane, row = k / PL, col = k - row * PL;
            piece_row[i] = min(row, kAttendTile - 1);
            piece_off[i] = (BLOCKS ? (row & 15) * (int)a.row_stride : 0) + (col < PL - 1 ? min(16 * col, RB - 16) : RB - 16);
            piece_to[i] = piece_row[i] * P + (col < PL - 1 ? 16 * col : P - 16);
        }
        // the tokens of a tile that are there and seen
        auto seen = [&](int tile) {
            const int left = len - tile, skip = t_low - tile;
            uint32_t mask = left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1u;
            if (skip > 0) mask &= 0xFFFFFFFFu << skip;
            return mask;
        };
        // asks for a tile's pieces; returns the mask of its tokens
        auto load_tile = [&](int tile) {
            uint32_t mask = seen(tile);
            if constexpr (BLOCKS) {
                const int at = 2 * ((tile - tile0) / kAttendUnit);
                const uint64_t ok = __builtin_amdgcn_ballot_w64(entry_ok);
                mask &= ((ok >> at) & 1 ? 0x0000FFFFu : 0u) | ((ok >> (at + 1)) & 1 ? 0xFFFF0000u : 0u);
                const int64_t e0 = lane_of64(entry, at), e1 = lane_of64(entry, at + 1);
#pragma unroll
                for (int i = 0; i < KU; ++i) {
                    const int64_t e = (64 * i + 63) / PL < 16 ? e0 : 64 * i / PL >= 16 ? e1 : piece_row[i] < 16 ? e0 : e1;
                    if ((64 * (i + 1) <= kAttendTile * PL || 64 * i + lane < kAttendTile * PL) &&
                        (mask == 0xFFFFFFFFu || ((mask >> piece_row[i]) & 1))) {
                        kreg[i] = piece_at(a.pages[0] + e + (uint32_t)piece_off[i]);
                        vreg[i] = piece_at(a.pages[1] + e + (uint32_t)piece_off[i]);
                    }
                }
            } else {
                const int tok = tile + (lane & 31);
                const bool ok = (unsigned)page < (unsigned)a.num_pages;
                const int64_t off = ok ? page * a.page_stride + (tok - (int)a.page_size((uint32_t)tok) * (int)a.page_size.d) * a.row_stride + head_off : 0;
                mask &= (uint32_t)__builtin_amdgcn_ballot_w64(ok);
#pragma unroll
                for (int i = 0; i < KU; ++i) {
                    const int64_t e = ((int64_t)__shfl((int)(off >> 32), piece_row[i]) << 32) | (uint32_t)__shfl((int)off, piece_row[i]);
                    if ((64 * (i + 1) <= kAttendTile * PL || 64 * i + lane < kAttendTile * PL) && ((mask >> piece_row[i]) & 1)) {
                        kreg[i] = piece_at(a.pages[0] + e + piece_off[i]);
                        vreg[i] = piece_at(a.pages[1] + e + piece_off[i]);
                    }
                }
            }
            return mask;
        };

        // the queries, behind the pages in the queue, and the first tile
        // ---- queries: operands of the first product, and their sums over both groups of channels ----
        const int qi = qt * kAttendRows + (n & (Q - 1));   // among the queries of the K/V head
        const bool q_live = qi < a.share;
        const uint16_t* qrow = a.q + b * a.ldq + (int64_t)(hk * a.share + (q_live ? qi : 0)) * a.ldqh;
        int h_here = a.r - 8 * g, l_here = low - 8 * g;   // (kept from the compiler, which would hold the comparisons for all heads)
        asm volatile("" : "+v"(h_here), "+v"(l_here));
        Piece16 raw_h[HS], raw_l[LS ? LS : 1];
#pragma unroll
        for (int s = 0; s < HS; ++s) {
            raw_h[s] = Piece16{0u, 0u, 0u, 0u};
            if (q_live && 32 * s < h_here) raw_h[s] = *reinterpret_cast<const Piece16*>(qrow + 8 * (4 * s + g));
        }
#pragma unroll
        for (int s = 0; s < LS; ++s) {
            raw_l[s] = Piece16{0u, 0u, 0u, 0u};
            // (the last four alone: with the four in front of them)
            if (q_live && 32 * s < l_here)
                raw_l[s] = *reinterpret_cast<const Piece16*>(qrow + a.r + 8 * (4 * s + g) - (l_here - 32 * s == 4 ? 4 : 0));
        }
        uint32_t next_mask = 0;
        if constexpr (BLOCKS) set_entries(tile0);
        if (tile0 < t_end) next_mask = load_tile(tile0);
        if constexpr (!BLOCKS) load_page(tile0 + kAttendUnit);

        if (a.r & 4) {   // pieces of which four channels are the group's
#pragma unroll
            for (int s = 0; s < HS; ++s)
                if (h_here - 32 * s == 4) raw_h[s].z = raw_h[s].w = 0u;
#pragma unroll
            for (int s = 0; s < LS; ++s)
                if (l_here - 32 * s == 4) raw_l[s] = Piece16{raw_l[s].z, raw_l[s].w, 0u, 0u};
        }
        v4u_att qh[HS], ql[LS ? LS : 1];
        float sum_h = 0.0f, sum_l = 0.0f;
#pragma unroll
        for (int s = 0; s < HS; ++s) {
            qh[s] = (v4u_att){raw_h[s].x, raw_h[s].y, raw_h[s].z, raw_h[s].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) sum_h += __uint_as_float(qh[s][i] << 16) + __uint_as_float(qh[s][i] & 0xFFFF0000u);
        }
#pragma unroll
        for (int s = 0; s < LS; ++s) {
            const Piece16 p = raw_l[s];
            const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) sum_l += __uint_as_float(w[i] << 16) + __uint_as_float(w[i] & 0xFFFF0000u);
            // in the order in which the codes of a dword become operands: 0 4 1 5 2 6 3 7
            ql[s] = (v4u_att){__builtin_amdgcn_perm(p.z, p.x, 0x05040100u), __builtin_amdgcn_perm(p.z, p.x, 0x07060302u),
                              __builtin_amdgcn_perm(p.w, p.y, 0x05040100u), __builtin_amdgcn_perm(p.w, p.y, 0x07060302u)};
        }
        // the sums of a lane's own four queries: what lane 4 g + i (Q = 8: 4 (g & 1) + i) has summed
        sum_h = rows_sum(sum_h);
        sum_l = rows_sum(sum_l);
        const int own = Q == 8 ? 4 * (g & 1) : 4 * g;
        float qsum_h[4], qsum_l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            qsum_h[i] = __shfl(sum_h, own + i);
            qsum_l[i] = __shfl(sum_l, own + i);
        }


        for (int tt = tile0; tt < t_end; tt += kAttendUnit) {
            const uint32_t mask = next_mask;
#pragma unroll
            for (int i = 0; i < KU; ++i) {
                if (64 * (i + 1) <= kAttendTile * PL || 64 * i + lane < kAttendTile * PL) {
                    *reinterpret_cast<uint4*>(kt + piece_to[i]) = kreg[i];
                    *reinterpret_cast<uint4*>(vt + piece_to[i]) = vreg[i];
                }
            }
            const int next = tt + kAttendUnit;
            if (next < t_end) {
                if constexpr (BLOCKS) {
                    if (next - tile0 >= 32 * kAttendUnit) {
                        tile0 = next;
                        load_entries(next);
                        set_entries(next);
                    }
                }
                next_mask = load_tile(next);
                if constexpr (!BLOCKS) load_page(next + kAttendUnit);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();

            // ---- what the tile's work reads of LDS, asked for at once; values' codes only where they leave registers for it (32 x
            // 4096: 256 channels in 8 bits 132 us against 162, 32 of 256 82.5 against 92.1, heads of 64 36.3 against 37.6, of 128 46.9
            // and 47.1; where both groups are wide they do not fit: 64 of 256 351 against 119; 64 of 128 56.3 against 57.3, left) ----
            constexpr bool kEarly = HT <= 2 || (NL == 0 && HT == 16);
            uint2 kh[2][HS];
            uint32_t kl[2][LS ? LS : 1];
            float4 kpar[NT], vpar[NT];
            uint32_t vh[8][kEarly ? HT : 1], vl[8][NL < 8 ? 1 : NL / 8];
            auto vrow = [&](int e) { return vt + (16 * (e >> 2) + 4 * g + (e & 3)) * P; };
            auto own_token = [&](int h) { return Q == 8 ? 16 * (g >> 1) + n : 16 * h + n; };   // of the softmax
            auto read_low = [&](uint32_t (&c)[NL < 8 ? 1 : NL / 8], int e) {
                const uint8_t* p = vrow(e) + a.r + n * (NL / 2);
                if constexpr (NL == 4) c[0] = *reinterpret_cast<const uint16_t*>(p);
                else
#pragma unroll
                    for (int k = 0; k < NL / 8; ++k) c[k] = reinterpret_cast<const uint32_t*>(p)[k];
            };
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint8_t* row = kt + (16 * h + n) * P;
#pragma unroll
                for (int s = 0; s < HS; ++s) kh[h][s] = *reinterpret_cast<const uint2*>(row + 8 * (4 * s + g));
#pragma unroll
                for (int s = 0; s < LS; ++s) kl[h][s] = *reinterpret_cast<const uint32_t*>(row + a.r + 4 * (4 * s + g));
            }
#pragma unroll
            for (int h = 0; h < NT; ++h) {
                kpar[h] = *reinterpret_cast<const float4*>(kt + own_token(h) * P + P - 16);
                vpar[h] = *reinterpret_cast<const float4*>(vt + own_token(h) * P + P - 16);
            }
            if constexpr (kEarly) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
#pragma unroll
                    for (int j = 0; j < HT; ++j) vh[e][j] = vrow(e)[16 * j + n];
                    if constexpr (NL > 0) read_low(vl[e], e);
                }
            }
            __builtin_amdgcn_sched_barrier(0);

            // ---- scores ----
            v4f_att sh[2], sl[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) sh[h] = sl[h] = (v4f_att){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < HS; ++s) {
                if (s == 0 || 32 * s < a.r) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint2 c = kh[h][s];
                        v4u_att o;
                        o[0] = upper_halves((float)(c.x & 0xFFu), (float)((c.x >> 8) & 0xFFu));
                        o[1] = upper_halves((float)((c.x >> 16) & 0xFFu), (float)(c.x >> 24));
                        o[2] = upper_halves((float)(c.y & 0xFFu), (float)((c.y >> 8) & 0xFFu));
                        o[3] = upper_halves((float)((c.y >> 16) & 0xFFu), (float)(c.y >> 24));
                        sh[h] = attend_mfma(qh[s], o, sh[h]);
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < LS; ++s) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t c = kl[h][s];
                    v4u_att o;
                    o[0] = key_bits(c << 3);
                    o[1] = key_bits(c >> 1);
                    o[2] = key_bits(c >> 5);
                    o[3] = key_bits(c >> 9);
                    sl[h] = attend_mfma(ql[s], o, sl[h]);
                }
            }
            float x[NT][4];
#pragma unroll
            for (int h = 0; h < NT; ++h) {
                const float4 par = kpar[h];
                const float z = fmaf(par.z, -16.0f, par.w);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float dh = Q == 8 ? (g & 2 ? sh[1][i] : sh[0][i]) : sh[h][i];
                    float v = fmaf(dh, par.x, qsum_h[i] * par.y);
                    if constexpr (NL > 0) {
                        const float dl = Q == 8 ? (g & 2 ? sl[1][i] : sl[0][i]) : sl[h][i];
                        v = fmaf(dl, par.z, fmaf(qsum_l[i], z, v));
                    }
                    x[h][i] = v;
                }
            }
            if (a.softcap > 0.0f) {
#pragma unroll
                for (int h = 0; h < NT; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[h][i] = soft_cap(x[h][i] * a.scale, a.softcap, inv_cap);
            }
            if (mask != 0xFFFFFFFFu) {   // what is not seen has no weight, and its constants may be anything
#pragma unroll
                for (int h = 0; h < NT; ++h) {
                    const bool there = (mask >> own_token(h)) & 1;
                    vpar[h].x = there ? vpar[h].x : 0.0f;
                    vpar[h].y = there ? vpar[h].y : 0.0f;
                    vpar[h].z = there ? vpar[h].z : 0.0f;
                    vpar[h].w = there ? vpar[h].w : 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[h][i] = there ? x[h][i] : -inf;
                }
            }
            float over[NT][4];   // by how many powers of two a score is over the maximum
            bool rise = false;
#pragma unroll
            for (int h = 0; h < NT; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    over[h][i] = fmaf(x[h][i], sc2, -m2[i]);
                    rise |= over[h][i] > kAttendSlack;
                }

            // ---- the running maximum, where it has to rise ----
            if (__builtin_amdgcn_ballot_w64(rise) != 0) {
                float back[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float top = x[0][i];
                    if constexpr (NT == 2) top = fmaxf(top, x[1][i]);
                    top = row_max16(top);
                    if constexpr (Q == 8) top = halves_max(top);
                    const float m_new = fmaxf(m2[i], top * sc2);
                    back[i] = __builtin_amdgcn_exp2f(m2[i] - m_new);
                    m2[i] = m_new;
#pragma unroll
                    for (int h = 0; h < NT; ++h) over[h][i] = fmaf(x[h][i], sc2, -m_new);
                    l[i] *= back[i];
                    zero_h[i] *= back[i];
                    zero_l[i] *= back[i];
                }
                // the factor of query n (Q = 8: n % 8), from a lane that has it among its own
                const int from_lane = Q == 8 ? 16 * ((n >> 2) & 1) : 16 * (n >> 2);
                const float f0 = __shfl(back[0], from_lane), f1 = __shfl(back[1], from_lane);
                const float f2 = __shfl(back[2], from_lane), f3 = __shfl(back[3], from_lane);
                const float f = n & 2 ? (n & 1 ? f3 : f2) : (n & 1 ? f1 : f0);
#pragma unroll
                for (int j = 0; j < HT; ++j) acch[j] *= f;
#pragma unroll
                for (int j = 0; j < NL; ++j) accl[j] *= f;
            }

            // ---- weights, times both groups' scales, to LDS; zero-points take in the codes' offsets ----
#pragma unroll
            for (int h = 0; h < NT; ++h) {
                const float4 par = vpar[h];
                const float zh = fmaf(par.x, n & 1 ? 255.0f : 0.0f, par.y), zl = fmaf(par.z, n & 1 ? 143.0f : -128.0f, par.w);
                // as the second product counts tokens: 4 g + i, i < 4, then 16 more
                const int tok = own_token(h), pos = 8 * ((tok >> 2) & 3) + 4 * (tok >> 4) + (tok & 3);
                uint8_t* dst = pt + own * kAttendPRow + 2 * pos;
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    float p[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        p[e] = __builtin_amdgcn_exp2f(over[h][i + e]);
                        l[i + e] += p[e];
                        zero_h[i + e] = fmaf(p[e], zh, zero_h[i + e]);
                        zero_l[i + e] = fmaf(p[e], zl, zero_l[i + e]);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {   // the 8-bit group's rows, then the 4-bit group's: first numbers, then second ones
                        const float s = k ? par.z : par.x, w0 = p[0] * s, w1 = p[1] * s;
                        const uint32_t big = pack_bf16_pair(w0, w1);
                        const float r0 = w0 - __uint_as_float(big << 16), r1 = w1 - __uint_as_float(big & 0xFFFF0000u);
                        const uint32_t rest = pack_bf16_pair(r0, r1);
                        const float mid = k ? (n & 1 ? -135.5f : 135.5f) : (n & 1 ? -127.5f : 127.5f);
                        float(&zero)[4] = k ? zero_l : zero_h;
                        zero[i] = fmaf(r0 - __uint_as_float(rest << 16), mid, zero[i]);
                        zero[i + 1] = fmaf(r1 - __uint_as_float(rest & 0xFFFF0000u), mid, zero[i + 1]);
                        *reinterpret_cast<uint16_t*>(dst + (2 * Q * k + i) * kAttendPRow) = (uint16_t)big;
                        *reinterpret_cast<uint16_t*>(dst + (2 * Q * k + i + 1) * kAttendPRow) = (uint16_t)(big >> 16);
                        *reinterpret_cast<uint16_t*>(dst + (2 * Q * k + Q + i) * kAttendPRow) = (uint16_t)rest;
                        *reinterpret_cast<uint16_t*>(dst + (2 * Q * k + Q + i + 1) * kAttendPRow) = (uint16_t)(rest >> 16);
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();

            // ---- weighted sums of the values' codes ----
            const v4u_att* pw = reinterpret_cast<const v4u_att*>(pt + n * kAttendPRow + 16 * g);
            constexpr int kPart = Q * kAttendPRow / 16;   // from truncations to remainders (Q = 8: they are this product's columns 8 to 15)
            {
                const v4u_att w = pw[0];
#pragma unroll
                for (int j = 0; j < HT; ++j) {
                    if (j == 0 || 16 * j < a.r) {
                        v4u_att o;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t c0, c1;
                            if constexpr (kEarly) {
                                c0 = vh[2 * i][j];
                                c1 = vh[2 * i + 1][j];
                            } else {
                                c0 = vrow(2 * i)[16 * j + n];
                                c1 = vrow(2 * i + 1)[16 * j + n];
                            }
                            o[i] = upper_halves((float)c0, (float)(c1 ^ 255u)) ^ 0x80000000u;
                        }
                        acch[j] = attend_mfma(o, w, acch[j]);
                        if constexpr (Q == 16) acch[j] = attend_mfma(o, pw[kPart], acch[j]);
                    }
                }
            }
            if constexpr (NL > 0) {
                const v4u_att w = pw[2 * kPart];
                if constexpr (!kEarly) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) read_low(vl[e], e);
                }
#pragma unroll
                for (int k = 0; k < NL / 4; ++k) {   // four channels at a time: half a dword of two tokens in one
                    uint32_t two[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        two[i] = __builtin_amdgcn_perm(~vl[2 * i + 1][k >> 1], vl[2 * i][k >> 1], k & 1 ? 0x07060302u : 0x05040100u);
                    v4u_att o[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[j][i] = value_bits(two[i] >> (4 * j));
                        accl[4 * k + j] = attend_mfma(o[j], w, accl[4 * k + j]);
                    }
                    if constexpr (Q == 16) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) accl[4 * k + j] = attend_mfma(o[j], pw[3 * kPart], accl[4 * k + j]);
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }

        // ---- the four wavefronts' results together ----
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                float& v = k == 0 ? l[i] : k == 1 ? zero_h[i] : zero_l[i];
                v = row_sum16(v);
                if constexpr (Q == 8) v = halves_sum(v);
            }
        }
        if constexpr (Q == 8) {
#pragma unroll
            for (int j = 0; j < HT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acch[j][i] += lane_xor<8>(acch[j][i]);
#pragma unroll
            for (int j = 0; j < NL; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) accl[j][i] += lane_xor<8>(accl[j][i]);
        }
        __syncthreads();   // every wavefront is through with its rows
        const int rows = min(a.share - qt * kAttendRows, kAttendRows);
        float* red = reinterpret_cast<float*>(lds);                           // [wave][rows][d]
        float4* ml = reinterpret_cast<float4*>(lds + a.lds_red);              // [wave][16]: maximum, sum, zero-points' sums
        if (n == 0 && (Q == 16 || g < 2)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) ml[wave * kAttendRows + own + i] = make_float4(m2[i], l[i], zero_h[i], zero_l[i]);
        }
        // both groups have a multiple of 4 channels, so that four in a row from a multiple of 4 on are of one group or of none.
        // (What the limits are is kept from the compiler: it would take the comparisons out of the loop, each in registers.)
        int h_left = a.r - 4 * g, l_left = low - 4 * g * NL;
        asm volatile("" : "+v"(h_left), "+v"(l_left));
        if (n < Q && n < rows) {
            float* row = red + (wave * rows + n) * a.d;
#pragma unroll
            for (int j = 0; j < HT; ++j) {
                if (16 * j < h_left) *reinterpret_cast<v4f_att*>(row + 16 * j + 4 * g) = acch[j];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < NL; j += 4) {
                    const v4f_att o = {accl[j][i], accl[j + 1][i], accl[j + 2][i], accl[j + 3][i]};
                    if (i * NL + j < l_left) *reinterpret_cast<v4f_att*>(row + a.r + (4 * g + i) * NL + j) = o;
                }
        }
        __syncthreads();
        // a head in one piece is done; a piece of one is partial result 0 of its workgroup, or 1 behind another head
        const bool whole = n_units == units;
        const int64_t slot = 2 * (int64_t)w0 + !first_head;
        first_head = false;
        if (t == 0) {
            int32_t* join = a.joins + ((int64_t)b * heads + head) * 2;
            if (first_unit == 0) join[0] = (int32_t)slot;
            if (first_unit + n_units == units) join[1] = (int32_t)w0;
        }
        const int fours = a.d >> 2;   // four channels to a thread, of one group
        for (int e = t; e < rows * fours; e += kAttendThreads) {
            const int row = (int)((uint32_t)e * (uint32_t)a.fours_magic >> 16), ch = 4 * (e - row * fours);
            float4 v[kAttendWaves];
            v4f_att part_o[kAttendWaves];
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) {
                v[w] = ml[w * kAttendRows + row];
                part_o[w] = *reinterpret_cast<const v4f_att*>(red + (w * rows + row) * a.d + ch);
            }
            const float top = fmaxf(fmaxf(v[0].x, v[1].x), fmaxf(v[2].x, v[3].x));
            float sum = 0.0f;
            v4f_att o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(v[w].x - top), z = ch < a.r ? v[w].z : v[w].w;
                sum = fmaf(f, v[w].y, sum);
                o += f * (part_o[w] + z);
            }
            const int qhead = hk * a.share + qt * kAttendRows + row;
            if (whole) {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                uint16_t* dst = a.out + b * a.ldo + qhead * a.ldoh + ch;
                *reinterpret_cast<Piece8*>(dst) = Piece8{pack_bf16_pair(o[0] * inv, o[1] * inv), pack_bf16_pair(o[2] * inv, o[3] * inv)};
                if (ch == 0 && a.lse)
                    a.lse[(int64_t)b * a.heads_k * a.share + qhead] = sum == 0.0f ? -inf : top * 0.69314718055994530942f + logf(sum);
            } else {
                *reinterpret_cast<v4f_att*>(a.part_acc + (slot * a.rows + row) * a.d + ch) = o;
                if (ch == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * kAttendRows + row) * 2) = make_float2(top, sum);
            }
        }
        __syncthreads();   // before the rows of the next head come to LDS
    }
}

// Joins the partial results of the heads that several workgroups had, and writes the queries of sequences without tokens; a
// workgroup to a head's queries, or to one of them (grid.y) where there are few.
//   m = max m_i, f_i = 2^(m_i - m), out = sum f_i acc_i / sum f_i l_i, lse = m ln 2 + ln sum f_i l_i
// Few partial results, the usual case: four channels of a query to a thread, all its reads at once.  More: all threads to one
// query after the other, in three barriers each.
// Bound by the launch and two dependent reads: by a trace 3.8 us for 8 heads of 4 queries in 7 parts, 5.6 for 8 of 8 in 64.  A workgroup
// to every query always: 256 x 512 59.5 us with the main kernel instead of 56.5; to every head always: 1 x 8192 22.1 instead of 15.1,
// 1 x 131072 with 64 queries 68.5 instead of 49.0.  512 threads instead of 256: 256 x 512 an eighth more.
__global__ __launch_bounds__(kAttendThreads) void attend_join_kernel(const AttendArgs a) {
    __shared__ float weight[kAttendMaxGrid], weight_sum[kAttendMaxGrid], part[2 * kAttendWaves];
    __shared__ float4 red[kAttendThreads];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int heads = a.heads_k * a.qtiles;
    const int b = blockIdx.x / heads, head = blockIdx.x - b * heads;
    const int hk = head / a.qtiles, qt = head - hk * a.qtiles;
    const int32_t* join = a.joins + (int64_t)blockIdx.x * 2;
    const int slot0 = join[0], w_last = join[1];   // (nobody wrote them for a sequence without tokens)
    const int rows = min(a.share - qt * kAttendRows, kAttendRows);
    const int row0 = gridDim.y > 1 ? blockIdx.y : 0, row1 = gridDim.y > 1 ? min(row0 + 1, rows) : rows;
    const int q0 = hk * a.share + qt * kAttendRows;   // the query head of row 0
    uint16_t* out = a.out + b * a.ldo + q0 * a.ldoh;
    float* lse = a.lse ? a.lse + (int64_t)b * a.heads_k * a.share + q0 : nullptr;
    const float inf = __builtin_huge_valf();
    const int fours = a.d >> 2;
    auto write = [&](int row, int ch, const float4& o, float top, float sum) {
        const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<Piece8*>(out + row * a.ldoh + ch) = Piece8{pack_bf16_pair(o.x * f, o.y * f), pack_bf16_pair(o.z * f, o.w * f)};
        if (ch == 0 && lse) lse[row] = sum == 0.0f ? -inf : top * 0.69314718055994530942f + logf(sum);
    };
    const bool empty = attend_len(a, b) == 0;
    const int w_first = slot0 >> 1, count = w_last - w_first + 1;
    if (!empty && count == 1) return;
    auto slot = [&](int i) { return (int64_t)(i == 0 ? slot0 : 2 * (w_first + i)); };
    if (empty || count <= kAttendJoinFew) {
        for (int e = row0 * fours + t; e < row1 * fours; e += kAttendThreads) {
            const int row = (int)((uint32_t)e * (uint32_t)a.fours_magic >> 16), ch = 4 * (e - row * fours);
            float4 v[kAttendJoinFew], o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float2 ml[kAttendJoinFew];
            float top = kAttendNone, sum = 0.0f;
            if (!empty) {
#pragma unroll
                for (int i = 0; i < kAttendJoinFew; ++i)
                    if (i < count) {
                        ml[i] = *reinterpret_cast<const float2*>(a.part_ml + (slot(i) * kAttendRows + row) * 2);
                        v[i] = *reinterpret_cast<const float4*>(a.part_acc + (slot(i) * a.rows + row) * a.d + ch);
                    }
#pragma unroll
                for (int i = 0; i < kAttendJoinFew; ++i)
                    if (i < count) top = fmaxf(top, ml[i].x);
#pragma unroll
                for (int i = 0; i < kAttendJoinFew; ++i)
                    if (i < count) {
                        const float f = __builtin_amdgcn_exp2f(ml[i].x - top);
                        sum = fmaf(f, ml[i].y, sum);
                        o.x = fmaf(f, v[i].x, o.x);
                        o.y = fmaf(f, v[i].y, o.y);
                        o.z = fmaf(f, v[i].z, o.z);
                        o.w = fmaf(f, v[i].w, o.w);
                    }
            }
            write(row, ch, o, top, sum);
        }
        return;
    }
    // four channels to a thread, what threads are left over the partial results, four of which are on their way at a time; the
    // first four are asked for before their weights are known
    const int groups = kAttendThreads / fours, group = t / fours, ch = 4 * (t - group * fours);
    for (int row = row0; row < row1; ++row) {
        float4 v[4];
        auto load_four = [&](int i) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[k] = *reinterpret_cast<const float4*>(a.part_acc + (slot(min(i + k * groups, count - 1)) * a.rows + row) * a.d + ch);
        };
        if (group < groups) load_four(group);
        float top = kAttendNone, sum = 0.0f;
        for (int i = t; i < count; i += kAttendThreads) {
            const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (slot(i) * kAttendRows + row) * 2);
            weight[i] = ml.x;
            weight_sum[i] = ml.y;
            top = fmaxf(top, ml.x);
        }
        top = halves_max(fmaxf(row_max16(top), lane_xor<16>(row_max16(top))));
        if (lane == 0) part[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        for (int i = t; i < count; i += kAttendThreads) {
            const float f = __builtin_amdgcn_exp2f(weight[i] - top);
            weight[i] = f;
            sum = fmaf(f, weight_sum[i], sum);
        }
        sum = row_sum16(sum);
        sum = rows_sum(sum);
        if (lane == 0) part[kAttendWaves + wave] = sum;
        __syncthreads();
        sum = (part[kAttendWaves] + part[kAttendWaves + 1]) + (part[kAttendWaves + 2] + part[kAttendWaves + 3]);
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (group < groups) {
            for (int i = group; i < count; i += 4 * groups) {
                if (i != group) load_four(i);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float f = i + k * groups < count ? weight[i + k * groups] : 0.0f;
                    if (f != 0.0f) {   // (a workgroup that saw nothing)
                        o.x = fmaf(f, v[k].x, o.x);
                        o.y = fmaf(f, v[k].y, o.y);
                        o.z = fmaf(f, v[k].z, o.z);
                        o.w = fmaf(f, v[k].w, o.w);
                    }
                }
            }
        }
        red[t] = o;
        __syncthreads();
        if (t < fours) {
            for (int k = 1; k < groups; ++k) {
                const float4 v = red[k * fours + t];
                o.x += v.x;
                o.y += v.y;
                o.z += v.z;
                o.w += v.w;
            }
            write(row, 4 * t, o, top, sum);
        }
        __syncthreads();   // before the next query's weights
    }
}

}  // namespace resq
