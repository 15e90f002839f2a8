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
// Queries of one K/V head are the columns of both products; a wavefront takes 32 tokens at a time.
//   S (tokens x queries) = K codes x Q: lane l ends with query l % 16 and tokens 4 (l / 16) + i and 16 + those, i < 4
//   O (channels x queries) += V codes^T x P: its operand P wants of lane l query l % 16 and any eight tokens, which the codes
//   of V are then taken of too: the eight it has.  Softmax weights never move between lanes.
// A 4-bit code becomes a bf16 number by being put under the leading bits of 16 (keys) or 128 (values): one shift and one
// and-or for two codes.  The constants leave again: 16 sum(q) with the accumulator's start; for values every second token has
// the code's complement and the opposite sign, c + 128 and c - 143, so that the sums stay small, and what remains is a sum of
// weights.  P goes in as two bf16 numbers, a truncation and its remainder (16 bits in all, so that the output's rounding to
// bf16 is the one that counts).
//
// The work is cut into units of 128 tokens of one head (four wavefronts, 32 tokens each); all units of the call in a row are
// dealt to the workgroups in runs of equal length, whatever the sequences' lengths are (they are read on the GPU).  A head
// that ends up with several workgroups is joined by a second kernel from their maxima, sums and partial outputs.
//
// Bound: HBM, 2 row bytes per token and K/V head.
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
constexpr int kAttendMaxGrid = 1024;
constexpr int kAttendRows = 16;                              // queries of a workgroup at most
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
    int num_pages, page_size;
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
    int blocks16;      // 16 rows of a page from a multiple of 16 on are contiguous and 16-byte aligned
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
// max and sum over the four lanes l % 16 + 16 k: swaps of halves and of rows of 16 lanes
__device__ __forceinline__ float rows_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
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

// Bytes from row to row in LDS: what the kernel's groups of channels take, so that every address is a lane's base and a
// constant, and 16 more than a multiple of 32, so that 16 rows, and rows 4 apart, spread over all banks.  A row's scales and
// zero-points are its last 16 bytes there.
__host__ __device__ constexpr int attend_row(int NL, int HT) { return HT * 16 + NL * 8 + 16 < 272 ? HT * 16 + NL * 8 + 16 : 272; }
__host__ __device__ constexpr int attend_pitch(int NL, int HT) { return (attend_row(NL, HT) + 15) / 32 * 32 + 16; }
// a number that all lanes have, in scalar registers
__device__ __forceinline__ int64_t uniform64(int64_t x) {
    return ((int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
// NL: 4-bit channels of a lane in the second product (16 NL channels in all), HT: 16-channel tiles of the 8-bit group,
// BLOCKS: 16 rows of a page from a multiple of 16 on are contiguous pieces of 16 bytes
template <int NL, int HT, bool BLOCKS, int OCC>
__global__ __launch_bounds__(kAttendThreads, OCC) void attend_kv_cache_kernel(const AttendArgs a) {
    constexpr int LS = NL / 2, HS = (HT + 1) / 2;   // steps of 32 channels of the first product
    constexpr int P = attend_pitch(NL, HT);
    constexpr int KU = (attend_row(NL, HT) + 63) / 64;   // 16-byte pieces of 16 rows that a lane moves
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ int64_t part[kAttendWaves], found_start;
    __shared__ int found_b;

    const int t = threadIdx.x, lane = t & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int heads = a.heads_k * a.qtiles;   // heads' query tiles of a sequence

    // ---- the run of units that is this workgroup's ----
    const int per = (a.B + kAttendThreads - 1) / kAttendThreads;
    const int b0 = min(t * per, a.B), b1 = min(b0 + per, a.B);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += (int64_t)attend_units(a, attend_len(a, b)) * heads;
    int64_t upto = mine;
    for (int k = 1; k < 64; k <<= 1) {
        const int64_t u = __shfl_up(upto, k);
        if (lane >= k) upto += u;
    }
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    int64_t total = 0, before = 0;
    for (int w = 0; w < kAttendWaves; ++w) {
        if (w == wave) before = total;
        total += part[w];
    }
    int64_t start = before + upto - mine;   // of this thread's first sequence
    total = uniform64(total);
    const int64_t W = total < (int64_t)gridDim.x ? total : (int64_t)gridDim.x;
    const int64_t w0 = blockIdx.x;
    if (w0 >= W) return;
    int64_t u = total * w0 / W;
    const int64_t u_end = total * (w0 + 1) / W;
    if (start <= u && u < start + mine) {
        for (int b = b0; b < b1; ++b) {
            const int64_t units = (int64_t)attend_units(a, attend_len(a, b)) * heads;
            if (u < start + units) {
                found_b = b;
                found_start = start;
                break;
            }
            start += units;
        }
    }
    __syncthreads();
    int b = __builtin_amdgcn_readfirstlane(found_b);
    int64_t seq_start = uniform64(found_start);
    const int64_t u_first = u;

    const int RB = a.row_bytes, low = a.d - a.r, par_off = a.r + (low >> 1);
    uint8_t* kt = lds + wave * (2 * kAttendTile * P);
    uint8_t* vt = kt + kAttendTile * P;
    int to[2 * KU];   // where the halves of a lane's pieces go
    if constexpr (BLOCKS) {
#pragma unroll
        for (int i = 0; i < 2 * KU; ++i) {
            const int at = (i >> 1) * 1024 + lane * 16 + (i & 1) * 8, row = at / RB, col = at - row * RB;
            to[i] = row * P + col + (col < par_off ? 0 : P - 16 - par_off);
        }
    }
    const float inv_cap = a.softcap > 0.0f ? 1.0f / a.softcap : 0.0f;
    const float kLog2e = 1.44269504088896340736f;
    const float sc2 = a.softcap > 0.0f ? kLog2e : a.scale * kLog2e;
    const float inf = __builtin_huge_valf();

    const CodeBits key_bits(0x00780078u, 0x41804180u), value_bits(0x000F000Fu, 0xC3004300u);

    while (u < u_end) {
        // ---- the next head in the run ----
        const int len = __builtin_amdgcn_readfirstlane(attend_len(a, b));
        const int units = attend_units(a, len);
        const int64_t seq_units = (int64_t)units * heads;
        if (u >= seq_start + seq_units) {
            seq_start += seq_units;
            ++b;
            continue;
        }
        const int head = (int)((u - seq_start) / units), first_unit = (int)((u - seq_start) - (int64_t)head * units);
        const int n_units = (int)(units - first_unit < u_end - u ? units - first_unit : u_end - u);
        const int hk = head / a.qtiles, qt = head - hk * a.qtiles;
        const int t_low = attend_first(a, len), from = t_low & ~(kAttendTile - 1);
        const int t_begin = from + first_unit * kAttendUnit;
        const int t_end = min(len, t_begin + n_units * kAttendUnit);
        const int64_t head_off = hk * a.head_stride;
        const int32_t* table = a.table + b * a.ld_table;

        // ---- queries: operands of the first product, and their sums over both groups of channels ----
        const int qi = qt * kAttendRows + n;   // among the queries of the K/V head
        const bool q_live = qi < a.share;
        const uint16_t* qrow = a.q + b * a.ldq + (int64_t)(hk * a.share + (q_live ? qi : 0)) * a.ldqh;
        v4u_att qh[HS], ql[LS ? LS : 1];
        int r_here = a.r, low_here = low;
        asm volatile("" : "+s"(r_here), "+s"(low_here));
        float sum_h = 0.0f, sum_l = 0.0f;
#pragma unroll
        for (int s = 0; s < HS; ++s) {
            const int ch = 8 * (4 * s + g);
            qh[s] = (v4u_att){0u, 0u, 0u, 0u};
            if (q_live && ch < r_here) {
                const Piece16 p = *reinterpret_cast<const Piece16*>(qrow + ch);
                qh[s] = (v4u_att){p.x, p.y, p.z, p.w};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sum_h += __uint_as_float(qh[s][i] << 16) + __uint_as_float(qh[s][i] & 0xFFFF0000u);
        }
#pragma unroll
        for (int s = 0; s < LS; ++s) {
            const int ch = 8 * (4 * s + g);
            Piece16 p{0u, 0u, 0u, 0u};
            if (q_live && ch < low_here) p = *reinterpret_cast<const Piece16*>(qrow + a.r + ch);
            const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) sum_l += __uint_as_float(w[i] << 16) + __uint_as_float(w[i] & 0xFFFF0000u);
            // in the order in which the codes of a dword become operands: 0 4 1 5 2 6 3 7
            ql[s] = (v4u_att){__builtin_amdgcn_perm(p.z, p.x, 0x05040100u), __builtin_amdgcn_perm(p.z, p.x, 0x07060302u),
                              __builtin_amdgcn_perm(p.w, p.y, 0x05040100u), __builtin_amdgcn_perm(p.w, p.y, 0x07060302u)};
        }
        sum_h = rows_sum(sum_h);
        sum_l = rows_sum(sum_l);

        v4f_att acch[HT], accl[NL ? NL : 1];
#pragma unroll
        for (int j = 0; j < HT; ++j) acch[j] = (v4f_att){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NL; ++j) accl[j] = (v4f_att){0.0f, 0.0f, 0.0f, 0.0f};
        float m2 = -inf, l = 0.0f, zero_h = 0.0f, zero_l = 0.0f;   // m2: maximum times log2 e

        // ---- rows of a tile to LDS ----
        uint4 kreg[2 * KU], vreg[2 * KU];   // (where a block is not there they keep what they had: codes of some kind)
#pragma unroll
        for (int i = 0; i < 2 * KU; ++i) kreg[i] = vreg[i] = make_uint4(0u, 0u, 0u, 0u);
        int64_t entry = 0;        // BLOCKS: offset of block lane % 2 of the wavefront's tile lane / 2, counted from tile0
        bool entry_ok = false;
        int tile0 = t_begin + wave * kAttendTile;
        auto load_entries = [&](int from_token) {
            const int tok = from_token + (lane >> 1) * kAttendUnit + (lane & 1) * 16;
            int page = -1;
            if (tok < t_end) page = table[tok / a.page_size];
            entry_ok = (unsigned)page < (unsigned)a.num_pages;
            entry = entry_ok ? page * a.page_stride + (tok % a.page_size) * a.row_stride + head_off : 0;
        };
        // the tokens of the tile at token tt that are there and seen
        auto seen = [&](int tt) {
            const int left = len - tt, skip = t_low - tt;
            uint32_t mask = left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1u;
            if (skip > 0) mask &= 0xFFFFFFFFu << skip;
            return mask;
        };
        // whole blocks of 16 rows, 16 bytes per lane and load; returns the tile's mask
        auto load_blocks = [&](int tt) {
            const int at = 2 * ((tt - tile0) / kAttendUnit);
            const uint64_t ok = __builtin_amdgcn_ballot_w64(entry_ok);
            const bool ok0 = (ok >> at) & 1, ok1 = (ok >> (at + 1)) & 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!(h ? ok1 : ok0)) continue;
                const int64_t e = ((int64_t)__builtin_amdgcn_readlane((int)(entry >> 32), at + h) << 32) |
                                  (uint32_t)__builtin_amdgcn_readlane((int)entry, at + h);
                const uint8_t* kp = a.pages[0] + e;
                const uint8_t* vp = a.pages[1] + e;
#pragma unroll
                for (int i = 0; i < KU; ++i) {   // RB pieces in a block
                    if (i * 64 + lane < RB) {
                        kreg[h * KU + i] = *reinterpret_cast<const uint4*>(kp + (uint32_t)(i * 1024 + lane * 16));
                        vreg[h * KU + i] = *reinterpret_cast<const uint4*>(vp + (uint32_t)(i * 1024 + lane * 16));
                    }
                }
            }
            return seen(tt) & ((ok0 ? 0x0000FFFFu : 0u) | (ok1 ? 0xFFFF0000u : 0u));
        };
        auto store_blocks = [&]() {
#pragma unroll
            for (int i = 0; i < KU; ++i) {
                if (i * 64 + lane < RB) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 k = kreg[h * KU + i], v = vreg[h * KU + i];
                        *reinterpret_cast<uint2*>(kt + h * 16 * P + to[2 * i]) = make_uint2(k.x, k.y);
                        *reinterpret_cast<uint2*>(kt + h * 16 * P + to[2 * i + 1]) = make_uint2(k.z, k.w);
                        *reinterpret_cast<uint2*>(vt + h * 16 * P + to[2 * i]) = make_uint2(v.x, v.y);
                        *reinterpret_cast<uint2*>(vt + h * 16 * P + to[2 * i + 1]) = make_uint2(v.z, v.w);
                    }
                }
            }
        };
        // rows anywhere, 4 bytes per lane and load, row by row through the table; rows that are not there become zeros
        auto move_rows = [&](int tt) {
            const int tok = tt + (lane & 31);
            int page = -1;
            if (tok < len && tok >= t_low) page = table[tok / a.page_size];
            const bool ok = (unsigned)page < (unsigned)a.num_pages;
            const int64_t off = ok ? page * a.page_stride + (tok % a.page_size) * a.row_stride + head_off : 0;
            const uint32_t mask = (uint32_t)__builtin_amdgcn_ballot_w64(ok);
            const int words = RB >> 2;
            for (int i = 0; i < kAttendTile * words; i += 256) {
                uint32_t kw[4], vw[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int word = i + 64 * j + lane;
                    const int row = min(word / words, kAttendTile - 1), col = word - row * words;
                    const int64_t at = ((int64_t)__shfl((int)(off >> 32), row) << 32) | (uint32_t)__shfl((int)off, row);
                    kw[j] = vw[j] = 0u;
                    if (word < kAttendTile * words && ((mask >> row) & 1)) {
                        kw[j] = *reinterpret_cast<const uint32_t*>(a.pages[0] + at + 4 * col);
                        vw[j] = *reinterpret_cast<const uint32_t*>(a.pages[1] + at + 4 * col);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int word = i + 64 * j + lane, row = word / words, col = 4 * (word - row * words);
                    if (row < kAttendTile) {
                        const int at = row * P + col + (col < par_off ? 0 : P - 16 - par_off);
                        *reinterpret_cast<uint32_t*>(kt + at) = kw[j];
                        *reinterpret_cast<uint32_t*>(vt + at) = vw[j];
                    }
                }
            }
            return mask;
        };

        uint32_t next_mask = 0;
        if (BLOCKS && tile0 < t_end) {
            load_entries(tile0);
            next_mask = load_blocks(tile0);
        }
        for (int tt = tile0; tt < t_end; tt += kAttendUnit) {
            uint32_t mask;
            if constexpr (BLOCKS) {
                mask = next_mask;
                store_blocks();
                const int nt = tt + kAttendUnit;
                if (nt < t_end) {
                    if (nt - tile0 >= 32 * kAttendUnit) {
                        tile0 = nt;
                        load_entries(nt);
                    }
                    next_mask = load_blocks(nt);
                }
            } else {
                mask = move_rows(tt);
            }
            const bool full = mask == 0xFFFFFFFFu;
            // For the values' sums a token's zero-points take in the offsets of its codes there; a token that is not seen gets
            // zeros, since its weight of 0 would not make 0 of what may be anything.
            if (lane < kAttendTile) {
                float4* par = reinterpret_cast<float4*>(vt + lane * P + P - 16);
                float4 v = *par;
                v.y = fmaf(v.x, lane & 1 ? 255.0f : 0.0f, v.y);
                v.w = fmaf(v.z, lane & 1 ? 143.0f : -128.0f, v.w);
                if (!((mask >> lane) & 1)) v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                *par = v;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();

            __builtin_amdgcn_sched_barrier(0);
            // ---- scores ----
            float x[8];
            v4f_att sh[2], sl[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                sh[h] = (v4f_att){0.0f, 0.0f, 0.0f, 0.0f};
                sl[h] = (v4f_att){-16.0f * sum_l, -16.0f * sum_l, -16.0f * sum_l, -16.0f * sum_l};
            }
#pragma unroll
            for (int s = 0; s < HS; ++s) {
                if (s == 0 || 32 * s < a.r) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint2 c = *reinterpret_cast<const uint2*>(kt + (16 * h + n) * P + 8 * (4 * s + g));
                        v4u_att o;
                        o[0] = upper_halves((float)(c.x & 0xFFu), (float)((c.x >> 8) & 0xFFu));
                        o[1] = upper_halves((float)((c.x >> 16) & 0xFFu), (float)(c.x >> 24));
                        o[2] = upper_halves((float)(c.y & 0xFFu), (float)((c.y >> 8) & 0xFFu));
                        o[3] = upper_halves((float)((c.y >> 16) & 0xFFu), (float)(c.y >> 24));
                        sh[h] = attend_mfma(o, qh[s], sh[h]);
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < LS; ++s) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t c = *reinterpret_cast<const uint32_t*>(kt + (16 * h + n) * P + a.r + 4 * (4 * s + g));
                    v4u_att o;
                    o[0] = key_bits(c << 3);
                    o[1] = key_bits(c >> 1);
                    o[2] = key_bits(c >> 5);
                    o[3] = key_bits(c >> 9);
                    sl[h] = attend_mfma(o, ql[s], sl[h]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);   // (here and below: what a later phase reads does not come earlier, for registers)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float4 par = *reinterpret_cast<const float4*>(kt + (16 * (e >> 2) + 4 * g + (e & 3)) * P + P - 16);
                float v = fmaf(sh[e >> 2][e & 3], par.x, sum_h * par.y);
                if constexpr (NL > 0) v = fmaf(sl[e >> 2][e & 3], par.z, fmaf(sum_l, par.w, v));
                x[e] = v;
            }
            __builtin_amdgcn_sched_barrier(0);
            if (a.softcap > 0.0f) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = soft_cap(x[e] * a.scale, a.softcap, inv_cap);
            }
            if (!full) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(((mask >> (4 * g)) >> (16 * (e >> 2) + (e & 3))) & 1)) x[e] = -inf;
            }

            // ---- the running maximum and sum ----
            float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            top = rows_max(top) * sc2;
            if (__builtin_amdgcn_ballot_w64(top > m2) != 0) {
                const float m_new = fmaxf(m2, top);
                const float back = m_new == -inf ? 0.0f : __builtin_amdgcn_exp2f(m2 - m_new);
                m2 = m_new;
                l *= back;
                zero_h *= back;
                zero_l *= back;
#pragma unroll
                for (int j = 0; j < HT; ++j) acch[j] *= back;
#pragma unroll
                for (int j = 0; j < NL; ++j) accl[j] *= back;
            }
            const float base = m2 == -inf ? 0.0f : m2;
            float ph[8], pl[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float4 par = *reinterpret_cast<const float4*>(vt + (16 * (e >> 2) + 4 * g + (e & 3)) * P + P - 16);
                const float p = __builtin_amdgcn_exp2f(fmaf(x[e], sc2, -base));
                l += p;
                ph[e] = p * par.x;
                pl[e] = p * par.z;
                zero_h = fmaf(p, par.y, zero_h);
                zero_l = fmaf(p, par.w, zero_l);
            }

            __builtin_amdgcn_sched_barrier(0);
            // ---- weighted sums of the values' codes ----
            auto weights = [&](const float (&p)[8], v4u_att& first, v4u_att& rest) {   // truncation and remainder
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p0 = p[2 * i], p1 = p[2 * i + 1];
                    first[i] = upper_halves(p0, p1);
                    rest[i] = upper_halves(p0 - __uint_as_float(__float_as_uint(p0) & 0xFFFF0000u),
                                           p1 - __uint_as_float(__float_as_uint(p1) & 0xFFFF0000u));
                }
            };
            auto vrow = [&](int e) { return vt + (16 * (e >> 2) + 4 * g + (e & 3)) * P; };
            {
                v4u_att w, w2;
                weights(ph, w, w2);
#pragma unroll
                for (int j = 0; j < HT; ++j) {
                    if (j == 0 || 16 * j < a.r) {
                        v4u_att o;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t c0 = vrow(2 * i)[16 * j + n], c1 = vrow(2 * i + 1)[16 * j + n];
                            o[i] = upper_halves((float)c0, (float)(c1 ^ 255u)) ^ 0x80000000u;
                        }
                        acch[j] = attend_mfma(o, w, acch[j]);
                        acch[j] = attend_mfma(o, w2, acch[j]);
                    }
                }
            }
            if constexpr (NL > 0) {
                v4u_att w, w2;
                weights(pl, w, w2);
                uint32_t c[8][NL < 8 ? 1 : NL / 8];   // a lane's codes of each token
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint8_t* p = vrow(e) + a.r + n * (NL / 2);
                    if constexpr (NL == 4) c[e][0] = *reinterpret_cast<const uint16_t*>(p);
                    else
#pragma unroll
                        for (int k = 0; k < NL / 8; ++k) c[e][k] = reinterpret_cast<const uint32_t*>(p)[k];
                }
#pragma unroll
                for (int k = 0; k < NL / 4; ++k) {   // four channels at a time: half a dword of two tokens in one
                    uint32_t two[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        two[i] = __builtin_amdgcn_perm(~c[2 * i + 1][k >> 1], c[2 * i][k >> 1], k & 1 ? 0x07060302u : 0x05040100u);
                    v4u_att o[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[j][i] = value_bits(two[i] >> (4 * j));
                        accl[4 * k + j] = attend_mfma(o[j], w, accl[4 * k + j]);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) accl[4 * k + j] = attend_mfma(o[j], w2, accl[4 * k + j]);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }

        // ---- the four wavefronts' results together ----
        l = rows_sum(l);
        zero_h = rows_sum(zero_h);
        zero_l = rows_sum(zero_l);
        __syncthreads();   // every wavefront is through with its rows
        const int rows = min(a.share - qt * kAttendRows, kAttendRows);
        float* red = reinterpret_cast<float*>(lds);                           // [wave][rows][d]
        float* ml = reinterpret_cast<float*>(lds + a.lds_red);                // [wave][16][2]
        // (limits of their own: comparisons with the ones above would be made once, for all heads, and kept in too many registers)
        int r_end = a.r, low_end = low;
        asm volatile("" : "+s"(r_end), "+s"(low_end));
        if (n < rows) {
            float* row = red + (wave * rows + n) * a.d;
            if (g == 0) {
                ml[(wave * kAttendRows + n) * 2] = m2;
                ml[(wave * kAttendRows + n) * 2 + 1] = l;
            }
#pragma unroll
            for (int j = 0; j < HT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * j + 4 * g + i < r_end) row[16 * j + 4 * g + i] = acch[j][i] + zero_h;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < NL; ++j)
                    if ((4 * g + i) * NL + j < low_end) row[a.r + (4 * g + i) * NL + j] = accl[j][i] + zero_l;
        }
        __syncthreads();
        // a head in one piece is done; a piece of one is partial result 0 of its workgroup, or 1 behind another head
        const bool whole = n_units == units;
        const int64_t slot = 2 * w0 + (u != u_first);
        if (t == 0) {
            int32_t* join = a.joins + ((int64_t)b * heads + head) * 2;
            if (first_unit == 0) join[0] = (int32_t)slot;
            if (first_unit + n_units == units) join[1] = (int32_t)w0;
        }
        const int pairs = a.d >> 1;
        for (int e = t; e < rows * pairs; e += kAttendThreads) {
            const int row = e / pairs, ch = 2 * (e - row * pairs);
            float top = -inf, sum = 0.0f, o0 = 0.0f, o1 = 0.0f;
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) top = fmaxf(top, ml[(w * kAttendRows + row) * 2]);
            const float base = top == -inf ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(ml[(w * kAttendRows + row) * 2] - base);
                sum = fmaf(f, ml[(w * kAttendRows + row) * 2 + 1], sum);
                o0 = fmaf(f, red[(w * rows + row) * a.d + ch], o0);
                o1 = fmaf(f, red[(w * rows + row) * a.d + ch + 1], o1);
            }
            const int64_t qhead = hk * a.share + qt * kAttendRows + row;
            if (whole) {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                uint16_t* dst = a.out + b * a.ldo + qhead * a.ldoh + ch;
                reinterpret_cast<Piece4*>(dst)->x = pack_bf16_pair(o0 * inv, o1 * inv);
                if (ch == 0 && a.lse)
                    a.lse[(int64_t)b * a.heads_k * a.share + qhead] = sum == 0.0f ? -inf : top * 0.69314718055994530942f + logf(sum);
            } else {
                float* dst = a.part_acc + (slot * a.rows + row) * a.d + ch;
                dst[0] = o0;
                dst[1] = o1;
                if (ch == 0) {
                    a.part_ml[(slot * kAttendRows + row) * 2] = top;
                    a.part_ml[(slot * kAttendRows + row) * 2 + 1] = sum;
                }
            }
        }
        __syncthreads();   // before the rows of the next head come to LDS
        u += n_units;
    }
}

// Joins the partial results of the heads that several workgroups had, one workgroup to a query; and writes the queries of
// sequences without tokens.
__global__ __launch_bounds__(kAttendThreads) void attend_join_kernel(const AttendArgs a) {
    __shared__ float weight[kAttendMaxGrid], part[2 * kAttendWaves];
    __shared__ float4 red[kAttendThreads];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int heads_q = a.heads_k * a.share;
    const int b = blockIdx.x / heads_q, qhead = blockIdx.x - b * heads_q;
    const int hk = qhead / a.share, qi = qhead - hk * a.share, qt = qi / kAttendRows, row = qi - qt * kAttendRows;
    const int32_t* join = a.joins + ((int64_t)b * a.heads_k * a.qtiles + hk * a.qtiles + qt) * 2;
    const int slot0 = join[0], w_last = join[1];   // (nobody wrote them for a sequence without tokens)
    uint16_t* dst = a.out + b * a.ldo + qhead * a.ldoh;
    const float inf = __builtin_huge_valf();
    if (attend_len(a, b) == 0) {
        for (int c = t; c < a.d; c += kAttendThreads) dst[c] = 0;
        if (t == 0 && a.lse) a.lse[blockIdx.x] = -inf;
        return;
    }
    const int w_first = slot0 >> 1, count = w_last - w_first + 1;
    if (count == 1) return;
    auto slot = [&](int i) { return (int64_t)(i == 0 ? slot0 : 2 * (w_first + i)); };
    float top = -inf;
    for (int i = t; i < count; i += kAttendThreads) {
        weight[i] = a.part_ml[(slot(i) * kAttendRows + row) * 2];
        top = fmaxf(top, weight[i]);
    }
    top = wave_max(top);
    if (lane == 0) part[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    const float base = top == -inf ? 0.0f : top;
    float sum = 0.0f;
    for (int i = t; i < count; i += kAttendThreads) {
        const float f = __builtin_amdgcn_exp2f(weight[i] - base);
        weight[i] = f;
        sum = fmaf(f, a.part_ml[(slot(i) * kAttendRows + row) * 2 + 1], sum);
    }
    for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
    if (lane == 0) part[kAttendWaves + wave] = sum;
    __syncthreads();
    sum = (part[kAttendWaves] + part[kAttendWaves + 1]) + (part[kAttendWaves + 2] + part[kAttendWaves + 3]);
    // four channels to a thread, what threads are left over the partial results, four of which are on their way at a time
    const int fours = a.d >> 2, groups = kAttendThreads / fours, group = t / fours, ch = 4 * (t - group * fours);
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (group < groups) {
        for (int i = group; i < count; i += 4 * groups) {
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int j = min(i + k * groups, count - 1);
                v[k] = *reinterpret_cast<const float4*>(a.part_acc + (slot(j) * a.rows + row) * a.d + ch);
            }
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
        const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
        Piece8 p{pack_bf16_pair(o.x * f, o.y * f), pack_bf16_pair(o.z * f, o.w * f)};
        *reinterpret_cast<Piece8*>(dst + 4 * t) = p;
        if (t == 0 && a.lse) a.lse[blockIdx.x] = sum == 0.0f ? -inf : top * 0.69314718055994530942f + logf(sum);
    }
}

}  // namespace resq
