// Attention of one new token of each sequence over a prefix that all sequences of the batch share, in pages of compact K/V rows
// (resq_kv_row.hip.h): for each K/V head the queries of all sequences are rows of one product, so that the prefix is read and made into
// numbers once for 256 of them and not once for each sequence.  The sequences' own tokens are resq_attend.hip.h's; a last kernel joins both.
//   k_t = code * s + z of each group, x = scale * q . k_t, capped or not; out = sum e^(x - lse) v, as there
//
// A workgroup makes a tile of 64 rows (of 32 for heads above 128: what LDS and registers hold) into fp16 numbers in LDS and has 256 queries
// attend to it (resq_flash.hip.h), in two groups of wavefronts half a tile apart as the prompts' kernel has them; the first makes the keys
// of the tile behind, the second the values, each in its turn at the vector ALU.  A value is rounded to fp16, half a step 2^-11 of itself,
// an eighth of what bf16 loses, which would add as much again to the error of a bf16 result.  A key is two such numbers, itself and
// what its rounding left out, 2^-22 of it: with one the log-sum-exp, an fp32 result, was off by up to 10^-3 of itself.  (The products that
// this takes more, a third of all, are made while the vector ALU is at work; what making them costs there is 464 -> 525 us of the largest
// case below.)  fp16's range is made up for by powers of two: of a query (its largest channel becomes 2^13), of a wavefront's keys of a
// tile, and of the values of all tokens so far.  What is below 2^-27 of the largest number there loses bits, down to 2^-38 of it.
//
// What bounds it is the vector ALU: 600 instructions of a wavefront to a tile, more than half of them from codes to numbers, of which a turn
// is made of some 4200 cycles (of values) to 4800 (of keys); the matrix cores' turn takes 2100, 1536 of them products.  Measured on MI355X (all four kernels of a
// call, the own tokens' attention and the joins beside this one): 200 queries of 64 heads over 30001 tokens, 8 K/V heads of 128: 508 us,
// 390 TFLOP/s (capped 637); 64 of 32 heads over 8192 62 us, 31 of them here; 4 over 1000 27 us, 13 here, the latency of page, row and result; 64 of 16 heads on 8 over
// 8192, heads of 192 70 us, of 256, for which registers do not suffice, 171.  On the way, at
// 200 queries: loads in branches, each of which waited for all before it, 842 us; without 732; places of a piece made anew in place of kept in
// scratch memory 577; factors of the keys in the softmax's own multiplications 464; keys in two numbers 525, the join by a wavefront to a query 507.  Loads made in the other
// turn, at the matrix cores, where there is time: 468 for 464, they come too late then.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "resq_flash.hip.h"

namespace resq {

constexpr int kPrefixThreads = 512;
constexpr int kPrefixWaves = kPrefixThreads / 64;
constexpr int kPrefixJoinSmall = 64, kPrefixJoinLarge = 256;
constexpr int kPrefixRows = kFlashRows * kPrefixWaves;   // of a workgroup
__host__ __device__ constexpr int prefix_keys_of(int d) { return d <= 128 ? 64 : 32; }   // of a tile: what registers and LDS hold
constexpr int kPrefixLeast = 2;                          // tiles of a part at least

struct PrefixArgs {
    const uint16_t* q;
    int64_t ldq, ldqh;
    int B, heads_k, d, r, row_bytes;
    FastDiv share, parts, heads;
    const int32_t* prefix_len;
    const int32_t* prefix_table;
    int max_prefix;        // tokens that the prefix's table can name
    const int32_t* lens;   // own tokens of each sequence, below 0: the sequence is not there
    int max_own;           // that a sequence's table can name
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
    float* part_ml;        // [tile, head, part][256][2]: maximum (times log2 e) and sum (workspace)
    float* part_acc;       // [tile, head, part][256][d]: weighted sums (workspace)
};

// The tokens of the prefix that some row may see, [begin, end) with begin a multiple of a tile, and the parts they are cut into.
struct PrefixKeys {
    int begin, end, per, parts;
};
__device__ __forceinline__ PrefixKeys prefix_keys(const PrefixArgs& a) {
    PrefixKeys k;
    const int tile = prefix_keys_of(a.d);
    k.end = min(max(a.prefix_len[0], 0), a.max_prefix);
    k.begin = max(k.end - a.window, 0) & -tile;   // (own tokens leave fewer)
    const int tiles = (k.end - k.begin + tile - 1) / tile;
    const int parts = min((int)a.parts.d, max(tiles / kPrefixLeast, 1));
    k.per = (tiles + parts - 1) / parts;
    k.parts = k.per ? (tiles + k.per - 1) / k.per : 0;
    return k;
}

// 2^e of exponent bits e, and 2^13 over it, which makes numbers below 2^(e + 1) ones below 2^14
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)e << 23); }
__device__ __forceinline__ int exponent_of(float x) { return max((int)(__float_as_uint(x) >> 23), 27); }   // x >= 0; bits, 127 is 2^0
__device__ __forceinline__ float to_half_range(int e) { return two_to(267 - e); }

template <int W, bool CAP>
__global__ __launch_bounds__(kPrefixThreads, 2) void attend_prefix_kernel(const PrefixArgs a) {
    using Tile = FlashTile<W>;
    constexpr int KEYS = prefix_keys_of(W), kTileBytes = KEYS * Tile::kPitch;
    constexpr int kGroups = kPrefixWaves / 2, kGroup = KEYS / kGroups;   // tokens of a wavefront
    constexpr int kLanes = kPrefixThreads / 2 / KEYS;   // threads of a token's keys (values)
    constexpr int kUnits = Tile::kPieces / kLanes;      // pieces of 8 channels of a thread
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // two tiles of keys, two of values, two of what the keys' rounding left out
    // of each wavefront's tokens of a tile: the exponent of keys (values), which tokens there are, and which of them have an 8-bit (4-bit)
    // group of values that is not finite
    typedef typename std::conditional<kGroup == 16, uint16_t, uint8_t>::type Bits;
    struct alignas(16) About {
        uint8_t e[kGroups];
        Bits there[kGroups], odd_high[kGroups], odd_low[kGroups];
    };
    constexpr int kAbout = sizeof(About) / 4, kWords = KEYS / 32;
    static_assert(kGroups == 4 && kGroup * kGroups == KEYS && (kAbout == 4 || kAbout == 8));
    __shared__ About about[2][2];   // [buffer][keys or values]

    const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6), group = wave >> 2;   // what it makes: 0 keys, 1 values
    const int unit = (int)a.heads(blockIdx.x), hk = (int)blockIdx.x - unit * a.heads_k;
    const int tile = (int)a.parts(unit), piece = unit - tile * (int)a.parts.d;
    const PrefixKeys keys = prefix_keys(a);
    if (piece >= keys.parts) return;
    const int begin = keys.begin + piece * keys.per * KEYS, end = min(keys.end, begin + keys.per * KEYS);
    const int n_all = (end - begin + KEYS - 1) / KEYS;
    const float inf = __builtin_huge_valf();

    // ---- rows of a tile: read two tiles ahead, made into numbers one ahead ----
    const int my_token = kGroup * (wave & 3) + lane % kGroup, my_unit = lane / kGroup;
    const uint8_t* pages = a.pages[group] + hk * a.head_stride;
    int page_next = -1;
    bool there = false;
    uint2 code[kUnits];
    float par[4];
    auto load_page = [&](int n) __attribute__((always_inline)) {
        const int tok = begin + n * KEYS + my_token;
        page_next = -1;
        if (tok < end) page_next = a.prefix_table[a.page_size((uint32_t)tok)];
    };
    // (a token that is not there: the first row of the first page in its place, of which nothing is used.  No branches: a load behind
    // one would wait for the loads in front of it.)
    auto load = [&](int n) __attribute__((always_inline)) {
        const int tok = begin + n * KEYS + my_token;
        there = (unsigned)page_next < (unsigned)a.num_pages;
        const int64_t off = page_next * a.page_stride + (tok - (int)a.page_size((uint32_t)tok) * (int)a.page_size.d) * a.row_stride;
        const uint8_t* src = pages + (there ? off : 0);
        const Piece16 p = *reinterpret_cast<const Piece16*>(src + a.row_bytes - 16);
        par[0] = __uint_as_float(p.x);
        par[1] = __uint_as_float(p.y);
        par[2] = __uint_as_float(p.z);
        par[3] = __uint_as_float(p.w);
        int unit0 = my_unit;
        asm volatile("" : "+v"(unit0));   // made anew here: kept over the products, the offsets would go to scratch memory
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            // a piece of the 8-bit group, eight bytes, of the 4-bit one, four, or of both, four and two, which follow each other (behind the
            // head: any); ch >= r where (ch + r) / 2 <= ch
            const int ch = 8 * (unit0 + u * kLanes);
            const Piece8 c = *reinterpret_cast<const Piece8*>(src + min(min(ch, (ch + a.r) >> 1), a.row_bytes - 8));
            code[u] = make_uint2(c.x, c.y);
        }
    };
    // least: the exponent that values are counted in so far
    auto store_of = [&](auto values, int n, int least) __attribute__((always_inline)) {
        constexpr int group = decltype(values)::value;
        // (the pieces' order in a row is by exclusive or: piece my_unit + kLanes u stands where piece my_unit stands, but for u)
        uint32_t at = (2 * group + (n & 1)) * kTileBytes + (group ? Tile::value_at(my_token, my_unit) : Tile::key_at(my_token, my_unit));
        int unit0 = my_unit;
        asm volatile("" : "+v"(at), "+v"(unit0));
        // (what a row holds as the numbers of a group without channels is nothing)
#pragma unroll
        for (int i = 0; i < 4; ++i) par[i] = there && (i < 2 ? a.r > 0 : a.r < a.d) ? par[i] : 0.0f;
        float high = 0.0f, low = 0.0f;   // the groups' largest magnitudes
        if (a.r > 0) high = fmaxf(fabsf(par[1]), fabsf(fmaf(255.0f, par[0], par[1])));
        if (a.r < a.d) low = fmaxf(fabsf(par[3]), fabsf(fmaf(15.0f, par[2], par[3])));
        // (of numbers that are not finite keys keep what they have, values are left out: `odd` below)
        const bool odd_high = !(fabsf(par[0]) + fabsf(par[1]) < inf), odd_low = !(fabsf(par[2]) + fabsf(par[3]) < inf);
        const float top = fmaxf(odd_high || !(high < inf) ? 0.0f : high, odd_low || !(low < inf) ? 0.0f : low);
        int e = exponent_of(rows_max(row_max16(top)));
        if (group) e = max(e, least);
        const float f = to_half_range(e);
        const float fh = group && odd_high ? 0.0f : f, fl = group && odd_low ? 0.0f : f;
        const float sh = fh == 0.0f ? 0.0f : par[0] * fh, zh = fh == 0.0f ? 0.0f : par[1] * fh;
        const float sl = fl == 0.0f ? 0.0f : par[2] * fl, zl = fl == 0.0f ? 0.0f : par[3] * fl;
        auto number = [](uint32_t codes, int i) __attribute__((always_inline)) { return (float)(codes >> (8 * i) & 255u); };
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const uint2 c = code[u];
            const int ch0 = 8 * kLanes * u;
            v4u_flash o, rest;   // numbers, and what their rounding leaves out
            auto two = [&](float v0, float v1) __attribute__((always_inline)) {
                const uint32_t bits = flash_pack<true>(v0, v1);
                if constexpr (group != 0) return make_uint2(bits, 0u);
                const v2h_flash h = __builtin_bit_cast(v2h_flash, bits);
                return make_uint2(bits, flash_pack<true>(fmaf((float)h[0], -1.0f, v0), fmaf((float)h[1], -1.0f, v1)));
            };
            auto put = [&](uint2 a0, uint2 a1, uint2 a2, uint2 a3) __attribute__((always_inline)) {
                o = (v4u_flash){a0.x, a1.x, a2.x, a3.x};
                rest = (v4u_flash){a0.y, a1.y, a2.y, a3.y};
            };
            auto low = [&]() __attribute__((always_inline)) {
                const uint32_t even = c.x & 0x0F0F0F0Fu, odd = c.x >> 4 & 0x0F0F0F0Fu;
                auto pair = [&](int i) __attribute__((always_inline)) { return two(fmaf(number(even, i), sl, zl), fmaf(number(odd, i), sl, zl)); };
                put(pair(0), pair(1), pair(2), pair(3));
            };
            if (ch0 >= a.r) {   // (the same for all)
                low();
            } else {
                const int ch = 8 * unit0 + ch0;
                if (ch >= a.r) {
                    low();
                } else {
                    const bool mixed = ch + 8 > a.r;
                    const uint32_t second = mixed ? (c.y & 0xFu) | (c.y & 0xF0u) << 4 | (c.y & 0xF00u) << 8 | (c.y & 0xF000u) << 12 : c.y;
                    const float s2 = mixed ? sl : sh, z2 = mixed ? zl : zh;
                    auto pair = [&](uint32_t codes, int i, float s, float z) __attribute__((always_inline)) {
                        return two(fmaf(number(codes, i), s, z), fmaf(number(codes, i + 1), s, z));
                    };
                    put(pair(c.x, 0, sh, zh), pair(c.x, 2, sh, zh), pair(second, 0, s2, z2), pair(second, 2, s2, z2));
                }
            }
            *reinterpret_cast<v4u_flash*>(lds + (at ^ 16 * kLanes * u)) = o;
            if constexpr (group == 0) {
                const bool nothing = odd_high || odd_low;   // (an infinity less itself)
                rest = (v4u_flash){nothing ? 0u : rest[0], nothing ? 0u : rest[1], nothing ? 0u : rest[2], nothing ? 0u : rest[3]};
                *reinterpret_cast<v4u_flash*>(lds + 4 * kTileBytes + (at ^ 16 * kLanes * u)) = rest;
            }
        }
        // the first lanes speak for the tokens
        const int some = (int)(__builtin_amdgcn_ballot_w64(there) & ((1 << kGroup) - 1)), high_bits = (int)(__builtin_amdgcn_ballot_w64(odd_high) & ((1 << kGroup) - 1));
        const int low_bits = (int)(__builtin_amdgcn_ballot_w64(odd_low) & ((1 << kGroup) - 1));
        if (lane == 0) {
            About& of = about[n & 1][group];
            of.e[wave & 3] = (uint8_t)e;
            of.there[wave & 3] = (Bits)some;
            of.odd_high[wave & 3] = (Bits)high_bits;
            of.odd_low[wave & 3] = (Bits)low_bits;
        }
    };
    auto store = [&](int n, int least) __attribute__((always_inline)) {   // (one branch, the same for a wavefront)
        if (group) store_of(std::integral_constant<int, 1>(), n, least);
        else store_of(std::integral_constant<int, 0>(), n, least);
    };
    static_assert(kLanes * kGroup == 64 && (kLanes & (kLanes - 1)) == 0);
    load_page(0);
    load(0);
    load_page(1);
    store(0, 27);
    load(1);
    load_page(2);

    // ---- the own row ----
    const int rows = a.B * (int)a.share.d, row = tile * kPrefixRows + wave * kFlashRows + (lane & 31);
    const bool live = row < rows;
    const int b = (int)a.share(live ? row : 0), head = hk * (int)a.share.d + (live ? row : 0) - b * (int)a.share.d;
    const int own = min(a.lens[b], a.max_own);
    // the first token that the row sees, own tokens count for the window too (a row that is not there sees all: nothing comes of it)
    const int from = live && own >= 0 ? (int)max((int64_t)keys.end + own - a.window, (int64_t)0) : 0;
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
        top = halves_max(top);
        const int e = exponent_of(top < inf ? top : 0.0f);
        const float f = to_half_range(e);
#pragma unroll
        for (int s = 0; s < Tile::kSteps; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r.q[s][i] = flash_pack<true>(__uint_as_float(r.q[s][i] << 16) * f, __uint_as_float(r.q[s][i] & 0xFFFF0000u) * f);
        qf = a.scale * two_to(e - 13) * 1.44269504088896340736f;
    }
    const FlashCap<false> cap(CAP ? a.softcap : 1.0f, 1.0f);

    constexpr int kAhead = W <= 128 && !CAP ? 2 : 0;   // (capped scores need the registers)
    FlashTurn<W, KEYS, kAhead> s;
    int value_e = 27;        // the exponent of the values that are weighed, and of all before
    uint32_t odd = 0;        // bit 0 (1): a value of the 8-bit (4-bit) group that the row sees is not finite
    auto keys_in = [&](int n) { return lds + (n & 1) * kTileBytes; };
    auto values_in = [&](int n) { return lds + (2 + (n & 1)) * kTileBytes; };
    auto turn = [&](int n) __attribute__((always_inline)) {
        flash_after_products();
        const uint32_t word = reinterpret_cast<const uint32_t*>(about[n & 1])[lane & (2 * kAbout - 1)];   // all of both
        r.ask_ahead(s, values_in(n));
        // ---- what this tile is counted in ----
        auto read = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane((int)word, i); };
        const uint32_t ke = read(0), ve_all = read(kAbout);
        uint32_t seen[kWords], high[kWords], low[kWords], missing = 0, odd_here = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            seen[i] = read(1 + i);
            high[i] = read(kAbout + 1 + kWords + i);
            low[i] = read(kAbout + 1 + 2 * kWords + i);
            missing |= ~seen[i];
            odd_here |= high[i] | low[i];
        }
        float unit[kGroups], up[kGroups];
        int ve[kGroups], e_new = value_e;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            unit[g] = fmaxf(qf * two_to((int)(ke >> (8 * g) & 255u) - 13), 1.17549435e-38f);   // (not 0, which would make a NaN of -inf)
            ve[g] = (int)(ve_all >> (8 * g) & 255u);
            e_new = max(e_new, ve[g]);
        }
        bool scaled = false;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            up[g] = two_to(max(127 + ve[g] - e_new, 0));
            scaled |= ve[g] != e_new;
        }
        if (e_new != value_e) {
            const float back = two_to(max(127 + value_e - e_new, 0));
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) r.acc[c] *= back;
            value_e = e_new;
        }
        // ---- keys that are not there, or behind the row's window ----
        const int key0 = begin + n * KEYS, behind = from - key0;
        if (missing != 0 || __builtin_amdgcn_ballot_w64(behind > 0) != 0) {
            uint32_t sees[kWords];   // the row's keys of both halves
#pragma unroll
            for (int kb = 0; kb < kWords; ++kb) {
                const int gone = min(max(behind - 32 * kb, 0), 32);
                sees[kb] = seen[kb] & (gone == 32 ? 0u : 0xFFFFFFFFu << gone);
                odd |= ((sees[kb] & high[kb]) != 0 ? 1u : 0u) | ((sees[kb] & low[kb]) != 0 ? 2u : 0u);
                sees[kb] >>= 4 * half;
            }
            r.mask(s, [&](int c) { return (sees[c >> 5] >> (c & 31) & 1) != 0; });
        } else if (odd_here != 0) {
#pragma unroll
            for (int kb = 0; kb < kWords; ++kb) odd |= (high[kb] != 0 ? 1u : 0u) | (low[kb] != 0 ? 2u : 0u);
        }
        r.template softmax<KEYS, CAP, true>(s, unit, cap);
        if (scaled) {
#pragma unroll
            for (int g = 0; g < KEYS / 16; ++g) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t bits = s.p[g][e];
                    const v2h_flash two = __builtin_bit_cast(v2h_flash, bits);
                    const float f = up[(8 * g + 2 * e) / (KEYS / 2 / kGroups)];
                    s.p[g][e] = flash_pack<true>((float)two[0] * f, (float)two[1] * f);
                }
            }
        }
        // ---- the tile behind ----
        if (n + 1 < n_all) {
            store(n + 1, value_e);
            if (n + 2 < n_all) {
                load(n + 2);
                load_page(n + 3);
            }
        }
        flash_after_making();
    };

    flash_landed();
    if (group) flash_after_products();
    r.template products<KEYS, false, true>(s, keys_in(0), nullptr, 4 * kTileBytes);
    turn(0);
    for (int n = 1; n < n_all; ++n) {
        r.template products<KEYS, true, true>(s, keys_in(n), values_in(n - 1), 4 * kTileBytes);
        turn(n);
    }
    r.weigh_rest(s, values_in(n_all - 1));
    if (!group) flash_after_products();

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
            const int ch = 32 * c + 8 * (i >> 2) + 4 * half;   // four channels of one group
            const bool nan = (odd & (ch < a.r ? 1u : 2u)) != 0;
            const float w = nan ? __builtin_nanf("") : f;
            if (ch < a.d)
                *reinterpret_cast<float4*>(dst + ch) = make_float4(r.acc[c][i] * w, r.acc[c][i + 1] * w, r.acc[c][i + 2] * w, r.acc[c][i + 3] * w);
        }
    if (half == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * kPrefixRows + at) * 2) = make_float2(r.m, sum);
}

// Joins the parts of the prefix and the own tokens' result, whose maximum is its log-sum-exp and whose sum is 1: a workgroup to a query,
// four channels to a thread, what threads are left over the parts.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void attend_prefix_join_kernel(const PrefixArgs a) {
    __shared__ float weight[THREADS + 1], sums[THREADS + 1], top_of[THREADS / 64];
    __shared__ float4 red[THREADS];
    const int t = threadIdx.x, fours = a.d >> 2, heads_q = a.heads_k * (int)a.share.d;
    const int b = (int)(blockIdx.x / (uint32_t)heads_q), head = (int)(blockIdx.x - (uint32_t)b * heads_q);
    const int hk = (int)a.share(head), row = b * (int)a.share.d + head - hk * (int)a.share.d;
    const int parts = prefix_keys(a).parts;   // at most THREADS
    const float inf = __builtin_huge_valf();
    uint16_t* out = a.out + b * a.ldo + head * a.ldoh;
    if (a.lens[b] < 0) {
        if (t < fours) *reinterpret_cast<Piece8*>(out + 4 * t) = Piece8{0u, 0u};
        if (t == 0 && a.lse) a.lse[blockIdx.x] = -inf;
        return;
    }
    const int64_t slot = ((int64_t)(row / kPrefixRows) * a.heads_k + hk) * a.parts.d;
    const float* ml = a.part_ml + (slot * kPrefixRows + row % kPrefixRows) * 2;
    const float* acc = a.part_acc + (slot * kPrefixRows + row % kPrefixRows) * a.d;
    // weight i < parts: a part's; weight `parts`: the own tokens'
    float2 mine = make_float2(kFlashNone, 0.0f);
    if (t < parts) mine = *reinterpret_cast<const float2*>(ml + (int64_t)t * kPrefixRows * 2);
    float own = a.own_lse[blockIdx.x] * 1.44269504088896340736f;
    const float own_sum = own == -inf ? 0.0f : 1.0f;
    if (own == -inf) own = kFlashNone;
    float top = rows_max(row_max16(mine.x));
    if ((t & 63) == 0) top_of[t >> 6] = top;
    __syncthreads();
    top = own;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) top = fmaxf(top, top_of[w]);
    const float f = __builtin_amdgcn_exp2f(mine.x - top), f_own = __builtin_amdgcn_exp2f(own - top);
    if (t < parts) {
        weight[t] = f;
        sums[t] = f == 0.0f && mine.y == mine.y ? 0.0f : f * mine.y;   // (of a part whose keys the row does not see, or that weigh nothing)
    }
    if (t == 0) {
        weight[parts] = own_sum == 0.0f ? 0.0f : f_own;
        sums[parts] = own_sum == 0.0f ? 0.0f : f_own;
    }
    __syncthreads();
    const int groups = THREADS / fours, group = t / fours, ch = 4 * (t - group * fours);
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add = [&](float w, const float4& v) {   // (of weight 0 too: a part whose tokens weigh nothing may have NaN, which stays)
        o.x = fmaf(w, v.x, o.x);
        o.y = fmaf(w, v.y, o.y);
        o.z = fmaf(w, v.z, o.z);
        o.w = fmaf(w, v.w, o.w);
    };
    if (group < groups) {
        for (int i = group; i < parts; i += 4 * groups) {
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const float4*>(acc + (int64_t)min(i + k * groups, parts - 1) * kPrefixRows * a.d + ch);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k * groups < parts) add(weight[i + k * groups], v[k]);
        }
        if (group == 0) add(weight[parts], *reinterpret_cast<const float4*>(a.own_out + (int64_t)blockIdx.x * a.d + ch));
    }
    red[t] = o;
    __syncthreads();
    if (t >= fours) return;
    for (int k = 1; k < groups; ++k) {
        const float4 v = red[k * fours + t];
        o.x += v.x;
        o.y += v.y;
        o.z += v.z;
        o.w += v.w;
    }
    float sum = 0.0f;
    for (int i = 0; i <= parts; ++i) sum += sums[i];
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *reinterpret_cast<Piece8*>(out + 4 * t) = Piece8{pack_bf16_pair(o.x * inv, o.y * inv), pack_bf16_pair(o.z * inv, o.w * inv)};
    if (t == 0 && a.lse) a.lse[blockIdx.x] = sum == 0.0f ? -inf : top * 0.69314718055994530942f + logf(sum);
}

}  // namespace resq
