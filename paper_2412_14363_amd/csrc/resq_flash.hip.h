// Attention of many rows of queries over tiles of keys and values, one pass with the running maximum and sum of the softmax: what the
// kernels for whole prompts and for shared prefixes have in common.
//
// A wavefront has 32 rows (queries of one K/V head).  Its scores are taken transposed, S^T (keys x rows) = K x Q^T, on the 32x32x16
// matrix cores: a lane then has one row, l % 32, and of 32 keys the sixteen 8 (i / 4) + 4 (l / 32) + i % 4, so that a row's maximum and
// sum stay in its two lanes and factors of a row are a lane's own.  The weights are the other product's operand as they lie,
//   O^T (channels x rows) += V^T x P^T,
// if that product counts its keys as the lanes have them: lane half h's eight of a step t are 16 t + 4 h + 0..3 and 8 more, which is
// how the values are read, with the transposing LDS read that gives a lane four keys of one channel.
//
// LDS: rows of a power of two of 16-byte pieces.  A key's piece c is at c ^ (row % 16): sixteen rows of one piece, what a read of K takes
// at a time, lie on all banks.  A value's is at c ^ 4 (row % 4): a read of V takes 64 bytes of four rows at a time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_lanes.hip.h"
#include "resq_layout.h"

namespace resq {

constexpr int kFlashRows = 32;          // of a wavefront
constexpr float kFlashNone = -3.0e38f;  // the maximum of no scores: finite, so that differences stay numbers
// weights in fp16 are 2^10 times what they are: those down to 2^-24 of the largest one keep all their bits, and 2^-35 is the smallest
constexpr float kFlashHalfBias = 10.0f;
// by how many powers of two a score may be over the running maximum before that rises (in fp16 weights stay below 2^15)
constexpr float kFlashSlack = 8.0f, kFlashHalfSlack = 5.0f;

typedef float v16f_flash __attribute__((ext_vector_type(16)));
typedef uint32_t v4u_flash __attribute__((ext_vector_type(4)));
typedef uint32_t v2u_flash __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf_flash __attribute__((ext_vector_type(8)));
typedef _Float16 v8h_flash __attribute__((ext_vector_type(8)));
typedef _Float16 v2h_flash __attribute__((ext_vector_type(2)));
typedef float v2f_flash __attribute__((ext_vector_type(2)));
typedef short v4s_flash __attribute__((ext_vector_type(4)));

// c (32 x 32) += a (rows of the result) x b (its columns), 16 steps, operands in bf16 or fp16
template <bool F16>
__device__ __forceinline__ v16f_flash flash_mfma(const v4u_flash& a, const v4u_flash& b, const v16f_flash& c) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h_flash, a), __builtin_bit_cast(v8h_flash, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf_flash, a), __builtin_bit_cast(v8bf_flash, b), c, 0, 0, 0);
}
template <bool F16>
__device__ __forceinline__ uint32_t flash_pack(float lo, float hi) {   // rounded to nearest even
    if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f_flash){lo, hi}, v2h_flash));
    else return pack_bf16_pair(lo, hi);
}
#define FlashLds __attribute__((address_space(3)))
__device__ __forceinline__ uint32_t flash_lds(const uint8_t* p) { return (uint32_t)(uintptr_t)(const FlashLds uint8_t*)p; }
__device__ __forceinline__ v2u_flash flash_read_tr(FlashLds uint8_t* p) {
    return __builtin_bit_cast(v2u_flash, __builtin_amdgcn_ds_read_tr16_b64_v4i16((FlashLds v4s_flash*)p));
}

// 16 bytes of each lane from base + off to lds + 16 lane in LDS, on their way past the compiler: it would have every later read of LDS wait
// for them.  flash_landed() is the wait, and the workgroup's meeting behind it.
__device__ __forceinline__ void flash_fetch(uint32_t lds, const uint8_t* base, uint32_t off) {
    // (both are the wavefront's, which the compiler loses sight of where many registers are taken)
    lds = __builtin_amdgcn_readfirstlane(lds);
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    base = reinterpret_cast<const uint8_t*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 |
                                            (uint32_t)__builtin_amdgcn_readfirstlane((int)at));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void flash_landed() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Ends of a wavefront's turn at the matrix cores (it has read all that it needed of the keys, and of the values before), and of its turn
// at the vector ALU (what it has fetched but the last LATER moves is there).
__device__ __forceinline__ void flash_after_products() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_setprio 0\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void flash_after_making() {   // ... where it writes to LDS itself
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_setprio 3\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
template <int LATER>
__device__ __forceinline__ void flash_after_softmax() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_setprio 3\n\ts_barrier" ::"n"(LATER) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A capped score in base 2: B tanh(y / B) = y f(t), t = (y / B)^2, B = cap log2 e, off by a few roundings of itself (2^-19.9 at most) however
// large the cap is, where 1 - 2 / (1 + e^(2 y / B)) would be off by 2^-21 of the cap.  f is P / Q, fitted for the least relative error up to
// |y| = 8.7 B, from where on y f is B to fp32 (2^-25.9; all terms are positive, so that nothing cancels), or where a wavefront's scores of
// a tile are all within 0.33 B, as scores below a cap mostly are, a polynomial (2^-25.2).  Measured on MI355X: 24 ragged prompts of heads of 64
// 185 us, 259 by P / Q everywhere, 177 by the exponential and its reciprocal; 8192 tokens, heads of 128, 662 with all scores within 0.33 B, 885 with
// larger ones in every tile, 666 by the exponential.
// UNIT: of products that make y = unit x, one unit for all, which is then in the numerators; else of y itself.
template <bool UNIT>
struct FlashCap {
    float unit, most, small, inv;   // 8.7 B, 0.33 B and 1 / B, for UNIT of x, in scalar registers
    __device__ __forceinline__ FlashCap(float cap, float unit_) : unit(scalar(unit_)) {
        inv = 0.69314718055994530942f / cap;
        if constexpr (UNIT) {
            inv = fminf(inv * unit, 3.4028235e38f);
            cap /= unit;
        }
        most = scalar(fminf(12.5514472f * cap, 3.4028235e38f));
        small = scalar(0.47608936f * cap);
        inv = scalar(inv);
    }
    __device__ static __forceinline__ float scalar(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
    // A constant in a vector register from here on: kept over a loop it would take another's place, which goes to scratch memory, and reads of
    // that wait for tiles on their way to LDS (a few of them there: 8192 tokens, heads of 128, 1016 us for 688; 200 queries over 30001 tokens 723 for 658).
    __device__ static __forceinline__ float here(float x) {
        asm volatile("" : "+v"(x));
        return x;
    }
    __device__ __forceinline__ float of(float c) const { return UNIT ? scalar(unit * c) : c; }
    __device__ __forceinline__ float small_factor(float y, float c2) const {   // c2: here(of(kSmall2))
        const float u = y * inv, t = u * u;
        return fmaf(fmaf(fmaf(of(-0.04965299f), t, c2), t, of(-0.333328575f)), t, of(1.0f));
    }
    // y within +-most (which makes a number of NaN)
    __device__ __forceinline__ float within(float y) const { return __builtin_amdgcn_fmed3f(y, -most, most); }
    __device__ __forceinline__ float factor(float y, float p3, float q3) const {   // here(of(kP3)), here(kQ3)
        const float u = y * inv, t = u * u;
        const float p = fmaf(fmaf(fmaf(fmaf(of(1.39620733e-8f), t, p3), t, of(3.52193834e-3f)), t, of(0.134032145f)), t, of(1.0f));
        const float q = fmaf(fmaf(fmaf(fmaf(8.02389081e-7f, t, q3), t, 2.59772241e-2f), t, 0.467365384f), t, 1.0f);
        return p * __builtin_amdgcn_rcpf(q);
    }
    __device__ __forceinline__ float operator()(float y) const {
        const float x = within(y);
        return x * factor(x, of(kP3), kQ3);
    }
    static constexpr float kSmall2 = 0.133066013f, kP3 = 2.10437538e-5f, kQ3 = 3.32875614e-4f;
};

// Layout of a tile: W channels (a multiple of 32) in rows of a power of two of pieces.
template <int W>
struct FlashTile {
    static constexpr int kPieces = W <= 64 ? 8 : W <= 128 ? 16 : 32;
    static constexpr int kPitch = 16 * kPieces;
    static constexpr int kSteps = W / 16;    // of the first product
    static constexpr int kBlocks = W / 32;   // tiles of channels of the second one
    // (rows of 128 bytes: two of them make up the banks)
    __device__ static __forceinline__ int key_at(int row, int piece) {
        return row * kPitch + 16 * (piece ^ (kPieces == 8 ? (row >> 1) & 7 : row & 15));
    }
    __device__ static __forceinline__ int value_at(int row, int piece) {
        return row * kPitch + 16 * (piece ^ (kPieces == 8 ? 4 * ((row >> 1) & 1) : 4 * (row & 3)));
    }
};

// What goes from one turn of a wavefront to the next: scores and weights of the tile at hand, and its values, which are asked for in front of
// the softmax where registers allow it.
template <int W, int KEYS, int AHEAD>   // AHEAD: sixteens of keys whose values are asked for in front of the softmax
struct FlashTurn {
    static constexpr int kAhead = AHEAD;
    v16f_flash x[KEYS / 32];
    v4u_flash p[KEYS / 16];
    v4u_flash v[kAhead ? kAhead : 1][FlashTile<W>::kBlocks];
};

// A lane's row: its query as the first product's operand, its running maximum (times log2 e) and sum (over the lane's own keys), and
// its weighted sums of values.
template <int W, bool F16>
struct FlashRow {
    using Tile = FlashTile<W>;
    v4u_flash q[Tile::kSteps];
    v16f_flash acc[Tile::kBlocks];
    float m, l;

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int c = 0; c < Tile::kBlocks; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[c][i] = 0.0f;
        m = kFlashNone;
        l = 0.0f;
    }
    // keys [32 kb, 32 kb + 32) of a tile, channels 16 t .. 16 t + 15, as the first product's operand.  (A piece's number is in the lower bits of
    // its place, so that what t does to the address is one exclusive or.)
    __device__ __forceinline__ v4u_flash keys(const uint8_t* kt, int kb, int t) const {
        const int lane = threadIdx.x & 63;
        const uint32_t at = ((uint32_t)Tile::key_at(lane & 31, lane >> 5) ^ (32u * t)) + flash_lds(kt);
        return *reinterpret_cast<const FlashLds v4u_flash*>(reinterpret_cast<const FlashLds uint8_t*>((uintptr_t)at) + 32 * kb * Tile::kPitch);
    }
    // values of keys 16 t .. 16 t + 15 and channels [32 c, 32 c + 32), as the second product's operand
    __device__ __forceinline__ v4u_flash values(const uint8_t* vals, int t, int c) const {
        const int lane = threadIdx.x & 63;
        const int row = 4 * (lane >> 5) + ((lane >> 2) & 3), piece = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        const uint32_t at = ((uint32_t)(Tile::value_at(row, piece) + 8 * (lane & 1)) ^ (64u * c)) + flash_lds(vals);
        FlashLds uint8_t* p = reinterpret_cast<FlashLds uint8_t*>((uintptr_t)at) + 16 * t * Tile::kPitch;
        const v2u_flash a = flash_read_tr(p), b = flash_read_tr(p + 8 * Tile::kPitch);
        return (v4u_flash){a[0], a[1], b[0], b[1]};
    }

    // ---- a tile in two turns, one at the matrix cores and one at the vector ALU ----
    // weighted sums of the tile before (PV), whose weights and first values are at hand, and scores of this one; what a product needs of
    // LDS is asked for eight products ahead.  LOW: `low` bytes behind the keys' tile is one of what their rounding to 16 bits left out.
    template <int KEYS, bool PV, bool LOW, int AHEAD>
    __device__ __forceinline__ void products(FlashTurn<W, KEYS, AHEAD>& s, const uint8_t* kt, const uint8_t* vals_before, int low = 0) {
        constexpr int kAhead = PV ? AHEAD : 0, kRest = PV && kAhead ? KEYS / 16 - kAhead : 0;
        constexpr int kFirst = W <= 128 ? Tile::kSteps : 4;   // (all that registers allow)
        v4u_flash k[KEYS / 32][Tile::kSteps], v[kRest ? kRest : 1][Tile::kBlocks];
#pragma unroll
        for (int t = 0; t < kFirst; ++t) k[0][t] = keys(kt, 0, t);
#pragma unroll
        for (int g = 0; g < kRest; ++g)
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) v[g][c] = values(vals_before, kAhead + g, c);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (PV) {
            if constexpr (kAhead == 0) weigh<KEYS>(s.p, vals_before);
#pragma unroll
            for (int g = 0; g < kAhead; ++g)
#pragma unroll
                for (int c = 0; c < Tile::kBlocks; ++c) acc[c] = flash_mfma<F16>(s.v[g][c], s.p[g], acc[c]);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int kb = 1; kb < KEYS / 32; ++kb)
#pragma unroll
            for (int t = 0; t < Tile::kSteps; ++t) k[kb][t] = keys(kt, kb, t);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < kRest; ++g)
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) acc[c] = flash_mfma<F16>(v[g][c], s.p[kAhead + g], acc[c]);
#pragma unroll
        for (int kb = 0; kb < KEYS / 32; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s.x[kb][i] = 0.0f;
#pragma unroll
        for (int t = 0; t < Tile::kSteps; ++t) {
#pragma unroll
            for (int kb = 0; kb < KEYS / 32; ++kb)
                s.x[kb] = flash_mfma<F16>(kb == 0 && t >= kFirst ? keys(kt, kb, t) : k[kb][t], q[t], s.x[kb]);
            if constexpr (LOW) {   // (into the registers that the products behind leave)
#pragma unroll
                for (int kb = 0; kb < KEYS / 32; ++kb)
                    if (t < kFirst) k[kb][t] = keys(kt + low, kb, t);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (LOW) {
#pragma unroll
            for (int t = 0; t < Tile::kSteps; ++t)
#pragma unroll
                for (int kb = 0; kb < KEYS / 32; ++kb) s.x[kb] = flash_mfma<F16>(t >= kFirst ? keys(kt + low, kb, t) : k[kb][t], q[t], s.x[kb]);
        }
    }
    template <int KEYS, int AHEAD>
    __device__ __forceinline__ void weigh_rest(const FlashTurn<W, KEYS, AHEAD>& s, const uint8_t* vt) {
#pragma unroll
        for (int g = 0; g < KEYS / 16; ++g)
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) acc[c] = flash_mfma<F16>(g < AHEAD ? s.v[g < AHEAD ? g : 0][c] : values(vt, g, c), s.p[g], acc[c]);
    }
    template <int KEYS>
    __device__ __forceinline__ void weigh(const v4u_flash (&p)[KEYS / 16], const uint8_t* vt) {
#pragma unroll
        for (int g = 0; g < KEYS / 16; ++g)
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) acc[c] = flash_mfma<F16>(values(vt, g, c), p[g], acc[c]);
    }
    // The same where some row of the wavefront does not see some key.  Its weight 0 is no part of the row's sum, but would make a NaN of an
    // infinity or NaN among the key's values: those are left out here.  True: there are some, which belong to the rows that see them.
    template <int KEYS>
    __device__ __forceinline__ bool weigh_finite(const v4u_flash (&p)[KEYS / 16], const uint8_t* vt) {
        typedef short v2s __attribute__((ext_vector_type(2)));
        constexpr uint32_t kExp = F16 ? 0x7C00u : 0x7F80u, kUp = 0x8000u - kExp;
        uint32_t found = 0;
#pragma unroll
        for (int g = 0; g < KEYS / 16; ++g)
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) {
                v4u_flash o = values(vt, g, c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t odd = (o[e] & (kExp << 16 | kExp)) + (kUp << 16 | kUp);   // the sign bit of a half that is not finite
                    found |= odd;
                    o[e] &= ~__builtin_bit_cast(uint32_t, __builtin_bit_cast(v2s, odd) >> 15);
                }
                acc[c] = flash_mfma<F16>(o, p[g], acc[c]);
            }
        return __builtin_amdgcn_ballot_w64((found & 0x80008000u) != 0) != 0;
    }
    // a value that weigh_finite left out, or 0
    __device__ static __forceinline__ float odd_value(uint32_t u) {
        const uint32_t mag = u & 0x7FFFu;
        if constexpr (F16) return mag < 0x7C00u ? 0.0f : __uint_as_float((u & 0x8000u) << 16 | 0x7F800000u | (mag & 0x3FFu) << 13);
        return mag < 0x7F80u ? 0.0f : __uint_as_float(u << 16);
    }
    template <int KEYS, int AHEAD>
    __device__ __forceinline__ void ask_ahead(FlashTurn<W, KEYS, AHEAD>& s, const uint8_t* vt) {
#pragma unroll
        for (int g = 0; g < AHEAD; ++g)
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) s.v[g][c] = values(vt, g, c);
        __builtin_amdgcn_sched_barrier(0);
    }
    // scores of keys that the row does not see become -inf; sees(c): whether it sees key c + 4 half of the tile
    template <int KEYS, int AHEAD, typename Sees>
    __device__ __forceinline__ void mask(FlashTurn<W, KEYS, AHEAD>& s, Sees sees) {
#pragma unroll
        for (int kb = 0; kb < KEYS / 32; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s.x[kb][i] = sees(32 * kb + 8 * (i >> 2) + (i & 3)) ? s.x[kb][i] : -__builtin_huge_valf();
    }
    // Weights of the tile at hand; MASKED: there may be scores of -inf.  unit, not negative: what makes a product a score of base 2, one for all
    // or UNITS for as many parts of the tile.
    template <int KEYS, bool CAP, bool MASKED, int AHEAD, int UNITS>
    __device__ __forceinline__ void softmax(FlashTurn<W, KEYS, AHEAD>& s, const float (&unit)[UNITS], const FlashCap<UNITS == 1>& cap) {
        constexpr float kBias = F16 ? kFlashHalfBias : 0.0f, kSlack = F16 ? kFlashHalfSlack : kFlashSlack;
        constexpr int kOf = KEYS / 2 / UNITS;   // numbers of a lane that share a unit
        constexpr bool kOwnUnit = CAP && UNITS == 1;   // the cap has it
        auto& x = s.x;
        // the largest of what each unit's numbers are, that all make a score of
        auto most_of = [&](auto number, auto larger) __attribute__((always_inline)) {
            float most;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                float tops[2] = {number(x[kOf * u >> 4][kOf * u & 15]), number(x[kOf * u >> 4][(kOf * u & 15) + 1])};
#pragma unroll
                for (int i = kOf * u + 2; i < kOf * u + kOf; ++i) tops[i & 1] = larger(tops[i & 1], number(x[i >> 4][i & 15]));
                const float top = larger(tops[0], tops[1]) * (kOwnUnit ? 1.0f : unit[u]);
                most = u == 0 ? top : larger(most, top);
            }
            return most;
        };
        auto top_of = [&]() __attribute__((always_inline)) { return most_of([](float v) { return v; }, [](float a, float b) { return fmaxf(a, b); }); };
        auto raise = [&](float top) __attribute__((always_inline)) {
            const float m_new = fmaxf(m, halves_max(top));
            const float back = __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= back;
#pragma unroll
            for (int c = 0; c < Tile::kBlocks; ++c) acc[c] *= back;
        };
        // ---- the running maximum, where a score is 2^kSlack times what it allows ----
        float size = 0.0f;   // the largest magnitude of what is seen, or NaN, which capping would lose and the sum keeps
        if constexpr (CAP) {
            size = most_of([](float v) { return MASKED && v == -__builtin_huge_valf() ? 0.0f : fabsf(v); },
                           [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
            l = size == size ? l : size;
            if (__builtin_amdgcn_ballot_w64(!(size * (kOwnUnit ? cap.unit : 1.0f) <= m + kSlack)) != 0) {
                const float top = cap(top_of());
                if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0) raise(top);
            }
        } else {
            const float top = top_of();
            if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0) raise(top);
        }
        // ---- weights, rounded once as the product's operand (their sum is taken unrounded) ----
        const float base = kBias - m;
        auto weigh_all = [&](auto weight) __attribute__((always_inline)) {
            float sums[2] = {0.0f, 0.0f};
#pragma unroll
            for (int kb = 0; kb < KEYS / 32; ++kb)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float p0 = weight(x[kb][i], unit[(16 * kb + i) / kOf]), p1 = weight(x[kb][i + 1], unit[(16 * kb + i + 1) / kOf]);
                    sums[0] += p0;
                    sums[1] += p1;
                    s.p[2 * kb + (i >> 3)][(i & 7) >> 1] = flash_pack<F16>(p0, p1);
                }
            l += sums[0] + sums[1];
        };
        if constexpr (!CAP) {
            weigh_all([&](float v, float of) { return __builtin_amdgcn_exp2f(fmaf(v, of, base)); });
        } else if (__builtin_amdgcn_ballot_w64(!(size <= cap.small)) == 0) {
            const float c2 = cap.here(cap.of(cap.kSmall2));
            weigh_all([&](float v, float of) {
                const float y = kOwnUnit ? v : v * of, w = __builtin_amdgcn_exp2f(fmaf(y, cap.small_factor(y, c2), base));
                return MASKED && v == -__builtin_huge_valf() ? 0.0f : w;   // (the cap of what is not seen is no score)
            });
        } else {
            const float p3 = cap.here(cap.of(cap.kP3)), q3 = cap.here(cap.kQ3);
            weigh_all([&](float v, float of) {
                const float y = cap.within(kOwnUnit ? v : v * of), w = __builtin_amdgcn_exp2f(fmaf(y, cap.factor(y, p3, q3), base));
                return MASKED && v == -__builtin_huge_valf() ? 0.0f : w;
            });
        }
    }
};

}  // namespace resq
