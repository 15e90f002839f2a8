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
__device__ __forceinline__ v2u_flash flash_read_tr(const uint8_t* p) {
    return __builtin_bit_cast(v2u_flash, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                             (__attribute__((address_space(3))) v4s_flash*)(__attribute__((address_space(3))) uint8_t*)p));
}

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
    // scores of keys [32 kb, 32 kb + 32) of a tile
    __device__ __forceinline__ v16f_flash scores(const uint8_t* keys, int kb) const {
        const int lane = threadIdx.x & 63;
        v16f_flash s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
        for (int t = 0; t < Tile::kSteps; ++t) {
            const v4u_flash k = *reinterpret_cast<const v4u_flash*>(keys + 32 * kb * Tile::kPitch + Tile::key_at(lane & 31, 2 * t + (lane >> 5)));
            s = flash_mfma<F16>(k, q[t], s);
        }
        return s;
    }
    // values of keys 16 t .. 16 t + 15 and channels [32 c, 32 c + 32), as the second product's operand
    __device__ __forceinline__ v4u_flash values(const uint8_t* vals, int t, int c) const {
        const int lane = threadIdx.x & 63;
        const int row = 4 * (lane >> 5) + ((lane >> 2) & 3), piece = 4 * c + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        const uint8_t* p = vals + 16 * t * Tile::kPitch + Tile::value_at(row, piece) + 8 * (lane & 1);
        const v2u_flash a = flash_read_tr(p), b = flash_read_tr(p + 8 * Tile::kPitch);
        return (v4u_flash){a[0], a[1], b[0], b[1]};
    }
};

}  // namespace resq
