// Attention of one new token of each sequence over the paged cache of compact K/V rows.
//   x_t = scale * q . k_t, k_t = code * s + z (not rounded), capped to cap * tanh(x_t / cap) where there is a cap
//   out = sum_t exp(x_t - m) v_t / sum_t exp(x_t - m), lse = m + log(sum)
// over the tokens t < len of the sequence (the last `window` of them where there is a window) whose page exists.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_kv_row.hip.h"
#include "resq_lanes.hip.h"

namespace resq {

constexpr int kAttendThreads = 256;
constexpr int kAttendMaxHead = 256;

struct AttendArgs {
    const uint16_t* q;
    int64_t ldq, ldqh;
    int B, heads_k, share, d, r;
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
};

__device__ __forceinline__ float kv_value(const uint8_t* row, int d, int r, int c) {
    const float* par = reinterpret_cast<const float*>(row + r + (d - r) / 2);
    if (c < r) return fmaf((float)row[c], par[0], par[1]);
    return fmaf((float)((row[r + (c - r) / 2] >> (4 * (c & 1))) & 15), par[2], par[3]);
}

// one workgroup to a query head of a sequence, 256 tokens at a time
__global__ __launch_bounds__(kAttendThreads) void attend_kv_cache_kernel(const AttendArgs a) {
    __shared__ float q[kAttendMaxHead], p[kAttendThreads], red[8];
    __shared__ const uint8_t* rows[kAttendThreads];
    const int t = threadIdx.x, head = blockIdx.x, b = blockIdx.y, hk = head / a.share;
    const int len = min(max(a.lens[b], 0), a.max_len);
    if (t < a.d) q[t] = bf16_bits_to_f32(a.q[b * a.ldq + head * a.ldqh + t]);
    float m = -__builtin_huge_valf(), l = 0.0f, acc = 0.0f;
    for (int t0 = a.window && len > a.window ? len - a.window : 0; t0 < len; t0 += kAttendThreads) {
        __syncthreads();
        const int tok = t0 + t;
        int page = -1;
        if (tok < len) page = a.table[b * a.ld_table + tok / a.page_size];
        const bool seen = (unsigned)page < (unsigned)a.num_pages;
        const int64_t off = seen ? page * a.page_stride + hk * a.head_stride + (tok % a.page_size) * a.row_stride : 0;
        float x = -__builtin_huge_valf();
        rows[t] = seen ? a.pages[1] + off : nullptr;
        if (seen) {
            x = 0.0f;
            for (int c = 0; c < a.d; ++c) x = fmaf(q[c], kv_value(a.pages[0] + off, a.d, a.r, c), x);
            x *= a.scale;
            if (a.softcap > 0.0f) x = a.softcap * tanhf(x / a.softcap);
        }
        const float top = wave_max(x);
        if ((t & 63) == 0) red[t >> 6] = top;
        __syncthreads();
        const float m_new = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float base = m_new == -__builtin_huge_valf() ? 0.0f : m_new;
        const float e = expf(x - base), back = expf(m - base);
        p[t] = e;
        float sum = e;
        for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
        if ((t & 63) == 0) red[4 + (t >> 6)] = sum;
        __syncthreads();
        l = l * back + (red[4] + red[5]) + (red[6] + red[7]);
        acc *= back;
        m = m_new;
        if (t < a.d)
            for (int i = 0; i < kAttendThreads; ++i)
                if (rows[i]) acc = fmaf(p[i], kv_value(rows[i], a.d, a.r, t), acc);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (t < a.d) a.out[b * a.ldo + head * a.ldoh + t] = (uint16_t)pack_bf16_pair(acc * inv, 0.0f);
    if (t == 0 && a.lse) a.lse[(int64_t)b * a.heads_k * a.share + head] = l == 0.0f ? -__builtin_huge_valf() : m + logf(l);
}

}  // namespace resq
