// The paged K/V cache: the plan of a step (pages and slots of new tokens, from request lengths), the writer and the reader.
//
// A slot is page * page_size + row; the compact row of head h of the token in it (resq_kv_row.hip.h: codes, then scales and
// zero-points) lies at pages + page * page_stride + h * head_stride + row * row_stride.  Slots are checked against the number
// of pages before they become addresses: what lies outside is skipped.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq_kv_row.hip.h"
#include "resq_lanes.hip.h"

namespace resq {

constexpr int kKvThreads = 256;

// ---------------------------------------------------------------------------
// The plan.  Request b holds lens[b] tokens in ceil(lens[b] / page_size) pages, named by its row of the block table, and gets
// news[b] more: its tokens' places in the batch are a prefix sum, the pages it lacks another one, taken off the front of the
// free list.  One workgroup makes the sums and checks them (nothing changes unless everything fits); then every token finds
// its request by bisection of the first sum, and the token that opens a page writes the page's entry.
// Latency: 8 bytes in and 16 out per request, 8 out per token.
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;

struct KvPlanArgs {
    const int32_t* lens;
    const int32_t* news;
    int B;
    int page_size;
    int num_pages;
    const int32_t* free_pages;
    int64_t n_free;
    const int32_t* taken;   // entries of free_pages handed out before
    int32_t* table;
    int64_t ld_table;
    int width;              // entries of a table row
    int max_tokens;
    int32_t* lens_out;
    int32_t* cu_tokens;     // [B + 1]
    int32_t* cu_pages;      // [B + 1]
    int32_t* positions;     // [max_tokens]
    int32_t* slots;         // [max_tokens]
    int32_t* state;         // taken after the call, status
};

// exclusive prefix sums of two 64-bit counts over the block's threads, and their totals
__device__ __forceinline__ void block_scan2(int64_t& a, int64_t& b, int64_t& total_a, int64_t& total_b, int64_t (*part)[2]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sa = a, sb = b;
    for (int k = 1; k < 64; k <<= 1) {
        const int64_t ua = __shfl_up(sa, k), ub = __shfl_up(sb, k);
        if (lane >= k) {
            sa += ua;
            sb += ub;
        }
    }
    if (lane == 63) {
        part[wave][0] = sa;
        part[wave][1] = sb;
    }
    __syncthreads();
    int64_t before_a = 0, before_b = 0;
    total_a = total_b = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
        if (w == wave) {
            before_a = total_a;
            before_b = total_b;
        }
        total_a += part[w][0];
        total_b += part[w][1];
    }
    a = before_a + sa - a;
    b = before_b + sb - b;
}

__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(const KvPlanArgs p) {
    __shared__ int64_t part[kPlanThreads / 64][2];
    __shared__ int flags;
    const int t = threadIdx.x;
    const int per = (p.B + kPlanThreads - 1) / kPlanThreads;   // consecutive requests of a thread
    const int b0 = min(t * per, p.B), b1 = min(b0 + per, p.B);
    if (t == 0) flags = 0;
    const int taken = *p.taken;
    int64_t tokens = 0, pages = 0;
    int bad = taken < 0 ? 2 : 0;
    for (int b = b0; b < b1; ++b) {
        const int64_t len = p.lens[b], add = p.news[b];
        if (len < 0 || add < 0) {
            bad |= 2;
            continue;
        }
        const int64_t all = (len + add + p.page_size - 1) / p.page_size;
        if (all > p.width) bad |= 1;
        tokens += add;
        pages += all - (len + p.page_size - 1) / p.page_size;
    }
    int64_t total_tokens, total_pages;
    block_scan2(tokens, pages, total_tokens, total_pages, part);   // (its barrier is behind flags = 0)
    if (bad) atomicOr(&flags, bad);
    __syncthreads();
    const int status = flags & 2 ? 4 : total_tokens > p.max_tokens ? 3 : flags & 1 ? 2 : taken + total_pages > p.n_free ? 1 : 0;
    for (int b = b0; b < b1; ++b) {
        const int len = p.lens[b], add = p.news[b];
        p.cu_tokens[b] = status ? 0 : (int)tokens;
        p.cu_pages[b] = status ? 0 : (int)pages;
        p.lens_out[b] = status ? len : len + add;
        tokens += add;
        pages += ((int64_t)len + add + p.page_size - 1) / p.page_size - ((int64_t)len + p.page_size - 1) / p.page_size;
    }
    if (t == 0) {
        p.cu_tokens[p.B] = status ? 0 : (int)total_tokens;
        p.cu_pages[p.B] = status ? 0 : (int)total_pages;
        p.state[0] = status ? taken : taken + (int)total_pages;
        p.state[1] = status;
    }
}

__global__ __launch_bounds__(256) void kv_plan_tokens_kernel(const KvPlanArgs p) {
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= p.max_tokens) return;
    if (t >= p.cu_tokens[p.B]) {   // behind the last token, and after a refusal: nothing to write
        p.positions[t] = 0;
        p.slots[t] = -1;
        return;
    }
    int lo = 0, hi = p.B;   // the last request that begins at or before t
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.cu_tokens[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int first = p.cu_tokens[lo];
    const int old = p.lens_out[lo] - (p.cu_tokens[lo + 1] - first);
    const int pos = old + (t - first);
    const int at = pos / p.page_size, row = pos - at * p.page_size;
    const int have = (int)(((int64_t)old + p.page_size - 1) / p.page_size);
    int32_t* entry = p.table + (int64_t)lo * p.ld_table + at;
    int page;
    if (at >= have) {
        page = p.free_pages[(int64_t)(p.state[0] - p.cu_pages[p.B]) + p.cu_pages[lo] + (at - have)];
        if (row == 0) *entry = page;   // a new page's first row is new too
    } else {
        page = *entry;
    }
    p.positions[t] = pos;
    p.slots[t] = (unsigned)page < (unsigned)p.num_pages ? page * p.page_size + row : -1;
}

// ---------------------------------------------------------------------------
// The writer and the reader: one row per token, head and kind (blockIdx.y: keys, values), G lanes to a row.
// Bound by HBM at prefill sizes (2 d_head bytes of bf16 and a row of codes per row), by the launch at a step's.
// ---------------------------------------------------------------------------
struct KvPagesArgs {
    const uint16_t* x[2];       // bf16 [tokens, heads, d], keys and values
    int64_t ld[2], ldh[2];      // elements from token to token and from head to head
    int64_t tokens;
    int heads, d, r;
    const int32_t* slots;
    uint8_t* pages[2];
    int64_t page_stride, head_stride, row_stride;   // bytes
    int page_size;
    uint32_t num_slots;
};

__device__ __forceinline__ int64_t kv_row_offset(const KvPagesArgs& a, uint32_t slot, int head) {
    const uint32_t page = slot / (uint32_t)a.page_size, row = slot - page * (uint32_t)a.page_size;
    return page * a.page_stride + head * a.head_stride + row * a.row_stride;
}

template <int G>
__global__ __launch_bounds__(kKvThreads) void append_kv_cache_kernel(const KvPagesArgs a) {
    const int gl = threadIdx.x & (G - 1), kind = blockIdx.y;
    const int64_t rows = a.tokens * a.heads;
    const int64_t m_raw = (int64_t)blockIdx.x * (kKvThreads / G) + threadIdx.x / G;
    const int64_t m = m_raw < rows ? m_raw : rows - 1;   // groups past the last row quantize it and store nothing
    const int64_t token = m / a.heads;
    const int head = (int)(m - token * a.heads);
    const uint32_t slot = (uint32_t)a.slots[token];
    const uint16_t* x = a.x[kind] + token * a.ld[kind] + head * a.ldh[kind];
    const uint4 v = gl < (a.d >> 3) ? reinterpret_cast<const uint4*>(x)[gl] : make_uint4(0u, 0u, 0u, 0u);
    const bool wanted = m_raw < rows && slot < a.num_slots;
    quantize_kv_row<G>(v, gl, a.d, a.r, wanted ? a.pages[kind] + kv_row_offset(a, slot, head) : nullptr);
}

template <int G>
__global__ __launch_bounds__(kKvThreads) void gather_kv_cache_kernel(const KvPagesArgs a) {
    const int gl = threadIdx.x & (G - 1), kind = blockIdx.y;
    const int64_t m = (int64_t)blockIdx.x * (kKvThreads / G) + threadIdx.x / G;
    if (m >= a.tokens * a.heads || gl >= (a.d >> 3)) return;
    const int64_t token = m / a.heads;
    const int head = (int)(m - token * a.heads);
    const uint32_t slot = (uint32_t)a.slots[token];
    uint4 o = make_uint4(0u, 0u, 0u, 0u);
    if (slot < a.num_slots) o = dequantize_kv_piece(a.pages[kind] + kv_row_offset(a, slot, head), gl, a.d, a.r);
    uint16_t* x = const_cast<uint16_t*>(a.x[kind]) + token * a.ld[kind] + head * a.ldh[kind];
    reinterpret_cast<uint4*>(x)[gl] = o;
}

}  // namespace resq
