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
// free list.  Sums first, and checks (nothing changes unless everything fits); then every token finds its request by bisection
// of the first sum, and the token that opens a page writes the page's entry.
// Latency: 8 bytes in and 16 out per request, 8 out per token.  Up to kPlanRequests requests (whose sums fit LDS) take one launch:
// every workgroup makes the sums for itself and serves some of the tokens; outputs that lie on inputs allow one workgroup only,
// which reads them all before it writes.  Else the sums go through memory to a second kernel.  In a captured graph 3.2 us for
// 32 requests of a token, 3.7 for 4096 tokens, 5.9 for 1024 requests, 19 for 4096 (16 to a thread).
// ---------------------------------------------------------------------------
constexpr int kPlanRequests = 4096;
constexpr int kPlanThreads = 256;
constexpr int kPlanTokens = 256;              // of a workgroup
constexpr int kPlanTokensInPlace = 1024;      // of the only one

struct KvPlanArgs {
    const int32_t* lens;
    const int32_t* news;
    int B;
    FastDiv page_size;
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

// inclusive sums over the lanes of a wavefront
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t shifted64(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xF, false);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t wave_scan64(int64_t x) {
    x += shifted64<0x111, 0xF>(x);   // row_shr by 1, 2, 4, 8
    x += shifted64<0x112, 0xF>(x);
    x += shifted64<0x114, 0xF>(x);
    x += shifted64<0x118, 0xF>(x);
    x += shifted64<0x142, 0xA>(x);   // row_bcast:15, row_bcast:31
    return x + shifted64<0x143, 0xC>(x);
}
// exclusive prefix sums of two 64-bit counts over the block's threads, and their totals
__device__ __forceinline__ void block_scan2(int64_t& a, int64_t& b, int64_t& total_a, int64_t& total_b, int64_t (*part)[2]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t sa = wave_scan64(a), sb = wave_scan64(b);
    if (lane == 63) {
        part[wave][0] = sa;
        part[wave][1] = sb;
    }
    __syncthreads();
    int64_t before_a = 0, before_b = 0;
    total_a = total_b = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
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

__device__ __forceinline__ int64_t plan_pages(const KvPlanArgs& p, int64_t tokens) {   // pages of so many tokens, below 2^32
    return tokens <= 0x7FFFFFFF ? (tokens == 0 ? 0 : p.page_size((uint32_t)tokens - 1) + 1) : (tokens - 1) / p.page_size.d + 1;
}

// The sums of a workgroup of kPlanThreads: each thread's requests b0 .. b1 in a row, its first request's sums, the totals and the
// status.  Sums are in 64 bits; those that are handed out fit 32.
struct PlanSums {
    int b0, b1;
    int64_t tokens, pages, total_tokens, total_pages;
    int taken, status;
};
__device__ __forceinline__ PlanSums plan_sums(const KvPlanArgs& p) {
    __shared__ int64_t part[kPlanThreads / 64][2];
    __shared__ int flags;
    const int t = threadIdx.x;
    PlanSums s;
    const int per = (p.B + kPlanThreads - 1) / kPlanThreads;
    s.b0 = min(t * per, p.B);
    s.b1 = min(s.b0 + per, p.B);
    if (t == 0) flags = 0;
    s.taken = *p.taken;
    s.tokens = s.pages = 0;
    int bad = s.taken < 0 ? 2 : 0;
    for (int b = s.b0; b < s.b1; ++b) {
        const int64_t len = p.lens[b], add = p.news[b];
        if (len < 0 || add < 0) {
            bad |= 2;
            continue;
        }
        const int64_t all = plan_pages(p, len + add);
        if (all > p.width) bad |= 1;
        s.tokens += add;
        s.pages += all - plan_pages(p, len);
    }
    block_scan2(s.tokens, s.pages, s.total_tokens, s.total_pages, part);   // (its barrier is behind flags = 0)
    if (bad) atomicOr(&flags, bad);
    __syncthreads();
    s.status = flags & 2 ? 4 : s.total_tokens > p.max_tokens ? 3 : flags & 1 ? 2 : s.taken + s.total_pages > p.n_free ? 1 : 0;
    return s;
}
// what goes out per request; request(b, old length, first token, first page) for the caller's own use
template <typename F>
__device__ __forceinline__ void plan_write(const KvPlanArgs& p, const PlanSums& s, bool write, F request) {
    int64_t tokens = s.tokens, pages = s.pages;
    for (int b = s.b0; b < s.b1; ++b) {
        const int len = p.lens[b], add = p.news[b];
        request(b, len, (int)tokens, (int)pages);
        if (write) {
            p.cu_tokens[b] = s.status ? 0 : (int)tokens;
            p.cu_pages[b] = s.status ? 0 : (int)pages;
            p.lens_out[b] = s.status ? len : len + add;
        }
        if (s.status == 0) {
            tokens += add;
            pages += plan_pages(p, (int64_t)len + add) - plan_pages(p, len);
        }
    }
    if (write && threadIdx.x == 0) {
        p.cu_tokens[p.B] = s.status ? 0 : (int)s.total_tokens;
        p.cu_pages[p.B] = s.status ? 0 : (int)s.total_pages;
        p.state[0] = s.status ? s.taken : s.taken + (int)s.total_pages;
        p.state[1] = s.status;
    }
}
// position and slot of token t: token `place` of those that request b, which held `old`, gets; pages: the request's first new one
// in the free list
__device__ __forceinline__ void plan_token(const KvPlanArgs& p, int t, int b, int old, int place, int64_t pages) {
    const int pos = old + place;
    const int at = (int)p.page_size((uint32_t)pos), row = pos - at * (int)p.page_size.d;
    const int have = (int)plan_pages(p, old);
    int32_t* entry = p.table + (int64_t)b * p.ld_table + at;
    int page;
    if (at >= have) {
        page = p.free_pages[pages + (at - have)];
        if (row == 0) *entry = page;   // a new page's first row is new too
    } else {
        page = *entry;
    }
    p.positions[t] = pos;
    p.slots[t] = (unsigned)page < (unsigned)p.num_pages ? page * (int)p.page_size.d + row : -1;
}
__device__ __forceinline__ void plan_no_token(const KvPlanArgs& p, int t) {
    p.positions[t] = 0;
    p.slots[t] = -1;
}

__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(const KvPlanArgs p, int tokens_per_block) {
    extern __shared__ int plan_lds[];   // [B] each: old lengths, first tokens, first pages
    int *olds = plan_lds, *firsts = plan_lds + p.B, *pages = plan_lds + 2 * p.B;
    const PlanSums s = plan_sums(p);
    plan_write(p, s, blockIdx.x == 0, [&](int b, int old, int token, int page) {
        olds[b] = old;
        firsts[b] = token;
        pages[b] = page;
    });
    __syncthreads();
    const int begin = blockIdx.x * tokens_per_block, end = min(begin + tokens_per_block, p.max_tokens);
    const int total = s.status ? 0 : (int)s.total_tokens;
    for (int t = begin + threadIdx.x; t < end; t += kPlanThreads) {
        if (t >= total) {   // behind the last token, and after a refusal
            plan_no_token(p, t);
            continue;
        }
        int lo = 0, hi = p.B;   // the last request that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (firsts[mid] <= t) lo = mid;
            else hi = mid;
        }
        plan_token(p, t, lo, olds[lo], t - firsts[lo], (int64_t)s.taken + pages[lo]);
    }
}

__global__ __launch_bounds__(kPlanThreads) void kv_plan_sums_kernel(const KvPlanArgs p) {
    const PlanSums s = plan_sums(p);
    plan_write(p, s, true, [](int, int, int, int) {});
}

__global__ __launch_bounds__(256) void kv_plan_tokens_kernel(const KvPlanArgs p) {
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= p.max_tokens) return;
    if (t >= p.cu_tokens[p.B]) return plan_no_token(p, t);
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.cu_tokens[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int first = p.cu_tokens[lo];
    plan_token(p, t, lo, p.lens_out[lo] - (p.cu_tokens[lo + 1] - first), t - first,
               (int64_t)(p.state[0] - p.cu_pages[p.B]) + p.cu_pages[lo]);
}

// ---------------------------------------------------------------------------
// The writer, G lanes to a row of keys or values (blockIdx.y), and the reader, G lanes to both of a token and head (so that twice
// the bytes are on their way: 21.5 instead of 25.3 us for 16384 tokens of 8 heads of 128; the writer has the quantizer's arithmetic,
// and takes longer so: 8.8 instead of 7.9 for 2911 tokens).
// The reader is bound by HBM (16384 tokens, 90 MB at least: 19.4 us from the last-level cache where slots come in runs of a page, 20.7 in
// no order, when it fetches whole lines for 88-byte rows, 53 MB for 23; 28.5 on memory that no cache has), the writer by the
// quantizer's instructions, some 270 per wavefront of four rows (27.4 us, 3.3 TB/s), both by the launch at a step's sizes (16 tokens: 2.8
// and 3.0 us).  With a head's tokens in a row where they lie so in the pages, and such workgroups in a row on one die, runs take 17.7
// and 18.1 us, but 256 channels on memory that no cache has 58 instead of 53.8, and slots in no order 22.2 and 22.9 instead of 21.5.
// ---------------------------------------------------------------------------
struct KvPagesArgs {
    const uint16_t* x[2];       // bf16 [tokens, heads, d], keys and values
    int64_t ld[2], ldh[2];      // elements from token to token and from head to head
    uint32_t rows;              // tokens * heads
    FastDiv heads;
    int d, r;
    const int32_t* slots;
    uint8_t* pages[2];
    int64_t page_stride, head_stride, row_stride;   // bytes
    FastDiv page_size;
    uint32_t num_slots;
};

__device__ __forceinline__ int64_t kv_row_offset(const KvPagesArgs& a, uint32_t slot, uint32_t head) {
    const uint32_t page = a.page_size(slot), row = slot - page * a.page_size.d;
    return page * a.page_stride + head * a.head_stride + row * a.row_stride;
}

template <int G, int C>
__global__ __launch_bounds__(kKvThreads) void append_kv_cache_kernel(const KvPagesArgs a) {
    const int gl = threadIdx.x & (G - 1), kind = blockIdx.y;
    const uint32_t m_raw = blockIdx.x * (kKvThreads / G) + threadIdx.x / G;
    const uint32_t m = min(m_raw, a.rows - 1);   // groups past the last row quantize it and store nothing
    const uint32_t token = a.heads(m), head = m - token * a.heads.d;
    const uint32_t slot = (uint32_t)a.slots[token];
    const uint16_t* x = a.x[kind] + token * a.ld[kind] + head * a.ldh[kind];
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (gl < a.d / C) {
        if constexpr (C == 8) {
            v = reinterpret_cast<const uint4*>(x)[gl];
        } else {
            const uint2 half = reinterpret_cast<const uint2*>(x)[gl];
            v.x = half.x;
            v.y = half.y;
        }
    }
    const bool wanted = m_raw < a.rows && slot < a.num_slots;
    quantize_kv_row<G, C>(v, gl, a.d, a.r, wanted ? a.pages[kind] + kv_row_offset(a, slot, head) : nullptr);
}

template <int G, int C>
__global__ __launch_bounds__(kKvThreads) void gather_kv_cache_kernel(const KvPagesArgs a) {
    const int gl = threadIdx.x & (G - 1);
    const uint32_t m = blockIdx.x * (kKvThreads / G) + threadIdx.x / G;
    if (m >= a.rows || gl >= a.d / C) return;
    const uint32_t token = a.heads(m), head = m - token * a.heads.d;
    const uint32_t slot = (uint32_t)a.slots[token];
    if constexpr (C == 4) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint2 o = make_uint2(0u, 0u);
            if (slot < a.num_slots) o = dequantize_kv_half_piece(a.pages[k] + kv_row_offset(a, slot, head), gl, a.d, a.r);
            reinterpret_cast<uint2*>(const_cast<uint16_t*>(a.x[k]) + token * a.ld[k] + head * a.ldh[k])[gl] = o;
        }
        return;
    }
    uint4 o[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
    if (slot < a.num_slots) {
        const int64_t off = kv_row_offset(a, slot, head);
#pragma unroll
        for (int k = 0; k < 2; ++k) o[k] = dequantize_kv_piece(a.pages[k] + off, gl, a.d, a.r);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
        reinterpret_cast<uint4*>(const_cast<uint16_t*>(a.x[k]) + token * a.ld[k] + head * a.ldh[k])[gl] = o[k];
}

}  // namespace resq
