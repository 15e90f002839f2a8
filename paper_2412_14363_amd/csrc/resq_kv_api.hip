// C ABI of the generation step's side of the library: position embedding, paged K/V cache, attention over it.
// Argument checks on the host, then launches on the caller's stream.  See include/resq.h for the contract of every entry.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "resq.h"
#include "resq_attend.hip.h"
#include "resq_kv.hip.h"
#include "resq_launch.h"
#include "resq_rope.hip.h"

using namespace resq;

namespace {

constexpr int64_t kInt32Max = 0x7FFFFFFF;
constexpr int64_t kMaxAttendLen = 1 << 30;

// rows of `width` elements, ld from one to the next of n and ldh from one to the next of heads, that do not overlap
inline bool rows_apart(int64_t n, int64_t ld, int64_t heads, int64_t ldh, int64_t width) {
    if ((n > 1 && ld < width) || (heads > 1 && ldh < width)) return false;
    return n <= 1 || heads <= 1 || ld >= (heads - 1) * ldh + width || ldh >= (n - 1) * ld + width;
}

// a head's row in pages: as everywhere, or with an 8-bit group of an odd multiple of four channels, at even addresses then
inline bool page_head_ok(int64_t d_head, int64_t r) {
    return kv_head_ok(d_head, r) || (kv_head_ok(d_head, r - 4) && r < d_head && d_head <= 256);
}

struct PagesGeometry {
    int64_t num_pages, page_size, heads, page_stride, head_stride, row_stride;
};

// checks the pages of a cache; strides of axes with one entry do not matter and become 0
int check_pages(PagesGeometry& g, const void* k_pages, const void* v_pages, int64_t d_head, int64_t r) {
    if (!page_head_ok(d_head, r) || g.num_pages < 1 || g.page_size < 1 || g.num_pages > kInt32Max / g.page_size || g.heads < 1 ||
        g.heads > 65535)
        return RESQ_ERR_SHAPE;
    const int64_t need = r + (d_head - r) / 2 + 16;
    if (g.num_pages == 1) g.page_stride = 0;
    if (g.heads == 1) g.head_stride = 0;
    if (g.page_size == 1) g.row_stride = 0;
    if ((g.num_pages > 1 && g.page_stride < need) || (g.heads > 1 && g.head_stride < need) ||
        (g.page_size > 1 && g.row_stride < need))
        return RESQ_ERR_BUFFER;
    if (!k_pages || !v_pages) return RESQ_ERR_NULL;
    const int align = r % 8 ? 2 : 4;
    if (!aligned(k_pages, align) || !aligned(v_pages, align) || g.page_stride % align || g.head_stride % align || g.row_stride % align)
        return RESQ_ERR_ALIGN;
    return RESQ_OK;
}

// what the paged writer and the reader check alike; done: nothing to do
int make_pages_args(KvPagesArgs& a, bool& done, const void* k, int64_t ldk, int64_t ldkh, const void* v, int64_t ldv, int64_t ldvh,
                    int64_t tokens, int64_t heads, int64_t d_head, int64_t r, const int32_t* slots, const void* k_pages,
                    const void* v_pages, int64_t num_pages, int64_t page_size, int64_t page_stride, int64_t head_stride,
                    int64_t row_stride) {
    done = true;
    if (tokens < 0 || tokens > kInt32Max || ldk < 0 || ldkh < 0 || ldv < 0 || ldvh < 0) return RESQ_ERR_SHAPE;
    PagesGeometry g{num_pages, page_size, heads, page_stride, head_stride, row_stride};
    const int rc = check_pages(g, k_pages, v_pages, d_head, r);
    if (rc == RESQ_ERR_SHAPE || rc == RESQ_ERR_BUFFER) return rc;
    const int64_t lanes = (d_head <= 128 ? 16 : d_head <= 256 ? 32 : 64) * (r % 8 ? 2 : 1);   // of a row (below)
    if (tokens > kInt32Max / heads || !launch_fits(tokens * heads + 63, lanes)) return RESQ_ERR_SHAPE;
    if (tokens == 0) return RESQ_OK;
    if (!k || !v || !slots) return RESQ_ERR_NULL;
    if (rc != RESQ_OK) return rc;
    if (!aligned(k, 16) || !aligned(v, 16) || (tokens > 1 && (ldk % 8 || ldv % 8)) || (heads > 1 && (ldkh % 8 || ldvh % 8)) ||
        !aligned(slots, 4))
        return RESQ_ERR_ALIGN;
    a.x[0] = static_cast<const uint16_t*>(k);
    a.x[1] = static_cast<const uint16_t*>(v);
    a.ld[0] = tokens > 1 ? ldk : 0;
    a.ld[1] = tokens > 1 ? ldv : 0;
    a.ldh[0] = heads > 1 ? ldkh : 0;
    a.ldh[1] = heads > 1 ? ldvh : 0;
    a.rows = (uint32_t)(tokens * heads);
    a.heads = FastDiv((uint32_t)heads);
    a.d = (int)d_head;
    a.r = (int)r;
    a.slots = slots;
    a.pages[0] = static_cast<uint8_t*>(const_cast<void*>(k_pages));
    a.pages[1] = static_cast<uint8_t*>(const_cast<void*>(v_pages));
    a.page_stride = g.page_stride;
    a.head_stride = g.head_stride;
    a.row_stride = g.row_stride;
    a.page_size = FastDiv((uint32_t)page_size);
    a.num_slots = (uint32_t)(num_pages * page_size);
    done = false;
    return RESQ_OK;
}

// layout of the attention's workspace: where each head's partial results are, then their maxima and sums, then their weighted
// sums, two results to a workgroup
struct AttendWorkspace {
    size_t ml, acc, bytes;
    int rows;
};
AttendWorkspace attend_workspace(int64_t B, int64_t heads_k, int64_t share, int64_t d_head) {
    AttendWorkspace w;
    w.rows = (int)(share < kAttendRows ? share : kAttendRows);
    const size_t heads = (size_t)B * heads_k * ((share + kAttendRows - 1) / kAttendRows);
    w.ml = (heads * 2 * sizeof(int32_t) + 255) / 256 * 256;
    w.acc = w.ml + (size_t)2 * kAttendMaxGrid * kAttendRows * 2 * sizeof(float);
    w.bytes = w.acc + (size_t)2 * kAttendMaxGrid * w.rows * d_head * sizeof(float);
    return w;
}

template <int NL, int HT, int OCC>
int launch_attend(const AttendArgs& a, int64_t units, hipStream_t st) {
    const int Q = a.share <= 8 ? 8 : 16;
    int lds = attend_tiles_bytes(NL, HT) + kAttendWaves * attend_weights_bytes(Q);
    const int red = kAttendWaves * a.rows * a.d * (int)sizeof(float);
    if (lds < red) lds = red;
    AttendArgs args = a;
    args.lds_red = lds;
    lds += kAttendWaves * kAttendRows * (int)sizeof(float4);
    void (*kernel)(const AttendArgs);
    if (Q == 8) kernel = a.blocks16 ? attend_kv_cache_kernel<NL, HT, 8, true, OCC> : attend_kv_cache_kernel<NL, HT, 8, false, OCC>;
    else kernel = a.blocks16 ? attend_kv_cache_kernel<NL, HT, 16, true, OCC> : attend_kv_cache_kernel<NL, HT, 16, false, OCC>;
    if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                               lds) != hipSuccess)
        return RESQ_ERR_HIP;
    // as many workgroups as run at once, one run each: no head begins more often than that asks for (four times as many: 1 x 131072
    // 67.1 us instead of 49.0, 256 x 512 58.6 instead of 56.5)
    const int64_t grid = units < 256 * OCC ? (units + 7) / 8 * 8 : 256 * OCC;   // a multiple of the dies
    launch(kernel, dim3((unsigned)grid), dim3(kAttendThreads), (size_t)lds, st, args);
    const int64_t heads = (int64_t)a.B * a.heads_k * a.qtiles;
    launch(attend_join_kernel, dim3((unsigned)heads, heads < kAttendJoinSplit ? (unsigned)a.rows : 1), dim3(kAttendThreads), 0, st, args);
    return launch_status();
}

}  // namespace

extern "C" {

int resq_kv_slots(const int32_t* lens, const int32_t* new_tokens, int64_t B, int64_t page_size, int64_t num_pages,
                  const int32_t* free_pages, int64_t n_free, const int32_t* taken, int32_t* block_table, int64_t ld_table,
                  int64_t width, int64_t max_tokens, int32_t* lens_out, int32_t* cu_tokens, int32_t* cu_pages,
                  int32_t* positions, int32_t* slots, int32_t* state, void* stream) {
    if (B < 1 || B > 65536 || page_size < 1 || num_pages < 1 || num_pages > kInt32Max / page_size || n_free < 0 ||
        n_free > kInt32Max || width < 1 || width > kInt32Max / page_size || (B > 1 && ld_table < width) || max_tokens < 1 ||
        max_tokens > kInt32Max - 256)
        return RESQ_ERR_SHAPE;
    if (!lens || !new_tokens || (n_free > 0 && !free_pages) || !taken || !block_table || !lens_out || !cu_tokens || !cu_pages ||
        !positions || !slots || !state)
        return RESQ_ERR_NULL;
    for (const void* p : {(const void*)lens, (const void*)new_tokens, (const void*)free_pages, (const void*)taken,
                          (const void*)block_table, (const void*)lens_out, (const void*)cu_tokens, (const void*)cu_pages,
                          (const void*)positions, (const void*)slots, (const void*)state})
        if (!aligned(p, 4)) return RESQ_ERR_ALIGN;
    const KvPlanArgs p{lens, new_tokens, (int)B, FastDiv((uint32_t)page_size), (int)num_pages, free_pages, n_free, taken, block_table, ld_table,
                       (int)width, (int)max_tokens, lens_out, cu_tokens, cu_pages, positions, slots, state};
    hipStream_t st = static_cast<hipStream_t>(stream);
    // One launch where it can be, see resq_kv.hip.h: 3.3 us for 32 requests of a token, two take 4.4; 32 and 1024 tokens in place 4.0 and
    // 5.0.  In place one workgroup has to serve all tokens: 16384 of them 8.2 us, two launches 5.2, from 1024 or so on they are even.  1024
    // tokens to a workgroup where there can be several, instead of 256: 5.4 for 3.5 (1024 tokens).
    const bool in_place = lens == lens_out || taken == state;
    if (B <= kPlanRequests && (!in_place || max_tokens <= kPlanTokensInPlace)) {
        const int per_block = in_place ? kPlanTokensInPlace : kPlanTokens;
        launch(kv_plan_kernel, dim3((unsigned)((max_tokens + per_block - 1) / per_block)), dim3(kPlanThreads), 3 * B * sizeof(int), st, p,
               per_block);
        return launch_status();
    }
    launch(kv_plan_sums_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
    launch(kv_plan_tokens_kernel, dim3((unsigned)((max_tokens + 255) / 256)), dim3(256), 0, st, p);
    return launch_status();
}

int resq_rope_frequencies(int64_t rot, double base, int scaling, double factor, double low, double high, int64_t original_len,
                          double* freq, float* mscale) {
    if (rot < 2 || rot > kRopeMaxHead || rot % 2 || !(base > 1.0) || !isfinite(base) || scaling < 0 || scaling > 4) return RESQ_ERR_SHAPE;
    if (scaling != RESQ_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return RESQ_ERR_SHAPE;
    if (scaling >= RESQ_ROPE_BANDS && (!(low > 0.0) || !(high > low) || !isfinite(high) || original_len < 1)) return RESQ_ERR_SHAPE;
    if (!freq || !mscale) return RESQ_ERR_NULL;
    const double turn = 6.283185307179586477;
    *mscale = 1.0f;
    double first = 0.0, last = 0.0;
    if (scaling == RESQ_ROPE_BASE && rot > 2) base *= pow(factor, (double)rot / (double)(rot - 2));
    if (scaling == RESQ_ROPE_RAMP) {   // the pairs that make `high` and `low` turns over the original length
        const double per = rot / (2.0 * log(base));
        first = fmax(floor(per * log(original_len / (high * turn))), 0.0);
        last = fmin(ceil(per * log(original_len / (low * turn))), (double)(rot - 1));
        if (last <= first) last = first + 0.001;
        *mscale = (float)(0.1 * log(factor) + 1.0);
    }
    for (int64_t i = 0; i < rot / 2; ++i) {
        const double f = pow(base, -2.0 * (double)i / (double)rot);
        double keep = 1.0;   // share of the frequency that stays as it is; the rest is divided by the factor
        if (scaling == RESQ_ROPE_LINEAR) keep = 0.0;
        if (scaling == RESQ_ROPE_BANDS) keep = fmin(fmax((original_len * f / turn - low) / (high - low), 0.0), 1.0);
        if (scaling == RESQ_ROPE_RAMP) keep = 1.0 - fmin(fmax(((double)i - first) / (last - first), 0.0), 1.0);
        freq[i] = keep * f + (1.0 - keep) * (f / factor);
    }
    return RESQ_OK;
}

int resq_rope_heads(const void* x, int64_t ldx, int64_t ldxh, int64_t tokens, int64_t heads_q, int64_t heads_k, int64_t d_head,
                    const void* w_q, const void* w_k, float eps, const int32_t* positions, const double* freq, int64_t rot,
                    int interleaved, float mscale, void* y, int64_t ldy, int64_t ldyh, void* stream) {
    const int64_t heads = heads_q + heads_k;
    if (tokens < 0 || tokens > kInt32Max || heads_q < 0 || heads_k < 0 || heads_q > 65535 || heads_k > 65535 || heads < 1 || d_head < 2 ||
        d_head > kRopeMaxHead || d_head % 2 || rot < 0 || rot > d_head || rot % 2 || ldx < 0 || ldxh < 0 || !(eps >= 0.0f) ||
        !isfinite(eps) || !rows_apart(tokens, ldy, heads, ldyh, d_head))
        return RESQ_ERR_SHAPE;
    const bool norm = w_q || w_k;
    if (tokens == 0) return RESQ_OK;
    if (!x || !y || (rot > 0 && (!positions || !freq)) || (norm && ((heads_q > 0 && !w_q) || (heads_k > 0 && !w_k)))) return RESQ_ERR_NULL;
    if (tokens == 1) ldx = ldy = 0;
    if (heads == 1) ldxh = ldyh = 0;
    if (x == y && (ldx != ldy || ldxh != ldyh)) return RESQ_ERR_SHAPE;
    if (!aligned(x, 2) || !aligned(y, 2) || !aligned(w_q, 2) || !aligned(w_k, 2) || !aligned(positions, 4) || !aligned(freq, 8))
        return RESQ_ERR_ALIGN;
    const RopeArgs a{static_cast<const uint16_t*>(x), ldx, ldxh, tokens, (int)heads, (int)heads_q, (int)d_head,
                     static_cast<const uint16_t*>(w_q), static_cast<const uint16_t*>(w_k), eps, positions, freq, (int)rot,
                     interleaved != 0, mscale, static_cast<uint16_t*>(y), ldy, ldyh};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool any = !(aligned(x, 16) && aligned(y, 16) && ldx % 8 == 0 && ldxh % 8 == 0 && ldy % 8 == 0 && ldyh % 8 == 0 && d_head % 8 == 0 &&
                       rot % (interleaved ? 2 : 16) == 0);
    // Lanes to a head, and tokens to a workgroup: as many as give 256 threads an angle each, while 512 workgroups remain; with fewer
    // tokens than that a workgroup takes one round of heads.  Us at heads of 64, 24 of them, 8192 tokens: 9.0, one token to a
    // workgroup 16.1; 2048 tokens of 40 heads of 128 8.0 and 8.7; 1024 with 512 / 128 workgroups as the least 5.3 / 5.9.  All heads of
    // one token in one workgroup 3.0, in rounds of 32 2.7; 2048 tokens in such rounds 8.9, whole 8.0.
    const int64_t lanes = interleaved ? (d_head + 15) / 16 : (rot / 2 + 7) / 8 + (d_head - rot + 15) / 16;
    const int lg = lanes <= 4 ? 4 : lanes <= 8 ? 8 : lanes <= 16 ? 16 : lanes <= 32 ? 32 : 64, groups = 256 / lg;
    int tb_log2 = 0;
    while ((2 << tb_log2) <= groups && (rot >> 1) * (2 << tb_log2) <= 256 && tokens >= ((int64_t)512 << (tb_log2 + 1))) ++tb_log2;
    const int per_block = tokens < 512 ? groups >> tb_log2 : (int)heads;
    const dim3 grid((unsigned)((tokens + (1 << tb_log2) - 1) >> tb_log2), (unsigned)((heads + per_block - 1) / per_block));
    const size_t lds = (size_t)(rot ? rot >> 1 : 1) * sizeof(float2) << tb_log2;
    if (!launch_fits(grid.x, 256)) return RESQ_ERR_SHAPE;
#define RESQ_LAUNCH_ROPE(LG)                                                                                                \
    launch(any ? rope_pieces_kernel<LG, true> : rope_pieces_kernel<LG, false>, grid, dim3(256), lds, st, a, tb_log2, per_block)
    switch (lg) {
        case 4: RESQ_LAUNCH_ROPE(4); break;
        case 8: RESQ_LAUNCH_ROPE(8); break;
        case 16: RESQ_LAUNCH_ROPE(16); break;
        case 32: RESQ_LAUNCH_ROPE(32); break;
        default: launch(rope_pieces_kernel<64, true>, grid, dim3(256), lds, st, a, tb_log2, per_block); break;
    }
#undef RESQ_LAUNCH_ROPE
    return launch_status();
}

int resq_append_kv_cache(const void* k, int64_t ldk, int64_t ldkh, const void* v, int64_t ldv, int64_t ldvh, int64_t tokens,
                         int64_t heads, int64_t d_head, int64_t r, const int32_t* slots, void* k_pages, void* v_pages,
                         int64_t num_pages, int64_t page_size, int64_t page_stride, int64_t head_stride, int64_t row_stride,
                         void* stream) {
    KvPagesArgs a;
    bool done;
    const int rc = make_pages_args(a, done, k, ldk, ldkh, v, ldv, ldvh, tokens, heads, d_head, r, slots, k_pages, v_pages, num_pages,
                                   page_size, page_stride, head_stride, row_stride);
    if (rc != RESQ_OK || done) return rc;
#define RESQ_LAUNCH_APPEND(G, C)                                                                                       \
    launch(append_kv_cache_kernel<G, C>, dim3((a.rows + kKvThreads / G - 1) / (kKvThreads / G), 2), dim3(kKvThreads), 0,   \
           static_cast<hipStream_t>(stream), a)
    if (r % 8) {
        if (d_head <= 128) RESQ_LAUNCH_APPEND(32, 4);
        else RESQ_LAUNCH_APPEND(64, 4);
    } else if (d_head <= 128) RESQ_LAUNCH_APPEND(16, 8);
    else if (d_head <= 256) RESQ_LAUNCH_APPEND(32, 8);
    else RESQ_LAUNCH_APPEND(64, 8);
#undef RESQ_LAUNCH_APPEND
    return launch_status();
}

int resq_gather_kv_cache(const void* k_pages, const void* v_pages, int64_t num_pages, int64_t page_size, int64_t page_stride,
                         int64_t head_stride, int64_t row_stride, const int32_t* slots, int64_t tokens, int64_t heads,
                         int64_t d_head, int64_t r, void* k, int64_t ldk, int64_t ldkh, void* v, int64_t ldv, int64_t ldvh,
                         void* stream) {
    KvPagesArgs a;
    bool done;
    if (!rows_apart(tokens, ldk, heads, ldkh, d_head) || !rows_apart(tokens, ldv, heads, ldvh, d_head)) return RESQ_ERR_SHAPE;
    const int rc = make_pages_args(a, done, k, ldk, ldkh, v, ldv, ldvh, tokens, heads, d_head, r, slots, k_pages, v_pages, num_pages,
                                   page_size, page_stride, head_stride, row_stride);
    if (rc != RESQ_OK || done) return rc;
#define RESQ_LAUNCH_GATHER(G, C)                                                                                       \
    launch(gather_kv_cache_kernel<G, C>, dim3((a.rows + kKvThreads / G - 1) / (kKvThreads / G)), dim3(kKvThreads), 0,      \
           static_cast<hipStream_t>(stream), a)
    if (r % 8) {
        if (d_head <= 128) RESQ_LAUNCH_GATHER(32, 4);
        else RESQ_LAUNCH_GATHER(64, 4);
    } else if (d_head <= 128) RESQ_LAUNCH_GATHER(16, 8);
    else if (d_head <= 256) RESQ_LAUNCH_GATHER(32, 8);
    else RESQ_LAUNCH_GATHER(64, 8);
#undef RESQ_LAUNCH_GATHER
    return launch_status();
}

size_t resq_attend_kv_cache_workspace_bytes(int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head) {
    if (B < 1 || B > 65535 || heads_q < 1 || heads_q > 65535 || heads_k < 1 || heads_q % heads_k || d_head < 8 ||
        d_head > kAttendMaxHead || d_head % 8)
        return 0;
    return attend_workspace(B, heads_k, heads_q / heads_k, d_head).bytes;
}

int resq_attend_kv_cache(const void* q, int64_t ldq, int64_t ldqh, int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head,
                         int64_t r, const int32_t* lens, const int32_t* block_table, int64_t ld_table, int64_t width,
                         const void* k_pages, const void* v_pages, int64_t num_pages, int64_t page_size, int64_t page_stride,
                         int64_t head_stride, int64_t row_stride, float scale, float softcap, int64_t window, void* out,
                         int64_t ldo, int64_t ldoh, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    const size_t need = resq_attend_kv_cache_workspace_bytes(B, heads_q, heads_k, d_head);
    if (need == 0 || ldq < 0 || ldqh < 0 || width < 1 || width > kInt32Max || (B > 1 && ld_table < width) || !(scale > 0.0f) ||
        !isfinite(scale) || !(softcap == 0.0f || softcap >= FLT_MIN) || !isfinite(softcap) || window < 0 || !rows_apart(B, ldo, heads_q, ldoh, d_head))
        return RESQ_ERR_SHAPE;
    PagesGeometry g{num_pages, page_size, heads_k, page_stride, head_stride, row_stride};
    const int rc = check_pages(g, k_pages, v_pages, d_head, r);
    if (rc != RESQ_OK && rc != RESQ_ERR_NULL && rc != RESQ_ERR_ALIGN) return rc;
    if (!q || !lens || !block_table || !out || !workspace) return RESQ_ERR_NULL;
    if (rc != RESQ_OK) return rc;
    if (!aligned(q, 2) || !aligned(out, 2) || !aligned(lens, 4) || !aligned(block_table, 4) || !aligned(lse, 4) ||
        !aligned(workspace, 256))
        return RESQ_ERR_ALIGN;
    if (workspace_bytes < need) return RESQ_ERR_BUFFER;
    const int64_t longest = width > kMaxAttendLen / page_size ? kMaxAttendLen : width * page_size;
    // units of the longest sequences that the table can name: counted in 32 bits
    const int64_t qtiles = (heads_q / heads_k + kAttendRows - 1) / kAttendRows;
    const int64_t units = B * heads_k * qtiles * ((longest + kAttendUnit - 1) / kAttendUnit + kAttendHeadCost);
    if (units > kInt32Max || !launch_fits(B * heads_q, kAttendThreads)) return RESQ_ERR_SHAPE;
    AttendArgs a;
    a.q = static_cast<const uint16_t*>(q);
    a.ldq = ldq;
    a.ldqh = ldqh;
    a.B = (int)B;
    a.heads_k = (int)heads_k;
    a.share = (int)(heads_q / heads_k);
    a.d = (int)d_head;
    a.r = (int)r;
    a.lens = lens;
    a.table = block_table;
    a.ld_table = ld_table;
    a.pages[0] = static_cast<const uint8_t*>(k_pages);
    a.pages[1] = static_cast<const uint8_t*>(v_pages);
    a.num_pages = (int)num_pages;
    a.page_size = FastDiv((uint32_t)page_size);
    a.page_stride = g.page_stride;
    a.head_stride = g.head_stride;
    a.row_stride = g.row_stride;
    a.row_bytes = (int)(r + (d_head - r) / 2 + 16);
    a.qtiles = (int)qtiles;
    const AttendWorkspace w = attend_workspace(B, heads_k, a.share, d_head);
    a.joins = static_cast<int32_t*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + w.ml);
    a.part_acc = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + w.acc);
    a.rows = w.rows;
    a.blocks16 = page_size % 16 == 0 && g.row_stride < (1 << 26);
    a.fours_magic = 65536 / (a.d / 4) + 1;
    a.lds_red = 0;
    a.max_len = (int)longest;
    a.window = window < kMaxAttendLen ? (int)window : 0;
    a.scale = scale;
    a.softcap = softcap;
    a.out = static_cast<uint16_t*>(out);
    a.ldo = ldo;
    a.ldoh = ldoh;
    a.lse = lse;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t low = d_head - r;
    // The smallest kernel that holds the head's two groups of channels, in as many workgroups to a compute unit as its registers allow
    // without spilling vector registers in the loop over tiles (<0, 16> in pages that are no multiple of 16 rows has one to four there; some
    // others have up to 28 around it, once a head).  32 x 4096, in us: the next larger kernel for 128 (r = 16) 48.3 instead of 46.9, 64 (8)
    // 43.7 instead of 36.3, 256 (32) 103.5 instead of 82.5; a workgroup less 54.7 for 46.9, 37.7 for 36.3 (128, r = 32: 62.4 for 51.1); one more,
    // with spills, 310 for 82.5 (256, r = 32), 781 for 132.5 (r = 256), 57.2 for 57.3 (128, r = 64).
    if (low == 0) return r <= 64 ? launch_attend<0, 4, 3>(a, units, st) : r <= 128 ? launch_attend<0, 8, 2>(a, units, st)
                                                                                   : launch_attend<0, 16, 1>(a, units, st);
    if (low <= 64) return r <= 16 ? launch_attend<4, 1, 3>(a, units, st) : r <= 64 ? launch_attend<4, 4, 2>(a, units, st)
                                                                                   : launch_attend<4, 16, 1>(a, units, st);
    if (low <= 128) return r <= 16 ? launch_attend<8, 1, 2>(a, units, st) : r <= 32 ? launch_attend<8, 2, 2>(a, units, st)
                           : r <= 64 ? launch_attend<8, 4, 2>(a, units, st) : launch_attend<8, 16, 1>(a, units, st);
    return r <= 32 ? launch_attend<16, 2, 1>(a, units, st) : launch_attend<16, 8, 1>(a, units, st);
}

}  // extern "C"
