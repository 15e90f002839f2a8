// C ABI of what stands around a layer's products beside the generation step: attention over whole prompts,
// attention of a batch behind a shared prefix, the norms between blocks.
// Argument checks on the host, then launches on the caller's stream.  See include/resq.h for the contract of every entry.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "resq.h"
#include "resq_launch.h"
#include "resq_norm.hip.h"
#include "resq_prefix.hip.h"
#include "resq_prompts.hip.h"

using namespace resq;

namespace {

constexpr int64_t kInt32Max = 0x7FFFFFFF;
constexpr int64_t kMaxTokens = 1 << 30;   // so that a place minus a window stays in 32 bits
constexpr int64_t kMaxStride = 1 << 24;   // of keys and values from token to token: a tile's offsets stay in 32 bits
constexpr int kMaxHead = 256;

// sizes that both entries of the prompts' attention check, and what they have in common
struct PromptPlan {
    int waves;           // of a workgroup
    int64_t tiles;       // of its rows, at most
    int keys, parts, least;
    size_t acc, bytes;   // workspace: maxima and sums, weighted sums behind them
};
bool prompt_plan(PromptPlan& p, int64_t tokens_q, int64_t tokens_k, int64_t B, int64_t heads_q, int64_t heads_k, int64_t d) {
    if (tokens_q < 0 || tokens_q > kMaxTokens || tokens_k < 0 || tokens_k > kMaxTokens || B < 1 || B > 65535 || heads_q < 1 || heads_q > 65535 ||
        heads_k < 1 || heads_q % heads_k || d < 8 || d > kMaxHead || d % 8)
        return false;
    const int64_t share = heads_q / heads_k;
    if (tokens_q * heads_q > kInt32Max - 65536) return false;   // rows are counted in 32 bits
    p.waves = d <= 64 ? 4 : 8;   // (24 ragged prompts of heads of 64, window and cap, by eight: 292 us for 207)
    const int rows = prompt_rows(p.waves);
    p.tiles = (tokens_q * share + B * (rows - 1)) / rows;
    p.keys = d <= 128 ? 64 : 32;
    p.least = 512 / p.keys;
    const int64_t units = p.tiles * heads_k;
    // a workgroup to a compute unit, or two of the small ones (three chunks behind up to 30000 tokens in twice as many parts: 358 us for 336;
    // from 256 workgroups on parts cost more than the longest one, 2048 tokens of 32 heads in two 91 us for 69)
    const int64_t enough = p.waves == 8 ? 256 : 512;
    int64_t parts = units >= 256 || units == 0 ? 1 : (enough + units - 1) / units;
    const int64_t most = (tokens_k / p.keys + p.least) / p.least;
    if (parts > most) parts = most;
    p.parts = (int)(parts > 64 ? 64 : parts);
    if (!launch_fits(units * p.parts, 64 * p.waves) || units * p.parts > kInt32Max) return false;
    const size_t slots = p.parts > 1 ? (size_t)units * p.parts : 0;
    p.acc = slots * rows * 2 * sizeof(float);
    p.bytes = p.acc + slots * rows * d * sizeof(float);
    if (p.bytes == 0) p.bytes = 256;
    return true;
}

template <int W, int KEYS, int WAVES, int OCC>
int launch_prompts(const PromptArgs& a, const PromptPlan& p, hipStream_t st) {
    const int lds = 6 * KEYS * FlashTile<W>::kPitch;
    const auto kernel = a.softcap > 0.0f ? attend_prompts_kernel<W, KEYS, WAVES, OCC, true> : attend_prompts_kernel<W, KEYS, WAVES, OCC, false>;
    if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                               lds) != hipSuccess)
        return RESQ_ERR_HIP;
    launch(kernel, dim3((unsigned)(p.tiles * a.heads.d * p.parts)), dim3(64 * WAVES), (size_t)lds, st, a);
    if (p.parts > 1)
        launch(attend_prompts_join_kernel<KEYS, WAVES>, dim3((unsigned)(p.tiles * a.heads.d), 16), dim3(64 * WAVES), 0, st, a);
    return launch_status();
}

// workspace of the attention behind a shared prefix: that of the own tokens' attention, its results, then the prefix's parts
struct PrefixPlan {
    int64_t tiles;   // of 256 rows
    int parts;
    size_t own, out, lse, ml, acc, bytes;
};
constexpr size_t whole(size_t n) { return (n + 255) / 256 * 256; }
bool prefix_plan(PrefixPlan& p, int64_t B, int64_t heads_q, int64_t heads_k, int64_t d) {
    p.own = resq_attend_kv_cache_workspace_bytes(B, heads_q, heads_k, d);   // 0 for sizes that it refuses
    if (p.own == 0 || B * heads_q >= 1 << 24) return false;
    p.tiles = (B * (heads_q / heads_k) + kPrefixRows - 1) / kPrefixRows;
    const int64_t units = p.tiles * heads_k;
    p.parts = units >= 256 ? 1 : (int)(256 / units);   // a workgroup to a compute unit
    p.out = whole(p.own);
    p.lse = p.out + whole((size_t)B * heads_q * d * sizeof(float));
    p.ml = p.lse + whole((size_t)B * heads_q * sizeof(float));
    p.acc = p.ml + (size_t)units * p.parts * kPrefixRows * 2 * sizeof(float);
    p.bytes = p.acc + (size_t)units * p.parts * kPrefixRows * d * sizeof(float);
    return true;
}

template <int W>
int launch_prefix(const PrefixArgs& a, const PrefixPlan& p, hipStream_t st) {
    const int lds = 6 * prefix_keys_of(W) * FlashTile<W>::kPitch;
    const auto kernel = a.softcap > 0.0f ? attend_prefix_kernel<W, true> : attend_prefix_kernel<W, false>;
    if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                               lds) != hipSuccess)
        return RESQ_ERR_HIP;
    launch(kernel, dim3((unsigned)(p.tiles * a.heads_k * p.parts)), dim3(kPrefixThreads), (size_t)lds, st, a);
    // few parts come with many queries, and then workgroups begin one after the other: 12800 queries of 4 parts 27 us by four wavefronts each, 11.6
    // by one; 2048 of 32 parts 65.4 us a call for 66.4
    const bool small = p.parts <= 8;
    launch(small ? attend_prefix_join_kernel<kPrefixJoinSmall> : attend_prefix_join_kernel<kPrefixJoinLarge>,
           dim3((unsigned)a.B * a.heads_k * a.share.d), dim3(small ? kPrefixJoinSmall : kPrefixJoinLarge), 0, st, a);
    return launch_status();
}

template <int T, int P>
int launch_norm(const NormArgs& a, bool wide, hipStream_t st) {
    constexpr int threads = T < 256 ? 256 : T;
    const int64_t blocks = (a.tokens + threads / T - 1) / (threads / T);
    if (!launch_fits(blocks, threads)) return RESQ_ERR_SHAPE;
    launch(wide ? norm_residual_kernel<T, P, float> : norm_residual_kernel<T, P, uint16_t>, dim3((unsigned)blocks), dim3(threads), 0, st, a);
    return launch_status();
}

}  // namespace

extern "C" {

size_t resq_attend_prompts_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head) {
    PromptPlan p;
    return prompt_plan(p, tokens_q, tokens_k, B, heads_q, heads_k, d_head) ? p.bytes : 0;
}

int resq_attend_prompts(const void* q, int64_t ldq, int64_t ldqh, int64_t tokens_q, const void* k, int64_t ldk, int64_t ldkh, const void* v,
                        int64_t ldv, int64_t ldvh, int64_t tokens_k, const int32_t* cu_q, const int32_t* cu_k, int64_t B, int64_t heads_q,
                        int64_t heads_k, int64_t d_head, float scale, float softcap, int64_t window, void* out, int64_t ldo, int64_t ldoh,
                        float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (tokens_k == 1 && ldk >= 0 && ldv >= 0) ldk = ldv = 0;
    PromptPlan p;
    if (!prompt_plan(p, tokens_q, tokens_k, B, heads_q, heads_k, d_head) || ldq < 0 || ldqh < 0 || ldk < 0 || ldkh < 0 || ldv < 0 ||
        ldvh < 0 || !(scale > 0.0f) || !isfinite(scale) || !(softcap == 0.0f || softcap >= FLT_MIN) || !isfinite(softcap) || window < 0 ||
        ldk >= kMaxStride || ldv >= kMaxStride || !rows_apart(tokens_q, ldo, heads_q, ldoh, d_head))
        return RESQ_ERR_SHAPE;
    if (tokens_q == 0) return RESQ_OK;
    if (!q || (tokens_k > 0 && (!k || !v)) || !cu_q || !cu_k || !out || !workspace) return RESQ_ERR_NULL;
    if (tokens_q == 1) ldq = ldo = 0;
    if (heads_q == 1) ldqh = ldoh = 0;
    if (heads_k == 1) ldkh = ldvh = 0;
    if (out == q && (ldq != ldo || ldqh != ldoh)) return RESQ_ERR_SHAPE;
    if (!aligned(q, 2) || !aligned(out, 2) || !aligned(k, 16) || !aligned(v, 16) || ldk % 8 || ldkh % 8 || ldv % 8 || ldvh % 8 ||
        !aligned(cu_q, 4) || !aligned(cu_k, 4) || !aligned(lse, 4) || !aligned(workspace, 256))
        return RESQ_ERR_ALIGN;
    if (workspace_bytes < p.bytes) return RESQ_ERR_BUFFER;
    PromptArgs a;
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.ldq = ldq;
    a.ldqh = ldqh;
    a.ldk = ldk;
    a.ldkh = ldkh;
    a.ldv = ldv;
    a.ldvh = ldvh;
    a.cu_q = cu_q;
    a.cu_k = cu_k;
    a.B = (int)B;
    a.tokens_q = (int)tokens_q;
    a.tokens_k = (int)tokens_k;
    a.heads_k = (int)heads_k;
    a.d = (int)d_head;
    a.share = FastDiv((uint32_t)(heads_q / heads_k));
    a.heads = FastDiv((uint32_t)heads_k);
    a.parts = FastDiv((uint32_t)p.parts);
    a.scale = scale;
    a.softcap = softcap;
    a.window = window > 0 && window < kMaxTokens ? (int)window : (int)kMaxTokens;
    a.least = p.least;
    a.out = static_cast<uint16_t*>(out);
    a.ldo = ldo;
    a.ldoh = ldoh;
    a.lse = lse;
    a.part_ml = static_cast<float*>(workspace);
    a.part_acc = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + p.acc);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d_head <= 64) return launch_prompts<64, 64, 4, 3>(a, p, st);
    if (d_head <= 96) return launch_prompts<96, 64, 8, 2>(a, p, st);
    if (d_head <= 128) return launch_prompts<128, 64, 8, 2>(a, p, st);
    if (d_head <= 192) return launch_prompts<192, 32, 8, 2>(a, p, st);
    return launch_prompts<256, 32, 8, 2>(a, p, st);
}

size_t resq_attend_kv_prefix_workspace_bytes(int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head) {
    PrefixPlan p;
    return prefix_plan(p, B, heads_q, heads_k, d_head) ? p.bytes : 0;
}

int resq_attend_kv_prefix(const void* q, int64_t ldq, int64_t ldqh, int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head, int64_t r,
                          const int32_t* prefix_len, const int32_t* prefix_table, int64_t prefix_width, const int32_t* lens,
                          const int32_t* block_table, int64_t ld_table, int64_t width, const void* k_pages, const void* v_pages,
                          int64_t num_pages, int64_t page_size, int64_t page_stride, int64_t head_stride, int64_t row_stride, float scale,
                          float softcap, int64_t window, void* out, int64_t ldo, int64_t ldoh, float* lse, void* workspace,
                          size_t workspace_bytes, void* stream) {
    PrefixPlan p;
    if (!prefix_plan(p, B, heads_q, heads_k, d_head) || prefix_width < 1 || prefix_width > kInt32Max || !rows_apart(B, ldo, heads_q, ldoh, d_head))
        return RESQ_ERR_SHAPE;
    if (!prefix_len || !prefix_table || !out || !workspace) return RESQ_ERR_NULL;
    if (B == 1) ldq = ldo = 0;
    if (heads_q == 1) ldqh = ldoh = 0;
    if (out == q && (ldq != ldo || ldqh != ldoh)) return RESQ_ERR_SHAPE;
    if (!aligned(prefix_len, 4) || !aligned(prefix_table, 4) || !aligned(out, 2) || !aligned(lse, 4)) return RESQ_ERR_ALIGN;
    if (workspace_bytes < p.bytes) return aligned(workspace, 256) ? RESQ_ERR_BUFFER : RESQ_ERR_ALIGN;
    uint8_t* space = static_cast<uint8_t*>(workspace);
    float *own_out = reinterpret_cast<float*>(space + p.out), *own_lse = reinterpret_cast<float*>(space + p.lse);
    // checks everything else, and launches nothing where it refuses
    const int rc = attend_kv_cache_call(q, ldq, ldqh, B, heads_q, heads_k, d_head, r, lens, block_table, ld_table, width, k_pages, v_pages, num_pages,
                                        page_size, page_stride, head_stride, row_stride, scale, softcap, window, nullptr, 0, 0, own_lse, own_out,
                                        workspace, p.own, stream);
    if (rc != RESQ_OK) return rc;
    PrefixArgs a;
    a.q = static_cast<const uint16_t*>(q);
    a.ldq = ldq;
    a.ldqh = ldqh;
    a.B = (int)B;
    a.heads_k = (int)heads_k;
    a.d = (int)d_head;
    a.r = (int)r;
    a.row_bytes = (int)(r + (d_head - r) / 2 + 16);
    a.share = FastDiv((uint32_t)(heads_q / heads_k));
    a.parts = FastDiv((uint32_t)p.parts);
    a.heads = FastDiv((uint32_t)heads_k);
    a.prefix_len = prefix_len;
    a.prefix_table = prefix_table;
    a.max_prefix = (int)(prefix_width > kMaxTokens / page_size ? kMaxTokens : prefix_width * page_size);
    a.lens = lens;
    a.max_own = (int)(width > kMaxTokens / page_size ? kMaxTokens : width * page_size);
    a.pages[0] = static_cast<const uint8_t*>(k_pages);
    a.pages[1] = static_cast<const uint8_t*>(v_pages);
    a.num_pages = (int)num_pages;
    a.page_size = FastDiv((uint32_t)page_size);
    a.page_stride = page_stride;
    a.head_stride = head_stride;
    a.row_stride = row_stride;
    a.scale = scale;
    a.softcap = softcap;
    a.window = window > 0 && window < kMaxTokens ? (int)window : (int)kMaxTokens;
    a.own_out = own_out;
    a.own_lse = own_lse;
    a.out = static_cast<uint16_t*>(out);
    a.ldo = ldo;
    a.ldoh = ldoh;
    a.lse = lse;
    a.part_ml = reinterpret_cast<float*>(space + p.ml);
    a.part_acc = reinterpret_cast<float*>(space + p.acc);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d_head <= 64) return launch_prefix<64>(a, p, st);
    if (d_head <= 96) return launch_prefix<96>(a, p, st);
    if (d_head <= 128) return launch_prefix<128>(a, p, st);
    if (d_head <= 192) return launch_prefix<192>(a, p, st);
    return launch_prefix<256>(a, p, st);
}

int resq_norm_residual(const void* y, int64_t ldy, const void* gate, int64_t ldg, const void* h, int64_t ldh, int h_is_fp32, int64_t tokens,
                       int64_t width, const void* w_pre, const void* w_post, float w_offset, float eps, float alpha, void* h_out,
                       int64_t ldho, void* x, int64_t ldx, void* stream) {
    if (tokens < 0 || width < 1 || width > kNormMaxWidth || ldy < 0 || ldg < 0 || ldh < 0 || !(eps >= 0.0f) || !isfinite(eps) ||
        !isfinite(w_offset) || !isfinite(alpha) || (tokens > 1 && ((h_out && ldho < width) || (x && ldx < width))))
        return RESQ_ERR_SHAPE;
    if (tokens == 0) return RESQ_OK;
    if (!h || (!h_out && !x) || (x && !w_pre) || ((gate || w_post) && !y)) return RESQ_ERR_NULL;
    if (tokens == 1) ldy = ldg = ldh = ldho = ldx = 0;
    if ((h_out == h && ldho != ldh) || (x && x == y && ldx != ldy)) return RESQ_ERR_SHAPE;
    const uintptr_t of_h = h_is_fp32 ? 4 : 2;
    if (!aligned(y, 2) || !aligned(gate, 2) || !aligned(h, of_h) || !aligned(h_out, of_h) || !aligned(x, 2) || !aligned(w_pre, 2) ||
        !aligned(w_post, 2))
        return RESQ_ERR_ALIGN;
    const NormArgs a{static_cast<const uint16_t*>(y), ldy, static_cast<const uint16_t*>(gate), ldg, h, ldh,
                     static_cast<const uint16_t*>(w_post), static_cast<const uint16_t*>(w_pre), w_offset, eps, alpha, h_out, ldho,
                     static_cast<uint16_t*>(x), ldx, tokens, (int)width};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool wide = h_is_fp32 != 0;
    if (width <= 512) return launch_norm<64, 1>(a, wide, st);
    if (width <= 1024) return launch_norm<128, 1>(a, wide, st);
    if (width <= 2048) return launch_norm<256, 1>(a, wide, st);
    if (width <= 4096) return launch_norm<512, 1>(a, wide, st);
    if (width <= 8192) return launch_norm<1024, 1>(a, wide, st);
    if (width <= 16384) return launch_norm<1024, 2>(a, wide, st);
    return launch_norm<1024, 4>(a, wide, st);
}

}  // extern "C"
