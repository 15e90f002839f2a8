// What the kernels around a layer's products use of the device beside hip_runtime.h's: 32x32x16 products, the transposing read of LDS, loads
// straight to LDS, and LDS at addresses of 32 bits.
#pragma once
#include <sanitizer/asan_interface.h>

#include <deque>

#include <hip/hip_runtime.h>

namespace model {

// LDS in the lowest 2 GiB, of its exact size: what is around it may not be touched
constexpr size_t kLdsRoom = 1 << 20;
inline int low_lds(void** p, size_t, size_t bytes) {
    static void* room = mmap(nullptr, kLdsRoom, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_32BIT, -1, 0);
    if (room == MAP_FAILED || bytes > kLdsRoom / 2) return 1;
    *p = static_cast<char*>(room) + kLdsRoom / 4;
    ASAN_POISON_MEMORY_REGION(room, kLdsRoom);
    ASAN_UNPOISON_MEMORY_REGION(*p, bytes);
    return 0;
}
inline void low_lds_done(void*) {}

// Loads straight to LDS of a lane, in order: at once, or, where `late`, when they are waited for.
struct Fetch {
    uint32_t to;
    const uint8_t* from;
};
inline bool late = false;
inline std::deque<Fetch> fetches[kMaxThreads];
inline void deliver(const Fetch& f) { memcpy(reinterpret_cast<void*>((uintptr_t)f.to), f.from, 16); }
inline void fetch(uint32_t to, const uint8_t* base, uint32_t off) {
    const Fetch f{to + 16 * (cur->tid & 63), base + off};
    if (late) fetches[cur->tid].push_back(f);
    else deliver(f);
}
inline void wait_but(size_t left) {   // for all but the last `left`
    auto& q = fetches[cur->tid];
    for (; q.size() > left; q.pop_front()) deliver(q.front());
}

// lane l has row (column) l % 32 of the operands, eight in a row from 8 (l / 32) on, and column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4 of
// the result
template <bool F16, typename A, typename C>
inline C mfma32(const A& a, const A& b, const C& c) {
    static float fa[kMaxThreads / 64][2][32][16], fb[kMaxThreads / 64][2][32][16];
    const int l = cur->tid & 63, w = cur->tid >> 6, p = cur->ops & 1;
    uint16_t na[8], nb[8];
    memcpy(na, &a, 16);
    memcpy(nb, &b, 16);
    auto number = [](uint16_t x) { return F16 ? (float)__builtin_bit_cast(_Float16, x) : real((uint64_t)x << 16); };
    for (int i = 0; i < 8; ++i) {
        fa[w][p][l & 31][8 * (l >> 5) + i] = number(na[i]);
        fb[w][p][l & 31][8 * (l >> 5) + i] = number(nb[i]);
    }
    meet(0x4001, 0);
    C r = c;
    for (int i = 0; i < 16; ++i) {
        const float *row = fa[w][p][8 * (i >> 2) + 4 * (l >> 5) + (i & 3)], *column = fb[w][p][l & 31];
        float s = 0.0f;
        for (int k = 0; k < 16; ++k) s += row[k] * column[k];
        r[i] += s;
    }
    return r;
}

// 16 lanes read four rows of 16 numbers, four lanes to a row; each gets one column's four
template <typename V>
inline V read_tr(V* p) {
    uint64_t mine;
    memcpy(&mine, p, 8);
    const int l = cur->tid & 63;
    const Meeting m = meet(0x4002, mine);
    uint64_t got = 0;
    for (int k = 0; k < 4; ++k) got |= (m((l & 48) + 4 * k + ((l & 15) >> 2)) >> (16 * (l & 3)) & 0xFFFF) << (16 * k);
    return __builtin_bit_cast(V, got);
}

}  // namespace model

#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) model::mfma32<false>(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, x, y, z) model::mfma32<true>(a, b, c)
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) model::read_tr(p)
#define __builtin_amdgcn_rsqf(x) (1.0f / sqrtf(x))
#define __builtin_amdgcn_fmed3f(x, lo, hi) fminf(fmaxf(x, lo), hi)   // (of NaN too: the lower bound)
