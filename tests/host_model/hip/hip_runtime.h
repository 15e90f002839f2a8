// A host model of what the kernels of the generation step use of the device: a workgroup's threads run as coroutines, the lanes of a
// wavefront meet at every exchange and every workgroup at its barriers, so that the kernels' own source runs on the CPU, built with
// the sanitizers for addresses and undefined behaviour.  Every buffer, LDS too, is a host allocation of its exact size.
// It knows nothing of time: between two meetings a lane runs alone, and what the source leaves to lockstep without a barrier
// between it is in the order of the lanes here.
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <sys/mman.h>

#include <algorithm>
#include <functional>
#include <vector>

#define __host__
#define __device__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static

// vectors of the compiler's own, whose alignment its sanitizer knows
typedef uint32_t uint2 __attribute__((ext_vector_type(2)));
typedef uint32_t uint4 __attribute__((ext_vector_type(4)));
typedef float float2 __attribute__((ext_vector_type(2)));
typedef float float4 __attribute__((ext_vector_type(4)));
inline uint2 make_uint2(uint32_t x, uint32_t y) { return (uint2){x, y}; }
inline uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return (uint4){x, y, z, w}; }
inline float2 make_float2(float x, float y) { return (float2){x, y}; }
inline float4 make_float4(float x, float y, float z, float w) { return (float4){x, y, z, w}; }
struct dim3 {
    uint32_t x, y, z;
    dim3(uint32_t x_ = 1, uint32_t y_ = 1, uint32_t z_ = 1) : x(x_), y(y_), z(z_) {}
};
using std::max;
using std::min;

namespace model {

[[noreturn]] inline void fail(const char* what) {
    fprintf(stderr, "host model: %s\n", what);
    abort();
}

// ---- coroutines ----------------------------------------------------------------------------------
// Only what a call has to keep is kept: the stack pointer, and on the stack the registers that a function leaves as they were.
extern "C" void model_switch(void** from, void* to);
__asm__(R"(
.text
.globl model_switch
.type model_switch, @function
model_switch:
    pushq %rbp
    pushq %rbx
    pushq %r12
    pushq %r13
    pushq %r14
    pushq %r15
    movq %rsp, (%rdi)
    movq %rsi, %rsp
    popq %r15
    popq %r14
    popq %r13
    popq %r12
    popq %rbx
    popq %rbp
    ret
)");

constexpr int kMaxThreads = 256;
constexpr size_t kStack = 1 << 20;
enum State { kReady, kAtBarrier, kDone };

struct Thread {
    void* sp;
    char* stack;
    State state;
    int ops;          // meetings of its wavefront so far
    uint32_t tid;
};
struct Wave {
    uint64_t slot[2][64][2];   // what the lanes bring to a meeting, by its parity (a lane is at most one ahead of another)
    int tag[2][64];
};
inline Thread threads[kMaxThreads];
inline Wave waves[kMaxThreads / 64];
inline Thread* cur;
inline void* scheduler;
inline dim3 block_idx, block_dim, grid_dim;
inline const std::function<void()>* body;
inline uint8_t* lds;

inline void to_scheduler() { model_switch(&cur->sp, scheduler); }
inline void entry() {
    (*body)();
    cur->state = kDone;
    while (true) to_scheduler();
}
// All lanes of the wavefront bring two words; afterwards lane l's are read by from(l).
struct Meeting {
    const Wave& w;
    int p;
    uint64_t operator()(int lane, int word = 0) const { return w.slot[p][lane & 63][word]; }
};
inline Meeting meet(int tag, uint64_t a, uint64_t b = 0) {
    Thread* me = cur;
    Wave& w = waves[me->tid >> 6];
    const int p = me->ops++ & 1, lane = me->tid & 63;
    w.slot[p][lane][0] = a;
    w.slot[p][lane][1] = b;
    w.tag[p][lane] = tag;
    to_scheduler();
    for (int l = 0; l < 64; ++l)
        if (w.tag[p][l] != tag) fail("lanes of a wavefront met at different places");
    return Meeting{w, p};
}
inline void barrier() {
    cur->state = kAtBarrier;
    to_scheduler();
}
inline void run_block(int n) {
    for (int t = 0; t < n; ++t) {
        Thread& th = threads[t];
        if (!th.stack) {
            th.stack = static_cast<char*>(mmap(nullptr, kStack, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0));
            if (th.stack == MAP_FAILED) fail("no memory for a stack");
        }
        void** sp = reinterpret_cast<void**>(th.stack + kStack - 64);
        *--sp = nullptr;   // entry() does not return
        *--sp = reinterpret_cast<void*>(&entry);
        for (int i = 0; i < 6; ++i) *--sp = nullptr;
        th.sp = sp;
        th.state = kReady;
        th.ops = 0;
        th.tid = t;
    }
    while (true) {
        bool done = true, waiting = true;
        for (int w = 0; w < n / 64; ++w) {
            Thread *t = threads + 64 * w, *live = nullptr;
            for (bool ready = true; ready;) {   // the lanes in turn, from one meeting to the next
                ready = false;
                live = nullptr;
                for (int l = 0; l < 64; ++l) {
                    if (t[l].state != kReady) continue;
                    cur = t + l;
                    model_switch(&scheduler, cur->sp);
                }
                for (int l = 0; l < 64; ++l) {
                    if (t[l].state == kDone) continue;
                    if (live && (t[l].state != live->state || t[l].ops != live->ops)) fail("lanes of a wavefront parted");
                    live = t + l;
                    ready = t[l].state == kReady;
                }
            }
            done &= !live;
            waiting &= live != nullptr;
        }
        if (done) return;
        if (!waiting) fail("a wavefront ended in front of a barrier");
        for (int t = 0; t < n; ++t)
            if (threads[t].state == kAtBarrier) threads[t].state = kReady;
    }
}
// One launch, workgroup after workgroup.  LDS holds something before, as it does on the device.
template <typename F>
inline void launch(F f, dim3 grid, dim3 block, size_t lds_bytes) {
    if (block.x > kMaxThreads || block.x % 64) fail("a workgroup of another size");
    const std::function<void()> call = f;
    body = &call;
    block_dim = block;
    grid_dim = grid;
    for (uint32_t y = 0; y < grid.y; ++y)
        for (uint32_t x = 0; x < grid.x; ++x) {
            block_idx = dim3(x, y);
            void* p = nullptr;
            if (lds_bytes && posix_memalign(&p, 16, lds_bytes)) fail("no memory for LDS");
            if (p) memset(p, 0xFF, lds_bytes);
            lds = static_cast<uint8_t*>(p);
            run_block((int)block.x);
            free(lds);
        }
}

inline uint64_t bits(float x) { uint32_t u; memcpy(&u, &x, 4); return u; }
inline float real(uint64_t x) { const uint32_t u = (uint32_t)x; float f; memcpy(&f, &u, 4); return f; }

// the lane that data-parallel-primitive control `ctrl` reads for lane l, or -1
inline int dpp_source(int ctrl, int l) {
    const int row = l & ~15, i = l & 15;
    if (ctrl <= 0xFF) return (l & ~3) | (ctrl >> (2 * (l & 3)) & 3);                       // quad_perm
    if (ctrl > 0x110 && ctrl < 0x120) return i >= (ctrl & 15) ? l - (ctrl & 15) : -1;      // row_shr
    if (ctrl > 0x120 && ctrl < 0x130) return row | ((i - (ctrl & 15)) & 15);               // row_ror
    if (ctrl == 0x140) return row | (15 - i);                                              // row_mirror
    if (ctrl == 0x141) return row | (i & 8) | (7 - (i & 7));                               // row_half_mirror
    if (ctrl == 0x142) return l >= 16 ? row - 1 : -1;                                      // row_bcast:15
    if (ctrl == 0x143) return l >= 32 ? 31 : -1;                                           // row_bcast:31
    fail("a lane exchange that is not modelled");
}
inline int update_dpp(int old, int x, int ctrl, int row_mask, int bank_mask, bool zero) {
    const int l = cur->tid & 63;
    const Meeting m = meet(0x1000 + ctrl, (uint32_t)x);
    if (!(row_mask >> (l >> 4) & 1) || !(bank_mask >> ((l >> 2) & 3) & 1)) return old;
    const int from = dpp_source(ctrl, l);
    return from < 0 ? (zero ? 0 : old) : (int)(uint32_t)m(from);
}
inline int swizzle(int x, int pattern) {
    const int l = cur->tid & 63;
    const Meeting m = meet(0x2000, (uint32_t)x);
    return (int)(uint32_t)m((l & 32) | ((((l & 31) & (pattern & 31)) | (pattern >> 5 & 31)) ^ (pattern >> 10 & 31)));
}
inline uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) {
    const uint64_t both = (uint64_t)hi << 32 | lo;
    uint32_t r = 0;
    for (int i = 0; i < 4; ++i) {
        const uint32_t s = sel >> (8 * i) & 0xFF;
        if (s > 7 && s != 0x0C) fail("a byte selector that is not modelled");
        r |= (s == 0x0C ? 0u : (uint32_t)(both >> (8 * s)) & 0xFFu) << (8 * i);
    }
    return r;
}
struct Pair { uint32_t v[2]; uint32_t operator[](int i) const { return v[i]; } };
// odd rows of the first operand change places with even rows of the second (16), its upper half with the lower one (32)
template <int N>
inline Pair permlane_swap(uint32_t x, uint32_t y) {
    const int l = cur->tid & 63;
    const Meeting m = meet(0x3000 + N, x, y);
    return l & N ? Pair{{(uint32_t)m(l - N, 1), y}} : Pair{{x, (uint32_t)m(l + N, 0)}};
}
// lane l has row (column) l % 16 of the operands, eight in a row from 8 (l / 16) on, and column l % 16, rows 4 (l / 16) + i of the result
template <typename A, typename C>
inline C mfma(const A& a, const A& b, const C& c) {
    uint32_t wa[4], wb[4];
    memcpy(wa, &a, 16);
    memcpy(wb, &b, 16);
    const int l = cur->tid & 63;
    static float fa[kMaxThreads / 64][2][64][8], fb[kMaxThreads / 64][2][64][8];
    const int wv = cur->tid >> 6, p = cur->ops & 1;
    for (int i = 0; i < 8; ++i) {
        fa[wv][p][l][i] = real((uint64_t)(wa[i >> 1] >> (16 * (i & 1)) & 0xFFFF) << 16);
        fb[wv][p][l][i] = real((uint64_t)(wb[i >> 1] >> (16 * (i & 1)) & 0xFFFF) << 16);
    }
    meet(0x4000, 0);
    C r = c;
    for (int i = 0; i < 4; ++i) {
        float s = 0.0f;
        for (int k = 0; k < 32; ++k) s += fa[wv][p][(k >> 3) * 16 + 4 * (l >> 4) + i][k & 7] * fb[wv][p][(k >> 3) * 16 + (l & 15)][k & 7];
        r[i] += s;
    }
    return r;
}

}  // namespace model

#define threadIdx (dim3(model::cur->tid))
#define blockIdx (model::block_idx)
#define blockDim (model::block_dim)
#define gridDim (model::grid_dim)
inline void __syncthreads() { model::barrier(); }
inline int __shfl(int x, int l) { return (int)(uint32_t)model::meet(0x5000, (uint32_t)x)(l); }
inline float __shfl(float x, int l) { return model::real(model::meet(0x5000, model::bits(x))(l)); }
inline float __shfl_xor(float x, int mask) { return model::real(model::meet(0x5001, model::bits(x))((model::cur->tid & 63) ^ mask)); }
inline uint32_t __float_as_uint(float x) { return (uint32_t)model::bits(x); }
inline int __float_as_int(float x) { return (int)model::bits(x); }
inline float __uint_as_float(uint32_t x) { return model::real(x); }
inline float __int_as_float(int x) { return model::real((uint32_t)x); }
inline int atomicOr(int* p, int v) { const int old = *p; *p |= v; return old; }
inline void sincospif(float x, float* s, float* c) {
    *s = (float)sin(M_PI * (double)x);
    *c = (float)cos(M_PI * (double)x);
}

#define __builtin_amdgcn_update_dpp(old, x, ctrl, rows, banks, zero) model::update_dpp((int)(old), (int)(x), ctrl, rows, banks, zero)
#define __builtin_amdgcn_ds_swizzle(x, pattern) model::swizzle(x, pattern)
#define __builtin_amdgcn_perm(a, b, sel) model::perm(a, b, sel)
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_rcpf(x) (1.0f / (x))
#define __builtin_amdgcn_permlane16_swap(x, y, a, b) model::permlane_swap<16>(x, y)
#define __builtin_amdgcn_permlane32_swap(x, y, a, b) model::permlane_swap<32>(x, y)
#define __builtin_amdgcn_readfirstlane(x) ((int)(uint32_t)model::meet(0x6000, (uint32_t)(x))(0))
#define __builtin_amdgcn_readlane(x, l) ((int)(uint32_t)model::meet(0x6001, (uint32_t)(x))(l))
#define __builtin_amdgcn_sched_barrier(x) ((void)0)
#define __builtin_amdgcn_fence(...) ((void)0)
#define __builtin_amdgcn_wave_barrier() ((void)model::meet(0x6002, 0))
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) model::mfma(a, b, c)
inline uint64_t model_ballot(bool x) {
    const model::Meeting m = model::meet(0x6003, x);
    uint64_t r = 0;
    for (int l = 0; l < 64; ++l) r |= (m(l) & 1) << l;
    return r;
}
#define __builtin_amdgcn_ballot_w64(x) model_ballot(x)
// round to nearest even, as the device's conversion does
extern "C" __bf16 __truncsfbf2(float x) {
    const uint32_t u = (uint32_t)model::bits(x);
    const uint16_t r = x != x ? (uint16_t)(u >> 16 | 0x40) : (uint16_t)((u + 0x7FFF + (u >> 16 & 1)) >> 16);
    return __builtin_bit_cast(__bf16, r);
}

// ---- what the entry points use of the runtime ------------------------------------------------------
typedef void* hipStream_t;
typedef void* hipEvent_t;
typedef int hipError_t;
constexpr int hipSuccess = 0, hipFuncAttributeMaxDynamicSharedMemorySize = 0;
inline int hipGetLastError() { return hipSuccess; }
inline int hipFuncSetAttribute(const void*, int, int) { return hipSuccess; }
template <typename... KArgs, typename... Args>
inline void hipExtLaunchKernelGGL(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t lds_bytes, hipStream_t, hipEvent_t, hipEvent_t, int,
                                  Args... args) {
    model::launch([=] { kernel(args...); }, grid, block, lds_bytes);
}

// empty assembly, by which the kernels keep values from the compiler
#define asm
#define volatile(...)
