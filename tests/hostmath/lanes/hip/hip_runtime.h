// What layers.h and tc_layers.cpp need of HIP to be compiled for the host and run lane by lane, for the addresses that they form: every load and
// store is made, on memory that the sanitizer watches.  Nothing passes between lanes (a sum over them is a lane's own value, a matrix instruction returns its
// sums as they were), so that results mean nothing; LDS that a lane has not written itself holds zeros (the compiler's -ftrivial-auto-var-init=zero).
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>
#include <vector>

#define __device__
#define __host__
#define __global__
#define __shared__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __align__(n) __attribute__((aligned(n)))
#define address_space(n)
#define amdgpu_waves_per_eu(...)
#define asm
#define volatile(...)

struct dim3 {
    uint32_t x, y;
    dim3(uint64_t x_ = 1, uint64_t y_ = 1) : x((uint32_t)x_), y((uint32_t)y_) {}
};
struct uint2 { uint32_t x, y; };
struct uint4 { uint32_t x, y, z, w; };
struct float2 { float x, y; };
inline uint2 make_uint2(uint32_t x, uint32_t y) { return {x, y}; }
inline uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return {x, y, z, w}; }
inline float2 make_float2(float x, float y) { return {x, y}; }
inline dim3 threadIdx, blockIdx, gridDim;
inline void __syncthreads() {}

namespace lanes {
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
struct Rsrc {
    const char* base;
    uint32_t bytes;
};
/* a piece that begins outside the buffer reads zeros; one that begins inside has to lie inside, and in memory */
template <class V>
V load(const Rsrc& r, uint32_t offset, uint32_t from) {
    V v;
    memset(&v, 0, sizeof v);
    if (offset >= r.bytes) return v;
    if (offset + sizeof v > r.bytes) {
        fprintf(stderr, "a buffer load crosses its end: %u of %u\n", offset, r.bytes);
        abort();
    }
    memcpy(&v, r.base + offset + from, sizeof v);
    return v;
}
inline void load_to_lds(const Rsrc& r, void* lds, uint32_t size, uint32_t offset) {
    if (size != 16) abort();
    const u4 v = load<u4>(r, offset, 0);
    memcpy((char*)lds + (threadIdx.x & 63) * 16, &v, 16);
}
inline uint32_t perm(uint32_t hi, uint32_t lo, uint32_t which) {
    const uint64_t both = (uint64_t)hi << 32 | lo;
    uint32_t v = 0;
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = which >> 8 * i & 0xFF;
        v |= (w < 8 ? (uint32_t)(both >> 8 * w) & 0xFF : w == 0x0C ? 0u : 0xFFu) << 8 * i;
    }
    return v;
}
/* runs some of the workgroups of a grid, the first and last ones of each axis among them, one lane after the other */
void take_lds(size_t bytes);
extern uint32_t most_blocks;
extern bool skipped;                 /* set where not all workgroups of a launch were run */
template <class F>
void launch(dim3 grid, dim3 block, size_t lds, const F& f) {
    if (!grid.x || !grid.y || (uint64_t)grid.x * block.x > 0xFFFFFFFFull || block.x > 1024) {
        fprintf(stderr, "a launch that the runtime refuses: %u x %u of %u\n", grid.x, grid.y, block.x);
        abort();
    }
    take_lds(lds);
    gridDim = grid;
    auto some = [](uint32_t n, uint32_t most) {
        std::vector<uint32_t> v;
        if (n > most) skipped = true;
        for (uint32_t i = 0; i < n; i += n > most ? (n + most - 1) / most : 1) v.push_back(i);
        for (uint32_t i = n > 2 ? n - 2 : 0; i < n; ++i)
            if (std::find(v.begin(), v.end(), i) == v.end()) v.push_back(i);
        return v;
    };
    const auto ys = some(grid.y, most_blocks), xs = some(grid.x, most_blocks);
    for (uint32_t y : ys)
        for (uint32_t x : xs) {
            blockIdx = dim3(x, y);
            for (uint32_t t = 0; t < block.x; ++t) {
                threadIdx = dim3(t, 0);
                f();
            }
        }
}
}  // namespace lanes
typedef lanes::Rsrc __amdgpu_buffer_rsrc_t;
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, n, flags) (lanes::Rsrc{(const char*)(p), (uint32_t)(n)})
#define __builtin_amdgcn_raw_buffer_load_b16(r, o, s, a) lanes::load<uint16_t>(r, o, s)
#define __builtin_amdgcn_raw_buffer_load_b64(r, o, s, a) lanes::load<lanes::u2>(r, o, s)
#define __builtin_amdgcn_raw_buffer_load_b128(r, o, s, a) lanes::load<lanes::u4>(r, o, s)
#define __builtin_amdgcn_raw_ptr_buffer_load_lds(r, l, n, o, s, i, a) lanes::load_to_lds(r, (void*)(l), n, o)
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) (*(p))
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_readfirstlane(v) (v)
#define __builtin_amdgcn_readlane(v, l) (v)
#define __builtin_amdgcn_mov_dpp(v, c, r, b, z) (v)
#define __builtin_amdgcn_perm(a, b, s) lanes::perm(a, b, s)
#define __builtin_amdgcn_alignbit(h, l, s) (uint32_t)((((uint64_t)(h) << 32 | (l)) >> ((s) & 31)))
#define __builtin_amdgcn_rcpf(x) (1.0f / (x))
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_frexp_mantf(x) lanes_mant(x)
#define __builtin_amdgcn_frexp_expf(x) lanes_exp(x)
#define __builtin_amdgcn_fence(...)
#define __builtin_amdgcn_sched_group_barrier(...)
inline int lanes_exp(float x) {
    int e = 0;
    if (std::isfinite(x)) (void)frexpf(x, &e);
    return e;
}
inline float lanes_mant(float x) {
    int e;
    return std::isfinite(x) ? frexpf(x, &e) : x;
}
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) lanes::launch(grid, block, lds, [&] { (kernel)(__VA_ARGS__); })
inline int hipGetLastError() { return 0; }
enum { hipFuncAttributeMaxDynamicSharedMemorySize };
inline int hipFuncSetAttribute(const void*, int, int) { return 0; }
