/*
 * Kernels of the layer operators (gfx950): 8-bit checkpoints, norms and their gradients, matrix products with their
 * epilogue and their gradients.
 */
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace tc {
namespace layers {

typedef float f4 __attribute__((ext_vector_type(4)));
template <class T> struct Vec {
    typedef T v8 __attribute__((ext_vector_type(8)));
};

/* ---- activations: value and slope ------------------------------------------------------------------
 * The upper tail of the normal distribution is exp(-a^2 / 2) R(a), where R falls slowly from 1/2 to 0.4 / a: t times a polynomial of degree 7 in
 * t = 1 / (1 + 0.3 a), whose coefficients make the largest relative error over 0 <= a <= 13.5 least (1.3e-7; found by linear programming over 3000 points; with float32
 * roundings 4.3e-7).  So values far below zero are rounded to their type once too, down to float32's normal range, where the tail becomes 0 (z < -13.2).  gelu = max(z, 0) - |z| tail: some
 * 25 operations, where the library's erf alone takes 40; in the epilogue of a product of 8192 x 4096 -> 11008 (z kept) they add 56 us to 618.  |z| is held at 14, beyond
 * which every factor has become 0, so that infinities (values before the activation that overflowed) do not turn into NaNs; NaNs stay. */
__device__ __forceinline__ float held_at_14(float z) {
    const float a = fabsf(z);
    return a > 14.0f ? 14.0f : a;
}
__device__ __forceinline__ float normal_tail(float a, float& bell) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, a, 1.0f));
    bell = __builtin_amdgcn_exp2f(-0.72134752044448170f * (a * a));
    float s = 0.035931729f;
    s = fmaf(t, s, -0.158275947f);
    s = fmaf(t, s, 0.208206490f);
    s = fmaf(t, s, -0.055393755f);
    s = fmaf(t, s, 0.129469156f);
    s = fmaf(t, s, 0.099637508f);
    s = fmaf(t, s, 0.120798364f);
    s = fmaf(t, s, 0.119626395f);
    return bell * (t * s);
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z)); }
__device__ __forceinline__ float activate(float z, int act) {
    if (act == TC_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (act == TC_ACT_GELU) {
        float bell;
        const float a = held_at_14(z);
        return fmaf(-a, normal_tail(a, bell), z < 0.0f ? 0.0f : z);
    }
    if (act == TC_ACT_SILU) return (z < -104.0f ? -104.0f : z) * sigmoid(z);
    return z;
}
__device__ __forceinline__ float slope(float z, int act) {
    if (act == TC_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    if (act == TC_ACT_GELU) {
        float bell;
        const float a = held_at_14(z), tail = normal_tail(a, bell);
        return fmaf(copysignf(a, z), 0.3989422804014327f * bell, z < 0.0f ? tail : 1.0f - tail);
    }
    if (act == TC_ACT_SILU) {
        const float s = sigmoid(z), far = z < -104.0f ? -104.0f : z > 104.0f ? 104.0f : z;
        return fmaf(far, s * (1.0f - s), s);
    }
    return 1.0f;
}

/* ---- sums and maxima of a wave or of the waves that share a row --------------------------------------
 * Within sixteen lanes by moves between neighbours (one instruction each, no LDS), the four sixteens through scalar registers. */
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float lane_of(float v, int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); }
__device__ __forceinline__ float wave_sum(float v) {
    v += moved<0xB1>(v);         /* the other one of a pair, the other pair of four */
    v += moved<0x4E>(v);
    v += moved<0x141>(v);        /* eight lanes mirrored, sixteen lanes mirrored */
    v += moved<0x140>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, moved<0xB1>(v));
    v = fmaxf(v, moved<0x4E>(v));
    v = fmaxf(v, moved<0x141>(v));
    v = fmaxf(v, moved<0x140>(v));
    return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
/* TH lanes of the workgroup (TH / 64 whole waves) together.  cells: TH / 64 floats of LDS of this group that nobody else uses between this
 * call's barrier and a later one; every lane of the workgroup makes the call. */
template <int TH>
__device__ __forceinline__ float group_sum(float v, float* cells, int t) {
    v = wave_sum(v);
    if (TH == 64) return v;
    if ((t & 63) == 0) cells[t >> 6] = v;
    __syncthreads();
    v = cells[0];
    for (int w = 1; w < TH / 64; ++w) v += cells[w];
    return v;
}
template <int TH>
__device__ __forceinline__ float group_max(float v, float* cells, int t) {
    v = wave_max(v);
    if (TH == 64) return v;
    if ((t & 63) == 0) cells[t >> 6] = v;
    __syncthreads();
    v = cells[0];
    for (int w = 1; w < TH / 64; ++w) v = fmaxf(v, cells[w]);
    return v;
}
/* two sums at one barrier */
template <int TH>
__device__ __forceinline__ void group_sum2(float& u, float& v, float2* cells, int t) {
    u = wave_sum(u);
    v = wave_sum(v);
    if (TH == 64) return;
    if ((t & 63) == 0) cells[t >> 6] = make_float2(u, v);
    __syncthreads();
    u = cells[0].x;
    v = cells[0].y;
    for (int w = 1; w < TH / 64; ++w) {
        u += cells[w].x;
        v += cells[w].y;
    }
}

/* ---- rows in registers -------------------------------------------------------------------------------
 * TH lanes hold a row of at most TH * 8 * NCH entries, 8 NCH to a lane: lane t's chunk c is the eight entries from (c TH + t) 8 on, one
 * access of 16 bytes (8 bytes of int8), at any address that is aligned to an entry.  Rows are kept as they were read and unpacked when used. */
template <class V>
__device__ __forceinline__ V unaligned(const void* p) {
    V v;
    __builtin_memcpy(&v, p, sizeof v);
    return v;
}
/* Eight entries of which only the last `count` are wanted, moved to the front, zeros behind them.  The last piece of a row is read as
 * the row's last eight entries (which are all there) and moved so. */
__device__ __forceinline__ void to_front(uint32_t (&w)[4], uint32_t count) {
    const uint32_t n = 8 - count;
    if (n & 4) {
        w[0] = w[2];
        w[1] = w[3];
        w[2] = w[3] = 0;
    }
    if (n & 2) {
        w[0] = w[1];
        w[1] = w[2];
        w[2] = w[3];
        w[3] = 0;
    }
    if (n & 1) {
#pragma unroll
        for (int i = 0; i < 3; ++i) w[i] = w[i] >> 16 | w[i + 1] << 16;
        w[3] >>= 16;
    }
}
__device__ __forceinline__ void to_front(uint32_t (&w)[2], uint32_t count) {
    const uint32_t n = 8 - count, s = (n & 3) * 8;
    if (n & 4) {
        w[0] = w[1];
        w[1] = 0;
    }
    w[0] = __builtin_amdgcn_alignbit(w[1], w[0], s);
    w[1] >>= s;
}
/* the first `count` of the eight entries from p on, one by one, zeros behind them: for rows that have fewer than eight */
__device__ __forceinline__ void read_piece(const uint16_t* p, uint32_t count, uint32_t (&w)[4]) {
    w[0] = w[1] = w[2] = w[3] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if ((uint32_t)j < count) w[j >> 1] |= (uint32_t)p[j] << (j & 1) * 16;
}
__device__ __forceinline__ void read_piece(const uint8_t* p, uint32_t count, uint32_t (&w)[2]) {
    w[0] = w[1] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if ((uint32_t)j < count) w[j >> 2] |= (uint32_t)p[j] << (j & 3) * 8;
}
template <int TH>
__device__ __forceinline__ uint32_t row_col(int t, int c) { return ((uint32_t)c * TH + t) * 8; }
__device__ __forceinline__ uint32_t entries_at(uint32_t k, uint32_t cols) { return k >= cols ? 0 : cols - k < 8 ? cols - k : 8; }
template <class T, int TH, bool SHORT>
struct Raw {
    uint32_t w[4];
    __device__ __forceinline__ void load(const T* p, int t, int c, uint32_t cols) {
        const uint32_t k = row_col<TH>(t, c);
        if (SHORT) {
            read_piece((const uint16_t*)p + k, entries_at(k, cols), w);
            return;
        }
        uint4 x = make_uint4(0, 0, 0, 0);
        if (k < cols) x = unaligned<uint4>(p + (k + 8 <= cols ? k : cols - 8));
        w[0] = x.x;
        w[1] = x.y;
        w[2] = x.z;
        w[3] = x.w;
    }
    /* once all loads are under way: the last piece of a row that is no whole number of pieces */
    __device__ __forceinline__ void trim(int t, int c, uint32_t cols) {
        if (SHORT || (cols & 7) == 0) return;
        const uint32_t count = entries_at(row_col<TH>(t, c), cols);
        if (count && count < 8) to_front(w, count);
    }
    __device__ __forceinline__ float get(int j) const { return (float)__builtin_bit_cast(T, (uint16_t)(w[j >> 1] >> (j & 1) * 16)); }
    /* from here on the values are unpacked anew, not kept */
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(w[i]));
    }
};
template <int TH, bool SHORT>
struct RawQ {
    uint32_t w[2];
    __device__ __forceinline__ void load(const int8_t* p, int t, int c, uint32_t cols) {
        const uint32_t k = row_col<TH>(t, c);
        if (SHORT) {
            read_piece((const uint8_t*)p + k, entries_at(k, cols), w);
            return;
        }
        uint2 x = make_uint2(0, 0);
        if (k < cols) x = unaligned<uint2>(p + (k + 8 <= cols ? k : cols - 8));
        w[0] = x.x;
        w[1] = x.y;
    }
    /* once all loads are under way: the last piece of a row that is no whole number of pieces */
    __device__ __forceinline__ void trim(int t, int c, uint32_t cols) {
        if (SHORT || (cols & 7) == 0) return;
        const uint32_t count = entries_at(row_col<TH>(t, c), cols);
        if (count && count < 8) to_front(w, count);
    }
    __device__ __forceinline__ float get(int j) const { return (float)((int)(w[j >> 2] << (24 - (j & 3) * 8)) >> 24); }
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(w[i]));
    }
};
template <class T, int TH, bool SHORT>
__device__ __forceinline__ void load8(const T* p, int t, int c, uint32_t cols, float* v) {
    Raw<T, TH, SHORT> r;
    r.load(p, t, c, cols);
    r.trim(t, c, cols);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = r.get(j);
}
template <int TH, bool SHORT>
__device__ __forceinline__ void load8q(const int8_t* p, float scale, int t, int c, uint32_t cols, float* v) {
    RawQ<TH, SHORT> r;
    r.load(p, t, c, cols);
    r.trim(t, c, cols);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = scale * r.get(j);
}
/* eight values to entries k .. of a row of n; `past`: past the caches */
template <class T>
__device__ __forceinline__ void put8(T* row, uint32_t k, uint32_t n, const float* v, bool past = false) {
    typedef typename Vec<T>::v8 anywhere __attribute__((aligned(2)));
    typename Vec<T>::v8 x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (T)v[j];
    if (k + 8 <= n) {
        if (past) {
            asm volatile("");            /* (else the compiler makes one plain store of the two) */
            __builtin_nontemporal_store(x, (anywhere*)(row + k));
        } else *(anywhere*)(row + k) = x;
    } else
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (k + j < n) row[k + j] = x[j];
}
template <class T, int TH>
__device__ __forceinline__ void store8(T* p, int t, int c, uint32_t cols, const float* v, bool past = false) { put8<T>(p, row_col<TH>(t, c), cols, v, past); }

/* ---- 8-bit checkpoints ------------------------------------------------------------------------------- */
struct RowArgs {
    const void* src;
    void* dst;
    float* scale;
    uint64_t ld_src, ld_dst;
    uint32_t rows, cols;
    bool past;                       /* the 16-bit output goes past the caches */
};
/* The row is scaled by a power of two so that amax, the largest finite magnitude, lies in [1, 2): nothing overflows or gets lost (but entries
 * below 2^-126 of amax, whose q is 0 either way).  x and amax have at most 11 significant bits, so t = 127 x has 18 and is exact in
 * float32, and a quotient t / amax that is not half way between two whole numbers is at least 2^-20 of itself away from that.  One correction of
 * t (1 / amax) by the exact remainder gives a quotient within 2^-23 of itself, and exactly the quotient where that is half a whole
 * number: rounding it, half to even, is then rounding t / amax.  Added to 1.5 * 2^23 its low byte is q.
 * Rows with infinities or NaNs, or an amax out of the range of these scalings, take the careful way: q from the whole number next to the quotient by the
 * sign of the remainder t - q amax.
 * Bound by memory, some ten operations an entry: 8192 x 11008 in 58 us, 4.7 GB a millisecond (29 operations an entry, the careful way for all: 107 us).  Rows longer than the registers hold (NCH = 0) are read twice. */
__device__ __forceinline__ float quantised(float x, float amax, float inv, int e) {
    const float t = 127.0f * ldexpf(x, e);
    float q = rintf(t * inv);
    const float r = 2.0f * fmaf(-q, amax, t);
    const float toward = r > 0.0f ? 1.0f : -1.0f;
    const bool over = fabsf(r) > amax;
    const bool tie = fabsf(r) == amax && ((int)q & 1);
    if (over || tie) q += toward;
    q = fminf(fmaxf(q, -127.0f), 127.0f);
    return x != x ? 0.0f : (fabsf(x) == INFINITY ? copysignf(127.0f, x) : q);
}
__device__ __forceinline__ float finite_magnitude(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.0f;
}
template <class T, int TH, int NCH, bool SHORT = false>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void checkpoint_encode(const RowArgs a) {
    __shared__ float cells[2][16];
    const int t = threadIdx.x % TH;
    constexpr uint32_t SETS = TH < 256 ? 256 / TH : 1;
    const int chunks = NCH ? NCH : (a.cols + TH * 8 - 1) / (TH * 8);
    /* where waves share a row, all of them run the same rounds; where they do not, there is no barrier */
    for (uint64_t row = (uint64_t)blockIdx.x * SETS + threadIdx.x / TH; row < a.rows; row += (uint64_t)gridDim.x * SETS) {
        const T* src = (const T*)a.src + row * a.ld_src;
        int8_t* dst = (int8_t*)a.dst + row * a.ld_dst;
        Raw<T, TH, SHORT> x[NCH ? NCH : 1];
        /* magnitudes compare like their bits, two at a time */
        typedef uint16_t s2 __attribute__((ext_vector_type(2)));
        s2 top = {0, 0};
#pragma unroll
        for (int c = 0; c < (NCH ? NCH : 1); ++c) x[c].load(src, t, c, a.cols);
        for (int c = 0; c < chunks; ++c) {
            if (!NCH) x[0].load(src, t, c, a.cols);
            x[NCH ? c : 0].trim(t, c, a.cols);
#pragma unroll
            for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(s2, x[NCH ? c : 0].w[i] & 0x7FFF7FFFu));
        }
        float m = fmaxf((float)top[0], (float)top[1]);                                 /* bits as whole numbers, exact */
        m = group_max<TH>(m, cells[0], t);
        const uint16_t bits = (uint16_t)m;
        m = (float)__builtin_bit_cast(T, bits);
        const bool numbers = m < INFINITY;
        if (!numbers) {
            m = 0.0f;
            for (int c = 0; c < chunks; ++c) {
                if (!NCH) {
                    x[0].load(src, t, c, a.cols);
                    x[0].trim(t, c, a.cols);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) m = fmaxf(m, finite_magnitude(x[NCH ? c : 0].get(j)));
            }
            m = group_max<TH>(m, cells[1], t);
        }
        if (t == 0) a.scale[row] = m / 127.0f;
        const int e = m > 0.0f ? -ilogbf(m) : 0;
        const float amax = m > 0.0f ? ldexpf(m, e) : 1.0f, inv = 1.0f / amax;
        const bool plain = numbers && e > -100 && e < 100;
        const float times127 = plain ? ldexpf(127.0f, e) : 0.0f, quick = times127 * inv;
        for (int c = 0; c < chunks; ++c) {
            if (!NCH) {
                x[0].load(src, t, c, a.cols);
                x[0].trim(t, c, a.cols);
            }
            const Raw<T, TH, SHORT>& r = x[NCH ? c : 0];
            uint32_t q[8];
            if (plain) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float v = r.get(j), n = v * times127, near = v * quick;
                    q[j] = __builtin_bit_cast(uint32_t, fmaf(fmaf(-near, amax, n), inv, near) + 12582912.0f);
                }
            } else {
                for (int j = 0; j < 8; ++j) q[j] = (uint32_t)(int)quantised(r.get(j), amax, inv, e);
            }
            {
                const uint32_t k = row_col<TH>(t, c);
                uint2 w;
                w.x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0C0C0400u), __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u), 0x05040100u);
                w.y = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[7], q[6], 0x0C0C0400u), __builtin_amdgcn_perm(q[5], q[4], 0x0C0C0400u), 0x05040100u);
                if (k + 8 <= a.cols) __builtin_memcpy(dst + k, &w, 8);
                else
#pragma unroll
                    for (int j = 0; j < 7; ++j)
                        if (k + j < a.cols) dst[k + j] = (int8_t)q[j];
            }
        }
        if (TH > 64) __syncthreads();                    /* the cells are free again */
    }
}
/* 256 lanes take 2048 entries of a row */
template <class T, bool SHORT>
__global__ __launch_bounds__(256) void checkpoint_decode(const RowArgs a) {
    for (uint64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        float v[8];
        load8q<256, SHORT>((const int8_t*)a.src + row * a.ld_src, a.scale[row], threadIdx.x, blockIdx.x, a.cols, v);
        store8<T, 256>((T*)a.dst + row * a.ld_dst, threadIdx.x, blockIdx.x, a.cols, v, a.past);
    }
}

/* ---- norms --------------------------------------------------------------------------------------------
 * A row is read once and stays in registers: its mean, then the mean square about it (no difference of large sums), then y.
 * Short calls are launches (one row of 4096: 2.3 us in the kernel, 4.6 a call); 487 x 4096 4.3 us. */
struct NormArgs {
    const void* x;
    const float* scale;              /* x is int8 where this is set */
    const void *gamma, *beta;
    void* y;
    float *mean, *rstd;
    uint64_t ldx, ldy;
    uint32_t rows, cols;
    float eps;
    int centred;
};
template <class T, int TH, int NCH, bool SHORT = false>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void norm_forward(const NormArgs a) {
    __shared__ float cells[2][16];
    const int t = threadIdx.x % TH;
    constexpr uint32_t SETS = TH < 256 ? 256 / TH : 1;
    const float per = 1.0f / (float)a.cols;
    Raw<T, TH, SHORT> g[NCH], b[NCH];                 /* under way while the sums are formed */
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        if (a.gamma) g[c].load((const T*)a.gamma, t, c, a.cols);
        if (a.beta) b[c].load((const T*)a.beta, t, c, a.cols);
    }
    bool trimmed = false;
    for (uint64_t row = (uint64_t)blockIdx.x * SETS + threadIdx.x / TH; row < a.rows; row += (uint64_t)gridDim.x * SETS) {
        float x[NCH][8];
        if (a.scale) {
            const float scale = a.scale[row];
            RawQ<TH, SHORT> r[NCH];
#pragma unroll
            for (int c = 0; c < NCH; ++c) r[c].load((const int8_t*)a.x + row * a.ldx, t, c, a.cols);
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                r[c].trim(t, c, a.cols);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] = scale * r[c].get(j);
            }
        } else {
            Raw<T, TH, SHORT> r[NCH];
#pragma unroll
            for (int c = 0; c < NCH; ++c) r[c].load((const T*)a.x + row * a.ldx, t, c, a.cols);
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                r[c].trim(t, c, a.cols);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] = r[c].get(j);
            }
        }
        float mean = 0.0f;
        if (a.centred) {
            float s = 0.0f;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) s += x[c][j];
            mean = group_sum<TH>(s, cells[0], t) * per;
        }
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = row_col<TH>(t, c) + j < a.cols ? x[c][j] - mean : 0.0f;
                x[c][j] = d;
                s += d * d;
            }
        const float rstd = 1.0f / sqrtf(group_sum<TH>(s, cells[1], t) * per + a.eps);
        if (!trimmed)
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                if (a.gamma) g[c].trim(t, c, a.cols);
                if (a.beta) b[c].trim(t, c, a.cols);
            }
        trimmed = true;
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = x[c][j] * rstd;
                if (a.gamma) v *= g[c].get(j);
                if (a.beta) v += b[c].get(j);
                x[c][j] = v;
            }
            store8<T, TH>((T*)a.y + row * a.ldy, t, c, a.cols, x[c]);
        }
        if (TH > 64) __syncthreads();                /* the cells are free again */
    }
}

/* The gradient: a workgroup of LANES lanes takes LANES / TH rows at a time and every gridDim-th such set; a lane keeps the sums of dy xh and dy
 * for its columns over all of them, so that gamma's and beta's gradients cost one partial row per workgroup and no second
 * pass over the activations.  The next two sets' loads are under way while this one's two sums are formed, at one barrier a set.  The row sets of a workgroup are added in order through LDS; column_sums adds the workgroups.
 * Partial sums leave in pieces of 32 bytes: entry by entry 29 x 11008 took 19 us instead of 11, 512 x 4096 16 instead of 13.
 * Bound by memory: 16384 x 4096 from int8 rows in 78 us, 335 MB, 4.3 GB a millisecond (copies reach 5.2).  Rows beyond 8192 (16384) entries keep some 50 (480) bytes
 * a lane in scratch memory, 29 x 32768 takes 41 us. */
struct NormBackArgs {
    const void *dy, *x;
    const float* scale;
    const void* gamma;
    const float *mean, *rstd;
    void* dx;
    float* part;                     /* [gridDim][2][cols]; null: no sums wanted */
    uint64_t lddy, ldx, lddx;
    uint32_t rows, cols;
    int centred;
    bool past;                       /* dx goes past the caches */
};
template <class T, bool EIGHT, int TH, int NCH, int LANES, bool SHORT = false>
__global__ __launch_bounds__(LANES) void norm_backward(const NormBackArgs a) {
    extern __shared__ float lds[];
    constexpr int SETS = LANES / TH;
    __shared__ float2 cells[3][16];
    const int t = threadIdx.x % TH, set = threadIdx.x / TH;
    float dg[NCH][8], db[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[c][j] = db[c][j] = 0.0f;
    Raw<T, TH, SHORT> gamma[NCH];
    if (a.gamma)
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            gamma[c].load((const T*)a.gamma, t, c, a.cols);
            gamma[c].trim(t, c, a.cols);
        }
    const float per = 1.0f / (float)a.cols;
    const uint64_t step = (uint64_t)gridDim.x * SETS;
    /* A row is kept as it was read and unpacked twice, for the sums and for dx: three rows' raw bits take fewer registers than one row's values (values kept across the barrier spilled: 16384 x 4096 in 179 us).
     * Where a lane has more than one chunk of a row there is no room for the next ones. */
    constexpr bool AHEAD = NCH == 1;
    typedef typename std::conditional<EIGHT, RawQ<TH, SHORT>, Raw<T, TH, SHORT>>::type RawX;
    struct Row {
        RawX x[NCH];
        Raw<T, TH, SHORT> dy[NCH];
        float mean, rstd, scale;
    };
    auto fetch = [&](Row& to, uint64_t row) {
        const bool live = row < a.rows;
        const uint32_t cols = live ? a.cols : 0;
        const uint64_t r = live ? row : 0;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            if constexpr (EIGHT) to.x[c].load((const int8_t*)a.x + r * a.ldx, t, c, cols);
            else to.x[c].load((const T*)a.x + r * a.ldx, t, c, cols);
            to.dy[c].load((const T*)a.dy + r * a.lddy, t, c, cols);
        }
        to.rstd = a.rstd[r];
        to.mean = a.centred ? a.mean[r] : 0.0f;
        to.scale = EIGHT ? a.scale[r] : 1.0f;
    };
    auto work = [&](Row& now, uint64_t row, float2* cell) {
        const uint32_t cols = row < a.rows ? a.cols : 0;
        float sg = 0.0f, sgx = 0.0f;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            now.x[c].trim(t, c, cols);
            now.dy[c].trim(t, c, cols);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = row_col<TH>(t, c) + j < cols;
                const float h = in ? (now.x[c].get(j) * now.scale - now.mean) * now.rstd : 0.0f, d = now.dy[c].get(j);
                dg[c][j] += d * h;
                db[c][j] += d;
                const float g = a.gamma ? d * gamma[c].get(j) : d;
                sg += g;
                sgx += g * h;
            }
        }
        if (!a.dx) return;
        group_sum2<TH>(sg, sgx, cell, t);
        const float mg = a.centred ? sg * per : 0.0f, mgx = sgx * per;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            now.x[c].forget();
            now.dy[c].forget();
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float h = (now.x[c].get(j) * now.scale - now.mean) * now.rstd, d = now.dy[c].get(j), g = a.gamma ? d * gamma[c].get(j) : d;
                v[j] = now.rstd * (g - mg - h * mgx);
            }
            store8<T, TH>((T*)a.dx + row * a.lddx, t, c, cols, v, a.past);
        }
    };
    /* every lane of the workgroup makes the same rounds; the cells go round by three, so one barrier a round is enough */
    const uint64_t begin = (uint64_t)blockIdx.x * SETS;
    if constexpr (AHEAD) {
        Row rows[3];
        fetch(rows[0], begin + set);
        fetch(rows[1], begin + step + set);
        for (uint64_t first = begin; first < a.rows; first += 3 * step) {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                if (first + i * step >= a.rows) break;
                fetch(rows[(i + 2) % 3], first + (i + 2) * step + set);
                work(rows[i], first + i * step + set, cells[i] + set * (TH / 64));
            }
        }
    } else {
        Row one;
        int turn = 0;
        for (uint64_t first = begin; first < a.rows; first += step, turn ^= 1) {
            fetch(one, first + set);
            work(one, first + set, cells[turn] + set * (TH / 64));
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* part = a.part + ((uint64_t)blockIdx.x * 2 + which) * a.cols;
        for (int s = 0; s < SETS; ++s) {
            if (SETS > 1) __syncthreads();
            if (set != s) continue;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                const uint32_t k = row_col<TH>(t, c);
                if (k >= a.cols) continue;
                const float* mine = which ? db[c] : dg[c];
                f4 v[2] = {{mine[0], mine[1], mine[2], mine[3]}, {mine[4], mine[5], mine[6], mine[7]}};
                f4* sum = (f4*)(lds + k);            /* (LDS has room for whole pieces of eight) */
                if (s) {
                    v[0] += sum[0];
                    v[1] += sum[1];
                }
                if (s + 1 < SETS) {
                    sum[0] = v[0];
                    sum[1] = v[1];
                } else if (k + 8 <= a.cols) __builtin_memcpy(part + k, v, 32);
                else
#pragma unroll
                    for (int j = 0; j < 7; ++j)
                        if (k + j < a.cols) part[k + j] = v[j / 4][j % 4];
            }
        }
    }
}
/* out[k] = sum over i < n of part[i * stride + k]: 64 columns to a workgroup, 16 waves that take every 16th partial row, joined in order */
struct ColumnSumArgs {
    const float* part;
    float* out[2];                   /* of the second one (blockIdx.y) the partial rows lie cols further on; null: not wanted */
    uint64_t stride;
    uint32_t n, cols;
};
__global__ __launch_bounds__(1024) void column_sums(const ColumnSumArgs a) {
    __shared__ float cells[16][64];
    const int w = threadIdx.x / 64, l = threadIdx.x % 64;
    const uint32_t k = blockIdx.x * 64 + l;
    float* out = a.out[blockIdx.y];
    if (!out) return;
    const float* part = a.part + (uint64_t)blockIdx.y * a.cols;
    float s = 0.0f;
    if (k < a.cols)
#pragma unroll 4
        for (uint32_t i = w; i < a.n; i += 16) s += part[i * a.stride + k];
    cells[w][l] = s;
    __syncthreads();
    if (w || k >= a.cols) return;
    for (int i = 1; i < 16; ++i) s += cells[i][l];
    out[k] = s;
}

/* ---- products ------------------------------------------------------------------------------------------
 * One kernel for the three products: out[q][p] = sum over r of P(p, r) Q(q, r), p the axis along which out lies in memory.
 *     y  = x w^T    p: outputs, q: rows,    r: inputs   P = w   r along memory    Q = x   r along memory
 *     dx = dz w     p: inputs,  q: rows,    r: outputs  P = w   r across memory   Q = dz  r along memory
 *     dw = dz^T x   p: inputs,  q: outputs, r: rows     P = x   r across memory   Q = dz  r across memory
 * P is the first operand of the matrix instruction and Q the second, so that a lane ends up with four neighbouring
 * entries of a row of out.  Tiles lie in LDS as they lie in memory: where r runs along memory, rows of BK r in 16-byte pieces, piece k
 * of row i in place k ^ turn(i); where it runs across, rows of the tile's p in 32-byte pieces, piece k of row r in place k ^ f(r), read through the transposing
 * LDS load.  With both rules the sixteen rows that a wave reads at once fall on all banks. */
struct Operand {
    const void* d;
    uint64_t ld;
};
struct ProductArgs {
    Operand p, q;
    uint32_t np, nq, nr;
    /* epilogue */
    void* out;
    uint64_t ldo;
    const float* p_scale;            /* forward, int8 weights: one for each p */
    const void* bias;                /* forward: one for each p */
    const void* residual;
    uint64_t ldres;
    void* z;
    uint64_t ldz;
    const float* factor;             /* gradients: everything times this number; null: 1 */
    const uint16_t* powers;          /* gradients in float16, int8 p: a power of two for each r, in float16, that its whole numbers are multiplied by */
    int act;
    bool past;                       /* out and z go past the caches */
    float* part;                     /* [split][nq][ldp] unfinished sums, where r is split; null: the whole of r in one go */
    uint64_t ldp;
    uint32_t r_split;                /* r of one split */
};
template <class T> __device__ __forceinline__ f4 mfma(typename Vec<T>::v8 a, typename Vec<T>::v8 b, f4 c);
template <> __device__ __forceinline__ f4 mfma<_Float16>(Vec<_Float16>::v8 a, Vec<_Float16>::v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
template <> __device__ __forceinline__ f4 mfma<__bf16>(Vec<__bf16>::v8 a, Vec<__bf16>::v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

/* A tile of an operand: SIDE of p (or q) by BK of r, 32 or 64 */
template <class T, bool ALONG, int SIDE, int BK>
struct Tile {
    typedef typename Vec<T>::v8 v8;
    typedef short s4 __attribute__((ext_vector_type(4)));
    static constexpr int ELEMENTS = SIDE * BK;
    __device__ static __forceinline__ int spread(int r) { return SIDE >= 128 ? (r & 3) | ((r >> 3) & 1) << 2 : r & 3; }
    __device__ static __forceinline__ int turn(int line) { return BK == 64 ? line & 7 : (line >> 1) & 3; }
    /* where the eight elements number `piece` of line `line` lie: line = p of r pieces, or r of p pieces */
    __device__ static __forceinline__ int place(int line, int piece) {
        if (ALONG) return line * BK + ((piece ^ turn(line)) << 3);
        return line * SIDE + ((((piece >> 1) ^ spread(line)) << 1 | (piece & 1)) << 3);
    }
    /* the matrix instruction's operand: sixteen of p from `side` on, r from 32 s on */
    __device__ static __forceinline__ v8 fragment(const T* lds, int side, int s, int lane) {
        if (ALONG) return *(const v8*)(lds + place(side + (lane & 15), s * 4 + (lane >> 4)));
        union {
            s4 half[2];
            v8 whole;
        } u;
        for (int h = 0; h < 2; ++h) {
            const int r = s * 32 + (lane >> 4) * 8 + h * 4 + ((lane & 15) >> 2);
            const int at = r * SIDE + ((((side >> 4) ^ spread(r)) << 4) | (lane & 3) << 2);
            u.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(lds + at));
        }
        return u.whole;
    }
};

/* The epilogue of eight entries of column p on.  What it needs for the columns is loaded once, by the constructor; what it needs for the entries,
 * the residual, by ask(), ahead of apply(). */
template <class T, bool FORWARD>
struct Finish {
    const ProductArgs& a;
    const uint32_t p;
    float scale[8], bias[8];
    typename Vec<T>::v8 res;
    __device__ __forceinline__ Finish(const ProductArgs& a_, uint32_t p_) : a(a_), p(p_) {
        if (!FORWARD) {
            scale[0] = a.factor ? a.factor[0] : 1.0f;
            return;
        }
        if (a.p_scale) {
#pragma unroll
            for (int i = 0; i < 8; ++i) scale[i] = p + i < a.np ? a.p_scale[p + i] : 0.0f;
        }
        if (a.bias) {
#pragma unroll
            for (int i = 0; i < 8; ++i) bias[i] = p + i < a.np ? (float)((const T*)a.bias)[p + i] : 0.0f;
        }
    }
    __device__ __forceinline__ void ask(uint32_t q) {
        if (!FORWARD || !a.residual || q >= a.nq || p >= a.np) return;
        const T* at = (const T*)a.residual + q * a.ldres + p;
        if (p + 8 <= a.np) res = unaligned<typename Vec<T>::v8>(at);
        else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (p + i < a.np) res[i] = at[i];
        }
    }
    __device__ __forceinline__ void apply(uint32_t q, float* v) const {
        if (q >= a.nq || p >= a.np) return;
        if (FORWARD) {
            if (a.p_scale) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= scale[i];
            }
            if (a.bias) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += bias[i];
            }
            if (a.z) put8<T>((T*)a.z + q * a.ldz, p, a.np, v, a.past);
            if (a.act != TC_ACT_NONE) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = activate(v[i], a.act);
            }
            if (a.residual) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += (float)res[i];
            }
        } else if (a.factor) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= scale[0];
        }
        put8<T>((T*)a.out + q * a.ldo, p, a.np, v, a.past);
    }
};
/* A wave's NP x NQ blocks of sixteen by sixteen, through a piece of LDS of its own (NP * 16 + 4 floats for each of sixteen q): a lane of
 * the matrix instruction holds four entries of a row, and memory wants whole lines.  The workgroup must have passed a barrier since
 * LDS was last read otherwise. */
template <int NP> constexpr int drain_bytes() { return 16 * (NP * 16 + 4) * 4; }
template <class T, bool FORWARD, int NP, int NQ>
__device__ __forceinline__ void drain(const ProductArgs& a, f4 (&acc)[NP][NQ], uint8_t* lds, uint32_t q0, uint32_t p0, uint32_t split, int lane) {
    float* buf = (float*)lds;
    constexpr int LD = NP * 16 + 4, GROUPS = NP * 2, ROWS = 64 / GROUPS;
    const uint32_t p = p0 + (lane % GROUPS) * 8, row = lane / GROUPS;
    Finish<T, FORWARD> end(a, p);
    end.ask(q0 + row);
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
#pragma unroll
        for (int i = 0; i < NP; ++i) *(f4*)(buf + (lane & 15) * LD + i * 16 + (lane >> 4) * 4) = acc[i][j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");        /* lanes read what others of the wave have written */
#pragma unroll 1
        for (int r = row; r < 16; r += ROWS) {
            const float* at = buf + r * LD + (lane % GROUPS) * 8;
            const f4 lo = *(const f4*)at, hi = *(const f4*)(at + 4);
            const uint32_t q = q0 + j * 16 + r;
            if (a.part) {
                if (q < a.nq && p < a.np) {
                    f4* to = (f4*)(a.part + (split * (uint64_t)a.nq + q) * a.ldp + p);
                    to[0] = lo;
                    to[1] = hi;
                }
            } else {
                float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                Finish<T, FORWARD> now = end;
                end.ask(q + ROWS);                       /* rows of this block, then of the next, are ROWS apart */
                now.apply(q, v);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

/* How a tile gets to LDS.  An operand whose rows can be read in aligned 16-byte pieces (int8: 8-byte ones) goes there directly, without
 * passing through registers.  That direct load writes the lanes' pieces side by side, so the places of a tile are dealt out
 * on the memory side: place n takes the piece that belongs there.  Buffer addresses: a piece outside the operand gets an offset past the buffer's end and reads
 * zeros.  int8 tiles pass through registers, where they become the other operand's type.  So do LOOSE operands, rows of any
 * alignment, length and stride: pieces at addresses that need not be aligned (1), or entry by entry where a row has fewer than eight (2). */
/* eight int8 in two words -> eight of T, exactly.  float16: a byte with its sign bit flipped is q + 128; put under the exponent of 1024 it reads 1152 + q. */
template <class T> __device__ __forceinline__ typename Vec<T>::v8 widen(uint32_t lo, uint32_t hi);
template <> __device__ __forceinline__ Vec<_Float16>::v8 widen<_Float16>(uint32_t lo, uint32_t hi) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    union {
        h2 h[4];
        Vec<_Float16>::v8 v;
    } u;
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    const h2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    u.h[0] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)) - bias;
    u.h[1] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)) - bias;
    u.h[2] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)) - bias;
    u.h[3] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)) - bias;
    return u.v;
}
template <> __device__ __forceinline__ Vec<__bf16>::v8 widen<__bf16>(uint32_t lo, uint32_t hi) {
    union {
        uint32_t w[4];
        Vec<__bf16>::v8 v;
    } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int w = (int)(i < 2 ? lo : hi), at = i & 1 ? 16 : 0;
        const float even = (float)(w << (24 - at) >> 24), odd = (float)(w << (16 - at) >> 24);
        u.w[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, odd), __builtin_bit_cast(uint32_t, even), 0x07060302u);      /* the upper halves: a whole number under 256 has no more */
    }
    return u.v;
}
template <class T, bool ALONG, bool EIGHT, int LOOSE, int SIDE, int TH, int BK>
struct Feed {
    typedef Tile<T, ALONG, SIDE, BK> tile;
    static constexpr int N = SIDE * BK / 8 / TH, PIECES = ALONG ? BK / 8 : SIDE / 8, SIZE = EIGHT ? 1 : 2;
    static constexpr bool HELD = EIGHT || LOOSE != 0, POWERS = EIGHT && !ALONG && std::is_same<T, _Float16>::value;
    static constexpr uint32_t NOWHERE = 0x80000000u;
    typedef typename std::conditional<EIGHT, uint2, uint4>::type Piece;
    typedef Piece Held[HELD ? N : 1];
    typename std::conditional<LOOSE != 0, uint64_t, uint32_t>::type off[N];
    const char* base;
    uint64_t step, ld;
    uint32_t nr, line_bytes, left;   /* left: of the operand's axis across the sum, from this tile on */
    uint32_t held_rest;              /* of the sum, from the tile in `held` on */
    const uint16_t* powers;
    uint32_t held_power[POWERS ? N : 1];
    __device__ static __forceinline__ int line_of(int n) { return n / PIECES; }
    __device__ static __forceinline__ int piece_of(int n) {
        const int line = n / PIECES, slot = n % PIECES;
        return ALONG ? slot ^ tile::turn(line) : ((slot >> 1) ^ tile::spread(line)) << 1 | (slot & 1);
    }
    /* LOOSE: how far before its place piece n has to be read to end with its row, `rest` of the sum being left; eight or more: nothing of it is the row's */
    __device__ __forceinline__ uint32_t back(int n, uint32_t rest) const {
        const uint32_t end = piece_of(n) * 8 + 8, has = ALONG ? rest : left;
        return end > has ? end - has : 0;
    }
    /* r from `r0` on, `nr_` of them */
    __device__ __forceinline__ void init(const Operand& o, uint64_t side0, uint32_t sides, uint32_t r0, uint32_t nr_, int t, const uint16_t* powers_ = nullptr) {
        nr = nr_;
        if constexpr (POWERS) powers = powers_ + r0;
        ld = o.ld;
        left = sides - (uint32_t)side0;
        line_bytes = (uint32_t)(o.ld * SIZE);
        base = (const char*)o.d + (ALONG ? side0 * o.ld + r0 : r0 * o.ld + side0) * SIZE;
        step = ALONG ? BK * SIZE : BK * o.ld * SIZE;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int n = i * TH + t, line = line_of(n), piece = piece_of(n);
            const bool in = (uint32_t)(ALONG ? line : piece * 8) < left;
            if (LOOSE) off[i] = ((ALONG && !in ? 0 : line) * o.ld + piece * 8) * SIZE;        /* a line too many reads the first one: its results are dropped */
            else off[i] = in ? line * line_bytes + piece * 8 * SIZE : NOWHERE;
        }
    }
    /* tile number k, to its place in LDS or into `held`; past the last one: zeros (LOOSE: nothing) */
    __device__ __forceinline__ void issue(T* lds, Held& held, uint32_t k, int t) {
        const uint32_t rest = __builtin_amdgcn_readfirstlane(nr > k * BK ? nr - k * BK : 0);      /* a saturating difference, which is a vector instruction */
        const char* at = base + (rest ? k * step : 0);
        if constexpr (POWERS) {          /* a line past the last one gets 0 */
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(powers + (rest ? k * BK : 0)), 0, (rest < BK ? rest : BK) * 2, 0x00020000);
#pragma unroll
            for (int i = 0; i < N; ++i) held_power[i] = __builtin_amdgcn_raw_buffer_load_b16(r, line_of(i * TH + t) * 2, 0, 0);
        }
        if constexpr (LOOSE == 1) {
            held_rest = rest;
            if (!rest) return;
            /* no load depends on a condition: pieces past an end are read where the row's last eight entries are, or from its last line, and put right by settle() */
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int n = i * TH + t;
                int64_t o = (int64_t)off[i] - (int64_t)back(n, rest) * SIZE;
                if (!ALONG && rest < BK && (uint32_t)line_of(n) >= rest) o -= (int64_t)(line_of(n) - (rest - 1)) * (int64_t)ld * SIZE;
                held[i] = unaligned<Piece>(at + o);
            }
        } else if constexpr (LOOSE == 2) {
            /* rows shorter than eight entries: one by one */
            typedef typename std::conditional<EIGHT, uint8_t, uint16_t>::type entry;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int n = i * TH + t;
                const uint32_t b = back(n, rest);
                const bool live = b < 8 && (ALONG ? (uint32_t)line_of(n) < left : (uint32_t)line_of(n) < rest);
                uint32_t w[EIGHT ? 2 : 4];
                read_piece((const entry*)(at + off[i]), live ? 8 - b : 0, w);
                held[i] = __builtin_bit_cast(Piece, w);
            }
        } else {
            const uint32_t span = ALONG ? NOWHERE - 1 : (rest < BK ? rest : BK) * line_bytes;
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, span, 0x00020000);
            if (ALONG && rest < BK) {    /* the last tile of r: pieces past its end go, for good */
                asm volatile("");        /* a branch, not eight selections in every step */
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if ((uint32_t)piece_of(i * TH + t) * 8 >= rest) off[i] = NOWHERE;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint32_t o = off[i];
                if constexpr (EIGHT) held[i] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, 0));
                else
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (i * TH + (t & ~63)) * 8), 16, o, 0, 0, 0);
            }
        }
    }
    __device__ __forceinline__ void settle(T* lds, Held& held, int t) {
        if constexpr (HELD) {
            /* the same for all lanes: whether this tile has pieces that issue() could not read where they are */
            const bool ragged = LOOSE == 1 && (held_rest < BK || (!ALONG && left < SIDE && left % 8));
#pragma unroll
            for (int i = 0; i < N; ++i) {
                typename Vec<T>::v8* to = (typename Vec<T>::v8*)(lds + (i * TH + t) * 8);
                uint32_t w[EIGHT ? 2 : 4];
                __builtin_memcpy(w, &held[i], sizeof w);
                if (LOOSE == 1 && ragged) {
                    asm volatile("");    /* a branch */
                    const int n = i * TH + t;
                    const uint32_t b = back(n, held_rest);
                    if (b >= 8 || (!ALONG && (uint32_t)line_of(n) >= held_rest))
#pragma unroll
                        for (uint32_t& x : w) x = 0;
                    else if (b) to_front(w, 8 - b);
                }
                if constexpr (POWERS) *to = widen<T>(w[0], w[1]) * __builtin_bit_cast(T, (uint16_t)held_power[i]);
                else if constexpr (EIGHT) *to = widen<T>(w[0], w[1]);
                else *to = __builtin_bit_cast(typename Vec<T>::v8, make_uint4(w[0], w[1], w[2], w[3]));
            }
        }
    }
};
/* Workgroups go to the eight XCDs in turn, each with an L2 of its own: an XCD takes neighbouring tiles, in blocks of four along q */
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t tiles_p, uint32_t tiles_q, uint32_t& tp, uint32_t& tq) {
    const uint32_t n = tiles_p * tiles_q, per = n / 8, more = n % 8, x = b % 8;
    const uint32_t i = x * per + (x < more ? x : more) + b / 8;
    const uint32_t DEEP = 4;
    const uint32_t band = i / (DEEP * tiles_p), first = band * DEEP, deep = tiles_q - first < DEEP ? tiles_q - first : DEEP;
    const uint32_t j = i - band * DEEP * tiles_p;
    /* the division runs in vector registers; buffer descriptors want scalar ones */
    tq = __builtin_amdgcn_readfirstlane(first + j % deep);
    tp = __builtin_amdgcn_readfirstlane(j / deep);
}
/* What both kernels below start with: the tile of this workgroup and its part of r */
#define TC_PRODUCT_PROLOGUE                                                                                                 \
    constexpr int TH = WP * WQ * 64, NP = SP / WP / 16, NQ = SQ / WQ / 16, STAGE = (SP + SQ) * BK;                          \
    typedef Feed<T, P_ALONG, P_EIGHT, LOOSE, SP, TH, BK> FP;                                                                \
    typedef Feed<T, Q_ALONG, false, LOOSE, SQ, TH, BK> FQ;                                                                  \
    extern __shared__ __align__(16) uint8_t lds_bytes[];                                                                    \
    T* const lds = (T*)lds_bytes;                                                                                           \
    const uint32_t tiles_p = (a.np + SP - 1) / SP, tiles_q = (a.nq + SQ - 1) / SQ;                                          \
    const uint32_t split = __builtin_amdgcn_readfirstlane(blockIdx.x / (tiles_p * tiles_q)), r0 = split * a.r_split;                                        \
    const uint32_t nr = a.nr - r0 < a.r_split ? a.nr - r0 : a.r_split, steps = (nr + BK - 1) / BK;                          \
    uint32_t tp, tq;                                                                                                        \
    tile_of(blockIdx.x % (tiles_p * tiles_q), tiles_p, tiles_q, tp, tq);                                                    \
    const uint64_t p0 = (uint64_t)tp * SP, q0 = (uint64_t)tq * SQ;                                                          \
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), wp = w % WP, wq = w / WP;         \
    FP fp;                                                                                                                  \
    FQ fq;                                                                                                                  \
    fp.init(a.p, p0, a.np, r0, nr, t, a.powers);                                                                            \
    fq.init(a.q, q0, a.nq, r0, nr, t);                                                                                      \
    f4 acc[NP][NQ] = {};
#define TC_WAIT_AND_MEET(n) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(n) : "memory")
#define TC_PRODUCT_EPILOGUE                                                                                                 \
    TC_WAIT_AND_MEET(0);                                                                                                    \
    drain<T, FORWARD, NP, NQ>(a, acc, lds_bytes + w * drain_bytes<NP>(), (uint32_t)q0 + wq * (SQ / WQ), (uint32_t)p0 + wp * (SP / WP), split, lane);

/* Two stages of 64 r: one is multiplied while the other is filled; the two or more workgroups that share a compute unit cover each other's waits. */
template <class T, bool P_ALONG, bool P_EIGHT, bool Q_ALONG, bool FORWARD, int LOOSE, int SP, int SQ, int WP, int WQ>
__global__ __launch_bounds__(WP * WQ * 64) void product_paired(const ProductArgs a) {
    constexpr int BK = 64;
    TC_PRODUCT_PROLOGUE
    typename FP::Held hp;
    typename FQ::Held hq;
    fp.issue(lds, hp, 0, t);
    fq.issue(lds + SP * BK, hq, 0, t);
    fp.settle(lds, hp, t);
    fq.settle(lds + SP * BK, hq, t);
#pragma unroll 1
    for (uint32_t k = 0; k < steps; ++k) {
        T* now = lds + (k & 1) * STAGE;
        T* next = lds + (~k & 1) * STAGE;
        TC_WAIT_AND_MEET(0);
        fp.issue(next, hp, k + 1, t);
        fq.issue(next + SP * BK, hq, k + 1, t);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            typename Vec<T>::v8 x[NP], y[NQ];
#pragma unroll
            for (int j = 0; j < NQ; ++j) y[j] = FQ::tile::fragment(now + SP * BK, wq * (SQ / WQ) + j * 16, s, lane);
#pragma unroll
            for (int i = 0; i < NP; ++i) x[i] = FP::tile::fragment(now, wp * (SP / WP) + i * 16, s, lane);
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < NQ; ++j) acc[i][j] = mfma<T>(x[i], y[j], acc[i][j]);
        }
        fp.settle(next, hp, t);
        fq.settle(next + SP * BK, hq, t);
    }
    TC_PRODUCT_EPILOGUE
}

/* Five stages of 32 r in all 160 KB of LDS, for tiles of 256 x 256, one workgroup to a compute unit.  While a stage is multiplied from registers, the next
 * one is read into the other set of registers and the loads of the three after that are under way: at a step's barrier
 * every wave has read the stage it multiplies and the next one has arrived (the loads of the two behind it may be
 * outstanding).  Loads past the last stage bring zeros, so that the loop has no branches and the count of outstanding loads is always the same.
 * 16-bit operands only: an int8 one of a product this large is widened beforehand, which costs less than its passage through registers. */
template <class T, bool P_ALONG, bool Q_ALONG, bool FORWARD, int SP, int SQ, int WP, int WQ>
__global__ __launch_bounds__(WP * WQ * 64) __attribute__((amdgpu_waves_per_eu(WP * WQ / 4, WP * WQ / 4))) void product_deep(const ProductArgs a) {
    constexpr int BK = 32, STAGES = 5;
    constexpr bool P_EIGHT = false;
    constexpr int LOOSE = 0;
    TC_PRODUCT_PROLOGUE
    constexpr int LOADS = FP::N + FQ::N;
    typename FP::Held hp;
    typename FQ::Held hq;
    typename Vec<T>::v8 x0[NP], y0[NQ], x1[NP], y1[NQ];
#define TC_READ(X, Y, place)                                                                                                            \
    _Pragma("unroll") for (int j = 0; j < NQ; ++j) Y[j] = FQ::tile::fragment(lds + (place) * STAGE + SP * BK, wq * (SQ / WQ) + j * 16, 0, lane); \
    _Pragma("unroll") for (int i = 0; i < NP; ++i) X[i] = FP::tile::fragment(lds + (place) * STAGE, wp * (SP / WP) + i * 16, 0, lane);
#define TC_ORDER                                                                                                                        \
    if (P_ALONG && Q_ALONG) {                                                                                                           \
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);                                                                              \
        _Pragma("unroll") for (int i = 0; i < NP + NQ; ++i) {                                                                           \
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                                                                                   \
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);                                                                          \
        }                                                                                                                               \
    }
#define TC_STEP(k, X, Y, X2, Y2)                                                                                                        \
    TC_WAIT_AND_MEET(LOADS * (STAGES - 3));                                                                                             \
    fp.issue(lds + put * STAGE, hp, (k) + STAGES - 1, t);                                                                                \
    fq.issue(lds + put * STAGE + SP * BK, hq, (k) + STAGES - 1, t);                                                                     \
    TC_READ(X2, Y2, next)                                                                                                               \
    _Pragma("unroll") for (int i = 0; i < NP; ++i)                                                                                      \
        _Pragma("unroll") for (int j = 0; j < NQ; ++j) acc[i][j] = mfma<T>(X[i], Y[j], acc[i][j]);                                      \
    TC_ORDER                                                                                                                            \
    put = put + 1 == STAGES ? 0 : put + 1;                                                                                              \
    next = next + 1 == STAGES ? 0 : next + 1;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) {
        fp.issue(lds + i * STAGE, hp, i, t);
        fq.issue(lds + i * STAGE + SP * BK, hq, i, t);
    }
    TC_WAIT_AND_MEET(LOADS * (STAGES - 2));
    TC_READ(x0, y0, 0)
    uint32_t next = 1, put = STAGES - 1;
#pragma unroll 1
    for (uint32_t k = 0; k < steps; k += 2) {
        TC_STEP(k, x0, y0, x1, y1)
        TC_STEP(k + 1, x1, y1, x0, y0)
    }
#undef TC_STEP
#undef TC_ORDER
#undef TC_READ
    TC_PRODUCT_EPILOGUE
}
#undef TC_PRODUCT_PROLOGUE
#undef TC_PRODUCT_EPILOGUE

/* int8 rows -> the same whole numbers in T, times a power of two for each row where `powers` has them, side by side with a stride of ldo: 256 lanes
 * take 2048 entries of a row */
template <class T>
__global__ __launch_bounds__(256) void widen_rows(const Operand o, const uint16_t* powers, T* out, uint64_t ldo, uint32_t rows, uint32_t cols) {
    const uint32_t col = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= cols) return;
    for (uint64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const uint2 q = *(const uint2*)((const int8_t*)o.d + row * o.ld + col);
        typename Vec<T>::v8 v = widen<T>(q.x, q.y);
        if (std::is_same<T, _Float16>::value && powers) v *= __builtin_bit_cast(T, powers[row]);
        *(typename Vec<T>::v8*)(out + row * ldo + col) = v;
    }
}

/* the parts of a split product, added in order, and its epilogue: eight entries to a lane */
template <class T, bool FORWARD>
__global__ __launch_bounds__(256) void join_parts(const ProductArgs a, uint32_t splits) {
    const uint32_t per = (a.np + 7) / 8;
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= (uint64_t)per * a.nq) return;
    const uint32_t q = (uint32_t)(n / per), p = (uint32_t)(n % per) * 8;
    Finish<T, FORWARD> end(a, p);
    end.ask(q);
    f4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
#pragma unroll 4
    for (uint32_t i = 0; i < splits; ++i) {
        const f4* at = (const f4*)(a.part + (i * (uint64_t)a.nq + q) * a.ldp + p);
        lo += at[0];
        hi += at[1];
    }
    float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    end.apply(q, v);
}

/* ---- a few rows -------------------------------------------------------------------------------------------------
 * y = x w^T for at most sixteen rows of x: the weights are read once and that is all it costs.  A workgroup has sixteen of w's rows and its waves share r; each goes from memory
 * straight into the matrix instruction: lane l takes 16 r of row l & 15, from 16 (l >> 4) on, the first eight of them for one
 * instruction and the last eight for the next (any order of r does, if both operands have the same).  The waves' sums are added in order.
 * A wave has four chunks of 64 r under way.  Sixteen waves where the weights are int8 and their rows therefore short (1 x 4096 -> 11008, cold:
 * 13.3 us; eight waves 15.3), eight otherwise.  Rows of whole, aligned pieces of sixteen. */
template <class T, bool EIGHT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void product_thin(const ProductArgs a) {
    typedef typename Vec<T>::v8 v8;
    __shared__ float sums[WAVES][256];
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t p0 = blockIdx.x * 16, line = lane & 15, at = (lane >> 4) * 16;
    constexpr int SIZE = EIGHT ? 1 : 2, WORDS = EIGHT ? 2 : 4;
    constexpr uint32_t NOWHERE = 0x80000000u;
    const bool has_p = p0 + line < a.np, has_q = line < a.nq;
    f4 acc = {0, 0, 0, 0};
    constexpr int AHEAD = 4;
    const uint32_t chunks = (a.nr + 63) / 64;
    for (uint32_t c = w; c < chunks; c += WAVES * AHEAD) {
        uint32_t x[AHEAD][2][WORDS], y[AHEAD][2][4];
        const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc((char*)a.p.d + p0 * a.p.ld * SIZE, 0, NOWHERE - 1, 0x00020000);
        const __amdgpu_buffer_rsrc_t rq = __builtin_amdgcn_make_buffer_rsrc((void*)a.q.d, 0, NOWHERE - 1, 0x00020000);
        const uint32_t op = (uint32_t)(line * a.p.ld + at) * SIZE, oq = (uint32_t)(line * a.q.ld + at) * 2;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const uint32_t r = (c + i * WAVES) * 64, from = r < a.nr ? r : 0;
            const bool in = r + at < a.nr;                 /* the rows are whole pieces of sixteen */
            const auto one = __builtin_amdgcn_raw_buffer_load_b128(rp, in && has_p ? op : NOWHERE, from * SIZE, 0);
            if constexpr (EIGHT) {
                x[i][0][0] = one[0];
                x[i][0][1] = one[1];
                x[i][1][0] = one[2];
                x[i][1][1] = one[3];
            } else {
                const auto two = __builtin_amdgcn_raw_buffer_load_b128(rp, in && has_p ? op + 16 : NOWHERE, from * SIZE, 0);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    x[i][0][k] = one[k];
                    x[i][1][k] = two[k];
                }
            }
            const auto lo = __builtin_amdgcn_raw_buffer_load_b128(rq, in && has_q ? oq : NOWHERE, from * 2, 0);
            const auto hi = __builtin_amdgcn_raw_buffer_load_b128(rq, in && has_q ? oq + 16 : NOWHERE, from * 2, 0);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                y[i][0][k] = lo[k];
                y[i][1][k] = hi[k];
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v8 u;
                if constexpr (EIGHT) u = widen<T>(x[i][h][0], x[i][h][1]);
                else u = __builtin_bit_cast(v8, make_uint4(x[i][h][0], x[i][h][1], x[i][h][2], x[i][h][3]));
                acc = mfma<T>(u, __builtin_bit_cast(v8, make_uint4(y[i][h][0], y[i][h][1], y[i][h][2], y[i][h][3])), acc);
            }
    }
    /* acc: q = lane & 15, p from 4 (lane >> 4) on */
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[w][(lane & 15) * 16 + (lane >> 4) * 4 + i] = acc[i];
    __syncthreads();
    if (t >= 32) return;
    const uint32_t q = t >> 1, p = (t & 1) * 8;
    Finish<T, true> end(a, p0 + p);
    end.ask(q);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = sums[0][q * 16 + p + i];
        for (int k = 1; k < WAVES; ++k) v[i] += sums[k][q * 16 + p + i];
    }
    end.apply(q, v);
}

/* ---- the gradient before the activation ------------------------------------------------------------------
 * dz = dy act'(z), and its sums over the rows.  int8 operands of the products that follow have a scale for each of the
 * rows that those products sum over; it is put into their other operand here, from the unrounded value: by_x = dz s_x[row] for dw,
 * by_w = dz s_w[column] for dx.  So whole numbers enter the matrix instruction exactly and one rounding of the gradient to its type is all there is.
 * bfloat16 has float32's range and takes the scale as it is.  float16 would lose rows whose scale is small beside the largest, so a scale is split into a number of
 * [1/2, 1), which goes to the gradient and cannot overflow, and a power of two, which goes to the whole numbers as they are widened: relative to the largest
 * scale's, which becomes 2^8, down to 2^-24 every q 2^k is a float16.  (Scales more than 2^32 below the largest leave the rest with the gradient.)  One row of 512 with an entry of
 * 5000 among others of N(0, 1), gradients of 1e-4: dw of the other columns is 3.3e-4 of its size off; with one power of two for all rows it was 0.41. */
struct SlopeArgs {
    const void *dy, *z;
    const float* z_scale;            /* z is int8 where this is set */
    void *dz, *by_x, *by_w;
    const float *x_scale, *w_scale;
    const float* m;                  /* float16: what scale_peak wrote */
    uint16_t *powers_x, *powers_w;   /* float16: the powers of two of x's and w's rows */
    float* part;                     /* [gridDim.y][cols] */
    uint64_t lddy, ldz, lddz;        /* by_x, by_w: cols side by side, padded to ld_by */
    uint64_t ld_by;
    uint32_t rows, cols;
    int act;
};
/* for the largest magnitude f 2^e of x's scales, f in [1/2, 1): m[0] = 2^(e - 8), which their product is multiplied by, m[1] = e; of w's: m[2], m[3].  e is
 * held above -110, so that m[0] is in the normal range. */
__global__ __launch_bounds__(1024) void scale_peak(const float* x, uint32_t nx, const float* w, uint32_t nw, float* m) {
    __shared__ float cells[16];
    const float* s = blockIdx.x ? w : x;
    const uint32_t n = s ? (blockIdx.x ? nw : nx) : 0;
    float v = 0.0f;
#pragma unroll 8
    for (uint32_t i = threadIdx.x; i < n; i += 1024) v = fmaxf(v, finite_magnitude(s[i]));
    v = group_max<1024>(v, cells, threadIdx.x);
    if (threadIdx.x) return;
    int e = v > 0.0f ? ilogbf(v) + 1 : 0;
    e = e < -110 ? -110 : e;
    m[2 * blockIdx.x] = ldexpf(1.0f, e - 8);
    m[2 * blockIdx.x + 1] = (float)e;
}
/* the scale s = f 2^e beside the largest one's 2^top: its power of two, 2^(8 + e - top) as a float16, and what is left for the gradient (0, infinities and NaNs: they themselves) */
__device__ __forceinline__ float split_scale(float s, int top, uint16_t& power) {
    const float f = __builtin_amdgcn_frexp_mantf(s);
    const int below = __builtin_amdgcn_frexp_expf(s) - top, held = below < -32 ? -32 : below > 0 ? 0 : below, k = held + 8;
    power = (uint16_t)(k < -14 ? 1 << (k + 24) : (k + 15) << 10);
    return below < -32 ? ldexpf(f, below + 32) : f;
}
/* A wave takes 512 columns (eight to a lane), the four waves of a workgroup every fourth of its rows. */
template <class T, bool SHORT>
__global__ __launch_bounds__(256) void slopes(const SlopeArgs a) {
    __shared__ float cells[4][512];
    const int w = threadIdx.x >> 6, t = threadIdx.x & 63, strip = blockIdx.x;
    const uint32_t k = row_col<64>(t, strip);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, ws[8];
    const int top_x = a.by_x && a.m ? (int)a.m[1] : 0, top_w = a.by_w && a.m ? (int)a.m[3] : 0;
    if (a.by_w)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            ws[j] = k + j < a.cols ? a.w_scale[k + j] : 0.0f;
            if (!a.m) continue;
            uint16_t power;
            ws[j] = split_scale(ws[j], top_w, power);
            if (blockIdx.y == 0 && w == 0 && k + j < a.cols) a.powers_w[k + j] = power;
        }
    for (uint64_t row = (uint64_t)blockIdx.y * 4 + w; row < a.rows; row += (uint64_t)gridDim.y * 4) {
        float v[8], z[8];
        load8<T, 64, SHORT>((const T*)a.dy + row * a.lddy, t, strip, a.cols, v);
        if (a.act != TC_ACT_NONE) {
            if (a.z_scale) load8q<64, SHORT>((const int8_t*)a.z + row * a.ldz, a.z_scale[row], t, strip, a.cols, z);
            else load8<T, 64, SHORT>((const T*)a.z + row * a.ldz, t, strip, a.cols, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= slope(z[j], a.act);
            put8<T>((T*)a.dz + row * a.lddz, k, a.cols, v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
        if (a.by_x) {
            float f = a.x_scale[row];
            if (a.m) {
                uint16_t power;
                f = split_scale(f, top_x, power);
                if (strip == 0 && t == 0) a.powers_x[row] = power;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = v[j] * f;
            put8<T>((T*)a.by_x + row * a.ld_by, k, a.cols, z);
        }
        if (a.by_w) {
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = v[j] * ws[j];
            put8<T>((T*)a.by_w + row * a.ld_by, k, a.cols, z);
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) cells[w][t * 8 + j] = sum[j];
    __syncthreads();
    const uint32_t first = strip * 512;
    for (uint32_t i = threadIdx.x; i < 512 && first + i < a.cols; i += 256)
        a.part[(uint64_t)blockIdx.y * a.cols + first + i] = (cells[0][i] + cells[1][i]) + (cells[2][i] + cells[3][i]);
}
/* The sums of dy alone, over few rows and in one launch: a workgroup takes 64 columns (eight to a lane), a wave eight rows at a time, and its
 * 128 partial rows are added in order.  501 x 4096: 5 us, where the two launches of many row sets cost 9.5. */
template <class T, bool SHORT>
__global__ __launch_bounds__(1024) void bias_sums(const T* dy, uint64_t ld, uint32_t rows, uint32_t cols, float* out) {
    __shared__ float cells[128][64];
    __shared__ float again[16][64];
    const int t = threadIdx.x, set = t >> 3, group = t & 7;
    const int chunk = blockIdx.x * 8 + group;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
    for (uint32_t row = set; row < rows; row += 128) {
        Raw<T, 1, SHORT> r;
        r.load(dy + row * ld, 0, chunk, cols);
        r.trim(0, chunk, cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += r.get(j);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) cells[set][group * 8 + j] = sum[j];
    __syncthreads();
    const int c = t & 63, part = t >> 6;
    float s = cells[part * 8][c];
#pragma unroll
    for (int i = 1; i < 8; ++i) s += cells[part * 8 + i][c];
    again[part][c] = s;
    __syncthreads();
    const uint32_t k = blockIdx.x * 64 + c;
    if (part || k >= cols) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += again[i][c];
    out[k] = s;
}
template <class T>
__global__ __launch_bounds__(256) void fill_rows(T* out, uint64_t ld, uint32_t rows, uint32_t cols) {
    const uint64_t n = (uint64_t)rows * cols;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) out[i / cols * ld + i % cols] = (T)0.0f;
}

}  // namespace layers
}  // namespace tc
