/*
 * Kernels of the layer operators (gfx950): 8-bit checkpoints, norms and their gradients, matrix products with their
 * epilogue and their gradients.
 */
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tc {
namespace layers {

typedef float f4 __attribute__((ext_vector_type(4)));
template <class T> struct Vec {
    typedef T v4 __attribute__((ext_vector_type(4)));
    typedef T v8 __attribute__((ext_vector_type(8)));
};
typedef int8_t q8 __attribute__((ext_vector_type(8)));

/* ---- activations: value and slope ------------------------------------------------------------------
 * Phi(z) by the rational form 7.1.26 of Abramowitz and Stegun's handbook: the upper tail of the normal distribution is
 * t (a1 + t (a2 + ..)) exp(-z^2 / 2) / 2 with t = 1 / (1 + p |z| / sqrt 2), within 7.5e-8 of it everywhere, which is the
 * size of a float32 rounding of Phi: 12 operations where the library's erf takes some 40.  Products with a factor that has
 * become 0 are 0, also at z = +-infinity, so that an overflowed value before the activation does not turn into a NaN. */
__device__ __forceinline__ float normal_tail(float z, float& bell) {
    const float a = fabsf(z) * 0.70710678118654752f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, a, 1.0f));
    bell = __expf(-0.5f * z * z);
    const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    return 0.5f * p * bell;
}
__device__ __forceinline__ float times(float z, float f) { return f == 0.0f ? 0.0f : z * f; }
__device__ __forceinline__ float activate(float z, int act) {
    if (act == TC_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (act == TC_ACT_GELU) {
        float bell;
        const float tail = normal_tail(z, bell);
        return times(z, z > 0.0f ? 1.0f - tail : tail);
    }
    if (act == TC_ACT_SILU) return times(z, __builtin_amdgcn_rcpf(1.0f + __expf(-z)));
    return z;
}
__device__ __forceinline__ float slope(float z, int act) {
    if (act == TC_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    if (act == TC_ACT_GELU) {
        float bell;
        const float tail = normal_tail(z, bell);
        return (z > 0.0f ? 1.0f - tail : tail) + times(z, 0.3989422804014327f * bell);
    }
    if (act == TC_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
        return s + times(z, s * (1.0f - s));
    }
    return 1.0f;
}

/* ---- sums and maxima of a wave or of the waves that share a row -------------------------------------- */
__device__ __forceinline__ float wave_sum(float v) {
    for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
    for (int k = 32; k; k >>= 1) v = fmaxf(v, __shfl_xor(v, k, 64));
    return v;
}
/* TH lanes of the workgroup (TH / 64 whole waves) together; cells: TH / 64 floats of LDS of this group.  Every lane of the workgroup calls it. */
template <int TH>
__device__ __forceinline__ float group_sum(float v, float* cells, int t) {
    v = wave_sum(v);
    if (TH == 64) return v;
    __syncthreads();
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
    __syncthreads();
    if ((t & 63) == 0) cells[t >> 6] = v;
    __syncthreads();
    v = cells[0];
    for (int w = 1; w < TH / 64; ++w) v = fmaxf(v, cells[w]);
    return v;
}

/* ---- rows in registers -------------------------------------------------------------------------------
 * TH lanes hold a row of at most TH * 8 * NCH entries, 8 NCH to a lane.  WIDE: lane t's chunk c is the eight entries from (c TH + t) 8
 * on, one 16-byte access (8 bytes of int8); rows that are not so aligned: entry (8 c + j) TH + t, so that the lanes of a
 * wave still read side by side. */
template <int TH, bool WIDE>
__device__ __forceinline__ uint32_t row_col(int t, int c, int j) {
    return WIDE ? ((uint32_t)c * TH + t) * 8 + j : ((uint32_t)c * 8 + j) * TH + t;
}
template <class T, int TH, bool WIDE>
__device__ __forceinline__ void load8(const T* p, int t, int c, uint32_t cols, float* v) {
    if (WIDE) {
        const uint32_t k = row_col<TH, true>(t, c, 0);
        typename Vec<T>::v8 x = {0, 0, 0, 0, 0, 0, 0, 0};
        if (k < cols) x = *(const typename Vec<T>::v8*)(p + k);
        for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
    } else {
        for (int j = 0; j < 8; ++j) {
            const uint32_t k = row_col<TH, false>(t, c, j);
            v[j] = k < cols ? (float)p[k] : 0.0f;
        }
    }
}
template <int TH, bool WIDE>
__device__ __forceinline__ void load8q(const int8_t* p, float scale, int t, int c, uint32_t cols, float* v) {
    if (WIDE) {
        const uint32_t k = row_col<TH, true>(t, c, 0);
        q8 x = {0, 0, 0, 0, 0, 0, 0, 0};
        if (k < cols) x = *(const q8*)(p + k);
        for (int j = 0; j < 8; ++j) v[j] = scale * (float)x[j];
    } else {
        for (int j = 0; j < 8; ++j) {
            const uint32_t k = row_col<TH, false>(t, c, j);
            v[j] = k < cols ? scale * (float)p[k] : 0.0f;
        }
    }
}
template <class T, int TH, bool WIDE>
__device__ __forceinline__ void store8(T* p, int t, int c, uint32_t cols, const float* v) {
    if (WIDE) {
        const uint32_t k = row_col<TH, true>(t, c, 0);
        typename Vec<T>::v8 x;
        for (int j = 0; j < 8; ++j) x[j] = (T)v[j];
        if (k < cols) *(typename Vec<T>::v8*)(p + k) = x;
    } else {
        for (int j = 0; j < 8; ++j) {
            const uint32_t k = row_col<TH, false>(t, c, j);
            if (k < cols) p[k] = (T)v[j];
        }
    }
}

/* ---- 8-bit checkpoints ------------------------------------------------------------------------------- */
struct RowArgs {
    const void* src;
    void* dst;
    float* scale;
    uint64_t ld_src, ld_dst;
    uint32_t rows, cols;
};
/* The largest finite magnitude is scaled by a power of two into [1, 2), and the row with it (exact but for entries below 2^-126 of it,
 * whose q is 0 either way), so that nothing overflows or gets lost.  With a 16-bit significand or less, 127 x is exact in
 * float32; a quotient from the rounded reciprocal is at most one off the nearest whole number, and the remainder 127 x - q amax, exact
 * too (q and amax have 7 and 11 bits), says which way.
 * Rows longer than the registers hold (NCH = 0) are read twice. */
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
template <class T, bool WIDE, int TH, int NCH>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void checkpoint_encode(const RowArgs a) {
    __shared__ float cells[16];
    const int t = threadIdx.x % TH;
    const uint32_t row = blockIdx.x * (TH < 256 ? 256 / TH : 1) + threadIdx.x / TH;
    if (row >= a.rows) return;                       /* whole waves, and only where no barrier follows */
    const T* src = (const T*)a.src + row * a.ld_src;
    int8_t* dst = (int8_t*)a.dst + row * a.ld_dst;
    const int chunks = NCH ? NCH : (a.cols + TH * 8 - 1) / (TH * 8);
    float x[NCH ? NCH : 1][8];
    float m = 0.0f;
    for (int c = 0; c < chunks; ++c) {
        float* v = x[NCH ? c : 0];
        load8<T, TH, WIDE>(src, t, c, a.cols, v);
        for (int j = 0; j < 8; ++j) m = fmaxf(m, finite_magnitude(v[j]));
    }
    m = group_max<TH>(m, cells, t);
    if (t == 0) a.scale[row] = m / 127.0f;
    const int e = m > 0.0f ? -ilogbf(m) : 0;
    const float amax = m > 0.0f ? ldexpf(m, e) : 1.0f, inv = 1.0f / amax;
    for (int c = 0; c < chunks; ++c) {
        float* v = x[NCH ? c : 0];
        if (!NCH) load8<T, TH, WIDE>(src, t, c, a.cols, v);
        if (WIDE) {
            const uint32_t k = row_col<TH, true>(t, c, 0);
            q8 q;
            for (int j = 0; j < 8; ++j) q[j] = (int8_t)quantised(v[j], amax, inv, e);
            if (k < a.cols) *(q8*)(dst + k) = q;
        } else {
            for (int j = 0; j < 8; ++j) {
                const uint32_t k = row_col<TH, false>(t, c, j);
                if (k < a.cols) dst[k] = (int8_t)quantised(v[j], amax, inv, e);
            }
        }
    }
}
/* 256 lanes take 2048 entries of a row */
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void checkpoint_decode(const RowArgs a) {
    const uint32_t per_row = (a.cols + 2047) / 2048;
    const uint32_t row = blockIdx.x / per_row;
    const int c = blockIdx.x % per_row;
    float v[8];
    load8q<256, WIDE>((const int8_t*)a.src + row * a.ld_src, a.scale[row], threadIdx.x, c, a.cols, v);
    store8<T, 256, WIDE>((T*)a.dst + row * a.ld_dst, threadIdx.x, c, a.cols, v);
}

/* ---- norms --------------------------------------------------------------------------------------------
 * A row is read once and stays in registers: its mean, then the mean square about it (no difference of large sums), then y. */
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
template <class T, bool WIDE, int TH, int NCH>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void norm_forward(const NormArgs a) {
    __shared__ float cells[16];
    const int t = threadIdx.x % TH;
    const uint32_t row = blockIdx.x * (TH < 256 ? 256 / TH : 1) + threadIdx.x / TH;
    if (row >= a.rows) return;
    float x[NCH][8];
    for (int c = 0; c < NCH; ++c) {
        if (a.scale) load8q<TH, WIDE>((const int8_t*)a.x + row * a.ldx, a.scale[row], t, c, a.cols, x[c]);
        else load8<T, TH, WIDE>((const T*)a.x + row * a.ldx, t, c, a.cols, x[c]);
    }
    const float per = 1.0f / (float)a.cols;
    float mean = 0.0f;
    if (a.centred) {
        float s = 0.0f;
        for (int c = 0; c < NCH; ++c)
            for (int j = 0; j < 8; ++j) s += x[c][j];
        mean = group_sum<TH>(s, cells, t) * per;
    }
    float s = 0.0f;
    for (int c = 0; c < NCH; ++c)
        for (int j = 0; j < 8; ++j) {
            const float d = row_col<TH, WIDE>(t, c, j) < a.cols ? x[c][j] - mean : 0.0f;
            x[c][j] = d;
            s += d * d;
        }
    const float rstd = 1.0f / sqrtf(group_sum<TH>(s, cells, t) * per + a.eps);
    if (t == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    for (int c = 0; c < NCH; ++c) {
        float g[8], b[8];
        if (a.gamma) load8<T, TH, WIDE>((const T*)a.gamma, t, c, a.cols, g);
        if (a.beta) load8<T, TH, WIDE>((const T*)a.beta, t, c, a.cols, b);
        for (int j = 0; j < 8; ++j) {
            float v = x[c][j] * rstd;
            if (a.gamma) v *= g[j];
            if (a.beta) v += b[j];
            x[c][j] = v;
        }
        store8<T, TH, WIDE>((T*)a.y + row * a.ldy, t, c, a.cols, x[c]);
    }
}

/* The gradient: a workgroup of 1024 lanes takes 1024 / TH rows at a time and every gridDim-th such set; a lane keeps the sums of dy xh and dy
 * for its columns over all of them, so that gamma's and beta's gradients cost one partial row per workgroup and no second
 * pass over the activations.  The row sets of a workgroup are added in order through LDS; column_sums adds the workgroups. */
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
};
static const int NORM_BACK_LANES = 1024;
template <class T, bool WIDE, int TH, int NCH>
__global__ __launch_bounds__(NORM_BACK_LANES) void norm_backward(const NormBackArgs a) {
    extern __shared__ float lds[];
    constexpr int SETS = NORM_BACK_LANES / TH;
    __shared__ float cells[2][16];
    const int t = threadIdx.x % TH, set = threadIdx.x / TH;
    float *cell0 = cells[0] + set * (TH / 64), *cell1 = cells[1] + set * (TH / 64);
    float dg[NCH][8], db[NCH][8];
    for (int c = 0; c < NCH; ++c)
        for (int j = 0; j < 8; ++j) dg[c][j] = db[c][j] = 0.0f;
    const float per = 1.0f / (float)a.cols;
    const uint64_t step = (uint64_t)gridDim.x * SETS;
    for (uint64_t first = (uint64_t)blockIdx.x * SETS; first < a.rows; first += step) {      /* the same number of rounds for every lane */
        const uint64_t row = first + set;
        const bool live = row < a.rows;
        const uint32_t cols = live ? a.cols : 0;
        const uint64_t r = live ? row : 0;
        const float mean = a.centred ? a.mean[r] : 0.0f, rstd = a.rstd[r];
        float xh[NCH][8], g[NCH][8];
        float sg = 0.0f, sgx = 0.0f;
        for (int c = 0; c < NCH; ++c) {
            if (a.scale) load8q<TH, WIDE>((const int8_t*)a.x + r * a.ldx, a.scale[r], t, c, cols, xh[c]);
            else load8<T, TH, WIDE>((const T*)a.x + r * a.ldx, t, c, cols, xh[c]);
            load8<T, TH, WIDE>((const T*)a.dy + r * a.lddy, t, c, cols, g[c]);
            float gm[8];
            if (a.gamma) load8<T, TH, WIDE>((const T*)a.gamma, t, c, a.cols, gm);
            for (int j = 0; j < 8; ++j) {
                const bool in = row_col<TH, WIDE>(t, c, j) < cols;
                const float h = in ? (xh[c][j] - mean) * rstd : 0.0f;
                const float dy = g[c][j];
                dg[c][j] += dy * h;
                db[c][j] += dy;
                const float gg = a.gamma ? dy * gm[j] : dy;
                xh[c][j] = h;
                g[c][j] = gg;
                sg += gg;
                sgx += gg * h;
            }
        }
        if (a.dx) {
            sg = group_sum<TH>(sg, cell0, t);
            sgx = group_sum<TH>(sgx, cell1, t);
            const float mg = a.centred ? sg * per : 0.0f, mgx = sgx * per;
            for (int c = 0; c < NCH; ++c) {
                for (int j = 0; j < 8; ++j) g[c][j] = rstd * (g[c][j] - mg - xh[c][j] * mgx);
                store8<T, TH, WIDE>((T*)a.dx + r * a.lddx, t, c, cols, g[c]);
            }
        }
    }
    if (!a.part) return;
    for (int which = 0; which < 2; ++which) {
        float* part = a.part + ((uint64_t)blockIdx.x * 2 + which) * a.cols;
        for (int s = 0; s < SETS; ++s) {
            __syncthreads();
            if (set == s)
                for (int c = 0; c < NCH; ++c)
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t k = row_col<TH, WIDE>(t, c, j);
                        if (k >= a.cols) continue;
                        float v = which ? db[c][j] : dg[c][j];
                        if (s) v += lds[k];
                        if (s + 1 < SETS) lds[k] = v;
                        else part[k] = v;
                    }
        }
    }
}
/* out[k] = sum over i < n of part[i * stride + k]: 64 columns to a workgroup, 16 waves that take every 16th partial row, joined in order */
struct ColumnSumArgs {
    const float* part;
    float* out;
    uint64_t stride;
    uint32_t n, cols;
};
__global__ __launch_bounds__(1024) void column_sums(const ColumnSumArgs a) {
    __shared__ float cells[16][64];
    const int w = threadIdx.x / 64, l = threadIdx.x % 64;
    const uint32_t k = blockIdx.x * 64 + l;
    float s = 0.0f;
    if (k < a.cols)
        for (uint32_t i = w; i < a.n; i += 16) s += a.part[i * a.stride + k];
    cells[w][l] = s;
    __syncthreads();
    if (w || k >= a.cols) return;
    for (int i = 1; i < 16; ++i) s += cells[i][l];
    a.out[k] = s;
}

/* ---- products ------------------------------------------------------------------------------------------
 * One kernel for the three products: out[q][p] = sum over r of P(p, r) Q(q, r), p the axis along which out lies in memory.
 *     y  = x w^T    p: outputs, q: rows,    r: inputs   P = w   r along memory    Q = x   r along memory
 *     dx = dz w     p: inputs,  q: rows,    r: outputs  P = w   r across memory   Q = dz  r along memory
 *     dw = dz^T x   p: inputs,  q: outputs, r: rows     P = x   r across memory   Q = dz  r across memory
 * P is the first operand of the matrix instruction and Q the second, so that a lane ends up with four neighbouring
 * entries of a row of out.  Tiles lie in LDS as they lie in memory: where r runs along memory, rows of 64 r in 16-byte pieces, piece k
 * of row i in place k ^ (i & 7); where it runs across, rows of the tile's p in 32-byte pieces, piece k of row r in place k ^ f(r), read through the transposing
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
    int act;
};
template <class T> __device__ __forceinline__ f4 mfma(typename Vec<T>::v8 a, typename Vec<T>::v8 b, f4 c);
template <> __device__ __forceinline__ f4 mfma<_Float16>(Vec<_Float16>::v8 a, Vec<_Float16>::v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
template <> __device__ __forceinline__ f4 mfma<__bf16>(Vec<__bf16>::v8 a, Vec<__bf16>::v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

static const int BK = 64;            /* r per step */

/* A tile of an operand: SIDE of p (or q) by BK of r */
template <class T, bool ALONG, bool EIGHT, int SIDE>
struct Tile {
    typedef typename Vec<T>::v8 v8;
    typedef short s4 __attribute__((ext_vector_type(4)));
    static constexpr int ELEMENTS = SIDE * BK;
    __device__ static __forceinline__ int spread(int r) { return SIDE >= 128 ? (r & 3) | ((r >> 3) & 1) << 2 : r & 3; }
    /* where the eight elements number `piece` of line `line` lie: line = p of r pieces, or r of p pieces */
    __device__ static __forceinline__ int place(int line, int piece) {
        if (ALONG) return line * BK + ((piece ^ (line & 7)) << 3);
        return line * SIDE + ((((piece >> 1) ^ spread(line)) << 1 | (piece & 1)) << 3);
    }
    /* eight elements along memory: (line, col .. col + 7) of an operand of lines x cols; outside: zeros */
    __device__ static __forceinline__ v8 fetch(const Operand& o, uint64_t line, uint64_t lines, uint64_t col, uint64_t cols) {
        v8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (line >= lines) return v;
        for (int j = 0; j < 8; ++j)
            if (col + j < cols) v[j] = EIGHT ? (T)(float)((const int8_t*)o.d)[line * o.ld + col + j] : ((const T*)o.d)[line * o.ld + col + j];
        return v;
    }
    /* elements n * 8 .. of the tile whose corner is (side0, r0), by lane t of TH */
    template <int TH>
    __device__ static __forceinline__ void fill(T* lds, const Operand& o, uint64_t side0, uint64_t sides, uint64_t r0, uint64_t nr, int t) {
        constexpr int PIECES = ALONG ? BK / 8 : SIDE / 8;
        for (int n = t; n < ELEMENTS / 8; n += TH) {
            const int line = n / PIECES, piece = n % PIECES;
            const v8 v = ALONG ? fetch(o, side0 + line, sides, r0 + piece * 8, nr) : fetch(o, r0 + line, nr, side0 + piece * 8, sides);
            *(v8*)(lds + place(line, piece)) = v;
        }
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

/* four neighbouring entries of a row of out, from column p on */
template <class T>
__device__ __forceinline__ void put4(void* base, uint64_t ld, uint32_t q, uint32_t p, uint32_t np, const float* v) {
    T* at = (T*)base + q * ld + p;
    if (p + 4 <= np && ((uintptr_t)at & 7u) == 0) {
        typename Vec<T>::v4 x;
        for (int i = 0; i < 4; ++i) x[i] = (T)v[i];
        *(typename Vec<T>::v4*)at = x;
    } else {
        for (int i = 0; i < 4; ++i)
            if (p + i < np) at[i] = (T)v[i];
    }
}
template <class T>
__device__ __forceinline__ void get4(const void* base, uint64_t ld, uint32_t q, uint32_t p, uint32_t np, float* v) {
    const T* at = (const T*)base + q * ld + p;
    if (p + 4 <= np && ((uintptr_t)at & 7u) == 0) {
        const typename Vec<T>::v4 x = *(const typename Vec<T>::v4*)at;
        for (int i = 0; i < 4; ++i) v[i] = (float)x[i];
    } else {
        for (int i = 0; i < 4; ++i) v[i] = p + i < np ? (float)at[i] : 0.0f;
    }
}
template <class T, bool FORWARD>
__device__ __forceinline__ void finish4(const ProductArgs& a, uint32_t q, uint32_t p, float* v) {
    if (q >= a.nq || p >= a.np) return;
    if (FORWARD) {
        for (int i = 0; i < 4; ++i) {
            if (p + i >= a.np) continue;
            if (a.p_scale) v[i] *= a.p_scale[p + i];
            if (a.bias) v[i] += (float)((const T*)a.bias)[p + i];
        }
        if (a.z) put4<T>(a.z, a.ldz, q, p, a.np, v);
        for (int i = 0; i < 4; ++i) v[i] = activate(v[i], a.act);
        if (a.residual) {
            float r[4];
            get4<T>(a.residual, a.ldres, q, p, a.np, r);
            for (int i = 0; i < 4; ++i) v[i] += r[i];
        }
    } else if (a.factor) {
        const float f = a.factor[0];
        for (int i = 0; i < 4; ++i) v[i] *= f;
    }
    put4<T>(a.out, a.ldo, q, p, a.np, v);
}

template <class T, bool P_ALONG, bool P_EIGHT, bool Q_ALONG, bool Q_EIGHT, bool FORWARD>
__global__ __launch_bounds__(256) void product(const ProductArgs a) {
    constexpr int SP = 128, SQ = 128;
    typedef Tile<T, P_ALONG, P_EIGHT, SP> TP;
    typedef Tile<T, Q_ALONG, Q_EIGHT, SQ> TQ;
    __shared__ __align__(16) T lp[TP::ELEMENTS];
    __shared__ __align__(16) T lq[TQ::ELEMENTS];
    const uint32_t tiles_p = (a.np + SP - 1) / SP;
    const uint64_t p0 = (uint64_t)(blockIdx.x % tiles_p) * SP, q0 = (uint64_t)(blockIdx.x / tiles_p) * SQ;
    const int t = threadIdx.x, lane = t & 63, wp = (t >> 6) & 1, wq = t >> 7;
    f4 acc[4][4] = {};
    for (uint32_t r0 = 0; r0 < a.nr; r0 += BK) {
        __syncthreads();
        TP::template fill<256>(lp, a.p, p0, a.np, r0, a.nr, t);
        TQ::template fill<256>(lq, a.q, q0, a.nq, r0, a.nr, t);
        __syncthreads();
        for (int s = 0; s < 2; ++s) {
            typename Vec<T>::v8 fp[4], fq[4];
            for (int i = 0; i < 4; ++i) fp[i] = TP::fragment(lp, wp * 64 + i * 16, s, lane);
            for (int j = 0; j < 4; ++j) fq[j] = TQ::fragment(lq, wq * 64 + j * 16, s, lane);
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma<T>(fp[i], fq[j], acc[i][j]);
        }
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            finish4<T, FORWARD>(a, (uint32_t)q0 + wq * 64 + j * 16 + (lane & 15), (uint32_t)p0 + wp * 64 + i * 16 + (lane >> 4) * 4, v);
        }
}

/* ---- the gradient before the activation ------------------------------------------------------------------
 * dz = dy act'(z), and its sums over the rows.  int8 operands of the products that follow have a scale for each of the
 * rows that those products sum over; it is put into their other operand here, from the unrounded value: by_x = dz s_x[row] / m_x for dw,
 * by_w = dz s_w[column] / m_w for dx.  So whole numbers enter the matrix instruction exactly and one rounding of the
 * gradient is all there is.  m is the power of two above the largest scale: it keeps float16 in its range and is put back, exactly, after the product. */
struct SlopeArgs {
    const void *dy, *z;
    const float* z_scale;            /* z is int8 where this is set */
    void *dz, *by_x, *by_w;
    const float *x_scale, *w_scale;
    const float* m;                  /* m_x, 1 / m_x, m_w, 1 / m_w */
    float* part;                     /* [gridDim.y][cols] */
    uint64_t lddy, ldz, lddz;        /* by_x, by_w: cols side by side, padded to ld_by */
    uint64_t ld_by;
    uint32_t rows, cols;
    int act;
};
__global__ __launch_bounds__(1024) void scale_peak(const float* x, uint32_t nx, const float* w, uint32_t nw, float* m) {
    __shared__ float cells[16];
    const float* s = blockIdx.x ? w : x;
    const uint32_t n = s ? (blockIdx.x ? nw : nx) : 0;
    float v = 0.0f;
    for (uint32_t i = threadIdx.x; i < n; i += 1024) v = fmaxf(v, finite_magnitude(s[i]));
    v = group_max<1024>(v, cells, threadIdx.x);
    if (threadIdx.x) return;
    int e = v > 0.0f ? ilogbf(v) + 1 : 0;
    e = e < -120 ? -120 : e > 120 ? 120 : e;
    m[2 * blockIdx.x] = ldexpf(1.0f, e);
    m[2 * blockIdx.x + 1] = ldexpf(1.0f, -e);
}
/* A wave takes 512 columns (eight to a lane), the four waves of a workgroup every fourth of its rows. */
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void slopes(const SlopeArgs a) {
    __shared__ float cells[4][512];
    const int w = threadIdx.x >> 6, t = threadIdx.x & 63;
    const uint32_t c0 = blockIdx.x * 512;
    const uint32_t cols = a.cols - c0 < 512 ? a.cols - c0 : 512;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, ws[8];
    const float mx = a.by_x ? a.m[1] : 0.0f, mw = a.by_w ? a.m[3] : 0.0f;
    if (a.by_w)
        for (int j = 0; j < 8; ++j) {
            const uint32_t k = row_col<64, WIDE>(t, 0, j);
            ws[j] = k < cols ? a.w_scale[c0 + k] * mw : 0.0f;
        }
    for (uint64_t row = (uint64_t)blockIdx.y * 4 + w; row < a.rows; row += (uint64_t)gridDim.y * 4) {
        float v[8], z[8];
        load8<T, 64, WIDE>((const T*)a.dy + row * a.lddy + c0, t, 0, cols, v);
        if (a.act != TC_ACT_NONE) {
            if (a.z_scale) load8q<64, WIDE>((const int8_t*)a.z + row * a.ldz + c0, a.z_scale[row], t, 0, cols, z);
            else load8<T, 64, WIDE>((const T*)a.z + row * a.ldz + c0, t, 0, cols, z);
            for (int j = 0; j < 8; ++j) v[j] *= slope(z[j], a.act);
            if (a.dz) store8<T, 64, WIDE>((T*)a.dz + row * a.lddz + c0, t, 0, cols, v);
        }
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
        if (a.by_x) {
            const float f = a.x_scale[row] * mx;
            for (int j = 0; j < 8; ++j) z[j] = v[j] * f;
            store8<T, 64, WIDE>((T*)a.by_x + row * a.ld_by + c0, t, 0, cols, z);
        }
        if (a.by_w) {
            for (int j = 0; j < 8; ++j) z[j] = v[j] * ws[j];
            store8<T, 64, WIDE>((T*)a.by_w + row * a.ld_by + c0, t, 0, cols, z);
        }
    }
    if (!a.part) return;
    for (int j = 0; j < 8; ++j) cells[w][row_col<64, WIDE>(t, 0, j)] = sum[j];
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < cols; k += 256)
        a.part[(uint64_t)blockIdx.y * a.cols + c0 + k] = (cells[0][k] + cells[1][k]) + (cells[2][k] + cells[3][k]);
}
template <class T>
__global__ __launch_bounds__(256) void fill_rows(T* out, uint64_t ld, uint32_t rows, uint32_t cols) {
    const uint64_t n = (uint64_t)rows * cols;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) out[i / cols * ld + i % cols] = (T)0.0f;
}

}  // namespace layers
}  // namespace tc
