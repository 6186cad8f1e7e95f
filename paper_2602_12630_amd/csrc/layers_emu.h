/*
 * The layer operators as plain loops on the host, from their definitions: what the CPU build of the tests runs in the place of
 * the kernels, so that the checks, the views and the outputs that a call leaves alone can be tested without a GPU.
 */
#pragma once
#include <math.h>
#include <string.h>

#include <vector>

namespace emu {

inline float half_value(uint16_t h) {
    const int e = h >> 10 & 31, m = h & 1023;
    const float v = e == 31 ? (m ? NAN : INFINITY) : e ? ldexpf((float)(m + 1024), e - 25) : ldexpf((float)m, -24);
    return h >> 15 ? -v : v;
}
inline uint16_t half_bits(float f) {
    const uint16_t s = signbit(f) ? 0x8000 : 0;
    const float a = fabsf(f);
    if (a != a) return s | 0x7E00;
    if (a >= 65520.0f) return s | 0x7C00;
    if (a < 6.103515625e-05f) return s | (uint16_t)rintf(ldexpf(a, 24));
    int e;
    const float m = frexpf(a, &e);                        /* a = m 2^e, m in [1/2, 1) */
    return s + (uint16_t)((e + 13) << 10) + (uint16_t)rintf(ldexpf(m, 11));      /* a mantissa rounded up to 2048 carries into the exponent */
}
inline float brain_value(uint16_t h) {
    const uint32_t u = (uint32_t)h << 16;
    float f;
    memcpy(&f, &u, 4);
    return f;
}
inline uint16_t brain_bits(float f) {
    uint32_t u;
    memcpy(&u, &f, 4);
    if (f != f) return (uint16_t)(u >> 16 | 0x40);
    return (uint16_t)((u + 0x7FFF + (u >> 16 & 1)) >> 16);
}
inline float load16(const void* p, size_t i, int dtype) {
    const uint16_t h = ((const uint16_t*)p)[i];
    return dtype == TC_F16 ? half_value(h) : brain_value(h);
}
inline void store16(void* p, size_t i, int dtype, double v) {
    ((uint16_t*)p)[i] = dtype == TC_F16 ? half_bits((float)v) : brain_bits((float)v);
}
inline double get(const tc_matrix* m, size_t r, size_t c) {
    const size_t i = r * m->ld + c;
    return m->dtype == TC_I8 ? (double)m->d_scale[r] * ((const int8_t*)m->d_data)[i] : load16(m->d_data, i, m->dtype);
}
inline void put(const tc_matrix* m, size_t r, size_t c, double v) { store16(m->d_data, r * m->ld + c, m->dtype, v); }
inline double phi(double z) { return 0.5 * erfc(-z / sqrt(2.0)); }
inline double activate(double z, int act) {
    if (act == TC_ACT_RELU) return z > 0 ? z : 0;
    if (act == TC_ACT_GELU) return z * phi(z);
    if (act == TC_ACT_SILU) return z / (1 + exp(-z));
    return z;
}
inline double slope(double z, int act) {
    if (act == TC_ACT_RELU) return z > 0 ? 1 : 0;
    if (act == TC_ACT_GELU) return phi(z) + z * exp(-0.5 * z * z) / sqrt(2 * M_PI);
    if (act == TC_ACT_SILU) {
        const double s = 1 / (1 + exp(-z));
        return s + z * s * (1 - s);
    }
    return 1;
}

inline void encode(int, const tc_matrix* src, const tc_matrix* dst) {
    for (size_t r = 0; r < src->rows; ++r) {
        double amax = 0;
        for (size_t c = 0; c < src->cols; ++c) {
            const double a = fabs(get(src, r, c));
            if (isfinite(a) && a > amax) amax = a;
        }
        dst->d_scale[r] = (float)amax / 127.0f;
        for (size_t c = 0; c < src->cols; ++c) {
            const double x = get(src, r, c);
            const double q = x != x ? 0 : isinf(x) ? copysign(127, x) : amax > 0 ? rint(127 * x / amax) : 0;
            ((int8_t*)dst->d_data)[r * dst->ld + c] = (int8_t)q;
        }
    }
}
inline void decode(int, const tc_matrix* src, const tc_matrix* dst) {
    for (size_t r = 0; r < src->rows; ++r)
        for (size_t c = 0; c < src->cols; ++c) put(dst, r, c, get(src, r, c));
}
inline void norm(int dtype, int kind, const tc_matrix* x, const void* gamma, const void* beta, float eps, const tc_matrix* y, float* mean, float* rstd) {
    for (size_t r = 0; r < x->rows; ++r) {
        double mu = 0, var = 0;
        if (kind == TC_NORM_LAYER) {
            for (size_t c = 0; c < x->cols; ++c) mu += get(x, r, c);
            mu /= x->cols;
        }
        for (size_t c = 0; c < x->cols; ++c) var += (get(x, r, c) - mu) * (get(x, r, c) - mu);
        const double s = 1 / sqrt(var / x->cols + eps);
        if (mean) mean[r] = (float)mu;
        if (rstd) rstd[r] = (float)s;
        for (size_t c = 0; c < x->cols; ++c)
            put(y, r, c, (get(x, r, c) - mu) * s * (gamma ? load16(gamma, c, dtype) : 1) + (beta ? load16(beta, c, dtype) : 0));
    }
}
inline void norm_backward(int dtype, int kind, const tc_matrix* dy, const tc_matrix* x, const void* gamma, const float* mean, const float* rstd,
                          const tc_matrix* dx, float* dgamma, float* dbeta, void*) {
    const size_t n = dy->cols;
    std::vector<double> dg(n, 0), db(n, 0), g(n), h(n);
    for (size_t r = 0; r < dy->rows; ++r) {
        double mg = 0, mgh = 0;
        for (size_t c = 0; c < n; ++c) {
            const double d = get(dy, r, c);
            h[c] = (get(x, r, c) - (kind == TC_NORM_LAYER ? mean[r] : 0)) * rstd[r];
            g[c] = d * (gamma ? load16(gamma, c, dtype) : 1);
            dg[c] += d * h[c];
            db[c] += d;
            mg += g[c] / n;
            mgh += g[c] * h[c] / n;
        }
        if (dx)
            for (size_t c = 0; c < n; ++c) put(dx, r, c, rstd[r] * (g[c] - (kind == TC_NORM_LAYER ? mg : 0) - h[c] * mgh));
    }
    for (size_t c = 0; c < n; ++c) {
        if (dgamma) dgamma[c] = (float)dg[c];
        if (dbeta) dbeta[c] = (float)db[c];
    }
}
inline void linear(int dtype, const tc_matrix* x, const tc_matrix* w, const void* bias, int act, const tc_matrix* residual, const tc_matrix* y, const tc_matrix* z, void*, size_t) {
    for (size_t r = 0; r < x->rows; ++r)
        for (size_t o = 0; o < w->rows; ++o) {
            double v = bias ? load16(bias, o, dtype) : 0;
            for (size_t i = 0; i < x->cols; ++i) v += get(x, r, i) * get(w, o, i);
            const double add = residual ? get(residual, r, o) : 0;
            if (z) put(z, r, o, v);
            put(y, r, o, activate(v, act) + add);
        }
}
inline void linear_backward(int, const tc_matrix* dy, const tc_matrix* x, const tc_matrix* w, int act, const tc_matrix* z, const tc_matrix* dz,
                            const tc_matrix* dx, const tc_matrix* dw, float* dbias, void*, size_t) {
    const size_t rows = dy->rows, out = dy->cols, in = dx ? dx->cols : dw ? dw->cols : 0;
    std::vector<double> d(rows * out);
    for (size_t r = 0; r < rows; ++r)
        for (size_t o = 0; o < out; ++o) {
            d[r * out + o] = get(dy, r, o) * (act == TC_ACT_NONE ? 1 : slope(get(z, r, o), act));
            if (act != TC_ACT_NONE) put(dz, r, o, d[r * out + o]);
        }
    for (size_t o = 0; dbias && o < out; ++o) {
        double s = 0;
        for (size_t r = 0; r < rows; ++r) s += d[r * out + o];
        dbias[o] = (float)s;
    }
    for (size_t r = 0; dx && r < rows; ++r)
        for (size_t i = 0; i < in; ++i) {
            double s = 0;
            for (size_t o = 0; o < out; ++o) s += d[r * out + o] * get(w, o, i);
            put(dx, r, i, s);
        }
    for (size_t o = 0; dw && o < out; ++o)
        for (size_t i = 0; i < in; ++i) {
            double s = 0;
            for (size_t r = 0; r < rows; ++r) s += d[r * out + o] * get(x, r, i);
            put(dw, o, i, s);
        }
}

}  // namespace emu
