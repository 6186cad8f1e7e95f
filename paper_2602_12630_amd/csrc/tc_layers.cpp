/*
 * Host side of the layer operators declared in include/tc.h: checks of the arguments and launches of the kernels of layers.h.
 *
 * Compiled by hipcc for gfx950 (product) or, with -DTC_HOST_EMU, by g++ with plain loops in the place of the
 * launches, which only CPU tests of the checks and of the views use.
 */
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "ctx.h"
#if defined(TC_HOST_EMU)
#include "layers_emu.h"
#else
#include "layers.h"
#endif

using namespace tc;

namespace {

#define TRY(call)                     \
    do {                              \
        int rc_ = (call);             \
        if (rc_ != TC_OK) return rc_; \
    } while (0)
#define REFUSE(code, msg) return ctx_fail(ctx, code, msg)

bool sixteen(int dtype) { return dtype == TC_F16 || dtype == TC_BF16; }

/* a view that the kernels may use: known type, sizes and stride in range, aligned to its elements */
int check_view(tc_ctx* ctx, const tc_matrix* m, bool eight_allowed) {
    if (!m) REFUSE(TC_ERR_ARG, "null matrix");
    if (!sixteen(m->dtype) && !(eight_allowed && m->dtype == TC_I8)) REFUSE(TC_ERR_ARG, "matrix of a type that this argument does not take");
    if (m->cols == 0 || m->cols > TC_LAYER_MAX_COLS || m->rows > 0x7FFFFFFFu) REFUSE(TC_ERR_SHAPE, "rows or columns out of range");
    if (m->ld < m->cols || m->ld > TC_LAYER_MAX_LD) REFUSE(TC_ERR_SHAPE, "row stride shorter than a row, or out of range");
    if (m->rows == 0) return TC_OK;
    if (!m->d_data) REFUSE(TC_ERR_ARG, "null matrix data");
    if (sixteen(m->dtype) && ((uintptr_t)m->d_data & 1u)) REFUSE(TC_ERR_ARG, "misaligned matrix");
    if (m->dtype == TC_I8) {
        if (!m->d_scale) REFUSE(TC_ERR_ARG, "int8 matrix without its scales");
        if ((uintptr_t)m->d_scale & 3u) REFUSE(TC_ERR_ARG, "misaligned scales");
    }
    return TC_OK;
}
int check_shape(tc_ctx* ctx, const tc_matrix* m, uint32_t rows, uint32_t cols) {
    if (m->rows != rows || m->cols != cols) REFUSE(TC_ERR_SHAPE, "matrices of shapes that do not fit together");
    return TC_OK;
}
int check_type(tc_ctx* ctx, const tc_matrix* m, int dtype) {
    if (m->dtype != dtype) REFUSE(TC_ERR_ARG, "matrices of different 16-bit types");
    return TC_OK;
}
int check_vector(tc_ctx* ctx, const void* p, unsigned element) {
    if ((uintptr_t)p & (element - 1)) REFUSE(TC_ERR_ARG, "misaligned vector");
    return TC_OK;
}
int check_workspace(tc_ctx* ctx, const void* ws, size_t have, size_t need) {
    if (!need) return TC_OK;
    if (!ws || have < need) REFUSE(TC_ERR_ARG, "workspace missing or too small");
    if ((uintptr_t)ws & 15u) REFUSE(TC_ERR_ARG, "workspace not aligned to 16 bytes");
    return TC_OK;
}
size_t up(size_t x, size_t a) { return (x + a - 1) / a * a; }

/* rows of the input gradient that one workgroup of its kernel has in flight */
uint32_t norm_back_sets(uint32_t rows, uint32_t cols) {
    if (rows < 1024) return cols <= 512 ? 4 : 1;
    return cols <= 512 ? 16 : cols <= 2048 ? 4 : cols <= 4096 ? 2 : 1;
}
/* workgroups of it: one for each compute unit, each leaves a partial row of gamma's and beta's gradients */
uint32_t norm_back_groups(uint32_t rows, uint32_t cols) {
    const uint32_t sets = norm_back_sets(rows, cols);
    return std::min<uint32_t>(256, (rows + sets - 1) / sets);
}
/* and the most that this or a smaller number of rows has: below 1024 rows a workgroup has fewer of them */
uint32_t norm_back_most_groups(uint32_t rows, uint32_t cols) {
    return std::max(norm_back_groups(rows, cols), norm_back_groups(std::min<uint32_t>(rows, 1023), cols));
}
/* sets of rows over which the gradient before the activation is spread: about eight workgroups for each compute unit */
uint32_t slope_groups(uint32_t rows, uint32_t cols) {
    const uint32_t strips = (cols + 511) / 512;
    return std::max<uint32_t>(1, std::min<uint32_t>((2048 + strips - 1) / strips, (rows + 15) / 16));
}
/* How a product of np x nq results over nr is laid out: the tile, and into how many parts r is split so that there are workgroups for
 * the whole chip. */
struct Layout {
    uint32_t np, nq, side, splits, r_split;
    uint64_t ldp;
    uint64_t tiles(uint32_t s) const { return (uint64_t)((np + s - 1) / s) * ((nq + s - 1) / s); }
    size_t part_bytes() const { return splits > 1 ? (size_t)splits * nq * ldp * 4 : 0; }
};
/* Chosen by what the layouts cost, in microseconds, measured over products of 10^9 to 10^12 multiply-adds: so much for a step of 64 r
 * with one, two .. workgroups on every compute unit (as many as LDS holds), one for a round of workgroups to start and finish in, and
 * for a split the writing and reading of its parts at 6 GB a millisecond and one more launch.  Within 10 % of the best layout
 * wherever both were timed: 8192 x 4096 -> 11008: 256 x 256 641 us, 128 x 128 672, 64 x 64 992; 487 x 11008 -> 4096: 128 x 128 in four parts
 * 52 us, whole 114, 256 x 256 in eight parts 61; 64 x 4096 -> 4096: 64 x 64 in eight parts 15 us, whole 33, 128 x 128 whole 42.  Layouts whose parts do
 * not fit into `room` bytes and tiles larger than `largest` are left out. */
Layout product_layout(uint32_t np, uint32_t nq, uint32_t nr, size_t room, uint32_t largest, double* least) {
    struct Rate {
        uint32_t side, deepest;
        double step[5];
    };
    static const Rate rates[3] = {{256, 1, {1.7}}, {128, 2, {0.75, 0.97}}, {64, 5, {0.48, 0.5, 0.62, 0.75, 0.9}}};
    static const uint32_t parts[] = {1, 2, 3, 4, 6, 8, 12, 16};
    Layout best = {np, nq, 64, 1, nr, up(np, 8)};
    *least = 1e300;
    if (!np || !nq || !nr) return best;              /* no rows: nothing is launched */
    for (const Rate& l : rates) {
        if (l.side > largest) continue;
        for (uint32_t splits : parts) {
            Layout p = {np, nq, l.side, 1, nr, up(np, 8)};
            if (splits > 1) {
                p.r_split = (uint32_t)up((nr + splits - 1) / splits, 64);
                p.splits = (nr + p.r_split - 1) / p.r_split;
                if (p.splits != splits || p.r_split < 256) break;
            }
            if (p.part_bytes() > room) break;
            const double groups = (double)p.tiles(l.side) * splits, steps = (p.r_split + 63) / 64;
            const uint32_t deep = (uint32_t)std::min<double>(l.deepest, std::ceil(groups / 256));
            double rounds = groups / (256.0 * deep);
            if (rounds < 3 || l.deepest == 1) rounds = std::ceil(rounds);
            double cost = rounds * (steps * l.step[deep - 1] + 1);
            if (splits > 1) cost += 4 + (double)p.part_bytes() * 2 / 6e6;
            if (cost < *least) {
                *least = cost;
                best = p;
            }
        }
    }
    return best;
}
/* The largest tiles are one to a compute unit, and a last round with few of them leaves most of the chip idle: where it pays, whole
 * rounds of them take the product up to `cut` of p (or q), and a launch of another layout takes the rest.  8192 x 4096 -> 11008 with gelu: 1376 tiles in
 * 732 us, 1280 of them and 384 of 128 x 128 in 682. */
struct ProductPlan {
    Layout whole, first, rest;
    uint32_t cut;                    /* 0: the product is done as a whole */
    bool cut_p;
    /* the parts of split sums; behind them, the 16-bit copy of an int8 operand, which the kernel of the largest tiles wants */
    size_t part_bytes() const { return std::max(whole.part_bytes(), cut ? rest.part_bytes() : 0); }
    size_t bytes(uint32_t nr) const { return part_bytes() + (whole.side == 256 ? up((size_t)whole.np * nr * 2, 256) : 0); }
};
ProductPlan product_plan(uint32_t np, uint32_t nq, uint32_t nr, size_t room = SIZE_MAX, uint32_t largest = 256) {
    ProductPlan p = {};
    double least;
    p.whole = product_layout(np, nq, nr, room, largest, &least);
    if (p.whole.side != 256 || p.whole.splits > 1) return p;
    const uint32_t tp = (np + 255) / 256, tq = (nq + 255) / 256, rounds = (uint32_t)(p.whole.tiles(256) / 256);
    for (int on_p = 0; on_p < 2; ++on_p) {
        const uint64_t lines = (uint64_t)rounds * 256 / (on_p ? tq : tp);            /* whole lines of tiles in whole rounds */
        if (lines == 0 || lines >= (on_p ? tp : tq)) continue;
        const uint32_t cut = (uint32_t)lines * 256;
        double a, b;
        const Layout first = product_layout(on_p ? cut : np, on_p ? nq : cut, nr, room, largest, &a),
                     rest = product_layout(on_p ? np - cut : np, on_p ? nq : nq - cut, nr, room, largest, &b);
        if (first.side != 256 || first.splits > 1 || a + b + 4 >= least) continue;
        least = a + b + 4;
        p.first = first;
        p.rest = rest;
        p.cut = cut;
        p.cut_p = on_p;
    }
    return p;
}
/* The plan in a workspace of `room` bytes, which may be that of a larger call: sizes do not only grow with the rows (more rows may need no split).  Where there
 * is less than the best plan wants, it is the best one that fits, at the least one without parts and with int8 operands through registers. */
ProductPlan product_plan_in(uint32_t np, uint32_t nq, uint32_t nr, size_t room, bool eight) {
    ProductPlan p = product_plan(np, nq, nr, room);
    if (!eight || p.whole.side != 256 || p.bytes(nr) <= room) return p;
    const size_t copy = p.bytes(nr) - p.part_bytes();
    return room >= copy ? product_plan(np, nq, nr, room - copy) : product_plan(np, nq, nr, room, 128);
}
/* workspace of the linear gradients: where each part lies */
struct BackPlan {
    size_t by_x, by_w, part, m, powers_x, powers_w, split, bytes;
    uint64_t ld_by;
};
/* in = 0: neither dx nor dw is wanted */
BackPlan back_plan(uint32_t rows, uint32_t in, uint32_t out) {
    BackPlan b;
    b.ld_by = up(out, 8);
    const size_t scaled = up((size_t)rows * b.ld_by * 2, 256);
    b.by_x = 0;
    b.by_w = scaled;
    b.part = 2 * scaled;
    b.m = b.part + up((size_t)slope_groups(rows, out) * out * 4, 256);
    b.powers_x = b.m + 256;
    b.powers_w = b.powers_x + up((size_t)rows * 2, 256);
    b.split = b.powers_w + up((size_t)out * 2, 256);
    b.bytes = b.split + (in ? std::max(product_plan(in, rows, out).bytes(out), product_plan(in, out, rows).bytes(rows)) : 0);
    return b;
}

}  // namespace

#if !defined(TC_HOST_EMU)
namespace {
using namespace tc::layers;
#define LAUNCH(kernel, grid, block, lds, args)                                              \
    do {                                                                                    \
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(block), lds, ctx_stream(ctx), args);          \
        int e_ = (int)hipGetLastError();                                                    \
        if (e_) return ctx_fail_hip(ctx, e_, "launch of " #kernel);                         \
    } while (0)

/* Whether a 16-bit output is written past the caches.  The last-level cache holds 256 MB: from half of that on, an output would drive out what the call
 * and the next one read, and little of it is left when it is read itself.  256 MB decoded: 57 us against 70, with a norm that reads them 162
 * against 166; the gradient of a norm of 128 MB 74 against 85, with a checkpoint of it 128 against 125; 8192 x 4096 -> 11008 672 against 686.  Smaller outputs
 * are better read from the cache: 64 MB decoded and normalised 46 us past it, 44 through it.  (A norm's own output gains nothing.) */
bool past_caches(const tc_matrix* m) { return (uint64_t)m->rows * m->cols * 2 >= 128u << 20; }
/* workgroups for `sets` sets of rows; the kernels go round until all are done */
uint32_t row_grid(uint64_t sets) { return (uint32_t)std::min<uint64_t>(sets, 1u << 20); }
template <class T>
int encode_rows(tc_ctx* ctx, const RowArgs& a) {
    const uint32_t c = a.cols;
    if (c < 8) LAUNCH((checkpoint_encode<T, 64, 1, true>), row_grid(((uint64_t)a.rows + 3) / 4), 256, 0, a);
    else if (c <= 512) LAUNCH((checkpoint_encode<T, 64, 1>), row_grid(((uint64_t)a.rows + 3) / 4), 256, 0, a);
    else if (c <= 2048) LAUNCH((checkpoint_encode<T, 256, 1>), row_grid(a.rows), 256, 0, a);
    else if (c <= 4096) LAUNCH((checkpoint_encode<T, 256, 2>), row_grid(a.rows), 256, 0, a);
    else if (c <= 8192) LAUNCH((checkpoint_encode<T, 256, 4>), row_grid(a.rows), 256, 0, a);
    else if (c <= 16384) LAUNCH((checkpoint_encode<T, 256, 8>), row_grid(a.rows), 256, 0, a);
    else LAUNCH((checkpoint_encode<T, 1024, 0>), row_grid(a.rows), 1024, 0, a);
    return TC_OK;
}
template <class T>
int norm_rows(tc_ctx* ctx, const NormArgs& a) {
    const uint32_t c = a.cols;
    if (c < 8) LAUNCH((norm_forward<T, 64, 1, true>), row_grid(((uint64_t)a.rows + 3) / 4), 256, 0, a);
    else if (c <= 512) LAUNCH((norm_forward<T, 64, 1>), row_grid(((uint64_t)a.rows + 3) / 4), 256, 0, a);
    else if (c <= 2048) LAUNCH((norm_forward<T, 256, 1>), row_grid(a.rows), 256, 0, a);
    else if (c <= 4096) LAUNCH((norm_forward<T, 256, 2>), row_grid(a.rows), 256, 0, a);
    else if (c <= 8192) LAUNCH((norm_forward<T, 256, 4>), row_grid(a.rows), 256, 0, a);
    else if (c <= 16384) LAUNCH((norm_forward<T, 1024, 2>), row_grid(a.rows), 1024, 0, a);
    else LAUNCH((norm_forward<T, 1024, 4>), row_grid(a.rows), 1024, 0, a);
    return TC_OK;
}
template <class T, bool EIGHT>
int norm_back_rows(tc_ctx* ctx, const NormBackArgs& a, uint32_t groups) {
    const uint32_t c = a.cols, sets = norm_back_sets(a.rows, c);
    const size_t lds = sets > 1 ? up(c, 8) * 4 : 0;
    if (a.rows < 1024) {                             /* few rows: smaller workgroups, so that they go to more compute units */
        if (c < 8) LAUNCH((norm_backward<T, EIGHT, 64, 1, 256, true>), groups, 256, lds, a);
        else if (c <= 512) LAUNCH((norm_backward<T, EIGHT, 64, 1, 256>), groups, 256, lds, a);
        else if (c <= 2048) LAUNCH((norm_backward<T, EIGHT, 256, 1, 256>), groups, 256, lds, a);
        else if (c <= 4096) LAUNCH((norm_backward<T, EIGHT, 512, 1, 512>), groups, 512, lds, a);
        else if (c <= 8192) LAUNCH((norm_backward<T, EIGHT, 1024, 1, 1024>), groups, 1024, lds, a);
        else if (c <= 16384) LAUNCH((norm_backward<T, EIGHT, 1024, 2, 1024>), groups, 1024, lds, a);
        else LAUNCH((norm_backward<T, EIGHT, 1024, 4, 1024>), groups, 1024, lds, a);
    } else {
        if (c < 8) LAUNCH((norm_backward<T, EIGHT, 64, 1, 1024, true>), groups, 1024, lds, a);
        else if (c <= 512) LAUNCH((norm_backward<T, EIGHT, 64, 1, 1024>), groups, 1024, lds, a);
        else if (c <= 2048) LAUNCH((norm_backward<T, EIGHT, 256, 1, 1024>), groups, 1024, lds, a);
        else if (c <= 4096) LAUNCH((norm_backward<T, EIGHT, 512, 1, 1024>), groups, 1024, lds, a);
        else if (c <= 8192) LAUNCH((norm_backward<T, EIGHT, 1024, 1, 1024>), groups, 1024, lds, a);
        else if (c <= 16384) LAUNCH((norm_backward<T, EIGHT, 1024, 2, 1024>), groups, 1024, lds, a);
        else LAUNCH((norm_backward<T, EIGHT, 1024, 4, 1024>), groups, 1024, lds, a);
    }
    return TC_OK;
}
int sum_columns(tc_ctx* ctx, const float* part, uint64_t stride, uint32_t n, uint32_t cols, float* out, float* second) {
    const ColumnSumArgs a{part, {out, second}, stride, n, cols};
    LAUNCH(column_sums, dim3((cols + 63) / 64, second ? 2 : 1), 1024, 0, a);
    return TC_OK;
}
template <class T>
int clear_rows(tc_ctx* ctx, void* out, uint64_t ld, uint32_t rows, uint32_t cols) {
    const uint64_t n = (uint64_t)rows * cols;
    hipLaunchKernelGGL(fill_rows<T>, dim3((uint32_t)std::min<uint64_t>(2048, (n + 255) / 256)), dim3(256), 0, ctx_stream(ctx), (T*)out, ld, rows, cols);
    int e = (int)hipGetLastError();
    return e ? ctx_fail_hip(ctx, e, "launch of fill_rows") : TC_OK;
}
/* whether an operand can be read in pieces of eight elements (sixteen: `twice`): aligned rows of whole pieces, and a tile's addresses within 31 bits */
bool in_pieces(const Operand& o, uint32_t along_memory, bool eight, bool twice = false) {
    const uint32_t piece = twice ? 16 : 8;
    return ((uintptr_t)o.d & (eight ? piece - 1 : 15u)) == 0 && o.ld % piece == 0 && along_memory % piece == 0 && o.ld < (1u << 21);
}
template <class K>
int launch_product(tc_ctx* ctx, K* kernel, const ProductArgs& a, uint64_t grid, int threads, size_t lds) {
    if (grid * threads > 0xFFFFFFFFull) REFUSE(TC_ERR_SHAPE, "product too large for one launch");
    LAUNCH(kernel, (uint32_t)grid, threads, lds, a);
    return TC_OK;
}
/* A kernel that uses more than the 64 KB of LDS that every kernel may has to say so once on each GPU; `said` has a bit for each. */
int allow_lds(tc_ctx* ctx, const void* kernel, size_t bytes, std::atomic<uint64_t>& said) {
    const uint64_t bit = 1ull << (ctx_device(ctx) & 63);
    if (said.load(std::memory_order_relaxed) & bit) return TC_OK;
    int e = (int)hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e) return ctx_fail_hip(ctx, e, "LDS of a product");
    said.fetch_or(bit, std::memory_order_relaxed);
    return TC_OK;
}
/* one product by one layout; loose: 0, or how its operands have to be read (see Feed) */
template <class T, bool P_ALONG, bool P_EIGHT, bool Q_ALONG, bool FORWARD>
int multiply_by(tc_ctx* ctx, ProductArgs a, const Layout& l, int loose, float* part) {
    a.r_split = l.r_split;
    if (l.splits > 1) {
        a.part = part;
        a.ldp = l.ldp;
    }
    const uint64_t tiles128 = l.tiles(128) * l.splits, tiles64 = l.tiles(64) * l.splits;
    const size_t lds256 = 5 * 512 * 32 * 2, lds128 = 2 * 256 * 64 * 2, lds64 = 2 * 128 * 64 * 2;
    if (loose == 2) TRY(launch_product(ctx, product_paired<T, P_ALONG, P_EIGHT, Q_ALONG, FORWARD, 2, 64, 64, 2, 2>, a, tiles64, 256, lds64));
    else if (loose && l.side > 64) TRY(launch_product(ctx, product_paired<T, P_ALONG, P_EIGHT, Q_ALONG, FORWARD, 1, 128, 128, 2, 2>, a, tiles128, 256, lds128));
    else if (loose) TRY(launch_product(ctx, product_paired<T, P_ALONG, P_EIGHT, Q_ALONG, FORWARD, 1, 64, 64, 2, 2>, a, tiles64, 256, lds64));
    else if (l.side == 256) {
        if constexpr (P_EIGHT) REFUSE(TC_ERR_STATE, "internal: int8 operand that was not widened");
        else {
            auto* kernel = product_deep<T, P_ALONG, Q_ALONG, FORWARD, 256, 256, 2, 4>;
            static std::atomic<uint64_t> said{0};
            TRY(allow_lds(ctx, (const void*)kernel, lds256, said));
            TRY(launch_product(ctx, kernel, a, l.tiles(256) * l.splits, 512, lds256));
        }
    } else if (l.side == 128) TRY(launch_product(ctx, product_paired<T, P_ALONG, P_EIGHT, Q_ALONG, FORWARD, 0, 128, 128, 2, 2>, a, tiles128, 256, lds128));
    else TRY(launch_product(ctx, product_paired<T, P_ALONG, P_EIGHT, Q_ALONG, FORWARD, 0, 64, 64, 2, 2>, a, tiles64, 256, lds64));
    if (l.splits > 1) {
        const uint64_t pieces8 = (uint64_t)((a.np + 7) / 8) * a.nq;
        hipLaunchKernelGGL((join_parts<T, FORWARD>), dim3((uint32_t)((pieces8 + 255) / 256)), dim3(256), 0, ctx_stream(ctx), a, l.splits);
        int e = (int)hipGetLastError();
        if (e) return ctx_fail_hip(ctx, e, "launch of join_parts");
    }
    return TC_OK;
}
/* 16-bit operands in whole pieces, in the one or two launches of the plan */
template <class T, bool P_ALONG, bool Q_ALONG, bool FORWARD>
int multiply_planned(tc_ctx* ctx, const ProductArgs& a, const ProductPlan& plan, float* part) {
    if (!plan.cut) return multiply_by<T, P_ALONG, false, Q_ALONG, FORWARD>(ctx, a, plan.whole, 0, part);
    const uint64_t cut = plan.cut;
    ProductArgs first = a, rest = a;
    auto behind = [](const void* p, uint64_t elements) { return p ? (const char*)p + elements * sizeof(T) : nullptr; };
    if (plan.cut_p) {
        first.np = plan.cut;
        rest.np = a.np - plan.cut;
        rest.p.d = behind(a.p.d, P_ALONG ? cut * a.p.ld : cut);
        rest.out = (void*)behind(a.out, cut);
        rest.p_scale = a.p_scale ? a.p_scale + cut : nullptr;
        rest.bias = behind(a.bias, cut);
        rest.residual = behind(a.residual, cut);
        rest.z = (void*)behind(a.z, cut);
    } else {
        first.nq = plan.cut;
        rest.nq = a.nq - plan.cut;
        rest.q.d = behind(a.q.d, Q_ALONG ? cut * a.q.ld : cut);
        rest.out = (void*)behind(a.out, cut * a.ldo);
        rest.residual = behind(a.residual, cut * a.ldres);
        rest.z = (void*)behind(a.z, cut * a.ldz);
    }
    TRY((multiply_by<T, P_ALONG, false, Q_ALONG, FORWARD>(ctx, first, plan.first, 0, part)));
    return multiply_by<T, P_ALONG, false, Q_ALONG, FORWARD>(ctx, rest, plan.rest, 0, part);
}
template <class T, bool P_ALONG, bool P_EIGHT, bool Q_ALONG, bool FORWARD>
int multiply(tc_ctx* ctx, ProductArgs a, float* part, size_t room) {
    /* Up to sixteen rows: a pass over the weights alone, 1 x 4096 -> 4096 in 6.9 us against 10.5 by tiles.  Every workgroup reads all of x, though:
     * beyond eight rows, 16-bit weights that are past the caches' help go by tiles (16 x 4096 -> 11008: 18.4 us against 25.0). */
    if constexpr (FORWARD) {
        const bool few = a.nq <= 8 || (a.nq <= 16 && (P_EIGHT || (uint64_t)a.np * a.nr <= 1u << 25));
        constexpr int waves = P_EIGHT ? 16 : 8;
        if (few && in_pieces(a.p, a.nr, P_EIGHT, true) && in_pieces(a.q, a.nr, false, true))
            return launch_product(ctx, product_thin<T, P_EIGHT, waves>, a, (a.np + 15) / 16, waves * 64, 0);
    }
    const ProductPlan plan = product_plan_in(a.np, a.nq, a.nr, part ? room : 0, P_EIGHT);
    const uint32_t along_p = P_ALONG ? a.nr : a.np, along_q = Q_ALONG ? a.nr : a.nq;
    if (!in_pieces(a.p, along_p, P_EIGHT) || !in_pieces(a.q, along_q, false))
        return multiply_by<T, P_ALONG, P_EIGHT, Q_ALONG, FORWARD>(ctx, a, plan.whole, along_p < 8 || along_q < 8 ? 2 : 1, part);
    if constexpr (P_EIGHT) {
        if (plan.whole.side != 256) return multiply_by<T, P_ALONG, true, Q_ALONG, FORWARD>(ctx, a, plan.whole, 0, part);
        const uint32_t lines = P_ALONG ? a.np : a.nr, cols = along_p;
        T* wide = (T*)((uint8_t*)part + plan.part_bytes());
        hipLaunchKernelGGL(widen_rows<T>, dim3((cols + 2047) / 2048, std::min<uint32_t>(lines, 65535)), dim3(256), 0, ctx_stream(ctx), a.p, a.powers, wide, cols, lines, cols);
        int e = (int)hipGetLastError();
        if (e) return ctx_fail_hip(ctx, e, "launch of widen_rows");
        a.p = Operand{wide, cols};
    }
    return multiply_planned<T, P_ALONG, Q_ALONG, FORWARD>(ctx, a, plan, part);
}

template <class T>
int run_encode(tc_ctx* ctx, const tc_matrix* src, const tc_matrix* dst) {
    const RowArgs a{src->d_data, dst->d_data, dst->d_scale, src->ld, dst->ld, src->rows, src->cols, false};
    return encode_rows<T>(ctx, a);
}
template <class T>
int run_decode(tc_ctx* ctx, const tc_matrix* src, const tc_matrix* dst) {
    const RowArgs a{src->d_data, dst->d_data, src->d_scale, src->ld, dst->ld, src->rows, src->cols, past_caches(dst)};
    const dim3 grid((a.cols + 2047) / 2048, std::min<uint32_t>(a.rows, 65535));
    if (a.cols < 8) LAUNCH((checkpoint_decode<T, true>), grid, 256, 0, a);
    else LAUNCH((checkpoint_decode<T, false>), grid, 256, 0, a);
    return TC_OK;
}
template <class T>
int run_norm(tc_ctx* ctx, int kind, const tc_matrix* x, const void* gamma, const void* beta, float eps, const tc_matrix* y, float* mean, float* rstd) {
    const NormArgs a{x->d_data, x->dtype == TC_I8 ? x->d_scale : nullptr, gamma, beta, y->d_data, mean, rstd, x->ld, y->ld, x->rows, x->cols, eps, kind == TC_NORM_LAYER};
    return norm_rows<T>(ctx, a);
}
template <class T>
int run_norm_backward(tc_ctx* ctx, int kind, const tc_matrix* dy, const tc_matrix* x, const void* gamma, const float* mean, const float* rstd,
                      const tc_matrix* dx, float* dgamma, float* dbeta, void* ws) {
    const uint32_t groups = norm_back_groups(dy->rows, dy->cols);
    float* part = dgamma || dbeta ? (float*)ws : nullptr;
    const NormBackArgs a{dy->d_data, x->d_data, x->dtype == TC_I8 ? x->d_scale : nullptr, gamma, mean, rstd, dx ? dx->d_data : nullptr, part,
                         dy->ld, x->ld, dx ? dx->ld : 0, dy->rows, dy->cols, kind == TC_NORM_LAYER, past_caches(dy)};
    TRY((a.scale ? norm_back_rows<T, true>(ctx, a, groups) : norm_back_rows<T, false>(ctx, a, groups)));
    return part ? sum_columns(ctx, part, 2 * (uint64_t)dy->cols, groups, dy->cols, dgamma, dbeta) : TC_OK;
}
template <class T>
int run_linear(tc_ctx* ctx, const tc_matrix* x, const tc_matrix* w, const void* bias, int act, const tc_matrix* residual, const tc_matrix* y, const tc_matrix* z,
               void* ws, size_t ws_bytes) {
    ProductArgs a = {};
    a.p = Operand{w->d_data, w->ld};
    a.q = Operand{x->d_data, x->ld};
    a.np = w->rows;
    a.nq = x->rows;
    a.nr = w->cols;
    a.out = y->d_data;
    a.ldo = y->ld;
    a.p_scale = w->dtype == TC_I8 ? w->d_scale : nullptr;
    a.bias = bias;
    if (residual) { a.residual = residual->d_data; a.ldres = residual->ld; }
    if (z) { a.z = z->d_data; a.ldz = z->ld; }
    a.act = act;
    a.past = past_caches(y);
    return a.p_scale ? multiply<T, true, true, true, true>(ctx, a, (float*)ws, ws_bytes) : multiply<T, true, false, true, true>(ctx, a, (float*)ws, ws_bytes);
}
template <class T>
int run_linear_backward(tc_ctx* ctx, const tc_matrix* dy, const tc_matrix* x, const tc_matrix* w, int act, const tc_matrix* z, const tc_matrix* dz,
                        const tc_matrix* dx, const tc_matrix* dw, float* dbias, void* ws, size_t ws_bytes) {
    const uint32_t rows = dy->rows, out = dy->cols;
    const BackPlan plan = back_plan(rows, dx ? dx->cols : dw ? dw->cols : 0, out);
    const size_t room = ws_bytes - plan.split;
    uint8_t* base = (uint8_t*)ws;
    /* float16: the scales' powers of two apart from the rest of them (see slopes) */
    float *m = std::is_same<T, _Float16>::value ? (float*)(base + plan.m) : nullptr, *parts = (float*)(base + plan.split);
    const bool by_x = dw && x->dtype == TC_I8, by_w = dx && w->dtype == TC_I8;
    if (m && (by_x || by_w)) {
        hipLaunchKernelGGL(scale_peak, dim3(2), dim3(1024), 0, ctx_stream(ctx), by_x ? x->d_scale : nullptr, rows, by_w ? w->d_scale : nullptr, out, m);
        int e = (int)hipGetLastError();
        if (e) return ctx_fail_hip(ctx, e, "launch of scale_peak");
    }
    /* (whatever else the call asks for, so that a sum does not depend on that) */
    const bool direct = act == TC_ACT_NONE && dbias && rows <= 2048;
    if (direct) {
        const T* d = (const T*)dy->d_data;
        const dim3 grid((out + 63) / 64), block(1024);
        if (out < 8) hipLaunchKernelGGL((bias_sums<T, true>), grid, block, 0, ctx_stream(ctx), d, dy->ld, rows, out, dbias);
        else hipLaunchKernelGGL((bias_sums<T, false>), grid, block, 0, ctx_stream(ctx), d, dy->ld, rows, out, dbias);
        int e = (int)hipGetLastError();
        if (e) return ctx_fail_hip(ctx, e, "launch of bias_sums");
        dbias = nullptr;
    }
    if (act != TC_ACT_NONE || by_x || by_w || dbias) {
        SlopeArgs s = {};
        s.dy = dy->d_data;
        s.lddy = dy->ld;
        if (act != TC_ACT_NONE) {
            s.z = z->d_data;
            s.z_scale = z->dtype == TC_I8 ? z->d_scale : nullptr;
            s.ldz = z->ld;
            s.dz = dz->d_data;
            s.lddz = dz->ld;
        }
        s.by_x = by_x ? base + plan.by_x : nullptr;
        s.by_w = by_w ? base + plan.by_w : nullptr;
        s.x_scale = by_x ? x->d_scale : nullptr;
        s.w_scale = by_w ? w->d_scale : nullptr;
        s.m = m;
        s.powers_x = (uint16_t*)(base + plan.powers_x);
        s.powers_w = (uint16_t*)(base + plan.powers_w);
        s.part = dbias ? (float*)(base + plan.part) : nullptr;
        s.ld_by = plan.ld_by;
        s.rows = rows;
        s.cols = out;
        s.act = act;
        const uint32_t groups = slope_groups(rows, out);
        const dim3 grid((out + 511) / 512, groups);
        if (out < 8) LAUNCH((slopes<T, true>), grid, 256, 0, s);
        else LAUNCH((slopes<T, false>), grid, 256, 0, s);
        if (dbias) TRY(sum_columns(ctx, s.part, out, groups, out, dbias, nullptr));
    }
    const Operand plain = act == TC_ACT_NONE ? Operand{dy->d_data, dy->ld} : Operand{dz->d_data, dz->ld};
    if (dx) {
        ProductArgs a = {};
        a.p = Operand{w->d_data, w->ld};
        a.q = by_w ? Operand{base + plan.by_w, plan.ld_by} : plain;
        a.np = w->cols;
        a.nq = rows;
        a.nr = out;
        a.out = dx->d_data;
        a.ldo = dx->ld;
        a.factor = by_w && m ? m + 2 : nullptr;
        a.powers = by_w && m ? (const uint16_t*)(base + plan.powers_w) : nullptr;
        a.past = past_caches(dx);
        TRY((by_w ? multiply<T, false, true, true, false>(ctx, a, parts, room) : multiply<T, false, false, true, false>(ctx, a, parts, room)));
    }
    if (dw) {
        ProductArgs a = {};
        a.p = Operand{x->d_data, x->ld};
        a.q = by_x ? Operand{base + plan.by_x, plan.ld_by} : plain;
        a.np = x->cols;
        a.nq = out;
        a.nr = rows;
        a.out = dw->d_data;
        a.ldo = dw->ld;
        a.factor = by_x ? m : nullptr;
        a.powers = by_x && m ? (const uint16_t*)(base + plan.powers_x) : nullptr;
        a.past = past_caches(dw);
        TRY((by_x ? multiply<T, false, true, false, false>(ctx, a, parts, room) : multiply<T, false, false, false, false>(ctx, a, parts, room)));
    }
    return TC_OK;
}
}  // namespace
#endif

#if defined(TC_HOST_EMU)
#define RUN(name, dtype, ...) (emu::name(dtype, __VA_ARGS__), TC_OK)
#else
#define RUN(name, dtype, ...) ((dtype) == TC_F16 ? run_##name<_Float16>(ctx, __VA_ARGS__) : run_##name<__bf16>(ctx, __VA_ARGS__))
#endif

extern "C" int tc_checkpoint_encode(tc_ctx* ctx, const tc_matrix* src, const tc_matrix* dst) {
    if (!ctx) return TC_ERR_ARG;
    TRY(check_view(ctx, src, false));
    TRY(check_view(ctx, dst, true));
    if (dst->dtype != TC_I8) REFUSE(TC_ERR_ARG, "a checkpoint is int8");
    TRY(check_shape(ctx, dst, src->rows, src->cols));
    if (!src->rows) return TC_OK;
    TRY(ctx_use_device(ctx));
    return RUN(encode, src->dtype, src, dst);
}
extern "C" int tc_checkpoint_decode(tc_ctx* ctx, const tc_matrix* src, const tc_matrix* dst) {
    if (!ctx) return TC_ERR_ARG;
    TRY(check_view(ctx, src, true));
    if (src->dtype != TC_I8) REFUSE(TC_ERR_ARG, "a checkpoint is int8");
    TRY(check_view(ctx, dst, false));
    TRY(check_shape(ctx, dst, src->rows, src->cols));
    if (!src->rows) return TC_OK;
    TRY(ctx_use_device(ctx));
    return RUN(decode, dst->dtype, src, dst);
}

extern "C" int tc_norm(tc_ctx* ctx, int kind, const tc_matrix* x, const void* d_gamma, const void* d_beta, float eps, const tc_matrix* y,
                       float* d_mean, float* d_rstd) {
    if (!ctx) return TC_ERR_ARG;
    if (kind != TC_NORM_LAYER && kind != TC_NORM_RMS) REFUSE(TC_ERR_ARG, "unknown norm");
    if (!(eps > 0.0f && eps < 1.0f)) REFUSE(TC_ERR_ARG, "eps outside (0, 1)");
    TRY(check_view(ctx, x, true));
    TRY(check_view(ctx, y, false));
    if (x->dtype != TC_I8) TRY(check_type(ctx, x, y->dtype));
    TRY(check_shape(ctx, y, x->rows, x->cols));
    if (x->cols > TC_NORM_MAX_COLS) REFUSE(TC_ERR_SHAPE, "rows longer than TC_NORM_MAX_COLS");
    TRY(check_vector(ctx, d_gamma, 2));
    TRY(check_vector(ctx, d_beta, 2));
    TRY(check_vector(ctx, d_mean, 4));
    TRY(check_vector(ctx, d_rstd, 4));
    if (!x->rows) return TC_OK;
    TRY(ctx_use_device(ctx));
    return RUN(norm, y->dtype, kind, x, d_gamma, d_beta, eps, y, d_mean, d_rstd);
}
extern "C" int tc_norm_backward_workspace(uint32_t rows, uint32_t cols, size_t* bytes) {
    if (!bytes) return TC_ERR_ARG;
    if (rows > 0x7FFFFFFFu || cols == 0 || cols > TC_NORM_MAX_COLS) return TC_ERR_SHAPE;
    *bytes = (size_t)norm_back_most_groups(rows, cols) * 2 * cols * 4;
    return TC_OK;
}
extern "C" int tc_norm_backward(tc_ctx* ctx, int kind, const tc_matrix* dy, const tc_matrix* x, const void* d_gamma, const float* d_mean,
                                const float* d_rstd, const tc_matrix* dx, float* d_dgamma, float* d_dbeta, void* d_workspace,
                                size_t workspace_bytes) {
    if (!ctx) return TC_ERR_ARG;
    if (kind != TC_NORM_LAYER && kind != TC_NORM_RMS) REFUSE(TC_ERR_ARG, "unknown norm");
    TRY(check_view(ctx, dy, false));
    TRY(check_view(ctx, x, true));
    if (x->dtype != TC_I8) TRY(check_type(ctx, x, dy->dtype));
    TRY(check_shape(ctx, x, dy->rows, dy->cols));
    if (dx) {
        TRY(check_view(ctx, dx, false));
        TRY(check_type(ctx, dx, dy->dtype));
        TRY(check_shape(ctx, dx, dy->rows, dy->cols));
    }
    if (dy->cols > TC_NORM_MAX_COLS) REFUSE(TC_ERR_SHAPE, "rows longer than TC_NORM_MAX_COLS");
    if (dy->rows && (!d_rstd || (kind == TC_NORM_LAYER && !d_mean))) REFUSE(TC_ERR_ARG, "statistics of the forward pass missing");
    TRY(check_vector(ctx, d_gamma, 2));
    TRY(check_vector(ctx, d_mean, 4));
    TRY(check_vector(ctx, d_rstd, 4));
    TRY(check_vector(ctx, d_dgamma, 4));
    TRY(check_vector(ctx, d_dbeta, 4));
    if (!dx && !d_dgamma && !d_dbeta) return TC_OK;
    if (d_dgamma || d_dbeta) {
        size_t need = 0;
        TRY(tc_norm_backward_workspace(dy->rows, dy->cols, &need));
        TRY(check_workspace(ctx, d_workspace, workspace_bytes, need));
    }
    TRY(ctx_use_device(ctx));
    if (!dy->rows) {
#if !defined(TC_HOST_EMU)
        if (d_dgamma) TRY(clear_rows<float>(ctx, d_dgamma, dy->cols, 1, dy->cols));
        if (d_dbeta) TRY(clear_rows<float>(ctx, d_dbeta, dy->cols, 1, dy->cols));
        return TC_OK;
#endif
    }
    return RUN(norm_backward, dy->dtype, kind, dy, x, d_gamma, d_mean, d_rstd, dx, d_dgamma, d_dbeta, d_workspace);
}

static bool linear_sizes(uint32_t rows, uint32_t in, uint32_t out) {
    return rows <= 0x7FFFFFFFu && in >= 1 && in <= TC_LAYER_MAX_COLS && out >= 1 && out <= TC_LAYER_MAX_COLS;
}
extern "C" int tc_linear_workspace(uint32_t rows, uint32_t in, uint32_t out, size_t* bytes) {
    if (!bytes) return TC_ERR_ARG;
    if (!linear_sizes(rows, in, out)) return TC_ERR_SHAPE;
    *bytes = product_plan(out, rows, in).bytes(in);
    return TC_OK;
}
extern "C" int tc_linear(tc_ctx* ctx, const tc_matrix* x, const tc_matrix* w, const void* d_bias, int activation, const tc_matrix* residual,
                         const tc_matrix* y, const tc_matrix* z, void* d_workspace, size_t workspace_bytes) {
    if (!ctx) return TC_ERR_ARG;
    if (activation < TC_ACT_NONE || activation > TC_ACT_SILU) REFUSE(TC_ERR_ARG, "unknown activation");
    TRY(check_view(ctx, x, false));
    TRY(check_view(ctx, w, true));
    if (!w->rows) REFUSE(TC_ERR_SHAPE, "weights without rows");
    if (w->dtype != TC_I8) TRY(check_type(ctx, w, x->dtype));
    if (w->cols != x->cols || w->rows > TC_LAYER_MAX_COLS) REFUSE(TC_ERR_SHAPE, "weights whose shape does not fit the input");
    const tc_matrix* outs[3] = {y, residual, z};
    for (int i = 0; i < 3; ++i) {
        if (i && !outs[i]) continue;
        TRY(check_view(ctx, outs[i], false));
        TRY(check_type(ctx, outs[i], x->dtype));
        TRY(check_shape(ctx, outs[i], x->rows, w->rows));
    }
    TRY(check_vector(ctx, d_bias, 2));
    size_t most = 0;
    TRY(tc_linear_workspace(x->rows, x->cols, w->rows, &most));
    workspace_bytes = d_workspace ? std::min(workspace_bytes, most) : 0;
    TRY(check_workspace(ctx, d_workspace, workspace_bytes, workspace_bytes ? 1 : 0));
    if (!x->rows) return TC_OK;
    TRY(ctx_use_device(ctx));
    return RUN(linear, x->dtype, x, w, d_bias, activation, residual, y, z, d_workspace, workspace_bytes);
}
extern "C" int tc_linear_backward_workspace(uint32_t rows, uint32_t in, uint32_t out, size_t* bytes) {
    if (!bytes) return TC_ERR_ARG;
    if (!linear_sizes(rows, in, out)) return TC_ERR_SHAPE;
    *bytes = back_plan(rows, in, out).bytes;
    return TC_OK;
}
extern "C" int tc_linear_backward(tc_ctx* ctx, const tc_matrix* dy, const tc_matrix* x, const tc_matrix* w, int activation, const tc_matrix* z,
                                  const tc_matrix* dz, const tc_matrix* dx, const tc_matrix* dw, float* d_dbias, void* d_workspace,
                                  size_t workspace_bytes) {
    if (!ctx) return TC_ERR_ARG;
    if (activation < TC_ACT_NONE || activation > TC_ACT_SILU) REFUSE(TC_ERR_ARG, "unknown activation");
    TRY(check_view(ctx, dy, false));
    const uint32_t rows = dy->rows, out = dy->cols;
    uint32_t in = 0;
    if (activation == TC_ACT_NONE) {
        if (z || dz) REFUSE(TC_ERR_ARG, "without an activation z and dz must be null");
    } else {
        TRY(check_view(ctx, z, true));
        TRY(check_view(ctx, dz, false));
        if (z->dtype != TC_I8) TRY(check_type(ctx, z, dy->dtype));
        TRY(check_type(ctx, dz, dy->dtype));
        TRY(check_shape(ctx, z, rows, out));
        TRY(check_shape(ctx, dz, rows, out));
    }
    if (dx) {
        TRY(check_view(ctx, dx, false));
        TRY(check_type(ctx, dx, dy->dtype));
        in = dx->cols;
        TRY(check_shape(ctx, dx, rows, in));
        TRY(check_view(ctx, w, true));
        if (w->dtype != TC_I8) TRY(check_type(ctx, w, dy->dtype));
        TRY(check_shape(ctx, w, out, in));
    }
    if (dw) {
        TRY(check_view(ctx, dw, false));
        TRY(check_type(ctx, dw, dy->dtype));
        if (dx && dw->cols != in) REFUSE(TC_ERR_SHAPE, "matrices of shapes that do not fit together");
        in = dw->cols;
        TRY(check_shape(ctx, dw, out, in));
        TRY(check_view(ctx, x, true));
        if (x->dtype != TC_I8) TRY(check_type(ctx, x, dy->dtype));
        TRY(check_shape(ctx, x, rows, in));
    }
    TRY(check_vector(ctx, d_dbias, 4));
    TRY(check_workspace(ctx, d_workspace, workspace_bytes, back_plan(rows, in, out).split));
    TRY(ctx_use_device(ctx));
    if (!rows) {
#if !defined(TC_HOST_EMU)
        if (dw) TRY(dw->dtype == TC_F16 ? clear_rows<_Float16>(ctx, dw->d_data, dw->ld, out, in) : clear_rows<__bf16>(ctx, dw->d_data, dw->ld, out, in));
        if (d_dbias) TRY(clear_rows<float>(ctx, d_dbias, out, 1, out));
        return TC_OK;
#endif
    }
    return RUN(linear_backward, dy->dtype, dy, x, w, activation, z, dz, dx, dw, d_dbias, d_workspace, workspace_bytes);
}
