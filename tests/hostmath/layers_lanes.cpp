// The layer operators' own kernels and launches, lane by lane on the host under AddressSanitizer and UBSan: operands, outputs, parameters and
// workspaces are blocks of exactly their size, what lies between rows and LDS beyond what a launch asks for is poisoned, so that an access
// that the GPU would make silently, or fault on, stops this program.  Tiles on their way to LDS are besides compared with what belongs there.
// Built and run by tests/test_layers_lanes.py, with lanes/hip/hip_runtime.h in the place of HIP's.
#define TC_HOST_EMU
#include "../../paper_2602_12630_amd/csrc/ctx.h"
#undef TC_HOST_EMU
#include "../../paper_2602_12630_amd/csrc/tc_layers.cpp"

#include <sanitizer/asan_interface.h>

#include <memory>
#include <random>

namespace tc {
rt::stream_t ctx_stream(const tc_ctx*) { return {}; }
int ctx_device(const tc_ctx*) { return 0; }
int ctx_use_device(tc_ctx*) { return TC_OK; }
int ctx_fail(tc_ctx*, int code, const char* msg) {
    fprintf(stderr, "%s\n", msg);
    return code;
}
int ctx_fail_hip(tc_ctx*, int, const char*) { return TC_ERR_HIP; }
namespace layers {
__align__(16) uint8_t lds_bytes[160 * 1024];
float lds[1 << 15];
}  // namespace layers
}  // namespace tc
namespace lanes {
uint32_t most_blocks = 6;
bool skipped = false;
void take_lds(size_t bytes) {
    ASAN_UNPOISON_MEMORY_REGION(tc::layers::lds_bytes, sizeof tc::layers::lds_bytes);
    ASAN_UNPOISON_MEMORY_REGION(tc::layers::lds, sizeof tc::layers::lds);
    if (bytes > sizeof tc::layers::lds_bytes) abort();
    ASAN_POISON_MEMORY_REGION(tc::layers::lds_bytes + bytes, sizeof tc::layers::lds_bytes - bytes);
    if (bytes <= sizeof tc::layers::lds) ASAN_POISON_MEMORY_REGION((uint8_t*)tc::layers::lds + bytes, sizeof tc::layers::lds - bytes);
}
}  // namespace lanes

static std::mt19937 gen(1);
static const char* what = "";
#define OK(call)                                                                        \
    do {                                                                                \
        const int rc_ = (call);                                                         \
        if (rc_ != TC_OK) {                                                             \
            fprintf(stderr, "%s:%d: %s -> %d (%s)\n", __FILE__, __LINE__, #call, rc_, what); \
            exit(1);                                                                    \
        }                                                                               \
    } while (0)

/* a block of n bytes, and nothing beside it */
struct Block {
    std::unique_ptr<uint8_t[]> p;
    explicit Block(size_t n) : p(new uint8_t[n ? n : 1]()) {}
    void* at(size_t i = 0) { return p.get() + i; }
};
/* rows x cols with a stride, beginning `shift` elements into its block */
struct Mat {
    Block data, scale;
    tc_matrix m;
    size_t bytes;
    Mat(uint32_t rows, uint32_t cols, int dtype, uint32_t gap = 0, uint32_t shift = 0)
        : data((rows ? (size_t)(rows - 1) * (cols + gap) + cols + shift : 0) * (dtype == TC_I8 ? 1 : 2)), scale(dtype == TC_I8 ? rows * 4ull : 0) {
        const size_t size = dtype == TC_I8 ? 1 : 2;
        bytes = (rows ? (size_t)(rows - 1) * (cols + gap) + cols + shift : 0) * size;
        m = {data.at(shift * size), dtype == TC_I8 ? (float*)scale.at() : nullptr, rows, cols, cols + gap, dtype};
        const size_t some = std::min<size_t>(bytes, 100002);
        for (size_t i = 0; i < some; i += size) {
            if (size == 1) ((int8_t*)data.at())[i] = (int8_t)gen();
            else ((uint16_t*)data.at())[i / 2] = (uint16_t)(0x3800 + gen() % 1024);
        }
        for (size_t i = some; i < bytes; i += some) memcpy(data.at(i), data.at(), std::min(some, bytes - i));
        if (dtype == TC_I8)
            for (uint32_t r = 0; r < rows; ++r) m.d_scale[r] = 0.01f * (1 + gen() % 100);
        if (gap * size >= 16)
            for (uint32_t r = 0; r + 1 < rows; ++r) ASAN_POISON_MEMORY_REGION((uint8_t*)m.d_data + ((size_t)r * m.ld + cols) * size, gap * size);
        if (shift * size >= 8) ASAN_POISON_MEMORY_REGION(data.at(), shift * size / 8 * 8);
    }
    /* outputs: every entry has to be written, where all workgroups were run */
    void clear() {
        for (uint32_t r = 0; r < m.rows; ++r) {
            if (m.dtype == TC_I8) memset((int8_t*)m.d_data + r * m.ld, -128, m.cols);
            else std::fill_n((uint16_t*)m.d_data + r * m.ld, m.cols, 0x7EAD);
        }
    }
    void written(const char* name) const {
        if (lanes::skipped) return;
        for (uint32_t r = 0; r < m.rows; ++r)
            for (uint32_t c = 0; c < m.cols; ++c)
                if (m.dtype == TC_I8 ? ((int8_t*)m.d_data)[r * m.ld + c] == -128 : ((uint16_t*)m.d_data)[r * m.ld + c] == 0x7EAD) {
                    fprintf(stderr, "%s: entry (%u, %u) of %u x %u was not written (%s)\n", name, r, c, m.rows, m.cols, what);
                    exit(1);
                }
    }
    ~Mat() { ASAN_UNPOISON_MEMORY_REGION(data.at(), bytes); }
    const tc_matrix* operator&() const { return &m; }
};
static tc_ctx* const ctx = (tc_ctx*)16;

static void checkpoints_and_norms(uint32_t rows, uint32_t cols, int dtype, uint32_t gap, uint32_t shift) {
    what = "checkpoints and norms";
    Mat x(rows, cols, dtype, gap, shift), y(rows, cols, dtype, gap, shift), q(rows, cols, TC_I8, gap, shift);
    if (rows > 1) ((uint16_t*)x.m.d_data)[x.m.ld] = dtype == TC_F16 ? 0x7C00 : 0x7F80;
    lanes::skipped = false;
    q.clear();
    OK(tc_checkpoint_encode(ctx, &x, &q));
    q.written("checkpoint");
    y.clear();
    OK(tc_checkpoint_decode(ctx, &q, &y));
    y.written("decoded");
    if (cols > TC_NORM_MAX_COLS) return;
    Block gamma(2 * cols), beta(2 * cols), mean(4 * rows), rstd(4 * rows), dgamma(4 * cols), dbeta(4 * cols);
    memset(gamma.at(), 0, 2 * cols);
    memset(beta.at(), 0, 2 * cols);
    size_t need;
    OK(tc_norm_backward_workspace(rows, cols, &need));
    need = std::max<size_t>(need, 16);
    Block work(need);
    for (int kind = 0; kind < 2; ++kind)
        for (const tc_matrix* in : {&x, &q}) {
            lanes::skipped = false;
            y.clear();
            OK(tc_norm(ctx, kind, in, gamma.at(), kind ? nullptr : beta.at(), 1e-5f, &y, (float*)mean.at(), (float*)rstd.at()));
            y.written("norm");
            y.clear();
            OK(tc_norm_backward(ctx, kind, &x, in, kind ? nullptr : gamma.at(), (float*)mean.at(), (float*)rstd.at(), &y, (float*)dgamma.at(), (float*)dbeta.at(), work.at(), need));
            y.written("norm gradient");
        }
    OK(tc_norm_backward(ctx, 1, &x, &x, nullptr, nullptr, (float*)rstd.at(), nullptr, nullptr, (float*)dbeta.at(), work.at(), need));
}
static void products(uint32_t rows, uint32_t in, uint32_t out, int dtype, bool eight, uint32_t gap, uint32_t shift, int act, bool poor) {
    what = "products";
    Mat x(rows, in, dtype, gap, shift), w(out, in, eight ? TC_I8 : dtype, gap, shift), y(rows, out, dtype, gap, shift), z(rows, out, dtype, gap, shift), res(rows, out, dtype, gap, shift);
    Block bias(2 * out);
    memset(bias.at(), 0, 2 * out);
    size_t need;
    OK(tc_linear_workspace(rows, in, out, &need));
    if (poor) need = 0;
    {
        Block work(need);
        lanes::skipped = false;
        y.clear();
        z.clear();
        OK(tc_linear(ctx, &x, &w, bias.at(), act, &res, &y, &z, need ? work.at() : nullptr, need));
        y.written("y");
        z.written("z");
        OK(tc_linear(ctx, &x, &w, nullptr, act, nullptr, &y, nullptr, need ? work.at() : nullptr, need));
    }
    Mat x8(rows, in, TC_I8, gap, shift), z8(rows, out, TC_I8, gap, shift), dz(rows, out, dtype, gap, shift), dx(rows, in, dtype, gap, shift), dw(out, in, dtype, gap, shift);
    Block dbias(4 * out);
    OK(tc_linear_backward_workspace(rows, poor ? 1 : in, out, &need));
    Block work(need);
    const bool bent = act != TC_ACT_NONE;
    lanes::skipped = false;
    dx.clear();
    dw.clear();
    dz.clear();
    OK(tc_linear_backward(ctx, &y, eight ? &x8 : &x, &w, act, bent ? (eight ? &z8 : &z) : nullptr, bent ? &dz : nullptr, &dx, &dw, (float*)dbias.at(), work.at(), need));
    dx.written("dx");
    dw.written("dw");
    if (bent) dz.written("dz");
    OK(tc_linear_backward(ctx, &y, nullptr, nullptr, act, bent ? &z : nullptr, bent ? &dz : nullptr, nullptr, nullptr, (float*)dbias.at(), work.at(), need));
}

/* every place of a tile against the operand, for all tiles of a row of tiles and each way of reading them */
template <class T, bool ALONG, bool EIGHT, int LOOSE, int SIDE, int TH, int BK>
static void feed(uint32_t sides, uint32_t nr, uint32_t r0, uint32_t left_over, uint32_t gap) {
    typedef Feed<T, ALONG, EIGHT, LOOSE, SIDE, TH, BK> F;
    what = "tiles";
    const int dtype = EIGHT ? TC_I8 : std::is_same<T, _Float16>::value ? TC_F16 : TC_BF16;
    const uint32_t all = r0 + nr + left_over;                /* of the sum; this part has r0 .. r0 + nr */
    Mat m(ALONG ? sides : all, ALONG ? all : sides, dtype, gap, LOOSE ? 1 : 0);
    Block powers(2 * (size_t)all);
    for (uint32_t i = 0; i < all; ++i) ((uint16_t*)powers.at())[i] = (uint16_t)((15 + i % 5) << 10);
    const Operand o{m.m.d_data, m.m.ld};
    std::vector<F> f(TH);
    struct Pieces { typename F::Held v; };
    std::vector<Pieces> held(TH);
    std::vector<T> tile(SIDE * BK);
    const uint32_t last = (sides - 1) / SIDE * SIDE;
    for (uint32_t side0 : {0u, last}) {
        for (int t = 0; t < TH; ++t) f[t].init(o, side0, sides, r0, nr, t, F::POWERS ? (const uint16_t*)powers.at() : nullptr);
        for (uint32_t k = 0; k <= (nr + BK - 1) / BK + 1; ++k) {
            memset(tile.data(), 0xFF, sizeof(T) * tile.size());
            for (int t = 0; t < TH; ++t) {
                threadIdx = dim3(t, 0);
                f[t].issue(tile.data(), held[t].v, k, t);
            }
            for (int t = 0; t < TH; ++t) {
                threadIdx = dim3(t, 0);
                f[t].settle(tile.data(), held[t].v, t);
            }
            for (uint32_t side = 0; side < SIDE; ++side)
                for (uint32_t i = 0; i < BK; ++i) {
                    const uint32_t r = k * BK + i, line = ALONG ? side : i, along = ALONG ? i : side;
                    const bool in = side0 + side < sides && r < nr;
                    if (LOOSE && side0 + side >= sides) continue;        /* results that are dropped */
                    double want = 0;
                    if (in) {
                        const size_t at = ALONG ? (size_t)(side0 + side) * m.m.ld + r0 + r : (size_t)(r0 + r) * m.m.ld + side0 + side;
                        want = EIGHT ? (double)((int8_t*)m.m.d_data)[at] : (double)((T*)m.m.d_data)[at];
                        if (F::POWERS) want *= std::ldexp(1.0, (int)((r0 + r) % 5));
                    }
                    const double got = (double)tile[F::tile::place(line, along / 8) + along % 8];
                    if (got != want) {
                        fprintf(stderr, "tile %u from %u: entry (%u, %u) is %g, not %g (along %d eight %d loose %d side %d step %d; %u sides, r %u + %u of %u)\n", k, side0, side, i, got, want, ALONG, EIGHT,
                                LOOSE, SIDE, BK, sides, r0, nr, all);
                        exit(1);
                    }
                }
        }
    }
}
template <class T, bool ALONG, bool EIGHT>
static void feeds() {
    for (uint32_t gap : {0u, 16u})
        for (uint32_t r0 : {0u, 256u}) {
            for (uint32_t nr : {8u, 64u, 72u, 136u}) {
                if (gap) nr += 56;
                for (uint32_t sides : {8u, 64u, 72u, 136u, 264u}) {
                    feed<T, ALONG, EIGHT, 0, 64, 256, 64>(sides, nr, r0, r0 ? 64 : 0, gap);
                    feed<T, ALONG, EIGHT, 0, 128, 256, 64>(sides, nr, r0, r0 ? 64 : 0, gap);
                    if constexpr (!EIGHT) feed<T, ALONG, false, 0, 256, 512, 32>(sides, nr, r0, r0 ? 64 : 0, gap);
                }
            }
            for (uint32_t nr : {1u, 7u, 9u, 65u, 131u})
                for (uint32_t sides : {1u, 5u, 8u, 65u, 71u, 127u, 130u, 257u}) {
                    const bool pieces = (ALONG ? r0 + nr : sides) >= 8;
                    if (pieces) feed<T, ALONG, EIGHT, 1, 64, 256, 64>(sides, nr, r0, 0, gap);
                    if (pieces) feed<T, ALONG, EIGHT, 1, 128, 256, 64>(sides, nr, r0, r0 ? 3 : 0, gap);
                    feed<T, ALONG, EIGHT, 2, 64, 256, 64>(sides, nr, r0, r0 ? 2 : 0, gap);
                }
        }
}

int main() {
    feeds<_Float16, true, false>();
    feeds<_Float16, false, false>();
    feeds<_Float16, true, true>();
    feeds<_Float16, false, true>();
    feeds<__bf16, true, true>();
    feeds<__bf16, false, true>();
    puts("tiles");
    const uint32_t row_sizes[][2] = {{1, 1}, {3, 7}, {5, 8}, {9, 9}, {4, 512}, {5, 513}, {3, 520}, {700, 515}, {1030, 7}, {1030, 511}, {2, 2048}, {3, 2049}, {1027, 2047}, {7, 4096}, {3, 4101}, {1025, 4099}, {2, 8192},
                                     {3, 8199}, {2, 16384}, {3, 16385}, {2, 16390}, {2, 32768}, {3, 32767}, {2, 40001}};
    for (auto& s : row_sizes)
        for (uint32_t shift : {0u, 1u, 8u})
            checkpoints_and_norms(s[0], s[1], (s[0] + shift) % 2 ? TC_F16 : TC_BF16, shift * 2, shift);
    puts("rows");
    lanes::most_blocks = 24;
    const uint32_t sizes[][3] = {{1, 1, 1}, {1, 64, 128}, {2, 65, 7}, {3, 63, 130}, {8, 80, 40}, {9, 16, 24}, {16, 512, 96}, {17, 72, 129}, {16, 8, 264}, {65, 1027, 33}, {129, 640, 264}, {5, 5, 300},
                                 {9, 24, 515}, {5, 1025, 1030}, {70, 129, 513}, {3, 9, 1031}, {300, 328, 392}, {200, 200, 4104}, {300, 4104, 520}, {487, 1032, 1096}, {1100, 2056, 520}};
    for (auto& s : sizes)
        for (uint32_t shift : {0u, 1u, 8u})
            for (int eight = 0; eight < 2; ++eight)
                products(s[0], s[1], s[2], eight || (s[0] + shift) % 2 ? TC_F16 : TC_BF16, eight, shift * 2, shift, (s[0] + shift + eight) % 4, shift == 8);
    puts("products");
    lanes::most_blocks = 2;
    const uint32_t large[][3] = {{8200, 136, 8456}, {8456, 520, 8200}, {520, 8200, 8456}, {4104, 1040, 1040}, {4100, 1043, 2049}};
    for (auto& s : large)
        for (int eight = 0; eight < 2; ++eight) products(s[0], s[1], s[2], eight ? TC_F16 : TC_BF16, eight, 0, 0, eight ? 0 : 2, s[0] == 4104);
    puts("layers lanes: ok");
    return 0;
}
