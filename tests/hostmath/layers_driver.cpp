// The planning of the layer operators' products on the CPU: which layout a call takes in which workspace, and that everything it puts
// there fits.  Built and run by tests/test_layers_plans.py under AddressSanitizer and UBSan.
#include "../../paper_2602_12630_amd/csrc/tc_layers.cpp"

#include <cstdio>
#include <random>

namespace tc {  // what tc_lib.cpp has; no call is made here
rt::stream_t ctx_stream(const tc_ctx*) { return {}; }
int ctx_device(const tc_ctx*) { return 0; }
int ctx_use_device(tc_ctx*) { return TC_OK; }
int ctx_fail(tc_ctx*, int code, const char*) { return code; }
int ctx_fail_hip(tc_ctx*, int, const char*) { return TC_ERR_HIP; }
}  // namespace tc

#define REQUIRE(cond)                                                                                                       \
    do {                                                                                                                    \
        if (!(cond)) {                                                                                                      \
            std::fprintf(stderr, "%s:%d: %s does not hold (%u %u %u, %zu bytes)\n", __FILE__, __LINE__, #cond, np, nq, nr, room); \
            return 1;                                                                                                       \
        }                                                                                                                   \
    } while (0)

static bool same(const Layout& a, const Layout& b) { return a.np == b.np && a.nq == b.nq && a.side == b.side && a.splits == b.splits && a.r_split == b.r_split; }
static bool same(const ProductPlan& a, const ProductPlan& b) {
    return same(a.whole, b.whole) && a.cut == b.cut && (!a.cut || (a.cut_p == b.cut_p && same(a.first, b.first) && same(a.rest, b.rest)));
}
/* one launch: every part has some of r, and the parts lie in the workspace */
static int check_layout(const Layout& l, uint32_t np, uint32_t nq, uint32_t nr, size_t room) {
    REQUIRE(l.np == np && l.nq == nq && l.ldp >= np && l.ldp % 8 == 0);
    REQUIRE(l.splits >= 1 && (uint64_t)(l.splits - 1) * l.r_split < nr && (uint64_t)l.splits * l.r_split >= nr);
    REQUIRE(l.splits == 1 || (l.r_split % 64 == 0 && l.r_split >= 256));
    REQUIRE(l.part_bytes() <= room);
    return 0;
}
static int check_plan(uint32_t np, uint32_t nq, uint32_t nr, size_t room, bool eight) {
    const ProductPlan most = product_plan(np, nq, nr), p = product_plan_in(np, nq, nr, room, eight);
    if (room >= most.bytes(nr)) REQUIRE(same(p, most));
    if (check_layout(p.whole, np, nq, nr, room)) return 1;
    if (eight) REQUIRE(p.whole.side != 256 || p.bytes(nr) <= room);
    REQUIRE(p.part_bytes() <= room);
    if (p.cut) {
        REQUIRE(p.whole.side == 256 && p.first.side == 256 && p.first.splits == 1 && p.cut % 256 == 0 && p.cut < (p.cut_p ? np : nq));
        if (check_layout(p.first, p.cut_p ? p.cut : np, p.cut_p ? nq : p.cut, nr, room)) return 1;
        if (check_layout(p.rest, p.cut_p ? np - p.cut : np, p.cut_p ? nq : nq - p.cut, nr, room)) return 1;
    }
    return 0;
}
/* calls of r rows in the workspace of `rows` */
static int check_sizes(uint32_t rows, uint32_t r, uint32_t in, uint32_t out) {
    const uint32_t np = in, nq = out, nr = r;
    size_t room = 0, need = 0;
    REQUIRE(tc_linear_workspace(rows, in, out, &room) == TC_OK);
    for (int eight = 0; eight < 2; ++eight)
        if (check_plan(out, r, in, room, eight)) return 1;
    REQUIRE(tc_linear_backward_workspace(rows, in, out, &room) == TC_OK);
    for (uint32_t width : {0u, in}) {
        const BackPlan b = back_plan(r, width, out);
        REQUIRE(b.split <= room && b.by_w == up((size_t)r * b.ld_by * 2, 256) && b.part == 2 * b.by_w && b.m >= b.part + (size_t)slope_groups(r, out) * out * 4);
        REQUIRE(b.powers_x >= b.m + 16 && b.powers_w >= b.powers_x + 2 * (size_t)r && b.split >= b.powers_w + 2 * (size_t)out && b.split % 16 == 0);
        for (int eight = 0; eight < 2; ++eight)
            if (check_plan(in, r, out, room - b.split, eight) || check_plan(in, out, r, room - b.split, eight)) return 1;
    }
    if (in <= TC_NORM_MAX_COLS) {
        REQUIRE(tc_norm_backward_workspace(rows, in, &room) == TC_OK && tc_norm_backward_workspace(r, in, &need) == TC_OK);
        REQUIRE(need <= room && (size_t)norm_back_groups(r, in) * 2 * in * 4 <= need);
    }
    return 0;
}

int main() {
    std::mt19937_64 gen(1);
    auto any = [&](double most) { return (uint32_t)std::exp(std::uniform_real_distribution<>(0, std::log(most))(gen)); };
    const uint32_t widths[] = {1, 8, 64, 512, 1024, 4096, 11008};
    for (uint32_t in : widths)
        for (uint32_t out : widths)
            for (uint32_t rows : {1u, 1023u, 1024u, 1025u, 4096u, 8192u, 16384u, 65536u})
                for (uint32_t r = rows; r; r = r > 4096 ? r - 293 : r > 64 ? r - 61 : r - 1)
                    if (check_sizes(rows, r, in, out)) return 1;
    for (int i = 0; i < 200000; ++i) {
        const uint32_t rows = any(i % 10 ? 1e5 : 2147483647.0);
        if (check_sizes(rows, std::min(rows, any(rows + 1.0)), any(i % 4 ? 2e4 : 1048576.0), any(i % 4 ? 2e4 : 1048576.0))) return 1;
    }
    std::puts("layers driver: ok");
    return 0;
}
