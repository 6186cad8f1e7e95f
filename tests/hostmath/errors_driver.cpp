// Refused calls while the host has no memory left for their message: the code comes back, nothing is thrown across the C boundary.
// Built from the host build's sources and run by tests/test_host_errors.py.
#include "../../include/tc.h"

#include <cstdio>
#include <cstdlib>
#include <new>

static bool full = false;
void* operator new(size_t n) {
    void* p = full ? nullptr : std::malloc(n);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

#define REQUIRE(cond)                                                                     \
    do {                                                                                  \
        if (!(cond)) {                                                                    \
            std::fprintf(stderr, "%s:%d: %s does not hold\n", __FILE__, __LINE__, #cond); \
            return 1;                                                                     \
        }                                                                                 \
    } while (0)

int main() {
    tc_ctx* ctx = nullptr;
    REQUIRE(tc_ctx_create(&ctx, 0, nullptr) == TC_OK);
    uint16_t data[8] = {};
    tc_matrix m = {data, nullptr, 1, 8, 8, TC_F16};
    full = true;
    REQUIRE(tc_norm(ctx, 7, &m, nullptr, nullptr, 1e-5f, &m, nullptr, nullptr) == TC_ERR_ARG);
    REQUIRE(tc_checkpoint_encode(ctx, &m, &m) == TC_ERR_ARG);
    REQUIRE(tc_linear(ctx, &m, &m, nullptr, 9, nullptr, &m, nullptr, nullptr, 0) == TC_ERR_ARG);
    REQUIRE(tc_linear_backward(ctx, &m, nullptr, nullptr, 0, &m, nullptr, nullptr, nullptr, nullptr, nullptr, 0) == TC_ERR_ARG);
    REQUIRE(tc_encode_tensor(ctx, data, TC_BF16, 8, 1.0f, data) == TC_ERR_ARG);
    full = false;
    REQUIRE(tc_last_error(ctx) != nullptr);
    tc_ctx_destroy(ctx);
    std::puts("errors driver: ok");
    return 0;
}
