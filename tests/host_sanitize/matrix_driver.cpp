// Host-side exercise of the matrix entry points for the sanitizer build: the sizes of workspaces over many shapes (the
// layouts, the cost model that picks tiles and runs, the plan of the steps are all computed on the host) and every
// refusal. Nothing here launches a kernel.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "../../include/rtopk.h"

static int failures = 0;
#define EXPECT(cond)                                                         \
    do {                                                                     \
        if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++failures; } \
    } while (0)

int main()
{
    uint64_t bytes = 0, sum = 0;
    const uint64_t sizes[] = {0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 1500, 4096, 10007, 65536, 1u << 21, 1u << 22};
    for (uint64_t m : sizes)
        for (uint64_t n : sizes) {
            for (int along : {RTOPK_ROWS, RTOPK_COLUMNS})
                if (n) {
                    EXPECT(rtopk_quantize_i8_workspace_bytes(m, n, along, &bytes) == RTOPK_OK);
                    sum += bytes;
                }
            for (uint64_t k : sizes) {
                EXPECT(rtopk_matmul_i8_workspace_bytes(m, n, k, &bytes) == RTOPK_OK);
                EXPECT(bytes % 256 == 0);
                sum += bytes;
                if (!n || !k) continue;
                EXPECT(rtopk_linear_i8_workspace_bytes(m, k, n, &bytes) == RTOPK_OK);
                EXPECT(m <= 64 || bytes >= m * k);       // (fewer tokens may need none)
                sum += bytes;
                EXPECT(rtopk_linear_i8_backward_workspace_bytes(m, k, n, &bytes) == RTOPK_OK);
                EXPECT(bytes >= m * (n + k));
                sum += bytes;
            }
            if (!m || !n) continue;
            for (uint32_t count : {1u, 2u, 3u, 15u, 16u, 17u, 33u, 1000u})
                for (int products : {RTOPK_PRODUCTS_PAIRS, RTOPK_PRODUCTS_HALVES}) {
                    const bool fits = m <= 1u << 21 && n <= 1u << 21 && m * n < 1ull << 32;
                    uint64_t more = 0;
                    const int rc = rtopk_orthogonalize_workspace_bytes(count, m, n, products, &bytes);
                    EXPECT(rc == (fits ? RTOPK_OK : RTOPK_EINVAL));
                    EXPECT(rtopk_aggregate_update_orthogonal_workspace_bytes(count, m, n, products, &more) == rc);
                    if (fits) {
                        EXPECT(more >= bytes + 4 * m * n);
                        uint64_t turned = 0;
                        EXPECT(rtopk_orthogonalize_workspace_bytes(count, n, m, products, &turned) == RTOPK_OK && turned == bytes);
                        sum += bytes + more;
                    }
                }
        }
    EXPECT(rtopk_quantize_i8_workspace_bytes(UINT64_MAX, 5, RTOPK_ROWS, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_i8_workspace_bytes(5, UINT64_MAX, RTOPK_COLUMNS, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_i8_workspace_bytes(5, 5, 7, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_i8_workspace_bytes(5, 5, RTOPK_ROWS, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_matmul_i8_workspace_bytes(5, UINT64_MAX, 5, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_matmul_i8_workspace_bytes(5, 5, 5, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_linear_i8_workspace_bytes(5, 5, (1u << 22) + 1, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_linear_i8_workspace_bytes(5, 5, 5, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_linear_i8_backward_workspace_bytes(5, UINT64_MAX, 5, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_linear_i8_backward_workspace_bytes(5, 5, 5, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_orthogonalize_workspace_bytes(1, UINT64_MAX, UINT64_MAX, RTOPK_PRODUCTS_PAIRS, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_orthogonalize_workspace_bytes(0, 5, 5, RTOPK_PRODUCTS_PAIRS, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_orthogonalize_workspace_bytes(1, 5, 5, 2, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_orthogonalize_workspace_bytes(1, 5, 5, RTOPK_PRODUCTS_PAIRS, nullptr) == RTOPK_EINVAL);

    // the addresses of refused calls are never looked at
    void *p = (void *)0x1000, *q = (void *)0x40000000, *ws = (void *)0x80000000;
    float *scale = (float *)0x20000000;
    const uint64_t room = 1ull << 40;
    EXPECT(rtopk_quantize_i8(p, 9, 4, 8, 8, RTOPK_ROWS, (int8_t *)q, 8, scale, ws, room, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_i8(p, RTOPK_F32, 4, 8, 8, RTOPK_COLUMNS, (int8_t *)q, 4, scale, ws, 16, nullptr) == RTOPK_EWORKSPACE);
    EXPECT(rtopk_quantize_i8(p, RTOPK_F32, 4, 8, UINT64_MAX, RTOPK_ROWS, (int8_t *)q, 8, scale, ws, room, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_matmul_i8((int8_t *)p, scale, (int8_t *)q, scale, nullptr, 4, 4, UINT64_MAX, 16, 16, p, RTOPK_F32, 4, ws, room, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_linear_i8(p, RTOPK_BF16, 4, 8, 7, (int8_t *)q, scale, 4, 8, nullptr, p, RTOPK_BF16, 4, ws, room, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_linear_i8(p, RTOPK_BF16, 400, 800, 800, (int8_t *)q, scale, 400, 800, nullptr, (void *)0x60000000, RTOPK_BF16, 400, ws, 16, nullptr) == RTOPK_EWORKSPACE);
    EXPECT(rtopk_linear_i8_backward(p, p, RTOPK_BF16, 4, 8, 4, 4, 8, nullptr, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, ws, room, nullptr) == RTOPK_EINVAL);
    const void *xs[2] = {p, nullptr};
    void *outs[2] = {q, q};
    const float abc[3] = {3.4445f, -4.7750f, 2.0315f}, wild[3] = {1e30f, 1e30f, NAN};
    EXPECT(rtopk_orthogonalize(2, xs, RTOPK_F32, 8, 8, 8, 1, abc, 1e-7f, RTOPK_PRODUCTS_PAIRS, outs, RTOPK_F32, 8, ws, room, nullptr) == RTOPK_EINVAL);
    xs[1] = p;
    EXPECT(rtopk_orthogonalize(2, xs, RTOPK_F32, 8, 8, 7, 1, abc, 1e-7f, RTOPK_PRODUCTS_PAIRS, outs, RTOPK_F32, 8, ws, room, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_orthogonalize(2, xs, RTOPK_F32, 8, 8, 8, 1, wild, 1e-7f, RTOPK_PRODUCTS_PAIRS, outs, RTOPK_F32, 8, ws, room, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_orthogonalize(2, xs, RTOPK_F32, 8, 8, 8, 1, nullptr, 1e-7f, RTOPK_PRODUCTS_PAIRS, outs, RTOPK_F32, 8, ws, room, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_orthogonalize(2, xs, RTOPK_F32, 8, 8, 8, 1, abc, 1e-7f, RTOPK_PRODUCTS_PAIRS, outs, RTOPK_F32, 8, ws, 16, nullptr) == RTOPK_EWORKSPACE);
    std::printf("sum of sizes %llu, %d failures\n", (unsigned long long)sum, failures);
    return failures != 0;
}
