// Host-side exercise of the 4-bit products, layer norm and dropout for the sanitizer build: sizes of workspaces over many
// shapes, the plans, and refusals. Nothing here launches a kernel.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "../../include/rtopk.h"
#include "../../include/rtopk_diag.h"

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
            if (n) {
                EXPECT(rtopk_layer_norm_backward_workspace_bytes(m, n, &bytes) == RTOPK_OK && bytes % 256 == 0);
                EXPECT((m <= 2048 && m * n <= 1u << 21) == (bytes == 0));
                sum += bytes;
            }
            for (uint64_t k : sizes) {
                EXPECT(rtopk_matmul_mx4_workspace_bytes(m, n, k, &bytes) == RTOPK_OK && bytes % 256 == 0);
                sum += bytes;
                if (m && n) {
                    for (int on_lines : {0, 1}) {
                        rtopk_product_plan_t p;
                        EXPECT(rtopk_product_mx4_plan(m, n, k, on_lines, &p) == RTOPK_OK && p.tiles >= 1 && p.runs >= 1);
                        EXPECT(p.runs == 1 || bytes >= 4 * m * n * p.runs);
                    }
                }
                if (!n || !k) continue;
                EXPECT(rtopk_linear_mx4_workspace_bytes(m, k, n, &bytes) == RTOPK_OK);
                EXPECT(m <= 16 || bytes >= m * ((k + 1) / 2 + (k + 31) / 32));
                sum += bytes;
                EXPECT(rtopk_linear_mx4_backward_workspace_bytes(m, k, n, &bytes) == RTOPK_OK);
                EXPECT(bytes >= m * (2 * n + k) / 2);
                sum += bytes;
            }
        }
    EXPECT(rtopk_matmul_mx4_workspace_bytes(5, UINT64_MAX, 5, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_matmul_mx4_workspace_bytes(5, 5, 5, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_linear_mx4_workspace_bytes(5, UINT64_MAX, 5, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_linear_mx4_backward_workspace_bytes(UINT64_MAX, 5, 5, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_layer_norm_backward_workspace_bytes(UINT64_MAX, 5, &bytes) == RTOPK_EINVAL);
    EXPECT(rtopk_layer_norm_backward_workspace_bytes(5, 5, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_product_mx4_plan(5, 5, 5, 0, nullptr) == RTOPK_EINVAL);

    float x[64] = {}, y[64] = {};
    uint8_t q[64] = {}, s[64] = {};
    void *ws = reinterpret_cast<void *>(0x1000);
    EXPECT(rtopk_quantize_mx4(x, 0, UINT64_MAX, 8, 8, 0, 0, 1, 2, nullptr, q, 4, s, 8, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_mx4(x, 0, 8, 8, UINT64_MAX, 0, 0, 1, 2, nullptr, q, 4, s, 8, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_mx4(x, 0, 8, 8, 8, 0, 0, 1, 2, nullptr, q, 3, s, 8, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_mx4(x, 0, 8, 8, 8, 0, 0, 1, 2, nullptr, q, 4, s, 7, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_mx4(x, 0, 8, 8, 8, 1, 2, 1, 2, nullptr, q, 4, s, 8, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_quantize_mx4(nullptr, 0, 0, 8, 8, 0, 0, 1, 2, nullptr, nullptr, 4, nullptr, 0, nullptr) == RTOPK_OK);
    EXPECT(rtopk_dequantize_mx4(q, 8, UINT64_MAX, 4, s, 8, y, 0, 8, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_dequantize_mx4(nullptr, 0, 8, 4, nullptr, 0, nullptr, 0, 8, nullptr) == RTOPK_OK);
    EXPECT(rtopk_matmul_mx4(q, s, q, s, nullptr, 8, 8, 8, 4, 8, 4, 7, y, 0, 8, nullptr, 0, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_matmul_mx4(nullptr, nullptr, nullptr, nullptr, nullptr, 0, 8, 8, 4, 8, 4, 8, nullptr, 0, 8, nullptr, 0, nullptr) == RTOPK_OK);
    EXPECT(rtopk_linear_mx4(x, 0, 500, 900, 900, q, s, 700, 450, 700, nullptr, y, 0, 700, nullptr, 0, nullptr) == RTOPK_EWORKSPACE);
    EXPECT(rtopk_linear_mx4_backward(x, x, 0, 4, 8, 6, 6, 8, q, s, 3, 8, 0, 1, 2, nullptr, y, 8, y, 8, y, ws, 8, nullptr) == RTOPK_EWORKSPACE);
    EXPECT(rtopk_layer_norm(x, 0, 4, 8, 8, nullptr, nullptr, NAN, y, 0, 8, nullptr, nullptr, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_layer_norm(x, 0, 4, 8, 8, nullptr, nullptr, 1e-5f, y, 0, UINT64_MAX, nullptr, nullptr, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_layer_norm_backward(x, 0, x, 0, 5000, 8, 8, 8, x, x, nullptr, nullptr, 0, nullptr, 0, y, nullptr, ws, 8, nullptr) ==
           RTOPK_EWORKSPACE);
    EXPECT(rtopk_layer_norm_backward(x, 0, x, 0, 5000, 8, 8, 8, x, x, nullptr, nullptr, 0, nullptr, 0, nullptr, nullptr, ws, 8, nullptr) ==
           RTOPK_EINVAL);
    for (double p : {-1.0, 2.0, (double)NAN, (double)INFINITY, -(double)INFINITY})
        EXPECT(rtopk_dropout(x, 0, 4, 8, 8, nullptr, 0, y, 0, 8, p, 1, 2, nullptr, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_dropout(x, 0, UINT64_MAX, UINT64_MAX, UINT64_MAX, nullptr, 0, y, 0, UINT64_MAX, 0.5, 1, 2, nullptr, nullptr) == RTOPK_EINVAL);
    EXPECT(rtopk_dropout(nullptr, 0, 0, 8, 8, nullptr, 0, nullptr, 0, 8, 0.5, 1, 2, nullptr, nullptr) == RTOPK_OK);
    std::printf("sum %llu, %d failures\n", (unsigned long long)sum, failures);
    return failures != 0;
}
