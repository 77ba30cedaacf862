// The host side of the 4-bit products, layer norm and dropout with the runtime's launch replaced by a check of its shape: every
// launch of calls over many sizes, the largest among them, must be one that the device takes. Nothing runs on a GPU, and no
// pointer that is handed over is followed.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <map>
#include <string>
#include <vector>

#include "../../include/rtopk.h"

namespace {

// (kernels are registered before this file's own objects are made)
std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> all;
    return all;
}
struct Shape {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
};
std::vector<Shape> configured;
const char *call = "";
uint64_t sizes_of_call[3], launches;
int failures;

void expect(bool ok, const char *what, const void *kernel, const Shape &s)
{
    if (ok) return;
    ++failures;
    std::printf("%s(%llu, %llu, %llu): %s, %s: grid %u %u %u, block %u\n", call, (unsigned long long)sizes_of_call[0],
                (unsigned long long)sizes_of_call[1], (unsigned long long)sizes_of_call[2], what, names()[kernel].c_str(), s.grid.x, s.grid.y,
                s.grid.z, s.block.x);
}

}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *) { return nullptr; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *)
{
    names()[host] = name;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream)
{
    configured.push_back({grid, block, lds, stream});
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    const Shape s = configured.back();
    configured.pop_back();
    *grid = s.grid;
    *block = s.block;
    *lds = s.lds;
    *stream = s.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *kernel, dim3 grid, dim3 block, void **, size_t lds, hipStream_t stream)
{
    const Shape s{grid, block, lds, stream};
    ++launches;
    expect(grid.x && grid.y && grid.z, "no workgroups", kernel, s);
    expect((uint64_t)grid.x * block.x < 1ull << 32, "2^32 threads or more along x", kernel, s);
    expect(grid.y < 1u << 16 && grid.z < 1u << 16, "2^16 workgroups or more along y or z", kernel, s);
    expect(block.x <= 1024 && block.y == 1 && block.z == 1, "the workgroup's size", kernel, s);
    expect(lds <= 64 * 1024, "LDS", kernel, s);
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}

int main()
{
    const uint64_t most = 1ull << 22, sizes[] = {1, 3, 40, 64, 65, 700, 1500, 2049, 4096, 8193, 16385, 60'001, 1u << 18, (1u << 20) + 3, most - 64, most - 63, most};
    const uint64_t memory = 288'000'000'000;
    uint8_t *const p = (uint8_t *)0x100000, *const q = (uint8_t *)0x200000;
    float *const f = (float *)0x300000;
    auto expect_ok = [&](int rc) {
        if (rc == RTOPK_OK) return;
        ++failures;
        std::printf("%s(%llu, %llu, %llu) gave %d\n", call, (unsigned long long)sizes_of_call[0], (unsigned long long)sizes_of_call[1],
                    (unsigned long long)sizes_of_call[2], rc);
    };
    auto next = [&](const char *name, uint64_t a, uint64_t b, uint64_t c) {
        call = name;
        sizes_of_call[0] = a;
        sizes_of_call[1] = b;
        sizes_of_call[2] = c;
    };
    for (uint64_t rows : sizes)
        for (uint64_t cols : sizes) {
            if (rows * cols * 2 > memory) continue;
            uint64_t need = 0;
            for (int type : {RTOPK_F32, RTOPK_BF16, RTOPK_F16}) {
                for (int rounding : {RTOPK_NEAREST, RTOPK_DRAWN}) {
                    next("quantize_mx4", rows, cols, rounding);
                    expect_ok(rtopk_quantize_mx4(p, type, rows, cols, cols, RTOPK_ROWS, rounding, 1, 2, nullptr, q, (cols + 1) / 2, q, rows, nullptr));
                    expect_ok(rtopk_quantize_mx4(p, type, rows, cols, cols, RTOPK_COLUMNS, rounding, 1, 2, nullptr, q, (rows + 1) / 2, q, cols, nullptr));
                }
                next("dequantize_mx4", rows, cols, 0);
                expect_ok(rtopk_dequantize_mx4(q, rows, cols, (cols + 1) / 2, q, rows, p, type, cols, nullptr));
                next("layer_norm", rows, cols, 0);
                expect_ok(rtopk_layer_norm(p, type, rows, cols, cols, f, f, 1e-5f, q, type, cols, f, f, nullptr));
                next("layer_norm_backward", rows, cols, 0);
                expect_ok(rtopk_layer_norm_backward_workspace_bytes(rows, cols, &need));
                for (void *dx : {(void *)nullptr, (void *)q, (void *)p})
                    expect_ok(rtopk_layer_norm_backward(p, type, p, type, rows, cols, cols, cols, f, f, f, nullptr, 0, dx, cols, f, f, f, need, nullptr));
                next("dropout", rows, cols, 0);
                for (uint64_t apart : {0, 1})
                    expect_ok(rtopk_dropout(p, type, rows, cols, cols + apart, q, cols, q, type, cols, 0.5, 1, 2, nullptr, nullptr));
            }
            for (uint64_t k : sizes) {
                if (k * (rows + cols) / 2 > memory) continue;
                next("matmul_mx4", rows, cols, k);
                expect_ok(rtopk_matmul_mx4_workspace_bytes(rows, cols, k, &need));
                expect_ok(rtopk_matmul_mx4(p, p, p, p, f, rows, cols, k, (k + 1) / 2, rows, (k + 1) / 2, cols, q, RTOPK_BF16, cols, f, need, nullptr));
                next("linear_mx4", rows, k, cols);
                expect_ok(rtopk_linear_mx4_workspace_bytes(rows, k, cols, &need));
                expect_ok(rtopk_linear_mx4(p, RTOPK_BF16, rows, k, k, p, p, cols, (k + 1) / 2, cols, f, q, RTOPK_BF16, cols, f, need, nullptr));
                if (k * cols * 4 > memory || rows * k * 2 > memory) continue;
                next("linear_mx4_backward", rows, k, cols);
                expect_ok(rtopk_linear_mx4_backward_workspace_bytes(rows, k, cols, &need));
                for (int which = 1; which < 4; ++which)
                    expect_ok(rtopk_linear_mx4_backward(p, p, RTOPK_BF16, rows, k, cols, cols, k, p, p, (cols + 1) / 2, k, RTOPK_DRAWN, 1, 2, nullptr,
                                                        which & 1 ? q : nullptr, k, which & 2 ? (float *)q : nullptr, k, which & 2 ? f : nullptr, f, need,
                                                        nullptr));
            }
        }
    std::printf("%llu launches, %d failures\n", (unsigned long long)launches, failures);
    return failures != 0;
}
