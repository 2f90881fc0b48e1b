// Host-side logic of the operators around the tiled layers under AddressSanitizer + UndefinedBehaviorSanitizer (CPU only).
// Built by tests/test_step_abi_host.py; every call is sizing, or is stopped by the validation one byte short of its workspace.
#include <stdint.h>
#include <stdio.h>
#include <vector>

#include "alst_block_norm.h"
#include "alst_embedding.h"
#include "alst_grads.h"

static int failures = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) {                                                      \
            ++failures;                                                     \
            fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #cond);      \
        }                                                                   \
    } while (0)

static void* fake(uintptr_t a) { return reinterpret_cast<void*>(a); }

int main() {
    long calls = 0;
    for (int64_t N : {(int64_t)1, (int64_t)31, (int64_t)33, (int64_t)4097, (int64_t)131072, ((int64_t)1 << 30) - 1, (int64_t)1 << 30})
        for (int64_t H : {(int64_t)8, (int64_t)512, (int64_t)520, (int64_t)1600, (int64_t)16384, (int64_t)16392, (int64_t)1 << 20}) {
            for (int64_t V : {(int64_t)1, (int64_t)2, (int64_t)511, (int64_t)128256, (int64_t)1 << 18, (int64_t)1 << 24}) {
                const size_t w = alst_embedding_workspace_bytes(N, H, V);
                EXPECT(w > (size_t)N * 16);
                EXPECT(alst_embedding_backward(static_cast<const int32_t*>(fake(0x1000)), fake(0x2000), N, H, V, -100, 1.f, fake(0x3000),
                                               fake(0x4000), w - 1, 0, nullptr) == ALST_ERR_WORKSPACE);
                ++calls;
            }
            const size_t w = alst_block_norm_workspace_bytes(N, H);
            EXPECT((w > 0) == (H <= 16384));
            const int rc = alst_block_norm_backward(fake(0x1000), fake(0x2000), fake(0x3000), nullptr, 0, fake(0x4000), fake(0x5000),
                                                    nullptr, N, H, 1.f, 1e-6f, 0.f, fake(0x6000), fake(0x7000), nullptr, fake(0x8000),
                                                    fake(0x9000), fake(0xa000), w - 1, 0, nullptr);
            EXPECT(rc == (w ? ALST_ERR_WORKSPACE : ALST_ERR_SHAPE));
            ++calls;
        }
    for (int64_t count : {(int64_t)1, (int64_t)63, (int64_t)64, (int64_t)65, (int64_t)1000}) {
        std::vector<alst_grad_tensor> ts;
        for (int64_t i = 0; i < count; ++i)
            ts.push_back({fake(0x1000 + 4 * i), fake(0x1000 + 4 * i), i % 7 ? (int64_t)1 << (i % 35) : 0, (int32_t)(i & 1), 0});
        const size_t w = alst_grad_norm_workspace_bytes(count);
        EXPECT(alst_grad_norm_clip(ts.data(), count, 1.f, nullptr, nullptr, fake(0x4000), w - 1, nullptr) == ALST_ERR_WORKSPACE);
        ts.back().n = (int64_t)1 << 40;
        ts.back().fp32 = 1;
        ts.back().grad = ts.back().out = fake(0x1002);
        EXPECT(alst_grad_norm_clip(ts.data(), count, 1.f, nullptr, nullptr, fake(0x4000), w, nullptr) == ALST_ERR_ALIGN);
        calls += 2;
    }
    printf("step_sanitize: %ld calls, %d failures\n", calls, failures);
    return failures ? 1 : 0;
}
