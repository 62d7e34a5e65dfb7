// Host-code exercise of the group norm, the feed-forward block and the 8-bit projection of include/paraanya_ops.h
// against the host-sanitized copy of the library, without a GPU: workspace queries over sizes that take every part
// of the plans, calls that have nothing to do, and refusals (nothing is launched). Any sanitizer report ends the run
// with a non-zero status. The last line is "block_ops_driver ok".
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "paraanya_ops.h"

#define EXPECT(cond)                                                                                   \
    do {                                                                                               \
        if (!(cond)) {                                                                                 \
            fprintf(stderr, "%s:%d: expectation failed: %s (last error: %s)\n", __FILE__, __LINE__, #cond, \
                    paraanya_last_error());                                                            \
            exit(1);                                                                                   \
        }                                                                                              \
    } while (0)

int main() {
    void* const some = (void*)(uintptr_t)4096;       // never dereferenced
    float* const numbers = (float*)some;
    size_t n = 1;
    for (int64_t batch : {0, 1, 32, 65535})
        for (int64_t pixels : {0, 1, 1000, 70001, 1 << 30})
            for (int channels : {1, 7, 320, 4096, 1 << 20})
                for (int groups : {1, 7, 32, 4096, 1 << 20}) {
                    if (channels % groups != 0) continue;
                    for (int dtype : {PA_F32, PA_BF16}) {
                        pa_group_norm_t p = {batch, pixels, channels, groups, dtype, PA_F32, PA_ACT_SILU, 0, 1e-5, {}, {}, {}};
                        int64_t strides[2] = {pixels * channels, channels};
                        if (strides[0] > (1ll << 40)) continue;
                        for (int i = 0; i < 2; ++i) p.x_stride[i] = p.y_stride[i] = p.dx_stride[i] = strides[i];
                        const int want = channels / groups > PA_GROUP_MAX_CHANNELS ? PA_ERR_UNSUPPORTED : PA_OK;
                        n = 1;
                        EXPECT(paraanya_group_norm_workspace(&p, &n) == want && (want != PA_OK || n % 256 == 0));
                        if (want == PA_OK && batch > 0 && pixels > 0 && n > 0)
                            EXPECT(paraanya_group_norm(&p, some, some, some, some, numbers, numbers, some, n - 1, nullptr) == PA_ERR_INVALID_ARG);
                        n = 1;
                        EXPECT(paraanya_group_norm_backward_workspace(&p, &n) == want && (want != PA_OK || n % 256 == 0));
                        if (want == PA_OK && n > 0)
                            EXPECT(paraanya_group_norm_backward(&p, some, some, some, some, numbers, numbers, some, some, some, some, n - 1,
                                                                nullptr) == PA_ERR_INVALID_ARG);
                    }
                }
    pa_group_norm_t g = {2, 0, 8, 2, PA_F32, PA_F32, PA_ACT_NONE, 0, 1e-5, {0, 8}, {0, 8}, {0, 8}};
    EXPECT(paraanya_group_norm(&g, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == PA_OK);
    g.eps = NAN;
    EXPECT(paraanya_group_norm_workspace(&g, &n) == PA_ERR_INVALID_ARG);
    EXPECT(paraanya_group_norm_workspace(nullptr, &n) == PA_ERR_INVALID_ARG);
    puts("group norm ok");

    for (int64_t rows : {0, 1, 64, 65, 8192, 1 << 20})
        for (int in : {1, 64, 1100, 2048})
            for (int hidden : {1, 96, 2731, 8192})
                for (int dtype : {PA_BF16, PA_F16})
                    for (int alignment : {2, 16}) {
                        pa_feed_t p = {rows, in, hidden, 40, dtype, PA_ACT_GELU, alignment, in, in, in, hidden, 40};
                        size_t saved = 1, back = 1;
                        EXPECT(paraanya_feed_forward_saved(&p, &saved) == PA_OK && saved % 256 == 0);
                        EXPECT(paraanya_feed_forward_backward_workspace(&p, &back) == PA_OK && back % 256 == 0);
                        pa_feed_grad_t d = {some, some, some, some, some, some, some};
                        for (int with : {0, 1}) {
                            EXPECT(paraanya_feed_forward_workspace(&p, with, &n) == PA_OK && n % 256 == 0);
                            if (rows > 0 && n > 0)
                                EXPECT(paraanya_feed_forward(&p, some, some, some, some, some, some, some, some, with ? some : nullptr, saved,
                                                             some, n - 1, nullptr) == PA_ERR_INVALID_ARG);
                        }
                        if (rows > 0)
                            EXPECT(paraanya_feed_forward_backward(&p, &d, some, some, some, some, some, some, saved, some, back - 1, nullptr) ==
                                   PA_ERR_INVALID_ARG);
                    }
    puts("feed-forward block ok");

    pa_quantize_t q = {0, 100, PA_F16, 0, 100, 112};
    EXPECT(paraanya_quantize_rows(&q, nullptr, nullptr, nullptr, nullptr) == PA_OK);
    q.q_stride = 100;
    EXPECT(paraanya_quantize_rows(&q, nullptr, nullptr, nullptr, nullptr) == PA_ERR_INVALID_ARG);
    pa_int8_linear_t l = {0, 100, 32, PA_F16, 0, 112, 112, 32};
    EXPECT(paraanya_int8_linear(&l, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == PA_OK);
    l.rows = 4;
    EXPECT(paraanya_int8_linear(&l, (int8_t*)some, numbers, (int8_t*)some, numbers, nullptr, (void*)(uintptr_t)4097, nullptr) == PA_ERR_INVALID_ARG);
    puts("8-bit projection ok");
    puts("block_ops_driver ok");
    return 0;
}
