// Host-code exercise of include/paraanya_ops.h against the host-sanitized copy of the library, without a GPU:
// workspace queries over sizes that take every part of the workspaces, calls that have nothing to do, and
// refusals (nothing is launched). Any sanitizer report ends the run with a non-zero status. The last line is
// "ops_driver ok".
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

static pa_cross_t cross(int64_t batch, int64_t q_len, int64_t kv_len, int q_heads, int kv_heads, int dim) {
    pa_cross_t p = {};
    p.batch = batch, p.q_len = q_len, p.kv_len = kv_len, p.q_heads = q_heads, p.kv_heads = kv_heads, p.head_dim = dim;
    p.dtype = PA_BF16, p.scale = 0.125;
    const int64_t q[3] = {q_len * q_heads * dim, (int64_t)q_heads * dim, dim};
    const int64_t k[3] = {kv_len * kv_heads * dim, (int64_t)kv_heads * dim, dim};
    for (int i = 0; i < 3; ++i) p.q_stride[i] = p.o_stride[i] = q[i], p.k_stride[i] = p.v_stride[i] = k[i];
    return p;
}

int main() {
    void* const some = (void*)(uintptr_t)4096;       // never dereferenced
    size_t n = 1;
    for (int64_t q_len : {0, 1, 33, 1000, 2309, 1 << 19})
        for (int64_t kv_len : {0, 1, 77, 1541, 1 << 20})
            for (int heads : {1, 8, 128})
                for (int dim : {1, 40, 128}) {
                    pa_cross_t p = cross(2, q_len, kv_len, heads, heads > 1 ? heads / 4 : 1, dim);
                    n = 1;
                    EXPECT(paraanya_cross_attention_workspace(&p, &n) == PA_OK && n % 256 == 0);
                    n = 1;
                    EXPECT(paraanya_cross_attention_backward_workspace(&p, &n) == PA_OK && n % 256 == 0);
                    if (q_len > 0 && kv_len > 0 && n > 0) {
                        pa_cross_grad_t g = {};
                        for (int i = 0; i < 3; ++i) {
                            g.do_stride[i] = g.dq_stride[i] = p.q_stride[i];
                            g.dk_stride[i] = g.dv_stride[i] = p.k_stride[i];
                        }
                        EXPECT(paraanya_cross_attention_backward(&p, &g, some, some, some, some, some, (float*)some, some, some, some, nullptr,
                                                                 0, nullptr) == PA_ERR_INVALID_ARG);
                        EXPECT(paraanya_cross_attention_backward(&p, &g, some, some, some, some, some, (float*)some, some, some, some, some,
                                                                 n - 1, nullptr) == PA_ERR_INVALID_ARG);
                    }
                }
    pa_cross_t c = cross(0, 5, 9, 2, 1, 64);
    EXPECT(paraanya_cross_attention(&c, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == PA_OK);
    c = cross(2, 5, 9, 2, 1, 64);
    c.scale = NAN;
    EXPECT(paraanya_cross_attention_workspace(&c, &n) == PA_ERR_INVALID_ARG);
    c.scale = 1e300;
    EXPECT(paraanya_cross_attention_workspace(&c, &n) == PA_ERR_INVALID_ARG);
    EXPECT(paraanya_cross_attention_workspace(nullptr, &n) == PA_ERR_INVALID_ARG);
    puts("cross attention ok");

    for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)5003, (int64_t)1 << 40})
        for (int64_t cols : {1, 1024, 1333, PA_NORM_MAX_COLS}) {
            pa_norm_t p = {rows, cols, PA_F16, PA_F32, 1e-5, cols, cols, cols};
            EXPECT(paraanya_layer_norm_backward_workspace(&p, &n) == PA_OK && n % 256 == 0 && (n > 0) == (rows > 0));
        }
    pa_norm_t z = {0, 64, PA_F32, PA_F32, 1e-5, 64, 64, 64};
    EXPECT(paraanya_layer_norm(&z, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == PA_OK);
    puts("layer norm ok");

    for (int64_t rows : {0, 1, 8192, 1 << 30})
        for (int rank : {1, 16, 128}) {
            pa_lora_t p = {rows, 64, 32, rank, 2, 1, PA_BF16, 64, 64, 32, (int32_t*)some, (int32_t*)some, nullptr};
            EXPECT(paraanya_lora_linear_workspace(&p, &n) == PA_OK && n % 256 == 0);
            if (rows > 0) EXPECT(paraanya_lora_linear(&p, some, some, some, some, some, some, nullptr, 0, nullptr) == PA_ERR_INVALID_ARG);
        }
    puts("projection with adapters ok");
    puts("ops_driver ok");
    return 0;
}
