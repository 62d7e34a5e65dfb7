// What the operators of include/paraanya_ops.h launch, without a GPU: the functions by which compiled host code registers and
// launches kernels are defined here, so that the library's calls end in this file. Reads a call a line,
//
//     group <backward> <batch> <pixels> <channels> <groups> <dtype> <activation>
//     feed <backward> <rows> <in> <hidden> <out> <dtype> <activation> <alignment>
//     int8 <rows> <in> <out> <dtype>
//
// and prints for each its status and kernels: "call <status>", then "<name> <grid x y z> <block x y z>" a line.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <map>
#include <string>

#include "paraanya_ops.h"

namespace {
std::map<const void*, std::string>& names() {      // (filled by the library's constructors, ahead of main)
    static std::map<const void*, std::string> m;
    return m;
}
struct Dim3 {
    uint32_t x, y, z;
};
struct Configuration {
    Dim3 grid, block;
    size_t bytes;
    void* stream;
} pushed;
}  // namespace

#define EXPORT extern "C" __attribute__((visibility("default")))
EXPORT void** __hipRegisterFatBinary(const void*) {
    static void* handle;
    return &handle;
}
EXPORT void __hipUnregisterFatBinary(void**) {}
EXPORT void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
    names()[host] = name;
}
EXPORT void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
EXPORT int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t bytes, void* stream) {
    pushed = {grid, block, bytes, stream};
    return 0;
}
EXPORT int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* bytes, void** stream) {
    *grid = pushed.grid, *block = pushed.block, *bytes = pushed.bytes, *stream = pushed.stream;
    return 0;
}
EXPORT int hipLaunchKernel(const void* kernel, Dim3 g, Dim3 b, void**, size_t, void*) {
    printf("%s %u %u %u %u %u %u\n", names()[kernel].c_str(), g.x, g.y, g.z, b.x, b.y, b.z);
    return 0;
}
EXPORT int hipGetLastError() { return 0; }

int main() {
    void* const some = (void*)(uintptr_t)4096;       // never dereferenced
    float* const numbers = (float*)some;
    const size_t much = (size_t)1 << 60;
    char line[512];
    while (fgets(line, sizeof line, stdin)) {
        char op[16];
        long long a[9] = {};
        const int n = sscanf(line, "%15s %lld %lld %lld %lld %lld %lld %lld %lld", op, a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7) - 1;
        int rc = PA_ERR_INVALID_ARG;
        if (!strcmp(op, "group") && n == 7) {
            pa_group_norm_t p = {a[1], a[2], (int32_t)a[3], (int32_t)a[4], (int32_t)a[5], (int32_t)a[5], (int32_t)a[6], 0, 1e-5, {}, {}, {}};
            for (int64_t* s : {p.x_stride, p.y_stride, p.dx_stride}) s[0] = a[2] * a[3], s[1] = a[3];
            rc = a[0] ? paraanya_group_norm_backward(&p, some, some, some, some, numbers, numbers, some, some, some, some, much, nullptr)
                      : paraanya_group_norm(&p, some, some, some, some, numbers, numbers, some, much, nullptr);
        } else if (!strcmp(op, "feed") && n == 8) {
            const pa_feed_t p = {a[1], (int32_t)a[2], (int32_t)a[3], (int32_t)a[4], (int32_t)a[5], (int32_t)a[6], (int32_t)a[7],
                                 a[2], a[2], a[2], a[3], a[4]};
            const pa_feed_grad_t g = {some, some, some, some, some, some, some};
            rc = a[0] ? paraanya_feed_forward_backward(&p, &g, some, some, some, some, some, some, much, some, much, nullptr)
                      : paraanya_feed_forward(&p, some, some, some, some, some, some, some, some, some, much, some, much, nullptr);
        } else if (!strcmp(op, "int8") && n == 4) {
            const int64_t stride = (a[1] + 15) / 16 * 16;
            const pa_int8_linear_t p = {a[0], (int32_t)a[1], (int32_t)a[2], (int32_t)a[3], 0, stride, stride, a[2]};
            rc = paraanya_int8_linear(&p, (int8_t*)some, numbers, (int8_t*)some, numbers, some, some, nullptr);
        }
        printf("call %d\n", rc);
    }
    return 0;
}
