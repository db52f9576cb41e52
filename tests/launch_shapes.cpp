// The launches that the query-tower operators ask for, without a GPU: this
// program stands in for the runtime's launch functions, loads the library, calls
// the operators on pointers that nothing reads and checks every launch's shape. A
// launch may not have 2^32 threads in one direction.
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <vector>

#include "boa.h"

struct Dim {
    uint32_t x, y, z;
};

static std::vector<std::pair<Dim, Dim>> launches;
static int failures = 0;

extern "C" {
int __hipPushCallConfiguration(Dim grid, Dim block, size_t, void *)
{
    launches.push_back({grid, block});
    return 0;
}
int __hipPopCallConfiguration(Dim *grid, Dim *block, size_t *shared, void **stream)
{
    *grid = launches.back().first, *block = launches.back().second, *shared = 0, *stream = nullptr;
    return 0;
}
int hipLaunchKernel(const void *, Dim, Dim, void **, size_t, void *) { return 0; }
int hipGetLastError() { return 0; }
int hipFuncSetAttribute(const void *, int, int) { return 0; }
}

static void expect(bool ok, const char *what, long long a, long long b, long long c)
{
    if (ok) return;
    ++failures;
    printf("%s: %lld %lld %lld\n", what, a, b, c);
}

// Checks the launches since the last call; the blocks of all of them.
static int64_t look(const char *what, int rc, long long a, long long b, long long c)
{
    expect(rc == 0, what, a, b, c);
    expect(!launches.empty(), "no launch", a, b, c);
    int64_t blocks = 0;
    for (auto &[g, t] : launches) {
        const uint64_t most = 1ull << 32;
        expect(t.x >= 1 && t.x * t.y * t.z <= 1024, "threads of a block", t.x, t.y, t.z);
        expect(g.x >= 1 && g.y >= 1 && g.z >= 1, "no blocks", g.x, g.y, g.z);
        expect((uint64_t)g.x * t.x < most && (uint64_t)g.y * t.y < most && (uint64_t)g.z * t.z < most, what, a, b, c);
        expect(g.y < 65536 && g.z < 65536, "blocks in y or z", g.x, g.y, g.z);
        blocks += (int64_t)g.x * g.y * g.z;
    }
    launches.clear();
    return blocks;
}

int main(int argc, char **argv)
{
    void *lib = argc > 1 ? dlopen(argv[1], RTLD_NOW) : nullptr;
    if (!lib) {
        printf("no library: %s\n", argc > 1 ? dlerror() : "no path");
        return 2;
    }
    const auto norm = (decltype(&boa_layer_norm))dlsym(lib, "boa_layer_norm");
    const auto block = (decltype(&boa_block_norm))dlsym(lib, "boa_block_norm");
    const auto block_back = (decltype(&boa_block_norm_backward))dlsym(lib, "boa_block_norm_backward");
    const auto linear = (decltype(&boa_linear))dlsym(lib, "boa_linear");
    const auto linear_grad = (decltype(&boa_linear_grad))dlsym(lib, "boa_linear_grad");
    const auto orth = (decltype(&boa_orthogonalize))dlsym(lib, "boa_orthogonalize");
    char *const p = (char *)(1ull << 40);   // nothing reads it
    const int64_t room = INT64_MAX / 2;

    for (int32_t dtype : {BOA_T_F32, BOA_T_BF16, BOA_T_F16})
        for (int64_t rows : {int64_t(1), (int64_t(1) << 22), (int64_t(1) << 23), (int64_t(1) << 23) + 77, (int64_t(1) << 31) - 1})
            for (int32_t d : {1, 7, 8, 64, 255, 256, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 4104, 8191, 8192, 8193, 1 << 20}) {
                look("layer_norm", norm(p, rows, d, d, dtype, p, p, dtype, 1e-5f, p, nullptr, nullptr, nullptr), rows, d, dtype);
                for (int pre : {0, 1}) {
                    boa_block b{};
                    b.dtype = b.param_dtype = dtype, b.rows = rows, b.d = d, b.post = 1, b.pre = pre, b.scale = 1.0f, b.eps = 1e-5f;
                    b.x = b.f = p, b.x_stride = b.f_stride = d, b.h = p, b.y = p, b.stats = (float *)p;
                    const int64_t blocks = look("block_norm", block(&b, nullptr), rows, d, dtype);
                    if (d > 4096) expect(blocks == rows, "a block a row", blocks, rows, d);
                    b.dh = p, b.dh_stride = d, b.dx = b.df = b.dpost_weight = p, b.workspace = p, b.workspace_bytes = room;
                    look("block_norm_backward", block_back(&b, nullptr), rows, d, dtype);
                }
            }
    for (int32_t dtype : {BOA_T_F32, BOA_T_BF16, BOA_T_F16})
        for (int64_t M : {int64_t(1), int64_t(17), int64_t(1) << 20, (int64_t(1) << 30) + 100, int64_t(BOA_MAX_LINEAR_ROWS)})
            for (int32_t N : {1, 40, 4096, BOA_MAX_LINEAR})
                for (int32_t K : {1, 40, 4096, BOA_MAX_LINEAR}) {
                    if ((double)M * N > 1e12 || (double)M * K > 1e12) continue;
                    boa_dense l{};
                    l.dtype = l.param_dtype = dtype, l.activation = BOA_ACT_GELU, l.M = M, l.N = N, l.K = K, l.x = l.w = p;
                    l.x_stride = l.w_stride = K, l.y = l.pre = p, l.dy = p, l.dy_stride = N, l.dx = l.dw = l.dbias = p;
                    look("linear", linear(&l, p, room, nullptr), M, N, K);
                    look("linear_grad", linear_grad(&l, p, room, nullptr), M, N, K);
                }
    const float steps[6] = {3.4445f, -4.7750f, 2.0315f, 1.5f, -0.5f, 0.0f};
    for (int32_t dtype : {BOA_T_F32, BOA_T_BF16, BOA_T_F16})
        for (int64_t count : {1, 300, BOA_MAX_ORTH_COUNT})
            for (int32_t rows : {1, 16, 64, 65, 127, 128, 1000, BOA_MAX_ORTH})
                for (int32_t cols : {1, 16, 64, 65, 127, 128, 1000, BOA_MAX_ORTH}) {
                    if ((double)count * rows * cols > 1e11) continue;
                    boa_orth o{};
                    o.dtype = dtype, o.rows = rows, o.cols = cols, o.count = count, o.update = p, o.update_stride = cols;
                    o.update_batch = (int64_t)rows * cols, o.steps = 2, o.coefficients = steps, o.eps = 1e-7f, o.out = p;
                    look("orthogonalize", orth(&o, p, room, nullptr), count, rows, cols);
                }
    printf("%d failures\n", failures);
    return failures != 0;
}
