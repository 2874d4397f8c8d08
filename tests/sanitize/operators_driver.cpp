// Calls the host side of the operators around a verify call that needs no GPU (workspace planning over their whole range, and every argument error,
// found before anything is launched) in a build whose host code carries AddressSanitizer and UndefinedBehaviorSanitizer.  Built and run by
// tests/test_operators_sanitizers.py from csrc/operators.hip.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "fsd.h"

extern "C" int64_t fsd_max_vocab(int) { return 524288; }   // (the verify calls' file has it)

namespace {

int bad = 0;
void expect(int got, int want, const char* what) {
    if (got != want) { std::printf("%s: status %d, expected %d\n", what, got, want); ++bad; }
}
char* const fake = reinterpret_cast<char*>(0x100000);   // never dereferenced: every call below fails validation first
const int32_t* ints(size_t at) { return reinterpret_cast<const int32_t*>(fake + at); }
int32_t* outs(size_t at) { return reinterpret_cast<int32_t*>(fake + at); }

fsd_cache cache_of(int D, int H, int max_blocks) {
    return fsd_cache{fake, fake, reinterpret_cast<float*>(fake), reinterpret_cast<float*>(fake), ints(0x10000), ints(0x20000), 2, 10, H, D, max_blocks};
}
int chain(int B, int K, int rows, int V, int dtype, const fsd_conditions& c, const void* z, void* out, bool tree = false) {
    if (tree) return fsd_condition_tree(z, ints(0), ints(0), B, K, rows, V, dtype, &c, out, nullptr);
    return fsd_condition_chain(z, ints(0), B, K, rows, V, dtype, &c, out, nullptr);
}
int append(const fsd_cache* c, int B, int R, int dtype, const fsd_rotation* rot, int32_t* len, int32_t* status, int64_t stride, int depth = 0) {
    return fsd_cache_append(fake, fake, stride, B, R, dtype, ints(0x30000), depth ? ints(0x40000) : nullptr, depth, rot, c, len, status, nullptr);
}
int attend(const fsd_cache* c, int B, int R, int heads, int dtype, float scale, const fsd_rotation* rot, int32_t* status, size_t bytes, bool tree,
           void* workspace = fake, int64_t q_stride = 1 << 20) {
    const int64_t kv = 1 << 20;
    if (tree) return fsd_attend_tree(fake, fake, fake, q_stride, kv, ints(0x50000), B, R, heads, dtype, ints(0x60000), scale, rot, c, 1, fake, status, workspace, bytes, nullptr);
    return fsd_attend_chain(fake, fake, fake, q_stride, kv, B, R, heads, dtype, ints(0x60000), scale, rot, c, 1, fake, status, workspace, bytes, nullptr);
}

}  // namespace

int main() {
    // ---- workspace sizes: every layout of heads over the whole range of rows and sequences, none of them smaller than a smaller call's
    for (int D : {64, 128, 256})
        for (int H : {1, 2, 7, 8, 1024})
            for (int G : {1, 3, 8, 64}) {
                if (H * G > 1024) continue;
                size_t last = 0;
                for (int R : {1, 2, 9, 16, 17, 64, 65, 100, 1000, 2049}) {
                    const size_t n = fsd_attend_workspace_bytes(1, R, H * G, H, D), three = fsd_attend_workspace_bytes(3, R, H * G, H, D);
                    if (n == 0 || n % 256 != 0 || three <= n || (R > 64 && n < last)) { std::printf("workspace %d %d %d %d\n", R, G, H, D); ++bad; }
                    last = n;
                    const fsd_cache c = cache_of(D, H, 4);
                    for (bool tree : {false, true}) {
                        expect(attend(&c, 3, R, H * G, FSD_BF16, 0.1f, nullptr, nullptr, 255, tree), FSD_ERR_WORKSPACE, "attend workspace");
                        expect(attend(&c, 3, R, H * G, FSD_F16, 0.1f, nullptr, nullptr, 0, tree), FSD_ERR_WORKSPACE, "attend workspace, f16");
                        expect(attend(&c, 3, R, H * G, FSD_F16, 0.1f, nullptr, nullptr, size_t(1) << 60, tree, fake + 16), FSD_ERR_WORKSPACE, "attend workspace alignment");
                        expect(attend(&c, 3, R, H * G, FSD_BF16, 0.1f, nullptr, outs(0x20000), size_t(1) << 60, tree), FSD_ERR_LAYOUT, "attend report over lengths");
                        expect(attend(&c, 3, R, H * G, FSD_BF16, 0.1f, nullptr, outs(0x60000 - 8), size_t(1) << 60, tree), FSD_ERR_LAYOUT, "attend report over row counts");
                    }
                }
            }
    if (fsd_attend_workspace_bytes(65535, 256, 8, 8, 128) == 0 || fsd_attend_workspace_bytes(65535, 257, 8, 8, 128) != 0 ||
        fsd_attend_workspace_bytes(8191, 2048, 1024, 1024, 256) == 0 || fsd_attend_workspace_bytes(1, 1, 65, 1, 64) != 0) {
        std::printf("workspace limits\n");
        ++bad;
    }
    // ---- attention
    const float inf = INFINITY;
    const fsd_cache c = cache_of(128, 2, 4), longest = cache_of(64, 1, (1 << 25) - 2), too_long = cache_of(64, 1, (1 << 25) - 1), many = cache_of(64, 128, 1 << 24);
    const size_t big = size_t(1) << 60;
    const fsd_rotation table = {reinterpret_cast<const float*>(fake), 9, 128, FSD_ROPE_HALVES}, wide = {reinterpret_cast<const float*>(fake), 9, 144, 0},
                       none = {nullptr, 0, 0, 7}, style = {reinterpret_cast<const float*>(fake), 9, 64, 5};
    expect(attend(nullptr, 2, 9, 8, FSD_BF16, 0.1f, nullptr, nullptr, big, false), FSD_ERR_NULL, "attend cache");
    expect(attend(&c, 2, 9, 8, FSD_F32, 0.1f, nullptr, nullptr, big, false), FSD_ERR_DTYPE, "attend dtype");
    expect(attend(&c, 2, 9, 7, FSD_BF16, 0.1f, nullptr, nullptr, big, false), FSD_ERR_SHAPE, "attend heads");
    expect(attend(&c, 2, 2050, 8, FSD_BF16, 0.1f, nullptr, nullptr, big, true), FSD_ERR_SHAPE, "attend rows");
    expect(attend(&c, 2, 9, 8, FSD_BF16, inf, nullptr, nullptr, big, false), FSD_ERR_SHAPE, "attend scale");
    expect(attend(&c, 2, 9, 8, FSD_BF16, 3.0e38f, nullptr, nullptr, big, false), FSD_ERR_SHAPE, "attend scale in powers of two");
    expect(attend(&c, 2, 9, 8, FSD_BF16, 0.1f, &wide, nullptr, big, false), FSD_ERR_SHAPE, "attend rotation");
    expect(attend(&c, 2, 9, 8, FSD_BF16, 0.1f, &style, nullptr, big, false), FSD_ERR_MODE, "attend rotation style");
    expect(attend(&c, 2, 9, 8, FSD_BF16, 0.1f, &none, nullptr, 100, false), FSD_ERR_WORKSPACE, "attend without a table");
    expect(attend(&c, 2, 9, 8, FSD_BF16, 0.1f, &table, nullptr, big, false, fake, 1020), FSD_ERR_LAYOUT, "attend stride");
    expect(attend(&longest, 2, 9, 1, FSD_BF16, 0.1f, nullptr, nullptr, 100, false), FSD_ERR_WORKSPACE, "attend longest table");
    expect(attend(&too_long, 2, 9, 1, FSD_BF16, 0.1f, nullptr, nullptr, big, false), FSD_ERR_SHAPE, "attend too long a table");
    expect(attend(&many, 2, 9, 128, FSD_BF16, 0.1f, nullptr, nullptr, big, false), FSD_ERR_SHAPE, "attend units");
    // ---- appending
    expect(append(nullptr, 2, 9, FSD_F32, nullptr, nullptr, nullptr, 256), FSD_ERR_NULL, "append cache");
    expect(append(&c, 2, 9, 3, nullptr, nullptr, nullptr, 256), FSD_ERR_DTYPE, "append dtype");
    expect(append(&c, 0, 9, FSD_F16, nullptr, nullptr, nullptr, 256), FSD_ERR_SHAPE, "append B");
    expect(append(&c, 2, (1 << 20) + 1, FSD_F16, nullptr, nullptr, nullptr, 256), FSD_ERR_SHAPE, "append R");
    expect(append(&c, 65535, 1 << 20, FSD_F16, nullptr, nullptr, nullptr, 256), FSD_ERR_SHAPE, "append grid");
    expect(append(&c, 2, 9, FSD_F16, nullptr, nullptr, nullptr, 256, 2049), FSD_ERR_SHAPE, "append depth");
    expect(append(&c, 2, 9, FSD_F16, nullptr, nullptr, nullptr, 248), FSD_ERR_LAYOUT, "append stride");
    expect(append(&c, 2, 9, FSD_F16, nullptr, nullptr, nullptr, (int64_t(1) << 32) + 8), FSD_ERR_LAYOUT, "append far stride");
    expect(append(&c, 2, 9, FSD_F16, &wide, nullptr, nullptr, 256), FSD_ERR_SHAPE, "append rotation");
    expect(append(&c, 2, 9, FSD_F16, nullptr, outs(0x20004), nullptr, 256), FSD_ERR_LAYOUT, "append length over lengths");
    expect(append(&c, 2, 9, FSD_F16, nullptr, nullptr, outs(0x30000 - 4), 256), FSD_ERR_LAYOUT, "append report over accepted");
    expect(append(&c, 65535, 9, FSD_F16, nullptr, outs(0x70000), outs(0x70000 + 4 * 65534), 256), FSD_ERR_LAYOUT, "append report over length");
    expect(append(&c, 2, 9, FSD_F16, nullptr, outs(0x40000 + 4 * 15), nullptr, 256, 8), FSD_ERR_LAYOUT, "append length over path");
    // ---- conditioning
    fsd_conditions d{};
    expect(chain(2, 4, 5, 1000, FSD_F16, d, fake, fake), FSD_ERR_DTYPE, "condition dtype");
    expect(chain(2, 4, 3, 1000, FSD_F32, d, fake, fake), FSD_ERR_SHAPE, "condition rows");
    expect(chain(65535, 300, 300, 1000, FSD_F32, d, fake, fake), FSD_ERR_SHAPE, "condition B rows");
    expect(chain(2, 4, 5, 524289, FSD_F32, d, fake, fake), FSD_ERR_SHAPE, "condition V");
    expect(chain(2, 0, 1, 1000, FSD_F32, d, fake, fake, true), FSD_ERR_SHAPE, "condition tree of nothing");
    expect(chain(2, 4, 5, 1000, FSD_F32, d, fake + 2, fake), FSD_ERR_LAYOUT, "condition address");
    expect(chain(65535, 255, 256, 524288, FSD_F32, d, fake, fake + 4), FSD_ERR_LAYOUT, "condition overlap, 2^45 bytes");
    expect(chain(2, 4, 5, 1000, FSD_BF16, d, fake, fake + 2 * 5 * 1000 * 2 - 2, true), FSD_ERR_LAYOUT, "condition overlap");
    d.bias_count = 2147483647;
    expect(chain(2, 4, 5, 1000, FSD_F32, d, fake, fake), FSD_ERR_NULL, "condition biases");
    d.bias_count = 0;
    d.history_stride = (1 << 29) + 1;
    expect(chain(2, 4, 5, 1000, FSD_F32, d, fake, fake), FSD_ERR_SHAPE, "condition history");
    d.history_stride = 0;
    d.allowed = reinterpret_cast<const uint32_t*>(fake);
    d.allowed_contexts = 2;
    expect(chain(2, 4, 5, 1000, FSD_F32, d, fake, fake), FSD_ERR_SHAPE, "condition masks");
    std::printf("operators sanitizer driver: %d unexpected results\n", bad);
    return bad ? 1 : 0;
}
