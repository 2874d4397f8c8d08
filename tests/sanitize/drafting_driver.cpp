// Calls the host side of the operators around drafting that needs no GPU (workspace planning over its whole range, and argument errors, found before
// anything is launched) in a build whose host code carries AddressSanitizer and UndefinedBehaviorSanitizer.  Built and run by
// tests/test_drafting_sanitizers.py from csrc/drafting.hip.
#include <cstdint>
#include <cstdio>

#include "fsd.h"

extern "C" int64_t fsd_max_vocab(int) { return 524288; }   // (the verify calls' file has it)

namespace {

int bad = 0;
void expect(int got, int want, const char* what) {
    if (got != want) { std::printf("%s: status %d, expected %d\n", what, got, want); ++bad; }
}
char* place(int k) { return reinterpret_cast<char*>((static_cast<uintptr_t>(k) + 1) << 40); }   // never dereferenced: every call below fails validation first
int32_t* ints(int k) { return reinterpret_cast<int32_t*>(place(k)); }
float* floats(int k) { return reinterpret_cast<float*>(place(k)); }

int select(int B, int W, int V, int dtype, int n, int64_t stride, size_t bytes, float* out = floats(4)) {
    return fsd_beam_select(place(0), stride, floats(1), floats(2), ints(3), B, W, V, dtype, n, out, ints(5), ints(6), ints(7), place(8), bytes, nullptr);
}
fsd_cache cache_of(int layers, int blocks, int H, int D, int max_blocks, int at = 10) {
    return fsd_cache{place(at), place(at + 1), floats(at + 2), floats(at + 3), ints(at + 4), ints(at + 5), layers, blocks, H, D, max_blocks};
}
int fork(const fsd_cache* c, int B, int n, size_t bytes, int32_t* table = ints(33)) {
    return fsd_cache_fork(c, B, ints(30), ints(31), ints(32), ints(34), n, table, ints(35), ints(36), ints(37), ints(38), place(39), bytes, nullptr);
}
int compact(const fsd_cache* c, int B, size_t bytes, int32_t* table = ints(33)) {
    return fsd_cache_compact(c, B, ints(30), table, ints(36), ints(35), ints(37), ints(38), place(39), bytes, nullptr);
}

}  // namespace

int main() {
    // ---- selection: every size has a workspace, and one byte less is refused
    for (int dtype : {FSD_F32, FSD_BF16})
        for (int B : {1, 2, 7, 64, 1000, 65535})
            for (int W : {1, 3, 16, 256})
                for (int V : {1, 8, 2049, 32000, 65536, 128257, 524288})
                    for (int n : {1, 17, 128}) {
                        const size_t need = fsd_beam_workspace_bytes(B, W, V, n, dtype);
                        if (need == 0 || need % 256 != 0) { std::printf("workspace %d %d %d %d\n", B, W, V, n); ++bad; }
                        expect(select(B, W, V, dtype, n, V, need - 1), FSD_ERR_WORKSPACE, "select workspace");
                        expect(select(B, W, V, dtype, n, int64_t(1) << 32, need, floats(0)), FSD_ERR_LAYOUT, "select output over logits");
                        expect(select(B, W, V, dtype, n, V - 1, need), FSD_ERR_LAYOUT, "select stride");
                    }
    for (int W : {0, 257, -1, 2147483647}) expect(select(2, W, 100, FSD_F32, 4, 100, size_t(1) << 40), FSD_ERR_SHAPE, "select beams");
    for (int n : {0, 129, -5, 2147483647}) expect(select(2, 2, 100, FSD_F32, n, 100, size_t(1) << 40), FSD_ERR_SHAPE, "select n");
    for (int V : {0, 524289, -1, 2147483647}) expect(select(2, 2, V, FSD_BF16, 4, int64_t(1) << 31, size_t(1) << 40), FSD_ERR_SHAPE, "select V");
    expect(select(2, 2, 100, FSD_F16, 4, 100, size_t(1) << 40), FSD_ERR_DTYPE, "select dtype");
    // ---- states: sizes whose bytes would not fit a size_t
    expect(fsd_beam_reorder(place(0), ints(1), 32767, 65535, 1, 1, size_t(1) << 40, place(2), nullptr, nullptr), FSD_ERR_SHAPE, "reorder bytes");
    expect(fsd_beam_reorder(place(0), ints(1), 65535, 65535, 1, 1, 1, place(2), nullptr, nullptr), FSD_ERR_SHAPE, "reorder rows");
    expect(fsd_beam_reorder(place(0), ints(1), 1, 1, 65536, 1, 1, place(2), nullptr, nullptr), FSD_ERR_SHAPE, "reorder beams");
    expect(fsd_beam_reorder(place(0), ints(1), 3, 5, 7, 9, 1000, place(0) + 3 * 5 * 7 * 1000 - 1, nullptr, nullptr), FSD_ERR_LAYOUT, "reorder overlap");
    expect(fsd_beam_reorder(place(0), ints(1), 3, 5, 7, 9, 0, place(2), nullptr, nullptr), FSD_ERR_SHAPE, "reorder nothing");
    // ---- pages
    for (int P : {1, 5, 1023, 1024, 1025, 4096, 4097, 100000, 1 << 24})
        for (int n : {1, 2, 255, 256, 257, 65535}) {
            const size_t need = fsd_cache_fork_workspace_bytes(P, n);
            const fsd_cache c = cache_of(2, P, 3, 64, 4);
            if (need == 0 || need % 256 != 0) { std::printf("fork workspace %d %d\n", P, n); ++bad; }
            expect(fork(&c, 7, n, need - 1), FSD_ERR_WORKSPACE, "fork workspace");
            expect(fork(&c, 7, n, need, ints(14)), FSD_ERR_LAYOUT, "fork in place");
            const size_t room = fsd_cache_compact_workspace_bytes(P);
            expect(compact(&c, 7, room - 1), FSD_ERR_WORKSPACE, "compact workspace");
            expect(compact(&c, 7, room, ints(14) + 1), FSD_ERR_LAYOUT, "compact into a part of the table");
        }
    const fsd_cache wide = cache_of(1, 10, 1, 64, 32768), widest = cache_of(1, 10, 1, 64, (1 << 25) - 2), many = cache_of(1, (1 << 24) + 1, 1, 64, 4), c = cache_of(3, 10, 2, 128, 4);
    expect(fork(&wide, 65535, 65535, 100), FSD_ERR_WORKSPACE, "fork of most places");
    expect(fork(&widest, 65535, 65, 100), FSD_ERR_SHAPE, "fork of too many places");
    expect(fork(&widest, 65535, 64, 100), FSD_ERR_WORKSPACE, "fork of long tables");
    expect(fork(&many, 2, 2, size_t(1) << 40), FSD_ERR_SHAPE, "fork blocks");
    expect(compact(&many, 2, size_t(1) << 40), FSD_ERR_SHAPE, "compact blocks");
    expect(fork(nullptr, 2, 2, size_t(1) << 40), FSD_ERR_NULL, "fork cache");
    expect(compact(nullptr, 2, size_t(1) << 40), FSD_ERR_NULL, "compact cache");
    const fsd_cache other = cache_of(3, 2147483647, 2, 128, 4, 50), tall = cache_of(2147483647, 2147483647, 1024, 256, 4, 60), tall_too = cache_of(2147483647, 5, 1024, 256, 4, 70),
                    shifted = cache_of(3, 10, 2, 128, 4, 11);
    expect(fsd_cache_copy(&c, nullptr, ints(1), ints(2), nullptr, 4, nullptr, nullptr), FSD_ERR_NULL, "copy cache");
    expect(fsd_cache_copy(&c, &other, ints(1), ints(2), nullptr, 0, nullptr, nullptr), FSD_ERR_SHAPE, "copy nothing");
    expect(fsd_cache_copy(&c, &tall, ints(1), ints(2), nullptr, 4, nullptr, nullptr), FSD_ERR_SHAPE, "copy geometry");
    expect(fsd_cache_copy(&tall, &tall_too, ints(1), ints(2), nullptr, 2147483647, nullptr, nullptr), FSD_ERR_SHAPE, "copy units");
    expect(fsd_cache_copy(&c, &shifted, ints(1), ints(2), nullptr, 4, nullptr, nullptr), FSD_ERR_LAYOUT, "copy into half of a cache");
    expect(fsd_cache_copy(&c, &other, ints(1), ints(2), nullptr, 4, ints(1) + 3, nullptr), FSD_ERR_LAYOUT, "copy report");
    std::printf("drafting sanitizer driver: %d unexpected results\n", bad);
    return bad ? 1 : 0;
}
