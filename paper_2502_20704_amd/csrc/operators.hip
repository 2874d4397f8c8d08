// Host side and C ABI of the operators around a verify call: conditioning of logits (condition.h), the 8-bit paged
// cache's append (cache_append.h) and the attention that reads it (cache_attend.h).  Kernels for gfx950 (MI355X).

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <limits.h>
#include <cmath>
#include <type_traits>

#include "fsd.h"

#include "operators_common.h"
#include "operators_host.h"
#include "condition.h"
#include "cache_append.h"
#include "cache_attend.h"

namespace {

// ------------------------------------------------------------------------------------------ conditioning

constexpr long kConditionWGs = 1024;   // workgroups aimed at: 4 a compute unit, which is what their LDS allows at once

template <bool BF16>
void launch_condition(hipStream_t st, unsigned grid, size_t lds, bool tree, bool stream, const ConditionParams& P) {
    const dim3 g(grid), t(kWG);
    if (tree) {
        if (stream) hipLaunchKernelGGL((condition_rows<BF16, true, true>), g, t, lds, st, P);
        else hipLaunchKernelGGL((condition_rows<BF16, true, false>), g, t, lds, st, P);
    } else {
        if (stream) hipLaunchKernelGGL((condition_rows<BF16, false, true>), g, t, lds, st, P);
        else hipLaunchKernelGGL((condition_rows<BF16, false, false>), g, t, lds, st, P);
    }
}

int condition(const void* logits, const int32_t* tokens, const int32_t* parent, int B, int N, int rows, int V, int dtype,
              const fsd_conditions* conditions, void* out, bool tree, hipStream_t st) {
    if (!logits || !out || !conditions || (N > 0 && !tokens) || (tree && !parent)) return FSD_ERR_NULL;
    if (dtype != FSD_F32 && dtype != FSD_BF16) return FSD_ERR_DTYPE;
    if (B < 1 || B > kMaxBatch || N < (tree ? 1 : 0) || N > kMaxRows || rows < 1 || (rows != N && rows != N + 1) || V < 1 ||
        V > fsd_max_vocab(dtype) || static_cast<long>(B) * rows >= (1L << 24))
        return FSD_ERR_SHAPE;
    const fsd_conditions& c = *conditions;
    if (c.history_stride < 0 || c.history_stride > (1 << 29) || c.bias_count < 0) return FSD_ERR_SHAPE;
    if (c.bias_count > 0 && (!c.bias_tokens || !c.bias_values)) return FSD_ERR_NULL;
    if (c.allowed && c.allowed_contexts != 1 && c.allowed_contexts != N + 1) return FSD_ERR_SHAPE;
    const size_t es = dtype == FSD_BF16 ? 2 : 4;
    if ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out)) % es != 0) return FSD_ERR_LAYOUT;
    const size_t bytes = static_cast<size_t>(B) * rows * V * es;
    if (out != logits && overlap(logits, bytes, out, bytes)) return FSD_ERR_LAYOUT;
    ConditionParams P;
    P.logits = static_cast<const char*>(logits);
    P.out = static_cast<char*>(out);
    P.tokens = tokens;
    P.parent = parent;
    P.c = c;
    if (c.history_stride == 0) P.c.history = nullptr;
    P.B = B; P.N = N; P.rows = rows; P.V = V;
    P.target = rows == N + 1;
    // A workgroup's slice: the fewer, the fewer times a history is read; but a call of few rows wants workgroups on all compute units.
    P.slice = kConditionSlots * kWG * (dtype == FSD_BF16 ? 8 : 4);
    while (P.slice > 1024 && static_cast<long>(B) * rows * ((V + P.slice - 1) / P.slice) < kConditionWGs) P.slice /= 2;
    // (many biases: their places and the table share 64 KB with the tree)
    auto lds_of = [&](int slice) { return static_cast<size_t>(slice) * 4 + slice / 8 + static_cast<size_t>(c.bias_count < slice ? c.bias_count : slice) * 8 + 4; };
    while (P.slice > 1024 && lds_of(P.slice) > (52u << 10)) P.slice /= 2;
    P.nslices = (V + P.slice - 1) / P.slice;
    const long pieces = static_cast<long>(B) * P.nslices;
    long per = pieces * rows / kConditionWGs;
    if (per < 1) per = 1;
    if (per > rows) per = rows;
    P.ngroups = static_cast<int>((rows + per - 1) / per);
    P.rows_per_wg = (rows + P.ngroups - 1) / P.ngroups;
    P.ngroups = (rows + P.rows_per_wg - 1) / P.rows_per_wg;
    P.nwork = pieces * P.ngroups;
    const long grid = grid_over_xcds(P.nwork);
    if (grid > kMaxGroups) return FSD_ERR_SHAPE;
    P.side = c.bias_count < P.slice ? c.bias_count : P.slice;
    size_t lds = lds_of(P.slice);
    if (tree) lds += static_cast<size_t>(N) * 6;
    // Past the caches where the logits are more than these hold and lines are written whole: 64 sequences of 9 rows of 128256 bfloat16
    // entries 77 -> 73 us; but 48 of 17 rows of 128259 binary32 entries 203 -> 207, and a small call's reader finds its rows in the caches.
    const bool stream = bytes >= (64u << 20) && V * es % 16 == 0 && aligned16(logits) && aligned16(out);
    if (dtype == FSD_BF16) launch_condition<true>(st, static_cast<unsigned>(grid), lds, tree, stream, P);
    else launch_condition<false>(st, static_cast<unsigned>(grid), lds, tree, stream, P);
    return launched();
}

// ------------------------------------------------------------------------------------------ the cache

// A sequence's new length and report are written by one workgroup, which no other waits for: they must not lie in what all of them read, nor in one another.
bool report_overlaps(const int32_t* length, const int32_t* status, int B, const fsd_cache& c, const int32_t* first, size_t n_first, const int32_t* second,
                     size_t n_second) {
    const size_t own = static_cast<size_t>(B) * 4, table = own * static_cast<size_t>(c.max_blocks);
    auto meets = [&](const int32_t* out) {
        return overlap(out, own, c.cache_len, own) || overlap(out, own, c.block_table, table) || overlap(out, own, first, n_first * 4) ||
               overlap(out, own, second, n_second * 4);
    };
    return meets(length) || meets(status) || overlap(length, own, status, own);
}
// the rotation to hand to a kernel: none where there is no table
int check_rotation(const fsd_rotation* r, int head_dim, fsd_rotation* out) {
    *out = fsd_rotation{nullptr, 0, 0, FSD_ROPE_HALVES};
    if (!r || !r->table) return FSD_OK;
    if (r->rows < 1 || r->dim < 16 || r->dim % 16 != 0 || r->dim > head_dim) return FSD_ERR_SHAPE;
    if (r->style != FSD_ROPE_HALVES && r->style != FSD_ROPE_PAIRS) return FSD_ERR_MODE;
    if (!aligned16(r->table)) return FSD_ERR_LAYOUT;
    *out = *r;
    return FSD_OK;
}

template <int DT, int D>
void launch_append(hipStream_t st, const AppendParams& P, int tokens) {
    if (tokens <= kFew) hipLaunchKernelGGL((append_few<DT, D>), dim3((P.cache.kv_heads + 1) / 2, P.B, P.cache.layers), dim3(kWG), 0, st, P);
    else hipLaunchKernelGGL((append_many<DT, D>), dim3(P.npieces), dim3(kWG), 0, st, P);
}
template <int DT>
void launch_append_d(hipStream_t st, const AppendParams& P, int tokens) {
    if (P.cache.head_dim == 64) launch_append<DT, 64>(st, P, tokens);
    else if (P.cache.head_dim == 128) launch_append<DT, 128>(st, P, tokens);
    else launch_append<DT, 256>(st, P, tokens);
}

// ------------------------------------------------------------------------------------------ attention

// How many of a key head's rows (tokens times query heads of its group) an item takes: up to 64 attend_few (binary16 48, as its second parts take registers;
// at head_dim 256 32 and 16), beyond that attend_rows with 128.  64 sequences of up to 8192 tokens, 36 rows a key head: 171 us with attend_few, 200 with
// attend_rows.  Twice the rows an item (8 wavefronts, 256 workgroups): 162 us as well for trees of 244 rows, 115 in place of 110 for a prompt's 1000.
struct AttendShape { int rt, tile, workers; bool few; };
constexpr int rows_waves(int head_dim) { return head_dim == 256 ? 8 : 4; }   // of attend_rows: 16 sequences of 256 rows at head_dim 256 62 us with 8, 68 with 4
// Tiles of 16 rows of each of them: at head_dim 128 and 256 what registers hold beside the sums; at 64 they would hold more, which is not measured.
constexpr int rows_tiles(int head_dim) { return head_dim == 256 ? 1 : 2; }
AttendShape attend_shape(long rows, int head_dim, int dtype) {
    AttendShape s;
    const long tiles = (rows + 15) / 16;
    s.few = tiles <= (head_dim == 256 ? 2 : 4) - (dtype == FSD_F16 ? 1 : 0);
    s.rt = s.few ? static_cast<int>(tiles) : rows_tiles(head_dim);
    s.tile = 16 * s.rt * (s.few ? 1 : rows_waves(head_dim));
    // Two workgroups for each of the 256 compute units, or one of eight wavefronts: what their registers and LDS hold at once at head_dim 128 and 256.  (At
    // 64 three of most kinds would fit, and four of the smallest; not measured.)
    s.workers = s.few || head_dim != 256 ? 512 : 256;
    return s;
}
bool attend_sizes(int B, int R, int heads, int kv_heads, int head_dim) {
    return B >= 1 && B <= kMaxBatch && R >= 1 && R <= kMaxRows + 1 && static_cast<long>(B) * R < (1L << 24) && kv_heads >= 1 && heads >= kv_heads &&
           heads <= 1024 && heads % kv_heads == 0 && heads / kv_heads <= 64 && (head_dim == 64 || head_dim == 128 || head_dim == 256);
}
// Places of the workspace's parts (attend_prepare says what they hold), and its size.
struct AttendSpace {
    int row_tiles, tiles;
    size_t pieces, factor, key_scale, value_lift, row_lift, broken, sees, q16, k16, v16, part, bytes;
};
AttendSpace attend_space(const AttendShape& s, int B, int R, int heads, int H, int D, bool fine) {
    AttendSpace w;
    const long rows = static_cast<long>(R) * (heads / H), groups = (rows + s.tile - 1) / s.tile;
    w.row_tiles = static_cast<int>(groups * s.tile / 16);
    w.tiles = (R + kBlock - 1) / kBlock;
    const size_t bh = static_cast<size_t>(B) * H, bht = bh * w.tiles, parts = fine ? 2 : 1;
    size_t o = 0;
    auto take = [&o](size_t n) {
        const size_t at = o;
        o = (o + n + 255) / 256 * 256;
        return at;
    };
    take((static_cast<size_t>(B) + 2) * 8);                   // the plan
    w.pieces = take(bh * groups * 8);
    w.factor = take(bh * w.row_tiles * 64);
    w.key_scale = take(bht * kBlock * 4);
    w.value_lift = take(bht * 4);
    w.row_lift = take(bht * kBlock);
    w.broken = take(bht * 8);
    w.sees = take(static_cast<size_t>(B) * R * w.tiles * 8);
    w.q16 = take(bh * w.row_tiles * 32 * D * parts);
    w.k16 = take(bht * kBlock * 2 * D * parts);
    w.v16 = take(bht * kBlock * 2 * D);
    w.part = take(2 * static_cast<size_t>(s.workers) * s.tile * (D + 2) * 4);
    w.bytes = o;
    return w;
}

template <int D, int RT>
void launch_attend_few(hipStream_t st, const AttendParams& P) {
    const dim3 grid(static_cast<unsigned>(grid_over_xcds(P.workers)));
    if constexpr (RT < (D == 256 ? 2 : 4)) {
        if (P.dtype == FSD_F16) {
            hipLaunchKernelGGL((attend_few<D, RT, true>), grid, dim3(kWG), 0, st, P);
            return;
        }
    }
    hipLaunchKernelGGL((attend_few<D, RT, false>), grid, dim3(kWG), 0, st, P);
}
template <int D>
void launch_attend_rows(hipStream_t st, const AttendParams& P) {
    constexpr int RT = rows_tiles(D), NW = rows_waves(D);
    const dim3 grid(static_cast<unsigned>(grid_over_xcds(P.workers)));
    if (P.dtype == FSD_F16) hipLaunchKernelGGL((attend_rows<D, RT, NW, true>), grid, dim3(NW * 64), 0, st, P);
    else hipLaunchKernelGGL((attend_rows<D, RT, NW, false>), grid, dim3(NW * 64), 0, st, P);
}
template <int D>
void launch_attend(hipStream_t st, const AttendParams& P, const AttendShape& s, unsigned prepare, size_t lds, unsigned joins, int by_pieces) {
    const dim3 g(prepare, static_cast<unsigned>(P.B));
    if (P.dtype == FSD_F16) hipLaunchKernelGGL((attend_prepare<D, true>), g, dim3(kWG), lds, st, P);
    else hipLaunchKernelGGL((attend_prepare<D, false>), g, dim3(kWG), lds, st, P);
    if (!s.few) {
        launch_attend_rows<D>(st, P);
    } else if (s.rt == 1) {
        launch_attend_few<D, 1>(st, P);
    } else if (s.rt == 2) {
        launch_attend_few<D, 2>(st, P);
    } else if constexpr (D != 256) {
        if (s.rt == 3) launch_attend_few<D, 3>(st, P);
        else launch_attend_few<D, 4>(st, P);
    }
    hipLaunchKernelGGL((attend_join<D>), dim3(joins, static_cast<unsigned>(P.cache.kv_heads), static_cast<unsigned>(P.B)), dim3(kWG), 0, st, P, by_pieces);
}

int attend(const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride, const int32_t* parent, bool tree, int B, int R,
           int heads, int dtype, const int32_t* row_count, float scale, const fsd_rotation* rotation, const fsd_cache* cache, int layer,
           void* out, int32_t* row_status, void* workspace, size_t workspace_bytes, hipStream_t st) {
    if (!q || !k || !v || !out || (tree && !parent && R > 1)) return FSD_ERR_NULL;
    AttendParams P;
    int bad = check_cache(cache);
    if (bad == FSD_OK) bad = check_rotation(rotation, cache->head_dim, &P.rot);
    if (bad != FSD_OK) return bad;
    if (dtype != FSD_BF16 && dtype != FSD_F16) return FSD_ERR_DTYPE;
    const int H = cache->kv_heads, D = cache->head_dim;
    if (!attend_sizes(B, R, heads, H, D) || layer < 0 || layer >= cache->layers || !std::isfinite(scale * kLog2eF)) return FSD_ERR_SHAPE;
    if (q_stride < static_cast<int64_t>(heads) * D || kv_stride < static_cast<int64_t>(H) * D || q_stride % 8 != 0 || kv_stride % 8 != 0 ||
        q_stride > (1L << 32) || kv_stride > (1L << 32) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return FSD_ERR_LAYOUT;
    const AttendShape s = attend_shape(static_cast<long>(R) * (heads / H), D, dtype);
    const AttendSpace w = attend_space(s, B, R, heads, H, D, dtype == FSD_F16);
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < w.bytes) return FSD_ERR_WORKSPACE;
    P.q = q; P.k = k; P.v = v;
    P.q_stride = q_stride; P.kv_stride = kv_stride;
    P.parent = tree && R > 1 ? parent : nullptr;
    P.row_count = row_count;
    P.B = B; P.R = R; P.heads = heads; P.G = heads / H;
    P.dtype = dtype;
    P.scale = scale * kLog2eF;
    P.cache = *cache;
    P.layer = layer;
    P.out = out;
    P.status = row_status;
    char* base = static_cast<char*>(workspace);
    P.plan = reinterpret_cast<long*>(base);
    P.pieces = reinterpret_cast<int2*>(base + w.pieces);
    P.factor = reinterpret_cast<float*>(base + w.factor);
    P.key_scale = reinterpret_cast<float*>(base + w.key_scale);
    P.value_lift = reinterpret_cast<int*>(base + w.value_lift);
    P.row_lift = reinterpret_cast<unsigned char*>(base + w.row_lift);
    P.broken = reinterpret_cast<unsigned long long*>(base + w.broken);
    P.sees = reinterpret_cast<unsigned long long*>(base + w.sees);
    P.q16 = base + w.q16;
    P.k16 = base + w.k16;
    P.v16 = base + w.v16;
    P.part = reinterpret_cast<float*>(base + w.part);
    P.workers = s.workers;
    P.tile = s.tile;
    P.row_tiles = w.row_tiles;
    P.tiles = w.tiles;
    auto for_dividing = [](int d) { return d == 1 ? 0u : static_cast<unsigned>(((1ul << 32) + d - 1) / d); };
    P.by_heads = for_dividing(heads);
    P.by_G = for_dividing(P.G);
    P.by_tile = for_dividing(s.tile);
    // Of attend_prepare a sequence's queries take 8 elements in each of two slots of a thread, a key head's tile D / 64 workgroups and one.
    const long prepare = 1 + (static_cast<long>(R) * heads * (D / 8) + 2 * kWG - 1) / (2 * kWG) + static_cast<long>(H) * P.tiles * (D / 64 + 1);
    // A workgroup of attend_join takes one row where the rows are few, else as many as its lanes hold (measured there).
    const int by_pieces = static_cast<long>(B) * R * heads <= 4096, row_groups = by_pieces ? 1 : 4 * kWG / D;
    const unsigned joins = static_cast<unsigned>((static_cast<long>(R) * P.G + row_groups - 1) / row_groups);
    const long units = (kStart + static_cast<long>(cache->max_blocks) + P.tiles) * H * (P.row_tiles * 16 / s.tile);   // of a sequence, at most
    if (prepare > kMaxGroups || units > INT_MAX) return FSD_ERR_SHAPE;
    if (report_overlaps(nullptr, row_status, B, *cache, row_count, static_cast<size_t>(B), P.parent, static_cast<size_t>(B) * (R - 1))) return FSD_ERR_LAYOUT;
    const size_t lds = P.parent ? static_cast<size_t>(R) * 6 : 0;
    if (D == 64) launch_attend<64>(st, P, s, static_cast<unsigned>(prepare), lds, joins, by_pieces);
    else if (D == 128) launch_attend<128>(st, P, s, static_cast<unsigned>(prepare), lds, joins, by_pieces);
    else launch_attend<256>(st, P, s, static_cast<unsigned>(prepare), lds, joins, by_pieces);
    return launched();
}

}  // namespace

extern "C" {

int fsd_condition_chain(const void* logits, const int32_t* cand_tokens, int B, int K, int rows, int V, int dtype,
                        const fsd_conditions* conditions, void* out, void* hip_stream) {
    return condition(logits, cand_tokens, nullptr, B, K, rows, V, dtype, conditions, out, false, static_cast<hipStream_t>(hip_stream));
}

int fsd_condition_tree(const void* logits, const int32_t* node_tokens, const int32_t* parent, int B, int N, int rows, int V, int dtype,
                       const fsd_conditions* conditions, void* out, void* hip_stream) {
    return condition(logits, node_tokens, parent, B, N, rows, V, dtype, conditions, out, true, static_cast<hipStream_t>(hip_stream));
}

int fsd_cache_append(const void* k, const void* v, int64_t token_stride, int B, int R, int dtype, const int32_t* accept_len,
                     const int32_t* path_nodes, int max_depth, const fsd_rotation* rotation, const fsd_cache* cache,
                     int32_t* cache_len_out, int32_t* row_status, void* hip_stream) {
    if (!k || !v || !accept_len) return FSD_ERR_NULL;
    AppendParams P;
    int bad = check_cache(cache);
    if (bad == FSD_OK) bad = check_rotation(rotation, cache->head_dim, &P.rot);
    if (bad != FSD_OK) return bad;
    if (dtype != FSD_F32 && dtype != FSD_BF16 && dtype != FSD_F16) return FSD_ERR_DTYPE;
    const int H = cache->kv_heads;
    if (B < 1 || B > kMaxBatch || R < 1 || R > (1 << 20) || (path_nodes && (max_depth < 1 || max_depth > kMaxRows))) return FSD_ERR_SHAPE;
    if (token_stride < static_cast<int64_t>(H) * cache->head_dim || token_stride % 8 != 0 || token_stride > (1L << 32) || !aligned16(k) ||
        !aligned16(v))
        return FSD_ERR_LAYOUT;
    P.k = static_cast<const char*>(k);
    P.v = static_cast<const char*>(v);
    P.stride = token_stride;
    P.B = B; P.R = R; P.max_depth = max_depth;
    P.max_rows = path_nodes && max_depth + 1 < R ? max_depth + 1 : R;
    P.accept_len = accept_len;
    P.path = path_nodes;
    P.cache = *cache;
    P.len_out = cache_len_out;
    P.status = row_status;
    // few rows: two wavefronts a head, whichever blocks they touch; else a workgroup for each block
    P.slots = P.max_rows <= kFew ? 1 : (P.max_rows - 1 + kBlock - 1) / kBlock + 1;
    const long pieces = static_cast<long>(cache->layers) * B * H * P.slots;
    if (P.max_rows <= kFew ? cache->layers > 65535 : pieces > kMaxGroups) return FSD_ERR_SHAPE;
    P.npieces = static_cast<unsigned>(pieces);                // (append_many's grid)
    if (report_overlaps(cache_len_out, row_status, B, *cache, accept_len, static_cast<size_t>(B), path_nodes, static_cast<size_t>(B) * max_depth))
        return FSD_ERR_LAYOUT;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (dtype == FSD_F32) launch_append_d<FSD_F32>(st, P, P.max_rows);
    else if (dtype == FSD_BF16) launch_append_d<FSD_BF16>(st, P, P.max_rows);
    else launch_append_d<FSD_F16>(st, P, P.max_rows);
    return launched();
}

size_t fsd_attend_workspace_bytes(int B, int R, int heads, int kv_heads, int head_dim) {
    if (!attend_sizes(B, R, heads, kv_heads, head_dim)) return 0;
    const long rows = static_cast<long>(R) * (heads / kv_heads);
    const size_t a = attend_space(attend_shape(rows, head_dim, FSD_BF16), B, R, heads, kv_heads, head_dim, false).bytes;
    const size_t c = attend_space(attend_shape(rows, head_dim, FSD_F16), B, R, heads, kv_heads, head_dim, true).bytes;
    return a > c ? a : c;
}

int fsd_attend_chain(const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride, int B, int R, int heads, int dtype,
                     const int32_t* row_count, float scale, const fsd_rotation* rotation, const fsd_cache* cache, int layer, void* out,
                     int32_t* row_status, void* workspace, size_t workspace_bytes, void* hip_stream) {
    return attend(q, k, v, q_stride, kv_stride, nullptr, false, B, R, heads, dtype, row_count, scale, rotation, cache, layer, out, row_status,
                  workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
}

int fsd_attend_tree(const void* q, const void* k, const void* v, int64_t q_stride, int64_t kv_stride, const int32_t* parent, int B, int R,
                    int heads, int dtype, const int32_t* row_count, float scale, const fsd_rotation* rotation, const fsd_cache* cache, int layer,
                    void* out, int32_t* row_status, void* workspace, size_t workspace_bytes, void* hip_stream) {
    return attend(q, k, v, q_stride, kv_stride, parent, true, B, R, heads, dtype, row_count, scale, rotation, cache, layer, out, row_status,
                  workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
