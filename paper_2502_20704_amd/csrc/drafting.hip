// Host side and C ABI of the operators around drafting: the best continuations of beams and the states that follow them (beam_select.h), and the pages of
// the 8-bit paged cache (cache_pages.h).  Kernels for gfx950 (MI355X).

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <limits.h>

#include "fsd.h"

#include "operators_common.h"
#include "operators_host.h"
#include "beam_select.h"
#include "cache_pages.h"

namespace {

// parts of a workspace, one behind the other on 256-byte boundaries
struct Space {
    size_t bytes = 0;
    size_t take(size_t n) {
        const size_t at = bytes;
        bytes = (bytes + n + 255) / 256 * 256;
        return at;
    }
};
inline bool workspace_fits(const void* workspace, size_t have, size_t need) {
    return workspace && reinterpret_cast<uintptr_t>(workspace) % 256 == 0 && have >= need;
}
// runs of bytes; whether one of the first n_out meets another of them or one of the rest
struct Run { const void* at; size_t bytes; };
bool any_overlap(const Run* runs, int n_out, int n) {
    for (int i = 0; i < n_out; ++i)
        for (int k = i + 1; k < n; ++k)
            if (overlap(runs[i].at, runs[i].bytes, runs[k].at, runs[k].bytes)) return true;
    return false;
}
inline bool misaligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

// ------------------------------------------------------------------------------------------ selection

// How a row is cut.  Into as many slices as fill the GPU once (four workgroups of four wavefronts a compute unit, what their registers allow), each of several
// chunks; in a call of few rows into chunks, and these made smaller while compute units are left over.  Long bfloat16 rows (from 65536 entries and 2^23 in all): by
// the kernel with the table, two workgroups of eight wavefronts a compute unit, the slices so many that these have about equally many.  Whole calls with and
// without the table, 16 continuations of 8 beams: 8 sequences of 128256 entries 23.3 and 22.6 us, 12 27.8 and 22.8, 16 27.8 and 25.2, 32 30.1 and 35.0, 64 39.6 and 52.3,
// 128 65.3 and 84.2, 12 of 256000 29.0 and 29.6; shorter rows lose by it (64 of 32000 24.8 and 24.9, 128 37.3 and 34.1, 256 62.2 and 54.8), as each pays for its beginning and end.
// (Of rows of 128256 entries 96 and 128 are taken by the table's kernel and lose by it; the border pays from about 192 on.)
struct BeamShape { int slots, len, S; bool table; };
constexpr long kBeamWGs = 1024, kBeamFew = 512, kTableWGs = 512;
constexpr int kTableSlots = 2;
bool beam_shape(int B, int W, int V, int n, int dtype, BeamShape* s) {
    if (dtype != FSD_F32 && dtype != FSD_BF16) return false;
    if (B < 1 || B > kMaxBatch || W < 1 || W > kBeamWidest || n < 1 || n > kBeamMost || V < 1 || V > fsd_max_vocab(dtype)) return false;
    const int E = dtype == FSD_BF16 ? 8 : 4;
    const long rows = static_cast<long>(B) * W;
    auto chunks = [&](int slots) { return (V + kWG * E * slots - 1) / (kWG * E * slots); };
    s->slots = 4;
    while (s->slots > 1 && rows * chunks(s->slots) < kBeamFew) s->slots /= 2;
    int S = chunks(s->slots);
    s->table = dtype == FSD_BF16 && V >= 65536 && rows * V >= 1L << 23;
    if (s->table) {
        // (slices of 32768 entries at least; beginning and end of one cost about as much as 6000 entries)
        double best = 0.0;
        S = 1;
        for (int k = 1; k <= 8 && V / k >= 32768 && rows * k <= kMaxGroups; ++k) {
            const double cost = static_cast<double>((rows * k + kTableWGs - 1) / kTableWGs) * (static_cast<double>(V) / k + 6000.0);
            if (k == 1 || cost < best) best = cost, S = k;
        }
    } else if (rows * S > kBeamWGs) {
        // two to four workgroups a compute unit, so many slices that the busiest unit has least to do; beginning and end of one cost about as much as this many
        // entries (192 binary32 rows of 128259 entries, n = 60: 2 slices 36.6 us, 4 31.8, 5 33.6, 6 35.9)
        const double ends = 10000.0 + 200.0 * n;
        const int least = static_cast<int>((kBeamWGs / 2 + rows - 1) / rows), most = static_cast<int>(kBeamWGs / rows);
        double best = 0.0;
        S = least;
        for (int k = least; k <= most; ++k) {
            const double cost = static_cast<double>((rows * k + 255) / 256) * (static_cast<double>(V) / k + ends);
            if (k == least || cost < best) best = cost, S = k;
        }
    }
    s->len = ((V + S - 1) / S + E - 1) / E * E;              // slices of one length, so that none of them is a remnant
    s->S = (V + s->len - 1) / s->len;
    // A slice of one slot a thread has no use for more; one of a few goes in smaller chunks where its registers keep other workgroups waiting (3330 rows of 4032 bfloat16
    // entries 34.3 and 24.5 us, 3968 of 5120 76 and 67, 528 of 1152 10.8 and 7.9; 144 rows of 13696 binary32 entries 15.2 and 15.4, 64 of 32000 8.7 and 9.0).
    if (!s->table && s->len <= kWG * E) s->slots = 1;
    else if (!s->table && s->slots > 2 && s->len <= kWG * E * s->slots && rows * s->S > kBeamWGs) s->slots = 2;
    return rows * s->S <= kMaxGroups;
}
struct BeamSpace { size_t lists, stat, cand, bytes; };
// (as much as any call of these or smaller sizes needs, of either type: beam_shape makes at most 1535 slices besides one a row, or of a long bfloat16 row min(8, V / 32768))
BeamSpace beam_space(int B, int W, int V, int n) {
    Space a;
    BeamSpace w;
    const int of_long_row = V < 65536 ? 1 : V / 32768 < 8 ? V / 32768 : 8;
    const size_t lists = w.lists = static_cast<size_t>(B) * W * of_long_row + 1536;
    w.stat = a.take(lists * sizeof(double2));
    w.cand = a.take(lists * n * sizeof(float2));
    w.bytes = a.bytes;
    return w;
}
template <bool BF16>
void launch_beam_slices(hipStream_t st, const BeamShape& s, const BeamParams& P) {
    const dim3 g(P.units), t(kWG);
    if constexpr (BF16) {
        if (s.table) {
            hipLaunchKernelGGL((beam_slices<true, kTableSlots, true>), dim3(P.units < kTableWGs ? P.units : static_cast<unsigned>(kTableWGs)), dim3(512), 0, st, P);
            return;
        }
    }
    if (s.slots == 1) hipLaunchKernelGGL((beam_slices<BF16, 1, false>), g, t, 0, st, P);
    else if (s.slots == 2) hipLaunchKernelGGL((beam_slices<BF16, 2, false>), g, t, 0, st, P);
    else hipLaunchKernelGGL((beam_slices<BF16, 4, false>), g, t, 0, st, P);
}

// ------------------------------------------------------------------------------------------ pages

constexpr int kMostBlocks = 1 << 24;
constexpr long kCopyWGs = 2048;        // workgroups that share the pages' bytes: 8 a compute unit

PagesPair pages_pair(const fsd_cache& a, const fsd_cache& b) {
    PagesPair p;
    p.k_from = static_cast<const char*>(a.k_codes);
    p.v_from = static_cast<const char*>(a.v_codes);
    p.k_to = static_cast<char*>(b.k_codes);
    p.v_to = static_cast<char*>(b.v_codes);
    p.ks_from = a.k_scale;
    p.vs_from = a.v_scale;
    p.ks_to = b.k_scale;
    p.vs_to = b.v_scale;
    p.blocks_from = a.num_blocks;
    p.blocks_to = b.num_blocks;
    p.layers = a.layers;
    p.heads = a.kv_heads;
    p.head_bytes = kBlock * a.head_dim;
    return p;
}
inline size_t codes_bytes(const fsd_cache& c) { return static_cast<size_t>(c.layers) * c.num_blocks * c.kv_heads * kBlock * c.head_dim; }
inline size_t scale_bytes(const fsd_cache& c) { return static_cast<size_t>(c.layers) * c.num_blocks * c.kv_heads * 4; }
inline int chunks_of(int num_blocks) { return (num_blocks + kPagesChunk - 1) / kPagesChunk; }
inline unsigned copy_groups(long units) { return static_cast<unsigned>(units < kCopyWGs ? units : kCopyWGs); }

struct ForkSpace { size_t counts, claim, free_list, free_count, seq, fresh, copies, at, copy_seq, totals, bytes; };
ForkSpace fork_space(int P, int n) {
    Space a;
    ForkSpace w;
    const size_t blocks = static_cast<size_t>(P) * 4, seqs = static_cast<size_t>(n);
    w.counts = a.take(2 * blocks);
    w.claim = a.take(blocks);
    w.free_list = a.take(blocks);
    w.free_count = a.take(static_cast<size_t>(chunks_of(P)) * 4);
    w.seq = a.take(seqs * sizeof(int4));
    w.fresh = a.take(seqs * 4);
    w.copies = a.take(seqs * 4);
    w.at = a.take(seqs * sizeof(int2));
    w.copy_seq = a.take(seqs * 4);
    w.totals = a.take(12);
    w.bytes = a.bytes;
    return w;
}
struct CompactSpace { size_t used_count, number, from, to, count, totals, bytes; };
CompactSpace compact_space(int P) {
    Space a;
    CompactSpace w;
    const size_t half = (static_cast<size_t>(P) / 2 + 1) * 4;
    w.used_count = a.take(static_cast<size_t>(chunks_of(P)) * 4);
    w.number = a.take(static_cast<size_t>(P) * 4);
    w.from = a.take(half);
    w.to = a.take(half);
    w.count = a.take(half);
    w.totals = a.take(8);
    w.bytes = a.bytes;
    return w;
}
bool fork_sizes(int P, int n) { return P >= 1 && P <= kMostBlocks && n >= 1 && n <= kMaxBatch; }

}  // namespace

extern "C" {

size_t fsd_beam_workspace_bytes(int B, int beams, int V, int n, int dtype) {
    BeamShape s;
    return beam_shape(B, beams, V, n, dtype, &s) ? beam_space(B, beams, V, n).bytes : 0;
}

int fsd_beam_select(const void* logits, int64_t row_stride, const float* scores, const float* weights, const int32_t* done, int B, int beams, int V, int dtype,
                    int n, float* scores_out, int32_t* parent, int32_t* tokens, int32_t* row_status, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!logits || !scores_out || !parent || !tokens) return FSD_ERR_NULL;
    if (dtype != FSD_F32 && dtype != FSD_BF16) return FSD_ERR_DTYPE;
    BeamShape s;
    if (!beam_shape(B, beams, V, n, dtype, &s)) return FSD_ERR_SHAPE;
    const size_t es = dtype == FSD_BF16 ? 2 : 4, in = static_cast<size_t>(B) * beams * 4, out = static_cast<size_t>(B) * n * 4;
    if (row_stride < V || row_stride > (1L << 32) || reinterpret_cast<uintptr_t>(logits) % es != 0 || misaligned4(scores) || misaligned4(weights) ||
        misaligned4(done) || misaligned4(scores_out) || misaligned4(parent) || misaligned4(tokens) || misaligned4(row_status))
        return FSD_ERR_LAYOUT;
    const BeamSpace w = beam_space(B, beams, V, n);
    if (!workspace_fits(workspace, workspace_bytes, w.bytes)) return FSD_ERR_WORKSPACE;
    if (static_cast<size_t>(B) * beams * s.S > w.lists) return FSD_ERR_SHAPE;   // (never)
    const size_t read = (static_cast<size_t>(B) * beams - 1) * static_cast<size_t>(row_stride) * es + static_cast<size_t>(V) * es;
    const Run runs[] = {{scores_out, out}, {parent, out}, {tokens, out}, {row_status, static_cast<size_t>(B) * 4}, {workspace, w.bytes},
                        {scores, in}, {weights, in}, {done, in}, {logits, read}};
    if (any_overlap(runs, 5, 9)) return FSD_ERR_LAYOUT;
    char* base = static_cast<char*>(workspace);
    BeamParams P;
    P.logits = static_cast<const char*>(logits);
    P.row_stride = static_cast<size_t>(row_stride) * es;
    P.scores = scores;
    P.weights = weights;
    P.done = done;
    P.B = B; P.W = beams; P.V = V; P.n = n;
    P.len = s.len; P.S = s.S; P.lists = beams * s.S;
    P.by_S = s.S == 1 ? 0u : static_cast<unsigned>(((1ul << 32) + s.S - 1) / s.S);
    P.stat = reinterpret_cast<double2*>(base + w.stat);
    P.cand = reinterpret_cast<float2*>(base + w.cand);
    P.scores_out = scores_out;
    P.parent = parent;
    P.tokens = tokens;
    P.status = row_status;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    P.units = static_cast<unsigned>(static_cast<long>(B) * P.lists);
    if (dtype == FSD_BF16) launch_beam_slices<true>(st, s, P);
    else launch_beam_slices<false>(st, s, P);
    const dim3 sequences(static_cast<unsigned>(B));
    // A round of the merge takes the first entries of all lists, and it is over where a round reaches nothing.  One beam that has all of the best has n / S of them in
    // each of its lists, so rounds of n * beams entries and a third hold what counts; longer ones cost as many registers and instructions where lists are few.  256 threads of
    // 4 entries, 512 of 4 and 512 of 16, by n * beams: 32: 5.5, 5.8, 8.1 us; 128: 6.3, 6.5, 9.1; 720: 9.2, 11.6, 13.4; 960: 16.6, 13.9, 23.0; 2376: 23.3, 16.7, 24.0;
    // 3840: 219, 18.4, 23.5; 8192: 669, 36.0, 25.2; 25600: 57, 35.4, 25.7.
    const long deep = static_cast<long>(n) * beams;
    if (P.lists * n <= 256 * 4 || (deep * 4 / 3 <= 256 * 4 && P.lists <= 512)) hipLaunchKernelGGL((beam_merge<256, 4>), sequences, dim3(256), 0, st, P);
    else if (deep <= 2 * 512 * 4 && P.lists <= 1024) hipLaunchKernelGGL((beam_merge<512, 4>), sequences, dim3(512), 0, st, P);
    else hipLaunchKernelGGL((beam_merge<512, 16>), sequences, dim3(512), 0, st, P);
    return launched();
}

int fsd_beam_reorder(const void* states, const int32_t* parent, int layers, int B, int beams, int n, size_t row_bytes, void* out, int32_t* row_status,
                     void* hip_stream) {
    if (!states || !parent || !out) return FSD_ERR_NULL;
    if (layers < 1 || layers > 65535 || B < 1 || B > kMaxBatch || beams < 1 || beams > 65535 || n < 1 || n > 65535 || row_bytes < 1 || row_bytes > (1ul << 40))
        return FSD_ERR_SHAPE;
    const long pairs = static_cast<long>(layers) * B, rows = pairs * n;
    if (pairs * (beams > n ? beams : n) >= (1L << 31)) return FSD_ERR_SHAPE;
    if (misaligned4(parent) || misaligned4(row_status)) return FSD_ERR_LAYOUT;
    ReorderParams P;
    P.pieces = static_cast<int>((row_bytes + kReorderPiece - 1) / kReorderPiece);
    // (rows of 2^40 bytes are 2^26 pieces: the product is in range; whether the bytes are is the memory's matter)
    P.units = rows * P.pieces;
    const unsigned __int128 in_bytes = static_cast<unsigned __int128>(row_bytes) * pairs * beams, out_bytes = static_cast<unsigned __int128>(row_bytes) * rows;
    if ((in_bytes >> 62) != 0 || (out_bytes >> 62) != 0) return FSD_ERR_SHAPE;
    const Run runs[] = {{out, static_cast<size_t>(out_bytes)}, {row_status, static_cast<size_t>(B) * 4}, {states, static_cast<size_t>(in_bytes)},
                        {parent, static_cast<size_t>(B) * n * 4}};
    if (any_overlap(runs, 2, 4)) return FSD_ERR_LAYOUT;
    P.states = static_cast<const char*>(states);
    P.parent = parent;
    P.out = static_cast<char*>(out);
    P.status = row_status;
    P.row = row_bytes;
    P.rows = rows;
    P.B = B; P.W = beams; P.n = n;
    const long most = 1L << 20;
    hipLaunchKernelGGL(beam_reorder, dim3(static_cast<unsigned>(P.units < most ? P.units : most)), dim3(kWG), 0, static_cast<hipStream_t>(hip_stream), P);
    return launched();
}

size_t fsd_cache_fork_workspace_bytes(int num_blocks, int n) { return fork_sizes(num_blocks, n) ? fork_space(num_blocks, n).bytes : 0; }

int fsd_cache_fork(const fsd_cache* cache, int B, const int32_t* refs, const int32_t* parent, const int32_t* lengths, const int32_t* room, int n,
                   int32_t* block_table_out, int32_t* cache_len_out, int32_t* refs_out, int32_t* free_blocks, int32_t* row_status, void* workspace,
                   size_t workspace_bytes, void* hip_stream) {
    if (!refs || !parent || !block_table_out || !cache_len_out || !refs_out) return FSD_ERR_NULL;
    const int bad = check_cache(cache);
    if (bad != FSD_OK) return bad;
    const fsd_cache& c = *cache;
    if (B < 1 || B > kMaxBatch || !fork_sizes(c.num_blocks, n) || static_cast<long>(n) * c.max_blocks >= INT_MAX) return FSD_ERR_SHAPE;
    if (misaligned4(refs) || misaligned4(parent) || misaligned4(lengths) || misaligned4(room) || misaligned4(block_table_out) || misaligned4(cache_len_out) ||
        misaligned4(refs_out) || misaligned4(free_blocks) || misaligned4(row_status) || misaligned4(c.block_table) || misaligned4(c.cache_len))
        return FSD_ERR_LAYOUT;
    const ForkSpace w = fork_space(c.num_blocks, n);
    if (!workspace_fits(workspace, workspace_bytes, w.bytes)) return FSD_ERR_WORKSPACE;
    const size_t per = static_cast<size_t>(c.max_blocks) * 4, seqs = static_cast<size_t>(n) * 4, blocks = static_cast<size_t>(c.num_blocks) * 4;
    const Run runs[] = {{block_table_out, n * per}, {cache_len_out, seqs}, {free_blocks, 4}, {row_status, seqs}, {workspace, w.bytes}, {refs_out, blocks},
                        {refs_out == refs ? nullptr : refs, blocks}, {parent, seqs}, {lengths, seqs}, {room, seqs}, {c.block_table, B * per},
                        {c.cache_len, static_cast<size_t>(B) * 4}, {c.k_codes, codes_bytes(c)}, {c.v_codes, codes_bytes(c)}, {c.k_scale, scale_bytes(c)},
                        {c.v_scale, scale_bytes(c)}};
    if (any_overlap(runs, 6, 16)) return FSD_ERR_LAYOUT;
    char* base = static_cast<char*>(workspace);
    auto ints = [base](size_t at) { return reinterpret_cast<int*>(base + at); };
    ForkParams P;
    P.table = c.block_table;
    P.lens = c.cache_len;
    P.parent = parent;
    P.keep = lengths;
    P.room = room;
    P.refs = refs;
    P.B = B; P.M = c.max_blocks; P.P = c.num_blocks; P.n = n;
    P.table_out = block_table_out;
    P.len_out = cache_len_out;
    P.refs_out = refs_out;
    P.free_out = free_blocks;
    P.status = row_status;
    P.counts = reinterpret_cast<unsigned long*>(base + w.counts);
    P.claim = ints(w.claim);
    P.free_list = ints(w.free_list);
    P.free_count = ints(w.free_count);
    P.seq = reinterpret_cast<int4*>(base + w.seq);
    P.fresh = ints(w.fresh);
    P.copies = ints(w.copies);
    P.at = reinterpret_cast<int2*>(base + w.at);
    P.copy_seq = ints(w.copy_seq);
    P.totals = ints(w.totals);
    P.pair = pages_pair(c, c);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const int chunks = chunks_of(P.P);
    const dim3 t(kWG);
    const unsigned movers = copy_groups(static_cast<long>(n) * c.layers * c.kv_heads);
    if (P.P <= kSmallBlocks && n <= kSmallWG && (static_cast<long>(B) + n) * P.M <= kSmallPlaces) {
        hipLaunchKernelGGL(fork_small, dim3(1), dim3(kSmallWG), 0, st, P);
        hipLaunchKernelGGL(fork_move, dim3(movers), t, 0, st, P);
        return launched();
    }
    const long clear = (static_cast<long>(P.P) + kWG - 1) / kWG;
    hipLaunchKernelGGL(fork_clear, dim3(static_cast<unsigned>(clear < 2048 ? clear : 2048)), t, 0, st, P);
    hipLaunchKernelGGL(fork_mark, dim3(static_cast<unsigned>(B + n)), t, 0, st, P);
    hipLaunchKernelGGL(fork_count, dim3(static_cast<unsigned>(chunks + (n + kWG / 64 - 1) / (kWG / 64))), t, 0, st, P, chunks);
    hipLaunchKernelGGL(fork_list, dim3(static_cast<unsigned>(chunks + (n + kWG - 1) / kWG)), t, 0, st, P, chunks);
    hipLaunchKernelGGL(fork_apply, dim3(static_cast<unsigned>(chunks + n) + movers), t, 0, st, P, chunks);
    return launched();
}

int fsd_cache_copy(const fsd_cache* src, const fsd_cache* dst, const int32_t* src_blocks, const int32_t* dst_blocks, const int32_t* tokens, int n,
                   int32_t* page_status, void* hip_stream) {
    if (!src_blocks || !dst_blocks) return FSD_ERR_NULL;
    int bad = check_cache(src);
    if (bad == FSD_OK) bad = check_cache(dst);
    if (bad != FSD_OK) return bad;
    if (n < 1 || src->layers != dst->layers || src->kv_heads != dst->kv_heads || src->head_dim != dst->head_dim) return FSD_ERR_SHAPE;
    const long units = static_cast<long>(n) * src->layers;   // (times heads: under 2^31 * 2^31)
    if (units >= (1L << 40) / src->kv_heads) return FSD_ERR_SHAPE;
    const size_t list = static_cast<size_t>(n) * 4;
    const bool one = src->k_codes == dst->k_codes && src->v_codes == dst->v_codes && src->k_scale == dst->k_scale && src->v_scale == dst->v_scale &&
                     src->num_blocks == dst->num_blocks;
    const Run runs[] = {{dst->k_codes, codes_bytes(*dst)}, {dst->v_codes, codes_bytes(*dst)}, {dst->k_scale, scale_bytes(*dst)}, {dst->v_scale, scale_bytes(*dst)},
                        {page_status, list}, {src_blocks, list}, {dst_blocks, list}, {tokens, list},
                        {one ? nullptr : src->k_codes, codes_bytes(*src)}, {one ? nullptr : src->v_codes, codes_bytes(*src)},
                        {one ? nullptr : src->k_scale, scale_bytes(*src)}, {one ? nullptr : src->v_scale, scale_bytes(*src)}};
    if (any_overlap(runs, 5, 12) || misaligned4(src_blocks) || misaligned4(dst_blocks) || misaligned4(tokens) || misaligned4(page_status)) return FSD_ERR_LAYOUT;
    CopyParams P;
    P.pair = pages_pair(*src, *dst);
    P.from = src_blocks;
    P.to = dst_blocks;
    P.tokens = tokens;
    P.status = page_status;
    P.n = n;
    P.units = units * src->kv_heads;
    const long most = 1L << 20;
    hipLaunchKernelGGL(pages_copy, dim3(static_cast<unsigned>(P.units < most ? P.units : most)), dim3(kWG), 0, static_cast<hipStream_t>(hip_stream), P);
    return launched();
}

size_t fsd_cache_compact_workspace_bytes(int num_blocks) { return fork_sizes(num_blocks, 1) ? compact_space(num_blocks).bytes : 0; }

int fsd_cache_compact(const fsd_cache* cache, int B, const int32_t* refs, int32_t* block_table_out, int32_t* refs_out, int32_t* remap, int32_t* used_blocks,
                      int32_t* row_status, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!refs || !block_table_out || !refs_out) return FSD_ERR_NULL;
    const int bad = check_cache(cache);
    if (bad != FSD_OK) return bad;
    const fsd_cache& c = *cache;
    if (B < 1 || B > kMaxBatch || !fork_sizes(c.num_blocks, 1)) return FSD_ERR_SHAPE;
    if (misaligned4(refs) || misaligned4(block_table_out) || misaligned4(refs_out) || misaligned4(remap) || misaligned4(used_blocks) || misaligned4(row_status) ||
        misaligned4(c.block_table))
        return FSD_ERR_LAYOUT;
    const CompactSpace w = compact_space(c.num_blocks);
    if (!workspace_fits(workspace, workspace_bytes, w.bytes)) return FSD_ERR_WORKSPACE;
    const size_t table = static_cast<size_t>(B) * c.max_blocks * 4, blocks = static_cast<size_t>(c.num_blocks) * 4;
    const Run runs[] = {{remap, blocks}, {used_blocks, 4}, {row_status, static_cast<size_t>(B) * 4}, {workspace, w.bytes}, {block_table_out, table}, {refs_out, blocks},
                        {block_table_out == c.block_table ? nullptr : c.block_table, table}, {refs_out == refs ? nullptr : refs, blocks},
                        {c.k_codes, codes_bytes(c)}, {c.v_codes, codes_bytes(c)}, {c.k_scale, scale_bytes(c)}, {c.v_scale, scale_bytes(c)}};
    if (any_overlap(runs, 6, 12)) return FSD_ERR_LAYOUT;
    char* base = static_cast<char*>(workspace);
    auto ints = [base](size_t at) { return reinterpret_cast<int*>(base + at); };
    CompactParams P;
    P.table = c.block_table;
    P.refs = refs;
    P.B = B; P.M = c.max_blocks; P.P = c.num_blocks;
    P.table_out = block_table_out;
    P.refs_out = refs_out;
    P.remap = remap;
    P.used_out = used_blocks;
    P.status = row_status;
    P.used_count = ints(w.used_count);
    P.number = ints(w.number);
    P.from = ints(w.from);
    P.to = ints(w.to);
    P.count = ints(w.count);
    P.totals = ints(w.totals);
    P.pair = pages_pair(c, c);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const int chunks = chunks_of(P.P);
    const dim3 t(kWG);
    const unsigned movers = copy_groups(static_cast<long>(c.num_blocks / 2 + 1) * c.layers * c.kv_heads);
    if (P.P <= kSmallBlocks && B <= kSmallWG && static_cast<long>(B) * P.M <= kSmallPlaces) {
        hipLaunchKernelGGL(compact_small, dim3(1), dim3(kSmallWG), 0, st, P);
        hipLaunchKernelGGL(compact_move, dim3(movers), t, 0, st, P);
        return launched();
    }
    hipLaunchKernelGGL(compact_count, dim3(static_cast<unsigned>(chunks)), t, 0, st, P);
    hipLaunchKernelGGL(compact_list, dim3(static_cast<unsigned>(chunks)), t, 0, st, P, chunks);
    hipLaunchKernelGGL(compact_apply, dim3(static_cast<unsigned>(chunks + B) + movers), t, 0, st, P, chunks);
    return launched();
}

}  // extern "C"
