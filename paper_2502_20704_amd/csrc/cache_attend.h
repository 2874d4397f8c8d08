// Attention of a step's rows over the 8-bit paged cache and over one another (fsd_attend_*).
// Part of libfsd (gfx950); included by operators.hip, which holds the host side and the C ABI.
//
//   out_r = sum_t w_t v_t / sum_t w_t,  w_t = exp(scale q_r . k_t),  over the cached tokens and the rows that row r sees
//
// One pass over the cache with a running maximum and sum.  The rows of one key head (tokens x query heads of its
// group) are the columns of the matrix instruction (16x16x32, binary16 operands, binary32 sums); a wavefront takes 16 RT
// of them and goes over cache blocks of 64 tokens:
//   S' = K Q'    4 tiles of 16 tokens; the key bytes go from memory to registers (16 bytes a lane and load, 64 contiguous
//                bytes a token) and are widened there: e4m3 to binary16 is exact, so a block's scale stays outside
//   P  = exp2    of S' times the row's and the block's scales.  Token 16 g + 4 s + i of the block is row 4 g + i of tile s: a lane
//                of group g then holds the 16 weights of its group's tokens, which is what the second product wants
//                as its operand: the weights never change lanes
//   O' += V' P   V' is the block's values with the token index running fastest, as the cache holds them
// The order of a head's dimensions inside the products is as free as that of the tokens: lane group g takes dimensions
// 64 i + 16 g .. + 15 of queries and keys alike.
//
// A block's value scale enters the weights' exponent: p = exp2(s + log2(vs) - m), with m the running maximum of s + log2(vs), and
// sum += p / vs.  So p is at most 2^15 whatever the scales are (binary16 holds it), codes enter the product exactly,
// and O' / sum is the result.  m is kept 7 below the maximum, so that weights lose less at binary16's small end (2^-25 absolutely, beside 2^7), and
// follows only where the maximum is more than 15 above it: a rescaling of O' is rare.  A block whose value scale is far below one before
// it (values that are all zero have the smallest scale there is) may add nothing to O' and yet much to the sum: there the sum takes exp2(s - m) itself.
//
// The rows' own values are held in binary16 in units of that kind: of a tile of 64 rows, or of each row where the rows of a tile differ in size by more
// than 2^6, as a result must not lose bits beside values that its row does not see.
//
// Kernels: attend_prepare turns queries and the rows' keys, brings them and the rows' values into binary16's range by powers of two and lays them
// out in the workspace as the matrix instruction takes them, so that no piece of the work does this again; it deals out the work, which takes the
// lengths, and reports the sequences.  attend_few (few rows a key head) or attend_rows is the pass over cache and rows: every workgroup gets the same number of
// blocks, whichever sequences and heads they belong to.  attend_join puts together what lies across the border of two workgroups.
//
// Measured (us; e4m3 cache, head_dim 128, 8 key heads and 32 heads unless said, bfloat16):
//   1 sequence of 2048 tokens, 1 row             prepare  5.2  few    8  join  4   three kernels' starts and ends, each one chain of requests
//   64 of up to 8192, 9 rows                             14          147        7.5 memory and the barrier a block: 4.2 TB/s of a read's 5.8
//   2 of up to 131072, 5 rows, 28 on 4, binary16           8.7         63        6   the same, 4.0 TB/s; products twice, in two parts
//   32 of up to 4096, trees of 61 rows                   18.5  rows  132       14.5 a wavefront's chain of products, weights and sums, one block after the other:
//                                                                                 the matrix unit works 34 % of the time, vector instructions 52 %; with
//                                                                                 244 of 256 rows in use, 580 TFLOP/s
//   3 of up to 7000, 1000 rows, 16 on 16, head_dim 64    11.7         81-98     7.5 the same, 25 and 55 %
#ifndef FSD_CSRC_CACHE_ATTEND_H_
#define FSD_CSRC_CACHE_ATTEND_H_

#include "operators_common.h"

namespace {

typedef float float2_t __attribute__((ext_vector_type(2)));

constexpr float kRoom = 7.0f;      // powers of two that a weight formed anew is above 1
constexpr float kLazy = 15.0f;     // how far (likewise) weights may pass 1 before they are scaled down again
constexpr float kUnit = 10.0f;     // sums are in units of 2^10: value scales from 2^-100 on leave room for 2^22 tokens, those up to 2^119 do not vanish
constexpr float kPerUnit = 0x1p-10f;
constexpr int kLeast = 100;        // units of the rows' values are 2^-100 to 2^119
constexpr float kNarrow = 0x1p-6f; // a tile's values have one unit where the smallest row (its largest magnitude) is no further below the largest
constexpr float kLog2eF = 1.44269504088896340736f;

struct AttendParams {
    const void* q;
    const void* k;
    const void* v;
    long q_stride, kv_stride;
    const int32_t* parent;         // [B, R-1], trees
    const int32_t* row_count;
    int B, R, heads, G;            // G: query heads of a key head
    int dtype;
    float scale;                   // times log2(e)
    fsd_rotation rot;
    fsd_cache cache;
    int layer;
    void* out;
    int32_t* status;
    int workers;                   // workgroups of attend_rows
    int tile;                      // rows of an item
    int row_tiles;                 // of 16 rows, of a (sequence, key head): whole items
    int tiles;                     // of 64 tokens of the R rows
    unsigned by_heads, by_G, by_tile;   // for dividing by heads, G and tile
    // workspace
    long* plan;                    // [0] units of a workgroup, [1 + b] units of the sequences before b
    int2* pieces;                  // [B, kv_heads, groups] of an item: its first slot, and how many workers share it
    float* factor;                 // [B, kv_heads, row_tiles * 16] of the products of a row: its power of two back, scale, log2(e)
    float* key_scale;              // [B, kv_heads, tiles, 64]
    int* value_lift;               // [B, kv_heads, tiles] log2 of what a tile's values are in units of, plus kLeast; -1: each row's are in units of their own
    unsigned char* row_lift;       // [B, kv_heads, tiles, 64] these, where they are
    unsigned long long* broken;    // [B, kv_heads, tiles] tokens of a tile with a value that is not finite
    unsigned long long* sees;      // [B, R, tiles] trees: tokens of a tile that a row sees
    char* q16;                     // [B, kv_heads, row_tiles, 2 * (D / 64)] fragments of 1 KB; binary16 inputs: second parts behind them
    char* k16;                     // [B, kv_heads, tiles, 4 * 2 * (D / 64)] fragments; second parts likewise
    char* v16;                     // [B, kv_heads, tiles, 2 * (D / 16)] fragments
    float* part;                   // results of pieces: two slots a worker, [rows of an item][D], then [rows][2] each
};

// The work is a line of units.  An item is one (sequence, key head, run of `tile` rows); its units are the blocks of the sequence's
// cache, then its tiles of 64 rows; kStart more stand for what an item costs at its beginning, whoever begins it.
// (64 sequences of 300 to 2048 tokens, 8 key heads: 211 us with 3, 205 with 6, 201 with 10; 25-row trees: best with 3 to 6.)
constexpr int kStart = 6;
struct Share { int rows, blocks, tiles, groups; };
__device__ __forceinline__ Share share_of(const AttendParams& P, int b) {
    Share s;
    const int most = P.cache.max_blocks * kBlock;
    s.rows = P.row_count ? max(0, min(P.row_count[b], P.R)) : P.R;
    s.blocks = (max(0, min(P.cache.cache_len[b], most)) + kBlock - 1) / kBlock;
    s.tiles = (s.rows + kBlock - 1) / kBlock;
    s.groups = (s.rows * P.G + P.tile - 1) / P.tile;
    return s;
}
__device__ __forceinline__ int units_of(const Share& s) { return kStart + s.blocks + s.tiles; }          // of an item
__device__ __forceinline__ long units_of_sequence(const AttendParams& P, const Share& s) {
    return static_cast<long>(units_of(s)) * s.groups * P.cache.kv_heads;
}

// Deals the line out: every worker takes `per` units in a row, so that all have the same.  A workgroup's work.
__device__ __forceinline__ void deal(const AttendParams& P) {
    __shared__ long sums[kWG / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    long base = 0;
    for (int b0 = 0; b0 < P.B; b0 += kWG) {
        const int b = b0 + tid;
        const long n = b < P.B ? units_of_sequence(P, share_of(P, b)) : 0l;
        long up = n;                                          // inclusive sum over the wavefront
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long y = __shfl_up(up, o, 64);
            if (lane >= o) up += y;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = up;
        __syncthreads();
        long first = base + up - n;
        for (int i = 0; i < wave; ++i) first += sums[i];
        if (b < P.B) P.plan[1 + b] = first;
        for (int i = 0; i < kWG / 64; ++i) base += sums[i];
    }
    if (tid == 0) {
        const long per = (base + P.workers - 1) / P.workers;
        P.plan[0] = per < 1 ? 1 : per;
        P.plan[1 + P.B] = base;
    }
}

// n / d for n d < 2^32, with by = ceil(2^32 / d).  (The division that the compiler writes out is 30 instructions, and the kernels around the products
// are bound by theirs.)
__device__ __forceinline__ int divided(int n, int d, unsigned by) { return d == 1 ? n : static_cast<int>(__umulhi(static_cast<unsigned>(n), by)); }

__device__ __forceinline__ half8_t widened(unsigned lo, unsigned hi) {
    half8_t r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const half2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(i ? hi : lo, 1.0f, false);
        const half2_t b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(i ? hi : lo, 1.0f, true);
        r[4 * i] = a.x; r[4 * i + 1] = a.y; r[4 * i + 2] = b.x; r[4 * i + 3] = b.y;
    }
    return r;
}
// (the type of queries, keys, values and results matters at both ends of a piece only: it is no template argument)
__device__ __forceinline__ void store4(int dtype, void* base, size_t at, const float4_t& x) {
    uint2 w;
    if (dtype == FSD_BF16) {
        w.x = bf16_bits(x[0]) | bf16_bits(x[1]) << 16;
        w.y = bf16_bits(x[2]) | bf16_bits(x[3]) << 16;
    } else {
        auto two = [](float a, float b) {
            half2_t h;
            h.x = static_cast<_Float16>(a);
            h.y = static_cast<_Float16>(b);
            return __builtin_bit_cast(unsigned, h);
        };
        w.x = two(x[0], x[1]);
        w.y = two(x[2], x[3]);
    }
    *reinterpret_cast<uint2*>(static_cast<unsigned short*>(base) + at) = w;
}
__device__ __forceinline__ float byte_of(unsigned w, int i) { return static_cast<float>(w >> (8 * i) & 0xFFu); }   // (one instruction)
// maximum over the four lanes that hold one column
__device__ __forceinline__ float column_max(float v) {
    v = __builtin_fmaxf(v, __shfl_xor(v, 16, 64));
    return __builtin_fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float column_sum(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}
// What is relative to 2^from becomes relative to 2^to by this factor's square: a sum of weights may be as large as the step is far (scales of values lie up to
// 2^219 apart), and outlives it only in two halves.
__device__ __forceinline__ float back_from(float from, float to) {
    return to == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(0.5f * (from - to));
}
// the power of two that brings `most` into [2^at, 2 * 2^at), as an exponent
__device__ __forceinline__ int to_half_range(float most, int at, int limit) { return min(at + 127 - static_cast<int>(__float_as_uint(most) >> 23), limit); }
// queries and keys: as large as products allow; values (as an exponent): as large as the cache's codes, so that their scales are alike (nothing but zeros
// gets the smallest unit there is, as in the cache)
__device__ __forceinline__ float key_range(float most) { return most > 0.0f ? pow2(to_half_range(most, 13, 126)) : 1.0f; }
__device__ __forceinline__ int value_range(float most) { return to_half_range(most, 8, kLeast); }
// maximum over the 16 lanes of a row, in all of them: lanes 1 and 2 apart, then mirrored in halves and as a whole
__device__ __forceinline__ float row_max(float v) {
    auto other = [&](auto ctrl) {
        return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    v = __builtin_fmaxf(v, other(std::integral_constant<int, 0xB1>()));
    v = __builtin_fmaxf(v, other(std::integral_constant<int, 0x4E>()));
    v = __builtin_fmaxf(v, other(std::integral_constant<int, 0x141>()));
    return __builtin_fmaxf(v, other(std::integral_constant<int, 0x140>()));
}

constexpr int kMaxNodes = 2048;
constexpr int kWalk = 256;          // nodes of trees whose depths are found by walking

__device__ __forceinline__ int not_kept(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// The value is in its register from here on: the compiler waits for what it has requested here, and not in a loop behind, where it
// would wait for the fetches as well.
template <typename T>
__device__ __forceinline__ void settle(T& x) {
    asm volatile("" : "+v"(x));
}

// ---- blocks come to LDS without passing through registers: a lane's 16 bytes of a fragment land at 16 * lane of its 1 KB, and
// the same lane (or the same lane of another wavefront) reads them back, so that nothing is exchanged between lanes

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ unsigned lds_address(const unsigned char* p) {
    return static_cast<unsigned>(reinterpret_cast<uintptr_t>((const lds_void*)(p)));
}
// from: this lane's 16 bytes; to: the same for all lanes.  (In assembly, as the reads below, because the compiler would have every access of
// LDS wait for every fetch in flight.  What it counts itself is less than what there is: its own waits are long enough.)
__device__ __forceinline__ void fetch_1k(const char* from, const unsigned char* to) {
    asm volatile("s_mov_b32 m0, %1\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, off"
                 :: "v"(from), "s"(__builtin_amdgcn_readfirstlane(static_cast<int>(lds_address(to)))) : "memory", "m0");
}
// four fragments 1 KB apart
__device__ __forceinline__ void read_4k(unsigned at, u32x4 (&w)[4]) {
    asm volatile("ds_read_b128 %0, %4\n\t"
                 "ds_read_b128 %1, %4 offset:1024\n\t"
                 "ds_read_b128 %2, %4 offset:2048\n\t"
                 "ds_read_b128 %3, %4 offset:3072\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]) : "v"(at) : "memory");
}
__device__ __forceinline__ void read_2k(unsigned at, u32x4 (&w)[2]) {
    asm volatile("ds_read_b128 %0, %2\n\t"
                 "ds_read_b128 %1, %2 offset:1024\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(w[0]), "=&v"(w[1]) : "v"(at) : "memory");
}
__device__ __forceinline__ void read_1k(unsigned at, u32x4& w) {
    asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(w) : "v"(at) : "memory");
}
template <int N, int M>
__device__ __forceinline__ void read_some(unsigned at, u32x4 (&w)[M]) {
    static_assert((N == 1 || N == 2 || N == 4) && N <= M, "fragments");
    if constexpr (N == 1) read_1k(at, w[0]);
    else if constexpr (N == 2) read_2k(at, reinterpret_cast<u32x4(&)[2]>(w));
    else read_4k(at, reinterpret_cast<u32x4(&)[4]>(w));
}
// A barrier that leaves fetches under way: what the wavefronts exchange goes through LDS by ordinary stores.
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// waits until at most N of this wavefront's fetches are under way
template <int N>
__device__ __forceinline__ void wait_fetches() {
    static_assert(N < 64, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// a b + c, with b given in two parts where FINE
template <bool FINE>
__device__ __forceinline__ float4_t product(const half8_t& a, const half8_t& b, const half8_t& b2, float4_t c) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    if constexpr (FINE) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b2, c, 0, 0, 0);
    return c;
}
// y times a power of two in binary16: the first part, and with FINE what is left in a second
template <bool FINE>
__device__ __forceinline__ void two_parts(const float (&y)[8], float by, half8_t& a, half8_t& c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float z = y[e] * by;
        a[e] = static_cast<_Float16>(z);
        if constexpr (FINE) c[e] = static_cast<_Float16>(z - static_cast<float>(a[e]));
    }
}

// Queries and the rows' keys and values in the layout of the products; the plan; the sequences' reports.  Grid: pieces of work, sequences.  The first workgroup
// deals the work out; of the others each belongs to one sequence and takes some query rows, or keys or values of one tile of 64 rows of a key head.  What it costs is latencies: everything a thread reads
// is requested at once, and nothing changes places between threads.
// FINE (binary16 inputs): a turned query or key is held in two parts of 11 bits, as one rounding of them would cost more than that of the result:
// 0.00047 of the result's norm in place of 0.00027 at 131072 tokens.
template <int D, bool FINE>
__global__ __launch_bounds__(kWG) void attend_prepare(AttendParams P) {
    constexpr int kType = FINE ? FSD_F16 : FSD_BF16, kI = D / 64, kPer = D / 8, kThreads = kWG;
    __shared__ __align__(16) float most_of[2][kBlock];
    __shared__ unsigned long long broken;
    extern __shared__ short tree[];                           // trees: [R] parent's row, [R] depth, [R] ancestors found so far
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (blockIdx.x == 0) {
        if (blockIdx.y == 0) deal(P);
        return;
    }
    const int H = P.cache.kv_heads, R = P.R, G = P.G, all_tiles = H * P.tiles * (kI + 1), at_block = static_cast<int>(blockIdx.x) - 1;
    const bool is_tile = at_block < all_tiles;                // (tiles first: they take longest)
    const int b = static_cast<int>(blockIdx.y);
    const Share share = share_of(P, b);
    const int len = max(0, min(P.cache.cache_len[b], P.cache.max_blocks * kBlock));
    short* up = tree;
    short* depth = tree + R;
    short* stands = tree + 2 * R;
    bool bad_tree = false;
    const bool deep = P.parent && R - 1 > kWalk;              // paths may be too long to walk up for every row
    if (P.parent) {
        const int32_t* parent = P.parent + static_cast<size_t>(b) * (R - 1);
        for (int r = tid; r < R; r += kThreads) {
            int p = -1;                                       // row 0 has none, and those behind the sequence's last row are not looked at
            if (r > 0 && r < share.rows) {
                p = parent[r - 1];
                const bool bad = p < -1 || p >= r - 1;
                bad_tree |= bad;
                p = bad ? 0 : p + 1;
            }
            up[r] = static_cast<short>(p);
        }
        __syncthreads();
    }
    if (deep) {
        // in deep ones by doubling: after step i a row knows its 2^i-th ancestor and how far that is
        for (int r = tid; r < R; r += kThreads) {
            stands[r] = up[r];
            depth[r] = up[r] >= 0 ? 1 : 0;
        }
        __syncthreads();
        for (;;) {
            constexpr int kEach = (kMaxNodes + kThreads) / kThreads;
            short jump[kEach], more[kEach];
            bool moved = false;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = tid + i * kThreads, p = r < R ? stands[r] : -1;
                jump[i] = p > 0 ? stands[p] : static_cast<short>(-1);
                more[i] = p > 0 ? depth[p] : static_cast<short>(0);
                moved |= p > 0;
            }
            if (!__syncthreads_or(moved)) break;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = tid + i * kThreads;
                if (r >= R) continue;
                depth[r] = static_cast<short>(depth[r] + more[i]);
                stands[r] = jump[i];
            }
            __syncthreads();
        }
    }
    // (a cache of nearly 2^31 tokens and the rows behind it: more than an int holds)
    auto position = [&](int r) -> unsigned {
        const unsigned n = static_cast<unsigned>(len);
        if (!P.parent) return n + static_cast<unsigned>(r);
        if (deep) return n + static_cast<unsigned>(depth[r]);
        unsigned way = 0;
        for (int at = r; at > 0; at = up[at]) ++way;
        return n + way;
    };
    auto table_row = [&](unsigned pos) { return P.rot.table ? static_cast<int>(min(pos, static_cast<unsigned>(P.rot.rows) - 1u)) : 0; };
    constexpr int kSlots = 2;                                 // rows of which a thread takes 8 dimensions, D / 8 neighbours the whole of a row

    if (!is_tile) {
        const int part = at_block - all_tiles;
        if (part == 0 && P.status) {                          // the sequence's report
            const int32_t* table = P.cache.block_table + static_cast<size_t>(b) * P.cache.max_blocks;
            bool bad = P.cache.cache_len[b] < 0 || P.cache.cache_len[b] > P.cache.max_blocks * kBlock ||
                       (P.row_count && (P.row_count[b] < 0 || P.row_count[b] > R));
            for (int i = tid; i < share.blocks; i += kThreads) bad |= table[i] < 0 || table[i] >= P.cache.num_blocks;
            if (P.rot.table)
                for (int r = tid; r < share.rows; r += kThreads) bad |= position(r) >= static_cast<unsigned>(P.rot.rows);
            bad = __syncthreads_or(bad);
            bad_tree = __syncthreads_or(bad_tree);
            if (tid == 0) P.status[b] = (bad ? FSD_ROW_BAD_CACHE : 0) | (bad_tree ? FSD_ROW_BAD_PARENT : 0);
        }
        const size_t parts = static_cast<size_t>(P.B) * H * P.row_tiles * 2 * kI * 1024;
        const int n = share.rows * P.heads, row0 = part * (kSlots * kThreads / kPer) + tid / kPer, dim = tid % kPer * 8;
        if (row0 >= n) return;
        size_t at[kSlots];
        int dims[kSlots], pos[kSlots], row[kSlots];
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            row[i] = row0 + i * (kThreads / kPer);
            const int there = min(row[i], n - 1), r = divided(there, P.heads, P.by_heads);
            at[i] = (static_cast<size_t>(b) * R + r) * P.q_stride + static_cast<size_t>(there - r * P.heads) * D;
            dims[i] = dim;
            pos[i] = table_row(position(r));
        }
        float y[kSlots][8];
        load_turned<kSlots>(kType, P.q, at, dims, P.rot, pos, y);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, finite_abs(y[i][e]));
#pragma unroll
            for (int o = kPer / 2; o > 0; o >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, o, 64));
            if (row[i] >= n) continue;
            const float by = key_range(most);
            half8_t a, c;
            two_parts<FINE>(y[i], P.scale < 0.0f ? -by : by, a, c);  // (a negative scale goes in here: a larger product is always a larger score)
            const int r = divided(row[i], P.heads, P.by_heads), head = row[i] - r * P.heads, h = divided(head, G, P.by_G), rho = r * G + head - h * G;
            const size_t bh = static_cast<size_t>(b) * H + h, fragment = (bh * P.row_tiles + rho / 16) * 2 * kI + dim / 64 * 2 + (dim / 8 & 1);
            char* to = P.q16 + fragment * 1024 + ((dim / 16 & 3) * 16 + (rho & 15)) * 16;
            *reinterpret_cast<half8_t*>(to) = a;
            if constexpr (FINE) *reinterpret_cast<half8_t*>(to + parts) = c;
            if (dim == 0) P.factor[bh * P.row_tiles * 16 + rho] = __builtin_fabsf(P.scale) / by;
        }
        return;
    }
    // kI workgroups a tile and head for the keys, one for the values
    const int kind = at_block % (kI + 1), tile = at_block / (kI + 1) % P.tiles, h = at_block / (kI + 1) / P.tiles % H, t0 = tile * kBlock, n = min(kBlock, share.rows - t0);
    const size_t bht = (static_cast<size_t>(b) * H + h) * P.tiles + tile, size = static_cast<size_t>(P.B) * H * P.tiles * 8 * kI * 1024;
    const size_t base = (static_cast<size_t>(b) * R + t0) * P.kv_stride + static_cast<size_t>(h) * D;
    if (kind < kI) {
        // keys: every token scaled by a power of two of its own.  (What lies behind the last row is not written: no weight comes of it.)
        const int first = kind * (kBlock / kI) + tid / kPer, dim = tid % kPer * 8;
        if (first >= n) return;
        size_t at[kSlots];
        int dims[kSlots], pos[kSlots];
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            const int t = min(first + i * (kThreads / kPer), n - 1);
            at[i] = base + t * P.kv_stride;
            dims[i] = dim;
            pos[i] = table_row(position(t0 + t));
        }
        float y[kSlots][8];
        load_turned<kSlots>(kType, P.k, at, dims, P.rot, pos, y);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            const int t = first + i * (kThreads / kPer);
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, finite_abs(y[i][e]));
#pragma unroll
            for (int o = kPer / 2; o > 0; o >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, o, 64));
            if (t >= n) continue;
            const float by = key_range(most);
            half8_t a, c;
            two_parts<FINE>(y[i], by, a, c);
            const int fragment = (t >> 2 & 3) * 2 * kI + dim / 64 * 2 + (dim / 8 & 1), place = (dim / 16 & 3) * 16 + (t >> 4) * 4 + (t & 3);
            char* to = P.k16 + bht * (8 * kI * 1024) + fragment * 1024 + place * 16;
            *reinterpret_cast<half8_t*>(to) = a;
            if constexpr (FINE) *reinterpret_cast<half8_t*>(to + size) = c;
            if (dim == 0) P.key_scale[bht * kBlock + t] = 1.0f / by;
        }
        return;
    }
    if (n <= 0) return;
    // values: a thread takes 8 tokens of one dimension, which lie in one of the product's fragments; its tokens are the same in all units
    constexpr int kUnits = kBlock * D / 8 / kThreads;
    unsigned raw[kUnits][4];
    const unsigned short* values = static_cast<const unsigned short*>(P.v) + base;
    const int t = (lane >> 4) * 16 + (wave & 1) * 8;          // the first of them
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int d = (tid + i * kThreads) / 128 * 16 + (lane & 15);
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[i][e] = 0;
        if (t >= n) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned w = values[min(t + e, n - 1) * P.kv_stride + d];   // (behind the last row it comes again, and is blanked)
            raw[i][e / 2] |= (t + e < n ? w : 0u) << (16 * (e & 1));
        }
    }
    // Values are scaled by a power of two, for all rows of the tile where they are of one size, else for each its own: what a row sees must not be lost
    // beside what it does not see.  One that is not finite is noted, as no weight of 0 makes it harmless.  (A row's dimensions lie in 16 lanes of this
    // wavefront and of the one two further.)
    float most[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) most[e] = 0.0f;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        float y[8];
        unpack8(P.dtype, u32x4{raw[i][0], raw[i][1], raw[i][2], raw[i][3]}, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) most[e] = __builtin_fmaxf(most[e], finite_abs(y[e]));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) most[e] = row_max(most[e]);
    if ((lane & 15) == 0) {
#pragma unroll
        for (int e = 0; e < 8; e += 4) *reinterpret_cast<float4_t*>(&most_of[wave >> 1][t + e]) = float4_t{most[e], most[e + 1], most[e + 2], most[e + 3]};
    }
    if (tid == 0) broken = 0;
    __syncthreads();
    const float of_row = __builtin_fmaxf(most_of[0][lane], most_of[1][lane]);
    const float high = column_max(row_max(of_row)), least = -column_max(row_max(of_row > 0.0f ? -of_row : -__builtin_inff()));
    const bool narrow = least >= high * kNarrow;
    float by[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) by[e] = pow2(value_range(high));
    if (!narrow) {
#pragma unroll
        for (int e = 0; e < 8; ++e) by[e] = pow2(value_range(__builtin_fmaxf(most_of[0][t + e], most_of[1][t + e])));
        if (wave == 0) P.row_lift[bht * kBlock + lane] = static_cast<unsigned char>(kLeast - value_range(of_row));
    }
    if (tid == 0) P.value_lift[bht] = narrow ? kLeast - value_range(high) : -1;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        float y[8];
        unpack8(P.dtype, u32x4{raw[i][0], raw[i][1], raw[i][2], raw[i][3]}, y);
        half8_t a;
        unsigned long long bad = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool finite = __builtin_fabsf(y[e]) < __builtin_inff();
            if (!finite) bad |= 1ull << (t + e);
            a[e] = static_cast<_Float16>(finite ? y[e] * by[e] : 0.0f);
        }
        if (bad != 0) atomicOr(&broken, bad);
        *reinterpret_cast<half8_t*>(P.v16 + bht * (8 * kI * 1024) + static_cast<size_t>(tid + i * kThreads) * 16) = a;
    }
    __syncthreads();
    if (tid == 0) P.broken[bht] = broken;
    if (P.parent && h == 0) {                                 // who of this tile lies on the way to a row
        for (int r = t0 + tid; r < share.rows; r += kThreads) {
            unsigned long long bits = 0;
            int at = r;
            while (at >= t0 + kBlock) at = up[at];
            for (; at >= t0; at = up[at]) bits |= 1ull << (at - t0);
            P.sees[(static_cast<size_t>(b) * R + r) * P.tiles + tile] = bits;
        }
    }
}

// An item, or the part of one that a worker has
struct Item {
    int b, h, group, len, nrho;    // nrho: (row, head) pairs of the sequence
    int first, last;               // cached blocks
    int tile0, tile1;              // tiles of the rows themselves
    bool whole;
    size_t slot;                   // for the result where it is not whole
};
// A worker's way along the line.  (All of it is the same for every thread of the workgroup.)
struct Line {
    long per, worker, begin, finish, x, before;
    int b;
    __device__ __forceinline__ explicit Line(const AttendParams& P) {
        per = P.plan[0];
        const long total = P.plan[1 + P.B];
        worker = spread_over_xcds(blockIdx.x, (total + per - 1) / per);   // (of those that have units, however few)
        begin = x = worker < 0 ? total : per * worker;
        finish = begin + per < total ? begin + per : total;
        b = 0;                                                // the sequence in which the units begin: 64 of them looked at at once
        for (int n = P.B; n > 1;) {                           // (of those that begin at the same unit the last one has units)
            const int lane = static_cast<int>(threadIdx.x) & 63, step = (n + 63) / 64;
            const unsigned long long up_to = __ballot(lane * step < n && P.plan[1 + b + min(lane * step, n - 1)] <= begin);
            const int past = (__popcll(up_to) - 1) * step;
            b += past;
            n = min(step, n - past);
        }
        before = P.plan[1 + b];                               // units before sequence b
    }
    __device__ __forceinline__ bool more() const { return x < finish; }
    __device__ __forceinline__ Item next(const AttendParams& P) {
        while (x >= P.plan[2 + b]) before = P.plan[1 + ++b];
        const Share share = share_of(P, b);
        const int units = units_of(share), item = static_cast<int>(static_cast<unsigned>(x - before) / static_cast<unsigned>(units));
        const long item0 = before + static_cast<long>(item) * units;
        const int u0 = static_cast<int>(x - item0), u1 = static_cast<int>(finish - item0 < units ? finish - item0 : units);
        const int end = max(0, u1 - kStart);
        Item it;
        it.b = b;
        it.group = item % share.groups;
        it.h = item / share.groups;
        it.len = max(0, min(P.cache.cache_len[b], P.cache.max_blocks * kBlock));
        it.nrho = share.rows * P.G;
        it.first = max(0, u0 - kStart);
        it.last = min(share.blocks, end);
        const int row1 = min(share.rows - 1, (it.group * P.tile + P.tile - 1) / P.G);   // last row of the item
        it.tile0 = max(0, it.first - share.blocks);
        it.tile1 = min(row1 / kBlock + 1, end - share.blocks);
        it.whole = u0 == 0 && u1 == units;
        // slot 0: of the item in which this worker's units begin; slot 1: of one that begins behind that and goes on with the next worker
        it.slot = 2 * static_cast<size_t>(worker) + (item0 > begin ? 1 : 0);
        if (u0 == 0 && threadIdx.x == 0) {                    // for the join: the item's first slot and its workers
            const long w1 = (item0 + units - 1) / per;
            P.pieces[(static_cast<size_t>(b) * P.cache.kv_heads + it.h) * (P.row_tiles * 16 / P.tile) + it.group] =
                make_int2(static_cast<int>(it.slot), static_cast<int>(w1 - worker) + 1);
        }
        x = item0 + u1;
        return it;
    }
};

template <int D>
struct AttendShapeOf {
    static constexpr int kI = D / 64;                         // 64-dimension steps of a head
    static constexpr int kT = D / 16;                         // tiles of 16 dimensions; also the fragments of a block's keys, and of its values
    static constexpr int kStage = 2 * kT * 1024;              // a block; also a tile's keys, and its values, in binary16
};

// Many rows: each of NW wavefronts takes 16 RT rows of its own and goes over all blocks, which they fetch together, four stages deep.  A block's fragment
// read from LDS and widened serves RT products; RT = 2 is what registers hold beside the sums at head_dim 128.
// FINE: see attend_prepare.
template <int D, int RT, int NW, bool FINE>
__global__ __launch_bounds__(NW * 64, 2) void attend_rows(AttendParams P) {
    using Shape = AttendShapeOf<D>;
    constexpr int kI = Shape::kI, kT = Shape::kT;
    __shared__ __align__(16) unsigned char lds[4 * Shape::kStage];   // blocks in flight
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int G = P.G, H = P.cache.kv_heads, R = P.R;
    Line line(P);
    while (line.more()) {
        // (what follows from a thread's number is worked out anew for every item: kept in registers from one to the next, as the
        // compiler would, it leaves the loop over blocks too few of them)
        const int tid = not_kept(thread), lane = tid & 63, col = lane & 15, g = lane >> 4;
        const Item it = line.next(P);
        const int b = it.b, h = it.h, group = it.group, first = it.first, last = it.last, tile0 = it.tile0, tile1 = it.tile1, len = it.len, nrho = it.nrho;
        const int rho0 = group * P.tile + wave * 16 * RT;   // first (row, head) pair of this wavefront
        const int32_t* table = P.cache.block_table + static_cast<size_t>(b) * P.cache.max_blocks;
        const size_t bh = static_cast<size_t>(b) * H + h;

        // 64 cached blocks at a time: a lane looks up one block's number and scales.  (The first of them together with the queries, so that an item
        // begins with two round trips and not with four.)
        const size_t layer0 = static_cast<size_t>(P.layer) * P.cache.num_blocks;
        int my_id = 0;
        auto look = [&](int j0) { my_id = table[min(j0 + lane, last - 1)]; };
        if (first < last) look(first);
        // ---- queries
        half8_t q[RT][2 * kI], q2[FINE ? RT : 1][2 * kI];
        float factor[RT];                                     // of the products of a row: its power of two back, scale, log2(e)
        int row_of[RT];                                       // the row, -1 behind the last
        const size_t parts = static_cast<size_t>(P.B) * H * P.row_tiles * 2 * kI * 1024;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int rho = rho0 + rt * 16 + col;
            row_of[rt] = rho < nrho ? rho / G : -1;
            factor[rt] = P.factor[bh * P.row_tiles * 16 + rho];
            const char* from = P.q16 + ((bh * P.row_tiles + rho0 / 16 + rt) * 2 * kI) * 1024 + lane * 16;
#pragma unroll
            for (int i = 0; i < 2 * kI; ++i) {
                q[rt][i] = *reinterpret_cast<const half8_t*>(from + i * 1024);
                if constexpr (FINE) q2[rt][i] = *reinterpret_cast<const half8_t*>(from + parts + i * 1024);
            }
        }
        bool good = false;
        float my_ks = 1.0f, my_vs = 1.0f;
        auto look_further = [&](int j0) {
            good = j0 + lane < last && my_id >= 0 && my_id < P.cache.num_blocks;
            if (!good) my_id = 0;                             // in bounds, and neither its tokens nor its scales count
            const size_t at = (layer0 + my_id) * H + h;
            const float ks = P.cache.k_scale[at], vs = P.cache.v_scale[at];
            my_ks = good ? ks : 1.0f;
            my_vs = good ? __builtin_fmaxf(vs, 0x1p-100f) : 0x1p-100f;
        };
        if (first < last) look_further(first);
        // (columns behind the last row hold anything; they are never stored, and must not hold up the others)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            if (row_of[rt] < 0) {
                const half8_t zero = {};
                factor[rt] = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * kI; ++i) {
                    q[rt][i] = zero;
                    if constexpr (FINE) q2[rt][i] = zero;
                }
            }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            settle(factor[rt]);
#pragma unroll
            for (int i = 0; i < 2 * kI; ++i) {
                settle(q[rt][i]);
                if constexpr (FINE) settle(q2[rt][i]);
            }
        }
        float4_t o[RT][kT];
        float most_vs = 0.0f;                                 // largest value scale so far
        float m[RT], l[RT];                                   // maximum of s + log2(value scale), less kRoom; sum (of all lanes of the column)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -__builtin_inff();
            l[rt] = 0.0f;
#pragma unroll
            for (int t = 0; t < kT; ++t) o[rt][t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const _Float16 one = static_cast<_Float16>(1.0f);
        const half8_t ones = {one, one, one, one, one, one, one, one};

        auto raise = [&](const float (&high)[RT]) {           // to maxima that have run away
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float to = __builtin_fmaxf(m[rt], column_max(high[rt]) - kRoom);
                const float root = back_from(m[rt], to), by = root * root;
                m[rt] = to;
                l[rt] = l[rt] * root * root;
#pragma unroll
                for (int t = 0; t < kT; ++t) o[rt][t] *= by;
            }
        };
        // Weights of 64 tokens from their products.  With `part` only those of kept(rt) count (a bit for each of the 16 tokens of this
        // lane's group).  Their sum is a product with ones: two instructions of the matrix unit for 16 additions, and it sums what the second product
        // will use.
        auto weigh = [&](float4_t (&s)[RT][4], float ks, float vs, auto part, auto kept, half8_t (&p)[RT][2]) {
            const float lift = __builtin_amdgcn_logf(vs), inv_vs = __builtin_amdgcn_rcpf(vs) * kPerUnit;   // (exact for powers of two)
            // 2^6 below: a weight of 2^-25 that binary16 loses is 2^-26 of the largest
            const bool low = vs < most_vs * 0x1p-6f;
            most_vs = __builtin_fmaxf(most_vs, vs);
            float high[RT], f[RT];
            bool over = false;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                f[rt] = factor[rt] * ks;
                if constexpr (part) {
                    const unsigned keep = kept(rt);
#pragma unroll
                    for (int j = 0; j < 16; ++j) s[rt][j / 4][j % 4] = keep >> j & 1u ? s[rt][j / 4][j % 4] : -3.0e38f;
                }
                float top = s[rt][0][0];
#pragma unroll
                for (int j = 1; j < 16; ++j) top = __builtin_fmaxf(top, s[rt][j / 4][j % 4]);
                high[rt] = fmaf(top, f[rt], lift);
                if constexpr (part) high[rt] = kept(rt) != 0u ? high[rt] : -__builtin_inff();   // (a factor near 0 takes a masked product to a score near 0)
                over |= high[rt] > m[rt] + kLazy;
            }
            if (__any(over)) raise(high);
            if (low) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float from = -kUnit - (m[rt] == -__builtin_inff() ? 0.0f : m[rt]);
                    const unsigned keep = part ? kept(rt) : 0xFFFFu;
                    float sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum += keep >> j & 1u ? __builtin_amdgcn_exp2f(fmaf(s[rt][j / 4][j % 4], f[rt], from)) : 0.0f;
                    l[rt] += column_sum(sum);
                }
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float from = lift - (m[rt] == -__builtin_inff() ? 0.0f : m[rt]);
                const unsigned keep = part ? kept(rt) : 0xFFFFu;
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    float2_t w;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        w[e] = __builtin_amdgcn_exp2f(fmaf(s[rt][j / 4][j % 4 + e], f[rt], from));
                        if constexpr (part) w[e] = keep >> (j + e) & 1u ? w[e] : 0.0f;
                    }
                    const half2_t two = __builtin_convertvector(w, half2_t);
                    p[rt][j / 8][j % 8] = two.x;
                    p[rt][j / 8][j % 8 + 1] = two.y;
                }
                float4_t z = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
                z = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p[rt][0], z, 0, 0, 0);
                z = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p[rt][1], z, 0, 0, 0);
                l[rt] = fmaf(z[0], low ? 0.0f : inv_vs, l[rt]);
            }
        };
        const std::integral_constant<bool, true> in_part;
        const std::integral_constant<bool, false> in_full;

        // ---- cached blocks
        {
            const size_t per_block = static_cast<size_t>(H) * kBlock * D;
            const char* kbase = static_cast<const char*>(P.cache.k_codes) + (layer0 * H + h) * (static_cast<size_t>(kBlock) * D) + ((col >> 2) * 16 + (col & 3)) * D + g * 16;
            const char* vbase = static_cast<const char*>(P.cache.v_codes) + (layer0 * H + h) * (static_cast<size_t>(kBlock) * D) + (g * D + col) * 16;
            unsigned char* flight = lds;
            // fragment f of the keys is tile f / kI, 64-dimension step f % kI; of the values tile f
            auto fetch_key = [&](size_t id, int f, unsigned char* to) { fetch_1k(kbase + id * per_block + (f / kI) * 4 * D + (f % kI) * 64, to + f * 1024); };
            auto fetch_value = [&](size_t id, int f, unsigned char* to) { fetch_1k(vbase + id * per_block + f * 256, to + (kT + f) * 1024); };
            auto products = [&](unsigned at, float4_t (&s)[RT][4]) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int t = 0; t < 4; ++t) s[rt][t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int f0 = 0; f0 < kT; f0 += 4) {
                    u32x4 w[4];
                    read_4k(at + f0 * 1024, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int f = f0 + e, t = f / kI, k = 2 * (f % kI);
                        const half8_t a = widened(w[e].x, w[e].y), c = widened(w[e].z, w[e].w);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            s[rt][t] = product<FINE>(a, q[rt][k], q2[FINE ? rt : 0][k], s[rt][t]);
                            s[rt][t] = product<FINE>(c, q[rt][k + 1], q2[FINE ? rt : 0][k + 1], s[rt][t]);
                        }
                    }
                }
            };
            // mine: how many of the 16 tokens of this lane's group there are.  What lies behind the last one may be anything: a weight of 0
            // would not make a NaN harmless
            auto sums = [&](unsigned at, const half8_t (&p)[RT][2], auto part, int mine) {
#pragma unroll
                for (int t0 = 0; t0 < kT; t0 += 4) {
                    u32x4 w[4];
                    read_4k(at + (kT + t0) * 1024, w);
                    if constexpr (part) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int bytes = max(0, min(4, mine - 4 * i));
                            const unsigned keep = bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1u;
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[e][i] &= keep;
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const half8_t a = widened(w[e].x, w[e].y), c = widened(w[e].z, w[e].w);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            o[rt][t0 + e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, p[rt][0], o[rt][t0 + e], 0, 0, 0);
                            o[rt][t0 + e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c, p[rt][1], o[rt][t0 + e], 0, 0, 0);
                        }
                    }
                }
            };
            for (int j0 = first; j0 < last; j0 += 64) {
                const int n = min(64, last - j0);
                if (j0 > first) {
                    look(j0);
                    look_further(j0);
                }
                const unsigned long long fine = __ballot(good);
                auto id_of = [&](int i) { return static_cast<size_t>(__builtin_amdgcn_readlane(my_id, i)); };
                auto float_of = [](float y, int i) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(y), i)); };
                // tokens of the i-th block that count
                auto left_of = [&](int i) { return fine >> i & 1ull ? len - (j0 + i) * kBlock : 0; };
                // blocks all of whose tokens count come first and have a loop of their own: only a sequence's last block has others
                // (a number out of range apart).  (With selections between the two the compiler makes a hundred instructions more a block.)
                const int full = n > 0 && fine == ~0ull >> (64 - n) ? n - (left_of(n - 1) < kBlock ? 1 : 0) : 0;
                settle(my_id);
                settle(my_ks);
                settle(my_vs);
                wait_fetches<0>();                            // (nothing of the loads above is counted below)
                // four stages: while block i is worked on, the three behind it are under way; a wavefront fetches every NW-th fragment
                constexpr int kMine = 2 * kT / NW;
                static_assert(2 * kT % NW == 0, "every wavefront fetches as many fragments");
                auto fetch_block = [&](int i) {
                    const size_t id = id_of(min(i, n - 1));
                    unsigned char* to = flight + i % 4 * Shape::kStage;
#pragma unroll
                    for (int e = 0; e < kMine; ++e) {
                        const int f = wave + e * NW;
                        if (f < kT) fetch_key(id, f, to);
                        else fetch_value(id, f - kT, to);
                    }
                };
                __syncthreads();                          // (the stages are free)
                fetch_block(0);
                fetch_block(1);
                fetch_block(2);
                auto step = [&](int i, auto part) {
                    wait_fetches<2 * kMine>();
                    __builtin_amdgcn_s_barrier();         // block i is there, and everyone is done with block i - 1
                    fetch_block(i + 3);
                    if (rho0 < nrho) {
                        const unsigned at = lds_address(flight + i % 4 * Shape::kStage) + lane * 16;
                        float4_t s[RT][4];
                        half8_t p[RT][2];
                        products(at, s);
                        const int mine = max(0, min(16, left_of(i) - 16 * g));
                        weigh(s, float_of(my_ks, i), float_of(my_vs, i), part, [&](int) { return (1u << mine) - 1u; }, p);
                        sums(at, p, part, mine);
                    }
                };
                int i = 0;
                for (; i < full; ++i) step(i, in_full);
                for (; i < n; ++i) step(i, in_part);
                wait_fetches<0>();
            }
        }
        // ---- the tail: the rows themselves, in binary16
        {
            // Weights where the rows of a tile have units of their own: each token's is in its weight's exponent (`lift`).  They lie far apart, so the sum
            // takes every weight without its own.  (Seldom: two exponentials a weight are well enough.)
            auto weigh_rows = [&](float4_t (&s)[RT][4], u32x4 lift, const unsigned (&see)[RT], half8_t (&p)[RT][2]) {
                float high[RT];
                bool over = false;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    high[rt] = -__builtin_inff();
                    settle(lift);                             // (its bytes are taken out anew each time: as numbers they would fill 16 registers)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float x = see[rt] >> j & 1u ? fmaf(s[rt][j / 4][j % 4], factor[rt], byte_of(lift[j / 4], j % 4)) : -__builtin_inff();
                        s[rt][j / 4][j % 4] = x;
                        high[rt] = __builtin_fmaxf(high[rt], x);
                    }
                    high[rt] -= kLeast;
                    over |= high[rt] > m[rt] + kLazy;
                }
                if (__any(over)) raise(high);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float from = (m[rt] == -__builtin_inff() ? 0.0f : m[rt]) + kLeast;
                    settle(lift);
                    float sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum += __builtin_amdgcn_exp2f(s[rt][j / 4][j % 4] - from - byte_of(lift[j / 4], j % 4) + (kLeast - kUnit));
#pragma unroll
                    for (int j = 0; j < 16; j += 2) {
                        const float2_t w = {__builtin_amdgcn_exp2f(s[rt][j / 4][j % 4] - from), __builtin_amdgcn_exp2f(s[rt][j / 4][j % 4 + 1] - from)};
                        const half2_t two = __builtin_convertvector(w, half2_t);
                        p[rt][j / 8][j % 8] = two.x;
                        p[rt][j / 8][j % 8 + 1] = two.y;
                    }
                    l[rt] += column_sum(sum);
                }
                most_vs = __builtin_inff();                   // (any unit may have been among them: tiles behind this one are summed without theirs, too)
            };
            // weights and sums of tile `tile`, whose keys lie at `keys` and whose values come when values() is called
            auto one_tile = [&](int tile, auto keys, auto values) {
                const size_t bht = bh * P.tiles + tile;
                const int t0 = tile * kBlock;
                float4_t s[RT][4];
                keys(s);
                const float* scales = P.key_scale + bht * kBlock + g * 16;
                const unsigned spoilt = static_cast<unsigned>(P.broken[bht] >> (16 * g)) & 0xFFFFu;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    float4_t ks = *reinterpret_cast<const float4_t*>(scales + 4 * t);   // of rows 4 g .. of token tile t
#pragma unroll
                    for (int i = 0; i < 4; ++i) ks[i] = spoilt >> (4 * t + i) & 1u ? __builtin_nanf("") : ks[i];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) s[rt][t] *= ks;
                }
                unsigned see[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const int r = row_of[rt];
                    if (r < t0) see[rt] = 0u;
                    else if (P.parent) see[rt] = static_cast<unsigned>(P.sees[(static_cast<size_t>(b) * R + r) * P.tiles + tile] >> (16 * g)) & 0xFFFFu;
                    else see[rt] = (1u << max(0, min(16, r - t0 - 16 * g + 1))) - 1u;         // rows t0 + 16 g .. r
                }
                const int one_lift = P.value_lift[bht];
                half8_t p[RT][2];
                if (one_lift >= 0) weigh(s, 1.0f, pow2(one_lift - kLeast), in_part, [&](int rt) { return see[rt]; }, p);
                else weigh_rows(s, *reinterpret_cast<const u32x4*>(P.row_lift + bht * kBlock + g * 16), see, p);
                values(p);
            };
            auto products16 = [&](unsigned at, auto second, float4_t (&s)[RT][4]) {   // second: the keys' second parts, or the first ones again
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (!second) s[rt][t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int f0 = 0; f0 < 8 * kI; f0 += 4) {
                    u32x4 w[4];
                    read_4k(at + f0 * 1024, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int f = f0 + e, t = f / (2 * kI), k = f % (2 * kI);
                        const half8_t a = __builtin_bit_cast(half8_t, w[e]);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            if constexpr (second) s[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q[rt][k], s[rt][t], 0, 0, 0);
                            else s[rt][t] = product<FINE>(a, q[rt][k], q2[FINE ? rt : 0][k], s[rt][t]);
                        }
                    }
                }
            };
            auto sums16 = [&](unsigned at, const half8_t (&p)[RT][2]) {
#pragma unroll
                for (int f0 = 0; f0 < 2 * kT; f0 += 4) {
                    u32x4 w[4];
                    read_4k(at + f0 * 1024, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
                            o[rt][(f0 + e) / 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, w[e]), p[rt][(f0 + e) & 1], o[rt][(f0 + e) / 2], 0, 0, 0);
                }
            };
            const std::integral_constant<bool, false> first_parts;
            const std::integral_constant<bool, true> second_parts;
            const size_t size = static_cast<size_t>(P.B) * H * P.tiles * Shape::kStage;
            const char* k16 = P.k16 + bh * P.tiles * Shape::kStage + lane * 16;
            const char* v16 = P.v16 + bh * P.tiles * Shape::kStage + lane * 16;
            if (tile0 < tile1) {
                // stages: keys, values (and the keys' second parts); without the latter the next tile is under way in the other two
                __syncthreads();                              // (the blocks' stages are free)
                constexpr int kMine = 2 * kT / NW;
                auto fetch = [&](const char* from, int stage) {
#pragma unroll
                    for (int e = 0; e < kMine; ++e) fetch_1k(from + (wave + e * NW) * 1024, lds + stage * Shape::kStage + (wave + e * NW) * 1024);
                };
                auto fetch_tile = [&](int tile, int stage) {
                    fetch(k16 + static_cast<size_t>(tile) * Shape::kStage, stage);
                    fetch(v16 + static_cast<size_t>(tile) * Shape::kStage, stage + 1);
                    if constexpr (FINE) fetch(k16 + size + static_cast<size_t>(tile) * Shape::kStage, stage + 2);
                };
                fetch_tile(tile0, 0);
                for (int tile = tile0; tile < tile1; ++tile) {
                    const int stage = FINE ? 0 : (tile - tile0) % 2 * 2;
                    wait_fetches<0>();
                    __builtin_amdgcn_s_barrier();             // the tile is there, and everyone is done with the one before
                    if (!FINE && tile + 1 < tile1) fetch_tile(tile + 1, 2 - stage);
                    const unsigned at = lds_address(lds + stage * Shape::kStage) + lane * 16;
                    if (rho0 < nrho && (min(rho0 + 16 * RT, nrho) - 1) / G >= tile * kBlock)
                        one_tile(tile, [&](float4_t (&s)[RT][4]) {
                            products16(at, first_parts, s);
                            if constexpr (FINE) products16(at + 2 * Shape::kStage, second_parts, s);
                        }, [&](const half8_t (&p)[RT][2]) { sums16(at + Shape::kStage, p); });
                    if constexpr (FINE) {
                        __builtin_amdgcn_s_barrier();
                        if (tile + 1 < tile1) fetch_tile(tile + 1, 0);
                    }
                }
                __syncthreads();
            }
        }

        if (it.whole) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int rho = rho0 + rt * 16 + col;
                if (rho >= nrho) continue;
                const int r = rho / G, head = h * G + (rho - r * G);
                const float inv = kPerUnit / l[rt];
                const size_t at = ((static_cast<size_t>(b) * R + r) * P.heads + head) * D;
#pragma unroll
                for (int t = 0; t < kT; ++t) store4(P.dtype, P.out, at + t * 16 + g * 4, o[rt][t] * inv);
            }
        } else {
            float* part = P.part + it.slot * P.tile * (D + 2);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int rho = rho0 + rt * 16 + col, at = wave * 16 * RT + rt * 16 + col;
                if (rho >= nrho) continue;
#pragma unroll
                for (int t = 0; t < kT; ++t) *reinterpret_cast<float4_t*>(part + static_cast<size_t>(at) * D + t * 16 + g * 4) = o[rt][t];
                if (g == 0) {
                    part[static_cast<size_t>(P.tile) * D + 2 * at] = m[rt];
                    part[static_cast<size_t>(P.tile) * D + 2 * at + 1] = l[rt];
                }
            }
        }
    }
}

// Few rows (up to 16 RT = 64): four wavefronts share every block without doing anything twice.  Wavefront w takes the products of
// token tile w with all rows, and the sums of a quarter of the dimensions: it fetches and widens a quarter of the keys and a quarter of the
// values, its own, and only the weights go round, through LDS, with one barrier a block (two buffers: who is a block ahead writes
// the other one).  A wavefront that sees a maximum run away says so beside its weights; then all of them agree on a new one and form the weights again.
// O' is complete in every dimension, so nothing is joined between wavefronts but the sums of weights.  (With blocks dealt to the wavefronts of
// attend_rows instead, 64 sequences of up to 8192 tokens and 36 rows a key head take 200 us in place of 171: a quarter of its rows are padding.)
template <int D, int RT, bool FINE>
__global__ __launch_bounds__(kWG, 2) void attend_few(AttendParams P) {
    using Shape = AttendShapeOf<D>;
    constexpr int kI = Shape::kI, kT = Shape::kT, kV = kT / 4;          // kV: tiles of 16 dimensions of a wavefront
    constexpr int kPart = (kI + kV) * 1024;                             // a block's keys and values of a wavefront
    constexpr int kStages = D == 256 ? 2 : RT == 4 ? 3 : 4;             // (two workgroups a compute unit)
    __shared__ __align__(16) unsigned char lds[4 * kStages * kPart];    // a wavefront's blocks in flight lie side by side
    __shared__ __align__(16) unsigned char weights[2][RT * 2 * 1024];   // of a block, as the second product takes them
    __shared__ __align__(16) int over[2][4];
    __shared__ float highs[4][16 * RT];
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int H = P.cache.kv_heads, R = P.R, G = P.G;
    int turn = 0;                                                       // which of the two buffers is next
    Line line(P);
    while (line.more()) {
        const int tid = not_kept(thread), lane = tid & 63, col = lane & 15, g = lane >> 4;
        const Item it = line.next(P);
        const int b = it.b, h = it.h, len = it.len, first = it.first, last = it.last, rho0 = it.group * P.tile;
        const int32_t* table = P.cache.block_table + static_cast<size_t>(b) * P.cache.max_blocks;
        const size_t bh = static_cast<size_t>(b) * H + h;

        // 64 cached blocks at a time: a lane looks up one block's number and scales.  (The first of them together with the queries, so that an item
        // begins with two round trips and not with four.)
        const size_t layer0 = static_cast<size_t>(P.layer) * P.cache.num_blocks;
        int my_id = 0;
        auto look = [&](int j0) { my_id = table[min(j0 + lane, last - 1)]; };
        if (first < last) look(first);
        half8_t q[RT][2 * kI], q2[FINE ? RT : 1][2 * kI];
        float factor[RT];                                               // of the products of a row: its power of two back, scale, log2(e)
        int row_of[RT];                                                 // the row, -1 behind the last
        const size_t parts = static_cast<size_t>(P.B) * H * P.row_tiles * 2 * kI * 1024;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int rho = rho0 + rt * 16 + col;
            row_of[rt] = rho < it.nrho ? rho / G : -1;
            factor[rt] = P.factor[bh * P.row_tiles * 16 + rho];
            const char* from = P.q16 + ((bh * P.row_tiles + rho0 / 16 + rt) * 2 * kI) * 1024 + lane * 16;
#pragma unroll
            for (int i = 0; i < 2 * kI; ++i) {
                q[rt][i] = *reinterpret_cast<const half8_t*>(from + i * 1024);
                if constexpr (FINE) q2[rt][i] = *reinterpret_cast<const half8_t*>(from + parts + i * 1024);
            }
        }
        bool good = false;
        float my_ks = 1.0f, my_vs = 1.0f;
        auto look_further = [&](int j0) {
            good = j0 + lane < last && my_id >= 0 && my_id < P.cache.num_blocks;
            if (!good) my_id = 0;                             // in bounds, and neither its tokens nor its scales count
            const size_t at = (layer0 + my_id) * H + h;
            const float ks = P.cache.k_scale[at], vs = P.cache.v_scale[at];
            my_ks = good ? ks : 1.0f;
            my_vs = good ? __builtin_fmaxf(vs, 0x1p-100f) : 0x1p-100f;
        };
        if (first < last) look_further(first);
        // (columns behind the last row hold anything; they are never stored, and must not hold up the others)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            if (row_of[rt] < 0) {
                const half8_t zero = {};
                factor[rt] = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * kI; ++i) {
                    q[rt][i] = zero;
                    if constexpr (FINE) q2[rt][i] = zero;
                }
            }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            settle(factor[rt]);
#pragma unroll
            for (int i = 0; i < 2 * kI; ++i) {
                settle(q[rt][i]);
                if constexpr (FINE) settle(q2[rt][i]);
            }
        }
        float4_t o[RT][kV];
        float most_vs = 0.0f;                                           // largest value scale so far
        float m[RT], l[RT];                                             // maximum of s + log2(value scale), less kRoom; sum of this lane's tokens' weights
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -__builtin_inff();
            l[rt] = 0.0f;
#pragma unroll
            for (int t = 0; t < kV; ++t) o[rt][t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }

        // From this wavefront's products to everyone's weights p.  With `part` only the tokens of kept(rt) count (a bit for each of this
        // lane's four).  `rows`: each token's values are in units of their own (lifts: log2 and kLeast); these lie far apart, so
        // the sum takes every weight without its own.
        auto weigh = [&](float4_t (&s)[RT], float ks, float vs, auto part, auto kept, auto rows, unsigned lifts, half8_t (&p)[RT][2]) {
            const float lift = __builtin_amdgcn_logf(vs), inv_vs = __builtin_amdgcn_rcpf(vs) * kPerUnit;   // (exact for powers of two)
            const bool low = vs < most_vs * 0x1p-60f;                   // weights may vanish in binary32
            most_vs = __builtin_fmaxf(most_vs, vs);
            float high[RT], f[RT];
            bool run = false;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                f[rt] = factor[rt] * ks;
                if constexpr (rows) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[rt][i] = kept(rt) >> i & 1u ? fmaf(s[rt][i], f[rt], byte_of(lifts, i)) : -__builtin_inff();
                } else if constexpr (part) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[rt][i] = kept(rt) >> i & 1u ? s[rt][i] : -3.0e38f;
                }
                high[rt] = __builtin_fmaxf(__builtin_fmaxf(s[rt][0], s[rt][1]), __builtin_fmaxf(s[rt][2], s[rt][3]));
                high[rt] = rows ? high[rt] - kLeast : fmaf(high[rt], f[rt], lift);
                if constexpr (part && !rows) high[rt] = kept(rt) != 0u ? high[rt] : -__builtin_inff();   // (a factor near 0 takes a masked product to a score near 0)
                run |= high[rt] > m[rt] + kLazy;
            }
            float sum[RT];
            unsigned char* box = weights[turn] + (wave >> 1) * 1024 + lane * 16 + (wave & 1) * 8;
            auto form = [&]() {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float base = m[rt] == -__builtin_inff() ? 0.0f : m[rt];
                    float w[4];
                    if constexpr (rows) {
                        sum[rt] = 0.0f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = s[rt][i] - (base + kLeast);
                            w[i] = __builtin_amdgcn_exp2f(x);
                            sum[rt] += __builtin_amdgcn_exp2f(x - byte_of(lifts, i) + (kLeast - kUnit));
                        }
                    } else {
                        const float from = lift - base;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            w[i] = __builtin_amdgcn_exp2f(fmaf(s[rt][i], f[rt], from));
                            if constexpr (part) w[i] = kept(rt) >> i & 1u ? w[i] : 0.0f;
                        }
                        sum[rt] = ((w[0] + w[1]) + (w[2] + w[3])) * inv_vs;
                        if (low) {
                            sum[rt] = 0.0f;
#pragma unroll
                            for (int i = 0; i < 4; ++i) sum[rt] += !part || (kept(rt) >> i & 1u) ? __builtin_amdgcn_exp2f(fmaf(s[rt][i], f[rt], from - lift - kUnit)) : 0.0f;
                        }
                    }
                    const float2_t lo = {w[0], w[1]}, hi = {w[2], w[3]};
                    uint2 y;
                    y.x = __builtin_bit_cast(unsigned, __builtin_convertvector(lo, half2_t));
                    y.y = __builtin_bit_cast(unsigned, __builtin_convertvector(hi, half2_t));
                    *reinterpret_cast<uint2*>(box + rt * 2048) = y;
                }
            };
            form();
            const bool mine = __any(run);
            if (lane == 0) over[turn][wave] = mine ? 1 : 0;
            meet();
            if ((over[turn][0] | over[turn][1] | over[turn][2] | over[turn][3]) != 0) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float top = column_max(high[rt]);
                    if (g == 0) highs[wave][rt * 16 + col] = top;
                }
                meet();
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    float to = m[rt];
#pragma unroll
                    for (int w = 0; w < 4; ++w) to = __builtin_fmaxf(to, highs[w][rt * 16 + col] - kRoom);
                    const float root = back_from(m[rt], to), by = root * root;
                    m[rt] = to;
                    l[rt] = l[rt] * root * root;
#pragma unroll
                    for (int t = 0; t < kV; ++t) o[rt][t] *= by;
                }
                form();
                meet();
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                l[rt] += sum[rt];
#pragma unroll
                for (int k = 0; k < 2; ++k) p[rt][k] = *reinterpret_cast<const half8_t*>(weights[turn] + (rt * 2 + k) * 1024 + lane * 16);
            }
            turn ^= 1;
        };
        const std::integral_constant<bool, true> in_part;
        const std::integral_constant<bool, false> in_full;
        unsigned char* flight = lds + wave * kStages * kPart;

        // ---- cached blocks
        {
            const size_t per_block = static_cast<size_t>(H) * kBlock * D;
            const char* kbase = static_cast<const char*>(P.cache.k_codes) + (layer0 * H + h) * (static_cast<size_t>(kBlock) * D) + ((col >> 2) * 16 + (col & 3) + 4 * wave) * D + g * 16;
            const char* vbase = static_cast<const char*>(P.cache.v_codes) + (layer0 * H + h) * (static_cast<size_t>(kBlock) * D) + (g * D + wave * kV * 16 + col) * 16;
            for (int j0 = first; j0 < last; j0 += 64) {
                const int n = min(64, last - j0);
                if (j0 > first) {
                    look(j0);
                    look_further(j0);
                }
                const unsigned long long fine = __ballot(good);
                auto float_of = [](float y, int i) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(y), i)); };
                // tokens of the i-th block that count
                auto left_of = [&](int i) { return fine >> i & 1ull ? len - (j0 + i) * kBlock : 0; };
                // blocks all of whose tokens count come first and have a loop of their own: only a sequence's last block has others
                // (a number out of range apart)
                const int full = fine == ~0ull >> (64 - n) ? n - (left_of(n - 1) < kBlock ? 1 : 0) : 0;
                auto fetch = [&](int i) {                               // (behind the last one it comes again, unused: the count of fetches stays)
                    const size_t id = static_cast<size_t>(__builtin_amdgcn_readlane(my_id, min(i, n - 1)));
                    unsigned char* to = flight + i % kStages * kPart;
#pragma unroll
                    for (int f = 0; f < kI; ++f) fetch_1k(kbase + id * per_block + f * 64, to + f * 1024);
#pragma unroll
                    for (int f = 0; f < kV; ++f) fetch_1k(vbase + id * per_block + f * 256, to + (kI + f) * 1024);
                };
                settle(my_id);
                settle(my_ks);
                settle(my_vs);
                wait_fetches<0>();                                      // (nothing of the loads above is counted below)
#pragma unroll
                for (int i = 0; i < kStages; ++i) fetch(i);
                auto step = [&](int i, auto part) {
                    const unsigned at = lds_address(flight + i % kStages * kPart) + lane * 16;
                    float4_t s[RT];
                    half8_t p[RT][2];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) s[rt] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
                    wait_fetches<(kStages - 1) * (kI + kV) + kV>();
                    u32x4 w[kI > kV ? kI : kV];
                    read_some<kI>(at, w);
#pragma unroll
                    for (int f = 0; f < kI; ++f) {
                        const half8_t a = widened(w[f].x, w[f].y), c = widened(w[f].z, w[f].w);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            s[rt] = product<FINE>(a, q[rt][2 * f], q2[FINE ? rt : 0][2 * f], s[rt]);
                            s[rt] = product<FINE>(c, q[rt][2 * f + 1], q2[FINE ? rt : 0][2 * f + 1], s[rt]);
                        }
                    }
                    const int mine = max(0, min(16, left_of(i) - 16 * g));          // of the 16 tokens of this lane's group
                    const unsigned keep = ((1u << mine) - 1u) >> (4 * wave) & 15u;
                    weigh(s, float_of(my_ks, i), float_of(my_vs, i), part, [&](int) { return keep; }, in_full, 0u, p);
                    wait_fetches<(kStages - 1) * (kI + kV)>();
                    read_some<kV>(at + kI * 1024, w);
#pragma unroll
                    for (int t = 0; t < kV; ++t) {
                        // what lies behind the last token may be anything: a weight of 0 would not make a NaN harmless
                        if constexpr (part) {
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int bytes = max(0, min(4, mine - 4 * k));
                                w[t][k] = bytes == 4 ? w[t][k] : w[t][k] & ((1u << (8 * bytes)) - 1u);
                            }
                        }
                        const half8_t a = widened(w[t].x, w[t].y), c = widened(w[t].z, w[t].w);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, p[rt][0], o[rt][t], 0, 0, 0);
                            o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c, p[rt][1], o[rt][t], 0, 0, 0);
                        }
                    }
                    fetch(i + kStages);
                };
                int i = 0;
                for (; i < full; ++i) step(i, in_full);
                for (; i < n; ++i) step(i, in_part);
                wait_fetches<0>();
            }
        }

        // ---- the tail: the rows themselves, in binary16 (straight from memory: there is one tile, seldom two)
        for (int tile = it.tile0; tile < it.tile1; ++tile) {
            const size_t bht = bh * P.tiles + tile, size = static_cast<size_t>(P.B) * H * P.tiles * Shape::kStage;
            const int t0 = tile * kBlock;
            const char* keys = P.k16 + bht * Shape::kStage + wave * 2 * kI * 1024 + lane * 16;
            const char* values = P.v16 + bht * Shape::kStage + wave * kV * 2048 + lane * 16;
            half8_t a[2 * kI], a2[FINE ? 2 * kI : 1], v[2 * kV];
#pragma unroll
            for (int k = 0; k < 2 * kI; ++k) {
                a[k] = *reinterpret_cast<const half8_t*>(keys + k * 1024);
                if constexpr (FINE) a2[k] = *reinterpret_cast<const half8_t*>(keys + size + k * 1024);
            }
#pragma unroll
            for (int k = 0; k < 2 * kV; ++k) v[k] = *reinterpret_cast<const half8_t*>(values + k * 1024);
            float4_t ks = *reinterpret_cast<const float4_t*>(P.key_scale + bht * kBlock + g * 16 + 4 * wave);
            const unsigned spoilt = static_cast<unsigned>(P.broken[bht] >> (16 * g + 4 * wave)) & 15u;
            const int one_lift = P.value_lift[bht];                                 // (the same for everyone, and so is the way taken below, with its barriers)
#pragma unroll
            for (int i = 0; i < 4; ++i) ks[i] = spoilt >> i & 1u ? __builtin_nanf("") : ks[i];   // (of those a row sees every weight is NaN then)
            float4_t s[RT];
            half8_t p[RT][2];
            unsigned see[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                s[rt] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < 2 * kI; ++k) {
                    s[rt] = product<FINE>(a[k], q[rt][k], q2[FINE ? rt : 0][k], s[rt]);
                    if constexpr (FINE) s[rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a2[k], q[rt][k], s[rt], 0, 0, 0);
                }
                s[rt] *= ks;
                const int r = row_of[rt], r0 = t0 + 16 * g + 4 * wave;            // this lane's tokens: rows r0 .. r0 + 3
                if (r < t0) see[rt] = 0u;
                else if (P.parent) see[rt] = static_cast<unsigned>(P.sees[(static_cast<size_t>(b) * R + r) * P.tiles + tile] >> (16 * g + 4 * wave)) & 15u;
                else see[rt] = (1u << max(0, min(4, r - r0 + 1))) - 1u;
            }
            auto seen = [&](int rt) { return see[rt]; };
            if (one_lift >= 0) weigh(s, 1.0f, pow2(one_lift - kLeast), in_part, seen, in_full, 0u, p);
            else weigh(s, 1.0f, 1.0f, in_part, seen, in_part, *reinterpret_cast<const unsigned*>(P.row_lift + bht * kBlock + g * 16 + 4 * wave), p);
#pragma unroll
            for (int t = 0; t < 2 * kV; ++t)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][t / 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[t], p[rt][t & 1], o[rt][t / 2], 0, 0, 0);
        }

        // ---- sums of all wavefronts' weights
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float sum = column_sum(l[rt]);
            if (g == 0) highs[wave][rt * 16 + col] = sum;
        }
        meet();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) l[rt] = (highs[0][rt * 16 + col] + highs[1][rt * 16 + col]) + (highs[2][rt * 16 + col] + highs[3][rt * 16 + col]);
        meet();
        if (it.whole) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int rho = rho0 + rt * 16 + col;
                if (rho >= it.nrho) continue;
                const int r = rho / G, head = h * G + (rho - r * G);
                const float inv = kPerUnit / l[rt];
                const size_t at = ((static_cast<size_t>(b) * R + r) * P.heads + head) * D + wave * kV * 16 + g * 4;
#pragma unroll
                for (int t = 0; t < kV; ++t) store4(P.dtype, P.out, at + t * 16, o[rt][t] * inv);
            }
        } else {
            float* part = P.part + it.slot * P.tile * (D + 2);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int at = rt * 16 + col;
                if (rho0 + at >= it.nrho) continue;
#pragma unroll
                for (int t = 0; t < kV; ++t) *reinterpret_cast<float4_t*>(part + static_cast<size_t>(at) * D + wave * kV * 16 + t * 16 + g * 4) = o[rt][t];
                if (g == 0 && wave == 0) {
                    part[static_cast<size_t>(P.tile) * D + 2 * at] = m[rt];
                    part[static_cast<size_t>(P.tile) * D + 2 * at + 1] = l[rt];
                }
            }
        }
    }
}

// Joins the items that several workers share.  D / 4 lanes hold a row's dimensions, four each; such groups of lanes take a row each, or (by_pieces)
// those of a workgroup share the pieces of one row, where the call has few rows and their pieces may be many: 1 row of 32 heads 16.9 us in place of
// 19.5, but 64 sequences of 9 rows 183 in place of 171.  8 pieces are requested at once.
// Grid: runs of a key head's rows, key heads, sequences.
template <int D>
__global__ __launch_bounds__(kWG) void attend_join(AttendParams P, int by_pieces) {
    constexpr int kLanes = D / 4, kGroups = kWG / kLanes;
    __shared__ float stats[kGroups][2];
    __shared__ __align__(16) float4_t sums[kGroups][kLanes];
    const int b = static_cast<int>(blockIdx.z), h = static_cast<int>(blockIdx.y), at_row = static_cast<int>(blockIdx.x);
    const int d = static_cast<int>(threadIdx.x) % kLanes * 4, which = static_cast<int>(threadIdx.x) / kLanes;
    const int nrho = (P.row_count ? max(0, min(P.row_count[b], P.R)) : P.R) * P.G, H = P.cache.kv_heads;
    const int rho = by_pieces ? at_row : at_row * kGroups + which, group = divided(rho, P.tile, P.by_tile), at = rho - group * P.tile;
    int2 piece = make_int2(0, 0);
    if (rho < nrho) piece = P.pieces[(static_cast<size_t>(b) * H + h) * (P.row_tiles * 16 / P.tile) + group];
    const int n = piece.y, step = by_pieces ? kGroups : 1;
    if (by_pieces ? n <= 1 : !__any(n > 1)) return;           // (with by_pieces n is the workgroup's)
    const size_t size = static_cast<size_t>(P.tile) * (D + 2);
    const size_t stat = static_cast<size_t>(P.tile) * D + 2 * at, mine = static_cast<size_t>(at) * D + d;
    float top = -__builtin_inff(), sum = 0.0f;
    float4_t acc = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // as many pieces at once as there are, up to 8
    auto some = [&](int s0, auto once) {
        constexpr int kOnce = decltype(once)::value;
        float4_t y[kOnce];
        float m[kOnce], l[kOnce], high = top;
#pragma unroll
        for (int k = 0; k < kOnce; ++k) {
            const int s = s0 + k * step;
            m[k] = -__builtin_inff();
            l[k] = 0.0f;
            y[k] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
            if (s < n) {
                // slots: the first worker's, then the first ones of the workers behind it
                const float* p = P.part + (s == 0 ? piece.x : piece.x / 2 * 2 + 2 * s) * size;
                m[k] = p[stat];
                l[k] = p[stat + 1];
                y[k] = *reinterpret_cast<const float4_t*>(p + mine);
            }
        }
#pragma unroll
        for (int k = 0; k < kOnce; ++k) high = __builtin_fmaxf(high, m[k]);
        const float back = back_from(top, high);
        top = high;
        sum = sum * back * back;
        acc *= back * back;
#pragma unroll
        for (int k = 0; k < kOnce; ++k) {
            const float root = back_from(m[k], high), by = root * root;
            sum = fmaf(l[k] * root, root, sum);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(y[k][e], by, acc[e]);
        }
    };
    int s0 = by_pieces ? which : 0;
    if (!__any(s0 + 2 * step < n)) some(s0, std::integral_constant<int, 2>());
    else for (; s0 < n; s0 += 8 * step) some(s0, std::integral_constant<int, 8>());
    if (by_pieces) {
        if (d == 0) {
            stats[which][0] = top;
            stats[which][1] = sum;
        }
        sums[which][d / 4] = acc;
        __syncthreads();
        if (which != 0) return;
        float high = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < kGroups; ++w) high = __builtin_fmaxf(high, stats[w][0]);
        sum = 0.0f;
        acc = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kGroups; ++w) {
            const float root = back_from(stats[w][0], high);
            sum = fmaf(stats[w][1] * root, root, sum);
            acc += sums[w][d / 4] * (root * root);
        }
    }
    if (n <= 1) return;
    const int r = divided(rho, P.G, P.by_G), head = h * P.G + rho - r * P.G;
    store4(P.dtype, P.out, ((static_cast<size_t>(b) * P.R + r) * P.heads + head) * D + d, acc * (kPerUnit / sum));
}

}  // namespace

#endif  // FSD_CSRC_CACHE_ATTEND_H_
