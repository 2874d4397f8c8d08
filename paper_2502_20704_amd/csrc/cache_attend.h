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
// sum += p / vs.  So p is at most 2^8 whatever the scales are (binary16 holds it), codes enter the product exactly,
// and O' / sum is the result.  m follows the maximum only where that is more than 2^8 above it: a rescaling of O' is rare.
//
// Three kernels: attend_prepare turns queries and the rows' keys, brings them and the rows' values into binary16's range by powers of two and lays them
// out in the workspace as the matrix instruction takes them, so that no piece of the work does this again; it deals out the work, which takes the
// lengths, and reports the sequences.  attend_rows is the pass over cache and rows: every workgroup gets the same number of blocks, whichever sequences and
// heads they belong to.  attend_join puts together what lies across the border of two workgroups.
#ifndef FSD_CSRC_CACHE_ATTEND_H_
#define FSD_CSRC_CACHE_ATTEND_H_

#include "operators_common.h"

namespace {

typedef float float2_t __attribute__((ext_vector_type(2)));

constexpr float kLazy = 8.0f;      // how far (in powers of two) weights may pass 1 before they are scaled down again
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
    int least;                     // units of a workgroup, at least
    int tile;                      // rows of an item
    int row_tiles;                 // of 16 rows, of a (sequence, key head): whole items
    int tiles;                     // of 64 tokens of the R rows
    int query_groups;              // workgroups of attend_prepare that a sequence's queries take
    // workspace
    long* plan;                    // [0] units of a workgroup, [1 + b] units of the sequences before b
    int2* pieces;                  // [B, kv_heads, groups] of an item: its first slot, and how many workers share it
    float* factor;                 // [B, kv_heads, row_tiles * 16] of the products of a row: its power of two back, scale, log2(e)
    float* key_scale;              // [B, kv_heads, tiles, 64]
    float* value_scale;            // [B, kv_heads, tiles]
    unsigned long long* broken;    // [B, kv_heads, tiles] tokens of a tile with a value that is not finite
    unsigned long long* sees;      // [B, R, tiles] trees: tokens of a tile that a row sees
    char* q16;                     // [B, kv_heads, row_tiles, 2 * (D / 64)] fragments of 1 KB; binary16 inputs: second parts behind them
    char* k16;                     // [B, kv_heads, tiles, 4 * 2 * (D / 64)] fragments; second parts likewise
    char* v16;                     // [B, kv_heads, tiles, 2 * (D / 16)] fragments
    float* part;                   // results of pieces: two slots a worker, [rows of an item][D], then [rows][2] each
};

// The work is a line of units.  An item is one (sequence, key head, run of `tile` rows); its units are the blocks of the sequence's
// cache, then its tiles of 64 rows; kStart more stand for what an item costs at its beginning, whoever begins it.
constexpr int kStart = 2;
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
        P.plan[0] = per < P.least ? P.least : per;
        P.plan[1 + P.B] = base;
    }
}

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
// maximum over the four lanes that hold one column
__device__ __forceinline__ float column_max(float v) {
    v = __builtin_fmaxf(v, __shfl_xor(v, 16, 64));
    return __builtin_fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float column_sum(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}
// the power of two that brings `most` into [2^13, 2^14) (1 where there is nothing to bring there), as an exponent
__device__ __forceinline__ int to_half_range(float most) {
    const int e = static_cast<int>(__float_as_uint(most) >> 23) - 127;
    return most > 0.0f ? min(13 - e, 126) : 0;
}

constexpr int kMaxNodes = 2048;

__device__ __forceinline__ int not_kept(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// ---- blocks come to LDS without passing through registers: a lane's 16 bytes of a fragment land at 16 * lane of its 1 KB, and
// the same lane (or the same lane of another wavefront) reads them back, so that nothing is exchanged between lanes

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) void global_void;

__device__ __forceinline__ void fetch_1k(const char* from, unsigned char* to) {   // from: this lane's 16 bytes; to: the same for all lanes
    __builtin_amdgcn_global_load_lds((global_void*)(from), (lds_void*)(to), 16, 0, 0);
}
__device__ __forceinline__ unsigned lds_address(const unsigned char* p) {
    return static_cast<unsigned>(reinterpret_cast<uintptr_t>((const lds_void*)(p)));
}
// four fragments 1 KB apart.  (In assembly because the compiler would wait for every fetch in flight before it reads LDS.)
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
// y times a power of two in binary16: the first part, and what is left in a second
__device__ __forceinline__ void two_parts(const float (&y)[8], float by, half8_t& a, half8_t& c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float z = y[e] * by;
        a[e] = static_cast<_Float16>(z);
        c[e] = static_cast<_Float16>(z - static_cast<float>(a[e]));
    }
}

// Queries and the rows' keys and values in the layout of the products; the plan; the sequences' reports.  Workgroup 0 deals the work out; of the others
// each belongs to one sequence and takes some of its query rows, or one tile of 64 rows of a key head.
// FINE (binary16 inputs): a turned query or key is held in two parts of 11 bits, as one rounding of them would cost more than that of the result:
// 0.00047 of the result's norm in place of 0.00025 at 131072 tokens.
template <int D>
__global__ __launch_bounds__(kWG) void attend_prepare(AttendParams P) {
    constexpr int kI = D / 64, kPer = D / 8, kThreads = kWG;
    __shared__ __align__(16) _Float16 turned[kBlock * D];     // values: [16-dimension tile][2][lane][8]
    __shared__ float most_of[kWG / 64];
    __shared__ unsigned long long broken;
    extern __shared__ short tree[];                           // trees: [R] parent's row, [R] depth, [R] ancestors found so far
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (blockIdx.x == 0) {
        deal(P);
        return;
    }
    const int H = P.cache.kv_heads, R = P.R, G = P.G;
    const int per_sequence = P.query_groups + H * P.tiles, b = static_cast<int>((blockIdx.x - 1) / per_sequence), part = static_cast<int>((blockIdx.x - 1) % per_sequence);
    const Share share = share_of(P, b);
    const int len = max(0, min(P.cache.cache_len[b], P.cache.max_blocks * kBlock));
    short* up = tree;
    short* depth = tree + R;
    short* stands = tree + 2 * R;
    bool bad_tree = false;
    if (P.parent) {
        // depths by doubling: after step i a row knows its 2^i-th ancestor and how far that is
        const int32_t* parent = P.parent + static_cast<size_t>(b) * (R - 1);
        for (int r = tid; r < R; r += kThreads) {
            int p = -1;                                   // row 0 has none
            if (r > 0) {
                p = parent[r - 1];
                const bool bad = p < -1 || p >= r - 1;
                bad_tree |= bad;
                p = bad ? 0 : p + 1;
            }
            up[r] = static_cast<short>(p);
            stands[r] = static_cast<short>(p);
            depth[r] = r > 0 ? 1 : 0;
        }
        bad_tree = __syncthreads_or(bad_tree);
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
    auto position = [&](int r) { return len + (P.parent ? depth[r] : r); };
    auto table_row = [&](int pos) { return P.rot.table ? min(pos, P.rot.rows - 1) : 0; };
    const bool fine = P.dtype == FSD_F16;

    if (part < P.query_groups) {
        if (part == 0 && P.status) {                          // the sequence's report
            const int32_t* table = P.cache.block_table + static_cast<size_t>(b) * P.cache.max_blocks;
            bool bad = P.cache.cache_len[b] < 0 || P.cache.cache_len[b] > P.cache.max_blocks * kBlock ||
                       (P.row_count && (P.row_count[b] < 0 || P.row_count[b] > R));
            for (int i = tid; i < share.blocks; i += kThreads) bad |= table[i] < 0 || table[i] >= P.cache.num_blocks;
            if (P.rot.table)
                for (int r = tid; r < share.rows; r += kThreads) bad |= position(r) >= P.rot.rows;
            bad = __syncthreads_or(bad);
            if (tid == 0) P.status[b] = (bad ? FSD_ROW_BAD_CACHE : 0) | (bad_tree ? FSD_ROW_BAD_PARENT : 0);
        }
        // a thread takes 8 dimensions of a row, D / 8 neighbours the whole of it
        const size_t parts = static_cast<size_t>(P.B) * H * P.row_tiles * 2 * kI * 1024;
        const int n = share.rows * P.heads;
        for (int u = part * kThreads + tid; u / kPer < n; u += P.query_groups * kThreads) {
            const int r = u / kPer / P.heads, head = u / kPer % P.heads, dim = u % kPer * 8, h = head / G, rho = r * G + head % G;
            const size_t at[1] = {(static_cast<size_t>(b) * R + r) * P.q_stride + static_cast<size_t>(head) * D};
            const int dims[1] = {dim}, pos[1] = {table_row(position(r))};
            float y[1][8];
            load_turned<1>(P.dtype, P.q, at, dims, P.rot, pos, y);
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, finite_abs(y[0][e]));
#pragma unroll
            for (int o = kPer / 2; o > 0; o >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, o, 64));
            const float by = pow2(max(to_half_range(most), -126));
            half8_t a, c;
            two_parts(y[0], P.scale < 0.0f ? -by : by, a, c);  // (a negative scale goes in here: a larger product is always a larger score)
            const size_t bh = static_cast<size_t>(b) * H + h, fragment = (bh * P.row_tiles + rho / 16) * 2 * kI + dim / 64 * 2 + (dim / 8 & 1);
            char* to = P.q16 + fragment * 1024 + ((dim / 16 & 3) * 16 + (rho & 15)) * 16;
            *reinterpret_cast<half8_t*>(to) = a;
            if (fine) *reinterpret_cast<half8_t*>(to + parts) = c;
            if (dim == 0) P.factor[bh * P.row_tiles * 16 + rho] = __builtin_fabsf(P.scale) / by;
        }
        return;
    }
    const int tile = (part - P.query_groups) % P.tiles, h = (part - P.query_groups) / P.tiles, t0 = tile * kBlock, n = min(kBlock, share.rows - t0);
    if (n <= 0) return;
    const size_t bht = (static_cast<size_t>(b) * H + h) * P.tiles + tile, size = static_cast<size_t>(P.B) * H * P.tiles * 8 * kI * 1024;
    const size_t base = (static_cast<size_t>(b) * R + t0) * P.kv_stride + static_cast<size_t>(h) * D;
    constexpr int kUnits = kBlock * kPer / kThreads;
    u32x4 raw[kUnits];                                        // values as they are
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int u = tid + i * kThreads, t = u / kPer;
        raw[i] = u32x4{0, 0, 0, 0};
        if (t < n) raw[i] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned short*>(P.v) + base + t * P.kv_stride + u % kPer * 8);
    }
    // keys: every token scaled by a power of two of its own.  (What lies behind the last row is not written: no weight comes of it.)
    for (int u = tid; u / kPer < n; u += kThreads) {
        const int t = u / kPer, dim = u % kPer * 8;
        const size_t at[1] = {base + t * P.kv_stride};
        const int dims[1] = {dim}, pos[1] = {table_row(position(t0 + t))};
        float y[1][8];
        load_turned<1>(P.dtype, P.k, at, dims, P.rot, pos, y);
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, finite_abs(y[0][e]));
#pragma unroll
        for (int o = kPer / 2; o > 0; o >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, o, 64));
        const float by = pow2(max(to_half_range(most), -126));
        half8_t a, c;
        two_parts(y[0], by, a, c);
        const int fragment = (t >> 2 & 3) * 2 * kI + dim / 64 * 2 + (dim / 8 & 1), place = (dim / 16 & 3) * 16 + (t >> 4) * 4 + (t & 3);
        char* to = P.k16 + bht * (8 * kI * 1024) + fragment * 1024 + place * 16;
        *reinterpret_cast<half8_t*>(to) = a;
        if (fine) *reinterpret_cast<half8_t*>(to + size) = c;
        if (dim == 0) P.key_scale[bht * kBlock + t] = 1.0f / by;
    }
    // values: all scaled by one power of two; one that is not finite is noted, as no weight of 0 makes it harmless
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        float y[8];
        unpack8(P.dtype, raw[i], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, finite_abs(y[e]));
    }
    most = wave_max_all(most);
    if (lane == 0) most_of[wave] = most;
    if (tid == 0) broken = 0;
    __syncthreads();
    most = __builtin_fmaxf(__builtin_fmaxf(most_of[0], most_of[1]), __builtin_fmaxf(most_of[2], most_of[3]));
    const float by = pow2(max(to_half_range(most), -126));
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int u = tid + i * kThreads, t = u / kPer, dim = u % kPer * 8;
        float y[8];
        unpack8(P.dtype, raw[i], y);
        bool good = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool finite = __builtin_fabsf(y[e]) < __builtin_inff();
            good &= finite;
            const int d = dim + e;                            // tile d / 16, half t / 8 % 2, lane (t / 16) * 16 + d % 16, place t % 8
            turned[((d / 16 * 2 + (t >> 3 & 1)) * 64 + (t >> 4) * 16 + d % 16) * 8 + (t & 7)] = static_cast<_Float16>(finite ? y[e] * by : 0.0f);
        }
        if (!good) atomicOr(&broken, 1ull << t);
    }
    __syncthreads();
    char* to = P.v16 + bht * (8 * kI * 1024);
    for (int i = tid; i < kBlock * D / 8; i += kThreads) *reinterpret_cast<half8_t*>(to + i * 16) = *reinterpret_cast<const half8_t*>(turned + i * 8);
    if (tid == 0) {
        P.value_scale[bht] = 1.0f / by;
        P.broken[bht] = broken;
    }
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

// LDS of a workgroup: blocks in flight, or the join of the wavefronts' results
template <int D, int RT, int NW, bool BYKEYS, bool FINE>
struct AttendShapeOf {
    static constexpr int kI = D / 64;                         // 64-dimension steps of a head
    static constexpr int kT = D / 16;                         // tiles of 16 dimensions; also the fragments of a block's keys, and of its values
    static constexpr int kStage = 2 * kT * 1024;              // a block; also a tile's keys, and its values, in binary16
    static constexpr int kStages = BYKEYS ? 1 : 4;
    static constexpr int kFlight = kStages * kStage * (BYKEYS ? NW : 1);
    static constexpr int kJoin = BYKEYS ? 2 * RT * kT * 64 * 16 : 0;   // two wavefronts' sums
    static constexpr int kBytes = kJoin > kFlight ? kJoin : kFlight;
};

// BYKEYS: the wavefronts take the same rows (16 RT) and each every NW-th block; otherwise each its own 16 RT rows and all blocks.
// FINE: see attend_prepare.
template <int D, int RT, int NW, bool BYKEYS, bool FINE>
__global__ __launch_bounds__(NW * 64, 2) void attend_rows(AttendParams P) {
    using Shape = AttendShapeOf<D, RT, NW, BYKEYS, FINE>;
    constexpr int kI = Shape::kI, kT = Shape::kT;
    __shared__ __align__(16) unsigned char lds[Shape::kBytes];
    __shared__ float stat[2][NW][16 * RT];                    // maximum and sum of every wavefront's columns
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int G = P.G, H = P.cache.kv_heads, R = P.R;
    const long worker = spread_over_xcds(blockIdx.x, P.workers), per = P.plan[0], total = P.plan[1 + P.B];
    const long begin = per * worker, finish = begin + per < total ? begin + per : total;
    if (worker < 0 || begin >= finish) return;
    int b = 0;                                                // the sequence in which the units begin
    for (int n = P.B; n > 1;) {                               // (of those that begin at the same unit the last one has units)
        const int half = n / 2;
        if (P.plan[1 + b + half] <= begin) b += half;
        n -= half;
    }
    long before = P.plan[1 + b];                              // units before sequence b

    for (long x = begin; x < finish;) {
        // (what follows from a thread's number is worked out anew for every item: kept in registers from one to the next, as the
        // compiler would, it leaves the loop over blocks too few of them)
        const int tid = not_kept(thread), lane = tid & 63, col = lane & 15, g = lane >> 4;
        // ---- which item, and which of its units
        while (x >= P.plan[2 + b]) before = P.plan[1 + ++b];
        const Share share = share_of(P, b);
        const int units = units_of(share), item = static_cast<int>(static_cast<unsigned>(x - before) / static_cast<unsigned>(units));
        const int group = item % share.groups, h = item / share.groups;
        const long item0 = before + static_cast<long>(item) * units;
        const int u0 = static_cast<int>(x - item0), u1 = static_cast<int>(finish - item0 < units ? finish - item0 : units);
        const int first = max(0, u0 - kStart), end = max(0, u1 - kStart);    // cached blocks, then tiles
        x = item0 + u1;

        const int len = max(0, min(P.cache.cache_len[b], P.cache.max_blocks * kBlock));
        const int rho0 = group * P.tile + (BYKEYS ? 0 : wave * 16 * RT);      // first (row, head) pair of this wavefront
        const int nrho = share.rows * G;
        const int row1 = min(share.rows - 1, (group * P.tile + P.tile - 1) / G);   // last row of the item
        const int last = min(share.blocks, end), tile0 = max(0, first - share.blocks), tile1 = min(row1 / kBlock + 1, end - share.blocks);
        const int32_t* table = P.cache.block_table + static_cast<size_t>(b) * P.cache.max_blocks;
        const size_t bh = static_cast<size_t>(b) * H + h;

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
        float4_t o[RT][kT];
        float m[RT], l[RT];                                   // maximum of s + log2(value scale); sum (of all lanes of the column)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -__builtin_inff();
            l[rt] = 0.0f;
#pragma unroll
            for (int t = 0; t < kT; ++t) o[rt][t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const _Float16 one = static_cast<_Float16>(1.0f);
        const half8_t ones = {one, one, one, one, one, one, one, one};

        // Weights of 64 tokens from their products.  With `part` only those of kept(rt) count (a bit for each of the 16 tokens of this
        // lane's group), and those of spoilt(rt) are NaN.  Their sum is a product with ones: two instructions of the matrix unit for
        // 16 additions, and it sums what the second product will use.
        auto weigh = [&](float4_t (&s)[RT][4], float ks, float vs, bool part, auto kept, auto spoilt, half8_t (&p)[RT][2]) {
            const float lift = __builtin_amdgcn_logf(vs), inv_vs = 1.0f / vs;
            float high[RT], f[RT];
            bool over = false;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                f[rt] = factor[rt] * ks;
                if (part) {
                    const unsigned keep = kept(rt);
#pragma unroll
                    for (int j = 0; j < 16; ++j) s[rt][j / 4][j % 4] = keep >> j & 1u ? s[rt][j / 4][j % 4] : -3.0e38f;
                }
                float top = s[rt][0][0];
#pragma unroll
                for (int j = 1; j < 16; ++j) top = __builtin_fmaxf(top, s[rt][j / 4][j % 4]);
                high[rt] = fmaf(top, f[rt], lift);
                over |= high[rt] > m[rt] + kLazy;
            }
            if (__any(over)) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float to = __builtin_fmaxf(m[rt], column_max(high[rt]));
                    const float by = to == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - to);
                    m[rt] = to;
                    l[rt] *= by;
#pragma unroll
                    for (int t = 0; t < kT; ++t) o[rt][t] *= by;
                }
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float from = lift - (m[rt] == -__builtin_inff() ? 0.0f : m[rt]);
                const unsigned keep = part ? kept(rt) : 0xFFFFu, spoil = part ? spoilt(rt) : 0u;
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    float2_t w;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        w[e] = __builtin_amdgcn_exp2f(fmaf(s[rt][j / 4][j % 4 + e], f[rt], from));
                        if (part) w[e] = keep >> (j + e) & 1u ? (spoil >> (j + e) & 1u ? __builtin_nanf("") : w[e]) : 0.0f;
                    }
                    const half2_t two = __builtin_convertvector(w, half2_t);
                    p[rt][j / 8][j % 8] = two.x;
                    p[rt][j / 8][j % 8 + 1] = two.y;
                }
                float4_t z = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
                z = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p[rt][0], z, 0, 0, 0);
                z = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p[rt][1], z, 0, 0, 0);
                l[rt] = fmaf(z[0], inv_vs, l[rt]);
            }
        };
        auto nothing = [](int) { return 0u; };

        // ---- cached blocks
        {
            const size_t per_block = static_cast<size_t>(H) * kBlock * D;
            const size_t layer0 = static_cast<size_t>(P.layer) * P.cache.num_blocks;
            const char* kbase = static_cast<const char*>(P.cache.k_codes) + (layer0 * H + h) * (static_cast<size_t>(kBlock) * D) + ((col >> 2) * 16 + (col & 3)) * D + g * 16;
            const char* vbase = static_cast<const char*>(P.cache.v_codes) + (layer0 * H + h) * (static_cast<size_t>(kBlock) * D) + (g * D + col) * 16;
            unsigned char* flight = lds + (BYKEYS ? wave * Shape::kStages * Shape::kStage : 0);
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
            auto sums = [&](unsigned at, const half8_t (&p)[RT][2], bool part, int mine) {
#pragma unroll
                for (int t0 = 0; t0 < kT; t0 += 4) {
                    u32x4 w[4];
                    read_4k(at + (kT + t0) * 1024, w);
                    if (part) {
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
            constexpr int kStep = BYKEYS ? NW : 1;
            // 64 blocks at a time: a lane looks up one block's number and scales
            for (int j0 = first; j0 < last; j0 += 64 * kStep) {
                const int mine0 = j0 + (BYKEYS ? wave : 0);
                const int n = min(64, (last - mine0 + kStep - 1) / kStep);   // blocks of this wavefront
                int my_id = 0;
                float my_ks = 1.0f, my_vs = 1.0f;
                bool good = false;
                if (lane < n) {
                    my_id = table[mine0 + lane * kStep];
                    good = my_id >= 0 && my_id < P.cache.num_blocks;
                    if (!good) my_id = 0;                      // in bounds, and none of its tokens counts
                    const size_t at = (layer0 + my_id) * H + h;
                    my_ks = P.cache.k_scale[at];
                    my_vs = __builtin_fmaxf(P.cache.v_scale[at], 0x1p-100f);
                }
                const unsigned long long fine = __ballot(good);
                auto id_of = [&](int i) { return static_cast<size_t>(__builtin_amdgcn_readlane(my_id, i)); };
                auto float_of = [](float y, int i) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(y), i)); };
                // tokens of the i-th block that count
                auto left_of = [&](int i) { return fine >> i & 1ull ? len - (mine0 + i * kStep) * kBlock : 0; };
                wait_fetches<0>();                            // (nothing of the loads above is counted below)
                if constexpr (BYKEYS) {
                    if (n > 0) {
                        const size_t id = id_of(0);
#pragma unroll
                        for (int f = 0; f < kT; ++f) fetch_key(id, f, flight);
#pragma unroll
                        for (int f = 0; f < kT; ++f) fetch_value(id, f, flight);
                    }
                    const unsigned at = lds_address(flight) + lane * 16;
                    for (int i = 0; i < n; ++i) {
                        const size_t next = id_of(min(i + 1, n - 1));   // (behind the last one it comes again, unused)
                        float4_t s[RT][4];
                        half8_t p[RT][2];
                        wait_fetches<kT>();
                        products(at, s);
#pragma unroll
                        for (int f = 0; f < kT; ++f) fetch_key(next, f, flight);
                        const int left = left_of(i);
                        const bool part = left < kBlock;
                        const int mine = max(0, min(16, left - 16 * g));
                        weigh(s, float_of(my_ks, i), float_of(my_vs, i), part, [&](int) { return (1u << mine) - 1u; }, nothing, p);
                        wait_fetches<kT>();
                        sums(at, p, part, mine);
#pragma unroll
                        for (int f = 0; f < kT; ++f) fetch_value(next, f, flight);
                    }
                    wait_fetches<0>();
                } else {
                    // three stages: while block i is worked on, the two behind it are under way; a wavefront fetches every NW-th fragment
                    constexpr int kMine = 2 * kT / NW;
                    static_assert(2 * kT % NW == 0, "every wavefront fetches as many fragments");
                    auto fetch_block = [&](int i) {
                        const size_t id = id_of(min(i, n - 1));
                        unsigned char* to = flight + i % 3 * Shape::kStage;
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
                    for (int i = 0; i < n; ++i) {
                        wait_fetches<kMine>();
                        __builtin_amdgcn_s_barrier();         // block i is there, and everyone is done with block i - 1
                        fetch_block(i + 2);
                        if (rho0 < nrho) {
                            const unsigned at = lds_address(flight + i % 3 * Shape::kStage) + lane * 16;
                            float4_t s[RT][4];
                            half8_t p[RT][2];
                            products(at, s);
                            const int left = left_of(i);
                            const bool part = left < kBlock;
                            const int mine = max(0, min(16, left - 16 * g));
                            weigh(s, float_of(my_ks, i), float_of(my_vs, i), part, [&](int) { return (1u << mine) - 1u; }, nothing, p);
                            sums(at, p, part, mine);
                        }
                    }
                    wait_fetches<0>();
                }
            }
        }
        // ---- the tail: the rows themselves, in binary16
        __syncthreads();
        {
            // weights and sums of tile `tile`, whose keys lie at `keys` and whose values come when values() is called
            auto one_tile = [&](int tile, auto keys, auto values) {
                const size_t bht = bh * P.tiles + tile;
                const int t0 = tile * kBlock;
                float4_t s[RT][4];
                keys(s);
                const float* scales = P.key_scale + bht * kBlock + g * 16;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const float4_t ks = *reinterpret_cast<const float4_t*>(scales + 4 * t);   // of rows 4 g .. of token tile t
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
                const unsigned spoilt = static_cast<unsigned>(P.broken[bht] >> (16 * g)) & 0xFFFFu;
                half8_t p[RT][2];
                weigh(s, 1.0f, P.value_scale[bht], true, [&](int rt) { return see[rt]; }, [&](int) { return spoilt; }, p);
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
            if constexpr (BYKEYS) {
                unsigned char* flight = lds + wave * Shape::kStage;
                const unsigned at = lds_address(flight) + lane * 16;
                auto fetch = [&](const char* from) {
#pragma unroll
                    for (int f = 0; f < 2 * kT; ++f) fetch_1k(from + f * 1024, flight + f * 1024);
                };
                for (int tile = tile0; tile < tile1; ++tile) {
                    if (tile % NW != wave) continue;
                    fetch(k16 + static_cast<size_t>(tile) * Shape::kStage);
                    one_tile(tile, [&](float4_t (&s)[RT][4]) {
                        wait_fetches<0>();
                        products16(at, first_parts, s);
                        if constexpr (FINE) {
                            fetch(k16 + size + static_cast<size_t>(tile) * Shape::kStage);
                            wait_fetches<0>();
                            products16(at, second_parts, s);
                        }
                        fetch(v16 + static_cast<size_t>(tile) * Shape::kStage);
                    }, [&](const half8_t (&p)[RT][2]) {
                        wait_fetches<0>();
                        sums16(at, p);
                    });
                }
                __syncthreads();
            } else if (tile0 < tile1) {
                // stages: keys, values (and the keys' second parts); without the latter the next tile is under way in the other two
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

        // ---- with BYKEYS the wavefronts' results are put together
        if constexpr (BYKEYS) {
            if (g == 0) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    stat[0][wave][rt * 16 + col] = m[rt];
                    stat[1][wave][rt * 16 + col] = l[rt];
                }
            }
            __syncthreads();
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float top = -__builtin_inff();
                for (int w = 0; w < NW; ++w) top = __builtin_fmaxf(top, stat[0][w][rt * 16 + col]);
                const float from = top == -__builtin_inff() ? 0.0f : top;
                float sum = 0.0f;
                for (int w = 0; w < NW; ++w) sum += stat[1][w][rt * 16 + col] * __builtin_amdgcn_exp2f(stat[0][w][rt * 16 + col] - from);
                const float by = __builtin_amdgcn_exp2f(m[rt] - from);
                m[rt] = top;
                l[rt] = sum;
#pragma unroll
                for (int t = 0; t < kT; ++t) o[rt][t] *= by;
            }
            float4_t* box = reinterpret_cast<float4_t*>(lds);
            static_assert(!BYKEYS || NW == 4, "the steps of the join");
#pragma unroll
            for (int step = 2; step >= 1; --step) {           // wavefronts 2, 3 to 0, 1, then 1 to 0
                if (wave >= step && wave < 2 * step) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int t = 0; t < kT; ++t) box[((wave - step) * RT * kT + rt * kT + t) * 64 + lane] = o[rt][t];
                }
                __syncthreads();
                if (wave < step) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int t = 0; t < kT; ++t) o[rt][t] += box[(wave * RT * kT + rt * kT + t) * 64 + lane];
                }
                __syncthreads();
            }
        }
        if (u0 == 0 && tid == 0) {                            // for the join: the item's first slot and its workers
            const long w1 = (item0 + units - 1) / per;
            P.pieces[bh * (P.row_tiles * 16 / P.tile) + group] = make_int2(static_cast<int>(2 * worker + (item0 > begin ? 1 : 0)), static_cast<int>(w1 - worker) + 1);
        }
        if (!BYKEYS || wave == 0) {
            if (u0 == 0 && u1 == units) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const int rho = rho0 + rt * 16 + col;
                    if (rho >= nrho) continue;
                    const int r = rho / G, head = h * G + (rho - r * G);
                    const float inv = 1.0f / l[rt];
                    const size_t at = ((static_cast<size_t>(b) * R + r) * P.heads + head) * D;
#pragma unroll
                    for (int t = 0; t < kT; ++t) store4(P.dtype, P.out, at + t * 16 + g * 4, o[rt][t] * inv);
                }
            } else {
                // slot 0: of the item in which this worker's units begin; slot 1: of one that begins behind that and goes on with the next worker
                float* part = P.part + (2 * static_cast<size_t>(worker) + (item0 > begin ? 1 : 0)) * P.tile * (D + 2);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const int rho = rho0 + rt * 16 + col, at = (BYKEYS ? 0 : wave * 16 * RT) + rt * 16 + col;
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
}

// Joins the items that several workers share: a wavefront a (row, head), the pieces in their order.
template <int D>
__global__ __launch_bounds__(kWG) void attend_join(AttendParams P, int per_sequence) {
    constexpr int kLanes = D / 4, kAtOnce = 64 / kLanes;      // lanes with 4 dimensions each; pieces a wavefront takes at once
    const int b = blockIdx.x / per_sequence, lane = threadIdx.x & 63, d = lane % kLanes * 4, which = lane / kLanes;
    const int nrho = (P.row_count ? max(0, min(P.row_count[b], P.R)) : P.R) * P.G, H = P.cache.kv_heads;
    const int i = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x % per_sequence) * (kWG / 64) + static_cast<int>(threadIdx.x >> 6));
    if (i >= nrho * H) return;
    const int h = i / nrho, rho = i % nrho, group = rho / P.tile, at = rho % P.tile;
    const int2 piece = P.pieces[(static_cast<size_t>(b) * H + h) * (P.row_tiles * 16 / P.tile) + group];
    const int n = piece.y;
    if (n == 1) return;
    const size_t size = static_cast<size_t>(P.tile) * (D + 2);
    // slots: the first worker's, then the first ones of the workers behind it
    auto slot = [&](int s) { return P.part + (s == 0 ? piece.x : piece.x / 2 * 2 + 2 * s) * size; };
    const size_t stat = static_cast<size_t>(P.tile) * D + 2 * at, mine = static_cast<size_t>(at) * D + d;
    float top = -__builtin_inff();
    for (int s = lane; s < n; s += 64) top = __builtin_fmaxf(top, slot(s)[stat]);
    top = wave_max_all(top);
    const float from = top == -__builtin_inff() ? 0.0f : top;
    float sum = 0.0f;
    float4_t acc = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kOnce = 8;                                  // requests in flight
    for (int s0 = 0; s0 < n; s0 += kOnce * kAtOnce) {
        float4_t y[kOnce];
        float m[kOnce], l[kOnce];
#pragma unroll
        for (int k = 0; k < kOnce; ++k) {
            const int s = s0 + k * kAtOnce + which;
            m[k] = -__builtin_inff();
            l[k] = 0.0f;
            y[k] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
            if (s < n) {
                const float* p = slot(s);
                m[k] = p[stat];
                l[k] = p[stat + 1];
                y[k] = *reinterpret_cast<const float4_t*>(p + mine);
            }
        }
#pragma unroll
        for (int k = 0; k < kOnce; ++k) {
            const float by = __builtin_amdgcn_exp2f(m[k] - from);
            sum = fmaf(l[k], by, sum);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(y[k][e], by, acc[e]);
        }
    }
#pragma unroll
    for (int o = kLanes; o < 64; o <<= 1) {
        sum += __shfl_xor(sum, o, 64);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
    }
    const int r = rho / P.G, head = h * P.G + rho % P.G;
    if (which == 0) store4(P.dtype, P.out, ((static_cast<size_t>(b) * P.R + r) * P.heads + head) * D + d, acc * (1.0f / sum));
}

}  // namespace

#endif  // FSD_CSRC_CACHE_ATTEND_H_
