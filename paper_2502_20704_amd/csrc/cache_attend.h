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
// The rows themselves (the tail) are turned, scaled by powers of two into binary16's range and laid out in LDS as a cache block
// is, 64 of them at a time, and go through the same code, with the mask of the chain or the tree.
//
// Work is dealt by the kernel itself, which alone knows the lengths: pieces of `chunk` blocks of one (sequence, key head, rows),
// chunk chosen so that the device is filled about once.  Pieces of a sequence that has several are joined by attend_join.
#ifndef FSD_CSRC_CACHE_ATTEND_H_
#define FSD_CSRC_CACHE_ATTEND_H_

#include "operators_common.h"

namespace {

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
    float* part;                   // partial results, one for every piece: [rows of a piece][D], then [rows][2]
    int target;                    // pieces aimed at
    int least;                     // blocks of a piece, at least
    int tile;                      // rows of a piece
};

// What a sequence's share of the work is: rows and cache blocks, and pieces once the chunk is known
struct Share { int rows, blocks, groups; };
__device__ __forceinline__ Share share_of(const AttendParams& P, int b) {
    Share s;
    const int most = P.cache.max_blocks * kBlock;
    s.rows = P.row_count ? max(0, min(P.row_count[b], P.R)) : P.R;
    s.blocks = (max(0, min(P.cache.cache_len[b], most)) + kBlock - 1) / kBlock;
    s.groups = (s.rows * P.G + P.tile - 1) / P.tile;
    return s;
}
__device__ __forceinline__ int splits_of(const Share& s, int chunk) { return max(1, (s.blocks + chunk - 1) / chunk); }

// The chunk (blocks of a piece), and which piece workgroup `block` has: sequence b (-1: none is left), piece `local` of it.  With a
// `sequence` (>= 0) that one's first slot instead.  All threads of the workgroup call it.
struct Dealt { int chunk, b, local, slot; };   // slot: of the first piece of b, among those that need one
__device__ __forceinline__ Dealt deal(const AttendParams& P, long block, int sequence) {
    __shared__ long sums[kWG / 64];
    __shared__ long carry_of[kWG / 64];
    __shared__ int found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    long mine = 0;
    for (int b = tid; b < P.B; b += kWG) {
        const Share s = share_of(P, b);
        mine += static_cast<long>(s.blocks) * s.groups;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
    if (lane == 0) sums[wave] = mine;
    if (tid < 3) found[tid] = -1;
    __syncthreads();
    const long all = (sums[0] + sums[1] + sums[2] + sums[3]) * P.cache.kv_heads;
    Dealt d;
    d.chunk = static_cast<int>(max(static_cast<long>(P.least), (all + P.target - 1) / P.target));
    // first over everything (how many pieces there are), then the wanted one; sums of pieces below, above them sums of the
    // pieces of sequences that have several (those need a slot: twice the target at most, as ceil(x) <= 2 x for x > 1)
    long base = 0, wanted = -1;
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1) {
            if (sequence < 0) wanted = spread_over_xcds(block, base & 0xFFFFFFFFl);
            base = 0;
        }
        for (int b0 = 0; b0 < P.B; b0 += kWG) {
            const int b = b0 + tid;
            long n = 0;
            if (b < P.B) {
                const Share s = share_of(P, b);
                const int splits = splits_of(s, d.chunk);
                n = static_cast<long>(splits) * s.groups * P.cache.kv_heads;
                if (splits > 1) n |= n << 32;
            }
            long up = n;                                      // inclusive sum over the wavefront
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const long y = __shfl_up(up, o, 64);
                if (lane >= o) up += y;
            }
            __syncthreads();
            if (lane == 63) carry_of[wave] = up;
            __syncthreads();
            long before = base;
            for (int w = 0; w < wave; ++w) before += carry_of[w];
            before += up - n;
            const long first = before & 0xFFFFFFFFl;
            if (pass == 1 && b < P.B && (sequence >= 0 ? b == sequence : wanted >= first && wanted < first + (n & 0xFFFFFFFFl))) {
                found[0] = b;
                found[1] = static_cast<int>(wanted - first);
                found[2] = static_cast<int>(before >> 32);
            }
            for (int w = 0; w < kWG / 64; ++w) base += carry_of[w];
        }
        __syncthreads();
    }
    d.b = found[0];
    d.local = found[1];
    d.slot = found[2];
    return d;
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
__device__ __forceinline__ void load8_16bit(int dtype, const void* base, size_t at, float* x) {
    if (dtype == FSD_BF16) load8<FSD_BF16>(base, at, x);
    else load8<FSD_F16>(base, at, x);
}
__device__ __forceinline__ void load8_16bit_turned(int dtype, const void* base, size_t at, int d, const fsd_rotation& rot, int pos, float* x) {
    if (dtype == FSD_BF16) load8_turned<FSD_BF16>(base, at, d, rot, pos, x);
    else load8_turned<FSD_F16>(base, at, d, rot, pos, x);
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

// LDS of a piece: the tail's keys and values, or the join of the wavefronts' results; then the tree
template <int D, int RT, bool BYKEYS>
struct AttendLds {
    static constexpr int kKeyRow = D + 8;                                    // binary16, padded: rows on other banks
    static constexpr int kTail = kBlock * kKeyRow * 2 + kBlock * D * 2;
    static constexpr int kJoin = BYKEYS ? 2 * RT * (D / 16) * 64 * 16 : 0;   // two wavefronts' sums
    static constexpr int kBytes = kTail > kJoin ? kTail : kJoin;
};

// BYKEYS: the four wavefronts take the same rows (16 RT) and every fourth block; otherwise each its own 16 RT rows and all blocks
template <int D, int RT, bool BYKEYS>
__global__ __launch_bounds__(kWG) void attend_rows(AttendParams P) {
    using Lds = AttendLds<D, RT, BYKEYS>;
    constexpr int kI = D / 64;                                // 64-dimension steps of a head
    constexpr int kT = D / 16;                                // tiles of 16 dimensions
    __shared__ __align__(16) unsigned char lds[Lds::kBytes];
    __shared__ float stat[2][4][16 * RT];                     // maximum and sum of every wavefront's columns
    __shared__ float most_of[2][4];
    __shared__ unsigned long long broken;                     // tokens of the tail's tile with a value that is not finite
    __shared__ unsigned long long sees[kWG + 8];              // rows of the tail's tile that a row of the piece sees
    extern __shared__ short tree[];                           // trees: [R] parent's row, [R] depth, [R] row where a walk stands
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;

    const Dealt d = deal(P, blockIdx.x, -1);
    if (blockIdx.x == 0 && P.status)                          // sequences without rows have no piece to report them
        for (int b = tid; b < P.B; b += kWG)
            if (share_of(P, b).rows == 0) P.status[b] = P.row_count[b] < 0 ? FSD_ROW_BAD_CACHE : 0;
    if (d.b < 0) return;
    const int b = d.b;
    const Share share = share_of(P, b);
    const int splits = splits_of(share, d.chunk);
    const int group = d.local % share.groups, split = d.local / share.groups % splits, h = d.local / share.groups / splits;
    const int len = max(0, min(P.cache.cache_len[b], P.cache.max_blocks * kBlock));
    const int G = P.G, H = P.cache.kv_heads, R = P.R;
    const int ntail = share.rows;
    const int rho0 = group * P.tile + (BYKEYS ? 0 : wave * 16 * RT);      // first (row, head) pair of this wavefront
    const int nrho = share.rows * G;
    const int row0 = group * P.tile / G, row1 = min(share.rows - 1, (group * P.tile + P.tile - 1) / G);   // rows of the piece
    short* up = tree;
    short* depth = tree + R;
    short* stands = tree + 2 * R;
    bool bad_tree = false;
    if (P.parent) {
        // depths by doubling: after step i a row knows its 2^i-th ancestor and how far that is
        const int32_t* parent = P.parent + static_cast<size_t>(b) * (R - 1);
        for (int r = tid; r < R; r += kWG) {
            int p = -1;                                       // row 0 has none
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
            constexpr int kEach = (kMaxNodes + kWG) / kWG;
            short jump[kEach], more[kEach];
            bool moved = false;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = tid + i * kWG, p = r < R ? stands[r] : -1;
                jump[i] = p > 0 ? stands[p] : static_cast<short>(-1);
                more[i] = p > 0 ? depth[p] : static_cast<short>(0);
                moved |= p > 0;
            }
            if (!__syncthreads_or(moved)) break;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = tid + i * kWG;
                if (r >= R) continue;
                depth[r] = static_cast<short>(depth[r] + more[i]);
                stands[r] = jump[i];
            }
            __syncthreads();
        }
        for (int r = tid; r < R; r += kWG) stands[r] = static_cast<short>(r);
        __syncthreads();
    }
    auto position = [&](int r) { return len + (P.parent ? depth[r] : r); };
    auto table_row = [&](int pos) { return P.rot.table ? min(pos, P.rot.rows - 1) : 0; };
    const int32_t* table = P.cache.block_table + static_cast<size_t>(b) * P.cache.max_blocks;

    if (h == 0 && group == 0 && split == 0 && P.status) {     // this piece reports the sequence
        bool bad = P.cache.cache_len[b] < 0 || P.cache.cache_len[b] > P.cache.max_blocks * kBlock ||
                   (P.row_count && (P.row_count[b] < 0 || P.row_count[b] > R));
        for (int i = tid; i < share.blocks; i += kWG) bad |= table[i] < 0 || table[i] >= P.cache.num_blocks;
        if (P.rot.table)
            for (int r = tid; r < share.rows; r += kWG) bad |= position(r) >= P.rot.rows;
        bad = __syncthreads_or(bad);
        if (tid == 0) P.status[b] = (bad ? FSD_ROW_BAD_CACHE : 0) | (bad_tree ? FSD_ROW_BAD_PARENT : 0);
    }

    // ---- queries: turned, and scaled by a power of two for each row so that binary16 holds them
    half8_t q[RT][2 * kI];
    float factor[RT];                                         // of the products of a row: its power of two back, scale, log2(e)
    int row_of[RT];                                           // the row, -1 behind the last
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int rho = rho0 + rt * 16 + col;
        const bool there = rho < nrho;
        const int r = there ? rho / G : 0, head = h * G + (there ? rho - r * G : 0);
        row_of[rt] = there ? r : -1;
        float x[2 * kI][8];
        float most = 0.0f;
        const size_t at = (static_cast<size_t>(b) * R + r) * P.q_stride + static_cast<size_t>(head) * D;
        const int pos = table_row(position(r));
#pragma unroll
        for (int i = 0; i < 2 * kI; ++i) {
            load8_16bit_turned(P.dtype, P.q, at, (i / 2) * 64 + g * 16 + (i & 1) * 8, P.rot, pos, x[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, finite_abs(x[i][e]));
        }
        most = column_max(most);
        const int e2 = to_half_range(most);
        const float by = pow2(max(e2, -126));
#pragma unroll
        for (int i = 0; i < 2 * kI; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) q[rt][i][e] = static_cast<_Float16>(x[i][e] * by);
        factor[rt] = P.scale / by;
    }
    float4_t o[RT][kT];
    float m[RT], l[RT];                                       // of s + log2(value scale); the sum is this lane's tokens' alone
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -__builtin_inff();
        l[rt] = 0.0f;
#pragma unroll
        for (int t = 0; t < kT; ++t) o[rt][t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // weights of 64 tokens from their products; keep(rt) has a bit for each of the 16 tokens of this lane's group
    auto weigh = [&](float4_t (&s)[RT][4], float ks, float vs, auto keep, half8_t (&p)[RT][2]) {
        const float lift = __builtin_amdgcn_logf(vs), inv_vs = 1.0f / vs;
        float high[RT];
        bool over = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float f = factor[rt] * ks;
            const unsigned kept = keep(rt);
            high[rt] = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = fmaf(s[rt][j][i], f, lift);
                    x = kept >> (4 * j + i) & 1u ? x : -__builtin_inff();
                    s[rt][j][i] = x;
                    high[rt] = __builtin_fmaxf(high[rt], x);
                }
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
            const float from = m[rt] == -__builtin_inff() ? 0.0f : m[rt];
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = __builtin_amdgcn_exp2f(s[rt][j][i] - from);
                    sum += w;
                    p[rt][j / 2][(j & 1) * 4 + i] = static_cast<_Float16>(w);
                }
            l[rt] = fmaf(sum, inv_vs, l[rt]);
        }
    };

    // ---- cached blocks
    const int first = split * d.chunk, last = min(share.blocks, first + d.chunk);
    const size_t per_block = static_cast<size_t>(H) * kBlock * D;
    const size_t layer0 = static_cast<size_t>(P.layer) * P.cache.num_blocks;
    const char* kbase = static_cast<const char*>(P.cache.k_codes) + layer0 * per_block + static_cast<size_t>(h) * kBlock * D;
    const char* vbase = static_cast<const char*>(P.cache.v_codes) + layer0 * per_block + static_cast<size_t>(h) * kBlock * D;
    for (int j = first + (BYKEYS ? wave : 0); j < last; j += BYKEYS ? 4 : 1) {
        const int id = table[j];
        if (id < 0 || id >= P.cache.num_blocks) continue;
        const char* kb = kbase + id * per_block;
        const char* vb = vbase + id * per_block;
        u32x4 kw[4][kI], vw[kT];
        const int token = (col >> 2) * 16 + (col & 3);        // + 4 s
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < kI; ++i)
                kw[s][i] = *reinterpret_cast<const u32x4*>(kb + (token + 4 * s) * D + i * 64 + g * 16);
#pragma unroll
        for (int t = 0; t < kT; ++t) vw[t] = *reinterpret_cast<const u32x4*>(vb + (g * D + t * 16 + col) * 16);
        const size_t si = (layer0 + id) * H + h;
        const float ks = P.cache.k_scale[si], vs = __builtin_fmaxf(P.cache.v_scale[si], 0x1p-100f);
        float4_t s[RT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            half8_t kf[2 * kI];
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                kf[2 * i] = widened(kw[t][i].x, kw[t][i].y);
                kf[2 * i + 1] = widened(kw[t][i].z, kw[t][i].w);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                s[rt][t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 2 * kI; ++i) s[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i], q[rt][i], s[rt][t], 0, 0, 0);
            }
        }
        half8_t p[RT][2];
        const int left = len - j * kBlock;                    // tokens of the sequence in this block
        unsigned held = 0xFFFFu;                              // of the 16 of this lane's group
        if (left < kBlock) {
            const int mine = max(0, min(16, left - 16 * g));
            held = (1u << mine) - 1u;
            // what lies behind the last token may be anything: a weight of 0 would not make a NaN harmless
#pragma unroll
            for (int t = 0; t < kT; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int bytes = max(0, min(4, mine - 4 * w));
                    vw[t][w] = bytes == 4 ? vw[t][w] : vw[t][w] & ((1u << (8 * bytes)) - 1u);
                }
        }
        weigh(s, ks, vs, [&](int) { return held; }, p);
#pragma unroll
        for (int t = 0; t < kT; ++t) {
            const half8_t v0 = widened(vw[t].x, vw[t].y), v1 = widened(vw[t].z, vw[t].w);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[rt][0], o[rt][t], 0, 0, 0);
                o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[rt][1], o[rt][t], 0, 0, 0);
            }
        }
    }

    // ---- the tail: the rows themselves, 64 at a time from the last ones any row of the piece sees
    if (split == splits - 1) {
        _Float16* tk = reinterpret_cast<_Float16*>(lds);
        _Float16* tv = tk + kBlock * Lds::kKeyRow;
        for (int tile = row1 / kBlock; tile >= 0; --tile) {
            const int t0 = tile * kBlock, n = min(kBlock, ntail - t0);
            constexpr int kPer = D / 8, kUnits = kBlock * kPer / kWG;
            float x[kUnits][8];
            float scale_k = 1.0f, scale_v = 1.0f;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < kUnits; ++i) {
                    const int u = tid + i * kWG, t = u / kPer, dim = u % kPer * 8;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
                    if (t < n) {
                        const size_t at = (static_cast<size_t>(b) * R + t0 + t) * P.kv_stride + static_cast<size_t>(h) * D;
                        if (which == 0) load8_16bit_turned(P.dtype, P.k, at, dim, P.rot, table_row(position(t0 + t)), x[i]);
                        else load8_16bit(P.dtype, P.v, at + dim, x[i]);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) most = __builtin_fmaxf(most, finite_abs(x[i][e]));
                }
                most = wave_max_all(most);
                if (lane == 0) most_of[which][wave] = most;
                if (which == 0 && tid == 0) broken = 0;
                __syncthreads();                              // (also: the tile before this one is no longer read)
                most = __builtin_fmaxf(__builtin_fmaxf(most_of[which][0], most_of[which][1]), __builtin_fmaxf(most_of[which][2], most_of[which][3]));
                const float by = pow2(max(to_half_range(most), -126));
                (which == 0 ? scale_k : scale_v) = 1.0f / by;
#pragma unroll
                for (int i = 0; i < kUnits; ++i) {
                    const int u = tid + i * kWG, t = u / kPer, dim = u % kPer * 8;
                    half8_t y;
                    if (which == 1) {                         // no weight of 0 makes them harmless to rows that do not see them
                        bool fine = true;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const bool good = __builtin_fabsf(x[i][e]) < __builtin_inff();
                            x[i][e] = good ? x[i][e] : 0.0f;
                            fine &= good;
                        }
                        if (!fine) atomicOr(&broken, 1ull << t);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = static_cast<_Float16>(x[i][e] * by);
                    if (which == 0) {
                        *reinterpret_cast<half8_t*>(tk + t * Lds::kKeyRow + dim) = y;
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) tv[(t / 16 * D + dim + e) * 16 + t % 16] = y[e];
                    }
                }
            }
            if (P.parent) {                                   // who of this tile lies on the way to a row of the piece
                for (int r = row0 + tid; r <= row1; r += kWG) {
                    unsigned long long bits = 0;
                    int at = stands[r];
                    for (; at >= t0; at = up[at]) bits |= 1ull << (at - t0);
                    stands[r] = static_cast<short>(at);
                    sees[r - row0] = bits;
                }
            }
            __syncthreads();
            if (BYKEYS ? (tile & 3) == wave : rho0 < nrho && (rho0 + 16 * RT - 1) / G >= t0) {
                float4_t s[RT][4];
                const int token = (col >> 2) * 16 + (col & 3);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    half8_t kf[2 * kI];
#pragma unroll
                    for (int i = 0; i < 2 * kI; ++i)
                        kf[i] = *reinterpret_cast<const half8_t*>(tk + (token + 4 * t) * Lds::kKeyRow + (i / 2) * 64 + g * 16 + (i & 1) * 8);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        s[rt][t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int i = 0; i < 2 * kI; ++i) s[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i], q[rt][i], s[rt][t], 0, 0, 0);
                    }
                }
                half8_t p[RT][2];
                auto keep = [&](int rt) -> unsigned {
                    const int r = row_of[rt];
                    if (r < 0) return 0u;
                    if (P.parent) return static_cast<unsigned>(sees[r - row0] >> (16 * g)) & 0xFFFFu;
                    const int upto = max(0, min(16, r - t0 - 16 * g + 1));     // rows t0 + 16 g .. r
                    return (1u << upto) - 1u;
                };
                weigh(s, scale_k, scale_v, keep, p);
                if (broken != 0) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
                        if (keep(rt) & static_cast<unsigned>(broken >> (16 * g)) & 0xFFFFu) l[rt] = __builtin_nanf("");
                }
#pragma unroll
                for (int t = 0; t < kT; ++t) {
                    const half8_t* from = reinterpret_cast<const half8_t*>(tv + (g * D + t * 16 + col) * 16);
                    const half8_t v0 = from[0], v1 = from[1];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[rt][0], o[rt][t], 0, 0, 0);
                        o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[rt][1], o[rt][t], 0, 0, 0);
                    }
                }
            }
            __syncthreads();
        }
    }

    // ---- the columns' sums, and with BYKEYS the four wavefronts' results put together
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) l[rt] = column_sum(l[rt]);
    if constexpr (BYKEYS) {
        __syncthreads();
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
            for (int w = 0; w < 4; ++w) top = __builtin_fmaxf(top, stat[0][w][rt * 16 + col]);
            const float from = top == -__builtin_inff() ? 0.0f : top;
            float sum = 0.0f;
            for (int w = 0; w < 4; ++w) sum += stat[1][w][rt * 16 + col] * __builtin_amdgcn_exp2f(stat[0][w][rt * 16 + col] - from);
            const float by = __builtin_amdgcn_exp2f(m[rt] - from);
            m[rt] = top;
            l[rt] = sum;
#pragma unroll
            for (int t = 0; t < kT; ++t) o[rt][t] *= by;
        }
        float4_t* box = reinterpret_cast<float4_t*>(lds);
#pragma unroll
        for (int step = 2; step >= 1; --step) {               // wavefronts 2, 3 to 0, 1, then 1 to 0
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
        if (wave != 0) return;
    }
    if (splits == 1) {
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
        float* part = P.part + static_cast<size_t>(d.slot + d.local) * P.tile * (D + 2);
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

// Joins the pieces of a sequence that has several: a wavefront a (row, head), the pieces in their order.
template <int D>
__global__ __launch_bounds__(kWG) void attend_join(AttendParams P, int per_sequence) {
    const int b = blockIdx.x / per_sequence;
    const Dealt d = deal(P, 0, b);
    const Share share = share_of(P, b);
    const int splits = splits_of(share, d.chunk);
    if (splits == 1) return;
    const int lane = threadIdx.x & 63, nrho = share.rows * P.G;
    const int i = blockIdx.x % per_sequence * (kWG / 64) + (threadIdx.x >> 6);
    if (i >= nrho * P.cache.kv_heads) return;
    const int h = i / nrho, rho = i % nrho, group = rho / P.tile, at = rho % P.tile;
    const size_t size = static_cast<size_t>(P.tile) * (D + 2);
    const float* part = P.part + (static_cast<size_t>(d.slot) + static_cast<size_t>(h) * splits * share.groups + group) * size;
    const size_t step = static_cast<size_t>(share.groups) * size;
    float top = -__builtin_inff();
    for (int s = lane; s < splits; s += 64) top = __builtin_fmaxf(top, part[s * step + static_cast<size_t>(P.tile) * D + 2 * at]);
    top = wave_max_all(top);
    const float from = top == -__builtin_inff() ? 0.0f : top;
    float sum = 0.0f, acc[D / 64];
#pragma unroll
    for (int e = 0; e < D / 64; ++e) acc[e] = 0.0f;
    for (int s = 0; s < splits; ++s) {
        const float* p = part + s * step;
        const float by = __builtin_amdgcn_exp2f(p[static_cast<size_t>(P.tile) * D + 2 * at] - from);
        sum = fmaf(p[static_cast<size_t>(P.tile) * D + 2 * at + 1], by, sum);
#pragma unroll
        for (int e = 0; e < D / 64; ++e) acc[e] = fmaf(p[static_cast<size_t>(at) * D + lane + e * 64], by, acc[e]);
    }
    const int r = rho / P.G, head = h * P.G + rho % P.G;
    const size_t to = ((static_cast<size_t>(b) * P.R + r) * P.heads + head) * D;
    const float inv = 1.0f / sum;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
        const float y = acc[e] * inv;
        unsigned short* out = static_cast<unsigned short*>(P.out) + to + lane + e * 64;
        if (P.dtype == FSD_BF16) *out = static_cast<unsigned short>(bf16_bits(y));
        else *out = __builtin_bit_cast(unsigned short, static_cast<_Float16>(y));
    }
}

}  // namespace

#endif  // FSD_CSRC_CACHE_ATTEND_H_
