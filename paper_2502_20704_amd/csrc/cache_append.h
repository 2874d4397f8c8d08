// Appending keys and values to the 8-bit paged cache (fsd_cache_append).
// Part of libfsd (gfx950); included by operators.hip, which holds the host side and the C ABI.
//
//   s = smallest 2^e, e >= -100, with |x| <= 448 s over the finite x appended to the block, but not under the block's own
//   old codes: round(code s_old / s);  new codes: round(x / s), e4m3, ties to even
//
// A piece of work is one (layer, sequence, block, head): nothing is shared between two of them, so they need not agree
// on anything.  A piece holds the block's new keys in registers (at most head_dim / 32 slots of 8 elements a lane),
// finds their largest magnitude, and writes codes; then the same for the values.  A step's accepted rows (at most 16 of them) are a
// wavefront's work, a prompt's 64 a workgroup's.
#ifndef FSD_CSRC_CACHE_APPEND_H_
#define FSD_CSRC_CACHE_APPEND_H_

#include "operators_common.h"

namespace {

constexpr int kLeastExponent = -100;

struct AppendParams {
    const char* k;
    const char* v;
    long stride;                 // elements from one token to the next
    int B, R, max_depth, max_rows;
    const int32_t* accept_len;
    const int32_t* path;         // [B, max_depth], or null
    fsd_rotation rot;
    fsd_cache cache;
    int32_t* len_out;
    int32_t* status;
    int slots;                   // blocks that a sequence's rows can touch
    unsigned npieces;
};

// 1 / s of the smallest power of two s with most <= 448 s, and s itself
__device__ __forceinline__ float block_scale(float most) {
    const unsigned bits = __float_as_uint(most);
    const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);   // 448 = 1.75 * 2^8
    return pow2(max(e, kLeastExponent));
}

// four values (of magnitude at most 448, or not finite: NaN) as e4m3 codes
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
    auto held = [](float x) { return __builtin_fabsf(x) < __builtin_inff() ? x : __builtin_nanf(""); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(held(a), held(b), 0, false);
    return static_cast<unsigned>(__builtin_amdgcn_cvt_pk_fp8_f32(held(c), held(d), w, true));
}
// four codes times a factor (<= 1), rounded again
__device__ __forceinline__ unsigned rescaled4(unsigned w, float f) {
    return codes4(__builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), 0) * f, __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), 1) * f,
                  __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), 2) * f, __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), 3) * f);
}

// LANES: the lanes that share a piece, a wavefront (at most 16 new tokens) or a workgroup (64)
template <int DT, int D, int LANES>
__global__ __launch_bounds__(kWG) void append_rows(AppendParams P) {
    constexpr int kTokens = LANES / 4;                       // new tokens a piece can hold
    constexpr int kSlots = kTokens * D / 8 / LANES;          // slots of 8 elements a lane: D / 32
    constexpr int kPer = D / 8;                              // slots of a token
    // the values' codes change places here: [group of 16 tokens][d][16], a token's byte for 8 consecutive d from one lane
    __shared__ float most_of[8];
    __shared__ __align__(16) unsigned char turned[LANES == kWG ? D * kBlock : 16];
    __shared__ int bad_any;
    const int lane = threadIdx.x % LANES;
    const int H = P.cache.kv_heads;
    const unsigned piece = blockIdx.x * (kWG / LANES) + threadIdx.x / LANES;
    if (piece >= P.npieces) return;                           // (wavefronts of the last workgroup; a whole workgroup never)
    const int h = static_cast<int>(piece % H);
    const int slot = static_cast<int>(piece / H % P.slots);
    const int b = static_cast<int>(piece / H / P.slots % P.B), layer = static_cast<int>(piece / H / P.slots / P.B);

    const long len = P.cache.cache_len[b];
    const long count = static_cast<long>(P.accept_len[b]) + 1;
    const long room = static_cast<long>(P.cache.max_blocks) * kBlock;
    const int32_t* path = P.path ? P.path + static_cast<size_t>(b) * P.max_depth : nullptr;
    const int32_t* table = P.cache.block_table + static_cast<size_t>(b) * P.cache.max_blocks;
    // the sequence is appended whole or not at all: every piece looks at all of it
    bool bad = count < 0 || count > P.max_rows || len < 0 || len + count > room ||
               (count > 0 && P.rot.table != nullptr && len + count > P.rot.rows);
    if (!bad && count > 0) {
        if (path)
            for (int i = lane; i < count - 1; i += LANES) bad |= path[i] < 0 || path[i] >= P.R - 1;
        for (long i = len / kBlock + lane; i <= (len + count - 1) / kBlock; i += LANES) bad |= table[i] < 0 || table[i] >= P.cache.num_blocks;
    }
    if constexpr (LANES == 64) {
        bad = __any(bad);
    } else {
        if (threadIdx.x == 0) bad_any = 0;
        __syncthreads();
        if (bad) bad_any = 1;
        __syncthreads();
        bad = bad_any != 0;
    }
    if (h == 0 && slot == 0 && layer == 0 && lane == 0) {
        if (P.len_out) P.len_out[b] = static_cast<int32_t>(bad ? len : len + count);
        if (P.status) P.status[b] = bad ? FSD_ROW_BAD_CACHE : 0;
    }
    if (bad || count <= 0) return;
    const long block = len / kBlock + slot;                   // of the sequence
    const long from = block * kBlock > len ? block * kBlock : len, to = (block + 1) * kBlock < len + count ? (block + 1) * kBlock : len + count;
    if (from >= to) return;
    const int fill = static_cast<int>(from - block * kBlock);   // tokens of the sequence that the block holds already
    const int n = static_cast<int>(to - from);
    const size_t at = (static_cast<size_t>(layer) * P.cache.num_blocks + table[block]) * H + h;   // block and head
    unsigned char* kc = static_cast<unsigned char*>(P.cache.k_codes) + at * (kBlock * D);
    unsigned char* vc = static_cast<unsigned char*>(P.cache.v_codes) + at * (kBlock * D);

    float x[kSlots][8];
    auto largest = [&]() {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < kSlots; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = __builtin_fmaxf(m, finite_abs(x[i][e]));
        m = wave_max_all(m);
        if constexpr (LANES != 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) most_of[threadIdx.x >> 6] = m;
            __syncthreads();
            m = __builtin_fmaxf(__builtin_fmaxf(most_of[0], most_of[1]), __builtin_fmaxf(most_of[2], most_of[3]));
        }
        return m;
    };
    size_t head[kSlots];
    int dim[kSlots], pos[kSlots];
    bool there[kSlots];
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
        const int u = lane + i * LANES, t = u / kPer;
        there[i] = t < n;
        const long i0 = from - len + (there[i] ? t : 0);      // which of the accepted rows (the first one where there is none)
        const long row = path == nullptr || i0 == 0 ? i0 : path[i0 - 1] + 1;
        head[i] = (static_cast<size_t>(static_cast<long>(layer) * P.B + b) * P.R + row) * P.stride + static_cast<size_t>(h) * D;
        dim[i] = u % kPer * 8;
        pos[i] = static_cast<int>(len + i0);
    }
    auto blank = [&]() {
#pragma unroll
        for (int i = 0; i < kSlots; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = there[i] ? x[i][e] : 0.0f;
    };
    // the scale in force, and what the old codes are multiplied by
    auto scale_of = [&](float* scale, float most, float& ratio) {
        float s = block_scale(most);
        ratio = 1.0f;
        if (fill > 0) {
            const float old = scale[at];
            s = __builtin_fmaxf(s, old);
            ratio = old / s;
        }
        return s;
    };
    // ---- keys
    load_turned<kSlots>(DT, P.k, head, dim, P.rot, pos, x);
    blank();
    {
        float ratio;
        const float s = scale_of(P.cache.k_scale, largest(), ratio), inv = 1.0f / s;
        if (ratio != 1.0f) {
            unsigned* w = reinterpret_cast<unsigned*>(kc);
            for (int i = lane; i < fill * (D / 4); i += LANES) w[i] = rescaled4(w[i], ratio);
        }
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            const int u = lane + i * LANES, t = u / kPer, d = u % kPer * 8;
            if (t < n) {
                uint2 w;
                w.x = codes4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv);
                w.y = codes4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv);
                *reinterpret_cast<uint2*>(kc + (fill + t) * D + d) = w;
            }
        }
        // (every lane has read the old scale: the barriers or the shuffles of `largest` of the values stand between)
#pragma unroll
        for (int i = 0; i < kSlots; ++i) load8<DT>(P.v, head[i] + dim[i], x[i]);
        blank();
        const float most = largest();
        if (lane == 0) P.cache.k_scale[at] = s;
        float vratio;
        const float vs = scale_of(P.cache.v_scale, most, vratio), vinv = 1.0f / vs;
        if constexpr (LANES == 64) {
            // few tokens: the bytes go straight to their places; old ones first, in words of 4 tokens
            if (vratio != 1.0f) {
                const int words = (fill + 3) / 4;             // of a row of d: 4 a group
                for (int i = lane; i < words * D; i += 64) {
                    const int q = i / D, d = i % D;
                    unsigned* w = reinterpret_cast<unsigned*>(vc + (q / 4 * D + d) * 16) + q % 4;
                    const unsigned old = *w, keep = q * 4 + 4 <= fill ? 0u : ~0u << (8 * (fill - q * 4));
                    *w = (rescaled4(old, vratio) & ~keep) | (old & keep);
                }
                __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");   // before the new bytes of the same words
            }
#pragma unroll
            for (int i = 0; i < kSlots; ++i) {
                const int u = lane + i * LANES, t = u / kPer, d = u % kPer * 8;
                if (t < n) {
                    const int place = fill + t;
                    unsigned char* p = vc + (place / 16 * D + d) * 16 + place % 16;
                    const unsigned lo = codes4(x[i][0] * vinv, x[i][1] * vinv, x[i][2] * vinv, x[i][3] * vinv);
                    const unsigned hi = codes4(x[i][4] * vinv, x[i][5] * vinv, x[i][6] * vinv, x[i][7] * vinv);
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e * 16] = static_cast<unsigned char>((e < 4 ? lo : hi) >> (e % 4 * 8));
                }
            }
        } else {
            // the whole block is put together in LDS and written in 16-byte pieces, one group of 16 tokens of one d each
#pragma unroll
            for (int i = 0; i < kSlots; ++i) {
                const int u = lane + i * LANES, t = u / kPer, d = u % kPer * 8;
                const int place = fill + t;
                if (t < n) {
                    unsigned char* p = turned + (place / 16 * D + d) * 16 + place % 16;
                    const unsigned lo = codes4(x[i][0] * vinv, x[i][1] * vinv, x[i][2] * vinv, x[i][3] * vinv);
                    const unsigned hi = codes4(x[i][4] * vinv, x[i][5] * vinv, x[i][6] * vinv, x[i][7] * vinv);
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e * 16] = static_cast<unsigned char>((e < 4 ? lo : hi) >> (e % 4 * 8));
                }
            }
            __syncthreads();
            const int end = fill + n;
            for (int i = lane; i < (kBlock / 16) * D; i += LANES) {
                const int first = i / D * 16;                 // of the group's tokens
                if (first >= end) continue;
                unsigned* to = reinterpret_cast<unsigned*>(vc + static_cast<size_t>(i) * 16);
                const unsigned* made = reinterpret_cast<const unsigned*>(turned + static_cast<size_t>(i) * 16);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int t0 = first + q * 4;             // the word's first token
                    if (t0 >= end) continue;
                    unsigned w = made[q];
                    if (t0 < fill || t0 + 4 > end) {          // a word that is not new throughout
                        unsigned old = to[q];
                        unsigned is_new = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (t0 + e >= fill && t0 + e < end) is_new |= 0xFFu << (8 * e);
                        if (vratio != 1.0f && t0 < fill) old = rescaled4(old, vratio);
                        w = (w & is_new) | (old & ~is_new);
                    }
                    to[q] = w;
                }
            }
        }
        if constexpr (LANES != 64) __syncthreads();           // (every lane has read the old scale)
        if (lane == 0) P.cache.v_scale[at] = vs;
    }
}

}  // namespace

#endif  // FSD_CSRC_CACHE_APPEND_H_
