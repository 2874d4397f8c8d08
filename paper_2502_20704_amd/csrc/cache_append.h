// Appending keys and values to the 8-bit paged cache (fsd_cache_append).
// Part of libfsd (gfx950); included by operators.hip, which holds the host side and the C ABI.
//
//   s = smallest 2^e, e >= -100, with |x| <= 448 s over the finite x appended to the block, but not under the block's own
//   old codes: round(code s_old / s);  new codes: round(x / s), e4m3, ties to even
//
// A block of a head is one piece of work: nothing is shared between two of them, so they need not agree on anything.  Its new keys
// are in registers when their largest magnitude is known, and are then written as codes; so are its new values, which are requested
// together with the keys.  What bounds both kernels is how much is requested at once.
//   append_few   a step's accepted rows (at most 16): a wavefront a head, which takes the blocks they touch (one, seldom two) in turn
//   append_many  a prompt's: a workgroup a block and head
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
    int slots;                   // append_many: blocks that a sequence's rows can touch
    unsigned npieces;
};

// 1 / s of the smallest power of two s with most <= 448 s, and s itself
__device__ __forceinline__ float block_scale(float most) {
    const unsigned bits = __float_as_uint(most);
    const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);   // 448 = 1.75 * 2^8
    return pow2(max(e, kLeastExponent));
}

// four values of magnitude at most 448 as e4m3 codes; one that is not finite becomes NaN, as all beyond the range do
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<unsigned>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}
// four codes times a factor (<= 1), rounded again
__device__ __forceinline__ unsigned rescaled4(unsigned w, float f) {
    return codes4(__builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), 0) * f, __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), 1) * f,
                  __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), 2) * f, __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), 3) * f);
}

// What a sequence's rows need to be appended.  It is appended whole or not at all: every piece looks at all of it.
struct Appended {
    long len, count;
    const int32_t* path;
    const int32_t* table;
    int R;
    bool bad;                    // lengths or positions out of range; the same for everyone
    __device__ __forceinline__ Appended(const AppendParams& P, int b) {
        len = P.cache.cache_len[b];
        count = static_cast<long>(P.accept_len[b]) + 1;
        path = P.path ? P.path + static_cast<size_t>(b) * P.max_depth : nullptr;
        table = P.cache.block_table + static_cast<size_t>(b) * P.cache.max_blocks;
        R = P.R;
        bad = count < 0 || count > P.max_rows || len < 0 || len + count > static_cast<long>(P.cache.max_blocks) * kBlock ||
              (count > 0 && P.rot.table != nullptr && len + count > P.rot.rows);
    }
    // whether this lane finds a path node or a block out of range (asked where the lengths are in range, and something is appended)
    __device__ __forceinline__ bool look(const AppendParams& P, int lane, int lanes) const {
        bool found = false;
        if (path)
#pragma unroll 1
            for (int i = lane; i < count - 1; i += lanes) found |= path[i] < 0 || path[i] >= P.R - 1;
#pragma unroll 1
        for (long i = len / kBlock + lane; i <= (len + count - 1) / kBlock; i += lanes) found |= table[i] < 0 || table[i] >= P.cache.num_blocks;
        return found;
    }
    // row of k and v that is the i-th to be appended (in bounds, also where it has not been looked at)
    __device__ __forceinline__ long row(long i) const { return path == nullptr || i == 0 ? i : max(0, min(R - 1, path[i - 1] + 1)); }
};
__device__ __forceinline__ void report(const AppendParams& P, int b, const Appended& a, bool bad) {
    if (P.len_out) P.len_out[b] = static_cast<int32_t>(bad ? a.len : a.len + a.count);
    if (P.status) P.status[b] = bad ? FSD_ROW_BAD_CACHE : 0;
}
// the scale in force, and what old codes are multiplied by
__device__ __forceinline__ float scale_in_force(float most, int fill, float old, float& ratio) {
    float s = block_scale(most);
    ratio = 1.0f;
    if (fill > 0) {
        s = __builtin_fmaxf(s, old);
        ratio = old / s;
    }
    return s;
}
template <int NS>
__device__ __forceinline__ float largest_of(const float (&x)[NS][8]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) m = __builtin_fmaxf(m, __builtin_fabsf(x[i][e]));   // (a NaN is passed over)
    if (__any(m == __builtin_inff())) {                       // only finite ones count
        m = 0.0f;
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = __builtin_fmaxf(m, finite_abs(x[i][e]));
    }
    return wave_max_all(m);
}
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float by) {
    return make_uint2(codes4(x[0] * by, x[1] * by, x[2] * by, x[3] * by), codes4(x[4] * by, x[5] * by, x[6] * by, x[7] * by));
}
// the keys of a block's first `fill` tokens, rounded to a larger scale
template <int D>
__device__ __forceinline__ void rescale_keys(unsigned char* kc, int fill, float ratio, int lane, int lanes) {
    uint2* w = reinterpret_cast<uint2*>(kc);
#pragma unroll 1                                              // (rare: not worth the registers)
    for (int i = lane; i < fill * (D / 8); i += lanes) {
        const uint2 old = w[i];
        w[i] = make_uint2(rescaled4(old.x, ratio), rescaled4(old.y, ratio));
    }
}

template <int DT, int D, int TOKENS>
__global__ __launch_bounds__(kWG) void append_few(AppendParams P) {
    constexpr int kPer = D / 8, kSlots = TOKENS * kPer / 64;  // slots of 8 elements: of a token, of a lane
    const int lane = threadIdx.x % 64, H = P.cache.kv_heads;
    const unsigned piece = blockIdx.x * (kWG / 64) + threadIdx.x / 64;
    if (piece >= P.npieces) return;
    const int h = static_cast<int>(piece % H), b = static_cast<int>(piece / H % P.B), layer = static_cast<int>(piece / H / P.B);
    const Appended a(P, b);
    const bool bad = a.bad || (a.count > 0 && __any(a.look(P, lane, 64)));
    if (h == 0 && layer == 0 && lane == 0) report(P, b, a, bad);
    if (bad || a.count <= 0) return;
    const size_t rows = (static_cast<size_t>(layer) * P.B + b) * P.R;
    for (long from = a.len; from < a.len + a.count;) {
        const long block = from / kBlock, to = (block + 1) * kBlock < a.len + a.count ? (block + 1) * kBlock : a.len + a.count;
        const int fill = static_cast<int>(from - block * kBlock);   // tokens of the sequence that the block holds already
        const int n = static_cast<int>(to - from);
        const size_t at = (static_cast<size_t>(layer) * P.cache.num_blocks + a.table[block]) * H + h;   // block and head
        unsigned char* kc = static_cast<unsigned char*>(P.cache.k_codes) + at * (kBlock * D);
        unsigned char* vc = static_cast<unsigned char*>(P.cache.v_codes) + at * (kBlock * D);
        const float old_k = P.cache.k_scale[at], old_v = P.cache.v_scale[at];
        size_t head[kSlots];
        int dim[kSlots], pos[kSlots], token[kSlots];
        Raw8 raw[kSlots];
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            const int u = lane + i * 64, t = u / kPer;
            token[i] = t < n ? t : -1;
            const long i0 = from - a.len + (t < n ? t : 0);   // (the first one where there is none)
            head[i] = (rows + a.row(i0)) * P.stride + static_cast<size_t>(h) * D;
            dim[i] = u % kPer * 8;
            pos[i] = static_cast<int>(a.len + i0);
        }
#pragma unroll
        for (int i = 0; i < kSlots; ++i)
            if (i * 64 / kPer < n) request8(DT, P.v, head[i] + dim[i], raw[i]);
        float x[kSlots][8];
        if (kSlots > 1 && n * kPer <= 64) {                   // one slot a lane holds them all
            const size_t one_head[1] = {head[0]};
            const int one_dim[1] = {dim[0]}, one_pos[1] = {pos[0]};
            float y[1][8];
            load_turned<1>(DT, P.k, one_head, one_dim, P.rot, one_pos, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[0][e] = y[0][e];
        } else {
            load_turned<kSlots, 1>(DT, P.k, head, dim, P.rot, pos, x);
        }
#pragma unroll
        for (int i = 0; i < kSlots; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = token[i] >= 0 ? x[i][e] : 0.0f;
        float ratio;
        const float ks = scale_in_force(largest_of<kSlots>(x), fill, old_k, ratio), kinv = 1.0f / ks;
        if (ratio != 1.0f) rescale_keys<D>(kc, fill, ratio, lane, 64);
#pragma unroll
        for (int i = 0; i < kSlots; ++i)
            if (token[i] >= 0) *reinterpret_cast<uint2*>(kc + (fill + token[i]) * D + dim[i]) = codes8(x[i], kinv);
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = 0.0f;
            if (token[i] >= 0) unpack8(DT, raw[i], y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = y[e];
        }
        const float vs = scale_in_force(largest_of<kSlots>(x), fill, old_v, ratio), vinv = 1.0f / vs;
        if (ratio != 1.0f) {
            const int words = (fill + 3) / 4;                 // of a row of d: 4 a group
#pragma unroll 1
            for (int i = lane; i < words * D; i += 64) {
                const int q = i / D, d = i % D;
                unsigned* w = reinterpret_cast<unsigned*>(vc + (q / 4 * D + d) * 16) + q % 4;
                const unsigned old = *w, keep = q * 4 + 4 <= fill ? 0u : ~0u << (8 * (fill - q * 4));
                *w = (rescaled4(old, ratio) & ~keep) | (old & keep);
            }
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");   // before the new bytes of the same words
        }
#pragma unroll
        for (int i = 0; i < kSlots; ++i)
            if (token[i] >= 0) {
                const int place = fill + token[i];
                unsigned char* p = vc + (place / 16 * D + dim[i]) * 16 + place % 16;
                const uint2 w = codes8(x[i], vinv);
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e * 16] = static_cast<unsigned char>((e < 4 ? w.x : w.y) >> (e % 4 * 8));
            }
        if (lane == 0) {
            P.cache.k_scale[at] = ks;
            P.cache.v_scale[at] = vs;
        }
        from = to;
    }
}

template <int DT, int D>
__global__ __launch_bounds__(kWG) void append_many(AppendParams P) {
    constexpr int kPer = D / 8, kSlots = kBlock * kPer / kWG; // slots of 8 elements: of a token, of a thread (keys)
    constexpr int kQuads = kBlock / 4 * kPer;                 // values: 8 dimensions of 4 places that lie side by side
    constexpr int kMine = (kQuads + kWG - 1) / kWG;
    __shared__ float most_of[2][kWG / 64];
    __shared__ int bad_any;
    const int tid = threadIdx.x, wave = tid >> 6, H = P.cache.kv_heads;
    const unsigned piece = blockIdx.x;
    const int h = static_cast<int>(piece % H);
    const int slot = static_cast<int>(piece / H % P.slots);
    const int b = static_cast<int>(piece / H / P.slots % P.B), layer = static_cast<int>(piece / H / P.slots / P.B);
    const Appended a(P, b);
    if (tid == 0) bad_any = 0;
    const long block = a.len / kBlock + slot;                 // of the sequence
    const long from = block * kBlock > a.len ? block * kBlock : a.len, to = (block + 1) * kBlock < a.len + a.count ? (block + 1) * kBlock : a.len + a.count;
    const bool first = h == 0 && slot == 0 && layer == 0;
    if (a.bad || from >= to) {                                // (slot 0 of a sequence with nothing to append; or a slot behind its last block)
        if (first && tid == 0) report(P, b, a, a.bad);
        return;
    }
    const int fill = static_cast<int>(from - block * kBlock); // tokens of the sequence that the block holds already
    const int n = static_cast<int>(to - from);
    const size_t rows = (static_cast<size_t>(layer) * P.B + b) * P.R;
    auto head_of = [&](int t) { return (rows + a.row(from - a.len + t)) * P.stride + static_cast<size_t>(h) * D; };

    Raw8 raw[kMine][4];                                       // values of 4 places; those that are not new are the nearest new ones
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int u = tid + i * kWG, place = u / kPer * 4;
        if (u >= kQuads || place + 4 <= fill || place >= fill + n) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) request8(DT, P.v, head_of(max(0, min(n - 1, place + e - fill))) + u % kPer * 8, raw[i][e]);
    }
    float x[kSlots][8];
    size_t head[kSlots];
    int dim[kSlots], pos[kSlots];
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
        const int u = tid + i * kWG, t = min(u / kPer, n - 1);
        head[i] = head_of(t);
        dim[i] = u % kPer * 8;
        pos[i] = static_cast<int>(from + t);
    }
    load_turned<kSlots, 2>(DT, P.k, head, dim, P.rot, pos, x);   // (a token that comes again does not change the largest)
    // (what the rows are is requested above, whatever is found here: it is in bounds)
    const bool found = a.look(P, tid, kWG);
    __syncthreads();
    if (found) bad_any = 1;
    __syncthreads();
    if (first && tid == 0) report(P, b, a, bad_any != 0);
    if (bad_any != 0) return;
    const size_t at = (static_cast<size_t>(layer) * P.cache.num_blocks + a.table[block]) * H + h;   // block and head
    unsigned char* kc = static_cast<unsigned char*>(P.cache.k_codes) + at * (kBlock * D);
    unsigned char* vc = static_cast<unsigned char*>(P.cache.v_codes) + at * (kBlock * D);
    const float old_k = P.cache.k_scale[at], old_v = P.cache.v_scale[at];
    const float high_k = largest_of<kSlots>(x);
    float high_v = 0.0f;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int u = tid + i * kWG, place = u / kPer * 4;
        if (u >= kQuads || place + 4 <= fill || place >= fill + n) continue;
        float y[4][8], m = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) unpack8(DT, raw[i][e], y[e]);
#pragma unroll
        for (int e = 0; e < 32; ++e) m = __builtin_fmaxf(m, __builtin_fabsf(y[e / 8][e % 8]));
        if (m == __builtin_inff()) {
            m = 0.0f;
#pragma unroll
            for (int e = 0; e < 32; ++e) m = __builtin_fmaxf(m, finite_abs(y[e / 8][e % 8]));
        }
        high_v = __builtin_fmaxf(high_v, m);
    }
    high_v = wave_max_all(high_v);
    if ((tid & 63) == 0) {
        most_of[0][wave] = high_k;
        most_of[1][wave] = high_v;
    }
    __syncthreads();
    auto most = [&](int i) { return __builtin_fmaxf(__builtin_fmaxf(most_of[i][0], most_of[i][1]), __builtin_fmaxf(most_of[i][2], most_of[i][3])); };
    float kratio, vratio;
    const float ks = scale_in_force(most(0), fill, old_k, kratio), kinv = 1.0f / ks;
    const float vs = scale_in_force(most(1), fill, old_v, vratio), vinv = 1.0f / vs;
    if (kratio != 1.0f) rescale_keys<D>(kc, fill, kratio, tid, kWG);
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
        const int t = (tid + i * kWG) / kPer;
        if (t < n) *reinterpret_cast<uint2*>(kc + (fill + t) * D + dim[i]) = codes8(x[i], kinv);
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int u = tid + i * kWG, place = u / kPer * 4, d = u % kPer * 8;
        if (u >= kQuads || place >= fill + n) continue;
        const bool any_new = place + 4 > fill;
        if (!any_new && vratio == 1.0f) continue;
        float y[4][8];
        unsigned is_new = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (place + e >= fill && place + e < fill + n) is_new |= 0xFFu << (8 * e);
            if (any_new) {
                unpack8(DT, raw[i][e], y[e]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) y[e][k] = 0.0f;
            }
        }
        unsigned held = 0;                                    // bytes of tokens that the block held before
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (place + e < fill) held |= 0xFFu << (8 * e);
        unsigned char* p = vc + (place / 16 * D + d) * 16 + place % 16;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            unsigned w = codes4(y[0][k] * vinv, y[1][k] * vinv, y[2][k] * vinv, y[3][k] * vinv);
            if (is_new != ~0u) {                              // a word that is not new throughout
                const unsigned old = *reinterpret_cast<const unsigned*>(p + k * 16);
                const unsigned kept = vratio != 1.0f ? (rescaled4(old, vratio) & held) | (old & ~held) : old;
                w = (w & is_new) | (kept & ~is_new);
            }
            *reinterpret_cast<unsigned*>(p + k * 16) = w;
        }
    }
    if (tid == 0) {
        P.cache.k_scale[at] = ks;
        P.cache.v_scale[at] = vs;
    }
}

}  // namespace

#endif  // FSD_CSRC_CACHE_APPEND_H_
