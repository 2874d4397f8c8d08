// Appending keys and values to the 8-bit paged cache (fsd_cache_append).
// Part of libfsd (gfx950); included by operators.hip, which holds the host side and the C ABI.
//
//   s = smallest 2^e, e >= -100, with |x| <= 448 s over the finite x appended to the block, but not under the block's own
//   old codes: round(code s_old / s);  new codes: round(x / s), e4m3, ties to even
//
// A block of a head is one piece of work: nothing is shared between two of them, so they need not agree on anything.  Its new keys
// are in registers when their largest magnitude is known, and are then written as codes; so are its new values.
// Measured: the accepted rows of 64 trees, 8 key heads of 128, 32 layers: 44 us for 148 MB of traffic (the codes of a dimension's 16 tokens
// lie together, so values are read and written 2 KB at a time; without that, 50 MB), in pieces of 128 bytes to 2 KB all over 1.6 GB: neither more
// wavefronts a compute unit (6 in place of 4: 49 us) nor a sequence's heads in one XCD (47) change that.  24576 prompt tokens: 56 us for 252 MB, 4.5 TB/s:
// of the 201 read 100 are keys and values, the rest the rotation's table, as a block's heads lie on all eight XCDs and each fetches its rows.
//   append_few   a step's accepted rows (at most 16): a wavefront for a head's keys and one for its values, which take the blocks they touch (one, seldom
//                two) in turn
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
// `slots` times 16 old codes, rounded to a larger scale.  (Few calls have such blocks, but one that has waits for them: four slots at once.)
__device__ __forceinline__ void rescale(unsigned char* codes, int slots, float ratio, int lane, int lanes) {
    constexpr int kOnce = 4;
    u32x4* w = reinterpret_cast<u32x4*>(codes);
#pragma unroll 1
    for (int i = lane; i < slots; i += kOnce * lanes) {
        u32x4 z[kOnce];
#pragma unroll
        for (int e = 0; e < kOnce; ++e) z[e] = w[min(i + e * lanes, slots - 1)];
#pragma unroll
        for (int e = 0; e < kOnce; ++e) {
#pragma unroll
            for (int k = 0; k < 4; ++k) z[e][k] = rescaled4(z[e][k], ratio);
            if (i + e * lanes < slots) w[i + e * lanes] = z[e];
        }
    }
}

constexpr int kFew = 16;         // rows of append_few: they touch two blocks, and two runs of 16 tokens of a block, at most

// The rows of a step that append_few takes, looked up once by a wavefront: lane i holds the i-th row's place in k and v, lanes 0 and 1 the blocks.
struct Few {
    long len, count;
    int row, block;
    bool bad;                    // for everyone
    __device__ __forceinline__ Few(const AppendParams& P, int b, int lane) {
        len = P.cache.cache_len[b];
        count = static_cast<long>(P.accept_len[b]) + 1;
        row = lane;
        if (P.path != nullptr && lane > 0 && lane <= min(P.max_depth, kFew)) row = P.path[static_cast<size_t>(b) * P.max_depth + lane - 1] + 1;
        bad = count < 0 || count > P.max_rows || len < 0 || len + count > static_cast<long>(P.cache.max_blocks) * kBlock ||
              (count > 0 && P.rot.table != nullptr && len + count > P.rot.rows);
        block = 0;
        if (bad || count == 0) return;
        bool found = false;
        if (lane < 2 && len / kBlock + lane <= (len + count - 1) / kBlock) {
            block = P.cache.block_table[static_cast<size_t>(b) * P.cache.max_blocks + len / kBlock + lane];
            found = block < 0 || block >= P.cache.num_blocks;
        }
        if (lane > 0 && lane < count) found |= row < 1 || row >= P.R;
        row = max(0, min(P.R - 1, row));                      // (requested before it has been looked at)
        bad = __any(found);
    }
};

// Keys: D / 8 lanes a token, 8 dimensions each; a token's codes are a run of D bytes.  SLOTS: such steps over the wavefront's lanes, which hold
// 512 / D tokens each.
template <int DT, int D, int SLOTS>
__device__ __forceinline__ void append_keys(const AppendParams& P, size_t at, int fill, int n, size_t rows, int h, int row, int i0, int pos0, int lane) {
    constexpr int kPer = D / 8, kAtOnce = 64 / kPer;
    unsigned char* kc = static_cast<unsigned char*>(P.cache.k_codes) + at * (kBlock * D);
    const float old = P.cache.k_scale[at];
    float x[SLOTS][8];
    const int dim[1] = {lane % kPer * 8};
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
        if (i > 0 && i * kAtOnce >= n) continue;
        const int t = i * kAtOnce + lane / kPer, there = min(t, n - 1);   // (the last one again: it does not change the largest)
        const size_t head[1] = {(rows + __shfl(row, i0 + there, 64)) * P.stride + static_cast<size_t>(h) * D};
        const int pos[1] = {pos0 + there};
        load_turned<1>(DT, P.k, head, dim, P.rot, pos, reinterpret_cast<float(&)[1][8]>(x[i]));
    }
    float ratio;
    const float s = scale_in_force(largest_of<SLOTS>(x), fill, old, ratio), inv = 1.0f / s;
    if (ratio != 1.0f) rescale(kc, fill * (D / 16), ratio, lane, 64);
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        const int t = i * kAtOnce + lane / kPer;
        if (t < n) *reinterpret_cast<uint2*>(kc + (fill + t) * D + dim[0]) = codes8(x[i], inv);
    }
    if (lane == 0) P.cache.k_scale[at] = s;
}

// Values: D / 64 dimensions a lane, all tokens of which it has: a dimension's codes of 16 tokens are 16 bytes, so whole ones are read, changed and written.
// (With a lane a token's 8 dimensions, as for keys, and stores of single bytes that step took 54 us.)  N: tokens, at most.
template <int DT, int D, int N>
__device__ __forceinline__ void append_values(const AppendParams& P, size_t at, int fill, int n, size_t rows, int h, int row, int i0, int lane) {
    constexpr int kE = D / 64, kBytes = kE * (DT == FSD_F32 ? 4 : 2);
    unsigned char* vc = static_cast<unsigned char*>(P.cache.v_codes) + at * (kBlock * D);
    const float old_s = P.cache.v_scale[at];
    struct alignas(kBytes) Raw { unsigned char of[kBytes]; };
    Raw raw[N];
#pragma unroll
    for (int t = 0; t < N; ++t) {
        raw[t] = Raw{};
        if (t >= n) continue;
        const size_t r = rows + __builtin_amdgcn_readlane(row, i0 + t);
        raw[t] = *reinterpret_cast<const Raw*>(P.v + (r * P.stride + static_cast<size_t>(h) * D + lane * kE) * (DT == FSD_F32 ? 4 : 2));
    }
    const int run = fill / 16, f = fill % 16;                 // the first of the two runs of 16 tokens, and the first new place in it
    const bool two = f + n > 16;
    u32x4* to = reinterpret_cast<u32x4*>(vc) + run * D + lane * kE;
    u32x4 old[2][kE];
#pragma unroll
    for (int e = 0; e < kE; ++e) {
        old[0][e] = to[e];
        old[1][e] = u32x4{0u, 0u, 0u, 0u};
        if (two) old[1][e] = to[D + e];
    }
    float y[N][kE], m = 0.0f;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            if constexpr (DT == FSD_F32) y[t][e] = __builtin_bit_cast(float, *reinterpret_cast<const unsigned*>(raw[t].of + 4 * e));
            else if constexpr (DT == FSD_BF16) y[t][e] = __uint_as_float(static_cast<unsigned>(*reinterpret_cast<const unsigned short*>(raw[t].of + 2 * e)) << 16);
            else y[t][e] = static_cast<float>(*reinterpret_cast<const _Float16*>(raw[t].of + 2 * e));
            m = __builtin_fmaxf(m, __builtin_fabsf(y[t][e]));  // (a NaN is passed over)
        }
    if (__any(m == __builtin_inff())) {                       // only finite ones count
        m = 0.0f;
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int e = 0; e < kE; ++e) m = __builtin_fmaxf(m, finite_abs(y[t][e]));
    }
    float ratio;
    const float s = scale_in_force(wave_max_all(m), fill, old_s, ratio), inv = 1.0f / s;
    if (ratio != 1.0f) {                                      // (rare)
        rescale(vc, run * D, ratio, lane, 64);
#pragma unroll
        for (int e = 0; e < kE; ++e)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int held = max(0, min(4, f - 4 * k));    // of this word's tokens
                const unsigned keep = held == 4 ? ~0u : (1u << (8 * held)) - 1u, now = old[0][e][k];
                old[0][e][k] = (rescaled4(now, ratio) & keep) | (now & ~keep);
            }
    }
    // The new codes of a dimension move to their place in the runs by bytes, then by words; `places`: which bytes of these words are new
    const unsigned places = ((1u << n) - 1u) << (f & 3);
    auto put = [&](auto word) {
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            unsigned before = 0u;
#pragma unroll
            for (int j = 0; j <= N / 4; ++j) {
                unsigned c = 0u;
                if (j < N / 4) c = codes4(y[4 * (j % (N / 4))][e] * inv, y[4 * (j % (N / 4)) + 1][e] * inv, y[4 * (j % (N / 4)) + 2][e] * inv, y[4 * (j % (N / 4)) + 3][e] * inv);
                const unsigned w = static_cast<unsigned>((static_cast<unsigned long long>(c) << 32 | before) >> (32 - 8 * (f & 3)));
                const unsigned bits = places >> (4 * j) & 15u, is_new = (bits * 0x00204081u & 0x01010101u) * 0xFFu;
                constexpr int at0 = decltype(word)::value;
                const int k = at0 + j;
                old[k / 4][e][k % 4] = (w & is_new) | (old[k / 4][e][k % 4] & ~is_new);
                before = c;
            }
        }
    };
    switch (f / 4) {
        case 0: put(std::integral_constant<int, 0>()); break;
        case 1: put(std::integral_constant<int, 1>()); break;
        case 2: put(std::integral_constant<int, 2>()); break;
        default: put(std::integral_constant<int, 3>()); break;
    }
#pragma unroll
    for (int e = 0; e < kE; ++e) {
        to[e] = old[0][e];
        if (two) to[D + e] = old[1][e];
    }
    if (lane == 0) P.cache.v_scale[at] = s;
}

// Grid: two wavefronts for each key head, sequences, layers.
template <int DT, int D>
__global__ __launch_bounds__(kWG) void append_few(AppendParams P) {
    const int lane = threadIdx.x % 64, H = P.cache.kv_heads;
    const int at_wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (kWG / 64) + threadIdx.x / 64), h = at_wave / 2;
    if (h >= H) return;
    const bool values = at_wave & 1;
    const int b = static_cast<int>(blockIdx.y), layer = static_cast<int>(blockIdx.z);
    const Few a(P, b, lane);
    if (h == 0 && layer == 0 && lane == 0 && !values) {
        if (P.len_out) P.len_out[b] = static_cast<int32_t>(a.bad ? a.len : a.len + a.count);
        if (P.status) P.status[b] = a.bad ? FSD_ROW_BAD_CACHE : 0;
    }
    if (a.bad || a.count <= 0) return;
    const size_t rows = (static_cast<size_t>(layer) * P.B + b) * P.R;
    int done = 0;
    for (int which = 0; done < a.count; ++which) {            // the blocks: one, seldom two
        const int fill = which == 0 ? static_cast<int>(a.len % kBlock) : 0;   // tokens of the sequence that the block holds already
        const int n = min(static_cast<int>(a.count) - done, kBlock - fill);
        const size_t at = (static_cast<size_t>(layer) * P.cache.num_blocks + __builtin_amdgcn_readlane(a.block, which)) * H + h;   // block and head
        const int pos0 = static_cast<int>(a.len) + done;
        // (few tokens: most of the instructions are left out)
        if (values) {
            if (n <= 4) append_values<DT, D, 4>(P, at, fill, n, rows, h, a.row, done, lane);
            else append_values<DT, D, kFew>(P, at, fill, n, rows, h, a.row, done, lane);
        } else {
            if (n <= 512 / D) append_keys<DT, D, 1>(P, at, fill, n, rows, h, a.row, done, pos0, lane);
            else append_keys<DT, D, kFew * D / 512>(P, at, fill, n, rows, h, a.row, done, pos0, lane);
        }
        done += n;
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
    if (kratio != 1.0f) rescale(kc, fill * (D / 16), kratio, tid, kWG);
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
