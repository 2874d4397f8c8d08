// Device helpers of the operators around a verify call (condition.h, cache_append.h, cache_attend.h).
// Part of libfsd (gfx950).
#ifndef FSD_CSRC_OPERATORS_COMMON_H_
#define FSD_CSRC_OPERATORS_COMMON_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fsd.h"

namespace {

constexpr int kWG = 256;          // threads per workgroup (4 wavefronts of 64)
constexpr int kBlock = FSD_CACHE_BLOCK;
constexpr int kXcds = 8;

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));

// Workgroups are dealt to the 8 XCDs, each with an L2 of its own, in turn.  This gives an XCD a run of consecutive pieces
// of work instead, so that those that read the same thing (a sequence's history, a head's cache blocks) meet in one L2.
// -1: nothing left for this workgroup (the grid has 8 * ceil(n / 8) of them).
__device__ __forceinline__ long spread_over_xcds(long block, long n) {
    const long per = (n + kXcds - 1) / kXcds, at = block % kXcds * per + block / kXcds;
    return block / kXcds < per && at < n ? at : -1;
}
inline long grid_over_xcds(long n) { return (n + kXcds - 1) / kXcds * kXcds; }

// ---- logits, in 16-byte slots at any address of whole elements

// (STREAM: past the caches, for what is not read again soon)
template <bool STREAM = false>
__device__ __forceinline__ uint4 load_any16(const char* p) {
    const u32x4_any* at = reinterpret_cast<const u32x4_any*>(p);
    u32x4_any v;
    if constexpr (STREAM) v = __builtin_nontemporal_load(at);
    else v = *at;
    return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool STREAM = false>
__device__ __forceinline__ void store_any16(char* p, const uint4& w) {
    u32x4_any v;
    v.x = w.x; v.y = w.y; v.z = w.z; v.w = w.w;
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(p));
    else *reinterpret_cast<u32x4_any*>(p) = v;
}
template <bool BF16>
__device__ __forceinline__ uint4 neg_inf_slot() {
    const unsigned w = BF16 ? 0xFF80FF80u : 0xFF800000u;
    return make_uint4(w, w, w, w);
}
__device__ __forceinline__ unsigned bf16_bits(float z) {
    return static_cast<unsigned>(__builtin_bit_cast(unsigned short, static_cast<__bf16>(z)));   // to nearest, ties to even
}
// the slot with -inf in the entries that `ok` lacks
template <bool BF16>
__device__ __forceinline__ uint4 masked_slot(const uint4& r, unsigned ok) {
    unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        auto all = [&](int bit) { return static_cast<unsigned>(static_cast<int>(ok << (31 - bit)) >> 31); };   // the bit, 32 times
        const unsigned keep = BF16 ? (all(2 * i) & 0xFFFFu) | (all(2 * i + 1) & 0xFFFF0000u) : all(i);
        w[i] = (w[i] & keep) | ((BF16 ? 0xFF80FF80u : 0xFF800000u) & ~keep);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool BF16>
__device__ __forceinline__ float load_logit(const char* row, int e) {
    if constexpr (BF16) return __uint_as_float(static_cast<unsigned>(reinterpret_cast<const unsigned short*>(row)[e]) << 16);
    else return reinterpret_cast<const float*>(row)[e];
}
template <bool BF16>
__device__ __forceinline__ void store_logit(char* row, int e, float z) {
    if constexpr (BF16) reinterpret_cast<unsigned short*>(row)[e] = static_cast<unsigned short>(bf16_bits(z));
    else reinterpret_cast<float*>(row)[e] = z;
}
template <bool BF16>
__device__ __forceinline__ void copy_logit(char* out, const char* in, int e) {
    if constexpr (BF16) reinterpret_cast<unsigned short*>(out)[e] = reinterpret_cast<const unsigned short*>(in)[e];
    else reinterpret_cast<unsigned*>(out)[e] = reinterpret_cast<const unsigned*>(in)[e];
}

// ---- keys, values and queries: 8 elements in a row

// what lies in 16 bytes (8 elements of 16 bits) as numbers
__device__ __forceinline__ void unpack8(int dtype, const u32x4& a, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned w = a[i];                              // (a bit cast of the vector's element itself takes element 0)
        const half2_t h = __builtin_bit_cast(half2_t, w);
        x[2 * i] = dtype == FSD_BF16 ? __uint_as_float(w << 16) : static_cast<float>(h.x);
        x[2 * i + 1] = dtype == FSD_BF16 ? __uint_as_float(w & 0xFFFF0000u) : static_cast<float>(h.y);
    }
}
// 8 elements as they lie in memory: 16 bits each in lo, or 32 bits in lo and hi
struct Raw8 { u32x4 lo, hi; };
__device__ __forceinline__ void request8(int dtype, const void* base, size_t at, Raw8& r) {
    if (dtype == FSD_F32) {
        const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const float*>(base) + at);
        r.lo = p[0];
        r.hi = p[1];
    } else {
        r.lo = *reinterpret_cast<const u32x4*>(static_cast<const unsigned short*>(base) + at);
    }
}
__device__ __forceinline__ void unpack8(int dtype, const Raw8& r, float* x) {
    if (dtype == FSD_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(r.lo[i]);
            x[4 + i] = __uint_as_float(r.hi[i]);
        }
    } else {
        unpack8(dtype, r.lo, x);
    }
}

// NS slots of 8 elements, d[i] .. d[i]+7 (d a multiple of 8) of the head that begins at element at[i], turned by the table's row
// pos[i].  All loads of up to ONCE slots are requested before the first is used: one memory latency, not one for each.
template <int NS, int ONCE = 4>
__device__ __forceinline__ void load_turned(int dtype, const void* base, const size_t (&at)[NS], const int (&d)[NS], const fsd_rotation& rot,
                                            const int (&pos)[NS], float (&x)[NS][8]) {
    const int n = rot.dim / 2;
    constexpr int kOnce = NS < ONCE ? NS : ONCE;
#pragma unroll
    for (int i0 = 0; i0 < NS; i0 += kOnce) {
        Raw8 own[kOnce];
#pragma unroll
        for (int e = 0; e < kOnce; ++e) request8(dtype, base, at[i0 + e] + d[i0 + e], own[e]);
        if (rot.table == nullptr) {
#pragma unroll
            for (int e = 0; e < kOnce; ++e) unpack8(dtype, own[e], x[i0 + e]);
        } else if (rot.style == FSD_ROPE_HALVES) {
            Raw8 other[kOnce];
            u32x4 c[kOnce][2], s[kOnce][2];
#pragma unroll
            for (int e = 0; e < kOnce; ++e) {
                const int i = i0 + e;
                const bool low = d[i] < n, in = d[i] < rot.dim;
                request8(dtype, base, at[i] + (low ? d[i] + n : in ? d[i] - n : d[i]), other[e]);
                const float* t = rot.table + static_cast<size_t>(pos[i]) * rot.dim + (low ? d[i] : in ? d[i] - n : 0);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    c[e][k] = *reinterpret_cast<const u32x4*>(t + 4 * k);
                    s[e][k] = *reinterpret_cast<const u32x4*>(t + n + 4 * k);
                }
            }
#pragma unroll
            for (int e = 0; e < kOnce; ++e) {
                const int i = i0 + e;
                const bool low = d[i] < n, in = d[i] < rot.dim;
                float y[8];
                unpack8(dtype, own[e], x[i]);
                unpack8(dtype, other[e], y);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const unsigned cb = c[e][k / 4][k % 4], sb = s[e][k / 4][k % 4];
                    const float a = x[i][k] * __uint_as_float(cb), b = y[k] * __uint_as_float(sb);
                    x[i][k] = in ? (low ? a - b : a + b) : x[i][k];
                }
            }
        } else {
            u32x4 c[kOnce], s[kOnce];
#pragma unroll
            for (int e = 0; e < kOnce; ++e) {
                const int i = i0 + e;
                const float* t = rot.table + static_cast<size_t>(pos[i]) * rot.dim + (d[i] < rot.dim ? d[i] / 2 : 0);
                c[e] = *reinterpret_cast<const u32x4*>(t);
                s[e] = *reinterpret_cast<const u32x4*>(t + n);
            }
#pragma unroll
            for (int e = 0; e < kOnce; ++e) {
                const int i = i0 + e;
                const bool in = d[i] < rot.dim;
                unpack8(dtype, own[e], x[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned cb = c[e][k], sb = s[e][k];
                    const float cc = __uint_as_float(cb), ss = __uint_as_float(sb), a = x[i][2 * k], b = x[i][2 * k + 1];
                    x[i][2 * k] = in ? a * cc - b * ss : a;
                    x[i][2 * k + 1] = in ? b * cc + a * ss : b;
                }
            }
        }
    }
}

// |x|, or 0 where x is not finite
__device__ __forceinline__ float finite_abs(float x) {
    const float a = __builtin_fabsf(x);
    return a < __builtin_inff() ? a : 0.0f;
}
__device__ __forceinline__ float wave_max_all(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = __builtin_fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
// 2^e as a number, -126 <= e <= 127
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<unsigned>(e + 127) << 23); }

}  // namespace

#endif  // FSD_CSRC_OPERATORS_COMMON_H_
