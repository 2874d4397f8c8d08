// The best continuations of a sequence's beams (fsd_beam_select) and the states that follow them (fsd_beam_reorder).
// Part of libfsd (gfx950).
//
// beam_slices goes over the logits once: a workgroup takes a slice of one beam's row, adds up its exponentials and writes its n best entries, best
// first.  beam_merge, a workgroup a sequence, makes the normalisers of the beams from the slices' sums and takes the n best of all slices' lists.
//
// Whole numbers come out of it, so the order matters to the last bit: two beams' entries may lie as near to one another as their normalisers' errors.
// Exponentials, sums and ranks are binary64 therefore.  A binary64 fma issues like a binary32 one here (2.0 ns a wavefront and SIMD, as an addition or
// a conversion), the hardware's binary32 exponential takes 3.8: 16 instructions an entry where binary32 would take 9, and an error of 2^-34 in place of 2^-25.
//
// What bounds it (64 x 8 rows of 128256 bfloat16 entries, a tenth of the beams finished, 118 MB: 36 us; reading them alone 18): vector instructions, 11.9
// an entry, take 21 us of it, the table's reads 14 of the LDS's time beside them; the rest is what a wavefront waits for within a slot (four of them on a SIMD) and each
// row's end (bound, list, ranks, about 4 us), which only the other workgroup of the compute unit overlaps, and that is in step with it (512 rows are one a workgroup).
// (Without the sums it took 13 us less, without slots put aside 6, without the making of the table 2; the next slice's first requests before this one's end change
// nothing.)  16 x 12 rows of 128259 binary32 entries, n = 60, 98 MB: 30 us; the list
// of 60 takes as many instructions as the exponentials, and all workgroups begin and end together (exponentials by a table of 512 powers and degree 2, 3 instructions
// an entry less, change nothing).  Merging: 5 us for one sequence of 4 beams, 6 for 64 of 8, 9 at n = 60: a chain of round trips and barriers.  128 x 8 bfloat16 rows of
// 32000, without the table: 29.5 us, reading 11.
#ifndef FSD_CSRC_BEAM_SELECT_H_
#define FSD_CSRC_BEAM_SELECT_H_

#include <type_traits>

#include "operators_common.h"

namespace {

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

constexpr int kBeamMost = 128;      // n
constexpr int kBeamWidest = 256;    // beams
constexpr int kWaveList = 256;      // entries of a wavefront's part of a slice that stand in LDS before the n best are taken from all
constexpr unsigned short kTableBase = 0x397F;   // bits of the last bfloat16 number under 2^-12
constexpr unsigned short kTableEnd = 2 * (0x4280 - kTableBase);   // entries: 0; 2^-12, -2^-12 and so on to the last numbers under 64; two and the last one for 64 and over
constexpr unsigned short kTurnedInf = 0xFF01;   // -inf with its sign behind the rest
constexpr int kAside = 112;         // slots of a wavefront's that stand there until they are taken apart
constexpr double kLog2e64 = 1.4426950408889634074;
constexpr double kExpOf0 = 0.9999999999616819;      // what exp_within gives for 0

struct BeamParams {
    const char* logits;
    size_t row_stride;              // bytes
    const float *scores, *weights;
    const int* done;
    int B, W, V, n;
    int len, S, lists;              // entries of a slice (a multiple of a 16-byte slot's), slices of a row, W * S
    unsigned units;                 // B * W * S
    unsigned by_S;                  // ceil(2^32 / S), 0 where S is 1
    float2* cand;                   // [B, n, W * S]: logit and token of a list's entry, best first; -inf behind the last
    double2* stat;                  // [B, W * S]: a number r and the sum of e^(z - r); -inf and 0 where no entry counts
    float* scores_out;
    int *parent, *tokens, *status;
};

// e^x, off by 2^-34 of it, for |x| up to 700: x log2 e as a whole number k and a rest of at most 1/2; the rest's power by a polynomial of degree 7
// (fitted to the smallest largest relative error on [-1/2, 1/2], 4.03e-11), k added to its exponent.  NaN stays NaN.
__device__ __forceinline__ double exp_within(double x) {
    constexpr double kWhole = 6755399441055744.0;            // 1.5 * 2^52: what is added to it comes out whole, in the low word
    const double k = __builtin_fma(x, kLog2e64, kWhole), f = __builtin_fma(x, kLog2e64, kWhole - k);
    double p = 1.520192135287937e-05;
    p = __builtin_fma(p, f, 0.00015469291148729867);
    p = __builtin_fma(p, f, 0.001333392256490547);
    p = __builtin_fma(p, f, 0.009618027253635145);
    p = __builtin_fma(p, f, 0.05550410353445615);
    p = __builtin_fma(p, f, 0.24022651198157982);
    p = __builtin_fma(p, f, 0.693147180728448);
    p = __builtin_fma(p, f, kExpOf0);
    return __builtin_amdgcn_ldexp(p, static_cast<int>(__builtin_bit_cast(unsigned long, k)));
}
// for any x <= 0: nothing under -700
__device__ __forceinline__ double exp_below(double x) {
    const double e = exp_within(x < -700.0 ? -700.0 : x);
    return x < -700.0 ? 0.0 : e;
}
// what all lanes have alike, as a scalar
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ unsigned uniform(unsigned x) { return static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(x))); }

// Over 16 lanes by rotations within them (no round trip through LDS), over the wavefront's four rows of 16 by scalars.  The sums' order is fixed.
template <int N>
__device__ __forceinline__ int rotated(int x) { return __builtin_amdgcn_update_dpp(x, x, 0x120 | N, 0xF, 0xF, false); }
template <int N>
__device__ __forceinline__ double rotated(double x) {
    const unsigned long u = __builtin_bit_cast(unsigned long, x);
    const unsigned lo = static_cast<unsigned>(rotated<N>(static_cast<int>(u))), hi = static_cast<unsigned>(rotated<N>(static_cast<int>(u >> 32)));
    return __builtin_bit_cast(double, static_cast<unsigned long>(hi) << 32 | lo);
}
__device__ __forceinline__ double row_sum(double x) {          // of 16 lanes
    x += rotated<8>(x);
    x += rotated<4>(x);
    x += rotated<2>(x);
    x += rotated<1>(x);
    return x;
}
__device__ __forceinline__ double row_max(double x) {
    double y;
    y = rotated<8>(x), x = y > x ? y : x;
    y = rotated<4>(x), x = y > x ? y : x;
    y = rotated<2>(x), x = y > x ? y : x;
    y = rotated<1>(x), x = y > x ? y : x;
    return x;
}
__device__ __forceinline__ unsigned long lane_word(unsigned long u, int lane) {
    return static_cast<unsigned long>(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(u >> 32), lane))) << 32 |
           static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(u), lane));
}
__device__ __forceinline__ double lane_value(double x, int lane) { return __builtin_bit_cast(double, lane_word(__builtin_bit_cast(unsigned long, x), lane)); }
__device__ __forceinline__ double wave_sum_64(double x) {
    x = row_sum(x);
    return (lane_value(x, 0) + lane_value(x, 16)) + (lane_value(x, 32) + lane_value(x, 48));
}
__device__ __forceinline__ float wave_largest(float x) {
    auto larger = [](float a, int b) { return __builtin_fmaxf(a, __int_as_float(b)); };
    x = larger(x, rotated<8>(__float_as_int(x)));
    x = larger(x, rotated<4>(__float_as_int(x)));
    x = larger(x, rotated<2>(__float_as_int(x)));
    x = larger(x, rotated<1>(__float_as_int(x)));
    const int u = __float_as_int(x);
    const float a = __int_as_float(__builtin_amdgcn_readlane(u, 0)), b = __int_as_float(__builtin_amdgcn_readlane(u, 16)),
                c = __int_as_float(__builtin_amdgcn_readlane(u, 32)), d = __int_as_float(__builtin_amdgcn_readlane(u, 48));
    return __builtin_fmaxf(__builtin_fmaxf(a, b), __builtin_fmaxf(c, d));
}

// bits of a number in an order in which larger numbers have larger words (0 and -0 differ: give it neither as -0)
__device__ __forceinline__ unsigned ordered(float x) {
    const unsigned u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(unsigned o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
constexpr unsigned kLeastOrdered = 0x00800000u;   // of the lowest finite number

// the largest of three, without the instructions that make quiet NaNs of others first
__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}
// x, but no less than -700 (by its word: those of negative numbers grow with the distance from 0; a NaN of this sign is lost, which is looked for elsewhere)
__device__ __forceinline__ float at_least_700_below(float x) {
    const unsigned u = __float_as_uint(x), least = 0xC42F0000u;
    return __uint_as_float(u < least ? u : least);
}

// entry e of a 16-byte slot
template <bool BF16>
__device__ __forceinline__ float slot_entry(const u32x4& r, int e) {
    if constexpr (BF16) return __uint_as_float(e & 1 ? r[e / 2] & 0xFFFF0000u : r[e / 2] << 16);
    else return __uint_as_float(r[e]);
}

__device__ __forceinline__ float score_of(const BeamParams& P, long at) { return P.scores ? P.scores[at] : 0.0f; }
__device__ __forceinline__ bool beam_runs(const BeamParams& P, long at) {   // whether a beam's row is read
    const float score = score_of(P, at);
    const int done = P.done ? P.done[at] : 0;                // (both requested together)
    return (score > -__builtin_inff()) & (done == 0);        // (a score that is NaN is reported without its row)
}

// A slice's n best entries where more than kWaveList of a wavefront's reach the bound that its lanes gave (rows of equal entries, or in order): the n-th largest
// is found bit by bit, then what is above it and, from the lowest index on, what equals it go into the list.  Returns how many.  (It reads the entries
// again rather than keep the calling kernel's registers in memory: 16 passes, 32 for binary32, and two more, entry by entry, over what the caches hold.  64 x 8 rows
// of 128256 bfloat16 entries of which a mask of a finite number leaves 5: the kernel takes 1840 us, unmasked 35, masked by -inf 31; 16 x 12 binary32 rows of 128259, n = 60: 1530, 32, 24.)
template <bool BF16, int NW>
__device__ __noinline__ int slice_cut(const char* z, int begin, int end, int n, unsigned long* list, int* lds, int tid) {
    const int wave = tid / 64, lane = tid % 64, len = end - begin;
    auto over_wg = [&](int c) {                              // the sum of all threads' c
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
        __syncthreads();
        if (lane == 0) lds[wave] = c;
        __syncthreads();
        int all = 0;
        for (int w = 0; w < NW; ++w) all += lds[w];
        return all;
    };
    auto word_at = [&](int k) { return ordered(load_logit<BF16>(z, begin + k) + 0.0f); };
    unsigned least = 0;
    for (int bit = 31; bit >= (BF16 ? 16 : 0); --bit) {
        const unsigned c = least | 1u << bit;
        int have = 0;
        for (int k = tid; k < len; k += 64 * NW) have += word_at(k) >= c;
        if (over_wg(have) >= n) least = c;
    }
    // (an ordered word's low 16 bits are those of a bfloat16 entry's zeros: all 0 of a positive one, all 1 of a negative one)
    if (BF16 && !(least & 0x80000000u)) least |= 0xFFFFu;
    if (least < kLeastOrdered) least = kLeastOrdered;
    int above = 0;
    for (int k = tid; k < len; k += 64 * NW) above += word_at(k) > least;
    const int more = over_wg(above);
    if (tid == 0) lds[NW] = 0;
    int before = 0;                                          // entries that equal it, of those behind us
    __syncthreads();
    for (int k0 = 0; k0 < len; k0 += 64 * NW) {
        const int k = k0 + tid;
        const unsigned o = k < len ? word_at(k) : 0u;
        const unsigned long same = __ballot(o == least);
        __syncthreads();
        if (lane == 0) lds[wave] = __popcll(same);
        __syncthreads();
        int at = before + __popcll(same & ((1ul << lane) - 1));
        for (int w = 0; w < wave; ++w) at += lds[w];
        for (int w = 0; w < NW; ++w) before += lds[w];
        if (o > least || (o == least && at < n - more)) list[atomicAdd(&lds[NW], 1)] = static_cast<unsigned long>(o) << 32 | ~static_cast<unsigned>(k);
    }
    __syncthreads();
    return lds[NW];
}

// Of a wavefront's list (in LDS) those that reach the bound, in their order; how many.
__device__ __forceinline__ int keep_reaching(unsigned long* list, int count, unsigned bound, int lane) {
    int kept = 0;
    for (int k0 = 0; k0 < count; k0 += 64) {
        __builtin_amdgcn_wave_barrier();                     // (lanes read what others have written; no instruction, an order for the compiler)
        const unsigned long x = k0 + lane < count ? list[k0 + lane] : 0;
        const bool keep = static_cast<unsigned>(x >> 32) >= bound;
        const unsigned long who = __ballot(keep);
        if (keep) list[kept + __popcll(who & ((1ul << lane) - 1))] = x;   // (at or before where it was read; a wavefront's LDS instructions are done in order)
        kept += __popcll(who);
    }
    return kept;
}

// The slots that a wavefront put aside, 64 entries at a time: those that reach the bound go into its list of `count`.  How many it has then; 2^16 more where they
// are too many for it.
template <bool BF16>
__device__ __forceinline__ int slots_apart(const u32x4* slots, const int* places, int aside, unsigned long* list, int count, unsigned least, int lane) {
    constexpr int E = BF16 ? 8 : 4;
    const float from = from_ordered(least);
    bool full = false;
    __builtin_amdgcn_wave_barrier();
    for (int s0 = 0; s0 < aside; s0 += 64 / E) {
        const int k = s0 + lane / E;
        bool is = false;
        float x = 0.0f;
        int at = 0;
        if (k < aside) {
            const unsigned* words = reinterpret_cast<const unsigned*>(slots + k);
            const int e = lane % E;
            if constexpr (BF16) x = __uint_as_float(e & 1 ? words[e / 2] & 0xFFFF0000u : words[e / 2] << 16);
            else x = __uint_as_float(words[e]);
            at = places[k] * E + e;
            is = x >= from;
        }
        const unsigned long who = __ballot(is);
        const int n_who = __popcll(who);
        // make room: what is under the bound by now goes
        if (count + n_who > kWaveList) count = keep_reaching(list, count, least, lane);
        const int to = count + __popcll(who & ((1ul << lane) - 1));
        if (is && to < kWaveList) list[to] = static_cast<unsigned long>(ordered(x + 0.0f)) << 32 | ~static_cast<unsigned>(at);
        count += n_who;
        if (count > kWaveList) full = true, count = kWaveList;
    }
    return count + (full ? 0x10000 : 0);
}

// 2 a + b of either half of a word, in one instruction
__device__ __forceinline__ u16x2 twice_and(u16x2 a, u16x2 b) {
    u16x2 x;
    asm("v_pk_mad_u16 %0, %1, 2, %2 op_sel_hi:[1,0,1]" : "=v"(x) : "v"(a), "v"(b));
    return x;
}
// eight times the lower (0) or upper (1) half of a word, in one instruction
template <int HALF>
__device__ __forceinline__ unsigned eight_times(unsigned both) {
    unsigned x;
    if constexpr (HALF == 0) asm("v_mad_u32_u16 %0, %1, 8, 0" : "=v"(x) : "v"(both));
    else asm("v_mad_u32_u16 %0, %1, 8, 0 op_sel:[1,0,0,0]" : "=v"(x) : "v"(both));
    return x;
}

// Of the entries of a slot that are nearer to 0 than the table goes, and count as 0: what that leaves out (what the table has for 0 goes, so that one error remains)
__device__ __forceinline__ double rest_of_small(u32x4 slot) {
    double rest = 0.0;
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
        const unsigned w = j == 0 ? slot[0] : j == 1 ? slot[1] : j == 2 ? slot[2] : slot[3];
        if ((w & 0x7FFFu) - 1u < kTableBase) rest += exp_within(static_cast<double>(__uint_as_float(w << 16))) - kExpOf0;
        if ((w >> 16 & 0x7FFFu) - 1u < kTableBase) rest += exp_within(static_cast<double>(__uint_as_float(w & 0xFFFF0000u))) - kExpOf0;
    }
    return rest;
}

// The wavefront's q-th largest of its lanes' words, to the upper 20 bits
template <bool BF16>
__device__ __forceinline__ unsigned wave_bound(unsigned word, int q) {
    unsigned bound = 0;
    for (int bit = 31; bit >= (BF16 ? 16 : 12); --bit) {
        const unsigned c = bound | 1u << bit;
        if (__popcll(__ballot(word >= c)) >= q) bound = c;
    }
    return bound;
}

// Slices of rows, one after the other in a workgroup, in chunks of NS slots of 16 bytes a thread; where a slot has been added up, that of the next chunk is requested in its
// place.  Of the entries seen so far a wavefront's q-th largest lane maximum, q = n / wavefronts rounded up, is reached by q of its own at least, so
// the least of the wavefronts' by n of the slice: what reaches that bound (few more than n entries where the values lie as those of logits do) is put
// into LDS and ranked there at the end.  Wavefronts tell one another their bounds without waiting: an older one of another's bounds as well.
// Exponentials are added up as e^z: binary64 has the range where logits are of the size that models give them.  Where they are not, the slice is gone over again.
// TABLE: exponentials of bfloat16 numbers are read from a table of all of them from 2^-12 to 64 of either sign (and 0, and those under -64, which
// count as nothing), which a workgroup makes once and keeps for all of its slices: 7 instructions an entry where the polynomial takes 16 (51 -> 38 us for the rows above at that step).
template <bool BF16, int NS, bool TABLE>
__global__ void __launch_bounds__(TABLE ? 512 : kWG, 4) beam_slices(const BeamParams P) {
    constexpr int NW = TABLE ? 8 : 4, T = NW * 64;
    static_assert(BF16 || !TABLE, "a table of bfloat16 numbers");
    constexpr int E = BF16 ? 8 : 4, kChunk = T * NS;        // (slots of a chunk)
    constexpr unsigned kNone = BF16 ? 0xFF80FF80u : 0xFF800000u;   // -inf
    __shared__ unsigned long list[NW * kWaveList];
    __shared__ u32x4 aside_slot[NW][kAside];
    __shared__ int aside_at[NW][kAside];
    __shared__ double table[TABLE ? kTableEnd + 1 : 1];
    __shared__ double wave_sum[NW], wave_ref[NW];
    __shared__ unsigned bounds[NW];
    __shared__ int lds[NW + 1];
    const int tid = threadIdx.x, wave = uniform(tid / 64), lane = tid % 64;
    bool begun = false;                                       // the table is there
    for (unsigned unit = blockIdx.x; unit < P.units; unit += gridDim.x) {
        const unsigned row = unit / static_cast<unsigned>(P.S);
        const int slice = static_cast<int>(unit - row * static_cast<unsigned>(P.S));
        if (!beam_runs(P, row)) continue;
        const int begin = slice * P.len, end = begin + P.len < P.V ? begin + P.len : P.V;
        const char* const z = P.logits + static_cast<size_t>(row) * P.row_stride;
        const char* const at_begin = z + static_cast<size_t>(begin) * (16 / E);
        const int slots = (end - begin) / E, all_slots = (end - begin + E - 1) / E;   // whole ones; and with a last one that is not
        // (Threads without a slot request the last one again, and where there is none some of the workspace: requests without branches go out together, and what
        // waits for one of them need not wait for the others.)
        const char* const at_slots = slots > 0 ? at_begin : reinterpret_cast<const char*>(P.stat);
        const int last_slot = slots > 0 ? slots - 1 : 0;
        auto request = [&](int slot) {
            const int from = slot < last_slot ? slot : last_slot;
            return static_cast<u32x4>(*reinterpret_cast<const u32x4_any*>(at_slots + static_cast<unsigned>(from) * 16u));
        };
        u32x4 r[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) r[i] = request(i * T + tid);
        if (TABLE && !begun) {                                    // (while the first requests are on their way; the barrier before its first use comes below)
            begun = true;
            for (int k = tid; k <= kTableEnd; k += T) {
                const double x = k == 0 ? 0.0 : static_cast<double>(__uint_as_float(static_cast<unsigned>(kTableBase + (k + 1) / 2) << 16));
                table[k] = k >= kTableEnd - 1 ? 0.0 : exp_within(k & 1 ? x : -x);
            }
        }
        // the entries behind the last whole slot: its thread takes them one by one
        u32x4 last = {kNone, kNone, kNone, kNone};
        if (slots < all_slots) {
            const int whole = begin + slots * E;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (whole + e < end) {
                    if constexpr (BF16) {
                        const unsigned h = reinterpret_cast<const unsigned short*>(z)[whole + e];
                        last[e / 2] = e & 1 ? (last[e / 2] & 0xFFFFu) | h << 16 : (last[e / 2] & 0xFFFF0000u) | h;
                    } else {
                        last[e] = reinterpret_cast<const unsigned*>(z)[whole + e];
                    }
                }
        }
        auto behind = [&](u32x4& slot, int k) {                   // slots that the slice does not have, or not whole
#pragma unroll
            for (int j = 0; j < 4; ++j) slot[j] = k < slots ? slot[j] : k == slots ? last[j] : kNone;
        };

        unsigned long* const mine_list = list + wave * kWaveList;
        int count = 0;                                            // of the wavefront's list
        bool full = false;                                        // whether more were to go into it than it holds
        int aside = 0;
        // its share of n: by how many of its lanes have a slot, where not all do (a share that some lanes could not reach would let everything through: a row's last
        // slice, of 1776 bfloat16 entries, n = 128: 30 -> 13 us)
        int q = (P.n + NW - 1) / NW;
        if (all_slots < T) {
            const int lanes = all_slots - wave * 64, some = lanes < 0 ? 0 : lanes < 64 ? lanes : 64;
            q = (P.n * some + all_slots - 1) / all_slots;
        }
        unsigned least = kLeastOrdered;
        auto take_apart = [&]() {
            const int to = slots_apart<BF16>(aside_slot[wave], aside_at[wave], aside, mine_list, count, least, lane);
            count = to & 0xFFFF;
            full |= to > 0xFFFF;
            aside = 0;
        };
        auto all_bounds = [&]() {
            unsigned bound = 0xFFFFFFFFu;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const unsigned theirs = uniform(__hip_atomic_load(&bounds[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
                bound = theirs < bound ? theirs : bound;
            }
            least = bound > least ? bound : least;
        };
        auto slot_max = [&](const u32x4& slot) {
            float m = -__builtin_inff();
#pragma unroll
            for (int e = 0; e < E; e += 2) m = max3(m, slot_entry<BF16>(slot, e), slot_entry<BF16>(slot, e + 1));
            return m;
        };

        // The same of a bfloat16 slot with an entry over 0; of others, one of their entries.  (As 16-bit numbers those over 0 lie above the others, in their order.)
        auto slot_max_over_0 = [&](const u32x4& slot) {
            const i16x2 a = __builtin_elementwise_max(__builtin_bit_cast(i16x2, static_cast<unsigned>(slot[0])), __builtin_bit_cast(i16x2, static_cast<unsigned>(slot[1])));
            const i16x2 b = __builtin_elementwise_max(__builtin_bit_cast(i16x2, static_cast<unsigned>(slot[2])), __builtin_bit_cast(i16x2, static_cast<unsigned>(slot[3])));
            const unsigned m = __builtin_bit_cast(unsigned, __builtin_elementwise_max(a, b));
            const int low = static_cast<int>(m << 16), high = static_cast<int>(m & 0xFFFF0000u);
            return __int_as_float(low > high ? low : high);
        };

        // the first chunk's bound
        float mine = -__builtin_inff();                           // the lane's largest so far
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            if (kChunk > slots) behind(r[i], i * T + tid);
            mine = __builtin_fmaxf(mine, slot_max(r[i]));
        }
        {
            const unsigned bound = wave_bound<BF16>(ordered(mine + 0.0f), q);
            if (lane == 0) __hip_atomic_store(&bounds[wave], bound, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
        __syncthreads();
        all_bounds();

        bool broken = false;                                      // an entry is NaN or +inf
        u16x2 most_turned = {0, 0};                               // (TABLE: tells a NaN, the only ones beyond -inf)
        double sum[2] = {0.0, 0.0};
        // (The last chunk apart from the others: where a branch may or may not request, each slot's wait is one for all requests before it, and 98 MB of binary32 rows
        // take 31.3 us, not 30.)
        auto over_chunk = [&](int first, auto more) {
            const float from = from_ordered(least);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const int slot = first + i * T + tid;
                if (!decltype(more)::value && first + kChunk > slots) behind(r[i], slot);
                const float top = TABLE && from > 0.0f ? slot_max_over_0(r[i]) : slot_max(r[i]);
                mine = __builtin_fmaxf(mine, top);
                // a slot with an entry that reaches the bound is put aside whole, to be taken apart with others
                const unsigned long who = __ballot(top >= from);
                if (who != 0) {
                    if (top >= from) {
                        const int k = aside + __popcll(who & ((1ul << lane) - 1));
                        aside_slot[wave][k] = r[i];
                        aside_at[wave][k] = slot;
                    }
                    aside += __popcll(who);
                    if (aside > kAside - 64) take_apart();
                }
                if constexpr (!TABLE) {
#pragma unroll
                    for (int e = 0; e < E; e += 2) broken |= __builtin_isunordered(slot_entry<BF16>(r[i], e), slot_entry<BF16>(r[i], e + 1));
                }
                if constexpr (TABLE) {                            // (also where it does not hold: then all of it is gone over again)
                    u16x2 least_index = {0xFFFF, 0xFFFF}, index[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const u16x2 v = __builtin_bit_cast(u16x2, static_cast<unsigned>(r[i][j]));
                        const u16x2 turned = twice_and(v, v >> static_cast<unsigned short>(15));   // the sign behind the rest
                        most_turned = __builtin_elementwise_max(most_turned, turned);
                        index[j] = __builtin_elementwise_min(__builtin_elementwise_sub_sat(turned, u16x2{2 * kTableBase + 1, 2 * kTableBase + 1}), u16x2{kTableEnd, kTableEnd});
                        least_index = __builtin_elementwise_min(least_index, index[j]);
                    }
                    double e[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const unsigned both = __builtin_bit_cast(unsigned, index[j]);
                        e[2 * j] = *reinterpret_cast<const double*>(reinterpret_cast<const char*>(table) + eight_times<0>(both));
                        e[2 * j + 1] = *reinterpret_cast<const double*>(reinterpret_cast<const char*>(table) + eight_times<1>(both));
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j & 1] += e[j];
                    if (__ballot(least_index.x == 0 || least_index.y == 0) != 0) {
                        sum[0] += rest_of_small(r[i]);            // (in a few slots of a hundred)
                    }
                } else {
                    // (what is under -700 counts as -700: nothing beside a largest entry of -600 or more)
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        sum[0] += exp_within(static_cast<double>(at_least_700_below(slot_entry<BF16>(r[i], e))));
                        sum[1] += exp_within(static_cast<double>(at_least_700_below(slot_entry<BF16>(r[i], e + 1))));
                    }
                }
                if constexpr (decltype(more)::value) r[i] = request(slot + kChunk);
            }
        };
        int first = 0;
        for (int chunk = 0; first + kChunk < all_slots; first += kChunk, ++chunk) {
            over_chunk(first, std::true_type{});
            // the bound anew where the entries seen have doubled
            if ((chunk & (chunk + 1)) == 0 && chunk > 0) {
                const unsigned bound = wave_bound<BF16>(ordered(mine + 0.0f), q);
                if (lane == 0) __hip_atomic_store(&bounds[wave], bound, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            }
            if ((chunk & (chunk - 1)) == 0) all_bounds();     // (the others' by then)
        }
        over_chunk(first, std::false_type{});
        if constexpr (TABLE) broken = most_turned.x > kTurnedInf || most_turned.y > kTurnedInf;
        const float top = wave_largest(mine);
        double ref = top > -__builtin_inff() ? 0.0 : -__builtin_inf();
        if ((TABLE ? top >= 64.0f || top < -20.0f : top > 600.0f || top < -600.0f) && top > -__builtin_inff()) {
            // again, as e^(z - top)
            ref = top;
            sum[0] = sum[1] = 0.0;
            for (int slot = tid; slot < all_slots; slot += T) {
                u32x4 x = request(slot);
                behind(x, slot);
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e & 1] += exp_below(static_cast<double>(slot_entry<BF16>(x, e)) - ref);
            }
        }
        double s = wave_sum_64(sum[0] + sum[1]);
        if (!(top > -__builtin_inff())) s = 0.0;
        // One entry (or one beside which the others are nothing) has its sum without an error: what is certain has the beam's score itself, and ties with others that have.
        if (s == exp_within(static_cast<double>(top) - ref)) ref = top, s = 1.0;   // (NaN where there is no entry)
        const bool any_broken = __ballot(broken || !(mine < __builtin_inff())) != 0;
        // the final bound, made of all wavefronts' entries
        {
            const unsigned bound = wave_bound<BF16>(ordered(mine + 0.0f), q);
            if (lane == 0) {
                wave_ref[wave] = ref;
                wave_sum[wave] = any_broken ? __builtin_nan("") : s;
                __hip_atomic_store(&bounds[wave], bound, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            }
        }
        __syncthreads();
        all_bounds();
        take_apart();
        count = keep_reaching(mine_list, count, least, lane);
        if (lane == 0) lds[wave] = full ? kWaveList + 1 : count;
        __syncthreads();
        int counts[NW], have = 0, most = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            counts[w] = uniform(lds[w]);
            have += counts[w];
            most = counts[w] > most ? counts[w] : most;
        }
        const size_t at = static_cast<size_t>(row) * P.S + slice;   // of [B, W * S]
        const int b = static_cast<int>(row / static_cast<unsigned>(P.W));
        const size_t lists = P.lists, column = at - static_cast<size_t>(b) * lists;
        float2* const cand = P.cand + static_cast<size_t>(b) * P.n * lists + column;
        auto put = [&](int rank, unsigned long me) {
            if (rank < P.n)
                cand[rank * lists] = make_float2(from_ordered(static_cast<unsigned>(me >> 32)), __uint_as_float(static_cast<unsigned>(begin) + ~static_cast<unsigned>(me)));
        };
        if (most <= 64) {
            // a lane holds an entry of each wavefront's; a wavefront finds the ranks of its own one after the other
            unsigned long other[NW];
#pragma unroll
            for (int w = 0; w < NW; ++w) other[w] = lane < counts[w] ? list[w * kWaveList + lane] : 0;
            const unsigned long own = lane < count ? mine_list[lane] : 0;
            int my_rank = 0;
#pragma unroll 4
            for (int k = 0; k < count; ++k) {
                const unsigned long me = lane_word(own, k);
                int rank = 0;
#pragma unroll
                for (int w = 0; w < NW; ++w) rank += __popcll(__ballot(other[w] > me));
                my_rank = lane == k ? rank : my_rank;
            }
            if (lane < count) put(my_rank, own);
        } else {
            if (most > kWaveList) {
                __syncthreads();                                  // (all have read the counts)
                have = slice_cut<BF16, NW>(z, begin, end, P.n, list, lds, tid);
#pragma unroll
                for (int w = 0; w < NW; ++w) counts[w] = w == 0 ? have : 0;   // (at most n of them)
                count = wave == 0 ? have : 0;
            }
            // a lane two entries of its wavefront's, which all are compared with (a broadcast each)
            for (int k = lane; k < count; k += 128) {
                const unsigned long me = mine_list[k], next = k + 64 < count ? mine_list[k + 64] : ~0ul;
                int rank = 0, rank_next = 0;
#pragma unroll
                for (int w = 0; w < NW; ++w)
#pragma unroll 8
                    for (int j = 0; j < counts[w]; ++j) {
                        const unsigned long theirs = list[w * kWaveList + j];
                        rank += theirs > me;
                        rank_next += theirs > next;
                    }
                put(rank, me);
                if (k + 64 < count) put(rank_next, next);
            }
        }
        for (int k = have + tid; k < P.n; k += T) cand[k * lists] = make_float2(-__builtin_inff(), 0.0f);
        if (tid == T - 1) {
            double m = -__builtin_inf(), total = 0.0;
            for (int w = 0; w < NW; ++w) m = wave_ref[w] > m ? wave_ref[w] : m;
            for (int w = 0; w < NW; ++w) {
                const double d = wave_ref[w] - m;                 // (NaN where the slice has no entry)
                total += d < 0.0 ? (wave_ref[w] > -__builtin_inf() ? wave_sum[w] * exp_below(d) : wave_sum[w]) : wave_sum[w];
            }
            P.stat[at] = make_double2(m, total);
        }
        __syncthreads();                                          // (the next slice's bounds and lists go where these were)
    }
}

// ------------------------------------------------------------------------------------------ merging

// A continuation: its rank, (beam, token + 1), its logit.  A rank's rounding may take logits of one beam for equal: then the logits decide.
// As a word, the lower of which comes first among equal ranks: 8 bits of the beam, 32 of the logit, the larger the lower, 20 of token + 1.
__device__ __forceinline__ unsigned long found_word(int beam, float z, int token1) {
    return static_cast<unsigned long>(beam) << 52 | static_cast<unsigned long>(~ordered(z)) << 20 | static_cast<unsigned>(token1);
}
// of a logit, given its row's normaliser
__device__ __forceinline__ double log_share(float z, double2 norm) { return (static_cast<double>(z) - norm.x) - norm.y; }
constexpr int kMergeFew = 256;      // entries that are put into order as they are; of more, the n best are looked for first

// 64-bit order of binary64 numbers, as ordered() is for binary32 ones; the upper word
__device__ __forceinline__ unsigned ordered_high(double x) {
    const unsigned u = static_cast<unsigned>(__builtin_bit_cast(unsigned long, x) >> 32);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A sequence a workgroup of T threads.  All entries of its lists (or EACH a thread at a time) are ranked in registers; a wavefront's q-th largest, q =
// n / wavefronts rounded up, bounds the n-th largest of all from below as in beam_slices, and the few that reach the least of these are ordered in LDS.
template <int T, int EACH>
__global__ void __launch_bounds__(T) beam_merge(const BeamParams P) {
    constexpr int NW = T / 64, kRoom = T + kBeamMost;
    __shared__ double key[kRoom + 8];
    __shared__ unsigned long found[kRoom + 8];
    __shared__ double best_key[kBeamMost];
    __shared__ unsigned long best[kBeamMost];
    // A row's normaliser in two parts, a number r and log of the sum of e^(z - r): in one, the logarithm would be lost beside an r of 2^53 (a row of the
    // type's lowest number, from a mask that leaves nothing, would have continuations of probability 1).
    __shared__ double2 norm[kBeamWidest];
    __shared__ float base[kBeamWidest];                       // a beam's score; NaN: its list does not count
    __shared__ float so_far[kBeamWidest];
    __shared__ float factor[kBeamWidest];
    __shared__ unsigned wave_bound[NW], wave_alone[NW];
    __shared__ int wave_count[2][NW];
    __shared__ int have, bad;
    const int tid = threadIdx.x, wave = uniform(tid / 64), b = blockIdx.x, W = P.W, S = P.S, n = P.n;
    const int lists = P.lists;
    const long first = static_cast<long>(b) * W;
    const size_t out = static_cast<size_t>(b) * n;
    const float2* cand = P.cand + out * lists;
    if (tid == 0) have = 0, bad = 0;
    const int total = lists * n;                              // (at most 2^21)
    const int column_step = T % lists;
    float z[EACH];
    int token[EACH];
    // entry k of the lists: the (k / lists)-th of list k % lists
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int k = k0 + i * T + tid;
            const float2 c = k < total ? cand[k] : make_float2(-__builtin_inff(), 0.0f);
            z[i] = c.x;
            token[i] = static_cast<int>(__float_as_uint(c.y));
        }
    };
    load(0);                                                  // (on the way while the normalisers are made)
    __syncthreads();
    // normalisers: 16 lanes a beam
    for (int w0 = 0; w0 < W; w0 += T / 16) {
        const int w = w0 + tid / 16, part = tid % 16;
        double m = -__builtin_inf(), s = 0.0;
        float score = 0.0f, by = 1.0f;
        bool lives = false, ended = false, runs = false, broken = false;
        const double2* stat = P.stat + (first + w) * S;
        double2 own = make_double2(m, 0.0);
        if (w < W && part < S) own = stat[part];              // (of a beam that does not run, anything: requested together with what says so)
        if (w < W) {
            score = score_of(P, first + w);
            if (P.weights) by = P.weights[first + w];
            ended = P.done && P.done[first + w];
            lives = !(score <= -__builtin_inff());
            broken = lives && !(score < __builtin_inff() && by > 0.0f && by < __builtin_inff());
            runs = lives && score == score && !ended;
        }
        if (runs) {
            m = own.x;
            broken |= own.y != own.y;
            for (int k = part + 16; k < S; k += 16) {
                const double2 x = stat[k];
                m = x.x > m ? x.x : m;
                broken |= x.y != x.y;
            }
        }
        m = row_max(m);
        if (runs && m > -__builtin_inf()) {
            // (exact powers: the polynomial's error enters an entry's exponential and, where a slice's wavefronts differ, that of their distance; 4.03e-11 a third time
            // would be more than 2^-33)
            if (own.x > -__builtin_inf()) s = own.y * exp(own.x - m);
            for (int k = part + 16; k < S; k += 16) {
                const double2 x = stat[k];
                if (x.x > -__builtin_inf()) s += x.y * exp(x.x - m);
            }
        }
        s = row_sum(s);
        if (broken) bad = 1;                                  // (whoever writes it writes the same)
        if (w < W && part == 0) {
            const bool counts = runs && m > -__builtin_inf();
            norm[w] = counts ? make_double2(m, log(s)) : make_double2(0.0, 0.0);
            base[w] = counts ? score : __builtin_nanf("");
            factor[w] = by;
            so_far[w] = score;
            if (lives && ended && !broken) {                  // a finished beam, as it stands
                const int at = atomicAdd(&have, 1);
                key[at] = static_cast<double>(score) * static_cast<double>(by);
                found[at] = found_word(w, 0.0f, 0);
            }
        }
    }
    __syncthreads();
    if (bad) {
        for (int i = tid; i < n; i += T) {
            P.scores_out[out + i] = -__builtin_inff();
            P.parent[out + i] = -1;
            P.tokens[out + i] = -1;
        }
        if (tid == 0 && P.status) P.status[b] = FSD_ROW_NONFINITE;
        return;
    }
    auto beam_of = [&](int l) { return P.by_S ? static_cast<int>(__umulhi(static_cast<unsigned>(l), P.by_S)) : l; };
    double last_key = -__builtin_inf();                       // the n-th best of what has been ordered
    unsigned long last = ~0ul;
    int count = uniform(have);
    __syncthreads();
    // the n best of found[0 .. count) to its front, best first
    auto order = [&]() {
        if (tid < 8) key[count + tid] = -__builtin_inf();
        __syncthreads();
        if (count <= 128) {                                   // a lane holds two of them; a wavefront finds the ranks of its share one after the other
            const int lane = tid % 64;
            const double k0 = lane < count ? key[lane] : -__builtin_inf(), k1 = lane + 64 < count ? key[lane + 64] : -__builtin_inf();
            const unsigned long f0 = lane < count ? found[lane] : ~0ul, f1 = lane + 64 < count ? found[lane + 64] : ~0ul;
            int rank0 = 0, rank1 = 0;
            auto rank_of = [&](double mine, unsigned long me) {
                return __popcll(__ballot((k0 > mine) | ((k0 == mine) & (f0 < me)))) + __popcll(__ballot((k1 > mine) | ((k1 == mine) & (f1 < me))));
            };
            const int in_first = count < 64 ? count : 64;
#pragma unroll 4
            for (int k = wave; k < in_first; k += NW) {
                const int rank = rank_of(lane_value(k0, k), lane_word(f0, k));
                rank0 = lane == k ? rank : rank0;
            }
#pragma unroll 4
            for (int k = 64 + wave; k < count; k += NW) {
                const int rank = rank_of(lane_value(k1, k - 64), lane_word(f1, k - 64));
                rank1 = lane == k - 64 ? rank : rank1;
            }
            if (lane < count && lane % NW == wave && rank0 < n) best_key[rank0] = k0, best[rank0] = f0;
            if (lane + 64 < count && (lane + 64) % NW == wave && rank1 < n) best_key[rank1] = k1, best[rank1] = f1;
        } else {                                              // a thread an entry, which all others are compared with (a broadcast each)
            for (int k = tid; k < count; k += T) {
                const double mine = key[k];
                const unsigned long me = found[k];
                int rank = 0;
                for (int j = 0; j < count; j += 8) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) rank += (key[j + u] > mine) | ((key[j + u] == mine) & (found[j + u] < me));
                }
                if (rank < n) {
                    best_key[rank] = mine;
                    best[rank] = me;
                }
            }
        }
        __syncthreads();
        count = count < n ? count : n;
        for (int k = tid; k < count; k += T) {
            key[k] = best_key[k];
            found[k] = best[k];
        }
        if (count == n) last_key = best_key[n - 1], last = best[n - 1];
        if (tid == 0) have = count;
        __syncthreads();
    };
    for (int k0 = 0; k0 < total; k0 += T * EACH) {
        double rank[EACH];
        double most = -__builtin_inf();
        {
            int l = (k0 + tid) % lists;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int w = beam_of(l);
                const float from = base[w];
                rank[i] = -__builtin_inf();
                if (from == from && z[i] > -__builtin_inff())
                    rank[i] = (static_cast<double>(from) + log_share(z[i], norm[w])) * static_cast<double>(factor[w]);
                most = rank[i] > most ? rank[i] : most;
                l += column_step;
                l -= l >= lists ? lists : 0;
            }
        }
        // Lists fall: where no entry of a whole row of them (their r-th ones) reaches the n-th best so far, none behind it does.
        if (k0 > 0 && count == n && !__syncthreads_or(most >= last_key) && 2 * lists <= T * EACH) break;
        const unsigned word = ordered_high(most);
        const int q = (n + NW - 1) / NW;
        unsigned bound = 0, alone = 0;                        // its q-th largest, and its n-th: what n of its own reach bounds the n-th of all as well
        for (int bit = 31; bit >= 12; --bit) {                // (the upper 20 bits)
            const unsigned c = bound | 1u << bit, d = alone | 1u << bit;
            if (__popcll(__ballot(word >= c)) >= q) bound = c;
            if (__popcll(__ballot(word >= d)) >= n) alone = d;
        }
        if (tid % 64 == 0) wave_bound[wave] = bound, wave_alone[wave] = alone;
        __syncthreads();
        for (int i = 0; i < NW; ++i) bound = wave_bound[i] < bound ? wave_bound[i] : bound;
        for (int i = 0; i < NW; ++i) bound = wave_alone[i] > bound ? wave_alone[i] : bound;
        // (an entry that is none has the word of -inf; every other one a larger word)
        const unsigned none = ordered_high(-__builtin_inf());
        bound = bound > none ? bound : none + 1;
        int reach, at, all;                                   // of the wavefront; where its first goes; of the workgroup
        auto places = [&]() {                                 // of the wavefront's entries that reach the bound (in any order: they are put into order afterwards)
            reach = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) reach += __popcll(__ballot(ordered_high(rank[i]) >= bound && rank[i] >= last_key));
            at = 0;
            if (tid % 64 == 0 && reach != 0) at = atomicAdd(&have, reach);
            at = __builtin_amdgcn_readfirstlane(at);
            __syncthreads();
            all = uniform(have);
        };
        places();
        if (all - count > kMergeFew) {
            // A bound far under the n-th largest (one beam's lists have most of the best): bit by bit, by all entries
            bound = 0;
            for (int bit = 31; bit >= 0; --bit) {
                const unsigned c = bound | 1u << bit;
                int n_c = 0;
#pragma unroll
                for (int i = 0; i < EACH; ++i) n_c += __popcll(__ballot(ordered_high(rank[i]) >= c));
                if (tid % 64 == 0) wave_count[bit & 1][wave] = n_c;
                __syncthreads();
                n_c = 0;
                for (int i = 0; i < NW; ++i) n_c += wave_count[bit & 1][i];
                if (n_c >= n) bound = c;
            }
            bound = bound > none ? bound : none + 1;
            if (tid == 0) have = count;
            __syncthreads();
            places();
        }
        if (all <= kRoom) {
            if (reach != 0) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const bool is = ordered_high(rank[i]) >= bound && rank[i] >= last_key;
                    const unsigned long who = __ballot(is);
                    if (is) {
                        const int to = at + __popcll(who & ((1ul << (tid % 64)) - 1));
                        key[to] = rank[i];
                        found[to] = found_word(beam_of((k0 + i * T + tid) % lists), z[i], token[i] + 1);
                    }
                    at += __popcll(who);
                }
            }
            if (k0 + T * EACH < total) load(k0 + T * EACH);       // (on the way meanwhile)
            count = all;
            __syncthreads();
            order();
        } else {
            // more than there is room for (equal ranks, lists of very unequal length): one entry a thread at a time
            __syncthreads();
            if (tid == 0) have = count;
            __syncthreads();
            if (count > n) order();
#pragma unroll 1
            for (int i = 0; i < EACH; ++i) {
                const int k = k0 + i * T + tid;
                double mine = rank[0];
#pragma unroll
                for (int j = 1; j < EACH; ++j) mine = i == j ? rank[j] : mine;
                if (mine > -__builtin_inf()) {
                    const float2 c = cand[k];
                    const unsigned long me = found_word(beam_of(k % lists), c.x, static_cast<int>(__float_as_uint(c.y)) + 1);
                    if (mine > last_key || (mine == last_key && me < last)) {
                        const int to = atomicAdd(&have, 1);
                        key[to] = mine;
                        found[to] = me;
                    }
                }
                __syncthreads();
                count = uniform(have);
                __syncthreads();
                if (count > n) order();
            }
            if (k0 + T * EACH < total) load(k0 + T * EACH);
            order();
        }
    }
    for (int i = tid; i < n; i += T) {
        const bool some = i < count;
        float s = -__builtin_inff();
        int beam = -1, token1 = 0;
        if (some) {
            const unsigned long me = found[i];
            beam = static_cast<int>(me >> 52);
            token1 = static_cast<int>(me & 0xFFFFFu);
            s = so_far[beam];
            if (token1 > 0) s = static_cast<float>(static_cast<double>(s) + log_share(from_ordered(~static_cast<unsigned>(me >> 20)), norm[beam]));
        }
        P.scores_out[out + i] = s;
        P.parent[out + i] = beam;
        P.tokens[out + i] = token1 - 1;
    }
    if (tid == 0 && P.status) P.status[b] = 0;
}

// ------------------------------------------------------------------------------------------ states

// A piece of a row a workgroup at a time, 16 bytes a thread and step on whatever address (a wavefront's kilobyte is one run, so that the hardware splits
// few of them).  Bound by the bytes: 163 MB read and written in 30 us, 5.4 TB/s, part of it in the caches; 53 KB in 2.8, a launch.
struct ReorderParams {
    const char* states;
    const int* parent;
    char* out;
    int* status;
    size_t row;                     // bytes
    long rows;                      // layers * B * n
    int B, W, n;
    int pieces;                     // of a row, of kReorderPiece bytes
    long units;                     // rows * pieces
};
constexpr int kReorderPiece = 16384;
typedef unsigned u32x4_bytes __attribute__((ext_vector_type(4), aligned(1)));

__global__ void __launch_bounds__(kWG) beam_reorder(const ReorderParams P) {
    const int tid = threadIdx.x;
    for (long u = blockIdx.x; u < P.units; u += gridDim.x) {
        const long row = u / P.pieces;
        const int piece = static_cast<int>(u - row * P.pieces);
        const long lb = row / P.n;
        const int i = static_cast<int>(row - lb * P.n), b = static_cast<int>(lb % P.B);
        const int w = P.parent[static_cast<size_t>(b) * P.n + i];
        const size_t begin = static_cast<size_t>(piece) * kReorderPiece, left = P.row - begin;
        const int bytes = left < kReorderPiece ? static_cast<int>(left) : kReorderPiece;
        const bool some = w >= 0 && w < P.W;
        const char* from = P.states + (static_cast<size_t>(lb) * P.W + (some ? w : 0)) * P.row + begin;
        char* to = P.out + static_cast<size_t>(row) * P.row + begin;
        const int slots = bytes / 16;
        for (int k = tid; k < slots; k += kWG) {
            u32x4_bytes x = {0, 0, 0, 0};
            if (some) x = *reinterpret_cast<const u32x4_bytes*>(from + k * 16);
            *reinterpret_cast<u32x4_bytes*>(to + k * 16) = x;
        }
        const int tail = slots * 16 + tid;
        if (tail < bytes) to[tail] = some ? from[tail] : 0;
        if (P.status && i == 0 && piece == 0 && lb < P.B && tid < 64) {   // a sequence's report, by one wavefront
            int wrong = 0;
            for (int k = tid; k < P.n; k += 64) {
                const int p = P.parent[static_cast<size_t>(b) * P.n + k];
                wrong |= p < -1 || p >= P.W;
            }
            if (__ballot(wrong != 0) != 0) wrong = 1;
            if (tid == 0) P.status[b] = wrong ? FSD_ROW_BAD_PARENT : 0;
        }
    }
}

}  // namespace

#endif  // FSD_CSRC_BEAM_SELECT_H_
