// The best continuations of a sequence's beams (fsd_beam_select) and the states that follow them (fsd_beam_reorder).
// Part of libfsd (gfx950).
//
// beam_slices goes over the logits once: a workgroup has a slice of one beam's row in registers, adds up its exponentials and writes its n
// best entries, best first.  beam_merge, a workgroup a sequence, makes the normalisers of the beams from the slices' sums and takes the n best of
// all slices' lists.  Order matters to the last bit (two beams' entries may lie as near to one another as their normalisers' errors), so
// exponentials, sums and ranks are binary64; on this machine a binary64 fma issues like a binary32 one, and the hardware's binary32
// exponential takes four times as long, so that this costs what a corrected binary32 exponential would.
#ifndef FSD_CSRC_BEAM_SELECT_H_
#define FSD_CSRC_BEAM_SELECT_H_

#include "operators_common.h"

namespace {

constexpr int kBeamMost = 128;      // n
constexpr int kBeamWidest = 256;    // beams
constexpr int kBeamList = 1024;     // entries of a slice that stand in LDS before the n best are taken from them
constexpr double kLog2e64 = 1.4426950408889634074;

struct BeamParams {
    const char* logits;
    size_t row_stride;              // bytes
    const float *scores, *weights;
    const int* done;
    int B, W, V, n;
    int len, S, lists;              // entries of a slice (a multiple of a 16-byte slot's), slices of a row, W * S
    float2* cand;                   // [B, n, W * S]: logit and token of a list's entry, best first
    int* count;                     // [B, W * S]
    double2* stat;                  // [B, W * S]: largest logit, sum of e^(z - largest)
    float* scores_out;
    int *parent, *tokens, *status;
};

// e^d for d <= 0, off by 2^-34 of it (under -690: next to nothing, NaN: NaN): d log2 e as a whole number k and a rest of at most 1/2; the rest's power by a
// polynomial of degree 7 (fitted to the smallest largest relative error on [-1/2, 1/2]), k into its exponent's bits.
__device__ __forceinline__ double exp_64(double d) {
    constexpr double kWhole = 6755399441055744.0;            // 1.5 * 2^52: what is added to it comes out whole, in the low word
    const double k = __builtin_fma(d, kLog2e64, kWhole), f = __builtin_fma(d, kLog2e64, kWhole - k);
    double p = 1.520192135287937e-05;
    p = __builtin_fma(p, f, 0.00015469291148729867);
    p = __builtin_fma(p, f, 0.001333392256490547);
    p = __builtin_fma(p, f, 0.009618027253635145);
    p = __builtin_fma(p, f, 0.05550410353445615);
    p = __builtin_fma(p, f, 0.24022651198157982);
    p = __builtin_fma(p, f, 0.693147180728448);
    p = __builtin_fma(p, f, 0.9999999999616819);
    const unsigned long bits = __builtin_bit_cast(unsigned long, p);
    unsigned hi = static_cast<unsigned>(bits >> 32) + (static_cast<unsigned>(__builtin_bit_cast(unsigned long, k)) << 20);
    hi = d < -690.0 ? 0u : hi;                               // (the low word alone is less than 2^-1042)
    return __builtin_bit_cast(double, static_cast<unsigned long>(hi) << 32 | (bits & 0xFFFFFFFFul));
}
// bits of a number in an order in which larger numbers have larger words (0 and -0 differ: give it neither as -0)
__device__ __forceinline__ unsigned ordered(float x) {
    const unsigned u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(unsigned o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
constexpr unsigned kLeastOrdered = 0x00800000u;   // of the lowest finite number

template <bool BF16>
__device__ __forceinline__ float slot_entry(const uint4& r, int e) {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
    if constexpr (BF16) return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    else return __uint_as_float(w[e]);
}

__device__ __forceinline__ float score_of(const BeamParams& P, long at) { return P.scores ? P.scores[at] : 0.0f; }
__device__ __forceinline__ bool beam_runs(const BeamParams& P, long at) {   // whether a beam's row is read
    return score_of(P, at) > -__builtin_inff() && !(P.done && P.done[at]);   // (a score that is NaN is reported without its row)
}

// A slice's n best entries where more than kBeamList reach the bound that its lanes gave (rows of equal entries, or in order): the n-th largest
// is found bit by bit, then what is above it and, from the lowest index on, what equals it go into the list.  Returns how many.
template <bool BF16, int NS>
__device__ int slice_cut(const uint4 (&r)[NS], int n, unsigned long* list, int* lds, int tid) {
    constexpr int E = BF16 ? 8 : 4;
    const int wave = tid / 64, lane = tid % 64;
    auto over_wg = [&](int c) {                              // the sum of all threads' c
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
        __syncthreads();
        if (lane == 0) lds[wave] = c;
        __syncthreads();
        return lds[0] + lds[1] + lds[2] + lds[3];
    };
    unsigned least = 0;
    for (int bit = 31; bit >= (BF16 ? 16 : 0); --bit) {
        const unsigned c = least | 1u << bit;
        int have = 0;
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) have += ordered(slot_entry<BF16>(r[i], e) + 0.0f) >= c;
        if (over_wg(have) >= n) least = c;
    }
    // (of bfloat16 entries the low 16 bits: 0 of a positive one, 1 of a negative one, so that this is its lowest word or one that no entry has)
    if (BF16 && !(least & 0x80000000u)) least |= 0xFFFFu;
    if (least < kLeastOrdered) least = kLeastOrdered;
    int above = 0;
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) above += ordered(slot_entry<BF16>(r[i], e) + 0.0f) > least;
    const int more = over_wg(above);
    if (tid == 0) lds[4] = 0;
    int before = 0;                                          // entries that equal it, of the slots behind us
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < NS; ++i) {
        uint4 slot = r[0];
#pragma unroll
        for (int k = 1; k < NS; ++k) slot = i == k ? r[k] : slot;
        int same = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) same += ordered(slot_entry<BF16>(slot, e) + 0.0f) == least;
        int upto = same;                                     // of this and the lanes below
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int other = __shfl_up(upto, o, 64);
            if (lane >= o) upto += other;
        }
        __syncthreads();
        if (lane == 63) lds[wave] = upto;
        __syncthreads();
        int at = before + upto - same;
        for (int w = 0; w < wave; ++w) at += lds[w];
        before += lds[0] + lds[1] + lds[2] + lds[3];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const unsigned o = ordered(slot_entry<BF16>(slot, e) + 0.0f);
            const bool equal = o == least;
            if (o > least || (equal && at < n - more)) {
                const int k = atomicAdd(&lds[4], 1);
                list[k] = static_cast<unsigned long>(o) << 32 | ~static_cast<unsigned>((i * kWG + tid) * E + e);
            }
            at += equal;
        }
    }
    __syncthreads();
    return lds[4];
}

// One slice of a row a workgroup, NS slots of 16 bytes a thread.  A wavefront's q-th largest lane maximum, q = n / 4 rounded up, is
// reached by q entries of its own at least, so the least of the four wavefronts' by n of the slice: what reaches that bound (a few more than n entries
// where the values lie as those of logits do) is written to LDS and ranked there.
template <bool BF16, int NS>
__global__ void __launch_bounds__(kWG) beam_slices(const BeamParams P) {
    constexpr int E = BF16 ? 8 : 4;
    __shared__ unsigned long list[kBeamList];
    __shared__ double wave_sum[4];
    __shared__ float wave_top[4];
    __shared__ unsigned wave_bound[4];
    __shared__ int lds[5];
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const long row = blockIdx.x / P.S;
    const int slice = static_cast<int>(blockIdx.x - row * P.S);
    if (!beam_runs(P, row)) return;
    const int begin = slice * P.len, end = begin + P.len < P.V ? begin + P.len : P.V;
    const char* z = P.logits + static_cast<size_t>(row) * P.row_stride;
    uint4 r[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int at = begin + (i * kWG + tid) * E;
        if (at + E <= end) r[i] = load_any16(z + static_cast<size_t>(at) * (16 / E));
        else r[i] = neg_inf_slot<BF16>();
    }
    // the entries behind the row's last whole slot: its thread takes them one by one
    const int whole = begin + (end - begin) / E * E;
    if (whole < end) {
        const int slot = (end - begin) / E;
        unsigned w[4];
        const uint4 none = neg_inf_slot<BF16>();
        w[0] = none.x; w[1] = none.y; w[2] = none.z; w[3] = none.w;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (whole + e < end) {
                if constexpr (BF16) {
                    const unsigned h = reinterpret_cast<const unsigned short*>(z)[whole + e];
                    w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | h << 16 : (w[e / 2] & 0xFFFF0000u) | h;
                } else {
                    w[e] = reinterpret_cast<const unsigned*>(z)[whole + e];
                }
            }
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i * kWG + tid == slot) r[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (tid == 0) lds[4] = 0;

    float mine = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) mine = __builtin_fmaxf(mine, slot_entry<BF16>(r[i], e));
    const float top = wave_max_all(mine);

    // the wavefront's bound, to the upper 20 bits
    const unsigned word = ordered(mine + 0.0f);
    const int q = (P.n + 3) / 4;
    unsigned bound = 0;
    for (int bit = 31; bit >= (BF16 ? 16 : 12); --bit) {
        const unsigned c = bound | 1u << bit;
        if (__popcll(__ballot(word >= c)) >= q) bound = c;
    }

    // the wavefront's sum (NaN stays in it)
    const double highest = top;
    double sum[2] = {0.0, 0.0};
    if (top > -__builtin_inff()) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e & 1] += exp_64(static_cast<double>(slot_entry<BF16>(r[i], e)) - highest);
    }
    double s = sum[0] + sum[1];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    // an entry that is NaN or +inf: largest and sum are no numbers then (a wavefront of NaN alone has no largest entry)
    bool broken = false;
    if (!(top > -__builtin_inff())) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = slot_entry<BF16>(r[i], e);
                broken |= x != x;
            }
        broken = __ballot(broken) != 0;
    }
    if (lane == 0) {
        wave_top[wave] = top;
        wave_sum[wave] = broken || !(top < __builtin_inff()) ? __builtin_nan("") : s;
        wave_bound[wave] = bound;
    }
    __syncthreads();
    unsigned least = wave_bound[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) least = wave_bound[w] < least ? wave_bound[w] : least;
    if (least < kLeastOrdered) least = kLeastOrdered;
    const float from = from_ordered(least);
    const size_t at = static_cast<size_t>(row) * P.S + slice;   // of [B, W * S]
    if (tid == 0) {
        double m = -__builtin_inf(), total = 0.0;
        for (int w = 0; w < 4; ++w) m = wave_top[w] > m ? static_cast<double>(wave_top[w]) : m;
        for (int w = 0; w < 4; ++w) {
            const double ws = wave_sum[w];
            if (ws != ws) total = ws;
            else if (wave_top[w] > -__builtin_inff()) total += ws * exp_64(static_cast<double>(wave_top[w]) - m);
        }
        P.stat[at] = make_double2(m, total);
    }

    if (mine >= from) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = slot_entry<BF16>(r[i], e);
                if (x >= from) {
                    const int k = atomicAdd(&lds[4], 1);
                    if (k < kBeamList) list[k] = static_cast<unsigned long>(ordered(x + 0.0f)) << 32 | ~static_cast<unsigned>((i * kWG + tid) * E + e);
                }
            }
    }
    __syncthreads();
    int have = lds[4];
    if (have > kBeamList) have = slice_cut<BF16, NS>(r, P.n, list, lds, tid);
    const int b = static_cast<int>(row / P.W);
    const size_t lists = P.lists, column = at - static_cast<size_t>(b) * lists;
    for (int k = tid; k < have; k += kWG) {
        const unsigned long me = list[k];
        int rank = 0;
        for (int j = 0; j < have; ++j) rank += list[j] > me;
        if (rank < P.n)
            P.cand[(static_cast<size_t>(b) * P.n + rank) * lists + column] =
                make_float2(from_ordered(static_cast<unsigned>(me >> 32)), __uint_as_float(static_cast<unsigned>(begin) + ~static_cast<unsigned>(me)));
    }
    if (tid == 0) P.count[at] = have < P.n ? have : P.n;
}

// ------------------------------------------------------------------------------------------ merging

constexpr int kNoBeam = kBeamWidest;

// A continuation: its rank, (beam, token + 1), its logit.  A rank's rounding may take logits of one beam for equal: then the logits decide.
struct Ranked { double key; int beam, token1; float z; };
__device__ __forceinline__ bool before(const Ranked& a, const Ranked& b) {
    if (a.key != b.key) return a.key > b.key;
    if (a.beam != b.beam) return a.beam < b.beam;
    return a.z != b.z ? a.z > b.z : a.token1 < b.token1;
}

// A sequence a workgroup.  The lists' first entries come first, then their second ones, and so on: after the first few hundred of them
// the n-th best so far turns nearly all others away, and where as many in a row as there are lists were turned away, so are all behind them.
__global__ void __launch_bounds__(kWG) beam_merge(const BeamParams P) {
    __shared__ Ranked found[3 * kWG];
    __shared__ Ranked best[kBeamMost];
    __shared__ double norm[kBeamWidest];
    __shared__ int have, bad;
    const int tid = threadIdx.x, b = blockIdx.x, W = P.W, S = P.S, n = P.n;
    const long lists = P.lists;
    const long first = static_cast<long>(b) * W;
    const float* weights = P.weights ? P.weights + first : nullptr;
    const int* done = P.done ? P.done + first : nullptr;
    if (tid == 0) have = 0, bad = 0;
    __syncthreads();
    // normalisers: 16 lanes a beam
    for (int w0 = 0; w0 < W; w0 += kWG / 16) {
        const int w = w0 + tid / 16, part = tid % 16;
        double m = -__builtin_inf(), s = 0.0;
        bool runs = false, broken = false;
        if (w < W) {
            const float score = score_of(P, first + w);
            const bool lives = !(score <= -__builtin_inff());
            const bool ended = done && done[w];
            broken = lives && !(score < __builtin_inff());
            if (lives && weights) broken |= !(weights[w] > 0.0f && weights[w] < __builtin_inff());
            runs = lives && score == score && !ended;
        }
        const double2* stat = P.stat + static_cast<size_t>(b) * lists + static_cast<size_t>(w) * S;
        if (runs) {
            for (int k = part; k < S; k += 16) {
                const double2 x = stat[k];
                m = x.x > m ? x.x : m;
                broken |= x.y != x.y;
            }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            const double other = __shfl_xor(m, o, 16);
            m = other > m ? other : m;
        }
        if (runs && m > -__builtin_inf()) {
            for (int k = part; k < S; k += 16) {
                const double2 x = stat[k];
                if (x.x > -__builtin_inf()) s += x.y * exp_64(x.x - m);
            }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) s += __shfl_xor(s, o, 16);
        if (broken) bad = 1;                                  // (whoever writes it writes the same)
        if (w < W && part == 0) {
            norm[w] = runs && m > -__builtin_inf() ? m + log(s) : 0.0;
        }
    }
    __syncthreads();
    const size_t out = static_cast<size_t>(b) * n;
    if (bad) {
        for (int i = tid; i < n; i += kWG) {
            P.scores_out[out + i] = -__builtin_inff();
            P.parent[out + i] = -1;
            P.tokens[out + i] = -1;
        }
        if (tid == 0 && P.status) P.status[b] = FSD_ROW_NONFINITE;
        return;
    }
    // finished beams, as they stand
    if (done && tid < W && done[tid] && score_of(P, first + tid) > -__builtin_inff()) {
        const float s = score_of(P, first + tid);
        const double by = weights ? static_cast<double>(weights[tid]) : 1.0;
        found[atomicAdd(&have, 1)] = Ranked{static_cast<double>(s) * by, tid, 0, 0.0f};
    }
    __syncthreads();
    Ranked last = {-__builtin_inf(), kNoBeam, 0, 0.0f};      // the n-th best of what has been ranked
    auto rank_found = [&](int count) {                        // the n best of found[0 .. count) to its front, best first
        for (int k = tid; k < count; k += kWG) {
            const Ranked me = found[k];
            int rank = 0;
            for (int j = 0; j < count; ++j) rank += before(found[j], me);
            if (rank < n) best[rank] = me;
        }
        __syncthreads();
        const int left = count < n ? count : n;
        for (int k = tid; k < left; k += kWG) found[k] = best[k];
        if (left == n) last = best[n - 1];
        if (tid == 0) have = left;
        __syncthreads();
    };
    const long total = lists * n;
    long quiet = 0;
    int count = have;
    __syncthreads();
    for (long k0 = 0; k0 < total && quiet < lists; k0 += kWG) {
        const long k = k0 + tid;
        bool take = false;
        Ranked me = {0.0, 0, 0, 0.0f};
        if (k < total) {
            const int r = static_cast<int>(k / lists), l = static_cast<int>(k - static_cast<long>(r) * lists), w = l / S;
            if (beam_runs(P, first + w) && r < P.count[static_cast<size_t>(b) * lists + l]) {
                const float2 c = P.cand[(out + r) * lists + l];
                const double s = static_cast<double>(score_of(P, first + w)) + (static_cast<double>(c.x) - norm[w]);
                me = Ranked{weights ? s * static_cast<double>(weights[w]) : s, w, static_cast<int>(__float_as_uint(c.y)) + 1, c.x};
                take = before(me, last);
            }
        }
        if (take) found[atomicAdd(&have, 1)] = me;
        __syncthreads();
        const int now = have;
        __syncthreads();
        quiet = now == count ? quiet + kWG : 0;
        count = now;
        if (count >= 2 * kWG || (count > n && last.beam == kNoBeam)) {
            rank_found(count);
            count = have;
            __syncthreads();
        }
    }
    rank_found(count);
    count = have;
    for (int i = tid; i < n; i += kWG) {
        const bool some = i < count;
        const Ranked me = found[some ? i : 0];
        float s = -__builtin_inff();
        if (some) {
            s = score_of(P, first + me.beam);
            if (me.token1 > 0) s = static_cast<float>(static_cast<double>(s) + (static_cast<double>(me.z) - norm[me.beam]));
        }
        P.scores_out[out + i] = s;
        P.parent[out + i] = some ? me.beam : -1;
        P.tokens[out + i] = some ? me.token1 - 1 : -1;
    }
    if (tid == 0 && P.status) P.status[b] = 0;
}

// ------------------------------------------------------------------------------------------ states

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
