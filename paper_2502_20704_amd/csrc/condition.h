// Penalties for repeated tokens, biases and grammar masks on the rows of a verify call (fsd_condition_*).
// Part of libfsd (gfx950); included by operators.hip, which holds the host side and the C ABI.
//
//   z1 = seen ? (z > 0 ? z / r : z r) : z;  z2 = z1 - f count - (count ? p : 0);  z3 = z2 + bias;  -inf where not allowed
//
// A workgroup takes a run of `slice` vocabulary entries and some rows of one sequence.  It goes over the sequence's
// history once and counts in LDS the tokens that fall into its slice (integer atomics: the order does not matter), then
// streams its rows: one bit an entry tells whether the table says anything about it, so that nearly every 16-byte
// slot is copied (or masked) as it is.  What a row's own way adds is put into the table when the row needs it: along a chain
// the contexts contain one another and each row adds one candidate; in a tree a row takes away and adds what its way and that of the row before
// do not share, of tokens in the slice only (most rows: nothing).  No row keeps another one waiting otherwise: there is no barrier between them.
//
// What bounds it is memory: 64 x 9 rows of 128256 bfloat16 entries 71 us (4.2 TB/s read and written; a copy of that size 58), 32 trees of 60 rows under
// a mask each 186 (of 492 MB 291 are read, as slots without an allowed entry are not: 4.2 TB/s), 48 x 17 rows of 128259 binary32 entries with histories of
// 32768 201 (4.2 TB/s).  One row of 32000: 4.5 us, a kernel's start and its two round trips, history and row.
// Deep trees: one thread walks between two rows' ways, so numbering that keeps neighbours' ways alike is cheap.  8 sequences of 2048 candidates and 32000
// bfloat16 entries, as a chain 600 us, as a tree that is a chain 820, random parents 620, but two chains whose nodes come in turn 10450.
#ifndef FSD_CSRC_CONDITION_H_
#define FSD_CSRC_CONDITION_H_

#include "operators_common.h"

namespace {

constexpr unsigned kInPrompt = 1u << 31;   // of a token's word; the low bits count its generated occurrences
constexpr unsigned kElsewhere = 1u << 30;  // the token has a bias: the low bits say where its word and its bias stand
constexpr int kConditionSlots = 4;         // 16-byte slots of a row that a thread takes, at most

struct ConditionParams {
    const char* logits;
    char* out;
    const int32_t* tokens;    // [B, N]
    const int32_t* parent;    // [B, N], trees
    fsd_conditions c;
    int B, N, rows, V;
    int target;               // rows are contexts 0 .. N (target rows); 0: row r is the context of node r's parent
    int slice, nslices, rows_per_wg, ngroups;
    int side;                 // biased tokens a slice can have
    long nwork;
};

// logit after penalties and bias; inv is 1 / r (a product costs one rounding of 2^-24 more than the quotient, and 20 instructions less)
__device__ __forceinline__ float conditioned(float z, unsigned word, float r, float inv, float f, float p, bool biased, float bias) {
    if (word != 0) z *= z > 0.0f ? inv : r;
    const unsigned count = word & ~kInPrompt;
    if (count != 0) {
        z = z - f * static_cast<float>(count);
        z = z - p;
    }
    return biased ? z + bias : z;
}

// Wavefronts a SIMD: bfloat16 has LDS for 4 workgroups a compute unit; binary32 tables are half as large, and 6 of them take 48 sequences of
// 17 rows of 128259 entries 203 us where 5 take 242 (1536 workgroups: one round in place of 1.2).  That leaves binary32 80 registers, two short: they are
// spilled before the loop over rows and read again once a row.
template <bool BF16, bool TREE, bool STREAM>
__global__ __launch_bounds__(kWG, BF16 ? 4 : 6) void condition_rows(ConditionParams P) {
    constexpr int VE = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;
    extern __shared__ unsigned lds[];
    const long work = spread_over_xcds(blockIdx.x, P.nwork);
    if (work < 0) return;
    const int group = static_cast<int>(work % P.ngroups);
    const int si = static_cast<int>(work / P.ngroups % P.nslices), b = static_cast<int>(work / P.ngroups / P.nslices);
    const int v0 = si * P.slice, n = min(P.slice, P.V - v0);
    const int r0 = group * P.rows_per_wg, r1 = min(P.rows, r0 + P.rows_per_wg);
    const int tid = threadIdx.x, nb = P.c.bias_count;
    unsigned* table = lds;                                   // [slice] a word for every token
    unsigned* touched = table + P.slice;                     // [slice / 32] its word or its bias says something
    unsigned* side = touched + P.slice / 32;                 // [side][2] of biased tokens: word, 1 + index of the last bias
    unsigned* taken = side + 2 * P.side;                     // how many of them there are
    short* up = reinterpret_cast<short*>(taken + 1);         // trees: [N] parent
    short* here = up + (TREE ? P.N : 0);                     // trees: [N] token - v0, or -1
    short* near = here + (TREE ? P.N : 0);                   // trees: [N] the last node on the way to a node, itself included, with a token here, or -1

    for (int i = tid; i < P.slice + P.slice / 32 + 2 * P.side + 1; i += kWG) lds[i] = 0;
    const int32_t* tokens = P.tokens + static_cast<size_t>(b) * P.N;
    if constexpr (TREE) {
        const int32_t* parent = P.parent + static_cast<size_t>(b) * P.N;
        for (int j = tid; j < P.N; j += kWG) {
            const int p = parent[j];
            up[j] = static_cast<short>(p < -1 || p >= j ? -1 : p);
            const unsigned at = static_cast<unsigned>(tokens[j]) - static_cast<unsigned>(v0);
            here[j] = static_cast<short>(at < static_cast<unsigned>(n) ? at : 0xFFFFu);
        }
    }
    __syncthreads();
    auto touch = [&](unsigned at) { atomicOr(&touched[at >> 5], 1u << (at & 31)); };
    auto place = [&](int t, unsigned& at) {                  // whether a token is of this slice, and where
        at = static_cast<unsigned>(t) - static_cast<unsigned>(v0);
        return at < static_cast<unsigned>(n);
    };
    if (nb > 0) {
        // biased tokens move out of the table: one of those that name a token finds it a place, then the last one is noted there
        const int32_t* list = P.c.bias_tokens + static_cast<size_t>(b) * nb;
        unsigned at;
        for (int i = tid; i < nb; i += kWG)
            if (place(list[i], at) && atomicCAS(&table[at], 0u, kElsewhere) == 0u) {
                atomicOr(&table[at], atomicAdd(taken, 1u));
                touch(at);
            }
        __syncthreads();
        for (int i = tid; i < nb; i += kWG)
            if (place(list[i], at)) atomicMax(&side[2 * (table[at] & ~kElsewhere) + 1], static_cast<unsigned>(i) + 1u);
    }
    auto word_of = [&](unsigned at) -> unsigned* {
        const unsigned w = nb > 0 ? table[at] : 0u;
        return (w & kElsewhere) != 0 ? &side[2 * (w & ~kElsewhere)] : &table[at];
    };
    auto say = [&](unsigned at, unsigned add) {
        atomicAdd(word_of(at), add);
        touch(at);
    };
    if (P.c.history) {
        const int32_t* h = P.c.history + static_cast<size_t>(b) * P.c.history_stride;
        int len = P.c.history_len ? P.c.history_len[b] : P.c.history_stride;
        len = max(0, min(len, P.c.history_stride));
        const int prompt = P.c.prompt_len ? P.c.prompt_len[b] : 0;
        auto one = [&](int i, int t) {
            unsigned at;
            if (!place(t, at)) return;
            if (i < prompt) {
                atomicOr(word_of(at), kInPrompt);
                touch(at);
            } else {
                say(at, 1u);
            }
        };
        // (four requests of 16 bytes a thread in flight: the histories of a sequence's slices come from one L2, what counts is latency)
        constexpr int kOnce = 4 * kWG, kAhead = 4;
        auto four = [&](int e, const uint4& x) { one(e, x.x); one(e + 1, x.y); one(e + 2, x.z); one(e + 3, x.w); };
        int i = 0;
        for (; i + kAhead * kOnce <= len; i += kAhead * kOnce) {
            uint4 x[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) x[k] = load_any16(reinterpret_cast<const char*>(h + i + k * kOnce + 4 * tid));
#pragma unroll
            for (int k = 0; k < kAhead; ++k) four(i + k * kOnce + 4 * tid, x[k]);
        }
        for (; i + kOnce <= len; i += kOnce) four(i + 4 * tid, load_any16(reinterpret_cast<const char*>(h + i + 4 * tid)));
        for (i += tid; i < len; i += kWG) one(i, h[i]);
    }
    if constexpr (TREE) {
        for (int j0 = 0; j0 < P.N; j0 += kWG) {              // (as many nodes at a time as there are threads: a walk ends where those before know)
            if (j0 > 0) __syncthreads();
            if (j0 + tid < P.N) {
                int j = j0 + tid;
                while (j >= j0 && here[j] < 0) j = up[j];
                near[j0 + tid] = static_cast<short>(j < 0 || j >= j0 ? j : near[j]);
            }
        }
    } else {
        for (int j = tid; j < min(r0, P.N); j += kWG) {      // the candidates on the way to the first row
            unsigned at;
            if (place(tokens[j], at)) say(at, 1u);
        }
    }
    __syncthreads();
    const float rep = P.c.repetition ? P.c.repetition[b] : 1.0f, inv_rep = 1.0f / rep;
    const float freq = P.c.frequency ? P.c.frequency[b] : 0.0f, pres = P.c.presence ? P.c.presence[b] : 0.0f;
    const float* bias = P.c.bias_values + static_cast<size_t>(b) * nb;
    const int words = (P.V + 31) / 32;

    // From the way that the table holds (its last node with a token here) to another one: of the two ways' ends the one with the larger number is not on
    // the other way, as a parent's is smaller.  What is taken out leaves its bit (a zero word says nothing).
    auto move = [&](int from, int to) {
        while (from != to) {
            const bool out = from > to;
            const int end = out ? from : to, above = up[end], next_end = above < 0 ? -1 : near[above];
            say(static_cast<unsigned>(here[end]), out ? 0xFFFFFFFFu : 1u);   // (-1 or 1)
            from = out ? next_end : from;
            to = out ? to : next_end;
        }
    };
    auto adjusted = [&](float z, int at) {
        unsigned w = table[at], last = 0;
        if ((w & kElsewhere) != 0) {
            const unsigned* s = &side[2 * (w & ~kElsewhere)];
            w = s[0];
            last = s[1];
        }
        return conditioned(z, w, rep, inv_rep, freq, pres, last != 0, last != 0 ? bias[last - 1] : 0.0f);
    };
    auto meet = []() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };   // (of LDS: what is requested stays so)
    // A thread's slots of a row are requested while it works on the row before, their masks one row earlier still: a slot
    // without an allowed entry is not read.
    constexpr unsigned kAll = (1u << VE) - 1u;
    auto row_at = [&](int r) { return ((static_cast<size_t>(b) * P.rows + r) * P.V + v0) * ES; };
    auto masks = [&](int r, unsigned (&ok)[kConditionSlots]) {
        if (P.c.allowed && r < r1) {
            const int context = P.c.allowed_contexts == 1 ? 0 : TREE && !P.target ? up[r] + 1 : r;
            const uint32_t* mask = P.c.allowed + (static_cast<size_t>(b) * P.c.allowed_contexts + context) * words + v0 / 32;
            int id = tid;
            if constexpr (TREE && !BF16) asm volatile("" : "+v"(id));   // (the places worked out anew for every row: kept, they would take registers that are spilled)
#pragma unroll
            for (int k = 0; k < kConditionSlots; ++k) {
                const int at = (id + k * kWG) * VE;
                ok[k] = at < n ? mask[at >> 5] : 0u;
            }
        } else {
#pragma unroll
            for (int k = 0; k < kConditionSlots; ++k) ok[k] = ~0u;
        }
    };
    auto mask_of = [&](unsigned word, int k) { return word >> ((tid + k * kWG) * VE & 31) & kAll; };
    auto request = [&](int r, const unsigned (&ok)[kConditionSlots], uint4 (&w)[kConditionSlots]) {
        if (r >= r1) return;
        const char* in = P.logits + row_at(r);
#pragma unroll
        for (int k = 0; k < kConditionSlots; ++k) {
            const int at = (tid + k * kWG) * VE;
            if (at + VE <= n && mask_of(ok[k], k) != 0) w[k] = load_any16<STREAM>(in + static_cast<size_t>(at) * ES);
        }
    };
    unsigned ok[kConditionSlots], ok1[kConditionSlots], ok2[kConditionSlots];
    uint4 now[kConditionSlots], next[kConditionSlots];
    masks(r0, ok);
    masks(r0 + 1, ok1);
    request(r0, ok, now);
    int held = -1;                                            // trees: the way that the table holds
    for (int r = r0; r < r1; ++r) {
        request(r + 1, ok1, next);
        masks(r + 2, ok2);
        if constexpr (TREE) {
            const int last = P.target ? r - 1 : __builtin_amdgcn_readfirstlane(up[r]);   // (the same for every thread)
            const int to = last < 0 ? -1 : __builtin_amdgcn_readfirstlane(near[last]);
            if (to != held) {
                meet();
                if (tid == 0) move(held, to);
                meet();
                held = to;
            }
        } else if (r > r0) {                                  // (uniform: every thread reads the same token)
            unsigned at;
            if (place(tokens[r - 1], at)) {
                meet();
                if (tid == 0) say(at, 1u);
                meet();
            }
        }
        const char* in = P.logits + row_at(r);
        char* out = P.out + row_at(r);
#pragma unroll
        for (int k = 0; k < kConditionSlots; ++k) {
            const int at = (tid + k * kWG) * VE;
            if (at >= n) continue;
            const unsigned let = mask_of(ok[k], k);
            if (at + VE <= n) {
                uint4 w = neg_inf_slot<BF16>();
                if (let != 0) {
                    // one touched entry of every lane's slot at a time: there are few, and each costs a wavefront the same
                    unsigned a = now[k].x, c = now[k].y, d = now[k].z, f = now[k].w;
                    for (unsigned t = (touched[at >> 5] >> (at & 31)) & let; t != 0; t &= t - 1) {
                        const int e = __builtin_ctz(t), i = BF16 ? e >> 1 : e, up_by = BF16 ? 16 * (e & 1) : 0;
                        const unsigned of = (BF16 ? 0xFFFFu : ~0u) << up_by, old = i < 2 ? (i == 0 ? a : c) : (i == 2 ? d : f);
                        const float z = adjusted(__uint_as_float(BF16 ? (old >> up_by) << 16 : old), at + e);
                        const unsigned put = (old & ~of) | (BF16 ? bf16_bits(z) << up_by : __float_as_uint(z));
                        a = i == 0 ? put : a;
                        c = i == 1 ? put : c;
                        d = i == 2 ? put : d;
                        f = i == 3 ? put : f;
                    }
                    w = make_uint4(a, c, d, f);
                    if (let != kAll) w = masked_slot<BF16>(w, let);
                }
                store_any16<STREAM>(out + static_cast<size_t>(at) * ES, w);
            } else {
                for (int e = 0; at + e < n; ++e) {            // the end of a ragged row
                    float z = load_logit<BF16>(in, at + e);
                    if (!(let >> e & 1u)) {
                        store_logit<BF16>(out, at + e, -__builtin_inff());
                    } else if ((touched[at >> 5] >> ((at + e) & 31)) & 1u) {
                        z = adjusted(z, at + e);
                        store_logit<BF16>(out, at + e, z);
                    } else {
                        copy_logit<BF16>(out, in, at + e);
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kConditionSlots; ++k) {
            now[k] = next[k];
            ok[k] = ok1[k];
            ok1[k] = ok2[k];
        }
    }
}

}  // namespace

#endif  // FSD_CSRC_CONDITION_H_
