// Penalties for repeated tokens, biases and grammar masks on the rows of a verify call (fsd_condition_*).
// Part of libfsd (gfx950); included by operators.hip, which holds the host side and the C ABI.
//
//   z1 = seen ? (z > 0 ? z / r : z r) : z;  z2 = z1 - f count - (count ? p : 0);  z3 = z2 + bias;  -inf where not allowed
//
// A workgroup takes a run of `slice` vocabulary entries and some rows of one sequence.  It goes over the sequence's
// history once and counts in LDS the tokens that fall into its slice (integer atomics: the order does not matter), then
// streams its rows: one bit an entry tells whether the table says anything about it, so that nearly every 16-byte
// slot is copied (or masked) as it is.  What a row's own way adds is put into the table when the row needs it: along a chain
// the contexts contain one another and each row adds one candidate; in a tree the few rows whose way has a token in
// the slice add it and take it away again.  No row keeps another one waiting otherwise: there is no barrier between them.
#ifndef FSD_CSRC_CONDITION_H_
#define FSD_CSRC_CONDITION_H_

#include "operators_common.h"

namespace {

constexpr unsigned kInPrompt = 1u << 31;   // of a table word; the rest counts generated occurrences

struct ConditionParams {
    const char* logits;
    char* out;
    const int32_t* tokens;    // [B, N]
    const int32_t* parent;    // [B, N], trees
    fsd_conditions c;
    int B, N, rows, V;
    int target;               // rows are contexts 0 .. N (target rows); 0: row r is the context of node r's parent
    int slice, nslices, rows_per_wg, ngroups;
    long nwork;
};

// logit after penalties and bias
__device__ __forceinline__ float conditioned(float z, unsigned word, float r, float f, float p, bool biased, float bias) {
    if (word != 0) z = z > 0.0f ? __fdiv_rn(z, r) : z * r;
    const unsigned count = word & ~kInPrompt;
    if (count != 0) {
        z = z - f * static_cast<float>(count);
        z = z - p;
    }
    return biased ? z + bias : z;
}

template <bool BF16, bool TREE>
__global__ __launch_bounds__(kWG) void condition_rows(ConditionParams P) {
    constexpr int VE = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;
    extern __shared__ unsigned lds[];
    const long work = spread_over_xcds(blockIdx.x, P.nwork);
    if (work < 0) return;
    const int group = static_cast<int>(work % P.ngroups);
    const int si = static_cast<int>(work / P.ngroups % P.nslices), b = static_cast<int>(work / P.ngroups / P.nslices);
    const int v0 = si * P.slice, n = min(P.slice, P.V - v0);
    const int r0 = group * P.rows_per_wg, r1 = min(P.rows, r0 + P.rows_per_wg);
    const int tid = threadIdx.x, nb = P.c.bias_count;
    unsigned* table = lds;                                   // [slice]
    unsigned* touched = table + P.slice;                     // [slice / 32] the table or the biases say something
    unsigned* which = touched + P.slice / 32;                // [slice] with biases: 1 + index of the last of this token
    unsigned* wayed = which + (nb ? P.slice : 0);            // trees: [rows_per_wg / 32 + 1] the row's way has a token here
    short* up = reinterpret_cast<short*>(wayed + (TREE ? P.rows_per_wg / 32 + 1 : 0));   // trees: [N] parent
    short* here = up + (TREE ? P.N : 0);                     // trees: [N] token - v0, or -1

    for (int i = tid; i < P.slice + P.slice / 32 + (nb ? P.slice : 0) + (TREE ? P.rows_per_wg / 32 + 1 : 0); i += kWG) lds[i] = 0;
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
    auto say = [&](unsigned at, unsigned add) {
        atomicAdd(&table[at], add);
        atomicOr(&touched[at >> 5], 1u << (at & 31));
    };
    if (P.c.history) {
        const int32_t* h = P.c.history + static_cast<size_t>(b) * P.c.history_stride;
        int len = P.c.history_len ? P.c.history_len[b] : P.c.history_stride;
        len = max(0, min(len, P.c.history_stride));
        int prompt = P.c.prompt_len ? P.c.prompt_len[b] : 0;
        auto one = [&](int i, int t) {
            const unsigned at = static_cast<unsigned>(t) - static_cast<unsigned>(v0);
            if (at < static_cast<unsigned>(n)) {
                if (i < prompt) {
                    atomicOr(&table[at], kInPrompt);
                    atomicOr(&touched[at >> 5], 1u << (at & 31));
                } else {
                    say(at, 1u);
                }
            }
        };
        int i = tid;
        for (; i + 3 * kWG < len; i += 4 * kWG) {            // four requests in flight
            const int t0 = h[i], t1 = h[i + kWG], t2 = h[i + 2 * kWG], t3 = h[i + 3 * kWG];
            one(i, t0); one(i + kWG, t1); one(i + 2 * kWG, t2); one(i + 3 * kWG, t3);
        }
        for (; i < len; i += kWG) one(i, h[i]);
    }
    for (int i = tid; i < nb; i += kWG) {
        const unsigned at = static_cast<unsigned>(P.c.bias_tokens[static_cast<size_t>(b) * nb + i]) - static_cast<unsigned>(v0);
        if (at < static_cast<unsigned>(n)) {
            atomicMax(&which[at], static_cast<unsigned>(i) + 1u);
            atomicOr(&touched[at >> 5], 1u << (at & 31));
        }
    }
    if constexpr (TREE) {
        for (int r = r0 + tid; r < r1; r += kWG) {
            bool any = false;
            for (int j = P.target ? r - 1 : up[r]; j >= 0 && !any; j = up[j]) any = here[j] >= 0;
            if (any) atomicOr(&wayed[(r - r0) >> 5], 1u << ((r - r0) & 31));
        }
    } else {
        for (int j = tid; j < min(r0, P.N); j += kWG) {      // the candidates on the way to the first row
            const unsigned at = static_cast<unsigned>(tokens[j]) - static_cast<unsigned>(v0);
            if (at < static_cast<unsigned>(n)) say(at, 1u);
        }
    }
    __syncthreads();
    const float rep = P.c.repetition ? P.c.repetition[b] : 1.0f;
    const float freq = P.c.frequency ? P.c.frequency[b] : 0.0f, pres = P.c.presence ? P.c.presence[b] : 0.0f;
    const float* bias = P.c.bias_values + static_cast<size_t>(b) * nb;
    const int words = (P.V + 31) / 32;

    // a node's token is taken into the table, or out of it (the bit stays: a zero word says nothing)
    auto along = [&](int r, unsigned add) {
        if (tid == 0) {
            for (int j = P.target ? r - 1 : up[r]; j >= 0; j = up[j])
                if (here[j] >= 0) say(static_cast<unsigned>(here[j]), add);
        }
    };
    auto adjusted = [&](float z, int at) {
        const unsigned w = nb ? which[at] : 0u;
        return conditioned(z, table[at], rep, freq, pres, w != 0, w != 0 ? bias[w - 1] : 0.0f);
    };
    for (int r = r0; r < r1; ++r) {
        bool mine = false;
        if constexpr (TREE) {
            mine = (wayed[(r - r0) >> 5] >> ((r - r0) & 31)) & 1u;
            if (mine) {
                __syncthreads();
                along(r, 1u);
                __syncthreads();
            }
        } else if (r > r0) {                                  // (uniform: every thread reads the same token)
            const unsigned at = static_cast<unsigned>(tokens[r - 1]) - static_cast<unsigned>(v0);
            if (at < static_cast<unsigned>(n)) {
                __syncthreads();
                if (tid == 0) say(at, 1u);
                __syncthreads();
            }
        }
        const int context = TREE && !P.target ? up[r] + 1 : r;
        const size_t row = (static_cast<size_t>(b) * P.rows + r) * P.V + v0;
        const char* in = P.logits + row * ES;
        char* out = P.out + row * ES;
        const uint32_t* mask = nullptr;
        if (P.c.allowed)
            mask = P.c.allowed + (static_cast<size_t>(b) * P.c.allowed_contexts + (P.c.allowed_contexts > 1 ? context : 0)) * words + v0 / 32;
        constexpr unsigned kAll = (1u << VE) - 1u;
        for (int at = tid * VE; at < n; at += kWG * VE) {
            unsigned ok = mask ? (mask[at >> 5] >> (at & 31)) & kAll : kAll;
            if (at + VE <= n) {
                uint4 w = neg_inf_slot<BF16>();
                if (ok != 0) {                                // (a slot without an allowed entry is not read)
                    w = load_any16(in + static_cast<size_t>(at) * ES);
                    unsigned t = (touched[at >> 5] >> (at & 31)) & ok;
                    if ((t | (ok ^ kAll)) != 0) {
                        float z[VE];
                        unpack_slot<BF16>(w, z);
                        const uint4 raw = w;
#pragma unroll
                        for (int e = 0; e < VE; ++e)
                            if (t >> e & 1u) z[e] = adjusted(z[e], at + e);
                        w = repack_slot<BF16>(raw, z, t, ok);
                    }
                }
                store_any16(out + static_cast<size_t>(at) * ES, w);
            } else {
                for (int e = 0; at + e < n; ++e) {            // the end of a ragged row
                    float z = load_logit<BF16>(in, at + e);
                    if ((touched[at >> 5] >> ((at + e) & 31)) & 1u) {
                        z = adjusted(z, at + e);
                        if (ok >> e & 1u) store_logit<BF16>(out, at + e, z);
                    } else if (ok >> e & 1u) {
                        copy_logit<BF16>(out, in, at + e);
                    }
                    if (!(ok >> e & 1u)) store_logit<BF16>(out, at + e, -__builtin_inff());
                }
            }
        }
        if (TREE && mine) {
            __syncthreads();
            along(r, 0xFFFFFFFFu);                            // (adds -1)
            __syncthreads();
        }
    }
}

}  // namespace

#endif  // FSD_CSRC_CONDITION_H_
