// Pages of the 8-bit paged cache: which sequence names which blocks (fsd_cache_fork), pages copied (fsd_cache_copy) and moved to
// the front (fsd_cache_compact).  Part of libfsd (gfx950).
//
// Who gets which block has to come out the same on every run, so nothing hangs on the order in which workgroups come: counts and minima by
// integer atomics, places of blocks and sequences by sums over what lies in front of them, one kernel behind the other.
//
// What bounds it: where many pages move, their bytes (1.21 GB read and written by pages_copy in 240 us, 5.05 TB/s; a large copy reaches 4.9 here); where few do, the
// launches that follow one another, 3 to 5 us each, and in fork_mark the atomics.  256 sequences of some 40000 tokens in one layer: fork_clear 3.0, fork_mark 9.9,
// fork_count 4.2, fork_list 5.9, fork_apply 4.4 us with the few copies in it; 128 beams in 16 layers, 140 MB of begun pages: fork_small 9.4, fork_move 22 us.
// Compacting a pool of 1200 blocks, 540 of them in use, 8 layers: compact_small 9, compact_move 136 us for 623 MB (4.6 TB/s); one of 6000 blocks, one layer, 390 MB:
// compact_count 4.9, compact_list 6.2, compact_apply 83.
#ifndef FSD_CSRC_CACHE_PAGES_H_
#define FSD_CSRC_CACHE_PAGES_H_

#include "operators_common.h"

namespace {

constexpr int kPagesChunk = 1024;   // blocks, or places, that a workgroup goes over at once
constexpr int kNobody = 0x7FFFFFFF;
// What one workgroup does by itself, its blocks' counts in LDS: the launches behind one another take 14 to 17 us on the device and 10 more on the host than
// one.  One sequence's 4 beams: 5.2 us; 128 beams of 11 places: 9.4; at the limits here as long as the several kernels.
constexpr int kSmallWG = 1024, kSmallBlocks = 4096, kSmallPlaces = 8192;

// the sum of all threads' v, and of those below
template <int T = kWG>
__device__ __forceinline__ int scan_wg(int v, int tid, int* lds, int* total) {
    int upto = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int other = __shfl_up(upto, o, 64);
        if (tid % 64 >= o) upto += other;
    }
    __syncthreads();
    if (tid % 64 == 63) lds[tid / 64] = upto;
    __syncthreads();
    int before = upto - v, all = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) {
        before += w < tid / 64 ? lds[w] : 0;
        all += lds[w];
    }
    *total = all;
    return before;
}
__device__ __forceinline__ int sum_wg(const int* from, long n, int tid, int* lds) {
    int mine = 0, all;
    for (long i = tid; i < n; i += kWG) mine += from[i];
    scan_wg(mine, tid, lds, &all);
    return all;
}

// ------------------------------------------------------------------------------------------ bytes of pages

struct PagesPair {                  // two caches of one geometry (or one cache twice)
    const char *k_from, *v_from;
    char *k_to, *v_to;
    const float *ks_from, *vs_from;
    float *ks_to, *vs_to;
    long blocks_from, blocks_to;
    int layers, heads, head_bytes;  // head_bytes: of a block's codes of one head
};
// Of block `from` in the one cache to block `to` in the other: a layer's head, its first `groups` groups of 16 tokens.  Keys and values have them at the front of
// a head's codes alike.
// (A workgroup has both of a head's runs of 4 to 16 KB on their way at once.  Requests and stores past the caches: 3 % faster at 1.2 GB, and slower where the
// pages lie in them.)
__device__ __forceinline__ void move_head(const PagesPair& P, long from, long to, int layer, int head, int groups, int tid) {
    const long src = (static_cast<long>(layer) * P.blocks_from + from) * P.heads + head, dst = (static_cast<long>(layer) * P.blocks_to + to) * P.heads + head;
    const u32x4* k = reinterpret_cast<const u32x4*>(P.k_from + src * P.head_bytes);
    const u32x4* v = reinterpret_cast<const u32x4*>(P.v_from + src * P.head_bytes);
    u32x4* ko = reinterpret_cast<u32x4*>(P.k_to + dst * P.head_bytes);
    u32x4* vo = reinterpret_cast<u32x4*>(P.v_to + dst * P.head_bytes);
    const int slots = P.head_bytes / 64 * groups;            // of 16 bytes
    if (tid == 0) P.ks_to[dst] = P.ks_from[src];
    if (tid == 64) P.vs_to[dst] = P.vs_from[src];
    for (int i = tid; i < slots; i += kWG) {
        const u32x4 a = k[i], b = v[i];
        ko[i] = a;
        vo[i] = b;
    }
}

struct CopyParams {
    PagesPair pair;
    const int *from, *to, *tokens;
    int* status;
    int n;
    long units;                     // n * layers * heads
};
__global__ void __launch_bounds__(kWG) pages_copy(const CopyParams P) {
    const int tid = threadIdx.x;
    for (long u = blockIdx.x; u < P.units; u += gridDim.x) {
        const long kl = u / P.pair.heads;
        const int head = static_cast<int>(u - kl * P.pair.heads), k = static_cast<int>(kl / P.pair.layers), layer = static_cast<int>(kl - static_cast<long>(k) * P.pair.layers);
        const int from = P.from[k], to = P.to[k], tokens = P.tokens ? P.tokens[k] : kBlock;
        const bool none = from == -1 || to == -1;
        const bool good = from >= 0 && from < P.pair.blocks_from && to >= 0 && to < P.pair.blocks_to && tokens >= 0 && tokens <= kBlock;
        if (good) move_head(P.pair, from, to, layer, head, (tokens + 15) / 16, tid);
        if (P.status && layer == 0 && head == 0 && tid == 0) P.status[k] = good || none ? 0 : FSD_ROW_BAD_CACHE;
    }
}

// ------------------------------------------------------------------------------------------ forking

struct ForkParams {
    const int *table, *lens, *parent, *keep, *room, *refs;
    int B, M, P, n;                 // old sequences, places of a table's row, blocks, new sequences
    int *table_out, *len_out, *refs_out, *free_out, *status;
    unsigned long* counts;          // [P] of a block: places of the old tables, and in the upper half whole places of the new ones
    int* claim;                     // [P] the first other place that wants to keep it
    int* free_list;                 // [P]
    int* free_count;                // [chunks of P]
    int4* seq;                      // [n] tokens, full places, needed places, status
    int* fresh;                     // [n] blocks that a sequence needs
    int* copies;                    // [n] whether the first of them takes over what a begun block holds
    int2* at;                       // [n] fresh and copies of the sequences in front of it
    int* copy_seq;                  // [n] the sequences with a copy
    int* totals;                    // free blocks, fresh ones, copies
    PagesPair pair;
};
// claim, after fork_list: the place that keeps the block; kNobody where several or others hold it; -1 - (its number among the free ones)

__global__ void __launch_bounds__(kWG) fork_clear(const ForkParams P) {
    for (long i = blockIdx.x * static_cast<long>(kWG) + threadIdx.x; i < P.P; i += static_cast<long>(gridDim.x) * kWG) {
        P.counts[i] = 0;
        P.claim[i] = kNobody;
    }
}

// Workgroups 0 .. B-1: an old sequence's places, and those of the new sequence of its number if that goes on from it (one atomic for both: a serving step's
// sequences nearly all do); the others: a new sequence's places.
__global__ void __launch_bounds__(kWG) fork_mark(const ForkParams P) {
    const int tid = threadIdx.x, M = P.M;
    const bool is_old = blockIdx.x < static_cast<unsigned>(P.B);
    const int i = is_old ? static_cast<int>(blockIdx.x) : static_cast<int>(blockIdx.x) - P.B;
    const int p = i < P.n ? P.parent[i] : -1;
    const bool goes_on = p == i && i < P.B, is_new = is_old ? goes_on : !goes_on;
    const bool some = is_new && p >= 0 && p < P.B;
    int full = 0, need = 0;
    if (is_new) {
        __shared__ int wrong_place;
        int status = p < -1 || p >= P.B ? FSD_ROW_BAD_PARENT : 0;
        const long most = static_cast<long>(M) * kBlock;
        const int held = some ? P.lens[p] : 0, room = P.room ? P.room[i] : 0;
        int have = P.keep && some ? P.keep[i] : held;
        if (held < 0 || held > most || have < 0 || have > held || room < 0 || room > most - have) status |= FSD_ROW_BAD_CACHE;
        if (tid == 0) wrong_place = 0;
        __syncthreads();
        if (status == 0) {
            const int* row = P.table + static_cast<size_t>(some ? p : 0) * M;
            for (int j = tid; j < (have + kBlock - 1) / kBlock; j += kWG) {
                const int e = row[j];
                if (e < 0 || e >= P.P) wrong_place = 1;
            }
        }
        __syncthreads();
        if (wrong_place) status |= FSD_ROW_BAD_CACHE;
        if (status != 0) have = 0;
        full = have / kBlock;
        need = status != 0 ? 0 : static_cast<int>((static_cast<long>(have) + room + kBlock - 1) / kBlock);
        if (tid == 0) P.seq[i] = make_int4(have, full, need, status);
    }
    if (!is_old && !some) return;
    const int* row = P.table + static_cast<size_t>(is_old ? i : p) * M;
    for (int j = tid; j < (is_old ? M : need); j += kWG) {
        const int e = row[j];
        if (e < 0 || e >= P.P) continue;
        const unsigned long more = (is_old ? 1ul : 0ul) + (j < full ? 1ul << 32 : 0ul);
        if (more != 0) atomicAdd(&P.counts[e], more);
        if (j >= full && j < need) atomicMin(&P.claim[e], i * M + j);
    }
}

// of a block: places that are none of the old sequences'; whole places of the new ones
__device__ __forceinline__ int others(const ForkParams& P, int e) {
    const int o = P.refs[e] - static_cast<int>(static_cast<unsigned>(P.counts[e]));
    return o > 0 ? o : 0;
}
__device__ __forceinline__ int shared(const ForkParams& P, int e) { return static_cast<int>(P.counts[e] >> 32); }

// workgroups 0 .. chunks-1: how many of a chunk's blocks are free; the others: how many blocks new sequences need, a wavefront each
__global__ void __launch_bounds__(kWG) fork_count(const ForkParams P, int chunks) {
    __shared__ int lds[kWG / 64];
    const int tid = threadIdx.x;
    if (static_cast<int>(blockIdx.x) < chunks) {
        int mine = 0, all;
        for (int k = 0; k < kPagesChunk / kWG; ++k) {
            const long e = blockIdx.x * static_cast<long>(kPagesChunk) + k * kWG + tid;
            if (e < P.P) mine += others(P, static_cast<int>(e)) == 0 && shared(P, static_cast<int>(e)) == 0 && P.claim[e] == kNobody;
        }
        scan_wg(mine, tid, lds, &all);
        if (tid == 0) P.free_count[blockIdx.x] = all;
        return;
    }
    const int i = (static_cast<int>(blockIdx.x) - chunks) * (kWG / 64) + tid / 64, lane = tid % 64;
    if (i >= P.n) return;
    const int4 q = P.seq[i];
    const int p = P.parent[i];
    const bool some = p >= 0 && p < P.B;
    const int* row = P.table + static_cast<size_t>(some ? p : 0) * P.M;
    int fresh = 0, copy = 0;
    for (int j0 = q.y; j0 < q.z; j0 += 64) {
        const int j = j0 + lane;
        bool is = false;
        if (j < q.z) {
            const int e = some ? row[j] : -1;
            is = !(e >= 0 && e < P.P && P.claim[e] == i * P.M + j && shared(P, e) == 0 && others(P, e) == 0);
        }
        const unsigned long which = __ballot(is);
        if (j0 == q.y) copy = (which & 1) && q.x % kBlock != 0;
        fresh += __popcll(which);
    }
    if (lane == 0) {
        P.fresh[i] = fresh;
        P.copies[i] = copy;
    }
}

// workgroups 0 .. chunks-1: a chunk's free blocks into the list; the others: 256 new sequences each
__global__ void __launch_bounds__(kWG) fork_list(const ForkParams P, int chunks) {
    __shared__ int lds[kWG / 64];
    const int tid = threadIdx.x;
    if (static_cast<int>(blockIdx.x) < chunks) {
        int number = sum_wg(P.free_count, blockIdx.x, tid, lds);
        for (int k = 0; k < kPagesChunk / kWG; ++k) {
            const long e = blockIdx.x * static_cast<long>(kPagesChunk) + k * kWG + tid;
            bool free = false, alone = false;
            if (e < P.P) {
                alone = others(P, static_cast<int>(e)) == 0 && shared(P, static_cast<int>(e)) == 0;
                free = alone && P.claim[e] == kNobody;
            }
            int all;
            const int own = number + scan_wg(free, tid, lds, &all);
            number += all;
            if (free) {
                P.free_list[own] = static_cast<int>(e);
                P.claim[e] = -1 - own;
            } else if (e < P.P && !alone) {
                P.claim[e] = kNobody;
            }
        }
        if (static_cast<int>(blockIdx.x) == chunks - 1 && tid == 0) P.totals[0] = number;
        return;
    }
    const int i0 = (static_cast<int>(blockIdx.x) - chunks) * kWG, i = i0 + tid;
    const int fresh0 = sum_wg(P.fresh, i0, tid, lds), copies0 = sum_wg(P.copies, i0, tid, lds);
    const int fresh = i < P.n ? P.fresh[i] : 0, copy = i < P.n ? P.copies[i] : 0;
    int all_fresh, all_copies;
    const int a = fresh0 + scan_wg(fresh, tid, lds, &all_fresh), c = copies0 + scan_wg(copy, tid, lds, &all_copies);
    if (i < P.n) {
        P.at[i] = make_int2(a, c);
        if (copy) P.copy_seq[c] = i;
    }
    if (i0 + kWG >= P.n && tid == 0) {
        P.totals[1] = fresh0 + all_fresh;
        P.totals[2] = copies0 + all_copies;
    }
}

// What begun blocks hold to those that take over, a layer's head at a time; this workgroup is one of `step`
__device__ __forceinline__ void move_begun(const ForkParams& P, long first, long step) {
    if (P.totals[1] > P.totals[0]) return;
    const long units = static_cast<long>(P.totals[2]) * P.pair.layers * P.pair.heads;
    for (long u = first; u < units; u += step) {
        const long kl = u / P.pair.heads;
        const int head = static_cast<int>(u - kl * P.pair.heads), k = static_cast<int>(kl / P.pair.layers), layer = static_cast<int>(kl - static_cast<long>(k) * P.pair.layers);
        const int i = P.copy_seq[k];
        const int4 q = P.seq[i];
        const int from = P.table[static_cast<size_t>(P.parent[i]) * P.M + q.y], to = P.free_list[P.at[i].x];
        move_head(P.pair, from, to, layer, head, (q.x % kBlock + 15) / 16, threadIdx.x);
    }
}

// Workgroups 0 .. chunks-1: a chunk's counts; the next n: a new sequence's row; the rest share the copies.
__global__ void __launch_bounds__(kWG) fork_apply(const ForkParams P, int chunks) {
    __shared__ int lds[kWG / 64];
    const int tid = threadIdx.x, M = P.M;
    const int total_free = P.totals[0], total_fresh = P.totals[1];
    const bool is_short = total_fresh > total_free;
    if (static_cast<int>(blockIdx.x) < chunks) {
        for (int k = 0; k < kPagesChunk / kWG; ++k) {
            const long e = blockIdx.x * static_cast<long>(kPagesChunk) + k * kWG + tid;
            if (e >= P.P) break;
            const int c = P.claim[e], refs = P.refs[e];
            const int held = others(P, static_cast<int>(e)) + shared(P, static_cast<int>(e)) + (c < 0 ? -1 - c < total_fresh : c != kNobody);
            P.refs_out[e] = is_short ? refs : held;
        }
        if (blockIdx.x == 0 && tid == 0 && P.free_out) P.free_out[0] = total_free - total_fresh;
        return;
    }
    if (static_cast<int>(blockIdx.x) < chunks + P.n) {
        const int i = static_cast<int>(blockIdx.x) - chunks;
        const int4 q = P.seq[i];
        const int p = P.parent[i];
        const bool some = p >= 0 && p < P.B;
        const int* row = P.table + static_cast<size_t>(some ? p : 0) * M;
        int* out = P.table_out + static_cast<size_t>(i) * M;
        int number = P.at[i].x;
        for (int j0 = 0; j0 < M; j0 += kWG) {
            const int j = j0 + tid;
            int e = -1;
            bool fresh = false;
            if (!is_short && j < q.z) {
                e = some ? row[j] : -1;
                if (j >= q.y) fresh = !(e >= 0 && e < P.P && P.claim[e] == i * M + j);
            }
            if (!is_short && j0 + kWG > q.y && j0 < q.z) {   // (the same for all threads)
                int all;
                const int own = number + scan_wg(fresh, tid, lds, &all);
                number += all;
                if (fresh) e = P.free_list[own];
            }
            if (j < M) out[j] = e;
        }
        if (tid == 0) {
            P.len_out[i] = is_short ? 0 : q.x;
            if (P.status) P.status[i] = q.w | (is_short ? FSD_ROW_NO_BLOCKS : 0);
        }
        return;
    }
    move_begun(P, static_cast<long>(blockIdx.x) - chunks - P.n, static_cast<long>(gridDim.x) - chunks - P.n);
}

// All of it but the copies in one workgroup, as fork_clear to fork_apply do it.  counts: places of the old tables, and in the upper half full places
// of the new ones (either at most kSmallPlaces).
__global__ void __launch_bounds__(kSmallWG) fork_small(const ForkParams P) {
    __shared__ unsigned counts[kSmallBlocks];
    __shared__ int claim[kSmallBlocks];
    __shared__ int have[kSmallWG], full[kSmallWG], need[kSmallWG], from[kSmallWG], status[kSmallWG];   // (from: the parent, -1 for none)
    __shared__ int lds[kSmallWG / 64];
    const int tid = threadIdx.x, M = P.M, n = P.n;
    for (int e = tid; e < P.P; e += kSmallWG) {
        counts[e] = 0;
        claim[e] = kNobody;
    }
    if (tid < n) {
        const int p = P.parent[tid];
        const bool some = p >= 0 && p < P.B;
        const long most = static_cast<long>(M) * kBlock;
        const int held = some ? P.lens[p] : 0, room = P.room ? P.room[tid] : 0;
        const int h = P.keep && some ? P.keep[tid] : held;
        int st = p < -1 || p >= P.B ? FSD_ROW_BAD_PARENT : 0;
        if (held < 0 || held > most || h < 0 || h > held || room < 0 || room > most - h) st |= FSD_ROW_BAD_CACHE;
        from[tid] = some ? p : -1;
        have[tid] = st == 0 ? h : 0;
        full[tid] = st == 0 ? h / kBlock : 0;
        need[tid] = st == 0 ? static_cast<int>((static_cast<long>(h) + room + kBlock - 1) / kBlock) : 0;
        status[tid] = st;
    }
    __syncthreads();
    for (long k = tid; k < static_cast<long>(P.B) * M; k += kSmallWG) {
        const int e = P.table[k];
        if (e >= 0 && e < P.P) atomicAdd(&counts[e], 1u);
    }
    // from here on a thread a place of the new sequences, in order
    const int places = n * M;
    auto old_entry = [&](int i, int j) { return P.table[static_cast<size_t>(from[i]) * M + j]; };
    for (int k = tid; k < places; k += kSmallWG) {
        const int i = k / M, j = k - i * M;
        if (j * kBlock < have[i]) {
            const int e = old_entry(i, j);
            if (e < 0 || e >= P.P) status[i] = FSD_ROW_BAD_CACHE;   // (it was 0: it has tokens)
        }
    }
    __syncthreads();
    if (tid < n && status[tid] != 0) have[tid] = full[tid] = need[tid] = 0;
    __syncthreads();
    for (int k = tid; k < places; k += kSmallWG) {
        const int i = k / M, j = k - i * M;
        if (j < need[i] && from[i] >= 0) {
            const int e = old_entry(i, j);
            if (j < full[i]) atomicAdd(&counts[e], 0x10000u);
            else if (e >= 0 && e < P.P) atomicMin(&claim[e], k);
        }
    }
    __syncthreads();
    // the free ones in order, and how many places of others and of whole blocks name a block
    int total_free = 0;
    for (int e0 = 0; e0 < P.P; e0 += kSmallWG) {
        const int e = e0 + tid;
        bool free = false;
        if (e < P.P) {
            const unsigned c = counts[e];
            int other = P.refs[e] - static_cast<int>(c & 0xFFFFu);
            other = other > 0 ? other : 0;
            const bool alone = other == 0 && c < 0x10000u;
            free = alone && claim[e] == kNobody;
            if (!alone) claim[e] = kNobody;
            counts[e] = static_cast<unsigned>(other) + (c >> 16);
        }
        int all;
        const int number = total_free + scan_wg<kSmallWG>(free, tid, lds, &all);
        total_free += all;
        if (free) {
            P.free_list[number] = e;
            claim[e] = -1 - number;
        }
    }
    __threadfence_block();
    __syncthreads();
    // the new table; places that need a block are numbered, and in the upper half of the words those of them that take over what a begun block holds
    unsigned total = 0;
    for (int k0 = 0; k0 < places; k0 += kSmallWG) {
        const int k = k0 + tid, i = k < places ? k / M : 0, j = k - i * M;
        int e = -1, old = -1;
        bool fresh = false, begun = false;
        if (k < places && j < need[i]) {
            if (from[i] >= 0) old = old_entry(i, j);
            e = old;
            fresh = j >= full[i] && !(old >= 0 && old < P.P && claim[old] == k);
            begun = fresh && j * kBlock < have[i];
        }
        int all;
        const unsigned number = total + static_cast<unsigned>(scan_wg<kSmallWG>(static_cast<int>(fresh ? begun ? 0x10001u : 1u : 0u), tid, lds, &all));
        total += static_cast<unsigned>(all);
        if (fresh) e = static_cast<int>(number & 0xFFFFu) < total_free ? P.free_list[number & 0xFFFFu] : -1;
        if (begun) P.seq[number >> 16] = make_int4(old, e, (have[i] % kBlock + 15) / 16, 0);
        if (k < places) P.table_out[k] = e;
    }
    const int total_fresh = static_cast<int>(total & 0xFFFFu);
    const bool is_short = total_fresh > total_free;
    if (tid < n) {
        P.len_out[tid] = is_short ? 0 : have[tid];
        if (P.status) P.status[tid] = status[tid] | (is_short ? FSD_ROW_NO_BLOCKS : 0);
    }
    if (tid == 0) {
        P.totals[2] = is_short ? 0 : static_cast<int>(total >> 16);
        if (P.free_out) P.free_out[0] = total_free - total_fresh;
    }
    for (int e = tid; e < P.P; e += kSmallWG) {
        const int c = claim[e], refs = P.refs[e];
        P.refs_out[e] = is_short ? refs : static_cast<int>(counts[e]) + (c < 0 ? -1 - c < total_fresh : c != kNobody);
    }
    if (is_short)
        for (int k = tid; k < places; k += kSmallWG) P.table_out[k] = -1;   // (written by this thread before, too)
}
// P.seq: block, block, groups of a copy
__global__ void __launch_bounds__(kWG) fork_move(const ForkParams P) {
    const long units = static_cast<long>(P.totals[2]) * P.pair.layers * P.pair.heads;
    for (long u = blockIdx.x; u < units; u += gridDim.x) {
        const long kl = u / P.pair.heads;
        const int head = static_cast<int>(u - kl * P.pair.heads), k = static_cast<int>(kl / P.pair.layers), layer = static_cast<int>(kl - static_cast<long>(k) * P.pair.layers);
        const int4 m = P.seq[k];
        move_head(P.pair, m.x, m.y, layer, head, m.z, threadIdx.x);
    }
}

// ------------------------------------------------------------------------------------------ compacting

struct CompactParams {
    const int *table, *refs;
    int B, M, P;
    int *table_out, *refs_out, *remap, *used_out, *status;
    int* used_count;                // [chunks of P]
    int* number;                    // [P] -1: free; its own number: used and stays; P + k: the k-th that moves
    int *from, *to, *count;         // [P / 2 + 1] of a move: the block, where it goes, how many places name it
    int* totals;                    // used blocks, moves
    PagesPair pair;
};

__global__ void __launch_bounds__(kWG) compact_count(const CompactParams P) {
    __shared__ int lds[kWG / 64];
    const int tid = threadIdx.x;
    int mine = 0, all;
    for (int k = 0; k < kPagesChunk / kWG; ++k) {
        const long e = blockIdx.x * static_cast<long>(kPagesChunk) + k * kWG + tid;
        if (e < P.P) mine += P.refs[e] > 0;
    }
    scan_wg(mine, tid, lds, &all);
    if (tid == 0) P.used_count[blockIdx.x] = all;
}

// With U blocks in use, block e and u of the used ones in front of it: a free e < U is the (e - u)-th hole, a used e >= U the (u - (those in front
// of U))-th to move; there are as many of the one as of the other.
__global__ void __launch_bounds__(kWG) compact_list(const CompactParams P, int chunks) {
    __shared__ int lds[kWG / 64];
    __shared__ int part;
    const int tid = threadIdx.x;
    const int used = sum_wg(P.used_count, chunks, tid, lds);
    int in_front = sum_wg(P.used_count, blockIdx.x, tid, lds);
    // used blocks in front of block U
    const int border = used / kPagesChunk;
    int below = sum_wg(P.used_count, border, tid, lds);
    {
        int mine = 0, all;
        for (int k = 0; k < kPagesChunk / kWG; ++k) {
            const long e = border * static_cast<long>(kPagesChunk) + k * kWG + tid;
            if (e < used) mine += P.refs[e] > 0;
        }
        scan_wg(mine, tid, lds, &all);
        below += all;
    }
    if (tid == 0) part = below;
    __syncthreads();
    for (int k = 0; k < kPagesChunk / kWG; ++k) {
        const long e = blockIdx.x * static_cast<long>(kPagesChunk) + k * kWG + tid;
        const int refs = e < P.P ? P.refs[e] : 0;
        const bool is = refs > 0;
        int all;
        const int u = in_front + scan_wg(is, tid, lds, &all);
        in_front += all;
        if (e >= P.P) continue;
        int number = -1;
        if (is && e < used) {
            number = static_cast<int>(e);
        } else if (is) {
            const int m = u - part;
            P.from[m] = static_cast<int>(e);
            P.count[m] = refs;
            number = P.P + m;
        } else if (e < used) {
            P.to[e - u] = static_cast<int>(e);
        }
        P.number[e] = number;
    }
    if (blockIdx.x == 0 && tid == 0) {
        P.totals[0] = used;
        P.totals[1] = used - part;
    }
}

// Pages that move, a layer's head at a time; this workgroup is one of `step`
__device__ __forceinline__ void move_pages(const CompactParams& P, long first, long step) {
    const long units = static_cast<long>(P.totals[1]) * P.pair.layers * P.pair.heads;
    for (long u = first; u < units; u += step) {
        const long kl = u / P.pair.heads;
        const int head = static_cast<int>(u - kl * P.pair.heads), k = static_cast<int>(kl / P.pair.layers), layer = static_cast<int>(kl - static_cast<long>(k) * P.pair.layers);
        move_head(P.pair, P.from[k], P.to[k], layer, head, kBlock / 16, threadIdx.x);
    }
}

// Workgroups 0 .. chunks-1: a chunk's counts and new numbers; the next B: a sequence's row; the rest share the moves.
__global__ void __launch_bounds__(kWG) compact_apply(const CompactParams P, int chunks) {
    const int tid = threadIdx.x, M = P.M;
    auto moved = [&](int e) {
        const int v = P.number[e];
        return v < P.P ? v : P.to[v - P.P];
    };
    if (static_cast<int>(blockIdx.x) < chunks) {
        __shared__ int lds[kWG / 64];
        const int used = P.totals[0];
        int holes = 0;                                        // in front of this chunk
        {
            const long begin = blockIdx.x * static_cast<long>(kPagesChunk);
            holes = static_cast<int>(begin) - sum_wg(P.used_count, blockIdx.x, tid, lds);
        }
        for (int k = 0; k < kPagesChunk / kWG; ++k) {
            const long e = blockIdx.x * static_cast<long>(kPagesChunk) + k * kWG + tid;
            const int v = e < P.P ? P.number[e] : 0;
            int all;
            const int hole = holes + scan_wg(e < P.P && v < 0, tid, lds, &all);
            holes += all;
            if (e >= P.P) continue;
            const int refs = P.refs[e];                       // (refs_out may be the same memory: each entry is read by the thread that writes it)
            P.refs_out[e] = e >= used ? 0 : v >= 0 ? refs : P.count[hole];
            if (P.remap) P.remap[e] = v < P.P ? v : P.to[v - P.P];
        }
        if (blockIdx.x == 0 && tid == 0 && P.used_out) P.used_out[0] = used;
        return;
    }
    if (static_cast<int>(blockIdx.x) < chunks + P.B) {
        __shared__ int wrong_place;
        const int b = static_cast<int>(blockIdx.x) - chunks;
        const int* row = P.table + static_cast<size_t>(b) * M;
        int* out = P.table_out + static_cast<size_t>(b) * M;
        if (tid == 0) wrong_place = 0;
        __syncthreads();
        for (int j = tid; j < M; j += kWG) {
            const int e = row[j];
            const int to = e >= 0 && e < P.P ? moved(e) : -1;
            if (e >= 0 && to < 0) wrong_place = 1;
            out[j] = to;
        }
        __syncthreads();
        if (tid == 0 && P.status) P.status[b] = wrong_place ? FSD_ROW_BAD_CACHE : 0;
        return;
    }
    move_pages(P, static_cast<long>(blockIdx.x) - chunks - P.B, static_cast<long>(gridDim.x) - chunks - P.B);
}

// All of it but the moves in one workgroup
__global__ void __launch_bounds__(kSmallWG) compact_small(const CompactParams P) {
    __shared__ int number[kSmallBlocks];                      // as P.number, but of a moved one where it goes
    __shared__ int to[kSmallBlocks / 2 + 1];
    __shared__ int count[kSmallBlocks / 2 + 1];
    __shared__ int lds[kSmallWG / 64];
    __shared__ int wrong[kSmallWG];                           // (B <= kSmallWG)
    const int tid = threadIdx.x;
    int used = 0;
    for (int e0 = 0; e0 < P.P; e0 += kSmallWG) {
        int all;
        scan_wg<kSmallWG>(e0 + tid < P.P && P.refs[e0 + tid] > 0, tid, lds, &all);
        used += all;
    }
    // used blocks in front of one, holes in front of one and movers in front of one
    int holes = 0, movers = 0;
    for (int e0 = 0; e0 < P.P; e0 += kSmallWG) {
        const int e = e0 + tid, refs = e < P.P ? P.refs[e] : 0;
        const bool hole = e < used && refs <= 0, mover = e >= used && refs > 0;
        int all_holes, all_movers;
        const int h = holes + scan_wg<kSmallWG>(hole, tid, lds, &all_holes), m = movers + scan_wg<kSmallWG>(mover, tid, lds, &all_movers);
        holes += all_holes;
        movers += all_movers;
        if (hole) {
            to[h] = e;
            P.to[h] = e;
        }
        if (mover) {
            count[m] = refs;
            P.from[m] = e;
        }
        if (e < P.P) number[e] = hole ? -2 - h : mover ? P.P + m : refs > 0 ? e : -1;
    }
    __syncthreads();
    for (int e = tid; e < P.P; e += kSmallWG) {
        const int v = number[e], goes = v >= P.P ? to[v - P.P] : v < 0 ? -1 : v;
        const int refs = v <= -2 ? count[-2 - v] : v == e ? P.refs[e] : 0;
        P.refs_out[e] = refs;
        if (P.remap) P.remap[e] = goes;
        number[e] = goes;
    }
    wrong[tid] = 0;
    if (tid == 0) {
        P.totals[0] = used;
        P.totals[1] = movers;
        if (P.used_out) P.used_out[0] = used;
    }
    __syncthreads();
    for (int k = tid; k < P.B * P.M; k += kSmallWG) {
        const int e = P.table[k], goes = e >= 0 && e < P.P ? number[e] : -1;
        if (e >= 0 && goes < 0) wrong[k / P.M] = FSD_ROW_BAD_CACHE;
        P.table_out[k] = goes;
    }
    __syncthreads();
    if (P.status && tid < P.B) P.status[tid] = wrong[tid];
}
__global__ void __launch_bounds__(kWG) compact_move(const CompactParams P) { move_pages(P, blockIdx.x, gridDim.x); }

}  // namespace

#endif  // FSD_CSRC_CACHE_PAGES_H_
