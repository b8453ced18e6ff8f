// Eviction from the cache by accumulated attention weight: a session that has more
// than `limit` tokens falls back to m of them (block-level allocation, §5.1; the
// paged block pool of §6).  In every layer and KV head on its own the tokens
//   of the first `first` slots, then the latest ones (position >= next - recent),
//   then those of the largest weight, of equal ones those in lower slots
// stay, m in all.  Attention does not depend on the order of its keys, so nothing is
// shifted: with the evicted slots below m in ascending order and the tokens that stay
// behind m in ascending order, the i-th token moves into the i-th slot.  Their numbers
// are equal, sources lie behind m and targets below, so all moves are independent.
#include <algorithm>

#include "common.h"

namespace ls {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Slots whose ranking keys are kept in LDS (a longer session's are computed again for
// each pass): tables of up to 160 columns, and wider ones.
constexpr int kEvKeysShort = 2560, kEvKeysLong = 16384;
constexpr int kBins = 2048;                  // of a ranking key's 11 bits
constexpr int kEvMoves = kBins / 2;          // moves at a time (their slots, where the bins were)
static_assert(kMaxCacheBlocks * kBlock <= kEvKeysLong * 32, "a bit for each slot where the keys would be");
constexpr int kPlanThreads = 1024;
constexpr int kEvSlices = 8;

struct EvictArgs {
    uint16_t *pool;                // layer base of the first layer
    int64_t num_blocks;
    int32_t num_kv_heads;
    int32_t num_sessions;
    const int32_t *lens;           // [S]
    const int32_t *tables;         // [S][max_blocks]
    int32_t max_blocks;
    int32_t budget, limit, recent;
    const int32_t *first;          // [S] or null
    const int32_t *next_pos;       // [S]
    const float *weights;          // layer base of the first layer, [layers][num_blocks][Hkv][16]
    const int32_t *positions;
    float *weights_next;
    int32_t *positions_next;
    int32_t *next_lens;            // [S]
    int32_t *ring;                 // or null
    int32_t ring_size;
    const int64_t *counts;
    int64_t *next_counts;
    int32_t slices;                // workgroups that share a (session, KV head, layer)
    bool plans;                    // workgroup 0 plans, and the others check the lengths for themselves
    unsigned int *err;
};

__device__ __forceinline__ int blocks_of(int tokens) { return (int)(((int64_t)tokens + kBlock - 1) / kBlock); }

// Tokens that session s keeps of its L.
__device__ __forceinline__ int keeps(const EvictArgs &a, int s, int L) {
    if (L <= a.limit) return L;
    const int first = a.first ? min(max(a.first[s], 0), L) : 0;
    return (int)min((int64_t)L, max((int64_t)a.budget, (int64_t)first + a.recent));
}

// Blocks that session s gives back; its length may be wrong.
__device__ __forceinline__ unsigned gives(const EvictArgs &a, int s, bool &wrong) {
    const int L = a.lens[s];
    if (L < 0 || L > (int64_t)a.max_blocks * kBlock) {
        wrong = true;
        return 0u;
    }
    return a.ring ? (unsigned)(blocks_of(L) - blocks_of(keeps(a, s, L))) : 0u;
}
// Sums of blocks saturate at INT32_MAX, more than any ring has room for.
__device__ __forceinline__ unsigned add(unsigned x, unsigned y) { return min(x + y, (unsigned)INT32_MAX); }

// Exclusive prefix sum over the threads, and the total (the former: of sums that have not saturated).
template <int kThreads>
__device__ __forceinline__ unsigned scan(unsigned v, unsigned &total, unsigned *sm_wave) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    unsigned x = v;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const unsigned y = __shfl_up(x, off);
        if (lane >= off) x = add(x, y);
    }
    __syncthreads();
    if (lane == kWave - 1) sm_wave[wave] = x;
    __syncthreads();
    unsigned before = 0u;
    total = 0u;
    for (int w = 0; w < kThreads / kWave; ++w) {
        if (w == wave) before = total;
        total = add(total, sm_wave[w]);
    }
    return before + x - v;
}

// What keeps the whole call from being served (0: nothing), and the blocks that go back.
template <int kThreads>
__device__ __forceinline__ unsigned refusal(const EvictArgs &a, int64_t taken, int64_t given, unsigned &total, unsigned *sm_wave) {
    unsigned v = 0u;
    bool wrong = false;
    for (int s = threadIdx.x; s < a.num_sessions; s += kThreads) v = add(v, gives(a, s, wrong));
    scan<kThreads>(v, total, sm_wave);
    if (__syncthreads_or(wrong)) return LS_DEVERR_LENGTH;
    const int64_t avail = given - taken;
    if (a.ring && (taken < 0 || avail < 0 || avail > a.ring_size || total == INT32_MAX || total > a.ring_size - avail))
        return LS_DEVERR_FREE_LIST;
    return 0u;
}

// Lengths after the call, and the blocks behind them to the ring: one workgroup.  All
// sessions are served or none.
template <int kThreads>
__device__ __forceinline__ void plan(const EvictArgs &a, unsigned *sm_wave, unsigned *sm_at, int *sm_col) {
    const int tid = threadIdx.x, S = a.num_sessions;
    // (before anything is written: the counters may advance in place)
    int64_t taken = 0, given = 0;
    if (a.ring) {
        taken = a.counts[0];
        given = a.counts[1];
    }
    unsigned total;
    const unsigned bad = refusal<kThreads>(a, taken, given, total, sm_wave);
    if (tid == 0) {
        if (bad) flag_error(a.err, bad);
        if (a.ring) {
            a.next_counts[0] = taken;
            a.next_counts[1] = given + (bad ? 0 : total);
        }
    }
    unsigned carry = 0u;
    for (int s0 = 0; s0 < S; s0 += kThreads) {
        const int s = s0 + tid;
        unsigned n = 0u;
        int m = 0;
        if (s < S) {
            const int L = m = a.lens[s];
            if (!bad) {
                m = keeps(a, s, L);
                n = a.ring ? (unsigned)(blocks_of(L) - blocks_of(m)) : 0u;
            }
            a.next_lens[s] = m;
        }
        unsigned all;
        sm_at[tid] = scan<kThreads>(n, all, sm_wave);
        sm_col[tid] = blocks_of(m);
        __syncthreads();
        // thread = block that goes back: the last session whose blocks begin at or before it
        for (unsigned i = tid; i < all; i += kThreads) {
            int e = 0;
#pragma unroll
            for (int step = kThreads / 2; step > 0; step >>= 1)
                if (sm_at[e + step] <= i) e += step;
            const int id = a.tables[(int64_t)(s0 + e) * a.max_blocks + sm_col[e] + (i - sm_at[e])];
            if (id < 0 || id >= a.num_blocks) flag_error(a.err, LS_DEVERR_BLOCK_ID);
            a.ring[(given + carry + i) % a.ring_size] = id;
        }
        carry += all;
        __syncthreads();
    }
}

__global__ __launch_bounds__(kPlanThreads) void evict_plan_kernel(EvictArgs a) {
    __shared__ unsigned sm_wave[kPlanThreads / kWave], sm_at[kPlanThreads];
    __shared__ int sm_col[kPlanThreads];
    plan<kPlanThreads>(a, sm_wave, sm_at, sm_col);
}

// Order of two weights as that of two unsigned words: NaN (1) below all, -0 as 0.
__device__ __forceinline__ uint32_t rank_key(float w) {
    if (w != w) return 1u;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Bits of a ballot below this lane, added to x.
__device__ __forceinline__ unsigned count_below(uint64_t mask, unsigned x) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, x));
}

// Weights and positions of four consecutive slots.
struct Quad {
    f32x4 w;
    i32x4 p;
};

// One (session, KV head, layer) per workgroup, or one of `slices` that all rank the
// tokens and share the moves (entries apart: none of them writes what another reads).
//
// Ranking keys are words in the order of the weights.  The evict-th smallest is found
// from its digits of 11, 11 and 10 bits by counting; keys below it go, and of those
// equal to it the ones in the highest slots.  Then waves go over their contiguous
// shares of the slots, 256 at a time (a lane has four consecutive ones, 16 bytes of
// an entry array), and number the holes below m and the tokens that stay behind it.
//
// Bound by the moves' sectors: a token's V values are 2 bytes in each of D rows of 32 bytes.
// Measured: 64 sessions, about half of them cut to 2048 tokens, 8 layers of 4 heads of
// 128, 125 us a call, 160 MB written (1.5 TB/s; 95 MB needed in all); 8 prompts of up to
// 16384 cut to 1024, 4 layers, 144 us, 103 MB written and 323 read.  43 and 42 us
// without the moves.  Entries and counters in place: 121 and 189 us.  V tiles of blocks with holes,
// read and written whole: 152 us for 127.
template <int D, int kThreads, int kKeys>
__global__ __launch_bounds__(kThreads) void evict_kernel(EvictArgs a) {
    constexpr int kWaves = kThreads / kWave;
    constexpr int kStep = 4 * kWave;               // slots of a wave's step
    __shared__ __attribute__((aligned(16))) uint32_t sm_key[kKeys];
    __shared__ __attribute__((aligned(16))) uint32_t sm_bin[kBins];
    __shared__ uint64_t sm_flags[kKeys / 64];
    __shared__ unsigned sm_wave[2][kWaves];
    __shared__ uint32_t sm_digit, sm_rest, sm_ties;
    static_assert(2 * kThreads <= kBins, "the plan fits the bins");
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int H = a.num_kv_heads, S = a.num_sessions, slices = a.slices;
    int x = blockIdx.x, h = blockIdx.y, la = blockIdx.z;
    unsigned bad = 0u;
    if (a.plans) {
        if (x-- == 0) {
            plan<kThreads>(a, sm_wave[0], sm_bin, reinterpret_cast<int *>(sm_bin) + kThreads);
            return;
        }
        h = x / (S * slices) % H;
        la = x / (S * slices) / H;
        x %= S * slices;
        unsigned total;
        bad = refusal<kThreads>(a, a.ring ? a.counts[0] : 0, a.ring ? a.counts[1] : 0, total, sm_wave[0]);
    }
    const int slice = x / S, s = x % S;
    const int32_t *table = a.tables + (int64_t)s * a.max_blocks;
    const int64_t entries = (int64_t)la * a.num_blocks * H * kBlock;
    const float *weights = a.weights + entries;
    const int32_t *positions = a.positions + entries;
    float *weights_next = a.weights_next + entries;
    int32_t *positions_next = a.positions_next + entries;
    const bool apart = a.weights_next != a.weights;
    const int L = (int)min((int64_t)max(a.lens[s], 0), (int64_t)a.max_blocks * kBlock);
    const int m = bad ? L : a.plans ? keeps(a, s, L) : min(max(a.next_lens[s], 0), L);
    const bool cut = m < L;
    if (!cut && (!apart || slice)) return;
    // First entry of a block, or -1: it is not in the pool.
    auto block_entry = [&](int col) -> int64_t {
        const int id = table[col];
        return id < 0 || id >= a.num_blocks ? -1 : ((int64_t)id * H + h) * kBlock;
    };
    auto load = [&](int64_t e) { return Quad{*reinterpret_cast<const f32x4 *>(weights + e), *reinterpret_cast<const i32x4 *>(positions + e)}; };
    if (!cut) {
        for (int t = tid * 4; t < L; t += kThreads * 4) {
            const int64_t e = block_entry(t / kBlock);
            if (e < 0) continue;
            const Quad x = load(e + t % kBlock);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t + i < L) {
                    weights_next[e + t % kBlock + i] = x.w[i];
                    positions_next[e + t % kBlock + i] = x.p[i];
                }
        }
        return;
    }
    const int first = a.first ? min(max(a.first[s], 0), m) : 0;
    const int64_t late = (int64_t)a.next_pos[s] - a.recent;
    // Keys of slots t .. t + 3: the largest for first and latest tokens.  Absent ones cannot move or be moved
    // to: below m the largest (at most t slots come before slot t, so all of these stay), behind it 0 (no more
    // than L - m, so all of these go).
    auto keys_of = [&](int t, bool &missing) -> u32x4 {
        const int64_t e = block_entry(t / kBlock);
        u32x4 k = {0u, 0u, 0u, 0u};
        if (e < 0) {
            missing = true;
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = t + i < m ? 0xFFFFFFFFu : 0u;
        } else {
            const Quad x = load(e + t % kBlock);
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = x.p[i] >= late ? 0xFFFFFFFFu : rank_key(x.w[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < first) k[i] = 0xFFFFFFFFu;
        return k;
    };
    const bool cached = L <= kKeys;
    bool missing = false;
    if (cached) {
#pragma unroll 4
        for (int t = tid * 4; t < L; t += kThreads * 4) *reinterpret_cast<u32x4 *>(&sm_key[t]) = keys_of(t, missing);
    } else {
        for (int t = tid * kBlock; t < L; t += kThreads * kBlock) missing = missing || block_entry(t / kBlock) < 0;
    }
    if (missing && la == 0 && h == 0 && slice == 0) flag_error(a.err, LS_DEVERR_BLOCK_ID);
    auto keys = [&](int t) -> u32x4 {
        bool unused;
        return cached ? *reinterpret_cast<const u32x4 *>(&sm_key[t]) : keys_of(t, unused);
    };
    // ---- the evict-th smallest key (a table's slots behind L are no tokens)
    uint32_t prefix = 0u, rest = (uint32_t)(L - m);    // of the keys that begin with prefix, the rest-th smallest
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass < 2 ? 11 : 10;
        for (int i = tid; i < kBins; i += kThreads) sm_bin[i] = 0u;
        __syncthreads();
        for (int t = tid * 4; t < L; t += kThreads * 4) {
            const u32x4 k = keys(t);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t + i < L && (pass == 0 || k[i] >> (shift + bits) == prefix >> (shift + bits)))
                    atomicAdd(&sm_bin[(k[i] >> shift) & ((1u << bits) - 1u)], 1u);
        }
        __syncthreads();
        // A thread has kBins / kThreads bins: the one in which the count passes `rest`.
        constexpr int kPer = kBins / kThreads;
        unsigned own[kPer], x = 0u;
#pragma unroll
        for (int i = 0; i < kPer; ++i) x += own[i] = sm_bin[tid * kPer + i];
        const unsigned mine = x;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const unsigned y = __shfl_up(x, off);
            if (lane >= off) x += y;
        }
        if (lane == kWave - 1) sm_wave[0][wave] = x;
        __syncthreads();
        unsigned before = x - mine;
        for (int w = 0; w < wave; ++w) before += sm_wave[0][w];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (before < rest && rest <= before + own[i]) {
                sm_digit = (uint32_t)(tid * kPer + i);
                sm_rest = rest - before;
                sm_ties = own[i];              // (in the last pass: keys equal to the one found)
            }
            before += own[i];
        }
        __syncthreads();
        prefix |= sm_digit << shift;
        rest = sm_rest;
    }
    // ---- numbers of ties, holes and moving tokens
    const int steps = (L + kStep - 1) / kStep, per = (steps + kWaves - 1) / kWaves;
    const int t_begin = min(wave * per, steps) * kStep, t_end = min((wave + 1) * per, steps) * kStep;
    // Sums of a wave's value over the waves before, and over all.
    auto wave_sums = [&](unsigned v, int which, unsigned &all) {
        if (lane == 0) sm_wave[which][wave] = v;
        __syncthreads();
        unsigned before = 0u;
        all = 0u;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) before = all;
            all += sm_wave[which][w];
        }
        return before;
    };
    const unsigned ties_stay = sm_ties - rest;
    unsigned seen = 0u;                             // ties before the wave's slots, where some stay and some go
    if (ties_stay) {
        unsigned ties = 0u, all_ties;
        for (int t0 = t_begin; t0 < t_end; t0 += kStep) {
            const int t = t0 + lane * 4;
            const u32x4 k = t < L ? keys(t) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 4; ++i) ties += __popcll(__ballot(t + i < L && k[i] == prefix));
        }
        seen = wave_sums(ties, 1, all_ties);
    }
    // Which of the lane's four tokens stay; seen: ties before the step, and after it.
    auto stays = [&](int t, const u32x4 &k, unsigned &seen, bool (&yes)[4]) {
        if (!ties_stay) {
#pragma unroll
            for (int i = 0; i < 4; ++i) yes[i] = t + i < L && k[i] > prefix;
            return;
        }
        unsigned mine = seen;                       // ties before the lane's first slot
        uint64_t tie[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            tie[i] = __ballot(t + i < L && k[i] == prefix);
            mine = count_below(tie[i], mine);
            seen += __popcll(tie[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            yes[i] = t + i < L && (k[i] > prefix || (k[i] == prefix && mine < ties_stay));
            mine += (tie[i] >> lane) & 1u;
        }
    };
    // A bit for each slot whose token stays: four words a step, bit = lane.  Without keys in
    // LDS they take the keys' place; moves in place change what keys are computed from.
    uint64_t *flags = cached ? sm_flags : reinterpret_cast<uint64_t *>(sm_key);
    unsigned holes = 0u, movers = 0u, all_holes, all_movers;
    for (int t0 = t_begin; t0 < t_end; t0 += kStep) {
        const int t = t0 + lane * 4;
        bool yes[4];
        const u32x4 k = t < L ? keys(t) : u32x4{0u, 0u, 0u, 0u};
        stays(t, k, seen, yes);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            holes += __popcll(__ballot(t + i < m && !yes[i]));
            movers += __popcll(__ballot(t + i >= m && yes[i]));
            const uint64_t f = __ballot(yes[i]);
            if (lane == 0) flags[t0 / 64 + i] = f;
        }
    }
    __syncthreads();
    unsigned hole0 = wave_sums(holes, 0, all_holes), mover0 = wave_sums(movers, 1, all_movers);
    // (all_holes = all_movers, since m tokens stay)
    if (apart && slice == 0)
        for (int t = tid * 4; t < m; t += kThreads * 4) {
            const int64_t e = block_entry(t / kBlock);
            if (e < 0) continue;
            const Quad x = load(e + t % kBlock);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t + i < m && (flags[t / kStep * 4 + i] >> (t % kStep / 4)) & 1u) {
                    weights_next[e + t % kBlock + i] = x.w[i];
                    positions_next[e + t % kBlock + i] = x.p[i];
                }
        }
    // ---- the moves, a batch at a time
    int *sm_from = reinterpret_cast<int *>(sm_bin), *sm_to = sm_from + kEvMoves;
    const unsigned share = (all_movers + slices - 1) / slices, last = min((slice + 1) * share, all_movers);
    // A move takes D / 8 lanes: 16 bytes of K each, and 8 dims of V that are D / 8 apart, so that
    // neighbours' 2-byte elements, 32 bytes apart, fall into the same lines.
    constexpr int kLanes = D / 8;
    for (unsigned base = slice * share; base < last; base += kEvMoves) {
        const unsigned n = min(last - base, (unsigned)kEvMoves);
        __syncthreads();                           // the batch before has been read
        unsigned hole = hole0, mover = mover0;
        for (int t0 = t_begin; t0 < t_end; t0 += kStep) {
            const int t = t0 + lane * 4;
            uint64_t f[4], go[4], come[4];
            unsigned i_hole = hole, i_mover = mover;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[i] = flags[t0 / 64 + i];
                const bool yes = (f[i] >> lane) & 1u;
                come[i] = __ballot(t + i < m && !yes);
                go[i] = __ballot(t + i >= m && yes);
                i_hole = count_below(come[i], i_hole);
                i_mover = count_below(go[i], i_mover);
                hole += __popcll(come[i]);
                mover += __popcll(go[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if ((come[i] >> lane) & 1u) {
                    if (i_hole - base < n) sm_to[i_hole - base] = t + i;
                    ++i_hole;
                }
                if ((go[i] >> lane) & 1u) {
                    if (i_mover - base < n) sm_from[i_mover - base] = t + i;
                    ++i_mover;
                }
            }
        }
        __syncthreads();
        const int c = tid % kLanes;
        uint16_t *slab = a.pool + (int64_t)la * a.num_blocks * 2 * H * (kBlock * D);
#pragma unroll 2
        for (unsigned x = tid / kLanes; x < n; x += kThreads / kLanes) {
            const int from = sm_from[x], to = sm_to[x], fo = from % kBlock, too = to % kBlock;
            const int fb = table[from / kBlock], tb = table[to / kBlock];
            if (fb < 0 || fb >= a.num_blocks || tb < 0 || tb >= a.num_blocks) continue;
            const uint16_t *fk = slab + ((int64_t)fb * 2 * H + h) * (kBlock * D), *fv = fk + (int64_t)H * (kBlock * D);
            uint16_t *tk = slab + ((int64_t)tb * 2 * H + h) * (kBlock * D), *tv = tk + (int64_t)H * (kBlock * D);
            const u32x4 kv = *reinterpret_cast<const u32x4 *>(fk + (c * kBlock + fo) * 8);
            uint16_t v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fv[(e * kLanes + c) * kBlock + fo];
            const int64_t ef = ((int64_t)fb * H + h) * kBlock + fo, et = ((int64_t)tb * H + h) * kBlock + too;
            float w = 0.f;
            int p = 0;
            if (c == 0) {
                w = weights[ef];
                p = positions[ef];
            }
            *reinterpret_cast<u32x4 *>(tk + (c * kBlock + too) * 8) = kv;
#pragma unroll
            for (int e = 0; e < 8; ++e) tv[(e * kLanes + c) * kBlock + too] = v[e];
            if (c == 0) {
                weights_next[et] = w;
                positions_next[et] = p;
            }
        }
    }
}

}  // namespace

hipError_t launch_evict(const PoolGeom &p, int32_t layer_begin, int32_t layer_count, const EvictCall &c, unsigned int *err,
                        hipStream_t stream) {
    const int64_t entries = (int64_t)layer_begin * p.num_blocks * p.num_kv_heads * kBlock;
    EvictArgs a = {};
    a.pool = p.layer_base(layer_begin);
    a.num_blocks = p.num_blocks;
    a.num_kv_heads = p.num_kv_heads;
    a.num_sessions = c.num_sessions;
    a.lens = c.seq_lens;
    a.tables = c.block_tables;
    a.max_blocks = c.max_blocks;
    a.budget = c.budget;
    a.limit = c.limit;
    a.recent = c.recent;
    a.first = c.first_lens;
    a.next_pos = c.next_positions;
    a.weights = c.weights + entries;
    a.positions = c.positions + entries;
    a.weights_next = c.weights_next + entries;
    a.positions_next = c.positions_next + entries;
    a.next_lens = c.next_lens;
    a.ring = c.free_ring;
    a.ring_size = c.ring_size;
    a.counts = c.free_counts;
    a.next_counts = c.next_counts;
    a.err = err;
    // With entries apart, and workgroups for a part of the CUs only, several share a (session, KV head,
    // layer)'s moves.
    const int64_t whole = (int64_t)c.num_sessions * p.num_kv_heads * layer_count, cus = stream_cus(p, stream);
    a.slices = c.weights_next != c.weights && whole ? (int)std::max<int64_t>(1, std::min<int64_t>(kEvSlices, 2 * cus / whole)) : 1;
    // Up to a thousand sessions, whose lengths a workgroup reads in a microsecond, one launch does all
    // (but where the plan would write the counters that the others read, and in grids of 2^32 threads).
    a.plans = whole && (!c.free_ring || c.next_counts != c.free_counts) && c.num_sessions <= kPlanThreads && whole * a.slices < 1 << 21;
    const dim3 grid = a.plans ? dim3((unsigned)(1 + whole * a.slices))
                              : dim3((unsigned)(c.num_sessions * a.slices), (unsigned)p.num_kv_heads, (unsigned)layer_count);
    if (!a.plans) {
        hipLaunchKernelGGL(evict_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
        if (hipError_t e = hipGetLastError()) return e;
        if (!whole) return hipSuccess;
    }
    // By the table's width, as the lengths are on the device: in workgroups of four waves if every
    // session's keys fit (64 sessions cut to 2048 as above 125 us, cut to 1024 109), else of sixteen (the same
    // sessions in tables of 1024 columns 153 and 132; cut to 4096 194).
    const bool narrow = (int64_t)c.max_blocks * kBlock <= kEvKeysShort;
#define LS_EVICT(D, THREADS, KEYS) hipLaunchKernelGGL((evict_kernel<D, THREADS, KEYS>), grid, dim3(THREADS), 0, stream, a)
    if (p.head_dim == 128) {
        if (narrow) LS_EVICT(128, 256, kEvKeysShort);
        else LS_EVICT(128, 1024, kEvKeysLong);
    } else {
        if (narrow) LS_EVICT(64, 256, kEvKeysShort);
        else LS_EVICT(64, 1024, kEvKeysLong);
    }
#undef LS_EVICT
    return hipGetLastError();
}

}  // namespace ls
