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

constexpr int kEvThreads = 256;
constexpr int kEvWaves = kEvThreads / kWave;
constexpr int kEvMoves = 2048;               // moves at a time (LDS)
// Tokens whose ranking keys are kept in LDS (a longer session's are computed again for
// each pass): caches around a budget of 2048, and long prompts.
constexpr int kEvKeysShort = 2304, kEvKeysLong = 16384;
constexpr int kBins = 256;                   // of a ranking key's 8 bits
constexpr int kPlanThreads = 1024;

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
    unsigned int *err;
};

__device__ __forceinline__ int blocks_of(int tokens) { return (int)(((int64_t)tokens + kBlock - 1) / kBlock); }

// Tokens that session s keeps of its L.
__device__ __forceinline__ int keeps(const EvictArgs &a, int s, int L) {
    if (L <= a.limit) return L;
    const int first = a.first ? min(max(a.first[s], 0), L) : 0;
    return (int)min((int64_t)L, max((int64_t)a.budget, (int64_t)first + a.recent));
}

// Lengths after the call, and the blocks behind them to the ring: one workgroup.  All
// sessions are served or none.
__global__ __launch_bounds__(kPlanThreads) void evict_plan_kernel(EvictArgs a) {
    __shared__ unsigned sm_wave[kPlanThreads / kWave];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, S = a.num_sessions;
    const int64_t cap = (int64_t)a.max_blocks * kBlock;
    int64_t taken = 0, given = 0;
    if (a.ring) {
        taken = a.counts[0];
        given = a.counts[1];
    }
    auto gives = [&](int s, bool &wrong) -> unsigned {
        const int L = a.lens[s];
        if (L < 0 || L > cap) {
            wrong = true;
            return 0u;
        }
        return a.ring ? (unsigned)(blocks_of(L) - blocks_of(keeps(a, s, L))) : 0u;
    };
    // Exclusive prefix sum over the threads, and the total.
    auto scan = [&](unsigned v, unsigned &total) {
        unsigned x = v;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const unsigned y = __shfl_up(x, off);
            if (lane >= off) x += y;
        }
        __syncthreads();
        if (lane == kWave - 1) sm_wave[wave] = x;
        __syncthreads();
        unsigned before = 0u;
        total = 0u;
        for (int w = 0; w < kPlanThreads / kWave; ++w) {
            if (w == wave) before = total;
            total += sm_wave[w];
        }
        return before + x - v;
    };
    unsigned v = 0u, total;
    bool wrong = false;
    for (int s = tid; s < S; s += kPlanThreads) v += gives(s, wrong);
    scan(v, total);
    unsigned bad = __syncthreads_or(wrong) ? LS_DEVERR_LENGTH : 0u;
    if (a.ring && !bad) {
        const int64_t avail = given - taken;
        if (taken < 0 || avail < 0 || avail > a.ring_size || total > a.ring_size - avail) bad = LS_DEVERR_FREE_LIST;
    }
    if (tid == 0) {
        if (bad) flag_error(a.err, bad);
        if (a.ring) {
            a.next_counts[0] = taken;
            a.next_counts[1] = given + (bad ? 0 : total);
        }
    }
    unsigned carry = 0u;
    for (int s0 = 0; s0 < S; s0 += kPlanThreads) {
        const int s = s0 + tid;
        unsigned n = 0u;
        int L = 0, m = 0;
        if (s < S) {
            L = m = a.lens[s];
            if (!bad) {
                m = keeps(a, s, L);
                n = a.ring ? (unsigned)(blocks_of(L) - blocks_of(m)) : 0u;
            }
            a.next_lens[s] = m;
        }
        unsigned all;
        unsigned at = carry + scan(n, all);
        for (unsigned i = 0; i < n; ++i, ++at) {
            const int id = a.tables[(int64_t)s * a.max_blocks + blocks_of(m) + i];
            if (id < 0 || id >= a.num_blocks) flag_error(a.err, LS_DEVERR_BLOCK_ID);
            a.ring[(given + at) % a.ring_size] = id;
        }
        carry += all;
    }
}

// Order of two weights as that of two unsigned words: NaN below all, -0 as 0.
__device__ __forceinline__ uint32_t rank_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One (session, KV head, layer) per workgroup.
template <int D, int kKeys>
__global__ __launch_bounds__(kEvThreads) void evict_kernel(EvictArgs a) {
    __shared__ uint32_t sm_key[kKeys];
    __shared__ uint32_t sm_bin[kBins];
    __shared__ unsigned sm_wave[2][kEvWaves];
    __shared__ int sm_from[kEvMoves], sm_to[kEvMoves];
    __shared__ uint32_t sm_digit, sm_rest;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int s = blockIdx.x, h = blockIdx.y, la = blockIdx.z, H = a.num_kv_heads;
    const int32_t *table = a.tables + (int64_t)s * a.max_blocks;
    const int64_t entries = (int64_t)la * a.num_blocks * H * kBlock;
    const float *weights = a.weights + entries;
    const int32_t *positions = a.positions + entries;
    float *weights_next = a.weights_next + entries;
    int32_t *positions_next = a.positions_next + entries;
    const bool apart = a.weights_next != a.weights;
    const int L = (int)min((int64_t)max(a.lens[s], 0), (int64_t)a.max_blocks * kBlock);
    const int m = min(max(a.next_lens[s], 0), L);
    // Entry of a slot, or -1: its block is not in the pool.
    auto entry = [&](int t) -> int64_t {
        const int id = table[t / kBlock];
        return id < 0 || id >= a.num_blocks ? -1 : ((int64_t)id * H + h) * kBlock + t % kBlock;
    };
    const bool cut = m < L;
    if (apart)
        for (int t = tid; t < m; t += kEvThreads) {
            const int64_t e = entry(t);
            if (e < 0) continue;
            weights_next[e] = weights[e];
            positions_next[e] = positions[e];
        }
    if (!cut) return;
    const int first = a.first ? min(max(a.first[s], 0), m) : 0;
    const int64_t late = (int64_t)a.next_pos[s] - a.recent;
    const int evict = L - m;                       // of the slots [first, L)
    auto key_at = [&](int t) -> uint32_t {
        const int64_t e = entry(t);
        if (e < 0) return 0u;
        return positions[e] >= late ? 0xFFFFFFFFu : rank_key(weights[e]);
    };
    const bool cached = L <= kKeys;
    bool missing = false;
    if (cached)
        for (int t = first + tid; t < L; t += kEvThreads) sm_key[t] = key_at(t);
    for (int t = tid * kBlock; t < L; t += kEvThreads * kBlock) missing = missing || entry(t) < 0;
    if (missing && la == 0 && h == 0) flag_error(a.err, LS_DEVERR_BLOCK_ID);
    __syncthreads();
    auto key = [&](int t) -> uint32_t { return cached ? sm_key[t] : key_at(t); };
    // ---- the evict-th smallest key, eight bits at a time
    uint32_t prefix = 0u, rest = (uint32_t)evict;  // of the keys that begin with prefix, the rest-th smallest
    for (int shift = 24; shift >= 0; shift -= 8) {
        sm_bin[tid] = 0u;
        __syncthreads();
        for (int t = first + tid; t < L; t += kEvThreads) {
            const uint32_t k = key(t);
            if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&sm_bin[(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        // thread = bin: keys in the bins up to and with its own
        unsigned x = sm_bin[tid];
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const unsigned y = __shfl_up(x, off);
            if (lane >= off) x += y;
        }
        if (lane == kWave - 1) sm_wave[0][wave] = x;
        __syncthreads();
        for (int w = 0; w < wave; ++w) x += sm_wave[0][w];
        const unsigned before = x - sm_bin[tid];
        if (before < rest && rest <= x) {
            sm_digit = (uint32_t)tid;
            sm_rest = rest - before;
        }
        __syncthreads();
        prefix |= sm_digit << shift;
        rest = sm_rest;
    }
    // Keys below `prefix` go, and of those equal to it the `rest` in the highest slots.
    const int per = (L - first + kEvThreads - 1) / kEvThreads;
    const int t0 = min(first + tid * per, L), t1 = min(t0 + per, L);
    auto scan = [&](unsigned v, int which, unsigned &total) {
        unsigned x = v;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const unsigned y = __shfl_up(x, off);
            if (lane >= off) x += y;
        }
        if (lane == kWave - 1) sm_wave[which][wave] = x;
        __syncthreads();
        unsigned before = 0u;
        total = 0u;
        for (int w = 0; w < kEvWaves; ++w) {
            if (w == wave) before = total;
            total += sm_wave[which][w];
        }
        return before + x - v;
    };
    unsigned ties = 0u, all_ties;
    for (int t = t0; t < t1; ++t) ties += key(t) == prefix;
    const unsigned ties_before = scan(ties, 0, all_ties);
    const unsigned ties_stay = all_ties - rest;
    auto stays = [&](uint32_t k, unsigned &seen) {  // in the order of the slots
        const bool tie = k == prefix, yes = k > prefix || (tie && seen < ties_stay);
        seen += tie;
        return yes;
    };
    // Of the thread's slots those below m, and those behind it.
    const int h1 = max(min(t1, m), t0), u0 = min(max(t0, m), t1);
    unsigned seen = ties_before, holes = 0u, movers = 0u, all_holes, all_movers;
    for (int t = t0; t < h1; ++t) holes += !stays(key(t), seen);
    const unsigned mover_seen0 = seen;
    for (int t = u0; t < t1; ++t) movers += stays(key(t), seen);
    __syncthreads();
    unsigned i = scan(holes, 0, all_holes), j = scan(movers, 1, all_movers);
    // ---- the moves.  A batch writes weights in place, which keys that are not in LDS are
    // computed from: a thread goes on behind its last hole, in slots not yet written.
    constexpr int kLanes = D / 8;                  // of a move: 16 bytes of K and 8 dims of V each
    unsigned hole_seen = ties_before, mover_seen = mover_seen0;
    int th = t0, tu = u0;
    for (unsigned base = 0u; base < all_movers; base += kEvMoves) {
        __syncthreads();
        for (const unsigned end = base + kEvMoves; th < h1 && i < end; ++th)
            if (!stays(key(th), hole_seen)) sm_to[i++ - base] = th;
        for (const unsigned end = base + kEvMoves; tu < t1 && j < end; ++tu)
            if (stays(key(tu), mover_seen)) sm_from[j++ - base] = tu;
        __syncthreads();
        const int n = (int)min(all_movers - base, (unsigned)kEvMoves);
        for (int x = tid / kLanes; x < n; x += kEvThreads / kLanes) {
            const int64_t from = entry(sm_from[x]), to = entry(sm_to[x]);
            if (from < 0 || to < 0) continue;
            const int c = tid % kLanes;
            // entry = (block Hkv + h) 16 + slot; a block has 2 Hkv tiles
            const int64_t fb = from / kBlock / H, tb = to / kBlock / H;
            const int fo = (int)(from % kBlock), to_o = (int)(to % kBlock);
            uint16_t *slab = a.pool + (int64_t)la * a.num_blocks * 2 * H * (kBlock * D);
            const uint16_t *fk = slab + (fb * 2 * H + h) * (int64_t)(kBlock * D), *fv = fk + (int64_t)H * (kBlock * D);
            uint16_t *tk = slab + (tb * 2 * H + h) * (int64_t)(kBlock * D), *tv = tk + (int64_t)H * (kBlock * D);
            const uint4 kv = *reinterpret_cast<const uint4 *>(fk + (c * kBlock + fo) * 8);
            uint16_t v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fv[(c * 8 + e) * kBlock + fo];
            *reinterpret_cast<uint4 *>(tk + (c * kBlock + to_o) * 8) = kv;
#pragma unroll
            for (int e = 0; e < 8; ++e) tv[(c * 8 + e) * kBlock + to_o] = v[e];
            if (c == 0) {
                weights_next[to] = weights[from];
                positions_next[to] = positions[from];
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
    hipLaunchKernelGGL(evict_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (!c.num_sessions) return hipSuccess;
    const dim3 grid((unsigned)c.num_sessions, (unsigned)p.num_kv_heads, (unsigned)layer_count);
    const bool narrow = (int64_t)c.max_blocks * kBlock <= kEvKeysShort;
#define LS_EVICT(D, KEYS) hipLaunchKernelGGL((evict_kernel<D, KEYS>), grid, dim3(kEvThreads), 0, stream, a)
    if (p.head_dim == 128) {
        if (narrow) LS_EVICT(128, kEvKeysShort);
        else LS_EVICT(128, kEvKeysLong);
    } else {
        if (narrow) LS_EVICT(64, kEvKeysShort);
        else LS_EVICT(64, kEvKeysLong);
    }
#undef LS_EVICT
    return hipGetLastError();
}

}  // namespace ls
