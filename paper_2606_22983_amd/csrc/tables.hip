// Block tables and slot maps from the sessions' lengths, on the GPU: the
// bookkeeping of a step (block-level allocation, §5.1; the paged block pool of
// §6) without the host.  Free blocks stand in a ring of ids in device memory:
// with counters `taken` and `given`, ids [taken, given) of it (modulo its size)
// are free.  A step of S sessions, session s with L_s tokens in the pool and n_s
// new ones:
//   cu[s]    = n_0 + .. + n_{s-1}                    rows of q, k_new, v_new
//   need_s   = ceil((L_s + n_s) / 16) - ceil(L_s / 16)  blocks taken
//   dead(x)  = blocks behind those of the first tokens that end before x - W + 1,
//              the first key a query at position x sees
//   gives_s  = dead(L_s + n_s) - dead(L_s)           blocks no later step sees
// Sessions take and give in their order, each its blocks in ascending order.
#include "common.h"

namespace ls {

namespace {

constexpr int kTabThreads = 1024;
constexpr int kTabWaves = kTabThreads / kWave;

struct TablesArgs {
    int64_t num_blocks;
    int32_t num_sessions;
    const int32_t *lens;           // [S] tokens in the pool
    const int32_t *new_lens;       // [S]
    int32_t *tables;               // [S][max_blocks]
    int32_t max_blocks;
    int32_t *ring;                 // [ring_size], or null: the tables hold every block
    int32_t ring_size;
    const int64_t *counts;         // taken, given
    int64_t *next_counts;
    int32_t window;                // 0: nothing is given back
    int32_t sinks;
    int32_t total;                 // slots
    int32_t max_new;
    int32_t *next_lens;            // [S]
    int32_t *cu;                   // [S+1]
    int32_t *reused;               // [S], or null
    int64_t *slots;                // [total]
    unsigned int *err;
};

struct SessionStep {
    int L, n, b0, need, d0, gives; // lengths; first block taken, count; first block given (behind the sinks'), count
};

__device__ __forceinline__ int dead_blocks(const TablesArgs &a, int x) {
    if (!a.window || x < a.window) return 0;
    return max((x - a.window + 1) / kBlock - (a.sinks + kBlock - 1) / kBlock, 0);
}

// Session s's step; false: lengths that the call cannot serve.
__device__ __forceinline__ bool session_step(const TablesArgs &a, int s, SessionStep &t) {
    t.L = a.lens[s];
    t.n = a.new_lens[s];
    const bool ok = t.L >= 0 && t.n >= 0 && t.n <= a.max_new && (int64_t)t.L + t.n <= (int64_t)a.max_blocks * kBlock;
    if (!ok) t.L = t.n = 0;
    t.b0 = (t.L + kBlock - 1) / kBlock;
    t.need = a.ring ? (t.L + t.n + kBlock - 1) / kBlock - t.b0 : 0;
    t.d0 = a.ring ? dead_blocks(a, t.L) : 0;
    t.gives = a.ring ? dead_blocks(a, t.L + t.n) - t.d0 : 0;
    return ok;
}

__device__ __forceinline__ int ring_at(int first, int i, int size) {
    const int at = first - size + i;                 // (first, i < size: no overflow)
    return at < 0 ? at + size : at;
}

// One workgroup for the whole step: its latency is what a step's bookkeeping
// costs, and a step of a decode batch moves a few KB.  `width` lanes (a power of
// two, at least as many as the longest turn has tokens, up to a wave) share a
// session when blocks and slots are written.
__global__ __launch_bounds__(kTabThreads) void tables_kernel(TablesArgs a, int width) {
    __shared__ int64_t sm_sum[3][kTabWaves];
    __shared__ unsigned sm_scan[3][kTabWaves];
    __shared__ SessionStep sm_step[kTabThreads];
    __shared__ int sm_cu[kTabThreads], sm_take[kTabThreads], sm_give[kTabThreads];
    __shared__ unsigned sm_bad;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int S = a.num_sessions;
    if (tid == 0) sm_bad = 0u;
    __syncthreads();
    // ---- totals: the step is refused as a whole when some length is out of
    // range, or rows, free blocks or the ring's room do not suffice.
    int64_t sum[3] = {0, 0, 0};
    bool good = true;
    for (int s = tid; s < S; s += kTabThreads) {
        SessionStep t;
        good = session_step(a, s, t) && good;
        sum[0] += t.n;
        sum[1] += t.need;
        sum[2] += t.gives;
    }
    if (!good) atomicOr(&sm_bad, LS_DEVERR_LENGTH);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        for (int off = 32; off > 0; off >>= 1) sum[k] += __shfl_xor(sum[k], off);
        if (lane == 0) sm_sum[k][wave] = sum[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        sum[k] = 0;
        for (int w = 0; w < kTabWaves; ++w) sum[k] += sm_sum[k][w];
    }
    unsigned bad = sm_bad;
    if (sum[0] > a.total) bad |= LS_DEVERR_LENGTH;
    int64_t taken = 0, given = 0;
    if (a.ring) {
        taken = a.counts[0];
        given = a.counts[1];
        const int64_t avail = given - taken;
        if (taken < 0 || avail < 0 || avail > a.ring_size || sum[1] > avail || sum[2] > a.ring_size - avail)
            bad |= LS_DEVERR_FREE_LIST;
    }
    __syncthreads();                                 // every thread has the counts (next_counts may be the same memory)
    if (bad) {
        if (tid == 0) flag_error(a.err, bad);
        sum[0] = sum[1] = sum[2] = 0;
    }
    if (tid == 0 && a.ring) {
        a.next_counts[0] = taken + sum[1];
        a.next_counts[1] = given + sum[2];
    }
    for (int64_t i = sum[0] + tid; i < a.total; i += kTabThreads) a.slots[i] = -1;
    if (tid == 0) a.cu[0] = 0;
    const int take0 = a.ring && !bad ? (int)(taken % a.ring_size) : 0, give0 = a.ring && !bad ? (int)(given % a.ring_size) : 0;
    unsigned carry[3] = {0u, 0u, 0u};
    const int first_kept = (a.sinks + kBlock - 1) / kBlock;
    for (int s0 = 0; s0 < S; s0 += kTabThreads) {
        // ---- prefix sums over this chunk of sessions.
        const int s = s0 + tid;
        SessionStep t = {0, 0, 0, 0, 0, 0};
        if (s < S) {
            const int L = a.lens[s];
            session_step(a, s, t);
            if (bad) t.n = t.need = t.gives = 0;
            if (a.reused) a.reused[s] = L;
            a.next_lens[s] = L + t.n;
        }
        const unsigned v[3] = {(unsigned)t.n, (unsigned)t.need, (unsigned)t.gives};
        unsigned x[3] = {v[0], v[1], v[2]};
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1)
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const unsigned y = __shfl_up(x[k], off);
                if (lane >= off) x[k] += y;
            }
        if (lane == kWave - 1)
#pragma unroll
            for (int k = 0; k < 3; ++k) sm_scan[k][wave] = x[k];
        __syncthreads();
        unsigned before[3], all[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            before[k] = carry[k] + x[k] - v[k];
            all[k] = 0;
            for (int w = 0; w < kTabWaves; ++w) {
                const unsigned y = sm_scan[k][w];
                if (w < wave) before[k] += y;
                all[k] += y;
            }
            carry[k] += all[k];
        }
        sm_step[tid] = t;
        sm_cu[tid] = (int)before[0];
        sm_take[tid] = (int)before[1];
        sm_give[tid] = (int)before[2];
        if (s < S) a.cu[s + 1] = (int)(before[0] + v[0]);
        __syncthreads();
        // ---- blocks and slots: `width` lanes per session.
        if (!bad) {
            const int li = tid % width;
            for (int e = tid / width; e < min(kTabThreads, S - s0); e += kTabThreads / width) {
                const SessionStep u = sm_step[e];
                if (!u.n) continue;
                int32_t *row = a.tables + (int64_t)(s0 + e) * a.max_blocks;
                // Id of the session's block j: taken in this step, or in the table.
                auto id_of = [&](int j) {
                    const int i = j - u.b0;
                    return i >= 0 && i < u.need ? a.ring[ring_at(take0, ring_at(sm_take[e], i, a.ring_size), a.ring_size)] : row[j];
                };
                auto inside = [&](int id) { return id >= 0 && id < a.num_blocks; };
                for (int i = li; i < u.n; i += width) {
                    const int pos = u.L + i, id = id_of(pos / kBlock);
                    const bool ok = inside(id);
                    if (!ok) flag_error(a.err, LS_DEVERR_BLOCK_ID);
                    a.slots[sm_cu[e] + i] = ok ? (int64_t)id * kBlock + pos % kBlock : -1;
                }
                for (int i = li; i < u.gives; i += width) {
                    const int id = id_of(first_kept + u.d0 + i);
                    if (!inside(id)) flag_error(a.err, LS_DEVERR_BLOCK_ID);
                    a.ring[ring_at(give0, ring_at(sm_give[e], i, a.ring_size), a.ring_size)] = id;
                }
                for (int i = li; i < u.need; i += width) row[u.b0 + i] = id_of(u.b0 + i);
            }
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_tables(const PoolGeom &p, int32_t num_sessions, const int32_t *seq_lens, const int32_t *new_lens,
                         int32_t *block_tables, int32_t max_blocks, int32_t *free_ring, int32_t ring_size,
                         const int64_t *free_counts, int64_t *next_counts, int32_t window, int32_t sinks,
                         int32_t total_tokens, int32_t max_new_len, int32_t *next_lens, int32_t *cu_new_lens,
                         int32_t *reused_lens, int64_t *slot_map, unsigned int *err, hipStream_t stream) {
    TablesArgs a;
    a.num_blocks = p.num_blocks;
    a.num_sessions = num_sessions;
    a.lens = seq_lens;
    a.new_lens = new_lens;
    a.tables = block_tables;
    a.max_blocks = max_blocks;
    a.ring = free_ring;
    a.ring_size = ring_size;
    a.counts = free_counts;
    a.next_counts = next_counts;
    a.window = window;
    a.sinks = sinks;
    a.total = total_tokens;
    a.max_new = max_new_len;
    a.next_lens = next_lens;
    a.cu = cu_new_lens;
    a.reused = reused_lens;
    a.slots = slot_map;
    a.err = err;
    int width = 1;
    while (width < max_new_len && width < kWave) width *= 2;
    hipLaunchKernelGGL(tables_kernel, dim3(1), dim3(kTabThreads), 0, stream, a, width);
    return hipGetLastError();
}

}  // namespace ls
