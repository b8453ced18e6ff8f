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

constexpr int kTabRows = 4;             // rows per thread up to which one workgroup does the whole step

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
    int L, n;                      // tokens in the pool, new ones
    unsigned need, gives;          // blocks taken, given back
};

// Blocks behind those of the first tokens that a query at position x or later does not see.
__device__ __forceinline__ int dead_blocks(const TablesArgs &a, int x) {
    if (!a.window || x < a.window) return 0;
    return max((x - a.window + 1) / kBlock - (a.sinks + kBlock - 1) / kBlock, 0);
}

// Session s's step; false: lengths that the call cannot serve.
__device__ __forceinline__ bool session_step(const TablesArgs &a, int s, SessionStep &t) {
    t.L = a.lens[s];
    t.n = a.new_lens[s];
    const bool ok = t.L >= 0 && t.n >= 0 && t.n <= a.max_new && (int64_t)t.L + t.n <= (int64_t)a.max_blocks * kBlock;
    const int L = ok ? t.L : 0, n = ok ? t.n : 0;
    t.n = n;
    t.need = a.ring ? (unsigned)((L + n + kBlock - 1) / kBlock - (L + kBlock - 1) / kBlock) : 0u;
    t.gives = a.ring ? (unsigned)(dead_blocks(a, L + n) - dead_blocks(a, L)) : 0u;
    return ok;
}

// Sums of rows that saturate at INT32_MAX, more than any slot map holds.
__device__ __forceinline__ unsigned add_rows(unsigned x, unsigned y) { return min(x + y, (unsigned)INT32_MAX); }

__device__ __forceinline__ int ring_at(int first, unsigned i, int size) {
    const int at = first - size + (int)i;            // (first, i < size: no overflow)
    return at < 0 ? at + size : at;
}

// Thread = new token.  Everything that a token brings follows from its position
// p: its slot; the table entry of the block it opens (p a multiple of 16); the
// block that the next position's window leaves behind (dead(p + 1) =
// dead(p) + 1).  What hangs on the other sessions are three prefix sums (rows,
// blocks taken, blocks given), which every workgroup makes for itself, kThreads
// sessions at a time.  A step of a decode batch moves a few KB, so the chain of
// latencies is what it costs (lengths, scan, ids, stores), and one workgroup
// without a second pass over the lengths is the shortest; a step of many rows is
// spread over as many workgroups as it has kThreads rows.
//
// write_state: lengths, prefix sums and counters are written, by workgroup 0.
// Where they are the inputs' own memory and there are other workgroups, which
// still read them, a launch of one workgroup without rows does that afterwards.
template <int kThreads>
__global__ __launch_bounds__(kThreads) void tables_kernel(TablesArgs a, int rows_per_wg, int write_state) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ unsigned sm_scan[3][kWaves];
    __shared__ unsigned sm_bad[kWaves];
    __shared__ int sm_cu[kThreads + 1], sm_len[kThreads];
    __shared__ unsigned sm_take[kThreads], sm_give[kThreads];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int S = a.num_sessions;
    int64_t taken = 0, given = 0;
    if (a.ring) {
        taken = a.counts[0];
        given = a.counts[1];
    }
    // Prefix sums of the chunk of sessions from s0 on: exclusive ones in `before`, totals in `all`.
    // bad: lengths that cannot be served (of any of the chunk's sessions).
    auto scan = [&](int s0, SessionStep &t, unsigned (&before)[3], unsigned (&all)[3], bool &bad) {
        t = SessionStep{0, 0, 0u, 0u};
        const bool wrong = s0 + tid < S && !session_step(a, s0 + tid, t);
        const unsigned v[3] = {(unsigned)t.n, t.need, t.gives};
        unsigned x[3] = {v[0], v[1], v[2]};
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const unsigned y0 = __shfl_up(x[0], off), y1 = __shfl_up(x[1], off), y2 = __shfl_up(x[2], off);
            if (lane >= off) {
                x[0] = add_rows(x[0], y0);
                x[1] += y1;
                x[2] += y2;
            }
        }
        const bool any_wrong = __any(wrong);
        if (lane == kWave - 1) {
#pragma unroll
            for (int k = 0; k < 3; ++k) sm_scan[k][wave] = x[k];
            sm_bad[wave] = any_wrong;
        }
        __syncthreads();
        unsigned first[3] = {0u, 0u, 0u}, is_bad = 0u;
        all[0] = all[1] = all[2] = 0u;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) {
                first[0] = all[0];
                first[1] = all[1];
                first[2] = all[2];
            }
            all[0] = add_rows(all[0], sm_scan[0][w]);
            all[1] += sm_scan[1][w];
            all[2] += sm_scan[2][w];
            is_bad |= sm_bad[w];
        }
        bad = is_bad != 0u;
        before[0] = add_rows(first[0], x[0]) - v[0];
        before[1] = first[1] + x[1] - v[1];
        before[2] = first[2] + x[2] - v[2];
    };
    SessionStep t;
    unsigned before[3], all[3];
    bool wrong;
    scan(0, t, before, all, wrong);
    // ---- totals: the step is refused as a whole when some length is out of
    // range, or rows, free blocks or the ring's room do not suffice.
    unsigned sum[3] = {all[0], all[1], all[2]};
    for (int s0 = kThreads; s0 < S; s0 += kThreads) {
        SessionStep u;
        unsigned b[3], c[3];
        bool w;
        __syncthreads();                             // (the last chunk's sums are read)
        scan(s0, u, b, c, w);
        wrong = wrong || w;
        sum[0] = add_rows(sum[0], c[0]);
        sum[1] += c[1];
        sum[2] += c[2];
    }
    unsigned bad = wrong || sum[0] > (unsigned)a.total ? LS_DEVERR_LENGTH : 0u;
    if (a.ring && !bad) {
        const int64_t avail = given - taken;
        if (taken < 0 || avail < 0 || avail > a.ring_size || sum[1] > avail || sum[2] > a.ring_size - avail)
            bad = LS_DEVERR_FREE_LIST;
    }
    if (bad) sum[0] = sum[1] = sum[2] = 0u;
    __syncthreads();                                 // every wave has the counters and lengths (outputs may be the same memory)
    if (write_state && blockIdx.x == 0 && tid == 0) {
        if (bad) flag_error(a.err, bad);
        a.cu[0] = 0;
        if (a.ring) {
            a.next_counts[0] = taken + sum[1];
            a.next_counts[1] = given + sum[2];
        }
    }
    const int take0 = a.ring && !bad ? (int)(taken % a.ring_size) : 0, give0 = a.ring && !bad ? (int)(given % a.ring_size) : 0;
    const int64_t row0 = (int64_t)blockIdx.x * rows_per_wg, row1 = min(row0 + rows_per_wg, (int64_t)a.total);
    const int first_kept = (a.sinks + kBlock - 1) / kBlock;
    unsigned carry[3] = {0u, 0u, 0u};
    for (int s0 = 0;;) {
        const int s = s0 + tid;
        if (bad) t.n = 0;
        if (write_state && blockIdx.x == 0 && s < S) {
            if (a.reused) a.reused[s] = t.L;
            a.next_lens[s] = t.L + t.n;
            a.cu[s + 1] = bad ? 0 : (int)(carry[0] + before[0]) + t.n;
        }
        sm_cu[tid] = (int)(carry[0] + before[0]);
        sm_len[tid] = t.L;
        sm_take[tid] = carry[1] + before[1];
        sm_give[tid] = carry[2] + before[2];
        const int chunk_rows = (int)(carry[0] + all[0]);               // rows of the sessions up to this chunk's last
        if (tid == 0) sm_cu[kThreads] = chunk_rows;
        __syncthreads();
        // ---- this workgroup's rows of the chunk's sessions
        if (!bad)
            for (int64_t r = max(row0, (int64_t)carry[0]) + tid; r < min(row1, (int64_t)chunk_rows); r += kThreads) {
                int e = 0;                           // the row's session: the last one that starts at or before it
#pragma unroll
                for (int step = kThreads / 2; step > 0; step >>= 1)
                    if (sm_cu[e + step] <= r) e += step;
                const int L = sm_len[e], i = (int)r - sm_cu[e], pos = L + i, b0 = (L + kBlock - 1) / kBlock;
                int32_t *row = a.tables + (int64_t)(s0 + e) * a.max_blocks;
                // Id of the session's block j: taken in this step, or in the table.
                auto id_of = [&](int j) {
                    return a.ring && j >= b0
                               ? a.ring[ring_at(take0, (unsigned)ring_at((int)sm_take[e], (unsigned)(j - b0), a.ring_size), a.ring_size)]
                               : row[j];
                };
                auto inside = [&](int id) { return id >= 0 && id < a.num_blocks; };
                const int j = pos / kBlock, id = id_of(j);
                const bool ok = inside(id);
                a.slots[r] = ok ? (int64_t)id * kBlock + pos % kBlock : -1;
                if (a.ring && pos % kBlock == 0) row[j] = id;
                const int dead = a.ring ? dead_blocks(a, pos) : 0;
                int gone = 0;
                if (a.ring && dead_blocks(a, pos + 1) > dead) {
                    gone = id_of(first_kept + dead);
                    const unsigned k = sm_give[e] + (unsigned)(dead - dead_blocks(a, L));
                    a.ring[ring_at(give0, k, a.ring_size)] = gone;
                }
                if (!ok || !inside(gone)) flag_error(a.err, LS_DEVERR_BLOCK_ID);
            }
        carry[0] = add_rows(carry[0], all[0]);
        carry[1] += all[1];
        carry[2] += all[2];
        s0 += kThreads;
        if (s0 >= S) break;
        __syncthreads();
        scan(s0, t, before, all, wrong);
    }
    for (int64_t r = max(row0, (int64_t)sum[0]) + tid; r < row1; r += kThreads) a.slots[r] = -1;
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
    const bool small = num_sessions <= 256;
    const int threads = small ? 256 : 1024;
    auto launch = [&](int64_t grid, int rows, int state) {
        if (small) hipLaunchKernelGGL(tables_kernel<256>, dim3((unsigned)grid), dim3(256), 0, stream, a, rows, state);
        else hipLaunchKernelGGL(tables_kernel<1024>, dim3((unsigned)grid), dim3(1024), 0, stream, a, rows, state);
        return hipGetLastError();
    };
    if (total_tokens <= kTabRows * threads) return launch(1, total_tokens, 1);
    const bool same = next_lens == seq_lens || (free_ring && next_counts == free_counts);
    const hipError_t e = launch(((int64_t)total_tokens + threads - 1) / threads, threads, same ? 0 : 1);
    return e != hipSuccess || !same ? e : launch(1, 0, 1);
}

}  // namespace ls
