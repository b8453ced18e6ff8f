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
// blocks taken, blocks given), which every workgroup makes for itself, kPer
// consecutive sessions a thread.  A step moves a few KB, so the chain of latencies
// is what it costs (lengths, scan, ids, stores), and one pass over the lengths with
// a thread for each row is the shortest (256 sessions of one row: 3.6 us inside a
// graph, of which 2.5 are what any launch takes; 32 turns of 19817 rows in all: 4.4).
//
// write_state: lengths, prefix sums and counters are written, by workgroup 0.
// Where they are the inputs' own memory and there are other workgroups, which
// still read them, a launch of one workgroup without rows does that afterwards.
template <int kThreads, int kPer>
__global__ __launch_bounds__(kThreads) void tables_kernel(TablesArgs a, int rows_per_wg, int write_state) {
    constexpr int kWaves = kThreads / kWave;
    constexpr int kChunk = kThreads * kPer;       // sessions at a time
    __shared__ unsigned sm_scan[3][kWaves];
    __shared__ unsigned sm_bad[kWaves];
    __shared__ int sm_cu[kChunk], sm_len[kChunk];
    __shared__ unsigned sm_take[kChunk], sm_give[kChunk];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int S = a.num_sessions;
    int64_t taken = 0, given = 0;
    if (a.ring) {
        taken = a.counts[0];
        given = a.counts[1];
    }
    // Adds session s's step to v; false as session_step.
    auto add = [&](int s, SessionStep &t, unsigned (&v)[3]) {
        const bool ok = session_step(a, s, t);
        v[0] = add_rows(v[0], (unsigned)t.n);
        v[1] += t.need;
        v[2] += t.gives;
        return ok;
    };
    // Prefix sums of the threads' v: exclusive ones in `before`, totals in `all`; whether any thread's is wrong.
    auto scan = [&](const unsigned (&v)[3], bool wrong, unsigned (&before)[3], unsigned (&all)[3]) {
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
        // What the lanes before have: the difference, but for rows that have saturated
        // (the step is refused then, and no prefix sum used).
        before[0] = x[0] - v[0];
        before[1] = x[1] - v[1];
        before[2] = x[2] - v[2];
        if (lane == kWave - 1) {
#pragma unroll
            for (int k = 0; k < 3; ++k) sm_scan[k][wave] = x[k];
            sm_bad[wave] = any_wrong;
        }
        __syncthreads();
        unsigned is_bad = 0u;
        all[0] = all[1] = all[2] = 0u;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) {
                before[0] += all[0];
                before[1] += all[1];
                before[2] += all[2];
            }
            all[0] = add_rows(all[0], sm_scan[0][w]);
            all[1] += sm_scan[1][w];
            all[2] += sm_scan[2][w];
            is_bad |= sm_bad[w];
        }
        return is_bad != 0u;
    };
    SessionStep t[kPer];
    unsigned before[3], all[3];
    // The thread's sessions of the chunk from s0 on, and their sums.
    auto chunk = [&](int s0) {
        unsigned v[3] = {0u, 0u, 0u};
        bool wrong = false;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            t[k] = SessionStep{0, 0, 0u, 0u};
            if (s0 + tid * kPer + k < S && !add(s0 + tid * kPer + k, t[k], v)) wrong = true;
        }
        return scan(v, wrong, before, all);
    };
    bool wrong = chunk(0);
    // ---- totals: the step is refused as a whole when some length is out of
    // range, or rows, free blocks or the ring's room do not suffice.
    unsigned sum[3] = {all[0], all[1], all[2]};
    if (S > kChunk) {
        unsigned v[3] = {0u, 0u, 0u}, b[3], rest[3];
        bool w = false;
        for (int s = kChunk + tid; s < S; s += kThreads) {
            SessionStep u;
            if (!add(s, u, v)) w = true;
        }
        __syncthreads();                             // (the first chunk's sums are read)
        wrong = scan(v, w, b, rest) || wrong;
        sum[0] = add_rows(sum[0], rest[0]);
        sum[1] += rest[1];
        sum[2] += rest[2];
    }
    unsigned bad = wrong || sum[0] > (unsigned)a.total ? LS_DEVERR_LENGTH : 0u;
    if (a.ring && !bad) {
        const int64_t avail = given - taken;
        if (taken < 0 || avail < 0 || avail > a.ring_size || sum[1] > avail || sum[2] > a.ring_size - avail)
            bad = LS_DEVERR_FREE_LIST;
    }
    if (bad) sum[0] = sum[1] = sum[2] = 0u;
    const bool state = write_state && blockIdx.x == 0;
    __syncthreads();                                 // every wave has the counters and the chunk's lengths (outputs may be the same memory)
    if (state && tid == 0) {
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
        unsigned at[3] = {carry[0] + before[0], carry[1] + before[1], carry[2] + before[2]};
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int e = tid * kPer + k, s = s0 + e;
            if (bad) t[k].n = 0;
            if (state && s < S) {
                if (a.reused) a.reused[s] = t[k].L;
                a.next_lens[s] = t[k].L + t[k].n;
                a.cu[s + 1] = bad ? 0 : (int)at[0] + t[k].n;
            }
            sm_cu[e] = (int)at[0];
            sm_len[e] = t[k].L;
            sm_take[e] = at[1];
            sm_give[e] = at[2];
            at[0] += (unsigned)t[k].n;
            at[1] += t[k].need;
            at[2] += t[k].gives;
        }
        const int chunk_rows = (int)(carry[0] + all[0]);               // rows of the sessions up to this chunk's last
        __syncthreads();
        // ---- this workgroup's rows of the chunk's sessions
        if (!bad)
            for (int64_t r = max(row0, (int64_t)carry[0]) + tid; r < min(row1, (int64_t)chunk_rows); r += kThreads) {
                int e = 0;                           // the row's session: the last one that starts at or before it
#pragma unroll
                for (int step = kChunk / 2; step > 0; step >>= 1)
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
        s0 += kChunk;
        if (s0 >= S || (!state && carry[0] >= row1)) break;
        __syncthreads();
        chunk(s0);
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
    // Threads per workgroup, sessions per thread and workgroups (us inside a graph).
    // - State apart from the inputs: a thread per row, 256 in a workgroup, for more
    //   than 256 sessions 4 of them a thread (256 sessions of 4 rows 3.8, against 5.5
    //   when one workgroup does all rows; 1024 sessions of one row 4.9, against 5.7 in
    //   one workgroup of 1024 threads with a session each).  Past 1024 sessions 1024
    //   threads, so that up to 4096 make one pass (4096 sessions 9.8; 14.6 with 256 threads).
    // - State in place: the two launches that several workgroups take cost 6.9 (256
    //   sessions), 9.3 (1024) and 16.7 (2048), so one workgroup does the step while
    //   its rows are few: up to 512 with 256 threads (two rows of 256 sessions: 4.4,
    //   5.6 with 1024), up to 2048, or 4096 with many sessions, with 1024 (8 rows of
    //   256 sessions 6.9, 4 rows of 1024 sessions 8.8, a row of 2048 sessions 9.1).
    const bool same = next_lens == seq_lens || (free_ring && next_counts == free_counts);
    const bool many = num_sessions > 256, most = num_sessions > 1024;
    const bool one = same && total_tokens <= (many ? 4096 : 2048);
    const int threads = most || (one && (many || total_tokens > 512)) ? 1024 : 256;
    auto launch = [&](int64_t grid, int rows, int state) {
#define LS_TABLES(THREADS, PER) \
    hipLaunchKernelGGL((tables_kernel<THREADS, PER>), dim3((unsigned)grid), dim3(THREADS), 0, stream, a, rows, state)
        if (most) LS_TABLES(1024, 4);
        else if (threads == 1024) LS_TABLES(1024, 1);
        else if (many) LS_TABLES(256, 4);
        else LS_TABLES(256, 1);
#undef LS_TABLES
        return hipGetLastError();
    };
    if (one || total_tokens <= threads) return launch(1, total_tokens, 1);
    const hipError_t e = launch(((int64_t)total_tokens + threads - 1) / threads, threads, same ? 0 : 1);
    return e != hipSuccess || !same ? e : launch(1, 0, 1);
}

}  // namespace ls
