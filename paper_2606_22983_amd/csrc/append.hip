// KV append of a next turn's tokens (prefill over reused context, §5): write
// their K and V rows into their pool slots before attention reads them.  Slot
// of logical token t of session s: block block_tables[s][t / 16], offset
// t % 16; K tiles are chunk-major ([D/8][16 tokens][8 dims]), V tiles
// dim-major ([D][16 tokens]).  (The decode step's own token is written by the
// decode kernel.)
//
// And the append of rows by a slot map (kv_append): row i goes to slot
// slots[i] = block * 16 + offset, wherever the map says.
#include "common.h"

namespace ls {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kAppendThreads = 256;

// Workgroup (session s, j, KV head g) appends the turn's tokens of the pool
// blocks j, j + bps, ... that the turn touches (bps workgroups per session:
// normally one block each; a turn longer than max_new_len still gets every
// block).  Per block it writes 16-byte chunks.  A K chunk is 8 dims of one
// token, i.e. 16 contiguous bytes of that token's k_new row.  A V chunk is 8
// tokens of one dim, gathered from 8 rows through LDS.  The turn's first and
// last blocks may be shared with other tokens (the reused context before it,
// nothing after it): K chunks of other tokens are left alone, and a V chunk
// that mixes the turn's tokens with others is read, merged and written back
// (no other workgroup writes this tile in the launch).
template <int D>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(
    uint16_t *__restrict__ layer_pool, int64_t num_blocks, int32_t num_kv_heads,
    const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new,
    const int32_t *__restrict__ block_tables, int32_t max_blocks, const int32_t *__restrict__ cu,
    const int32_t *__restrict__ ctx, int32_t total_tokens, int32_t blocks_per_session, unsigned int *err,
    uint32_t *__restrict__ counters) {
    __shared__ __attribute__((aligned(16))) uint16_t sv[kBlock][D];
    const int s = blockIdx.x / blocks_per_session;
    const int j = blockIdx.x % blocks_per_session;
    const int g = blockIdx.y;
    const int tid = threadIdx.x;
    // The item counters of the prefill that follows on the stream: cleared here
    // rather than by a launch of their own, which costs ~4.5 us.
    if (counters && blockIdx.x == 0 && g == 0 && tid < kPrefillCounters) counters[tid] = 0u;
    const int c = ctx[s];
    const int n = cu[s + 1] - cu[s];
    // Nothing to append, or lengths that do not fit the token arrays (flagged by prefill).
    if (n <= 0 || c < 0 || cu[s] < 0 || cu[s + 1] > total_tokens) return;
    const int first = c / kBlock, last = (c + n - 1) / kBlock;
    constexpr int kChunks = D / 8 * kBlock;                     // 16-byte chunks per tile
    const int64_t tile = (int64_t)kBlock * D;
    for (int jb = first + j; jb <= last; jb += blocks_per_session) {
        if (jb >= max_blocks) {
            if (tid == 0) flag_error(err, LS_DEVERR_LENGTH);
            return;
        }
        const int32_t blk = block_tables[(int64_t)s * max_blocks + jb];
        if (blk < 0 || blk >= num_blocks) {
            if (tid == 0) flag_error(err, LS_DEVERR_BLOCK_ID);
            continue;
        }
        const int t_lo = max(c, jb * kBlock) - jb * kBlock;        // the turn's slots of this block: [t_lo, t_hi)
        const int t_hi = min(c + n, (jb + 1) * kBlock) - jb * kBlock;
        const int64_t row0 = (int64_t)cu[s] + (jb * kBlock - c);   // new-token index of slot 0 (may be negative)
        uint16_t *ktile = layer_pool + ((int64_t)blk * 2 * num_kv_heads + g) * tile;
        uint16_t *vtile = ktile + (int64_t)num_kv_heads * tile;

        // K: chunk ci = (dim chunk ci / 16, token ci % 16), contiguous across threads.
        for (int ci = tid; ci < kChunks; ci += kAppendThreads) {
            const int t = ci % kBlock;
            if (t < t_lo || t >= t_hi) continue;
            const u32x4 v =
                *reinterpret_cast<const u32x4 *>(k_new + ((row0 + t) * num_kv_heads + g) * D + (ci / kBlock) * 8);
            *reinterpret_cast<u32x4 *>(ktile + ci * 8) = v;
        }
        // V: the block's rows into LDS, then chunk ci = (dim ci / 2, tokens 8 * (ci % 2) ..).
        __syncthreads();                                        // the previous block's LDS reads are done
        for (int ci = tid; ci < kChunks; ci += kAppendThreads) {
            const int t = ci / (D / 8), d8 = ci % (D / 8);
            if (t < t_lo || t >= t_hi) continue;
            *reinterpret_cast<u32x4 *>(&sv[t][d8 * 8]) =
                *reinterpret_cast<const u32x4 *>(v_new + ((row0 + t) * num_kv_heads + g) * D + d8 * 8);
        }
        __syncthreads();
        for (int ci = tid; ci < 2 * D; ci += kAppendThreads) {
            const int d = ci / 2, t0 = (ci % 2) * 8;
            const int lo = max(t_lo, t0), hi = min(t_hi, t0 + 8);
            if (lo >= hi) continue;
            u32x4 *dst = reinterpret_cast<u32x4 *>(vtile + (int64_t)d * kBlock + t0);
            u32x4 w = (lo == t0 && hi == t0 + 8) ? u32x4{0u, 0u, 0u, 0u} : *dst;
            for (int t = lo; t < hi; ++t) {
                const uint32_t half = sv[t][d];
                const int k = (t - t0) >> 1, sh = ((t - t0) & 1) * 16;
                w[k] = (w[k] & ~(0xFFFFu << sh)) | (half << sh);
            }
            *dst = w;
        }
    }
}

// Workgroup (kRows consecutive rows, KV head).  Bound by bandwidth when there are
// many rows, each read and written once (19817 rows of 4 heads x 128 dims, 162 MB:
// 28.8 us or 5.64 TB/s while half of it stays cached, 45 us or 3.6 TB/s from HBM;
// 6.17 is what a plain read and write of as much reaches), by latency when there
// are few (2.6 us inside a graph for one row, 3.4 for 256 lone slots of 2 heads).  K goes straight
// from registers to its tile: a wave moves up to 16 rows x 4 chunks of 16 bytes, so
// that consecutive slots make 256 contiguous bytes.  V is turned through LDS: a
// slot's values lie 32 bytes apart in the dim-major tile, and only with the
// neighbouring slots at hand do they make whole 16-byte stores.  The rows are
// therefore cut into segments, of consecutive rows in consecutive slots of one
// block, and a segment belongs to the workgroup that holds its first row, which
// reads up to 15 rows of the next workgroup's for it (which then skips them):
// any order of slots is served, runs of a session's tokens by whole 32-byte
// lines.  Half segments shorter than 8 slots are stored value by value; a read,
// a merge and a wider write would race with other calls' slots of the block.
constexpr int kAppendAhead = 15;                  // rows past its own that a workgroup may read

template <int D, int kRows>
__global__ __launch_bounds__(kAppendThreads) void append_slots_kernel(
    uint16_t *__restrict__ layer_pool, int64_t num_blocks, int32_t num_kv_heads, const uint16_t *__restrict__ k_new,
    const uint16_t *__restrict__ v_new, int64_t k_stride, int64_t v_stride, const int64_t *__restrict__ slots,
    int32_t total, unsigned int *err) {
    static_assert(kRows + kAppendAhead < kWave, "a lane per row, and the row that ends the last segment");
    constexpr int kRun = kRows < kBlock ? kRows : kBlock;       // rows whose chunks a K store interleaves
    static_assert(kRows % kRun == 0, "whole runs");
    constexpr int kChunks = D / 8;                              // 16-byte chunks of a row
    constexpr int kPitch = D + 8;                               // (16 bytes of padding: a column's two halves in distinct banks)
    __shared__ __attribute__((aligned(16))) uint16_t sv[kRows + kAppendAhead][kPitch];
    __shared__ int64_t sm_slot[kWave];                          // -1: left out
    __shared__ int64_t sm_tile[kRows];                          // segments: V tile (elements from block 0's),
    __shared__ uint32_t sm_segment[kRows];                      // first row | first slot << 8 | rows << 16
    __shared__ int sm_segments, sm_begin, sm_end;               // rows [begin, end) are in segments that start here
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int g = blockIdx.y;
    const int64_t row0 = (int64_t)blockIdx.x * kRows;
    const int rows = (int)min((int64_t)kRows + kAppendAhead, total - row0);      // rows there are to look at
    // K rows, and with few rows, where latency counts, V rows too, are requested
    // before the slots are known.
    auto k_row = [&](int c) { return c % kRun + c / (kRun * kChunks) * kRun; };
    auto k_chunk = [&](int c) { return c / kRun % kChunks; };
    constexpr int kLoadsK = (kRows * kChunks + kAppendThreads - 1) / kAppendThreads;
    constexpr bool kEarly = kRows <= kBlock;
    u32x4 kreg[kLoadsK], vreg[kEarly ? kLoadsK : 1];
#pragma unroll
    for (int i = 0; i < kLoadsK; ++i) {
        const int c = tid + i * kAppendThreads, r = min(k_row(c), rows - 1);
        if (kRows * kChunks % kAppendThreads == 0 || c < kRows * kChunks)
            kreg[i] = *reinterpret_cast<const u32x4 *>(k_new + (row0 + r) * k_stride + g * D + k_chunk(c) * 8);
    }
    if constexpr (kEarly)
#pragma unroll
        for (int i = 0; i < kLoadsK; ++i) {
            const int c = tid + i * kAppendThreads, r = min(c / kChunks, rows - 1);
            if (kRows * kChunks % kAppendThreads == 0 || c < kRows * kChunks)
                vreg[i] = *reinterpret_cast<const u32x4 *>(v_new + (row0 + r) * v_stride + g * D + c % kChunks * 8);
        }
    if (wave == 0) {
        const int64_t raw = lane < rows ? slots[row0 + lane] : -1;
        const bool past = raw >= num_blocks * kBlock;
        if (past && lane < kRows && g == 0) flag_error(err, LS_DEVERR_BLOCK_ID);
        const int64_t slot = past ? -1 : raw;
        int64_t before = __shfl_up(slot, 1);
        if (lane == 0) before = row0 > 0 ? slots[row0 - 1] : -1;
        // (a row left out counts as a first row, and is dropped from the list)
        const bool first = slot < 0 || before < 0 || slot != before + 1 || slot % kBlock == 0;
        const uint64_t firsts = __ballot(first);
        const uint64_t mine = __ballot(first && slot >= 0 && lane < kRows);
        if ((mine >> lane) & 1) {
            const int k = __popcll(mine & ((1ull << lane) - 1));
            const uint32_t n = (uint32_t)__builtin_ctzll(firsts >> (lane + 1)) + 1;      // (the lanes past the rows are firsts)
            sm_segment[k] = (uint32_t)lane | (uint32_t)(slot % kBlock) << 8 | n << 16;
            sm_tile[k] = ((slot / kBlock) * 2 + 1) * num_kv_heads * (kBlock * D);
        }
        sm_slot[lane] = slot;
        if (lane == 0) {
            const int last = mine ? 63 - __builtin_clzll(mine) : 0;
            sm_segments = __popcll(mine);
            sm_begin = mine ? __builtin_ctzll(mine) : 0;
            sm_end = mine ? last + 1 + __builtin_ctzll(firsts >> (last + 1)) : 0;
        }
    }
    __syncthreads();
    const int begin = sm_begin, end = sm_end, segments = sm_segments;
    const int64_t tile = (int64_t)kBlock * D;
    uint16_t *const head = layer_pool + g * tile;               // K tile of block 0
    // ---- V rows to LDS
    if constexpr (kEarly)
#pragma unroll
        for (int i = 0; i < kLoadsK; ++i) {
            const int c = tid + i * kAppendThreads;
            if (c < kRows * kChunks) *reinterpret_cast<u32x4 *>(&sv[c / kChunks][c % kChunks * 8]) = vreg[i];
        }
    for (int c = tid + (kEarly ? kRows * kChunks : 0); c < (kRows + kAppendAhead) * kChunks; c += kAppendThreads) {
        const int r = c / kChunks, d8 = c % kChunks;
        if (r >= begin && r < end)
            *reinterpret_cast<u32x4 *>(&sv[r][d8 * 8]) =
                *reinterpret_cast<const u32x4 *>(v_new + (row0 + r) * v_stride + g * D + d8 * 8);
    }
    // ---- K
#pragma unroll
    for (int i = 0; i < kLoadsK; ++i) {
        const int c = tid + i * kAppendThreads;
        if (c >= kRows * kChunks) break;
        const int64_t slot = sm_slot[k_row(c)];
        if (slot < 0) continue;
        uint16_t *ktile = head + (slot / kBlock) * 2 * num_kv_heads * tile;
        *reinterpret_cast<u32x4 *>(ktile + (k_chunk(c) * kBlock + slot % kBlock) * 8) = kreg[i];
    }
    __syncthreads();
    // ---- V: a thread has one dim of every (kAppendThreads / D)-th segment.
    const int d = tid % D;
    for (int k = tid / D; k < segments; k += kAppendThreads / D) {
        const uint32_t seg = sm_segment[k];
        uint16_t *dst = head + sm_tile[k] + d * kBlock;
        const int o = (int)(seg >> 8) & 0xFF, end_slot = o + (int)(seg >> 16);
        const uint16_t *src = &sv[seg & 0xFF][d] - o * kPitch;  // slot t's value: src[t * kPitch]
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int lo = max(o, half * 8), hi = min(end_slot, half * 8 + 8);
            if (hi - lo == 8) {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] = src[(half * 8 + 2 * e) * kPitch] | (uint32_t)src[(half * 8 + 2 * e + 1) * kPitch] << 16;
                *reinterpret_cast<u32x4 *>(dst + half * 8) = w;
            } else {
                for (int t = lo; t < hi; ++t) dst[t] = src[t * kPitch];
            }
        }
    }
}

}  // namespace

hipError_t launch_append_slots(const PoolGeom &p, int layer, int32_t total_tokens, const uint16_t *k_new,
                               const uint16_t *v_new, int64_t k_stride, int64_t v_stride, const int64_t *slot_map,
                               unsigned int *err, hipStream_t stream) {
    // Rows per workgroup by how many workgroups that leaves each CU (us inside a
    // graph, 128 dims, 2 KV heads).  Fewer than one of 16 rows: 4, since a slot
    // without its neighbours costs 128 narrow stores, which then spread over more
    // CUs (256 lone slots 3.4 against 4.6; runs of 16 slots the same, 2.9).  From 8 of
    // 48 rows on, 48: less of what the next workgroup's segments need is read twice
    // (65536 rows 21.2 against 21.9); below, 16 (32768 rows 12.1 either way, 16384 rows 6.5 against 7.8).
    const int64_t cus = p.num_cus > 0 ? p.num_cus : 256;
    auto groups = [&](int rows) { return ((int64_t)total_tokens + rows - 1) / rows * p.num_kv_heads; };
    const int rows = groups(48) >= 8 * cus ? 48 : groups(16) >= cus ? 16 : 4;
    const dim3 grid((unsigned)(groups(rows) / p.num_kv_heads), (unsigned)p.num_kv_heads);
#define LS_APPEND(DD, ROWS) \
    hipLaunchKernelGGL((append_slots_kernel<DD, ROWS>), grid, dim3(kAppendThreads), 0, stream, p.layer_base(layer), \
                       p.num_blocks, p.num_kv_heads, k_new, v_new, k_stride, v_stride, slot_map, total_tokens, err)
    if (p.head_dim == 128) {
        if (rows == 48) LS_APPEND(128, 48);
        else if (rows == 16) LS_APPEND(128, 16);
        else LS_APPEND(128, 4);
    } else {
        if (rows == 48) LS_APPEND(64, 48);
        else if (rows == 16) LS_APPEND(64, 16);
        else LS_APPEND(64, 4);
    }
#undef LS_APPEND
    return hipGetLastError();
}

hipError_t launch_append_prefill(const PoolGeom &p, int layer, int32_t num_sessions, int32_t total_tokens,
                                 int32_t max_new_len, const uint16_t *k_new, const uint16_t *v_new,
                                 const int32_t *cu_new_lens, const int32_t *reused_lens,
                                 const int32_t *block_tables, int32_t max_blocks, uint32_t *counters,
                                 unsigned int *err, hipStream_t stream) {
    if (num_sessions <= 0 || max_new_len <= 0) return hipSuccess;
    // A turn of n tokens touches at most (n + 15) / 16 + 1 blocks (one more
    // when it starts inside a block).
    const int32_t bps = (max_new_len + kBlock - 1) / kBlock + 1;
    const int64_t grid = (int64_t)num_sessions * bps;
    if (grid > 0x7FFFFFFFLL) return hipErrorInvalidConfiguration;
    const dim3 g((unsigned)grid, (unsigned)p.num_kv_heads);
    if (p.head_dim == 128)
        hipLaunchKernelGGL(append_kernel<128>, g, dim3(kAppendThreads), 0, stream, p.layer_base(layer),
                           p.num_blocks, p.num_kv_heads, k_new, v_new, block_tables, max_blocks, cu_new_lens,
                           reused_lens, total_tokens, bps, err, counters);
    else
        hipLaunchKernelGGL(append_kernel<64>, g, dim3(kAppendThreads), 0, stream, p.layer_base(layer),
                           p.num_blocks, p.num_kv_heads, k_new, v_new, block_tables, max_blocks, cu_new_lens,
                           reused_lens, total_tokens, bps, err, counters);
    return hipGetLastError();
}

}  // namespace ls
