// Accumulated attention weights of a turn: what the last rows of the turn's queries
// attend to (next-turn prefill over reused context, §5, §3), summed per key and KV
// head, so that an eviction can tell the keys that later tokens will use.
//
// With rows i at positions p_i of the observed queries of one KV head (tokens times
// query heads) and scores x_it = scale q_i.k_t for t <= p_i,
//   w_t += sum_i e^(x_it - m_i) / l_i,   m_i = max_t x_it,   l_i = sum_t e^(x_it - m_i).
// l is known only after all keys, so the scores are computed twice, from K alone (V is
// not read), in three launches:
//   rows    (m, l) of each row over each chunk of keys
//   sums    their sum over the chunks, as m and 1 / l
//   keys    e^(x - m) / l summed over the rows, added to the weights
// The exponential is that of fma(product, scale, -round(m scale)), one operation: what m loses
// by rounding is in p and in l, and cancels (RowScale).  (With log2(l) + m as one word a score of 2^14
// put a weight off by 2^-10.  Subtracting products before the scale takes an operation a score more: 283
// us for the batch below where this takes 272, and the one word took 270.)
// A wave keeps the K tiles of its blocks in registers, as the A operand of
// S^T[16 tokens x 16 rows] = K . Q^T, and walks over the rows 16 at a time, so K is
// read once a launch however many rows there are, and the rows (a few hundred KB)
// come from L2.  A lane's scores belong to one row (lane % 16): sums over keys end
// with two lane exchanges, sums over rows stay in the lane until the last row.
// Bound by the matrix and exponential units when rows are many, by latency when few.
// Measured: 32 turns, 64 observed rows each over up to 8192 tokens, 32 / 4 heads of 128, 272
// to 285 us a call, as cards differ (rows' launch 158, keys' 137 at best; 720-755 TFLOP/s of
// products); one turn, 32 rows over 2090 tokens, 20 us (8.5, 4.5 and 6.5).  Wider waves (8 blocks,
// 301 us), a persistent grid (368) and four waves a SIMD (289) were slower than the 264 they were
// compared with.
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace ls {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kObThreads = 256;
constexpr int kObWaves = kObThreads / kWave;
constexpr int kObRows = 1024;                // rows of a KV head at a time (the workspace); more take another round
constexpr float kNoMax = -0x1.fffffep127f;   // maximum of no key: no finite product is below it
constexpr int kRawBuffer = 0x00020000;

struct ObserveArgs {
    const uint16_t *pool;          // layer base
    int64_t num_blocks;
    int32_t num_kv_heads, group;
    const uint16_t *q;             // [T][Hq][D]
    const int32_t *cu;             // [S + 1]
    const int32_t *reused;         // [S]
    int32_t num_sessions, total, max_new;
    const int32_t *tables;         // [S][max_blocks]
    int32_t max_blocks;
    int32_t rows;                  // observed tokens of a turn
    float scale_log2;
    int32_t row0;                  // first row of the round
    int32_t row_cap;               // rows of the round, at most
    int32_t chunks;                // chunks of a table, at most
    float2 *part;                  // [S][Hkv][chunks][row_cap] (m, l), m before scaling
    f32x4 *whole;                  // [S][Hkv][row_cap] (round(m scale), scale, 1 / l) over all keys
    float *weights;                // layer base, [num_blocks][Hkv][16]
    int32_t *positions;
    const int32_t *begin;          // [S] or null
    const int32_t *first;          // [S] or null
    unsigned int *err;
};

// A session's turn.
struct Turn {
    int q0;                        // row of q of its first token
    int n, c;                      // new tokens, tokens before (0 and 0: not a turn that can be)
    int j0;                        // first observed token
    int rows;                      // rows of the round (tokens x group)
};

__device__ __forceinline__ Turn turn_of(const ObserveArgs &a, int s, bool may_flag) {
    Turn t;
    t.q0 = a.cu[s];
    t.n = a.cu[s + 1] - t.q0;
    t.c = a.reused[s];
    if (t.q0 < 0 || t.n < 0 || t.n > a.max_new || t.n > a.total - t.q0 || t.c < 0 || (int64_t)t.c + t.n > (int64_t)a.max_blocks * kBlock) {
        if (may_flag) flag_error(a.err, LS_DEVERR_LENGTH);
        t.q0 = t.n = t.c = 0;
    }
    t.j0 = max(t.n - a.rows, 0);
    t.rows = min(max((t.n - t.j0) * a.group - a.row0, 0), a.row_cap);
    return t;
}

__device__ __forceinline__ float max_xor_16_32(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_xor_16_32(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The scale (log2) that a row with the largest product m takes, and m scale rounded.  The largest score's
// exponential is 2^rounding, where it would be 1 with an exact m scale: half a step of m scale.  It stays
// within 2^64 because a row whose m scale passes 2^31 takes a scale smaller by a power of two, with |m scale|
// in [2^29, 2^31).  Its fp32 products, where they differ, are then still 2^5 apart, a share of 2^-32 (and
// twice that or more with the whole scale).
struct RowScale {
    float scale, m, rounding;
    __device__ __forceinline__ RowScale(float product, float scale_log2) {
        // (exponents apart: the product of the two may be past the largest number.  The biased one of 0 is the least.)
        const int e = (int)(__float_as_uint(product) >> 23 & 255u) - 126 + __builtin_amdgcn_frexp_expf(scale_log2);
        scale = __builtin_amdgcn_ldexpf(scale_log2, min(31 - e, 0));
        m = product * scale;
        rounding = __builtin_fmaf(product, scale, -m);
    }
};

typedef __attribute__((address_space(3))) void lds_void;

// Four tiles of 16 rows, one loaded by each wave: a tile's k-step is a kilobyte, in the
// order of the lanes that take it as the B operand.
template <int D>
struct RowStage {
    __attribute__((aligned(1024))) uint8_t q[kObWaves][D / 32][1024];
};
struct SumStage {
    __attribute__((aligned(1024))) f32x4 row[kObWaves][kWave];      // lane: its row's
};

// One chunk of kObWaves * KB blocks of a (session, KV head); wave w has blocks
// w KB .. w KB + KB - 1 of it.  kKeys false: the rows' launch, true: the keys'.
//
// The rows come through LDS, four tiles a stage, loaded a stage ahead (each wave
// reading its rows from L2 one tile ahead took longer: a tile takes some 400 cycles, a
// load up to 4000 when all CUs read).  One barrier a stage publishes the next one and
// frees the one before.
template <int D, int KB, bool kKeys>
__global__ __launch_bounds__(kObThreads, 3) void observe_kernel(ObserveArgs a) {
    // (arrays of their own: reads of one stage do not wait for the loads of another)
    __shared__ RowStage<D> sq0, sq1;
    __shared__ SumStage sl0, sl1;
    __shared__ float2 sm[3][kObWaves][kObWaves * 16];      // (m, l) of a stage's rows, by wave
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, c16 = lane % 16, g4 = lane / 16;
    const int H = a.num_kv_heads, G = a.group;
    // (A session's chunks are spread over the XCDs: rows are few, and lengths differ.)
    const int chunk = blockIdx.x, h = blockIdx.y, s = blockIdx.z;
    const Turn t = turn_of(a, s, kKeys && chunk == 0 && h == 0 && a.row0 == 0);
    const int keys = t.c + t.n, col0 = (chunk * kObWaves + wave) * KB;
    if (t.n == 0 || (a.row0 && !t.rows) || chunk * kObWaves * KB * kBlock >= keys) return;
    const int64_t pair = (int64_t)s * H + h;
    const int p0 = t.c + t.j0;                     // position of the first observed token
    const int gs = __builtin_ctz(G);               // (G is 1, 2, 4 or 8)
    // Rows before this one see none of the chunk's keys.
    const int unseen = max(chunk * kObWaves * KB * kBlock - p0, 0) * G - a.row0;
    const int tile0 = max(unseen, 0) / 16, tiles = (t.rows + 15) / 16;
    // ---- the wave's K tiles (ids: lane b has block b's; -1: no key or not in the pool)
    bf16x8 k[KB][D / 32];
    int ids = -1;
    if (lane < KB && (col0 + lane) * kBlock < keys) {
        ids = a.tables[(int64_t)s * a.max_blocks + col0 + lane];
        if (ids < 0 || ids >= a.num_blocks) {
            if (kKeys) flag_error(a.err, LS_DEVERR_BLOCK_ID);
            ids = -1;
        }
    }
    int id[KB];
    bool absent = false;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
        id[b] = __builtin_amdgcn_readlane(ids, b);
        absent = absent || id[b] < 0;
        const uint16_t *kt = a.pool + ((int64_t)max(id[b], 0) * 2 * H + h) * (kBlock * D);
        const __amdgpu_buffer_rsrc_t rk =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(kt), 0, id[b] < 0 ? 0 : kBlock * D * 2, kRawBuffer);
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
            k[b][ks] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rk, lane * 16, ks * 4 * kBlock * 16, 0));
    }
    const int wkey0 = col0 * kBlock;               // the wave's first key
    float sum[kKeys ? KB : 1][4] = {};
    // ---- the rows.  (The round's first row is a token's first: row0 is a multiple of 1024.)
    const __amdgpu_buffer_rsrc_t rq = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(a.q + ((int64_t)(t.q0 + t.j0 + (a.row0 >> gs)) * H + h) * G * D), 0, INT32_MAX, kRawBuffer);
    const __amdgpu_buffer_rsrc_t rl =
        __builtin_amdgcn_make_buffer_rsrc(a.whole + pair * a.row_cap, 0, kKeys ? INT32_MAX : 0, kRawBuffer);
    // Lanes of no row, and stages behind the last, read the last row.
    auto load_stage = [&](RowStage<D> &sq, SumStage &sl, int tile_first) {
        const int row = min((tile_first + wave) * 16 + c16, t.rows - 1);
        const int off = ((row >> gs) * (H * G) + (row & (G - 1))) * (D * 2) + g4 * 16;
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (lds_void *)sq.q[wave][ks], 16, off + ks * 64, 0, 0, 0);
        if constexpr (kKeys) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rl, (lds_void *)sl.row[wave], 16, row * 16, 0, 0, 0);
        }
    };
    auto stage_barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);        // vmcnt(0) lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // ---- products of a tile, and what is made of them (by the rows' launch one tile later, in the
    // same code: the matrix unit has the next tile's while the vector unit has this one's)
    f32x4 acc[2][KB];
    f32x4 whole = {};
    auto products = [&](const RowStage<D> &sq, const SumStage &sl, int i, f32x4 (&to)[KB]) {
        if constexpr (kKeys) whole = sl.row[i][lane];
        bf16x8 q[D / 32];
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) q[ks] = *reinterpret_cast<const bf16x8 *>(&sq.q[i][ks][lane * 16]);
#pragma unroll
        for (int b = 0; b < KB; ++b) to[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
            for (int b = 0; b < KB; ++b) to[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[b][ks], q[ks], to[b], 0, 0, 0);
    };
    // Some row of the tile does not see every key of the wave.  (A branch around code of its
    // own: as selects in the common code the masks cost as much as the sums.)
    auto is_partial = [&](int tile) { return p0 + ((a.row0 + tile * 16) >> gs) < wkey0 + KB * kBlock - 1 || absent; };
    auto consume = [&](const f32x4 (&of)[KB], int tile, auto partial) {
        const int row = tile * 16 + c16, pos = p0 + ((a.row0 + row) >> gs);
        auto unseen = [&](int b, int e) {
            return decltype(partial)::value && (wkey0 + b * kBlock + 4 * g4 + e > pos || id[b] < 0);
        };
        float x[KB][4];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[b][e] = unseen(b, e) ? -INFINITY : of[b][e];
        if constexpr (kKeys) {
            const float inv = row < t.rows ? whole.z : 0.f;    // (no row: no weight)
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][e], whole.y, -whole.x));
                    // (unseen: 0, also of a row whose sum is no number)
                    sum[b][e] = unseen(b, e) ? sum[b][e] : __builtin_fmaf(p, inv, sum[b][e]);
                }
        } else {
            float m = kNoMax, l = 0.f;
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, x[b][e]);
            // (the scale is positive: the largest product has the largest score)
            m = max_xor_16_32(m);
            const RowScale rs(m, a.scale_log2);
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) l += __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][e], rs.scale, -rs.m));
            l = sum_xor_16_32(l);
            const int n = tile - tile0;
            if (g4 == 0) sm[n / kObWaves % 3][wave][n % kObWaves * 16 + c16] = make_float2(m, l);
        }
    };
    float2 *part = a.part + (pair * a.chunks + chunk) * a.row_cap;
    if constexpr (!kKeys)
        for (int row = tid; row < min(tile0 * 16, t.rows); row += kObThreads) part[row] = make_float2(kNoMax, 0.f);
    const int count = tiles - tile0, stages = (count + kObWaves - 1) / kObWaves;
    // The rows of a finished stage over the waves' keys, by one wave.
    auto store_rows = [&](int st) {
        const int row = (tile0 + st * kObWaves) * 16 + lane;
        if (kKeys || wave != st % kObWaves || row >= t.rows) return;
        float m = kNoMax, l = 0.f;
#pragma unroll
        for (int w = 0; w < kObWaves; ++w) m = fmaxf(m, sm[st % 3][w][lane].x);
#pragma unroll
        for (int w = 0; w < kObWaves; ++w) {
            const float2 of = sm[st % 3][w][lane];
            l += __builtin_amdgcn_exp2f((of.x - m) * a.scale_log2 - RowScale(of.x, a.scale_log2).rounding) * of.y;
        }
        part[row] = make_float2(m, l);
    };
    auto stage = [&](int st, RowStage<D> &sq, SumStage &sl, RowStage<D> &ahead_q, SumStage &ahead_l) {
        load_stage(ahead_q, ahead_l, tile0 + (st + 1) * kObWaves);
        if (st >= 2) store_rows(st - 2);           // (its last tile was finished in stage st - 1)
#pragma unroll
        for (int i = 0; i < kObWaves; ++i) {
            const int n = st * kObWaves + i;
            if (n >= count) break;
            if constexpr (kKeys) {
                // (at once: the sums take the registers that a tile's products would wait in, and a
                // third wave per SIMD gives as much: 152 us for the next-turn batch, 174 one later)
                products(sq, sl, i, acc[0]);
                if (is_partial(tile0 + n)) consume(acc[0], tile0 + n, std::true_type());
                else consume(acc[0], tile0 + n, std::false_type());
            } else if (n == 0) {
                products(sq, sl, i, acc[i & 1]);
            } else if (is_partial(tile0 + n - 1)) {
                products(sq, sl, i, acc[i & 1]);
                consume(acc[(i + 1) & 1], tile0 + n - 1, std::true_type());
            } else {
                products(sq, sl, i, acc[i & 1]);
                consume(acc[(i + 1) & 1], tile0 + n - 1, std::false_type());
            }
        }
        stage_barrier();
    };
    if (count > 0) {
        load_stage(sq0, sl0, tile0);
        stage_barrier();
        for (int st = 0;;) {
            stage(st, sq0, sl0, sq1, sl1);
            if (++st >= stages) break;
            stage(st, sq1, sl1, sq0, sl0);
            if (++st >= stages) break;
        }
        if constexpr (!kKeys) {
            if (count & 1) consume(acc[0], tiles - 1, std::true_type());
            else consume(acc[1], tiles - 1, std::true_type());
            __syncthreads();
            if (stages >= 2) store_rows(stages - 2);
            store_rows(stages - 1);
        }
    }
    if constexpr (kKeys) {
        // ---- sums over the 16 rows' lanes; lane 16 g4 + b has the wave's block b
        const int first = a.first ? a.first[s] : 0, begin = a.begin ? a.begin[s] : t.c;
#pragma unroll
        for (int b = 0; b < KB; ++b) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int off = 1; off < 16; off <<= 1) sum[b][e] += __shfl_xor(sum[b][e], off);
            if (c16 == b && id[b] >= 0) {
                const int64_t at = ((int64_t)id[b] * H + h) * kBlock + 4 * g4;
                const f32x4 was = *reinterpret_cast<const f32x4 *>(a.weights + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = wkey0 + b * kBlock + 4 * g4 + e;
                    if (key < first || key >= keys) continue;
                    const bool fresh = key >= t.c && a.row0 == 0;
                    a.weights[at + e] = fresh ? sum[b][e] : was[e] + sum[b][e];
                    if (fresh) a.positions[at + e] = begin + (key - t.c);
                }
            }
        }
    }
}

// What the keys' launch takes of each row.
__global__ __launch_bounds__(kObThreads) void observe_sum_kernel(ObserveArgs a, int chunk_tokens) {
    const int h = blockIdx.y, s = blockIdx.z, row = blockIdx.x * kObThreads + threadIdx.x;
    const Turn t = turn_of(a, s, false);
    if (row >= t.rows) return;
    const int64_t pair = (int64_t)s * a.num_kv_heads + h;
    const int pos = t.c + t.j0 + (a.row0 + row) / a.group, chunks = pos / chunk_tokens + 1;
    const float2 *p = a.part + pair * a.chunks * a.row_cap + row;
    // (eight chunks at a time, so that their loads are in flight together)
    float m = kNoMax, l = 0.f;
    for (int k0 = 0; k0 < chunks; k0 += 8) {
        float2 v[8];
        float now = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[(int64_t)min(k0 + i, chunks - 1) * a.row_cap];
#pragma unroll
        for (int i = 0; i < 8; ++i) now = fmaxf(now, v[i].x);
        l *= __builtin_amdgcn_exp2f((m - now) * a.scale_log2);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k0 + i < chunks) l += __builtin_amdgcn_exp2f((v[i].x - now) * a.scale_log2) * v[i].y;
        m = now;
    }
    // (a row without a key, all of its blocks absent: no weight)
    const RowScale rs(m, a.scale_log2);
    a.whole[pair * a.row_cap + row] = f32x4{rs.m, rs.scale, l > 0.f || l != l ? __builtin_amdgcn_exp2f(-rs.rounding) / l : 0.f, 0.f};
}

template <int D, int KB>
hipError_t launch_observe_t(ObserveArgs a, int32_t whole_rows, hipStream_t stream) {
    constexpr int kChunkTokens = kObWaves * KB * kBlock;
    const dim3 grid((unsigned)a.chunks, (unsigned)a.num_kv_heads, (unsigned)a.num_sessions);
    for (a.row0 = 0; a.row0 < whole_rows; a.row0 += a.row_cap) {
        hipLaunchKernelGGL((observe_kernel<D, KB, false>), grid, dim3(kObThreads), 0, stream, a);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL(observe_sum_kernel, dim3((unsigned)((a.row_cap + kObThreads - 1) / kObThreads), (unsigned)a.num_kv_heads, (unsigned)a.num_sessions),
                           dim3(kObThreads), 0, stream, a, kChunkTokens);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL((observe_kernel<D, KB, true>), grid, dim3(kObThreads), 0, stream, a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

constexpr size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

ObservePlan plan_observe(const PoolGeom &p, int32_t num_sessions, int32_t num_q_heads, int32_t max_new_len, int32_t rows,
                         int32_t max_blocks) {
    const int64_t G = num_q_heads / p.num_kv_heads, pairs = (int64_t)num_sessions * p.num_kv_heads;
    const int64_t cus = p.num_cus > 0 ? p.num_cus : 256;
    ObservePlan o;
    // (a turn fits its table)
    o.whole_rows = (int32_t)(std::min({(int64_t)rows, (int64_t)max_new_len, (int64_t)max_blocks * kBlock}) * G);
    o.row_cap = std::min(o.whole_rows, kObRows);
    // Blocks per wave: as many as leave every CU two workgroups, if the sessions fill their tables (their
    // lengths are on the device).  In tables of 1024 columns the one turn above takes 26 us for 20, eight first
    // turns of up to 700 tokens (all rows, 8 heads of 64) 110 for 29, the 32 turns 340 for 281 on one card.
    o.blocks = 4;
    while (o.blocks > 1 && pairs * ((max_blocks + kObWaves * o.blocks - 1) / (kObWaves * o.blocks)) < 2 * cus) o.blocks /= 2;
    o.chunks = (max_blocks + kObWaves * o.blocks - 1) / (kObWaves * o.blocks);
    o.whole_at = align256((size_t)pairs * (size_t)o.chunks * (size_t)o.row_cap * sizeof(float2));
    o.total = o.whole_at + align256((size_t)pairs * (size_t)o.row_cap * sizeof(f32x4));
    return o;
}

hipError_t launch_observe(const PoolGeom &p, int layer, int32_t num_sessions, int32_t num_q_heads, const ObserveCall &c,
                          const ObservePlan &plan, unsigned int *err, hipStream_t stream) {
    uint8_t *ws = static_cast<uint8_t *>(c.workspace);
    const int64_t entries = (int64_t)layer * p.num_blocks * p.num_kv_heads * kBlock;
    ObserveArgs a = {};
    a.pool = p.layer_base(layer);
    a.num_blocks = p.num_blocks;
    a.num_kv_heads = p.num_kv_heads;
    a.group = num_q_heads / p.num_kv_heads;
    a.q = c.q;
    a.cu = c.cu_new_lens;
    a.reused = c.reused_lens;
    a.num_sessions = num_sessions;
    a.total = c.total_new_tokens;
    a.max_new = c.max_new_len;
    a.tables = c.block_tables;
    a.max_blocks = c.max_blocks;
    a.rows = c.rows;
    a.scale_log2 = c.scale * 1.4426950408889634f;
    a.row_cap = plan.row_cap;
    a.chunks = plan.chunks;
    a.part = reinterpret_cast<float2 *>(ws);
    a.whole = reinterpret_cast<f32x4 *>(ws + plan.whole_at);
    a.weights = c.weights + entries;
    a.positions = c.positions + entries;
    a.begin = c.first_positions;
    a.first = c.first_lens;
    a.err = err;
#define LS_OBSERVE(D) \
    (plan.blocks == 4   ? launch_observe_t<D, 4>(a, plan.whole_rows, stream) \
     : plan.blocks == 2 ? launch_observe_t<D, 2>(a, plan.whole_rows, stream) \
                        : launch_observe_t<D, 1>(a, plan.whole_rows, stream))
    return p.head_dim == 128 ? LS_OBSERVE(128) : LS_OBSERVE(64);
#undef LS_OBSERVE
}

}  // namespace ls
