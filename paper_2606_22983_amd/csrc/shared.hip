// Decode of a batch whose sessions share prefixes, and decode that accumulates
// the attention weight of every key (the batched decode step of §2.1 and §6 over
// the block tables of §5.1).
//
// With keys t of session s, scores x_t = scale q.k_t and row state (m, l, O) =
// (max x, sum e^(x - m), sum e^(x - m) v) over a set of keys, the states of two
// disjoint sets add up by the log-sum-exp rule.  A group's sessions have their
// first 16 P keys in common: the state over these is computed for all query rows
// of the group at once, as one matrix of (members x query heads per KV head) rows
// against K and V tiles that are read once per 64 rows, and each session's own
// keys are walked for it alone.
//
// Work: segments = (group, KV head, tile of 64 rows) over the group's blocks, then
// (session, KV head) over its own blocks.  A block of a segment costs some units
// (kCost*, from measurement); one workgroup per CU takes an equal contiguous share
// of all units, so it works on a few parts of segments.  Its four waves take a
// part's pairs of blocks in turn, each with a state of its own, and merge through
// LDS.  A segment that one workgroup has whole, without a shared prefix, is written
// out at once; other parts leave their state in the workspace, at slot (segment +
// workgroup), which no other part has, and a second kernel adds them up per row.
//
// Accumulated weights: the probability of a key is known only once its row's sum
// is, so the first kernel leaves the scores of the own keys (fp32, 4 bytes a head
// where K and V take 4 D of them a KV head) and the second one reads them back,
// sums e^(x - m) / l over the query heads of a KV head and adds that to the key's
// weight.
//
// Products: S^T[16 tokens x 16 rows] = K . Q^T (MFMA 16x16x32), whose accumulator
// layout (lane: row lane % 16, tokens 4 (lane / 16) + i) of a pair of blocks is
// the B operand of O^T[16 dims x 16 rows] += V^T . P^T (16x16x32 over the pair's 32
// tokens, in the order that the lanes hold them).  Probabilities are rounded to
// bf16 there, by 2^-9 of themselves at most half a step, while sums, maxima and
// accumulated weights take the fp32 ones.
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace ls {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kShThreads = 256;
constexpr int kShWaves = kShThreads / kWave;
constexpr int kShBatch = 2048;               // sessions (LDS)
constexpr int kTileRows = 64;                // rows of a prefix segment
constexpr int kRank = 11;                    // bits of a member's rank (kShBatch of them)
// Units of a block: own keys (bound by HBM), a prefix tile of 16, 32 or 64 rows.
constexpr int kCostOwn = 4;
constexpr int kCostTile1 = 2, kCostTile2 = 3, kCostTile4 = 4;
constexpr int kLeastUnits = kShWaves * 2 * kCostOwn;     // a pair of blocks for each wave
constexpr float kNoMax = -1.0e30f;           // running maximum of no key
// The running maximum moves only when a score passes it by this much (log2), so that
// probabilities reach 2^8 and most pairs of blocks need no rescaling.
constexpr float kMaxSlack = 8.0f;
constexpr int kRawBuffer = 0x00020000;       // raw buffer, 32-bit data format
constexpr int kStream = 2;                   // non-temporal: own keys are read once

// How a session's parts are found by the second kernel.
struct ShRecord {
    int64_t own_pos;               // first unit of (s, KV head 0); a KV head further: own_blocks * kCostOwn
    int64_t tile_pos;              // first unit of its prefix tile at KV head 0
    int64_t tile_stride;           // units per KV head of its group
    int32_t own_blocks;            // 0: no own key
    int32_t prefix_blocks;         // 0: no prefix
    int32_t tile_seg;              // prefix segment at KV head 0
    int32_t tile_seg_stride;       // prefix segments per KV head of its group
    int32_t tile_row;              // its first row in the tile
    int32_t tile_cost;             // units of a block of the tile
    int32_t keys;                  // L
    int32_t unused;
};
struct ShHeader {
    int64_t share;                 // units per workgroup
    int64_t own_base;              // first unit of the own segments
    int64_t own_units;             // own blocks of all sessions, per KV head
    int64_t unused;
};

struct SharedArgs {
    uint16_t *pool;                // layer base
    int64_t num_blocks;
    int32_t num_kv_heads, group;
    const uint16_t *q;             // [S][Hq][D]
    uint16_t *out;                 // [S][Hq][D]
    const int32_t *tables;         // [S][max_blocks]
    int32_t max_blocks;
    const int32_t *lens;           // [S]
    int32_t num_sessions;
    int32_t num_groups, num_members;
    const int32_t *starts;         // [num_groups + 1]
    const int32_t *members;        // [num_members]
    const int32_t *prefix;         // [num_groups] blocks
    float scale_log2;
    ShHeader *header;
    ShRecord *records;             // [S]
    float *tile_ml;                // [tile slots][64][2]
    float *tile_acc;               // [tile slots][64][D]
    float *own_ml;                 // [own slots][G][2]
    float *own_acc;                // [own slots][G][D]
    // Accumulated weights
    float *scores;                 // [num_blocks][Hkv][G][16]
    float *weights;                // layer base, [num_blocks][Hkv][16]
    int32_t *positions;            // the same
    const int32_t *reused;         // [S], or null: no key is new
    const int32_t *begin;          // [S] position of the first new key, or null: its slot
    const int32_t *first;          // [S] keys that no weight is kept for, or null
    unsigned int *err;
};

__device__ __forceinline__ int tile_cost(int rows) {
    return rows <= 16 ? kCostTile1 : rows <= 32 ? kCostTile2 : kCostTile4;
}
// Units per block of all tiles of a group of `rows` rows.
__device__ __forceinline__ int group_cost(int rows) {
    const int rest = rows % kTileRows;
    return rows / kTileRows * kCostTile4 + (rest ? tile_cost(rest) : 0);
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

// Two blocks of K and V in registers.
template <int D>
struct PairRegs {
    u32x4 k[2][D / 32];            // K[token lane % 16][8 dims of k-step]
    u32x2 v[2][D / 16];            // V^T[dim 16 dt + lane % 16][tokens 4 (lane / 16) .. + 3]
};

// (id < 0: a descriptor of no bytes, nothing is fetched and zeros arrive)
template <int D, int kPolicy>
__device__ __forceinline__ void load_pair(PairRegs<D> &r, const uint16_t *pool, int num_kv_heads, int g,
                                          const int (&id)[2], int koff, int voff) {
    constexpr int kTile = kBlock * D;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const uint16_t *kt = pool + ((int64_t)(id[b] < 0 ? 0 : id[b]) * 2 * num_kv_heads + g) * kTile;
        const uint16_t *vt = kt + (int64_t)num_kv_heads * kTile;
        const int bytes = id[b] < 0 ? 0 : kTile * 2;
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(kt), 0, bytes, kRawBuffer);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(vt), 0, bytes, kRawBuffer);
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
            r.k[b][ks] = __builtin_amdgcn_raw_buffer_load_b128(rk, koff, ks * 4 * kBlock * 16, kPolicy);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt)
            r.v[b][dt] = __builtin_amdgcn_raw_buffer_load_b64(rv, voff, dt * 16 * kBlock * 2, kPolicy);
    }
}

template <int D>
struct ShLds {
    // The schedule
    uint32_t cum[kShBatch + 1];    // own blocks of the sessions before
    int32_t len[kShBatch];
    int32_t owner[kShBatch];       // its place among the members, or -1
    uint16_t gid[kShBatch];
    int32_t start[kShBatch + 1];
    int32_t prefix[kShBatch];      // blocks of the group
    uint32_t lead[kShBatch];       // longest member: length, then lowest rank
    uint32_t gunits[kShBatch + 1]; // units per KV head of the groups before
    uint32_t gsegs[kShBatch + 1];  // tiles per KV head of the groups before
    unsigned scan[2][kShWaves];
    // The merge of a part's waves
    float m[kShWaves][kTileRows], l[kShWaves][kTileRows];
    __attribute__((aligned(16))) f32x4 o[kShWaves][2][D / 16][kWave];
};

// Exclusive prefix sums of two values per thread, and their totals.
__device__ __forceinline__ void scan2(unsigned (&v)[2], unsigned (&total)[2], unsigned (*sm)[kShWaves]) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    unsigned x[2] = {v[0], v[1]};
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const unsigned y0 = __shfl_up(x[0], off), y1 = __shfl_up(x[1], off);
        if (lane >= off) {
            x[0] += y0;
            x[1] += y1;
        }
    }
    __syncthreads();
    if (lane == kWave - 1) {
        sm[0][wave] = x[0];
        sm[1][wave] = x[1];
    }
    __syncthreads();
    total[0] = total[1] = 0;
    unsigned before[2] = {0, 0};
#pragma unroll
    for (int w = 0; w < kShWaves; ++w) {
        if (w == wave) {
            before[0] = total[0];
            before[1] = total[1];
        }
        total[0] += sm[0][w];
        total[1] += sm[1][w];
    }
    v[0] = before[0] + x[0] - v[0];
    v[1] = before[1] + x[1] - v[1];
}

// A part of a segment: blocks [j0, j1) of a table row.
struct ShPart {
    const int32_t *table;          // its table row
    int head;                      // KV head
    int j0, j1;
    int longest;                   // no row sees a key from here on
};

// The states of R tiles of 16 rows over the wave's pairs of a part.  row_len: keys
// that the lane's row of each tile sees, shortest: that all rows see; rows: scores of
// the tile's first ones are kept.
template <int D, int R, bool kScores, int kPolicy>
__device__ __forceinline__ void walk(const SharedArgs &a, const ShPart &part, const uint16_t *const (&qrow)[R],
                                     const int (&row_len)[R], int shortest, int rows, float (&m)[R], float (&lsum)[R],
                                     f32x4 (&o)[R][D / 16]) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c16 = lane % 16, g4 = lane / 16;
    bf16x8 qop[R][D / 32];
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) qop[r][ks] = *reinterpret_cast<const bf16x8 *>(qrow[r] + ks * 32 + g4 * 8);
        m[r] = kNoMax;
        lsum[r] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) o[r][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int blocks = part.j1 - part.j0, pairs = (blocks + 1) / 2;
    const int mine = pairs > wave ? (pairs - wave + kShWaves - 1) / kShWaves : 0;     // pairs of this wave
    const int koff = lane * 16, voff = c16 * kBlock * 2 + g4 * 8;
    // Ids of the wave's next 32 pairs: lane 2 i + b holds block b of pair i.
    int ids = -1;
    auto fetch_ids = [&](int i0) {
        const int j = part.j0 + 2 * (wave + kShWaves * (i0 + lane / 2)) + lane % 2;
        int id = -1;
        if (j < part.j1) {
            id = part.table[j];
            if (id < 0 || id >= a.num_blocks) {
                flag_error(a.err, LS_DEVERR_BLOCK_ID);
                id = -1;
            }
        }
        ids = id;
    };
    auto pair_ids = [&](int i, int (&id)[2]) {
        id[0] = __builtin_amdgcn_readlane(ids, (2 * i) % kWave);
        id[1] = __builtin_amdgcn_readlane(ids, (2 * i + 1) % kWave);
    };
    PairRegs<D> regs[2];
    int id[2][2] = {{-1, -1}, {-1, -1}};
    auto fetch = [&](PairRegs<D> &r, int (&which)[2], int i) {
        if (i >= mine) return;
        if (i % (kWave / 2) == 0) fetch_ids(i);
        pair_ids(i, which);
        load_pair<D, kPolicy>(r, a.pool, a.num_kv_heads, part.head, which, koff, voff);
    };
    auto work = [&](PairRegs<D> &t, const int (&which)[2], int i) {
        const int tok0 = (part.j0 + 2 * (wave + kShWaves * i)) * kBlock;
        // A pair some of whose keys some row does not see.
        const bool partial = tok0 + 2 * kBlock > shortest || which[0] < 0 || which[1] < 0;
        if (partial) {
            // Slots that no row sees may hold anything (NaN included): zero their V.
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int valid = part.longest - tok0 - b * kBlock - 4 * g4;
                const uint32_t lo = valid >= 2 ? 0xFFFFFFFFu : valid == 1 ? 0x0000FFFFu : 0u;
                const uint32_t hi = valid >= 4 ? 0xFFFFFFFFu : valid == 3 ? 0x0000FFFFu : 0u;
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) {
                    t.v[b][dt].x &= lo;
                    t.v[b][dt].y &= hi;
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[b][ks]), qop[r][ks], s[b], 0, 0, 0);
            float x[2][4];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[b][e] = s[b][e] * a.scale_log2;
                    if (partial && (tok0 + b * kBlock + 4 * g4 + e >= row_len[r] || which[b] < 0)) x[b][e] = -INFINITY;
                }
            if constexpr (kScores) {
                if (c16 < rows)
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        if (which[b] >= 0)
                            *reinterpret_cast<f32x4 *>(a.scores + (((int64_t)which[b] * a.num_kv_heads + part.head) * a.group + c16) * kBlock + 4 * g4) =
                                f32x4{x[b][0], x[b][1], x[b][2], x[b][3]};
            }
            const float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                                    fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
            if (__any(top > m[r] + kMaxSlack)) {
                const float now = fmaxf(m[r], max_xor_16_32(top));
                const float alpha = __builtin_amdgcn_exp2f(m[r] - now);
                lsum[r] *= alpha;
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) o[r][dt] *= alpha;
                m[r] = now;
            }
            float p[2][4];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[b][e] = __builtin_amdgcn_exp2f(x[b][e] - m[r]);
            lsum[r] += ((p[0][0] + p[0][1]) + (p[0][2] + p[0][3])) + ((p[1][0] + p[1][1]) + (p[1][2] + p[1][3]));
            const u32x4 pb = {pack_bf16x2(p[0][0], p[0][1]), pack_bf16x2(p[0][2], p[0][3]),
                              pack_bf16x2(p[1][0], p[1][1]), pack_bf16x2(p[1][2], p[1][3])};
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                const u32x4 va = {t.v[0][dt].x, t.v[0][dt].y, t.v[1][dt].x, t.v[1][dt].y};
                o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), __builtin_bit_cast(bf16x8, pb),
                                                                   o[r][dt], 0, 0, 0);
            }
        }
    };
    fetch(regs[0], id[0], 0);
    for (int i = 0; i < mine; i += 2) {
        fetch(regs[1], id[1], i + 1);
        work(regs[0], id[0], i);
        if (i + 1 >= mine) break;
        fetch(regs[0], id[0], i + 2);
        work(regs[1], id[1], i + 1);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) lsum[r] = sum_xor_16_32(lsum[r]);
}

// Where a part's state goes.
struct ShSink {
    float *ml;                     // [rows][2], or null
    float *acc;                    // [rows][D], or null: the output itself
    uint16_t *out;                 // [rows][D]
    int rows;
};

// Adds the waves' states up and writes them.
template <int D, int R>
__device__ __forceinline__ void merge(ShLds<D> &sm, const float (&m)[R], const float (&lsum)[R],
                                      const f32x4 (&o)[R][D / 16], const ShSink &sink) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c16 = lane % 16, g4 = lane / 16;
    constexpr int kHalf = R < 2 ? R : 2;       // tiles at a time
    if (g4 == 0)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sm.m[wave][r * 16 + c16] = m[r];
            sm.l[wave][r * 16 + c16] = lsum[r];
        }
#pragma unroll
    for (int r0 = 0; r0 < R; r0 += kHalf) {
        if (r0) __syncthreads();               // the half before has been read
#pragma unroll
        for (int r = 0; r < kHalf; ++r)
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) sm.o[wave][r][dt][lane] = o[r0 + r][dt];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kHalf; ++r) {
            const int row = (r0 + r) * 16 + c16;
            float top = kNoMax, e[kShWaves], l = 0.f;
#pragma unroll
            for (int w = 0; w < kShWaves; ++w) top = fmaxf(top, sm.m[w][row]);
#pragma unroll
            for (int w = 0; w < kShWaves; ++w) {
                e[w] = __builtin_amdgcn_exp2f(sm.m[w][row] - top);
                l += e[w] * sm.l[w][row];
            }
            const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
            for (int k = 0; k < D / 16 / kShWaves; ++k) {
                const int dt = wave + k * kShWaves;
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kShWaves; ++w) x += sm.o[w][r][dt][lane] * e[w];
                if (row < sink.rows) {
                    const int at = row * D + dt * 16 + 4 * g4;
                    if (sink.acc) *reinterpret_cast<f32x4 *>(sink.acc + at) = x;
                    else *reinterpret_cast<uint2 *>(sink.out + at) =
                        make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
                }
            }
            if (sink.ml && wave == 0 && g4 == 0 && row < sink.rows) {
                sink.ml[2 * row] = top;
                sink.ml[2 * row + 1] = l;
            }
        }
    }
    __syncthreads();                           // the next part writes sm again
}

template <int D, bool kWeights>
__global__ __launch_bounds__(kShThreads) void shared_kernel(SharedArgs a) {
    __shared__ ShLds<D> sm;
    const int tid = threadIdx.x, lane = tid % kWave, c16 = lane % 16;
    const int S = a.num_sessions, G = a.group, H = a.num_kv_heads;
    const bool first_wg = blockIdx.x == 0;
    const int gs = __builtin_ctz(G);           // (G is 1, 2, 4 or 8)
    // ---- the schedule, made by every workgroup for itself
    int ng = a.num_groups;
    bool bad = false;
    for (int g = tid; g < ng; g += kShThreads) {
        const int x = a.starts[g], y = a.starts[g + 1], pb = a.prefix[g];
        bad = bad || x < 0 || y < x || y > a.num_members || pb < 0 || pb > a.max_blocks || (g == 0 && x != 0) ||
              (g == ng - 1 && y != a.num_members);
        sm.start[g] = x;
        sm.start[g + 1] = y;                   // (the same value from two threads)
        sm.prefix[g] = pb;
        sm.lead[g] = 0u;
    }
    for (int s = tid; s < S; s += kShThreads) {
        sm.owner[s] = -1;
        const int raw = a.lens[s], cap = a.max_blocks * kBlock;
        if (first_wg && (raw < 0 || raw > cap)) flag_error(a.err, LS_DEVERR_LENGTH);
        sm.len[s] = max(min(raw, cap), 0);
    }
    bad = __syncthreads_or(bad);
    if (ng && !bad) {
        bool wrong = false;
        for (int i = tid; i < a.num_members; i += kShThreads) {
            const int s = a.members[i];
            if (s < 0 || s >= S) {
                wrong = true;
                continue;
            }
            int lo = 0, hi = ng;                // the last group that starts at or before i and has it
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (sm.start[mid] <= i) lo = mid;
                else hi = mid;
            }
            if (atomicExch(&sm.owner[s], i) != -1) wrong = true;
            sm.gid[s] = (uint16_t)lo;
            atomicMax(&sm.lead[lo], (uint32_t)sm.len[s] << kRank | (uint32_t)(kShBatch - 1 - (i - sm.start[lo])));
        }
        bad = __syncthreads_or(wrong);
    }
    if (bad) {
        // Groups that cannot be: every session is computed on its own.
        if (first_wg && tid == 0) flag_error(a.err, LS_DEVERR_GROUP);
        ng = 0;
        __syncthreads();
        for (int s = tid; s < S; s += kShThreads) sm.owner[s] = -1;
        __syncthreads();
    }
    {
        const int per = (ng + kShThreads - 1) / kShThreads;
        unsigned v[2] = {0, 0}, all[2];
        for (int g = tid * per; g < min(ng, (tid + 1) * per); ++g) {
            const int rows = (sm.start[g + 1] - sm.start[g]) * G, longest = (int)(sm.lead[g] >> kRank);
            const int pb = min(sm.prefix[g], (longest + kBlock - 1) / kBlock);
            sm.prefix[g] = pb;
            sm.gunits[g] = (unsigned)(group_cost(rows) * pb);
            sm.gsegs[g] = (unsigned)((rows + kTileRows - 1) / kTileRows);
            v[0] += sm.gunits[g];
            v[1] += sm.gsegs[g];
        }
        scan2(v, all, sm.scan);
        for (int g = tid * per; g < min(ng, (tid + 1) * per); ++g) {
            const unsigned u = sm.gunits[g], t = sm.gsegs[g];
            sm.gunits[g] = v[0];
            sm.gsegs[g] = v[1];
            v[0] += u;
            v[1] += t;
        }
        if (tid == 0) {
            sm.gunits[ng] = all[0];
            sm.gsegs[ng] = all[1];
        }
    }
    __syncthreads();
    {
        const int per = (S + kShThreads - 1) / kShThreads;
        unsigned v[2] = {0, 0}, all[2];
        auto own = [&](int s) {
            const int pb = sm.owner[s] >= 0 ? sm.prefix[sm.gid[s]] : 0;
            return max((sm.len[s] + kBlock - 1) / kBlock - pb, 0);
        };
        for (int s = tid * per; s < min(S, (tid + 1) * per); ++s) v[0] += (unsigned)own(s);
        scan2(v, all, sm.scan);
        for (int s = tid * per; s < min(S, (tid + 1) * per); ++s) {
            sm.cum[s] = v[0];
            v[0] += (unsigned)own(s);
        }
        if (tid == 0) sm.cum[S] = all[0];
    }
    __syncthreads();
    const int64_t own_base = (int64_t)H * sm.gunits[ng];
    const int64_t units = own_base + (int64_t)H * sm.cum[S] * kCostOwn;
    int64_t share = (units + gridDim.x - 1) / gridDim.x;
    if (share < kLeastUnits) share = kLeastUnits;
    if (first_wg) {
        if (tid == 0) *a.header = ShHeader{share, own_base, (int64_t)sm.cum[S], 0};
        for (int s = tid; s < S; s += kShThreads) {
            ShRecord r = {};
            r.own_blocks = (int)(sm.cum[s + 1] - sm.cum[s]);
            r.own_pos = own_base + (int64_t)H * sm.cum[s] * kCostOwn;
            r.keys = sm.len[s];
            if (sm.owner[s] >= 0) {
                const int g = sm.gid[s], rows = (sm.start[g + 1] - sm.start[g]) * G, row = (sm.owner[s] - sm.start[g]) * G;
                const int tile = row / kTileRows;
                r.prefix_blocks = sm.prefix[g];
                r.tile_pos = (int64_t)H * sm.gunits[g] + (int64_t)tile * kCostTile4 * sm.prefix[g];
                r.tile_stride = sm.gunits[g + 1] - sm.gunits[g];
                r.tile_seg = (int)(H * sm.gsegs[g]) + tile;
                r.tile_seg_stride = (int)(sm.gsegs[g + 1] - sm.gsegs[g]);
                r.tile_row = row % kTileRows;
                r.tile_cost = tile_cost(min(kTileRows, rows - tile * kTileRows));
            }
            a.records[s] = r;
        }
    }
    // Consecutive shares on one XCD: the tiles of a group and KV head read the same K and V.
    const int W = gridDim.x;
    const int w = W % 8 == 0 ? (int)(blockIdx.x % 8) * (W / 8) + (int)(blockIdx.x / 8) : (int)blockIdx.x;
    const int64_t u0 = (int64_t)w * share, u1 = min(u0 + share, units);
    // Blocks of the segment at `pos` that are this workgroup's.
    auto range = [&](int64_t pos, int blocks, int cost, int &j0, int &j1) {
        j0 = u0 > pos ? (int)((u0 - pos + cost - 1) / cost) : 0;
        j1 = u1 - pos >= (int64_t)blocks * cost ? blocks : (int)((u1 - pos + cost - 1) / cost);
    };
    int64_t at = u0;
    // ---- prefix tiles
    if (at < min(u1, own_base)) {
        int g = 0, hi = ng;
        while (hi - g > 1) {
            const int mid = (g + hi) / 2;
            if ((int64_t)H * sm.gunits[mid] <= at) g = mid;
            else hi = mid;
        }
        for (; g < ng && (int64_t)H * sm.gunits[g] < min(u1, own_base); ++g) {
            const int64_t stride = sm.gunits[g + 1] - sm.gunits[g];
            if (!stride) continue;
            const int pb = sm.prefix[g], rows = (sm.start[g + 1] - sm.start[g]) * G, tiles = (rows + kTileRows - 1) / kTileRows;
            const int64_t gpos = (int64_t)H * sm.gunits[g];
            const int lead = kShBatch - 1 - (int)(sm.lead[g] & (kShBatch - 1));
            const int lead_s = a.members[sm.start[g] + lead];
            for (int h = at > gpos ? (int)((at - gpos) / stride) : 0; h < H && gpos + h * stride < u1; ++h) {
                const int64_t hpos = gpos + h * stride;
                for (int t = at > hpos ? (int)((at - hpos) / ((int64_t)pb * kCostTile4)) : 0; t < tiles; ++t) {
                    const int64_t pos = hpos + (int64_t)t * pb * kCostTile4;
                    if (pos >= u1) break;
                    const int n = min(kTileRows, rows - t * kTileRows), cost = tile_cost(n);
                    ShPart part;
                    range(pos, pb, cost, part.j0, part.j1);
                    if (part.j0 >= part.j1) continue;
                    part.table = a.tables + (int64_t)lead_s * a.max_blocks;
                    part.head = h;
                    part.longest = (int)(sm.lead[g] >> kRank);
                    const int64_t slot = (int64_t)H * sm.gsegs[g] + (int64_t)h * tiles + t + w;
                    const ShSink sink = {a.tile_ml + slot * kTileRows * 2, a.tile_acc + slot * kTileRows * D, nullptr, n};
                    auto run = [&](auto tag) {
                        constexpr int R = decltype(tag)::value;
                        const uint16_t *qrow[R];
                        int row_len[R], shortest = INT32_MAX;
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            // (lanes of no row take the last one: a load under a condition waits for the one before)
                            const int row = t * kTileRows + min(r * 16 + c16, n - 1);
                            const int s = a.members[sm.start[g] + (row >> gs)];
                            qrow[r] = a.q + ((int64_t)s * H * G + h * G + (row & (G - 1))) * D;
                            row_len[r] = sm.len[s];
                            shortest = min(shortest, row_len[r]);
                        }
#pragma unroll
                        for (int off = 1; off < 16; off <<= 1) shortest = min(shortest, __shfl_xor(shortest, off));
                        shortest = __builtin_amdgcn_readfirstlane(shortest);
                        float m[R], lsum[R];
                        f32x4 o[R][D / 16];
                        walk<D, R, false, 0>(a, part, qrow, row_len, shortest, n, m, lsum, o);
                        merge<D, R>(sm, m, lsum, o, sink);
                    };
                    if (n <= 16) run(std::integral_constant<int, 1>{});
                    else if (n <= 32) run(std::integral_constant<int, 2>{});
                    else run(std::integral_constant<int, 4>{});
                }
            }
        }
        at = own_base;
    }
    // ---- own keys
    if (at < u1) {
        const int64_t rel = (at - own_base) / kCostOwn / H;       // blocks per KV head before
        int s = 0, hi = S;                      // the last session that starts at or before it
        while (hi - s > 1) {
            const int mid = (s + hi) / 2;
            if ((int64_t)sm.cum[mid] <= rel) s = mid;
            else hi = mid;
        }
        for (; s < S; ++s) {
            const int64_t spos = own_base + (int64_t)H * sm.cum[s] * kCostOwn;
            if (spos >= u1) break;
            const int nb = (int)(sm.cum[s + 1] - sm.cum[s]);
            if (!nb) continue;
            const int pb = sm.owner[s] >= 0 ? sm.prefix[sm.gid[s]] : 0, L = sm.len[s];
            const int64_t stride = (int64_t)nb * kCostOwn;
            for (int h = at > spos ? (int)((at - spos) / stride) : 0; h < H; ++h) {
                const int64_t pos = spos + h * stride;
                if (pos >= u1) break;
                int j0, j1;
                range(pos, nb, kCostOwn, j0, j1);
                if (j0 >= j1) continue;
                ShPart part = {a.tables + (int64_t)s * a.max_blocks, h, pb + j0, pb + j1, L};
                const bool whole = !pb && j0 == 0 && j1 == nb;
                const int64_t slot = (int64_t)s * H + h + w;
                const int64_t row0 = (int64_t)s * H * G + h * G;
                const ShSink sink = {!whole || kWeights ? a.own_ml + slot * G * 2 : nullptr, whole ? nullptr : a.own_acc + slot * G * D,
                                     a.out + row0 * D, G};
                const uint16_t *qrow[1] = {a.q + (row0 + min(c16, G - 1)) * D};
                const int row_len[1] = {L};
                float m[1], lsum[1];
                f32x4 o[1][D / 16];
                walk<D, 1, kWeights, kStream>(a, part, qrow, row_len, L, G, m, lsum, o);
                merge<D, 1>(sm, m, lsum, o, sink);
            }
        }
    }
}

// Calls f(slot, part workgroup) for every part of a segment's blocks.
template <typename F>
__device__ __forceinline__ void each_part(int64_t share, int64_t pos, int blocks, int cost, int64_t seg, F f) {
    const int64_t end = pos + (int64_t)blocks * cost;
    for (int64_t w = pos / share; w * share < end; ++w) {
        const int64_t lo = w * share - pos, hi = lo + share;
        const int64_t j0 = lo > 0 ? (lo + cost - 1) / cost : 0, j1 = hi >= (int64_t)blocks * cost ? blocks : (hi + cost - 1) / cost;
        if (j0 < j1) f(seg + w);
    }
}

// Row state of (session, query head): top is the largest maximum, sum the whole sum.
template <typename F>
__device__ __forceinline__ void row_state(const SharedArgs &a, const ShRecord &r, int64_t share, int s, int h, int head,
                                          float &top, float &sum, F f) {
    // f(ml, acc row index or such) is called for every part in a fixed order, twice.
    top = kNoMax;
    sum = 0.f;
    const int H = a.num_kv_heads, G = a.group;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        auto visit = [&](const float *ml, int64_t acc_row, bool tile) {
            if (pass == 0) {
                top = fmaxf(top, ml[0]);
            } else {
                const float e = __builtin_amdgcn_exp2f(ml[0] - top);
                sum += e * ml[1];
                f(e, acc_row, tile);
            }
        };
        if (r.prefix_blocks)
            each_part(share, r.tile_pos + h * r.tile_stride, r.prefix_blocks, r.tile_cost,
                      (int64_t)r.tile_seg + (int64_t)h * r.tile_seg_stride, [&](int64_t slot) {
                          const int64_t row = slot * kTileRows + r.tile_row + head;
                          visit(a.tile_ml + row * 2, row, true);
                      });
        if (r.own_blocks)
            each_part(share, r.own_pos + (int64_t)h * r.own_blocks * kCostOwn, r.own_blocks, kCostOwn, (int64_t)s * H + h,
                      [&](int64_t slot) {
                          const int64_t row = slot * G + head;
                          visit(a.own_ml + row * 2, row, false);
                      });
    }
}

// Workgroups below `combine` add up rows of the output, D / 4 threads a row; the
// others take equal shares of the own blocks and add their probabilities to the
// weights, four threads a (block, KV head).
template <int D, bool kWeights>
__global__ __launch_bounds__(kShThreads) void shared_merge_kernel(SharedArgs a, int combine) {
    __shared__ uint32_t sm_cum[kWeights ? kShBatch + 1 : 1];
    __shared__ float sm_top[8], sm_inv[8];
    const int tid = threadIdx.x, H = a.num_kv_heads, G = a.group, S = a.num_sessions;
    const ShHeader head = *a.header;
    if ((int)blockIdx.x < combine) {
        constexpr int kLanes = D / 4;
        const int64_t row = (int64_t)blockIdx.x * (kShThreads / kLanes) + tid / kLanes;
        if (row >= (int64_t)S * H * G) return;
        const int s = (int)(row / (H * G)), h = (int)(row % (H * G)) / G, e4 = tid % kLanes * 4;
        const ShRecord r = a.records[s];
        if (r.own_blocks && !r.prefix_blocks) {
            // written already, if the workgroup that has its first block has the last one too
            const int64_t pos = r.own_pos + (int64_t)h * r.own_blocks * kCostOwn;
            if ((pos / head.share + 1) * head.share - pos > (int64_t)(r.own_blocks - 1) * kCostOwn) return;
        }
        float top, sum;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        row_state(a, r, head.share, s, h, (int)(row % G), top, sum, [&](float e, int64_t at, bool tile) {
            x += *reinterpret_cast<const f32x4 *>((tile ? a.tile_acc : a.own_acc) + at * D + e4) * e;
        });
        const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
        *reinterpret_cast<uint2 *>(a.out + row * D + e4) =
            make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
        return;
    }
    if constexpr (kWeights) {
        for (int s = tid; s < S; s += kShThreads) sm_cum[s] = (uint32_t)((a.records[s].own_pos - head.own_base) / kCostOwn / H);
        if (tid == 0) sm_cum[S] = (uint32_t)head.own_units;
        __syncthreads();
        const int64_t all = head.own_units * H, n = gridDim.x - combine, w = blockIdx.x - combine;
        int64_t per = (all + n - 1) / n;
        per = max(per, (int64_t)(kShThreads / 4));
        const int64_t b0 = w * per, b1 = min(b0 + per, all);
        if (b0 >= b1) return;
        int s = 0, hi = S;
        while (hi - s > 1) {
            const int mid = (s + hi) / 2;
            if ((int64_t)sm_cum[mid] * H <= b0) s = mid;
            else hi = mid;
        }
        for (; s < S && (int64_t)sm_cum[s] * H < b1; ++s) {
            const ShRecord r = a.records[s];
            if (!r.own_blocks) continue;
            const int first = a.first ? a.first[s] : 0;
            const int old = a.reused ? a.reused[s] : INT32_MAX;      // keys from here on are new
            const int begin = a.reused ? (a.begin ? a.begin[s] : old) : 0;
            const int64_t spos = (int64_t)sm_cum[s] * H;
            for (int h = b0 > spos ? (int)((b0 - spos) / r.own_blocks) : 0; h < H; ++h) {
                const int64_t pos = spos + (int64_t)h * r.own_blocks;
                if (pos >= b1) break;
                __syncthreads();                                     // the segment before is done with sm_top
                if (tid < G) {
                    float top, sum;
                    row_state(a, r, head.share, s, h, tid, top, sum, [](float, int64_t, bool) {});
                    sm_top[tid] = top;
                    sm_inv[tid] = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                }
                __syncthreads();
                const int j0 = (int)max(b0 - pos, (int64_t)0), j1 = (int)min(b1 - pos, (int64_t)r.own_blocks);
                for (int j = j0 + tid / 4; j < j1; j += kShThreads / 4) {
                    const int col = r.prefix_blocks + j, t0 = col * kBlock + tid % 4 * 4;
                    const int id = a.tables[(int64_t)s * a.max_blocks + col];
                    if (id < 0 || id >= a.num_blocks || t0 >= r.keys || t0 + 4 <= first) continue;
                    const float *x = a.scores + ((int64_t)id * H + h) * G * kBlock + tid % 4 * 4;
                    f32x4 p = {0.f, 0.f, 0.f, 0.f};
                    for (int k = 0; k < G; ++k) {
                        const f32x4 y = *reinterpret_cast<const f32x4 *>(x + k * kBlock);
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[e] += __builtin_amdgcn_exp2f(y[e] - sm_top[k]) * sm_inv[k];
                    }
                    const int64_t at = ((int64_t)id * H + h) * kBlock + tid % 4 * 4;
                    const f32x4 was = *reinterpret_cast<const f32x4 *>(a.weights + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = t0 + e;
                        if (t < first || t >= r.keys) continue;
                        a.weights[at + e] = t >= old ? p[e] : was[e] + p[e];
                        if (t >= old) a.positions[at + e] = begin + (t - old);
                    }
                }
            }
        }
    }
}

template <int D>
hipError_t launch_shared_t(const SharedArgs &a, int grid, hipStream_t stream) {
    const int64_t rows = (int64_t)a.num_sessions * a.num_kv_heads * a.group;
    const int combine = (int)((rows + kShThreads / (D / 4) - 1) / (kShThreads / (D / 4)));
    if (a.weights) {
        hipLaunchKernelGGL((shared_kernel<D, true>), dim3(grid), dim3(kShThreads), 0, stream, a);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL((shared_merge_kernel<D, true>), dim3(combine + 4 * grid), dim3(kShThreads), 0, stream, a, combine);
    } else {
        hipLaunchKernelGGL((shared_kernel<D, false>), dim3(grid), dim3(kShThreads), 0, stream, a);
        if (hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL((shared_merge_kernel<D, false>), dim3(combine), dim3(kShThreads), 0, stream, a, combine);
    }
    return hipGetLastError();
}

constexpr size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

SharedPlan plan_shared(const PoolGeom &p, int32_t num_sessions, int32_t num_q_heads, int32_t num_groups,
                       int32_t num_members, bool weights) {
    const int64_t H = p.num_kv_heads, G = num_q_heads / p.num_kv_heads, W = p.num_cus > 0 ? p.num_cus : 256;
    SharedPlan s;
    // (a slot per segment and one per workgroup; a group has a tile that is not full)
    s.tile_slots = num_groups ? (size_t)(H * ((int64_t)num_members * G / kTileRows + num_groups) + W) : 0;
    s.own_slots = (size_t)(num_sessions * H + W);
    s.at[0] = 0;
    s.at[1] = s.at[0] + align256(sizeof(ShHeader));
    s.at[2] = s.at[1] + align256((size_t)num_sessions * sizeof(ShRecord));
    s.at[3] = s.at[2] + align256(s.tile_slots * kTileRows * 2 * sizeof(float));
    s.at[4] = s.at[3] + align256(s.tile_slots * kTileRows * (size_t)p.head_dim * sizeof(float));
    s.at[5] = s.at[4] + align256(s.own_slots * (size_t)G * 2 * sizeof(float));
    s.at[6] = s.at[5] + align256(s.own_slots * (size_t)G * (size_t)p.head_dim * sizeof(float));
    s.total = s.at[6] + (weights ? (size_t)p.num_blocks * (size_t)num_q_heads * kBlock * sizeof(float) : 0);
    return s;
}

hipError_t launch_shared(const PoolGeom &p, int layer, int32_t num_sessions, int32_t num_q_heads, const SharedCall &c,
                         const SharedPlan &plan, unsigned int *err, hipStream_t stream) {
    uint8_t *ws = static_cast<uint8_t *>(c.workspace);
    SharedArgs a = {};
    a.pool = p.layer_base(layer);
    a.num_blocks = p.num_blocks;
    a.num_kv_heads = p.num_kv_heads;
    a.group = num_q_heads / p.num_kv_heads;
    a.q = c.q;
    a.out = c.out;
    a.tables = c.block_tables;
    a.max_blocks = c.max_blocks;
    a.lens = c.context_lens;
    a.num_sessions = num_sessions;
    a.num_groups = c.num_groups;
    a.num_members = c.num_members;
    a.starts = c.group_starts;
    a.members = c.group_members;
    a.prefix = c.prefix_blocks;
    a.scale_log2 = c.scale * 1.4426950408889634f;
    a.header = reinterpret_cast<ShHeader *>(ws + plan.at[0]);
    a.records = reinterpret_cast<ShRecord *>(ws + plan.at[1]);
    a.tile_ml = reinterpret_cast<float *>(ws + plan.at[2]);
    a.tile_acc = reinterpret_cast<float *>(ws + plan.at[3]);
    a.own_ml = reinterpret_cast<float *>(ws + plan.at[4]);
    a.own_acc = reinterpret_cast<float *>(ws + plan.at[5]);
    a.scores = reinterpret_cast<float *>(ws + plan.at[6]);
    const int64_t entries = (int64_t)layer * p.num_blocks * p.num_kv_heads * kBlock;
    a.weights = c.weights ? c.weights + entries : nullptr;
    a.positions = c.positions ? c.positions + entries : nullptr;
    a.reused = c.reused_lens;
    a.begin = c.first_positions;
    a.first = c.first_lens;
    a.err = err;
    const int cus = stream_cus(p, stream), most = p.num_cus > 0 ? p.num_cus : 256;
    const int grid = std::min(cus, most);
    return p.head_dim == 128 ? launch_shared_t<128>(a, grid, stream) : launch_shared_t<64>(a, grid, stream);
}

}  // namespace ls
