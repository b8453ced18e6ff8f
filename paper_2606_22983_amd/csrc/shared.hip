// Decode of a batch whose sessions share prefixes, and decode that accumulates
// the attention weight of every key (the batched decode step of §2.1 and §6 over
// the block tables of §5.1).
//
// With keys t of session s, scores x_t = scale q.k_t and row state (m, l, O) =
// (max x, sum e^(x - m), sum e^(x - m) v) over a set of keys, the states of two
// disjoint sets add up by the log-sum-exp rule.  A group's sessions have their
// first 16 P keys in common: the state over these is computed for all query rows
// of the group at once, as one matrix of (members x query heads per KV head) rows
// against K and V tiles that are read once per tile of rows, and each session's own
// keys are walked for it alone.
//
// Work: segments = (group, KV head, tile of up to 16 or 128 rows) over the group's blocks,
// then (session, KV head) over its own blocks.  A block of a segment costs some units
// (kCost*).  Of the workgroups, of four waves, two for each CU, as many as the units say are for
// prefixes and the others for own blocks, on every XCD; each takes an equal contiguous
// share of the one or the other, so it works on a few parts of segments.  A part with up to 16
// rows (own keys, small groups): the waves take its pairs of blocks in turn, straight
// into registers, each with a state of its own, and merge through LDS.  With more rows:
// the pairs go through LDS, and every wave takes them all, for 16 or 32 rows of its own.
// A workgroup goes through most of the code once or twice a launch, and fetching
// instructions for the first time took as long as the work: loops are not unrolled, and
// masked and whole pairs share their code.  A segment that one workgroup has whole, without a shared
// prefix, is written out at once; other parts leave their state in the workspace, at slot
// (segment + workgroup), which no other part has (prefix tiles at row 16 places before +
// 128 workgroup), and a second kernel adds them up.
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
// bf16 there, by half a step (2^-8 of themselves) at most, while sums, maxima and
// accumulated weights take the fp32 ones.
//
// Bound by HBM where own keys are many, else by latency.  Measured (head_dim 128, both
// kernels, a call): 64 sessions behind 4096 shared tokens, 32 / 4 heads, 51 us, 162 MB read;
// 256 sessions in 8 groups, 16 / 2 heads, 57 us, 219 MB (4.7 TB/s in the first kernel); 3
// sessions behind 640 shared tokens 19 us (13.6 and 3.0 on the GPU).  With weights, 64
// sessions of up to 16384 tokens 173 us, 783 MB needed; the scores' stores take 31 of them.
// The decode of each session's own table, one launch with a prefix that stays in the caches,
// takes 72 (lengths on the host) or 78 us, 57 or 64, and 8 in these three: sharing pays from
// some 10^8 members x shared tokens x KV heads x D on (4 heads of 128: 128 members behind 1024
// tokens 33 us for 31, behind 4096 51 for 74; 32 behind 4096 33 for 31, behind 16384 55 for 84).
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
constexpr int kShPerCu = 2;                  // workgroups
// Sessions, members and groups that a kernel's LDS has room for: with the few, two
// workgroups fit a CU, with the most one (the other half of the grid follows): 512 sessions of
// 50 to 500 own tokens, half of them in 8 groups, 16 / 2 heads of 128, take 52 us, 600 78.
constexpr int kShFew = 512, kShMost = 2048;
// Rows of a prefix segment: 128 (two tiles of 16 per wave), but 16 in groups of up to 64,
// where four parts of 16 cost no more than one of 128 and a wave waits for less.
constexpr int kTileRows = 128, kFewRows = 16, kFewMost = 64;
constexpr int kRank = 11;                    // bits of a member's rank (kShMost of them)
static_assert(kShMost == 1 << kRank && kShMost == kMaxCacheSessions, "ranks fit");
// Units: of an own block and a block of a prefix tile of up to 16 rows (whose pairs the
// waves share), of a block of a larger tile, and of what beginning a part takes (3 us, where
// an own block of D 128 takes 0.4 and a tile's 1.5: without them, workgroups that got many
// short segments ended last by far).
constexpr int kCostFew = 1, kCostTile = 4, kCostPart = 8;
// The least share.
constexpr int kLeastTile = kCostPart + 4 * kCostTile, kLeastOwn = kCostPart + 2 * kShWaves;
constexpr float kNoMax = -0x1.fffffep127f;   // running maximum of no key: no finite score is below it
// The running maximum moves only when a score passes it by this much (log2), so that
// probabilities reach 2^8 and most pairs of blocks need no rescaling.
constexpr float kMaxSlack = 8.0f;
constexpr int kRawBuffer = 0x00020000;       // raw buffer, 32-bit data format
constexpr int kStream = 2;                   // non-temporal: own keys are read once

// What the second kernel knows of a session.
struct ShRecord {
    int32_t own_blocks;            // 0: no own key
    int32_t prefix_blocks;         // 0: no prefix
    int32_t tile_seg;              // first 16-row place of its prefix tile at KV head 0
    int32_t tile_seg_stride;       // places per KV head of its group
    int32_t tile_row;              // its first row in the tile
    int32_t keys;                  // weights are kept of those before this one: L, or 0
    uint32_t own_before;           // own blocks of the sessions before
    uint32_t own_all;              // of all sessions
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
    ShRecord *records;             // [S]
    int32_t *tile_first, *tile_last;     // [first place of a prefix tile] workgroups of its first and last part
    int32_t *own_first, *own_last;       // [S][Hkv]
    float *tile_ml;                // [16 first places + 128 workgroups][2]
    float *tile_acc;               // the same [D]
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

__device__ __forceinline__ int tile_cost(int rows) { return rows <= kFewRows ? kCostFew : kCostTile; }
__device__ __forceinline__ int tile_size(int rows) { return rows <= kFewMost ? kFewRows : kTileRows; }
// 16-row places that the tiles of a group take per KV head.
__device__ __forceinline__ int tile_places(int rows) {
    const int size = tile_size(rows);
    return (rows + size - 1) / size * (size / kFewRows);
}
// Units of all tiles of a group of `rows` rows over `blocks` blocks, per KV head.
__device__ __forceinline__ int group_cost(int rows, int blocks) {
    const int size = tile_size(rows), rest = rows % size;
    if (!blocks) return 0;
    return rows / size * (tile_cost(size) * blocks + kCostPart) + (rest ? tile_cost(rest) * blocks + kCostPart : 0);
}
// Keys of session s, clipped to its table.
__device__ __forceinline__ int keys_of(const SharedArgs &a, int s) {
    return max(min(a.lens[s], a.max_blocks * kBlock), 0);
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

// K tile of a block and KV head (id < 0: a descriptor of no bytes, nothing is fetched).
template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const uint16_t *pool, int num_kv_heads, int g, int id, bool v) {
    const uint16_t *t = pool + ((int64_t)(id < 0 ? 0 : id) * 2 * num_kv_heads + g + (v ? num_kv_heads : 0)) * (kBlock * D);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(t), 0, id < 0 ? 0 : kBlock * D * 2, kRawBuffer);
}

// Two pairs of blocks in LDS, as in the pool; there waves merge, too, and the schedule is made.
template <int D>
struct StageLds {
    __attribute__((aligned(1024))) uint8_t tile[8][kBlock * D * 2];     // K, K, V, V
};

template <int kMost>
struct ShPlan {
    uint32_t cum[kMost + 1];       // own blocks of the sessions before
    uint32_t cost[kMost + 1];      // and those with what beginning them takes
    uint16_t pb[kMost];            // blocks that the session shares
    uint8_t pad[kMost];            // slots of its last block without a token
    uint16_t gid[kMost];
    uint16_t start[kMost + 1];     // of the group's members
    uint16_t prefix[kMost];        // blocks of the group
    uint32_t lead[kMost];          // its longest member: length, then lowest rank
    uint16_t lead_s[kMost];        // that member
    uint32_t units[kMost + 1];     // units per KV head of the groups before
    uint16_t segs[kMost + 1];      // places of their tiles, per KV head
    unsigned scan[2][kShWaves];
    float m[kShWaves][16], l[kShWaves][16];       // the merge of a part's waves
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
    int longest;                   // no row sees a key from here on (and one that sees fewer is not used)
};

// State of a tile of 16 rows: row lane % 16, dims 16 dt + 4 (lane / 16) + i.
template <int D>
struct RowState {
    float m, l;
    f32x4 o[D / 16];
    __device__ __forceinline__ void clear() {
        m = kNoMax;
        l = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Scores x (log2) of a pair's keys: their probabilities as the operand of the second product.
    __device__ __forceinline__ bf16x8 take(const float (&x)[2][4]) {
        const float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                                fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
        if (__any(top > m + kMaxSlack)) {
            const float now = fmaxf(m, max_xor_16_32(top));
            const float alpha = __builtin_amdgcn_exp2f(m - now);
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) o[dt] *= alpha;
            m = now;
        }
        float p[2][4];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) p[b][e] = __builtin_amdgcn_exp2f(x[b][e] - m);
        l += ((p[0][0] + p[0][1]) + (p[0][2] + p[0][3])) + ((p[1][0] + p[1][1]) + (p[1][2] + p[1][3]));
        const u32x4 pb = {pack_bf16x2(p[0][0], p[0][1]), pack_bf16x2(p[0][2], p[0][3]), pack_bf16x2(p[1][0], p[1][1]),
                          pack_bf16x2(p[1][2], p[1][3])};
        return __builtin_bit_cast(bf16x8, pb);
    }
};

// Scores of a pair's products.  The row sees keys before row_len; absent: a bit per block
// that is not in the pool.
__device__ __forceinline__ void scores_of(const f32x4 (&s)[2], float scale_log2, int tok0, int row_len, int absent, float (&x)[2][4]) {
    const int left = row_len - tok0 - 4 * (int)(threadIdx.x % kWave / 16);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int seen = absent >> b & 1 ? 0 : left - b * kBlock;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[b][e] = e < seen ? s[b][e] * scale_log2 : -INFINITY;
    }
}
// Tokens t and t + 1 of V: zeros from `longest` on.  Slots that no row sees may hold anything
// (NaN included).
__device__ __forceinline__ uint32_t seen_v(uint32_t two, int t, int longest) {
    return t + 1 < longest ? two : t < longest ? two & 0x0000FFFFu : 0u;
}

// The id of a part's block, or -1 (none, or not in the pool).
__device__ __forceinline__ int part_id(const SharedArgs &a, const ShPart &part, int j) {
    if (j >= part.j1) return -1;
    const int id = part.table[j];
    if (id >= 0 && id < a.num_blocks) return id;
    flag_error(a.err, LS_DEVERR_BLOCK_ID);
    return -1;
}

// Up to 16 rows: the wave's pairs of the part.  qrow, row_len: of the lane's row.  K of the
// next pair is requested when the first product has taken this one's, V when the second has.
template <int D, bool kScores, int kPolicy>
__device__ __forceinline__ void walk(const SharedArgs &a, const ShPart &part, const uint16_t *qrow, int row_len,
                                     RowState<D> &st) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c16 = lane % 16, g4 = lane / 16;
    const int pairs = (part.j1 - part.j0 + 1) / 2;
    const int mine = pairs > wave ? (pairs - wave + kShWaves - 1) / kShWaves : 0;     // pairs of this wave
    const int koff = lane * 16, voff = c16 * kBlock * 2 + g4 * 8;
    int ids = -1;                              // of the wave's next 32 pairs: lane 2 i + b holds block b of pair i
    auto fetch_ids = [&](int i) {
        ids = part_id(a, part, part.j0 + 2 * (wave + kShWaves * (i + lane / 2)) + lane % 2);
        // (waited for here, so that the loop's other loads need not be)
        __builtin_amdgcn_s_waitcnt(0x0F70);
    };
    bf16x8 qop[D / 32];
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) qop[ks] = *reinterpret_cast<const bf16x8 *>(qrow + ks * 32 + g4 * 8);
    fetch_ids(0);
    st.clear();
    u32x4 k[2][D / 32];                        // K[token lane % 16][8 dims of k-step]
    u32x2 v[2][D / 16];                        // V^T[dim 16 dt + lane % 16][tokens 4 (lane / 16) .. + 3]
    auto load_k = [&](const int (&id)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const __amdgpu_buffer_rsrc_t r = tile_rsrc<D>(a.pool, a.num_kv_heads, part.head, id[b], false);
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) k[b][ks] = __builtin_amdgcn_raw_buffer_load_b128(r, koff, ks * 4 * kBlock * 16, kPolicy);
        }
    };
    auto load_v = [&](const int (&id)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const __amdgpu_buffer_rsrc_t r = tile_rsrc<D>(a.pool, a.num_kv_heads, part.head, id[b], true);
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) v[b][dt] = __builtin_amdgcn_raw_buffer_load_b64(r, voff, dt * 16 * kBlock * 2, kPolicy);
        }
    };
    int id[2] = {__builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1)};
    load_k(id);
    load_v(id);
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        const int tok0 = (part.j0 + 2 * (wave + kShWaves * i)) * kBlock;
        f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[b][ks]), qop[ks], s[b], 0, 0, 0);
        const int now[2] = {id[0], id[1]};
        // (Behind the last pair nothing is fetched, but by as many loads.)
        if ((i + 1) % (kWave / 2) == 0) fetch_ids(i + 1);
        id[0] = __builtin_amdgcn_readlane(ids, 2 * (i + 1) % kWave);
        id[1] = __builtin_amdgcn_readlane(ids, (2 * (i + 1) + 1) % kWave);
        load_k(id);
        float x[2][4];
        scores_of(s, a.scale_log2, tok0, row_len, (now[0] < 0) | (now[1] < 0) << 1, x);
        if constexpr (kScores) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
                if (c16 < a.group && now[b] >= 0)
                    *reinterpret_cast<f32x4 *>(a.scores + (((int64_t)now[b] * a.num_kv_heads + part.head) * a.group + c16) * kBlock + 4 * g4) =
                        f32x4{x[b][0], x[b][1], x[b][2], x[b][3]};
        }
        const bf16x8 p = st.take(x);
        if (tok0 + 2 * kBlock > part.longest) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) {
                    v[b][dt].x = seen_v(v[b][dt].x, tok0 + b * kBlock + 4 * g4, part.longest);
                    v[b][dt].y = seen_v(v[b][dt].y, tok0 + b * kBlock + 4 * g4 + 2, part.longest);
                }
        }
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            const u32x4 va = {v[0][dt].x, v[0][dt].y, v[1][dt].x, v[1][dt].y};
            st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), p, st.o[dt], 0, 0, 0);
        }
        load_v(id);
    }
    st.l = sum_xor_16_32(st.l);
}

// Where a part's state goes.
struct ShSink {
    float *ml;                     // [rows][2], or null
    float *acc;                    // [rows][D], or null: the output itself
    uint16_t *out;                 // [rows][D]
    int rows;
};

// Adds the waves' states of 16 rows up and writes them.
template <int D, int kMost>
__device__ __forceinline__ void merge(ShPlan<kMost> &sm, StageLds<D> *buf, const RowState<D> &st, const ShSink &sink) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c16 = lane % 16, g4 = lane / 16;
    // [wave][D / 16][64] of 16 bytes
    auto slot = [&](int w, int dt) { return reinterpret_cast<f32x4 *>(buf) + (w * (D / 16) + dt) * kWave + lane; };
    static_assert(sizeof(StageLds<D>) == kShWaves * (D / 16) * kWave * sizeof(f32x4), "a state per wave");
    if (g4 == 0) {
        sm.m[wave][c16] = st.m;
        sm.l[wave][c16] = st.l;
    }
    if (c16 < sink.rows)
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) *slot(wave, dt) = st.o[dt];
    __syncthreads();
    if (c16 < sink.rows) {
        float top = kNoMax, e[kShWaves], l = 0.f;
#pragma unroll
        for (int w = 0; w < kShWaves; ++w) top = fmaxf(top, sm.m[w][c16]);
#pragma unroll
        for (int w = 0; w < kShWaves; ++w) {
            e[w] = __builtin_amdgcn_exp2f(sm.m[w][c16] - top);
            l += e[w] * sm.l[w][c16];
        }
        const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
        for (int k = 0; k < D / 16 / kShWaves; ++k) {
            const int dt = wave + k * kShWaves, at = c16 * D + dt * 16 + 4 * g4;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kShWaves; ++w) x += *slot(w, dt) * e[w];
            if (sink.acc) *reinterpret_cast<f32x4 *>(sink.acc + at) = x;
            else *reinterpret_cast<uint2 *>(sink.out + at) =
                make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
        }
        if (sink.ml && wave == 0 && g4 == 0) {
            sink.ml[2 * c16] = top;
            sink.ml[2 * c16 + 1] = l;
        }
    }
    __syncthreads();                           // the next part writes there again
}

// More rows: tiles `wave` and `wave` + 4 of 16 of them are this wave's (count of them),
// and every pair of the part goes through LDS, two a stage: each wave loads one of a pair's
// four tiles into registers a stage ahead and stores it beside the stage at work.
template <int D>
__device__ __forceinline__ void tile_walk(const SharedArgs &a, const ShPart &part, StageLds<D> *buf, const uint16_t *const (&qrow)[2],
                                          const int (&row_len)[2], int count, float *ml, float *acc, int rows) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c16 = lane % 16, g4 = lane / 16;
    constexpr int kLoads = kBlock * D * 2 / 1024;        // of a tile, a kilobyte each
    const int pairs = (part.j1 - part.j0 + 1) / 2, stages = (pairs + 1) / 2;
    int ids = -1;                              // of 64 blocks, 16 stages
    auto fetch_ids = [&](int st) {
        ids = part_id(a, part, part.j0 + 4 * st + lane);
        __builtin_amdgcn_s_waitcnt(0x0F70);
    };
    bf16x8 qop[2][D / 32];
    RowState<D> rs[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) qop[r][ks] = *reinterpret_cast<const bf16x8 *>(qrow[r] + ks * 32 + g4 * 8);
        rs[r].clear();
    }
    u32x4 ahead[2][kLoads];                    // tile `wave` of each pair: K, K, V, V
    // Requests a stage (behind the last nothing, by as many loads); a bit per block that is absent.
    auto load = [&](int st) {
        if (st % (kWave / 4) == 0) fetch_ids(st);
        int absent = 0;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int id0 = __builtin_amdgcn_readlane(ids, (4 * st + 2 * p) % kWave), id1 = __builtin_amdgcn_readlane(ids, (4 * st + 2 * p + 1) % kWave);
            const __amdgpu_buffer_rsrc_t r = tile_rsrc<D>(a.pool, a.num_kv_heads, part.head, wave % 2 ? id1 : id0, wave >= 2);
#pragma unroll
            for (int kb = 0; kb < kLoads; ++kb) ahead[p][kb] = __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, kb * 1024, 0);
            absent |= (id0 < 0 ? 1 : 0) << (2 * p) | (id1 < 0 ? 2 : 0) << (2 * p);
        }
        return absent;
    };
    auto store = [&](int st) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int tok = (part.j0 + 4 * st + 2 * p + wave % 2) * kBlock;
            if (wave >= 2 && tok + kBlock > part.longest) {
                // 16 bytes: eight tokens of a dim
                const int t = tok + lane % 2 * 8;
#pragma unroll
                for (int kb = 0; kb < kLoads; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) ahead[p][kb][e] = seen_v(ahead[p][kb][e], t + 2 * e, part.longest);
            }
#pragma unroll
            for (int kb = 0; kb < kLoads; ++kb)
                *reinterpret_cast<u32x4 *>(buf[st & 1].tile[4 * p + wave] + kb * 1024 + lane * 16) = ahead[p][kb];
        }
    };
    int absent = load(0);
    store(0);
    int absent_next = load(1);
#pragma unroll 1
    for (int st = 0; st < stages; ++st) {
        // The stage's stores are done; loads stay in flight.
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);    // lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (count)
#pragma unroll 1
            for (int p = 0; p < min(2, pairs - 2 * st); ++p) {
                const uint8_t(*t)[kBlock * D * 2] = buf[st & 1].tile + 4 * p;
                const int tok0 = (part.j0 + 4 * st + 2 * p) * kBlock;
                f32x4 s[2][2] = {};
#pragma unroll
                for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const bf16x8 k = *reinterpret_cast<const bf16x8 *>(t[b] + ks * 1024 + lane * 16);
#pragma unroll
                        for (int r = 0; r < 2; ++r) s[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qop[r][ks], s[r][b], 0, 0, 0);
                    }
                bf16x8 pr[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float x[2][4];
                    scores_of(s[r], a.scale_log2, tok0, row_len[r], absent >> (2 * p), x);
                    pr[r] = rs[r].take(x);
                }
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) {
                    const int at = (dt * 16 + c16) * kBlock * 2 + g4 * 8;
                    const u32x2 v0 = *reinterpret_cast<const u32x2 *>(t[2] + at), v1 = *reinterpret_cast<const u32x2 *>(t[3] + at);
                    const u32x4 va = {v0.x, v0.y, v1.x, v1.y};
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        rs[r].o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), pr[r], rs[r].o[dt], 0, 0, 0);
                }
            }
        store(st + 1);                         // (the stage before, whose buffer it is, was left at the barrier)
        absent = absent_next;
        absent_next = load(st + 2);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = (wave + r * kShWaves) * 16 + c16;
        const float l = sum_xor_16_32(rs[r].l);
        if (row < rows) {
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4 *>(acc + (int64_t)row * D + dt * 16 + 4 * g4) = rs[r].o[dt];
            if (g4 == 0) *reinterpret_cast<float2 *>(ml + 2 * row) = make_float2(rs[r].m, l);
        }
    }
    __syncthreads();
}

template <int D, int kMost, bool kWeights>
__global__ __launch_bounds__(kShThreads, kMost == kShFew ? kShPerCu : 1) void shared_kernel(SharedArgs a) {
    __shared__ ShPlan<kMost> sm;
    __shared__ StageLds<D> buf[2];
    int32_t *const owner = reinterpret_cast<int32_t *>(buf[0].tile[0]);   // a session's place among the members, or -1
    static_assert(kShMost * 4 <= sizeof(StageLds<D>), "owners fit a buffer");
    const int tid = threadIdx.x, lane = tid % kWave, c16 = lane % 16;
    const int S = a.num_sessions, G = a.group, H = a.num_kv_heads;
    const bool first_wg = blockIdx.x == 0;
    const int gs = __builtin_ctz(G);           // (G is 1, 2, 4 or 8)
    // ---- the schedule, made by every workgroup for itself (its loads all at once)
    constexpr int kPer = kMost / kShThreads;
    int32_t *const len = reinterpret_cast<int32_t *>(buf[1].tile[0]);
    int ng = a.num_groups;
    bool bad = false;
    {
        int ld_len[kPer], ld_member[kPer], ld_x[kPer], ld_y[kPer], ld_pb[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = tid + k * kShThreads;
            ld_len[k] = a.lens[min(i, S - 1)];
            if (ng) {
                ld_member[k] = a.members[min(i, a.num_members - 1)];
                ld_x[k] = a.starts[min(i, ng)];
                ld_y[k] = a.starts[min(i + 1, ng)];
                ld_pb[k] = a.prefix[min(i, ng - 1)];
            }
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = tid + k * kShThreads;
            if (i < S) {
                owner[i] = -1;
                if (first_wg && (ld_len[k] < 0 || ld_len[k] > a.max_blocks * kBlock)) flag_error(a.err, LS_DEVERR_LENGTH);
                len[i] = max(min(ld_len[k], a.max_blocks * kBlock), 0);
            }
            if (i < ng) {
                const int x = ld_x[k], y = ld_y[k], pb = ld_pb[k];
                bad = bad || x < 0 || y < x || y > a.num_members || pb < 0 || pb > a.max_blocks || (i == 0 && x != 0) ||
                      (i == ng - 1 && y != a.num_members);
                sm.start[i] = (uint16_t)x;
                if (i == ng - 1) sm.start[ng] = (uint16_t)y;
                sm.prefix[i] = (uint16_t)pb;
                sm.lead[i] = 0u;
            }
        }
        bad = __syncthreads_or(bad);
        if (ng && !bad) {
            bool wrong = false;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int i = tid + k * kShThreads, s = ld_member[k];
                if (i >= a.num_members) continue;
                if (s < 0 || s >= S) {
                    wrong = true;
                    continue;
                }
                int lo = 0, hi = ng;           // the last group that starts at or before i
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (sm.start[mid] <= i) lo = mid;
                    else hi = mid;
                }
                if (atomicExch(&owner[s], i) != -1) wrong = true;
                sm.gid[s] = (uint16_t)lo;
                atomicMax(&sm.lead[lo], (uint32_t)len[s] << kRank | (uint32_t)(kShMost - 1 - (i - sm.start[lo])));
            }
            bad = __syncthreads_or(wrong);
            if (!bad)
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const int i = tid + k * kShThreads, s = ld_member[k];
                    if (i >= a.num_members) continue;
                    const int g = sm.gid[s];
                    if (kShMost - 1 - (i - sm.start[g]) == (int)(sm.lead[g] & (kShMost - 1))) sm.lead_s[g] = (uint16_t)s;
                }
        }
    }
    if (bad) {
        // Groups that cannot be: every session is computed on its own, and no weight is kept.
        if (first_wg && tid == 0) flag_error(a.err, LS_DEVERR_GROUP);
        ng = 0;
        __syncthreads();
        for (int s = tid; s < S; s += kShThreads) owner[s] = -1;
    }
    {
        const int per = (ng + kShThreads - 1) / kShThreads;
        unsigned v[2] = {0, 0}, all[2];
        for (int g = tid * per; g < min(ng, (tid + 1) * per); ++g) {
            const int rows = (sm.start[g + 1] - sm.start[g]) * G, longest = (int)(sm.lead[g] >> kRank);
            const int pb = min((int)sm.prefix[g], (longest + kBlock - 1) / kBlock);
            sm.prefix[g] = (uint16_t)pb;
            v[0] += (unsigned)group_cost(rows, pb);
            v[1] += (unsigned)tile_places(rows);
        }
        if (ng) scan2(v, all, sm.scan);
        else all[0] = all[1] = 0u;
        for (int g = tid * per; g < min(ng, (tid + 1) * per); ++g) {
            const int rows = (sm.start[g + 1] - sm.start[g]) * G;
            sm.units[g] = v[0];
            sm.segs[g] = (uint16_t)v[1];
            v[0] += (unsigned)group_cost(rows, sm.prefix[g]);
            v[1] += (unsigned)tile_places(rows);
        }
        if (tid == 0) {
            sm.units[ng] = all[0];
            sm.segs[ng] = (uint16_t)all[1];
        }
    }
    __syncthreads();
    {
        const int per = (S + kShThreads - 1) / kShThreads;
        unsigned v[2] = {0, 0}, all[2];
        auto own = [&](int s, int pb) { return (unsigned)max((len[s] + kBlock - 1) / kBlock - pb, 0); };
        for (int s = tid * per; s < min(S, (tid + 1) * per); ++s) {
            // A member that does not see all of the prefix's keys is computed on its own: 0 x V of a key that
            // the others see is NaN where that V is not finite.
            int pb = 0;
            if (owner[s] >= 0) {
                const int g = sm.gid[s], all_pb = sm.prefix[g], longest = (int)(sm.lead[g] >> kRank);
                if (len[s] >= min(all_pb * kBlock, longest)) pb = all_pb;
            }
            sm.pb[s] = (uint16_t)pb;
            sm.pad[s] = (uint8_t)(-len[s] & (kBlock - 1));
            const unsigned n = own(s, sm.pb[s]);
            v[0] += n;
            v[1] += n ? n + kCostPart : 0u;
        }
        scan2(v, all, sm.scan);
        for (int s = tid * per; s < min(S, (tid + 1) * per); ++s) {
            const unsigned n = own(s, sm.pb[s]);
            sm.cum[s] = v[0];
            sm.cost[s] = v[1];
            v[0] += n;
            v[1] += n ? n + kCostPart : 0u;
        }
        if (tid == 0) {
            sm.cum[S] = all[0];
            sm.cost[S] = all[1];
        }
    }
    __syncthreads();
    if (first_wg) {
        for (int s = tid; s < S; s += kShThreads) {
            ShRecord r = {};
            r.own_blocks = (int)(sm.cum[s + 1] - sm.cum[s]);
            r.own_before = sm.cum[s];
            r.own_all = sm.cum[S];
            // (which blocks are shared is not known of groups that cannot be: their scores and entries are several sessions')
            r.keys = bad ? 0 : len[s];
            if (owner[s] >= 0) {
                const int g = sm.gid[s], row = (owner[s] - sm.start[g]) * G, size = tile_size((sm.start[g + 1] - sm.start[g]) * G);
                r.prefix_blocks = sm.pb[s];
                if (!sm.pb[s] && sm.prefix[g]) r.keys = 0;           // (all of them are the prefix's)
                r.tile_seg = H * sm.segs[g] + row / size * (size / kFewRows);
                r.tile_seg_stride = sm.segs[g + 1] - sm.segs[g];
                r.tile_row = row % size;
            }
            a.records[s] = r;
        }
    }
    __syncthreads();                           // the buffers of owners and lengths are used again
    // Workgroups for prefixes and for own blocks, the same of each on every XCD (8, where workgroup b
    // runs on b % 8), and consecutive shares on one: the tiles of a group and KV head read the same K and V.
    // (There are two workgroups at least, so both kinds get one where there is work of both.)
    const int W = gridDim.x, xcds = W % 8 || W < 16 ? 1 : 8, b = blockIdx.x / xcds, x = blockIdx.x % xcds;
    const int units_tile = H * (int)sm.units[ng], units_own = H * (int)sm.cost[S];
    int tile_wgs = units_tile ? (int)((float)(W / xcds) * units_tile / ((float)units_tile + units_own) + 0.5f) : 0;
    if (units_tile) tile_wgs = max(tile_wgs, 1);
    if (units_own) tile_wgs = min(tile_wgs, W / xcds - 1);
    const int own_wgs = W / xcds - tile_wgs;
    // Blocks of the segment at `pos` that are in [u0, u1).
    auto range = [](int u0, int u1, int pos, int blocks, int cost, int &j0, int &j1) {
        const int from = pos + kCostPart;
        j0 = u0 > from ? min((u0 - from + cost - 1) / cost, blocks) : 0;
        j1 = u1 > from ? min((u1 - from + cost - 1) / cost, blocks) : 0;
    };
    auto prefix_tiles = [&]() {
        const int n = tile_wgs * xcds, wp = x * tile_wgs + b, all = units_tile, share = max((all + n - 1) / n, kLeastTile);
        if (wp > all / share) return;
        const int at = wp * share, u1 = min(at + share, all);
        if (at >= u1) return;
        int g = 0, hi = ng;
        while (hi - g > 1) {
            const int mid = (g + hi) / 2;
            if (H * (int)sm.units[mid] <= at) g = mid;
            else hi = mid;
        }
        for (; g < ng && H * (int)sm.units[g] < u1; ++g) {
            const int stride = (int)(sm.units[g + 1] - sm.units[g]);
            if (!stride) continue;
            const int pb = sm.prefix[g], first = sm.start[g], rows = (sm.start[g + 1] - first) * G;
            const int size = tile_size(rows), tiles = (rows + size - 1) / size, full = pb * tile_cost(size) + kCostPart;
            const int gpos = H * (int)sm.units[g];
            const int lead_s = sm.lead_s[g];
            for (int h = at > gpos ? (at - gpos) / stride : 0; h < H && gpos + h * stride < u1; ++h) {
                const int hpos = gpos + h * stride;
                for (int t = at > hpos ? (at - hpos) / full : 0; t < tiles; ++t) {
                    const int pos = hpos + t * full;
                    if (pos >= u1) break;
                    const int n = min(size, rows - t * size);
                    ShPart part;
                    range(at, u1, pos, pb, tile_cost(n), part.j0, part.j1);
                    if (part.j0 >= part.j1) continue;
                    part.table = a.tables + (int64_t)lead_s * a.max_blocks;
                    part.head = h;
                    part.longest = (int)(sm.lead[g] >> kRank);
                    const int seg = H * sm.segs[g] + (h * tiles + t) * (size / kFewRows);
                    const int64_t row0 = (int64_t)seg * kFewRows + (int64_t)wp * kTileRows;
                    float *ml = a.tile_ml + row0 * 2, *acc = a.tile_acc + row0 * D;
                    if (tid == 0) {
                        if (part.j0 == 0) a.tile_first[seg] = wp;
                        if (part.j1 == pb) a.tile_last[seg] = wp;
                    }
                    // (lanes of no row take the last one: a load under a condition waits for the one before)
                    auto row_of = [&](int row, const uint16_t *&qrow, int &len) {
                        const int x = t * size + min(row, n - 1), s = a.members[first + (x >> gs)];
                        qrow = a.q + ((int64_t)s * H * G + h * G + (x & (G - 1))) * D;
                        len = keys_of(a, s);
                    };
                    if (n <= 16) {
                        const uint16_t *qrow;
                        int row_len;
                        row_of(c16, qrow, row_len);
                        RowState<D> st;
                        walk<D, false, 0>(a, part, qrow, row_len, st);
                        merge<D>(sm, buf, st, ShSink{ml, acc, nullptr, n});
                    } else {
                        const int wave = tid / kWave;
                        const uint16_t *qrow[2];
                        int row_len[2];
                        row_of(wave * 16 + c16, qrow[0], row_len[0]);
                        row_of((wave + kShWaves) * 16 + c16, qrow[1], row_len[1]);
                        const int count = (wave * 16 < n) + ((wave + kShWaves) * 16 < n);
                        tile_walk<D>(a, part, buf, qrow, row_len, count, ml, acc, n);
                    }
                }
            }
        }
    };
    auto own_keys = [&]() {
        const int n = own_wgs * xcds, wo = x * own_wgs + b - tile_wgs, all = units_own, share = max((all + n - 1) / n, kLeastOwn);
        if (wo > all / share) return;
        const int at = wo * share, u1 = min(at + share, all);
        if (at >= u1) return;
        const int rel = at / H;                 // units per KV head before
        int s = 0, hi = S;                      // the last session that starts at or before it
        while (hi - s > 1) {
            const int mid = (s + hi) / 2;
            if ((int)sm.cost[mid] <= rel) s = mid;
            else hi = mid;
        }
        for (; s < S; ++s) {
            const int spos = H * (int)sm.cost[s];
            if (spos >= u1) break;
            const int nb = (int)(sm.cum[s + 1] - sm.cum[s]);
            if (!nb) continue;
            const int pb = sm.pb[s], L = (pb + nb) * kBlock - sm.pad[s];
            for (int h = at > spos ? (at - spos) / (nb + kCostPart) : 0; h < H; ++h) {
                const int pos = spos + h * (nb + kCostPart);
                if (pos >= u1) break;
                int j0, j1;
                range(at, u1, pos, nb, 1, j0, j1);
                if (j0 >= j1) continue;
                const ShPart part = {a.tables + (int64_t)s * a.max_blocks, h, pb + j0, pb + j1, L};
                const bool whole = !pb && j0 == 0 && j1 == nb;
                const int seg = s * H + h;
                const int64_t slot = (int64_t)seg + wo, row0 = (int64_t)seg * G;
                if (tid == 0) {
                    if (j0 == 0) a.own_first[seg] = wo;
                    if (j1 == nb) a.own_last[seg] = wo;
                }
                const ShSink sink = {!whole || kWeights ? a.own_ml + slot * G * 2 : nullptr, whole ? nullptr : a.own_acc + slot * G * D,
                                     a.out + row0 * D, G};
                RowState<D> st;
                walk<D, kWeights, kStream>(a, part, a.q + (row0 + min(c16, G - 1)) * D, L, st);
                merge<D>(sm, buf, st, sink);
            }
        }
    };
    if (b < tile_wgs) prefix_tiles();
    else own_keys();
}

// The parts of a row: those of its prefix tile, then its own.
struct RowParts {
    int prefix, own;               // how many
    int64_t prefix_row, own_row;   // rows of the first ones in tile_ml, own_ml
};
__device__ __forceinline__ RowParts parts_of(const SharedArgs &a, const ShRecord &r, int s, int h, int head) {
    RowParts p = {0, 0, 0, 0};
    const int seg = s * a.num_kv_heads + h, tile = r.tile_seg + h * r.tile_seg_stride;
    if (r.prefix_blocks) {
        const int w = a.tile_first[tile];
        p.prefix = a.tile_last[tile] - w + 1;
        p.prefix_row = (int64_t)tile * kFewRows + (int64_t)w * kTileRows + r.tile_row + head;
    }
    if (r.own_blocks) {
        const int w = a.own_first[seg];
        p.own = a.own_last[seg] - w + 1;
        p.own_row = ((int64_t)seg + w) * a.group + head;
    }
    return p;
}

// Workgroups below `combine` add up rows of the output, D / 4 threads a row; the waves of
// the others take equal shares of the own blocks and add their probabilities to the
// weights, four threads a (block, KV head).  Bound by the scores' scattered reads: 64 long
// sessions 17 us for 70 MB read and written (19 with shares of a workgroup each), one of 1789
// tokens 3.8.
template <int D, bool kWeights>
__global__ __launch_bounds__(kShThreads) void shared_merge_kernel(SharedArgs a, int combine) {
    __shared__ uint32_t sm_cum[kWeights ? kShMost + 1 : 1];
    const int tid = threadIdx.x, H = a.num_kv_heads, G = a.group, S = a.num_sessions;
    if ((int)blockIdx.x < combine) {
        constexpr int kLanes = D / 4, kAhead = 8;
        const int64_t row = (int64_t)blockIdx.x * (kShThreads / kLanes) + tid / kLanes;
        if (row >= (int64_t)S * H * G) return;
        const int s = (int)(row / (H * G)), h = (int)(row % (H * G)) / G, e4 = tid % kLanes * 4;
        const ShRecord r = a.records[s];
        const RowParts n = parts_of(a, r, s, h, (int)(row % G));
        if (n.own == 1 && !n.prefix) return;               // written already
        // kAhead parts at a time, so that their loads are in flight together
        float top = kNoMax, sum = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        const int parts = n.prefix + n.own;
        for (int i0 = 0; i0 < parts; i0 += kAhead) {
            float2 ml[kAhead];
            f32x4 o[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int i = min(i0 + k, parts - 1);
                const bool tile = i < n.prefix;
                const int64_t at = tile ? n.prefix_row + (int64_t)i * kTileRows : n.own_row + (int64_t)(i - n.prefix) * G;
                ml[k] = reinterpret_cast<const float2 *>(tile ? a.tile_ml : a.own_ml)[at];
                o[k] = *reinterpret_cast<const f32x4 *>((tile ? a.tile_acc : a.own_acc) + at * D + e4);
            }
            float now = top;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) now = fmaxf(now, ml[k].x);
            const float old = __builtin_amdgcn_exp2f(top - now);
            sum *= old;
            x *= old;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const float e = i0 + k < parts ? __builtin_amdgcn_exp2f(ml[k].x - now) : 0.f;
                if (i0 + k < parts) {
                    sum += e * ml[k].y;
                    x += o[k] * e;
                }
            }
            top = now;
        }
        const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
        *reinterpret_cast<uint2 *>(a.out + row * D + e4) =
            make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
        return;
    }
    if constexpr (kWeights) {
        for (int s = tid; s < S; s += kShThreads) sm_cum[s] = a.records[s].own_before;
        const uint32_t own_all = a.records[0].own_all;
        if (tid == 0) sm_cum[S] = own_all;
        __syncthreads();
        // Shares are a wave's: with a workgroup's, the second segment of a share waited for the first.
        constexpr int kQuads = kWave / 4;                            // blocks at a time
        const int lane = tid % kWave;
        const int all = (int)own_all * H, n = (gridDim.x - combine) * kShWaves, w = (blockIdx.x - combine) * kShWaves + tid / kWave;
        const int per = max((all + n - 1) / n, kQuads);
        if (w > all / per) return;
        const int b0 = w * per, b1 = min(b0 + per, all);
        if (b0 >= b1) return;
        int s = 0, hi = S;
        while (hi - s > 1) {
            const int mid = (s + hi) / 2;
            if ((int)sm_cum[mid] * H <= b0) s = mid;
            else hi = mid;
        }
        for (; s < S && (int)sm_cum[s] * H < b1; ++s) {
            const ShRecord r = a.records[s];
            if (!r.own_blocks) continue;
            const int first = a.first ? a.first[s] : 0;
            const int old = a.reused ? a.reused[s] : INT32_MAX;      // keys from here on are new
            const int begin = a.reused ? (a.begin ? a.begin[s] : old) : 0;
            const int spos = (int)sm_cum[s] * H;
            for (int h = b0 > spos ? (b0 - spos) / r.own_blocks : 0; h < H; ++h) {
                const int pos = spos + h * r.own_blocks;
                if (pos >= b1) break;
                // The rows' whole sums: lane = (part, query head), eight parts at a time
                float top = kNoMax, sum = 0.f;
                {
                    const RowParts p = parts_of(a, r, s, h, min(lane % 8, G - 1));
                    for (int i = lane / 8; i < p.prefix + p.own; i += kWave / 8) {
                        const bool tile = i < p.prefix;
                        const int64_t row = tile ? p.prefix_row + (int64_t)i * kTileRows : p.own_row + (int64_t)(i - p.prefix) * G;
                        const float2 ml = reinterpret_cast<const float2 *>(tile ? a.tile_ml : a.own_ml)[row];
                        const float now = fmaxf(top, ml.x);
                        sum = sum * __builtin_amdgcn_exp2f(top - now) + ml.y * __builtin_amdgcn_exp2f(ml.x - now);
                        top = now;
                    }
#pragma unroll
                    for (int off = 8; off < kWave; off <<= 1) {
                        const float t2 = __shfl_xor(top, off), s2 = __shfl_xor(sum, off), now = fmaxf(top, t2);
                        sum = sum * __builtin_amdgcn_exp2f(top - now) + s2 * __builtin_amdgcn_exp2f(t2 - now);
                        top = now;
                    }
                }
                const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                const int j0 = max(b0 - pos, 0), j1 = min(b1 - pos, r.own_blocks);
                for (int j = j0 + lane / 4; j - lane / 4 < j1; j += kQuads) {
                    const int col = r.prefix_blocks + j, t0 = col * kBlock + lane % 4 * 4;
                    const int id = j < j1 ? a.tables[(int64_t)s * a.max_blocks + col] : -1;
                    const bool use = id >= 0 && id < a.num_blocks && t0 < r.keys && t0 + 4 > first;
                    const int64_t tile = (int64_t)(use ? id : 0) * H + h, at = tile * kBlock + lane % 4 * 4;
                    const float *x = a.scores + tile * G * kBlock + lane % 4 * 4;
                    const f32x4 was = *reinterpret_cast<const f32x4 *>(a.weights + at);
                    f32x4 p = {0.f, 0.f, 0.f, 0.f}, y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = *reinterpret_cast<const f32x4 *>(x + min(k, G - 1) * kBlock);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float m = __shfl(top, k), scale = k < G ? __shfl(inv, k) : 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (k < G) p[e] += __builtin_amdgcn_exp2f(y[k][e] - m) * scale;
                    }
                    if (!use) continue;
                    if (t0 >= first && t0 + 4 <= r.keys && t0 + 4 <= old) {
                        *reinterpret_cast<f32x4 *>(a.weights + at) = was + p;
                        continue;
                    }
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
    const bool few = a.num_sessions <= kShFew;               // (members and groups are no more)
#define LS_SHARED(MOST, W) hipLaunchKernelGGL((shared_kernel<D, MOST, W>), dim3(grid), dim3(kShThreads), 0, stream, a)
    if (a.weights) {
        if (few) LS_SHARED(kShFew, true);
        else LS_SHARED(kShMost, true);
    } else {
        if (few) LS_SHARED(kShFew, false);
        else LS_SHARED(kShMost, false);
    }
#undef LS_SHARED
    if (hipError_t e = hipGetLastError()) return e;
    if (a.weights)
        hipLaunchKernelGGL((shared_merge_kernel<D, true>), dim3(combine + 2 * grid), dim3(kShThreads), 0, stream, a, combine);
    else
        hipLaunchKernelGGL((shared_merge_kernel<D, false>), dim3(combine), dim3(kShThreads), 0, stream, a, combine);
    return hipGetLastError();
}

constexpr size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

SharedPlan plan_shared(const PoolGeom &p, int32_t num_sessions, int32_t num_q_heads, int32_t num_groups,
                       int32_t num_members, bool weights) {
    const int64_t H = p.num_kv_heads, G = num_q_heads / p.num_kv_heads, W = kShPerCu * (p.num_cus > 0 ? p.num_cus : 256);
    SharedPlan s;
    // (a slot per segment and one per workgroup.  A group's rows round up to 16, those of more than 64 to 128.)
    const int64_t rows = (int64_t)num_members * G, large = std::min<int64_t>(num_groups, rows / (kFewMost + 1));
    const size_t tiles = num_groups ? (size_t)(H * (rows / kFewRows + num_groups + (kTileRows / kFewRows - 1) * large)) : 0;
    const size_t tile_rows = num_groups ? tiles * kFewRows + (size_t)W * kTileRows : 0, own_slots = (size_t)(num_sessions * H + W);
    const size_t sizes[] = {(size_t)num_sessions * sizeof(ShRecord),
                            tiles * 2 * sizeof(int32_t),
                            (size_t)(num_sessions * H) * 2 * sizeof(int32_t),
                            tile_rows * 2 * sizeof(float),
                            tile_rows * (size_t)p.head_dim * sizeof(float),
                            own_slots * (size_t)G * 2 * sizeof(float),
                            own_slots * (size_t)G * (size_t)p.head_dim * sizeof(float),
                            weights ? (size_t)p.num_blocks * (size_t)num_q_heads * kBlock * sizeof(float) : 0};
    static_assert(sizeof sizes / sizeof *sizes == sizeof s.at / sizeof *s.at, "an offset each");
    s.tiles = tiles;
    s.total = 0;
    for (size_t i = 0; i < sizeof sizes / sizeof *sizes; ++i) {
        s.at[i] = s.total;
        s.total += align256(sizes[i]);
    }
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
    a.records = reinterpret_cast<ShRecord *>(ws + plan.at[0]);
    a.tile_first = reinterpret_cast<int32_t *>(ws + plan.at[1]);
    a.tile_last = a.tile_first + plan.tiles;
    a.own_first = reinterpret_cast<int32_t *>(ws + plan.at[2]);
    a.own_last = a.own_first + (int64_t)num_sessions * p.num_kv_heads;
    a.tile_ml = reinterpret_cast<float *>(ws + plan.at[3]);
    a.tile_acc = reinterpret_cast<float *>(ws + plan.at[4]);
    a.own_ml = reinterpret_cast<float *>(ws + plan.at[5]);
    a.own_acc = reinterpret_cast<float *>(ws + plan.at[6]);
    a.scores = reinterpret_cast<float *>(ws + plan.at[7]);
    const int64_t entries = (int64_t)layer * p.num_blocks * p.num_kv_heads * kBlock;
    a.weights = c.weights ? c.weights + entries : nullptr;
    a.positions = c.positions ? c.positions + entries : nullptr;
    a.reused = c.reused_lens;
    a.begin = c.first_positions;
    a.first = c.first_lens;
    a.err = err;
    const int cus = stream_cus(p, stream), most = p.num_cus > 0 ? p.num_cus : 256;
    const int grid = kShPerCu * std::min(cus, most);
    return p.head_dim == 128 ? launch_shared_t<128>(a, grid, stream) : launch_shared_t<64>(a, grid, stream);
}

}  // namespace ls
