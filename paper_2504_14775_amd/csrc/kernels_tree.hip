// Attention of trees of drafted tokens over the paged pool (contract: include/gllm_branch.h).
//
// A sequence has n nodes, whose keys and values stand behind its c cached ones, and node i sees the c cached positions, its
// ancestors and itself.  Per KV head the n nodes times the g query heads of the group are n*g independent columns over one
// stream of keys: S^T = K.Q^T, softmax down the columns with a running reference, O^T += V^T.P^T, by the inner step of
// attn_core.h.  Column j is head j % g of node j / g, so that any g fills the groups of 16 columns.
//
// Which keys a column sees differs in the last blocks only (blocks of 32 keys; the tree starts in block c / 32): there a
// node has one 32-bit word per block, bit k for key k of the block, from the closure of the parent links (tree_visibility).
// Everything in front is seen by all columns and goes through a loop without masks.
//
// Work: 4 * d * columns multiplications and additions per key and KV head against 4 * d bytes of keys and values, so the kernels go with
// the keys' stream from HBM up to some 200 columns, and with the inner step (matrix and vector instructions) above.  Measured (one layer;
// keys in HBM; means of thirty launches): 32 single tokens behind 300 to 20000 keys (32 heads on 8, 615 MB) 99 + 4.8 us, 6.2 TB/s; 16 trees of 64
// nodes behind 1000 to 8000 (64 on 8) 178 to 187 + 18.5 us on three cards, the second figure the joining of the parts (the fastest 163 + 16.4); calls
// that follow one another without a profiler take 102 and 168.
#include "attn_core.h"

#include <atomic>

namespace {

constexpr int kTreeNodes = kMaxTreeNodes;   // one per thread
static_assert(kTreeNodes == 256, "a node per thread of a workgroup");
constexpr int kTreeWords = kTreeNodes / 32;
constexpr int kTreeStages = 3;

// A unit of work: the keys of blocks blk_begin .. blk_end - 1 for the columns of one tile of a sequence.
struct TreeUnit {
    int32_t seq, tile, row0, n, c;
    int32_t blk_begin, blk_end;  // equal where the sequence breaks a rule: zeros
    int32_t parts, part;
    int32_t slot;                // parts > 1: place of the unit among those with partial results
    int32_t cut_tile;            // and of its tile among those with such units
};

// What the closure of a tree takes in LDS: rows of `stride` words per node (odd, so that neighbouring nodes lie in different
// banks), the words of the nodes that are used, and, above 64 nodes, the parent links.
struct TreeLds {
    uint32_t* vis;    // [nodes][stride]: word w of a node: keys 32w .. 32w+31 behind the first key of block c / 32
    uint32_t* used;   // [kTreeWords + 1], as a row of vis: all cached keys and all used nodes
    uint32_t* raw;    // [kTreeWords]
    int* up;          // [nodes]
    int nodes, words, stride;
    __host__ __device__ TreeLds(void* p, int max_nodes) {
        nodes = max_nodes <= 64 ? max_nodes : kTreeNodes;
        words = (max_nodes + 31) / 32 + 1;
        stride = words | 1;
        used = (uint32_t*)p;
        raw = used + kTreeWords + 1;
        vis = raw + kTreeWords;
        up = (int*)(vis + nodes * stride);
    }
    __host__ __device__ int bytes(int max_nodes) const { return (2 * kTreeWords + 1 + nodes * stride + (max_nodes > 64 ? nodes : 0)) * 4; }
};

// The words of all nodes of a tree of n nodes behind c cached keys.  Every round joins to a node's set that of the node at the
// end of its link and doubles the link: a tree is done in log2 of its depth rounds.  A link that leads to no root is -2 at the
// end, and the node's words are zero.
//
// Up to 64 nodes, one per lane: every wave does it for itself, in registers, and all write the same words (no barrier).
__device__ __forceinline__ void tree_visibility_wave(const TreeLds& t, int given, int n, int c) {
    const int i = threadIdx.x & 63, sh = c & 31;
    int p = i < n && given >= -1 && given < i ? given : -2;
    uint64_t set = 1ull << i;
    while (__any(p >= 0)) {
        const int from = max(p, 0);
        const uint32_t lo = __shfl((int)(uint32_t)set, from), hi = __shfl((int)(uint32_t)(set >> 32), from);
        const int next = __shfl(p, from);
        if (p >= 0) {
            set |= (uint64_t)hi << 32 | lo;
            p = next;
        }
    }
    const uint64_t used = __ballot(p == -1);
    const uint32_t prefix = (1u << sh) - 1u;  // every used node sees the cached keys of the first block
    auto words = [&](uint64_t bits, uint32_t* to, bool on) {
        const uint32_t lo = (uint32_t)bits, hi = (uint32_t)(bits >> 32);
        to[0] = on ? lo << sh | prefix : 0u;
        if (t.words > 1) to[1] = on ? (uint32_t)(bits << sh >> 32) : 0u;
        if (t.words > 2) to[2] = on && sh ? hi >> (32 - sh) : 0u;
    };
    if (i < t.nodes) words(set, t.vis + i * t.stride, p == -1);
    if (i == 0) words(used, t.used, true);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Up to 256 nodes, one per thread; ends with a barrier.
__device__ __forceinline__ void tree_visibility_group(const TreeLds& t, int given, int n, int c) {
    const int i = threadIdx.x, words = t.words - 1, sh = c & 31;
    uint32_t* mine = t.vis + i * t.stride;
    int p = i < n && given >= -1 && given < i ? given : -2;
    t.up[i] = p;
    for (int w = 0; w < words; ++w) mine[w] = w == i >> 5 ? 1u << (i & 31) : 0u;
    __syncthreads();
    for (;;) {
        uint32_t b[kTreeWords];
        int next = p;
        if (p >= 0) {
            next = t.up[p];
#pragma unroll
            for (int w = 0; w < kTreeWords; ++w) b[w] = w < words ? t.vis[p * t.stride + w] : 0u;
        }
        if (!__syncthreads_or(p >= 0)) break;
        if (p >= 0) {
#pragma unroll
            for (int w = 0; w < kTreeWords; ++w)
                if (w < words) mine[w] |= b[w];
            t.up[i] = next;
        }
        p = next;
        __syncthreads();
    }
    const uint64_t valid = __ballot(p == -1);
    if ((i & 63) == 0) {
        t.raw[i / 32] = (uint32_t)valid;
        t.raw[i / 32 + 1] = (uint32_t)(valid >> 32);
    }
    uint32_t low = 0u;  // moved up by the cached keys of the first block, which every used node sees
    const uint32_t prefix = (1u << sh) - 1u;
    for (int w = 0; w <= words; ++w) {
        const uint32_t b = w < words ? mine[w] : 0u;
        const uint32_t moved = (uint32_t)((((uint64_t)b << 32 | low) << sh) >> 32) | (w == 0 ? prefix : 0u);
        mine[w] = p == -1 ? moved : 0u;
        low = b;
    }
    __syncthreads();
    if (i <= words) {
        const uint32_t b = i < words ? t.raw[i] : 0u, below = i > 0 ? t.raw[i - 1] : 0u;
        t.used[i] = (uint32_t)((((uint64_t)b << 32 | below) << sh) >> 32) | (i == 0 ? prefix : 0u);
    }
    __syncthreads();
}

// The parent of this thread's node, fetched in front of the rest; all threads call the other with it.
__device__ __forceinline__ int tree_parent(const TreeArgs& a, int row0, int n) {
    const int i = a.max_nodes <= 64 ? threadIdx.x & 63 : threadIdx.x;
    return i < n ? a.parents[row0 + i] : -2;
}
__device__ __forceinline__ void tree_visibility(const TreeArgs& a, const TreeLds& t, int given, int n, int c) {
    if (a.max_nodes <= 64) tree_visibility_wave(t, given, n, c);
    else tree_visibility_group(t, given, n, c);
}

// ---- the plan --------------------------------------------------------------------------------------------------------------
//
// The lengths stand on the device.  The keys of a sequence are cut into parts of at most `share` blocks, equal to within one
// block, so that all parts of all sequences come to about tree_target workgroups; the tiles of a part, neighbours in the launch but for
// the KV heads, read the same keys at the same time.
constexpr int kTreeMinShare = 8;      // fewest blocks worth a workgroup
// Workgroups that the keys are cut into, over all KV heads: as many as run at one time.  Every part of a tile writes and reads partial
// results of (d + 2) floats a column, at 64 columns as much as four blocks of keys.  us at 512 / 768 / 1024 / 2048: one sequence of 30000
// keys, 64 nodes (8B heads) 58 / 69 / 75 / 98, 64 sequences of 500 to 4000 keys, 8 nodes (70B heads) 108 / 118 / 118 / 131.  Of 16 columns they
// are small, and shorter parts fill the end of the launch better: 32 single tokens behind 300 to 20000 keys 105 / 102 / 103 / 107.
constexpr int tree_target(int n_kv, int tile_cols) { return (tile_cols == 16 ? 768 : 512) / n_kv > 0 ? (tile_cols == 16 ? 768 : 512) / n_kv : 1; }
// Units with partial results: a sequence is cut where it has more blocks than a share, and then into fewer parts than twice its
// blocks by the share; a share is at least the blocks of all tiles by the target.
constexpr int tree_max_slots(int n_kv, int tile_cols) { return 2 * tree_target(n_kv, tile_cols); }
// (and their tiles: every one of them has more blocks than a share)
constexpr int tree_max_cut_tiles(int n_kv, int tile_cols) { return tree_target(n_kv, tile_cols); }

struct SeqPlan {
    int32_t row0, n, c, tiles, blocks;
    bool bad;  // its rows break the order of the rows
};
__device__ __forceinline__ SeqPlan seq_plan(const TreeArgs& a, int s, int tile_cols) {
    SeqPlan p{0, 0, 0, 0, 0, false};
    if (s >= a.num_seqs) return p;
    const int r0 = a.row_begin[s], r1 = a.row_end[s];
    p.c = a.cached_len[s];
    p.bad = r0 < 0 || r1 < r0 || r1 > a.num_rows;
    p.row0 = r0;
    p.n = p.bad ? 0 : r1 - r0;
    p.tiles = (p.n * (a.n_q / a.n_kv) + tile_cols - 1) / tile_cols;  // (num_rows * group fits 31 bits: the launcher)
    if (p.n > 0 && p.n <= a.max_nodes && p.c >= 0 && (int64_t)p.c + p.n <= min((int64_t)a.table_stride * kPage, (int64_t)kMaxPositions)) p.blocks = (p.c + p.n + 31) / 32;
    return p;
}

// Sums over a wave by lane shifts, lane 63 has all of them; x of a lane becomes that of it and the lanes in front.
template <int CTRL, int ROWS>
__device__ __forceinline__ int lanes_below(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
template <typename T, int CTRL, int ROWS>
__device__ __forceinline__ void scan_step(T& x) { x += __builtin_bit_cast(T, lanes_below<CTRL, ROWS>(__builtin_bit_cast(int, x))); }
template <typename T>
__device__ __forceinline__ void scan_wave(T& x) {
    scan_step<T, 0x111, 0xf>(x);  // by 1, 2, 4 and 8 lanes in a row of 16
    scan_step<T, 0x112, 0xf>(x);
    scan_step<T, 0x114, 0xf>(x);
    scan_step<T, 0x118, 0xf>(x);
    scan_step<T, 0x142, 0xa>(x);  // the last lane of a row to the next row, of both to the upper half
    scan_step<T, 0x143, 0xc>(x);
}
__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// Blocks of a share, from those of all tiles.  (The sum is exact up to 2^24, and by 1e-4 of itself more from there on, which is more than the
// roundings of its additions, 2^-24 of it each, take away: kTreeMaxSeqs / 4096 of a lane and 15 over lanes and runs.  A share is never less
// than the blocks by the target: the units with partial results would outgrow their places.)
constexpr int kTreeMaxSeqs = 1 << 22;
static_assert(kTreeMaxSeqs / (64 * 64) + 15 < 16777216 / 10000, "the sum of all blocks");
__device__ __forceinline__ int share_of(float total, int n_kv, int tile_cols) {
    const float target = (float)tree_target(n_kv, tile_cols);
    const float even = total < 16777216.f ? ceilf(total / target) : total / target * 1.0001f + 1.f;
    return (int)fminf(fmaxf(even, (float)kTreeMinShare), 1e9f);
}
// The units of a sequence.  They are in order of their size, in quarters of a share, so that the last workgroups to start are short ones;
// in a quarter by sequence, part and tile.
__device__ __forceinline__ int split_seq(const SeqPlan& q, int share, int& parts, int& quarter) {
    parts = max(1, (q.blocks - 1) / share + 1);
    const int size = (q.blocks - 1) / parts + 1;
    quarter = 4 * (int64_t)size > 3 * (int64_t)share ? 0 : 2 * (int64_t)size > share ? 1 : 4 * (int64_t)size > share ? 2 : 3;
    return q.tiles * parts;
}
// The unit of place `place`, if it is one of the 64 sequences from s0 on, one per lane, of whose `mine` units (0: not looked at) the first is
// at place `before`.  slots, cut_tiles: those of the sequences in front, on return of these too.
__device__ __forceinline__ bool unit_of(const SeqPlan& q, int parts, int units, int mine, int before, int place, int s0, int& slots, int& cut_tiles, TreeUnit& u) {
    const bool cut = parts > 1;
    int cut_upto = cut ? units : 0, tiles_upto = cut ? q.tiles : 0;
    scan_wave(cut_upto);
    scan_wave(tiles_upto);
    const int at = place - before;
    const uint64_t who = __ballot(at >= 0 && at < mine);
    if (who) {
        const int l = __builtin_ctzll(who), i = lane_value(at, l), tiles = lane_value(q.tiles, l), blocks = lane_value(q.blocks, l);
        u.seq = s0 + l;
        u.row0 = lane_value(q.row0, l);
        u.n = lane_value(q.n, l);
        u.c = lane_value(q.c, l);
        u.parts = lane_value(parts, l);
        u.part = i / tiles;
        u.tile = i - u.part * tiles;
        u.slot = slots + lane_value(cut_upto - (cut ? units : 0), l) + i;
        u.cut_tile = cut_tiles + lane_value(tiles_upto - (cut ? q.tiles : 0), l) + u.tile;
        const int each = blocks / u.parts, more = blocks - each * u.parts;  // the first `more` parts have a block more
        u.blk_begin = u.part * each + min(u.part, more);
        u.blk_end = u.blk_begin + each + (u.part < more);
        return true;
    }
    slots += lane_value(cut_upto, 63);
    cut_tiles += lane_value(tiles_upto, 63);
    return false;
}

// Up to 64 sequences every wave works the plan out for itself, all of them with the same arithmetic, without LDS and barriers.  More are
// planned by a launch of their own, which cuts them into up to 64 runs of whole waves and leaves what stands in front of each; a wave then looks
// at the runs and at one of them.  us of single tokens behind 300 to 700 keys (8B heads), for itself / by
// the launch: 128 sequences of 500 to 4000 keys 149 / 152, 256 105 / 86, 1024 668 / 330, 4096 7531 / 1306 (6.1 TB/s): a square law against a
// launch of 5.4 us at 256, 5.7 at 1024 and 12.3 at 4096 sequences, of which the stream's launch hides the start.
constexpr int kPlanRuns = 64;
struct TreePlan {
    int32_t share, units;               // units: none where the rows break their order
    int32_t start[4];                   // place of the first unit of a quarter
    int32_t before[4][kPlanRuns];       // place of a run's first unit in a quarter
    int32_t slots[kPlanRuns], cut_tiles[kPlanRuns];  // in front of a run
};
__host__ __device__ inline int plan_run(int num_seqs) { return (num_seqs + 64 * kPlanRuns - 1) / (64 * kPlanRuns) * 64; }  // sequences

// false behind the last unit.  cut_tiles: behind it the number of tiles whose keys are cut, or -1 where the plan's launch has written it.
__device__ __forceinline__ bool tree_unit(const TreeArgs& a, const TreePlan* plan, int place, int tile_cols, TreeUnit& u, int& cut_tiles) {
    const int lane = threadIdx.x & 63;
    int slots = 0;
    if (a.num_seqs > 64) {
        cut_tiles = -1;
        if (place >= plan->units) return false;
        const int share = plan->share;
        const int quarter = (place >= plan->start[1]) + (place >= plan->start[2]) + (place >= plan->start[3]);
        const int first = plan->before[quarter][lane];
        const int run = __popcll(__ballot(first <= place)) - 1, begin = run * plan_run(a.num_seqs), end = min(begin + plan_run(a.num_seqs), a.num_seqs);
        int at = lane_value(first, run), cut = plan->cut_tiles[run];
        slots = plan->slots[run];
        for (int s0 = begin; s0 < end; s0 += 64) {
            const SeqPlan q = seq_plan(a, s0 + lane, tile_cols);
            int parts, its;
            const int units = split_seq(q, share, parts, its), mine = its == quarter ? units : 0;
            int x = mine;
            scan_wave(x);
            if (unit_of(q, parts, units, mine, at + x - mine, place, s0, slots, cut, u)) return true;
            at += lane_value(x, 63);
        }
        return false;
    }
    const SeqPlan p = seq_plan(a, lane, tile_cols);
    cut_tiles = 0;
    if (__any(p.bad)) return false;  // rows in no order may belong to two sequences: the launch would have no place for their units
    float total = (float)p.tiles * (float)p.blocks;
    scan_wave(total);
    total = __builtin_bit_cast(float, lane_value(__builtin_bit_cast(int, total), 63));
    int parts, quarter, before = 0, start = 0;
    const int units = split_seq(p, share_of(total, a.n_kv, tile_cols), parts, quarter);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        int x = quarter == c ? units : 0;
        scan_wave(x);
        if (quarter == c) before = start + x - units;
        start += lane_value(x, 63);
    }
    return unit_of(p, parts, units, units, before, place, 0, slots, cut_tiles, u);
}

// One workgroup; wave w has the runs w, w + 16, ...
__global__ __launch_bounds__(1024) void tree_plan_kernel(TreeArgs a, TreePlan* plan, int32_t* count, int tile_cols) {
    __shared__ float totals[kPlanRuns];
    __shared__ int sums[6][kPlanRuns];  // of a run: units of each quarter, slots, tiles that are cut
    __shared__ int any_bad;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int len = plan_run(a.num_seqs);
    if (threadIdx.x < kPlanRuns) {
        totals[threadIdx.x] = 0.f;
        for (int k = 0; k < 6; ++k) sums[k][threadIdx.x] = 0;
    }
    if (threadIdx.x == 0) any_bad = 0;
    __syncthreads();
    for (int run = wave; run < kPlanRuns && run * len < a.num_seqs; run += 16) {
        float total = 0.f;
        bool bad = false;
        for (int s0 = run * len; s0 < min((run + 1) * len, a.num_seqs); s0 += 64) {
            const SeqPlan q = seq_plan(a, s0 + lane, tile_cols);
            total += (float)q.tiles * (float)q.blocks;
            bad |= q.bad;
        }
        scan_wave(total);
        if (lane == 63) totals[run] = total;
        if (bad) any_bad = 1;
    }
    __syncthreads();
    float total = totals[lane];
    scan_wave(total);
    const int share = share_of(__builtin_bit_cast(float, lane_value(__builtin_bit_cast(int, total), 63)), a.n_kv, tile_cols);
    for (int run = wave; run < kPlanRuns && run * len < a.num_seqs; run += 16) {
        int sum[6] = {0, 0, 0, 0, 0, 0};
        for (int s0 = run * len; s0 < min((run + 1) * len, a.num_seqs); s0 += 64) {
            const SeqPlan q = seq_plan(a, s0 + lane, tile_cols);
            int parts, quarter;
            const int units = split_seq(q, share, parts, quarter);
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] += quarter == c ? units : 0;
            sum[4] += parts > 1 ? units : 0;
            sum[5] += parts > 1 ? q.tiles : 0;
        }
#pragma unroll
        for (int k = 0; k < 6; ++k) {
            scan_wave(sum[k]);
            if (lane == 63) sums[k][run] = sum[k];
        }
    }
    __syncthreads();
    if (wave > 0) return;
    int start = 0;
#pragma unroll
    for (int k = 0; k < 6; ++k) {
        const int own = sums[k][lane];
        int upto = own;
        scan_wave(upto);
        const int all = lane_value(upto, 63);
        if (k < 4) {
            if (lane == 0) plan->start[k] = start;
            plan->before[k][lane] = lane * len < a.num_seqs ? start + upto - own : INT32_MAX;
            start += all;
        } else {
            (k == 4 ? plan->slots : plan->cut_tiles)[lane] = upto - own;
            if (k == 5 && lane == 0) *count = any_bad ? 0 : all;
        }
    }
    if (lane == 0) {
        plan->share = share;
        plan->units = any_bad ? 0 : start;
    }
}

// ---- partial results ------------------------------------------------------------------------------------------------------
//
// Workspace: the plan of many sequences, a record per tile whose keys are cut, then per (slot, KV head) the reference and the sum of each column of the tile,
// then their unnormalised outputs.  A column of a sum below zero is an unused node's.
struct TreeRecord {
    int32_t row0, n, tile, parts;
    int32_t slot, step;  // of the first part, and slots from a part to the next one
    int32_t pad[2];
};
struct TreeParts {
    int32_t* count;  // records
    TreePlan* plan;
    TreeRecord* rec;
    f32x2* ml;       // [slot][n_kv][tile_cols]
    float* o;        // [slot][n_kv][tile_cols][d]
};
__host__ __device__ inline size_t tree_parts(TreeParts& t, void* base, int n_kv, int d, int tile_cols) {
    const size_t cols = (size_t)tree_max_slots(n_kv, tile_cols) * n_kv * tile_cols;
    char* p = (char*)base;
    t.count = (int32_t*)p;
    t.plan = (TreePlan*)(p + 256);
    constexpr size_t head = 256 + (sizeof(TreePlan) + 255) / 256 * 256;
    t.rec = (TreeRecord*)(p + head);
    size_t off = head + (tree_max_cut_tiles(n_kv, tile_cols) * sizeof(TreeRecord) + 255) / 256 * 256;
    t.ml = (f32x2*)(p + off);
    off += cols * 8;
    t.o = (float*)(p + off);
    return off + cols * d * 4;
}
__device__ __forceinline__ void write_record(const TreeParts& parts, const TreeUnit& it, int cols, int tile_cols) {
    if (it.part == 0) parts.rec[it.cut_tile] = TreeRecord{it.row0, it.n, it.tile, it.parts, it.slot, (cols + tile_cols - 1) / tile_cols, {}};
}

// ---- the last blocks -------------------------------------------------------------------------------------------------------
//
// A lane holds 8 of a block's keys: bit v of `seen` says whether its column sees key v, of `keep` whether any used node does.
__device__ __forceinline__ void hide_scores(float (&sc)[8], uint32_t seen) {
#pragma unroll
    for (int v = 0; v < 8; ++v)
        if (!(seen >> v & 1)) sc[v] = -INFINITY;  // (a column may see nothing of a block: no finite stand-in)
}
__device__ __forceinline__ uint32_t pair_mask(uint32_t bits, int w) { return (bits >> (2 * w) & 1 ? 0xFFFFu : 0u) | (bits >> (2 * w + 1) & 1 ? 0xFFFF0000u : 0u); }
// Bit 15 or 31 of a value that is not finite.
__device__ __forceinline__ uint32_t not_finite(uint32_t pair) { return ((pair & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
// V operands of the block: 0 * NaN is NaN, so the values that no node sees are emptied, and those of a used node that are not finite too:
// they may reach the columns that see them only, whose outputs become NaN here.
// (vf: the dims blocks from b0 on.)
template <int D, int NB, int N>
__device__ __forceinline__ void clean_values(u32x4 (&vf)[N], int b0, uint32_t keep, const uint32_t (&seen)[NB], AttnState<D, NB>& st) {
    uint32_t bad = 0u;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t m = pair_mask(keep, w);
#pragma unroll
        for (int b = 0; b < N; ++b) {
            vf[b][w] &= m;
            bad |= not_finite(vf[b][w]);
        }
    }
    if (!__any(bad != 0u)) return;
#pragma unroll
    for (int b = 0; b < N; ++b) {
        u32x4 mark, sees;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t off = not_finite(vf[b][w]);
            mark[w] = (off >> 15 & 1 ? 0x3F80u : 0u) | (off >> 31 ? 0x3F800000u : 0u);  // bf16 ones
            vf[b][w] &= ~((off >> 15 & 1 ? 0xFFFFu : 0u) | (off >> 31 ? 0xFFFF0000u : 0u));
        }
#pragma unroll
        for (int c = 0; c < NB; ++c) {
#pragma unroll
            for (int w = 0; w < 4; ++w) sees[w] = pair_mask(seen[c], w) & 0x3F803F80u;
            const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, mark), __builtin_bit_cast(bf16x8, sees), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (hit[v] > 0.f) st.o[c][b0 + b][v] = NAN;
        }
    }
}

// One workgroup of 4 waves per (unit, KV head), of tiles of 64*NB columns: a block of 32 keys is brought into LDS once and
// read by all waves, each of which has NB groups of 16 columns (the ring and the operand layout are those of prefill attention).
//
// What bounds it: of a block a wave takes 16*NB matrix instructions of 16 cycles and some 56*NB vector ones (per score a maximum, a
// multiplication and addition, a sum, half a conversion, and an exponential of four times their length), and its workgroup passes 64 KiB
// through LDS (at NB = 1 as much for half the columns).  At NB = 2 the matrix cores are busy for 0.40 of the time, the vector units for 0.50; a block takes 1.18 us with two
// workgroups on a compute unit, 0.92 PFLOP/s, and 16 trees of 64 nodes (64 heads on 8, 1000 to 8000 keys) come to 0.7 with the start of
// the units and their last, masked blocks.  Tried without gain: the scores of the next block between the exponentials of this one (a ring
// of four), raised wave priority in either part (169 -> 167 to 173 us with the joining), three workgroups a compute unit at NB = 2 (spills).
template <int D, int NB>
__global__ __launch_bounds__(256, 2) void tree_attention_kernel(TreeArgs a) {
    constexpr int PAGE_BYTES = D * kPage * 2, IPB = PAGE_BYTES / 1024, NS = kTreeStages, TILE = 64 * NB;
    // (one LDS object: with a second one the compiler waits for all loads into the ring before it reads from it)
    extern __shared__ __attribute__((aligned(1024))) unsigned char tree_lds[];
    auto& ring = *reinterpret_cast<unsigned char(*)[NS][4][PAGE_BYTES]>(tree_lds);  // [stage][K0,K1,V0,V1]
    const TreeLds tree(tree_lds + NS * 4 * PAGE_BYTES, a.max_nodes);
    const int kvh = blockIdx.x % a.n_kv, g = a.n_q / a.n_kv;
    TreeUnit it;
    TreeParts parts;
    tree_parts(parts, a.workspace, a.n_kv, D, TILE);
    int cut_tiles;
    if (!tree_unit(a, parts.plan, blockIdx.x / a.n_kv, TILE, it, cut_tiles)) {
        if (cut_tiles >= 0 && blockIdx.x + 1 == gridDim.x && threadIdx.x == 0) *parts.count = cut_tiles;  // (the last workgroup is behind the last unit)
        return;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, G = lane >> 4;
    const int cols = it.n * g;

    bf16x8 qf[NB][D / 32];
    int node[NB];
    bool stored[NB];
    auto load_q = [&]() {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            const bf16_t* qrow = a.q + (int64_t)(it.row0 + node[c]) * a.ld_q + (int64_t)(kvh * g + min(it.tile * TILE + (wave * NB + c) * 16 + r, cols - 1) - node[c] * g) * D;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) qf[c][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + (s * 4 + G) * 8));
        }
    };
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        const int col = it.tile * TILE + (wave * NB + c) * 16 + r;
        stored[c] = col < cols;
        node[c] = min(col, cols - 1) / g;
    }
    AttnState<D, NB> st;
    init_state<D, NB>(st);
    bool used[NB] = {};
    if (it.blk_begin < it.blk_end) {
        const int n_full = it.c / 32, last_page = (it.c + it.n - 1) / kPage;
        const bool sees_tree = it.blk_end > n_full;  // (one part at least: its last block holds the last node)
        const int32_t* bt = a.block_tables + (a.bt_off ? (int64_t)a.bt_off[it.seq] : (int64_t)it.seq * a.table_stride);
        // wave w brings in piece w of a block: K page 0, K page 1, V page 0, V page 1
        const bf16_t* pool = wave < 2 ? a.k_pool : a.v_pool;
        // this wave's pages of 64 blocks, one per lane.  (A load per block would be waited for behind the loads into the ring, which come
        // back in order: all of them would have to be there)
        int ids_base = 0, ids = 0;
        auto fetch_ids = [&](int blk) {
            ids_base = blk;
            ids = min(max(bt[min((blk + lane) * 2 + (wave & 1), last_page)], 0), a.num_blocks - 1);
        };
        auto page_id = [&](int blk) -> int { return __builtin_amdgcn_readlane(ids, blk - ids_base); };
        auto issue_block = [&](int64_t page, int stage) {
            const int src_lane = wave == 1 ? lane ^ 4 : lane;  // K page 1 lies four slots shifted, against bank conflicts
            const char* src = reinterpret_cast<const char*>(pool + (page * a.n_kv + kvh) * (int64_t)(D * kPage)) + src_lane * 16;
#pragma unroll
            for (int i = 0; i < IPB; ++i)
                __builtin_amdgcn_global_load_lds((gptr_t)(src + i * 1024), (lptr_t)(&ring[stage][wave][i * 1024]), 16, 0, 0);
        };
        // The keys are asked for first: they come from HBM, the rest from the caches.
        const int parent = sees_tree ? tree_parent(a, it.row0, it.n) : -2;
        fetch_ids(it.blk_begin);
#pragma unroll
        for (int i = 0; i < NS - 1; ++i) issue_block(page_id(it.blk_begin + i), i);
        load_q();
        const int kpage = r >> 3, kslot = ((r >> 2) & 1) * 8 + (r & 3);
        // Raw scores of the block in `stage`.
        auto scores = [&](int stage, float (&sc)[NB][8]) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                u32x4 kf[D / 32];
#pragma unroll
                for (int s = 0; s < D / 32; ++s) kf[s] = *reinterpret_cast<const u32x4*>(&ring[stage][kpage][((s * 4 + G) * 16 + ((kslot + 4 * t) ^ (4 * kpage))) * 16]);
#pragma unroll
                for (int c = 0; c < NB; ++c) {
                    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < D / 32; ++s) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[s]), qf[c][s], x, 0, 0, 0);
#pragma unroll
                    for (int v = 0; v < 4; ++v) sc[c][4 * t + v] = x[v];
                }
            }
        };
        auto block_step = [&](int stage, int blk, auto masked) {
            constexpr bool MASKED = decltype(masked)::value;
            float sc[NB][8];
            scores(stage, sc);
            uint32_t seen[NB];
            if (MASKED)
#pragma unroll
                for (int c = 0; c < NB; ++c) {
                    seen[c] = tree.vis[node[c] * tree.stride + blk - n_full] >> (G * 8);
                    hide_scores(sc[c], seen[c]);
                }
            constexpr int PORTION = 4;  // dims blocks
            u32x4 vf[PORTION];
            auto read_v = [&](int b0) {
#pragma unroll
                for (int b = 0; b < PORTION; ++b) vf[b] = *reinterpret_cast<const u32x4*>(&ring[stage][2 + (G >> 1)][(b0 + b) * 512 + r * 32 + (G & 1) * 16]);
            };
            raise_reference<D, NB, true>(st, sc, a.scale_log2);
            read_v(0);
            bf16x8 pb[NB];
            block_weights<D, NB>(st, sc, a.scale_log2, pb);
#pragma unroll
            for (int b0 = 0; b0 < D / 16; b0 += PORTION) {
                if (b0 > 0) read_v(b0);
                if (MASKED) clean_values<D, NB, PORTION>(vf, b0, tree.used[blk - n_full] >> (G * 8), seen, st);
#pragma unroll
                for (int b = 0; b < PORTION; ++b)
#pragma unroll
                    for (int c = 0; c < NB; ++c)
                        st.o[c][b0 + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[b]), pb[c], st.o[c][b0 + b], 0, 0, 0);
            }
        };
        if (sees_tree) tree_visibility(a, tree, parent, it.n, it.c);
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            if (!sees_tree) continue;
            const int at = (it.c & 31) + node[c];
            used[c] = tree.vis[node[c] * tree.stride + (at >> 5)] >> (at & 31) & 1;
        }
        const bool idle = it.tile * TILE + wave * NB * 16 >= cols;  // (the same for the wave)
        // No node sees a later one: the last block of the tile, and of the wave, is that of its last node.  (A part may be left without blocks.
        // 64 trees of 256 nodes behind 10 to 500 keys, 8B heads: 252 -> 220 us.)
        auto stop = [&](int columns) { return (it.c + (min(it.tile * TILE + columns, cols) - 1) / g) / 32 + 1; };
        const int nblk = min(it.blk_end, stop(TILE)) - it.blk_begin, full = min(nblk, max(n_full - it.blk_begin, 0)), mine = stop((wave + 1) * NB * 16) - it.blk_begin;
        // every wave always issues its piece (indices past the end read the last page again into a stage nobody reads), so the
        // count of outstanding loads is the same in every iteration
        auto advance = [&](int i) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * IPB) : "memory");
            __syncthreads();  // block i has landed; nobody reads the stage of the block before it any more
            const int next = it.blk_begin + i + NS - 1;
            if (next >= ids_base + 64) fetch_ids(next);
            issue_block(page_id(next), (i + NS - 1) % NS);
        };
        // blocks that all columns see, then the last ones
        for (int i = 0; i < full; ++i) {
            advance(i);
            if (!idle) block_step(i % NS, it.blk_begin + i, std::false_type{});
        }
        for (int i = full; i < nblk; ++i) {
            advance(i);
            if (!idle && i < mine) block_step(i % NS, it.blk_begin + i, std::true_type{});
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no LDS fill may outlive the workgroup
    }
    if (it.parts > 1 && kvh == 0 && threadIdx.x == 0) write_record(parts, it, cols, TILE);
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        float l = st.l[c];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (!stored[c]) continue;
        const int tcol = (wave * NB + c) * 16 + r, col = it.tile * TILE + tcol;
        if (it.parts > 1) {
            const int64_t at = ((int64_t)it.slot * a.n_kv + kvh) * TILE + tcol;
#pragma unroll
            for (int b = 0; b < D / 16; ++b) *reinterpret_cast<f32x4*>(parts.o + at * D + b * 16 + G * 4) = st.o[c][b];
            if (G == 0) parts.ml[at] = f32x2{st.m[c], it.part + 1 == it.parts && !used[c] ? -1.f : l};
            continue;
        }
        const float inv = 1.0f / l;
        bf16_t* orow = a.out + (int64_t)(it.row0 + node[c]) * a.ld_o + (int64_t)(kvh * g + col - node[c] * g) * D;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) {
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
            if (used[c])
#pragma unroll
                for (int v = 0; v < 4; ++v) o[v] = st.o[c][b][v] * inv;
            *reinterpret_cast<bf16x4*>(orow + b * 16 + G * 4) = __builtin_convertvector(o, bf16x4);
        }
    }
}

// Few columns (tiles of 16*NB): the keys are a stream from HBM, and each wave takes a run of the unit's blocks for all columns, operands
// straight to registers as in decode attention (load_kv: score tile t is page t, a lane has keys 4G .. 4G+3 of both pages).  The
// waves' results are joined through LDS, a group of 16 columns at a time.  Bound by HBM: 6.2 TB/s at 32 single tokens behind 300 to 20000
// keys (a bare read in this way reaches 6.2); one short sequence is all latency (6.0 us at 64 keys and less).
template <int D>
struct StreamLds {
    float o[4][16][D + 4];
    float m[4][16], l[4][16];
};
template <int D, int NB>
__global__ __launch_bounds__(256, NB == 1 ? 2 : 1) void tree_stream_kernel(TreeArgs a) {
    constexpr int TILE = 16 * NB;
    __shared__ StreamLds<D> join;
    extern __shared__ uint32_t tree_words[];
    const TreeLds tree(tree_words, a.max_nodes);
    const int kvh = blockIdx.x % a.n_kv, g = a.n_q / a.n_kv;
    TreeUnit it;
    TreeParts parts;
    tree_parts(parts, a.workspace, a.n_kv, D, TILE);
    int cut_tiles;
    if (!tree_unit(a, parts.plan, blockIdx.x / a.n_kv, TILE, it, cut_tiles)) {
        if (cut_tiles >= 0 && blockIdx.x + 1 == gridDim.x && threadIdx.x == 0) *parts.count = cut_tiles;  // (the last workgroup is behind the last unit)
        return;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, G = lane >> 4;
    const int cols = it.n * g;
    const int n_full = it.c / 32, last_page = max(it.c + it.n - 1, 0) / kPage;
    const int run = (it.blk_end - it.blk_begin + 3) / 4;
    const int b_begin = min(it.blk_begin + wave * run, it.blk_end), b_end = min(b_begin + run, it.blk_end);
    const int32_t* bt = a.block_tables + (a.bt_off ? (int64_t)a.bt_off[it.seq] : (int64_t)it.seq * a.table_stride);
    int ids_base = 2 * b_begin, ids = 0;  // page ids, one per lane
    auto fetch_ids = [&](int base) {
        ids_base = base;
        ids = min(max(bt[min(base + lane, last_page)], 0), a.num_blocks - 1);
    };
    auto load_block = [&](KvFrag<D>& f, int blk) {
        const int p0 = min(2 * blk, last_page) - ids_base, p1 = min(2 * blk + 1, last_page) - ids_base;
        load_kv<D>(f, a.k_pool, a.v_pool, (int64_t)__builtin_amdgcn_readlane(ids, p0), (int64_t)__builtin_amdgcn_readlane(ids, p1), a.n_kv, kvh, lane);
    };
    KvFrag<D> fa, fb;
    const bool sees_tree = it.blk_begin < it.blk_end && it.blk_end > n_full;
    const int parent = sees_tree ? tree_parent(a, it.row0, it.n) : -2;
    if (b_begin < b_end) {
        fetch_ids(2 * b_begin);
        load_block(fa, b_begin);
    }
    bf16x8 qf[NB][D / 32];
    int node[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        const int cc = min(it.tile * TILE + c * 16 + r, cols - 1);
        node[c] = cc / g;
        const bf16_t* qrow = a.q + (int64_t)(it.row0 + node[c]) * a.ld_q + (int64_t)(kvh * g + cc - node[c] * g) * D;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) qf[c][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + (s * 4 + G) * 8));
    }
    if (sees_tree) tree_visibility(a, tree, parent, it.n, it.c);
    AttnState<D, NB> st;
    init_state<D, NB>(st);
    auto attend = [&](KvFrag<D>& f) {
        float sc[NB][8];
#pragma unroll
        for (int c = 0; c < NB; ++c) score_group<D>(sc[c], f.k, qf[c]);
        update_groups<D, NB, false>(st, sc, a.scale_log2, []() {}, [&]() -> const u32x4 (&)[D / 16] { return f.v; });
    };
    auto next_block = [&](KvFrag<D>& f, int blk) {
        if (2 * blk + 1 >= ids_base + 64) fetch_ids(2 * blk);
        load_block(f, blk);
    };
    // blocks that all columns see, the next one on its way; then the last ones
    int blk = b_begin;
    const int b_full = min(b_end, n_full);
    while (blk + 1 < b_full) {
        next_block(fb, blk + 1);
        attend(fa);
        if (blk + 2 < b_end) next_block(fa, blk + 2);
        attend(fb);
        blk += 2;
    }
    if (blk < b_full) {
        attend(fa);
        if (++blk < b_end) next_block(fa, blk);
    }
    while (blk < b_end) {
        float sc[NB][8];
        uint32_t seen[NB];
        auto mine = [&](uint32_t word) { return (word >> (4 * G) & 15u) | (word >> (16 + 4 * G) & 15u) << 4; };
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            score_group<D>(sc[c], fa.k, qf[c]);
            seen[c] = mine(tree.vis[node[c] * tree.stride + blk - n_full]);
            hide_scores(sc[c], seen[c]);
        }
        clean_values<D, NB, D / 16>(fa.v, 0, mine(tree.used[blk - n_full]), seen, st);
        update_groups<D, NB, false>(st, sc, a.scale_log2, []() {}, [&]() -> const u32x4 (&)[D / 16] { return fa.v; });
        if (++blk < b_end) next_block(fa, blk);
    }
    if (it.parts > 1 && kvh == 0 && threadIdx.x == 0) write_record(parts, it, cols, TILE);
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        float l = st.l[c];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (c > 0) __syncthreads();
        if (G == 0) {
            join.m[wave][r] = st.m[c];
            join.l[wave][r] = l;
        }
#pragma unroll
        for (int b = 0; b < D / 16; ++b) *reinterpret_cast<f32x4*>(&join.o[wave][r][b * 16 + G * 4]) = st.o[c][b];
        __syncthreads();
        const int col0 = it.tile * TILE + c * 16, here = min(16, cols - col0);
        for (int i = threadIdx.x; i < here * (D / 4); i += 256) {
            const int j = i / (D / 4), e = i % (D / 4) * 4, col = col0 + j, nd = col / g;
            float m = kNegBig, ls = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) m = fmaxf(m, join.m[w][j]);
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float x = __builtin_amdgcn_exp2f(join.m[w][j] - m);
                const f32x4 o = *reinterpret_cast<const f32x4*>(&join.o[w][j][e]);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[v] += o[v] * x;
                ls += join.l[w][j] * x;
            }
            const int at = (it.c & 31) + nd;
            const bool used = sees_tree && tree.vis[nd * tree.stride + (at >> 5)] >> (at & 31) & 1;
            if (it.parts > 1) {
                const int64_t place = ((int64_t)it.slot * a.n_kv + kvh) * TILE + c * 16 + j;
                *reinterpret_cast<f32x4*>(parts.o + place * D + e) = acc;
                if (e == 0) parts.ml[place] = f32x2{m, it.part + 1 == it.parts && !used ? -1.f : ls};
                continue;
            }
            const float inv = 1.0f / ls;
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[v] = used ? acc[v] * inv : 0.f;
            *reinterpret_cast<bf16x4*>(a.out + (int64_t)(it.row0 + nd) * a.ld_o + (int64_t)(kvh * g + col - nd * g) * D + e) =
                __builtin_convertvector(acc, bf16x4);
        }
    }
}

// The partial results of all tiles joined, in order of the parts: a work item is (record, KV head, 1024 / D columns), a thread per four dims
// of a column.  The kernel is all latency: kMergeBatch parts are asked for at a time, where there are fewer the last one again (18.5 us, 16.5 the
// fastest, at 512 workgroups' results of 128 columns, 34 MB; 4.8 at those of 32 single tokens).
constexpr int kMergeBatch = 12;
constexpr int kMergeGroups = 2048;  // workgroups
template <int D>
__device__ __forceinline__ void merge_columns(const TreeArgs& a, const TreeParts& parts, const TreeRecord& rec, int kvh, int tcol, int tile_cols) {
    const int g = a.n_q / a.n_kv, e = threadIdx.x % (D / 4) * 4, col = rec.tile * tile_cols + tcol;
    if (col >= rec.n * g) return;
    const int64_t step = (int64_t)rec.step * a.n_kv * tile_cols, first = ((int64_t)rec.slot * a.n_kv + kvh) * tile_cols + tcol;
    float m = kNegBig, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    bool used = true;
    for (int p0 = 0; p0 < rec.parts; p0 += kMergeBatch) {
        f32x2 ml[kMergeBatch];
        f32x4 o[kMergeBatch];
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) {
            const int64_t at = first + min(p0 + u, rec.parts - 1) * step;
            ml[u] = parts.ml[at];
            o[u] = *reinterpret_cast<const f32x4*>(parts.o + at * D + e);
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) top = fmaxf(top, ml[u][0]);
        const float down = __builtin_amdgcn_exp2f(m - top);
        l *= down;
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[v] *= down;
        m = top;
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) {
            if (p0 + u >= rec.parts) continue;
            const float w = __builtin_amdgcn_exp2f(ml[u][0] - m);
            used = !(ml[u][1] < 0.f);
            l += ml[u][1] * w;
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[v] += o[u][v] * w;
        }
    }
    const float inv = 1.0f / l;
#pragma unroll
    for (int v = 0; v < 4; ++v) acc[v] = used ? acc[v] * inv : 0.f;
    *reinterpret_cast<bf16x4*>(a.out + (int64_t)(rec.row0 + col / g) * a.ld_o + (int64_t)(kvh * g + col % g) * D + e) = __builtin_convertvector(acc, bf16x4);
}
template <int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, int tile_cols) {
    constexpr int COLS = 1024 / D;
    TreeParts parts;
    tree_parts(parts, a.workspace, a.n_kv, D, tile_cols);
    const int groups = (tile_cols + COLS - 1) / COLS, per_record = a.n_kv * groups;
    int work = blockIdx.x;
    TreeRecord rec = parts.rec[min(work / per_record, tree_max_cut_tiles(a.n_kv, tile_cols) - 1)];  // (behind the last one: anything)
    const int total = *parts.count * per_record;
    while (work < total) {
        const int rest = work % per_record;
        work += gridDim.x;
        const TreeRecord next = parts.rec[min(work / per_record, tree_max_cut_tiles(a.n_kv, tile_cols) - 1)];
        merge_columns<D>(a, parts, rec, rest % a.n_kv, rest / a.n_kv * COLS + (int)threadIdx.x / (D / 4), tile_cols);
        rec = next;
    }
}

}  // namespace

// Columns of a tile.  Up to 32 all columns of a KV head are in one, whose waves stream keys of their own.  Above, tiles of 64 (three
// workgroups per compute unit, half the partial results) against 128 (two, and half the passes through LDS), us: 26 nodes behind 2500 keys,
// 104 columns 14.7 / 17.0, 32 x 32 nodes (8B heads) 128 columns 93 / 100, 16 x 64 nodes (8B) 256 columns 108 / 110, 48 ragged trees (14B)
// up to 300 columns 110 / 114, 16 x 64 nodes (70B) 512 columns 173 / 165, four of 128 nodes (8B) 512 columns 75 / 69, four of 200 nodes (70B) 1600
// columns 185 / 182.  The rule goes by the columns alone, and loses where few KV heads leave few workgroups: 16 x 60 nodes of 16 heads on one KV
// head, 960 columns, 56 / 68.
static int tree_tile_cols(int n_q, int n_kv, int max_nodes) {
    const int64_t cols = (int64_t)max_nodes * (n_q / n_kv);
    return cols <= 16 ? 16 : cols <= 32 ? 32 : cols < 512 ? 64 : 128;
}

size_t tree_workspace_bytes(int n_q, int n_kv, int d, int max_nodes) {
    TreeParts t;
    return tree_parts(t, nullptr, n_kv, d, tree_tile_cols(n_q, n_kv, max_nodes));
}

template <int D, int NB>
static hipError_t launch_tiles(const TreeArgs& a, dim3 grid, int lds, hipStream_t stream) {
    constexpr int ring = kTreeStages * 4 * D * kPage * 2;
    static std::atomic<uint64_t> allowed{0};  // devices on which this kernel may use the LDS that it asks for
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(tree_attention_kernel<D, NB>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                ring + TreeLds(nullptr, kTreeNodes).bytes(kTreeNodes));
        if (e != hipSuccess) return e;
        if (dev < 64) allowed.fetch_or(1ull << dev);
    }
    tree_attention_kernel<D, NB><<<grid, 256, ring + lds, stream>>>(a);
    return hipSuccess;
}

template <int D>
static hipError_t launch_tree(const TreeArgs& a, int tile_cols, int64_t units, hipStream_t stream) {
    const dim3 grid((unsigned)(units * a.n_kv));
    const int lds = TreeLds(nullptr, a.max_nodes).bytes(a.max_nodes);
    hipError_t e = hipSuccess;
    if (a.num_seqs > 64) {
        TreeParts parts;
        tree_parts(parts, a.workspace, a.n_kv, D, tile_cols);
        tree_plan_kernel<<<1, 1024, 0, stream>>>(a, parts.plan, parts.count, tile_cols);
    }
    if (tile_cols == 16) tree_stream_kernel<D, 1><<<grid, 256, lds, stream>>>(a);
    else if (tile_cols == 32) tree_stream_kernel<D, 2><<<grid, 256, lds, stream>>>(a);
    else if (tile_cols == 64) e = launch_tiles<D, 1>(a, grid, lds, stream);
    else e = launch_tiles<D, 2>(a, grid, lds, stream);
    if (e != hipSuccess) return e;
    // no sequence can be cut whose table has no more pages than the fewest blocks of a part
    if (a.table_stride > 2 * kTreeMinShare) tree_merge_kernel<D><<<kMergeGroups, 256, 0, stream>>>(a, tile_cols);
    return hipGetLastError();
}

hipError_t launch_tree_attention(const TreeArgs& a, hipStream_t stream) {
    if (a.num_seqs <= 0 || a.num_rows <= 0) return hipSuccess;
    const int g = a.n_q / a.n_kv, tile_cols = tree_tile_cols(a.n_q, a.n_kv, a.max_nodes);
    // no more tiles than whole ones in all rows and a partly filled one per sequence; cutting the keys adds no more units than there
    // are shares; and one place behind the last unit
    const int64_t units = (int64_t)a.num_rows * g / tile_cols + a.num_seqs + tree_target(a.n_kv, tile_cols) + 1;
    if (a.num_seqs > kTreeMaxSeqs || units * a.n_kv > INT32_MAX || (int64_t)a.num_rows * g > INT32_MAX) return hipErrorInvalidValue;
    if (a.d == 128) return launch_tree<128>(a, tile_cols, units, stream);
    if (a.d == 64) return launch_tree<64>(a, tile_cols, units, stream);
    return hipErrorInvalidValue;
}
