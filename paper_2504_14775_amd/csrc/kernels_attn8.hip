// Attention of hybrid batches over the 8-bit pool (contract: include/gllm_cache8.h).
//
// Per KV head the n rows of a sequence times the g query heads of the group are n*g columns over one stream of keys, column j being head
// j % g of row j / g:  S^T = K.Q^T, softmax down the columns with a running reference, O^T += V^T.P^T, in transposed form so that the
// scores a lane receives are the operand that it supplies (kernels_attn.hip).  A code times its page's scale is a value: codes become bf16
// without rounding (4 bits of mantissa).  The key scale s_k of a page multiplies its scores.  Its value scale s_v = 2^e f, 1 <= f < 2, is shared out: the
// codes take 2^e as they become bf16, which has the exponents for it (2^-109 .. 2^109), and the weights f,
//     p f = 2^(s c s_k - m + log2 f),   c = scale * log2(e),
// in the one multiply-add that the exponential's argument takes anyway; a lane holds keys of one page only, so that its part of the sum of
// the weights is that of p f times 1 / f.  (Weights of p s_v would leave float's range under small scales, and be missing from the sum of the weights.)
//
// Up to 16 columns (decode rows), or 32 where no sequence of a call can have more, the keys are a stream from HBM: stream_wave.  More go in tiles whose
// keys pass through LDS: tile_unit.
// The keys of long sequences are shared among waves, or units, by a plan made on the device, and the parts' results joined by a second launch.
//
// Roundings: queries, codes as bf16 (exact), weights p f and the output are bf16, all else float.  A weight rounded to bf16 is what a matrix
// instruction takes; its error, up to 2^-8 of it, is in the output's tolerance.  Tiles sum the rounded weights (one instruction for two of them, and
// the error of a weight cancels where all values agree), streams, which have instructions to spare, the unrounded.
//
// Measured (8 KV heads of 128): 32 decode rows behind 300 .. 20000 keys, 308 MB, 58 us with the joining, 53 + 5, 5.8 TB/s inside the kernel (a copy
// reaches 5.2); 64 behind a window of 1024, 33 us; 251 decode rows and 1802 chunk rows together, 938 MB and 63 GFLOP, 201 us; a chunk of 4096 behind
// 4096 keys, 64 heads, 825 GFLOP that count, 796 us, 1.04 PFLOP/s (a large product reaches 1.42).
#include "cache8.h"

#include <algorithm>
#include <atomic>

namespace {

typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr float kNegBig = -1.0e30f;
constexpr int kBlock = 64;  // keys, four pages

// ---- the plan --------------------------------------------------------------------------------------------------------------
//
// The lengths stand on the device.  Sequences of up to 16 columns (32) are streams: their blocks of 64 keys, one sequence behind the other, are dealt
// in equal runs to the waves of some workgroups.  The others have tiles of 256 columns, each a unit of work of its own or, where there are few of
// them, several, which share its keys.  The stream's workgroups are the first of the launch. Streams of 32 columns need 393 registers, which the
// launch with tiles has not: there those of 17 columns and more are tiles.  us as tiles / as streams (8B heads): 32 sequences of 5 rows behind up to
// 8000 keys 165 / 58, of 8 166 / 64, 100 of up to 8 behind up to 700 68 / 45.
constexpr int kStreamCols = 16, kWideCols = 32, kTileCols = 256;

// A unit of work of a tile: a part of its keys.
struct Unit {
    int32_t seq, row0, n, c;
    int32_t tile, part, parts;
    int32_t place;               // parts > 1: of its partial results, in columns
    int32_t step;                // and from a part's to the next one's
    int32_t cut_tile;            // and of its tile among those with such units
};

// Fewest blocks worth a unit.  us at 2 / 3 / 6 / 10 (8B heads): a chunk of 64 behind 1000 keys 20.6 / 20.8 / 23.8 / 28.7, of 512 behind none 26.7 /
// 26.7 / 28.9 / 29.3, of 32 behind 4000 21.1 / 21.1 / 21.4 / 25.3, 4 of 128 behind up to 700 28.2 / 28.3 / 30.7 / 35.5.
constexpr int kMinShare = 2;
constexpr int kWhole = 6;        // most blocks of a stream that is never cut
constexpr int kGroups = 256;     // workgroups that run at one time: one on each compute unit
// All of these are for each KV head.
__host__ __device__ constexpr int per_head(int total, int n_kv) { return total / n_kv > 0 ? total / n_kv : 1; }
// Workgroups of the stream at most.
template <bool TILES, int COLS>
__host__ __device__ constexpr int max_workers(int n_kv, int d) { return per_head(TILES || d == 128 || COLS > kStreamCols ? kGroups : 2 * kGroups, n_kv); }
// Units that the keys of tiles are cut into.  Every part of a tile writes and reads partial results of (d + 2) floats a column, as much as eight
// blocks of keys.  us at 128 / 256 / 512: a chunk of 901 behind 2011 keys (14B heads) 95 / 99 / 99, of 4096 behind none (8B) 155 / 156 / 220, 251
// decode rows beside 1802 chunk rows (14B) 201 / 224 / 262, 100 rows behind 6000 keys 41 / 39 / 43.
__host__ __device__ constexpr int target_units(int n_kv) { return per_head(kGroups / 2, n_kv); }
// Tiles with partial results and columns of these.  A tile is cut where its sequence has more blocks than a share, into at most ceil(blocks /
// share) parts; the shares of all are at least half their blocks by the target (seq_plan: twice the weight is at least the blocks).
__host__ __device__ constexpr int max_cut_tiles(int n_kv) { return 2 * target_units(n_kv); }
__host__ __device__ constexpr int max_places(int n_kv) { return 4 * target_units(n_kv) * kTileCols; }

// The blocks that the rows i0 .. i1 of a sequence see, counted without those between the first tokens that stay and the window.
struct Seen {
    int32_t sink_blocks, skip;   // block v is v, or v + skip from sink_blocks on
    int32_t blocks;
    __device__ __forceinline__ int actual(int v) const { return v < sink_blocks ? v : v + skip; }
};
__device__ __forceinline__ Seen seen_blocks(const Attn8Args& a, int c, int i0, int i1) {
    const int high = (c + i1) / kBlock;
    if (a.window == 0) return Seen{0, 0, high + 1};
    const int low = max(c + i0 - a.window + 1, 0) / kBlock;
    const int sink = min(a.sinks / kBlock + (a.sinks % kBlock > 0), low);
    return Seen{sink, low - sink, high - low + 1 + sink};
}
// Most blocks that `rows` rows of a sequence see of its own.
__host__ __device__ inline int64_t most_blocks(int64_t own, int64_t rows, int window, int sinks) {
    const int64_t near = (window + rows + kBlock - 2) / kBlock + 1 + sinks / kBlock + 1;
    return window > 0 && near < own ? near : own;
}

struct SeqPlan {
    int32_t row0, n, c, stream;       // stream: its blocks, or none
    int32_t tiles, blocks;            // blocks: of the tile that sees most, at most
    float weight;                     // tiles times about their blocks, at least half of tiles * blocks
    bool broken, unordered;           // a rule: zeros
};
template <int COLS>
__device__ __forceinline__ SeqPlan seq_plan(const Attn8Args& a, int s) {
    SeqPlan p{0, 0, 0, 0, 0, 0, 0.f, false, false};
    if (s >= a.num_seqs) return p;
    const int r0 = a.row_start[s], r1 = a.row_start[s + 1], g = a.n_q / a.n_kv;
    p.c = a.cached_len[s];
    p.unordered = r0 < 0 || r1 < r0 || r1 > a.num_rows;
    p.row0 = r0;
    p.n = p.unordered ? 0 : r1 - r0;
    if (p.n == 0) return p;
    p.broken = p.n > a.max_new || p.c < 0 || (int64_t)p.c + p.n > min((int64_t)a.table_stride * kPage, (int64_t)kMaxPositions);
    if (p.broken) return p;
    const int64_t cols = (int64_t)p.n * g;
    if (cols <= COLS) {
        p.stream = seen_blocks(a, p.c, 0, p.n - 1).blocks;
    } else {
        p.tiles = (int)((cols + kTileCols - 1) / kTileCols);
        p.blocks = (int)most_blocks((p.c + p.n - 1) / kBlock + 1, kTileCols / g + 2, a.window, a.sinks);
        p.weight = (float)p.tiles * (p.tiles > 1 ? fminf((float)p.blocks, (2.f * p.c + p.n) * (0.5f / kBlock) + 2.f) : (float)p.blocks);
    }
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
template <typename T>
__device__ __forceinline__ T lane_value(T x, int lane) { return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); }

// What follows from the sums over all sequences.  (Weights are multiples of 1/128, and their sums exact up to 2^17.  From there on the share is by
// 1e-4 of itself larger, which is more than the roundings of the additions, 2^-24 of the sum each, take away, kMaxAttn8Seqs / 4096 of a lane and 15
// over lanes and runs.)
static_assert(kMaxAttn8Seqs / (64 * 64) + 15 < 16777216 / 10000, "the sum of all weights");
// A block of a tile keeps a compute unit busy for 2.0 us, one of a stream, where half of the units draw all that the memory gives, for 0.35.  us at 4
// / 6 / 8: 251 decode rows beside 1802 chunk rows (14B heads) 208 / 201 / 211, 256 beside 1792 (8B) 148 / 131 / 142, 32 beside 4 x 128 55 / 56 / 47.
constexpr float kTileCost = 6.f;
// Blocks of a wave of the stream, where there are few: us at 2 / 4 / 8, one sequence of 3000 keys (8B heads) 12.8 / 15.0 / 17.7, of 20000 18.9 / 17.9
// / 21.7.
constexpr int kFewBlocks = 2;
template <bool TILES, int COLS>
__device__ __forceinline__ int workers_of(float stream, float tiles, int n_kv, int d) {
    if (!(stream > 0.f)) return 0;
    const int most = max_workers<TILES, COLS>(n_kv, d);
    const float fair = TILES ? rintf(stream / (stream + kTileCost * tiles) * (float)most) : (float)most;
    return (int)fmaxf(fminf(fair, ceilf(stream / (float)(kFewBlocks * (TILES ? 8 : 4)))), 1.f);
}
__device__ __forceinline__ int share_of(float tiles, int n_kv) {
    const float target = (float)target_units(n_kv);
    const float even = tiles < 131072.f ? ceilf(tiles / target) : tiles / target * 1.0001f + 1.f;
    return (int)fminf(fmaxf(even, (float)kMinShare), 1e9f);
}
// The units of a sequence's tiles.  They are in order of their size, in quarters of a share, so that the last workgroups to start are short ones;
// in a quarter by sequence, part and tile, the last tiles, which see most, first.
__device__ __forceinline__ int split_seq(const SeqPlan& q, int share, int& parts, int& quarter) {
    parts = max(1, (q.blocks - 1) / share + 1);
    const int size = (q.blocks - 1) / parts + 1;
    quarter = 4 * (int64_t)size > 3 * (int64_t)share ? 0 : 2 * (int64_t)size > share ? 1 : 4 * (int64_t)size > share ? 2 : 3;
    return q.tiles * parts;
}
// The unit of place `place`, if it is one of the 64 sequences from s0 on, one per lane, of whose `mine` units (0: not looked at) the first is
// at place `before`.  places, cut_tiles: those of the sequences in front, on return of these too.
__device__ __forceinline__ bool unit_of(const SeqPlan& q, int parts, int units, int mine, int before, int place, int s0, int& places, int& cut_tiles, Unit& u) {
    const bool cut = parts > 1;
    int cut_upto = cut ? units * kTileCols : 0, tiles_upto = cut ? q.tiles : 0;
    scan_wave(cut_upto);
    scan_wave(tiles_upto);
    const int at = place - before;
    const uint64_t who = __ballot(at >= 0 && at < mine);
    if (who) {
        const int l = __builtin_ctzll(who), i = lane_value(at, l), tiles = lane_value(q.tiles, l);
        u.seq = s0 + l;
        u.row0 = lane_value(q.row0, l);
        u.n = lane_value(q.n, l);
        u.c = lane_value(q.c, l);
        u.parts = lane_value(parts, l);
        u.part = i / tiles;
        u.tile = tiles - 1 - (i - u.part * tiles);
        u.step = tiles * kTileCols;
        u.place = places + lane_value(cut_upto - (cut ? units * kTileCols : 0), l) + u.part * u.step + u.tile * kTileCols;
        u.cut_tile = cut_tiles + lane_value(tiles_upto - (cut ? q.tiles : 0), l) + u.tile;
        return true;
    }
    places += lane_value(cut_upto, 63);
    cut_tiles += lane_value(tiles_upto, 63);
    return false;
}

// Up to 64 sequences, 256 where there are streams only, every wave works the plan out for itself, all of them with the same arithmetic, without LDS
// and barriers.  More are planned by a launch of their own, which cuts them into up to 64 runs of whole waves and leaves what stands in front of
// each.  Above 64 a wave then looks at the runs and at some of their sequences.  (us with that launch and without, decode rows behind 300 .. 700 keys
// (8B heads): 128 38.2 / 35.1, 256 59.1 / 57.4; 65 behind 64 .. 300 15.9 / 12.5.  With tiles there are many workgroups without work, and each would
// plan first: 253 sequences, 2 of them chunks, 201 / 227.)
constexpr int kOwnRuns = 4;
template <bool TILES>
__host__ __device__ constexpr bool plans_alone(int num_seqs) { return num_seqs <= (TILES ? 64 : 64 * kOwnRuns); }
constexpr int kPlanRuns = 64;
struct Plan {
    int32_t share, units, workers;      // units, workers: none where the rows break their order
    int32_t broken;                     // whether any sequence breaks a rule
    int64_t stream;                     // blocks of all streams
    int64_t stream_before[kPlanRuns];   // in front of a run
    int32_t start[4];                   // place of the first unit of a quarter
    int32_t before[4][kPlanRuns];       // place of a run's first unit in a quarter
    int32_t places[kPlanRuns], cut_tiles[kPlanRuns];  // in front of a run
};
__host__ __device__ inline int plan_run(int num_seqs) { return (num_seqs + 64 * kPlanRuns - 1) / (64 * kPlanRuns) * 64; }  // sequences

// The work of a workgroup's place: a worker of the stream, a unit of a tile, or none.
struct Job {
    int workers;          // of the stream
    int64_t stream;       // blocks of all streams
    bool is_unit;
    Unit unit;
    int cut_tiles;        // behind the last unit: tiles whose keys are cut, or -1 where the plan's launch has written it
    bool broken;
    SeqPlan seqs;         // up to 64 sequences: that of this lane
    int64_t before;       // more, and planned here: blocks of the streams in front of run `lane`
};
template <bool TILES, int COLS>
__device__ __forceinline__ void find_job(const Attn8Args& a, const Plan* plan, int place, Job& j) {
    const int lane = threadIdx.x & 63;
    int places = 0;
    j.is_unit = false;
    j.cut_tiles = 0;
    if (!TILES && a.num_seqs > 64 && plans_alone<TILES>(a.num_seqs)) {
        SeqPlan q[kOwnRuns];
        bool unordered = false, broken = false;
        j.stream = 0;
        j.before = INT64_MAX;
#pragma unroll
        for (int r = 0; r < kOwnRuns; ++r) q[r] = seq_plan<COLS>(a, 64 * r + lane);
#pragma unroll
        for (int r = 0; r < kOwnRuns; ++r) {
            unordered |= q[r].unordered;
            broken |= q[r].broken;
            uint32_t blocks = (uint32_t)q[r].stream;
            scan_wave(blocks);
            if (lane == r && 64 * r < a.num_seqs) j.before = j.stream;
            j.stream += lane_value(blocks, 63);
        }
        const bool none = __any(unordered);
        j.broken = !none && __any(broken);
        j.workers = none ? 0 : workers_of<TILES, COLS>((float)j.stream, 0.f, a.n_kv, a.d);
        return;
    }
    if (a.num_seqs > 64) {
        j.workers = plan->workers;
        j.stream = plan->stream;
        j.broken = plan->broken;
        j.cut_tiles = -1;
        place -= j.workers;
        if (!TILES || place < 0 || place >= plan->units) return;
        const int share = plan->share;
        const int quarter = (place >= plan->start[1]) + (place >= plan->start[2]) + (place >= plan->start[3]);
        const int first = plan->before[quarter][lane];
        const int run = __popcll(__ballot(first <= place)) - 1, begin = run * plan_run(a.num_seqs), end = min(begin + plan_run(a.num_seqs), a.num_seqs);
        int at = lane_value(first, run), cut = plan->cut_tiles[run];
        places = plan->places[run];
        for (int s0 = begin; s0 < end; s0 += 64) {
            const SeqPlan q = seq_plan<COLS>(a, s0 + lane);
            int parts, its;
            const int units = split_seq(q, share, parts, its), mine = its == quarter ? units : 0;
            int x = mine;
            scan_wave(x);
            if (unit_of(q, parts, units, mine, at + x - mine, place, s0, places, cut, j.unit)) {
                j.is_unit = true;
                return;
            }
            at += lane_value(x, 63);
        }
        return;
    }
    j.seqs = seq_plan<COLS>(a, lane);
    j.broken = __any(j.seqs.broken);
    uint32_t blocks = (uint32_t)j.seqs.stream;  // (64 times 2^25 at most)
    scan_wave(blocks);
    j.stream = lane_value(blocks, 63);
    float tiles = 0.f;
    if (TILES) {
        tiles = j.seqs.weight;
        scan_wave(tiles);
        tiles = lane_value(tiles, 63);
    }
    j.workers = workers_of<TILES, COLS>((float)j.stream, tiles, a.n_kv, a.d);
    if (__any(j.seqs.unordered)) {  // rows in no order may belong to two sequences
        j.workers = 0;
        j.broken = false;
        return;
    }
    place -= j.workers;
    if (!TILES || place < 0) return;
    int parts, quarter, before = 0, start = 0;
    const int units = split_seq(j.seqs, share_of(tiles, a.n_kv), parts, quarter);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        int x = quarter == c ? units : 0;
        scan_wave(x);
        if (quarter == c) before = start + x - units;
        start += lane_value(x, 63);
    }
    j.is_unit = unit_of(j.seqs, parts, units, units, before, place, 0, places, j.cut_tiles, j.unit);
}

// One workgroup; wave w has the runs w, w + 16, ...
template <bool TILES, int COLS>
__global__ __launch_bounds__(1024) void attention8_plan_kernel(Attn8Args a, Plan* plan, int32_t* count) {
    __shared__ float totals[2][kPlanRuns];
    __shared__ int64_t stream[kPlanRuns];
    __shared__ int sums[6][kPlanRuns];  // of a run: units of each quarter, places, tiles that are cut
    __shared__ int any_unordered, any_broken;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int len = plan_run(a.num_seqs);
    if (threadIdx.x < kPlanRuns) {
        totals[0][threadIdx.x] = totals[1][threadIdx.x] = 0.f;
        stream[threadIdx.x] = 0;
        for (int k = 0; k < 6; ++k) sums[k][threadIdx.x] = 0;
    }
    if (threadIdx.x == 0) any_unordered = any_broken = 0;
    __syncthreads();
    for (int run = wave; run < kPlanRuns && run * len < a.num_seqs; run += 16) {
        float total = 0.f;
        int64_t blocks = 0;
        bool unordered = false, broken = false;
        for (int s0 = run * len; s0 < min((run + 1) * len, a.num_seqs); s0 += 64) {
            const SeqPlan q = seq_plan<COLS>(a, s0 + lane);
            total += q.weight;
            blocks += q.stream;
            unordered |= q.unordered;
            broken |= q.broken;
        }
        scan_wave(total);
#pragma unroll
        for (int by = 1; by < 64; by *= 2) blocks += __shfl_xor(blocks, by);
        if (lane == 63) {
            totals[0][run] = total;
            stream[run] = blocks;
        }
        if (unordered) any_unordered = 1;
        if (broken) any_broken = 1;
    }
    __syncthreads();
    float total = totals[0][lane];
    scan_wave(total);
    total = lane_value(total, 63);
    const int share = share_of(total, a.n_kv);
    if (TILES) {
        for (int run = wave; run < kPlanRuns && run * len < a.num_seqs; run += 16) {
            int sum[6] = {0, 0, 0, 0, 0, 0};
            for (int s0 = run * len; s0 < min((run + 1) * len, a.num_seqs); s0 += 64) {
                const SeqPlan q = seq_plan<COLS>(a, s0 + lane);
                int parts, quarter;
                const int units = split_seq(q, share, parts, quarter);
#pragma unroll
                for (int c = 0; c < 4; ++c) sum[c] += quarter == c ? units : 0;
                sum[4] += parts > 1 ? units * kTileCols : 0;
                sum[5] += parts > 1 ? q.tiles : 0;
            }
#pragma unroll
            for (int k = 0; k < 6; ++k) {
                scan_wave(sum[k]);
                if (lane == 63) sums[k][run] = sum[k];
            }
        }
        __syncthreads();
    }
    if (wave > 0) return;
    int64_t blocks = stream[lane];
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const int64_t y = __shfl_up(blocks, by);
        if (lane >= by) blocks += y;
    }
    plan->stream_before[lane] = lane * len < a.num_seqs ? blocks - stream[lane] : INT64_MAX;
    const int64_t all_blocks = __shfl(blocks, 63);
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
            (k == 4 ? plan->places : plan->cut_tiles)[lane] = upto - own;
            if (k == 5 && lane == 0) *count = any_unordered ? 0 : all;
        }
    }
    if (lane == 0) {
        plan->share = share;
        plan->units = any_unordered ? 0 : start;
        plan->workers = any_unordered ? 0 : workers_of<TILES, COLS>((float)all_blocks, total, a.n_kv, a.d);
        plan->broken = any_unordered ? 0 : any_broken;
        plan->stream = all_blocks;
    }
}

// ---- partial results ------------------------------------------------------------------------------------------------------
//
// Workspace: the plan of many sequences; the waves of the stream; a record per tile whose keys are cut; then per KV head and column of a part the
// reference and the sum, then the unnormalised outputs, of the stream and of the tiles.  A wave of the stream has places for two streams that
// are not its own alone: the one that its run begins with, and the one that it ends with.
struct StreamRecord {       // of a sequence, or, of more than 64, of the one that begins in a wave's run and goes on in the next one's
    int32_t row0, cols, waves;  // waves: that have a part of it, or none
    int32_t wave, place;    // of the first part, in streams; those of the others are the first ones of their waves
};
struct Record {
    int32_t row0, n, tile;
    int32_t place, step, parts, pad[2];
};
struct Parts {
    int32_t* count;    // records
    int32_t* waves;    // waves of the stream
    Plan* plan;
    StreamRecord* stream;
    Record* rec;
    f32x2 *stream_ml, *ml;  // [n_kv][2 * max waves][columns of a stream], [n_kv][places]
    float *stream_o, *o;    // and [d]
    int64_t max_waves, places;
};
template <bool TILES, int COLS>
__host__ __device__ inline size_t parts_in(Parts& t, void* base, int n_kv, int d) {
    t.max_waves = max_workers<TILES, COLS>(n_kv, d) * (TILES ? 8 : 4);
    t.places = TILES ? max_places(n_kv) : 0;
    char* p = (char*)base;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* at = p + off;
        off += (bytes + 255) / 256 * 256;
        return at;
    };
    t.count = (int32_t*)take(256);
    t.waves = t.count + 1;
    t.plan = (Plan*)take(sizeof(Plan));
    t.stream = (StreamRecord*)take((t.max_waves > 64 ? t.max_waves : 64) * sizeof(StreamRecord));
    t.rec = (Record*)take(TILES ? max_cut_tiles(n_kv) * sizeof(Record) : 0);
    const size_t stream_cols = (size_t)n_kv * 2 * t.max_waves * COLS, cols = (size_t)n_kv * t.places;
    t.stream_ml = (f32x2*)take(stream_cols * 8);
    t.stream_o = (float*)take(stream_cols * d * 4);
    t.ml = (f32x2*)take(cols * 8);
    t.o = (float*)take(cols * d * 4);
    return off;
}

// ---- common to both kinds of units -------------------------------------------------------------------------------------

// A barrier that waits for this wave's reads and writes of LDS only: __syncthreads() would wait for the loads on their way too.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Four codes times a power of two as bf16, without rounding.
__device__ __forceinline__ u32x2 widen(uint32_t codes, float power) {
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, true))};
}
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi, float power = 1.0f) {
    const u32x2 a = widen(lo, power), b = widen(hi, power);
    return u32x4{a[0], a[1], b[0], b[1]};
}
// Bit 7 of every byte that is no number.
__device__ __forceinline__ uint32_t no_numbers(uint32_t codes) { return ((codes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// What a page's scales come to: the factor of its scores, log2 of that of its weights, and one over that; and the power of two that its values take.
struct PageScale {
    float keys, log_values, per_value;
    // Returns the power of two.
    __device__ __forceinline__ float of(f32x2 s, float scale_log2) {
        // (neither 0 nor infinite: the products with hidden keys' scores and with 0 stay what they are)
        keys = fminf(fmaxf(fminf(fmaxf(s[0], kScaleMin), kScaleMax) * scale_log2, 0x1p-126f), 0x1p127f);
        const uint32_t v = __builtin_bit_cast(uint32_t, fminf(fmaxf(s[1], kScaleMin), kScaleMax));
        const float f = __builtin_bit_cast(float, (v & 0x007FFFFFu) | 0x3F800000u);
        log_values = __builtin_amdgcn_logf(f);
        per_value = __builtin_amdgcn_rcpf(f);
        return __builtin_bit_cast(float, v & 0x7F800000u);
    }
};

// ---- streams ---------------------------------------------------------------------------------------------------------------
//
// Each wave takes a run of blocks for all columns of their sequences, operands straight to registers.  Matrix instructions of 16x16x32: the row 4q +
// i of score tile t is slot 4t + i of page q, so that a lane of group G receives the 16 slots of page G.  An instruction that loads keys takes runs
// of 256 bytes from each of the four pages, one that loads values the 16 slots of 16 dims of each.  The keys of the next block are asked for when the
// scores of this one are made, its values when this one's outputs are, into the same registers; so there is always half a block on its way, and the
// waves that share a compute unit hide each other's work.  Bound by HBM: 16 KB a block and KV head for 32 matrix instructions, whose unit is busy for
// 1/15 of the time.  Two blocks in registers would spill; without equal runs (parts of whole blocks per sequence, so many to each) 71 us instead of
// 57 for 32 decode rows behind 300 .. 20000 keys.

// A value that all lanes have, for the compiler to know.
__device__ __forceinline__ int64_t of_wave(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}
// Where the run of wave w begins.
__device__ __forceinline__ int64_t run_begin(int64_t blocks, int waves, int w) { return of_wave((int64_t)((uint64_t)blocks * (uint32_t)w / (uint32_t)waves)); }

template <int D, bool TILES, int COLS>
__device__ __forceinline__ void stream_wave(const Attn8Args& a, const Job& job, const Parts& parts, int kvh, int w, int waves) {
    constexpr int SETS = COLS / 16;  // of 16 columns, which share the keys and values
    const int lane = threadIdx.x & 63;
    const int r = lane & 15, G = lane >> 4, g = a.n_q / a.n_kv;
    // The run.  A stream of few blocks, up to kWhole, belongs to the wave in whose run its last one lies.  The parts of a longer one are those of all waves
    // from its first to its last: with more than kWhole blocks in a call no run behind one that is not empty is empty.  (With kFewBlocks of 2 there are
    // at least as many blocks as waves, or seven blocks to eight waves, of which the first has none.)
    const int64_t lo = run_begin(job.stream, waves, w), hi = run_begin(job.stream, waves, w + 1);

    // 64 sequences, one per lane, of which those up to lane `at` have been dealt with; `upto` blocks up to the end of this lane's, counted from all.
    SeqPlan q;
    int s0 = 0, at = -1;
    int64_t before = 0;   // in front of the 64
    uint32_t upto = 0;
    auto look = [&]() {
        upto = (uint32_t)q.stream;
        scan_wave(upto);
    };
    if (a.num_seqs > 64) {
        const int64_t first = plans_alone<TILES>(a.num_seqs) ? job.before : parts.plan->stream_before[lane];
        const int run = __popcll(__ballot(first <= lo)) - 1;
        s0 = run * plan_run(a.num_seqs);
        before = of_wave(__shfl(first, run));
        q = seq_plan<COLS>(a, s0 + lane);
    } else {
        q = job.seqs;
    }
    look();

    struct Segment {      // the blocks begin .. end - 1 of a sequence's
        int seq, row0, n, c, begin, end, blocks;
        int64_t start;    // of the sequence in the stream
    };
    auto next_segment = [&](Segment& seg) -> bool {
        for (;;) {
            uint64_t rest = __ballot(q.stream > 0 && before + (int64_t)upto > lo);
            if (at >= 0) rest &= at >= 63 ? 0 : ~((2ull << at) - 1);
            if (rest) {
                at = __builtin_ctzll(rest);
                seg.seq = s0 + at;
                seg.row0 = lane_value(q.row0, at);
                seg.n = lane_value(q.n, at);
                seg.c = lane_value(q.c, at);
                seg.blocks = lane_value(q.stream, at);
                const int64_t end = before + (int64_t)lane_value(upto, at);
                seg.start = end - seg.blocks;
                if (seg.blocks <= kWhole) {
                    if (end > hi) return false;
                    seg.begin = 0;
                    seg.end = seg.blocks;
                    return true;
                }
                if (seg.start >= hi) return false;
                seg.begin = (int)(seg.start < lo ? lo - seg.start : 0);
                seg.end = (int)((end < hi ? end : hi) - seg.start);
                if (seg.begin < seg.end) return true;
                continue;
            }
            before += (int64_t)lane_value(upto, 63);
            s0 += 64;
            at = -1;
            if (s0 >= a.num_seqs || before >= hi) return false;
            q = seq_plan<COLS>(a, s0 + lane);
            look();
        }
    };
    // Page ids, of 16 blocks from `base` on, one per lane, as they stand in the table.
    auto table_ids = [&](const Segment& s, const Seen& seen, int base) {
        return a.block_tables[(int64_t)s.seq * a.table_stride + min(seen.actual(base + lane / 4) * 4 + lane % 4, (s.c + s.n - 1) / kPage)];
    };
    // operands: keys [tile][64 dims], row r = slot 4t + r % 4 of page r / 4, dims 16 (4p + G) ..; values [16 dims], dim 16b + r of page G
    u32x4 k[4][D / 64], v[D / 16];
    bf16x8 qf[SETS][D / 64][2], qn[SETS][D / 64][2];  // queries of this segment, and of the next one
    f32x2 scale = {1.f, 1.f}, scale_next = {1.f, 1.f};  // of page G
    const uint8_t* values_at = nullptr;
    int ids = 0, ids_base = 0;
    auto load_keys = [&](int b) {
        constexpr int PH = D * kPage;  // bytes of a page's head
        const int i = (b - ids_base) * 4;
        const int64_t page = (int64_t)__shfl(ids, i + G) * a.n_kv + kvh;
        const uint8_t* at = a.k_pool + ((int64_t)__shfl(ids, i + (r >> 2)) * a.n_kv + kvh) * PH + G * 64 + (r & 3) * 16;
        values_at = a.v_pool + page * PH + r * kPage;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int p = 0; p < D / 64; ++p) k[t][p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + t * (4 * D) + p * 256));
        scale_next = a.scales[page];
    };
    auto load_values = [&]() {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) v[b] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(values_at + b * 256));
    };
    auto load_queries = [&](const Segment& s) {
        const int cols = s.n * g;
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            const int col = min(16 * c + r, cols - 1), row = col / g;
            const bf16_t* qrow = a.q + (int64_t)(s.row0 + row) * a.ld_q + (int64_t)(kvh * g + col - row * g) * D;
#pragma unroll
            for (int p = 0; p < D / 64; ++p)
#pragma unroll
                for (int h = 0; h < 2; ++h) qn[c][p][h] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + 64 * p + 16 * G + 8 * h));
        }
    };

    f32x4 o[SETS][D / 16];
    float m[SETS], l[SETS];
    int pos[SETS], low[SETS], pos_min = 0, low_max = 0;  // a column sees keys up to pos and above low, or below sinks
    auto enter = [&](const Segment& s) {
        const int cols = s.n * g;
        pos_min = s.c;
        low_max = a.window > 0 ? s.c + s.n - 1 - a.window : -1;
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            pos[c] = s.c + min(16 * c + r, cols - 1) / g;
            low[c] = a.window > 0 ? pos[c] - a.window : -1;
            m[c] = kNegBig;
            l[c] = 0.f;
#pragma unroll
            for (int b = 0; b < D / 16; ++b) o[c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < D / 64; ++p)
#pragma unroll
                for (int h = 0; h < 2; ++h) qf[c][p][h] = qn[c][p][h];
        }
    };
    StreamRecord record{0, 0, 0, 0, 0};
    auto finish = [&](const Segment& s) {
        const int cols = s.n * g;
        const bool one = s.end - s.begin == s.blocks;  // the only part
        const int place = 2 * w + (s.start + s.begin > lo);  // the first stream of the run, or the last
#pragma unroll
        for (int c = 0; c < SETS; ++c) {
            float sum = l[c] + __shfl_xor(l[c], 16);
            sum += __shfl_xor(sum, 32);
            const int col = 16 * c + r;
            if (col >= cols) continue;
            if (one) {
                const float inv = 1.0f / sum;
                const int row = col / g;
                bf16_t* orow = a.out + (int64_t)(s.row0 + row) * a.ld_o + (int64_t)(kvh * g + col - row * g) * D + G * 4;
#pragma unroll
                for (int b = 0; b < D / 16; ++b) *reinterpret_cast<bf16x4*>(orow + b * 16) = __builtin_convertvector(o[c][b] * inv, bf16x4);
            } else {
                const int64_t at = ((int64_t)kvh * 2 * parts.max_waves + place) * COLS + col;
#pragma unroll
                for (int b = 0; b < D / 16; ++b) *reinterpret_cast<f32x4*>(parts.stream_o + at * D + b * 16 + G * 4) = o[c][b];
                if (G == 0) parts.stream_ml[at] = f32x2{m[c], sum};
            }
        }
        if (one) {
            if (a.num_seqs <= 64 && kvh == 0 && lane == 0) parts.stream[s.seq] = StreamRecord{0, 0, 0, 0, 0};
            return;
        }
        if (s.begin == 0) {  // the wave of its last block: the last one whose run does not begin behind it
            const int last = (int)(((uint64_t)(s.start + s.blocks) * (uint32_t)waves - 1) / (uint64_t)job.stream);
            record = StreamRecord{s.row0, cols, last - w + 1, w, place};
            if (a.num_seqs <= 64 && kvh == 0 && lane == 0) parts.stream[s.seq] = record;
        }
    };
    Segment seg{}, then{};
    Seen seen{0, 0, 0}, seen_then{0, 0, 0};
    int ids_then = 0, ids_ahead = 0;  // pages that the next segment begins with, of the next 16 blocks
    auto look_ahead = [&]() -> bool {
        if (!next_segment(then)) return false;
        seen_then = seen_blocks(a, then.c, 0, then.n - 1);
        ids_then = table_ids(then, seen_then, then.begin);
        return true;
    };
    auto begin_next = [&]() {  // its keys
        ids = min(max(ids_then, 0), a.num_blocks - 1);
        ids_base = then.begin;
        load_keys(ids_base);
        load_queries(then);
    };
    bool more = look_ahead();
    if (more) {
        begin_next();
        load_values();
        seg = then;
        seen = seen_then;
        scale = scale_next;
        enter(seg);
        more = look_ahead();
        for (int b = seg.begin;;) {
            const bool same = b + 1 < seg.end;
            const int key0 = seen.actual(b) * kBlock;
            f32x4 s[SETS][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int c = 0; c < SETS; ++c) s[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int p = 0; p < D / 64; ++p)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bf16x8 kf = __builtin_bit_cast(bf16x8, widen8(k[t][p][2 * h], k[t][p][2 * h + 1]));
#pragma unroll
                        for (int c = 0; c < SETS; ++c) s[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c][p][h], s[c][t], 0, 0, 0);
                    }
            }
            __builtin_amdgcn_sched_barrier(0);  // (the keys of the next block take the place of these)
            if (same) {
                if (b - ids_base == 12 && ids_base + 16 < seg.end) ids_ahead = table_ids(seg, seen, ids_base + 16);
                if (b + 1 - ids_base == 16) {
                    ids = min(max(ids_ahead, 0), a.num_blocks - 1);
                    ids_base = b + 1;
                }
                load_keys(b + 1);
            } else if (more) {
                begin_next();
            }
            PageScale ps;
            const float power = ps.of(scale, a.scale_log2);
            if (key0 + kBlock - 1 > pos_min || (key0 <= low_max && key0 + kBlock > a.sinks)) {  // not all keys are seen by all columns
                // values that are no numbers may reach the columns that see them only: they are emptied and the key's scores are no numbers
                u32x4 bad = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int b16 = 0; b16 < D / 16; ++b16)
#pragma unroll
                    for (int x = 0; x < 4; ++x) bad[x] |= no_numbers(v[b16][x]);
                if (__any((bad[0] | bad[1] | bad[2] | bad[3]) != 0u)) {
#pragma unroll
                    for (int b16 = 0; b16 < D / 16; ++b16)
#pragma unroll
                        for (int x = 0; x < 4; ++x) v[b16][x] &= ~((no_numbers(v[b16][x]) >> 7) * 0xFFu);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int by = 1; by < 16; by *= 2) bad[x] |= (uint32_t)__shfl_xor((int)bad[x], by);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = key0 + G * kPage + 4 * t + i;
#pragma unroll
                        for (int c = 0; c < SETS; ++c) {
                            const bool hidden = (key > pos[c]) | ((key <= low[c]) & (key >= a.sinks));
                            s[c][t][i] = hidden ? -INFINITY : bad[t] >> (8 * i + 7) & 1 ? NAN : s[c][t][i];
                        }
                    }
            }
            bf16x8 wt[SETS][2];
#pragma unroll
            for (int c = 0; c < SETS; ++c) {
                float top = fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3]));
#pragma unroll
                for (int t = 1; t < 4; ++t) top = fmaxf(top, fmaxf(fmaxf(s[c][t][0], s[c][t][1]), fmaxf(s[c][t][2], s[c][t][3])));
                top *= ps.keys;
                if (__any(top > m[c])) {  // the reference moves to the running maximum, the same in the four lanes of a column
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), m[c]);
                    const float down = __builtin_amdgcn_exp2f(m[c] - top);
                    m[c] = top;
                    l[c] *= down;
#pragma unroll
                    for (int b16 = 0; b16 < D / 16; ++b16)
#pragma unroll
                        for (int x = 0; x < 4; ++x) o[c][b16][x] *= down;
                }
                const float shift = ps.log_values - m[c];
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    f32x8 p;
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        p[x] = __builtin_amdgcn_exp2f(fmaf(s[c][2 * j + x / 4][x % 4], ps.keys, shift));
                        sum += p[x];
                    }
                    wt[c][j] = __builtin_convertvector(p, bf16x8);
                }
                l[c] += sum * ps.per_value;
            }
#pragma unroll
            for (int b16 = 0; b16 < D / 16; ++b16)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, widen8(v[b16][2 * j], v[b16][2 * j + 1], power));
#pragma unroll
                    for (int c = 0; c < SETS; ++c) o[c][b16] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, wt[c][j], o[c][b16], 0, 0, 0);
                }
            __builtin_amdgcn_sched_barrier(0);
            if (same || more) load_values();
            scale = scale_next;
            if (same) {
                ++b;
                continue;
            }
            finish(seg);
            if (!more) break;
            seg = then;
            seen = seen_then;
            b = seg.begin;
            enter(seg);
            more = look_ahead();
        }
    }
    if (a.num_seqs > 64 && kvh == 0 && lane == 0) parts.stream[w] = record;
}

// ---- tiles of columns --------------------------------------------------------------------------------------------------------
//
// One workgroup of 8 waves, 32 columns a wave, matrix instructions of 32x32x16.  Keys come in blocks of 64, four pages: each thread asks for a piece
// of their codes and of their values a block ahead, puts it into LDS as bf16 when it has come, and all waves read these, half a block (two pages)
// after the other.  (Codes through a ring in LDS, four blocks deep, cost 4 to 5 % more: the reads and waits of what every thread had asked for itself.)
// The row 8a + 4h + b of a score tile is slot 4a + b of page h of the half, so that the lanes of half h receive the 16 slots of page h.
//   keys as bf16    [half][D / 8][32 rows][8 dims], row x of piece c at x ^ 4 (c / 2 % 4): the writes of 16 lanes hit different banks
//   values as bf16  [page][2 halves of the slots][D][8 slots]
// The exponentials of a half run beside the scores of the next one and in front of its own outputs; what a phase reads from LDS is asked for in the
// phase before.
//
// What bounds it, a chunk of 4096 behind 4096 keys: 796 us, 1.04 PFLOP/s.  Per block of 64 keys (2.0 us) the matrix cores are busy for 0.9 us, the
// vector units for about 1.1 (32 exponentials and some 170 others a wave), LDS, which each wave reads all keys and values from, for 1.1; a wave's
// chain goes through all three, and there are two waves on a SIMD to hide each other's waits, all that the registers allow.  What each costs, with
// data that does not change, so that the clock stays up (which is worth 5 to 8 % itself): staging and barriers 8 %, exponentials 8 %, reads of LDS
// nothing.  Steps to here: 4 waves of 64 columns, 32 keys at a time, 1143 us, matrix and vector instructions in a given order 1002, 8 waves of 32 and
// blocks of 64 keys 846, the compiler's own order 823.  No gain: raised priority of half of the waves, a reference that moves when a sum of weights
// has grown (a fifth fewer vector instructions), instructions held in the order of the source (3 % slower).

// Blocks that LDS holds: with four a barrier after every second round is enough.  us with two / four: 64 dims, 14 heads on 2, a chunk of 4096 behind
// 4096 228 / 212, 8 heads on 8, four chunks of 1024 behind up to 4096 87 / 84; 128 dims, a chunk of 4096 behind 4096 (64 heads on 8) 829 / 827, of 8191
// in a window 317 / 320 (these four on one card, on which the chunk of 4096 takes 4 % more than stands above).
template <int D>
constexpr int kStages = D == 64 ? 4 : 2;
constexpr int kHalf = 32, kWindow = 64;
struct PageEntry {
    int32_t id;
    float power;
    PageScale scale;
};
template <int D>
struct TileLds {
    unsigned char keys[kStages<D>][2][kHalf * D * 2];
    unsigned char values[kStages<D>][2][kHalf * D * 2];
    PageEntry pages[2][kWindow * 4];                // of 64 blocks and the next 64
    uint32_t bad[2 * kStages<D>][2];                             // of a half: bit 16h + t: slot t of page h has values that are no numbers
};
constexpr float kSlack = 32.0f;  // a reference lags by up to this: weights stay below 2^33

template <int D>
__device__ __forceinline__ void tile_unit(const Attn8Args& a, const Unit& it, const Parts& parts, int kvh, TileLds<D>& lds) {
    constexpr int PH = D * kPage;         // bytes of a page's head
    constexpr int AHEAD = kStages<D> / 2; // blocks that values in LDS are ahead of the round; keys are one more
    constexpr bool BOTH = D == 128;       // a thread has a piece of keys and one of values; or the lower waves keys, the upper ones values
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, h = lane >> 5, g = a.n_q / a.n_kv;
    const int cols = it.n * g, col0 = it.tile * kTileCols, ncols = min(kTileCols, cols - col0);
    const int i0 = col0 / g, i1 = (col0 + ncols - 1) / g;
    const Seen seen = seen_blocks(a, it.c, i0, i1);
    const int each = seen.blocks / it.parts, more = seen.blocks - each * it.parts;
    const int first = it.part * each + min(it.part, more), blocks = each + (it.part < more);
    const int last_page = (it.c + it.n - 1) / kPage;
    const int32_t* bt = a.block_tables + (int64_t)it.seq * a.table_stride;
    auto key_of = [&](int b) { return seen.actual(first + b) * kBlock; };  // first key of block b

    const int tcol = wave * 32 + r, col = col0 + min(tcol, ncols - 1), row = col / g;
    const bool idle = wave * 32 >= ncols;  // (its pieces are wanted all the same)
    const int pos = it.c + row, low = a.window > 0 ? pos - a.window : -1;  // this column sees keys up to pos and above low, or below sinks
    const int wave_min = it.c + (col0 + min(wave * 32, ncols - 1)) / g, wave_max = it.c + (col0 + min((wave + 1) * 32, ncols) - 1) / g;
    auto partly = [&](int key0, int n, int lo, int hi) { return key0 + n - 1 > lo || (a.window > 0 && key0 <= hi - a.window && key0 + n > a.sinks); };
    bf16x8 qf[D / 16];
    const bf16_t* qrow = a.q + (int64_t)(it.row0 + row) * a.ld_q + (int64_t)(kvh * g + col - row * g) * D;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) qf[k] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + k * 16 + h * 8));

    f32x16 o[D / 32];
    float m = kNegBig, l = 0.f;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[t][v] = 0.f;

    if (blocks > 0) {
        // Page ids and scales, 64 blocks and the next 64 in LDS.
        auto page_of = [&](int x) { return min(max(bt[min(key_of(min(x / 4, blocks - 1)) / kPage + x % 4, last_page)], 0), a.num_blocks - 1); };
        auto entry = [&](int x, int id, f32x2 sc) {
            PageEntry e;
            e.id = id;
            e.power = e.scale.of(sc, a.scale_log2);
            lds.pages[x / (kWindow * 4) % 2][x % (kWindow * 4)] = e;
        };
        auto entry_of = [&](int b, int q) -> const PageEntry& { return lds.pages[b / kWindow % 2][b % kWindow * 4 + q]; };
        // The pieces of a side of a block are 16 bytes, 4D of them, page after page.
        const bool has_keys = BOTH || wave < 4, has_values = BOTH || wave >= 4;
        const int piece = BOTH ? threadIdx.x : threadIdx.x & 255, page = piece / D, piece_at = piece % D;
        const int64_t piece_off = (int64_t)kvh * PH + piece_at * 16, page_step = (int64_t)a.n_kv * PH;
        // (behind the last block its pieces again)
        auto load_keys = [&](int id) { return has_keys ? *reinterpret_cast<const u32x4*>(a.k_pool + id * page_step + piece_off) : u32x4{0u, 0u, 0u, 0u}; };
        auto load_values = [&](int id) { return has_values ? *reinterpret_cast<const u32x4*>(a.v_pool + id * page_step + piece_off) : u32x4{0u, 0u, 0u, 0u}; };
        auto id_of = [&](int j) { return entry_of(min(j, blocks - 1), page).id; };  // (the same for the wave; read a round before it is wanted)
        auto power_of = [&](int j) { return entry_of(min(j, blocks - 1), page).power; };
        // Values that are no numbers may reach the columns that see them only: where not all rows of the tile see all keys of a block they are emptied, and
        // the key's scores are no numbers, in all waves: also in one that sees all keys itself.
        auto emptied = [&](int b) { return partly(key_of(b), kBlock, it.c + i0, it.c + i1); };  // (the same for all waves)
        auto clean = [&](int b, u32x4& x) {
            if (!has_values || !emptied(min(b, blocks - 1))) return;
            uint32_t some = 0u;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t n = no_numbers(x[w]);
                x[w] &= ~((n >> 7) * 0xFFu);
                some |= ((n >> 7 & 1) | (n >> 14 & 2) | (n >> 21 & 4) | (n >> 28 & 8)) << (4 * w);
            }
            if (some) atomicOr(&lds.bad[b % (2 * kStages<D>)][page / 2], some << (16 * (page % 2)));
        };
        // where the two halves of a piece go as bf16
        const int chunk = piece_at % (D / 4) / 4, key_row = (8 * (piece_at / (D / 4)) + 4 * (page % 2) + piece_at % 4) ^ (4 * (chunk & 3));
        const int keys_at = (page / 2) * (kHalf * D * 2) + (2 * chunk * 32 + key_row) * 16, values_at = (2 * page * D + piece_at) * 16;
        auto put_keys = [&](int b, u32x4 lo, u32x4 hi) {
            if (!has_keys) return;
            unsigned char* to = &lds.keys[b % kStages<D>][0][0] + keys_at;
            *reinterpret_cast<u32x4*>(to) = lo;
            *reinterpret_cast<u32x4*>(to + 32 * 16) = hi;
        };
        auto put_values = [&](int b, u32x4 lo, u32x4 hi) {
            if (!has_values) return;
            unsigned char* to = &lds.values[b % kStages<D>][0][0] + values_at;
            *reinterpret_cast<u32x4*>(to) = lo;
            *reinterpret_cast<u32x4*>(to + D * 16) = hi;
        };
        auto largest = [&](const f32x16& s) {
            float x = s[0];
#pragma unroll
            for (int v = 1; v < 16; ++v) x = fmaxf(x, s[v]);
            return x;
        };
        // Masks, and the reference that a half needs.
        auto settle = [&](int b, int half, f32x16& s, float top, const PageScale& sc) {
            const int key0 = key_of(b) + half * kHalf;
            if (emptied(b)) {  // (wherever a wave does not see a half whole, the tile does not see the block whole)
                const uint32_t flags = __builtin_amdgcn_readfirstlane(lds.bad[b % (2 * kStages<D>)][half]);
                if (flags || partly(key0, kHalf, wave_min, wave_max)) {
                    const uint32_t bad = flags >> (16 * h);
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int key = key0 + h * kPage + v;
                        const bool hidden = (key > pos) | ((key <= low) & (key >= a.sinks));
                        s[v] = hidden ? -INFINITY : bad >> v & 1 ? NAN : s[v];
                    }
                    top = largest(s);
                }
            }
            top *= sc.keys;
            if (__any(top > m + kSlack)) {
                const float up = fmaxf(m, fmaxf(top, __shfl_xor(top, 32))), down = __builtin_amdgcn_exp2f(m - up);
                m = up;
                l *= down;
#pragma unroll
                for (int t = 0; t < D / 32; ++t)
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[t][v] *= down;
            }
        };
        bf16x8 kf[D / 16], vf[D / 32][2];
        auto read_key = [&](int b, int half, int k) { kf[k] = *reinterpret_cast<const bf16x8*>(lds.keys[b % kStages<D>][half] + ((2 * k + h) * 32 + (r ^ (4 * (k & 3)))) * 16); };
        auto read_value = [&](int b, int half, int x) {
            vf[x % (D / 32)][x / (D / 32)] = *reinterpret_cast<const bf16x8*>(lds.values[b % kStages<D>][half] + ((2 * h + x / (D / 32)) * D + x % (D / 32) * 32 + r) * 16);
        };
        // One half, of block b: its weights and outputs from the scores s, and the scores of the next one, whose keys are in kf, into s; the keys of the one behind
        // that are read into kf.  extra(x): what else goes behind output x.
        auto half_block = [&](int b, int half, f32x16& s, float& top, const PageScale& now, auto extra) {
            constexpr int SCORES = D / 16, OUTPUTS = D / 32 * 2;
            u32x4 w[2];
            f32x16 next;
            float sum = 0.f;
            const float shift = now.log_values - m;
#pragma unroll
            for (int v = 0; v < 16; ++v) next[v] = 0.f;
            // Two weights, and their sum as they are rounded.
            auto pair = [&](int q) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(s[2 * q], now.keys, shift)), p1 = __builtin_amdgcn_exp2f(fmaf(s[2 * q + 1], now.keys, shift));
                const bf16x2 p = __builtin_convertvector(f32x2{p0, p1}, bf16x2);
                w[q / 4][q % 4] = __builtin_bit_cast(uint32_t, p);
                sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(s16x2, p), s16x2{0x3F80, 0x3F80}, sum, false);
            };
#pragma unroll
            for (int x = 0; x < SCORES; ++x) {
                next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[x], qf[x], next, 0, 0, 0);
                read_value(b, half, x);
#pragma unroll
                for (int y = 8 * x / SCORES; y < 8 * (x + 1) / SCORES; ++y) pair(y);
            }
            l += sum * now.per_value;
#pragma unroll
            for (int x = 0; x < OUTPUTS; ++x) {
                const int t = x % (D / 32), j = x / (D / 32);
                o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t][j], __builtin_bit_cast(bf16x8, w[j]), o[t], 0, 0, 0);
                read_key(b + 1, half, x);
                extra(x);
#pragma unroll
                for (int y = 16 * x / OUTPUTS; y < 16 * (x + 1) / OUTPUTS; ++y) top = y == 0 ? next[y] : fmaxf(top, next[y]);
            }
            s = next;
        };
        static_assert(D / 16 == D / 32 * 2, "as many scores as outputs");

        if (threadIdx.x < 4 * kStages<D>) (&lds.bad[0][0])[threadIdx.x] = 0u;
        {
            const int id = page_of(threadIdx.x);
            entry(threadIdx.x, id, a.scales[(int64_t)id * a.n_kv + kvh]);
        }
        __syncthreads();
        auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
        u32x4 rk, rv;  // the next pieces
        {
            constexpr bool MORE = AHEAD == 2;
            const int id0 = uniform(id_of(0)), id1 = uniform(id_of(1)), id2 = uniform(id_of(2)), id3 = MORE ? uniform(id_of(3)) : 0;
            const u32x4 k0 = load_keys(id0), k1 = load_keys(id1);
            u32x4 k2{}, v1{};
            if (MORE) k2 = load_keys(id2);
            u32x4 v0 = load_values(id0);
            if (MORE) v1 = load_values(id1);
            rk = load_keys(MORE ? id3 : id2);
            rv = load_values(MORE ? id2 : id1);
            put_keys(0, widen8(k0[0], k0[1]), widen8(k0[2], k0[3]));
            put_keys(1, widen8(k1[0], k1[1]), widen8(k1[2], k1[3]));
            if (MORE) put_keys(2, widen8(k2[0], k2[1]), widen8(k2[2], k2[3]));
            clean(0, v0);
            put_values(0, widen8(v0[0], v0[1], power_of(0)), widen8(v0[2], v0[3], power_of(0)));
            if (MORE) {
                clean(1, v1);
                put_values(1, widen8(v1[0], v1[1], power_of(1)), widen8(v1[2], v1[3], power_of(1)));
            }
        }
        lds_barrier();
        int id_keys = id_of(AHEAD + 2), id_values = id_of(AHEAD + 1);
        f32x16 s;
        float top = 0.f;
        PageScale now = entry_of(0, h).scale;
        if (!idle) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                read_key(0, 0, k);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], qf[k], s, 0, 0, 0);
            }
            settle(0, 0, s, largest(s), now);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) read_key(0, 1, k);
        }
        lds_barrier();  // the keys of block 0 have been read, and others may take their place
        int window_id = 0;
        f32x2 window_scale = {0.f, 0.f};
        for (int b = 0; b < blocks; ++b) {
            const int behind = b % kWindow;
            if (behind <= 2 && b >= kWindow) {  // the pages of the next window but one, in three rounds
                const int x = (b / kWindow + 1) * kWindow * 4 + (int)threadIdx.x;
                if (threadIdx.x < kWindow * 4) {
                    if (behind == 0) window_id = page_of(x);
                    else if (behind == 1) window_scale = a.scales[(int64_t)window_id * a.n_kv + kvh];
                    else entry(x, window_id, window_scale);
                }
            }
            // A round reads the keys of block b + 1, the values of block b and the flags of b and b + 1, and writes the keys of block b + AHEAD + 1,
            // the values and the flags of block b + AHEAD: what AHEAD rounds on is read, and AHEAD rounds ago was, as that of other blocks.
            const int next_keys = uniform(id_keys), next_values = uniform(id_values);
            id_keys = id_of(b + AHEAD + 3);
            id_values = id_of(b + AHEAD + 2);
            const float power = power_of(b + AHEAD);  // of the values in rv
            if (threadIdx.x < 2) lds.bad[(b + 2 * AHEAD + (AHEAD == 1)) % (2 * kStages<D>)][threadIdx.x] = 0u;
            const PageScale then = entry_of(b, 2 + h).scale, after = entry_of(min(b + 1, blocks - 1), h).scale;
            u32x4 wide[4];
            if (!idle) {
                half_block(b, 0, s, top, now, [&](int x) {
                    if (x == 1) wide[0] = widen8(rk[0], rk[1]);
                    if (x == 3) {
                        wide[1] = widen8(rk[2], rk[3]);
                        rk = load_keys(next_keys);
                    }
                });
                put_keys(b + AHEAD + 1, wide[0], wide[1]);
                settle(b, 1, s, top, then);
                clean(b + AHEAD, rv);
                half_block(b, 1, s, top, then, [&](int x) {
                    if (x == 1) wide[2] = widen8(rv[0], rv[1], power);
                    if (x == 3) {
                        wide[3] = widen8(rv[2], rv[3], power);
                        rv = load_values(next_values);
                    }
                });
            } else {
                put_keys(b + AHEAD + 1, widen8(rk[0], rk[1]), widen8(rk[2], rk[3]));
                rk = load_keys(next_keys);
                clean(b + AHEAD, rv);
                wide[2] = widen8(rv[0], rv[1], power);
                wide[3] = widen8(rv[2], rv[3], power);
                rv = load_values(next_values);
            }
            put_values(b + AHEAD, wide[2], wide[3]);
            if (AHEAD == 1 || b % 2 == 1) lds_barrier();
            now = after;
            if (!idle && b + 1 < blocks) settle(b + 1, 0, s, top, now);
        }
    }
    l += __shfl_xor(l, 32);
    if (tcol >= ncols) return;
    if (it.parts > 1) {
        const int64_t place = kvh * parts.places + it.place + tcol;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<f32x4*>(parts.o + place * D + t * 32 + b * 8 + h * 4) = f32x4{o[t][4 * b], o[t][4 * b + 1], o[t][4 * b + 2], o[t][4 * b + 3]};
        if (h == 0) parts.ml[place] = f32x2{m, l};
        return;
    }
    const float inv = 1.0f / l;
    bf16_t* orow = a.out + (int64_t)(it.row0 + row) * a.ld_o + (int64_t)(kvh * g + col - row * g) * D;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 x = {o[t][4 * b] * inv, o[t][4 * b + 1] * inv, o[t][4 * b + 2] * inv, o[t][4 * b + 3] * inv};
            *reinterpret_cast<bf16x4*>(orow + t * 32 + b * 8 + h * 4) = __builtin_convertvector(x, bf16x4);
        }
}

// The rows of sequences that break a rule become zeros, by one wave.
template <int D, int COLS>
__device__ __forceinline__ void write_zeros(const Attn8Args& a, int kvh) {
    const int lane = threadIdx.x & 63, g = a.n_q / a.n_kv;
    for (int s0 = 0; s0 < a.num_seqs; s0 += 64) {
        const SeqPlan q = seq_plan<COLS>(a, s0 + lane);
        for (uint64_t todo = __ballot(q.broken); todo; todo &= todo - 1) {
            const int l = __builtin_ctzll(todo), row0 = lane_value(q.row0, l), n = lane_value(q.n, l);
            for (int i = 0; i < n; ++i)
                for (int e = lane * 4; e < g * D; e += 256) *reinterpret_cast<u32x2*>(a.out + (int64_t)(row0 + i) * a.ld_o + (int64_t)kvh * g * D + e) = u32x2{0u, 0u};
        }
    }
}

// Threads of a workgroup: four waves where there are streams only (of 64 dims and 16 columns two workgroups to a compute unit), eight with tiles.
template <bool TILES>
constexpr int kThreads = TILES ? 512 : 256;

template <int D, bool TILES, int COLS>
__global__ __launch_bounds__(kThreads<TILES>, COLS > kStreamCols ? 1 : 2) void attention8_kernel(Attn8Args a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char attn8_lds[];
    constexpr int WAVES = kThreads<TILES> / 64;
    const int kvh = blockIdx.x % a.n_kv, place = blockIdx.x / a.n_kv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Parts parts;
    parts_in<TILES, COLS>(parts, a.workspace, a.n_kv, D);
    Job job;
    find_job<TILES, COLS>(a, parts.plan, place, job);
    if (blockIdx.x + a.n_kv >= gridDim.x) {  // behind the last unit
        if (job.broken && wave == 0) write_zeros<D, COLS>(a, kvh);
        if (a.num_seqs <= 64 && kvh == 0 && wave == 0 && (int)(threadIdx.x & 63) < a.num_seqs && (job.workers == 0 || job.seqs.stream == 0))
            parts.stream[threadIdx.x & 63] = StreamRecord{0, 0, 0, 0, 0};
        if (kvh == 0 && threadIdx.x == 0) {
            if (job.cut_tiles >= 0) *parts.count = job.cut_tiles;
            *parts.waves = job.workers * WAVES;
        }
        return;
    }
    if (place < job.workers) {
        stream_wave<D, TILES, COLS>(a, job, parts, kvh, place * WAVES + wave, job.workers * WAVES);
        return;
    }
    if constexpr (TILES) {
        if (!job.is_unit) return;
        const Unit& it = job.unit;
        if (it.parts > 1 && it.part == 0 && kvh == 0 && threadIdx.x == 0) parts.rec[it.cut_tile] = Record{it.row0, it.n, it.tile, it.place, it.step, it.parts, {}};
        tile_unit<D>(a, it, parts, kvh, *reinterpret_cast<TileLds<D>*>(attn8_lds));
    }
}

// Partial results of a column joined: parts first, first + step, ... of n, of which `at` says the places; BATCH of them are asked for at a time, where
// there are fewer the last one again.
struct Joined {
    float m, l;
    f32x4 o;
};
template <int BATCH, typename At>
__device__ __forceinline__ Joined join_batches(const f32x2* ml, const float* o, int first, int step, int n, int d, int e, At at) {
    Joined j{kNegBig, 0.f, {0.f, 0.f, 0.f, 0.f}};
    for (int p0 = first; p0 < n; p0 += BATCH * step) {
        f32x2 x[BATCH];
        f32x4 y[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int64_t place = at(min(p0 + u * step, n - 1));
            x[u] = ml[place];
            y[u] = *reinterpret_cast<const f32x4*>(o + place * d + e);
        }
        float top = j.m;
#pragma unroll
        for (int u = 0; u < BATCH; ++u) top = fmaxf(top, x[u][0]);
        const float down = __builtin_amdgcn_exp2f(j.m - top);
        j.l *= down;
        j.o *= down;
        j.m = top;
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (p0 + u * step >= n) continue;
            const float w = __builtin_amdgcn_exp2f(x[u][0] - j.m);
            j.l += x[u][1] * w;
            j.o += y[u] * w;
        }
    }
    return j;
}
template <typename At>
__device__ __forceinline__ Joined join_parts(const f32x2* ml, const float* o, int first, int step, int n, int d, int e, At at) {
    const int mine = (n - first + step - 1) / step;
    if (mine <= 2) return join_batches<2>(ml, o, first, step, n, d, e, at);
    if (mine <= 4) return join_batches<4>(ml, o, first, step, n, d, e, at);
    return join_batches<12>(ml, o, first, step, n, d, e, at);
}
// All latency.  The first workgroups take some columns of a stream and a KV head each: D/4 threads have a column, or, where that leaves threads over,
// each so many of its parts; the others as many columns of a cut tile as there are D/4 threads.  (Few streams have many parts: with all columns of a
// stream in a workgroup 8 rows behind 20000 keys take 59 us instead of 25.)
template <int D, bool TILES, int COLS, int THREADS>
__global__ __launch_bounds__(THREADS) void attention8_merge_kernel(Attn8Args a, int stream_groups, int split) {
    constexpr int LANES = D / 4, TEAMS = THREADS / LANES;
    Parts parts;
    parts_in<TILES, COLS>(parts, a.workspace, a.n_kv, D);
    const int g = a.n_q / a.n_kv, team = threadIdx.x / LANES, e = threadIdx.x % LANES * 4;
    auto out_of = [&](int row, int head) { return reinterpret_cast<bf16x4*>(a.out + (int64_t)row * a.ld_o + (int64_t)head * D + e); };
    if ((int)blockIdx.x < stream_groups) {
        __shared__ Joined joined[TEAMS][LANES];
        const int kvh = blockIdx.x % a.n_kv, i = blockIdx.x / a.n_kv / split, each = (COLS + split - 1) / split, col0 = blockIdx.x / a.n_kv % split * each;
        if (a.num_seqs > 64 && i >= *parts.waves) return;
        const StreamRecord rec = parts.stream[i];
        const int cols = min(rec.cols - col0, each);
        if (rec.waves == 0 || cols <= 0) return;
        const int shares = cols < TEAMS ? TEAMS / cols : 1, share = team % shares;
        for (int c = team / shares; shares > 1 || c < cols; c += TEAMS / shares) {
            const bool mine = c < cols;
            const int col = col0 + c;
            Joined j{kNegBig, 0.f, {0.f, 0.f, 0.f, 0.f}};
            if (mine)
                j = join_parts(parts.stream_ml, parts.stream_o, share, shares, rec.waves, D, e,
                               [&](int p) { return ((int64_t)kvh * 2 * parts.max_waves + (p == 0 ? rec.place : 2 * (rec.wave + p))) * COLS + col; });
            if (shares > 1) {
                joined[team][threadIdx.x % LANES] = j;
                __syncthreads();
                if (share > 0 || !mine) return;  // (one pass)
                float top = j.m, l = 0.f;
                for (int x = 1; x < shares; ++x) top = fmaxf(top, joined[team + x][threadIdx.x % LANES].m);
                f32x4 o = {0.f, 0.f, 0.f, 0.f};
                for (int x = 0; x < shares; ++x) {
                    const Joined& y = joined[team + x][threadIdx.x % LANES];
                    const float by = __builtin_amdgcn_exp2f(y.m - top);
                    l += y.l * by;
                    o += y.o * by;
                }
                j = Joined{top, l, o};
            }
            if (mine) *out_of(rec.row0 + col / g, kvh * g + col % g) = __builtin_convertvector(j.o * (1.0f / j.l), bf16x4);
            if (shares > 1) return;
        }
        return;
    }
    if constexpr (TILES) {
        constexpr int GROUPS = kTileCols / TEAMS;
        const int per_record = a.n_kv * GROUPS, total = *parts.count * per_record;
        for (int work = blockIdx.x - stream_groups; work < total; work += gridDim.x - stream_groups) {
            const Record rec = parts.rec[work / per_record];
            const int rest = work % per_record, kvh = rest % a.n_kv, tcol = rest / a.n_kv * TEAMS + team, col = rec.tile * kTileCols + tcol;
            if (col >= rec.n * g) continue;
            const int64_t first = kvh * parts.places + rec.place + tcol;
            const Joined j = join_parts(parts.ml, parts.o, 0, 1, rec.parts, D, e, [&](int p) { return first + (int64_t)p * rec.step; });
            *out_of(rec.row0 + col / g, kvh * g + col % g) = __builtin_convertvector(j.o * (1.0f / j.l), bf16x4);
        }
    }
}

}  // namespace

// The most columns that a sequence of a call can have.
static int64_t most_cols(int n_q, int n_kv, int max_new) { return (int64_t)max_new * (n_q / n_kv); }

size_t attention8_workspace_bytes(int n_q, int n_kv, int d, int max_new) {
    Parts t;
    const int64_t cols = most_cols(n_q, n_kv, max_new);
    if (cols <= kStreamCols) return parts_in<false, kStreamCols>(t, nullptr, n_kv, d);
    return cols <= kWideCols ? parts_in<false, kWideCols>(t, nullptr, n_kv, d) : parts_in<true, kStreamCols>(t, nullptr, n_kv, d);
}

template <int D, bool TILES, int COLS>
static gllm_status launch(const Attn8Args& a, hipStream_t stream) {
    // the stream's workgroups; no more tiles than whole ones in all rows and a partly filled one per sequence, and cutting the keys adds no more units
    // than twice the target; and one place behind the last unit
    const int g = a.n_q / a.n_kv;
    const int64_t tiles = TILES ? (int64_t)a.num_rows * g / kTileCols + a.num_seqs : 0;
    const int64_t places = max_workers<TILES, COLS>(a.n_kv, D) + tiles + (TILES ? 2 * target_units(a.n_kv) : 0) + 1;
    Parts parts;
    parts_in<TILES, COLS>(parts, a.workspace, a.n_kv, D);
    // the joining: no sequence can be cut that has no more blocks than these
    const int64_t own = ceil_div(a.table_stride, kBlock / kPage), rows = TILES ? kTileCols / g + 2 : COLS / g;
    const bool joined = most_blocks(own, rows, a.window, a.sinks) > (TILES && kMinShare < kWhole ? kMinShare : kWhole);
    const int64_t records = a.num_seqs <= 64 ? a.num_seqs : std::min<int64_t>(parts.max_waves, (int64_t)a.num_seqs * most_blocks(own, COLS / g, a.window, a.sinks) + 8);
    // columns of few streams are spread over workgroups
    const int64_t split = std::max<int64_t>(1, std::min<int64_t>(COLS / 4, kGroups / (records * a.n_kv))), stream_groups = records * a.n_kv * split;
    const int64_t tile_groups = TILES ? std::min<int64_t>(2048, std::min<int64_t>(max_cut_tiles(a.n_kv), tiles) * a.n_kv * (kTileCols * D / 1024)) : 0;
    const int join_threads = a.num_seqs <= 64 ? 512 : 256;
    if (places * a.n_kv * kThreads<TILES> > UINT32_MAX || (joined && (stream_groups + tile_groups) * join_threads > UINT32_MAX)) return GLLM_E_CAPACITY;
    if (!plans_alone<TILES>(a.num_seqs)) attention8_plan_kernel<TILES, COLS><<<1, 1024, 0, stream>>>(a, parts.plan, parts.count);
    const int lds = TILES ? sizeof(TileLds<D>) : 0;
    if (TILES) {
        static std::atomic<uint64_t> allowed{0};  // devices on which this kernel may use the LDS that it asks for
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess) return GLLM_E_HIP;
        if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(attention8_kernel<D, TILES, COLS>), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
                return GLLM_E_HIP;
            if (dev < 64) allowed.fetch_or(1ull << dev);
        }
    }
    attention8_kernel<D, TILES, COLS><<<(unsigned)(places * a.n_kv), kThreads<TILES>, lds, stream>>>(a);
    if (joined) {
        const dim3 grid((unsigned)(stream_groups + tile_groups));
        if (a.num_seqs <= 64) attention8_merge_kernel<D, TILES, COLS, 512><<<grid, 512, 0, stream>>>(a, (int)stream_groups, (int)split);
        else attention8_merge_kernel<D, TILES, COLS, 256><<<grid, 256, 0, stream>>>(a, (int)stream_groups, (int)split);
    }
    return hipGetLastError() == hipSuccess ? GLLM_OK : GLLM_E_HIP;
}

template <int D>
static gllm_status launch_for(const Attn8Args& a, hipStream_t stream) {
    const int64_t cols = most_cols(a.n_q, a.n_kv, a.max_new);
    if (cols <= kStreamCols) return launch<D, false, kStreamCols>(a, stream);
    return cols <= kWideCols ? launch<D, false, kWideCols>(a, stream) : launch<D, true, kStreamCols>(a, stream);
}

gllm_status launch_attention8(const Attn8Args& a, hipStream_t stream) {
    if (a.num_seqs <= 0 || a.num_rows <= 0) return GLLM_OK;
    if (a.num_seqs > kMaxAttn8Seqs || (int64_t)a.num_rows * (a.n_q / a.n_kv) > INT32_MAX) return GLLM_E_CAPACITY;
    if (a.d == 128) return launch_for<128>(a, stream);
    if (a.d == 64) return launch_for<64>(a, stream);
    return GLLM_E_UNSUPPORTED;
}
