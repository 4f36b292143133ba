// Attention of hybrid batches over the 8-bit pool (contract: include/gllm_cache8.h).
//
// Per KV head the n rows of a sequence times the g query heads of the group are n*g columns over one stream of keys, column j being head
// j % g of row j / g:  S^T = K.Q^T, softmax down the columns with a running reference, O^T += V^T.P^T, in transposed form so that the
// scores a lane receives are the operand that it supplies (kernels_attn.hip).  A code times its page's scale is a value: codes become bf16
// without rounding (4 bits of mantissa), the key scale s_k of a page multiplies its scores and the value scale s_v its weights,
//     p s_v = 2^(s c s_k - m + log2 s_v),   c = scale * log2(e),
// both in the one multiply-add that the exponential's argument takes anyway; a lane holds keys of one page only, so that its part of the sum of
// the weights is that of p s_v times 1 / s_v.
//
// Up to 16 columns (decode rows) the keys are a stream from HBM: stream_unit.  More go in tiles whose keys pass through LDS: tile_unit.
// The keys of long sequences are cut into parts, planned on the device, and the parts' results joined by a second launch.
#include "cache8.h"

#include <atomic>

namespace {

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr float kNegBig = -1.0e30f;
constexpr int kBlock = 64;  // keys, four pages

// ---- the plan --------------------------------------------------------------------------------------------------------------

// Columns of a tile by the columns of a sequence.
constexpr int kStreamCols = 16, kTileCols = 256;
__host__ __device__ constexpr int tile_cols(int64_t cols) { return cols <= kStreamCols ? kStreamCols : kTileCols; }

// A unit of work: a part of the keys for the columns of one tile of a sequence.
struct Unit {
    int32_t seq, row0, n, c;
    int32_t width;               // tile_cols()
    int32_t tile, part, parts;
    bool broken;                 // the sequence breaks a rule: zeros
    int32_t place;               // parts > 1: of its partial results, in columns
    int32_t step;                // and from a part's to the next one's
    int32_t cut_tile;            // and of its tile among those with such units
};

constexpr int kMinShare = 6;     // fewest blocks worth a workgroup
// Workgroups that the keys are cut into, over all KV heads.
template <bool TILES>
__host__ __device__ constexpr int target_units(int n_kv) { return (TILES ? 512 : 768) / n_kv > 0 ? (TILES ? 512 : 768) / n_kv : 1; }
// Columns of partial results, and tiles that have them.  A sequence is cut where it has more blocks than a share, into at most ceil(blocks /
// share) parts; the shares of all are at least half their blocks by the target (seq_plan: twice the weight is at least the blocks).
template <bool TILES>
__host__ __device__ constexpr int max_cut_tiles(int n_kv) { return 2 * target_units<TILES>(n_kv); }
template <bool TILES>
__host__ __device__ constexpr int max_places(int n_kv) { return 4 * target_units<TILES>(n_kv) * (TILES ? kTileCols : kStreamCols); }

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

struct SeqPlan {
    int32_t row0, n, c, width, tiles, blocks;  // blocks: of the tile that sees most, at most
    float weight;                              // tiles times about their blocks, at least half of tiles * blocks
    bool broken, unordered;
};
__device__ __forceinline__ SeqPlan seq_plan(const Attn8Args& a, int s) {
    SeqPlan p{0, 0, 0, kStreamCols, 0, 0, 0.f, true, false};
    if (s >= a.num_seqs) return p;
    const int r0 = a.row_start[s], r1 = a.row_start[s + 1], g = a.n_q / a.n_kv;
    p.c = a.cached_len[s];
    p.unordered = r0 < 0 || r1 < r0 || r1 > a.num_rows;
    p.row0 = r0;
    p.n = p.unordered ? 0 : r1 - r0;
    p.broken = p.n > a.max_new || p.c < 0 || (int64_t)p.c + p.n > min((int64_t)a.table_stride * kPage, (int64_t)kMaxPositions);
    p.width = (int64_t)a.max_new * g <= kStreamCols ? kStreamCols : tile_cols((int64_t)p.n * g);  // (a call of short sequences has stream units only)
    p.tiles = (p.n * g + p.width - 1) / p.width;  // (num_rows * g fits 31 bits: the launcher)
    if (p.broken || p.n == 0) return p;
    const int all = (p.c + p.n - 1) / kBlock + 1;
    p.blocks = all;
    if (a.window > 0) {
        const int64_t near = ((int64_t)a.window + p.width / g + 1 + kBlock - 2) / kBlock + 1 + a.sinks / kBlock + 1;
        p.blocks = (int)min((int64_t)all, near);
    }
    p.weight = (float)p.tiles * (p.tiles > 1 ? min((float)p.blocks, (2.f * p.c + p.n) * (0.5f / kBlock) + 2.f) : (float)p.blocks);
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
__device__ __forceinline__ float lane_value(float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); }

// Blocks of a share.  (The sum is exact up to 2^24, and by 1e-4 of itself more from there on, which is more than the roundings of its additions,
// 2^-24 of it each, take away: kMaxAttn8Seqs / 4096 of a lane and 15 over lanes and runs.)
static_assert(kMaxAttn8Seqs / (64 * 64) + 15 < 16777216 / 10000, "the sum of all weights");
template <bool TILES>
__device__ __forceinline__ int share_of(float total, int n_kv) {
    const float target = (float)target_units<TILES>(n_kv);
    const float even = total < 16777216.f ? ceilf(total / target) : total / target * 1.0001f + 1.f;
    return (int)fminf(fmaxf(even, (float)kMinShare), 1e9f);
}
// The units of a sequence.  They are in order of their size, in quarters of a share, so that the last workgroups to start are short ones;
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
    int cut_upto = cut ? units * q.width : 0, tiles_upto = cut ? q.tiles : 0;
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
        u.width = lane_value(q.width, l);
        u.broken = lane_value((int)q.broken, l);
        u.parts = lane_value(parts, l);
        u.part = i / tiles;
        u.tile = tiles - 1 - (i - u.part * tiles);
        u.step = tiles * u.width;
        u.place = places + lane_value(cut_upto - (cut ? units * q.width : 0), l) + u.part * u.step + u.tile * u.width;
        u.cut_tile = cut_tiles + lane_value(tiles_upto - (cut ? q.tiles : 0), l) + u.tile;
        return true;
    }
    places += lane_value(cut_upto, 63);
    cut_tiles += lane_value(tiles_upto, 63);
    return false;
}

// Up to 64 sequences every wave works the plan out for itself, all of them with the same arithmetic, without LDS and barriers.  More are
// planned by a launch of their own, which cuts them into up to 64 runs of whole waves and leaves what stands in front of each; a wave then looks
// at the runs and at one of them.
constexpr int kPlanRuns = 64;
struct Plan {
    int32_t share, units;               // units: none where the rows break their order
    int32_t start[4];                   // place of the first unit of a quarter
    int32_t before[4][kPlanRuns];       // place of a run's first unit in a quarter
    int32_t places[kPlanRuns], cut_tiles[kPlanRuns];  // in front of a run
};
__host__ __device__ inline int plan_run(int num_seqs) { return (num_seqs + 64 * kPlanRuns - 1) / (64 * kPlanRuns) * 64; }  // sequences

// false behind the last unit.  cut_tiles: behind it the number of tiles whose keys are cut, or -1 where the plan's launch has written it.
template <bool TILES>
__device__ __forceinline__ bool find_unit(const Attn8Args& a, const Plan* plan, int place, Unit& u, int& cut_tiles) {
    const int lane = threadIdx.x & 63;
    int places = 0;
    if (a.num_seqs > 64) {
        cut_tiles = -1;
        if (place >= plan->units) return false;
        const int share = plan->share;
        const int quarter = (place >= plan->start[1]) + (place >= plan->start[2]) + (place >= plan->start[3]);
        const int first = plan->before[quarter][lane];
        const int run = __popcll(__ballot(first <= place)) - 1, begin = run * plan_run(a.num_seqs), end = min(begin + plan_run(a.num_seqs), a.num_seqs);
        int at = lane_value(first, run), cut = plan->cut_tiles[run];
        places = plan->places[run];
        for (int s0 = begin; s0 < end; s0 += 64) {
            const SeqPlan q = seq_plan(a, s0 + lane);
            int parts, its;
            const int units = split_seq(q, share, parts, its), mine = its == quarter ? units : 0;
            int x = mine;
            scan_wave(x);
            if (unit_of(q, parts, units, mine, at + x - mine, place, s0, places, cut, u)) return true;
            at += lane_value(x, 63);
        }
        return false;
    }
    const SeqPlan p = seq_plan(a, lane);
    cut_tiles = 0;
    if (__any(p.unordered)) return false;  // rows in no order may belong to two sequences: the launch would have no place for their units
    float total = p.weight;
    scan_wave(total);
    total = lane_value(total, 63);
    int parts, quarter, before = 0, start = 0;
    const int units = split_seq(p, share_of<TILES>(total, a.n_kv), parts, quarter);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        int x = quarter == c ? units : 0;
        scan_wave(x);
        if (quarter == c) before = start + x - units;
        start += lane_value(x, 63);
    }
    return unit_of(p, parts, units, units, before, place, 0, places, cut_tiles, u);
}

// One workgroup; wave w has the runs w, w + 16, ...
template <bool TILES>
__global__ __launch_bounds__(1024) void attention8_plan_kernel(Attn8Args a, Plan* plan, int32_t* count) {
    __shared__ float totals[kPlanRuns];
    __shared__ int sums[6][kPlanRuns];  // of a run: units of each quarter, places, tiles that are cut
    __shared__ int any_unordered;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int len = plan_run(a.num_seqs);
    if (threadIdx.x < kPlanRuns) {
        totals[threadIdx.x] = 0.f;
        for (int k = 0; k < 6; ++k) sums[k][threadIdx.x] = 0;
    }
    if (threadIdx.x == 0) any_unordered = 0;
    __syncthreads();
    for (int run = wave; run < kPlanRuns && run * len < a.num_seqs; run += 16) {
        float total = 0.f;
        bool unordered = false;
        for (int s0 = run * len; s0 < min((run + 1) * len, a.num_seqs); s0 += 64) {
            const SeqPlan q = seq_plan(a, s0 + lane);
            total += q.weight;
            unordered |= q.unordered;
        }
        scan_wave(total);
        if (lane == 63) totals[run] = total;
        if (unordered) any_unordered = 1;
    }
    __syncthreads();
    float total = totals[lane];
    scan_wave(total);
    const int share = share_of<TILES>(lane_value(total, 63), a.n_kv);
    for (int run = wave; run < kPlanRuns && run * len < a.num_seqs; run += 16) {
        int sum[6] = {0, 0, 0, 0, 0, 0};
        for (int s0 = run * len; s0 < min((run + 1) * len, a.num_seqs); s0 += 64) {
            const SeqPlan q = seq_plan(a, s0 + lane);
            int parts, quarter;
            const int units = split_seq(q, share, parts, quarter);
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] += quarter == c ? units : 0;
            sum[4] += parts > 1 ? units * q.width : 0;
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
            (k == 4 ? plan->places : plan->cut_tiles)[lane] = upto - own;
            if (k == 5 && lane == 0) *count = any_unordered ? 0 : all;
        }
    }
    if (lane == 0) {
        plan->share = share;
        plan->units = any_unordered ? 0 : start;
    }
}

// ---- partial results ------------------------------------------------------------------------------------------------------
//
// Workspace: the plan of many sequences, a record per tile whose keys are cut, then per KV head and column of a part the reference and the sum,
// then the unnormalised outputs.
struct Record {
    int32_t row0, n, tile, width;
    int32_t place, step, parts, pad;
};
struct Parts {
    int32_t* count;  // records
    Plan* plan;
    Record* rec;
    f32x2* ml;       // [n_kv][places]
    float* o;        // [n_kv][places][d]
    int64_t places;
};
template <bool TILES>
__host__ __device__ inline size_t parts_in(Parts& t, void* base, int n_kv, int d) {
    t.places = max_places<TILES>(n_kv);
    const size_t cols = (size_t)t.places * n_kv;
    char* p = (char*)base;
    t.count = (int32_t*)p;
    t.plan = (Plan*)(p + 256);
    constexpr size_t head = 256 + (sizeof(Plan) + 255) / 256 * 256;
    t.rec = (Record*)(p + head);
    size_t off = head + (max_cut_tiles<TILES>(n_kv) * sizeof(Record) + 255) / 256 * 256;
    t.ml = (f32x2*)(p + off);
    off += (cols * 8 + 255) / 256 * 256;
    t.o = (float*)(p + off);
    return off + cols * d * 4;
}

// ---- common to both kinds of units -------------------------------------------------------------------------------------

// A barrier that waits for this wave's reads and writes of LDS only: __syncthreads() would wait for the loads into the ring too.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Four codes as bf16, without rounding.
__device__ __forceinline__ u32x2 widen(uint32_t codes) {
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, true))};
}
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi) {
    const u32x2 a = widen(lo), b = widen(hi);
    return u32x4{a[0], a[1], b[0], b[1]};
}
// Bit 7 of every byte that is no number.
__device__ __forceinline__ uint32_t no_numbers(uint32_t codes) { return ((codes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// What a page's scales come to: the factor of its scores, log2 of that of its weights, and one over that.
struct PageScale {
    float keys, log_values, per_value;
    __device__ __forceinline__ void of(f32x2 s, float scale_log2) {
        keys = fminf(fmaxf(s[0], kScaleMin), kScaleMax) * scale_log2;
        const float v = fminf(fmaxf(s[1], kScaleMin), kScaleMax);
        log_values = __builtin_amdgcn_logf(v);
        per_value = __builtin_amdgcn_rcpf(v);
    }
};

// ---- few columns -----------------------------------------------------------------------------------------------------------
//
// Each wave takes a run of the unit's blocks for all columns, operands straight to registers.  Matrix instructions of 16x16x32: the row 4q + i of
// score tile t is slot 4t + i of page q, so that a lane of group G receives the 16 slots of page G.  An instruction that loads keys takes runs of
// 256 bytes from each of the four pages, one that loads values the 16 slots of 16 dims of each.
template <int D>
struct Frag {
    u32x4 k[4][D / 64];  // [tile][64 dims]: row r = slot 4t + r % 4 of page r / 4, dims 16 (4p + G) ..
    u32x4 v[D / 16];     // [16 dims]: dim 16b + r of page G
};
template <int D, int WAVES>
struct StreamLds {
    float o[WAVES][16][D + 4];
    float m[WAVES][16], l[WAVES][16];
};

template <int D, int WAVES>
__device__ __forceinline__ void stream_unit(const Attn8Args& a, const Unit& it, const Parts& parts, int kvh, StreamLds<D, WAVES>& join) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, G = lane >> 4, g = a.n_q / a.n_kv;
    const int cols = it.n * g;
    const Seen seen = seen_blocks(a, it.c, 0, it.n - 1);
    const int each = seen.blocks / it.parts, more = seen.blocks - each * it.parts;
    const int first = it.broken ? 0 : it.part * each + min(it.part, more), last = it.broken ? 0 : first + each + (it.part < more);
    const int run = (last - first + WAVES - 1) / WAVES;
    const int b_begin = min(first + wave * run, last), b_end = min(b_begin + run, last);
    const int last_page = max(it.c + it.n - 1, 0) / kPage;
    const int32_t* bt = a.block_tables + (int64_t)it.seq * a.table_stride;

    int ids_base = b_begin, ids = 0;  // pages of 16 blocks, one per lane, with their scales
    PageScale ps;
    auto fetch_ids = [&](int base) {
        ids_base = base;
        ids = min(max(bt[min(seen.actual(base + lane / 4) * 4 + lane % 4, last_page)], 0), a.num_blocks - 1);
        ps.of(a.scales[(int64_t)ids * a.n_kv + kvh], a.scale_log2);
    };
    auto load_block = [&](Frag<D>& f, int b) {
        constexpr int PH = D * kPage;  // bytes of a page's head
        const int at = (b - ids_base) * 4;
        const uint8_t* k = a.k_pool + ((int64_t)__shfl(ids, at + (r >> 2)) * a.n_kv + kvh) * PH + G * 64 + (r & 3) * 16;
        const uint8_t* v = a.v_pool + ((int64_t)__shfl(ids, at + G) * a.n_kv + kvh) * PH + r * kPage;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int p = 0; p < D / 64; ++p) f.k[t][p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k + t * (4 * D) + p * 256));
#pragma unroll
        for (int b16 = 0; b16 < D / 16; ++b16) f.v[b16] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(v + b16 * 256));
    };
    Frag<D> fa, fb;
    if (b_begin < b_end) {
        fetch_ids(b_begin);
        load_block(fa, b_begin);
    }
    bf16x8 qf[D / 64][2];
    const int col = min(it.tile * kStreamCols + r, cols - 1), row = col / g;
    const bf16_t* qrow = a.q + (int64_t)(it.row0 + row) * a.ld_q + (int64_t)(kvh * g + col - row * g) * D;
#pragma unroll
    for (int p = 0; p < D / 64; ++p)
#pragma unroll
        for (int h = 0; h < 2; ++h) qf[p][h] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + 64 * p + 16 * G + 8 * h));

    f32x4 o[D / 16];
    float m = kNegBig, l = 0.f;
#pragma unroll
    for (int b = 0; b < D / 16; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int pos = it.c + row, low = a.window > 0 ? pos - a.window : -1;  // this column sees keys up to pos and above low, or below sinks
    const int pos_min = it.c, low_max = a.window > 0 ? it.c + it.n - 1 - a.window : -1;
    auto attend = [&](Frag<D>& f, int b) {
        const int key0 = seen.actual(b) * kBlock, at = (b - ids_base) * 4 + G;
        const float factor = __shfl(ps.keys, at), log_values = __shfl(ps.log_values, at), per_value = __shfl(ps.per_value, at);
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < D / 64; ++p)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, widen8(f.k[t][p][2 * h], f.k[t][p][2 * h + 1])), qf[p][h], s[t], 0, 0, 0);
        }
        if (key0 + kBlock - 1 > pos_min || (key0 <= low_max && key0 + kBlock > a.sinks)) {  // not all keys are seen by all columns
            // values that are no numbers may reach the columns that see them only: they are emptied and the key's scores are no numbers
            u32x4 bad = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int b16 = 0; b16 < D / 16; ++b16)
#pragma unroll
                for (int w = 0; w < 4; ++w) bad[w] |= no_numbers(f.v[b16][w]);
            if (__any((bad[0] | bad[1] | bad[2] | bad[3]) != 0u)) {
#pragma unroll
                for (int b16 = 0; b16 < D / 16; ++b16)
#pragma unroll
                    for (int w = 0; w < 4; ++w) f.v[b16][w] &= ~((no_numbers(f.v[b16][w]) >> 7) * 0xFFu);
#pragma unroll
                for (int w = 0; w < 4; ++w)
#pragma unroll
                    for (int by = 1; by < 16; by *= 2) bad[w] |= (uint32_t)__shfl_xor((int)bad[w], by);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = key0 + G * kPage + 4 * t + i;
                    const bool hidden = (key > pos) | ((key <= low) & (key >= a.sinks));
                    s[t][i] = hidden ? -INFINITY : bad[t] >> (8 * i + 7) & 1 ? NAN : s[t][i];
                }
        }
        float top = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
#pragma unroll
        for (int t = 1; t < 4; ++t) top = fmaxf(top, fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])));
        top *= factor;
        if (__any(top > m)) {  // the reference moves to the running maximum, the same in the four lanes of a column
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), m);
            const float down = __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= down;
#pragma unroll
            for (int b16 = 0; b16 < D / 16; ++b16)
#pragma unroll
                for (int v = 0; v < 4; ++v) o[b16][v] *= down;
        }
        const float shift = log_values - m;
        float sum = 0.f;
        bf16x8 w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            f32x8 p;
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                p[v] = __builtin_amdgcn_exp2f(fmaf(s[2 * j + v / 4][v % 4], factor, shift));
                sum += p[v];
            }
            w[j] = __builtin_convertvector(p, bf16x8);
        }
        l += sum * per_value;
#pragma unroll
        for (int b16 = 0; b16 < D / 16; ++b16)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                o[b16] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, widen8(f.v[b16][2 * j], f.v[b16][2 * j + 1])), w[j], o[b16], 0, 0, 0);
    };
    for (int b = b_begin; b < b_end; b += 2) {  // (16 blocks of page ids: an even number, so that they run out in front of fa only)
        if (b + 1 < b_end) load_block(fb, b + 1);
        attend(fa, b);
        if (b + 2 < b_end && b + 2 < ids_base + 16) load_block(fa, b + 2);
        if (b + 1 < b_end) attend(fb, b + 1);
        if (b + 2 < b_end && b + 2 >= ids_base + 16) {
            fetch_ids(b + 2);
            load_block(fa, b + 2);
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (G == 0) {
        join.m[wave][r] = m;
        join.l[wave][r] = l;
    }
#pragma unroll
    for (int b = 0; b < D / 16; ++b) *reinterpret_cast<f32x4*>(&join.o[wave][r][b * 16 + G * 4]) = o[b];
    __syncthreads();
    const int here = min(kStreamCols, cols - it.tile * kStreamCols);
    for (int i = threadIdx.x; i < here * (D / 4); i += 64 * WAVES) {
        const int j = i / (D / 4), e = i % (D / 4) * 4, cc = it.tile * kStreamCols + j, rr = cc / g;
        float ms = kNegBig, ls = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) ms = fmaxf(ms, join.m[w][j]);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float x = __builtin_amdgcn_exp2f(join.m[w][j] - ms);
            const f32x4 ow = *reinterpret_cast<const f32x4*>(&join.o[w][j][e]);
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[v] += ow[v] * x;
            ls += join.l[w][j] * x;
        }
        if (it.parts > 1) {
            const int64_t place = kvh * parts.places + it.place + j;
            *reinterpret_cast<f32x4*>(parts.o + place * D + e) = acc;
            if (e == 0) parts.ml[place] = f32x2{ms, ls};
            continue;
        }
        const float inv = it.broken ? 0.f : 1.0f / ls;
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[v] *= inv;
        *reinterpret_cast<bf16x4*>(a.out + (int64_t)(it.row0 + rr) * a.ld_o + (int64_t)(kvh * g + cc - rr * g) * D + e) = __builtin_convertvector(acc, bf16x4);
    }
}

// ---- tiles of columns --------------------------------------------------------------------------------------------------------
//
// One workgroup of 8 waves, 32 columns a wave, matrix instructions of 32x32x16.  Keys come in blocks of 64, four pages: their codes go from HBM
// into a ring in LDS, each thread turns the pieces that it asked for into bf16, and all waves read these, half a block (two pages) after the other.
// The row 8a + 4h + b of a score tile is slot 4a + b of page h of the half, so that the lanes of half h receive the 16 slots of page h.
//   keys as bf16    [half][D / 8][32 rows][8 dims], row x of piece c at x ^ 4 (c / 2 % 4): the writes of 16 lanes hit different banks
//   values as bf16  [page][2 halves of the slots][D][8 slots]
// The exponentials of a half run beside the scores of the next one and in front of its own outputs; what a phase reads from LDS is asked for in the
// phase before.
constexpr int kHalf = 32, kRaw = 4, kKeyStages = 2, kValueStages = 2, kWindow = 64;
struct PageEntry {
    int32_t id;
    PageScale scale;
};
template <int D>
struct TileLds {
    unsigned char raw[kRaw][2][kBlock * D];         // [block][keys, values]: codes as loaded; the keys of block j with the values of block j - 1
    unsigned char keys[kKeyStages][2][kHalf * D * 2];
    unsigned char values[kValueStages][2][kHalf * D * 2];
    PageEntry pages[2][kWindow * 4];                // of 64 blocks and the next 64
    uint32_t bad[4][2];                             // of a half: bit 16h + t: slot t of page h has values that are no numbers
};
constexpr float kSlack = 32.0f;  // a reference lags by up to this: weights stay below 2^32

template <int D>
__device__ __forceinline__ void tile_unit(const Attn8Args& a, const Unit& it, const Parts& parts, int kvh, TileLds<D>& lds) {
    constexpr int PH = D * kPage;         // bytes of a page's head
    constexpr bool BOTH = D == 128;       // a thread has a piece of keys and one of values; or the lower waves keys, the upper ones values
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, h = lane >> 5, g = a.n_q / a.n_kv;
    const int cols = it.n * g, col0 = it.tile * it.width, ncols = min(it.width, cols - col0);
    const int i0 = col0 / g, i1 = (col0 + ncols - 1) / g;
    const Seen seen = seen_blocks(a, it.c, i0, i1);
    const int each = seen.blocks / it.parts, more = seen.blocks - each * it.parts;
    const int first = it.part * each + min(it.part, more), blocks = it.broken ? 0 : each + (it.part < more);
    const int last_page = max(it.c + it.n - 1, 0) / kPage;
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
            e.scale.of(sc, a.scale_log2);
            lds.pages[x / (kWindow * 4) % 2][x % (kWindow * 4)] = e;
        };
        auto entry_of = [&](int b, int q) -> const PageEntry& { return lds.pages[b / kWindow % 2][b % kWindow * 4 + q]; };
        // The pieces of a side of a block are 16 bytes, 4D of them, page after page.
        const bool has_keys = BOTH || wave < 4, has_values = BOTH || wave >= 4;
        const int piece = BOTH ? threadIdx.x : threadIdx.x & 255, page = piece / D, piece_at = piece % D;
        const int64_t piece_off = (int64_t)kvh * PH + piece_at * 16, page_step = (int64_t)a.n_kv * PH;
        // every wave issues its pieces (of the last block again behind it), so that the number on their way is the same in every round
        auto issue = [&](int j, int id_keys, int id_values) {  // the keys of block j and the values of block j - 1
            unsigned char* to = &lds.raw[j % kRaw][0][0] + wave * 1024;
            if (has_keys) __builtin_amdgcn_global_load_lds((gptr_t)(a.k_pool + id_keys * page_step + piece_off), (lptr_t)to, 16, 0, 0);
            if (has_values) __builtin_amdgcn_global_load_lds((gptr_t)(a.v_pool + id_values * page_step + piece_off), (lptr_t)(to + (BOTH ? kBlock * D : 0)), 16, 0, 0);
        };
        auto id_of = [&](int j) { return entry_of(min(max(j, 0), blocks - 1), page).id; };  // (the same for the wave; read a round before it is wanted)
        auto raw_keys = [&](int j) { return *reinterpret_cast<const u32x4*>(&lds.raw[j % kRaw][0][0] + threadIdx.x * 16); };  // which have come
        auto raw_values = [&](int j) { return *reinterpret_cast<const u32x4*>(&lds.raw[j % kRaw][0][0] + threadIdx.x * 16 + (BOTH ? kBlock * D : 0)); };
        // Values that are no numbers may reach the columns that see them only: where not all rows see all keys they are emptied, and the key's scores are
        // no numbers.
        auto clean = [&](int b, u32x4& x) {
            if (!has_values || !partly(key_of(min(b, blocks - 1)), kBlock, it.c + i0, it.c + i1)) return;  // (the same for the wave)
            uint32_t some = 0u;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t n = no_numbers(x[w]);
                x[w] &= ~((n >> 7) * 0xFFu);
                some |= ((n >> 7 & 1) | (n >> 14 & 2) | (n >> 21 & 4) | (n >> 28 & 8)) << (4 * w);
            }
            if (some) atomicOr(&lds.bad[b % 4][page / 2], some << (16 * (page % 2)));
        };
        // where the two halves of a piece go as bf16
        const int chunk = piece_at % (D / 4) / 4, key_row = (8 * (piece_at / (D / 4)) + 4 * (page % 2) + piece_at % 4) ^ (4 * (chunk & 3));
        const int keys_at = (page / 2) * (kHalf * D * 2) + (2 * chunk * 32 + key_row) * 16, values_at = (2 * page * D + piece_at) * 16;
        auto put_keys = [&](int b, u32x4 lo, u32x4 hi) {
            if (!has_keys) return;
            unsigned char* to = &lds.keys[b % kKeyStages][0][0] + keys_at;
            *reinterpret_cast<u32x4*>(to) = lo;
            *reinterpret_cast<u32x4*>(to + 32 * 16) = hi;
        };
        auto put_values = [&](int b, u32x4 lo, u32x4 hi) {
            if (!has_values) return;
            unsigned char* to = &lds.values[b % kValueStages][0][0] + values_at;
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
            if (partly(key0, kHalf, wave_min, wave_max)) {
                const uint32_t bad = lds.bad[b % 4][half] >> (16 * h);
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int key = key0 + h * kPage + v;
                    const bool hidden = (key > pos) | ((key <= low) & (key >= a.sinks));
                    s[v] = hidden ? -INFINITY : bad >> v & 1 ? NAN : s[v];
                }
                top = largest(s);
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
        auto read_key = [&](int b, int half, int k) { kf[k] = *reinterpret_cast<const bf16x8*>(lds.keys[b % kKeyStages][half] + ((2 * k + h) * 32 + (r ^ (4 * (k & 3)))) * 16); };
        auto read_value = [&](int b, int half, int x) {
            vf[x % (D / 32)][x / (D / 32)] = *reinterpret_cast<const bf16x8*>(lds.values[b % kValueStages][half] + ((2 * h + x / (D / 32)) * D + x % (D / 32) * 32 + r) * 16);
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

        if (threadIdx.x < 8) (&lds.bad[0][0])[threadIdx.x] = 0u;
        {
            const int id = page_of(threadIdx.x);
            entry(threadIdx.x, id, a.scales[(int64_t)id * a.n_kv + kvh]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kRaw; ++j) issue(j, __builtin_amdgcn_readfirstlane(id_of(j)), __builtin_amdgcn_readfirstlane(id_of(j - 1)));
        // the keys of blocks 0 and 1, the values of block 0
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kRaw - 2) * (BOTH ? 2 : 1)) : "memory");
        {
            u32x4 x = raw_keys(0);
            put_keys(0, widen8(x[0], x[1]), widen8(x[2], x[3]));
            x = raw_keys(1);
            put_keys(1, widen8(x[0], x[1]), widen8(x[2], x[3]));
            x = raw_values(1);
            clean(0, x);
            put_values(0, widen8(x[0], x[1]), widen8(x[2], x[3]));
        }
        lds_barrier();
        int id_keys = id_of(kRaw), id_values = id_of(kRaw - 1);
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
        lds_barrier();  // the keys of block 0 have been read, and those of block 2 may take their place
        int window_id = 0;
        f32x2 window_scale = {0.f, 0.f};
        for (int b = 0; b < blocks; ++b) {
            // the keys of block b + 2 and the values of block b + 1 have come, and nobody reads the stages that they go to any more
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kRaw - 3) * (BOTH ? 2 : 1)) : "memory");
            const int behind = b % kWindow;
            if (behind <= 2 && b >= kWindow) {  // the pages of the next window but one, in three rounds
                const int x = (b / kWindow + 1) * kWindow * 4 + (int)threadIdx.x;
                if (threadIdx.x < kWindow * 4) {
                    if (behind == 0) window_id = page_of(x);
                    else if (behind == 1) window_scale = a.scales[(int64_t)window_id * a.n_kv + kvh];
                    else entry(x, window_id, window_scale);
                }
            }
            issue(b + kRaw, __builtin_amdgcn_readfirstlane(id_keys), __builtin_amdgcn_readfirstlane(id_values));
            u32x4 rk = raw_keys(b + 2), rv = raw_values(b + 2);
            id_keys = id_of(b + kRaw + 1);
            id_values = id_of(b + kRaw);
            if (threadIdx.x < 2) lds.bad[(b + 3) % 4][threadIdx.x] = 0u;
            const PageScale then = entry_of(b, 2 + h).scale, after = entry_of(min(b + 1, blocks - 1), h).scale;
            clean(b + 1, rv);
            u32x4 wide[4];
            if (!idle) {
                half_block(b, 0, s, top, now, [&](int x) {
                    if (x == 1) wide[0] = widen8(rk[0], rk[1]);
                    if (x == 3) wide[1] = widen8(rk[2], rk[3]);
                });
                put_keys(b + 2, wide[0], wide[1]);
                settle(b, 1, s, top, then);
                half_block(b, 1, s, top, then, [&](int x) {
                    if (x == 1) wide[2] = widen8(rv[0], rv[1]);
                    if (x == 3) wide[3] = widen8(rv[2], rv[3]);
                });
            } else {
                wide[0] = widen8(rk[0], rk[1]);
                wide[1] = widen8(rk[2], rk[3]);
                wide[2] = widen8(rv[0], rv[1]);
                wide[3] = widen8(rv[2], rv[3]);
            }
            if (idle) put_keys(b + 2, wide[0], wide[1]);
            put_values(b + 1, wide[2], wide[3]);
            lds_barrier();
            now = after;
            if (!idle && b + 1 < blocks) settle(b + 1, 0, s, top, now);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no LDS fill may outlive the workgroup
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
    const float inv = it.broken ? 0.f : 1.0f / l;
    bf16_t* orow = a.out + (int64_t)(it.row0 + row) * a.ld_o + (int64_t)(kvh * g + col - row * g) * D;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 x = {o[t][4 * b] * inv, o[t][4 * b + 1] * inv, o[t][4 * b + 2] * inv, o[t][4 * b + 3] * inv};
            *reinterpret_cast<bf16x4*>(orow + t * 32 + b * 8 + h * 4) = __builtin_convertvector(x, bf16x4);
        }
}

// Threads of a workgroup: four waves where there are stream units only, two workgroups to a compute unit, eight with tiles.
template <bool TILES>
constexpr int kThreads = TILES ? 512 : 256;

template <int D, bool TILES>
__global__ __launch_bounds__(kThreads<TILES>, 2) void attention8_kernel(Attn8Args a) {
    // (one LDS object: with a second one the compiler waits for all loads into the ring before it reads from it)
    extern __shared__ __attribute__((aligned(1024))) unsigned char attn8_lds[];
    const int kvh = blockIdx.x % a.n_kv;
    Unit it;
    Parts parts;
    parts_in<TILES>(parts, a.workspace, a.n_kv, D);
    int cut_tiles;
    if (!find_unit<TILES>(a, parts.plan, blockIdx.x / a.n_kv, it, cut_tiles)) {
        if (cut_tiles >= 0 && blockIdx.x + 1 == gridDim.x && threadIdx.x == 0) *parts.count = cut_tiles;  // (the last workgroup is behind the last unit)
        return;
    }
    if (it.parts > 1 && it.part == 0 && kvh == 0 && threadIdx.x == 0)
        parts.rec[it.cut_tile] = Record{it.row0, it.n, it.tile, it.width, it.place, it.step, it.parts, 0};
    if (!TILES || it.width == kStreamCols) stream_unit<D, kThreads<TILES> / 64>(a, it, parts, kvh, *reinterpret_cast<StreamLds<D, kThreads<TILES> / 64>*>(attn8_lds));
    else tile_unit<D>(a, it, parts, kvh, *reinterpret_cast<TileLds<D>*>(attn8_lds));
}

// The partial results of all tiles joined, in order of the parts: a work item is (record, KV head, 1024 / D columns), a thread per four dims
// of a column.  The kernel is all latency: kMergeBatch parts are asked for at a time, where there are fewer the last one again.
constexpr int kMergeBatch = 12;
constexpr int kMergeGroups = 2048;  // workgroups
template <int D>
__device__ __forceinline__ void merge_columns(const Attn8Args& a, const Parts& parts, const Record& rec, int kvh, int tcol) {
    const int g = a.n_q / a.n_kv, e = threadIdx.x % (D / 4) * 4, col = rec.tile * rec.width + tcol;
    if (tcol >= rec.width || col >= rec.n * g) return;
    const int64_t first = kvh * parts.places + rec.place + tcol;
    float m = kNegBig, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < rec.parts; p0 += kMergeBatch) {
        f32x2 ml[kMergeBatch];
        f32x4 o[kMergeBatch];
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) {
            const int64_t at = first + (int64_t)min(p0 + u, rec.parts - 1) * rec.step;
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
            l += ml[u][1] * w;
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[v] += o[u][v] * w;
        }
    }
    const float inv = 1.0f / l;
#pragma unroll
    for (int v = 0; v < 4; ++v) acc[v] *= inv;
    *reinterpret_cast<bf16x4*>(a.out + (int64_t)(rec.row0 + col / g) * a.ld_o + (int64_t)(kvh * g + col % g) * D + e) = __builtin_convertvector(acc, bf16x4);
}
template <int D, bool TILES>
__global__ __launch_bounds__(256) void attention8_merge_kernel(Attn8Args a) {
    constexpr int COLS = 1024 / D;
    Parts parts;
    parts_in<TILES>(parts, a.workspace, a.n_kv, D);
    const int groups = (TILES ? kTileCols : kStreamCols) / COLS, per_record = a.n_kv * groups;
    int work = blockIdx.x;
    Record rec = parts.rec[min(work / per_record, max_cut_tiles<TILES>(a.n_kv) - 1)];  // (behind the last one: anything)
    const int total = *parts.count * per_record;
    while (work < total) {
        const int rest = work % per_record;
        work += gridDim.x;
        const Record next = parts.rec[min(work / per_record, max_cut_tiles<TILES>(a.n_kv) - 1)];
        merge_columns<D>(a, parts, rec, rest % a.n_kv, rest / a.n_kv * COLS + (int)threadIdx.x / (D / 4));
        rec = next;
    }
}

}  // namespace

static bool has_tiles(int n_q, int n_kv, int max_new) { return (int64_t)max_new * (n_q / n_kv) > kStreamCols; }

size_t attention8_workspace_bytes(int n_q, int n_kv, int d, int max_new) {
    Parts t;
    return has_tiles(n_q, n_kv, max_new) ? parts_in<true>(t, nullptr, n_kv, d) : parts_in<false>(t, nullptr, n_kv, d);
}

template <int D, bool TILES>
static hipError_t launch(const Attn8Args& a, hipStream_t stream) {
    // no more tiles than whole ones in all rows and a partly filled one per sequence; cutting the keys adds no more units than twice the
    // shares; and one place behind the last unit
    const int64_t units = (int64_t)a.num_rows * (a.n_q / a.n_kv) / (TILES ? kTileCols : kStreamCols) + a.num_seqs + 2 * target_units<TILES>(a.n_kv) + 1;
    if (units * a.n_kv > INT32_MAX) return hipErrorInvalidValue;
    Parts parts;
    parts_in<TILES>(parts, a.workspace, a.n_kv, D);
    if (a.num_seqs > 64) attention8_plan_kernel<TILES><<<1, 1024, 0, stream>>>(a, parts.plan, parts.count);
    int lds = sizeof(StreamLds<D, kThreads<TILES> / 64>);
    if (TILES) {
        lds = sizeof(TileLds<D>) > lds ? sizeof(TileLds<D>) : lds;
        static std::atomic<uint64_t> allowed{0};  // devices on which this kernel may use the LDS that it asks for
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(attention8_kernel<D, TILES>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            if (e != hipSuccess) return e;
            if (dev < 64) allowed.fetch_or(1ull << dev);
        }
    }
    attention8_kernel<D, TILES><<<(unsigned)(units * a.n_kv), kThreads<TILES>, lds, stream>>>(a);
    // no sequence can be cut whose table has no more pages than the fewest blocks of a part
    if (a.table_stride > kBlock / kPage * kMinShare) attention8_merge_kernel<D, TILES><<<kMergeGroups, 256, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_attention8(const Attn8Args& a, hipStream_t stream) {
    if (a.num_seqs <= 0 || a.num_rows <= 0) return hipSuccess;
    if (a.num_seqs > kMaxAttn8Seqs || (int64_t)a.num_rows * (a.n_q / a.n_kv) > INT32_MAX) return hipErrorInvalidValue;
    const bool tiles = has_tiles(a.n_q, a.n_kv, a.max_new);
    if (a.d == 128) return tiles ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
    if (a.d == 64) return tiles ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
    return hipErrorInvalidValue;
}
