// Several continuations of one sequence: entry points of include/gllm_branch.h, and the kernels of all of them but tree attention
// (kernels_tree.hip).
#include "../../include/gllm_branch.h"
#include "common.h"

#include <algorithm>
#include <cmath>
#include <vector>

namespace {

static_assert(GLLM_TREE_MAX_NODES == 256, "a thread per node");

// ---- acceptance and the move of accepted keys and values ---------------------------------------------------------------

struct CommitArgs {
    const int32_t *tokens, *parents, *sampled, *row_start, *cached_len, *block_tables;
    int32_t table_stride, num_seqs, num_rows;
    bf16_t *k_pool, *v_pool;
    int32_t num_layers, num_blocks, n_kv;
    int32_t per_group, groups;  // (layer, head)s of a workgroup, workgroups of a sequence
    int32_t *path, *count, *next_token;
};

// A workgroup has a sequence and per_group of its (layer, KV head)s; each of them walks the tree itself (a few steps of one wave over at most 256 nodes in
// registers), so that one launch does both; the sequence's first one writes the result of the walk.
// The moves of the (layer, head)s, those of one in order of the path, are made kMoves at a time, all read before the first is written: position
// i takes what stands at path[i] >= i, so that no slot is written before it has been read.
//
// Bound by HBM where there is much to move, and by how V lies there: a token's values are 2 bytes of every 32, so that its 256 bytes of a
// head are in all 32 128-byte lines of a (page, head), which a move reads and writes.  64 trees of 60 nodes in 12 layers (8 KV heads of
// 128): 31 MB of keys and values moved, 73 MB read and 33 MB written, 36 us (mean of thirty launches, 34 the fastest); one tree of 26 nodes
// 6.4 us, a launch and the walk.
// (A thread has a 16-byte piece of K, and V elements of neighbouring dims.)
constexpr int kMoves = 16;
// Workgroups that the (layer, head)s are spread over: two rounds of those that run at one time.  (us at 1024 / 2048 / 4096 / one for each, 64 trees
// of 60 nodes: 12 layers, 6144 of them, 45 / 35 / 35 / 38; 20 layers, 10240, 81 / 66 / 64 / 65.)
constexpr int kCommitGroups = 4096;
template <int D>
__global__ __launch_bounds__(256) void tree_commit_kernel(CommitArgs a) {
    __shared__ int32_t drawn[GLLM_TREE_MAX_NODES], path[GLLM_TREE_MAX_NODES];
    __shared__ int accepted, last_drawn;
    const int s = blockIdx.x / a.groups, part0 = blockIdx.x % a.groups * a.per_group, t = threadIdx.x;
    const int r0 = a.row_start[s], r1 = a.row_start[s + 1], c = a.cached_len[s];
    const bool rows_ok = r0 >= 0 && r1 >= r0 && r1 <= a.num_rows;
    const int n = rows_ok ? r1 - r0 : 0;
    const bool fits = n > 0 && n <= GLLM_TREE_MAX_NODES && c >= 0 && (int64_t)c + n <= min((int64_t)a.table_stride * kPage, (int64_t)kMaxPositions);
    if (fits) {
        if (t < n) drawn[t] = a.sampled[r0 + t];
        __syncthreads();
        if (t < 64) {
            int32_t up[4], tok[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = t + 64 * u;
                up[u] = -2;
                tok[u] = 0;
                if (i < n) {
                    up[u] = a.parents[r0 + i];
                    tok[u] = a.tokens[r0 + i];
                    if (up[u] >= i) up[u] = -2;
                }
            }
            int cur = __builtin_amdgcn_readfirstlane(up[0]) == -1 ? 0 : -1, m = 0, last = -1;
            while (cur >= 0) {  // (a child's index is larger than its parent's)
                if (t == 0) path[m] = cur;
                ++m;
                last = drawn[cur];
                int next = -1;
#pragma unroll
                for (int u = 3; u >= 0; --u) {
                    const uint64_t hit = __ballot(up[u] == cur && tok[u] == last);
                    if (hit) next = 64 * u + __builtin_ctzll(hit);
                }
                cur = next;
            }
            if (t == 0) {
                accepted = m;
                last_drawn = last;
            }
        }
        __syncthreads();
    }
    const int m = fits ? accepted : 0;
    if (part0 == 0) {
        for (int i = t; i < n; i += 256) a.path[r0 + i] = i < m ? path[i] : -1;
        if (t == 0) {
            a.count[s] = m;
            a.next_token[s] = m > 0 ? last_drawn : -1;
        }
    }
    if (!a.k_pool || m == 0) return;
    int first = 0;
    while (first < m && path[first] == first) ++first;  // (the same for all threads)
    if (first == m) return;

    const int32_t* bt = a.block_tables + (int64_t)s * a.table_stride;
    const int moves = m - first, todo = min(a.per_group, a.num_layers * a.n_kv - part0) * moves;  // (behind the first, all nodes move)
    auto page_at = [&](int part, int pos) -> int64_t {  // element offset of the (page, head), -1 for an id outside the pool
        const int id = bt[pos / kPage], layer = part / a.n_kv;
        return id >= 0 && id < a.num_blocks ? (((int64_t)layer * a.num_blocks + id) * a.n_kv + part - layer * a.n_kv) * (D * kPage) : -1;
    };
    constexpr int KP = kMoves * (D / 8) / 256, VP = kMoves * D / 256;  // 16-byte pieces of K, elements of V per thread
    static_assert(kMoves * (D / 8) % 128 == 0 && kMoves * D % 256 == 0, "whole passes");
    for (int j0 = 0; j0 < todo; j0 += kMoves) {
        u32x4 kv[KP > 0 ? KP : 1];
        bf16_t vv[VP];
        auto move = [&](int j, int64_t& from, int64_t& to, int& fs, int& ts) {
            from = to = -1;
            if (j >= todo) return;
            const int part = part0 + j / moves, i = first + j % moves;
            const int sp = c + path[i], dp = c + i;
            from = page_at(part, sp);
            to = page_at(part, dp);
            if (from < 0 || to < 0) from = to = -1;
            fs = sp % kPage;
            ts = dp % kPage;
        };
        auto for_k = [&](auto&& f) {
#pragma unroll
            for (int u = 0; u < (KP > 0 ? KP : 1); ++u) {
                const int x = t + u * 256;
                if (x >= kMoves * (D / 8)) continue;
                int64_t from, to;
                int fs = 0, ts = 0;
                move(j0 + x / (D / 8), from, to, fs, ts);
                if (from >= 0) f(u, a.k_pool + from + (x % (D / 8)) * (kPage * 8) + fs * 8, a.k_pool + to + (x % (D / 8)) * (kPage * 8) + ts * 8);
            }
        };
        auto for_v = [&](auto&& f) {
#pragma unroll
            for (int u = 0; u < VP; ++u) {
                const int x = t + u * 256;
                int64_t from, to;
                int fs = 0, ts = 0;
                move(j0 + x / D, from, to, fs, ts);
                if (from >= 0) f(u, a.v_pool + from + (x % D) * kPage + fs, a.v_pool + to + (x % D) * kPage + ts);
            }
        };
        for_k([&](int u, const bf16_t* src, bf16_t*) { kv[u] = *reinterpret_cast<const u32x4*>(src); });
        for_v([&](int u, const bf16_t* src, bf16_t*) { vv[u] = *src; });
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (what has been asked for is here before another wave writes)
        __syncthreads();
        for_k([&](int u, const bf16_t*, bf16_t* dst) { *reinterpret_cast<u32x4*>(dst) = kv[u]; });
        for_v([&](int u, const bf16_t*, bf16_t* dst) { *dst = vv[u]; });
    }
}

// ---- beam selection -----------------------------------------------------------------------------------------------------
//
// Two launches.  beam_rows: a workgroup passes once over a segment of a row of logits and keeps its `keep` largest (no other
// token of the segment can be among the best of the sequence) beside the segment's largest logit and sum of exponentials.
// beam_merge: a workgroup per sequence adds up the sums of its rows and picks the best of what the segments kept.
// The order among beams hangs on the sums: they and the scores are held in 64 bits, so that the order is that of exact
// arithmetic but where scores of two beams agree to some 1e-10; in a beam it is that of the logits.
//
// Measured (64 sequences of 8 beams over a vocabulary of 152064, keep 16: 311 MB): 91 + 8.1 us, means of thirty launches (88 + 7.6 the fastest), of
// which HBM would take 50.  What bounds beam_rows are vector instructions and their latency, 27 a logit, 12 of them in 64 bits (the exponential),
// with one pass on its way while the last one is worked on: at 128 rows it takes 30 us, without exponentials and without lists behind the first
// pass 16.  Reading past the caches takes 94 us where a plain load takes 96.  Rows that do not start on a 16-byte boundary: 18.3 us where aligned ones
// take 16.6 (80 rows of 50261).  beam_merge is latency: four dependent steps (sums, logarithms, the bound, the lists above it, all in one queue so
// that up to 8 loads are on their way: both launches of 32 beams that keep 64 53 -> 47 us).

constexpr int kBeamWaves = 4;
constexpr int kBeamTokenBits = 24, kBeamMaxVocab = 1 << kBeamTokenBits;
constexpr int kBeamLists = 1280;  // most segments of the rows of a sequence
constexpr int kBeamList = 384;  // places of a wave's list: the 64 kept at most, the 256 of one pass, and a whole number per lane

// Keys in the order of the numbers, 0 for what is no candidate (minus infinity, not a number).
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);  // (one zero)
    return x > -INFINITY ? b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u) : 0u;
}
// The least number whose key is above `key`, which is a number's, one less, or 0; infinity for infinity's own (candidates of the same key
// are sorted out by their index).
__device__ __forceinline__ float above_key(uint32_t key) {
    constexpr uint32_t kInfinity = 0xFF800000u;
    const uint32_t k = min(key + 1, kInfinity);
    return key == 0u ? -3.402823466e38f : __builtin_bit_cast(float, k >> 31 ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t order_key(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);
    return x > -INFINITY ? b ^ (b >> 63 ? ~0ull : 1ull << 63) : 0ull;
}

// Bit by bit the largest v with at least `need` of the wave's keys >= v, U per lane, of which those that are `in` count; it stops
// early at a v that exactly `need` keys reach, most often after the bits in which the need-th key differs from the next one.  count: the keys
// that reach v.  There have to be `need` of them.
template <int U>
__device__ __forceinline__ uint32_t reach_of(const uint32_t (&key)[U], const bool (&in)[U], int need, int& count) {
    uint32_t v = 0;
    count = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) count += __popcll(__ballot(in[u]));
#pragma unroll 1
    for (int bit = 31; bit >= 0 && count != need; --bit) {
        const uint32_t probe = v | 1u << bit;
        int above = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) above += __popcll(__ballot(in[u] && key[u] >= probe));
        if (above >= need) {
            v = probe;
            count = above;
        }
    }
    return v;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ void max_step(float& x) {
    const int b = __builtin_bit_cast(int, x);
    x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, ROWS, 0xf, false)));
}
// The largest x of the wave, in all lanes: by lane shifts (lane 63 has it).
__device__ __forceinline__ float wave_max(float x) {
    max_step<0x111, 0xf>(x);
    max_step<0x112, 0xf>(x);
    max_step<0x114, 0xf>(x);
    max_step<0x118, 0xf>(x);
    max_step<0x142, 0xa>(x);
    max_step<0x143, 0xc>(x);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// 2^f for |f| <= 1/2 in 64 bits, off by at most 4.7e-11 of itself: the polynomial of degree 7 that is 1 at 0 and whose largest relative error is
// least.  (1 at 0: what has the weight 1 keeps it whatever the reference, so that rows of the same sum have the same logarithm.)
__device__ __forceinline__ double exp2_unit(double f) {
    double p = 1.5196149292421300e-05;
    p = fma(p, f, 1.5466756939974918e-04);
    p = fma(p, f, 1.3333935089590121e-03);
    p = fma(p, f, 9.6180381297376900e-03);
    p = fma(p, f, 5.5504103659446753e-02);
    p = fma(p, f, 2.4022651066581255e-01);
    p = fma(p, f, 6.9314718070454884e-01);
    return fma(p, f, 1.0);
}
// 2^y for any y <= 1000.
__device__ __forceinline__ double exp2_wide(double y) {
    y = fmax(y, -1400.0);
    const double n = rint(y);
    return ldexp(exp2_unit(y - n), (int)n);
}
constexpr double kLog2E = 1.4426950408889634;
// 2^(x log2(e) - r) for a whole number r, given kRound - r, where the exponent lies within +-1020: without the instructions on 64 bits that
// take longer than a multiplication.  The sum with 1.5 * 2^52 rounds x log2(e) to a whole number, which stands, less r, in the low bits,
// and is added to the exponent of the result.
constexpr double kRound = 6755399441055744.0;
__device__ __forceinline__ double exp_near(float x, double round_less_r) {
    const double t = fma((double)x, kLog2E, round_less_r);
    u32x2 p = __builtin_bit_cast(u32x2, exp2_unit(fma((double)x, kLog2E, round_less_r - t)));
    p[1] += __builtin_bit_cast(u32x2, t)[0] << 20;
    return __builtin_bit_cast(double, p);
}

__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The candidates of one wave, in LDS: by the key, the highest first, equal keys by the index, the lowest first.
template <typename Key, typename Idx>
struct WaveList {
    Key* key;
    Idx* idx;
    int n;      // the same in all lanes
    int lane;
    // Adds the lanes' candidates that `pass`; there has to be room for 64.
    __device__ __forceinline__ void add(bool pass, Key k, Idx i) {
        const uint64_t who = __ballot(pass);
        if (pass) {
            const int at = n + __popcll(who & ((1ull << lane) - 1));
            key[at] = k;
            idx[at] = i;
        }
        n += __popcll(who);
    }
    // Leaves the k best.  Returns a key that all of them reach, or 0 where there were no more than k.
    __device__ __forceinline__ Key keep_best(int k) {
        if (n <= k) return 0;
        return n <= 128 ? best_of<2>(k) : n <= 256 ? best_of<4>(k) : best_of<kBeamList / 64>(k);
    }
    template <int U>
    __device__ __forceinline__ Key best_of(int k) {
        wave_fence();
        Key mine[U];
        Idx at[U];
        uint32_t part[U];
        bool tied[U], kept[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = lane + 64 * u;
            tied[u] = i < n;
            kept[u] = false;
            mine[u] = tied[u] ? key[i] : 0;
            at[u] = tied[u] ? idx[i] : 0;
        }
        // by the key's words, upper one first, then by the index: those above the need-th value of a word are kept, those that
        // agree in it go on
        Key low = 0;
        int need = k;
#pragma unroll
        for (int word = 0; word < (int)(sizeof(Key) + sizeof(Idx)) / 4; ++word) {
            if (need == 0) continue;
            const int down = (int)sizeof(Key) * 8 - 32 * (word + 1);  // of the key, below zero behind its last word
#pragma unroll
            for (int u = 0; u < U; ++u) part[u] = down >= 0 ? (uint32_t)(mine[u] >> (down & 63)) : ~(uint32_t)(at[u] >> (down + (int)sizeof(Idx) * 8 & 63));
            int count;
            const uint32_t v = reach_of(part, tied, need, count);
            if (down >= 0) low |= (Key)v << (down & 63);
            if (count == need) {
#pragma unroll
                for (int u = 0; u < U; ++u) kept[u] |= tied[u] && part[u] >= v;
                need = 0;
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    kept[u] |= tied[u] && part[u] > v;
                    need -= __popcll(__ballot(tied[u] && part[u] > v));
                    tied[u] = tied[u] && part[u] == v;
                }
            }
        }
        wave_fence();
        n = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) add(kept[u], mine[u], at[u]);
        wave_fence();
        return low;
    }
};

struct BeamArgs {
    const float* logits;
    int64_t ld;
    const float* scores;
    int32_t num_seqs, beams, vocab, keep, segs, seg_len;
    // workspace: per (row, segment) the sum, the largest logit, and `keep` values with their tokens (-1: none)
    double* sum;
    float* top;
    float* value;
    int32_t* token;
    float* out_scores;
    int32_t *out_beams, *out_tokens;
};

constexpr int kBeamQuads = 4;                        // four-column loads of a lane and pass
constexpr int kBeamPass = 256 * kBeamQuads;          // columns of a wave's pass
constexpr float kBeamSlack = 60.f;

// Columns `at` .. of a wave's pass; minus infinity behind the end.
template <bool VEC>
__device__ __forceinline__ void load_pass(f32x4 (&x)[kBeamQuads], const float* __restrict__ x0, int at, int end, int lane) {
#pragma unroll
    for (int j = 0; j < kBeamQuads; ++j) {
        const int col = at + (j * 64 + lane) * 4;
        x[j] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (VEC) {
            if (col < end) x[j] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(x0 + col));  // (read once)
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < end) x[j][e] = x0[col + e];
        }
    }
}
// (a bare maximum: fmaxf first makes every loaded value quiet.  Not a number: low.)
__device__ __forceinline__ float at_least(float x, float low) { return __builtin_amdgcn_fmed3f(x, low, INFINITY); }

template <bool VEC>
__global__ __launch_bounds__(256, 4) void beam_rows_kernel(BeamArgs a) {
    __shared__ uint32_t keys[kBeamWaves][kBeamList], idxs[kBeamWaves][kBeamList];
    __shared__ double wave_sum[kBeamWaves];
    __shared__ float wave_top[kBeamWaves];
    __shared__ int wave_n[kBeamWaves];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = blockIdx.x / a.segs, seg = blockIdx.x % a.segs;
    const float* x0 = a.logits + (int64_t)row * a.ld;
    const int begin = seg * a.seg_len, end = min(a.vocab, begin + a.seg_len);
    WaveList<uint32_t, uint32_t> list{keys[wave], idxs[wave], 0, lane};
    float bar = above_key(0);  // candidates are not below it
    // The sum of exp(x - ref); where ref is below 1000 in magnitude, of 2^(x log2(e) - r), r = ref log2(e) rounded to a whole number (one
    // subtraction in 64 bits less per logit, of sixteen operations).
    float ref = -INFINITY;
    double sum = 0.0, r = 0.0;  // (sum: of this lane)
    float most = -INFINITY;     // this lane's largest
    auto near = [&](float x) { return fabsf(x) < 1000.f; };
    auto refer_to = [&](float x) {  // (the same for the wave)
        const double was = near(ref) ? r : (double)ref * kLog2E;
        r = rint((double)x * kLog2E);
        sum = ref == -INFINITY || x == INFINITY ? 0.0 : sum * exp2_wide(was - (near(x) ? r : (double)x * kLog2E));
        ref = x;
    };
    auto raise = [&]() {
        const uint32_t floor = list.keep_best(a.keep);
        if (floor > 0) bar = fmaxf(bar, above_key(floor));
    };
    f32x4 x[kBeamQuads], next[kBeamQuads];
    const int first = begin + wave * kBeamPass, step = kBeamWaves * kBeamPass;
    if (first < end) load_pass<VEC>(x, x0, first, end, lane);
    // Every wave passes over columns in ascending order, so that behind keep_best an equal key comes with a larger index and loses.
#pragma unroll 1
    for (int at = first; at < end; at += step) {
        if (at + step < end) load_pass<VEC>(next, x0, at + step, end, lane);
        if (VEC && at + kBeamPass > end) {  // (the same for the wave)
#pragma unroll
            for (int j = 0; j < kBeamQuads; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at + (j * 64 + lane) * 4 + e >= end) x[j][e] = -INFINITY;
        }
        if (at == first) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < kBeamQuads; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, x[j][e]);
            const float now = wave_max(top);
            if (now > -INFINITY) refer_to(now);
            // at least `keep` candidates are not below the keep-th largest of the lanes' maxima
            const uint32_t lane_top[1] = {order_key(top)};
            const bool in[1] = {lane_top[0] > 0};
            int count;
            if (__popcll(__ballot(in[0])) >= a.keep) bar = above_key(max(reach_of(lane_top, in, a.keep, count), 1u) - 1);
        }
        // what is lower weighs 1e-304; a quad's maximum is exact where it is higher
        const float low = near(ref) ? ref - 700.f : -INFINITY;
        float quad[kBeamQuads], top = low;
#pragma unroll
        for (int j = 0; j < kBeamQuads; ++j) {
            quad[j] = low;
#pragma unroll
            for (int e = 0; e < 4; ++e) quad[j] = fmaxf(quad[j], at_least(x[j][e], low));
            top = fmaxf(top, quad[j]);
        }
        most = fmaxf(most, top);
        if (__any(top > ref + kBeamSlack || (top > ref && ref == -INFINITY))) refer_to(wave_max(top));
        if (near(ref)) {
            const double c = kRound - r;
#pragma unroll
            for (int j = 0; j < kBeamQuads; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += exp_near(at_least(x[j][e], ref - 700.f), c);
        } else if (ref > -INFINITY) {
#pragma unroll
            for (int j = 0; j < kBeamQuads; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)  // (not x * log2(e) - ref * log2(e): logits may be the type's lowest value)
                    sum += x[j][e] == ref ? 1.0 : ref < INFINITY ? exp2_wide(((double)x[j][e] - (double)ref) * kLog2E) : 0.0;
        }
        if (__any(top >= bar)) {
#pragma unroll
            for (int j = 0; j < kBeamQuads; ++j) {
                if (!__any(quad[j] >= bar)) continue;
                if (list.n + 256 > kBeamList) raise();
#pragma unroll
                for (int e = 0; e < 4; ++e) list.add(x[j][e] >= bar, order_key(x[j][e]), (uint32_t)(at + (j * 64 + lane) * 4 + e));
            }
            if (list.n >= 2 * a.keep) raise();  // (the sooner the bar is high the fewer candidates come: in pass p about keep / p)
        }
#pragma unroll
        for (int j = 0; j < kBeamQuads; ++j) x[j] = next[j];
    }
    // what goes out is the sum by the largest logit: the merge takes it for that of the best candidate too
    const float largest = wave_max(most);
    if (near(ref)) sum *= exp2_wide(r - (double)largest * kLog2E);
    else if (largest > ref) sum *= exp2_wide(((double)ref - (double)largest) * kLog2E);
    if (list.n > 64) list.keep_best(a.keep);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) {
        wave_sum[wave] = sum;
        wave_top[wave] = largest;
        wave_n[wave] = list.n;
    }
    __syncthreads();
    if (wave > 0) return;
    // the first wave's list takes in the others', of at most 64 each (keys and indices decide, not the places)
    for (int w = 1; w < kBeamWaves; ++w) {
        const int n = wave_n[w];
        list.add(lane < n, lane < n ? keys[w][lane] : 0u, lane < n ? idxs[w][lane] : 0u);
    }
    list.keep_best(a.keep);
    wave_fence();
    const int64_t place = (int64_t)blockIdx.x;
    if (lane < a.keep) {
        const bool there = lane < list.n;
        const uint32_t i = there ? list.idx[lane] : 0u;
        a.token[place * a.keep + lane] = there ? (int32_t)i : -1;
        a.value[place * a.keep + lane] = there ? x0[i] : 0.f;
    }
    if (lane == 0) {
        float m = -INFINITY;
        for (int w = 0; w < kBeamWaves; ++w) m = fmaxf(m, wave_top[w]);
        double total = 0.0;
        for (int w = 0; w < kBeamWaves; ++w)
            if (wave_top[w] > -INFINITY) total += wave_top[w] == m ? wave_sum[w] : wave_sum[w] * exp2_wide(((double)wave_top[w] - (double)m) * kLog2E);
        a.top[place] = m;
        a.sum[place] = total;
    }
}

__global__ __launch_bounds__(256) void beam_merge_kernel(BeamArgs a) {
    __shared__ uint64_t keys[kBeamWaves][kBeamList], idxs[kBeamWaves][kBeamList];
    __shared__ double lse[GLLM_BEAM_MAX_BEAMS];   // log of the sum without the largest logit
    __shared__ float tops[GLLM_BEAM_MAX_BEAMS], so_far[GLLM_BEAM_MAX_BEAMS];
    __shared__ float list_top[kBeamLists];
    __shared__ double list_sum[kBeamLists];
    __shared__ uint16_t queue[kBeamWaves][kBeamLists / kBeamWaves];  // a wave's lists that are looked into
    __shared__ int wave_n[kBeamWaves];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int s = blockIdx.x;
    const int64_t row0 = (int64_t)s * a.beams;
    const int lists = a.beams * a.segs;
    if ((int)threadIdx.x < a.beams) so_far[threadIdx.x] = a.scores[row0 + threadIdx.x];
    for (int i = threadIdx.x; i < lists; i += 256) {
        list_top[i] = a.top[row0 * a.segs + i];
        list_sum[i] = a.sum[row0 * a.segs + i];
    }
    // Few candidates are all asked for at once, without a look at the lists' first ones.  (us of both launches, all at once / by the lists: 64 places
    // 13.2 / 17.3, 256 14.2 / 17.5, 600 24.7 / 28.1, 1024 17.9 / 19.2 and 17.0 / 18.7.  With 6 instead of 4, 1216 and 1536 places take 18.5 and 18.8
    // instead of 19.3, and all smaller ones 0.2 to 0.4 more.)
    constexpr int FEW = 4;
    static_assert(FEW * 64 <= kBeamList, "a wave's candidates have room");
    const bool few = lists * a.keep <= FEW * 256;
    int32_t few_token[FEW];
    float few_value[FEW];
#pragma unroll
    for (int t = 0; t < FEW; ++t) {
        const int i = (t * kBeamWaves + wave) * 64 + lane;
        few_token[t] = -1;
        few_value[t] = 0.f;
        if (few && i < lists * a.keep) {
            few_token[t] = a.token[row0 * a.segs * a.keep + i];
            few_value[t] = a.value[row0 * a.segs * a.keep + i];
        }
    }
    __syncthreads();
    // sixteen lanes to a beam
    for (int b0 = 0; b0 < a.beams; b0 += 4 * kBeamWaves) {
        const int b = b0 + wave * 4 + lane / 16, at = min(b, a.beams - 1) * a.segs;
        float m = -INFINITY;
        for (int i = lane % 16; i < a.segs; i += 16) m = fmaxf(m, list_top[at + i]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
        double total = 0.0;
        for (int i = lane % 16; i < a.segs; i += 16) {
            const float t = list_top[at + i];
            if (t > -INFINITY) total += t == m ? list_sum[at + i] : list_sum[at + i] * exp2_wide(((double)t - (double)m) * kLog2E);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) total += __shfl_xor(total, o);
        if (lane % 16 == 0 && b < a.beams) {
            tops[b] = m;
            // the logarithm in 32 bits and a step of Newton's method, whose error is half the square of the first one's
            const double y = (double)__logf((float)total);
            lse[b] = total > 0.0 ? y + (total * exp2_wide(-y * kLog2E) - 1.0) : 0.0;
        }
    }
    __syncthreads();
    auto score = [&](float x, int b) {  // of a logit of beam b; 0: no candidate
        const float cum = so_far[b], m = tops[b];
        if (!(cum > -INFINITY && cum < INFINITY) || x == -INFINITY) return (uint64_t)0;  // (x: the largest logit of a list that is empty)
        return order_key((double)cum + ((x == m ? 0.0 : (double)x - (double)m) - lse[b]));
    };
    // What orders equal scores: the beam, then the logit, whose differences the score may have swallowed, then the token.  The segments kept the
    // best of their row by the last two, so that nothing they left out comes in front of what they kept.
    constexpr int kBeamAt = kBeamTokenBits + 32;
    static_assert(GLLM_BEAM_MAX_BEAMS <= 1 << (64 - kBeamAt), "a beam has room");
    auto place_of = [](int b, float x, int token) { return (uint64_t)b << kBeamAt | (uint64_t)~order_key(x) << kBeamTokenBits | (uint32_t)token; };
    WaveList<uint64_t, uint64_t> list{keys[wave], idxs[wave], 0, lane};
    if (few) {
#pragma unroll
        for (int t = 0; t < FEW; ++t) {
            const int b = ((t * kBeamWaves + wave) * 64 + lane) / (a.segs * a.keep);
            const uint64_t k = few_token[t] >= 0 ? score(few_value[t], b) : 0;
            list.add(k > 0, k, place_of(b, few_value[t], few_token[t]));
        }
    } else {
        // What the segments kept is a list each.  At least `keep` candidates are not below the keep-th best of the lists' largest ones: of a
        // wave's lists first, then of those that all waves have found, and few lists are left to be looked into.
        constexpr int U = kBeamLists / 256;
        uint64_t best[U];
        uint32_t high[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = (u * 64 + lane) * kBeamWaves + wave;
            best[u] = 0;
            if (i < lists) best[u] = score(list_top[i], i / a.segs);
            high[u] = (uint32_t)(best[u] >> 32);
        }
        bool in[U];
        int found = 0, count;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            in[u] = best[u] > 0;
            found += __popcll(__ballot(in[u]));
        }
        const uint32_t own = found >= a.keep ? reach_of(high, in, a.keep, count) : 0u;
        uint32_t* const heads = reinterpret_cast<uint32_t*>(&idxs[0][0]);  // [kBeamWaves][64]: of each wave's lists the first keep that reach its bound
        {
            heads[wave * 64 + lane] = 0;
            wave_fence();
            int at = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool take = in[u] && high[u] >= own;
                const uint64_t who = __ballot(take);
                const int to = at + __popcll(who & ((1ull << lane) - 1));
                if (take && to < 64) heads[wave * 64 + to] = high[u];
                at += __popcll(who);
            }
        }
        __syncthreads();
        uint64_t floor = 1;
        {
            uint32_t every[kBeamWaves];
            bool of[kBeamWaves];
            int there = 0;
#pragma unroll
            for (int w = 0; w < kBeamWaves; ++w) {
                every[w] = heads[w * 64 + lane];
                of[w] = every[w] > 0;
                there += __popcll(__ballot(of[w]));
            }
            if (there >= a.keep) floor = max(floor, (uint64_t)reach_of(every, of, a.keep, count) << 32);
        }
        __syncthreads();  // (the heads have been read)
        int room = 1;  // lanes to a list
        while (room < a.keep) room *= 2;
        const int at_once = 64 / room, mine = lane / room, e = lane % room;
        int queued = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool take = best[u] >= floor;
            const uint64_t who = __ballot(take);
            if (take) queue[wave][queued + __popcll(who & ((1ull << lane) - 1))] = (uint16_t)((u * 64 + lane) * kBeamWaves + wave);
            queued += __popcll(who);
        }
        wave_fence();
        constexpr int STEPS = 8;  // on their way at one time
        for (int q0 = 0; q0 < queued; q0 += STEPS * at_once) {
            int32_t token[STEPS];
            float value[STEPS];
            int beam[STEPS];
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                const int q = q0 + t * at_once + mine;
                token[t] = -1;
                value[t] = 0.f;
                beam[t] = 0;
                if (q < queued && e < a.keep) {
                    const int i = queue[wave][q];
                    const int64_t place = (row0 * a.segs + i) * a.keep + e;
                    beam[t] = i / a.segs;
                    token[t] = a.token[place];
                    value[t] = a.value[place];
                }
            }
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                if (q0 + t * at_once >= queued) continue;
                const uint64_t k = token[t] >= 0 ? score(value[t], beam[t]) : 0;
                if (list.n + 64 > kBeamList) floor = max(floor, list.keep_best(a.keep));
                list.add(k >= floor, k, place_of(beam[t], value[t], token[t]));
            }
        }
    }
    if (list.n > 64) list.keep_best(a.keep);
    if (lane == 0) wave_n[wave] = list.n;
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < kBeamWaves; ++w) {
        const int n = wave_n[w];
        list.add(lane < n, lane < n ? keys[w][lane] : 0ull, lane < n ? idxs[w][lane] : 0ull);
    }
    list.keep_best(a.keep);
    wave_fence();
    // the place of each of the at most 64 is the number of those in front of it (the index is looked at where keys are equal only)
    const bool there = lane < list.n;
    const uint64_t k = there ? list.key[lane] : 0ull;
    const uint64_t i = there ? list.idx[lane] : 0ull;
    auto of_lane = [](uint64_t x, int l) { return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, l); };
    int rank = 0;
    bool ties = false;
    for (int j = 0; j < list.n; ++j) {
        const uint64_t kj = of_lane(k, j);
        rank += kj > k;
        ties |= kj == k && j != lane;
    }
    if (__any(there && ties))
        for (int j = 0; j < list.n; ++j) rank += of_lane(k, j) == k && of_lane(i, j) < i;
    const int64_t out = (int64_t)s * a.keep;
    if (there) {
        const uint64_t bits = k >> 63 ? k ^ (1ull << 63) : ~k;
        a.out_scores[out + rank] = (float)__builtin_bit_cast(double, bits);
        a.out_beams[out + rank] = (int32_t)(i >> kBeamAt);
        a.out_tokens[out + rank] = (int32_t)i & (kBeamMaxVocab - 1);
    } else if (lane < a.keep) {
        a.out_scores[out + lane] = -INFINITY;
        a.out_beams[out + lane] = -1;
        a.out_tokens[out + lane] = -1;
    }
}

// Segments of a row: no more workgroups than run at one time (four per compute unit), unless there are more rows, each with at least one
// pass of its four waves.  (us at 512 / 1024 / 1536 / 2048: 64 sequences of 8 beams, vocabulary 152064, 99 / 94 / 102 / 103; 16 of 8 beams,
// 128256, 42 / 41 / 49 / 48; 8 of 32 beams that keep 64 95 / 89 / 98 / 103: segments that start late end late, and each finds its bar anew.)
constexpr int kBeamTarget = 1024;
int beam_segments(int num_seqs, int beams, int vocab) {
    const int64_t rows = std::max<int64_t>(1, (int64_t)num_seqs * beams), most = ceil_div(vocab, kBeamWaves * kBeamPass);
    return (int)std::min({most, std::max<int64_t>(1, kBeamTarget / rows), (int64_t)kBeamLists / beams});
}

bool beam_sizes_ok(int num_seqs, int beams, int vocab, int keep) {
    return num_seqs >= 0 && beams >= 1 && beams <= GLLM_BEAM_MAX_BEAMS && vocab >= 1 && vocab <= kBeamMaxVocab && keep >= 1 && keep <= GLLM_BEAM_MAX_KEEP &&
           (int64_t)num_seqs * beams <= 1 << 22;
}

// ---- page copies --------------------------------------------------------------------------------------------------------

constexpr int kCopyPairs = 448;  // pages of a launch: the list travels with the launch, whose arguments may take 4 KiB
struct CopyArgs {
    u32x4 *k, *v;
    int64_t layer_vecs;   // 16-byte pieces of a layer of either pool
    int32_t page_vecs;    // and of a page
    int32_t src[kCopyPairs], dst[kCopyPairs];
};
static_assert(sizeof(CopyArgs) <= 4096 - 256, "launch arguments");

// grid (pairs, layers, 2): a workgroup copies the page's part of a layer in one pool, 4 KiB of it per step (16 bytes a thread).  Bound by
// HBM: 160 pages in 20 layers (8 KV heads of 128, 210 MB read and as many written) 72 us, 5.8 TB/s; 3 pages 3.8 us (means of thirty launches).
__global__ __launch_bounds__(256) void copy_pages_kernel(CopyArgs a) {
    u32x4* pool = (blockIdx.z ? a.v : a.k) + blockIdx.y * a.layer_vecs;
    const u32x4* src = pool + (int64_t)a.src[blockIdx.x] * a.page_vecs;
    u32x4* dst = pool + (int64_t)a.dst[blockIdx.x] * a.page_vecs;
    for (int i = threadIdx.x; i < a.page_vecs; i += 256) dst[i] = src[i];
}

gllm_status launched() { return hipGetLastError() == hipSuccess ? GLLM_OK : GLLM_E_HIP; }

bool misaligned(const void* p, int to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) != 0; }

float base2(float scale) { return (float)(scale * 1.4426950408889634); }  // of scores whose exponentials are taken in base 2

bool tree_shape_ok(int n_q, int n_kv, int d, int max_nodes) {
    return n_q >= 1 && n_kv >= 1 && n_q % n_kv == 0 && n_q / n_kv <= 16 && (d == 64 || d == 128) && max_nodes >= 1 && max_nodes <= GLLM_TREE_MAX_NODES;
}

}  // namespace

extern "C" {

size_t gllm_op_tree_attention_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_nodes) {
    return tree_shape_ok(n_q_heads, n_kv_heads, head_dim, max_nodes) ? tree_workspace_bytes(n_q_heads, n_kv_heads, head_dim, max_nodes) : 0;
}

gllm_status gllm_op_tree_attention(const void* q, int64_t ld_q, const void* k_pool, const void* v_pool, int64_t num_blocks,
                                   const int32_t* block_tables, int32_t block_table_stride, const int32_t* cached_len,
                                   const int32_t* row_start, const int32_t* parents, int32_t num_seqs, int32_t num_rows,
                                   int32_t max_nodes, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                                   void* out, int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (num_seqs < 0 || num_rows < 0 || max_nodes < 1 || num_blocks < 1 || num_blocks > INT32_MAX || block_table_stride < 1 || n_q_heads < 1 || n_kv_heads < 1 ||
        !(scale > 0.f) || !std::isfinite(base2(scale)))
        return GLLM_E_INVALID;
    if (!tree_shape_ok(n_q_heads, n_kv_heads, head_dim, max_nodes)) return GLLM_E_UNSUPPORTED;
    if (num_seqs == 0 || num_rows == 0) return GLLM_OK;
    if (!q || !k_pool || !v_pool || !block_tables || !cached_len || !row_start || !parents || !out || !workspace) return GLLM_E_INVALID;
    if (ld_q < (int64_t)n_q_heads * head_dim || ld_out < (int64_t)n_q_heads * head_dim) return GLLM_E_INVALID;
    if (ld_q % 8 != 0 || ld_out % 4 != 0 || misaligned(q, 16) || misaligned(k_pool, 16) || misaligned(v_pool, 16) || misaligned(out, 8) || misaligned(workspace, 16))
        return GLLM_E_INVALID;
    if (workspace_bytes < tree_workspace_bytes(n_q_heads, n_kv_heads, head_dim, max_nodes)) return GLLM_E_CAPACITY;
    TreeArgs a{};
    a.q = (const bf16_t*)q; a.ld_q = ld_q;
    a.k_pool = (const bf16_t*)k_pool; a.v_pool = (const bf16_t*)v_pool; a.num_blocks = (int32_t)num_blocks;
    a.block_tables = block_tables; a.table_stride = block_table_stride; a.bt_off = nullptr;
    a.cached_len = cached_len; a.row_begin = row_start; a.row_end = row_start + 1; a.parents = parents;
    a.num_seqs = num_seqs; a.num_rows = num_rows; a.max_nodes = max_nodes;
    a.out = (bf16_t*)out; a.ld_o = ld_out;
    a.n_q = n_q_heads; a.n_kv = n_kv_heads; a.d = head_dim;
    a.scale_log2 = base2(scale);
    a.workspace = workspace;
    const hipError_t e = launch_tree_attention(a, (hipStream_t)stream);
    return e == hipSuccess ? GLLM_OK : e == hipErrorInvalidValue ? GLLM_E_CAPACITY : GLLM_E_HIP;
}

gllm_status gllm_op_tree_commit(const int32_t* tokens, const int32_t* parents, const int32_t* sampled, const int32_t* row_start,
                                const int32_t* cached_len, const int32_t* block_tables, int32_t block_table_stride,
                                int32_t num_seqs, int32_t num_rows, void* k_pool, void* v_pool, int32_t num_layers,
                                int64_t num_blocks, int32_t n_kv_heads, int32_t head_dim, int32_t* path, int32_t* count,
                                int32_t* next_token, void* stream) {
    if (num_seqs < 0 || num_rows < 0 || block_table_stride < 1 || !k_pool != !v_pool) return GLLM_E_INVALID;
    if (k_pool) {
        if (num_layers < 1 || num_blocks < 1 || num_blocks > INT32_MAX || n_kv_heads < 1 || misaligned(k_pool, 16) || misaligned(v_pool, 16)) return GLLM_E_INVALID;
        if (head_dim != 64 && head_dim != 128) return GLLM_E_UNSUPPORTED;
        if ((int64_t)num_layers * n_kv_heads > INT32_MAX / std::max(1, num_seqs)) return GLLM_E_CAPACITY;
    }
    if (num_seqs == 0) return GLLM_OK;
    if (!row_start || !cached_len || !block_tables || !count || !next_token) return GLLM_E_INVALID;
    if (num_rows > 0 && (!tokens || !parents || !sampled || !path)) return GLLM_E_INVALID;
    const int64_t parts = k_pool ? (int64_t)num_layers * n_kv_heads : 1;
    const int32_t per_group = (int32_t)std::max<int64_t>(1, ceil_div(parts * num_seqs, kCommitGroups));
    const CommitArgs a{tokens, parents, sampled, row_start, cached_len, block_tables, block_table_stride, num_seqs, num_rows,
                       (bf16_t*)k_pool, (bf16_t*)v_pool, k_pool ? num_layers : 0, (int32_t)(k_pool ? num_blocks : 0), k_pool ? n_kv_heads : 0,
                       per_group, (int32_t)ceil_div(parts, per_group),
                       path, count, next_token};
    const dim3 grid((unsigned)num_seqs * (unsigned)a.groups);
    if (k_pool && head_dim == 64) tree_commit_kernel<64><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    else tree_commit_kernel<128><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    return launched();
}

size_t gllm_op_beam_select_workspace_bytes(int32_t num_seqs, int32_t beams, int32_t vocab, int32_t keep) {
    if (!beam_sizes_ok(num_seqs, beams, vocab, keep)) return 0;
    const size_t places = (size_t)std::max(1, num_seqs) * beams * beam_segments(num_seqs, beams, vocab);
    return places * (8 + 4 + (size_t)keep * 8);
}

gllm_status gllm_op_beam_select(const float* logits, int64_t ld_logits, const float* scores, int32_t num_seqs, int32_t beams,
                                int32_t vocab, int32_t keep, float* out_scores, int32_t* out_beams, int32_t* out_tokens,
                                void* workspace, size_t workspace_bytes, void* stream) {
    if (num_seqs < 0 || beams < 1 || vocab < 1 || keep < 1 || ld_logits < vocab) return GLLM_E_INVALID;
    if (!beam_sizes_ok(num_seqs, beams, vocab, keep)) return GLLM_E_UNSUPPORTED;
    if (num_seqs == 0) return GLLM_OK;
    if (!logits || !scores || !out_scores || !out_beams || !out_tokens || !workspace || misaligned(logits, 4) || misaligned(workspace, 16)) return GLLM_E_INVALID;
    if (workspace_bytes < gllm_op_beam_select_workspace_bytes(num_seqs, beams, vocab, keep)) return GLLM_E_CAPACITY;
    BeamArgs a{};
    a.logits = logits; a.ld = ld_logits; a.scores = scores;
    a.num_seqs = num_seqs; a.beams = beams; a.vocab = vocab; a.keep = keep;
    a.segs = beam_segments(num_seqs, beams, vocab);
    a.seg_len = (int32_t)round_up(ceil_div(vocab, a.segs), kBeamPass);  // (the last ones may be short of it, or empty)
    const int64_t places = (int64_t)num_seqs * beams * a.segs;
    a.sum = (double*)workspace;
    a.top = (float*)(a.sum + places);
    a.value = a.top + places;
    a.token = (int32_t*)(a.value + places * keep);
    a.out_scores = out_scores; a.out_beams = out_beams; a.out_tokens = out_tokens;
    // four logits at a time from rows that all start on a 16-byte boundary (a quad does not pass a row's end then)
    if (!misaligned(logits, 16) && ld_logits % 4 == 0) beam_rows_kernel<true><<<(unsigned)places, 256, 0, (hipStream_t)stream>>>(a);
    else beam_rows_kernel<false><<<(unsigned)places, 256, 0, (hipStream_t)stream>>>(a);
    if (hipGetLastError() != hipSuccess) return GLLM_E_HIP;
    beam_merge_kernel<<<num_seqs, 256, 0, (hipStream_t)stream>>>(a);
    return launched();
}

gllm_status gllm_op_copy_pages(void* k_pool, void* v_pool, int32_t num_layers, int64_t num_blocks, int32_t n_kv_heads,
                               int32_t head_dim, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
    if (n < 0 || num_layers < 1 || num_layers > 65535 || num_blocks < 1 || num_blocks > INT32_MAX || n_kv_heads < 1) return GLLM_E_INVALID;
    if (head_dim != 64 && head_dim != 128) return GLLM_E_UNSUPPORTED;
    if ((int64_t)n_kv_heads * head_dim * 2 > INT32_MAX) return GLLM_E_UNSUPPORTED;
    if (n == 0) return GLLM_OK;
    if (!k_pool || !v_pool || !src || !dst || misaligned(k_pool, 16) || misaligned(v_pool, 16)) return GLLM_E_INVALID;
    for (int32_t i = 0; i < n; ++i)
        if (src[i] < 0 || src[i] >= num_blocks || dst[i] < 0 || dst[i] >= num_blocks) return GLLM_E_BLOCK_RANGE;
    try {
        std::vector<int32_t> to(dst, dst + n);
        std::sort(to.begin(), to.end());
        if (std::adjacent_find(to.begin(), to.end()) != to.end()) return GLLM_E_BLOCK_ALIAS;
        for (int32_t i = 0; i < n; ++i)
            if (std::binary_search(to.begin(), to.end(), src[i])) return GLLM_E_BLOCK_ALIAS;
    } catch (const std::exception&) {
        return GLLM_E_CAPACITY;
    }
    CopyArgs a{};
    a.k = (u32x4*)k_pool;
    a.v = (u32x4*)v_pool;
    a.page_vecs = n_kv_heads * head_dim * 2;
    a.layer_vecs = num_blocks * a.page_vecs;
    for (int32_t i0 = 0; i0 < n; i0 += kCopyPairs) {
        const int32_t m = std::min(n - i0, kCopyPairs);
        std::copy(src + i0, src + i0 + m, a.src);
        std::copy(dst + i0, dst + i0 + m, a.dst);
        copy_pages_kernel<<<dim3((unsigned)m, (unsigned)num_layers, 2), 256, 0, (hipStream_t)stream>>>(a);
        if (hipGetLastError() != hipSuccess) return GLLM_E_HIP;
    }
    return GLLM_OK;
}

}  // extern "C"
