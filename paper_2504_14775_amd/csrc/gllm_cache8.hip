// A KV cache held in 8 bits: entry points of include/gllm_cache8.h, and the kernels of all of them but attention (kernels_attn8.hip).
#include "../../include/gllm_cache8.h"
#include "cache8.h"

#include <algorithm>
#include <cmath>

namespace {

// ---- the arrays of a step ------------------------------------------------------------------------------------------------

struct MapsArgs {
    const int32_t *new_tokens, *cached_len, *free_pages;
    int32_t* block_tables;
    int32_t *row_start, *positions, *slots, *needed;
    int32_t num_seqs, num_free, table_stride, num_blocks, num_rows;
};

constexpr int kMapsThreads = 256, kMapsPer = 4, kMapsTile = kMapsThreads * kMapsPer;  // sequences looked at together
constexpr int kMapsGroups = 256;                                                      // workgroups at most

// Sums over a wave by lane shifts: x of a lane becomes that of it and the lanes in front.
template <int CTRL, int ROWS>
__device__ __forceinline__ void scan_step(int64_t& x) {
    const int lo = __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
    x += (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
}
__device__ __forceinline__ int64_t scan_wave(int64_t x) {
    scan_step<0x111, 0xf>(x);  // by 1, 2, 4 and 8 lanes in a row of 16
    scan_step<0x112, 0xf>(x);
    scan_step<0x114, 0xf>(x);
    scan_step<0x118, 0xf>(x);
    scan_step<0x142, 0xa>(x);  // the last lane of a row to the next row, of both to the upper half
    scan_step<0x143, 0xc>(x);
    return x;
}

// Every workgroup adds up the lengths of all sequences for itself (from the caches: 8 bytes a sequence), a tile of 1024 at a time, and then writes
// the rows of every n-th run of 256, finding a row's sequence by bisection in LDS; so there is one launch and nothing that a workgroup waits for.
// All latency: lengths, sums over a wave and four waves, the bisection's ten reads of LDS, a page id.  64 sequences 5.8 us, 512 with 4000 rows 6.9 (a
// call 7: of the host); with the rows' runs found by divisions 9.5.
__global__ __launch_bounds__(kMapsThreads) void step_maps_kernel(MapsArgs a) {
    __shared__ int64_t wave_rows[4], wave_pages[4];
    __shared__ int32_t start[kMapsTile + 1], taken[kMapsTile], cached[kMapsTile];  // of a sequence: first row, first free page, cached length (-1: broken)
    __shared__ int fit;                                                           // rows up to here have a place
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    int64_t rows_before = 0, pages_before = 0;
    int first = 0;  // rows of the tiles in front
    if (t == 0) fit = 0;
    if (t == 0 && blockIdx.x == 0) a.row_start[0] = 0;
    const int64_t most = min((int64_t)a.table_stride * kPage, (int64_t)kMaxPositions);
    // the runs of 256 rows are dealt to the workgroups in turn: this thread's row of the first run of its own that reaches behind row r0
    const int64_t step = (int64_t)gridDim.x * kMapsThreads;
    auto my_row = [&](int r0) {
        const uint32_t run = (uint32_t)r0 / kMapsThreads, turn = run % gridDim.x;
        return (int64_t)(run - turn + blockIdx.x + (blockIdx.x < turn ? gridDim.x : 0)) * kMapsThreads + t;
    };
    for (int s0 = 0; s0 < a.num_seqs; s0 += kMapsTile) {
        int32_t n[kMapsPer], c[kMapsPer], need[kMapsPer];
        int64_t rows = 0, pages = 0;
#pragma unroll
        for (int i = 0; i < kMapsPer; ++i) {
            const int s = s0 + t * kMapsPer + i;
            n[i] = s < a.num_seqs ? max(a.new_tokens[s], 0) : 0;
            c[i] = s < a.num_seqs ? a.cached_len[s] : 0;
        }
#pragma unroll
        for (int i = 0; i < kMapsPer; ++i) {
            const bool good = c[i] >= 0 && (int64_t)c[i] + n[i] <= most;
            if (!good) c[i] = -1;
            need[i] = good ? (c[i] + n[i] + (kPage - 1)) / kPage - (c[i] + (kPage - 1)) / kPage : 0;
            rows += n[i];
            pages += need[i];
        }
        const int64_t rows_upto = scan_wave(rows), pages_upto = scan_wave(pages);
        if (lane == 63) {
            wave_rows[wave] = rows_upto;
            wave_pages[wave] = pages_upto;
        }
        __syncthreads();  // (and the rows of the tile before have been written)
        int64_t end = rows_before + rows_upto - rows, page = pages_before + pages_upto - pages;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) {
                end += wave_rows[w];
                page += wave_pages[w];
            }
            rows_before += wave_rows[w];
            pages_before += wave_pages[w];
        }
        int64_t ends[kMapsPer];
        int top = 0;
#pragma unroll
        for (int i = 0; i < kMapsPer; ++i) {
            cached[t * kMapsPer + i] = c[i];
            taken[t * kMapsPer + i] = (int32_t)min(page, (int64_t)INT32_MAX);
            page += need[i];
            end += n[i];
            ends[i] = end;
            if (end <= a.num_rows) top = (int)end;
        }
        if (t == 0) start[0] = first;
        atomicMax(&fit, top);
        __syncthreads();
        const int all = fit;
#pragma unroll
        for (int i = 0; i < kMapsPer; ++i) {
            const int e = ends[i] <= a.num_rows ? (int)ends[i] : all, s = s0 + t * kMapsPer + i;
            start[t * kMapsPer + i + 1] = e;
            if (s < a.num_seqs && (s0 / kMapsTile) % gridDim.x == blockIdx.x) a.row_start[s + 1] = e;
        }
        __syncthreads();
        for (int64_t r = my_row(first); r < all; r += step) {
            if (r < first) continue;
            int lo = 0, hi = kMapsTile;  // the sequence with start[lo] <= r < start[lo + 1]: the last one that starts at r or in front
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (start[mid] <= r) lo = mid;
                else hi = mid;
            }
            int pos = 0, slot = -1;
            if (cached[lo] >= 0) {
                pos = cached[lo] + (int)(r - start[lo]);
                const int entry = pos / kPage, held = (cached[lo] + (kPage - 1)) / kPage;
                int32_t* at = a.block_tables + (int64_t)(s0 + lo) * a.table_stride + entry;
                int id;
                if (entry >= held) {
                    const int64_t i = (int64_t)taken[lo] + entry - held;
                    id = i < a.num_free ? a.free_pages[i] : -1;
                    if (pos % kPage == 0) *at = id;
                } else {
                    id = *at;
                }
                if (id >= 0 && id < a.num_blocks) slot = id * kPage + pos % kPage;
            }
            a.positions[r] = pos;
            a.slots[r] = slot;
        }
        first = all;
    }
    __syncthreads();
    if (t == 0 && blockIdx.x == 0) {
        a.needed[0] = (int32_t)min(rows_before, (int64_t)INT32_MAX);
        a.needed[1] = (int32_t)min(pages_before, (int64_t)INT32_MAX);
    }
    for (int64_t r = my_row(fit); r < a.num_rows; r += step) {
        if (r < fit) continue;
        a.positions[r] = 0;
        a.slots[r] = -1;
    }
}

// ---- norm, rotation and store ------------------------------------------------------------------------------------------

struct Store8Args {
    const void* qkv;
    int64_t ld_qkv;
    const bf16_t *q_gain, *k_gain;
    float eps;
    const float* rope;
    int32_t max_position;
    const int32_t *positions, *slots;
    int32_t num_rows, n_q, n_kv;
    bf16_t* q_out;
    int64_t ld_q;
    uint8_t *k_pool, *v_pool;
    float* scales;
    int64_t num_slots;
};

template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p);
template <>
__device__ __forceinline__ f32x4 load4<float>(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
template <>
__device__ __forceinline__ f32x4 load4<bf16_t>(const bf16_t* p) { return __builtin_convertvector(*reinterpret_cast<const bf16x4*>(p), f32x4); }

__device__ __forceinline__ float max_wave(float x) {
#pragma unroll
    for (int by = 1; by < 64; by *= 2) x = fmaxf(x, __shfl_xor(x, by));
    return x;
}
// The magnitude of a finite value; of any other 0.
__device__ __forceinline__ float finite_abs(float x) {
    x = fabsf(x);
    return x < INFINITY ? x : 0.f;
}
// Codes of four values by `scale`, inv its reciprocal, and of those that are not finite the code that is no number.  (The quotient is corrected
// by its remainder, so that it is that of a division and no value next to the border of two codes gets the wrong one.)
__device__ __forceinline__ uint32_t codes4(f32x4 x, float scale, float inv) {
    float y[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        y[v] = x[v] * inv;
        y[v] = fmaf(fmaf(-y[v], scale, x[v]), inv, y[v]);
        y[v] = fminf(fmaxf(y[v], -kCodeMax), kCodeMax);
        if (!(fabsf(x[v]) < INFINITY)) y[v] = NAN;
    }
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
}
__device__ __forceinline__ uint32_t scaled_codes(uint32_t c, float by) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * by, lo[1] * by, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * by, hi[1] * by, r, true);
}

// The scale of a page side for the largest new magnitude m, and the power of two by which kept codes are divided.  (m / 448 in 32 bits, as the
// scale itself; a page grows by whole powers of two so that its kept codes are exact but for the smallest ones, however often it grows.)
__device__ __forceinline__ float page_scale(float m, bool begun, float old, int& halvings) {
    const float fit = fmaxf(m / kCodeMax, kScaleMin);
    halvings = 0;
    if (begun) return fit;
    if (!(old > 0.f && old < INFINITY)) old = kScaleMin;
    const float mf = __builtin_amdgcn_frexp_mantf(fit), mo = __builtin_amdgcn_frexp_mantf(old);
    halvings = max(__builtin_amdgcn_frexp_expf(fit) - __builtin_amdgcn_frexp_expf(old) + (mf > mo ? 1 : 0), 0);
    return __builtin_ldexpf(old, halvings);
}

// One head of a row in D/8 lanes: elements e .. e+3 and their partners D/2 further, normalised and rotated.
template <int D>
__device__ __forceinline__ void norm_rotate(f32x4& lo, f32x4& hi, const bf16_t* gain, float eps, const float* rope, int e) {
    if (gain) {
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < 4; ++v) sum += lo[v] * lo[v] + hi[v] * hi[v];
#pragma unroll
        for (int by = 1; by < D / 8; by *= 2) sum += __shfl_xor(sum, by);
        const float inv = 1.0f / sqrtf(sum * (1.0f / D) + eps);
        const f32x4 gl = load4<bf16_t>(gain + e), gh = load4<bf16_t>(gain + e + D / 2);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            lo[v] *= inv * gl[v];
            hi[v] *= inv * gh[v];
        }
    }
    const f32x4 c01 = *reinterpret_cast<const f32x4*>(rope + 2 * e), c23 = *reinterpret_cast<const f32x4*>(rope + 2 * e + 4);
    const f32x4 co = {c01[0], c01[2], c23[0], c23[2]}, si = {c01[1], c01[3], c23[1], c23[3]};
    f32x4 a, b;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        a[v] = lo[v] * co[v] - hi[v] * si[v];
        b[v] = hi[v] * co[v] + lo[v] * si[v];
    }
    lo = a;
    hi = b;
}

// A wave has kQueryPasses passes over query heads of a row, all asked for at one time, or the keys, or the values, of one KV head of the pages whose
// first rows are among 16 rows: a page's largest magnitude then needs no more than a wave, and there is one pass over the projection.  The pages
// among these that receive one row only (decode rows) are done together, D/8 lanes to each, the others one after another (1024 decode rows 23 -> 17
// us).  Bound by HBM for chunks: 8192 rows of 64 + 16 heads of 128 in float, 491 MB, 94 us, 5.2 TB/s, what a copy reaches; queries alone 75, pages
// alone 23.  2053 rows of 40 + 16 heads, 251 of them single, 85 MB: 20 us, of which 15 for the pages alone, whose chain (slots, rows, largest
// magnitude, kept codes, stores) is the longer one, so that they are the first workgroups (26 us behind the queries).  64 decode rows 9 us, latency.
// Query passes 1 / 2 / 4: 77 / 75 / 78 us for the queries of the 8192 rows.
constexpr int kQueryPasses = 2;

// The rows of a page and their slots in it, in order of the rows.
struct PageRows {
    const u32x2* run;  // LDS
    int n, first;      // first: the lowest slot
    bool whole;        // all slots, in order
    __device__ __forceinline__ int row(int t) const { return (int)run[t][0]; }
    __device__ __forceinline__ int slot(int t) const { return (int)run[t][1]; }
};

template <int D, typename T>
__device__ __forceinline__ void store_queries(const Store8Args& a, int r, int part) {
    constexpr int LANES = D / 8, PER = 64 / LANES;  // lanes of a head, heads of a pass
    const int lane = threadIdx.x & 63, sub = lane / LANES, e = lane % LANES * 4;
    const T* x = static_cast<const T*>(a.qkv) + (int64_t)r * a.ld_qkv + e;
    f32x4 lo[kQueryPasses], hi[kQueryPasses];
    const int head0 = part * kQueryPasses * PER;
#pragma unroll
    for (int i = 0; i < kQueryPasses; ++i) {
        if (head0 + i * PER >= a.n_q) break;
        const T* at = x + (int64_t)min(head0 + i * PER + sub, a.n_q - 1) * D;
        lo[i] = load4<T>(at);
        hi[i] = load4<T>(at + D / 2);
    }
    const int64_t slot = a.slots[r];
    const float* rope = a.rope + (int64_t)min(max(a.positions[r], 0), a.max_position - 1) * D;
    if (slot < 0 || slot >= a.num_slots) return;
#pragma unroll
    for (int i = 0; i < kQueryPasses; ++i) {
        if (head0 + i * PER >= a.n_q) break;
        norm_rotate<D>(lo[i], hi[i], a.q_gain, a.eps, rope, e);
        const int h = head0 + i * PER + sub;
        if (h < a.n_q) {
            bf16_t* o = a.q_out + (int64_t)r * a.ld_q + (int64_t)h * D + e;
            *reinterpret_cast<bf16x4*>(o) = __builtin_convertvector(lo[i], bf16x4);
            *reinterpret_cast<bf16x4*>(o + D / 2) = __builtin_convertvector(hi[i], bf16x4);
        }
    }
}

template <int D, typename T>
__device__ __forceinline__ void store_keys(const Store8Args& a, const PageRows& p, int64_t page, int h) {
    constexpr int LANES = D / 8, PER = 64 / LANES, IT = kPage / PER;  // lanes of a head, tokens of a pass, passes
    const int lane = threadIdx.x & 63, sub = lane / LANES, e = lane % LANES * 4;
    float* scale_at = a.scales + (page * a.n_kv + h) * 2;
    const float old = p.first > 0 ? *scale_at : 0.f;
    f32x4 lo[IT], hi[IT];
    int pos[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        if (i * PER >= p.n) break;
        const int row = p.row(min(i * PER + sub, p.n - 1));  // (lanes past the page's rows repeat the last one)
        const T* x = static_cast<const T*>(a.qkv) + (int64_t)row * a.ld_qkv + (int64_t)(a.n_q + h) * D + e;
        lo[i] = load4<T>(x);
        hi[i] = load4<T>(x + D / 2);
        pos[i] = a.positions[row];
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        if (i * PER >= p.n) break;
        norm_rotate<D>(lo[i], hi[i], a.k_gain, a.eps, a.rope + (int64_t)min(max(pos[i], 0), a.max_position - 1) * D, e);
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, fmaxf(finite_abs(lo[i][v]), finite_abs(hi[i][v])));
    }
    int halvings;
    const float scale = page_scale(max_wave(m), p.first == 0, old, halvings), inv = 1.0f / scale;
    uint8_t* base = a.k_pool + (page * a.n_kv + h) * (D * kPage);
    if (halvings > 0) {
        const float by = __builtin_ldexpf(1.0f, -halvings);
        for (int x = lane; x < D; x += 64) {  // 16-byte pieces: 16 dims of one slot
            if (x / (D / 4) * 4 + x % 4 >= p.first) continue;
            u32x4* at = reinterpret_cast<u32x4*>(base + x * 16);
            u32x4 c = *at;
#pragma unroll
            for (int v = 0; v < 4; ++v) c[v] = scaled_codes(c[v], by);
            *at = c;
        }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int t = i * PER + sub;
        if (t >= p.n) continue;
        const int s = p.slot(t);
        uint8_t* at = base + s / 4 * (4 * D) + s % 4 * 16 + e % 16;
        *reinterpret_cast<uint32_t*>(at + e / 16 * 64) = codes4(lo[i], scale, inv);
        *reinterpret_cast<uint32_t*>(at + (e + D / 2) / 16 * 64) = codes4(hi[i], scale, inv);
    }
    if (lane == 0) *scale_at = scale;
}

// The values of a dim in the slots in front of `first` times `by`.
__device__ __forceinline__ void keep_scaled(void* values, int first, float by) {
    u32x4* at = static_cast<u32x4*>(values);
    u32x4 was = *at;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int mine = min(max(first - 4 * v, 0), 4);
        const uint32_t mask = mine == 4 ? 0xFFFFFFFFu : (1u << (8 * mine)) - 1u;
        was[v] = (was[v] & ~mask) | (scaled_codes(was[v], by) & mask);
    }
    *at = was;
}

template <int D, typename T>
__device__ __forceinline__ void store_values(const Store8Args& a, const PageRows& p, int64_t page, int h) {
    constexpr int DIMS = D / 64;  // of a lane, next to each other
    typedef T pair_t __attribute__((ext_vector_type(DIMS)));
    const int lane = threadIdx.x & 63;
    float* scale_at = a.scales + (page * a.n_kv + h) * 2 + 1;
    const float old = p.first > 0 ? *scale_at : 0.f;
    float x[kPage][DIMS], m = 0.f;
#pragma unroll
    for (int t = 0; t < kPage; ++t) {
#pragma unroll
        for (int j = 0; j < DIMS; ++j) x[t][j] = 0.f;
        if (t >= p.n) continue;
        const T* at = static_cast<const T*>(a.qkv) + (int64_t)p.row(t) * a.ld_qkv + (int64_t)(a.n_q + a.n_kv + h) * D + lane * DIMS;
        const pair_t y = *reinterpret_cast<const pair_t*>(at);
#pragma unroll
        for (int j = 0; j < DIMS; ++j) x[t][j] = (float)y[j];
    }
#pragma unroll
    for (int t = 0; t < kPage; ++t)
#pragma unroll
        for (int j = 0; j < DIMS; ++j) m = fmaxf(m, finite_abs(x[t][j]));
    int halvings;
    const float scale = page_scale(max_wave(m), p.first == 0, old, halvings), inv = 1.0f / scale;
    uint8_t* base = a.v_pool + (page * a.n_kv + h) * (D * kPage) + lane * DIMS * kPage;
    const float by = __builtin_ldexpf(1.0f, -halvings);
#pragma unroll
    for (int j = 0; j < DIMS; ++j) {
        u32x4* at = reinterpret_cast<u32x4*>(base + j * kPage);
        u32x4 c;
#pragma unroll
        for (int v = 0; v < 4; ++v) c[v] = codes4(f32x4{x[4 * v][j], x[4 * v + 1][j], x[4 * v + 2][j], x[4 * v + 3][j]}, scale, inv);
        if (p.whole) {
            *at = c;
            continue;
        }
        if (halvings > 0) keep_scaled(at, p.first, by);
        uint8_t* b = reinterpret_cast<uint8_t*>(at);
#pragma unroll
        for (int t = 0; t < kPage; ++t)
            if (t < p.n) b[p.slot(t)] = (uint8_t)(c[t / 4] >> (8 * (t % 4)));
    }
    if (lane == 0) *scale_at = scale;
}

// Keys (or values) of a KV head for n rows that are the only ones of their pages; list: row and slot of each.
template <int D, bool KEYS, typename T>
__device__ __forceinline__ void store_singles(const Store8Args& a, const u32x2* list, int n, int h) {
    constexpr int LANES = D / 8, PER = 64 / LANES, IT = kPage / PER;
    const int lane = threadIdx.x & 63, sub = lane / LANES, e = lane % LANES * 4;
    f32x4 lo[IT], hi[IT];
    float old[IT];
    int pos[IT], slot[IT];
    uint8_t* const pool = KEYS ? a.k_pool : a.v_pool;
    auto scale_of = [&](int i) { return a.scales + ((int64_t)(slot[i] / kPage) * a.n_kv + h) * 2 + (KEYS ? 0 : 1); };
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        if (i * PER >= n) break;
        const u32x2 of = list[min(i * PER + sub, n - 1)];
        const T* x = static_cast<const T*>(a.qkv) + (int64_t)of[0] * a.ld_qkv + (int64_t)(a.n_q + (KEYS ? 0 : a.n_kv) + h) * D + e;
        lo[i] = load4<T>(x);
        hi[i] = load4<T>(x + D / 2);
        slot[i] = (int)of[1];
        old[i] = *scale_of(i);
        pos[i] = KEYS ? a.positions[of[0]] : 0;
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        if (i * PER >= n) break;
        if (KEYS) norm_rotate<D>(lo[i], hi[i], a.k_gain, a.eps, a.rope + (int64_t)min(max(pos[i], 0), a.max_position - 1) * D, e);
        float m = 0.f;
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, fmaxf(finite_abs(lo[i][v]), finite_abs(hi[i][v])));
#pragma unroll
        for (int by = 1; by < LANES; by *= 2) m = fmaxf(m, __shfl_xor(m, by));
        if (i * PER + sub >= n) continue;
        const int first = slot[i] % kPage;
        int halvings;
        const float scale = page_scale(m, first == 0, old[i], halvings), inv = 1.0f / scale, by = __builtin_ldexpf(1.0f, -halvings);
        uint8_t* base = pool + ((int64_t)(slot[i] / kPage) * a.n_kv + h) * (D * kPage);
        const uint32_t cl = codes4(lo[i], scale, inv), ch = codes4(hi[i], scale, inv);
        if (KEYS) {
            if (halvings > 0) {
                for (int x = lane % LANES; x < D; x += LANES) {  // 16-byte pieces: 16 dims of one slot
                    if (x / (D / 4) * 4 + x % 4 >= first) continue;
                    u32x4* at = reinterpret_cast<u32x4*>(base + x * 16);
                    u32x4 c = *at;
#pragma unroll
                    for (int v = 0; v < 4; ++v) c[v] = scaled_codes(c[v], by);
                    *at = c;
                }
            }
            uint8_t* at = base + first / 4 * (4 * D) + first % 4 * 16 + e % 16;
            *reinterpret_cast<uint32_t*>(at + e / 16 * 64) = cl;
            *reinterpret_cast<uint32_t*>(at + (e + D / 2) / 16 * 64) = ch;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint8_t* at = base + (e + j % 4 + (j < 4 ? 0 : D / 2)) * kPage;
                if (halvings > 0) keep_scaled(at, first, by);
                at[first] = (uint8_t)((j < 4 ? cl : ch) >> (8 * (j % 4)));
            }
        }
        if (lane % LANES == 0) *scale_of(i) = scale;
    }
}

template <int D, typename T>
__global__ __launch_bounds__(256) void norm_rope_store8_kernel(Store8Args a, int query_groups, int query_parts) {
    __shared__ u32x2 lists[4][kPage];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int page_groups = (int)gridDim.x - query_groups;
    if ((int)blockIdx.x >= page_groups) {
        const int64_t id = (int64_t)((int)blockIdx.x - page_groups) * 4 + wave;
        const int r = (int)(id / query_parts);
        if (r < a.num_rows) store_queries<D, T>(a, r, (int)(id - (int64_t)r * query_parts));
        return;
    }
    const int64_t id = (int64_t)blockIdx.x * 4 + wave;
    const int64_t block = id / (2 * a.n_kv), r0 = block * kPage;
    const int task = (int)(id - block * (2 * a.n_kv)), h = task / 2;
    if (r0 >= a.num_rows) return;
    // lanes 15 .. 30 have the rows among which first ones are looked for, the 15 lanes on either side those that may be of the same page
    const int64_t at = r0 - (kPage - 1) + lane;
    int slot = lane < 3 * kPage - 2 && at >= 0 && at < a.num_rows ? a.slots[at] : -1;
    if (slot >= a.num_slots) slot = -1;
    const int page = slot < 0 ? -1 : slot / kPage, s = slot % kPage;
    u32x2* const list = lists[wave];
    auto write_list = [&](uint64_t who, int what) {
        __builtin_amdgcn_wave_barrier();
        if (who >> lane & 1) list[__popcll(who & ((1ull << lane) - 1))] = u32x2{(uint32_t)at, (uint32_t)what};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    const int above = __shfl_up(page, 1);  // (by all lanes, also those without a page)
    uint64_t firsts = __ballot(page >= 0 && page != above) & (((1ull << kPage) - 1) << (kPage - 1)), singles = 0;
    for (uint64_t todo = firsts; todo; todo &= todo - 1) {
        const int l = __builtin_ctzll(todo), of = __builtin_amdgcn_readlane(page, l);
        const uint64_t same = __ballot(page == of) & (((1ull << (2 * kPage - 1)) - 1) << (l - (kPage - 1))), this_one = 1ull << l;
        if (same & (this_one - 1)) firsts &= ~this_one;  // a row further up is of this page
        else if (same == this_one) singles |= this_one;
    }
    if (singles) {
        write_list(singles, slot);
        if (task % 2 == 0) store_singles<D, true, T>(a, list, __popcll(singles), h);
        else store_singles<D, false, T>(a, list, __popcll(singles), h);
    }
    for (uint64_t todo = firsts & ~singles; todo; todo &= todo - 1) {
        const int l = __builtin_ctzll(todo), of = __builtin_amdgcn_readlane(page, l);
        const uint64_t same = __ballot(page == of) & (((1ull << kPage) - 1) << l);
        const bool mine = same >> lane & 1;
        PageRows p;
        p.run = list;
        p.n = __popcll(same);
        write_list(same, s);
        uint32_t held = mine ? 1u << s : 0u;  // the slots that are written
#pragma unroll
        for (int by = 1; by < 64; by *= 2) held |= (uint32_t)__shfl_xor((int)held, by);
        p.first = __builtin_ctz(held);
        p.whole = p.n == kPage && __all(!mine || s == lane - l);
        if (task % 2 == 0) store_keys<D, T>(a, p, of, h);
        else store_values<D, T>(a, p, of, h);
    }
}

gllm_status launched() { return hipGetLastError() == hipSuccess ? GLLM_OK : GLLM_E_HIP; }

bool misaligned(const void* p, int to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) != 0; }

float base2(float scale) { return (float)(scale * 1.4426950408889634); }  // of scores whose exponentials are taken in base 2

bool attention_shape_ok(int n_q, int n_kv, int d, int max_new) {
    return n_q > 0 && n_kv > 0 && max_new > 0 && n_q % n_kv == 0 && n_q / n_kv <= 16 && (d == 64 || d == 128);
}

}  // namespace

gllm_status gllm_op_step_maps(const int32_t* new_tokens, const int32_t* cached_len, int32_t num_seqs, const int32_t* free_pages,
                              int32_t num_free, int32_t* block_tables, int32_t block_table_stride, int64_t num_blocks, int32_t num_rows,
                              int32_t* row_start, int32_t* positions, int32_t* slots, int32_t* needed, void* stream) {
    if (num_seqs < 0 || num_free < 0 || num_rows < 0 || block_table_stride < 1 || num_blocks < 1) return GLLM_E_INVALID;
    if (num_blocks > GLLM_CACHE8_MAX_BLOCKS) return GLLM_E_UNSUPPORTED;
    if (num_seqs > kMaxAttn8Seqs) return GLLM_E_CAPACITY;
    if (!row_start || !needed || (num_seqs > 0 && (!new_tokens || !cached_len || !block_tables)) || (num_free > 0 && !free_pages) ||
        (num_rows > 0 && (!positions || !slots)))
        return GLLM_E_INVALID;
    const MapsArgs a{new_tokens, cached_len, free_pages, block_tables, row_start, positions, slots, needed, num_seqs, num_free,
                     block_table_stride, (int32_t)num_blocks, num_rows};
    const int groups = (int)std::min<int64_t>(kMapsGroups, std::max<int64_t>(1, ceil_div(num_rows, kMapsThreads)));
    step_maps_kernel<<<groups, kMapsThreads, 0, (hipStream_t)stream>>>(a);
    return launched();
}

gllm_status gllm_op_norm_rope_store8(const void* qkv, int64_t ld_qkv, int32_t rows_type, const void* q_gain, const void* k_gain, double eps,
                                     const float* rope, int32_t max_position, const int32_t* positions, const int32_t* slots,
                                     int32_t num_rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, void* q_out, int64_t ld_q,
                                     void* k_pool, void* v_pool, float* scales, int64_t num_blocks, void* stream) {
    if (num_rows < 0 || n_q_heads < 1 || n_kv_heads < 1 || max_position < 1 || num_blocks < 1 || !(eps >= 0.0) || !std::isfinite((float)eps) ||
        (eps > 0.0 && (float)eps == 0.f) || (rows_type != GLLM_ROWS_F32 && rows_type != GLLM_ROWS_BF16))
        return GLLM_E_INVALID;
    if ((head_dim != 64 && head_dim != 128) || (int64_t)n_q_heads + 2 * (int64_t)n_kv_heads > 65535 || num_blocks > GLLM_CACHE8_MAX_BLOCKS)
        return GLLM_E_UNSUPPORTED;
    if (num_rows == 0) return GLLM_OK;
    if (!qkv || !rope || !positions || !slots || !q_out || !k_pool || !v_pool || !scales) return GLLM_E_INVALID;
    if (ld_qkv < ((int64_t)n_q_heads + 2 * n_kv_heads) * head_dim || ld_q < (int64_t)n_q_heads * head_dim || ld_qkv % 4 != 0 || ld_q % 4 != 0)
        return GLLM_E_INVALID;
    if (misaligned(qkv, rows_type == GLLM_ROWS_F32 ? 16 : 8) || (q_gain && misaligned(q_gain, 8)) || (k_gain && misaligned(k_gain, 8)) || misaligned(rope, 16) ||
        misaligned(q_out, 8) || misaligned(k_pool, 16) || misaligned(v_pool, 16) || misaligned(scales, 8))
        return GLLM_E_INVALID;
    const Store8Args a{qkv, ld_qkv, (const bf16_t*)q_gain, (const bf16_t*)k_gain, (float)eps, rope, max_position, positions, slots, num_rows,
                       n_q_heads, n_kv_heads, (bf16_t*)q_out, ld_q, (uint8_t*)k_pool, (uint8_t*)v_pool, scales, num_blocks * kPage};
    const int64_t parts = ceil_div(n_q_heads, kQueryPasses * (512 / head_dim));
    const int64_t queries = ceil_div(num_rows * parts, 4), pages = ceil_div(ceil_div(num_rows, kPage) * 2 * n_kv_heads, 4);
    if ((queries + pages) * 256 > UINT32_MAX) return GLLM_E_CAPACITY;
    const dim3 grid((unsigned)(queries + pages));
#define GLLM_STORE8(D_, T_) norm_rope_store8_kernel<D_, T_><<<grid, 256, 0, (hipStream_t)stream>>>(a, (int)queries, (int)parts)
    if (head_dim == 128 && rows_type == GLLM_ROWS_F32) GLLM_STORE8(128, float);
    else if (head_dim == 128) GLLM_STORE8(128, bf16_t);
    else if (rows_type == GLLM_ROWS_F32) GLLM_STORE8(64, float);
    else GLLM_STORE8(64, bf16_t);
#undef GLLM_STORE8
    return launched();
}

size_t gllm_op_attention8_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_new) {
    return attention_shape_ok(n_q_heads, n_kv_heads, head_dim, max_new) ? attention8_workspace_bytes(n_q_heads, n_kv_heads, head_dim, max_new) : 0;
}

gllm_status gllm_op_attention8(const void* q, int64_t ld_q, const void* k_pool, const void* v_pool, const float* scales, int64_t num_blocks,
                               const int32_t* block_tables, int32_t block_table_stride, const int32_t* cached_len,
                               const int32_t* row_start, int32_t num_seqs, int32_t num_rows, int32_t max_new, int32_t window, int32_t sinks,
                               int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float scale, void* out, int64_t ld_out,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (num_seqs < 0 || num_rows < 0 || max_new < 1 || num_blocks < 1 || block_table_stride < 1 || n_q_heads < 1 || n_kv_heads < 1 || window < 0 || sinks < 0 ||
        (sinks > 0 && window == 0) || !(scale > 0.f) || !std::isfinite(base2(scale)))
        return GLLM_E_INVALID;
    if (!attention_shape_ok(n_q_heads, n_kv_heads, head_dim, max_new) || num_blocks > GLLM_CACHE8_MAX_BLOCKS) return GLLM_E_UNSUPPORTED;
    if (num_seqs == 0 || num_rows == 0) return GLLM_OK;
    if (!q || !k_pool || !v_pool || !scales || !block_tables || !cached_len || !row_start || !out || !workspace) return GLLM_E_INVALID;
    if (ld_q < (int64_t)n_q_heads * head_dim || ld_out < (int64_t)n_q_heads * head_dim) return GLLM_E_INVALID;
    if (ld_q % 8 != 0 || ld_out % 4 != 0 || misaligned(q, 16) || misaligned(k_pool, 16) || misaligned(v_pool, 16) || misaligned(scales, 8) || misaligned(out, 8) ||
        misaligned(workspace, 16))
        return GLLM_E_INVALID;
    if (workspace_bytes < attention8_workspace_bytes(n_q_heads, n_kv_heads, head_dim, max_new) || num_seqs > kMaxAttn8Seqs) return GLLM_E_CAPACITY;
    Attn8Args a{};
    a.q = (const bf16_t*)q; a.ld_q = ld_q;
    a.k_pool = (const uint8_t*)k_pool; a.v_pool = (const uint8_t*)v_pool; a.scales = (const f32x2*)scales; a.num_blocks = (int32_t)num_blocks;
    a.block_tables = block_tables; a.table_stride = block_table_stride;
    a.cached_len = cached_len; a.row_start = row_start;
    a.num_seqs = num_seqs; a.num_rows = num_rows; a.max_new = max_new;
    a.window = window; a.sinks = sinks;
    a.out = (bf16_t*)out; a.ld_o = ld_out;
    a.n_q = n_q_heads; a.n_kv = n_kv_heads; a.d = head_dim;
    a.scale_log2 = base2(scale);
    a.workspace = workspace;
    return launch_attention8(a, (hipStream_t)stream);
}
