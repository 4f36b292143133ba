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
__device__ __forceinline__ int64_t scan_wave64(int64_t x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const int64_t y = __shfl_up(x, by);
        if (lane >= by) x += y;
    }
    return x;
}

// Every workgroup adds up the lengths of all sequences for itself (from the caches: 8 bytes a sequence), a tile of 1024 at a time, and then
// writes the rows of every n-th run of 256, finding a row's sequence by bisection in LDS; so there is one launch and nothing that a
// workgroup waits for.  All latency.
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
        const int64_t rows_upto = scan_wave64(rows), pages_upto = scan_wave64(pages);
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
        for (int64_t r0 = (int64_t)(first / kMapsThreads) * kMapsThreads; r0 < all; r0 += kMapsThreads) {
            const int64_t r = r0 + t;
            if ((r0 / kMapsThreads) % gridDim.x != blockIdx.x || r < first || r >= all) continue;
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
    for (int64_t r0 = (int64_t)(fit / kMapsThreads) * kMapsThreads; r0 < a.num_rows; r0 += kMapsThreads) {
        const int64_t r = r0 + t;
        if ((r0 / kMapsThreads) % gridDim.x != blockIdx.x || r < fit || r >= a.num_rows) continue;
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

// A workgroup has a row: its query heads, and, where it is the first row of a page, the keys and values of all rows of the page; a wave takes a page's keys (or values) of one KV head, so that their largest magnitude needs no more than a wave.
template <int D, typename T>
__global__ __launch_bounds__(256) void norm_rope_store8_kernel(Store8Args a) {
    constexpr int LANES = D / 8, PER = 64 / LANES;  // lanes of a head, heads (or tokens) of a wave
    __shared__ u32x2 run[4][kPage];                 // rows and slots of a page
    const int r = blockIdx.x, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t slot = a.slots[r];
    if (slot < 0 || slot >= a.num_slots) return;
    const T* qkv = static_cast<const T*>(a.qkv);
    const int sub = lane / LANES, e = lane % LANES * 4;
    auto rope_of = [&](int row) { return a.rope + (int64_t)min(max(a.positions[row], 0), a.max_position - 1) * D; };
    const int q_tasks = (a.n_q + PER - 1) / PER;
    for (int task = wave; task < q_tasks; task += 4) {
        const int h = task * PER + sub, hh = min(h, a.n_q - 1);
        const T* x = qkv + (int64_t)r * a.ld_qkv + (int64_t)hh * D + e;
        f32x4 lo = load4<T>(x), hi = load4<T>(x + D / 2);
        norm_rotate<D>(lo, hi, a.q_gain, a.eps, rope_of(r), e);
        if (h < a.n_q) {
            bf16_t* o = a.q_out + (int64_t)r * a.ld_q + (int64_t)h * D + e;
            *reinterpret_cast<bf16x4*>(o) = __builtin_convertvector(lo, bf16x4);
            *reinterpret_cast<bf16x4*>(o + D / 2) = __builtin_convertvector(hi, bf16x4);
        }
    }
    // the rows of the page: lane 15 is this row, lanes 15 .. 30 those of the page that this workgroup stores, if none in front is one
    const int at = r - (kPage - 1) + lane;
    const int64_t other = lane < 2 * kPage - 1 && at >= 0 && at < a.num_rows ? a.slots[at] : -1;
    const uint64_t same = __ballot(other >= 0 && other / kPage == slot / kPage);
    if (same & ((1ull << (kPage - 1)) - 1)) return;
    const int n = __popcll(same);
    if (same >> lane & 1) run[wave][__popcll(same & ((1ull << lane) - 1))] = u32x2{(uint32_t)at, (uint32_t)(other % kPage)};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    int first = same >> lane & 1 ? (int)(other % kPage) : kPage;  // the lowest slot
#pragma unroll
    for (int by = 1; by < 64; by *= 2) first = min(first, __shfl_xor(first, by));
    const bool whole = n == kPage && __all(!(same >> lane & 1) || other % kPage == lane - (kPage - 1));  // all slots, in order
    auto row_of = [&](int t) { return (int)run[wave][t][0]; };
    auto slot_of = [&](int t) { return (int)run[wave][t][1]; };
    const int64_t page = slot / kPage;
    for (int task = wave; task < 2 * a.n_kv; task += 4) {
        const int h = task >> 1;
        float* scale_at = a.scales + (page * a.n_kv + h) * 2 + (task & 1);
        const float old = first > 0 ? *scale_at : 0.f;
        int halvings;
        if (task % 2 == 0) {
            constexpr int IT = kPage / PER;
            f32x4 lo[IT], hi[IT];
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const int t = min(i * PER + sub, n - 1);  // (lanes past the page's rows repeat the last one)
                const T* x = qkv + (int64_t)row_of(t) * a.ld_qkv + (int64_t)(a.n_q + h) * D + e;
                lo[i] = load4<T>(x);
                hi[i] = load4<T>(x + D / 2);
            }
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                norm_rotate<D>(lo[i], hi[i], a.k_gain, a.eps, rope_of(row_of(min(i * PER + sub, n - 1))), e);
#pragma unroll
                for (int v = 0; v < 4; ++v) m = fmaxf(m, fmaxf(finite_abs(lo[i][v]), finite_abs(hi[i][v])));
            }
            const float scale = page_scale(max_wave(m), first == 0, old, halvings), inv = 1.0f / scale;
            uint8_t* base = a.k_pool + (page * a.n_kv + h) * (D * kPage);
            if (halvings > 0) {
                const float by = __builtin_ldexpf(1.0f, -halvings);
                for (int p = lane; p < D; p += 64) {  // 16-byte pieces: 16 dims of one slot
                    if (p / (D / 4) * 4 + p % 4 >= first) continue;
                    u32x4* at = reinterpret_cast<u32x4*>(base + p * 16);
                    u32x4 c = *at;
#pragma unroll
                    for (int v = 0; v < 4; ++v) c[v] = scaled_codes(c[v], by);
                    *at = c;
                }
            }
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const int t = i * PER + sub;
                if (t >= n) continue;
                const int s = slot_of(t);
                uint8_t* at = base + s / 4 * (4 * D) + s % 4 * 16 + e % 16;
                *reinterpret_cast<uint32_t*>(at + e / 16 * 64) = codes4(lo[i], scale, inv);
                *reinterpret_cast<uint32_t*>(at + (e + D / 2) / 16 * 64) = codes4(hi[i], scale, inv);
            }
            if (lane == 0) *scale_at = scale;
        } else {
            constexpr int DIMS = D / 64;  // of a lane, next to each other
            float x[kPage][DIMS], m = 0.f;
#pragma unroll
            for (int t = 0; t < kPage; ++t)
#pragma unroll
                for (int j = 0; j < DIMS; ++j) x[t][j] = t < n ? (float)qkv[(int64_t)row_of(t) * a.ld_qkv + (int64_t)(a.n_q + a.n_kv + h) * D + lane * DIMS + j] : 0.f;
#pragma unroll
            for (int t = 0; t < kPage; ++t)
#pragma unroll
                for (int j = 0; j < DIMS; ++j) m = fmaxf(m, finite_abs(x[t][j]));
            const float scale = page_scale(max_wave(m), first == 0, old, halvings), inv = 1.0f / scale;
            uint8_t* base = a.v_pool + (page * a.n_kv + h) * (D * kPage) + lane * DIMS * kPage;
            const float by = __builtin_ldexpf(1.0f, -halvings);
#pragma unroll
            for (int j = 0; j < DIMS; ++j) {
                u32x4* at = reinterpret_cast<u32x4*>(base + j * kPage);
                u32x4 c;
#pragma unroll
                for (int v = 0; v < 4; ++v) c[v] = codes4(f32x4{x[4 * v][j], x[4 * v + 1][j], x[4 * v + 2][j], x[4 * v + 3][j]}, scale, inv);
                if (whole) {
                    *at = c;
                    continue;
                }
                // the bytes of the slots written are new, those in front of the first are kept, the others stay
                u32x4 was = *at;
                uint8_t* b = reinterpret_cast<uint8_t*>(at);
                if (halvings > 0) {
                    u32x4 kept;
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        kept[v] = scaled_codes(was[v], by);
                        const int mine = min(max(first - 4 * v, 0), 4);
                        const uint32_t mask = mine == 4 ? 0xFFFFFFFFu : (1u << (8 * mine)) - 1u;
                        was[v] = (was[v] & ~mask) | (kept[v] & mask);
                    }
                    *at = was;
                }
#pragma unroll
                for (int t = 0; t < kPage; ++t)
                    if (t < n) b[slot_of(t)] = (uint8_t)(c[t / 4] >> (8 * (t % 4)));
            }
            if (lane == 0) *scale_at = scale;
        }
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
    if (num_rows < 0 || n_q_heads < 1 || n_kv_heads < 1 || max_position < 1 || num_blocks < 1 || !(eps >= 0.0) || !std::isfinite(eps) ||
        (rows_type != GLLM_ROWS_F32 && rows_type != GLLM_ROWS_BF16))
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
    const dim3 grid((unsigned)num_rows);
    if (head_dim == 128 && rows_type == GLLM_ROWS_F32) norm_rope_store8_kernel<128, float><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    else if (head_dim == 128) norm_rope_store8_kernel<128, bf16_t><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    else if (rows_type == GLLM_ROWS_F32) norm_rope_store8_kernel<64, float><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    else norm_rope_store8_kernel<64, bf16_t><<<grid, 256, 0, (hipStream_t)stream>>>(a);
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
    const hipError_t e = launch_attention8(a, (hipStream_t)stream);
    return e == hipSuccess ? GLLM_OK : e == hipErrorInvalidValue ? GLLM_E_CAPACITY : GLLM_E_HIP;
}
