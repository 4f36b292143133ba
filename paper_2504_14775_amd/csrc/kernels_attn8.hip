// Attention of hybrid batches over the 8-bit pool (contract: include/gllm_cache8.h): a wave per row and query head, 64 keys at a time.
#include "cache8.h"

namespace {

template <int D>
__global__ __launch_bounds__(256) void attention8_kernel(Attn8Args a) {
    __shared__ float qs[4][D], ps[4][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t task = (int64_t)blockIdx.x * 4 + wave;
    if (task >= (int64_t)a.num_rows * a.n_q) return;
    const int r = (int)(task / a.n_q), h = (int)(task % a.n_q), kvh = h / (a.n_q / a.n_kv);
    int mine = -1;
    bool bad = false;
    for (int s = lane; s < a.num_seqs; s += 64) {
        const int r0 = a.row_start[s], r1 = a.row_start[s + 1];
        bad |= r0 < 0 || r1 < r0 || r1 > a.num_rows;
        if (r >= r0 && r < r1) mine = s;
    }
    if (__any(bad) || !__any(mine >= 0)) return;
    const int s = __builtin_amdgcn_readlane(mine, __builtin_ctzll(__ballot(mine >= 0)));
    const int r0 = a.row_start[s], n = a.row_start[s + 1] - r0, c = a.cached_len[s];
    bf16_t* out = a.out + (int64_t)r * a.ld_o + (int64_t)h * D;
    float o[D / 64] = {}, l = 0.f, m = -INFINITY;
    if (n <= a.max_new && c >= 0 && (int64_t)c + n <= min((int64_t)a.table_stride * kPage, (int64_t)kMaxPositions)) {
        for (int i = lane; i < D; i += 64) qs[wave][i] = (float)a.q[(int64_t)r * a.ld_q + (int64_t)h * D + i];
        const int pos = c + r - r0, low = a.window > 0 ? max(0, pos - a.window + 1) : 0;
        for (int b = 0; b <= pos; b += 64) {
            if (b >= a.sinks && b + 63 < low) {
                b = low / 64 * 64 - 64;
                continue;
            }
            const int key = b + lane;
            const bool seen = key <= pos && (key >= low || key < a.sinks);
            int64_t page = 0;
            float x = -INFINITY, vs = 0.f;
            if (seen) {
                page = min(max(a.block_tables[(int64_t)s * a.table_stride + key / kPage], 0), a.num_blocks - 1);
                f32x2 sc = a.scales[page * a.n_kv + kvh];
                sc[0] = fminf(fmaxf(sc[0], kScaleMin), kScaleMax);
                vs = fminf(fmaxf(sc[1], kScaleMin), kScaleMax);
                const int slot = key % kPage;
                const uint8_t* k = a.k_pool + (page * a.n_kv + kvh) * (D * kPage) + slot / 4 * (4 * D) + slot % 4 * 16;
                x = 0.f;
                for (int e = 0; e < D; e += 4) {
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(k + e / 16 * 64 + e % 16);
                    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
                    x += lo[0] * qs[wave][e] + lo[1] * qs[wave][e + 1] + hi[0] * qs[wave][e + 2] + hi[1] * qs[wave][e + 3];
                }
                x *= sc[0] * a.scale_log2;
            }
            float top = x;
            for (int by = 1; by < 64; by *= 2) top = fmaxf(top, __shfl_xor(top, by));
            top = fmaxf(top, m);
            if (!(top > -INFINITY)) continue;
            const float down = __builtin_amdgcn_exp2f(m - top), p = __builtin_amdgcn_exp2f(x - top);
            m = top;
            l = l * down + p;
            ps[wave][lane] = p * vs;
            for (int j = 0; j < D / 64; ++j) o[j] *= down;
            for (uint64_t todo = __ballot(seen); todo; todo &= todo - 1) {
                const int i = __builtin_ctzll(todo);
                const int64_t at = ((int64_t)__builtin_amdgcn_readlane((int)page, i) * a.n_kv + kvh) * (D * kPage) + (b + i) % kPage;
                for (int j = 0; j < D / 64; ++j) o[j] += ps[wave][i] * __builtin_amdgcn_cvt_f32_fp8((int)a.v_pool[at + (lane + 64 * j) * kPage], 0);
            }
        }
        for (int by = 1; by < 64; by *= 2) l += __shfl_xor(l, by);
    }
    for (int j = 0; j < D / 64; ++j) out[lane + 64 * j] = l != 0.f ? (bf16_t)(o[j] / l) : (bf16_t)0.f;
}

}  // namespace

size_t attention8_workspace_bytes(int n_q, int n_kv, int d, int max_new) { return 256; }

hipError_t launch_attention8(const Attn8Args& a, hipStream_t stream) {
    const int64_t groups = ceil_div((int64_t)a.num_rows * a.n_q, 4);
    if (groups > INT32_MAX) return hipErrorInvalidValue;
    if (a.d == 128) attention8_kernel<128><<<(unsigned)groups, 256, 0, stream>>>(a);
    else attention8_kernel<64><<<(unsigned)groups, 256, 0, stream>>>(a);
    return hipGetLastError();
}
