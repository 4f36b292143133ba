// The inner step of attention over the paged pool that the kernels of kernels_attn.hip and kernels_tree.hip share: a block of 32 keys
// (two pages) against groups of 16 columns, in transposed form (kernels_attn.hip says why and which lane holds what).
#pragma once
#include "common.h"

namespace {

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

constexpr float kNegBig = -1.0e30f;

// K and V operands of one block of 32 keys (two pages) for a decode row.  Score tile t is page t, so a lane of group G ends
// up with keys 4G .. 4G+3 of either page, and its V operand is those slots of both.
template <int D>
struct KvFrag {
    u32x4 k[2][D / 32];  // [page][k-step]: operand row r = slot r
    u32x4 v[D / 16];     // [16-dim block]: slots 4G .. 4G+3 of dim r, first page in the low half
};

// Every instruction takes whole 128-byte lines: with lane groups owning 8 consecutive keys (as in the prefill kernel) a
// K line is split over two instructions, and a line loaded with the non-temporal hint is fetched for each (4 % more
// traffic: 512 rows of 1024 .. 8192 keys, 3 layers 4313 -> 4216 us; 251 rows of 64 .. 1100 keys, 8 layers 2224 -> 2182 us).
// The hint itself: a decode row's K and V are read once and never again, and without it the stream is allocated in the
// caches on its way (5.78 -> 6.20 TB/s on 256 rows of 512 .. 4096 keys; a bare streaming read without the hint sustains
// 5.9 - 6.2, with it 6.5).
template <int D>
__device__ __forceinline__ void load_kv(KvFrag<D>& f, const bf16_t* __restrict__ kp, const bf16_t* __restrict__ vp,
                                        int64_t page0, int64_t page1, int n_kv, int kvh, int lane) {
    constexpr int64_t PH = (int64_t)D * kPage;  // elements of one (page, head)
    const int r = lane & 15, G = lane >> 4;
    // K page layout [d/8 groups][16 slots][8]: 16 bytes per (group, slot); V page layout [d][16 slots]
    const bf16_t* k0 = kp + (page0 * n_kv + kvh) * PH + (G * kPage + r) * 8;
    const bf16_t* k1 = kp + (page1 * n_kv + kvh) * PH + (G * kPage + r) * 8;
    const bf16_t* v0 = vp + (page0 * n_kv + kvh) * PH + r * kPage + G * 4;
    const bf16_t* v1 = vp + (page1 * n_kv + kvh) * PH + r * kPage + G * 4;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        f.k[0][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k0 + s * 512));
        f.k[1][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k1 + s * 512));
    }
#pragma unroll
    for (int b = 0; b < D / 16; ++b) {
        const u32x2 lo = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(v0 + b * 256));
        const u32x2 hi = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(v1 + b * 256));
        f.v[b] = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
}

// State of NB column groups across the key loop.
template <int D, int NB>
struct AttnState {
    f32x4 o[NB][D / 16];
    float m[NB];
    float l[NB];
};

// Masks the V fragments of keys >= valid_end (slots that hold no data yet may contain any bit pattern,
// also NaN, and 0 * NaN would poison the P.V product).  v[b] holds this lane's keys key0 .. key0+3 and key1 .. key1+3 of
// dims block b, two per register.
template <int D>
__device__ __forceinline__ void mask_unwritten_v(u32x4 (&v)[D / 16], int key0, int key1, int valid_end) {
    uint32_t m[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int nv = valid_end - ((w < 2 ? key0 : key1) + 2 * (w & 1));
        m[w] = nv >= 2 ? 0xFFFFFFFFu : (nv == 1 ? 0x0000FFFFu : 0u);
    }
#pragma unroll
    for (int b = 0; b < D / 16; ++b)
#pragma unroll
        for (int w = 0; w < 4; ++w) v[b][w] &= m[w];
}

// One column group against one block of 32 keys, in two phases so that callers
// can fetch the V fragments only after the K fragments are dead.
// Phase 1: raw scores q.k of this lane's 8 keys (not yet scaled).  Lane group G receives rows 4G .. 4G+3 of both operand
// fragments; the caller's choice of the keys in those rows decides which keys these are (key0 .. key0+3 from fragment 0,
// key1 .. key1+3 from fragment 1), and the V operand of the P.V product has to hold the same ones.
template <int D>
__device__ __forceinline__ void score_group(float (&sc)[8], const u32x4 (&kf)[2][D / 32], const bf16x8 (&qf)[D / 32]) {
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[0][s]), qf[s], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[1][s]), qf[s], s1, 0, 0, 0);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        sc[v] = s0[v];
        sc[4 + v] = s1[v];
    }
}
// Scores of keys past `limit` (the last key visible to this lane's column) become a huge negative.
__device__ __forceinline__ void mask_scores(float (&sc)[8], int key0, int key1, int limit) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (key0 + v > limit) sc[v] = kNegBig;
        if (key1 + v > limit) sc[4 + v] = kNegBig;
    }
}

// Phase 2, for all NB column groups of a wave at once: softmax update in base 2 and O^T += V^T P^T.
//
// m is the reference exponent of a column (identical in the four lanes that share the column); p =
// 2^(s*c - m) with c = log2(e)/sqrt(d).  Softmax does not care which reference is used as long as nothing
// overflows.  DEFER = true lets the reference lag: it is only moved (to the exact running maximum: two
// cross-lane exchanges per group, then m, l and the accumulators are rescaled) when some lane sees a score
// more than 64 above it -- always in a wave's first block, where the reference is still the huge negative
// start value, and practically never afterwards -- so p stays below 2^64, sums of 2^13 of them stay finite,
// and the common path has no cross-lane traffic and no rescaling at all: a lane-local maximum, one wave vote,
// the exponentials, the MFMAs.  DEFER = false moves the reference whenever a lane's maximum exceeds it (the
// textbook order): the memory-bound decode kernel, with one group per wave, gains nothing from deferring.
constexpr float kRefSlack = 64.0f;

// Moves the references for the scores of a block.
template <int D, int NB, bool DEFER>
__device__ __forceinline__ void raise_reference(AttnState<D, NB>& st, const float (&sc)[NB][8], float scale_log2) {
    float lm[NB];
    bool low = false;
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        float x = sc[c][0];
#pragma unroll
        for (int v = 1; v < 8; ++v) x = fmaxf(x, sc[c][v]);
        lm[c] = x * scale_log2;
        low |= DEFER ? lm[c] > st.m[c] + kRefSlack : lm[c] > st.m[c];
    }
    if (__any(low)) {  // wave-uniform
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            float bm = fmaxf(lm[c], __shfl_xor(lm[c], 16));
            bm = fmaxf(bm, __shfl_xor(bm, 32));
            const float m_new = fmaxf(st.m[c], bm);
            const float alpha = __builtin_amdgcn_exp2f(st.m[c] - m_new);
            st.l[c] *= alpha;
#pragma unroll
            for (int b = 0; b < D / 16; ++b)
#pragma unroll
                for (int v = 0; v < 4; ++v) st.o[c][b][v] *= alpha;
            st.m[c] = m_new;
        }
    }
}
// The weights of the block by the present references, the operand of the P.V product, and their sums.  The operand is rounded to bf16, since the
// matrix instruction takes both operands in the type of V: each weight is off by at most 2^-8 of itself, independently, on top of an output that
// is rounded to bf16 anyway (error of an output against 64 bits 0.0018 to 0.0023 of its size, 0.0017 with weights of 32 bits).  The sums take the
// weights as they were.
template <int D, int NB>
__device__ __forceinline__ void block_weights(AttnState<D, NB>& st, const float (&sc)[NB][8], float scale_log2, bf16x8 (&pb)[NB]) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        f32x8 p;
        float psum = 0.f;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            p[v] = __builtin_amdgcn_exp2f(fmaf(sc[c][v], scale_log2, -st.m[c]));
            psum += p[v];
        }
        st.l[c] += psum;
        pb[c] = __builtin_convertvector(p, bf16x8);
    }
}

// issue_v() is called before the exponentials (a caller that fetches V from LDS starts its reads there),
// get_v() after them (it returns the fragments, waiting for them if need be).
template <int D, int NB, bool DEFER, typename IssueV, typename GetV>
__device__ __forceinline__ void update_groups(AttnState<D, NB>& st, const float (&sc)[NB][8], float scale_log2,
                                              IssueV&& issue_v, GetV&& get_v) {
    raise_reference<D, NB, DEFER>(st, sc, scale_log2);
    issue_v();
    bf16x8 pb[NB];
    block_weights<D, NB>(st, sc, scale_log2, pb);
    const u32x4 (&vf)[D / 16] = get_v();
#pragma unroll
    for (int b = 0; b < D / 16; ++b)
#pragma unroll
        for (int c = 0; c < NB; ++c)
            st.o[c][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[b]), pb[c], st.o[c][b], 0, 0, 0);
}

template <int D, int NB>
__device__ __forceinline__ void init_state(AttnState<D, NB>& st) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        st.m[c] = kNegBig;
        st.l[c] = 0.f;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) st.o[c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
}

}  // namespace
