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
#include "attn_core.h"

namespace {

constexpr int kTreeNodes = 256;             // most nodes of a tree: one per thread
constexpr int kTreeWords = kTreeNodes / 32;
constexpr int kTreeStages = 3;

struct TreeItem {
    int32_t seq, tile, row0, n, c, pad;
};

// What the closure of a tree takes in LDS: rows of `stride` words per node (odd, so that neighbouring nodes lie in different
// banks), the parent links, and the words of the nodes that are used.
__host__ __device__ inline int tree_row_words(int max_nodes) { return (max_nodes / 32 + 2) | 1; }
__host__ __device__ inline int tree_lds_bytes(int max_nodes) { return (kTreeNodes * tree_row_words(max_nodes) + kTreeNodes + 2 * (kTreeWords + 1) + 16) * 4; }
struct TreeLds {
    uint32_t* vis;    // [node][stride]: word w of a node: keys 32w .. 32w+31 behind the first key of block c / 32
    int* up;          // [node]
    uint32_t* used;   // [kTreeWords + 1], as a row of vis: all cached keys and all used nodes
    uint32_t* raw;    // [kTreeWords]
    int* scratch;     // [16]
    int stride;
    __device__ TreeLds(void* p, int max_nodes) {
        stride = tree_row_words(max_nodes);
        vis = (uint32_t*)p;
        up = (int*)(vis + kTreeNodes * stride);
        used = (uint32_t*)(up + kTreeNodes);
        raw = used + kTreeWords + 1;
        scratch = (int*)(raw + kTreeWords + 1);
    }
};

// The words of all nodes of a tree of n <= max_nodes nodes behind c cached keys.  Every round joins to a node's set that of the
// node at the end of its link and doubles the link: the depth of the tree is passed in log2 of it rounds.  A link that leads
// to no root is -2 at the end, and the node's words are zero.  All 256 threads; ends with a barrier.
__device__ __forceinline__ void tree_visibility(const TreeLds& t, const int32_t* __restrict__ parents, int n, int c, int max_nodes) {
    const int i = threadIdx.x, words = (max_nodes + 31) / 32, sh = c & 31;
    uint32_t* mine = t.vis + i * t.stride;
    int p = -2;
    if (i < n) {
        const int given = parents[i];
        p = given >= -1 && given < i ? given : -2;
    }
    t.up[i] = p;
    for (int w = 0; w < words; ++w) mine[w] = w == i >> 5 ? 1u << (i & 31) : 0u;
    __syncthreads();
    for (;;) {
        uint32_t b[kTreeWords];
        int next = p;
        if (p >= 0) {
            next = t.up[p];
            for (int w = 0; w < kTreeWords; ++w) b[w] = w < words ? t.vis[p * t.stride + w] : 0u;
        }
        if (!__syncthreads_or(p >= 0)) break;
        if (p >= 0) {
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

// The workgroup's place in the list of all (sequence, tile of columns): the sequence and tile of place `item`.  Sequences that
// break a rule keep their place with n or c as found; the caller sees to that.  False behind the last one.  All threads.
__device__ __forceinline__ bool tree_locate(const TreeArgs& a, int item, int tile_cols, TreeItem& it, int* scratch) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = a.n_q / a.n_kv;
    int64_t before = 0;
    for (int s0 = 0; s0 < a.num_seqs; s0 += 256) {
        const int s = s0 + threadIdx.x;
        int tiles = 0, r0 = 0, n = 0, c = 0;
        if (s < a.num_seqs) {
            r0 = a.row_begin[s];
            const int r1 = a.row_end[s];
            c = a.cached_len[s];
            if (r0 >= 0 && r1 > r0 && r1 <= a.num_rows) n = r1 - r0;
            tiles = (int)(((int64_t)n * g + tile_cols - 1) / tile_cols);
        }
        int sum = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(sum, o);
            if (lane >= o) sum += x;
        }
        if (lane == 63) scratch[wave] = sum;
        if (threadIdx.x == 0) scratch[4] = -1;
        __syncthreads();
        int64_t first = before + sum - tiles;
        for (int w = 0; w < wave; ++w) first += scratch[w];
        before += (int64_t)scratch[0] + scratch[1] + scratch[2] + scratch[3];
        if (item >= first && item < first + tiles) {
            scratch[4] = s;
            scratch[5] = (int)(item - first);
            scratch[6] = r0;
            scratch[7] = n;
            scratch[8] = c;
        }
        __syncthreads();
        if (scratch[4] >= 0) {
            it = TreeItem{scratch[4], scratch[5], scratch[6], scratch[7], scratch[8], 0};
            return true;
        }
        __syncthreads();
    }
    return false;
}

// One workgroup of 4 waves per (sequence, tile of 64*NB columns, KV head): a block of 32 keys is brought into LDS once and
// read by all waves, each of which has NB groups of 16 columns (the ring and the operand layout are those of prefill attention).
template <int D, int NB>
__global__ __launch_bounds__(256, 2) void tree_attention_kernel(TreeArgs a) {
    constexpr int PAGE_BYTES = D * kPage * 2, IPB = PAGE_BYTES / 1024, NS = kTreeStages, TILE = 64 * NB;
    __shared__ __attribute__((aligned(1024))) unsigned char ring[NS][4][PAGE_BYTES];  // [stage][K0,K1,V0,V1]
    extern __shared__ uint32_t tree_words[];
    const TreeLds tree(tree_words, a.max_nodes);
    const int kvh = blockIdx.x % a.n_kv, g = a.n_q / a.n_kv;
    TreeItem it;
    if (!tree_locate(a, blockIdx.x / a.n_kv, TILE, it, tree.scratch)) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, G = lane >> 4;
    const bool fits = it.n <= a.max_nodes && it.c >= 0 && (int64_t)it.c + it.n <= (int64_t)a.table_stride * kPage;
    const int cols = it.n * g;  // (n <= num_rows, g <= 16: the launcher sees that it fits)

    bf16x8 qf[NB][D / 32];
    int node[NB];
    bool stored[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        const int col = it.tile * TILE + (wave * NB + c) * 16 + r, cc = min(col, cols - 1);
        stored[c] = col < cols;
        node[c] = cc / g;
        const bf16_t* qrow = a.q + (int64_t)(it.row0 + node[c]) * a.ld_q + (int64_t)(kvh * g + cc - node[c] * g) * D;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) qf[c][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + (s * 4 + G) * 8));
    }
    AttnState<D, NB> st;
    init_state<D, NB>(st);
    bool used[NB] = {};
    if (fits) {
        const int nblk = (it.c + it.n + 31) / 32, n_full = it.c / 32, last_page = (it.c + it.n - 1) / kPage;
        const int32_t* bt = a.block_tables + (a.bt_off ? (int64_t)a.bt_off[it.seq] : (int64_t)it.seq * a.table_stride);
        // wave w brings in piece w of a block: K page 0, K page 1, V page 0, V page 1
        const bf16_t* pool = wave < 2 ? a.k_pool : a.v_pool;
        auto page_id = [&](int blk) -> int { return min(max(bt[min(blk * 2 + (wave & 1), last_page)], 0), a.num_blocks - 1); };
        auto issue_block = [&](int64_t page, int stage) {
            const int src_lane = wave == 1 ? lane ^ 4 : lane;  // K page 1 lies four slots shifted, against bank conflicts
            const char* src = reinterpret_cast<const char*>(pool + (page * a.n_kv + kvh) * (int64_t)(D * kPage)) + src_lane * 16;
#pragma unroll
            for (int i = 0; i < IPB; ++i)
                __builtin_amdgcn_global_load_lds((gptr_t)(src + i * 1024), (lptr_t)(&ring[stage][wave][i * 1024]), 16, 0, 0);
        };
        auto block_step = [&](int stage, int blk, auto masked) {
            constexpr bool MASKED = decltype(masked)::value;
            float sc[NB][8];
            u32x4 kf[2][D / 32];
            const int kpage = r >> 3, kslot = ((r >> 2) & 1) * 8 + (r & 3);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int s = 0; s < D / 32; ++s)
                    kf[t][s] = *reinterpret_cast<const u32x4*>(&ring[stage][kpage][((s * 4 + G) * 16 + ((kslot + 4 * t) ^ (4 * kpage))) * 16]);
            uint32_t seen[NB];
#pragma unroll
            for (int c = 0; c < NB; ++c) {
                score_group<D>(sc[c], kf, qf[c]);
                if (MASKED) {
                    seen[c] = tree.vis[node[c] * tree.stride + blk - n_full] >> (G * 8);
#pragma unroll
                    for (int v = 0; v < 8; ++v)
                        if (!(seen[c] >> v & 1)) sc[c][v] = -INFINITY;  // (a column may see nothing of a block: no finite stand-in)
                }
            }
            u32x4 vf[D / 16];
            update_groups<D, NB, true>(
                st, sc, a.scale_log2, []() {},
                [&]() -> const u32x4 (&)[D / 16] {
#pragma unroll
                    for (int b = 0; b < D / 16; ++b) vf[b] = *reinterpret_cast<const u32x4*>(&ring[stage][2 + (G >> 1)][b * 512 + r * 32 + (G & 1) * 16]);
                    if (MASKED) {
                        // values of unused nodes and of slots past the last one may be anything: 0 * NaN is NaN
                        const uint32_t keep = tree.used[blk - n_full] >> (G * 8);
                        uint32_t bad = 0u;
#pragma unroll
                        for (int b = 0; b < D / 16; ++b)
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                vf[b][w] &= (keep >> (2 * w) & 1 ? 0xFFFFu : 0u) | (keep >> (2 * w + 1) & 1 ? 0xFFFF0000u : 0u);
                                bad |= ((vf[b][w] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
                            }
                        if (__any(bad != 0u)) {
                            // a used node's value is not finite: it may reach the columns that see it only.  Its place is
                            // emptied here, and the outputs of the columns that see it become NaN
#pragma unroll
                            for (int b = 0; b < D / 16; ++b) {
                                u32x4 mark;
#pragma unroll
                                for (int w = 0; w < 4; ++w) {
                                    const uint32_t off = ((vf[b][w] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;  // bit 15 or 31 of a bad one
                                    mark[w] = (off >> 15 & 1 ? 0x3F80u : 0u) | (off >> 31 ? 0x3F800000u : 0u);
                                    vf[b][w] &= (off >> 15 & 1 ? 0u : 0xFFFFu) | (off >> 31 ? 0u : 0xFFFF0000u);
                                }
#pragma unroll
                                for (int c = 0; c < NB; ++c) {
                                    u32x4 sees;
#pragma unroll
                                    for (int w = 0; w < 4; ++w)
                                        sees[w] = (seen[c] >> (2 * w) & 1 ? 0x3F80u : 0u) | (seen[c] >> (2 * w + 1) & 1 ? 0x3F800000u : 0u);
                                    const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, mark), __builtin_bit_cast(bf16x8, sees),
                                                                                             f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                                    for (int v = 0; v < 4; ++v)
                                        if (hit[v] > 0.f) st.o[c][b][v] = NAN;
                                }
                            }
                        }
                    }
                    return vf;
                });
        };
        tree_visibility(tree, a.parents + it.row0, it.n, it.c, a.max_nodes);
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            const int at = (it.c & 31) + node[c];
            used[c] = tree.vis[node[c] * tree.stride + (at >> 5)] >> (at & 31) & 1;
        }
        // every wave always issues its piece (indices past the end read the last page again into a stage nobody reads), so the
        // count of outstanding loads is the same in every iteration
#pragma unroll
        for (int i = 0; i < NS - 1; ++i) issue_block(page_id(i), i);
        int pid_next = page_id(NS - 1);
        const bool idle = it.tile * TILE + wave * NB * 16 >= cols;  // (the same for the wave)
        for (int blk = 0; blk < nblk; ++blk) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * IPB) : "memory");
            __syncthreads();  // block blk has landed; nobody reads stage (blk - 1) % NS any more
            issue_block(pid_next, (blk + NS - 1) % NS);
            pid_next = page_id(blk + NS);
            if (idle) continue;
            if (blk < n_full) block_step(blk % NS, blk, std::false_type{});
            else block_step(blk % NS, blk, std::true_type{});
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no LDS fill may outlive the workgroup
    }
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        float l = st.l[c];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (!stored[c]) continue;
        const float inv = 1.0f / l;
        const int col = it.tile * TILE + (wave * NB + c) * 16 + r;
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

}  // namespace

size_t tree_workspace_bytes(int n_q, int n_kv, int d, int max_nodes) {
    (void)n_q; (void)n_kv; (void)d; (void)max_nodes;
    return 256;
}

hipError_t launch_tree_attention(const TreeArgs& a, hipStream_t stream) {
    if (a.num_seqs <= 0 || a.num_rows <= 0) return hipSuccess;
    const int g = a.n_q / a.n_kv;
    // no more tiles than whole ones in all rows and a partly filled one per sequence
    const int64_t items = (int64_t)a.num_rows * g / 64 + a.num_seqs;
    if (items * a.n_kv > INT32_MAX || (int64_t)a.num_rows * g > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(items * a.n_kv));
    const int lds = tree_lds_bytes(a.max_nodes);
    if (a.d == 128) tree_attention_kernel<128, 1><<<grid, 256, lds, stream>>>(a);
    else if (a.d == 64) tree_attention_kernel<64, 1><<<grid, 256, lds, stream>>>(a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}
