// The commit of a drafted tree's accepted path: which tokens the model's choices keep, and their keys' and values' way
// to the places behind the cached tokens, in every layer.
//
// The path is a chain of dependent looks at the tree, the rows are copies.  A workgroup reads its sequence's tree once, a
// token a thread, and each of its waves walks the path for itself (four tokens a lane, a step compares all at once), so
// nothing passes between workgroups and one launch does both.  A wave then moves its share of the (layer, keys or values,
// head) blocks, four in flight: a kept token's 64 columns lie in one block at its old and its new place, and the i-th goes
// to place i of the tree, which is never behind the old one and never a later one's, so whole groups read in ascending
// order and then written lose nothing.
//
// Captured: one sequence, 4 of 16 tokens kept in 24 layers of 20 heads, 3.8 us (2.5 without a move), 16 sequences that
// keep 1 to 8 8.0 us: rows of 128 bytes, 17 MB.  A thousand waves that each read the tree from memory took 16 us for it.
#include <algorithm>

#include "decode_entry.hpp"

namespace ftts {

constexpr int kTcWaves = 4, kTcNodes = FTTS_MAX_TREE / kWave;  // tokens of the tree a lane holds
constexpr int kTcWide = 512;   // workgroups that fill the card: from there on a wave takes more blocks
constexpr int kTcAhead = 4;    // blocks that a wave has in flight

struct CommitArgs {
    const int32_t *tokens, *parents, *choices, *row_offsets;
    int rows, B;
    const int32_t *block_table, *seq_lens;
    int max_pages, n_pages, n_layer, n_kv_head;
    char* base;
    int32_t *path, *counts, *next_tokens, *new_lens;
    int max_path;
    int groups;  // workgroups of a sequence
};

// COLS: bytes of a token's columns in a block (64 of 2 or 4).
template <int COLS>
__global__ __launch_bounds__(kTcWaves * 64) void tree_commit_kernel(const CommitArgs a) {
    static_assert(kTcWaves * kWave == FTTS_MAX_TREE, "a thread a token of the tree");
    __shared__ int3 s_node[FTTS_MAX_TREE];            // token, parent, choice
    __shared__ int s_path[kTcWaves][FTTS_MAX_TREE];   // a wave's own copy
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / a.groups, mine = blockIdx.x % a.groups * kTcWaves + wave, waves = a.groups * kTcWaves;
    const int r0 = min(max(a.row_offsets[b], 0), a.rows), all = min(max(a.row_offsets[b + 1], r0), a.rows) - r0;
    const int n = min(all, FTTS_MAX_TREE), len = a.seq_lens[b];
    const int past = len < all ? -1 : len - all;  // (compared first: a length may be -2^31)
    if ((int)threadIdx.x < n) {
        const int r = r0 + threadIdx.x;
        s_node[threadIdx.x] = make_int3(a.tokens[r], a.parents[r], a.choices[r]);
    }
    __syncthreads();
    int* path = s_path[wave];
    int kept = 0, next = -1;
    if (n > 0 && past >= 0) {
        int token[kTcNodes], parent[kTcNodes];  // of tokens 64 k + lane
#pragma unroll
        for (int k = 0; k < kTcNodes; ++k) {
            const int j = k * kWave + lane;
            const int3 x = s_node[j];  // (behind the tree's end: whatever is there, under a parent that is none)
            token[k] = x.x;
            parent[k] = j < n ? x.y : -1;
        }
        for (int cur = 0; cur >= 0;) {
            if (lane == 0) path[kept] = cur;
            ++kept;
            next = __builtin_amdgcn_readfirstlane(s_node[cur].z);
            int child = -1;
#pragma unroll
            for (int k = kTcNodes - 1; k >= 0; --k) {
                const unsigned long long hit = __ballot(parent[k] == cur && token[k] == next && k * kWave + lane > cur);
                if (hit) child = k * kWave + __builtin_ctzll(hit);
            }
            cur = kept < a.max_path && next >= 0 ? child : -1;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (mine == 0) {
        for (int i = lane; i < a.max_path; i += kWave) a.path[(size_t)b * a.max_path + i] = i < kept ? path[i] : -1;
        if (lane == 0) {
            a.counts[b] = kept;
            a.next_tokens[b] = next;
            a.new_lens[b] = kept > 0 ? past + kept : len;
        }
    }
    // lane (i, piece): the group's i-th token, 16 bytes of its columns
    constexpr int kLanes = COLS / 16, kRows = kWave / kLanes;
    const int heads2 = 2 * a.n_kv_head, blocks = a.n_layer * heads2;
    const size_t page_bytes = (size_t)kPage * COLS, layer_bytes = (size_t)a.n_pages * heads2 * page_bytes;
    auto place = [&](int64_t t, int64_t& at) {  // of own token t in a (layer 0, keys, head 0) block
        const int64_t page = t / kPage;
        const int phys = page < a.max_pages ? a.block_table[(size_t)b * a.max_pages + page] : -1;
        at = (int64_t)phys * heads2 * page_bytes + (t % kPage) * COLS;
        return phys >= 0 && phys < a.n_pages;
    };
    for (int i0 = 0; i0 < kept; i0 += kRows) {
        const int i = i0 + lane / kLanes, from = i < kept ? path[i] : i;
        if (!__any(from != i)) continue;
        int64_t src = 0, dst = 0;
        // (in 64 bits: lanes behind the path look past a length that may be 2^31 - 1)
        const bool there = place((int64_t)past + from, src), move = place((int64_t)past + i, dst) && there && from != i;
        src += lane % kLanes * 16;
        dst += lane % kLanes * 16;
        for (int u0 = mine; u0 < blocks; u0 += kTcAhead * waves) {
            // (every lane's rows are in before one is written over; past the last block the last one is moved again, alike)
            u32x4_t x[kTcAhead];
            char* at[kTcAhead];
#pragma unroll
            for (int k = 0; k < kTcAhead; ++k) {
                const uint32_t u = u0 + k * waves < blocks ? u0 + k * waves : u0;
                at[k] = a.base + u / (uint32_t)heads2 * layer_bytes + u % (uint32_t)heads2 * page_bytes;
            }
            if (move) {
#pragma unroll
                for (int k = 0; k < kTcAhead; ++k) x[k] = *reinterpret_cast<const u32x4_t*>(at[k] + src);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
                for (int k = 0; k < kTcAhead; ++k) *reinterpret_cast<u32x4_t*>(at[k] + dst) = x[k];
            }
        }
    }
}

}  // namespace ftts

using namespace ftts;

extern "C" int ftts_tree_commit(const int32_t* tokens, const int32_t* parents, const int32_t* choices,
                                const int32_t* row_offsets, int32_t n_rows, int32_t B, const ftts_page_table* pt,
                                const ftts_kv_pool* kv, int32_t kv_dtype, int32_t n_layer, int32_t n_kv_head, int32_t* path,
                                int32_t max_path, int32_t* counts, int32_t* next_tokens, int32_t* new_lens, void* stream) {
    if (kv_dtype != FTTS_F32 && kv_dtype != FTTS_BF16) return set_error(FTTS_E_DTYPE, "tree_commit: kv_dtype must be FTTS_F32 or FTTS_BF16");
    if (!pt || !pt->block_table || !pt->seq_lens) return set_error(FTTS_E_INVALID_ARG, "tree_commit: page table is NULL");
    if (!kv || !kv->base) return set_error(FTTS_E_INVALID_ARG, "tree_commit: pool is NULL");
    if (B < 1 || B > FTTS_MAX_BATCH) return set_error(FTTS_E_SHAPE, "tree_commit: B must be in [1, %d]", FTTS_MAX_BATCH);
    if (n_rows < 0 || n_rows > (1 << 24)) return set_error(FTTS_E_RANGE, "tree_commit: n_rows must be in [0, 2^24]");
    if (pt->max_pages < 1 || pt->max_pages > kMaxPages)
        return set_error(FTTS_E_SHAPE, "tree_commit: max_pages must be in [1, %d]", kMaxPages);
    if (kv->n_pages < 1 || n_layer < 1 || n_kv_head < 1 || n_kv_head > 256 || (int64_t)n_layer * n_kv_head > (1 << 16))
        return set_error(FTTS_E_SHAPE, "tree_commit: bad pool dimensions");
    if (max_path < 1 || max_path > FTTS_MAX_TREE) return set_error(FTTS_E_SHAPE, "tree_commit: max_path must be in [1, %d]", FTTS_MAX_TREE);
    if (!row_offsets || !path || !counts || !next_tokens || !new_lens) return set_error(FTTS_E_INVALID_ARG, "tree_commit: NULL pointer");
    if (n_rows > 0 && (!tokens || !parents || !choices)) return set_error(FTTS_E_INVALID_ARG, "tree_commit: tokens/parents/choices is NULL");
    if (reinterpret_cast<uintptr_t>(kv->base) & 15u) return set_error(FTTS_E_ALIGN, "tree_commit: pool is not 16-byte aligned");
    const size_t nb = 4u * (size_t)B, nr = 4u * (size_t)n_rows;
    const int cols = kv_dtype == FTTS_F32 ? 256 : 128;
    const size_t pool = (size_t)n_layer * kv->n_pages * 2 * n_kv_head * kPage * cols;
    const struct { const void* p; size_t n; } in[] = {{tokens, nr}, {parents, nr}, {choices, nr}, {row_offsets, nb + 4},
                                                      {pt->block_table, nb * pt->max_pages}, {pt->seq_lens, nb}},
        out[] = {{path, nb * max_path}, {counts, nb}, {next_tokens, nb}, {new_lens, nb}, {kv->base, pool}};
    auto overlap = [](const void* x, size_t nx, const void* y, size_t ny) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
        return x && y && nx && ny && p < q + ny && q < p + nx;
    };
    for (int i = 0; i < 5; ++i) {
        if (reinterpret_cast<uintptr_t>(out[i].p) & 3u) return set_error(FTTS_E_ALIGN, "tree_commit: output not 4-byte aligned");
        for (const auto& x : in)
            if (overlap(out[i].p, out[i].n, x.p, x.n)) return set_error(FTTS_E_INVALID_ARG, "tree_commit: an output overlaps an input");
        for (int j = 0; j < i; ++j)
            if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return set_error(FTTS_E_INVALID_ARG, "tree_commit: two outputs overlap");
    }
    for (const auto& x : in)
        if (reinterpret_cast<uintptr_t>(x.p) & 3u) return set_error(FTTS_E_ALIGN, "tree_commit: input not 4-byte aligned");
    const int blocks = n_layer * 2 * n_kv_head;
    CommitArgs a{tokens, parents, choices, row_offsets, n_rows, B, pt->block_table, pt->seq_lens, pt->max_pages, kv->n_pages,
                 n_layer, n_kv_head, reinterpret_cast<char*>(kv->base), path, counts, next_tokens, new_lens, max_path, 0};
    a.groups = std::min((blocks + kTcWaves * kTcAhead - 1) / (kTcWaves * kTcAhead), std::max(kTcWide / B, 1));
    const dim3 g((unsigned)(a.groups * B)), t(kTcWaves * 64);
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    if (kv_dtype == FTTS_F32) hipLaunchKernelGGL(tree_commit_kernel<256>, g, t, 0, st, a);
    else hipLaunchKernelGGL(tree_commit_kernel<128>, g, t, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "tree_commit launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}
