// Attention of trees of drafted tokens over the paged cache.
//
// Row i of sequence b (n_b rows, L_b own tokens) sees the P tokens of the prefix, the own tokens before the tree,
// 0 .. L_b - n_b - 1, and the tree's tokens whose bits its mask has:  o = sum_j p_j v_j / sum_j p_j,
// p_j = exp(q . k_j / 8 - m).
//
// A wave a row and head: lane t scores token t of a page, then sums dim t over the page's tokens that are seen.
#include <algorithm>
#include <cmath>

#include "decode_entry.hpp"

namespace ftts {

struct TreeArgs {
    const void* q;
    void* o;
    int64_t q_ld, o_ld;
    const void* kv_base;
    int n_pages, layer, n_head, n_kv_head, max_pages;
    const int32_t* block_table;
    const int32_t* seq_lens;
    const int32_t* row_offsets;
    const uint64_t* masks;
    int mask_words;
    const int32_t* prefix_pages;
    int prefix_len;
    int B, rows;
};

// The tree's tokens j0 .. j0 + 63 that a row sees, of n: bits of its mask (j0 may be negative: tokens before the tree,
// all of them seen).
__device__ __forceinline__ uint64_t tree_bits(const uint64_t* mask, int words, int j0, int n) {
    if (j0 <= -kPage) return ~0ull;
    auto word = [&](int w) { return w >= 0 && w < words ? mask[w] : 0ull; };
    const int w = j0 >> 6, s = j0 & 63;  // (a floor)
    uint64_t bits = word(w) >> s | (s ? word(w + 1) << (64 - s) : 0);
    if (j0 < 0) bits |= (1ull << -j0) - 1;
    const int left = n - j0;
    return left >= 64 ? bits : left <= 0 ? 0 : bits & ((1ull << left) - 1);
}

constexpr int kTreeWaves = 4;
template <bool F32>
__global__ __launch_bounds__(kTreeWaves * 64) void tree_row_kernel(const TreeArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * kTreeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = (int)(id / a.n_head), head = (int)(id % a.n_head), kh = head / (a.n_head / a.n_kv_head);
    if (row >= a.rows) return;
    const int lo = lane < a.B ? a.row_offsets[lane] : 0, hi = lane < a.B ? a.row_offsets[lane + 1] : 0;
    const int first = min(max(lo, 0), a.rows), n_of = min(max(hi, first), a.rows) - first;
    const unsigned long long whose = __ballot(lane < a.B && row >= first && row < first + n_of);
    if (!whose) return;
    const int b = __builtin_ctzll(whose), n = __builtin_amdgcn_readlane(n_of, b), past = a.seq_lens[b] - n;
    const int own = past < 0 ? 0 : (int)min((int64_t)past + n, (int64_t)a.max_pages * kPage);
    const int n_pre = past < 0 ? 0 : (a.prefix_len + kPage - 1) / kPage, pages = n_pre + (own + kPage - 1) / kPage;
    float q[kHeadDim];
#pragma unroll
    for (int d = 0; d < kHeadDim; ++d) q[d] = ld_act<F32>(a.q, (size_t)row * a.q_ld + head * kHeadDim + d);
    float m = -INFINITY, l = 0.f, o = 0.f;
    bool saw = false;
    for (int j = 0; j < pages; ++j) {
        const int k = j - n_pre, phys = k < 0 ? a.prefix_pages[j] : a.block_table[(size_t)b * a.max_pages + k];
        if (phys < 0 || phys >= a.n_pages) continue;
        const int tokens = min(k < 0 ? a.prefix_len - j * kPage : own - k * kPage, kPage);
        uint64_t seen = tokens == kPage ? ~0ull : (1ull << tokens) - 1;
        if (k >= 0) seen &= tree_bits(a.masks + (size_t)row * a.mask_words, a.mask_words, k * kPage - past, n);
        if (!seen) continue;
        saw = true;
        const size_t key = kv_offset(a.layer, a.n_pages, phys, 0, a.n_kv_head, kh, 0), val = key + (size_t)a.n_kv_head * kPage * kHeadDim;
        float s = -INFINITY;
        if (seen >> lane & 1) {
            s = 0.f;
#pragma unroll
            for (int d = 0; d < kHeadDim; ++d) s = fmaf(q[d], ld_act<F32>(a.kv_base, key + lane * kHeadDim + d), s);
            s *= 0.125f;
        }
        const float mn = fmaxf(m, wave_max(s)), ref = mn == -INFINITY ? 0.f : mn, keep = expf(m - ref);
        const float p = seen >> lane & 1 ? expf(s - ref) : 0.f;
        m = mn;
        l = l * keep + wave_sum(p);
        o *= keep;
        for (uint64_t x = seen; x; x &= x - 1) {
            const int t = __builtin_ctzll(x);
            o = fmaf(__shfl(p, t, kWave), ld_act<F32>(a.kv_base, val + t * kHeadDim + lane), o);
        }
    }
    // where nothing is seen 0, where every score is -inf NaN
    st_act<F32>(a.o, (size_t)row * a.o_ld + head * kHeadDim + lane, saw ? o / l : 0.f);
}

static hipError_t launch_tree_attention(int dtype, const TreeArgs& a, hipStream_t st) {
    const dim3 g((unsigned)(((int64_t)a.rows * a.n_head + kTreeWaves - 1) / kTreeWaves)), t(kTreeWaves * 64);
    (void)hipGetLastError();
    if (dtype == FTTS_F32) hipLaunchKernelGGL(tree_row_kernel<true>, g, t, 0, st, a);
    else hipLaunchKernelGGL(tree_row_kernel<false>, g, t, 0, st, a);
    return hipGetLastError();
}

static size_t tree_attention_bytes() { return 256; }

}  // namespace ftts

using namespace ftts;

namespace {

int check_shape(const ftts_attn_shape* s, int B, int n_rows, int prefix_len, int max_pages) {
    if (!s) return set_error(FTTS_E_INVALID_ARG, "tree_attention: shape is NULL");
    if (s->dtype != FTTS_F32 && s->dtype != FTTS_BF16)
        return set_error(FTTS_E_DTYPE, "tree_attention: dtype must be FTTS_F32 or FTTS_BF16");
    if (s->d_head != kHeadDim) return set_error(FTTS_E_UNSUPPORTED, "tree_attention: d_head must be 64 (got %d)", s->d_head);
    if (s->n_head < 1 || s->n_head > 256 || s->n_kv_head < 1 || s->n_head % s->n_kv_head)
        return set_error(FTTS_E_SHAPE, "tree_attention: n_head must be in [1, 256] and a multiple of n_kv_head");
    if (B < 1 || B > FTTS_MAX_BATCH) return set_error(FTTS_E_SHAPE, "tree_attention: B must be in [1, %d]", FTTS_MAX_BATCH);
    if (n_rows < 0 || n_rows > (1 << 24) || (int64_t)n_rows * s->n_head > 0x7FFFFFFF)
        return set_error(FTTS_E_RANGE, "tree_attention: n_rows must be in [0, 2^24] and n_rows * n_head below 2^31");
    if (prefix_len < 0 || prefix_len > FTTS_MAX_SHARED_PREFIX)
        return set_error(FTTS_E_RANGE, "tree_attention: prefix length must be in [0, %d]", FTTS_MAX_SHARED_PREFIX);
    if (max_pages < 1 || max_pages > kMaxPages)
        return set_error(FTTS_E_SHAPE, "tree_attention: max_pages must be in [1, %d]", kMaxPages);
    return FTTS_OK;
}

}  // namespace

extern "C" {

size_t ftts_tree_attention_workspace_bytes(const ftts_attn_shape* shape, int32_t B, int32_t n_rows, int32_t prefix_len,
                                           int32_t max_pages) {
    if (check_shape(shape, B, n_rows, prefix_len, max_pages) != FTTS_OK) return 0;
    return tree_attention_bytes();
}

int ftts_tree_attention(const ftts_attn_shape* shape, const void* q, int64_t q_stride, const int32_t* row_offsets,
                        int32_t n_rows, int32_t B, const int64_t* masks, int32_t mask_words,
                        const ftts_shared_prefix* prefix, const ftts_page_table* pt, const ftts_kv_pool* kv, int32_t layer,
                        void* out, int64_t out_stride, void* ws, size_t ws_bytes, void* stream) {
    const int P = prefix ? prefix->len : 0;
    if (!pt) return set_error(FTTS_E_INVALID_ARG, "tree_attention: page table is NULL");
    if (int rc = check_shape(shape, B, n_rows, P, pt->max_pages)) return rc;
    if (!kv || !kv->base) return set_error(FTTS_E_INVALID_ARG, "tree_attention: pool is NULL");
    if (!pt->block_table || !pt->seq_lens) return set_error(FTTS_E_INVALID_ARG, "tree_attention: block_table/seq_lens is NULL");
    if (kv->n_pages < 1 || layer < 0) return set_error(FTTS_E_SHAPE, "tree_attention: n_pages must be >= 1 and layer >= 0");
    if (P > 0 && !prefix->pages) return set_error(FTTS_E_INVALID_ARG, "tree_attention: prefix pages is NULL");
    if (mask_words < 1 || mask_words > FTTS_MAX_TREE / 64)
        return set_error(FTTS_E_SHAPE, "tree_attention: mask_words must be in [1, %d]", FTTS_MAX_TREE / 64);
    if (!row_offsets) return set_error(FTTS_E_INVALID_ARG, "tree_attention: row_offsets is NULL");
    if (n_rows == 0) return FTTS_OK;
    if (!q || !out || !masks) return set_error(FTTS_E_INVALID_ARG, "tree_attention: q/out/masks is NULL");
    if (reinterpret_cast<uintptr_t>(masks) & 7u) return set_error(FTTS_E_ALIGN, "tree_attention: masks not 8-byte aligned");
    const int64_t piece = shape->dtype == FTTS_F32 ? 4 : 8;  // elements in 16 bytes
    for (const int64_t st : {q_stride, out_stride})
        if (st < 64LL * shape->n_head || st > (1LL << 31) || st % piece)
            return set_error(FTTS_E_SHAPE, "tree_attention: a stride must be a multiple of %d, at least 64 * n_head", (int)piece);
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(kv->base)) & 15u)
        return set_error(FTTS_E_ALIGN, "tree_attention: q, out and the pool must be 16-byte aligned");
    if (!ws) return set_error(FTTS_E_INVALID_ARG, "tree_attention: workspace is NULL");
    if (reinterpret_cast<uintptr_t>(ws) & 15u) return set_error(FTTS_E_ALIGN, "tree_attention: workspace is not 16-byte aligned");
    const size_t need = ftts_tree_attention_workspace_bytes(shape, B, n_rows, P, pt->max_pages);
    if (ws_bytes < need) return set_error(FTTS_E_WORKSPACE, "tree_attention: workspace too small: %zu < %zu", ws_bytes, need);
    TreeArgs a{};
    a.q = q;
    a.o = out;
    a.q_ld = q_stride;
    a.o_ld = out_stride;
    a.kv_base = kv->base;
    a.n_pages = kv->n_pages;
    a.layer = layer;
    a.n_head = shape->n_head;
    a.n_kv_head = shape->n_kv_head;
    a.max_pages = pt->max_pages;
    a.block_table = pt->block_table;
    a.seq_lens = pt->seq_lens;
    a.row_offsets = row_offsets;
    a.masks = reinterpret_cast<const uint64_t*>(masks);
    a.mask_words = mask_words;
    a.prefix_pages = P > 0 ? prefix->pages : nullptr;
    a.prefix_len = P;
    a.B = B;
    a.rows = n_rows;
    const hipError_t e = launch_tree_attention(shape->dtype, a, (hipStream_t)stream);
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "tree_attention launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

}  // extern "C"
