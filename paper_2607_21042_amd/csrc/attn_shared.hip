// Attention of a batch of sequences that continue one shared prefix, over the paged cache.
//
// Row i of sequence b (n_b rows, L_b own tokens) sees the P tokens of the prefix and own tokens
// 0 .. L_b - n_b + i:  o = sum_j p_j v_j / sum_j p_j,  p_j = exp(q . k_j / 8 - m).
//
// One wave per row and query head walks the pages of the prefix and then the sequence's own with
// a running maximum and sum: lane j scores token j of a page, and lane d then sums dimension d
// over the tokens that the row sees (the others are not read).
#include "decode_entry.hpp"

namespace ftts {

constexpr int kSaWaves = 4;

template <bool F32>
__global__ __launch_bounds__(kSaWaves * 64) void shared_row_kernel(const SharedAttnArgs a) {
    const int64_t id = (int64_t)blockIdx.x * kSaWaves + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (id >= (int64_t)a.rows * a.n_head) return;
    const int r = (int)(id / a.n_head), h = (int)(id % a.n_head), kh = h / (a.n_head / a.n_kv_head);
    int b = r, i = 0, n = 1;
    if (a.row_offsets) {
        if (r < a.row_offsets[0] || r >= a.row_offsets[a.B]) return;
        int lo = 0, hi = a.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.row_offsets[mid] <= r) lo = mid;
            else hi = mid - 1;
        }
        b = lo;
        i = r - a.row_offsets[b];
        n = a.row_offsets[b + 1] - a.row_offsets[b];
    }
    const int len = a.seq_lens[b];
    const int own = len < 0 ? 0 : (int)min((int64_t)len - n + i + 1, (int64_t)a.max_pages * kPage);
    const float q = ld_act<F32>(a.q, (size_t)r * a.q_ld + h * kHeadDim + lane) * 0.125f;
    float m = -INFINITY, l = 0.f, o = 0.f;
    auto page = [&](int phys, int seen) {  // the first `seen` tokens of a page
        if (phys < 0 || phys >= a.n_pages) return;
        const size_t kb = kv_offset(a.layer, a.n_pages, phys, 0, a.n_kv_head, kh, 0);
        const size_t vb = kv_offset(a.layer, a.n_pages, phys, 1, a.n_kv_head, kh, 0);
        float s = 0.f;
        for (int d = 0; d < kHeadDim; ++d) {
            const float qd = __shfl(q, d, kWave);
            if (lane < seen) s = fmaf(qd, ld_act<F32>(a.kv_base, kb + lane * kHeadDim + d), s);
        }
        if (lane >= seen) s = -INFINITY;
        const float mn = fmaxf(m, wave_max(s));
        const float ref = mn == -INFINITY ? 0.f : mn;
        const float f = expf(m - ref), p = expf(s - ref);
        m = mn;
        l = l * f + wave_sum(p);
        o *= f;
        for (int j = 0; j < seen; ++j) o = fmaf(__shfl(p, j, kWave), ld_act<F32>(a.kv_base, vb + j * kHeadDim + lane), o);
    };
    if (len >= 0)
        for (int t = 0; t < a.prefix_len; t += kPage) page(a.prefix_pages[t / kPage], min(kPage, a.prefix_len - t));
    for (int t = 0; t < own; t += kPage) page(a.block_table[(size_t)b * a.max_pages + t / kPage], min(kPage, own - t));
    st_act<F32>(a.o, (size_t)r * a.o_ld + h * kHeadDim + lane, l == 0.f ? 0.f : o / l);
}

hipError_t launch_shared_attention(int dtype, const SharedAttnArgs& a, hipStream_t st) {
    const dim3 g((unsigned)(((int64_t)a.rows * a.n_head + kSaWaves - 1) / kSaWaves)), t(kSaWaves * 64);
    if (dtype == FTTS_F32) hipLaunchKernelGGL(shared_row_kernel<true>, g, t, 0, st, a);
    else hipLaunchKernelGGL(shared_row_kernel<false>, g, t, 0, st, a);
    return hipGetLastError();
}

}  // namespace ftts

using namespace ftts;

namespace {

int check_shape(const ftts_attn_shape* s, int B, int n_rows, int prefix_len, int max_pages) {
    if (!s) return set_error(FTTS_E_INVALID_ARG, "shared_attention: shape is NULL");
    if (s->dtype != FTTS_F32 && s->dtype != FTTS_BF16)
        return set_error(FTTS_E_DTYPE, "shared_attention: dtype must be FTTS_F32 or FTTS_BF16");
    if (s->d_head != kHeadDim) return set_error(FTTS_E_UNSUPPORTED, "shared_attention: d_head must be 64 (got %d)", s->d_head);
    if (s->n_head < 1 || s->n_head > 256 || s->n_kv_head < 1 || s->n_head % s->n_kv_head)
        return set_error(FTTS_E_SHAPE, "shared_attention: n_head must be in [1, 256] and a multiple of n_kv_head");
    if (B < 1 || B > FTTS_MAX_BATCH) return set_error(FTTS_E_SHAPE, "shared_attention: B must be in [1, %d]", FTTS_MAX_BATCH);
    if (n_rows < 0 || n_rows > (1 << 24)) return set_error(FTTS_E_RANGE, "shared_attention: n_rows must be in [0, 2^24]");
    if (prefix_len < 0 || prefix_len > FTTS_MAX_SHARED_PREFIX)
        return set_error(FTTS_E_RANGE, "shared_attention: prefix length must be in [0, %d]", FTTS_MAX_SHARED_PREFIX);
    if (max_pages < 1 || max_pages > kMaxPages)
        return set_error(FTTS_E_SHAPE, "shared_attention: max_pages must be in [1, %d]", kMaxPages);
    return FTTS_OK;
}

}  // namespace

extern "C" {

size_t ftts_shared_attention_workspace_bytes(const ftts_attn_shape* shape, int32_t B, int32_t n_rows,
                                             int32_t prefix_len, int32_t max_pages) {
    if (check_shape(shape, B, n_rows, prefix_len, max_pages) != FTTS_OK) return 0;
    return 256;
}

int ftts_shared_attention(const ftts_attn_shape* shape, const void* q, int64_t q_stride, const int32_t* row_offsets,
                          int32_t n_rows, int32_t B, const ftts_shared_prefix* prefix, const ftts_page_table* pt,
                          const ftts_kv_pool* kv, int32_t layer, void* out, int64_t out_stride, void* ws,
                          size_t ws_bytes, void* stream) {
    const int P = prefix ? prefix->len : 0;
    if (!pt) return set_error(FTTS_E_INVALID_ARG, "shared_attention: page table is NULL");
    if (int rc = check_shape(shape, B, n_rows, P, pt->max_pages)) return rc;
    if (!kv || !kv->base) return set_error(FTTS_E_INVALID_ARG, "shared_attention: pool is NULL");
    if (!pt->block_table || !pt->seq_lens) return set_error(FTTS_E_INVALID_ARG, "shared_attention: block_table/seq_lens is NULL");
    if (kv->n_pages < 1 || layer < 0) return set_error(FTTS_E_SHAPE, "shared_attention: n_pages must be >= 1 and layer >= 0");
    if (P > 0 && !prefix->pages) return set_error(FTTS_E_INVALID_ARG, "shared_attention: prefix pages is NULL");
    if (!row_offsets && n_rows != B) return set_error(FTTS_E_SHAPE, "shared_attention: n_rows must be B without row_offsets");
    if (n_rows == 0) return FTTS_OK;
    if (!q || !out) return set_error(FTTS_E_INVALID_ARG, "shared_attention: q/out is NULL");
    const int64_t piece = shape->dtype == FTTS_F32 ? 4 : 8;  // elements in 16 bytes
    for (const int64_t st : {q_stride, out_stride})
        if (st < 64LL * shape->n_head || st > (1LL << 31) || st % piece)
            return set_error(FTTS_E_SHAPE, "shared_attention: a stride must be a multiple of %d, at least 64 * n_head", (int)piece);
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(kv->base)) & 15u)
        return set_error(FTTS_E_ALIGN, "shared_attention: q, out and the pool must be 16-byte aligned");
    if (!ws) return set_error(FTTS_E_INVALID_ARG, "shared_attention: workspace is NULL");
    if (reinterpret_cast<uintptr_t>(ws) & 15u) return set_error(FTTS_E_ALIGN, "shared_attention: workspace is not 16-byte aligned");
    const size_t need = ftts_shared_attention_workspace_bytes(shape, B, n_rows, P, pt->max_pages);
    if (ws_bytes < need) return set_error(FTTS_E_WORKSPACE, "shared_attention: workspace too small: %zu < %zu", ws_bytes, need);
    SharedAttnArgs a{};
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
    a.prefix_pages = P > 0 ? prefix->pages : nullptr;
    a.prefix_len = P;
    a.B = B;
    a.rows = n_rows;
    (void)hipGetLastError();
    const hipError_t e = launch_shared_attention(shape->dtype, a, (hipStream_t)stream);
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "shared_attention launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

}  // extern "C"
