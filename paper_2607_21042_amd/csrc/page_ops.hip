// Block tables and slot maps from request lengths, and the write of new keys and values into
// their pages by slot.
#include <algorithm>

#include "decode_entry.hpp"

namespace ftts {

// ---- tables ---------------------------------------------------------------------------------
// A request's share of the free pages and of the packed rows is a prefix sum over the requests
// before it, at most 1024 of them: every workgroup does that scan for itself, one request a
// thread, and then fills its part of the table and of the slot map, so one launch serves both
// and nothing passes between workgroups.  A run of four rows finds its request by bisecting the row offsets in
// LDS, and its page from the kept entries or from the free list directly (never from the entries
// that another workgroup is writing).
//
// Small calls are latency, so they take one element a thread and, up to 256 requests, 256 threads a workgroup; from
// kTabWide elements on a thread fills four, with one division or bisection for them, one page lookup where they
// share it, and one store where they start on 16 bytes.  Traced: one request of 256 tokens 2.9 us, a step of 48
// requests 3.6, 1024 requests of 753,857 tokens in all 11 (two dependent trips to memory and the scan; 3.3 MB).
constexpr int kTabThreads = 1024, kTabWide = 1 << 16;

struct TableArgs {
    const int32_t *cached, *added, *free_pages;
    int B, n_free, n_pages, max_pages, max_rows;
    int32_t *table, *row_offsets, *seq_lens, *slots, *counts;
};

template <typename T>
__device__ __forceinline__ T scan_wave(T v, int lane) {  // inclusive
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const T u = __shfl_up(v, d, kWave);
        if (lane >= d) v += u;
    }
    return v;
}

template <int PER>
__global__ __launch_bounds__(kTabThreads) void build_tables_kernel(const TableArgs a) {
    __shared__ int64_t w_rows[kTabThreads / kWave];
    __shared__ int w_take[kTabThreads / kWave], s_refused, s_taken;
    __shared__ int s_row[kTabThreads + 1];   // first row of each request, and behind the last
    __shared__ int s_first[kTabThreads];     // index in the free list of its first new page, or -1: refused
    __shared__ int s_cached[kTabThreads], s_has[kTabThreads], s_need[kTabThreads];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int cached = t < a.B && a.cached ? a.cached[t] : 0, added = t < a.B ? a.added[t] : 0;
    if (t == 0) s_refused = s_taken = 0;
    const int64_t end = (int64_t)cached + added, most = (int64_t)a.max_pages * kPage;
    const bool fits = cached >= 0 && added >= 0 && end <= most;
    const int has = (int)((min((int64_t)max(cached, 0), most) + kPage - 1) / kPage);
    const int need = fits ? (int)((end + kPage - 1) / kPage) : has;
    int64_t rows = scan_wave((int64_t)max(added, 0), lane);
    int take = scan_wave(need - has, lane);
    if (lane == 63) {
        w_rows[w] = rows;
        w_take[w] = take;
    }
    __syncthreads();
    for (int i = 0; i < w; ++i) {
        rows += w_rows[i];
        take += w_take[i];
    }
    const bool ok = fits && (need == has || take <= a.n_free);
    const int top = (int)min(rows, (int64_t)0x7FFFFFFF);
    s_row[t + 1] = top;
    if (t == 0) s_row[0] = 0;
    s_first[t] = ok ? take - (need - has) : -1;
    s_cached[t] = cached;
    s_has[t] = has;
    s_need[t] = ok ? need : has;
    if (t < a.B && !ok) atomicAdd(&s_refused, 1);
    if (ok && need > has) atomicMax(&s_taken, take);  // (the accepted ones' ends ascend)
    __syncthreads();
    if (blockIdx.x == 0) {
        if (t < a.B) {
            a.row_offsets[t + 1] = top;
            if (a.seq_lens) a.seq_lens[t] = ok ? (int)end : max(cached, 0);
        }
        if (t == 0) {
            a.row_offsets[0] = 0;
            a.counts[0] = s_taken;
            a.counts[1] = s_refused;
        }
    }
    // (cells stay below 2^20, rows at 2^24, a step at 2^20)
    const uint32_t step = gridDim.x * blockDim.x * PER, i0 = (blockIdx.x * blockDim.x + t) * PER;
    const uint32_t cells = (uint32_t)a.B * a.max_pages, max_rows = a.max_rows;
    for (uint32_t i = i0; i < cells; i += step) {
        int b = i / (uint32_t)a.max_pages, p = i - b * a.max_pages;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (i + k >= cells) break;
            const int kept = s_has[b];
            if (p >= kept) a.table[i + k] = p < s_need[b] ? a.free_pages[s_first[b] + p - kept] : -1;
            if (++p == a.max_pages) p = 0, ++b;
        }
    }
    const bool whole = PER == 4 && (reinterpret_cast<uintptr_t>(a.slots) & 15u) == 0;
    for (uint32_t r0 = i0; r0 < max_rows; r0 += step) {
        int slot[PER], lo = 0, hi = a.B - 1;  // the last request that begins at or before r0
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_row[mid] <= (int)r0) lo = mid;
            else hi = mid - 1;
        }
        int at_lo = -1, at_page = -1, phys = -1;  // the page last looked up
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r = (int)r0 + k;
            slot[k] = -1;
            while (lo < a.B && s_row[lo + 1] <= r) ++lo;  // (past empty ones; B: behind the last)
            if (lo < a.B && s_first[lo] >= 0) {
                const int tok = s_cached[lo] + r - s_row[lo], page = tok / kPage, kept = s_has[lo];
                if (lo != at_lo || page != at_page) {
                    phys = page < kept ? a.table[(size_t)lo * a.max_pages + page] : a.free_pages[s_first[lo] + page - kept];
                    at_lo = lo;
                    at_page = page;
                }
                if (phys >= 0 && phys < a.n_pages) slot[k] = phys * kPage + tok % kPage;
            }
        }
        if (whole && r0 + PER <= max_rows) {
            *reinterpret_cast<int4*>(a.slots + r0) = make_int4(slot[0], slot[PER > 1 ? 1 : 0], slot[PER > 2 ? 2 : 0], slot[PER > 3 ? 3 : 0]);
        } else {
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (r0 + k < max_rows) a.slots[r0 + k] = slot[k];
        }
    }
}

// ---- append ----------------------------------------------------------------------------------
// One wave a row: lane j moves pieces j, j + 64, ... of 8 elements, keys' before values'.  Bound by memory: 10,827 rows
// of 20 heads 22 us, 5.0 TB/s (what a copy of 1 GiB reaches); 32 rows 3.4 us, a launch and two trips.
constexpr int kAppWaves = 4;

struct AppendArgs {
    const void *k, *v;
    int64_t k_ld, v_ld;
    int rows, n_pages, layer, n_head;
    const int32_t* slots;
    void* base;
};

template <bool SRC32, bool DST32>
__global__ __launch_bounds__(kAppWaves * 64) void append_kv_kernel(const AppendArgs a) {
    const int r = blockIdx.x * kAppWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (r >= a.rows) return;
    const int slot = a.slots[r];
    if (slot < 0 || slot / kPage >= a.n_pages) return;
    const int half = 8 * a.n_head;  // pieces of a row's keys
    for (int j = lane; j < 2 * half; j += kWave) {
        const int kv = j >= half, p = j - kv * half;
        const size_t src = (size_t)r * (kv ? a.v_ld : a.k_ld) + 8 * p;
        const void* from = kv ? a.v : a.k;
        const size_t dst = kv_offset(a.layer, a.n_pages, slot / kPage, kv, a.n_head, p >> 3, slot % kPage) + 8 * (p & 7);
        if constexpr (SRC32) {
            const float4* s = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(from) + src);
            const float4 x = s[0], y = s[1];
            if constexpr (DST32) {
                float4* d = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.base) + dst);
                d[0] = x;
                d[1] = y;
            } else {
                auto pair = [](float lo, float hi) { return (uint32_t)f32_to_bf16(lo) | ((uint32_t)f32_to_bf16(hi) << 16); };
                *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.base) + dst) =
                    make_uint4(pair(x.x, x.y), pair(x.z, x.w), pair(y.x, y.y), pair(y.z, y.w));
            }
        } else {
            *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.base) + dst) =
                *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(from) + src);
        }
    }
}

}  // namespace ftts

using namespace ftts;

namespace {

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && na && nb && x < y + nb && y < x + na;
}

}  // namespace

extern "C" {

int ftts_build_tables(const int32_t* cached, const int32_t* added, int32_t B, const int32_t* free_pages,
                      int32_t n_free, int32_t n_pages, int32_t* block_table, int32_t max_pages, int32_t* row_offsets,
                      int32_t* seq_lens, int32_t* slots, int32_t max_rows, int32_t* counts, void* stream) {
    if (!added || !block_table || !row_offsets || !counts) return set_error(FTTS_E_INVALID_ARG, "build_tables: NULL pointer");
    if (B < 1 || B > FTTS_MAX_TABLE_BATCH)
        return set_error(FTTS_E_SHAPE, "build_tables: B must be in [1, %d]", FTTS_MAX_TABLE_BATCH);
    if (max_pages < 1 || max_pages > kMaxPages)
        return set_error(FTTS_E_SHAPE, "build_tables: max_pages must be in [1, %d]", kMaxPages);
    if (n_pages < 1 || n_pages > (1 << 25) - 1) return set_error(FTTS_E_SHAPE, "build_tables: n_pages must be in [1, 2^25)");
    if (n_free < 0 || (n_free > 0 && !free_pages)) return set_error(FTTS_E_INVALID_ARG, "build_tables: bad free_pages");
    if (max_rows < 0 || max_rows > (1 << 24)) return set_error(FTTS_E_RANGE, "build_tables: max_rows must be in [0, 2^24]");
    if (max_rows > 0 && !slots) return set_error(FTTS_E_INVALID_ARG, "build_tables: slots is NULL");
    const struct { const void* p; size_t n; } in[] = {{cached, 4u * (size_t)B}, {added, 4u * (size_t)B}, {free_pages, 4u * (size_t)n_free}},
        out[] = {{block_table, 4u * (size_t)B * max_pages}, {row_offsets, 4u * ((size_t)B + 1)}, {seq_lens, 4u * (size_t)B},
                 {slots, 4u * (size_t)max_rows}, {counts, 8}};
    for (int i = 0; i < 5; ++i) {
        if (reinterpret_cast<uintptr_t>(out[i].p) & 3u) return set_error(FTTS_E_ALIGN, "build_tables: output not 4-byte aligned");
        for (const auto& x : in)
            if (overlap(out[i].p, out[i].n, x.p, x.n)) return set_error(FTTS_E_INVALID_ARG, "build_tables: an output overlaps an input");
        for (int j = 0; j < i; ++j)
            if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return set_error(FTTS_E_INVALID_ARG, "build_tables: two outputs overlap");
    }
    for (const auto& x : in)
        if (reinterpret_cast<uintptr_t>(x.p) & 3u) return set_error(FTTS_E_ALIGN, "build_tables: input not 4-byte aligned");
    TableArgs a{cached, added, free_pages, B, n_free, n_pages, max_pages, max_rows, block_table, row_offsets, seq_lens, slots, counts};
    const int64_t n = std::max<int64_t>((int64_t)B * max_pages, max_rows);
    const bool wide = n >= kTabWide;
    const int threads = B <= 256 && !wide ? 256 : kTabThreads, fill = threads * (wide ? 4 : 1);
    const dim3 g((unsigned)std::max<int64_t>(std::min<int64_t>((n + fill - 1) / fill, 256), 1));
    (void)hipGetLastError();
    if (wide) hipLaunchKernelGGL(build_tables_kernel<4>, g, dim3(threads), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(build_tables_kernel<1>, g, dim3(threads), 0, (hipStream_t)stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "build_tables launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

int ftts_append_kv(int32_t src_dtype, int32_t kv_dtype, const void* k, int64_t k_stride, const void* v,
                   int64_t v_stride, int32_t n_rows, const int32_t* slots, const ftts_kv_pool* kv, int32_t layer,
                   int32_t n_kv_head, void* stream) {
    if ((src_dtype != FTTS_F32 && src_dtype != FTTS_BF16) || (kv_dtype != FTTS_F32 && kv_dtype != FTTS_BF16))
        return set_error(FTTS_E_DTYPE, "append_kv: dtypes must be FTTS_F32 or FTTS_BF16");
    if (src_dtype == FTTS_BF16 && kv_dtype == FTTS_F32) return set_error(FTTS_E_DTYPE, "append_kv: bf16 rows into an fp32 pool");
    if (!kv || !kv->base) return set_error(FTTS_E_INVALID_ARG, "append_kv: pool is NULL");
    if (n_rows < 0 || n_rows > (1 << 24)) return set_error(FTTS_E_RANGE, "append_kv: n_rows must be in [0, 2^24]");
    if (n_kv_head < 1 || n_kv_head > 256) return set_error(FTTS_E_SHAPE, "append_kv: n_kv_head must be in [1, 256]");
    if (kv->n_pages < 1 || layer < 0) return set_error(FTTS_E_SHAPE, "append_kv: n_pages must be >= 1 and layer >= 0");
    if (n_rows == 0) return FTTS_OK;
    if (!k || !v || !slots) return set_error(FTTS_E_INVALID_ARG, "append_kv: NULL pointer");
    const int64_t piece = src_dtype == FTTS_F32 ? 4 : 8;  // elements in 16 bytes
    for (const int64_t st : {k_stride, v_stride})
        if (st < 64LL * n_kv_head || st > (1LL << 31) || st % piece)
            return set_error(FTTS_E_SHAPE, "append_kv: a stride must be a multiple of %d, at least 64 * n_kv_head", (int)piece);
    if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(kv->base)) & 15u)
        return set_error(FTTS_E_ALIGN, "append_kv: k, v and the pool must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(slots) & 3u) return set_error(FTTS_E_ALIGN, "append_kv: slots not 4-byte aligned");
    const AppendArgs a{k, v, k_stride, v_stride, n_rows, kv->n_pages, layer, n_kv_head, slots, kv->base};
    const dim3 g((n_rows + kAppWaves - 1) / kAppWaves), t(kAppWaves * 64);
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    if (src_dtype == FTTS_BF16) hipLaunchKernelGGL((append_kv_kernel<false, false>), g, t, 0, st, a);
    else if (kv_dtype == FTTS_BF16) hipLaunchKernelGGL((append_kv_kernel<true, false>), g, t, 0, st, a);
    else hipLaunchKernelGGL((append_kv_kernel<true, true>), g, t, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "append_kv launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

}  // extern "C"
