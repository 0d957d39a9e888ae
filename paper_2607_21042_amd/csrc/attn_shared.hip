// Attention of a batch of sequences that continue one shared prefix, over the paged cache.
//
// Row i of sequence b (n_b rows, L_b own tokens) sees the P tokens of the prefix and own tokens
// 0 .. L_b - n_b + i:  o = sum_j p_j v_j / sum_j p_j,  p_j = exp(q . k_j / 8 - m).
//
// A softmax over two disjoint sets of tokens is joined from (m, l, o) of each: m = max(m1, m2),
// l = l1 e^(m1 - m) + l2 e^(m2 - m), o likewise.  So the batch's rows meet the prefix as one
// matrix, whatever sequence they belong to, and each sequence's rows meet its own pages; both
// kinds of work are cut along the tokens into workgroups that leave partial results, and a
// second kernel joins them.
#include <algorithm>

#include "attn_tile.hpp"
#include "decode_entry.hpp"

namespace ftts {

constexpr int kSaWaves = 4, kSaQ = 32;

// How a call is cut: prefix rows in row_tiles tiles of 32, own rows in own_tiles (an upper bound
// where the rows per sequence are on the device); c_pre and c_own pages a workgroup, s_pre and
// s_own workgroups along the tokens; partials of slot s (prefix slots first) at ml + s * T H and
// o + s * T H * 64.
struct SharedPlan {
    int row_tiles, own_tiles, c_pre, s_pre, c_own, s_own;
    float2* ml;
    float* o;
};

// The rows of a workgroup: 32 (token, query head) pairs that read one key head.
struct RowTile {
    int row, head;   // this lane's pair; row -1: none
    int lim;         // the tokens of the segment that it sees
    int most;        // the largest lim of the tile
    bool inactive;   // the sequence has no length
};

// Tile `tile` of all rows (the prefix's side).
__device__ __forceinline__ RowTile prefix_rows(const SharedAttnArgs& a, int tile, int kh, int ql) {
    const int g = a.n_head / a.n_kv_head, idx = tile * kSaQ + ql;
    RowTile t;
    t.row = idx / g < a.rows ? idx / g : -1;
    t.head = kh * g + idx % g;
    t.lim = t.most = a.prefix_len;
    t.inactive = false;
    return t;
}
// Own tile `tile`: its sequence goes to b (B: past the last one).
__device__ __forceinline__ RowTile own_rows(const SharedAttnArgs& a, int tile, int kh, int lane, int ql, int& b) {
    const int g = a.n_head / a.n_kv_head;
    int n = 1, row0, in;  // rows and first row of the sequence, tile of the sequence
    if (!a.row_offsets) {
        const int per = (g + kSaQ - 1) / kSaQ;
        b = row0 = tile / per;
        in = tile - b * per;
    } else {
        static_assert(FTTS_MAX_BATCH <= kWave, "one sequence per lane");
        const int lo = lane < a.B ? a.row_offsets[lane] : 0, hi = lane < a.B ? a.row_offsets[lane + 1] : 0;
        const int first = min(max(lo, 0), a.rows), rows = min(max(hi, first), a.rows) - first;
        int end = (rows * g + kSaQ - 1) / kSaQ;  // (rows * n_head < 2^31)
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int u = __shfl_up(end, d, kWave);
            if (lane >= d) end += u;
        }
        b = __popcll(__ballot(lane < a.B && end <= tile));
        if (b >= a.B) return RowTile{-1, 0, 0, 0, false};
        row0 = __builtin_amdgcn_readlane(first, b);
        n = __builtin_amdgcn_readlane(rows, b);
        in = tile - (b ? __builtin_amdgcn_readlane(end, b - 1) : 0);
    }
    const int len = a.seq_lens[b], idx = in * kSaQ + ql, last = min(in * kSaQ + kSaQ, n * g) - 1;
    auto seen = [&](int i) {  // own tokens that row i of the sequence sees
        return len < 0 ? 0 : (int)min(max((int64_t)len - n + i + 1, (int64_t)0), (int64_t)a.max_pages * kPage);
    };
    RowTile t;
    t.row = idx <= last ? row0 + idx / g : -1;
    t.head = kh * g + idx % g;
    t.most = seen(last / g);
    t.lim = idx <= last ? seen(idx / g) : t.most;  // (a lane without a row asks for no mask)
    t.inactive = len < 0;
    return t;
}

// A wave's running attention of 32 rows: O^T as in AtState, the maximum (exp2 domain; -inf: nothing seen
// yet) and the sum over this lane's half of the keys.
struct SaState {
    at_f32x16 o0, o1;
    float m, l;
};

// Masks tokens at or past lim (k0: the tile's first token), moves the maximum where a tile exceeds it by
// more than 2^8, and gives the weights as bf16 pairs and (LO) what their rounding left, in bf16 too.
template <bool LO>
__device__ __forceinline__ void sa_softmax(SaState& a, at_f32x16 (&s)[2], int k0, int lim, int hh, uint32_t (&pw)[16],
                                           uint32_t (&pl)[LO ? 16 : 1]) {
    const float kScale = 0.125f * 1.44269504088896340736f;  // 1/sqrt(64) * log2(e)
    if (__any(lim < k0 + kAtK)) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (k0 + 32 * b + (i >> 2) * 8 + hh * 4 + (i & 3) >= lim) s[b][i] = -INFINITY;
    }
    float tmax = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) tmax = fmaxf(tmax, fmaxf(s[0][i], s[1][i]));
    {
        const RowPair pr = swap32(tmax);
        tmax = fmaxf(pr.a, pr.b) * kScale;
    }
    if (__any(tmax > a.m + 8.f)) {
        const float mn = fmaxf(a.m, tmax), alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(a.m - mn);
        a.m = mn;
        a.l *= alpha;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            a.o0[i] *= alpha;
            a.o1[i] *= alpha;
        }
    }
    const float ref = a.m == -INFINITY ? 0.f : a.m;  // nothing seen: every score is -inf and every weight 0
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[b][i], kScale, -ref));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], kScale, -ref));
            const uint32_t w = bf16x2_rne(x, y);
            pw[b * 8 + i / 2] = w;
            a.l += x + y;
            if constexpr (LO) pl[b * 8 + i / 2] = bf16x2_rne(x - bf16lo(w), y - bf16hi(w));
        }
}
// O^T += V^T P^T over a tile's 64 keys (k slots as at_read_v gives them).
__device__ __forceinline__ void sa_pv(SaState& a, const uint64_t (&v)[2][2][4], const uint32_t (&pw)[16]) {
#pragma unroll
    for (int st = 0; st < 4; ++st) {
        const at_bf16x8 pb = at_op(make_uint4(pw[4 * st], pw[4 * st + 1], pw[4 * st + 2], pw[4 * st + 3]));
        auto vop = [&](int d) {
            return at_op(make_uint4((uint32_t)v[d][0][st], (uint32_t)(v[d][0][st] >> 32), (uint32_t)v[d][1][st],
                                    (uint32_t)(v[d][1][st] >> 32)));
        };
        a.o0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop(0), pb, a.o0, 0, 0, 0);
        a.o1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop(1), pb, a.o1, 0, 0, 0);
    }
}
// Values that are not finite, in a tile that some row sees in part: in one product with the rest their 0 x inf = NaN
// would reach the rows that do not see them.  They become 0 in the operands (returns whether there were any) ...
__device__ __forceinline__ bool sa_take_out(uint64_t (&v)[2][2][4]) {
    uint32_t bad = 0;
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                uint32_t x[2] = {(uint32_t)v[d][e][st], (uint32_t)(v[d][e][st] >> 32)};
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t lo = (x[w] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u;
                    const uint32_t hi = (x[w] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u;
                    bad |= lo | hi;
                    x[w] &= ~(lo | hi);
                }
                v[d][e][st] = (uint64_t)x[1] << 32 | x[0];
            }
    return __any(bad != 0);
}
// ... and are added here where the weight is not 0.  vt: the tile in LDS; the weights go through 4 KB of it (wl, rows
// of 64 keys).
__device__ __forceinline__ void sa_add_not_finite(SaState& a, const char* vt, char* wl, const uint32_t (&pw)[16], int lane) {
    const int ql = lane & 31, hh = lane >> 5;
#pragma unroll
    for (int j = 0; j < 16; ++j)
        *reinterpret_cast<uint32_t*>(wl + ql * 128 + 2 * (32 * (j >> 3) + ((j >> 1) & 3) * 8 + hh * 4 + 2 * (j & 1))) = pw[j];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    for (int key = 0; key < kAtK; ++key) {
        const float p = bf16_to_f32(*reinterpret_cast<const uint16_t*>(wl + ql * 128 + 2 * key));
        const char* row = vt + key * 128 + hh * 8;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint2 x = *reinterpret_cast<const uint2*>(row + ((c ^ ((key >> 1) & 7)) << 4));
            const float f[4] = {bf16lo(x.x), bf16hi(x.x), bf16lo(x.y), bf16hi(x.y)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float y = p != 0.f && !(fabsf(f[i]) < INFINITY) ? p * f[i] : 0.f;
                if (c < 4) a.o0[4 * (c & 3) + i] += y;
                else a.o1[4 * (c & 3) + i] += y;
            }
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// One workgroup per key head, 32 rows and run of pages: the 4 waves take its pages in turn (wave w: w, w + 4, ...)
// by direct-to-LDS loads into a stage of their own, the next page's K (V) on its way once this one's is in
// registers, no barrier in the loop; their (m, l, o) are joined through LDS.  PROMPT: several rows a sequence, so a
// tile's rows may see different tokens.
template <bool PROMPT>
__global__ __launch_bounds__(kSaWaves * 64, 2) void shared_part_kernel(const SharedAttnArgs a, const SharedPlan pl) {
    constexpr int kWeights = PROMPT ? kSaQ * 128 : 0;
    __shared__ __attribute__((aligned(1024))) char smem[kSaWaves * (kAtStage + kWeights)];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ql = lane & 31, hh = lane >> 5;
    int id = blockIdx.x, kh, slot, page0, pages;
    RowTile t;
    const int32_t* ids;
    // Prefix work first: the row tiles of one (key head, run of pages) are 8 workgroups apart, so that one XCD
    // (workgroups are dealt to the 8 in turn) reads the run through its L2.
    const int n_pre = (a.n_kv_head * pl.s_pre + 7) / 8 * 8 * pl.row_tiles;
    if (id < n_pre) {
        const int pair = id / (8 * pl.row_tiles) * 8 + id % 8, tile = id / 8 % pl.row_tiles;
        if (pair >= a.n_kv_head * pl.s_pre) return;
        kh = pair % a.n_kv_head;
        slot = pair / a.n_kv_head;
        t = prefix_rows(a, tile, kh, ql);
        page0 = slot * pl.c_pre;
        pages = min(pl.c_pre, (a.prefix_len + kPage - 1) / kPage - page0);
        ids = a.prefix_pages + page0;
    } else {
        id -= n_pre;
        kh = id % a.n_kv_head;
        const int sp = id / a.n_kv_head % pl.s_own, tile = id / a.n_kv_head / pl.s_own;
        int b;
        t = own_rows(a, tile, kh, lane, ql, b);
        if (b >= a.B) return;
        slot = pl.s_pre + sp;
        page0 = sp * pl.c_own;
        pages = min(pl.c_own, (t.most + kPage - 1) / kPage - page0);
        ids = a.block_table + (size_t)b * a.max_pages + page0;
    }
    const int64_t rows_heads = (int64_t)a.rows * a.n_head;
    const int64_t part = slot * rows_heads + (int64_t)t.row * a.n_head + t.head;
    if (pages <= 0) {  // (an inactive sequence is marked by a negative sum)
        if (t.row >= 0 && tid < kSaQ) pl.ml[part] = make_float2(-INFINITY, t.inactive ? -1.f : 0.f);
        return;
    }
    char* own = smem + wave * kAtStage;
    char* wl = smem + kSaWaves * kAtStage + wave * kWeights;
    const int n = pages > wave ? (pages - wave + kSaWaves - 1) / kSaWaves : 0;  // this wave's pages
    int phys_l = 0;
    // the wave's page ids, 64 at a time (lane j: page j of the round)
    auto fetch_ids = [&](int j0) { phys_l = j0 + lane < n ? ids[wave + kSaWaves * (j0 + lane)] : -1; };
    auto load = [&](int j, int kv) {  // the wave's page j, K (kv 0) or V; nothing of an invalid page
        int phys = __builtin_amdgcn_readlane(phys_l, j & 63);
        const bool ok = phys >= 0 && phys < a.n_pages;
        const int left = t.most - (page0 + wave + kSaWaves * j) * kPage;
        const int bytes = ok ? min(left, kPage) * (kHeadDim * 2) : 0;
        const uint16_t* src = reinterpret_cast<const uint16_t*>(a.kv_base) +
                              kv_offset(a.layer, a.n_pages, ok ? phys : 0, kv, a.n_kv_head, kh, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = i * 8 + (lane >> 3);
            buffer_to_lds16(src, bytes, own + kv * kAtTile + i * 1024, row * 128 + (((lane & 7) ^ ((row >> 1) & 7)) << 4), 0);
        }
        return ok;
    };
    uint4 qr[4];
    {
        const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + (size_t)max(t.row, 0) * a.q_ld + t.head * kHeadDim;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) qr[kk] = *reinterpret_cast<const uint4*>(qp + kk * 16 + hh * 8);
    }
    const AtAddr ad = at_addresses(lds_address(own), lane);
    SaState st;
#pragma unroll
    for (int i = 0; i < 16; ++i) st.o0[i] = st.o1[i] = 0.f;
    st.m = -INFINITY;
    st.l = 0.f;
    bool ok = false;
    if (n > 0) {
        fetch_ids(0);
        ok = load(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load(0, 1);
    }
    for (int j = 0; j < n; ++j) {
        const bool more = j + 1 < n, seen = ok;
        const int k0 = (page0 + wave + kSaWaves * j) * kPage;
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // K is in (this wave's own loads), V's 8 loads may be out
        __builtin_amdgcn_sched_barrier(0);
        uint4 ka[4], kb[4];
        at_read_k(ad, 0, ka, kb);
        at_wait_lds();
        at_tie4(ka);
        at_tie4(kb);
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            if (((j + 1) & 63) == 0) fetch_ids(j + 1);
            ok = load(j + 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        at_f32x16 s[2];
        at_scores(ka, kb, qr, s);
        uint32_t pw[16], plo[16];
        sa_softmax<true>(st, s, k0, seen ? t.lim : 0, hh, pw, plo);
        __builtin_amdgcn_sched_barrier(0);
        if (more) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // V is in, the next K may be out
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        uint64_t v[2][2][4];
        at_read_v(ad, 0, v);
        at_wait_lds();
        at_tie_v(v);
        __builtin_amdgcn_sched_barrier(0);
        // (rows without a token in the tile have weights of 0, those past a tile's end zeros for values)
        if (PROMPT && __any(t.lim < min(t.most, k0 + kAtK)) && sa_take_out(v)) sa_add_not_finite(st, own + kAtTile, wl, pw, lane);
        if (more) load(j + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
        sa_pv(st, v, pw);
        sa_pv(st, v, plo);
    }
    __syncthreads();  // every wave has read its stage: the partials of waves 1 .. 3 go there, lane for lane
    float* mrg = reinterpret_cast<float*>(smem);  // [3][34][64]
    if (wave > 0) {
        float* mw = mrg + (wave - 1) * 34 * 64;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            mw[i * 64 + lane] = st.o0[i];
            mw[(16 + i) * 64 + lane] = st.o1[i];
        }
        mw[32 * 64 + lane] = st.m;
        mw[33 * 64 + lane] = st.l;
    }
    __syncthreads();
    if (wave > 0) return;
    float mm = st.m;
#pragma unroll
    for (int w = 0; w < kSaWaves - 1; ++w) mm = fmaxf(mm, mrg[(w * 34 + 32) * 64 + lane]);
    const float ref = mm == -INFINITY ? 0.f : mm;
    const float f0 = exp2f(st.m - ref);
    st.l *= f0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        st.o0[i] *= f0;
        st.o1[i] *= f0;
    }
#pragma unroll
    for (int w = 0; w < kSaWaves - 1; ++w) {
        const float* mw = mrg + w * 34 * 64;
        const float f = exp2f(mw[32 * 64 + lane] - ref);
        st.l += mw[33 * 64 + lane] * f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            st.o0[i] += mw[i * 64 + lane] * f;
            st.o1[i] += mw[(16 + i) * 64 + lane] * f;
        }
    }
    const RowPair ls = swap32(st.l);
    if (t.row < 0) return;
    if (hh == 0) pl.ml[part] = make_float2(mm, ls.a + ls.b);
    float4* out = reinterpret_cast<float4*>(pl.o + part * kHeadDim) + hh;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        out[2 * g] = make_float4(st.o0[4 * g], st.o0[4 * g + 1], st.o0[4 * g + 2], st.o0[4 * g + 3]);
        out[8 + 2 * g] = make_float4(st.o1[4 * g], st.o1[4 * g + 1], st.o1[4 * g + 2], st.o1[4 * g + 3]);
    }
}

// Joins the partials: 16 lanes per (row, head), 4 dims each.
template <bool F32>
__global__ __launch_bounds__(256) void shared_join_kernel(const SharedAttnArgs a, const SharedPlan pl) {
    const int64_t rows_heads = (int64_t)a.rows * a.n_head, rh = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (rh >= rows_heads) return;
    const int r = (int)(rh / a.n_head), h = (int)(rh % a.n_head), d = (threadIdx.x & 15) * 4;
    if (a.row_offsets && (r < a.row_offsets[0] || r >= a.row_offsets[a.B])) return;
    const int S = pl.s_pre + pl.s_own;
    float m = -INFINITY;
    bool inactive = false;
    for (int s = 0; s < S; ++s) {
        const float2 x = pl.ml[s * rows_heads + rh];
        m = fmaxf(m, x.x);
        inactive |= x.y < 0.f;
    }
    float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    if (!inactive)
        for (int s = 0; s < S; ++s) {
            const float2 x = pl.ml[s * rows_heads + rh];
            if (x.y == 0.f) continue;  // nothing seen there (and nothing written)
            const float f = exp2f(x.x - (m == -INFINITY ? 0.f : m));
            const float4 y = *reinterpret_cast<const float4*>(pl.o + (s * rows_heads + rh) * kHeadDim + d);
            l = fmaf(x.y, f, l);
            o[0] = fmaf(y.x, f, o[0]);
            o[1] = fmaf(y.y, f, o[1]);
            o[2] = fmaf(y.z, f, o[2]);
            o[3] = fmaf(y.w, f, o[3]);
        }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const size_t at = (size_t)r * a.o_ld + h * kHeadDim + d;
    if constexpr (F32)
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.o) + at) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    else
        *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.o) + at) =
            make_uint2(bf16x2_rne(o[0] * inv, o[1] * inv), bf16x2_rne(o[2] * inv, o[3] * inv));
}

// ---- fp32: one wave per row and head ---------------------------------------------------------
// Lane j scores token j of a page, and lane d then sums dimension d over the tokens that the row
// sees (the others are not read).
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
    const float q = ld_act<true>(a.q, (size_t)r * a.q_ld + h * kHeadDim + lane) * 0.125f;
    float m = -INFINITY, l = 0.f, o = 0.f;
    auto page = [&](int phys, int seen) {  // the first `seen` tokens of a page
        if (phys < 0 || phys >= a.n_pages) return;
        const size_t kb = kv_offset(a.layer, a.n_pages, phys, 0, a.n_kv_head, kh, 0);
        const size_t vb = kv_offset(a.layer, a.n_pages, phys, 1, a.n_kv_head, kh, 0);
        float s = 0.f;
        for (int d = 0; d < kHeadDim; ++d) {
            const float qd = __shfl(q, d, kWave);
            if (lane < seen) s = fmaf(qd, ld_act<true>(a.kv_base, kb + lane * kHeadDim + d), s);
        }
        if (lane >= seen) s = -INFINITY;
        const float mn = fmaxf(m, wave_max(s));
        const float ref = mn == -INFINITY ? 0.f : mn;
        const float f = expf(m - ref), p = expf(s - ref);
        m = mn;
        l = l * f + wave_sum(p);
        o *= f;
        for (int j = 0; j < seen; ++j) o = fmaf(__shfl(p, j, kWave), ld_act<true>(a.kv_base, vb + j * kHeadDim + lane), o);
    };
    if (len >= 0)
        for (int t = 0; t < a.prefix_len; t += kPage) page(a.prefix_pages[t / kPage], min(kPage, a.prefix_len - t));
    for (int t = 0; t < own; t += kPage) page(a.block_table[(size_t)b * a.max_pages + t / kPage], min(kPage, own - t));
    st_act<true>(a.o, (size_t)r * a.o_ld + h * kHeadDim + lane, l == 0.f ? 0.f : o / l);
}

constexpr int kGroups = 1536, kMaxSplit = 64;

// Workgroups along the tokens: as many pages each (a multiple of the 4 waves) as keep the call near
// kGroups workgroups, at most kMaxSplit of them for the prefix.
static SharedPlan shared_plan(int n_head, int n_kv_head, int B, int rows, bool prompt, int prefix_len, int max_pages) {
    const int g = n_head / n_kv_head;
    SharedPlan p{};
    p.row_tiles = (int)(((int64_t)rows * g + kSaQ - 1) / kSaQ);
    p.own_tiles = prompt ? (int)((int64_t)rows * g / kSaQ) + B : B * ((g + kSaQ - 1) / kSaQ);
    const int pages = (prefix_len + kPage - 1) / kPage;
    int c = kSaWaves;
    for (;; c += kSaWaves) {
        p.s_pre = (pages + c - 1) / c;
        p.s_own = (max_pages + c - 1) / c;
        const int64_t n = (int64_t)n_kv_head * ((int64_t)p.row_tiles * p.s_pre + (int64_t)p.own_tiles * p.s_own);
        if (p.s_pre <= kMaxSplit && (n <= kGroups || c >= std::max(pages, max_pages))) break;
    }
    p.c_pre = p.c_own = c;
    return p;
}

// An upper bound of the partials of every call up to these sizes: a call has either one slot on each side or at
// most kGroups workgroups of 32 rows, and its slots hold at least 4 pages each.
size_t shared_attention_bytes(int n_head, int rows, int prefix_len, int max_pages) {
    const int pages = (prefix_len + kPage - 1) / kPage;
    const int64_t rh = (int64_t)rows * n_head, slots = std::min((pages + 3) / 4, kMaxSplit) + (max_pages + 3) / 4;
    const int64_t n = std::max(std::min(slots * rh, (int64_t)kGroups * kSaQ), std::min<int64_t>(slots, 2) * rh);
    return (size_t)n * (kHeadDim + 2) * 4 + 256;
}

hipError_t launch_shared_attention(int dtype, const SharedAttnArgs& a, void* ws, hipStream_t st) {
    if (dtype == FTTS_F32) {
        const dim3 g((unsigned)(((int64_t)a.rows * a.n_head + kSaWaves - 1) / kSaWaves)), t(kSaWaves * 64);
        hipLaunchKernelGGL(shared_row_kernel, g, t, 0, st, a);
        return hipGetLastError();
    }
    SharedPlan p = shared_plan(a.n_head, a.n_kv_head, a.B, a.rows, a.row_offsets != nullptr, a.prefix_len, a.max_pages);
    const int64_t rows_heads = (int64_t)a.rows * a.n_head;
    p.o = reinterpret_cast<float*>(ws);
    p.ml = reinterpret_cast<float2*>(p.o + (p.s_pre + p.s_own) * rows_heads * kHeadDim);
    const int64_t groups = (int64_t)((a.n_kv_head * p.s_pre + 7) / 8 * 8) * p.row_tiles + (int64_t)a.n_kv_head * p.own_tiles * p.s_own;
    const dim3 g((unsigned)groups), t(kSaWaves * 64);
    if (a.row_offsets) hipLaunchKernelGGL(shared_part_kernel<true>, g, t, 0, st, a, p);
    else hipLaunchKernelGGL(shared_part_kernel<false>, g, t, 0, st, a, p);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL(shared_join_kernel<false>, dim3((unsigned)((rows_heads + 15) / 16)), dim3(256), 0, st, a, p);
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
    if (n_rows < 0 || n_rows > (1 << 24) || (int64_t)n_rows * s->n_head > 0x7FFFFFFF)
        return set_error(FTTS_E_RANGE, "shared_attention: n_rows must be in [0, 2^24] and n_rows * n_head below 2^31");
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
    return shared_attention_bytes(shape->n_head, n_rows, prefix_len, max_pages);
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
    const hipError_t e = launch_shared_attention(shape->dtype, a, ws, (hipStream_t)stream);
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "shared_attention launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

}  // extern "C"
