// Attention of a batch of sequences that continue one shared prefix, over the paged cache.
//
// Row i of sequence b (n_b rows, L_b own tokens) sees the P tokens of the prefix and own tokens
// 0 .. L_b - n_b + i:  o = sum_j p_j v_j / sum_j p_j,  p_j = exp(q . k_j / 8 - m).
//
// A softmax over two disjoint sets of tokens is joined from (m, l, o) of each: m = max(m1, m2),
// l = l1 e^(m1 - m) + l2 e^(m2 - m), o likewise.  Four kernels share that, chosen by rules on sizes
// (shared_whole, tile_plan):
//   cut    (shared_part_*_kernel): the batch's rows meet the prefix as one matrix, whatever sequence they
//          belong to, and each sequence's rows meet its own pages; both kinds of work are cut along the tokens into
//          workgroups that leave partial results, and a second kernel joins them.  Bound by reading the pages once.
//   whole  one row a sequence and few pages: a workgroup a sequence and key head, no partials.
//   tile   many rows: 128 rows, of one sequence or of several, share each page on its way through LDS; a long chain of
//          pages of few tiles is cut into parts, which the second kernel joins.  Bound by vector and matrix work.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

#include "attn_tile.hpp"
#include "decode_entry.hpp"

namespace ftts {

constexpr int kSaWaves = 2, kSaQ = 32;

// How a call is cut: prefix rows in row_tiles tiles of q_pre, own rows in own_tiles of q_own (an upper bound
// where the rows per sequence are on the device); c_pre and c_own pages a workgroup, s_pre and
// s_own workgroups along the tokens; partials of slot s (prefix slots first) at ml + s * T H and
// o + s * T H * 64.
struct SharedPlan {
    int q_pre, q_own, row_tiles, own_tiles, c_pre, s_pre, c_own, s_own;
    float2* ml;
    float* o;
};

// The rows of a workgroup: up to 32 (token, query head) pairs that read one key head.
struct RowTile {
    int row, head;   // this lane's pair; row -1: none
    int lim;         // the tokens of the segment that it sees
    int most;        // the largest lim of the tile
    bool inactive;   // the sequence has no length
};

// Tile `tile` of `size` of all rows (the prefix's side).
__device__ __forceinline__ RowTile prefix_rows(const SharedAttnArgs& a, int tile, int size, int kh, int ql) {
    const int g = a.n_head / a.n_kv_head, idx = tile * size + ql;
    RowTile t;
    t.row = idx / g < a.rows ? idx / g : -1;
    t.head = kh * g + idx % g;
    t.lim = t.most = a.prefix_len;
    t.inactive = false;
    return t;
}
// A run of the rows of one sequence: (token, head) pairs first .. first + size - 1 of its n * g.
struct OwnTile {
    int b, row0, n, len, first;  // sequence (B: past the last one), its first row, rows and length
};
// Tile `tile` of `size` pairs.  Whole waves call it.
__device__ __forceinline__ OwnTile own_tile(const SharedAttnArgs& a, int tile, int size, int lane) {
    const int g = a.n_head / a.n_kv_head;
    OwnTile t;
    if (!a.row_offsets) {
        const int per = (g + size - 1) / size;
        t.b = t.row0 = tile / per;
        t.n = 1;
        t.first = (tile - t.b * per) * size;
    } else {
        static_assert(FTTS_MAX_BATCH <= kWave, "one sequence per lane");
        const int lo = lane < a.B ? a.row_offsets[lane] : 0, hi = lane < a.B ? a.row_offsets[lane + 1] : 0;
        const int first = min(max(lo, 0), a.rows), rows = min(max(hi, first), a.rows) - first;
        int end = (rows * g + size - 1) / size;  // (rows * n_head < 2^31)
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int u = __shfl_up(end, d, kWave);
            if (lane >= d) end += u;
        }
        t.b = __popcll(__ballot(lane < a.B && end <= tile));
        if (t.b >= a.B) return t;
        t.row0 = __builtin_amdgcn_readlane(first, t.b);
        t.n = __builtin_amdgcn_readlane(rows, t.b);
        t.first = (tile - (t.b ? __builtin_amdgcn_readlane(end, t.b - 1) : 0)) * size;
    }
    t.len = a.seq_lens[t.b] + a.len_add;
    if (a.active && !a.active[t.b]) t.len = -1;
    return t;
}
// Own tokens that the i-th row of the sequence sees.
__device__ __forceinline__ int own_seen(const SharedAttnArgs& a, int len, int n, int i) {
    return len < 0 ? 0 : (int)min(max((int64_t)len - n + i + 1, (int64_t)0), (int64_t)a.max_pages * kPage);
}
__device__ __forceinline__ int own_seen(const SharedAttnArgs& a, const OwnTile& t, int i) { return own_seen(a, t.len, t.n, i); }
// The `size` pairs from `first` on.
__device__ __forceinline__ RowTile own_rows(const SharedAttnArgs& a, const OwnTile& o, int first, int size, int kh, int ql) {
    const int g = a.n_head / a.n_kv_head, idx = first + ql, last = min(first + size, o.n * g) - 1;
    RowTile t;
    t.row = idx <= last ? o.row0 + idx / g : -1;
    t.head = kh * g + idx % g;
    t.most = last >= first ? own_seen(a, o, last / g) : 0;
    t.lim = idx <= last ? own_seen(a, o, idx / g) : t.most;  // (a lane without a row asks for no mask)
    t.inactive = o.len < 0;
    return t;
}

// A staged tile's K operands, and its V operands (SO: byte offset of the stage), in one assembly block with the wait:
// nothing is in flight in a register that the compiler holds for written.
template <int SO>
__device__ __forceinline__ void sa_read_k(const AtAddr& r, uint4 (&ka)[4], uint4 (&kb)[4]) {
    at_bf16x8 x[8];
    asm volatile(
        "ds_read_b128 %0, %8 offset:%12\n\tds_read_b128 %1, %9 offset:%12\n\t"
        "ds_read_b128 %2, %10 offset:%12\n\tds_read_b128 %3, %11 offset:%12\n\t"
        "ds_read_b128 %4, %8 offset:%13\n\tds_read_b128 %5, %9 offset:%13\n\t"
        "ds_read_b128 %6, %10 offset:%13\n\tds_read_b128 %7, %11 offset:%13\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(r.kr[0]), "v"(r.kr[1]), "v"(r.kr[2]), "v"(r.kr[3]), "n"(SO), "n"(SO + 4096)
        : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        ka[i] = __builtin_bit_cast(uint4, x[i]);
        kb[i] = __builtin_bit_cast(uint4, x[4 + i]);
    }
}
template <int SO>
__device__ __forceinline__ void sa_read_v(const AtAddr& r, uint64_t (&v)[2][2][4]) {
#define SA_TR(O, A, S) "ds_read_b64_tr_b16 %" #O ", %" #A " offset:%" #S "\n\t"
    asm volatile(
        SA_TR(0, 16, 20) SA_TR(1, 16, 21) SA_TR(2, 16, 22) SA_TR(3, 16, 23)
        SA_TR(4, 17, 20) SA_TR(5, 17, 21) SA_TR(6, 17, 22) SA_TR(7, 17, 23)
        SA_TR(8, 18, 20) SA_TR(9, 18, 21) SA_TR(10, 18, 22) SA_TR(11, 18, 23)
        SA_TR(12, 19, 20) SA_TR(13, 19, 21) SA_TR(14, 19, 22) SA_TR(15, 19, 23)
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(v[0][0][0]), "=&v"(v[0][0][1]), "=&v"(v[0][0][2]), "=&v"(v[0][0][3]), "=&v"(v[0][1][0]), "=&v"(v[0][1][1]),
          "=&v"(v[0][1][2]), "=&v"(v[0][1][3]), "=&v"(v[1][0][0]), "=&v"(v[1][0][1]), "=&v"(v[1][0][2]), "=&v"(v[1][0][3]),
          "=&v"(v[1][1][0]), "=&v"(v[1][1][1]), "=&v"(v[1][1][2]), "=&v"(v[1][1][3])
        : "v"(r.vr[0][0]), "v"(r.vr[1][0]), "v"(r.vr[0][1]), "v"(r.vr[1][1]), "n"(SO), "n"(SO + 2048), "n"(SO + 4096), "n"(SO + 6144)
        : "memory");
#undef SA_TR
}

// A page of one key head as its loads see it: where its keys (its values: n_kv_head blocks on) begin, and how many
// tokens of it are seen, 0 for a page outside the pool.  One a lane, computed 64 at a time: a loop's scalar work per page is
// what the vector units wait for.
struct PageRef {
    uint32_t lo, hi;
    int tokens;
};
__device__ __forceinline__ PageRef page_ref(const SharedAttnArgs& a, int kh, int esize, int phys, int left) {
    const bool ok = phys >= 0 && phys < a.n_pages;
    const uint64_t off = kv_offset(a.layer, a.n_pages, ok ? phys : 0, 0, a.n_kv_head, kh, 0) * esize;
    return {(uint32_t)off, (uint32_t)(off >> 32), ok ? max(min(left, kPage), 0) : 0};
}
__device__ __forceinline__ const char* page_at(const SharedAttnArgs& a, const PageRef& r, int lane) {
    return reinterpret_cast<const char*>(a.kv_base) +
           ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)r.hi, lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)r.lo, lane));
}

// A wave's running attention of 32 rows: O^T as in AtState, the maximum (exp2 domain; -inf: nothing seen
// yet) and the sum over this lane's half of the keys.
typedef __bf16 sa_bf16x2 __attribute__((ext_vector_type(2)));
struct SaState {
    at_f32x16 o0, o1;
    float m, l;
};

// A maximum of kSaLowest marks a row that has seen tokens, all with a score of -inf: it has no softmax unless others join.
constexpr float kSaLowest = -3.402823466e38f;
__device__ __forceinline__ float sa_marked(float m, bool saw) { return saw && m == -INFINITY ? kSaLowest : m; }
// 1 / l: where nothing has been seen 0, where every score was -inf NaN.
__device__ __forceinline__ float sa_inverse(float l, float m) { return l != 0.f ? 1.0f / l : m == kSaLowest ? NAN : 0.f; }

__device__ __forceinline__ void sa_init(SaState& a) {
#pragma unroll
    for (int i = 0; i < 16; ++i) a.o0[i] = a.o1[i] = 0.f;
    a.m = -INFINITY;
    a.l = 0.f;
}

// Masks tokens at or past lim (k0: the tile's first token).
__device__ __forceinline__ void sa_mask(at_f32x16 (&s)[2], int k0, int lim, int hh) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k0 + 32 * b + (i >> 2) * 8 + hh * 4 + (i & 3) >= lim) s[b][i] = -INFINITY;
}
constexpr float kSaScale = 0.125f * 1.44269504088896340736f;  // 1/sqrt(64) * log2(e)
// Moves the maximum where a tile exceeds it by more than 2^8.
template <int N>
__device__ __forceinline__ void sa_maximum(SaState& a, const at_f32x16 (&s)[N]) {
    // (the maximum that passes NaN on: one instruction for three operands, and none to quieten them)
    float tmax = s[0][0];
#pragma unroll
    for (int i = 1; i < 16 * N; ++i) tmax = __builtin_elementwise_maximum(tmax, s[i >> 4][i & 15]);
    {
        const RowPair pr = swap32(tmax);
        tmax = __builtin_elementwise_maximum(pr.a, pr.b) * kSaScale;
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
}
// Weights x, y >= 0 in two bf16 parts each, the larger one below the weight, so that what is left is above 0 where the
// weight is: with both times an infinite value the product stays infinite (a part of 0, or below it, would make NaN of
// it).  Within 2^-16 of the weight: the larger part leaves less than 2^-7 of it, rounded by 2^-9 of that.
__device__ __forceinline__ uint32_t sa_split(float x, float y, uint32_t& left) {
    const uint32_t a = __builtin_elementwise_sub_sat(__float_as_uint(x), 1u), b = __builtin_elementwise_sub_sat(__float_as_uint(y), 1u);
    left = bf16x2_rne(x - __uint_as_float(a & 0xFFFF0000u), y - __uint_as_float(b & 0xFFFF0000u));
    return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
// The weights as bf16 pairs, their sum over this lane's half of the keys and (LO) their second parts.
template <bool LO>
__device__ __forceinline__ float sa_weights(const SaState& a, const at_f32x16 (&s)[2], uint32_t (&pw)[16], uint32_t (&pl)[LO ? 16 : 1]) {
    const float ref = a.m == -INFINITY ? 0.f : a.m;  // nothing seen: every score is -inf and every weight 0
    float l = 0.f;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[b][i], kSaScale, -ref));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], kSaScale, -ref));
            if constexpr (LO) {
                l += x + y;
                pw[b * 8 + i / 2] = sa_split(x, y, pl[b * 8 + i / 2]);
            } else {
                const uint32_t w = bf16x2_rne(x, y);
                pw[b * 8 + i / 2] = w;
                l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(sa_bf16x2, w), __builtin_bit_cast(sa_bf16x2, 0x3F803F80u), l, false);
            }
        }
    return l;
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
// would reach the rows that do not see them.  Whether there are any: the sums of all values by dimension, a product
// with ones, tell (finite ones that overflow fp32 only send the tile the slow way).  x: registers for it.
__device__ __forceinline__ bool sa_not_finite(const uint64_t (&v)[2][2][4], at_f32x16 (&x)[2]) {
    const at_bf16x8 ones = at_op(make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
    float z = 0.f;
#pragma unroll
    for (int d = 0; d < 2; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[d][i] = 0.f;
#pragma unroll
        for (int st = 0; st < 4; ++st)
            x[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                at_op(make_uint4((uint32_t)v[d][0][st], (uint32_t)(v[d][0][st] >> 32), (uint32_t)v[d][1][st], (uint32_t)(v[d][1][st] >> 32))),
                ones, x[d], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) z = fmaf(x[d][i], 0.f, z);
    }
    return __any(z != 0.f);  // (NaN)
}
// Then they become 0 in the operands ...
__device__ __forceinline__ void sa_take_out(uint64_t (&v)[2][2][4]) {
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                uint32_t x[2] = {(uint32_t)v[d][e][st], (uint32_t)(v[d][e][st] >> 32)};
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if ((x[w] & 0x7F80u) == 0x7F80u) x[w] &= 0xFFFF0000u;
                    if ((x[w] & 0x7F800000u) == 0x7F800000u) x[w] &= 0xFFFFu;
                }
                v[d][e][st] = (uint64_t)x[1] << 32 | x[0];
            }
}
// ... and are added here to the rows that see the token, at a weight of 0 too.  vt: the tile in LDS; seen: its tokens that
// this lane's row sees.
__device__ __forceinline__ void sa_add_not_finite(SaState& a, const char* vt, const uint32_t (&pw)[16], int seen, int hh) {
    uint32_t p[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) p[j] = pw[j];
#pragma unroll 1
    for (int j = 0; j < 16; ++j) {  // pair j of both halves of the wave: 4 keys
        const auto w = __builtin_amdgcn_permlane32_swap(p[0], p[0], false, false);
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {
            const uint32_t x = k < 2 ? w[0] : w[1];
            const float pk = k & 1 ? bf16hi(x) : bf16lo(x);
            const int key = 32 * (j >> 3) + ((j >> 1) & 3) * 8 + (k >> 1) * 4 + 2 * (j & 1) + (k & 1);
            const char* row = vt + key * 128 + hh * 8;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint2 v = *reinterpret_cast<const uint2*>(row + ((c ^ ((key >> 1) & 7)) << 4));
                const float f[4] = {bf16lo(v.x), bf16hi(v.x), bf16lo(v.y), bf16hi(v.y)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y = key < seen && !(fabsf(f[i]) < INFINITY) ? pk * f[i] : 0.f;
                    if (c < 4) a.o0[4 * (c & 3) + i] += y;
                    else a.o1[4 * (c & 3) + i] += y;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 15; ++i) p[i] = p[i + 1];
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// Four fp32 queries as bf16, and what their rounding left, in bf16 too: scores then see 16 bits of each, as in the
// decode step without a prefix (8 bits alone let two scores of 100 move against each other by 0.04 and more).
__device__ __forceinline__ uint2 sa_round_q(const float4& x, uint2& left) {
    const uint2 r = make_uint2(bf16x2_rne(x.x, x.y), bf16x2_rne(x.z, x.w));
    left = make_uint2(bf16x2_rne(x.x - bf16lo(r.x), x.y - bf16hi(r.x)), bf16x2_rne(x.z - bf16lo(r.y), x.w - bf16hi(r.y)));
    return r;
}
// Adds the scores of the queries' second part.
__device__ __forceinline__ void sa_scores_left(const uint4 (&ka)[4], const uint4 (&kb)[4], const uint4 (&ql)[4], at_f32x16 (&s)[2]) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at_op(b ? kb[kk] : ka[kk]), at_op(ql[kk]), s[b], 0, 0, 0);
}

// A page id asked for before it is known whether the page is seen (a plain load could be moved behind that): the ids
// then come with the lengths instead of a trip to memory after them.
__device__ __forceinline__ int early_id(const int32_t* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
}

// What a workgroup of the cut call does: a tile of rows, one key head, a run of pages.
struct PartWork {
    RowTile t;
    const int32_t* ids;  // its pages
    int size, kh, page0, pages;
    int id0;             // page 2 * lane + wave of the run
    int64_t part;        // where this lane's row leaves its partial
};
// Prefix work comes first: the row tiles of one (key head, run of pages) are 8 workgroups apart, so that one XCD
// (workgroups are dealt to the 8 in turn) reads the run through its L2.  False: nothing to do (what has no pages
// says so in its slot).
template <bool SIZES>  // tiles as the plan says, else 32 rows
__device__ __forceinline__ bool part_work(const SharedAttnArgs& a, const SharedPlan& pl, int tid, PartWork& w) {
    const int lane = tid & 63, j0 = (tid >> 6) + kSaWaves * lane;
    int id = blockIdx.x, slot;
    const int n_pre = (a.n_kv_head * pl.s_pre + 7) / 8 * 8 * pl.row_tiles;
    if (id < n_pre) {
        const int pair = id / (8 * pl.row_tiles) * 8 + id % 8, tile = id / 8 % pl.row_tiles;
        if (pair >= a.n_kv_head * pl.s_pre) return false;
        w.kh = pair % a.n_kv_head;
        slot = pair / a.n_kv_head;
        w.size = SIZES ? pl.q_pre : kSaQ;
        w.t = prefix_rows(a, tile, w.size, w.kh, lane & (w.size - 1));
        w.page0 = slot * pl.c_pre;
        w.pages = min(pl.c_pre, (a.prefix_len + kPage - 1) / kPage - w.page0);
        w.ids = a.prefix_pages + w.page0;
        w.id0 = early_id(w.ids + min(j0, w.pages - 1));
    } else {
        id -= n_pre;
        w.kh = id % a.n_kv_head;
        const int sp = id / a.n_kv_head % pl.s_own, tile = id / a.n_kv_head / pl.s_own;
        w.page0 = sp * pl.c_own;
        w.size = SIZES ? pl.q_own : kSaQ;
        const OwnTile o = own_tile(a, tile, w.size, lane);
        if (o.b >= a.B) return false;
        w.ids = a.block_table + (size_t)o.b * a.max_pages + w.page0;
        w.id0 = early_id(w.ids + min(j0, a.max_pages - 1 - w.page0));
        w.t = own_rows(a, o, o.first, w.size, w.kh, lane & (w.size - 1));
        slot = pl.s_pre + sp;
        w.pages = min(pl.c_own, (w.t.most + kPage - 1) / kPage - w.page0);
    }
    w.part = slot * ((int64_t)a.rows * a.n_head) + (int64_t)w.t.row * a.n_head + w.t.head;
    if (w.pages > 0) return true;
    // (an inactive sequence is marked by a negative sum)
    if (w.t.row >= 0 && tid < w.size) pl.ml[w.part] = make_float2(-INFINITY, w.t.inactive ? -1.f : 0.f);
    return false;
}
// Joins the waves' results through LDS (every wave is done with smem) and leaves the partial.
__device__ __forceinline__ void part_finish(const SharedPlan& pl, const PartWork& w, SaState& st, char* smem, int wave, int lane) {
    static_assert(kSaWaves == 2, "one wave hands over to the other");
    __syncthreads();
    float* mw = reinterpret_cast<float*>(smem);  // [34][64], lane for lane
    if (wave > 0) {
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
    const float m1 = mw[32 * 64 + lane], mm = fmaxf(st.m, m1), ref = mm == -INFINITY ? 0.f : mm;
    const float f0 = exp2f(st.m - ref), f1 = exp2f(m1 - ref);
    const RowPair ls = swap32(st.l * f0 + mw[33 * 64 + lane] * f1);
    if (w.t.row < 0) return;
    const int hh = lane >> 5;
    if (hh == 0) pl.ml[w.part] = make_float2(mm, ls.a + ls.b);
    float4* out = reinterpret_cast<float4*>(pl.o + w.part * kHeadDim) + hh;
    auto sum = [&](const at_f32x16& o, int at, int i) { return o[i] * f0 + mw[(at + i) * 64 + lane] * f1; };
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        out[2 * g] = make_float4(sum(st.o0, 0, 4 * g), sum(st.o0, 0, 4 * g + 1), sum(st.o0, 0, 4 * g + 2), sum(st.o0, 0, 4 * g + 3));
        out[8 + 2 * g] = make_float4(sum(st.o1, 16, 4 * g), sum(st.o1, 16, 4 * g + 1), sum(st.o1, 16, 4 * g + 2), sum(st.o1, 16, 4 * g + 3));
    }
}

// Tiles of 4 rows (one row a sequence): products of 16 blocks of 4x4.  Scores: a block's 4 keys by the 4 rows, so that
// lane (block, row) holds 4 keys' scores; values: 4 rows by a block's 4 dims, the weights of one block's keys handed to
// all blocks by the instruction.  The state: the lane's row's maximum, its sum over the lane's keys, and the 4 rows'
// outputs in dim `lane`.
constexpr int kFew = 4;
typedef float few_f32x4 __attribute__((ext_vector_type(4)));
struct FewState {
    float m = -INFINITY, l = 0.f;
    few_f32x4 o[2] = {};  // (two chains of products)
    bool saw = false;     // a token
};
// The scores p of a page (-inf: not seen) to weights.
__device__ __forceinline__ void few_weights(FewState& a, float (&p)[4]) {
    float tmax = __builtin_elementwise_maximum(__builtin_elementwise_maximum(p[0], p[1]), __builtin_elementwise_maximum(p[2], p[3]));
#pragma unroll
    for (int d = 4; d < 16; d <<= 1) tmax = __builtin_elementwise_maximum(tmax, __shfl_xor(tmax, d, kWave));
    const RowPair p16 = swap16(tmax);
    const RowPair p32 = swap32(__builtin_elementwise_maximum(p16.a, p16.b));
    tmax = __builtin_elementwise_maximum(p32.a, p32.b) * kSaScale;
    if (__any(tmax > a.m + 8.f)) {  // as sa_maximum
        const float mn = fmaxf(a.m, tmax), alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(a.m - mn);
        a.m = mn;
        a.l *= alpha;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __shfl(alpha, i, kWave);
            a.o[0][i] *= x;
            a.o[1][i] *= x;
        }
    }
    const float ref = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], kSaScale, -ref));
        a.l += p[i];
    }
}
// As part_finish.
__device__ __forceinline__ void few_finish(const SharedPlan& pl, const PartWork& w, FewState& st, char* smem, int wave, int lane) {
    static_assert(kSaWaves == 2, "one wave hands over to the other");
    st.o[0] += st.o[1];
    st.m = sa_marked(st.m, st.saw);
#pragma unroll
    for (int d = 4; d < kWave; d <<= 1) st.l += __shfl_xor(st.l, d, kWave);
    __syncthreads();
    float* mw = reinterpret_cast<float*>(smem) + lane;  // [6][64], lane for lane
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) mw[i * 64] = st.o[0][i];
        mw[4 * 64] = st.m;
        mw[5 * 64] = st.l;
    }
    __syncthreads();
    if (wave > 0) return;
    const float m1 = mw[4 * 64], mm = fmaxf(st.m, m1), ref = mm == -INFINITY ? 0.f : mm;
    const float f0 = exp2f(st.m - ref), f1 = exp2f(m1 - ref), l = st.l * f0 + mw[5 * 64] * f1;
    if (lane < kFew && w.t.row >= 0) pl.ml[w.part] = make_float2(mm, l);
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // row i: its weights and its partial's place are lane i's
        const float o = st.o[0][i] * __shfl(f0, i, kWave) + mw[i * 64] * __shfl(f1, i, kWave);
        const int64_t part = __shfl(w.part, i, kWave);
        if (__shfl(w.t.row, i, kWave) >= 0) pl.o[part * kHeadDim + lane] = o;
    }
}

// bf16: K and V through LDS as in shared_part_kernel.  In a graph, with the join, 32 sequences of 64-700 tokens behind
// 1500, 20 heads, 18.2 us (tiles of 32 rows: 20.1), 8 of 30-500 behind 700 10.1 (11.3).  Two groups of 4 rows a tile, for 5 to 8 query
// heads a key head, were slower than one tile of 32: 14.4 us for 24 sequences of 20/4 heads (13.6).
typedef short few_s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ few_s16x4 few_op(uint32_t x, uint32_t y) { return __builtin_bit_cast(few_s16x4, make_uint2(x, y)); }
// fp32 queries: lane (block, row) rounds its 4 dims of the row, and through LDS (at s0, where the first page's values
// land afterwards) every lane gets both parts of its row: a sixteenth of the rounding, and one load a lane.  A step of 24
// layers behind 1500 tokens, 32, 8 and 1 sequences: 1383, 1118 and 845 us; where every lane rounds its row 1399, 1134 and
// 867; 8-bit queries 1390, 1121 and 842.
__device__ __forceinline__ void few_exchange_q(const float4& x, uint32_t s0, int lane, uint4 (&q)[8], uint4 (&ql)[8]) {
    uint2 left;
    const uint2 r = sa_round_q(x, left);
    const uint32_t row = s0 + (lane & 3) * 272, to = row + (lane >> 2) * 8;  // (256 bytes a row, and 16 so that rows lie in other banks)
    at_bf16x8 o[16];
    asm volatile(
        "ds_write_b64 %16, %18\n\tds_write_b64 %16, %19 offset:128\n\ts_waitcnt lgkmcnt(0)\n\t"
        "ds_read_b128 %0, %17\n\tds_read_b128 %1, %17 offset:16\n\tds_read_b128 %2, %17 offset:32\n\tds_read_b128 %3, %17 offset:48\n\t"
        "ds_read_b128 %4, %17 offset:64\n\tds_read_b128 %5, %17 offset:80\n\tds_read_b128 %6, %17 offset:96\n\tds_read_b128 %7, %17 offset:112\n\t"
        "ds_read_b128 %8, %17 offset:128\n\tds_read_b128 %9, %17 offset:144\n\tds_read_b128 %10, %17 offset:160\n\tds_read_b128 %11, %17 offset:176\n\t"
        "ds_read_b128 %12, %17 offset:192\n\tds_read_b128 %13, %17 offset:208\n\tds_read_b128 %14, %17 offset:224\n\tds_read_b128 %15, %17 offset:240\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]), "=&v"(o[4]), "=&v"(o[5]), "=&v"(o[6]), "=&v"(o[7]),
          "=&v"(o[8]), "=&v"(o[9]), "=&v"(o[10]), "=&v"(o[11]), "=&v"(o[12]), "=&v"(o[13]), "=&v"(o[14]), "=&v"(o[15])
        : "v"(to), "v"(row), "v"(__builtin_bit_cast(few_s16x4, r)), "v"(__builtin_bit_cast(few_s16x4, left))
        : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = __builtin_bit_cast(uint4, o[i]);
        ql[i] = __builtin_bit_cast(uint4, o[8 + i]);
    }
}
// A page's keys, lane by key (kr: its 16-byte pieces).
__device__ __forceinline__ void few_read_k(const uint32_t (&kr)[8], uint4 (&k)[8]) {
    at_bf16x8 x[8];
    asm volatile(
        "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
        "ds_read_b128 %4, %12\n\tds_read_b128 %5, %13\n\tds_read_b128 %6, %14\n\tds_read_b128 %7, %15\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(kr[0]), "v"(kr[1]), "v"(kr[2]), "v"(kr[3]), "v"(kr[4]), "v"(kr[5]), "v"(kr[6]), "v"(kr[7])
        : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = __builtin_bit_cast(uint4, x[i]);
}
// v[b] = values of keys 4 b .. 4 b + 3 in dim `lane` (vr: the lane's 8 bytes of keys 4 b .. + 3, b % 4).
__device__ __forceinline__ void few_read_v(const uint32_t (&vr)[4], uint64_t (&v)[16]) {
#define SA_TR(O, A, S) "ds_read_b64_tr_b16 %" #O ", %" #A " offset:" #S "\n\t"
    asm volatile(
        SA_TR(0, 16, 0) SA_TR(1, 17, 0) SA_TR(2, 18, 0) SA_TR(3, 19, 0) SA_TR(4, 16, 2048) SA_TR(5, 17, 2048) SA_TR(6, 18, 2048)
        SA_TR(7, 19, 2048) SA_TR(8, 16, 4096) SA_TR(9, 17, 4096) SA_TR(10, 18, 4096) SA_TR(11, 19, 4096) SA_TR(12, 16, 6144)
        SA_TR(13, 17, 6144) SA_TR(14, 18, 6144) SA_TR(15, 19, 6144) "s_waitcnt lgkmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7]),
          "=&v"(v[8]), "=&v"(v[9]), "=&v"(v[10]), "=&v"(v[11]), "=&v"(v[12]), "=&v"(v[13]), "=&v"(v[14]), "=&v"(v[15])
        : "v"(vr[0]), "v"(vr[1]), "v"(vr[2]), "v"(vr[3])
        : "memory");
#undef SA_TR
}
template <int... B>  // the blocks of 4 keys; pl: the weights' second parts
__device__ __forceinline__ void few_pv(FewState& a, few_s16x4 p, few_s16x4 pl, const uint64_t (&v)[16], std::integer_sequence<int, B...>) {
    ((a.o[0] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(p, __builtin_bit_cast(few_s16x4, v[B]), a.o[0], 4, B, 0),
      a.o[1] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(pl, __builtin_bit_cast(few_s16x4, v[B]), a.o[1], 4, B, 0)), ...);
}
// The wave's n pages, which fetch hands over one a lane, 64 at a time.
template <bool Q32, typename Fetch>
__device__ __forceinline__ void few_pages(const SharedAttnArgs& a, const RowTile& t, int n, char* own, int lane, FewState& st, Fetch fetch) {
    const size_t to_v = (size_t)a.n_kv_head * kAtTile;
    PageRef page{};
    auto load = [&](int j, int kv) {  // as shared_part_kernel's
        const int tokens = __builtin_amdgcn_readlane(page.tokens, j & 63);
        const char* src = page_at(a, page, j & 63) + kv * to_v;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = i * 8 + (lane >> 3);
            buffer_to_lds16(src, tokens * 128, own + kv * kAtTile + i * 1024, row * 128 + (((lane & 7) ^ ((row >> 1) & 7)) << 4), 0);
        }
        return tokens;
    };
    uint4 q[8], ql[Q32 ? 8 : 1];
    const size_t q0 = (size_t)max(t.row, 0) * a.q_ld + t.head * kHeadDim;
    float4 q32;  // Q32: lane (block, row) takes dims 4 block .. + 3 of the row
    if constexpr (Q32) {
        q32 = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + q0 + (lane & ~3));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.q) + q0 + 8 * i);
    }
    uint32_t kr[8], vr[4];
    {
        const uint32_t s0 = lds_address(own);
        const int i16 = lane & 15;
#pragma unroll
        for (int c = 0; c < 8; ++c) kr[c] = s0 + lane * 128 + ((c ^ ((lane >> 1) & 7)) << 4);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int row = 4 * b + (i16 >> 2), piece = 2 * (lane >> 4) + ((i16 & 3) >> 1);
            vr[b] = s0 + kAtTile + row * 128 + ((piece ^ ((row >> 1) & 7)) << 4) + (i16 & 1) * 8;
        }
    }
    int next = 0;
    if (n > 0) {
        page = fetch(0);
        st.saw = __any(page.tokens > 0);
        next = load(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (Q32) {
            few_exchange_q(q32, lds_address(own + kAtTile), lane, q, ql);
            __builtin_amdgcn_sched_barrier(0);
        }
        load(0, 1);
    }
    for (int j = 0; j < n; ++j) {
        const bool more = j + 1 < n;
        const int tokens = next;
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // K is in (this wave's own loads), V's 8 loads may be out
        __builtin_amdgcn_sched_barrier(0);
        uint4 k[8];
        few_read_k(kr, k);
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            if (((j + 1) & 63) == 0) {
                page = fetch(j + 1);
                st.saw |= __any(page.tokens > 0);
            }
            next = load(j + 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        few_f32x4 s[2] = {}, sl[2] = {};
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            s[0] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(few_op(k[c].x, k[c].y), few_op(q[c].x, q[c].y), s[0], 0, 0, 0);
            s[1] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(few_op(k[c].z, k[c].w), few_op(q[c].z, q[c].w), s[1], 0, 0, 0);
            if constexpr (Q32) {
                sl[0] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(few_op(k[c].x, k[c].y), few_op(ql[c].x, ql[c].y), sl[0], 0, 0, 0);
                sl[1] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(few_op(k[c].z, k[c].w), few_op(ql[c].z, ql[c].w), sl[1], 0, 0, 0);
            }
        }
        if constexpr (Q32) {
            s[0] += sl[0];
            s[1] += sl[1];
        }
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = (lane & ~3) + i < tokens ? s[0][i] + s[1][i] : -INFINITY;
        few_weights(st, p);
        uint32_t l0, l1;
        const uint32_t h0 = sa_split(p[0], p[1], l0), h1 = sa_split(p[2], p[3], l1);
        __builtin_amdgcn_sched_barrier(0);
        if (more) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // V is in, the next K may be out
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        uint64_t v[16];
        few_read_v(vr, v);
        __builtin_amdgcn_sched_barrier(0);
        if (more) load(j + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
        few_pv(st, few_op(h0, h1), few_op(l0, l1), v, std::make_integer_sequence<int, 16>{});
    }
}
template <bool Q32>
__device__ __forceinline__ void few_part(const SharedAttnArgs& a, const SharedPlan& pl, const PartWork& w, char* smem, int wave, int lane) {
    const int n = w.pages > wave ? (w.pages - wave + kSaWaves - 1) / kSaWaves : 0;  // this wave's pages
    FewState st;
    few_pages<Q32>(a, w.t, n, smem + wave * kAtStage, lane, st, [&](int j0) {
        const int j = w.page0 + wave + kSaWaves * (j0 + lane);
        const int id = j0 == 0 ? w.id0 : j0 + lane < n ? w.ids[j - w.page0] : -1;
        return page_ref(a, w.kh, 2, id, j0 + lane < n ? w.t.most - j * kPage : 0);
    });
    few_finish(pl, w, st, smem, wave, lane);
}

// bf16: the waves take a run's pages in turn (wave w: w, w + 2, ...) by direct-to-LDS loads into a stage of their own,
// the next page's K (V) on its way once this one's is in registers; no barrier in the loop.  The weights go into the
// products in two bf16 parts (sa_split), so that only the output is rounded (the second product is free where
// reading bounds).  PROMPT: several rows a sequence, so a tile's rows may see different tokens.
//
// Two waves a workgroup: one wave each measured 1-2 us better for 32 short sequences and 2 worse behind long prefixes,
// four 1-3 worse nearly everywhere (more idle waves at a run's end).  Calls in a row, the join included: 32 sequences of
// 64-700 tokens behind 1500, 20 heads, 17.8 us for 76 MB; 64 of 100-900 behind 16,001 53 us for 255 MB (a read reaches
// 5.9 TB/s: 12.9 and 43 us); 24 of up to 1200 behind 5000, 20 query and 4 key heads, 12.9 for 22 MB: there a chain of
// page ids, keys, products, values and the hand-over, not bytes.
template <bool PROMPT, bool Q32>
__global__ __launch_bounds__(kSaWaves * 64, 2) void shared_part_kernel(const SharedAttnArgs a, const SharedPlan pl) {
    __shared__ __attribute__((aligned(1024))) char smem[kSaWaves * kAtStage];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hh = lane >> 5;
    PartWork w;
    if (!part_work<!PROMPT>(a, pl, tid, w)) return;
    if (!PROMPT && w.size == kFew) return few_part<Q32>(a, pl, w, smem, wave, lane);
    const RowTile& t = w.t;
    char* own = smem + wave * kAtStage;
    const int n = w.pages > wave ? (w.pages - wave + kSaWaves - 1) / kSaWaves : 0;  // this wave's pages
    const size_t to_v = (size_t)a.n_kv_head * kAtTile;  // from a page's keys to its values
    PageRef page{};
    auto fetch = [&](int j0) {  // the wave's pages j0 .. j0 + 63, one a lane
        const int j = w.page0 + wave + kSaWaves * (j0 + lane);
        const int id = j0 == 0 ? w.id0 : j0 + lane < n ? w.ids[j - w.page0] : -1;
        page = page_ref(a, w.kh, 2, id, j0 + lane < n ? t.most - j * kPage : 0);
    };
    auto load = [&](int j, int kv) {  // the wave's page j, K (kv 0) or V; zeros for what is not seen
        const int tokens = __builtin_amdgcn_readlane(page.tokens, j & 63);
        const char* src = page_at(a, page, j & 63) + kv * to_v;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = i * 8 + (lane >> 3);
            buffer_to_lds16(src, tokens * 128, own + kv * kAtTile + i * 1024, row * 128 + (((lane & 7) ^ ((row >> 1) & 7)) << 4), 0);
        }
        return tokens > 0;
    };
    uint4 qr[4], ql[Q32 ? 4 : 1];
    const size_t q0 = (size_t)max(t.row, 0) * a.q_ld + t.head * kHeadDim;
    if constexpr (Q32) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const float4* qp = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + q0 + hh * 8 + kk * 16);
            uint2 l0, l1;
            const uint2 r0 = sa_round_q(qp[0], l0), r1 = sa_round_q(qp[1], l1);
            qr[kk] = make_uint4(r0.x, r0.y, r1.x, r1.y);
            ql[kk] = make_uint4(l0.x, l0.y, l1.x, l1.y);
        }
    } else {
        at_load_q(reinterpret_cast<const uint16_t*>(a.q) + q0, hh, qr);
    }
    const AtAddr ad = at_addresses(lds_address(own), lane);
    SaState st;
    sa_init(st);
    bool ok = false, saw = false;
    if (n > 0) {
        fetch(0);
        ok = load(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load(0, 1);
    }
    for (int j = 0; j < n; ++j) {
        const bool more = j + 1 < n, seen = ok;
        const int k0 = (w.page0 + wave + kSaWaves * j) * kPage;
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // K is in (this wave's own loads), V's 8 loads may be out
        __builtin_amdgcn_sched_barrier(0);
        uint4 ka[4], kb[4];
        sa_read_k<0>(ad, ka, kb);
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            if (((j + 1) & 63) == 0) fetch(j + 1);
            ok = load(j + 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        at_f32x16 s[2];
        at_scores(ka, kb, qr, s);
        if constexpr (Q32) sa_scores_left(ka, kb, ql, s);
        uint32_t pw[16], plo[16];
        const int lim = seen ? t.lim : 0;
        saw |= lim > k0;
        if (__any(lim < k0 + kAtK)) sa_mask(s, k0, lim, hh);
        sa_maximum(st, s);
        st.l += sa_weights<true>(st, s, pw, plo);
        __builtin_amdgcn_sched_barrier(0);
        if (more) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // V is in, the next K may be out
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        uint64_t v[2][2][4];
        sa_read_v<0>(ad, v);
        __builtin_amdgcn_sched_barrier(0);
        // (rows without a token in the tile have weights of 0, those past a tile's end zeros for values)
        if (PROMPT && __any(t.lim < min(t.most, k0 + kAtK)) && sa_not_finite(v, s)) {
            sa_add_not_finite(st, own + kAtTile, pw, lim - k0, hh);
            sa_read_v<0>(ad, v);
            sa_take_out(v);
        }
        if (more) load(j + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
        sa_pv(st, v, pw);
        sa_pv(st, v, plo);
    }
    st.m = sa_marked(st.m, saw);
    part_finish(pl, w, st, smem, wave, lane);
}

// fp32: the same on 32-token halves of pages (the same 16 KB a stage) with fp32 matrix products, all sums in fp32.  A
// 16-byte piece c of row r lies at c ^ (r % 16).  K as the first operand: lane (key, hh) holds dims 32 hh .. + 31, one
// a step; V: lane (dim, hh) holds the key that element i of the scores is for.  Bound by the products: 8192 cycles a
// wave and page, whatever the rows, so a wave takes one page where there are enough.
constexpr int kSfK = 32;
__device__ __forceinline__ void sf_read_k(const uint32_t (&kr)[8], float4 (&k)[8]) {
    at_bf16x8 x[8];  // (any 16-byte register type)
    asm volatile(
        "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
        "ds_read_b128 %4, %12\n\tds_read_b128 %5, %13\n\tds_read_b128 %6, %14\n\tds_read_b128 %7, %15\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(kr[0]), "v"(kr[1]), "v"(kr[2]), "v"(kr[3]), "v"(kr[4]), "v"(kr[5]), "v"(kr[6]), "v"(kr[7])
        : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = __builtin_bit_cast(float4, x[i]);
}
// v[i] = value of key (i/4)*8 + hh*4 + i%4 in dim lane % 32 (+ 32: the addresses of the other half of a row).
__device__ __forceinline__ void sf_read_v(const uint32_t (&a)[8], int flip, float (&v)[16]) {
#define SF_R(O, A, OFF) "ds_read_b32 %" #O ", %" #A " offset:" #OFF "\n\t"
    asm volatile(
        SF_R(0, 16, 0) SF_R(1, 17, 256) SF_R(2, 18, 512) SF_R(3, 19, 768)
        SF_R(4, 20, 2048) SF_R(5, 21, 2304) SF_R(6, 22, 2560) SF_R(7, 23, 2816)
        SF_R(8, 16, 4096) SF_R(9, 17, 4352) SF_R(10, 18, 4608) SF_R(11, 19, 4864)
        SF_R(12, 20, 6144) SF_R(13, 21, 6400) SF_R(14, 22, 6656) SF_R(15, 23, 6912)
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7]),
          "=&v"(v[8]), "=&v"(v[9]), "=&v"(v[10]), "=&v"(v[11]), "=&v"(v[12]), "=&v"(v[13]), "=&v"(v[14]), "=&v"(v[15])
        : "v"(a[0 ^ flip]), "v"(a[1 ^ flip]), "v"(a[2 ^ flip]), "v"(a[3 ^ flip]), "v"(a[4 ^ flip]), "v"(a[5 ^ flip]),
          "v"(a[6 ^ flip]), "v"(a[7 ^ flip])
        : "memory");
#undef SF_R
}
// As sa_add_not_finite.
__device__ __forceinline__ void sf_add_not_finite(SaState& a, const char* vt, const at_f32x16& pw, int seen, int hh) {
    at_f32x16 p = pw;
#pragma unroll 1
    for (int j = 0; j < 16; ++j) {
        const RowPair w = swap32(p[0]);
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
            const float pk = k ? w.b : w.a;
            const int key = (j >> 2) * 8 + k * 4 + (j & 3);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float4 v = *reinterpret_cast<const float4*>(vt + key * 256 + (((2 * c + hh) ^ (key & 15)) << 4));
                const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y = key < seen && !(fabsf(f[i]) < INFINITY) ? pk * f[i] : 0.f;
                    if (c < 4) a.o0[4 * (c & 3) + i] += y;
                    else a.o1[4 * (c & 3) + i] += y;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 15; ++i) p[i] = p[i + 1];
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// fp32, tiles of 4 rows: 1024 cycles of 4x4x1 products a page where a tile of 32 takes 8192.  K goes through LDS, whole
// pages; V's rows go straight into registers, lane by dim.  8 sequences of 30-500 tokens behind 700, 20 heads: 12.9 us
// with the join (tiles of 32: 19.2), 32 of them 24.6 (37.3); there bound by reading (105 MB), here by the chain.
__device__ __forceinline__ void sf_load_v(const char* src, int bytes, int lane, float (&v)[kPage]) {
#ifdef __HIP_DEVICE_COMPILE__
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(src), 0, bytes, 0x00020000);
#pragma unroll
    for (int k = 0; k < kPage; ++k)
        v[k] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, lane * 4 + k * 256, 0, 0));
#endif
}
template <int... B>  // the blocks of 4 keys
__device__ __forceinline__ void sf_few_pv(FewState& a, const float (&p)[4], const float (&v)[kPage], std::integer_sequence<int, B...>) {
    ((a.o[0] = __builtin_amdgcn_mfma_f32_4x4x1f32(p[0], v[4 * B], a.o[0], 4, B, 0),
      a.o[1] = __builtin_amdgcn_mfma_f32_4x4x1f32(p[1], v[4 * B + 1], a.o[1], 4, B, 0),
      a.o[0] = __builtin_amdgcn_mfma_f32_4x4x1f32(p[2], v[4 * B + 2], a.o[0], 4, B, 0),
      a.o[1] = __builtin_amdgcn_mfma_f32_4x4x1f32(p[3], v[4 * B + 3], a.o[1], 4, B, 0)), ...);
}
__device__ __forceinline__ void sf_few_part(const SharedAttnArgs& a, const SharedPlan& pl, const PartWork& w, char* smem, int wave, int lane) {
    const int n = w.pages > wave ? (w.pages - wave + kSaWaves - 1) / kSaWaves : 0;  // this wave's pages
    const size_t to_v = (size_t)a.n_kv_head * (kPage * kHeadDim * 4);
    char* own = smem + wave * kAtStage;
    PageRef page{};
    auto fetch = [&](int j0) {  // the wave's pages j0 .. j0 + 63, one a lane
        const int j = w.page0 + wave + kSaWaves * (j0 + lane);
        const int id = j0 == 0 ? w.id0 : j0 + lane < n ? w.ids[j - w.page0] : -1;
        page = page_ref(a, w.kh, 4, id, j0 + lane < n ? w.t.most - j * kPage : 0);
    };
    float4 q[16];
    {
        const float* qp = reinterpret_cast<const float*>(a.q) + (size_t)max(w.t.row, 0) * a.q_ld + w.t.head * kHeadDim;
#pragma unroll
        for (int i = 0; i < 16; ++i) q[i] = *reinterpret_cast<const float4*>(qp + 4 * i);
    }
    FewState st;
    float v[kPage];
    for (int u = 0; u < n; ++u) {
        if ((u & 63) == 0) {
            fetch(u);
            st.saw |= __any(page.tokens > 0);
        }
        const int tokens = __builtin_amdgcn_readlane(page.tokens, u & 63);
        const char* src = page_at(a, page, u & 63);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = i * 4 + (lane >> 4);
            buffer_to_lds16(src, tokens * 256, own + i * 1024, row * 256 + (((lane & 15) ^ (row & 15)) << 4), 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        sf_load_v(src + to_v, tokens * 256, lane, v);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(63)" ::: "memory");  // the 16 loads of K are in, 63 of V's 64 may be out
        __builtin_amdgcn_sched_barrier(0);
        few_f32x4 s[4] = {};
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            const float4 k = *reinterpret_cast<const float4*>(own + lane * 256 + ((c ^ (lane & 15)) << 4));
            s[0] = __builtin_amdgcn_mfma_f32_4x4x1f32(k.x, q[c].x, s[0], 0, 0, 0);
            s[1] = __builtin_amdgcn_mfma_f32_4x4x1f32(k.y, q[c].y, s[1], 0, 0, 0);
            s[2] = __builtin_amdgcn_mfma_f32_4x4x1f32(k.z, q[c].z, s[2], 0, 0, 0);
            s[3] = __builtin_amdgcn_mfma_f32_4x4x1f32(k.w, q[c].w, s[3], 0, 0, 0);
        }
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = (lane & ~3) + i < tokens ? (s[0][i] + s[1][i]) + (s[2][i] + s[3][i]) : -INFINITY;
        few_weights(st, p);
        sf_few_pv(st, p, v, std::make_integer_sequence<int, 16>{});
        __builtin_amdgcn_sched_barrier(0);
    }
    few_finish(pl, w, st, smem, wave, lane);
}

template <bool PROMPT>
__global__ __launch_bounds__(kSaWaves * 64, 2) void shared_part_f32_kernel(const SharedAttnArgs a, const SharedPlan pl) {
    __shared__ __attribute__((aligned(1024))) char smem[kSaWaves * kAtStage];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ql = lane & 31, hh = lane >> 5;
    PartWork w;
    if (!part_work<!PROMPT>(a, pl, tid, w)) return;
    if (!PROMPT && w.size == kFew) return sf_few_part(a, pl, w, smem, wave, lane);
    const RowTile& t = w.t;
    char* own = smem + wave * kAtStage;
    const int n = w.pages > wave ? 2 * ((w.pages - wave + kSaWaves - 1) / kSaWaves) : 0;  // this wave's half pages
    const size_t to_v = (size_t)a.n_kv_head * (kPage * kHeadDim * 4);  // from a page's keys to its values
    PageRef page{};
    auto fetch = [&](int j0) {  // the wave's pages j0 .. j0 + 63, one a lane
        const int j = w.page0 + wave + kSaWaves * (j0 + lane);
        const int id = j0 == 0 ? w.id0 : 2 * (j0 + lane) < n ? w.ids[j - w.page0] : -1;
        page = page_ref(a, w.kh, 4, id, 2 * (j0 + lane) < n ? t.most - j * kPage : 0);
    };
    auto first = [&](int u) { return (w.page0 + wave + kSaWaves * (u >> 1)) * kPage + (u & 1) * kSfK; };
    auto load = [&](int u, int kv) {  // half page u, K (kv 0) or V; zeros for what is not seen
        const int j = (u >> 1) & 63, tokens = __builtin_amdgcn_readlane(page.tokens, j);
        const char* src = page_at(a, page, j) + kv * to_v + (u & 1) * kAtTile;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = i * 4 + (lane >> 4);
            buffer_to_lds16(src, max(min(tokens - (u & 1) * kSfK, kSfK), 0) * 256, own + kv * kAtTile + i * 1024,
                            row * 256 + (((lane & 15) ^ (row & 15)) << 4), 0);
        }
        return tokens > 0;
    };
    float4 q[8];
    {
        const float* qp = reinterpret_cast<const float*>(a.q) + (size_t)max(t.row, 0) * a.q_ld + t.head * kHeadDim + hh * 32;
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = *reinterpret_cast<const float4*>(qp + 4 * i);
    }
    uint32_t kr[8], vr[8];
    {
        const uint32_t s0 = lds_address(own);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            kr[c] = s0 + ql * 256 + (((hh * 8 + c) ^ (ql & 15)) << 4);
            // c = 4 (i / 4 % 2) + i % 4 for element i
            vr[c] = s0 + kAtTile + hh * 1024 + (((ql >> 2) ^ ((c >> 2) * 8 + hh * 4 + (c & 3))) << 4) + (ql & 3) * 4;
        }
    }
    SaState st;
    sa_init(st);
    bool ok = false, saw = false;
    if (n > 0) {
        fetch(0);
        ok = load(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load(0, 1);
    }
    for (int u = 0; u < n; ++u) {
        const bool more = u + 1 < n, seen = ok;
        const int k0 = first(u);
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // K is in (this wave's own loads), V's 8 loads may be out
        __builtin_amdgcn_sched_barrier(0);
        float4 k[8];
        sf_read_k(kr, k);
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            if (((u + 1) & 127) == 0) fetch((u + 1) >> 1);
            ok = load(u + 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        at_f32x16 s[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i].x, q[i].x, s[0], 0, 0, 0);
            s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i].y, q[i].y, s[0], 0, 0, 0);
            s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i].z, q[i].z, s[0], 0, 0, 0);
            s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i].w, q[i].w, s[0], 0, 0, 0);
        }
        const int lim = seen ? t.lim : 0;
        saw |= lim > k0;
        if (__any(lim < k0 + kSfK)) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (k0 + (i >> 2) * 8 + hh * 4 + (i & 3) >= lim) s[0][i] = -INFINITY;
        }
        sa_maximum(st, s);
        const float ref = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[0][i] = __builtin_amdgcn_exp2f(fmaf(s[0][i], kSaScale, -ref));
            st.l += s[0][i];
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // V is in, the next K may be out
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        float v0[16], v1[16];
        sf_read_v(vr, 0, v0);
        sf_read_v(vr, 4, v1);
        __builtin_amdgcn_sched_barrier(0);
        if (PROMPT && __any(t.lim < min(t.most, k0 + kSfK))) {
            float z = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) z = fmaf(v0[i], 0.f, fmaf(v1[i], 0.f, z));
            if (__any(z != 0.f)) {  // (NaN: a value that is not finite, in a tile that some row sees in part)
                sf_add_not_finite(st, own + kAtTile, s[0], lim - k0, hh);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    v0[i] = fabsf(v0[i]) < INFINITY ? v0[i] : 0.f;
                    v1[i] = fabsf(v1[i]) < INFINITY ? v1[i] : 0.f;
                }
            }
        }
        if (more) load(u + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            st.o0 = __builtin_amdgcn_mfma_f32_32x32x2f32(v0[i], s[0][i], st.o0, 0, 0, 0);
            st.o1 = __builtin_amdgcn_mfma_f32_32x32x2f32(v1[i], s[0][i], st.o1, 0, 0, 0);
        }
    }
    st.m = sa_marked(st.m, saw);
    part_finish(pl, w, st, smem, wave, lane);
}

// The rows of a workgroup of shared_tile_kernel, (token, head) pairs first .. end - 1 counted over all rows, and the chain of
// pages that they see: the prefix's, then their sequences' own, sequence after sequence.  Sequence i is lane i's.
struct TilePages {
    int first, end, n_pre, n_own;
    uint64_t seqs;              // the sequences with rows here
    int row0, n, len;           // a sequence's first row, rows and length
    int most, start;            // its own tokens that some row here sees, its first page's place among all own ones
};
// PACK: tiles of all rows, whatever sequence they are of; else each sequence's rows begin a tile.
template <bool PACK>
__device__ __forceinline__ TilePages tile_pages(const SharedAttnArgs& a, int tile, int size, int lane) {
    static_assert(FTTS_MAX_BATCH <= kWave, "one sequence per lane");
    const int g = a.n_head / a.n_kv_head;
    const bool in = lane < a.B;
    const int lo = in ? a.row_offsets[lane] : 0, hi = in ? a.row_offsets[lane + 1] : 0;
    TilePages t;
    t.len = in ? a.seq_lens[lane] : -1;
    t.row0 = min(max(lo, 0), a.rows);
    t.n = min(max(hi, t.row0), a.rows) - t.row0;
    if constexpr (PACK) {
        t.first = tile * size;
        t.end = min(t.first + size, a.rows * g);  // (rows * n_head < 2^31)
        t.seqs = __ballot(t.n > 0 && t.row0 <= (t.end - 1) / g && t.row0 + t.n > t.first / g);
    } else {
        const int own = (t.n * g + size - 1) / size;
        int upto = own;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int u = __shfl_up(upto, d, kWave);
            if (lane >= d) upto += u;
        }
        const int b = __popcll(__ballot(in && upto <= tile));
        if (b >= a.B) {
            t.first = t.end = 0;
            return t;
        }
        const int r0 = __builtin_amdgcn_readlane(t.row0, b);
        t.first = r0 * g + (tile - __builtin_amdgcn_readlane(upto - own, b)) * size;
        t.end = min(t.first + size, (r0 + __builtin_amdgcn_readlane(t.n, b)) * g);
        t.seqs = 1ull << b;
    }
    const bool here = t.seqs >> lane & 1;
    t.most = here ? own_seen(a, t.len, t.n, min((t.end - 1) / g - t.row0, t.n - 1)) : 0;
    t.n_pre = __any(here && t.len >= 0) ? (a.prefix_len + kPage - 1) / kPage : 0;
    const int pages = (t.most + kPage - 1) / kPage;
    int upto = pages;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int u = __shfl_up(upto, d, kWave);
        if (lane >= d) upto += u;
    }
    t.start = upto - pages;
    t.n_own = __builtin_amdgcn_readlane(upto, kWave - 1);
    return t;
}

// Many rows: one workgroup per key head and run of 128 rows, whose waves (32 rows each) share 64-token tiles of the
// prefix and then of the sequences' own pages.  Where many short prompts follow a long prefix a run goes over sequences'
// ends (packed: a wave passes the own pages of sequences that it has no row of), else each sequence begins one.  Tiles
// come in whole pages of a head, 8 KB of keys and of values, by direct-to-LDS loads into two stages, a tile ahead; one
// barrier a tile; three workgroups a CU.  The weights go into the products as bf16, rounded once as in the
// prefill's own attention, and their sum takes the rounded ones (error against 64 bits 2.3e-3; two parts as in the cut
// would give 1.7e-3 for a quarter more time).
//
// Four prompts of 1500-2300 rows behind 8000 tokens, 20 heads: 491 us, 800 TFLOP/s (a library product of 8192^3: 1460);
// 32 of 20-220 behind 600 36 us (a tile for each sequence: 44).  Counted for the long ones: matrix units busy 34% of the
// time, vector units 49% (32 exponentials of 8 cycles and about 114 operations of 4 a tile of 32 rows and a page), both
// at once 10%, and 15% of the units' time at the launch's ends.  Measured and not taken: three stages, 64 rows a wave
// (spills), two waves a workgroup (more loads), the next tile's scores under this one's exponentials (two waves a SIMD:
// 637 us), half a tile's weights under the other half's products (spills: 525), the maximum of the first tile alone with
// a second pass where a sum overflows (488, not worth its second path).
constexpr int kStWaves = 4;
template <bool PACK, bool CUT>
__global__ __launch_bounds__(kStWaves * 64, 3) void shared_tile_kernel(const SharedAttnArgs a, int tiles, const SharedPlan pl) {
    constexpr int kRows = kStWaves * kSaQ, kLoads = 8 / kStWaves;
    __shared__ __attribute__((aligned(1024))) char smem[2 * kAtStage];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ql = lane & 31, hh = lane >> 5;
    // Each XCD (workgroups are dealt to the 8 in turn) gets a contiguous run of (key head, tile), tiles fastest, so
    // that a head's pages are read through one L2.
    int tile, kh, part = 0;
    {
        const int T = gridDim.x, i = blockIdx.x, x = i & 7, q = T >> 3, r = T & 7;
        const int t = (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + (i >> 3);
        tile = t % tiles;
        kh = t / tiles;
        if constexpr (CUT) {
            part = kh % pl.s_pre;
            kh /= pl.s_pre;
        }
    }
    const int g = a.n_head / a.n_kv_head;
    const TilePages o = tile_pages<PACK>(a, tile, kRows, lane);
    if (o.first >= o.end) return;
    const int P = a.prefix_len, all = o.n_pre + o.n_own;
    const int per = CUT ? (all + pl.s_pre - 1) / pl.s_pre : all, j0 = CUT ? min(part * per, all) : 0, n = min(per, all - j0);
    // This lane's pair, the tile's last one where it is past it (which is not written twice).
    const int pair = o.first + wave * kSaQ + ql, row = min(pair, o.end - 1) / g, head = kh * g + min(pair, o.end - 1) % g;
    bool inactive = false;
    int seq = -1, own_lim = 0, pre_lim = 0;  // its sequence, the own tokens and those of the prefix that it sees
    for (uint64_t m = o.seqs; m; m &= m - 1) {
        const int b = __builtin_ctzll(m), r0 = __builtin_amdgcn_readlane(o.row0, b), rn = __builtin_amdgcn_readlane(o.n, b);
        const int len = __builtin_amdgcn_readlane(o.len, b);
        if (row < r0 || row >= r0 + rn) continue;
        seq = b;
        own_lim = own_seen(a, len, rn, row - r0);
        inactive = len < 0;
        pre_lim = inactive ? 0 : P;
    }
    const bool rows = o.first + wave * kSaQ < o.end;
    SaState st;
    sa_init(st);
    uint4 qr[4];
    at_load_q(reinterpret_cast<const uint16_t*>(a.q) + (size_t)row * a.q_ld + head * kHeadDim, hh, qr);
    const size_t to_v = (size_t)a.n_kv_head * kAtTile;  // from a page's keys to its values
    PageRef page{};
    int whose = 0;  // the page's sequence (kWave: the prefix) and its number there, in the low 24 bits
    auto fetch = [&](int i) {  // the workgroup's pages i .. i + 63, one a lane
        const int j = j0 + i + lane, own = j - o.n_pre;
        const int32_t* id = own < 0 ? a.prefix_pages + j : nullptr;
        int left = P - j * kPage;
        whose = kWave << 24 | j;
        for (uint64_t m = o.seqs; m; m &= m - 1) {
            const int b = __builtin_ctzll(m), k = own - __builtin_amdgcn_readlane(o.start, b);
            const int most = __builtin_amdgcn_readlane(o.most, b);
            if (k < 0 || own < 0 || k * kPage >= most) continue;
            id = a.block_table + (size_t)b * a.max_pages + k;
            left = most - k * kPage;
            whose = b << 24 | k;
        }
        page = page_ref(a, kh, 2, id && j < all ? *id : -1, left);
    };
    uint32_t vo[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = (wave * kLoads + i) * 8 + (lane >> 3);
        vo[i] = row * 128 + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
    }
    auto load = [&](int j, int so) {  // this wave's part of tile j into the stage at so; zeros for what is not seen
        if ((j & 63) == 0) fetch(j);
        const int tokens = __builtin_amdgcn_readlane(page.tokens, j & 63);
        const char* src = page_at(a, page, j & 63);
        char* dst = smem + so + wave * kLoads * 1024;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            buffer_to_lds16(src, tokens * 128, dst + i * 1024, vo[i], 0);
            buffer_to_lds16(src + to_v, tokens * 128, dst + kAtTile + i * 1024, vo[i], 0);
        }
        return tokens;
    };
    const AtAddr ad = at_addresses(lds_address(smem), lane);
    bool saw = false;
    int next = n > 0 ? load(0, 0) : 0, next_whose = n > 0 ? __builtin_amdgcn_readlane(whose, 0) : 0;
    auto step = [&](auto stage, int j) {  // tile j, in the stage at SO
        constexpr int SO = decltype(stage)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's loads of tile j
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();  // tile j is in; every wave has read tile j - 1
        __builtin_amdgcn_sched_barrier(0);
        const int tokens = next, of = next_whose >> 24, k0 = (next_whose & 0xFFFFFF) * kPage;
        if (j + 1 < n) {
            next = load(j + 1, kAtStage - SO);
            next_whose = __builtin_amdgcn_readlane(whose, (j + 1) & 63);
        }
        const int lim = of == kWave ? pre_lim : !PACK || of == seq ? own_lim : 0;
        if (tokens == 0 || !rows || !__any(lim > k0)) return;  // nothing for this wave
        saw |= lim > k0;
        const bool mask = __any(lim < k0 + kAtK);
        uint4 ka[4], kb[4];
        at_f32x16 s[2];
        uint64_t v[2][2][4];
        uint32_t pw[16], none[1];
        sa_read_k<SO>(ad, ka, kb);
        __builtin_amdgcn_sched_barrier(0);
        at_scores(ka, kb, qr, s);
        __builtin_amdgcn_sched_barrier(0);
        sa_read_v<SO>(ad, v);
        __builtin_amdgcn_sched_barrier(0);
        if (mask) sa_mask(s, k0, lim, hh);
        sa_maximum(st, s);
        st.l += sa_weights<false>(st, s, pw, none);
        if (mask && __any(lim < k0 + tokens) && sa_not_finite(v, s)) {
            sa_add_not_finite(st, smem + SO + kAtTile, pw, lim - k0, hh);
            sa_read_v<SO>(ad, v);
            sa_take_out(v);
        }
        sa_pv(st, v, pw);
    };
    for (int j = 0; j < n; j += 2) {
        step(std::integral_constant<int, 0>{}, j);
        if (j + 1 < n) step(std::integral_constant<int, kAtStage>{}, j + 1);
    }
    const RowPair ls = swap32(st.l);
    st.m = sa_marked(st.m, saw);
    const float l = ls.a + ls.b, inv = sa_inverse(l, st.m);
    if constexpr (CUT) {
        if (pair >= o.end || seq < 0) return;
        const int64_t at = part * ((int64_t)a.rows * a.n_head) + (int64_t)row * a.n_head + head;
        if (hh == 0) pl.ml[at] = make_float2(st.m, inactive ? -1.f : l);
        float4* to = reinterpret_cast<float4*>(pl.o + at * kHeadDim) + hh;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            to[2 * e] = make_float4(st.o0[4 * e], st.o0[4 * e + 1], st.o0[4 * e + 2], st.o0[4 * e + 3]);
            to[8 + 2 * e] = make_float4(st.o1[4 * e], st.o1[4 * e + 1], st.o1[4 * e + 2], st.o1[4 * e + 3]);
        }
        return;
    }
    uint16_t* out = reinterpret_cast<uint16_t*>(a.o) + (size_t)row * a.o_ld + head * kHeadDim + hh * 8;
    const bool write = pair < o.end && seq >= 0;
    // 8 dims of a piece are in both halves of the wave: one half takes even pieces, the other odd ones
#pragma unroll
    for (int g4 = 0; g4 < 8; g4 += 2) {
        const at_f32x16& x = g4 < 4 ? st.o0 : st.o1;
        const int e = 4 * (g4 & 3);
        const auto r0 = __builtin_amdgcn_permlane32_swap(bf16x2_rne(x[e] * inv, x[e + 1] * inv), bf16x2_rne(x[e + 4] * inv, x[e + 5] * inv), false, false);
        const auto r1 = __builtin_amdgcn_permlane32_swap(bf16x2_rne(x[e + 2] * inv, x[e + 3] * inv), bf16x2_rne(x[e + 6] * inv, x[e + 7] * inv), false, false);
        if (write) *reinterpret_cast<uint4*>(out + g4 * 8) = make_uint4(r0[0], r1[0], r0[1], r1[1]);
    }
}

// Short contexts, one row a sequence: one workgroup per key head and sequence takes the prefix's pages and the
// sequence's own, its waves in turn, and writes the result at once: the prefix is read by every sequence (through
// L2), but there is one launch and no partial.  Bound by its chain (ids, keys, products, values, hand-over): 4
// sequences of up to 90 tokens behind 134, 20 heads, 5.3 us (cut: 7.2).  FEW: up to 4 query heads a key head, in tiles
// of 4 rows (of 32: 6.4); the decode step's form (Q32) has one query head a key head.
constexpr int kSwWaves = 4;
template <bool Q32, bool FEW>
__global__ __launch_bounds__(kSwWaves * 64, 2) void shared_whole_kernel(const SharedAttnArgs a) {
    static_assert(FEW || !Q32, "fp32 queries come in tiles of 4 rows");
    __shared__ __attribute__((aligned(1024))) char smem[kSwWaves * kAtStage];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hh = lane >> 5;
    const int kh = blockIdx.x % a.n_kv_head;
    const int n_pre = (a.prefix_len + kPage - 1) / kPage, j0 = wave + kSwWaves * lane;
    constexpr int size = FEW ? kFew : kSaQ;
    const OwnTile o = own_tile(a, blockIdx.x / a.n_kv_head, size, lane);
    const int id0 = early_id(j0 < n_pre ? a.prefix_pages + j0
                                        : a.block_table + (size_t)o.b * a.max_pages + min(j0 - n_pre, a.max_pages - 1));
    const RowTile t = own_rows(a, o, o.first, size, kh, lane & (size - 1));
    const int P = a.prefix_len, pages = t.inactive ? 0 : n_pre + (t.most + kPage - 1) / kPage;
    const int n = pages > wave ? (pages - wave + kSwWaves - 1) / kSwWaves : 0;  // this wave's pages: wave, wave + 4, ...
    char* own = smem + wave * kAtStage;
    const size_t to_v = (size_t)a.n_kv_head * kAtTile;  // from a page's keys to its values
    // lane i: the wave's i-th page (the launcher bounds them by 64)
    const PageRef page = page_ref(a, kh, 2, id0, j0 >= pages ? 0 : j0 < n_pre ? P - j0 * kPage : t.most - (j0 - n_pre) * kPage);
    if constexpr (FEW) {
        FewState few;
        few_pages<Q32>(a, t, n, own, lane, few, [&](int) { return page; });
        few.o[0] += few.o[1];
        few.m = sa_marked(few.m, few.saw);
#pragma unroll
        for (int d = 4; d < kWave; d <<= 1) few.l += __shfl_xor(few.l, d, kWave);
        __syncthreads();
        float* mrg = reinterpret_cast<float*>(smem);  // [4][6][64]
        float* mw = mrg + wave * 6 * 64 + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) mw[i * 64] = few.o[0][i];
        mw[4 * 64] = few.m;
        mw[5 * 64] = few.l;
        __syncthreads();
        static_assert(kSwWaves == kFew, "a wave sums a row");
        const int row = __shfl(t.row, wave, kWave), head = __shfl(t.head, wave, kWave);
        if (row < 0) return;
        float mm = -INFINITY, l = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < kSwWaves; ++w) mm = fmaxf(mm, mrg[(w * 6 + 4) * 64 + wave]);
        const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
        for (int w = 0; w < kSwWaves; ++w) {
            const float f = exp2f(mrg[(w * 6 + 4) * 64 + wave] - ref);
            l += mrg[(w * 6 + 5) * 64 + wave] * f;
            x += mrg[(w * 6 + wave) * 64 + lane] * f;
        }
        x *= sa_inverse(l, mm);
        const size_t at = (size_t)row * a.o_ld + head * kHeadDim + lane;
        if (Q32 && a.o_f32) reinterpret_cast<float*>(a.o)[at] = x;
        else reinterpret_cast<uint16_t*>(a.o)[at] = (uint16_t)bf16x2_rne(x, 0.f);
        return;
    }
    auto load = [&](int i, int kv) {  // the wave's i-th page, K (kv 0) or V; zeros for what is not seen
        const int tokens = __builtin_amdgcn_readlane(page.tokens, i);
        const char* src = page_at(a, page, i) + kv * to_v;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int row = k * 8 + (lane >> 3);
            buffer_to_lds16(src, tokens * 128, own + kv * kAtTile + k * 1024, row * 128 + (((lane & 7) ^ ((row >> 1) & 7)) << 4), 0);
        }
    };
    uint4 qr[4];
    at_load_q(reinterpret_cast<const uint16_t*>(a.q) + (size_t)max(t.row, 0) * a.q_ld + t.head * kHeadDim, hh, qr);
    const AtAddr ad = at_addresses(lds_address(own), lane);
    SaState st;
    sa_init(st);
    if (n > 0) {
        load(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load(0, 1);
    }
    for (int i = 0; i < n; ++i) {
        const bool more = i + 1 < n;
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // K is in (this wave's own loads), V's 8 loads may be out
        __builtin_amdgcn_sched_barrier(0);
        uint4 ka[4], kb[4];
        sa_read_k<0>(ad, ka, kb);
        __builtin_amdgcn_sched_barrier(0);
        if (more) load(i + 1, 0);
        __builtin_amdgcn_sched_barrier(0);
        at_f32x16 s[2];
        at_scores(ka, kb, qr, s);
        uint32_t pw[16], plo[16];
        const int lim = __builtin_amdgcn_readlane(page.tokens, i);  // (all rows see as much)
        if (lim < kAtK) sa_mask(s, 0, lim, hh);
        sa_maximum(st, s);
        st.l += sa_weights<true>(st, s, pw, plo);
        __builtin_amdgcn_sched_barrier(0);
        if (more) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // V is in, the next K may be out
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        uint64_t v[2][2][4];
        sa_read_v<0>(ad, v);
        __builtin_amdgcn_sched_barrier(0);
        if (more) load(i + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
        sa_pv(st, v, pw);
        sa_pv(st, v, plo);
    }
    st.m = sa_marked(st.m, __any(page.tokens > 0));
    // the waves' (m, l, O) through LDS, lane for lane; each wave then sums a quarter of the dims
    __syncthreads();
    float* mrg = reinterpret_cast<float*>(smem);  // [4][34][64]
    {
        float* mw = mrg + wave * 34 * 64;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            mw[i * 64 + lane] = st.o0[i];
            mw[(16 + i) * 64 + lane] = st.o1[i];
        }
        mw[32 * 64 + lane] = st.m;
        mw[33 * 64 + lane] = st.l;
    }
    __syncthreads();
    float mm = -INFINITY, l = 0.f, x[8];
#pragma unroll
    for (int w = 0; w < kSwWaves; ++w) mm = fmaxf(mm, mrg[(w * 34 + 32) * 64 + lane]);
    const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
    for (int w = 0; w < kSwWaves; ++w) {
        const float* mw = mrg + w * 34 * 64;
        const float f = exp2f(mw[32 * 64 + lane] - ref);
        l += mw[33 * 64 + lane] * f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += mw[(8 * wave + i) * 64 + lane] * f;
    }
    const RowPair ls = swap32(l);
    const float inv = sa_inverse(ls.a + ls.b, mm);
    if (t.row < 0) return;
    // element 8 wave + i: dims 16 wave + 8 (i / 4) + 4 hh + i % 4
    const size_t at = (size_t)t.row * a.o_ld + t.head * kHeadDim + 16 * wave + 4 * hh;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const float y[4] = {x[4 * g] * inv, x[4 * g + 1] * inv, x[4 * g + 2] * inv, x[4 * g + 3] * inv};
        *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.o) + at + 8 * g) = make_uint2(bf16x2_rne(y[0], y[1]), bf16x2_rne(y[2], y[3]));
    }
}

// Joins the partials, one wave per (row, head): lane s weighs slot s (64 at a time), then 4 groups of 16 lanes sum
// every fourth slot, 4 dims a lane (16 lanes that walk all slots in turn took 20 us for 25 slots of 480 rows; this 5).
constexpr int kJoinWaves = 4, kJoinEarly = 4;
template <bool F32>
__global__ __launch_bounds__(kJoinWaves * 64) void shared_join_kernel(const SharedAttnArgs a, const SharedPlan pl) {
    const int lane = threadIdx.x & 63;
    const int64_t rows_heads = (int64_t)a.rows * a.n_head, rh = (int64_t)blockIdx.x * kJoinWaves + (threadIdx.x >> 6);
    if (rh >= rows_heads) return;
    const int r = (int)(rh / a.n_head), h = (int)(rh % a.n_head), grp = lane >> 4, d = (lane & 15) * 4;
    if (a.row_offsets && (r < a.row_offsets[0] || r >= a.row_offsets[a.B])) return;
    const int S = pl.s_pre + pl.s_own;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    bool inactive = false;
    for (int s0 = 0; s0 < S; s0 += kWave) {
        const float2 x = s0 + lane < S ? pl.ml[(s0 + lane) * rows_heads + rh] : make_float2(-INFINITY, 0.f);
        auto partial = [&](int s) { return *reinterpret_cast<const float4*>(pl.o + ((s0 + s) * rows_heads + rh) * kHeadDim + d); };
        float4 early[kJoinEarly];  // asked for with the weights; where nothing was written the weight is 0 and they are dropped
#pragma unroll
        for (int i = 0; i < kJoinEarly; ++i) early[i] = partial(min(4 * i + grp, min(kWave, S - s0) - 1));
        inactive |= __any(x.y < 0.f);
        const float mn = fmaxf(m, wave_max(x.x)), ref = mn == -INFINITY ? 0.f : mn;
        const float f = x.y == 0.f ? 0.f : exp2f(x.x - ref);  // (a sum of 0: nothing seen there, and nothing written)
        const float keep = exp2f(m - ref);
        m = mn;
        l = l * keep + wave_sum(x.y == 0.f ? 0.f : x.y * f);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= keep;
        const int n = min(kWave, S - s0);
        const unsigned long long live = __ballot(x.y != 0.f);
        auto add = [&](int s4, const float4& y) {  // (every lane stays: the weights come from all of them)
            const int s = s4 + grp;
            const float w = __shfl(f, s & 63, kWave);
            if (s >= n || !(live >> s & 1)) return;
            o[0] = fmaf(y.x, w, o[0]);
            o[1] = fmaf(y.y, w, o[1]);
            o[2] = fmaf(y.z, w, o[2]);
            o[3] = fmaf(y.w, w, o[3]);
        };
#pragma unroll
        for (int i = 0; i < kJoinEarly; ++i) add(4 * i, early[i]);
#pragma unroll 4
        for (int s4 = 4 * kJoinEarly; s4 < n; s4 += 4) {
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            if (s4 + grp < n) y = partial(s4 + grp);
            add(s4, y);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const RowPair p16 = swap16(o[i]);
        const float half = p16.a + p16.b;
        const RowPair p32 = swap32(half);
        o[i] = p32.a + p32.b;
    }
    if (grp != 0) return;
    const float inv = inactive ? 0.f : sa_inverse(l, m);
    if (inactive) o[0] = o[1] = o[2] = o[3] = 0.f;
    const size_t at = (size_t)r * a.o_ld + h * kHeadDim + d;
    if constexpr (F32)
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.o) + at) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    else
        *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.o) + at) =
            make_uint2(bf16x2_rne(o[0] * inv, o[1] * inv), bf16x2_rne(o[2] * inv, o[3] * inv));
}

// Pages a workgroup.  Own side: 4 (two a wave; fp32, bound by its products: one a wave), more where the table is so
// wide that the grid would pass kOwnGroups workgroups (most of them past their sequence's end).  Prefix: so many that
// about kPreFew workgroups share it (few rows: bound by reading, and each workgroup leaves 8 KB of partials) or
// kPreMany (many rows, or fp32: bound by the products), at most kMaxSplit along it.
//
// Tiles of 4 rows (one row a sequence): a sequence's own rows and the prefix's take them where they are up to 4 a key
// head.  fp32: they cost each row as much in products as tiles of 32, but read the pages 8 times as often.  So a
// sequence's own rows take them up to 8 a key head (two tiles), and the prefix's also up to 16 or where the whole prefix
// is little work (a tile, key head and page each): 4 sequences of 20/4 heads behind 700 8.6 us (32 rows: 11.8),
// 16 of 12/12 behind 3000 15.2 (18.9), 32 of 20/20 behind 700 27.7 (24.7).
constexpr int kOwnGroups = 8192, kPreFew = 256, kPreMany = 640, kMaxSplit = 64;
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

static SharedPlan shared_plan(bool f32, int n_head, int n_kv_head, int B, int rows, bool prompt, int prefix_len, int max_pages) {
    const int g = n_head / n_kv_head;
    const int64_t pages = ceil_div(prefix_len, kPage);
    SharedPlan p{};
    const int64_t few = prompt ? 0 : ceil_div((int64_t)rows * g, kFew);
    p.q_pre = few && (f32 ? few <= 4 || few * n_kv_head * pages <= 1024 : few == 1) ? kFew : kSaQ;
    p.q_own = few && g <= (f32 ? 2 : 1) * kFew ? kFew : kSaQ;
    p.row_tiles = (int)ceil_div((int64_t)rows * g, p.q_pre);
    p.own_tiles = prompt ? (int)((int64_t)rows * g / kSaQ) + B : B * (int)ceil_div(g, p.q_own);
    const int64_t groups = f32 || p.row_tiles > 4 ? kPreMany : kPreFew;
    const int64_t c_pre = std::max({(int64_t)2, ceil_div(pages * n_kv_head * p.row_tiles, groups), ceil_div(pages, kMaxSplit)});
    const int64_t c_own = std::max((int64_t)(f32 ? 2 : 4), ceil_div((int64_t)max_pages * n_kv_head * p.own_tiles, kOwnGroups));
    p.c_pre = (int)std::min(ceil_div(c_pre, 2) * 2, std::max(pages, (int64_t)1));
    p.c_own = (int)std::min(ceil_div(c_own, 2) * 2, (int64_t)max_pages);
    p.s_pre = (int)ceil_div(pages, p.c_pre);
    p.s_own = (int)ceil_div(max_pages, p.c_own);
    return p;
}

// How shared_tile_kernel takes a call: 128-row tiles, whether they go over sequences' ends, and the workgroups along a
// tile's chain of pages.
struct TilePlan {
    int tiles, parts;  // tiles 0: the call is cut into tiles of 32
    bool pack;
};
// A tile's pages are one chain, 0.8 us a page (packed: 0.88) while a unit has one workgroup, 256 of them, and so many
// times that where it has more; in its own tiles a sequence has half of one to spare, packed it meets the own pages of
// 1 + (B - 1) / tiles sequences.  Parts of a chain pay for another launch and a row's partials, 0.7 us a page (packed:
// 0.77), and half a round of units more where the last one is not full.  Tiles of 32 pay for the other launch, 1.65 ns
// for 32 rows and a page (own pages, often past a sequence's end: 0.8 of that), and 0.53 ns for a row's partials.
// Fitted to 29,004 calls of tiles of 32, of 128 and packed (20/20, 20/4, 32/16, 12/12, 8/8 and 8/1 heads, 1 to 64
// sequences of 1 to 1024 rows, prefixes of 0 to 8100 tokens), and 8,954 calls of those and of 2 to 16 parts: the least of
// eleven times missed costs 1.5% of a call on average.  Tiles of 32, of 128 and packed, us, 20 heads: 32 sequences of
// 4 rows each behind 1000 tokens 13 / 23 / 67, of 20-220 behind 600 97 / 45 / 37, 64 of 36-58 behind 4000 190 / 176 / 91,
// 24 of 52-191 with up to 695 tokens behind 563 106 / 46 / 79.  Tiles of 32, of 128 and those in 2, 4 and 8 parts: one of
// 1024 behind 6000 103 / 121 / 83 / 65 / 67, 2 of 56-361 behind 6000, 20/4 heads, 58 / 112 / 66 / 47 / 42.  Own lengths
// are on the device, so the table's width stands for them.
static TilePlan tile_plan(const SharedAttnArgs& a) {
    TilePlan best{0, 1, false};
    if (!a.row_offsets) return best;
    const int64_t pairs = (int64_t)a.rows * (a.n_head / a.n_kv_head), tiles = ceil_div(pairs, kStWaves * kSaQ), pages = ceil_div(a.prefix_len, kPage);
    const double KH = a.n_kv_head, own = a.max_pages, row_heads = (double)a.rows * a.n_head;
    double least = 9.0 + 1.65e-3 * KH * ((double)ceil_div(pairs, kSaQ) * pages + 0.8 * ((double)pairs / kSaQ + a.B) * own) + 0.53e-3 * row_heads;
    for (const bool pack : {false, true}) {
        const double units = KH * (pack ? (double)tiles : (double)pairs / (kStWaves * kSaQ) + 0.5 * a.B) / 256;
        const double chain = pages + 1.1 * own * (pack ? 1.0 + (double)(a.B - 1) / tiles : 1.0);
        const int64_t n = pack ? tiles : pairs / (kStWaves * kSaQ) + a.B;
        // (parts of 4 pages or more in 2048 workgroups or fewer: within shared_attention_bytes)
        for (int parts = 1; parts == 1 || (parts <= 16 && 4 * parts <= pages + a.max_pages && n * a.n_kv_head * parts <= 2048); parts *= 2) {
            const double rate = pack ? 1.1 : 1.0, u = units * parts;
            const double t = parts == 1 ? 5.5 + 0.8 * rate * chain * std::max(1.0, u)
                                        : 13.0 + 0.7 * rate * (chain / parts + 0.5) * std::max(1.0, 0.5 * (u + std::ceil(u))) +
                                              0.03e-3 * parts * row_heads;
            if (t > least || (pack && t == least)) continue;
            least = t;
            best = {(int)n, parts, pack};
        }
    }
    return best;
}

// Whether shared_whole_kernel takes a call of one row a sequence.  Its chain is a quarter of a sequence's pages (0.32 us
// a page while about 240 workgroups run), and every sequence reads the prefix; the cut pays for another launch and 1.3 ns
// for 32 rows and a page.  Fitted to 18,489 calls of both (20/20, 12/12, 8/8, 4/4, 32/16, 20/4 and 8/1 heads, 1 to 64
// sequences of up to 1200 tokens behind 0 to 2900): the worse of the two costs 0.12% of a call on average.  Whole and cut,
// us, 20 heads: 1 sequence of 50 behind 60 4.2 / 7.0, 8 of 250 behind 250 6.2 / 8.8, 8 of 250 behind 1000 9.3 / 9.4, 32 of 250
// behind 60 12.6 / 13.3, 32 of 1200 behind 2000 55 / 43.  The table's width stands for the own lengths (for the cut, up to
// 16 pages of it: a wide table is rarely full).
static bool shared_whole(const SharedAttnArgs& a) {
    if (a.row_offsets || ceil_div(a.prefix_len, kPage) + a.max_pages > kWave * kSwWaves) return false;
    const double g = a.n_head / a.n_kv_head, pages = (double)ceil_div(a.prefix_len, kPage), own = a.max_pages;
    const double tiles = (double)a.B * ceil_div(a.n_head / a.n_kv_head, kSaQ);
    const double whole = 3.5 + 0.32 * (pages + own) * std::max(1.0, tiles * a.n_kv_head / 240);
    const double cut = 8.5 + 1.3e-3 * a.n_kv_head * (pages * std::ceil(a.B * g / kSaQ) + tiles * std::min(own, 16.0));
    return whole <= cut;
}

// An upper bound of the partials of every call up to these sizes, from the least pages a workgroup, and from the
// most workgroups of 32 rows where more than one shares a side.
size_t shared_attention_bytes(int n_head, int rows, int prefix_len, int max_pages) {
    const int64_t rh = (int64_t)rows * n_head, pages = ceil_div(prefix_len, kPage);
    const int64_t most = std::min<int64_t>(ceil_div(pages, 2), kMaxSplit) + ceil_div(max_pages, 2);
    const int64_t n = std::min(most * rh, (int64_t)(kOwnGroups + kPreMany) * kSaQ + 2 * rh);
    return (size_t)n * (kHeadDim + 2) * 4 + 256;
}

// How a call runs (ftts_shared_attention_plan hands it out).
struct SharedChoice {
    int kernel, slots;  // FTTS_SHARED_*; partials a row
    TilePlan tile;
    SharedPlan cut;
};
static SharedChoice shared_choice(bool f32, const SharedAttnArgs& a) {
    SharedChoice c{};
    if (!f32) c.tile = tile_plan(a);
    if (c.tile.tiles > 0) {
        c.kernel = c.tile.pack ? FTTS_SHARED_PACKED : FTTS_SHARED_TILE;
        c.slots = c.tile.parts > 1 ? c.tile.parts : 0;
    } else if (!f32 && shared_whole(a)) {
        c.kernel = FTTS_SHARED_WHOLE;
    } else {
        c.kernel = FTTS_SHARED_CUT;
        c.cut = shared_plan(f32, a.n_head, a.n_kv_head, a.B, a.rows, a.row_offsets != nullptr, a.prefix_len, a.max_pages);
        c.slots = c.cut.s_pre + c.cut.s_own;
    }
    return c;
}

hipError_t launch_shared_attention(int dtype, const SharedAttnArgs& a, void* ws, size_t ws_bytes, hipStream_t st) {
    const bool f32 = dtype == FTTS_F32;
    // (the decode step's forms)
    if (a.q_f32 || a.o_f32 || a.active || a.len_add) {
        if (a.row_offsets || a.n_head > kFew * a.n_kv_head) return hipErrorInvalidValue;
    }
    const SharedChoice c = shared_choice(f32, a);
    const TilePlan& tp = c.tile;
    const int64_t rows_heads = (int64_t)a.rows * a.n_head;
    const dim3 jg((unsigned)((rows_heads + kJoinWaves - 1) / kJoinWaves)), jt(kJoinWaves * 64);
    SharedPlan p = c.cut;
    if (c.slots > 0) {
        if ((size_t)c.slots * rows_heads * (kHeadDim + 2) * 4 > ws_bytes) return hipErrorInvalidValue;
        p.o = reinterpret_cast<float*>(ws);
        p.ml = reinterpret_cast<float2*>(p.o + c.slots * rows_heads * kHeadDim);
    }
    if (tp.tiles > 0) {
        const dim3 wg((unsigned)(tp.tiles * a.n_kv_head * tp.parts)), wt(kStWaves * 64);
        if (tp.parts > 1) {
            p.s_pre = tp.parts;  // (for the join)
            if (tp.pack) hipLaunchKernelGGL((shared_tile_kernel<true, true>), wg, wt, 0, st, a, tp.tiles, p);
            else hipLaunchKernelGGL((shared_tile_kernel<false, true>), wg, wt, 0, st, a, tp.tiles, p);
            if (hipError_t e = hipGetLastError()) return e;
            hipLaunchKernelGGL(shared_join_kernel<false>, jg, jt, 0, st, a, p);
        } else if (tp.pack) {
            hipLaunchKernelGGL((shared_tile_kernel<true, false>), wg, wt, 0, st, a, tp.tiles, p);
        } else {
            hipLaunchKernelGGL((shared_tile_kernel<false, false>), wg, wt, 0, st, a, tp.tiles, p);
        }
        return hipGetLastError();
    }
    if (c.kernel == FTTS_SHARED_WHOLE) {
        const int64_t own_tiles = a.B * ceil_div(a.n_head / a.n_kv_head, kSaQ);
        const dim3 wg((unsigned)(own_tiles * a.n_kv_head)), wt(kSwWaves * 64);
        const bool few = a.n_head <= kFew * a.n_kv_head;
        if (a.q_f32) hipLaunchKernelGGL((shared_whole_kernel<true, true>), wg, wt, 0, st, a);
        else if (few) hipLaunchKernelGGL((shared_whole_kernel<false, true>), wg, wt, 0, st, a);
        else hipLaunchKernelGGL((shared_whole_kernel<false, false>), wg, wt, 0, st, a);
        return hipGetLastError();
    }
    const int64_t groups = (int64_t)((a.n_kv_head * p.s_pre + 7) / 8 * 8) * p.row_tiles + (int64_t)a.n_kv_head * p.own_tiles * p.s_own;
    const dim3 g((unsigned)groups), t(kSaWaves * 64);
    if (f32 && a.row_offsets) hipLaunchKernelGGL(shared_part_f32_kernel<true>, g, t, 0, st, a, p);
    else if (f32) hipLaunchKernelGGL(shared_part_f32_kernel<false>, g, t, 0, st, a, p);
    else if (a.row_offsets) hipLaunchKernelGGL((shared_part_kernel<true, false>), g, t, 0, st, a, p);
    else if (a.q_f32) hipLaunchKernelGGL((shared_part_kernel<false, true>), g, t, 0, st, a, p);
    else hipLaunchKernelGGL((shared_part_kernel<false, false>), g, t, 0, st, a, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (f32 || a.o_f32) hipLaunchKernelGGL(shared_join_kernel<true>, jg, jt, 0, st, a, p);
    else hipLaunchKernelGGL(shared_join_kernel<false>, jg, jt, 0, st, a, p);
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

int ftts_shared_attention_plan(const ftts_attn_shape* shape, int32_t B, int32_t n_rows, int32_t prompts, int32_t prefix_len,
                               int32_t max_pages, ftts_shared_launch* out) {
    if (!out) return set_error(FTTS_E_INVALID_ARG, "shared_attention_plan: out is NULL");
    if (int rc = check_shape(shape, B, n_rows, prefix_len, max_pages)) return rc;
    if (n_rows < 1 || (!prompts && n_rows != B))
        return set_error(FTTS_E_SHAPE, "shared_attention_plan: n_rows must be at least 1, and B without row offsets");
    const int32_t offsets = 0;  // (the rules ask only whether there are any)
    SharedAttnArgs a{};
    a.n_head = shape->n_head;
    a.n_kv_head = shape->n_kv_head;
    a.max_pages = max_pages;
    a.row_offsets = prompts ? &offsets : nullptr;
    a.prefix_len = prefix_len;
    a.B = B;
    a.rows = n_rows;
    const SharedChoice c = shared_choice(shape->dtype == FTTS_F32, a);
    const bool cut = c.kernel == FTTS_SHARED_CUT;
    *out = ftts_shared_launch{c.kernel, cut ? 0 : c.tile.tiles > 0 ? c.tile.parts : 1, c.cut.q_pre, c.cut.q_own,
                              cut && prefix_len > 0 ? c.cut.c_pre : 0, c.cut.c_own, c.slots};
    return FTTS_OK;
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
    const hipError_t e = launch_shared_attention(shape->dtype, a, ws, ws_bytes, (hipStream_t)stream);
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "shared_attention launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

}  // extern "C"
