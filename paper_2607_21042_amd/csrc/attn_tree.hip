// Attention of trees of drafted tokens over the paged cache.
//
// Row i of sequence b (n_b rows, L_b own tokens) sees the P tokens of the prefix, the own tokens before the tree,
// 0 .. L_b - n_b - 1, and the tree's tokens whose bits its mask has:  o = sum_j p_j v_j / sum_j p_j,
// p_j = exp(q . k_j / 8 - m).
//
// A workgroup takes a tile of 32 (row, query head) pairs of one sequence that read one key head, and a run of the pages
// that the sequence sees, cut into parts where the calls' tiles are few and the pages many; the shared-prefix attention's
// second kernel joins the parts.  Its waves take the run's half pages in turn and join their sums through LDS.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_rows.hpp"
#include "decode_entry.hpp"

namespace ftts {

// The bits of tokens 0 .. n - 1.
__device__ __forceinline__ uint64_t low_bits(int n) { return n >= 64 ? ~0ull : (1ull << max(n, 0)) - 1; }

// How a call is cut: tiles of 32 rows of a sequence, its chain of pages in so many equal parts; partials of part p (where
// there are several) at ml + p * T H and o + p * T H * 64.
struct TreePlan {
    int tiles, parts;
    bool blocks;  // (tree_work)
    float2* ml;
    float* o;
};

// What a workgroup does: a tile of one sequence's (token, query head) pairs that read one key head, a run of the pages
// that the sequence sees, the prefix's before its own.
struct TreeWork {
    int b, kh, row0, n, first;  // the tile's first pair of the sequence's n * g
    int past, own, n_pre;       // own tokens before the tree (-1: inactive), and in all; pages of the prefix
    int j0, pages;              // of the run
    int part;
};
// Inclusive sums over the wave's lanes.
__device__ __forceinline__ int sum_up(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // by 1, 2, 4 and 8 lanes within rows of 16,
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // then each row's last lane to the next row,
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // and the first half's to the second
    return v;
}
// False: no such tile.
__device__ __forceinline__ bool tree_work(const TreeArgs& a, const TreePlan& pl, int size, int lane, TreeWork& w) {
    static_assert(FTTS_MAX_BATCH <= kWave, "one sequence per lane");
    // Heads fastest, so that neighbouring blocks of a page are read at about the same time (heads times parts are a multiple
    // of 8, where there are parts: a sequence's tiles are then on one XCD).  blocks: in blocks of 8 tiles
    // whose (head, tile) pairs go to the 8 XCDs (workgroups are dealt to them in turn) in runs, tiles fastest: a sequence's
    // tiles, and in a block all sequences behind a prefix, read a head's pages through one L2.
    int tile, i = blockIdx.x;
    if (pl.blocks) {
        const int per = 8 * a.n_kv_head, lin = (i % per & 7) * a.n_kv_head + (i % per >> 3);
        tile = i / per * 8 + (lin & 7);
        w.kh = lin >> 3;
        w.part = 0;
    } else {
        w.kh = i % a.n_kv_head;
        i /= a.n_kv_head;
        w.part = i % pl.parts;
        tile = i / pl.parts;
    }
    const int g = a.n_head / a.n_kv_head;
    const bool in = lane < a.B;
    const int lo = in ? a.row_offsets[lane] : 0, hi = in ? a.row_offsets[lane + 1] : 0, length = in ? a.seq_lens[lane] : -1;
    const int first = min(max(lo, 0), a.rows), rows = min(max(hi, first), a.rows) - first, mine = (rows * g + size - 1) / size;
    // Longer sequences first, in four classes: begun last they would end last, by themselves.
    const int len = min(max(length, 0), kMaxPages * kPage), most = (int)wave_max((float)len);
    const int of = 4 * len > 3 * most ? 0 : 2 * len > most ? 1 : 4 * len > most ? 2 : 3;
    int upto = 0, before = 0;  // tiles up to this sequence's last one
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int sum = sum_up(of == c ? mine : 0);
        upto = of == c ? before + sum : upto;
        before += __builtin_amdgcn_readlane(sum, kWave - 1);
    }
    const unsigned long long whose = __ballot(in && tile < upto && tile >= upto - mine);
    if (!whose) return false;
    w.b = __builtin_ctzll(whose);
    w.row0 = __builtin_amdgcn_readlane(first, w.b);
    w.n = __builtin_amdgcn_readlane(rows, w.b);
    w.first = (tile - __builtin_amdgcn_readlane(upto - mine, w.b)) * size;
    const int own = __builtin_amdgcn_readlane(length, w.b);
    w.past = own < w.n ? -1 : own - w.n;  // (compared first: a length may be -2^31)
    w.own = w.past < 0 ? 0 : (int)min((int64_t)w.past + w.n, (int64_t)a.max_pages * kPage);
    w.n_pre = w.past < 0 ? 0 : (a.prefix_len + kPage - 1) / kPage;
    const int every = w.n_pre + (w.own + kPage - 1) / kPage, per = (every + pl.parts - 1) / pl.parts;
    w.j0 = w.part * per;
    w.pages = max(min(per, every - w.j0), 0);
    return true;
}

// A row's mask: lane (row, hh) holds words 2 hh and 2 hh + 1.
struct TreeMask {
    uint64_t even, odd;
};
__device__ __forceinline__ TreeMask tree_mask(const TreeArgs& a, int row, int hh) {
    const uint64_t* m = a.masks + (size_t)row * a.mask_words;
    return {2 * hh < a.mask_words ? m[2 * hh] : 0, 2 * hh + 1 < a.mask_words ? m[2 * hh + 1] : 0};
}
// The tree's tokens j0 .. j0 + 31 that the lane's row sees, of cnt that are there: bits of its mask (j0 may be negative:
// tokens before the tree, all of them seen).
__device__ __forceinline__ uint32_t tree_seen(const TreeMask m, int j0, int cnt, int lane) {
    const uint32_t there = (uint32_t)low_bits(cnt);
    if (j0 <= -32) return there;
    auto word = [lane, even = m.even, odd = m.odd](int i) -> uint64_t {  // (i is the same for the whole wave)
        if (i < 0 || i >= FTTS_MAX_TREE / 64) return 0;
        const uint64_t x = i & 1 ? odd : even;
        const int from = (lane & 31) | (i >> 1) << 5;
        return (uint64_t)(uint32_t)__shfl((int)(x >> 32), from, kWave) << 32 | (uint32_t)__shfl((int)x, from, kWave);
    };
    const int w = j0 >> 6, s = j0 & 63;  // (a floor)
    uint64_t bits = word(w) >> s;
    if (s > 32) bits |= word(w + 1) << (64 - s);
    if (j0 < 0) bits |= low_bits(-j0);
    return (uint32_t)bits & there;
}

// A run's pages meet a tile in halves of 32 tokens: K and V of 4 KB each in a wave's stage, 128-byte rows whose 16-byte
// pieces are XOR-swizzled by (row / 2) % 8.  The lane's keys of a half are (i / 4) * 8 + hh * 4 + i % 4, i < 16.
constexpr int kThK = 32, kThTile = kThK * kHeadDim * 2, kThStage = 2 * kThTile;

// K operands kr, V blocks vr by (second 8 keys, second 32 dims): as at_addresses.
struct ThAddr {
    uint32_t kr[4], vr[2][2];
};
__device__ __forceinline__ ThAddr th_addresses(uint32_t s0, int lane) {
    const int ql = lane & 31, hh = lane >> 5, i16 = lane & 15, g16 = (lane >> 4) & 1;
    ThAddr r;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) r.kr[kk] = s0 + ql * 128 + (((2 * kk + hh) ^ ((ql >> 1) & 7)) << 4);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const int row = e * 8 + hh * 4 + (i16 >> 2), piece = d * 4 + g16 * 2 + ((i16 & 3) >> 1);
            r.vr[e][d] = s0 + kThTile + row * 128 + ((piece ^ ((row >> 1) & 7)) << 4) + (i16 & 1) * 8;
        }
    return r;
}
// (one assembly block with its wait: nothing is in flight in a register that the compiler holds for written)
__device__ __forceinline__ void th_read_k(const ThAddr& r, uint4 (&k)[4]) {
    at_bf16x8 x[4];
    asm volatile(
        "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
        : "v"(r.kr[0]), "v"(r.kr[1]), "v"(r.kr[2]), "v"(r.kr[3])
        : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = __builtin_bit_cast(uint4, x[i]);
}
__device__ __forceinline__ void th_read_v(const ThAddr& r, uint64_t (&v)[2][2][2]) {  // [dims][keys][step]
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:2048\n\t"
        "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:2048\n\t"
        "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:2048\n\t"
        "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:2048\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(v[0][0][0]), "=&v"(v[0][0][1]), "=&v"(v[0][1][0]), "=&v"(v[0][1][1]), "=&v"(v[1][0][0]), "=&v"(v[1][0][1]),
          "=&v"(v[1][1][0]), "=&v"(v[1][1][1])
        : "v"(r.vr[0][0]), "v"(r.vr[1][0]), "v"(r.vr[0][1]), "v"(r.vr[1][1])
        : "memory");
}
__device__ __forceinline__ at_bf16x8 th_vop(const uint64_t (&v)[2][2][2], int d, int st) {
    return at_op(make_uint4((uint32_t)v[d][0][st], (uint32_t)(v[d][0][st] >> 32), (uint32_t)v[d][1][st], (uint32_t)(v[d][1][st] >> 32)));
}
__device__ __forceinline__ void th_pv(SaState& a, const uint64_t (&v)[2][2][2], const uint32_t (&pw)[8]) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        const at_bf16x8 p = at_op(make_uint4(pw[4 * st], pw[4 * st + 1], pw[4 * st + 2], pw[4 * st + 3]));
        a.o0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(th_vop(v, 0, st), p, a.o0, 0, 0, 0);
        a.o1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(th_vop(v, 1, st), p, a.o1, 0, 0, 0);
    }
}
// Masks what a row does not see.
__device__ __forceinline__ void th_hide(at_f32x16& s, uint32_t seen, int hh) {
    const uint32_t x = seen >> (4 * hh);
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (!(x >> ((i >> 2) * 8 + (i & 3)) & 1)) s[i] = -INFINITY;
}
// As sa_not_finite.
__device__ __forceinline__ bool th_not_finite(const uint64_t (&v)[2][2][2]) {
    const at_bf16x8 ones = at_op(make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
    at_f32x16 x;
    float z = 0.f;
#pragma unroll
    for (int d = 0; d < 2; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
        for (int st = 0; st < 2; ++st) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(th_vop(v, d, st), ones, x, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) z = fmaf(x[i], 0.f, z);
    }
    return __any(z != 0.f);  // (NaN)
}
// Values that are not finite are taken out of the operands and reach the rows that see their token by themselves, after
// the loop: which rows meet one, of either sign (a NaN counts for both), is a product of indicators, made for two bf16 at
// once: bit 15 of each half where it holds, then bit 14, 2.0 in bf16.
__device__ __forceinline__ void th_add_not_finite(SaState& a, const uint64_t (&v)[2][2][2], uint32_t seen, int hh) {
    const uint32_t x = seen >> (4 * hh);
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int sign = 0; sign < 2; ++sign) {
            at_f32x16 n;
#pragma unroll
            for (int i = 0; i < 16; ++i) n[i] = 0.f;
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                uint32_t of[4], sees[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t w = (uint32_t)(v[d][r >> 1][st] >> (32 * (r & 1))), odd = ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
                    const uint32_t nan = ((w & 0x007F007Fu) + 0x007F007Fu) << 8, bits = x >> ((2 * st + (r >> 1)) * 8 + 2 * (r & 1));
                    of[r] = (odd & ((sign ? w : ~w) | nan)) >> 1;
                    sees[r] = (bits << 14 & 0x4000u) | (bits << 29 & 0x40000000u);
                }
                n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at_op(make_uint4(of[0], of[1], of[2], of[3])),
                                                            at_op(make_uint4(sees[0], sees[1], sees[2], sees[3])), n, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) (d ? a.o1 : a.o0)[i] += n[i] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
            __builtin_amdgcn_sched_barrier(0);  // (one after the other)
        }
}
__device__ __forceinline__ void th_take_out(uint64_t (&v)[2][2][2]) {
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                uint32_t x[2] = {(uint32_t)v[d][e][st], (uint32_t)(v[d][e][st] >> 32)};
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if ((x[w] & 0x7F80u) == 0x7F80u) x[w] &= 0xFFFF0000u;
                    if ((x[w] & 0x7F800000u) == 0x7F800000u) x[w] &= 0xFFFFu;
                }
                v[d][e][st] = (uint64_t)x[1] << 32 | x[0];
            }
}

// Joins the W waves' results of one tile through LDS and writes the output, or the run's partial: each wave a part of the
// dims.  Every wave is done with smem.
template <bool F32, int W>
__device__ __forceinline__ void tree_finish(const TreeArgs& a, const TreePlan& pl, const TreeWork& w, const SaState& st, int row, int head,
                                            char* smem, int wave, int lane) {
    constexpr int kMine = 32 / W;  // elements of a lane's 32
    float* mrg = reinterpret_cast<float*>(smem);  // [W][34][64], lane for lane
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
    float mm = -INFINITY, l = 0.f, x[kMine];
#pragma unroll
    for (int u = 0; u < W; ++u) mm = fmaxf(mm, mrg[(u * 34 + 32) * 64 + lane]);
    const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
    for (int i = 0; i < kMine; ++i) x[i] = 0.f;
#pragma unroll
    for (int u = 0; u < W; ++u) {
        const float* mw = mrg + u * 34 * 64;
        const float f = exp2f(mw[32 * 64 + lane] - ref);
        l += mw[33 * 64 + lane] * f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) x[i] += mw[(kMine * wave + i) * 64 + lane] * f;
    }
    const RowPair ls = swap32(l);
    l = ls.a + ls.b;
    if (row < 0) return;
    // element e = kMine wave + i: dims 8 (e / 4) + 4 hh + e % 4
    const int d = 8 * (kMine * wave / 4) + 4 * (lane >> 5) + kMine * wave % 4;
    constexpr int kRun = kMine < 4 ? kMine : 4;  // dims side by side
    const int64_t slot = (int64_t)w.part * a.rows * a.n_head + (int64_t)row * a.n_head + head;
    const bool part = pl.parts > 1;
    if (part && wave == 0 && lane < 32) pl.ml[slot] = make_float2(mm, l);
    const float scale = part ? 1.f : sa_inverse(l, mm);
    const size_t at = part ? slot * kHeadDim + d : (size_t)row * a.o_ld + head * kHeadDim + d;
#pragma unroll
    for (int g = 0; g < kMine / kRun; ++g) {
        float y[kRun];
#pragma unroll
        for (int i = 0; i < kRun; ++i) y[i] = x[kRun * g + i] * scale;
        if (F32 || part) {
            float* to = (part ? pl.o : reinterpret_cast<float*>(a.o)) + at + 8 * g;
            if constexpr (kRun == 4) *reinterpret_cast<float4*>(to) = make_float4(y[0], y[1], y[2], y[3]);
            else *reinterpret_cast<float2*>(to) = make_float2(y[0], y[1]);
        } else {
            uint16_t* to = reinterpret_cast<uint16_t*>(a.o) + at + 8 * g;
            if constexpr (kRun == 4) *reinterpret_cast<uint2*>(to) = make_uint2(bf16x2_rne(y[0], y[1]), bf16x2_rne(y[2], y[3]));
            else *reinterpret_cast<uint32_t*>(to) = bf16x2_rne(y[0], y[1]);
        }
    }
}

// bf16: the waves take the halves of the run's pages in turn (wave w: w, w + W, ...) by direct-to-LDS loads into a stage of
// their own, the next half's K (V) on its way once this one's is in registers; no barrier in the loop.  Halves before the
// tree come first and need no mask; those of the tree follow.  Queries and masks are waited for before the loop: a wait for
// them in it would be one for the next half's loads too.
//
// Bound by reading where the pages are many (a half costs a wave 1,285 cycles of vector work, two waves a SIMD hide the
// loads up to 5.1 TB/s), by one tile's chain of halves, start and hand-over (5 us) where they are few.  Traced: 32 trees of
// 8-64 tokens behind 64-1,200 at 20 heads, 123 MB, 32.5 us; 4 of 40-64 behind 6,000-14,000, 188 MB, 46.4 and the join 4.9;
// one of 16 behind 300 7.5.  A wave a row without matrix products took 1,352 us for the first and 4,113 for the second.
// Slower or level: whole pages a step, two tiles a wave (spills), four waves a SIMD, two halves in flight, 16 waves.
template <int W>
__global__ __launch_bounds__(W * 64, W == 4 ? 3 : 4) void tree_tile_kernel(const TreeArgs a, const TreePlan pl) {
    __shared__ __attribute__((aligned(1024))) char smem[W * 34 * 256];  // the stages, then the waves' results
    static_assert(sizeof(smem) >= W * kThStage, "");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31, hh = lane >> 5;
    TreeWork w;
    if (!tree_work(a, pl, 32, lane, w)) return;
    const int g = a.n_head / a.n_kv_head, pairs = w.n * g, idx = w.first + ql, last = min(idx, pairs - 1);
    const int row = w.row0 + last / g, head = w.kh * g + last % g;  // this lane's pair, the tile's last one where it is past it
    char* own = smem + wave * kThStage;
    const int halves = 2 * w.pages, n = halves > wave ? (halves - wave + W - 1) / W : 0;  // this wave's halves
    const size_t to_v = (size_t)a.n_kv_head * kAtTile;  // from a page's keys to its values
    PageRef page{};
    auto fetch = [&](int i0) {  // the wave's halves i0 .. i0 + 63, one a lane
        const int i = i0 + lane, u = wave + W * i, j = w.j0 + (u >> 1), k = j - w.n_pre;
        const int id = i >= n ? -1 : k < 0 ? a.prefix_pages[j] : a.block_table[(size_t)w.b * a.max_pages + k];
        page = page_ref(a, w.kh, 2, id, i >= n ? 0 : k < 0 ? a.prefix_len - j * kPage : w.own - k * kPage);
        page.tokens = min(max(page.tokens - (u & 1) * kThK, 0), kThK);
    };
    if (n > 0) fetch(0);
    uint4 qr[4];
    at_load_q(reinterpret_cast<const uint16_t*>(a.q) + (size_t)row * a.q_ld + head * kHeadDim, hh, qr);
    TreeMask mask = tree_mask(a, row, hh);
    auto load = [&](int i, int kv) {  // the wave's i-th half, K (kv 0) or V; zeros for what is not there
        const int tokens = __builtin_amdgcn_readlane(page.tokens, i & 63);
        const char* src = page_at(a, page, i & 63) + kv * to_v + (wave & 1) * kThTile;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = k * 8 + (lane >> 3);
            buffer_to_lds16(src, tokens * 128, own + kv * kThTile + k * 1024, r * 128 + (((lane & 7) ^ ((r >> 1) & 7)) << 4), 0);
        }
        return tokens;
    };
    static_assert(W % 2 == 0, "a wave's halves are all first or all second ones");
    const ThAddr ad = th_addresses(lds_address(own), lane);
    SaState st;
    sa_init(st);
    bool saw = false, odd = false;  // a token; a value that is not finite where rows see different tokens
    int next = 0;
    if (n > 0) {
        next = load(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load(0, 1);
    }
    auto tree0 = [&](int i) { return (w.j0 + ((wave + W * i) >> 1) - w.n_pre) * kPage + (wave & 1) * kThK - w.past; };
    auto step = [&](auto of_tree, int i) {  // half i; of_tree: rows may see different tokens of it
        constexpr bool TREE = decltype(of_tree)::value;
        const bool more = i + 1 < n;
        const int tokens = next;
        asm volatile("s_waitcnt vmcnt(4)" ::: "memory");  // K is in (this wave's own loads), V's 4 loads may be out
        __builtin_amdgcn_sched_barrier(0);
        uint4 k[4];
        th_read_k(ad, k);
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            if (((i + 1) & 63) == 0) fetch(i + 1);
            next = load(i + 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        at_f32x16 s[1];
#pragma unroll
        for (int e = 0; e < 16; ++e) s[0][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at_op(k[kk]), at_op(qr[kk]), s[0], 0, 0, 0);
        uint32_t seen = 0;
        if constexpr (TREE) {
            seen = tree_seen(mask, tree0(i), tokens, lane);
            th_hide(s[0], seen, hh);
            saw |= seen != 0;
        } else {
            if (tokens < kThK) th_hide(s[0], (uint32_t)low_bits(tokens), hh);
            saw |= tokens > 0;
        }
        sa_maximum(st, s);
        const float ref = st.m == -INFINITY ? 0.f : st.m;  // nothing seen: every score is -inf and every weight 0
        uint32_t pw[8], plo[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[0][e], kSaScale, -ref)), y = __builtin_amdgcn_exp2f(fmaf(s[0][e + 1], kSaScale, -ref));
            st.l += x + y;
            pw[e / 2] = sa_split(x, y, plo[e / 2]);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");  // V is in, the next K may be out
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        uint64_t v[2][2][2];
        th_read_v(ad, v);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (TREE) {
            if (__any(seen != (uint32_t)low_bits(tokens)) && th_not_finite(v)) {
                th_take_out(v);
                odd = true;
            }
        }
        if (more) load(i + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
        th_pv(st, v, pw);
        th_pv(st, v, plo);
    };
    // (queries and masks are waited for here: the compiler would wait for them in the loop, and so for the next half's loads)
    at_tie4(qr);
    asm volatile("" : "+v"(mask.even), "+v"(mask.odd));
    // halves that end before the tree are seen whole: the wave's first ones, of the run's 2 (n_pre - j0) + past / 32
    const int before = 2 * (w.n_pre - w.j0) + (w.past < 0 ? 0 : w.past / kThK), whole = min(max(before - wave + W - 1, 0) / W, n);
    for (int i = 0; i < whole; ++i) step(std::false_type{}, i);
    for (int i = whole; i < n; ++i) step(std::true_type{}, i);
    if (odd)
#pragma unroll 1
        for (int i = whole; i < n; ++i) {
            fetch(i);  // (to lane 0)
            const int tokens = __builtin_amdgcn_readlane(page.tokens, 0);
            load(0, 1);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            uint64_t v[2][2][2];
            th_read_v(ad, v);
            th_add_not_finite(st, v, tree_seen(mask, tree0(i), tokens, lane), hh);
        }
    st.m = sa_marked(st.m, saw);
    __syncthreads();
    tree_finish<false, W>(a, pl, w, st, idx < pairs ? row : -1, head, smem, wave, lane);
}

// fp32: the same with fp32 matrix products, all sums in fp32: 4096 cycles of products (1.7 us) a wave and half page, whatever
// the tile's rows.  4 trees of 8-32 behind 50-700 at 20 heads, 20 MB, 15.0 us and the join 4.0: a wave has one to three half
// pages there, and products are 26% of the waves' cycles (4.9 M of 19 M); start, loads and hand-over are the rest.
constexpr int kTfTile = kSfK * kHeadDim * 4, kTfStage = 2 * kTfTile;
// As th_add_not_finite; v0, v1: values of the keys that element i is for, in dims lane % 32 and 32 + lane % 32.
__device__ __forceinline__ void tf_add_not_finite(SaState& a, const float (&v0)[16], const float (&v1)[16], uint32_t seen, int hh) {
    const uint32_t x = seen >> (4 * hh);
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int sign = 0; sign < 2; ++sign) {
            at_f32x16 n;
#pragma unroll
            for (int i = 0; i < 16; ++i) n[i] = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float v = d ? v1[i] : v0[i], of = fabsf(v) < INFINITY || v == (sign ? INFINITY : -INFINITY) ? 0.f : 1.f;
                n = __builtin_amdgcn_mfma_f32_32x32x2f32(of, x >> ((i >> 2) * 8 + (i & 3)) & 1 ? 1.f : 0.f, n, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) (d ? a.o1 : a.o0)[i] += n[i] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
            __builtin_amdgcn_sched_barrier(0);  // (one after the other)
        }
}
template <int W>
__global__ __launch_bounds__(W * 64, 2) void tree_tile_f32_kernel(const TreeArgs a, const TreePlan pl) {
    __shared__ __attribute__((aligned(1024))) char smem[W * kTfStage];  // the stages, then the waves' results
    static_assert(kTfStage >= 34 * 256, "");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31, hh = lane >> 5;
    TreeWork w;
    if (!tree_work(a, pl, 32, lane, w)) return;
    const int g = a.n_head / a.n_kv_head, pairs = w.n * g, idx = w.first + ql, last = min(idx, pairs - 1);
    const int row = w.row0 + last / g, head = w.kh * g + last % g;  // this lane's pair, the tile's last one where it is past it
    char* own = smem + wave * kTfStage;
    const int halves = 2 * w.pages, n = halves > wave ? (halves - wave + W - 1) / W : 0;  // this wave's halves
    const size_t to_v = (size_t)a.n_kv_head * (kPage * kHeadDim * 4);  // from a page's keys to its values
    PageRef page{};
    auto fetch = [&](int i0) {  // the wave's halves i0 .. i0 + 63, one a lane
        const int i = i0 + lane, u = wave + W * i, j = w.j0 + (u >> 1), k = j - w.n_pre;
        const int id = i >= n ? -1 : k < 0 ? a.prefix_pages[j] : a.block_table[(size_t)w.b * a.max_pages + k];
        page = page_ref(a, w.kh, 4, id, i >= n ? 0 : k < 0 ? a.prefix_len - j * kPage : w.own - k * kPage);
        page.tokens = min(max(page.tokens - (u & 1) * kSfK, 0), kSfK);
    };
    if (n > 0) fetch(0);
    float4 q[8];
    {
        const float* qp = reinterpret_cast<const float*>(a.q) + (size_t)row * a.q_ld + head * kHeadDim + hh * 32;
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = *reinterpret_cast<const float4*>(qp + 4 * i);
    }
    TreeMask mask = tree_mask(a, row, hh);
    static_assert(W % 2 == 0, "a wave's halves are all first or all second ones");
    auto load = [&](int i, int kv) {  // the wave's i-th half, K (kv 0) or V; zeros for what is not there
        const int tokens = __builtin_amdgcn_readlane(page.tokens, i & 63);
        const char* src = page_at(a, page, i & 63) + kv * to_v + (wave & 1) * kTfTile;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int r = k * 4 + (lane >> 4);
            buffer_to_lds16(src, tokens * 256, own + kv * kTfTile + k * 1024, r * 256 + (((lane & 15) ^ (r & 15)) << 4), 0);
        }
        return tokens;
    };
    uint32_t kr[8], vr[8];
    {
        const uint32_t s0 = lds_address(own);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            kr[c] = s0 + ql * 256 + (((hh * 8 + c) ^ (ql & 15)) << 4);
            // c = 4 (i / 4 % 2) + i % 4 for element i
            vr[c] = s0 + kTfTile + hh * 1024 + (((ql >> 2) ^ ((c >> 2) * 8 + hh * 4 + (c & 3))) << 4) + (ql & 3) * 4;
        }
    }
    SaState st;
    sa_init(st);
    bool saw = false, odd = false;  // a token; a value that is not finite where rows see different tokens
    int next = 0;
    if (n > 0) {
        next = load(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load(0, 1);
    }
    auto tree0 = [&](int i) { return (w.j0 + ((wave + W * i) >> 1) - w.n_pre) * kPage + (wave & 1) * kSfK - w.past; };
    auto step = [&](auto of_tree, int i) {  // half i; of_tree: rows may see different tokens of it
        constexpr bool TREE = decltype(of_tree)::value;
        const bool more = i + 1 < n;
        const int tokens = next;
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // K is in (this wave's own loads), V's 8 loads may be out
        __builtin_amdgcn_sched_barrier(0);
        float4 k[8];
        sf_read_k(kr, k);
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            if (((i + 1) & 63) == 0) fetch(i + 1);
            next = load(i + 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        at_f32x16 s[1];
#pragma unroll
        for (int e = 0; e < 16; ++e) s[0][e] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e].x, q[e].x, s[0], 0, 0, 0);
            s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e].y, q[e].y, s[0], 0, 0, 0);
            s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e].z, q[e].z, s[0], 0, 0, 0);
            s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e].w, q[e].w, s[0], 0, 0, 0);
        }
        uint32_t seen = 0;
        if constexpr (TREE) {
            seen = tree_seen(mask, tree0(i), tokens, lane);
            th_hide(s[0], seen, hh);
            saw |= seen != 0;
        } else {
            if (tokens < kSfK) th_hide(s[0], (uint32_t)low_bits(tokens), hh);
            saw |= tokens > 0;
        }
        sa_maximum(st, s);
        const float ref = st.m == -INFINITY ? 0.f : st.m;  // nothing seen: every score is -inf and every weight 0
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[0][e] = __builtin_amdgcn_exp2f(fmaf(s[0][e], kSaScale, -ref));
            st.l += s[0][e];
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // V is in, the next K may be out
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        float v0[16], v1[16];
        sf_read_v(vr, 0, v0);
        sf_read_v(vr, 4, v1);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (TREE) {
            float z = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) z = fmaf(v0[e], 0.f, fmaf(v1[e], 0.f, z));
            if (__any(seen != (uint32_t)low_bits(tokens)) && __any(z != 0.f)) {  // (NaN)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    v0[e] = fabsf(v0[e]) < INFINITY ? v0[e] : 0.f;
                    v1[e] = fabsf(v1[e]) < INFINITY ? v1[e] : 0.f;
                }
                odd = true;
            }
        }
        if (more) load(i + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            st.o0 = __builtin_amdgcn_mfma_f32_32x32x2f32(v0[e], s[0][e], st.o0, 0, 0, 0);
            st.o1 = __builtin_amdgcn_mfma_f32_32x32x2f32(v1[e], s[0][e], st.o1, 0, 0, 0);
        }
    };
    // (as in tree_tile_kernel)
#pragma unroll
    for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(q[i].x), "+v"(q[i].y), "+v"(q[i].z), "+v"(q[i].w));
    asm volatile("" : "+v"(mask.even), "+v"(mask.odd));
    const int before = 2 * (w.n_pre - w.j0) + (w.past < 0 ? 0 : w.past / kSfK), whole = min(max(before - wave + W - 1, 0) / W, n);
    for (int i = 0; i < whole; ++i) step(std::false_type{}, i);
    for (int i = whole; i < n; ++i) step(std::true_type{}, i);
    if (odd)
#pragma unroll 1
        for (int i = whole; i < n; ++i) {
            fetch(i);  // (to lane 0)
            const int tokens = __builtin_amdgcn_readlane(page.tokens, 0);
            load(0, 1);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            float v0[16], v1[16];
            sf_read_v(vr, 0, v0);
            sf_read_v(vr, 4, v1);
            tf_add_not_finite(st, v0, v1, tree_seen(mask, tree0(i), tokens, lane), hh);
        }
    st.m = sa_marked(st.m, saw);
    __syncthreads();
    tree_finish<true, W>(a, pl, w, st, idx < pairs ? row : -1, head, smem, wave, lane);
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of 32 rows that so many sequences have at most; in one part many of them go in blocks of 8 (captured, 32 trees of
// 8-64 tokens behind up to 1200: 32.6 us, 38.4 without the blocks; few tiles would leave a block's idle).
static int64_t tree_tiles(int n_head, int n_kv_head, int rows, int B, int parts) {
    const int64_t n = (int64_t)rows * (n_head / n_kv_head) / 32 + B;
    return parts == 1 && n >= 16 ? ceil_div(n, 8) * 8 : n;
}
// A grid has fewer than 2^32 threads.
static bool tree_fits(int64_t workgroups, int waves) { return workgroups * waves * kWave < 1LL << 32; }

// Parts pay for a second launch and a row's partials, 8 waves a workgroup for fewer workgroups at once and a longer hand-
// over.  In bf16 a part's chain of pages costs 0.40 us a page with 4 waves and 0.25 with 8 while fewer than 590 (270)
// workgroups run, and so many times that where there are more, with a bend between.  Fitted to 1,455 calls (fp32: 963) of 1
// to 64 sequences, trees of 1 to 256, 20/20, 20/4, 12/12, 12/2, 32/16, 8/1 and 4/4 heads, up to 16,000 own tokens behind up
// to 5000 (2000 and 1000), each run with 4 and 8 waves in 1 to 48 parts: the choice costs 1.1% (1.7%) of a call on average,
// always 4 waves and one part 33% (43%), 8 waves 25% (44%).  Own lengths are on the device, so the table's width stands for
// them.
constexpr int kTreeMaxParts = 48, kTreeMaxSlots = 1 << 18;  // partials of a call: 69 MB at most
struct TreeCost {
    double begun, own;       // of a sequence's tiles the one that is begun, of the table's width what is filled
    double room[2], page[2]; // workgroups at once, us a page of the chain: 4 waves, 8 waves
    double eight, bend;      // us for 8 waves; how sharp the bend is
    double join, partial;    // us for the second launch, and a partial
    double group;            // us a workgroup
};
static TreePlan tree_plan(const TreeArgs& a, bool f32, int& waves) {
    static constexpr TreeCost kCost[2] = {{0.75, 0.83, {590, 270}, {0.40, 0.246}, 1.0, 3.9, 2.7, 0.155e-3, 4.9e-3},
                                          {1.40, 1.37, {400, 306}, {0.48, 0.367}, 1.4, 3.1, 1.27, 0.168e-3, 4.5e-3}};
    const TreeCost& c = kCost[f32];
    const double g = a.n_head / a.n_kv_head, units = a.n_kv_head * (a.rows * g / 32 + c.begun * a.B), row_heads = (double)a.rows * a.n_head;
    const int64_t pages = ceil_div(a.prefix_len, kPage) + a.max_pages;
    const double chain = ceil_div(a.prefix_len, kPage) + c.own * a.max_pages;
    TreePlan p{};
    double least = 1e30;
    // (4 trees of 40-64 behind 6,000-14,000, 20 heads: 51 us in 4 parts, 64 in 3 and 70 in 5, whose tiles read through two L2)
    const int step = a.n_kv_head % 8 == 0 ? 1 : a.n_kv_head % 4 == 0 ? 2 : a.n_kv_head % 2 == 0 ? 4 : 8;
    for (const int n : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, kTreeMaxParts}) {
        const int parts = n > 1 ? (int)ceil_div(n, step) * step : 1;
        if (n > 1 && (2 * parts > pages || parts * row_heads > kTreeMaxSlots)) break;
        const int64_t tiles = tree_tiles(a.n_head, a.n_kv_head, a.rows, a.B, parts);
        for (const int e : {0, 1}) {
            if (!tree_fits(tiles * a.n_kv_head * parts, e ? 8 : 4)) continue;  // (4 waves and one part: check_shape)
            const double full = units * parts / c.room[e];
            const double t = e * c.eight + c.page[e] * chain / parts * std::pow(1.0 + std::pow(full, c.bend), 1.0 / c.bend) +
                             (parts > 1 ? c.join + c.partial * parts * row_heads : 0) + c.group * units * parts;
            if (t >= least) continue;
            least = t;
            p.parts = parts;
            p.tiles = (int)tiles;
            waves = e ? 8 : 4;
        }
    }
    p.blocks = p.parts == 1 && p.tiles >= 16;
    return p;
}

size_t tree_attention_bytes(int n_head, int rows) {
    return (size_t)std::min<int64_t>((int64_t)rows * n_head * kTreeMaxParts, kTreeMaxSlots) * (kHeadDim + 2) * 4 + 256;
}

hipError_t launch_tree_attention(int dtype, const TreeArgs& a, void* ws, size_t ws_bytes, hipStream_t st) {
    const bool f32 = dtype == FTTS_F32;
    int waves = 4;
    TreePlan p = tree_plan(a, f32, waves);
    const int64_t slots = p.parts > 1 ? (int64_t)p.parts * a.rows * a.n_head : 0;
    if ((size_t)slots * (kHeadDim + 2) * 4 > ws_bytes) return hipErrorInvalidValue;
    p.o = reinterpret_cast<float*>(ws);
    p.ml = reinterpret_cast<float2*>(p.o + slots * kHeadDim);
    const dim3 wg((unsigned)(p.tiles * a.n_kv_head * p.parts)), wt(waves * 64);
    (void)hipGetLastError();
    if (f32 && waves == 8) hipLaunchKernelGGL(tree_tile_f32_kernel<8>, wg, wt, 0, st, a, p);
    else if (f32) hipLaunchKernelGGL(tree_tile_f32_kernel<4>, wg, wt, 0, st, a, p);
    else if (waves == 8) hipLaunchKernelGGL(tree_tile_kernel<8>, wg, wt, 0, st, a, p);
    else hipLaunchKernelGGL(tree_tile_kernel<4>, wg, wt, 0, st, a, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.parts == 1) return hipSuccess;
    SharedAttnArgs join{};
    join.o = a.o;
    join.o_ld = a.o_ld;
    join.n_head = a.n_head;
    join.rows = a.rows;
    join.row_offsets = a.row_offsets;
    join.B = a.B;
    return launch_attn_join(f32, join, p.parts, p.ml, p.o, st);
}

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
    if (n_rows < 0 || n_rows > (1 << 24)) return set_error(FTTS_E_RANGE, "tree_attention: n_rows must be in [0, 2^24]");
    const int64_t groups = tree_tiles(s->n_head, s->n_kv_head, n_rows, B, 1) * s->n_kv_head;
    if (!tree_fits(groups, 4))
        return set_error(FTTS_E_RANGE, "tree_attention: %lld tiles of 32 rows and heads, a launch takes fewer than 2^24", (long long)groups);
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
    return tree_attention_bytes(shape->n_head, n_rows);
}

int ftts_tree_attention_plan(const ftts_attn_shape* shape, int32_t B, int32_t n_rows, int32_t prefix_len, int32_t max_pages,
                             ftts_tree_launch* out) {
    if (!out) return set_error(FTTS_E_INVALID_ARG, "tree_attention_plan: out is NULL");
    if (int rc = check_shape(shape, B, n_rows, prefix_len, max_pages)) return rc;
    if (n_rows < 1) return set_error(FTTS_E_SHAPE, "tree_attention_plan: n_rows must be at least 1");
    TreeArgs a{};
    a.n_head = shape->n_head;
    a.n_kv_head = shape->n_kv_head;
    a.max_pages = max_pages;
    a.prefix_len = prefix_len;
    a.B = B;
    a.rows = n_rows;
    int waves = 4;
    const TreePlan p = tree_plan(a, shape->dtype == FTTS_F32, waves);
    *out = ftts_tree_launch{waves, p.parts, p.tiles, p.blocks};
    return FTTS_OK;
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
    const hipError_t e = launch_tree_attention(shape->dtype, a, ws, ws_bytes, (hipStream_t)stream);
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "tree_attention launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

}  // extern "C"
