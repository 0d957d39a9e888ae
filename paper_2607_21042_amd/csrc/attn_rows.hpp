// What the attention kernels over the paged cache share: a wave's products of 32 rows with pages of 64 tokens that
// direct-to-LDS loads bring into a stage, its running softmax, weights in two bf16 parts, values that are not finite.
#pragma once
#include "attn_tile.hpp"

namespace ftts {

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
template <typename Args>
__device__ __forceinline__ PageRef page_ref(const Args& a, int kh, int esize, int phys, int left) {
    const bool ok = phys >= 0 && phys < a.n_pages;
    const uint64_t off = kv_offset(a.layer, a.n_pages, ok ? phys : 0, 0, a.n_kv_head, kh, 0) * esize;
    return {(uint32_t)off, (uint32_t)(off >> 32), ok ? max(min(left, kPage), 0) : 0};
}
template <typename Args>
__device__ __forceinline__ const char* page_at(const Args& a, const PageRef& r, int lane) {
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
// Then they become 0 in the operands (and are added by themselves to the rows that see the token).
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

// fp32: halves of a page, 32 tokens, as the first operand of products of 32x32x2.  A 16-byte piece c of row r lies at
// c ^ (r % 16).  K: lane (key, hh) holds dims 32 hh .. + 31, one a step (kr: its 16-byte pieces).
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

}  // namespace ftts
