// Pieces of the bf16 attention kernels: a wave's products of 32 queries with a 64-key tile of K
// and V that direct-to-LDS loads have brought in, 128-byte rows whose 16-byte pieces are
// XOR-swizzled by (row / 2) % 8 (two rows share the 256 bytes that a 16-byte read takes a cycle).
#pragma once
#include "gemm_epilogue.hpp"

namespace ftts {

typedef __bf16 at_bf16x8 __attribute__((ext_vector_type(8)));
typedef float at_f32x16 __attribute__((ext_vector_type(16)));

constexpr int kAtK = 64;
constexpr int kAtTile = kAtK * kHeadDim * 2;   // bytes of a K (or V) tile
constexpr int kAtStage = 2 * kAtTile;

// LDS reads in inline assembly (the compiler would wait for every direct-to-LDS load in
// flight before each); used only after at_wait and at_tie.
template <int OFF>
__device__ __forceinline__ uint4 at_read(uint32_t addr) {
    at_bf16x8 r;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "n"(OFF) : "memory");
    return __builtin_bit_cast(uint4, r);
}
template <int OFF>
__device__ __forceinline__ uint64_t at_read_tr(uint32_t addr) {
    uint64_t r;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "n"(OFF) : "memory");
    return r;
}
template <typename T, int N>
__device__ __forceinline__ void at_tie(T (&o)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(o[i])::"memory");
}
__device__ __forceinline__ void at_tie4(uint4 (&o)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        at_bf16x8 v = __builtin_bit_cast(at_bf16x8, o[i]);
        asm volatile("" : "+v"(v)::"memory");
        o[i] = __builtin_bit_cast(uint4, v);
    }
}
__device__ __forceinline__ at_bf16x8 at_op(uint4 v) { return __builtin_bit_cast(at_bf16x8, v); }

// Q as the second operand of S^T = K Q^T: lane (q, hh) holds dims kk*16 + hh*8 .. +7.
__device__ __forceinline__ void at_load_q(const uint16_t* qrow, int hh, uint4 (&qr)[4]) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) qr[kk] = *reinterpret_cast<const uint4*>(qrow + kk * 16 + hh * 8);
}
// s[b][i] = raw score of key 32 b + (i/4)*8 + hh*4 + i%4 of the tile and the lane's query.
__device__ __forceinline__ void at_scores(const uint4 (&ka)[4], const uint4 (&kb)[4], const uint4 (&qr)[4], at_f32x16 (&s)[2]) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at_op(b ? kb[kk] : ka[kk]), at_op(qr[kk]), s[b], 0, 0, 0);
    }
}
// Lane addresses of a staged tile: K operands kr, V blocks vr by (second 8 keys, second 32 dims).
struct AtAddr {
    uint32_t kr[4], vr[2][2];
};
__device__ __forceinline__ AtAddr at_addresses(uint32_t s0, int lane) {
    const int ql = lane & 31, hh = lane >> 5, i16 = lane & 15, g16 = (lane >> 4) & 1;
    AtAddr r;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) r.kr[kk] = s0 + ql * 128 + (((2 * kk + hh) ^ ((ql >> 1) & 7)) << 4);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const int row = e * 8 + hh * 4 + (i16 >> 2), piece = d * 4 + g16 * 2 + ((i16 & 3) >> 1);
            r.vr[e][d] = s0 + kAtTile + row * 128 + ((piece ^ ((row >> 1) & 7)) << 4) + (i16 & 1) * 8;
        }
    return r;
}
__device__ __forceinline__ void at_read_k(const AtAddr& r, uint32_t so, uint4 (&ka)[4], uint4 (&kb)[4]) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) ka[kk] = at_read<0>(r.kr[kk] + so);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) kb[kk] = at_read<4096>(r.kr[kk] + so);
}
__device__ __forceinline__ void at_read_v(const AtAddr& r, uint32_t so, uint64_t (&v)[2][2][4]) {
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            v[d][e][0] = at_read_tr<0>(r.vr[e][d] + so);
            v[d][e][1] = at_read_tr<2048>(r.vr[e][d] + so);
            v[d][e][2] = at_read_tr<4096>(r.vr[e][d] + so);
            v[d][e][3] = at_read_tr<6144>(r.vr[e][d] + so);
        }
}
__device__ __forceinline__ void at_tie_v(uint64_t (&v)[2][2][4]) {
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e) at_tie(v[d][e]);
}
__device__ __forceinline__ void at_wait_lds() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

}  // namespace ftts
