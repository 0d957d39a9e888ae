// Rows turned by their positions, and keys and values turned on their way into their pages.
//
// A pair (a, b) of a head's columns becomes scale (a cos t - b sin t, b cos t + a sin t), t = 2 pi p turns[i]: one
// complex product, 6 operations for 4 (8) bytes, so what bounds it is memory, and in small calls the launch and two
// dependent trips (slot, then rows beside the angles).
//
// A wave takes a part of a row, 64 pieces of 8 columns once or twice, which it asks for at once.  A row's heads share
// its angles: lane i makes pair i's cosine and sine once, and a piece's 8 columns are the same in every head that the
// lane meets, so each lane then keeps the 8 (4) pairs of its own.  The angle is reduced in fp64 to within an eighth of
// a turn: a product in fp32 would lose position 2^20 of a pair that turns by a radian to 0.06 rad.
//
// A workgroup's waves take the same part of four rows in turn, so four tokens of a page are written together.  10,827
// rows of 20 heads of queries, keys and values, 166 MB: 38.8 us, 4.3 TB/s, 86% of a large copy's rate; waves that took
// whole rows in two rounds of four pieces 42.9 (longer batches are slower: 49.4 with eight pieces).  9,746 rows of 20
// heads turned alone, 50 MB: 12.0 us (12.8).  The smallest calls take 2.8 us, their launch and the two trips.
#include <algorithm>
#include <cmath>

#include "decode_entry.hpp"

namespace ftts {

constexpr int kRotWaves = 4, kRotAhead = 2;  // waves a workgroup; pieces of a lane
constexpr int kRotEnough = 2048;             // waves that fill the card: fewer rows are cut into smaller parts

struct RotArgs {
    const void *q, *k, *v;
    int64_t q_ld, k_ld, v_ld;
    int rows, n_head, n_kv_head, parts;
    int half;                // pairs turned in each head
    float scale;
    const int32_t* positions;
    const int32_t* slots;    // null: every row, queries only
    void* q_out;
    int64_t q_out_ld;
    void* base;
    int n_pages, layer;
    double turns[FTTS_ROTARY_MAX_PAIRS];
};

// Where a pair's columns lie: neighbours, or half of the turned columns apart, which is whole pieces or not.
enum { ROT_PAIRS, ROT_HALVES, ROT_HALVES_ANY };

template <bool F32>
struct RotPiece {  // 8 columns as they come
    uint4 x[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ void rot_unpack(const RotPiece<F32>& r, float (&x)[8]) {
    if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[4 * i] = __uint_as_float(r.x[i].x);
            x[4 * i + 1] = __uint_as_float(r.x[i].y);
            x[4 * i + 2] = __uint_as_float(r.x[i].z);
            x[4 * i + 3] = __uint_as_float(r.x[i].w);
        }
    } else {
        const uint32_t w[4] = {r.x[0].x, r.x[0].y, r.x[0].z, r.x[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16lo(w[i]);
            x[2 * i + 1] = bf16hi(w[i]);
        }
    }
}
template <bool F32>
__device__ __forceinline__ void rot_store(void* p, size_t at, const float (&x)[8]) {
    if constexpr (F32) {
        float4* d = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + at);
        d[0] = make_float4(x[0], x[1], x[2], x[3]);
        d[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        auto pair = [](float lo, float hi) { return (uint32_t)f32_to_bf16(lo) | ((uint32_t)f32_to_bf16(hi) << 16); };
        *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p) + at) =
            make_uint4(pair(x[0], x[1]), pair(x[2], x[3]), pair(x[4], x[5]), pair(x[6], x[7]));
    }
}

// Cosine and sine of `turns` turns a position, p positions on.
__device__ __forceinline__ float2 rot_unit(int p, double turns) {
    const double t = (double)p * turns, quarter = 4.0 * (t - floor(t)), n = rint(quarter);
    float c, s;
    sincospif(0.5f * (float)(quarter - n), &s, &c);  // within an eighth of a turn: rounded by 2^-28 turns
    switch ((int)n & 3) {
        case 1: return make_float2(-s, c);
        case 2: return make_float2(-c, -s);
        case 3: return make_float2(s, -c);
        default: return make_float2(c, s);
    }
}

template <bool SRC32, bool DST32, int LAYOUT>
__global__ __launch_bounds__(kRotWaves * 64) void turn_rows_kernel(const RotArgs a) {
    constexpr bool kAny = LAYOUT == ROT_HALVES_ANY;
    __shared__ float stage[kAny ? kRotWaves * kWave * 8 : 1];  // a wave's pieces in fp32
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = blockIdx.x * kRotWaves + wave, part = blockIdx.y;
    if (row >= a.rows) return;
    const int slot = a.slots ? a.slots[row] : 0;
    if (a.slots && (slot < 0 || slot / kPage >= a.n_pages)) return;
    const int n_q = 8 * a.n_head, n_k = 8 * a.n_kv_head, all = n_q + 2 * n_k;
    RotPiece<SRC32> in[kRotAhead];
    auto load = [&](int j, RotPiece<SRC32>& r) {
        if (j >= all) return;
        const int of = j < n_q ? 0 : j < n_q + n_k ? 1 : 2, p = j - (of > 0) * n_q - (of > 1) * n_k;
        const void* from = of == 0 ? a.q : of == 1 ? a.k : a.v;
        const size_t at = (size_t)row * (of == 0 ? a.q_ld : of == 1 ? a.k_ld : a.v_ld) + 8 * p;
        if constexpr (SRC32) {
            const uint4* s = reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(from) + at);
            r.x[0] = s[0];
            r.x[1] = s[1];
        } else {
            r.x[0] = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(from) + at);
        }
    };
    const int step = kWave * a.parts, j0 = part * kWave + lane;
#pragma unroll
    for (int u = 0; u < kRotAhead; ++u) load(j0 + u * step, in[u]);

    const float2 unit = rot_unit(a.positions[row], a.turns[lane & 31]);
    const float cv = unit.x * a.scale, sv = unit.y * a.scale;
    // this lane's columns 8 c .. 8 c + 7 of every head; columns from 2 half on pass
    const int c0 = 8 * (lane & 7), turned = 2 * a.half;
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = c0 + i, pair = LAYOUT == ROT_PAIRS ? e >> 1 : e < a.half ? e : e - a.half;
        const bool second = LAYOUT == ROT_PAIRS ? i & 1 : e >= a.half;
        cs[i] = __shfl(cv, pair & 31, kWave);
        const float s = __shfl(sv, pair & 31, kWave);
        sn[i] = second ? s : -s;
    }
    auto turn = [&](const float (&x)[8], bool turns, float (&y)[8]) {
        float z[8];  // the other column of each pair
        if constexpr (LAYOUT == ROT_PAIRS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = x[i ^ 1];
        } else if constexpr (LAYOUT == ROT_HALVES) {
            const int other = c0 < a.half ? lane + a.half / 8 : lane - a.half / 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = __shfl(x[i], other & 63, kWave);
        } else {
            float* own = stage + wave * kWave * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) own[8 * lane + i] = x[i];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = c0 + i, o = e < a.half ? e + a.half : e < turned ? e - a.half : e;
                z[i] = own[8 * (lane & ~7) + o];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = turns && c0 + i < turned ? fmaf(x[i], cs[i], z[i] * sn[i]) : x[i];
    };
#pragma unroll
    for (int u = 0; u < kRotAhead; ++u) {
        if (part * kWave + u * step >= all) break;  // (the same for the whole wave)
        const int j = j0 + u * step;
        float x[8] = {}, y[8];
        if (j < all) rot_unpack<SRC32>(in[u], x);
        turn(x, j < n_q + n_k, y);
        if (j >= all) continue;
        if (j < n_q) {
            rot_store<DST32>(a.q_out, (size_t)row * a.q_out_ld + 8 * j, y);
        } else {
            const int kv = j >= n_q + n_k, p = j - n_q - kv * n_k;
            rot_store<DST32>(a.base, kv_offset(a.layer, a.n_pages, slot / kPage, kv, a.n_kv_head, p >> 3, slot % kPage) + 8 * (p & 7), y);
        }
    }
}

static hipError_t launch_turn(int src, int dst, int layout, const RotArgs& args, hipStream_t st) {
    RotArgs a = args;
    const int pieces = 8 * a.n_head + 16 * a.n_kv_head, turns = (pieces + kWave - 1) / kWave;
    a.parts = std::min(std::max((kRotEnough + a.rows - 1) / a.rows, (turns + kRotAhead - 1) / kRotAhead), turns);
    const dim3 g((unsigned)((a.rows + kRotWaves - 1) / kRotWaves), a.parts), t(kRotWaves * 64);
    const int form = layout == FTTS_ROTARY_PAIRS ? ROT_PAIRS : a.half % 8 == 0 ? ROT_HALVES : ROT_HALVES_ANY;
#define FTTS_TURN(S, D)                                                                                      \
    do {                                                                                                     \
        if (form == ROT_PAIRS) hipLaunchKernelGGL((turn_rows_kernel<S, D, ROT_PAIRS>), g, t, 0, st, a);      \
        else if (form == ROT_HALVES) hipLaunchKernelGGL((turn_rows_kernel<S, D, ROT_HALVES>), g, t, 0, st, a); \
        else hipLaunchKernelGGL((turn_rows_kernel<S, D, ROT_HALVES_ANY>), g, t, 0, st, a);                   \
    } while (0)
    (void)hipGetLastError();
    if (src == FTTS_BF16) FTTS_TURN(false, false);
    else if (dst == FTTS_BF16) FTTS_TURN(true, false);
    else FTTS_TURN(true, true);
#undef FTTS_TURN
    return hipGetLastError();
}

}  // namespace ftts

using namespace ftts;

namespace {

int check_rotary(const char* call, int src, int dst, const ftts_rotary* r, int n_rows) {
    if ((src != FTTS_F32 && src != FTTS_BF16) || (dst != FTTS_F32 && dst != FTTS_BF16))
        return set_error(FTTS_E_DTYPE, "%s: dtypes must be FTTS_F32 or FTTS_BF16", call);
    if (src == FTTS_BF16 && dst == FTTS_F32) return set_error(FTTS_E_DTYPE, "%s: bf16 rows into fp32", call);
    if (!r) return set_error(FTTS_E_INVALID_ARG, "%s: rotation is NULL", call);
    if (r->dim < 2 || r->dim > kHeadDim || r->dim % 2)
        return set_error(FTTS_E_SHAPE, "%s: turned columns must be even, 2 to 64 (got %d)", call, r->dim);
    if (r->layout != FTTS_ROTARY_HALVES && r->layout != FTTS_ROTARY_PAIRS)
        return set_error(FTTS_E_INVALID_ARG, "%s: unknown layout %d", call, r->layout);
    if (!std::isfinite(r->scale)) return set_error(FTTS_E_RANGE, "%s: scale must be finite", call);
    for (int i = 0; i < r->dim / 2; ++i)
        if (!(std::fabs(r->turns[i]) <= 1.0)) return set_error(FTTS_E_RANGE, "%s: turns[%d] must be in [-1, 1]", call, i);
    if (n_rows < 0 || n_rows > (1 << 24)) return set_error(FTTS_E_RANGE, "%s: n_rows must be in [0, 2^24]", call);
    return FTTS_OK;
}

// A strided array of rows of whole heads.
struct Rows {
    const void* p;
    int64_t stride;  // elements
    int heads, esize;
};
int check_rows(const char* call, const char* name, const Rows& r) {
    if (!r.p) return set_error(FTTS_E_INVALID_ARG, "%s: %s is NULL", call, name);
    if (r.stride < 64LL * r.heads || r.stride > (1LL << 31) || r.stride * r.esize % 16)
        return set_error(FTTS_E_SHAPE, "%s: the stride of %s must be a multiple of 16 bytes, at least 64 * heads", call, name);
    if (reinterpret_cast<uintptr_t>(r.p) & 15u) return set_error(FTTS_E_ALIGN, "%s: %s is not 16-byte aligned", call, name);
    return FTTS_OK;
}
// Whether two arrays of n rows share bytes: not where they are different columns of the same rows.
bool collide(const Rows& a, const Rows& b, int n) {
    const uint64_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    const uint64_t sa = a.stride * a.esize, sb = b.stride * b.esize, wa = 64ull * a.heads * a.esize, wb = 64ull * b.heads * b.esize;
    if (x >= y + (n - 1) * sb + wb || y >= x + (n - 1) * sa + wa) return false;
    if (n == 1 || sa != sb) return true;
    const uint64_t d = y >= x ? (y - x) % sa : (sa - (x - y) % sa) % sa;
    return d < wa || d + wb > sa;
}
bool same(const Rows& a, const Rows& b, int n) { return a.p == b.p && a.esize == b.esize && (n == 1 || a.stride == b.stride); }

RotArgs rot_args(const ftts_rotary& r, int n_rows, const int32_t* positions) {
    RotArgs a{};
    a.rows = n_rows;
    a.half = r.dim / 2;
    a.scale = r.scale;
    a.positions = positions;
    for (int i = 0; i < a.half; ++i) a.turns[i] = r.turns[i];
    return a;
}

}  // namespace

extern "C" {

int ftts_rotary_init(int32_t dim, int32_t layout, double base, int32_t scaling, double factor, double original, double slow,
                     double fast, ftts_rotary* out) {
    if (!out) return set_error(FTTS_E_INVALID_ARG, "rotary_init: out is NULL");
    if (dim < 2 || dim > kHeadDim || dim % 2)
        return set_error(FTTS_E_SHAPE, "rotary_init: turned columns must be even, 2 to 64 (got %d)", dim);
    if (layout != FTTS_ROTARY_HALVES && layout != FTTS_ROTARY_PAIRS)
        return set_error(FTTS_E_INVALID_ARG, "rotary_init: unknown layout %d", layout);
    if (scaling < FTTS_ROTARY_PLAIN || scaling > FTTS_ROTARY_PARTS)
        return set_error(FTTS_E_INVALID_ARG, "rotary_init: unknown scaling %d", scaling);
    if (!(base > 1.0) || !std::isfinite(base)) return set_error(FTTS_E_RANGE, "rotary_init: base must be finite and above 1");
    if (scaling != FTTS_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
        return set_error(FTTS_E_RANGE, "rotary_init: factor must be finite and at least 1");
    if (scaling == FTTS_ROTARY_BASE && dim < 4) return set_error(FTTS_E_SHAPE, "rotary_init: a larger base needs 4 columns");
    if (scaling == FTTS_ROTARY_PARTS && (!(original >= 1.0) || !std::isfinite(original) || !(slow >= 0.0) || !(fast > slow) ||
                                         !std::isfinite(fast)))
        return set_error(FTTS_E_RANGE, "rotary_init: needs original >= 1 and 0 <= slow < fast, finite");
    if (scaling == FTTS_ROTARY_BASE) base *= std::pow(factor, (double)dim / (dim - 2));
    if (!std::isfinite(base)) return set_error(FTTS_E_RANGE, "rotary_init: the larger base is not finite");
    const double two_pi = 6.283185307179586476925;
    ftts_rotary r{};
    r.dim = dim;
    r.layout = layout;
    r.scale = 1.f;
    for (int i = 0; i < dim / 2; ++i) {
        double t = std::pow(base, -2.0 * i / dim) / two_pi;
        if (scaling == FTTS_ROTARY_LINEAR) t /= factor;
        if (scaling == FTTS_ROTARY_PARTS) {
            const double keep = std::min(std::max((original * t - slow) / (fast - slow), 0.0), 1.0);
            t = t * keep + t / factor * (1.0 - keep);
        }
        r.turns[i] = t;
    }
    if (scaling == FTTS_ROTARY_PARTS) r.scale = (float)(0.1 * std::log(factor) + 1.0);
    *out = r;
    return FTTS_OK;
}

int ftts_rotate(int32_t src_dtype, int32_t dst_dtype, const ftts_rotary* rot, const void* x, int64_t x_stride,
                int32_t n_rows, int32_t n_head, const int32_t* positions, void* out, int64_t out_stride, void* stream) {
    if (int rc = check_rotary("rotate", src_dtype, dst_dtype, rot, n_rows)) return rc;
    if (n_head < 1 || n_head > 256) return set_error(FTTS_E_SHAPE, "rotate: n_head must be in [1, 256]");
    if (n_rows == 0) return FTTS_OK;
    const Rows in{x, x_stride, n_head, src_dtype == FTTS_F32 ? 4 : 2}, to{out, out_stride, n_head, dst_dtype == FTTS_F32 ? 4 : 2};
    if (int rc = check_rows("rotate", "x", in)) return rc;
    if (int rc = check_rows("rotate", "out", to)) return rc;
    if (!positions) return set_error(FTTS_E_INVALID_ARG, "rotate: positions is NULL");
    if (reinterpret_cast<uintptr_t>(positions) & 3u) return set_error(FTTS_E_ALIGN, "rotate: positions not 4-byte aligned");
    if (!same(in, to, n_rows) && collide(in, to, n_rows)) return set_error(FTTS_E_INVALID_ARG, "rotate: out overlaps x");
    RotArgs a = rot_args(*rot, n_rows, positions);
    a.q = x;
    a.q_ld = x_stride;
    a.n_head = n_head;
    a.q_out = out;
    a.q_out_ld = out_stride;
    const hipError_t e = launch_turn(src_dtype, dst_dtype, rot->layout, a, (hipStream_t)stream);
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "rotate launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

int ftts_append_rotated(int32_t src_dtype, int32_t kv_dtype, const ftts_rotary* rot, const void* q, int64_t q_stride,
                        int32_t n_head, void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride, const void* v,
                        int64_t v_stride, int32_t n_rows, const int32_t* positions, const int32_t* slots,
                        const ftts_kv_pool* kv, int32_t layer, int32_t n_kv_head, void* stream) {
    const char* me = "append_rotated";
    if (int rc = check_rotary(me, src_dtype, kv_dtype, rot, n_rows)) return rc;
    if (!kv || !kv->base) return set_error(FTTS_E_INVALID_ARG, "append_rotated: pool is NULL");
    if (n_head < 0 || n_head > 256 || n_kv_head < 1 || n_kv_head > 256)
        return set_error(FTTS_E_SHAPE, "append_rotated: n_head must be in [0, 256] and n_kv_head in [1, 256]");
    if (kv->n_pages < 1 || layer < 0) return set_error(FTTS_E_SHAPE, "append_rotated: n_pages must be >= 1 and layer >= 0");
    if (reinterpret_cast<uintptr_t>(kv->base) & 15u) return set_error(FTTS_E_ALIGN, "append_rotated: pool is not 16-byte aligned");
    if (n_head == 0 && (q || q_out)) return set_error(FTTS_E_SHAPE, "append_rotated: queries of 0 heads");
    if (n_rows == 0) return FTTS_OK;
    const int es = src_dtype == FTTS_F32 ? 4 : 2, ed = kv_dtype == FTTS_F32 ? 4 : 2;
    const Rows rq{q, q_stride, n_head, es}, to{q_out, q_out_stride, n_head, ed}, rk{k, k_stride, n_kv_head, es}, rv{v, v_stride, n_kv_head, es};
    if (int rc = check_rows(me, "k", rk)) return rc;
    if (int rc = check_rows(me, "v", rv)) return rc;
    if (!positions || !slots) return set_error(FTTS_E_INVALID_ARG, "append_rotated: positions/slots is NULL");
    if ((reinterpret_cast<uintptr_t>(positions) | reinterpret_cast<uintptr_t>(slots)) & 3u)
        return set_error(FTTS_E_ALIGN, "append_rotated: positions/slots not 4-byte aligned");
    RotArgs a = rot_args(*rot, n_rows, positions);
    if (n_head > 0) {
        if (int rc = check_rows(me, "q", rq)) return rc;
        if (int rc = check_rows(me, "q_out", to)) return rc;
        if ((!same(rq, to, n_rows) && collide(rq, to, n_rows)) || collide(rk, to, n_rows) || collide(rv, to, n_rows))
            return set_error(FTTS_E_INVALID_ARG, "append_rotated: q_out overlaps q, k or v");
        a.q = q;
        a.q_ld = q_stride;
        a.n_head = n_head;
        a.q_out = q_out;
        a.q_out_ld = q_out_stride;
    }
    a.k = k;
    a.v = v;
    a.k_ld = k_stride;
    a.v_ld = v_stride;
    a.n_kv_head = n_kv_head;
    a.slots = slots;
    a.base = kv->base;
    a.n_pages = kv->n_pages;
    a.layer = layer;
    const hipError_t e = launch_turn(src_dtype, kv_dtype, rot->layout, a, (hipStream_t)stream);
    if (e != hipSuccess) return set_error(FTTS_E_HIP, "append_rotated launch: %s", hipGetErrorString(e));
    return FTTS_OK;
}

}  // extern "C"
