// The turn of pairs of dimensions by a token's position, and the commit that turns on the way, shared by sk_rotate.hip and the attention kernel that turns
// its own rows (sk_kernels.hip).
//
// Pair i of the first `rotary` dimensions is a point in the plane that a token at position p turns by the angle p f_i:
//   (a, b) -> (a cos - b sin, a sin + b cos) * factor
// Turns add up: what moves a key from one position to another is the turn by the difference, whatever position it had.
//
// Angles.  p f_i exceeds what 32 bits hold long before it does so for p: at position 10^6 a float's angle is off by 0.03.  Only the
// part of a full turn that is left counts, and that is an integer product: step_i = f_i / (2 pi) as a fraction of 2^64, p step_i modulo 2^64,
// of which the upper 32 bits are kept (2^-32 of a turn; step_i itself is off by 2^-65 of one a position, 2^-34 at position 2^31).  The upper two bits of
// those, rounded, are the quadrant; what is left, at most pi / 4, goes through the series of sine and cosine, whose next terms are
// below 2^-28.
//
// Which products join an addition is written out: a row has the same bits whichever kernel turns it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "sk_internal.h"

namespace sk_turn {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

__device__ __forceinline__ uint32_t phase_of(const int32_t p, const uint64_t step)
{
    const uint32_t lo = (uint32_t)step, hi = (uint32_t)(step >> 32);
    return __umulhi((uint32_t)p, lo) + (uint32_t)p * hi - (p < 0 ? lo : 0u);      // bits 32 to 63 of p * step
}

// cos and sin of a phase (2^32: a full turn)
__device__ __forceinline__ f32x2 cos_sin(const uint32_t phase)
{
#pragma clang fp contract(off)
    const uint32_t quadrant = (phase + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(phase - (quadrant << 30)) * 1.4629180792671596e-09f;      // 2 pi / 2^32
    const float y = x * x;
    float s = fmaf(y, 2.7557319e-06f, -1.9841270e-04f);                                        // 1/9!, 1/7!, 1/5!, 1/3!
    s = fmaf(y, s, 8.3333333e-03f);
    s = fmaf(y, s, -1.6666667e-01f);
    s = fmaf(y * x, s, x);
    float c = fmaf(y, -2.7557319e-07f, 2.4801587e-05f);                                        // 1/10!, 1/8!, 1/6!, 1/4!, 1/2!
    c = fmaf(y, c, -1.3888889e-03f);
    c = fmaf(y, c, 4.1666667e-02f);
    c = fmaf(y, c, -0.5f);
    c = fmaf(y, c, 1.f);
    const float a = quadrant & 1 ? s : c, b = quadrant & 1 ? c : s;
    return f32x2{__uint_as_float(__float_as_uint(a) ^ ((quadrant + 1) & 2) << 30), __uint_as_float(__float_as_uint(b) ^ (quadrant & 2) << 30)};
}

// Steps of the eight pairs of a unit, asked for ahead of the rows that they turn (units that do not turn have some too)
struct Steps { uint64_t of[8]; };
__device__ __forceinline__ Steps steps_of(const sk_rotation& rot, const int unit)
{
    Steps s;
#pragma unroll
    for (int i = 0; i < 8; ++i) s.of[i] = rot.step[8 * unit + i];
    return s;
}
// cos and sin of those pairs
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ Turn turn_of(const Steps& steps, const int32_t position, const float factor)
{
#pragma clang fp contract(off)
    Turn t;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const f32x2 cs = cos_sin(phase_of(position, steps.of[i]));
        t.c[i] = cs.x * factor; t.s[i] = cs.y * factor;
    }
    return t;
}

// A unit of a row: sixteen elements that one thread turns (eight pairs) or, behind the rotary dimensions, passes on.  Halves: eight
// elements of either half; neighbours: sixteen in a row.
template <bool F32> struct Unit { u32x4 x[F32 ? 4 : 2]; };
struct Place { int lo, hi; };      // byte offsets of its two stretches of eight elements
template <bool F32> __device__ __forceinline__ Place place_of(const sk_rotation& rot, const int unit)
{
    constexpr int EL = F32 ? 4 : 2;
    if (16 * unit < rot.rotary && !rot.interleaved) return Place{8 * unit * EL, (rot.rotary / 2 + 8 * unit) * EL};
    return Place{16 * unit * EL, (16 * unit + 8) * EL};
}
template <bool F32> __device__ __forceinline__ Unit<F32> load_unit(const unsigned char* row, const Place at)
{
    Unit<F32> u;
    constexpr int H = F32 ? 2 : 1;
#pragma unroll
    for (int i = 0; i < H; ++i) { u.x[i] = *(const u32x4*)(row + at.lo + 16 * i); u.x[H + i] = *(const u32x4*)(row + at.hi + 16 * i); }
    return u;
}
template <bool F32> __device__ __forceinline__ void store_unit(unsigned char* row, const Place at, const Unit<F32>& u)
{
    constexpr int H = F32 ? 2 : 1;
#pragma unroll
    for (int i = 0; i < H; ++i) { *(u32x4*)(row + at.lo + 16 * i) = u.x[i]; *(u32x4*)(row + at.hi + 16 * i) = u.x[H + i]; }
}

__device__ __forceinline__ float low(const uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(const uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(const float a, const float b)       // the one rounding of a turned element
{
    const bf16x2 r = __builtin_convertvector(f32x2{a, b}, bf16x2);
    return __builtin_bit_cast(uint32_t, r);
}

template <bool F32> __device__ __forceinline__ Unit<F32> turned(const Unit<F32>& u, const Turn& t, const bool interleaved)
{
#pragma clang fp contract(off)
    Unit<F32> r;
    float a[8], b[8];
    if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a[i] = __uint_as_float(interleaved ? u.x[i >> 1][2 * (i & 1)] : u.x[i >> 2][i & 3]);
            b[i] = __uint_as_float(interleaved ? u.x[i >> 1][2 * (i & 1) + 1] : u.x[2 + (i >> 2)][i & 3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t wa = interleaved ? u.x[i >> 2][i & 3] : u.x[0][i >> 1], wb = interleaved ? wa : u.x[1][i >> 1];
            a[i] = interleaved || !(i & 1) ? low(wa) : high(wa);
            b[i] = interleaved || (i & 1) ? high(wb) : low(wb);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = fmaf(a[i], t.c[i], -(b[i] * t.s[i])), y = fmaf(a[i], t.s[i], b[i] * t.c[i]);
        a[i] = x; b[i] = y;
    }
    if constexpr (F32) {
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            const float n = w & 1 ? b[w >> 1] : a[w >> 1], h = w < 8 ? a[w & 7] : b[w & 7];
            r.x[w >> 2][w & 3] = __float_as_uint(interleaved ? n : h);
        }
    } else {
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const uint32_t n = pack(a[w], b[w]), h = w < 4 ? pack(a[2 * w], a[2 * w + 1]) : pack(b[2 * w - 8], b[2 * w - 7]);
            r.x[w >> 2][w & 3] = interleaved ? n : h;
        }
    }
    return r;
}

// One (16-token group, KV head) of a commit or staging list, as the plain commit does it but for k.
// Bound: memory or round trips (256 tokens of 32/8 heads of 128: 4.6 us of the device's time, q's rows with them, against 4.8 for the plain commit alone;
// 4,096: 100 MB in 19 us, 5.3 TB/s).
template <int D, bool F32>
__device__ __forceinline__ void commit_group(const sk_geom& g, const sk_rotation& rot, const int32_t* positions, const int32_t pos0, const void* k, const void* v,
                                             const sk_scatter& it, const int head, int32_t* tables_rw, unsigned char* base, uint16_t* vt)
{
    constexpr int U = D / 16, ROWB = D * (F32 ? 4 : 2), PR = ROWB / 16, LD = D + 8;
    const int tid = threadIdx.x, row = tid / U, unit = tid % U;
    unsigned char* dst = base + it.dst_off + (int64_t)head * (it.to_eph ? g.eph_head_stride : g.head_stride);
    unsigned char* vdst = dst + (it.to_eph ? g.eph_v_off : g.v_off);
    if (it.tbl_index >= 0 && head == 0 && tid == 0) tables_rw[it.tbl_index] = it.block_id;
    const bool mine = row < it.count;
    const Steps steps = steps_of(rot, unit);
    int32_t position = pos0 + it.src_tok0 + row;
    if (mine && positions) position = positions[it.src_tok0 + row];
    const Place at = place_of<F32>(rot, unit);
    Unit<F32> u;
    if (mine) u = load_unit<F32>((const unsigned char*)k + ((int64_t)(it.src_tok0 + row) * g.Hkv + head) * ROWB, at);
    constexpr int NV = (16 * PR + 255) / 256;      // pieces of v that a thread takes
    u32x4 y[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int p = tid + 256 * i, r = p / PR;
        if (r < it.count) y[i] = *(const u32x4*)((const unsigned char*)v + ((int64_t)(it.src_tok0 + r) * g.Hkv + head) * ROWB + (p % PR) * 16);
    }
    if (mine) {
        if (16 * unit < rot.rotary) u = turned<F32>(u, turn_of(steps, position, rot.factor), rot.interleaved);
        store_unit<F32>(dst + (it.dst_slot0 + row) * ROWB, at, u);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int p = tid + 256 * i, r = p / PR;
        if (r < it.count) {
            if constexpr (F32) *(u32x4*)(vdst + (it.dst_slot0 + r) * ROWB + (p % PR) * 16) = y[i];
            else *(u32x4*)(vt + r * LD + (p % PR) * 8) = y[i];
        }
    }
    if constexpr (!F32) {                           // transposed within the group of 16 slots; slots behind the last token are 0
        __syncthreads();
        if (tid >= 2 * D) return;
        const int first = it.dst_slot0 & 15, dim = tid >> 1, s0 = (tid & 1) * 8 - first;
        uint16_t* vd = (uint16_t*)vdst + (size_t)(it.dst_slot0 >> 4) * D * 16 + dim * 16 + (tid & 1) * 8;
        uint32_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = (s0 + j >= 0 && s0 + j < it.count) ? vt[(s0 + j) * LD + dim] : 0u;
        if (first == 0) *(u32x4*)vd = u32x4{e[0] | (e[1] << 16), e[2] | (e[3] << 16), e[4] | (e[5] << 16), e[6] | (e[7] << 16)};
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (s0 + j >= 0) vd[j] = (uint16_t)e[j];
        }
    }
}

}  // namespace sk_turn
