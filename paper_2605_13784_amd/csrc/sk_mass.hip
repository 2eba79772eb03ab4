// Attention weight that cached tokens receive, summed over a call's query rows (include/sk.h: sk_session_attention_mass), gfx950.
//
//   mass[g][j] = keep * mass[g][j] + sum over the rows (i, h) of KV head g of exp(scale * q_ih . k_gj - lse_ih)
//
// The row's log-sum-exp is known, so no maximum is looked for and no weight is kept: a score becomes a weight (one FMA, one
// exponential) and joins its key's sum (one addition).  Scores come from the matrix pipe with the keys as its columns
// (S = Q K^T): a lane then holds 16 rows of ONE key, whose weights it adds in registers, and only its two halves (and the
// waves that share keys) meet at the end.  The keys stay in registers, read once; the rows pass by.
// Bound: K's stream from HBM for few rows; for many the exponentials and the matrix products, which take the same time.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>
#include "../../include/sk.h"
#include "sk_internal.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kItems = 48;            // sessions of a launch, carried in its arguments

struct Item {
    int32_t tbl_off;      // of the session's block table
    int32_t q_tok0, n_tok;
    int32_t n_keys;       // retained tokens
    int32_t hole_lo, hole_n;          // retained token j lies at storage index j, from hole_lo on at j + hole_n
    int32_t first_vis;    // keys that token 0 sees: token i sees those below first_vis + i * causal
    int32_t causal;
    int32_t tile0;        // the launch's key tiles before this item's (a tile: the keys of a workgroup)
    int32_t pad;
    const float* in;
    float* out;
    int64_t in_stride, out_stride;
};

struct Args {
    sk_geom g;
    const unsigned char* q;
    const float* lse;
    float keep;
    int32_t n_items;
    Item item[kItems];
};

// A wave's operand of 32 rows x D elements: lane holds row (lane % 32), in bf16 elements 16 s + 8 (lane / 32) .. + 7 of each step s of
// the matrix instruction, in fp32 the half (lane / 32) of the row (both operands in the same order: a product does not depend on it).
template <int D, bool F32> struct Operand { u32x4 v[F32 ? D / 8 : D / 16]; };

template <int D, bool F32>
__device__ __forceinline__ void load_operand(Operand<D, F32>& o, const unsigned char* row, const int half)
{
    constexpr int N = F32 ? D / 8 : D / 16;
    const unsigned char* p = row + (F32 ? half * (D * 2) : half * 16);
#pragma unroll
    for (int s = 0; s < N; ++s) o.v[s] = *(const u32x4*)(p + s * (F32 ? 16 : 32));
}

template <int D, bool F32>
__device__ __forceinline__ f32x16 product(const Operand<D, F32>& a, const Operand<D, F32>& b)
{
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
    constexpr int N = F32 ? D / 8 : D / 16;
#pragma unroll
    for (int s = 0; s < N; ++s) {
        if constexpr (F32) {
            const f32x4 x = __builtin_bit_cast(f32x4, a.v[s]), y = __builtin_bit_cast(f32x4, b.v[s]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
        } else {
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v[s]), __builtin_bit_cast(bf16x8, b.v[s]), acc, 0, 0, 0);
        }
    }
    return acc;
}

// Workgroup (key tile, KV head) of four waves: 4 / WR of them side by side along the keys, KT x 32 keys each, and WR that take
// the row tiles in turn.
template <int D, bool F32, int KT, int WR>
__global__ __launch_bounds__(256) void sk_mass_kernel(const Args A)
{
    __shared__ float sums[WR > 1 ? WR : 1][KT * 32];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    const int Hkv = A.g.Hkv, G = A.g.G;
    const int tile = blockIdx.x / Hkv, head = blockIdx.x - tile * Hkv;
    // the item that this tile belongs to: the last one that starts at or before it
    int it = 0;
    if (A.n_items > 1) {
        const int t0 = lane < A.n_items ? A.item[lane].tile0 : 0x7fffffff;
        it = __builtin_amdgcn_readfirstlane(__popcll(__ballot(t0 <= tile)) - 1);
    }
    const Item I = A.item[it];
    const int k0 = (tile - I.tile0) * (KT * 32 * (4 / WR)) + (wave / WR) * (KT * 32);
    const int row_bytes = D * (F32 ? 4 : 2);

    Operand<D, F32> key[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        int j = k0 + 32 * t + col;
        j = j < I.n_keys ? j : I.n_keys - 1;              // (a key behind the last one is not written)
        const int st = j + (j >= I.hole_lo ? I.hole_n : 0);
        const int blk = A.g.tables[I.tbl_off + (st >> A.g.log2B)];
        load_operand<D, F32>(key[t], A.g.kv + (int64_t)head * A.g.head_stride + (int64_t)blk * A.g.blk_stride + (int64_t)(st & (A.g.B - 1)) * row_bytes, half);
    }
    float sum[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) sum[t] = 0.f;

    const int n_rows = I.n_tok * G;
    // tokens below `tok0` see none of the wave's keys
    int tok0 = I.causal ? k0 - I.first_vis + 1 : 0;
    tok0 = tok0 > 0 ? tok0 : 0;
    const float c = A.g.scale_log2e;
    const int step = WR > 1 ? 32 * WR : 32;
    for (int r0 = (tok0 * G & ~31) + (WR > 1 ? 32 * (wave % WR) : 0); r0 < n_rows && k0 < I.n_keys; r0 += step) {
        Operand<D, F32> q;
        float l;
        {
            const int r = r0 + col < n_rows ? r0 + col : n_rows - 1;
            const int tok = (int)((unsigned)r / (unsigned)G), h = head * G + (r - tok * G);
            const int64_t at = (int64_t)(I.q_tok0 + tok) * A.g.Hq + h;
            load_operand<D, F32>(q, A.q + at * row_bytes, half);
            l = A.lse[at] * kLog2e;
            // a row that is left out: weight exp2(0 - inf), whatever its q holds
            if (r0 + col >= n_rows || __builtin_isinf(l)) {
                l = __builtin_inff();
#pragma unroll
                for (int s = 0; s < (F32 ? D / 8 : D / 16); ++s) q.v[s] = u32x4{0, 0, 0, 0};
            }
        }
        const int row = 4 * half;                         // the accumulator's register v: row (v & 3) + 8 (v >> 2) + 4 half
        // (the first row of the tile sees the fewest keys)
        const int least = I.first_vis + I.causal * (r0 / G);
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const f32x16 s = product<D, F32>(q, key[t]);
            const int j = k0 + 32 * t + col;
            const bool edge = k0 + 32 * t + 31 >= least;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int r = row + (v & 3) + 8 * (v >> 2);
                float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, -__shfl(l, r, 64)));
                if (edge && I.causal) w = j < I.first_vis + (int)((unsigned)(r0 + r) / (unsigned)G) ? w : 0.f;
                sum[t] += w;
            }
        }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) sum[t] += __shfl_xor(sum[t], 32, 64);
    if (WR > 1) {
#pragma unroll
        for (int t = 0; t < KT; ++t) if (half == 0) sums[wave % WR][32 * t + col] = sum[t];
        __syncthreads();
        if (wave % WR != 0) return;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int w = 1; w < WR; ++w) sum[t] += sums[w][32 * t + col];
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        const int j = k0 + 32 * t + col;
        if (half == 0 && j < I.n_keys) {
            float m = sum[t];
            if (I.in) m += A.keep * I.in[head * I.in_stride + j];
            I.out[head * I.out_stride + j] = m;
        }
    }
}

template <int D, bool F32>
int launch(const Args& A, const int wr, const int tiles, hipStream_t st)
{
    const dim3 grid((unsigned)tiles * (unsigned)A.g.Hkv), block(256);
    if (wr == 4) hipLaunchKernelGGL((sk_mass_kernel<D, F32, 2, 4>), grid, block, 0, st, A);
    else hipLaunchKernelGGL((sk_mass_kernel<D, F32, 1, 1>), grid, block, 0, st, A);
    return (int)hipGetLastError();
}

// The items of one call, which share q and lse.
struct Call {
    int32_t n_items;
    const int32_t *session_id, *causal, *cu_tokens;
    const void* q;
    const float* lse;
    const float* const* in;       // null: none
    const int64_t* in_stride;
    float keep;
    float* const* out;
    const int64_t* out_stride;
};

int check(sk_pool* p, const Call& C)
{
    if (C.cu_tokens[0] != 0) return SK_E_INVAL;
    sk_session_view V;
    for (int32_t i = 0; i < C.n_items; ++i) {
        const int rc = sk_view_session(p, C.session_id[i], &V);
        if (rc) return rc;
        const int64_t T = (int64_t)C.cu_tokens[i + 1] - C.cu_tokens[i], n = V.retained;
        if (T < 0 || (C.causal && C.causal[i] != 0 && T > n)) return SK_E_INVAL;
        if (!V.device) continue;
        if (n == 0) continue;
        if (!C.out[i] || (uintptr_t)C.out[i] & 3 || C.out_stride[i] < n) return SK_E_INVAL;
        if (C.in && C.keep != 0.f && (!C.in[i] || (uintptr_t)C.in[i] & 3 || C.in_stride[i] < n ||
                                      sk_rows_overlap(C.in[i], C.in_stride[i], C.out[i], C.out_stride[i], V.g.Hkv, n))) return SK_E_INVAL;
        if (T > 0 && (!C.q || !C.lse || ((uintptr_t)C.q | (uintptr_t)C.lse) & 15)) return SK_E_INVAL;
    }
    if (!sk_sessions_differ(p, C.n_items, C.session_id)) return SK_E_INVAL;
    if (!V.device) return SK_E_NODEVICE;
    return C.cu_tokens[C.n_items] > V.max_batch_tokens ? SK_E_WORKSPACE : SK_OK;
}

int run(sk_pool* p, const Call& C, void* stream)
{
    const int rc = check(p, C);
    if (rc) return rc;
    hipStream_t st = (hipStream_t)stream;
    sk_session_view V;
    int64_t keys = 0, rows = 0;
    for (int32_t i = 0; i < C.n_items; ++i) {
        sk_view_session(p, C.session_id[i], &V);
        keys += V.retained;
        rows = std::max<int64_t>(rows, (int64_t)(C.cu_tokens[i + 1] - C.cu_tokens[i]) * V.g.G);
    }
    // few keys and several row tiles: the waves of a workgroup share their keys and take the rows in turn
    const int wr = rows > 32 && keys * V.g.Hkv < 512 * 128 ? 4 : 1;
    const int tile_keys = wr == 4 ? 64 : 128;
    Args A;
    A.q = (const unsigned char*)C.q; A.lse = C.lse; A.keep = C.keep;
    for (int32_t i = 0; i < C.n_items;) {
        A.n_items = 0;
        int64_t tiles = 0;
        for (; i < C.n_items && A.n_items < kItems; ++i) {
            sk_view_session(p, C.session_id[i], &V);
            A.g = V.g;
            if (V.retained == 0) continue;
            const int64_t t = (V.retained + tile_keys - 1) / tile_keys;
            if (A.n_items > 0 && (tiles + t) * V.g.Hkv >= (int64_t(1) << 31)) break;      // a launch's workgroups are counted in 31 bits
            Item& I = A.item[A.n_items++];
            I.tbl_off = V.tbl_off; I.q_tok0 = C.cu_tokens[i]; I.n_tok = C.cu_tokens[i + 1] - C.cu_tokens[i];
            I.n_keys = (int32_t)V.retained; I.hole_lo = (int32_t)V.frozen; I.hole_n = (int32_t)(V.win - V.frozen);
            I.causal = C.causal && C.causal[i] != 0 ? 1 : 0;
            I.first_vis = I.causal ? I.n_keys - I.n_tok + 1 : I.n_keys;
            I.tile0 = (int32_t)tiles; I.pad = 0;
            I.in = C.in && C.keep != 0.f ? C.in[i] : nullptr; I.in_stride = I.in ? C.in_stride[i] : 0;
            I.out = C.out[i]; I.out_stride = C.out_stride[i];
            tiles += t;
        }
        if (A.n_items == 0) break;                        // (only empty sessions were left)
        int e;
        if (A.g.elem == 4) e = A.g.d == 128 ? launch<128, true>(A, wr, (int)tiles, st) : launch<64, true>(A, wr, (int)tiles, st);
        else e = A.g.d == 128 ? launch<128, false>(A, wr, (int)tiles, st) : launch<64, false>(A, wr, (int)tiles, st);
        if (e) return sk_note_hip_error(e);
        sk_count_launch(p);
    }
    return SK_OK;
}

}  // namespace

extern "C" {

int sk_session_attention_mass(sk_pool* p, int32_t id, const void* q, const float* lse, int32_t n_tok, int32_t causal, const float* mass_in,
                              int64_t mass_in_stride, float keep, float* mass_out, int64_t mass_out_stride, void* hip_stream)
{
    if (!p || n_tok < 0) return SK_E_INVAL;
    const int32_t cu[2] = {0, n_tok};
    return run(p, Call{1, &id, &causal, cu, q, lse, mass_in ? &mass_in : nullptr, &mass_in_stride, keep, &mass_out, &mass_out_stride}, hip_stream);
}

int sk_batch_attention_mass(sk_pool* p, int32_t n_items, const int32_t* session_id, const int32_t* causal, const int32_t* cu_tokens,
                            const void* q, const float* lse, const float* const* mass_in, const int64_t* mass_in_stride, float keep,
                            float* const* mass_out, const int64_t* mass_out_stride, void* hip_stream)
{
    if (!p || n_items < 0) return SK_E_INVAL;
    if (n_items == 0) return SK_OK;
    if (!session_id || !cu_tokens || !mass_out || !mass_out_stride || (mass_in && !mass_in_stride)) return SK_E_INVAL;
    return run(p, Call{n_items, session_id, causal, cu_tokens, q, lse, mass_in, mass_in_stride, keep, mass_out, mass_out_stride}, hip_stream);
}

}  // extern "C"
