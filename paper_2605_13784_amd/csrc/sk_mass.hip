// Attention weight that cached tokens receive, summed over a call's query rows (include/sk.h: sk_session_attention_mass), gfx950.
//
//   mass[g][j] = keep * mass[g][j] + sum over the rows (i, h) of KV head g of exp(scale * q_ih . k_gj - lse_ih)
//
// The row's log-sum-exp is known, so no maximum is looked for and no weight is kept: a score becomes a weight (one FMA, one
// exponential) and joins its key's sum (one addition).  Scores come from the matrix pipe with the keys as its columns
// (S = Q K^T): a lane then holds 16 rows of ONE key, whose weights it adds in registers, and only its two halves (and the
// waves that share keys) meet at the end.  The keys stay in registers, read once; the rows pass by.
// Bound: K's stream from HBM for few rows (one token at 131,072 cached, 268 MB, 41 us: 6.5 TB/s, the rate of a plain read); for many
// the exponentials and the matrix products, which overlap in part (256 tokens at 32,768, 6.9e10 operations, 72 us: 0.95 PFLOP/s).
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
    sk_div by_group;
    int32_t run, lds_rows;            // stream: key tiles of a workgroup, one behind the other; rows that its LDS holds
    int32_t parts;                    // parts of an item's rows
    float* part_sums;                 // [tile][part][head][keys of a tile]
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

template <int D, bool F32, int KT>
__device__ __forceinline__ void products(const Operand<D, F32>& a, const Operand<D, F32> (&b)[KT], f32x16 (&acc)[KT])
{
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[t][v] = 0.f;
    constexpr int N = F32 ? D / 8 : D / 16;
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            if constexpr (F32) {
                const f32x4 x = __builtin_bit_cast(f32x4, a.v[s]), y = __builtin_bit_cast(f32x4, b[t].v[s]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc[t], 0, 0, 0);
            } else {
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v[s]), __builtin_bit_cast(bf16x8, b[t].v[s]), acc[t], 0, 0, 0);
            }
        }
}

__device__ __forceinline__ int divide(const int n, const sk_div d) { return d.mul ? (int)(__umulhi((uint32_t)n, d.mul) >> d.shift) : n; }

// The item that workgroup tile `tile` belongs to: the last one that starts at or before it.
__device__ __forceinline__ int item_of(const Args& A, const int tile, const int lane)
{
    if (A.n_items == 1) return 0;
    const int t0 = lane < A.n_items ? A.item[lane].tile0 : 0x7fffffff;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(t0 <= tile)) - 1);
}

// Where retained key j's row lies (one behind the last: the last one's; its sum is not written): block and slot, and its byte offset.
struct Place {
    int32_t block, slot;
    __device__ __forceinline__ void find(const Args& A, const Item& I, int j)
    {
        j = j < I.n_keys ? j : I.n_keys - 1;
        const int st = j + (j >= I.hole_lo ? I.hole_n : 0);
        block = A.g.tables[I.tbl_off + (st >> A.g.log2B)];
        slot = st & (A.g.B - 1);
    }
    __device__ __forceinline__ int64_t at(const Args& A, const int row_bytes) const { return (int64_t)block * A.g.blk_stride + (int64_t)slot * row_bytes; }
};

// Query rows of an item on their way to LDS: a workgroup of THREADS threads takes ROWS of them at a time, THREADS / ROWS threads a row, whose
// pieces of 16 bytes lie next to each other.  In LDS rows lie 16 bytes further apart than they are long, so that the 16 rows that a
// quarter of a wave reads at once start in different banks.
template <int D, bool F32, int ROWS, int THREADS>
struct Rows {
    static constexpr int ROWB = D * (F32 ? 4 : 2), PITCH = ROWB + 16, TPR = THREADS / ROWS, NP = ROWB / 16 / TPR;
    u32x4 piece[NP];
    float l;
    int see;
    __device__ __forceinline__ void fetch(const Args& A, const Item& I, const int head, const int first, const int n_rows)
    {
        int r = first + (int)threadIdx.x / TPR;
        const bool there = r < n_rows;
        r = there ? r : n_rows - 1;
        const int tok = divide(r, A.by_group);
        const int64_t at = (int64_t)(I.q_tok0 + tok) * A.g.Hq + head * A.g.G + (r - tok * A.g.G);
        const u32x4* p = (const u32x4*)(A.q + at * ROWB) + threadIdx.x % TPR * NP;
#pragma unroll
        for (int i = 0; i < NP; ++i) piece[i] = p[i];
        l = there ? A.lse[at] : __builtin_inff();
        see = I.first_vis + I.causal * tok;
    }
    // norm: log2 sum exp2, infinite for a row that is left out: its weights are exp2(0 - inf), whatever its q holds; sees: the keys that
    // it sees, none for a row that is left out (a key that only such rows would see, their own padding, may hold no number)
    __device__ __forceinline__ void store(unsigned char* rows, float* norm, int* sees) const
    {
        const int r = (int)threadIdx.x / TPR;
        const bool out = __builtin_isinf(l);
        u32x4* p = (u32x4*)(rows + r * PITCH) + threadIdx.x % TPR * NP;
#pragma unroll
        for (int i = 0; i < NP; ++i) p[i] = out ? u32x4{0, 0, 0, 0} : piece[i];
        if (threadIdx.x % TPR == 0) { norm[r] = out ? __builtin_inff() : l * kLog2e; sees[r] = out ? 0 : see; }
    }
};

// Adds the weights that the 32 rows of an LDS tile give the keys of a lane: key k0 + 32 t + lane % 32 of each operand t.  `edge`: some of
// the rows may not see all of the wave's keys.
template <int D, bool F32, int KT>
__device__ __forceinline__ void add_weights(const unsigned char* rows, const float* norm, const int* sees, const Operand<D, F32> (&key)[KT], const int k0,
                                            const bool edge, const float c, const int lane, float (&sum)[KT])
{
    constexpr int PITCH = D * (F32 ? 4 : 2) + 16;
    const int half = lane >> 5, col = lane & 31;
    Operand<D, F32> q;
    load_operand<D, F32>(q, rows + col * PITCH, half);
    f32x16 s[KT];
    products<D, F32, KT>(q, key, s);
    // the accumulator's register v: row (v & 3) + 8 (v >> 2) + 4 half
    if (edge) {
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
            const f32x4 n = *(const f32x4*)&norm[8 * v4 + 4 * half];
            const int4 m = *(const int4*)&sees[8 * v4 + 4 * half];
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                const int j = k0 + 32 * t + col;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][4 * v4 + e], c, -n[e]));
                    sum[t] += j < (e == 0 ? m.x : e == 1 ? m.y : e == 2 ? m.z : m.w) ? w : 0.f;
                }
            }
        }
    } else {
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
            const f32x4 n = *(const f32x4*)&norm[8 * v4 + 4 * half];
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[t] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][4 * v4 + e], c, -n[e]));
        }
    }
}

// Waits for the operands here: left to itself the compiler waits inside the loop that uses them, for every load that is in flight by
// then, the next rows' among them.
template <int D, bool F32, int KT>
__device__ __forceinline__ void arrived(Operand<D, F32> (&key)[KT])
{
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int s = 0; s < (F32 ? D / 8 : D / 16); ++s) asm volatile("" : "+v"(key[t].v[s]));
}

// Few rows (at most few_rows() a KV head): they stay in LDS, and the keys stream past.  Workgroup (run of key tiles, KV head) of four waves
// side by side along the keys, 32 each.  A wave asks for 32 keys, waits for them and multiplies; while it does, the other waves' loads are in
// flight, and there are up to six to a SIMD, as small operands and no second set of them leave the registers for that.  (With the next keys
// asked for before the products, twice the registers and half the waves, 32 tokens at 32,768 keys 16.9 -> 18.2 us, 131,072 49.5 -> 52.7.)
constexpr int few_rows(const int d, const int elem) { return d * elem == 512 ? 64 : 128; }        // (of LDS that a launch may ask for)
template <int D, bool F32> constexpr int few_rows_bytes(const int rows) { return rows * (D * (F32 ? 4 : 2) + 16 + 8); }
template <int D, bool F32>
__global__ __launch_bounds__(256, F32 && D == 128 ? 4 : 6) void sk_mass_stream(const Args A)
{
    constexpr int KEYS = 128, ROWB = D * (F32 ? 4 : 2), PITCH = ROWB + 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char rows[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    const int wg = blockIdx.x / A.g.Hkv, head = blockIdx.x - wg * A.g.Hkv;
    const Item I = A.item[item_of(A, wg, lane)];
    const int first = (wg - I.tile0) * A.run * KEYS + wave * 32;
    const int last = first + A.run * KEYS < I.n_keys ? first + A.run * KEYS : I.n_keys;
    const unsigned char* kv = A.g.kv + (int64_t)head * A.g.head_stride;
    const int n_rows = I.n_tok * A.g.G;
    float* norm = (float*)(rows + A.lds_rows * PITCH);
    int* sees = (int*)(norm + A.lds_rows);

    Place at;
    at.find(A, I, first + col);
    for (int r = 0; r < n_rows; r += 64) {
        Rows<D, F32, 64, 256> R;
        R.fetch(A, I, head, r, n_rows);
        R.store(rows + r * PITCH, norm + r, sees + r);
    }
    __syncthreads();
    for (int k0 = first; k0 < last; k0 += KEYS) {
        const int j = k0 + col;
        Operand<D, F32> key[1];
        load_operand<D, F32>(key[0], kv + at.at(A, ROWB), half);
        const float in = I.in ? I.in[head * I.in_stride + (j < I.n_keys ? j : 0)] : 0.f;
        at.find(A, I, j + KEYS);
        arrived<D, F32, 1>(key);
        float sum[1] = {0.f};
        for (int r = 0; r < n_rows; r += 32)
            add_weights<D, F32, 1>(rows + r * PITCH, norm + r, sees + r, key, k0, k0 + 32 > I.first_vis, A.g.scale_log2e, lane, sum);
        sum[0] += __shfl_xor(sum[0], 32, 64);
        if (half == 0 && j < I.n_keys) I.out[head * I.out_stride + j] = I.in ? sum[0] + A.keep * in : sum[0];
    }
}

// Many rows: the keys stay in registers, and the rows pass by.  Workgroup (key tile, part of the rows, KV head) of four waves side by side
// along the keys, KT x 32 each, or twice as many, which share a step's rows.  Rows go through LDS, 64 at a time, loaded one step ahead.  Where the keys make few workgroups the rows are
// cut into parts, whose sums a second launch adds up.
template <int D, bool F32, int KT, int SHARES>
__global__ __launch_bounds__(256 * SHARES, 2) void sk_mass_rows(const Args A)
{
    constexpr int ROWB = D * (F32 ? 4 : 2), PITCH = ROWB + 16, ROWS = 64, KEYS = 128 * KT;
    __shared__ __attribute__((aligned(16))) unsigned char rows[2][ROWS * PITCH];
    __shared__ __attribute__((aligned(16))) float norm[2][ROWS];
    __shared__ __attribute__((aligned(16))) int sees[2][ROWS];
    __shared__ float others[SHARES > 1 ? KEYS : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3;
    const int share = SHARES > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
    const int half = lane >> 5, col = lane & 31;
    const int rest = blockIdx.x / A.g.Hkv, head = blockIdx.x - rest * A.g.Hkv;
    const int wg = rest / A.parts, part = rest - wg * A.parts;
    const Item I = A.item[item_of(A, wg, lane)];
    const int key0 = (wg - I.tile0) * KEYS, k0 = key0 + wave * (KT * 32);
    Operand<D, F32> key[KT];
    Place at[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) at[t].find(A, I, k0 + 32 * t + col);
#pragma unroll
    for (int t = 0; t < KT; ++t) load_operand<D, F32>(key[t], A.g.kv + (int64_t)head * A.g.head_stride + at[t].at(A, ROWB), half);
    float sum[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) sum[t] = 0.f;
    // tokens below `tok0` see none of the workgroup's keys
    int begin = 0, end = I.n_tok * A.g.G;
    if (I.causal && key0 >= I.first_vis) begin = (key0 - I.first_vis + 1) * A.g.G & ~31;
    if (A.parts > 1) {
        const int steps = end > begin ? (end - begin + A.parts * ROWS - 1) / (A.parts * ROWS) : 0;
        begin += part * steps * ROWS;
        end = begin + steps * ROWS < end ? begin + steps * ROWS : end;
    }
    const int n_rows = I.n_tok * A.g.G;
    const bool edge = k0 + 32 * KT > I.first_vis;
    Rows<D, F32, ROWS, 256 * SHARES> R;
    if (begin < end) { R.fetch(A, I, head, begin, n_rows); R.store(rows[0], norm[0], sees[0]); }
    arrived<D, F32, KT>(key);
    __syncthreads();
    // Waves of a SIMD go at different priorities: at equal ones they fall into step, all at the matrix pipe or all at the vector pipe.
    const int slot = __builtin_amdgcn_s_getreg(4 | (3 << 11)) & 3;
    if (slot == 1) __builtin_amdgcn_s_setprio(1);
    else if (slot == 2) __builtin_amdgcn_s_setprio(2);
    else if (slot == 3) __builtin_amdgcn_s_setprio(3);
    int buf = 0;
    for (int r0 = begin; r0 < end; r0 += ROWS, buf ^= 1) {
        const bool more = r0 + ROWS < end;
        if (more) R.fetch(A, I, head, r0 + ROWS, n_rows);
#pragma unroll
        for (int r = 32 * share; r < ROWS; r += 32 * SHARES) {
            // (apart, then to the others: a chain of as many additions as a lane has rows loses more than its terms do: 256 tokens over
            // 32,768 keys are off by 1.7e-7 of the sums' norm, 2.7e-7 in one chain, in the same time)
            float w[KT] = {};
            add_weights<D, F32, KT>(rows[buf] + r * PITCH, norm[buf] + r, sees[buf] + r, key, k0, edge, A.g.scale_log2e, lane, w);
#pragma unroll
            for (int t = 0; t < KT; ++t) sum[t] += w[t];
        }
        if (more) R.store(rows[buf ^ 1], norm[buf ^ 1], sees[buf ^ 1]);
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) sum[t] += __shfl_xor(sum[t], 32, 64);
    if (SHARES > 1) {
        if (share == 1 && half == 0) {
#pragma unroll
            for (int t = 0; t < KT; ++t) others[wave * (KT * 32) + 32 * t + col] = sum[t];
        }
        __syncthreads();
        if (share == 1) return;
#pragma unroll
        for (int t = 0; t < KT; ++t) sum[t] += others[wave * (KT * 32) + 32 * t + col];
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        const int j = k0 + 32 * t + col;
        if (half != 0 || j >= I.n_keys) continue;
        if (A.parts > 1) { A.part_sums[(int64_t)blockIdx.x * KEYS + (j - key0)] = sum[t]; continue; }
        if (I.in) sum[t] += A.keep * I.in[head * I.in_stride + j];
        I.out[head * I.out_stride + j] = sum[t];
    }
}

// Adds up the parts: workgroup (key tile, KV head), a thread a key.
__global__ __launch_bounds__(256) void sk_mass_join(const Args A, const int tile_keys)
{
    const int wg = blockIdx.x / A.g.Hkv, head = blockIdx.x - wg * A.g.Hkv;
    const Item I = A.item[item_of(A, wg, threadIdx.x & 63)];
    for (int k = threadIdx.x; k < tile_keys; k += 256) {
        const int j = (wg - I.tile0) * tile_keys + k;
        if (j >= I.n_keys) break;
        const float in = I.in ? I.in[head * I.in_stride + j] : 0.f;
        const float* p = A.part_sums + ((int64_t)wg * A.parts * A.g.Hkv + head) * tile_keys + k;
        float sum = 0.f;
#pragma unroll 4
        for (int i = 0; i < A.parts; ++i) sum += p[(int64_t)i * A.g.Hkv * tile_keys];
        I.out[head * I.out_stride + j] = I.in ? sum + A.keep * in : sum;
    }
}

template <int D, bool F32>
int launch(const Args& A, const int kt, const int tiles, hipStream_t st)
{
    const dim3 grid((unsigned)tiles * (unsigned)A.parts * (unsigned)A.g.Hkv), block(256);
    if (kt == 0) hipLaunchKernelGGL((sk_mass_stream<D, F32>), grid, block, (few_rows_bytes<D, F32>(A.lds_rows)), st, A);
    else if constexpr (F32) hipLaunchKernelGGL((sk_mass_rows<D, F32, 1, 1>), grid, block, 0, st, A);
    else if (kt == 4) hipLaunchKernelGGL((sk_mass_rows<D, F32, 4, 1>), grid, block, 0, st, A);
    // At most a workgroup to a CU: eight waves, two to a SIMD, one at the matrix pipe while the other is at the vector unit.  us, four / eight:
    // 256 tokens at 2,600 keys 24.1 / 19.9, 64 there 9.0 / 8.5; 20 tokens of 33 heads at 9,000 keys of one 14.0 / 11.6.  With more, waves of other workgroups
    // do that: 64 at 9,001 12.7 / 17.0, 512 at 2,600 in parts 22.8 / 28.4.  (fp32: no difference.)
    else if (A.parts == 1 && tiles * A.g.Hkv <= 256) hipLaunchKernelGGL((sk_mass_rows<D, F32, 1, 2>), grid, dim3(512), 0, st, A);
    else hipLaunchKernelGGL((sk_mass_rows<D, F32, 1, 1>), grid, block, 0, st, A);
    if (A.parts > 1) hipLaunchKernelGGL(sk_mass_join, dim3((unsigned)tiles * (unsigned)A.g.Hkv), block, 0, st, A, 128 * kt);
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

// How the rows kernel cuts a call: keys of a wave / 32, and parts of the rows.  `keys` are the items' added up, `rows` those of the longest.
// Waves of 128 keys read an LDS row once for twice as many products as waves of 64, and make two workgroups to a CU: taken where they
// fill the device (512), by the keys alone or, for rows long enough that a part still has eight steps of 64, by parts of them.  Otherwise
// waves of 32 keys, four workgroups to a CU, in parts of at least four steps.  us (rows of a KV head; keys x KV heads), 32 keys a wave / 128:
// 1,024; 262,144 104 / 75; 512; 262,144 48 / 40; 512; 118,400 24 / 31; 539; 36,004 17.4 / 31.5; in the best parts of each 8,192; 32,768 68 / 69,
// 8,192; 131,072 321 / 255, 2,048; 20,800 22 / 24, whole 45.6 / 101.  fp32: operands of twice the size and products of eight times the time, so 32
// keys a wave, and parts of two steps; 256; 16,384 23.7 whole, 17.9 in two.
void cut_rows(const sk_geom& g, const int64_t keys, const int64_t rows, int& kt, int& parts)
{
    const int64_t steps = (rows + 63) / 64, w4 = std::max<int64_t>(1, keys * g.Hkv / 512), w1 = std::max<int64_t>(1, keys * g.Hkv / 128);
    int64_t p = 1;
    kt = 4;
    if (g.elem == 4) { kt = 1; p = std::min<int64_t>(512 / w1, steps / 2); }
    else if (w4 < 448) {
        p = 512 / w4;
        if (steps < 8 * p) { kt = 1; p = std::min<int64_t>(1024 / w1, steps / 4); }
        if (rows <= 1024) { kt = 1; p = 1; }
    }
    parts = (int)std::max<int64_t>(1, std::min<int64_t>(p, 16));
}

// The items with few rows, or those with many, in as many launches as their descriptions need.
int launch_items(sk_pool* p, const Call& C, const bool few, hipStream_t st)
{
    sk_session_view V;
    int64_t keys = 0, rows = 0;
    auto belongs = [&](const int32_t i) {
        sk_view_session(p, C.session_id[i], &V);
        return V.retained > 0 && ((int64_t)(C.cu_tokens[i + 1] - C.cu_tokens[i]) * V.g.G <= few_rows(V.g.d, V.g.elem)) == few;
    };
    for (int32_t i = 0; i < C.n_items; ++i)
        if (belongs(i)) { keys += V.retained; rows = std::max<int64_t>(rows, (int64_t)(C.cu_tokens[i + 1] - C.cu_tokens[i]) * V.g.G); }
    if (keys == 0) return SK_OK;
    Args A;
    A.g = V.g; A.q = (const unsigned char*)C.q; A.lse = C.lse; A.keep = C.keep; A.by_group = sk_make_div((uint32_t)V.g.G);
    A.run = 1; A.part_sums = (float*)V.scratch;
    A.lds_rows = few ? (int)(rows + 63) / 64 * 64 : 0;
    int kt = 0, parts = 1, tile_keys = 128;
    if (few) {
        // Workgroups of several key tiles start, and load their rows, less often; as long as there are six to a CU.  us for runs of 1, 2, 4, 8:
        // 32 tokens at 32,768 keys 21.0, 17.2, 21.4, 30.0; one at 131,072 43.6, 41.3, 42.7, 46.2; 32 there, where a tile's products take longer than its
        // keys to arrive, 76.7, 62.2, 54.7, 50.8; 48 sessions of 2K-64K keys 405, 367, 375, 388; 16 tokens at 9,001 7.6, 8.1, 10.7, 18.5.
        const int64_t tiles = keys / tile_keys * V.g.Hkv;
        A.run = tiles < 1536 ? 1 : rows <= 64 || tiles < 4096 ? 2 : 8;
        tile_keys *= A.run;
    } else {
        cut_rows(V.g, keys, rows, kt, parts);
        tile_keys = 128 * kt;
    }
    for (int32_t i = 0; i < C.n_items;) {
        A.n_items = 0;
        int64_t tiles = 0;
        for (; i < C.n_items && A.n_items < kItems; ++i) {
            if (!belongs(i)) continue;
            const int64_t t = (V.retained + tile_keys - 1) / tile_keys;
            if (A.n_items > 0 && (tiles + t) * parts * V.g.Hkv >= (int64_t(1) << 31)) break;      // a launch's workgroups are counted in 31 bits
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
        if (A.n_items == 0) break;
        // (sums of parts that the workspace does not hold: many short sessions)
        A.parts = (int)std::max<int64_t>(1, std::min<int64_t>(parts, (int64_t)(V.scratch_bytes / 4) / (tiles * V.g.Hkv * tile_keys)));
        int e;
        if (A.g.elem == 4) e = A.g.d == 128 ? launch<128, true>(A, kt, (int)tiles, st) : launch<64, true>(A, kt, (int)tiles, st);
        else e = A.g.d == 128 ? launch<128, false>(A, kt, (int)tiles, st) : launch<64, false>(A, kt, (int)tiles, st);
        if (e) return sk_note_hip_error(e);
        sk_count_launch(p);
        if (A.parts > 1) sk_count_launch(p);
    }
    return SK_OK;
}

int run(sk_pool* p, const Call& C, void* stream)
{
    int rc = check(p, C);
    if (rc == SK_OK) rc = launch_items(p, C, true, (hipStream_t)stream);
    if (rc == SK_OK) rc = launch_items(p, C, false, (hipStream_t)stream);
    return rc;
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
