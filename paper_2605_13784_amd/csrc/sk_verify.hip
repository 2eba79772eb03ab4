// Verification of drafted tokens for gfx950 (include/sk.h: sk_verify).
//
// With p the target's and q the draft's softmax of logit / T at a place, a drafted token x stays while u q(x) < p(x); the first that does
// not is replaced by the token that u' finds in the running sum of max(p - q, 0), and behind k that stay one is drawn from p.  What
// leaves has the target's distribution whatever the draft's is.
//
// A comparison next to a border turns on the last bits of a sum over a whole vocabulary, so that sums and exponentials are formed in 64
// bits: the vector unit adds and multiplies those at the rate of 32-bit ones, and a row's bytes take longer to arrive.
//
// Three launches: maxima and sums of all rows, in parts; the sums of the stretches of the one row per sequence that is drawn from; the draw.
// Bound: the logits, read once (and the drawn row again, once, and one stretch of it).
#include <hip/hip_runtime.h>
#include <cstring>

#include "../../include/sk.h"
#include "sk_internal.h"
#include "sk_order.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPieces = 8;                         // 16-byte pieces of a thread in the first launch
constexpr int kStretch = 4096;                     // logits of a workgroup in the second
constexpr int kMaxRows = 2 * SK_VERIFY_MAX_DRAFT + 1;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct Part { double sum; float max; int32_t at; };       // of a part of a row: sum of 2^((x - max) scale), lowest index of max (greedy)

struct Args {
    const unsigned char *target, *draft;
    int64_t target_stride, draft_stride;           // bytes
    int32_t n_draft, vocab, parts, stretches;
    const int32_t* tokens;
    const float* uniform;
    const float* temperature;
    Part* part;                                    // [sequence][target rows, then draft rows][part]
    double* sums;                                  // [sequence][stretch]
    int32_t *n_accepted, *out_tokens;
    float* logprob;
};

// 2^d for d <= 0: the integer part goes to the exponent, the rest through the series of exp, whose next term is below 2^-47
__device__ __forceinline__ double power_of_two(double d)
{
    d = __builtin_fmax(d, -1100.0);                // (-inf, and NaN of -inf * 0: nothing)
    const double n = __builtin_rint(d), f = (d - n) * 0.6931471805599453;
    double r = 1.0 / 39916800;
    r = __builtin_fma(r, f, 1.0 / 3628800); r = __builtin_fma(r, f, 1.0 / 362880); r = __builtin_fma(r, f, 1.0 / 40320);
    r = __builtin_fma(r, f, 1.0 / 5040); r = __builtin_fma(r, f, 1.0 / 720); r = __builtin_fma(r, f, 1.0 / 120);
    r = __builtin_fma(r, f, 1.0 / 24); r = __builtin_fma(r, f, 1.0 / 6); r = __builtin_fma(r, f, 0.5);
    r = __builtin_fma(r, f, 1.0); r = __builtin_fma(r, f, 1.0);
    return __builtin_ldexp(r, (int)n);
}

template <bool F32> __device__ __forceinline__ float logit(const unsigned char* row, const int i)
{
    if (F32) return ((const float*)row)[i];
    return __uint_as_float((uint32_t)((const uint16_t*)row)[i] << 16);
}

__device__ __forceinline__ double shuffled(const double x, const int mask)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __shfl_xor((int)(uint32_t)b, mask, 64), hi = __shfl_xor((int)(uint32_t)(b >> 32), mask, 64);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += shuffled(x, m);
    return x;
}
__device__ __forceinline__ float wave_max(const float x) { return sk_order::value_of(__builtin_amdgcn_readfirstlane(sk_order::wave_max(sk_order::rank_of(x)))); }

// The exponent's factor of a sequence: log2(e) / T; greedy sequences, whose log probabilities are those of the logits as they are, have T = 1.
__device__ __forceinline__ double scale_of(const Args& A, const int seq, bool& greedy)
{
    const float t = A.temperature ? A.temperature[seq] : 1.f;
    greedy = !(t > 0.f);
    return 1.4426950408889634 / (greedy ? 1.0 : (double)t);
}

// Tokens that a sequence has drafted: those in front of the first outside the vocabulary.
__device__ __forceinline__ int drafted(const Args& A, const int seq)
{
    const int lane = threadIdx.x & 63;
    const bool ends = lane >= A.n_draft || (uint32_t)A.tokens[(int64_t)seq * A.n_draft + lane] >= (uint32_t)A.vocab;
    return __builtin_ctzll(__ballot(ends));        // (fewer than a wave's lanes)
}

__device__ __forceinline__ const unsigned char* row_of(const Args& A, const int seq, const int r)
{
    if (r <= A.n_draft) return A.target + ((int64_t)seq * (A.n_draft + 1) + r) * A.target_stride;
    return A.draft + ((int64_t)seq * A.n_draft + r - A.n_draft - 1) * A.draft_stride;
}

// ---- first launch: maximum and sum of a part of a row ----

template <bool F32>
__global__ __launch_bounds__(kThreads) void sk_verify_rows(const Args A, const int rows)
{
    constexpr int EL = F32 ? 4 : 2, N = 16 / EL;
    __shared__ Part of_wave[kWaves];
    const int part = blockIdx.x % A.parts, row = blockIdx.x / A.parts, seq = row / rows, r = row - seq * rows;
    const int n = drafted(A, seq), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    bool greedy;
    const double scale = scale_of(A, seq, greedy);
    if (r <= A.n_draft ? r > n : greedy || r - A.n_draft - 1 >= n) return;
    const unsigned char* x = row_of(A, seq, r);
    // pieces of 16 bytes as they lie in memory; the first and last may reach beyond the row
    const int lead = (int)((uintptr_t)x & 15) / EL;
    float v[kPieces * N];
    const float none = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int at = ((part * kPieces + i) * kThreads + (int)threadIdx.x) * N - lead;
        if (at >= 0 && at + N <= A.vocab) {
            const u32x4 w = *(const u32x4*)(x + (int64_t)at * EL);
#pragma unroll
            for (int e = 0; e < N; ++e)
                v[i * N + e] = F32 ? __uint_as_float(w[e % 4]) : __uint_as_float(e & 1 ? w[e / 2 % 4] & 0xffff0000u : w[e / 2 % 4] << 16);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[i * N + e] = at + e >= 0 && at + e < A.vocab ? logit<F32>(x, at + e) : none;
        }
    }
    float m = none;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPieces * N; ++i) { m = fmaxf(m, v[i]); bad |= !(v[i] < __builtin_inff()); }
    m = wave_max(m);
    const float m0 = m == none ? 0.f : m;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kPieces * N; ++i) sum += power_of_two(((double)v[i] - (double)m0) * scale);
    sum = wave_sum(sum);
    int at = INT32_MAX;
    if (greedy) {
#pragma unroll
        for (int i = kPieces * N - 1; i >= 0; --i)
            if (v[i] == m) at = ((part * kPieces + i / N) * kThreads + (int)threadIdx.x) * N - lead + i % N;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) at = min(at, __shfl_xor(at, s, 64));
    }
    if (__ballot(bad)) sum = __builtin_nan("");
    if (lane == 0) of_wave[wave] = Part{sum, m, at};
    __syncthreads();
    if (threadIdx.x == 0) {
        Part p = of_wave[0];
        for (int w = 1; w < kWaves; ++w) {
            const Part o = of_wave[w];
            const float top = fmaxf(p.max, o.max), t0 = top == none ? 0.f : top;
            const int32_t first = p.max > o.max ? p.at : p.max < o.max ? o.at : min(p.at, o.at);
            p = Part{p.sum * power_of_two(((double)p.max - t0) * scale) + o.sum * power_of_two(((double)o.max - t0) * scale), top, first};
        }
        A.part[((int64_t)seq * rows + r) * A.parts + part] = p;
    }
}

// ---- which tokens stay ----

struct Row { double total; float max; int32_t at; };      // of a whole row: sum of 2^((x - max) scale); 0: no probabilities
struct Decision {
    Row row[kMaxRows];
    int n;                    // drafted
    int accepted;
    bool greedy, valid;       // valid: the row that is drawn from has probabilities
    bool less;                // the draft's probabilities are taken off
    double scale;
};

template <bool F32>
__device__ __forceinline__ void decide(const Args& A, const int rows, const int seq, Decision& D)
{
    const int n = drafted(A, seq), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    bool greedy;
    const double scale = scale_of(A, seq, greedy);
    const float none = -__builtin_inff();
    const int n_rows = n + 1 + (A.draft && !greedy ? n : 0);
    for (int i = wave; i < n_rows; i += kWaves) {
        const int r = i <= n ? i : A.n_draft + 1 + (i - n - 1);
        const Part* p = A.part + ((int64_t)seq * rows + r) * A.parts;
        float m = none;
        for (int c = lane; c < A.parts; c += 64) m = fmaxf(m, p[c].max);
        m = wave_max(m);
        const float m0 = m == none ? 0.f : m;
        double sum = 0.0;
        int at = INT32_MAX;
        for (int c = lane; c < A.parts; c += 64) {
            const Part o = p[c];
            sum += o.sum * power_of_two(((double)o.max - m0) * scale);
            if (o.max == m) at = min(at, o.at);
        }
        sum = wave_sum(sum);
#pragma unroll
        for (int s = 1; s < 64; s *= 2) at = min(at, __shfl_xor(at, s, 64));
        if (lane == 0) D.row[r] = Row{sum > 0.0 ? sum : 0.0, m, at};      // (NaN: none)
    }
    __syncthreads();
    if (wave == 0) {
        bool stays = false;
        if (lane < n) {
            const int32_t t = A.tokens[(int64_t)seq * A.n_draft + lane];
            const Row p = D.row[lane];
            if (p.total == 0.0) stays = false;
            else if (greedy) stays = t == p.at;
            else {
                const double px = power_of_two(((double)logit<F32>(row_of(A, seq, lane), t) - (double)p.max) * scale) / p.total;
                double qx = 1.0;
                bool none_drafted = false;
                if (A.draft) {
                    const Row q = D.row[A.n_draft + 1 + lane];
                    none_drafted = q.total == 0.0;
                    qx = none_drafted ? 1.0 : power_of_two(((double)logit<F32>(row_of(A, seq, A.n_draft + 1 + lane), t) - (double)q.max) * scale) / q.total;
                }
                stays = !none_drafted && (double)A.uniform[(int64_t)seq * (A.n_draft + 1) + lane] * qx < px;
            }
        }
        const uint64_t out = ~__ballot(stays);
        if (lane == 0) {
            const int a = min(n, out ? __builtin_ctzll(out) : 64);
            D.n = n; D.accepted = a; D.greedy = greedy; D.scale = scale;
            D.valid = D.row[a].total > 0.0;
            D.less = a < n && (!A.draft || (!greedy && D.row[A.n_draft + 1 + a].total > 0.0));
        }
    }
    __syncthreads();
}

// What a logit of the row that is drawn from counts for.
template <bool F32> struct Weights {
    const unsigned char *p, *q;
    double scale, p_max, p_inv, q_max, q_inv;
    int32_t without;          // a draft without probabilities: its token
    __device__ __forceinline__ Weights(const Args& A, const Decision& D, const int seq)
    {
        const int a = D.accepted;
        p = row_of(A, seq, a);
        scale = D.scale; p_max = D.row[a].max; p_inv = 1.0 / D.row[a].total;
        q = nullptr; q_max = q_inv = 0.0; without = -1;
        if (D.less && A.draft) { const Row& r = D.row[A.n_draft + 1 + a]; q = row_of(A, seq, A.n_draft + 1 + a); q_max = r.max; q_inv = 1.0 / r.total; }
        else if (D.less) without = A.tokens[(int64_t)seq * A.n_draft + a];
    }
    __device__ __forceinline__ double operator()(const int i) const
    {
        double w = power_of_two(((double)logit<F32>(p, i) - p_max) * scale) * p_inv;
        if (q) w = __builtin_fmax(w - power_of_two(((double)logit<F32>(q, i) - q_max) * scale) * q_inv, 0.0);
        return i == without ? 0.0 : w;
    }
};

// ---- second launch: the sum of a stretch of the drawn row ----

template <bool F32>
__global__ __launch_bounds__(kThreads) void sk_verify_stretches(const Args A, const int rows)
{
    __shared__ Decision D;
    __shared__ double of_wave[kWaves];
    const int stretch = blockIdx.x % A.stretches, seq = blockIdx.x / A.stretches;
    decide<F32>(A, rows, seq, D);
    if (D.greedy || !D.valid) return;
    const Weights<F32> w(A, D, seq);
    double sum = 0.0;
#pragma unroll 4
    for (int i = 0; i < kStretch / kThreads; ++i) {
        const int t = stretch * kStretch + i * kThreads + threadIdx.x;
        if (t < A.vocab) sum += w(t);
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) A.sums[(int64_t)seq * A.stretches + stretch] = of_wave[0] + of_wave[1] + of_wave[2] + of_wave[3];
}

// ---- third launch: the draw, and what a sequence's outputs are ----

// The token that the sequence's last number finds in the running sum of the row's weights, for the whole workgroup.
template <bool F32>
__device__ __forceinline__ int draw(const Args& A, const Decision& D, const int seq)
{
    constexpr int EACH = kStretch / kThreads;
    __shared__ double of_thread[kThreads];
    __shared__ int chosen;
    __shared__ double left;
    const int tid = threadIdx.x;
    const Weights<F32> w(A, D, seq);
    const double* sums = A.sums + (int64_t)seq * A.stretches;
    if (tid == 0) {
        double total = 0.0, before = 0.0, at_last = 0.0;
        for (int c = 0; c < A.stretches; ++c) total += sums[c];
        const double limit = __builtin_fmax((double)A.uniform[(int64_t)seq * (A.n_draft + 1) + A.n_draft], 0.0) * total;
        int c = 0, last = 0;
        for (; c < A.stretches; ++c) {
            if (sums[c] > 0.0) { last = c; at_last = before; }
            if (before + sums[c] > limit) break;
            before += sums[c];
        }
        if (c == A.stretches) { c = last; before = at_last; }
        chosen = total > 0.0 ? c : -1; left = limit - before;
    }
    __syncthreads();
    // nothing is left of the target: p and q are one, and the drafted token is as good
    if (chosen < 0) return A.tokens[(int64_t)seq * A.n_draft + D.accepted];
    const int begin = chosen * kStretch + tid * EACH;
    double mine = 0.0;
    for (int i = 0; i < EACH; ++i)
        if (begin + i < A.vocab) mine += w(begin + i);
    of_thread[tid] = mine;
    __syncthreads();
    if (tid == 0) {
        double before = 0.0, at_last = 0.0;
        int t = 0, last = 0;
        for (; t < kThreads; ++t) {
            if (of_thread[t] > 0.0) { last = t; at_last = before; }
            if (before + of_thread[t] > left) break;
            before += of_thread[t];
        }
        if (t == kThreads) { t = last; before = at_last; }
        const int from = chosen * kStretch + t * EACH;
        int found = from;
        for (int i = 0; i < EACH && from + i < A.vocab; ++i) {
            const double x = w(from + i);
            if (x > 0.0) found = from + i;         // (the last that counts, where roundings leave the sum below the limit)
            before += x;
            if (before > left && x > 0.0) break;
        }
        chosen = found;
    }
    __syncthreads();
    return chosen;
}

template <bool F32>
__global__ __launch_bounds__(kThreads) void sk_verify_draw(const Args A, const int rows)
{
    __shared__ Decision D;
    const int seq = blockIdx.x, tid = threadIdx.x;
    decide<F32>(A, rows, seq, D);
    const int a = D.accepted;
    int token = -1;
    if (D.valid) token = D.greedy ? D.row[a].at : draw<F32>(A, D, seq);
    if (tid == 0) A.n_accepted[seq] = a;
    if (tid <= A.n_draft) {
        const int32_t t = tid < a ? A.tokens[(int64_t)seq * A.n_draft + tid] : tid == a ? token : -1;
        A.out_tokens[(int64_t)seq * (A.n_draft + 1) + tid] = t;
        if (A.logprob) {
            float l = 0.f;
            if (tid <= a) {
                const Row r = D.row[tid];
                l = t < 0 ? __builtin_nanf("") : (float)(((double)logit<F32>(row_of(A, seq, tid), t) - (double)r.max) * (D.scale * 0.6931471805599453) - log(r.total));
            }
            A.logprob[(int64_t)seq * (A.n_draft + 1) + tid] = l;
        }
    }
}

int64_t parts_of(const int dtype_bytes, const int32_t vocab)
{
    const int n = 16 / dtype_bytes;
    return ((int64_t)vocab + n - 1 + kPieces * kThreads * n - 1) / (kPieces * kThreads * n);
}
bool sizes_ok(const int32_t n_seq, const int32_t n_draft, const int32_t vocab)
{
    return n_seq > 0 && n_draft >= 0 && n_draft <= SK_VERIFY_MAX_DRAFT && vocab >= 1 && vocab <= SK_VERIFY_MAX_VOCAB &&
           (int64_t)n_seq * (n_draft + 1) <= SK_VERIFY_MAX_ROWS;
}

}  // namespace

extern "C" {

size_t sk_verify_workspace_bytes(int32_t n_seq, int32_t n_draft, int32_t vocab)
{
    if (!sizes_ok(n_seq, n_draft, vocab)) return 0;
    // (for either type of the logits: fp32 ones have more parts)
    const int64_t stretches = ((int64_t)vocab + kStretch - 1) / kStretch;
    return size_t(n_seq) * (size_t(2 * n_draft + 1) * size_t(parts_of(4, vocab)) * sizeof(Part) + size_t(stretches) * 8);
}

int sk_verify(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int dtype, int32_t n_seq, int32_t n_draft, int32_t vocab,
              const int32_t* tokens, const float* uniform, const float* temperature, void* workspace, size_t workspace_bytes,
              int32_t* n_accepted, int32_t* out_tokens, float* logprob, void* hip_stream)
{
    if (dtype != SK_F32 && dtype != SK_BF16) return SK_E_DTYPE;
    if (n_seq < 0) return SK_E_INVAL;
    if (n_seq == 0) return SK_OK;
    if (!sizes_ok(n_seq, n_draft, vocab) || target_stride < vocab || (draft && draft_stride < vocab)) return SK_E_INVAL;
    if (target_stride > (int64_t(1) << 40) || (draft && draft_stride > (int64_t(1) << 40))) return SK_E_INVAL;
    if (!target || !uniform || !n_accepted || !out_tokens || (n_draft > 0 && !tokens)) return SK_E_INVAL;
    const int el = dtype == SK_F32 ? 4 : 2;
    auto off = [](const void* p, const uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; };
    if (off(target, el) || off(draft, el) || off(tokens, 4) || off(uniform, 4) || off(temperature, 4) || off(n_accepted, 4) || off(out_tokens, 4) || off(logprob, 4)) return SK_E_INVAL;
    if (!workspace || off(workspace, 16)) return SK_E_INVAL;
    if (workspace_bytes < sk_verify_workspace_bytes(n_seq, n_draft, vocab)) return SK_E_WORKSPACE;
    Args A;
    A.target = (const unsigned char*)target; A.draft = n_draft > 0 ? (const unsigned char*)draft : nullptr;
    A.target_stride = target_stride * el; A.draft_stride = draft_stride * el;
    A.n_draft = n_draft; A.vocab = vocab;
    A.parts = (int32_t)parts_of(el, vocab); A.stretches = (vocab + kStretch - 1) / kStretch;
    A.tokens = tokens; A.uniform = uniform; A.temperature = temperature;
    const int rows = n_draft + 1 + (A.draft ? n_draft : 0);
    A.part = (Part*)workspace;
    A.sums = (double*)(A.part + (int64_t)n_seq * rows * A.parts);
    A.n_accepted = n_accepted; A.out_tokens = out_tokens; A.logprob = logprob;
    if ((int64_t)n_seq * rows * A.parts >= (int64_t(1) << 31) || (int64_t)n_seq * A.stretches >= (int64_t(1) << 31)) return SK_E_INVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    const dim3 block(kThreads), first((unsigned)(n_seq * rows) * (unsigned)A.parts), second((unsigned)n_seq * (unsigned)A.stretches);
    if (dtype == SK_F32) {
        hipLaunchKernelGGL(sk_verify_rows<true>, first, block, 0, st, A, rows);
        hipLaunchKernelGGL(sk_verify_stretches<true>, second, block, 0, st, A, rows);
        hipLaunchKernelGGL(sk_verify_draw<true>, dim3(n_seq), block, 0, st, A, rows);
    } else {
        hipLaunchKernelGGL(sk_verify_rows<false>, first, block, 0, st, A, rows);
        hipLaunchKernelGGL(sk_verify_stretches<false>, second, block, 0, st, A, rows);
        hipLaunchKernelGGL(sk_verify_draw<false>, dim3(n_seq), block, 0, st, A, rows);
    }
    return sk_status_of((int)hipGetLastError());
}

}  // extern "C"
