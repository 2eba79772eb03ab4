// Verification of drafted tokens for gfx950 (include/sk.h: sk_verify).
//
// With p the target's and q the draft's softmax of logit / T at a place, a drafted token x stays while u q(x) < p(x); the first that does
// not is replaced by the token that u' finds in the running sum of max(p - q, 0), and behind k that stay one is drawn from p.  What
// leaves has the target's distribution whatever the draft's is.
//
// A comparison next to a border turns on the last bits of a sum over a whole vocabulary, so that sums and exponentials are formed in 64
// bits, which the vector unit adds and multiplies at the rate of 32-bit ones.  Exponentials of 32 bits are off by up to 2^-23 of themselves, and the border between any two
// of 128,256 tokens would move by as much of the total; a number that falls between the old place and the new finds another token.
//
// Maxima and sums of all rows, in parts; the sums of the stretches of the one row per sequence that is drawn from; the draw.  Where there are few rows, that is two
// launches, the draw being the business of the workgroup that is its sequence's last to have a sum; where there are many, three, of which the first is two with a small
// one between them, and the second has a small one in front.
#include <hip/hip_runtime.h>
#include <cstring>

#include "../../include/sk.h"
#include "sk_internal.h"
#include "sk_order.h"

// Which products join an addition is written out: the launches have to agree on every weight.
#pragma clang fp contract(off)

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kEach = 32, kEachFew = 8;            // logits of a lane; where there are few rows.  A stretch is a wave's, a part a workgroup's
constexpr int kApart = 64;                         // words from a sequence's count of workgroups to the next: additions to one line wait for each other
constexpr int kFirstPlaces = 2;                    // places whose rows come first, where there are many rows
constexpr int64_t kPartsInTwo = 8192;              // parts of rows from which they do
constexpr int64_t kAtATime = 2048;                 // workgroups that the chip runs at a time, eight to each of 256 units
constexpr int kMaxRows = 2 * SK_VERIFY_MAX_DRAFT + 1;
constexpr int64_t kMaxWgs = (int64_t(1) << 32) / kThreads - 1;      // of a launch, which has fewer than 2^32 threads

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef u32x4 __attribute__((aligned(2))) u32x4_anywhere;      // (the hardware loads 16 bytes from any address)

// Of a part of a row, or of all of it: sum of 2^(x scale - e) with a whole number e next to the maximum's, so that parts meet without a rounding;
// the lowest index of the maximum (greedy sequences).
struct Part { double sum, e; float max; int32_t at; };
struct Sum { double sum, e; };                     // of a stretch

// What a sequence draws from.
struct Chosen {
    double scale, p_e, p_inv, q_e, q_inv;
    float p_max, q_max;
    int32_t place;            // the row that is drawn from; -1: the token is known
    int32_t less;             // 0: p; 1: p - q; 2: p without the drafted token
};

struct Args {
    const unsigned char *target, *draft;
    int64_t target_stride, draft_stride;           // bytes
    int32_t n_draft, vocab, parts, stretches, rows;
    const int32_t* tokens;
    const float* uniform;
    const float* temperature;
    Part* part;                                    // [sequence][target rows, then draft rows][part]
    Sum* of_stretch;                               // [sequence][target rows][stretch]
    float* given;                                  // [sequence][rows]: the logit of the row's drafted token
    int32_t* ended;                                // [sequence]: nothing behind place0 counts (where rows come in two launches)
    int32_t place0, places, drafts;                // of a launch of rows: its first place, target rows and draft rows of a sequence
    Chosen* chosen;                                // [sequence], for a launch of draws
    uint32_t* arrived;                             // [sequence][kApart]: workgroups that have their sums, where the last one draws (few rows)
    double* sums;                                  // [sequence][stretch]: of the weights of the drawn row
    int32_t *n_accepted, *out_tokens;
    float* logprob;
};

// 2^f for |f| <= 1/2: the polynomial through the values at Chebyshev's ten points, moved by 2^-46 to be 1 at 0; within 2^-44 of itself.
__device__ __forceinline__ double power_of_fraction(const double f)
{
    double r = 1.0205905320493103e-07;
    r = __builtin_fma(r, f, 1.3259645243929057e-06); r = __builtin_fma(r, f, 1.5252672925346873e-05); r = __builtin_fma(r, f, 1.5403433751254997e-04);
    r = __builtin_fma(r, f, 1.3333558200793719e-03); r = __builtin_fma(r, f, 9.618129193934304e-03); r = __builtin_fma(r, f, 5.550410866465168e-02);
    r = __builtin_fma(r, f, 0.2402265069564034); r = __builtin_fma(r, f, 0.6931471805599462);
    return __builtin_fma(r, f, 1.0);
}
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// From 2^50 on, x scale is a whole number and two different logits lie further apart than 2^1000: only the maximum counts.
constexpr double kFar = 1125899906842624.0;

// 2^(x scale - e), where e is no less than a whole number next to the row's largest x scale, and below 2^50 in magnitude
__device__ __forceinline__ double near_weight(const float x, const double scale, const double e)
{
    const double d = __builtin_fmax(__builtin_fma((double)x, scale, -e), -1100.0);      // (-inf, and NaN of -inf * 0: nothing)
    const double n = __builtin_rint(d);
    return __builtin_ldexp(power_of_fraction(d - n), (int)n);
}
__device__ __forceinline__ double weight_of(const float x, const double scale, const double e, const float max)
{
    return __builtin_fabs(e) < kFar ? near_weight(x, scale, e) : x == max ? 1.0 : 0.0;
}
// The same for many, where |e| is below 2^50 and no x scale further from e than 2^10: the distance is rounded into the low bits of a sum, from where its integer part is
// added to the exponent's.  `base` is that sum's other part.
constexpr double kRounds = 6755399441055744.0;     // 1.5 * 2^52
constexpr double kLeast = -1000.0;
__device__ __forceinline__ double weight_within(const float x, const double scale, const double base)
{
    const double t = __builtin_fma((double)x, scale, base);
    u32x2 r = __builtin_bit_cast(u32x2, power_of_fraction(__builtin_fma((double)x, scale, base - t)));
    r.y += __builtin_bit_cast(u32x2, t).x << 20;
    return __builtin_bit_cast(double, r);
}
// The same wherever x is, what lies further below e counting 2^-1000
__device__ __forceinline__ double weight_or_least(const float x, const double scale, const double e)
{
    const double d = __builtin_fmax(__builtin_fma((double)x, scale, -e), kLeast), t = d + kRounds;
    u32x2 r = __builtin_bit_cast(u32x2, power_of_fraction(d - (t - kRounds)));
    r.y += __builtin_bit_cast(u32x2, t).x << 20;
    return __builtin_bit_cast(double, r);
}
constexpr double kNothing = 0x1p-980;              // what the least makes of a row's weights, and more, is taken off the drawn ones: nothing is left of it, and others do not feel it
// The logarithm of a token's probability
__device__ __forceinline__ float log_probability(const float x, const double scale, const double e, const float max, const double inverse)
{
    const double d = __builtin_fabs(e) < kFar ? __builtin_fma((double)x, scale, -e) : ((double)x - (double)max) * scale;
    return (float)(d * 0.6931471805599453 + log(inverse));
}
// A sum from exponent `from` to the larger one `to`
__device__ __forceinline__ double at_exponent(const double sum, const double from, const double to)
{
    return __builtin_ldexp(sum, (int)__builtin_fmax(from - to, -2200.0));
}
// The exponent of a maximum; of none, lower than any other
constexpr double kNoExponent = -1.0e300;
__device__ __forceinline__ double exponent_of(const float max, const double scale)
{
    const double e = __builtin_rint((double)max * scale);
    return max == -__builtin_inff() ? kNoExponent : e;
}

// Maximum and minimum of three (the library's take an instruction more for each operand, for the sake of signalling NaNs: a row that has one has no probabilities, whatever these say)
__device__ __forceinline__ float max_of(const float a, const float b, const float c) { float r; asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c)); return r; }
__device__ __forceinline__ float min_of(const float a, const float b, const float c) { float r; asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c)); return r; }

template <bool F32> __device__ __forceinline__ float logit(const unsigned char* row, const int i)
{
    if (F32) return ((const float*)row)[i];
    return __uint_as_float((uint32_t)((const uint16_t*)row)[i] << 16);
}

// Logit e of a piece of 16 bytes
template <bool F32> __device__ __forceinline__ float element(const u32x4 w, const int e)
{
    if (F32) return __uint_as_float(w[e & 3]);
    return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
}

// Sums and maxima over a row of 16 lanes and over a wave, in every lane, by lane exchanges within the vector unit.
template <int CTRL> __device__ __forceinline__ double dpp(const double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)sk_order::dpp<CTRL>((uint32_t)(b >> 32)) << 32 | sk_order::dpp<CTRL>((uint32_t)b));
}
__device__ __forceinline__ double row_sum(double x) { x += dpp<0xB1>(x); x += dpp<0x4E>(x); x += dpp<0x141>(x); return x + dpp<0x140>(x); }
__device__ __forceinline__ float row_max(float x)
{
    auto of = [](float y, uint32_t z) { return fmaxf(y, __uint_as_float(z)); };
    x = of(x, sk_order::dpp<0xB1>(__float_as_uint(x))); x = of(x, sk_order::dpp<0x4E>(__float_as_uint(x)));
    x = of(x, sk_order::dpp<0x141>(__float_as_uint(x))); return of(x, sk_order::dpp<0x140>(__float_as_uint(x)));
}
__device__ __forceinline__ int row_min(int x)
{
    x = min(x, (int)sk_order::dpp<0xB1>(x)); x = min(x, (int)sk_order::dpp<0x4E>(x)); x = min(x, (int)sk_order::dpp<0x141>(x));
    return min(x, (int)sk_order::dpp<0x140>(x));
}
__device__ __forceinline__ double wave_sum(double x)
{
    x = row_sum(x);
#pragma unroll
    for (int far = 0; far < 2; ++far) {
        const uint64_t b = __builtin_bit_cast(uint64_t, x);
        const uint32_t l = (uint32_t)b, h = (uint32_t)(b >> 32);
        uint32_t l0, l1, h0, h1;
        if (far) { const auto r = __builtin_amdgcn_permlane32_swap(l, l, false, false); const auto q = __builtin_amdgcn_permlane32_swap(h, h, false, false); l0 = r[0]; l1 = r[1]; h0 = q[0]; h1 = q[1]; }
        else { const auto r = __builtin_amdgcn_permlane16_swap(l, l, false, false); const auto q = __builtin_amdgcn_permlane16_swap(h, h, false, false); l0 = r[0]; l1 = r[1]; h0 = q[0]; h1 = q[1]; }
        x = __builtin_bit_cast(double, (uint64_t)h0 << 32 | l0) + __builtin_bit_cast(double, (uint64_t)h1 << 32 | l1);
    }
    return x;
}
__device__ __forceinline__ float wave_max(const float x) { return sk_order::value_of(__builtin_amdgcn_readfirstlane(sk_order::wave_max(sk_order::rank_of(x)))); }
__device__ __forceinline__ double of_lane(const double x, const int lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__shfl((int)(b >> 32), lane, 64) << 32 | (uint32_t)__shfl((int)(uint32_t)b, lane, 64));
}
// Sum over the lanes up to and with this one: within a row of 16 lanes by shifts of it, then the last lane of a row added to the rows behind it.
template <int CTRL, int ROWS, bool BOUND> __device__ __forceinline__ double shifted(const double x)
{
    u32x2 b = __builtin_bit_cast(u32x2, x);
    b.x = __builtin_amdgcn_update_dpp(0u, b.x, CTRL, ROWS, 0xf, BOUND);
    b.y = __builtin_amdgcn_update_dpp(0u, b.y, CTRL, ROWS, 0xf, BOUND);
    return __builtin_bit_cast(double, b);
}
__device__ __forceinline__ double wave_running_sum(double x)
{
    x += shifted<0x111, 0xf, true>(x); x += shifted<0x112, 0xf, true>(x); x += shifted<0x114, 0xf, true>(x); x += shifted<0x118, 0xf, true>(x);
    x += shifted<0x142, 0xa, false>(x); return x + shifted<0x143, 0xc, false>(x);
}

// The exponent's factor of a sequence: log2(e) / T; greedy sequences, whose log probabilities are those of the logits as they are, have T = 1.
__device__ __forceinline__ double scale_of(const Args& A, const int seq, bool& greedy)
{
    const float t = A.temperature ? A.temperature[seq] : 1.f;
    greedy = !(t > 0.f);
    return 1.4426950408889634 / (greedy ? 1.0 : (double)t);
}

// Tokens that a sequence has drafted, those in front of the first outside the vocabulary, from one a lane.
__device__ __forceinline__ int drafted(const Args& A, const int32_t token)
{
    return __builtin_ctzll(__ballot((int)(threadIdx.x & 63) >= A.n_draft || (uint32_t)token >= (uint32_t)A.vocab));      // (fewer than a wave's lanes)
}
__device__ __forceinline__ int32_t token_of_lane(const Args& A, const int seq)
{
    const int lane = threadIdx.x & 63;
    return lane < A.n_draft ? A.tokens[(int64_t)seq * A.n_draft + lane] : -1;
}

__device__ __forceinline__ const unsigned char* row_of(const Args& A, const int seq, const int r)
{
    if (r <= A.n_draft) return A.target + ((int64_t)seq * (A.n_draft + 1) + r) * A.target_stride;
    return A.draft + ((int64_t)seq * A.n_draft + r - A.n_draft - 1) * A.draft_stride;
}

// ---- first launch: maximum and sum of a part of a row ----

// Bound: vector instructions beside HBM.  256 rows of 128,256 fp32 logits (131 MB) in 27 us, 4.9 TB/s; 19.6 instructions to a wave's 64 logits, of which the loop's 14 of 64 bits and one
// of 32, take 76 % of the cycles.  With every logit's distance clamped, and the copies that a maximum of two and a row of three logits in the same code cost, 24.5 instructions and 30.5 us.  Of
// 576 rows in one launch, at that time 61-68 us: 16 logits a lane 70, 64 64.5; several parts a workgroup, the next one's loads in flight while it computes, 72-77 (a third fewer waves);
// loads ahead of the look at the sequence 67; without the exponentials 43 (6.9 TB/s).
template <bool F32, int EACH>
__global__ __launch_bounds__(kThreads) void sk_verify_rows(const Args A)
{
    constexpr int EL = F32 ? 4 : 2, N = 16 / EL, P = EACH / N;      // P pieces of 16 bytes
    __shared__ Part of_wave[kWaves];
    const int part = blockIdx.x % A.parts, row = blockIdx.x / A.parts, rows = A.places + A.drafts, seq = row / rows, of_seq = row - seq * rows;
    const int place = A.place0 + (of_seq < A.places ? of_seq : of_seq - A.places), r = of_seq < A.places ? place : A.n_draft + 1 + place;
    if (A.place0 > 0 && A.ended[seq]) return;
    if (EACH == kEachFew && part == 0 && of_seq == 0 && threadIdx.x == 0) A.arrived[seq * kApart] = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t tokens = token_of_lane(A, seq);
    const int n = drafted(A, tokens);
    bool greedy;
    const double scale = scale_of(A, seq, greedy);
    if (r <= A.n_draft ? place > n : greedy || place >= n) return;
    const unsigned char* x = row_of(A, seq, r);
    const float none = -__builtin_inff();
    const int stretch = part * kWaves + wave, at0 = stretch * 64 * EACH + lane * N;      // piece i: N logits from at0 + i * 64 * N on
    if (place < n) {
        const int32_t t = __builtin_amdgcn_readlane(tokens, place);
        if (t / (64 * EACH) == stretch && lane == 0) A.given[(int64_t)seq * A.rows + r] = logit<F32>(x, t);
    }
    float m;
    double e, total;
    int at = INT32_MAX;
    // of a lane's logits, the i-th of which is index(i) of the row
    auto sum_up = [&](auto& v, auto index) __attribute__((always_inline)) {
        constexpr int M = sizeof(v) / sizeof(float);
        m = v[0];
        float low = v[0];
#pragma unroll
        for (int i = 1; i < M; i += 2) { const int k = i + 1 < M ? i + 1 : i; m = max_of(m, v[i], v[k]); low = min_of(low, v[i], v[k]); }
        m = wave_max(m);
        e = exponent_of(m, scale);
        double sum[2] = {0.0, 0.0};
        if (__builtin_fabs(e) < kFar && __all(__builtin_fma((double)low, scale, -e) >= kLeast)) {        // (a NaN makes the sum one)
            const double base = kRounds - e;
#pragma unroll
            for (int i = 0; i < M; ++i) sum[i & 1] += weight_within(v[i], scale, base);
        } else {
            bool bad = m == __builtin_inff();
#pragma unroll
            for (int i = 0; i < M; ++i) bad |= v[i] != v[i];
            if (__builtin_fabs(e) < kFar) {
#pragma unroll
                for (int i = 0; i < M; ++i) sum[i & 1] += weight_or_least(v[i], scale, e);
            } else if (m != none) {
#pragma unroll
                for (int i = 0; i < M; ++i) sum[0] += v[i] == m ? 1.0 : 0.0;
            }
            if (bad) sum[0] = __builtin_nan("");
        }
        total = wave_sum(sum[0] + sum[1]);
        if (greedy) {
#pragma unroll
            for (int i = M - 1; i >= 0; --i) at = v[i] == m ? index(i) : at;
#pragma unroll
            for (int s = 1; s < 64; s *= 2) at = min(at, __shfl_xor(at, s, 64));
        }
    };
    if (A.vocab >= N) {
        float v[EACH];
        u32x4 w[P];
        const int last = A.vocab - N;
        if ((stretch + 1) * 64 * EACH <= A.vocab) {
            const unsigned char* from = x + (int64_t)at0 * EL;
#pragma unroll
            for (int i = 0; i < P; ++i) w[i] = *(const u32x4_anywhere*)(from + i * 1024);
#pragma unroll
            for (int i = 0; i < EACH; ++i) v[i] = element<F32>(w[i / N], i % N);
        } else {
            // A piece that reaches behind the row is read N logits in front of its end, of which those count that are its own.
#pragma unroll
            for (int i = 0; i < P; ++i) w[i] = *(const u32x4_anywhere*)(x + (int64_t)min(at0 + i * 64 * N, last) * EL);
#pragma unroll
            for (int i = 0; i < EACH; ++i) v[i] = i % N >= at0 + i / N * 64 * N - last ? element<F32>(w[i / N], i % N) : none;
        }
        sum_up(v, [&](const int i) { return min(at0 + i / N * 64 * N, last) + i % N; });
    } else {
        float v[1] = {stretch == 0 && lane < A.vocab ? logit<F32>(x, lane) : none};
        sum_up(v, [&](int) { return lane; });
    }
    if (lane == 0) {
        of_wave[wave] = Part{total, e, m, at};
        if (r <= A.n_draft) A.of_stretch[((int64_t)seq * (A.n_draft + 1) + r) * A.stretches + stretch] = Sum{total, e};
    }
    __syncthreads();
    if (threadIdx.x < 64) {                        // lanes 0 to 3 have the waves'
        const Part p = lane < kWaves ? of_wave[lane] : Part{0.0, kNoExponent, none, INT32_MAX};
        const float top = row_max(p.max);
        const double to = exponent_of(top, scale), all = row_sum(at_exponent(p.sum, p.e, to));
        const int first = row_min(p.max == top ? p.at : INT32_MAX);
        if (lane == 0) A.part[((int64_t)seq * A.rows + r) * A.parts + part] = Part{all, to, top, first};
    }
}

// ---- which tokens stay ----

// Whole rows from their parts, which meet in sixteen lanes each: those of the first `places` places (rows that were not computed hold anything, and are
// not looked at).  sum 0: no probabilities.
__device__ __forceinline__ void join_rows(const Args& A, const int seq, const int places, const double scale, Part* row)
{
    constexpr int kParts = 4;                      // of a lane, asked for at once
    const int tid = threadIdx.x, n = places + (A.draft ? min(places, A.n_draft) : 0);
    for (int i = tid >> 4; i < n; i += kThreads / 16) {
        const int r = i < places ? i : A.n_draft + 1 + i - places;
        const Part* p = A.part + ((int64_t)seq * A.rows + r) * A.parts;
        Part o = {0.0, kNoExponent, -__builtin_inff(), INT32_MAX};
        for (int c0 = tid & 15; c0 < A.parts; c0 += 16 * kParts) {
            Part y[kParts];
#pragma unroll
            for (int j = 0; j < kParts; ++j) y[j] = p[min(c0 + 16 * j, A.parts - 1)];
#pragma unroll
            for (int j = 0; j < kParts; ++j) {
                if (c0 + 16 * j >= A.parts) continue;
                const double to = __builtin_fmax(o.e, y[j].e);
                o = Part{at_exponent(o.sum, o.e, to) + at_exponent(y[j].sum, y[j].e, to), to, fmaxf(o.max, y[j].max),
                         y[j].max > o.max ? y[j].at : y[j].max == o.max ? min(o.at, y[j].at) : o.at};
            }
        }
        const float top = row_max(o.max);
        const double to = exponent_of(top, scale), sum = row_sum(at_exponent(o.sum, o.e, to));
        const int at = row_min(o.max == top ? o.at : INT32_MAX);
        if ((tid & 15) == 0) row[r] = Part{sum > 0.0 ? sum : 0.0, to, top, at};      // (NaN: none)
    }
}

// A drafted token's logits in its two rows, and its number, for the lanes of a wave
__device__ __forceinline__ void given_of(const Args& A, const int seq, const int lane, float& xp, float& xq, float& u)
{
    xp = A.given[(int64_t)seq * A.rows + lane];
    xq = A.draft ? A.given[(int64_t)seq * A.rows + A.n_draft + 1 + lane] : 0.f;
    u = A.uniform[(int64_t)seq * (A.n_draft + 1) + lane];
}
__device__ __forceinline__ bool token_stays(const Args& A, const int place, const int32_t token, const bool greedy, const double scale, const float xp, const float xq,
                                            const float u, const Part* row)
{
    const Part p = row[place];
    if (!(p.sum > 0.0)) return false;
    if (greedy) return token == p.at;
    const double px = weight_of(xp, scale, p.e, p.max) / p.sum;
    if (!A.draft) return (double)u < px;
    const Part q = row[A.n_draft + 1 + place];
    return q.sum > 0.0 && (double)u * (weight_of(xq, scale, q.e, q.max) / q.sum) < px;
}

// Where rows come in two launches: which sequences' drafts end within the first, for good or by a token that does not stay.
__global__ __launch_bounds__(kThreads) void sk_verify_ends(const Args A)
{
    __shared__ Part row[kMaxRows];
    const int seq = blockIdx.x, tid = threadIdx.x;
    bool greedy;
    const double scale = scale_of(A, seq, greedy);
    const int32_t token = token_of_lane(A, seq);
    const int n = min(drafted(A, token), A.place0);
    float xp = 0.f, xq = 0.f, u = 0.f;
    if (tid < n) given_of(A, seq, tid, xp, xq, u);
    join_rows(A, seq, A.place0, scale, row);
    __syncthreads();
    if (tid < 64) {
        const uint64_t out = ~__ballot(tid < n && token_stays(A, tid, token, greedy, scale, xp, xq, u, row));
        if (tid == 0) A.ended[seq] = (int)__builtin_ctzll(out) < A.place0;
    }
}

// ---- second launch: the sums of the stretches of the row that is drawn from, and the draw ----
//
// Every workgroup finds by itself which row that is (a launch for it would cost as much), unless there are many.  Bound: round trips one behind the other, four to the sums (5 us for one
// sequence of 128,256 logits), four more to the drawn token (8.7; in a launch of its own 5.3 + 3.4 and the gap between them, and 2.5 us more of the host).  Where there are many rows, two rows' way and
// their exponentials: 64 sequences 14.0 us, of which reading 66 MB takes 13 (21.7 where every workgroup decides); there a workgroup that waits until its sum has arrived keeps another from
// starting (38 us with the draw, 29 in two launches).

// What a logit of the row that is drawn from counts for.
template <bool F32> struct Weights {
    const unsigned char *p, *q;
    Chosen c;
    int32_t without;
    __device__ __forceinline__ Weights(const Args& A, const Chosen& chosen, const int seq) : c(chosen)
    {
        p = row_of(A, seq, c.place);
        q = c.less == 1 ? row_of(A, seq, A.n_draft + 1 + c.place) : p;
        without = c.less == 2 ? A.tokens[(int64_t)seq * A.n_draft + c.place] : -1;
    }
    // Where no exponent is far, as nearly always, what a logit has to pass holds no branch: `visit` is called with a function of two logits and an index.
    template <class V> __device__ __forceinline__ void each(V visit) const
    {
        const bool near = __builtin_fabs(c.p_e) < kFar && __builtin_fabs(c.q_e) < kFar;
        if (near && c.less == 1)
            visit([&](const float x, const float y, int) __attribute__((always_inline)) {
                return __builtin_fmax(__builtin_fma(weight_or_least(x, c.scale, c.p_e), c.p_inv, -kNothing) - weight_or_least(y, c.scale, c.q_e) * c.q_inv, 0.0);
            });
        else if (near)
            visit([&](const float x, float, const int i) __attribute__((always_inline)) {
                const double w = __builtin_fmax(__builtin_fma(weight_or_least(x, c.scale, c.p_e), c.p_inv, -kNothing), 0.0);
                return i == without ? 0.0 : w;
            });
        else
            visit([&](const float x, const float y, const int i) __attribute__((always_inline)) { return (*this)(x, y, i); });
    }
    // of logits x and y of the two rows, at index i
    __device__ __forceinline__ double operator()(const float x, const float y, const int i) const
    {
        auto weight = [&](const float z, const double e, const float max) { return __builtin_fabs(e) < kFar ? weight_or_least(z, c.scale, e) : z == max ? 1.0 : 0.0; };
        double w = __builtin_fma(weight(x, c.p_e, c.p_max), c.p_inv, -kNothing);
        if (c.less == 1) w -= weight(y, c.q_e, c.q_max) * c.q_inv;
        return i == without ? 0.0 : __builtin_fmax(w, 0.0);
    }
};

constexpr int kSums = 4;                           // stretches of a lane that are asked for at once

// The token that the sequence's last number finds in the running sum of the row's weights: the stretch, by every wave for itself, then the thread, then
// its logit.  Where roundings leave the sum below the limit, or the number is 1 or more, the last that counts is taken at each step.  `summed(i)` is what has been added up
// for stretch i if less is 1, or 2 and the drafted token is in it; `first` holds it for the first ones.
template <bool F32, int STRETCH, class SUMMED>
__device__ __forceinline__ void draw(const Args& A, const int seq, const Weights<F32>& w, const float number, const SUMMED summed, double (&first)[kSums])
{
    constexpr int EACH = STRETCH / kThreads;       // logits of a thread, one behind the other
    __shared__ double of_wave[kWaves];
    __shared__ uint64_t over_of[kWaves], some_of[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Chosen& c = w.c;
    // The target's own sums.  One below 2^-960 is none: all of its logits, 2^11 at most, may be nothing.
    const Sum* known = A.of_stretch + ((int64_t)seq * (A.n_draft + 1) + c.place) * A.stretches;
    auto known_sum = [&](const int i, const double again) {
        const Sum k = known[min(i, A.stretches - 1)];
        const double x = at_exponent(k.sum, k.e, c.p_e) * c.p_inv;
        return c.less == 2 && i == w.without / STRETCH ? again : x < 0x1p-960 ? 0.0 : x;
    };
    if (c.less != 1) {
#pragma unroll
        for (int j = 0; j < kSums; ++j) first[j] = known_sum(64 * j + lane, first[j]);
    }
    auto stretch_sum = [&](const int base) {
        if (base + lane >= A.stretches) return 0.0;
        if (base < 64 * kSums) return base < 128 ? (base ? first[1] : first[0]) : base == 128 ? first[2] : first[3];
        return c.less == 1 ? summed(base + lane) : known_sum(base + lane, summed(base + lane));
    };
    double total = 0.0;
    for (int base = 0; base < A.stretches; base += 64) total += stretch_sum(base);
    total = wave_sum(total);
    const double limit = __builtin_fmax((double)number, 0.0) * total;
    double before = 0.0, left = 0.0;
    int stretch = -1;
    for (int base = 0; base < A.stretches; base += 64) {
        const double mine = stretch_sum(base), running = before + wave_running_sum(mine);
        const uint64_t over = __ballot(mine > 0.0 && running > limit), some = __ballot(mine > 0.0);
        if (some) {
            const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);
            stretch = base + l;
            left = limit - (l ? of_lane(running, l - 1) : before);
        }
        if (over) break;
        before = of_lane(running, 63);
    }
    const int64_t to = (int64_t)seq * (A.n_draft + 1) + c.place;
    if (stretch < 0) {                             // nothing is left of the target: p and q are one, and the drafted token is as good
        if (tid == 0) {
            const int token = c.less ? A.tokens[(int64_t)seq * A.n_draft + c.place] : 0;
            A.out_tokens[to] = token;
            if (A.logprob) A.logprob[to] = log_probability(logit<F32>(row_of(A, seq, c.place), token), c.scale, c.p_e, c.p_max, c.p_inv);
        }
        return;
    }
    const int begin = stretch * STRETCH + tid * EACH;
    float x[EACH], y[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int t = min(begin + i, A.vocab - 1);
        x[i] = logit<F32>(w.p, t);
        y[i] = logit<F32>(w.q, t);
    }
    double weight[EACH], mine = 0.0;
    w.each([&](auto one) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) { const double z = one(x[i], y[i], begin + i); weight[i] = begin + i < A.vocab ? z : 0.0; mine += weight[i]; }
    });
    double running = wave_running_sum(mine);
    if (lane == 63) of_wave[wave] = running;
    __syncthreads();
    double in_front = 0.0;
    for (int i = 0; i < wave; ++i) in_front += of_wave[i];
    const uint64_t over = __ballot(mine > 0.0 && in_front + running > left), some = __ballot(mine > 0.0);
    if (lane == 0) { over_of[wave] = over; some_of[wave] = some; }
    __syncthreads();
    int chosen_wave = -1, chosen_lane = 0;
    for (int i = kWaves - 1; i >= 0; --i) {
        if (over_of[i]) { chosen_wave = i; chosen_lane = __builtin_ctzll(over_of[i]); }
        else if (some_of[i] && chosen_wave < 0) { chosen_wave = i; chosen_lane = 63 - __builtin_clzll(some_of[i]); }
    }
    if (wave != chosen_wave || lane != chosen_lane) return;
    double sum = in_front + running - mine;
    int token = begin;
    float its = x[0];
    bool passed = false;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (!passed && weight[i] > 0.0) { token = begin + i; its = x[i]; }
        sum += weight[i];
        passed |= weight[i] > 0.0 && sum > left;
    }
    A.out_tokens[to] = token;
    if (A.logprob) A.logprob[to] = log_probability(its, c.scale, c.p_e, c.p_max, c.p_inv);
}

// By a workgroup: how many of a sequence's tokens stay, and what it draws from; everything that it returns but a token that is still to be drawn.
__device__ __forceinline__ void decide(const Args& A, const int seq, const bool writes, Part* row, Chosen& chosen)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const float none = -__builtin_inff();
    bool greedy;
    const double scale = scale_of(A, seq, greedy);
    const int32_t token = token_of_lane(A, seq);
    const int n = drafted(A, token);
    // a drafted token's logits, for the lanes of the first wave
    float xp = none, xq = none, u = 0.f;
    if (tid < n) given_of(A, seq, lane, xp, xq, u);
    join_rows(A, seq, A.n_draft + 1, scale, row);
    __syncthreads();
    if (tid < 64) {
        const bool stays = lane < n && token_stays(A, lane, token, greedy, scale, xp, xq, u, row);
        const uint64_t out = ~__ballot(stays);
        const int a = min(n, (int)__builtin_ctzll(out));            // (lanes from n on are out)
        const Part p = row[a];
        const bool valid = p.sum > 0.0;
        if (lane == 0) {
            Chosen c = {scale, p.e, 1.0 / p.sum, 0.0, 0.0, p.max, 0.f, valid && !greedy ? a : -1, 0};
            if (a < n && !A.draft) c.less = 2;
            else if (a < n && !greedy && row[A.n_draft + 1 + a].sum > 0.0) {
                const Part q = row[A.n_draft + 1 + a];
                c.less = 1; c.q_e = q.e; c.q_inv = 1.0 / q.sum; c.q_max = q.max;
            }
            chosen = c;
            if (writes) A.n_accepted[seq] = a;
        }
        if (writes && lane <= A.n_draft && (lane != a || !valid || greedy)) {       // everything but a token that is still to be drawn
            const int32_t t = lane < a ? token : lane == a && valid && greedy ? p.at : -1;
            const int64_t at = (int64_t)seq * (A.n_draft + 1) + lane;
            A.out_tokens[at] = t;
            if (A.logprob) {
                float l = 0.f;
                if (lane < a || (lane == a && valid && greedy)) {
                    const Part r = row[lane];
                    l = log_probability(lane < a ? xp : p.max, scale, r.e, r.max, 1.0 / r.sum);
                } else if (lane == a && !valid) l = __builtin_nanf("");
                A.logprob[at] = l;
            }
        }
    }
}

// ... in a launch of its own, where there are many workgroups
__global__ __launch_bounds__(kThreads) void sk_verify_decide(const Args A)
{
    __shared__ Part row[kMaxRows];
    decide(A, blockIdx.x, true, row, A.chosen[blockIdx.x]);
}

template <bool F32, int EACH, bool DECIDES>
__global__ __launch_bounds__(kThreads) void sk_verify_stretches(const Args A)
{
    // eight logits to a lane: a workgroup has one stretch, or four
    constexpr int EL = F32 ? 4 : 2, N = 16 / EL, P = 8 / N, kOfThisWg = kThreads * 8, kOfWg = kOfThisWg / (64 * EACH);
    constexpr bool kDraws = EACH == kEachFew;
    static_assert(kOfWg == (kDraws ? kWaves : 1) && (DECIDES || !kDraws), "");
    __shared__ double of_wave[kWaves];
    __shared__ int draws;
    Chosen chosen;
    const int wgs = A.stretches / kOfWg, wg = blockIdx.x % wgs, seq = blockIdx.x / wgs, tid = threadIdx.x, lane = tid & 63;
    const float number = A.uniform[(int64_t)seq * (A.n_draft + 1) + A.n_draft];
    if constexpr (DECIDES) {
        __shared__ Part row[kMaxRows];
        __shared__ Chosen found;
        decide(A, seq, wg == 0, row, found);
        __syncthreads();
        chosen = found;
        if (!kDraws && wg == 0 && tid == 0) A.chosen[seq] = chosen;
    } else chosen = A.chosen[seq];
    // The target's own sums are known; without the drafted token, all but those of its stretch.
    if (chosen.place < 0 || (chosen.less == 0 && !(kDraws && wg == 0))) return;
    const Weights<F32> w(A, chosen, seq);
    if (w.c.less == 2 && w.without / kOfThisWg != wg) return;
    double again = 0.0, *sums = A.sums + (int64_t)seq * A.stretches;
    if (w.c.less > 0) {
        const int sub = wg * kWaves + (tid >> 6);
        double sum = 0.0;
        if (A.vocab >= N) {                        // pieces of 16 bytes as in the first launch
            const int at0 = sub * 512 + lane * N, last = A.vocab - N;
            u32x4 x[P], y[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int64_t at = (int64_t)min(at0 + i * 64 * N, last) * EL;
                x[i] = *(const u32x4_anywhere*)(w.p + at);
                y[i] = *(const u32x4_anywhere*)(w.q + at);
            }
            w.each([&](auto one) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const int first = at0 + i * 64 * N, from = min(first, last);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const double z = one(element<F32>(x[i], e), element<F32>(y[i], e), from + e);
                        sum += from + e >= first ? z : 0.0;
                    }
                }
            });
        } else {
            for (int i = lane; i < A.vocab && sub == 0; i += 64) sum += w(logit<F32>(w.p, i), logit<F32>(w.q, i), i);
        }
        sum = wave_sum(sum);
        if (lane == 0) of_wave[tid >> 6] = sum;
        __syncthreads();
        if (!kDraws) {                             // the workgroup is one stretch
            if (tid == 0) sums[wg] = of_wave[0] + of_wave[1] + of_wave[2] + of_wave[3];
            return;
        }
        if (w.c.less == 2) again = of_wave[w.without / (64 * EACH) % kWaves];
        else {
            // Sums leave by stores that write through, and have arrived behind the wait, before the workgroup is counted: whoever counts the last one finds all.  Nobody waits.
            if (tid == 0) {
#pragma unroll
                for (int i = 0; i < kWaves; ++i) __hip_atomic_store(&sums[wg * kWaves + i], of_wave[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                asm volatile("" : : : "memory");
                __builtin_amdgcn_s_waitcnt(0);
                asm volatile("" : : : "memory");
                draws = __hip_atomic_fetch_add(&A.arrived[seq * kApart], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == (uint32_t)wgs;
            }
            __syncthreads();
            if (!draws) return;
        }
    }
    if (!kDraws) return;
    auto summed = [&](const int i) { return w.c.less == 1 ? __hip_atomic_load(&sums[min(i, A.stretches - 1)], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : again; };
    double first[kSums];
#pragma unroll
    for (int j = 0; j < kSums; ++j) first[j] = summed(64 * j + lane);
    draw<F32, 64 * EACH>(A, seq, w, number, summed, first);
}

// The draw in a launch of its own, where there are many rows.  Bound: three round trips (6.2 us for 64 sequences).
template <bool F32>
__global__ __launch_bounds__(kThreads) void sk_verify_draw(const Args A)
{
    const int seq = blockIdx.x, lane = threadIdx.x & 63;
    const double* sums = A.sums + (int64_t)seq * A.stretches;
    auto summed = [&](const int i) { return sums[min(i, A.stretches - 1)]; };
    const float number = A.uniform[(int64_t)seq * (A.n_draft + 1) + A.n_draft];
    double first[kSums];
#pragma unroll
    for (int j = 0; j < kSums; ++j) first[j] = summed(64 * j + lane);
    const Chosen c = A.chosen[seq];
    if (c.place < 0) return;
    draw<F32, 64 * kEach>(A, seq, Weights<F32>(A, c, seq), number, summed, first);
}

int64_t parts_of(const int64_t each, const int32_t vocab) { return (vocab + each * kThreads - 1) / (each * kThreads); }
// Logits of a lane.  us per call in a stream of them, eight (two launches) -> 32 (three), fp32 rows of 128,256 logits with their draft's: 1 x 4 12.7 -> 15.2, 4 x 4 16.5 -> 17.5, 7 x 4 (1,008
// parts of 32) 20.9 -> 21.4, 10 x 4 25.0 -> 24.9, 14 x 4 29.0 -> 29.0, 24 x 4 43 -> 38; bf16 rows of 50,257 16 x 3 17.0 -> 19.5, 64 x 3 39.5 -> 34.4; without a draft 16 x 0 10.9 -> 13.4, 40 x 0 15.3 ->
// 17.0, 64 x 0 (1,024 parts) 19.8 -> 20.4, 300 x 0 rows of 32,000 (1,200) 30 -> 25.  Eight, and the draws in a launch of their own: 1 x 4 13.8, 4 x 4 17.5, 16 x 0 13.8; with sequences' counts
// next to each other 4 x 4 18.8, 10 x 4 29.5.
int each_of(const int64_t rows, const int32_t vocab) { return rows * parts_of(kEach, vocab) < 1024 ? kEachFew : kEach; }
bool sizes_ok(const int32_t n_seq, const int32_t n_draft, const int32_t vocab)
{
    return n_seq > 0 && n_draft >= 0 && n_draft <= SK_VERIFY_MAX_DRAFT && vocab >= 1 && vocab <= SK_VERIFY_MAX_VOCAB &&
           (int64_t)n_seq * (n_draft + 1) <= SK_VERIFY_MAX_ROWS;
}
// What a call keeps, in the order in which it lies in the workspace
size_t lay_out(Args& A, const int each, void* workspace, const int32_t n_seq)
{
    const int64_t parts = (int64_t)n_seq * A.rows * A.parts, stretches = (int64_t)n_seq * A.stretches;
    uintptr_t at = (uintptr_t)workspace;
    auto take = [&](const int64_t n, const size_t bytes) { const uintptr_t p = at; at += size_t(n) * bytes; return (void*)p; };
    A.part = (Part*)take(parts, sizeof(Part));
    A.of_stretch = (Sum*)take(stretches * (A.n_draft + 1), sizeof(Sum));
    A.given = (float*)take((int64_t)n_seq * A.rows, sizeof(float));
    A.ended = (int32_t*)take(n_seq + ((n_seq * (int64_t)A.rows + n_seq) & 1), sizeof(int32_t));
    A.arrived = (uint32_t*)take(each == kEachFew ? n_seq * kApart : 0, sizeof(uint32_t));
    A.chosen = (Chosen*)take(n_seq, sizeof(Chosen));
    A.sums = (double*)take(stretches, sizeof(double));
    return size_t(at - (uintptr_t)workspace);
}
int cut(Args& A, const int32_t n_seq, const int32_t n_draft, const int32_t vocab, const bool draft)
{
    A.n_draft = n_draft; A.vocab = vocab;
    A.rows = n_draft + 1 + (draft ? n_draft : 0);
    const int each = each_of((int64_t)n_seq * A.rows, vocab);
    A.parts = (int32_t)parts_of(each, vocab); A.stretches = A.parts * kWaves;
    return each;
}

// The launches of n_seq sequences
int launch(Args& A, const int each, const int dtype, const int32_t n_seq, void* workspace, hipStream_t st)
{
    lay_out(A, each, workspace, n_seq);
    const dim3 block(kThreads), second((unsigned)n_seq * (each == kEach ? A.stretches : A.stretches / kWaves)), each_seq((unsigned)n_seq);
    // Where there are many rows, those of the first two places come first, and the others only of sequences whose draft is still standing.  us per call, all
    // rows at once -> in two launches, rows of 128,256 logits with their draft's, by what share of the drafted tokens is accepted (each row at the nearest one measured):
    //   accepted of the drafted            0.95-0.98     0.8           0.65          0.4           0.2           0.05
    //   64 x 4 (9,216 parts)                72 ->  80     70 ->  76     74 ->  72     78 ->  69     79 ->  66     79 ->  59
    //   64 x 8 (17,408)                    120 -> 132    126 -> 131    130 -> 124    136 -> 121    138 -> 104    137 ->  64
    //   128 x 4 (18,432)                   129 -> 141    138 -> 139    142 -> 140    151 -> 127    154 -> 113    155 ->  99
    //   128 x 4, bf16                      113 -> 127    125 -> 117    132 -> 115    140 -> 109    144 -> 103    144 ->  95
    //   256 x 4, bf16 of 32,000 (9,216)     63 ->  69     63 ->  71     65 ->  70     69 ->  67     71 ->  63     73 ->  60
    //   64 x 16 of 50,257 (14,784)         104 -> 117    104 -> 117        -         107 -> 103    109 ->  74    108 ->  56
    //   32 x 8 (8,704)                      64 ->  73     65 ->  67     65 ->  66     67 ->  61     69 ->  56     70 ->  48
    //   64 x 3, bf16 (7,168)                52 ->  57     52 ->  58     54 ->  59     57 ->  60     61 ->  58     61 ->  57
    //   32 x 4 (4,608)                      40 ->  49     41 ->  49     43 ->  49     45 ->  48     46 ->  47     46 ->  40
    // A token that stays with 0.9, 0.8 or 0.7, if those in front do, makes that share 0.77, 0.59 and 0.44 for four drafted tokens, 0.64, 0.42 and 0.27 for eight.  From the border on the
    // two launches cost up to 14 % where nearly everything stays, and save from about 0.6 on downwards, up to half; below it they rarely save.
    const bool in_two = each == kEach && A.n_draft > kFirstPlaces && (int64_t)n_seq * A.rows * A.parts >= kPartsInTwo;
    const int split = in_two ? kFirstPlaces : 0;
    // Where its workgroups are more than run at a time, the second launch finds the row that is drawn from decided by one in front of it.  us per call, 0.7 to 0.05 of the drafted
    // accepted, by every workgroup -> by a launch: 14 x 4 (896 workgroups) 28.8 -> 30.4, 24 x 4 (1,536) 37.9 -> 38.3, 32 x 4 (2,048) 43-45 -> 43-45, 64 x 3 bf16 (4,096) 60-64 -> 57-62, 64 x 4 (4,096) 62-79 -> 59-74,
    // 64 x 8 67-123 -> 63-117, 128 x 2 (8,192) 87-102 -> 84-97.
    const bool apart = (int64_t)second.x > kAtATime;
#define SK_VERIFY(F32, EACH)                                                                                                                 \
    for (int from = 0; from <= A.n_draft;) {                                                                                                 \
        const int to = from == 0 && split ? split : A.n_draft + 1;                                                                           \
        A.place0 = from; A.places = to - from; A.drafts = !A.draft ? 0 : to <= A.n_draft ? A.places : A.places - 1;                          \
        hipLaunchKernelGGL((sk_verify_rows<F32, EACH>), dim3((unsigned)n_seq * (A.places + A.drafts) * A.parts), block, 0, st, A);           \
        A.place0 = from = to;                                                                                                                \
        if (to <= A.n_draft) hipLaunchKernelGGL(sk_verify_ends, each_seq, block, 0, st, A);                                                     \
    }                                                                                                                                        \
    if (EACH == kEach && apart) {                                                                                                            \
        hipLaunchKernelGGL(sk_verify_decide, each_seq, block, 0, st, A);                                                                     \
        hipLaunchKernelGGL((sk_verify_stretches<F32, EACH, EACH == kEachFew>), second, block, 0, st, A);                                     \
    } else hipLaunchKernelGGL((sk_verify_stretches<F32, EACH, true>), second, block, 0, st, A);                                              \
    if (EACH != kEachFew) hipLaunchKernelGGL(sk_verify_draw<F32>, each_seq, block, 0, st, A)
    if (dtype == SK_F32) {
        if (each == kEach) { SK_VERIFY(true, kEach); } else { SK_VERIFY(true, kEachFew); }
    } else {
        if (each == kEach) { SK_VERIFY(false, kEach); } else { SK_VERIFY(false, kEachFew); }
    }
#undef SK_VERIFY
    return (int)hipGetLastError();
}

}  // namespace

extern "C" {

size_t sk_verify_workspace_bytes(int32_t n_seq, int32_t n_draft, int32_t vocab)
{
    if (!sizes_ok(n_seq, n_draft, vocab)) return 0;
    size_t most = 0;                               // with a draft's rows or without them, whose cut may be another
    for (int draft = 0; draft < 2; ++draft) {
        Args A = {};
        const int each = cut(A, n_seq, n_draft, vocab, draft != 0);
        const size_t bytes = lay_out(A, each, nullptr, n_seq);
        if (bytes > most) most = bytes;
    }
    return most;
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
    const size_t scratch = sk_verify_workspace_bytes(n_seq, n_draft, vocab);
    if (workspace_bytes < scratch) return SK_E_WORKSPACE;
    {   // what is written, first, lies apart from everything else
        const int64_t places = (int64_t)n_seq * (n_draft + 1), drafts = (int64_t)n_seq * n_draft;
        struct { const void* at; size_t bytes; } a[] = {
            {n_accepted, size_t(n_seq) * 4}, {out_tokens, size_t(places) * 4}, {logprob, size_t(places) * 4}, {workspace, scratch},
            {target, size_t((places - 1) * target_stride + vocab) * el}, {draft, drafts ? size_t((drafts - 1) * draft_stride + vocab) * el : 0},
            {tokens, size_t(drafts) * 4}, {uniform, size_t(places) * 4}, {temperature, size_t(n_seq) * 4}};
        for (int i = 0; i < 4; ++i)
            for (int j = i + 1; j < 9; ++j) {
                const uintptr_t x = (uintptr_t)a[i].at, y = (uintptr_t)a[j].at;
                if (x && y && x < y + a[j].bytes && y < x + a[i].bytes) return SK_E_INVAL;
            }
    }
    Args A;
    A.target = (const unsigned char*)target; A.draft = n_draft > 0 ? (const unsigned char*)draft : nullptr;
    A.target_stride = target_stride * el; A.draft_stride = draft_stride * el;
    A.tokens = tokens; A.uniform = uniform; A.temperature = temperature;
    const int each = cut(A, n_seq, n_draft, vocab, A.draft != nullptr);
    A.n_accepted = n_accepted; A.out_tokens = out_tokens; A.logprob = logprob;
    hipStream_t st = (hipStream_t)hip_stream;
    // Sequences of a launch: all, except where its grid would be too large (2^20 rows of more than 24,576 logits).
    const int32_t second_wgs = each == kEach ? A.stretches : A.stretches / kWaves, all = n_seq;
    const int32_t at_once = (int32_t)(kMaxWgs / (second_wgs > A.rows * A.parts ? second_wgs : A.rows * A.parts));
    for (int32_t s0 = 0; s0 < all; s0 += n_seq) {
        n_seq = all - s0 < at_once ? all - s0 : at_once;
        const int e = launch(A, each, dtype, n_seq, workspace, st);
        if (e) return sk_status_of(e);
        const int64_t places = (int64_t)n_seq * (n_draft + 1), drafts = (int64_t)n_seq * n_draft;
        A.target += places * A.target_stride; A.uniform += places; A.out_tokens += places; A.n_accepted += n_seq;
        if (A.draft) A.draft += drafts * A.draft_stride;
        if (A.tokens) A.tokens += drafts;
        if (A.temperature) A.temperature += n_seq;
        if (A.logprob) A.logprob += places;
    }
    return SK_OK;
}

}  // extern "C"
