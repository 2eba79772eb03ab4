// Log probabilities of given tokens, normaliser, entropy and best alternatives of logit rows (include/sk.h: sk_logprobs), gfx950.
//
// One pass over the logits.  A wave keeps, per lane, the running maximum m and the sums of a softmax against it,
//   S = sum exp(x - m),   Z = sum exp(x - m) (x - m),
// which move to a larger maximum m' = m - delta (delta < 0) by S' = e^delta S, Z' = e^delta (Z + delta S).  Then
//   lse = m + log S,   log p(t) = (x_t - m) - log S,   entropy = log S - Z / S,
// the last a sum of two terms that are never negative, so that nothing cancels in a row that is nearly certain.
// The best alternatives come from the same registers: a wave knows a bound that at least `n_top` of the logits it has seen
// reach, appends what lies above to a short list in LDS, and cuts the list back to the best n_top when it is full, which raises the
// bound.  The bound is first the n_top-th largest of the 64 lanes' maxima, found by counting lanes two bits at a time; the waves of a workgroup
// tell each other theirs, and what the highest leaves of their lists is put in order by counting larger ones.
// Bound: reading the logits once; about ten vector instructions per logit beside it.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <limits.h>
#include "../../include/sk.h"
#include "sk_internal.h"
#include "sk_order.h"

namespace {

using namespace sk_order;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kTile = 2048;           // logits that a wave takes at once, 32 in a lane
constexpr int kWaves = 4;             // of a workgroup, where a row is cut into parts or there are many
constexpr int kWavesAlone = 16;       // of one that takes a whole row, where there are few
constexpr int kList = 256;            // entries of a wave's list of candidates
constexpr float kLog2e = 1.4426950408889634f;

struct Args {
    const void* logits;
    int64_t row_stride;
    int32_t vocab, n_tokens, n_top;
    int32_t parts, tiles;             // workgroups to a row; tiles that each of their waves takes
    const int32_t* tokens;
    float *logprob, *lse, *entropy;
    int32_t* top_idx;
    float* top_logprob;
    float4* stats;                    // [rows][parts * kWaves]: m, S, Z
    uint64_t* keys;                   // [rows][parts * kWaves][n_top]
};

// A wave's candidates: rank << 32 | ~index, so that of equal logits the one of lower index is the larger key.
struct Top {
    uint64_t* list;         // LDS, kList entries
    int n, k;
    uint32_t* bound;        // LDS: the highest rank that some wave knows n_top logits of its row to reach
    float floor;            // a logit that is smaller is none of the best; one that equals it only with an index below floor_idx
    int32_t floor_idx;

    __device__ __forceinline__ void init(uint64_t* l, uint32_t* b, const int kk) { list = l; bound = b; n = 0; k = kk; floor = -__builtin_inff(); floor_idx = INT_MIN; }

    // Cuts a list of more than k entries to its k best.
    __device__ __forceinline__ void cut(const int lane)
    {
        constexpr int N = kList / 64;
        wave_order();
        uint32_t hi[N], lo[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint64_t x = 64 * j + lane < n ? list[64 * j + lane] : 0;
            hi[j] = (uint32_t)(x >> 32); lo[j] = (uint32_t)x;
        }
        int hits;
        const uint32_t t = bound_of(hi, k, hits);
        uint32_t tie = 0;                                 // of equal ranks, those whose ~index reaches this
        floor = t <= kRankNone ? -__builtin_inff() : value_of(t);
        floor_idx = INT_MIN;                              // (what lies in front of a row has negative indices)
        if (hits > k) {
            int over = 0;
            uint32_t l[N];
#pragma unroll
            for (int j = 0; j < N; ++j) { over += lanes(hi[j] > t); l[j] = hi[j] == t ? lo[j] : 0; }
            int h;
            tie = bound_of(l, k - over, h);
            floor_idx = (int32_t)~tie;
        } else if (t > kRankNone) {                       // what equals the bound, if anything does: a lower index, which a later step of the tile may bring, takes its place
            uint32_t last = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) last = max(last, hi[j] == t ? ~lo[j] : 0u);
            floor_idx = (int32_t)__builtin_amdgcn_readfirstlane(wave_max(last));
        }
        int at = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const bool stays = hi[j] > t || (hi[j] == t && lo[j] >= tie);
            const uint64_t m = __ballot(stays);
            if (stays) list[at + lanes_before(m)] = (uint64_t)hi[j] << 32 | lo[j];
            at += __popcll(m);
        }
        n = at;
        wave_order();
    }
    // Adds the keys of the lanes in `m`; the caller has seen that there is room for them.
    __device__ __forceinline__ void add(const uint64_t m, const bool mine, const uint64_t key)
    {
        if (mine) list[n + lanes_before(m)] = key;
        n += __popcll(m);
    }
    __device__ __forceinline__ bool full() const { return n > kList - 64; }
    __device__ __forceinline__ bool takes(const float x, const int32_t i) const
    {
        return x > floor || (x == floor && i < floor_idx);
    }
    // The smallest number that is taken among those whose indices are `first` and higher.
    __device__ __forceinline__ float least(const int32_t first) const
    {
        return floor_idx <= first ? value_of(rank_of(floor) + 1) : floor;
    }
    // Before numbers of which at least k reach rank t are offered: none below that is among the best.
    __device__ __forceinline__ void raise(const uint32_t t)
    {
        const float f = value_of(t);
        if (t > kRankNone && f > floor) { floor = f; floor_idx = INT_MAX; }
    }
    // Tells the other waves, and hears from them.
    __device__ __forceinline__ void share(const int lane)
    {
        if (lane == 0) atomicMax(bound, rank_of(floor));
        raise(__builtin_amdgcn_readfirstlane(__hip_atomic_load(bound, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)));
    }
};

// The 32 logits of this lane in tile `tile` of a row; what lies outside the row is -inf.  `row`: rounded down to 16 bytes, `skip` the
// elements of another row that come first.
template <bool BF16>
__device__ __forceinline__ void load_tile(const unsigned char* __restrict__ row, const int skip, const int64_t total, const int tile, const int lane, float (&x)[32])
{
    constexpr int V = BF16 ? 8 : 4, NV = 32 / V;          // logits to a 16-byte piece, pieces to a lane
    const int64_t first = (int64_t)tile * kTile;
    u32x4 p[NV];
    if (first >= skip && first + kTile <= total) {
        const u32x4* src = (const u32x4*)row + first / V + lane;
#pragma unroll
        for (int u = 0; u < NV; ++u) p[u] = __builtin_nontemporal_load(src + 64 * u);
    } else {                                              // pieces that reach over an end are put together from what lies inside
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int64_t e = first + (int64_t)V * (lane + 64 * u);
            if (e >= skip && e + V <= total) p[u] = __builtin_nontemporal_load((const u32x4*)row + e / V);
            else {
                uint32_t w[V];
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    const bool in = e + c >= skip && e + c < total;
                    if (BF16) w[c] = in ? ((const uint16_t*)row)[e + c] : 0xff80u;
                    else w[c] = in ? ((const uint32_t*)row)[e + c] : 0xff800000u;
                }
                if (BF16) p[u] = u32x4{w[0] | w[1 % V] << 16, w[2 % V] | w[3 % V] << 16, w[4 % V] | w[5 % V] << 16, w[6 % V] | w[7 % V] << 16};
                else p[u] = u32x4{w[0], w[1], w[2], w[3]};
            }
        }
    }
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (BF16) { x[u * V + 2 * c] = __uint_as_float(p[u][c] << 16); x[u * V + 2 * c + 1] = __uint_as_float(p[u][c] & 0xffff0000u); }
            else x[u * V + c] = __uint_as_float(p[u][c]);
        }
}

struct Sums { float m, s, z; };

__device__ __forceinline__ float exp_of(const float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
__device__ __forceinline__ float finite_or_0(const float m) { return m == -__builtin_inff() ? 0.f : m; }

// The sums of `a`, moved to the maximum M >= a.m (not -inf).  A side that saw nothing but -inf (or NaN, which stays one) has no z.  (e^-200 is
// 0 in 32 bits: a side that saw nothing but a mask's 1e38s counts 0, and not 0 times a product that is infinite.)
__device__ __forceinline__ Sums moved(const Sums a, const float M)
{
    const float d = fmaxf(a.m - M, -200.f), f = exp_of(d);
    return Sums{M, a.s * f, a.m == -__builtin_inff() ? 0.f : f * (a.z + d * a.s)};
}

__device__ __forceinline__ Sums wave_sums(Sums a)
{
    float M = a.m;
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) M = fmaxf(M, __shfl_xor(M, i, 64));
    a = moved(a, finite_or_0(M));
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) { a.s += __shfl_xor(a.s, i, 64); a.z += __shfl_xor(a.z, i, 64); }
    a.m = M;
    return a;
}

template <bool BF16>
struct Row {
    const unsigned char* logits;
    float m, log_s;
    bool none;                        // nothing above -inf
    __device__ __forceinline__ Row(const Args& A, const int r) : logits((const unsigned char*)A.logits + (int64_t)r * A.row_stride * (BF16 ? 2 : 4)) {}
    __device__ __forceinline__ void of(const Sums a) { m = finite_or_0(a.m); log_s = logf(a.s); none = a.s == 0.f; }
    __device__ __forceinline__ float at(const int32_t i) const
    {
        return BF16 ? __uint_as_float((uint32_t)((const uint16_t*)logits)[i] << 16) : ((const float*)logits)[i];
    }
    __device__ __forceinline__ float log_p(const float x) const { return none ? -__builtin_inff() : (x - m) - log_s; }
};

// Joins the sums and lists (of at most 64 entries) of a workgroup's W waves and writes the row's results.
template <bool BF16, bool TOP, int W>
__device__ __forceinline__ void finish_row(const Args& A, const int r, Sums a, const Top& top, const int wave, const int lane)
{
    __shared__ float4 stat[W];
    __shared__ __attribute__((aligned(16))) uint64_t best[TOP ? 64 * W : 1];
    __shared__ int n_best, places[TOP ? 64 * W : 1];
    if (TOP) {
        uint32_t known = rank_of(top.floor);
        if (2 * top.n > 3 * top.k) {                      // (a list of several tiles says more than the bound that it came in by)
            const uint32_t rk[1] = {lane < top.n ? (uint32_t)(top.list[lane] >> 32) : 0};
            int hits;
            known = bound_of(rk, top.k, hits);
        }
        if (lane == 0) atomicMax(top.bound, known);
    }
    if (lane == 0) stat[wave] = float4{a.m, a.s, a.z, 0.f};
    if (TOP) places[threadIdx.x] = 0;
    if (threadIdx.x == 0) n_best = 0;
    Row<BF16> row(A, r);
    int32_t t = -1;
    float x = 0.f;
    if (wave == 1 && lane < A.n_tokens) {                 // on their way while the others arrive
        t = A.tokens[(int64_t)r * A.n_tokens + lane];
        if (t >= 0 && t < A.vocab) x = row.at(t);
    }
    __syncthreads();
    if (TOP) {
        // What the highest of the waves' bounds leaves.
        const uint32_t least = *top.bound;
        const uint64_t key = lane < top.n ? top.list[lane] : 0;
        const uint64_t m = __ballot((uint32_t)(key >> 32) >= least && key != 0);
        if (m) {
            int at = 0;
            if (lane == 0) at = atomicAdd(&n_best, __popcll(m));
            at = __builtin_amdgcn_readfirstlane(at);
            if (m >> lane & 1) best[at + lanes_before(m)] = key;
        }
        __syncthreads();
    }
    const int n = TOP ? n_best : 0, i = threadIdx.x;
    // A key's place is the number of larger ones.  Of more than a wave's, the waves that no keys are left for count in a part of the others.
    int place = 0;
    if (TOP && n > 64) {
        const int groups = (n + 63) / 64, shares = W / groups, group = wave % groups, share = wave / groups;
        if (share < shares) {
            const uint64_t key = best[64 * group + lane];
#pragma unroll 8
            for (int j = share; j < n; j += shares) place += best[j] > key;
            atomicAdd(&places[64 * group + lane], place);
        }
        __syncthreads();
        place = places[i];
    }
    if (wave > 1 && 64 * wave >= n) return;
    a = Sums{-__builtin_inff(), 0.f, 0.f};
    float M = a.m;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, stat[w].x);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const Sums b = moved(Sums{stat[w].x, stat[w].y, stat[w].z}, finite_or_0(M));
        a.s += b.s; a.z += b.z;
    }
    a.m = M;
    row.of(a);
    if (wave == 1) {
        if (lane == 0) {
            if (A.lse) A.lse[r] = row.none ? -__builtin_inff() : row.m + row.log_s;
            if (A.entropy) A.entropy[r] = row.none ? 0.f : row.log_s - a.z / a.s;
        }
        for (int j = lane; j < A.n_tokens; j += 64) {
            if (j >= 64) {
                t = A.tokens[(int64_t)r * A.n_tokens + j];
                if (t >= 0 && t < A.vocab) x = row.at(t);
            }
            A.logprob[(int64_t)r * A.n_tokens + j] = t >= 0 && t < A.vocab ? row.log_p(x) : 0.f;
        }
    }
    if (!TOP) return;
    if (64 * wave < n) {
        const uint64_t key = i < n ? best[i] : 0;
        if (n <= 64) {
#pragma unroll 8
            for (int j = 0; j < n; ++j) place += best[j] > key;
        }
        if (i < n && place < A.n_top) {
            A.top_idx[(int64_t)r * A.n_top + place] = (int32_t)~(uint32_t)key;
            if (A.top_logprob) A.top_logprob[(int64_t)r * A.n_top + place] = row.log_p(value_of((uint32_t)(key >> 32)));
        }
    }
    if (n < A.n_top && wave == 0) {                       // the other places go to the lowest indices that have none
        uint64_t taken = 0;
        for (int j = 0; j < n; ++j) {
            const uint32_t k = ~(uint32_t)best[j];
            taken |= k < 64 ? uint64_t(1) << k : 0;
        }
        const bool free = !(taken >> lane & 1);
        const int fill = n + lanes_before(__ballot(free));
        if (free && fill < A.n_top) {
            A.top_idx[(int64_t)r * A.n_top + fill] = lane;
            if (A.top_logprob) A.top_logprob[(int64_t)r * A.n_top + fill] = row.log_p(row.at(lane));
        }
    }
}

// Workgroup (part, row): its W waves take the row's tiles part * W * tiles + wave, + W, ..
template <bool BF16, bool TOP, int W>
__global__ __launch_bounds__(64 * W) void sk_logprobs_scan(const Args A)
{
    __shared__ uint64_t lists[W][kList];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = blockIdx.x / A.parts, part = blockIdx.x - r * A.parts;
    constexpr int EL = BF16 ? 2 : 4, V = 16 / EL;
    const uintptr_t row = (uintptr_t)A.logits + (uintptr_t)((int64_t)r * A.row_stride * EL);
    const int skip = (int)(row & 15) / EL;
    const int64_t total = (int64_t)skip + A.vocab;
    Sums a = {-__builtin_inff(), 0.f, 0.f};
    Top top;
    __shared__ uint32_t bound;
    if (TOP) {
        top.init(lists[wave], &bound, A.n_top);
        if (threadIdx.x == 0) bound = 0;
        __syncthreads();
    }
    for (int i = 0; i < A.tiles; ++i) {
        const int tile = (part * A.tiles + i) * W + wave;
        if ((int64_t)tile * kTile >= total) break;
        float x[32];
        load_tile<BF16>((const unsigned char*)(row & ~(uintptr_t)15), skip, total, tile, lane, x);
        float most[4];                                    // maxima of eight logits each
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            most[e] = x[8 * e];
#pragma unroll
            for (int f = 1; f < 8; ++f) most[e] = fmaxf(most[e], x[8 * e + f]);
        }
        const float mx = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
        const float M = fmaxf(a.m, mx), Mf = finite_or_0(M);
        a = moved(a, Mf);
        a.m = M;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const float d = x[e] - Mf, w = exp_of(d);
            a.s += w;
            a.z += w * fmaxf(d, -200.f);                  // e^-200 is 0 in 32 bits: a logit of -inf adds 0 and not 0 * inf
        }
        if (TOP) {
            if (top.floor == -__builtin_inff()) {                          // the k-th largest of the lanes' maxima, if as many lanes have one
                const uint32_t rk[1] = {mx > -__builtin_inff() ? rank_of(mx) : 0};
                int hits = lanes(rk[0] != 0);
                if (hits >= top.k) top.raise(bound_of(rk, top.k, hits));
            }
            top.share(lane);
            const int32_t first = (int32_t)((int64_t)tile * kTile - skip);
            const float least = top.least(first);
            int done = 32;                                // of the 32 steps, a logit of each lane
            if (__ballot(mx >= least)) {
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    if (done < 32 || !__ballot(most[p] >= least)) continue;
#pragma unroll
                    for (int e = 8 * p; e < 8 * p + 8; ++e) {
                        const uint64_t m = __ballot(x[e] >= least);
                        if (!m) continue;
                        if (top.full()) { done = e; break; }
                        top.add(m, x[e] >= least, (uint64_t)rank_of(x[e]) << 32 | (uint32_t)~(first + V * lane + (e / V) * 64 * V + e % V));
                    }
                }
            }
            // A list that is full before the tile is through (thousands of equal logits, as a mask writes them) is cut in
            // between, and the rest of the tile read again, a logit at a time.  (Nothing of this stands behind each of the steps above:
            // a kernel of one tile runs most of its code once, from a cold instruction cache.)
            for (;;) {
#pragma clang loop unroll(disable)
                for (; done < 32 && !top.full(); ++done) {
                    const int32_t idx = first + V * lane + (done / V) * 64 * V + done % V;
                    float y = -__builtin_inff();
                    if (idx >= 0 && idx < A.vocab) y = BF16 ? __uint_as_float((uint32_t)((const uint16_t*)row)[idx] << 16) : ((const float*)row)[idx];
                    const bool takes = top.takes(y, idx);
                    top.add(__ballot(takes), takes, (uint64_t)rank_of(y) << 32 | (uint32_t)~idx);
                }
                if (top.n > 64) top.cut(lane);
                if (done == 32) break;
            }
        }
    }
    a = wave_sums(a);
    if (W == kWavesAlone || A.parts == 1) {
        finish_row<BF16, TOP, W>(A, r, a, top, wave, lane);
        return;
    }
    const int64_t slot = (int64_t)blockIdx.x * W + wave;
    if (lane == 0) A.stats[slot] = float4{a.m, a.s, a.z, 0.f};
    if (TOP) {                                            // its best in order, 0 in the places that none fills
        wave_order();
        const uint64_t key = lane < top.n ? top.list[lane] : 0;
        int place = lane < top.n ? 0 : lane;
#pragma unroll 4
        for (int j = 0; j < top.n; ++j) place += top.list[j] > key && key;
        if (place < A.n_top) A.keys[slot * A.n_top + place] = key;
    }
}

// Rows cut into several parts: one workgroup to a row joins them.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(64 * kWaves) void sk_logprobs_join(const Args A)
{
    __shared__ uint64_t lists[kWaves][kList];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = blockIdx.x, n = A.parts * kWaves;
    Sums a = {-__builtin_inff(), 0.f, 0.f};
    for (int i = threadIdx.x; i < n; i += 64 * kWaves) {
        const float4 b = A.stats[(int64_t)r * n + i];
        const float M = fmaxf(a.m, b.x), Mf = finite_or_0(M);
        const Sums p = moved(a, Mf), q = moved(Sums{b.x, b.y, b.z}, Mf);
        a = Sums{M, p.s + q.s, p.z + q.z};
    }
    a = wave_sums(a);
    Top top;
    __shared__ uint32_t bound;
    if (TOP) {
        top.init(lists[wave], &bound, A.n_top);
        if (threadIdx.x == 0) bound = 0;
        __syncthreads();
        const int64_t all = (int64_t)n * A.n_top;
        const uint64_t* keys = A.keys + (int64_t)r * all;
        constexpr int N = 8;
        for (int64_t i0 = threadIdx.x; i0 - threadIdx.x < all; i0 += N * 64 * kWaves) {
            uint64_t key[N];
#pragma unroll
            for (int j = 0; j < N; ++j) key[j] = i0 + j * 64 * kWaves < all ? keys[i0 + j * 64 * kWaves] : 0;
            if (top.floor == -__builtin_inff()) {                          // as in the scan, by the lanes' maxima
                uint32_t most[1] = {(uint32_t)(key[0] >> 32)};
#pragma unroll
                for (int j = 1; j < N; ++j) most[0] = max(most[0], (uint32_t)(key[j] >> 32));
                int hits = lanes(most[0] != 0);
                if (hits >= top.k) top.raise(bound_of(most, top.k, hits));
            }
            top.share(lane);
            auto takes = [&](const uint64_t x) { return x != 0 && top.takes(value_of((uint32_t)(x >> 32)), (int32_t)~(uint32_t)x); };
            int done = N;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const bool t = takes(key[j]);
                const uint64_t m = __ballot(t);
                if (!m) continue;
                if (top.full()) { done = j; break; }
                top.add(m, t, key[j]);
            }
            for (;;) {
#pragma clang loop unroll(disable)
                for (; done < N && !top.full(); ++done) {
                    const int64_t i = i0 + done * 64 * kWaves;
                    const uint64_t x = i < all ? keys[i] : 0;
                    const bool t = takes(x);
                    top.add(__ballot(t), t, x);
                }
                if (top.n > 64) top.cut(lane);
                if (done == N) break;
            }
        }
    }
    finish_row<BF16, TOP, kWaves>(A, r, a, top, wave, lane);
}

// How a call is cut: waves of a workgroup, workgroups to a row and tiles to a wave.
void cut_rows(const int32_t rows, const int32_t vocab, int32_t& waves, int32_t& parts, int32_t& tiles)
{
    const int64_t all = (int64_t(vocab) + 7 + kTile - 1) / kTile, groups = (all + kWaves - 1) / kWaves, rounds = (all + kWavesAlone - 1) / kWavesAlone;
    // Up to a row to a CU: a workgroup of sixteen waves takes all of it, in one launch; where its waves take several tiles each, from as many rows
    // on that parts of them would fill the device anyhow.  us in parts / alone, 5 and 20 alternatives:
    //   fp32    1 x 9,000  10.7 / 7.5, 12.0 / 9.0     200 x 9,000  12.7 / 8.7, 14.3 / 9.9     1 x 32,000  10.2 / 9.5, 12.0 / 12.4    200 x 32,000  15.5 / 11.5, 17.6 / 15.7
    //          64 x 50,257 13.1 / 13.3, 15.4 / 16.6   200 x 50,257 17.8 / 14.4, 20.6 / 17.6  128 x 128,256 21.8 / 21.2, 25.2 / 28.5  200 x 128,256 28.3 / 23.4, 33.4 / 29.4
    //   bf16   64 x 50,257 14.0 / 12.5, 16.5 / 16.5   200 x 50,257 18.9 / 13.5, 22.5 / 17.2    1 x 128,256 11.6 / 18.0, 14.4 / 25.0  200 x 128,256 27.0 / 21.5, 32.5 / 30.0
    // (300 rows are a second round: 300 x 32,000 17.2 / 20.1.)  What one group of four waves takes at once is as fast either way.
    waves = kWavesAlone; parts = 1; tiles = (int32_t)rounds;
    if (rows <= 256 && groups > 1 && rows >= 64 * (rounds - 1)) return;
    // Else a row cut in parts has a list and an end for every part, and a second launch joins them; whole, the bound of its list holds for more
    // tiles.  us with 20 alternatives, logits not in a cache (fp32, bf16), 1, 2, 4, 8, 16 parts:
    //   1,024 x 128,256   90.8  99.5  97.9  97.7 103 / 76.5 89.4 97.0 100 114       64 x 128,256   52.2 37.7 26.7 21.9 19.5 / 53.8 40.5 28.5 23.4 19.3
    //     600 x 128,256   66.3  64.9  63.8  63.2 65.8 / 67.3 59.6 64.9 66.0 72.7   1,024 x 32,000   32.4 37.3 / 32.2 38.8
    //     300 x 128,256   58.0  46.3  40.4  40.1 39.8 / 59.2 49.0 40.2 41.5 42.9
    // So whole from three rows to a CU, one for rows of at most two workgroups' work (500 x 16,384, 5: 14.2 -> 12.1), and else about 2,048
    // workgroups, eight to a CU.
    waves = kWaves;
    int64_t t = rows >= (groups <= 2 ? 256 : 768) ? groups : (rows * groups + 2047) / 2048;
    t = t < 1 ? 1 : t > groups ? groups : t;
    parts = int32_t((groups + t - 1) / t);
    tiles = int32_t((groups + parts - 1) / parts);
}

size_t stats_bytes(const int32_t rows, const int32_t parts) { return (size_t)rows * parts * kWaves * sizeof(float4); }

}  // namespace

extern "C" {

size_t sk_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t n_top)
{
    if (rows <= 0 || vocab < 1 || n_top < 0 || n_top > SK_LOGPROBS_MAX_TOP) return 0;
    int32_t waves, parts, tiles;
    cut_rows(rows, vocab, waves, parts, tiles);
    return parts == 1 ? 0 : stats_bytes(rows, parts) + (size_t)rows * parts * kWaves * n_top * sizeof(uint64_t);
}

int sk_logprobs(const void* logits, int dtype, int32_t rows, int32_t vocab, int64_t row_stride, const int32_t* tokens, int32_t n_tokens,
                int32_t n_top, void* workspace, size_t workspace_bytes, float* logprob, float* lse, float* entropy,
                int32_t* top_idx, float* top_logprob, void* hip_stream)
{
    if (dtype != SK_F32 && dtype != SK_BF16) return SK_E_DTYPE;
    if (rows < 0 || rows > SK_LOGPROBS_MAX_ROWS || vocab < 1 || vocab > SK_LOGPROBS_MAX_VOCAB || row_stride < vocab) return SK_E_INVAL;
    if (n_tokens < 0 || n_top < 0 || n_top > SK_LOGPROBS_MAX_TOP || n_top > vocab) return SK_E_INVAL;
    if (rows == 0) return SK_OK;
    if (!logits || (n_tokens > 0 && (!tokens || !logprob)) || (n_top > 0 && !top_idx)) return SK_E_INVAL;
    if ((uintptr_t)logits % (dtype == SK_BF16 ? 2 : 4) || (uintptr_t)workspace % 16) return SK_E_INVAL;
    Args A;
    int32_t waves;
    cut_rows(rows, vocab, waves, A.parts, A.tiles);
    const size_t need = sk_logprobs_workspace_bytes(rows, vocab, n_top);
    if (need > 0 && !workspace) return SK_E_INVAL;
    if (workspace_bytes < need) return SK_E_WORKSPACE;
    A.logits = logits; A.row_stride = row_stride; A.vocab = vocab; A.n_tokens = n_tokens; A.n_top = n_top;
    A.tokens = tokens; A.logprob = logprob; A.lse = lse; A.entropy = entropy; A.top_idx = top_idx; A.top_logprob = top_logprob;
    A.stats = (float4*)workspace;
    A.keys = (uint64_t*)((unsigned char*)workspace + stats_bytes(rows, A.parts));
    hipStream_t st = (hipStream_t)hip_stream;
    const dim3 grid((unsigned)rows * (unsigned)A.parts);
#define SK_LOGPROBS(kernel, grid, waves, ...)                                                                       \
    do {                                                                                                            \
        const dim3 block(64 * (waves));                                                                             \
        if (dtype == SK_BF16) {                                                                                     \
            if (n_top > 0) hipLaunchKernelGGL((kernel<true, true __VA_OPT__(,) __VA_ARGS__>), grid, block, 0, st, A);          \
            else hipLaunchKernelGGL((kernel<true, false __VA_OPT__(,) __VA_ARGS__>), grid, block, 0, st, A);                   \
        } else {                                                                                                    \
            if (n_top > 0) hipLaunchKernelGGL((kernel<false, true __VA_OPT__(,) __VA_ARGS__>), grid, block, 0, st, A);         \
            else hipLaunchKernelGGL((kernel<false, false __VA_OPT__(,) __VA_ARGS__>), grid, block, 0, st, A);                  \
        }                                                                                                           \
    } while (0)
    if (waves == kWavesAlone) SK_LOGPROBS(sk_logprobs_scan, grid, kWavesAlone, kWavesAlone);
    else SK_LOGPROBS(sk_logprobs_scan, grid, kWaves, kWaves);
    if (A.parts > 1) SK_LOGPROBS(sk_logprobs_join, dim3(rows), kWaves);
#undef SK_LOGPROBS
    return sk_status_of((int)hipGetLastError());
}

}  // extern "C"
