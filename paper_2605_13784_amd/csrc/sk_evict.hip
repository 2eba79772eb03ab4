// Eviction of the tokens with the lowest accumulated weight (include/sk.h: sk_session_evict_lowest), gfx950.
//
// First what leaves: per list (a KV head, or all together) the n-th smallest sum, as a number of 32 bits that orders like the float,
// found by histograms of its leading bits and, among the few that share those, by counting lanes; then the indices of what
// stays are written in order.  One launch with a workgroup to a list where the list fits LDS; longer lists are cut among workgroups, in
// five launches.  Then the move: a workgroup takes 64 consecutive slots of one KV head, reads what goes there and writes it.  K and V
// bytes are copied, never computed with.
// Bound: the selection by latency, the move by HBM (what stays is read once and written once; V, transposed in groups of 16
// tokens, is read in whole groups).
//
// Where the tokens go.  If the free list has a block for every one that would be written, what stays goes there and the old blocks
// are given back: nothing that is read is written.  If not, stretches of what stays go to the workspace in their new order and
// from there to their places, a launch each: a token never moves to a higher slot, so that no stretch writes over what a later one reads.
// (Moving in place in one launch was built and measured: workgroups that read 64 slots, say so, and write when those before them whose
// tokens lie there have said so.  Its three device-scope round trips for each workgroup, one behind the other, cost more than the
// way by the workspace: 131,072 tokens to 65,536 370 us, 14,800 of 64 dims to 11,303 37 us; to free blocks 130 and 10 us.)
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/sk.h"
#include "sk_internal.h"
#include "sk_order.h"

namespace {

using namespace sk_order;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kSlots = 64;            // slots that a workgroup of the move takes
constexpr int kSelectThreads = 1024;
constexpr int kBinBits = 13, kBins = 1 << kBinBits;       // leading bits that a histogram counts
constexpr int kKept = 30 * 1024;      // sums that one workgroup keeps in LDS; longer lists are cut into
constexpr int kPart = 4096, kPartThreads = 256;           // parts of this many, whose histograms have
constexpr int kPartBits = 11, kPartBins = 1 << kPartBits; // fewer bins to clear, merge and look through
constexpr int kFew = 256;             // sums that one wave finishes the search among

struct Args {
    sk_geom g;
    int32_t tbl_off, n_lists, per_head;
    int32_t win, frozen;
    int32_t len, new_len, first;      // storage indices, see sk_evict
    int32_t n_evict, n_cand;
    int32_t blk0, n_blk, n_fresh;
    const float* in;
    int64_t in_stride;
    float* out;
    int64_t out_stride;
    const int32_t* table_new;         // pinned
    int32_t* tables_rw;
    unsigned char* kv_rw;
    // scratch
    int32_t* keep;                    // [n_lists][new_len - win]: what stays, counted from win, ascending
    float* sums;                      // per_head == 0: [n_cand]
    int32_t* old_table;               // n_fresh > 0: the n_blk entries and those behind them that are read, as they were
    float* old_sums;                  // out == in: a copy of in's entries behind the frozen ones, [Hkv][len - win]
    int32_t n_old;
    unsigned char* staged;            // chunk by chunk and head by head K and V as they will lie, or null: to their places at once
    int32_t chunk0;                   // first chunk of a launch
    // ... of lists that are cut into parts
    int32_t n_parts;
    uint32_t* histogram;              // [n_lists][kPartBins]
    uint32_t* some;                   // [n_lists][n_cand]: sums that share the leading bits of the n-th smallest
    uint32_t *n_some, *emitting;      // [n_lists] each: how many; parts that have started to write what stays
    uint64_t* counted;                // [n_lists][n_parts]: of a part, sums below the n-th smallest, and equal ones + 1
    uint2* found;                     // [n_lists]: the n-th smallest, and how many that equal it leave
    uint32_t* clear;                  // n_clear words that are cleared: the counts above
    int64_t n_clear;
};

// Orders sums as unsigned numbers, of which the lowest leave first; a NaN is larger than any.  (The complement of none of them is 0.)
__device__ __forceinline__ uint32_t place_of(const float x) { return x != x ? 0xfffffffeu : rank_of(x); }

// Exclusive sum over the workgroup's threads.
template <int WAVES>
__device__ __forceinline__ int before_me(const int x, int* waves)
{
    const int s = wave_running_sum(x), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int base = 0;
    for (int w = 0; w < WAVES; ++w) base += w < wave ? waves[w] : 0;
    return base + s - x;
}

// Clears what the launches behind count with, puts the table in place, and lists the newest, which all stay: workgroup i of n.
__device__ __forceinline__ void prepare(const Args& A, const int i, const int n)
{
    const int64_t first = (int64_t)i * blockDim.x + threadIdx.x, step = (int64_t)n * blockDim.x;
    for (int64_t k = first; k < A.n_clear; k += step) A.clear[k] = 0;
    if (A.old_sums) {
        const int64_t m = A.len - A.win;
        for (int64_t k = first; k < m * A.g.Hkv; k += step) A.old_sums[k] = A.in[k / m * A.in_stride + A.frozen + k % m];
    }
    if (A.n_fresh > 0) {
        int32_t* table = A.tables_rw + A.tbl_off + A.blk0;
        for (int64_t k = first; k < A.n_old; k += step) {
            A.old_table[k] = table[k];
            if (k < A.n_blk) table[k] = A.table_new[k];
        }
    }
    const int64_t kept = A.new_len - A.win, newest = kept - (A.n_cand - A.n_evict);
    for (int64_t k = first; k < newest * A.n_lists; k += step) {
        const int64_t list = k / newest, j = A.n_cand - A.n_evict + k % newest;
        A.keep[list * kept + j] = (int32_t)(j + A.n_evict);
    }
}

__device__ __forceinline__ const float* sums_of(const Args& A, const int list)
{
    return A.per_head ? A.in + list * A.in_stride + A.frozen : A.sums;
}

struct Search {
    uint32_t bins[kBins], few[kFew];
    int waves[kSelectThreads / 64];
    uint32_t bin, lowest, highest;
    int before, count, n_few, left;
};

// The bin in which the left-th smallest lies, from the counts of the bins in LDS, BINS / THREADS consecutive ones to a thread;
// `before`: how many lie below it.
template <int THREADS, int BINS>
__device__ __forceinline__ void find_bin(const uint32_t* bins, const int left, int* waves, uint32_t& bin, int& before, int& count)
{
    constexpr int own = BINS / THREADS;
    u32x4 n[own / 4];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < own / 4; ++k) { n[k] = ((const u32x4*)bins)[threadIdx.x * (own / 4) + k]; mine += n[k].x + n[k].y + n[k].z + n[k].w; }
    int b = before_me<THREADS / 64>(mine, waves);
    if (b < left && left <= b + mine) {
#pragma unroll
        for (int k = 0; k < own; ++k) {
            const int m = n[k / 4][k % 4];
            if (b < left && left <= b + m) { bin = threadIdx.x * own + k; before = b; count = m; }
            b += m;
        }
    }
    __syncthreads();
}

__device__ __forceinline__ void empty(Search& S)
{
    for (int b = threadIdx.x; b < kBins / 4; b += kSelectThreads) ((u32x4*)S.bins)[b] = u32x4{0, 0, 0, 0};
    if (threadIdx.x == 0) S.n_few = 0;
}

// The left-th smallest of 4 * n4 numbers (four at a time: keys(i); any that pad the end are as large as others at least), among those
// whose bits from `shift` on are those of `limit` (the bins are empty at the start); `left` becomes the number of those equal to it that are among the left smallest.  All threads.
template <class Keys>
__device__ __forceinline__ void search(Search& S, const Keys keys, const int n4, int shift, uint32_t& limit, int& left)
{
    const int tid = threadIdx.x, lane = tid & 63;
    while (shift > 0) {
        const int above = shift, width = shift < kBinBits ? shift : kBinBits;
        shift -= width;
        const uint32_t mask = (1u << width) - 1;
#pragma unroll 2
        for (int i = tid; i < n4; i += kSelectThreads) {
            const u32x4 x = keys(i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t b = x[e] >> shift & mask;
                if (above == 32 || x[e] >> above == limit >> above) atomicAdd(&S.bins[b], 1u);
            }
        }
        __syncthreads();
        find_bin<kSelectThreads, kBins>(S.bins, left, S.waves, S.bin, S.before, S.count);
        limit |= S.bin << shift;
        left -= S.before;
        if (shift == 0) break;
        if (S.count > kFew) {
            empty(S);
            __syncthreads();
            continue;
        }
        // few share these bits: one wave looks at all of them
#pragma unroll 2
        for (int i = tid; i < n4; i += kSelectThreads) {
            const u32x4 x = keys(i);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (x[e] >> shift == limit >> shift) S.few[atomicAdd(&S.n_few, 1)] = x[e];
        }
        __syncthreads();
        if (tid < 64) {
            constexpr int N = kFew / 64;
            uint32_t y[N];                                // complements: the largest of those are looked for
#pragma unroll
            for (int j = 0; j < N; ++j) y[j] = 64 * j + lane < S.n_few ? ~S.few[64 * j + lane] : 0;
            int hits, more = 0;
            const uint32_t t = bound_of(y, left, hits);
#pragma unroll
            for (int j = 0; j < N; ++j) more += lanes(y[j] > t);
            if (lane == 0) { S.bin = ~t; S.left = hits == left ? 0x7fffffff : left - more; }      // (all that reach t leave)
        }
        __syncthreads();
        limit = S.bin; left = S.left;
        return;
    }
}

// Whether a sum stays, by the n-th smallest; `same_before`: how many of its equals lie in front of the wave's 64.
__device__ __forceinline__ bool stays(const bool there, const uint32_t x, const uint32_t limit, const int left, int& same_before)
{
    const uint64_t eq = __ballot(there && x == limit);
    bool s = there && x > limit;
    if (eq) {
        if (there && x == limit) s = same_before + lanes_before(eq) >= left;
        same_before += __popcll(eq);
    }
    return s;
}

// One choice for all heads: the sum of the rows, head by head.  The workgroups behind those of the candidates prepare.
__global__ __launch_bounds__(256) void sk_evict_sums(const Args A)
{
    const int n_sums = (A.n_cand + 255) / 256;
    if ((int)blockIdx.x >= n_sums) { prepare(A, blockIdx.x - n_sums, gridDim.x - n_sums); return; }
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= A.n_cand) return;
    const float* in = A.in + A.frozen + i;
    float s = in[0];
#pragma unroll 8
    for (int h = 1; h < A.g.Hkv; ++h) s += in[h * A.in_stride];
    A.sums[i] = s;
}

// Workgroups 0 .. n_lists - 1: one list each, of at most kKept candidates.  The others, if there are any, prepare.
__global__ __launch_bounds__(kSelectThreads) void sk_evict_select(const Args A)
{
    __shared__ Search S;
    __shared__ uint32_t kept[kKept];
    __shared__ int n_less[kSelectThreads / 64], n_same[kSelectThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int list = blockIdx.x;
    if (list >= A.n_lists) { prepare(A, list - A.n_lists, gridDim.x - A.n_lists); return; }
    const int c = A.n_cand, n4 = (c + 3) / 4;
    const float* in = sums_of(A, list);
    empty(S);
    if (tid == 0) { S.lowest = 0xffffffffu; S.highest = 0; }
    __syncthreads();
    uint32_t hi = 0, lo = 0;              // largest, and largest complement
    for (int i0 = tid; i0 < 4 * n4; i0 += 8 * kSelectThreads) {       // (a loop's rest of single loads would be a round trip each)
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = in[i0 + e * kSelectThreads < c ? i0 + e * kSelectThreads : c - 1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = i0 + e * kSelectThreads;
            const uint32_t x = i < c ? place_of(f[e]) : 0xffffffffu;
            if (i < 4 * n4) kept[i] = x;
            if (i < c) { hi = hi > x ? hi : x; lo = lo > ~x ? lo : ~x; }
        }
    }
    hi = wave_max(hi); lo = wave_max(lo);
    if (lane == 0) { atomicMax(&S.highest, hi); atomicMin(&S.lowest, ~lo); }
    __syncthreads();
    // The bits that are looked through start where the sums differ: bins for the range that there is.  (Bins for all floats are
    // few for the octaves of real sums: the lanes of a wave queue up at them, and hundreds share one.)
    uint32_t limit = 0;
    int left = A.n_evict;
    if (left > 0) {
        const uint32_t base = S.lowest, range = S.highest - base;
        search(S, [&](const int i) { return ((const u32x4*)kept)[i] - base; }, n4, range ? 32 - __builtin_clz(range) : 0, limit, left);
        limit += base;
    }
    // what stays: a wave takes a stretch of E rows of 64
    const int E = (c + kSelectThreads - 1) / kSelectThreads, begin = wave * E * 64, end = begin + E * 64 < c ? begin + E * 64 : c;
    int less = 0, same = 0;
#pragma unroll 4
    for (int i = begin + lane; i < end; i += 64) { less += kept[i] < limit; same += kept[i] == limit; }
    less = wave_sum(less); same = wave_sum(same);
    if (lane == 0) { n_less[wave] = less; n_same[wave] = same; }
    __syncthreads();
    int same_before = 0, less_before = 0;
    for (int w = 0; w < wave; ++w) { same_before += n_same[w]; less_before += n_less[w]; }
    int at = begin - less_before - (same_before < left ? same_before : left);
    int32_t* keep = A.keep + (int64_t)list * (A.new_len - A.win);
    for (int i0 = begin + lane; i0 - lane < end; i0 += 4 * 64) {
        uint32_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = kept[i0 + 64 * e < end ? i0 + 64 * e : 0];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + 64 * e;
            const bool s = stays(i < end, x[e], limit, left, same_before);
            const uint64_t m = __ballot(s);
            if (s) keep[at + lanes_before(m)] = i;
            at += __popcll(m);
        }
    }
}

// ---- longer lists: workgroup (part, list) of 256 threads takes kPart candidates, 16 to a thread ----

__global__ __launch_bounds__(kSelectThreads) void sk_evict_prepare(const Args A) { prepare(A, blockIdx.x, gridDim.x); }

// The candidates of a part: thread t's e-th is the part's 1,024 (t / 64) + 64 e + t % 64.
__device__ __forceinline__ void load_part(const Args& A, const int list, const int part, uint32_t (&x)[kPart / kPartThreads])
{
    const float* in = sums_of(A, list);
    const int first = part * kPart + (threadIdx.x >> 6) * (kPart / 4) + (threadIdx.x & 63);
    float f[kPart / kPartThreads];
#pragma unroll
    for (int e = 0; e < kPart / kPartThreads; ++e) f[e] = in[first + 64 * e < A.n_cand ? first + 64 * e : A.n_cand - 1];
#pragma unroll
    for (int e = 0; e < kPart / kPartThreads; ++e) x[e] = first + 64 * e < A.n_cand ? place_of(f[e]) : 0xffffffffu;
}

__global__ __launch_bounds__(kPartThreads) void sk_evict_count(const Args A)
{
    __shared__ uint32_t bins[kPartBins];
    const int list = blockIdx.x % A.n_lists, part = blockIdx.x / A.n_lists;
    uint32_t x[kPart / kPartThreads];
    load_part(A, list, part, x);
    for (int b = threadIdx.x; b < kPartBins / 4; b += kPartThreads) ((u32x4*)bins)[b] = u32x4{0, 0, 0, 0};
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPart / kPartThreads; ++e) if (x[e] != 0xffffffffu) atomicAdd(&bins[x[e] >> (32 - kPartBits)], 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < kPartBins; b += kPartThreads)
        if (bins[b]) atomicAdd(&A.histogram[(int64_t)list * kPartBins + b], bins[b]);
}

// The candidates that share the leading bits of the n-th smallest.
__global__ __launch_bounds__(kPartThreads) void sk_evict_gather(const Args A)
{
    __shared__ uint32_t bins[kPartBins], some[kPart], bin;
    __shared__ int waves[kPartThreads / 64], before, count, n, at;
    const int list = blockIdx.x % A.n_lists, part = blockIdx.x / A.n_lists;
    uint32_t x[kPart / kPartThreads];
    load_part(A, list, part, x);
    if (threadIdx.x == 0) n = 0;
#pragma unroll
    for (int b = 0; b < kPartBins / 4 / kPartThreads; ++b)
        ((u32x4*)bins)[b * kPartThreads + threadIdx.x] = ((const u32x4*)(A.histogram + (int64_t)list * kPartBins))[b * kPartThreads + threadIdx.x];
    __syncthreads();
    find_bin<kPartThreads, kPartBins>(bins, A.n_evict, waves, bin, before, count);
#pragma unroll
    for (int e = 0; e < kPart / kPartThreads; ++e)
        if (x[e] >> (32 - kPartBits) == bin && x[e] != 0xffffffffu) some[atomicAdd(&n, 1)] = x[e];
    __syncthreads();
    if (threadIdx.x == 0) {
        if (n > 0) at = atomicAdd(&A.n_some[list], (uint32_t)n);
        if (part == 0) A.found[list] = uint2{bin << (32 - kPartBits), (uint32_t)(A.n_evict - before)};
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPartThreads) A.some[(int64_t)list * A.n_cand + at + i] = some[i];
}

// The n-th smallest itself, one workgroup to a list.
__global__ __launch_bounds__(kSelectThreads) void sk_evict_search(const Args A)
{
    __shared__ Search S;
    __shared__ uint32_t kept[kKept];
    const int list = blockIdx.x, n = A.n_some[list], n4 = (n + 3) / 4;
    const uint32_t* some = A.some + (int64_t)list * A.n_cand;
    uint32_t limit = A.found[list].x;
    int left = A.found[list].y;
    auto at = [&](const int i) { return i < n ? some[i] : 0xffffffffu; };
    empty(S);
    if (n <= kKept) {
        for (int i0 = threadIdx.x; i0 < 4 * n4; i0 += 4 * kSelectThreads) {
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = some[i0 + e * kSelectThreads < n ? i0 + e * kSelectThreads : n - 1];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = i0 + e * kSelectThreads;
                if (i < 4 * n4) kept[i] = i < n ? x[e] : 0xffffffffu;
            }
        }
        __syncthreads();
        search(S, [&](const int i) { return ((const u32x4*)kept)[i]; }, n4, 32 - kPartBits, limit, left);
    } else {
        __syncthreads();
        search(S, [&](const int i) { return u32x4{at(4 * i), at(4 * i + 1), at(4 * i + 2), at(4 * i + 3)}; }, n4, 32 - kPartBits, limit, left);
    }
    if (threadIdx.x == 0) A.found[list] = uint2{limit, (uint32_t)left};
}

// What stays, in order: a part counts what leaves, says so, and adds up what the parts before it have said.  Parts are handed out in
// the order in which workgroups start, so each waits only for workgroups that are running and have nothing to wait for before they say it.
__global__ __launch_bounds__(kPartThreads) void sk_evict_emit(const Args A)
{
    __shared__ int ticket, n_less[kPartThreads / 64], n_same[kPartThreads / 64], less_of[kPartThreads / 64], same_of[kPartThreads / 64];
    const int list = blockIdx.x % A.n_lists, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x == 0) ticket = (int)__hip_atomic_fetch_add(&A.emitting[list], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const int part = ticket;
    uint32_t x[kPart / kPartThreads];
    load_part(A, list, part, x);
    uint32_t limit = 0;
    int left = 0;
    if (A.n_evict > 0) { limit = A.found[list].x; left = (int)A.found[list].y; }
    int less = 0, same = 0;
#pragma unroll
    for (int e = 0; e < kPart / kPartThreads; ++e) { less += x[e] < limit; same += x[e] == limit; }
    less = wave_sum(less); same = wave_sum(same);
    if (lane == 0) { n_less[wave] = less; n_same[wave] = same; }
    __syncthreads();
    uint64_t* counted = A.counted + (int64_t)list * A.n_parts;
    if (threadIdx.x == 0) {
        int l = 0, s = 0;
        for (int w = 0; w < kPartThreads / 64; ++w) { l += n_less[w]; s += n_same[w]; }
        __hip_atomic_store(&counted[part], (uint64_t)l << 32 | (uint32_t)(s + 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    less = same = 0;
    for (int p = threadIdx.x; p < part; p += kPartThreads) {
        uint64_t y;
        while ((y = __hip_atomic_load(&counted[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) == 0) __builtin_amdgcn_s_sleep(1);
        less += (int)(y >> 32); same += (int)(uint32_t)y - 1;
    }
    less = wave_sum(less); same = wave_sum(same);
    if (lane == 0) { less_of[wave] = less; same_of[wave] = same; }
    __syncthreads();
    int less_before = 0, same_before = 0;
    for (int w = 0; w < kPartThreads / 64; ++w) {
        less_before += less_of[w] + (w < wave ? n_less[w] : 0);
        same_before += same_of[w] + (w < wave ? n_same[w] : 0);
    }
    const int begin = part * kPart + wave * (kPart / 4);
    int at = begin - less_before - (same_before < left ? same_before : left);
    int32_t* keep = A.keep + (int64_t)list * (A.new_len - A.win);
#pragma unroll
    for (int e = 0; e < kPart / kPartThreads; ++e) {
        const int i = begin + 64 * e + lane;
        const bool s = stays(i < A.n_cand, x[e], limit, left, same_before);
        const uint64_t m = __ballot(s);
        if (s) keep[at + lanes_before(m)] = i;
        at += __popcll(m);
    }
}

// Writes what a workgroup holds of a chunk: thread t the pieces t, t + 256, .. of its K rows and, fp32, of its V rows; bf16, two pieces of
// dimension t % D of the 16-slot group t / D, + 256 / D, ..
template <int D, bool F32, int N>
__device__ __forceinline__ void put(const Args& A, const int head, const int t0, const int n_valid, const int64_t* to, const u32x4 (&k)[N], const u32x4 (&v)[N])
{
    constexpr int ROWB = D * (F32 ? 4 : 2), PR = ROWB / 16, VG = 256 / D;
    const int tid = threadIdx.x;
    unsigned char* dst = A.kv_rw + (int64_t)head * A.g.head_stride;
    const int s0 = t0 & (A.g.B - 1);      // (a group of 16 slots lies in one block; blocks hold whole groups)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int p = tid + 256 * i, r = p / PR;
        if (r < n_valid) {
            unsigned char* row = dst + to[r >> 4] + (int64_t)((s0 + r) & (A.g.B - 1)) * ROWB + (p % PR) * 16;
            *(u32x4*)row = k[i];
            if (F32) *(u32x4*)(row + A.g.v_off) = v[i];
        }
    }
    if constexpr (!F32) {
        const int dim = tid % D;
#pragma unroll
        for (int i = 0; i < kSlots / 16 / VG; ++i) {
            const int group = tid / D + VG * i;
            if (16 * group < n_valid) {
                unsigned char* at = dst + to[group] + A.g.v_off + ((((s0 + 16 * group) & (A.g.B - 1)) >> 4) * D + dim) * 32;
                *(u32x4*)at = v[2 * i];
                *(u32x4*)(at + 16) = v[2 * i + 1];
            }
        }
    }
}

// Workgroup (chunk, KV head) of the move.
template <int D, bool F32>
__global__ __launch_bounds__(256, F32 ? 2 : 4) void sk_evict_move(const Args A)
{
    constexpr int ROWB = D * (F32 ? 4 : 2), PR = ROWB / 16, N = kSlots * PR / 256;     // 16-byte pieces of a row, of a thread
    __shared__ int64_t from[kSlots];      // byte offset of the slot's block and KV head
    __shared__ int slot[kSlots];          // slot within that block
    __shared__ uint8_t pick[kSlots];      // bf16: which of the groups that go to this slot's one, slot within it
    __shared__ int64_t group_at[kSlots];  // bf16: byte offset of V of the groups that go to group g, from 16 g on
    __shared__ int n_groups[kSlots / 16];
    __shared__ int64_t to[kSlots / 16];   // of the four groups: byte offset of the block and KV head
    __shared__ int last_moves;
    const int tid = threadIdx.x;
    const int Hkv = A.g.Hkv;
    const int chunk = A.chunk0 + blockIdx.x / Hkv, head = blockIdx.x % Hkv;
    const int t0 = A.first + chunk * kSlots;
    const int n_valid = A.new_len - t0 < kSlots ? A.new_len - t0 : kSlots;               // slots that hold something afterwards
    const unsigned char* kv = A.g.kv + (int64_t)head * A.g.head_stride;
    const int32_t* table = A.g.tables + A.tbl_off;
    const int32_t* source = A.n_fresh > 0 ? A.old_table : table + A.blk0;                // entries from blk0 on
    const int32_t* keep = A.keep + (A.per_head ? (int64_t)head * (A.new_len - A.win) : 0);
    int src = 0;
    if (tid < kSlots) {
        const int t = t0 + (tid < n_valid ? tid : n_valid - 1);                          // (a slot behind the end: the last one's again)
        if (n_valid > 0) {
            src = t < A.win ? t : A.win + keep[t - A.win];
            from[tid] = (int64_t)source[(src >> A.g.log2B) - A.blk0] * A.g.blk_stride;
            slot[tid] = src & (A.g.B - 1);
            if (tid == n_valid - 1) last_moves = src != t;
            if (!F32) {                   // tokens of one group of 16 slots share the loads of it
                const int before = __shfl_up(src, 1, 64);
                const bool first = tid % 16 == 0 || src >> 4 != before >> 4;
                const uint64_t m = __ballot(first) >> (tid & 48) & 0xffff;
                const int g = __popcll(m & ((2u << (tid & 15)) - 1)) - 1;
                pick[tid] = (uint8_t)(g << 4 | (src & 15));
                if (first) group_at[(tid & 48) + g] = from[tid] + A.g.v_off + (int64_t)((src & (A.g.B - 1)) >> 4) * (D * 32);
                if (tid % 16 == 15) n_groups[tid >> 4] = g + 1;
            }
        }
    } else if (tid < kSlots + kSlots / 16) {
        const int t = t0 + 16 * (tid - kSlots);
        if (t < A.new_len) to[tid - kSlots] = (int64_t)table[t >> A.g.log2B] * A.g.blk_stride;
    }
    // the sums that go to these places
    float sum = 0.f;
    const float* in = A.old_sums ? A.old_sums + (int64_t)head * (A.len - A.win) - A.win : A.in + head * A.in_stride + A.frozen - A.win;    // by storage index, from win on
    if (A.out && tid < n_valid && t0 + tid >= A.win) sum = in[src];
    __syncthreads();
    // where nothing in front has left and no block is replaced, everything is in its place
    const bool moves = n_valid > 0 && (A.n_fresh > 0 || last_moves);
    u32x4 k[N], v[N];
    constexpr int VG = 256 / D;           // V^T: groups of 16 slots that the workgroup reads at once, a thread one dimension of a group
    if (moves) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = tid + 256 * i, r = p / PR;
            const unsigned char* row = kv + from[r] + (int64_t)slot[r] * ROWB + (p % PR) * 16;
            k[i] = *(const u32x4*)row;
            if (F32) v[i] = *(const u32x4*)(row + A.g.v_off);
        }
        if constexpr (!F32) {
            // A thread holds one dimension of a group: 32 bytes of each group that something comes from, kBatch groups at a time,
            // of which it picks 16 bits for each of the 16 slots.  (Which, is the same for the whole wave.)
            const int dim = tid % D;
            constexpr int kBatch = 4;
#pragma unroll
            for (int i = 0; i < kSlots / 16 / VG; ++i) {
                const int group = __builtin_amdgcn_readfirstlane(tid / D + VG * i), n = __builtin_amdgcn_readfirstlane(n_groups[group]);
                uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                const uint32_t mine = pick[16 * group + (tid & 15)];
                for (int g0 = 0; g0 < n; g0 += kBatch) {
                    typedef __attribute__((ext_vector_type(32))) uint32_t u32x32;
                    u32x32 x;
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        const int g = g0 + j < n ? g0 + j : n - 1;
                        const u32x4* p = (const u32x4*)(kv + group_at[16 * group + g] + dim * 32);
                        const u32x4 a = p[0], b = p[1];
#pragma unroll
                        for (int e = 0; e < 4; ++e) { x[8 * j + e] = a[e]; x[8 * j + 4 + e] = b[e]; }
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint32_t from_slot = __builtin_amdgcn_readlane(mine, e);
                        const uint32_t g = (from_slot >> 4) - g0;
                        if (g < kBatch) {
                            const uint32_t y = x[g * 8 + (from_slot >> 1 & 7)] >> (from_slot & 1) * 16;
                            w[e >> 1] |= e & 1 ? y << 16 : y & 0xffffu;
                        }
                    }
                }
                v[2 * i] = u32x4{w[0], w[1], w[2], w[3]};
                v[2 * i + 1] = u32x4{w[4], w[5], w[6], w[7]};
            }
        }
    }
    if (A.out) {
        float* out = A.out + head * A.out_stride + A.frozen - A.win;
        if (tid < kSlots && t0 + tid >= A.win && t0 + tid < A.len) out[t0 + tid] = sum;
        if (chunk == 0 && A.out != A.in)
            for (int j = tid; j < A.frozen; j += 256) A.out[head * A.out_stride + j] = A.in[head * A.in_stride + j];
    }
    if (!moves) return;
    if (A.staged) {
        u32x4* dst = (u32x4*)(A.staged + (int64_t)blockIdx.x * (2 * kSlots * ROWB)) + tid;
#pragma unroll
        for (int i = 0; i < N; ++i) { dst[256 * i] = k[i]; dst[256 * (N + i)] = v[i]; }
        return;
    }
    put<D, F32>(A, head, t0, n_valid, to, k, v);
}

// The chunks of a launch from the workspace to their places.
template <int D, bool F32>
__global__ __launch_bounds__(256) void sk_evict_put(const Args A)
{
    constexpr int ROWB = D * (F32 ? 4 : 2), N = kSlots * (ROWB / 16) / 256;
    __shared__ int64_t to[kSlots / 16];
    const int chunk = A.chunk0 + blockIdx.x / A.g.Hkv, head = blockIdx.x % A.g.Hkv;
    const int t0 = A.first + chunk * kSlots, n_valid = A.new_len - t0 < kSlots ? A.new_len - t0 : kSlots, last = t0 + n_valid - 1;
    if (n_valid <= 0) return;
    const int32_t* keep = A.keep + (A.per_head ? (int64_t)head * (A.new_len - A.win) : 0);
    if (A.n_fresh == 0 && (last < A.win || A.win + keep[last - A.win] == last)) return;      // (did not move, see there)
    if (threadIdx.x < kSlots / 16) {
        const int t = t0 + 16 * threadIdx.x;
        if (t < A.new_len) to[threadIdx.x] = (int64_t)A.g.tables[A.tbl_off + (t >> A.g.log2B)] * A.g.blk_stride;
    }
    const u32x4* src = (const u32x4*)(A.staged + (int64_t)blockIdx.x * (2 * kSlots * ROWB)) + threadIdx.x;
    u32x4 k[N], v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) { k[i] = src[256 * i]; v[i] = src[256 * (N + i)]; }
    __syncthreads();
    put<D, F32>(A, head, t0, n_valid, to, k, v);
}

template <class T> T* take(unsigned char*& at, int64_t n) { T* p = (T*)at; at += (size_t(n) * sizeof(T) + 255) / 256 * 256; return p; }

}  // namespace

extern "C" int sk_session_evict_lowest(sk_pool* p, int32_t id, const float* mass_in, int64_t mass_in_stride, int64_t n_evict, int64_t n_recent,
                                       int32_t per_head, float* mass_out, int64_t mass_out_stride, void* hip_stream)
{
    sk_session_view V;
    int rc = sk_view_session(p, id, &V);
    if (rc) return rc;
    const int64_t n = V.retained, Hkv = V.g.Hkv;
    if (V.device && n > 0) {
        if (!mass_in || (uintptr_t)mass_in & 3 || mass_in_stride < n) return SK_E_INVAL;
        if (mass_out && ((uintptr_t)mass_out & 3 || mass_out_stride < n ||
                         sk_rows_overlap(mass_in, mass_in_stride, mass_out, mass_out_stride, Hkv, n))) return SK_E_INVAL;
    }
    sk_evict E;
    rc = sk_evict_begin(p, id, n_evict, n_recent, &E);
    if (rc) return rc;
    Args A = {};
    int64_t chunks = 0, round = 0;
    if (V.device && n > 0) {
        A.g = V.g;
        A.tbl_off = V.tbl_off; A.per_head = per_head || Hkv == 1 ? 1 : 0; A.n_lists = A.per_head ? (int32_t)Hkv : 1;
        A.win = (int32_t)V.win; A.frozen = (int32_t)V.frozen; A.len = (int32_t)E.len; A.new_len = (int32_t)E.new_len; A.first = (int32_t)E.first;
        A.n_evict = (int32_t)E.n_evict; A.n_cand = (int32_t)E.n_cand;
        A.blk0 = (int32_t)E.blk0; A.n_blk = (int32_t)E.n_blk; A.n_fresh = (int32_t)E.n_fresh;
        A.in = mass_in; A.in_stride = mass_in_stride; A.out = mass_out; A.out_stride = mass_out_stride;
        A.table_new = E.table; A.tables_rw = E.tables_rw; A.kv_rw = E.kv_rw;
        chunks = (E.len - E.first + kSlots - 1) / kSlots;
        if (chunks < 1) chunks = 1;                       // (no token behind the frozen ones: their sums are copied)
        A.n_old = (int32_t)((E.len + V.g.B - 1) / V.g.B - E.blk0);
        unsigned char* at = V.scratch;
        A.keep = take<int32_t>(at, (int64_t)A.n_lists * (E.new_len - V.win));
        A.sums = take<float>(at, A.per_head ? 0 : E.n_cand);
        A.old_table = take<int32_t>(at, A.n_old);
        A.old_sums = mass_out == mass_in ? take<float>(at, Hkv * (E.len - V.win)) : nullptr;
        if (A.n_cand > kKept) {
            const int64_t lists = A.n_lists;
            A.n_parts = (A.n_cand + kPart - 1) / kPart;
            A.clear = A.n_some = take<uint32_t>(at, lists);
            A.emitting = take<uint32_t>(at, lists);
            A.histogram = take<uint32_t>(at, lists * kPartBins);
            A.counted = take<uint64_t>(at, lists * A.n_parts);
            A.n_clear = (uint32_t*)at - A.clear;
            A.some = take<uint32_t>(at, lists * A.n_cand);
            A.found = take<uint2>(at, lists);
        }
        round = chunks;
        if (E.n_fresh < E.n_blk && n_evict > 0) {         // by way of the workspace, as many chunks at a time as it holds
            A.staged = at;
            const int64_t chunk_bytes = Hkv * 2 * kSlots * V.g.d * V.g.elem;
            round = (int64_t)(V.scratch_bytes - (size_t)(at - V.scratch)) / chunk_bytes;
            if (at > V.scratch + V.scratch_bytes || round < 1) return SK_E_WORKSPACE;
        }
        if ((size_t)(at - V.scratch) > V.scratch_bytes || chunks * Hkv >= (int64_t(1) << 31)) return SK_E_WORKSPACE;
    }
    // (nothing to evict and no sums to copy: nothing to do on the device)
    const bool runs = V.device && n > 0 && (n_evict > 0 || (mass_out && mass_out != mass_in));
    int launches = 1;
    hipStream_t st = (hipStream_t)hip_stream;
    if (sk_injected(p, SK_SITE_EVICT_SELECT)) return SK_E_HIP;
    if (runs) {
        const int64_t work = A.n_clear + A.n_old + A.n_lists * (E.len - V.win - E.n_cand) + (A.old_sums ? Hkv * (E.len - V.win) : 0);
        const unsigned others = (unsigned)(work / (8 * kSelectThreads) < 63 ? work / (8 * kSelectThreads) + 1 : 64);
        const bool sums = !A.per_head && A.n_cand > 0;    // (a launch that the preparation goes along with)
        if (sums) {
            hipLaunchKernelGGL(sk_evict_sums, dim3((unsigned)((A.n_cand + 255) / 256) + others * (kSelectThreads / 256)), dim3(256), 0, st, A);
            ++launches;
        }
        if (A.n_parts == 0) hipLaunchKernelGGL(sk_evict_select, dim3(A.n_lists + (sums ? 0 : others)), dim3(kSelectThreads), 0, st, A);
        else {
            const dim3 parts((unsigned)A.n_lists * (unsigned)A.n_parts);
            if (!sums) { hipLaunchKernelGGL(sk_evict_prepare, dim3(others), dim3(kSelectThreads), 0, st, A); ++launches; }
            if (n_evict > 0) {
                hipLaunchKernelGGL(sk_evict_count, parts, dim3(kPartThreads), 0, st, A);
                hipLaunchKernelGGL(sk_evict_gather, parts, dim3(kPartThreads), 0, st, A);
                hipLaunchKernelGGL(sk_evict_search, dim3(A.n_lists), dim3(kSelectThreads), 0, st, A);
            }
            hipLaunchKernelGGL(sk_evict_emit, parts, dim3(kPartThreads), 0, st, A);
            launches += n_evict > 0 ? 3 : 0;
        }
        const int e = (int)hipGetLastError();
        sk_evict_listed(p, E, hip_stream);
        if (e) {      // (an error that an earlier call left behind shows up here too, with the kernel on the stream)
            sk_evict_undo(p, E, hip_stream);
            return sk_note_hip_error(e);
        }
    }
    int e = 0;
    bool moved = false;
    auto failed = [&] { return sk_injected(p, SK_SITE_EVICT_MOVE) ? (int)hipErrorUnknown : 0; };
    if (!runs) e = failed();
    for (int64_t c = 0; runs && c < chunks && !e; c += round) {
        const dim3 grid((unsigned)((chunks - c < round ? chunks - c : round) * Hkv)), block(256);
        A.chunk0 = (int32_t)c;
#define SK_EVICT(kernel)                                                                                            \
    if ((e = failed()) == 0) {                                                                                      \
        if (A.g.elem == 4) {                                                                                        \
            if (A.g.d == 128) hipLaunchKernelGGL((kernel<128, true>), grid, block, 0, st, A);                       \
            else hipLaunchKernelGGL((kernel<64, true>), grid, block, 0, st, A);                                     \
        } else {                                                                                                    \
            if (A.g.d == 128) hipLaunchKernelGGL((kernel<128, false>), grid, block, 0, st, A);                      \
            else hipLaunchKernelGGL((kernel<64, false>), grid, block, 0, st, A);                                    \
        }                                                                                                           \
        ++launches;                                                                                                 \
        e = (int)hipGetLastError();                                                                                 \
        moved = true;                                                                                               \
    }
        SK_EVICT(sk_evict_move)
        if (A.staged && !e) SK_EVICT(sk_evict_put)
#undef SK_EVICT
    }
    if (e) {
        if (moved && A.old_sums)                          // sums in place: as they were
            for (int64_t h = 0; h < Hkv; ++h)
                (void)hipMemcpyAsync(mass_out + h * mass_out_stride + V.frozen, A.old_sums + h * (E.len - V.win), size_t(E.len - V.win) * 4, hipMemcpyDeviceToDevice, st);
        if (runs) sk_evict_undo(p, E, hip_stream);
        return sk_note_hip_error(e);
    }
    for (; runs && launches > 0; --launches) sk_count_launch(p);
    sk_evict_end(p, E);
    return SK_OK;
}
