// Eviction of the tokens with the lowest accumulated weight (include/sk.h: sk_session_evict_lowest), gfx950.
//
// Two launches.  The first finds, per list (a KV head, or all together), the n-th smallest sum as a number of 32 bits that orders
// like the float, eleven bits at a time by histograms, and writes the indices of what stays in order.  The second moves: a
// workgroup takes 64 consecutive slots of one KV head, reads what goes there and writes it.  K and V bytes are copied, never computed with.
// Bound: the selection by round trips to the L2 (a workgroup for each list), the move by HBM (what stays is read once and written
// once; V, transposed in groups of 16 tokens, is read in whole groups).
//
// Moving in place.  A token never moves to a higher slot.  A workgroup first reads all that it will write, then says so, and writes
// once those before it, whose tokens lie in its 64 slots, have said so too.  Workgroups take their slots in the order in which they
// start (a counter), so everyone waits only for workgroups that are running already and wait for nobody in order to read:
// every wait ends.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/sk.h"
#include "sk_internal.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kSlots = 64;            // slots that a workgroup of the move takes
constexpr int kBins = 2048;
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

struct Args {
    sk_geom g;
    int32_t tbl_off, n_lists, per_head, in_place;
    int32_t win, frozen;
    int32_t len, new_len, first;      // storage indices, see sk_evict
    int32_t n_evict, n_cand;
    int32_t blk0, n_blk, n_fresh;
    int32_t n_chunks;                 // groups of kSlots slots from `first` to len
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
    uint32_t* started;                // [Hkv]
    uint32_t* has_read;               // [Hkv][n_chunks]
    int32_t n_old;
};

__device__ __forceinline__ uint32_t rank_of(const float x)      // orders floats as unsigned numbers; -0 is +0, NaN the largest
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return x != x ? 0xffffffffu : u ^ (uint32_t)((int32_t)u >> 31 | INT32_MIN);
}

__device__ __forceinline__ int lanes_before(const uint64_t m)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// Exclusive sum over the workgroup's threads; `all` receives the total.
__device__ __forceinline__ int before_me(const int x, int& all, int* waves /*[kSelectWaves]*/)
{
    int s = x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) { const int y = __shfl_up(s, i, 64); s += lane >= i ? y : 0; }
    __syncthreads();
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int base = 0;
    all = 0;
    for (int w = 0; w < kSelectWaves; ++w) { base += w < wave ? waves[w] : 0; all += waves[w]; }
    return base + s - x;
}

// Workgroups 0 .. n_lists - 1: one list each.  The others clear what the move counts with, and put the table in place.
__global__ __launch_bounds__(kSelectThreads) void sk_evict_select(const Args A)
{
    __shared__ int bins[kBins];
    __shared__ int waves[kSelectWaves], found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int list = blockIdx.x;
    if (list >= A.n_lists) {
        const int64_t i0 = (int64_t)(list - A.n_lists) * kSelectThreads + tid, step = (int64_t)(gridDim.x - A.n_lists) * kSelectThreads;
        for (int64_t i = i0; i < (int64_t)A.g.Hkv * (A.n_chunks + 1); i += step) A.started[i] = 0;      // (has_read lies behind it)
        if (A.n_fresh > 0) {
            int32_t* table = A.tables_rw + A.tbl_off + A.blk0;
            for (int64_t i = i0; i < A.n_old; i += step) {
                A.old_table[i] = table[i];
                if (i < A.n_blk) table[i] = A.table_new[i];
            }
        }
        return;
    }
    const int c = A.n_cand;
    const float* in = A.in + list * A.in_stride + A.frozen;
    if (!A.per_head) {
        for (int i = tid; i < c; i += kSelectThreads) {
            float s = in[i];
            for (int h = 1; h < A.g.Hkv; ++h) s += in[h * A.in_stride + i];
            A.sums[i] = s;
        }
        in = A.sums;
        __syncthreads();
    }
    // the n_evict-th smallest: `prefix` its leading bits, `left` its place among the sums that share them
    uint32_t prefix = 0;
    int left = A.n_evict;
    if (A.n_evict > 0) {
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
            for (int b = tid; b < kBins; b += kSelectThreads) bins[b] = 0;
            __syncthreads();
            for (int i0 = tid; i0 < c; i0 += 4 * kSelectThreads) {
                float x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) x[u] = i0 + u * kSelectThreads < c ? in[i0 + u * kSelectThreads] : 0.f;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t r = rank_of(x[u]);
                    const bool in_it = i0 + u * kSelectThreads < c && (pass == 0 || r >> (shift + width) == prefix >> (shift + width));
                    const int b = (int)(r >> shift & ((1u << width) - 1));
                    // (sums that are all the same, zeros above all, would queue up at one counter)
                    const uint64_t who = __ballot(in_it);
                    if (!who) continue;
                    const int one = __shfl(b, __ffsll((unsigned long long)who) - 1, 64);
                    if (__ballot(in_it && b == one) == who) { if (lane == 0) atomicAdd(&bins[one], __popcll(who)); }
                    else if (in_it) atomicAdd(&bins[b], 1);
                }
            }
            __syncthreads();
            int all;
            const int x0 = bins[2 * tid], x1 = bins[2 * tid + 1];
            const int at = before_me(x0 + x1, all, waves);
            if (at < left && left <= at + x0) { found[0] = 2 * tid; found[1] = at; }
            else if (at + x0 < left && left <= at + x0 + x1) { found[0] = 2 * tid + 1; found[1] = at + x0; }
            __syncthreads();
            prefix |= (uint32_t)found[0] << shift;
            left -= found[1];
            __syncthreads();
        }
    }
    // What stays: each wave a stretch of the candidates; of the sums that equal the n_evict-th smallest the first `left` leave.
    const bool none = A.n_evict == 0;
    const int stretch = ((c + kSelectWaves - 1) / kSelectWaves + 63) & ~63;
    const int a = wave * stretch < c ? wave * stretch : c, b = a + stretch < c ? a + stretch : c;
    int less = 0, same = 0;
    for (int i = a; i < b; i += 64) {
        const bool in_it = i + lane < b;
        const uint32_t r = in_it ? rank_of(in[i + lane]) : 0xffffffffu;
        less += __popcll(__ballot(in_it && r < prefix));
        same += __popcll(__ballot(in_it && r == prefix));
    }
    __shared__ int n_less[kSelectWaves], n_same[kSelectWaves];
    if (lane == 0) { n_less[wave] = less; n_same[wave] = same; }
    __syncthreads();
    int same_before = 0, less_before = 0;
    for (int w = 0; w < wave; ++w) { same_before += n_same[w]; less_before += n_less[w]; }
    if (none) { same_before = less_before = 0; left = 0; }
    int at = a - (none ? 0 : less_before + (same_before < left ? same_before : left));
    int32_t* keep = A.keep + (int64_t)list * (A.new_len - A.win);
    for (int i = a; i < b; i += 64) {
        const bool in_it = i + lane < b;
        const uint32_t r = in_it ? rank_of(in[i + lane]) : 0;
        const uint64_t eq = __ballot(in_it && r == prefix);
        const bool stays = in_it && (none || r > prefix || (r == prefix && same_before + lanes_before(eq) >= left));
        const uint64_t m = __ballot(stays);
        if (stays) keep[at + lanes_before(m)] = i + lane;
        at += __popcll(m);
        same_before += __popcll(eq);
    }
    for (int i = c - A.n_evict + tid; i < A.new_len - A.win; i += kSelectThreads) keep[i] = i + A.n_evict;      // the newest
}

__device__ __forceinline__ void used(u32x4& x) { asm volatile("" : "+v"(x)); }

// Workgroup (chunk, KV head) of the move.
template <int D, bool F32>
__global__ __launch_bounds__(256) void sk_evict_move(const Args A)
{
    constexpr int ROWB = D * (F32 ? 4 : 2), PR = ROWB / 16, N = kSlots * PR / 256;     // 16-byte pieces of a row, of a thread
    __shared__ int64_t from[kSlots];      // byte offset of the slot's block and KV head
    __shared__ int slot[kSlots];          // slot within that block
    __shared__ int64_t to[kSlots / 16];   // of the four groups: byte offset of the block and KV head
    __shared__ int last_moves, ticket;
    const int tid = threadIdx.x;
    const int Hkv = A.g.Hkv;
    int chunk = blockIdx.x / Hkv;
    const int head = blockIdx.x - chunk * Hkv;
    if (A.in_place) {
        if (tid == 0) ticket = (int)__hip_atomic_fetch_add(&A.started[head], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        chunk = ticket;
    }
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
        }
    } else if (tid < kSlots + kSlots / 16) {
        const int t = t0 + 16 * (tid - kSlots);
        if (t < A.new_len) to[tid - kSlots] = (int64_t)table[t >> A.g.log2B] * A.g.blk_stride;
    }
    // the sums that go to these places
    float sum = 0.f;
    const float* in = A.in + head * A.in_stride + A.frozen - A.win;                      // by storage index, from win on
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
            const int dim = tid % D;
#pragma unroll
            for (int i = 0; i < kSlots / 16 / VG; ++i) {
                const int group = tid / D + VG * i;
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int r = 16 * group + e;
                    const uint32_t x = *(const uint16_t*)(kv + from[r] + A.g.v_off + ((slot[r] >> 4) * D + dim) * 32 + (slot[r] & 15) * 2);
                    w[e >> 1] = e & 1 ? w[e >> 1] | x << 16 : x;
                }
                v[2 * i] = u32x4{w[0], w[1], w[2], w[3]};
                v[2 * i + 1] = u32x4{w[4], w[5], w[6], w[7]};
            }
        }
    }
    if (A.in_place) {
        // all of it has arrived: say so, and wait for those whose tokens lie in these slots
#pragma unroll
        for (int i = 0; i < N; ++i) if (moves) { used(k[i]); used(v[i]); }
        asm volatile("" : "+v"(sum));
        __syncthreads();
        uint32_t* flags = A.has_read + (int64_t)head * A.n_chunks;
        if (tid == 0) __hip_atomic_store(&flags[chunk], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int back = (A.n_evict + kSlots - 1) / kSlots;
        for (int f = (chunk > back ? chunk - back : 0) + tid; f < chunk; f += 256)
            while (__hip_atomic_load(&flags[f], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0) __builtin_amdgcn_s_sleep(1);
        __syncthreads();
    }
    if (A.out) {
        float* out = A.out + head * A.out_stride + A.frozen - A.win;
        if (tid < kSlots && t0 + tid >= A.win && t0 + tid < A.len) out[t0 + tid] = sum;
        if (chunk == 0 && A.out != A.in)
            for (int j = tid; j < A.frozen; j += 256) A.out[head * A.out_stride + j] = A.in[head * A.in_stride + j];
    }
    if (!moves) return;
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
    int64_t chunks = 0;
    if (V.device && n > 0) {
        A.g = V.g;
        A.tbl_off = V.tbl_off; A.per_head = per_head ? 1 : 0; A.n_lists = per_head ? (int32_t)Hkv : 1;
        A.win = (int32_t)V.win; A.frozen = (int32_t)V.frozen; A.len = (int32_t)E.len; A.new_len = (int32_t)E.new_len; A.first = (int32_t)E.first;
        A.n_evict = (int32_t)E.n_evict; A.n_cand = (int32_t)E.n_cand;
        A.blk0 = (int32_t)E.blk0; A.n_blk = (int32_t)E.n_blk; A.n_fresh = (int32_t)E.n_fresh;
        A.in = mass_in; A.in_stride = mass_in_stride; A.out = mass_out; A.out_stride = mass_out_stride;
        A.in_place = E.n_fresh < E.n_blk || mass_out == mass_in;
        A.table_new = E.table; A.tables_rw = E.tables_rw; A.kv_rw = E.kv_rw;
        chunks = (E.len - E.first + kSlots - 1) / kSlots;
        if (chunks < 1) chunks = 1;                       // (no token behind the frozen ones: their sums are copied)
        A.n_chunks = (int32_t)chunks;
        A.n_old = (int32_t)((E.len + V.g.B - 1) / V.g.B - E.blk0);
        unsigned char* at = E.scratch;
        A.keep = take<int32_t>(at, (int64_t)A.n_lists * (E.new_len - V.win));
        A.sums = take<float>(at, A.per_head ? 0 : E.n_cand);
        A.old_table = take<int32_t>(at, A.n_old);
        A.started = take<uint32_t>(at, Hkv * (chunks + 1));
        A.has_read = A.started + Hkv;
        if ((size_t)(at - E.scratch) > E.scratch_bytes || chunks * Hkv >= (int64_t(1) << 31)) return SK_E_WORKSPACE;
    }
    // (nothing to evict and no sums to copy: nothing to do on the device)
    const bool runs = V.device && n > 0 && (n_evict > 0 || (mass_out && mass_out != mass_in));
    hipStream_t st = (hipStream_t)hip_stream;
    if (sk_injected(p, SK_SITE_EVICT_SELECT)) return SK_E_HIP;
    if (runs) {
        const int64_t others = (Hkv * (chunks + 1) + A.n_old) / (8 * kSelectThreads) + 1;
        hipLaunchKernelGGL(sk_evict_select, dim3((unsigned)(A.n_lists + (others < 64 ? others : 64))), dim3(kSelectThreads), 0, st, A);
        const int e = (int)hipGetLastError();
        sk_evict_listed(p, E, hip_stream);
        if (e) {      // (an error that an earlier call left behind shows up here too, with the kernel on the stream)
            sk_evict_undo(p, E, hip_stream);
            return sk_note_hip_error(e);
        }
        sk_count_launch(p);
    }
    int e = sk_injected(p, SK_SITE_EVICT_MOVE) ? (int)hipErrorUnknown : 0;
    if (runs && !e) {
        const dim3 grid((unsigned)(chunks * Hkv)), block(256);
        if (A.g.elem == 4) {
            if (A.g.d == 128) hipLaunchKernelGGL((sk_evict_move<128, true>), grid, block, 0, st, A);
            else hipLaunchKernelGGL((sk_evict_move<64, true>), grid, block, 0, st, A);
        } else {
            if (A.g.d == 128) hipLaunchKernelGGL((sk_evict_move<128, false>), grid, block, 0, st, A);
            else hipLaunchKernelGGL((sk_evict_move<64, false>), grid, block, 0, st, A);
        }
        e = (int)hipGetLastError();
    }
    if (e) {
        if (runs) sk_evict_undo(p, E, hip_stream);
        return sk_note_hip_error(e);
    }
    if (runs) sk_count_launch(p);
    sk_evict_end(p, E);
    return SK_OK;
}
