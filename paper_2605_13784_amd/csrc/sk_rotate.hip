// Position rotation for gfx950: q and k turned by their tokens' positions on the way into the cache (sk_session_append_rotated,
// sk_batch_step_rotated) or beside it (sk_rotate), and cached keys turned on by a difference of positions (sk_session_shift).
// The mathematics: sk_turn.h.
#include <hip/hip_runtime.h>
#include <cmath>
#include <cstring>

#include "../../include/sk.h"
#include "sk_internal.h"
#include "sk_turn.h"

namespace {

using namespace sk_turn;

// ---- rows beside the cache --------------------------------------------------------------------------

// Workgroup `wg` of those that turn [n_tok][n_heads][D] x into y: a stretch of tokens and HEADS heads, for which a thread forms its
// sines and cosines once.  A thread has eight pairs, both halves of each: nothing is exchanged, and a row is read and written in whole lines.
// Bound: memory for long calls (4,096 tokens of 32/8 heads of 128: 84 MB in 14.5 us, 5.8 TB/s with the last-level cache's help), the launch and one round trip
// for short ones (32 tokens: 3.3 us of the device's time, 0.35 of them for the steps, which come with the arguments).
template <int D, bool F32, int HEADS>
__device__ __forceinline__ void turn_rows(const sk_rotation& rot, const int32_t* positions, const int32_t pos0, const int n_tok, const int n_heads,
                                          const void* x, void* y, const int wg)
{
    constexpr int U = D / 16, ROWB = D * (F32 ? 4 : 2), TOK = 256 / U;
    const int head_groups = (n_heads + HEADS - 1) / HEADS, stretch = wg / head_groups, head0 = (wg - stretch * head_groups) * HEADS;
    const int unit = threadIdx.x % U, tok = stretch * TOK + threadIdx.x / U;
    if (tok >= n_tok) return;
    const Steps steps = steps_of(rot, unit);
    const int32_t position = positions ? positions[tok] : pos0 + tok;
    const bool turns = 16 * unit < rot.rotary;
    const Place at = place_of<F32>(rot, unit);
    const int64_t row = ((int64_t)tok * n_heads + head0) * ROWB;
    Unit<F32> u[HEADS];
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
        if (head0 + h < n_heads) u[h] = load_unit<F32>((const unsigned char*)x + row + h * ROWB, at);
    if (turns) {
        const Turn t = turn_of(steps, position, rot.factor);
#pragma unroll
        for (int h = 0; h < HEADS; ++h) u[h] = turned<F32>(u[h], t, rot.interleaved);
    }
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
        if (head0 + h < n_heads) store_unit<F32>((unsigned char*)y + row + h * ROWB, at, u[h]);
}

template <int D, bool F32, int HEADS>
__global__ __launch_bounds__(256) void sk_turn_rows(const void* q, void* q_out, const int Hq, const void* k, void* k_out, const int Hkv,
                                                    const int32_t* positions, const int32_t pos0, const int n_tok, const int q_wgs, const sk_rotation rot)
{
    if ((int)blockIdx.x < q_wgs) turn_rows<D, F32, HEADS>(rot, positions, pos0, n_tok, Hq, q, q_out, blockIdx.x);
    else turn_rows<D, F32, HEADS>(rot, positions, pos0, n_tok, Hkv, k, k_out, blockIdx.x - q_wgs);
}

// ---- the commit, turning on the way -------------------------------------------------------------------

struct CommitArgs {
    sk_geom g;
    sk_div by_heads;
    const void *k, *v, *q;
    void* q_out;
    const int32_t* positions;
    int32_t pos0, n_tok, commit_wgs;
    const sk_scatter* items;
    int32_t* tables_rw;
    unsigned char *kv_rw, *eph_rw;
    sk_rotation rot;
};

// `item(i)` is the i-th group that the launch commits; behind their workgroups lie those of q.
template <int D, bool F32, int HEADS, class ITEM>
__device__ __forceinline__ void commit_or_turn(const CommitArgs& A, ITEM item)
{
    __shared__ __attribute__((aligned(16))) uint16_t vt[F32 ? 8 : 16 * (D + 8)];
    const int wg = blockIdx.x;
    if (wg >= A.commit_wgs) { turn_rows<D, F32, HEADS>(A.rot, A.positions, A.pos0, A.n_tok, A.g.Hq, A.q, A.q_out, wg - A.commit_wgs); return; }
    const int i = A.by_heads.mul ? (int)(__umulhi((uint32_t)wg, A.by_heads.mul) >> A.by_heads.shift) : wg, head = wg - i * A.g.Hkv;
    const sk_scatter it = item(i);
    if (it.to_eph == SK_COPY_LIST) {
        const int at = head * 256 + threadIdx.x;
        if (at < it.count) ((u32x4*)(A.eph_rw + it.dst_off))[at] = ((const u32x4*)A.items)[it.src_tok0 + at];
        return;
    }
    commit_group<D, F32>(A.g, A.rot, A.positions, A.pos0, A.k, A.v, it, head, A.tables_rw, it.to_eph ? A.eph_rw : A.kv_rw, vt);
}

// Groups of a list, which may lie in host memory: read at once
template <int D, bool F32, int HEADS>
__global__ __launch_bounds__(256) void sk_turn_commit(const CommitArgs A)
{
    commit_or_turn<D, F32, HEADS>(A, [&](const int i) { return A.items[i]; });
}
// Groups of a stretch of tokens
template <int D, bool F32, int HEADS>
__global__ __launch_bounds__(256) void sk_turn_commit_blocks(const CommitArgs A, const sk_block_list L)
{
    commit_or_turn<D, F32, HEADS>(A, [&](const int i) {
        const int group = (L.first >> 4) + i, t0 = max(L.first, 16 * group), t1 = min(L.first + L.count, 16 * group + 16), b = t0 >> A.g.log2B;
        const int32_t block = L.id[b - L.blk0];
        return sk_scatter{(int64_t)block * A.g.blk_stride, t0 - L.first, t1 - t0, t0 & (A.g.B - 1), 0, b >= L.first_new ? L.tbl_off + b : -1, block};
    });
}

// ---- keys in the cache, turned on ---------------------------------------------------------------------

constexpr int kShiftTokens = 64;                   // tokens of a workgroup

struct ShiftArgs {
    sk_geom g;
    unsigned char* kv_rw;
    int32_t* tables_rw;
    const int32_t* list;          // pairs of a block and what it is replaced by, from blk0 on, where they are not in the arguments
    int32_t replaces;             // 0: no block is replaced
    int32_t tbl_off, blk0;
    int32_t start, end;           // storage indices: the first of a group, and behind the last token
    int32_t lo, hi;               // turned: [lo, hi) without [hole_lo, hole_hi)
    int32_t hole_lo, hole_hi;
    int32_t delta;
    const int32_t* deltas;        // by retained token from the stretch's first on, or null
    int64_t delta_stride;         // from one KV head to the next
    int32_t first;                // retained index of the stretch's first token
    sk_rotation rot;
};

// Workgroup (64 tokens, KV head): K rows are read, turned and written where they lie, or with their whole group, and its V, to the block that
// replaces theirs.  One difference for all takes one set of sines and cosines a thread; one a row takes one each (some 250 operations, which hide behind the
// rows' way).  Bound: memory.  131,072 tokens of 8 heads of 128 in a fork's shared blocks: 1.07 GB in 202 us, 5.3 TB/s, what a plain copy
// reaches; 64 tokens to a workgroup 202 us, 128 211; 2,600 tokens 7.1 and 8.9 us.
template <int D, bool F32>
__device__ __forceinline__ void turn_cached(const ShiftArgs& A, const int32_t* list)
{
    constexpr int U = D / 16, ROWB = D * (F32 ? 4 : 2), ROWS = 256 / U, N = kShiftTokens / ROWS;
    constexpr int GB = 16 * ROWB;                  // bytes of a group's V
    const int tid = threadIdx.x, span = blockIdx.x / A.g.Hkv, head = blockIdx.x - span * A.g.Hkv;
    const int t0 = A.start + span * kShiftTokens, unit = tid % U;
    unsigned char* kv = A.kv_rw + (int64_t)head * A.g.head_stride;
    auto block_of = [&](const int t, int& from, int& to) {
        const int b = t >> A.g.log2B;
        if (A.replaces) { from = list[2 * (b - A.blk0)]; to = list[2 * (b - A.blk0) + 1]; }
        else from = to = A.g.tables[A.tbl_off + b];
    };
    const Place at = place_of<F32>(A.rot, unit);
    const bool turns = 16 * unit < A.rot.rotary;
    const Steps steps = steps_of(A.rot, unit);
    Unit<F32> u[N];
    unsigned char* to_row[N];
    bool moves[N], writes[N];
    int32_t by[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int t = t0 + tid / U + i * ROWS;
        moves[i] = turns && t >= A.lo && t < A.hi && !(t >= A.hole_lo && t < A.hole_hi);
        writes[i] = false;
        by[i] = A.delta;
        if (moves[i] && A.deltas) by[i] = A.deltas[head * A.delta_stride + (t >= A.hole_hi ? t - (A.hole_hi - A.hole_lo) : t) - A.first];
        if (t < A.end) {
            int from, to;
            block_of(t, from, to);
            const int64_t row = (int64_t)(t & (A.g.B - 1)) * ROWB;
            writes[i] = moves[i] || from != to;
            to_row[i] = kv + (int64_t)to * A.g.blk_stride + row;
            if (writes[i]) u[i] = load_unit<F32>(kv + (int64_t)from * A.g.blk_stride + row, at);
        }
    }
    // V of blocks that are replaced: whole groups of 16 slots
    if (A.replaces) {
        constexpr int PV = GB / 16;                // pieces of a group
#pragma unroll
        for (int i = 0; i < kShiftTokens / 16 * PV / 256; ++i) {
            const int p = tid + 256 * i, t = t0 + p / PV * 16;
            if (t >= A.end) continue;
            int from, to;
            block_of(t, from, to);
            if (from == to) continue;
            const int64_t off = A.g.v_off + (int64_t)((t & (A.g.B - 1)) >> 4) * GB + (p % PV) * 16;
            *(u32x4*)(kv + (int64_t)to * A.g.blk_stride + off) = *(const u32x4*)(kv + (int64_t)from * A.g.blk_stride + off);
        }
        if (head == 0 && tid < kShiftTokens / 16) {
            const int t = t0 + 16 * tid;
            if (t < A.end && (t & (A.g.B - 1)) == 0) A.tables_rw[A.tbl_off + (t >> A.g.log2B)] = list[2 * ((t >> A.g.log2B) - A.blk0) + 1];
        }
    }
    // one turn for all, or one a row
    Turn turn = turn_of(steps, by[0], 1.f);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i > 0 && A.deltas) turn = turn_of(steps, by[i], 1.f);
        if (!writes[i]) continue;
        if (moves[i] && by[i] != 0) u[i] = turned<F32>(u[i], turn, A.rot.interleaved);
        store_unit<F32>(to_row[i], at, u[i]);
    }
}

template <int D, bool F32>
__global__ __launch_bounds__(256) void sk_turn_cached(const ShiftArgs A) { turn_cached<D, F32>(A, A.list); }
struct PairList { int32_t pair[2 * SK_SHIFT_ARGS_MAX]; };
template <int D, bool F32>
__global__ __launch_bounds__(256) void sk_turn_cached_args(const ShiftArgs A, const PairList L) { turn_cached<D, F32>(A, L.pair); }

// ---- launches -----------------------------------------------------------------------------------------

#define SK_BY_SHAPE(g, CALL)                                                          \
    do {                                                                              \
        if ((g).elem == 4) { if ((g).d == 128) { CALL(128, true); } else { CALL(64, true); } } \
        else { if ((g).d == 128) { CALL(128, false); } else { CALL(64, false); } }    \
    } while (0)

unsigned row_wgs(const sk_geom& g, const int n_tok, const int n_heads, const int heads)
{
    const int tok = 256 / (g.d / 16);
    return unsigned((n_tok + tok - 1) / tok) * unsigned((n_heads + heads - 1) / heads);
}

// Heads of a thread: two where one each gives more workgroups than the chip runs at a time.  us per call in a stream of them, one head a thread -> two -> four:
//                          512 tokens          1,024               2,048                4,096                 8,192
//   bf16 32/8 d 128  rows   5.1 -> 5.2 -> 5.1   6.3 -> 5.6 -> 5.8   9.6 ->  8.0 ->  8.0  16.0 -> 14.5 -> 12.9  27.1 -> 27.1 -> 25.7
//                  commit   6.4 -> 6.5 -> 6.5   7.3 -> 6.6 -> 6.7  11.4 ->  9.4 -> 10.8  17.9 -> 17.9 -> 19.0  34.2 -> 35.2 -> 36.2
//   bf16 32/8 d 64 commit   6.4 -> 6.4 -> 6.3   6.6 -> 6.4 -> 6.4   7.4 ->  6.8 ->  6.8  11.6 -> 10.5 -> 10.8  22.3 -> 22.1 -> 24.9
//   fp32 8/2 d 128 commit   6.3 -> 6.5 -> 6.6   6.4 -> 6.7 -> 6.4   6.5 ->  6.7 ->  7.3  10.4 ->  9.2 -> 11.3  22.0 -> 20.8 -> 25.6
// (one is kept below for the calls that wait for each other: half the rows to a thread)
bool two_heads(const sk_geom& g, const int n_tok) { return row_wgs(g, n_tok, g.Hq, 1) >= 1024; }

int launch_rows(const sk_geom& g, const sk_turned& t, const void* q, const void* k, void* k_out, void* stream)
{
    const bool two = two_heads(g, t.n_tok);
    const unsigned q_wgs = q ? row_wgs(g, t.n_tok, g.Hq, two ? 2 : 1) : 0, k_wgs = k ? row_wgs(g, t.n_tok, g.Hkv, two ? 2 : 1) : 0;
    if (q_wgs + k_wgs == 0) return 0;
    hipStream_t st = (hipStream_t)stream;
#define SK_ROWS(D, F32)                                                                                                                        \
    if (two) hipLaunchKernelGGL((sk_turn_rows<D, F32, 2>), dim3(q_wgs + k_wgs), dim3(256), 0, st, q, t.q_out, g.Hq, k, k_out, g.Hkv, t.positions, t.pos0, t.n_tok, (int)q_wgs, *t.rot); \
    else hipLaunchKernelGGL((sk_turn_rows<D, F32, 1>), dim3(q_wgs + k_wgs), dim3(256), 0, st, q, t.q_out, g.Hq, k, k_out, g.Hkv, t.positions, t.pos0, t.n_tok, (int)q_wgs, *t.rot)
    SK_BY_SHAPE(g, SK_ROWS);
#undef SK_ROWS
    return (int)hipGetLastError();
}

int launch_commit(const sk_geom& g, const sk_turned& t, const void* k, const void* v, const sk_scatter* items, const sk_block_list* to, int32_t n_items,
                  int32_t* tables_rw, unsigned char* kv_rw, unsigned char* eph_rw, void* stream)
{
    CommitArgs A;
    A.g = g; A.by_heads = sk_make_div((uint32_t)g.Hkv);
    A.k = k; A.v = v; A.q = t.q; A.q_out = t.q_out;
    A.positions = t.positions; A.pos0 = t.pos0; A.n_tok = t.n_tok;
    A.commit_wgs = n_items * g.Hkv;
    A.items = items; A.tables_rw = tables_rw; A.kv_rw = kv_rw; A.eph_rw = eph_rw;
    A.rot = *t.rot;
    const bool two = two_heads(g, t.n_tok);
    const dim3 grid((unsigned)A.commit_wgs + (t.q ? row_wgs(g, t.n_tok, g.Hq, two ? 2 : 1) : 0)), block(256);
    hipStream_t st = (hipStream_t)stream;
#define SK_COMMIT(D, F32)                                                                                       \
    if (to) { if (two) hipLaunchKernelGGL((sk_turn_commit_blocks<D, F32, 2>), grid, block, 0, st, A, *to);     \
              else hipLaunchKernelGGL((sk_turn_commit_blocks<D, F32, 1>), grid, block, 0, st, A, *to); }        \
    else if (two) hipLaunchKernelGGL((sk_turn_commit<D, F32, 2>), grid, block, 0, st, A);                      \
    else hipLaunchKernelGGL((sk_turn_commit<D, F32, 1>), grid, block, 0, st, A)
    SK_BY_SHAPE(g, SK_COMMIT);
#undef SK_COMMIT
    return (int)hipGetLastError();
}
int launch_scatter(const sk_geom& g, const sk_turned& t, const void* k, const void* v, const sk_scatter* items, int32_t n_items,
                   int32_t* tables_rw, unsigned char* kv_rw, unsigned char* eph_rw, void* stream)
{
    return launch_commit(g, t, k, v, items, nullptr, n_items, tables_rw, kv_rw, eph_rw, stream);
}
int launch_blocks(const sk_geom& g, const sk_turned& t, const void* k, const void* v, const sk_block_list& to, int32_t* tables_rw, unsigned char* kv_rw, void* stream)
{
    return launch_commit(g, t, k, v, nullptr, &to, (to.first + to.count + 15) / 16 - to.first / 16, tables_rw, kv_rw, nullptr, stream);
}

// The part of a turn, in 2^-64, that a pair of frequency f (at most 2^20) turns a position: f / (2 pi) less its whole turns, to the nearest.  f is a 53-bit m over 2^s, with s
// from 33 on, and m / (2 pi) is formed in whole numbers, from 128 bits of 1 / (2 pi), before anything is dropped: whole turns take no bits off what is left of them.  (A quotient of 64 bits
// has lost 19 of them at f = 10^6, which is 1.3e-4 rad at position 2^31.)
uint64_t step_of(const double f)
{
    constexpr uint64_t kInverseHigh = 0x28be60db9391054aull, kInverseLow = 0x7f09d5f47d4d3770ull;
    int e;
    const uint64_t m = (uint64_t)std::ldexp(std::frexp(std::fabs(f), &e), 53);
    const int s = 53 - e;
    const unsigned __int128 turns = (unsigned __int128)m * kInverseHigh + (uint64_t)((unsigned __int128)m * kInverseLow >> 64);      // f / (2 pi) in 2^-(64 + s), by less than one too few
    const uint64_t step = s > 127 ? 0 : (uint64_t)((turns + ((unsigned __int128)1 << (s - 1))) >> s);
    return f < 0 ? 0 - step : step;
}

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

sk_turned make_turned(const sk_geom& g, const sk_rotation* rot, const void* q, void* q_out, const int32_t* positions, int32_t pos0, int32_t n_tok)
{
    sk_turned t;
    t.rot = rot; t.positions = positions; t.pos0 = pos0; t.n_tok = n_tok; t.q = q; t.q_out = q_out;
    t.rows = launch_rows; t.scatter = launch_scatter; t.blocks = launch_blocks;
    t.small = sk_small_turns(g, *rot, n_tok) ? sk_launch_attention_small_turned : nullptr;
    return t;
}

}  // namespace

extern "C" {

int sk_pool_set_rotation(sk_pool* p, int32_t rotary_dim, int32_t interleaved, const double* inv_freq, float factor)
{
    if (!p) return SK_E_INVAL;
    sk_geom g;
    sk_geom_of(p, &g);
    if (rotary_dim <= 0 || rotary_dim % 16 || rotary_dim > g.d) return SK_E_SHAPE;
    if (!inv_freq || !(std::fabs(factor) <= 3.0e38f)) return SK_E_INVAL;
    for (int i = 0; i < rotary_dim / 2; ++i)
        if (!(std::fabs(inv_freq[i]) <= 1e6)) return SK_E_INVAL;
    sk_rotation r = {};
    r.rotary = rotary_dim; r.interleaved = interleaved != 0; r.factor = factor;
    for (int i = 0; i < rotary_dim / 2; ++i) r.step[i] = step_of(inv_freq[i]);
    *sk_rotation_of(p) = r;
    return SK_OK;
}

int sk_rotate(sk_pool* p, const void* q, const void* k, int32_t n_tok, const int32_t* positions, int32_t pos0, void* q_out, void* k_out, void* hip_stream)
{
    if (!p || !sk_rotation_of(p)->rotary || n_tok < 0) return SK_E_INVAL;
    if (n_tok == 0) return SK_OK;
    sk_geom g;
    const bool device = sk_geom_of(p, &g);
    if ((int64_t)n_tok * g.Hq > (int64_t(1) << 27)) return SK_E_INVAL;      // (a grid has fewer than 2^32 threads)
    if (!device) return SK_E_NODEVICE;
    if ((!q && !k) || (!q) != (!q_out) || (!k) != (!k_out)) return SK_E_INVAL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(q_out, 16) || !aligned(k_out, 16) || !aligned(positions, 4)) return SK_E_INVAL;
    if (!positions && pos0 > INT32_MAX - (n_tok - 1)) return SK_E_INVAL;
    const sk_turned t = make_turned(g, sk_rotation_of(p), q, q_out, positions, pos0, n_tok);
    if (!sk_turned_apart(g, t, n_tok, k, nullptr, k_out, nullptr, SK_F32, nullptr)) return SK_E_INVAL;
    if (sk_injected(p, SK_SITE_SCATTER)) return SK_E_HIP;
    const int e = launch_rows(g, t, q, k, k_out, hip_stream);
    if (e) return sk_note_hip_error(e);
    sk_count_launch(p);
    return SK_OK;
}

int sk_session_append_rotated(sk_pool* p, int32_t id, const void* q, const void* k, const void* v, int32_t L, const int32_t* positions, int32_t pos0,
                              void* q_out, void* out, int out_dtype, float* lse, void* hip_stream)
{
    if (!p || !sk_rotation_of(p)->rotary || L < 0) return SK_E_INVAL;
    sk_session_view V;
    const int rc = sk_view_session(p, id, &V);
    if (rc) return rc;
    sk_turned t = make_turned(V.g, sk_rotation_of(p), q, q_out, positions, pos0, L);
    if (L > 0 && !positions && pos0 > INT32_MAX - (L - 1)) return SK_E_INVAL;
    if (L > 0 && V.device) {
        if ((!q) != (!q_out) || !aligned(q_out, 16) || !aligned(positions, 4)) return SK_E_INVAL;
        if (!sk_turned_apart(V.g, t, L, k, v, nullptr, out, out_dtype, lse)) return SK_E_INVAL;
    }
    return sk_append_turned(p, id, t, k, v, L, out, out_dtype, lse, hip_stream);
}

int sk_batch_step_rotated(sk_pool* p, int32_t n_items, const int32_t* session_id, const int32_t* op, const int32_t* cu_tokens, const int32_t* positions,
                          const void* q, const void* k, const void* v, void* q_out, void* out, int out_dtype, float* lse, void* hip_stream)
{
    if (!p || !sk_rotation_of(p)->rotary) return SK_E_INVAL;
    if (!aligned(q_out, 16) || !aligned(positions, 4)) return SK_E_INVAL;
    sk_geom g;
    (void)sk_geom_of(p, &g);
    sk_turned t = make_turned(g, sk_rotation_of(p), q, q_out, positions, 0, 0);
    return sk_batch_turned(p, n_items, session_id, op, cu_tokens, t, k, v, out, out_dtype, lse, hip_stream);
}

int sk_session_shift(sk_pool* p, int32_t id, int64_t first, int64_t count, int32_t delta, const int32_t* deltas, int64_t delta_stride, void* hip_stream)
{
    if (!p || !sk_rotation_of(p)->rotary) return SK_E_INVAL;
    sk_session_view V;
    int rc = sk_view_session(p, id, &V);
    if (rc) return rc;
    if (first < 0 || count < 0 || first > V.retained - count) return SK_E_INVAL;
    if (!aligned(deltas, 4) || (deltas && delta_stride != 0 && delta_stride < count)) return SK_E_INVAL;
    if (count == 0 || (!deltas && delta == 0)) return SK_OK;
    auto stored = [&](const int64_t j) { return j < V.frozen ? j : j - V.frozen + V.win; };
    const int64_t lo = stored(first), hi = stored(first + count - 1) + 1;
    sk_shift E;
    PairList pairs;
    rc = sk_shift_begin(p, id, lo, hi, pairs.pair, &E);
    if (rc) return rc;
    if (sk_injected(p, SK_SITE_SCATTER)) return SK_E_HIP;
    if (V.device) {
        // an error that an earlier call of the thread left behind is told before anything is launched: what comes back behind the launch is its own
        int e = (int)hipGetLastError();
        if (e) return sk_note_hip_error(e);
        ShiftArgs A = {};
        A.g = V.g; A.kv_rw = E.kv_rw; A.tables_rw = E.tables_rw; A.list = E.list; A.replaces = E.n_fresh > 0; A.tbl_off = V.tbl_off; A.blk0 = (int32_t)E.blk0;
        // of replaced blocks everything that holds tokens, otherwise the groups of the stretch
        const int64_t start = A.replaces ? E.blk0 * V.g.B : lo / 16 * 16, behind = (E.blk0 + E.n_blk) * V.g.B;
        const int64_t end = A.replaces ? (behind < E.len ? behind : E.len) : hi;
        A.start = (int32_t)start; A.end = (int32_t)end; A.lo = (int32_t)lo; A.hi = (int32_t)hi;
        A.hole_lo = (int32_t)V.frozen; A.hole_hi = (int32_t)V.win;
        A.delta = delta; A.deltas = deltas; A.delta_stride = delta_stride; A.first = (int32_t)first;
        A.rot = *sk_rotation_of(p);
        const dim3 grid((unsigned)((end - start + kShiftTokens - 1) / kShiftTokens * V.g.Hkv)), block(256);
#define SK_SHIFT(D, F32)                                                                                                        \
    if (E.pairs) hipLaunchKernelGGL((sk_turn_cached_args<D, F32>), grid, block, 0, (hipStream_t)hip_stream, A, pairs);            \
    else hipLaunchKernelGGL((sk_turn_cached<D, F32>), grid, block, 0, (hipStream_t)hip_stream, A)
        SK_BY_SHAPE(V.g, SK_SHIFT);
#undef SK_SHIFT
        e = (int)hipGetLastError();
        if (e) return sk_note_hip_error(e);
        sk_shift_listed(p, E, hip_stream);
        sk_count_launch(p);
    }
    sk_shift_end(p, E);
    return SK_OK;
}

}  // extern "C"
