// Random walk over the host half of rotated appends and of shifts, among the calls that share and free blocks (metadata-only pools), meant to
// be built with -fsanitize=address,undefined on the host pass and run by tests/test_rotation_host.py.  Checks a shadow model as it goes; exits
// non-zero on a mismatch (the sanitizers abort by themselves).
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <vector>

#include <hip/hip_runtime_api.h>

#include "../include/sk.h"

static uint64_t rng_state = 0x5EED0011ull;
static uint32_t rnd(uint32_t n) { rng_state = rng_state * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)(rng_state >> 33) % n; }

#define CHECK(c) do { if (!(c)) { std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

struct Shadow { int64_t len = 0, frozen = 0; };
typedef std::map<int32_t, std::vector<int32_t>> Tables;

static Tables tables(sk_pool* p, const std::map<int32_t, Shadow>& live)
{
    Tables t;
    for (auto& kv : live) {
        const int32_t* at = nullptr;
        int64_t n = 0;
        CHECK(sk_session_block_table(p, kv.first, &at, &n) == SK_OK);
        t[kv.first].assign(at, at + n);
    }
    return t;
}

static std::map<int32_t, int> holders_of(const Tables& t)
{
    std::map<int32_t, int> h;
    for (auto& kv : t)
        for (int32_t b : kv.second) h[b]++;
    return h;
}

static void walk(const int n_ops, const int block_tokens)
{
    sk_pool_desc d = {};
    d.dtype = SK_BF16; d.n_q_heads = 8; d.n_kv_heads = 4; d.head_dim = 64;
    d.block_tokens = block_tokens; d.max_sessions = 8; d.n_blocks = 24000 / block_tokens; d.max_batch_tokens = 10000;
    d.flags = SK_POOL_METADATA_ONLY;
    sk_pool* p = nullptr;
    CHECK(sk_pool_create(&d, &p) == SK_OK && p);
    double f[32];
    for (int i = 0; i < 32; ++i) f[i] = 1.0 / (1 + i);
    CHECK(sk_session_append_rotated(p, 0, nullptr, nullptr, nullptr, 1, nullptr, 0, nullptr, nullptr, SK_F32, nullptr, nullptr) == SK_E_INVAL);
    CHECK(sk_pool_set_rotation(p, 64, 1, f, 1.f) == SK_OK && sk_pool_set_rotation(p, 32, 0, f, 1.f) == SK_OK);
    std::map<int32_t, Shadow> live;
    int replaced = 0, full = 0, failed = 0, steps = 0;
    for (int it = 0; it < n_ops; ++it) {
        const uint32_t op = rnd(100);
        if (live.empty() || op < 6) {
            int32_t id = -1;
            if (sk_session_create(p, &id) == SK_OK) live[id] = Shadow();
            else CHECK((int)live.size() == d.max_sessions);
            continue;
        }
        auto itr = live.begin();
        std::advance(itr, rnd((uint32_t)live.size()));
        const int32_t id = itr->first;
        Shadow& s = itr->second;
        const Tables before = tables(p, live);
        int64_t free_before = 0, free_now = 0;
        CHECK(sk_pool_blocks_free(p, &free_before) == SK_OK);
        if (op < 30) {                                       // a rotated append, sometimes with a failure ordered
            const int32_t L = 1 + (int32_t)rnd(rnd(8) ? 500 : 9000);
            const int sites[3] = {SK_SITE_BLOCK_COPY, SK_SITE_SCATTER, SK_SITE_ATTENTION};
            const int site = rnd(8) < 3 ? sites[rnd(3)] : SK_SITE_NONE;
            CHECK(sk_pool_inject_failure(p, site, site ? 1 + (int32_t)rnd(2) : 0) == SK_OK);
            const int rc = sk_session_append_rotated(p, id, nullptr, nullptr, nullptr, L, nullptr, (int32_t)rnd(1000000), nullptr, nullptr, SK_F32, nullptr, nullptr);
            CHECK(sk_pool_inject_failure(p, 0, 0) == SK_OK);
            if (rc == SK_OK) s.len += L;
            else {
                CHECK((rc == SK_E_HIP && site != SK_SITE_NONE) || rc == SK_E_NOMEM);
                ++(rc == SK_E_NOMEM ? full : failed);
                // as it was, but for the private copy of a shared last block, which a launch may have made its own
                const Tables after = tables(p, live);
                CHECK(sk_pool_blocks_free(p, &free_now) == SK_OK && (free_now == free_before || free_now == free_before - 1));
                for (auto& kv : after) {
                    if (kv.first != id || free_now == free_before) { CHECK(kv.second == before.at(kv.first)); continue; }
                    const std::vector<int32_t>& was = before.at(id);
                    CHECK(kv.second.size() == was.size());
                    for (size_t i = 0; i + 1 < was.size(); ++i) CHECK(kv.second[i] == was[i]);
                }
            }
        } else if (op < 65) {                                // a shift
            const int64_t first = s.len ? (int64_t)rnd((uint32_t)s.len + 1) : 0, count = (int64_t)rnd((uint32_t)(s.len - first) + 1);
            const int sites[2] = {SK_SITE_RING, SK_SITE_SCATTER};
            const int site = rnd(8) < 3 ? sites[rnd(2)] : SK_SITE_NONE;
            CHECK(sk_pool_inject_failure(p, site, site ? 1 : 0) == SK_OK);
            const int rc = sk_session_shift(p, id, first, count, (int32_t)rnd(3) - 1, nullptr, 0, nullptr);
            CHECK(sk_pool_inject_failure(p, 0, 0) == SK_OK);
            const Tables after = tables(p, live);
            CHECK(sk_pool_blocks_free(p, &free_now) == SK_OK);
            if (rc != SK_OK) {
                CHECK((rc == SK_E_HIP && site != SK_SITE_NONE) || rc == SK_E_NOMEM);
                CHECK(after == before && free_now == free_before);
                ++(rc == SK_E_NOMEM ? full : failed);
            } else {
                const std::map<int32_t, int> was = holders_of(before), is = holders_of(after);
                int changed = 0;
                for (auto& kv : after) {
                    if (kv.first != id) { CHECK(kv.second == before.at(kv.first)); continue; }
                    CHECK(kv.second.size() == before.at(id).size());
                    for (size_t i = 0; i < kv.second.size(); ++i)
                        if (kv.second[i] != before.at(id)[i]) { ++changed; CHECK(was.at(before.at(id)[i]) > 1 && is.at(kv.second[i]) == 1); }
                }
                CHECK(free_now == free_before - changed);
                replaced += changed;
            }
            CHECK(sk_session_shift(p, id, 0, s.len + 1, 1, nullptr, 0, nullptr) == SK_E_INVAL);
            CHECK(sk_session_shift(p, id, INT64_MAX, 1, 1, nullptr, 0, nullptr) == SK_E_INVAL);
            CHECK(sk_session_shift(p, id, 1, INT64_MAX, 1, nullptr, 0, nullptr) == SK_E_INVAL);
        } else if (op < 70) {                                // a ragged step
            std::vector<int32_t> ids, ops, cu(1, 0);
            int64_t room = d.max_batch_tokens;
            for (auto& kv : live) {
                const int32_t T = (int32_t)rnd(300);
                if (room < T || (rnd(4) == 0 && !ids.empty())) continue;
                room -= T;
                ids.push_back(kv.first);
                ops.push_back(kv.second.len > 0 ? (int32_t)rnd(3) : (int32_t)rnd(2) * SK_OP_QUERY_B);
                cu.push_back(cu.back() + T);
            }
            const int site = rnd(4) ? SK_SITE_NONE : rnd(2) ? SK_SITE_SCATTER : SK_SITE_ATTENTION;
            CHECK(sk_pool_inject_failure(p, site, site ? 1 : 0) == SK_OK);
            const int rc = sk_batch_step_rotated(p, (int32_t)ids.size(), ids.data(), ops.data(), cu.data(), nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                                                 SK_F32, nullptr, nullptr);
            CHECK(sk_pool_inject_failure(p, 0, 0) == SK_OK);
            if (rc == SK_OK) {
                ++steps;
                for (size_t i = 0; i < ids.size(); ++i)
                    if (ops[i] == SK_OP_APPEND) live[ids[i]].len += cu[i + 1] - cu[i];
            } else CHECK((rc == SK_E_HIP && site != SK_SITE_NONE) || rc == SK_E_NOMEM);
        } else if (op < 77) {
            const int64_t n = s.len > s.frozen ? (int64_t)rnd((uint32_t)(s.len - s.frozen) + 1) / 3 : 0;
            if (sk_session_evict_oldest(p, id, n, nullptr) == SK_OK) s.len -= n;
        } else if (op < 82) {
            const int64_t nf = s.frozen + (int64_t)rnd((uint32_t)(s.len - s.frozen) / 4 + 1);
            if (sk_session_freeze(p, id, nf) == SK_OK) s.frozen = nf;
        } else if (op < 87) {
            const int64_t nl = s.len - (s.len ? (int64_t)rnd((uint32_t)s.len + 1) / 2 : 0);
            CHECK(sk_session_truncate(p, id, nl) == SK_OK);
            s.len = nl;
            if (s.frozen > nl) s.frozen = nl;
        } else if (op < 95) {
            const int64_t np = s.len ? (int64_t)rnd((uint32_t)s.len + 1) : 0;
            int32_t fid = -1;
            if (sk_session_fork(p, id, np, &fid, nullptr) == SK_OK) { live[fid].len = np; live[fid].frozen = s.frozen < np ? s.frozen : np; }
        } else if (op < 97) {
            const int64_t n = s.len > s.frozen ? (int64_t)rnd((uint32_t)(s.len - s.frozen) + 1) / 3 : 0;
            if (sk_session_evict_lowest(p, id, nullptr, 0, n, 0, 1, nullptr, 0, nullptr) == SK_OK) s.len -= n;
        } else {
            CHECK(sk_session_destroy(p, id) == SK_OK);
            live.erase(id);
        }
        CHECK(sk_pool_blocks_free(p, &free_now) == SK_OK);
        std::map<int32_t, int> holders;
        for (auto& kv : tables(p, live)) {
            int64_t len = 0;
            CHECK(sk_session_length(p, kv.first, &len) == SK_OK && len == live.at(kv.first).len);
            const int64_t nb = (int64_t)kv.second.size(), least = (len + block_tokens - 1) / block_tokens;
            CHECK(nb >= least && nb <= least + 2);
            for (int32_t b : kv.second) { CHECK(b >= 0 && b < d.n_blocks); holders[b]++; }
        }
        CHECK((int64_t)holders.size() + free_now == d.n_blocks);
    }
    CHECK(replaced > 50 && full > 0 && failed > 10 && steps > 10);
    for (auto& kv : live) CHECK(sk_session_destroy(p, kv.first) == SK_OK);
    int64_t left = 0;
    CHECK(sk_pool_blocks_free(p, &left) == SK_OK && left == d.n_blocks);
    CHECK(sk_pool_destroy(p) == SK_OK);
}

// The workspace of sk_verify: enough whatever is asked, never for what is refused.
static void workspaces()
{
    for (int it = 0; it < 20000; ++it) {
        const int32_t n = 1 + (int32_t)rnd(rnd(2) ? 300 : 40000), k = (int32_t)rnd(34), v = 1 + (int32_t)rnd(rnd(2) ? 1000 : 1 << 21);
        const size_t bytes = sk_verify_workspace_bytes(n, k, v);
        if (k > SK_VERIFY_MAX_DRAFT || (int64_t)n * (k + 1) > SK_VERIFY_MAX_ROWS) CHECK(bytes == 0);
        else CHECK(bytes >= size_t(n) * size_t(k + 1) * 16 && bytes % 8 == 0);
    }
}

int main(int argc, char** argv)
{
    const int n_ops = argc > 1 ? std::atoi(argv[1]) : 6000;
    for (int block_tokens : {16, 64, 256}) walk(n_ops, block_tokens);
    workspaces();
    std::printf("host walk ok\n");
    return 0;
}
