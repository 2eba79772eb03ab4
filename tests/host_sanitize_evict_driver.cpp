// Random walk over the host half of the eviction by weight, among the calls that share and free blocks, and over the checks of the
// attention weights (metadata-only pools), meant to be built with -fsanitize=address,undefined on the host pass and run by
// tests/test_host_sanitizers.py.  Checks a shadow model as it goes; exits non-zero on a mismatch (the sanitizers abort by themselves).
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <vector>

#include <hip/hip_runtime_api.h>

#include "../include/sk.h"
#include "../paper_2605_13784_amd/csrc/sk_internal.h"

static uint64_t rng_state = 0x5EED0010ull;
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

static void walk(const int n_ops, const int block_tokens)
{
    sk_pool_desc d = {};
    d.dtype = SK_BF16; d.n_q_heads = 8; d.n_kv_heads = 4; d.head_dim = 64;
    d.block_tokens = block_tokens; d.max_sessions = 8; d.n_blocks = 4800 / block_tokens; d.max_batch_tokens = 2048;
    d.flags = SK_POOL_METADATA_ONLY;
    sk_pool* p = nullptr;
    CHECK(sk_pool_create(&d, &p) == SK_OK && p);
    std::map<int32_t, Shadow> live;
    int evicted = 0, full = 0, failed = 0;
    for (int it = 0; it < n_ops; ++it) {
        const uint32_t op = rnd(100);
        int64_t free_before = 0;
        CHECK(sk_pool_blocks_free(p, &free_before) == SK_OK);
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
        if (op < 40) {
            const int32_t L = 1 + (int32_t)rnd(700);
            if (sk_session_append(p, id, nullptr, nullptr, nullptr, L, nullptr, SK_F32, nullptr, nullptr) == SK_OK) s.len += L;
        } else if (op < 72) {                                // the eviction, sometimes with a failure ordered
            const int64_t recent = rnd(3) ? (int64_t)rnd(80) : 0, room = s.len - s.frozen - recent;
            const int64_t n = room > 0 ? (int64_t)rnd((uint32_t)room + 1) : 0;
            const int sites[4] = {SK_SITE_RING, SK_SITE_EVICT_SELECT, SK_SITE_EVICT_MOVE, SK_SITE_NONE};
            const int site = sites[rnd(8) < 3 ? rnd(3) : 3];
            CHECK(sk_pool_inject_failure(p, site, site ? 1 : 0) == SK_OK);
            const int rc = sk_session_evict_lowest(p, id, nullptr, 0, n, recent, (int32_t)rnd(2), nullptr, 0, nullptr);
            CHECK(sk_pool_inject_failure(p, 0, 0) == SK_OK);
            const Tables after = tables(p, live);
            int64_t free_now = 0;
            CHECK(sk_pool_blocks_free(p, &free_now) == SK_OK);
            if (rc != SK_OK) {
                CHECK((rc == SK_E_HIP && site != SK_SITE_NONE) || rc == SK_E_NOMEM);
                CHECK(after == before && free_now == free_before);
                ++(rc == SK_E_NOMEM ? full : failed);
            } else {
                s.len -= n;
                evicted += n > 0;
                for (auto& kv : after)
                    if (kv.first != id) CHECK(kv.second == before.at(kv.first));
                // what is written again, every block behind the frozen tokens' last whole one at least, is held by this session alone
                std::map<int32_t, int> holders;
                for (auto& kv : after)
                    for (int32_t b : kv.second) holders[b]++;
                const std::vector<int32_t>& t = after.at(id);
                if (n > 0)
                    for (size_t i = size_t(s.frozen / block_tokens) + 2; i < t.size(); ++i) CHECK(holders[t[i]] == 1);
            }
            CHECK(sk_session_evict_lowest(p, id, nullptr, 0, s.len - s.frozen + 1, 0, 1, nullptr, 0, nullptr) == SK_E_INVAL);
            CHECK(sk_session_evict_lowest(p, id, nullptr, 0, -1, 0, 1, nullptr, 0, nullptr) == SK_E_INVAL);
            CHECK(sk_session_evict_lowest(p, id, nullptr, 0, 1, s.len, 1, nullptr, 0, nullptr) == SK_E_INVAL);
            CHECK(sk_session_evict_lowest(p, id, nullptr, 0, 0, INT64_MAX, 1, nullptr, 0, nullptr) == SK_OK);
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
        } else if (op < 98) {                                // the weights: what can be refused without a device is, and the rest ends there
            std::vector<int32_t> ids, causal, cu(1, 0);
            std::vector<float*> out;
            std::vector<int64_t> stride;
            for (auto& kv : live) {
                ids.push_back(kv.first);
                causal.push_back((int32_t)rnd(2) && kv.second.len >= 5);
                cu.push_back(cu.back() + (int32_t)rnd(5));
                out.push_back(nullptr);
                stride.push_back(0);
            }
            const int32_t n = (int32_t)ids.size();
            auto call = [&](const int32_t* which) {
                return sk_batch_attention_mass(p, n, which, causal.data(), cu.data(), nullptr, nullptr, nullptr, nullptr, 1.f, out.data(), stride.data(), nullptr);
            };
            CHECK(call(ids.data()) == SK_E_NODEVICE && call(ids.data()) == SK_E_NODEVICE);
            if (n > 1) {
                std::vector<int32_t> twice = ids;
                twice[n - 1] = twice[0];
                causal[n - 1] = 0;
                CHECK(call(twice.data()) == SK_E_INVAL);
                twice[0] = d.max_sessions;
                CHECK(call(twice.data()) == SK_E_BADSESSION);
            }
            CHECK(sk_session_attention_mass(p, id, nullptr, nullptr, (int32_t)s.len + 1, 1, nullptr, 0, 1.f, nullptr, 0, nullptr) == SK_E_INVAL);
        } else {
            CHECK(sk_session_destroy(p, id) == SK_OK);
            live.erase(id);
        }
        int64_t free_now = 0;
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
    CHECK(evicted > 50 && full > 0 && failed > 10);
    for (auto& kv : live) CHECK(sk_session_destroy(p, kv.first) == SK_OK);
    int64_t f = 0;
    CHECK(sk_pool_blocks_free(p, &f) == SK_OK && f == d.n_blocks);
    CHECK(sk_pool_destroy(p) == SK_OK);
}

// Arrays of sums that a call reads and writes: an entry that both have is found, wherever they lie.
static void overlaps()
{
    static float memory[4096];
    for (int it = 0; it < 200000; ++it) {
        const int64_t rows = 1 + rnd(5), n = 1 + rnd(12), sa = n + rnd(20), sb = rnd(2) ? sa : n + (int64_t)rnd(20);
        const int64_t a = rnd(300), b = rnd(3) ? rnd(300) : a;
        bool meet = false;
        for (int64_t i = 0; i < rows; ++i)
            for (int64_t j = 0; j < rows; ++j) {
                const int64_t x = (a + i * sa) - (b + j * sb);
                meet |= x < n && -x < n;
            }
        const bool same = a == b && (sa == sb || rows == 1);
        const bool found = sk_rows_overlap(memory + a, sa, memory + b, sb, rows, n);
        if (meet && !same) CHECK(found);
        if (a == b && sa == sb) CHECK(!found);
        if (!meet) CHECK(!found);
    }
}

int main(int argc, char** argv)
{
    const int n_ops = argc > 1 ? std::atoi(argv[1]) : 12000;
    for (int block_tokens : {16, 64, 256}) walk(n_ops, block_tokens);
    overlaps();
    std::printf("host walk ok\n");
    return 0;
}
