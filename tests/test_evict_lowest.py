"""sk_session_evict_lowest: which tokens leave (by sum, then by age), that the others are there bit for bit and in order, what
becomes of blocks, forks and sums, and attention over what is left.  Everything but that last part is exact."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2605_13784_amd as sk
from gpu_common import compare
from workloads import synth

D64 = synth.Shape("bf16", 8, 4, 64)
ODD = synth.Shape("bf16", 6, 3, 128)
F32_WIDE = synth.Shape("f32", 4, 2, 128)


class Model:
    """What the session holds, by hand: K and V [n][Hkv][d] as raw bits (row j is every head's own j-th token), sums [Hkv][n]."""

    def __init__(self, shape, k, v, frozen=0):
        self.shape, self.K, self.V, self.frozen = shape, k, v, frozen

    def evict(self, mass, n_evict, n_recent, per_head):
        n, hkv = self.K.shape[0], self.shape.n_kv_heads
        m = n - n_evict
        last = max(n - n_recent, self.frozen)
        rows = mass
        if not per_head:
            total = mass[0].copy()
            for g in range(1, hkv):
                total = total + mass[g]                    # fp32, head by head
            rows = np.repeat(total[None], hkv, 0)
        K, V, out = np.empty_like(self.K[:m]), np.empty_like(self.V[:m]), np.zeros_like(mass)
        for g in range(hkv):
            gone = self.frozen + np.argsort(rows[g, self.frozen:last], kind="stable")[:n_evict]
            left = np.delete(np.arange(n), gone)
            K[:, g], V[:, g], out[g, :m] = self.K[left, g], self.V[left, g], mass[g, left]
        self.K, self.V = K, V
        return out


def _check(pool, sid, model):
    assert pool.sk_session_length(sid) == model.K.shape[0]
    if model.K.shape[0]:
        k, v = pool.sk_session_gather(sid)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(synth.to_raw(k.cpu()), model.K)
        np.testing.assert_array_equal(synth.to_raw(v.cpu()), model.V)


def _attend(pool, sid, model, gen, T=5):
    """A query over what is left, against the oracle."""
    shape = model.shape
    q = synth.draw(gen, (T, shape.n_q_heads, shape.head_dim), shape.dtype)
    out, lse = pool.sk_session_query(sid, q.cuda())
    ro, rl = oracle.attention(shape.dtype, synth.to_raw(q), model.K, model.V, None, None, None, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                              shape.head_dim ** -0.5)
    compare("query", out, lse, ro, rl, shape.dtype)


def _make(shape, gen, n, block, frozen=0, evicted=0, spare=9, max_sessions=3):
    blocks = -(-(n + evicted) // block) + spare
    pool = sk.Pool(shape.dtype, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, block, blocks, max_sessions=max_sessions, max_batch_tokens=8192, kv_fill=0xFF)
    pool.sk_pool_set_alloc_order(synth.permutation(gen, blocks))
    sid = pool.sk_session_create()
    _, k, v = synth.draw_qkv(gen, n + evicted, shape)
    for t in range(0, n + evicted, 8192):
        pool.sk_session_append(sid, None, k[t:t + 8192].cuda(), v[t:t + 8192].cuda())
    if frozen:
        pool.sk_session_freeze(sid, frozen)
    if evicted:
        pool.sk_session_evict_oldest(sid, evicted)
    k, v = (synth.to_raw(torch.cat([x[:frozen], x[frozen + evicted:]])) for x in (k, v))
    return pool, sid, Model(shape, k, v, frozen)


def _mass(gen, hkv, n, kind="spread"):
    if kind == "spread":
        return torch.exp(1.5 * torch.randn((hkv, n), generator=gen))
    if kind == "equal":
        return torch.full((hkv, n), 0.25)
    if kind == "zero":
        return torch.zeros((hkv, n)) * torch.where(torch.arange(n) % 2 == 0, 1.0, -1.0)      # +0 and -0 are equal
    if kind == "few":
        return torch.randint(0, 4, (hkv, n), generator=gen).float()
    if kind == "rising":
        return torch.arange(n).float().repeat(hkv, 1) * 2.0 ** -10
    if kind == "falling":
        return -torch.arange(n).float().repeat(hkv, 1)
    if kind == "near":                                         # differ in the last bits only
        return (torch.full((hkv, n), 1.0).view(torch.int32) + torch.randint(0, 50, (hkv, n), generator=gen, dtype=torch.int32)).view(torch.float32)
    assert kind == "odd"                                       # negative sums, infinities and NaN
    x = torch.randn((hkv, n), generator=gen)
    x[:, ::7], x[:, 3::11], x[:, 5::13] = float("nan"), float("inf"), -float("inf")
    return x


CASES = [(D64, 200, 16, 0, 0, 100, 0, True), (D64, 200, 16, 0, 0, 1, 0, True), (D64, 200, 16, 0, 0, 200, 0, True), (D64, 200, 16, 0, 0, 0, 0, True),
         (D64, 1, 16, 0, 0, 1, 0, True), (D64, 17, 16, 3, 0, 5, 4, False), (D64, 333, 64, 37, 0, 63, 50, True), (D64, 333, 64, 64, 0, 64, 0, False),
         (D64, 1000, 256, 100, 0, 65, 1000 - 100 - 65, True), (D64, 1000, 1024, 1, 0, 500, 10, True), (D64, 700, 16, 20, 35, 300, 64, True),
         (D64, 700, 64, 0, 100, 333, 1, False), (ODD, 650, 16, 15, 3, 129, 17, True), (ODD, 1500, 64, 500, 70, 900, 100, True),
         (synth.CFG2, 2600, 16, 0, 0, 1300, 64, True), (synth.CFG2, 4099, 16, 100, 5, 257, 300, True), (synth.CFG2, 9001, 64, 500, 1000, 4000, 333, False),
         (synth.CFG1, 500, 16, 0, 0, 250, 10, True), (synth.CFG1, 777, 64, 33, 40, 100, 0, False), (F32_WIDE, 600, 16, 10, 20, 64, 64, True),
         (D64, 30000, 16, 0, 0, 1000, 0, True), (D64, 30000, 256, 1234, 77, 15000, 5000, True), (D64, 40000, 16, 0, 0, 39000, 0, False),
         (synth.CFG2, 36000, 16, 7, 0, 1500, 0, True)]         # the last in two stretches where it moves by way of the workspace


@pytest.mark.gpu
@pytest.mark.parametrize("room", [False, True])               # free blocks for what stays, or too few
@pytest.mark.parametrize("shape,n,block,frozen,evicted,n_evict,n_recent,per_head", CASES)
def test_what_leaves_and_what_stays(shape, n, block, frozen, evicted, n_evict, n_recent, per_head, room):
    gen = synth.generator(10, stream=n + n_evict)
    pool, sid, model = _make(shape, gen, n, block, frozen, evicted, spare=9 + (n // block if room else 0))
    before = pool.sk_session_block_table(sid)
    mass = _mass(gen, shape.n_kv_heads, n + 3)
    place = mass.cuda()
    free = pool.sk_pool_blocks_free()
    held = len(pool.sk_session_block_table(sid))
    want = model.evict(mass[:, :n].numpy(), n_evict, n_recent, per_head)
    assert pool.sk_session_evict_lowest(sid, place, n_evict, n_recent, per_head) is place
    torch.cuda.synchronize()
    np.testing.assert_array_equal(place[:, :n].cpu().numpy(), want)
    assert torch.equal(place[:, n:].cpu(), mass[:, n:])
    _check(pool, sid, model)
    if room and n_evict and n > n_evict + frozen + block:
        assert not set(pool.sk_session_block_table(sid)[frozen // block + 2 + evicted // block:]) & set(before)
    elif not room and n > n_evict + 20 * block + frozen:
        assert pool.sk_session_block_table(sid) == before[:len(pool.sk_session_block_table(sid))]
    assert held - len(pool.sk_session_block_table(sid)) == pool.sk_pool_blocks_free() - free >= n_evict // block
    if n > n_evict:
        _attend(pool, sid, model, gen)
    # it goes on: tokens are appended, and some leave again
    q, k, v = synth.draw_qkv(gen, 100 if n < 20000 else 40, shape)
    model.K, model.V = np.concatenate([model.K, synth.to_raw(k)]), np.concatenate([model.V, synth.to_raw(v)])
    pool.sk_session_append(sid, q.cuda(), k.cuda(), v.cuda())
    n2 = model.K.shape[0]
    mass = _mass(gen, shape.n_kv_heads, n2, "few")
    more = min(n2 - frozen, 37)
    want = model.evict(mass.numpy(), more, 0, not per_head)
    out = pool.sk_session_evict_lowest(sid, mass.cuda(), more, 0, not per_head, mass_out=torch.full((shape.n_kv_heads, n2 + 1), -1.0, device="cuda"))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(out[:, :n2].cpu().numpy(), want)
    assert (out[:, n2:] == -1.0).all()
    _check(pool, sid, model)


@pytest.mark.gpu
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("kind", ["equal", "zero", "few", "rising", "falling", "near", "odd"])
@pytest.mark.parametrize("n", [90, 3000])
def test_orders_of_sums(n, kind, per_head):
    gen = synth.generator(10, stream=n)
    pool, sid, model = _make(D64, gen, n, 16, 11)
    mass = _mass(gen, 4, n, kind)
    before = mass.cuda()
    with np.errstate(invalid="ignore"):
        want = model.evict(mass.numpy(), n // 3, 7, per_head)
    out = pool.sk_session_evict_lowest(sid, before, n // 3, 7, per_head, mass_out=torch.empty_like(before))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(out.cpu().numpy(), want)
    _check(pool, sid, model)


@pytest.mark.gpu
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("kind", ["equal", "zero", "few", "rising", "falling", "near", "odd"])
def test_orders_of_long_lists(kind, per_head):
    """More candidates than one workgroup looks through, and as many that share their leading bits."""
    gen = synth.generator(10, stream=8)
    n = 70001
    pool, sid, model = _make(D64, gen, n, 64, 1003, spare=1200)
    mass = _mass(gen, 4, n, kind)
    place = mass.cuda()
    with np.errstate(invalid="ignore"):
        want = model.evict(mass.numpy(), 30007, 513, per_head)
    pool.sk_session_evict_lowest(sid, place, 30007, 513, per_head)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(place.cpu().numpy(), want)
    _check(pool, sid, model)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,block,frozen,evicted,prefix", [(D64, 16, 0, 0, 500), (D64, 64, 100, 70, 391), (synth.CFG2, 16, 37, 0, 320), (F32_WIDE, 16, 10, 20, 333)])
def test_forks_keep_what_they_share(shape, block, frozen, evicted, prefix):
    """A fork is cut, then its source, then the fork again: blocks that both hold are replaced and never written."""
    gen = synth.generator(10, stream=prefix)
    n = 500
    pool, a, model = _make(shape, gen, n, block, frozen, evicted, spare=2 * (n // block + 3))
    b = pool.sk_session_fork(a, prefix)
    other = Model(shape, model.K[:prefix], model.V[:prefix], min(frozen, prefix))
    for sid, mine, n_evict in ((b, other, 200), (a, model, 150), (b, other, 30), (a, model, 1)):
        mass = _mass(gen, shape.n_kv_heads, mine.K.shape[0])
        want = mine.evict(mass.numpy(), n_evict, 20, True)
        place = mass.cuda()
        pool.sk_session_evict_lowest(sid, place, n_evict, 20)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(place.cpu().numpy(), want)
        _check(pool, a, model)
        _check(pool, b, other)
        _attend(pool, sid, mine, gen)
    pool.sk_session_destroy(a)
    _check(pool, b, other)
    pool.sk_session_destroy(b)
    assert pool.sk_pool_blocks_free() == pool.desc.n_blocks


@pytest.mark.gpu
def test_stream_held_to_a_budget():
    """The operators as they are used together: append, its weights, a question, its weights and log probabilities, eviction down
    to the budget; the model follows with the sums that the library reports."""
    shape = synth.CFG2
    gen = synth.generator(10, stream=5)
    pool, sid, model = _make(shape, gen, 64, 16, spare=80)
    pool.sk_session_freeze(sid, 16)
    model.frozen = 16
    mass = torch.zeros((8, 1200), device="cuda")
    head = torch.randn((32 * 128, 1000), generator=gen).cuda()
    for step, L in enumerate([300, 77, 256, 1, 130, 300]):
        q, k, v = synth.draw_qkv(gen, L, shape)
        out, lse = pool.sk_session_append(sid, q.cuda(), k.cuda(), v.cuda())
        model.K, model.V = np.concatenate([model.K, synth.to_raw(k)]), np.concatenate([model.V, synth.to_raw(v)])
        pool.sk_session_attention_mass(sid, q.cuda(), lse, causal=True, mass_in=mass, keep=0.9)
        q = synth.draw(gen, (9, 32, 128), "bf16")
        out, lse = pool.sk_session_query(sid, q.cuda())
        pool.sk_session_attention_mass(sid, q.cuda(), lse, mass_in=mass)
        logits = out.view(9, -1) @ head
        logprob, _, entropy, top, top_logprob = sk.sk_logprobs(logits, n_top=3)
        i1, i2, _, _, gap = sk.sk_top2(logits)
        torch.cuda.synchronize()
        assert torch.equal(top[:, 0], i1) and torch.equal(top[:, 1], i2) and (entropy >= 0).all()
        n = model.K.shape[0]
        # both calls' rows give every KV head a weight of one each (to the library's 1e-3 in lse)
        if n > 500:
            sums = mass[:, :n].cpu().numpy().copy()
            want = model.evict(sums, n - 500, 64, step % 2 == 0)
            pool.sk_session_evict_lowest(sid, mass, n - 500, 64, step % 2 == 0)
            torch.cuda.synchronize()
            np.testing.assert_array_equal(mass[:, :n].cpu().numpy(), want)
            assert (mass[:, 500:] == 0).all()
        _check(pool, sid, model)
        _attend(pool, sid, model, gen, 33)


@pytest.mark.gpu
def test_blocks_at_the_end_of_a_large_pool():
    """Offsets beyond 2^35: weights and eviction of a session in the last blocks of 40 GiB."""
    shape, n = synth.CFG2, 700
    gen = synth.generator(10, stream=11)
    blocks = (40 << 30) // (64 << 10)
    pool = sk.Pool("bf16", 32, 8, 128, 16, blocks, max_sessions=2, max_session_tokens=4096, max_batch_tokens=8192)
    pool.sk_pool_set_alloc_order(np.arange(blocks, dtype=np.int32)[::-1].copy())
    sid = pool.sk_session_create()
    q, k, v = synth.draw_qkv(gen, n, shape)
    pool.sk_session_append(sid, None, k.cuda(), v.cuda())
    model = Model(shape, synth.to_raw(k), synth.to_raw(v))
    out, lse = pool.sk_session_query(sid, q[:40].cuda())
    mass = pool.sk_session_attention_mass(sid, q[:40].cuda(), lse)
    few = pool.sk_session_attention_mass(sid, q[:5].cuda(), lse[:5])
    torch.cuda.synchronize()
    for T, got in ((40, mass), (5, few)):
        w = torch.exp(torch.einsum("thd,nhd->thn", q[:T].double(), k.double().repeat_interleave(4, 1)) * 128 ** -0.5 - lse[:T].double().cpu()[:, :, None])
        w = w.sum(0).view(8, 4, n).sum(1)
        assert torch.all((got.double().cpu() - w).abs() <= 1e-4 * w)       # rounding: 40 * 4 terms, scores below 2^6: 2^-24 * 2^9 = 3e-5
    want = model.evict(mass.cpu().numpy(), 300, 10, True)
    pool.sk_session_evict_lowest(sid, mass, 300, 10)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(mass.cpu().numpy(), want)
    assert min(pool.sk_session_block_table(sid)) >= blocks - 100
    _check(pool, sid, model)


@pytest.mark.gpu
@pytest.mark.parametrize("site", [sk.SK_SITE_RING, sk.SK_SITE_EVICT_SELECT, sk.SK_SITE_EVICT_MOVE])
def test_call_that_fails_on_the_device_leaves_the_session(site):
    gen = synth.generator(10, stream=6)
    pool, a, model = _make(D64, gen, 300, 16, spare=40)
    b = pool.sk_session_fork(a, 300)
    mass = _mass(gen, 4, 300)
    place = mass.cuda()
    free = pool.sk_pool_blocks_free()
    pool.sk_pool_inject_failure(site, 1)
    with pytest.raises(sk.SkError) as e:
        pool.sk_session_evict_lowest(b, place, 100)
    assert e.value.status == sk.SK_E_HIP
    torch.cuda.synchronize()
    assert torch.equal(place.cpu(), mass) and pool.sk_pool_blocks_free() == free
    _check(pool, a, model)
    _check(pool, b, model)
    other = Model(D64, model.K, model.V)
    other.evict(mass.numpy(), 100, 0, True)
    pool.sk_session_evict_lowest(b, place, 100)
    _check(pool, b, other)
    _check(pool, a, model)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,block,seed", [(D64, 16, 0), (D64, 16, 1), (D64, 64, 2), (synth.CFG1, 16, 3), (ODD, 16, 4), (D64, 256, 5)])
def test_random_walk_with_other_calls(shape, block, seed):
    """Sessions of a pool that is often full: appended to, cut in every way there is, forked, destroyed; all of them read back after each eviction."""
    rng, gen = np.random.default_rng(seed), synth.generator(10, stream=40 + seed)
    blocks = 2400 // block
    pool = sk.Pool(shape.dtype, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, block, blocks, max_sessions=5, max_batch_tokens=1024, kv_fill=0xFF)
    pool.sk_pool_set_alloc_order(synth.permutation(gen, blocks))
    models, refused, evicted = {}, 0, 0
    for step in range(90):
        sid = int(rng.choice(sorted(models))) if models else None
        op = rng.choice(["append", "append", "evict", "evict", "evict", "oldest", "truncate", "fork", "freeze", "destroy"], p=[.2, .15, .2, .1, .1, .06, .05, .07, .05, .02])
        try:
            if sid is None or (op == "append" and len(models) < 5 and rng.random() < 0.3):
                sid = pool.sk_session_create()
                models[sid] = Model(shape, *(synth.to_raw(x[:0]) for x in synth.draw_qkv(gen, 1, shape)[1:]))
                op = "append"
            m = models[sid]
            n = m.K.shape[0]
            if op == "append":
                _, k, v = synth.draw_qkv(gen, int(rng.integers(1, 500)), shape)
                pool.sk_session_append(sid, None, k.cuda(), v.cuda())
                m.K, m.V = np.concatenate([m.K, synth.to_raw(k)]), np.concatenate([m.V, synth.to_raw(v)])
            elif op == "evict":
                recent = int(rng.integers(0, 80))
                count = int(rng.integers(0, max(n - m.frozen - recent, 0) + 1))
                per_head, in_place = bool(rng.integers(2)), bool(rng.integers(2))
                mass = _mass(gen, shape.n_kv_heads, n + 2, str(rng.choice(["spread", "few", "near", "equal"])))
                place = mass.cuda()
                out = pool.sk_session_evict_lowest(sid, place, count, min(recent, n), per_head, mass_out=None if in_place else torch.zeros_like(place))
                torch.cuda.synchronize()
                want = m.evict(mass[:, :n].numpy(), count, min(recent, n), per_head)
                np.testing.assert_array_equal(out[:, :n].cpu().numpy(), want)
                evicted += count > 0
                for other in models:
                    _check(pool, other, models[other])
            elif op == "oldest":
                count = int(rng.integers(0, max(n - m.frozen, 0) + 1)) // 3
                pool.sk_session_evict_oldest(sid, count)
                m.K, m.V = (np.concatenate([x[:m.frozen], x[m.frozen + count:]]) for x in (m.K, m.V))
            elif op == "truncate":
                count = int(rng.integers(n // 2, n + 1))
                pool.sk_session_truncate(sid, count)
                m.K, m.V, m.frozen = m.K[:count], m.V[:count], min(m.frozen, count)
            elif op == "fork" and len(models) < 5:
                prefix = int(rng.integers(0, n + 1))
                new = pool.sk_session_fork(sid, prefix)
                models[new] = Model(shape, m.K[:prefix], m.V[:prefix], min(m.frozen, prefix))
            elif op == "freeze":
                count = int(rng.integers(m.frozen, min(m.frozen + 100, n) + 1)) if n >= m.frozen else m.frozen
                pool.sk_session_freeze(sid, count)
                m.frozen = count
            elif op == "destroy":
                pool.sk_session_destroy(sid)
                del models[sid]
        except sk.SkError as e:
            assert e.status == (sk.SK_E_INVAL if op == "freeze" else sk.SK_E_NOMEM), (step, op)
            refused += 1
    assert evicted > 5 and refused > 0
    for sid, m in models.items():
        _check(pool, sid, m)
        if m.K.shape[0]:
            _attend(pool, sid, m, gen)
        pool.sk_session_destroy(sid)
    assert pool.sk_pool_blocks_free() == blocks


# ---- host half, without a GPU ---------------------------------------------------------------------------

def _meta(**kw):
    args = dict(dtype="bf16", n_q_heads=8, n_kv_heads=4, head_dim=64, block_tokens=16, n_blocks=64, max_sessions=4, metadata_only=True)
    return sk.Pool(**{**args, **kw})


def _state(p, sids):
    return [(p.sk_session_length(s), p.sk_session_block_table(s)) for s in sids], p.sk_pool_blocks_free()


def test_host_half_and_refusals_without_a_gpu():
    p = _meta()
    a = p.sk_session_create()
    p.reserve(a, 200)
    p.sk_session_freeze(a, 30)
    free = p.sk_pool_blocks_free()
    before = _state(p, [a])
    for n_evict, n_recent in ((171, 0), (100, 71), (1, 170), (1, 500), (-1, 0), (1, -1)):
        with pytest.raises(sk.SkError) as e:
            p.sk_session_evict_lowest(a, None, n_evict, n_recent)
        assert e.value.status == sk.SK_E_INVAL
    with pytest.raises(sk.SkError) as e:
        p.sk_session_evict_lowest(3, None, 0)
    assert e.value.status == sk.SK_E_BADSESSION
    assert sk.lib().sk_session_evict_lowest(None, 0, None, 0, 0, 0, 0, None, 0, None) == sk.SK_E_INVAL
    assert _state(p, [a]) == before
    p.sk_session_evict_lowest(a, None, 0, 500)                # nothing to evict: as it was
    assert _state(p, [a]) == before
    p.sk_session_evict_lowest(a, None, 100, 70)
    assert p.sk_session_length(a) == 100 and p.sk_pool_blocks_free() == free + 6
    table = p.sk_session_block_table(a)                       # what is frozen stays where it is, the rest goes to free blocks
    assert table[:1] == before[0][0][1][:1] and len(table) == 7 and not set(table[1:]) & set(before[0][0][1])
    p.sk_session_evict_oldest(a, 20)                          # and the window goes on behind it
    p.sk_session_evict_lowest(a, None, 50)
    assert p.sk_session_length(a) == 30 and p.sk_pool_get_stats()["tokens_evicted"] == 170
    with pytest.raises(sk.SkError):
        p.sk_session_evict_lowest(a, None, 1)                 # only the frozen tokens are left
    p.reserve(a, 5)
    assert p.sk_session_length(a) == 35


def test_a_full_pool_needs_no_blocks():
    p = _meta(n_blocks=15)
    a = p.sk_session_create()
    p.reserve(a, 200)                                         # 13 blocks, 2 free
    table = p.sk_session_block_table(a)
    p.sk_session_evict_lowest(a, None, 100, 70)               # 7 blocks would be written: in place
    assert p.sk_session_length(a) == 100 and p.sk_session_block_table(a) == table[:7] and p.sk_pool_blocks_free() == 8
    p.sk_session_evict_lowest(a, None, 1)
    assert p.sk_session_length(a) == 99 and not set(p.sk_session_block_table(a)) & set(table[:7]) and p.sk_pool_blocks_free() == 8


def test_shared_blocks_are_replaced_and_counted():
    p = _meta(n_blocks=20)
    a = p.sk_session_create()
    p.reserve(a, 160)                                         # 10 blocks
    p.sk_session_freeze(a, 40)
    b = p.sk_session_fork(a, 155)                             # shares 9, holds a copy of the last: 9 free
    tables = _state(p, [a, b])[0]
    assert p.sk_pool_blocks_free() == 9
    p.sk_session_evict_lowest(b, None, 20)                    # 135 tokens, blocks 2..8 are replaced, the last one goes
    assert p.sk_session_length(b) == 135 and p.sk_pool_blocks_free() == 9 - 7 + 1
    tb = p.sk_session_block_table(b)
    assert tb[:2] == tables[0][1][:2] and not set(tb[2:]) & set(tables[0][1]) and p.sk_session_block_table(a) == tables[0][1]
    c = p.sk_session_fork(a, 160)
    before = _state(p, [a, b, c])
    with pytest.raises(sk.SkError) as e:
        p.sk_session_evict_lowest(c, None, 1)                 # 8 blocks to replace, 3 free
    assert e.value.status == sk.SK_E_NOMEM and _state(p, [a, b, c]) == before
    p.sk_session_evict_lowest(c, None, 80)                    # 80 left: blocks 2, 3 and 4
    assert p.sk_pool_blocks_free() == 0
    for s in (a, b, c):
        p.sk_session_destroy(s)
    assert p.sk_pool_blocks_free() == 20


@pytest.mark.parametrize("site", [sk.SK_SITE_RING, sk.SK_SITE_EVICT_SELECT, sk.SK_SITE_EVICT_MOVE])
def test_call_that_fails_changes_nothing(site):
    p = _meta()
    a = p.sk_session_create()
    p.reserve(a, 200)
    b = p.sk_session_fork(a, 200)
    before = _state(p, [a, b])
    p.sk_pool_inject_failure(site, 1)
    with pytest.raises(sk.SkError) as e:
        p.sk_session_evict_lowest(b, None, 50)
    assert e.value.status == sk.SK_E_HIP and _state(p, [a, b]) == before
    p.sk_session_evict_lowest(b, None, 50)
    assert p.sk_session_length(b) == 150


def test_injected_sites_end_with_the_eviction():
    p = _meta()
    assert sk.lib().sk_pool_inject_failure(p.h, sk.SK_SITE_EVICT_MOVE + 1, 1) == sk.SK_E_INVAL
    assert sk.lib().sk_pool_inject_failure(p.h, -1, 1) == sk.SK_E_INVAL


@pytest.mark.gpu
def test_refusals():
    pool, sid, model = _make(D64, synth.generator(10), 100, 16)
    L, a = sk.lib(), 1 << 20                                  # an address that a refused call does not use
    good = dict(i=a, si=128, n=10, r=0, o=a, so=128)

    def call(**kw):
        x = {**good, **kw}
        return L.sk_session_evict_lowest(pool.h, sid, x["i"], x["si"], x["n"], x["r"], 1, x["o"], x["so"], None)

    for bad in (dict(i=None), dict(i=a + 2), dict(si=99), dict(o=a + 1), dict(so=99), dict(so=129), dict(o=a + 400), dict(o=a - 4), dict(o=a + 128 * 4),
                dict(n=101), dict(n=50, r=51), dict(n=-1), dict(r=-1)):
        assert call(**bad) == sk.SK_E_INVAL, bad
    _check(pool, sid, model)
    empty = pool.sk_session_create()
    assert L.sk_session_evict_lowest(pool.h, empty, None, 0, 0, 5, 1, None, 0, None) == sk.SK_OK
    assert L.sk_session_evict_lowest(pool.h, empty, None, 0, 1, 0, 1, None, 0, None) == sk.SK_E_INVAL
    # no sums kept
    mass = _mass(synth.generator(10, stream=7), 4, 100).cuda()
    assert L.sk_session_evict_lowest(pool.h, sid, ctypes.c_void_p(mass.data_ptr()), 100, 10, 0, 0, None, 0, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == sk.SK_OK
    model.evict(mass.cpu().numpy(), 10, 0, False)
    _check(pool, sid, model)


MANY_HEADS = synth.Shape("bf16", 32, 32, 64)


def _make_with_a_small_workspace(gen, n, frozen, evicted):
    """A session of MANY_HEADS, 8 KiB a token, in a pool that has too few free blocks and a workspace that holds about 8,200 tokens of it."""
    shape, blocks = MANY_HEADS, -(-(n + evicted) // 16) + 9
    pool = sk.Pool("bf16", 32, 32, 64, 16, blocks, max_sessions=3, max_batch_tokens=64, kv_fill=0xFF)
    pool.sk_pool_set_alloc_order(synth.permutation(gen, blocks))
    sid = pool.sk_session_create()
    k, v = (torch.randint(-0x7000, 0x7000, (n + evicted, 32, 64), generator=gen, dtype=torch.int16).view(torch.bfloat16) for _ in range(2))
    kd, vd = k.cuda(), v.cuda()
    for t in range(0, n + evicted, 64):
        pool.sk_session_append(sid, None, kd[t:t + 64], vd[t:t + 64])
    pool.sk_session_freeze(sid, frozen)
    pool.sk_session_evict_oldest(sid, evicted)
    k, v = (synth.to_raw(torch.cat([x[:frozen], x[frozen + evicted:]])) for x in (k, v))
    return pool, sid, Model(shape, k, v, frozen)


@pytest.mark.gpu
@pytest.mark.parametrize("n,n_evict,n_recent,per_head", [(20011, 700, 50, True), (19001, 6000, 0, True), (20011, 3333, 10000, False)])
def test_moves_in_several_stretches(n, n_evict, n_recent, per_head):
    """Too few free blocks, and a workspace that holds less than half of what stays."""
    gen = synth.generator(10, stream=n_evict)
    pool, sid, model = _make_with_a_small_workspace(gen, n, 23, 11)
    launches = pool.sk_pool_get_stats()["launches"]
    mass = _mass(gen, 32, n)
    place = mass.cuda()
    want = model.evict(mass.numpy(), n_evict, n_recent, per_head)
    pool.sk_session_evict_lowest(sid, place, n_evict, n_recent, per_head)
    torch.cuda.synchronize()
    assert pool.sk_pool_get_stats()["launches"] - launches >= 1 + 2 * 2 + (not per_head)       # selection, and move and put of each stretch
    np.testing.assert_array_equal(place.cpu().numpy(), want)
    _check(pool, sid, model)


@pytest.mark.gpu
@pytest.mark.parametrize("launch", [2, 3, 4])
def test_a_launch_that_fails_between_the_moves(launch):
    """Too few free blocks, sums in place: the launches are move and put, stretch by stretch.  Up to the first put nothing has changed; behind
    it the tokens that are not frozen are undefined, and all else is as it was."""
    n, frozen, n_evict = 19001, 23, 1500
    gen = synth.generator(10, stream=launch)
    pool, sid, model = _make_with_a_small_workspace(gen, n, frozen, 11)
    fork = pool.sk_session_fork(sid, 60)
    other = Model(MANY_HEADS, model.K[:60], model.V[:60])
    mass = _mass(gen, 32, n + 3)
    place = mass.cuda()

    def state():
        return pool.sk_session_length(sid), pool.sk_session_block_table(sid), pool.sk_pool_blocks_free(), pool.sk_pool_get_stats()["tokens_evicted"]

    before = state()
    pool.sk_pool_inject_failure(sk.SK_SITE_EVICT_MOVE, launch)
    with pytest.raises(sk.SkError) as e:
        pool.sk_session_evict_lowest(sid, place, n_evict, 5)
    assert e.value.status == sk.SK_E_HIP
    torch.cuda.synchronize()
    assert state() == before and torch.equal(place.cpu(), mass)
    _check(pool, fork, other)
    if launch == 2:
        _check(pool, sid, model)
        want = model.evict(mass[:, :n].numpy(), n_evict, 5, True)
        pool.sk_session_evict_lowest(sid, place, n_evict, 5)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(place[:, :n].cpu().numpy(), want)
    else:
        pool.sk_session_truncate(sid, frozen)
        model = Model(MANY_HEADS, model.K[:frozen], model.V[:frozen], frozen)
    _check(pool, sid, model)
    _check(pool, fork, other)


@pytest.mark.gpu
@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("shape,n,block,n_evict,per_head", [(D64, 700, 16, 300, True), (ODD, 900, 64, 77, False), (F32_WIDE, 600, 16, 64, True), (D64, 33000, 64, 1000, False)])
def test_sums_that_are_not_kept(shape, n, block, n_evict, per_head, room):
    gen = synth.generator(10, stream=n)
    pool, sid, model = _make(shape, gen, n, block, 20, 5, spare=9 + (n // block if room else 0))
    mass = _mass(gen, shape.n_kv_heads, n + 1)
    place = mass.cuda()
    model.evict(mass[:, :n].numpy(), n_evict, 6, per_head)
    assert pool.sk_session_evict_lowest(sid, place, n_evict, 6, per_head, mass_out=False) is None
    torch.cuda.synchronize()
    assert torch.equal(place.cpu(), mass)
    _check(pool, sid, model)


@pytest.mark.gpu
def test_sums_of_a_stream_grow_by_a_weight_of_one_a_row():
    """Sums in place over appends, queries and evictions: every row of a call adds a weight of one to each KV head, to the 1e-3 that the
    library states for lse, and an eviction takes away what the tokens that leave had."""
    shape = synth.CFG2
    gen = synth.generator(10, stream=13)
    pool, sid, model = _make(shape, gen, 64, 16, spare=80)
    mass = torch.zeros((8, 1200), device="cuda")
    total = torch.zeros(8, dtype=torch.float64)
    for L in (300, 1, 77, 256):
        q, k, v = (x.cuda() for x in synth.draw_qkv(gen, L, shape))
        _, lse = pool.sk_session_append(sid, q, k, v)
        pool.sk_session_attention_mass(sid, q, lse, causal=True, mass_in=mass)
        for T in (9, 32):
            _, lse = pool.sk_session_query(sid, q[:T]) if T <= L else pool.sk_session_query(sid, q[:1].repeat(T, 1, 1))
            pool.sk_session_attention_mass(sid, q[:T] if T <= L else q[:1].repeat(T, 1, 1), lse, mass_in=mass)
        torch.cuda.synchronize()
        grown = mass.double().sum(1).cpu() - total
        assert torch.all((grown / ((L + 41) * shape.group) - 1).abs() <= 1.1e-3)
        n = pool.sk_session_length(sid)
        if n > 300:
            pool.sk_session_evict_lowest(sid, mass, n - 300, 64)
        total = mass.double().sum(1).cpu()


@pytest.mark.gpu
def test_a_workspace_that_holds_no_stretch_is_an_error():
    """Thousands of KV heads and a small batch limit: 64 tokens do not fit the workspace.  Without free blocks the call is refused and changes
    nothing, with them it needs none."""
    heads, n = 5000, 100
    shape = synth.Shape("bf16", heads, heads, 64)
    pool = sk.Pool("bf16", heads, heads, 64, 16, 8, max_sessions=1, max_batch_tokens=1)
    sid = pool.sk_session_create()
    k = torch.randint(-0x7000, 0x7000, (n, heads, 64), generator=synth.generator(10), dtype=torch.int16).view(torch.bfloat16)
    for t in range(n):
        pool.sk_session_append(sid, None, k[t:t + 1].cuda(), k[t:t + 1].cuda())
    model = Model(shape, synth.to_raw(k), synth.to_raw(k))
    mass = _mass(synth.generator(10, stream=1), heads, n)
    place = mass.cuda()
    table, free = pool.sk_session_block_table(sid), pool.sk_pool_blocks_free()
    for per_head in (True, False):
        with pytest.raises(sk.SkError) as e:
            pool.sk_session_evict_lowest(sid, place, 10, 0, per_head)
        assert e.value.status == sk.SK_E_WORKSPACE
    torch.cuda.synchronize()
    assert pool.sk_session_block_table(sid) == table and pool.sk_pool_blocks_free() == free == 1 and torch.equal(place.cpu(), mass)
    _check(pool, sid, model)
    pool.sk_session_truncate(sid, 17)
    model.K, model.V = model.K[:17], model.V[:17]
    want = model.evict(mass[:, :17].numpy(), 3, 2, True)
    pool.sk_session_evict_lowest(sid, place, 3, 2)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(place[:, :17].cpu().numpy(), want)
    _check(pool, sid, model)
