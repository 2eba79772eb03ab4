"""Seeded random walks over sessions whose keys are rotated: rotated and plain appends, steps, forks, truncations, evictions by age and by weight, and
shifts by one number, by token and by head, each compared with arrays that are kept beside them; what a shift has written is checked against the
definition in 64 bits from the keys before it (tests/test_rotation.py says how far it may be off), everything else bit for bit."""
import numpy as np
import pytest
import torch

import paper_2605_13784_amd as sk
from workloads import synth
from test_rotation import _check, _pool, _rows

pytestmark = pytest.mark.gpu

LAYERS = [("bf16", 8, 2, 128), ("bf16", 6, 3, 64), ("f32", 4, 2, 64), ("bf16", 32, 8, 128)]


@pytest.mark.parametrize("seed", range(9100, 9124))
def test_random_operations(seed):
    rng, gen = np.random.default_rng(seed), synth.generator(25, stream=seed)
    layer = LAYERS[seed % len(LAYERS)]
    dtype, _, hkv, d = layer
    block = int(rng.choice([16, 64, 256]))
    rotary, interleaved = [(d, False), (d, True), (48, False), (32, True)][int(rng.integers(4))]
    factor = float(rng.choice([1.0, 1.25]))
    pool = _pool(layer, rotary, interleaved, block=block, n_blocks=12000 // block, max_sessions=4, factor=factor, max_batch_tokens=4096)
    held, frozen = {}, {}                                      # session -> K, V on the host

    def check(sid):
        k, v = (x.cpu() for x in pool.sk_session_gather(sid))
        assert k.shape[0] == pool.sk_session_length(sid)
        assert torch.equal(k.view(torch.int16), held[sid][0].view(torch.int16)) and torch.equal(v.view(torch.int16), held[sid][1].view(torch.int16))

    def grow(sid, k, v):
        held[sid] = tuple(torch.cat([a, b]).contiguous() for a, b in zip(held[sid], (k, v)))

    first = pool.sk_session_create()
    held[first], frozen[first] = tuple(torch.zeros((0, hkv, d), dtype=synth.torch_dtype(dtype)) for _ in range(2)), 0
    for _ in range(40):
        sid = int(rng.choice(sorted(held)))
        n, kind = held[sid][0].shape[0], int(rng.integers(10))
        if kind <= 2 or n == 0:                                # a rotated append, with attention, without, or without q
            T = int(rng.choice([1, 2, 17, 60, 200, 700, 1500]))
            if sum(len(h[0]) for h in held.values()) + T > 9000:
                continue
            q, k, v = (x.cuda() for x in _rows(gen, T, layer))
            positions = torch.randint(-1000, 1 << 20, (T,), generator=gen, dtype=torch.int32).cuda() if rng.random() < 0.5 else None
            pos0 = 0 if positions is not None else int(rng.integers(1 << 20))
            _, want = pool.sk_rotate(None, k, positions=positions, pos0=pos0)
            at = positions.cpu().numpy() if positions is not None else pos0 + np.arange(T)
            _check(want, k.cpu(), at[:, None], rotary, interleaved, dtype, factor)
            pool.sk_session_append_rotated(sid, q if rng.random() < 0.7 else None, k, v, positions=positions, pos0=pos0, attend=rng.random() < 0.6)
            grow(sid, want.cpu(), v.cpu())
        elif kind == 3 and len(held) < 4:
            m = int(rng.integers(n + 1))
            fork = pool.sk_session_fork(sid, m)
            held[fork], frozen[fork] = tuple(x[:m].contiguous() for x in held[sid]), min(frozen[sid], m)
        elif kind == 4:
            m = n - int(rng.integers(n // 3 + 1))
            pool.sk_session_truncate(sid, m)
            held[sid], frozen[sid] = tuple(x[:m].contiguous() for x in held[sid]), min(frozen[sid], m)
        elif kind == 5:                                        # the oldest leave, the others move up
            f, m = frozen[sid], int(rng.integers((n - frozen[sid]) // 2 + 1))
            pool.sk_session_evict_oldest(sid, m)
            held[sid] = tuple(torch.cat([x[:f], x[f + m:]]) for x in held[sid])
            n -= m
            check(sid)
            pool.sk_session_shift(sid, -m, first=f)
            k = pool.sk_session_gather(sid)[0].cpu()
            _check(k[f:], held[sid][0][f:], np.full((n - f, 1), -m), rotary, interleaved, dtype)
            held[sid] = (torch.cat([held[sid][0][:f], k[f:]]), held[sid][1])
        elif kind == 6:                                        # those of lowest weight, head by head; every head's own numbers
            f, m = frozen[sid], int(rng.integers((n - frozen[sid]) // 3 + 1))
            mass = torch.rand((hkv, n), generator=gen)
            try:
                pool.sk_session_evict_lowest(sid, mass.cuda(), m, mass_out=False)
            except sk.SkError as e:
                assert e.status == sk.SK_E_NOMEM
                continue
            stay = np.ones((hkv, n), bool)
            for g in range(hkv):
                stay[g, f + np.argsort(mass[g, f:].numpy(), kind="stable")[:m]] = False
            kept = np.stack([np.nonzero(stay[g])[0] for g in range(hkv)])                # [Hkv][n - m]
            held[sid] = tuple(torch.stack([x[torch.from_numpy(kept[g]), g] for g in range(hkv)], 1).contiguous() for x in held[sid])
            check(sid)
            delta = torch.from_numpy((np.arange(n - m)[None, :] - kept).astype(np.int32))
            try:
                pool.sk_session_shift(sid, delta.cuda())
            except sk.SkError as e:
                assert e.status == sk.SK_E_NOMEM
                check(sid)
                continue
            k = pool.sk_session_gather(sid)[0].cpu()
            _check(k, held[sid][0], delta.numpy().T, rotary, interleaved, dtype)
            held[sid] = (k, held[sid][1])
        elif kind == 7:                                        # a stretch by anything
            a = int(rng.integers(n + 1))
            m = int(rng.integers(n - a + 1))
            delta = torch.randint(-3000, 3000, (m,), generator=gen, dtype=torch.int32)
            try:
                pool.sk_session_shift(sid, delta.cuda(), first=a, count=m)
            except sk.SkError as e:
                assert e.status == sk.SK_E_NOMEM
                check(sid)
                continue
            k = pool.sk_session_gather(sid)[0].cpu()
            _check(k[a:a + m], held[sid][0][a:a + m], delta.numpy()[:, None], rotary, interleaved, dtype)
            held[sid] = (torch.cat([held[sid][0][:a], k[a:a + m], held[sid][0][a + m:]]), held[sid][1])
        elif kind == 8:                                        # a step over all sessions
            ids = sorted(held)
            T = [int(rng.integers(40)) for _ in ids]
            T[0] += 1
            ops = [int(rng.choice([sk.SK_OP_APPEND, sk.SK_OP_QUERY_B] + ([sk.SK_OP_QUERY_A] if held[s][0].shape[0] else []))) for s in ids]
            cu = np.concatenate([[0], np.cumsum(T)])
            q, k, v = (x.cuda() for x in _rows(gen, int(cu[-1]), layer))
            positions = torch.randint(0, 1 << 20, (int(cu[-1]),), generator=gen, dtype=torch.int32).cuda()
            want = pool.sk_rotate(None, k, positions=positions)[1].cpu()
            pool.sk_batch_step_rotated(ids, ops, cu, positions, q, k, v)
            for s, o, a, b in zip(ids, ops, cu, cu[1:]):
                if o == sk.SK_OP_APPEND:
                    grow(s, want[a:b], v[a:b].cpu())
        elif len(held) > 1 and rng.random() < 0.5:
            pool.sk_session_destroy(sid)
            held.pop(sid)
        elif frozen[sid] == 0 and n > 4:
            try:
                pool.sk_session_freeze(sid, 3)
                frozen[sid] = 3
            except sk.SkError as e:                            # tokens behind it have left already
                assert e.status == sk.SK_E_INVAL
        for s in sorted(held):
            check(s)
    for s in sorted(held):                                     # what a query reads is what the cache holds
        n = held[s][0].shape[0]
        if n:
            q = _rows(gen, 3, layer)[0].cuda()
            pool2 = _pool(layer, rotary, interleaved, block=16, n_blocks=n // 16 + 1)
            fresh = pool2.sk_session_create()
            for t in range(0, n, 4096):
                pool2.sk_session_append(fresh, None, held[s][0][t:t + 4096].cuda(), held[s][1][t:t + 4096].cuda())
            a, b = pool.sk_session_query(s, q)[1], pool2.sk_session_query(fresh, q)[1]
            assert torch.allclose(a, b, atol=1e-3, rtol=0)     # (cut otherwise: the sums' order differs)
