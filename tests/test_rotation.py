"""Position rotation: rows beside the cache, on the way into it, and keys turned on where they lie, against the definition in 64 bits.

Tolerance of a turned element x cos a - y sin a (or x sin a + y cos a), both times the factor.  The angle's part of a turn is off by 2^-32 of
one from the phase's lower bits and 2^-34 from the step (times 2 pi: below 2^-28); the rest of a quadrant, at most pi / 4, loses 2^-24 of itself on its way
to a float, 2^-23 with the constant and the product by it; the series' next terms are below 2^-28, its last operations round by 2^-24 each and the inner
ones by less than that together.  So a sine or cosine is within 2^-22 of itself absolutely, with the factor's product 2^-24 more, and the two
products and their sum round by 2^-24 of |x| + |y| at most three times: 2^-21 factor (|x| + |y|).  Then one rounding to the pool's type."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2605_13784_amd as sk
from workloads import synth

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
LAYERS = [("bf16", 8, 2, 128), ("bf16", 6, 2, 64), ("bf16", 32, 8, 128), ("bf16", 5, 1, 64), ("f32", 4, 4, 64), ("f32", 6, 2, 128)]
TURNS = [(128, False), (128, True), (64, False), (64, True), (32, False), (48, True), (16, False), (112, False)]


def _freqs(rotary, base=10000.0):
    return base ** (-np.arange(0, rotary, 2) / rotary)


def _pool(layer, rotary, interleaved, block=16, n_blocks=64, factor=1.0, base=10000.0, **kw):
    pool = sk.Pool(*layer, block, n_blocks, **kw)
    pool.sk_pool_set_rotation(_freqs(rotary, base), interleaved=interleaved, factor=factor)
    return pool


def _expected(x, position, rotary, interleaved, factor=1.0, base=10000.0):
    """x [.., d] on the host, position broadcasting against [..] -> turned in 64 bits, |x| + |y| of each element's pair (0 beside them)."""
    x = x.double().numpy()
    pairs = [(2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2) for i in range(rotary // 2)]
    a, b = [p[0] for p in pairs], [p[1] for p in pairs]
    angle = np.asarray(position, np.float64)[..., None] * _freqs(rotary, base)
    out, size = x.copy(), np.zeros_like(x)
    out[..., a] = factor * (x[..., a] * np.cos(angle) - x[..., b] * np.sin(angle))
    out[..., b] = factor * (x[..., a] * np.sin(angle) + x[..., b] * np.cos(angle))
    size[..., a] = size[..., b] = abs(factor) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return out, size


def _check(got, x, position, rotary, interleaved, dtype, factor=1.0, base=10000.0):
    want, size = _expected(x, position, rotary, interleaved, factor, base)
    tol = 2.0 ** -21 * size
    tol = tol + np.where(size > 0, HALF_STEP[dtype] * (np.abs(want) + tol), 0.0)
    diff = np.abs(got.cpu().double().numpy() - want)
    assert np.all(diff <= tol), (diff - tol).max()


def _rows(gen, T, layer):
    dtype, hq, hkv, d = layer
    return synth.draw(gen, (T, hq, d), dtype), synth.draw(gen, (T, hkv, d), dtype), synth.draw(gen, (T, hkv, d), dtype)


# ---- without a GPU -----------------------------------------------------------------------------------

def _host_pool(n_blocks=32, **kw):
    return sk.Pool("bf16", 4, 2, 64, 16, n_blocks, max_sessions=4, metadata_only=True, **kw)


def _status(f, *a, **kw):
    try:
        f(*a, **kw)
        return sk.SK_OK
    except sk.SkError as e:
        return e.status


def test_a_rotation_is_checked():
    pool = _host_pool()
    assert _status(pool.sk_pool_set_rotation, np.ones(4)) == sk.SK_E_SHAPE            # 8 dimensions
    assert _status(pool.sk_pool_set_rotation, np.ones(0)) == sk.SK_E_SHAPE
    assert _status(pool.sk_pool_set_rotation, np.ones(40)) == sk.SK_E_SHAPE           # more than a row has
    for bad in (np.nan, np.inf, 1e7, -1e7):
        f = np.ones(16)
        f[5] = bad
        assert _status(pool.sk_pool_set_rotation, f) == sk.SK_E_INVAL
    assert _status(pool.sk_pool_set_rotation, np.ones(16), factor=float("nan")) == sk.SK_E_INVAL
    assert _status(pool.sk_pool_set_rotation, np.ones(16), factor=float("inf")) == sk.SK_E_INVAL
    assert sk.lib().sk_pool_set_rotation(pool.h, 32, 0, None, 1.0) == sk.SK_E_INVAL
    assert sk.lib().sk_pool_set_rotation(None, 32, 0, None, 1.0) == sk.SK_E_INVAL
    sid = pool.sk_session_create()
    pool.reserve(sid, 20)
    L, p = sk.lib(), 4096
    # none of the refused ones counts
    assert L.sk_rotate(pool.h, p, None, 1, None, 0, p, None, None) == sk.SK_E_INVAL
    assert L.sk_session_append_rotated(pool.h, sid, None, None, None, 1, None, 0, None, None, sk.SK_F32, None, None) == sk.SK_E_INVAL
    assert _status(pool.sk_session_shift, sid, 1) == sk.SK_E_INVAL
    pool.sk_pool_set_rotation(np.ones(32), interleaved=True)
    assert L.sk_rotate(pool.h, p, None, 1, None, 0, p, None, None) == sk.SK_E_NODEVICE
    assert L.sk_rotate(pool.h, p, None, -1, None, 0, p, None, None) == sk.SK_E_INVAL
    most = (1 << 27) // pool.Hq
    assert L.sk_rotate(pool.h, p, None, most + 1, None, 0, p, None, None) == sk.SK_E_INVAL
    assert L.sk_rotate(pool.h, p, None, most, None, 0, p, None, None) == sk.SK_E_NODEVICE
    assert L.sk_rotate(pool.h, None, None, 0, None, 0, None, None, None) == sk.SK_OK
    assert _status(pool.sk_session_shift, sid, 1) == sk.SK_OK


def test_stretches_of_a_shift_are_checked():
    pool = _host_pool()
    pool.sk_pool_set_rotation(np.ones(32))
    sid = pool.sk_session_create()
    pool.reserve(sid, 100)
    for first, count in ((-1, 5), (0, -1), (0, 101), (101, 0), (100, 1), (1 << 62, 1 << 62)):
        assert _status(pool.sk_session_shift, sid, 3, first, count) == sk.SK_E_INVAL
    assert _status(pool.sk_session_shift, sid, 3, 100, 0) == sk.SK_OK
    assert _status(pool.sk_session_shift, 3, 3, 0, 0) == sk.SK_E_BADSESSION
    L = sk.lib()
    assert L.sk_session_shift(pool.h, sid, 0, 10, 0, 4098, 10, None) == sk.SK_E_INVAL      # not aligned to its elements
    assert L.sk_session_shift(pool.h, sid, 0, 10, 0, 4096, 9, None) == sk.SK_E_INVAL       # rows that meet


def test_append_rotated_on_the_host():
    pool = _host_pool(8)
    pool.sk_pool_set_rotation(np.ones(32))
    sid = pool.sk_session_create()
    L = sk.lib()

    def append(n, pos0=0):
        return L.sk_session_append_rotated(pool.h, sid, None, None, None, n, None, pos0, None, None, sk.SK_F32, None, None)

    assert append(40) == sk.SK_OK and pool.sk_session_length(sid) == 40
    assert append(100) == sk.SK_E_NOMEM and append(-1) == sk.SK_E_INVAL and append(2, 2 ** 31 - 2) == sk.SK_OK
    assert append(2, 2 ** 31 - 1) == sk.SK_E_INVAL and append(1, -2 ** 31) == sk.SK_OK
    assert pool.sk_session_length(sid) == 43 and append(0) == sk.SK_OK
    for site in (sk.SK_SITE_SCATTER, sk.SK_SITE_ATTENTION):
        pool.sk_pool_inject_failure(site)
        before = pool.sk_session_block_table(sid), pool.sk_pool_blocks_free()
        assert append(30) == sk.SK_E_HIP
        assert pool.sk_session_length(sid) == 43 and (pool.sk_session_block_table(sid), pool.sk_pool_blocks_free()) == before
    pool.sk_pool_inject_failure(0, 0)


def test_a_short_append_comes_past_as_many_sites_as_it_has_launches():
    """A metadata-only pool visits the sites of failures as a device pool does: once where the attention launch turns the rows and commits them,
    twice where a launch in front of it turns them (the commit is the attention launch's in both)."""
    for pairs, launches in ((32, 1), (16, 1), (8, 2)):
        pool = _host_pool(8)
        pool.sk_pool_set_rotation(np.ones(pairs))
        sid = pool.sk_session_create()
        pool.reserve(sid, 20)
        L = sk.lib()

        def append():
            return L.sk_session_append_rotated(pool.h, sid, None, None, None, 1, None, 20, None, None, sk.SK_F32, None, None)

        before = pool.sk_session_block_table(sid), pool.sk_pool_blocks_free()
        for countdown in range(1, launches + 1):
            pool.sk_pool_inject_failure(sk.SK_SITE_SCATTER, countdown)
            assert append() == sk.SK_E_HIP
            assert pool.sk_session_length(sid) == 20 and (pool.sk_session_block_table(sid), pool.sk_pool_blocks_free()) == before
        pool.sk_pool_inject_failure(sk.SK_SITE_SCATTER, launches + 1)
        assert append() == sk.SK_OK and pool.sk_session_length(sid) == 21
        pool.sk_pool_inject_failure(0, 0)


class _OnCard:
    """What the binding looks at of a tensor, with nothing behind it."""
    is_cuda = True

    def __init__(self, n, dtype=torch.bfloat16, is_cuda=True):
        self.n, self.dtype, self.is_cuda = n, dtype, is_cuda

    shape = property(lambda self: (self.n // 128,))

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 24


def test_the_binding_checks_the_arrays_of_rotated_calls():
    """A type or a length that is not the call's own would have kernels read and write behind an array: refused in the binding, which knows them.
    (Nothing is computed: the pool holds metadata only.)"""
    pool = _host_pool(64)                                      # 4 query heads, 2 KV heads of 64: 256 and 128 elements a token
    pool.sk_pool_set_rotation(np.ones(32))
    sids = [pool.sk_session_create() for _ in range(3)]
    for sid in sids:
        pool.reserve(sid, 20)
    T = 9
    good = dict(positions=_OnCard(T, torch.int32), q=_OnCard(T * 256), k=_OnCard(T * 128), v=_OnCard(T * 128), q_out=_OnCard(T * 256), out=_OnCard(T * 256, torch.float32),
                lse=_OnCard(T * 4, torch.float32))
    wrong = [dict(k=_OnCard(T * 128, torch.float32)), dict(v=_OnCard(T * 128, torch.float16)), dict(k=_OnCard(T * 128, is_cuda=False)), dict(v=_OnCard(T * 128, is_cuda=False)),
             dict(out=_OnCard(T * 256)), dict(out=_OnCard(T * 256 - 4, torch.float32)), dict(out=_OnCard(T * 256, torch.float32, False)), dict(lse=_OnCard(T * 4)),
             dict(lse=_OnCard(T * 4 - 1, torch.float32)), dict(lse=_OnCard(T * 4, torch.float32, False)), dict(q=_OnCard(T * 256, torch.float32)), dict(q_out=_OnCard(T * 256 - 64)),
             dict(positions=_OnCard(T - 1, torch.int32)), dict(positions=_OnCard(T, torch.int64))]

    def step(ops, **kw):
        return pool.sk_batch_step_rotated(sids, ops, [0, 4, 6, T], **{**good, **kw}, stream=0)

    A, B, C = sk.SK_OP_APPEND, sk.SK_OP_QUERY_A, sk.SK_OP_QUERY_B
    step([A, B, C])
    step([B, B, B], out=_OnCard(50 * 256, torch.float32), lse=_OnCard(50 * 4, torch.float32))           # room for more
    for bad in wrong + [dict(k=_OnCard(T * 128 - 128)), dict(v=_OnCard(128))]:
        with pytest.raises(AssertionError):
            step([A, B, C], **bad)
    # what no item reads of k and v may be missing
    assert step([A, C, B], k=_OnCard(6 * 128), v=_OnCard(6 * 128))
    assert step([B, B, B], k=None, v=None)
    with pytest.raises(AssertionError):
        step([A, C, B], k=_OnCard(6 * 128), v=_OnCard(5 * 128))
    assert [pool.sk_session_length(s) for s in sids] == [28, 20, 20]

    pool.kv_mem = True                                         # (the binding checks arrays of pools that have memory)
    try:
        def append(**kw):
            a = {**good, **kw}
            return pool.sk_session_append_rotated(sids[1], a.pop("q"), a.pop("k"), a.pop("v"), pos0=0, **a, stream=0)

        append()
        for bad in wrong + [dict(v=_OnCard(T * 128 + 128)), dict(v=_OnCard(T * 128 - 128))]:
            with pytest.raises(AssertionError):
                append(**bad)
        assert pool.sk_session_length(sids[1]) == 29
    finally:
        pool.kv_mem = None


def test_a_list_of_shared_blocks_in_pinned_memory():
    pool = _host_pool(1000)
    pool.sk_pool_set_rotation(np.ones(32))
    a = pool.sk_session_create()
    pool.reserve(a, 4096), pool.reserve(a, 16 * 400 - 4096)
    b = pool.sk_session_fork(a, 16 * 400)
    before = pool.sk_session_block_table(b)
    for site in (sk.SK_SITE_RING, sk.SK_SITE_SCATTER):
        pool.sk_pool_inject_failure(site)
        assert _status(pool.sk_session_shift, b, 7) == sk.SK_E_HIP
        assert pool.sk_session_block_table(b) == before and pool.sk_pool_blocks_free() == 600
    pool.sk_session_shift(b, 7)
    assert not set(pool.sk_session_block_table(b)) & set(before) and pool.sk_pool_blocks_free() == 200


@pytest.mark.parametrize("launch,kept", [(1, 0), (2, 1), (3, 1)])
def test_a_long_append_that_fails_between_its_launches(launch, kept):
    """Its blocks travel in the arguments of several launches.  The copy of a shared last block stays once a launch has pointed the device's
    table at it; everything else is taken back."""
    pool = sk.Pool("bf16", 4, 2, 64, 16, 2000, max_sessions=2, max_batch_tokens=20000, metadata_only=True)
    pool.sk_pool_set_rotation(np.ones(32))
    a = pool.sk_session_create()
    pool.reserve(a, 40)
    b = pool.sk_session_fork(a, 48 - 8)
    pool.sk_session_truncate(a, 20)                            # ends inside a block that the fork holds too
    tables, free = pool.sk_session_block_table(a), pool.sk_pool_blocks_free()
    pool.sk_pool_inject_failure(sk.SK_SITE_SCATTER, launch)
    L = sk.lib()
    assert L.sk_session_append_rotated(pool.h, a, None, None, None, 18000, None, 0, None, None, sk.SK_F32, None, None) == sk.SK_E_HIP
    assert pool.sk_session_length(a) == 20 and pool.sk_pool_blocks_free() == free - kept
    now = pool.sk_session_block_table(a)
    assert now[:1] == tables[:1] and (now[1] != tables[1]) == bool(kept)
    assert L.sk_session_append_rotated(pool.h, a, None, None, None, 18000, None, 0, None, None, sk.SK_F32, None, None) == sk.SK_OK
    assert pool.sk_session_length(a) == 18020 and pool.sk_session_length(b) == 40


def test_shared_blocks_are_replaced_and_others_are_not():
    pool = _host_pool(24)
    pool.sk_pool_set_rotation(np.ones(32))
    a = pool.sk_session_create()
    pool.reserve(a, 150)                                       # ten blocks
    b = pool.sk_session_fork(a, 150)                           # nine shared, one of its own
    ta, tb = pool.sk_session_block_table(a), pool.sk_session_block_table(b)
    pool.sk_session_shift(b, 0)                                # nothing to do
    assert pool.sk_session_block_table(b) == tb
    pool.sk_session_shift(b, 7, first=35, count=40)            # tokens 35..74: blocks 2, 3, 4
    now = pool.sk_session_block_table(b)
    assert pool.sk_session_block_table(a) == ta
    assert now[:2] == tb[:2] and now[5:] == tb[5:] and not set(now[2:5]) & set(ta + tb)
    assert pool.sk_pool_blocks_free() == 24 - 10 - 1 - 3
    pool.sk_session_shift(b, 7, first=35, count=40)            # its own by now
    assert pool.sk_session_block_table(b) == now
    pool.sk_session_shift(a, 7, first=40, count=1)             # the other holder's block 2 has one holder
    assert pool.sk_session_block_table(a) == ta
    pool.sk_pool_inject_failure(sk.SK_SITE_SCATTER)
    assert _status(pool.sk_session_shift, b, 7) == sk.SK_E_HIP
    assert pool.sk_session_block_table(b) == now
    # more shared blocks than are free: refused, nothing changed
    c = pool.sk_session_create()
    pool.reserve(c, 16 * (pool.sk_pool_blocks_free() - 5))
    assert _status(pool.sk_session_shift, b, 7) == sk.SK_E_NOMEM
    assert pool.sk_session_block_table(b) == now and pool.sk_pool_blocks_free() == 5
    for s in (a, b, c):
        pool.sk_session_destroy(s)
    assert pool.sk_pool_blocks_free() == 24


def _inverse_turn(bits=400):
    """1 / (2 pi) in units of 2^-bits, pi by Machin's formula in whole numbers."""
    one = 1 << (bits + 64)

    def arctan_of_inverse(n):
        term, total, k = one // n, 0, 1
        while term:
            total += term // k if k % 4 == 1 else -(term // k)
            term //= n * n
            k += 2
        return total

    return (one << bits) // (8 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239)))


def _turns(frequency, position, bits=400):
    """The part of a turn, in units of 2^-bits, that a pair of a frequency has turned at a position."""
    num, den = float(frequency).as_integer_ratio()
    return int(position) * num * _INVERSE_TURN // den % (1 << bits)


_INVERSE_TURN = _inverse_turn()
FAST = np.array([(-1) ** i * 10.0 ** (6 * i / 63) for i in range(62)] + [2 * np.pi, 1e6])      # every frequency that a pool takes, above 1


def _steps(pool):
    """What the library keeps of a pool's frequencies (sk_rotation_of in csrc/sk_internal.h): the pairs' parts of a turn a position, in 2^-64."""
    of = getattr(sk.lib(), "_Z14sk_rotation_ofP7sk_pool")
    of.restype, of.argtypes = ctypes.c_void_p, [ctypes.c_void_p]
    at = of(pool.h)
    rotary = ctypes.c_int32.from_address(at).value
    return list((ctypes.c_uint64 * (rotary // 2)).from_address(at + 16))


def test_steps_against_whole_numbers():
    """A step is the nearest 64-bit fraction of a turn, whatever the frequency: half a unit, and no more than 2^-20 of one from what forms it."""
    pool = sk.Pool("bf16", 4, 2, 128, 16, 32, metadata_only=True)
    lists = [FAST, -FAST, _freqs(128), np.concatenate([10.0 ** -np.arange(0, 32), -10.0 ** -np.arange(0, 32)]),
             np.array([0.0, -0.0, 5e-324, 1.0, 2.0 ** -52, np.pi, -np.pi, 2 * np.pi, np.nextafter(2 * np.pi, 0), np.nextafter(2 * np.pi, 7), 999999.9999, -1e6, 2.0 ** 19, 710.0, 355.0, 1e-19])]
    for f in lists:
        pool.sk_pool_set_rotation(f)
        steps = _steps(pool)
        assert len(steps) == f.size
        for x, step in zip(f, steps):
            off = (step << 336) - _turns(x, 1)
            off = (off + (1 << 399)) % (1 << 400) - (1 << 399)
            assert abs(off) <= (1 << 335) + (1 << 316), (x, off / 2.0 ** 336)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("sign", [1, -1])
def test_fast_pairs_at_far_positions(interleaved, sign):
    """Frequencies up to the largest that a pool takes, positions up to the largest there are: angles of up to 3.4e8 turns."""
    pool = sk.Pool("f32", 1, 1, 128, 16, 4)
    pool.sk_pool_set_rotation(sign * FAST, interleaved=interleaved)
    positions = [1, -1, 7, 1000, 4097, 131071, -131072, 10 ** 7, 10 ** 9, 2 ** 31 - 1, -2 ** 31 + 1, -2 ** 31]
    q = synth.draw(synth.generator(39), (len(positions), 1, 128), "f32")
    got, _ = pool.sk_rotate(q.cuda(), positions=torch.tensor(positions, dtype=torch.int32, device="cuda"))
    got = got.cpu().double().numpy()[:, 0]
    x = q.double().numpy()[:, 0]
    a, b = (x[:, ::2], x[:, 1::2]) if interleaved else (x[:, :64], x[:, 64:])
    angle = 2 * np.pi * np.array([[_turns(sign * f, p) / 2 ** 400 for f in FAST] for p in positions])
    size = np.abs(a) + np.abs(b)
    for y, want in ((got[:, ::2] if interleaved else got[:, :64], a * np.cos(angle) - b * np.sin(angle)),
                    (got[:, 1::2] if interleaved else got[:, 64:], a * np.sin(angle) + b * np.cos(angle))):
        tol = 2.0 ** -21 * size
        assert np.all(np.abs(y - want) <= tol + HALF_STEP["f32"] * (np.abs(want) + tol)), (np.abs(y - want) / size).max()


# ---- rows beside the cache ---------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("layer", LAYERS)
@pytest.mark.parametrize("rotary,interleaved", TURNS)
def test_rows_against_the_definition(layer, rotary, interleaved):
    if rotary > layer[3]:
        rotary = layer[3]
    gen = synth.generator(11, stream=rotary + layer[1])
    for T, factor, base in ((1, 1.0, 10000.0), (33, 1.25, 500000.0), (200, 1.0, 10000.0)):
        pool = _pool(layer, rotary, interleaved, factor=factor, base=base)
        q, k, _ = _rows(gen, T, layer)
        got_q, got_k = pool.sk_rotate(q.cuda(), k.cuda(), pos0=1000003)
        torch.cuda.synchronize()
        position = 1000003 + np.arange(T)[:, None]
        _check(got_q, q, position, rotary, interleaved, layer[0], factor, base)
        _check(got_k, k, position, rotary, interleaved, layer[0], factor, base)
        # what lies behind the rotary dimensions is passed on bit for bit
        assert torch.equal(got_q.cpu()[..., rotary:], q[..., rotary:]) and torch.equal(got_k.cpu()[..., rotary:], k[..., rotary:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_positions_in_any_order_and_far_away(dtype):
    layer = (dtype, 4, 2, 128)
    pool = _pool(layer, 128, False)
    gen = synth.generator(12)
    positions = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 7, 7, 2 ** 24 + 1, 2 ** 30, -2 ** 30, 123456789, 3, 2, 1, 0, 65536], dtype=torch.int32)
    q, k, _ = _rows(gen, 16, layer)
    got_q, got_k = pool.sk_rotate(q.cuda(), k.cuda(), positions=positions.cuda())
    # (the reference's own angle, p f in doubles, is off by 2^-53 p f: 2^-22 at these ends, which its tolerance does not hold; phases modulo 1 of long doubles do)
    f = _freqs(128).astype(np.longdouble)
    turns = positions.numpy().astype(np.longdouble)[:, None] * (f / np.longdouble("6.283185307179586476925286766559005768"))
    angle = (2 * np.pi * (turns - np.floor(turns)).astype(np.float64))[:, None, :]
    for got, x in ((got_q, q), (got_k, k)):
        a, b = x.double().numpy()[..., :64], x.double().numpy()[..., 64:]
        want = np.concatenate([a * np.cos(angle) - b * np.sin(angle), a * np.sin(angle) + b * np.cos(angle)], -1)
        size = np.tile(np.abs(a) + np.abs(b), 2)
        tol = 2.0 ** -21 * size
        assert np.all(np.abs(got.cpu().double().numpy() - want) <= tol + HALF_STEP[dtype] * (np.abs(want) + tol))
    # position 0 is the row itself
    assert torch.equal(got_q[0].cpu(), q[0]) and torch.equal(got_k[14].cpu(), k[14])


@pytest.mark.gpu
def test_each_alone_in_place_and_many_rows():
    layer = ("bf16", 32, 8, 128)
    pool = _pool(layer, 128, False, n_blocks=8)
    gen = synth.generator(13)
    q, k, _ = _rows(gen, 2100, layer)                          # several heads to a thread
    qd, kd = q.cuda(), k.cuda()
    both = pool.sk_rotate(qd, kd, pos0=5)
    torch.cuda.synchronize()
    _check(both[0], q, 5 + np.arange(2100)[:, None], 128, False, "bf16")
    _check(both[1], k, 5 + np.arange(2100)[:, None], 128, False, "bf16")
    assert torch.equal(pool.sk_rotate(qd, None, pos0=5)[0], both[0])
    assert torch.equal(pool.sk_rotate(None, kd, pos0=5)[1], both[1])
    assert torch.equal(pool.sk_rotate(qd[:50], kd[:50], pos0=5)[0], both[0][:50])        # one head to a thread: the same bits
    pool.sk_rotate(qd, kd, pos0=5, q_out=qd, k_out=kd)
    assert torch.equal(qd, both[0]) and torch.equal(kd, both[1])
    with pytest.raises(sk.SkError):                            # outputs that overlap inputs otherwise
        pool.sk_rotate(qd[:100], None, q_out=qd[1:101])
    with pytest.raises(sk.SkError):
        pool.sk_rotate(None, kd[:100], k_out=kd[1:101])
    flat = torch.zeros(100 * 32 * 128 + 100 * 8 * 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sk.SkError):
        pool.sk_rotate(qd[:100], kd[:100], q_out=flat[:100 * 4096], k_out=flat[100 * 4096 - 1024:100 * 5120 - 1024])


@pytest.mark.gpu
def test_a_captured_rotation_follows_its_positions():
    layer = ("bf16", 8, 2, 128)
    pool = _pool(layer, 128, False)
    gen = synth.generator(14)
    sid = pool.sk_session_create()
    _, k0, v0 = _rows(gen, 300, layer)
    pool.sk_session_append(sid, None, k0.cuda(), v0.cuda())
    q, k, v = (x.cuda() for x in _rows(gen, 4, layer))
    positions = torch.arange(300, 304, dtype=torch.int32, device="cuda")
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    out, lse = torch.empty(q.shape, device="cuda"), torch.empty(q.shape[:2], device="cuda")

    def step():
        pool.sk_rotate(q, k, positions=positions, q_out=q_out, k_out=k_out)
        pool.sk_session_query(sid, q_out, k_out, v, out=out, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for p in (300, 17, 100000):
        positions.copy_(torch.arange(p, p + 4, dtype=torch.int32))
        q.copy_(_rows(gen, 4, layer)[0])
        graph.replay()
        got = [t.clone() for t in (q_out, k_out, out, lse)]
        step()
        for a, b in zip(got, (q_out, k_out, out, lse)):
            assert torch.equal(a, b)
        _check(got[0], q.cpu(), p + np.arange(4)[:, None], 128, False, "bf16")


# ---- on the way into the cache -----------------------------------------------------------------------

def _same(pool_a, a, pool_b, b):
    for x, y in zip(pool_a.sk_session_gather(a), pool_b.sk_session_gather(b)):
        assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("layer", LAYERS)
@pytest.mark.parametrize("block,rotary,interleaved", [(16, 64, False), (64, 48, True)])
def test_append_is_a_rotation_and_an_append(layer, block, rotary, interleaved):
    """q_out, the cache, and attention bit for bit those of sk_rotate and sk_session_append: short appends, long ones, lists in the arguments and in
    pinned memory, at lengths that end inside blocks, behind evicted tokens."""
    pools = [_pool(layer, rotary, interleaved, block=block, n_blocks=8192 // block, max_sessions=2) for _ in range(2)]
    gen = synth.generator(15, stream=block + layer[1])
    sids = [p.sk_session_create() for p in pools]
    at = 0
    for T in (1, 3, 16, 13, 33, 130, 1, 257, 1400, 2):
        q, k, v = (x.cuda() for x in _rows(gen, T, layer))
        positions = None
        if T % 2:
            positions = torch.randint(0, 100000, (T,), generator=gen, dtype=torch.int32).cuda()
        kw = dict(positions=positions, pos0=0 if positions is not None else at)
        got_q, out, lse = pools[0].sk_session_append_rotated(sids[0], q, k, v, **kw)
        want_q, want_k = pools[1].sk_rotate(q, k, **kw)
        want = pools[1].sk_session_append(sids[1], want_q, want_k, v)
        assert torch.equal(got_q, want_q) and torch.equal(lse, want[1]) and torch.equal(out, want[0]), T
        _same(pools[0], sids[0], pools[1], sids[1])
        at += T
        if T == 130:
            for p, s in zip(pools, sids):
                p.sk_session_freeze(s, 7)
                p.sk_session_evict_oldest(s, 60)
    # a position left out is the session's length
    q, k, v = (x.cuda() for x in _rows(gen, 5, layer))
    n = pools[0].sk_session_length(sids[0])
    got_q = pools[0].sk_session_append_rotated(sids[0], q, k, v)[0]
    assert torch.equal(got_q, pools[1].sk_rotate(q, pos0=n)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("switch", ["SK_FORCE_SIMPLE", "SK_NO_SMALL", "SK_FUSE", "SK_NO_256"])
@pytest.mark.parametrize("layer", [("bf16", 8, 2, 128), ("bf16", 16, 1, 64)])
def test_append_whatever_kernel_attends(monkeypatch, switch, layer):
    monkeypatch.setenv(switch, "1")
    pools = [_pool(layer, 64, False, n_blocks=200) for _ in range(2)]
    gen = synth.generator(26)
    sids = [p.sk_session_create() for p in pools]
    for T in (1, 20, 150, 400, 7):
        q, k, v = (x.cuda() for x in _rows(gen, T, layer))
        got_q, out, lse = pools[0].sk_session_append_rotated(sids[0], q, k, v, pos0=5 * T)
        want_q, want_k = pools[1].sk_rotate(q, k, pos0=5 * T)
        want = pools[1].sk_session_append(sids[1], want_q, want_k, v)
        assert torch.equal(got_q, want_q) and torch.equal(out, want[0]) and torch.equal(lse, want[1])
        _same(pools[0], sids[0], pools[1], sids[1])


@pytest.mark.gpu
@pytest.mark.parametrize("distrust", ["0", "1"])
@pytest.mark.parametrize("layer", [("bf16", 8, 8, 128), ("bf16", 8, 2, 64), ("bf16", 32, 8, 128), ("bf16", 7, 1, 128), ("bf16", 32, 1, 64)])
@pytest.mark.parametrize("rotary,interleaved", [(128, False), (64, False), (32, False), (128, True), (48, True), (16, True)])
def test_short_appends_whose_attention_turns_them(monkeypatch, distrust, layer, rotary, interleaved):
    """Up to 16 tokens and 32 rows a KV head: one launch, as far as its lanes hold both elements of a pair.  Sessions of no tokens, of a few, of several parts,
    with evicted ones; also with the last workgroup computing every part again."""
    monkeypatch.setenv("SK_SMALL_DISTRUST", distrust)
    rotary = min(rotary, layer[3])
    pools = [_pool(layer, rotary, interleaved, n_blocks=400, max_sessions=1, factor=1.125) for _ in range(2)]
    gen = synth.generator(28, stream=rotary + layer[1])
    sids = [p.sk_session_create() for p in pools]
    G = layer[1] // layer[2]
    for n in (0, 5, 33, 700, 4000):
        for T in sorted({1, 2, min(16, 32 // G), min(17, max(1, 32 // G)), min(32, max(1, 32 // G))}):
            q, k, v = (x.cuda() for x in _rows(gen, T, layer))
            positions = torch.randint(-5, 1 << 20, (T,), generator=gen, dtype=torch.int32).cuda() if T % 2 else None
            before = pools[0].sk_pool_get_stats()["launches"]
            got_q, out, lse = pools[0].sk_session_append_rotated(sids[0], q, k, v, positions=positions, pos0=n)
            launches = pools[0].sk_pool_get_stats()["launches"] - before - (not pools[0].sk_pool_last_launch()["fused_merge"] and pools[0].sk_pool_last_launch()["n_splits"] > 1)
            inside = T <= 16 and T * G <= 32 and (interleaved or rotary in (layer[3], layer[3] // 2))
            assert launches == (1 if inside else 2)
            want_q, want_k = pools[1].sk_rotate(q, k, positions=positions, pos0=n)
            want, want_lse = pools[1].sk_session_append(sids[1], want_q, want_k, v)
            assert torch.equal(got_q, want_q) and torch.equal(out, want) and torch.equal(lse, want_lse), (n, T)
            _same(pools[0], sids[0], pools[1], sids[1])
        if n == 33:
            for p, s in zip(pools, sids):
                p.sk_session_freeze(s, 3)
                p.sk_session_evict_oldest(s, 9)
        grow = max(0, n * 2 - pools[0].sk_session_length(sids[0]))
        if grow:
            _, k, v = (x.cuda() for x in _rows(gen, min(grow, 4000), layer))
            for p, s in zip(pools, sids):
                p.sk_session_append(s, None, k, v)


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [("bf16", 8, 2, 128), ("f32", 4, 4, 64)])
def test_an_append_behind_a_shared_last_block(layer):
    """The session's end lies in a block that a fork holds too: the append takes a copy of its own, and the fork reads what it read."""
    pool, plain = _pool(layer, 64, False, max_sessions=2), _pool(layer, 64, False, max_sessions=2)
    gen = synth.generator(27)
    a, k, v = _cached(pool, gen, 100, layer)
    fork = pool.sk_session_fork(a, 96)
    pool.sk_session_truncate(a, 87)
    ref = plain.sk_session_create()
    plain.sk_session_append(ref, None, k[:87].cuda(), v[:87].cuda())
    for T in (1, 50):
        q, k1, v1 = (x.cuda() for x in _rows(gen, T, layer))
        got = pool.sk_session_append_rotated(a, q, k1, v1, pos0=3)
        want_q, want_k = plain.sk_rotate(q, k1, pos0=3)
        want = plain.sk_session_append(ref, want_q, want_k, v1)
        assert torch.equal(got[0], want_q) and torch.equal(got[1], want[0]) and torch.equal(got[2], want[1])
        _same(pool, a, plain, ref)
        got_k, got_v = (x.cpu() for x in pool.sk_session_gather(fork))
        assert torch.equal(got_k, k[:96]) and torch.equal(got_v, v[:96])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_append_whose_blocks_take_several_launches(dtype):
    layer, T = (dtype, 2, 1, 64), 9000
    pools = [_pool(layer, 64, False, n_blocks=700, max_batch_tokens=T) for _ in range(2)]
    gen = synth.generator(23)
    q, k, v = (x.cuda() for x in _rows(gen, T, layer))
    sids = [p.sk_session_create() for p in pools]
    for p, s in zip(pools, sids):
        p.sk_session_append(s, None, k[:5].contiguous(), v[:5].contiguous())
    for positions, pos0 in ((None, 77), (torch.randint(0, 1 << 20, (T,), generator=gen, dtype=torch.int32).cuda(), 0)):
        got_q, _, _ = pools[0].sk_session_append_rotated(sids[0], q, k, v, positions=positions, pos0=pos0, attend=False)
        want_q, want_k = pools[1].sk_rotate(q, k, positions=positions, pos0=pos0)
        pools[1].sk_session_append(sids[1], None, want_k, v)
        assert torch.equal(got_q, want_q)
        _same(pools[0], sids[0], pools[1], sids[1])
        for p, s in zip(pools, sids):
            p.sk_session_truncate(s, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("by", ["all", "head"])
def test_shift_of_more_shared_blocks_than_travel_in_the_arguments(by):
    layer = ("bf16", 2, 2, 64)
    pool = _pool(layer, 64, False, n_blocks=1100, max_sessions=2)
    gen = synth.generator(24)
    source, k, v = _cached(pool, gen, 8000, layer)
    for first in (0, 3000):                                    # 500 shared blocks; 313
        fork = pool.sk_session_fork(source, 8000)
        delta = _deltas(gen, by, 2, 8000 - first)
        pool.sk_session_shift(fork, delta if by == "all" else delta.cuda(), first=first)
        got_k, got_v = (x.cpu() for x in pool.sk_session_gather(fork))
        assert torch.equal(got_v, v) and torch.equal(got_k[:first], k[:first])
        _check(got_k[first:], k[first:], np.full((8000 - first, 2), delta) if by == "all" else delta.numpy().T, 64, False, "bf16")
        src_k, src_v = (x.cpu() for x in pool.sk_session_gather(source))
        assert torch.equal(src_k, k) and torch.equal(src_v, v)
        pool.sk_session_destroy(fork)


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [("bf16", 8, 2, 128), ("f32", 4, 4, 64)])
@pytest.mark.parametrize("T", [1, 5, 40, 300])
def test_commit_alone_results_over_inputs_and_in_place(layer, T):
    pools = [_pool(layer, 64, False, max_sessions=4) for _ in range(2)]
    gen = synth.generator(16, stream=T)
    q, k, v = (x.cuda() for x in _rows(gen, T, layer))
    ref = pools[1].sk_session_create()
    want_q, want_k = pools[1].sk_rotate(q, k, pos0=9)
    want, want_lse = pools[1].sk_session_append(ref, want_q, want_k, v)
    p = pools[0]
    # neither q nor attention; q without attention
    for kw in (dict(q=None), dict(q=q, attend=False)):
        s = p.sk_session_create()
        got_q, out, lse = p.sk_session_append_rotated(s, kw.pop("q"), k, v, pos0=9, **kw)
        assert out is None and lse is None and (got_q is None or torch.equal(got_q, want_q))
        _same(p, s, pools[1], ref)
        p.sk_session_destroy(s)
    # q turned in place
    s, q2 = p.sk_session_create(), q.clone()
    got_q, out, lse = p.sk_session_append_rotated(s, q2, k, v, pos0=9, q_out=q2)
    assert got_q is q2 and torch.equal(q2, want_q) and torch.equal(out, want) and torch.equal(lse, want_lse)
    p.sk_session_destroy(s)
    # the output over q, k, v, which lie one behind the other (its type is the pool's)
    want2 = pools[1].sk_session_truncate(ref, 0) or pools[1].sk_session_append(ref, want_q, want_k, v, out_dtype=layer[0])[0]
    for over in "qkv":
        s = p.sk_session_create()
        flat = torch.cat([q.flatten(), k.flatten(), v.flatten(), q.flatten()])
        n, m = q.numel(), k.numel()
        at = {"q": 0, "k": n, "v": n + m}[over]
        got_q, out, _ = p.sk_session_append_rotated(s, flat[:n].view_as(q), flat[n:n + m].view_as(k), flat[n + m:n + 2 * m].view_as(v), pos0=9,
                                                    out=flat[at:at + n].view_as(q), out_dtype=layer[0])
        assert torch.equal(out, want2) and torch.equal(got_q, want_q), over
        _same(p, s, pools[1], ref)
        p.sk_session_destroy(s)
    # q_out over what the call reads or writes otherwise is refused, and nothing changes
    s = p.sk_session_create()
    big = torch.zeros(4 * q.numel(), dtype=q.dtype, device="cuda")
    for kw in (dict(q=big[:q.numel()].view_as(q), q_out=big[16:16 + q.numel()].view_as(q)), dict(k=big[:k.numel()].view_as(k), q_out=big[:q.numel()].view_as(q)),
               dict(v=big[:k.numel()].view_as(k), q_out=big[:q.numel()].view_as(q)),
               dict(out=big[:q.numel()].view_as(q), out_dtype=layer[0], q_out=big[:q.numel()].view_as(q))):
        args = {"q": q, "k": k, "v": v, **kw}
        with pytest.raises(sk.SkError) as e:
            p.sk_session_append_rotated(s, args.pop("q"), args.pop("k"), args.pop("v"), pos0=9, **args)
        assert e.value.status == sk.SK_E_INVAL and p.sk_session_length(s) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [("bf16", 8, 2, 128), ("bf16", 14, 2, 64), ("f32", 6, 2, 128)])
@pytest.mark.parametrize("sessions,most", [(2, 5), (9, 40), (40, 90)])
def test_a_ragged_step_is_a_rotation_and_a_step(layer, sessions, most):
    pools = [_pool(layer, 64, True, n_blocks=2048, max_sessions=sessions) for _ in range(2)]
    gen = synth.generator(17, stream=sessions)
    r = np.random.RandomState(sessions)
    ids = []
    for p in pools:
        ids.append([p.sk_session_create() for _ in range(sessions)])
    lengths = r.randint(1, 300, sessions)
    for n, a, b in zip(lengths, *ids):
        _, k, v = (x.cuda() for x in _rows(gen, int(n), layer))
        for p, s in zip(pools, (a, b)):
            p.sk_session_append(s, None, k, v)
    for kinds in ([sk.SK_OP_APPEND], [sk.SK_OP_QUERY_A], [sk.SK_OP_QUERY_B], [0, 1, 2]):
        ops = [kinds[i % len(kinds)] for i in range(sessions)]
        cu = np.concatenate([[0], np.cumsum(r.randint(0, most + 1, sessions))])
        cu[-1] += cu[-1] == 0
        T = int(cu[-1])
        q, k, v = (x.cuda() for x in _rows(gen, T, layer))
        positions = torch.randint(0, 1 << 20, (T,), generator=gen, dtype=torch.int32).cuda()
        in_place = q.clone()
        got_q, out, lse = pools[0].sk_batch_step_rotated(ids[0], ops, cu, positions, in_place, k, v, q_out=in_place if kinds[0] != 2 else None)
        want_q, want_k = pools[1].sk_rotate(q, k, positions=positions)
        want, want_lse = pools[1].sk_batch_step(ids[1], ops, cu, want_q, want_k, v)
        assert torch.equal(got_q, want_q) and torch.equal(out, want) and torch.equal(lse, want_lse)
        for a, b in zip(*ids):
            _same(pools[0], a, pools[1], b)
    lengths = [pools[0].sk_session_length(x) for x in ids[0]]
    with pytest.raises(sk.SkError) as e:                       # positions must be given
        pools[0].sk_batch_step_rotated(ids[0], ops, cu, None, q, k, v)
    assert e.value.status == sk.SK_E_INVAL and [pools[0].sk_session_length(x) for x in ids[0]] == lengths
    L = sk.lib()
    assert L.sk_batch_step_rotated(pools[0].h, 0, None, None, None, None, None, None, None, None, None, sk.SK_F32, None, None) == sk.SK_OK


@pytest.mark.gpu
def test_another_stream_than_the_current_one():
    layer = ("bf16", 8, 2, 128)
    pools = [_pool(layer, 128, False) for _ in range(2)]
    gen = synth.generator(18)
    q, k, v = (x.cuda() for x in _rows(gen, 200, layer))
    sids = [p.sk_session_create() for p in pools]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pools[0].sk_session_append_rotated(sids[0], q, k, v, stream=side)
    pools[0].sk_session_shift(sids[0], 11, first=50, stream=side)
    more = pools[0].sk_rotate(q, pos0=3, stream=side)[0]
    side.synchronize()
    want = pools[1].sk_session_append_rotated(sids[1], q, k, v)
    pools[1].sk_session_shift(sids[1], 11, first=50)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.equal(more, pools[1].sk_rotate(q, pos0=3)[0])
    torch.cuda.synchronize()
    _same(pools[0], sids[0], pools[1], sids[1])


# ---- keys turned on where they lie ----------------------------------------------------------------------

def _cached(pool, gen, n, layer):
    sid = pool.sk_session_create()
    _, k, v = _rows(gen, n, layer)
    for t in range(0, n, 4096):
        pool.sk_session_append(sid, None, k[t:t + 4096].cuda(), v[t:t + 4096].cuda())
    return sid, k, v


def _deltas(gen, by, hkv, count):
    if by == "all":
        return -37
    shape = (count,) if by == "token" else (hkv, count)
    return torch.randint(-5000, 5000, shape, generator=gen, dtype=torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [("bf16", 8, 2, 128), ("bf16", 6, 3, 64), ("f32", 4, 2, 64), ("f32", 3, 1, 128)])
@pytest.mark.parametrize("block", [16, 64, 256])
@pytest.mark.parametrize("by", ["all", "token", "head"])
@pytest.mark.parametrize("shared", [False, True])
def test_shift_against_the_definition(layer, block, by, shared):
    """Stretches that begin and end inside groups and blocks, with a frozen head and evicted tokens between; a fork's, whose source keeps its keys."""
    dtype, _, hkv, d = layer
    rotary, interleaved = (d, False) if block != 64 else (48, True)
    pool = _pool(layer, rotary, interleaved, block=block, n_blocks=4096 // block, max_sessions=3, factor=1.5)
    gen = synth.generator(19, stream=block)
    n = 700
    source, k, v = _cached(pool, gen, n, layer)
    pool.sk_session_freeze(source, 21)
    pool.sk_session_evict_oldest(source, 150)
    k, v = torch.cat([k[:21], k[171:]]), torch.cat([v[:21], v[171:]])
    n = 550
    sid = pool.sk_session_fork(source, n) if shared else source
    for first, count in ((21, n - 21), (5, 40), (0, n), (300, 1), (n - 1, 1), (64, 64), (333, 100), (10, 0)):
        delta = _deltas(gen, by, hkv, count)
        on_gpu = delta
        if by == "token":
            on_gpu = delta.cuda()
        elif by == "head":                                      # rows that lie apart
            wide = torch.full((hkv, count + 9), 1 << 30, dtype=torch.int32)
            wide[:, :count] = delta
            on_gpu = wide.cuda()[:, :count]
        pool.sk_session_shift(sid, on_gpu, first=first, count=count)
        got_k, got_v = pool.sk_session_gather(sid)
        torch.cuda.synchronize()
        assert torch.equal(got_v.cpu(), v)
        got_k = got_k.cpu()
        assert torch.equal(got_k[:first], k[:first]) and torch.equal(got_k[first + count:], k[first + count:])
        if count:
            move = np.full((count, hkv), delta) if by == "all" else np.broadcast_to(delta.numpy()[:, None] if by == "token" else delta.numpy().T, (count, hkv))
            _check(got_k[first:first + count], k[first:first + count], move, rotary, interleaved, dtype)
            assert torch.equal(got_k[..., rotary:], k[..., rotary:])
        k = got_k
    if shared:
        src_k, src_v = pool.sk_session_gather(source)
        pool2 = _pool(layer, rotary, interleaved, block=block, n_blocks=4096 // block)
        again, k2, v2 = _cached(pool2, synth.generator(19, stream=block), 700, layer)
        assert torch.equal(src_k.cpu(), torch.cat([k2[:21], k2[171:]])) and torch.equal(src_v.cpu(), torch.cat([v2[:21], v2[171:]]))
    # appends and attention go on behind it
    q, k1, v1 = _rows(gen, 20, layer)
    out, _ = pool.sk_session_append(sid, q.cuda(), k1.cuda(), v1.cuda())
    got_k, got_v = pool.sk_session_gather(sid)
    assert torch.equal(got_k.cpu(), torch.cat([k, k1])) and torch.equal(got_v.cpu(), torch.cat([v, v1])) and bool(torch.isfinite(out).all())


@pytest.mark.gpu
def test_a_delta_of_zero_leaves_every_bit():
    layer = ("bf16", 4, 2, 128)
    pool = _pool(layer, 128, False, max_sessions=2)
    gen = synth.generator(20)
    sid = pool.sk_session_create()
    k = torch.randint(-2 ** 15, 2 ** 15, (100, 2, 128), generator=gen, dtype=torch.int16).view(torch.bfloat16)      # any bits: NaN, infinities, zeros of both signs
    v = torch.randint(-2 ** 15, 2 ** 15, (100, 2, 128), generator=gen, dtype=torch.int16).view(torch.bfloat16)
    pool.sk_session_append(sid, None, k.cuda(), v.cuda())
    pool.sk_session_shift(sid, torch.zeros((2, 100), dtype=torch.int32, device="cuda"))
    fork = pool.sk_session_fork(sid, 100)
    pool.sk_session_shift(fork, torch.zeros(100, dtype=torch.int32, device="cuda"))
    for s in (sid, fork):
        got_k, got_v = pool.sk_session_gather(s)
        assert torch.equal(got_k.cpu().view(torch.int16), k.view(torch.int16)) and torch.equal(got_v.cpu().view(torch.int16), v.view(torch.int16))


@pytest.mark.gpu
def test_a_captured_shift_turns_the_keys_again():
    layer = ("f32", 2, 1, 64)
    pool = _pool(layer, 64, False)
    gen = synth.generator(21)
    sid, k, _ = _cached(pool, gen, 90, layer)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pool.sk_session_shift(sid, 3, first=10)
    for i in range(1, 5):
        graph.replay()
        torch.cuda.synchronize()
        got = pool.sk_session_gather(sid)[0].cpu()
        want, size = _expected(k[10:], 3 * i, 64, False)
        # each pass adds its own error, and a rounding
        assert np.all(np.abs(got[10:].double().numpy() - want) <= i * (2.0 ** -21 * 2 + 2.0 ** -24 * 2) * size)
        assert torch.equal(got[:10], k[:10])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_sliding_window_keeps_its_positions(dtype):
    """Append, evict, move the window's positions, over and over: the cache holds the raw keys turned by their places in the window, and a query
    at the window's end attends as a session does that was made of them.

    fp32, after m moves: each turns by an angle that is off by 2^-22 and rounds its products, (m + 1) 2^-21 (|x| + |y|) with growth below
    2; bf16: m + 1 roundings of 2^-8 of an element that is at most |x| + |y|."""
    layer = (dtype, 4, 2, 64)
    pool = _pool(layer, 64, False, block=16, n_blocks=40, max_sessions=2)
    gen = synth.generator(22)
    sid, sink, window = pool.sk_session_create(), 4, 200
    raw = torch.zeros((0, 2, 64))
    moves = 0
    for step in range(30):
        T = [1, 17, 40, 3][step % 4]
        q, k, v = _rows(gen, T, layer)
        pool.sk_session_append_rotated(sid, q.cuda(), k.cuda(), v.cuda())                 # at the session's length
        raw = torch.cat([raw, k.float()])
        if pool.sk_session_length(sid) > sink and moves == 0:
            pool.sk_session_freeze(sid, sink)
        over = pool.sk_session_length(sid) - window
        if over > 0:
            pool.sk_session_evict_oldest(sid, over)
            pool.sk_session_shift(sid, -over, first=sink)
            raw = torch.cat([raw[:sink], raw[sink + over:]])
            moves += 1
    assert moves > 8
    got = pool.sk_session_gather(sid)[0].cpu()
    want, size = _expected(raw, np.arange(len(raw))[:, None], 64, False)
    per = 2.0 ** -20 if dtype == "f32" else 2.0 ** -8 + 2.0 ** -20
    assert np.all(np.abs(got.double().numpy() - want) <= (moves + 1) * per * size)
