"""sk_verify: drafted tokens against the definition in 64 bits.  Whole results are compared exactly: a decision, or a drawn token, differs
from the definition's only where a number lies within some 2^-44 of a border, which no input here does (every case says how near its numbers come).
Log probabilities are formed in 64 bits and rounded once: 2^-24 of themselves, and 2^-40 for what is left of sums and logarithms."""
import numpy as np
import pytest
import torch

import paper_2605_13784_amd as sk
from workloads import synth


def _softmax(z, T):
    """p, log p of a row of logits at a temperature, or None if it has no probabilities."""
    z = z.astype(np.float64)
    if np.isnan(z).any() or np.isposinf(z).any() or np.isneginf(z).all():
        return None
    m = z.max()
    d = np.where(np.isneginf(z), -np.inf, (z - m) / T if np.isfinite(T) else 0.0)
    with np.errstate(under="ignore"):
        s = np.exp(d).sum()
        return np.exp(d) / s, d - np.log(s)


def _define(target, draft, tokens, u, temperature):
    """One sequence -> accepted, tokens, log probabilities, distance of the numbers that decide from their borders."""
    k, V = len(tokens), target.shape[1]
    T = 1.0 if temperature is None else float(temperature)
    greedy = not T > 0
    out, logp, near = [], [], 1.0
    for i in range(k + 1):
        row = _softmax(target[i], 1.0 if greedy else T)
        t = int(tokens[i]) if i < k else -1
        drafted = 0 <= t < V
        if row is None:
            return i, out + [-1], logp + [np.nan], near
        p, lp = row
        if greedy:
            best = int(np.argmax(target[i]))
            out.append(best), logp.append(lp[best])
            if drafted and t == best:
                continue
            return i, out, logp, near
        w = p
        if drafted:
            q = np.zeros(V)
            if draft is None:
                q[t] = 1.0
            else:
                d = _softmax(draft[i], T)
                q = None if d is None else d[0]
            if q is not None:
                ui = float(u[i])
                if ui == ui:
                    near = min(near, abs(ui * q[t] - p[t]) / max(p[t], 1e-300) if ui * q[t] != p[t] or p[t] > 0 else 1.0)
                if ui * q[t] < p[t]:
                    out.append(t), logp.append(lp[t])
                    continue
                w = np.maximum(p - q, 0.0)
        c = np.cumsum(w)
        if c[-1] <= 0:
            return i, out + [t], logp + [lp[t]], near
        v = float(u[k])
        x = max(v, 0.0) * c[-1] if v == v else 0.0
        at = int(np.searchsorted(c, x, side="right"))
        if at == V:
            at = int(np.nonzero(w)[0][-1])
        else:
            near = min(near, abs(c[at] - x) / c[-1], abs(x - (c[at - 1] if at else 0.0)) / c[-1] if x > 0 and at and c[at - 1] > 0 else 1.0)
        return i, out + [at], logp + [lp[at]], near
    raise AssertionError


def _check(target, tokens, u, draft=None, temperature=None, least=2.0 ** -40, target_gpu=None, draft_gpu=None, **kw):
    n, places, V = target.shape
    got = sk.sk_verify(target.cuda() if target_gpu is None else target_gpu, tokens.cuda(), u.cuda(),
                       draft=None if draft is None else (draft.cuda() if draft_gpu is None else draft_gpu),
                       temperature=None if temperature is None else temperature.cuda(), **kw)
    torch.cuda.synchronize()
    accepted, out, logp = (None if x is None else x.cpu().numpy() for x in got)
    for s in range(n):
        a, t, lp, near = _define(target[s].float().numpy(), None if draft is None else draft[s].float().numpy(), tokens[s].numpy(), u[s].numpy(),
                                 None if temperature is None else temperature[s])
        assert near > least, (s, near)                        # (of the inputs, not of the result)
        assert accepted[s] == a and list(out[s]) == t + [-1] * (places - len(t)), (s, a, t, accepted[s], out[s])
        if logp is not None:
            lp = np.array(lp + [0.0] * (places - len(lp)))
            with np.errstate(over="ignore"):
                ok = np.isfinite(lp.astype(np.float32))       # (below the least float, 3.4e38, is -inf: the token's logit over a tiny temperature)
            np.testing.assert_array_equal(logp[s][~ok], np.where(np.isnan(lp[~ok]), np.nan, -np.inf))
            assert np.all(np.abs(logp[s][ok] - lp[ok]) <= 2.0 ** -24 * np.abs(lp[ok]) + 2.0 ** -40 * (1 + np.abs(lp[ok])))
    return accepted


def _case(gen, n, k, V, dtype, near=1.0, spread=2.5):
    """Logits, a draft's near them, tokens drawn from the draft, numbers."""
    t = synth.torch_dtype(dtype)
    x = (spread * torch.randn((n, k + 1, V), generator=gen)).to(t)
    y = (x[:, :k].float() + near * torch.randn((n, k, V), generator=gen)).to(t)
    tokens = torch.zeros((n, k), dtype=torch.int32)
    for i in range(k):
        g = -torch.log(-torch.log(torch.rand((n, V), generator=gen).clamp(1e-9, 1 - 1e-7)))
        tokens[:, i] = (y[:, i].float() + g).argmax(1)
    return x, y, tokens, torch.rand((n, k + 1), generator=gen)


def test_refusals_without_a_gpu():
    L = sk.lib()
    p = 1 << 24                                               # addresses that no call below gets as far as using
    q, r = 2 * p, 3 * p
    good = dict(target=p, target_stride=100, draft=p, draft_stride=100, dtype=sk.SK_F32, n_seq=3, n_draft=2, vocab=100, tokens=p, uniform=p, temperature=p,
                ws=q, ws_bytes=1 << 20, n_accepted=r, out_tokens=r + 64, logprob=r + 128, stream=None)

    def call(**kw):
        return L.sk_verify(*{**good, **kw}.values())

    for bad in (dict(n_seq=-1), dict(n_draft=-1), dict(n_draft=sk.SK_VERIFY_MAX_DRAFT + 1), dict(vocab=0), dict(vocab=-5), dict(target_stride=99),
                dict(draft_stride=99), dict(vocab=sk.SK_VERIFY_MAX_VOCAB + 1, target_stride=1 << 22, draft_stride=1 << 22), dict(n_seq=sk.SK_VERIFY_MAX_ROWS),
                dict(target=None), dict(tokens=None), dict(uniform=None), dict(n_accepted=None), dict(out_tokens=None), dict(target=p + 2),
                dict(draft=p + 1), dict(dtype=sk.SK_BF16, target=p + 1), dict(tokens=p + 2), dict(uniform=p + 1), dict(temperature=p + 2), dict(ws=q + 8), dict(ws=None),
                dict(n_accepted=r + 2), dict(out_tokens=r + 65), dict(logprob=r + 130), dict(target_stride=1 << 41),
                # outputs over inputs, over each other, over the workspace, and that over an input
                dict(n_accepted=p + 3596), dict(out_tokens=p + 2000), dict(logprob=p), dict(out_tokens=r + 8), dict(logprob=r + 96), dict(n_accepted=q + 16),
                dict(ws=p + 16), dict(tokens=r + 80), dict(uniform=r + 160), dict(temperature=r)):
        assert call(**bad) == sk.SK_E_INVAL, bad
    assert call(dtype=2) == sk.SK_E_DTYPE
    need = L.sk_verify_workspace_bytes(3, 2, 100)
    assert need > 0 and call(ws_bytes=need - 1) == sk.SK_E_WORKSPACE
    assert call(n_seq=0, target=None) == sk.SK_OK
    for n, k, v in ((0, 2, 100), (3, -1, 100), (3, 33, 100), (3, 2, 0), (1 << 20, 1, 10)):
        assert L.sk_verify_workspace_bytes(n, k, v) == 0


SIZES = [(1, 0, 1), (2, 1, 1), (3, 1, 2), (5, 2, 5), (9, 3, 64), (4, 4, 255), (3, 2, 4095), (3, 2, 4096), (3, 2, 4097), (2, 3, 8191), (2, 1, 8192), (2, 3, 16385),
         (1, 8, 32000), (5, 5, 50257), (2, 4, 131072), (70, 1, 300), (3, 32, 130), (1, 0, 70001), (40, 0, 999), (300, 2, 77)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("n,k,V", SIZES)
def test_against_the_definition(dtype, drawn, n, k, V):
    gen = synth.generator(30, stream=n * 1000 + k * 100 + V)
    x, y, tokens, u = _case(gen, n, k, V, dtype, near=0.7)
    if not drawn and k:                                       # looked-up tokens that the target likes
        tokens[:, 0] = x[:, 0].float().argmax(1)
    _check(x, tokens, u, draft=y if drawn else None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_temperatures_and_drafts_that_end_early(dtype):
    gen = synth.generator(31)
    n, k, V = 24, 4, 700
    x, y, tokens, u = _case(gen, n, k, V, dtype, near=0.3)
    temperature = torch.tensor([0.0, 1.0, 0.5, 2.0, 1e-3, 50.0, float("inf"), float("nan"), -1.0, 0.7, 1e-38, 1e30] * 2)
    for s in range(n):
        if not temperature[s] > 0:
            tokens[s] = x[s, :k].float().argmax(1)            # greedy sequences that accept
    tokens[3, 0] = -1
    tokens[5, 2] = V
    tokens[9, 1] = -2 ** 31
    tokens[10, 3] = 2 ** 31 - 1
    tokens[12, 2] = -5                                        # a greedy one
    tokens[20, 1] = (tokens[20, 1] + 1) % V                   # a greedy one that rejects
    accepted = _check(x, tokens, u, draft=y, temperature=temperature)
    assert accepted.max() == k and accepted.min() == 0
    _check(x, tokens, u, temperature=temperature)


def _odd_rows(dtype, V):
    gen = synth.generator(32, stream=V)
    n, k = 16, 2
    x, y, tokens, u = _case(gen, n, k, V, dtype, near=0.5)
    lowest = torch.finfo(synth.torch_dtype(dtype)).min
    inf = float("inf")
    x[0, :, V // 2:] = -inf                                   # a draft that offers what the target forbids
    x[1, 0] = -inf                                            # nothing at all
    x[2, 1] = -inf
    x[3, 0, V - 1] = float("nan")
    x[4, 0, 0] = inf
    y[5, 0] = -inf                                            # a draft row without probabilities
    y[6, 0, 1] = float("nan")
    y[7, 1, 0] = inf
    x[8] = 1.25                                               # all equal
    y[8] = 1.25
    x[9, :, 1:] = lowest                                      # masked with the type's lowest number
    x[10] = lowest
    x[11, 0, :V - 1] = -inf                                   # one token is left, in the last place
    x[12, :, ::2] = -inf
    y[12, :, 1::2] = -inf                                     # nothing in common
    x[13] = x[13] * 30.0
    y[13] = x[13, :2]                                         # the same distribution: everything stays
    x[14, :, :-1] = -inf
    y[14, :, :-1] = -inf
    tokens[14] = V - 1
    x[15, :, 0] = 3.0e38 if dtype == "f32" else 3.0e38
    return x, y, tokens, u


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3, 40, 5000, 9001])
def test_masks_equal_logits_and_rows_without_probabilities(dtype, V):
    x, y, tokens, u = _odd_rows(dtype, V)
    n = 16
    temperature = torch.ones(n)
    _check(x, tokens, u, draft=y, temperature=temperature)
    _check(x, tokens, u, temperature=temperature)
    _check(x, tokens, u, draft=y, temperature=torch.zeros(n))
    tokens[:, 0] = torch.where(torch.isnan(x[:, 0].float()), torch.zeros(()), x[:, 0].float()).argmax(1)
    _check(x, tokens, u, draft=y, temperature=torch.full((n,), 0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3, 40, 9001])
def test_masks_equal_logits_and_rows_without_probabilities_among_many_rows(dtype, V):
    x, y, tokens, u = (t.repeat((20,) + (1,) * (t.dim() - 1)) for t in _odd_rows(dtype, V))
    u[16:] = torch.rand((304, 3), generator=synth.generator(42))
    temperature = torch.ones(320)
    temperature[160:240] = 0.0
    _check(x, tokens, u, draft=y, temperature=temperature)
    _check(x, tokens, u, temperature=temperature)


@pytest.mark.gpu
def test_numbers_at_the_ends_of_their_range():
    gen = synth.generator(33)
    n, k, V = 12, 2, 6000
    x, y, tokens, _ = _case(gen, n, k, V, "f32")
    x[:, :, :3] = -float("inf")                               # the first and last tokens have no weight
    x[:, :, -3:] = -float("inf")
    ends = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 7.0, -0.5, float("nan"), float("inf"), -float("inf"), 2.0 ** -149, 1.0 - 2.0 ** -24, 0.0, 1.0])
    u = ends[:, None].repeat(1, k + 1)
    _check(x, tokens, u, draft=y, least=-1.0)                 # (a number of 0 lies on its border: 0 q < p)
    u[:, :k] = 2.0                                            # (what stays has p > 2 q)
    u[:, k] = ends
    _check(x, tokens, u, draft=y, least=-1.0)
    # a looked-up token that is the only one left, and a number that rejects it: nothing remains but the token
    x = torch.full((1, 2, 50), -float("inf"))
    x[0, :, 17] = 0.5
    assert _check(x, torch.tensor([[17]], dtype=torch.int32), torch.tensor([[1.0, 0.5]]), least=-1.0)[0] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 1100])
def test_weights_below_the_least_double(dtype, n):
    """2,048 logits that lie 2^-1075.3 below the largest: none of them has a weight, though all together would have 2^-1064."""
    V, T = 6000, 1.4426950408889634 / 1075.3
    x = torch.full((n, 2, V), -float("inf"), dtype=synth.torch_dtype(dtype))
    x[:, :, :2048] = -1.0
    x[:, :, 5000] = 0.0
    temperature = torch.full((n,), T, dtype=torch.float32)
    # a number of 0 finds the first token that has a weight, behind the draft and behind nothing; a number of 1 rejects the only one that has: nothing remains but the token
    u = torch.tensor([[0.0, 0.0], [1.0, 0.0], [0.5, 2.0 ** -149]]).repeat((n + 2) // 3, 1)[:n]
    tokens = torch.full((n, 1), 5000, dtype=torch.int32)
    _check(x, tokens, u, temperature=temperature, least=-1.0)
    _check(x[:, 1:], tokens[:, :0], u[:, 1:], temperature=temperature, least=-1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift,pad", [(0, 1), (1, 0), (3, 5), (7, 2)])
def test_rows_that_start_anywhere(dtype, shift, pad):
    gen = synth.generator(34, stream=shift)
    n, k, V = 5, 3, 4099
    x, y, tokens, u = _case(gen, n, k, V, dtype, near=0.4)

    def placed(a, places):
        flat = torch.full((shift + n * places * (V + pad) + 8,), float("nan"), dtype=a.dtype, device="cuda")         # what lies beside a row must not count
        view = flat[shift:shift + n * places * (V + pad)].view(n, places, V + pad)[:, :, :V]
        view.copy_(a)
        return view

    _check(x, tokens, u, draft=y, target_gpu=placed(x, k + 1), draft_gpu=placed(y, k))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drawn", [True, False])
def test_many_rows_whose_later_places_wait_for_the_first(dtype, drawn):
    """600 sequences of up to 4 drafted tokens over 16,400 logits: sequences that end at every place, by a token that does not stay, by the draft's end and greedily,
    some of them in rows without probabilities behind the place where they end (which do not count)."""
    gen = synth.generator(40)
    n, k, V = 600, 4, 16400
    x, y, tokens, u = _case(gen, n, k, V, dtype, near=0.4)
    for s in range(n):
        if s % 7 < k:
            tokens[s, s % 7] = -1
        if s % 11 == 0:
            x[s, 3] = float("nan")
        if s % 13 == 0:
            y[s, 2] = -float("inf")
        if s % 17 == 0:
            x[s, 1] = -float("inf")
    if not drawn:
        tokens[:, 0] = torch.where(tokens[:, 0] >= 0, x[:, 0].float().argmax(1).to(torch.int32), tokens[:, 0])
    temperature = torch.where(torch.arange(n) % 5 == 0, 0.0, 1.0)
    for s in range(0, n, 10):
        tokens[s] = torch.nan_to_num(x[s, :k].float(), nan=0.0).argmax(1)
    accepted = _check(x, tokens, u, draft=y if drawn else None, temperature=temperature)
    assert set(accepted) == set(range(k + 1))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("n,k,V", [(1, 4, 151936), (2, 3, 131073), (2, 2, 262144), (3, 1, 202048), (1, 0, 1 << 21), (1, 1, 1 << 21)])
def test_rows_of_more_stretches_than_a_lane_keeps(dtype, drawn, n, k, V):
    """Behind 131,072 logits a row of the few-rows form has more than 256 stretches of 512 (four a lane) and 64 parts of 2,048 (four for each of sixteen lanes)."""
    gen = synth.generator(50, stream=n * 1000 + k * 100 + V % 97)
    x, y, tokens, u = _case(gen, n, k, V, dtype, near=0.7)
    if not drawn and k:
        tokens[:, 0] = x[:, 0].float().argmax(1)
    _check(x, tokens, u, draft=y if drawn else None)


def _behind(gen, n, k, V, at, dtype):
    """Rows whose probabilities lie in the last logits, from `at` on; what is in front has none (sequences 0, 3, ..), next to none (1, 4, ..) or half (2, 5, ..)."""
    x, y, tokens, u = _case(gen, n, k, V, dtype, near=0.7)
    tail = V - at
    for rows in (x, y):
        rows[0::3, :, :at] = -float("inf")
        rows[1::3, :, :at] -= 60.0
        rows[2::3, :, at:] += float(np.log(at / tail))         # as much as in front
    for i in range(k):
        g = -torch.log(-torch.log(torch.rand((n, V), generator=gen).clamp(1e-9, 1 - 1e-7)))
        tokens[:, i] = (y[:, i].float() + g).argmax(1)
    return x, y, tokens, u


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,V,at", [(6, 2, 133000, 131072), (3, 3, 151936, 151936 - 300), (3, 1, 262144, 262143), (9, 0, 132100, 131072),
                                      (9, 16, 524288 + 700, 524288), (40, 1, 524288 + 9000, 524288 + 8192), (200, 0, 524288 + 33, 524288)])
def test_rows_whose_weight_lies_in_their_last_stretches(dtype, n, k, V, at):
    """Behind stretch 256 and part 64, of either form (32 logits a lane have them from 524,288 on): draws, what is left of a drafted token, a looked-up token that is
    rejected there, the maximum of a greedy sequence and its lowest index among equals."""
    rows = n * (2 * k + 1)
    gen = synth.generator(51, stream=n * 100 + k)
    x, y, tokens, u = _behind(gen, n, k, V, at, dtype)
    places = min(n, 8 if rows > 30 else n)
    some = list(range(places))                                 # (the definition in 64 bits takes 0.1 s a row)

    def check(**kw):
        got = sk.sk_verify(x.cuda(), tokens.cuda(), u.cuda(), **{a: b.cuda() for a, b in kw.items()})
        for s in some:
            temperature = kw.get("temperature")
            a, t, lp, near = _define(x[s].float().numpy(), kw["draft"][s].float().numpy() if "draft" in kw else None, tokens[s].numpy(), u[s].numpy(),
                                     None if temperature is None else temperature[s])
            assert near > 2.0 ** -40
            assert int(got[0][s]) == a and got[1][s].tolist() == t + [-1] * (k + 1 - len(t)), s
            lp = np.array(lp)
            assert np.all(np.abs(got[2][s, :len(lp)].cpu().numpy() - lp) <= 2.0 ** -24 * np.abs(lp) + 2.0 ** -40 * (1 + np.abs(lp)))
        return got

    got = check(**({"draft": y} if k else {}))
    assert (got[1][:, 0] >= at).float().mean() >= 0.5
    if k:
        u[:, :k] = 0.9375                                      # looked-up tokens that do not stay: each has half its row's weight or less
        tokens[:, 0] = x[:, 0, at:].float().argmax(1).int() + at
        check()
    x[:, :, V - 1] = x.float().amax(2).to(x.dtype)             # greedy: two largest ones, the lower in front
    if k:
        tokens[:] = torch.from_numpy(np.argmax(x[:, :k].float().numpy(), 2)).int()
    got = check(temperature=torch.zeros(n))
    assert (got[0] == k).all()
    x[:, :, V - 1] += 1.0
    check(temperature=torch.zeros(n))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,k,V,drawn", [("f32", 512, 8, 5000, True), ("bf16", 512, 8, 5000, True), ("f32", 512, 16, 5000, False), ("bf16", 512, 16, 5000, False),
                                               ("f32", 32, 8, 128256, True)])
def test_later_places_wait_and_every_workgroup_decides(dtype, n, k, V, drawn):
    """8,192 parts and more, so that places come in two launches, with few enough sequences and stretches that every workgroup of the sums finds what is drawn from by itself: parts of
    rows that nobody computed hold what the workspace held before, NaN here.  Sequences end at every place."""
    gen = synth.generator(52, stream=n + k)
    x, y, tokens, u = _case(gen, n, k, V, dtype, near=0.3)
    for s in range(n):
        e = s % (k + 2)
        if not drawn:                                          # (looked up: what the target likes best, and numbers that let it stay)
            tokens[s] = x[s, :k].float().argmax(1)
            u[s, :k] *= 0.001
        if e < k:
            if s % 4 == 0:
                tokens[s, e] = -1
            elif s % 4 == 1:                                   # nothing in the target
                x[s, e, int(tokens[s, e])] = -float("inf")
            elif s % 4 == 2:
                x[s, e] = float("nan")
            else:
                u[s, e] = 2.0                                  # (stays only where p > 2 q)
            if s % 5 == 0:
                x[s, e + 1:] = float("nan")                    # behind the end: not looked at
    temperature = torch.where(torch.arange(n) % 7 == 3, 0.0, 1.0)
    need = sk.lib().sk_verify_workspace_bytes(n, k, V)
    accepted = _check(x, tokens, u, draft=y if drawn else None, temperature=temperature, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert len(set(accepted)) > min(k, 6)


@pytest.mark.gpu
def test_more_rows_than_one_grid_has_workgroups_for():
    """2^20 rows of 32,769 bf16 logits (68.7 GB, offsets far behind 32 bits): more than 2^24 workgroups, so that the last sequences are a second run of launches.
    Every stretch of sequences gives what a call of its own gives, and rows on both sides of the border what the definition does."""
    n, V, step = 1 << 20, 4 * 8192 + 1, 1 << 16
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GiB of device memory")
    gen = torch.Generator(device="cuda").manual_seed(41)
    some = (2.5 * torch.randn((4099, V), generator=gen, device="cuda")).bfloat16()
    target = torch.empty((n, 1, V), dtype=torch.bfloat16, device="cuda")
    for i in range(0, n, 4099):
        target[i:i + 4099, 0] = some[:min(4099, n - i)]
    u = torch.rand((n, 1), generator=gen, device="cuda")
    temperature = 0.5 + torch.rand(n, generator=gen, device="cuda")
    temperature[::5] = 0.0                                    # greedy
    tokens = torch.empty((n, 0), dtype=torch.int32, device="cuda")
    accepted, out, logp = sk.sk_verify(target, tokens, u, temperature=temperature)
    torch.cuda.synchronize()
    assert not accepted.any()
    for i in range(0, n, step):
        one = sk.sk_verify(target[i:i + step], tokens[i:i + step], u[i:i + step], temperature=temperature[i:i + step])
        assert torch.equal(one[1], out[i:i + step]) and torch.equal(one[2], logp[i:i + step]), i
    border = ((1 << 24) - 1) // 20                            # sequences of the first run
    for i in [0, 1, border - 2, border - 1, border, border + 1, n - 1]:
        _, t, lp, near = _define(target[i].float().cpu().numpy(), None, [], u[i].cpu().numpy(), float(temperature[i]))
        assert near > 2.0 ** -40 and int(out[i, 0]) == t[0] and abs(float(logp[i, 0]) - lp[0]) <= 2.0 ** -24 * abs(lp[0]) + 2.0 ** -40 * (1 + abs(lp[0])), i
    del target, some


@pytest.mark.gpu
def test_what_it_draws_has_the_targets_distribution():
    """Frequencies of the first token over 2^17 sequences, for a draft that is far from the target, a looked-up token and none: within 5 deviations."""
    gen = synth.generator(35)
    n, V = 1 << 17, 7
    p_logits, q_logits = 1.5 * torch.randn(V, generator=gen), 1.5 * torch.randn(V, generator=gen)
    p = torch.softmax(p_logits.double(), 0)
    for kind in ("draft", "looked up", "none"):
        k = 0 if kind == "none" else 1
        x = p_logits.expand(n, k + 1, V).contiguous().cuda()
        y = q_logits.expand(n, k, V).contiguous().cuda() if kind == "draft" else None
        tokens = torch.full((n, k), 2, dtype=torch.int32)
        if kind == "draft":
            tokens[:, 0] = torch.multinomial(torch.softmax(q_logits, 0), n, replacement=True, generator=gen)
        u = torch.rand((n, k + 1), generator=gen)
        _, out, logp = sk.sk_verify(x, tokens.cuda(), u.cuda(), draft=y)
        first = out[:, 0].cpu().long()
        count = torch.bincount(first, minlength=V).double()
        assert torch.all((count - n * p).abs() <= 5 * torch.sqrt(n * p * (1 - p))), kind
        assert torch.allclose(logp[:, 0].cpu().double(), torch.log(p)[first], atol=1e-6, rtol=0)


@pytest.mark.gpu
def test_outputs_left_out_none_at_all_and_other_streams():
    gen = synth.generator(36)
    x, y, tokens, u = _case(gen, 6, 3, 20000, "f32", near=0.5)
    want = [t.clone() for t in sk.sk_verify(x.cuda(), tokens.cuda(), u.cuda(), draft=y.cuda())]
    out = sk.verify_outputs(6, 3, "cuda:0")
    got = sk.sk_verify(x.cuda(), tokens.cuda(), u.cuda(), draft=y.cuda(), outputs=(out[0], out[1], None))
    assert got[2] is None and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    none = sk.sk_verify(x.cuda()[:0], tokens.cuda()[:0], u.cuda()[:0], draft=y.cuda()[:0])
    assert none[0].shape == (0,) and none[1].shape == (0, 4)
    xd, yd, td, ud = x.cuda(), y.cuda(), tokens.cuda(), u.cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    both = [sk.sk_verify(xd, td, ud, draft=yd, stream=s) for s in streams]
    torch.cuda.synchronize()
    for got in both:
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_captured_and_replayed():
    gen = synth.generator(37)
    n, k, V = 5, 4, 33000
    cases = [_case(gen, n, k, V, "bf16", near=0.5) for _ in range(4)]
    static = [t.cuda() for t in cases[0]]
    workspace = torch.empty(sk.lib().sk_verify_workspace_bytes(n, k, V), dtype=torch.uint8, device="cuda")
    outputs = sk.verify_outputs(n, k, "cuda:0")

    def call():
        sk.sk_verify(static[0], static[2], static[3], draft=static[1], workspace=workspace, outputs=outputs)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for case in cases:
        for a, b in zip(static, case):
            a.copy_(b)
        workspace.fill_(0xA5)
        graph.replay()
        got = [t.clone() for t in outputs]
        want = sk.sk_verify(static[0], static[2], static[3], draft=static[1])
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_drafting_step_over_sessions(dtype):
    """Drafted tokens go into their sessions' caches turned by their positions, the target's rows for them are verified, what does not stay is taken out
    again, and the next step goes on behind: cache and positions as if only what stayed had ever been appended; then the window slides."""
    hq, hkv, d, V, k, n = 4, 2, 64, 997, 3, 6
    gen = synth.generator(38)
    pools = [sk.Pool(dtype, hq, hkv, d, 16, 200, max_sessions=n) for _ in range(2)]
    for p in pools:
        p.sk_pool_set_rotation(10000.0 ** (-np.arange(0, d, 2) / d))
    t = synth.torch_dtype(dtype)
    embed = [torch.randn((V, h, d), generator=gen).to(t).cuda() for h in (hq, hkv, hkv)]      # q, k, v of a token
    head = (0.7 * torch.randn((hq * d, V), generator=gen)).cuda()
    ids = [[p.sk_session_create() for _ in range(n)] for p in pools]
    history = [list(torch.randint(0, V, (20 + 7 * s,), generator=gen).numpy()) for s in range(n)]
    for pool, sids in zip(pools, ids):
        for sid, h in zip(sids, history):
            x = torch.tensor(h[:-1], device="cuda")
            pool.sk_session_append_rotated(sid, *(e[x] for e in embed))
    cu = [i * (k + 1) for i in range(n + 1)]
    seen = []
    for step in range(6):
        # the last token of a sequence and k drafted ones behind it, the draft's choice a noisy one of the target's kind
        last = torch.tensor([h[-1] for h in history], dtype=torch.int32)
        draft_logits = 2.0 * torch.randn((n, k, V), generator=gen)
        if step % 2:
            draft_logits[:, 0, :] = -float("inf")
            draft_logits[:, 0, 5] = 0.0                                          # certain of a token
        g = -torch.log(-torch.log(torch.rand((n, k, V), generator=gen).clamp(1e-9, 1 - 1e-7)))
        drafted = (draft_logits + g).argmax(2).to(torch.int32)
        rows = torch.cat([last[:, None], drafted], 1).flatten().long().cuda()
        lengths = [pools[0].sk_session_length(s) for s in ids[0]]
        positions = torch.cat([torch.arange(m, m + k + 1, dtype=torch.int32) for m in lengths]).cuda()
        q_out, out, _ = pools[0].sk_batch_step_rotated(ids[0], [sk.SK_OP_APPEND] * n, cu, positions, *(e[rows] for e in embed))
        logits = (out.view(n * (k + 1), hq * d) @ head).view(n, k + 1, V)
        logits[:, 0] += 4.0 * torch.nn.functional.one_hot(drafted[:, 0].long(), V).cuda() * (step % 3)       # likes the first drafted token in some steps
        u = torch.rand((n, k + 1), generator=gen)
        accepted, tokens, _ = sk.sk_verify(logits, drafted.cuda(), u.cuda(), draft=draft_logits.cuda())
        accepted, tokens = accepted.cpu().numpy(), tokens.cpu().numpy()
        for s in range(n):
            a, want, _, near = _define(logits[s].cpu().numpy(), draft_logits[s].numpy(), drafted[s].numpy(), u[s].numpy(), None)
            assert near > 2.0 ** -40 and accepted[s] == a and list(tokens[s][:a + 1]) == want
            seen.append(a)
            pools[0].sk_session_truncate(ids[0][s], lengths[s] + 1 + a)
            new = [history[s][-1]] + list(tokens[s][:a])                          # what is in the cache now; the drawn token comes with the next step
            pools[1].sk_session_append_rotated(ids[1][s], *(e[torch.tensor(new, device="cuda")] for e in embed))
            history[s] += list(tokens[s][:a + 1])
            for x, y in zip(pools[0].sk_session_gather(ids[0][s]), pools[1].sk_session_gather(ids[1][s])):
                assert torch.equal(x, y)
    assert max(seen) > 0 and min(seen) < k
    for pool, sids in zip(pools, ids):
        for sid in sids:
            pool.sk_session_freeze(sid, 4)
            pool.sk_session_evict_oldest(sid, 9)
            pool.sk_session_shift(sid, -9, first=4)
    q = torch.randn((2, hq, d), generator=gen).to(t).cuda()
    for a, b in zip(*ids):
        m = pools[0].sk_session_length(a)
        x, y = (p.sk_session_query(s, p.sk_rotate(q, pos0=m)[0])[0] for p, s in zip(pools, (a, b)))
        assert torch.equal(x, y)
