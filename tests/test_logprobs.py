"""sk_logprobs: log probabilities of given tokens, normaliser, entropy and best alternatives of logit rows, against their
definitions in 64 bits.  Indices are compared exactly; the order of equal logits is by index.

Tolerance.  A lane adds at most n = 32 * ceil(vocab / 8192) + 32 weights one behind the other, the lanes' and parts' sums meet in
fewer than 32 more additions, each rounding by at most 2^-24 of the sum; a weight exp(d) is off by 2^-24 |d| (the rounded d) and
2^-22 (the product with log2 e, the hardware's exponential), and weights with |d| > 32 count for less than 2^-24 of a row of 2^21
logits together.  So S is within (n + 32 + 32 + 4) 2^-24 of itself, log S within as much absolutely, and with the roundings of
x - m, of their difference and of logf (2 ulp) a result within that + 2^-23 (|result| + |log S| + 1).  The entropy has Z / S beside it,
whose terms carry the same relative errors."""
import numpy as np
import pytest
import torch

import paper_2605_13784_amd as sk
from workloads import synth


def _tolerance(vocab, size):
    n = 32 * -(-vocab // 8192) + 32
    return (n + 68) * 2.0 ** -24 + 2.0 ** -23 * (np.abs(size) + np.log(vocab) + 1)


def _expected(x, tokens, n_top):
    z = x.double()
    m = z.max(1, keepdim=True)[0]
    none = torch.isneginf(m)
    m0 = torch.where(none, torch.zeros_like(m), m)
    s = torch.exp(z - m0).sum(1, keepdim=True)
    lse = torch.where(none, m, m + torch.log(s))
    p = torch.where(none, torch.full_like(z, -np.inf), (z - m0) - torch.log(s))           # (z - lse is 0 where m is 1e38: 64 bits do not hold m + log s)
    q = torch.where(none, torch.zeros_like(z), torch.exp(p))
    entropy = -torch.where(q > 0, q * p, torch.zeros_like(q)).sum(1)
    valid = (tokens >= 0) & (tokens < x.shape[1])
    given = torch.where(valid, torch.gather(p, 1, tokens.long().clamp(0, x.shape[1] - 1)), torch.zeros((), dtype=torch.float64))
    order = np.argsort(-z.numpy(), axis=1, kind="stable")[:, :n_top]
    return given.numpy(), lse[:, 0].numpy(), entropy.numpy(), order, np.take_along_axis(p.numpy(), order, 1)


def _close(got, want, tol):
    got = got.cpu().double().numpy()
    finite = np.isfinite(want)
    np.testing.assert_array_equal(got[~finite], want[~finite])
    assert np.all(np.abs(got[finite] - want[finite]) <= np.broadcast_to(tol, want.shape)[finite])


def _check(xd, x, tokens, n_top, **kw):
    logprob, lse, entropy, top_idx, top_logprob = sk.sk_logprobs(xd, tokens.cuda(), n_top, **kw)
    torch.cuda.synchronize()
    given, l, h, order, tp = _expected(x, tokens, n_top)
    vocab = x.shape[1]
    np.testing.assert_array_equal(top_idx.cpu().numpy(), order)
    _close(logprob, given, _tolerance(vocab, np.where(np.isfinite(given), given, 0)))
    _close(lse, l, _tolerance(vocab, np.where(np.isfinite(l), l, 0)))
    _close(entropy, h, 2 * _tolerance(vocab, h))
    _close(top_logprob, tp, _tolerance(vocab, np.where(np.isfinite(tp), tp, 0)))


def test_refusals_without_a_gpu():
    L = sk.lib()
    p = 4096                                                  # an address that no call below gets as far as using
    good = dict(logits=p, dtype=sk.SK_F32, rows=2, vocab=100, stride=100, tokens=p, n_tokens=1, n_top=3, ws=p, ws_bytes=1 << 20,
                logprob=p, lse=p, entropy=p, top_idx=p, top_logprob=p, stream=None)

    def call(**kw):
        return L.sk_logprobs(*{**good, **kw}.values())

    for bad in (dict(rows=-1), dict(rows=sk.SK_LOGPROBS_MAX_ROWS + 1), dict(vocab=0), dict(vocab=sk.SK_LOGPROBS_MAX_VOCAB + 1, stride=1 << 22),
                dict(stride=99), dict(n_tokens=-1), dict(n_top=-1), dict(n_top=sk.SK_LOGPROBS_MAX_TOP + 1), dict(vocab=2, n_top=3),
                dict(logits=None), dict(tokens=None), dict(logprob=None), dict(top_idx=None), dict(logits=p + 2), dict(ws=p + 8),
                dict(dtype=sk.SK_BF16, logits=p + 1), dict(vocab=40000, stride=40000, ws=None)):
        assert call(**bad) == sk.SK_E_INVAL, bad
    assert call(dtype=2) == sk.SK_E_DTYPE
    need = L.sk_logprobs_workspace_bytes(2, 40000, 3)
    assert need > 0 and call(vocab=40000, stride=40000, ws_bytes=need - 1) == sk.SK_E_WORKSPACE
    assert call(rows=0, logits=None) == sk.SK_OK
    assert L.sk_logprobs_workspace_bytes(0, 100, 3) == 0 and L.sk_logprobs_workspace_bytes(4, 100, 33) == 0
    assert L.sk_logprobs_workspace_bytes(1 << 20, 1 << 21, 32) == 0        # a row to a workgroup: nothing to keep


def _planted(x, n_top):
    """Rows in which an order or a mask can go wrong, as far as there are rows."""
    rows, vocab = x.shape
    last = vocab - 1

    def one(i, f):
        if i < rows:
            f(x[i])
    one(1, lambda r: r.fill_(-1.25))                                                        # all equal
    one(2, lambda r: (r.fill_(-np.inf), r[last].fill_(1.0)))                                # a single one above -inf, in the last place
    one(3, lambda r: r.fill_(-np.inf))
    one(4, lambda r: r.copy_(torch.arange(vocab, dtype=torch.float32) / 64))                # rising: the list is renewed all the way
    one(5, lambda r: r.copy_(-torch.arange(vocab, dtype=torch.float32) / 64))
    one(6, lambda r: r.copy_((torch.arange(vocab) * 7919 % 5).float()))                     # five values only
    one(7, lambda r: (r.fill_(-np.inf), r[vocab // 2:].fill_(-0.0), r[vocab // 2 + 1::2].fill_(0.0)))    # +0 and -0 are equal
    one(8, lambda r: r.mul_(40.0))                                                          # nearly certain
    one(9, lambda r: r.sub_(3.0e4))
    return x


SIZES = [(1, 1, 0, 1), (1, 2, 0, 2), (10, 3, 1, 3), (10, 31, 0, 8), (10, 64, 4, 32), (10, 65, 0, 32), (10, 2047, 0, 5), (10, 2048, 0, 20),
         (10, 2049, 3, 20), (10, 8193, 0, 32), (10, 16400, 1, 1), (10, 50257, 0, 8), (1, 131072, 0, 20), (2, 262145, 0, 32), (1030, 9001, 0, 20), (1100, 130, 5, 4),
         (70, 40001, 3, 32), (130, 70001, 0, 7), (256, 33000, 1, 1), (12, 150001, 0, 32), (300, 20000, 0, 20)]      # several tiles to a wave of sixteen; parts


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,n_top", SIZES)
def test_against_the_definition(dtype, rows, vocab, pad, n_top):
    gen = synth.generator(8, stream=rows + vocab)
    buf = 2.5 * torch.randn((rows, vocab + pad), generator=gen)
    _planted(buf[:, :vocab], n_top)
    buf[:, vocab:] = 1e30                                     # what lies behind a row must not count
    buf = buf.to(synth.torch_dtype(dtype))
    x = buf[:, :vocab].float()
    tokens = torch.randint(0, vocab, (rows, 3), generator=gen, dtype=torch.int32)
    tokens[:, 1] = torch.where(torch.arange(rows) % 3 == 0, -100, vocab - 1).to(torch.int32)
    tokens[rows // 2, 2] = vocab                              # one behind the last
    _check(buf.cuda()[:, :vocab], x, tokens, n_top)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 3, 5])
def test_rows_that_start_anywhere(dtype, shift):
    gen = synth.generator(8, stream=shift)
    flat = (2.5 * torch.randn(7 * 2051 + 8, generator=gen)).to(synth.torch_dtype(dtype))
    x = flat[shift:shift + 7 * 2051].view(7, 2051)
    xd = flat.cuda()[shift:shift + 7 * 2051].view(7, 2051)
    _check(xd, x.float(), torch.randint(0, 2051, (7, 1), generator=gen, dtype=torch.int32), 9)


@pytest.mark.gpu
def test_without_tokens_or_alternatives():
    x = torch.randn((3, 5000), generator=synth.generator(8))
    _check(x.cuda(), x, torch.zeros((3, 0), dtype=torch.int32), 0)
    logprob, lse, entropy, top_idx, top_logprob = sk.sk_logprobs(x.cuda())
    assert logprob.shape == (3, 0) and top_idx.shape == (3, 0) and lse.shape == (3,)
    # optional outputs left out
    out = sk.logprobs_outputs(3, 1, 2, "cuda:0")
    got = sk.sk_logprobs(x.cuda(), torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"), 2, outputs=(out[0], None, None, out[3], None))
    torch.cuda.synchronize()
    assert got[1] is None and int(got[3][0, 0]) == int(x[0].argmax())
    assert sk.sk_logprobs(x.cuda()[:0])[1].shape == (0,)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [70, 300, 5000, 50257])
def test_masks_of_the_lowest_value(vocab, dtype):
    """Tokens masked with the type's lowest number: alone, in stretches that a lane, a wave or a workgroup sees nothing else of, everywhere,
    and beside the largest numbers, where differences overflow."""
    t = synth.torch_dtype(dtype)
    low, high = torch.finfo(t).min, torch.finfo(t).max
    x = (2.5 * torch.randn((8, vocab), generator=synth.generator(8, stream=9))).to(t).float()
    x[0, ::2] = low
    x[1, : vocab - 9] = low
    x[2, 9:] = low
    x[3, :] = low
    x[4, torch.arange(vocab) % 64 != 5] = low
    x[5, :] = low
    x[5, 7:16] = high
    x[6, 20:] = low
    x[6, 3] = high
    x[7, vocab // 3:] = -0.5 * high
    tokens = torch.tensor([[1], [vocab - 1], [0], [2], [5], [8], [3], [0]], dtype=torch.int32)
    _check(x.to(t).cuda(), x, tokens, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [300, 40000])
def test_rows_with_nan_and_infinity(vocab):
    x = torch.randn((4, vocab), generator=synth.generator(8, stream=2))
    x[0, vocab // 2] = np.nan
    x[1, vocab - 1] = np.inf
    x[2, :] = np.nan
    tokens = torch.tensor([[3], [4], [5], [6]], dtype=torch.int32)
    logprob, lse, entropy, top_idx, top_logprob = sk.sk_logprobs(x.cuda(), tokens.cuda(), 8)
    torch.cuda.synchronize()
    for t in (logprob, lse, entropy, top_logprob):
        assert torch.isnan(t[:3]).all() and torch.isfinite(t[3:]).all()
    for r in range(4):
        ids = top_idx[r].tolist()
        assert len(set(ids)) == 8 and min(ids) >= 0 and max(ids) < vocab
    _check(x[3:].cuda(), x[3:], tokens[3:], 8)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(2, 20011), (1100, 20011), (5, 90011)])
def test_captured_and_replayed_on_new_logits(rows, vocab):
    """Two captured calls with workspaces of their own, replayed several times with eager calls in between."""
    gen = synth.generator(8, stream=rows)
    x = [torch.randn((rows, vocab), generator=gen).cuda() for _ in range(2)]
    tokens = torch.randint(0, vocab, (rows, 2), generator=gen, dtype=torch.int32).cuda()
    need = max(16, sk.lib().sk_logprobs_workspace_bytes(rows, vocab, 6))
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [sk.logprobs_outputs(rows, 2, 6, "cuda:0") for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        for i in range(2):
            sk.sk_logprobs(x[i], tokens, 6, workspace=ws[i], outputs=outs[i])
        with torch.cuda.graph(graph, stream=stream):
            for i in range(2):
                sk.sk_logprobs(x[i], tokens, 6, workspace=ws[i], outputs=outs[i])
    torch.cuda.synchronize()
    for _ in range(3):
        for i in range(2):
            x[i].copy_(torch.randn((rows, vocab), generator=gen).cuda())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            want = sk.sk_logprobs(x[i], tokens, 6)
            torch.cuda.synchronize()
            for a, b in zip(outs[i], want):
                assert torch.equal(a, b)


@pytest.mark.gpu
def test_agrees_with_the_greedy_sampler():
    """The two largest logits are those of sk_top2, and their gap that of the log probabilities."""
    x = (2.5 * torch.randn((5, 128256), generator=synth.generator(8, stream=4))).cuda()
    i1, i2, v1, v2, gap = sk.sk_top2(x)
    _, lse, _, top_idx, top_logprob = sk.sk_logprobs(x, n_top=2)
    torch.cuda.synchronize()
    assert torch.equal(top_idx[:, 0], i1) and torch.equal(top_idx[:, 1], i2)
    assert torch.all((top_logprob[:, 0] - top_logprob[:, 1] - gap).abs() <= 2.0 ** -23 * 16)


@pytest.mark.gpu
def test_workspace_too_small_is_an_error():
    x = torch.zeros((2, 40000), device="cuda")
    with pytest.raises(sk.SkError) as e:
        sk.sk_logprobs(x, n_top=4, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == sk.SK_E_WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,length,lower,twos", [("bf16", 2048, (0, 0), (5, 80, 81, 82)), ("f32", 2048, (100, 256), (40, 258, 296, 297))])
def test_an_equal_logit_of_lower_index_comes_behind_a_cut(dtype, length, lower, twos):
    """A flat row fills a wave's list in the middle of a tile, with exactly n_top logits of the largest value listed; one more of that
    value follows, whose index is lower than some of theirs (a tile's steps are not in the order of indices)."""
    x = torch.full((1, length), 1.0)
    x[:, lower[0]:lower[1]] = -5.0
    x[0, list(twos)] = 2.0
    _check(x.to(synth.torch_dtype(dtype)).cuda(), x, torch.zeros((1, 1), dtype=torch.int32), 3)


def _tied(rows, vocab, gen):
    """Flat rows with a lower stretch at their start, in which a larger value is repeated many times by few lanes of one tile."""
    x = torch.full((rows, vocab), 1.0)
    for r in range(rows):
        stretch = int(torch.randint(0, 400, (1,), generator=gen))
        x[r, stretch:stretch + int(torch.randint(1, 400, (1,), generator=gen))] = -5.0
        first = int(torch.randint(0, max(vocab - 600, 1), (1,), generator=gen)) if r % 2 else 0
        lanes = torch.randint(0, min(64, vocab // 8), (1 + r % 9,), generator=gen)
        for _ in range(6):
            at = first + 8 * lanes + torch.randint(0, 8, lanes.shape, generator=gen)
            x[r, at.clamp(max=vocab - 1)] = 2.0
            at = first + 256 + 4 * lanes + torch.randint(0, 4, lanes.shape, generator=gen)
            x[r, at.clamp(max=vocab - 1)] = 2.0
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad", [(150, 2048, 0), (150, 2051, 2), (40, 9001, 0), (40, 40001, 3), (900, 5003, 0)])
def test_ties_at_the_last_place_in_flat_rows(rows, vocab, pad, dtype):
    gen = synth.generator(8, stream=rows + vocab + 1)
    buf = torch.full((rows, vocab + pad), 3.0)
    buf[:, :vocab] = _tied(rows, vocab, gen)
    buf = buf.to(synth.torch_dtype(dtype))
    x, xd = buf[:, :vocab].float(), buf.cuda()[:, :vocab]
    for n_top in (1, 2, 3, 5, 8, 13, 20, 32):
        _check(xd, x, torch.zeros((rows, 1), dtype=torch.int32), n_top)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_over_parts_of_several_tiles(dtype):
    """Rows in parts whose waves take two tiles each: what a later wave of a part reports has lower indices than some of an earlier one."""
    rows, vocab = 100, 262144
    gen = synth.generator(8, stream=12)
    x = torch.full((rows, vocab), 1.0)
    for r in range(rows):                                     # in tiles that are all over one part, or all over the row
        at = torch.randint(0, 8 * 2048 if r % 2 else vocab, (20 + r,), generator=gen)
        x[r, at] = 2.0
    x = x.to(synth.torch_dtype(dtype))
    assert sk.lib().sk_logprobs_workspace_bytes(rows, vocab, 32) == rows * 17 * 4 * (16 + 8 * 32)      # 17 parts of a row's 129 tiles: two to a wave
    for n_top in (5, 32):
        _check(x.cuda(), x.float(), torch.zeros((rows, 1), dtype=torch.int32), n_top)


@pytest.mark.gpu
@pytest.mark.parametrize("call", ["logprobs", "top2"])
@pytest.mark.parametrize("handle", [False, True])
def test_scratch_of_a_call_on_another_stream_is_not_handed_out_before_it_has_run(call, handle):
    """The workspace that the binding makes and drops: as long as the stream of the call is busy, tensors of the current one do not get it."""
    rows, vocab = (100, 262144) if call == "logprobs" else (4200, 128256)
    L = sk.lib()
    need = L.sk_logprobs_workspace_bytes(rows, vocab, 32) if call == "logprobs" else L.sk_top2_workspace_bytes(rows, vocab)
    assert need > 1 << 20                                     # apart from small tensors
    x = torch.randn((rows, vocab), device="cuda")
    want = [t.clone() for t in (sk.sk_logprobs(x, n_top=32) if call == "logprobs" else sk.sk_top2(x))]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    a = torch.empty(need, dtype=torch.uint8, device="cuda")
    place = a.data_ptr()
    del a
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)                         # tens of milliseconds
    stream = side.cuda_stream if handle else side
    got = sk.sk_logprobs(x, n_top=32, stream=stream) if call == "logprobs" else sk.sk_top2(x, stream=stream)
    b = torch.empty(need, dtype=torch.uint8, device="cuda")
    busy = not side.query()
    assert busy and b.data_ptr() != place
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    # a call on the current stream takes that place and leaves it to the next tensor
    del b
    torch.cuda.empty_cache()
    a = torch.empty(need, dtype=torch.uint8, device="cuda")
    place = a.data_ptr()
    del a
    got = sk.sk_logprobs(x, n_top=32) if call == "logprobs" else sk.sk_top2(x)
    assert torch.empty(need, dtype=torch.uint8, device="cuda").data_ptr() == place
