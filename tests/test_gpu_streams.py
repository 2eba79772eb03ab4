"""Calls on a stream that is named: what the binding makes for them, and the caller drops at once, does not get into other tensors before
the stream has come that far."""
import pytest
import torch

import paper_2605_13784_amd as sk
from workloads import synth

SHAPE = synth.CFG2
N = 700


def _pool():
    gen = synth.generator(11, stream=1)
    pool = sk.Pool("bf16", 32, 8, 128, 16, 128, max_sessions=4)
    sids = [pool.sk_session_create() for _ in range(2)]
    q, k, v = (x.cuda() for x in synth.draw_qkv(gen, N, SHAPE))
    for sid in sids:
        pool.sk_session_append(sid, None, k, v)
    return pool, sids, q, k, v


def _calls():
    pool, (a, b), q, k, v = _pool()
    lse = torch.zeros((64, 32), device="cuda")
    x = torch.randn((64, 128256), device="cuda")
    at = [0, 32, 64]
    return {
        "append": lambda s: pool.sk_session_append(a, q[:64], k[:64], v[:64], stream=s),
        "query": lambda s: pool.sk_session_query(a, q[:64], stream=s),
        "batch": lambda s: pool.sk_batch_step([a, b], [sk.SK_OP_QUERY_A] * 2, at, q[:64], k[:64], v[:64], stream=s),
        "questions": lambda s: pool.sk_session_query_shared_prefix(a, q[:32], k[:32], v[:32], q[:64].view(2, 32, 32, 128), k[:64].view(2, 32, 8, 128),
                                                                   v[:64].view(2, 32, 8, 128), stream=s),
        "gather": lambda s: pool.sk_session_gather(a, stream=s),
        "mass": lambda s: (pool.sk_session_attention_mass(a, q[:64], lse, stream=s),),
        "mass of a batch": lambda s: pool.sk_batch_attention_mass([a, b], at, q[:64], lse, stream=s),
        "top2": lambda s: sk.sk_top2(x, stream=s),
        "top2 static": lambda s: sk.sk_top2_static(x, stream=s),
        "logprobs": lambda s: sk.sk_logprobs(x, torch.zeros(64, dtype=torch.int32, device="cuda"), n_top=4, stream=s)}


def _taken_again(places):
    """Of memory at `places` (address -> bytes), what tensors of the same sizes get now (so many that free places in front run out)."""
    got = [torch.empty(size, dtype=torch.uint8, device="cuda") for size in places.values() for _ in range(50)]
    return {t.data_ptr() for t in got} & set(places)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["append", "query", "batch", "questions", "gather", "mass", "mass of a batch", "top2", "top2 static", "logprobs"])
def test_outputs_that_are_dropped_while_their_stream_is_busy(name):
    call = _calls()[name]
    side = torch.cuda.Stream()
    call(None)                                                # (so that the library has loaded what it needs)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(50_000_000)                     # tens of milliseconds
        made = call(stream)
        places = {t.data_ptr(): t.numel() * t.element_size() for t in made}
        del made
        taken = _taken_again(places)
        assert not side.query() and not taken
        torch.cuda.synchronize()
    made = call(None)                                         # on the current stream they are there for the next tensors
    places = {t.data_ptr(): t.numel() * t.element_size() for t in made}
    del made
    assert _taken_again(places)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_the_default_stream_by_its_handle():
    x = torch.randn((64, 128256), device="cuda")
    want = sk.sk_logprobs(x, n_top=4)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = sk.sk_logprobs(x, n_top=4, stream=0)
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))
