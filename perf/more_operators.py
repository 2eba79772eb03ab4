"""Operators around a session's positions and its drafted tokens, as cases that can be timed and compared.

A case is a dict of plain values.  Five kinds:

  append    tokens are committed to a session with the position rotation applied on the way: k rotated into the cache, v as it is, q
            rotated beside it; with "attend" the tokens' causal attention over cache and chunk too.  For pair i of the first
            "rotary" dimensions and angle a = position * inv_freq[i]:  (x, y) -> factor * (x cos a - y sin a, x sin a + y cos a)
  step      the same in a ragged step over many sessions, of tokens that are not committed
  rotate    q and k of a query are rotated
  shift     the positions of cached keys move: each key of a stretch is rotated by its token's difference (one for all, one a
            token, or one a token and KV head).  A pass does that to a fork of the session, so that every pass finds the same cache
  verify    drafted tokens are accepted or rejected by the target's and the draft's probabilities from given uniform numbers, and
            the token behind the accepted ones is drawn

With `own` false a pass computes these from their formulas with elementary torch operations; with `own` true it calls the
library.  Inputs are drawn on the GPU from the seed alone: N(0,1) for projections, N(0, 2.5) for logits, a draft's logits near its
target's, drafted tokens drawn from the draft's distribution.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"

# layer shapes: (dtype, query heads, KV heads, head_dim)
SHAPES = [("bf16", 32, 8, 128), ("bf16", 64, 8, 128), ("bf16", 28, 4, 128), ("bf16", 12, 4, 128), ("bf16", 32, 8, 64),
          ("bf16", 14, 2, 64), ("f32", 4, 4, 64), ("f32", 8, 2, 128)]


def _layer(shape, rotary=None, interleaved=False, base=10000.0, factor=1.0, block=16):
    return {**dict(zip(("dtype", "hq", "hkv", "dim"), shape)), "rotary": rotary or shape[3], "interleaved": interleaved, "base": base,
            "factor": factor, "block": block}


def _append(name, layer, tokens, pos0, gaps=False, cached=0, attend=False):
    return {"name": name, "kind": "append", **layer, "tokens": tokens, "pos0": pos0, "gaps": gaps, "cached": cached, "attend": attend}


def _step(name, layer, sessions, shortest, longest, most, mix):
    return {"name": name, "kind": "step", **layer, "sessions": sessions, "shortest": shortest, "longest": longest, "most": most, "mix": mix}


def _rotate(name, layer, tokens, pos0, gaps=False):
    return {"name": name, "kind": "rotate", **layer, "tokens": tokens, "pos0": pos0, "gaps": gaps}


def _shift(name, layer, cached, first, by, delta):
    return {"name": name, "kind": "shift", **layer, "cached": cached, "first": first, "by": by, "delta": delta}


def _verify(name, seqs, drafted, vocab, dtype="f32", draft=True, near=1.0, greedy=0, pad=0):
    return {"name": name, "kind": "verify", "seqs": seqs, "drafted": drafted, "vocab": vocab, "dtype": dtype, "draft": draft, "near": near,
            "greedy": greedy, "pad": pad}


def listed():
    main = ("bf16", 32, 8, 128)
    return [
        # one decoded token at the shortest context of the latency curves, its attention with it
        _append("append_1_at_2600", _layer(main, base=500000.0), 1, 2600, cached=2600, attend=True),
        # the benchmark's data plane: the commit of a 256-token chunk at position 32,768
        _append("append_256_at_32k", _layer(main, base=500000.0), 256, 32768),
        # an fp32 layer that rotates a part of its dimensions, neighbours in pairs, by scaled angles; positions with gaps, odd sizes
        _append("append_777_f32_partial", _layer(("f32", 8, 2, 128), 64, True, factor=1.2, block=64), 777, 100001, gaps=True),
        # a long prompt's tokens, as many as one call takes
        _append("append_4096", _layer(main, base=500000.0), 4096, 0),
        # a decoding step of 48 young sessions, one to four drafted tokens each
        _step("step_48_sessions", _layer(main, base=500000.0), 48, 64, 1024, 4, 4),
        # the benchmark's query plane: 32 tokens of a question behind 32,768
        _rotate("rotate_32_at_32k", _layer(main, base=500000.0), 32, 32768),
        # a window of the latency curves' shortest length slides by 256 tokens
        _shift("shift_2600", _layer(main, base=500000.0), 2600, 64, "all", -256),
        # behind an eviction that chose by head: every head's tokens moved by numbers of their own; a part of 64 dimensions rotates
        _shift("shift_14801_by_head", _layer(("bf16", 32, 8, 64), 32, block=64), 14801, 500, "head", -3500),
        # the long context, a frozen head before it
        _shift("shift_128k", _layer(main, base=500000.0, block=64), 131072, 1000, "all", -4096),
        # one sequence, four drafted tokens: what a single user waits for
        _verify("verify_1x4", 1, 4, 128256),
        # tokens drafted by looking them up (no probabilities), bf16 rows of odd length, greedy sequences among them
        _verify("verify_16x3_bf16_odd", 16, 3, 50257, dtype="bf16", draft=False, greedy=4),
        # a full step of a drafting server
        _verify("verify_64x4", 64, 4, 128256),
    ]


# ---- drawn cases --------------------------------------------------------------------------------------

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_layer(rng):
    shape = rng.choice(SHAPES + [SHAPES[0]] * 3)
    return _layer(shape, rng.choice([shape[3], shape[3], shape[3] // 2, 32, 48]), rng.random() < 0.35, rng.choice([10000.0, 500000.0, 1000000.0]),
                  rng.choice([1.0, 1.0, 1.0, 1.1]), rng.choice([16, 16, 16, 64, 256]))


def _draw_once(rng):
    kind = rng.choices(["append", "step", "rotate", "shift", "verify"], [5, 1, 2, 4, 4])[0]
    layer = _draw_layer(rng)
    f32 = layer["dtype"] == "f32"
    gaps = rng.random() < 0.3
    pos0 = _log_int(rng, 1, 1000000) - 1
    if kind == "append":
        if rng.random() < 0.3:
            B = layer["block"]
            tokens = min(B, _log_int(rng, 1, 32))
            cached = _log_int(rng, 64, 4096 if f32 else 16384) // B * B + rng.randint(0, B - tokens)
            c = _append("", layer, tokens, pos0, gaps, cached, True)
        else:
            c = _append("", layer, _log_int(rng, 1, 1024 if f32 else 4096), pos0, gaps)
    elif kind == "step":
        c = _step("", layer, rng.randint(2, 48), _log_int(rng, 16, 256), _log_int(rng, 257, 2048), _log_int(rng, 1, 16), rng.randrange(1 << 16))
    elif kind == "rotate":
        c = _rotate("", layer, _log_int(rng, 1, 2048), pos0, gaps)
    elif kind == "shift":
        cached = _log_int(rng, 256, 16384 if f32 else 131072)
        c = _shift("", layer, cached, rng.choice([0, rng.randint(0, cached // 2)]), rng.choice(["all", "all", "token", "head"]),
                   rng.choice([-1, -1, 1]) * _log_int(rng, 1, 100000))
    else:
        c = _verify("", _log_int(rng, 1, 64), rng.choice([0, 1, 2, 3, 4, 5, 8]), _log_int(rng, 1000, 131072), rng.choice(["f32", "f32", "bf16"]),
                    rng.random() < 0.7, rng.choice([0.3, 1.0, 1.0, 3.0]), rng.choice([0, 0, 2, 5]), rng.choice([0, 0, rng.randint(1, 64)]))
    c.pop("name", None)
    return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] * 100, w["flops"])


def draw(rng):
    dearest = max(_cost(c) for c in listed())
    while True:
        c = _draw_once(rng)
        if _cost(c) <= dearest:
            return c


# ---- what a case comes down to ----------------------------------------------------------------------

def _items(case):
    """(cached, tokens) of each session of a ragged step."""
    r = np.random.RandomState(case["mix"])
    n = case["sessions"]
    lengths = [int(case["shortest"] * (case["longest"] / case["shortest"]) ** u) for u in r.uniform(size=n)]
    return list(zip(lengths, [int(x) for x in r.randint(1, case["most"] + 1, size=n)]))


def work(case):
    """Each input read once, each result written once; the rotations' and the attention's products."""
    if case["kind"] == "verify":
        el = 2 if case["dtype"] == "bf16" else 4
        rows = case["seqs"] * (case["drafted"] + 1) + (case["seqs"] * case["drafted"] if case["draft"] else 0)
        return {"bytes": rows * case["vocab"] * el + case["seqs"] * (16.0 * (case["drafted"] + 1) + 8), "flops": 4.0 * rows * case["vocab"]}
    el = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, d, r = case["hq"], case["hkv"], case["dim"], case["rotary"]
    row = hkv * d * el                                       # one token's keys
    if case["kind"] == "shift":
        moved = case["cached"] - case["first"] // case["block"] * case["block"]
        deltas = 4.0 * {"all": 0, "token": 1, "head": hkv}[case["by"]] * (case["cached"] - case["first"])
        return {"bytes": 4.0 * moved * row + deltas, "flops": 3.0 * moved * hkv * r}
    items = _items(case) if case["kind"] == "step" else [(case.get("cached", 0), case["tokens"])]
    T = sum(t for _, t in items)
    nbytes = 2.0 * T * (hq * d * el + row) + (0 if case["kind"] == "rotate" else 2.0 * T * row)
    flops = 3.0 * T * (hq + hkv) * r
    if case["kind"] == "step" or case.get("attend"):
        nbytes += sum(n for n, _ in items) * 2 * row + T * hq * d * el
        flops += sum(4.0 * d * hq * (t * n + t * (t + 1) / 2) for n, t in items)
    return {"bytes": nbytes, "flops": flops}


# ---- inputs -----------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed) & 0x7FFFFFFF)


def _normal(gen, shape, dtype="f32"):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _inv_freq(case):
    return case["base"] ** (-np.arange(0, case["rotary"], 2, dtype=np.float64) / case["rotary"])


def _positions(case, gen, tokens):
    """Consecutive ones, or with gaps of up to three tokens that other sequences of the text have taken out."""
    if not case.get("gaps"):
        return None
    steps = torch.randint(1, 5, (tokens,), generator=gen, device=DEVICE, dtype=torch.int64)
    return (case["pos0"] + torch.cumsum(steps, 0) - steps).to(torch.int32)


def _draw_rows(case, gen, T):
    q = _normal(gen, (T, case["hq"], case["dim"]), case["dtype"])
    return q, _normal(gen, (T, case["hkv"], case["dim"]), case["dtype"]), _normal(gen, (T, case["hkv"], case["dim"]), case["dtype"])


def _draw_append(case, gen):
    s = dict(zip("qkv", _draw_rows(case, gen, case["tokens"])))
    s["positions"] = _positions(case, gen, case["tokens"])
    if case.get("attend"):
        _, s["kc"], s["vc"] = _draw_rows({**case, "hq": 1}, gen, case["cached"])
    return s


def _draw_step(case, gen):
    items = _items(case)
    s = dict(zip("qkv", _draw_rows(case, gen, sum(t for _, t in items))))
    s["positions"] = torch.cat([torch.arange(n, n + t, device=DEVICE, dtype=torch.int32) for n, t in items])
    s["cu"] = [int(x) for x in np.concatenate([[0], np.cumsum([t for _, t in items])])]
    s["caches"] = [_draw_rows({**case, "hq": 1}, gen, n)[1:] for n, _ in items]
    return s


def _draw_shift(case, gen):
    _, k, v = _draw_rows({**case, "hq": 1}, gen, case["cached"])
    n = case["cached"] - case["first"]
    delta = case["delta"]
    if case["by"] != "all":                                  # what an eviction moves: a little more with every token, up to delta
        shape = (n,) if case["by"] == "token" else (case["hkv"], n)
        left = torch.rand(shape, generator=gen, device=DEVICE) < min(0.9, abs(delta) / n)
        delta = (torch.cumsum(left, -1) * (1 if case["delta"] > 0 else -1)).to(torch.int32)
    return {"k": k, "v": v, "delta": delta}


def _draw_verify(case, gen):
    n, kd, V = case["seqs"], case["drafted"], case["vocab"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    x = 2.5 * _normal(gen, (n, kd + 1, V + case["pad"]))
    x[::3, :, V - V // 8:V] = -math.inf                      # constrained sequences: a part of the vocabulary is not allowed
    y = x[:, :kd] + case["near"] * _normal(gen, (n, kd, V + case["pad"]))
    temperature = 0.5 + torch.rand((n,), generator=gen, device=DEVICE)
    x, y = x.to(dtype)[:, :, :V], y.to(dtype)[:, :, :V]
    # drafted tokens follow the draft's distribution: the largest of logit / T + Gumbel noise
    tokens = torch.empty((n, kd), dtype=torch.int32, device=DEVICE)
    for i in range(kd):
        noise = -torch.log(-torch.log(torch.rand((n, V), generator=gen, device=DEVICE).clamp(1e-9, 1 - 1e-7)))
        tokens[:, i] = (y[:, i].float() / temperature[:, None] + noise).argmax(1)
    if kd:
        tokens[torch.rand((n,), generator=gen, device=DEVICE) < 1.0 / 8, kd - 1] = -1        # fewer drafted than the most
    if case["greedy"]:
        temperature[::case["greedy"]] = 0.0
        if kd:
            tokens[::case["greedy"], 0] = x[::case["greedy"], 0].float().argmax(1).to(torch.int32)
    u = torch.rand((n, kd + 1), generator=gen, device=DEVICE)
    return {"target": x, "draft": y if case["draft"] else None, "tokens": tokens, "u": u, "temperature": temperature}


def _commit(pool, sid, k, v, piece=4096):
    for t in range(0, k.shape[0], piece):
        pool.sk_session_append(sid, None, k[t:t + piece].contiguous(), v[t:t + piece].contiguous())


def _make_pool(case, blocks, sessions):
    import paper_2605_13784_amd as sk
    pool = sk.Pool(case["dtype"], case["hq"], case["hkv"], case["dim"], case["block"], blocks, max_sessions=sessions)
    pool.sk_pool_set_rotation(_inv_freq(case), interleaved=case["interleaved"], factor=case["factor"])
    return pool


def prepare(case, seed):
    gen = _generator(seed)
    s = {"case": case}
    B = case.get("block", 16)
    if case["kind"] == "verify":
        s.update(_draw_verify(case, gen))
        if own:
            import paper_2605_13784_amd as sk
            s["outputs"] = sk.verify_outputs(case["seqs"], case["drafted"], DEVICE)
            need = sk.lib().sk_verify_workspace_bytes(case["seqs"], case["drafted"], case["vocab"])
            s["workspace"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEVICE)
        return s
    s["inv_freq"] = torch.from_numpy(_inv_freq(case)).to(DEVICE)
    if case["kind"] == "shift":
        s.update(_draw_shift(case, gen))
        n, first = case["cached"], case["first"] // B
        if own:
            # blocks for the session, for the copy of its last, partly filled one, and for those that the fork's moved keys go to
            held, copy, fresh = -(-n // B), 1 if n % B else 0, n // B - first
            pool = s["pool"] = _make_pool(case, held + copy + fresh, 2)
            s["sid"], s["fork"] = pool.sk_session_create(), None
            _commit(pool, s["sid"], s.pop("k"), s.pop("v"))
            k, v = _pool_blocks(case, pool.kv_mem)
            s["cache"] = ([k[:, held + copy:], v[:, held + copy:]] if fresh else []) + (_slots(k[:, held], v[:, held], 0, n % B) if copy else [])
        else:
            s["k"], s["v"] = s["k"].transpose(0, 1).contiguous(), s["v"].transpose(0, 1).contiguous()       # as the pool holds them
        return s
    if case["kind"] == "step":
        s.update(_draw_step(case, gen))
        if own:
            items = _items(case)
            pool = s["pool"] = _make_pool(case, sum(-(-n // B) for n, _ in items), len(items))
            s["sids"] = [pool.sk_session_create() for _ in items]
            for sid, (k, v) in zip(s["sids"], s.pop("caches")):
                _commit(pool, sid, k, v)
    else:
        s.update(_draw_append(case, gen))
        if own:
            n, T = case.get("cached", 0), case["tokens"]
            pool = s["pool"] = _make_pool(case, -(-(n + T) // B), 1)
            s["sid"] = None
            if case.get("attend"):
                s["sid"] = pool.sk_session_create()
                _commit(pool, s["sid"], s.pop("kc"), s.pop("vc"))
            if case["kind"] == "append":
                k, v = _pool_blocks(case, pool.kv_mem)
                last, r = (n + T) // B, (n + T) % B
                if case["attend"]:
                    s["cache"] = _slots(k[:, n // B], v[:, n // B], n % B, T)
                else:
                    s["cache"] = ([k[:, :last], v[:, :last]] if last else []) + (_slots(k[:, last], v[:, last], 0, r) if r else [])
    if own:
        s["q_out"] = torch.empty_like(s["q"])
        if case["kind"] == "rotate":
            s["k_out"] = torch.empty_like(s["k"])
        elif case["kind"] == "step" or case["attend"]:
            s["out"] = torch.empty_like(s["q"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------

def _pool_blocks(case, kv_mem):
    """A pool's blocks as K [Hkv][block][slot][d] and V [Hkv][block][group][slot][d], views of its memory: per KV head and block K row
    by row, then V transposed within groups of 16 tokens (bf16) or row by row (fp32)."""
    B, d, hkv = case["block"], case["dim"], case["hkv"]
    mem = kv_mem.view(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32).view(hkv, -1, 2, B * d)
    n = mem.shape[1]
    v = mem[:, :, 1].view(hkv, n, B // 16, d, 16).transpose(3, 4) if case["dtype"] == "bf16" else mem[:, :, 1].view(hkv, n, B // 16, 16, d)
    return mem[:, :, 0].view(hkv, n, B, d), v


def _slots(k, v, first, count):
    """Slots first .. first + count - 1 of one block: K [Hkv][count][d], and V 16-slot group by group."""
    got, t = [k[:, first:first + count]], first
    while t < first + count:
        end = min(first + count, (t // 16 + 1) * 16)
        got.append(v[:, t // 16, t % 16:t % 16 + end - t])
        t = end
    return got


def _run_own(s, case):
    import paper_2605_13784_amd as sk
    if case["kind"] == "verify":
        return list(sk.sk_verify(s["target"], s["tokens"], s["u"], draft=s["draft"], temperature=s["temperature"], workspace=s["workspace"],
                                 outputs=s["outputs"]))
    pool = s["pool"]
    if case["kind"] == "rotate":
        return list(pool.sk_rotate(s["q"], s["k"], positions=s["positions"], pos0=case["pos0"], q_out=s["q_out"], k_out=s["k_out"]))
    if case["kind"] == "step":
        ops = [sk.SK_OP_QUERY_B] * case["sessions"]
        return list(pool.sk_batch_step_rotated(s["sids"], ops, s["cu"], s["positions"], s["q"], s["k"], s["v"], q_out=s["q_out"], out=s["out"],
                                               out_dtype=case["dtype"])[:2])
    if case["kind"] == "append":
        if case["attend"]:
            pool.sk_session_truncate(s["sid"], case["cached"])
            got = pool.sk_session_append_rotated(s["sid"], s["q"], s["k"], s["v"], positions=s["positions"], pos0=case["pos0"], q_out=s["q_out"],
                                                 out=s["out"], out_dtype=case["dtype"])
            return s["cache"] + list(got[:2])
        if s["sid"] is not None:
            pool.sk_session_destroy(s["sid"])
        s["sid"] = pool.sk_session_create()
        got = pool.sk_session_append_rotated(s["sid"], s["q"], s["k"], s["v"], positions=s["positions"], pos0=case["pos0"], q_out=s["q_out"],
                                             attend=False)
        return s["cache"] + [got[0]]
    if s["fork"] is not None:                                # the blocks go back in the order in which they are taken again
        pool.sk_session_truncate(s["fork"], case["cached"] // case["block"] * case["block"])
        pool.sk_session_destroy(s["fork"])
    s["fork"] = pool.sk_session_fork(s["sid"], case["cached"])
    pool.sk_session_shift(s["fork"], s["delta"], first=case["first"])
    return s["cache"]


def _turn(case, x, position, inv_freq, factor):
    """Rows [.., d] turned by the angles of positions that broadcast against [..]: angles in 64 bits, products in 32, rounded once."""
    r = case["rotary"]
    angle = position.double()[..., None] * inv_freq
    cos, sin = (factor * torch.cos(angle)).float(), (factor * torch.sin(angle)).float()
    if case["interleaved"]:
        a, b = x[..., 0:r:2].float(), x[..., 1:r:2].float()
    else:
        a, b = x[..., :r // 2].float(), x[..., r // 2:r].float()
    out = x.clone()
    first, second = (a * cos - b * sin).to(x.dtype), (a * sin + b * cos).to(x.dtype)
    if case["interleaved"]:
        out[..., 0:r:2], out[..., 1:r:2] = first, second
    else:
        out[..., :r // 2], out[..., r // 2:r] = first, second
    return out


def _token_positions(case, s):
    if s["positions"] is not None:
        return s["positions"]
    return torch.arange(case["pos0"], case["pos0"] + case["tokens"], device=DEVICE)


def _blocks(case, x, blocks):
    """[tokens][Hkv][d] -> [Hkv][block][slot][d], the last block partly filled."""
    y = torch.zeros((case["hkv"], blocks * case["block"], case["dim"]), dtype=x.dtype, device=DEVICE)
    y[:, :x.shape[0]] = x.transpose(0, 1)
    return y.view(case["hkv"], blocks, case["block"], case["dim"])


def _groups(case, x):
    """[Hkv][block][slot][d] -> [Hkv][block][group][slot][d]"""
    return x.view(*x.shape[:2], case["block"] // 16, 16, case["dim"])


def _laid_out(case, k, v, n):
    """What an append leaves in the cache, behind n cached tokens."""
    B, T = case["block"], k.shape[0]
    if case["attend"]:                                       # within one block
        kb = torch.zeros((case["hkv"], B, case["dim"]), dtype=k.dtype, device=DEVICE)
        vb = torch.zeros_like(kb)
        kb[:, n % B:n % B + T], vb[:, n % B:n % B + T] = k.transpose(0, 1), v.transpose(0, 1)
        return _slots(kb, vb.view(case["hkv"], B // 16, 16, case["dim"]), n % B, T)
    last, r = T // B, T % B
    kb = _blocks(case, k, last + (r > 0))
    vb = _groups(case, _blocks(case, v, last + (r > 0)))
    return ([kb[:, :last], vb[:, :last]] if last else []) + (_slots(kb[:, last], vb[:, last], 0, r) if r else [])


def _plain_attention(case, q, k, v, n):
    """Causal attention of the newest tokens: token i of q sees n + i + 1 of the keys."""
    T, hkv, d = q.shape[0], case["hkv"], case["dim"]
    G = case["hq"] // hkv
    rows = q.view(T, hkv, G, d).permute(1, 0, 2, 3).reshape(hkv, T * G, d).float()
    x = torch.bmm(rows, k.permute(1, 2, 0).float().contiguous()) * d ** -0.5
    sees = (n + 1 + torch.arange(T, device=DEVICE)).repeat_interleave(G)
    x = torch.where(torch.arange(n + T, device=DEVICE)[None, :] < sees[:, None], x, torch.full((), -math.inf, device=DEVICE))
    w = torch.exp(x - x.max(2, keepdim=True)[0])
    out = torch.bmm(w, v.transpose(0, 1).float().contiguous()) / w.sum(2, keepdim=True)
    return out.view(hkv, T, G, d).permute(1, 0, 2, 3).reshape(T, case["hq"], d).to(q.dtype)


def _plain_shift(case, s):
    B, n, first = case["block"], case["cached"], case["first"]
    delta = s["delta"] if case["by"] != "all" else torch.full((n - first,), case["delta"], device=DEVICE)
    b0, whole, r = first // B, n // B, n % B
    k = s["k"][:, b0 * B:].clone()
    k[:, first - b0 * B:] = _turn(case, s["k"][:, first:], delta, s["inv_freq"], 1.0)
    v = s["v"][:, b0 * B:].clone()
    w, got = whole - b0, []
    if w:
        got = [k[:, :w * B].reshape(case["hkv"], w, B, case["dim"]), _groups(case, v[:, :w * B].reshape(case["hkv"], w, B, case["dim"]))]
    if r:
        vb = torch.zeros((case["hkv"], B, case["dim"]), dtype=v.dtype, device=DEVICE)
        vb[:, :r] = v[:, w * B:]
        got += _slots(k[:, w * B:], vb.view(case["hkv"], B // 16, 16, case["dim"]), 0, r)
    return got


def _plain_verify(case, s):
    """Probabilities and their running sums in 64 bits: the number drawn lies next to the border of two tokens now and then."""
    n, kd, V = case["seqs"], case["drafted"], case["vocab"]
    greedy = s["temperature"] <= 0
    T = torch.where(greedy, torch.ones((), device=DEVICE), s["temperature"]).double()[:, None, None]

    def log_softmax(x):
        z = x.double() / T
        z = z - z.max(2, keepdim=True)[0]
        return z - torch.log(torch.exp(z).sum(2, keepdim=True))

    lp = log_softmax(s["target"])
    p = torch.exp(lp)
    best = s["target"].float().max(2, keepdim=True)[0]
    best = torch.where(s["target"].float() == best, torch.arange(V, device=DEVICE), V).min(2)[0]      # the lowest index of the largest
    valid = (s["tokens"] >= 0) & (s["tokens"] < V)
    at = s["tokens"].clamp(0, V - 1).long()[:, :, None]
    px = torch.gather(p[:, :kd], 2, at)[:, :, 0]
    if s["draft"] is not None:
        q = torch.exp(log_softmax(s["draft"]))
        qx = torch.gather(q, 2, at)[:, :, 0]
    else:
        q = torch.zeros((n, kd, V), dtype=torch.float64, device=DEVICE).scatter_(2, at, 1.0)
        qx = torch.ones_like(px)
    taken = torch.where(greedy[:, None], s["tokens"] == best[:, :kd], s["u"][:, :kd].double() * qx < px) & valid
    accepted = torch.cumprod(taken.long(), 1).sum(1)
    # the row that is drawn from: what the draft left of the rejected token's, or the target's own behind the last drafted token
    seq = torch.arange(n, device=DEVICE)
    w = p[seq, accepted]
    if kd:
        last = accepted.clamp(max=kd - 1)
        rejected = (accepted < kd) & valid[seq, last]
        w = torch.where(rejected[:, None], (w - q[seq, last]).clamp(min=0.0), w)
    c = torch.cumsum(w, 1)
    drawn = (c <= s["u"][:, kd:].double() * c[:, -1:]).sum(1)
    drawn = torch.where(greedy, best[seq, accepted], drawn)
    tokens = torch.full((n, kd + 1), -1, dtype=torch.int32, device=DEVICE)
    place = torch.arange(kd + 1, device=DEVICE)
    tokens[:, :kd] = torch.where(place[:kd] < accepted[:, None], s["tokens"], tokens[:, :kd])
    tokens[seq, accepted] = drawn.to(torch.int32)
    logprob = torch.gather(lp, 2, tokens.clamp(min=0).long()[:, :, None])[:, :, 0]
    return [accepted.to(torch.int32), tokens, torch.where(tokens >= 0, logprob, torch.zeros((), dtype=torch.float64, device=DEVICE)).float()]


def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["kind"] == "verify":
        return _plain_verify(case, s)
    if case["kind"] == "shift":
        return _plain_shift(case, s)
    position = (s["positions"] if case["kind"] == "step" else _token_positions(case, s))[:, None]
    q, k = (_turn(case, x, position, s["inv_freq"], case["factor"]) for x in (s["q"], s["k"]))
    if case["kind"] == "rotate":
        return [q, k]
    if case["kind"] == "append":
        got = _laid_out(case, k, s["v"], case["cached"]) + [q]
        if case["attend"]:
            got.append(_plain_attention(case, q, torch.cat([s["kc"], k]), torch.cat([s["vc"], s["v"]]), case["cached"]))
        return got
    parts = [_plain_attention(case, q[a:b], torch.cat([kc, k[a:b]]), torch.cat([vc, s["v"][a:b]]), kc.shape[0])
             for a, b, (kc, vc) in zip(s["cu"], s["cu"][1:], s["caches"])]
    return [q, torch.cat(parts)]


# ---- from the definitions, in 64 bits -----------------------------------------------------------------

def _exact_turn(case, x, position, factor):
    """Pairs as complex numbers times factor * exp(i * angle)."""
    r, x = case["rotary"], x.double()
    f = torch.from_numpy(_inv_freq(case)).to(DEVICE)
    angle = position.double().unsqueeze(-1) * f
    turn = float(factor) * torch.polar(torch.ones_like(angle), angle)
    if case["interleaved"]:
        z = torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous()) * turn
        head = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * turn
        head = torch.cat([z.real, z.imag], -1)
    return torch.cat([head, x[..., r:]], -1)


def _exact_attention(case, q, k, v, n):
    """q and k as the pool's type holds them."""
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    q, k, v = q.to(t).double(), k.to(t).double(), v.double()
    out = torch.empty_like(q)
    for i in range(q.shape[0]):
        for h in range(case["hq"]):
            g = h // (case["hq"] // case["hkv"])
            x = k[:n + i + 1, g] @ q[i, h] / math.sqrt(case["dim"])
            out[i, h] = torch.softmax(x, 0) @ v[:n + i + 1, g]
    return out


def _exact_blocks(case, x, t0, t1):
    """[Hkv][tokens][d], tokens t0 .. t1 - 1 in whole blocks"""
    return x[:, t0:t1].reshape(case["hkv"], (t1 - t0) // case["block"], case["block"], case["dim"])


def _exact_cache(case, k, v, start):
    """[Hkv][tokens][d]: whole blocks, then what is left of them, from slot `start` of a block on if there are no whole ones."""
    B, T = case["block"], k.shape[1]
    got, t = [], 0
    if start is None:
        t = T // B * B
        if t:
            kb, vb = _exact_blocks(case, k, 0, t), _exact_blocks(case, v, 0, t)
            got = [kb, vb.reshape(case["hkv"], t // B, B // 16, 16, case["dim"])]
        if t == T:
            return got
        start = 0
    got.append(k[:, t:])
    cuts = sorted({0, T - t} | {c for c in range(16 - start % 16, T - t, 16)})
    return got + [v[:, t + a:t + b] for a, b in zip(cuts, cuts[1:])]


def _exact_verify(case, s):
    n, kd, V = case["seqs"], case["drafted"], case["vocab"]
    accepted, tokens = np.zeros(n, np.int32), np.full((n, kd + 1), -1, np.int32)
    logprob = torch.zeros((n, kd + 1), dtype=torch.float64, device=DEVICE)
    given, u, temperature = s["tokens"].cpu().numpy(), s["u"].cpu().numpy().astype(np.float64), s["temperature"].cpu().numpy()
    for i in range(n):
        T = float(temperature[i])
        for j in range(kd + 1):
            z = s["target"][i, j].double()
            lp = torch.log_softmax(z / T if T > 0 else z, 0)
            p = lp.exp()
            t = int(given[i, j]) if j < kd else -1
            w, took = p, False
            if T <= 0:
                top = int((z == z.max()).nonzero()[0, 0])
                took = t == top
            elif t >= 0:
                if s["draft"] is not None:
                    q = torch.softmax(s["draft"][i, j].double() / T, 0)
                else:
                    q = torch.zeros_like(p)
                    q[t] = 1.0
                took = u[i, j] * float(q[t]) < float(p[t])
                w = torch.relu(p - q)
            if not took:
                if T <= 0:
                    t = top
                else:
                    c = torch.cumsum(w, 0)
                    t = int(torch.searchsorted(c, c[-1] * u[i, kd], right=True))
            tokens[i, j], logprob[i, j] = t, lp[t]
            accepted[i] = j
            if not took:
                break
    return [torch.from_numpy(accepted).to(DEVICE), torch.from_numpy(tokens).to(DEVICE), logprob]


def exact(case, seed):
    gen = _generator(seed)
    if case["kind"] == "verify":
        return _exact_verify(case, _draw_verify(case, gen))
    if case["kind"] == "shift":
        s = _draw_shift(case, gen)
        k, v = s["k"].transpose(0, 1).double(), s["v"].transpose(0, 1).double()
        delta = s["delta"] if case["by"] != "all" else torch.tensor(case["delta"], device=DEVICE)
        f = case["first"]
        b0 = f // case["block"] * case["block"]
        k = torch.cat([k[:, b0:f], _exact_turn(case, k[:, f:], delta, 1.0)], 1)
        return _exact_cache(case, k, v[:, b0:], None)
    if case["kind"] == "step":
        s = _draw_step(case, gen)
        q, k = (_exact_turn(case, s[x], s["positions"][:, None], case["factor"]) for x in "qk")
        parts = [_exact_attention(case, q[a:b], torch.cat([kc.double(), k[a:b]]), torch.cat([vc, s["v"][a:b]]), kc.shape[0])
                 for a, b, (kc, vc) in zip(s["cu"], s["cu"][1:], s["caches"])]
        return [q, torch.cat(parts)]
    s = _draw_append(case, gen)
    position = _token_positions(case, s)
    q, k = (_exact_turn(case, s[x], position[:, None], case["factor"]) for x in "qk")
    if case["kind"] == "rotate":
        return [q, k]
    n = case["cached"]
    got = _exact_cache(case, k.transpose(0, 1), s["v"].transpose(0, 1).double(), n % case["block"] if case["attend"] else None) + [q]
    if case["attend"]:
        got.append(_exact_attention(case, q, torch.cat([s["kc"].double(), k]), torch.cat([s["vc"], s["v"]]), n))
    return got
