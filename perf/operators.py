"""Operators of a session's upkeep and of its answers, as cases that can be timed and compared.

A case is a dict of plain values.  Four kinds:

  mass      the attention weight that the cached tokens of one session receive from a call's query rows, added
            up per KV head and token:  mass[g][j] = keep * mass[g][j] + sum over rows i and heads h of group g of
            exp(scale * q[i][h] . k[g][j] - lse[i][h])
  mass_batch  the same for the items of a ragged step over many sessions, in one call
  evict     the tokens of lowest accumulated weight leave a session, the others move together in order.  A pass evicts
            from a fork of the session, so that every pass finds the same cache
  logprobs  log probabilities of given tokens, normaliser, entropy and the best alternatives of logit rows

With `own` false a pass computes these from their formulas with elementary torch operations; with `own` true it calls
the library.  Inputs are drawn on the GPU from the seed alone: N(0,1) for projected, position-encoded activations as
everywhere in this repository, log-normal for accumulated weights (a few tokens hold most of it), N(0, 2.5) for logits.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"

# layer shapes: (dtype, query heads, KV heads, head_dim)
SHAPES = [("bf16", 32, 8, 128), ("bf16", 64, 8, 128), ("bf16", 28, 4, 128), ("bf16", 12, 4, 128), ("bf16", 32, 8, 64),
          ("bf16", 14, 2, 64), ("f32", 4, 4, 64), ("f32", 8, 2, 128)]


def _layer(shape):
    return dict(zip(("dtype", "hq", "hkv", "dim"), shape))


def _mass(name, shape, cached, tokens, causal=False, keep=1.0, block=16, frozen=0, evicted=0):
    return {"name": name, "kind": "mass", **_layer(shape), "cached": cached, "tokens": tokens, "causal": causal, "keep": keep,
            "block": block, "frozen": frozen, "evicted": evicted}


def _evict(name, shape, cached, evict, recent, frozen=0, per_head=True, block=16):
    return {"name": name, "kind": "evict", **_layer(shape), "cached": cached, "evict": evict, "recent": recent, "frozen": frozen,
            "per_head": per_head, "block": block}


def _logprobs(name, rows, vocab, tokens, top, dtype="f32", pad=0):
    return {"name": name, "kind": "logprobs", "rows": rows, "vocab": vocab, "tokens": tokens, "top": top, "dtype": dtype, "pad": pad}


def listed():
    layer = ("bf16", 32, 8, 128)
    return [
        # one decoded token at the shortest context of the latency curves: the bookkeeping beside every generated token
        _mass("mass_1_at_2600", layer, 2600, 1),
        # the benchmark's query plane: 32 tokens of a question against 32,768 cached ones
        _mass("mass_32_at_32k", layer, 32768, 32),
        # the benchmark's data plane: the 256 tokens just appended, each up to its own position, on top of decayed sums
        _mass("mass_256_append_at_32k", layer, 32768, 256, causal=True, keep=0.9),
        # a window behind a frozen head with evicted tokens in between, seven query heads per KV head, odd sizes
        _mass("mass_77_window_9001", ("bf16", 28, 4, 128), 9001, 77, causal=True, block=64, frozen=500, evicted=1000),
        # the fp32 path at its workload's size
        _mass("mass_16_f32_1k", ("f32", 4, 4, 64), 1024, 16),
        # a step of the multi-tenant workload: 48 sessions of 2K-64K cached tokens, queries of 1 to 16 tokens
        {"name": "mass_48_sessions", "kind": "mass_batch", **_layer(layer), "block": 16, "sessions": 48, "shortest": 2048, "longest": 65536,
         "most": 16, "mix": 4},
        # the shortest context of the latency curves, cut to a budget of half its tokens
        _evict("evict_2600_to_1300", layer, 2600, 1300, 64),
        # a head_dim 64 layer at the longer context, a frozen head, odd sizes, one choice for all heads
        _evict("evict_14800_to_11303", ("bf16", 32, 8, 64), 14800, 3497, 333, frozen=500, per_head=False, block=64),
        # the long context cut to half
        _evict("evict_128k_to_64k", layer, 131072, 65536, 1024, block=64),
        # one decoded token and its five best alternatives
        _logprobs("logprobs_1_top5", 1, 128256, 1, 5),
        # bf16 logits in rows of odd length that lie next to each other, three candidates a row
        _logprobs("logprobs_200_bf16_odd", 200, 50257, 3, 8, dtype="bf16"),
        # a prompt of 1,024 tokens scored, with alternatives
        _logprobs("logprobs_1024_top20", 1024, 128256, 1, 20),
    ]


# ---- drawn cases --------------------------------------------------------------------------------------

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choices(["mass", "mass_batch", "evict", "logprobs"], [5, 1, 4, 4])[0]
    block = rng.choice([16, 16, 16, 64, 256])
    shape = rng.choice(SHAPES + [SHAPES[0]] * 3)
    f32 = shape[0] == "f32"
    if kind == "mass":
        causal = rng.random() < 0.4
        cached = _log_int(rng, 64, 16384 if f32 else 131072)
        tokens = min(cached, _log_int(rng, 1, 2048 if causal else 128))
        window = rng.random() < 0.25
        frozen = rng.randint(0, min(500, cached)) if window else 0
        c = _mass("", shape, cached, tokens, causal, rng.choice([0.0, 1.0, 0.9]), block, frozen, _log_int(rng, 10, 2000) if window else 0)
    elif kind == "mass_batch":
        c = {"kind": kind, **_layer(shape), "block": block, "sessions": rng.randint(2, 48), "shortest": _log_int(rng, 64, 2048),
             "longest": _log_int(rng, 2100, 8192 if f32 else 65536), "most": _log_int(rng, 1, 64), "mix": rng.randrange(1 << 16)}
    elif kind == "evict":
        cached = _log_int(rng, 1024, 16384 if f32 else 131072)
        frozen = rng.choice([0, rng.randint(1, 500)])
        recent = rng.randint(0, cached // 8)
        # (a block's worth at least: fewer free no memory)
        c = _evict("", shape, cached, _log_int(rng, block, cached - frozen - recent), recent, frozen, rng.random() < 0.6, block)
    else:
        c = _logprobs("", _log_int(rng, 1, 1024), _log_int(rng, 1000, 131072), rng.choice([0, 1, 1, 2, 4]), rng.choice([0, 1, 5, 20, 32]),
                      rng.choice(["f32", "f32", "bf16"]), rng.choice([0, 0, rng.randint(1, 64)]))
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
    ratio = max(1.0, case["longest"] / case["shortest"])
    lengths = [int(case["shortest"] * ratio ** u) for u in r.uniform(size=n)]
    return list(zip(lengths, [int(x) for x in r.randint(1, case["most"] + 1, size=n)]))


def work(case):
    """Each input read once, each result written once; the products of rows and keys."""
    if case["kind"] == "logprobs":
        el = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["rows"] * (case["vocab"] * el + 8 + 8 * case["tokens"] + 8 * case["top"]),
                "flops": 4.0 * case["rows"] * case["vocab"]}
    el = 2 if case["dtype"] == "bf16" else 4
    row = case["hkv"] * case["dim"] * el                     # one token's keys
    if case["kind"] == "evict":
        kept = case["cached"] - case["evict"] - case["frozen"] // case["block"] * case["block"]
        return {"bytes": 2.0 * 2 * kept * row + 8.0 * case["hkv"] * case["cached"], "flops": float(case["hkv"] * case["cached"])}
    nbytes = flops = 0.0
    for n, T in ([(case["cached"], case["tokens"])] if case["kind"] == "mass" else _items(case)):
        pairs = T * n - (T * (T - 1) / 2.0 if case.get("causal") else 0)
        nbytes += n * row + T * case["hq"] * (case["dim"] * el + 4) + n * case["hkv"] * (8 if case.get("keep", 1.0) else 4)
        flops += 2.0 * case["dim"] * case["hq"] * pairs
    return {"bytes": nbytes, "flops": flops}


# ---- inputs -----------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed) & 0x7FFFFFFF)


def _normal(gen, shape, dtype="f32"):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _weights(gen, shape):
    """Accumulated weights: log-normal, some tokens never looked at."""
    w = torch.exp(1.5 * _normal(gen, shape))
    return torch.where(torch.rand(shape, generator=gen, device=DEVICE) < 1.0 / 64, torch.zeros((), device=DEVICE), w)


def _heads(x, hkv):
    """[T][Hq][d] -> [Hkv][T * G][d]: the rows that read one KV head, token by token."""
    T, hq, d = x.shape
    return x.view(T, hkv, hq // hkv, d).permute(1, 0, 2, 3).reshape(hkv, T * (hq // hkv), d)


def _visible(case, n, T):
    """Keys that each row of a KV head sees: its own position's and those before it, or all."""
    G = case["hq"] // case["hkv"]
    if not case.get("causal"):
        return torch.full((T * G,), n, device=DEVICE, dtype=torch.int64)
    return (n - T + 1 + torch.arange(T, device=DEVICE)).repeat_interleave(G)


def _lse(case, q, k):
    """Log-sum-exp of each row's scaled scores, as the attention call over the same rows leaves it: [T][Hq]."""
    T, n = q.shape[0], k.shape[0]
    G = case["hq"] // case["hkv"]
    visible = _visible(case, n, T)
    keys = torch.arange(n, device=DEVICE)
    out = torch.empty((case["hkv"], T * G), dtype=torch.float32, device=DEVICE)
    for g in range(case["hkv"]):
        kg = k[:, g].float()
        for r in range(0, T * G, 512):
            s = (_heads(q, case["hkv"])[g, r:r + 512].float() @ kg.t()) * case["dim"] ** -0.5
            s.masked_fill_(keys >= visible[r:r + 512, None], -math.inf)
            out[g, r:r + 512] = torch.logsumexp(s, 1)
    return out.view(case["hkv"], T, G).permute(1, 0, 2).reshape(T, case["hq"]).contiguous()


def _draw_mass(case, gen, n, T, evicted=0):
    """q, the session's K and V with `evicted` tokens that leave it behind the frozen ones, lse and sums so far."""
    held = n + evicted
    q = _normal(gen, (T, case["hq"], case["dim"]), case["dtype"])
    k = _normal(gen, (held, case["hkv"], case["dim"]), case["dtype"])
    f = case.get("frozen", 0)
    kept = torch.cat([k[:f], k[f + evicted:]]) if evicted else k
    return {"q": q, "k": k, "kept": kept, "lse": _lse(case, q, kept), "mass": _weights(gen, (case["hkv"], n))}


def _draw_evict(case, gen):
    shape = (case["cached"], case["hkv"], case["dim"])
    k, v = _normal(gen, shape, case["dtype"]), _normal(gen, shape, case["dtype"])
    return {"k": k, "v": v, "mass": _weights(gen, (case["hkv"], case["cached"]))}


def _draw_logprobs(case, gen):
    rows, vocab = case["rows"], case["vocab"]
    x = 2.5 * _normal(gen, (rows, vocab + case["pad"]))
    x[::4, vocab - vocab // 8:vocab] = -math.inf             # constrained rows: a part of the vocabulary is not allowed
    x = x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)[:, :vocab]
    tokens = torch.randint(0, vocab, (rows, case["tokens"]), generator=gen, device=DEVICE, dtype=torch.int32)
    tokens[torch.rand(tokens.shape, generator=gen, device=DEVICE) < 1.0 / 16] = -1      # padding
    return {"logits": x, "tokens": tokens}


def _commit(pool, sid, k, v, piece=4096):
    for t in range(0, k.shape[0], piece):
        pool.sk_session_append(sid, None, k[t:t + piece].contiguous(), v[t:t + piece].contiguous())


def _make_pool(case, blocks, sessions):
    import paper_2605_13784_amd as sk
    return sk.Pool(case["dtype"], case["hq"], case["hkv"], case["dim"], case["block"], blocks, max_sessions=sessions)


def prepare(case, seed):
    gen = _generator(seed)
    s = {"case": case}
    B = case.get("block", 16)
    if case["kind"] == "logprobs":
        s.update(_draw_logprobs(case, gen))
        if own:
            import paper_2605_13784_amd as sk
            s["outputs"] = sk.logprobs_outputs(case["rows"], case["tokens"], case["top"], DEVICE)
            s["workspace"] = torch.empty(max(16, sk.lib().sk_logprobs_workspace_bytes(case["rows"], case["vocab"], case["top"])),
                                         dtype=torch.uint8, device=DEVICE)
    elif case["kind"] == "mass":
        s.update(_draw_mass(case, gen, case["cached"], case["tokens"], case["evicted"]))
        if own:
            pool = s["pool"] = _make_pool(case, -(-(case["cached"] + case["evicted"]) // B), 1)
            sid = s["sid"] = pool.sk_session_create()
            _commit(pool, sid, s["k"], s["k"])
            if case["frozen"]:
                pool.sk_session_freeze(sid, case["frozen"])
            if case["evicted"]:
                pool.sk_session_evict_oldest(sid, case["evicted"])
            s["mass_out"] = torch.empty_like(s["mass"])
        s.pop("k")
    elif case["kind"] == "mass_batch":
        items = _items(case)
        drawn = [_draw_mass(case, gen, n, T) for n, T in items]
        s["q"], s["lse"] = torch.cat([x["q"] for x in drawn]), torch.cat([x["lse"] for x in drawn])
        s["cu"] = [int(x) for x in np.concatenate([[0], np.cumsum([T for _, T in items])])]
        s["mass"] = [x["mass"] for x in drawn]
        if own:
            pool = s["pool"] = _make_pool(case, sum(-(-n // B) for n, _ in items), len(items))
            s["sids"] = [pool.sk_session_create() for _ in items]
            for sid, x in zip(s["sids"], drawn):
                _commit(pool, sid, x["k"], x["k"])
            s["mass_out"] = [torch.empty_like(m) for m in s["mass"]]
        else:
            s["keys"] = [x["kept"] for x in drawn]
    else:
        s.update(_draw_evict(case, gen))
        n, first = case["cached"], case["frozen"] // B
        if own:
            # blocks for the session, for the copy of its last, partly filled one, and for what a fork keeps behind the
            # blocks that hold frozen tokens only: a fork finds the same ones free each time
            held, copy = -(-n // B), 1 if n % B else 0
            fresh = -(-(n - case["evict"]) // B) - first
            pool = s["pool"] = _make_pool(case, held + copy + fresh, 2)
            sid = s["sid"] = pool.sk_session_create()
            _commit(pool, sid, s.pop("k"), s.pop("v"))
            if case["frozen"]:
                pool.sk_session_freeze(sid, case["frozen"])
            s["fork"] = None
            s["mass_out"] = torch.empty_like(s["mass"])
            s["cache"] = _pieces(case, *_pool_blocks(case, pool.kv_mem, [(0, first), (held + copy, held + copy + fresh)]))
        else:
            # as the pool holds them, a head's tokens next to each other
            s["k"], s["v"] = s["k"].transpose(0, 1).contiguous(), s["v"].transpose(0, 1).contiguous()
    return s


# ---- one pass ---------------------------------------------------------------------------------------

def _pool_blocks(case, kv_mem, ranges):
    """Ranges of a pool's blocks as K [Hkv][block][slot][d] and V [Hkv][block][group][slot][d], views of its memory: per KV
    head and block K row by row, then V transposed within groups of 16 tokens (bf16) or row by row (fp32)."""
    B, d, hkv = case["block"], case["dim"], case["hkv"]
    mem = kv_mem.view(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32).view(hkv, -1, 2, B * d)
    k = [mem[:, a:b, 0].view(hkv, b - a, B, d) for a, b in ranges]
    if case["dtype"] == "bf16":
        return k, [mem[:, a:b, 1].view(hkv, b - a, B // 16, d, 16).transpose(3, 4) for a, b in ranges]
    return k, [mem[:, a:b, 1].view(hkv, b - a, B // 16, 16, d) for a, b in ranges]


def _pieces(case, k, v):
    """The kept tokens' K and V among blocks: whole blocks, and the tokens, 16-token groups and rest of the last, partly filled one."""
    r = (case["cached"] - case["evict"]) % case["block"]
    if not r:
        return k + v
    tail = [k[-1][:, -1, :r], v[-1][:, -1, :r // 16], v[-1][:, -1, r // 16, :r % 16]]
    return k[:-1] + [k[-1][:, :-1]] + v[:-1] + [v[-1][:, :-1]] + tail


def _run_own(s, case):
    import paper_2605_13784_amd as sk
    if case["kind"] == "logprobs":
        logprob, lse, entropy, top, top_logprob = sk.sk_logprobs(s["logits"], s["tokens"], case["top"], workspace=s["workspace"], outputs=s["outputs"])
        return [logprob, lse, entropy, top, top_logprob]
    pool = s["pool"]
    if case["kind"] == "mass":
        return pool.sk_session_attention_mass(s["sid"], s["q"], s["lse"], causal=case["causal"], mass_in=s["mass"], keep=case["keep"],
                                              mass_out=s["mass_out"])
    if case["kind"] == "mass_batch":
        return pool.sk_batch_attention_mass(s["sids"], s["cu"], s["q"], s["lse"], mass_in=s["mass"], mass_out=s["mass_out"])
    if s["fork"] is not None:
        pool.sk_session_destroy(s["fork"])
    s["fork"] = pool.sk_session_fork(s["sid"], case["cached"])
    mass = pool.sk_session_evict_lowest(s["fork"], s["mass"], case["evict"], n_recent=case["recent"], per_head=case["per_head"],
                                        mass_out=s["mass_out"])
    return s["cache"] + [mass]


def _plain_mass(case, q, k, lse, mass, keep):
    """Scores of a KV head's rows and keys, their weights by the rows' log-sum-exp, summed over the rows."""
    n, T, hkv = k.shape[0], q.shape[0], case["hkv"]
    rows, norm = _heads(q, hkv).float(), _heads(lse[:, :, None], hkv)
    s = torch.bmm(rows, k.permute(1, 2, 0).float().contiguous()) * case["dim"] ** -0.5
    w = torch.exp(s - norm)
    if case.get("causal"):
        w = torch.where(torch.arange(n, device=DEVICE)[None, :] < _visible(case, n, T)[:, None], w, torch.zeros((), device=DEVICE))
    w = w.sum(1)
    return w if keep == 0.0 else keep * mass + w


def _plain_evict(case, k, v, mass):
    n, f, gone = case["cached"], case["frozen"], case["evict"]
    score = mass
    if not case["per_head"]:                                 # one choice for all heads, by the heads' sum in their order
        score = mass[0]
        for g in range(1, case["hkv"]):
            score = score + mass[g]
        score = score[None]
    order = torch.sort(score[:, f:n - case["recent"]], dim=1, stable=True)[1]          # equal weights: the older token first
    keep = torch.ones((score.shape[0], n), dtype=torch.bool, device=DEVICE)
    keep.scatter_(1, f + order[:, :gone], False)
    index = keep.nonzero()[:, 1].view(score.shape[0], n - gone).expand(case["hkv"], n - gone)
    out = torch.zeros_like(mass)
    out[:, :n - gone] = torch.gather(mass, 1, index)
    B, first = case["block"], f // case["block"]
    blocks = -(-(n - gone) // B)

    def cut(x):                                              # into blocks, the last one partly filled
        y = torch.zeros((case["hkv"], blocks * B, case["dim"]), dtype=x.dtype, device=DEVICE)
        torch.gather(x, 1, index[:, :, None].expand(-1, -1, case["dim"]), out=y[:, :n - gone])
        return y.view(case["hkv"], blocks, B, case["dim"])

    kb, vb = cut(k), cut(v).view(case["hkv"], blocks, B // 16, 16, case["dim"])
    return _pieces(case, [kb[:, :first], kb[:, first:]], [vb[:, :first], vb[:, first:]]) + [out]


def _plain_logprobs(case, x, tokens):
    x = x.float()
    m = x.max(1, keepdim=True)[0]
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    # p log p, nothing where p is 0
    entropy = torch.log(total[:, 0]) - torch.where(e > 0, e * (x - m), torch.zeros((), device=DEVICE)).sum(1) / total[:, 0]
    given = torch.gather(x, 1, tokens.clamp(min=0).long()) - lse
    given = torch.where((tokens >= 0) & (tokens < case["vocab"]), given, torch.zeros((), device=DEVICE))
    value, index = torch.sort(x, dim=1, descending=True, stable=True)                  # equal logits: the lower index first
    return [given, lse[:, 0], entropy, index[:, :case["top"]].to(torch.int32), value[:, :case["top"]] - lse]


def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["kind"] == "logprobs":
        return _plain_logprobs(case, s["logits"], s["tokens"])
    if case["kind"] == "mass":
        return _plain_mass(case, s["q"], s["kept"], s["lse"], s["mass"], case["keep"])
    if case["kind"] == "mass_batch":
        return [_plain_mass(case, s["q"][a:b], k, s["lse"][a:b], m, 1.0)
                for a, b, k, m in zip(s["cu"], s["cu"][1:], s["keys"], s["mass"])]
    return _plain_evict(case, s["k"], s["v"], s["mass"])


# ---- from the definitions, in 64 bits -----------------------------------------------------------------

def _exact_mass(case, x, n, T, keep):
    G, scale = case["hq"] // case["hkv"], 1.0 / math.sqrt(case["dim"])
    total = torch.zeros((case["hkv"], n), dtype=torch.float64, device=DEVICE)
    for h in range(case["hq"]):
        keys = x["kept"][:, h // G].double().t().contiguous()
        for i in range(0, T, 256):
            w = torch.exp(scale * (x["q"][i:i + 256, h].double() @ keys) - x["lse"][i:i + 256, h].double()[:, None])
            if case.get("causal"):
                w = torch.tril(w, diagonal=n - T + i)
            total[h // G] += w.sum(0)
    return total if keep == 0.0 else total + keep * x["mass"].double()


def _exact_evict(case, x):
    n, f, last, gone = case["cached"], case["frozen"], case["cached"] - case["recent"], case["evict"]
    mass = x["mass"].cpu().numpy()
    left, out = [], np.zeros((case["hkv"], n), np.float64)
    for g in range(case["hkv"]):
        score = mass[g]
        if not case["per_head"]:                             # the sum is defined in 32 bits, head by head
            score = np.zeros(n, np.float32)
            for h in range(case["hkv"]):
                score = score + mass[h]
        leaves = f + np.lexsort((np.arange(last - f), score[f:last]))[:gone]
        left.append(np.delete(np.arange(n), leaves))
        out[g, :n - gone] = mass[g][left[-1]]
    B, b0 = case["block"], f // case["block"]
    m = n - gone
    whole = m // B

    def tokens(t, a, b):                                     # [Hkv][b - a][d]
        return torch.stack([t[torch.from_numpy(left[g][a:b]).to(DEVICE), g] for g in range(case["hkv"])]).double()

    def cut(t, shape):
        return [tokens(t, 0, b0 * B).view(case["hkv"], b0, *shape), tokens(t, b0 * B, whole * B).view(case["hkv"], whole - b0, *shape)]

    d = case["dim"]
    got = cut(x["k"], (B, d)) + cut(x["v"], (B // 16, 16, d))
    if m % B:
        groups = m % B // 16
        got += [tokens(x["k"], whole * B, m), tokens(x["v"], whole * B, whole * B + groups * 16).view(case["hkv"], groups, 16, d),
                tokens(x["v"], whole * B + groups * 16, m)]
    return got + [torch.from_numpy(out).to(DEVICE)]


def _exact_logprobs(case, x):
    ids = x["tokens"].long()
    given = torch.zeros(ids.shape, dtype=torch.float64, device=DEVICE)
    lse, entropy = (torch.empty(case["rows"], dtype=torch.float64, device=DEVICE) for _ in range(2))
    top = torch.empty((case["rows"], case["top"]), dtype=torch.int32, device=DEVICE)
    top_logprob = torch.empty((case["rows"], case["top"]), dtype=torch.float64, device=DEVICE)
    for i in range(case["rows"]):
        z = x["logits"][i].double()
        p = torch.log_softmax(z, 0)
        lse[i] = torch.logsumexp(z, 0)
        entropy[i] = torch.special.entr(p.exp()).sum()
        order = torch.argsort(-z, stable=True)[:case["top"]]
        top[i], top_logprob[i] = order.to(torch.int32), p[order]
        given[i] = torch.where(ids[i] >= 0, p[ids[i].clamp(min=0)], torch.zeros((), dtype=torch.float64, device=DEVICE))
    return [given, lse, entropy, top, top_logprob]


def exact(case, seed):
    gen = _generator(seed)
    if case["kind"] == "logprobs":
        return _exact_logprobs(case, _draw_logprobs(case, gen))
    if case["kind"] == "evict":
        return _exact_evict(case, _draw_evict(case, gen))
    if case["kind"] == "mass":
        return _exact_mass(case, _draw_mass(case, gen, case["cached"], case["tokens"], case["evicted"]), case["cached"], case["tokens"], case["keep"])
    return [_exact_mass(case, _draw_mass(case, gen, n, T), n, T, 1.0) for n, T in _items(case)]
