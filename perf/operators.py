"""Cases of the operators that write and read the 8-bit paged KV pool.

``append``: the new tokens' queries and keys get their rotary positions, and
keys and values go into the pool as E4M3 codes with one power-of-two scale per
block and KV head.  ``attend``: attention of the new tokens over the pool
(decodes, drafts of a few tokens, prefill chunks), with the scores' tanh cap,
the rows' log-sum-exp and the blocks' accumulated attention weight where a
program asks for them.  ``evict``: the blocks with the least accumulated
weight leave their requests; tables, lengths and weights are compacted and the
freed slots listed.

The plain forms below are written from the formulas in elementary torch
operations over padded batches.  Head counts and head sizes are those of the
pool's geometry (8 KV heads of 128, 16 tokens a block) and its shares under
tensor parallelism, with other common ones in the drawn cases; lengths follow
the chat and agentic prompt laws of ``synth``, chunks are of 512 tokens.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -100


# ------------------------------------------------------------------- cases

def listed():
    llm = dict(heads=32, kv_heads=8, dim=128, block=16, dtype="bf16")
    big = dict(heads=64, kv_heads=8, dim=128, block=16, dtype="bf16")
    plain = dict(cap=0.0, window=0, lse=False)
    half = dict(rotary=128, interleaved=False)
    return [
        # one request's next token: the latency of the write
        dict(name="append_1", kind="append", n=1, new=1, law="chat", top=8192, shape=1, **llm, **half),
        # a full decode batch of a 64-head model
        dict(name="append_128", kind="append", n=128, new=1, law="chat", top=8192, shape=2, **big,
             **half),
        # sixteen prefill chunks, interleaved pairs on half of the head, float16
        dict(name="append_chunks_8192", kind="append", n=16, new=512, law="agent", top=8192, shape=3,
             rotary=64, interleaved=True, **dict(llm, dtype="f16")),
        # one request's next token over a short context: latency of the read
        dict(name="decode_1", kind="attend", n=1, new=1, law="chat", top=777, shape=4, **llm, **plain),
        # a full decode batch of chat requests, weights gathered for eviction
        dict(name="decode_128", kind="attend", n=128, new=1, law="chat", top=8192, shape=5, **big,
             **dict(plain, window=1)),
        # a few long contexts: the read of a long cache
        dict(name="decode_long_4", kind="attend", n=4, new=1, law="long", top=131071, shape=6, **llm,
             **dict(plain, lse=True)),
        # drafts of one to eight tokens verified over agentic contexts, capped scores, float16
        dict(name="draft_32", kind="attend", n=32, new=-8, law="agent", top=16384, shape=7,
             **dict(llm, block=32, dtype="f16"), cap=50.0, window=8, lse=True),
        # one prefill chunk late in a long prompt
        dict(name="chunk_512", kind="attend", n=1, new=512, law="long", top=32001, shape=8, **llm, **plain),
        # a step's whole token cap: sixteen chunks of a 64-head model, the
        # last 16 tokens of each gather weights
        dict(name="chunks_8192", kind="attend", n=16, new=512, law="agent", top=8192, shape=9, **big,
             **dict(plain, window=16, lse=True)),
        # one request over its budget
        dict(name="evict_1", kind="evict", n=1, law="agent", top=8192, block=16, shape=10, keep=0.5,
             sink=1, recent=4),
        # a decode batch
        dict(name="evict_128", kind="evict", n=128, law="agent", top=32768, block=16, shape=11, keep=0.5,
             sink=1, recent=4),
        # long contexts cut to an eighth
        dict(name="evict_long_64", kind="evict", n=64, law="long", top=131072, block=16, shape=12,
             keep=0.125, sink=4, recent=64),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(8, 1, 128), (16, 2, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (16, 16, 64), (24, 8, 64),
         (16, 8, 256), (40, 8, 128)]


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "evict"])
    shape = rng.randrange(100, 1 << 30)
    block = rng.choice([16, 16, 32, 64, 128])
    if kind == "evict":
        return dict(kind=kind, n=_log(rng, 1, 128), law=rng.choice(["chat", "agent", "long"]),
                    top=_log(rng, 300, 32768), block=block, shape=shape,
                    keep=round(rng.uniform(0.1, 1.1), 3), sink=rng.randrange(0, 5),
                    recent=rng.randrange(1, 33))
    heads, kv_heads, dim = rng.choice(HEADS)
    model = dict(heads=heads, kv_heads=kv_heads, dim=dim, block=block, dtype=rng.choice(["bf16", "f16"]))
    if kind == "append":
        new = rng.choice([1, -8, _log(rng, 2, 512)])
        return dict(kind=kind, n=_log(rng, 1, 128 if abs(new) <= 8 else 8), new=new,
                    law=rng.choice(["chat", "agent"]), top=_log(rng, 600, 8192), shape=shape,
                    rotary=rng.choice([dim, dim // 2, dim // 4]), interleaved=rng.random() < 0.5, **model)
    form = rng.choice(["decode", "decode", "draft", "chunk"])
    more = dict(cap=rng.choice([0.0, 0.0, 30.0]), window=rng.choice([0, 0, 1, 5]), lse=rng.random() < 0.5)
    if form == "chunk":
        return dict(kind=kind, n=_log(rng, 1, 8), new=_log(rng, 9, 512), law=rng.choice(["chat", "agent"]),
                    top=_log(rng, 600, 8192), shape=shape, **model, **more)
    n = _log(rng, 1, 128)
    return dict(kind=kind, n=n, new=1 if form == "decode" else -8,
                law=rng.choice(["chat", "agent", "long"]), top=_log(rng, 64, min(65536, 300000 // n)),
                shape=shape, **model, **more)


def _lengths(case):
    """New tokens and cached tokens (the new ones included) of each request:
    part of the case, the same for every seed."""
    r = np.random.default_rng(case["shape"])
    n, top = case["n"], case["top"]
    if case["law"] == "chat":
        old = np.exp(r.normal(6, 1, n))
    elif case["law"] == "agent":
        old = np.exp(r.normal(9, 0.7, n))
    else:
        old = top * r.uniform(0.75, 1.0, n)
    old = np.clip(np.rint(old).astype(np.int64), 1, top)
    old[0] = top  # one request reaches the top of the range
    if case["kind"] == "evict":
        return np.zeros(n, np.int64), old
    new = case["new"]
    new = r.integers(1, -new + 1, n) if new < 0 else np.full(n, new, np.int64)
    return new, np.maximum(old, new)


# ----------------------------------------------------------------- prepare

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _ints(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int64)).to(device=DEV, dtype=dtype)


def _chunk_bytes(case):
    """The codes of a block's K or V over all heads, then one scale a head."""
    return case["kv_heads"] * case["block"] * case["dim"], -(-4 * case["kv_heads"] // 16) * 16


def _pool(case, slots, g):
    """A pool of one layer, [K and V, slots, bytes], filled as earlier tokens
    leave it: codes up to the format's largest, scales of powers of two."""
    codes, tail = _chunk_bytes(case)
    pool = torch.zeros(2, slots, codes + tail, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 26) // codes)
    for kv in range(2):
        for a in range(0, slots, step):
            b = min(slots, a + step)
            x = torch.randn(b - a, codes, generator=g, device=DEV).mul_(110).clamp_(-448, 448)
            pool[kv, a:b, :codes] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    e = torch.randint(-8, -5, (2, slots, tail // 4), generator=g, device=DEV)
    pool[:, :, codes:] = torch.exp2(e.float()).view(torch.uint8)
    return pool


def _frequencies(rotary):
    """Turns a position in 2^-64: base 500000, contexts stretched eightfold
    for the slow half of the pairs."""
    j = np.arange(rotary // 2)
    f = 500000.0 ** (-2.0 * j / rotary) / (2 * math.pi)
    f[len(j) // 2:] /= 8
    return torch.from_numpy(np.rint(f * 2.0 ** 64).astype(np.uint64).view(np.int64).copy()).to(DEV)


def prepare(case, seed):
    g = _generator(seed)
    new, length = _lengths(case)
    n, bt = case["n"], case["block"]
    blocks = -(-length // bt)
    rows = np.concatenate([[0], np.cumsum(blocks)])
    entries = int(rows[-1])
    # every request's blocks lie anywhere in the pool; one slot is nobody's
    slots = torch.randperm(entries, generator=g, device=DEV).to(torch.int32)
    s = dict(case=case, n=n, entries=entries, length=_ints(length), rows=_ints(rows), slots=slots,
             most_blocks=int(blocks.max()), most_new=int(new.max()) if n else 0)
    if case["kind"] == "evict":
        # accumulated weights: a few blocks hold most, many hold exactly none
        w = torch.rand(entries, generator=g, device=DEV).pow_(8)
        s["weight"] = torch.where(w < 1e-4, torch.zeros_like(w), w)
        s["keep"] = _ints(np.maximum(1, np.rint(blocks * case["keep"])))
        for name, size in (("length_out", n), ("rows_out", n + 1), ("slots_out", entries),
                           ("freed", entries), ("n_freed", 1)):
            s[name] = torch.zeros(size, dtype=torch.int32, device=DEV)
        s["weight_out"] = torch.zeros(entries, device=DEV)
        if own:
            from paper_2608_06557_amd import device
            s["op"] = device.DeviceKvEvict(bt, s["length"], s["rows"], s["slots"], s["weight"], s["keep"],
                                           sink=case["sink"], recent=case["recent"],
                                           out=(s["length_out"], s["rows_out"], s["slots_out"],
                                                s["weight_out"], s["freed"], s["n_freed"]))
        return s
    dt = TYPES[case["dtype"]]
    tokens = int(new.sum())
    s["pool"] = _pool(case, entries + 1, g)
    s["offsets"] = _ints(np.concatenate([[0], np.cumsum(new)]))
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    # queries, keys and values of the new tokens side by side, as a fused
    # projection leaves them
    x = torch.randn(tokens, heads + 2 * kv_heads, dim, generator=g, device=DEV)
    x *= torch.exp2(torch.randn(heads + 2 * kv_heads, 1, generator=g, device=DEV) * 0.5)
    x = x.to(dt)
    s["q"], s["k"], s["v"] = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    s["out"] = torch.zeros(tokens, heads, dim, dtype=dt, device=DEV)
    if case["kind"] == "append":
        s["freq"] = _frequencies(case["rotary"])
        first = np.repeat(length - new, new)
        s["positions"] = _ints(first + np.arange(tokens) - np.repeat(np.cumsum(new) - new, new))
    else:
        s["scale"] = dim ** -0.5
        s["lse"] = torch.zeros(tokens, heads, device=DEV) if case["lse"] else None
        s["weight"] = torch.rand(entries, generator=g, device=DEV) if case["window"] else None
    if own:
        from paper_2608_06557_amd import device
        kv = device.DeviceKvPool(s["pool"][None], kv_heads, dim, bt)
        batch = device.KvBatch(s["offsets"], s["length"], s["rows"], s["slots"], tokens, s["most_new"])
        if case["kind"] == "append":
            s["op"] = device.DeviceKvAppend(kv, batch, s["q"], s["k"], s["v"], s["out"], s["positions"],
                                            s["freq"], interleaved=case["interleaved"])
        else:
            s["op"] = device.DeviceAttention(kv, batch, s["q"], s["out"], s["scale"], softcap=case["cap"],
                                             lse=s["lse"], block_weight=s["weight"],
                                             weight_window=case["window"])
    return s


# --------------------------------------------------------------------- run

def _padded_blocks(s):
    """Table entry of each request's b-th block, [n, most blocks], and
    whether it has one."""
    b = torch.arange(s["most_blocks"], device=DEV)
    first, last = s["rows"][:-1, None].long(), s["rows"][1:, None].long()
    entry = first + b
    return torch.minimum(entry, last - 1).clamp_(min=0), entry < last


def _k_codes(case, bytes_):
    """[..., head, token, dim] of K codes as they lie in a chunk."""
    h, bt, d = case["kv_heads"], case["block"], case["dim"]
    lead = bytes_.shape[:-1]
    x = bytes_.reshape(*lead, h, bt // 16, d // 64, 16, 64).transpose(-3, -2)
    return x.reshape(*lead, h, bt, d)


def _k_bytes(case, codes):
    h, bt, d = case["kv_heads"], case["block"], case["dim"]
    lead = codes.shape[:-3]
    x = codes.reshape(*lead, h, bt // 16, 16, d // 64, 64).transpose(-3, -2)
    return x.reshape(*lead, h * bt * d)


def _v_codes(case, bytes_):
    """The same of V codes: 16 tokens by 64 dims lie as 4 groups of tokens,
    16 dims, 4 dims 16 apart, 4 tokens."""
    h, bt, d = case["kv_heads"], case["block"], case["dim"]
    lead = bytes_.shape[:-1]
    m = len(lead)
    x = bytes_.reshape(*lead, h, bt // 16, d // 64, 4, 16, 4, 4)
    at = tuple(range(m))
    x = x.permute(*at, m, m + 1, m + 3, m + 6, m + 2, m + 5, m + 4)
    return x.reshape(*lead, h, bt, d)


def _v_bytes(case, codes):
    h, bt, d = case["kv_heads"], case["block"], case["dim"]
    lead = codes.shape[:-3]
    m = len(lead)
    x = codes.reshape(*lead, h, bt // 16, 4, 4, d // 64, 4, 16)
    at = tuple(range(m))
    x = x.permute(*at, m, m + 1, m + 4, m + 2, m + 6, m + 5, m + 3)
    return x.reshape(*lead, h * bt * d)


def _split(case, chunks):
    """E4M3 codes (bytes) and scales [..., head] of chunks [..., bytes]."""
    codes, _ = _chunk_bytes(case)
    scale = chunks[..., codes:].contiguous().view(torch.float32)[..., :case["kv_heads"]]
    return chunks[..., :codes].contiguous(), scale


def _values(case, kv, chunks):
    """What chunks stand for: [..., head, token, dim] in 32 bits."""
    codes, scale = _split(case, chunks)
    codes = _v_codes(case, codes) if kv else _k_codes(case, codes)
    return codes.view(torch.float8_e4m3fn).float() * scale[..., None, None]


def _stored(case, s):
    """The pool as codes and scales, as views."""
    codes, _ = _chunk_bytes(case)
    return {"codes": s["pool"][..., :codes].view(torch.float8_e4m3fn),
            "scales": s["pool"][..., codes:codes + 4 * case["kv_heads"]].view(torch.float32)}


def _rotate(case, x, turns):
    """Rotary positions in 32 bits; `turns` [tokens, pairs]."""
    r = case["rotary"]
    a = turns * (2 * math.pi)
    c, d = torch.cos(a)[:, None], torch.sin(a)[:, None]
    x = x.float()
    if case["interleaved"]:
        u, v = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([u * c - v * d, v * c + u * d], -1).flatten(-2)
    else:
        u, v = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([u * c - v * d, v * c + u * d], -1)
    return torch.cat([y, x[..., r:]], -1)


def _append(case, s):
    # fractions of a turn, from whole numbers that wrap
    turns = ((s["positions"].long()[:, None] * s["freq"]) >> 40).float() * 2.0 ** -24
    q, k = _rotate(case, s["q"], turns), _rotate(case, s["k"], turns)
    s["out"].copy_(q)
    bt, n = case["block"], s["n"]
    count = s["offsets"][1:] - s["offsets"][:-1]
    first = (s["length"] - count).long()
    # each request's blocks that get tokens, [n, most]
    most = (s["most_new"] + bt - 2) // bt + 1
    block = first[:, None] // bt + torch.arange(most, device=DEV)
    has = block * bt < s["length"][:, None]
    entry = torch.where(has, s["rows"][:-1, None] + block, 0)
    slot = torch.where(has, s["slots"][entry], s["entries"]).long()
    # the new token of each of their places, and the places that hold older ones
    token = block[..., None] * bt + torch.arange(bt, device=DEV)
    fresh = (token >= first[:, None, None]) & (token < s["length"][:, None, None])
    held = (token < first[:, None, None])[:, :, None, :, None]
    row = torch.where(fresh, s["offsets"][:-1, None, None] + token - first[:, None, None], 0).long()
    fresh = fresh[:, :, None, :, None]
    for kv, x in ((0, k), (1, s["v"].float())):
        chunks = s["pool"][kv][slot]
        x = torch.where(fresh, x[row].transpose(2, 3), 0.0)
        m, e = torch.frexp(x.abs().amax((-2, -1)))
        scale = torch.exp2((e - 9 + (m > 0.875)).float()).clamp_(min=MIN_SCALE)
        codes, old = _split(case, chunks)
        scale = torch.where((first[:, None] > block * bt)[..., None], torch.maximum(old, scale), scale)
        codes = (_v_codes if kv else _k_codes)(case, codes).view(torch.float8_e4m3fn)
        older = (codes.float() * (old / scale)[..., None, None]).to(torch.float8_e4m3fn)
        both = torch.where(held, older.view(torch.uint8), codes.view(torch.uint8))
        fine = (x / scale[..., None, None]).to(torch.float8_e4m3fn)
        both = torch.where(fresh, fine.view(torch.uint8), both)
        size = codes.shape[-3] * bt * case["dim"]
        chunks[..., :size] = (_v_bytes if kv else _k_bytes)(case, both)
        chunks[..., size:size + 4 * case["kv_heads"]] = scale.contiguous().view(torch.uint8)
        s["pool"][kv].index_copy_(0, slot.flatten(), chunks.flatten(0, 1))
    return {"q": s["out"], **{k: v[:, :-1] for k, v in _stored(case, s).items()}}


def _attend(case, s):
    n, h, d, most = s["n"], case["kv_heads"], case["dim"], s["most_new"]
    group = case["heads"] // h
    entry, has = _padded_blocks(s)
    slot = s["slots"][entry].long()
    held = torch.arange(s["most_blocks"] * case["block"], device=DEV) < s["length"][:, None]

    def side(kv):
        x = _values(case, kv, s["pool"][kv][slot]).transpose(1, 2).flatten(2, 3)
        return torch.where(held[:, None, :, None], x, 0.0)

    k = side(0)
    count = s["offsets"][1:] - s["offsets"][:-1]
    t = torch.arange(most, device=DEV)
    live = t < count[:, None]
    row = torch.where(live, s["offsets"][:-1, None] + t, 0).long()
    q = s["q"].float()[row].reshape(n, most, h, group, d).permute(0, 2, 1, 3, 4).reshape(n, h, -1, d)
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"])
    del k
    if case["cap"]:
        x = x.div_(case["cap"]).tanh_().mul_(case["cap"])
    x = x.view(n, h, most, group, -1)
    last = (s["length"] - count)[:, None] + t
    seen = torch.arange(x.shape[-1], device=DEV) <= last[..., None]
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).flatten(2)
    x.div_(torch.where(total > 0, total, 1.0))
    o = torch.matmul(x.flatten(2, 3), side(1)).view(n, h, most, group, d)
    o = o.permute(0, 2, 1, 3, 4).flatten(2, 3)
    # rows of no token go to a row that is dropped
    tokens = s["out"].shape[0]
    to = torch.where(live, row, tokens).flatten()

    def packed(a):
        return a.new_empty(tokens + 1, *a.shape[2:]).index_copy_(0, to, a.flatten(0, 1))[:tokens]

    s["out"].copy_(packed(o))
    got = {"out": s["out"]}
    if s["lse"] is not None:
        s["lse"].copy_(packed(lse))
        got["lse"] = s["lse"]
    if s["weight"] is not None:
        late = live & (t >= (count - case["window"])[:, None])
        w = torch.where(late[:, None, :, None, None], x, 0.0).sum((1, 2, 3))
        w = w.view(n, -1, case["block"]).sum(-1)
        s["weight"].index_add_(0, entry.flatten(), torch.where(has, w, 0.0).flatten())
        got["weight"] = s["weight"]
    return got


def _evict(case, s):
    bt, n, most = case["block"], s["n"], s["most_blocks"]
    entry, has = _padded_blocks(s)
    blocks = (s["length"] + bt - 1) // bt
    b = torch.arange(most, device=DEV)
    free = (b >= case["sink"]) & (b < (blocks - case["recent"])[:, None])
    count = torch.minimum((blocks - s["keep"]).clamp(min=0), free.sum(1, dtype=torch.int32))
    w = torch.where(free, s["weight"][entry], math.inf)
    rank = torch.empty(n, most, dtype=torch.int64, device=DEV)
    rank.scatter_(1, torch.sort(w, dim=1, stable=True).indices, b.expand(n, most).contiguous())
    gone = free & (rank < count[:, None])
    stay = has & ~gone
    s["length_out"].copy_(s["length"] - count * bt)
    s["rows_out"][1:] = torch.cumsum(blocks - count, 0)
    end = s["entries"]

    def listed_in(mask, first, source, out):
        at = torch.where(mask, first[:, None] + torch.cumsum(mask, 1) - 1, end)
        wide = torch.zeros(end + 1, dtype=out.dtype, device=DEV)
        wide[at.flatten()] = source[entry].flatten()
        out.copy_(wide[:end])

    first = torch.cumsum(count, 0) - count
    listed_in(stay, s["rows_out"][:-1], s["slots"], s["slots_out"])
    listed_in(stay, s["rows_out"][:-1], s["weight"], s["weight_out"])
    listed_in(gone, first, s["slots"], s["freed"])
    s["n_freed"].copy_(count.sum().view(1))
    return _evicted(s)


def _evicted(s):
    return {k: s[k] for k in ("length_out", "rows_out", "slots_out", "weight_out", "freed", "n_freed")}


def run(state):
    s = state
    case = s["case"]
    if not own:
        return {"append": _append, "attend": _attend, "evict": _evict}[case["kind"]](case, s)
    s["op"].run()
    if case["kind"] == "append":
        return {"q": s["out"], **{k: v[:, :-1] for k, v in _stored(case, s).items()}}
    if case["kind"] == "evict":
        return _evicted(s)
    got = {"out": s["out"]}
    if s["lse"] is not None:
        got["lse"] = s["lse"]
    if s["weight"] is not None:
        got["weight"] = s["weight"]
    return got


# -------------------------------------------------------------------- work

def work(case):
    new, length = _lengths(case)
    if case["kind"] == "evict":
        # slot and weight of each block in, the same out
        return {"bytes": int(16 * (-(-length // case["block"])).sum() + 16 * case["n"]), "flops": 0}
    tokens, d, h, kv = int(new.sum()), case["dim"], case["heads"], case["kv_heads"]
    if case["kind"] == "append":
        # queries in and out, keys and values in at 16 bits and out at 8
        return {"bytes": tokens * d * (4 * h + 2 * kv * 3), "flops": 3 * tokens * case["rotary"] * (h + kv)}
    cached, blocks = int(length.sum()), int((-(-length // case["block"])).sum())
    pairs = int((new * length - new * (new - 1) // 2).sum())
    moved = 2 * cached * kv * d + 8 * blocks * kv + 4 * tokens * h * d
    moved += (4 * tokens * h if case["lse"] else 0) + (8 * blocks if case["window"] else 0)
    return {"bytes": moved, "flops": 4 * h * d * pairs}


# ------------------------------------------------------------------- exact

def _round_e4m3(x):
    """The nearest value of four significant bits, at least 2^-9 apart, ties
    to even."""
    step = torch.exp2((torch.frexp(x).exponent - 4).clamp_(min=-9).double())
    return torch.round(x / step) * step


def _exact_pool(s):
    """K and V as numbers [K and V][slot, head, token, dim] in 64 bits."""
    case = s["case"]
    return [_values(case, kv, s["pool"][kv]).double() for kv in range(2)]


def _exact_append(s):
    case, r = s["case"], s["case"]["rotary"]
    f = s["freq"].cpu().numpy().view(np.uint64)
    p = s["positions"].cpu().numpy().astype(np.uint64)
    with np.errstate(over="ignore"):
        turns = (p[:, None] * f[None]).view(np.int64).astype(np.float64) * 2.0 ** -64
    turns = torch.from_numpy(turns).to(DEV)
    unit = torch.polar(torch.ones_like(turns), 2 * math.pi * turns)[:, None]

    def turned(x):
        x = x.double()
        y = x.clone()
        i = slice(0, r, 2) if case["interleaved"] else slice(0, r // 2)
        j = slice(1, r, 2) if case["interleaved"] else slice(r // 2, r)
        z = torch.complex(x[..., i].contiguous(), x[..., j].contiguous()) * unit
        y[..., i], y[..., j] = z.real, z.imag
        return y

    codes, _ = _chunk_bytes(case)
    bt = case["block"]
    kept, scales = [], []
    off, length = s["offsets"].tolist(), s["length"].tolist()
    rows, slots = s["rows"].tolist(), s["slots"].tolist()
    for kv, x in ((0, turned(s["k"])), (1, s["v"].double())):
        raw, scale = _split(case, s["pool"][kv])
        code = (_v_codes if kv else _k_codes)(case, raw).view(torch.float8_e4m3fn).double()
        scale = scale.double().clone()
        for i in range(s["n"]):
            t, at = off[i], length[i] - (off[i + 1] - off[i])
            while at < length[i]:
                slot, o = slots[rows[i] + at // bt], at % bt
                m = min(bt - o, length[i] - at)
                y = x[t:t + m].transpose(0, 1)
                need = torch.exp2(torch.ceil(torch.log2(y.abs().amax((-2, -1)) / E4M3_MAX))).clamp_(min=MIN_SCALE)
                if o:
                    need = torch.maximum(need, scale[slot])
                    code[slot, :, :o] = _round_e4m3(code[slot, :, :o] * (scale[slot] / need)[:, None, None])
                code[slot, :, o:o + m] = _round_e4m3(y / need[:, None, None])
                scale[slot] = need
                t, at = t + m, at + m
        kept.append((_v_bytes if kv else _k_bytes)(case, code))
        scales.append(scale)
    return {"q": turned(s["q"]), "codes": torch.stack(kept)[:, :-1], "scales": torch.stack(scales)[:, :-1]}


def _exact_attend(s):
    case = s["case"]
    h, d, bt = case["kv_heads"], case["dim"], case["block"]
    group = case["heads"] // h
    off, length = s["offsets"].tolist(), s["length"].tolist()
    rows = s["rows"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    weight = s["weight"].double() if s["weight"] is not None else None
    for i in range(s["n"]):
        c, l = off[i + 1] - off[i], length[i]
        slot = s["slots"][rows[i]:rows[i + 1]].long()
        k, v = (_values(case, kv, s["pool"][kv][slot]).double().transpose(0, 1).reshape(h, -1, d)[:, :l]
                for kv in range(2))
        seen = (torch.arange(l, device=DEV) <= torch.arange(l - c, l, device=DEV)[:, None])
        for j in range(h):
            q = s["q"][off[i]:off[i + 1], j * group:(j + 1) * group].double().transpose(0, 1)
            x = torch.matmul(q, k[j].T) * s["scale"]
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            x = x.masked_fill(~seen, -math.inf)
            z = torch.logsumexp(x, -1)
            p = torch.exp(x - z[..., None])
            out[off[i]:off[i + 1], j * group:(j + 1) * group] = torch.matmul(p, v[j]).transpose(0, 1)
            lse[off[i]:off[i + 1], j * group:(j + 1) * group] = z.T
            if weight is not None:
                w = p[:, -min(case["window"], c):].sum((0, 1))
                w = torch.nn.functional.pad(w, (0, len(slot) * bt - l))
                weight[rows[i]:rows[i + 1]] += w.view(-1, bt).sum(-1)
    got = {"out": out}
    if s["lse"] is not None:
        got["lse"] = lse
    if weight is not None:
        got["weight"] = weight
    return got


def _exact_evict(s):
    case, bt = s["case"], s["case"]["block"]
    length, rows, keep = s["length"].tolist(), s["rows"].tolist(), s["keep"].tolist()
    slots, weight = s["slots"].cpu().numpy(), s["weight"].cpu().numpy().astype(np.float64)
    out = {k: np.zeros(s[k].shape, np.int64) for k in ("length_out", "rows_out", "slots_out", "freed", "n_freed")}
    out["weight_out"] = np.zeros(s["entries"])
    put = freed = 0
    for i in range(s["n"]):
        nb = -(-length[i] // bt)
        can = list(range(case["sink"], max(case["sink"], nb - case["recent"])))
        can.sort(key=lambda b: (weight[rows[i] + b], b))
        gone = sorted(can[:max(0, nb - keep[i])])
        stay = np.setdiff1d(np.arange(nb), gone)
        out["length_out"][i] = length[i] - bt * len(gone)
        out["slots_out"][put:put + len(stay)] = slots[rows[i] + stay]
        out["weight_out"][put:put + len(stay)] = weight[rows[i] + stay]
        put += len(stay)
        out["rows_out"][i + 1] = put
        for b in gone:
            out["freed"][freed] = slots[rows[i] + b]
            freed += 1
    out["n_freed"][0] = freed
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[case["kind"]](s)
