"""Cases of the operators that read less of the 8-bit paged KV pool.

``shared``: attention of a batch whose neighbouring requests share their first
blocks, which are read once for all of a group's rows.  ``bounds``: the largest
and least key of each block, per head and dim, as whole numbers in units of
four scales.  ``select``: for each new token and KV head the blocks whose
bounds promise the largest scores.  ``sparse``: attention over the selected
blocks.

The plain forms below are written from the formulas in elementary torch
operations over padded batches.  Head counts and sizes are those of the pool's
geometry (8 KV heads of 128, 16 tokens a block) and its shares under tensor
parallelism, with other common ones in the drawn cases; lengths follow the
chat and agentic prompt laws of ``synth``, families of parallel samples share
prefixes of 1 to 32 Ki tokens, chunks are of 512 tokens.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------- cases

def listed():
    llm = dict(heads=32, kv_heads=8, dim=128, block=16, dtype="bf16")
    big = dict(heads=64, kv_heads=8, dim=128, block=16, dtype="bf16")
    return [
        # four parallel samples of one prompt: the latency of a small batch
        dict(name="shared_family_4", kind="shared", groups=1, members=4, prefix=4096, least=1.0, new=1,
             law="chat", top=300, shape=1, cap=0.0, lse=False, **llm),
        # a decode batch of 32 families of four over prefixes of 1 to 32 Ki tokens
        dict(name="shared_families_128", kind="shared", groups=32, members=4, prefix=32768, least=0.03, new=1,
             law="chat", top=4096, shape=2, cap=0.0, lse=False, **big),
        # a decode batch behind one system prompt
        dict(name="shared_prompt_128", kind="shared", groups=1, members=128, prefix=8192, least=1.0, new=1,
             law="chat", top=2048, shape=3, cap=0.0, lse=True, **big),
        # drafts of one to eight tokens in groups of uneven size, some of one request; capped scores, float16
        dict(name="shared_drafts_48", kind="shared", groups=12, members=-8, prefix=12000, least=0.1, new=-8,
             law="chat", top=3000, shape=4, cap=30.0, lse=True, **dict(llm, block=32, dtype="f16")),
        # a decode batch's blocks after a token was written
        dict(name="bounds_128", kind="bounds", n=128, new=1, whole=False, law="chat", top=8192, shape=5, **big),
        # sixteen prefill chunks' blocks
        dict(name="bounds_chunks_8192", kind="bounds", n=16, new=512, whole=False, law="agent", top=8192,
             shape=6, **llm),
        # the next token of one request of 32 Ki tokens: the latency of a selection
        dict(name="select_1", kind="select", n=1, new=1, law="long", top=32768, keep=64, sink=1, recent=4,
             shape=7, **llm),
        # a decode batch of agentic requests, an eighth of 16 Ki tokens kept
        dict(name="select_128", kind="select", n=128, new=1, law="agent", top=32768, keep=128, sink=1,
             recent=8, shape=8, **big),
        # one prefill chunk late in a long prompt, float16
        dict(name="select_chunk_512", kind="select", n=1, new=512, law="long", top=32001, keep=64, sink=1,
             recent=4, shape=9, **dict(llm, dtype="f16")),
        # the next token of one request over 1 Ki tokens
        dict(name="sparse_1", kind="sparse", n=1, new=1, law="long", top=32768, keep=64, shape=10, cap=0.0,
             lse=False, **llm),
        # a decode batch over 2 Ki tokens each
        dict(name="sparse_128", kind="sparse", n=128, new=1, law="agent", top=32768, keep=128, shape=11,
             cap=0.0, lse=True, **big),
        # one prefill chunk, each token over its own 1 Ki tokens
        dict(name="sparse_chunk_512", kind="sparse", n=1, new=512, law="long", top=32001, keep=64, shape=12,
             cap=0.0, lse=False, **llm),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(8, 1, 128), (16, 2, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (16, 16, 64), (24, 8, 64),
         (16, 8, 256), (40, 8, 128)]


def draw(rng):
    kind = rng.choice(["shared", "shared", "bounds", "select", "sparse"])
    heads, kv_heads, dim = rng.choice(HEADS)
    block = rng.choice([16, 16, 32, 64, 128])
    case = dict(kind=kind, heads=heads, kv_heads=kv_heads, dim=dim, block=block,
                dtype=rng.choice(["bf16", "f16"]), shape=rng.randrange(100, 1 << 30))
    more = dict(cap=rng.choice([0.0, 0.0, 30.0]), lse=rng.random() < 0.5)
    law = rng.choice(["chat", "agent", "long"])
    if kind == "shared":
        n = _log(rng, 2, 128)
        groups = _log(rng, 1, n)
        return dict(case, groups=groups, members=rng.choice([1, -1]) * -(-n // groups),
                    prefix=_log(rng, 200, min(32768, 1200000 // n)), least=round(rng.uniform(0.02, 1.0), 3),
                    new=rng.choice([1, 1, -8, _log(rng, 2, 64) if n <= 16 else 1]), law="chat",
                    top=_log(rng, 64, 2048), **more)
    if kind == "bounds":
        new = rng.choice([1, -8, _log(rng, 2, 512)])
        return dict(case, n=_log(rng, 1, 128 if abs(new) <= 8 else 16), new=new, whole=rng.random() < 0.3,
                    law=law, top=_log(rng, 600, 8192))
    form = rng.choice(["decode", "decode", "draft", "chunk"])
    keep = _log(rng, 4, 2048 // block)
    case.update(new={"decode": 1, "draft": -8}.get(form) or _log(rng, 9, 512), law=law, keep=keep,
                n=_log(rng, 1, {"decode": 128, "draft": 16}.get(form, 1)))
    case.update(top=_log(rng, 256, min(65536, 600000 // case["n"])))
    if kind == "select":
        sink = rng.randrange(0, 3)
        return dict(case, sink=sink, recent=rng.randrange(1, keep - sink + 1) if keep - sink < 9 else
                    rng.randrange(1, 9))
    return dict(case, **more)


def _prompt(r, law, n, top):
    if law == "chat":
        x = np.exp(r.normal(6, 1, n))
    elif law == "agent":
        x = np.exp(r.normal(9, 0.7, n))
    else:
        x = top * r.uniform(0.75, 1.0, n)
    x = np.clip(np.rint(x).astype(np.int64), 1, top)
    x[0] = top  # one request reaches the top of the range
    return x


def _layout(case):
    """What is part of the case and the same for every seed: new and cached
    tokens (the new ones included) of each request, for each the first of its
    group and the tokens that it shares with it, and the table as numbers of
    blocks."""
    r = np.random.default_rng(case["shape"])
    bt = case["block"]
    if case["kind"] == "shared":
        g, m = case["groups"], case["members"]
        size = r.integers(1, -m + 1, g) if m < 0 else np.full(g, m)
        n = int(size.sum())
        prefix = case["prefix"] * np.exp(r.uniform(math.log(case["least"]), 0, g))
        prefix[0] = case["prefix"]
        prefix = np.maximum(1, np.rint(prefix / bt).astype(np.int64)) * bt
        leader = np.repeat(np.cumsum(size) - size, size)
        shared = np.repeat(prefix, size)
    else:
        n = case["n"]
        leader, shared = np.arange(n), np.zeros(n, np.int64)
    old = _prompt(r, case["law"], n, case["top"])
    new = case["new"]
    new = r.integers(1, -new + 1, n) if new < 0 else np.full(n, new, np.int64)
    length = shared + np.maximum(old, new)
    blocks = -(-length // bt)
    rows = np.concatenate([[0], np.cumsum(blocks)])
    ids = np.empty(int(rows[-1]), np.int64)
    made = 0
    for i in range(n):
        own_blocks = int(blocks[i])
        at = int(rows[i])
        held = int(shared[i] // bt) if leader[i] != i else 0
        ids[at:at + held] = ids[rows[leader[i]]:rows[leader[i]] + held]
        ids[at + held:at + own_blocks] = made + np.arange(own_blocks - held)
        made += own_blocks - held
    return dict(n=n, new=new, length=length, leader=leader, shared=shared, blocks=blocks, rows=rows, ids=ids,
                made=made)


# ----------------------------------------------------------------- prepare

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _ints(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int64)).to(device=DEV, dtype=dtype)


def _chunk_bytes(case):
    """The codes of a block's K or V over all heads, one scale a head, and the
    bounds of K: the largest keys in K's chunk, the least in V's."""
    codes = case["kv_heads"] * case["block"] * case["dim"]
    scales = -(-4 * case["kv_heads"] // 16) * 16
    return codes, scales, case["kv_heads"] * case["dim"]


def _pool(case, slots, g):
    """A pool of one layer, [K and V, slots, bytes], filled as earlier tokens
    leave it: codes up to the format's largest, scales of powers of two.  Keys
    have dims of unlike size, and neighbouring tokens have something in
    common."""
    codes, scales, bounds = _chunk_bytes(case)
    h, bt, d = case["kv_heads"], case["block"], case["dim"]
    pool = torch.zeros(2, slots, codes + scales + bounds, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 26) // codes)
    size = torch.exp2(torch.randn(h, 1, d, generator=g, device=DEV) * 0.7) * 40
    for kv in range(2):
        for a in range(0, slots, step):
            b = min(slots, a + step)
            x = torch.randn(b - a, h, bt, d, generator=g, device=DEV)
            if kv == 0:
                x = (x + torch.randn(b - a, h, 1, d, generator=g, device=DEV)).mul_(size)
            else:
                x = x.mul_(110)
            x = x.clamp_(-448, 448).to(torch.float8_e4m3fn)
            pool[kv, a:b, :codes] = (_v_bytes if kv else _k_bytes)(case, x.view(torch.uint8))
            if kv == 0 and case["kind"] == "select":
                x = x.float()
                pool[0, a:b, codes + scales:] = _whole(torch.ceil(x.amax(2) / 4))
                pool[1, a:b, codes + scales:] = _whole(torch.floor(x.amin(2) / 4))
    e = torch.randint(-8, -5, (2, slots, scales // 4), generator=g, device=DEV)
    pool[:, :, codes:codes + scales] = torch.exp2(e.float()).view(torch.uint8)
    return pool


def _whole(x):
    return x.to(torch.int8).flatten(1).view(torch.uint8)


def prepare(case, seed):
    g = _generator(seed)
    lay = _layout(case)
    n, bt = lay["n"], case["block"]
    h, heads, dim = case["kv_heads"], case["heads"], case["dim"]
    tokens = int(lay["new"].sum())
    # blocks lie anywhere in the pool; one slot is nobody's
    where = torch.randperm(lay["made"], generator=g, device=DEV).to(torch.int32)
    s = dict(case=case, n=n, tokens=tokens, entries=len(lay["ids"]), free=lay["made"], length=_ints(lay["length"]),
             rows=_ints(lay["rows"]), slots=where[_ints(lay["ids"], torch.int64)], leader=_ints(lay["leader"]),
             shared=_ints(lay["shared"]), most_blocks=int(lay["blocks"].max()), most_new=int(lay["new"].max()),
             offsets=_ints(np.concatenate([[0], np.cumsum(lay["new"])])))
    s["pool"] = _pool(case, lay["made"] + 1, g)
    s["most_shared"] = int(np.bincount(lay["leader"], lay["new"]).max())
    if case["kind"] == "bounds":
        s["upper"], s["lower"] = _bounds_view(case, s)
    else:
        # queries of the new tokens beside their keys and values, as a fused
        # projection leaves them
        x = torch.randn(tokens, heads + 2 * h, dim, generator=g, device=DEV)
        x *= torch.exp2(torch.randn(heads + 2 * h, 1, generator=g, device=DEV) * 0.5)
        s["q"] = x.to(TYPES[case["dtype"]])[:, :heads]
    if case["kind"] in ("shared", "sparse"):
        s["scale"] = dim ** -0.5
        s["out"] = torch.zeros(tokens, heads, dim, dtype=TYPES[case["dtype"]], device=DEV)
        s["lse"] = torch.zeros(tokens, heads, device=DEV) if case["lse"] else None
    if case["kind"] == "select":
        s["selected"] = torch.zeros(tokens, h, case["keep"], dtype=torch.int32, device=DEV)
    if case["kind"] == "sparse":
        s["selected"] = _selection(case, s, g)
    if own:
        from paper_2608_06557_amd import device
        kv = device.DeviceKvPool(s["pool"][None], h, dim, bt, bounds=True)
        batch = device.KvBatch(s["offsets"], s["length"], s["rows"], s["slots"], tokens, s["most_new"])
        if case["kind"] == "shared":
            s["op"] = device.DeviceSharedAttention(kv, batch, s["leader"], s["shared"], s["most_shared"], s["q"],
                                                   s["out"], s["scale"], softcap=case["cap"], lse=s["lse"])
        elif case["kind"] == "bounds":
            s["op"] = device.DeviceKvBounds(kv, batch, whole=case["whole"])
        elif case["kind"] == "select":
            s["op"] = device.DeviceKvSelect(kv, batch, s["q"], s["selected"], sink=case["sink"],
                                            recent=case["recent"])
        else:
            s["op"] = device.DeviceSelectedAttention(kv, batch, s["q"], s["selected"], s["out"], s["scale"],
                                                     softcap=case["cap"], lse=s["lse"])
    return s


def _rows(s):
    """[n, most new]: each request's rows, and whether it has them."""
    count = s["offsets"][1:] - s["offsets"][:-1]
    t = torch.arange(s["most_new"], device=DEV)
    live = t < count[:, None]
    return torch.where(live, s["offsets"][:-1, None] + t, 0).long(), live, count


def _token_requests(s):
    """Of each row its request, and the last cached token that it sees."""
    count = s["offsets"][1:] - s["offsets"][:-1]
    i = torch.repeat_interleave(torch.arange(s["n"], device=DEV), count, output_size=s["tokens"])
    last = s["length"][i] - s["offsets"][1:][i] + torch.arange(s["tokens"], device=DEV)
    return i, last


def _selection(case, s, g):
    """Blocks as a selection leaves them: the first, the newest two, and others
    on which neighbouring tokens mostly agree."""
    i, last = _token_requests(s)
    b = torch.arange(s["most_blocks"], device=DEV)
    x = torch.rand(s["n"], case["kv_heads"], s["most_blocks"], generator=g, device=DEV)[i]
    x += torch.rand(x.shape, generator=g, device=DEV).mul_(0.5)
    own_block = (last // case["block"])[:, None, None]
    x = torch.where((b == 0) | (b > own_block - 2), 3.0, x)
    x = torch.where(b > own_block, -1.0, x)
    keep = min(case["keep"], s["most_blocks"])
    top, at = torch.topk(x, keep, dim=-1)
    at = torch.sort(torch.where(top >= 0, at, 1 << 30), -1).values
    out = torch.full((s["tokens"], case["kv_heads"], case["keep"]), -1, dtype=torch.int32, device=DEV)
    out[..., :keep] = torch.where(at < 1 << 30, at, -1)
    return out


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


def _scales(case, chunks):
    codes, _, _ = _chunk_bytes(case)
    return chunks[..., codes:codes + 4 * case["kv_heads"]].contiguous().view(torch.float32)


def _values(case, kv, chunks):
    """What chunks stand for: [..., head, token, dim] in 32 bits."""
    codes, _, _ = _chunk_bytes(case)
    x = (_v_codes if kv else _k_codes)(case, chunks[..., :codes].contiguous())
    return x.view(torch.float8_e4m3fn).float() * _scales(case, chunks)[..., None, None]


def _bounds_view(case, s):
    """The bounds of all blocks but nobody's: [K: largest, V: least, slots, head * dim]."""
    codes, scales, bounds = _chunk_bytes(case)
    return s["pool"][:, :-1, codes + scales:codes + scales + bounds].view(torch.int8)


def _weighted(x, v):
    """Softmax over the last dimension of scores that may be -inf, the values'
    average by it and the log sum."""
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    return torch.matmul(x, v).div_(torch.where(total > 0, total, 1.0)), lse


def _capped(case, x):
    return x.div_(case["cap"]).tanh_().mul_(case["cap"]) if case["cap"] else x


def _shared(case, s):
    n, h, d, most = s["n"], case["kv_heads"], case["dim"], s["most_new"]
    group = case["heads"] // h
    slot = s["slots"][_padded_blocks(s)[0]].long()
    held = torch.arange(s["most_blocks"] * case["block"], device=DEV) < s["length"][:, None]

    def side(kv):
        x = _values(case, kv, s["pool"][kv][slot]).transpose(1, 2).flatten(2, 3)
        return torch.where(held[:, None, :, None], x, 0.0)

    row, live, count = _rows(s)
    q = s["q"].float()[row].reshape(n, most, h, group, d).permute(0, 2, 1, 3, 4).reshape(n, h, -1, d)
    x = _capped(case, torch.matmul(q, side(0).transpose(-1, -2)).mul_(s["scale"]))
    x = x.view(n, h, most, group, -1)
    last = (s["length"] - count)[:, None] + torch.arange(most, device=DEV)
    seen = torch.arange(x.shape[-1], device=DEV) <= last[..., None]
    x = x.masked_fill_(~seen[:, None, :, None], -math.inf).flatten(2, 3)
    o, lse = _weighted(x, side(1))
    o = o.view(n, h, most, group, d).permute(0, 2, 1, 3, 4).flatten(2, 3)
    lse = lse.view(n, h, most, group).permute(0, 2, 1, 3).flatten(2)
    # rows of no token go to a row that is dropped
    to = torch.where(live, row, s["tokens"]).flatten()

    def packed(a):
        return a.new_empty(s["tokens"] + 1, *a.shape[2:]).index_copy_(0, to, a.flatten(0, 1))[:s["tokens"]]

    s["out"].copy_(packed(o))
    if s["lse"] is not None:
        s["lse"].copy_(packed(lse))
    return _attended(s)


def _attended(s):
    return {"out": s["out"]} if s["lse"] is None else {"out": s["out"], "lse": s["lse"]}


def _bounds(case, s):
    bt = case["block"]
    count = s["offsets"][1:] - s["offsets"][:-1]
    first = torch.zeros_like(s["length"]) if case["whole"] else (s["length"] - count) // bt
    most = s["most_blocks"] if case["whole"] else (s["most_new"] + bt - 2) // bt + 1
    block = first[:, None] + torch.arange(most, device=DEV)
    has = (block * bt < s["length"][:, None]) & ((count[:, None] > 0) | case["whole"])
    entry = torch.where(has, s["rows"][:-1, None] + block, 0)
    slot = torch.where(has, s["slots"][entry], s["free"]).long()
    codes, scales, size = _chunk_bytes(case)
    x = _k_codes(case, s["pool"][0][slot][..., :codes].contiguous()).view(torch.float8_e4m3fn).float()
    live = (block[..., None] * bt + torch.arange(bt, device=DEV) < s["length"][:, None, None])[:, :, None, :, None]
    upper = torch.ceil(torch.where(live, x, -math.inf).amax(-2).mul_(0.25))
    lower = torch.floor(torch.where(live, x, math.inf).amin(-2).mul_(0.25))
    at = slice(codes + scales, codes + scales + size)
    for kv, y in ((0, upper), (1, lower)):
        y = torch.where(has[..., None, None], y, 0.0).to(torch.int8)
        s["pool"][kv, :, at].index_copy_(0, slot.flatten(), y.view(torch.uint8).flatten(2).flatten(0, 1))
    return {"upper": s["upper"], "lower": s["lower"]}


def _select(case, s):
    n, h, d, most, bt = s["n"], case["kv_heads"], case["dim"], s["most_new"], case["block"]
    group, keep = case["heads"] // h, case["keep"]
    slot = s["slots"][_padded_blocks(s)[0]].long()
    codes, scales, size = _chunk_bytes(case)
    both = s["pool"][:, :, codes + scales:codes + scales + size].view(torch.int8)
    # [n, h, blocks, 2 dims]
    bound = torch.cat([both[kv][slot].view(n, -1, h, d) for kv in (0, 1)], -1).float().transpose(1, 2)
    # queries in whole numbers of a power of two, up to 127
    x = s["q"].float()
    m, e = torch.frexp(x.abs().amax(-1))
    e = (e - 7 + (m > 127 / 128)).clamp_(min=-100)
    x = torch.round(torch.ldexp(x, -e[..., None]))
    top = e.view(-1, h, group).amax(-1, keepdim=True)
    weight = torch.exp2((e.view(-1, h, group) - top).clamp_(min=-126).float())
    row, live, count = _rows(s)
    x = torch.cat([x.clamp(min=0), x.clamp(max=0)], -1)[row]  # [n, most, heads, 2 dims]
    x = x.reshape(n, most, h, group, 2 * d).permute(0, 2, 1, 3, 4).reshape(n, h, -1, 2 * d)
    # whole numbers under 2^24: exact
    score = torch.matmul(x, bound.transpose(-1, -2)).view(n, h, most, group, -1)
    score = score.mul_(weight[row].transpose(1, 2)[..., None]).amax(3)
    scale = _scales(case, s["pool"][0][:, :codes + scales])[slot].transpose(1, 2)  # [n, h, blocks]
    score = score.mul_(scale[:, :, None])
    own_block = (((s["length"] - count)[:, None] + torch.arange(most, device=DEV)) // bt)[:, None, :, None]
    b = torch.arange(score.shape[-1], device=DEV)
    score = torch.where((b < case["sink"]) | (b > own_block - case["recent"]), math.inf, score)
    score = torch.where(b > own_block, -math.inf, score)
    at = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :keep]
    at = torch.where(at > own_block, 1 << 30, at)
    at = torch.sort(at, -1).values
    got = torch.full((n, h, most, keep), -1, dtype=torch.int32, device=DEV)
    got[..., :at.shape[-1]] = torch.where(at < 1 << 30, at, -1)
    to = torch.where(live, row, s["tokens"]).flatten()
    wide = got.new_empty(s["tokens"] + 1, h, keep)
    s["selected"].copy_(wide.index_copy_(0, to, got.transpose(1, 2).flatten(0, 1))[:s["tokens"]])
    return {"selected": s["selected"]}


def _sparse(case, s):
    h, d, bt, t = case["kv_heads"], case["dim"], case["block"], s["tokens"]
    i, last = _token_requests(s)
    listed_ = s["selected"] >= 0
    block = torch.where(listed_, s["selected"], 0)
    slot = s["slots"][s["rows"][:-1][i][:, None, None] + block].long()  # [tokens, h, keep]
    head = torch.arange(h, device=DEV)[:, None]
    codes, _, _ = _chunk_bytes(case)
    seen = block[..., None] * bt + torch.arange(bt, device=DEV) <= last[:, None, None, None]
    seen = (seen & listed_[..., None]).flatten(2)[:, :, None]  # [tokens, h, 1, keep * bt]

    def side(kv):
        x = s["pool"][kv]
        size = bt * d
        # [slots, h, bytes of a head's codes] -> [tokens, h, keep, bytes]
        x = x[:, :codes].unflatten(1, (h, size))[slot, head]
        one = dict(case, kv_heads=1)
        x = (_v_codes if kv else _k_codes)(one, x).view(torch.float8_e4m3fn).float()
        x = x.squeeze(-3) * _scales(case, s["pool"][kv])[slot, head][..., None, None]
        return torch.where(seen.transpose(-1, -2), x.flatten(2, 3), 0.0)

    q = s["q"].float().reshape(t, h, -1, d)
    x = _capped(case, torch.matmul(q, side(0).transpose(-1, -2)).mul_(s["scale"]))
    o, lse = _weighted(x.masked_fill_(~seen, -math.inf), side(1))
    s["out"].copy_(o.flatten(1, 2))
    if s["lse"] is not None:
        s["lse"].copy_(lse.flatten(1))
    return _attended(s)


def run(state):
    s = state
    case = s["case"]
    if not own:
        return {"shared": _shared, "bounds": _bounds, "select": _select, "sparse": _sparse}[case["kind"]](case, s)
    s["op"].run()
    if case["kind"] == "bounds":
        return {"upper": s["upper"], "lower": s["lower"]}
    if case["kind"] == "select":
        return {"selected": s["selected"]}
    return _attended(s)


# -------------------------------------------------------------------- work

def work(case):
    lay = _layout(case)
    new, length, bt = lay["new"], lay["length"], case["block"]
    tokens, d, h, kv = int(new.sum()), case["dim"], case["heads"], case["kv_heads"]
    if case["kind"] == "bounds":
        first = np.zeros_like(length) if case["whole"] else (length - new) // bt * bt
        blocks = int((-(-length // bt) - first // bt).sum())
        # codes in, two bounds of 8 bits out
        return {"bytes": kv * d * (int((length - first).sum()) + 2 * blocks), "flops": 0}
    if case["kind"] == "select":
        blocks = lay["blocks"]
        pairs = sum(int(((np.arange(l - c, l)) // bt + 1).sum()) for c, l in zip(new, length))
        return {"bytes": int(blocks.sum()) * kv * (2 * d + 4) + 2 * tokens * h * d + 4 * tokens * kv * case["keep"],
                "flops": 4 * h * d * pairs}
    rows = 4 * tokens * h * d + (4 * tokens * h if case["lse"] else 0)
    if case["kind"] == "shared":
        # shared tokens once for the first of a group
        first = lay["leader"] == np.arange(lay["n"])
        cached = int(np.where(first, length, length - lay["shared"]).sum())
        pairs = int((new * length - new * (new - 1) // 2).sum())
        return {"bytes": 2 * cached * kv * d + 8 * lay["made"] * kv + rows, "flops": 4 * h * d * pairs}
    keep = case["keep"] * bt
    pairs = sum(int(np.minimum(np.arange(l - c, l) + 1, keep).sum()) for c, l in zip(new, length))
    cached = int(np.minimum(length, new * keep).sum())
    return {"bytes": 2 * cached * kv * d + 8 * (cached // bt) * kv + 4 * tokens * kv * case["keep"] + rows,
            "flops": 4 * h * d * pairs}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    """Attention in 64 bits, request by request over all of its cached tokens,
    those that a row does not see or did not select masked.  Bounds and
    selections are whole numbers."""
    global own
    if case["kind"] in ("bounds", "select"):
        return None
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    h, d, bt = case["kv_heads"], case["dim"], case["block"]
    group = case["heads"] // h
    off, length, rows = s["offsets"].tolist(), s["length"].tolist(), s["rows"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for i in range(s["n"]):
        c, l, blocks = off[i + 1] - off[i], length[i], rows[i + 1] - rows[i]
        slot = s["slots"][rows[i]:rows[i + 1]].long()
        k, v = (_values(case, kv, s["pool"][kv][slot]).double().transpose(0, 1).reshape(h, -1, d)[:, :l]
                for kv in range(2))
        seen = torch.arange(l, device=DEV) <= torch.arange(l - c, l, device=DEV)[:, None]
        for j in range(h):
            mask = seen
            if case["kind"] == "sparse":
                at = s["selected"][off[i]:off[i + 1], j].long()
                chosen = torch.zeros(c, blocks + 1, dtype=torch.bool, device=DEV)
                chosen.scatter_(1, torch.where(at < 0, blocks, at), True)
                mask = seen & chosen[:, :blocks].repeat_interleave(bt, 1)[:, :l]
            q = s["q"][off[i]:off[i + 1], j * group:(j + 1) * group].double().transpose(0, 1)
            x = torch.matmul(q, k[j].T) * s["scale"]
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            x = x.masked_fill(~mask, -math.inf)
            z = torch.logsumexp(x, -1)
            p = torch.exp(x - z[..., None])
            out[off[i]:off[i + 1], j * group:(j + 1) * group] = torch.matmul(p, v[j]).transpose(0, 1)
            lse[off[i]:off[i + 1], j * group:(j + 1) * group] = z.T
    return {"out": out} if s["lse"] is None else {"out": out, "lse": lse}
