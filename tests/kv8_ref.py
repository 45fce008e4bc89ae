"""Test-only reference of the 8-bit KV cache's operators, in 64 bits on the
CPU, straight from the formulas in include/cascade.h."""
from __future__ import annotations

import numpy as np
import torch

E4M3 = torch.float8_e4m3fn
F64 = torch.float64


# ------------------------------------------------------------------ layout

def chunk_bytes(h, d, bt):
    return h * bt * d + -(-4 * h // 16) * 16


def code_offsets(h, d, bt, side):
    """Byte of each code in a chunk, [head, token, dim]."""
    hh, tt, dd = np.meshgrid(np.arange(h), np.arange(bt), np.arange(d), indexing="ij")
    t, sub = tt % 16, (hh * bt + tt // 16 * 16) * d
    if side == 0:
        at = ((dd // 64) * 16 + t) * 64 + dd % 64
    else:
        at = (((dd // 64) * 4 + t // 4) * 16 + dd % 16) * 16 + (dd % 64) // 16 * 4 + t % 4
    return torch.from_numpy(sub + at)


def codes_of(chunks, h, d, bt, side):
    """E4M3 codes (bytes) [..., head, token, dim] of chunks [..., bytes]."""
    return chunks[..., code_offsets(h, d, bt, side)]


def scales_of(chunks, h, d, bt):
    n = h * bt * d
    return chunks[..., n:n + 4 * h].contiguous().view(torch.float32)


def values_of(chunks, h, d, bt, side):
    x = codes_of(chunks, h, d, bt, side).view(E4M3).to(torch.float32).to(F64)
    return x * scales_of(chunks, h, d, bt).to(F64)[..., None, None]


def store(chunks, codes, scales, h, d, bt, side):
    """Write codes (bytes [slot, head, token, dim]) and scales into chunks."""
    chunks[:, code_offsets(h, d, bt, side).flatten()] = codes.flatten(1)
    n = h * bt * d
    chunks[:, n:n + 4 * h] = scales.to(torch.float32).contiguous().view(torch.uint8)


def random_pool(rng, layers, slots, h, d, bt, pad=0, spread=2, stale_nan=False):
    """Pool bytes [layers, 2, slots, chunk + pad] of random codes and scales."""
    pool = torch.zeros(layers, 2, slots, chunk_bytes(h, d, bt) + pad, dtype=torch.uint8)
    for layer in range(layers):
        for side in range(2):
            x = torch.from_numpy(rng.normal(0, 100, (slots, h, bt, d))).clamp(-448, 448)
            codes = x.float().to(E4M3).view(torch.uint8)
            e = rng.integers(-7 - spread, -6 + spread, (slots, h))
            view = pool[layer, side]
            store(view, codes, torch.from_numpy(2.0 ** e), h, d, bt, side)
    return pool


# -------------------------------------------------------------------- rope

def theta(kind, R, base, factor=1.0, length=0.0, low=1.0, high=4.0):
    """Radians a position of each pair and the rotation's scale."""
    j = np.arange(R // 2, dtype=np.float64)
    if kind == "base":
        return (base * factor ** (R / (R - 2))) ** (-2 * j / R), 1.0
    t = base ** (-2 * j / R)
    if kind == "plain":
        return t, 1.0
    if kind == "linear":
        return t / factor, 1.0
    if kind == "bands":
        wave = 2 * np.pi / t
        s = (length / wave - low) / (high - low)
        mid = (1 - s) * t / factor + s * t
        return np.where(wave > length / low, t / factor, np.where(wave < length / high, t, mid)), 1.0
    turn = lambda b: R * np.log(length / (2 * np.pi * b)) / (2 * np.log(base))
    a, b = max(np.floor(turn(high)), 0), min(np.ceil(turn(low)), R - 1)
    if b <= a:
        b = a + 0.001
    s = 1 - np.clip((j - a) / (b - a), 0, 1)
    return (1 - s) * t / factor + s * t, 0.1 * np.log(factor) + 1


def fixed(radians):
    return np.floor(np.asarray(radians) / (2 * np.pi) * 2.0 ** 64).astype(np.uint64)


def rotate(x, positions, freq, interleaved, scale=1.0):
    """x [tokens, heads, dims] in 64 bits; freq uint64[R / 2]."""
    x = x.to(F64).clone()
    R = 2 * len(freq)
    if R == 0:
        return x
    with np.errstate(over="ignore"):
        f = np.asarray(positions).astype(np.uint64)[:, None] * np.asarray(freq, np.uint64)[None]
    a = torch.from_numpy(f.view(np.int64).astype(np.float64) * 2.0 ** -64 * 2 * np.pi)[:, None]
    c, s = torch.cos(a) * scale, torch.sin(a) * scale
    i, j = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    u, v = x[..., i].clone(), x[..., j].clone()
    x[..., i], x[..., j] = u * c - v * s, v * c + u * s
    return x


# ------------------------------------------------------------------ append

def scale_for(amax):
    """Smallest power of two with amax <= 448 scales, at least 2^-100."""
    a = np.asarray(amax, np.float64)
    m, e = np.frexp(a)  # a = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = np.where(a > 0, e - 9 + (m > 0.875), -100)
    return 2.0 ** np.maximum(e, -100)


def round_e4m3(x):
    """Values of E4M3 nearest to x (64 bits), ties to even."""
    m, e = torch.frexp(x)
    step = torch.exp2(torch.clamp(e - 4, min=-9).to(F64))
    return torch.round(x / step) * step


def append(pool_side, x, b, h, d, bt, side):
    """The pool's chunks [slots, bytes] of one side after x [tokens, h, d]
    (64 bits): code values [slots, h, bt, d] and scales [slots, h], and where
    a new element went."""
    val = codes_of(pool_side, h, d, bt, side).view(E4M3).float().to(F64)
    sc = scales_of(pool_side, h, d, bt).to(F64).clone()
    fresh = torch.zeros(val.shape, dtype=torch.bool)
    want = torch.zeros_like(val)
    for i in range(b["n"]):
        first, count = int(b["off"][i]), int(b["off"][i + 1] - b["off"][i])
        length, row = int(b["len"][i]), int(b["rows"][i])
        t = 0
        while t < count:
            at = length - count + t
            slot, o = int(b["slots"][row + at // bt]), at % bt
            m = min(bt - o, count - t)
            y = x[first + t:first + t + m].transpose(0, 1)  # [h, m, d]
            s = torch.from_numpy(scale_for(y.abs().amax((1, 2)).numpy()))
            if o:
                s = torch.maximum(s, sc[slot])
                grown = s > sc[slot]
                old = round_e4m3(val[slot, :, :o] * (sc[slot] / s)[:, None, None])
                val[slot, :, :o] = torch.where(grown[:, None, None], old, val[slot, :, :o])
            sc[slot] = s
            want[slot, :, o:o + m] = y / s[:, None, None]
            val[slot, :, o:o + m] = round_e4m3(want[slot, :, o:o + m])
            fresh[slot, :, o:o + m] = True
            t += m
    return val, sc, fresh, want


# --------------------------------------------------------------- attention

def attend(pool_layer, q, b, h, d, bt, scale, cap=0.0, window=0, kinds=None):
    """out, lse [tokens, heads], weight [entries] in 64 bits, and the sums of
    |v| weights that bound the rounding: dict."""
    T, H = q.shape[:2]
    G = H // h
    out = torch.zeros(T, H, d, dtype=F64)
    mass = torch.zeros(T, H, d, dtype=F64)      # sum of p |v|
    reach = torch.zeros(T, H, d, dtype=F64)     # sum of |v|
    lse = torch.full((T, H), -np.inf, dtype=F64)
    err = torch.zeros(T, H, dtype=F64)          # largest sum of |q k| of a row
    w = torch.zeros(len(b["slots"]), dtype=F64)
    k_all, v_all = (values_of(pool_layer[s], h, d, bt, s) for s in range(2))
    for i in range(b["n"]):
        first, count = int(b["off"][i]), int(b["off"][i + 1] - b["off"][i])
        length, row = int(b["len"][i]), int(b["rows"][i])
        if count == 0:
            continue
        nb = -(-length // bt)
        sl = b["slots"][row:row + nb].long()
        k = k_all[sl].transpose(0, 1).reshape(h, nb * bt, d)[:, :length]
        v = v_all[sl].transpose(0, 1).reshape(h, nb * bt, d)[:, :length]
        wt = torch.zeros(nb * bt, dtype=F64)
        for t in range(count):
            n = length - count + t + 1
            if n <= 0:
                continue
            for hh in range(H):
                x = q[first + t, hh].to(F64)
                kk, vv = k[hh // G, :n], v[hh // G, :n]
                s = kk @ x * scale
                err[first + t, hh] = (kk.abs() @ x.abs()).max() * abs(scale)
                if cap:
                    s = cap * torch.tanh(s / cap)
                z = torch.logsumexp(s, 0)
                p = torch.exp(s - z)
                out[first + t, hh] = p @ vv
                mass[first + t, hh] = p @ vv.abs()
                reach[first + t, hh] = vv.abs().sum(0)
                lse[first + t, hh] = z
                if t >= count - window:
                    wt[:n] += p
        w[row:row + nb] += wt.view(nb, bt).sum(1)
    return dict(out=out, lse=lse, weight=w, mass=mass, reach=reach, err=err)


# ------------------------------------------------------------------- evict

def evict(b, weight, keep, sink, recent, bt):
    n = b["n"]
    length, rows, slots, ws, freed = [], [0], [], [], []
    for i in range(n):
        l, row = int(b["len"][i]), int(b["rows"][i])
        nb = -(-l // bt)
        can = range(min(sink, nb), max(min(sink, nb), nb - recent))
        key = lambda j: (np.isnan(weight[row + j]), weight[row + j], j)
        gone = set(sorted(can, key=key)[:max(0, nb - int(keep[i]))])
        length.append(l - bt * len(gone))
        for j in range(nb):
            if j in gone:
                freed.append(int(b["slots"][row + j]))
            else:
                slots.append(int(b["slots"][row + j]))
                ws.append(weight[row + j])
        rows.append(len(slots))
    return length, rows, slots, ws, freed


# ------------------------------------------------------------------ inputs

def batch(rng, counts, lengths, bt, slack=0, spare=3):
    """A batch over shuffled distinct slots; every row has `slack` entries too
    many."""
    counts, lengths = np.asarray(counts), np.asarray(lengths)
    blocks = -(-lengths // bt) + slack
    rows = np.concatenate([[0], np.cumsum(blocks)]).astype(np.int32)
    pool = int(rows[-1]) + spare
    slots = rng.permutation(pool)[:rows[-1]].astype(np.int32)
    if slack:  # entries past a request's blocks name no slot
        for i in range(len(counts)):
            slots[rows[i + 1] - slack:rows[i + 1]] = -7
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32))
    return dict(n=len(counts), off=t(off), len=t(lengths), rows=t(rows), slots=t(slots), pool=pool,
                tokens=int(off[-1]), most=int(counts.max()) if len(counts) else 0)
