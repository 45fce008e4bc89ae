"""Test-only reference of the operators over bounds and selected blocks, in 64
bits on the CPU, straight from the formulas in include/cascade.h."""
from __future__ import annotations

import numpy as np
import torch

from tests import kv8_ref as ref


def bounds_of(pool_layer, b, h, d, bt, whole):
    """{slot: (upper, lower) int64 [h, d]} of the blocks that a call writes."""
    code = ref.codes_of(pool_layer[0], h, d, bt, 0).view(ref.E4M3).float().to(ref.F64).numpy()
    got = {}
    for i in range(b["n"]):
        length, row = int(b["len"][i]), int(b["rows"][i])
        first = 0 if whole else max(0, length - int(b["off"][i + 1] - b["off"][i])) // bt
        if not whole and b["off"][i + 1] == b["off"][i]:
            continue
        for k in range(first, -(-length // bt)):
            slot = int(b["slots"][row + k])
            x = code[slot][:, :min(bt, length - k * bt)]
            got[slot] = (np.ceil(x.max(1) / 4).astype(np.int64), np.floor(x.min(1) / 4).astype(np.int64))
    return got


def bounds_in(pool_layer, h, d, bt):
    """(upper, lower) int64 [slots, h, d] as they lie in the chunks."""
    n = ref.chunk_bytes(h, d, bt)
    return tuple(pool_layer[s][:, n:n + h * d].contiguous().view(torch.int8).numpy().astype(np.int64)
                 .reshape(-1, h, d) for s in range(2))


def whole_queries(q):
    """Whole numbers [tokens, heads, d] and exponents [tokens, heads]."""
    x = np.nan_to_num(q.to(ref.F64).numpy(), nan=0.0, posinf=0.0, neginf=0.0)
    most = np.abs(x).max(-1)
    e = np.full(most.shape, -100, np.int64)
    some = most > 0
    e[some] = np.maximum(np.ceil(np.log2(most[some] / 127)), -100).astype(np.int64)
    # the logarithm may be off by one at a power of two
    e = np.where(most > 127 * 2.0 ** e, e + 1, e)
    e = np.where((most <= 127 * 2.0 ** (e - 1)) & (e > -100), e - 1, e)
    return np.rint(x / 2.0 ** e[..., None]).astype(np.int64), e


def select(pool_layer, q, b, h, d, bt, keep, sink, recent):
    """[tokens, h, keep]; tokens of no request are -7."""
    T, H = q.shape[:2]
    G = H // h
    n, e = whole_queries(q)
    upper, lower = bounds_in(pool_layer, h, d, bt)
    scale = ref.scales_of(pool_layer[0], h, d, bt).to(ref.F64).numpy()
    out = np.full((T, h, keep), -7, np.int64)
    for i in range(b["n"]):
        first, count = int(b["off"][i]), int(b["off"][i + 1] - b["off"][i])
        length, row = int(b["len"][i]), int(b["rows"][i])
        for j in range(count):
            last = length - count + j
            blocks = 0 if last < 0 else last // bt + 1
            slots = b["slots"][row:row + blocks].numpy()
            for k in range(h):
                if blocks <= keep:
                    out[first + j, k] = list(range(blocks)) + [-1] * (keep - blocks)
                    continue
                best = np.full(blocks, -np.inf)
                top = e[first + j, k * G:(k + 1) * G].max()
                for g in range(k * G, (k + 1) * G):
                    x = n[first + j, g]
                    s = upper[slots, k] @ np.maximum(x, 0) + lower[slots, k] @ np.minimum(x, 0)
                    best = np.maximum(best, s * 2.0 ** max(e[first + j, g] - top, -126))
                best = best * scale[slots, k]
                forced = set(range(sink)) | set(range(blocks - recent, blocks))
                others = [t for t in range(blocks) if t not in forced]
                others.sort(key=lambda t: (-best[t], t))
                out[first + j, k] = sorted(forced | set(others[:keep - len(forced)]))
    return torch.from_numpy(out).to(torch.int32)


def attend(pool_layer, q, b, selected, h, d, bt, scale, cap=0.0):
    """As ref.attend over the listed blocks."""
    T, H = q.shape[:2]
    G = H // h
    out, mass, reach = (torch.zeros(T, H, d, dtype=ref.F64) for _ in range(3))
    lse, err = torch.full((T, H), -np.inf, dtype=ref.F64), torch.zeros(T, H, dtype=ref.F64)
    k_all, v_all = (ref.values_of(pool_layer[s], h, d, bt, s) for s in range(2))
    for i in range(b["n"]):
        first, count = int(b["off"][i]), int(b["off"][i + 1] - b["off"][i])
        length, row = int(b["len"][i]), int(b["rows"][i])
        for j in range(count):
            last = length - count + j
            for k in range(h):
                blocks = [int(x) for x in selected[first + j, k] if x >= 0]
                at = [(int(b["slots"][row + x]), t) for x in blocks for t in range(bt) if x * bt + t <= last]
                if not at:
                    continue
                sl, tk = (torch.tensor(z) for z in zip(*at))
                kk, vv = k_all[sl, k, tk], v_all[sl, k, tk]
                for g in range(k * G, (k + 1) * G):
                    x = q[first + j, g].to(ref.F64)
                    s = kk @ x * scale
                    err[first + j, g] = (kk.abs() @ x.abs()).max() * abs(scale)
                    if cap:
                        s = cap * torch.tanh(s / cap)
                    z = torch.logsumexp(s, 0)
                    p = torch.exp(s - z)
                    out[first + j, g], mass[first + j, g] = p @ vv, p @ vv.abs()
                    reach[first + j, g], lse[first + j, g] = vv.abs().sum(0), z
    return dict(out=out, lse=lse, mass=mass, reach=reach, err=err)


def random_bounds(rng, pool_layer, h, d, bt, few=False):
    """Bounds of any values; `few`: of few different ones, so that scores tie."""
    n, slots = ref.chunk_bytes(h, d, bt), pool_layer.shape[1]
    most = 1 if few else 113
    x = np.sort(rng.integers(-most + 1 if not few else -1, most + (1 if few else 0), (2, slots, h * d)), 0)[::-1]
    if few:
        x = np.repeat(x[:, :, :1], h * d, 2)
    for s in range(2):
        pool_layer[s][:, n:n + h * d] = torch.from_numpy(x[s].astype(np.int8).copy()).view(torch.uint8)
