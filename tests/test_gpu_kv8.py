"""GPU tests of the 8-bit KV cache's operators (cascade_kv_append,
cascade_attention, cascade_kv_evict) against the 64-bit reference.

Tolerances.  u is the unit roundoff of the rows' type: 2^-8 for bfloat16's 8
significant bits, 2^-11 for float16's 11.

append, queries: the hardware sine and cosine are within 2^-22 of exact (1.3e-7
measured over the circle) and the turn is cut to 24 bits (2 pi 2^-25): an
element is off by 2^-20 (|a| + |b|) of its pair at most, then rounded once.
append, codes: a code's value is the E4M3 number next to x / scale, where x is
off by as much; so it is no further from the exact quotient than the nearest
one is, plus twice that.

attention: scores carry 32-bit errors.  A sum of D products in 32 bits is off
by at most (D + 8) 2^-24 sum|q k|; the product with the scale, the cap, the
difference from m (up to |s| + 8 large) and exp2 add 2^-21 (|s| + 16).  With e
the sum of these, weights are off by 2 e relatively (numerator and sum).  Each
weight is rounded to the rows' type (u; below float16's normal range 2^-25,
against a sum of at least 1, since m is at most the row's maximum), the result
once more (u), partial sums in 32 bits add 2^-16.
"""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


def on_gpu(b):
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in b.items()}


def make_batch(dev, g):
    return dev.KvBatch(g["off"], g["len"], g["rows"], g["slots"], g["tokens"], g["most"])


def rows(rng, t, h, d, dt, spread=1.0):
    x = rng.normal(0, 1, (t, h, d)) * np.exp2(rng.normal(0, spread, (1, h, 1)))
    return torch.from_numpy(x).to(dt)


# ------------------------------------------------------------------ append

APPEND = [
    # heads, kv heads, dim, block, type, rotary, interleaved, counts, lengths
    (8, 2, 128, 16, "bf16", 128, False, [1], [1]),
    (8, 2, 128, 16, "bf16", 128, False, [1, 1, 1], [16, 17, 700]),
    (4, 4, 64, 16, "f16", 64, True, [16, 15, 17, 0, 1], [16, 31, 40, 9, 33]),
    (6, 2, 256, 16, "bf16", 64, False, [40, 3], [45, 3]),
    (4, 1, 128, 32, "f16", 32, True, [70, 1, 33], [75, 32, 65]),
    (3, 3, 64, 128, "bf16", 16, False, [300, 5, 128], [301, 130, 256]),
    (2, 1, 256, 64, "f16", 256, True, [64, 65, 1], [64, 100, 1]),
    (16, 8, 128, 16, "bf16", 0, False, [530, 9], [541, 12]),
    (16, 5, 64, 64, "bf16", 48, False, [600, 1, 1], [650, 64, 65]),
]


@pytest.mark.parametrize("case", APPEND, ids=[f"{c[0]}h{c[1]}kv{c[2]}d{c[3]}bt-{c[4]}-r{c[5]}" for c in APPEND])
def test_append(dev, case):
    H, h, d, bt, name, R, inter, counts, lengths = case
    dt, u = TYPES[name], U[name]
    rng = np.random.default_rng(sum(counts) + d)
    b = ref.batch(rng, counts, lengths, bt, slack=1)
    layers, layer = 2, 1
    # old scales below and above what the new tokens need: some blocks grow
    pool = ref.random_pool(rng, layers, b["pool"], h, d, bt, pad=32, spread=3)
    before = pool.clone()
    T = b["tokens"]
    x = torch.cat([rows(rng, T, H, d, dt), rows(rng, T, h, d, dt, 2), rows(rng, T, h, d, dt, 2)], 1)
    pos = rng.integers(0, 1 << 20, T).astype(np.int32)
    pos[0] = 2 ** 31 - 1
    th, _ = ref.theta("plain", max(R, 2), 10000.0)
    freq = ref.fixed(th)[:R // 2]
    mult = 1.0 if R == 0 else 1.25
    g, xg = on_gpu(b), x.cuda()
    gpool = pool.cuda()
    kv = dev.DeviceKvPool(gpool, h, d, bt)
    q_out = torch.zeros(T, H, d, dtype=dt, device="cuda")
    op = dev.DeviceKvAppend(
        kv, make_batch(dev, g), xg[:, :H], xg[:, H:H + h], xg[:, H + h:], q_out,
        torch.from_numpy(pos).cuda(), torch.from_numpy(freq.view(np.int64).copy()).cuda() if R else None,
        inter, mult, layer)
    op.run()
    torch.cuda.synchronize()
    kv.check()
    got = gpool.cpu()
    assert torch.equal(got[0], before[0])                  # the other layer
    n = ref.chunk_bytes(h, d, bt)
    assert torch.equal(got[1, :, :, n:], before[1, :, :, n:])  # the padding
    qe = ref.rotate(x[:, :H], pos, freq, inter, mult)
    size = x[:, :H].to(ref.F64).abs().amax(2, keepdim=True) * 2 * mult
    assert ((q_out.cpu().to(ref.F64) - qe).abs() <= u * qe.abs() + 2.0 ** -20 * size).all()
    for side, e in ((0, ref.rotate(x[:, H:H + h], pos, freq, inter, mult)), (1, x[:, H + h:].to(ref.F64))):
        val, sc, fresh, want = ref.append(before[1, side], e, b, h, d, bt, side)
        raw = ref.codes_of(got[1, side], h, d, bt, side)
        have = raw.view(ref.E4M3).float().to(ref.F64)
        assert torch.equal(ref.scales_of(got[1, side], h, d, bt).to(ref.F64), sc)
        # older tokens and places past the end: to the byte
        exact = ref.codes_of(before[1, side], h, d, bt, side)
        touched = torch.zeros(val.shape[0], dtype=torch.bool)
        assert torch.equal(have[~fresh], val[~fresh])
        same_scale = (ref.scales_of(before[1, side], h, d, bt).to(ref.F64) == sc)[..., None, None].expand_as(raw)
        assert torch.equal(raw[~fresh & same_scale], exact[~fresh & same_scale])
        slack = 0.0
        if side == 0 and R:
            big = e.abs().amax()  # of any pair
            slack = 2.0 ** -20 * 2 * 2 * big / sc[..., None, None]
        off, best = (have - want).abs(), (ref.round_e4m3(want) - want).abs()
        assert (off <= best + 2 * slack + 1e-12)[fresh].all()
        if side == 1 or R == 0:
            assert torch.equal(have[fresh], val[fresh])


def test_append_in_place_and_strided(dev):
    """Queries turned in place inside a fused projection; then the same with
    contiguous copies gives the same bytes."""
    rng = np.random.default_rng(5)
    H, h, d, bt = 8, 2, 128, 16
    b = ref.batch(rng, [3, 20], [19, 20], bt)
    g = on_gpu(b)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    x = rows(rng, b["tokens"], H + 2 * h + 1, d, torch.bfloat16).cuda()
    freq = torch.from_numpy(ref.fixed(ref.theta("plain", 64, 1e4)[0]).view(np.int64).copy()).cuda()
    pos = torch.arange(b["tokens"], dtype=torch.int32, device="cuda") * 977
    outs = []
    for strided in (True, False):
        y = x.clone()
        kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
        q, k, v = y[:, :H], y[:, H:H + h], y[:, H + h:H + 2 * h]
        if not strided:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        dev.DeviceKvAppend(kv, make_batch(dev, g), q, k, v, q, pos, freq).run()
        kv.check()
        outs.append((q.clone(), kv.pool))
        if strided:
            assert torch.equal(y[:, H:], x[:, H:])
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_append_without_queries_and_repeated(dev):
    """No queries, no rotation; a second write of the same tokens changes
    nothing, and tokens written one by one meet those written at once where
    the first token has the largest elements."""
    rng = np.random.default_rng(6)
    h, d, bt = 2, 64, 16
    b = ref.batch(rng, [30], [37], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt, spread=0)
    k = rows(rng, 30, h, d, torch.float16)
    k[::9] = k[::9] * 0 + 30.0
    v = k.flip(0).contiguous()
    v[::9] = 30.0
    g = on_gpu(b)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
    op = dev.DeviceKvAppend(kv, make_batch(dev, g), None, k.cuda(), v.cuda())
    op.run()
    first = kv.pool.clone()
    op.run()
    assert torch.equal(kv.pool, first)
    one = dev.DeviceKvPool(pool.cuda(), h, d, bt)
    for t in range(30):
        s = dict(g, off=torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                 len=torch.tensor([7 + t + 1], dtype=torch.int32, device="cuda"), tokens=1, most=1)
        dev.DeviceKvAppend(one, make_batch(dev, s), None, k[t:t + 1].cuda(), v[t:t + 1].cuda()).run()
    one.check()
    assert torch.equal(one.pool, first)


def test_append_extreme_values(dev):
    """Zeros, the type's largest and smallest; NaN and infinities are refused
    by the status word and stored as 0."""
    h, d, bt = 1, 64, 16
    rng = np.random.default_rng(7)
    b = ref.batch(rng, [16, 1, 1, 1], [16, 1, 1, 1], bt)
    g = on_gpu(b)
    k = torch.zeros(19, h, d, dtype=torch.bfloat16)
    k[16] = torch.finfo(torch.bfloat16).max
    k[17] = 2.0 ** -120
    k[18] = 1.0
    kv = dev.DeviceKvPool(torch.zeros(1, 2, b["pool"], ref.chunk_bytes(h, d, bt), dtype=torch.uint8).cuda(),
                          h, d, bt)
    dev.DeviceKvAppend(kv, make_batch(dev, g), None, k.cuda(), k.cuda()).run()
    kv.check()
    for side in range(2):
        val, sc, fresh, _ = ref.append(torch.zeros_like(kv.pool[0, side].cpu()), k.to(ref.F64), b, h, d, bt, side)
        got = ref.values_of(kv.pool[0, side].cpu(), h, d, bt, side)
        assert torch.equal(got, val * sc[..., None, None]) and torch.isfinite(got).all()
    k[3, 0, 5], k[18, 0, 7] = float("nan"), float("-inf")
    op = dev.DeviceKvAppend(kv, make_batch(dev, g), None, k.cuda(), k.cuda())
    op.run()
    with pytest.raises(RuntimeError):
        kv.check()
    got = ref.values_of(kv.pool[0, 0].cpu(), h, d, bt, 0)
    assert torch.isfinite(got).all()
    assert got[b["slots"][0], 0, 3, 5] == 0 and got[b["slots"][3], 0, 0, 7] == 0


@pytest.mark.parametrize("fault", ["slot", "negative slot", "position", "length", "offsets", "row"])
def test_append_refuses_bad_device_data(dev, fault):
    """A bad request is reported and not written; the others are."""
    rng = np.random.default_rng(8)
    h, d, bt = 2, 64, 16
    b = ref.batch(rng, [2, 2, 2], [20, 21, 22], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    k = rows(rng, 6, h, d, torch.bfloat16)
    pos = torch.arange(6, dtype=torch.int32)
    freq = torch.from_numpy(ref.fixed(ref.theta("plain", 64, 1e4)[0]).view(np.int64).copy()).cuda()
    bad = {k_: v.clone() if torch.is_tensor(v) else v for k_, v in b.items()}
    if fault == "slot":
        bad["slots"][3] = b["pool"]
    elif fault == "negative slot":
        bad["slots"][3] = -1
    elif fault == "position":
        pos[2] = -1
    elif fault == "length":
        bad["len"][1] = 1
    elif fault == "offsets":
        bad["off"][2] = 1 << 20
    else:
        bad["len"][1] = 50
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
    dev.DeviceKvAppend(kv, make_batch(dev, on_gpu(bad)), None, k.cuda(), k.cuda(), None, pos.cuda(), freq).run()
    with pytest.raises(RuntimeError):
        kv.check()
    touched = {int(b["slots"][int(b["rows"][i]) + 1]) for i in (0, 2)}
    for slot in range(b["pool"]):
        same = torch.equal(kv.pool[0, :, slot].cpu(), pool[0, :, slot])
        if slot not in touched:
            if not (fault == "position" and slot == int(b["slots"][3])):  # its values have no position
                assert same, slot
        elif fault != "offsets":  # (then the next request's rows are unknown too)
            assert not same


# --------------------------------------------------------------- attention

ATTEND = [
    # heads, kv heads, dim, block, type, cap, window, counts, lengths
    (8, 2, 128, 16, "bf16", 0.0, 0, [1], [1]),
    (8, 2, 128, 16, "bf16", 0.0, 1, [1, 1, 1, 1, 1], [2, 15, 16, 17, 33]),
    (4, 1, 64, 16, "f16", 0.0, 2, [1, 0, 2, 3], [130, 40, 64, 95]),
    (4, 4, 256, 32, "bf16", 20.0, 3, [1, 4, 2], [300, 70, 31]),
    (14, 2, 128, 16, "f16", 5.0, 1, [2, 1, 9], [257, 128, 9]),
    (20, 4, 64, 64, "bf16", 0.0, 4, [3, 12], [129, 65]),
    (32, 1, 128, 128, "bf16", 0.0, 1, [1, 1], [200, 513]),
    (8, 2, 128, 16, "bf16", 0.0, 7, [40, 1, 70], [90, 300, 70]),
    (6, 3, 64, 16, "f16", 30.0, 64, [150, 3], [190, 5]),
    (128, 1, 64, 16, "bf16", 0.0, 2, [3, 1], [50, 20]),
    (2, 2, 256, 16, "f16", 0.0, 0, [65, 129], [65, 400]),
    # new tokens without any cached one before them, and rows that see nothing
    (8, 2, 128, 16, "bf16", 0.0, 3, [5, 2, 1], [3, 0, 4]),
    (8, 2, 128, 16, "f16", 0.0, 2, [80, 20], [37, 0]),
]


def bounds(e, name, d, scale_abs):
    """(out, lse, weight) tolerances of a reference result."""
    u = U[name]
    s = torch.where(torch.isfinite(e["lse"]), e["lse"].abs(), 0.0) + e["err"]
    eps = (d + 8) * 2.0 ** -24 * e["err"] + 2.0 ** -21 * (s + 16)
    out = e["mass"] * (2 * eps[..., None] + u + 2.0 ** -16) + u * e["out"].abs() + 1e-30
    if name == "f16":
        out = out + 2.0 ** -24 * e["reach"] + 2.0 ** -25
    return out, 2 * eps, eps


def run_attention(dev, pool, q, g, h, d, bt, scale, cap=0.0, window=0, want_lse=True, workspace=None,
                  stream=None, layer=0):
    kv = dev.DeviceKvPool(pool, h, d, bt)
    T, H = q.shape[:2]
    out = torch.full((T, H, d), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((T, H), 7.0, device="cuda") if want_lse else None
    w = torch.zeros(len(g["slots"]), device="cuda") if window else None
    op = dev.DeviceAttention(kv, make_batch(dev, g), q, out, scale, cap, lse, w, window, layer, workspace)
    if workspace is None:
        op.workspace.fill_(0xff)  # any content: here NaN
    op.run(stream)
    torch.cuda.synchronize()
    kv.check()
    return out, lse, w


def check_attention(got, e, name, d, window):
    out, lse, w = got
    to, tl, tw = bounds(e, name, d, 1.0)
    off = (out.cpu().to(ref.F64) - e["out"]).abs()
    assert (off <= to).all(), float((off / to).max())
    if lse is not None:
        x = lse.cpu().to(ref.F64)
        none = torch.isinf(e["lse"])
        assert torch.equal(torch.isinf(x), none) and (x[none] < 0).all()
        assert ((x - e["lse"]).abs() <= tl)[~none].all()
    if window:
        rel = 2 * float(tw.max()) + 2.0 ** -18
        assert ((w.cpu().to(ref.F64) - e["weight"]).abs() <= rel * e["weight"] + 1e-30).all()


@pytest.mark.parametrize("case", ATTEND, ids=[f"{c[0]}h{c[1]}kv{c[2]}d{c[3]}bt-{c[4]}-n{max(c[7])}-l{max(c[8])}" for c in ATTEND])
def test_attention(dev, case):
    H, h, d, bt, name, cap, window, counts, lengths = case
    rng = np.random.default_rng(sum(lengths) + H)
    b = ref.batch(rng, counts, lengths, bt, slack=2)
    pool = ref.random_pool(rng, 2, b["pool"], h, d, bt, pad=16)
    # everything past a request's last token is NaN codes
    for i in range(b["n"]):
        l, row = int(b["len"][i]), int(b["rows"][i])
        if l % bt:
            for side in range(2):
                at = ref.code_offsets(h, d, bt, side)[:, l % bt:].flatten()
                pool[1, side, int(b["slots"][row + l // bt]), at] = 0x7f
    q = rows(rng, b["tokens"], H, d, TYPES[name])
    scale = 1.7 * d ** -0.5
    e = ref.attend(pool[1], q, b, h, d, bt, scale, cap, window)
    got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, scale, cap, window, layer=1)
    check_attention(got, e, name, d, window)


def test_attention_cut_over_workgroups(dev):
    """Long requests are cut and joined; a few heads, one and several rows,
    beside short ones."""
    rng = np.random.default_rng(3)
    H, h, d, bt = 4, 1, 64, 16
    for counts, lengths, window in (([1, 1, 2], [9001, 5, 4097], 2), ([40, 1], [5000, 777], 3),
                                    ([200], [6003], 1)):
        b = ref.batch(rng, counts, lengths, bt)
        pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
        q = rows(rng, b["tokens"], H, d, torch.bfloat16)
        e = ref.attend(pool[0], q, b, h, d, bt, 0.3, 0.0, window)
        got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, 0.3, 0.0, window)
        check_attention(got, e, "bf16", d, window)
        again = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, 0.3, 0.0, window)
        assert all(torch.equal(x, y) for x, y in zip(got, again))


def test_attention_peaked_and_flat_scores(dev):
    """Rows whose maximum grows late by far more than the lag that m may
    have, rows of equal scores, and a scale of 0."""
    rng = np.random.default_rng(4)
    H, h, d, bt = 4, 2, 64, 16
    b = ref.batch(rng, [1, 2], [400, 333], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt, spread=0)
    q = rows(rng, b["tokens"], H, d, torch.float16)
    for scale in (8.0, 0.0, -0.4):
        e = ref.attend(pool[0], q, b, h, d, bt, scale, 0.0, 1)
        got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, scale, 0.0, 1)
        check_attention(got, e, "f16", d, 1)


def test_attention_strided_rows_and_nan_queries(dev):
    """Rows with strides of their own; a NaN query spoils its own row only."""
    rng = np.random.default_rng(9)
    H, h, d, bt = 8, 2, 128, 16
    b = ref.batch(rng, [3, 1, 30], [40, 100, 77], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    g = on_gpu(b)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    base = run_attention(dev, pool.cuda(), q.cuda(), g, h, d, bt, 0.09)
    wide = torch.zeros(H, b["tokens"], d + 8, dtype=q.dtype, device="cuda")
    qs = wide.transpose(0, 1)[..., :d]
    qs.copy_(q)
    qs[5, 3] = float("nan")
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
    out = torch.zeros(b["tokens"], 2 * H, d, dtype=q.dtype, device="cuda")[:, ::2]
    dev.DeviceAttention(kv, make_batch(dev, g), qs, out, 0.09).run()
    bad = torch.zeros(b["tokens"], H, dtype=torch.bool)
    bad[5, 3] = True
    assert torch.isnan(out[5, 3]).all()
    assert torch.equal(out.cpu()[~bad], base[0].cpu()[~bad])


def test_attention_many_requests(dev):
    """More requests than a workgroup's threads, most without new tokens."""
    rng = np.random.default_rng(10)
    H, h, d, bt = 4, 2, 64, 16
    counts = (np.arange(700) % 7 == 0).astype(int)
    counts[350] = 40
    lengths = np.maximum(rng.integers(1, 60, 700), counts)
    b = ref.batch(rng, counts, lengths, bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    e = ref.attend(pool[0], q, b, h, d, bt, 0.2, 0.0, 1)
    got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, 0.2, 0.0, 1)
    check_attention(got, e, "bf16", d, 1)


def test_attention_on_another_stream_and_in_a_graph(dev):
    rng = np.random.default_rng(11)
    H, h, d, bt = 8, 2, 128, 16
    b = ref.batch(rng, [1, 1, 30], [600, 33, 200], bt)
    g = on_gpu(b)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt).cuda()
    q = rows(rng, b["tokens"], H, d, torch.bfloat16).cuda()
    want = run_attention(dev, pool, q, g, h, d, bt, 0.1, 0.0, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run_attention(dev, pool, q, g, h, d, bt, 0.1, 0.0, 2, stream=side)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    kv = dev.DeviceKvPool(pool, h, d, bt)
    out, w = torch.zeros_like(want[0]), torch.zeros_like(want[2])
    op = dev.DeviceAttention(kv, make_batch(dev, g), q, out, 0.1, block_weight=w, weight_window=2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.run()
    for i in range(3):
        w.zero_()
        out.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(w, want[2])
        q.mul_(1.0)


@pytest.mark.parametrize("fault", ["slot", "length", "offsets", "row"])
def test_attention_reports_bad_device_data(dev, fault):
    """Reported; the other requests are answered."""
    rng = np.random.default_rng(12)
    H, h, d, bt = 4, 2, 64, 16
    b = ref.batch(rng, [1, 1, 1], [40, 50, 60], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q = rows(rng, 3, H, d, torch.bfloat16)
    e = ref.attend(pool[0], q, b, h, d, bt, 0.2)
    g = on_gpu(b)
    if fault == "slot":
        g["slots"][int(b["rows"][1]) + 1] = b["pool"] + 5
    elif fault == "length":
        g["len"][1] = -1
    elif fault == "offsets":
        g["off"][1:3] = torch.tensor([1, 9], dtype=torch.int32)
    else:
        g["len"][1] = 1000
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
    out = torch.zeros(3, H, d, dtype=q.dtype, device="cuda")
    dev.DeviceAttention(kv, make_batch(dev, g), q.cuda(), out, 0.2).run()
    with pytest.raises(RuntimeError):
        kv.check()
    to = bounds(e, "bf16", d, 1.0)[0]
    fine = [0, 2] if fault != "offsets" else [0]
    assert ((out.cpu().to(ref.F64) - e["out"]).abs() <= to)[fine].all()


# ------------------------------------------------------------------- evict

@pytest.mark.parametrize("bt,sink,recent,lengths,keep", [
    (16, 0, 1, [1], [0]),
    (16, 1, 2, [0, 16, 17, 160, 500], [1, 1, 1, 4, 31]),
    (32, 0, 1, [3200, 10, 999], [0, 0, 1000]),
    (16, 3, 5, [40000, 16 * 1024, 16 * 1025, 100], [100, 1000, 1024, 2]),
    (1, 0, 1, [5000, 3], [17, 1]),
    (128, 200, 300, [128 * 600, 128 * 400], [0, 0]),
])
def test_evict(dev, bt, sink, recent, lengths, keep):
    rng = np.random.default_rng(sum(lengths))
    b = ref.batch(rng, np.zeros(len(lengths), int), lengths, bt, slack=1)
    n = len(b["slots"])
    for values in ("random", "ties", "odd"):
        w = rng.random(n).astype(np.float32) ** 6
        if values == "ties":
            w = np.floor(w * 4).astype(np.float32)
        if values == "odd":
            w[rng.random(n) < 0.3] = rng.choice([0.0, -0.0, -1.5, np.inf, -np.inf, np.nan, 1e-40, 3.4e38])
            w[rng.random(n) < 0.1] = np.nan
        e = ref.evict(b, w, keep, sink, recent, bt)
        g = on_gpu(b)
        k = torch.tensor(keep, dtype=torch.int32, device="cuda")
        op = dev.DeviceKvEvict(bt, g["len"], g["rows"], g["slots"], torch.from_numpy(w).cuda(), k, sink, recent)
        op.run()
        assert int(op.status) == 0
        assert op.kv_len_out.tolist() == e[0]
        assert op.row_offsets_out.tolist() == e[1]
        kept, gone = len(e[2]), len(e[4])
        assert op.slots_out[:kept].tolist() == e[2]
        assert np.array_equal(op.weight_out[:kept].cpu().numpy(), np.asarray(e[3], np.float32), equal_nan=True)
        assert int(op.n_freed) == gone and op.freed[:gone].tolist() == e[4]
        assert not op.slots_out[kept:].any() and not op.freed[gone:].any()


def test_evict_bad_requests(dev):
    rng = np.random.default_rng(2)
    b = ref.batch(rng, [0, 0, 0], [100, 100, 100], 16)
    w = torch.rand(len(b["slots"])).cuda()
    for fault in ("len", "keep", "row"):
        g = on_gpu(b)
        keep = torch.full((3,), 3, dtype=torch.int32, device="cuda")
        if fault == "len":
            g["len"][1] = 200
        elif fault == "keep":
            keep[1] = -1
        else:
            g["rows"][2] = 1 << 30
        op = dev.DeviceKvEvict(16, g["len"], g["rows"], g["slots"], w, keep)
        op.run()
        assert int(op.status) == -1
        assert op.row_offsets_out[1] == 3


def test_evict_nothing(dev):
    z = lambda *a: torch.zeros(*a, dtype=torch.int32, device="cuda")
    op = dev.DeviceKvEvict(16, z(0), z(1), z(0), torch.zeros(0, device="cuda"), z(0),
                           out=(z(1), z(1) + 5, z(1), torch.zeros(1, device="cuda"), z(1), z(1) + 5))
    op.run()
    assert int(op.row_offsets_out[0]) == 0 and int(op.n_freed) == 0


# ------------------------------------------------------ the cycle, together

def test_written_evicted_moved_and_read(dev):
    """A request's tokens are written in chunks and single tokens, attended
    with weights, cut, its blocks moved through staging by the pool's own
    copy, and attended again: each read against the reference on the bytes in
    the pool."""
    from paper_2608_06557_amd import cascade
    rng = np.random.default_rng(13)
    H, h, d, bt, L = 8, 2, 128, 16, 2
    n, nb = 2, 12
    kv = dev.DeviceKvPool.empty(L, 40, h, d, bt)
    slots = torch.from_numpy(rng.permutation(40)[:n * nb].astype(np.int32))
    table = torch.tensor([0, nb, 2 * nb], dtype=torch.int32)
    have = np.zeros(n, int)
    freq, mult = dev.rope_frequencies(128, 10000.0)
    weight = torch.zeros(n * nb, device="cuda")
    for counts in ([33, 64], [1, 1], [1, 5], [70, 1]):
        counts = np.array(counts)
        have += counts
        off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        b = dict(n=n, off=torch.from_numpy(off), len=torch.from_numpy(have.astype(np.int32)), rows=table,
                 slots=slots, tokens=int(off[-1]), most=int(counts.max()))
        g = on_gpu(b)
        x = rows(rng, b["tokens"], H + 2 * h, d, torch.bfloat16).cuda()
        pos = torch.from_numpy(np.concatenate([np.arange(l - c, l) for l, c in zip(have, counts)]).astype(np.int32)).cuda()
        q = torch.empty(b["tokens"], H, d, dtype=torch.bfloat16, device="cuda")
        out = torch.empty_like(q)
        batch = make_batch(dev, g)
        for layer in range(L):
            dev.DeviceKvAppend(kv, batch, x[:, :H], x[:, H:H + h], x[:, H + h:], q, pos, freq, False, mult,
                               layer).run()
            w = weight if layer == L - 1 else None
            dev.DeviceAttention(kv, batch, q, out, d ** -0.5, block_weight=w, weight_window=4, layer=layer).run()
            kv.check()
            e = ref.attend(kv.pool[layer].cpu(), q.cpu(), b, h, d, bt, d ** -0.5)
            check_attention((out, None, None), e, "bf16", d, 0)
    op = dev.DeviceKvEvict(bt, g["len"], g["rows"], g["slots"], weight,
                           torch.tensor([5, 4], dtype=torch.int32, device="cuda"), 1, 2)
    op.run()
    e = ref.evict(b, weight.cpu().numpy(), [5, 4], 1, 2, bt)
    rows_out, kept = op.row_offsets_out.cpu(), int(op.row_offsets_out[-1])
    assert rows_out.tolist() == e[1] == [0, 5, 9]
    # spill what stays, and restore it into other slots
    free = [s for s in range(40) if s not in set(op.slots_out[:kept].tolist())][:kept]
    move = np.zeros((kept, 4), np.int32)
    move[:, 2], move[:, 3] = op.slots_out[:kept].cpu().numpy(), np.arange(kept)
    back = move.copy()
    back[:, 2] = free
    staging = torch.zeros(kept * 2 * L * kv.chunk_bytes, dtype=torch.uint8, device="cuda")
    count = torch.tensor([kept], dtype=torch.int32, device="cuda")
    sh = dev.stream_handle()
    mv, bk = torch.from_numpy(move).cuda(), torch.from_numpy(back).cuda()
    for fn, m in ((cascade.cascade_pack, mv), (cascade.cascade_unpack, bk)):
        assert fn(kv.c_pool, staging.data_ptr(), kept, m.data_ptr(), count.data_ptr(), kept,
                  kv.status.data_ptr(), sh) == 0
    b2 = dict(n=n, off=torch.tensor([0, 1, 2], dtype=torch.int32), len=op.kv_len_out.cpu(), rows=rows_out,
              slots=torch.tensor(free, dtype=torch.int32), tokens=2, most=1)
    q2 = rows(rng, 2, H, d, torch.bfloat16)
    got = []
    for s in (op.slots_out[:kept].clone(), b2["slots"].cuda()):
        got.append(run_attention(dev, kv.pool, q2.cuda(), dict(on_gpu(b2), slots=s), h, d, bt, d ** -0.5, layer=1))
    assert all(torch.equal(a, c) for a, c in zip(got[0][:2], got[1][:2]))
    e = ref.attend(kv.pool[1].cpu(), q2, b2, h, d, bt, d ** -0.5)
    check_attention(got[1], e, "bf16", d, 0)
