"""cascade_kv_bounds and cascade_kv_select, whose results are whole numbers and
have to be equal, and cascade_attention_selected (tolerances of
tests/test_gpu_kv8.py), against the 64-bit reference."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests import sparse_ref as sref
from tests.test_gpu_kv8 import TYPES, check_attention, make_batch, on_gpu, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


def make_pool(rng, layers, b, h, d, bt, pad=0, spread=2):
    """With room for bounds, of 0x55, and `pad` bytes behind them."""
    pool = ref.random_pool(rng, layers, b["pool"], h, d, bt, pad=h * d + pad, spread=spread)
    pool[..., ref.chunk_bytes(h, d, bt):] = 0x55
    return pool


# ------------------------------------------------------------------ bounds

BOUNDS = [
    # kv heads, dim, block, whole, counts, lengths
    (2, 128, 16, False, [1], [1]),
    (8, 128, 16, False, [1, 1, 0, 1, 1], [16, 17, 40, 33, 700]),
    (3, 64, 32, False, [40, 3, 100, 32], [41, 3, 131, 64]),
    (1, 256, 128, False, [130, 1, 300], [257, 128, 300]),
    (5, 128, 64, True, [0, 0, 3, 0], [0, 1, 700, 64]),
    (4, 64, 16, True, [0] * 5, [15, 16, 17, 0, 5000]),
    (2, 64, 16, False, [5, 20], [3, 0]),             # new tokens that are not cached
    (1, 128, 16, False, [1200, 900, 1, 777], [1300, 900, 30, 779]),
    (1, 64, 16, True, [0] * 3, [20000, 9, 16000]),
]


@pytest.mark.parametrize("case", BOUNDS, ids=[f"kv{c[0]}d{c[1]}bt{c[2]}-{i}" for i, c in enumerate(BOUNDS)])
def test_bounds(dev, case):
    h, d, bt, whole, counts, lengths = case
    rng = np.random.default_rng(d + sum(lengths))
    b = ref.batch(rng, counts, lengths, bt, slack=1)
    pool = make_pool(rng, 2, b, h, d, bt, pad=32)
    for i in range(b["n"]):  # past a request's end there may be anything
        l, row = int(b["len"][i]), int(b["rows"][i])
        if l % bt:
            at = ref.code_offsets(h, d, bt, 0)[:, l % bt:].flatten()
            pool[1, 0, int(b["slots"][row + l // bt]), at] = 0x7f
    before = pool.clone()
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    dev.DeviceKvBounds(kv, make_batch(dev, on_gpu(b)), whole, layer=1).run()
    torch.cuda.synchronize()
    kv.check()
    got = kv.pool.cpu()
    want = before.clone()
    n = ref.chunk_bytes(h, d, bt)
    for slot, both in sref.bounds_of(before[1], b, h, d, bt, whole).items():
        for s in range(2):
            want[1, s, slot, n:n + h * d] = torch.from_numpy(both[s].astype(np.int8)).view(torch.uint8).flatten()
    assert torch.equal(got, want)  # and nothing else has changed


def test_bounds_of_every_code(dev):
    """Each finite code alone, and against its negative."""
    h, d, bt = 1, 64, 16
    codes = torch.tensor([c for c in range(256) if c & 0x7f != 0x7f], dtype=torch.uint8)
    slots = 2 * len(codes)
    pool = torch.zeros(1, 2, slots, ref.chunk_bytes(h, d, bt) + h * d, dtype=torch.uint8)
    x = torch.zeros(slots, h, bt, d, dtype=torch.uint8)
    x[:len(codes)] = codes[:, None, None, None]
    x[len(codes):] = codes[:, None, None, None]
    x[len(codes):, :, 1::2] ^= 0x80
    ref.store(pool[0, 0], x, torch.ones(slots, h), h, d, bt, 0)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32)
    b = dict(n=1, off=i32([0, 0]), len=i32([slots * bt]), rows=i32([0, slots]), slots=torch.arange(slots, dtype=torch.int32),
             tokens=0, most=0)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    dev.DeviceKvBounds(kv, make_batch(dev, on_gpu(b)), True).run()
    kv.check()
    upper, lower = sref.bounds_in(kv.pool[0].cpu(), h, d, bt)
    for slot, (u, l) in sref.bounds_of(pool[0], b, h, d, bt, True).items():
        assert np.array_equal(upper[slot], u) and np.array_equal(lower[slot], l), slot


@pytest.mark.parametrize("fault", ["slot", "negative slot", "length", "offsets", "row"])
def test_bounds_refuse_bad_device_data(dev, fault):
    rng = np.random.default_rng(3)
    h, d, bt = 2, 64, 16
    b = ref.batch(rng, [1, 2, 1], [40, 50, 20], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    want = sref.bounds_of(pool[0], b, h, d, bt, False)
    bad = {k: v.clone() if torch.is_tensor(v) else v for k, v in b.items()}
    spoil(bad, b, fault, 3)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    dev.DeviceKvBounds(kv, make_batch(dev, on_gpu(bad))).run()
    with pytest.raises(RuntimeError):
        kv.check()
    got = sref.bounds_in(kv.pool[0].cpu(), h, d, bt)
    slot = int(b["slots"][int(b["rows"][0]) + 2])  # the first request's
    assert np.array_equal(got[0][slot], want[slot][0]) and np.array_equal(got[1][slot], want[slot][1])


def spoil(bad, b, fault, at):
    """Something of the second request that is outside the domain."""
    row = int(b["rows"][1])
    if fault == "slot":
        bad["slots"][row + at] = b["pool"]
    elif fault == "negative slot":
        bad["slots"][row + at] = -1
    elif fault == "length":
        bad["len"][1] = 1 << 20
    elif fault == "offsets":
        bad["off"][2] = 1 << 20
    else:
        bad["rows"][2] = 1 << 20


# ------------------------------------------------------------------ select

SELECT = [
    # heads, kv heads, dim, block, type, keep, sink, recent, counts, lengths
    (8, 2, 128, 16, "bf16", 4, 1, 1, [1], [1]),
    (8, 2, 128, 16, "bf16", 4, 1, 2, [1, 1, 0, 1], [64, 65, 900, 700]),
    (4, 4, 64, 16, "f16", 8, 0, 1, [2, 1, 3], [400, 128, 129]),
    (14, 2, 128, 32, "bf16", 5, 2, 3, [1, 1], [3000, 700]),       # nothing but sink and recent
    (12, 1, 256, 16, "f16", 7, 0, 3, [3, 1], [333, 2000]),
    (20, 1, 64, 16, "bf16", 6, 1, 1, [5, 1], [500, 1000]),        # 20 heads: two row sets
    (128, 1, 64, 64, "f16", 3, 0, 1, [2], [900]),
    (2, 2, 128, 16, "bf16", 9, 1, 2, [70, 1], [1000, 60]),
    (6, 3, 64, 128, "bf16", 4, 1, 1, [200, 30], [2000, 31]),
    (16, 1, 128, 16, "f16", 64, 1, 4, [9], [3999]),
    (8, 8, 128, 16, "bf16", 100, 0, 5, [5, 7], [3, 0]),           # rows that see nothing
    (2, 1, 64, 16, "bf16", 300, 2, 9, [1, 1], [60000, 4801]),     # more blocks than registers hold
]


def run_select(dev, kv, q, g, keep, sink, recent, layer=0, stream=None, check=True):
    got = torch.full((q.shape[0], kv.kv_heads, keep), -7, dtype=torch.int32, device="cuda")
    op = dev.DeviceKvSelect(kv, make_batch(dev, g), q, got, sink, recent, layer)
    op.workspace.fill_(0xff)
    op.run(stream)
    torch.cuda.synchronize()
    if check:
        kv.check()
    return got


@pytest.mark.parametrize("few", [False, True], ids=["", "ties"])
@pytest.mark.parametrize("case", SELECT, ids=[f"{c[0]}h{c[1]}kv{c[2]}d{c[3]}bt-{c[4]}-{i}" for i, c in enumerate(SELECT)])
def test_select(dev, case, few):
    H, h, d, bt, name, keep, sink, recent, counts, lengths = case
    rng = np.random.default_rng(sum(lengths) + H)
    b = ref.batch(rng, counts, lengths, bt, slack=2)
    pool = make_pool(rng, 2, b, h, d, bt, pad=16, spread=1 if few else 3)
    sref.random_bounds(rng, pool[1], h, d, bt, few)
    q = rows(rng, b["tokens"] + 2, H, d, TYPES[name], 3.0)  # the last two rows are no request's
    want = sref.select(pool[1], q, b, h, d, bt, keep, sink, recent)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    got = run_select(dev, kv, q.cuda(), on_gpu(b), keep, sink, recent, layer=1)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_select_extreme_queries(dev, name):
    """Zeros, the type's largest and least numbers, exactly 127 and just above,
    halves between whole numbers, heads of very unlike size."""
    rng = np.random.default_rng(8)
    H, h, d, bt = 4, 1, 64, 16
    dt = TYPES[name]
    b = ref.batch(rng, [1] * 8, [1500] * 8, bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, 8, H, d, dt)
    q[0] = 0
    q[1, :, ::2], q[1, :, 1::2] = torch.finfo(dt).max, -torch.finfo(dt).max
    q[2] = torch.finfo(dt).smallest_normal * torch.sign(q[2].float()).to(dt) / 2
    q[3] = torch.round(q[3].float() * 30).clamp(-127, 127).to(dt)
    q[3, :, 0] = 127
    q[4] = q[3]
    q[4, :, 0] = 127.5 if name == "f16" else 128
    q[5] = (torch.round(q[5].float() * 20) + 0.5).clamp(-100.5, 100.5).to(dt)
    q[5, :, 0] = 120
    q[6, 0] *= 2.0 ** 10
    q[6, 1:] *= 2.0 ** -20
    q[7, 1] = 0
    want = sref.select(pool[0], q, b, h, d, bt, 9, 0, 1)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    assert torch.equal(run_select(dev, kv, q.cuda(), on_gpu(b), 9, 0, 1).cpu(), want)
    q[5, 2, 7], q[6, 0, 3], q[6, 3, 2] = float("nan"), float("inf"), float("-inf")
    want = sref.select(pool[0], q, b, h, d, bt, 9, 0, 1)
    assert torch.equal(run_select(dev, kv, q.cuda(), on_gpu(b), 9, 0, 1, check=False).cpu(), want)
    with pytest.raises(RuntimeError):
        kv.check()


def test_select_most_requests(dev):
    """2048 requests, of none to a few hundred blocks."""
    rng = np.random.default_rng(9)
    counts = rng.integers(0, 3, 2048)
    lengths = counts + np.where(rng.random(2048) < 0.02, rng.integers(0, 5000, 2048), rng.integers(0, 200, 2048))
    b = ref.batch(rng, counts, lengths, 16)
    pool = make_pool(rng, 1, b, 1, 64, 16)
    sref.random_bounds(rng, pool[0], 1, 64, 16)
    q = rows(rng, b["tokens"], 2, 64, torch.bfloat16)
    kv = dev.DeviceKvPool(pool.cuda(), 1, 64, 16, bounds=True)
    got = run_select(dev, kv, q.cuda(), on_gpu(b), 5, 1, 1)
    assert torch.equal(got.cpu(), sref.select(pool[0], q, b, 1, 64, 16, 5, 1, 1))


@pytest.mark.parametrize("scores", ["", "ties", "two values", "far apart", "infinite", "one above"])
def test_select_many_rows(dev, scores):
    """Enough rows for a wave each; scores that fall into one part of their
    range, or have none."""
    rng = np.random.default_rng(10)
    H, h, d, bt, keep = 8, 8, 64, 16, 20
    b = ref.batch(rng, [3, 290], [2000, 5100], bt)
    pool = make_pool(rng, 1, b, h, d, bt, spread=1)
    sref.random_bounds(rng, pool[0], h, d, bt, scores == "ties")
    n = ref.chunk_bytes(h, d, bt) - 32
    scale = pool[0, 0, :, n:n + 32].contiguous().view(torch.float32)
    if scores == "two values":  # all scores alike but for the scale
        for s in range(2):
            pool[0, s, :, n + 32:] = pool[0, s, :1, n + 32:]
        scale[:] = 1.0
        scale[torch.from_numpy(rng.permutation(b["pool"])[:15])] = 2.0
    elif scores == "far apart":
        scale[:] = torch.exp2(torch.from_numpy(rng.integers(-90, 90, scale.shape)).float())
    elif scores == "infinite":
        scale[::40] = float("inf")
    elif scores == "one above":
        scale[7] = 2.0 ** 40
    pool[0, 0, :, n:n + 32] = scale.view(torch.uint8)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    want = sref.select(pool[0], q, b, h, d, bt, keep, 1, 2)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    got = run_select(dev, kv, q.cuda(), on_gpu(b), keep, 1, 2)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("fault", ["slot", "negative slot", "length", "offsets", "row"])
def test_select_refuses_bad_device_data(dev, fault):
    rng = np.random.default_rng(3)
    h, d, bt = 2, 64, 16
    b = ref.batch(rng, [1, 2, 1], [140, 150, 120], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, 4, 4, d, torch.bfloat16)
    want = sref.select(pool[0], q, b, h, d, bt, 4, 1, 1)
    bad = {k: v.clone() if torch.is_tensor(v) else v for k, v in b.items()}
    spoil(bad, b, fault, 3)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    got = run_select(dev, kv, q.cuda(), on_gpu(bad), 4, 1, 1, check=False).cpu()
    with pytest.raises(RuntimeError):
        kv.check()
    assert torch.equal(got[0], want[0])


# ---------------------------------------------------------------- attention

ATTEND = [
    # heads, kv heads, dim, block, type, cap, lse, keep, counts, lengths
    (8, 2, 128, 16, "bf16", 0.0, True, 1, [1], [1]),
    (8, 2, 128, 16, "bf16", 0.0, False, 4, [1, 1, 0, 1], [64, 65, 900, 700]),
    (4, 4, 64, 16, "f16", 20.0, True, 33, [2, 1, 3], [800, 128, 129]),
    (14, 2, 128, 32, "bf16", 0.0, True, 5, [1, 1], [3000, 33]),
    (12, 1, 256, 16, "f16", 0.0, True, 40, [3, 1], [333, 2000]),
    (20, 1, 64, 64, "bf16", 100.0, True, 9, [5, 1], [500, 1000]),
    (128, 1, 128, 16, "f16", 0.0, False, 3, [2], [900]),
    (40, 1, 256, 128, "bf16", 5.0, True, 6, [2, 1], [900, 1]),
    (2, 2, 128, 16, "bf16", 0.0, True, 9, [70, 1], [1000, 60]),
    (4, 2, 64, 16, "bf16", 0.0, True, 600, [1, 1], [12000, 4801]),  # cut into parts
    (4, 1, 64, 16, "f16", 0.0, True, 5000, [1], [60001]),           # of more blocks than a part may have
    (8, 8, 128, 16, "bf16", 0.0, True, 7, [5, 7], [3, 0]),          # rows that see nothing
]


def random_lists(rng, b, h, bt, keep, empty=0.1):
    """Ascending lists of any length, with or without the token's own block;
    rows behind the last request's name nothing sensible."""
    out = np.full((b["tokens"], h, keep), -1, np.int32)
    for i in range(b["n"]):
        first, count = int(b["off"][i]), int(b["off"][i + 1] - b["off"][i])
        for j in range(count):
            last = int(b["len"][i]) - count + j
            blocks = 0 if last < 0 else last // bt + 1
            for k in range(h):
                n = 0 if rng.random() < empty else int(rng.integers(0, min(keep, blocks) + 1))
                if rng.random() < 0.3:
                    n = min(keep, blocks)
                out[first + j, k, :n] = np.sort(rng.choice(blocks, n, replace=False)) if n else []
                if n and rng.random() < 0.5:
                    out[first + j, k, n - 1] = blocks - 1
    return torch.from_numpy(out)


def run_selected(dev, kv, q, g, lists, scale, cap=0.0, want_lse=True, layer=0, stream=None, check=True):
    out = torch.full(tuple(q.shape), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(tuple(q.shape[:2]), 7.0, device="cuda") if want_lse else None
    op = dev.DeviceSelectedAttention(kv, make_batch(dev, g), q, lists, out, scale, cap, lse, layer)
    op.workspace.fill_(0xff)
    op.run(stream)
    torch.cuda.synchronize()
    if check:
        kv.check()
    return out, lse, None


@pytest.mark.parametrize("case", ATTEND, ids=[f"{c[0]}h{c[1]}kv{c[2]}d{c[3]}bt-{c[4]}-{i}" for i, c in enumerate(ATTEND)])
def test_selected_attention(dev, case):
    H, h, d, bt, name, cap, want_lse, keep, counts, lengths = case
    rng = np.random.default_rng(sum(lengths) + H)
    b = ref.batch(rng, counts, lengths, bt, slack=1)
    pool = make_pool(rng, 2, b, h, d, bt)
    for i in range(b["n"]):  # everything past a request's last token is NaN codes
        l, row = int(b["len"][i]), int(b["rows"][i])
        if l % bt:
            for side in range(2):
                at = ref.code_offsets(h, d, bt, side)[:, l % bt:].flatten()
                pool[1, side, int(b["slots"][row + l // bt]), at] = 0x7f
    q = rows(rng, b["tokens"], H, d, TYPES[name])
    lists = random_lists(rng, b, h, bt, keep)
    scale = 1.7 * d ** -0.5
    e = sref.attend(pool[1], q, b, lists, h, d, bt, scale, cap)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    args = (dev, kv, q.cuda(), on_gpu(b), lists.cuda(), scale, cap, want_lse, 1)
    got = run_selected(*args)
    check_attention(got, e, name, d, 0)
    again = run_selected(*args)
    assert torch.equal(got[0], again[0]) and (not want_lse or torch.equal(got[1], again[1]))


@pytest.mark.parametrize("e", [-100, -20, 9, 80])
def test_selected_attention_scales_out_of_range(dev, e):
    """Scales that float16 does not hold: keys' are made good by the queries
    and the scale, values' small ones vanish."""
    rng = np.random.default_rng(14)
    H, h, d, bt = 4, 2, 64, 16
    b = ref.batch(rng, [1, 2], [200, 77], bt)
    pool = make_pool(rng, 1, b, h, d, bt, spread=0)
    n = ref.chunk_bytes(h, d, bt) - 16
    scales = torch.full((b["pool"], h), 2.0 ** e)
    scales[::2] = 2.0 ** (e + 1)
    pool[0, 0, :, n:n + 4 * h] = scales.view(torch.uint8)
    if e < 10:
        pool[0, 1, :, n:n + 4 * h] = (scales * 2.0 ** (-7 - e if e > 0 else 0)).contiguous().view(torch.uint8)
    q = rows(rng, 3, H, d, torch.float16)
    lists = random_lists(rng, b, h, bt, 6, 0.0)
    scale = 2.0 ** (-e - 10)
    want = sref.attend(pool[0], q, b, lists, h, d, bt, scale)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    check_attention(run_selected(dev, kv, q.cuda(), on_gpu(b), lists.cuda(), scale), want, "f16", d, 0)


@pytest.mark.parametrize("fault", ["behind", "order", "twice", "after the end", "slot", "offsets"])
def test_selected_attention_refuses_bad_lists(dev, fault):
    rng = np.random.default_rng(15)
    H, h, d, bt = 4, 2, 64, 16
    b = ref.batch(rng, [1, 2, 1], [140, 150, 120], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    q = rows(rng, 4, H, d, torch.bfloat16)
    lists = torch.tensor([0, 2, 5, 7, -1], dtype=torch.int32).expand(4, h, 5).clone()
    e = sref.attend(pool[0], q, b, lists, h, d, bt, 0.2)
    bad, listed = {k: v.clone() if torch.is_tensor(v) else v for k, v in b.items()}, lists.clone()
    if fault == "behind":
        listed[2, 1, 3] = 10
    elif fault == "order":
        listed[2, 1, 1] = 6
    elif fault == "twice":
        listed[2, 1, 1] = 0
    elif fault == "after the end":
        listed[2, 1, 1] = -1
    else:
        spoil(bad, b, fault, 5)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    got = run_selected(dev, kv, q.cuda(), on_gpu(bad), listed.cuda(), 0.2, check=False)
    with pytest.raises(RuntimeError):
        kv.check()
    check_attention((got[0].cpu()[:1], got[1].cpu()[:1], None), {k: v[:1] for k, v in e.items()}, "bf16", d, 0)


# ----------------------------------------------------------------- together

def test_written_bounded_selected_attended_and_moved(dev):
    """Chunks and single tokens enter as a program would do it; the selection
    meets the reference on the cache as it is; with every block kept the attention is
    the plain one; spilled and restored blocks bring their bounds along."""
    from paper_2608_06557_amd import cascade as cx
    rng = np.random.default_rng(21)
    H, h, d, bt, keep = 8, 2, 128, 16, 6
    total = [333, 150, 64]
    b = ref.batch(rng, [0, 0, 0], total, bt, spare=40)
    kv = dev.DeviceKvPool.empty(1, b["pool"], h, d, bt, bounds=True)
    x = rows(rng, sum(total), H + 2 * h, d, torch.bfloat16).cuda()
    start = np.concatenate([[0], np.cumsum(total)])
    held = np.zeros(3, int)
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32)
    for step in ([100, 150, 1], [232, 0, 1], [1, 0, 61], [0, 0, 1]):
        at = np.concatenate([start[i] + held[i] + np.arange(c) for i, c in enumerate(step)]).astype(int)
        held += step
        off = i32(np.concatenate([[0], np.cumsum(step)]))
        c = dict(b, off=off, len=i32(held), tokens=int(sum(step)), most=max(step))
        g = on_gpu(c)
        y = x[torch.from_numpy(at).cuda()]
        batch = make_batch(dev, g)
        dev.DeviceKvAppend(kv, batch, None, y[:, H:H + h], y[:, H + h:]).run()
        dev.DeviceKvBounds(kv, batch).run()
    kv.check()
    once = kv.pool.clone()
    c = dict(b, off=i32([0, 2, 3, 4]), len=i32(held), tokens=4, most=2)
    g, q = on_gpu(c), rows(rng, 4, H, d, torch.bfloat16)
    dev.DeviceKvBounds(kv, make_batch(dev, g), whole=True).run()
    assert torch.equal(kv.pool, once)  # they were up to date
    want = sref.select(once[0].cpu(), q, c, h, d, bt, keep, 1, 2)
    lists = run_select(dev, kv, q.cuda(), g, keep, 1, 2)
    assert torch.equal(lists.cpu(), want)
    e = sref.attend(once[0].cpu(), q, c, want, h, d, bt, 0.09)
    got = run_selected(dev, kv, q.cuda(), g, lists, 0.09)
    check_attention(got, e, "bf16", d, 0)
    every = run_select(dev, kv, q.cuda(), g, 30, 1, 2)
    check_attention(run_selected(dev, kv, q.cuda(), g, every, 0.09), ref.attend(once[0].cpu(), q, c, h, d, bt, 0.09),
                    "bf16", d, 0)
    # the first request leaves and comes back into other slots
    n = -(-total[0] // bt)
    free = sorted(set(range(b["pool"])) - set(b["slots"].tolist()))[:n]
    staging = torch.zeros(n * 2 * kv.chunk_bytes, dtype=torch.uint8, device="cuda")
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    for copy, slots in ((cx.cascade_pack, b["slots"][:n].tolist()), (cx.cascade_unpack, free)):
        moves = np.zeros(n, dev.MOVE_DTYPE)
        moves["pool_slot"], moves["staging_slot"] = slots, np.arange(n)
        m = torch.from_numpy(moves.view(np.int32).copy()).cuda()
        assert copy(kv.c_pool, staging.data_ptr(), n, m.data_ptr(), count.data_ptr(), n, kv.status.data_ptr(),
                    dev.stream_handle()) == 0
    g["slots"][:n] = i32(free).cuda()
    lists2 = run_select(dev, kv, q.cuda(), g, keep, 1, 2)
    assert torch.equal(lists2, lists)
    again = run_selected(dev, kv, q.cuda(), g, lists2, 0.09)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


def test_select_and_attend_on_another_stream_and_in_graphs(dev):
    """Bounds, selection and attention in one graph; two graphs share their
    workspaces and are replayed in turn."""
    rng = np.random.default_rng(22)
    H, h, d, bt, keep = 8, 2, 128, 16, 9
    b = ref.batch(rng, [1, 2, 30], [900, 700, 400], bt)
    g = on_gpu(b)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    batch = make_batch(dev, g)
    dev.DeviceKvBounds(kv, batch).run()
    qs = [rows(rng, b["tokens"], H, d, torch.bfloat16).cuda() for _ in range(2)]
    want = []
    for q in qs:
        lists = run_select(dev, kv, q, g, keep, 1, 1)
        want.append((lists, run_selected(dev, kv, q, g, lists, 0.1)[0]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lists = run_select(dev, kv, qs[0], g, keep, 1, 1, stream=side)
    assert torch.equal(lists, want[0][0])
    assert torch.equal(run_selected(dev, kv, qs[0], g, lists, 0.1, stream=side)[0], want[0][1])
    made, w1, w2 = [], None, None
    for q in qs:
        lists, out = torch.zeros_like(want[0][0]), torch.zeros_like(q)
        ops = [dev.DeviceKvBounds(kv, batch), dev.DeviceKvSelect(kv, batch, q, lists, 1, 1, workspace=w1),
               dev.DeviceSelectedAttention(kv, batch, q, lists, out, 0.1, workspace=w2)]
        w1, w2 = ops[1].workspace, ops[2].workspace
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for op in ops:
                op.run()
        made.append((graph, ops, lists, out))
    for _ in range(3):
        for k in (0, 1, 1, 0):
            graph, _, lists, out = made[k]
            lists.fill_(-5)
            out.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(lists, want[k][0]) and torch.equal(out, want[k][1])
    kv.check()
