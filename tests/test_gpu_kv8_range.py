"""cascade_attention of float16 rows over caches whose values float16 does not
hold (tolerances of tests/test_gpu_kv8.py: the codes' values are exact whatever
their scales, so no term is added)."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_kv8 import bounds, check_attention, make_batch, on_gpu, rows, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


def with_infinities(got, want, d):
    """Results that round to infinity as what was wanted, where that is within its
    tolerance of 65520, from which on the type has infinity, or over it."""
    out = got[0].cpu().to(ref.F64)
    may = torch.isinf(out) & (want["out"] * out.sign() + bounds(want, "f16", d, 1.0)[0] >= 65520)
    return torch.where(may, want["out"], out), got[1], got[2]


SHAPES = [([1, 3], [70, 200]), ([9, 1], [130, 33]), ([80, 1], [333, 40]), ([300], [1500])]


@pytest.mark.parametrize("counts,lengths", SHAPES, ids=[str(c[0]) for c in SHAPES])
@pytest.mark.parametrize("d,bt", [(64, 16), (128, 32), (128, 16), (256, 16)])
@pytest.mark.parametrize("side", [0, 1])
@pytest.mark.parametrize("low,high", [(6, 11), (-34, -12), (40, 60)])
def test_scales_out_of_the_types_range(dev, counts, lengths, d, bt, side, low, high):
    """Keys or values of blocks and heads with scales 2^low .. 2^high; for keys
    the scale of the scores makes up for them."""
    if side and low == 40:  # (results would not fit the type)
        low, high = 5, 8
    rng = np.random.default_rng(d + low)
    H, h = 4, 2
    b = ref.batch(rng, counts, lengths, bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    e = rng.integers(low, high + 1, (b["pool"], h))
    n = ref.chunk_bytes(h, d, bt) - 16
    pool[0, side, :, n:n + 4 * h] = torch.from_numpy((2.0 ** e).astype(np.float32)).view(torch.uint8)
    scale = d ** -0.5 * (1.0 if side else 2.0 ** (-6 - (low + high) / 2))
    q = rows(rng, b["tokens"], H, d, torch.float16)
    want = ref.attend(pool[0], q, b, h, d, bt, scale, 0.0, 2)
    got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, scale, 0.0, 2)
    check_attention(with_infinities(got, want, d), want, "f16", d, 2)


@pytest.mark.parametrize("count", [1, 8, 90])
def test_appended_values_at_the_types_end(dev, count):
    """Values of +-65504 round to a code that stands for 65536.  Tokens that do
    not see them keep their results to the bit; those that do get the average."""
    rng = np.random.default_rng(4)
    H, h, d, bt = 4, 2, 128, 16
    b = ref.batch(rng, [count, count], [count + 50, count + 30], bt)
    g = on_gpu(b)
    T = b["tokens"]
    q, k, v = rows(rng, T, H, d, torch.float16), rows(rng, T, h, d, torch.float16), rows(rng, T, h, d, torch.float16)
    start = ref.random_pool(rng, 1, b["pool"], h, d, bt).cuda()
    results = []
    for big in (False, True):
        vv, kk = v.clone(), k.clone()
        if big:  # the last token of request 0
            vv[count - 1, :, ::2], vv[count - 1, :, 1::2] = 65504.0, -65504.0
        kv = dev.DeviceKvPool(start.clone(), h, d, bt)
        dev.DeviceKvAppend(kv, make_batch(dev, g), None, kk.cuda(), vv.cuda()).run()
        kv.check()
        want = ref.attend(kv.pool[0].cpu(), q, b, h, d, bt, 0.05)
        got = run_attention(dev, kv.pool, q.cuda(), g, h, d, bt, 0.05)
        check_attention(got, want, "f16", d, 0)
        assert torch.isfinite(got[0]).all()
        results.append(got[0])
    assert torch.equal(results[0][count:], results[1][count:])  # the other request


def test_rotated_keys_over_the_types_end(dev):
    """Pairs of 65504 turned by an eighth of a circle and scaled: 1.4 * 1.25
    times as large; queries as small as the type allows."""
    rng = np.random.default_rng(5)
    H, h, d, bt = 4, 2, 64, 16
    b = ref.batch(rng, [6], [40], bt)
    g = on_gpu(b)
    k = torch.full((6, h, d), 65504.0, dtype=torch.float16)
    v = rows(rng, 6, h, d, torch.float16)
    q = (rows(rng, 6, H, d, torch.float16).float() * 2.0 ** -18).half()
    freq = torch.full((d // 2,), 1 << 61, dtype=torch.int64, device="cuda")
    pos = torch.tensor([1, 9, 17, 1, 1, 25], dtype=torch.int32, device="cuda")
    kv = dev.DeviceKvPool(ref.random_pool(rng, 1, b["pool"], h, d, bt).cuda(), h, d, bt)
    dev.DeviceKvAppend(kv, make_batch(dev, g), None, k.cuda(), v.cuda(), None, pos, freq, False, 1.25).run()
    kv.check()
    stored = ref.values_of(kv.pool[0, 0].cpu(), h, d, bt, 0)
    assert stored.abs().max() > 110000
    want = ref.attend(kv.pool[0].cpu(), q, b, h, d, bt, 0.7)
    check_attention(run_attention(dev, kv.pool, q.cuda(), g, h, d, bt, 0.7), want, "f16", d, 0)
