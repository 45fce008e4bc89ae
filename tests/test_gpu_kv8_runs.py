"""cascade_kv_append over batches of short and of long runs, few and many: the
codes and scales are the reference's whichever way the work is divided."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_kv8 import make_batch, on_gpu, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


@pytest.mark.parametrize("n,low,high", [(512, 1, 1), (513, 1, 1), (900, 0, 2), (2048, 1, 1), (30, 14, 18), (33, 15, 17),
                                        (70, 0, 15), (2, 256, 257), (5, 0, 511), (40, 1, 60)])
@pytest.mark.parametrize("bt", [16, 64])
def test_runs(dev, n, low, high, bt):
    rng = np.random.default_rng(n + bt)
    h, d = 3, 64
    counts = rng.integers(low, high + 1, n)
    b = ref.batch(rng, counts, counts + rng.integers(0, 40, n), bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt, spread=3)
    k, v = (rows(rng, b["tokens"], h, d, torch.bfloat16, 2) for _ in range(2))
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
    dev.DeviceKvAppend(kv, make_batch(dev, on_gpu(b)), None, k.cuda(), v.cuda()).run()
    kv.check()
    for side, x in enumerate((k, v)):
        val, sc, _, _ = ref.append(pool[0, side], x.to(ref.F64), b, h, d, bt, side)
        got = kv.pool[0, side].cpu()
        assert torch.equal(ref.scales_of(got, h, d, bt).to(ref.F64), sc)
        assert torch.equal(ref.codes_of(got, h, d, bt, side).view(ref.E4M3).float().to(ref.F64), val)
