"""Key bounds of requests in tables of very many entries."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests import sparse_ref as sref
from tests.test_gpu_kv8 import make_batch, on_gpu
from tests.test_gpu_sparse import make_pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


@pytest.mark.parametrize("entries", [1 << 25, 1 << 27])
def test_whole_bounds_of_a_long_table(dev, entries):
    """More entries than a launch of four to a workgroup takes."""
    rng = np.random.default_rng(36)
    h, d, bt = 3, 64, 16
    b = ref.batch(rng, [0, 2, 0], [90, 500, 33], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    want = sref.bounds_of(pool[0], b, h, d, bt, True)
    g, first = on_gpu(b), int(b["rows"][2])
    gap = torch.full((entries,), -1, dtype=torch.int32, device="cuda")
    g["slots"] = torch.cat([g["slots"][:first], gap, g["slots"][first:]])
    g["rows"] = torch.cat([g["rows"][:2], g["rows"][2:] + entries])
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    dev.DeviceKvBounds(kv, make_batch(dev, g), whole=True).run()
    kv.check()
    upper, lower = sref.bounds_in(kv.pool[0].cpu(), h, d, bt)
    for slot, (u, l) in want.items():
        assert np.array_equal(upper[slot], u) and np.array_equal(lower[slot], l)
