"""Block selection where more than 16 query heads read a KV head, whose scores
are taken in parts."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests import sparse_ref as sref
from tests.test_gpu_kv8 import on_gpu, rows
from tests.test_gpu_sparse import make_pool, run_select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


@pytest.mark.parametrize("first", [True, False], ids=["zeros first", "zeros last"])
def test_infinite_scales_over_many_heads(dev, first):
    """Of 40 heads the largest sum is 0 and others' are negative: by an infinite
    K scale that is no number, and the largest, whichever heads come first."""
    rng = np.random.default_rng(30)
    H, h, d, bt, keep = 40, 1, 64, 16, 12
    b = ref.batch(rng, [2], [1600], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    n = ref.chunk_bytes(h, d, bt)
    odd = b["slots"][40:50].long()  # ten blocks whose keys are all below 0
    for s in range(2):
        pool[0, s, odd, n:n + h * d] = 0xfb
    pool[0, 0, odd, n - 16:n - 12] = torch.tensor([float("inf")]).view(torch.uint8)
    q = rows(rng, 2, H, d, torch.bfloat16).abs() + 0.5
    q[:, slice(0, 16) if first else slice(32, 40)] = 0
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    got = run_select(dev, kv, q.cuda(), on_gpu(b), keep, 1, 1).cpu()
    assert (got == torch.tensor([0] + list(range(40, 50)) + [99])).all()
