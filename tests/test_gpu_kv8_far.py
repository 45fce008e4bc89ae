"""The 8-bit cache in a pool whose slots, sides and layers lie more than 2^32
bytes apart (tolerances of tests/test_gpu_kv8.py)."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_kv8 import check_attention, make_batch, on_gpu, rows, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


@pytest.mark.parametrize("counts,lengths", [([3, 1], [37, 20]), ([80], [90])], ids=["few", "tiles"])
def test_far_slots(dev, counts, lengths):
    rng = np.random.default_rng(1)
    H, h, d, bt = 4, 2, 64, 16
    b = ref.batch(rng, counts, lengths, bt)
    near = ref.random_pool(rng, 2, b["pool"], h, d, bt)
    size = ref.chunk_bytes(h, d, bt)
    gap = (5 << 30) // b["pool"] // 16 * 16  # between slots; sides and layers lie 5 GiB apart
    room = torch.empty(4 * b["pool"] * gap, dtype=torch.uint8, device="cuda")
    far = room.view(2, 2, b["pool"], gap)
    far[..., :size] = near.cuda()
    g = on_gpu(b)
    k, v = (rows(rng, b["tokens"], h, d, torch.bfloat16).cuda() for _ in range(2))
    pools = []
    for pool in (near.cuda(), far):
        kv = dev.DeviceKvPool(pool, h, d, bt)
        dev.DeviceKvAppend(kv, make_batch(dev, g), None, k, v, layer=1).run()
        kv.check()
        pools.append(pool)
    assert torch.equal(pools[1][..., :size], pools[0])
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    e = ref.attend(pools[0][1].cpu(), q, b, h, d, bt, 0.2, 0.0, 2)
    got = run_attention(dev, far, q.cuda(), g, h, d, bt, 0.2, 0.0, 2, layer=1)
    check_attention(got, e, "bf16", d, 2)
    want = run_attention(dev, pools[0], q.cuda(), g, h, d, bt, 0.2, 0.0, 2, layer=1)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
