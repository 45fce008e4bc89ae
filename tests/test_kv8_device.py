"""The 8-bit cache's Python classes without a GPU: what they hand to the library
and what they refuse before they do."""
import os

import pytest
import torch

from paper_2608_06557_amd import cascade as cx
from paper_2608_06557_amd import device


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(cx.LIB_PATH):
        from paper_2608_06557_amd import build
        build.build()
    return cx.load()


def i32(*a, **kw):
    return torch.tensor(a, dtype=torch.int32, **kw)


def pool():
    return device.DeviceKvPool(torch.zeros(1, 2, 3, 16 * 64 + 16, dtype=torch.uint8), 1, 64, 16)


def test_weights_of_an_empty_table_are_not_asked_for():
    """An empty tensor has no address, which the library would refuse."""
    b = device.KvBatch(i32(0, 2), i32(0), i32(0, 0), i32(), 2, 2)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    op = device.DeviceAttention(pool(), b, q, q, 0.1, block_weight=torch.zeros(0), weight_window=3)
    assert op.c_args.weight_window == 0 and not op.c_args.block_weight
    b = device.KvBatch(i32(0, 2), i32(2), i32(0, 1), i32(1), 2, 2)
    op = device.DeviceAttention(pool(), b, q, q, 0.1, block_weight=torch.zeros(1), weight_window=3)
    assert op.c_args.weight_window == 3 and op.c_args.block_weight


def test_tensors_of_another_device_are_refused():
    kv, elsewhere = pool(), torch.device("meta")
    parts = (i32(0, 2), i32(2), i32(0, 1), i32(1))
    for i in range(4):
        with pytest.raises(ValueError):
            device.KvBatch(*[t.to(elsewhere) if j == i else t for j, t in enumerate(parts)], 2, 2)
    b, far = device.KvBatch(*parts, 2, 2), device.KvBatch(*[t.to(elsewhere) for t in parts], 2, 2)
    q, k = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    args = (q, k, k, q, i32(0, 1), torch.zeros(32, dtype=torch.int64))
    device.DeviceKvAppend(kv, b, *args)
    for i in range(6):
        with pytest.raises(ValueError):
            device.DeviceKvAppend(kv, b, *[t.to(elsewhere) if j == i else t for j, t in enumerate(args)])
    with pytest.raises(ValueError):
        device.DeviceKvAppend(kv, far, *args)
    more = dict(lse=torch.zeros(2, 4), block_weight=torch.zeros(1), weight_window=1,
                workspace=torch.zeros(256, dtype=torch.uint8))
    device.DeviceAttention(kv, b, q, q, 0.1, **more)
    for bad in (dict(q=q.to(elsewhere)), dict(out=q.to(elsewhere)), dict(lse=more["lse"].to(elsewhere)),
                dict(block_weight=more["block_weight"].to(elsewhere)),
                dict(workspace=more["workspace"].to(elsewhere)), dict(batch=far)):
        given = dict(batch=b, q=q, out=q, scale=0.1, **more)
        given.update(bad)
        with pytest.raises(ValueError):
            device.DeviceAttention(kv, **given)
    args = (parts[1], parts[2], parts[3], torch.zeros(1), i32(1))
    device.DeviceKvEvict(16, *args)
    for i in range(5):
        with pytest.raises(ValueError):
            device.DeviceKvEvict(16, *[t.to(elsewhere) if j == i else t for j, t in enumerate(args)])


def test_an_eviction_is_checked_as_the_pool_is():
    op = device.DeviceKvEvict(16, i32(2), i32(0, 1), i32(1), torch.zeros(1), i32(1))
    op.check()
    for code in (cx.EINVAL, cx.ENOSPC):
        op.status.fill_(code)
        with pytest.raises(RuntimeError, match=cx.cascade_strerror(code)):
            op.check()
