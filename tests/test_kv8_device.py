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
