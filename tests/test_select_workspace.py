"""The workspace of cascade_kv_select: how it grows, and what the Python class
takes of it (no GPU)."""
import os

import pytest
import torch

from paper_2608_06557_amd import cascade as cx
from paper_2608_06557_amd import device
from tests.test_kv8_sparse_host import FAKE, ROWS, TABLE, batch, fmt, pool


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(cx.LIB_PATH):
        from paper_2608_06557_amd import build
        build.build()
    return cx.load()


def size(f=fmt(), **kw):
    return cx.cascade_kv_select_workspace_bytes(f, batch(**kw))


def test_size():
    one = 4 * (1000 + 16 * 3) * 8
    assert size(n=3, tokens=9, most=1, entries=1000) == one + 256
    assert size(n=3, tokens=9, most=5, entries=1000) == 5 * one + 256
    assert size(n=3, tokens=9, most=500, entries=1000) == 9 * one + 256  # no request has more than all
    assert size(tokens=-1) == 0
    top = 2 ** 31 - 1
    sizes = [size(fmt(h=256), n=2048, tokens=t, most=t, entries=top) for t in (1, 2, 32767, 32768, 32769, top)]
    assert sizes == sorted(sizes) and sizes[-1] < 1 << 57  # and nothing passes 64 bits


def test_smaller_workspaces_are_taken():
    def call(b, w):
        a = cx.Select(cx.BF16, 32, 8, 1, 1, ROWS, 0)  # no place for lists: refused behind the size
        return cx.cascade_kv_select(pool(), 0, fmt(), b, TABLE, a, FAKE, w, 0, 0)

    b = dict(n=3, tokens=600, most=512, entries=1000)
    least = size(**dict(b, most=1))
    assert call(batch(**b), least) == cx.EINVAL and call(batch(**b), least - 1) == cx.ENOSPC
    for empty in (dict(b, tokens=0), dict(b, most=0)):
        assert call(batch(**empty), size(**empty)) == cx.OK
        assert call(batch(**empty), size(**empty) - 1) == cx.ENOSPC


def test_tables_that_no_launch_takes_are_refused():
    a = cx.Select(cx.BF16, 8, 8, 1, 1, ROWS, FAKE)
    got = cx.cascade_kv_select(pool(), 0, fmt(), batch(entries=2 ** 31 - 1), TABLE, a, FAKE, 1 << 60, 0, 0)
    assert got == cx.EINVAL


def test_a_batch_of_decodes_and_a_chunk():
    """127 single tokens beside one chunk of 512 over 84608 blocks: not the
    chunk's rows for each of them."""
    kv = device.DeviceKvPool.empty(1, 1, 8, 64, 16, "cpu", bounds=True)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    b = device.KvBatch(i32(129), i32(128), i32(129), i32(84608), 639, 512)
    q, lists = torch.zeros(639, 8, 64, dtype=torch.bfloat16), i32(639, 8, 16)
    full = cx.cascade_kv_select_workspace_bytes(kv.c_format, b.c_batch)
    assert full > 1400 * 10 ** 6
    op = device.DeviceKvSelect(kv, b, q, lists, most_blocks=2001)
    assert op.workspace.numel() == 256 + (256 + 4 * 639 * 8 * 2016) < 50 * 10 ** 6
    # and no more than without a bound
    few = device.KvBatch(i32(129), i32(128), i32(129), i32(84608), 128, 1)
    for most in (0, 2001, 2 ** 31 - 1):
        op = device.DeviceKvSelect(kv, few, q, lists, most_blocks=most)
        assert op.workspace.numel() == 256 + cx.cascade_kv_select_workspace_bytes(kv.c_format, few.c_batch)


def test_workspaces_by_tokens():
    def call(w, most):
        a = cx.Select(cx.BF16, 32, 8, 1, 1, ROWS, 0, most)  # no place for lists: refused behind the size
        return cx.cascade_kv_select(pool(), 0, fmt(), batch(n=3, tokens=5, most=5, entries=3000), TABLE, a, FAKE, w, 0, 0)

    by_tokens, least = 256 + 4 * 5 * 8 * 112, size(n=3, tokens=5, most=1, entries=3000)
    assert by_tokens < least
    for most in (97, 100, 112):
        assert call(by_tokens, most) == cx.EINVAL and call(by_tokens - 1, most) == cx.ENOSPC
    assert call(by_tokens, 113) == call(by_tokens, 0) == call(least - 1, 2 ** 31 - 1) == cx.ENOSPC
    assert call(1 << 40, -1) == cx.EINVAL


def test_sizes_that_pass_64_bits():
    top = 2 ** 31 - 1
    a = cx.Select(cx.BF16, 256, 8, 1, 1, ROWS, FAKE, top)
    b = batch(n=2048, tokens=top, most=top, entries=top)
    big = pool(chunk=1 << 40, ls=0, ks=0, ss=0)
    assert cx.cascade_kv_select(big, 0, fmt(h=256), b, TABLE, a, FAKE, 1 << 30, 0, 0) != cx.OK
