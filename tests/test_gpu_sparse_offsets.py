"""Bounds, selections and attention over them where a batch's offsets fall
somewhere: requests before are right, and nothing depends on the workspace."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests import sparse_ref as sref
from tests.test_gpu_kv8 import check_attention, make_batch, on_gpu, rows
from tests.test_gpu_sparse import make_pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


FALLS = ["row to the first", "row into the one before", "row far ahead", "tokens to the first", "tokens back"]


def fallen(fault, chunk):
    """A batch of four requests, and the same with offsets that fall at the
    second one."""
    rng = np.random.default_rng(40)
    counts = [2, 3, 2, 1] if not chunk else [70, 3, 90, 1]
    b = ref.batch(rng, counts, [3000, 200, 900, 700], 16)
    bad = {k: v.clone() if torch.is_tensor(v) else v for k, v in b.items()}
    bad["most"] = b["tokens"]  # or a request that has others' tokens is out of the domain for that alone
    if fault == "row to the first":
        bad["rows"][2] = 0
    elif fault == "row into the one before":
        bad["rows"][2] = int(b["rows"][1]) - 100
    elif fault == "row far ahead":
        bad["rows"][1] = int(b["rows"][3])
    elif fault == "tokens to the first":
        bad["off"][2] = 0
    else:
        bad["off"][2] = 1
    return rng, b, bad


@pytest.mark.parametrize("chunk", [False, True], ids=["few rows", "many rows"])
@pytest.mark.parametrize("by_tokens", [False, True], ids=["", "by tokens"])
@pytest.mark.parametrize("fault", FALLS)
def test_select(dev, fault, by_tokens, chunk):
    H, h, d, bt, keep = 8, 2, 64, 16, 12
    rng, b, bad = fallen(fault, chunk)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    want = sref.select(pool[0], q, b, h, d, bt, keep, 1, 2)
    pool, g = pool.cuda(), on_gpu(bad)
    results = []
    for fill in (0xff, 0, 0x40):
        kv = dev.DeviceKvPool(pool, h, d, bt, bounds=True)
        got = torch.full(tuple(want.shape), -7, dtype=torch.int32, device="cuda")
        op = dev.DeviceKvSelect(kv, make_batch(dev, g), q.cuda(), got, 1, 2, most_blocks=200 if by_tokens else 0)
        op.workspace.fill_(fill)
        op.run()
        with pytest.raises(RuntimeError):
            kv.check()
        results.append(got.cpu())
    n = int(b["off"][1])
    for got in results:
        assert torch.equal(got, results[0])
        assert torch.equal(got[:n], want[:n]) and (got[n:] == -7).all()


@pytest.mark.parametrize("chunk", [False, True], ids=["few rows", "many rows"])
@pytest.mark.parametrize("whole", [False, True], ids=["", "whole"])
@pytest.mark.parametrize("fault", FALLS)
def test_bounds(dev, fault, whole, chunk):
    h, d, bt = 2, 64, 16
    rng, b, bad = fallen(fault, chunk)
    pool = make_pool(rng, 1, b, h, d, bt)
    want = sref.bounds_of(pool[0], dict(b, n=1), h, d, bt, whole)  # the first request's
    if fault == "row far ahead":
        want = {}  # its row reaches over others' blocks: it is theirs too
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    dev.DeviceKvBounds(kv, make_batch(dev, on_gpu(bad)), whole).run()
    with pytest.raises(RuntimeError):
        kv.check()
    upper, lower = sref.bounds_in(kv.pool[0].cpu(), h, d, bt)
    for slot, (u, l) in want.items():
        assert np.array_equal(upper[slot], u) and np.array_equal(lower[slot], l), slot


@pytest.mark.parametrize("keep", [12, 5000])  # the second is cut into parts
@pytest.mark.parametrize("fault", FALLS)
def test_selected_attention(dev, fault, keep):
    H, h, d, bt = 8, 2, 64, 16
    rng, b, bad = fallen(fault, False)
    pool = make_pool(rng, 1, b, h, d, bt)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    lists = torch.full((b["tokens"], h, keep), -1, dtype=torch.int32)
    lists[..., :10] = torch.arange(10)
    e = sref.attend(pool[0], q, b, lists, h, d, bt, 0.2)
    n = int(b["off"][1])
    results = []
    for fill in (0xff, 0x40):
        kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
        out = torch.full(tuple(q.shape), 7.0, dtype=q.dtype, device="cuda")
        lse = torch.full(tuple(q.shape[:2]), 7.0, device="cuda")
        op = dev.DeviceSelectedAttention(kv, make_batch(dev, on_gpu(bad)), q.cuda(), lists.cuda(), out, 0.2, lse=lse)
        op.workspace.fill_(fill)
        op.run()
        with pytest.raises(RuntimeError):
            kv.check()
        part = {k: v[:n] for k, v in e.items()}
        check_attention((out[:n].cpu(), lse[:n].cpu(), None), part, "bf16", d, 0)
        results.append((out, lse))
    assert all(torch.equal(x, y) for x, y in zip(*results))
