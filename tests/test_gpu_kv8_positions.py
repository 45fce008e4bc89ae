"""cascade_kv_append where positions are negative or requests without new
tokens are outside the domain: what is reported, and what is left as it was."""
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


@pytest.mark.parametrize("inter", [False, True])
def test_negative_positions_are_not_written(dev, inter):
    """A query with a negative position keeps its place in q_out, and the new
    tokens of a block with one are not written, keys and values; all others
    are, as without it."""
    rng = np.random.default_rng(1)
    H, h, d, bt = 4, 2, 64, 16
    b = ref.batch(rng, [20, 1, 3], [24, 40, 16], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    x = rows(rng, b["tokens"], H + 2 * h, d, torch.bfloat16).cuda()
    freq = torch.from_numpy(ref.fixed(ref.theta("plain", 64, 1e4)[0]).view(np.int64).copy()).cuda()
    g = on_gpu(b)
    # new token 13 of request 0 is its 18th cached token, in its second block; token 20 is request 1's
    bad_tokens, bad_slots = [13, 20], [int(b["slots"][1]), int(b["slots"][int(b["rows"][1]) + 2])]
    got = []
    for bad in ([], bad_tokens):
        pos = torch.arange(b["tokens"], dtype=torch.int32) * 31
        pos[bad] = torch.tensor([-1, -2 ** 31], dtype=torch.int32)[:len(bad)]
        kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
        q_out = torch.full((b["tokens"], H, d), 7.0, dtype=torch.bfloat16, device="cuda")
        dev.DeviceKvAppend(kv, make_batch(dev, g), x[:, :H], x[:, H:H + h], x[:, H + h:], q_out, pos.cuda(), freq,
                           inter).run()
        if bad:
            with pytest.raises(RuntimeError):
                kv.check()
        else:
            kv.check()
        got.append((q_out, kv.pool[0]))
    fine = [t for t in range(b["tokens"]) if t not in bad_tokens]
    assert torch.equal(got[1][0][fine], got[0][0][fine])
    assert (got[1][0][bad_tokens] == 7.0).all()
    for slot in range(b["pool"]):
        want = pool[0, :, slot].cuda() if slot in bad_slots else got[0][1][:, slot]
        assert torch.equal(got[1][1][:, slot], want), slot


@pytest.mark.parametrize("fault", ["length", "long", "row", "row end", "offsets"])
@pytest.mark.parametrize("at", [0, 1, 3])
def test_bad_requests_without_new_tokens_are_reported(dev, fault, at):
    rng = np.random.default_rng(2)
    h, d, bt = 2, 64, 16
    counts = [1, 1, 2, 1]
    counts[at] = 0
    b = ref.batch(rng, counts, [20, 21, 22, 30], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    k = rows(rng, b["tokens"], h, d, torch.bfloat16).cuda()
    g = on_gpu(b)
    if fault == "length":
        g["len"][at] = -1
    elif fault == "long":
        g["len"][at] = 33
    elif fault == "row":
        g["rows"][at] = -1
    elif fault == "row end":
        g["rows"][at + 1] = 1 << 30
    else:
        g["off"][at + 1] -= 1
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
    dev.DeviceKvAppend(kv, make_batch(dev, g), None, k, k).run()
    with pytest.raises(RuntimeError):
        kv.check()
    if fault in ("length", "long"):  # otherwise a neighbour is bad too
        clean = dev.DeviceKvPool(pool.cuda(), h, d, bt)
        dev.DeviceKvAppend(clean, make_batch(dev, on_gpu(b)), None, k, k).run()
        clean.check()
        assert torch.equal(kv.pool, clean.pool)
