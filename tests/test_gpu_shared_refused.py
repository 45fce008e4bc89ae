"""What cascade_attention_shared leaves alone: rows of requests and groups that
it refuses, whatever the workspace holds, and good groups beside bad ones
(tolerances of tests/test_gpu_kv8.py)."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_kv8 import check_attention, make_batch, on_gpu, rows
from tests.test_gpu_shared_attention import shared_batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


def attend_over(dev, pool, q, b, h, d, bt, most, workspace=None):
    """(out, lse, op) into rows of 7, by a workspace that holds what it did."""
    g = on_gpu(b)
    kv = dev.DeviceKvPool(pool, h, d, bt)
    out = torch.full(tuple(q.shape), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(tuple(q.shape[:2]), 7.0, device="cuda")
    op = dev.DeviceSharedAttention(kv, make_batch(dev, g), g["leader"], g["shared"], most, q, out, 0.2, lse=lse,
                                   workspace=workspace)
    op.run()
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), op


# what is wrong, and the rows that are left: of requests 0 to 5 rows 0, 1, 2, 3 and 4, 5, 6; groups 0 1, 2 3 4 and 5
FAULTS = {
    "length odd": [2, 3, 4, 5], "group": [2, 3, 4, 5], "middle": [3, 4], "last": [2, 3, 4, 5],
    "leader negative": [3, 4, 5], "leader apart": [5], "alone": [6], "offsets": [2, 3, 4, 5], "nothing": [],
}


@pytest.mark.parametrize("heads", [(4, 2), (32, 1)], ids=["few rows", "row tiles"])
@pytest.mark.parametrize("fault", FAULTS)
def test_refused_rows_stay(dev, fault, heads):
    (H, h), d, bt = heads, 64, 16
    rng = np.random.default_rng(12)
    b = shared_batch(rng, [(32, [(1, 4), (1, 9)]), (64, [(1, 5), (2, 30), (1, 1)]), (16, [(1, 3)])], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q, other = (rows(rng, b["tokens"], H, d, torch.bfloat16) for _ in range(2))
    e = ref.attend(pool[0], q, b, h, d, bt, 0.2)
    pool = pool.cuda()
    # an earlier call's states and parts, of other queries
    before = attend_over(dev, pool, other.cuda(), b, h, d, bt, b["most_shared"])[2].workspace.clone()
    most = b["most_shared"]
    if fault == "length odd":
        b["shared"][2] = 40
    elif fault == "group":
        most = 3
    elif fault == "middle":
        b["len"][3] = 1 << 20
    elif fault == "last":
        b["len"][4] = 1 << 20
    elif fault == "leader negative":
        b["leader"][3] = -1
    elif fault == "leader apart":
        b["leader"][4] = 0
    elif fault == "alone":
        b["len"][5] = 1 << 20
    elif fault == "offsets":  # the next one has more new tokens than any may have
        b["off"][4] = 2
    results = []
    for fill in (lambda w: w.copy_(before), lambda w: w.zero_(), lambda w: w.fill_(0xff), lambda w: w.fill_(1)):
        w = before.clone()
        fill(w)
        results.append(attend_over(dev, pool, q.cuda(), b, h, d, bt, most, w))
    out, lse, op = results[0]
    if fault == "nothing":
        op.kv.check()
    else:
        with pytest.raises(RuntimeError):
            op.kv.check()
    left = FAULTS[fault]
    good = [t for t in range(b["tokens"]) if t not in left]
    for out, lse, _ in results:
        assert (out[left] == 7).all() and (lse[left] == 7).all()
        part = {k: v[good] for k, v in e.items() if k != "weight"}
        check_attention((out[good], lse[good], None), part, "bf16", d, 0)
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])


# leaders that name a request apart from them, or no first one; the rows that are left, and the groups beside
APART = {
    "behind one": ([0, 1, 0, 0], [2, 3], []),
    "behind a group": ([0, 0, 2, 2, 0, 0], [4, 5], [(0, 2), (2, 4)]),
    "of a member": ([0, 0, 1, 1], [2, 3], [(0, 2)]),
    "of the next": ([1, 1, 1, 3], [0], [(1, 3)]),
    "of a group far behind": ([0] * 70 + [70] * 70 + [0] * 70, list(range(140, 210)), [(0, 70), (70, 140)]),
    "across waves": ([0] * 30 + [29] * 100 + [130] * 140 + [127] * 30, list(range(30, 130)) + list(range(270, 300)),
                     [(0, 30), (130, 270)]),
}


@pytest.mark.parametrize("case", APART)
def test_groups_that_are_no_neighbours_leave_others_alone(dev, case):
    """Requests that name a first one they do not follow are refused, and what
    lies between is right."""
    leader, left, groups = APART[case]
    rng = np.random.default_rng(13)
    H, h, d, bt, n = 4, 2, 64, 16, len(leader)
    shared = 3200 if n < 9 else 256
    b = shared_batch(rng, [(0, [(1, shared + 800 if n < 9 else shared + 60)])] * n, bt)
    for first, end in groups:
        at = int(b["rows"][first])
        for i in range(first + 1, end):
            row = int(b["rows"][i])
            b["slots"][row:row + shared // bt] = b["slots"][at:at + shared // bt].clone()
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q = rows(rng, n, H, d, torch.bfloat16)
    e = ref.attend(pool[0], q, b, h, d, bt, 0.2)
    b["leader"] = torch.tensor(leader, dtype=torch.int32)
    b["shared"][:] = shared
    out, lse, op = attend_over(dev, pool.cuda(), q.cuda(), b, h, d, bt, n)
    with pytest.raises(RuntimeError):
        op.kv.check()
    good = [t for t in range(n) if t not in left]
    part = {k: v[good] for k, v in e.items() if k != "weight"}
    check_attention((out[good], lse[good], None), part, "bf16", d, 0)
    assert (out[left] == 7).all() and (lse[left] == 7).all()


def test_a_group_whose_offsets_fall_inside(dev):
    """Its rows end before the first request's do: what they miss is left, by
    whatever workspace (rows that two requests have are either's)."""
    rng = np.random.default_rng(14)
    H, h, d, bt = 4, 2, 64, 16
    b = shared_batch(rng, [(64, [(5, 20), (1, 30), (2, 40)]), (0, [(4, 30)])], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q, other = (rows(rng, b["tokens"], H, d, torch.bfloat16) for _ in range(2))
    e = ref.attend(pool[0], q, b, h, d, bt, 0.2)
    pool = pool.cuda()
    before = attend_over(dev, pool, other.cuda(), b, h, d, bt, b["most_shared"])[2].workspace.clone()
    b["off"] = torch.tensor([0, 5, 2, 4, 12], dtype=torch.int32)  # the second is refused, the third has rows 2 and 3
    b["len"][3] = 1 << 20  # and the last, which would have row 4
    for fill in (lambda w: w.copy_(before), lambda w: w.fill_(0xff), lambda w: w.fill_(2)):
        w = before.clone()
        fill(w)
        out, lse, op = attend_over(dev, pool, q.cuda(), b, h, d, bt, b["most_shared"], w)
        with pytest.raises(RuntimeError):
            op.kv.check()
        part = {k: v[:2] for k, v in e.items() if k != "weight"}
        check_attention((out[:2], lse[:2], None), part, "bf16", d, 0)
        assert (out[4:] == 7).all() and (lse[4:] == 7).all()
