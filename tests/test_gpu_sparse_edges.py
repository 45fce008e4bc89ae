"""Attention over shared prefixes and selected blocks, bounds and selections
where sizes, strides and places are at their ends (tolerances of
tests/test_gpu_kv8.py)."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests import sparse_ref as sref
from tests.test_gpu_kv8 import check_attention, make_batch, on_gpu, rows
from tests.test_gpu_shared_attention import run_shared, shared_batch
from tests.test_gpu_sparse import make_pool, random_lists, run_select, run_selected

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


@pytest.mark.parametrize("name,d", [("bf16", 128), ("f16", 256), ("f16", 64)])
def test_most_requests_in_groups_of_whole_tiles(dev, name, d):
    """2048 requests, a group of over 1024 rows among them: the largest lists
    beside the largest tiles."""
    rng = np.random.default_rng(5)
    groups = [(32, [(1, 1 + i % 9) for i in range(640)]), (0, [(1, 3)] * 408), (16, [(1, 2)] * 2), (48, [(1, 5)] * 998)]
    b = shared_batch(rng, groups, 16)
    pool = ref.random_pool(rng, 1, b["pool"], 1, d, 16)
    q = rows(rng, b["tokens"], 2, d, {"bf16": torch.bfloat16, "f16": torch.float16}[name])
    e = ref.attend(pool[0], q, b, 1, d, 16, 0.1)
    check_attention(run_shared(dev, pool.cuda(), q.cuda(), on_gpu(b), 1, d, 16, 0.1), e, name, d, 0)


def test_rows_behind_the_last_request_stay(dev):
    """A padded batch: rows that no request has are neither read nor written."""
    rng = np.random.default_rng(6)
    H, h, d, bt, T = 8, 2, 128, 16, 9
    b = shared_batch(rng, [(320, [(1, 9), (2, 30)]), (0, [(3, 20)])], bt)
    n = b["tokens"]
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, T, H, d, torch.bfloat16)
    q[n:] = float("nan")
    g = dict(on_gpu(b), tokens=T)
    e = ref.attend(pool[0], q[:n], b, h, d, bt, 0.1)
    out, lse, _ = run_shared(dev, pool.cuda(), q.cuda(), g, h, d, bt, 0.1)
    check_attention((out[:n], lse[:n], None), e, "bf16", d, 0)
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    before = kv.pool.clone()
    dev.DeviceKvBounds(kv, make_batch(dev, g)).run()
    kv.check()
    changed = (kv.pool != before).flatten(3).any(3)[0].any(0).nonzero().flatten().tolist()
    tails = {int(b["slots"][int(b["rows"][i]) + k]) for i in range(3)
             for k in range(int(b["len"][i] - (b["off"][i + 1] - b["off"][i])) // bt, (int(b["len"][i]) - 1) // bt + 1)}
    assert set(changed) <= tails
    for keep in (3, 30):
        got = run_select(dev, kv, q.cuda(), g, keep, 1, 1)
        want = sref.select(kv.pool[0].cpu(), q[:n], b, h, d, bt, keep, 1, 1)
        assert torch.equal(got[:n].cpu(), want) and (got[n:] == -7).all()
        lists = got.clone()
        lists[n:] = 1 << 30
        out, lse, _ = run_selected(dev, kv, q.cuda(), g, lists, 0.1)
        e = sref.attend(kv.pool[0].cpu(), q[:n], b, want, h, d, bt, 0.1)
        check_attention((out[:n], lse[:n], None), e, "bf16", d, 0)
        assert (out[n:] == 7).all() and (lse[n:] == 7).all()


def test_strided_rows(dev):
    """Rows inside a fused projection, heads far apart, every second head of a
    wider output: the same results as of rows side by side."""
    rng = np.random.default_rng(7)
    H, h, d, bt = 8, 2, 64, 32
    b = shared_batch(rng, [(640, [(1, 9), (2, 30), (40, 41)]), (0, [(3, 300)])], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    g = on_gpu(b)
    q = rows(rng, b["tokens"], H, d, torch.float16).cuda()
    wide = torch.full((H, b["tokens"], d + 24), 3.0, dtype=q.dtype, device="cuda")
    qs = wide.transpose(0, 1)[..., 8:8 + d]
    qs.copy_(q)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    batch = make_batch(dev, g)
    lists = run_select(dev, kv, q, g, 5, 1, 1)
    assert torch.equal(run_select(dev, kv, qs, g, 5, 1, 1), lists)
    for run in (lambda q, out: dev.DeviceSharedAttention(kv, batch, g["leader"], g["shared"], b["most_shared"], q, out, 0.1),
                lambda q, out: dev.DeviceSelectedAttention(kv, batch, q, lists, out, 0.1)):
        near = torch.zeros_like(q)
        run(q, near).run()
        room = torch.full((b["tokens"], 2 * H, d), 5.0, dtype=q.dtype, device="cuda")
        run(qs, room[:, ::2]).run()
        torch.cuda.synchronize()
        assert torch.equal(room[:, ::2], near) and (room[:, 1::2] == 5).all()
    kv.check()


def test_far_slots_and_scores(dev):
    """Slots, sides and layers more than 2^32 bytes apart, and scores of
    requests whose places in the workspace are."""
    rng = np.random.default_rng(1)
    H, h, d, bt = 4, 2, 64, 16
    b = shared_batch(rng, [(64, [(1, 20), (1, 9)]), (0, [(2, 90)])], bt)
    near = make_pool(rng, 2, b, h, d, bt)
    size = near.shape[-1]
    gap = (5 << 30) // b["pool"] // 16 * 16
    far = torch.empty(4 * b["pool"] * gap, dtype=torch.uint8, device="cuda").view(2, 2, b["pool"], gap)
    far[..., :size] = near.cuda()
    g = on_gpu(b)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16).cuda()
    results = []
    for pool in (near.cuda(), far):
        kv = dev.DeviceKvPool(pool, h, d, bt, bounds=True)
        dev.DeviceKvBounds(kv, make_batch(dev, g), whole=True, layer=1).run()
        lists = run_select(dev, kv, q, g, 4, 1, 1, layer=1)
        out, lse, _ = run_selected(dev, kv, q, g, lists, 0.2, layer=1)
        shared = run_shared(dev, pool, q, g, h, d, bt, 0.2, layer=1)
        results.append((pool[..., :size].clone(), lists, out, lse, *shared[:2]))
    assert all(torch.equal(x, y) for x, y in zip(*results))
    want = sref.select(results[0][0][1].cpu(), q.cpu(), b, h, d, bt, 4, 1, 1)
    assert torch.equal(results[0][1].cpu(), want)
    # as many new tokens as a batch might have, and rows far along the table
    slack = 1 << 18
    c = {k: v.clone() if torch.is_tensor(v) else v for k, v in b.items()}
    c["rows"] += slack
    c["rows"][0] = 0
    c["slots"] = torch.cat([c["slots"][:int(b["rows"][1])], torch.zeros(slack, dtype=torch.int32), c["slots"][int(b["rows"][1]):]])
    c["most"] = 2100
    assert len(c["slots"]) * c["most"] * h * 4 > 1 << 32
    kv = dev.DeviceKvPool(results[0][0], h, d, bt, bounds=True)
    assert torch.equal(run_select(dev, kv, q, on_gpu(c), 4, 1, 1, layer=1), results[0][1])


def test_one_workspace_for_batches_of_any_size(dev):
    """Made for the largest batch, used by smaller ones in turn."""
    rng = np.random.default_rng(8)
    H, h, d, bt = 4, 2, 64, 16
    sizes = [[(1, 5000)] * 2, [(1, 40)] * 60, [(3, 700), (1, 9)]]
    batches = [shared_batch(rng, [(160, m)], bt) for m in sizes]
    spaces = {}
    for turn in range(2):
        for b in batches:
            pool = make_pool(rng, 1, b, h, d, bt)
            sref.random_bounds(rng, pool[0], h, d, bt)
            g = on_gpu(b)
            q = rows(rng, b["tokens"], H, d, torch.bfloat16)
            kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
            batch = make_batch(dev, g)
            out, out2 = torch.zeros_like(q).cuda(), torch.zeros_like(q).cuda()
            lists = torch.zeros(b["tokens"], h, 200, dtype=torch.int32, device="cuda")
            made = [lambda w: dev.DeviceSharedAttention(kv, batch, g["leader"], g["shared"], b["most_shared"], q.cuda(), out, 0.2, workspace=w),
                    lambda w: dev.DeviceKvSelect(kv, batch, q.cuda(), lists, 1, 1, workspace=w),
                    lambda w: dev.DeviceSelectedAttention(kv, batch, q.cuda(), lists, out2, 0.2, workspace=w)]
            for k, make in enumerate(made):
                if turn:
                    make(spaces[k]).run()
                else:
                    op = make(None)
                    if k not in spaces or op.workspace.numel() > spaces[k].numel():
                        spaces[k] = op.workspace
            torch.cuda.synchronize()
            kv.check()
            if not turn:
                continue
            e = ref.attend(pool[0], q, b, h, d, bt, 0.2)
            check_attention((out, None, None), e, "bf16", d, 0)
            want = sref.select(pool[0], q, b, h, d, bt, 200, 1, 1)
            assert torch.equal(lists.cpu(), want)
            check_attention((out2, None, None), sref.attend(pool[0], q, b, want, h, d, bt, 0.2), "bf16", d, 0)


def test_nothing_new_and_nothing_cached(dev):
    """Batches of no request, without new tokens, and without cached ones."""
    rng = np.random.default_rng(9)
    H, h, d, bt = 4, 2, 64, 16
    for counts, lengths in (([], []), ([0, 0], [40, 0]), ([2, 1], [0, 0]), ([3], [1])):
        b = shared_batch(rng, [(0, [(c, l)]) for c, l in zip(counts, lengths)], bt) if counts else dict(
            ref.batch(rng, [0], [0], bt), n=0)
        if not counts:
            b.update(off=torch.zeros(1, dtype=torch.int32), len=torch.zeros(0, dtype=torch.int32),
                     rows=torch.zeros(1, dtype=torch.int32), leader=torch.zeros(0, dtype=torch.int32),
                     shared=torch.zeros(0, dtype=torch.int32), most_shared=0)
        pool = make_pool(rng, 1, b, h, d, bt)
        sref.random_bounds(rng, pool[0], h, d, bt)
        g, q = on_gpu(b), rows(rng, max(b["tokens"], 1), H, d, torch.bfloat16)
        kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
        for whole in (False, True):
            dev.DeviceKvBounds(kv, make_batch(dev, g), whole).run()
        n = b["tokens"]
        out, lse, _ = run_shared(dev, pool.cuda(), q.cuda(), g, h, d, bt, 0.2)
        lists = run_select(dev, kv, q.cuda(), g, 4, 1, 1)
        out2, lse2, _ = run_selected(dev, kv, q.cuda(), g, lists, 0.2)
        if n:
            e = ref.attend(pool[0], q, b, h, d, bt, 0.2)
            check_attention((out[:n], lse[:n], None), e, "bf16", d, 0)
            check_attention((out2[:n], lse2[:n], None), e, "bf16", d, 0)
            assert torch.equal(lists.cpu(), sref.select(kv.pool[0].cpu(), q, b, h, d, bt, 4, 1, 1))
        else:
            assert (out == 7).all() and (out2 == 7).all() and (lists == -7).all()


@pytest.mark.parametrize("scale,cap", [(8.0, 0.0), (0.0, 0.0), (-0.4, 0.0), (0.1, 100.0), (-0.1, 100.0), (3.0, 2.0)])
@pytest.mark.parametrize("H", [8, 32])
def test_selected_peaked_flat_and_capped_scores(dev, H, scale, cap):
    """Up to 8 heads and over 8 of a KV head; a NaN query spoils its own row only."""
    rng = np.random.default_rng(4)
    h, d, bt = 2, 128, 16
    b = ref.batch(rng, [1, 2], [700, 333], bt)
    pool = make_pool(rng, 1, b, h, d, bt, spread=0)
    q = rows(rng, 3, H, d, torch.float16)
    lists = random_lists(rng, b, h, bt, 30, 0.0)
    e = sref.attend(pool[0], q, b, lists, h, d, bt, scale, cap)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    base = run_selected(dev, kv, q.cuda(), on_gpu(b), lists.cuda(), scale, cap)
    check_attention(base, e, "f16", d, 0)
    q[1, 3, 5] = float("nan")
    got = run_selected(dev, kv, q.cuda(), on_gpu(b), lists.cuda(), scale, cap)
    bad = torch.zeros(3, H, dtype=torch.bool)
    bad[1, 3] = True
    if scale:  # of none of the query nothing is left
        assert torch.isnan(got[0][1, 3]).all()
    assert torch.equal(got[0].cpu()[~bad], base[0].cpu()[~bad])


@pytest.mark.parametrize("heads", [8, 40], ids=["", "wide"])
@pytest.mark.parametrize("counts", [[3, 2], [3, 290]], ids=["few rows", "many rows"])
def test_scores_that_are_no_numbers_are_the_largest(dev, counts, heads):
    """The first of the blocks whose K scale is NaN, beside those that are
    listed anyway."""
    rng = np.random.default_rng(27)
    h, d, bt, keep = 8, 64, 16, 20
    b = ref.batch(rng, counts, [2000, 5100], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    n = ref.chunk_bytes(h, d, bt) - 32
    scale = pool[0, 0, :, n:n + 32].contiguous().view(torch.float32)
    for i in range(2):
        scale[b["slots"][int(b["rows"][i]) + 10:int(b["rows"][i]) + 50].long()] = float("nan")
    pool[0, 0, :, n:n + 32] = scale.view(torch.uint8)
    q = rows(rng, b["tokens"], heads if heads == 8 else 8 * heads, d, torch.bfloat16)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    got = run_select(dev, kv, q.cuda(), on_gpu(b), keep, 1, 2).cpu()
    for i in range(2):
        for j in range(counts[i]):
            last = int(b["len"][i]) - counts[i] + j
            want = [0] + list(range(10, 27)) + [last // bt - 1, last // bt]
            assert (got[int(b["off"][i]) + j] == torch.tensor(want)).all()


@pytest.mark.parametrize("blocks", [180, 5300])  # the second is more than a workgroup's registers hold
@pytest.mark.parametrize("scores", ["", "ties", "two values", "infinite", "one above", "far apart"])
def test_select_few_rows_of_any_scores(dev, scores, blocks):
    """Rows that a workgroup each takes: scores that fall into one part of their
    range, or have none."""
    rng = np.random.default_rng(28)
    H, h, d, bt, keep = 4, 4, 64, 16, 41
    b = ref.batch(rng, [1, 2, 0], [blocks * 16 - 3, blocks * 8, 50], bt)
    pool = make_pool(rng, 1, b, h, d, bt, spread=1)
    sref.random_bounds(rng, pool[0], h, d, bt, scores == "ties")
    n = ref.chunk_bytes(h, d, bt) - 16
    scale = pool[0, 0, :, n:n + 16].contiguous().view(torch.float32)
    if scores == "two values":  # all scores alike but for the scale
        for s in range(2):
            pool[0, s, :, n + 16:] = pool[0, s, :1, n + 16:]
        scale[:] = 1.0
        scale[torch.from_numpy(rng.permutation(b["pool"])[:15])] = 2.0
    elif scores == "infinite":
        scale[::40] = float("inf")
    elif scores == "one above":
        scale[7] = 2.0 ** 40
    elif scores == "far apart":
        scale[:] = torch.exp2(torch.from_numpy(rng.integers(-90, 90, scale.shape)).float())
    pool[0, 0, :, n:n + 16] = scale.view(torch.uint8)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    want = sref.select(pool[0], q, b, h, d, bt, keep, 1, 2)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    assert torch.equal(run_select(dev, kv, q.cuda(), on_gpu(b), keep, 1, 2).cpu(), want)


@pytest.mark.parametrize("h", [3, 8])
def test_select_long_spans(dev, h):
    """Workgroups of over 200 table entries, and a request that begins and ends
    inside one; heads that do not divide the XCDs evenly."""
    rng = np.random.default_rng(29)
    d, bt, keep = 64, 16, 9
    group = 16 if h == 3 else 6
    b = ref.batch(rng, [300, 2, 40], [24000, 900, 8000], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, b["tokens"], group * h, d, torch.float16)
    want = sref.select(pool[0], q, b, h, d, bt, keep, 1, 2)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    assert torch.equal(run_select(dev, kv, q.cuda(), on_gpu(b), keep, 1, 2).cpu(), want)
