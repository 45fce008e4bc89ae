"""cascade_attention_shared against the 64-bit reference of plain attention
over the same tables (tolerances of tests/test_gpu_kv8.py: a row's sums fall
into two runs of tokens, whose errors those bounds count already)."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_kv8 import TYPES, check_attention, make_batch, on_gpu, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


def shared_batch(rng, groups, bt, slack=0):
    """`groups`: (shared tokens, [(new, own tokens with the new ones), ...])."""
    counts, own, shared, leader, held = [], [], [], [], []
    for tokens, members in groups:
        first = len(counts)
        for c, o in members:
            leader.append(first)
            shared.append(tokens if len(counts) == first else -99)  # of the first only
            held.append(tokens)
            counts.append(c)
            own.append(o)
    lengths = np.array(held) + np.array(own)
    b = ref.batch(rng, counts, lengths, bt, slack)
    for i, (first, tokens) in enumerate(zip(leader, held)):
        k = tokens // bt
        b["slots"][b["rows"][i]:b["rows"][i] + k] = b["slots"][b["rows"][first]:b["rows"][first] + k].clone()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32)
    per = np.bincount(leader, counts)
    b.update(leader=i32(leader), shared=i32(shared), most_shared=int(per.max()))
    return b


def run_shared(dev, pool, q, g, h, d, bt, scale, cap=0.0, want_lse=True, layer=0, stream=None, check=True,
               most=None):
    kv = dev.DeviceKvPool(pool, h, d, bt)
    out = torch.full(tuple(q.shape), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(tuple(q.shape[:2]), 7.0, device="cuda") if want_lse else None
    op = dev.DeviceSharedAttention(kv, make_batch(dev, g), g["leader"], g["shared"],
                                   g["most_shared"] if most is None else most, q, out, scale, cap, lse, layer)
    op.workspace.fill_(0xff)  # any content: here NaN
    op.run(stream)
    torch.cuda.synchronize()
    if check:
        kv.check()
    return out, lse, None


def stale(pool_layer, b, h, d, bt):
    """Everything past a request's last token is NaN codes."""
    for i in range(b["n"]):
        l, row = int(b["len"][i]), int(b["rows"][i])
        if l % bt:
            for side in range(2):
                at = ref.code_offsets(h, d, bt, side)[:, l % bt:].flatten()
                pool_layer[side, int(b["slots"][row + l // bt]), at] = 0x7f


SHARED = [
    # heads, kv heads, dim, block, type, cap, lse, groups
    (8, 2, 128, 16, "bf16", 0.0, True, [(32, [(1, 1), (1, 20), (1, 7)])]),
    (8, 2, 128, 16, "bf16", 0.0, False, [(0, [(1, 5)]), (16, [(1, 1)]), (48, [(1, 40), (1, 1)]), (0, [(3, 9)])]),
    (4, 1, 64, 16, "f16", 0.0, True, [(112, [(2, 3), (0, 40), (1, 30)]), (16, [(0, 5), (3, 3)]), (64, [(0, 0)])]),
    (4, 4, 256, 32, "bf16", 20.0, True, [(320, [(1, 70)] * 9), (32, [(2, 2)])]),
    (14, 2, 128, 16, "f16", 5.0, True, [(257 * 16, [(2, 9), (1, 33), (1, 1)]), (16, [(9, 12)])]),
    (32, 1, 128, 128, "bf16", 0.0, True, [(128, [(1, 129), (1, 3)]), (512, [(1, 1)] * 5)]),
    # groups of more rows than a wave's tiles hold; requests of few and many rows
    (8, 1, 128, 16, "bf16", 0.0, True, [(400, [(1, 1 + i) for i in range(40)]), (32, [(1, 1)] * 2)]),
    (16, 2, 64, 32, "f16", 100.0, True, [(96, [(12, 12), (30, 64)]), (992, [(1, 9)] * 20)]),
    (4, 2, 256, 16, "f16", 0.0, False, [(160, [(70, 70), (1, 2)]), (3008, [(1, 1)] * 33)]),
    (8, 2, 128, 16, "bf16", 0.0, False, [(48, [(90, 100), (20, 300)]), (0, [(80, 85)]), (2064, [(40, 40), (40, 50)])]),
    (128, 1, 64, 64, "bf16", 0.0, True, [(64, [(1, 1), (2, 70)]), (128, [(1, 5)])]),
]


@pytest.mark.parametrize("case", SHARED, ids=[f"{c[0]}h{c[1]}kv{c[2]}d{c[3]}bt-{c[4]}-{i}" for i, c in enumerate(SHARED)])
def test_shared(dev, case):
    H, h, d, bt, name, cap, want_lse, groups = case
    rng = np.random.default_rng(H + d + len(groups))
    b = shared_batch(rng, groups, bt, slack=1)
    pool = ref.random_pool(rng, 2, b["pool"], h, d, bt, pad=16)
    stale(pool[1], b, h, d, bt)
    q = rows(rng, b["tokens"], H, d, TYPES[name])
    scale = 1.7 * d ** -0.5
    e = ref.attend(pool[1], q, b, h, d, bt, scale, cap)
    args = (dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, scale, cap, want_lse, 1)
    got = run_shared(*args)
    check_attention(got, e, name, d, 0)
    again = run_shared(*args)
    assert torch.equal(got[0], again[0]) and (not want_lse or torch.equal(got[1], again[1]))


@pytest.mark.parametrize("scale", [8.0, 0.0, -0.4])
def test_shared_peaked_and_flat_scores(dev, scale):
    """Rows whose maximum lies far below or above the shared tokens'."""
    rng = np.random.default_rng(4)
    H, h, d, bt = 4, 2, 64, 16
    b = shared_batch(rng, [(400, [(1, 30), (2, 300), (1, 1)]), (16, [(1, 600)])], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt, spread=0)
    q = rows(rng, b["tokens"], H, d, torch.float16)
    e = ref.attend(pool[0], q, b, h, d, bt, scale)
    check_attention(run_shared(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, scale), e, "f16", d, 0)


def test_shared_most_requests(dev):
    """2048 requests in groups of every size; some without new tokens."""
    rng = np.random.default_rng(5)
    groups, left = [], 2048
    while left:
        m = min(left, int(rng.integers(1, 60)))
        groups.append((16 * int(rng.integers(0, 4)), [(int(c), int(c) + int(rng.integers(0, 20)))
                                                      for c in rng.integers(0, 3, m)]))
        left -= m
    b = shared_batch(rng, groups, 16)
    pool = ref.random_pool(rng, 1, b["pool"], 1, 64, 16)
    q = rows(rng, b["tokens"], 2, 64, torch.bfloat16)
    e = ref.attend(pool[0], q, b, 1, 64, 16, 0.2)
    check_attention(run_shared(dev, pool.cuda(), q.cuda(), on_gpu(b), 1, 64, 16, 0.2), e, "bf16", 64, 0)


def test_shared_on_another_stream_and_in_graphs(dev):
    """Two graphs that share a workspace, replayed in turn."""
    rng = np.random.default_rng(11)
    H, h, d, bt = 8, 2, 128, 16
    b = shared_batch(rng, [(640, [(1, 9)] * 12), (32, [(30, 200), (1, 1)])], bt)
    g = on_gpu(b)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt).cuda()
    qs = [rows(rng, b["tokens"], H, d, torch.bfloat16).cuda() for _ in range(2)]
    want = [run_shared(dev, pool, q, g, h, d, bt, 0.1) for q in qs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run_shared(dev, pool, qs[0], g, h, d, bt, 0.1, stream=side)
    assert torch.equal(got[0], want[0][0]) and torch.equal(got[1], want[0][1])
    kv = dev.DeviceKvPool(pool, h, d, bt)
    outs, graphs, ws = [], [], None
    for q in qs:
        out = torch.zeros_like(q)
        op = dev.DeviceSharedAttention(kv, make_batch(dev, g), g["leader"], g["shared"], b["most_shared"], q, out,
                                       0.1, lse=torch.zeros(tuple(q.shape[:2]), device="cuda"), workspace=ws)
        ws = op.workspace
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            op.run()
        outs.append(out)
        graphs.append((graph, op))
    for _ in range(3):
        for k in (0, 1, 1, 0):
            outs[k].fill_(3.0)
            graphs[k][0].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[k], want[k][0])
    kv.check()


@pytest.mark.parametrize("fault", ["leader behind", "leader negative", "leader apart", "not a leader", "length odd",
                                   "length negative", "length long", "slot", "row", "group"])
def test_shared_refuses_bad_groups(dev, fault):
    """The status word says so, and groups beside the bad one are right."""
    rng = np.random.default_rng(12)
    H, h, d, bt = 4, 2, 64, 16
    b = shared_batch(rng, [(32, [(1, 4), (1, 9)]), (64, [(1, 5), (2, 30), (1, 1)]), (16, [(1, 3)])], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    e = ref.attend(pool[0], q, b, h, d, bt, 0.2)
    most = None
    if fault == "leader behind":
        b["leader"][3] = 4
    elif fault == "leader negative":
        b["leader"][3] = -1
    elif fault == "leader apart":
        b["leader"][4] = 0
    elif fault == "not a leader":
        b["leader"][4] = 3
    elif fault == "length odd":
        b["shared"][2] = 40
    elif fault == "length negative":
        b["shared"][2] = -16
    elif fault == "length long":
        b["shared"][2] = 80
    elif fault == "slot":
        b["slots"][int(b["rows"][3]) + 3] = b["slots"][int(b["rows"][3]) + 4]
    elif fault == "row":
        b["rows"][3:] += 1 << 20
    else:
        most = 3
    g = on_gpu(b)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt)
    out = torch.zeros(tuple(q.shape), dtype=q.dtype, device="cuda")
    lse = torch.zeros(tuple(q.shape[:2]), device="cuda")
    dev.DeviceSharedAttention(kv, make_batch(dev, g), g["leader"], g["shared"],
                              b["most_shared"] if most is None else most, q.cuda(), out, 0.2, lse=lse).run()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError):
        kv.check()
    good = [0, 1] if fault == "row" else [0, 1, 6]
    part = {k: v[good] for k, v in e.items() if k != "weight"}
    check_attention((out.cpu()[good], lse.cpu()[good], None), part, "bf16", d, 0)
