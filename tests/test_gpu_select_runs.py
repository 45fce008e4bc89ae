"""Block selection by workspaces that do not hold all scores: the new tokens are
taken in runs, with the same result."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests import sparse_ref as sref
from tests.test_gpu_kv8 import make_batch, on_gpu, rows
from tests.test_gpu_sparse import make_pool, run_select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


def one_token(b, h):
    """Bytes of the scores of a new token of each request."""
    return 4 * (len(b["slots"]) + 16 * b["n"]) * h


def select_in(dev, kv, q, g, keep, sink, recent, size, most=0, check=True):
    """By a workspace of `size` bytes, full of NaN."""
    got = torch.full((q.shape[0], kv.kv_heads, keep), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    assert ws.data_ptr() % 256 == 0
    op = dev.DeviceKvSelect(kv, make_batch(dev, g), q, got, sink, recent, workspace=ws, most_blocks=most)
    op.run()
    torch.cuda.synchronize()
    if check:
        kv.check()
    return got, op


RUNS = [
    # heads, kv heads, dim, block, type, keep, sink, recent, counts, lengths
    (8, 2, 128, 16, "bf16", 6, 1, 2, [1, 1, 75, 0, 5], [400, 90, 600, 50, 300]),  # decodes, a chunk and drafts
    (8, 8, 64, 16, "f16", 20, 1, 2, [3, 290], [700, 900]),                        # a wave to a row
    (40, 1, 64, 32, "bf16", 5, 0, 1, [70, 2], [900, 400]),                        # 40 heads of a KV head
    (6, 3, 256, 16, "bf16", 9, 0, 3, [130, 130, 1], [400, 260, 3]),
    (2, 2, 64, 16, "f16", 50, 1, 1, [40], [39]),                                  # rows that see nothing
    (2, 1, 64, 16, "bf16", 400, 1, 1, [90, 1], [900, 700]),                       # nothing to choose
]


@pytest.mark.parametrize("case", RUNS, ids=[f"{c[0]}h{c[1]}kv{c[2]}d{c[3]}bt-{c[4]}-{i}" for i, c in enumerate(RUNS)])
def test_runs_of_tokens(dev, case):
    H, h, d, bt, name, keep, sink, recent, counts, lengths = case
    rng = np.random.default_rng(sum(lengths) + H)
    b = ref.batch(rng, counts, lengths, bt, slack=1)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, b["tokens"] + 2, H, d, {"bf16": torch.bfloat16, "f16": torch.float16}[name], 3.0)
    want = sref.select(pool[0], q, b, h, d, bt, keep, sink, recent)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    g, one = on_gpu(b), one_token(b, h)
    for tokens in (1, 2, 3.5, 17, 64, 65, 128, 1000):
        got, _ = select_in(dev, kv, q.cuda(), g, keep, sink, recent, int(tokens * one) + 256)
        assert torch.equal(got.cpu(), want), tokens
    # by tokens, where that takes less; by runs where it does not fit
    most = max(-(-l // bt) for l in lengths)
    by_tokens = 4 * b["tokens"] * h * (-(-most // 16) * 16)
    for size in (by_tokens, by_tokens - 4, one):
        if size >= one or size == by_tokens < one * b["most"]:
            got, _ = select_in(dev, kv, q.cuda(), g, keep, sink, recent, size + 256, most)
            assert torch.equal(got.cpu(), want), size
    with pytest.raises(RuntimeError):
        select_in(dev, kv, q.cuda(), g, keep, sink, recent, one + 255)


def test_runs_in_graphs(dev):
    """Two graphs of several runs that share a workspace, replayed in turn."""
    rng = np.random.default_rng(31)
    H, h, d, bt, keep = 8, 2, 64, 16, 7
    b = ref.batch(rng, [1, 150, 3], [900, 1500, 700], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    g = on_gpu(b)
    batch = make_batch(dev, g)
    ws = torch.zeros(20 * one_token(b, h) + 256, dtype=torch.uint8, device="cuda")
    made = []
    for _ in range(2):
        q = rows(rng, b["tokens"], H, d, torch.bfloat16)
        got = torch.zeros(b["tokens"], h, keep, dtype=torch.int32, device="cuda")
        op = dev.DeviceKvSelect(kv, batch, q.cuda(), got, 1, 1, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            op.run()
        made.append((graph, op, got, sref.select(pool[0], q, b, h, d, bt, keep, 1, 1)))
    for _ in range(3):
        for k in (0, 1, 1, 0):
            graph, _, got, want = made[k]
            got.fill_(-3)
            ws.fill_(0xff)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got.cpu(), want)
    kv.check()


def test_more_new_tokens_than_a_run_may_have(dev):
    """A prompt of 33 thousand tokens at once: by all that a run takes, and by
    runs of 1024; the last rows against the formula."""
    rng = np.random.default_rng(32)
    H, h, d, bt, keep, n = 2, 1, 64, 16, 5, 33000
    b = ref.batch(rng, [n], [n + 10], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    q = rows(rng, n, H, d, torch.bfloat16)
    g, one = on_gpu(b), one_token(b, h)
    got, _ = select_in(dev, kv, q.cuda(), g, keep, 1, 1, 32768 * one + 256)
    few, _ = select_in(dev, kv, q.cuda(), g, keep, 1, 1, 1024 * one + 256)
    assert torch.equal(got, few)
    one_more = on_gpu(dict(b, slots=torch.cat([b["slots"], torch.zeros(100, dtype=torch.int32)])))  # by tokens
    got, _ = select_in(dev, kv, q.cuda(), one_more, keep, 1, 1, 4 * n * h * 2064 + 256, most=2064)
    assert torch.equal(got, few)
    last = dict(b, off=torch.tensor([0, 9], dtype=torch.int32), tokens=9, most=9)
    want = sref.select(pool[0], q[-9:], last, h, d, bt, keep, 1, 1)
    assert torch.equal(got[-9:].cpu(), want)


def test_scores_over_4_gib(dev):
    """A request far along the table, whose scores lie behind 2^32 bytes."""
    rng = np.random.default_rng(33)
    H, h, d, bt, keep = 8, 8, 64, 16, 6
    b = ref.batch(rng, [1, 4], [200, 500], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, 5, H, d, torch.bfloat16)
    want = sref.select(pool[0], q, b, h, d, bt, keep, 1, 1)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    slack, first = 1 << 25, int(b["rows"][1])
    g = on_gpu(b)
    gap = torch.zeros(slack, dtype=torch.int32, device="cuda")
    g["slots"] = torch.cat([g["slots"][:first], gap, g["slots"][first:]])
    g["rows"] = torch.cat([g["rows"][:1], g["rows"][1:] + slack])
    got, op = select_in(dev, kv, q.cuda(), g, keep, 1, 1, 4 * one_token(g, h) + 256)
    assert op.ws_bytes > 1 << 32
    assert torch.equal(got.cpu(), want)
    assert torch.equal(run_select(dev, kv, q.cuda(), g, keep, 1, 1).cpu(), want)  
    got, op = select_in(dev, kv, q.cuda(), g, keep, 1, 1, 1 << 20, most=32)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("size", [1 << 20, 1100])  # by tokens, and by runs
def test_requests_of_more_blocks_than_told_are_refused(dev, size):
    rng = np.random.default_rng(34)
    H, h, d, bt, keep = 4, 2, 64, 16, 5
    b = ref.batch(rng, [2, 3, 1], [300, 340, 200], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, 6, H, d, torch.bfloat16)
    want = sref.select(pool[0], q, b, h, d, bt, keep, 1, 1)
    want[2:5] = -7
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    got, _ = select_in(dev, kv, q.cuda(), on_gpu(b), keep, 1, 1, size, most=19, check=False)
    with pytest.raises(RuntimeError):
        kv.check()
    assert torch.equal(got.cpu(), want)


def test_far_rows_by_tokens(dev):
    """Scores by tokens behind 2^32 bytes of the workspace."""
    rng = np.random.default_rng(35)
    H, h, d, bt, keep, T = 2, 2, 64, 16, 6, 70000
    b = ref.batch(rng, [T, 2], [T, 500], bt)
    pool = make_pool(rng, 1, b, h, d, bt)
    sref.random_bounds(rng, pool[0], h, d, bt)
    q = rows(rng, T + 2, H, d, torch.bfloat16)
    last = dict(b, off=torch.tensor([0, 4, 6], dtype=torch.int32), tokens=6, most=4)
    want = sref.select(pool[0], q[-6:], last, h, d, bt, keep, 1, 1)
    kv = dev.DeviceKvPool(pool.cuda(), h, d, bt, bounds=True)
    most = 1 << 13
    size = 4 * (T + 2) * h * most + 256
    assert size > 1 << 32
    g = on_gpu(b)
    g["slots"] = torch.cat([g["slots"], torch.zeros(20 * most, dtype=torch.int32, device="cuda")])  # or by requests
    got, _ = select_in(dev, kv, q.cuda(), g, keep, 1, 1, size, most=most)
    assert torch.equal(got[-6:].cpu(), want)
