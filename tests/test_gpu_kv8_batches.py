"""cascade_attention and cascade_kv_evict over the largest batches, tables at
the lengths where the work's division changes, and row tiles with and without
log sums (tolerances of tests/test_gpu_kv8.py)."""
import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_kv8 import check_attention, on_gpu, rows, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    from paper_2608_06557_amd import cascade, device
    assert torch.cuda.is_available()
    cascade.load()
    return device


def attend(dev, seed, H, h, d, counts, lengths, window=0, want_lse=True, name="bf16"):
    rng = np.random.default_rng(seed)
    b = ref.batch(rng, counts, lengths, 16)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, 16)
    q = rows(rng, b["tokens"], H, d, {"bf16": torch.bfloat16, "f16": torch.float16}[name])
    e = ref.attend(pool[0], q, b, h, d, 16, d ** -0.5, 0.0, window)
    got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, 16, d ** -0.5, 0.0, window, want_lse)
    check_attention(got, e, name, d, window)


def test_most_requests(dev):
    """2048 requests: single tokens, none, and two chunks of many rows."""
    rng = np.random.default_rng(0)
    counts = rng.integers(0, 2, 2048)
    lengths = counts + rng.integers(0, 40, 2048)
    for i, c in ((17, 90), (2047, 70)):
        counts[i], lengths[i] = c, c + 11
    attend(dev, 1, 2, 1, 128, counts, lengths, window=2)


@pytest.mark.parametrize("length", [511, 512, 513, 1024, 1025])
@pytest.mark.parametrize("count", [1, 9])
def test_short_tables(dev, length, count):
    attend(dev, length, 8, 2, 64, [count], [length], window=1)
    attend(dev, length, 8, 2, 128, [count, 1], [length // 2, length // 2], name="f16")


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("want_lse", [False, True])
def test_row_tiles(dev, d, want_lse):
    """One request uncut, one cut, one of less than a tile."""
    attend(dev, d, 4, 2, d, [150, 300, 40], [150, 2500, 2049], want_lse=want_lse)


def test_evict_most_requests(dev):
    rng = np.random.default_rng(6)
    lengths = rng.integers(0, 300, 2048)
    lengths[3], lengths[700] = 20000, 160000  # of more blocks than threads, and than they hold
    b = ref.batch(rng, np.zeros(2048, int), lengths, 16)
    n = len(b["slots"])
    w = np.floor(rng.random(n) * 50).astype(np.float32)
    keep = rng.integers(0, 12, 2048)
    keep[3], keep[700] = 400, 5000
    e = ref.evict(b, w, keep, 1, 2, 16)
    g = on_gpu(b)
    op = dev.DeviceKvEvict(16, g["len"], g["rows"], g["slots"], torch.from_numpy(w).cuda(),
                           torch.tensor(keep, dtype=torch.int32, device="cuda"), 1, 2)
    op.run()
    assert int(op.status) == 0
    assert op.kv_len_out.tolist() == e[0] and op.row_offsets_out.tolist() == e[1]
    assert op.slots_out[:len(e[2])].tolist() == e[2] and op.freed[:len(e[4])].tolist() == e[4]
    assert int(op.n_freed) == len(e[4])


def test_few_row_tiles_are_cut(dev):
    """Row tiles too few to fill the GPU, of lengths that many would leave whole."""
    attend(dev, 7, 8, 4, 128, [70], [2000], window=3)
    attend(dev, 8, 4, 2, 256, [138, 100], [753, 641])
    attend(dev, 9, 4, 2, 64, [90, 1, 120], [1500, 1500, 1100], window=2, name="f16")
