"""cascade_attention where new tokens outnumber cached ones: the rows that see
nothing get zeros and lse -infinity, the others their attention (tolerances of
tests/test_gpu_kv8.py)."""
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


def attend(dev, seed, H, h, d, counts, lengths, window=0, name="bf16", bt=16):
    rng = np.random.default_rng(seed)
    b = ref.batch(rng, counts, lengths, bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q = rows(rng, b["tokens"], H, d, {"bf16": torch.bfloat16, "f16": torch.float16}[name])
    e = ref.attend(pool[0], q, b, h, d, bt, d ** -0.5, 0.0, window)
    got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, d ** -0.5, 0.0, window)
    check_attention(got, e, name, d, window)
    first = 0
    for c, l in zip(counts, lengths):  # to the bit
        assert not got[0][first:first + max(c - l, 0)].any()
        assert (got[1][first:first + max(c - l, 0)] == -np.inf).all()
        first += c


@pytest.mark.parametrize("H,h,d,count,length", [(1, 1, 128, 2000, 100), (4, 2, 64, 1500, 37), (2, 1, 256, 900, 130),
                                                (4, 1, 128, 1100, 1090), (2, 2, 128, 3000, 1300)])
def test_row_tiles_longer_than_the_cache(dev, H, h, d, count, length):
    attend(dev, count, H, h, d, [count], [length], window=3)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("counts,lengths", [([1], [0]), ([5, 1, 2], [0, 0, 0]), ([1, 1], [0, 600]),
                                            ([6, 1, 40], [0, 33, 30]), ([20, 70], [0, 0]), ([9, 3], [2, 700])])
def test_first_requests_without_cached_tokens(dev, d, counts, lengths):
    """The first table row among them, and whole batches without a table, as
    padding requests leave them."""
    attend(dev, d, 4, 2, d, counts, lengths, window=2 if sum(lengths) else 0)


def test_nothing_in_front_of_the_table_counts(dev):
    """A request without tokens has no part of the table: what lies in front of
    it, here slots outside the pool, is not reported."""
    H, h, d, bt = 8, 2, 128, 16
    rng = np.random.default_rng(3)
    b = ref.batch(rng, [1, 1], [0, 9], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q = rows(rng, 2, H, d, torch.bfloat16)
    g = on_gpu(b)
    held = torch.full((9,), 1 << 20, dtype=torch.int32, device="cuda")  # slots outside the pool
    held[8] = g["slots"][0]
    e = ref.attend(pool[0], q, b, h, d, bt, 0.1)
    got = run_attention(dev, pool.cuda(), q.cuda(), dict(g, slots=held[8:]), h, d, bt, 0.1)
    check_attention(got, e, "bf16", d, 0)


def test_weights_of_an_empty_table(dev):
    """Block weights asked for where no request has a block."""
    attend(dev, 5, 4, 2, 64, [3, 1], [0, 0], window=2)
