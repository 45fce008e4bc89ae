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
