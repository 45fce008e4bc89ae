"""cascade_attention with tanh caps from the smallest to the largest numbers
(tolerances of tests/test_gpu_kv8.py, which know no cap: a capped score is as
accurate as one without, however far below the cap it lies)."""
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


@pytest.mark.parametrize("cap", [1e-40, 0.01, 64.0, 64.5, 300.0, 1e4, 1e6, 1e15, 3.4e38])
@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("counts,lengths", [([1, 4], [130, 70]), ([90], [200])], ids=["few", "tiles"])
def test_caps(dev, cap, name, counts, lengths):
    rng = np.random.default_rng(6)
    H, h, d, bt = 4, 2, 128, 16
    b = ref.batch(rng, counts, lengths, bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q = rows(rng, b["tokens"], H, d, {"bf16": torch.bfloat16, "f16": torch.float16}[name])
    q[0, 0] = 0.0  # scores of 0
    for scale in (d ** -0.5, 3.0):  # scores of a few, and of hundreds
        want = ref.attend(pool[0], q, b, h, d, bt, scale, cap, 2)
        got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, scale, cap, 2)
        check_attention(got, want, name, d, 2)


def test_largest_scale(dev):
    """A scale whose product with log2(e) no float holds: the largest score
    takes all."""
    rng = np.random.default_rng(7)
    H, h, d, bt = 2, 1, 64, 16
    b = ref.batch(rng, [1, 70], [40, 90], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt)
    q = rows(rng, b["tokens"], H, d, torch.bfloat16)
    q[1, 0] = 0.0
    got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, 3.4e38)[0]
    assert not torch.isnan(got[1, 0]).any()
    want = ref.attend(pool[0], q, b, h, d, bt, 0.0)["out"][1, 0]
    assert torch.allclose(got[1, 0].cpu().double(), want, rtol=2.0 ** -6, atol=2.0 ** -6)
