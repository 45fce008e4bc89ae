"""cascade_attention's row tiles over blocks of every size, with block weights,
lengths that end inside a block and inside a run of 32 tokens, cut and uncut,
alone and beside requests of few rows (tolerances of tests/test_gpu_kv8.py)."""
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


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("bt", [16, 32, 64, 128])
@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("counts,lengths,window", [
    ([90], [200], 5),            # uncut
    ([70], [2500], 64),          # cut, as few row tiles are
    ([130, 1, 75], [397, 85, 1111], 3),  # beside a single token
], ids=["uncut", "cut", "beside"])
def test_row_tiles_in_blocks(dev, d, bt, name, counts, lengths, window):
    rng = np.random.default_rng(d + bt + len(counts))
    H, h = 4, 2
    b = ref.batch(rng, counts, lengths, bt, slack=1)
    pool = ref.random_pool(rng, 2, b["pool"], h, d, bt, pad=16)
    # places past a request's last token are NaN codes
    for i in range(b["n"]):
        l, row = int(b["len"][i]), int(b["rows"][i])
        if l % bt:
            for side in range(2):
                at = ref.code_offsets(h, d, bt, side)[:, l % bt:].flatten()
                pool[1, side, int(b["slots"][row + l // bt]), at] = 0x7f
    q = rows(rng, b["tokens"], H, d, {"bf16": torch.bfloat16, "f16": torch.float16}[name])
    e = ref.attend(pool[1], q, b, h, d, bt, d ** -0.5, 0.0, window)
    got = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, d ** -0.5, 0.0, window, layer=1)
    check_attention(got, e, name, d, window)
    # and without log sums, whose kernels take the weights' sum another way
    out = run_attention(dev, pool.cuda(), q.cuda(), on_gpu(b), h, d, bt, d ** -0.5, want_lse=False, layer=1)
    check_attention(out, e, name, d, 0)
