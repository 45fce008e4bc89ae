"""examples/kv_serving.py at a small size: its tables stay sound through
eviction, spill and restore, and its last attention is that of the cache's
bytes (tolerances of tests/test_gpu_kv8.py)."""
import importlib.util
import os

import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_kv8 import check_attention

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "kv_serving.py")


def test_kv_serving():
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("kv_serving", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    said = []
    server = example.serve(requests=4, tokens=8, budget=12, longest=700, layers=2, heads=8, kv_heads=2,
                           dim=64, seed=3, tell=said.append)
    assert any(" 0 dropped" not in line for line in said if line.startswith("batch"))
    held = [s for r in server.requests for s in r.slots]
    assert sorted(held + server.free) == list(range(server.kv.pool.shape[2]))
    for r in server.requests:
        assert len(r.made) >= 8 and len(r.slots) <= 12 and r.away is None
        assert len(r.slots) == -(-r.cached // 16) == r.weight.numel()
        assert r.seen == len(r.prompt) + len(r.made) - 1
    last = server.last
    b = dict(n=len(last["live"]), off=last["offsets"].cpu(), len=server.length.cpu(),
             rows=server.entries.cpu(), slots=server.slots.cpu(), tokens=int(last["offsets"][-1]),
             most=max(last["counts"]))
    e = ref.attend(server.kv.pool[1].cpu(), last["q"].cpu(), b, 2, 64, 16, 64 ** -0.5)
    check_attention((last["y"], None, None), e, "bf16", 64, 0)
