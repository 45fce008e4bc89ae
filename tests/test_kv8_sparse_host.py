"""The calls over shared prefixes, bounds and selected blocks without a GPU:
struct layouts, sizes, refusals before any launch, and their Python classes."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2608_06557_amd import cascade as cx
from paper_2608_06557_amd import device
from tests import kv8_ref as ref
from tests import sparse_ref as sref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 4096  # never dereferenced: every call below fails a host-side check or launches nothing
E = cx.EINVAL


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(cx.LIB_PATH):
        from paper_2608_06557_amd import build
        build.build()
    return cx.load()


def test_struct_layout_matches_header(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "cascade.h"', "int main(){"]
    want = []
    for name, py in (("cascade_shared_t", cx.Shared), ("cascade_select_t", cx.Select)):
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(py))
        for f, _ in py._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(py, f).offset)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in got] == want


SIZE = 16 * 8 * 128 + 32 + 8 * 128  # of a chunk with bounds


def pool(**kw):
    f = dict(base=FAKE, layers=2, slots=10, chunk=SIZE, ls=20 * SIZE, ks=10 * SIZE, ss=SIZE)
    f.update(kw)
    return cx.KvPool(f["base"], f["layers"], f["slots"], f["chunk"], f["ls"], f["ks"], f["ss"])


def fmt(bt=16, h=8, d=128):
    return cx.KvFormat(bt, h, d)


def batch(n=1, tokens=1, most=1, entries=4, off=FAKE, length=FAKE):
    return cx.KvBatch(n, tokens, most, entries, off, length)


TABLE = cx.BlockTable(FAKE, FAKE)
ROWS = cx.Rows(FAKE, 4096, 128)
BAD_POOLS = [None, pool(base=0), pool(base=FAKE + 8), pool(slots=0), pool(layers=0), pool(ls=8), pool(ks=24),
             pool(ss=8), pool(ss=-16)]
BAD_ROWS = [cx.Rows(0, 4096, 128), cx.Rows(FAKE + 8, 4096, 128), cx.Rows(FAKE, 4100, 128), cx.Rows(FAKE, 4096, 4),
            cx.Rows(FAKE, -4096, 128)]
BAD_BATCHES = [None, batch(n=-1), batch(n=2049), batch(tokens=-1), batch(most=-1), batch(entries=-1), batch(off=0),
               batch(length=0)]
BAD_TABLES = [None, cx.BlockTable(0, FAKE), cx.BlockTable(FAKE, 0)]
BAD_FORMATS = [None, fmt(d=96), fmt(bt=8), fmt(h=0)]
EMPTY = [batch(n=0), batch(tokens=0), batch(most=0)]


def refused(call):
    for p in BAD_POOLS:
        assert call(p=p) == E
    for b in BAD_BATCHES:
        assert call(b=b) == E
    for t in BAD_TABLES:
        assert call(t=t) == E
    for f in BAD_FORMATS:
        assert call(f=f) == E
    assert call(layer=2) == E and call(layer=-1) == E


def refused_workspace(call, size):
    assert call(w=0) == E and call(w=FAKE + 16) == E
    assert size > 0 and call(size=size - 1) == cx.ENOSPC
    for b in EMPTY:
        assert call(b=b) == cx.OK


def attention(dt=cx.BF16, heads=32, scale=0.1, cap=0.0, q=ROWS, out=ROWS, lse=0, w=0, window=0):
    return cx.Attention(dt, heads, scale, cap, q, out, lse, w, window)


def refused_attention(call):
    nan, inf = float("nan"), float("inf")
    for a in (attention(dt=2), attention(dt=-1), attention(heads=0), attention(heads=33), attention(heads=-8),
              attention(heads=8 * 129), attention(scale=nan), attention(scale=inf), attention(cap=nan),
              attention(cap=-1.0), attention(w=FAKE, window=1), attention(window=1), attention(w=FAKE), None):
        assert call(a=a) == E
    for r in BAD_ROWS:
        assert call(a=attention(q=r)) == E and call(a=attention(out=r)) == E


def test_shared_refusals():
    def call(p=pool(), layer=0, f=fmt(), b=batch(), t=TABLE, a=attention(), s=cx.Shared(FAKE, FAKE, 1), w=FAKE,
             size=1 << 40):
        return cx.cascade_attention_shared(p, layer, f, b, t, a, s, w, size, 0, 0)

    refused(call)
    refused_attention(call)
    refused_workspace(call, cx.cascade_attention_shared_workspace_bytes(fmt(), batch(), 32))
    for s in (None, cx.Shared(0, FAKE, 1), cx.Shared(FAKE, 0, 1), cx.Shared(FAKE, FAKE, -1)):
        assert call(s=s) == E
    for f, b, heads in ((fmt(d=96), batch(), 32), (fmt(), None, 32), (fmt(), batch(), 33), (fmt(), batch(tokens=-1), 32)):
        assert cx.cascade_attention_shared_workspace_bytes(f, b, heads) == 0
    sizes = [cx.cascade_attention_shared_workspace_bytes(fmt(), batch(tokens=n), 32) for n in (1, 10, 1000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[-1] >= (1 << 20) * 32 * 130 * 4


def test_bounds_refusals():
    def call(p=pool(), layer=0, f=fmt(), b=batch(), t=TABLE, whole=0):
        return cx.cascade_kv_bounds(p, layer, f, b, t, whole, 0, 0)

    refused(call)
    assert call(whole=2) == E and call(whole=-1) == E
    assert call(p=pool(chunk=SIZE - 16)) == E  # no room for bounds
    assert call(b=batch(n=0)) == cx.OK and call(b=batch(tokens=0)) == cx.OK
    assert call(b=batch(entries=0), whole=1) == cx.OK
    assert cx.cascade_kv_bounds_bytes(fmt()) == 8 * 128 and cx.cascade_kv_bounds_bytes(fmt(d=96)) == 0


def test_select_refusals():
    def args(dt=cx.BF16, heads=32, keep=8, sink=1, recent=1, q=ROWS, selected=FAKE):
        return cx.Select(dt, heads, keep, sink, recent, q, selected)

    def call(p=pool(), layer=0, f=fmt(), b=batch(), t=TABLE, a=args(), w=FAKE, size=1 << 40):
        return cx.cascade_kv_select(p, layer, f, b, t, a, w, size, 0, 0)

    refused(call)
    refused_workspace(call, cx.cascade_kv_select_workspace_bytes(fmt(), batch()))
    assert call(p=pool(chunk=SIZE - 16)) == E
    for a in (None, args(dt=2), args(heads=0), args(heads=33), args(heads=8 * 129), args(keep=0), args(keep=65537),
              args(sink=-1), args(recent=0), args(sink=8), args(recent=8), args(sink=2 ** 31 - 1, recent=2 ** 31 - 1),
              args(selected=0)):
        assert call(a=a) == E
    for r in BAD_ROWS:
        assert call(a=args(q=r)) == E
    for f, b in ((fmt(d=96), batch()), (fmt(), None), (fmt(), batch(most=-1)), (fmt(), batch(entries=-1))):
        assert cx.cascade_kv_select_workspace_bytes(f, b) == 0
    big = batch(n=16, tokens=8192, most=512, entries=1 << 20)
    assert cx.cascade_kv_select_workspace_bytes(fmt(), big) >= (1 << 20) * 512 * 8 * 4  # over 2^32


def test_selected_attention_refusals():
    def call(p=pool(), layer=0, f=fmt(), b=batch(), t=TABLE, a=attention(), s=FAKE, keep=8, w=FAKE, size=1 << 40):
        return cx.cascade_attention_selected(p, layer, f, b, t, a, s, keep, w, size, 0, 0)

    refused(call)
    refused_attention(call)
    refused_workspace(call, cx.cascade_attention_selected_workspace_bytes(fmt(), batch(), 32, 8))
    assert call(s=0) == E and call(keep=0) == E and call(keep=65537) == E
    for f, b, heads, keep in ((fmt(d=96), batch(), 32, 8), (fmt(), None, 32, 8), (fmt(), batch(), 33, 8),
                              (fmt(), batch(), 32, 0), (fmt(), batch(tokens=-1), 32, 8)):
        assert cx.cascade_attention_selected_workspace_bytes(f, b, heads, keep) == 0
    # one made for any batch serves all
    size = {cx.cascade_attention_selected_workspace_bytes(fmt(), batch(tokens=n), 32, k)
            for n in (1, 7, 128, 8192) for k in (1, 64, 4096)}
    assert len(size) == 1
    longer = [cx.cascade_attention_selected_workspace_bytes(fmt(), batch(tokens=n), 32, 65536) for n in (1, 128, 8192)]
    assert longer == sorted(longer) and longer[-1] >= 8192 * 32 * 16 * 130 * 4


# ------------------------------------------------------------------ Python

def i32(*a, **kw):
    return torch.tensor(a, dtype=torch.int32, **kw)


def test_pools_with_bounds():
    plain = device.kv_chunk_bytes(2, 64, 16)
    assert device.kv_chunk_bytes(2, 64, 16, True) == plain + 128
    kv = device.DeviceKvPool.empty(1, 3, 2, 64, 16, "cpu", bounds=True)
    assert kv.pool.shape == (1, 2, 3, plain + 128) and kv.c_pool.chunk_bytes == plain + 128 == kv.chunk_bytes
    with pytest.raises(ValueError):
        device.DeviceKvPool(torch.zeros(1, 2, 3, plain, dtype=torch.uint8), 2, 64, 16, bounds=True)
    bare = device.DeviceKvPool.empty(1, 3, 2, 64, 16, "cpu")
    b = device.KvBatch(i32(0, 1), i32(1), i32(0, 1), i32(0), 1, 1)
    q, lists = torch.zeros(1, 4, 64, dtype=torch.float16), torch.zeros(1, 2, 5, dtype=torch.int32)
    for make in (lambda p: device.DeviceKvBounds(p, b), lambda p: device.DeviceKvSelect(p, b, q, lists)):
        make(kv)
        with pytest.raises(ValueError):
            make(bare)
    device.DeviceSelectedAttention(bare, b, q, lists, q, 0.1)  # reads no bounds


def test_arguments_that_do_not_fit_are_refused():
    kv = device.DeviceKvPool.empty(1, 3, 2, 64, 16, "cpu", bounds=True)
    b = device.KvBatch(i32(0, 2), i32(2), i32(0, 1), i32(0), 2, 2)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    good = dict(q=q, out=q, selected=torch.zeros(2, 2, 5, dtype=torch.int32), leader=i32(0), shared_len=i32(0),
                lse=torch.zeros(2, 4), workspace=torch.zeros(1 << 10, dtype=torch.uint8))
    far = torch.device("meta")

    def shared(**kw):
        a = dict(good, **kw)
        return device.DeviceSharedAttention(kv, b, a["leader"], a["shared_len"], 2, a["q"], a["out"], 0.1, lse=a["lse"],
                                            workspace=a["workspace"])

    def select(**kw):
        a = dict(good, **kw)
        return device.DeviceKvSelect(kv, b, a["q"], a["selected"], workspace=a["workspace"])

    def attend(**kw):
        a = dict(good, **kw)
        return device.DeviceSelectedAttention(kv, b, a["q"], a["selected"], a["out"], 0.1, lse=a["lse"],
                                              workspace=a["workspace"])

    uses = {shared: ("q", "out", "leader", "shared_len", "lse", "workspace"),
            select: ("q", "selected", "workspace"), attend: ("q", "out", "selected", "lse", "workspace")}
    wrong = dict(q=[q[:1], q[..., :32], q.float(), q.transpose(1, 2)], out=[q[:1], q.half()],
                 selected=[good["selected"][:1], good["selected"][:, :1], good["selected"].long(),
                           good["selected"][..., :0], good["selected"].transpose(1, 2), good["selected"][0]],
                 leader=[i32(), torch.zeros(1)], shared_len=[i32(), torch.zeros(1)],
                 lse=[torch.zeros(1, 4), torch.zeros(2, 4).double()],
                 workspace=[torch.zeros(1 << 10), torch.zeros(64, 64, dtype=torch.uint8).t()])
    for make, names in uses.items():
        make()
        for name in names:
            for bad in [good[name].to(far)] + wrong[name]:
                with pytest.raises((ValueError, TypeError)):
                    make(**{name: bad})
    # a workspace that is too small is the library's to refuse
    op = attend()
    with pytest.raises(RuntimeError, match=cx.cascade_strerror(cx.ENOSPC)):
        device._raise(op._call(0))


# ----------------------------------------------------- the reference itself

def test_reference_bounds_and_queries():
    """Hand values of the roundings, and that a score bounds every key's."""
    q = torch.tensor([[[127.0, -63.5, 0.5, 1.5]], [[128.0, 1.0, 2.0, 3.0]], [[0.0, 0, 0, 0]], [[254.0, -1.0, 1, 3]]])
    n, e = sref.whole_queries(q)
    assert e.flatten().tolist() == [0, 1, -100, 1]
    assert n[:, 0].tolist() == [[127, -64, 0, 2], [64, 0, 1, 2], [0, 0, 0, 0], [127, 0, 0, 2]]
    rng = np.random.default_rng(1)
    h, d, bt = 2, 64, 16
    b = ref.batch(rng, [0], [200], bt)
    pool = ref.random_pool(rng, 1, b["pool"], h, d, bt, pad=h * d)
    n = ref.chunk_bytes(h, d, bt)
    for slot, both in sref.bounds_of(pool[0], b, h, d, bt, True).items():
        for s in range(2):
            pool[0, s, slot, n:] = torch.from_numpy(both[s].astype(np.int8)).view(torch.uint8).flatten()
    upper, lower = sref.bounds_in(pool[0], h, d, bt)
    code = ref.codes_of(pool[0, 0], h, d, bt, 0).view(ref.E4M3).float().numpy()
    assert (np.abs(upper) <= 112).all() and (np.abs(lower) <= 112).all()
    for k, slot in enumerate(b["slots"].tolist()):
        c = code[slot][:, :min(bt, 200 - k * bt)]
        x = rng.normal(0, 50, (h, 1, d))
        bound = (np.maximum(x[:, 0], 0) * upper[slot] + np.minimum(x[:, 0], 0) * lower[slot]).sum(-1) * 4
        assert ((c * x).sum(-1).max(-1) <= bound).all()
