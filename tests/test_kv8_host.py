"""The 8-bit KV cache's calls without a GPU: struct layouts, sizes, refusals
before any launch, rotary frequency tables, and the reference of the GPU tests
checked against hand values and against itself."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2608_06557_amd import cascade as cx
from tests import kv8_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "cascade.h")
FAKE = 4096  # never dereferenced: every call below fails a host-side check or launches nothing


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(cx.LIB_PATH):
        from paper_2608_06557_amd import build
        build.build()
    return cx.load()


STRUCTS = {"cascade_kv_format_t": cx.KvFormat, "cascade_kv_batch_t": cx.KvBatch,
           "cascade_rows_t": cx.Rows, "cascade_rope_t": cx.Rope,
           "cascade_rope_spec_t": cx.RopeSpec, "cascade_attention_t": cx.Attention,
           "cascade_evict_t": cx.Evict}


def test_struct_layout_matches_header(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "cascade.h"', "int main(){"]
    want = []
    for name, py in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(py))
        for f, _ in py._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(py, f).offset)
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in got] == want


def test_chunk_bytes():
    assert cx.cascade_kv_chunk_bytes(cx.KvFormat(16, 8, 128)) == 16 * 8 * 128 + 32
    assert cx.cascade_kv_chunk_bytes(cx.KvFormat(128, 1, 64)) == 128 * 64 + 16
    assert cx.cascade_kv_chunk_bytes(cx.KvFormat(32, 5, 256)) == ref.chunk_bytes(5, 256, 32)
    for bad in ((8, 8, 128), (48, 8, 128), (256, 8, 128), (16, 0, 128), (16, 257, 128), (16, 8, 96), (16, 8, 512)):
        assert cx.cascade_kv_chunk_bytes(cx.KvFormat(*bad)) == 0


def fmt(**kw):
    return cx.KvFormat(kw.get("bt", 16), kw.get("h", 8), kw.get("d", 128))


def pool(**kw):
    size = 16 * 8 * 128 + 32
    f = dict(base=FAKE, layers=2, slots=10, chunk=size, ls=20 * size, ks=10 * size, ss=size)
    f.update(kw)
    return cx.KvPool(f["base"], f["layers"], f["slots"], f["chunk"], f["ls"], f["ks"], f["ss"])


def batch(n=1, tokens=1, most=1, entries=4, off=FAKE, length=FAKE):
    return cx.KvBatch(n, tokens, most, entries, off, length)


TABLE = cx.BlockTable(FAKE, FAKE)
ROWS = cx.Rows(FAKE, 4096, 128)
BAD_POOLS = [pool(base=0), pool(base=FAKE + 8), pool(slots=0), pool(layers=0), pool(chunk=16 * 8 * 128 + 16),
             pool(ls=8), pool(ks=24), pool(ss=8), pool(ss=-16)]
BAD_ROWS = [cx.Rows(0, 4096, 128), cx.Rows(FAKE + 8, 4096, 128), cx.Rows(FAKE, 4100, 128), cx.Rows(FAKE, 4096, 4),
            cx.Rows(FAKE, -4096, 128)]
BAD_BATCHES = [batch(n=-1), batch(n=2049), batch(tokens=-1), batch(most=-1), batch(entries=-1), batch(off=0),
               batch(length=0)]


def test_append_refusals():
    rope = cx.Rope(128, 0, FAKE, 1.0)

    def call(p=pool(), layer=0, f=fmt(), b=batch(), t=TABLE, dt=cx.BF16, heads=32, q=ROWS, qo=ROWS, k=ROWS, v=ROWS,
             r=rope, pos=FAKE):
        return cx.cascade_kv_append(p, layer, f, b, t, dt, heads, q, qo, k, v, r, pos, 0, 0)

    E = cx.EINVAL
    for p in BAD_POOLS:
        assert call(p=p) == E
    for b in BAD_BATCHES:
        assert call(b=b) == E
    for r in BAD_ROWS:
        assert call(q=r) == E and call(qo=r) == E and call(k=r) == E and call(v=r) == E
    assert call(layer=2) == E and call(layer=-1) == E
    assert call(f=fmt(d=96)) == E and call(f=None) == E and call(p=None) == E and call(b=None) == E
    assert call(t=None) == E and call(t=cx.BlockTable(0, FAKE)) == E and call(t=cx.BlockTable(FAKE, 0)) == E
    assert call(dt=2) == E and call(dt=-1) == E
    assert call(q=None) == E and call(qo=None) == E and call(k=None) == E and call(v=None) == E
    assert call(heads=0) == E and call(heads=-4) == E
    assert call(pos=0) == E
    for bad in (cx.Rope(129, 0, FAKE, 1.0), cx.Rope(24, 0, FAKE, 1.0), cx.Rope(256, 0, FAKE, 1.0),
                cx.Rope(-16, 0, FAKE, 1.0), cx.Rope(64, 0, 0, 1.0), cx.Rope(64, 0, FAKE, float("nan"))):
        assert call(r=bad) == E
    # nothing to do
    assert call(b=batch(n=0)) == cx.OK and call(b=batch(tokens=0)) == cx.OK


def test_attention_refusals():
    ws = cx.cascade_attention_workspace_bytes(fmt(), batch(), 32, 0)

    def args(dt=cx.BF16, heads=32, scale=0.1, cap=0.0, q=ROWS, out=ROWS, lse=0, w=0, window=0):
        return cx.Attention(dt, heads, scale, cap, q, out, lse, w, window)

    def call(a=args(), p=pool(), layer=0, f=fmt(), b=batch(), t=TABLE, w=FAKE, size=1 << 40):
        return cx.cascade_attention(p, layer, f, b, t, a, w, size, 0, 0)

    E = cx.EINVAL
    for p in BAD_POOLS:
        assert call(p=p) == E
    for b in BAD_BATCHES:
        assert call(b=b) == E
    for r in BAD_ROWS:
        assert call(args(q=r)) == E and call(args(out=r)) == E
    assert call(None) == E and call(p=None) == E and call(f=None) == E and call(b=None) == E and call(t=None) == E
    assert call(layer=2) == E and call(f=fmt(bt=24)) == E
    for bad in (args(dt=3), args(heads=0), args(heads=12), args(heads=8 * 129), args(heads=-8), args(scale=float("inf")),
                args(cap=-1.0), args(cap=float("nan")), args(w=FAKE), args(w=FAKE, window=65), args(window=1)):
        assert call(bad) == E
    assert call(w=0) == E and call(w=FAKE + 16) == E
    assert call(size=ws - 1) == cx.ENOSPC
    more = cx.cascade_attention_workspace_bytes(fmt(), batch(), 32, 4)
    assert more > ws
    assert call(args(w=FAKE, window=4), size=more - 1) == cx.ENOSPC
    assert call(b=batch(n=0)) == cx.OK and call(b=batch(tokens=0)) == cx.OK and call(b=batch(most=0)) == cx.OK


def test_attention_workspace_size():
    size = cx.cascade_attention_workspace_bytes
    for d in (64, 128, 256):
        f = fmt(d=d)
        last = 0
        for tokens, entries in ((0, 0), (1, 1), (100, 50), (8192, 100000)):
            w = size(f, batch(tokens=tokens, entries=entries), 32, 8)
            assert w % 256 == 0 and w >= last > -1
            last = w
            assert 0 < size(f, batch(tokens=tokens, entries=entries), 32, 0) <= w
    assert size(fmt(d=32), batch(), 32, 0) == 0 and size(fmt(), batch(), 33, 0) == 0
    assert size(fmt(), batch(), 32, 65) == 0 and size(fmt(), batch(tokens=-1), 32, 0) == 0


def test_evict_refusals():
    def args(**kw):
        f = dict(n=1, n_entries=4, block_tokens=16, sink=0, recent=1)
        f.update({k: FAKE for k in ("kv_len", "keep_blocks", "block_weight", "kv_len_out", "row_offsets_out",
                                    "slots_out", "weight_out", "freed", "n_freed")})
        f.update(kw)
        return cx.Evict(**f)

    E = cx.EINVAL
    call = lambda a, t=TABLE: cx.cascade_kv_evict(t, a, 0, 0)
    for kw in (dict(n=-1), dict(n=2049), dict(n_entries=-1), dict(block_tokens=0), dict(sink=-1), dict(recent=0),
               *[{k: 0} for k in ("kv_len", "keep_blocks", "block_weight", "kv_len_out", "row_offsets_out",
                                  "slots_out", "weight_out", "freed", "n_freed")]):
        assert call(args(**kw)) == E, kw
    assert call(None) == E and call(args(), None) == E
    assert call(args(), cx.BlockTable(0, FAKE)) == E and call(args(), cx.BlockTable(FAKE, 0)) == E


SPECS = [("plain", cx.ROPE_PLAIN, 128, 10000.0, 1.0, 0.0, 1.0, 4.0),
         ("linear", cx.ROPE_LINEAR, 64, 10000.0, 4.0, 0.0, 1.0, 4.0),
         ("base", cx.ROPE_BASE, 128, 500000.0, 8.0, 0.0, 1.0, 4.0),
         ("bands", cx.ROPE_BANDS, 128, 500000.0, 8.0, 8192.0, 1.0, 4.0),
         ("ramp", cx.ROPE_RAMP, 128, 10000.0, 16.0, 4096.0, 1.0, 32.0),
         ("ramp", cx.ROPE_RAMP, 32, 1000000.0, 4.0, 32768.0, 1.0, 32.0),
         ("plain", cx.ROPE_PLAIN, 16, 1.5, 1.0, 0.0, 1.0, 4.0)]


@pytest.mark.parametrize("spec", SPECS, ids=[f"{s[0]}-{s[2]}" for s in SPECS])
def test_rope_frequencies(spec):
    name, kind, R, base, factor, length, low, high = spec
    rc, freq, scale = cx.cascade_rope_frequencies(cx.RopeSpec(kind, R, base, factor, length, low, high))
    th, want = ref.theta(name, R, base, factor, length, low, high)
    assert rc == 0 and len(freq) == R // 2
    got = freq.astype(np.float64) * 2.0 ** -64 * 2 * np.pi
    # pow, log and a few products in 64 bits
    assert np.allclose(got, th, rtol=2.0 ** -46, atol=2.0 ** -60)
    assert abs(scale - want) <= 2.0 ** -23 * want


def test_rope_refusals():
    call = lambda *a: cx.cascade_rope_frequencies(cx.RopeSpec(*a))[0]
    ok = (cx.ROPE_RAMP, 64, 10000.0, 2.0, 4096.0, 1.0, 32.0)
    assert call(*ok) == cx.OK
    for i, bads in enumerate([(-1, 5), (0, 8, 40, 272), (1.0, 0.5, float("inf"), float("nan")),
                              (0.5, float("nan")), (0.0, float("nan")), (0.0, -1.0), (1.0, 0.5, float("inf"))]):
        for bad in bads:
            a = list(ok)
            a[i] = bad
            assert call(*a) == cx.EINVAL, (i, bad)
    f = cx._kv().cascade_rope_frequencies
    s = C.c_float()
    assert f(None, FAKE, C.byref(s)) == cx.EINVAL
    spec = cx.RopeSpec(*ok)
    assert f(C.byref(spec), None, C.byref(s)) == cx.EINVAL
    assert f(C.byref(spec), FAKE, None) == cx.EINVAL


def test_python_side_refuses_what_does_not_fit():
    from paper_2608_06557_amd import device
    with pytest.raises(ValueError):
        device.kv_chunk_bytes(8, 100)
    p = torch.zeros(1, 2, 3, 16 * 64 + 16, dtype=torch.uint8)
    kv = device.DeviceKvPool(p, 1, 64, 16)
    for bad in (p[0], p.int(), p[..., :-16], torch.zeros(1, 3, 3, 2000, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            device.DeviceKvPool(bad, 1, 64, 16)
    i = lambda *a: torch.tensor(a, dtype=torch.int32)
    b = device.KvBatch(i(0, 2), i(2), i(0, 1), i(0), 2, 2)
    for bad in ((i(0), i(2), i(0, 1), i(0)), (i(0, 2).long(), i(2), i(0, 1), i(0)),
                (i(0, 2), i(2), i(0, 9, 1)[::2].contiguous()[:1], i(0))):
        with pytest.raises(ValueError):
            device.KvBatch(*bad, 2, 2)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    for bad in ((q, k[:1], k, q), (q, k, k.half(), q), (q, q, k, q), (q[:1], k, k, q), (q, k, k, q[:, :2])):
        with pytest.raises(ValueError):
            device.DeviceKvAppend(kv, b, bad[0], bad[1], bad[2], bad[3])
    with pytest.raises(TypeError):
        device.DeviceKvAppend(kv, b, None, k.float(), k.float())
    with pytest.raises(ValueError):  # no positions for a rotation
        device.DeviceKvAppend(kv, b, None, k, k, None, i(0), torch.zeros(32, dtype=torch.int64))
    for bad in ((q, q[:, :2]), (q[:1], q[:1]), (q, q.half()), (q[..., :32], q[..., :32])):
        with pytest.raises(ValueError):
            device.DeviceAttention(kv, b, bad[0], bad[1], 0.1)
    with pytest.raises(ValueError):
        device.DeviceAttention(kv, b, q, q.transpose(1, 2).contiguous().transpose(1, 2), 0.1)
    with pytest.raises(ValueError):
        device.DeviceAttention(kv, b, q, q, 0.1, block_weight=torch.zeros(1), weight_window=65)


# ------------------------------------------- the reference itself, by hand

def test_reference_layout_is_a_bijection_and_as_the_header_says():
    for h, d, bt in ((2, 64, 16), (3, 128, 32), (1, 256, 128)):
        for side in range(2):
            at = ref.code_offsets(h, d, bt, side)
            assert torch.equal(at.flatten().sort().values, torch.arange(h * bt * d))
    k, v = ref.code_offsets(2, 128, 32, 0), ref.code_offsets(2, 128, 32, 1)
    # head 1, token 19 (sub-block 1, t = 3), dim 70
    base = (1 * 32 + 16) * 128
    assert int(k[1, 19, 70]) == base + ((70 // 64) * 16 + 3) * 64 + 6
    assert int(v[1, 19, 70]) == base + ((1 * 4 + 0) * 16 + 70 % 16) * 16 + 0 * 4 + 3


def test_reference_rounding_and_scales():
    codes = torch.arange(256, dtype=torch.uint8).view(ref.E4M3).float()
    codes = codes[torch.isfinite(codes)].double()
    assert torch.equal(ref.round_e4m3(codes), codes)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(20000, generator=g, dtype=torch.float64) * 60
    x = torch.cat([x.clamp(-448, 448), x * 1e-4, torch.tensor([0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0])])
    near = (x[:, None] - codes.unique()[None]).abs().min(1).values
    assert torch.allclose((ref.round_e4m3(x) - x).abs(), near, rtol=0, atol=0)
    assert torch.equal(ref.round_e4m3(x), x.float().to(ref.E4M3).double())
    assert ref.round_e4m3(torch.tensor([17.0, 19.0], dtype=torch.float64)).tolist() == [16.0, 20.0]  # ties
    for a, s in ((448.0, 1.0), (448.5, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.0, 2.0 ** -100), (1e-35, 2.0 ** -100)):
        assert float(ref.scale_for(a)) == s


def test_reference_rotation_by_differences():
    """Turning keeps lengths, and the product of two turned vectors depends on
    the difference of their positions only."""
    rng = np.random.default_rng(0)
    f = ref.fixed(ref.theta("plain", 64, 10000.0)[0])
    x = torch.from_numpy(rng.normal(size=(4, 1, 128)))
    for inter in (False, True):
        a = ref.rotate(x[:2], [5, 1000005], f, inter)
        b = ref.rotate(x[2:3].expand(2, 1, 128), [3, 1000003], f, inter)
        assert torch.allclose(a.square().sum(-1), x[:2].square().sum(-1), rtol=1e-12)
        same = ref.rotate(torch.cat([x[:1], x[:1]]), [5, 1000005], f, inter)
        dots = (same * b).sum(-1)
        assert torch.allclose(dots[0], dots[1], rtol=1e-9)


def test_reference_attention_by_hand():
    h, d, bt = 1, 64, 16
    p = torch.zeros(2, 3, ref.chunk_bytes(h, d, bt), dtype=torch.uint8)
    codes = torch.zeros(3, h, bt, d)
    codes[1, 0, 0, 0], codes[1, 0, 1, 0] = 1.0, 2.0
    for side in range(2):
        ref.store(p[side], codes.to(ref.E4M3).view(torch.uint8), torch.full((3, h), 0.5), h, d, bt, side)
    q = torch.zeros(1, 1, d)
    q[0, 0, 0] = 2.0
    b = ref.batch(np.random.default_rng(0), [1], [2], bt)
    b["slots"][0] = 1
    e = ref.attend(p, q, b, h, d, bt, 1.0, 0.0, 1)  # scores 1 and 2, values 0.5 and 1
    w = np.exp([1.0, 2.0]) / np.exp([1.0, 2.0]).sum()
    assert np.isclose(float(e["out"][0, 0, 0]), 0.5 * w[0] + w[1])
    assert np.isclose(float(e["lse"][0, 0]), np.log(np.exp(1) + np.exp(2))) and np.isclose(float(e["weight"][0]), 1.0)


def test_reference_evict_by_hand():
    b = ref.batch(np.random.default_rng(0), [0, 0], [80, 33], 16)
    w = np.array([9, 1, 0, 1, 5, 2, 0, 7], np.float32)
    b["slots"][:] = torch.arange(8)
    got = ref.evict(b, w, [3, 1], 1, 1, 16)
    assert got[0] == [48, 17] and got[1] == [0, 3, 5]
    assert got[2] == [0, 3, 4, 5, 7] and got[4] == [1, 2, 6]


def test_no_new_call_is_left_out_of_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    for name in ("cascade_kv_append", "cascade_attention", "cascade_kv_evict"):
        assert re.search(rf"\b{name}\(", text)
