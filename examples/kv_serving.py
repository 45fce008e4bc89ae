"""Requests served over the 8-bit paged KV cache, as an engine would between
two scheduling steps: prompts enter in chunks beside single tokens of running
requests, every layer writes its keys and values (cascade_kv_append) and reads
the cache (cascade_attention), the last layer gathers how much weight each
block receives, requests over their budget lose their least-read blocks
(cascade_kv_evict), and one request is spilled to staging and restored into
other slots (cascade_pack, cascade_unpack).  The model is random weights:
projections are torch's, everything on the cache is the library's.

    python examples/kv_serving.py [--requests 6] [--tokens 24] [--budget 64]
"""
import argparse
import os
import sys
import time

import numpy as np

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2608_06557_amd import cascade as cx  # noqa: E402
from paper_2608_06557_amd import device as dev  # noqa: E402


class Model:
    """Random attention layers over a small vocabulary."""

    def __init__(self, layers, heads, kv_heads, dim, vocab, seed):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: (torch.randn(*s, generator=g, device="cuda") / s[0] ** 0.5).bfloat16()
        width = 8 * dim
        self.layers, self.heads, self.kv_heads, self.dim = layers, heads, kv_heads, dim
        self.embed = (torch.randn(vocab, width, generator=g, device="cuda")).bfloat16()
        self.qkv = [rand(width, (heads + 2 * kv_heads) * dim) for _ in range(layers)]
        self.out = [rand(heads * dim, width) for _ in range(layers)]
        self.freq, self.rope_scale = dev.rope_frequencies(dim, 500000.0)


class Request:
    def __init__(self, prompt):
        self.prompt, self.made = list(prompt), []
        self.seen = 0      # tokens written, the next one's position
        self.cached = 0    # of them in the cache
        self.slots = []    # their blocks
        self.weight = None  # what each block has received, on the device
        self.away = None   # staging buffer while the request is spilled

    def take(self, chunk):
        """The tokens that the request puts into the next batch."""
        return (self.prompt + self.made)[self.seen:][:chunk]


class Server:
    def __init__(self, model, requests, slots, budget, block=16, chunk=256, window=8):
        import torch
        self.torch, self.model, self.requests = torch, model, requests
        self.block, self.budget, self.chunk, self.window = block, budget, chunk, window
        self.kv = dev.DeviceKvPool.empty(model.layers, slots, model.kv_heads, model.dim, block)
        self.free = list(range(slots))
        self.workspace = None

    def i32(self, values):
        return self.torch.tensor(list(values), dtype=self.torch.int32, device="cuda")

    def step(self):
        """One batch over all requests that are here; returns its size."""
        torch, m = self.torch, self.model
        live = [r for r in self.requests if r.away is None]
        rows = [r.take(self.chunk) for r in live]
        for r, new in zip(live, rows):
            r.cached += len(new)
            more = -(-r.cached // self.block) - len(r.slots)
            r.slots += [self.free.pop(0) for _ in range(more)]
            pad = torch.zeros(more, device="cuda")
            r.weight = pad if r.weight is None else torch.cat([r.weight, pad])
        counts = [len(new) for new in rows]
        tokens = sum(counts)
        offsets = self.i32(np.concatenate([[0], np.cumsum(counts)]))
        entries = self.i32(np.concatenate([[0], np.cumsum([len(r.slots) for r in live])]))
        self.length = self.i32(r.cached for r in live)
        self.entries, self.slots = entries, self.i32(s for r in live for s in r.slots)
        self.weight = torch.cat([r.weight for r in live])
        positions = self.i32(p for r, c in zip(live, counts) for p in range(r.seen, r.seen + c))
        batch = dev.KvBatch(offsets, self.length, entries, self.slots, tokens, max(counts))

        x = m.embed[self.i32(t for new in rows for t in new).long()]
        q = torch.empty(tokens, m.heads, m.dim, dtype=x.dtype, device="cuda")
        y = torch.empty_like(q)
        for layer in range(m.layers):
            # the projection's rows are read in place, by their strides
            qkv = (x @ m.qkv[layer]).view(tokens, m.heads + 2 * m.kv_heads, m.dim)
            dev.DeviceKvAppend(self.kv, batch, qkv[:, :m.heads], qkv[:, m.heads:m.heads + m.kv_heads],
                               qkv[:, m.heads + m.kv_heads:], q, positions, m.freq,
                               rope_scale=m.rope_scale, layer=layer).run()
            last = layer == m.layers - 1
            read = dev.DeviceAttention(self.kv, batch, q, y, m.dim ** -0.5,
                                       block_weight=self.weight if last else None,
                                       weight_window=self.window, layer=layer,
                                       workspace=self.workspace if not last else None)
            if not last:
                self.workspace = read.workspace if layer == 0 else self.workspace
            read.run()
            x = torch.nn.functional.rms_norm(x + y.view(tokens, -1) @ m.out[layer], x.shape[-1:])
        self.workspace = None  # the next batch has another size
        ends = (offsets[1:] - 1).long()
        made = (x[ends] @ m.embed.t()).argmax(-1).tolist()
        self.kv.check()
        for i, (r, c) in enumerate(zip(live, counts)):
            r.seen += c
            first = int(entries[i])
            r.weight = self.weight[first:first + len(r.slots)].clone()
            if r.seen >= len(r.prompt) + len(r.made):
                r.made.append(made[i])
        self.last = dict(live=live, q=q, y=y, offsets=offsets, counts=counts)
        return tokens

    def evict(self):
        """Requests over the budget keep their first block, the newest two and
        of the others those that were read most."""
        live = self.last["live"]
        if max(len(r.slots) for r in live) <= self.budget:
            return 0
        op = dev.DeviceKvEvict(self.block, self.length, self.entries, self.slots, self.weight,
                               self.i32([self.budget] * len(live)), sink=1, recent=2)
        op.run()
        op.check()
        at, kept = op.row_offsets_out.tolist(), op.slots_out.tolist()
        gone = op.freed[:int(op.n_freed)].tolist()
        for i, (r, length) in enumerate(zip(live, op.kv_len_out.tolist())):
            r.cached, r.slots = length, kept[at[i]:at[i + 1]]
            r.weight = op.weight_out[at[i]:at[i + 1]].clone()
        self.free += gone
        return len(gone)

    def move(self, r, slots, staging, copy):
        n = len(slots)
        moves = np.zeros(n, dev.MOVE_DTYPE)
        moves["pool_slot"], moves["staging_slot"] = slots, np.arange(n)
        m = self.torch.from_numpy(moves.view(np.int32).copy()).cuda()
        count = self.i32([n])
        rc = copy(self.kv.c_pool, staging.data_ptr(), n, m.data_ptr(), count.data_ptr(), n,
                  self.kv.status.data_ptr(), dev.stream_handle())
        if rc:
            raise RuntimeError(cx.cascade_strerror(rc))
        self.kv.check()

    def spill(self, r):
        size = 2 * self.model.layers * self.kv.chunk_bytes
        staging = self.torch.empty(len(r.slots) * size, dtype=self.torch.uint8, device="cuda")
        self.move(r, r.slots, staging, cx.cascade_pack)
        self.free += r.slots
        r.away = staging

    def restore(self, r):
        r.slots = [self.free.pop(0) for _ in r.slots]
        self.move(r, r.slots, r.away, cx.cascade_unpack)
        r.away = None


def serve(requests=6, tokens=24, budget=64, longest=2000, layers=3, heads=32, kv_heads=8, dim=128,
          seed=0, tell=print):
    import torch
    rng = np.random.default_rng(seed)
    model = Model(layers, heads, kv_heads, dim, 1024, seed)
    lengths = rng.integers(1, longest + 1, requests)
    todo = [Request(rng.integers(0, 1024, n).tolist()) for n in lengths]
    server = Server(model, todo, requests * (budget + 32), budget)
    turn = 0
    while any(len(r.made) < tokens for r in todo):
        began = time.perf_counter()
        rows = server.step()
        dropped = server.evict()
        torch.cuda.synchronize()
        took = time.perf_counter() - began
        if turn == 3:
            server.spill(todo[0])
        if turn == 5:
            server.restore(todo[0])
        tell(f"batch {turn}: {rows} tokens, {sum(len(r.slots) for r in todo)} blocks cached, "
             f"{dropped} dropped, {1e3 * took:.2f} ms")
        turn += 1
    for i, r in enumerate(todo):
        tell(f"request {i}: {len(r.prompt)} + {len(r.made)} tokens, {len(r.slots)} blocks, "
             f"ends {r.made[-4:]}")
    return server


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("requests", 6), ("tokens", 24), ("budget", 64), ("longest", 2000)):
        ap.add_argument("--" + name, type=int, default=default)
    serve(**vars(ap.parse_args()))
