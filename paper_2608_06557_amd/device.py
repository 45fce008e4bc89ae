"""Device-memory plumbing around the C ABI, using torch for allocation and
streams only.  Uploads a workload (numpy arrays from ``synth``), holds the
output and workspace buffers, enqueues ``cascade_step`` / ``cascade_pack`` /
``cascade_unpack`` and reads results back."""
from __future__ import annotations

import numpy as np

from . import cascade as cx

REQ_FIELDS = [("id", np.int64), ("slo_class", np.uint8), ("state", np.uint8),
              ("queue_tier", np.uint8), ("prefix_tier", np.uint8), ("arrival_ns", np.int64),
              ("n_in", np.int32), ("n_out_pred", np.int32), ("n_prefix", np.int32),
              ("n_progress", np.int32)]
MOVE_DTYPE = np.dtype([("req", np.int32), ("blk", np.int32), ("pool_slot", np.int32),
                       ("staging_slot", np.int32)])


def _torch():
    import torch
    return torch


def to_device(a: np.ndarray, device, dtype=None):
    """Upload an array; empty arrays become a 1-element buffer so that every
    pointer handed to the library is valid."""
    torch = _torch()
    a = np.ascontiguousarray(a if dtype is None else a.astype(dtype, copy=False))
    if a.dtype == np.uint64:
        a = a.view(np.int64)
    if a.size == 0:
        a = np.zeros(1, a.dtype)
    return torch.from_numpy(a.copy()).to(device)


def stream_handle(stream=None) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    # torch.cuda.current_stream().cuda_stream, which takes 2.9 us where this takes 0.3
    torch = _torch()
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


class DeviceStep:
    """Buffers for one workload and its cascade_step outputs."""

    def __init__(self, w: dict, device="cuda:0", slot_cap: int | None = None,
                 unpack_cap: int | None = None, pack_cap: int | None = None):
        torch = _torch()
        self.device = torch.device(device)
        self.n = n = int(len(w["id"]))
        p = w["params"]
        self.params = cx.make_params(p)
        self.num_blocks = int(p["num_blocks"])
        self.inp = {k: to_device(np.asarray(w[k]), self.device, dt) for k, dt in REQ_FIELDS}
        self.ro = to_device(np.asarray(w["row_offsets"]), self.device, np.int32)
        self.slots = to_device(np.asarray(w["slots"]), self.device, np.int32)
        self.free = to_device(np.asarray(w["free_slots"]), self.device, np.int32)
        self.n_free = int(len(w["free_slots"]))
        # shared-prefix restores: a prefix_group array in the workload
        self.pg = (to_device(np.asarray(w["prefix_group"]), self.device, np.int32)
                   if w.get("prefix_group") is not None else None)
        nb = self.num_blocks
        self.caps = (nb if slot_cap is None else slot_cap, nb if unpack_cap is None else unpack_cap,
                     nb if pack_cap is None else pack_cap)
        nn = max(n, 1)
        z = lambda k, dt: torch.zeros(max(k, 1), dtype=dt, device=self.device)
        self.out = {"budget_ns": z(nn, torch.int64), "action": z(nn, torch.uint8),
                    "queue_tier_out": z(nn, torch.uint8), "tokens_granted": z(nn, torch.int32),
                    "restore_blocks": z(nn, torch.int32), "order": z(nn, torch.int32),
                    "alloc_begin": z(nn, torch.int32), "alloc_count": z(nn, torch.int32),
                    "admitted": z(nn, torch.int32)}
        self.slot_list = z(self.caps[0], torch.int32)
        self.unpack_moves = z(4 * max(self.caps[1], 1), torch.int32)
        self.pack_moves = z(4 * max(self.caps[2], 1), torch.int32)
        self.unpack_hazard = z(self.caps[1], torch.int32)
        self.pack_hazard = z(self.caps[2], torch.int32)
        self.info = z(cx.INFO_LEN, torch.int32)
        if self.pg is not None:
            self.out["share_leader"] = z(nn, torch.int32)
        self.ws_bytes = cx.cascade_step_workspace_bytes(n)
        self.ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.device)
        self.ws_ptr = (self.ws.data_ptr() + 255) & ~255

        self.c_req = cx.Requests(n, *[self.inp[k].data_ptr() for k, _ in REQ_FIELDS],
                                 self.pg.data_ptr() if self.pg is not None else None)
        self.c_table = cx.BlockTable(self.ro.data_ptr(), self.slots.data_ptr())
        self.c_tier = cx.TierState(self.num_blocks, self.n_free, self.free.data_ptr())
        o = self.out
        self.c_out = cx.Outputs(
            o["budget_ns"].data_ptr(), o["action"].data_ptr(), o["queue_tier_out"].data_ptr(),
            o["tokens_granted"].data_ptr(), o["restore_blocks"].data_ptr(), o["order"].data_ptr(),
            o["alloc_begin"].data_ptr(), o["alloc_count"].data_ptr(), o["admitted"].data_ptr(),
            self.slot_list.data_ptr(), self.unpack_moves.data_ptr(), self.pack_moves.data_ptr(),
            self.caps[0], self.caps[1], self.caps[2], self.info.data_ptr(),
            self.unpack_hazard.data_ptr(), self.pack_hazard.data_ptr(),
            o["share_leader"].data_ptr() if self.pg is not None else None)

    def run(self, stream=None) -> int:
        """Enqueue one step; returns the host-side return code."""
        return cx.cascade_step(self.c_req, self.c_table, self.c_tier, self.params, self.c_out,
                               self.ws_ptr, self.ws_bytes, stream_handle(stream))

    def run_noalloc(self, stream=None) -> int:
        """The same step through cascade_step_noalloc (no workspace)."""
        return cx.cascade_step_noalloc(self.c_req, self.c_table, self.c_tier, self.params,
                                       self.c_out, stream_handle(stream))

    def n_unpack_ptr(self) -> int:
        return self.info.data_ptr() + 4 * cx.INFO_N_UNPACK

    def n_pack_ptr(self) -> int:
        return self.info.data_ptr() + 4 * cx.INFO_N_PACK

    def fetch(self) -> dict:
        """Synchronise and return every output as numpy (trimmed to counts)."""
        torch = _torch()
        torch.cuda.synchronize(self.device)
        info = self.info.cpu().numpy()
        n = self.n
        res = {k: v.cpu().numpy()[:n] for k, v in self.out.items()}
        res["status"] = int(info[cx.INFO_STATUS])
        res["n_admitted"] = int(info[cx.INFO_N_ADMITTED])
        res["n_slot_list"] = int(info[cx.INFO_N_SLOT_LIST])
        res["n_unpack"] = int(info[cx.INFO_N_UNPACK])
        res["n_pack"] = int(info[cx.INFO_N_PACK])
        res["admitted"] = res["admitted"][:res["n_admitted"]]
        res["slot_list"] = self.slot_list.cpu().numpy()[:min(res["n_slot_list"], self.caps[0])]
        um = self.unpack_moves.cpu().numpy().view(MOVE_DTYPE)
        pm = self.pack_moves.cpu().numpy().view(MOVE_DTYPE)
        res["unpack_moves"] = um[:min(res["n_unpack"], self.caps[1])]
        res["pack_moves"] = pm[:min(res["n_pack"], self.caps[2])]
        res["unpack_hazard"] = self.unpack_hazard.cpu().numpy()[:len(res["unpack_moves"])]
        res["pack_hazard"] = self.pack_hazard.cpu().numpy()[:len(res["pack_moves"])]
        return res


def kv_pool_struct(base_ptr: int, geom: dict) -> cx.KvPool:
    return cx.KvPool(base_ptr, int(geom["num_layers"]), int(geom["num_blocks"]),
                     int(geom["chunk_bytes"]), int(geom["layer_stride"]),
                     int(geom["kv_stride"]), int(geom["slot_stride"]))


def fill_pattern_(t, seed: int, word_offset: int = 0, chunk_words: int = 1 << 26,
                  progress=None) -> None:
    """Fill a uint8 device tensor with the counter-based 32-bit pattern of
    ``synth.hash32_torch`` (word k holds hash32(word_offset + k, seed)).
    ``progress(msg)``, if given, is called about every 16 GB."""
    torch = _torch()
    from .synth import hash32_torch
    w = t.view(torch.int32)
    nw = w.numel()
    every = max(1, (4 << 30) // chunk_words)
    for k, s in enumerate(range(0, nw, chunk_words)):
        e = min(nw, s + chunk_words)
        idx = torch.arange(word_offset + s, word_offset + e, device=t.device, dtype=torch.int64)
        h = hash32_torch(idx, seed)
        w[s:e] = (h - ((h >> 31) << 32)).to(torch.int32)
        if progress is not None and (k + 1) % every == 0:
            torch.cuda.synchronize(t.device)
            progress(f"filled {4 * e / 1e9:.0f} of {4 * nw / 1e9:.0f} GB")


def index_capacity(n_entries: int) -> int:
    """Slots for an index of n_entries facts: a power of two, load <= 1/2."""
    cap = 64
    while cap < 2 * max(n_entries, 1):
        cap *= 2
    return cap


class DevicePrefix:
    """Device buffers of one prefix-hit lookup: the index built from
    (hash, tier) facts and the requests' block-hash CSR."""

    def __init__(self, pw: dict, device="cuda:0", capacity: int | None = None):
        torch = _torch()
        self.device = torch.device(device)
        self.n = int(len(pw["n_in"]))
        self.n_entries = int(len(pw["index_hashes"]))
        self.capacity = capacity or index_capacity(self.n_entries)
        self.bt = int(pw["block_tokens"])
        nbytes = cx.cascade_prefix_index_bytes(self.capacity)
        assert nbytes > 0, self.capacity
        self.index = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.ih = to_device(np.asarray(pw["index_hashes"]), self.device)
        self.it = to_device(np.asarray(pw["index_tiers"]), self.device, np.uint8)
        self.off = to_device(np.asarray(pw["block_offsets"]), self.device, np.int32)
        self.bh = to_device(np.asarray(pw["block_hashes"]), self.device)
        self.n_in = to_device(np.asarray(pw["n_in"]), self.device, np.int32)
        self.n_prefix = torch.zeros(max(self.n, 1), dtype=torch.int32, device=self.device)
        self.tier = torch.zeros(max(self.n, 1), dtype=torch.uint8, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)

    def build(self, stream=None) -> int:
        s = stream_handle(stream)
        rc = cx.cascade_prefix_index_clear(self.index.data_ptr(), self.capacity, s)
        return rc or cx.cascade_prefix_index_insert(self.index.data_ptr(), self.capacity,
                                                    self.ih.data_ptr(), self.it.data_ptr(),
                                                    self.n_entries, self.status.data_ptr(), s)

    def probe(self, stream=None) -> int:
        return cx.cascade_prefix_probe(self.index.data_ptr(), self.capacity, self.n,
                                       self.off.data_ptr(), self.bh.data_ptr(),
                                       self.n_in.data_ptr(), self.bt, self.n_prefix.data_ptr(),
                                       self.tier.data_ptr(), self.status.data_ptr(),
                                       stream_handle(stream))

    def fetch(self) -> dict:
        torch = _torch()
        torch.cuda.synchronize(self.device)
        return {"status": int(self.status.item()),
                "n_prefix": self.n_prefix.cpu().numpy()[:self.n],
                "prefix_tier": self.tier.cpu().numpy()[:self.n]}


def event_handles(k: int, stream=None) -> list:
    """k HIP events (torch-owned), recorded once so that each has a handle."""
    torch = _torch()
    evs = [torch.cuda.Event() for _ in range(k)]
    s = stream if stream is not None else torch.cuda.current_stream()
    for e in evs:
        e.record(s)
    torch.cuda.synchronize()
    return evs, [int(e.cuda_event) for e in evs]


def index_facts(keys: np.ndarray, masks: np.ndarray):
    """(hash, tier) facts whose insertion gives each key its tier set."""
    keys = np.asarray(keys, np.uint64)
    masks = np.asarray(masks, np.uint8)
    hs, ts = [], []
    for t in range(3):
        sel = (masks >> t) & 1 == 1
        hs.append(keys[sel])
        ts.append(np.full(int(sel.sum()), t, np.uint8))
    return np.concatenate(hs), np.concatenate(ts)


def index_contents(index_bytes: np.ndarray):
    """Keys (ascending) and tier sets of the occupied slots of a device index
    read back."""
    slots = np.frombuffer(index_bytes.tobytes(), dtype=np.dtype(
        [("key", np.uint64), ("tiers", np.uint32), ("pad", np.uint32)]))
    occ = slots[slots["key"] != 0]
    order = np.argsort(occ["key"], kind="stable")
    return occ["key"][order], occ["tiers"][order]


class DeviceTiers:
    """Slot tables of the three tiers (HBM, DRAM, NVMe), the prefix index and
    the buffers of one reclamation chain HBM -> DRAM -> NVMe: each tier's
    demoted blocks are the next tier's incoming ones, one status word."""

    def __init__(self, tables: list, needs, index_keys=None, index_masks=None,
                 device="cuda:0", capacity: int | None = None):
        torch = _torch()
        self.device = torch.device(device)
        self.n = [int(len(t["block_hash"])) for t in tables]
        self.needs = [int(x) for x in needs]
        self.bh = [to_device(np.asarray(t["block_hash"], np.uint64), self.device)
                   for t in tables]
        self.lu = [to_device(np.asarray(t["last_use_ns"], np.int64), self.device)
                   for t in tables]
        self.held = [to_device(np.asarray(t["held"], np.uint8), self.device) for t in tables]
        self.tabs = [cx.TierTable(self.n[t], self.bh[t].data_ptr(), self.lu[t].data_ptr(),
                                  self.held[t].data_ptr()) for t in range(3)]
        # tier t takes at most the previous tier's outgoing capacity
        self.max_in = [0, 0, 0]
        self.max_out = [0, 0, 0]
        for t in range(3):
            self.max_in[t] = self.max_out[t - 1] if t > 0 else 0
            self.max_out[t] = self.needs[t] + self.max_in[t] if t < 2 else 0
        self.out = [torch.zeros(max(self.max_out[t], 1) * cx.DEMOTION_DTYPE.itemsize,
                                dtype=torch.uint8, device=self.device) for t in range(3)]
        self.n_out = torch.zeros(3, dtype=torch.int32, device=self.device)
        self.freed = [torch.full((max(self.needs[t], 1),), -1, dtype=torch.int32,
                                 device=self.device) for t in range(3)]
        self.placed = [torch.full((max(self.max_in[t], 1),), -1, dtype=torch.int32,
                                  device=self.device) for t in range(3)]
        self.ws_bytes = max(cx.cascade_reclaim_workspace_bytes(n) for n in self.n)
        self.ws = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.index = None
        self.capacity = 0
        if index_keys is not None:
            hs, ts = index_facts(index_keys, index_masks)
            self.capacity = capacity or index_capacity(len(index_keys))
            self.index = torch.empty(cx.cascade_prefix_index_bytes(self.capacity),
                                     dtype=torch.uint8, device=self.device)
            s = stream_handle()
            rc = cx.cascade_prefix_index_clear(self.index.data_ptr(), self.capacity, s)
            ih = to_device(hs, self.device)
            it = to_device(ts, self.device, np.uint8)
            rc = rc or cx.cascade_prefix_index_insert(self.index.data_ptr(), self.capacity,
                                                      ih.data_ptr(), it.data_ptr(), len(hs),
                                                      self.status.data_ptr(), s)
            assert rc == 0, rc
            torch.cuda.synchronize(self.device)
            assert int(self.status.item()) == 0

    def call(self, t: int, stream=None) -> int:
        """Enqueue tier t's reclamation (its incoming = tier t-1's outgoing)."""
        v = self
        inc = v.out[t - 1].data_ptr() if t > 0 else 0
        n_inc = v.n_out[t - 1:t].data_ptr() if t > 0 else 0
        return cx.cascade_tier_reclaim(
            t, v.tabs[t], v.needs[t], inc, n_inc, v.max_in[t],
            v.out[t].data_ptr() if t < 2 else 0, v.n_out[t:t + 1].data_ptr(), v.max_out[t],
            v.freed[t].data_ptr(), v.placed[t].data_ptr(),
            v.index.data_ptr() if v.index is not None else 0, v.capacity, v.ws.data_ptr(),
            v.ws_bytes, v.status.data_ptr(), stream_handle(stream))

    def run(self, stream=None, tiers=(0, 1, 2)) -> int:
        for t in tiers:
            rc = self.call(t, stream)
            if rc:
                return rc
        return 0

    def chain_args(self):
        """The chain call's arguments over the same buffers, with a workspace
        of its own (the three per-tier workspaces back to back)."""
        torch = _torch()
        if getattr(self, "ws_chain", None) is None:
            self.ws_chain_bytes = cx.cascade_tier_chain_workspace_bytes(self.n)
            self.ws_chain = torch.zeros(self.ws_chain_bytes, dtype=torch.uint8,
                                        device=self.device)
            c = cx.TierChain()
            for t in range(3):
                c.table[t] = self.tabs[t]
                c.need[t] = self.needs[t]
                c.freed[t] = self.freed[t].data_ptr()
                c.placed[t] = self.placed[t].data_ptr() if t > 0 else 0
            for t in range(2):
                c.outgoing[t] = self.out[t].data_ptr()
                c.n_outgoing_dev[t] = self.n_out[t:t + 1].data_ptr()
                c.max_outgoing[t] = self.max_out[t]
            self.chain = c
        return self.chain

    def run_chain(self, stream=None) -> int:
        """The whole chain in one cascade_tier_reclaim_chain call."""
        c = self.chain_args()
        return cx.cascade_tier_reclaim_chain(
            c, self.index.data_ptr() if self.index is not None else 0, self.capacity,
            self.ws_chain.data_ptr(), self.ws_chain_bytes, self.status.data_ptr(),
            stream_handle(stream))

    def fetch(self) -> dict:
        torch = _torch()
        torch.cuda.synchronize(self.device)
        n_out = self.n_out.cpu().numpy()
        res = {"status": int(self.status.item()), "tiers": []}
        for t in range(3):
            n_in = int(n_out[t - 1]) if t > 0 else 0
            no = int(n_out[t]) if t < 2 else 0
            out = np.frombuffer(self.out[t].cpu().numpy().tobytes(), cx.DEMOTION_DTYPE)[:no]
            res["tiers"].append({
                "freed": self.freed[t].cpu().numpy()[:self.needs[t]],
                "placed": self.placed[t].cpu().numpy()[:n_in],
                "outgoing": out, "n_outgoing": no,
                "block_hash": self.bh[t].cpu().numpy().view(np.uint64)[:self.n[t]],
                "last_use_ns": self.lu[t].cpu().numpy()[:self.n[t]]})
        if self.index is not None:
            res["index"] = index_contents(self.index.cpu().numpy())
        return res


# ------------------------------------------------------- the 8-bit KV cache

def kv_chunk_bytes(kv_heads: int, head_dim: int, block_tokens: int = 16, bounds: bool = False) -> int:
    """Bytes of one block's K or V of one layer in the 8-bit cache, with the
    bounds of its keys or without."""
    fmt = cx.KvFormat(block_tokens, kv_heads, head_dim)
    size = cx.cascade_kv_chunk_bytes(fmt)
    if size == 0:
        raise ValueError(f"no 8-bit cache of {kv_heads} heads of {head_dim} dims in blocks of "
                         f"{block_tokens} tokens")
    return size + (cx.cascade_kv_bounds_bytes(fmt) if bounds else 0)


def _raise(rc: int) -> None:
    if rc:
        raise RuntimeError(cx.cascade_strerror(rc))


def _dtype(t) -> int:
    torch = _torch()
    try:
        return {torch.bfloat16: cx.BF16, torch.float16: cx.F16}[t.dtype]
    except KeyError:
        raise TypeError(f"rows are bfloat16 or float16, not {t.dtype}") from None


def kv_rows(t) -> cx.Rows:
    """A [tokens, heads, dims] tensor of 16-bit elements, dims contiguous."""
    _dtype(t)
    if t.dim() != 3 or t.stride(2) != 1:
        raise ValueError("rows are [tokens, heads, dims] with the dims side by side")
    return cx.Rows(t.data_ptr(), t.stride(0), t.stride(1))


def _check_array(t, dtype, size: int, name: str) -> int:
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < size:
        raise ValueError(f"{name}: a contiguous tensor of at least {size} {dtype} is needed")
    return t.data_ptr()


def _check_device(device, *tensors) -> None:
    """Addresses of another device's memory, or the host's, would be read as
    this one's."""
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"a tensor lies on {t.device}, not {device}")


def _launch(call, device, stream) -> None:
    """The call on `stream`, or on the current one of the tensors' device."""
    torch = _torch()
    if device.type == "cuda" and device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            _raise(call(stream_handle(stream)))
    else:
        _raise(call(stream_handle(stream)))


class DeviceKvPool:
    """A pool of the 8-bit cache over a byte tensor [layers, 2 (K, V), slots,
    bytes]; the last dimension holds at least a chunk and may be padded.
    `bounds`: chunks hold the bounds of their keys too (DeviceKvBounds)."""

    def __init__(self, pool, kv_heads: int, head_dim: int, block_tokens: int = 16, bounds: bool = False):
        torch = _torch()
        size = kv_chunk_bytes(kv_heads, head_dim, block_tokens, bounds)
        if pool.dtype != torch.uint8 or pool.dim() != 4 or pool.shape[1] != 2 or \
                pool.shape[3] < size or pool.stride(3) != 1:
            raise ValueError(f"a uint8 tensor [layers, 2, slots, bytes >= {size}] is needed")
        self.pool, self.kv_heads, self.head_dim = pool, kv_heads, head_dim
        self.block_tokens, self.chunk_bytes, self.bounds = block_tokens, size, bounds
        self.c_format = cx.KvFormat(block_tokens, kv_heads, head_dim)
        self.c_pool = cx.KvPool(pool.data_ptr(), pool.shape[0], pool.shape[2], size,
                                pool.stride(0), pool.stride(1), pool.stride(2))
        self.status = torch.zeros(1, dtype=torch.int32, device=pool.device)

    @classmethod
    def empty(cls, layers: int, slots: int, kv_heads: int, head_dim: int, block_tokens: int = 16,
              device="cuda:0", bounds: bool = False):
        """A new pool of zeros."""
        size = kv_chunk_bytes(kv_heads, head_dim, block_tokens, bounds)
        return cls(_torch().zeros(layers, 2, slots, size, dtype=_torch().uint8, device=device),
                   kv_heads, head_dim, block_tokens, bounds)

    def check(self) -> None:
        """Synchronise and raise if a call found bad device data."""
        _raise(int(self.status.item()))


class KvBatch:
    """A ragged batch over device tensors (int32): token_offsets[n + 1],
    kv_len[n], and the block table's row_offsets[n + 1] and slots.  `tokens`
    rows, at most `most_new` of one request."""

    def __init__(self, token_offsets, kv_len, row_offsets, slots, tokens: int, most_new: int):
        i32 = _torch().int32
        n = int(kv_len.numel())
        self.tensors = (token_offsets, kv_len, row_offsets, slots)
        _check_device(kv_len.device, *self.tensors)
        self.n, self.tokens = n, int(tokens)
        self.c_batch = cx.KvBatch(n, tokens, most_new, slots.numel(),
                                  _check_array(token_offsets, i32, n + 1, "token_offsets"),
                                  _check_array(kv_len, i32, n, "kv_len"))
        self.c_table = cx.BlockTable(_check_array(row_offsets, i32, n + 1, "row_offsets"),
                                     _check_array(slots, i32, 0, "slots"))


def rope_frequencies(rotary_dim: int, base: float = 10000.0, kind: int = cx.ROPE_PLAIN,
                     factor: float = 1.0, original_len: float = 0.0, low: float = 1.0,
                     high: float = 4.0, device="cuda:0"):
    """(frequency tensor, scale) of rotary positions, see
    cascade_rope_frequencies."""
    rc, freq, scale = cx.cascade_rope_frequencies(
        cx.RopeSpec(kind, rotary_dim, base, factor, original_len, low, high))
    _raise(rc)
    return to_device(freq, device), scale


class DeviceKvAppend:
    """cascade_kv_append with its arguments laid out: `run` writes k and v
    [tokens, KV heads, dims] into `layer` and the turned queries into q_out.
    freq None: no rotation; q None: no queries."""

    def __init__(self, kv: DeviceKvPool, batch: KvBatch, q, k, v, q_out=None, positions=None,
                 freq=None, interleaved: bool = False, rope_scale: float = 1.0, layer: int = 0):
        torch = _torch()
        for t, heads in ((k, kv.kv_heads), (v, kv.kv_heads), (q, None), (q_out, None)):
            if t is not None and (t.shape[0] < batch.tokens or t.shape[2] != kv.head_dim or
                                  t.dtype != k.dtype or t.shape[1] != (heads or q.shape[1])):
                raise ValueError("rows do not fit the batch, the heads or each other")
        self.kv, self.batch, self.layer = kv, batch, layer
        self.tensors = (q, k, v, q_out, positions, freq)
        _check_device(kv.pool.device, *self.tensors, *batch.tensors)
        self.dtype, self.q_heads = _dtype(k), 0 if q is None else q.shape[1]
        self.c_rows = [None if t is None else kv_rows(t) for t in (q, q_out, k, v)]
        self.c_rope, self.positions = None, None
        if freq is not None:
            self.c_rope = cx.Rope(2 * freq.numel(), int(interleaved),
                                  _check_array(freq, torch.int64, 0, "freq"), rope_scale)
            self.positions = _check_array(positions, torch.int32, batch.tokens, "positions")
        self._call = cx.kv_call("cascade_kv_append", kv.c_pool, layer, kv.c_format, batch.c_batch,
                                batch.c_table, self.dtype, self.q_heads, *self.c_rows,
                                self.c_rope, self.positions, kv.status.data_ptr())

    def run(self, stream=None) -> None:
        _launch(self._call, self.kv.pool.device, stream)


class DeviceAttention:
    """cascade_attention with its arguments and workspace laid out: `run`
    writes the attention of q [tokens, query heads, dims] over `layer` to out,
    and lse [tokens, query heads] and block_weight (one per table entry, added
    to) where they are given.  A workspace may be shared by calls that follow
    each other on one stream."""

    def __init__(self, kv: DeviceKvPool, batch: KvBatch, q, out, scale: float,
                 softcap: float = 0.0, lse=None, block_weight=None, weight_window: int = 0,
                 layer: int = 0, workspace=None):
        torch = _torch()
        if q.shape != out.shape or q.dtype != out.dtype or q.shape[0] < batch.tokens or \
                q.shape[2] != kv.head_dim:
            raise ValueError("q and out do not fit the batch, the pool or each other")
        self.kv, self.batch, self.layer = kv, batch, layer
        self.tensors = (q, out, lse, block_weight)
        _check_device(kv.pool.device, *self.tensors, *batch.tensors, workspace)
        heads, f32 = q.shape[1], torch.float32
        weighs = block_weight is not None and batch.c_batch.n_entries > 0  # or nothing to add to
        self.c_args = cx.Attention(
            _dtype(q), heads, scale, softcap, kv_rows(q), kv_rows(out),
            None if lse is None else _check_array(lse, f32, batch.tokens * heads, "lse"),
            _check_array(block_weight, f32, batch.c_batch.n_entries, "block_weight") if weighs else None,
            weight_window if weighs else 0)
        self.ws_bytes = cx.cascade_attention_workspace_bytes(kv.c_format, batch.c_batch, heads,
                                                             self.c_args.weight_window)
        if self.ws_bytes == 0:
            raise ValueError("query heads or weight_window outside the domain")
        if workspace is None:
            workspace = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=q.device)
        self.workspace = workspace
        self.ws_ptr = (workspace.data_ptr() + 255) & ~255
        self.ws_bytes = workspace.data_ptr() + workspace.numel() - self.ws_ptr
        self._call = cx.kv_call("cascade_attention", kv.c_pool, layer, kv.c_format, batch.c_batch,
                                batch.c_table, self.c_args, self.ws_ptr, self.ws_bytes,
                                kv.status.data_ptr())

    def run(self, stream=None) -> None:
        _launch(self._call, self.kv.pool.device, stream)


def _workspace(workspace, size: int, device):
    """(tensor, its first address on 256 bytes, bytes from there) of a call's
    workspace, a new one if none is given."""
    torch = _torch()
    if workspace is None:
        workspace = torch.empty(size + 256, dtype=torch.uint8, device=device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("a workspace is a contiguous uint8 tensor")
    at = (workspace.data_ptr() + 255) & ~255
    return workspace, at, max(workspace.data_ptr() + workspace.numel() - at, 0)


class DeviceSharedAttention:
    """cascade_attention_shared with its arguments and workspace laid out:
    DeviceAttention of a batch whose neighbours share their first tokens.
    `leader` (int32, one per request) names the first request of each one's
    group and `shared_len` there the tokens that the group shares;
    `most_shared` is the most new tokens of one group."""

    def __init__(self, kv: DeviceKvPool, batch: KvBatch, leader, shared_len, most_shared: int, q, out,
                 scale: float, softcap: float = 0.0, lse=None, layer: int = 0, workspace=None):
        torch = _torch()
        if q.shape != out.shape or q.dtype != out.dtype or q.shape[0] < batch.tokens or \
                q.shape[2] != kv.head_dim:
            raise ValueError("q and out do not fit the batch, the pool or each other")
        self.kv, self.batch, self.layer = kv, batch, layer
        self.tensors = (q, out, lse, leader, shared_len)
        _check_device(kv.pool.device, *self.tensors, *batch.tensors, workspace)
        heads, i32 = q.shape[1], torch.int32
        self.c_args = cx.Attention(
            _dtype(q), heads, scale, softcap, kv_rows(q), kv_rows(out),
            None if lse is None else _check_array(lse, torch.float32, batch.tokens * heads, "lse"), None, 0)
        self.c_shared = cx.Shared(_check_array(leader, i32, batch.n, "leader"),
                                  _check_array(shared_len, i32, batch.n, "shared_len"), most_shared)
        size = cx.cascade_attention_shared_workspace_bytes(kv.c_format, batch.c_batch, heads)
        if size == 0:
            raise ValueError("query heads outside the domain")
        self.workspace, self.ws_ptr, self.ws_bytes = _workspace(workspace, size, q.device)
        self._call = cx.kv_call("cascade_attention_shared", kv.c_pool, layer, kv.c_format, batch.c_batch,
                                batch.c_table, self.c_args, self.c_shared, self.ws_ptr, self.ws_bytes,
                                kv.status.data_ptr())

    def run(self, stream=None) -> None:
        _launch(self._call, self.kv.pool.device, stream)


def _needs_bounds(kv: DeviceKvPool) -> None:
    if not kv.bounds:
        raise ValueError("the pool's chunks hold no bounds: make it with bounds=True")


class DeviceKvBounds:
    """cascade_kv_bounds with its arguments laid out: `run` brings the bounds of
    the batch's keys in `layer` up to date, in the blocks of the new tokens or,
    with `whole`, in all blocks."""

    def __init__(self, kv: DeviceKvPool, batch: KvBatch, whole: bool = False, layer: int = 0):
        _needs_bounds(kv)
        self.kv, self.batch, self.layer = kv, batch, layer
        _check_device(kv.pool.device, *batch.tensors)
        self._call = cx.kv_call("cascade_kv_bounds", kv.c_pool, layer, kv.c_format, batch.c_batch,
                                batch.c_table, int(whole), kv.status.data_ptr())

    def run(self, stream=None) -> None:
        _launch(self._call, self.kv.pool.device, stream)


def _selection(selected, kv: DeviceKvPool, batch: KvBatch) -> int:
    """Address of a selection [tokens, KV heads, blocks]."""
    if selected.dim() != 3 or selected.shape[0] < batch.tokens or selected.shape[1] != kv.kv_heads or \
            selected.shape[2] < 1:
        raise ValueError("a selection is [tokens, KV heads, blocks]")
    return _check_array(selected, _torch().int32, 0, "selected")


class DeviceKvSelect:
    """cascade_kv_select with its arguments and workspace laid out: `run` writes
    the blocks that q [tokens, query heads, dims] reads in `layer` to `selected`
    (int32 [tokens, KV heads, blocks]), the first `sink` and the last `recent` among
    them.  The pool's bounds have to be up to date (DeviceKvBounds).  `most_blocks`,
    if it is known, is the most blocks of one request: single tokens beside a chunk
    need a fraction of the workspace then.  By a smaller workspace than its own the
    tokens are taken in runs."""

    def __init__(self, kv: DeviceKvPool, batch: KvBatch, q, selected, sink: int = 0, recent: int = 1,
                 layer: int = 0, workspace=None, most_blocks: int = 0):
        _needs_bounds(kv)
        if q.shape[0] < batch.tokens or q.shape[2] != kv.head_dim:
            raise ValueError("q does not fit the batch or the pool")
        self.kv, self.batch, self.layer = kv, batch, layer
        self.tensors = (q, selected)
        _check_device(kv.pool.device, *self.tensors, *batch.tensors, workspace)
        self.c_args = cx.Select(_dtype(q), q.shape[1], selected.shape[-1], sink, recent, kv_rows(q),
                                _selection(selected, kv, batch), most_blocks)
        size = cx.cascade_kv_select_workspace_bytes(kv.c_format, batch.c_batch)
        if most_blocks > 0:
            size = min(size, 256 + 4 * batch.tokens * kv.kv_heads * (-(-most_blocks // 16) * 16))
        self.workspace, self.ws_ptr, self.ws_bytes = _workspace(workspace, size, q.device)
        self._call = cx.kv_call("cascade_kv_select", kv.c_pool, layer, kv.c_format, batch.c_batch,
                                batch.c_table, self.c_args, self.ws_ptr, self.ws_bytes,
                                kv.status.data_ptr())

    def run(self, stream=None) -> None:
        _launch(self._call, self.kv.pool.device, stream)


class DeviceSelectedAttention:
    """cascade_attention_selected with its arguments and workspace laid out:
    DeviceAttention of each token and KV head over the blocks that `selected`
    (int32 [tokens, KV heads, blocks], as DeviceKvSelect writes it) lists."""

    def __init__(self, kv: DeviceKvPool, batch: KvBatch, q, selected, out, scale: float,
                 softcap: float = 0.0, lse=None, layer: int = 0, workspace=None):
        torch = _torch()
        if q.shape != out.shape or q.dtype != out.dtype or q.shape[0] < batch.tokens or \
                q.shape[2] != kv.head_dim:
            raise ValueError("q and out do not fit the batch, the pool or each other")
        self.kv, self.batch, self.layer = kv, batch, layer
        self.tensors = (q, out, lse, selected)
        _check_device(kv.pool.device, *self.tensors, *batch.tensors, workspace)
        heads, keep = q.shape[1], selected.shape[-1]
        self.c_args = cx.Attention(
            _dtype(q), heads, scale, softcap, kv_rows(q), kv_rows(out),
            None if lse is None else _check_array(lse, torch.float32, batch.tokens * heads, "lse"), None, 0)
        size = cx.cascade_attention_selected_workspace_bytes(kv.c_format, batch.c_batch, heads, keep)
        if size == 0:
            raise ValueError("query heads or selected blocks outside the domain")
        self.workspace, self.ws_ptr, self.ws_bytes = _workspace(workspace, size, q.device)
        self._call = cx.kv_call("cascade_attention_selected", kv.c_pool, layer, kv.c_format, batch.c_batch,
                                batch.c_table, self.c_args, _selection(selected, kv, batch), keep,
                                self.ws_ptr, self.ws_bytes, kv.status.data_ptr())

    def run(self, stream=None) -> None:
        _launch(self._call, self.kv.pool.device, stream)


class DeviceKvEvict:
    """cascade_kv_evict with its arguments laid out: `run` writes the tight
    table of what stays to kv_len_out, row_offsets_out, slots_out and
    weight_out, and the dropped slots to freed, n_freed of them (`out`: these
    six tensors, else new ones)."""

    def __init__(self, block_tokens: int, kv_len, row_offsets, slots, block_weight, keep_blocks,
                 sink: int = 0, recent: int = 1, out=None):
        torch = _torch()
        i32, n, entries = torch.int32, int(kv_len.numel()), int(slots.numel())
        if out is None:
            new = lambda k, dt=i32: torch.zeros(max(k, 1), dtype=dt, device=kv_len.device)
            out = (new(n), new(n + 1), new(entries), new(entries, torch.float32), new(entries),
                   new(1))
        self.tensors = (kv_len, row_offsets, slots, block_weight, keep_blocks)
        _check_device(kv_len.device, *self.tensors, *out)
        self.kv_len_out, self.row_offsets_out, self.slots_out = out[:3]
        self.weight_out, self.freed, self.n_freed = out[3:]
        p = _check_array
        self.status = torch.zeros(1, dtype=i32, device=kv_len.device)
        self.c_table = cx.BlockTable(p(row_offsets, i32, n + 1, "row_offsets"),
                                     p(slots, i32, 0, "slots"))
        self.c_args = cx.Evict(
            n, entries, block_tokens, sink, recent, p(kv_len, i32, n, "kv_len"),
            p(keep_blocks, i32, n, "keep_blocks"),
            p(block_weight, torch.float32, entries, "block_weight"),
            p(out[0], i32, n, "kv_len_out"), p(out[1], i32, n + 1, "row_offsets_out"),
            p(out[2], i32, entries, "slots_out"), p(out[3], torch.float32, entries, "weight_out"),
            p(out[4], i32, entries, "freed"), p(out[5], i32, 1, "n_freed"))
        self._call = cx.kv_call("cascade_kv_evict", self.c_table, self.c_args,
                                self.status.data_ptr())

    def run(self, stream=None) -> None:
        _launch(self._call, self.status.device, stream)

    def check(self) -> None:
        """Synchronise and raise if a call found bad device data."""
        _raise(int(self.status.item()))
