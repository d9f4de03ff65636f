"""Device-memory plumbing around the C-ABI calls: allocates the KV pool / workspace with torch,
uploads a workload's wGraph, node KV and paths, and forwards to the library.  No attention or
table arithmetic lives here; PyTorch only supplies memory and streams."""
from __future__ import annotations

import os
import weakref
from typing import NamedTuple, Optional

import numpy as np
import torch

from . import binding as B
from . import workloads as W

GUARD_BYTES = 4096   # canary band on either side of every buffer the library is given
GUARD_VALUE = 0xA5
_live = weakref.WeakSet()


def verify_all_guards() -> None:
    """Checks the canary bands of every live PathAttention (an out-of-bounds write by a kernel lands
    there first); raises AssertionError naming the buffer."""
    for pa in list(_live):
        pa.verify_guards()


def _bits_to_tensor(bits: np.ndarray, device) -> torch.Tensor:
    return torch.from_numpy(bits.view(np.int16)).to(device).view(torch.bfloat16)


def tensor_to_f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().to(torch.float64).cpu().numpy()


class Projection:
    """A shared weight [out, in] with the low-rank adapters that rows may name: a [adapters, rank, in], b [adapters, out, rank],
    scale fp32 [adapters] (None: 1).  bf16, on one device; kept alive here.  The weight's rows may lie apart, the adapters are contiguous.  b with an infinity or a
    NaN is refused: such an adapter gives no results of use and makes a call slow.  (Looked at here, once; written to it later they stay in its own rows.)"""

    def __init__(self, weight: torch.Tensor, a: Optional[torch.Tensor] = None, b: Optional[torch.Tensor] = None,
                 scale: Optional[torch.Tensor] = None):
        if weight.dtype != torch.bfloat16 or weight.dim() != 2 or weight.stride(1) != 1 or not weight.is_cuda:
            raise ValueError("weight: a bf16 tensor [out, in] on a CUDA device, entries of a row next to each other")
        out_dim, in_dim = weight.shape
        adapters = rank = 0
        if a is not None or b is not None:
            if a is None or b is None or a.dim() != 3 or b.dim() != 3 or a.dtype != torch.bfloat16 or b.dtype != torch.bfloat16 or \
                    a.shape[2] != in_dim or tuple(b.shape) != (a.shape[0], out_dim, a.shape[1]) or not a.is_contiguous() or \
                    not b.is_contiguous() or a.device != weight.device or b.device != weight.device:
                raise ValueError(f"a, b: contiguous bf16 tensors [adapters, rank, {in_dim}] and [adapters, {out_dim}, rank] on {weight.device}")
            adapters, rank = a.shape[:2]
            if b.numel() and not bool(torch.isfinite(torch.stack(torch.aminmax(b))).all()):  # (a NaN comes through either)
                raise ValueError("b: finite entries")
        if scale is not None and (a is None or scale.dtype != torch.float32 or tuple(scale.shape) != (adapters,) or not scale.is_contiguous() or
                                  scale.device != weight.device):
            raise ValueError(f"scale: a contiguous fp32 tensor [{adapters}] on {weight.device}")
        self.weight, self.a, self.b, self.scale = weight, a, b, scale
        self.in_dim, self.out_dim, self.adapters, self.index = in_dim, out_dim, adapters, weight.get_device()
        self._scratch = {}
        # (a weight of one row may have any stride)
        stride = weight.stride(0) if out_dim > 1 else -(-in_dim // 8) * 8
        self.desc = B.ProjectionDesc(in_dim, out_dim, weight.data_ptr(), stride, adapters, rank, _ptr(a), _ptr(b), _ptr(scale))

    def scratch_bytes(self, rows: int) -> int:
        """gf_adapter_project_scratch_bytes."""
        n = self._scratch.get(rows)
        if n is None:
            n = self._scratch[rows] = B.gf_adapter_project_scratch_bytes(self.desc, rows)
        return n


class TokenLogprobs(NamedTuple):
    """Per row: the given token's log probability, the entropy, the log-sum-exp, and the most likely tokens with theirs."""
    logprob: Optional[torch.Tensor]
    entropy: torch.Tensor
    lse: torch.Tensor
    top_ids: torch.Tensor
    top_logprobs: torch.Tensor


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _current_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# (building a torch.cuda.Stream object costs as much as a kernel launch)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)


def _ints(t: torch.Tensor, n: int, index: int) -> bool:
    """A contiguous int32 tensor [n] on the CUDA device `index`."""
    return t.dtype is torch.int32 and t.dim() == 1 and t.numel() == n and t.is_contiguous() and t.get_device() == index


class PathAttention:
    """One wGraph handle with its pool and workspace, fed from a `workloads.Workload`."""

    def __init__(self, w: W.Workload, device: str = "cuda:0", layers: Optional[int] = None,
                 policy: Optional[tuple] = None, extra_tiles: int = 0, max_residual_nodes: int = 0,
                 kv4_nodes=(), extra_kv4_tiles: int = 0):
        """kv4_nodes: the nodes whose state is held in 4 bits (write_nodes and write_node go by it).  Either pool
        is sized for the used nodes that it holds, plus the extra tiles."""
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required (the path has no CPU fallback)")
        self.w = w
        self.dev = torch.device(device)
        torch.cuda.set_device(self.dev)
        self.layers = w.num_layers if layers is None else layers
        self.policy = policy
        chunk = policy[0] if policy is not None else 256
        used = w.used_nodes()
        self.kv4_nodes = frozenset(int(v) for v in kv4_nodes)
        node_tiles = (w.node_len[used].astype(np.int64) + B.GF_TILE_TOKENS - 1) // B.GF_TILE_TOKENS
        in4 = np.isin(used, np.fromiter(self.kv4_nodes, np.int64, len(self.kv4_nodes)))
        tiles = max(int(node_tiles[~in4].sum()) + extra_tiles, 1)
        kv4_tiles = int(node_tiles[in4].sum()) + extra_kv4_tiles
        self.pool_bytes = tiles * B.gf_pool_bytes_per_tile(w.head_dim) * w.num_kv_heads * self.layers
        self._guards = []
        # the pool must start on a 1024-byte boundary; the caching allocator only promises 512
        self.pool = self.guarded(self.pool_bytes, "kv pool", align=1024)
        pair_len = w.node_len[w.path_node].astype(np.int64)
        max_slots = int(((pair_len + chunk - 1) // chunk).sum()) + 1
        max_items = max_slots
        self.ws_bytes = B.gf_workspace_bytes(w.num_nodes, len(w.edge_src), w.num_requests,
                                             len(w.path_node), max_items, max_slots, w.num_q_heads,
                                             w.head_dim) + 64 * max_residual_nodes * self.layers + 256
        self.ws = self.guarded(self.ws_bytes, "workspace", align=256)
        st, self.g = B.gf_wgraph_create(
            num_nodes=w.num_nodes, num_shared_nodes=w.num_shared_nodes, edge_src=w.edge_src,
            edge_dst=w.edge_dst, num_layers=self.layers, num_q_heads=w.num_q_heads,
            num_kv_heads=w.num_kv_heads, head_dim=w.head_dim, kv_pool_ptr=self.pool.data_ptr(),
            kv_pool_bytes=self.pool_bytes, workspace_ptr=self.ws.data_ptr(), workspace_bytes=self.ws_bytes,
            max_residual_nodes=max_residual_nodes)
        B.check(st, "gf_wgraph_create")
        if self.kv4_nodes or kv4_tiles:
            nbytes = max(kv4_tiles, 1) * B.gf_kv4_bytes_per_tile(w.head_dim) * w.num_kv_heads * self.layers
            self.pool4 = self.guarded(nbytes, "4-bit kv pool", align=1024)
            B.check(B.gf_kv4_pool_attach(self.g, self.pool4.data_ptr(), nbytes), "gf_kv4_pool_attach")
        self.path_ptr = torch.from_numpy(w.path_ptr.astype(np.int32)).to(self.dev)
        self.path_node = torch.from_numpy(w.path_node.astype(np.int32)).to(self.dev)
        self._lib, self._index = B.lib(), self.pool.get_device()
        self.tables = None
        self._qtab = None
        _live.add(self)

    def guarded(self, nbytes: int, name: str, align: int = 256) -> torch.Tensor:
        """A uint8 device buffer of nbytes with a canary band before and after it."""
        raw = torch.empty(nbytes + 2 * GUARD_BYTES + align, dtype=torch.uint8, device=self.dev)
        lo = GUARD_BYTES + (-(raw.data_ptr() + GUARD_BYTES)) % align
        raw[lo - GUARD_BYTES:lo].fill_(GUARD_VALUE)
        raw[lo + nbytes:lo + nbytes + GUARD_BYTES].fill_(GUARD_VALUE)
        self._guards.append((name, raw, lo, nbytes))
        return raw[lo:lo + nbytes]

    # True: the results and scratch of append_slots, project and token_logprobs are guarded too, and kept until the handle is closed (for tests: GF_GUARD_OUTPUTS=1, or set
    # on a handle)
    guard_outputs = os.environ.get("GF_GUARD_OUTPUTS") == "1"

    def _guarded_new(self, shape: tuple, dtype: torch.dtype, name: str) -> torch.Tensor:
        n = int(np.prod(shape, dtype=np.int64))
        return self.guarded(n * torch.empty((), dtype=dtype).element_size(), name).view(dtype).view(shape)

    def guarded_like(self, t: torch.Tensor, name: str) -> torch.Tensor:
        return self.guarded(t.numel() * t.element_size(), name).view(t.dtype).view(t.shape)

    def verify_guards(self) -> None:
        if not self._guards:
            return
        torch.cuda.synchronize(self.dev)
        for name, raw, lo, nbytes in self._guards:
            before = raw[lo - GUARD_BYTES:lo]
            after = raw[lo + nbytes:lo + nbytes + GUARD_BYTES]
            assert bool((before == GUARD_VALUE).all()), f"canary before the {name} was overwritten"
            assert bool((after == GUARD_VALUE).all()), f"canary after the {name} was overwritten"

    def close(self):
        if self.g is not None:
            self.verify_guards()
            B.gf_wgraph_destroy(self.g)
            self.g = None
            self._guards = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def stream(self) -> int:
        return _raw_stream(self.pool.device.index)

    # ---- inputs -------------------------------------------------------------------------
    def _fill(self, key: int, count: int, out: torch.Tensor, start: int = 0):
        if self._qtab is None:
            self._qtab = torch.from_numpy(W.quantile_table().view(np.int16)).to(self.dev)
        if B.gfgen_fill_bf16(self._qtab.data_ptr(), key, start, count, out.data_ptr(), self.stream) != 0:
            raise RuntimeError("input fill kernel failed to launch")

    def write_nodes(self, source: str = "device", skip=(), only=None):
        """gf_node_kv_write for every used node (except those in `skip`; or exactly the nodes in `only`)
        and every materialised layer.  source="device" generates the bits with the fill kernel, "host"
        with numpy (identical bits)."""
        w = self.w
        used = w.used_nodes() if only is None else np.asarray(sorted(only), dtype=np.int64)
        if len(skip):
            used = used[~np.isin(used, list(skip))]
        if len(used) == 0:
            return
        per_tok = w.num_kv_heads * w.head_dim
        nmax = int(w.node_len[used].max())
        kbuf = torch.empty(nmax * per_tok, dtype=torch.bfloat16, device=self.dev)
        vbuf = torch.empty(nmax * per_tok, dtype=torch.bfloat16, device=self.dev)
        for layer in range(self.layers):
            for v in used.tolist():
                n = int(w.node_len[v])
                if source == "device":
                    self._fill(W.stream_key(w.seed, W.KIND_K, layer, v), n * per_tok, kbuf)
                    self._fill(W.stream_key(w.seed, W.KIND_V, layer, v), n * per_tok, vbuf)
                    if w.v_scale_log2:
                        vbuf[:n * per_tok].mul_(2.0 ** w.v_scale_log2)  # a power of two: exact in bf16
                    for token, kvh, row in w.planted_rows(layer, v):  # inputs with planted key rows
                        at = (token * w.num_kv_heads + kvh) * w.head_dim
                        kbuf[at:at + w.head_dim].copy_(_bits_to_tensor(row, self.dev))
                    kp, vp = kbuf.data_ptr(), vbuf.data_ptr()
                else:
                    kb, vb = w.node_kv_bits(layer, v)
                    kt, vt = _bits_to_tensor(kb, self.dev), _bits_to_tensor(vb, self.dev)
                    kp, vp = kt.data_ptr(), vt.data_ptr()
                write = B.gf_node_kv4_write if v in self.kv4_nodes else B.gf_node_kv_write
                B.check(write(self.g, v, layer, kp, vp, n, self.stream), "gf_node_kv_write")
                if source != "device":
                    torch.cuda.current_stream(self.dev).synchronize()  # kt/vt are freed next turn
        torch.cuda.current_stream(self.dev).synchronize()

    def write_node(self, node: int, layer: int, k: torch.Tensor, v: torch.Tensor) -> None:
        """gf_node_kv_write, or gf_node_kv4_write for a node of `kv4_nodes`, of bf16 tensors [tokens, Hkv, D]."""
        self._check_kv(k, v)
        write = B.gf_node_kv4_write if node in self.kv4_nodes else B.gf_node_kv_write
        B.check(write(self.g, node, layer, k.data_ptr(), v.data_ptr(), k.shape[0], self.stream), "gf_node_kv_write")

    def load_node(self, node: int, layer: int):
        """gf_node_kv_read into two new bf16 tensors [tokens, Hkv, D]; nothing is waited for."""
        st, n, _ = B.gf_node_extent(self.g, node)
        B.check(st, "gf_node_extent")
        both = self.pool.new_empty((2, n, self.w.num_kv_heads, self.w.head_dim), dtype=torch.bfloat16)
        k = both.data_ptr()
        B.check(B.gf_node_kv_read(self.g, node, layer, k, k + both.numel(), self.stream), "gf_node_kv_read")
        return both.unbind(0)

    def _check_kv(self, k: torch.Tensor, v: torch.Tensor) -> None:
        row = (self.w.num_kv_heads, self.w.head_dim)
        if k.dtype is v.dtype is torch.bfloat16 and k.shape == v.shape and k.dim() == 3 and k.shape[1:] == row and k.is_contiguous() and \
                v.is_contiguous() and k.get_device() == v.get_device() == self.pool.get_device():
            return
        raise ValueError(f"k, v: two contiguous bf16 tensors [tokens, {row[0]}, {row[1]}] on {self.pool.device}")

    def new_nodes(self):
        """The last node of every path: in an extend batch, the request's new segment."""
        w = self.w
        return [int(w.path_node[w.path_ptr[r + 1] - 1]) for r in range(w.num_requests)]

    def write_prefix_nodes(self, source: str = "device"):
        """Like write_nodes, but the requests' new segments are only reserved (their K/V arrive with
        gf_path_attention_extend_append)."""
        w = self.w
        new = set(self.new_nodes())
        self.write_nodes(source, skip=new)
        for v in sorted(new):
            B.check(B.gf_node_kv_reserve(self.g, v, int(w.node_len[v]), self.stream), "gf_node_kv_reserve")

    def new_kv(self, layer: int):
        """K and V of the new segments, request-major rows in the order of the queries: two tensors
        [num_q_rows, Hkv, D] (generated on the host, identical bits to what write_nodes stores)."""
        w = self.w
        ks, vs = [], []
        for v in self.new_nodes():
            kb, vb = w.node_kv_bits(layer, v)
            ks.append(kb)
            vs.append(vb)
        return (_bits_to_tensor(np.concatenate(ks, axis=0), self.dev), _bits_to_tensor(np.concatenate(vs, axis=0), self.dev))

    def make_q(self, layer: int, source: str = "device") -> torch.Tensor:
        w = self.w
        rows = int(w.q_row_ptr()[-1])
        if source == "device":
            q = torch.empty((rows, w.num_q_heads, w.head_dim), dtype=torch.bfloat16, device=self.dev)
            self._fill(W.stream_key(w.seed, W.KIND_Q, layer, 0), q.numel(), q)
            if w.q_scale_log2:
                q.mul_(2.0 ** w.q_scale_log2)  # a power of two: exact in bf16
            return q
        return _bits_to_tensor(w.q_bits(layer), self.dev)

    # ---- the path ---------------------------------------------------------------------------
    def build(self, mode: Optional[int] = None, deferred: bool = False):
        """gf_build_path_tables.  deferred=True (decode only) enqueues the build without waiting and
        returns None; sizes and errors are then reported by info() / status()."""
        w = self.w
        if mode is None:
            mode = B.GF_MODE_EXTEND if w.mode == "extend" else B.GF_MODE_DECODE
        if deferred:
            mode |= B.GF_MODE_DEFERRED
        st, t = B.gf_build_path_tables(self.g, w.num_requests, len(w.path_node), self.path_ptr.data_ptr(),
                                       self.path_node.data_ptr(), mode, self.policy, self.stream)
        self.tables = t
        B.check(st, "gf_build_path_tables")
        return None if deferred else B.gf_tables_info(t)

    def info(self):
        return B.gf_tables_info(self.tables)

    def decode(self, layer: int, q: torch.Tensor, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None):
        if out is None:
            out = self.guarded_like(q, "decode output")
        B.check(B.gf_path_attention_decode(self.g, self.tables, layer, q.data_ptr(), out.data_ptr(),
                                           None if lse is None else lse.data_ptr(), self.stream),
                "gf_path_attention_decode")
        return out

    def extend(self, layer: int, q: torch.Tensor, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None):
        if out is None:
            out = self.guarded_like(q, "extend output")
        B.check(B.gf_path_attention_extend(self.g, self.tables, layer, q.data_ptr(), out.data_ptr(),
                                           None if lse is None else lse.data_ptr(), self.stream),
                "gf_path_attention_extend")
        return out

    def extend_append(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                      out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
        if out is None:
            out = self.guarded_like(q, "extend output")
        B.check(B.gf_path_attention_extend_append(self.g, self.tables, layer, q.data_ptr(), k_new.data_ptr(),
                                                  v_new.data_ptr(), out.data_ptr(),
                                                  None if lse is None else lse.data_ptr(), self.stream),
                "gf_path_attention_extend_append")
        return out

    # ---- nodes that grow ---------------------------------------------------------------------
    def open_node(self, node: int, room: int) -> None:
        """gf_node_kv_open: an unwritten node gets room for that many tokens and holds none."""
        B.check(B.gf_node_kv_open(self.g, node, room, self.stream), "gf_node_kv_open")

    def close_node(self, node: int, tokens: int) -> None:
        """gf_node_kv_close: the node has this many tokens from here on."""
        B.check(B.gf_node_kv_close(self.g, node, tokens, self.stream), "gf_node_kv_close")

    def _refuse_ints(self, **tensors) -> None:
        """(The checks of the calls below stand in one expression each: a decode step makes many of them, at 0.1 us a question.)"""
        n = {name: want for name, (_, want) in tensors.items()}
        raise ValueError(", ".join(f"{name}: a contiguous int32 tensor [{want}]" for name, want in n.items()) + f" on {self.pool.device}")

    def append_slots(self, nodes: torch.Tensor, counts: torch.Tensor, num_new: int, held: Optional[torch.Tensor] = None):
        """gf_append_slots: request r gets counts[r] tokens in the open node nodes[r], behind the held[r] that stay (None: behind all
        that it holds).  Token slots of the num_new rows and the nodes' new lengths, int32.  Build the tables anew after it."""
        n, ix = nodes.numel(), self._index
        if not (_ints(nodes, n, ix) and _ints(counts, n, ix) and (held is None or _ints(held, n, ix))):
            self._refuse_ints(nodes=(nodes, "requests"), counts=(counts, "requests"), held=(held, "requests"))
        if num_new < 0:
            raise ValueError("num_new: at least 0")
        slots, lens = nodes.new_empty(num_new), torch.empty_like(nodes)
        if self.guard_outputs:
            slots, lens = self._guarded_new((num_new,), torch.int32, "slots"), self._guarded_new((n,), torch.int32, "lengths")
        st = self._lib.gf_append_slots(self.g, n, nodes.data_ptr(), None if held is None else held.data_ptr(), counts.data_ptr(), num_new,
                                       slots.data_ptr(), lens.data_ptr(), _raw_stream(ix))
        if st:
            B.check(st, "gf_append_slots")
        return slots, lens

    def append(self, layer: int, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> None:
        """gf_node_kv_append of bf16 rows [new, Hkv, D], which may be parts of wider rows (heads next to each other)."""
        n, ix, hkv, d = slots.numel(), self._index, self.w.num_kv_heads, self.w.head_dim
        ks, vs = k.stride(), v.stride()
        if not (_ints(slots, n, ix) and k.dtype is v.dtype is torch.bfloat16 and k.shape == v.shape == (n, hkv, d) and
                k.get_device() == v.get_device() == ix and ks[2] == vs[2] == 1 and (hkv == 1 or ks[1] == vs[1] == d)):
            raise ValueError(f"slots: a contiguous int32 tensor [new]; k, v: bf16 tensors [new, {hkv}, {d}], the entries of a token next to each "
                             f"other; on {self.pool.device}")
        many = n > 1  # (one row may have any stride)
        st = self._lib.gf_node_kv_append(self.g, layer, n, slots.data_ptr(), k.data_ptr(), ks[0] if many else 0, v.data_ptr(), vs[0] if many else 0,
                                         _raw_stream(ix))
        if st:
            B.check(st, "gf_node_kv_append")

    # ---- before and behind the attention -------------------------------------------------------
    def project(self, projection: Projection, x: torch.Tensor, adapters: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """gf_adapter_project: x [rows, in] times the shared weight, each row with the adapter that adapters[row] names (-1, or
        adapters None: none).  [rows, out] in bf16 or fp32, into `out` where given."""
        p, ix = projection, self._index
        xs = x.stride()
        if not (x.dtype is torch.bfloat16 and len(xs) == 2 and x.shape[1] == p.in_dim and xs[1] == 1 and x.get_device() == p.index == ix):
            raise ValueError(f"x: a bf16 tensor [rows, {p.in_dim}] on {self.pool.device} like the projection, entries of a row next to each other")
        rows = x.shape[0]
        if adapters is not None and not (p.adapters and _ints(adapters, rows, ix)):
            if not p.adapters:
                raise ValueError("adapters: the projection has none")
            self._refuse_ints(adapters=(adapters, rows))
        if out is None:
            if dtype not in (torch.bfloat16, torch.float32):
                raise ValueError("dtype: bf16 or fp32")
            out = x.new_empty(rows, p.out_dim) if dtype is torch.bfloat16 else x.new_empty(rows, p.out_dim, dtype=dtype)
            if self.guard_outputs:
                out = self._guarded_new((rows, p.out_dim), dtype, "projection")
            ys = p.out_dim
        else:
            dtype = out.dtype
            if dtype not in (torch.bfloat16, torch.float32) or out.shape != (rows, p.out_dim) or out.stride(1) != 1 or out.get_device() != ix:
                raise ValueError(f"out: a bf16 or fp32 tensor [{rows}, {p.out_dim}] on {self.pool.device}, entries of a row next to each other")
            ys = out.stride(0) if rows > 1 else p.out_dim
        if rows == 0:
            return out
        scratch, nbytes = None, 0
        if adapters is not None:
            nbytes = p.scratch_bytes(rows)
            scratch = self.guarded(nbytes, "projection scratch") if self.guard_outputs else adapters.new_empty(nbytes + 3 >> 2)
        st = self._lib.gf_adapter_project(self.g, p.desc, rows, x.data_ptr(), xs[0] if rows > 1 else p.in_dim,
                                          None if adapters is None else adapters.data_ptr(), out.data_ptr(), ys, dtype is torch.float32,
                                          None if scratch is None else scratch.data_ptr(), nbytes, _raw_stream(ix))
        if st:
            B.check(st, "gf_adapter_project")
        return out

    def token_logprobs(self, logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0) -> TokenLogprobs:
        """gf_token_logprobs of bf16 or fp32 logits [rows, vocab]: log probabilities of the given tokens (-1: none), entropy,
        log-sum-exp, and the `top` most likely tokens with their log probabilities."""
        ix, strides = self._index, logits.stride()
        fp32 = logits.dtype is torch.float32
        if not ((fp32 or logits.dtype is torch.bfloat16) and len(strides) == 2 and (strides[1] == 1 or logits.shape[1] == 1) and logits.get_device() == ix):
            raise ValueError(f"logits: a bf16 or fp32 tensor [rows, vocab] on {self.pool.device}, entries of a row next to each other")
        rows, vocab = logits.shape
        if tokens is not None and not _ints(tokens, rows, ix):
            self._refuse_ints(tokens=(tokens, rows))
        if not 0 <= top <= min(B.GF_MAX_TOP, vocab):
            raise ValueError(f"top: 0 to {min(B.GF_MAX_TOP, vocab)}")
        stats = logits.new_empty(3, rows, dtype=torch.float32)
        top_ids, top_logprobs = logits.new_empty(rows, top, dtype=torch.int32), stats.new_empty(rows, top)
        if self.guard_outputs:
            stats = self._guarded_new((3, rows), torch.float32, "token statistics")
            top_ids, top_logprobs = self._guarded_new((rows, top), torch.int32, "top ids"), self._guarded_new((rows, top), torch.float32, "top log probabilities")
        at = stats.data_ptr()
        out = B.Logprobs(None if tokens is None else at, at + 4 * rows, at + 8 * rows, top_ids.data_ptr() if top else None,
                         top_logprobs.data_ptr() if top else None)
        st = self._lib.gf_token_logprobs(self.g, rows, vocab, logits.data_ptr(), strides[0] if rows > 1 else vocab, fp32,
                                         None if tokens is None else tokens.data_ptr(), top, out, _raw_stream(ix))
        if st:
            B.check(st, "gf_token_logprobs")
        logprob, entropy, lse = stats.unbind(0)
        return TokenLogprobs(None if tokens is None else logprob, entropy, lse, top_ids, top_logprobs)

    # ---- eviction by accumulated attention weight --------------------------------------------
    def new_weights(self) -> torch.Tensor:
        """Zeroed weights for every token slot of both pools: fp32 [layers, Hkv, slots]."""
        shape = (self.layers, self.w.num_kv_heads, B.gf_weight_slots(self.g))
        buf = self.guarded(4 * shape[0] * shape[1] * shape[2], "attention weights").view(torch.float32).view(shape)
        return buf.zero_()

    def node_slot(self, node: int) -> int:
        """The first token slot of a node."""
        st, _, slot = B.gf_node_extent(self.g, node)
        B.check(st, "gf_node_extent")
        return slot

    def node_weights(self, weights: torch.Tensor, node: int) -> torch.Tensor:
        """A view of one node's weights: [layers, Hkv, tokens]."""
        st, n, slot = B.gf_node_extent(self.g, node)
        B.check(st, "gf_node_extent")
        return weights.narrow(2, slot, n)

    def clear_node_weights(self, weights: torch.Tensor, node: int) -> None:
        """Zeroes one node's weights.  A node that takes the token slots of a released one finds that one's sums there:
        call this before the first step that accumulates into it.  (The destinations of `evict` are filled by it.)"""
        self._check_weights(weights)
        self.node_weights(weights, node).zero_()

    def clear_slot_weights(self, weights: torch.Tensor, slots: torch.Tensor) -> None:
        """Zeroes the weights of the token slots that `append_slots` gave to new tokens (-1: none), which tokens taken back may have had before: call
        this before the first step that accumulates into them.  Nothing is waited for."""
        self._check_weights(weights)
        if not _ints(slots, slots.numel(), self._index):
            self._refuse_ints(slots=(slots, "new"))
        if slots.numel() == 0:
            return
        # (-1 stands for the largest slot named; where none is, all stand for slot 0, which keeps what it has)
        last = slots.amax()
        at = torch.where(slots >= 0, slots, last.clamp(min=0)).long()
        weights.index_copy_(2, at, weights.index_select(2, at).masked_fill_(last >= 0, 0.0))

    def _check_weights(self, weights: torch.Tensor) -> None:
        shape = (self.layers, self.w.num_kv_heads, B.gf_weight_slots(self.g))
        if weights.dtype != torch.float32 or weights.device != self.pool.device or not weights.is_contiguous() or \
                weights.shape != shape:
            raise ValueError(f"weights: a contiguous fp32 tensor {list(shape)} on {self.pool.device}")

    def attention_weights(self, layer: int, q: torch.Tensor, lse: torch.Tensor, weights: torch.Tensor,
                          accumulate: bool = True) -> torch.Tensor:
        """gf_path_attention_weights: adds to `weights` (or sets) what every token of the batch's paths received in
        the decode step of q and lse.  With nodes that have weights already beside new ones in a batch: accumulate, the
        new ones cleared before (clear_node_weights)."""
        self._check_weights(weights)
        rows = (self.w.num_requests, self.w.num_q_heads)
        if q.dtype != torch.bfloat16 or not q.is_contiguous() or tuple(q.shape) != rows + (self.w.head_dim,) or q.device != self.pool.device:
            raise ValueError(f"q: a contiguous bf16 tensor {[*rows, self.w.head_dim]} on {self.pool.device}")
        if lse.dtype != torch.float32 or not lse.is_contiguous() or tuple(lse.shape) != rows or lse.device != self.pool.device:
            raise ValueError(f"lse: a contiguous fp32 tensor {list(rows)} on {self.pool.device}")
        B.check(B.gf_path_attention_weights(self.g, self.tables, layer, q.data_ptr(), lse.data_ptr(), accumulate,
                                            weights.data_ptr(), self.stream), "gf_path_attention_weights")
        return weights

    def evict(self, entries, weights: torch.Tensor):
        """gf_node_kv_evict of (node, src_node, keep, keep_first, keep_last) entries; every entry's kept indices,
        int32 [layers, Hkv, kept]."""
        self._check_weights(weights)
        sizes = []
        for e in entries:
            st, n, _ = B.gf_node_extent(self.g, e[1])
            B.check(st, "gf_node_extent")
            sizes.append(max(min(n, e[2]), 0))
        hkv = self.w.num_kv_heads
        kept = self.pool.new_empty((max(self.layers * hkv * sum(sizes), 1),), dtype=torch.int32)
        B.check(B.gf_node_kv_evict(self.g, entries, weights.data_ptr(), kept.data_ptr(), self.stream), "gf_node_kv_evict")
        out, at = [], 0
        for m in sizes:
            out.append(kept.as_strided((self.layers, hkv, m), (hkv * m, m, 1), at))
            at += self.layers * hkv * m
        return out

    def read_node(self, node: int, layer: int):
        """gf_node_kv_read: (K, V) uint16 bit patterns [len, Hkv, D] of a node's layer."""
        w = self.w
        st, n, _ = B.gf_node_extent(self.g, node)
        B.check(st, "gf_node_extent")
        k = torch.empty((max(n, 1), w.num_kv_heads, w.head_dim), dtype=torch.bfloat16, device=self.dev)
        v = torch.empty_like(k)
        B.check(B.gf_node_kv_read(self.g, node, layer, k.data_ptr(), v.data_ptr(), self.stream), "gf_node_kv_read")
        torch.cuda.current_stream(self.dev).synchronize()
        return (k[:n].view(torch.int16).cpu().numpy().view(np.uint16), v[:n].view(torch.int16).cpu().numpy().view(np.uint16))

    def edge_scores(self, inputs: dict, tasks_per_pass: Optional[int] = None) -> torch.Tensor:
        """gf_edge_scores over `inputs` (see workloads.scoring_inputs): fp32 [num_tasks, num_edges]."""
        t = {k: torch.from_numpy(np.ascontiguousarray(v)).to(self.dev) for k, v in inputs.items() if k != "b3"}
        sc = B.Scorer(inputs["w_gcn1"].shape[0], inputs["w_gcn1"].shape[1], inputs["w2"].shape[0],
                      t["w_gcn1"].data_ptr(), t["w_gcn2"].data_ptr(), t["w1"].data_ptr(), t["b1"].data_ptr(),
                      t["w2"].data_ptr(), t["b2"].data_ptr(), t["w3"].data_ptr(), float(inputs["b3"]))
        nt = inputs["x_task"].shape[0]
        nbytes = B.gf_edge_scores_scratch_bytes(self.g, sc, nt, nt if tasks_per_pass is None else tasks_per_pass)
        scratch = self.guarded(nbytes, "scoring scratch")
        scores = self.guarded(nt * len(self.w.edge_src) * 4, "edge scores").view(torch.float32).view(nt, len(self.w.edge_src))
        B.check(B.gf_edge_scores(self.g, sc, t["x_op"].data_ptr(), nt, t["x_task"].data_ptr(), scores.data_ptr(),
                                 scratch.data_ptr(), nbytes, self.stream), "gf_edge_scores")
        torch.cuda.current_stream(self.dev).synchronize()   # the inputs in `t` are freed on return
        return scores

    def status(self) -> int:
        return B.gf_last_status(self.g, self.stream)
