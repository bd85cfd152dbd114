"""Thin ctypes binding of the C ABI in include/tova.h.

Argument marshalling only: every step of the decode path runs in the CUDA
library.  torch is used for device memory and streams.  Loading fails loudly
if the library has not been built; nothing here computes on the CPU.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

from . import build as _build

TOVA_DTYPE_FP32 = 0
TOVA_DTYPE_BF16 = 1
TOVA_POLICY_TOVA = 0
TOVA_POLICY_WINDOW = 1
TOVA_POLICY_TOVA_HEAD = 2
TOVA_POLICY_H2O_LAYER = 3
TOVA_POLICY_H2O_HEAD = 4
TOVA_POS_AUTO = -1       # "the previous token's position + 1"
TOVA_ROPE_HALF, TOVA_ROPE_INTERLEAVED = 0, 1
TOVA_ROPE_PLAIN, TOVA_ROPE_LINEAR, TOVA_ROPE_NTK, TOVA_ROPE_YARN, TOVA_ROPE_BANDS = 0, 1, 2, 3, 4
TOVA_FORMAT_PLAIN, TOVA_FORMAT_INT8, TOVA_FORMAT_E4M3 = 0, 1, 2


class TovaError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: status {code} ({strerror(code)})")
        self.code = code


class tova_config(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("sm_scale", ctypes.c_float), ("evict", ctypes.c_int32)]


class tova_rope_config(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("scaling", ctypes.c_int32), ("base", ctypes.c_double),
                ("factor", ctypes.c_double), ("blend_low", ctypes.c_double), ("blend_high", ctypes.c_double),
                ("amplitude", ctypes.c_double), ("original_context", ctypes.c_int32)]


class tova_quant_config(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("dtype", ctypes.c_int32), ("format", ctypes.c_int32)]


class tova_tree_config(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("capacity", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("format", ctypes.c_int32), ("sm_scale", ctypes.c_float)]


class tova_verify_config(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_nodes", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("row_stride", ctypes.c_int64)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded CUDA library (built on first use if nvcc is present)."""
    global _lib
    if _lib is None:
        path = _build.LIB_PATH
        if not os.path.exists(path):
            path = _build.build()
        L = ctypes.CDLL(path)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.tova_cache_bytes.restype = ctypes.c_size_t
        L.tova_cache_bytes.argtypes = [ctypes.POINTER(tova_config)]
        L.tova_cache_init.restype = ctypes.c_int
        L.tova_cache_init.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(tova_config), vp,
                                      ctypes.c_size_t, vp]
        L.tova_decode_step.restype = ctypes.c_int
        L.tova_decode_step.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp]
        L.tova_prefill.restype = ctypes.c_int
        L.tova_prefill.argtypes = [vp, vp, vp, vp, i32, i32, vp, vp, vp]
        L.tova_decode_step_host.restype = ctypes.c_int
        L.tova_decode_step_host.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp]
        L.tova_cache_read.restype = ctypes.c_int
        L.tova_cache_read.argtypes = [vp, vp, vp, vp, vp, vp, vp]
        L.tova_cache_set_chunk_rows.restype = ctypes.c_int
        L.tova_cache_set_chunk_rows.argtypes = [vp, i32]
        L.tova_cache_set_policy.restype = ctypes.c_int
        L.tova_cache_set_policy.argtypes = [vp, i32, i32]
        L.tova_prefill_workspace_bytes.restype = ctypes.c_size_t
        L.tova_prefill_workspace_bytes.argtypes = [ctypes.POINTER(tova_config)]
        L.tova_cache_set_prefill_workspace.restype = ctypes.c_int
        L.tova_cache_set_prefill_workspace.argtypes = [vp, vp, ctypes.c_size_t]
        L.tova_position_workspace_bytes.restype = ctypes.c_size_t
        L.tova_position_workspace_bytes.argtypes = [ctypes.POINTER(tova_config)]
        L.tova_cache_set_position_compression.restype = ctypes.c_int
        L.tova_cache_set_position_compression.argtypes = [vp, vp, ctypes.c_size_t, ctypes.c_float]
        L.tova_cache_read_compressed_positions.restype = ctypes.c_int
        L.tova_cache_read_compressed_positions.argtypes = [vp, vp, vp]
        L.tova_shard_table_bytes.restype = ctypes.c_size_t
        L.tova_shard_table_bytes.argtypes = [ctypes.POINTER(tova_config), i32]
        L.tova_cache_set_shard.restype = ctypes.c_int
        L.tova_cache_set_shard.argtypes = [vp, i32, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(vp)]
        L.tova_decode_step_scores.restype = ctypes.c_int
        L.tova_decode_step_scores.argtypes = [vp, vp, vp, vp, i32, vp, vp]
        L.tova_decode_step_commit.restype = ctypes.c_int
        L.tova_decode_step_commit.argtypes = [vp, vp, vp, vp, vp]
        L.tova_cache_set_chunk_cluster.restype = ctypes.c_int
        L.tova_cache_set_chunk_cluster.argtypes = [vp, i32]
        L.tova_cache_set_chunk_barriers.restype = ctypes.c_int
        L.tova_cache_set_chunk_barriers.argtypes = [vp, i32]
        L.tova_cache_read_scores.restype = ctypes.c_int
        L.tova_cache_read_scores.argtypes = [vp, vp, vp]
        L.tova_cache_units.restype = i32
        L.tova_cache_units.argtypes = [vp]
        L.tova_cache_set_fused_merge.restype = ctypes.c_int
        L.tova_cache_set_fused_merge.argtypes = [vp, i32]
        L.tova_cache_set_bulk_prefill.restype = ctypes.c_int
        L.tova_cache_set_bulk_prefill.argtypes = [vp, i32]
        L.tova_cache_set_deferred_eviction.restype = ctypes.c_int
        L.tova_cache_set_deferred_eviction.argtypes = [vp, i32]
        L.tova_cache_join.restype = ctypes.c_int
        L.tova_cache_join.argtypes = [vp, vp]
        L.tova_cache_len.restype = i32
        L.tova_cache_len.argtypes = [vp]
        L.tova_cache_launches.restype = i64
        L.tova_cache_launches.argtypes = [vp]
        L.tova_cache_destroy.restype = ctypes.c_int
        L.tova_cache_destroy.argtypes = [vp]
        L.tova_decode_step_static.restype = ctypes.c_int
        L.tova_decode_step_static.argtypes = [ctypes.POINTER(tova_config), vp, vp, vp, i32, vp, vp, vp,
                                              i32, vp, vp, vp, vp]
        sz = ctypes.c_size_t
        L.tova_rope_init.restype = ctypes.c_int
        L.tova_rope_init.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(tova_rope_config)]
        L.tova_rope_apply.restype = ctypes.c_int
        L.tova_rope_apply.argtypes = [vp, vp, i64, vp, i64, i32, vp, i32, i32, vp, i64, vp, i64, vp]
        L.tova_rope_destroy.restype = ctypes.c_int
        L.tova_rope_destroy.argtypes = [vp]
        L.tova_quant_write.restype = ctypes.c_int
        L.tova_quant_write.argtypes = [ctypes.POINTER(tova_quant_config), vp, i64, vp, i64, i32, vp, i32, vp, vp, vp,
                                       vp, vp]
        L.tova_quant_read.restype = ctypes.c_int
        L.tova_quant_read.argtypes = [ctypes.POINTER(tova_quant_config), vp, vp, vp, vp, i32, vp, i32, vp, vp, vp]
        L.tova_tree_workspace_bytes.restype = sz
        L.tova_tree_workspace_bytes.argtypes = [ctypes.POINTER(tova_tree_config), i32, i32]
        L.tova_tree_attention.restype = ctypes.c_int
        L.tova_tree_attention.argtypes = [ctypes.POINTER(tova_tree_config), vp, vp, vp, vp, vp, i32, vp, vp, vp, i32,
                                          vp, vp, vp, sz, vp]
        L.tova_cache_tree_workspace_bytes.restype = sz
        L.tova_cache_tree_workspace_bytes.argtypes = [vp, i32]
        L.tova_cache_tree_attention.restype = ctypes.c_int
        L.tova_cache_tree_attention.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.tova_verify_draft.restype = ctypes.c_int
        L.tova_verify_draft.argtypes = [ctypes.POINTER(tova_verify_config), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.tova_strerror.restype = ctypes.c_char_p
        L.tova_strerror.argtypes = [ctypes.c_int]
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().tova_strerror(int(code)).decode()


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise TovaError(rc, what)


def _p(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream: Optional[torch.cuda.Stream]):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def tova_cache_bytes(cfg: tova_config) -> int:
    return int(lib().tova_cache_bytes(ctypes.byref(cfg)))


class TovaCache:
    """State of one layer for `batch` sequences; the names follow the C ABI."""

    def __init__(self, batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, capacity: int,
                 dtype: int = TOVA_DTYPE_BF16, sm_scale: float = 0.0, evict: bool = True,
                 device: str = "cuda:0", stream: Optional[torch.cuda.Stream] = None):
        self.cfg = tova_config(batch, n_q_heads, n_kv_heads, head_dim, capacity, dtype,
                               float(sm_scale), 1 if evict else 0)
        nbytes = tova_cache_bytes(self.cfg)
        if nbytes == 0:
            raise TovaError(-2, "tova_cache_bytes rejected the configuration")
        self.device = torch.device(device)
        self.tdtype = torch.bfloat16 if dtype == TOVA_DTYPE_BF16 else torch.float32
        self.nbytes = nbytes
        with torch.cuda.device(self.device):
            self.mem = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            off = (-self.mem.data_ptr()) % 256
            self._base = self.mem.data_ptr() + off
            h = ctypes.c_void_p()
            _check(lib().tova_cache_init(ctypes.byref(h), ctypes.byref(self.cfg),
                                         ctypes.c_void_p(self._base), nbytes, _stream(stream)),
                   "tova_cache_init")
        self._h = h

    # -- C ABI calls ---------------------------------------------------------
    def tova_decode_step(self, q, k, v, pos: int, out, evicted_pos=None, stream=None) -> None:
        _check(lib().tova_decode_step(self._h, _p(q), _p(k), _p(v), int(pos), _p(out),
                                      _p(evicted_pos), _stream(stream)), "tova_decode_step")

    def tova_prefill(self, q, k, v, n_tokens: int, first_pos: int, out=None, evicted_pos=None,
                     stream=None) -> None:
        _check(lib().tova_prefill(self._h, _p(q), _p(k), _p(v), int(n_tokens), int(first_pos),
                                  _p(out), _p(evicted_pos), _stream(stream)), "tova_prefill")

    def tova_decode_step_host(self, q, k, v, pos: int, out, evicted_pos=None, stream=None) -> None:
        """q, k, v, out, evicted_pos are HOST tensors (pinned for async copies)."""
        _check(lib().tova_decode_step_host(self._h, _p(q), _p(k), _p(v), int(pos), _p(out),
                                           _p(evicted_pos), _stream(stream)), "tova_decode_step_host")

    def tova_cache_read(self, want_kv: bool = False, stream=None):
        """Returns dict(len [B], positions [B,cap], status int, K, V or None) on the host."""
        c = self.cfg
        ln = torch.empty(c.batch, dtype=torch.int32, device=self.device)
        units = self.tova_cache_units()
        ps = (torch.empty(c.batch, c.capacity, dtype=torch.int32, device=self.device) if units == 1 else
              torch.empty(c.batch, units, c.capacity, dtype=torch.int32, device=self.device))
        stt = torch.empty(1, dtype=torch.int32, device=self.device)
        K = V = None
        if want_kv:
            K = torch.empty(c.batch, c.n_kv_heads, c.capacity, c.head_dim, dtype=self.tdtype,
                            device=self.device)
            V = torch.empty_like(K)
        _check(lib().tova_cache_read(self._h, _p(ln), _p(ps), _p(K), _p(V), _p(stt), _stream(stream)),
               "tova_cache_read")
        torch.cuda.synchronize(self.device)
        return {"len": ln.cpu(), "positions": ps.cpu(), "status": int(stt.item()),
                "K": None if K is None else K.float().cpu(), "V": None if V is None else V.float().cpu()}

    def tova_cache_set_prefill_workspace(self, mem: Optional[torch.Tensor] = None, allocate: bool = True):
        """Gives the cache the scratch of the chunked prompt route: `mem`, a uint8 device tensor the caller
        keeps alive (it may serve several caches of one shape), or a fresh one when allocate is set.
        mem=None with allocate=False switches the route off.  Returns the tensor in use."""
        if mem is None and not allocate:
            _check(lib().tova_cache_set_prefill_workspace(self._h, None, 0), "tova_cache_set_prefill_workspace")
            self._prefill_ws = None
            return None
        need = int(lib().tova_prefill_workspace_bytes(ctypes.byref(self.cfg)))
        if need == 0:
            raise TovaError(-3, "tova_prefill_workspace_bytes rejected the configuration")
        if mem is None:
            mem = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        off = (-mem.data_ptr()) % 256
        _check(lib().tova_cache_set_prefill_workspace(self._h, ctypes.c_void_p(mem.data_ptr() + off),
                                                      mem.numel() - off), "tova_cache_set_prefill_workspace")
        self._prefill_ws = mem
        return mem

    def tova_cache_set_position_compression(self, rope_base: float = 10000.0, on: bool = True) -> None:
        """Switches the position compression on (allocating its workspace) or off; callers then pass q and k
        without rotary embedding."""
        if not on:
            _check(lib().tova_cache_set_position_compression(self._h, None, 0, 0.0), "tova_cache_set_position_compression")
            self._poscomp_ws = None
            return
        need = int(lib().tova_position_workspace_bytes(ctypes.byref(self.cfg)))
        mem = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        off = (-mem.data_ptr()) % 256
        _check(lib().tova_cache_set_position_compression(self._h, ctypes.c_void_p(mem.data_ptr() + off), need,
                                                         float(rope_base)), "tova_cache_set_position_compression")
        self._poscomp_ws = mem

    def tova_cache_read_compressed_positions(self, stream=None):
        c = self.cfg
        cp = torch.empty(c.batch, c.capacity + 1, dtype=torch.float64, device=self.device)
        _check(lib().tova_cache_read_compressed_positions(self._h, _p(cp), _stream(stream)),
               "tova_cache_read_compressed_positions")
        torch.cuda.synchronize(self.device)
        return cp.cpu()

    def tova_shard_table_bytes(self, world: int) -> int:
        return int(lib().tova_shard_table_bytes(ctypes.byref(self.cfg), int(world)))

    def tova_cache_set_shard(self, rank: int, world: int, n_q_heads_total: int, peer_tables, peer_flags=None) -> None:
        """peer_tables / peer_flags: lists of `world` device tensors (or data pointers) as mapped into this process;
        peer_flags None = the caller sums peer_tables[rank] over the ranks between scores and commit."""
        def ptrs(xs):
            arr = (ctypes.c_void_p * world)()
            for i, x in enumerate(xs):
                arr[i] = None if x is None else (x.data_ptr() if hasattr(x, "data_ptr") else int(x))
            return arr
        tabs = ptrs(peer_tables)
        flags = None if peer_flags is None else ptrs(peer_flags)
        self._shard_keep = (peer_tables, peer_flags)
        _check(lib().tova_cache_set_shard(self._h, int(rank), int(world), int(n_q_heads_total), tabs, flags),
               "tova_cache_set_shard")

    def tova_decode_step_scores(self, q, k, v, pos: int, out, stream=None) -> None:
        _check(lib().tova_decode_step_scores(self._h, _p(q), _p(k), _p(v), int(pos), _p(out), _stream(stream)),
               "tova_decode_step_scores")

    def tova_decode_step_commit(self, k, v, evicted_pos=None, stream=None) -> None:
        _check(lib().tova_decode_step_commit(self._h, _p(k), _p(v), _p(evicted_pos), _stream(stream)),
               "tova_decode_step_commit")

    def tova_cache_set_chunk_cluster(self, ctas: int) -> None:
        _check(lib().tova_cache_set_chunk_cluster(self._h, int(ctas)), "tova_cache_set_chunk_cluster")

    def tova_cache_set_chunk_barriers(self, per_token: int) -> None:
        _check(lib().tova_cache_set_chunk_barriers(self._h, int(per_token)), "tova_cache_set_chunk_barriers")

    def tova_cache_set_chunk_rows(self, rows: int) -> None:
        _check(lib().tova_cache_set_chunk_rows(self._h, int(rows)), "tova_cache_set_chunk_rows")

    def tova_cache_set_policy(self, policy: int, arg: int = 0) -> None:
        """policy: one of TOVA_POLICY_*; arg = i of the "+i" variants, or the recent window of H2O."""
        _check(lib().tova_cache_set_policy(self._h, int(policy), int(arg)), "tova_cache_set_policy")

    def tova_cache_units(self) -> int:
        return int(lib().tova_cache_units(self._h))

    def tova_cache_read_scores(self, stream=None):
        """H2O: accumulated attention weight of every slot, [B,U,cap] on the host."""
        c = self.cfg
        sc = torch.empty(c.batch, self.tova_cache_units() if self.tova_cache_units() > 1 else 1, c.capacity,
                         dtype=torch.float32, device=self.device)
        _check(lib().tova_cache_read_scores(self._h, _p(sc), _stream(stream)), "tova_cache_read_scores")
        torch.cuda.synchronize(self.device)
        return sc.cpu()

    def tova_cache_set_fused_merge(self, on: bool) -> None:
        _check(lib().tova_cache_set_fused_merge(self._h, 1 if on else 0), "tova_cache_set_fused_merge")

    def tova_cache_set_bulk_prefill(self, mode) -> None:
        """0 / False: prompt tokens one at a time; 1 / True: bulk fill (tcgen05 kernel where head_dim is 128);
        2: bulk fill with the warp-level MMA kernel."""
        _check(lib().tova_cache_set_bulk_prefill(self._h, int(mode)), "tova_cache_set_bulk_prefill")

    def tova_cache_set_deferred_eviction(self, on: bool) -> None:
        _check(lib().tova_cache_set_deferred_eviction(self._h, 1 if on else 0),
               "tova_cache_set_deferred_eviction")

    def tova_cache_join(self, stream=None) -> None:
        _check(lib().tova_cache_join(self._h, _stream(stream)), "tova_cache_join")

    def tova_cache_len(self) -> int:
        return int(lib().tova_cache_len(self._h))

    def tova_cache_launches(self) -> int:
        return int(lib().tova_cache_launches(self._h))

    def tova_cache_tree_workspace_bytes(self, n_nodes: int) -> int:
        n = int(lib().tova_cache_tree_workspace_bytes(self._h, int(n_nodes)))
        if n == _NO_SIZE:
            raise TovaError(-2, "tova_cache_tree_workspace_bytes rejected the shape")
        return n

    def tova_cache_tree_attention(self, q, k, v, n_nodes: int, out, workspace=None, parents=None, stream=None) -> None:
        """Attention of the drafted tokens q [N,B,H,D], k and v [N,B,Hkv,D] over this state and their tree; out
        [N,B,H,D] in the cache's dtype, workspace of tova_cache_tree_workspace_bytes(n_nodes) bytes."""
        c, N = self.cfg, int(n_nodes)
        row = N * c.batch * c.head_dim
        dev = self.mem.get_device()
        for x, n in ((q, row * c.n_q_heads), (k, row * c.n_kv_heads), (v, row * c.n_kv_heads), (out, row * c.n_q_heads)):
            _need(x, n, self.tdtype, dev)
        _need(parents, N * c.batch, torch.int32, dev)
        _need_workspace(workspace, dev)
        _call(lib().tova_cache_tree_attention, "tova_cache_tree_attention", dev, stream, self._h, _a(q), _a(k), _a(v), N,
              _a(parents), _a(out), _a(workspace), _bytes(workspace))

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h:
            lib().tova_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def tova_decode_step_static(cfg: tova_config, K, V, positions, n_live: int, q, k, v, pos: int, out,
                            evicted_pos=None, status=None, stream=None) -> None:
    """One decode step on caller-held state tensors, using the scratch array
    built into the library instead of a workspace: for callers that may not
    allocate device memory (see include/tova.h).  K, V [B,Hkv,cap,D] and
    positions [B,cap] are updated in place; the caller tracks n_live.  status: an
    int32 device tensor of one element that receives 0 or a device-side check's code."""
    _check(lib().tova_decode_step_static(ctypes.byref(cfg), _p(K), _p(V), _p(positions), int(n_live),
                                         _p(q), _p(k), _p(v), int(pos), _p(out), _p(evicted_pos),
                                         _p(status), _stream(stream)), "tova_decode_step_static")


# -- around the decode step: rotary positions, the 8-bit state, drafted tokens ------------------------------------
# These take torch tensors of any origin, so their types, sizes and devices are checked here before their addresses
# reach the library; the current device is switched to the tensors' where it is another.

_NO_SIZE = ctypes.c_size_t(-1).value
_TORCH_TYPE = {TOVA_DTYPE_BF16: torch.bfloat16, TOVA_DTYPE_FP32: torch.float32}
_CODE_TYPES = {TOVA_FORMAT_INT8: (torch.int8, torch.uint8), TOVA_FORMAT_E4M3: (torch.float8_e4m3fn, torch.uint8, torch.int8)}
_byref = ctypes.byref


def _a(t):
    return None if t is None else t.data_ptr()


def _bytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _misfit(t, numel, dtype, device: int):
    if t.dtype is not dtype and not (type(dtype) is tuple and t.dtype in dtype):
        raise TypeError(f"expected a tensor of {dtype}, got {t.dtype}")
    if t.get_device() != device or device < 0:
        raise ValueError(f"expected a tensor on the GPU of the other arguments, got one on {t.device}")
    raise ValueError(f"expected a contiguous tensor of at least {numel} elements, got {tuple(t.shape)} with strides {t.stride()}")


def _need(t, numel: int, dtype, device: int) -> None:
    """A contiguous tensor of at least `numel` elements of `dtype` (or of one of several) on GPU `device`; None passes."""
    if t is not None and not ((t.dtype is dtype or (type(dtype) is tuple and t.dtype in dtype)) and t.get_device() == device >= 0
                              and t.is_contiguous() and t.numel() >= numel):
        _misfit(t, numel, dtype, device)


def _need_workspace(t, device: int) -> None:
    if t is not None and not (t.get_device() == device >= 0 and t.is_contiguous()):
        _misfit(t, 0, t.dtype, device)


def _rows(t, n_tokens: int, batch: int, heads: int, dim: int, dtype, device: int) -> int:
    """Checks [T,B,heads,dim] with contiguous heads and evenly spaced (token, sequence) rows; their element stride."""
    if t.dtype is not dtype or t.get_device() != device or device < 0:
        _misfit(t, 0, dtype, device)
    T, B, H, D = t.shape
    s0, s1, s2, s3 = t.stride()
    if T < n_tokens or B != batch or H != heads or D != dim:
        raise ValueError(f"expected [{n_tokens},{batch},{heads},{dim}], got {tuple(t.shape)}")
    if batch == 1:
        s1 = s0 if n_tokens > 1 else heads * dim
    elif n_tokens > 1 and s0 != s1 * batch:
        s1 = -1
    if s1 < heads * dim or (s2 != dim and heads > 1) or s3 != 1:
        raise ValueError(f"rows of {tuple(t.shape)} with strides {t.stride()} are not evenly spaced with contiguous heads")
    return s1


def _shortcut(name, plain):
    """torch's own internal form of a call where it has one (a fifth of the time; a small call is as short as its checks)."""
    return getattr(torch._C, name, plain)


_raw_current_stream = _shortcut("_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = _shortcut("_cuda_getDevice", lambda: torch.cuda.current_device())


def _call(fn, what: str, device: int, stream, *args) -> None:
    """fn(*args, stream) with `device` current (switched to where it is not already); the stream is the caller's, or the
    current one of that device."""
    st = _raw_current_stream(device) if stream is None else stream.cuda_stream
    was = _current_device()
    if was == device:
        rc = fn(*args, st)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, st)
    if rc != 0:
        raise TovaError(rc, what)


class TovaRope:
    """Rotary positions of q and k; holds the frequencies (host memory only)."""

    def __init__(self, batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: int = TOVA_DTYPE_BF16,
                 rotary_dim: int = 0, layout: int = TOVA_ROPE_HALF, base: float = 10000.0,
                 scaling: int = TOVA_ROPE_PLAIN, factor: float = 1.0, original_context: int = 0,
                 blend_low: float = 0.0, blend_high: float = 0.0, amplitude: float = 0.0):
        self.cfg = tova_rope_config(batch, n_q_heads, n_kv_heads, head_dim, dtype, rotary_dim, layout, scaling, base,
                                    factor, blend_low, blend_high, amplitude, original_context)
        h = ctypes.c_void_p()
        _check(lib().tova_rope_init(_byref(h), _byref(self.cfg)), "tova_rope_init")
        self._h = h
        self._dims = (batch, n_q_heads, n_kv_heads, head_dim, _TORCH_TYPE[dtype])

    def tova_rope_apply(self, q, k, n_tokens: int, q_out, k_out, positions=None, first_pos: int = 0,
                        inverse: bool = False, stream=None) -> None:
        """q [T,B,H,D] and k [T,B,Hkv,D] (or None) into q_out, k_out; all may be evenly strided over (T, B).  inverse:
        the transposed map, for gradients."""
        B, H, Hkv, D, t = self._dims
        dev = q.get_device()
        qs, qos = _rows(q, n_tokens, B, H, D, t, dev), _rows(q_out, n_tokens, B, H, D, t, dev)
        ks = kos = 0
        if k is not None or k_out is not None:
            if k is None or k_out is None:
                raise ValueError("k and k_out come together")
            ks, kos = _rows(k, n_tokens, B, Hkv, D, t, dev), _rows(k_out, n_tokens, B, Hkv, D, t, dev)
        _need(positions, n_tokens * B, torch.int32, dev)
        _call(lib().tova_rope_apply, "tova_rope_apply", dev, stream, self._h, _a(q), qs, _a(k), ks, n_tokens, _a(positions),
              first_pos, 1 if inverse else 0, _a(q_out), qos, _a(k_out), kos)

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h:
            lib().tova_rope_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _need_state(cfg, format, codes, scale, dtype, device) -> None:
    rows = cfg.batch * cfg.n_kv_heads * cfg.capacity
    _need(codes, rows * cfg.head_dim, dtype if format == TOVA_FORMAT_PLAIN else _CODE_TYPES.get(format), device)
    _need(scale, rows, torch.float32, device)


def tova_quant_write(cfg: tova_quant_config, k, v, n_tokens: int, k_codes, k_scale, v_codes, v_scale, slots=None,
                     first_slot: int = 0, stream=None) -> None:
    """Rows k, v [T,B,Hkv,D] (evenly strided over (T, B)) into the 8-bit state: codes [B,Hkv,cap,D], scales
    [B,Hkv,cap]; slots [T,B] int32 or None = first_slot + token."""
    t, dev, B, H, D = _TORCH_TYPE.get(cfg.dtype), k.get_device(), cfg.batch, cfg.n_kv_heads, cfg.head_dim
    ks, vs = _rows(k, n_tokens, B, H, D, t, dev), _rows(v, n_tokens, B, H, D, t, dev)
    _need_state(cfg, cfg.format, k_codes, k_scale, None, dev)
    _need_state(cfg, cfg.format, v_codes, v_scale, None, dev)
    _need(slots, n_tokens * B, torch.int32, dev)
    _call(lib().tova_quant_write, "tova_quant_write", dev, stream, _byref(cfg), _a(k), ks, _a(v), vs, n_tokens, _a(slots),
          first_slot, _a(k_codes), _a(k_scale), _a(v_codes), _a(v_scale))


def tova_quant_read(cfg: tova_quant_config, k_codes, k_scale, v_codes, v_scale, n_tokens: int, k, v, slots=None,
                    first_slot: int = 0, stream=None) -> None:
    """The state's rows at slots [T,B] (None: first_slot + token) as k, v [T,B,Hkv,D] in cfg.dtype; k or v may be None."""
    if k is None and v is None:
        return
    t, dev, B = _TORCH_TYPE.get(cfg.dtype), (k if k is not None else v).get_device(), cfg.batch
    n = n_tokens * B * cfg.n_kv_heads * cfg.head_dim
    _need(k, n, t, dev)
    _need(v, n, t, dev)
    _need_state(cfg, cfg.format, k_codes, k_scale, None, dev)
    _need_state(cfg, cfg.format, v_codes, v_scale, None, dev)
    _need(slots, n_tokens * B, torch.int32, dev)
    _call(lib().tova_quant_read, "tova_quant_read", dev, stream, _byref(cfg), _a(k_codes), _a(k_scale), _a(v_codes),
          _a(v_scale), n_tokens, _a(slots), first_slot, _a(k), _a(v))


def tova_tree_workspace_bytes(cfg: tova_tree_config, n_live: int, n_nodes: int) -> int:
    n = int(lib().tova_tree_workspace_bytes(_byref(cfg), int(n_live), int(n_nodes)))
    if n == _NO_SIZE:
        raise TovaError(-2, "tova_tree_workspace_bytes rejected the shape")
    return n


def tova_tree_attention(cfg: tova_tree_config, K, V, n_live: int, q, k, v, n_nodes: int, out, workspace=None,
                        parents=None, lens=None, k_scale=None, v_scale=None, stream=None) -> None:
    """Attention of N drafted tokens q [N,B,H,D], k, v [N,B,Hkv,D] over a state K, V [B,Hkv,cap,D] (or its codes with
    their scales) and the tree parents [N,B] (None: a chain); lens [B] int32 (None: n_live rows each).  out [N,B,H,D]
    in the type of q."""
    t, dev, B, N = _TORCH_TYPE.get(cfg.dtype), q.get_device(), cfg.batch, n_nodes
    nq, nk = N * B * cfg.n_q_heads * cfg.head_dim, N * B * cfg.n_kv_heads * cfg.head_dim
    _need_state(cfg, cfg.format, K, k_scale, t, dev)
    _need_state(cfg, cfg.format, V, v_scale, t, dev)
    _need(q, nq, t, dev)
    _need(k, nk, t, dev)
    _need(v, nk, t, dev)
    _need(out, nq, t, dev)
    _need(parents, N * B, torch.int32, dev)
    _need(lens, B, torch.int32, dev)
    _need_workspace(workspace, dev)
    _call(lib().tova_tree_attention, "tova_tree_attention", dev, stream, _byref(cfg), _a(K), _a(V), _a(k_scale),
          _a(v_scale), _a(lens), n_live, _a(q), _a(k), _a(v), N, _a(parents), _a(out), _a(workspace), _bytes(workspace))


def tova_verify_draft(cfg: tova_verify_config, target, draft, tokens, u, u_sample, n_accepted, path, tokens_out,
                      parents=None, stream=None) -> None:
    """Which drafted tokens [N,B] the target's probabilities [N+1,B,V] accept, given u [N,B] and u_sample [B]; see
    include/tova.h.  draft: probabilities the children were drawn from, or None.  n_accepted [B], path [N,B] or None,
    tokens_out [N+1,B], int32."""
    t, dev, B, N = _TORCH_TYPE.get(cfg.dtype), target.get_device(), cfg.batch, cfg.n_nodes
    ld = cfg.row_stride or cfg.vocab
    need = ((N + 1) * B - 1) * ld + cfg.vocab
    _need(target, need, t, dev)
    _need(draft, (max(N, 1) * B - 1) * ld + cfg.vocab if parents is None else need, t, dev)
    _need(tokens, N * B, torch.int32, dev)
    _need(parents, N * B, torch.int32, dev)
    _need(u, N * B, torch.float32, dev)
    _need(u_sample, B, torch.float32, dev)
    _need(n_accepted, B, torch.int32, dev)
    _need(path, N * B, torch.int32, dev)
    _need(tokens_out, (N + 1) * B, torch.int32, dev)
    _call(lib().tova_verify_draft, "tova_verify_draft", dev, stream, _byref(cfg), _a(target), _a(draft), _a(tokens),
          _a(parents), _a(u), _a(u_sample), _a(n_accepted), _a(path), _a(tokens_out))


def to_device(x, dtype: int, device="cuda:0") -> torch.Tensor:
    """Upload a float32 numpy array (bf16-representable for bf16) in the cache dtype."""
    t = torch.from_numpy(x)
    if dtype == TOVA_DTYPE_BF16:
        t = t.to(torch.bfloat16)
    return t.to(device)
