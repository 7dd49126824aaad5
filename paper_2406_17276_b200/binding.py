"""Thin ctypes binding of the C ABI in include/opt_tree.h.

Argument marshalling only: every step runs in the CUDA library.  PyTorch is used
for device memory and streams.  There is no CPU fallback: if the library is not
built or no CUDA device is present, calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libopt_tree.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CUDA, ERR_TIMEOUT, ERR_INTERNAL = 0, -1, -2, -3, -4, -5

EXPORTS = ["opt_tree_workspace_bytes", "opt_tree_create", "opt_tree_destroy", "opt_tree_build", "opt_tree_mask",
           "opt_tree_verify", "opt_tree_row_softmax_topk", "opt_tree_step_host", "opt_tree_last_device_status",
           "opt_tree_launch_count", "opt_tree_strerror", "opt_tree_verify_static", "opt_tree_post_verify", "opt_tree_build_pruned", "opt_tree_layers_begin",
           "opt_tree_layers_step", "opt_tree_verify_sampled", "opt_tree_selftest_waits", "opt_tree_selftest_selection",
           "opt_tree_kv_workspace_bytes", "opt_tree_kv_create", "opt_tree_kv_destroy", "opt_tree_kv_append", "opt_tree_kv_attend",
           "opt_tree_kv_compact", "opt_tree_kv_last_device_status", "opt_tree_kv_launch_count"]


class Config(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("V", "H", "n", "k", "max_depth", "max_batch")]


class Out(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in
                ("token", "parent", "depth", "phat", "n_sel", "depth_reached", "expected_len", "esub_trace")]


class HostOut(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in
                ("token", "parent", "depth", "phat", "n_sel", "depth_reached", "expected_len", "mask", "position_ids",
                 "accept_len", "accept_tokens", "accept_nodes", "next_root")]


class KVConfig(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("q_heads", "kv_heads", "head_dim", "page", "num_pages", "max_pages", "max_batch", "max_step",
                                         "layers", "dtype")]


_lib = None


def lib():
    """Loads the shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2406_17276_b200.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        L.opt_tree_workspace_bytes.restype = C.c_size_t
        L.opt_tree_workspace_bytes.argtypes = [C.POINTER(Config)]
        L.opt_tree_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(Config)]
        L.opt_tree_destroy.argtypes = [C.c_void_p]
        L.opt_tree_build.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_float, C.POINTER(Out), C.c_void_p]
        L.opt_tree_mask.argtypes = [C.c_void_p, C.POINTER(Out), C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.opt_tree_verify.argtypes = [C.c_void_p, C.POINTER(Out), C.c_void_p, C.c_void_p, C.c_int32,
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.opt_tree_row_softmax_topk.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                                C.c_void_p]
        L.opt_tree_step_host.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                         C.c_float, C.POINTER(HostOut), C.c_void_p]
        L.opt_tree_last_device_status.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
        L.opt_tree_launch_count.restype = C.c_int64
        L.opt_tree_launch_count.argtypes = [C.c_void_p]
        L.opt_tree_verify_static.argtypes = [C.POINTER(Config), C.POINTER(Out), C.c_void_p, C.c_void_p, C.c_int32,
                                             C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.opt_tree_build_pruned.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_float, C.POINTER(Out), C.c_void_p,
                                            C.c_void_p]
        L.opt_tree_verify_sampled.argtypes = [C.c_void_p, C.POINTER(Out), C.c_void_p, C.c_void_p, C.c_int32, C.c_double,
                                              C.c_uint64, C.c_uint64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.opt_tree_layers_begin.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        L.opt_tree_layers_step.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.POINTER(Out), C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_void_p]
        L.opt_tree_post_verify.argtypes = [C.c_void_p, C.POINTER(Out), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.opt_tree_selftest_waits.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.opt_tree_selftest_selection.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32] + [C.c_void_p] * 5
        L.opt_tree_kv_workspace_bytes.restype = C.c_size_t
        L.opt_tree_kv_workspace_bytes.argtypes = [C.POINTER(KVConfig)]
        L.opt_tree_kv_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(KVConfig)]
        L.opt_tree_kv_destroy.argtypes = [C.c_void_p]
        rows, cache, step = C.c_void_p, C.c_void_p, C.c_void_p        # (plain addresses are handed over faster than typed pointers)
        L.opt_tree_kv_append.argtypes = [C.c_void_p, cache, C.c_int32, rows, rows, rows, rows, step, C.c_void_p, C.c_void_p]
        L.opt_tree_kv_attend.argtypes = [C.c_void_p, cache, C.c_int32, rows, step, C.c_float, rows, C.c_void_p, C.c_void_p]
        L.opt_tree_kv_compact.argtypes = [C.c_void_p, cache, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.opt_tree_kv_last_device_status.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
        L.opt_tree_kv_launch_count.restype = C.c_int64
        L.opt_tree_kv_launch_count.argtypes = [C.c_void_p]
        L.opt_tree_strerror.restype = C.c_char_p
        L.opt_tree_strerror.argtypes = [C.c_int]
        _lib = L
    return _lib


class OptTreeError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {lib().opt_tree_strerror(code).decode()} ({code})")


def _check(code: int, where: str):
    if code != OK:
        raise OptTreeError(code, where)


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(None)


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


@dataclass
class Tree:
    """Device tensors of one built batch (see opt_tree_out)."""
    token: torch.Tensor
    parent: torch.Tensor
    depth: torch.Tensor
    phat: torch.Tensor
    n_sel: torch.Tensor
    depth_reached: torch.Tensor
    expected_len: torch.Tensor
    esub_trace: torch.Tensor | None

    def c_struct(self) -> Out:
        return Out(*[t.data_ptr() if t is not None else None for t in
                     (self.token, self.parent, self.depth, self.phat, self.n_sel, self.depth_reached,
                      self.expected_len, self.esub_trace)])


class OptTree:
    """A library context: fixed (V, H, n, k, max_depth, max_batch), workspace allocated once."""

    def __init__(self, V: int, H: int, n: int, k: int, max_depth: int, max_batch: int, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the OPT-Tree library has no CPU fallback")
        self.cfg = Config(V, H, n, k, max_depth, max_batch)
        self.device = torch.device(device)
        self.W = (n + 63) // 64
        self._ctx = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().opt_tree_create(C.byref(self._ctx), C.byref(self.cfg)), "opt_tree_create")

    def close(self):
        if self._ctx:
            lib().opt_tree_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- allocation helpers (torch owns the memory) ----
    def alloc_tree(self, B: int, trace: bool = True) -> Tree:
        c, dev = self.cfg, self.device
        i32 = dict(dtype=torch.int32, device=dev)
        f64 = dict(dtype=torch.float64, device=dev)
        return Tree(torch.empty((B, c.n), **i32), torch.empty((B, c.n), **i32), torch.empty((B, c.n), **i32),
                    torch.empty((B, c.n), **f64), torch.empty(B, **i32), torch.empty(B, **i32), torch.empty(B, **f64),
                    torch.empty((B, c.max_depth), **f64) if trace else None)

    # ---- entry points (same names as the C ABI) ----
    def build(self, draft: torch.Tensor, root_token: torch.Tensor, delta: float, out: Tree | None = None) -> Tree:
        B = root_token.shape[0]
        out = out or self.alloc_tree(B)
        cs = out.c_struct()
        _check(lib().opt_tree_build(self._ctx, _ptr(draft), _ptr(root_token), B, C.c_float(delta), C.byref(cs), _stream()),
               "opt_tree_build")
        return out

    def build_pruned(self, draft: torch.Tensor, root_token: torch.Tensor, delta: float, out: Tree | None = None,
                     rows_read: torch.Tensor | None = None):
        """opt_tree_build_pruned: the same trees from fewer draft rows; returns (tree, rows_read [B] int32)."""
        B = root_token.shape[0]
        out = out or self.alloc_tree(B)
        if rows_read is None:
            rows_read = torch.empty(B, dtype=torch.int32, device=self.device)
        cs = out.c_struct()
        _check(lib().opt_tree_build_pruned(self._ctx, _ptr(draft), _ptr(root_token), B, C.c_float(delta), C.byref(cs),
                                           _ptr(rows_read), _stream()), "opt_tree_build_pruned")
        return out, rows_read

    def layers_begin(self, B: int):
        _check(lib().opt_tree_layers_begin(self._ctx, B, _stream()), "opt_tree_layers_begin")

    def layers_step(self, frontier_logits: torch.Tensor, delta: float, tree: Tree, nxt=None):
        """One layer of the layer-by-layer build; frontier_logits is [B][stride][V] bf16 bits on the device.
        Returns (next_tokens [B][n], next_parent [B][n], next_count [B])."""
        B, stride = frontier_logits.shape[0], frontier_logits.shape[1]
        if nxt is None:
            i32 = dict(dtype=torch.int32, device=self.device)
            nxt = (torch.empty((B, self.cfg.n), **i32), torch.empty((B, self.cfg.n), **i32), torch.empty(B, **i32))
        cs = tree.c_struct()
        _check(lib().opt_tree_layers_step(self._ctx, _ptr(frontier_logits), stride, B, C.c_float(delta), C.byref(cs),
                                          _ptr(nxt[0]), _ptr(nxt[1]), _ptr(nxt[2]), _stream()), "opt_tree_layers_step")
        return nxt

    def mask(self, tree: Tree, base_pos: torch.Tensor | None = None, mask: torch.Tensor | None = None,
             position_ids: torch.Tensor | None = None):
        B = tree.token.shape[0]
        if mask is None:
            mask = torch.empty((B, self.cfg.n, self.W), dtype=torch.int64, device=self.device)   # uint64 bit patterns
        if position_ids is None:
            position_ids = torch.empty((B, self.cfg.n), dtype=torch.int32, device=self.device)
        cs = tree.c_struct()
        _check(lib().opt_tree_mask(self._ctx, C.byref(cs), B, _ptr(base_pos), _ptr(mask), _ptr(position_ids), _stream()),
               "opt_tree_mask")
        return mask, position_ids

    def verify(self, tree: Tree, target: torch.Tensor, root_token: torch.Tensor, out=None):
        B = tree.token.shape[0]
        D = self.cfg.max_depth
        if out is None:
            i32 = dict(dtype=torch.int32, device=self.device)
            out = (torch.empty(B, **i32), torch.empty((B, D + 1), **i32), torch.empty((B, D), **i32), torch.empty(B, **i32))
        cs = tree.c_struct()
        _check(lib().opt_tree_verify(self._ctx, C.byref(cs), _ptr(target), _ptr(root_token), B,
                                     _ptr(out[0]), _ptr(out[1]), _ptr(out[2]), _ptr(out[3]), _stream()), "opt_tree_verify")
        return out

    def post_verify(self, tree: Tree, mask: torch.Tensor, accept_len: torch.Tensor, accept_nodes: torch.Tensor, out=None):
        """Dense (n+1)x(n+1) attention mask and the cache keep list of the accepted path."""
        B, n, D = tree.token.shape[0], self.cfg.n, self.cfg.max_depth
        if out is None:
            out = (torch.empty((B, n + 1, n + 1), dtype=torch.uint8, device=self.device),
                   torch.empty((B, D + 1), dtype=torch.int32, device=self.device),
                   torch.empty(B, dtype=torch.int32, device=self.device))
        cs = tree.c_struct()
        _check(lib().opt_tree_post_verify(self._ctx, C.byref(cs), _ptr(mask), _ptr(accept_len), _ptr(accept_nodes), B,
                                          _ptr(out[0]), _ptr(out[1]), _ptr(out[2]), _stream()), "opt_tree_post_verify")
        return out

    def verify_sampled(self, tree: Tree, target: torch.Tensor, root_token: torch.Tensor, tau: float, seed: int, step: int,
                       out=None):
        B = tree.token.shape[0]
        D = self.cfg.max_depth
        if out is None:
            i32 = dict(dtype=torch.int32, device=self.device)
            out = (torch.empty(B, **i32), torch.empty((B, D + 1), **i32), torch.empty((B, D), **i32), torch.empty(B, **i32))
        cs = tree.c_struct()
        _check(lib().opt_tree_verify_sampled(self._ctx, C.byref(cs), _ptr(target), _ptr(root_token), B, C.c_double(tau),
                                             C.c_uint64(seed), C.c_uint64(step), _ptr(out[0]), _ptr(out[1]), _ptr(out[2]),
                                             _ptr(out[3]), _stream()), "opt_tree_verify_sampled")
        return out

    def row_softmax_topk(self, logits: torch.Tensor, rows: torch.Tensor):
        nrows = rows.shape[0]
        tok = torch.empty((nrows, self.cfg.k), dtype=torch.int32, device=self.device)
        prob = torch.empty((nrows, self.cfg.k), dtype=torch.float64, device=self.device)
        _check(lib().opt_tree_row_softmax_topk(self._ctx, _ptr(logits), _ptr(rows), nrows, _ptr(tok), _ptr(prob), _stream()),
               "opt_tree_row_softmax_topk")
        return tok, prob

    def alloc_host_out(self, B: int) -> dict:
        """Pinned host buffers for step_host."""
        c = self.cfg
        def pin(shape, dt):
            return torch.empty(shape, dtype=dt).pin_memory()
        return dict(token=pin((B, c.n), torch.int32), parent=pin((B, c.n), torch.int32), depth=pin((B, c.n), torch.int32),
                    phat=pin((B, c.n), torch.float64), n_sel=pin((B,), torch.int32), depth_reached=pin((B,), torch.int32),
                    expected_len=pin((B,), torch.float64), mask=pin((B, c.n, self.W), torch.int64),
                    position_ids=pin((B, c.n), torch.int32), accept_len=pin((B,), torch.int32),
                    accept_tokens=pin((B, c.max_depth + 1), torch.int32), accept_nodes=pin((B, c.max_depth), torch.int32),
                    next_root=pin((B,), torch.int32))

    def step_host(self, draft: torch.Tensor, target: torch.Tensor, root_token_host: torch.Tensor,
                  base_pos_host: torch.Tensor | None, delta: float, host_out: dict) -> dict:
        B = root_token_host.shape[0]
        ho = HostOut(*[host_out[f].data_ptr() for f, _ in HostOut._fields_])
        _check(lib().opt_tree_step_host(self._ctx, _ptr(draft), _ptr(target), _ptr(root_token_host), _ptr(base_pos_host),
                                        B, C.c_float(delta), C.byref(ho), _stream()), "opt_tree_step_host")
        return host_out

    def selftest_waits(self) -> torch.Tensor:
        """opt_tree_selftest_waits: one status word per kind of bounded wait (each should read ERR_TIMEOUT)."""
        res = torch.full((5,), 77, dtype=torch.int32, device=self.device)
        _check(lib().opt_tree_selftest_waits(self._ctx, _ptr(res), _stream()), "opt_tree_selftest_waits")
        return res

    def selftest_selection(self, rows: int, written: int, joint: bool):
        """opt_tree_selftest_selection: (status, tokens, parents, path values) of a selection of which `rows - written` rows never come."""
        res = torch.full((1,), 77, dtype=torch.int32, device=self.device)
        tok, par = (torch.full((self.cfg.n,), 77, dtype=torch.int32, device=self.device) for _ in range(2))
        ph = torch.full((self.cfg.n,), 77.0, dtype=torch.float64, device=self.device)
        _check(lib().opt_tree_selftest_selection(self._ctx, rows, written, int(joint), _ptr(res), _ptr(tok), _ptr(par), _ptr(ph), _stream()),
               "opt_tree_selftest_selection")
        return res, tok, par, ph

    def device_status(self) -> int:
        st = C.c_int32(0)
        _check(lib().opt_tree_last_device_status(self._ctx, C.byref(st)), "opt_tree_last_device_status")
        return st.value

    def launch_count(self) -> int:
        return int(lib().opt_tree_launch_count(self._ctx))


def verify_static(cfg: Config, tree: Tree, target: torch.Tensor, root_token: torch.Tensor, out, device_status: torch.Tensor | None = None):
    """opt_tree_verify_static: verification for callers that cannot allocate.  Needs no OptTree context; every
    buffer, outputs included, is the caller's (out = (accept_len, accept_tokens, accept_nodes, next_root))."""
    B = tree.token.shape[0]
    cs = tree.c_struct()
    _check(lib().opt_tree_verify_static(C.byref(cfg), C.byref(cs), _ptr(target), _ptr(root_token), B, _ptr(out[0]), _ptr(out[1]),
                                        _ptr(out[2]), _ptr(out[3]), _ptr(device_status), _stream()), "opt_tree_verify_static")
    return out


# ---- the paged 8-bit cache of the target model's attention layers ----

_current_device, _current_stream = torch.cuda.current_device, lambda index: torch.cuda.current_stream(index).cuda_stream
if torch.cuda.is_available():            # the same without the wrappers' checks, which cost more than the library's launch
    _current_device = getattr(torch._C, "_cuda_getDevice", _current_device)
    _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)

_grad_enabled = torch.is_grad_enabled
_ROW_TYPES = {torch.bfloat16: 0, torch.float16: 1}
_F8, _F32, _I32, _I64 = torch.float8_e4m3fn, torch.float32, torch.int32, torch.int64


def _index(device: torch.device) -> int:
    """A device as Tensor.get_device() numbers it."""
    return device.index if device.type == "cuda" else -1


# The structures of opt_tree_kv_* as bytes: packed faster than ctypes fills a Structure, and handed over by their address.
_CACHE, _STEP, _ROWS, _TURN = (struct.Struct(f).pack for f in ("@5P", "@2i5P", "@P3q", "@P3iPPf"))


def _no_gradients(name: str):
    if _grad_enabled():
        raise ValueError(f"{name}: asks for gradients, which the cache operators do not have; call them under torch.no_grad() or detach it")


def _addr(t, name: str, dtype, shape, index: int):
    """Address of a contiguous tensor of this type, shape and device; 0 for None."""
    if t is None:
        return 0
    if t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: a contiguous {dtype} tensor {tuple(shape)} on device {index} is needed, not {t.dtype} {tuple(t.shape)} on {t.device}")


class KVCache:
    """Cache tensors (torch owns the memory): k, v [layers][num_pages][kv_heads][page][head_dim] float8_e4m3fn, k_scale, v_scale
    [layers][num_pages][kv_heads] float32, block_table [B][max_pages] int32 (see opt_tree_kv_cache).  One object serves any number of calls."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "block_table", "shape", "table_shape", "index", "c")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, block_table: torch.Tensor):
        shape, table, index = k.shape, block_table.shape, k.get_device()
        if len(shape) != 5 or len(table) != 2:
            raise ValueError("k: [layers][num_pages][kv_heads][page][head_dim], block_table: [B][max_pages]")
        scales = shape[:3]
        self.c = _CACHE(_addr(k, "k", _F8, shape, index), _addr(v, "v", _F8, shape, index), _addr(k_scale, "k_scale", _F32, scales, index),
                        _addr(v_scale, "v_scale", _F32, scales, index), _addr(block_table, "block_table", _I32, table, index))
        self.k, self.v, self.k_scale, self.v_scale, self.block_table = k, v, k_scale, v_scale, block_table
        self.shape, self.table_shape, self.index = shape, table, index


class KVStep:
    """A step's tokens (see opt_tree_kv_step): the root and `nodes` nodes of each sequence.  One object serves a step's calls for all layers."""

    __slots__ = ("kv_len", "nodes", "base_pos", "position_ids", "mask")

    def __init__(self, kv_len: torch.Tensor, nodes: torch.Tensor | None = None, base_pos: torch.Tensor | None = None,
                 position_ids: torch.Tensor | None = None, mask: torch.Tensor | None = None):
        self.kv_len, self.nodes, self.base_pos, self.position_ids, self.mask = kv_len, nodes, base_pos, position_ids, mask

    def c_struct(self, B: int, T: int, device: torch.device | int) -> bytes:
        index = device if type(device) is int else _index(device)
        one, nodes, base, pos, mask = (B,), self.nodes, self.base_pos, self.position_ids, self.mask
        return _STEP(B, T, _addr(self.kv_len, "kv_len", _I32, one, index), 0 if nodes is None else _addr(nodes, "nodes", _I32, one, index),
                     0 if base is None else _addr(base, "base_pos", _I32, one, index),
                     0 if pos is None else _addr(pos, "position_ids", _I32, (B, T - 1), index),
                     0 if mask is None or T == 1 else _addr(mask, "mask", _I64, (B, T - 1, (T + 62) // 64), index))


class TreeKV:
    """A handle of the cache operators (opt_tree_kv_*): fixed sizes, workspace allocated once, on one device.  For serving: there is no backward
    pass, and inputs that ask for gradients are refused."""

    def __init__(self, q_heads: int, kv_heads: int, head_dim: int, page: int, num_pages: int, max_pages: int, max_batch: int, max_step: int,
                 layers: int = 1, dtype: torch.dtype = torch.bfloat16, device: str | torch.device | None = None):
        self._kv = C.c_void_p()
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the OPT-Tree library has no CPU fallback")
        if dtype not in _ROW_TYPES:
            raise ValueError(f"dtype: bfloat16 or float16, not {dtype}")
        self.device = torch.device("cuda" if device is None else device)
        if self.device.type != "cuda":
            raise ValueError(f"device: a CUDA device, not {self.device}")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.dtype = dtype
        self.cfg = KVConfig(q_heads, kv_heads, head_dim, page, num_pages, max_pages, max_batch, max_step, layers, _ROW_TYPES[dtype])
        self._sizes()
        with torch.cuda.device(self.device):
            _check(lib().opt_tree_kv_create(C.byref(self._kv), C.byref(self.cfg)), "opt_tree_kv_create")

    def _sizes(self):
        c = self.cfg
        self._cache_shape = (c.layers, c.num_pages, c.kv_heads, c.page, c.head_dim)
        self._q_heads, self._kv_heads, self._D, self._max_pages = c.q_heads, c.kv_heads, c.head_dim, c.max_pages
        self._scale, self._at = c.head_dim ** -0.5, _index(self.device)

    def close(self):
        if self._kv:
            lib().opt_tree_kv_destroy(self._kv)
            self._kv = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def alloc_cache(self, block_table: torch.Tensor) -> KVCache:
        L, N, H, P, D = self._cache_shape
        k, v = (torch.zeros((L, N, H, P, D), dtype=torch.uint8, device=self.device).view(_F8) for _ in range(2))
        ks, vs = (torch.ones((L, N, H), dtype=_F32, device=self.device) for _ in range(2))
        return KVCache(k, v, ks, vs, block_table)

    def _rows(self, t: torch.Tensor, name: str, shape) -> bytes:
        if t.requires_grad:
            _no_gradients(name)
        st = t.stride()
        if t.dtype is self.dtype and t.shape == shape and t.get_device() == self._at and st[3] == 1:
            return _ROWS(t.data_ptr(), st[0], st[1], st[2])
        raise ValueError(f"{name}: {self.dtype} {tuple(shape)} with contiguous rows on {self.device} is needed, not {t.dtype} {tuple(t.shape)} on {t.device}")

    def _weight(self, t: torch.Tensor, name: str) -> int:
        if t.requires_grad:
            _no_gradients(name)
        return _addr(t, name, self.dtype, (self._D,), self._at)

    def _cache(self, cache: KVCache, B: int) -> bytes:
        table = cache.table_shape
        if cache.shape == self._cache_shape and cache.index == self._at and table[1] == self._max_pages and table[0] >= B:
            return cache.c
        raise ValueError(f"cache: pages {self._cache_shape} and a block table [{B}][{self._max_pages}] on {self.device} are needed, "
                         f"not {tuple(cache.shape)} and {tuple(table)} on {cache.k.device}")

    def _call(self, name: str, *args):
        """Calls with the handle's device current and its current stream as the last argument."""
        at = self._at
        if _current_device() == at:
            code = getattr(_lib, name)(self._kv, *args, _current_stream(at))
        else:
            with torch.cuda.device(self.device):
                code = getattr(_lib, name)(self._kv, *args, _current_stream(at))
        if code != OK:
            raise OptTreeError(code, name)

    def append(self, cache: KVCache, layer: int, q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, step: KVStep,
               cos_sin: torch.Tensor | None = None, q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None, eps: float = 1e-6,
               interleaved: bool = False, q_out: torch.Tensor | None = None) -> torch.Tensor | None:
        """opt_tree_kv_append: norm and rotation of q and k, k and v into the cache; returns the rotated queries (q_out; None if q is None)."""
        B, T = k.shape[:2]
        at, rows, D, each = self._at, self._rows, self._D, (B, T, self._kv_heads, self._D)
        qr = qo = None
        if q is not None:
            shape = (B, T, self._q_heads, D)
            if q_out is None:
                q_out = torch.empty(shape, dtype=self.dtype, device=self.device)
            qr, qo = rows(q, "q", shape), rows(q_out, "q_out", shape)
        angles, positions, rot = 0, 0, 0
        if cos_sin is not None:
            positions, rot = cos_sin.shape
            if cos_sin.requires_grad:
                _no_gradients("cos_sin")
            angles = _addr(cos_sin, "cos_sin", _F32, (positions, rot), at)
        turn = _TURN(angles, positions, rot, 1 if interleaved else 0, 0 if q_norm is None else self._weight(q_norm, "q_norm"),
                     0 if k_norm is None else self._weight(k_norm, "k_norm"), eps)
        self._call("opt_tree_kv_append", self._cache(cache, B), layer, qr, rows(k, "k", each), rows(v, "v", each), qo, step.c_struct(B, T, at), turn)
        return q_out

    def attend(self, cache: KVCache, layer: int, q: torch.Tensor, step: KVStep, scale: float | None = None, out: torch.Tensor | None = None,
               lse: torch.Tensor | None = None) -> torch.Tensor:
        """opt_tree_kv_attend: attention of the step's tokens over the cache; scale defaults to head_dim ** -0.5."""
        B, T = q.shape[:2]
        heads, at = self._q_heads, self._at
        shape = (B, T, heads, self._D)
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        self._call("opt_tree_kv_attend", self._cache(cache, B), layer, self._rows(q, "q", shape), step.c_struct(B, T, at), self._scale if scale is None else scale,
                   self._rows(out, "out", shape), None if lse is None else _addr(lse, "lse", _F32, (B, T, heads), at))
        return out

    def compact(self, cache: KVCache, kv_len: torch.Tensor, kv_gather: torch.Tensor, kv_keep: torch.Tensor,
                new_len: torch.Tensor | None = None) -> torch.Tensor:
        """opt_tree_kv_compact: the accepted path's entries of all layers to the end of the prefix; returns the new lengths."""
        B, G = shape = kv_gather.shape
        if new_len is None:
            new_len = torch.empty_like(kv_len)
        one, at = (B,), self._at
        self._call("opt_tree_kv_compact", self._cache(cache, B), _addr(kv_len, "kv_len", _I32, one, at), _addr(kv_gather, "kv_gather", _I32, shape, at),
                   _addr(kv_keep, "kv_keep", _I32, one, at), G, B, _addr(new_len, "new_len", _I32, one, at))
        return new_len

    def device_status(self) -> int:
        st = C.c_int32(0)
        with torch.cuda.device(self.device):
            _check(lib().opt_tree_kv_last_device_status(self._kv, C.byref(st)), "opt_tree_kv_last_device_status")
        return st.value

    def launch_count(self) -> int:
        return int(lib().opt_tree_kv_launch_count(self._kv))
